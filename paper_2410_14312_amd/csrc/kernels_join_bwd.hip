// Norm joins, backward.  With the rows' statistics of the forward pass, fh = (f - m1) i1 and yh = (y - m2) i2:
//   t = du pre_gain, dh = dy + i2 (t - mean(t) - yh mean(t yh))                 (means of t only where the norm subtracts one)
//   dr = scale dh (+ what others have given r);  da = dh gain fh g (1 - g);  v = dh g gain, df = i1 (v - mean(v) - fh mean(v fh))
//   dpre_gain = sum du yh, dpre_shift = sum du, dscale = sum dh r, dgain = sum dh g fh over the rows
// One pass over memory: dy, du, x, r, y are read and dx, dr written once each.  A team goes over its share of the rows and keeps its sums over them in registers, which
// leave as one row of partial results; those are added up in a fixed order behind.
#include "launch.h"
#include "norm_join.hip.h"

namespace tmps {

template <typename T, int TEAM, int V, int N, bool JOIN, bool PRE>
__global__ __launch_bounds__(Team<TEAM>::kThreads) void norm_join_bwd_kernel(NormJoinBackward a, float* part, float* part_pre) {
    __shared__ float red[2][4 * 16];
    const int D = a.D;
    const float over_d = 1.0f / (float)D;
    int place = 0;
    float dgain[N][V], dscale[N][V], dpg[N][V], dps[N][V];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) dgain[i][e] = dscale[i][e] = dpg[i][e] = dps[i][e] = 0.0f;
    const int64_t step = (int64_t)gridDim.x * Team<TEAM>::kRows;
    for (int64_t row = (int64_t)blockIdx.x * Team<TEAM>::kRows + threadIdx.x / TEAM; row < a.rows; row += step) {
        float dh[N][V];
        const bool has_dy = !PRE || a.dy;
        if (has_dy) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = join_column<TEAM, V>(i);
                if (c < D) load_piece<V>((const T*)a.dy + row * D + c, dh[i]);
            }
        }
        if constexpr (PRE) {
            const float mean = a.pre_stats[row * a.stats_stride], rstd = a.pre_stats[row * a.stats_stride + 1];
            float t[N][V], yh[N][V], s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = join_column<TEAM, V>(i);
                if (c >= D) continue;
                float du[V], g[V];
                load_piece<V>((const T*)a.du + row * D + c, du);
                load_piece<V>((const T*)a.y + row * D + c, yh[i]);
                load_piece<V>(a.pre_gain + c, g);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    yh[i][e] = (yh[i][e] - mean) * rstd;
                    t[i][e] = du[e] * g[e];
                    s[0] = fmaf(t[i][e], yh[i][e], s[0]);
                    s[1] += t[i][e];
                    dpg[i][e] = fmaf(du[e], yh[i][e], dpg[i][e]);
                    dps[i][e] += du[e];
                }
            }
            Team<TEAM>::sums(s, red, place);
            const float m = a.rms ? 0.0f : s[1] * over_d, q = s[0] * over_d;
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float v = rstd * (t[i][e] - m - yh[i][e] * q);
                    dh[i][e] = has_dy ? dh[i][e] + v : v;
                }
        }
        if constexpr (JOIN) {
            const float mean = a.stats[row * a.stats_stride], rstd = a.stats[row * a.stats_stride + 1];
            const int wide = a.gate ? 2 * D : D;
            const T* const xr = (const T*)a.x + row * wide;
            T* const dxr = (T*)a.dx + row * wide;
            float fh[N][V], s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = join_column<TEAM, V>(i);
                if (c >= D) continue;
                float r[V], sc[V], g[V], o[V];
                load_piece<V>(xr + c, fh[i]);
                load_piece<V>((const T*)a.r + row * D + c, r);
                load_piece<V>(a.scale + c, sc);
                load_piece<V>(a.gain + c, g);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    fh[i][e] = (fh[i][e] - mean) * rstd;
                    dscale[i][e] = fmaf(dh[i][e], r[e], dscale[i][e]);
                    o[e] = dh[i][e] * sc[e];
                }
                if (a.add) {
                    float b[V];
                    load_piece<V>((const T*)a.add + row * D + c, b);
#pragma unroll
                    for (int e = 0; e < V; ++e) o[e] += b[e];
                }
                if (a.gate) {
                    float at[V], da[V];
                    load_piece<V>(xr + D + c, at);
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        float sg, rest;
                        gate_of<T>(at[e], sg, rest);
                        da[e] = dh[i][e] * g[e] * fh[i][e] * (sg * rest);
                        dh[i][e] *= sg;
                    }
                    if (a.dx) store_piece<V>(dxr + D + c, da);
                }
                if (a.dr) store_piece<V>((T*)a.dr + row * D + c, o);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    dgain[i][e] = fmaf(dh[i][e], fh[i][e], dgain[i][e]);
                    dh[i][e] *= g[e];
                    s[0] = fmaf(dh[i][e], fh[i][e], s[0]);
                    s[1] += dh[i][e];
                }
            }
            if (a.dx) {
                Team<TEAM>::sums(s, red, place);
                const float m = a.rms ? 0.0f : s[1] * over_d, q = s[0] * over_d;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int c = join_column<TEAM, V>(i);
                    if (c >= D) continue;
                    float o[V];
#pragma unroll
                    for (int e = 0; e < V; ++e) o[e] = rstd * (dh[i][e] - m - fh[i][e] * q);
                    store_piece<V>(dxr + c, o);
                }
            }
        } else if (a.dr) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = join_column<TEAM, V>(i);
                if (c < D) store_piece<V>((T*)a.dr + row * D + c, dh[i]);
            }
        }
    }
    // a row of partial results for each team
    const int64_t team = (int64_t)blockIdx.x * Team<TEAM>::kRows + threadIdx.x / TEAM;
    const int pre = a.rms ? 1 : 2;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = join_column<TEAM, V>(i);
        if (c >= D) continue;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if constexpr (JOIN) {
                part[team * 2 * D + c + e] = dgain[i][e];
                part[team * 2 * D + D + c + e] = dscale[i][e];
            }
            if constexpr (PRE) {
                part_pre[team * pre * D + c + e] = dpg[i][e];
                if (!a.rms) part_pre[team * pre * D + D + c + e] = dps[i][e];
            }
        }
    }
}

// Workgroups of the launch: enough to fill the device, and few enough that their partial results are little beside the rows.
static int bwd_groups(int64_t rows, int teams) {
    const int64_t groups = (rows + teams - 1) / teams;
    return (int)(groups < 512 ? groups : 512);
}
static int bwd_teams(int D) { return D <= 1024 ? 4 : 1; }   // rows that a workgroup has under way

size_t norm_join_part_elems(int64_t rows, int D) { return (size_t)bwd_groups(rows, bwd_teams(D)) * bwd_teams(D) * 2 * (size_t)D; }

template <typename T, int TEAM, int V, int N> static hipError_t bwd_launch(const NormJoinBackward& j, const Partials& part, const Partials& part_pre, hipStream_t s) {
    const int groups = bwd_groups(j.rows, Team<TEAM>::kRows);
    const dim3 grid(groups), block(Team<TEAM>::kThreads);
    hipError_t e;
    if (!j.x) e = launch_timed(kcLayerNorm, norm_join_bwd_kernel<T, TEAM, V, N, false, true>, grid, block, 0, s, j, part.ws, part_pre.ws);
    else if (!j.du) e = launch_timed(kcLayerNorm, norm_join_bwd_kernel<T, TEAM, V, N, true, false>, grid, block, 0, s, j, part.ws, part_pre.ws);
    else e = launch_timed(kcLayerNorm, norm_join_bwd_kernel<T, TEAM, V, N, true, true>, grid, block, 0, s, j, part.ws, part_pre.ws);
    if (e != hipSuccess) return e;
    const int slabs = groups * Team<TEAM>::kRows;
    const Reduction of_join{part.ws, j.dgain_dscale, 2 * (int64_t)j.D, slabs, true}, of_pre{part_pre.ws, j.dpre, (j.rms ? 1 : 2) * (int64_t)j.D, slabs, true};
    if (j.x && j.du && !part.later && !part_pre.later) return reduce_all(Reductions{of_join, of_pre}, s);
    if (j.x && (e = part.finish(of_join, s)) != hipSuccess) return e;
    return j.du ? part_pre.finish(of_pre, s) : hipSuccess;
}

template <typename T> static hipError_t bwd_type(const NormJoinBackward& j, const Partials& part, const Partials& part_pre, hipStream_t s) {
    if (j.D <= 64) return bwd_launch<T, 64, 1, 1>(j, part, part_pre, s);
    if (j.D <= 1024) return bwd_launch<T, 64, 1, 16>(j, part, part_pre, s);
    if (j.D <= 4096) return bwd_launch<T, 256, 1, 16>(j, part, part_pre, s);
    return bwd_launch<T, 1024, 1, 16>(j, part, part_pre, s);
}

// Sums over no rows.
__global__ __launch_bounds__(256) void join_no_rows_kernel(float* dgain_dscale, float* dpre, int n, int n_pre) {
    for (int i = threadIdx.x; i < n; i += 256) dgain_dscale[i] = 0.0f;
    for (int i = threadIdx.x; i < n_pre; i += 256) dpre[i] = 0.0f;
}

hipError_t norm_join_backward(int dtype, const NormJoinBackward& j, const Partials& part, const Partials& part_pre, hipStream_t s) {
    if (j.rows <= 0)
        return launch_timed(kcLayerNorm, join_no_rows_kernel, dim3(1), dim3(256), 0, s, j.dgain_dscale, j.dpre, j.x ? 2 * j.D : 0, j.du ? (j.rms ? 1 : 2) * j.D : 0);
    if (j.D < 1 || j.D > kJoinMaxFeatures || (!j.x && !j.du) || (!j.dy && !j.du)) return hipErrorInvalidValue;
    return dtype == kBF16 ? bwd_type<bf16_t>(j, part, part_pre, s) : bwd_type<float>(j, part, part_pre, s);
}

}  // namespace tmps
