// Norm joins, backward.  With the rows' statistics of the forward pass, fh = (f - m1) i1 and yh = (y - m2) i2:
//   t = du pre_gain, dh = dy + i2 (t - mean(t) - yh mean(t yh))                 (means of t only where the norm subtracts one)
//   dr = scale dh (+ what others have given r);  da = dh gain fh g (1 - g);  v = dh g gain, df = i1 (v - mean(v) - fh mean(v fh))
//   dpre_gain = sum du yh, dpre_shift = sum du, dscale = sum dh r, dgain = sum dh g fh over the rows
// One pass over memory: dy, du, x, r, y are read and dx, dr written once each.  A team goes over its share of the rows and keeps its sums over them in registers, which
// leave as one row of partial results; those are added up in a fixed order behind.
#include "launch.h"
#include "norm_join.hip.h"

namespace tmps {

constexpr int kBwdGroups = 512;

template <typename T, int TEAM, int V, int N, bool JOIN, bool PRE, bool GATE>
__global__ __launch_bounds__(Team<TEAM>::kThreads) void norm_join_bwd_kernel(NormJoinBackward a, float* part, float* part_pre) {
    __shared__ float red[2][4 * 16];
    __shared__ float fold[Team<TEAM>::kRows > 1 ? Team<TEAM>::kRows : 1][Team<TEAM>::kRows > 1 ? TEAM * V * N : 1];
    const int D = a.D;
    constexpr int wide = GATE ? 2 : 1;
    const float over_d = 1.0f / (float)D;
    int place = 0;
    float dgain[JOIN ? N : 1][V], dscale[JOIN ? N : 1][V], dpg[PRE ? N : 1][V], dps[PRE ? N : 1][V];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if constexpr (JOIN) dgain[i][e] = dscale[i][e] = 0.0f;
            if constexpr (PRE) dpg[i][e] = dps[i][e] = 0.0f;
        }
    float gain[JOIN ? N : 1][V], scale[JOIN ? N : 1][V], pre_gain[PRE ? N : 1][V];
    if constexpr (JOIN) {
        load_vector<TEAM, V, N>(gain, a.gain, D);
        load_vector<TEAM, V, N>(scale, a.scale, D);
    }
    if constexpr (PRE) load_vector<TEAM, V, N>(pre_gain, a.pre_gain, D);
    const int64_t step = (int64_t)gridDim.x * Team<TEAM>::kRows;
    for (int64_t row = (int64_t)blockIdx.x * Team<TEAM>::kRows + threadIdx.x / TEAM; row < a.rows; row += step) {
        RawPiece<T, V> rdy[N], rdu[PRE ? N : 1], ry[PRE ? N : 1], rf[JOIN ? N : 1], ra[GATE ? N : 1], rr[JOIN ? N : 1], radd[JOIN ? N : 1];
        const bool has_dy = !PRE || a.dy;
        if constexpr (PRE) {
            request_row<T, TEAM, V, N>(rdu, (const T*)a.du + row * D, D);
            request_row<T, TEAM, V, N>(ry, (const T*)a.y + row * D, D);
        }
        if (has_dy) request_row<T, TEAM, V, N>(rdy, (const T*)a.dy + row * D, D);
        if constexpr (JOIN) {
            request_row<T, TEAM, V, N>(rf, (const T*)a.x + row * D * wide, D);
            request_row<T, TEAM, V, N>(rr, (const T*)a.r + row * D, D);
            if constexpr (GATE) request_row<T, TEAM, V, N>(ra, (const T*)a.x + row * D * wide + D, D);
            if (a.add) request_row<T, TEAM, V, N>(radd, (const T*)a.add + row * D, D);
        }
        float dh[N][V];
        if constexpr (PRE) {
            const float mean = a.pre_stats[row * a.stats_stride], rstd = a.pre_stats[row * a.stats_stride + 1];
            float yh[N][V], s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (join_column<TEAM, V>(i) >= D) continue;
                float du[V];
                rdu[i].get(du);
                ry[i].get(yh[i]);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    yh[i][e] = (yh[i][e] - mean) * rstd;
                    dh[i][e] = du[e] * pre_gain[i][e];
                    s[0] = fmaf(dh[i][e], yh[i][e], s[0]);
                    s[1] += dh[i][e];
                    dpg[i][e] = fmaf(du[e], yh[i][e], dpg[i][e]);
                    dps[i][e] += du[e];
                }
            }
            Team<TEAM>::sums(s, red, place);
            const float m = a.rms ? 0.0f : s[1] * over_d, q = s[0] * over_d;
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (join_column<TEAM, V>(i) < D) {
#pragma unroll
                    for (int e = 0; e < V; ++e) dh[i][e] = rstd * fmaf(-yh[i][e], q, dh[i][e] - m);
                }
        }
        if (has_dy) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (join_column<TEAM, V>(i) < D) {
                    float dy[V];
                    rdy[i].get(dy);
#pragma unroll
                    for (int e = 0; e < V; ++e) dh[i][e] = PRE ? dh[i][e] + dy[e] : dy[e];
                }
        }
        if constexpr (JOIN) {
            const float mean = a.stats[row * a.stats_stride], rstd = a.stats[row * a.stats_stride + 1];
            T* const dxr = (T*)a.dx + row * D * wide;
            float fh[N][V], s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = join_column<TEAM, V>(i);
                if (c >= D) continue;
                float r[V], o[V];
                rf[i].get(fh[i]);
                rr[i].get(r);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    fh[i][e] = (fh[i][e] - mean) * rstd;
                    dscale[i][e] = fmaf(dh[i][e], r[e], dscale[i][e]);
                    o[e] = dh[i][e] * scale[i][e];
                }
                if (a.add) {
                    float b[V];
                    radd[i].get(b);
#pragma unroll
                    for (int e = 0; e < V; ++e) o[e] += b[e];
                }
                if (a.dr) store_piece<V>((T*)a.dr + row * D + c, o);
                if constexpr (GATE) {
                    float at[V], da[V];
                    ra[i].get(at);
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        float sg, rest;
                        gate_of<T>(at[e], sg, rest);
                        da[e] = dh[i][e] * gain[i][e] * fh[i][e] * (sg * rest);
                        dh[i][e] *= sg;
                    }
                    if (a.dx) store_piece<V>(dxr + D + c, da);
                }
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    dgain[i][e] = fmaf(dh[i][e], fh[i][e], dgain[i][e]);
                    dh[i][e] *= gain[i][e];
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
                    for (int e = 0; e < V; ++e) o[e] = rstd * fmaf(-fh[i][e], q, dh[i][e] - m);
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
    // The workgroup's row of partial results; its waves' sums, where they are teams of their own, are added up through LDS.
    auto leave = [&](const float (&v)[N][V], float* to) {
        if constexpr (Team<TEAM>::kRows > 1) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e) fold[threadIdx.x / TEAM][join_column<TEAM, V>(i) + e] = v[i][e];
            __syncthreads();
            for (int c = threadIdx.x; c < D; c += Team<TEAM>::kThreads) to[c] = (fold[0][c] + fold[1][c]) + (fold[2][c] + fold[3][c]);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = join_column<TEAM, V>(i);
                if (c >= D) continue;
#pragma unroll
                for (int e = 0; e < V; ++e) to[c + e] = v[i][e];
            }
        }
    };
    if constexpr (JOIN) {
        leave(dgain, part + (int64_t)blockIdx.x * 2 * D);
        leave(dscale, part + (int64_t)blockIdx.x * 2 * D + D);
    }
    if constexpr (PRE) {
        float* const to = part_pre + (int64_t)blockIdx.x * (a.rms ? 1 : 2) * D;
        leave(dpg, to);
        if (!a.rms) leave(dps, to + D);
    }
}

// Workgroups of the launch: enough to fill the device, and few enough that their partial results are little beside the rows.
static int bwd_groups(int64_t rows, int teams) {
    const int64_t groups = (rows + teams - 1) / teams;
    return (int)(groups < kBwdGroups ? groups : kBwdGroups);
}

// (any kernel's: the one whose teams are workgroups)
size_t norm_join_part_elems(int64_t rows, int D) { return (size_t)bwd_groups(rows, 1) * 2 * (size_t)D; }

template <typename T, int TEAM, int V, int N> static hipError_t bwd_launch(const NormJoinBackward& j, const Partials& part, const Partials& part_pre, hipStream_t s) {
    const int groups = bwd_groups(j.rows, Team<TEAM>::kRows);
    auto kern = !j.x ? norm_join_bwd_kernel<T, TEAM, V, N, false, true, false>
                : !j.du ? (j.gate ? norm_join_bwd_kernel<T, TEAM, V, N, true, false, true> : norm_join_bwd_kernel<T, TEAM, V, N, true, false, false>)
                        : (j.gate ? norm_join_bwd_kernel<T, TEAM, V, N, true, true, true> : norm_join_bwd_kernel<T, TEAM, V, N, true, true, false>);
    hipError_t e = launch_timed(kcLayerNorm, kern, dim3(groups), dim3(Team<TEAM>::kThreads), 0, s, j, part.ws, part_pre.ws);
    if (e != hipSuccess) return e;
    const Reduction of_join{part.ws, j.dgain_dscale, 2 * (int64_t)j.D, groups, true}, of_pre{part_pre.ws, j.dpre, (j.rms ? 1 : 2) * (int64_t)j.D, groups, true};
    if (j.x && j.du && !part.later && !part_pre.later) return reduce_all(Reductions{of_join, of_pre}, s);
    if (j.x && (e = part.finish(of_join, s)) != hipSuccess) return e;
    return j.du ? part_pre.finish(of_pre, s) : hipSuccess;
}

template <typename T> static hipError_t bwd_type(const NormJoinBackward& j, const Partials& part, const Partials& part_pre, hipStream_t s) {
    if (join_wide(j.D, {j.dy, j.du, j.x, j.r, j.y, j.gain, j.scale, j.pre_gain, j.add, j.dx, j.dr})) {
        if (j.D <= 512) return bwd_launch<T, 64, 8, 1>(j, part, part_pre, s);
        if (j.D <= 1024) return bwd_launch<T, 64, 8, 2>(j, part, part_pre, s);
        if (j.D <= 2048) return bwd_launch<T, 256, 8, 1>(j, part, part_pre, s);
        if (j.D <= 4096) return bwd_launch<T, 256, 8, 2>(j, part, part_pre, s);
        if (j.D <= 8192) return bwd_launch<T, 1024, 8, 1>(j, part, part_pre, s);
        return bwd_launch<T, 1024, 8, 2>(j, part, part_pre, s);
    }
    if (j.D <= 64) return bwd_launch<T, 64, 1, 1>(j, part, part_pre, s);
    if (j.D <= 256) return bwd_launch<T, 64, 1, 4>(j, part, part_pre, s);
    if (j.D <= 1024) return bwd_launch<T, 256, 1, 4>(j, part, part_pre, s);
    if (j.D <= 4096) return bwd_launch<T, 1024, 1, 4>(j, part, part_pre, s);
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
