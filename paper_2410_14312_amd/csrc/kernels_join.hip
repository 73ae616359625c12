// Norm joins, forward: y = scale r + g gain n(f) and u = n(y) pre_gain + pre_shift in one pass over memory.  Bound by memory: f, r (and the gate's argument) are
// read, y and u written once each.
#include "launch.h"
#include "norm_join.hip.h"

namespace tmps {

// Mean (0 with rms) and 1/std of a row in registers; the variance is that of the differences from the mean.
template <int TEAM, int V, int N> __device__ __forceinline__ void row_stats(const float (&v)[N][V], int D, bool rms, float& mean, float& rstd, float (*red)[4 * 16], int& place) {
    float s[1] = {0.0f};
    mean = 0.0f;
    if (!rms) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (join_column<TEAM, V>(i) < D) {
#pragma unroll
                for (int e = 0; e < V; ++e) s[0] += v[i][e];
            }
        Team<TEAM>::sums(s, red, place);
        mean = s[0] / (float)D;
        s[0] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (join_column<TEAM, V>(i) < D) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = v[i][e] - mean;
                s[0] = fmaf(d, d, s[0]);
            }
        }
    Team<TEAM>::sums(s, red, place);
    rstd = 1.0f / sqrtf(s[0] / (float)D + 1e-5f);
}

// A team to a row.
template <typename T, int TEAM, int V, int N, bool JOIN, bool PRE>
__global__ __launch_bounds__(Team<TEAM>::kThreads) void norm_join_fwd_kernel(NormJoin a) {
    __shared__ float red[2][4 * 16];
    const int D = a.D;
    int place = 0;
    const int64_t step = (int64_t)gridDim.x * Team<TEAM>::kRows;
    for (int64_t row = (int64_t)blockIdx.x * Team<TEAM>::kRows + threadIdx.x / TEAM; row < a.rows; row += step) {
        float y[N][V];
        T* const yr = (T*)a.y + row * D;
        if constexpr (JOIN) {
            const int wide = a.gate ? 2 * D : D;
            const T* const xr = (const T*)a.x + row * wide;
            const T* const rr = (const T*)a.r + row * D;
            float f[N][V];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = join_column<TEAM, V>(i);
                if (c < D) load_piece<V>(xr + c, f[i]);
            }
            float mean, rstd;
            row_stats<TEAM, V, N>(f, D, a.rms, mean, rstd, red, place);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = join_column<TEAM, V>(i);
                if (c >= D) continue;
                float r[V], g[V], sc[V];
                load_piece<V>(rr + c, r);
                load_piece<V>(a.gain + c, g);
                load_piece<V>(a.scale + c, sc);
                if (a.gate) {
                    float at[V];
                    load_piece<V>(xr + D + c, at);
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        float sg, rest;
                        gate_of<T>(at[e], sg, rest);
                        g[e] *= sg;
                    }
                }
#pragma unroll
                for (int e = 0; e < V; ++e) y[i][e] = to_f32(from_f32<T>(sc[e] * r[e] + g[e] * ((f[i][e] - mean) * rstd)));   // (the norm reads the stored result)
                store_piece<V>(yr + c, y[i]);
            }
            if (threadIdx.x % TEAM == 0) {
                a.stats[row * a.stats_stride] = mean;
                a.stats[row * a.stats_stride + 1] = rstd;
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = join_column<TEAM, V>(i);
                if (c < D) load_piece<V>(yr + c, y[i]);
            }
        }
        if constexpr (PRE) {
            float mean, rstd;
            row_stats<TEAM, V, N>(y, D, a.rms, mean, rstd, red, place);
            T* const ur = (T*)a.u + row * D;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = join_column<TEAM, V>(i);
                if (c >= D) continue;
                float g[V], b[V];
                load_piece<V>(a.pre_gain + c, g);
                if (a.pre_shift) load_piece<V>(a.pre_shift + c, b);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float n = (y[i][e] - mean) * rstd * g[e];
                    g[e] = a.pre_shift ? n + b[e] : n;
                }
                store_piece<V>(ur + c, g);
            }
            if (threadIdx.x % TEAM == 0) {
                a.pre_stats[row * a.stats_stride] = mean;
                a.pre_stats[row * a.stats_stride + 1] = rstd;
            }
        }
    }
}

template <typename T, int TEAM, int V, int N> static hipError_t fwd_launch(const NormJoin& j, hipStream_t s) {
    const int64_t groups = (j.rows + Team<TEAM>::kRows - 1) / Team<TEAM>::kRows;
    const dim3 grid((unsigned)(groups < (1 << 20) ? groups : 1 << 20)), block(Team<TEAM>::kThreads);
    if (!j.x) return launch_timed(kcLayerNorm, norm_join_fwd_kernel<T, TEAM, V, N, false, true>, grid, block, 0, s, j);
    if (!j.u) return launch_timed(kcLayerNorm, norm_join_fwd_kernel<T, TEAM, V, N, true, false>, grid, block, 0, s, j);
    return launch_timed(kcLayerNorm, norm_join_fwd_kernel<T, TEAM, V, N, true, true>, grid, block, 0, s, j);
}

template <typename T> static hipError_t fwd_type(const NormJoin& j, hipStream_t s) {
    if (j.D <= 64) return fwd_launch<T, 64, 1, 1>(j, s);
    if (j.D <= 1024) return fwd_launch<T, 64, 1, 16>(j, s);
    if (j.D <= 4096) return fwd_launch<T, 256, 1, 16>(j, s);
    return fwd_launch<T, 1024, 1, 16>(j, s);
}

hipError_t norm_join_forward(int dtype, const NormJoin& j, hipStream_t s) {
    if (j.rows <= 0) return hipSuccess;
    if (j.D < 1 || j.D > kJoinMaxFeatures) return hipErrorInvalidValue;
    return dtype == kBF16 ? fwd_type<bf16_t>(j, s) : fwd_type<float>(j, s);
}

}  // namespace tmps
