// Norm joins, forward: y = scale r + g gain n(f) and u = n(y) pre_gain + pre_shift in one pass over memory.  Bound by memory: f, r (and the gate's argument) are
// read, y and u written once each.
#include "launch.h"
#include "norm_join.hip.h"

namespace tmps {

constexpr int kFwdGroups = 2048;

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

// A team to a row at a time; the next row's pieces are requested before this one's are needed, parameters stay in registers.
template <typename T, int TEAM, int V, int N, bool JOIN, bool PRE, bool GATE>
__global__ __launch_bounds__(Team<TEAM>::kThreads) void norm_join_fwd_kernel(NormJoin a) {
    __shared__ float red[2][4 * 16];
    const int D = a.D;
    constexpr int wide = GATE ? 2 : 1;
    int place = 0;
    const int64_t step = (int64_t)gridDim.x * Team<TEAM>::kRows;
    int64_t row = (int64_t)blockIdx.x * Team<TEAM>::kRows + threadIdx.x / TEAM;
    if (row >= a.rows) return;   // (whole waves, or the whole workgroup)
    RawPiece<T, V> rf[N], ra[GATE ? N : 1], rr[N];
    auto request = [&](int64_t at) {
        if constexpr (JOIN) {
            request_row<T, TEAM, V, N>(rf, (const T*)a.x + at * D * wide, D);
            request_row<T, TEAM, V, N>(rr, (const T*)a.r + at * D, D);
            if constexpr (GATE) request_row<T, TEAM, V, N>(ra, (const T*)a.x + at * D * wide + D, D);
        } else {
            request_row<T, TEAM, V, N>(rf, (const T*)a.y + at * D, D);
        }
    };
    request(row);
    float gain[JOIN ? N : 1][V], scale[JOIN ? N : 1][V], pre_gain[PRE ? N : 1][V], pre_shift[PRE ? N : 1][V];
    if constexpr (JOIN) {
        load_vector<TEAM, V, N>(gain, a.gain, D);
        load_vector<TEAM, V, N>(scale, a.scale, D);
    }
    if constexpr (PRE) {
        load_vector<TEAM, V, N>(pre_gain, a.pre_gain, D);
        load_vector<TEAM, V, N>(pre_shift, a.pre_shift, a.pre_shift ? D : 0);
    }
    for (; row < a.rows; row += step) {
        float f[N][V], y[N][V];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            rf[i].get(f[i]);
            if constexpr (JOIN) {
                rr[i].get(y[i]);
#pragma unroll
                for (int e = 0; e < V; ++e) y[i][e] *= scale[i][e];
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) y[i][e] = f[i][e];
            }
        }
        float g[GATE ? N : 1][V];
        if constexpr (GATE) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                ra[i].get(g[i]);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float rest;
                    gate_of<T>(g[i][e], g[i][e], rest);
                    g[i][e] *= gain[i][e];
                }
            }
        }
        if (row + step < a.rows) request(row + step);
        T* const yr = (T*)a.y + row * D;
        if constexpr (JOIN) {
            float mean, rstd;
            row_stats<TEAM, V, N>(f, D, a.rms, mean, rstd, red, place);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = join_column<TEAM, V>(i);
                if (c >= D) continue;
#pragma unroll
                for (int e = 0; e < V; ++e) y[i][e] = to_f32(from_f32<T>(fmaf(GATE ? g[GATE ? i : 0][e] : gain[i][e], (f[i][e] - mean) * rstd, y[i][e])));   // (the norm reads the stored result)
                store_piece<V>(yr + c, y[i]);
            }
            if (threadIdx.x % TEAM == 0) {
                a.stats[row * a.stats_stride] = mean;
                a.stats[row * a.stats_stride + 1] = rstd;
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
#pragma unroll
                for (int e = 0; e < V; ++e) f[i][e] = fmaf((y[i][e] - mean) * rstd, pre_gain[i][e], pre_shift[i][e]);
                store_piece<V>(ur + c, f[i]);
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
    const dim3 grid((unsigned)(groups < kFwdGroups ? groups : kFwdGroups)), block(Team<TEAM>::kThreads);
    auto kern = !j.x ? norm_join_fwd_kernel<T, TEAM, V, N, false, true, false>
                : !j.u ? (j.gate ? norm_join_fwd_kernel<T, TEAM, V, N, true, false, true> : norm_join_fwd_kernel<T, TEAM, V, N, true, false, false>)
                       : (j.gate ? norm_join_fwd_kernel<T, TEAM, V, N, true, true, true> : norm_join_fwd_kernel<T, TEAM, V, N, true, true, false>);
    return launch_timed(kcLayerNorm, kern, grid, block, 0, s, j);
}

template <typename T> static hipError_t fwd_type(const NormJoin& j, hipStream_t s) {
    if (join_wide(j.D, {j.x, j.r, j.gain, j.scale, j.y, j.pre_gain, j.pre_shift, j.u})) {
        if (j.D <= 512) return fwd_launch<T, 64, 8, 1>(j, s);
        if (j.D <= 1024) return fwd_launch<T, 64, 8, 2>(j, s);
        if (j.D <= 2048) return fwd_launch<T, 256, 8, 1>(j, s);
        if (j.D <= 4096) return fwd_launch<T, 256, 8, 2>(j, s);
        if (j.D <= 8192) return fwd_launch<T, 1024, 8, 1>(j, s);
        return fwd_launch<T, 1024, 8, 2>(j, s);
    }
    if (j.D <= 64) return fwd_launch<T, 64, 1, 1>(j, s);
    if (j.D <= 256) return fwd_launch<T, 64, 1, 4>(j, s);
    if (j.D <= 1024) return fwd_launch<T, 256, 1, 4>(j, s);
    if (j.D <= 4096) return fwd_launch<T, 1024, 1, 4>(j, s);
    return fwd_launch<T, 1024, 1, 16>(j, s);
}

hipError_t norm_join_forward(int dtype, const NormJoin& j, hipStream_t s) {
    if (j.rows <= 0) return hipSuccess;
    if (j.D < 1 || j.D > kJoinMaxFeatures) return hipErrorInvalidValue;
    return dtype == kBF16 ? fwd_type<bf16_t>(j, s) : fwd_type<float>(j, s);
}

}  // namespace tmps
