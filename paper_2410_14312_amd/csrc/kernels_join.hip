// Norm joins, forward: y = scale r + g gain n(f) and u = n(y) pre_gain + pre_shift in one pass over memory.  Bound by memory: f, r (and the gate's argument) are
// read, y and u written once each.  With the norm behind it, in bf16 (us of a launch between two time stamps; a copy of as many bytes at the 5.1 TB/s that one of a gigabyte reaches):
// 8192 x 768 gated 16.9 (12.4), 16384 x 4096 103 (106), 8192 x 8192 100 (106), 32768 x 256 13.9 (13.3); in fp32 4096 x 1024 gated 15.2 (16.6).  Small ones are a launch and two or three sums over
// a team: 256 x 64 4 us.
#include "launch.h"
#include "norm_join.hip.h"

namespace tmps {

// Threads of a launch at most: eight waves to a SIMD, of which four or five are resident.  (With fewer, whole rounds of rows are left over: 8192 x 8192 in bf16 166 us with a quarter,
// 99 with half, 99 with all of them, 109 with twice as many.)
constexpr int kFwdThreads = 524288;

// Mean (0 with rms) and 1/std of a row in registers; the variance is that of the differences from the mean.
template <int TEAM, int N, int V, bool WHOLE>
__device__ __forceinline__ void row_stats(const float (&v)[N][V], const Pieces<TEAM, N, V, WHOLE>& p, bool rms, float& mean, float& rstd, float (*red)[2 * 16], int& place) {
    float s[1] = {0.0f};
    mean = 0.0f;
    if (!rms) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (p.any(i)) {
#pragma unroll
                for (int e = 0; e < V; ++e) s[0] += p.own(i, e) ? v[i][e] : 0.0f;
            }
        Team<TEAM>::sums(s, red, place);
        mean = s[0] / (float)p.D;
        s[0] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (p.any(i)) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = p.own(i, e) ? v[i][e] - mean : 0.0f;
                s[0] = fmaf(d, d, s[0]);
            }
        }
    Team<TEAM>::sums(s, red, place);
    rstd = 1.0f / sqrtf(s[0] / (float)p.D + 1e-5f);
}

// A team to a row at a time; the next row's pieces are requested before this one's are needed, parameters stay in registers.  (With 16 features a thread, the widest rows, there are
// no registers for either: parameters come from the caches with each row.)
template <typename T, int TEAM, int N, bool WHOLE, bool JOIN, bool PRE, bool GATE>
__global__ __launch_bounds__(Team<TEAM>::kThreads) void norm_join_fwd_kernel(NormJoin a) {
    __shared__ float red[2][2 * 16];
    constexpr int V = kPiece<T>;
    const int D = a.D;
    constexpr int wide = GATE ? 2 : 1;
    constexpr bool KEEP = N * V == 8;
    const Pieces<TEAM, N, V, WHOLE> p{D};
    int place = 0;
    const int64_t step = (int64_t)gridDim.x * Team<TEAM>::kRows;
    int64_t row = (int64_t)blockIdx.x * Team<TEAM>::kRows + threadIdx.x / TEAM;
    if (row >= a.rows) return;   // (teams of a workgroup with barriers are the whole of it)
    uint4 rf[N], ra[GATE ? N : 1], rr[N];
    auto request = [&](int64_t at) {
        if constexpr (JOIN) {
            request_row(rf, (const T*)a.x + at * D * wide, p);
            request_row(rr, (const T*)a.r + at * D, p);
            if constexpr (GATE) request_row(ra, (const T*)a.x + at * D * wide + D, p);
        } else {
            request_row(rf, (const T*)a.y + at * D, p);
        }
    };
    if constexpr (KEEP) request(row);
    float gain[KEEP ? N : 1][V], scale[KEEP ? N : 1][V], pre_gain[KEEP ? N : 1][V], pre_shift[KEEP ? N : 1][V];
    if constexpr (KEEP) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (JOIN) {
                load_vector(gain[i], a.gain, p, i);
                load_vector(scale[i], a.scale, p, i);
            }
            if constexpr (PRE) {
                load_vector(pre_gain[i], a.pre_gain, p, i);
                load_vector(pre_shift[i], a.pre_shift, p, i);
            }
        }
    }
    for (; row < a.rows; row += step) {
        if constexpr (!KEEP) request(row);
        float f[N][V], y[N][V], g[GATE ? N : 1][V];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            unpack(rf[i], f[i]);
            if constexpr (JOIN) unpack(rr[i], y[i]);
            else {
#pragma unroll
                for (int e = 0; e < V; ++e) y[i][e] = f[i][e];
            }
            if constexpr (GATE) unpack(ra[i], g[i]);
        }
        if constexpr (KEEP)
            if (row + step < a.rows) request(row + step);
        T* const yr = (T*)a.y + row * D;
        if constexpr (JOIN) {
            float mean, rstd;
            row_stats(f, p, a.rms, mean, rstd, red, place);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (!p.any(i)) continue;
                if constexpr (!KEEP) {
                    load_vector(gain[0], a.gain, p, i);
                    load_vector(scale[0], a.scale, p, i);
                }
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float w = gain[KEEP ? i : 0][e];
                    if constexpr (GATE) {
                        float on, rest;
                        gate_of<T>(g[i][e], on, rest);
                        w *= on;
                    }
                    y[i][e] = fmaf(w, (f[i][e] - mean) * rstd, y[i][e] * scale[KEEP ? i : 0][e]);
                }
                const uint4 stored = pack(y[i]);
                store_packed(yr, p, i, stored);
                unpack(stored, y[i]);   // (the norm reads the stored result)
            }
            if (threadIdx.x % TEAM == 0) {
                a.stats[row * a.stats_stride] = mean;
                a.stats[row * a.stats_stride + 1] = rstd;
            }
        }
        if constexpr (PRE) {
            float mean, rstd;
            row_stats(y, p, a.rms, mean, rstd, red, place);
            T* const ur = (T*)a.u + row * D;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (!p.any(i)) continue;
                if constexpr (!KEEP) {
                    load_vector(pre_gain[0], a.pre_gain, p, i);
                    load_vector(pre_shift[0], a.pre_shift, p, i);
                }
#pragma unroll
                for (int e = 0; e < V; ++e) f[i][e] = fmaf((y[i][e] - mean) * rstd, pre_gain[KEEP ? i : 0][e], pre_shift[KEEP ? i : 0][e]);
                store_piece(ur, p, i, f[i]);
            }
            if (threadIdx.x % TEAM == 0) {
                a.pre_stats[row * a.stats_stride] = mean;
                a.pre_stats[row * a.stats_stride + 1] = rstd;
            }
        }
    }
}

template <typename T, int TEAM, int N, bool WHOLE> static hipError_t fwd_launch(const NormJoin& j, hipStream_t s) {
    const int64_t groups = (j.rows + Team<TEAM>::kRows - 1) / Team<TEAM>::kRows;
    const int most = kFwdThreads / Team<TEAM>::kThreads;
    const dim3 grid((unsigned)(groups < most ? groups : most)), block(Team<TEAM>::kThreads);
    auto kern = !j.x ? norm_join_fwd_kernel<T, TEAM, N, WHOLE, false, true, false>
                : !j.u ? (j.gate ? norm_join_fwd_kernel<T, TEAM, N, WHOLE, true, false, true> : norm_join_fwd_kernel<T, TEAM, N, WHOLE, true, false, false>)
                       : (j.gate ? norm_join_fwd_kernel<T, TEAM, N, WHOLE, true, true, true> : norm_join_fwd_kernel<T, TEAM, N, WHOLE, true, true, false>);
    return launch_timed(kcLayerNorm, kern, grid, block, 0, s, j);
}

template <typename T> static hipError_t fwd_type(const NormJoin& j, hipStream_t s) {
    if (join_whole<T>(j.D, {j.x, j.r, j.gain, j.scale, j.y, j.pre_gain, j.pre_shift, j.u})) {
        if (j.D <= 128) return fwd_launch<T, 16, kOne<T>, true>(j, s);
        if (j.D <= 256) return fwd_launch<T, 32, kOne<T>, true>(j, s);
        if (j.D <= 512) return fwd_launch<T, 64, kOne<T>, true>(j, s);
        if (j.D <= 1024) return fwd_launch<T, 128, kOne<T>, true>(j, s);
        if (j.D <= 2048) return fwd_launch<T, 256, kOne<T>, true>(j, s);
        if (j.D <= 4096) return fwd_launch<T, 512, kOne<T>, true>(j, s);
        if (j.D <= 8192) return fwd_launch<T, 1024, kOne<T>, true>(j, s);
        return fwd_launch<T, 1024, 2 * kOne<T>, true>(j, s);
    }
    if (j.D <= 128) return fwd_launch<T, 16, kOne<T>, false>(j, s);
    if (j.D <= 512) return fwd_launch<T, 64, kOne<T>, false>(j, s);
    if (j.D <= 1024) return fwd_launch<T, 128, kOne<T>, false>(j, s);
    if (j.D <= 2048) return fwd_launch<T, 256, kOne<T>, false>(j, s);
    if (j.D <= 4096) return fwd_launch<T, 512, kOne<T>, false>(j, s);
    if (j.D <= 8192) return fwd_launch<T, 1024, kOne<T>, false>(j, s);
    return fwd_launch<T, 1024, 2 * kOne<T>, false>(j, s);
}

hipError_t norm_join_forward(int dtype, const NormJoin& j, hipStream_t s) {
    if (j.rows <= 0) return hipSuccess;
    if (j.D < 1 || j.D > kJoinMaxFeatures) return hipErrorInvalidValue;
    return dtype == kBF16 ? fwd_type<bf16_t>(j, s) : fwd_type<float>(j, s);
}

}  // namespace tmps
