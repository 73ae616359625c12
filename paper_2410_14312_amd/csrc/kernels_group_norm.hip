// Group norm with its activation, and its gradients.  Three forms, all bound by memory:
//   rows  one position a sample: each group of a sample is a row of its own, held in the registers of a team of threads, one pass (8192 rows of 24 groups of 64 in bf16: 10.4 us, a copy's rate);
//   held  a sample's map fits the registers of a workgroup: one pass (8 maps of 64 x 64: 6.9 us; 277 of 25 x 944 in bf16: 22);
//   maps  larger ones: sums of slices of positions, the samples' sums, and a second pass over the map (32 of 3136 x 256 in bf16: 35 us, back 62, of which 9 for the sums of slices and samples).
// Of a group's values the mean is taken first and the differences from it squared; what several threads or slices have is joined as (number, mean, sum of squared differences).
#include <algorithm>

#include "launch.h"
#include "mixer.h"
#include "norm_join.hip.h"

#pragma clang fp contract(off)

namespace tmps {

// xhat = (x - mean) rstd and z = gain xhat + shift, the same bits in both passes (and so a ReLU's border).  The mean is taken off first: of values that are all the same nothing is left.
__device__ __forceinline__ float norm_z(float x, float mean, float rstd, float gain, float shift, float& xhat) {
    xhat = (x - mean) * rstd;
    return fmaf(gain, xhat, shift);
}

// The hardware's exponential and reciprocal are off by some 2^-23, enough for results of 8 bits, not for fp32.
template <typename T> __device__ __forceinline__ float norm_sigmoid(float z) {
    if constexpr (sizeof(T) == 2) return __builtin_amdgcn_rcpf(1.0f + __expf(-z));
    return 1.0f / (1.0f + expf(-z));
}
template <typename T> __device__ __forceinline__ float norm_act(int act, float z) {
    if (act == kNormActRelu) return z > 0.0f ? z : (z != z ? z : 0.0f);
    if (act == kNormActGelu) return sizeof(T) == 2 ? gelu_f(z) : z * (0.5f + 0.5f * erff(z * 0.70710678118654752f));
    if (act == kNormActSilu) return z * norm_sigmoid<T>(z);
    return z;
}
// (the activation is asked for once)
template <typename T, int V> __device__ __forceinline__ void norm_act_all(int act, float (&z)[V]) {
    if (act == kNormActSilu) {
#pragma unroll
        for (int e = 0; e < V; ++e) z[e] = norm_act<T>(kNormActSilu, z[e]);
    } else if (act == kNormActRelu) {
#pragma unroll
        for (int e = 0; e < V; ++e) z[e] = norm_act<T>(kNormActRelu, z[e]);
    } else if (act == kNormActGelu) {
#pragma unroll
        for (int e = 0; e < V; ++e) z[e] = norm_act<T>(kNormActGelu, z[e]);
    }
}
template <typename T> __device__ __forceinline__ float norm_act_grad(int act, float z, float dy) {
    if (act == kNormActRelu) return z > 0.0f ? dy : 0.0f;
    if (act == kNormActGelu)
        return dy * (sizeof(T) == 2 ? gelu_grad_f(z) : 0.5f + 0.5f * erff(z * 0.70710678118654752f) + z * 0.3989422804014327f * expf(-0.5f * z * z));
    if (act == kNormActSilu) {
        const float g = norm_sigmoid<T>(z);
        return dy * (g * (1.0f + z * (1.0f - g)));
    }
    return dy;
}

// (count, mean, sum of squared differences) of two sets as one
__device__ __forceinline__ void join_moments(float& n, float& mean, float& m2, float n2, float mean2, float m22) {
    if (n2 == 0.0f) return;
    const float d = mean2 - mean, share = n2 * __builtin_amdgcn_rcpf(n + n2);   // (off by a step, of the means' difference)
    mean = fmaf(d, share, mean);
    m2 += fmaf(d * (n * share), d, m22);
    n += n2;
}

// ------------------------------------------------------------------------------------------------ rows
constexpr int kGroupRowThreads = 524288;   // threads of a launch at most; backward, where teams leave partial results, kBackRowThreads
constexpr int kBackRowThreads = 262144;     // (4000 rows of 4096 in bf16: 43 us, with 524288 51, with 131072 68)

// The rows are the samples' groups; a team's rows are a whole number of samples apart, so that its group's parameters stay in registers.
template <typename T, int TEAM, int N, bool WHOLE> __global__ __launch_bounds__(Team<TEAM>::kThreads) void group_rows_fwd_kernel(GroupNorm a, int64_t step) {
    __shared__ float red[2][2 * 16];
    constexpr int V = kPiece<T>;
    const int D = a.channels / a.groups;
    const Pieces<TEAM, N, V, WHOLE> p{D};
    const int64_t rows = a.samples * a.groups;
    int64_t row = (int64_t)blockIdx.x * Team<TEAM>::kRows + threadIdx.x / TEAM;
    if (row >= step) return;   // (teams of a workgroup with barriers are the whole of it)
    int place = 0;
    const int group = (int)(row % a.groups);
    const float part = 1.0f / (float)D;   // (a quotient and a root of every row, by the library, would be a fifth of its instructions; the hardware's root is off by a step)
    float gain[N][V], shift[N][V];
    uint4 next[N];
    request_row(next, (const T*)a.x + row * D, p);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        load_vector(gain[i], a.gain + (int64_t)group * D, p, i);
        load_vector(shift[i], a.shift ? a.shift + (int64_t)group * D : nullptr, p, i);
    }
    for (; row < rows; row += step) {
        float v[N][V];
        float s[1] = {0.0f}, mean = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            unpack(next[i], v[i]);
            if (!a.rms && p.any(i)) {
#pragma unroll
                for (int e = 0; e < V; ++e) s[0] += p.own(i, e) ? v[i][e] : 0.0f;
            }
        }
        if (row + step < rows) request_row(next, (const T*)a.x + (row + step) * D, p);
        if (!a.rms) {
            Team<TEAM>::sums(s, red, place);
            mean = s[0] * part;
        }
        const auto squares = [&](float of) {
            s[0] = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (p.any(i)) {
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float d = p.own(i, e) ? v[i][e] - of : 0.0f;
                        s[0] = fmaf(d, d, s[0]);
                    }
                }
            Team<TEAM>::sums(s, red, place);
        };
        if (a.rms) squares(0.0f);
        else squares(mean);
        // Where the values lie far from 0 for what they differ by (or their squares are beyond a float), what the sum and the share have rounded is added to the mean, and the differences are
        // taken anew: of values that are all the same the mean is then the value in every bit.  (For every row it is one more sum of the team: 4096 rows of 4096 in bf16 21 us instead of 17.)
        if (!a.rms && mean != 0.0f && s[0] * part <= 0x1p-16f * (mean * mean)) {
            s[0] = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (p.any(i)) {
#pragma unroll
                    for (int e = 0; e < V; ++e) s[0] += p.own(i, e) ? v[i][e] - mean : 0.0f;
                }
            Team<TEAM>::sums(s, red, place);
            mean = fmaf(s[0], part, mean);
            squares(mean);
        }
        const float rstd = __builtin_amdgcn_rsqf(fmaf(s[0], part, 1e-5f));
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (!p.any(i)) continue;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float xhat;
                v[i][e] = norm_z(v[i][e], mean, rstd, gain[i][e], shift[i][e], xhat);
            }
            norm_act_all<T>(a.act, v[i]);
            store_piece((T*)a.y + row * D, p, i, v[i]);
        }
        if (threadIdx.x % TEAM == 0) {
            a.stats[2 * row] = mean;
            a.stats[2 * row + 1] = rstd;
        }
    }
}

// part: [step / groups][2][channels], the sums of each team's rows.
template <typename T, int TEAM, int N, bool WHOLE> __global__ __launch_bounds__(Team<TEAM>::kThreads) void group_rows_bwd_kernel(GroupNormBackward a, int64_t step, float* part) {
    __shared__ float red[2][2 * 16];
    constexpr int V = kPiece<T>;
    const int D = a.channels / a.groups;
    const Pieces<TEAM, N, V, WHOLE> p{D};
    const int64_t rows = a.samples * a.groups;
    int64_t row = (int64_t)blockIdx.x * Team<TEAM>::kRows + threadIdx.x / TEAM;
    if (row >= step) return;
    int place = 0;
    const int group = (int)(row % a.groups);
    const float share = 1.0f / (float)D;
    float* const mine = part + (row / a.groups) * 2 * (int64_t)a.channels + (int64_t)group * D;
    float gain[N][V], shift[N][V], dgain[N][V], dshift[N][V];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        load_vector(gain[i], a.gain + (int64_t)group * D, p, i);
        load_vector(shift[i], a.shift ? a.shift + (int64_t)group * D : nullptr, p, i);
#pragma unroll
        for (int e = 0; e < V; ++e) dgain[i][e] = dshift[i][e] = 0.0f;
    }
    uint4 nx[N], ng[N];
    request_row(nx, (const T*)a.x + row * D, p);
    request_row(ng, (const T*)a.dy + row * D, p);
    for (; row < rows; row += step) {
        const float mean = a.stats[2 * row], rstd = a.stats[2 * row + 1];
        float xhat[N][V], g[N][V];
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < N; ++i) {
            unpack(nx[i], xhat[i]);
            unpack(ng[i], g[i]);
        }
        if (row + step < rows) {
            request_row(nx, (const T*)a.x + (row + step) * D, p);
            request_row(ng, (const T*)a.dy + (row + step) * D, p);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (!p.any(i)) continue;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if (!p.own(i, e)) continue;
                const float z = norm_z(xhat[i][e], mean, rstd, gain[i][e], shift[i][e], xhat[i][e]);
                const float dz = norm_act_grad<T>(a.act, z, g[i][e]);
                dgain[i][e] = fmaf(dz, xhat[i][e], dgain[i][e]);
                dshift[i][e] += dz;
                g[i][e] = dz * gain[i][e];
                s[0] += g[i][e];
                s[1] = fmaf(g[i][e], xhat[i][e], s[1]);
            }
        }
        Team<TEAM>::sums(s, red, place);
        const float of_mean = a.rms ? 0.0f : s[0] * share, of_xhat = s[1] * share;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (!p.any(i)) continue;
#pragma unroll
            for (int e = 0; e < V; ++e) g[i][e] = (fmaf(-xhat[i][e], of_xhat, g[i][e]) - of_mean) * rstd;
            store_piece((T*)a.dx + row * D, p, i, g[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (!p.any(i)) continue;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if (!p.own(i, e)) continue;
            mine[p.at(i) + e] = dgain[i][e];
            mine[a.channels + p.at(i) + e] = dshift[i][e];
        }
    }
}

// ------------------------------------------------------------------------------------------------ maps
// A thread has a piece of channels and every `lanes`-th position of its workgroup's slice.  A workgroup has up to 256 pieces; a last piece that begins earlier comes out the same as
// the one before it where both hold a channel.
template <typename T> struct MapPlace {
    static constexpr int V = kPiece<T>;
    int C, pieces, width, lanes, lane, at;   // pieces of a row; of this workgroup; positions side by side; this thread's; its first channel
    bool any;
    __device__ __forceinline__ MapPlace(int channels, int block, int threads, int most = 256) : C(channels), pieces((channels + V - 1) / V) {
        width = min(pieces - block * 256, most);
        lanes = threads / width;
        lane = (int)threadIdx.x / width;
        any = lane < lanes;
        at = min((block * 256 + (int)threadIdx.x % width) * V, max(C - V, 0));
    }
    __device__ __forceinline__ uint4 request(const T* row) const {
        if (C >= V) return load16_any(row + at);
        struct Values { T v[V]; } f;
#pragma unroll
        for (int e = 0; e < V; ++e) f.v[e] = e < C ? row[e] : T(0.0f);
        return __builtin_bit_cast(uint4, f);
    }
    __device__ __forceinline__ void store(T* row, const float (&v)[V]) const {
        if (C >= V) {
            store16_any(row + at, pack(v));
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (e < C) row[e] = from_f32<T>(v[e]);
        }
    }
    // its channels' numbers of a vector (null: zeros)
    __device__ __forceinline__ void params(float (&v)[V], const float* p) const {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = 0.0f;
        if (!p) return;
        if (C >= V) {
#pragma unroll
            for (int e = 0; e < V; e += 4) {
                float f[4];
                unpack(load16_any(p + at + e), f);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[e + k] = f[k];
            }
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = p[min(e, C - 1)];
        }
    }
    // f(e, group) of each
    template <class F> __device__ __forceinline__ void groups(int size, F&& f) const {
        int g = at / size, end = (g + 1) * size;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if (min(at + e, C - 1) >= end) ++g, end += size;
            f(e, g);
        }
    }
    // the two numbers of their groups
    __device__ __forceinline__ void pairs(float (&first)[V], float (&second)[V], const float* p, int size) const {
        groups(size, [&](int e, int g) {
            const any_u32x2_t u = *reinterpret_cast<const any_u32x2_t*>(p + 2 * g);
            const uint32_t a = u[0], b = u[1];
            first[e] = __builtin_bit_cast(float, a);
            second[e] = __builtin_bit_cast(float, b);
        });
    }
};

constexpr int kMapBlock = 8, kMapPairs = 4;   // positions whose values, or values and gradients, a thread has at a time

// Mean and sum of squared differences, by channel, of up to B positions' values; the first `many` count.  With rms the mean is 0.
template <typename T, int B> __device__ __forceinline__ void block_moments(const uint4 (&u)[B], int many, bool rms, float (&mean)[kPiece<T>], float (&m2)[kPiece<T>]) {
    constexpr int V = kPiece<T>;
#pragma unroll
    for (int e = 0; e < V; ++e) mean[e] = m2[e] = 0.0f;
    if (!rms && many > 0) {
        // (that of the differences from the first one, so that of values that are all the same it is the value in every bit)
        float first[V];
        unpack(u[0], first);
#pragma unroll
        for (int k = 1; k < B; ++k)
            if (k < many) {
                float v[V];
                unpack(u[k], v);
#pragma unroll
                for (int e = 0; e < V; ++e) mean[e] += v[e] - first[e];
            }
        const float by = 1.0f / (float)many;
#pragma unroll
        for (int e = 0; e < V; ++e) mean[e] = fmaf(mean[e], by, first[e]);
    }
#pragma unroll
    for (int k = 0; k < B; ++k)
        if (k < many) {
            float v[V];
            unpack(u[k], v);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = v[e] - mean[e];
                m2[e] = fmaf(d, d, m2[e]);
            }
        }
}

// Mean and sum of squared differences of every channel over a slice: part [sample][slice][channels][2].
template <typename T> __global__ __launch_bounds__(256) void group_map_moments_kernel(const T* x, int64_t positions, int channels, int64_t slice, int slices, bool rms, float* part) {
    constexpr int V = kPiece<T>;
    __shared__ float fold[256][2 * V + 1];
    const MapPlace<T> p(channels, blockIdx.y, 256);
    const int64_t sample = blockIdx.x / slices, cut = blockIdx.x % slices;
    const int64_t t0 = cut * slice, t1 = min(t0 + slice, positions);
    const T* const rows = x + sample * positions * channels;
    float n = 0.0f, mean[V], m2[V];
#pragma unroll
    for (int e = 0; e < V; ++e) mean[e] = m2[e] = 0.0f;
    if (p.any) {
        for (int64_t t = t0 + p.lane; t < t1; t += (int64_t)p.lanes * kMapBlock) {
            uint4 u[kMapBlock];
            const int many = (int)min<int64_t>(kMapBlock, (t1 - t + p.lanes - 1) / p.lanes);
#pragma unroll
            for (int k = 0; k < kMapBlock; ++k) u[k] = p.request(rows + min(t + (int64_t)k * p.lanes, t1 - 1) * channels);
            float bm[V], b2[V];
            block_moments<T>(u, many, rms, bm, b2);
            const float all = n + (float)many, share = (float)many / all, between = n * share;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = bm[e] - mean[e];
                mean[e] = fmaf(d, share, mean[e]);
                m2[e] += fmaf(d * between, d, b2[e]);   // (of the first positions' 0: no square of d, which may be infinite)
            }
            n = all;
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
        fold[threadIdx.x][e] = mean[e];
        fold[threadIdx.x][V + e] = m2[e];
    }
    fold[threadIdx.x][2 * V] = n;
    __syncthreads();
    float* const mine = part + (sample * slices + cut) * channels * 2;
    for (int i = threadIdx.x; i < p.width * V; i += 256) {
        const int k = i / V, e = i % V;
        float c = fold[k][2 * V], m = fold[k][e], s = fold[k][V + e];
        for (int l = 1; l < p.lanes; ++l) {
            const float* f = fold[l * p.width + k];
            join_moments(c, m, s, f[2 * V], f[e], f[V + e]);
        }
        const int first = ((int)blockIdx.y * 256 + k) * V, ch = min(first, max(channels - V, 0)) + e;
        if (ch >= first && ch < channels) {
            mine[2 * ch] = m;
            mine[2 * ch + 1] = s;
        }
    }
}

// Moments of a group from those of the LANES lanes that share it.
template <int LANES> __device__ __forceinline__ void join_lanes(float& n, float& mean, float& m2) {
#pragma unroll
    for (int d = LANES / 2; d > 0; d >>= 1) {
        const float n2 = __shfl_xor(n, d), mean2 = __shfl_xor(mean, d), m22 = __shfl_xor(m2, d);
        // (the same in both lanes: the lower one's first)
        const bool low = (threadIdx.x & d) == 0;
        float an = low ? n : n2, am = low ? mean : mean2, as = low ? m2 : m22;
        const float bn = low ? n2 : n, bm = low ? mean2 : mean, bs = low ? m22 : m2;
        if (an == 0.0f) an = bn, am = bm, as = bs;
        else join_moments(an, am, as, bn, bm, bs);
        n = an; mean = am; m2 = as;
    }
}

// The groups' means and 1/std from those of the slices' channels: WAVES waves to a group, eight of a lane's under way at a time.
template <int WAVES> __global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void group_map_stats_kernel(const float* part, int64_t samples, int64_t positions, int channels, int groups,
                                                                                                              int64_t slice, int slices, bool rms, float* stats) {
    __shared__ float waves[WAVES][3];
    constexpr int kThreads = 64 * WAVES;
    const int64_t g = WAVES == 1 ? (int64_t)blockIdx.x * 4 + threadIdx.x / 64 : blockIdx.x;
    if (g >= samples * groups) return;   // (of workgroups with a barrier none)
    const int64_t sample = g / groups;
    const int size = channels / groups, first = (int)(g % groups) * size, lane = (int)threadIdx.x % kThreads;
    const int all = size * slices, last = (int)(positions - (slices - 1) * slice);   // (slices are as many as there are workgroups at most: 2^11, channels 2^16)
    const float2* const from = reinterpret_cast<const float2*>(part) + sample * slices * channels + first;
    float n = 0.0f, mean = 0.0f, m2 = 0.0f;
    for (int i0 = lane; i0 < all; i0 += kThreads * 8) {
        float2 f[8];
        float many[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t i = (uint32_t)min(i0 + kThreads * k, all - 1), cut = i / (uint32_t)size;
            f[k] = from[(int64_t)cut * channels + (i - cut * (uint32_t)size)];
            many[k] = i0 + kThreads * k >= all ? 0.0f : (int)cut == slices - 1 ? (float)last : (float)slice;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (n == 0.0f) n = many[k], mean = f[k].x, m2 = f[k].y;
            else join_moments(n, mean, m2, many[k], f[k].x, f[k].y);
        }
    }
    join_lanes<64>(n, mean, m2);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) {
            waves[threadIdx.x / 64][0] = n;
            waves[threadIdx.x / 64][1] = mean;
            waves[threadIdx.x / 64][2] = m2;
        }
        __syncthreads();
#pragma unroll
        for (int w = 1; w < WAVES; ++w) join_moments(n, mean, m2, waves[w][0], waves[w][1], waves[w][2]);
    }
    if (lane == 0) {
        stats[2 * g] = rms ? 0.0f : mean;
        stats[2 * g + 1] = 1.0f / sqrtf(m2 / ((float)size * (float)positions) + 1e-5f);
    }
}

template <typename T> __global__ __launch_bounds__(256) void group_map_apply_kernel(GroupNorm a, int64_t slice, int slices) {
    constexpr int V = kPiece<T>;
    const MapPlace<T> p(a.channels, blockIdx.y, 256);
    if (!p.any) return;
    const int64_t sample = blockIdx.x / slices, cut = blockIdx.x % slices;
    const int64_t t0 = cut * slice, t1 = min(t0 + slice, a.positions);
    const int size = a.channels / a.groups;
    const float* const stats = a.stats + sample * a.groups * 2;
    float mean[V], rstd[V], gain[V], shift[V];
    p.pairs(mean, rstd, stats, size);
    p.params(gain, a.gain);
    p.params(shift, a.shift);
    const T* const x = (const T*)a.x + sample * a.positions * a.channels;
    T* const y = (T*)a.y + sample * a.positions * a.channels;
    for (int64_t t = t0 + p.lane; t < t1; t += (int64_t)p.lanes * kMapPairs) {
        uint4 u[kMapPairs];
#pragma unroll
        for (int k = 0; k < kMapPairs; ++k) u[k] = p.request(x + min(t + (int64_t)k * p.lanes, t1 - 1) * a.channels);
#pragma unroll
        for (int k = 0; k < kMapPairs; ++k) {
            const int64_t at = t + (int64_t)k * p.lanes;
            if (at >= t1) continue;
            float v[V];
            unpack(u[k], v);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float xhat;
                v[e] = norm_z(v[e], mean[e], rstd[e], gain[e], shift[e], xhat);
            }
            norm_act_all<T>(a.act, v);
            p.store(y + at * a.channels, v);
        }
    }
}

// Sums of dz xhat and of dz of every channel over a slice: part [sample][slice][2][channels].
template <typename T> __global__ __launch_bounds__(256) void group_map_sums_kernel(GroupNormBackward a, int64_t slice, int slices, float* part) {
    constexpr int V = kPiece<T>;
    __shared__ float fold[256][2 * V];
    const MapPlace<T> p(a.channels, blockIdx.y, 256);
    const int64_t sample = blockIdx.x / slices, cut = blockIdx.x % slices;
    const int64_t t0 = cut * slice, t1 = min(t0 + slice, a.positions);
    float with_xhat[V], alone[V];
#pragma unroll
    for (int e = 0; e < V; ++e) with_xhat[e] = alone[e] = 0.0f;
    if (p.any) {
        const int size = a.channels / a.groups;
        const float* const stats = a.stats + sample * a.groups * 2;
        float mean[V], rstd[V], gain[V], shift[V];
        p.pairs(mean, rstd, stats, size);
        p.params(gain, a.gain);
        p.params(shift, a.shift);
        const T* const x = (const T*)a.x + sample * a.positions * a.channels;
        const T* const dy = (const T*)a.dy + sample * a.positions * a.channels;
        for (int64_t t = t0 + p.lane; t < t1; t += (int64_t)p.lanes * kMapPairs) {
            uint4 ux[kMapPairs], ug[kMapPairs];
#pragma unroll
            for (int k = 0; k < kMapPairs; ++k) {
                const int64_t row = min(t + (int64_t)k * p.lanes, t1 - 1) * a.channels;
                ux[k] = p.request(x + row);
                ug[k] = p.request(dy + row);
            }
#pragma unroll
            for (int k = 0; k < kMapPairs; ++k) {
                if (t + (int64_t)k * p.lanes >= t1) continue;
                float v[V], g[V];
                unpack(ux[k], v);
                unpack(ug[k], g);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float xhat;
                    const float z = norm_z(v[e], mean[e], rstd[e], gain[e], shift[e], xhat);
                    const float dz = norm_act_grad<T>(a.act, z, g[e]);
                    with_xhat[e] = fmaf(dz, xhat, with_xhat[e]);
                    alone[e] += dz;
                }
            }
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
        fold[threadIdx.x][e] = with_xhat[e];
        fold[threadIdx.x][V + e] = alone[e];
    }
    __syncthreads();
    float* const mine = part + (sample * slices + cut) * 2 * a.channels;
    for (int i = threadIdx.x; i < 2 * p.width * V; i += 256) {
        const int which = i / (p.width * V), k = i / V % p.width, e = i % V;
        float s = 0.0f;
        for (int l = 0; l < p.lanes; ++l) s += fold[l * p.width + k][which * V + e];
        const int first = ((int)blockIdx.y * 256 + k) * V, ch = min(first, max(a.channels - V, 0)) + e;
        if (ch >= first && ch < a.channels) mine[which * (int64_t)a.channels + ch] = s;
    }
}

// The slices' sums of a sample's channels added up, and of them each group's means of gain dz and of gain dz xhat over its values.  A workgroup has whole groups, `columns` channels of a
// sample: sums [sample][2][channels], means [samples][groups][2].
__global__ __launch_bounds__(512) void group_map_fold_kernel(const float* part, const float* gain, int64_t positions, int channels, int groups, int columns, int slices, bool rms, float* sums,
                                                             float* means) {
    __shared__ float fold[512];
    const int blocks = (channels + columns - 1) / columns;
    const int64_t sample = blockIdx.x / blocks;
    const int c0 = (int)(blockIdx.x % blocks) * columns, width = min(columns, channels - c0), size = channels / groups;
    const float* const from = part + sample * slices * 2 * channels;
    float* const to = sums + sample * 2 * channels;
    // (lanes of slices to a sum: as many as fill the workgroup)
    const int lanes = max(1, 512 / (2 * width)), lane = (int)threadIdx.x / (2 * width);
    for (int i0 = 0; i0 < 2 * width; i0 += 512) {
        const int i = lanes > 1 ? (int)threadIdx.x % (2 * width) : i0 + (int)threadIdx.x;
        const bool any = i < 2 * width && lane < lanes;
        const int64_t column = (int64_t)(i / width) * channels + c0 + i % width;
        float s = 0.0f;
        if (any)
            for (int z = lanes > 1 ? lane : 0; z < slices; z += lanes * 8) {
                float v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = from[(int64_t)min(z + k * lanes, slices - 1) * 2 * channels + column];
#pragma unroll
                for (int k = 0; k < 8; ++k) s += z + k * lanes < slices ? v[k] : 0.0f;
            }
        if (lanes > 1) {
            fold[threadIdx.x] = s;
            __syncthreads();
            if (lane == 0)
                for (int l = 1; l < lanes; ++l) s += fold[l * 2 * width + i];
        }
        if (any && (lanes == 1 || lane == 0)) to[column] = s;
    }
    __threadfence_block();
    __syncthreads();
    // eight lanes to a group
    const float n = (float)size * (float)positions;
    for (int g = (int)threadIdx.x / 8; g < width / size; g += 64) {
        float with_xhat = 0.0f, alone = 0.0f;
        for (int i = threadIdx.x % 8; i < size; i += 8) {
            const int c = c0 + g * size + i;
            with_xhat = fmaf(gain[c], to[c], with_xhat);
            alone = fmaf(gain[c], to[channels + c], alone);
        }
#pragma unroll
        for (int d = 4; d > 0; d >>= 1) {
            with_xhat += __shfl_xor(with_xhat, d);
            alone += __shfl_xor(alone, d);
        }
        if (threadIdx.x % 8 == 0) {
            float* const mean = means + (sample * groups + c0 / size + g) * 2;
            mean[0] = rms ? 0.0f : alone / n;
            mean[1] = with_xhat / n;
        }
    }
}

template <typename T> __global__ __launch_bounds__(256) void group_map_apply_bwd_kernel(GroupNormBackward a, int64_t slice, int slices, const float* means) {
    constexpr int V = kPiece<T>;
    const MapPlace<T> p(a.channels, blockIdx.y, 256);
    if (!p.any) return;
    const int64_t sample = blockIdx.x / slices, cut = blockIdx.x % slices;
    const int64_t t0 = cut * slice, t1 = min(t0 + slice, a.positions);
    const int size = a.channels / a.groups;
    const float *const stats = a.stats + sample * a.groups * 2, *const of = means + sample * a.groups * 2;
    float mean[V], rstd[V], gain[V], shift[V], alone[V], with_xhat[V];
    p.pairs(mean, rstd, stats, size);
    p.pairs(alone, with_xhat, of, size);
    p.params(gain, a.gain);
    p.params(shift, a.shift);
    const T* const x = (const T*)a.x + sample * a.positions * a.channels;
    const T* const dy = (const T*)a.dy + sample * a.positions * a.channels;
    T* const dx = (T*)a.dx + sample * a.positions * a.channels;
    for (int64_t t = t0 + p.lane; t < t1; t += (int64_t)p.lanes * kMapPairs) {
        uint4 ux[kMapPairs], ug[kMapPairs];
#pragma unroll
        for (int k = 0; k < kMapPairs; ++k) {
            const int64_t row = min(t + (int64_t)k * p.lanes, t1 - 1) * a.channels;
            ux[k] = p.request(x + row);
            ug[k] = p.request(dy + row);
        }
#pragma unroll
        for (int k = 0; k < kMapPairs; ++k) {
            const int64_t at = t + (int64_t)k * p.lanes;
            if (at >= t1) continue;
            float v[V], g[V];
            unpack(ux[k], v);
            unpack(ug[k], g);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float xhat;
                const float z = norm_z(v[e], mean[e], rstd[e], gain[e], shift[e], xhat);
                const float dz = norm_act_grad<T>(a.act, z, g[e]) * gain[e];
                v[e] = (fmaf(-xhat, with_xhat[e], dz) - alone[e]) * rstd[e];
            }
            p.store(dx + at * a.channels, v);
        }
    }
}

// ------------------------------------------------------------------------------------------------ held
// A workgroup has a sample, its threads every `lanes`-th position of a piece of channels each.
constexpr int kHeldPieces = 8, kHeldPairs = 4;   // of a thread: values, values and gradients
constexpr int kHeldGroups = 512;

// Lanes that share an item of `items` of a workgroup's.
__device__ __forceinline__ int lanes_each(int threads, int items) {
    int n = 1;
    while (n < 64 && 2 * n * items <= threads) n *= 2;
    return n;
}

template <typename T, int THREADS> __global__ __launch_bounds__(THREADS) void group_held_fwd_kernel(GroupNorm a) {
    constexpr int V = kPiece<T>;
    __shared__ float fold[THREADS][2 * V + 1];
    __shared__ float group_stats[kHeldGroups][2];
    const MapPlace<T> p(a.channels, 0, THREADS, THREADS);
    const int64_t sample = blockIdx.x;
    const int positions = (int)a.positions, size = a.channels / a.groups;
    const T* const x = (const T*)a.x + sample * a.positions * a.channels;
    uint4 u[kHeldPieces];
    const int many = p.any && p.lane < positions ? (positions - p.lane + p.lanes - 1) / p.lanes : 0;
#pragma unroll
    for (int k = 0; k < kHeldPieces; ++k)
        if (k * p.lanes < positions) u[k] = p.request(x + (int64_t)min(p.lane + k * p.lanes, positions - 1) * a.channels);
    float mean[V], m2[V], gain[V], shift[V];
    p.params(gain, a.gain);
    p.params(shift, a.shift);
    block_moments<T>(u, many, a.rms, mean, m2);
#pragma unroll
    for (int e = 0; e < V; ++e) {
        fold[threadIdx.x][e] = mean[e];
        fold[threadIdx.x][V + e] = m2[e];
    }
    fold[threadIdx.x][2 * V] = (float)many;
    __syncthreads();
    // the channels' moments, to the rows of the first lane
    {
        const int items = p.width * V, sub = lanes_each(THREADS, items), h = threadIdx.x % sub;
        for (int i0 = 0; i0 < items; i0 += THREADS / sub) {
            const int i = i0 + (int)threadIdx.x / sub, k = min(i, items - 1) / V, e = i % V;
            float n = 0.0f, m = 0.0f, s = 0.0f;
            for (int l = h; l < p.lanes; l += sub) {
                const float* const f = fold[l * p.width + k];
                if (n == 0.0f) n = f[2 * V], m = f[e], s = f[V + e];
                else join_moments(n, m, s, f[2 * V], f[e], f[V + e]);
            }
            for (int d = 1; d < sub; d <<= 1) {
                const float n2 = __shfl_xor(n, d), mean2 = __shfl_xor(m, d), m22 = __shfl_xor(s, d);
                if (n == 0.0f) n = n2, m = mean2, s = m22;
                else join_moments(n, m, s, n2, mean2, m22);
            }
            __syncthreads();
            if (i < items && h == 0) {
                fold[k][e] = m;
                fold[k][V + e] = s;
            }
        }
    }
    __syncthreads();
    {
        const int sub = lanes_each(THREADS, a.groups), h = threadIdx.x % sub;
        for (int g0 = 0; g0 < a.groups; g0 += THREADS / sub) {
            const int g = min(g0 + (int)threadIdx.x / sub, a.groups - 1);
            float n = 0.0f, m = 0.0f, s = 0.0f;
            for (int i = h; i < size; i += sub) {
                const int c = g * size + i, k = c / V, e = c - min(k * V, max(a.channels - V, 0));
                if (n == 0.0f) n = (float)positions, m = fold[k][e], s = fold[k][V + e];
                else join_moments(n, m, s, (float)positions, fold[k][e], fold[k][V + e]);
            }
            for (int d = 1; d < sub; d <<= 1) {
                const float n2 = __shfl_xor(n, d), mean2 = __shfl_xor(m, d), m22 = __shfl_xor(s, d);
                if (n == 0.0f) n = n2, m = mean2, s = m22;
                else join_moments(n, m, s, n2, mean2, m22);
            }
            if (h == 0 && g0 + (int)threadIdx.x / sub < a.groups) {
                const float rstd = 1.0f / sqrtf(s / ((float)size * (float)positions) + 1e-5f), to = a.rms ? 0.0f : m;
                group_stats[g][0] = to;
                group_stats[g][1] = rstd;
                a.stats[(sample * a.groups + g) * 2] = to;
                a.stats[(sample * a.groups + g) * 2 + 1] = rstd;
            }
        }
    }
    __syncthreads();
    float rstd[V];
    p.pairs(mean, rstd, &group_stats[0][0], size);
    T* const y = (T*)a.y + sample * a.positions * a.channels;
#pragma unroll
    for (int k = 0; k < kHeldPieces; ++k) {
        if (k >= many) continue;
        float v[V];
        unpack(u[k], v);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float xhat;
            v[e] = norm_z(v[e], mean[e], rstd[e], gain[e], shift[e], xhat);
        }
        norm_act_all<T>(a.act, v);
        p.store(y + (int64_t)(p.lane + k * p.lanes) * a.channels, v);
    }
}

// sums: [sample][2][channels]
template <typename T, int THREADS> __global__ __launch_bounds__(THREADS) void group_held_bwd_kernel(GroupNormBackward a, float* sums) {
    constexpr int V = kPiece<T>;
    __shared__ float fold[THREADS][2 * V];
    __shared__ float group_means[kHeldGroups][2];
    const MapPlace<T> p(a.channels, 0, THREADS, THREADS);
    const int64_t sample = blockIdx.x;
    const int positions = (int)a.positions, size = a.channels / a.groups;
    const T* const x = (const T*)a.x + sample * a.positions * a.channels;
    const T* const dy = (const T*)a.dy + sample * a.positions * a.channels;
    const float* const stats = a.stats + sample * a.groups * 2;
    uint4 ux[kHeldPairs], ug[kHeldPairs];
    const int many = p.any && p.lane < positions ? (positions - p.lane + p.lanes - 1) / p.lanes : 0;
#pragma unroll
    for (int k = 0; k < kHeldPairs; ++k)
        if (k * p.lanes < positions) {
            const int64_t row = (int64_t)min(p.lane + k * p.lanes, positions - 1) * a.channels;
            ux[k] = p.request(x + row);
            ug[k] = p.request(dy + row);
        }
    float mean[V], rstd[V], gain[V], shift[V], with_xhat[V], alone[V];
    p.pairs(mean, rstd, stats, size);
    p.params(gain, a.gain);
    p.params(shift, a.shift);
#pragma unroll
    for (int e = 0; e < V; ++e) with_xhat[e] = alone[e] = 0.0f;
    // xhat and dz of piece k
    const auto parts = [&](int k, float (&v)[V], float (&g)[V]) {
        unpack(ux[k], v);
        unpack(ug[k], g);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float xhat;
            const float z = norm_z(v[e], mean[e], rstd[e], gain[e], shift[e], xhat);
            g[e] = norm_act_grad<T>(a.act, z, g[e]);
            v[e] = xhat;
        }
    };
#pragma unroll
    for (int k = 0; k < kHeldPairs; ++k) {
        if (k >= many) continue;
        float v[V], g[V];
        parts(k, v, g);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            with_xhat[e] = fmaf(g[e], v[e], with_xhat[e]);
            alone[e] += g[e];
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
        fold[threadIdx.x][e] = with_xhat[e];
        fold[threadIdx.x][V + e] = alone[e];
    }
    __syncthreads();
    float* const mine = sums + sample * 2 * a.channels;
    {
        const int items = 2 * p.width * V, sub = lanes_each(THREADS, items), h = threadIdx.x % sub;
        for (int i0 = 0; i0 < items; i0 += THREADS / sub) {
            const int i = i0 + (int)threadIdx.x / sub, at = min(i, items - 1), which = at / (p.width * V), k = at / V % p.width, e = at % V;
            float s = 0.0f;
            for (int l = h; l < p.lanes; l += sub) s += fold[l * p.width + k][which * V + e];
            for (int d = 1; d < sub; d <<= 1) s += __shfl_xor(s, d);
            __syncthreads();
            if (i < items && h == 0) {
                fold[k][which * V + e] = s;
                const int ch = min(k * V, max(a.channels - V, 0)) + e;
                if (ch >= k * V && ch < a.channels) mine[which * (int64_t)a.channels + ch] = s;
            }
        }
    }
    __syncthreads();
    {
        const int sub = lanes_each(THREADS, a.groups), h = threadIdx.x % sub;
        const float n = (float)size * (float)positions;
        for (int g0 = 0; g0 < a.groups; g0 += THREADS / sub) {
            const int g = min(g0 + (int)threadIdx.x / sub, a.groups - 1);
            float with = 0.0f, without = 0.0f;
            for (int i = h; i < size; i += sub) {
                const int c = g * size + i, k = c / V, e = c - min(k * V, max(a.channels - V, 0));
                with = fmaf(a.gain[c], fold[k][e], with);
                without = fmaf(a.gain[c], fold[k][V + e], without);
            }
            for (int d = 1; d < sub; d <<= 1) {
                with += __shfl_xor(with, d);
                without += __shfl_xor(without, d);
            }
            if (h == 0) {
                group_means[g][0] = a.rms ? 0.0f : without / n;
                group_means[g][1] = with / n;
            }
        }
    }
    __syncthreads();
    p.pairs(alone, with_xhat, &group_means[0][0], size);
    T* const dx = (T*)a.dx + sample * a.positions * a.channels;
#pragma unroll
    for (int k = 0; k < kHeldPairs; ++k) {
        if (k >= many) continue;
        float v[V], g[V];
        parts(k, v, g);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = (fmaf(-v[e], with_xhat[e], g[e] * gain[e]) - alone[e]) * rstd[e];
        p.store(dx + (int64_t)(p.lane + k * p.lanes) * a.channels, v);
    }
}

// ------------------------------------------------------------------------------------------------ launches
// Slices of a sample's positions: as many as give the chip 2048 workgroups, of at least 32 positions, or four, and no fewer than eight, of a thread's where there are few side by side (1521 positions of 528 channels: 34 us in 48 slices of 32, 17 in 191 of 8).
constexpr int kMapGroups = 2048, kMapPositions = 32;
constexpr int kStatGroups = 1024;   // groups of all samples from which a wave to each is enough (60 groups of 4080 slices' channels each: 24 us a wave to each, 4.6 with several)
constexpr int kFoldColumns = 64;   // channels whose slices' sums a workgroup adds up, in whole groups
static int fold_columns(int size) { return (kFoldColumns + size - 1) / size * size; }
struct MapPlan {
    int64_t slice;
    int slices, blocks;   // blocks: of 256 pieces of channels
};
static int64_t map_slices(int64_t positions, int channels, int V) {
    const int lanes = 256 / std::min((channels + V - 1) / V, 256), least = std::max(8, std::min(kMapPositions, 4 * lanes));
    return (positions + least - 1) / least;
}
static MapPlan map_plan(int64_t samples, int64_t positions, int channels, int V) {
    MapPlan m;
    m.blocks = ((channels + V - 1) / V + 255) / 256;
    int64_t want = (kMapGroups + samples * m.blocks - 1) / (samples * m.blocks);
    want = std::max<int64_t>(1, std::min(want, map_slices(positions, channels, V)));
    m.slice = (positions + want - 1) / want;
    m.slices = (int)((positions + m.slice - 1) / m.slice);
    return m;
}

// Teams of a launch of rows: a whole number of samples' groups.
static int64_t row_teams(int64_t samples, int groups, int team, int rows_each, int threads) {
    const int64_t rows = samples * groups, most = threads / team;
    int64_t n = (samples + rows_each - 1) / rows_each;
    if (n * groups > most) n = most / groups;
    if (n < 1) n = 1;
    return n * groups < rows ? n * groups : rows;
}
constexpr int kRowsEachBack = 8;

constexpr int kRowFeatures = 16384;   // of a group in the form by rows
static bool by_rows(int64_t positions, int channels, int groups) { return positions == 1 && channels / groups <= kRowFeatures; }

// Threads that hold a sample's map, `pieces` of a thread's (0: more than a workgroup has).
static int held_threads(int64_t positions, int channels, int groups, int V, int pieces) {
    const int width = (channels + V - 1) / V;
    if (groups > kHeldGroups) return 0;
    for (int threads : {256, 1024})
        if (width <= threads && positions <= (int64_t)(threads / width) * pieces) return threads;
    return 0;
}

// Whether every launch of a forward and a backward pass can be had.
bool group_norm_fits(int dtype, int64_t samples, int64_t positions, int channels, int groups) {
    if (samples > INT32_MAX) return false;
    // (below, products of samples with groups or slices are under 2^58)
    if (samples == 0 || by_rows(positions, channels, groups)) return true;   // (teams are counted by the chip)
    const int V = dtype == kBF16 ? 8 : 4, size = channels / groups, columns = fold_columns(size);
    const MapPlan m = map_plan(samples, positions, channels, V);
    return launchable(samples * m.slices, 256) && launchable((samples * groups + 3) / 4, 256) && launchable(samples * ((channels + columns - 1) / columns), 512) &&
           launchable(samples, std::max(256, std::max(held_threads(positions, channels, groups, V, kHeldPieces), held_threads(positions, channels, groups, V, kHeldPairs))));
}

// (as much as any call of no more samples and positions takes)
size_t group_norm_workspace_bytes(int dtype, int64_t samples, int64_t positions, int channels, int groups, bool backward) {
    if (by_rows(positions, channels, groups)) return backward ? (size_t)row_teams(samples, groups, 4, kRowsEachBack, kBackRowThreads) / groups * 2 * channels * sizeof(float) : 0;
    const int V = dtype == kBF16 ? 8 : 4;
    const int64_t blocks = map_plan(samples, positions, channels, V).blocks, most = std::min(samples * map_slices(positions, channels, V), samples + kMapGroups / blocks + 1);
    return ((size_t)most * 2 * channels + (backward ? (size_t)samples * 2 * (groups + channels) : 0)) * sizeof(float);
}

template <typename T, int TEAM, int N, bool WHOLE> static hipError_t rows_fwd(const GroupNorm& a, hipStream_t s) {
    const int64_t teams = row_teams(a.samples, a.groups, TEAM, 1, kGroupRowThreads);
    const dim3 grid((unsigned)((teams + Team<TEAM>::kRows - 1) / Team<TEAM>::kRows));
    return launch_timed(kcLayerNorm, group_rows_fwd_kernel<T, TEAM, N, WHOLE>, grid, dim3(Team<TEAM>::kThreads), 0, s, a, teams);
}
template <typename T, int TEAM, int N, bool WHOLE> static hipError_t rows_bwd(const GroupNormBackward& a, float* part, hipStream_t s) {
    const int64_t teams = row_teams(a.samples, a.groups, TEAM, kRowsEachBack, kBackRowThreads);
    const dim3 grid((unsigned)((teams + Team<TEAM>::kRows - 1) / Team<TEAM>::kRows));
    const hipError_t e = launch_timed(kcLayerNorm, group_rows_bwd_kernel<T, TEAM, N, WHOLE>, grid, dim3(Team<TEAM>::kThreads), 0, s, a, teams, part);
    if (e != hipSuccess) return e;
    return reduce_all(Reductions(1, Reduction{part, a.dparams, 2 * (int64_t)a.channels, (int)(teams / a.groups), true}), s);
}

// (a team's threads have eight features each: of rows of 64 a team of 16 would leave half without any, 14.3 us for 8192 rows of 24 groups in bf16, a team of 8 10.4)
#define TMPS_GROUP_ROWS(fn, WHOLE, D, ...)                               \
    if (D <= 32) return fn<T, 4, kOne<T>, WHOLE>(__VA_ARGS__);           \
    if (D <= 64) return fn<T, 8, kOne<T>, WHOLE>(__VA_ARGS__);           \
    if (D <= 128) return fn<T, 16, kOne<T>, WHOLE>(__VA_ARGS__);         \
    if (D <= 256) return fn<T, 32, kOne<T>, WHOLE>(__VA_ARGS__);         \
    if (D <= 512) return fn<T, 64, kOne<T>, WHOLE>(__VA_ARGS__);         \
    if (D <= 2048) return fn<T, 256, kOne<T>, WHOLE>(__VA_ARGS__);       \
    if (D <= 8192) return fn<T, 1024, kOne<T>, WHOLE>(__VA_ARGS__);      \
    return fn<T, 1024, 2 * kOne<T>, WHOLE>(__VA_ARGS__)

template <typename T> static hipError_t rows_fwd_type(const GroupNorm& a, hipStream_t s) {
    const int D = a.channels / a.groups;
    if (join_whole<T>(D, {a.x, a.gain, a.shift, a.y})) { TMPS_GROUP_ROWS(rows_fwd, true, D, a, s); }
    TMPS_GROUP_ROWS(rows_fwd, false, D, a, s);
}
template <typename T> static hipError_t rows_bwd_type(const GroupNormBackward& a, float* part, hipStream_t s) {
    const int D = a.channels / a.groups;
    if (join_whole<T>(D, {a.dy, a.x, a.gain, a.shift, a.dx})) { TMPS_GROUP_ROWS(rows_bwd, true, D, a, part, s); }
    TMPS_GROUP_ROWS(rows_bwd, false, D, a, part, s);
}

template <typename T> static hipError_t forward_type(const GroupNorm& a, float* ws, hipStream_t s) {
    if (by_rows(a.positions, a.channels, a.groups)) return rows_fwd_type<T>(a, s);
    if (const int threads = held_threads(a.positions, a.channels, a.groups, kPiece<T>, kHeldPieces))
        return threads == 256 ? launch_timed(kcLayerNorm, group_held_fwd_kernel<T, 256>, dim3((unsigned)a.samples), dim3(256), 0, s, a)
                              : launch_timed(kcLayerNorm, group_held_fwd_kernel<T, 1024>, dim3((unsigned)a.samples), dim3(1024), 0, s, a);
    const MapPlan m = map_plan(a.samples, a.positions, a.channels, kPiece<T>);
    const dim3 grid((unsigned)(a.samples * m.slices), (unsigned)m.blocks);
    hipError_t e = launch_timed(kcLayerNorm, group_map_moments_kernel<T>, grid, dim3(256), 0, s, (const T*)a.x, a.positions, a.channels, m.slice, m.slices, a.rms, ws);
    if (e != hipSuccess) return e;
    const int64_t stats = a.samples * a.groups;
    e = stats >= kStatGroups ? launch_timed(kcLayerNorm, group_map_stats_kernel<1>, dim3((unsigned)((stats + 3) / 4)), dim3(256), 0, s, (const float*)ws, a.samples, a.positions,
                                            a.channels, a.groups, m.slice, m.slices, a.rms, a.stats)
                             : launch_timed(kcLayerNorm, group_map_stats_kernel<16>, dim3((unsigned)stats), dim3(1024), 0, s, (const float*)ws, a.samples, a.positions, a.channels,
                                            a.groups, m.slice, m.slices, a.rms, a.stats);
    if (e != hipSuccess) return e;
    return launch_timed(kcLayerNorm, group_map_apply_kernel<T>, grid, dim3(256), 0, s, a, m.slice, m.slices);
}

template <typename T> static hipError_t backward_type(const GroupNormBackward& a, float* ws, hipStream_t s) {
    if (by_rows(a.positions, a.channels, a.groups)) return rows_bwd_type<T>(a, ws, s);
    if (const int threads = held_threads(a.positions, a.channels, a.groups, kPiece<T>, kHeldPairs)) {
        const hipError_t e = threads == 256 ? launch_timed(kcLayerNorm, group_held_bwd_kernel<T, 256>, dim3((unsigned)a.samples), dim3(256), 0, s, a, ws)
                                            : launch_timed(kcLayerNorm, group_held_bwd_kernel<T, 1024>, dim3((unsigned)a.samples), dim3(1024), 0, s, a, ws);
        if (e != hipSuccess) return e;
        return reduce_all(Reductions(1, Reduction{ws, a.dparams, 2 * (int64_t)a.channels, (int)a.samples, true}), s);
    }
    const MapPlan m = map_plan(a.samples, a.positions, a.channels, kPiece<T>);
    float* const means = ws + a.samples * m.slices * 2 * (int64_t)a.channels;
    float* const sums = means + a.samples * a.groups * 2;
    const dim3 grid((unsigned)(a.samples * m.slices), (unsigned)m.blocks);
    hipError_t e = launch_timed(kcLayerNorm, group_map_sums_kernel<T>, grid, dim3(256), 0, s, a, m.slice, m.slices, ws);
    if (e != hipSuccess) return e;
    const int columns = fold_columns(a.channels / a.groups);
    const int64_t folds = a.samples * ((a.channels + columns - 1) / columns);
    e = launch_timed(kcLayerNorm, group_map_fold_kernel, dim3((unsigned)folds), dim3(512), 0, s, (const float*)ws, a.gain, a.positions, a.channels, a.groups, columns, m.slices, a.rms, sums,
                     means);
    if (e != hipSuccess) return e;
    e = launch_timed(kcLayerNorm, group_map_apply_bwd_kernel<T>, grid, dim3(256), 0, s, a, m.slice, m.slices, (const float*)means);
    if (e != hipSuccess) return e;
    return reduce_all(Reductions(1, Reduction{sums, a.dparams, 2 * (int64_t)a.channels, (int)a.samples, true}), s);
}

hipError_t group_norm_forward(int dtype, const GroupNorm& a, void* ws, hipStream_t s) {
    return dtype == kBF16 ? forward_type<bf16_t>(a, (float*)ws, s) : forward_type<float>(a, (float*)ws, s);
}
hipError_t group_norm_backward(int dtype, const GroupNormBackward& a, void* ws, hipStream_t s) {
    return dtype == kBF16 ? backward_type<bf16_t>(a, (float*)ws, s) : backward_type<float>(a, (float*)ws, s);
}

}  // namespace tmps
