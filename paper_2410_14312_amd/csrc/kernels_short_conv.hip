// A causal convolution of few taps along the positions, channels apart, with SiLU behind it, and its gradients.  Bound by memory: every number is read and written once.
#include "launch.h"
#include "mixer.h"
#include "pieces.hip.h"

#pragma clang fp contract(off)

namespace tmps {

// A thread has a piece of 16 bytes of neighbouring channels and a run of positions of a sample, whose inputs slide through its registers; a workgroup has 64 pieces of four runs that
// follow each other (the next sample's behind the last of one).  Rows whose channels are no whole pieces end in one that begins earlier: its first channels are also those of the piece before, and come out the same there.
constexpr int kConvRuns = 4;
constexpr int kConvRun = 16;       // forward: positions of a run
constexpr int kConvRunBack = 16;   // backward

template <typename T> struct ConvPiece {
    static constexpr int V = kPiece<T>;
    int C, at;   // channels, the first of this piece
    bool any;
    __device__ __forceinline__ ConvPiece(int piece, int channels) : C(channels), at(min(piece * V, max(channels - V, 0))), any(piece * V < channels) {}
    __device__ __forceinline__ void load(float (&v)[V], const T* row) const {
        if (C >= V) {
            unpack(load16_any(row + at), v);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = e < C ? to_f32(row[e]) : 0.0f;
        }
    }
    // (first: the first channel to store)
    __device__ __forceinline__ void store(T* row, const float (&v)[V], int first = 0) const {
        if (C >= V && first <= at) {
            store16_any(row + at, pack(v));
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (at + e < C && at + e >= first) row[at + e] = from_f32<T>(v[e]);
        }
    }
};

// What a thread has: a piece, a sample and a run's first position.
struct ConvPlace {
    int64_t group, sample, t0;   // the workgroup's four runs; its own
    int first, piece;            // the workgroup's first piece; its own
    __device__ __forceinline__ ConvPlace(int64_t positions, int run, int channels, int V) {
        const uint32_t blocks = (uint32_t)((channels + V * 64 - 1) / (V * 64)), runs = (uint32_t)((positions + run - 1) / run);
        group = blockIdx.x / blocks;
        first = (int)(blockIdx.x % blocks) * 64;
        piece = first + (int)(threadIdx.x & 63);
        const int64_t unit = group * kConvRuns + (threadIdx.x >> 6);
        sample = unit / runs;
        t0 = (unit - sample * runs) * run;
    }
};

template <typename T> __device__ __forceinline__ float conv_sigmoid(float z) {
    if constexpr (sizeof(T) == 2) return __builtin_amdgcn_rcpf(1.0f + __expf(-z));
    return 1.0f / (1.0f + expf(-z));
}

template <typename T, int K> struct ConvTaps {
    static constexpr int V = kPiece<T>;
    float w[K][V], bias[V];
    __device__ __forceinline__ ConvTaps(const ConvPiece<T>& p, const float* weight, const float* b) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int c = min(p.at + e, p.C - 1);
#pragma unroll
            for (int j = 0; j < K; ++j) w[j][e] = weight[(int64_t)c * K + j];
            bias[e] = b ? b[c] : 0.0f;
        }
    }
};

template <typename T, int K> __global__ __launch_bounds__(256) void short_conv_fwd_kernel(ShortConv a) {
    constexpr int V = kPiece<T>;
    const ConvPlace at(a.positions, kConvRun, a.channels, V);
    const ConvPiece<T> p(at.piece, a.channels);
    const int64_t sample = at.sample, t0 = at.t0;
    if (!p.any || sample >= a.samples) return;
    const ConvTaps<T, K> taps(p, a.weight, a.bias);
    const T* const x = (const T*)a.x + sample * a.positions * a.x_stride;
    T* const y = (T*)a.y + sample * a.positions * a.y_stride;
    const T* const tail = a.tail ? (const T*)a.tail + sample * (K - 1) * a.channels : nullptr;
    float u[K][V];   // the inputs of the positions t - K + 1 .. t
#pragma unroll
    for (int j = 0; j < K - 1; ++j) {
        const int64_t t = t0 - (K - 1) + j;
        if (t >= 0) {
            p.load(u[j + 1], x + t * a.x_stride);
        } else if (tail) {
            p.load(u[j + 1], tail + (K - 1 + t) * a.channels);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) u[j + 1][e] = 0.0f;
        }
    }
    const int64_t t1 = min(t0 + kConvRun, a.positions);
#pragma unroll 4
    for (int64_t t = t0; t < t1; ++t) {
#pragma unroll
        for (int j = 0; j < K - 1; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) u[j][e] = u[j + 1][e];
        p.load(u[K - 1], x + t * a.x_stride);
        float z[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            z[e] = taps.bias[e];
#pragma unroll
            for (int j = 0; j < K; ++j) z[e] = fmaf(taps.w[j][e], u[j][e], z[e]);
            if (a.silu) z[e] *= conv_sigmoid<T>(z[e]);
        }
        p.store(y + t * a.y_stride, z);
    }
    if (a.tail_out && t1 == a.positions) {
        T* const out = (T*)a.tail_out + sample * (K - 1) * a.channels;
#pragma unroll
        for (int j = 1; j < K; ++j) p.store(out + (int64_t)(j - 1) * a.channels, u[j], at.piece * V);
    }
}

// dz of the positions of a run and of the K - 1 behind it slides along as well: du[t] = sum_j w[j] dz[t + K - 1 - j].
template <typename T, int K> __global__ __launch_bounds__(256) void short_conv_bwd_kernel(ShortConvBackward a, float* part) {
    constexpr int V = kPiece<T>;
    __shared__ float fold[kConvRuns][K + 1][64 * V];
    const ConvPlace at(a.positions, kConvRunBack, a.channels, V);
    const ConvPiece<T> p(at.piece, a.channels);
    const int64_t sample = at.sample, t0 = at.t0;
    const int run = threadIdx.x >> 6;
    float dw[K + 1][V];
#pragma unroll
    for (int j = 0; j <= K; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) dw[j][e] = 0.0f;
    if (p.any && sample < a.samples) {
        const ConvTaps<T, K> taps(p, a.weight, a.bias);
        const T* const x = (const T*)a.x + sample * a.positions * a.x_stride;
        const T* const dy = (const T*)a.dy + sample * a.positions * a.dy_stride;
        T* const dx = (T*)a.dx + sample * a.positions * a.dx_stride;
        const T* const tail = a.tail ? (const T*)a.tail + sample * (K - 1) * a.channels : nullptr;
        const T* const dtail = a.dtail ? (const T*)a.dtail + sample * (K - 1) * a.channels : nullptr;
        const int64_t t1 = min(t0 + kConvRunBack, a.positions);
        float u[K][V], dz[K][V];   // inputs of t - K + 1 .. t; dz of the same
#pragma unroll
        for (int j = 0; j < K - 1; ++j) {
            const int64_t t = t0 - (K - 1) + j;
#pragma unroll
            for (int e = 0; e < V; ++e) u[j + 1][e] = dz[j + 1][e] = 0.0f;
            if (t >= 0) p.load(u[j + 1], x + t * a.x_stride);
            else if (tail) p.load(u[j + 1], tail + (K - 1 + t) * a.channels);
        }
        // (the gradient of the input at t - K + 1 is complete with dz of t; the first run also has those of the tail)
        for (int64_t t = t0; t < t1 + K - 1; ++t) {
#pragma unroll
            for (int j = 0; j < K - 1; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) u[j][e] = u[j + 1][e], dz[j][e] = dz[j + 1][e];
            if (t < a.positions) {
                float g[V];
                p.load(u[K - 1], x + t * a.x_stride);
                p.load(g, dy + t * a.dy_stride);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    if (a.silu) {
                        float z = taps.bias[e];
#pragma unroll
                        for (int j = 0; j < K; ++j) z = fmaf(taps.w[j][e], u[j][e], z);
                        const float s = conv_sigmoid<T>(z);
                        g[e] *= s * fmaf(z, 1.0f - s, 1.0f);
                    }
                    dz[K - 1][e] = g[e];
                    if (t < t1) {
#pragma unroll
                        for (int j = 0; j < K; ++j) dw[j][e] = fmaf(g[e], u[j][e], dw[j][e]);
                        dw[K][e] += g[e];
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) dz[K - 1][e] = 0.0f;
            }
            const int64_t of = t - (K - 1);
            if (of >= t0 || (t0 == 0 && a.dtail_in)) {
                float du[V];
                const int64_t back = of - (a.positions - (K - 1));   // its place in tail_out
#pragma unroll
                for (int e = 0; e < V; ++e) du[e] = 0.0f;
                if (dtail && back >= 0) p.load(du, dtail + back * a.channels);
#pragma unroll
                for (int e = 0; e < V; ++e) {
#pragma unroll
                    for (int j = 0; j < K; ++j) du[e] = fmaf(taps.w[j][e], dz[K - 1 - j][e], du[e]);
                }
                if (of >= 0) p.store(dx + of * a.dx_stride, du);
                else p.store((T*)a.dtail_in + (sample * (K - 1) + (K - 1) + of) * a.channels, du);
            }
        }
    }
#pragma unroll
    for (int j = 0; j <= K; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) fold[run][j][(threadIdx.x & 63) * V + e] = dw[j][e];
    __syncthreads();
    // partial results of a workgroup's runs: [channels][K], then, with a bias, [channels]
    const int sums = K + (a.bias ? 1 : 0);
    float* const mine = part + at.group * a.channels * sums;
    for (int i = threadIdx.x; i < sums * 64 * V; i += 256) {
        const int j = i / (64 * V), k = i % (64 * V), piece = at.first + k / V;
        const ConvPiece<T> q(piece, a.channels);
        const int c = q.at + k % V;
        if (!q.any || c >= a.channels || c < piece * V) continue;
        float sum = fold[0][j][k];
#pragma unroll
        for (int r = 1; r < kConvRuns; ++r) sum += fold[r][j][k];
        mine[j < K ? (int64_t)c * K + j : (int64_t)a.channels * K + c] = sum;
    }
}

// Groups of four runs.
static int64_t conv_groups(int64_t samples, int64_t positions, int run) { return (samples * ((positions + run - 1) / run) + kConvRuns - 1) / kConvRuns; }

size_t short_conv_part_elems(int64_t samples, int64_t positions, int channels, int taps) {
    return (size_t)conv_groups(samples, positions, kConvRunBack) * channels * (taps + 1);
}

// Workgroups of a launch (0: more than a launch takes).
template <typename T> static unsigned conv_grid(int64_t samples, int64_t positions, int channels, int run) {
    const int64_t blocks = conv_groups(samples, positions, run), pieces = ((channels + kPiece<T> - 1) / kPiece<T> + 63) / 64;
    return blocks <= INT32_MAX / pieces ? (unsigned)(blocks * pieces) : 0u;
}

template <typename T, int K> static hipError_t conv_fwd(const ShortConv& a, hipStream_t s) {
    const unsigned grid = conv_grid<T>(a.samples, a.positions, a.channels, kConvRun);
    return grid ? launch_timed(kcConvFwd, short_conv_fwd_kernel<T, K>, dim3(grid), dim3(256), 0, s, a) : hipErrorInvalidValue;
}
template <typename T, int K> static hipError_t conv_bwd(const ShortConvBackward& a, float* part, hipStream_t s) {
    const unsigned grid = conv_grid<T>(a.samples, a.positions, a.channels, kConvRunBack);
    return grid ? launch_timed(kcConvDgrad, short_conv_bwd_kernel<T, K>, dim3(grid), dim3(256), 0, s, a, part) : hipErrorInvalidValue;
}

#define TMPS_TAPS(fn, taps, ...)                      \
    switch (taps) {                                   \
        case 1: return fn<T, 1>(__VA_ARGS__);         \
        case 2: return fn<T, 2>(__VA_ARGS__);         \
        case 3: return fn<T, 3>(__VA_ARGS__);         \
        case 4: return fn<T, 4>(__VA_ARGS__);         \
        case 5: return fn<T, 5>(__VA_ARGS__);         \
        case 6: return fn<T, 6>(__VA_ARGS__);         \
        case 7: return fn<T, 7>(__VA_ARGS__);         \
        case 8: return fn<T, 8>(__VA_ARGS__);         \
    }                                                 \
    return hipErrorInvalidValue

template <typename T> static hipError_t conv_fwd_taps(const ShortConv& a, hipStream_t s) { TMPS_TAPS(conv_fwd, a.taps, a, s); }
template <typename T> static hipError_t conv_bwd_taps(const ShortConvBackward& a, float* part, hipStream_t s) { TMPS_TAPS(conv_bwd, a.taps, a, part, s); }

hipError_t short_conv_forward(int dtype, const ShortConv& a, hipStream_t s) {
    return dtype == kBF16 ? conv_fwd_taps<bf16_t>(a, s) : conv_fwd_taps<float>(a, s);
}

hipError_t short_conv_backward(int dtype, const ShortConvBackward& a, float* part, hipStream_t s) {
    const hipError_t e = dtype == kBF16 ? conv_bwd_taps<bf16_t>(a, part, s) : conv_bwd_taps<float>(a, part, s);
    if (e != hipSuccess) return e;
    const int64_t slabs = conv_groups(a.samples, a.positions, kConvRunBack);
    return reduce_all(Reductions(1, Reduction{part, a.dparams, (int64_t)a.channels * (a.taps + (a.bias ? 1 : 0)), (int)slabs, true}), s);
}

}  // namespace tmps
