// A causal convolution of few taps along the positions, channels apart, with SiLU behind it, and its gradients.  Bound by memory: every number is read and written once.  8192 rows of 1664
// channels in bf16, four taps: 17.5 us (3.1 TB/s; 10.8 at a copy's rate), back 28.0 with the sums of the partial results (16.2 at a copy's rate).
#include "launch.h"
#include "mixer.h"
#include "pieces.hip.h"

#pragma clang fp contract(off)

namespace tmps {

// A thread has a piece of V neighbouring channels and a run of positions of a sample, a few at a time, whose inputs are in its registers with the K - 1 before them; a workgroup has 64
// pieces of four runs that follow each other (the next sample's behind the last of one).  Rows whose channels are no whole pieces end in one that begins earlier: its first channels are
// also those of the piece before, and come out the same there.  NARROW: rows of fewer channels than a piece.
constexpr int kConvRuns = 4;
constexpr int kConvRun = 16;     // positions of a run
constexpr int kConvAhead = 2;    // positions at a time, as many more under way

// Forward 16 bytes; backward four channels, whose inputs, gradients and sums fit the registers of four waves of a SIMD.
template <typename T> constexpr int kConvForward = kPiece<T>;
constexpr int kConvBackward = 4;

template <typename T, int V, bool NARROW> struct ConvPiece {
    struct Values { T v[V]; };
    typedef std::conditional_t<V * sizeof(T) == 16, any_u32x4_t, any_u32x2_t> words_t;   // (at any address)
    int C, at;   // channels, the first of this piece
    uint32_t off;   // its place in a row
    bool any;
    __device__ __forceinline__ ConvPiece(int piece, int channels)
        : C(channels), at(NARROW ? 0 : min(piece * V, channels - V)), off((uint32_t)at * (uint32_t)sizeof(T)), any(piece * V < channels) {}
    __device__ __forceinline__ words_t request(const T* row) const {
        if constexpr (!NARROW) return *reinterpret_cast<const words_t*>(reinterpret_cast<const char*>(row) + off);
        Values f;
#pragma unroll
        for (int e = 0; e < V; ++e) f.v[e] = row[min(e, C - 1)];
        return __builtin_bit_cast(words_t, f);
    }
    static __device__ __forceinline__ void open(const words_t& u, float (&v)[V]) {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int e = 0; e < V / 2; ++e) {
                const uint32_t w = u[e];
                v[2 * e] = __builtin_bit_cast(float, w << 16);
                v[2 * e + 1] = __builtin_bit_cast(float, w & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const uint32_t w = u[e];   // (a vector's element has no address that its bits could be taken from)
                v[e] = __builtin_bit_cast(float, w);
            }
        }
    }
    __device__ __forceinline__ void load(float (&v)[V], const T* row) const { open(request(row), v); }
    __device__ __forceinline__ void store(T* row, const float (&v)[V]) const {
        Values f;
#pragma unroll
        for (int e = 0; e < V; ++e) f.v[e] = from_f32<T>(v[e]);
        if constexpr (!NARROW) {
            *reinterpret_cast<words_t*>(reinterpret_cast<char*>(row) + off) = __builtin_bit_cast(words_t, f);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (e < C) row[e] = f.v[e];
        }
    }
    // The channels from `first` on.
    __device__ __forceinline__ void store_from(T* row, const float (&v)[V], int first) const {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (at + e < C && at + e >= first) row[at + e] = from_f32<T>(v[e]);
    }
};

// What a thread has: a piece, a sample and a run's first position.
struct ConvPlace {
    int64_t group, sample, t0;   // the workgroup's four runs; its own
    int first, piece;            // the workgroup's first piece; its own
    __device__ __forceinline__ ConvPlace(int64_t positions, int channels, int V) {
        const uint32_t blocks = (uint32_t)((channels + V * 64 - 1) / (V * 64)), runs = (uint32_t)((positions + kConvRun - 1) / kConvRun);
        group = blockIdx.x / blocks;
        first = (int)(blockIdx.x % blocks) * 64;
        piece = first + (int)(threadIdx.x & 63);
        const int64_t unit = group * kConvRuns + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);   // (known to be the same for a wave: rows' addresses are scalars then)
        sample = unit / runs;
        t0 = (unit - sample * runs) * kConvRun;
    }
};

template <typename T> __device__ __forceinline__ float conv_sigmoid(float z) {
    if constexpr (sizeof(T) == 2) return __builtin_amdgcn_rcpf(1.0f + __expf(-z));
    return 1.0f / (1.0f + expf(-z));
}

template <int K, int V> struct ConvTaps {
    float w[K][V], bias[V];
    __device__ __forceinline__ ConvTaps(int at, int channels, const float* weight, const float* b) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int c = min(at + e, channels - 1);
#pragma unroll
            for (int j = 0; j < K; ++j) w[j][e] = weight[(int64_t)c * K + j];
            bias[e] = b ? b[c] : 0.0f;
        }
    }
};

// The K - 1 inputs before position t0, those before a sample's first from its tail.
template <typename T, int K, int V, bool NARROW, int N>
__device__ __forceinline__ void conv_before(float (&u)[N][V], const ConvPiece<T, V, NARROW>& p, const T* x, int64_t stride, const T* tail, int64_t t0) {
#pragma unroll
    for (int j = 0; j < K - 1; ++j) {
        const int64_t t = t0 - (K - 1) + j;
        if (t >= 0) {
            p.load(u[j], x + t * stride);
        } else if (tail) {
            p.load(u[j], tail + (K - 1 + t) * p.C);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) u[j][e] = 0.0f;
        }
    }
}

template <typename T, int K, bool NARROW> __global__ __launch_bounds__(256) void short_conv_fwd_kernel(ShortConv a) {
    constexpr int V = kConvForward<T>, A = kConvAhead;
    const ConvPlace at(a.positions, a.channels, V);
    const ConvPiece<T, V, NARROW> p(at.piece, a.channels);
    const int64_t sample = at.sample, t0 = at.t0;
    if (!p.any || sample >= a.samples) return;
    const T* const x = (const T*)a.x + sample * a.positions * a.x_stride;
    T* const y = (T*)a.y + sample * a.positions * a.y_stride;
    const T* const tail = a.tail ? (const T*)a.tail + sample * (K - 1) * a.channels : nullptr;
    const int64_t t1 = min(t0 + kConvRun, a.positions);
    typename ConvPiece<T, V, NARROW>::words_t next[A];
    const auto request = [&](int64_t from) {
#pragma unroll
        for (int k = 0; k < A; ++k) next[k] = p.request(x + min(from + k, t1 - 1) * a.x_stride);   // (behind the run its last one's again)
    };
    request(t0);
    const ConvTaps<K, V> taps(p.at, a.channels, a.weight, a.bias);
    // (where tail_out is the tail, what a piece that begins earlier has read of the piece before may be that one's outcome already)
    const bool own_only = p.at < at.piece * V && a.tail && a.tail_out == a.tail;
    float u[K - 1 + A][V];   // the inputs from position `from` - K + 1 on
    conv_before<T, K>(u, p, x, a.x_stride, tail, t0);
    for (int64_t from = t0; from < t1; from += A) {
#pragma unroll
        for (int k = 0; k < A; ++k) p.open(next[k], u[K - 1 + k]);
        if (from + A < t1) request(from + A);
        const int many = (int)min<int64_t>(A, t1 - from);
#pragma unroll
        for (int k = 0; k < A; ++k) {
            float z[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                z[e] = taps.bias[e];
#pragma unroll
                for (int j = 0; j < K; ++j) z[e] = fmaf(taps.w[j][e], u[k + j][e], z[e]);
            }
            if (a.silu) {
#pragma unroll
                for (int e = 0; e < V; ++e) z[e] *= conv_sigmoid<T>(z[e]);
            }
            if (k >= many) continue;
            if (own_only) p.store_from(y + (from + k) * a.y_stride, z, at.piece * V);
            else p.store(y + (from + k) * a.y_stride, z);
        }
        if (a.tail_out && from + A >= a.positions) {   // (the last positions': the inputs up to the last one)
            T* const out = (T*)a.tail_out + sample * (K - 1) * a.channels;
#pragma unroll
            for (int j = 0; j < K - 1; ++j)
#pragma unroll
                for (int k = 1; k <= A; ++k)
                    if (k == many) p.store_from(out + (int64_t)j * a.channels, u[k + j], at.piece * V);
        }
#pragma unroll
        for (int j = 0; j < K - 1; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) u[j][e] = u[A + j][e];
    }
}

// du[t] = sum_j w[j] dz[t + K - 1 - j]: dz of a run and of the K - 1 positions behind it, z being formed again.
template <typename T, int K, bool NARROW> __global__ __launch_bounds__(256) void short_conv_bwd_kernel(ShortConvBackward a, float* part) {
    constexpr int V = kConvBackward, A = kConvAhead;
    __shared__ float fold[kConvRuns][K + 1][64 * V];
    const ConvPlace at(a.positions, a.channels, V);
    const ConvPiece<T, V, NARROW> p(at.piece, a.channels);
    const int64_t sample = at.sample, t0 = at.t0;
    const int run = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    float dw[K + 1][V];
#pragma unroll
    for (int j = 0; j <= K; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) dw[j][e] = 0.0f;
    if (p.any && sample < a.samples) {
        const T* const x = (const T*)a.x + sample * a.positions * a.x_stride;
        const T* const dy = (const T*)a.dy + sample * a.positions * a.dy_stride;
        T* const dx = (T*)a.dx + sample * a.positions * a.dx_stride;
        const T* const tail = a.tail ? (const T*)a.tail + sample * (K - 1) * a.channels : nullptr;
        const T* const dtail = a.dtail ? (const T*)a.dtail + sample * (K - 1) * a.channels : nullptr;
        const int64_t t1 = min(t0 + kConvRun, a.positions), end = t1 + K - 1, last = min(end, a.positions) - 1;
        typename ConvPiece<T, V, NARROW>::words_t nx[A], ny[A];
        const auto request = [&](int64_t from) {
#pragma unroll
            for (int k = 0; k < A; ++k) {
                const int64_t t = min(from + k, last);
                nx[k] = p.request(x + t * a.x_stride);
                ny[k] = p.request(dy + t * a.dy_stride);
            }
        };
        request(t0);
        const ConvTaps<K, V> taps(p.at, a.channels, a.weight, a.bias);
        float u[K - 1 + A][V], dz[K - 1 + A][V];   // from position `from` - K + 1 on
        conv_before<T, K>(u, p, x, a.x_stride, tail, t0);
#pragma unroll
        for (int j = 0; j < K - 1; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) dz[j][e] = 0.0f;
        for (int64_t from = t0; from < end; from += A) {
#pragma unroll
            for (int k = 0; k < A; ++k) {
                p.open(nx[k], u[K - 1 + k]);
                p.open(ny[k], dz[K - 1 + k]);
            }
            if (from + A < end) request(from + A);
            if (a.silu) {
#pragma unroll
                for (int k = 0; k < A; ++k)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        float z = taps.bias[e];
#pragma unroll
                        for (int j = 0; j < K; ++j) z = fmaf(taps.w[j][e], u[k + j][e], z);
                        const float s = conv_sigmoid<T>(z);
                        dz[K - 1 + k][e] *= s * fmaf(z, 1.0f - s, 1.0f);
                    }
            }
#pragma unroll
            for (int k = 0; k < A; ++k) {
                const bool here = from + k < a.positions, mine = from + k < t1;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float g = dz[K - 1 + k][e] = here ? dz[K - 1 + k][e] : 0.0f;
                    if (!mine) continue;   // (no product with 0: an input may be infinite)
#pragma unroll
                    for (int j = 0; j < K; ++j) dw[j][e] = fmaf(g, u[k + j][e], dw[j][e]);
                    dw[K][e] += g;
                }
            }
            // (the gradient of the input K - 1 positions back is complete with a position's dz; the first run also has those of the tail)
#pragma unroll
            for (int k = 0; k < A; ++k) {
                const int64_t of = from + k - (K - 1);
                if (of >= t1 || (of < t0 && !(t0 == 0 && a.dtail_in))) continue;
                float du[V];
                const int64_t back = of - (a.positions - (K - 1));   // its place in tail_out
#pragma unroll
                for (int e = 0; e < V; ++e) du[e] = 0.0f;
                if (dtail && back >= 0) p.load(du, dtail + back * a.channels);
#pragma unroll
                for (int e = 0; e < V; ++e)
#pragma unroll
                    for (int j = 0; j < K; ++j) du[e] = fmaf(taps.w[j][e], dz[k + K - 1 - j][e], du[e]);
                if (of >= 0) p.store(dx + of * a.dx_stride, du);
                else p.store((T*)a.dtail_in + (sample * (K - 1) + (K - 1) + of) * a.channels, du);
            }
#pragma unroll
            for (int j = 0; j < K - 1; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) u[j][e] = u[A + j][e], dz[j][e] = dz[A + j][e];
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
        const ConvPiece<T, V, NARROW> q(piece, a.channels);
        const int c = q.at + k % V;
        if (!q.any || c >= a.channels || c < piece * V) continue;
        float sum = fold[0][j][k];
#pragma unroll
        for (int r = 1; r < kConvRuns; ++r) sum += fold[r][j][k];
        mine[j < K ? (int64_t)c * K + j : (int64_t)a.channels * K + c] = sum;
    }
}

// Groups of four runs.
static int64_t conv_groups(int64_t samples, int64_t positions) { return (samples * ((positions + kConvRun - 1) / kConvRun) + kConvRuns - 1) / kConvRuns; }

size_t short_conv_part_elems(int64_t samples, int64_t positions, int channels, int taps) {
    return (size_t)conv_groups(samples, positions) * channels * (taps + 1);
}

// Workgroups of a launch (0: more than a launch takes).
static unsigned conv_grid(int64_t samples, int64_t positions, int channels, int V) {
    const int64_t blocks = conv_groups(samples, positions), pieces = ((channels + V - 1) / V + 63) / 64;
    return launchable(blocks * pieces, 256) ? (unsigned)(blocks * pieces) : 0u;
}

template <typename T, int K> static hipError_t conv_fwd(const ShortConv& a, hipStream_t s) {
    const unsigned grid = conv_grid(a.samples, a.positions, a.channels, kConvForward<T>);
    if (!grid) return hipErrorInvalidValue;
    return launch_timed(kcConvFwd, a.channels < kConvForward<T> ? short_conv_fwd_kernel<T, K, true> : short_conv_fwd_kernel<T, K, false>, dim3(grid), dim3(256), 0, s, a);
}
template <typename T, int K> static hipError_t conv_bwd(const ShortConvBackward& a, float* part, hipStream_t s) {
    const unsigned grid = conv_grid(a.samples, a.positions, a.channels, kConvBackward);
    if (!grid) return hipErrorInvalidValue;
    return launch_timed(kcConvDgrad, a.channels < kConvBackward ? short_conv_bwd_kernel<T, K, true> : short_conv_bwd_kernel<T, K, false>, dim3(grid), dim3(256), 0, s, a, part);
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
    const int64_t slabs = conv_groups(a.samples, a.positions);
    return reduce_all(Reductions(1, Reduction{part, a.dparams, (int64_t)a.channels * (a.taps + (a.bias ? 1 : 0)), (int)slabs, true}), s);
}

}  // namespace tmps
