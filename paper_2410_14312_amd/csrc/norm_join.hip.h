// What the forward and the backward kernel of norm joins share: a row held in the registers of a team of threads, V neighbouring features N times a thread.
#pragma once
#include <initializer_list>

#include "gemm.hip.h"
#include "kernels.h"
#include "wave.hip.h"

// Products and sums are fused where fmaf says so and nowhere else: a row's results are then the same bit for bit whatever else its launch forms.
#pragma clang fp contract(off)

namespace tmps {

// A team is a wave, of which a workgroup has four, or a whole workgroup.
template <int TEAM> struct Team {
    static constexpr int kThreads = TEAM < 256 ? 256 : TEAM;
    static constexpr int kRows = kThreads / TEAM;   // teams of a workgroup
    static constexpr int kWaves = TEAM / 64;
    // Sums of K values over the team, the same in every thread.  red: K kWaves floats in LDS for each of two alternating places, so that one barrier a sum is enough: who
    // writes a place again has passed the barrier of the sum between, which nobody reaches before reading this one.
    template <int K> static __device__ __forceinline__ void sums(float (&v)[K], float (*red)[4 * 16], int& place) {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = wsum(v[k]);
        if constexpr (kWaves > 1) {
            const int wave = threadIdx.x >> 6;
            if ((threadIdx.x & 63) == 0) {
#pragma unroll
                for (int k = 0; k < K; ++k) red[place][k * kWaves + wave] = v[k];
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float t = red[place][k * kWaves];
#pragma unroll
                for (int w = 1; w < kWaves; ++w) t += red[place][k * kWaves + w];
                v[k] = t;
            }
            place ^= 1;
        }
    }
};

// Features of piece i of a thread begin at column(i); all of them are inside the row, or none.
template <int TEAM, int V> __device__ __forceinline__ int join_column(int i) { return ((int)(threadIdx.x % TEAM) + TEAM * i) * V; }

// A piece as it lies in memory: requested for the next row while this one is worked on, converted when its turn comes.
template <typename T, int V> struct RawPiece;
template <typename T> struct RawPiece<T, 8> : Raw8<T> {};
template <typename T> struct RawPiece<T, 1> {
    T v;
    __device__ __forceinline__ void load(const T* p) { v = p[0]; }
    __device__ __forceinline__ void get(float (&f)[1]) const { f[0] = to_f32(v); }
};
template <typename T, int TEAM, int V, int N> __device__ __forceinline__ void request_row(RawPiece<T, V> (&r)[N], const void* row, int D) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = join_column<TEAM, V>(i);
        if (c < D) r[i].load((const T*)row + c);
    }
}
template <int V, typename T> __device__ __forceinline__ void load_piece(const T* p, float (&v)[V]) {
    if constexpr (V == 8) load8(p, v);
    else v[0] = to_f32(p[0]);
}
template <int V, typename T> __device__ __forceinline__ void store_piece(T* p, const float (&v)[V]) {
    if constexpr (V == 8) store8(p, v);
    else p[0] = from_f32<T>(v[0]);
}

// A parameter's values of a thread's features (0 behind the row's end).
template <int TEAM, int V, int N> __device__ __forceinline__ void load_vector(float (&v)[N][V], const float* p, int D) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = join_column<TEAM, V>(i);
#pragma unroll
        for (int e = 0; e < V; ++e) v[i][e] = 0.0f;
        if (c < D) load_piece<V>(p + c, v[i]);
    }
}

// A gate and one minus it, each to its own last places (the difference of large a would lose them).  The hardware's exponential is off by |a| 2^-24: enough for results
// of 8 bits, not for fp32.
template <typename T> __device__ __forceinline__ void gate_of(float a, float& g, float& rest) {
    const float e = sizeof(T) == 2 ? __expf(-a) : expf(-a);
    g = 1.0f / (1.0f + e);
    rest = a < 0.0f ? 1.0f - g : e * g;
}

// Whether rows can be taken in pieces of 8 features: all of them on 16 bytes.
inline bool join_wide(int D, std::initializer_list<const void*> all) {
    uintptr_t bits = 0;
    for (const void* p : all) bits |= reinterpret_cast<uintptr_t>(p);
    return D % 8 == 0 && (bits & 15) == 0;
}

}  // namespace tmps
