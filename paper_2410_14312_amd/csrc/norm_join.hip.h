// What the forward and the backward kernel of norm joins share: a row held in the registers of a team of threads, 16 bytes of neighbouring features N times a thread.
#pragma once
#include <initializer_list>

#include "kernels.h"
#include "pieces.hip.h"
#include "wave.hip.h"

// Products and sums are fused where fmaf says so and nowhere else: a row's results are then the same bit for bit whatever else its launch forms.
#pragma clang fp contract(off)

namespace tmps {

// A team is 16, 32 or 64 lanes of a wave, in workgroups of four waves, or a whole workgroup.
template <int TEAM> struct Team {
    static constexpr int kThreads = TEAM <= 64 ? 256 : TEAM;
    static constexpr int kRows = kThreads / TEAM;   // teams of a workgroup
    static constexpr int kWaves = TEAM <= 64 ? 1 : TEAM / 64;
    static __device__ __forceinline__ float lanes_sum(float v) {
        if constexpr (TEAM >= 64) return wsum(v);
        if constexpr (TEAM == 32) {
            const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
            v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
        }
        v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x128, 0xF, 0xF, false));   // row_ror:8
        v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x124, 0xF, 0xF, false));   // row_ror:4
        v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x122, 0xF, 0xF, false));   // row_ror:2
        v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x121, 0xF, 0xF, false));   // row_ror:1
        return v;
    }
    // Sums of K values over the team, the same in every thread.  red: K kWaves floats in LDS for each of two alternating places, so that one barrier a sum is enough: who
    // writes a place again has passed the barrier of the sum between, which nobody reaches before reading this one.
    template <int K> static __device__ __forceinline__ void sums(float (&v)[K], float (*red)[2 * 16], int& place) {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = lanes_sum(v[k]);
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

template <typename T> constexpr int kOne = 8 / kPiece<T>;   // pieces of 8 features

// The features of piece i that are its own.
template <typename T, int TEAM, int N, int V, bool WHOLE> __device__ __forceinline__ void store_packed(T* row, const Pieces<TEAM, N, V, WHOLE>& p, int i, const uint4& u) {
    if (!p.any(i)) return;
    if constexpr (WHOLE) {
        *reinterpret_cast<uint4*>(row + p.at(i)) = u;
    } else if (p.column(i) + V <= p.D) {
        store16_any(row + p.at(i), u);
    } else {
        struct Features { T v[V]; } f = __builtin_bit_cast(Features, u);
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (p.own(i, e)) row[p.at(i) + e] = f.v[e];
    }
}
template <typename T, int TEAM, int N, int V, bool WHOLE> __device__ __forceinline__ void store_piece(T* row, const Pieces<TEAM, N, V, WHOLE>& p, int i, const float (&v)[V]) {
    store_packed(row, p, i, pack(v));
}

// A parameter's values of piece i (zeros where it has none).
template <int TEAM, int N, int V, bool WHOLE> __device__ __forceinline__ void load_vector(float (&v)[V], const float* from, const Pieces<TEAM, N, V, WHOLE>& p, int i) {
#pragma unroll
    for (int h = 0; h < V; h += 4) {
        uint4 u = make_uint4(0, 0, 0, 0);
        float f[4];
        if (from && p.any(i)) request16<WHOLE>(u, from, p.at(i) + h, p.D);
        unpack(u, f);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[h + e] = f[e];
    }
}

// A gate and one minus it, each to its own last places (the difference of large a would lose them).  The hardware's exponential is off by |a| 2^-24 and its reciprocal by a step:
// enough for results of 8 bits, not for fp32.
template <typename T> __device__ __forceinline__ void gate_of(float a, float& g, float& rest) {
    const float e = sizeof(T) == 2 ? __expf(-a) : expf(-a);
    g = sizeof(T) == 2 ? __builtin_amdgcn_rcpf(1.0f + e) : 1.0f / (1.0f + e);
    rest = a < 0.0f ? 1.0f - g : e * g;
}

// Whether all of a launch's pieces are on 16 bytes.
template <typename T> bool join_whole(int D, std::initializer_list<const void*> all) {
    uintptr_t bits = 0;
    for (const void* p : all) bits |= reinterpret_cast<uintptr_t>(p);
    return D % kPiece<T> == 0 && (bits & 15) == 0;
}

}  // namespace tmps
