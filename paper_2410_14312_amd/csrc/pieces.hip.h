// Rows in pieces of 16 bytes at any address: a thread's pieces of a row, and their features as floats.
#pragma once
#include "gemm.hip.h"

namespace tmps {

// A piece: V neighbouring features, 16 bytes.
template <typename T> constexpr int kPiece = 16 / sizeof(T);

typedef uint32_t any_u32x4_t __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t any_u32x2_t __attribute__((ext_vector_type(2), aligned(2)));

// (one instruction, of as many requests to memory as the address takes)
__device__ __forceinline__ uint4 load16_any(const void* p) {
    const any_u32x4_t v = *reinterpret_cast<const any_u32x4_t*>(p);
    return make_uint4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void store16_any(void* p, const uint4& u) { *reinterpret_cast<any_u32x4_t*>(p) = any_u32x4_t{u.x, u.y, u.z, u.w}; }

__device__ __forceinline__ void unpack(const uint4& u, float (&v)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[2 * e] = __builtin_bit_cast(float, w[e] << 16);
        v[2 * e + 1] = __builtin_bit_cast(float, w[e] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack(const uint4& u, float (&v)[4]) {
    const float4 f = __builtin_bit_cast(float4, u);
    v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
}
// (rounded to bf16 in pairs: one conversion makes two values in the halves of a register)
__device__ __forceinline__ uint4 pack(const float (&v)[8]) {
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{v[2 * e], v[2 * e + 1]}), bf16x2_t));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 pack(const float (&v)[4]) { return __builtin_bit_cast(uint4, make_float4(v[0], v[1], v[2], v[3])); }

// The pieces of a thread in every row.  WHOLE: all of the launch's pieces are on 16 bytes, and inside a row or behind it.  Otherwise they are 16 bytes at any address, which the
// memory unit takes in a request or two, and the piece that a row ends in begins as much earlier as it would reach beyond: its first features are also the piece's before it, which
// has them for its own.  (Loads of the last features one by one would have to be put together, and so waited for, where they are requested: 8000 x 1003 in bf16, backward, 52 us
// instead of 35.)  A row of fewer features than a piece is one that is put together all the same.
template <int TEAM, int N, int V, bool WHOLE> struct Pieces {
    int D;
    __device__ __forceinline__ int column(int i) const { return ((int)(threadIdx.x % TEAM) + TEAM * i) * V; }   // the first feature of its own
    __device__ __forceinline__ bool any(int i) const { return column(i) < D; }
    __device__ __forceinline__ int at(int i) const { return WHOLE ? column(i) : min(column(i), max(D - V, 0)); }   // the first feature it holds
    __device__ __forceinline__ bool own(int i, int e) const { return WHOLE || (at(i) + e >= column(i) && (D >= V || e < D)); }   // (of a piece that has any)
};

// 16 bytes of a row from feature c on, as they lie in memory: requested for the next row while this one is worked on, unpacked when their turn comes.
template <bool WHOLE, typename T> __device__ __forceinline__ void request16(uint4& u, const T* row, int c, int D) {
    if constexpr (WHOLE) {
        u = *reinterpret_cast<const uint4*>(row + c);
    } else if (c + kPiece<T> <= D) {
        u = load16_any(row + c);
    } else {
        struct Features { T v[kPiece<T>]; } f;
#pragma unroll
        for (int e = 0; e < kPiece<T>; ++e) f.v[e] = c + e < D ? row[c + e] : T(0.0f);
        u = __builtin_bit_cast(uint4, f);
    }
}
template <typename T, int TEAM, int N, int V, bool WHOLE> __device__ __forceinline__ void request_row(uint4 (&u)[N], const T* row, const Pieces<TEAM, N, V, WHOLE>& p) {
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (p.any(i)) request16<WHOLE>(u[i], row, p.at(i), p.D);
}
}  // namespace tmps
