// 16 bytes of neighbouring features at any address, and as floats.
#pragma once
#include "gemm.hip.h"

namespace tmps {

// A piece: V neighbouring features, 16 bytes.
template <typename T> constexpr int kPiece = 16 / sizeof(T);

typedef uint32_t any_u32x4_t __attribute__((ext_vector_type(4), aligned(2)));

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

}  // namespace tmps
