// What the kernels of the selective state space share: tiles of 16 x 16 by the matrix unit, operands from LDS by rows and by columns, the decays of a chunk of positions.
#pragma once
#include "mixer.h"
#include "pieces.hip.h"

namespace tmps {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef int16_t s16x4v_t __attribute__((ext_vector_type(4)));

constexpr int kScanChunk = 64;   // positions that a workgroup takes at a time

// Eight of the 32 numbers of a row (first operand) or column (second) that a lane holds: row or column lane % 16, numbers 8 (lane / 16) .. + 7; or, `split`, 4 (lane / 16) .. + 3 and
// 16 + 4 (lane / 16) .. + 3, which is how the results of two tiles lie (a lane has rows 4 (lane / 16) .. + 3 of column lane % 16).
template <typename T> struct Oct;
template <> struct Oct<bf16_t> {
    bf16x8_t v;
    __device__ __forceinline__ void set(int e, float x) { v[e] = (bf16_t)x; }
    __device__ __forceinline__ float get(int e) const { return (float)v[e]; }
};
template <> struct Oct<float> {
    float v[8];
    __device__ __forceinline__ void set(int e, float x) { v[e] = x; }
    __device__ __forceinline__ float get(int e) const { return v[e]; }
};

__device__ __forceinline__ f32x4_t mma(const Oct<bf16_t>& a, const Oct<bf16_t>& b, f32x4_t acc) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, acc, 0, 0, 0); }
__device__ __forceinline__ f32x4_t mma(const Oct<float>& a, const Oct<float>& b, f32x4_t acc) {
#pragma unroll
    for (int e = 0; e < 8; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[e], b.v[e], acc, 0, 0, 0);
    return acc;
}

// A number as the sum of K numbers of the operands' type (fp32: itself).
template <int K> __device__ __forceinline__ void terms_of(float x, int e, Oct<bf16_t> (&out)[K]) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
        out[k].set(e, x);
        if (k + 1 < K) x -= out[k].get(e);
    }
}
template <int K> __device__ __forceinline__ void terms_of(float x, int e, Oct<float> (&out)[K]) { out[0].set(e, x); }

// Numbers of a row of a tile that lie one behind the other from k0 on.
template <bool SPLIT> __device__ __forceinline__ Oct<bf16_t> along(const bf16_t* row, int k0, int lane) {
    Oct<bf16_t> o;
    if constexpr (SPLIT) {
        union { uint2 h[2]; bf16x8_t v; } u;
        u.h[0] = *reinterpret_cast<const uint2*>(row + k0 + 4 * (lane >> 4));
        u.h[1] = *reinterpret_cast<const uint2*>(row + k0 + 16 + 4 * (lane >> 4));
        o.v = u.v;
    } else {
        o.v = *reinterpret_cast<const bf16x8_t*>(row + k0 + 8 * (lane >> 4));
    }
    return o;
}
template <bool SPLIT> __device__ __forceinline__ Oct<float> along(const float* row, int k0, int lane) {
    Oct<float> o;
    const int first = SPLIT ? 4 * (lane >> 4) : 8 * (lane >> 4), second = SPLIT ? first + 16 : first + 4;
    const float4 a = *reinterpret_cast<const float4*>(row + k0 + first), b = *reinterpret_cast<const float4*>(row + k0 + second);
    o.v[0] = a.x; o.v[1] = a.y; o.v[2] = a.z; o.v[3] = a.w;
    o.v[4] = b.x; o.v[5] = b.y; o.v[6] = b.z; o.v[7] = b.w;
    return o;
}
// Numbers of a column, c0 + lane % 16, in the rows from k0 on.  bf16: transposing reads of four rows by 16 columns to each 16 lanes.
template <bool SPLIT> __device__ __forceinline__ Oct<bf16_t> across(const bf16_t* tile, int pitch, int k0, int c0, int lane) {
    typedef __attribute__((address_space(3))) s16x4v_t* lds_t;
    const int first = SPLIT ? 4 * (lane >> 4) : 8 * (lane >> 4), second = SPLIT ? first + 16 : first + 4;
    const bf16_t* const p = tile + (k0 + ((lane & 15) >> 2)) * pitch + c0 + (lane & 3) * 4;
    union { s16x4v_t h[2]; bf16x8_t v; } u;
    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(p + first * pitch));
    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(p + second * pitch));
    Oct<bf16_t> o;
    o.v = u.v;
    return o;
}
template <bool SPLIT> __device__ __forceinline__ Oct<float> across(const float* tile, int pitch, int k0, int c0, int lane) {
    Oct<float> o;
    const int first = SPLIT ? 4 * (lane >> 4) : 8 * (lane >> 4), second = SPLIT ? first + 16 : first + 4;
    const float* const p = tile + k0 * pitch + c0 + (lane & 15);
#pragma unroll
    for (int e = 0; e < 8; ++e) o.v[e] = p[((e < 4 ? first : second - 4) + e) * pitch];
    return o;
}

// Four neighbouring numbers.
__device__ __forceinline__ void four(const bf16_t* p, float (&v)[4]) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    v[0] = __builtin_bit_cast(float, u.x << 16); v[1] = __builtin_bit_cast(float, u.x & 0xffff0000u);
    v[2] = __builtin_bit_cast(float, u.y << 16); v[3] = __builtin_bit_cast(float, u.y & 0xffff0000u);
}
__device__ __forceinline__ void four(const float* p, float (&v)[4]) {
    const float4 f = *reinterpret_cast<const float4*>(p);
    v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
}
__device__ __forceinline__ void four_anywhere(const bf16_t* p, float (&v)[4]) {   // (at any address)
    const any_u32x2_t u = *reinterpret_cast<const any_u32x2_t*>(p);
    const uint32_t a = u[0], b = u[1];
    v[0] = __builtin_bit_cast(float, a << 16); v[1] = __builtin_bit_cast(float, a & 0xffff0000u);
    v[2] = __builtin_bit_cast(float, b << 16); v[3] = __builtin_bit_cast(float, b & 0xffff0000u);
}
__device__ __forceinline__ void four_anywhere(const float* p, float (&v)[4]) { unpack(load16_any(p), v); }
__device__ __forceinline__ void put_four(bf16_t* p, const float (&v)[4]) {   // (on 8 bytes)
    union { bf16_t h[4]; uint2 u; } k;
#pragma unroll
    for (int e = 0; e < 4; ++e) k.h[e] = (bf16_t)v[e];
    *reinterpret_cast<uint2*>(p) = k.u;
}
__device__ __forceinline__ void put_four(float* p, const float (&v)[4]) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
// The same anywhere in memory, those of them before `many`.
__device__ __forceinline__ void put_four_any(bf16_t* p, const float (&v)[4], int many) {
    union { bf16_t h[4]; any_u32x2_t u; } k;
#pragma unroll
    for (int e = 0; e < 4; ++e) k.h[e] = (bf16_t)v[e];
    if (many >= 4) *reinterpret_cast<any_u32x2_t*>(p) = k.u;
    else
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < many) p[e] = k.h[e];
}
__device__ __forceinline__ void put_four_any(float* p, const float (&v)[4], int many) {
    if (many >= 4) store16_any(p, pack(v));
    else
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < many) p[e] = v[e];
}
// A row's fours, `many` numbers from this one on (all: the row has whole fours, the same for all).
template <typename T> __device__ __forceinline__ void put_four_of(T* p, const float (&v)[4], int many, bool all) {
    if (all) {
        if (many > 0) put_four_any(p, v, 4);
    } else if (many > 0) {
        put_four_any(p, v, many);
    }
}
__device__ __forceinline__ void four_any(const float* p, float (&v)[4], int many) {
    if (many >= 4) unpack(load16_any(p), v);
    else
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = e < many ? p[e] : 0.0f;
}

// N pieces of 16 bytes of a chunk's rows, at(i, row, column): piece i's row and first column of those that are looked at, which begin `first` numbers into rows of `wide` (16 bytes at
// least).  The requests are loads without a branch (one in a branch would be waited for there), their places in a whole chunk a number of 32 bits each that is formed once: where a row of
// memory ends inside a piece, the piece begins as much earlier, and settle() moves what is its own to its place and puts zeros behind it.
template <typename T, int N> struct Requests {
    static constexpr int V = kPiece<T>;
    uint4 u[N];
    uint32_t off[N];
    static __device__ __forceinline__ uint32_t place(int r, int c, int stride, int first, int wide) { return (uint32_t)(r * stride + min(first + c, wide - V)) * (uint32_t)sizeof(T); }
    template <class At> __device__ __forceinline__ void places(int stride, int first, int wide, At&& at) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            int r, c;
            at(i, r, c);
            off[i] = place(r, c, stride, first, wide);
        }
    }
    // base: the chunk's first row of memory
    template <class At> __device__ __forceinline__ void request(const T* base, int stride, int rows, int first, int wide, At&& at) {
        uint32_t to[N];
#pragma unroll
        for (int i = 0; i < N; ++i) to[i] = off[i];
        if (rows < kScanChunk) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                int r, c;
                at(i, r, c);
                to[i] = place(min(r, rows - 1), c, stride, first, wide);
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) u[i] = load16_any(reinterpret_cast<const char*>(base) + to[i]);
    }
    // Zeros from row `rows` and column `columns` on.
    template <class At> __device__ __forceinline__ void settle(int rows, int columns, int first, int wide, At&& at) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            int r, c;
            at(i, r, c);
            if (columns % V) {
                uint64_t lo = u[i].x | (uint64_t)u[i].y << 32, hi = u[i].z | (uint64_t)u[i].w << 32;
                const int bits = max(first + c + V - wide, 0) * (int)sizeof(T) * 8, keep = (columns - c) * (int)sizeof(T) * 8;
                if (bits >= 64) lo = hi >> (bits & 63), hi = 0;
                else if (bits > 0) lo = lo >> bits | hi << (64 - bits), hi >>= bits;
                if (keep < 64) hi = 0, lo &= keep > 0 ? (uint64_t(1) << keep) - 1 : 0;
                else if (keep < 128) hi &= (uint64_t(1) << (keep - 64)) - 1;
                u[i] = make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
            }
            if (r >= rows || c >= columns) u[i] = make_uint4(0, 0, 0, 0);
        }
    }
};

// The rows of a chunk on their way from memory to LDS: requested while the chunk before is worked on.  W columns, zeros behind the valid rows and columns.
template <typename T, int W, int THREADS> struct ChunkRows : Requests<T, kScanChunk * W / kPiece<T> / THREADS> {
    static constexpr int V = kPiece<T>, kEach = W / V, kMany = kScanChunk * kEach / THREADS;
    static_assert(kScanChunk * kEach % THREADS == 0, "pieces of a chunk");
    using Requests<T, kMany>::u;
    static __device__ __forceinline__ void at(int i, int& r, int& c) {
        const int k = (int)threadIdx.x + i * THREADS;
        r = k / kEach;
        c = k % kEach * V;
    }
    __device__ __forceinline__ void places_all(int64_t stride, int first, int wide) { this->places((int)stride, first, wide, at); }
    __device__ __forceinline__ void request_all(const T* base, int64_t stride, int rows, int first, int wide) { this->request(base, (int)stride, rows, first, wide, at); }
    __device__ __forceinline__ void settle_all(int rows, int columns, int first, int wide) { this->settle(rows, columns, first, wide, at); }
    template <int PITCH> __device__ __forceinline__ void put(T* tile) const {
#pragma unroll
        for (int i = 0; i < kMany; ++i) {
            const int k = (int)threadIdx.x + i * THREADS;
            *reinterpret_cast<uint4*>(tile + k / kEach * PITCH + k % kEach * V) = u[i];
        }
    }
    // whether a number of this thread's is not finite
    __device__ __forceinline__ bool odd() const {
        uint32_t most = 0;   // exponents of all, the largest in each half
#pragma unroll
        for (int i = 0; i < kMany; ++i)
#pragma unroll
            for (uint32_t w : {u[i].x, u[i].y, u[i].z, u[i].w}) {
                if constexpr (sizeof(T) == 2) most = max(most, max(w & 0x7f800000u, w << 16 & 0x7f800000u));
                else most = max(most, w & 0x7f800000u);
            }
        return most == 0x7f800000u;
    }
};

// The steps and decays of a chunk, a position to a lane: delta, the sum of the exponents up to the position in units of log 2 (in two floats: of sums of hundreds their differences keep
// their last places), the decay from before the chunk, that to the end of the position's sixteen and that to the chunk's end, for the walks times delta, for the gradients alone; and for
// those the slope of softplus.  Positions behind the last have delta 0: they change nothing.
template <bool GRADIENTS> struct ChunkDecays {
    float delta[kScanChunk], sum[kScanChunk], rest[kScanChunk], from[kScanChunk], tile[kScanChunk], to[kScanChunk], slope[GRADIENTS ? kScanChunk : 4];
    float end;       // the decay over the whole chunk
    double total;    // its exponent
};
constexpr double kLog2eD = 1.4426950408889634074;
// A head's rate, e^a: from 2^100 on nothing is left of a state after any step.
__device__ __forceinline__ double rate_of(float a_log) {
    const double rate = exp((double)a_log);
    return rate > 0x1p100 ? 0x1p100 : rate;
}

__device__ __forceinline__ float softplus(float u) { return fmaxf(u, 0.0f) + log1pf(expf(-fabsf(u))); }

// 2^e, e <= 0: of an exponent of hundreds what its float has lost is put back, as 1 + its natural multiple.
__device__ __forceinline__ float exp2_of(double e) {
    const float hi = (float)e, rest = (float)(e - (double)hi);
    return __builtin_amdgcn_exp2f(hi) * fmaf(0.69314718f, fabsf(rest) < 1.0f ? rest : 0.0f, 1.0f);
}

// dt: the position's (any number behind the last row).
template <bool GRADIENTS> __device__ __forceinline__ void chunk_decays(ChunkDecays<GRADIENTS>& d, float dt, int rows, float bias, double rate, int lane) {
    const float u = dt + bias;
    const float delta = lane >= rows ? 0.0f : u != u ? u : softplus(u);
    // (an exponent of -1024 leaves nothing of what was before; of larger ones the sums' roundings would matter)
    const float most = 1024.0f * __builtin_amdgcn_rcpf((float)rate);
    double sum = -(double)(delta > most ? most : delta) * rate;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
        const double before = __shfl_up(sum, k);
        if (lane >= k) sum += before;
    }
    const double total = __shfl(sum, 63), of_tile = __shfl(sum, lane | 15);
    const float hi = (float)sum;
    d.delta[lane] = delta;
    d.sum[lane] = hi;
    d.rest[lane] = hi - hi == 0.0f ? (float)(sum - (double)hi) : 0.0f;
    d.from[lane] = exp2_of(sum);
    d.to[lane] = exp2_of(total - sum) * (GRADIENTS ? 1.0f : delta);
    d.tile[lane] = exp2_of(of_tile - sum);
    if constexpr (GRADIENTS) d.slope[lane] = lane < rows ? 1.0f / (1.0f + expf(-u)) : 0.0f;
    if (lane == 63) {
        d.end = exp2_of(total);
        d.total = total;
    }
}

// The decay from behind position s to behind position t >= s.
__device__ __forceinline__ float decay_between(float sum_t, float rest_t, float sum_s, float rest_s) { return __builtin_amdgcn_exp2f((sum_t - sum_s) + (rest_t - rest_s)); }

// Which heads, samples and stretches a workgroup has: neighbours, which read the same B and C, on one of the eight XCDs.
__device__ __forceinline__ int64_t xcd_order(int64_t block, int64_t blocks) { return (block & 7) * (blocks >> 3) + (block >> 3); }

}  // namespace tmps
