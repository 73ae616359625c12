// Gradients of the selective state space.
//
// Two walks leave, for every chunk of 64 positions, the state S before it and the gradient G of the state behind it (the recurrence's adjoint: G <- d_end G + sum_t d_t dy_t C_t').  Chunks
// are independent then.  With Z[t][s] = C_t . B_s, R[t][s] = dy_t . x_s, D the decays, w_s = D[end][s] delta_s, sums over s <= t:
//   dx_s = sum_t Z D delta_s dy_t + w_s G B_s + skip dy_s      dB_s = sum_t R D delta_s C_t + w_s G' x_s      dC_t = sum_s R D delta_s B_s + d_t S' dy_t
// With q = Z R D, the gradient of position t's own exponent is what passes through it: sum_{t' >= t > s} q[t'][s] delta_s, and of the states sum_{t' >= t} d_t' C_t' S' dy_t' +
// sum_{s < t} w_s x_s G B_s + d_end <S, G>.  The first is had from sums over the rows and columns of tiles of 16 positions, and over the pairs around a position inside its own: nothing is
// added that would have to be taken off again (what does not pass through it can be thousands of times larger, and a rate multiplies its roundings).  A workgroup has a chunk and, one after the other, a part of the heads that share its B and C, whose Z it forms
// once and whose gradients of B and C stay in its accumulators.  Products are formed by columns t and again by columns s: decayed, they are then operands as they lie in the accumulators.
// In bf16 calls these are the sum of two bf16 terms (2^-17 of themselves), S and G of three (2^-25), since gradients of exponents are fp32 sums over them: with one and two terms dx was off by
// 1.1e-3 beside the 1.7e-3 of its rounding, and da_log and ddt_bias by 1.1e-6 instead of 7.5e-7 and 3.5e-7.  (Sums of 32 bf16 products come out of the matrix unit 1.5e-10 of the products'
// sizes too low on average: over thousands of pairs of positions that is what is left of da_log's error, fp32 calls have 1.5e-7.)
// 16 x 512 positions of 24 heads of 64 x 64 in bf16: 43 us the walks (100 MB of states written, most of it read again from the last cache), 81 the chunks (64 with one and two terms; vector
// instructions and latency, two waves to a SIMD; 56 bytes of registers spill, addresses that are asked for once a head), 5 the parts' gradients of B and C, 5 the sums.
#include "launch.h"
#include "scan_walk.hip.h"
#include "wave.hip.h"

namespace tmps {

struct ScanGrad {
    ScanBackward b;
    const float *before, *behind;   // S and G: [samples, heads, chunks, PP * slices, NP]
    float* shared;                  // gradients of B and C of each part: [parts][rows][2 groups n] (null: one part, straight to dx)
    float* sums;                    // [samples * chunks][3 heads]
    int chunks, parts, each, slices;
};

// Sums of 16 values over the 16 lanes of a row: lane i of them has that of value i.  Each step halves the values: 45 instructions, where a sum of each in all lanes takes 64.
template <int CTRL, int N, int M> __device__ __forceinline__ void halve(float (&v)[M], bool upper) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float keep = upper ? v[i + N] : v[i], give = upper ? v[i] : v[i + N];
        v[i] = keep + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(give), CTRL, 0xF, 0xF, false));
    }
}
__device__ __forceinline__ float sixteen_sums(float (&v)[16], int lane) {
    halve<0x128, 8>(v, lane & 8);   // row_ror:8: lane ^ 8
    halve<0x141, 4>(v, lane & 4);   // row_half_mirror: lane ^ 7
    halve<0x1B, 2>(v, lane & 2);    // quad_perm 3, 2, 1, 0: lane ^ 3
    halve<0xB1, 1>(v, lane & 1);    // quad_perm 1, 0, 3, 2: lane ^ 1
    return v[0];
}
// The same of four values: lanes 4 i .. 4 i + 3 of them have that of value i.
__device__ __forceinline__ float four_sums(float (&v)[4], int lane) {
    halve<0x128, 2>(v, lane & 8);
    halve<0x141, 1>(v, lane & 4);
    v[0] += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v[0]), 0xB1, 0xF, 0xF, false));          // quad_perm 1, 0, 3, 2
    return v[0] + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v[0]), 0x4E, 0xF, 0xF, false));   // quad_perm 2, 3, 0, 1
}
// over the four lanes of a column
__device__ __forceinline__ float column_sum(float v) {
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// Whether LDS holds what two workgroups of a compute unit need.
template <typename T, int NP> constexpr bool kTwoGroups = sizeof(T) == 2 && NP <= 64;
// Heads whose decays are formed before, and whose steps' gradients behind the others, at a time, a wave each: four, or what LDS holds.
template <typename T, int NP> constexpr int kHeadsAtOnce = sizeof(T) == 4 && NP == 128 ? 2 : 4;

// Of a head's chunk: sums of q over the rows of each tile of 16 positions by column, over a row's columns of earlier tiles, over what passes through a position inside its tile, q of each
// position itself, C S' dy and x G B, and of each wave its parts of <S, G> and of dy x.
struct HeadSums {
    float columns[4][kScanChunk], row[kScanChunk], tile[kScanChunk], self[kScanChunk], of_c[kScanChunk], of_b[kScanChunk], parts[4][2];
};

template <typename T, int NP, int PT> __global__ __launch_bounds__(256, (kTwoGroups<T, NP> ? 2 : 1)) void scan_grad_kernel(ScanGrad a) {
    constexpr int V = kPiece<T>, PP = PT * 16, XP = PP + V, BP = NP + V, NT = NP / 16, NK = NP / 32, PK = PP / 32;
    constexpr int GT = kStateTerms<T>, RT = kResultTerms<T>;   // of S and G on their way to exponents' gradients, fp32; of those and decayed products to gradients of the type
    constexpr int kHeads = kHeadsAtOnce<T, NP>;
    constexpr int kState = PP * NP / 4 / 256;   // fours of a state of a thread
    __shared__ __attribute__((aligned(16))) T bs[kScanChunk * BP], cs[kScanChunk * BP], xs[kScanChunk * XP], dys[kScanChunk * XP], sg[GT * PP * BP];
    __shared__ __attribute__((aligned(16))) ChunkDecays<true> decays[kHeads];
    __shared__ HeadSums sums[kHeads];
    const ScanBackward& b = a.b;
    const Scan& f = b.f;
    const int64_t units = f.samples * a.chunks * f.groups * a.parts;
    int64_t unit = xcd_order(blockIdx.x, gridDim.x);
    if (unit >= units) return;
    const int part = (int)(unit % a.parts);
    unit /= a.parts;
    const int group = (int)(unit % f.groups);
    unit /= f.groups;
    const int chunk = (int)(unit % a.chunks);
    const int64_t sample = unit / a.chunks;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, col = lane & 15;
    const int rows = (int)min<int64_t>(kScanChunk, f.positions - (int64_t)chunk * kScanChunk);
    const int64_t row0 = sample * f.positions + (int64_t)chunk * kScanChunk;
    const int in_group = f.heads / f.groups, first = part * a.each, last = min(first + a.each, in_group);   // heads of the group
    const int64_t b_at = (int64_t)f.heads * f.dh + (int64_t)group * f.n, c_at = b_at + (int64_t)f.groups * f.n;
    const int own = 16 * wave + col;   // this lane's column: a position
    const int wide = (int)(f.heads * f.dh + 2 * f.groups * f.n), inner = f.heads * f.dh;

    {
        ChunkRows<T, NP, 256> r;
        const T* const base = (const T*)f.x + row0 * f.x_stride;
        r.places_all(f.x_stride, (int)b_at, wide);
        r.request_all(base, f.x_stride, rows, (int)b_at, wide);
        r.settle_all(rows, f.n, (int)b_at, wide);
        r.template put<BP>(bs);
        r.places_all(f.x_stride, (int)c_at, wide);
        r.request_all(base, f.x_stride, rows, (int)c_at, wide);
        r.settle_all(rows, f.n, (int)c_at, wide);
        r.template put<BP>(cs);
    }
    __syncthreads();
    f32x4_t z[4], zs[4];   // rows s, column t; rows t, column s
#pragma unroll
    for (int st = 0; st < 4; ++st) {
        z[st] = zs[st] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < NK; ++k) {
            if (st <= wave) z[st] = mma(along<false>(bs + (16 * st + col) * BP, 32 * k, lane), along<false>(cs + own * BP, 32 * k, lane), z[st]);
            if (st >= wave) zs[st] = mma(along<false>(cs + (16 * st + col) * BP, 32 * k, lane), along<false>(bs + own * BP, 32 * k, lane), zs[st]);
        }
    }
    f32x4_t db[NT], dc[NT];   // rows n, columns s and t
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) db[nt] = dc[nt] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

    const bool plain = rows == kScanChunk && f.dh % PP == 0;   // (no zeros to be put in)
    ChunkRows<T, PP, 256> rx, rd;
    rx.places_all(f.x_stride, 0, wide);
    rd.places_all(b.dy_stride, 0, inner);
    for (int h = first; h < last; ++h) {
        const int head = group * in_group + h;
        const float skip = f.skip[head];
        float dskip = 0.0f, meet = 0.0f;   // sums of dy x and of S G
        for (int slice = 0; slice < a.slices; ++slice) {
            const int p0 = slice * 64, width = min(64, f.dh - p0);
            const int at = head * f.dh + p0;
            const T *xg = (const T*)f.x + row0 * f.x_stride, *dyg = (const T*)b.dy + row0 * b.dy_stride;
            if (plain) {   // (the same places in each head's columns)
                xg += at;
                dyg += at;
            } else {
                rx.places_all(f.x_stride, at, wide);
                rd.places_all(b.dy_stride, at, inner);
            }
            rx.request_all(xg, f.x_stride, rows, at, wide);
            rd.request_all(dyg, b.dy_stride, rows, at, inner);
            float s4[kState][4], g4[kState][4];
            const int64_t of_state = (((sample * f.heads + head) * a.chunks + chunk) * a.slices + slice) * (int64_t)(PP * NP);
            const float *const before = a.before + of_state, *const behind = a.behind + of_state;
#pragma unroll
            for (int i = 0; i < kState; ++i) {
                four(before + 4 * threadIdx.x + 1024 * i, s4[i]);
                four(behind + 4 * threadIdx.x + 1024 * i, g4[i]);
            }
            __syncthreads();   // (what the head or slice before has left in LDS has been read)
            if (slice == 0 && (h - first) % kHeads == 0 && wave < kHeads && h + wave < last) {
                const int mine = head + wave;
                chunk_decays(decays[wave], to_f32(((const T*)f.dt)[(row0 + min(lane, rows - 1)) * f.dt_stride + mine]), rows, f.dt_bias[mine],
                                   rate_of(f.a_log[mine]) * kLog2eD, lane);
            }
            if (!plain) {
                rx.settle_all(rows, width, at, wide);
                rd.settle_all(rows, width, at, inner);
            }
            rx.template put<XP>(xs);
            rd.template put<XP>(dys);
            const auto put_state = [&](const float (&v)[kState][4]) {
#pragma unroll
                for (int i = 0; i < kState; ++i) {
                    const int k = (int)threadIdx.x + 256 * i, p = k / (NP / 4), n = k % (NP / 4) * 4;
                    float w[4] = {v[i][0], v[i][1], v[i][2], v[i][3]};
#pragma unroll
                    for (int term = 0; term < GT; ++term) {
                        put_four(sg + (term * PP + p) * BP + n, w);
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] -= (float)(T)w[e];
                    }
                }
            };
            put_state(s4);
#pragma unroll
            for (int i = 0; i < kState; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) meet = fmaf(s4[i][e], g4[i][e], meet);
            __syncthreads();
            const ChunkDecays<true>& d = decays[(h - first) % kHeads];
            HeadSums& sum = sums[(h - first) % kHeads];

            // by columns t
            f32x4_t dz[4];
            float from_row = 0.0f, of_self = 0.0f, q16[16], through[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            // (accumulated over a head's slices)
            const auto put_sum = [&](float& to, float v) { to = slice == 0 ? v : to + v; };
            Oct<T> dyf[PK];
#pragma unroll
            for (int k = 0; k < PK; ++k) dyf[k] = along<false>(dys + own * XP, 32 * k, lane);
            const float sum_t = d.sum[own], rest_t = d.rest[own];
#pragma unroll
            for (int st = 0; st < 4; ++st) {
                f32x4_t r = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
                dz[st] = r;
                if (st <= wave) {
#pragma unroll
                    for (int k = 0; k < PK; ++k) r = mma(along<false>(xs + (16 * st + col) * XP, 32 * k, lane), dyf[k], r);
                    float delta_s[4], decay[4];
                    four(d.delta + 16 * st + 4 * g, delta_s);
                    if (st < wave) {
                        // (by way of the end of the sixteen positions of s: neither factor is over one)
                        const float on = decay_between(sum_t, rest_t, d.sum[16 * st + 15], d.rest[16 * st + 15]);
                        four(d.tile + 16 * st + 4 * g, decay);
#pragma unroll
                        for (int e = 0; e < 4; ++e) decay[e] *= on;
                    } else {
                        float sum_s[4], rest_s[4];
                        four(d.sum + 16 * st + 4 * g, sum_s);
                        four(d.rest + 16 * st + 4 * g, rest_s);
#pragma unroll
                        for (int e = 0; e < 4; ++e) decay[e] = 4 * g + e <= col ? decay_between(sum_t, rest_t, sum_s[e], rest_s[e]) : 0.0f;
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float q = r[e] * (z[st][e] * decay[e]);
                        dz[st][e] = r[e] * (decay[e] * delta_s[e]);
                        if (st == wave) {   // (of a position itself nothing passes through)
                            const bool self = 4 * g + e == col;
                            of_self = self ? q : of_self;
                            dskip += self ? r[e] : 0.0f;
                            q = self ? 0.0f : q;
                            through[e] = q * delta_s[e];
                        } else {
                            from_row = fmaf(q, delta_s[e], from_row);
                        }
                        r[e] = q;
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) q16[4 * st + e] = r[e];
            }
            put_sum(sum.columns[wave][16 * (col >> 2) + 4 * g + (col & 3)], sixteen_sums(q16, lane));
            if (col >> 2 == g) put_sum(sum.self[own], of_self);
            {
                // inside the tile: of each t' what comes from the positions up to s, and of that, for the position behind s, the sum over t' from it on
#pragma unroll
                for (int e = 1; e < 4; ++e) through[e] += through[e - 1];
                const float below1 = __shfl_up(through[3], 16), below2 = __shfl_up(through[3], 32), below3 = __shfl_up(through[3], 48);
                const float below = ((g > 2 ? below3 : 0.0f) + (g > 1 ? below2 : 0.0f)) + (g > 0 ? below1 : 0.0f);
#pragma unroll
                for (int e = 0; e < 4; ++e) through[e] = col > 4 * g + e ? below + through[e] : 0.0f;
                const float over = four_sums(through, lane);
                const int t = 4 * g + (col >> 2) + 1;
                if ((col & 3) == 0 && t < 16) put_sum(sum.tile[16 * wave + t], over);
                if (lane == 1) sum.tile[16 * wave] = 0.0f;
            }
#pragma unroll
            for (int pair = 0; pair < 2; ++pair) {
                if (2 * pair > wave) continue;
                Oct<T> zf[RT];
#pragma unroll
                for (int e = 0; e < 8; ++e) terms_of(dz[2 * pair + e / 4][e % 4], e, zf);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const Oct<T> b = across<true>(bs, BP, 32 * pair, 16 * nt, lane);
#pragma unroll
                    for (int term = RT - 1; term >= 0; --term) dc[nt] = mma(b, zf[term], dc[nt]);
                }
            }
            float with_c = 0.0f;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                f32x4_t v = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int term = GT - 1; term >= 0; --term)
#pragma unroll
                    for (int k = 0; k < PK; ++k) v = mma(across<false>(sg + term * PP * BP, BP, 32 * k, 16 * nt, lane), dyf[k], v);
                float c[4];
                four(cs + own * BP + 16 * nt + 4 * g, c);
#pragma unroll
                for (int e = 0; e < 4; ++e) with_c = fmaf(v[e], c[e], with_c);
                dc[nt] += v * d.from[own];
            }
            from_row = column_sum(from_row);
            with_c = column_sum(with_c);
            if (g == 0) {
                put_sum(sum.row[own], from_row);
                put_sum(sum.of_c[own], with_c);
            }

            // by columns s: the same products anew, whose rows t are then operands as they lie
            Oct<T> xf[PK];
#pragma unroll
            for (int k = 0; k < PK; ++k) xf[k] = along<false>(xs + own * XP, 32 * k, lane);
            const float delta_own = d.delta[own];
            f32x4_t m[4];
            {
                const float sum_end = d.sum[16 * wave + 15], rest_end = d.rest[16 * wave + 15], tile_own = d.tile[own];
#pragma unroll
                for (int tt = 0; tt < 4; ++tt) {
                    f32x4_t r = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
                    m[tt] = dz[tt] = r;
                    if (tt < wave) continue;
#pragma unroll
                    for (int k = 0; k < PK; ++k) r = mma(along<false>(dys + (16 * tt + col) * XP, 32 * k, lane), xf[k], r);
                    float sum_r[4], rest_r[4];
                    four(d.sum + 16 * tt + 4 * g, sum_r);
                    four(d.rest + 16 * tt + 4 * g, rest_r);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float decay;
                        if (tt > wave) decay = tile_own * decay_between(sum_r[e], rest_r[e], sum_end, rest_end);
                        else decay = 4 * g + e >= col ? decay_between(sum_r[e], rest_r[e], sum_t, rest_t) : 0.0f;
                        decay *= delta_own;
                        m[tt][e] = zs[tt][e] * decay;
                        dz[tt][e] = r[e] * decay;
                    }
                }
            }
            f32x4_t dx[PT];
#pragma unroll
            for (int j = 0; j < PT; ++j) dx[j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int pair = 0; pair < 2; ++pair) {
                if (2 * pair + 1 < wave) continue;
                Oct<T> mf[RT], zf[RT];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    terms_of(m[2 * pair + e / 4][e % 4], e, mf);
                    terms_of(dz[2 * pair + e / 4][e % 4], e, zf);
                }
#pragma unroll
                for (int j = 0; j < PT; ++j) {
                    const Oct<T> dy = across<true>(dys, XP, 32 * pair, 16 * j, lane);
#pragma unroll
                    for (int term = RT - 1; term >= 0; --term) dx[j] = mma(dy, mf[term], dx[j]);
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const Oct<T> c = across<true>(cs, BP, 32 * pair, 16 * nt, lane);
#pragma unroll
                    for (int term = RT - 1; term >= 0; --term) db[nt] = mma(c, zf[term], db[nt]);
                }
            }
            __syncthreads();   // (S has been read)
            put_state(g4);
            __syncthreads();
            Oct<T> bf[NK];
#pragma unroll
            for (int k = 0; k < NK; ++k) bf[k] = along<false>(bs + own * BP, 32 * k, lane);
            const float to = delta_own * d.to[own];
#pragma unroll
            for (int j = 0; j < PT; ++j) {
                f32x4_t v = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int term = RT - 1; term >= 0; --term)
#pragma unroll
                    for (int k = 0; k < NK; ++k) v = mma(along<false>(sg + (term * PP + 16 * j + col) * BP, 32 * k, lane), bf[k], v);
                float dyv[4], out[4];
                four(dys + own * XP + 16 * j + 4 * g, dyv);
#pragma unroll
                for (int e = 0; e < 4; ++e) out[e] = fmaf(skip, dyv[e], fmaf(to, v[e], dx[j][e]));
                if (own < rows)
                    put_four_of((T*)b.dx + (row0 + own) * b.dx_stride + (int64_t)head * f.dh + p0 + 16 * j + 4 * g, out, width - 16 * j - 4 * g, width % 4 == 0);
            }
            float with_b = 0.0f;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                f32x4_t v = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int term = GT - 1; term >= 0; --term)
#pragma unroll
                    for (int k = 0; k < PK; ++k) v = mma(across<false>(sg + term * PP * BP, BP, 32 * k, 16 * nt, lane), xf[k], v);
                float bv[4];
                four(bs + own * BP + 16 * nt + 4 * g, bv);
#pragma unroll
                for (int e = 0; e < 4; ++e) with_b = fmaf(v[e], bv[e], with_b);
                db[nt] += v * to;
            }
            with_b = column_sum(with_b);
            if (g == 0) put_sum(sum.of_b[own], with_b);
        }
        const float meet_all = wsum(meet), skip_all = wsum(dskip);
        if (lane == 0) {
            sums[(h - first) % kHeads].parts[wave][0] = meet_all;
            sums[(h - first) % kHeads].parts[wave][1] = skip_all;
        }
        if ((h - first) % kHeads != kHeads - 1 && h + 1 < last) continue;
        // the heads' steps and parameters, a head to a wave
        __syncthreads();
        const int mine = h - (h - first) % kHeads + wave;
        if (wave < kHeads && mine <= h) {
            const int head = group * in_group + mine;
            const ChunkDecays<true>& d = decays[wave];
            const HeadSums& sum = sums[wave];
            const float rate = (float)rate_of(f.a_log[head]), delta = d.delta[lane], slope = d.slope[lane];
            // sums of q over the positions of each tile of 16, from the tile of position s (its own, below) on
            const int tile = lane >> 4;
            float later[4], in_tile = 0.0f, behind = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                later[w] = w > tile ? sum.columns[w][lane] : 0.0f;
                in_tile = w == tile ? sum.columns[w][lane] : in_tile;
                behind += later[w];
            }
            // tiles before t's to tiles behind it
            float over1 = tile == 0 ? delta * (later[2] + later[3]) : 0.0f, over2 = tile <= 1 ? delta * later[3] : 0.0f;
            over1 = wsum(over1);
            over2 = wsum(over2);
            // in tile order: from t on of rows, before t of columns
            float rows_on = sum.row[lane], columns_before = delta * behind;
#pragma unroll
            for (int k = 1; k < 16; k <<= 1) {
                const float on = __shfl_down(rows_on, k, 16), before = __shfl_up(columns_before, k, 16);
                if ((lane & 15) + k < 16) rows_on += on;
                if ((lane & 15) >= k) columns_before += before;
            }
            columns_before = __shfl_up(columns_before, 1, 16);
            columns_before = (lane & 15) ? columns_before : 0.0f;
            // of the states: from t on, and before t
            const float with_g = sum.of_b[lane];
            float states_on = d.from[lane] * sum.of_c[lane], states_before = delta * d.to[lane] * with_g;
#pragma unroll
            for (int k = 1; k < 64; k <<= 1) {
                const float on = __shfl_down(states_on, k), before = __shfl_up(states_before, k);
                if (lane + k < 64) states_on += on;
                if (lane >= k) states_before += before;
            }
            states_before = __shfl_up(states_before, 1);
            states_before = lane ? states_before : 0.0f;
            const float whole = d.end * ((sum.parts[0][0] + sum.parts[1][0]) + (sum.parts[2][0] + sum.parts[3][0]));
            const float of_exponent = (((sum.tile[lane] + rows_on) + columns_before) + (tile == 1 ? over1 : tile == 2 ? over2 : 0.0f)) + ((states_on + states_before) + whole);
            // (a step that leaves nothing of what was before: of its exponent's gradient there are only roundings, which such a rate would make large)
            const float by = delta * rate > 1024.0f ? 0.0f : -rate;
            const float ddelta = fmaf(by, of_exponent, (sum.self[lane] + (in_tile + behind)) + d.to[lane] * with_g), du = lane < rows ? ddelta * slope : 0.0f;
            if (lane < rows) ((T*)b.ddt)[(row0 + lane) * b.ddt_stride + head] = from_f32<T>(du);
            const float drate = wsum(lane < rows ? by * delta * of_exponent : 0.0f), dbias = wsum(du);
            if (lane == 0) {
                float* const to = a.sums + (sample * a.chunks + chunk) * 3 * f.heads + head;
                to[0] = drate;
                to[f.heads] = (sum.parts[0][1] + sum.parts[1][1]) + (sum.parts[2][1] + sum.parts[3][1]);
                to[2 * f.heads] = dbias;
            }
        }
    }
    if (own >= rows) return;
    const int64_t of_shared = 2 * (int64_t)f.groups * f.n;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int n = 16 * nt + 4 * g;
        if (n >= f.n) continue;
        const float vb[4] = {db[nt][0], db[nt][1], db[nt][2], db[nt][3]}, vc[4] = {dc[nt][0], dc[nt][1], dc[nt][2], dc[nt][3]};
        if (a.shared) {
            float* const to = a.shared + ((int64_t)part * f.samples * f.positions + row0 + own) * of_shared + (int64_t)group * f.n + n;
            put_four_any(to, vb, f.n - n);
            put_four_any(to + (int64_t)f.groups * f.n, vc, f.n - n);
        } else {
            T* const to = (T*)b.dx + (row0 + own) * b.dx_stride;
            put_four_any(to + b_at + n, vb, f.n - n);
            put_four_any(to + c_at + n, vc, f.n - n);
        }
    }
}

// Gradients of B and C: the parts' sums, rounded once.
template <typename T> __global__ __launch_bounds__(256) void scan_shared_kernel(ScanGrad a) {
    const Scan& f = a.b.f;
    const int64_t wide = 2 * (int64_t)f.groups * f.n, rows = f.samples * f.positions, i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= rows * wide) return;
    const int many = (int)min<int64_t>(4, rows * wide - i);
    float sum[4];
    four_any(a.shared + i, sum, many);
    for (int k = 1; k < a.parts; ++k) {
        float v[4];
        four_any(a.shared + k * rows * wide + i, v, many);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += v[e];
    }
    const int64_t row = i / wide, at = i % wide;
    T* const to = (T*)a.b.dx + (int64_t)f.heads * f.dh;
    if (many == 4 && at + 4 <= wide) {
        put_four_any(to + row * a.b.dx_stride + at, sum, 4);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < many) to[(i + e) / wide * a.b.dx_stride + (i + e) % wide] = from_f32<T>(sum[e]);
    }
}

// ------------------------------------------------------------------------------------------------ launches
// Parts of a group's heads: as many as give the chip 512 workgroups.
constexpr int kGradGroups = 512;
static void grad_plan(ScanGrad& a) {
    const Scan& f = a.b.f;
    a.chunks = (int)((f.positions + kScanChunk - 1) / kScanChunk);
    a.slices = (f.dh + 63) / 64;
    const int64_t groups = f.samples * a.chunks * f.groups;
    const int in_group = f.heads / f.groups;
    int64_t parts = (kGradGroups + groups - 1) / groups;
    if (parts > in_group) parts = in_group;
    a.each = (int)((in_group + parts - 1) / parts);
    a.parts = (in_group + a.each - 1) / a.each;
}

static size_t on256(size_t bytes) { return (bytes + 255) / 256 * 256; }

// The stretches' states, S, G, sums, and what the parts leave: as much as any call of no more samples and positions takes.
struct GradRoom {
    size_t walk, states, sums, shared;
    size_t all() const { return walk + 2 * states + sums + shared; }
};
static GradRoom grad_room(const Scan& f) {
    const int64_t chunks = (f.positions + kScanChunk - 1) / kScanChunk, of_chunks = f.samples * chunks;
    GradRoom r;
    r.walk = on256(2 * walk_stretch_bytes(f));
    r.states = on256((size_t)of_chunks * f.heads * padded_dh(f.dh) * padded_n(f.n) * sizeof(float));
    r.sums = on256((size_t)of_chunks * 3 * f.heads * sizeof(float));
    // (parts x chunks is at most the workgroups wanted and as many again as there are chunks)
    const int64_t most = std::min<int64_t>(of_chunks * (f.heads / f.groups), kGradGroups / f.groups + of_chunks);
    r.shared = f.heads == f.groups ? 0 : on256((size_t)most * kScanChunk * 2 * f.groups * f.n * sizeof(float));
    return r;
}

size_t scan_backward_workspace_bytes(int, const Scan& a) { return grad_room(a).all(); }

template <typename T> static hipError_t backward_type(const ScanBackward& b, void* ws, hipStream_t s) {
    const GradRoom room = grad_room(b.f);
    char* at = static_cast<char*>(ws);
    ScanGrad a;
    a.b = b;
    grad_plan(a);
    float* const before = reinterpret_cast<float*>(at + room.walk);
    float* const behind = reinterpret_cast<float*>(at + room.walk + room.states);
    a.before = before; a.behind = behind;
    a.sums = reinterpret_cast<float*>(at + room.walk + 2 * room.states);
    a.shared = a.parts > 1 ? reinterpret_cast<float*>(at + room.walk + 2 * room.states + room.sums) : nullptr;
    ScanWalk w = walk_of(b.f);
    w.chunk_states = before;
    walk_plan(w);
    ScanWalk back = w;
    back.x = b.dy; back.x_stride = b.dy_stride; back.x_wide = b.f.heads * b.f.dh; back.b_first = w.c_first;
    back.first_state = b.dstate; back.chunk_states = behind; back.final_state = b.dstate_in;
    const unsigned walks = walk_grid(w);
    const int64_t units = b.f.samples * a.chunks * b.f.groups * a.parts, blocks = (units + 7) / 8 * 8;
    const int64_t shared_blocks = ((b.f.samples * b.f.positions * 2 * b.f.groups * b.f.n + 3) / 4 + 255) / 256;
    if (!walks || !launchable(blocks, 256) || !launchable(shared_blocks, 256)) return hipErrorInvalidValue;
    hipError_t e = hipSuccess;
    if (w.stretches > 1) {
        walk_room(back, walk_room(w, at));
#define TMPS_OWNS(NP, PT) launch_timed(kcAttnBwd, scan_walks_kernel<T, NP, PT, kWalkOwn>, dim3(walks, 2), dim3(256), 0, s, w, back)
        e = TMPS_WALK(TMPS_OWNS, w);
        if (e != hipSuccess) return e;
        e = launch_timed(kcAttnBwd, scan_joins_kernel, dim3(join_grid(w), 2), dim3(256), 0, s, w, back, padded_n(w.n), padded_dh(w.dh) * padded_n(w.n));
        if (e != hipSuccess) return e;
    }
#define TMPS_WALKS(NP, PT) launch_timed(kcAttnBwd, scan_walks_kernel<T, NP, PT, kWalkStates>, dim3(walks, 2), dim3(256), 0, s, w, back)
    e = TMPS_WALK(TMPS_WALKS, w);
    if (e != hipSuccess) return e;
    const Scan& f = b.f;
    const dim3 grid((unsigned)blocks), block(256);
    if (f.dh > 32) {
        if (f.n <= 32) e = launch_timed(kcAttnBwd, scan_grad_kernel<T, 32, 4>, grid, block, 0, s, a);
        else if (f.n <= 64) e = launch_timed(kcAttnBwd, scan_grad_kernel<T, 64, 4>, grid, block, 0, s, a);
        else e = launch_timed(kcAttnBwd, scan_grad_kernel<T, 128, 4>, grid, block, 0, s, a);
    } else {
        if (f.n <= 32) e = launch_timed(kcAttnBwd, scan_grad_kernel<T, 32, 2>, grid, block, 0, s, a);
        else if (f.n <= 64) e = launch_timed(kcAttnBwd, scan_grad_kernel<T, 64, 2>, grid, block, 0, s, a);
        else e = launch_timed(kcAttnBwd, scan_grad_kernel<T, 128, 2>, grid, block, 0, s, a);
    }
    if (e != hipSuccess) return e;
    if (a.shared) {
        e = launch_timed(kcAttnBwd, scan_shared_kernel<T>, dim3((unsigned)shared_blocks), dim3(256), 0, s, a);
        if (e != hipSuccess) return e;
    }
    return reduce_all(Reductions(1, Reduction{a.sums, b.dparams, 3 * (int64_t)f.heads, (int)(f.samples * a.chunks), true}), s);
}

hipError_t scan_backward(int dtype, const ScanBackward& b, void* ws, hipStream_t s) { return dtype == kBF16 ? backward_type<bf16_t>(b, ws, s) : backward_type<float>(b, ws, s); }

}  // namespace tmps
