// The walk over the chunks of a head's positions with its state in the accumulators: forward with the results y, forward or backward for the states of the chunks alone.
#pragma once
#include <algorithm>
#include <type_traits>

#include "launch.h"
#include "scan.hip.h"

namespace tmps {

// States in workspaces have whole tiles, zeros behind the last feature.
inline int padded_n(int n) { return n <= 32 ? 32 : n <= 64 ? 64 : 128; }
inline int padded_dh(int dh) { return dh <= 32 ? 32 : (dh + 63) / 64 * 64; }

// The walk's operands: "x" and "b" are x and B going forward, dy and C going backward, where the state is the gradient of the state behind a chunk.
struct ScanWalk {
    const void *x, *b, *dt;         // rows of x, of B and C, of dt
    int64_t x_stride, bc_stride, dt_stride;
    int x_wide, bc_wide, b_first, c_first;   // numbers of a row, those before B and before C
    const float *a_log, *skip, *dt_bias;
    const float* first_state;    // before the first chunk of the walk: [samples, heads, dh, n] (null: zeros)
    void* y;
    int64_t y_stride;
    float* final_state;          // behind the last chunk (null: not wanted)
    float* chunk_states;         // before each chunk of the walk: [samples, heads, chunks, padded dh, NP] (null: not wanted)
    int64_t samples, positions;
    int heads, dh, groups, n;
    int chunks, stretches, each, slices, tiles;   // chunks of a sample, stretches of them and the chunks of one, slices of a head's features and their tiles of 16
    float* stretch_states;       // [samples, heads, stretches, padded dh, NP]: left by each, then before each
    double* stretch_totals;
};

inline ScanWalk walk_of(const Scan& a) {
    ScanWalk w;
    w.x = w.b = a.x;
    w.dt = a.dt; w.x_stride = w.bc_stride = a.x_stride; w.dt_stride = a.dt_stride;
    w.b_first = a.heads * a.dh; w.c_first = w.b_first + a.groups * a.n;
    w.x_wide = w.bc_wide = w.c_first + a.groups * a.n;
    w.a_log = a.a_log; w.skip = a.skip; w.dt_bias = a.dt_bias; w.first_state = a.state;
    w.y = nullptr; w.y_stride = 0; w.final_state = nullptr; w.chunk_states = nullptr;
    w.samples = a.samples; w.positions = a.positions; w.heads = a.heads; w.dh = a.dh; w.groups = a.groups; w.n = a.n;
    w.stretch_states = nullptr; w.stretch_totals = nullptr;
    return w;
}

template <typename T> constexpr int kStateTerms = sizeof(T) == 2 ? 3 : 1;    // of a state's increments: results in fp32
template <typename T> constexpr int kResultTerms = sizeof(T) == 2 ? 2 : 1;   // of states and decayed products on their way to results of the type

template <typename T, int NP, int PT, bool OUT> struct WalkTiles {
    static constexpr int V = kPiece<T>, PP = PT * 16, XP = PP + V, BP = NP + V;
    __attribute__((aligned(16))) T xs[kScanChunk * XP];
    __attribute__((aligned(16))) T bs[kScanChunk * BP];
    __attribute__((aligned(16))) T ss[OUT ? kResultTerms<T> * PP * BP : 8];
    __attribute__((aligned(16))) ChunkDecays<false> decays[4];
    int odd[2];
};

// What a walk leaves: results (and the state behind the last chunk), the states before its chunks, or each stretch's own state and exponent, from nothing.
enum { kWalkResults, kWalkStates, kWalkOwn };

// What one workgroup does: stretch, head, slice and sample number `unit`.
template <typename T, int NP, int PT, int LEAVES, bool REV> __device__ __forceinline__ void scan_walk(const ScanWalk& a, int64_t unit, WalkTiles<T, NP, PT, LEAVES == kWalkResults>& tiles) {
    constexpr bool OUT = LEAVES == kWalkResults;
    constexpr int V = kPiece<T>, PP = PT * 16, XP = PP + V, BP = NP + V, NT = NP / 16, TW = NT * PT / 4, NK = NP / 32;
    constexpr int RT = kResultTerms<T>, ST = kStateTerms<T>;
    T *const xs = tiles.xs, *const bs = tiles.bs, *const ss = tiles.ss;
    ChunkDecays<false>* const decays = tiles.decays;
    int* const odd = tiles.odd;
    const int slice = (int)(unit % a.slices);
    unit /= a.slices;
    const int head = (int)(unit % a.heads);
    unit /= a.heads;
    const int stretch = (int)(unit % a.stretches);
    const int64_t sample = unit / a.stretches;
    const int group = head / (a.heads / a.groups);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, col = lane & 15;
    const int p0 = slice * PP, width = max(min(PP, a.dh - p0), 0);   // (a slice behind the last feature has zeros)
    const double rate = rate_of(a.a_log[head]) * kLog2eD;
    const float bias = a.dt_bias[head];

    const int64_t rows0 = sample * a.positions;
    const T* const xg = (const T*)a.x + rows0 * a.x_stride;
    const T* const bg = (const T*)a.b + rows0 * a.bc_stride;
    const T* const dtg = (const T*)a.dt + rows0 * a.dt_stride + head;
    const int x_first = head * a.dh + min(p0, a.dh - 1), b_first = a.b_first + group * a.n, c_first = a.c_first + group * a.n;

    // this wave's tiles of the state: 16 features p, n tiles a few apart; rows n, columns p
    const int pt = wave % PT, nt0 = wave / PT;
    constexpr int NSTEP = 4 / PT;
    const int p = pt * 16 + col;   // in the slice
    f32x4_t state[TW];
    const int64_t of_head = (sample * a.heads + head) * a.dh * a.n + (int64_t)(p0 + p) * a.n;
    const int64_t whole = (int64_t)a.slices * PP * NP, in_whole = (int64_t)(p0 + p) * NP;
    const int64_t of_stretch = ((sample * a.heads + head) * a.stretches + stretch) * whole + in_whole;
    const auto n_of = [&](int k) { return (nt0 + k * NSTEP) * 16 + 4 * g; };
#pragma unroll
    for (int k = 0; k < TW; ++k) {
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (LEAVES == kWalkOwn) {
        } else if (a.stretches > 1) {
            four(a.stretch_states + of_stretch + n_of(k), v);
        } else if (a.first_state && p < width && n_of(k) < a.n) {
            four_any(a.first_state + of_head + n_of(k), v, a.n - n_of(k));
        }
        state[k] = f32x4_t{v[0], v[1], v[2], v[3]};
    }

    const int first = stretch * a.each, many = min(a.each, a.chunks - first);
    const auto chunk_of = [&](int i) { return REV ? first + many - 1 - i : first + i; };
    const auto rows_of = [&](int chunk) { return (int)min<int64_t>(kScanChunk, a.positions - (int64_t)chunk * kScanChunk); };
    constexpr int kC = (int)sizeof(T) / 2;   // pieces of eight numbers
    ChunkRows<T, PP, 256> xr;
    ChunkRows<T, NP, 256> br;
    Requests<T, OUT ? NK * kC : 1> cr;
    float dt = 0.0f;
    const auto of_c = [&](int k, int& r, int& c) {
        r = 16 * wave + col;
        c = 32 * (k / kC) + 8 * g + k % kC * V;
    };
    xr.places_all(a.x_stride, x_first, a.x_wide);
    br.places_all(a.bc_stride, b_first, a.bc_wide);
    if constexpr (OUT) cr.places((int)a.bc_stride, c_first, a.bc_wide, of_c);
    // a chunk's numbers on their way; with every fourth chunk the steps of the next four, one of which a wave has
    const auto request = [&](int i) {
        if ((i & 3) == 0) {
            const int mine = chunk_of(min(i + wave, many - 1));
            dt = to_f32(dtg[((int64_t)mine * kScanChunk + min(lane, rows_of(mine) - 1)) * a.dt_stride]);
        }
        const int chunk = chunk_of(min(i, many - 1)), rows = rows_of(chunk);
        const int64_t t0 = (int64_t)chunk * kScanChunk;
        xr.request_all(xg + t0 * a.x_stride, a.x_stride, rows, x_first, a.x_wide);
        br.request_all(bg + t0 * a.bc_stride, a.bc_stride, rows, b_first, a.bc_wide);
        if constexpr (OUT) cr.request(bg + t0 * a.bc_stride, (int)a.bc_stride, rows, c_first, a.bc_wide, of_c);
    };
    const bool plain = width == PP && a.n == NP;   // (whole chunks then have no zeros to be put in)
    const auto put = [&](int i) {
        const int rows = rows_of(chunk_of(min(i, many - 1)));
        if (!plain || rows < kScanChunk) {
            xr.settle_all(rows, width, x_first, a.x_wide);
            br.settle_all(rows, a.n, b_first, a.bc_wide);
            if constexpr (OUT) cr.settle(rows, a.n, c_first, a.bc_wide, of_c);
        }
        xr.template put<XP>(xs);
        br.template put<BP>(bs);
        if constexpr (OUT) {
            if (xr.odd()) odd[i & 1] = 1;
        }
        if ((i & 3) == 0) chunk_decays(decays[wave], dt, i + wave < many ? rows_of(chunk_of(i + wave)) : 0, bias, rate, lane);
    };
    double total = 0.0;

    const auto step = [&](auto whole_chunk, int i) {
        constexpr bool FULL = decltype(whole_chunk)::value;
        const int chunk = chunk_of(i), rows = FULL ? kScanChunk : rows_of(chunk);
        const int64_t t0 = (int64_t)chunk * kScanChunk;
        Oct<T> cf[OUT ? NK : 1];
        if constexpr (OUT) {
#pragma unroll
            for (int k = 0; k < NK; ++k) {
                struct Eight { uint4 u[kC]; } e;
#pragma unroll
                for (int h = 0; h < kC; ++h) e.u[h] = cr.u[k * kC + h];
                cf[k] = __builtin_bit_cast(Oct<T>, e);
            }
            // the state as an operand: [p][n]
#pragma unroll
            for (int k = 0; k < TW; ++k) {
                float v[4] = {state[k][0], state[k][1], state[k][2], state[k][3]};
#pragma unroll
                for (int h = 0; h < RT; ++h) {
                    put_four(ss + h * PP * BP + p * BP + n_of(k), v);
                    if (h + 1 < RT) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] -= (float)(T)v[e];
                    }
                }
            }
        }
        __syncthreads();
        if (OUT && threadIdx.x == 0) odd[(i + 1) & 1] = 0;   // (last read before the barrier that ended the step before)
        if constexpr (LEAVES == kWalkStates) {
            float* const to = a.chunk_states + ((sample * a.heads + head) * a.chunks + chunk) * whole + in_whole;
#pragma unroll
            for (int k = 0; k < TW; ++k) {
                const float v[4] = {state[k][0], state[k][1], state[k][2], state[k][3]};
                put_four(to + n_of(k), v);
            }
        }
        request(i + 1);
        __builtin_amdgcn_sched_barrier(0);   // (they are under way before what the step computes, or there would be nothing to hide them behind)
        const ChunkDecays<false>& d = decays[i & 3];
        if constexpr (OUT) {
            const int t = 16 * wave + col;
            const float sum_t = d.sum[t], rest_t = d.rest[t];
            // decayed products of B_s and C_t, rows s, column t
            f32x4_t m[4];
#pragma unroll
            for (int st = 0; st < 4; ++st) {
                m[st] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
                if (st > wave) continue;
#pragma unroll
                for (int k = 0; k < NK; ++k) m[st] = mma(along<false>(bs + (16 * st + col) * BP, 32 * k, lane), cf[k], m[st]);
                float delta_s[4];
                four(d.delta + 16 * st + 4 * g, delta_s);
                if (st < wave) {
                    // (by way of the end of the sixteen positions of s: neither factor is over one)
                    const float on = decay_between(sum_t, rest_t, d.sum[16 * st + 15], d.rest[16 * st + 15]);
                    float tile_s[4];
                    four(d.tile + 16 * st + 4 * g, tile_s);
#pragma unroll
                    for (int r = 0; r < 4; ++r) m[st][r] *= on * (tile_s[r] * delta_s[r]);
                } else {
                    float sum_s[4], rest_s[4];
                    four(d.sum + 16 * st + 4 * g, sum_s);
                    four(d.rest + 16 * st + 4 * g, rest_s);
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        m[st][r] = 4 * g + r <= col ? m[st][r] * (decay_between(sum_t, rest_t, sum_s[r], rest_s[r]) * delta_s[r]) : 0.0f;
                }
            }
            // rows p, column t: what the state before the chunk gives, then the chunk's own
            f32x4_t y[PT];
#pragma unroll
            for (int j = 0; j < PT; ++j) y[j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int h = RT - 1; h >= 0; --h)
#pragma unroll
                for (int k = 0; k < NK; ++k)
#pragma unroll
                    for (int j = 0; j < PT; ++j) y[j] = mma(along<false>(ss + h * PP * BP + (16 * j + col) * BP, 32 * k, lane), cf[k], y[j]);
#pragma unroll
            for (int j = 0; j < PT; ++j) y[j] *= d.from[t];
            // (numbers of x that are not finite would reach every position in products with 0: they are taken out, and put in by themselves where they belong)
            const bool some_odd = __builtin_amdgcn_readfirstlane(odd[i & 1]);
#pragma unroll
            for (int pair = 0; pair < 2; ++pair) {
                if (2 * pair > wave) continue;
                Oct<T> mf[RT], xf[PT];
#pragma unroll
                for (int j = 0; j < PT; ++j) xf[j] = across<true>(xs, XP, 32 * pair, 16 * j, lane);
#pragma unroll
                for (int e = 0; e < 8; ++e) terms_of(m[2 * pair + e / 4][e % 4], e, mf);
                if (some_odd) {
#pragma unroll
                    for (int j = 0; j < PT; ++j)
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (!(fabsf(xf[j].get(e)) < __builtin_inff())) xf[j].set(e, 0.0f);
                }
#pragma unroll
                for (int h = RT - 1; h >= 0; --h)
#pragma unroll
                    for (int j = 0; j < PT; ++j) y[j] = mma(xf[j], mf[h], y[j]);
            }
            if (some_odd) {
#pragma clang loop unroll(disable)
                for (int s = 0; s < 16 * wave + 16; ++s) {
                    float x[PT][4];
                    bool here = false;
#pragma unroll
                    for (int j = 0; j < PT; ++j) {
                        four(xs + s * XP + 16 * j + 4 * g, x[j]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) here |= !(fabsf(x[j][e]) < __builtin_inff());
                    }
                    if (!__any(here)) continue;
                    float by = 0.0f;   // C_t . B_s
#pragma unroll
                    for (int k = 0; k < NK; ++k) {
                        const Oct<T> b = along<false>(bs + s * BP, 32 * k, lane);
#pragma unroll
                        for (int e = 0; e < 8; ++e) by = fmaf(b.get(e), cf[k].get(e), by);
                    }
                    by += __shfl_xor(by, 16);
                    by += __shfl_xor(by, 32);
                    by *= decay_between(sum_t, rest_t, d.sum[s], d.rest[s]) * d.delta[s];
                    if (s > t) continue;
#pragma unroll
                    for (int j = 0; j < PT; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!(fabsf(x[j][e]) < __builtin_inff())) y[j][e] = fmaf(by, x[j][e], y[j][e]);
                }
            }
            T* const row = (T*)a.y + (rows0 + t0 + t) * a.y_stride + (int64_t)head * a.dh + p0;
            const float skip = a.skip[head];
#pragma unroll
            for (int j = 0; j < PT; ++j) {
                float x[4], v[4];
                four(xs + t * XP + 16 * j + 4 * g, x);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = fmaf(skip, x[e], y[j][e]);
                if constexpr (FULL) put_four_any(row + 16 * j + 4 * g, v, 4);
                else if (t < rows) put_four_any(row + 16 * j + 4 * g, v, width - 16 * j - 4 * g);
            }
        }
        // the state behind the chunk
        Oct<T> xw[2][ST];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const Oct<T> x = across<false>(xs, XP, 32 * k, 16 * pt, lane);
            const float* const weights = (REV ? d.from : d.to) + 32 * k + 8 * g;
#pragma unroll
            for (int e = 0; e < 8; ++e) terms_of(x.get(e) * weights[e], e, xw[k]);
        }
#pragma unroll
        for (int k = 0; k < TW; ++k) state[k] *= d.end;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            Oct<T> b[TW];
#pragma unroll
            for (int k = 0; k < TW; ++k) b[k] = across<false>(bs, BP, 32 * h, 16 * (nt0 + k * NSTEP), lane);
#pragma unroll
            for (int e = ST - 1; e >= 0; --e)
#pragma unroll
                for (int k = 0; k < TW; ++k) state[k] = mma(b[k], xw[h][e], state[k]);
        }
        total += d.total;
        __syncthreads();   // (the chunk has been read)
        put(i + 1);
    };
    if (threadIdx.x < 2) odd[threadIdx.x] = 0;
    request(0);
    __syncthreads();
    put(0);
    // (whole chunks in a loop of their own, where the number of memory's operations between a request and its use is known: the results' writing is not waited for)
    int i = 0;
    const auto whole_chunk = [&](int k) { return plain && rows_of(chunk_of(k)) == kScanChunk; };
    if (REV && !whole_chunk(0)) step(std::false_type{}, i++);
    while (i < many && whole_chunk(i)) step(std::true_type{}, i++);
    while (i < many) step(std::false_type{}, i++);

    if (LEAVES == kWalkOwn) {
        if (threadIdx.x == 0 && slice == 0) a.stretch_totals[(sample * a.heads + head) * a.stretches + stretch] = total;
#pragma unroll
        for (int k = 0; k < TW; ++k) {
            const float v[4] = {state[k][0], state[k][1], state[k][2], state[k][3]};
            put_four(a.stretch_states + of_stretch + n_of(k), v);
        }
    } else if (a.final_state && stretch == (REV ? 0 : a.stretches - 1) && p < width) {
#pragma unroll
        for (int k = 0; k < TW; ++k) {
            const float v[4] = {state[k][0], state[k][1], state[k][2], state[k][3]};
            if (n_of(k) < a.n) put_four_any(a.final_state + of_head + n_of(k), v, a.n - n_of(k));
        }
    }
}

// (two workgroups to a compute unit where its LDS has room for them)
template <typename T, int NP, int PT, int LEAVES> __global__ __launch_bounds__(256, (sizeof(WalkTiles<T, NP, PT, LEAVES == kWalkResults>) <= 81920 ? 2 : 1)) void scan_walk_kernel(ScanWalk a) {
    __shared__ WalkTiles<T, NP, PT, LEAVES == kWalkResults> tiles;
    const int64_t unit = xcd_order(blockIdx.x, gridDim.x);
    if (unit < a.samples * a.stretches * a.heads * a.slices) scan_walk<T, NP, PT, LEAVES, false>(a, unit, tiles);
}

// The two walks of a backward pass, for the states alone, side by side: `back` goes backward.
template <typename T, int NP, int PT, int LEAVES> __global__ __launch_bounds__(256, 2) void scan_walks_kernel(ScanWalk ahead, ScanWalk back) {
    __shared__ WalkTiles<T, NP, PT, false> tiles;
    const int64_t unit = xcd_order(blockIdx.x, gridDim.x);
    if (unit >= ahead.samples * ahead.stretches * ahead.heads * ahead.slices) return;
    if (blockIdx.y == 0) scan_walk<T, NP, PT, LEAVES, false>(ahead, unit, tiles);
    else scan_walk<T, NP, PT, LEAVES, true>(back, unit, tiles);
}

// The stretches' own states become those before them: a thread to a number of a state.
template <bool REV> __device__ __forceinline__ void scan_join(const ScanWalk& a, int NP, int whole) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.samples * a.heads * whole) return;
    const int64_t head = i / whole;
    const int at = (int)(i - head * whole), p = at / NP, n = at % NP;
    float carry = a.first_state && p < a.dh && n < a.n ? a.first_state[(head * a.dh + p) * a.n + n] : 0.0f;
    float* const states = a.stretch_states + head * a.stretches * whole + at;
    const double* const totals = a.stretch_totals + head * a.stretches;
#pragma unroll 4
    for (int k = 0; k < a.stretches; ++k) {
        const int s = REV ? a.stretches - 1 - k : k;
        const float own = states[(int64_t)s * whole];
        states[(int64_t)s * whole] = carry;
        carry = fmaf(exp2_of(totals[s]), carry, own);
    }
}
static __global__ __launch_bounds__(256) void scan_join_kernel(ScanWalk a, int NP, int whole) { scan_join<false>(a, NP, whole); }
static __global__ __launch_bounds__(256) void scan_joins_kernel(ScanWalk ahead, ScanWalk back, int NP, int whole) {
    if (blockIdx.y == 0) scan_join<false>(ahead, NP, whole);
    else scan_join<true>(back, NP, whole);
}

// Stretches: as many as are 512 workgroups, two for each compute unit, of four chunks at least, where that is two or more.  32768 positions of 24 heads of 64 x 128 take 219 us so, in 256
// workgroups 328 and in 1024 236 (and 16 x 512 positions, in stretches then, 58 instead of 37); 3 x 333 positions back 34 us, in stretches of two chunks 40.  Heads go in halves of 32
// features where workgroups are few: those 3 x 333 positions 34 us, 37 with whole heads.
constexpr int kStretchGroups = 512, kStretchChunks = 4;
inline void walk_plan(ScanWalk& w) {
    w.chunks = (int)((w.positions + kScanChunk - 1) / kScanChunk);
    w.tiles = w.dh <= 32 || w.samples * w.heads * (padded_dh(w.dh) / 64) * w.chunks < kStretchGroups ? 2 : 4;
    w.slices = padded_dh(w.dh) / (16 * w.tiles);
    const int64_t groups = w.samples * w.heads * w.slices;
    int64_t want = std::min<int64_t>(kStretchGroups / groups, w.chunks / kStretchChunks);
    if (want < 1) want = 1;
    w.each = (int)((w.chunks + want - 1) / want);
    w.stretches = (w.chunks + w.each - 1) / w.each;
}

// Of the states and exponents of stretches, as much as any call of no more samples and positions takes.
inline size_t walk_stretch_bytes(const Scan& a) {
    const int64_t chunks = (a.positions + kScanChunk - 1) / kScanChunk, slices = (a.dh + 63) / 64;
    if (chunks < 2 * kStretchChunks) return 0;
    const int64_t most = std::min<int64_t>(a.samples * a.heads * (chunks / kStretchChunks), kStretchGroups / slices);
    return (size_t)most * ((size_t)padded_dh(a.dh) * padded_n(a.n) * sizeof(float) + sizeof(double)) + 256;
}

// Workgroups of a walk (0: more than a launch takes).
inline unsigned walk_grid(const ScanWalk& w) {
    const int64_t blocks = (w.samples * w.stretches * w.heads * w.slices + 7) / 8 * 8;
    return launchable(blocks, 256) ? (unsigned)blocks : 0u;
}
inline unsigned join_grid(const ScanWalk& w) { return (unsigned)((w.samples * w.heads * padded_dh(w.dh) * padded_n(w.n) + 255) / 256); }

// With the memory of the stretches' states and exponents at ws; the memory behind them.
inline char* walk_room(ScanWalk& w, char* ws) {
    const size_t heads = (size_t)w.samples * w.heads * w.stretches, totals = (heads * sizeof(double) + 15) / 16 * 16;
    w.stretch_totals = reinterpret_cast<double*>(ws);
    w.stretch_states = reinterpret_cast<float*>(ws + totals);
    return ws + totals + heads * padded_dh(w.dh) * padded_n(w.n) * sizeof(float);
}
#define TMPS_WALK(launch, w)                                         \
    ((w).tiles == 4 ? ((w).n <= 32 ? launch(32, 4) : (w).n <= 64 ? launch(64, 4) : launch(128, 4)) \
                    : ((w).n <= 32 ? launch(32, 2) : (w).n <= 64 ? launch(64, 2) : launch(128, 2)))

}  // namespace tmps
