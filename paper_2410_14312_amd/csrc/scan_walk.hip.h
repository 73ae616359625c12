// The walk over the chunks of a head's positions with its state in the accumulators: forward with the results y, forward or backward for the states of the chunks alone.
#pragma once
#include <algorithm>

#include "launch.h"
#include "scan.hip.h"

namespace tmps {

// The walk's operands: "x" and "b" are x and B going forward, dy and C going backward, where the state is the gradient of the state behind a chunk.
struct ScanWalk {
    const void *x, *b, *c, *dt;
    int64_t x_stride, bc_stride, dt_stride;
    const float *a_log, *skip, *dt_bias;
    const float* first_state;    // before the first chunk of the walk: [samples, heads, dh, n] (null: zeros)
    void* y;
    int64_t y_stride;
    float* final_state;          // behind the last chunk (null: not wanted)
    float* chunk_states;         // before each chunk of the walk: [samples, heads, chunks, dh, n] (null: not wanted)
    int64_t samples, positions;
    int heads, dh, groups, n;
    int chunks, stretches, each, slices;   // chunks of a sample, stretches of them and the chunks of one, slices of a head's features
    float* stretch_states;       // [samples, heads, stretches, dh, n]: before each stretch, or with `own` left by each
    double* stretch_totals;
    bool own;                    // each stretch from nothing, for its own state and exponent alone
};

template <typename T> ScanWalk walk_of(const Scan& a) {
    ScanWalk w;
    w.x = a.x; w.b = (const T*)a.x + (int64_t)a.heads * a.dh; w.c = (const T*)w.b + (int64_t)a.groups * a.n;
    w.dt = a.dt; w.x_stride = w.bc_stride = a.x_stride; w.dt_stride = a.dt_stride;
    w.a_log = a.a_log; w.skip = a.skip; w.dt_bias = a.dt_bias; w.first_state = a.state;
    w.y = nullptr; w.y_stride = 0; w.final_state = nullptr; w.chunk_states = nullptr;
    w.samples = a.samples; w.positions = a.positions; w.heads = a.heads; w.dh = a.dh; w.groups = a.groups; w.n = a.n;
    w.stretch_states = nullptr; w.stretch_totals = nullptr; w.own = false;
    return w;
}

template <typename T> constexpr int kStateTerms = sizeof(T) == 2 ? 3 : 1;    // of a state's increments: results in fp32
template <typename T> constexpr int kResultTerms = sizeof(T) == 2 ? 2 : 1;   // of states and decayed products on their way to results of the type

template <typename T, int NP, int PT, bool OUT, bool REV> __global__ __launch_bounds__(256) void scan_walk_kernel(ScanWalk a) {
    constexpr int V = kPiece<T>, PP = PT * 16, XP = PP + V, BP = NP + V, NT = NP / 16, TW = NT * PT / 4, NK = NP / 32;
    constexpr int RT = kResultTerms<T>, ST = kStateTerms<T>;
    __shared__ __attribute__((aligned(16))) T xs[kScanChunk * XP];
    __shared__ __attribute__((aligned(16))) T bs[kScanChunk * BP];
    __shared__ __attribute__((aligned(16))) T ss[OUT ? RT * PP * BP : 8];
    __shared__ __attribute__((aligned(16))) ChunkDecays decays[4];
    __shared__ int odd[2];
    const int64_t units = a.samples * a.stretches * a.heads * a.slices;
    int64_t unit = xcd_order(blockIdx.x, gridDim.x);
    if (unit >= units) return;
    const int slice = (int)(unit % a.slices);
    unit /= a.slices;
    const int head = (int)(unit % a.heads);
    unit /= a.heads;
    const int stretch = (int)(unit % a.stretches);
    const int64_t sample = unit / a.stretches;
    const int group = head / (a.heads / a.groups);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, col = lane & 15;
    const int p0 = slice * 64, width = min(64, a.dh - p0);
    const double rate = exp((double)a.a_log[head]) * kLog2eD;
    const float bias = a.dt_bias[head];

    const int64_t rows0 = sample * a.positions;
    const T* const xg = (const T*)a.x + rows0 * a.x_stride + (int64_t)head * a.dh + p0;
    const T* const bg = (const T*)a.b + rows0 * a.bc_stride + (int64_t)group * a.n;
    const T* const cg = (const T*)a.c + rows0 * a.bc_stride + (int64_t)group * a.n;
    const T* const dtg = (const T*)a.dt + rows0 * a.dt_stride + head;

    // this wave's tiles of the state: 16 features p, n tiles a few apart; rows n, columns p
    const int pt = wave % PT, nt0 = wave / PT;
    constexpr int NSTEP = 4 / PT;
    const int p = pt * 16 + col;   // in the slice
    f32x4_t state[TW];
    const int64_t of_head = (sample * a.heads + head) * a.dh * a.n + (int64_t)(p0 + p) * a.n;
    const int64_t of_stretch = ((sample * a.heads + head) * a.stretches + stretch) * a.dh * a.n + (int64_t)(p0 + p) * a.n;
    const float* const from = a.own ? nullptr : a.stretches > 1 ? a.stretch_states + of_stretch : a.first_state ? a.first_state + of_head : nullptr;
    const auto n_of = [&](int k) { return (nt0 + k * NSTEP) * 16 + 4 * g; };
#pragma unroll
    for (int k = 0; k < TW; ++k) {
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (from && p < width && n_of(k) < a.n) four_any(from + n_of(k), v, a.n - n_of(k));
        state[k] = f32x4_t{v[0], v[1], v[2], v[3]};
    }

    const int first = stretch * a.each, many = min(a.each, a.chunks - first);
    const auto chunk_of = [&](int i) { return REV ? first + many - 1 - i : first + i; };
    const auto rows_of = [&](int chunk) { return (int)min<int64_t>(kScanChunk, a.positions - (int64_t)chunk * kScanChunk); };
    ChunkRows<T, PP, 256> xr;
    ChunkRows<T, NP, 256> br;
    Oct<T> cf[OUT ? NK : 1];
    const auto request = [&](int chunk) {
        const int64_t t0 = (int64_t)chunk * kScanChunk;
        const int rows = rows_of(chunk);
        xr.request(xg + t0 * a.x_stride, a.x_stride, rows, width);
        br.request(bg + t0 * a.bc_stride, a.bc_stride, rows, a.n);
    };
    double total = 0.0;
    if (threadIdx.x < 2) odd[threadIdx.x] = 0;
    request(chunk_of(0));
    for (int i = 0; i < many; ++i) {
        const int chunk = chunk_of(i), rows = rows_of(chunk);
        const int64_t t0 = (int64_t)chunk * kScanChunk;
        __syncthreads();   // (the chunk before has been read)
        if ((i & 3) == 0 && i + wave < many) {
            const int mine = chunk_of(i + wave);
            chunk_decays(decays[wave], dtg + (int64_t)mine * kScanChunk * a.dt_stride, a.dt_stride, rows_of(mine), bias, rate, lane);
        }
        xr.template put<XP>(xs);
        br.template put<BP>(bs);
        if constexpr (OUT) {
            if (xr.odd()) odd[i & 1] = 1;
            if (threadIdx.x == 0) odd[(i + 1) & 1] = 0;   // (last read before the barrier above)
            const int t = 16 * wave + col;
#pragma unroll
            for (int k = 0; k < NK; ++k) {
                struct Eight { uint4 u[sizeof(T) / 2]; } e;
#pragma unroll
                for (int h = 0; h < (int)sizeof(T) / 2; ++h)
                    e.u[h] = t < rows ? piece_until(cg + (t0 + t) * a.bc_stride, 32 * k + 8 * g + h * V, a.n) : make_uint4(0, 0, 0, 0);
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
                        for (int e = 0; e < 4; ++e) {
                            const float rest = v[e] - (float)(T)v[e];
                            v[e] = fabsf(rest) < 3.4e38f ? rest : 0.0f;
                        }
                    }
                }
            }
        }
        __syncthreads();
        if (i + 1 < many) request(chunk_of(i + 1));
        const ChunkDecays& d = decays[i & 3];
        if (a.chunk_states && p < width) {
            float* const to = a.chunk_states + (((sample * a.heads + head) * a.chunks + chunk) * a.dh + p0 + p) * a.n;
#pragma unroll
            for (int k = 0; k < TW; ++k) {
                const float v[4] = {state[k][0], state[k][1], state[k][2], state[k][3]};
                if (n_of(k) < a.n) put_four_any(to + n_of(k), v, a.n - n_of(k));
            }
        }
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
                float sum_s[4], rest_s[4], delta_s[4];
                four(d.sum + 16 * st + 4 * g, sum_s);
                four(d.rest + 16 * st + 4 * g, rest_s);
                four(d.delta + 16 * st + 4 * g, delta_s);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    m[st][r] = 16 * st + 4 * g + r <= t ? m[st][r] * (decay_between(sum_t, rest_t, sum_s[r], rest_s[r]) * delta_s[r]) : 0.0f;
            }
            // rows p, column t: what the state before the chunk gives, then the chunk's own
            f32x4_t y[PT];
#pragma unroll
            for (int j = 0; j < PT; ++j) {
                y[j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int h = RT - 1; h >= 0; --h)
#pragma unroll
                    for (int k = 0; k < NK; ++k) y[j] = mma(along<false>(ss + h * PP * BP + (16 * j + col) * BP, 32 * k, lane), cf[k], y[j]);
                y[j] *= d.from[t];
            }
            // (numbers of x that are not finite would reach every position in products with 0: they are taken out, and put in by themselves where they belong)
            const bool some_odd = odd[i & 1];
#pragma unroll
            for (int pair = 0; pair < 2; ++pair) {
                if (2 * pair > wave) continue;
                Oct<T> mf[RT];
#pragma unroll
                for (int e = 0; e < 8; ++e) terms_of(m[2 * pair + e / 4][e % 4], e, mf);
#pragma unroll
                for (int j = 0; j < PT; ++j) {
                    Oct<T> xf = across<true>(xs, XP, 32 * pair, 16 * j, lane);
                    if (some_odd) {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (!(fabsf(xf.get(e)) < __builtin_inff())) xf.set(e, 0.0f);
                    }
#pragma unroll
                    for (int h = RT - 1; h >= 0; --h) y[j] = mma(xf, mf[h], y[j]);
                }
            }
            if (some_odd) {
#pragma unroll
                for (int st = 0; st < 4; ++st)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        for (int h = 0; h < 4; ++h) {
                            const int s = 16 * st + 4 * h + r;
                            const float by = __shfl(m[st][r], 16 * h + col);
                            if (s > t) continue;
#pragma unroll
                            for (int j = 0; j < PT; ++j)
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const float x = to_f32(xs[s * XP + 16 * j + 4 * g + e]);
                                    if (!(fabsf(x) < __builtin_inff())) y[j][e] = fmaf(by, x, y[j][e]);
                                }
                        }
            }
            if (t < rows) {
                T* const row = (T*)a.y + (rows0 + t0 + t) * a.y_stride + (int64_t)head * a.dh + p0;
                const float skip = a.skip[head];
#pragma unroll
                for (int j = 0; j < PT; ++j) {
                    float x[4], v[4];
                    four(xs + t * XP + 16 * j + 4 * g, x);
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = fmaf(skip, x[e], y[j][e]);
                    if (16 * j + 4 * g < width) put_four_any(row + 16 * j + 4 * g, v, width - 16 * j - 4 * g);
                }
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
        for (int k = 0; k < TW; ++k) {
            state[k] *= d.end;
            const int nt = nt0 + k * NSTEP;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const Oct<T> b = across<false>(bs, BP, 32 * h, 16 * nt, lane);
#pragma unroll
                for (int e = ST - 1; e >= 0; --e) state[k] = mma(b, xw[h][e], state[k]);
            }
        }
        total += d.total;
    }
    if (a.own && threadIdx.x == 0 && slice == 0) a.stretch_totals[(sample * a.heads + head) * a.stretches + stretch] = total;
    float* const to = a.own ? a.stretch_states + of_stretch : a.final_state && stretch == (REV ? 0 : a.stretches - 1) ? a.final_state + of_head : nullptr;
    if (to && p < width) {
#pragma unroll
        for (int k = 0; k < TW; ++k) {
            const float v[4] = {state[k][0], state[k][1], state[k][2], state[k][3]};
            if (n_of(k) < a.n) put_four_any(to + n_of(k), v, a.n - n_of(k));
        }
    }
}

// The stretches' own states become those before them: a thread to a number of a state.
template <bool REV> __global__ __launch_bounds__(256) void scan_join_kernel(ScanWalk a) {
    const int64_t size = (int64_t)a.dh * a.n, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.samples * a.heads * size) return;
    const int64_t head = i / size, at = i % size;
    float carry = a.first_state ? a.first_state[i] : 0.0f;
    float* const states = a.stretch_states + head * a.stretches * size + at;
    const double* const totals = a.stretch_totals + head * a.stretches;
    for (int k = 0; k < a.stretches; ++k) {
        const int s = REV ? a.stretches - 1 - k : k;
        const float own = states[s * size];
        states[s * size] = carry;
        carry = fmaf(__builtin_amdgcn_exp2f((float)totals[s]), carry, own);
    }
}

// Stretches: as many as give the chip 512 workgroups, of four chunks at least.
constexpr int kStretchGroups = 512, kStretchChunks = 4;
inline void walk_plan(ScanWalk& w) {
    w.chunks = (int)((w.positions + kScanChunk - 1) / kScanChunk);
    w.slices = (w.dh + 63) / 64;
    const int64_t groups = w.samples * w.heads * w.slices;
    int64_t want = std::min<int64_t>((kStretchGroups + groups - 1) / groups, w.chunks / kStretchChunks);
    if (want < 1) want = 1;
    w.each = (int)((w.chunks + want - 1) / want);
    w.stretches = (w.chunks + w.each - 1) / w.each;
}

// Of the states and exponents of stretches, as much as any call of no more samples and positions takes.
inline size_t walk_stretch_bytes(const Scan& a) {
    const int64_t chunks = (a.positions + kScanChunk - 1) / kScanChunk, slices = (a.dh + 63) / 64;
    if (chunks < 2 * kStretchChunks) return 0;
    // samples x heads x stretches is at most the workgroups wanted / slices and as many again as there are samples and heads
    const int64_t most = std::min<int64_t>(a.samples * a.heads * (chunks / kStretchChunks), kStretchGroups / slices + a.samples * a.heads);
    return (size_t)most * ((size_t)a.dh * a.n * sizeof(float) + sizeof(double)) + 256;
}

template <typename T, bool OUT, bool REV> static hipError_t walk_launch(const ScanWalk& w, hipStream_t s) {
    const int64_t units = w.samples * w.stretches * w.heads * w.slices, blocks = (units + 7) / 8 * 8;
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    const dim3 grid((unsigned)blocks), block(256);
    const int kc = OUT ? kcAttnFwd : kcAttnBwd;
    if (w.dh > 32) {
        if (w.n <= 32) return launch_timed(kc, scan_walk_kernel<T, 32, 4, OUT, REV>, grid, block, 0, s, w);
        if (w.n <= 64) return launch_timed(kc, scan_walk_kernel<T, 64, 4, OUT, REV>, grid, block, 0, s, w);
        return launch_timed(kc, scan_walk_kernel<T, 128, 4, OUT, REV>, grid, block, 0, s, w);
    }
    if (w.n <= 32) return launch_timed(kc, scan_walk_kernel<T, 32, 2, OUT, REV>, grid, block, 0, s, w);
    if (w.n <= 64) return launch_timed(kc, scan_walk_kernel<T, 64, 2, OUT, REV>, grid, block, 0, s, w);
    return launch_timed(kc, scan_walk_kernel<T, 128, 2, OUT, REV>, grid, block, 0, s, w);
}

// A walk, in stretches where its plan has them.  ws: walk_stretch_bytes.
template <typename T, bool OUT, bool REV> static hipError_t walk_stretches(ScanWalk w, void* ws, hipStream_t s) {
    walk_plan(w);
    if (w.stretches > 1) {
        const size_t totals = (size_t)w.samples * w.heads * w.stretches * sizeof(double);
        w.stretch_totals = static_cast<double*>(ws);
        w.stretch_states = reinterpret_cast<float*>(static_cast<char*>(ws) + (totals + 15) / 16 * 16);
        ScanWalk own = w;
        own.own = true;
        own.chunk_states = nullptr;
        hipError_t e = walk_launch<T, false, REV>(own, s);
        if (e != hipSuccess) return e;
        const int64_t numbers = w.samples * w.heads * w.dh * w.n;
        if ((numbers + 255) / 256 > INT32_MAX) return hipErrorInvalidValue;
        e = launch_timed(OUT ? kcAttnFwd : kcAttnBwd, scan_join_kernel<REV>, dim3((unsigned)((numbers + 255) / 256)), dim3(256), 0, s, w);
        if (e != hipSuccess) return e;
    }
    return walk_launch<T, OUT, REV>(w, s);
}

}  // namespace tmps
