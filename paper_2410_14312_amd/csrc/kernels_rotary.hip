// Rotary positions: pairs (u, v) of a head's features turned by an angle, u' = u cos - v sin, v' = v cos + u sin.  The angle of pair i is the row's position on the
// pair's axis times base^(-j/n), j and n counted over all pairs or over the axis's own.
//
// Angles are formed as turns in 64 bits: a position of a million times a frequency of one is 1.6e5 turns, of which fp32 keeps 1/64 of a turn.  A frequency is off by less than 2^-50
// of itself, whatever its place on the ladder, so turns are off by 2^-50 of their number.  What is left of whole turns goes to fp32 (2^-25 of a turn at most, which is the larger part up
// to positions of 2^27), its sine and cosine from there.
//
// Bound by memory: the heads are read and written once.  (us of a launch between two time stamps; a copy of as many bytes at the 5.1 TB/s that one of a gigabyte reaches; a thread to a
// pair of one head): 16384 rows of 40 heads of 128 in bf16 67 (66; 238), 8192 of 24 of 64 14.4 (9.9; 31), in fp32 19.0 (19.8).  One row is a launch and one latency, 4.4 us.
#include "../../include/tmps.h"
#include "gemm.hip.h"
#include "kernels.h"
#include "launch.h"
#include "pieces.hip.h"

namespace tmps {

// What a launch's threads share.  step + rest: log2(base) / n of the ladder that each axis uses, the first with 24 bits, so that a pair's multiple of it is exact; first: the pair that
// stands at the ladder's top.
struct Ladders {
    double step[3], rest[3];
    int first[3], end[3];   // end: the first pair behind axis a's
};

struct RotaryShape {
    int64_t x_stride, y_stride, rows, pos_rows;
    int heads, turned, dh, pairs, interleaved;   // heads from `turned` on are copied
    const int32_t* pos;
    int grid_rows, grid_h, grid_w;
    float sign;   // -1: back
    Ladders l;
};

__device__ __forceinline__ int axis_of(const RotaryShape& a, int i) { return i < a.l.end[0] ? 0 : i < a.l.end[1] ? 1 : 2; }

// turns of pair i for a position of one: base^(-j/n) / (2 pi) as 2^(-j step) 2^(-j rest), the second, of an exponent below 2^-17, by its series (its third term is below 2^-54).  A step of
// 2^-52 of the exponential and three of 2^-53 of the products and the constant.  (Powers of base^(-1/n) would be off by its rounding j times over, 2^-44 at 4096 pairs.)
__device__ __forceinline__ double turns_of(const RotaryShape& a, int i, int axis) {
    const int j = i - a.l.first[axis];
    const double r = -0.69314718055994530942 * (j * a.l.rest[axis]);
    return 0.15915494309189533577 * exp2(-j * a.l.step[axis]) * fma(r, fma(0.5, r, 1.0), 1.0);
}

__device__ __forceinline__ int position(const RotaryShape& a, int64_t row, int axis) {
    if (a.pos) return a.pos[row % a.pos_rows * 3 + axis];
    const int r = (int)(row % a.grid_rows), w = r % a.grid_w, h = r / a.grid_w;
    return axis == 2 ? w : axis == 1 ? h % a.grid_h : h / a.grid_h;
}

__device__ __forceinline__ void turn(double turns, float sign, float& c, float& s) {
    const float t = (float)(turns - rint(turns));
    sincospif(2.0f * t, &s, &c);
    s *= sign;
}

// A thread to a pair (or to a feature behind the pairs) of one head of one row: heads of few pairs, and wide ones.  TABLE: frequencies are formed once a workgroup, in LDS.
template <typename T, bool TABLE> __global__ __launch_bounds__(256) void rotary_kernel(const T* x, T* y, RotaryShape a) {
    extern __shared__ double frequency[];
    if constexpr (TABLE) {
        for (int i = threadIdx.x; i < a.pairs; i += 256) frequency[i] = turns_of(a, i, axis_of(a, i));
        __syncthreads();
    }
    const int per_head = a.pairs + (a.dh - 2 * a.pairs);
    const int64_t n = a.rows * a.heads * per_head, step = (int64_t)gridDim.x * 256;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < n; t += step) {
        const int i = (int)(t % per_head);
        const int64_t rest = t / per_head, row = rest / a.heads;
        const int h = (int)(rest % a.heads) * a.dh;
        const T* const xr = x + row * a.x_stride + h;
        T* const yr = y + row * a.y_stride + h;
        if (h >= a.turned * a.dh) {
            yr[i] = xr[i];
            if (i < a.pairs) yr[per_head + i] = xr[per_head + i];
            continue;
        }
        if (i >= a.pairs) {
            yr[a.pairs + i] = xr[a.pairs + i];
            continue;
        }
        const int axis = axis_of(a, i);
        float c, s;
        turn(position(a, row, axis) * (TABLE ? frequency[i] : turns_of(a, i, axis)), a.sign, c, s);
        const int at = a.interleaved ? 2 * i : i, to = a.interleaved ? 2 * i + 1 : i + a.pairs;
        const float u = to_f32(xr[at]), v = to_f32(xr[to]);
        yr[at] = from_f32<T>(u * c - v * s);
        yr[to] = from_f32<T>(v * c + u * s);
    }
}

// A thread to 16 bytes of pairs (split: of both halves) in every row it comes to, for up to H heads, whose turns are the same: an angle's 64-bit product, sine and cosine are some 45
// instructions, a pair's turn in a head 8.  Frequencies are formed once a workgroup, in LDS, and a thread keeps its own.  A last task that would reach beyond the pairs begins
// earlier: it stores the same as the one before it or, where x is y and may already have been turned there, what is its own.  Tasks behind those of the pairs copy the features behind them, 16 bytes each.
template <typename T, int H, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rotary_pieces_kernel(const T* x, T* y, RotaryShape a, int tasks, int turning, int groups, int rows_each) {
    constexpr int V = kPiece<T>, NP = INTERLEAVED ? V / 2 : V;
    extern __shared__ double frequency[];
    for (int i = threadIdx.x; i < a.pairs; i += blockDim.x) frequency[i] = turns_of(a, i, axis_of(a, i));
    __syncthreads();
    const int task = threadIdx.x % tasks, group = threadIdx.x / tasks % groups, r = threadIdx.x / tasks / groups;
    if (r >= rows_each) return;
    const bool turns = task < turning;
    const int i0 = turns ? min(task * NP, a.pairs - NP) : 0;
    const int others = turns && x == y ? task * NP - i0 : 0;   // pairs that are the task's before it
    const int behind = 2 * a.pairs + (task - turning) * V;   // of a copying task
    double f[NP];
    bool on0[NP], on1[NP];
#pragma unroll
    for (int e = 0; e < NP; ++e) {
        f[e] = frequency[i0 + e];
        on0[e] = i0 + e < a.l.end[0];
        on1[e] = i0 + e < a.l.end[1];
    }
    const int64_t step = (int64_t)gridDim.x * rows_each;
    int64_t row = (int64_t)blockIdx.x * rows_each + r;
    // (the row's place among the positions, kept up by addition: a 64-bit remainder in each row is some hundred instructions)
    const int64_t places = a.pos ? a.pos_rows : a.grid_rows;
    int64_t place = row % places;
    const int64_t place_step = step % places;
    for (; row < a.rows; row += step) {
        const T* const xr = x + row * a.x_stride;
        T* const yr = y + row * a.y_stride;
        int p[3];
        if (a.pos) {
#pragma unroll
            for (int k = 0; k < 3; ++k) p[k] = a.pos[place * 3 + k];
        } else {
            const unsigned at = (unsigned)place, h = at / (unsigned)a.grid_w;
            p[2] = at % (unsigned)a.grid_w;
            p[1] = h % (unsigned)a.grid_h;
            p[0] = h / (unsigned)a.grid_h;
        }
        place += place_step;
        if (place >= places) place -= places;
        if (!turns) {
            const int n = a.dh - behind;
            if (n >= V) {
                for (int h0 = group; h0 < a.heads; h0 += H * groups) {
                    uint4 u[H];
#pragma unroll
                    for (int k = 0; k < H; ++k)
                        if (h0 + k * groups < a.heads) u[k] = load16_any(xr + (h0 + k * groups) * a.dh + behind);
#pragma unroll
                    for (int k = 0; k < H; ++k)
                        if (h0 + k * groups < a.heads) store16_any(yr + (h0 + k * groups) * a.dh + behind, u[k]);
                }
            } else {
                for (int h = group; h < a.heads; h += groups)
                    for (int e = 0; e < n; ++e) yr[h * a.dh + behind + e] = xr[h * a.dh + behind + e];
            }
            continue;
        }
        float c[NP], s[NP];
        bool ready = false;
        for (int h0 = group; h0 < a.heads; h0 += H * groups) {
            uint4 ru[H], rv[INTERLEAVED ? 1 : H];
#pragma unroll
            for (int k = 0; k < H; ++k) {
                const int h = h0 + k * groups;
                if (h < a.heads) {
                    const T* const at = xr + h * a.dh;
                    ru[k] = load16_any(at + (INTERLEAVED ? 2 * i0 : i0));
                    if constexpr (!INTERLEAVED) rv[k] = load16_any(at + a.pairs + i0);
                }
            }
            if (!ready) {
                ready = true;
#pragma unroll
                for (int e = 0; e < NP; ++e) turn((on0[e] ? p[0] : on1[e] ? p[1] : p[2]) * f[e], a.sign, c[e], s[e]);
            }
#pragma unroll
            for (int k = 0; k < H; ++k) {
                const int h = h0 + k * groups;
                if (h >= a.heads) continue;
                T* const at = yr + h * a.dh;
                float u[V], v[V];
                unpack(ru[k], u);
                if constexpr (!INTERLEAVED) unpack(rv[k], v);
                if (h < a.turned) {
#pragma unroll
                    for (int e = 0; e < NP; ++e) {
                        float& first = u[INTERLEAVED ? 2 * e : e];
                        float& second = INTERLEAVED ? u[INTERLEAVED ? 2 * e + 1 : 0] : v[e];
                        const float w = fmaf(first, c[e], -second * s[e]);
                        second = fmaf(second, c[e], first * s[e]);
                        first = w;
                    }
                }
                const uint4 pu = pack(u);
                uint4 pv;
                if constexpr (!INTERLEAVED) pv = pack(v);
                if (others == 0) {
                    store16_any(at + (INTERLEAVED ? 2 * i0 : i0), pu);
                    if constexpr (!INTERLEAVED) store16_any(at + a.pairs + i0, pv);
                } else {
                    struct Features { T v[V]; } fu = __builtin_bit_cast(Features, pu), fv;
                    if constexpr (!INTERLEAVED) fv = __builtin_bit_cast(Features, pv);
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        if (e < (INTERLEAVED ? 2 * others : others)) continue;
                        at[(INTERLEAVED ? 2 * i0 : i0) + e] = fu.v[e];
                        if constexpr (!INTERLEAVED) at[a.pairs + i0 + e] = fv.v[e];
                    }
                }
            }
        }
    }
}

// Workgroups of a launch at most: four to a compute unit, each with its frequencies formed once.  (8192 rows of 24 heads of 64 in bf16 a twelfth more with twice as many.)
constexpr int kRotaryGroups = 1024;

template <typename T, bool INTERLEAVED> static hipError_t rotary_pieces(const Rotary& r, const RotaryShape& a, hipStream_t s) {
    constexpr int V = kPiece<T>, NP = INTERLEAVED ? V / 2 : V;
    const int turning = (a.pairs + NP - 1) / NP, tasks = turning + (r.x == r.y ? 0 : (a.dh - 2 * a.pairs + V - 1) / V);
    // Heads to a thread: up to four, where that leaves the device enough threads; then the head groups with which whole rows fill whole waves best.
    const int64_t pieces = a.rows * tasks * a.heads;
    const int H = pieces >= (int64_t(1) << 20) ? 4 : pieces >= (int64_t(1) << 18) ? 2 : 1;
    const int most = 256 / tasks < a.heads ? 256 / tasks : a.heads, least = (a.heads + H - 1) / H < most ? (a.heads + H - 1) / H : most;
    int groups = least, best = 0;
    for (int g = least; g <= most && g < 2 * least; ++g) {
        const int used = 256 / (tasks * g) * tasks * g, full = used * 1024 / ((used + 63) / 64 * 64);
        if (full > best + 64) best = full, groups = g;
    }
    const int rows_each = 256 / (tasks * groups), threads = (rows_each * tasks * groups + 63) / 64 * 64;
    const int64_t blocks = (a.rows + rows_each - 1) / rows_each;
    auto kern = H == 4 ? rotary_pieces_kernel<T, 4, INTERLEAVED> : H == 2 ? rotary_pieces_kernel<T, 2, INTERLEAVED> : rotary_pieces_kernel<T, 1, INTERLEAVED>;
    return launch_timed(kcEmbedding, kern, dim3((unsigned)(blocks < kRotaryGroups ? blocks : kRotaryGroups)), dim3(threads), a.pairs * 8, s, (const T*)r.x, (T*)r.y, a, tasks, turning, groups, rows_each);
}

hipError_t rotary(int dtype, const Rotary& r, hipStream_t s) {
    if (r.rows <= 0) return hipSuccess;
    RotaryShape a;
    a.x_stride = r.x_stride; a.y_stride = r.y_stride; a.rows = r.rows; a.pos_rows = r.pos_rows;
    a.heads = r.heads + (r.x == r.y ? 0 : r.copied); a.turned = r.heads; a.dh = r.dh; a.pairs = r.pairs[0] + r.pairs[1] + r.pairs[2]; a.interleaved = r.flags & TMPS_FLAG_INTERLEAVED;
    a.pos = r.pos; a.grid_rows = r.grid_rows; a.grid_h = r.grid_h; a.grid_w = r.grid_w;
    a.sign = r.inverse ? -1.0f : 1.0f;
    int at = 0;
    for (int k = 0; k < 3; ++k) {
        const bool own = r.flags & TMPS_FLAG_OWN_LADDERS;
        const int n = own ? r.pairs[k] : a.pairs;
        a.l.first[k] = own ? at : 0;
        const long double step = n > 0 ? log2l((long double)r.base) / n : 0.0L;
        a.l.step[k] = (double)(float)step;
        a.l.rest[k] = (double)(step - (long double)a.l.step[k]);
        a.l.end[k] = at += r.pairs[k];
    }
    const int most = dtype == kBF16 ? 8 : 4;
    if (a.pairs >= (a.interleaved ? most / 2 : most) && a.dh <= 1016) {   // (tasks that 256 threads hold)
        if (dtype == kBF16) return a.interleaved ? rotary_pieces<bf16_t, true>(r, a, s) : rotary_pieces<bf16_t, false>(r, a, s);
        return a.interleaved ? rotary_pieces<float, true>(r, a, s) : rotary_pieces<float, false>(r, a, s);
    }
    const int64_t blocks = (a.rows * a.heads * (a.dh - a.pairs) + 255) / 256;
    // A table of more pairs than a workgroup has threads would cost each of them several frequencies for its one.  With a table, as many workgroups as the device holds, so that each
    // forms it once for many rows: 8192 rows of 24 heads of 64, 4 pairs, bf16 59 us, 65 with a workgroup to 256 features, 72 with a frequency formed for every turn.
    const bool table = a.pairs <= 256;
    const int64_t cap = table ? 2048 : 1 << 20;
    const dim3 grid((unsigned)(blocks < cap ? blocks : cap));
    const size_t lds = table ? (size_t)a.pairs * 8 : 0;
    if (dtype == kBF16) return launch_timed(kcEmbedding, table ? rotary_kernel<bf16_t, true> : rotary_kernel<bf16_t, false>, grid, dim3(256), lds, s, (const bf16_t*)r.x, (bf16_t*)r.y, a);
    return launch_timed(kcEmbedding, table ? rotary_kernel<float, true> : rotary_kernel<float, false>, grid, dim3(256), lds, s, (const float*)r.x, (float*)r.y, a);
}

}  // namespace tmps
