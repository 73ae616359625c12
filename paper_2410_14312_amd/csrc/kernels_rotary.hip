// Rotary positions: pairs (u, v) of a head's features turned by an angle, u' = u cos - v sin, v' = v cos + u sin.  The angle of pair i is the row's position on the
// pair's axis times base^(-j/n), j and n counted over all pairs or over the axis's own.
//
// Angles are formed as turns in 64 bits: a position of a million times a frequency of one is 1.6e5 turns, of which fp32 keeps 1/64 of a turn.  What is left of whole
// turns goes to fp32 (2^-25 of a turn at most), its sine and cosine from there.
#include "../../include/tmps.h"
#include "gemm.hip.h"
#include "kernels.h"
#include "launch.h"

namespace tmps {

// What a launch's threads share.  ratio: base^(-1/n) of the ladder that each axis uses, first: the pair that stands at the ladder's top.
struct Ladders {
    double ratio[3];
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

// x^n by squaring: the relative error of its at most 2 log2(n) products is below 2^-48.
__device__ __forceinline__ double power(double x, int n) {
    double r = 1.0;
    for (; n > 0; n >>= 1) {
        if (n & 1) r *= x;
        x *= x;
    }
    return r;
}

__device__ __forceinline__ int axis_of(const RotaryShape& a, int i) { return i < a.l.end[0] ? 0 : i < a.l.end[1] ? 1 : 2; }

// turns of pair i for a position of one
__device__ __forceinline__ double turns_of(const RotaryShape& a, int i, int axis) { return 0.15915494309189533577 * power(a.l.ratio[axis], i - a.l.first[axis]); }

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

// A thread to a pair (or to a feature behind the pairs) of one head of one row.
template <typename T> __global__ __launch_bounds__(256) void rotary_kernel(const T* x, T* y, RotaryShape a) {
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
        turn(position(a, row, axis) * turns_of(a, i, axis), a.sign, c, s);
        const int at = a.interleaved ? 2 * i : i, to = a.interleaved ? 2 * i + 1 : i + a.pairs;
        const float u = to_f32(xr[at]), v = to_f32(xr[to]);
        yr[at] = from_f32<T>(u * c - v * s);
        yr[to] = from_f32<T>(v * c + u * s);
    }
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
        a.l.ratio[k] = n > 0 ? pow((double)r.base, -1.0 / n) : 1.0;
        a.l.end[k] = at += r.pairs[k];
    }
    const int64_t n = a.rows * a.heads * (a.dh - a.pairs);
    const dim3 grid((unsigned)(n + 255 > (int64_t(1) << 28) ? 1 << 20 : (n + 255) / 256));
    if (dtype == kBF16) return launch_timed(kcEmbedding, rotary_kernel<bf16_t>, grid, dim3(256), 0, s, (const bf16_t*)r.x, (bf16_t*)r.y, a);
    return launch_timed(kcEmbedding, rotary_kernel<float>, grid, dim3(256), 0, s, (const float*)r.x, (float*)r.y, a);
}

}  // namespace tmps
