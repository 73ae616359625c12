// Stand-ins for the kernel launchers (paper_2410_14312_amd/csrc/kernels.h) that compute, on fp32 host memory and at once: dense layers without activation, residual joins, layer
// normalisation, norm joins, rotary positions.  The other launchers are those of kernel_stubs.cpp.  What no kernel promises is not kept here either: a dense layer's
// input gradient is written column by column while its operands are still read, and comes before the weight gradient where the two share a launch.
#include "arithmetic.h"

#define dense_forward stub_dense_forward
#define dense_dgrad stub_dense_dgrad
#define dense_wgrad stub_dense_wgrad
#define dense_backward stub_dense_backward
#define dense_wgrad_groups stub_dense_wgrad_groups
#define dense_wgrad_group stub_dense_wgrad_group
#define resadd_forward stub_resadd_forward
#define layernorm_forward stub_layernorm_forward
#define layernorm_backward stub_layernorm_backward
#include "kernel_stubs.cpp"
#undef dense_forward
#undef dense_dgrad
#undef dense_wgrad
#undef dense_backward
#undef dense_wgrad_groups
#undef dense_wgrad_group
#undef resadd_forward
#undef layernorm_forward
#undef layernorm_backward

#include <math.h>

#include <vector>

#include "../../include/tmps.h"

Arithmetic arithmetic;

namespace tmps {

hipError_t dense_forward(int, const void* x_, const void* w_, const float* bias, void* y_, int B, int Din, int Dout, int, int, const void* res_, void* again, float*, hipStream_t) {
    const float *x = (const float*)x_, *w = (const float*)w_, *res = (const float*)res_;
    float* y = (float*)y_;
    for (int b = 0; b < B; ++b)
        for (int o = 0; o < Dout; ++o) {
            float s = bias ? bias[o] : 0.0f;
            for (int i = 0; i < Din; ++i) s += x[(size_t)b * Din + i] * w[(size_t)o * Din + i];
            s += res ? res[(size_t)b * Dout + o] : 0.0f;
            y[(size_t)b * Dout + o] = s;
            if (again) ((float*)again)[(size_t)b * Dout + o] = s;
        }
    return hipSuccess;
}

hipError_t dense_dgrad(int, const void* dy_, const void* w_, void* dx_, const void* mask, int, const void* add_, int B, int Din, int Dout, float*, hipStream_t) {
    if (mask) return hipErrorInvalidValue;
    const float *dy = (const float*)dy_, *w = (const float*)w_, *add = (const float*)add_;
    float* dx = (float*)dx_;
    for (int i = 0; i < Din; ++i)
        for (int b = 0; b < B; ++b) {
            float s = 0.0f;
            for (int o = 0; o < Dout; ++o) s += dy[(size_t)b * Dout + o] * w[(size_t)o * Din + i];
            dx[(size_t)b * Din + i] = s + (add ? add[(size_t)b * Din + i] : 0.0f);
        }
    return hipSuccess;
}

hipError_t dense_wgrad(int, const void* dy_, const void* x_, float* gw, int B, int Din, int Dout, const Partials&, hipStream_t) {
    const float *dy = (const float*)dy_, *x = (const float*)x_;
    for (int o = 0; o < Dout; ++o) {
        float sum = 0.0f;
        for (int b = 0; b < B; ++b) sum += dy[(size_t)b * Dout + o];
        gw[(size_t)Dout * Din + o] = sum;
        for (int i = 0; i < Din; ++i) {
            float s = 0.0f;
            for (int b = 0; b < B; ++b) s += dy[(size_t)b * Dout + o] * x[(size_t)b * Din + i];
            gw[(size_t)o * Din + i] = s;
        }
    }
    return hipSuccess;
}

hipError_t dense_backward(int t, const void* dy, const void* x, const void* w, float* gw, void* dx, const void* mask, int mode, const void* add, int B, int Din, int Dout, float* ws,
                          const Partials& part, hipStream_t s) {
    const hipError_t e = dense_dgrad(t, dy, w, dx, mask, mode, add, B, Din, Dout, ws, s);
    return e != hipSuccess ? e : dense_wgrad(t, dy, x, gw, B, Din, Dout, part, s);
}

bool dense_wgrad_groups(int, int64_t, int, int) { return arithmetic.groups; }

hipError_t dense_wgrad_group(int t, const DenseWgradJob* jobs, int n, int64_t rows, float*, int64_t, hipStream_t s) {
    for (int k = 0; k < n; ++k) (void)dense_wgrad(t, jobs[k].dy, jobs[k].x, jobs[k].gw, (int)rows, jobs[k].Din, jobs[k].Dout, Partials(nullptr), s);
    return hipSuccess;
}

hipError_t resadd_forward(int, const void* a, const void* b, void* y, int64_t n, int relu, hipStream_t) {
    for (int64_t i = 0; i < n; ++i) {
        const float v = ((const float*)a)[i] + ((const float*)b)[i];
        ((float*)y)[i] = relu && v < 0.0f ? 0.0f : v;
    }
    return hipSuccess;
}

// (mean or 0, 1/std) of a row
static void stats_of(const float* v, int D, bool rms, float* st) {
    float m = 0.0f, q = 0.0f;
    for (int d = 0; d < D && !rms; ++d) m += v[d] / (float)D;
    for (int d = 0; d < D; ++d) q += (v[d] - m) * (v[d] - m) / (float)D;
    st[0] = m;
    st[1] = 1.0f / sqrtf(q + 1e-5f);
}
// the gradient through a row's norm, t that of its result
static std::vector<float> through_norm(const float* t, const float* v, int D, bool rms, const float* st) {
    float mean = 0.0f, along = 0.0f;
    for (int d = 0; d < D; ++d) {
        if (!rms) mean += t[d] / (float)D;
        along += t[d] * (v[d] - st[0]) * st[1] / (float)D;
    }
    std::vector<float> g(D);
    for (int d = 0; d < D; ++d) g[d] = st[1] * (t[d] - mean - (v[d] - st[0]) * st[1] * along);
    return g;
}

hipError_t layernorm_forward(int, const void* x_, const float* gamma, const float* beta, void* y_, float* stats, int64_t rows, int D, float, hipStream_t) {
    for (int64_t r = 0; r < rows; ++r) {
        const float* x = (const float*)x_ + r * D;
        stats_of(x, D, false, stats + 2 * r);
        for (int d = 0; d < D; ++d) ((float*)y_)[r * D + d] = (x[d] - stats[2 * r]) * stats[2 * r + 1] * gamma[d] + beta[d];
    }
    return hipSuccess;
}
hipError_t layernorm_backward(int, const void* dy_, const void* x_, const float* stats, const float* gamma, const void* add_, void* dx_, float* grads, const Partials&, int64_t rows, int D,
                              hipStream_t) {
    std::vector<float> sums(2 * D), t(D);
    for (int64_t r = 0; r < rows; ++r) {
        const float *dy = (const float*)dy_ + r * D, *x = (const float*)x_ + r * D, *add = add_ ? (const float*)add_ + r * D : nullptr;
        for (int d = 0; d < D; ++d) {
            sums[d] += dy[d] * (x[d] - stats[2 * r]) * stats[2 * r + 1];
            sums[D + d] += dy[d];
            t[d] = dy[d] * gamma[d];
        }
        const std::vector<float> g = through_norm(t.data(), x, D, false, stats + 2 * r);
        for (int d = 0; d < D && dx_; ++d) ((float*)dx_)[r * D + d] = g[d] + (add ? add[d] : 0.0f);
    }
    for (int k = 0; k < 2 * D; ++k) grads[k] = sums[k];
    return hipSuccess;
}

size_t norm_join_part_elems(int64_t, int D) { return 2 * (size_t)D; }

hipError_t norm_join_forward(int, const NormJoin& j, hipStream_t) {
    const int D = j.D, wide = j.gate ? 2 * D : D;
    for (int64_t r = 0; r < j.rows; ++r) {
        float* y = (float*)j.y + r * D;
        if (j.x) {
            const float *f = (const float*)j.x + r * wide, *res = (const float*)j.r + r * D;
            float* st = j.stats + r * j.stats_stride;
            stats_of(f, D, j.rms, st);
            for (int d = 0; d < D; ++d) y[d] = j.scale[d] * res[d] + (j.gate ? 1.0f / (1.0f + expf(-f[D + d])) : 1.0f) * j.gain[d] * (f[d] - st[0]) * st[1];
        }
        if (j.u) {
            float* st = j.pre_stats + r * j.stats_stride;
            stats_of(y, D, j.rms, st);
            for (int d = 0; d < D; ++d) ((float*)j.u)[r * D + d] = (y[d] - st[0]) * st[1] * j.pre_gain[d] + (j.pre_shift ? j.pre_shift[d] : 0.0f);
        }
    }
    return hipSuccess;
}

hipError_t norm_join_backward(int, const NormJoinBackward& j, const Partials&, const Partials&, hipStream_t) {
    const int D = j.D, wide = j.gate ? 2 * D : D;
    std::vector<float> sums(2 * D), pre(2 * D), t(D), dh(D);
    for (int64_t r = 0; r < j.rows; ++r) {
        const float* dy = j.dy ? (const float*)j.dy + r * D : nullptr;
        for (int d = 0; d < D; ++d) dh[d] = dy ? dy[d] : 0.0f;
        if (j.du) {
            const float *du = (const float*)j.du + r * D, *y = (const float*)j.y + r * D, *st = j.pre_stats + r * j.stats_stride;
            for (int d = 0; d < D; ++d) {
                pre[d] += du[d] * (y[d] - st[0]) * st[1];
                pre[D + d] += du[d];
                t[d] = du[d] * j.pre_gain[d];
            }
            const std::vector<float> g = through_norm(t.data(), y, D, j.rms, st);
            for (int d = 0; d < D; ++d) dh[d] += g[d];
        }
        if (!j.x) {
            for (int d = 0; d < D && j.dr; ++d) ((float*)j.dr)[r * D + d] = dh[d];
            continue;
        }
        const float *f = (const float*)j.x + r * wide, *res = (const float*)j.r + r * D, *st = j.stats + r * j.stats_stride, *add = j.add ? (const float*)j.add + r * D : nullptr;
        std::vector<float> da(D);
        for (int d = 0; d < D; ++d) {
            const float fh = (f[d] - st[0]) * st[1], g = j.gate ? 1.0f / (1.0f + expf(-f[D + d])) : 1.0f;
            sums[d] += dh[d] * g * fh;
            sums[D + d] += dh[d] * res[d];
            da[d] = dh[d] * j.gain[d] * fh * g * (1.0f - g);
            t[d] = dh[d] * g * j.gain[d];
        }
        const std::vector<float> df = through_norm(t.data(), f, D, j.rms, st);
        for (int d = 0; d < D && j.dr; ++d) ((float*)j.dr)[r * D + d] = j.scale[d] * dh[d] + (add ? add[d] : 0.0f);
        for (int d = 0; d < D && j.dx; ++d) {
            ((float*)j.dx)[r * wide + d] = df[d];
            if (j.gate) ((float*)j.dx)[r * wide + D + d] = da[d];
        }
    }
    for (int k = 0; k < 2 * D && j.x; ++k) j.dgain_dscale[k] = sums[k];
    for (int k = 0; k < (j.rms ? D : 2 * D) && j.du; ++k) j.dpre[k] = pre[k];
    return hipSuccess;
}

hipError_t rotary(int, const Rotary& r, hipStream_t) {
    const int pairs = r.pairs[0] + r.pairs[1] + r.pairs[2];
    const bool interleaved = r.flags & TMPS_FLAG_INTERLEAVED, own = r.flags & TMPS_FLAG_OWN_LADDERS;
    for (int64_t k = 0; k < r.rows; ++k) {
        const int place = (int)(k % r.grid_rows), across = r.grid_w * r.grid_h, at[3] = {place / across, place / r.grid_w % r.grid_h, place % r.grid_w};
        for (int h = 0; h < r.heads + (r.x == r.y ? 0 : r.copied); ++h) {
            const float* x = (const float*)r.x + k * r.x_stride + h * r.dh;
            float* y = (float*)r.y + k * r.y_stride + h * r.dh;
            for (int i = 0; i < pairs; ++i) {
                const int axis = i < r.pairs[0] ? 0 : i < r.pairs[0] + r.pairs[1] ? 1 : 2, first = axis == 0 ? 0 : axis == 1 ? r.pairs[0] : r.pairs[0] + r.pairs[1];
                const double angle = at[axis] * pow((double)r.base, own ? -(double)(i - first) / r.pairs[axis] : -(double)i / pairs) * (r.inverse ? -1.0 : 1.0);
                const double c = h < r.heads ? cos(angle) : 1.0, s = h < r.heads ? sin(angle) : 0.0;
                const int a = interleaved ? 2 * i : i, b = interleaved ? 2 * i + 1 : i + pairs;
                const double u = x[a], v = x[b];
                y[a] = (float)(u * c - v * s);
                y[b] = (float)(v * c + u * s);
            }
            for (int i = 2 * pairs; i < r.dh; ++i) y[i] = x[i];
        }
    }
    return hipSuccess;
}

size_t distill_workspace_elems(int64_t, int64_t, int) { return 0; }
hipError_t distill(int, const Distill&, float*, hipStream_t) { return hipErrorInvalidValue; }
int check_distill(int64_t, int64_t, float, float) { return TMPS_EUNSUPPORTED; }

}  // namespace tmps
