// Launchers of the operators of blocks that mix positions by a recurrence: a short convolution, a selective state space, group norm, clipping of gradients.
#pragma once
#include <stddef.h>

#include "kernels.h"

namespace tmps {

// Whether a launch takes so many workgroups (its threads are counted in 32 bits).
inline bool launchable(int64_t workgroups, int threads) { return workgroups < (int64_t(1) << 32) / threads; }

// Causal convolution of `taps` taps along the positions of each sample, channels apart, z = bias + sum_j weight[c][j] u[t - taps + 1 + j][c], and with silu
// y = z / (1 + exp(-z)).  u: x's rows (x_stride elements apart), before them those of tail ([samples, taps - 1, channels]; null: zeros).  tail_out (may be null, or tail for one
// position): the last taps - 1 inputs.
constexpr int kConvMaxTaps = 8;
struct ShortConv {
    const void* x;
    int64_t x_stride;
    const float *weight, *bias;   // bias may be null
    const void* tail;
    void* y;
    int64_t y_stride;
    void* tail_out;
    int64_t samples, positions;
    int channels, taps;
    bool silu;
};
hipError_t short_conv_forward(int dtype, const ShortConv& a, hipStream_t s);
// Its gradients from dy and, of tail_out, dtail (may be null): dx, dtail_in (may be null) and dparams: [channels][taps] of the weights, then, with a bias, [channels].
struct ShortConvBackward {
    const void* dy;
    int64_t dy_stride;
    const void* x;
    int64_t x_stride;
    const float *weight, *bias;
    const void *tail, *dtail;
    void* dx;
    int64_t dx_stride;
    void* dtail_in;
    float* dparams;
    int64_t samples, positions;
    int channels, taps;
    bool silu;
};
hipError_t short_conv_backward(int dtype, const ShortConvBackward& a, float* part, hipStream_t s);
size_t short_conv_part_elems(int64_t samples, int64_t positions, int channels, int taps);

// Selective state space: per sample and head (dh features p, n features of a state, heads / groups neighbouring heads with the same B and C)
//   delta = softplus(dt + dt_bias),  S_t = exp(-delta exp(a_log)) S_{t-1} + delta x_t B_t',  y_t = S_t C_t + skip x_t
// over rows [x (heads dh) | B (groups n) | C (groups n)].  state, state_out: [samples, heads, dh, n] (null: zeros; not wanted; one may be the other).
constexpr int kScanMaxState = 128;
constexpr int kScanSteps = 8;   // up to so many positions go one after the other
struct Scan {
    const void* x;
    int64_t x_stride;
    const void* dt;
    int64_t dt_stride;
    const float *a_log, *skip, *dt_bias;
    const float* state;
    void* y;
    int64_t y_stride;
    float* state_out;
    int64_t samples, positions;
    int heads, dh, groups, n;
};
size_t scan_workspace_bytes(const Scan& a);
hipError_t scan_forward(int dtype, const Scan& a, void* ws, hipStream_t s);
// Its gradients from dy and, of state_out, dstate (may be null): dx (rows as x's), ddt, dparams: [3][heads] of a_log, skip, dt_bias; dstate_in (may be null).
struct ScanBackward {
    Scan f;   // y and state_out are not looked at
    const void* dy;
    int64_t dy_stride;
    const float* dstate;
    void* dx;
    int64_t dx_stride;
    void* ddt;
    int64_t ddt_stride;
    float* dparams;
    float* dstate_in;
};
size_t scan_backward_workspace_bytes(int dtype, const Scan& a);
hipError_t scan_backward(int dtype, const ScanBackward& a, void* ws, hipStream_t s);

// Group norm over the positions and channels / groups neighbouring channels of a sample, and the activation behind it: xhat = (x - mean) / sqrt(var + 1e-5), with rms
// x / sqrt(mean(x^2) + 1e-5); y = act(gain xhat + shift) (shift may be null).  stats: (mean or 0, 1/std) of each sample's groups.
enum { kNormActNone = 0, kNormActRelu = 1, kNormActGelu = 2, kNormActSilu = 3 };
constexpr int kGroupNormMaxChannels = 1 << 16;
struct GroupNorm {
    const void* x;
    const float *gain, *shift;
    void* y;
    float* stats;
    int64_t samples, positions;
    int channels, groups, act;
    bool rms;
};
bool group_norm_fits(int dtype, int64_t samples, int64_t positions, int channels, int groups);
size_t group_norm_workspace_bytes(int dtype, int64_t samples, int64_t positions, int channels, int groups, bool backward);
hipError_t group_norm_forward(int dtype, const GroupNorm& a, void* ws, hipStream_t s);
// Its gradients: dx and dparams: [channels] of gain, then [channels] of shift (also where there is none).
struct GroupNormBackward {
    const void *dy, *x;
    const float *stats, *gain, *shift;
    void* dx;
    float* dparams;
    int64_t samples, positions;
    int channels, groups, act;
    bool rms;
};
hipError_t group_norm_backward(int dtype, const GroupNormBackward& a, void* ws, hipStream_t s);

// norm = the 2-norm of all arrays together, in 64 bits; out = in times limit / norm where that is less than one and the norm finite as a float.  out may be in, or null in all: the norm alone.
struct ClipArray {
    const void* in;
    void* out;
    int64_t n;
    int dtype;
};
size_t clip_workspace_bytes(const ClipArray* list, int n);
hipError_t clip_gradients(const ClipArray* list, int n, float limit, float* norm, void* ws, hipStream_t s);

}  // namespace tmps
