// Operators of blocks that mix positions by a recurrence, as calls of their own over the caller's memory: a short convolution, a selective state space, group norm, clipping of
// gradients.  Arguments are checked here.
#include <math.h>

#include <algorithm>
#include <initializer_list>
#include <new>
#include <vector>

#include "common.h"
#include "mixer.h"
#include "operands.h"

using namespace tmps;

namespace {

// Rows of `width` elements, `stride` elements apart: whether they are apart, and few enough for 63 bits of bytes.
int check_rows(const char* name, int64_t rows, int64_t width, int64_t stride) {
    if (rows > 1 && stride < width) return fail(TMPS_ESHAPE, "%s: rows of %lld elements overlap", name, (long long)width);
    if (rows > kMaxElems / width || (rows > 1 && stride > kMaxElems / rows)) return fail(TMPS_EUNSUPPORTED, "%s: too many rows", name);
    return TMPS_OK;
}
Range rows_at(const void* p, int64_t rows, int64_t width, int64_t stride, size_t esz) {
    if (rows == 1) return Range{p, (size_t)width * esz};
    return Range{p, (size_t)((rows - 1) * stride + width) * esz, (size_t)stride * esz, (size_t)width * esz};
}

int check_samples(int dtype, int64_t samples, int64_t positions) {
    if (!known(dtype)) return fail(TMPS_EINVAL, "unknown dtype %d", dtype);
    if (samples < 0 || positions < 1) return fail(TMPS_EINVAL, "positions must be positive, samples not negative");
    if (positions > INT32_MAX || samples > kMaxElems / positions) return fail(TMPS_EUNSUPPORTED, "too many positions");
    return TMPS_OK;
}

// Whether all are on whole elements.
bool whole(size_t bytes, std::initializer_list<const void*> all) {
    for (const void* p : all)
        if (!aligned(p, bytes)) return false;
    return true;
}

int room(const void* workspace, size_t bytes, size_t need) {
    if (need && (!workspace || bytes < need)) return fail(TMPS_ECAP, "the workspace holds %zu bytes, %zu are needed", workspace ? bytes : (size_t)0, need);
    if (need && !aligned(workspace, 16)) return fail(TMPS_ESHAPE, "the workspace is not on 16 bytes");
    return TMPS_OK;
}

// ------------------------------------------------------------------------------------------------ short convolution
int check_conv(int dtype, int flags, int64_t samples, int64_t positions, int channels, int taps) {
    const int rc = check_samples(dtype, samples, positions);
    if (rc != TMPS_OK) return rc;
    if (flags & ~TMPS_FLAG_SILU) return fail(TMPS_EINVAL, "unknown flags %d", flags);
    if (channels < 1 || taps < 1) return fail(TMPS_EINVAL, "channels and taps must be positive");
    if (taps > kConvMaxTaps) return fail(TMPS_EUNSUPPORTED, "more than %d taps", kConvMaxTaps);
    if (channels > (1 << 24)) return fail(TMPS_EUNSUPPORTED, "more than 2^24 channels");
    // (a launch has a workgroup for every 64 positions of 256 channels)
    const int64_t groups = (samples * ((positions + 15) / 16) + 3) / 4;
    if (!launchable(groups, 256) || !launchable(groups * ((channels + 255) / 256), 256)) return fail(TMPS_EUNSUPPORTED, "too many positions");
    return TMPS_OK;
}

}  // namespace

extern "C" int tmps_short_conv_forward(int dtype, int flags, int64_t samples, int64_t positions, int channels, int taps, const void* x, int64_t x_stride,
                                       const float* weight, const float* bias, const void* tail, void* y, int64_t y_stride, void* tail_out, void* hip_stream) {
    int rc = check_conv(dtype, flags, samples, positions, channels, taps);
    if (rc != TMPS_OK) return rc;
    if (samples == 0) return TMPS_OK;
    if (!x || !weight || !y) return fail(TMPS_EINVAL, "an argument is null");
    const int64_t rows = samples * positions;
    if ((rc = check_rows("x", rows, channels, x_stride)) != TMPS_OK || (rc = check_rows("y", rows, channels, y_stride)) != TMPS_OK) return rc;
    const size_t esz = act_bytes(dtype), tails = (size_t)samples * (taps - 1) * channels * esz;
    if (!whole(esz, {x, tail, y, tail_out}) || !whole(4, {weight, bias})) return fail(TMPS_ESHAPE, "a pointer is not on a whole element");
    const Range operands[] = {rows_at(x, rows, channels, x_stride, esz), {weight, (size_t)channels * taps * 4}, {bias, (size_t)channels * 4}, {tail, tails}};
    // (a position's thread has read the tail before it writes it; of several positions others may read it later)
    const Range results[] = {{tail_out, tails}, rows_at(y, rows, channels, y_stride, esz)};
    if (overlaps(operands, results, positions == 1 ? tail : nullptr)) return fail(TMPS_EINVAL, "a result overlaps an operand or another result (tail_out may be tail for one position)");
    ShortConv c;
    c.x = x; c.x_stride = x_stride; c.weight = weight; c.bias = bias; c.tail = tail; c.y = y; c.y_stride = y_stride; c.tail_out = tail_out;
    c.samples = samples; c.positions = positions; c.channels = channels; c.taps = taps; c.silu = flags & TMPS_FLAG_SILU;
    TMPS_HIP(short_conv_forward(dtype, c, (hipStream_t)hip_stream));
    return TMPS_OK;
}

extern "C" size_t tmps_short_conv_workspace(int64_t samples, int64_t positions, int channels, int taps) {
    if (samples < 1 || positions < 1 || positions > INT32_MAX || samples > kMaxElems / positions || channels < 1 || channels > (1 << 24) || taps < 1 || taps > kConvMaxTaps) return 0;
    return short_conv_part_elems(samples, positions, channels, taps) * sizeof(float);
}

extern "C" int tmps_short_conv_backward(int dtype, int flags, int64_t samples, int64_t positions, int channels, int taps, const void* dy, int64_t dy_stride, const void* x,
                                        int64_t x_stride, const float* weight, const float* bias, const void* tail, const void* dtail, void* dx, int64_t dx_stride,
                                        void* dtail_in, float* dparams, void* workspace, size_t workspace_bytes, void* hip_stream) {
    int rc = check_conv(dtype, flags, samples, positions, channels, taps);
    if (rc != TMPS_OK) return rc;
    if (samples == 0) return fail(TMPS_EUNSUPPORTED, "the gradients of no samples");
    if (!dy || !x || !weight || !dx || !dparams) return fail(TMPS_EINVAL, "an argument is null");
    const int64_t rows = samples * positions;
    if ((rc = check_rows("x", rows, channels, x_stride)) != TMPS_OK || (rc = check_rows("dy", rows, channels, dy_stride)) != TMPS_OK ||
        (rc = check_rows("dx", rows, channels, dx_stride)) != TMPS_OK)
        return rc;
    const size_t esz = act_bytes(dtype), tails = (size_t)samples * (taps - 1) * channels * esz, need = short_conv_part_elems(samples, positions, channels, taps) * sizeof(float);
    if (!whole(esz, {dy, x, tail, dtail, dx, dtail_in}) || !whole(4, {weight, bias, dparams})) return fail(TMPS_ESHAPE, "a pointer is not on a whole element");
    if ((rc = room(workspace, workspace_bytes, need)) != TMPS_OK) return rc;
    const Range operands[] = {rows_at(dy, rows, channels, dy_stride, esz), rows_at(x, rows, channels, x_stride, esz), {weight, (size_t)channels * taps * 4},
                              {bias, (size_t)channels * 4}, {tail, tails}, {dtail, tails}};
    const Range results[] = {rows_at(dx, rows, channels, dx_stride, esz), {dtail_in, tails}, {dparams, (size_t)channels * (taps + (bias ? 1 : 0)) * 4}, {workspace, need}};
    if (overlaps(operands, results)) return fail(TMPS_EINVAL, "a result or the workspace overlaps an operand or another result");
    ShortConvBackward c;
    c.dy = dy; c.dy_stride = dy_stride; c.x = x; c.x_stride = x_stride; c.weight = weight; c.bias = bias; c.tail = tail; c.dtail = dtail; c.dx = dx; c.dx_stride = dx_stride;
    c.dtail_in = dtail_in; c.dparams = dparams; c.samples = samples; c.positions = positions; c.channels = channels; c.taps = taps; c.silu = flags & TMPS_FLAG_SILU;
    try {
        TMPS_HIP(short_conv_backward(dtype, c, static_cast<float*>(workspace), (hipStream_t)hip_stream));
    } catch (const std::bad_alloc&) {
        return fail(TMPS_EINVAL, "out of host memory");
    }
    return TMPS_OK;
}

// ------------------------------------------------------------------------------------------------ selective state space
static int check_scan(int dtype, const tmps_scan_desc* desc, int64_t samples, int64_t positions) {
    const int rc = check_samples(dtype, samples, positions);
    if (rc != TMPS_OK) return rc;
    if (!desc) return fail(TMPS_EINVAL, "desc is null");
    if (desc->heads < 1 || desc->dh < 1 || desc->groups < 1 || desc->n < 1) return fail(TMPS_EINVAL, "heads, features, groups and state features must be positive");
    if (desc->heads % desc->groups) return fail(TMPS_ESHAPE, "%d heads in %d groups", desc->heads, desc->groups);
    if (desc->n > kScanMaxState) return fail(TMPS_EUNSUPPORTED, "states of more than %d features", kScanMaxState);
    if ((int64_t)desc->heads * desc->dh + 2 * (int64_t)desc->groups * desc->n > (1 << 24)) return fail(TMPS_EUNSUPPORTED, "rows of more than 2^24 features");
    const int64_t head_numbers = (int64_t)desc->heads * desc->dh * desc->n;   // (of a sample's states)
    if (samples > ((int64_t)INT32_MAX - 1) * 256 / head_numbers) return fail(TMPS_EUNSUPPORTED, "too many samples");
    // (numbers of the chunks' states, whole tiles of them: their places are 64-bit numbers)
    if ((double)samples * (double)((positions + 63) / 64) * desc->heads * (desc->dh + 63.0) * 128.0 > 0x1p50) return fail(TMPS_EUNSUPPORTED, "too many positions");
    return TMPS_OK;
}

// (rows are read 16 bytes at a time)
static int check_room(int dtype, const Scan& s, bool backward) {
    const int64_t least = 16 / (int64_t)act_bytes(dtype), inner = (int64_t)s.heads * s.dh;
    if ((backward || s.positions > kScanSteps) && (backward ? inner : inner + 2 * (int64_t)s.groups * s.n) < least)
        return fail(TMPS_EUNSUPPORTED, "rows of fewer than %d features", (int)least);
    return TMPS_OK;
}

// (places in a chunk of rows are numbers of 32 bits)
static int check_strides(int64_t rows, std::initializer_list<int64_t> strides) {
    for (int64_t s : strides)
        if (rows > 1 && s > (1 << 24)) return fail(TMPS_EUNSUPPORTED, "rows more than 2^24 elements apart");
    return TMPS_OK;
}

static Scan scan_of(const tmps_scan_desc* d, int64_t samples, int64_t positions) {
    Scan s = {};
    s.samples = samples; s.positions = positions; s.heads = d->heads; s.dh = d->dh; s.groups = d->groups; s.n = d->n;
    return s;
}

extern "C" size_t tmps_scan_workspace(const tmps_scan_desc* desc, int64_t samples, int64_t positions) {
    if (samples < 1 || check_scan(TMPS_F32, desc, samples, positions) != TMPS_OK) return 0;
    return scan_workspace_bytes(scan_of(desc, samples, positions));
}

extern "C" int tmps_scan_forward(int dtype, const tmps_scan_desc* desc, int64_t samples, int64_t positions, const void* x, int64_t x_stride, const void* dt, int64_t dt_stride,
                                 const float* a_log, const float* skip, const float* dt_bias, const float* state, void* y, int64_t y_stride, float* state_out,
                                 void* workspace, size_t workspace_bytes, void* hip_stream) {
    int rc = check_scan(dtype, desc, samples, positions);
    if (rc != TMPS_OK) return rc;
    if (samples == 0) return TMPS_OK;
    if (!x || !dt || !a_log || !skip || !dt_bias || !y) return fail(TMPS_EINVAL, "an argument is null");
    Scan s = scan_of(desc, samples, positions);
    const int64_t rows = samples * positions, wide = (int64_t)s.heads * s.dh + 2 * (int64_t)s.groups * s.n, inner = (int64_t)s.heads * s.dh;
    if ((rc = check_rows("x", rows, wide, x_stride)) != TMPS_OK || (rc = check_rows("dt", rows, s.heads, dt_stride)) != TMPS_OK ||
        (rc = check_rows("y", rows, inner, y_stride)) != TMPS_OK || (rc = check_strides(rows, {x_stride, dt_stride, y_stride})) != TMPS_OK || (rc = check_room(dtype, s, false)) != TMPS_OK)
        return rc;
    const size_t esz = act_bytes(dtype), heads = (size_t)s.heads * 4, states = (size_t)samples * inner * s.n * 4, need = scan_workspace_bytes(s);
    if (!whole(esz, {x, dt, y}) || !whole(4, {a_log, skip, dt_bias, state, state_out})) return fail(TMPS_ESHAPE, "a pointer is not on a whole element");
    if ((rc = room(workspace, workspace_bytes, need)) != TMPS_OK) return rc;
    const Range operands[] = {rows_at(x, rows, wide, x_stride, esz), rows_at(dt, rows, s.heads, dt_stride, esz), {a_log, heads}, {skip, heads}, {dt_bias, heads}, {state, states}};
    const Range results[] = {{state_out, states}, rows_at(y, rows, inner, y_stride, esz), {need ? workspace : nullptr, need}};
    if (overlaps(operands, results, state)) return fail(TMPS_EINVAL, "a result or the workspace overlaps an operand or another result (state_out may be state)");
    s.x = x; s.x_stride = x_stride; s.dt = dt; s.dt_stride = dt_stride; s.a_log = a_log; s.skip = skip; s.dt_bias = dt_bias; s.state = state;
    s.y = y; s.y_stride = y_stride; s.state_out = state_out;
    TMPS_HIP(scan_forward(dtype, s, workspace, (hipStream_t)hip_stream));
    return TMPS_OK;
}

extern "C" size_t tmps_scan_backward_workspace(int dtype, const tmps_scan_desc* desc, int64_t samples, int64_t positions) {
    if (samples < 1 || check_scan(dtype, desc, samples, positions) != TMPS_OK) return 0;
    return scan_backward_workspace_bytes(dtype, scan_of(desc, samples, positions));
}

extern "C" int tmps_scan_backward(int dtype, const tmps_scan_desc* desc, int64_t samples, int64_t positions, const void* dy, int64_t dy_stride, const float* dstate, const void* x,
                                  int64_t x_stride, const void* dt, int64_t dt_stride, const float* a_log, const float* skip, const float* dt_bias, const float* state, void* dx,
                                  int64_t dx_stride, void* ddt, int64_t ddt_stride, float* dparams, float* dstate_in, void* workspace, size_t workspace_bytes,
                                  void* hip_stream) {
    int rc = check_scan(dtype, desc, samples, positions);
    if (rc != TMPS_OK) return rc;
    if (samples == 0) return fail(TMPS_EUNSUPPORTED, "the gradients of no samples");
    if (!dy || !x || !dt || !a_log || !skip || !dt_bias || !dx || !ddt || !dparams) return fail(TMPS_EINVAL, "an argument is null");
    Scan s = scan_of(desc, samples, positions);
    const int64_t rows = samples * positions, wide = (int64_t)s.heads * s.dh + 2 * (int64_t)s.groups * s.n, inner = (int64_t)s.heads * s.dh;
    if ((rc = check_rows("x", rows, wide, x_stride)) != TMPS_OK || (rc = check_rows("dt", rows, s.heads, dt_stride)) != TMPS_OK ||
        (rc = check_rows("dy", rows, inner, dy_stride)) != TMPS_OK || (rc = check_rows("dx", rows, wide, dx_stride)) != TMPS_OK ||
        (rc = check_rows("ddt", rows, s.heads, ddt_stride)) != TMPS_OK || (rc = check_strides(rows, {x_stride, dt_stride, dy_stride, dx_stride, ddt_stride})) != TMPS_OK || (rc = check_room(dtype, s, true)) != TMPS_OK)
        return rc;
    const size_t esz = act_bytes(dtype), heads = (size_t)s.heads * 4, states = (size_t)samples * inner * s.n * 4, need = scan_backward_workspace_bytes(dtype, s);
    if (!whole(esz, {dy, x, dt, dx, ddt}) || !whole(4, {dstate, a_log, skip, dt_bias, state, dparams, dstate_in})) return fail(TMPS_ESHAPE, "a pointer is not on a whole element");
    if ((rc = room(workspace, workspace_bytes, need)) != TMPS_OK) return rc;
    const Range operands[] = {rows_at(dy, rows, inner, dy_stride, esz), {dstate, states}, rows_at(x, rows, wide, x_stride, esz), rows_at(dt, rows, s.heads, dt_stride, esz),
                              {a_log, heads}, {skip, heads}, {dt_bias, heads}, {state, states}};
    const Range results[] = {{dstate_in, states}, rows_at(dx, rows, wide, dx_stride, esz), rows_at(ddt, rows, s.heads, ddt_stride, esz), {dparams, 3 * heads}, {workspace, need}};
    if (overlaps(operands, results)) return fail(TMPS_EINVAL, "a result or the workspace overlaps an operand or another result");
    s.x = x; s.x_stride = x_stride; s.dt = dt; s.dt_stride = dt_stride; s.a_log = a_log; s.skip = skip; s.dt_bias = dt_bias; s.state = state;
    ScanBackward b;
    b.f = s; b.dy = dy; b.dy_stride = dy_stride; b.dstate = dstate; b.dx = dx; b.dx_stride = dx_stride; b.ddt = ddt; b.ddt_stride = ddt_stride; b.dparams = dparams;
    b.dstate_in = dstate_in;
    try {
        TMPS_HIP(scan_backward(dtype, b, workspace, (hipStream_t)hip_stream));
    } catch (const std::bad_alloc&) {
        return fail(TMPS_EINVAL, "out of host memory");
    }
    return TMPS_OK;
}

// ------------------------------------------------------------------------------------------------ group norm
static int act_of(int flags) { return flags & TMPS_FLAG_RELU ? kNormActRelu : flags & TMPS_FLAG_GELU ? kNormActGelu : flags & TMPS_FLAG_SILU ? kNormActSilu : kNormActNone; }

static int check_group_norm(int dtype, int flags, int64_t samples, int64_t positions, int channels, int groups) {
    const int rc = check_samples(dtype, samples, positions);
    if (rc != TMPS_OK) return rc;
    if (flags & ~(TMPS_FLAG_RELU | TMPS_FLAG_GELU | TMPS_FLAG_SILU | TMPS_FLAG_RMS)) return fail(TMPS_EINVAL, "unknown flags %d", flags);
    const int acts = flags & (TMPS_FLAG_RELU | TMPS_FLAG_GELU | TMPS_FLAG_SILU);
    if (acts & (acts - 1)) return fail(TMPS_EINVAL, "ReLU, GELU and SiLU are exclusive");
    if (channels < 1 || groups < 1) return fail(TMPS_EINVAL, "channels and groups must be positive");
    if (channels % groups) return fail(TMPS_ESHAPE, "%d channels in %d groups", channels, groups);
    if (channels > kGroupNormMaxChannels) return fail(TMPS_EUNSUPPORTED, "more than %d channels", kGroupNormMaxChannels);
    if (samples * positions > kMaxElems / channels || !group_norm_fits(dtype, samples, positions, channels, groups)) return fail(TMPS_EUNSUPPORTED, "too many rows");
    return TMPS_OK;
}

extern "C" size_t tmps_group_norm_workspace(int dtype, int64_t samples, int64_t positions, int channels, int groups, int backward) {
    if (samples < 1 || check_group_norm(dtype, 0, samples, positions, channels, groups) != TMPS_OK) return 0;
    return group_norm_workspace_bytes(dtype, samples, positions, channels, groups, backward != 0);
}

extern "C" int tmps_group_norm_forward(int dtype, int flags, int64_t samples, int64_t positions, int channels, int groups, const void* x, const float* gain, const float* shift,
                                       void* y, float* stats, void* workspace, size_t workspace_bytes, void* hip_stream) {
    int rc = check_group_norm(dtype, flags, samples, positions, channels, groups);
    if (rc != TMPS_OK) return rc;
    if (samples == 0) return TMPS_OK;
    if (!x || !gain || !y || !stats) return fail(TMPS_EINVAL, "an argument is null");
    const size_t esz = act_bytes(dtype), n = (size_t)samples * positions * channels * esz, v = (size_t)channels * 4;
    const size_t need = group_norm_workspace_bytes(dtype, samples, positions, channels, groups, false);
    if (!whole(esz, {x, y}) || !whole(4, {gain, shift, stats})) return fail(TMPS_ESHAPE, "a pointer is not on a whole element");
    if ((rc = room(workspace, workspace_bytes, need)) != TMPS_OK) return rc;
    const Range operands[] = {{x, n}, {gain, v}, {shift, v}};
    const Range results[] = {{y, n}, {stats, (size_t)samples * groups * 8}, {need ? workspace : nullptr, need}};
    if (overlaps(operands, results)) return fail(TMPS_EINVAL, "a result or the workspace overlaps an operand or another result");
    GroupNorm g;
    g.x = x; g.gain = gain; g.shift = shift; g.y = y; g.stats = stats; g.samples = samples; g.positions = positions; g.channels = channels; g.groups = groups;
    g.act = act_of(flags); g.rms = flags & TMPS_FLAG_RMS;
    TMPS_HIP(group_norm_forward(dtype, g, workspace, (hipStream_t)hip_stream));
    return TMPS_OK;
}

extern "C" int tmps_group_norm_backward(int dtype, int flags, int64_t samples, int64_t positions, int channels, int groups, const void* dy, const void* x, const float* stats,
                                        const float* gain, const float* shift, void* dx, float* dparams, void* workspace, size_t workspace_bytes, void* hip_stream) {
    int rc = check_group_norm(dtype, flags, samples, positions, channels, groups);
    if (rc != TMPS_OK) return rc;
    if (samples == 0) return fail(TMPS_EUNSUPPORTED, "the gradients of no samples");
    if (!dy || !x || !stats || !gain || !dx || !dparams) return fail(TMPS_EINVAL, "an argument is null");
    const size_t esz = act_bytes(dtype), n = (size_t)samples * positions * channels * esz, v = (size_t)channels * 4;
    const size_t need = group_norm_workspace_bytes(dtype, samples, positions, channels, groups, true);
    if (!whole(esz, {dy, x, dx}) || !whole(4, {stats, gain, shift, dparams})) return fail(TMPS_ESHAPE, "a pointer is not on a whole element");
    if ((rc = room(workspace, workspace_bytes, need)) != TMPS_OK) return rc;
    const Range operands[] = {{dy, n}, {x, n}, {stats, (size_t)samples * groups * 8}, {gain, v}, {shift, v}};
    const Range results[] = {{dx, n}, {dparams, 2 * v}, {workspace, need}};
    if (overlaps(operands, results)) return fail(TMPS_EINVAL, "a result or the workspace overlaps an operand or another result");
    GroupNormBackward g;
    g.dy = dy; g.x = x; g.stats = stats; g.gain = gain; g.shift = shift; g.dx = dx; g.dparams = dparams; g.samples = samples; g.positions = positions; g.channels = channels;
    g.groups = groups; g.act = act_of(flags); g.rms = flags & TMPS_FLAG_RMS;
    try {
        TMPS_HIP(group_norm_backward(dtype, g, workspace, (hipStream_t)hip_stream));
    } catch (const std::bad_alloc&) {
        return fail(TMPS_EINVAL, "out of host memory");
    }
    return TMPS_OK;
}

// ------------------------------------------------------------------------------------------------ clipping
static int check_clip(const tmps_array* arrays, int n) {
    if (n < 0 || (n > 0 && !arrays)) return fail(TMPS_EINVAL, "arrays is null, or a negative number of them");
    for (int i = 0; i < n; ++i) {
        const tmps_array& a = arrays[i];
        if (!known(a.dtype)) return fail(TMPS_EINVAL, "array %d: unknown dtype %d", i, a.dtype);
        if (a.n < 0 || (a.n > 0 && !a.data)) return fail(TMPS_EINVAL, "array %d is null, or has a negative number of elements", i);
        if (a.n > (int64_t(1) << 40)) return fail(TMPS_EUNSUPPORTED, "array %d has more than 2^40 elements", i);
        if (!aligned(a.data, act_bytes(a.dtype)) || !aligned(a.out, act_bytes(a.dtype))) return fail(TMPS_ESHAPE, "array %d is not on a whole element", i);
    }
    return TMPS_OK;
}

// The arrays that have elements.
static std::vector<ClipArray> clip_list(const tmps_array* arrays, int n) {
    std::vector<ClipArray> list;
    list.reserve(n);
    for (int i = 0; i < n; ++i)
        if (arrays[i].n) list.push_back(ClipArray{arrays[i].data, arrays[i].out, arrays[i].n, arrays[i].dtype});
    return list;
}

extern "C" size_t tmps_clip_workspace(const tmps_array* arrays, int n) {
    if (check_clip(arrays, n) != TMPS_OK) return 0;
    try {
        const std::vector<ClipArray> list = clip_list(arrays, n);
        return clip_workspace_bytes(list.data(), (int)list.size());
    } catch (const std::bad_alloc&) {
        return 0;
    }
}

// Whether no result lies over another array or its result.
static bool clip_apart(const std::vector<ClipArray>& list) {
    struct Part { uintptr_t begin, end; bool result; };
    std::vector<Part> parts;
    parts.reserve(2 * list.size());
    for (const ClipArray& a : list) {
        const uintptr_t in = reinterpret_cast<uintptr_t>(a.in), out = reinterpret_cast<uintptr_t>(a.out), bytes = (uintptr_t)a.n * act_bytes(a.dtype);
        if (a.in != a.out) parts.push_back(Part{in, in + bytes, false});
        if (a.out) parts.push_back(Part{out, out + bytes, true});
    }
    std::sort(parts.begin(), parts.end(), [](const Part& a, const Part& b) { return a.begin < b.begin; });
    uintptr_t any = 0, results = 0;   // the ends of those before
    for (const Part& p : parts) {
        if (p.begin < (p.result ? any : results)) return false;
        any = std::max(any, p.end);
        if (p.result) results = std::max(results, p.end);
    }
    return true;
}

extern "C" int tmps_clip_gradients(const tmps_array* arrays, int n, float limit, float* norm, void* workspace, size_t workspace_bytes, void* hip_stream) {
    int rc = check_clip(arrays, n);
    if (rc != TMPS_OK) return rc;
    if (!(limit >= 0.0f)) return fail(TMPS_EINVAL, "limit must not be negative");
    if (!norm) return fail(TMPS_EINVAL, "norm is null");
    if (!aligned(norm, 4)) return fail(TMPS_ESHAPE, "norm is not on a whole element");
    try {
        const std::vector<ClipArray> list = clip_list(arrays, n);
        const size_t need = clip_workspace_bytes(list.data(), (int)list.size());
        if ((rc = room(workspace, workspace_bytes, need)) != TMPS_OK) return rc;
        const Range of_norm{norm, 4}, of_ws{workspace, need};
        if (of_norm.meets(of_ws)) return fail(TMPS_EINVAL, "norm lies in the workspace");
        bool with = false, without = false;
        for (const ClipArray& a : list) {
            const size_t bytes = (size_t)a.n * act_bytes(a.dtype);
            const Range in{a.in, bytes}, out{a.out, bytes};
            if (in.meets(of_norm) || in.meets(of_ws) || out.meets(of_norm) || out.meets(of_ws)) return fail(TMPS_EINVAL, "an array or its result overlaps the norm or the workspace");
            (a.out ? with : without) = true;
        }
        if (with && without) return fail(TMPS_EINVAL, "some arrays have a result and others none");
        if (with && !clip_apart(list)) return fail(TMPS_EINVAL, "a result overlaps another array or its result");
        TMPS_HIP(clip_gradients(list.data(), (int)list.size(), limit, norm, workspace, (hipStream_t)hip_stream));
    } catch (const std::bad_alloc&) {
        return fail(TMPS_EINVAL, "out of host memory");
    }
    return TMPS_OK;
}
