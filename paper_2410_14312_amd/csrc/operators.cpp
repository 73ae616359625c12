// Operators as calls of their own, over the caller's memory: rotary positions, norm joins, distillation.  Arguments are checked here; the launchers are those that the
// layers of a stage use.
#include <float.h>
#include <math.h>

#include <new>

#include "common.h"
#include "kernels.h"
#include "operands.h"
#include "profile.h"

using namespace tmps;

extern "C" int tmps_rotary(int dtype, const tmps_rotary_desc* desc, const void* x, int64_t x_stride, void* y, int64_t y_stride, const int32_t* positions,
                           int64_t n_positions, int64_t rows, int inverse, void* hip_stream) {
    if (!known(dtype)) return fail(TMPS_EINVAL, "unknown dtype %d", dtype);
    if (!desc) return fail(TMPS_EINVAL, "desc is null");
    if (desc->heads < 1 || desc->dh < 1 || rows < 0) return fail(TMPS_EINVAL, "heads and features per head must be positive, rows not negative");
    int64_t pairs = 0;
    for (int k = 0; k < 3; ++k) {
        if (desc->pairs[k] < 0) return fail(TMPS_EINVAL, "negative number of pairs on axis %d", k);
        pairs += desc->pairs[k];
    }
    if (pairs < 1 || 2 * pairs > desc->dh) return fail(TMPS_ESHAPE, "%lld pairs of features in a head of %d", (long long)pairs, desc->dh);
    if (desc->flags & ~(TMPS_FLAG_INTERLEAVED | TMPS_FLAG_OWN_LADDERS)) return fail(TMPS_EINVAL, "unknown flags %d", desc->flags);
    if (!(desc->base > 0.0f) || !isfinite(desc->base)) return fail(TMPS_EINVAL, "base must be positive");
    const int64_t width = (int64_t)desc->heads * desc->dh, esz = (int64_t)act_bytes(dtype);
    if (width > INT32_MAX) return fail(TMPS_EUNSUPPORTED, "rows of more than 2^31 features");
    if (rows == 0) return TMPS_OK;
    if (!x || !y || !positions) return fail(TMPS_EINVAL, "x, y or positions is null");
    if (n_positions < 1) return fail(TMPS_EINVAL, "no positions");
    if (rows > 1 && (x_stride < width || y_stride < width)) return fail(TMPS_ESHAPE, "rows of %lld features overlap", (long long)width);
    if (rows > kMaxElems / width || (rows > 1 && (x_stride > kMaxElems / rows || y_stride > kMaxElems / rows))) return fail(TMPS_EUNSUPPORTED, "too many rows");
    if (!aligned(x, esz) || !aligned(y, esz) || !aligned(positions, 4)) return fail(TMPS_ESHAPE, "a pointer is not on a whole element");
    if (rows == 1) x_stride = y_stride = width;
    const Range in{x, (size_t)(((rows - 1) * x_stride + width) * esz)}, out{y, (size_t)(((rows - 1) * y_stride + width) * esz)};
    if (in.meets(out) && !(x == y && x_stride == y_stride)) {
        // (other columns of the same rows)
        const int64_t d = ((const char*)y - (const char*)x) / esz, e = x_stride == y_stride ? ((d % x_stride) + x_stride) % x_stride : 0;
        if (e < width || e > x_stride - width) return fail(TMPS_EINVAL, "y overlaps x without being x");
    }
    if (out.meets(Range{positions, (size_t)n_positions * 12})) return fail(TMPS_EINVAL, "y overlaps the positions");
    Rotary r;
    r.x = x; r.y = y; r.x_stride = x_stride; r.y_stride = y_stride; r.rows = rows; r.heads = desc->heads; r.dh = desc->dh;
    for (int k = 0; k < 3; ++k) r.pairs[k] = desc->pairs[k];
    r.flags = desc->flags; r.copied = 0;
    r.base = desc->base; r.inverse = inverse != 0; r.pos = positions; r.pos_rows = n_positions;
    r.grid_rows = r.grid_h = r.grid_w = 1;
    TMPS_HIP(rotary(dtype, r, (hipStream_t)hip_stream));
    return TMPS_OK;
}

static int check_join(int dtype, int flags, int64_t rows, int D) {
    if (!known(dtype)) return fail(TMPS_EINVAL, "unknown dtype %d", dtype);
    if (flags & ~(TMPS_FLAG_RMS | TMPS_FLAG_GATE)) return fail(TMPS_EINVAL, "unknown flags %d", flags);
    if (D < 1 || rows < 0) return fail(TMPS_EINVAL, "features must be positive, rows not negative");
    if (D > kJoinMaxFeatures) return fail(TMPS_EUNSUPPORTED, "rows of more than %d features", kJoinMaxFeatures);
    if (rows > kMaxElems / (2 * (int64_t)D)) return fail(TMPS_EUNSUPPORTED, "too many rows");
    return TMPS_OK;
}

extern "C" int tmps_norm_join_forward(int dtype, int flags, int64_t rows, int D, const void* x, const void* r, const float* gain, const float* scale, void* y,
                                      const float* pre_gain, const float* pre_shift, void* u, float* stats, void* hip_stream) {
    const int rc = check_join(dtype, flags, rows, D);
    if (rc != TMPS_OK) return rc;
    const bool rms = flags & TMPS_FLAG_RMS, gate = flags & TMPS_FLAG_GATE;
    if (rows == 0) return TMPS_OK;   // (arrays without elements may have no address)
    if ((u != nullptr) != (pre_gain != nullptr)) return fail(TMPS_EINVAL, "u and pre_gain go together");
    if (u ? (pre_shift != nullptr) == rms : pre_shift != nullptr) return fail(TMPS_EINVAL, "pre_shift belongs to a norm with a mean (no TMPS_FLAG_RMS) of the result");
    if (!x || !r || !gain || !scale || !y || !stats) return fail(TMPS_EINVAL, "an argument is null");
    const size_t esz = act_bytes(dtype), n = (size_t)rows * D * esz, v = (size_t)D * 4;
    for (const void* p : {x, r, (const void*)y, (const void*)u})
        if (!aligned(p, esz)) return fail(TMPS_ESHAPE, "a pointer is not on a whole element");
    for (const float* p : {gain, scale, pre_gain, pre_shift, (const float*)stats})
        if (!aligned(p, 4)) return fail(TMPS_ESHAPE, "a pointer is not on a whole element");
    const Range operands[] = {{x, gate ? 2 * n : n}, {r, n}, {gain, v}, {scale, v}, {pre_gain, v}, {pre_shift, v}};
    const Range results[] = {{y, n}, {u, n}, {stats, (size_t)rows * 16}};
    if (overlaps(operands, results, r)) return fail(TMPS_EINVAL, "a result overlaps an operand or another result (y may be r)");
    NormJoin j;
    j.x = x; j.r = r; j.gain = gain; j.scale = scale; j.y = y; j.stats = stats; j.pre_gain = pre_gain; j.pre_shift = pre_shift; j.u = u; j.pre_stats = stats + 2;
    j.stats_stride = 4; j.rows = rows; j.D = D; j.rms = rms; j.gate = gate;
    TMPS_HIP(norm_join_forward(dtype, j, (hipStream_t)hip_stream));
    return TMPS_OK;
}

extern "C" size_t tmps_norm_join_workspace(int64_t rows, int D) {
    if (rows < 1 || D < 1 || D > kJoinMaxFeatures) return 0;
    return 2 * norm_join_part_elems_up_to(rows, D) * sizeof(float);
}

extern "C" int tmps_norm_join_backward(int dtype, int flags, int64_t rows, int D, const void* dy, const void* du, const void* x, const void* r, const void* y,
                                       const float* stats, const float* gain, const float* scale, const float* pre_gain, void* dx, void* dr, float* dgain_dscale,
                                       float* dpre, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const int rc = check_join(dtype, flags, rows, D);
    if (rc != TMPS_OK) return rc;
    const bool rms = flags & TMPS_FLAG_RMS, gate = flags & TMPS_FLAG_GATE;
    if (!dgain_dscale || (du && !dpre)) return fail(TMPS_EINVAL, "an argument is null");
    const size_t part = rows > 0 ? norm_join_part_elems(rows, D) : 0, need = 2 * part * sizeof(float);   // (what the query gives is enough for fewer rows too)
    const size_t esz = act_bytes(dtype), n = (size_t)rows * D * esz, v = (size_t)D * 4;
    if (rows > 0) {
        if (!dy && !du) return fail(TMPS_EINVAL, "neither dy nor du is given");
        if (!x || !r || !stats || !gain || !scale || (du && (!y || !pre_gain))) return fail(TMPS_EINVAL, "an argument is null");
        if (!workspace || workspace_bytes < need) return fail(TMPS_ECAP, "the workspace holds %zu bytes, %zu are needed", workspace ? workspace_bytes : (size_t)0, need);
    }
    for (const void* p : {dy, du, x, r, y, (const void*)dx, (const void*)dr})
        if (!aligned(p, esz)) return fail(TMPS_ESHAPE, "a pointer is not on a whole element");
    for (const void* p : {(const void*)stats, (const void*)gain, (const void*)scale, (const void*)pre_gain, (const void*)dgain_dscale, (const void*)dpre, (const void*)workspace})
        if (!aligned(p, 4)) return fail(TMPS_ESHAPE, "a pointer is not on a whole element");
    const Range operands[] = {{dy, n}, {du, n}, {x, gate ? 2 * n : n}, {r, n}, {du ? y : nullptr, n}, {stats, (size_t)rows * 16}, {gain, v}, {scale, v}, {pre_gain, v}};
    const Range results[] = {{dr, n}, {dx, gate ? 2 * n : n}, {dgain_dscale, 2 * v}, {du || rows == 0 ? dpre : nullptr, rms ? v : 2 * v}, {rows > 0 ? workspace : nullptr, need}};
    if (overlaps(operands, results, dy)) return fail(TMPS_EINVAL, "a result or the workspace overlaps an operand or another result (dr may be dy)");
    NormJoinBackward j;
    j.dy = dy; j.du = du; j.x = x; j.r = r; j.y = y; j.stats = stats; j.pre_stats = stats ? stats + 2 : nullptr; j.gain = gain; j.scale = scale; j.pre_gain = pre_gain;
    j.add = nullptr; j.dx = dx; j.dr = dr; j.dgain_dscale = dgain_dscale; j.dpre = dpre; j.stats_stride = 4; j.rows = rows; j.D = D; j.rms = rms; j.gate = gate;
    if (rows == 0) j.x = dgain_dscale, j.du = dpre;   // (the gradients of no rows, which have no address, of which none is read)
    float* const ws = static_cast<float*>(workspace);
    try {
        TMPS_HIP(norm_join_backward(dtype, j, Partials(ws), Partials(ws ? ws + part : nullptr), (hipStream_t)hip_stream));
    } catch (const std::bad_alloc&) {
        return fail(TMPS_EINVAL, "out of host memory");
    }
    return TMPS_OK;
}

int tmps::check_distill(int64_t classes, int64_t k, float temperature, float alpha) {
    if (classes < 1 || k < 1) return fail(TMPS_EINVAL, "classes and k must be positive");
    if (classes > kDistillMaxClasses) return fail(TMPS_EUNSUPPORTED, "more than %d classes", kDistillMaxClasses);
    if (k > kDistillMaxEntries) return fail(TMPS_EUNSUPPORTED, "more than %d teacher entries a row", kDistillMaxEntries);
    // (the loss has its square for a factor: one that is nothing, or has lost places, would take the term along)
    const float square = temperature * temperature;
    if (!(temperature > 0.0f) || !isfinite(square) || square < FLT_MIN) return fail(TMPS_EINVAL, "temperature must be positive, its square within the range of a float");
    if (!(alpha >= 0.0f && alpha <= 1.0f)) return fail(TMPS_EINVAL, "alpha must lie in 0..1");
    return TMPS_OK;
}

extern "C" size_t tmps_distill_workspace(int64_t rows, int classes) {
    if (rows < 1 || classes < 1 || classes > kDistillMaxClasses) return 0;
    return distill_workspace_elems_up_to(rows, classes) * sizeof(float);
}

extern "C" int tmps_distill(int dtype, const tmps_distill_desc* desc, int64_t rows, const float* logits, const int32_t* labels, int64_t label_stride, const int32_t* ids,
                            const float* teacher, int64_t entry_stride, void* dlogits, float* row_loss, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (!known(dtype)) return fail(TMPS_EINVAL, "unknown dtype %d", dtype);
    if (!desc) return fail(TMPS_EINVAL, "desc is null");
    const int rc = tmps::check_distill(desc->classes, desc->k, desc->temperature, desc->alpha);
    if (rc != TMPS_OK) return rc;
    if (rows < 0) return fail(TMPS_EINVAL, "negative number of rows");
    if (!isfinite(desc->grad_scale)) return fail(TMPS_EINVAL, "grad_scale must be finite");
    if (rows == 0) return TMPS_OK;
    if (!logits || !row_loss || (desc->alpha > 0.0f && (!ids || !teacher))) return fail(TMPS_EINVAL, "an argument is null");
    if (desc->alpha > 0.0f && entry_stride < desc->k) return fail(TMPS_ESHAPE, "entries of one row overlap those of the next");
    if (labels && label_stride < 1) return fail(TMPS_ESHAPE, "label_stride must be positive");
    if (rows > kMaxElems / desc->classes || (desc->alpha > 0.0f && rows > kMaxElems / entry_stride) || (labels && rows > kMaxElems / label_stride))
        return fail(TMPS_EUNSUPPORTED, "too many rows");
    for (const void* p : {(const void*)logits, (const void*)labels, (const void*)ids, (const void*)teacher, (const void*)row_loss, (const void*)workspace})
        if (!aligned(p, 4)) return fail(TMPS_ESHAPE, "a pointer is not on a whole element");
    if (!aligned(dlogits, act_bytes(dtype))) return fail(TMPS_ESHAPE, "a pointer is not on a whole element");
    const size_t need = distill_workspace_elems(rows, rows, desc->classes) * sizeof(float), n = (size_t)rows * desc->classes;
    if (need && (!workspace || workspace_bytes < need))
        return fail(TMPS_ECAP, "the workspace holds %zu bytes, %zu are needed", workspace ? workspace_bytes : (size_t)0, need);
    const size_t entries = desc->alpha > 0.0f ? ((size_t)(rows - 1) * entry_stride + desc->k) * 4 : 0;
    const Range operands[] = {{logits, n * 4}, {labels, labels ? ((size_t)(rows - 1) * label_stride + 1) * 4 : 0}, {ids, entries}, {teacher, entries}};
    const Range results[] = {{dlogits, n * act_bytes(dtype)}, {row_loss, (size_t)rows * 4}, {workspace, need}};
    if (overlaps(operands, results)) return fail(TMPS_EINVAL, "a result or the workspace overlaps an operand or another result");
    Distill d;
    d.logits = logits; d.labels = labels; d.ids = ids; d.teacher = teacher; d.label_stride = label_stride; d.entry_stride = entry_stride; d.rows = rows;
    d.classes = desc->classes; d.k = desc->k; d.temperature = desc->temperature; d.alpha = desc->alpha; d.grad_scale = desc->grad_scale; d.dlogits = dlogits; d.row_loss = row_loss;
    d.plan_rows = rows;
    ProfileScope scope(kcSoftmaxCE, (hipStream_t)hip_stream);
    TMPS_HIP(distill(dtype, d, static_cast<float*>(workspace), (hipStream_t)hip_stream));
    return TMPS_OK;
}
