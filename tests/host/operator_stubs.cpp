// Stand-ins for the launchers of rotary positions, norm joins and distillation (paper_2410_14312_amd/csrc/kernels.h) in host-only sanitizer builds: nothing is launched; what a
// launch reads is read and what it writes is written, whole, so that a sanitizer sees a layout that is too small, and launches are counted.
#include "operator_stubs.h"

#include <string.h>

#include "../../include/tmps.h"
#include "../../paper_2410_14312_amd/csrc/kernels.h"

OperatorStubs operator_stubs;
static volatile unsigned char sink;

static void reads(const void* p, size_t bytes) {
    unsigned char sum = 0;
    for (size_t i = 0; p && i < bytes; ++i) sum += static_cast<const unsigned char*>(p)[i];
    sink = sum;
}
static void writes(void* p, size_t bytes) {
    if (p) memset(p, 1, bytes);
}

namespace tmps {

hipError_t rotary(int dtype, const Rotary& r, hipStream_t) {
    const size_t e = act_bytes(dtype);
    const bool in_place = r.x == r.y;
    ++(r.inverse ? operator_stubs.turned_back : operator_stubs.turned);
    if (in_place) ++operator_stubs.in_place;
    for (int64_t k = 0; k < r.rows; ++k) {
        const size_t n = (size_t)(r.heads + (in_place ? 0 : r.copied)) * r.dh * e;
        reads((const char*)r.x + k * r.x_stride * e, n);
        writes((char*)r.y + k * r.y_stride * e, n);
    }
    return hipSuccess;
}

hipError_t norm_join_forward(int dtype, const NormJoin& j, hipStream_t) {
    const size_t n = (size_t)j.rows * j.D * act_bytes(dtype);
    ++operator_stubs.joins;
    if (j.x && j.u) ++operator_stubs.joins_with_norm;
    reads(j.x, j.gate ? 2 * n : n);
    reads(j.r, n);
    if (j.x) writes(j.y, n);
    else reads(j.y, n);
    writes(j.u, n);
    for (const float* p : {j.gain, j.scale, j.pre_gain, j.pre_shift}) reads(p, (size_t)j.D * 4);
    for (int64_t r = 0; r < j.rows; ++r) {
        if (j.x) writes(j.stats + r * j.stats_stride, 8);
        if (j.u) writes(j.pre_stats + r * j.stats_stride, 8);
    }
    return hipSuccess;
}

size_t norm_join_part_elems(int64_t rows, int D) { return (size_t)(rows < 4 ? rows : 4) * 2 * (size_t)D; }

hipError_t norm_join_backward(int dtype, const NormJoinBackward& j, const Partials& part, const Partials& part_pre, hipStream_t) {
    const size_t n = (size_t)j.rows * j.D * act_bytes(dtype);
    ++operator_stubs.joins_back;
    if (!j.x && !j.du) return hipErrorInvalidValue;
    reads(j.dy, n);
    reads(j.du, n);
    reads(j.x, j.gate ? 2 * n : n);
    reads(j.r, n);
    if (j.du) reads(j.y, n);
    reads(j.add, n);
    if (j.x) writes(part.ws, norm_join_part_elems(j.rows, j.D) * 4);
    if (j.du) writes(part_pre.ws, norm_join_part_elems(j.rows, j.D) * 4);
    if (j.x && j.du && (part.ws < part_pre.ws ? part.ws + norm_join_part_elems(j.rows, j.D) > part_pre.ws : part_pre.ws + norm_join_part_elems(j.rows, j.D) > part.ws))
        return hipErrorInvalidValue;   // (one overlaps the other)
    if (j.x) writes(j.dx, j.gate ? 2 * n : n);
    writes(j.dr, n);
    if (j.x) writes(j.dgain_dscale, (size_t)j.D * 8);
    if (j.du) writes(j.dpre, (size_t)j.D * (j.rms ? 4 : 8));
    return hipSuccess;
}

size_t distill_workspace_elems(int64_t rows, int64_t plan_rows, int) { return (size_t)(rows + plan_rows); }

hipError_t distill(int dtype, const Distill& d, float* ws, hipStream_t) {
    const size_t n = (size_t)d.rows * d.classes;
    ++operator_stubs.distillations;
    reads(d.logits, n * 4);
    for (int64_t r = 0; r < d.rows; ++r) {
        reads(d.labels + r * d.label_stride, 4);
        reads(d.ids + r * d.entry_stride, (size_t)d.k * 4);
        reads(d.teacher + r * d.entry_stride, (size_t)d.k * 4);
    }
    writes(d.dlogits, n * act_bytes(dtype));
    writes(d.row_loss, (size_t)d.rows * 4);
    writes(ws, distill_workspace_elems(d.rows, d.plan_rows, d.classes) * 4);
    return hipSuccess;
}

int check_distill(int64_t classes, int64_t k, float temperature, float alpha) {
    return classes < 1 || k < 1 || !(temperature > 0.0f) || !(alpha >= 0.0f && alpha <= 1.0f) ? TMPS_EINVAL : k > kDistillMaxEntries ? TMPS_EUNSUPPORTED : TMPS_OK;
}

}  // namespace tmps
