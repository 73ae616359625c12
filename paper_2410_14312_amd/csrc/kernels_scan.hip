// Selective state space, forward: per sample and head S_t = exp(-delta_t e^a) S_{t-1} + delta_t x_t B_t', y_t = S_t C_t + skip x_t.
//
// In chunks of 64 positions it is products of matrices: with D[t][s] the decay from s to t, d_t that from before the chunk to t,
//   y_t = sum_{s <= t} (C_t . B_s) D[t][s] delta_s x_s + d_t S C_t + skip x_t,   S <- d_end S + sum_s D[end][s] delta_s x_s B_s'
// A workgroup walks the chunks of a head's (or 64 features' of it) positions with the state in its accumulators, fp32; as an operand of a product a state, and the matrix of decayed
// products, is the sum of bf16 terms.  Where there are few samples and heads the positions are cut into stretches: a first walk leaves each one's own state, which are joined, and a second
// walk starts from those.  A few positions go one after the other with the state in registers, which is a reading and a writing of it.
//
// Bound by the latency of a chunk's steps, each of which needs the one before: 4.5 us a chunk, two workgroups to a compute unit hiding part of it (vector instructions 44 % of the time there,
// LDS 35, the matrix unit 15).  16 x 512 positions of 24 heads of 64 x 64 in bf16: 36.7 us, 1.4 TB/s of operands and results; 32768 of one sample with states of 128: 219 us.  Eight waves to a
// workgroup have no registers for it and form the decayed products twice: 42.7 and 315.
#include <algorithm>

#include "launch.h"
#include "scan_walk.hip.h"
#include "wave.hip.h"

namespace tmps {

// ------------------------------------------------------------------------------------------------ single positions
// 16 lanes to a feature, which share its state's n, four neighbours to each (and as many 64 further, HALVES == 2); four features to each of 16 teams.  PLAIN: n is 64 HALVES and a head's
// features whole 64s: every access is whole and none is in a branch, so that all of a thread's states are under way together.  64 sequences of 24 heads of 64 x 64: 25 MB read and 25
// written in 10.8 us.  Eight positions of them take 21 us, nine in a chunk 26: up to kScanSteps go this way.
template <typename T, int HALVES, bool PLAIN> __global__ __launch_bounds__(256) void scan_steps_kernel(Scan a) {
    constexpr int kPasses = 4;
    const int64_t unit = blockIdx.x;
    const int head = (int)(unit % a.heads), group = head / (a.heads / a.groups);
    const int64_t sample = unit / a.heads;
    const int lane = threadIdx.x & 15, team = threadIdx.x >> 4, p0 = (int)(blockIdx.z * gridDim.y + blockIdx.y) * (16 * kPasses);
    if (p0 >= a.dh) return;
    const int64_t of_head = unit * a.dh * a.n;
    const T* const xr = (const T*)a.x + sample * a.positions * a.x_stride;
    const T* const dtr = (const T*)a.dt + sample * a.positions * a.dt_stride + head;
    T* const yr = (T*)a.y + sample * a.positions * a.y_stride + (int64_t)head * a.dh;
    const int64_t b_at = (int64_t)a.heads * a.dh + (int64_t)group * a.n, c_at = b_at + (int64_t)a.groups * a.n;
    float s[kPasses][HALVES][4];
#pragma unroll
    for (int k = 0; k < kPasses; ++k) {
        const int p = p0 + team + 16 * k;
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            const int n = 4 * lane + 64 * h;
#pragma unroll
            for (int e = 0; e < 4; ++e) s[k][h][e] = 0.0f;
            if (a.state) {
                if constexpr (PLAIN) unpack(load16_any(a.state + of_head + (int64_t)p * a.n + n), s[k][h]);
                else if (p < a.dh && n < a.n) four_any(a.state + of_head + (int64_t)p * a.n + n, s[k][h], a.n - n);
            }
        }
    }
    const double rate = rate_of(a.a_log[head]) * kLog2eD;
    const float skip = a.skip[head], bias = a.dt_bias[head];
    for (int64_t t = 0; t < a.positions; ++t) {
        const T* const row = xr + t * a.x_stride;
        float b[HALVES][4], c[HALVES][4], x[kPasses];
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            const int n = 4 * lane + 64 * h;
            if constexpr (PLAIN) {
                four_anywhere(row + b_at + n, b[h]);
                four_anywhere(row + c_at + n, c[h]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool any = n + e < a.n;
                    b[h][e] = any ? to_f32(row[b_at + (any ? n + e : 0)]) : 0.0f;
                    c[h][e] = any ? to_f32(row[c_at + (any ? n + e : 0)]) : 0.0f;
                }
            }
        }
#pragma unroll
        for (int k = 0; k < kPasses; ++k) {
            const int p = p0 + team + 16 * k;
            x[k] = PLAIN || p < a.dh ? to_f32(row[(int64_t)head * a.dh + p]) : 0.0f;
        }
        const float u = to_f32(dtr[t * a.dt_stride]) + bias, delta = u != u ? u : softplus(u);
        const float decay = exp2_of(-(double)delta * rate);
#pragma unroll
        for (int k = 0; k < kPasses; ++k) {
            const int p = p0 + team + 16 * k;
            const float add = delta * x[k];
            float y = 0.0f;
#pragma unroll
            for (int h = 0; h < HALVES; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[k][h][e] = fmaf(decay, s[k][h][e], add * b[h][e]);
                    y = fmaf(s[k][h][e], c[h][e], y);
                }
            y += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(y), 0x128, 0xF, 0xF, false));   // row_ror:8
            y += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(y), 0x124, 0xF, 0xF, false));   // row_ror:4
            y += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(y), 0x122, 0xF, 0xF, false));   // row_ror:2
            y += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(y), 0x121, 0xF, 0xF, false));   // row_ror:1
            if (lane == 0 && (PLAIN || p < a.dh)) yr[t * a.y_stride + p] = from_f32<T>(fmaf(skip, x[k], y));
        }
    }
    if (!a.state_out) return;
#pragma unroll
    for (int k = 0; k < kPasses; ++k) {
        const int p = p0 + team + 16 * k;
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            const int n = 4 * lane + 64 * h;
            if constexpr (PLAIN) store16_any(a.state_out + of_head + (int64_t)p * a.n + n, pack(s[k][h]));
            else if (p < a.dh && n < a.n) put_four_any(a.state_out + of_head + (int64_t)p * a.n + n, s[k][h], a.n - n);
        }
    }
}

// ------------------------------------------------------------------------------------------------ launches
size_t scan_workspace_bytes(const Scan& a) {
    if (a.positions <= kScanSteps) return 0;
    return walk_stretch_bytes(a);
}

template <typename T> static hipError_t forward_type(const Scan& a, void* ws, hipStream_t s) {
    if (a.positions <= kScanSteps) {
        const int64_t units = a.samples * a.heads;
        const unsigned cuts = (unsigned)(a.dh + 63) / 64, in_y = std::min(cuts, 32768u);   // (a launch has 65535 workgroups in its second direction)
        if (!launchable(units, 256)) return hipErrorInvalidValue;
        const bool whole = a.dh % 64 == 0;
        auto kern = a.n > 64 ? (whole && a.n == 128 ? scan_steps_kernel<T, 2, true> : scan_steps_kernel<T, 2, false>)
                             : (whole && a.n == 64 ? scan_steps_kernel<T, 1, true> : scan_steps_kernel<T, 1, false>);
        return launch_timed(kcAttnFwd, kern, dim3((unsigned)units, in_y, (cuts + in_y - 1) / in_y), dim3(256), 0, s, a);
    }
    ScanWalk w = walk_of(a);
    w.y = a.y; w.y_stride = a.y_stride;
    w.final_state = a.state_out;
    walk_plan(w);
    const unsigned grid = walk_grid(w);
    if (!grid) return hipErrorInvalidValue;
    if (w.stretches > 1) {
        walk_room(w, static_cast<char*>(ws));
#define TMPS_OWN(NP, PT) launch_timed(kcAttnFwd, scan_walk_kernel<T, NP, PT, kWalkOwn>, dim3(grid), dim3(256), 0, s, w)
        hipError_t e = TMPS_WALK(TMPS_OWN, w);
        if (e != hipSuccess) return e;
        e = launch_timed(kcAttnFwd, scan_join_kernel, dim3(join_grid(w)), dim3(256), 0, s, w, padded_n(w.n), padded_dh(w.dh) * padded_n(w.n));
        if (e != hipSuccess) return e;
    }
#define TMPS_OUT(NP, PT) launch_timed(kcAttnFwd, scan_walk_kernel<T, NP, PT, kWalkResults>, dim3(grid), dim3(256), 0, s, w)
    return TMPS_WALK(TMPS_OUT, w);
}

hipError_t scan_forward(int dtype, const Scan& a, void* ws, hipStream_t s) { return dtype == kBF16 ? forward_type<bf16_t>(a, ws, s) : forward_type<float>(a, ws, s); }

}  // namespace tmps
