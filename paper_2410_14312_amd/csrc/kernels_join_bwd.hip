// Norm joins, backward.  With the rows' statistics of the forward pass, fh = (f - m1) i1 and yh = (y - m2) i2:
//   t = du pre_gain, dh = dy + i2 (t - mean(t) - yh mean(t yh))                 (means of t only where the norm subtracts one)
//   dr = scale dh (+ what others have given r);  da = dh gain fh g (1 - g);  v = dh g gain, df = i1 (v - mean(v) - fh mean(v fh))
//   dpre_gain = sum du yh, dpre_shift = sum du, dscale = sum dh r, dgain = sum dh g fh over the rows
// One pass over memory: dy, du, x, r, y are read and dx, dr written once each.  A team goes over its share of the rows and keeps its sums over them in registers, which
// leave as one row of partial results; those are added up in a fixed order behind.  In bf16, with the norm, both launches, each between two time stamps (us; a copy of as many
// bytes at 5.1 TB/s): 8192 x 768 26.6 (17.4) and gated 31.9 (22.4), 8192 x 2048 53 (46), 16384 x 4096 177 (186), 8192 x 8192 189 (186); in fp32 4096 x 1024 gated 36.1 (30).  What short rows lack are waves: a
// SIMD's registers hold two or three.  Rows of more than 8192 features have more values than registers and spill some (2048 x 16384: 167, 93).
#include <algorithm>

#include "launch.h"
#include "norm_join.hip.h"

namespace tmps {

// Threads of a launch at most: two waves to a SIMD, which is what its registers hold, each with its next row under way.
constexpr int kBwdThreads = 131072;

// A thread's sums over its rows, of N pieces of V: in registers, or (SHARED) in LDS, where nobody else touches them.
template <int TEAM, int N, int V, bool SHARED> struct RowSums {
    float kept[SHARED ? 1 : N][V];
    float4* mine;
    __device__ __forceinline__ void get(int i, float (&v)[V]) const {
        if constexpr (SHARED) {
#pragma unroll
            for (int h = 0; h < V / 4; ++h) {
                const float4 u = mine[(i * (V / 4) + h) * TEAM];
                v[4 * h] = u.x, v[4 * h + 1] = u.y, v[4 * h + 2] = u.z, v[4 * h + 3] = u.w;
            }
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = kept[i][e];
        }
    }
    __device__ __forceinline__ void put(int i, const float (&v)[V]) {
        if constexpr (SHARED) {
#pragma unroll
            for (int h = 0; h < V / 4; ++h) mine[(i * (V / 4) + h) * TEAM] = make_float4(v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) kept[i][e] = v[e];
        }
    }
    __device__ __forceinline__ void start(float4* at) {
        mine = at + threadIdx.x;
        const float zeros[V] = {};
#pragma unroll
        for (int i = 0; i < N; ++i) put(i, zeros);
    }
    // sum += a b, or a
    __device__ __forceinline__ void add(int i, const float (&a)[V], const float (&b)[V]) {
        float v[V];
        get(i, v);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = fmaf(a[e], b[e], v[e]);
        put(i, v);
    }
    __device__ __forceinline__ void add(int i, const float (&a)[V]) {
        float v[V];
        get(i, v);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] += a[e];
        put(i, v);
    }
};

// A row's operand as numbers, of N pieces of V: formed once (KEPT, where the next row's pieces take its registers), or wherever it is wanted.
template <int N, int V, bool KEPT, typename F> struct Numbers {
    F form;
    float kept[KEPT ? N : 1][V];
    __device__ __forceinline__ explicit Numbers(F f) : form(f) {
        if constexpr (KEPT) {
#pragma unroll
            for (int i = 0; i < N; ++i) form(i, kept[i]);
        }
    }
    __device__ __forceinline__ void get(int i, float (&v)[V]) const {
        if constexpr (KEPT) {
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = kept[i][e];
        } else {
            form(i, v);
        }
    }
};
template <int N, int V, bool KEPT, typename F> __device__ __forceinline__ Numbers<N, V, KEPT, F> numbers(F f) { return Numbers<N, V, KEPT, F>(f); }

// NEXT (8192 x 768 gated 31.3 us without, 28.0 with; 16384 x 4096 197 and 171): a row's operands are requested as soon as those of the row before are taken, in two parts: what the
// norm of y needs, and what comes behind its sums.  Workgroups of 1024 threads have no registers for that: they form an operand's numbers again wherever they are used, hold two of
// the sums in LDS and take a join's parameters, with a norm behind, from the cache (not KEEP; 4096 x 5120 gated 84 us, 97 in registers; 8192 x 8192 185 and 186).  Sums in LDS
// and numbers formed again against registers for both, first launch: 8192 x 8192 185 and 201 us, 3000 x 5001 gated 91 and 152, 2048 x 16384 152 and 297, 2048 x 8193 with means 130
// and 376.  (Of a row of odd length the compiler would keep in registers which features are whose, of all pieces at once: hence the row's length anew in every row.)
template <typename T, int TEAM, int N, bool WHOLE, bool JOIN, bool PRE, bool GATE>
__global__ __launch_bounds__(Team<TEAM>::kThreads) void norm_join_bwd_kernel(NormJoinBackward a, float* part, float* part_pre) {
    constexpr int kRows = Team<TEAM>::kRows, V = kPiece<T>;
    constexpr bool KEEP = N * V == 8 && !(TEAM == 1024 && JOIN && PRE), NEXT = KEEP && TEAM < 1024;
    __shared__ float red[2][2 * 16];
    __shared__ float fold[kRows > 1 ? kRows : 1][kRows > 1 ? TEAM * V * N : 1];
    const int D = a.D;
    constexpr int wide = GATE ? 2 : 1;
    const float over_d = 1.0f / (float)D;
    Pieces<TEAM, N, V, WHOLE> p{D};
    int place = 0;
    // (two of the sums of a workgroup of 1024 threads are in LDS)
    constexpr bool SHARED = TEAM == 1024;
    constexpr int kEach = N * V / 4 * TEAM;
    __shared__ float4 shared_sums[SHARED ? 2 * kEach : 1];
    RowSums<TEAM, N, V, SHARED> dgain, dscale;
    RowSums<TEAM, N, V, SHARED && !JOIN> dpg, dps;
    if constexpr (JOIN) {
        dgain.start(shared_sums);
        dscale.start(shared_sums + (SHARED ? kEach : 0));
    }
    if constexpr (PRE) {
        dpg.start(shared_sums);
        dps.start(shared_sums + (SHARED ? kEach : 0));
    }
    float gain[KEEP ? N : 1][V], scale[KEEP ? N : 1][V], pre_gain[KEEP ? N : 1][V];
    if constexpr (KEEP) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (JOIN) {
                load_vector(gain[i], a.gain, p, i);
                load_vector(scale[i], a.scale, p, i);
            }
            if constexpr (PRE) load_vector(pre_gain[i], a.pre_gain, p, i);
        }
    }
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TEAM;
    uint4 rdy[N], rdu[PRE ? N : 1], ry[PRE ? N : 1], rf[JOIN ? N : 1], ra[GATE ? N : 1], rr[JOIN ? N : 1], radd[JOIN ? N : 1];
    float st[2], pre_st[2];
    const bool has_dy = !PRE || a.dy;
    auto request_first = [&](int64_t at) {
        if constexpr (PRE) {
            request_row(rdu, (const T*)a.du + at * D, p);
            request_row(ry, (const T*)a.y + at * D, p);
            pre_st[0] = a.pre_stats[at * a.stats_stride];
            pre_st[1] = a.pre_stats[at * a.stats_stride + 1];
        }
        if (has_dy) request_row(rdy, (const T*)a.dy + at * D, p);
    };
    auto request_second = [&](int64_t at) {
        if constexpr (JOIN) {
            request_row(rf, (const T*)a.x + at * D * wide, p);
            request_row(rr, (const T*)a.r + at * D, p);
            if constexpr (GATE) request_row(ra, (const T*)a.x + at * D * wide + D, p);
            if (a.add) request_row(radd, (const T*)a.add + at * D, p);
            st[0] = a.stats[at * a.stats_stride];
            st[1] = a.stats[at * a.stats_stride + 1];
        }
    };
    if (NEXT && row < a.rows) {
        request_first(row);
        request_second(row);
    }
    for (; row < a.rows; row += step) {
        const bool more = NEXT && row + step < a.rows;
        if constexpr (TEAM == 1024) asm volatile("" : "+s"(p.D));
        if constexpr (!NEXT) request_first(row);
        if constexpr (!NEXT && KEEP) request_second(row);
        float dh[N][V];
        auto dy = numbers<N, V, NEXT>([&](int i, float (&v)[V]) {
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = 0.0f;
            if (has_dy) unpack(rdy[i], v);
        });
        if constexpr (PRE) {
            const float mean = pre_st[0], rstd = pre_st[1];
            auto yh = numbers<N, V, NEXT>([&](int i, float (&v)[V]) {
                unpack(ry[i], v);
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] = (v[e] - mean) * rstd;
            });
            float s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (!p.any(i)) continue;
                float du[V], y[V];
                if constexpr (!KEEP) load_vector(pre_gain[0], a.pre_gain, p, i);
                unpack(rdu[i], du);
                yh.get(i, y);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    dh[i][e] = du[e] * pre_gain[KEEP ? i : 0][e];
                    const float t = p.own(i, e) ? dh[i][e] : 0.0f;
                    s[0] = fmaf(t, y[e], s[0]);
                    s[1] += t;
                }
                dpg.add(i, du, y);
                dps.add(i, du);
            }
            if (more) request_first(row + step);
            if constexpr (!KEEP) request_second(row);
            Team<TEAM>::sums(s, red, place);
            const float m = a.rms ? 0.0f : s[1] * over_d, q = s[0] * over_d;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (!p.any(i)) continue;
                float d[V], y[V];
                dy.get(i, d);
                yh.get(i, y);
#pragma unroll
                for (int e = 0; e < V; ++e) dh[i][e] = fmaf(rstd, fmaf(-y[e], q, dh[i][e] - m), d[e]);
            }
        } else {
            if (more) request_first(row + step);
            if constexpr (!KEEP) request_second(row);
#pragma unroll
            for (int i = 0; i < N; ++i) dy.get(i, dh[i]);
        }
        if constexpr (JOIN) {
            const float mean = st[0], rstd = st[1];
            T* const dxr = (T*)a.dx + row * D * wide;
            auto fh = numbers<N, V, NEXT>([&](int i, float (&v)[V]) {
                unpack(rf[i], v);
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] = (v[e] - mean) * rstd;
            });
            auto from_r = numbers<N, V, NEXT>([&](int i, float (&v)[V]) { unpack(rr[i], v); });
            auto gate = numbers<N, V, NEXT>([&](int i, float (&v)[V]) {
                if constexpr (GATE) unpack(ra[i], v);
            });
            auto given = numbers<N, V, NEXT>([&](int i, float (&v)[V]) {
                if (a.add) unpack(radd[i], v);
            });
            float s[2] = {0.0f, 0.0f};
            if (more) request_second(row + step);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                if (!p.any(i)) continue;
                if constexpr (!KEEP) {
                    load_vector(gain[0], a.gain, p, i);
                    load_vector(scale[0], a.scale, p, i);
                }
                float o[V], r[V], f[V];
                from_r.get(i, r);
                fh.get(i, f);
#pragma unroll
                for (int e = 0; e < V; ++e) o[e] = dh[i][e] * scale[KEEP ? i : 0][e];
                dscale.add(i, dh[i], r);
                if (a.add) {
                    float v[V];
                    given.get(i, v);
#pragma unroll
                    for (int e = 0; e < V; ++e) o[e] += v[e];
                }
                if (a.dr) store_piece((T*)a.dr + row * D, p, i, o);
                if constexpr (GATE) {
                    float da[V], at[V];
                    gate.get(i, at);
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        float sg, rest;
                        gate_of<T>(at[e], sg, rest);
                        da[e] = dh[i][e] * gain[KEEP ? i : 0][e] * f[e] * (sg * rest);
                        dh[i][e] *= sg;
                    }
                    if (a.dx) store_piece(dxr + D, p, i, da);
                }
                dgain.add(i, dh[i], f);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    dh[i][e] *= gain[KEEP ? i : 0][e];
                    const float t = p.own(i, e) ? dh[i][e] : 0.0f;
                    s[0] = fmaf(t, f[e], s[0]);
                    s[1] += t;
                }
            }
            if (a.dx) {
                Team<TEAM>::sums(s, red, place);
                const float m = a.rms ? 0.0f : s[1] * over_d, q = s[0] * over_d;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    if (!p.any(i)) continue;
                    float o[V], f[V];
                    fh.get(i, f);
#pragma unroll
                    for (int e = 0; e < V; ++e) o[e] = rstd * fmaf(-f[e], q, dh[i][e] - m);
                    store_piece(dxr, p, i, o);
                }
            }
        } else if (a.dr) {
#pragma unroll
            for (int i = 0; i < N; ++i) store_piece((T*)a.dr + row * D, p, i, dh[i]);
        }
    }
    // The workgroup's row of partial results; its teams' sums, where it has several, are added up through LDS.
    auto leave = [&](const auto& sums, float* to) {
        if constexpr (kRows > 1) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float v[V];
                sums.get(i, v);
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (p.any(i) && p.own(i, e)) fold[threadIdx.x / TEAM][p.at(i) + e] = v[e];
            }
            __syncthreads();
            for (int c = threadIdx.x; c < D; c += Team<TEAM>::kThreads) {
                float t[kRows];
#pragma unroll
                for (int k = 0; k < kRows; ++k) t[k] = fold[k][c];
#pragma unroll
                for (int h = kRows / 2; h > 0; h >>= 1)
#pragma unroll
                    for (int k = 0; k < h; ++k) t[k] += t[k + h];
                to[c] = t[0];
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float v[V];
                sums.get(i, v);
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (p.any(i) && p.own(i, e)) to[p.at(i) + e] = v[e];
            }
        }
    };
    if constexpr (JOIN) {
        leave(dgain, part + (int64_t)blockIdx.x * 2 * D);
        leave(dscale, part + (int64_t)blockIdx.x * 2 * D + D);
    }
    if constexpr (PRE) {
        float* const to = part_pre + (int64_t)blockIdx.x * (a.rms ? 1 : 2) * D;
        leave(dpg, to);
        if (!a.rms) leave(dps, to + D);
    }
}

// The team that takes rows of D features, and the launch's workgroups: no more than the device holds at a time, and as many rows to each.
static int bwd_team(int D, bool whole) {
    if (D <= 128) return 16;
    if (D <= 256 && whole) return 32;
    if (D <= 512) return 64;
    if (D <= 1024) return 128;
    if (D <= 2048) return 256;
    return D <= 4096 ? 512 : 1024;
}
static int bwd_most(int team) { return (team == 1024 ? 2 : 1) * kBwdThreads / (team <= 64 ? 256 : team); }
static int64_t bwd_full_groups(int64_t rows, int team) {
    const int teams = team <= 64 ? 256 / team : 1;
    return (rows + teams - 1) / teams;
}
static int bwd_groups(int64_t rows, int team) {
    const int most = bwd_most(team);
    const int64_t groups = bwd_full_groups(rows, team), few = groups / 512 < 6 ? groups / 512 : 6;
    // (up to six, where that still leaves two workgroups to a compute unit: a row of partial results is two to four of 4-byte values, written and read; 2999 x 1001 in fp32 20.6 and 9.7 us
    // for the two launches with three rows to a workgroup, 20.7 and 6.4 with six)
    const int64_t each = (groups + most - 1) / most > few ? (groups + most - 1) / most : few > 1 ? few : 1;
    return (int)((groups + each - 1) / each);
}

size_t norm_join_part_elems(int64_t rows, int D) {
    const int a = bwd_groups(rows, bwd_team(D, true)), b = bwd_groups(rows, bwd_team(D, false));
    return (size_t)(a > b ? a : b) * 2 * (size_t)D;
}

// (fewer rows may take more workgroups: 1023 of 768 features 1023, 1024 of them 512)
size_t norm_join_part_elems_up_to(int64_t rows, int D) {
    int64_t groups = 0;
    for (bool whole : {true, false}) {
        const int team = bwd_team(D, whole);
        const int64_t most = std::min<int64_t>(bwd_full_groups(rows, team), bwd_most(team));
        groups = std::max(groups, most);
    }
    return (size_t)groups * 2 * (size_t)D;
}

template <typename T, int TEAM, int N, bool WHOLE> static hipError_t bwd_launch(const NormJoinBackward& j, const Partials& part, const Partials& part_pre, hipStream_t s) {
    const int groups = bwd_groups(j.rows, TEAM);
    auto kern = !j.x ? norm_join_bwd_kernel<T, TEAM, N, WHOLE, false, true, false>
                : !j.du ? (j.gate ? norm_join_bwd_kernel<T, TEAM, N, WHOLE, true, false, true> : norm_join_bwd_kernel<T, TEAM, N, WHOLE, true, false, false>)
                        : (j.gate ? norm_join_bwd_kernel<T, TEAM, N, WHOLE, true, true, true> : norm_join_bwd_kernel<T, TEAM, N, WHOLE, true, true, false>);
    hipError_t e = launch_timed(kcLayerNorm, kern, dim3(groups), dim3(Team<TEAM>::kThreads), 0, s, j, part.ws, part_pre.ws);
    if (e != hipSuccess) return e;
    const Reduction of_join{part.ws, j.dgain_dscale, 2 * (int64_t)j.D, groups, true}, of_pre{part_pre.ws, j.dpre, (j.rms ? 1 : 2) * (int64_t)j.D, groups, true};
    if (j.x && j.du && !part.later && !part_pre.later) return reduce_all(Reductions{of_join, of_pre}, s);
    if (j.x && (e = part.finish(of_join, s)) != hipSuccess) return e;
    return j.du ? part_pre.finish(of_pre, s) : hipSuccess;
}

template <typename T> static hipError_t bwd_type(const NormJoinBackward& j, const Partials& part, const Partials& part_pre, hipStream_t s) {
    const bool whole = join_whole<T>(j.D, {j.dy, j.du, j.x, j.r, j.y, j.gain, j.scale, j.pre_gain, j.add, j.dx, j.dr});
    switch (bwd_team(j.D, whole)) {
        case 16: return whole ? bwd_launch<T, 16, kOne<T>, true>(j, part, part_pre, s) : bwd_launch<T, 16, kOne<T>, false>(j, part, part_pre, s);
        case 32: return bwd_launch<T, 32, kOne<T>, true>(j, part, part_pre, s);
        case 64: return whole ? bwd_launch<T, 64, kOne<T>, true>(j, part, part_pre, s) : bwd_launch<T, 64, kOne<T>, false>(j, part, part_pre, s);
        case 128: return whole ? bwd_launch<T, 128, kOne<T>, true>(j, part, part_pre, s) : bwd_launch<T, 128, kOne<T>, false>(j, part, part_pre, s);
        case 256: return whole ? bwd_launch<T, 256, kOne<T>, true>(j, part, part_pre, s) : bwd_launch<T, 256, kOne<T>, false>(j, part, part_pre, s);
        case 512: return whole ? bwd_launch<T, 512, kOne<T>, true>(j, part, part_pre, s) : bwd_launch<T, 512, kOne<T>, false>(j, part, part_pre, s);
    }
    if (j.D <= 8192) return whole ? bwd_launch<T, 1024, kOne<T>, true>(j, part, part_pre, s) : bwd_launch<T, 1024, kOne<T>, false>(j, part, part_pre, s);
    return whole ? bwd_launch<T, 1024, 2 * kOne<T>, true>(j, part, part_pre, s) : bwd_launch<T, 1024, 2 * kOne<T>, false>(j, part, part_pre, s);
}

// Sums over no rows.
__global__ __launch_bounds__(256) void join_no_rows_kernel(float* dgain_dscale, float* dpre, int n, int n_pre) {
    for (int i = threadIdx.x; i < n; i += 256) dgain_dscale[i] = 0.0f;
    for (int i = threadIdx.x; i < n_pre; i += 256) dpre[i] = 0.0f;
}

hipError_t norm_join_backward(int dtype, const NormJoinBackward& j, const Partials& part, const Partials& part_pre, hipStream_t s) {
    if (j.rows <= 0)
        return launch_timed(kcLayerNorm, join_no_rows_kernel, dim3(1), dim3(256), 0, s, j.dgain_dscale, j.dpre, j.x ? 2 * j.D : 0, j.du ? (j.rms ? 1 : 2) * j.D : 0);
    if (j.D < 1 || j.D > kJoinMaxFeatures || (!j.x && !j.du) || (!j.dy && !j.du)) return hipErrorInvalidValue;
    return dtype == kBF16 ? bwd_type<bf16_t>(j, part, part_pre, s) : bwd_type<float>(j, part, part_pre, s);
}

}  // namespace tmps
