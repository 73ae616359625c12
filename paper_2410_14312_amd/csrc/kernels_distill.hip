// Distillation from a teacher's largest logits.  With T the temperature, m the row's largest logit, q = softmax(z / T), s = softmax(z), and p the softmax of the
// teacher's entries over T:
//   loss = alpha T^2 sum_j p_j (log p_j - log q[id_j]) + (1 - alpha) (-log s[label])
//   d loss / dz = alpha T (q - sum_j p_j e[id_j]) + (1 - alpha) (s - e[label])
// Bound by memory: a row of logits is read, a row of gradients written.  Hence a row stays in registers between its largest logit, its two sums and its gradients, each of which takes
// every logit's exponentials again.  Of 8192 rows of 32000 logits, 64 entries, bf16 gradients, between two time stamps: 319 us, 4.5 TB/s (a copy of as many bytes 285 us; 293 us where T is 1 and one exponential
// does for both, 253 us without a teacher); the same of 1, 16, 256 entries: 301, 304, 338 us; 4096 rows of 16000 logits: 77 us, 4.7 TB/s; 16384 rows of 1000: 26 us; 2048 rows of
// 50257: 137 us, 4.1 TB/s; of 65000 207 us, 3.5 TB/s (one workgroup to a compute unit: nothing runs beside its loads); 64 rows of 100: 7 us, mostly the launch.
#include <algorithm>

#include "kernels.h"
#include "pieces.hip.h"
#include "wave.hip.h"

namespace tmps {

// What a launch does with its rows: all of it, or one of two launches over slices of rows: the slices' largest logits and sums, and everything else.
enum { kWholeRows = 0, kSliceSums = 1, kSliceRest = 2 };

// How rows are cut: `slices` of `length` logits each (the last may be shorter).
struct Slices {
    int slices, length;
};

// A team's reductions, the result in every thread: one barrier each, by alternating between two places in LDS (who writes a place again has passed the barrier between).  Teams
// of a wave need neither.
template <int TEAM> struct Reduce {
    static constexpr int kWaves = TEAM / 64;
    float (*red)[3 * 16];
    int place = 0;
    // v[0], or with MAX the largest v[0] (NaN is passed over), and the sums of the others
    template <bool MAX, int K> __device__ __forceinline__ void all(float (&v)[K]) {
        v[0] = MAX ? wmax(v[0]) : wsum(v[0]);
#pragma unroll
        for (int k = 1; k < K; ++k) v[k] = wsum(v[k]);
        if constexpr (kWaves > 1) {
            if ((threadIdx.x & 63) == 0) {
#pragma unroll
                for (int k = 0; k < K; ++k) red[place][k * 16 + (threadIdx.x >> 6)] = v[k];
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < K; ++k) {
                v[k] = red[place][k * 16];
#pragma unroll
                for (int w = 1; w < kWaves; ++w) {
                    const float o = red[place][k * 16 + w];
                    v[k] = MAX && k == 0 ? fmaxf(v[k], o) : v[k] + o;
                }
            }
            place ^= 1;
        }
    }
};

// What a team's lanes have written to LDS or memory is there for the others.  (A wave's operations on either complete in order; the compiler is kept from moving them.)
template <int TEAM> __device__ __forceinline__ void team_sync() {
    if constexpr (TEAM > 64) {
        __syncthreads();
    } else {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_wave_barrier();
    }
}

// Many entries' classes are put into a table in LDS, at least twice as large, to learn in one pass that none is there twice, and whether the label is among them.  (Up to 64
// are simply compared with one another: as fast at 64.  4096 rows of 2000 logits, 1000 entries: 40 us, compared 273 us; 8192 of 32000, 256 entries: 343 us, 361 us.)
constexpr int kFewEntries = 64;
constexpr __host__ __device__ int table_bits(int k) {
    int bits = 0;
    for (; k > kFewEntries && (1 << bits) < 2 * k; ++bits) {}
    return bits;
}
// words of LDS to a team
__host__ __device__ inline int entry_words(int k) { return 3 * ((k + 3) & ~3) + (k > kFewEntries ? 1 << table_bits(k) : 0); }
struct ClassTable {
    int* at;
    int bits;
    __device__ __forceinline__ int begin(int id) const { return (int)((uint32_t)id * 2654435769u >> (32 - bits)); }
    __device__ __forceinline__ int next(int i) const { return (i + 1) & ((1 << bits) - 1); }
    // whether it was there before
    __device__ __forceinline__ bool add(int id) const {
        for (int i = begin(id);; i = next(i)) {
            const int was = atomicCAS(at + i, -1, id);
            if (was == -1 || was == id) return was == id;
        }
    }
    __device__ __forceinline__ bool has(int id) const {
        for (int i = begin(id);; i = next(i))
            if (at[i] == -1 || at[i] == id) return at[i] == id;
    }
};

__device__ __forceinline__ void store4(bf16_t* p, const float (&v)[4]) {
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    const uint32_t a = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{v[0], v[1]}), bf16x2_t));
    const uint32_t b = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{v[2], v[3]}), bf16x2_t));
    *reinterpret_cast<any_u32x2_t*>(p) = any_u32x2_t{a, b};
}
__device__ __forceinline__ void store4(float* p, const float (&v)[4]) { store16_any(p, pack(v)); }

// (A base that all lanes share, one for every piece, and a 32-bit offset, the same for all pieces: no address and no offset in registers from a piece's load to its store.)
template <typename T> __device__ __forceinline__ T* at_bytes(T* base, uint32_t bytes) { return (T*)((char*)base + bytes); }

// A team to a row (or a slice of one), whose logits it keeps in registers and LDS: NV pieces of 4 a thread and NL in LDS, which nobody else touches, and of the up to three behind the
// last whole piece one to a lane.
// What a thread has no logit for is minus infinity: pieces are loaded, compared and added up without a branch.  The classes of the entries and of the label get their gradients
// once more, behind the others: the first entry of a class writes it, with what all of them and the label take away.
template <typename T, int TEAM, int NV, int NL, int MODE>
__global__ __launch_bounds__(TEAM == 64 ? 256 : TEAM, TEAM == 1024 ? 4 : NV <= 16 ? 4 : 2) void distill_rows_kernel(Distill d, Slices cut, float* sums, int64_t unit0) {
    constexpr int kTeams = TEAM == 64 ? 4 : 1;
    constexpr float kLog2e = 1.4426950408889634f;
    extern __shared__ __attribute__((aligned(16))) float entries[];   // of every team: classes, exponentials, the student's logits
    __shared__ float red[2][3 * 16];
    __shared__ uint4 stash[NL > 0 ? NL * TEAM : 1];
    Reduce<TEAM> reduce{red};
    const int lane = threadIdx.x % TEAM, team = TEAM == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : 0, k = d.k, C = d.classes;
    const float over_t = 1.0f / d.temperature, alpha = d.alpha, at_q = kLog2e * over_t, at_s = kLog2e;
    const int slots = (k + 3) & ~3;   // (entries in whole fours)
    const bool same = d.temperature == 1.0f;   // q is s
    const int64_t unit = unit0 + (int64_t)blockIdx.x * kTeams + team;
    if (unit >= d.rows * cut.slices) return;
    const int64_t row = MODE == kWholeRows ? unit : unit / cut.slices;
    const int slice = MODE == kWholeRows ? 0 : (int)(unit - row * cut.slices), from = slice * cut.length, n = MODE == kWholeRows ? C : min(cut.length, C - from);
    const int bits = table_bits(k);
    int* const ids = reinterpret_cast<int*>(entries) + team * entry_words(k);
    float* const p = reinterpret_cast<float*>(ids) + slots;
    float* const zs = p + slots;
    const ClassTable table{reinterpret_cast<int*>(zs) + slots, bits};
    const float* const zrow = d.logits + row * C;
    T* const g = d.dlogits ? (T*)d.dlogits + row * C + from : nullptr;
    const int whole = n & ~3;   // logits in whole pieces

    // What the row has to learn from.  top: the teacher's largest logit (over T come differences from it: a common part of large logits takes no places from them); how many ids are no class; how many repeat one.  (A NaN among the teacher's logits makes the row one.)
    const int label = d.labels && alpha < 1.0f ? d.labels[row * d.label_stride] : -1;
    const bool labelled = label >= 0 && label < C;
    float top[3] = {-INFINITY, labelled || label == -1 ? 0.0f : 1.0f, 0.0f};
    const bool tabled = MODE != kSliceSums && g && k > kFewEntries;
    if (alpha > 0.0f) {
        if (tabled) {
            for (int j = lane; j < 1 << bits; j += TEAM) table.at[j] = -1;
            team_sync<TEAM>();
        }
        for (int j = lane; j < k; j += TEAM) {
            const int id = d.ids[row * d.entry_stride + j];
            const bool entry = id >= 0 && id < C;
            const float t = entry ? d.teacher[row * d.entry_stride + j] : -INFINITY;
            ids[j] = entry ? id : -1;
            p[j] = t;
            top[0] = fmaxf(top[0], t != t ? INFINITY : t);
            top[1] += entry || id == -1 ? 0.0f : 1.0f;
            if (tabled && entry && table.add(id)) top[2] = 1.0f;
        }
        reduce.template all<true>(top);
    }
    const bool taught = top[0] != -INFINITY, bad = top[1] != 0.0f;
    if (!taught && !labelled) {   // nothing to learn, whatever the logits are
        if (MODE != kSliceSums) {
            if (g) {
                const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int i = 0; i < NV + NL; ++i)
                    if (lane * 4 < whole - i * TEAM * 4) store4(at_bytes(g + i * TEAM * 4, lane * 4 * (int)sizeof(T)), zero);
                if (lane < n - whole) g[whole + lane] = from_f32<T>(0.0f);
            }
            if (slice == 0 && lane == 0) d.row_loss[row] = bad ? NAN : 0.0f;
        }
        return;
    }
    // (the student's logits of the entries before the row's: what is requested first is there first)
    const bool first = MODE != kSliceSums && taught && lane < k && ids[lane] >= 0;
    const float z_first = first ? zrow[ids[lane]] : 0.0f, z_label = MODE != kSliceSums && labelled ? zrow[label] : 0.0f;
    uint4 raw[NV], aside[NL > 0 ? NL : 1];
    const float* const z = zrow + from;
    float extra = -INFINITY;
    float kl = 0.0f, most[2] = {-INFINITY, 0.0f};   // the row's largest logit; the sum of the teacher's exponentials
    auto request = [&](uint4& u, int i) {
        const int last = whole * 4 - 16, base = min(i * TEAM * 16, last);
        u = load16_any(at_bytes(reinterpret_cast<const char*>(z) + base, (uint32_t)min(lane * 16, last - base)));
    };
    auto finite = [&](uint4& u, int i) {
        const bool any = lane * 4 < whole - i * TEAM * 4;
        float v[4];
        unpack(u, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = any ? v[e] : -INFINITY;
        most[0] = fmaxf(most[0], fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])));
        u = pack(v);
    };
    if (lane < n - whole) extra = z[whole + lane];
    if constexpr (NL > 0) {   // (at most NV pieces under way: the registers that the row has; such a row has whole pieces)
#pragma unroll
        for (int i = 0; i < NL; ++i) request(aside[i], NV + i);
#pragma unroll
        for (int i = 0; i < NV - NL; ++i) request(raw[i], i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            finite(aside[i], NV + i);
            stash[i * TEAM + lane] = aside[i];
            request(raw[NV - NL + i], NV - NL + i);
            __builtin_amdgcn_sched_barrier(0);
        }
    } else if (whole > 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) request(raw[i], i);
    }
    if (MODE != kSliceSums) {
        if (taught) {
            for (int j = lane; j < k; j += TEAM) {
                const float t = (p[j] - top[0]) * over_t, e = ids[j] >= 0 ? expf(t) : 0.0f;
                zs[j] = j == lane ? z_first : ids[j] >= 0 ? zrow[ids[j]] : 0.0f;
                p[j] = e;
                most[1] += e;
                kl += e != 0.0f ? e * t : 0.0f;
            }
        }
        if (lane < slots - k) ids[k + lane] = -1;
    }
    float m, sq = 0.0f, ss = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) finite(raw[i], i);
    most[0] = fmaxf(most[0], extra);
    if constexpr (MODE == kSliceRest) {
        // (at most 256 slices: one to a thread)
        const float* const part = sums + (row * cut.slices + lane) * 3;
        const bool any = lane < cut.slices;
        const float mine = any ? part[0] : -INFINITY;
        most[0] = mine;
        reduce.template all<true>(most);
        m = most[0];
        sq = any ? part[1] * __builtin_amdgcn_exp2f((mine - m) * at_q) : 0.0f;
        ss = any ? part[2] * __builtin_amdgcn_exp2f((mine - m) * at_s) : 0.0f;
    } else {
        reduce.template all<true>(most);
        m = most[0];
    }
    const float teacher = most[1];
    // (of a slice without a finite logit the sums are those of what its logits are: nothing, or NaN)
    const float off = MODE == kSliceSums && m == -INFINITY ? 0.0f : m;
    const bool need_s = labelled && !(same && taught);
    // (left to itself the compiler has many pieces' exponentials under way at once, in registers that the row needs: hence the barriers to its scheduling)
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float v[4];
        unpack(raw[i], v);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] -= off;
        raw[i] = pack(v);
    }
    extra -= off;
    auto piece = [&](int i, float (&v)[4]) {   // a piece's logits minus the largest
        if (i < NV) {
            unpack(raw[i], v);
        } else {
            unpack(stash[(i - NV) * TEAM + lane], v);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] -= off;
        }
    };
    auto add_up = [&](float scale) {
        float t = __builtin_amdgcn_exp2f(extra * scale);
#pragma unroll
        for (int i = 0; i < NV + NL; ++i) {
            float v[4];
            piece(i, v);
#pragma unroll
            for (int e = 0; e < 4; ++e) t += __builtin_amdgcn_exp2f(v[e] * scale);
            __builtin_amdgcn_sched_barrier(0);
        }
        return t;
    };
    if constexpr (MODE != kSliceRest) {
        if (taught) sq = add_up(at_q);
        if (need_s) ss = add_up(at_s);
    }
    if (MODE != kSliceSums && taught) {
        for (int j = lane; j < k; j += TEAM)
            if (p[j] != 0.0f) kl -= p[j] * ((zs[j] - m) * over_t);
    }
    float total[3] = {sq, ss, kl};
    reduce.template all<false>(total);
    sq = total[0];
    ss = same && taught ? sq : total[1];
    if constexpr (MODE == kSliceSums) {
        if (lane == 0) {
            sums[unit * 3] = m;
            sums[unit * 3 + 1] = sq;
            sums[unit * 3 + 2] = ss;
        }
        return;
    }
    const float T_ = d.temperature, on_entry = taught ? alpha * T_ * d.grad_scale : 0.0f, on_label = labelled ? (1.0f - alpha) * d.grad_scale : 0.0f;
    if (slice == 0 && lane == 0) {
        float loss = taught ? alpha * T_ * T_ * (total[2] / teacher - logf(teacher) + logf(sq)) : 0.0f;
        if (labelled) loss += (1.0f - alpha) * (logf(ss) - (z_label - m));
        d.row_loss[row] = bad ? NAN : loss;
    }
    if (!g) return;
    // one exponential to a logit, or two
    const float w1 = taught ? on_entry / sq + (same && labelled ? on_label / ss : 0.0f) : on_label / ss, at1 = taught ? at_q : at_s, w2 = need_s && taught ? on_label / ss : 0.0f;
    auto gradient = [&](float v, bool two) {
        float o = w1 * __builtin_amdgcn_exp2f(v * at1);
        if (two) o = fmaf(w2, __builtin_amdgcn_exp2f(v * at_s), o);
        return o;
    };
    auto write = [&](bool two) {
#pragma unroll
        for (int i = 0; i < NV + NL; ++i) {
            float v[4];
            piece(i, v);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = gradient(v[e], two);
            if (lane * 4 < whole - i * TEAM * 4) store4(at_bytes(g + i * TEAM * 4, lane * 4 * (int)sizeof(T)), v);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const bool two = need_s && taught;
    if (two) write(true);
    else write(false);
    if (lane < n - whole) g[whole + lane] = from_f32<T>(gradient(extra, two));
    team_sync<TEAM>();
    const float share = taught ? on_entry / teacher : 0.0f;
    for (int j = taught ? lane : k + lane; j <= k; j += TEAM) {   // (the last is the label, for a class that no entry has)
        const int id = j < k ? ids[j] : label;
        if (id < from || id >= from + n) continue;
        int alike = 0;
        if (tabled && top[2] == 0.0f) {
            alike = j < k || (taught && table.has(id));
        } else {
            for (int i = 0; taught && i < slots; i += 4) {
                const int4 v = *reinterpret_cast<const int4*>(ids + i);
                alike += (v.x == id) + (v.y == id) + (v.z == id) + (v.w == id);
            }
        }
        float sum = 0.0f;
        if (j == k) {
            if (alike) continue;
        } else if (alike == 1) {
            sum = p[j];
        } else {   // (the sum in the entries' order)
            int firsts = j;
            for (int i = 0; i < k; ++i)
                if (ids[i] == id) {
                    firsts = min(firsts, i);
                    sum += p[i];
                }
            if (firsts != j) continue;
        }
        float o = gradient((j < k ? zs[j] : z_label) - m, two);
        if (id == label) o -= on_label;
        g[id - from] = from_f32<T>(fmaf(-share, sum, o));
    }
}

// Rows of more than 98304 logits are cut into slices that registers hold (1024 rows of 131072: 259 us), and few wide rows into as many as give every compute unit eight: one row of
// 98304 logits takes 13 us, whole 24, 64 rows 20 and 31; 8 rows of 50257 14 and 17; 8 rows of 32000 15 and 12.  (48 rows of 131071: 20 us, with two to a compute unit 26.)
constexpr int kWholeMax = 98304, kSliceMax = 32768;
constexpr int64_t kFewRows = 64;
static Slices cut_rows(int64_t rows, int classes) {
    const int64_t fit = classes > kWholeMax ? (classes + kSliceMax - 1) / kSliceMax : 1;
    int64_t slices = fit;
    if (rows <= kFewRows && classes > kSliceMax) {
        const int64_t wanted = (2048 + rows - 1) / rows, most = (classes + 4095) / 4096 < 256 ? (classes + 4095) / 4096 : 256;
        slices = wanted < most ? wanted : most;
        if (slices < fit) slices = fit;
    }
    const int64_t length = ((classes + slices - 1) / slices + 3) / 4 * 4;
    return Slices{(int)((classes + length - 1) / length), (int)length};
}

size_t distill_workspace_elems(int64_t rows, int64_t plan_rows, int classes) {
    const Slices cut = cut_rows(plan_rows, classes);
    return cut.slices > 1 ? (size_t)rows * cut.slices * 3 : 0;
}

// (few rows are cut into more slices than many)
size_t distill_workspace_elems_up_to(int64_t rows, int classes) {
    if (classes <= kSliceMax) return 0;
    size_t elems = distill_workspace_elems(rows, rows, classes);
    for (int64_t r = std::min(rows, kFewRows); r > 0; --r) elems = std::max(elems, distill_workspace_elems(r, r, classes));
    return elems;
}

// (A launch takes no loop over rows: what a lane has in each of them would be kept in registers that the row needs.)
template <typename T, int TEAM, int NV, int MODE, int NL = 0> static hipError_t launch_rows(const Distill& d, const Slices& cut, float* ws, hipStream_t s) {
    constexpr int teams = TEAM == 64 ? 4 : 1;
    const int64_t units = d.rows * cut.slices, at_once = int64_t(teams) << 20;
    for (int64_t unit = 0; unit < units; unit += at_once) {
        const int64_t n = units - unit < at_once ? units - unit : at_once;
        hipLaunchKernelGGL((distill_rows_kernel<T, TEAM, NV, NL, MODE>), dim3((unsigned)((n + teams - 1) / teams)), dim3(TEAM == 64 ? 256 : TEAM), (size_t)teams * entry_words(d.k) * 4, s, d, cut,
                           ws, unit);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T, int MODE> static hipError_t launch_slices(const Distill& d, const Slices& cut, float* ws, hipStream_t s) {
    if (cut.length <= 4096) return launch_rows<T, 256, 4, MODE>(d, cut, ws, s);
    if (cut.length <= 8192) return launch_rows<T, 256, 8, MODE>(d, cut, ws, s);
    return launch_rows<T, 512, 16, MODE>(d, cut, ws, s);
}

template <typename T> static hipError_t distill_type(const Distill& d, float* ws, hipStream_t s) {
    const Slices cut = cut_rows(d.plan_rows, d.classes);
    if (cut.slices > 1) {
        const hipError_t e = launch_slices<T, kSliceSums>(d, cut, ws, s);
        return e != hipSuccess ? e : launch_slices<T, kSliceRest>(d, cut, ws, s);
    }
    const int C = d.classes;
    // A wave to a row needs no barriers: 16384 rows of 1000 logits take 26 us, with 256 threads 58 us, rows of 2000 39 and 65 us.  With many entries it loses: 4096 rows of 2000,
    // 10 entries 15 and 21 us, 500 entries 32 and 31 us, 1000 entries 64 and 40 us.  The other teams, where two were measured: 8192 rows of 12000 by 256 threads 122 us, 512 133 us;
    // of 32000 by 512 317 us, 1024 (fewer registers to each, some spilled) 366 us; 2048 of 65000 by 512 202 us, 1024 206 us; of 90000 by 1024 329 us
    // (270 since a lane's offset is one for all pieces), 512 364 us, in slices 350 us.  Up to 51200 classes part of the row lies in LDS and a compute unit holds two rows: 2048 of 50257 136 us,
    // of 40000 111, by registers alone 176 and 159.  (Wider rows held so, 22 or 24 pieces in registers, spill: 2048 of 63000 235 to 282 us, by registers alone 204.)
    if (d.k <= 256) {
        if (C <= 256) return launch_rows<T, 64, 1, kWholeRows>(d, cut, ws, s);
        if (C <= 512) return launch_rows<T, 64, 2, kWholeRows>(d, cut, ws, s);
        if (C <= 1024) return launch_rows<T, 64, 4, kWholeRows>(d, cut, ws, s);
        if (C <= 2048) return launch_rows<T, 64, 8, kWholeRows>(d, cut, ws, s);
    }
    if (C <= 4096) return launch_rows<T, 256, 4, kWholeRows>(d, cut, ws, s);
    if (C <= 8192) return launch_rows<T, 256, 8, kWholeRows>(d, cut, ws, s);
    if (C <= 16384) return launch_rows<T, 256, 16, kWholeRows>(d, cut, ws, s);
    if (C <= 32768) return launch_rows<T, 512, 16, kWholeRows>(d, cut, ws, s);
    if (C <= 51200) return launch_rows<T, 512, 16, kWholeRows, 9>(d, cut, ws, s);
    if (C <= 65536) return launch_rows<T, 512, 32, kWholeRows>(d, cut, ws, s);
    return launch_rows<T, 1024, 24, kWholeRows>(d, cut, ws, s);
}

hipError_t distill(int dtype, const Distill& d, float* ws, hipStream_t s) {
    if (d.rows <= 0) return hipSuccess;
    return dtype == kBF16 ? distill_type<bf16_t>(d, ws, s) : distill_type<float>(d, ws, s);
}

}  // namespace tmps
