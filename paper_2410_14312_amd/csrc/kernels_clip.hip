// The norm of many arrays together, and the arrays scaled to at most a given norm.  Squares are added in 64 bits (no square of a float overflows there, and the sum of any number of
// them keeps 2^-50 of itself), in a fixed order: of a thread, a workgroup, all workgroups.  Bound by memory: all arrays are read for the norm and again for the scaling, which begins with
// what was read last, and is still in the last cache.  217 arrays of 337 MB: 98 us for the norm, 117 for the scaling.
#include "launch.h"
#include "mixer.h"
#include "pieces.hip.h"

namespace tmps {

// Arrays of a launch: as many as fit the 4 KiB that a kernel takes for arguments.
constexpr int kClipArrays = 120;
// Elements of a workgroup: so many that some three thousand workgroups have them all, each of which then adds up all workgroups' sums for itself (a launch less: 5 us), and no fewer than
// gives a thread four pieces.
constexpr int kClipLeast = 8192, kClipMost = 1 << 20, kClipWanted = 3072, kClipOwnSum = 6144;
struct ClipTable {
    const void* in[kClipArrays];
    void* out[kClipArrays];
    int64_t n[kClipArrays];
    uint32_t first[kClipArrays + 1];   // the first workgroup of each, bit 31: bf16
    int count, block;                  // arrays, elements of a workgroup
};
static_assert(sizeof(ClipTable) + 64 <= 4096, "a kernel's arguments");

static int64_t blocks_of(int64_t n, int block) { return (n + block - 1) / block; }
static int clip_block(const ClipArray* list, int n) {
    int64_t all = 0;
    for (int i = 0; i < n; ++i) all += list[i].n;
    int block = kClipLeast;
    while (block < kClipMost && all > (int64_t)block * kClipWanted) block *= 2;
    return block;
}

__device__ __forceinline__ int clip_find(const ClipTable& t, uint32_t block) {
    int lo = 0, hi = t.count;   // first[lo] <= block < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if ((t.first[mid] & 0x7fffffffu) <= block) lo = mid;
        else hi = mid;
    }
    return lo;
}

// f(values, the first one's place, how many) over a workgroup's elements in pieces of 16 bytes from `from` on, eight of a thread's under way at a time
template <typename T, class F> __device__ __forceinline__ void clip_pieces(const T* from, int n, F&& f) {
    constexpr int V = kPiece<T>, U = 8;
    int at = (int)threadIdx.x * V;
    for (; at + (U - 1) * 256 * V + V <= n; at += U * 256 * V) {
        uint4 u[U];
#pragma unroll
        for (int k = 0; k < U; ++k) u[k] = load16_any(from + at + k * 256 * V);
#pragma unroll
        for (int k = 0; k < U; ++k) {
            float v[V];
            unpack(u[k], v);
            f(v, at + k * 256 * V, V);
        }
    }
    for (; at < n; at += 256 * V) {
        float v[V];
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = at + e < n ? to_f32(from[at + e]) : 0.0f;
        f(v, at, min(V, n - at));
    }
}

// The same in every thread.
__device__ __forceinline__ double clip_block_sum(double v) {
    __shared__ double red[4];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// The norm and the factor of all workgroups' sums.  (Whether the norm is finite is asked of what is returned of it, which may not be where its 64 bits are.)
__device__ __forceinline__ double clip_norm(const double* part, int64_t n, float limit, double& scale) {
    double sum = 0.0;
#pragma unroll 8
    for (int64_t i = threadIdx.x; i < n; i += 256) sum += part[i];
    const double r = sqrt(clip_block_sum(sum));
    scale = r > (double)limit && (float)r < __builtin_inff() ? (double)limit / r : 1.0;
    return r;
}

__global__ __launch_bounds__(256) void clip_squares_kernel(ClipTable t, double* part) {
    const int a = clip_find(t, blockIdx.x);
    const int64_t begin = (int64_t)(blockIdx.x - (t.first[a] & 0x7fffffffu)) * t.block;
    const int n = (int)min<int64_t>(t.block, t.n[a] - begin);
    double sum = 0.0;
    auto add = [&](const auto& v, int, int) {
#pragma unroll
        for (float x : v) sum = fma((double)x, (double)x, sum);
    };
    if (t.first[a] >> 31) clip_pieces((const bf16_t*)t.in[a] + begin, n, add);
    else clip_pieces((const float*)t.in[a] + begin, n, add);
    sum = clip_block_sum(sum);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

__global__ __launch_bounds__(256) void clip_norm_kernel(const double* part, int64_t n, float limit, float* norm, double* scale) {
    double by;
    const double r = clip_norm(part, n, limit, by);
    if (threadIdx.x == 0) {
        *norm = (float)r;
        *scale = by;
    }
}

// scale: the factor, or null where each workgroup forms it from the `sums` of all.  Workgroups come in the opposite order of the first pass's.
__global__ __launch_bounds__(256) void clip_scale_kernel(ClipTable t, const double* scale, const double* part, int64_t sums, float limit, float* norm) {
    const uint32_t block = gridDim.x - 1 - blockIdx.x;
    const int a = clip_find(t, block);
    double all;
    if (scale) {
        all = *scale;
    } else {
        const double r = clip_norm(part, sums, limit, all);
        if (norm && block == 0 && threadIdx.x == 0) *norm = (float)r;
    }
    // (a factor below the normal range has few bits in a float, if any, where products have all: its power of two is apart)
    int power = 0;
    if (all < 0x1p-126) all = frexp(all, &power);
    const float by = (float)all;
    if (by == 1.0f && t.in[a] == t.out[a]) return;
    const int64_t begin = (int64_t)(block - (t.first[a] & 0x7fffffffu)) * t.block;
    const int n = (int)min<int64_t>(t.block, t.n[a] - begin);
    auto scaled = [&](auto* to) {
        return [=](auto& v, int at, int m) {
            constexpr int V = sizeof(v) / sizeof(v[0]);
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = __builtin_ldexpf(v[e] * by, power);
            if (m == V) {
                store16_any(to + at, pack(v));
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (e < m) to[at + e] = from_f32<std::remove_pointer_t<decltype(to)>>(v[e]);
            }
        };
    };
    if (t.first[a] >> 31) clip_pieces((const bf16_t*)t.in[a] + begin, n, scaled((bf16_t*)t.out[a] + begin));
    else clip_pieces((const float*)t.in[a] + begin, n, scaled((float*)t.out[a] + begin));
}

// The arrays from `i` on that one launch takes; returns its workgroups.
static int64_t clip_table(ClipTable& t, const ClipArray* list, int n, int block, int& i) {
    int64_t blocks = 0;
    t.count = 0;
    t.block = block;
    for (; i < n && t.count < kClipArrays && (t.count == 0 || launchable(blocks + blocks_of(list[i].n, block), 256)); ++i) {
        if (list[i].n <= 0) continue;
        t.in[t.count] = list[i].in; t.out[t.count] = list[i].out; t.n[t.count] = list[i].n;
        t.first[t.count] = (uint32_t)blocks | (list[i].dtype == kBF16 ? 0x80000000u : 0u);
        blocks += blocks_of(list[i].n, block);
        ++t.count;
    }
    t.first[t.count] = (uint32_t)blocks;
    return blocks;
}

size_t clip_workspace_bytes(const ClipArray* list, int n) {
    const int block = clip_block(list, n);
    int64_t blocks = 0;
    for (int i = 0; i < n; ++i) blocks += list[i].n > 0 ? blocks_of(list[i].n, block) : 0;
    return (size_t)(blocks + 1) * sizeof(double);
}

hipError_t clip_gradients(const ClipArray* list, int n, float limit, float* norm, void* ws, hipStream_t s) {
    double* const part = static_cast<double*>(ws);
    const int block = clip_block(list, n);
    std::vector<ClipTable> tables;
    std::vector<int64_t> blocks;
    int64_t total = 0;
    for (int i = 0; i < n;) {
        tables.emplace_back();
        blocks.push_back(clip_table(tables.back(), list, n, block, i));
        if (!blocks.back()) break;
        if (!launchable(blocks.back(), 256)) return hipErrorInvalidValue;
        const hipError_t e = launch_timed(kcSliceSum, clip_squares_kernel, dim3((unsigned)blocks.back()), dim3(256), 0, s, tables.back(), part + total);
        if (e != hipSuccess) return e;
        total += blocks.back();
    }
    const bool scaled = n > 0 && list[0].out;
    double* const scale = part + total;
    const bool own = scaled && total > 0 && total <= kClipOwnSum;
    if (!own) {
        const hipError_t e = launch_timed(kcSliceSum, clip_norm_kernel, dim3(1), dim3(256), 0, s, (const double*)part, total, limit, norm, scale);
        if (e != hipSuccess || !scaled) return e;
    }
    for (size_t k = tables.size(); k-- > 0;) {
        if (!blocks[k]) continue;
        const hipError_t e = launch_timed(kcAffine, clip_scale_kernel, dim3((unsigned)blocks[k]), dim3(256), 0, s, tables[k], own ? nullptr : (const double*)scale, (const double*)part, total,
                                          limit, k == 0 ? norm : nullptr);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace tmps
