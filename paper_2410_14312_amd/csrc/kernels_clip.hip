// The norm of many arrays together, and the arrays scaled to at most a given norm.  Squares are added in 64 bits (no square of a float overflows there, and the sum of any number of
// them keeps 2^-50 of itself), in a fixed order: of a thread, a workgroup, all workgroups.
#include "launch.h"
#include "mixer.h"
#include "pieces.hip.h"

namespace tmps {

// Arrays of a launch: as many as fit the 4 KiB that a kernel takes for arguments.
constexpr int kClipArrays = 120;
constexpr int kClipBlock = 16384;   // elements of a workgroup
struct ClipTable {
    const void* in[kClipArrays];
    void* out[kClipArrays];
    int64_t n[kClipArrays];
    uint32_t first[kClipArrays + 1];   // the first workgroup of each, bit 31: bf16
    int count;
};
static_assert(sizeof(ClipTable) + 32 <= 4096, "a kernel's arguments");

int64_t clip_blocks(int64_t n) { return (n + kClipBlock - 1) / kClipBlock; }

__device__ __forceinline__ int clip_find(const ClipTable& t, uint32_t block) {
    int lo = 0, hi = t.count;   // first[lo] <= block < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if ((t.first[mid] & 0x7fffffffu) <= block) lo = mid;
        else hi = mid;
    }
    return lo;
}

// f(values, how many) over a workgroup's elements in pieces of 16 bytes from `from` on
template <typename T, class F> __device__ __forceinline__ void clip_pieces(const T* from, int n, F&& f) {
    constexpr int V = kPiece<T>;
    constexpr int N = kClipBlock / (256 * V);
#pragma unroll 4
    for (int i = 0; i < N; ++i) {
        const int at = (i * 256 + (int)threadIdx.x) * V;
        if (at + V <= n) {
            float v[V];
            unpack(load16_any(from + at), v);
            f(v, at, V);
        } else if (at < n) {
            float v[V];
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = at + e < n ? to_f32(from[at + e]) : 0.0f;
            f(v, at, n - at);
        }
    }
}

__device__ __forceinline__ double clip_block_sum(double v) {
    __shared__ double red[256];
    red[threadIdx.x] = v;
    __syncthreads();
    for (int d = 128; d > 0; d >>= 1) {
        if ((int)threadIdx.x < d) red[threadIdx.x] += red[threadIdx.x + d];
        __syncthreads();
    }
    return red[0];
}

__global__ __launch_bounds__(256) void clip_squares_kernel(ClipTable t, double* part) {
    const int a = clip_find(t, blockIdx.x);
    const int64_t begin = (int64_t)(blockIdx.x - (t.first[a] & 0x7fffffffu)) * kClipBlock;
    const int n = (int)min<int64_t>(kClipBlock, t.n[a] - begin);
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

__global__ __launch_bounds__(256) void clip_norm_kernel(const double* part, int64_t n, float limit, float* norm, float* scale) {
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += 256) sum += part[i];
    sum = clip_block_sum(sum);
    if (threadIdx.x == 0) {
        const double r = sqrt(sum);
        *norm = (float)r;
        *scale = r > (double)limit && r < __builtin_inf() ? (float)((double)limit / r) : 1.0f;
    }
}

__global__ __launch_bounds__(256) void clip_scale_kernel(ClipTable t, const float* scale) {
    const int a = clip_find(t, blockIdx.x);
    const float by = *scale;
    if (by == 1.0f && t.in[a] == t.out[a]) return;
    const int64_t begin = (int64_t)(blockIdx.x - (t.first[a] & 0x7fffffffu)) * kClipBlock;
    const int n = (int)min<int64_t>(kClipBlock, t.n[a] - begin);
    auto scaled = [&](auto* to) {
        return [=](auto& v, int at, int m) {
            constexpr int V = sizeof(v) / sizeof(v[0]);
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] *= by;
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

// f(table, its workgroups, the workgroups before it) for the arrays in launches
template <class F> static hipError_t clip_tables(const ClipArray* list, int n, F&& f) {
    int64_t before = 0;
    for (int i = 0; i < n;) {
        ClipTable t;
        t.count = 0;
        int64_t blocks = 0;
        for (; i < n && t.count < kClipArrays && (t.count == 0 || blocks + clip_blocks(list[i].n) < (1 << 30)); ++i) {
            if (list[i].n <= 0) continue;
            t.in[t.count] = list[i].in; t.out[t.count] = list[i].out; t.n[t.count] = list[i].n;
            t.first[t.count] = (uint32_t)blocks | (list[i].dtype == kBF16 ? 0x80000000u : 0u);
            blocks += clip_blocks(list[i].n);
            ++t.count;
        }
        if (!t.count) break;
        t.first[t.count] = (uint32_t)blocks;
        const hipError_t e = f(t, blocks, before);
        if (e != hipSuccess) return e;
        before += blocks;
    }
    return hipSuccess;
}

size_t clip_workspace_bytes(int64_t blocks) { return (size_t)(blocks + 1) * sizeof(double); }

hipError_t clip_gradients(const ClipArray* list, int n, float limit, float* norm, void* ws, hipStream_t s) {
    double* const part = static_cast<double*>(ws);
    int64_t total = 0;
    hipError_t e = clip_tables(list, n, [&](const ClipTable& t, int64_t blocks, int64_t before) {
        total = before + blocks;
        return launch_timed(kcReduce, clip_squares_kernel, dim3((unsigned)blocks), dim3(256), 0, s, t, part + before);
    });
    if (e != hipSuccess) return e;
    float* const scale = reinterpret_cast<float*>(part + total);
    e = launch_timed(kcReduce, clip_norm_kernel, dim3(1), dim3(256), 0, s, (const double*)part, total, limit, norm, scale);
    if (e != hipSuccess || !list || n < 1 || !list[0].out) return e;
    return clip_tables(list, n, [&](const ClipTable& t, int64_t blocks, int64_t) {
        return launch_timed(kcUpdate, clip_scale_kernel, dim3((unsigned)blocks), dim3(256), 0, s, t, (const float*)scale);
    });
}

}  // namespace tmps
