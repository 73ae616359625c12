// Distillation from a teacher's largest logits.  With T the temperature, m the row's largest logit, q = softmax(z / T), s = softmax(z), and p the softmax of the
// teacher's entries over T:
//   loss = alpha T^2 sum_j p_j (log p_j - log q[id_j]) + (1 - alpha) (-log s[label])
//   d loss / dz = alpha T (q - sum_j p_j e[id_j]) + (1 - alpha) (s - e[label])
// Bound by memory: a row of logits is read, a row of gradients written.
#include "gemm.hip.h"
#include "kernels.h"
#include "wave.hip.h"

namespace tmps {

// The sum and maximum over a workgroup, the same in every thread; red: a float per wave.
template <int THREADS> __device__ __forceinline__ float block_sum(float v, float* red) {
    v = wsum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    float t = red[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) t += red[w];
    return t;
}
template <int THREADS> __device__ __forceinline__ float block_max(float v, float* red) {
    v = wmax(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    float t = red[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) t = fmaxf(t, red[w]);
    return t;
}

// A row's teacher: entries in LDS, their probabilities, and what the row has to learn from.
struct RowTeacher {
    bool taught, labelled, bad;   // bad: an id or label that is neither a class nor -1
    int label;
    float log_norm;               // of the teacher's logits over T
};

// ids: the entries' classes (-1: none); t: their logits over T; p: their probabilities.  Every thread of the workgroup takes part.
template <int THREADS> __device__ __forceinline__ RowTeacher read_teacher(const Distill& d, int64_t row, int* ids, float* t, float* p, float* red) {
    RowTeacher w;
    w.label = d.labels && d.alpha < 1.0f ? d.labels[row * d.label_stride] : -1;
    w.labelled = w.label >= 0 && w.label < d.classes;
    w.bad = !w.labelled && w.label != -1;
    w.taught = false;
    w.log_norm = 0.0f;
    if (d.alpha <= 0.0f) return w;
    const float over_t = 1.0f / d.temperature;
    float mx = -INFINITY, wrong = 0.0f;
    for (int j = threadIdx.x; j < d.k; j += THREADS) {
        const int id = d.ids[row * d.entry_stride + j];
        const bool entry = id >= 0 && id < d.classes;
        wrong = entry || id == -1 ? wrong : 1.0f;
        const float v = entry ? d.teacher[row * d.entry_stride + j] * over_t : -INFINITY;
        ids[j] = entry ? id : -1;
        t[j] = v;
        mx = v > mx || v != v ? v : mx;
    }
    w.bad |= block_max<THREADS>(wrong, red) > 0.0f;
    mx = block_max<THREADS>(mx, red);
    w.taught = mx != -INFINITY;
    if (!w.taught) return w;
    float sum = 0.0f;
    for (int j = threadIdx.x; j < d.k; j += THREADS) {
        p[j] = ids[j] >= 0 ? expf(t[j] - mx) : 0.0f;
        sum += p[j];
    }
    sum = block_sum<THREADS>(sum, red);
    for (int j = threadIdx.x; j < d.k; j += THREADS) p[j] /= sum;
    w.log_norm = mx + logf(sum);
    __syncthreads();
    return w;
}

// A workgroup to a row, which it reads for the maximum, for the sums and for the gradient.
template <typename T> __global__ __launch_bounds__(256) void distill_kernel(Distill d) {
    __shared__ int ids[kDistillMaxEntries];
    __shared__ float t[kDistillMaxEntries], p[kDistillMaxEntries], red[4];
    const int C = d.classes;
    const float over_t = 1.0f / d.temperature, alpha = d.alpha;
    for (int64_t row = blockIdx.x; row < d.rows; row += gridDim.x) {
        __syncthreads();   // (the row before is done with the entries)
        const RowTeacher w = read_teacher<256>(d, row, ids, t, p, red);
        const float* const z = d.logits + row * C;
        T* const g = d.dlogits ? (T*)d.dlogits + row * C : nullptr;
        if (!w.taught && !w.labelled) {   // nothing to learn: whatever the logits are
            if (g)
                for (int c = threadIdx.x; c < C; c += 256) g[c] = from_f32<T>(0.0f);
            if (threadIdx.x == 0) d.row_loss[row] = w.bad ? NAN : 0.0f;
            continue;
        }
        float mx = -INFINITY;
        for (int c = threadIdx.x; c < C; c += 256) mx = fmaxf(mx, z[c]);
        mx = block_max<256>(mx, red);
        float sq = 0.0f, ss = 0.0f;
        for (int c = threadIdx.x; c < C; c += 256) {
            const float v = z[c] - mx;
            sq += expf(v * over_t);
            ss += expf(v);
        }
        sq = block_sum<256>(sq, red);
        ss = block_sum<256>(ss, red);
        const float wq = w.taught ? alpha * d.temperature / sq * d.grad_scale : 0.0f, ws = w.labelled ? (1.0f - alpha) / ss * d.grad_scale : 0.0f;
        const float on_label = (1.0f - alpha) * d.grad_scale, on_entry = alpha * d.temperature * d.grad_scale;
        float kl = 0.0f;
        if (w.taught) {
            const float log_q = logf(sq);
            for (int j = threadIdx.x; j < d.k; j += 256)
                if (p[j] != 0.0f) kl += p[j] * ((t[j] - w.log_norm) - ((z[ids[j]] - mx) * over_t - log_q));
            kl = block_sum<256>(kl, red);
        }
        if (threadIdx.x == 0) {
            float loss = w.taught ? alpha * d.temperature * d.temperature * kl : 0.0f;
            if (w.labelled) loss += (1.0f - alpha) * (logf(ss) - (z[w.label] - mx));
            d.row_loss[row] = w.bad ? NAN : loss;
        }
        if (!g) continue;
        for (int c = threadIdx.x; c < C; c += 256) {
            const float v = z[c] - mx;
            float o = wq * expf(v * over_t) + ws * expf(v);
            if (w.labelled && c == w.label) o -= on_label;
            g[c] = from_f32<T>(o);
        }
        if (!w.taught) continue;
        __syncthreads();
        // The entries' classes once more, with what the teacher gives them: the first entry of a class writes it, with the sum of all.
        for (int j = threadIdx.x; j < d.k; j += 256) {
            const int id = ids[j];
            if (id < 0) continue;
            float sum = 0.0f;
            bool first = true;
            for (int i = 0; i < d.k; ++i)
                if (ids[i] == id) {
                    first = first && i >= j;
                    sum += p[i];
                }
            if (!first) continue;
            const float v = z[id] - mx;
            float o = wq * expf(v * over_t) + ws * expf(v) - on_entry * sum;
            if (w.labelled && id == w.label) o -= on_label;
            g[id] = from_f32<T>(o);
        }
    }
}

size_t distill_workspace_elems(int64_t rows, int64_t plan_rows, int classes) {
    (void)rows;
    (void)plan_rows;
    (void)classes;
    return 0;
}

hipError_t distill(int dtype, const Distill& d, float* ws, hipStream_t s) {
    (void)ws;
    if (d.rows <= 0) return hipSuccess;
    const dim3 grid((unsigned)(d.rows < (1 << 20) ? d.rows : 1 << 20));
    if (dtype == kBF16) hipLaunchKernelGGL(distill_kernel<bf16_t>, grid, dim3(256), 0, s, d);
    else hipLaunchKernelGGL(distill_kernel<float>, grid, dim3(256), 0, s, d);
    return hipGetLastError();
}

}  // namespace tmps
