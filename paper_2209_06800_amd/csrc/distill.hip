// The loss of a student against a teacher's top logits, and its gradient.
#include <cmath>

#include "train_common.h"

namespace mgg {

namespace {

using namespace train;

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kMaxTop = 1024;

struct DistillArgs {
    const void *logits, *top_ids, *top_logits;
    const float *row_weight;
    float *loss;
    void *grad;
    int64_t ld_logits, ld_ids, ld_top, ld_grad;
    int32_t n_classes, k;
    float temperature;
    int32_t ids64, top_bf16;
};

__device__ __forceinline__ int64_t entry_id(const DistillArgs &p, int64_t row, int j)
{
    return p.ids64 ? static_cast<const int64_t *>(p.top_ids)[row * p.ld_ids + j] : static_cast<const int32_t *>(p.top_ids)[row * p.ld_ids + j];
}
__device__ __forceinline__ float entry_logit(const DistillArgs &p, int64_t row, int j)
{
    return p.top_bf16 ? to_f32(static_cast<const Bf16 *>(p.top_logits)[row * p.ld_top + j]) : static_cast<const float *>(p.top_logits)[row * p.ld_top + j];
}

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) { const float o = __shfl_xor(v, off); v = v > o || v != v ? v : o; }
    return v;
}
__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

template <bool MAX>
__device__ __forceinline__ float block_join(float v, float *part)
{
    v = MAX ? wave_max(v) : wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
        if (MAX) v = v > part[w] || v != v ? v : part[w];
        else v += part[w];
    }
    return v;
}

// a block per row: maximum, sum, then the gradient
template <typename In, typename Out>
__global__ __launch_bounds__(kThreads) void distill_row_kernel(const DistillArgs p)
{
    __shared__ float part[kWaves];
    __shared__ int32_t id_of[kMaxTop];
    __shared__ float p_of[kMaxTop], z_of[kMaxTop];
    const int64_t row = blockIdx.x;
    const In *z = static_cast<const In *>(p.logits) + row * p.ld_logits;
    Out *dz = p.grad ? static_cast<Out *>(p.grad) + row * p.ld_grad : nullptr;
    const float weight = p.row_weight ? p.row_weight[row] : 1.f, inv_t = 1.f / p.temperature;
    float high = -INFINITY;
    for (int j = threadIdx.x; j < p.k; j += kThreads) {
        const int64_t id = entry_id(p, row, j);
        const bool there = id >= 0 && id < p.n_classes;
        const float t = there ? entry_logit(p, row, j) : -INFINITY;
        id_of[j] = there ? static_cast<int32_t>(id) : -1;
        p_of[j] = t;
        z_of[j] = there ? to_f32(z[id]) : 0.f;
        high = high > t || high != high ? high : t;
    }
    high = block_join<true>(high, part);
    float m = -INFINITY;
    if (weight != 0.f)
        for (int c = threadIdx.x; c < p.n_classes; c += kThreads) {
            const float x = to_f32(z[c]);
            m = m > x || m != m ? m : x;
        }
    m = block_join<true>(m, part);
    if (weight == 0.f || high == -INFINITY || m == -INFINITY) {
        if (threadIdx.x == 0) p.loss[row] = 0.f;
        if (dz)
            for (int c = threadIdx.x; c < p.n_classes; c += kThreads) from_f32(0.f, dz[c]);
        return;
    }
    float sum = 0.f;
    for (int c = threadIdx.x; c < p.n_classes; c += kThreads) sum += expf((to_f32(z[c]) - m) * inv_t);
    sum = block_join<false>(sum, part);
    const float log_sum = logf(sum);
    float p_sum = 0.f;
    for (int j = threadIdx.x; j < p.k; j += kThreads)
        if (id_of[j] >= 0) p_sum += expf((p_of[j] - high) * inv_t);
    p_sum = block_join<false>(p_sum, part);
    const float log_p_sum = logf(p_sum);
    float part_loss = 0.f;
    for (int j = threadIdx.x; j < p.k; j += kThreads) {
        const float log_p = (p_of[j] - high) * inv_t - log_p_sum, prob = id_of[j] >= 0 ? expf(log_p) : 0.f;
        if (prob != 0.f) part_loss += prob * (log_p - ((z_of[j] - m) * inv_t - log_sum));
        p_of[j] = prob;
    }
    part_loss = block_join<false>(part_loss, part);
    if (threadIdx.x == 0) p.loss[row] = weight * p.temperature * p.temperature * part_loss;
    if (!dz) return;
    const float factor = weight * p.temperature, inv_sum = 1.f / sum;
    for (int c = threadIdx.x; c < p.n_classes; c += kThreads) from_f32(factor * expf((to_f32(z[c]) - m) * inv_t) * inv_sum, dz[c]);
    __syncthreads();
    // the teacher's classes, each by its first entry
    for (int j = threadIdx.x; j < p.k; j += kThreads) {
        const int32_t id = id_of[j];
        if (id < 0) continue;
        float prob = 0.f;
        bool first = true;
        for (int i = 0; i < p.k; ++i)
            if (id_of[i] == id) {
                if (i < j) first = false;
                prob += p_of[i];
            }
        if (first) from_f32(factor * (expf((z_of[j] - m) * inv_t) * inv_sum - prob), dz[id]);
    }
}

}  // namespace

size_t distill_workspace(int64_t n_rows, int32_t n_classes) { return 256; }

mgg_status_t launch_distill(const Distill &q, void *workspace, hipStream_t stream)
{
    DistillArgs p{};
    p.logits = q.logits; p.top_ids = q.top_ids; p.top_logits = q.top_logits; p.row_weight = q.row_weight; p.loss = q.loss; p.grad = q.grad;
    p.ld_logits = q.ld_logits; p.ld_ids = q.ld_ids; p.ld_top = q.ld_top; p.ld_grad = q.ld_grad;
    p.n_classes = q.n_classes; p.k = q.k; p.temperature = q.temperature; p.ids64 = q.id_type == MGG_I64; p.top_bf16 = q.top_dtype == MGG_BF16;
    const dim3 grid(static_cast<unsigned>(q.n_rows)), block(kThreads);
    const bool in16 = q.logits_dtype == MGG_BF16, out16 = q.grad ? q.grad_dtype == MGG_BF16 : in16;
    if (in16 && out16) hipLaunchKernelGGL((distill_row_kernel<Bf16, Bf16>), grid, block, 0, stream, p);
    else if (in16) hipLaunchKernelGGL((distill_row_kernel<Bf16, float>), grid, block, 0, stream, p);
    else if (out16) hipLaunchKernelGGL((distill_row_kernel<float, Bf16>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((distill_row_kernel<float, float>), grid, block, 0, stream, p);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? MGG_OK : hip_fail(e, "distillation kernel launch");
}

}  // namespace mgg
