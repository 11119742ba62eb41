// Distillation from a teacher that is known by its top logits, mixed with the cross-entropy of the target: token losses and logit gradient.
//
//   p = softmax of the listed teacher logits / tau,   q = softmax(z / tau)
//   loss = (1 - w) (lse(z) - z_target) + w tau^2 sum_k p_k (log p_k - log q_{id k})
//   dz_j = s [(1 - w) (softmax(z)_j - [j = target]) + w tau (q_j - sum of the p_k whose id is j)]
//
// One workgroup per token: the maximum, both sums of exponentials, the gradient; then the target's and the listed columns again, where
// 1 - p and q - p are formed without cancellation of rounded values.  An id that is listed twice is written once, by its first entry, with the
// sum of their p in order.  fp32 arithmetic, one rounding, no atomics.
#include "lomo_kernels.h"

namespace lomo {

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
constexpr int NT = 256, WAVES = NT / 64;
constexpr float LOG2E = 1.4426950408889634f;

struct Distill {
    const uint16_t* z;
    const int32_t* ids;          // [T x K]
    const uint16_t* teacher;     // [T x K]
    const int32_t* target;       // [T]
    const float* scale_dev;      // read instead of `scale` when not null
    float* loss;
    uint16_t* dz;
    int64_t V;
    int K;
    float scale, tau, w;
};

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    return v;
}
__device__ __forceinline__ float block_max(float v, float* red) {
    v = wave_max(v);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    float total = red[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) total = fmaxf(total, red[i]);
    __syncthreads();
    return total;
}
__device__ __forceinline__ float block_sum(float v, float* red) {
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    float total = red[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) total += red[i];
    __syncthreads();
    return total;
}

// z and dz may be the same buffer.
__global__ __launch_bounds__(NT) void distill_kernel(Distill a) {
    extern __shared__ float lds[];      // p, z and id of the listed columns and of the target (the last)
    __shared__ float red[WAVES];
    float* p = lds;
    float* zk = lds + a.K + 1;
    int* id = reinterpret_cast<int*>(lds + 2 * (a.K + 1));
    const int64_t t = blockIdx.x;
    const uint16_t* row = a.z + t * a.V;
    uint16_t* out = a.dz + t * a.V;
    const int target = a.target[t];
    if (target < 0 || target >= a.V) {      // not counted
        if (threadIdx.x == 0) a.loss[t] = 0.f;
        for (int64_t c = (int64_t)threadIdx.x * 8; c < a.V; c += NT * 8) *reinterpret_cast<half8*>(out + c) = half8{};
        return;
    }
    const float scale = a.scale_dev != nullptr ? *a.scale_dev : a.scale, c2 = LOG2E / a.tau;

    // the teacher's probabilities; an id outside [0, V) is not listed
    float top = -INFINITY;
    for (int k = threadIdx.x; k <= a.K; k += NT) {
        const int i = k < a.K ? a.ids[t * a.K + k] : target;
        const bool in = i >= 0 && i < a.V;
        const float x = k < a.K && in ? (float)reinterpret_cast<const _Float16*>(a.teacher)[t * a.K + k] / a.tau : -INFINITY;
        id[k] = in ? i : -1;
        zk[k] = in ? (float)reinterpret_cast<const _Float16*>(row)[i] : 0.f;      // before anything is overwritten
        p[k] = x;
        top = fmaxf(top, x);
    }
    top = block_max(top, red);
    const bool taught = top > -INFINITY;      // otherwise nothing is listed and the soft term is left out
    float sum = 0.f;
    for (int k = threadIdx.x; k < a.K; k += NT) sum += taught ? expf(p[k] - top) : 0.f;
    const float teacher_lse = top + logf(block_sum(sum, red));

    float m = -INFINITY;
    for (int64_t c = (int64_t)threadIdx.x * 8; c < a.V; c += NT * 8) {
        const half8 x = *reinterpret_cast<const half8*>(row + c);
#pragma unroll
        for (int e = 0; e < 8; ++e) m = fmaxf(m, (float)x[e]);
    }
    m = block_max(m, red);
    float hard = 0.f, soft = 0.f;
    for (int64_t c = (int64_t)threadIdx.x * 8; c < a.V; c += NT * 8) {
        const half8 x = *reinterpret_cast<const half8*>(row + c);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = (float)x[e] - m;
            hard += __builtin_amdgcn_exp2f(d * LOG2E);
            soft += __builtin_amdgcn_exp2f(d * c2);
        }
    }
    hard = block_sum(hard, red);
    soft = block_sum(soft, red);

    const float w = taught ? a.w : 0.f, ah = scale * (1.f - a.w) / hard, as = scale * w * a.tau / soft;
    const float log_soft = logf(soft);
    float divergence = 0.f;
    for (int k = threadIdx.x; k < a.K; k += NT) {
        const float log_p = p[k] - teacher_lse, pk = taught ? expf(log_p) : 0.f;
        if (pk != 0.f) divergence += pk * (log_p - (zk[k] - m) / a.tau + log_soft);
        p[k] = pk;
    }
    divergence = block_sum(divergence, red);      // p is whole behind this
    if (threadIdx.x == 0) {
        float x = w * a.tau * a.tau * divergence;
        if (a.w != 1.f) x += (1.f - a.w) * (m - zk[a.K] + logf(hard));
        a.loss[t] = x;
    }
    for (int64_t c = (int64_t)threadIdx.x * 8; c < a.V; c += NT * 8) {
        const half8 x = *reinterpret_cast<const half8*>(row + c);
        half8 o;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = (float)x[e] - m;
            o[e] = (_Float16)fmaf(ah, __builtin_amdgcn_exp2f(d * LOG2E), as * __builtin_amdgcn_exp2f(d * c2));
        }
        *reinterpret_cast<half8*>(out + c) = o;
    }
    __syncthreads();      // the row is written; what follows replaces some of it
    for (int k = threadIdx.x; k <= a.K; k += NT) {
        const int i = id[k];
        if (i < 0) continue;
        float pk = 0.f;
        bool first = true;
        for (int j = 0; j < a.K; ++j) {
            if (id[j] != i) continue;
            first = first && j >= k;
            pk += p[j];
        }
        if (!first) continue;
        const float d = zk[k] - m;
        const float h = __builtin_amdgcn_exp2f(d * LOG2E) - (i == target ? hard : 0.f), s = __builtin_amdgcn_exp2f(d * c2) - pk * soft;
        reinterpret_cast<_Float16*>(out)[i] = (_Float16)fmaf(ah, h, as * s);
    }
}

}  // namespace

hipError_t launch_distill(const uint16_t* z, const int32_t* ids, const uint16_t* teacher, const int32_t* target, float scale,
                          const float* scale_dev, float tau, float w, float* loss, uint16_t* dz, int64_t T, int64_t V, int64_t K,
                          hipStream_t st) {
    const Distill a = {z, ids, teacher, target, scale_dev, loss, dz, V, (int)K, scale, tau, w};
    hipLaunchKernelGGL(distill_kernel, dim3((unsigned)T), dim3(NT), (size_t)(3 * (K + 1) * 4), st, a);
    return hipGetLastError();
}

}  // namespace lomo
