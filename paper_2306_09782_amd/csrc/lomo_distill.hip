// Distillation from a teacher that is known by its top logits, mixed with the cross-entropy of the target: token losses and logit gradient.
//
//   p = softmax of the listed teacher logits / tau,   q = softmax(z / tau)
//   loss = (1 - w) (lse(z) - z_target) + w tau^2 sum_k p_k (log p_k - log q_{id k})
//   dz_j = s [(1 - w) (softmax(z)_j - [j = target]) + w tau (q_j - sum of the p_k whose id is j)]
//
// One workgroup per token.  Bytes bound it: the row is read once, into registers where it fits (up to 163840 columns), and its
// sums of exponentials are formed while it arrives, each thread relative to the largest of its first eight columns: nothing
// overflows below 2^100, and a thread that meets a larger one starts again from there.  Then the gradient; then the target's and the
// listed columns once more, where 1 - p and q - p are formed without cancellation of rounded values.  An id that is listed twice is
// written once, by its first entry, with the sum of their p in order.  Exponentials are of base 2 with the reference inside the
// multiply-add.  fp32 arithmetic, one rounding, no atomics.
//
// Measured, us: 4096 x 32008, 64 listed 108 (524 MB, 4.9 TB/s; a large copy reaches 5.2), 4001 x 131080, 127 listed 475 (4.4 TB/s: one workgroup to a
// CU), 37 x 32000 11, where a row's way through memory and four meetings of its workgroup are the time.  Each listed column is compared with all ids at
// the end of its row: 4096 x 32008 with 64 / 256 / 1024 listed 120 / 157 / 869 (call after call on the same buffers).  Reading the row three times: 181, 864, 18.
#include "lomo_kernels.h"

namespace lomo {

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

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
    float scale, tau, inv_tau, w;
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
__device__ __forceinline__ float largest(half8 x) {
    _Float16 m[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) m[e] = __builtin_fmaxf16(x[e], x[e + 4]);
    return fmaxf(fmaxf((float)m[0], (float)m[1]), fmaxf((float)m[2], (float)m[3]));
}

// A share of a row: sums of 2^(z c - k) for the two c (of the logits as they are, and at the temperature); k = m c as rounded, so that sums
// with different m are moved by the difference of two numbers and not by that of two roundings.
template <bool BOTH>
struct Sums {
    float m, kh, ks, hard = 0.f, soft = 0.f;
    __device__ __forceinline__ Sums(float m, float ch, float cs) : m(m) { refer(ch, cs); }
    __device__ __forceinline__ void refer(float ch, float cs) {
        kh = m * ch;
        ks = m * cs;
        asm volatile("" : "+v"(kh), "+v"(ks));      // rounded here, not inside what uses them
    }
    __device__ __forceinline__ void move_to(float m_new, float ch, float cs) {
        const float h = kh, s = ks;
        m = m_new;
        refer(ch, cs);
        if constexpr (BOTH) hard *= __builtin_amdgcn_exp2f(h - kh);
        soft *= __builtin_amdgcn_exp2f(s - ks);
    }
    __device__ __forceinline__ void add(half8 x, float ch, float cs) {
        const float top = largest(x);
        if (__any((top - m) * fmaxf(ch, cs) > 100.f)) move_to(fmaxf(m, top), ch, cs);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (BOTH) hard += __builtin_amdgcn_exp2f(fmaf((float)x[e], ch, -kh));
            soft += __builtin_amdgcn_exp2f(fmaf((float)x[e], cs, -ks));
        }
    }
};

// Row of V columns by NT threads, CH chunks of 8 columns each in registers; CH = 0: any V, read again for the gradient.  BOTH: the two terms
// need exponentials of their own (0 < w < 1 and tau != 1); otherwise one is enough: at the temperature where the soft term has a
// weight, as they are where it has none.  z and dz may be the same buffer.
template <int NT, int CH, bool BOTH>
__global__ __launch_bounds__(NT, CH > 8 ? 4 : 8) void distill_kernel(Distill a) {
    constexpr int WAVES = NT / 64;
    extern __shared__ float lds[];      // teacher's logit and then p, z and id of the listed columns and of the target (the last)
    __shared__ float red[5][WAVES];
    float* p = lds;
    float* zk = lds + a.K + 1;
    int* id = reinterpret_cast<int*>(lds + 2 * (a.K + 1));
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t t = blockIdx.x;
    const uint16_t* row = a.z + t * a.V;
    uint16_t* out = a.dz + t * a.V;
    const int chunks = (int)(a.V >> 3);
    // the listed columns of this thread: the first is on its way while the row arrives
    auto listed = [&](int k) { return a.ids[t * a.K + k]; };
    auto logit = [&](int k) { return (float)reinterpret_cast<const _Float16*>(a.teacher)[t * a.K + k]; };
    int own = (int)threadIdx.x < a.K ? listed(threadIdx.x) : -1;
    const float own_logit = (int)threadIdx.x < a.K ? logit(threadIdx.x) : 0.f;
    const int target = a.target[t];
    if (target < 0 || target >= a.V) {      // not counted
        if (threadIdx.x == 0) a.loss[t] = 0.f;
        for (int c = threadIdx.x; c < chunks; c += NT) *reinterpret_cast<half8*>(out + (int64_t)c * 8) = half8{};
        return;
    }
    const float scale = a.scale_dev != nullptr ? *a.scale_dev : a.scale;
    const float ch = LOG2E, cs = BOTH || a.w > 0.f ? LOG2E / a.tau : LOG2E;

    half8 x[CH > 0 ? CH : 1];
    if constexpr (CH > 0) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = i * NT + (int)threadIdx.x;
            if (c < chunks) x[i] = __builtin_nontemporal_load(reinterpret_cast<const half8*>(row + (int64_t)c * 8));
        }
    }
    // the student's logit of a listed column, read before anything is overwritten; an id outside [0, V) is not listed
    auto column = [&](int i) { return i >= 0 && i < a.V ? (float)reinterpret_cast<const _Float16*>(row)[i] : 0.f; };
    if ((int)threadIdx.x == a.K) own = target;
    const float own_z = column(own);
    constexpr float LOWEST = -65504.f;      // finite from the start: masked logits may be -inf
    float m0 = LOWEST;
    if (CH > 0 && (int)threadIdx.x < chunks) m0 = fmaxf(m0, largest(x[0]));
    Sums<BOTH> s(m0, ch, cs);
    if constexpr (CH > 0) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            if (i * NT + (int)threadIdx.x < chunks) s.add(x[i], ch, cs);
            __builtin_amdgcn_sched_barrier(0);
        }
    } else {
        for (int c = threadIdx.x; c < chunks; c += NT) s.add(*reinterpret_cast<const half8*>(row + (int64_t)c * 8), ch, cs);
    }
    float top = -INFINITY;
    auto keep = [&](int k, int i, float z, float l) {
        const bool in = i >= 0 && i < a.V;
        p[k] = k < a.K && in ? l : -INFINITY;
        zk[k] = z;
        id[k] = in ? i : -1;
        top = fmaxf(top, p[k] != p[k] ? INFINITY : p[k]);      // a maximum passes over NaN, which is listed all the same
    };
    if ((int)threadIdx.x <= a.K) keep(threadIdx.x, own, own_z, own_logit);
    for (int k = threadIdx.x + NT; k <= a.K; k += NT) {
        const int i = k < a.K ? listed(k) : target;
        keep(k, i, column(i), k < a.K ? logit(k) : 0.f);
    }
    {
        const float m = wave_max(s.m);
        s.move_to(m, ch, cs);
        s.soft = wave_sum(s.soft);
        if constexpr (BOTH) s.hard = wave_sum(s.hard);
        top = wave_max(top);
        if (lane == 0) {
            red[0][wave] = m;
            red[1][wave] = s.soft;
            red[2][wave] = s.hard;
            red[3][wave] = top;
        }
    }
    __syncthreads();
    // the waves' shares, one to a lane
    const bool has = lane < WAVES;
    const float m = wave_max(has ? red[0][lane] : LOWEST);
    top = wave_max(has ? red[3][lane] : -INFINITY);
    Sums<BOTH> all(has ? red[0][lane] : LOWEST, ch, cs);
    all.soft = has ? red[1][lane] : 0.f;
    all.hard = has ? red[2][lane] : 0.f;
    all.move_to(m, ch, cs);
    all.soft = wave_sum(all.soft);
    if constexpr (BOTH) all.hard = wave_sum(all.hard);
    const float kh = all.kh, ks = all.ks, soft = all.soft, hard = BOTH ? all.hard : all.soft;
    const bool taught = a.w > 0.f && top > -INFINITY;      // otherwise it has no weight, or nothing is listed: the soft term is left out
    const float w = taught ? a.w : 0.f, as = scale * w * a.tau / soft, ah = scale * (1.f - a.w) / hard;
    const float alone = as + ah;              // of the one exponential
    {
        float sum = 0.f;
        for (int k = threadIdx.x; k < a.K; k += NT) {
            const float x = (p[k] - top) * a.inv_tau;      // of the difference, which is exact or nearly so: the logits themselves may be long at a small tau
            p[k] = x;
            sum += taught ? expf(x) : 0.f;
        }
        sum = wave_sum(sum);
        if (lane == 0) red[4][wave] = sum;
    }
    // the gradient but for the target and the teacher's shares
    auto gradient = [&](half8 z) {
        half8 o;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float es = __builtin_amdgcn_exp2f(fmaf((float)z[e], cs, -ks));
            if constexpr (BOTH) o[e] = (_Float16)fmaf(as, es, ah * __builtin_amdgcn_exp2f(fmaf((float)z[e], ch, -kh)));
            else o[e] = (_Float16)(alone * es);
        }
        return o;
    };
    __syncthreads();
    const float log_sum = logf(wave_sum(has ? red[4][lane] : 0.f)), log_soft = __builtin_amdgcn_logf(soft);
    float divergence = 0.f;
    for (int k = threadIdx.x; k < a.K; k += NT) {
        const float log_p = p[k] - log_sum, pk = taught ? expf(log_p) : 0.f;
        if (pk != 0.f) divergence += pk * (log_p - LN2 * (fmaf(zk[k], cs, -ks) - log_soft));
        p[k] = pk;
    }
    divergence = wave_sum(divergence);
    if (lane == 0) red[3][wave] = divergence;
    if constexpr (CH > 0) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = i * NT + (int)threadIdx.x;
            if (c < chunks) __builtin_nontemporal_store(gradient(x[i]), reinterpret_cast<half8*>(out + (int64_t)c * 8));
            __builtin_amdgcn_sched_barrier(0);
        }
    } else {
        for (int c = threadIdx.x; c < chunks; c += NT)
            *reinterpret_cast<half8*>(out + (int64_t)c * 8) = gradient(*reinterpret_cast<const half8*>(row + (int64_t)c * 8));
    }
    // p is whole, and every wave's part of the row is where other waves' stores find it: what follows replaces some of it
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const float sum = wave_sum(has ? red[3][lane] : 0.f);
    if (threadIdx.x == 0) {
        float l = w > 0.f ? w * a.tau * a.tau * sum : 0.f;
        if (a.w != 1.f) l += (1.f - a.w) * LN2 * (__builtin_amdgcn_logf(hard) - fmaf(zk[a.K], ch, -kh));      // no difference of long numbers
        a.loss[t] = l;
    }
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
        const float es = __builtin_amdgcn_exp2f(fmaf(zk[k], cs, -ks)), eh = BOTH ? __builtin_amdgcn_exp2f(fmaf(zk[k], ch, -kh)) : es;
        reinterpret_cast<_Float16*>(out)[i] = (_Float16)fmaf(ah, eh - (i == target ? hard : 0.f), as * (es - pk * soft));
    }
}

template <int NT, int CH>
hipError_t launch(const Distill& a, int64_t T, hipStream_t st) {
    const size_t lds = (size_t)(3 * (a.K + 1)) * 4;
    if (a.w > 0.f && a.w < 1.f && a.tau != 1.f) hipLaunchKernelGGL((distill_kernel<NT, CH, true>), dim3((unsigned)T), dim3(NT), lds, st, a);
    else hipLaunchKernelGGL((distill_kernel<NT, CH, false>), dim3((unsigned)T), dim3(NT), lds, st, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_distill(const uint16_t* z, const int32_t* ids, const uint16_t* teacher, const int32_t* target, float scale,
                          const float* scale_dev, float tau, float w, float* loss, uint16_t* dz, int64_t T, int64_t V, int64_t K,
                          hipStream_t st) {
    const Distill a = {z, ids, teacher, target, scale_dev, loss, dz, V, (int)K, scale, tau, 1.f / tau, w};
    const int64_t chunks = V / 8;
    // The smallest workgroup whose registers hold the row, so that several share a CU and one computes while another reads.  us, with the next larger instead:
    // 8192 x 8000 62 / 88 (256 and 512 threads), 4096 x 32008 108 / 161 (512 threads of eight chunks, 1024 of four), 2048 x 60000 108 / 152 (eight
    // chunks, twenty).  Twenty are what 128 registers have room for.
    if (chunks <= 256 * 4) return launch<256, 4>(a, T, st);
    if (chunks <= 512 * 8) return launch<512, 8>(a, T, st);
    if (chunks <= 1024 * 8) return launch<1024, 8>(a, T, st);
    if (chunks <= 1024 * 20) return launch<1024, 20>(a, T, st);
    return launch<1024, 0>(a, T, st);
}

}  // namespace lomo
