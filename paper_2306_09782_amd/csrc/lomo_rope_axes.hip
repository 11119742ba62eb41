// Rotary positions with several axes (time, height, width of images and video; text advances on all of them), and the same backwards.
//
//   y_c = x_c cos - x_{c + d/2} sin,   y_{c + d/2} = x_{c + d/2} cos + x_c sin,   cos, sin of row positions[axis of c][t], column c of the tables
//
// A thread has 8 neighbouring pairs of a token and turns them in several heads, four at a time in flight, so that the tables' values are
// read once for all of these.  fp32 arithmetic, one rounding.
//
// Bytes bound it.  Measured: 16384 tokens, 40 heads of 128 66.8 us (344 MB, 5.1 TB/s; a large copy reaches 5.2), 4096 tokens 14.6, 333 tokens, 10 heads
// of 64 4.6.
#include "lomo_kernels.h"

namespace lomo {

namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
constexpr int NT = 256;

struct RopeAxes {
    const uint16_t* x;
    uint16_t* y;
    int64_t ldx, ldy, T;
    const float* cosv;      // [P x d / 2]
    const float* sinv;
    const int32_t* pos;     // [axes x T]
    int64_t P;
    int heads, per, half, chunks;      // per: heads of a thread; chunks: of 8 pairs in half a head
    float sign;
    uint32_t one_axis;      // the chunks whose pairs have the same axis, where the tables can be read by 16 bytes
    uint8_t axis[128];
};

__global__ __launch_bounds__(NT) void rope_axes_kernel(RopeAxes a) {
    const int64_t i = (int64_t)blockIdx.x * NT + threadIdx.x;
    const int64_t t = i / a.chunks;
    const int c0 = (int)(i - t * a.chunks) * 8;
    if (t >= a.T) return;
    const int n0 = blockIdx.y * a.per, n1 = min(a.heads, n0 + a.per);
    const uint16_t* px = a.x + t * a.ldx + c0;
    uint16_t* py = a.y + t * a.ldy + c0;
    constexpr int BATCH = 4;
    half8 x1[BATCH], x2[BATCH];
    auto load = [&](int n) {
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const int64_t at = (int64_t)min(n + k, n1 - 1) * 2 * a.half;
            x1[k] = *reinterpret_cast<const half8*>(px + at);
            x2[k] = *reinterpret_cast<const half8*>(px + at + a.half);
        }
    };
    load(n0);
    float co[8], si[8];
    if (a.one_axis >> (c0 >> 3) & 1) {
        const int64_t p = a.pos[a.axis[c0] * a.T + t];
        const bool in = p >= 0 && p < a.P;      // any other position: the pairs stay as they are
        const float4* pc = reinterpret_cast<const float4*>(a.cosv + (in ? p * a.half + c0 : 0));
        const float4* ps = reinterpret_cast<const float4*>(a.sinv + (in ? p * a.half + c0 : 0));
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const float4 c4 = in ? pc[g] : float4{1.f, 1.f, 1.f, 1.f}, s4 = in ? ps[g] : float4{0.f, 0.f, 0.f, 0.f};
            co[4 * g] = c4.x; co[4 * g + 1] = c4.y; co[4 * g + 2] = c4.z; co[4 * g + 3] = c4.w;
            si[4 * g] = s4.x; si[4 * g + 1] = s4.y; si[4 * g + 2] = s4.z; si[4 * g + 3] = s4.w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int64_t p = a.pos[a.axis[c0 + e] * a.T + t];
            const bool in = p >= 0 && p < a.P;
            co[e] = in ? a.cosv[p * a.half + c0 + e] : 1.f;
            si[e] = in ? a.sinv[p * a.half + c0 + e] : 0.f;
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) si[e] *= a.sign;
    for (int n = n0; n < n1; n += BATCH) {
        half8 y1[BATCH], y2[BATCH];
#pragma unroll
        for (int k = 0; k < BATCH; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float u = (float)x1[k][e], v = (float)x2[k][e];
                y1[k][e] = (_Float16)fmaf(-v, si[e], u * co[e]);
                y2[k][e] = (_Float16)fmaf(u, si[e], v * co[e]);
            }
        if (n + BATCH < n1) load(n + BATCH);
#pragma unroll
        for (int k = 0; k < BATCH; ++k)
            if (n + k < n1) {
                const int64_t at = (int64_t)(n + k) * 2 * a.half;
                *reinterpret_cast<half8*>(py + at) = y1[k];
                *reinterpret_cast<half8*>(py + at + a.half) = y2[k];
            }
    }
}

}  // namespace

hipError_t launch_rope_axes(const uint16_t* x, int64_t ldx, uint16_t* y, int64_t ldy, const float* cosv, const float* sinv, int64_t P,
                            const int32_t* pos, const uint8_t* axis, int64_t T, int64_t heads, int64_t d, bool inverse, hipStream_t st) {
    RopeAxes a;
    a.x = x; a.y = y; a.ldx = ldx; a.ldy = ldy; a.T = T; a.cosv = cosv; a.sinv = sinv; a.pos = pos; a.P = P;
    a.heads = (int)heads; a.half = (int)(d / 2); a.chunks = (int)(d / 16);
    // heads of a thread: as many as leave two workgroups for every CU, up to 8 (8 at any size / 4 at any size / this, us: 333 tokens, 10 heads of 64 5.6 / 5.0
    // / 4.6, 16384 tokens, 40 heads of 128 66.8 / 69.4 / 66.8)
    const int64_t blocks = (T * a.chunks + NT - 1) / NT;
    a.per = 8;
    while (a.per > 1 && blocks * ((heads + a.per - 1) / a.per) < 2 * cu_count()) a.per /= 2;
    a.sign = inverse ? -1.f : 1.f;
    for (int64_t c = 0; c < d / 2; ++c) a.axis[c] = axis[c];
    a.one_axis = 0;
    if (((reinterpret_cast<uintptr_t>(cosv) | reinterpret_cast<uintptr_t>(sinv)) & 15u) == 0)
        for (int c = 0; c < a.chunks; ++c) {
            bool same = true;
            for (int e = 1; e < 8; ++e) same = same && axis[8 * c + e] == axis[8 * c];
            if (same) a.one_axis |= 1u << c;
        }
    const dim3 grid((unsigned)blocks, (unsigned)((heads + a.per - 1) / a.per));
    hipLaunchKernelGGL(rope_axes_kernel, grid, dim3(NT), 0, st, a);
    return hipGetLastError();
}

}  // namespace lomo
