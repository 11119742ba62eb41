// Rotary positions with several axes (time, height, width of images and video; text advances on all of them), and the same backwards.
//
//   y_c = x_c cos - x_{c + d/2} sin,   y_{c + d/2} = x_{c + d/2} cos + x_c sin,   cos, sin of row positions[axis of c][t], column c of the tables
//
// A thread has 8 neighbouring pairs of a token and turns them in several heads, so that the tables' values are read once for all of these; bytes
// bound it.  fp32 arithmetic, one rounding.
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
    uint8_t axis[128];
};

__global__ __launch_bounds__(NT) void rope_axes_kernel(RopeAxes a) {
    const int64_t i = (int64_t)blockIdx.x * NT + threadIdx.x;
    const int64_t t = i / a.chunks;
    const int c0 = (int)(i - t * a.chunks) * 8;
    if (t >= a.T) return;
    float co[8], si[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int64_t p = a.pos[a.axis[c0 + e] * a.T + t];
        const bool in = p >= 0 && p < a.P;      // any other position: the pair stays as it is
        co[e] = in ? a.cosv[p * a.half + c0 + e] : 1.f;
        si[e] = in ? a.sinv[p * a.half + c0 + e] * a.sign : 0.f;
    }
    const int n0 = blockIdx.y * a.per, n1 = min(a.heads, n0 + a.per);
    const uint16_t* px = a.x + t * a.ldx + c0;
    uint16_t* py = a.y + t * a.ldy + c0;
    for (int n = n0; n < n1; ++n) {
        const int64_t at = (int64_t)n * 2 * a.half;
        const half8 x1 = *reinterpret_cast<const half8*>(px + at), x2 = *reinterpret_cast<const half8*>(px + at + a.half);
        half8 y1, y2;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float u = (float)x1[e], v = (float)x2[e];
            y1[e] = (_Float16)fmaf(-v, si[e], u * co[e]);
            y2[e] = (_Float16)fmaf(u, si[e], v * co[e]);
        }
        *reinterpret_cast<half8*>(py + at) = y1;
        *reinterpret_cast<half8*>(py + at + a.half) = y2;
    }
}

}  // namespace

hipError_t launch_rope_axes(const uint16_t* x, int64_t ldx, uint16_t* y, int64_t ldy, const float* cosv, const float* sinv, int64_t P,
                            const int32_t* pos, const uint8_t* axis, int64_t T, int64_t heads, int64_t d, bool inverse, hipStream_t st) {
    RopeAxes a;
    a.x = x; a.y = y; a.ldx = ldx; a.ldy = ldy; a.T = T; a.cosv = cosv; a.sinv = sinv; a.pos = pos; a.P = P;
    a.heads = (int)heads; a.half = (int)(d / 2); a.chunks = (int)(d / 16);
    a.per = 8;
    a.sign = inverse ? -1.f : 1.f;
    for (int64_t c = 0; c < d / 2; ++c) a.axis[c] = axis[c];
    const dim3 grid((unsigned)((T * a.chunks + NT - 1) / NT), (unsigned)((heads + a.per - 1) / a.per));
    hipLaunchKernelGGL(rope_axes_kernel, grid, dim3(NT), 0, st, a);
    return hipGetLastError();
}

}  // namespace lomo
