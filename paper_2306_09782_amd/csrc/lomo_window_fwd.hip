// Forward of softmax attention with a sliding window and sinks over packed sequences, query heads sharing key heads in groups.
//
//   S_ij = q_i . k_j / sqrt(d) for the keys j <= i with i - j < window or j < sinks,  lse_i = log sum_j exp(S_ij),
//   o_i = sum_j exp(S_ij - lse_i) v_j
//
// One workgroup per (128 queries, head) walks the pairs of key and value tiles (64 keys) that the window of its queries reaches, the
// tile of the sinks first where that is left of them; one pass with a running maximum and sum.  The keys of the even and of the odd halves of
// the tiles have a maximum, a sum and an accumulator of their own (see lomo_attention_fwd.hip: less is rounded away), put together at
// the end.  Workgroups are numbered so that the heads of a group and neighbouring queries run on one XCD at a time.  Probabilities are
// rounded to fp16 relative to the running maximum, as the matrix cores take them; sums and accumulators are fp32; o is rounded once.
// Deterministic, and independent of what else is in the batch.
//
// A key that the mask hides from a query adds nothing to it, whatever its v holds: blocks that a mask cuts look for inf and NaN and
// take those out of the product, adding them to the queries that do see them.
#include "lomo_window_common.h"

namespace lomo {

namespace win {

struct FwdArgs {
    Batch b;
    const uint16_t* qkv;      // [T x (h + 2 g) D]
    uint16_t* o;              // [T x h D]
    float* lse;               // [T x h]
    int numbers, total;       // of 128-row pieces, of workgroups
};

}  // namespace win

template <int D>
__global__ __launch_bounds__(256, 2) void window_attention_forward_kernel(win::FwdArgs a) {
    using namespace win;
    extern __shared__ __attribute__((aligned(256))) uint16_t smem[];      // two pairs of tiles: K, V
    constexpr float C2 = SCALE<D> * LOG2E;

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, lh = lane >> 5;
    const uint32_t lds0 = (uint32_t)(uintptr_t)smem;
    const int window = a.b.window, sinks = a.b.sinks;

    // order: key heads, pieces, the heads of the group
    const int place = place_of_block(a.total), r = a.b.h / a.b.g;
    const int kv = place / (a.numbers * r), rest = place - kv * a.numbers * r;
    const int number = rest / r, n = kv * r + (rest - number * r);
    const int seq = sequence_of(a.b, number, ROWS, 1);
    if (seq < 0) return;
    const Rows s = rows_of(a.b, seq);
    const int nb = (s.len + ROWS - 1) / ROWS, at = number - first_piece(a.b, seq, ROWS, 1);
    if (at >= nb) return;
    const int q0 = (nb - 1 - at) * ROWS, qw = q0 + 32 * wave;      // the longest walks first
    const bool active = qw < s.len;
    const int query = qw + l32;

    const int64_t ld = (int64_t)(a.b.h + 2 * a.b.g) * D;
    const uint16_t* gq = a.qkv + (int64_t)s.start * ld + (int64_t)n * D;
    const uint16_t* gk = a.qkv + (int64_t)s.start * ld + (int64_t)(a.b.h + kv) * D;
    const uint16_t* gv = gk + (int64_t)a.b.g * D;

    // tiles of this workgroup: the sinks' where it is not among those of the window
    const int first = max(0, q0 - window + 1) / BLK, last = min(q0 + ROWS - 1, s.len - 1) / BLK;
    const int extra = sinks > 0 && first > 0 ? 1 : 0, tiles = last - first + 1 + extra;
    auto tile_at = [&](int i) { return i < extra ? 0 : first + i - extra; };

    const TileLoad<D> load(ld);
    const TileRead<D> rd(lds0);
    auto fetch = [&](int tile, int buf) {
        const int64_t off = (int64_t)tile * BLK * ld;
        const int rows = s.len - tile * BLK;
        load.issue(gk + off, rows, lds0 + (uint32_t)buf * (PAIR<D> * 2u), wave);
        load.issue(gv + off, rows, lds0 + (uint32_t)buf * (PAIR<D> * 2u) + TILE<D> * 2u, wave);
    };
    fetch(tile_at(0), 0);

    half8 fq[D / 16];
    if (active) load_fragments<D>(fq, gq + (int64_t)min(query, s.len - 1) * ld);

    // by half of the tiles; log2 domain; l_run is this lane's share (its half of the keys)
    constexpr int NC = D / 32;
    floatx16 accO[2][NC];
    float m_run[2], l_run[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        m_run[h] = -INFINITY;
        l_run[h] = 0.f;
#pragma unroll
        for (int i = 0; i < NC; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) accO[h][i][e] = 0.f;
    }

    auto scores = [&](const TileRead<D>& r0, floatx16& S) {
#pragma unroll
        for (int e = 0; e < 16; ++e) S[e] = 0.f;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) S = __builtin_amdgcn_mfma_f32_32x32x16_f16(r0.rows(0, ks), fq[ks], S, 0, 0, 0);
    };
    // What keys k0 .. k0 + 31 (S[e] <-> key k0 + 8 (e / 4) + 4 lh + e % 4) add to sum and output.
    auto half = [&](const TileRead<D>& r0, int k0, bool cut, floatx16& S, floatx16 (&O)[NC], float& m_run, float& l_run) {
        auto hidden = [&](int key) { return key > query || (query - key >= window && key >= sinks); };
        float scale = C2, bmax = -INFINITY;
        if (cut) {      // scaled and masked; the branch stays one
            scale = 1.f;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                float x = hidden(k0 + 8 * (e >> 2) + 4 * lh + (e & 3)) ? -INFINITY : S[e] * C2;
                asm volatile("" : "+v"(x));
                S[e] = x;
            }
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) bmax = fmaxf(bmax, S[e]);
        {
            const u32x2 sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(bmax), __float_as_uint(bmax), false, false);
            bmax = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
        }
        const float m_new = fmaxf(m_run, bmax * scale);
        const float m_ref = (m_new == -INFINITY) ? 0.f : m_new;      // a query that has seen no key yet
        float alpha = 1.f;
        if (__any(m_new > m_run)) {
            alpha = __builtin_amdgcn_exp2f(m_run - m_ref);
#pragma unroll
            for (int i = 0; i < NC; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) O[i][e] *= alpha;
            m_run = m_new;
        }
        float psum = 0.f;
        uint32_t pk[8];
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            const float p0 = __builtin_amdgcn_exp2f(fmaf(S[e], scale, -m_ref)), p1 = __builtin_amdgcn_exp2f(fmaf(S[e + 1], scale, -m_ref));
            psum += p0 + p1;
            pk[e >> 1] = pack2(p0, p1);
        }
        l_run = fmaf(l_run, alpha, psum);
        const bool dirty = cut && any_not_finite<D>(r0, TILE<D>);
        // o^T[column][query] += v^T[column][key] p^T[key][query], 16 keys at a time
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            const half8 fp = fragment_of(pk, ks);
            if (dirty) {
#pragma unroll
                for (int i = 0; i < NC; ++i)
                    O[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(finite_or_zero(r0.columns(TILE<D>, i, ks)), fp, O[i], 0, 0, 0);
            } else {
#pragma unroll
                for (int i = 0; i < NC; ++i) O[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(r0.columns(TILE<D>, i, ks), fp, O[i], 0, 0, 0);
            }
        }
        if (dirty) {      // what is not finite, to the queries that see its key
            const uint32_t block = r0.row_rd - 2u * (uint32_t)(l32 * D + ((8 * lh) ^ (swz<D>(l32) << 3))) + 2u * TILE<D>;
#pragma nounroll
            for (int key = 0; key < 32; ++key) {
#pragma unroll
                for (int i = 0; i < NC; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int c = 32 * i + 8 * (e >> 2) + 4 * lh + (e & 3);
                        const float x = (float)*(__attribute__((address_space(3))) const _Float16*)(block + 2u * (uint32_t)(key * D + (c ^ (swz<D>(key) << 3))));
                        if (not_finite(x) && !hidden(k0 + key)) O[i][e] += x;
                    }
            }
        }
    };

    for (int it = 0; it < tiles; ++it) {
        const int buf = it & 1, k0 = tile_at(it) * BLK;
        // the tiles have landed; everybody is done with the other pair
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (it + 1 < tiles) fetch(tile_at(it + 1), buf ^ 1);      // in flight while this pair is multiplied
        if (!active) continue;
        const Seen s0 = seen(qw, k0, window, sinks), s1 = seen(qw, k0 + 32, window, sinks);
        const TileRead<D> r0 = rd.at(buf * PAIR<D>), r1 = rd.at(buf * PAIR<D> + 32 * D);
        floatx16 S0, S1;
        if (s0 != NONE) scores(r0, S0);
        if (s1 != NONE) scores(r1, S1);
        if (s0 != NONE) half(r0, k0, s0 == SOME, S0, accO[0], m_run[0], l_run[0]);
        if (s1 != NONE) half(r1, k0 + 32, s1 == SOME, S1, accO[1], m_run[1], l_run[1]);
    }

    // ---- the two halves' common maximum and total sum (every query sees itself), then o
    if (!active) return;
    float l[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const u32x2 sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run[h]), __float_as_uint(l_run[h]), false, false);
        l[h] = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    }
    const float mt = fmaxf(m_run[0], m_run[1]);
    const float e0 = __builtin_amdgcn_exp2f(m_run[0] - mt), e1 = __builtin_amdgcn_exp2f(m_run[1] - mt);
    const float lt = fmaf(l[0], e0, l[1] * e1);
    const float f0 = e0 / lt, f1 = e1 / lt;
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) accO[0][i][e] = fmaf(accO[0][i][e], f0, accO[1][i][e] * f1);
    const bool own = query < s.len;
    const int64_t t = (int64_t)s.start + query;
    store_rows(accO[0], own ? a.o + (t * a.b.h + n) * D : nullptr);
    if (own && lh == 0) a.lse[t * a.b.h + n] = (mt + __builtin_amdgcn_logf(lt)) * LN2;
}

int64_t window_attention_pieces(int64_t T, int64_t B) { return win::pieces(T, B, win::ROWS, 1); }

template <int D>
static hipError_t launch_forward_of(const win::FwdArgs& a, hipStream_t st) {
    auto kern = window_attention_forward_kernel<D>;
    constexpr int lds = 2 * win::PAIR<D> * 2;
    static const hipError_t cfg = allow_dynamic_lds(kern, lds);
    if (cfg != hipSuccess) return cfg;
    hipLaunchKernelGGL(kern, dim3((unsigned)a.total), dim3(256), lds, st, a);
    return hipGetLastError();
}

hipError_t launch_window_attention_forward(const uint16_t* qkv, uint16_t* o, float* lse, const int32_t* off, int64_t T, int64_t B, int64_t h,
                                           int64_t g, int64_t d, int64_t window, int64_t sinks, hipStream_t st) {
    win::FwdArgs a;
    a.b = {off, (int)T, (int)B, (int)h, (int)g, (int)window, (int)sinks};
    a.qkv = qkv; a.o = o; a.lse = lse;
    a.numbers = (int)window_attention_pieces(T, B);
    a.total = (int)(a.numbers * h);
    return d == 128 ? launch_forward_of<128>(a, st) : launch_forward_of<64>(a, st);
}

}  // namespace lomo
