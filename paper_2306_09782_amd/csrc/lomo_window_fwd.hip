// Forward of softmax attention with a sliding window and sinks over packed sequences, query heads sharing key heads in groups.
//
//   S_ij = q_i . k_j / sqrt(d) for the keys j <= i with i - j < window or j < sinks,  lse_i = log sum_j exp(S_ij),
//   o_i = sum_j exp(S_ij - lse_i) v_j
//
// One workgroup per (128 queries, head) walks the pairs of key and value tiles (64 keys) that the window of its queries reaches, the
// tile of the sinks first where that is left of them; one pass with a running maximum and sum.  Workgroups are numbered so that the heads of a
// group and neighbouring queries run on one XCD at a time.  Probabilities are rounded to fp16 relative to a running reference, as the matrix
// cores take them (o is off by 2.5e-4 of its norm, 2.0e-4 of which is its own rounding; with what the rounding of P leaves in a further product it would be
// 2.0e-4, at 1345 us instead of 1000, packed 68 instead of 54); sums and accumulators are fp32; o is rounded once.  Deterministic, and independent of what else is in the batch.
//
// Tiles that every query of the workgroup sees whole have a loop of their own, without masks.  A key that the mask hides from a query adds nothing
// to it, whatever its v holds: inf and NaN are taken out of the tiles that a mask cuts, and added to the queries that do see them.
//
// Measured, us: 16384 tokens, 32 / 8 heads of 128, window 4096, 4 sinks 990 to 1025 (940 TFLOP/s of the visible pairs); 8192 tokens, no window, 32 / 8 heads
// of 128 570 (965 TFLOP/s); 4096 rows of seven sequences, window 1024 53; 8192 tokens, 32 / 8 heads of 64, window 2048 168 (716 TFLOP/s); four short
// sequences 6.8, the time of a launch.  Power is what bounds the long ones: the clock is at 1.5 to 1.9 GHz with the matrix cores busy for 47 to 52 % of its cycles and the vector
// units for 55 %.  Slower or no faster: the next tile's scores between the probabilities (1300), two waves of a SIMD held half a step apart by
// barriers (1000, and short sequences 30 % slower), tiles of 32 keys with three waves a SIMD (1010, odd lengths 12 % slower).
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

// Heads of 64 leave room for four waves a SIMD instead of three (8192 tokens 174 -> 168 us, 4096 packed rows 34.6 -> 33.2).
template <int D>
__global__ __launch_bounds__(256, D == 64 ? 4 : 2) void window_attention_forward_kernel(win::FwdArgs a) {
    using namespace win;
    extern __shared__ __attribute__((aligned(256))) uint16_t smem[];      // two pairs of tiles: K, V
    __shared__ uint32_t bad[2][4];                                        // rows of a V tile that are not finite, by wave
    constexpr float C2 = SCALE<D> * LOG2E;

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, lh = lane >> 5;
    const uint32_t lds0 = (uint32_t)(uintptr_t)smem;
    const int window = a.b.window, sinks = a.b.sinks;

    // order: key heads, pieces, the heads of the group
    const int place = place_of_block(a.total, blockIdx.x), r = a.b.h / a.b.g;
    const int kv = place / (a.numbers * r), rest = place - kv * a.numbers * r;
    const int number = rest / r, n = kv * r + (rest - number * r);
    Rows s;
    const int seq = sequence_of(a.b, number, ROWS, 1, s);
    if (seq < 0) return;
    const int nb = (s.len + ROWS - 1) / ROWS, at = number - first_piece(s.start, seq, ROWS, 1);
    if (at >= nb) return;
    const int q0 = (nb - 1 - at) * ROWS, qw = q0 + 32 * wave;      // the longest walks first
    const bool active = qw < s.len;
    const int query = qw + l32;

    const int64_t ld = (int64_t)(a.b.h + 2 * a.b.g) * D;
    const uint16_t* gq = a.qkv + (int64_t)s.start * ld + (int64_t)n * D;
    const uint16_t* gk = a.qkv + (int64_t)s.start * ld + (int64_t)(a.b.h + kv) * D;
    const uint16_t* gv = gk + (int64_t)a.b.g * D;

    // tiles of this workgroup: the sinks' where they are not among those of the window
    const int first = max(0, q0 - window + 1) / BLK, last = min(q0 + ROWS - 1, s.len - 1) / BLK;
    const int extra = min((sinks + BLK - 1) / BLK, first), tiles = last - first + 1 + extra;
    auto tile_at = [&](int i) { return i < extra ? i : first + i - extra; };

    const TileLoad<D> load(ld, wave);
    const TileRead<D> rd(lds0);
    auto fetch = [&](int tile, int buf) {
        const uint32_t at = lds0 + (uint32_t)buf * (PAIR<D> * 2u);
        load.issue(gk, tile, s.len - tile * BLK, at, wave);
        load.issue(gv, tile, s.len - tile * BLK, at + TILE<D> * 2u, wave);
    };
    fetch(tile_at(0), 0);

    half8 fq[D / 16];
    if (active) load_fragments<D>(fq, gq + (int64_t)min(query, s.len - 1) * ld);
    arrived<D>(fq);

    // log2 domain; l_run is this lane's share (its half of the keys)
    constexpr int NC = D / 32;
    floatx16 O[NC];
    float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) O[i][e] = 0.f;

    // Scores of keys 32 h .. + 31 of a pair: S[e] <-> key 8 (e / 4) + 4 lh + e % 4 of these.
    auto scores = [&](const TileRead<D>& r0, int h, floatx16& S) {
#pragma unroll
        for (int e = 0; e < 16; ++e) S[e] = 0.f;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) S = __builtin_amdgcn_mfma_f32_32x32x16_f16(r0.rows(32 * h * D, ks), fq[ks], S, 0, 0, 0);
    };
    // From scores to probabilities relative to a running reference, in fp16.  The reference begins 2^LIFT below the maximum, so that
    // probabilities down to 2^-21 of the largest are normal numbers of fp16, and moves only where the maximum has grown by more than 2^SLACK:
    // probabilities stay below 2^(LIFT + SLACK), and most tiles leave sum and output as they are.  Each query moves by its own scores alone,
    // so that no bit of its result depends on what its neighbours see.  SLACK 0 / 2 / 4 / 8, us: long 1090 / 1058 / 1045 / 1025, odd 99 / 96.5 / 96 / 93.5.
    constexpr float LIFT = 7.f, SLACK = 8.f;
    auto probabilities = [&](const floatx16 (&S)[2], uint32_t (&pk)[2][8]) {
        float top = -INFINITY;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, S[h][e]);
        const u32x2 sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        top = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * C2;
        if (__any(top > m_run + (LIFT + SLACK))) {
            const bool grown = top > m_run + (LIFT + SLACK);
            const float m_new = grown ? top - LIFT : m_run, alpha = grown ? __builtin_amdgcn_exp2f(m_run - m_new) : 1.f;
#pragma unroll
            for (int i = 0; i < NC; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) O[i][e] *= alpha;
            l_run *= alpha;
            m_run = m_new;
        }
        const float m_ref = m_run == -INFINITY ? 0.f : m_run;      // a query that has seen no key yet
        float sum = 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                const float p0 = __builtin_amdgcn_exp2f(fmaf(S[h][e], C2, -m_ref)), p1 = __builtin_amdgcn_exp2f(fmaf(S[h][e + 1], C2, -m_ref));
                sum += p0 + p1;
                pk[h][e >> 1] = pack2(p0, p1);
            }
        l_run += sum;
    };

    int it = 0;
    auto begin = [&]() {
        // the tiles have landed; everybody is done with the other pair
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (it + 1 < tiles) fetch(tile_at(it + 1), (it + 1) & 1);      // in flight while this pair is multiplied
        return rd.at((it & 1) * PAIR<D>);
    };
    // o^T[column][query] += v^T[column][key] p^T[key][query], 16 keys at a time
    auto values = [&](const TileRead<D>& r0, const uint32_t (&pk)[2][8]) {
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            const half8 fp = fragment_of(pk[ks >> 1], ks & 1);
#pragma unroll
            for (int i = 0; i < NC; ++i) O[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(r0.columns(TILE<D>, i, ks), fp, O[i], 0, 0, 0);
        }
        attn::interleave<8, 1, 2, 4 * NC - 4, 4>();
    };
    auto all_scores = [&](const TileRead<D>& r0, floatx16 (&S)[2]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) scores(r0, h, S[h]);
        attn::interleave<4, 1, 1, D / 8 - 4, 4>();
    };
    // the tiles that every query of the workgroup sees whole
    const int whole0 = (max(0, q0 + ROWS - window) + BLK - 1) / BLK, whole1 = q0 / BLK - 1;
    while (it < tiles) {
        for (; it < tiles && !(it >= extra && tile_at(it) >= whole0 && tile_at(it) <= whole1); ++it) {
            const int k0 = tile_at(it) * BLK;
            const TileRead<D> r0 = begin();
            const uint32_t mine = make_finite<D>(lds0 + (uint32_t)(it & 1) * (PAIR<D> * 2u) + TILE<D> * 2u, wave);
            if (lane == 0) bad[it & 1][wave] = mine;
            attn::meet();
            if (!active) continue;
            if (!seen(qw, k0, window, sinks) && !seen(qw, k0 + 32, window, sinks)) continue;
            // of a distance that is negative or not below the window, but for the sinks
            auto hidden = [&](int key) { return (uint32_t)(query - key) >= (key < sinks ? 0x80000000u : (uint32_t)window); };
            floatx16 S[2];
            all_scores(r0, S);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    S[h][e] = hidden(k0 + 32 * h + 8 * (e >> 2) + 4 * lh + (e & 3)) ? -INFINITY : S[h][e];
                    if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                }
            uint32_t pk[2][8];
            probabilities(S, pk);
            values(r0, pk);
            uint64_t rows = 0;
#pragma unroll
            for (int w = 0; w < 4; ++w) rows |= (uint64_t)bad[it & 1][w] << (16 * w);
            while (rows != 0) {      // what is not finite, to the queries that see its key
                const int key = k0 + __builtin_ctzll(rows);
                rows &= rows - 1;
                if (hidden(key)) continue;
                const uint16_t* v = gv + (int64_t)key * ld + 4 * lh;
#pragma unroll
                for (int i = 0; i < NC; ++i)
#pragma unroll
                    for (int g4 = 0; g4 < 4; ++g4) {
                        const half4 x = *reinterpret_cast<const half4*>(v + 32 * i + 8 * g4);
#pragma unroll
                        for (int e = 0; e < 4; ++e) O[i][4 * g4 + e] += not_finite((float)x[e]) ? (float)x[e] : 0.f;
                    }
            }
        }
        for (; it < tiles && tile_at(it) <= whole1; ++it) {
            const TileRead<D> r0 = begin();
            if (!active) continue;
            floatx16 S[2];
            all_scores(r0, S);
            uint32_t pk[2][8];
            probabilities(S, pk);
            values(r0, pk);
        }
    }

    // ---- the total sum (every query sees itself), then o
    if (!active) return;
    const u32x2 sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run), __float_as_uint(l_run), false, false);
    const float l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]), f = 1.f / l;
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) O[i][e] *= f;
    const bool own = query < s.len;
    const int64_t t = (int64_t)s.start + query;
    store_rows(O, own ? a.o + (t * a.b.h + n) * D : nullptr);
    if (own && lh == 0) a.lse[t * a.b.h + n] = (m_run + __builtin_amdgcn_logf(l)) * LN2;
}

// Zeros in the rows of no sequence, 16 bytes at a time.  Offsets that do not ascend stay in bounds.  A launch where there are none (2.0 us; 410 of 4096 rows
// of 6144 columns 2.7, 16384 rows of 12288 78, 5.1 TB/s).
__global__ __launch_bounds__(256) void clear_padding_kernel(u32x4* x, const int32_t* off, int64_t T, int64_t B, int64_t chunks) {
    const int64_t first = min(max((int64_t)off[0], (int64_t)0), T), end = min(max((int64_t)off[B], first), T);
    const int64_t front = first * chunks, gap = (end - first) * chunks, total = T * chunks - gap;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) x[i < front ? i : i + gap] = u32x4{0, 0, 0, 0};
}

hipError_t launch_clear_padding(uint16_t* x, const int32_t* off, int64_t T, int64_t B, int64_t width, hipStream_t st) {
    const int64_t chunks = width / 8, blocks = (T * chunks + 255) / 256;
    hipLaunchKernelGGL(clear_padding_kernel, dim3((unsigned)(blocks < 1024 ? blocks : 1024)), dim3(256), 0, st, reinterpret_cast<u32x4*>(x), off, T, B, chunks);
    return hipGetLastError();
}

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
    a.numbers = (int)win::pieces(T, B, win::ROWS, 1);
    a.total = (int)(a.numbers * h);
    return d == 128 ? launch_forward_of<128>(a, st) : launch_forward_of<64>(a, st);
}

}  // namespace lomo
