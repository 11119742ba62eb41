// Backward of softmax attention with a sliding window and sinks over packed sequences (the forward: lomo_window_fwd.hip), for the
// hand-on gradient of Algorithm 1.  Query i sees the keys j <= i with i - j < window or j < sinks:
//
//   P_ij = exp(q_i . k_j / sqrt(d) - lse_i),   dP_ij = do_i . v_j,   delta_i = do_i . o_i,   dS = P (dP - delta) / sqrt(d)
//   dq_i = sum_j dS_ij k_j;   dk_j = sum over the queries i of all heads of the group dS_ij q_i;   dv_j likewise of P_ij do_i
//
// Three deterministic kernels, no atomics.  The first: a workgroup per (128 queries, head) forms delta, walks the tiles of keys
// that the window reaches, and the sinks', and accumulates dq.  The second: a workgroup per (64 keys, key head) walks the query tiles
// whose window reaches the keys, for each head of the group, and accumulates dk and dv.  The sinks have queries beyond their window, up to
// the whole sequence: further workgroups of the second kernel sum over those, FAR_ROWS queries of all heads of a group each, into a
// slot of `sinks` fp32 rows in the workspace, where the sums over the window go too for these rows; the third adds the slots in order
// and rounds.  All recompute S, P, dP, dS in blocks of 32 x 32 per wave with the wave's own rows along the lanes.
//
// fp32 accumulation on the matrix cores.  P and dS pass through fp16 before the products that consume them; P is held times 2^15 there,
// so that the probabilities of a long window (2^-14 and less) keep all their bits, and dS times a power of two of its own row (below), so that
// gradients of any size do.  dq, dk, dv are rounded once.  Tiles that a mask cuts are
// made finite first, so that a pair which the mask hides adds nothing; a query that sees a key which is not finite has NaN in its gradient.
//
// Measured, us: 16384 tokens, 32 / 8 heads of 128, window 2048, 4 sinks 2130 (dq 800, dk and dv 1330; 605 TFLOP/s of the five products, 845 of
// the seven executed); 4096 rows of seven sequences, window 1024 192 to 198; 8192 tokens, 32 / 8 heads of 64, window 2048 635 (473 TFLOP/s); four short
// sequences 25.  Power bounds dq of the long ones: the clock falls to 1.8 GHz with the matrix cores busy for half of its cycles.  dk and dv have them busy for
// 36 % at 1.94 GHz and are bound by the bytes of their moving tiles: without tile loads they take 18 % less, and what takes stalls away changes
// nothing (three pairs of tiles in flight, one barrier a tile with the partner's half multiplied beside the next scores, no exponentials 1 %, no
// meeting of partners 1 %).  A packed batch is bound by its longest walk: two teams in a workgroup took it from 206 to 189 (short 29 -> 25; 16384 tokens,
// where there are walks enough, 2090 -> 2190).  Both teams on 128 keys and the same tiles: 2065 then, but 222 and 30, so the choice would be the
// sequence's: by its own length, window and group, since by the size of the call its bits would depend on its batch.
#include "lomo_window_common.h"

#include <algorithm>
#include <type_traits>

namespace lomo {

namespace win {

constexpr int FAR_ROWS = 512;      // 256 / 512 / 1024, us: long 2185 / 2160 / 2215, packed 194.5 / 192 / 194
constexpr float P_SCALE = 32768.f, P_LOG2 = 15.f;
template <int D>
constexpr float DS_SCALE = SCALE<D> / P_SCALE;      // of dP - delta where it meets P times P_SCALE

// dS passes through fp16 times 2^e, with an e for each query of dq and each key of dk.  It begins high and falls where a block has a dS beyond
// DS_TOP, to where the largest is 2^DS_TARGET .. 2^(DS_TARGET + 1); the sums fall with it.  So what is within 2^-21 of the largest that the row has met keeps all
// its bits, whatever the size of dO and v, and nothing overflows that the result holds.  A row's e follows from what the row sees alone.
constexpr int DS_FIRST = 60, DS_LAST = -60, DS_TARGET = 7;
constexpr float DS_TOP = 32768.f;
__device__ __forceinline__ float power_of_2(int n) { return __uint_as_float((uint32_t)(127 + n) << 23); }
// lower(n): e has fallen by n (0 for rows that stay).  A dS that is infinite before it is scaled stays so.
template <typename F>
__device__ __forceinline__ void keep_in_range(floatx16& dS, int& exponent, F&& lower) {
    float top = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) top = fmaxf(top, fabsf(dS[e]));
    if (__any(top > DS_TOP)) {
        const u32x2 sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        top = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
        const int n = top > DS_TOP && top < INFINITY ? min((int)(__float_as_uint(top) >> 23) - 127 - DS_TARGET, exponent - DS_LAST) : 0;
        const float f = power_of_2(-n);
#pragma unroll
        for (int e = 0; e < 16; ++e) dS[e] *= f;
        exponent -= n;
        lower(n);
    }
}
template <int N>
__device__ __forceinline__ void multiply_all(floatx16 (&x)[N], float f) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) x[i][e] *= f;
}
__device__ __forceinline__ void fragments(const floatx16& x, half8 (&f)[2]) {
    uint32_t pk[8];
#pragma unroll
    for (int e = 0; e < 16; e += 2) pk[e >> 1] = pack2(x[e], x[e + 1]);
    __builtin_amdgcn_sched_barrier(0);
    f[0] = fragment_of(pk, 0);
    f[1] = fragment_of(pk, 1);
}
template <int D>
constexpr float SCALE_LOG2 = D == 128 ? 3.5f : 3.f;      // log2(sqrt(D))

struct BwdArgs {
    Batch b;
    const uint16_t* qkv;      // [T x (h + 2 g) D]
    const uint16_t* o;        // [T x h D]
    const uint16_t* dO;       // [T x h D]
    const float* lse;         // [T x h]
    float* delta;             // [T x h], written by the dq kernel
    float* slots;             // [slot][g][dk | dv][sinks][D]
    uint16_t* dqkv;           // [T x (h + 2 g) D]
    int numbers_q, numbers_k, total_q, total_k;      // pieces of 128 queries, of 64 keys; workgroups for them
    int far;                                         // workgroups for the queries beyond the sinks' window
};

// Workgroups of the third kernel for a sequence and key head.
__host__ __device__ __forceinline__ constexpr int sinks_blocks(int sinks, int d) { return (2 * sinks * d + 255) / 256; }
// The sequence has pairs of a sink and a query beyond its window.
__device__ __forceinline__ bool has_far(const Batch& b, int len) { return b.sinks > 0 && len > b.window; }
template <int D>
__device__ __forceinline__ float* slot_at(const BwdArgs& a, int slot, int kv) {
    return a.slots + ((int64_t)slot * a.b.g + kv) * 2 * a.b.sinks * D;
}

// do . o of the lane's row.
template <int D>
__device__ __forceinline__ float row_product(const half8 (&fo)[D / 16], const half8 (&fd)[D / 16]) {
    float sum[D / 16];
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        sum[ks] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[ks] = fmaf((float)fo[ks][e], (float)fd[ks][e], sum[ks]);
    }
#pragma unroll
    for (int n2 = D / 32; n2 > 0; n2 >>= 1)
#pragma unroll
        for (int ks = 0; ks < n2; ++ks) sum[ks] += sum[ks + n2];
    const u32x2 sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum[0]), __float_as_uint(sum[0]), false, false);
    return __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
}

// S and, added to P, dP of a block: rows 0 .. 31 of the pair's tiles against the wave's fragments.
template <int D>
__device__ __forceinline__ void products(const TileRead<D>& r0, const half8 (&fx)[D / 16], const half8 (&fy)[D / 16], floatx16& S, floatx16& P) {
#pragma unroll
    for (int e = 0; e < 16; ++e) S[e] = 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        S = __builtin_amdgcn_mfma_f32_32x32x16_f16(r0.rows(0, ks), fx[ks], S, 0, 0, 0);
        P = __builtin_amdgcn_mfma_f32_32x32x16_f16(r0.rows(TILE<D>, ks), fy[ks], P, 0, 0, 0);
    }
    attn::interleave<4, 2, 2, D / 16 - 2, 4>();
    __builtin_amdgcn_sched_barrier(0);
}

// acc[i] += tile^T[column][row] f[row][lane's row], 32 rows at `off` of the tile.
template <int D>
__device__ __forceinline__ void multiply(const TileRead<D>& r0, int off, const half8 (&f)[2], floatx16 (&acc)[D / 32]) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int i = 0; i < D / 32; ++i) acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(r0.columns(off, i, ks), f[ks], acc[i], 0, 0, 0);
    attn::interleave<4, 1, 2, D / 16 - 2, 2>();
    __builtin_amdgcn_sched_barrier(0);
}
template <int N>
__device__ __forceinline__ void clear(floatx16 (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) x[i][e] = 0.f;
}

// P (times P_SCALE) and dS (times `scale` / DS_SCALE) of a block, for a wave that owns keys: queries qb .. qb + 31 (rows 0 .. 31 of the pair q, do;
// stats: their lse log2(e) - 15 and, BLK further on, -delta) against the lane's key.  CUT: without the pairs whose distance is not one of the
// `reach` from `near` on.
template <int D, bool CUT>
__device__ __forceinline__ void key_gradients(const TileRead<D>& r0, const float* stats, const half8 (&fk)[D / 16], const half8 (&fv)[D / 16],
                                              int distance, uint32_t reach, float scale, half8 (&fp)[2], floatx16& dS) {
    constexpr float C2 = SCALE<D> * LOG2E;
    const int lh = (threadIdx.x & 63) >> 5;
    floatx16 S, P;
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4) {
        const float4 d4 = *reinterpret_cast<const float4*>(stats + BLK + 8 * g4 + 4 * lh);
        P[4 * g4] = d4.x;
        P[4 * g4 + 1] = d4.y;
        P[4 * g4 + 2] = d4.z;
        P[4 * g4 + 3] = d4.w;
    }
    __builtin_amdgcn_sched_barrier(0);
    products<D>(r0, fk, fv, S, P);
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4) {
        const float4 l4 = *reinterpret_cast<const float4*>(stats + 8 * g4 + 4 * lh);
        const float lq[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float p = __builtin_amdgcn_exp2f(fmaf(C2, S[4 * g4 + e], -lq[e])), d = P[4 * g4 + e] * scale;
            if constexpr (CUT) {
                p = not_finite(d) ? NAN : p;
                asm volatile("" : "+v"(p), "+v"(d));      // selects, no branches
                const bool hidden = (uint32_t)(distance + 8 * g4 + e) >= reach;
                p = hidden ? 0.f : p;
                d = hidden ? 0.f : d;
            }
            S[4 * g4 + e] = p;
            dS[4 * g4 + e] = p * d;
        }
    }
    fragments(S, fp);
}

template <int D>
constexpr int DQ_LDS_BYTES = 2 * PAIR<D> * 2;
constexpr int STAT_BYTES = 2 * 2 * BLK * 4;      // lse and delta of the queries of two pairs
template <int D>
constexpr int KEY_LDS_BYTES = DQ_LDS_BYTES<D> + STAT_BYTES + attn::XCH_BYTES + 4 * 64 * 4;      // the last: exponents that go with the exchange

// The moving pairs of the kernel that owns keys: q and do of 64 queries of a head, and their lse and delta.  Rows behind the sequence are zeros; what
// they give is taken out with what the mask hides, since 0 * inf, for a key that is not finite, is not 0.
template <int D>
struct QueryTiles {
    const BwdArgs& a;
    Rows s;
    TileLoad<D> load_q, load_do;
    const uint16_t *q, *dO;      // of the sequence's first row, head 0
    const float* stat0;          // lse (wave 0) or delta (wave 1), likewise
    uint32_t lds0;
    float* stats;
    int wave, lane;
    float stat = 0.f;
    __device__ __forceinline__ QueryTiles(const BwdArgs& a, const Rows& s, uint32_t lds0, float* stats, int wave)
        : a(a), s(s), load_q((int64_t)(a.b.h + 2 * a.b.g) * D, wave), load_do((int64_t)a.b.h * D, wave),
          q(a.qkv + (int64_t)s.start * ((a.b.h + 2 * a.b.g) * D)), dO(a.dO + (int64_t)s.start * (a.b.h * D)), lds0(lds0), stats(stats),
          wave(wave), lane(threadIdx.x & 63) {
        stat0 = (wave == 0 ? a.lse : a.delta) + (int64_t)s.start * a.b.h;
    }
    __device__ __forceinline__ void fetch(int tile, int n, int buf) {
        const int left = s.len - tile * BLK;
        const uint32_t at = lds0 + (uint32_t)buf * (PAIR<D> * 2u);
        load_q.issue(q + n * D, tile, left, at, wave);
        load_do.issue(dO + n * D, tile, left, at + TILE<D> * 2u, wave);
        if (wave < 2) {
            const float* row = stat0 + (int64_t)tile * (BLK * a.b.h) + n;
            stat = row[(uint32_t)(min(lane, left - 1) * a.b.h)];
        }
    }
    // this wave's share of what fetch() brought; a barrier has to follow
    __device__ __forceinline__ void keep_stats(int buf) const {
        if (wave < 2) stats[(2 * buf + wave) * BLK + lane] = wave == 0 ? fmaf(stat, LOG2E, -P_LOG2) : -stat;
    }
};

}  // namespace win

template <int D>
__global__ __launch_bounds__(256, 2) void window_attention_dq_kernel(win::BwdArgs a) {
    using namespace win;
    extern __shared__ __attribute__((aligned(256))) uint16_t smem[];      // two pairs of tiles: K, V
    __shared__ uint32_t bad[2][4];                                        // rows of a K tile that are not finite, by wave
    constexpr float C2 = SCALE<D> * LOG2E;

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, lh = lane >> 5;
    const uint32_t lds0 = (uint32_t)(uintptr_t)smem;
    const int window = a.b.window, sinks = a.b.sinks;

    // order: key heads, pieces, the heads of the group
    const int place = place_of_block(a.total_q, blockIdx.x), r = a.b.h / a.b.g;
    const int kv = place / (a.numbers_q * r), rest = place - kv * a.numbers_q * r;
    const int number = rest / r, n = kv * r + (rest - number * r);
    Rows s;
    const int seq = sequence_of(a.b, number, ROWS, 1, s);
    if (seq < 0) return;
    const int nb = (s.len + ROWS - 1) / ROWS, at = number - first_piece(s.start, seq, ROWS, 1);
    if (at >= nb) return;
    const int q0 = (nb - 1 - at) * ROWS, qw = q0 + 32 * wave;      // the longest walks first
    const bool active = qw < s.len;
    const int query = qw + l32;
    const int64_t t = (int64_t)s.start + min(query, s.len - 1);

    const int64_t ld = (int64_t)(a.b.h + 2 * a.b.g) * D, ldo = (int64_t)a.b.h * D;
    const uint16_t* gk = a.qkv + (int64_t)s.start * ld + (int64_t)(a.b.h + kv) * D;
    const uint16_t* gv = gk + (int64_t)a.b.g * D;

    const int first = max(0, q0 - window + 1) / BLK, last = min(q0 + ROWS - 1, s.len - 1) / BLK;
    const int extra = sinks > 0 && first > 0 ? 1 : 0, tiles = last - first + 1 + extra;
    auto tile_at = [&](int i) { return i < extra ? 0 : first + i - extra; };

    const TileLoad<D> load(ld, wave);
    const TileRead<D> rd(lds0);
    auto fetch = [&](int tile, int buf) {
        const uint32_t at = lds0 + (uint32_t)buf * (PAIR<D> * 2u);
        load.issue(gk, tile, s.len - tile * BLK, at, wave);
        load.issue(gv, tile, s.len - tile * BLK, at + TILE<D> * 2u, wave);
    };
    fetch(tile_at(0), 0);

    half8 fq[D / 16], fd[D / 16];
    float lq = 0.f, delta = 0.f;
    if (active) {
        load_fragments<D>(fq, a.qkv + t * ld + (int64_t)n * D);
        load_fragments<D>(fd, a.dO + t * ldo + (int64_t)n * D);
        half8 fo[D / 16];
        load_fragments<D>(fo, a.o + t * ldo + (int64_t)n * D);
        lq = fmaf(a.lse[t * a.b.h + n], LOG2E, SCALE_LOG2<D> - DS_FIRST);      // so that P comes with the scale of dS
        delta = row_product<D>(fo, fd);
        if (lh == 0 && query < s.len) a.delta[t * a.b.h + n] = delta;
    }
    arrived<D>(fq);
    arrived<D>(fd);
    asm volatile("" : "+v"(lq));
    floatx16 acc[D / 32];
    clear(acc);
    int exponent = DS_FIRST;

    // dS of keys k0 .. k0 + 31 as fragments.  Bits of `rows`: keys that are not finite; a query that sees one has an lse and a delta that are not,
    // unless its score is -inf: then P is 0 and dS times the key is NaN in its infinite columns.
    auto gradients = [&](const TileRead<D>& r0, int k0, auto cut, uint32_t rows, half8 (&f)[2]) {
        floatx16 S, P;
#pragma unroll
        for (int e = 0; e < 16; ++e) P[e] = 0.f;
        products<D>(r0, fq, fd, S, P);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            S[e] = __builtin_amdgcn_exp2f(fmaf(C2, S[e], -lq));
            P[e] -= delta;
            if constexpr (decltype(cut)::value) {
                const int key = k0 + 8 * (e >> 2) + 4 * lh + (e & 3);
                const bool h = key > query | (query - key >= window & key >= sinks);
                float p = S[e], d = P[e];
                asm volatile("" : "+v"(p), "+v"(d));      // selects, no branches
                S[e] = h ? 0.f : p;
                P[e] = h ? 0.f : d;
            }
        }
        if (decltype(cut)::value && rows != 0) {
            const uint32_t own = rows >> (4 * lh);
#pragma unroll
            for (int e = 0; e < 16; ++e) S[e] = own >> (8 * (e >> 2) + (e & 3)) & 1 ? 0.f : S[e];
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) S[e] *= P[e];
        keep_in_range(S, exponent, [&](int n) {
            lq += (float)n;
            multiply_all(acc, power_of_2(-n));
        });
        fragments(S, f);
    };

    int it = 0;
    auto begin = [&]() {
        // the tiles have landed; everybody is done with the other pair
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (it + 1 < tiles) fetch(tile_at(it + 1), (it + 1) & 1);      // in flight while this pair is multiplied
        return rd.at((it & 1) * PAIR<D>);
    };
    // the tiles that every query of the workgroup sees whole
    const int whole0 = (max(0, q0 + ROWS - window) + BLK - 1) / BLK, whole1 = q0 / BLK - 1;
    while (it < tiles) {
        for (; it < tiles && !(it >= extra && tile_at(it) >= whole0 && tile_at(it) <= whole1); ++it) {
            const int k0 = tile_at(it) * BLK;
            const TileRead<D> r0 = begin();
            const uint32_t mine = make_finite<D>(lds0 + (uint32_t)(it & 1) * (PAIR<D> * 2u), wave);
            if (lane == 0) bad[it & 1][wave] = mine;
            attn::meet();
            if (!active) continue;
#pragma nounroll
            for (int h = 0; h < 2; ++h) {
                if (!seen(qw, k0 + 32 * h, window, sinks)) continue;
                const TileRead<D> r1 = r0.at(32 * h * D);
                uint32_t rows = __builtin_amdgcn_readfirstlane(bad[it & 1][2 * h] | bad[it & 1][2 * h + 1] << 16);
                half8 f[2];
                gradients(r1, k0 + 32 * h, std::true_type{}, rows, f);
                multiply<D>(r1, 0, f, acc);
                while (rows != 0) {      // what is not finite of a key, to the queries that see it
                    const int key = k0 + 32 * h + __builtin_ctz(rows);
                    rows &= rows - 1;
                    if (key > query || (query - key >= window && key >= sinks)) continue;
                    const uint16_t* k = gk + (int64_t)key * ld + 4 * lh;
#pragma unroll
                    for (int i = 0; i < D / 32; ++i)
#pragma unroll
                        for (int g4 = 0; g4 < 4; ++g4) {
                            const half4 x = *reinterpret_cast<const half4*>(k + 32 * i + 8 * g4);
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[i][4 * g4 + e] += not_finite((float)x[e]) ? NAN : 0.f;
                        }
                }
            }
        }
        for (; it < tiles && tile_at(it) <= whole1; ++it) {
            const TileRead<D> r0 = begin();
            if (!active) continue;
#pragma nounroll
            for (int h = 0; h < 2; ++h) {
                const TileRead<D> r1 = r0.at(32 * h * D);
                half8 f[2];
                gradients(r1, 0, std::false_type{}, 0u, f);
                multiply<D>(r1, 0, f, acc);
            }
        }
    }
    multiply_all(acc, power_of_2(-exponent));
    if (active) store_rows(acc, query < s.len ? a.dqkv + t * ld + (int64_t)n * D : nullptr);
}

// A workgroup has 64 keys and the queries whose distance to a key is within some bounds: of the first a.far workgroups the sinks and FAR_ROWS
// queries beyond the window, of the others a block of keys and the queries whose window reaches it.  Two teams of four waves, with tiles of
// their own, take one half each of the walk through the tiles of all heads of the group, and the first adds up: a walk is long where heads share
// their keys, and the longest one bounds a call.  In a team two waves have the same 32 keys; each forms P and dS of one half of the tile's
// queries, hands one of the two to the other through LDS, and sums dv (the first) or dk over all of them.
template <int D>
__global__ __launch_bounds__(512, 2) void window_attention_dkdv_kernel(win::BwdArgs a) {
    using namespace win;
    extern __shared__ __attribute__((aligned(256))) uint16_t smem[];      // of each team: lse and delta of two pairs of tiles; the pairs: Q, dO; what waves exchange

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) & 3, team = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
    const int part = wave >> 1, l32 = lane & 31, lh = lane >> 5;
    uint16_t* own_lds = smem + team * (KEY_LDS_BYTES<D> / 2);
    float* stats = reinterpret_cast<float*>(own_lds);      // [pair][lse log2(e) - 15 | delta DS_SCALE][64]
    uint16_t* tiles_at = own_lds + STAT_BYTES / 2;
    const uint32_t lds0 = (uint32_t)(uintptr_t)tiles_at;
    const attn::Exchange xch(tiles_at + 2 * PAIR<D>, wave);
    int* exponents = reinterpret_cast<int*>(tiles_at + 2 * PAIR<D> + attn::XCH_BYTES / 2) + lane;

    const int r = a.b.h / a.b.g;
    int seq, kv, k0, near, first, last;      // keys from k0 on; query tiles; the distance of the nearest query
    uint32_t reach;
    float* slot = nullptr;
    Rows s;
    if ((int)blockIdx.x < a.far) {
        const int number = blockIdx.x / a.b.g;
        kv = blockIdx.x - number * a.b.g;
        seq = sequence_of(a.b, number, FAR_ROWS, 2, s);
        if (seq < 0) return;
        const int piece = number - first_piece(s.start, seq, FAR_ROWS, 2) - 1;      // the first number is for the sums of the block of keys
        if (piece < 0 || !has_far(a.b, s.len)) return;
        const int from = max((int64_t)piece * FAR_ROWS, (int64_t)a.b.window), to = min((int64_t)s.len, (int64_t)(piece + 1) * FAR_ROWS);
        if (from >= to) return;
        k0 = 0;
        near = a.b.window;
        reach = 0x7fffffffu;
        first = from / BLK;
        last = (to - 1) / BLK;
        slot = slot_at<D>(a, number, kv);
    } else {
        // order: key heads, blocks
        const int place = place_of_block(a.total_k, (int)blockIdx.x - a.far);
        kv = place / a.numbers_k;
        const int number = place - kv * a.numbers_k;
        seq = sequence_of(a.b, number, BLK, 1, s);
        if (seq < 0) return;
        k0 = (number - first_piece(s.start, seq, BLK, 1)) * BLK;      // the longest walks first
        if (k0 >= s.len) return;
        near = 0;
        reach = (uint32_t)a.b.window;
        first = k0 / BLK;
        last = (int)min((int64_t)s.len - 1, (int64_t)k0 + BLK - 2 + a.b.window) / BLK;
        if (k0 == 0 && has_far(a.b, s.len)) slot = slot_at<D>(a, first_piece(s.start, seq, FAR_ROWS, 2), kv);
    }
    const int kw = k0 + 32 * (wave & 1), key = kw + l32;
    const bool active = kw < s.len && (near == 0 || kw < a.b.sinks);
    const int64_t ld = (int64_t)(a.b.h + 2 * a.b.g) * D;
    const int64_t t = (int64_t)s.start + min(key, s.len - 1);
    const uint32_t reach_key = min(reach, (uint32_t)max(s.len - key - near, 0));      // no further than the last query

    // the walk: (head, tile); this team's steps are `steps` from its `tile` and head `n` on, the other's tile is `other`
    const int per = last - first + 1, total = per * r, more = (total + 1) / 2, fewer = total - more;      // of the first team, of the second
    const int steps = team == 0 ? more : fewer;
    int tile = first + (team == 0 ? 0 : more % per), other = first + (team == 0 ? more % per : 0), n = kv * r + (team == 0 ? 0 : more / per);
    QueryTiles<D> tiles(a, s, lds0, stats, wave);
    if (steps > 0) tiles.fetch(tile, n, 0);

    half8 fk[D / 16], fv[D / 16];
    if (active) {
        load_fragments<D>(fk, a.qkv + t * ld + (int64_t)(a.b.h + kv) * D);
        load_fragments<D>(fv, a.qkv + t * ld + (int64_t)(a.b.h + a.b.g + kv) * D);
    }
    arrived<D>(fk);
    arrived<D>(fv);
    floatx16 acc[D / 32];      // dv or dk
    clear(acc);
    int exponent = DS_FIRST;      // of this wave's dS, and of the sums for dk
    float scale = power_of_2(DS_FIRST) * DS_SCALE<D>;
    const TileRead<D> rd(lds0);

    int it = 0;
    auto begin = [&]() {
        const int buf = it & 1;
        if (it < steps) tiles.keep_stats(buf);
        // the tiles have landed; everybody is done with the other pair
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        ++it;
        if (++tile > last) {
            tile = first;
            ++n;
        }
        if (++other > last) other = first;
        if (it < steps) tiles.fetch(tile, n, buf ^ 1);      // in flight while this pair is multiplied
        return buf;
    };
    auto lower = [&](int n) {
        const float f = power_of_2(-n);
        scale *= f;
        if (part == 1) multiply_all(acc, f);
    };
    auto own_gradients = [&](int buf, int distance, auto cut, half8 (&f)[2]) {
        half8 fp[2], fd[2];
        floatx16 dS;
        key_gradients<D, decltype(cut)::value>(rd.at(buf * PAIR<D> + 32 * part * D), stats + 2 * buf * BLK + 32 * part, fk, fv, distance, reach_key, scale, fp, dS);
        keep_in_range(dS, exponent, lower);
        fragments(dS, fd);
        exponents[64 * wave] = exponent;
        if (part == 0) xch.put(fd);
        else xch.put(fp);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) f[ks] = part == 0 ? fp[ks] : fd[ks];
    };
    // the partner's half; both go on with the lower exponent of the two
    auto others_gradients = [&](half8 (&f)[2]) {
        xch.get(f);
        const int other_exponent = exponents[64 * (wave ^ 2)];
        if (__any(other_exponent != exponent)) {
            if (part == 1) {
                const float down = power_of_2(-max(other_exponent - exponent, 0));
#pragma unroll
                for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[ks][e] = (_Float16)((float)f[ks][e] * down);
            }
            const int n = max(exponent - other_exponent, 0);
            exponent -= n;
            lower(n);
        }
    };
    // where half h of do (for dv) or q (for dk) is
    auto sums_of = [&](int buf, int h) { return rd.at(buf * PAIR<D> + (part == 0 ? TILE<D> : 0) + 32 * h * D); };
    // the query tiles that are within the bounds for every key of the workgroup, and within the sequence
    const int whole0 = (k0 + BLK - 1 + near + BLK - 1) / BLK, whole1 = min(near > 0 ? last : (k0 + a.b.window - BLK) / BLK, s.len / BLK - 1);
    auto whole = [&](int x) { return x >= whole0 && x <= whole1; };
    while (it < more) {
        while (it < more && !(it < fewer && whole(tile) && whole(other))) {
            const int qb = tile * BLK;
            const bool has = active && it < steps;
            const int buf = begin();
            make_finite<D>(lds0 + (uint32_t)buf * (PAIR<D> * 2u), wave);
            make_finite<D>(lds0 + (uint32_t)buf * (PAIR<D> * 2u) + TILE<D> * 2u, wave);
            attn::meet();
            // distances in each half: between qb + 32 h - (kw + 31) and qb + 32 h + 31 - kw
            auto some = [&](int h) { return has && qb + 32 * h + 31 - kw >= near && (near > 0 || qb + 32 * h - (kw + 31) < (int)reach); };
            half8 f[2];
            if (some(part)) {
                own_gradients(buf, qb + 32 * part + 4 * lh - key - near, std::true_type{}, f);
                multiply<D>(sums_of(buf, part), 0, f, acc);
            }
            attn::meet();
            if (some(1 - part)) {
                others_gradients(f);
                multiply<D>(sums_of(buf, 1 - part), 0, f, acc);
            }
        }
        while (it < fewer && whole(tile) && whole(other)) {
            const int buf = begin();
            half8 f[2];
            if (active) {
                own_gradients(buf, 0, std::false_type{}, f);
                multiply<D>(sums_of(buf, part), 0, f, acc);
            }
            attn::meet();
            if (!active) continue;
            others_gradients(f);
            multiply<D>(sums_of(buf, 1 - part), 0, f, acc);
        }
    }
    multiply_all(acc, part == 0 ? 1.f / P_SCALE : power_of_2(-exponent));
    // the second team's sums to the first
    float* sums = reinterpret_cast<float*>(smem) + wave * (D / 2 * 64) + lane;      // as much as two pairs of tiles
    __syncthreads();
    if (team == 1) {
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) sums[(16 * i + e) * 64] = acc[i][e];
    }
    __syncthreads();
    if (team == 1 || !active) return;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][e] += sums[(16 * i + e) * 64];
    const bool own = key < s.len, sink = own && key < a.b.sinks && slot != nullptr;
    if (near == 0) store_rows(acc, own && !sink ? a.dqkv + t * ld + (int64_t)(a.b.h + (1 - part) * a.b.g + kv) * D : nullptr);
    if (sink) {
        float* out = slot + (int64_t)((1 - part) * a.b.sinks + key) * D + 4 * lh;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int g4 = 0; g4 < 4; ++g4)
                *reinterpret_cast<float4*>(out + 32 * i + 8 * g4) = {acc[i][4 * g4], acc[i][4 * g4 + 1], acc[i][4 * g4 + 2], acc[i][4 * g4 + 3]};
    }
}

// The sinks' dk and dv: the sums over their window and over the pieces beyond it, in order.  One thread per element.
template <int D>
__global__ __launch_bounds__(256) void window_attention_sinks_kernel(win::BwdArgs a) {
    using namespace win;
    const int per = sinks_blocks(a.b.sinks, D), pair = blockIdx.x / per;
    const int seq = pair / a.b.g, kv = pair - seq * a.b.g;
    const Rows s = rows_of(a.b, seq);
    const int i = (blockIdx.x - pair * per) * 256 + threadIdx.x;
    const int which = i / (a.b.sinks * D), row = (i - which * a.b.sinks * D) / D, c = i % D;
    if (!has_far(a.b, s.len) || which > 1 || row >= s.len) return;
    const int base = first_piece(s.start, seq, FAR_ROWS, 2);
    const int from = a.b.window / FAR_ROWS, to = (s.len - 1) / FAR_ROWS;
    const int64_t step = (int64_t)a.b.g * 2 * a.b.sinks * D;
    const float* p = slot_at<D>(a, base, kv) + ((int64_t)which * a.b.sinks + row) * D + c;
    float sum = *p;
    for (int k = from; k <= to; k += 8) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = k + e <= to ? p[(k + e + 1) * step] : 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += x[e];
    }
    const _Float16 x = (_Float16)sum;
    a.dqkv[((int64_t)s.start + row) * (a.b.h + 2 * a.b.g) * D + (int64_t)(a.b.h + which * a.b.g + kv) * D + c] = __builtin_bit_cast(uint16_t, x);
}

// Threads of the largest launch.
int64_t window_attention_threads(int64_t T, int64_t B, int64_t h, int64_t g, int64_t d, int64_t sinks) {
    using namespace win;
    const int64_t rows = pieces(T, B, ROWS, 1) * h, keys = (pieces(T, B, BLK, 1) + pieces(T, B, FAR_ROWS, 2)) * g;
    return std::max(std::max(256 * rows, 512 * keys), 256 * B * g * sinks_blocks((int)sinks, (int)d));
}
size_t window_attention_delta_bytes(int64_t T, int64_t h) { return ((size_t)T * h * 4 + 255) & ~(size_t)255; }
size_t window_attention_ws_bytes(int64_t T, int64_t B, int64_t h, int64_t g, int64_t d, int64_t sinks) {
    return window_attention_delta_bytes(T, h) + (size_t)(win::pieces(T, B, win::FAR_ROWS, 2) * g * 2 * sinks * d) * 4;
}

template <int D>
static hipError_t launch_backward_of(const win::BwdArgs& a, hipStream_t st) {
    using namespace win;
    auto dq = window_attention_dq_kernel<D>;
    auto dkdv = window_attention_dkdv_kernel<D>;
    static const hipError_t cfg0 = allow_dynamic_lds(dq, DQ_LDS_BYTES<D>);
    if (cfg0 != hipSuccess) return cfg0;
    static const hipError_t cfg1 = allow_dynamic_lds(dkdv, 2 * KEY_LDS_BYTES<D>);
    if (cfg1 != hipSuccess) return cfg1;
    hipLaunchKernelGGL(dq, dim3((unsigned)a.total_q), dim3(256), DQ_LDS_BYTES<D>, st, a);
    hipLaunchKernelGGL(dkdv, dim3((unsigned)(a.far + a.total_k)), dim3(512), 2 * KEY_LDS_BYTES<D>, st, a);
    if (a.far > 0)
        hipLaunchKernelGGL(window_attention_sinks_kernel<D>, dim3((unsigned)(a.b.B * a.b.g * sinks_blocks(a.b.sinks, D))), dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_window_attention_backward(const uint16_t* qkv, const uint16_t* o, const uint16_t* dO, const float* lse, uint16_t* dqkv,
                                            const int32_t* off, int64_t T, int64_t B, int64_t h, int64_t g, int64_t d, int64_t window,
                                            int64_t sinks, void* ws, hipStream_t st) {
    win::BwdArgs a;
    a.b = {off, (int)T, (int)B, (int)h, (int)g, (int)window, (int)sinks};
    a.qkv = qkv; a.o = o; a.dO = dO; a.lse = lse; a.dqkv = dqkv;
    a.delta = static_cast<float*>(ws);
    a.slots = reinterpret_cast<float*>(static_cast<char*>(ws) + window_attention_delta_bytes(T, h));
    a.numbers_q = (int)win::pieces(T, B, win::ROWS, 1);
    a.numbers_k = (int)win::pieces(T, B, win::BLK, 1);
    a.total_q = (int)(a.numbers_q * h);
    a.total_k = (int)(a.numbers_k * g);
    a.far = sinks > 0 && T > window ? (int)(win::pieces(T, B, win::FAR_ROWS, 2) * g) : 0;      // no sequence is longer than T
    return d == 128 ? launch_backward_of<128>(a, st) : launch_backward_of<64>(a, st);
}

}  // namespace lomo
