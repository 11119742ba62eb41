// Backward of softmax attention with a sliding window and sinks over packed sequences (the forward: lomo_window_fwd.hip), for the
// hand-on gradient of Algorithm 1.  Query i sees the keys j <= i with i - j < window or j < sinks:
//
//   P_ij = exp(q_i . k_j / sqrt(d) - lse_i),   dP_ij = do_i . v_j,   delta_i = do_i . o_i,   dS = P (dP - delta) / sqrt(d)
//   dq_i = sum_j dS_ij k_j;   dk_j = sum over the queries i of all heads of the group dS_ij q_i;   dv_j likewise of P_ij do_i
//
// Four deterministic kernels, no atomics.  The first: a workgroup per (128 queries, head) forms delta, walks the tiles of keys
// that the window reaches, and the sinks', and accumulates dq.  The second: a workgroup per (128 keys, key head) walks the query tiles
// whose window reaches the keys, for each head of the group, and accumulates dk and dv.  The sinks have queries beyond their window, up to
// the whole sequence: the third kernel sums over those, FAR_ROWS queries of all heads of a group to a workgroup, each result a
// slot of `sinks` fp32 rows in the workspace, where the second puts its own sums of these rows; the fourth adds the slots in order
// and rounds.  All recompute S, P, dP, dS in blocks of 32 x 32 per wave with the wave's own rows along the lanes.
//
// fp32 accumulation on the matrix cores.  P and dS pass through fp16 before the products that consume them; P is held times 2^15 there,
// so that the probabilities of a long window (2^-14 and less) keep all their bits.  dq, dk, dv are rounded once.  Blocks that a mask
// cuts look for inf and NaN and take them out of the products, so that a pair which the mask hides adds nothing.
#include "lomo_window_common.h"

#include <type_traits>

namespace lomo {

namespace win {

constexpr int FAR_ROWS = 512;
constexpr float P_SCALE = 32768.f, P_LOG2 = 15.f;

struct BwdArgs {
    Batch b;
    const uint16_t* qkv;      // [T x (h + 2 g) D]
    const uint16_t* o;        // [T x h D]
    const uint16_t* dO;       // [T x h D]
    const float* lse;         // [T x h]
    float* delta;             // [T x h], written by the dq kernel
    float* slots;             // [slot][g][dk | dv][sinks][D]
    uint16_t* dqkv;           // [T x (h + 2 g) D]
    int numbers, total_q, total_k;      // of 128-row pieces; of workgroups
    int slot_numbers;
};

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

// S and dP of a block: rows 0 .. 31 of the pair's tiles against the wave's fragments.
template <int D>
__device__ __forceinline__ void products(const TileRead<D>& r0, const half8 (&fx)[D / 16], const half8 (&fy)[D / 16], floatx16& S, floatx16& P) {
#pragma unroll
    for (int e = 0; e < 16; ++e) S[e] = P[e] = 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        S = __builtin_amdgcn_mfma_f32_32x32x16_f16(r0.rows(0, ks), fx[ks], S, 0, 0, 0);
        P = __builtin_amdgcn_mfma_f32_32x32x16_f16(r0.rows(TILE<D>, ks), fy[ks], P, 0, 0, 0);
    }
    attn::interleave<4, 2, 2, D / 16 - 2, 4>();
    __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ bool any_not_finite(const floatx16& S, const floatx16& P) {
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 16; ++e) bad |= not_finite(S[e]) | not_finite(P[e]);
    return __any(bad);
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
// The same; dirty: without what is not finite in the tile.
template <int D>
__device__ __forceinline__ void multiply_finite(const TileRead<D>& r0, int off, const half8 (&f)[2], floatx16 (&acc)[D / 32], bool dirty) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
        half8 x[D / 32];
#pragma unroll
        for (int i = 0; i < D / 32; ++i) x[i] = r0.columns(off, i, ks);
        if (dirty) {
#pragma unroll
            for (int i = 0; i < D / 32; ++i) x[i] = finite_or_zero(x[i]);
        }
#pragma unroll
        for (int i = 0; i < D / 32; ++i) acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i], f[ks], acc[i], 0, 0, 0);
    }
}

template <int N>
__device__ __forceinline__ void clear(floatx16 (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) x[i][e] = 0.f;
}

// One block for a wave that owns keys: queries qb .. qb + 31 (rows 0 .. 31 of the pair q, do; stats: their lse log2(e) - 15 and, BLK
// further on, delta) against the lane's key.  CUT: without the pairs that `hidden(query)`.
template <int D, bool CUT, typename Hidden>
__device__ __forceinline__ void key_block(const TileRead<D>& r0, const float* stats, const half8 (&fk)[D / 16], const half8 (&fv)[D / 16], int qb,
                                          Hidden hidden, floatx16 (&dk)[D / 32], floatx16 (&dv)[D / 32]) {
    constexpr float C2 = SCALE<D> * LOG2E;
    const int lh = (threadIdx.x & 63) >> 5;
    floatx16 S, P;
    products<D>(r0, fk, fv, S, P);
    const bool dirty = CUT && any_not_finite(S, P);
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4) {
        const float4 l4 = *reinterpret_cast<const float4*>(stats + 8 * g4 + 4 * lh), d4 = *reinterpret_cast<const float4*>(stats + BLK + 8 * g4 + 4 * lh);
        const float lq[4] = {l4.x, l4.y, l4.z, l4.w}, dq[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            S[4 * g4 + e] = __builtin_amdgcn_exp2f(fmaf(C2, S[4 * g4 + e], -lq[e]));
            P[4 * g4 + e] -= dq[e];
            if constexpr (CUT) {
                const bool h = hidden(qb + 8 * g4 + 4 * lh + e);
                float p = S[4 * g4 + e], d = P[4 * g4 + e];
                p = not_finite(d) ? NAN : p;
                asm volatile("" : "+v"(p), "+v"(d));      // selects, no branches
                S[4 * g4 + e] = h ? 0.f : p;
                P[4 * g4 + e] = h ? 0.f : d;
            }
        }
        if (g4 & 1) __builtin_amdgcn_sched_barrier(0);
    }
    uint32_t pp[8], pd[8];
#pragma unroll
    for (int e = 0; e < 16; e += 2) {
        pp[e >> 1] = pack2(S[e], S[e + 1]);
        pd[e >> 1] = pack2(SCALE<D> / P_SCALE * S[e] * P[e], SCALE<D> / P_SCALE * S[e + 1] * P[e + 1]);
    }
    __builtin_amdgcn_sched_barrier(0);
    const half8 fp[2] = {fragment_of(pp, 0), fragment_of(pp, 1)}, fd[2] = {fragment_of(pd, 0), fragment_of(pd, 1)};
    if constexpr (CUT) {
        multiply_finite<D>(r0, TILE<D>, fp, dv, dirty);
        multiply_finite<D>(r0, 0, fd, dk, dirty);
    } else {
        multiply<D>(r0, TILE<D>, fp, dv);
        multiply<D>(r0, 0, fd, dk);
    }
}

template <int D>
constexpr int DQ_LDS_BYTES = 2 * PAIR<D> * 2;
constexpr int STAT_BYTES = 2 * 2 * BLK * 4;      // lse and delta of the queries of two pairs
template <int D>
constexpr int KEY_LDS_BYTES = DQ_LDS_BYTES<D> + STAT_BYTES;

// The moving pairs of the kernels that own keys: q and do of 64 queries of a head, and their lse and delta.  Rows behind the sequence are zeros with
// an lse of infinity: their probabilities are 0.
template <int D, int WAVES>
struct QueryTiles {
    const BwdArgs& a;
    Rows s;
    int64_t ld, ldo;
    TileLoad<D> load_q, load_do;
    uint32_t lds0;
    float* stats;
    int wave, lane;
    float stat = 0.f;
    __device__ __forceinline__ QueryTiles(const BwdArgs& a, const Rows& s, uint32_t lds0, float* stats)
        : a(a), s(s), ld((int64_t)(a.b.h + 2 * a.b.g) * D), ldo((int64_t)a.b.h * D), load_q(ld), load_do(ldo), lds0(lds0), stats(stats),
          wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), lane(threadIdx.x & 63) {}
    __device__ __forceinline__ void fetch(int tile, int n, int buf) {
        const int64_t t = (int64_t)s.start + tile * BLK;
        const int rows = s.len - tile * BLK;
        load_q.template issue<WAVES>(a.qkv + t * ld + (int64_t)n * D, rows, lds0 + (uint32_t)buf * (PAIR<D> * 2u), wave);
        load_do.template issue<WAVES>(a.dO + t * ldo + (int64_t)n * D, rows, lds0 + (uint32_t)buf * (PAIR<D> * 2u) + TILE<D> * 2u, wave);
        if (wave < 2) stat = lane < rows ? (wave == 0 ? a.lse : a.delta)[(t + lane) * a.b.h + n] : (wave == 0 ? INFINITY : 0.f);
    }
    // this wave's share of what fetch() brought; a barrier has to follow
    __device__ __forceinline__ void keep_stats(int buf) const {
        if (wave < 2) stats[(2 * buf + wave) * BLK + lane] = wave == 0 ? fmaf(stat, LOG2E, -P_LOG2) : stat;
    }
};

}  // namespace win

template <int D>
__global__ __launch_bounds__(256, 2) void window_attention_dq_kernel(win::BwdArgs a) {
    using namespace win;
    extern __shared__ __attribute__((aligned(256))) uint16_t smem[];      // two pairs of tiles: K, V
    constexpr float C2 = SCALE<D> * LOG2E;

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, lh = lane >> 5;
    const uint32_t lds0 = (uint32_t)(uintptr_t)smem;
    const int window = a.b.window, sinks = a.b.sinks;

    // order: key heads, pieces, the heads of the group
    const int place = place_of_block(a.total_q), r = a.b.h / a.b.g;
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
    const int64_t t = (int64_t)s.start + min(query, s.len - 1);

    const int64_t ld = (int64_t)(a.b.h + 2 * a.b.g) * D, ldo = (int64_t)a.b.h * D;
    const uint16_t* gk = a.qkv + (int64_t)s.start * ld + (int64_t)(a.b.h + kv) * D;
    const uint16_t* gv = gk + (int64_t)a.b.g * D;

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

    half8 fq[D / 16], fd[D / 16];
    float lq = 0.f, delta = 0.f;
    if (active) {
        load_fragments<D>(fq, a.qkv + t * ld + (int64_t)n * D);
        load_fragments<D>(fd, a.dO + t * ldo + (int64_t)n * D);
        half8 fo[D / 16];
        load_fragments<D>(fo, a.o + t * ldo + (int64_t)n * D);
        lq = a.lse[t * a.b.h + n] * LOG2E;
        delta = row_product<D>(fo, fd);
        if (lh == 0 && query < s.len) a.delta[t * a.b.h + n] = delta;
    }
    floatx16 acc[D / 32];
    clear(acc);

    // dS of keys k0 .. k0 + 31 as fragments
    auto gradients = [&](const TileRead<D>& r0, int k0, auto cut, half8 (&f)[2], bool& dirty) {
        floatx16 S, P;
        products<D>(r0, fq, fd, S, P);
        dirty = decltype(cut)::value && any_not_finite(S, P);
        uint32_t pk[8];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            S[e] = SCALE<D> * __builtin_amdgcn_exp2f(fmaf(C2, S[e], -lq));
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
#pragma unroll
        for (int e = 0; e < 16; e += 2) pk[e >> 1] = pack2(S[e] * P[e], S[e + 1] * P[e + 1]);
        __builtin_amdgcn_sched_barrier(0);
        f[0] = fragment_of(pk, 0);
        f[1] = fragment_of(pk, 1);
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
            if (!active) continue;
#pragma nounroll
            for (int h = 0; h < 2; ++h) {
                if (seen(qw, k0 + 32 * h, window, sinks) == NONE) continue;
                const TileRead<D> r1 = r0.at(32 * h * D);
                half8 f[2];
                bool dirty;
                gradients(r1, k0 + 32 * h, std::true_type{}, f, dirty);
                multiply_finite<D>(r1, 0, f, acc, dirty);
            }
        }
        for (; it < tiles && tile_at(it) <= whole1; ++it) {
            const TileRead<D> r0 = begin();
            if (!active) continue;
#pragma nounroll
            for (int h = 0; h < 2; ++h) {
                const TileRead<D> r1 = r0.at(32 * h * D);
                half8 f[2];
                bool dirty;
                gradients(r1, 0, std::false_type{}, f, dirty);
                multiply<D>(r1, 0, f, acc);
            }
        }
    }
    if (active) store_rows(acc, query < s.len ? a.dqkv + t * ld + (int64_t)n * D : nullptr);
}

template <int D>
__global__ __launch_bounds__(256, 2) void window_attention_dkdv_kernel(win::BwdArgs a) {
    using namespace win;
    extern __shared__ __attribute__((aligned(256))) uint16_t smem[];      // lse and delta of two pairs of tiles; the pairs: Q, dO

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31;
    float* stats = reinterpret_cast<float*>(smem);      // [pair][lse log2(e) - 15 | delta][64]
    const uint32_t lds0 = (uint32_t)(uintptr_t)(smem + STAT_BYTES / 2);
    const int window = a.b.window;

    // order: key heads, pieces
    const int place = place_of_block(a.total_k), r = a.b.h / a.b.g;
    const int kv = place / a.numbers, number = place - kv * a.numbers;
    const int seq = sequence_of(a.b, number, ROWS, 1);
    if (seq < 0) return;
    const Rows s = rows_of(a.b, seq);
    const int nb = (s.len + ROWS - 1) / ROWS, at = number - first_piece(a.b, seq, ROWS, 1);
    if (at >= nb) return;
    const int k0 = at * ROWS, kw = k0 + 32 * wave;      // the longest walks first
    const bool active = kw < s.len;
    const int key = kw + l32;
    const int64_t ld = (int64_t)(a.b.h + 2 * a.b.g) * D;
    const int64_t t = (int64_t)s.start + min(key, s.len - 1);

    // query tiles of one head, all heads of the group in turn
    const int first = k0 / BLK, last = (int)min((int64_t)s.len - 1, (int64_t)k0 + ROWS - 2 + window) / BLK;
    const int per = last - first + 1, steps = per * r;
    QueryTiles<D, 4> tiles(a, s, lds0, stats);
    tiles.fetch(first, kv * r, 0);

    half8 fk[D / 16], fv[D / 16];
    if (active) {
        load_fragments<D>(fk, a.qkv + t * ld + (int64_t)(a.b.h + kv) * D);
        load_fragments<D>(fv, a.qkv + t * ld + (int64_t)(a.b.h + a.b.g + kv) * D);
    }
    floatx16 dk[D / 32], dv[D / 32];
    clear(dk);
    clear(dv);
    const TileRead<D> rd(lds0);
    auto hidden = [&](int query) { return query < key | query - key >= window; };

    int it = 0, tile = first, n = kv * r;      // the pair that is next
    auto begin = [&](int& buf) {
        buf = it & 1;
        tiles.keep_stats(buf);
        // the tiles have landed; everybody is done with the other pair
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        ++it;
        if (++tile > last) {
            tile = first;
            ++n;
        }
        if (it < steps) tiles.fetch(tile, n, buf ^ 1);      // in flight while this pair is multiplied
    };
    // the query tiles that see every key of the workgroup
    const int whole0 = k0 / BLK + 2, whole1 = (k0 + window - BLK) / BLK;
    auto whole = [&]() { return tile >= whole0 && tile <= whole1; };
    while (it < steps) {
        while (it < steps && !whole()) {
            const int qb = tile * BLK;
            int buf;
            begin(buf);
            if (!active) continue;
#pragma nounroll
            for (int h = 0; h < 2; ++h)
                if (seen(qb + 32 * h, kw, window, 0) != NONE)
                    key_block<D, true>(rd.at(buf * PAIR<D> + 32 * h * D), stats + 2 * buf * BLK + 32 * h, fk, fv, qb + 32 * h, hidden, dk, dv);
        }
        while (it < steps && whole()) {
            int buf;
            begin(buf);
            if (!active) continue;
#pragma nounroll
            for (int h = 0; h < 2; ++h)
                key_block<D, false>(rd.at(buf * PAIR<D> + 32 * h * D), stats + 2 * buf * BLK + 32 * h, fk, fv, 0, hidden, dk, dv);
        }
    }
    if (!active) return;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) dv[i][e] *= 1.f / P_SCALE;
    const bool own = key < s.len, sink = own && key < a.b.sinks && has_far(a.b, s.len);
    uint16_t* out = own && !sink ? a.dqkv + t * ld + (int64_t)(a.b.h + kv) * D : nullptr;
    store_rows(dk, out);
    store_rows(dv, out == nullptr ? nullptr : out + (int64_t)a.b.g * D);
    if (sink) {
        float* slot = slot_at<D>(a, first_piece(a.b, seq, FAR_ROWS, 2), kv) + (int64_t)key * D + 4 * ((threadIdx.x & 63) >> 5);
        float* second = slot + (int64_t)a.b.sinks * D;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int g4 = 0; g4 < 4; ++g4) {
                *reinterpret_cast<float4*>(slot + 32 * i + 8 * g4) = {dk[i][4 * g4], dk[i][4 * g4 + 1], dk[i][4 * g4 + 2], dk[i][4 * g4 + 3]};
                *reinterpret_cast<float4*>(second + 32 * i + 8 * g4) = {dv[i][4 * g4], dv[i][4 * g4 + 1], dv[i][4 * g4 + 2], dv[i][4 * g4 + 3]};
            }
    }
}

// The sinks and FAR_ROWS queries, those beyond the window; a wave has 32 of each tile's 64, a workgroup 32 sinks.
template <int D>
__global__ __launch_bounds__(128, 1) void window_attention_far_kernel(win::BwdArgs a) {
    using namespace win;
    extern __shared__ __attribute__((aligned(256))) uint16_t smem[];      // as above

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, lh = lane >> 5;
    float* stats = reinterpret_cast<float*>(smem);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(smem + STAT_BYTES / 2);
    const int window = a.b.window, r = a.b.h / a.b.g;

    const int parts = (a.b.sinks + 31) / 32;
    const int number = blockIdx.x / (a.b.g * parts), rest = blockIdx.x - number * a.b.g * parts;
    const int kv = rest / parts, kw = 32 * (rest - kv * parts);      // these sinks
    const int seq = sequence_of(a.b, number, FAR_ROWS, 2);
    if (seq < 0) return;
    const Rows s = rows_of(a.b, seq);
    const int piece = number - first_piece(a.b, seq, FAR_ROWS, 2) - 1;      // the first number is the second kernel's slot
    if (piece < 0 || !has_far(a.b, s.len)) return;
    const int from = max((int64_t)piece * FAR_ROWS, (int64_t)window), to = min((int64_t)s.len, (int64_t)(piece + 1) * FAR_ROWS);
    if (from >= to || kw >= s.len) return;
    const int64_t ld = (int64_t)(a.b.h + 2 * a.b.g) * D;
    const int key = kw + l32;
    const int64_t t = (int64_t)s.start + min(key, s.len - 1);

    const int first = from / BLK, last = (to - 1) / BLK;
    const int per = last - first + 1, steps = per * r;
    QueryTiles<D, 2> tiles(a, s, lds0, stats);
    tiles.fetch(first, kv * r, 0);

    half8 fk[D / 16], fv[D / 16];
    load_fragments<D>(fk, a.qkv + t * ld + (int64_t)(a.b.h + kv) * D);
    load_fragments<D>(fv, a.qkv + t * ld + (int64_t)(a.b.h + a.b.g + kv) * D);
    floatx16 dk[D / 32], dv[D / 32];
    clear(dk);
    clear(dv);
    const TileRead<D> rd = TileRead<D>(lds0).at(32 * wave * D);
    auto hidden = [&](int query) { return query - key < window; };

    int tile = first, n = kv * r;
    for (int it = 0; it < steps; ++it) {
        const int buf = it & 1, qb = tile * BLK + 32 * wave;
        tiles.keep_stats(buf);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (++tile > last) {
            tile = first;
            ++n;
        }
        if (it + 1 < steps) tiles.fetch(tile, n, buf ^ 1);
        if (qb + 31 - kw < window) continue;      // none of them
        key_block<D, true>(rd.at(buf * PAIR<D>), stats + 2 * buf * BLK + 32 * wave, fk, fv, qb, hidden, dk, dv);
    }
    // the two waves' sums
    float* xch = reinterpret_cast<float*>(smem) + lane;      // [dk | dv][D / 2][64 lanes]: as much as a pair of tiles
    __syncthreads();
    if (wave == 1) {
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                xch[(16 * i + e) * 64] = dk[i][e];
                xch[(D / 2 + 16 * i + e) * 64] = dv[i][e];
            }
    }
    __syncthreads();
    if (wave == 1 || key >= min(a.b.sinks, s.len)) return;
    float* slot = slot_at<D>(a, number, kv) + (int64_t)key * D + 4 * lh;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int c = 32 * i + 8 * (e >> 2) + (e & 3);
            slot[c] = dk[i][e] + xch[(16 * i + e) * 64];
            slot[(int64_t)a.b.sinks * D + c] = (dv[i][e] + xch[(D / 2 + 16 * i + e) * 64]) * (1.f / P_SCALE);
        }
}

// The sinks' dk and dv: the second kernel's sums and the third's, in order.
template <int D>
__global__ __launch_bounds__(256) void window_attention_sinks_kernel(win::BwdArgs a) {
    using namespace win;
    const int seq = blockIdx.x / a.b.g, kv = blockIdx.x - seq * a.b.g;
    const Rows s = rows_of(a.b, seq);
    if (!has_far(a.b, s.len)) return;
    const int base = first_piece(a.b, seq, FAR_ROWS, 2);
    const int from = a.b.window / FAR_ROWS, to = (s.len - 1) / FAR_ROWS;
    const int64_t ld = (int64_t)(a.b.h + 2 * a.b.g) * D;
    const int64_t step = (int64_t)a.b.g * 2 * a.b.sinks * D;
    const int rows = min(a.b.sinks, s.len);
    for (int i = threadIdx.x; i < 2 * rows * D; i += 256) {
        const int which = i / (rows * D), row = (i - which * rows * D) / D, c = i % D;
        const float* p = slot_at<D>(a, base, kv) + ((int64_t)which * a.b.sinks + row) * D + c;
        float sum = *p;
        for (int k = from; k <= to; ++k) sum += p[(k + 1) * step];
        const _Float16 x = (_Float16)sum;
        a.dqkv[((int64_t)s.start + row) * ld + (int64_t)(a.b.h + which * a.b.g + kv) * D + c] = __builtin_bit_cast(uint16_t, x);
    }
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
    auto far = window_attention_far_kernel<D>;
    static const hipError_t cfg0 = allow_dynamic_lds(dq, DQ_LDS_BYTES<D>);
    if (cfg0 != hipSuccess) return cfg0;
    static const hipError_t cfg1 = allow_dynamic_lds(dkdv, KEY_LDS_BYTES<D>);
    if (cfg1 != hipSuccess) return cfg1;
    static const hipError_t cfg2 = allow_dynamic_lds(far, KEY_LDS_BYTES<D>);
    if (cfg2 != hipSuccess) return cfg2;
    hipLaunchKernelGGL(dq, dim3((unsigned)a.total_q), dim3(256), DQ_LDS_BYTES<D>, st, a);
    hipLaunchKernelGGL(dkdv, dim3((unsigned)a.total_k), dim3(256), KEY_LDS_BYTES<D>, st, a);
    if (a.b.sinks > 0 && a.b.T > a.b.window) {      // no sequence is longer than T
        hipLaunchKernelGGL(far, dim3((unsigned)(a.slot_numbers * a.b.g * ((a.b.sinks + 31) / 32))), dim3(128), KEY_LDS_BYTES<D>, st, a);
        hipLaunchKernelGGL(window_attention_sinks_kernel<D>, dim3((unsigned)(a.b.B * a.b.g)), dim3(256), 0, st, a);
    }
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
    a.numbers = (int)win::pieces(T, B, win::ROWS, 1);
    a.total_q = (int)(a.numbers * h);
    a.total_k = (int)(a.numbers * g);
    a.slot_numbers = (int)win::pieces(T, B, win::FAR_ROWS, 2);
    return d == 128 ? launch_backward_of<128>(a, st) : launch_backward_of<64>(a, st);
}

}  // namespace lomo
