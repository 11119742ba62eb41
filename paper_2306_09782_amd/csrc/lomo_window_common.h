// Pieces shared by the kernels of attention with a sliding window and sinks: which sequence a workgroup's rows belong to, tiles
// of D = 64 or 128 columns in LDS, their loads, fragment reads, and which pairs a mask leaves.
//
// Rows of q, k, v, o are packed: sequence b has the rows off[b] .. off[b + 1) - 1.  Query i of a sequence sees the keys j <= i
// with i - j < window or j < sinks.  A workgroup of four waves owns 128 rows (queries, or keys), 32 per wave, which stay in
// registers as MFMA fragments; pairs of [64 x D] tiles move along the sequence, double-buffered in LDS.  Scores are formed
// so that a lane owns one of the wave's rows; a block of 32 x 32 of them, one lane pair's sixteen registers, is what is masked,
// skipped or taken whole.
#pragma once
#include "lomo_attention_common.h"
#include "lomo_gemm_dma_common.h"

namespace lomo {
namespace win {

using attn::fragment_of;
using attn::pack2;
using attn::read8;
using attn::read_tr8;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int ROWS = 128, BLK = 64;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
template <int D>
constexpr int TILE = BLK * D;      // halves
template <int D>
constexpr int PAIR = 2 * TILE<D>;
template <int D>
constexpr float SCALE = D == 128 ? 0.08838834764831845f : 0.125f;      // 1 / sqrt(D)

// What the calls have in common.
struct Batch {
    const int32_t* off;      // [B + 1]
    int T, B, h, g;          // rows, sequences, query heads, key heads
    int window, sinks;
};

// A sequence's rows; offsets that do not ascend within [0, T] cannot lead outside the buffers.
struct Rows {
    int start, len;
};
__device__ __forceinline__ int clamped(const Batch& a, int b) { return min(max(a.off[b], 0), a.T); }
__device__ __forceinline__ Rows rows_of(const Batch& a, int b) {
    const int s = clamped(a, b), e = clamped(a, b + 1);
    return {s, max(e - s, 0)};
}

// Pieces of `unit` rows are numbered through all sequences without a table: those of sequence b begin at
// floor(off[b] / unit) + more * b, which leaves room for ceil(length / unit) + more - 1 of them.
__device__ __forceinline__ int first_piece(int start, int b, int unit, int more) { return start / unit + more * b; }
// The sequence that number i falls in, by a 64-way search of the wave, and its rows; -1: none.  The last round has the rows at hand.
__device__ __forceinline__ int sequence_of(const Batch& a, int i, int unit, int more, Rows& rows) {
    const int lane = threadIdx.x & 63;
    int lo = 0, n = a.B;
    while (true) {
        const int step = (n + 63) >> 6, at = lo + min(lane * step, n);      // at most off's last
        const int start = clamped(a, at);
        // how many from the first on: also where offsets do not ascend, the last of these begins at or before i
        const uint64_t before = __ballot(lane * step < n && first_piece(start, at, unit, more) <= i);
        const int count = ~before == 0 ? 64 : __builtin_ctzll(~before);
        if (count == 0) return -1;
        if (step > 1) {
            lo += (count - 1) * step;
            n = min(step, n - (count - 1) * step);
            continue;
        }
        const int seq = __builtin_amdgcn_readfirstlane(lo + count - 1);
        rows.start = __builtin_amdgcn_readlane(start, count - 1);
        const int end = count < 64 ? __builtin_amdgcn_readlane(start, count & 63) : clamped(a, seq + 1);
        rows.len = max(__builtin_amdgcn_readfirstlane(end) - rows.start, 0);
        return seq;
    }
}
inline int64_t pieces(int64_t T, int64_t B, int64_t unit, int64_t more) { return T / unit + more * B; }

// Place of workgroup `block` in an order of `total`, cut into one contiguous run for each XCD (block % 8), so that neighbours
// in the order meet in one L2.
__device__ __forceinline__ int place_of_block(int total, int block) {
    const int x = block & 7, local = block >> 3;
    const int q = total >> 3, r = total & 7;
    return x * q + (x < r ? x : r) + local;
}

// Chunk swizzle of a tile with 16-byte chunks: chunk c of row r sits at c ^ swz(r).  256-byte rows as in lomo_attention_common.h.  128-byte
// rows: rows r and r + 1 are on different halves of the banks anyway; r and r + 2 are 4 chunks apart (the four rows of a transposing read),
// the next two bits of r move by 1 .. 3 chunks (sixteen rows read at one column).
template <int D>
__device__ __forceinline__ int swz(int r) {
    if constexpr (D == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
    else return ((r & 2) << 1) | ((r >> 2) & 3);
}

// Load of [64 x D] tiles of rows `ld` elements apart, 64 of them less than 4 GiB.  Each of four waves fetches WROWS neighbouring rows, RPI with an
// instruction.  The instructions' swizzles differ from that of the first in two chunk bits; their offsets in memory and in LDS share the
// immediate, so that one value of M0 serves them all.
template <int D>
struct TileLoad {
    static constexpr int TROWS = BLK, WROWS = TROWS / 4, RPI = 512 / D, PER = WROWS / RPI;
    uint32_t voff, ld2, step;
    __device__ __forceinline__ TileLoad(int64_t ld, int wave) {
        const int lane = threadIdx.x & 63, rr = lane / (D / 8), c = lane % (D / 8);
        ld2 = 2u * (uint32_t)ld;
        step = RPI * ld2 - 1024u;      // what the scalar offset adds to the immediate
        voff = (uint32_t)rr * ld2 + (uint32_t)((c ^ swz<D>(rr) ^ ((WROWS * wave >> 2) & 3)) * 16);
    }
    // Row 0 of the tile is `tile` tiles from `rows0`, `left` rows of the sequence remain from there (any number); the others become zeros.
    __device__ __forceinline__ void issue(const uint16_t* rows0, int tile, int left, uint32_t lds, int wave) const {
        const char* base = reinterpret_cast<const char*>(rows0) + (uint64_t)(uint32_t)tile * (TROWS * ld2) + (uint64_t)((uint32_t)wave * WROWS * ld2);
        lds += (uint32_t)wave * (WROWS * D * 2u);
        uint32_t v[PER];
#pragma unroll
        for (int it = 0; it < PER; ++it) {
            v[it] = voff ^ (uint32_t)(((RPI * it >> 2) & 3) * 16);
            asm volatile("" : "+v"(v[it]));      // formed again each time, not kept in registers
        }
        if (left >= TROWS) {
            const auto srd = dma::make_srd(base, WROWS * ld2);
            if constexpr (PER == 4)
                asm volatile("s_mov_b32 m0, %8\n\ts_nop 0\n\t"
                             "buffer_load_dwordx4 %0, %4, 0 offen lds\n\t"
                             "buffer_load_dwordx4 %1, %4, %5 offen offset:0x400 lds\n\t"
                             "buffer_load_dwordx4 %2, %4, %6 offen offset:0x800 lds\n\t"
                             "buffer_load_dwordx4 %3, %4, %7 offen offset:0xc00 lds"
                             ::"v"(v[0]), "v"(v[1]), "v"(v[2]), "v"(v[3]), "s"(srd), "s"(step), "s"(2 * step), "s"(3 * step), "s"(lds) : "memory", "m0");
            else
                asm volatile("s_mov_b32 m0, %4\n\ts_nop 0\n\t"
                             "buffer_load_dwordx4 %0, %2, 0 offen lds\n\t"
                             "buffer_load_dwordx4 %1, %2, %3 offen offset:0x400 lds"
                             ::"v"(v[0]), "v"(v[1]), "s"(srd), "s"(step), "s"(lds) : "memory", "m0");
        } else {      // the descriptor ends behind the last row
            left -= WROWS * wave;
#pragma unroll
            for (int it = 0; it < PER; ++it) {
                const int n = min(left - RPI * it, RPI);
                dma::dma16(v[it], dma::make_srd(base + (uint64_t)(RPI * it) * ld2, n <= 0 ? 0u : (uint32_t)(n - 1) * ld2 + 2u * D), 0u, lds + 1024u * it);
            }
        }
    }
};

// Fragment reads from a tile at an LDS address that is a multiple of 256 bytes (see lomo_attention_common.h).
template <int D>
struct TileRead {
    uint32_t row_rd, tr0, tr1;
    __device__ __forceinline__ TileRead(uint32_t tile) {
        const int lane = threadIdx.x & 63;
        const int l32 = lane & 31, lh = lane >> 5;
        const int g4 = lane >> 4, j16 = lane & 15;
        const int mhalf = g4 & 1, kh = g4 >> 1, rib = j16 >> 2, piece = j16 & 3;
        const int tr_row = 8 * kh + rib, tr_col = 16 * mhalf + 4 * piece;
        row_rd = tile + 2u * (uint32_t)(l32 * D + ((8 * lh) ^ (swz<D>(l32) << 3)));
        tr0 = tile + 2u * (uint32_t)(tr_row * D + (tr_col ^ (swz<D>(tr_row) << 3)));
        tr1 = tile + 2u * (uint32_t)((tr_row + 4) * D + (tr_col ^ (swz<D>(tr_row + 4) << 3)));
    }
    __device__ __forceinline__ TileRead at(int halves) const {
        TileRead t = *this;
        t.row_rd += 2u * (uint32_t)halves;
        t.tr0 += 2u * (uint32_t)halves;
        t.tr1 += 2u * (uint32_t)halves;
        asm volatile("" : "+v"(t.row_rd), "+v"(t.tr0), "+v"(t.tr1));
        return t;
    }
    // rows 0 .. 31, columns 16 ks .. + 15: a lane holds eight consecutive columns of its row
    __device__ __forceinline__ half8 rows(int off, int ks) const { return read8((row_rd ^ (uint32_t)(32 * ks)) + 2u * (uint32_t)off); }
    // columns 32 i .. + 31, rows 16 ks .. + 15: a lane holds eight consecutive rows of its column
    __device__ __forceinline__ half8 columns(int off, int i, int ks) const {
        const uint32_t o = 2u * (uint32_t)(off + 16 * ks * D);
        return read_tr8((tr0 ^ (uint32_t)(64 * i)) + o, (tr1 ^ (uint32_t)(64 * i)) + o);
    }
};

// This lane's row as fragments: eight consecutive columns each.
template <int D>
__device__ __forceinline__ void load_fragments(half8 (&f)[D / 16], const uint16_t* row) {
    const int lh = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) f[ks] = *reinterpret_cast<const half8*>(row + 16 * ks + 8 * lh);
}
// Waits for them.  Without it the compiler, which does not see the loads to LDS, waits where they are used, in every turn of a loop: for all that
// is in flight there.
template <int D>
__device__ __forceinline__ void arrived(half8 (&f)[D / 16]) {
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) asm volatile("" : "+v"(f[ks]));
}

// acc[i][r]: column 32 i + 8 (r / 4) + 4 lh + r % 4 of the lane's row, rounded once.  Every lane takes part in the exchange; `row` is null for
// those that have no row.
template <int N>
__device__ __forceinline__ void store_rows(const floatx16 (&acc)[N], uint16_t* row) {
    const int lh = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        uint32_t pk[8];
#pragma unroll
        for (int r = 0; r < 16; r += 2) pk[r >> 1] = pack2(acc[i][r], acc[i][r + 1]);
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            const half8 f = fragment_of(pk, a);
            if (row != nullptr) *reinterpret_cast<half8*>(row + 32 * i + 16 * a + 8 * lh) = f;
        }
    }
}

// A product over a block that a mask cuts has zeros for the hidden pairs, and 0 * inf is not 0: the moving operand of such tiles is made
// finite in LDS first.  What sees the values all the same gets to know of them otherwise: their rows' lse and delta are not finite,
// and the forward adds them.  Each wave looks through the rows that it fetched; returned is one bit for each row that held any (uniform).
template <int D>
__device__ __forceinline__ uint32_t make_finite(uint32_t tile, int wave) {
    typedef __attribute__((address_space(3))) u32x4* chunk_p;
    using Load = TileLoad<D>;
    constexpr int RPI = Load::RPI, LANES = 64 / RPI;      // of a row
    const int lane = threadIdx.x & 63;
    uint32_t rows = 0;
#pragma unroll
    for (int it = 0; it < Load::PER; ++it) {
        chunk_p at = (chunk_p)(tile + (uint32_t)wave * (Load::WROWS * D * 2u) + (uint32_t)it * 1024u + (uint32_t)lane * 16u);
        u32x4 w = *at;
        uint32_t any = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t bad = (((w[e] & 0x7c007c00u) + 0x04000400u) & 0x80008000u) >> 15;      // an exponent of ones carries over
            any |= bad;
            w[e] &= ~(bad * 0xffffu);
        }
        const uint64_t lanes = __ballot(any != 0);
        if (lanes == 0) continue;
        *at = w;
#pragma unroll
        for (int r = 0; r < RPI; ++r) rows |= ((lanes >> (r * LANES)) & ((1ull << LANES) - 1)) != 0 ? 1u << (RPI * it + r) : 0u;
    }
    return rows;
}
__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }

// A mask leaves pairs of queries q0 .. q0 + 31 and keys k0 .. k0 + 31 (uniform in a wave).
__device__ __forceinline__ bool seen(int q0, int k0, int window, int sinks) {
    return k0 <= q0 + 31 && (q0 - (k0 + 31) < window || k0 < sinks);
}

}  // namespace win
}  // namespace lomo
