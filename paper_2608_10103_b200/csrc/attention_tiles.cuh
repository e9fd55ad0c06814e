// Attention for many query rows per KV head on the 5th-generation tensor cores, over binary16 keys and values of packed
// prompts or over the pages of the 4-bit cache.
//
// A CTA stays on its SM and takes row tiles one after another, longest first. A row tile is QT times 128 rows (queries x heads
// of a group) of one KV head, which walk the tokens in tiles of TN. Per tile: S = Q K^T (tcgen05.mma, operands in shared
// memory) into tensor memory; four warps, a thread per row, turn S into weights w = 2^(c s - m + 7), rounded to binary16, in the
// same place; O += w V (A operand in tensor memory). out = O / l with l the FP32 sum of the weights before rounding; m is
// a maximum seen earlier, renewed when a score passes it by 2^8 (see kv_attention.cuh), so that O rarely passes through
// registers. Scores, sums and statistics are FP32.
//
// Roles: a scheduler works out the next row tile while this one runs; a loader brings Q and, through a ring of tiles that runs
// on from one row tile into the next, K and V; an issuer for each 128 rows, so that neither waits for the other's softmax. Every 128 rows
// have two score buffers: the scores of the next tokens are computed while the softmax works on these.
//
// What bounds it, prompts at 128 d: 1530-1580 cycles per 64 tokens and pair of row tiles, which the products take by themselves: an
// instruction of Q K^T reads 128 rows of Q from shared memory, 64 cycles for 64 tokens as for 128, so that the two products come to 2 x (512 +
// 256). One buffer of 128 scores per row tile would halve the first, but scores -> maximum -> weights -> products then is a chain of 3400-3600
// cycles per 128 tokens (8192 tokens: 472-495 us against 453); tensor memory holds no more beside two results. The exponentials
// take 1024 cycles of the 1530. Tried and slower: two threads per row (684 us), the first half of the weights multiplied
// early; no faster: an eighth to half of the exponentials as polynomials, waits that spin. What would help is a pair of CTAs per pair of
// row tiles (cta_group::2), which leaves each tensor memory for two buffers of 128 scores: not built.
// A row tile's end, some 5000 cycles of which 2900 are its results' way out, is a sixth of a prompt of 1000 tokens.
// Measured, a few launches back to back: 8192 tokens, 32 heads on 8, 455 us (0.71 of the cuBLAS bf16 rate); 12 prompts of up to 2048 tokens
// 165 us; 4096 tokens of 256 d 265 us. In longer runs, and call by call with everything out of L2, the first two take 521 us (0.62) and 192: the
// clocks go down under the power limit, and 12 prompts' operands come from memory. 2 x 1024 queries over up to 8192 tokens in 4 bits 277-281 us, call
// by call 286: some 2700 cycles per 64 tokens. There the products are 2 x (512 + 512), the expansion of codes takes as long, and both want the
// same shared memory.
//
// Keys and values in binary16 come by tensor maps straight into the 128-byte swizzle: K-major for the first product and, read the
// other way round, MN-major for the second. Pages of 4-bit codes come by bulk copies, and warps write the same tiles from them. Keys
// are their codes, exact in binary16: a score is then scale (q . codes) + offset sum(q), by a table of two factors per token. Values are two
// tiles, multiplied one after the other: with the scale's first seven bits, and the middle of the range rounded to units of that, a value is
// exact in binary16 if the middle is no more than 16 of the scale's powers of two away from zero, as in every row with values of both signs; the second
// tile holds what is left, and what the first had to round where values lie further away, itself rounded to binary16 (2^-22 of the value; a tile is
// written twice then: 273 -> 373 us if all are such). (Keys and values rounded to binary16 once are 6e-4 of their norm away from the exact results, only
// values so 3.5e-4, this 2.5e-4; the rounded exact ones are 2e-4. Value scales folded into the weights, as in kv_attention_u4.cuh, need five
// factors a token for every row: what shared memory then hands to registers took longer, 340 us against 297.)
//
// What a masked place holds must not matter, but weight 0 times an infinity is NaN. A 4-bit token whose scale or
// offset is not finite gets zeros for values and a NaN for the scores' factor: NaN for the rows that see it, nothing for those that mask it.
// Binary16 values of tiles that hide a token from a row (a prompt's last tiles, a window's first ones) are looked at before they are multiplied, by
// the issuers while the softmax works on the scores (12 packed prompts 164 -> 166 us, 4096 tokens of 256 d 259 -> 265): what is not finite becomes 0 in
// shared memory, and is added to the results of the rows that see it, at the end. That costs a row tile 0.2 to 1 ms, however long its sequence is.
#pragma once

#include <cuda.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <type_traits>

#include "bounded_wait.cuh"
#include "kv_attention.cuh"
#include "kv_common.cuh"
#include "kv_host.cuh"
#include "ptx.cuh"

namespace b200gemm {

struct AttnTilesParams {
  int batch;
  const int* cu;
  const int* kv_len;  // null: each sequence's tokens are its rows
  int max_q, max_len, rows;
  int units;          // row tiles x KV heads at most, which scratch is there for
  int group, heads;   // query heads per KV head, KV heads
  const __half* q;
  long long q_token_stride, q_head_stride;
  __half* out;
  long long out_token_stride;
  float scale_log2;  // softmax_scale * log2(e)
  int causal, window;
  int split_rows;    // sequences of up to so many rows belong to another kernel
  int* status;
  // prompts
  const __half *k, *v;
  long long kv_token_stride, kv_head_stride;
  // 4-bit cache
  KvCacheU4View c;
  const int* table;
  int table_stride;
  // tokens of a row tile divided over several CTAs
  int splits;
  float* partial;     // [units][splits][ROWS][D + 4]
  unsigned* arrived;  // per unit, zero before and after
};

template <int D, bool U4>
struct AttnTileShape {
  static constexpr int QT = D <= 128 ? 2 : 1;    // row tiles of 128 per CTA
  static constexpr int TN = 64;                  // tokens per tile
  static constexpr int ROWS = 128 * QT;
  // Tiles of tokens that O takes up before it is split, see split_sums: 16384 tokens, in which 1e-4 of a result can be lost (8192 tokens: 5e-5, and
  // 1024 queries over 65536 tokens in 4 bits 1740 us instead of 1710; without it 1690).
  static constexpr int SUM_TILES = 16384 / TN;
  static constexpr int SOFTMAX_WARPS = 4 * QT;
  static constexpr int CONVERT_WARPS = U4 ? 12 : 0;
  // Warps that expand one tile of K or V together.  What a tile costs a warp is mostly waiting, so that several tiles are worked on
  // at a time, as far as there is room for their codes: tile by tile by all warps took 1.4 times as long.
  static constexpr int TILE_WARPS = D == 256 ? 4 : 2;
  static constexpr int GROUPS = 12 / TILE_WARPS;
  static constexpr int KINDS = U4 ? 3 : 2;       // tiles of the ring for TN tokens: K, V, and what V's binary16 leaves of it
  static constexpr int THREADS = 32 * (SOFTMAX_WARPS + 4 + CONVERT_WARPS);
  static constexpr int CHUNK = TN * 128;         // bytes of 64 d of a K or V tile
  static constexpr int TILE_BYTES = (D / 64) * CHUNK;
  static constexpr int Q_BYTES = QT * (D / 64) * 16384;
  static constexpr int SLOTS = U4 ? (D == 64 ? 12 : D == 128 ? 6 : 3) : (D == 64 ? 12 : D == 128 ? 8 : 4);  // tiles in the ring
  static constexpr int SLOT_OFFSET = Q_BYTES;
  static constexpr int RAW_BYTES = U4 ? TN * D / 2 : 0;  // codes of a K or V tile
  static constexpr int RAW_OFFSET = SLOT_OFFSET + SLOTS * TILE_BYTES;
  static constexpr int RAW_STAGES = D == 256 ? 2 : 4;  // rings of such tiles
  // A place of the ring of tiles, or of codes, belongs to one group of warps: it waits for every time that it is used, one by one, as a
  // barrier that tells a phase only from its neighbours needs it.
  static_assert(!U4 || (SLOTS % GROUPS == 0 && GROUPS % KINDS == 0 && RAW_STAGES * KINDS % GROUPS == 0), "places and groups");
  static constexpr int SCALE_OFFSET = RAW_OFFSET + 2 * RAW_STAGES * RAW_BYTES;
  static constexpr int SCALE_BYTES = U4 ? TN * 4 : 0;    // scales and offsets of a K or V tile
  // Ring of the scores' factors, four floats for two tokens.  They are written with a tile of K, up to SLOTS / KINDS tiles ahead of
  // the first product, and that up to two ahead of the softmax that reads them.
  static constexpr int TABLES = D == 256 ? 4 : 8;
  static_assert(TABLES >= SLOTS / KINDS + 2 || !U4, "no factor is replaced before it is read");
  static constexpr int TABLE_OFFSET = SCALE_OFFSET + 3 * RAW_STAGES * SCALE_BYTES;  // (of K and V with K's codes, of V with V's)
  static constexpr int TABLE_BYTES = U4 ? TN * 8 : 0;
  static constexpr int ITEM_OFFSET = TABLE_OFFSET + TABLES * TABLE_BYTES;
  static constexpr int ITEM_INTS = 16;
  static constexpr int BAR_OFFSET = ITEM_OFFSET + 2 * ITEM_INTS * 4;
  // item_full[2], item_empty[2], q_full, q_empty, s_full[4], p_full[4], o_done[2], drain[2], parts_written, parts_counted,
  // raw_full[2][4], raw_empty[2][4], table_full[8], turn_done[2][4], slot_full[], slot_empty[]
  static constexpr int BARS = 52 + 2 * SLOTS;
  static constexpr int MISC_OFFSET = BAR_OFFSET + BARS * 8;
  // 32 rows of OUT_COLUMNS results for each softmax warp, which leave as runs of 64 or 32 bytes; the pitch keeps rows off one another's
  // banks.  (Softmax warps of the 4-bit kernel have 128 registers up to 128 d: 16 columns at a time 292 -> 282 us there, at 256 d 619 -> 626,
  // on prompts 160 -> 165.)
  static constexpr int OUT_COLUMNS = U4 && D <= 128 ? 16 : 32;
  static constexpr int OUT_PITCH = OUT_COLUMNS * 2 + 16;
  static constexpr int OUT_OFFSET = MISC_OFFSET + 16;
  static constexpr int DYN_BYTES = OUT_OFFSET + SOFTMAX_WARPS * 32 * OUT_PITCH + 1024;
  static constexpr uint32_t O_COLUMN = 256;      // score (and weight) buffer i at TN i, two for each tile of rows; O behind them
  static_assert(DYN_BYTES <= 232448, "exceeds the 227 KB shared-memory limit per CTA");
  static_assert(O_COLUMN + QT * D <= 512, "tensor memory");
};

// What a CTA works on next.
struct AttnItem {
  int tiles;     // tiles of TN tokens; -1 = there is nothing more
  int row0;      // first row of the sequence in the packed arrays
  int n, base;   // its queries, the position of the first of them
  int seq, head;
  int query;     // first query of the row tile
  int active;    // tiles of 128 rows with a row in them
  int lo, hi;    // tokens
  int from;      // first token that any row sees
  int unit, split;
};
static_assert(sizeof(AttnItem) <= AttnTileShape<64, true>::ITEM_INTS * 4, "fits its place in shared memory");

__device__ __forceinline__ KvSeq attn_seq(const AttnTilesParams& p, int b, bool report) {
  KvSeq s;
  s.row0 = kv_ld(p.cu + b);
  s.n = kv_ld(p.cu + b + 1) - s.row0;
  s.len = p.kv_len ? kv_ld(p.kv_len + b) : 0;
  const int n = s.row0 < 0 ? 0 : max(0, min(s.n, min(p.max_q, p.rows - s.row0)));
  const int len = p.kv_len ? min(max(s.len, 0), p.max_len) : 0;
  if (report && (n != s.n || len != s.len)) kv_report(p.status);
  s.n = n;
  s.len = p.kv_len ? len : n;
  return s;
}

// The row tiles of all sequences, longest first (see kvt_item in kv_attention_tiles.cuh), by one warp, a lane per sequence.
template <int TN>
struct AttnOrder {
  const AttnTilesParams& p;
  int queries;  // of a row tile
  int all, longest;

  __device__ int tiles_of(const KvSeq& s) const {
    return static_cast<long long>(s.n) * p.group <= p.split_rows ? 0 : (s.n + queries - 1) / queries;
  }
  // Row tiles of a sequence that are at least x token tiles long: their last query sees beyond (x - 1) TN. A window is left out of
  // account: with one, the order is by position, and lengths are much alike but for a sequence's first tiles.
  __device__ int long_tiles(const KvSeq& s, int x) const {
    const int count = tiles_of(s);
    if (x <= 0) return count;
    if (!p.causal) return s.len > (x - 1) * TN ? count : 0;
    const int need = (x - 1) * TN - (s.len - s.n);  // first query that sees so far
    if (need <= 0) return count;
    return need < s.n ? count - need / queries : 0;
  }
  KvSeq mine;  // sequence `lane`
  __device__ KvSeq seq(int i) const { return i < 32 ? mine : attn_seq(p, i, false); }
  __device__ AttnOrder(const AttnTilesParams& params, int queries, bool report) : p(params), queries(queries), mine{} {
    const int lane = static_cast<int>(threadIdx.x) & 31;
    all = longest = 0;
    for (int i = lane; i < p.batch; i += 32) {
      const KvSeq s = attn_seq(p, i, report);
      if (i < 32) mine = s;
      longest = max(longest, s.len / TN + 1);
      all += tiles_of(s);
    }
    longest = static_cast<int>(__reduce_max_sync(0xffffffffu, static_cast<unsigned>(longest)));
    all = static_cast<int>(__reduce_add_sync(0xffffffffu, static_cast<unsigned>(all)));
  }
  // Where the last rank was: row tiles of x_lo token tiles (between x_lo and x_hi there are none), `beyond` of all sequences are longer, `upto`
  // that long or longer, `passed` of that length belong to sequences in front of `block`.
  int x_lo = 0, x_hi = 0, beyond = 0, upto = 0, block = 0, passed = 0;
  // (sequence, row tile) of a rank below `all`, none of them below the one before: looks on from there, as a search over all sequences for every rank
  // would take the square of their number (16384 sequences of 3 tokens: 84 ms).
  __device__ int2 at(int rank) {
    const int lane = static_cast<int>(threadIdx.x) & 31;
    if (p.batch == 1) return make_int2(0, all - 1 - rank);
    if (rank >= upto) {
      x_hi = upto == 0 ? longest + 1 : x_lo;
      beyond = upto;
      x_lo = 0;
      upto = all;
#pragma unroll 1
      while (x_hi - x_lo > 1) {  // more than rank tiles are x_lo long, `beyond` <= rank are x_hi long
        const int mid = (x_lo + x_hi) / 2;
        int c = 0;
        for (int i = lane; i < p.batch; i += 32) c += long_tiles(seq(i), mid);
        c = static_cast<int>(__reduce_add_sync(0xffffffffu, static_cast<unsigned>(c)));
        if (c > rank) {
          x_lo = mid;
          upto = c;
        } else {
          x_hi = mid;
          beyond = c;
        }
      }
      block = passed = 0;
    }
    int left = rank - beyond - passed;  // among the tiles of exactly that length, by sequence
#pragma unroll 1
    for (; block < p.batch; block += 32) {
      int same = 0, qt = 0;
      if (block + lane < p.batch) {
        const KvSeq s = seq(block + lane);
        const int longer = long_tiles(s, x_hi);
        same = long_tiles(s, x_lo) - longer;
        qt = tiles_of(s) - 1 - longer;  // its longest tile of that length
      }
      int incl = same;
      for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += up;
      }
      const unsigned holds = __ballot_sync(0xffffffffu, left < incl);
      if (holds) {
        const int from = __ffs(holds) - 1;
        return make_int2(block + from, __shfl_sync(0xffffffffu, qt - (left - (incl - same)), from));
      }
      const int here = __shfl_sync(0xffffffffu, incl, 31);
      left -= here;
      passed += here;
    }
    return make_int2(0, 0);  // (not reached: there are `rank - beyond` and more tiles of that length)
  }
};

namespace attn {

using ptx::add2;
using ptx::fma2;
using ptx::mul2;
using ptx::pair;
using ptx::unpair;
// Pairs of FP32 values, where they stand: the order of a pipeline written by hand.
__device__ __forceinline__ uint64_t fma2_here(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm volatile("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2_here(uint64_t a, uint64_t b) {
  uint64_t r;
  asm volatile("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float exp2_here(float x) {
  float r;
  asm volatile("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ uint32_t pack_here(float a, float b) {
  uint32_t r;
  asm volatile("cvt.rn.f16x2.f32 %0, %2, %1;" : "=r"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// 64 d of box_heads x box_tokens rows (see shared_row_map): coordinates d, head, row.
__device__ __forceinline__ void load_rows(uint32_t dst, const CUtensorMap* m, int d, int head, int row, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(d), "r"(head), "r"(row), "r"(bar)
      : "memory");
}
__device__ __forceinline__ bool not_finite2(uint32_t w) {  // either of two binary16
  return (w & 0x7c00u) == 0x7c00u || (w & 0x7c000000u) == 0x7c000000u;
}
__device__ __forceinline__ uint32_t fma_h2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}
__device__ __forceinline__ uint32_t add_h2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("add.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t sub_h2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("sub.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// Eight codes of a key as binary16 numbers, the subnormals c 2^-24 that they are as they stand, in the order of d.
__device__ __forceinline__ uint4 key_codes(uint32_t w) {
  const uint32_t a = w & 0x000f000fu, b = (w >> 4) & 0x000f000fu, c = (w >> 8) & 0x000f000fu, d = (w >> 12) & 0x000f000fu;
  return make_uint4(__byte_perm(a, b, 0x5410), __byte_perm(c, d, 0x5410), __byte_perm(a, b, 0x7632), __byte_perm(c, d, 0x7632));
}
// Eight codes of a value less 8, in the order d 0, 4, 1, 5, 2, 6, 3, 7: a nibble under the exponent of 1024 or of 64.
__device__ __forceinline__ uint4 value_codes(uint32_t w) {
  const uint32_t u = w >> 8;
  return make_uint4(sub_h2((w & 0x000f000fu) | 0x64006400u, 0x64086408u), sub_h2((w & 0x00f000f0u) | 0x54005400u, 0x54805480u),
                    sub_h2((u & 0x000f000fu) | 0x64006400u, 0x64086408u), sub_h2((u & 0x00f000f0u) | 0x54005400u, 0x54805480u));
}

// Two binary16 with 0 for what is not finite.
__device__ __forceinline__ uint32_t finite_or_zero2(uint32_t w) {
  return ((w & 0x7c00u) == 0x7c00u ? 0u : w & 0xffffu) | ((w & 0x7c000000u) == 0x7c000000u ? 0u : w & 0xffff0000u);
}

// A 4-bit value as two binary16, code - 8 times a factor plus a summand each: the scale's first seven bits and the rest; the middle (code 8)
// as a multiple of the unit that the former leaves, and the rest.
struct Value4Parts {
  float scale_hi, scale_lo, middle_hi, middle_lo;
  float round;  // 1.5 2^23 units
  __device__ uint32_t first() const { return kva::pack_halves(scale_hi, middle_hi); }
  __device__ uint32_t rest() const { return kva::pack_halves(scale_lo, middle_lo); }
  // Whether the first one may pass the 2^11 units that binary16 holds: 8 x 128 of the code's part and more than 1024 of the middle.
  __device__ bool far() const { return scale_hi != 0.0f && fabsf(middle_hi) * 0x1.8p13f > round; }
};
__device__ __forceinline__ Value4Parts value4_parts(uint32_t scale_offset) {
  Value4Parts x;
  const float2 f = kva::half2_of(scale_offset);
  x.scale_hi = __half2float(__ushort_as_half(static_cast<unsigned short>(scale_offset & 0xfff0u)));
  x.scale_lo = f.x - x.scale_hi;
  const float middle = fmaf(8.0f, f.x, f.y);
  // (a unit is 2^-6 of the scale's power of two, of 2^-14 below the normal range)
  x.round = __uint_as_float((__float_as_uint(fmaxf(fabsf(x.scale_hi), 0x1p-14f)) & 0x7f800000u) + (17u << 23) + 0x400000u);
  x.middle_hi = __half2float(__float2half_rn((middle + x.round) - x.round));
  x.middle_lo = middle - x.middle_hi;
  return x;
}
// The second binary16 of two codes with what rounding took from the first. All of that is exact: the middle and the first one lie within a factor of
// two of one another where the first was rounded, so that their difference is; with the code's part it is a rounding error, which has few bits.
__device__ __forceinline__ uint32_t value4_rest(uint32_t codes, uint32_t first_of, uint32_t rest_of) {
  const uint32_t factor = __byte_perm(first_of, 0, 0x1010), middle = __byte_perm(first_of, 0, 0x3232);
  const uint32_t lost = fma_h2(codes, factor, sub_h2(middle, fma_h2(codes, factor, middle)));
  return fma_h2(codes, __byte_perm(rest_of, 0, 0x1010), add_h2(__byte_perm(rest_of, 0, 0x3232), lost));
}

// Long sums. An instruction of 16 tokens cuts off up to two units of 2^-24 of what an accumulator holds, always towards zero: 131072 tokens of one
// sign in one sum lose 8.3e-4 of the result, more than its rounding to binary16. So a row's sums are split every 16384 tokens: their first eleven bits
// are put by as binary16, where the row's results will be (no scratch, and nothing shared), the rest stays and the sum goes on from there. The parts are
// exact. At the end they come together again.
// o: eight columns; held: what was put by, `factor` a unit of it; unit: of what is put by now, a power of two above the row's sum of weights; 0: the end.
__device__ __forceinline__ void split_sums(uint32_t* o, uint4* held, float factor, float unit) {
  uint32_t w[4] = {0, 0, 0, 0};
  if (factor != 0.0f) {
    const uint4 old = *held;
    w[0] = old.x; w[1] = old.y; w[2] = old.z; w[3] = old.w;
  }
  const float per = unit == 0.0f ? 0.0f : __uint_as_float(0x7f000000u - __float_as_uint(unit));
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const float2 old = kva::half2_of(w[u]);
    const float a = fmaf(old.x, factor, __uint_as_float(o[2 * u])), b = fmaf(old.y, factor, __uint_as_float(o[2 * u + 1]));
    o[2 * u] = __float_as_uint(a);
    o[2 * u + 1] = __float_as_uint(b);
    if (unit != 0.0f) {
      w[u] = kva::pack_halves(a * per, b * per);
      const float2 now = kva::half2_of(w[u]);
      // (an infinity is put by as a whole)
      o[2 * u] = fabsf(now.x) < INFINITY ? __float_as_uint(fmaf(-now.x, unit, a)) : 0u;
      o[2 * u + 1] = fabsf(now.y) < INFINITY ? __float_as_uint(fmaf(-now.y, unit, b)) : 0u;
    }
  }
  if (unit != 0.0f) *held = make_uint4(w[0], w[1], w[2], w[3]);
}

// Adds what is not finite in the values of tokens [first, last] of the packed arrays, 64 at most, to a row's results. An infinity has a
// weight above 0, however small, unless the row's score of it is -inf, which makes the product a NaN.
template <int D>
__device__ __noinline__ void add_not_finite(const AttnTilesParams& p, int row, int hq, int head, int first, int last) {
  const __half* const v = p.v + head * p.kv_head_stride;
  __half* const out = p.out + row * p.out_token_stride + static_cast<long long>(hq) * D;
  bool scored = false;
  uint64_t minus_inf = 0;  // tokens with that score, once one of them has an infinity
  auto score = [&]() {
    const __half* const q = p.q + row * p.q_token_stride + hq * p.q_head_stride;
    const __half* const k = p.k + head * p.kv_head_stride;
#pragma unroll 1
    for (int t = first; t <= last; ++t) {
      float sum = 0.0f;
#pragma unroll 2
      for (int d = 0; d < D; d += 8) {
        const uint4 a = ptx::ld_global_stream_v4(q + d), b = ptx::ld_global_stream_v4(k + t * p.kv_token_stride + d);
        const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float2 e = kva::half2_of(x[u]), f = kva::half2_of(y[u]);
          sum = fmaf(e.x, f.x, fmaf(e.y, f.y, sum));
        }
      }
      if (sum == -INFINITY) minus_inf |= 1ull << (t - first);
    }
    scored = true;
  };
#pragma unroll 1
  for (int d = 0; d < D; d += 8) {
    float sum[8];
    bool any = false;
#pragma unroll
    for (int u = 0; u < 8; ++u) sum[u] = 0.0f;
#pragma unroll 1
    for (int t0 = first; t0 <= last; t0 += 4) {
      uint4 x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = ptx::ld_global_stream_v4(v + min(t0 + i, last) * p.kv_token_stride + d);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
        if (t0 + i > last || !(not_finite2(w[0]) || not_finite2(w[1]) || not_finite2(w[2]) || not_finite2(w[3]))) continue;
        any = true;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const float y = __half2float(__ushort_as_half(static_cast<unsigned short>(w[u / 2] >> 16 * (u & 1))));
          if (fabsf(y) < INFINITY) continue;
          if (y == y && !scored) score();
          sum[u] += minus_inf >> (t0 + i - first) & 1 ? __int_as_float(0x7fffffff) : y;
        }
      }
    }
    if (!any) continue;
#pragma unroll
    for (int u = 0; u < 8; ++u) out[d + u] = __float2half_rn(__half2float(out[d + u]) + sum[u]);
  }
}

}  // namespace attn

// LONG: rows may see more than SUM_TILES tiles. (Calls whose bounds exclude it go without: over 4-bit pages the code for it takes
// 3 % by itself, 1640 -> 1690 us.)
template <int D, bool U4, bool LONG>
__global__ void __launch_bounds__(AttnTileShape<D, U4>::THREADS, 1)
attention_tiles_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
                       const __grid_constant__ CUtensorMap v_map, const __grid_constant__ AttnTilesParams p) {
  using namespace kva;
  using namespace attn;
  using T = AttnTileShape<D, U4>;
  constexpr int QT = T::QT, TN = T::TN, SLOTS = T::SLOTS;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = ptx::smem_addr(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* const base_ptr = smem_raw + (base - raw);
  const uint32_t bar0 = base + T::BAR_OFFSET;
  auto item_full = [&](int i) { return bar0 + 8u * i; };
  auto item_empty = [&](int i) { return bar0 + 8u * (2 + i); };
  const uint32_t q_full = bar0 + 8u * 4, q_empty = bar0 + 8u * 5;
  auto s_full = [&](int i) { return bar0 + 8u * (6 + i); };
  auto p_full = [&](int i) { return bar0 + 8u * (10 + i); };
  auto o_done = [&](int q) { return bar0 + 8u * (14 + q); };
  auto drain = [&](int q) { return bar0 + 8u * (16 + q); };
  const uint32_t parts_written = bar0 + 8u * 18, parts_counted = bar0 + 8u * 19;
  auto raw_full = [&](int which, int stage) { return bar0 + 8u * (20 + 4 * which + stage); };
  auto raw_empty = [&](int which, int stage) { return bar0 + 8u * (28 + 4 * which + stage); };
  auto table_full = [&](int i) { return bar0 + 8u * (36 + i); };
  auto turn_done = [&](int q, int w) { return bar0 + 8u * (44 + 4 * q + w); };
  auto slot_full = [&](int s) { return bar0 + 8u * (52 + s); };
  auto slot_empty = [&](int s) { return bar0 + 8u * (52 + SLOTS + s); };
  volatile uint32_t* const tmem_holder = reinterpret_cast<volatile uint32_t*>(base_ptr + T::MISC_OFFSET);
  volatile uint32_t* const abort_flag = tmem_holder + 1;
  volatile uint32_t* const last_flag = tmem_holder + 2;
  int* const cleared = reinterpret_cast<int*>(base_ptr + T::MISC_OFFSET + 12);  // 1 + the last item with a value taken out of its tiles

  const int tid = static_cast<int>(threadIdx.x), lane = tid & 31, warp = tid >> 5;
  constexpr int W_LOAD = T::SOFTMAX_WARPS, W_SCHEDULE = W_LOAD + 1, W_MMA = W_LOAD + 2;  // two issuers
  constexpr int CONSUMERS = T::SOFTMAX_WARPS + 1 + QT + T::CONVERT_WARPS;  // warps that read the items
  if (tid == 0) {
    ptx::grid_dep_launch_dependents();
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(item_full(i), 1);
      ptx::mbar_init(item_empty(i), CONSUMERS);
      ptx::mbar_init(s_full(2 * i), 1);
      ptx::mbar_init(s_full(2 * i + 1), 1);
      ptx::mbar_init(p_full(2 * i), 4);
      ptx::mbar_init(p_full(2 * i + 1), 4);
      ptx::mbar_init(o_done(i), 1);
      ptx::mbar_init(drain(i), 1);
      for (int stage = 0; stage < 4; ++stage) {
        ptx::mbar_init(raw_full(i, stage), 1);
        ptx::mbar_init(raw_empty(i, stage), i ? 2 * T::TILE_WARPS : T::TILE_WARPS);
      }
    }
    ptx::mbar_init(q_full, 1);
    ptx::mbar_init(q_empty, QT);
    ptx::mbar_init(parts_written, T::SOFTMAX_WARPS);
    ptx::mbar_init(parts_counted, 1);
    for (int i = 0; i < T::TABLES; ++i) ptx::mbar_init(table_full(i), T::TILE_WARPS);
    for (int i = 0; i < 8; ++i) ptx::mbar_init(turn_done(i >> 2, i & 3), 1);
    for (int i = 0; i < SLOTS; ++i) {
      ptx::mbar_init(slot_full(i), U4 ? T::TILE_WARPS : 1);
      ptx::mbar_init(slot_empty(i), QT);
    }
    *abort_flag = 0;
    *cleared = 0;
    ptx::fence_mbar_init();
  }
  if (warp == W_MMA) {
    ptx::tmem_alloc<1>(ptx::smem_addr(const_cast<uint32_t*>(tmem_holder)), 512);
    ptx::tmem_relinquish<1>();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  const uint32_t tmem = *tmem_holder;
  ptx::grid_dep_wait();

  const int per_tile = 128 / p.group;  // queries of 128 rows
  // The k-th item; false: give up.
  auto next_item = [&](int k, AttnItem& it) {
    bool ok = wait_bounded(item_full(k & 1), (k >> 1) & 1, abort_flag, p.status, DEV_TIMEOUT_PRODUCER);
    ok = __all_sync(0xffffffffu, ok);
    if (ok) it = *reinterpret_cast<const AttnItem*>(base_ptr + T::ITEM_OFFSET + (k & 1) * T::ITEM_INTS * 4);
    __syncwarp();
    if (ok && lane == 0) ptx::mbar_arrive(item_empty(k & 1));
    return ok;
  };

  // Every row of an item, of both its row tiles, which share the values in shared memory, sees the tokens [.x, .y].
  auto open_tokens = [&](const AttnItem& it) {
    return make_int2(p.window > 0 ? it.base + min(it.n, it.query + it.active * per_tile) - p.window : 0,
                     p.causal ? it.base + it.query : it.base + it.n - 1);
  };

  // A row's part of its results, where its tokens are divided: [D] sums, maximum, sum of weights.
  [[maybe_unused]] auto part_of = [&](const AttnItem& it, int row) {
    return p.partial + ((static_cast<long long>(it.unit) * p.splits + it.split) * T::ROWS + row) * (D + 4);
  };

  if constexpr (U4) {  // register shares: 256 x 128 + 512 x 56 of the 768 x 80 that the block was launched with, or 128 x 168 + 512 x 72 of 640 x 96
    if (warp < T::SOFTMAX_WARPS) {
      if constexpr (QT == 2)
        asm volatile("setmaxnreg.inc.sync.aligned.u32 128;");
      else
        asm volatile("setmaxnreg.inc.sync.aligned.u32 168;");
    } else {
      if constexpr (QT == 2)
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
      else
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    }
  }
  if (warp < T::SOFTMAX_WARPS) {
    // ------------------------------------------------------------------ softmax, one thread per row
    const int q = warp >> 2, r = (warp & 3) * 32 + lane;  // row of the 128
    const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t o_at = tmem + lane_base + T::O_COLUMN + static_cast<uint32_t>(q * D);
    const int in_tile = r / p.group, in_group = r - in_tile * p.group;
    const float c = p.scale_log2;
    const uint64_t c2 = pair(c, c);
    int done = 0;  // token tiles of this tile of rows so far
    int ring = 0;  // token tiles of the CTA before this item
    int joins = 0;
    int turns = 0;  // of this warp at the exponentials
    bool ok = true;
#pragma unroll 1
    for (int k = 0; ok; ++k) {
      AttnItem it;
      ok = next_item(k, it);
      if (!ok || it.tiles < 0) break;
      const int ring0 = ring;
      ring += it.tiles;
      if (q >= it.active) {
        // (the joining below is for all of these warps)
      } else {
        const int qi = it.query + q * per_tile + in_tile;  // query of the sequence
        const bool live = in_tile < per_tile && qi < it.n;
        const int hq = it.head * p.group + in_group;
        const int pos = p.causal ? it.base + qi : it.base + it.n - 1;  // sees tokens from .. pos
        const int from = p.window > 0 ? pos - p.window + 1 : 0;
        const int q0 = it.query + q * per_tile;
        const int all_hi = p.causal ? it.base + q0 : pos;
        const int all_lo = p.window > 0 ? it.base + min(it.n, q0 + per_tile) - p.window : 0;
        float m = -INFINITY, l = 0.0f;
        uint64_t q_sum2 = 0;  // the sum of the row's values, twice
        if constexpr (U4) {
          float sum = 0.0f;
          if (live) {
            const __half* const src = p.q + (static_cast<long long>(it.row0) + qi) * p.q_token_stride + hq * p.q_head_stride;
#pragma unroll 4
            for (int d = 0; d < D; d += 8) {
              uint32_t w[4];
              asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(src + d) : "memory");
#pragma unroll
              for (int v = 0; v < 4; ++v) {
                const float2 f = half2_of(w[v]);
                sum += f.x + f.y;
              }
            }
          }
          q_sum2 = pair(sum, sum);
        }
#pragma unroll 1
        for (int j = 0; ok && j < it.tiles;) {
          const int end = LONG ? min(it.tiles, j + T::SUM_TILES) : it.tiles;
#pragma unroll 1
          for (; j < end; ++j, ++done) {
            const int sb = 2 * q + (done & 1);  // score buffer
            const uint32_t s_at = tmem + lane_base + static_cast<uint32_t>(sb * TN);
            ok = wait_bounded(s_full(sb), (done >> 1) & 1, abort_flag, p.status, DEV_TIMEOUT_EPILOGUE);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            ptx::tc_fence_after_sync();
            uint32_t x[TN / 32][32];
#pragma unroll
            for (int h = 0; h < TN / 32; ++h) ptx::tmem_ld_32x32b_x32(s_at + h * 32, x[h]);
            ptx::tmem_wait_ld();
            if constexpr (U4) {  // scores in the units of the exponent: scale (q . codes) + offset sum(q)
              ok = wait_bounded(table_full((ring0 + j) % T::TABLES), ((ring0 + j) / T::TABLES) & 1, abort_flag, p.status, DEV_TIMEOUT_EPILOGUE);
              ok = __all_sync(0xffffffffu, ok);
              if (!ok) break;
              const uint32_t table = base + T::TABLE_OFFSET + static_cast<uint32_t>(((ring0 + j) % T::TABLES) * T::TABLE_BYTES);
#pragma unroll
              for (int h = 0; h < TN / 32; ++h)
#pragma unroll
                for (int v = 0; v < 32; v += 2) {
                  uint64_t a, b;
                  asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(a), "=l"(b) : "r"(table + (h * 32 + v) * 8) : "memory");
                  const float2 t = unpair(fma2(pair(__uint_as_float(x[h][v]), __uint_as_float(x[h][v + 1])), a, mul2(b, q_sum2)));
                  x[h][v] = __float_as_uint(t.x);
                  x[h][v + 1] = __float_as_uint(t.y);
                }
            }
            const int tok0 = it.lo + j * TN;
            if (tok0 + TN - 1 > all_hi || tok0 < all_lo) {
              const int last = pos - tok0, first = from - tok0;
#pragma unroll
              for (int h = 0; h < TN / 32; ++h)
#pragma unroll
                for (int v = 0; v < 32; ++v)
                  if (h * 32 + v > last || h * 32 + v < first) x[h][v] = 0xff800000u;  // -inf
            }
            float mx[8];  // (chains of their own)
#pragma unroll
            for (int u = 0; u < 8; ++u) mx[u] = fmaxf(__uint_as_float(x[0][u]), __uint_as_float(x[0][u + 8]));
#pragma unroll
            for (int i = 16; i < TN; i += 16)
#pragma unroll
              for (int u = 0; u < 8; ++u)
                mx[u] = max3(mx[u], __uint_as_float(x[(i + u) / 32][(i + u) % 32]), __uint_as_float(x[(i + u + 8) / 32][(i + u + 8) % 32]));
            float top = max3(max3(mx[0], mx[1], mx[2]), max3(mx[3], mx[4], mx[5]), fmaxf(mx[6], mx[7]));
            if constexpr (!U4) top *= c;
            const bool grow = top > m + 8.0f;
            if (__any_sync(0xffffffffu, grow)) {
              const float now = grow ? top : m;
              const float f = now == -INFINITY ? 1.0f : exp2_approx(m - now);
              m = now;
              l *= f;
              if (j > 0) {  // O of the tiles before, once their products are done
                ok = wait_bounded(o_done(q), (done - 1) & 1, abort_flag, p.status, DEV_TIMEOUT_EPILOGUE);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                ptx::tc_fence_after_sync();
#pragma unroll 1
                for (int d = 0; d < D; d += 16) {
                  uint32_t y[16];  // (few registers: the scores are in the others)
                  ptx::tmem_ld_32x32b_x16(o_at + d, y);
                  ptx::tmem_wait_ld();
#pragma unroll
                  for (int v = 0; v < 16; ++v) y[v] = __float_as_uint(__uint_as_float(y[v]) * f);
                  ptx::tmem_st_32x32b_x16(o_at + d, y);
                }
                ptx::tmem_wait_st();
              }
            }
            // The warps of an SM quarter that have a row tile each take turns at the exponentials, which one warp keeps busy.
            // (Left alone they fall into step: both at the exponentials, then both at everything else.)
            if (it.active == 2) {
              if (q == 1 || turns > 0)
                ok = wait_bounded(turn_done(q ^ 1, warp & 3), (q == 1 ? turns : turns - 1) & 1, abort_flag, p.status, DEV_TIMEOUT_EPILOGUE);
              ok = __all_sync(0xffffffffu, ok);
              if (!ok) break;
              ++turns;
            }
            // weights, two per column, over the scores: 32 tokens take 16 columns
            const float at_ref = KVA_WEIGHT_BITS - (m == -INFINITY ? 0.0f : m);
            const uint64_t at2 = pair(at_ref, at_ref);
            uint64_t sum[2] = {pair(0.0f, 0.0f), pair(0.0f, 0.0f)};
            {
              // Pair i is summed up and packed LAG pairs after its exponentials were asked for.
              constexpr int PAIRS = TN / 2, LAG = 4;
              auto exponent = [&](int i) {
                const uint64_t x2 = pair(__uint_as_float(x[i / 16][i % 16 * 2]), __uint_as_float(x[i / 16][i % 16 * 2 + 1]));
                return unpair(U4 ? add2_here(x2, at2) : fma2_here(x2, c2, at2));
              };
              float2 e[LAG + 1], t = exponent(0);
              uint32_t w[16];
#pragma unroll
              for (int i = 0; i < PAIRS + LAG; ++i) {
                if (i < PAIRS) {
                  e[i % (LAG + 1)].x = exp2_here(t.x);
                  e[i % (LAG + 1)].y = exp2_here(t.y);
                  if (i + 1 < PAIRS) t = exponent(i + 1);
                }
                if (i == PAIRS - 1 && it.active == 2 && lane == 0) ptx::mbar_arrive(turn_done(q, warp & 3));
                if (i >= LAG) {
                  const int o = i - LAG;
                  const float2 v = e[o % (LAG + 1)];
                  sum[o & 1] = add2_here(sum[o & 1], pair(v.x, v.y));
                  w[o % 16] = pack_here(v.x, v.y);
                  if (o % 16 == 15) ptx::tmem_st_32x32b_x16(s_at + (o / 16) * 16, w);
                }
              }
            }
            ptx::tmem_wait_st();
            if (j > 0 && j == end - 1) {
              // A barrier tells a phase from the one before or behind it only.  That S was there says that the products of the tile before
              // the last are done (they were issued earlier, by the same thread); the last one's are seen to here, in front of this one's,
              // so that the wait for these, below, is not taken in by them.
              ok = wait_bounded(o_done(q), (done - 1) & 1, abort_flag, p.status, DEV_TIMEOUT_EPILOGUE);
              ok = __all_sync(0xffffffffu, ok);
              if (!ok) break;
            }
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(p_full(sb));
            const float2 total = unpair(add2(sum[0], sum[1]));
            l += total.x + total.y;
          }
          if (!LONG || !ok || it.tiles <= T::SUM_TILES) break;
          // ---- long sums
          ok = wait_bounded(o_done(q), (done - 1) & 1, abort_flag, p.status, DEV_TIMEOUT_EPILOGUE);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          ptx::tc_fence_after_sync();
          const bool parts = U4 && it.split >= 0;
          __half* const mine = parts ? reinterpret_cast<__half*>(part_of(it, q * 128 + r)) + D
                                     : p.out + (static_cast<long long>(it.row0) + qi) * p.out_token_stride + static_cast<long long>(hq) * D;
          // (all rows have a place: eight columns of 32 rows side by side, or every access is to 32 lines)
          const bool dense = __all_sync(0xffffffffu, parts || live);
          // log2 of the unit of what was put by, with the reference of that time: in the row's place for results on their way out, which is free here
          const uint32_t held_at = base + T::OUT_OFFSET + static_cast<uint32_t>((warp * 32 + lane) * T::OUT_PITCH);
          float held = -INFINITY;
          if (j > T::SUM_TILES) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(held) : "r"(held_at) : "memory");
          const float factor = held == -INFINITY ? 0.0f : exp2_approx(held - m);
          const float unit = j == it.tiles ? 0.0f : l > 0.0f && l < 0x1p100f ? __uint_as_float((__float_as_uint(l) & 0x7f800000u) + 0x1000000u) : 1.0f;
#pragma unroll 1
          for (int d = 0; d < D; d += 16) {
            uint32_t y[16];
            ptx::tmem_ld_32x32b_x16(o_at + d, y);
            ptx::tmem_wait_ld();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int piece = (d / 8 + h) * 32 + lane;
              __half* const there = reinterpret_cast<__half*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(mine), piece / (D / 8))) + piece % (D / 8) * 8;
              if (dense || live) split_sums(y + 8 * h, reinterpret_cast<uint4*>(dense ? there : mine + d + 8 * h), factor, unit);
            }
            __syncwarp();
            ptx::tmem_st_32x32b_x16(o_at + d, y);
          }
          ptx::tmem_wait_st();
          held = m + (static_cast<float>(__float_as_uint(unit) >> 23) - 127.0f);
          asm volatile("st.shared.f32 [%0], %1;" ::"r"(held_at), "f"(held) : "memory");
        }
        if (!ok) break;
        // ---- the rows' results
        if (it.tiles > 0) {
          ok = wait_bounded(o_done(q), (done - 1) & 1, abort_flag, p.status, DEV_TIMEOUT_EPILOGUE);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          ptx::tc_fence_after_sync();
        }
        // (a row that sees a token has l > 0, or NaN; or all its scores are -inf, which makes it NaN)
        if (l == 0.0f && pos >= max(from, 0) && it.split < 0) l = __int_as_float(0x7fffffff);
        const float inv = l == 0.0f ? 0.0f : __fdividef(1.0f, l);
        float* const part = U4 && it.split >= 0 ? part_of(it, q * 128 + r) : nullptr;
        if (U4 && part && live) *reinterpret_cast<float2*>(part + D) = make_float2(m, l);
        __half* const dst = p.out + (static_cast<long long>(it.row0) + qi) * p.out_token_stride + static_cast<long long>(hq) * D;
        const unsigned alive = __ballot_sync(0xffffffffu, live);
        const uint32_t stage = base + T::OUT_OFFSET + static_cast<uint32_t>(warp * 32 * T::OUT_PITCH);
        constexpr int COLUMNS = T::OUT_COLUMNS, PIECES = COLUMNS / 8, RUN_ROWS = 32 / PIECES;  // 16-byte pieces of a run, rows that a store covers
        auto load_columns = [&](int d, uint32_t (&x)[COLUMNS]) {
          if constexpr (COLUMNS == 32)
            ptx::tmem_ld_32x32b_x32(o_at + d, x);
          else
            ptx::tmem_ld_32x32b_x16(o_at + d, x);
        };
        __half* run[PIECES];  // of rows lane / PIECES + RUN_ROWS i
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
          run[i] = reinterpret_cast<__half*>(
                       __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(dst), lane / PIECES + RUN_ROWS * i)) + lane % PIECES * 8;
        uint32_t x[COLUMNS];
#pragma unroll
        for (int v = 0; v < COLUMNS; ++v) x[v] = 0;
        if (it.tiles > 0) load_columns(0, x);
#pragma unroll 1
        for (int d = 0; d < D; d += COLUMNS) {
          ptx::tmem_wait_ld();
          uint32_t z[COLUMNS];
          // (columns of 4-bit values lie in the order in which words of codes come apart: 0, 4, 1, 5, ...)
#pragma unroll
          for (int v = 0; v < COLUMNS; ++v) z[v] = U4 ? x[(v & 24) + ((v & 7) < 4 ? 2 * (v & 7) : 2 * (v & 7) - 7)] : x[v];
          uint32_t y[COLUMNS / 2];
#pragma unroll
          for (int v = 0; v < COLUMNS / 2; ++v) y[v] = pack_halves(__uint_as_float(z[2 * v]) * inv, __uint_as_float(z[2 * v + 1]) * inv);
          if (U4 && part) {  // O as it stands, to be joined
#pragma unroll
            for (int v = 0; v < COLUMNS / 4; ++v)
              if (live) *reinterpret_cast<uint4*>(part + d + 4 * v) = make_uint4(z[4 * v], z[4 * v + 1], z[4 * v + 2], z[4 * v + 3]);
            __syncwarp();
          }
          if (it.tiles > 0 && d + COLUMNS < D) load_columns(d + COLUMNS, x);  // (on its way while these leave)
          if (!(U4 && part)) {
#pragma unroll
            for (int v = 0; v < PIECES; ++v) {
              ptx::st_shared_v4(stage + lane * T::OUT_PITCH + v * 16, y[4 * v], y[4 * v + 1], y[4 * v + 2], y[4 * v + 3]);
            }
            __syncwarp();
            uint4 w[PIECES];
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
              ptx::ld_shared_v4(stage + (lane / PIECES + RUN_ROWS * i) * T::OUT_PITCH + lane % PIECES * 16, w[i].x, w[i].y, w[i].z, w[i].w);
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
              if (alive >> (lane / PIECES + RUN_ROWS * i) & 1u) *reinterpret_cast<uint4*>(run[i] + d) = w[i];
            __syncwarp();
          }
        }
        ptx::tc_fence_before_sync();
        if constexpr (!U4) {
          if (live && *const_cast<volatile int*>(cleared) > k) {
            const int2 open = open_tokens(it);
#pragma unroll 1
            for (int j = 0; j < it.tiles; ++j) {
              const int tok = it.lo + j * TN, first = max(tok, from), last = min(tok + TN - 1, pos);
              if ((tok + TN - 1 > open.y || tok < open.x) && first <= last) add_not_finite<D>(p, it.row0 + qi, hq, it.head, it.row0 + first, it.row0 + last);
            }
          }
        }
        __syncwarp();
      }
      if (U4 && it.split >= 0) {
        // ---- the CTA that finishes a row tile last joins its parts, in their order
        __threadfence();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(parts_written);
        ok = wait_bounded(parts_written, joins & 1, abort_flag, p.status, DEV_TIMEOUT_EPILOGUE);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (tid == 0) {
          *last_flag = atomicAdd(p.arrived + it.unit, 1u) == static_cast<unsigned>(p.splits - 1);
          ptx::mbar_arrive(parts_counted);
        }
        ok = wait_bounded(parts_counted, joins & 1, abort_flag, p.status, DEV_TIMEOUT_EPILOGUE);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        ++joins;
        if (!*last_flag) continue;
        __threadfence();
        if (tid == 0) p.arrived[it.unit] = 0;
        const float* const parts = p.partial + static_cast<long long>(it.unit) * p.splits * T::ROWS * (D + 4);
#pragma unroll 1
        for (int i = tid; i < T::ROWS * (D / 4); i += 32 * T::SOFTMAX_WARPS) {
          const int rr = i / (D / 4), d = i % (D / 4) * 4;
          const int row = rr & 127, tile = rr >> 7, qin = row / p.group, qi = it.query + tile * per_tile + qin;
          if (tile >= it.active || qin >= per_tile || qi >= it.n) continue;
          const float* const mine = parts + rr * (D + 4);
          float top = -INFINITY, l = 0.0f;
          float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          for (int s = 0; s < p.splits; ++s) top = fmaxf(top, __ldcg(mine + static_cast<long long>(s) * T::ROWS * (D + 4) + D));
          const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll 4
          for (int s = 0; s < p.splits; ++s) {
            const float* const at = mine + static_cast<long long>(s) * T::ROWS * (D + 4);
            const float2 ml = __ldcg(reinterpret_cast<const float2*>(at + D));
            const float4 x = __ldcg(reinterpret_cast<const float4*>(at + d));
            const float f = exp2_approx(ml.x - ref);
            l = fmaf(ml.y, f, l);
            o.x = fmaf(x.x, f, o.x);
            o.y = fmaf(x.y, f, o.y);
            o.z = fmaf(x.z, f, o.z);
            o.w = fmaf(x.w, f, o.w);
          }
          if (l == 0.0f && it.base + qi >= 0) l = __int_as_float(0x7fffffff);
          const float inv = l == 0.0f ? 0.0f : __fdividef(1.0f, l);
          __half2* const dst = reinterpret_cast<__half2*>(
              p.out + (static_cast<long long>(it.row0) + qi) * p.out_token_stride +
              (static_cast<long long>(it.head) * p.group + (row - qin * p.group)) * D + d);
          dst[0] = __floats2half2_rn(o.x * inv, o.y * inv);
          dst[1] = __floats2half2_rn(o.z * inv, o.w * inv);
        }
      }
    }
  } else if (warp == W_SCHEDULE) {
    // ------------------------------------------------------------------ scheduler
    AttnOrder<TN> order(p, QT * per_tile, blockIdx.x == 0);
    // (sequences that overlap, or a count of row tiles that they make pass 32 bits: no row tile has a place behind the last)
    const bool fits = order.all >= 0 && static_cast<long long>(order.all) * p.heads <= p.units;
    if (!fits && blockIdx.x == 0 && lane == 0) kv_report(p.status);
    const int grid = static_cast<int>(gridDim.x), total = (fits ? order.all * p.heads : order.all < 0 ? 0 : p.units) * p.splits;
    bool ok = true;
#pragma unroll 1
    for (int k = 0, round = 0; ok; ++k, ++round) {
      // every other round backwards: who got the longest of one gets the shortest of the next
      const int at = round * grid + (round & 1 ? grid - 1 - static_cast<int>(blockIdx.x) : static_cast<int>(blockIdx.x));
      AttnItem it = {};
      it.tiles = -1;
      const bool more = at < total;  // (only the last round has gaps)
      if (more) {
        it.unit = at / p.splits;
        it.split = at - it.unit * p.splits;
        const int rank = it.unit / p.heads;
        it.head = it.unit - rank * p.heads;
        const int2 where = order.at(rank);
        const KvSeq s = attn_seq(p, where.x, false);
        it.seq = where.x;
        it.row0 = s.row0;
        it.n = s.n;
        it.base = s.len - s.n;
        it.query = where.y * QT * per_tile;
        const int queries = min(QT * per_tile, s.n - it.query);
        it.active = QT == 2 && queries > per_tile ? 2 : 1;
        it.hi = p.causal ? max(0, it.base + it.query + queries) : s.len;
        it.from = kv_first_seen(it.base + it.query, p.window);
        it.lo = it.from / TN * TN;
        it.tiles = max(0, (it.hi - it.lo + TN - 1) / TN);
        if (p.splits > 1) {  // this CTA's part of the tokens
          const int per = (it.tiles + p.splits - 1) / p.splits, first = min(it.tiles, it.split * per);
          it.tiles = min(it.tiles, first + per) - first;
          it.lo += first * TN;
          it.hi = min(it.hi, it.lo + it.tiles * TN);
        } else {
          it.split = -1;
        }
      }
      ok = wait_bounded(item_empty(k & 1), ((k >> 1) & 1) ^ 1, abort_flag, p.status, DEV_TIMEOUT_PRODUCER);
      ok = __all_sync(0xffffffffu, ok);
      if (ok && lane == 0) {
        *reinterpret_cast<AttnItem*>(base_ptr + T::ITEM_OFFSET + (k & 1) * T::ITEM_INTS * 4) = it;
        ptx::mbar_arrive(item_full(k & 1));
      }
      __syncwarp();
      if (!more) break;
    }
  } else if (warp == W_LOAD) {
    // ------------------------------------------------------------------ loader
    const uint32_t q_box = static_cast<uint32_t>(per_tile * p.group) * 128u;
    int tile = 0;  // tiles in the ring so far (FP16), tiles of tokens (4-bit)
    bool ok = true;
#pragma unroll 1
    for (int k = 0, used = 0; ok; ++k) {
      AttnItem it;
      ok = next_item(k, it);
      if (!ok || it.tiles < 0) break;
      if (it.tiles == 0) continue;
      ok = wait_bounded(q_empty, (used & 1) ^ 1, abort_flag, p.status, DEV_TIMEOUT_PRODUCER);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      ++used;
      if (lane == 0) {
        ptx::mbar_arrive_expect_tx(q_full, q_box * static_cast<uint32_t>(it.active * (D / 64)));
        for (int q = 0; q < it.active; ++q)
          for (int d = 0; d < D / 64; ++d)
            load_rows(base + (q * (D / 64) + d) * 16384, &q_map, d * 64, it.head * p.group, it.row0 + it.query + q * per_tile, q_full);
      }
      __syncwarp();
      if constexpr (!U4) {
#pragma unroll 1
        for (int j = 0; j < 2 * it.tiles; ++j, ++tile) {  // K, V by turns
          const int slot = tile % SLOTS;
          ok = wait_bounded(slot_empty(slot), ((tile / SLOTS) & 1) ^ 1, abort_flag, p.status, DEV_TIMEOUT_PRODUCER);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          if (lane == 0) {
            ptx::mbar_arrive_expect_tx(slot_full(slot), T::TILE_BYTES);
            for (int d = 0; d < D / 64; ++d)
              load_rows(base + T::SLOT_OFFSET + slot * T::TILE_BYTES + d * T::CHUNK, j & 1 ? &v_map : &k_map, d * 64, it.head,
                        it.row0 + it.lo + (j >> 1) * TN, slot_full(slot));
          }
          __syncwarp();
        }
      } else {
        // Lane g looks after the tile's g-th run of `run` tokens: one page, or half a tile's worth of a longer one.
        const int run = min(p.c.page, TN), runs = TN / run;
        const uint32_t run_bytes = static_cast<uint32_t>(run * D / 2);
        const int* const table = p.table + static_cast<long long>(it.seq) * p.table_stride;
        auto visible = [&](int j) {  // the lane's run of tile j, or a part of it
          const int tok = it.lo + j * TN + run * lane;
          return lane < runs && j < it.tiles && tok < it.hi && tok + run > it.from;
        };
        auto load_id = [&](int j) {  // its page, or -1
          return visible(j) ? kv_ld(table + ((it.lo + j * TN + run * lane) >> p.c.page_shift)) : -1;
        };
        int id = load_id(0);
#pragma unroll 1
        for (int j = 0; j < it.tiles && ok; ++j, ++tile) {
          const int id_next = load_id(j + 1);
          const bool in = visible(j);
          const bool good = in && id >= 0 && id < p.c.num_pages;
          if (in && !good) kv_report(p.status);
          const int tok = it.lo + j * TN + run * lane;
          const uint64_t token = good ? (static_cast<uint64_t>(id) * p.heads + it.head) * p.c.page + (tok & (p.c.page - 1)) : 0;
          const uint32_t count = static_cast<uint32_t>(__popc(__ballot_sync(0xffffffffu, good)));
#pragma unroll 1
          for (int which = 0; which < 2; ++which) {
            const int stage = tile % T::RAW_STAGES;
            const uint32_t full = raw_full(which, stage);
            ok = wait_bounded(raw_empty(which, stage), ((tile / T::RAW_STAGES) & 1) ^ 1, abort_flag, p.status, DEV_TIMEOUT_PRODUCER);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            // (runs that are left out keep what the buffers held)
            if (lane == 0) ptx::mbar_arrive_expect_tx(full, count * (run_bytes + static_cast<uint32_t>(run) * (which ? 4u : 8u)));
            __syncwarp();
            if (good) {
              ptx::bulk_load(base + T::RAW_OFFSET + (2 * stage + which) * T::RAW_BYTES + lane * run_bytes,
                             (which ? p.c.codes[1] : p.c.codes[0]) + token * (D / 2), run_bytes, full);
              const uint32_t scales = base + T::SCALE_OFFSET + stage * 3 * T::SCALE_BYTES + lane * run * 4;
              if (which == 0) ptx::bulk_load(scales, p.c.scales[0] + token, run * 4, full);
              ptx::bulk_load(scales + (which ? 2 : 1) * T::SCALE_BYTES, p.c.scales[1] + token, run * 4, full);
            }
          }
          id = id_next;
        }
      }
    }
    if (!ok) {
      // Gave up: let the copies in flight land before the CTA exits.
      const uint64_t start = ptx::globaltimer_ns();
      while (ptx::globaltimer_ns() - start < 1000000ull) {
      }
    }
  } else if (warp < W_MMA + QT && warp >= W_MMA) {
    // ------------------------------------------------------------------ MMA issuer of tile q of the rows
    // What addresses and control flow depend on is the same in all lanes; made from lane 0's, so that the compiler sees it and
    // keeps descriptors in uniform registers.
    const int q = __shfl_sync(0xffffffffu, warp, 0) - W_MMA;
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
    const bool elected = ptx::elect_one();
    constexpr uint32_t idesc_qk = ptx::make_idesc<ptx::KIND_F16>(128, TN);
    constexpr uint32_t idesc_pv = ptx::make_idesc<ptx::KIND_F16>(128, D) | ptx::IDESC_B_MN_MAJOR;
    const uint64_t q_desc = ptx::smem_desc_sw128(base + q * (D / 64) * 16384);
    const uint64_t k_desc = ptx::smem_desc_sw128(base + T::SLOT_OFFSET);
    const uint64_t v_desc = ptx::smem_desc_sw128_mn(base + T::SLOT_OFFSET, T::CHUNK);
    int slot = 0;          // of the next tile in the ring that has not been multiplied yet: V's, K's being up to two token tiles ahead
    uint32_t phase = 0;    // of that place
    int done = 0;          // token tiles of these rows
    bool ok = true;
    // `ahead` tiles on from there
    auto place = [&](int ahead, uint32_t& its_phase) {
      const int s = slot + ahead;
      its_phase = s >= SLOTS ? phase ^ 1u : phase;
      return s >= SLOTS ? s - SLOTS : s;
    };
    auto wait_all = [&](uint32_t bar, uint32_t parity) {
      const bool there = wait_bounded(bar, parity, abort_flag, p.status, DEV_TIMEOUT_MMA);
      return __all_sync(0xffffffffu, there) != 0;
    };
    auto advance = [&](int by) {
      slot += by;
      if (slot >= SLOTS) {
        slot -= SLOTS;
        phase ^= 1u;
      }
    };
    // What is not finite in a tile of values that hides tokens becomes 0, while the softmax still works on the scores. With two row tiles
    // both issuers may find the same values: they write the same, and neither multiplies before it has done so itself.
    [[maybe_unused]] auto take_out = [&](uint32_t values, int item) {
      uint32_t zero[4] = {0, 0, 0, 0};  // sums of the values times 0
#pragma unroll 8
      for (int i = lane * 16; i < T::TILE_BYTES; i += 512) {
        uint32_t w[4];
        ptx::ld_shared_v4(values + i, w[0], w[1], w[2], w[3]);
#pragma unroll
        for (int u = 0; u < 4; ++u) zero[u] = fma_h2(w[u], 0u, zero[u]);
      }
      if (((zero[0] | zero[1] | zero[2] | zero[3]) & 0x7fff7fffu) != 0) {  // a NaN among them
        atomicMax(cleared, item + 1);
        __threadfence_block();
#pragma unroll 1
        for (int i = lane * 16; i < T::TILE_BYTES; i += 512) {
          uint32_t w[4];
          ptx::ld_shared_v4(values + i, w[0], w[1], w[2], w[3]);
          ptx::st_shared_v4(values + i, finite_or_zero2(w[0]), finite_or_zero2(w[1]), finite_or_zero2(w[2]), finite_or_zero2(w[3]));
        }
        ptx::fence_proxy_async_smem();
      }
      __syncwarp();
    };
#pragma unroll 1
    for (int k = 0, used = 0; ok; ++k) {
      AttnItem it;
      ok = next_item(k, it);
      const int tiles = __shfl_sync(0xffffffffu, it.tiles, 0), active = __shfl_sync(0xffffffffu, it.active, 0);
      if (!ok || tiles < 0) break;
      if (tiles == 0) continue;
      ok = wait_all(q_full, used & 1);
      if (!ok) break;
      ++used;
      if (q >= active) {  // nothing to do but to let the ring go round
        if (elected) ptx::mbar_arrive(q_empty);
#pragma unroll 1
        for (int j = 0; j < T::KINDS * tiles && ok; ++j) {
          ok = wait_all(slot_full(slot), phase);
          if (ok && elected) ptx::mbar_arrive(slot_empty(slot));
          __syncwarp();
          advance(1);
        }
        continue;
      }
      // Scores of the token tile whose K lies `ahead` tiles on in the ring.
      auto qk = [&](int j, int ahead) {
        uint32_t its_phase;
        int at = place(ahead % SLOTS, its_phase);
        its_phase ^= static_cast<uint32_t>(ahead / SLOTS) & 1u;
        if (!wait_all(slot_full(at), its_phase)) return false;
        ptx::tc_fence_after_sync();
        const int sb = 2 * q + ((done + j) & 1);
        const uint64_t b = k_desc + static_cast<uint32_t>(at * (T::TILE_BYTES >> 4));
        if (elected) {
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)
            ptx::mma_ss<ptx::KIND_F16, 1>(tm + sb * TN, q_desc + static_cast<uint32_t>((kk >> 2) * (16384 >> 4) + (kk & 3) * 2),
                                          b + static_cast<uint32_t>((kk >> 2) * (T::CHUNK >> 4) + (kk & 3) * 2), idesc_qk, kk > 0);
          ptx::mma_commit<1>(s_full(sb));
          ptx::mma_commit<1>(slot_empty(at));
          if (j == tiles - 1) ptx::mma_commit<1>(q_empty);
        }
        __syncwarp();
        return true;
      };
      for (int j = 0; j < 2 && j < tiles && ok; ++j) ok = qk(j, T::KINDS * j);
      [[maybe_unused]] const int2 open = open_tokens(it);
#pragma unroll 1
      for (int j = 0; j < tiles && ok; ++j) {
        const int sb = 2 * q + ((done + j) & 1);
        int at[T::KINDS];
#pragma unroll
        for (int i = 1; i < T::KINDS; ++i) {
          uint32_t its_phase;
          at[i] = place(i, its_phase);
          ok = ok && wait_all(slot_full(at[i]), its_phase);
        }
        if constexpr (!U4) {
          const int tok0 = it.lo + j * TN;
          if (ok && (tok0 + TN - 1 > open.y || tok0 < open.x)) take_out(base + T::SLOT_OFFSET + at[1] * T::TILE_BYTES, k);
        }
        ok = ok && wait_all(p_full(sb), ((done + j) >> 1) & 1);
        if (!ok) break;
        ptx::tc_fence_after_sync();
        if (elected) {
#pragma unroll
          for (int i = 1; i < T::KINDS; ++i) {
            const uint64_t v = v_desc + static_cast<uint32_t>(at[i] * (T::TILE_BYTES >> 4));
#pragma unroll
            for (int kk = 0; kk < TN / 16; ++kk)
              ptx::mma_f16_ts(tm + T::O_COLUMN + q * D, tm + sb * TN + kk * 8, v + static_cast<uint32_t>(kk * (2048 >> 4)), idesc_pv,
                              j > 0 || i > 1 || kk > 0);
            if (i == T::KINDS - 1) ptx::mma_commit<1>(o_done(q));
            ptx::mma_commit<1>(slot_empty(at[i]));
          }
        }
        __syncwarp();
        // (the scores go where the weights are: the MMAs of this thread run in order)
        if (j + 2 < tiles) ok = qk(j + 2, 2 * T::KINDS);
        advance(T::KINDS);
      }
      done += tiles;
    }
    if (!ok && elected) {
      // Gave up: wait for the MMAs already issued before tensor memory is released.
      ptx::mma_commit<1>(drain(q));
      const uint64_t start = ptx::globaltimer_ns();
      while (!ptx::mbar_try_wait(drain(q), 0) && ptx::globaltimer_ns() - start < WAIT_LIMIT_NS) {
      }
    }
    __syncwarp();
  } else if (U4 && warp >= W_LOAD + 4) {
    // ------------------------------------------------------------------ K and V: 4-bit codes to binary16 tiles
    constexpr int AT_ONCE = 32 * T::TILE_WARPS;     // threads of a tile
    const int group = (warp - (W_LOAD + 4)) / T::TILE_WARPS, ct = tid % AT_ONCE;
    constexpr int PER_TOKEN = D / 32;               // 16-byte pieces of a token's codes: 32 d, 64 bytes of a row of a chunk
    constexpr int N = TN * PER_TOKEN / AT_ONCE;     // pieces per thread and tile
    constexpr int WARP_TOKENS = 32 / PER_TOKEN;     // tokens that a warp covers at a time (its lanes: neighbouring tokens, whose
                                                    // rows the swizzle keeps off one another's banks)
    const int piece = lane / WARP_TOKENS, t0 = ct / 32 * WARP_TOKENS + lane % WARP_TOKENS;
    int tile = 0;  // of the ring
    bool ok = true;
#pragma unroll 1
    for (int k = 0; ok; ++k) {
      AttnItem it;
      ok = next_item(k, it);
      if (!ok || it.tiles < 0) break;
      const int tile0 = tile;
      tile += T::KINDS * it.tiles;
#pragma unroll 1
      for (int i = tile0 + (group + T::GROUPS * SLOTS - tile0 % T::GROUPS) % T::GROUPS; i < tile; i += T::GROUPS) {
        const int nth = i / T::KINDS, kind = i - nth * T::KINDS, j = nth - tile0 / T::KINDS;  // token tile of the CTA, of the item
        const int which = kind > 0, slot = i % SLOTS, stage = nth % T::RAW_STAGES;
        ok = wait_bounded(raw_full(which, stage), (nth / T::RAW_STAGES) & 1, abort_flag, p.status, DEV_TIMEOUT_PRODUCER) &&
             wait_bounded(slot_empty(slot), ((i / SLOTS) & 1) ^ 1, abort_flag, p.status, DEV_TIMEOUT_PRODUCER);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        const uint32_t codes = base + T::RAW_OFFSET + (2 * stage + which) * T::RAW_BYTES + static_cast<uint32_t>(piece * 16);
        const uint32_t* const scales = reinterpret_cast<const uint32_t*>(base_ptr + T::SCALE_OFFSET + stage * 3 * T::SCALE_BYTES);
        const uint32_t to = base + T::SLOT_OFFSET + slot * T::TILE_BYTES + static_cast<uint32_t>((piece >> 1) * T::CHUNK);
        const int first = it.lo + j * TN;
        // (what stands for tokens that no row sees was not loaded or may be anything: zeros)
        auto seen = [&](int tok) { return first + tok < it.hi && first + tok >= it.from; };
        uint32_t of_token[TN / 32];  // V: factor and summand of tokens lane, lane + 32
        bool far = false;            // of these: the first tile may have had to round
        if (kind == 0) {  // the scores' factors; a NaN for a token whose key or value is not finite
#pragma unroll
          for (int tok = ct; tok < TN; tok += AT_ONCE) {
            const uint32_t mine = scales[tok];
            const float2 f = half2_of(mine);
            const bool good = !not_finite2(mine) && !not_finite2(scales[TN + tok]);
            float* const table = reinterpret_cast<float*>(base_ptr + T::TABLE_OFFSET + (nth % T::TABLES) * T::TABLE_BYTES) + (tok >> 1) * 4 + (tok & 1);
            table[0] = !seen(tok) ? 0.0f : good ? p.scale_log2 * f.x * 0x1p24f : __int_as_float(0x7fffffff);
            table[2] = seen(tok) && good ? p.scale_log2 * f.y : 0.0f;
          }
        } else {
#pragma unroll
          for (int u = 0; u < TN / 32; ++u) {
            const int tok = lane + 32 * u;
            const uint32_t mine = scales[2 * TN + tok];
            const Value4Parts x = value4_parts(mine);
            const uint32_t w = kind == 1 ? x.first() : x.rest();
            of_token[u] = seen(tok) && !not_finite2(mine) ? w : 0u;
            if (of_token[u] != 0 && x.far()) far = true;
          }
        }
#pragma unroll 4
        for (int u = 0; u < N; ++u) {
          const int tok = u * (AT_ONCE / PER_TOKEN) + t0;
          uint32_t w[4];
          ptx::ld_shared_v4(codes + tok * (D / 2), w[0], w[1], w[2], w[3]);
          const uint32_t at = to + static_cast<uint32_t>(tok * 128), sw = static_cast<uint32_t>(tok & 7);
          if (kind == 0) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              const uint4 x = key_codes(w[v]);
              ptx::st_shared_v4(at + (((static_cast<uint32_t>((piece & 1) * 4 + v)) ^ sw) << 4), x.x, x.y, x.z, x.w);
            }
          } else {
            // (the tokens of a warp's lanes lie within 32 of one another's multiple)
            uint32_t mine = __shfl_sync(0xffffffffu, of_token[0], tok & 31);
            const uint32_t later = __shfl_sync(0xffffffffu, of_token[1], tok & 31);
            if (tok >= 32) mine = later;
            const uint32_t factor = __byte_perm(mine, 0, 0x1010), summand = __byte_perm(mine, 0, 0x3232);
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              const uint4 x = value_codes(w[v]);
              ptx::st_shared_v4(at + (((static_cast<uint32_t>((piece & 1) * 4 + v)) ^ sw) << 4), fma_h2(x.x, factor, summand),
                                fma_h2(x.y, factor, summand), fma_h2(x.z, factor, summand), fma_h2(x.w, factor, summand));
            }
          }
        }
        if (kind == 2 && __any_sync(0xffffffffu, far)) {  // values far from zero for their range: the same once more, with what was rounded
#pragma unroll 1
          for (int u = 0; u < N; ++u) {
            const int tok = u * (AT_ONCE / PER_TOKEN) + t0;
            const uint32_t mine = scales[2 * TN + tok];
            const bool good = seen(tok) && !not_finite2(mine);
            const Value4Parts x = value4_parts(mine);
            const uint32_t first_of = good ? x.first() : 0u, rest_of = good ? x.rest() : 0u;
#pragma unroll 1
            for (int v = 0; v < 4; ++v) {
              uint32_t w;
              asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(codes + tok * (D / 2) + v * 4) : "memory");
              const uint4 c = value_codes(w);
              ptx::st_shared_v4(to + static_cast<uint32_t>(tok * 128) + ((static_cast<uint32_t>((piece & 1) * 4 + v) ^ static_cast<uint32_t>(tok & 7)) << 4),
                                value4_rest(c.x, first_of, rest_of), value4_rest(c.y, first_of, rest_of),
                                value4_rest(c.z, first_of, rest_of), value4_rest(c.w, first_of, rest_of));
            }
          }
        }
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          if (kind == 0) ptx::mbar_arrive(table_full(nth % T::TABLES));
          ptx::mbar_arrive(slot_full(slot));
          ptx::mbar_arrive(raw_empty(which, stage));
        }
      }
    }
  }

  // Every role gets here: all waits are bounded, and the last products have been waited for above.
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (warp == W_MMA) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc<1>(tmem, 512);
  }
}

// longest: what a row may see at most.
template <int D, bool U4>
int launch_attention_tiles(const SharedDevice& dev, int longest, int grid, cudaStream_t stream, const CUtensorMap& q, const CUtensorMap& k,
                           const CUtensorMap& v, const AttnTilesParams& p) {
  using T = AttnTileShape<D, U4>;
  auto with = [&](auto is_long) {
    constexpr auto kernel = attention_tiles_kernel<D, U4, decltype(is_long)::value>;
    const int rc = allow_smem<kernel>(dev, T::DYN_BYTES);
    return rc != GEMM_OK ? rc : launch(dev, kernel, dim3(grid), T::THREADS, T::DYN_BYTES, stream, q, k, v, p);
  };
  return longest > T::SUM_TILES * T::TN ? with(std::true_type{}) : with(std::false_type{});
}

}  // namespace b200gemm
