// Attention over the INT8 cache for few query rows per KV head (decoding, verification of a few
// tokens), and the general path for everything else.
//
// Mathematics.  The rows that share a KV head (queries x heads of its group) form one tile of
// 8 NR rows, so the cache is read once for all of them.  With page scales sk, sv, codes K, V and
// weights relative to a running reference m,
//     t = c sk (q . K) + log2 sv,   w = 2^(t - m + 7),   O = sum w V,   l = sum w / sv,   out = O / l,
// c = softmax_scale log2 e: the value scale is folded into the exponent, so that O needs one
// accumulator whatever the pages' scales are, and the softmax denominator takes it out again.  m is a
// maximum seen earlier, renewed when a score passes it by 2^8 (O and l are
// rescaled a few times per sequence instead of at every new maximum).  m, l, O and the scores are FP32;
// w is rounded to binary16 for the product with V (codes are exact in binary16): off by 2^-11 of itself,
// the rounding of the result, down to 2^-21 of the largest; a smaller one by up to 2^-32 of the largest.  The 2^7
// uses what binary16 has above a maximum of 2^8: without it weights lose bits from 2^-14 of the
// largest on and vanish at 2^-25, which long flat tails behind one large weight notice.
//
// q . K runs on the integer MMA, on the codes as they are: a row of q is held as
// q = s (254 q1 + q2) with int8 q1, q2 and s = max|q| / (127 * 254), i.e. to 1.6e-5 of the row's
// largest value, a thirtieth of the binary16 rounding of the weights.  Two exact INT32 sums per score
// take the place of 5 instructions for every four codes that binary16 operands would need.
// V has to meet fractional weights: a code becomes binary16 by placing code ^ 0x80 under the
// exponent of 1024 (prmt) and subtracting 1152.
//
// What bounds it: reading the codes once (2 D bytes a token and KV head).  So, as in few_rows.cuh, a
// thread fetches exactly the pieces its own fragments need, by cp.async into a ring nobody else
// reads: no barrier, no bank conflict, and DEPTH steps of 16 tokens in flight per warp.  The
// positions an MMA gives a thread are filled with whatever 16 bytes are contiguous: K's d order is
// permuted (q in the same order), V's d order is permuted over the rows of the result.
// Groups of eight rows fit the MMAs exactly: q1 and q2 of eight rows are the 16 rows of m16n8k32 against
// 8 tokens, and the sums come out where O^T = V^T w^T (m16n8k16: 16 d, 8 rows, 16 tokens) wants its weights,
// so nothing moves between lanes and a single decoding row pays for eight, not sixteen.
//
// Work split: the (sequence, row tile, head) units, cut into pieces of equal length.  With few units
// (at most a quarter of the CTAs) every CTA takes one piece of one unit; else the units, laid end to
// end in steps of 16 tokens, are cut into equal contiguous shares whatever their lengths are.  A CTA's
// warps share a piece; a piece that is not a whole unit leaves its m, l, O in scratch, and the CTA that
// finishes a unit last joins its pieces in their order (no second launch, and no dependence on who was
// last).  What runs once per CTA or piece is kept short and rolled up: between other kernels of a
// model its instructions are fetched anew each time, at some ten cycles an instruction.
//
// Measured (32 heads on 8 KV heads, 128 d): 64 sequences of up to 8192 tokens 131 us, 4.1 TB/s of codes; one of 131072
// tokens 72 us; one of 1000 tokens 10.6 us.  16 heads of 64 d, 131071 tokens, 4 queries: 58 us, 4.6 TB/s.  Two thirds of
// the copy rate: the issue slots are 0.3 busy, and a step waits for its own bytes, its shuffles and its MMAs in
// turn; the rings fill shared memory and the fragments the registers, so more warps would have shorter rings.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

#include "kv_cache.cuh"
#include "ptx.cuh"
#include "warp_pieces.cuh"

namespace b200gemm {

constexpr int KVA_WARPS = 4;
constexpr int KVA_THREADS = 32 * KVA_WARPS;
constexpr int KVA_STEP = 16;  // tokens per step
// What beginning a unit costs a CTA, in steps: the latencies of its q, page ids and first codes and the
// exchange between the warps, some 8-10 k cycles where four warps take 3 k for four steps.  Without it in the
// balance the CTAs with several short sequences were a fifth behind the others.
constexpr int KVA_UNIT_COST = 12;

// A weight of the reference is 2^7: with scores up to 2^8 beyond it, weights reach 2^15 of binary16's 65504.
constexpr float KVA_WEIGHT_BITS = 7.0f;
// A value scale as the exponent takes it.  Pages of zeros have none, but their tokens count in l; and 1 / sv times a
// weight must stay in FP32.  127 * 2^-40 = 1.2e-10 is nothing to a binary16 result (multiples of 6e-8).
__device__ __forceinline__ float kva_value_scale(float sv) { return sv < 0x1p-40f ? 0x1p-40f : sv; }

struct KvAttnParams {
  KvCacheView c;
  int batch;
  const int* cu;
  const int* kv_len;
  const int* table;
  int table_stride;
  int max_q;
  int rows;     // rows of q and out
  int max_len;  // tokens a row of the table can name
  int group;    // query heads per KV head
  const __half* q;
  long long q_token_stride, q_head_stride;
  __half* out;
  long long out_token_stride;
  float scale_log2;  // softmax_scale * log2(e)
  int window;        // 0 = all
  int split_rows;    // sequences of more than this many rows (queries x group) go to the tile kernel
  int* status;
  int min_share;     // steps per CTA at least
  int max_tiles;     // row tiles of a sequence at most
  float* partial;    // [2 * grid][rows * D + rows * 2]
  unsigned* arrived; // per unit, zero before and after
  int splits;        // tile kernel: CTAs a row tile's tokens are divided over
  float* long_sums;  // tile kernel: [slots][rows of a CTA][D] for CTAs with many tokens, or null
  unsigned* taken;   // per slot, zero before and after
  int slots;         // as many as CTAs can be resident
};

// A sequence's rows and length, cut to what the packed arrays, the table and the caller's bound allow.
struct KvSeq {
  int row0, n, len;
};
__device__ __forceinline__ KvSeq kv_seq_of(const KvAttnParams& p, int row0, int row1, int kv_len, bool report) {
  KvSeq s;
  s.row0 = row0;
  s.n = row1 - row0;
  s.len = kv_len;
  const int n = s.row0 < 0 ? 0 : max(0, min(s.n, min(p.max_q, p.rows - s.row0))), len = min(max(s.len, 0), p.max_len);
  if (report && (n != s.n || len != s.len)) kv_report(p.status);
  s.n = n;
  s.len = len;
  return s;
}
__device__ __forceinline__ KvSeq kv_seq(const KvAttnParams& p, int b, bool report) {
  const int row0 = kv_ld(p.cu + b), row1 = kv_ld(p.cu + b + 1), len = kv_ld(p.kv_len + b);
  return kv_seq_of(p, row0, row1, len, report);
}
// Tokens [lo, hi) that the queries [i0, i1) of a sequence see between them, lo rounded down to a step.
__device__ __forceinline__ void kv_visible(const KvAttnParams& p, const KvSeq& s, int i0, int i1,
                                           int& lo, int& hi) {
  const int base = s.len - s.n;  // position of query 0; may be negative
  hi = max(0, base + i1);
  lo = p.window > 0 ? max(0, base + i0 - p.window + 1) : 0;
  lo = lo / KVA_STEP * KVA_STEP;
  if (hi < lo) hi = lo;
}
__device__ __forceinline__ int kv_steps(int lo, int hi) {  // a unit has one step at least
  return max(1, (hi - lo + KVA_STEP - 1) / KVA_STEP);
}

namespace kva {

// Copies and loads at compile-time offsets from one base register (an address of its own per piece
// costs two or three instructions each, more than the copy).  bytes = 0 writes zeros and reads nothing.
template <int DST, int SRC, int BYTES>
__device__ __forceinline__ void cp_async(uint32_t dst, const void* src, int bytes) {
  if constexpr (BYTES == 16)
    asm volatile("cp.async.cg.shared.global [%0+%3], [%1+%4], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes), "n"(DST), "n"(SRC) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0+%3], [%1+%4], %5, %2;" ::"r"(dst), "l"(src), "r"(bytes), "n"(DST), "n"(SRC), "n"(BYTES) : "memory");
}
template <int OFF>
__device__ __forceinline__ void lds_v4(uint32_t at, uint32_t (&w)[4]) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4+%5];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at), "n"(OFF) : "memory");
}
template <int OFF>
__device__ __forceinline__ void lds_v2(uint32_t at, uint32_t& a, uint32_t& b) {
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2+%3];" : "=r"(a), "=r"(b) : "r"(at), "n"(OFF) : "memory");
}
template <int I>
struct Index {
  __host__ __device__ constexpr operator int() const { return I; }
};
// f(i) for i = 0 .. N-1, with i a constant expression inside f
template <int N, int I = 0, class F>
__device__ __forceinline__ void each(F&& f) {
  if constexpr (I < N) {
    f(Index<I>{});
    each<N, I + 1>(f);
  }
}
__device__ __forceinline__ uint32_t sub_1152(uint32_t h) {
  uint32_t r;
  asm("sub.f16x2 %0, %1, %2;" : "=r"(r) : "r"(h), "r"(0x64806480u));
  return r;
}
// bytes 0, 1 resp. 2, 3 of w (codes ^ 0x80) as two binary16 codes
__device__ __forceinline__ uint32_t lo_halves(uint32_t w) { return sub_1152(__byte_perm(w, 0x64646464u, 0x4140)); }
__device__ __forceinline__ uint32_t hi_halves(uint32_t w) { return sub_1152(__byte_perm(w, 0x64646464u, 0x4342)); }

__device__ __forceinline__ float exp2_approx(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float2 half2_of(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
// Four values of at most 127 as q1 + q2 / 254, int8 each, packed: rounding by adding 1.5 * 2^23, whose low
// byte then is the integer.
__device__ __forceinline__ void split_q(float a, float b, float c, float d, uint32_t& q1, uint32_t& q2) {
  constexpr float MAGIC = 12582912.0f;
  const float v[4] = {a, b, c, d};
  uint32_t h[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float r = v[i] + MAGIC;
    h[i] = __float_as_uint(r);
    l[i] = __float_as_uint(fmaf(v[i] - (r - MAGIC), 254.0f, MAGIC));
  }
  q1 = __byte_perm(__byte_perm(h[0], h[1], 0x0040), __byte_perm(h[2], h[3], 0x0040), 0x5410);
  q2 = __byte_perm(__byte_perm(l[0], l[1], 0x0040), __byte_perm(l[2], l[3], 0x0040), 0x5410);
}
__device__ __forceinline__ uint32_t pack_halves(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

}  // namespace kva

// Where a step's two scales travel: with its codes, a copy per lane (two more requests a step), or by lane, 32
// pages at a time like the ids (two shuffles).  At 64 d, where a step has six other requests, the latter is
// 27 % faster (16 x 131071 tokens: 79.5 -> 58 us); at 128 d the former by 2-8 %.
__host__ __device__ constexpr bool kva_scales_in_ring(int dim) { return dim >= 128; }
// Bytes of one ring slot of a warp: 16 tokens of K and V, and perhaps each lane's copy of both scales.
__host__ __device__ constexpr int kva_slot_bytes(int dim) { return KVA_STEP * 2 * dim + (kva_scales_in_ring(dim) ? 256 : 0); }
__host__ __device__ constexpr int kva_rows_floats(int rows, int dim) { return rows * (dim + 2); }
// Dynamic shared memory: the rings, reused for the warps' results; Q fragments where they are kept there.
// Fragments of q: 8 words a thread for 64 d and 8 rows; kept in registers up to 32 of them.
__host__ __device__ constexpr int kva_q_bytes(int dim, int nr) { return nr * (dim / 64) * 1024; }
__host__ __device__ constexpr bool kva_q_in_regs(int dim, int nr) { return dim * nr <= 256; }
// Steps that go through the softmax together (independent chains of arithmetic for a warp to overlap).
__host__ __device__ constexpr int kva_sub(int dim, int nr) { return dim * nr <= 256 ? 2 : 1; }
// Dynamic shared memory: q fragments, then the rings, reused for the warps' results and the weights of a join.
__host__ __device__ constexpr int kva_smem(int dim, int nr, int depth) {
  const int ring = KVA_WARPS * depth * kva_slot_bytes(dim);
  const int merge = KVA_WARPS * kva_rows_floats(8 * nr, dim) * 4;
  return (ring > merge ? ring : merge) + kva_q_bytes(dim, nr);
}
// CTAs an SM is meant to hold (registers: O takes dim * nr / 4 a thread).  At 128 d and 8 rows three with rings of
// four steps and 168 registers run 2-6 % ahead of four with three steps and 128 (which spill); two CTAs of
// six or eight warps behind them on long batches (64 x <= 8192 tokens: 127.6, 130.9, 136.9 us).
__host__ __device__ constexpr int kva_ctas(int dim, int nr) { return dim * nr <= 64 ? 4 : dim * nr <= 256 ? 3 : 2; }

template <int D, int NR, int DEPTH>
__global__ void __launch_bounds__(KVA_THREADS, kva_ctas(D, NR)) kv_attention_kernel(const KvAttnParams p) {
  using namespace kva;
  using namespace warp_pieces;
  constexpr int ROWS = 8 * NR;
  constexpr int KC = D / 64;                  // 64-byte pieces of a row of K
  constexpr int KP = 2 * KC;                  // 16-byte pieces of K per thread and step
  constexpr int VP = D >= 128 ? D / 128 : 1;  // pieces of V per token (8 bytes for D = 64)
  constexpr int VW = D == 64 ? 2 : 4;         // words of such a piece
  constexpr int OT = D / 16;                  // tiles of 16 d of the result
  constexpr int SUB = kva_sub(D, NR);
  constexpr bool Q_REGS = kva_q_in_regs(D, NR), SCALES_RING = kva_scales_in_ring(D);
  constexpr int SLOT = kva_slot_bytes(D);
  constexpr int PART = kva_rows_floats(ROWS, D);  // floats of a piece in scratch: O, then (m, l) a row
  constexpr int PITCH = D + 2;                    // floats of a row in the warps' exchange: O, m, l
  static_assert(DEPTH % SUB == 0 || SUB == 1 || DEPTH > SUB, "a ring holds the steps that are used together");
  extern __shared__ __align__(16) unsigned char kva_smem_raw[];
  __shared__ unsigned s_last;

  const int tid = static_cast<int>(threadIdx.x), lane = tid & 31, warp = tid >> 5;
  const int g = lane >> 2, t = lane & 3;
  if (tid == 0) ptx::grid_dep_launch_dependents();
  ptx::grid_dep_wait();

  // ---- this CTA's share.  Every warp works it out for itself (no barriers): lane i looks at the sequences
  // [i * chunk, (i + 1) * chunk).
  const int heads = p.c.heads;
  auto tiles_of = [&](const KvSeq& s) { return s.n * p.group > p.split_rows ? 0 : (s.n * p.group + ROWS - 1) / ROWS; };
  auto tile_steps = [&](const KvSeq& s, int qt, int& lo, int& hi) {
    int i0 = 0, i1 = s.n;
    if (s.n * p.group > ROWS) {
      i0 = qt * ROWS / p.group;
      i1 = min(s.n, ((qt + 1) * ROWS + p.group - 1) / p.group);
    }
    kv_visible(p, s, i0, i1, lo, hi);
    return kv_steps(lo, hi);
  };
  // A unit's weight: its pieces of at most `share` steps (one piece per CTA), or its steps and what beginning
  // a unit costs besides.
  int share = 0;
  bool one_piece = false;
  auto unit_weight_of = [&](int steps) { return one_piece ? (steps + share - 1) / share : steps + KVA_UNIT_COST; };
  auto seq_weight = [&](const KvSeq& s, int& units) {  // all heads and row tiles
    int sum = 0, lo, hi;
#pragma unroll 1
    for (int qt = tiles_of(s) - 1; qt >= 0; --qt) {
      sum += unit_weight_of(tile_steps(s, qt, lo, hi));
      ++units;
    }
    return sum * heads;
  };
  const int chunk = (p.batch + 31) / 32;
  const int b_first = min(p.batch, lane * chunk), b_last = min(p.batch, b_first + chunk);
  int begin = 0, end = 0, mine = 0, before = 0;
  // first pass: steps; second pass, with few units: pieces
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {
    int units = 0;
    mine = 0;
#pragma unroll 1
    for (int b = b_first; b < b_last; b += 4) {  // the loads of four sequences in flight together
      int row[5], len[4];
#pragma unroll
      for (int u = 0; u < 5; ++u) row[u] = kv_ld(p.cu + min(b + u, p.batch));
#pragma unroll
      for (int u = 0; u < 4; ++u) len[u] = kv_ld(p.kv_len + min(b + u, p.batch - 1));
#pragma unroll 1
      for (int u = 0; u < 4; ++u) {
        if (b + u < b_last)
          mine += seq_weight(kv_seq_of(p, row[0], row[1], len[0], pass == 0 && blockIdx.x == 0 && warp == 0), units);
        row[0] = row[1]; row[1] = row[2]; row[2] = row[3]; row[3] = row[4];
        len[0] = len[1]; len[1] = len[2]; len[2] = len[3];
      }
    }
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += up;
    }
    before = incl - mine;
    const int total = __shfl_sync(0xffffffffu, incl, 31), grid = static_cast<int>(gridDim.x);
    if (pass == 1) {  // one piece per CTA
      begin = static_cast<int>(blockIdx.x);
      end = min(begin + 1, total);
      break;
    }
    if (total == 0) return;
    const int n_units = static_cast<int>(__reduce_add_sync(0xffffffffu, static_cast<unsigned>(units))) * heads;
    one_piece = n_units * 4 <= grid;
    // (few units: their steps without the extra cost, over the CTAs that are not needed for a unit's odd end)
    share = max(p.min_share, one_piece ? (total - n_units * KVA_UNIT_COST - 1) / (grid - n_units) + 1 : (total - 1) / grid + 1);
    if (one_piece) continue;
    begin = static_cast<int>(min(static_cast<long long>(share) * blockIdx.x, static_cast<long long>(total)));
    end = min(begin + share, total);
    break;
  }
  if (begin >= end) return;
  // the sequence that holds it, and where in that
  int b = b_first, in_seq = begin - before;
  const bool here = in_seq >= 0 && in_seq < mine;
  if (here) {
    int units = 0;
#pragma unroll 1
    for (; b + 1 < b_last; ++b) {
      const int w = seq_weight(kv_seq(p, b, false), units);
      if (in_seq < w) break;
      in_seq -= w;
    }
  }
  const int holder = __ffs(__ballot_sync(0xffffffffu, here)) - 1;
  b = __shfl_sync(0xffffffffu, b, holder);
  in_seq = __shfl_sync(0xffffffffu, in_seq, holder);

  unsigned char* const rings = kva_smem_raw + kva_q_bytes(D, NR);
  const uint32_t ring_at = ptx::smem_addr(rings) + static_cast<uint32_t>(warp * DEPTH) * SLOT;
  const uint32_t q_at = ptx::smem_addr(kva_smem_raw) + lane * 16;
  float* const merge = reinterpret_cast<float*>(rings);

  bool first_piece = true;
#pragma unroll 1
  for (int at = begin; at < end; ++b) {
    const KvSeq s = kv_seq(p, b, false);
    const int tiles = tiles_of(s);
#pragma unroll 1
    for (int qt = 0; qt < tiles && at < end; ++qt) {
      int lo, hi;
      const int unit_steps = tile_steps(s, qt, lo, hi);
      // count c of a unit: its c-th piece of per_count steps, or step c - KVA_UNIT_COST of it
      const int unit_weight = unit_weight_of(unit_steps);
      const int per_count = one_piece ? (unit_steps + unit_weight - 1) / unit_weight : 1;
      const int cost = one_piece ? 0 : KVA_UNIT_COST;
      if (in_seq >= unit_weight * heads) {
        in_seq -= unit_weight * heads;
        continue;
      }
      int head = in_seq / unit_weight, c0 = in_seq - head * unit_weight;
      in_seq = 0;
#pragma unroll 1
      for (; head < heads && at < end; ++head, c0 = 0) {
        const int c1 = min(unit_weight, c0 + (end - at));
        const int s0 = max(0, c0 - cost) * per_count, s1 = min(unit_steps, max(0, c1 - cost) * per_count);
        if (cost && s1 == 0) {  // a share that ends inside what beginning the unit costs
          at += c1 - c0;
          continue;
        }
        // ------------------------------------------------ piece: steps [s0, s1) of this unit
        const int row_first = qt * ROWS;  // row = query * group + head in group
        const int rows = min(ROWS, s.n * p.group - row_first);
        const int per = max(0, s1 - s0 + KVA_WARPS - 1) / KVA_WARPS;
        const int w0 = min(s1, s0 + warp * per), w1 = min(s1, w0 + per);

        // ids of 32 pages at a time, one per lane, the next 32 on their way
        const int* const table = p.table + static_cast<long long>(b) * p.table_stride;
        const int last_page = (hi - 1) >> p.c.page_shift;  // (nothing visible: below every page)
        int id_first = (lo + w0 * KVA_STEP) >> p.c.page_shift;
        auto load_ids = [&](int first) { return first + lane <= last_page ? kv_ld(table + first + lane) : -1; };
        // (and the scales of those pages, once their ids are there)
        int ids = load_ids(id_first);
        [[maybe_unused]] float sks = 0.0f, svs = 0.0f, sks_next = 0.0f, svs_next = 0.0f;
        [[maybe_unused]] auto load_scales = [&](int id, float& k, float& v) {
          const bool ok = static_cast<uint32_t>(id) < static_cast<uint32_t>(p.c.num_pages);
          const long long ph = ok ? static_cast<long long>(id) * heads + head : 0;
          k = ok ? ptx::ld_global_f32(p.c.scales[0] + ph) : 0.0f;
          v = ok ? ptx::ld_global_f32(p.c.scales[1] + ph) : 1.0f;
        };

        // q: piece (group of rows, 64 d) i is converted by warp i % KVA_WARPS; its loads go out first
        float krow[NR];
        uint32_t q_bad = 0;  // bit n: row g of group n holds a NaN or an infinity
        uint32_t qx[NR][KC][8];
        {
#pragma unroll
          for (int n = 0; n < NR; ++n) {
            const int r = row_first + 8 * n + g, qi = r / p.group;
            const bool in = 8 * n + g < rows;
            const __half* const src = p.q + (static_cast<long long>(s.row0) + (in ? qi : 0)) * p.q_token_stride +
                                      (static_cast<long long>(head) * p.group + (in ? r - qi * p.group : 0)) * p.q_head_stride +
                                      t * 16;
#pragma unroll
            for (int c = 0; c < KC; ++c)
#pragma unroll
              for (int u = 0; u < 2; ++u) {
#pragma unroll
                for (int w = 0; w < 4; ++w) qx[n][c][4 * u + w] = 0;
                if (in)
                  asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];"
                               : "=r"(qx[n][c][4 * u]), "=r"(qx[n][c][4 * u + 1]), "=r"(qx[n][c][4 * u + 2]),
                                 "=r"(qx[n][c][4 * u + 3])
                               : "l"(src + c * 64 + u * 8) : "memory");
              }
          }
        }
        int ids_next = load_ids(id_first + 32);
        [[maybe_unused]] int s_first = id_first;  // the page of lane 0's scales

        // copies: one step of 16 tokens = rows g, g + 8 of K and rows 2t, 2t+1, 2t+8, 2t+9 of V
        const uint32_t page_bytes = static_cast<uint32_t>(heads) * p.c.page * D;  // of all heads: below 2^31
        const int head_row = head * p.c.page;
        int f_step = w0, f_slot = 0;
        uint32_t f_at = ring_at + lane * 16, f_at8 = ring_at + KP * 512 + lane * 8;  // 16- / 8-byte pieces
        auto fetch = [&]() {
          if (f_step < w1) {
            const int tok = lo + f_step * KVA_STEP;
            const int page = tok >> p.c.page_shift;
            if (page - id_first >= 32) {
              id_first += 32;
              ids = ids_next;
              if constexpr (!SCALES_RING) load_scales(ids, sks_next, svs_next);
              ids_next = load_ids(id_first + 32);
            }
            const uint32_t found = static_cast<uint32_t>(__shfl_sync(0xffffffffu, ids, page - id_first));
            const bool ok = found < static_cast<uint32_t>(p.c.num_pages);
            if (!ok && tok < hi && lane == 0) kv_report(p.status);
            const int bytes = ok ? 16 : 0;
            const uint32_t id = ok ? found : 0;
            const uint64_t off = static_cast<uint64_t>(id) * page_bytes +
                                 static_cast<uint32_t>((head_row + (tok & (p.c.page - 1))) * D);
            const int8_t* const kb = p.c.codes[0] + off + (g * D + t * 16);
            const int8_t* const vb = p.c.codes[1] + off + (2 * t * D + g * (D == 64 ? 8 : 16));
            each<2 * KC>([&](auto i) {
              constexpr int j = i / KC, c = i % KC;
              cp_async<i * 512, 8 * j * D + c * 64, 16>(f_at, kb, bytes);
            });
            each<4 * VP>([&](auto i) {
              constexpr int j = i / VP, c = i % VP, tr = (j & 1) + 8 * (j >> 1);
              if constexpr (D == 64)
                cp_async<j * 256, tr * D, 8>(f_at8, vb, bytes / 2);
              else
                cp_async<KP * 512 + i * 512, tr * D + c * 128, 16>(f_at, vb, bytes);
            });
            if constexpr (SCALES_RING) {
              const uint64_t ph = (static_cast<uint64_t>(id) * static_cast<uint32_t>(heads) + head) * 4;
              cp_async<KVA_STEP * 2 * D - KP * 512, 0, 4>(f_at8, reinterpret_cast<const char*>(p.c.scales[0]) + ph, bytes / 4);
              cp_async<KVA_STEP * 2 * D - KP * 512 + 4, 0, 4>(f_at8, reinterpret_cast<const char*>(p.c.scales[1]) + ph, bytes / 4);
            }
            ++f_step;
            const bool wrap = ++f_slot == DEPTH;
            f_slot = wrap ? 0 : f_slot;
            const uint32_t move = wrap ? static_cast<uint32_t>(-(DEPTH - 1) * SLOT) : SLOT;
            f_at += move;
            f_at8 += move;
          }
          cp_async_commit();
        };
#pragma unroll 1
        for (int d = 0; d < DEPTH; ++d) fetch();
        if constexpr (!SCALES_RING) load_scales(ids, sks, svs);  // (the ring spans fewer than 32 pages: these are still the first ones)

        // q as 254 q1 + q2 times a scale per row, in the d order of K's pieces
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          uint32_t top2 = 0;
#pragma unroll
          for (int c = 0; c < KC; ++c)
#pragma unroll
            for (int w = 0; w < 8; ++w) top2 = __vmaxu2(top2, qx[n][c][w] & 0x7fff7fffu);
          uint32_t top = max(top2 & 0xffffu, top2 >> 16);
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
          const float amax = __half2float(__ushort_as_half(static_cast<unsigned short>(top)));
          const float inv = amax > 0.0f ? __fdividef(127.0f, amax) : 0.0f;
          // (a row with an infinity or a NaN becomes NaN below, if it sees anything)
          q_bad |= top >= 0x7c00u ? 1u << n : 0u;
          krow[n] = p.scale_log2 * (top >= 0x7c00u ? 0.0f : amax * (1.0f / (127.0f * 254.0f)));
#pragma unroll
          for (int c = 0; c < KC; ++c)
            if (warp == (n * KC + c) % KVA_WARPS) {
              uint32_t q1[4], q2[4];
#pragma unroll
              for (int w = 0; w < 4; ++w) {  // word w of a piece of K holds d 4w .. 4w+3
                const float2 e0 = half2_of(qx[n][c][2 * w]), e1 = half2_of(qx[n][c][2 * w + 1]);
                split_q(e0.x * inv, e0.y * inv, e1.x * inv, e1.y * inv, q1[w], q2[w]);
              }
              const uint32_t dst = q_at + (n * KC + c) * 1024;
              ptx::st_shared_v4(dst, q1[0], q1[1], q1[2], q1[3]);
              ptx::st_shared_v4(dst + 512, q2[0], q2[1], q2[2], q2[3]);
            }
        }
        __syncthreads();
        uint32_t qf[Q_REGS ? NR * KC * 2 : 1][4];  // [rows, 64 d, (q1, q2)][word]
        if constexpr (Q_REGS)
          each<NR * KC * 2>([&](auto i) { lds_v4<i * 512>(q_at, qf[i]); });

        // O^T: o[n][i] = d (two per lane, see the exchange below) x rows 2t, 2t + 1 of group n;
        // m and l of row g of group n
        float o[NR][OT][4], mrow[NR], lrow[NR];
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          mrow[n] = -INFINITY;
          lrow[n] = 0.0f;
#pragma unroll
          for (int i = 0; i < OT; ++i)
#pragma unroll
            for (int v = 0; v < 4; ++v) o[n][i][v] = 0.0f;
        }
        // what every row of the tile sees
        const int base_pos = s.len - s.n;
        const int all_hi = base_pos + row_first / p.group;  // last token the first row sees
        const int all_lo = p.window > 0 ? base_pos + (row_first + rows - 1) / p.group - p.window + 1 : 0;

        int c_slot = 0;
#pragma unroll 1
        for (int st = w0; st < w1; st += SUB) {
          cp_async_wait<DEPTH - SUB>();
          // ---- scores: 8 NR rows x 16 SUB tokens, two exact integer sums each; this lane: row g of each
          // group, tokens 8 j + 2t, + 1
          float sc[SUB][NR][2][2], kk[SUB], lsv[SUB], inv_sv[SUB];
          uint32_t at16[SUB], at8[SUB];
          bool masked = false;
          each<SUB>([&](auto sub) {
            at16[sub] = ring_at + static_cast<uint32_t>(c_slot) * SLOT + lane * 16;
            at8[sub] = ring_at + static_cast<uint32_t>(c_slot) * SLOT + KP * 512 + lane * 8;
            c_slot = c_slot + 1 == DEPTH ? 0 : c_slot + 1;
            int sum[NR][2][4];
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
              for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int v = 0; v < 4; ++v) sum[n][j][v] = 0;
            each<KC>([&](auto c) {
              uint32_t kw[2][4];
              lds_v4<c * 512>(at16[sub], kw[0]);
              lds_v4<(KC + c) * 512>(at16[sub], kw[1]);
              each<NR>([&](auto n) {
                constexpr int base = (n * KC + c) * 2;
                uint32_t q1[4], q2[4];
                if constexpr (Q_REGS) {
#pragma unroll
                  for (int w = 0; w < 4; ++w) {
                    q1[w] = qf[base][w];
                    q2[w] = qf[base + 1][w];
                  }
                } else {
                  lds_v4<base * 512>(q_at, q1);
                  lds_v4<base * 512 + 512>(q_at, q2);
                }
#pragma unroll
                for (int w = 0; w < 4; w += 2)
#pragma unroll
                  for (int j = 0; j < 2; ++j)
                    mma_s8_m16n8k32(sum[n][j], q1[w], q2[w], q1[w + 1], q2[w + 1], kw[j][w], kw[j][w + 1]);
              });
            });
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
              for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int v = 0; v < 2; ++v)  // |254 q1 + q2| |k| D <= 32385 * 127 * 256 < 2^31
                  sc[sub][n][j][v] = static_cast<float>(sum[n][j][v] * 254 + sum[n][j][v + 2]);
            const bool dead = st + sub >= w1;  // the odd step out: nothing was fetched for it
            const int tok0 = lo + (st + sub) * KVA_STEP;
            float sv;
            if constexpr (SCALES_RING) {
              uint32_t sk_bits, sv_bits;
              lds_v2<KVA_STEP * 2 * D - KP * 512>(at8[sub], sk_bits, sv_bits);
              kk[sub] = __uint_as_float(sk_bits);
              sv = __uint_as_float(sv_bits);
            } else {
              const int page = tok0 >> p.c.page_shift;
              if (page - s_first >= 32) {  // the copies are ahead of this: the next 32 pages' scales are there
                s_first += 32;
                sks = sks_next;
                svs = svs_next;
              }
              kk[sub] = __shfl_sync(0xffffffffu, sks, page - s_first);
              sv = __shfl_sync(0xffffffffu, svs, page - s_first);
            }
            if (dead) {
              kk[sub] = 0.0f;
              sv = 1.0f;
            }
            // A page whose scale is not finite: NaN for the rows that see it, nothing (-inf below, which such factors
            // would turn into a NaN) for those that do not.
            if (!(fabsf(kk[sub]) < INFINITY && fabsf(sv) < INFINITY)) {
              kk[sub] = sv = 1.0f;
#pragma unroll
              for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int j = 0; j < 2; ++j) sc[sub][n][j][0] = sc[sub][n][j][1] = __int_as_float(0x7fffffff);
            }
            sv = kva_value_scale(sv);
            lsv[sub] = __log2f(sv);
            inv_sv[sub] = __fdividef(1.0f, sv);
            masked |= dead || tok0 + KVA_STEP - 1 > all_hi || tok0 < all_lo;
          });
          if (masked) {
#pragma unroll
            for (int n = 0; n < NR; ++n) {
              const int pos = base_pos + (row_first + 8 * n + g) / p.group;
              const int from = p.window > 0 ? pos - p.window + 1 : 0;
#pragma unroll
              for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                  for (int v = 0; v < 2; ++v) {
                    const int tok = lo + (st + sub) * KVA_STEP + 8 * j + 2 * t + v;
                    if (st + sub >= w1 || tok > pos || tok < from) sc[sub][n][j][v] = -INFINITY;
                  }
            }
          }
          uint32_t pw[SUB][NR][2];
#pragma unroll
          for (int n = 0; n < NR; ++n) {
            float k[SUB], top = -INFINITY;
#pragma unroll
            for (int sub = 0; sub < SUB; ++sub) {
              k[sub] = krow[n] * kk[sub];
              if (k[sub] == 0.0f) k[sub] = 1e-30f;  // (a hidden token's -inf must stay one)
              const float mx = fmaxf(fmaxf(sc[sub][n][0][0], sc[sub][n][0][1]), fmaxf(sc[sub][n][1][0], sc[sub][n][1][1]));
              top = fmaxf(top, fmaf(mx, k[sub], lsv[sub]));
            }
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            if (__any_sync(0xffffffffu, top > mrow[n] + 8.0f)) {
              const float now = fmaxf(mrow[n], top);
              const float f = now == -INFINITY ? 1.0f : exp2_approx(mrow[n] - now);
              mrow[n] = now;
              lrow[n] *= f;
              const float f0 = __shfl_sync(0xffffffffu, f, 8 * t), f1 = __shfl_sync(0xffffffffu, f, 8 * t + 4);
#pragma unroll
              for (int i = 0; i < OT; ++i) {
                o[n][i][0] *= f0;
                o[n][i][1] *= f1;
                o[n][i][2] *= f0;
                o[n][i][3] *= f1;
              }
            }
            const float ref = (mrow[n] == -INFINITY ? 0.0f : mrow[n]) - KVA_WEIGHT_BITS;
#pragma unroll
            for (int sub = 0; sub < SUB; ++sub) {
              const float at_ref = lsv[sub] - ref;
              float e[2][2];
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                e[j][0] = exp2_approx(fmaf(sc[sub][n][j][0], k[sub], at_ref));
                e[j][1] = exp2_approx(fmaf(sc[sub][n][j][1], k[sub], at_ref));
                pw[sub][n][j] = pack_halves(e[j][0], e[j][1]);
              }
              lrow[n] = fmaf((e[0][0] + e[0][1]) + (e[1][0] + e[1][1]), inv_sv[sub], lrow[n]);
            }
          }
          // ---- O^T += V^T w^T
          each<SUB>([&](auto sub) {
            each<VP>([&](auto c) {
              uint32_t vw[4][4];
              each<4>([&](auto j) {
                if constexpr (D == 64)
                  lds_v2<j * 256>(at8[sub], vw[j][0], vw[j][1]);
                else
                  lds_v4<KP * 512 + (j * VP + c) * 512>(at16[sub], vw[j]);
              });
#pragma unroll
              for (int w = 0; w < VW; ++w) {
                uint32_t pair[2][2];  // [tokens 2t,2t+1 / +8,+9][d 0,1 / 2,3 of the word] bytes interleaved by token
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                  const uint32_t a = vw[2 * h][w] ^ 0x80808080u, bb = vw[2 * h + 1][w] ^ 0x80808080u;
                  pair[h][0] = __byte_perm(a, bb, 0x5140);
                  pair[h][1] = __byte_perm(a, bb, 0x7362);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                  const uint32_t a0 = lo_halves(pair[0][i]), a1 = hi_halves(pair[0][i]);
                  const uint32_t a2 = lo_halves(pair[1][i]), a3 = hi_halves(pair[1][i]);
#pragma unroll
                  for (int n = 0; n < NR; ++n)
                    mma_f16_m16n8k16(o[n][(c * VW + w) * 2 + i], a0, a1, a2, a3, pw[sub][n][0], pw[sub][n][1]);
                }
              }
            });
            fetch();
          });
        }
        cp_async_wait<0>();

        // ---- join the warps: [warp][row][O, m, l]
        __syncthreads();  // every warp is done with its ring
        float* const mine_out = merge + warp * ROWS * PITCH;
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          lrow[n] += __shfl_xor_sync(0xffffffffu, lrow[n], 1);
          lrow[n] += __shfl_xor_sync(0xffffffffu, lrow[n], 2);
          if ((q_bad >> n & 1u) && base_pos + (row_first + 8 * n + g) / p.group >= 0) lrow[n] = __int_as_float(0x7fffffff);
          if (t == 0) *reinterpret_cast<float2*>(mine_out + (8 * n + g) * PITCH + D) = make_float2(mrow[n], lrow[n]);
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            if (8 * n + 2 * t + v >= rows) continue;
            float* const dst = mine_out + (8 * n + 2 * t + v) * PITCH + g * (4 * VW);
            // tile i = (c VW + w) 2 + u holds d = 128 c + 4 VW g + 4 w + 2 u and the one behind it
#pragma unroll
            for (int i = 0; i < OT; ++i)
              *reinterpret_cast<float2*>(dst + i / (2 * VW) * 128 + i % (2 * VW) * 2) = make_float2(o[n][i][v], o[n][i][v + 2]);
          }
        }
        __syncthreads();
        const bool whole = s0 == 0 && s1 == unit_steps;
        float* const part = p.partial + (2ll * blockIdx.x + (first_piece ? 0 : 1)) * PART;
        auto out_at = [&](int r) {
          const int row = row_first + r, qi = row / p.group;
          return p.out + (static_cast<long long>(s.row0) + qi) * p.out_token_stride +
                 (static_cast<long long>(head) * p.group + (row - qi * p.group)) * D;
        };
#pragma unroll 1
        for (int idx = tid; idx < rows * (D / 2); idx += KVA_THREADS) {
          const int r = idx / (D / 2), d = idx % (D / 2) * 2;
          const float* const src = merge + r * PITCH;
          float top = -INFINITY, a0 = 0.0f, a1 = 0.0f, l = 0.0f;
#pragma unroll
          for (int w = 0; w < KVA_WARPS; ++w) top = fmaxf(top, src[w * ROWS * PITCH + D]);
          const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll
          for (int w = 0; w < KVA_WARPS; ++w) {
            const float2 ml = *reinterpret_cast<const float2*>(src + w * ROWS * PITCH + D);
            const float2 x = *reinterpret_cast<const float2*>(src + w * ROWS * PITCH + d);
            const float f = exp2_approx(ml.x - ref);
            a0 = fmaf(x.x, f, a0);
            a1 = fmaf(x.y, f, a1);
            l = fmaf(ml.y, f, l);
          }
          if (whole) {
            const float inv = l == 0.0f ? 0.0f : __fdividef(1.0f, l);
            *reinterpret_cast<__half2*>(out_at(r) + d) = __floats2half2_rn(a0 * inv, a1 * inv);
          } else {
            *reinterpret_cast<float2*>(part + r * D + d) = make_float2(a0, a1);
            if (d == 0) *reinterpret_cast<float2*>(part + ROWS * D + 2 * r) = make_float2(top, l);
          }
        }
        if (!whole) {
          // ---- hand over; the last CTA of this unit joins.  Its pieces belong to the CTAs c_first .. c_last,
          // and are the first ones of those except perhaps in c_first.
          int c_first, c_last;
          bool second = false;
          if (one_piece) {
            c_first = static_cast<int>(blockIdx.x) - c0;
            c_last = c_first + unit_weight - 1;
          } else {
            const int u_begin = at - c0;  // of the unit; its first step counts `cost` later
            c_first = (u_begin + cost) / share;
            c_last = (u_begin + unit_weight - 1) / share;
            second = u_begin > share * c_first;
          }
          unsigned* const counter = p.arrived + (static_cast<long long>(b) * p.max_tiles + qt) * heads + head;
          __threadfence();
          __syncthreads();
          if (tid == 0) s_last = atomicAdd(counter, 1u);
          __syncthreads();
          const int pieces = c_last - c_first + 1;
          if (s_last == static_cast<unsigned>(pieces - 1)) {
            __threadfence();
            if (tid == 0) *counter = 0;
            auto piece_at = [&](int c) {
              return p.partial + (2ll * (c_first + c) + (c == 0 && second ? 1 : 0)) * PART;
            };
            // weights of the pieces, JOIN of them at a time: [row][piece], and what their sum of l comes to
            constexpr int JOIN = 128;
            constexpr int ACC = (ROWS * D / 4 + KVA_THREADS - 1) / KVA_THREADS;
            float4 acc[ACC];
#pragma unroll
            for (int a = 0; a < ACC; ++a) acc[a] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            float* const weight = merge;                  // [ROWS][JOIN]
            float* const state = merge + ROWS * JOIN;     // [ROWS][4]: reference, l, factor of what was summed before
#pragma unroll 1
            for (int first = 0; first < pieces; first += JOIN) {
              const int count = min(JOIN, pieces - first);
              __syncthreads();
              for (int r = warp; r < rows; r += KVA_WARPS) {  // a warp per row
                float2 ml[JOIN / 32];
                float top = first ? state[4 * r] : -INFINITY;
                const float was = top;
#pragma unroll
                for (int u = 0; u < JOIN / 32; ++u) {
                  ml[u] = make_float2(-INFINITY, 0.0f);
                  if (lane + 32 * u < count)
                    ml[u] = __ldcg(reinterpret_cast<const float2*>(piece_at(first + lane + 32 * u) + ROWS * D + 2 * r));
                  top = fmaxf(top, ml[u].x);
                }
#pragma unroll
                for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                const float ref = top == -INFINITY ? 0.0f : top;
                float l = 0.0f;
#pragma unroll
                for (int u = 0; u < JOIN / 32; ++u) {
                  const float w = exp2_approx(ml[u].x - ref);
                  weight[r * JOIN + lane + 32 * u] = w;
                  l = fmaf(ml[u].y, w, l);
                }
#pragma unroll
                for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
                if (lane == 0) {
                  const float f = exp2_approx(was - ref);  // 0 the first time
                  state[4 * r + 1] = first ? fmaf(state[4 * r + 1], f, l) : l;
                  state[4 * r] = top;
                  state[4 * r + 2] = f;
                }
              }
              __syncthreads();
#pragma unroll
              for (int a = 0; a < ACC; ++a) {
                const int idx = tid + a * KVA_THREADS;
                const int r = idx / (D / 4), d = idx % (D / 4) * 4;
                if (r >= rows) continue;
                const float f = state[4 * r + 2];
                acc[a].x *= f; acc[a].y *= f; acc[a].z *= f; acc[a].w *= f;
                // (weights beyond the last piece are 0)
                auto add = [&](int c0, auto batch) {
                  float4 x[batch];
#pragma unroll
                  for (int u = 0; u < batch; ++u)
                    x[u] = __ldcg(reinterpret_cast<const float4*>(piece_at(first + min(c0 + u, count - 1)) + r * D + d));
#pragma unroll
                  for (int u = 0; u < batch; ++u) {
                    const float w = weight[r * JOIN + c0 + u];
                    acc[a].x = fmaf(x[u].x, w, acc[a].x);
                    acc[a].y = fmaf(x[u].y, w, acc[a].y);
                    acc[a].z = fmaf(x[u].z, w, acc[a].z);
                    acc[a].w = fmaf(x[u].w, w, acc[a].w);
                  }
                };
                int c0 = 0;
#pragma unroll 1
                for (; count - c0 > 8; c0 += 16) add(c0, Index<16>{});
                if (c0 < count) add(c0, Index<8>{});
              }
            }
#pragma unroll
            for (int a = 0; a < ACC; ++a) {
              const int idx = tid + a * KVA_THREADS;
              const int r = idx / (D / 4), d = idx % (D / 4) * 4;
              if (r >= rows) continue;
              const float l = state[4 * r + 1], inv = l == 0.0f ? 0.0f : __fdividef(1.0f, l);
              __half2* const dst = reinterpret_cast<__half2*>(out_at(r) + d);
              dst[0] = __floats2half2_rn(acc[a].x * inv, acc[a].y * inv);
              dst[1] = __floats2half2_rn(acc[a].z * inv, acc[a].w * inv);
            }
          }
        }
        __syncthreads();  // the results are read: the rings may be filled again
        first_piece = false;
        at += c1 - c0;
      }
    }
  }
}

}  // namespace b200gemm
