// Attention over the 4-bit cache for few query rows per KV head (decoding, verification of a few tokens).
//
// Mathematics.  With a token's scale and offset (sk, ok) of its key, (sv, ov) of its value, codes K, V in 0 .. 15 and weights
// relative to a running reference m,
//     t = c (sk (q . K) + ok sum(q)) + log2 sv,   w = 2^(t - m + 7),   u = w / sv,   l = sum u,
//     O = sum w (V - 8) + sum u (ov + 8 sv),   out = O / l,
// c = softmax_scale log2 e.  Where sv is negative, 15 - V, -sv and ov + 15 sv stand for V, sv and ov.  The value scale is folded into
// the exponent, as in kv_attention.cuh (see there for m, the 2^7 and the bits of a weight), so that one accumulator serves tokens of any
// scale; the offsets are a single sum per row, in FP32.
// w is rounded to binary16 for the product with V; counting codes from the middle of their range halves what that rounding does,
// and keeps the sums small: a mean of many tokens is far below its terms, and the MMA's sums cut off what does not fit.
//
// q . K runs on the integer MMA, q held as 254 q1 + q2 in int8 each (kv_attention.cuh): eight codes of a word are two masks and a
// shift away from the int8 of two registers.  V has to meet fractional weights: a code in the low bits of a binary16 IS one, the
// subnormal c 2^-24, and its left neighbour 16 c 2^-24, so that one fused product each makes them (c - 8) 2^-9: eight registers of V
// fragments take two byte permutes, two shifts, eight masks and eight products.
//
// What bounds it: reading the codes once (D + 8 bytes a token and KV head), and issuing some 400 instructions per 32 tokens
// while they arrive.  As in kv_attention.cuh a warp fetches its own tokens, by cp.async, into a ring nobody else reads; here the
// lanes exchange pieces within the warp, so that every copy is 16 bytes and rows lie such that no load has a bank conflict: the
// row of a token and its 16-byte pieces are permuted by the token's low bits (`row_at`, `piece_at`).
//
// What a token's scale and offset come to (a logarithm, a reciprocal, four conversions) is worked out by one lane each and read
// back by the others through shared memory: eight lanes share a token, and each of them doing it for itself took 5-8 % longer.
//
// Work split, hand-over and joins are those of kv_attention.cuh, with one row tile per sequence.
//
// Measured, back to back (32 heads on 8 KV heads, 128 d): 64 sequences of up to 8192 tokens 74.4 us, 3.9 TB/s of the cache (call by
// call with everything out of L2 77 us); one of 1000 tokens 9.6 us. 16 heads of 64 d, 131071 tokens, 4 queries: 54.0 us, 2.8 TB/s. 0.6 of the issue slots are busy at 128 d; at 64 d, where half the
// codes meet as many scores, exponentials and factors, the instructions per byte are 1.5 times as many. Four CTAs per SM
// with rings of three steps at 128 d: 2 % slower than three with four; steps of 64 tokens at 64 d: -2 to +3 %; the scores' arithmetic by pairs
// of tokens, 7 % fewer instructions: 2 % faster at 64 d, level at 128 d, 9 % slower at 256 d (spills).
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

#include "kv_attention.cuh"
#include "kv_common.cuh"
#include "ptx.cuh"
#include "warp_pieces.cuh"

namespace b200gemm {

struct KvAttn4Params {
  KvCacheU4View c;
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
  float* partial;    // [2 * grid][rows * D + rows * 2]
  unsigned* arrived; // per unit, zero before and after
};

__host__ __device__ constexpr int kva4_step(int dim) { return dim == 256 ? 16 : 32; }  // tokens per step
// What beginning a unit costs a CTA, in steps (see KVA_UNIT_COST).
__host__ __device__ constexpr int kva4_unit_cost(int) { return 8; }  // (6: 1-2 % slower on batches, 16: 2 %)
// Bytes of one ring slot of a warp: a step's codes of K and V, and scales and offsets of both.
__host__ __device__ constexpr int kva4_slot_bytes(int dim) { return kva4_step(dim) * (dim + 8); }
// q fragments, and for each warp five factors of every token of a step.
__host__ __device__ constexpr int kva4_q_bytes(int dim, int nr) { return nr * (dim / 32) * 512 + KVA_WARPS * kva4_step(dim) * 20; }
__host__ __device__ constexpr int kva4_ctas(int dim, int nr) { return dim * nr <= 64 ? 4 : dim * nr <= 256 ? 3 : 2; }
__host__ __device__ constexpr int kva4_smem(int dim, int nr, int depth) {
  const int ring = KVA_WARPS * depth * kva4_slot_bytes(dim);
  const int merge = KVA_WARPS * 8 * nr * (dim + 4) * 4;
  const int join = 8 * nr * (128 + 4) * 4;
  return (ring > merge ? (ring > join ? ring : join) : (merge > join ? merge : join)) + kva4_q_bytes(dim, nr);
}

namespace kva4 {

// Where a token's row lies among the eight of its group, and a 16-byte piece within its row: such that the lanes (g, t) of a warp
// that read piece t of the rows g (K), or part g of the rows 2t or 2t + 1 (V), meet no bank twice.
template <int D>
__device__ __forceinline__ constexpr int row_at(int tok) {
  if (D == 64) return tok ^ (tok >> 2 & 1);
  if (D == 128) return tok ^ (tok >> 1 & 1);
  return tok;
}
template <int D>
__device__ __forceinline__ constexpr int piece_at(int tok, int piece) {
  if (D == 64) return piece;
  if (D == 128) return piece ^ ((tok >> 2 & 1) * 2);
  return piece ^ ((tok >> 1 & 3) * 2) ^ ((tok & 1) * 4);
}
template <int OFF>
__device__ __forceinline__ uint32_t lds(uint32_t at) {
  uint32_t r;
  asm volatile("ld.shared.b32 %0, [%1+%2];" : "=r"(r) : "r"(at), "n"(OFF) : "memory");
  return r;
}
// Codes in the lowest four bits of two binary16, or in the next four: (c - 8) 2^-9.
__device__ __forceinline__ uint32_t low_codes(uint32_t w) {
  uint32_t r;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(w & 0x000f000fu), "r"(0x78007800u), "r"(0xa400a400u));  // 2^15, -2^-6
  return r;
}
__device__ __forceinline__ uint32_t high_codes(uint32_t w) {
  uint32_t r;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(w & 0x00f000f0u), "r"(0x68006800u), "r"(0xa400a400u));  // 2^11, -2^-6
  return r;
}

}  // namespace kva4

template <int D, int NR, int DEPTH>
__global__ void __launch_bounds__(KVA_THREADS, kva4_ctas(D, NR)) kv_attention_u4_kernel(const KvAttn4Params p) {
  using namespace kva;
  using namespace kva4;
  using namespace warp_pieces;
  constexpr int ROWS = 8 * NR;
  constexpr int STEP = kva4_step(D), NT = STEP / 8;  // tokens of a step, groups of eight of them
  constexpr int KW = D / 32;                         // words of K per lane and token
  constexpr int VW = D / 64;                         // words of V per lane and token
  constexpr int OT = D / 16;                         // tiles of 16 d of the result
  constexpr int ROW = D / 2;                         // bytes of a token
  constexpr int SLOT = kva4_slot_bytes(D);
  constexpr int V_AT = STEP * ROW, S_AT = 2 * V_AT;  // in a slot: codes of V; (scale, offset) of K, then of V
  constexpr int COST = kva4_unit_cost(D);
  constexpr int PART = kva_rows_floats(ROWS, D);     // floats of a piece in scratch: O, then (m, l) a row
  constexpr int PITCH = D + 4;                       // floats of a row in the warps' exchange: O, m, l, z
  extern __shared__ __align__(16) unsigned char kva_smem_raw[];
  __shared__ unsigned s_last;

  const int tid = static_cast<int>(threadIdx.x), lane = tid & 31, warp = tid >> 5;
  const int g = lane >> 2, t = lane & 3;
  if (tid == 0) ptx::grid_dep_launch_dependents();
  ptx::grid_dep_wait();

  // ---- this CTA's share.  Every warp works it out for itself (no barriers): lane i looks at the sequences
  // [i * chunk, (i + 1) * chunk).
  const int heads = p.c.heads;
  auto seq_of = [&](int row0, int row1, int kv_len, bool report) {
    KvSeq s;
    s.row0 = row0;
    s.n = row0 < 0 ? 0 : max(0, min(row1 - row0, min(p.max_q, p.rows - row0)));
    s.len = min(max(kv_len, 0), p.max_len);
    if (report && (s.n != row1 - row0 || s.len != kv_len)) kv_report(p.status);
    return s;
  };
  // Steps of a sequence, 0 = it has no row here; [lo, hi): the tokens that its queries see between them, lo rounded down.
  auto steps_of = [&](const KvSeq& s, int& lo, int& hi) {
    if (s.n == 0 || static_cast<long long>(s.n) * p.group > p.split_rows) return 0;
    lo = kv_first_seen(s.len - s.n, p.window) / STEP * STEP;
    hi = max(s.len, lo);
    return max(1, (hi - lo + STEP - 1) / STEP);
  };
  // A unit's weight: its pieces of at most `share` steps (one piece per CTA), or its steps and what beginning
  // a unit costs besides.
  int share = 0;
  bool one_piece = false;
  auto unit_weight_of = [&](int steps) { return steps == 0 ? 0 : one_piece ? (steps + share - 1) / share : steps + COST; };
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
        if (b + u < b_last) {
          int lo, hi;
          const int steps = steps_of(seq_of(row[0], row[1], len[0], pass == 0 && blockIdx.x == 0 && warp == 0), lo, hi);
          units += steps > 0;
          mine += unit_weight_of(steps) * heads;
        }
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
    share = max(p.min_share, one_piece ? (total - n_units * COST - 1) / (grid - n_units) + 1 : (total - 1) / grid + 1);
    if (one_piece) continue;
    begin = static_cast<int>(min(static_cast<long long>(share) * blockIdx.x, static_cast<long long>(total)));
    end = min(begin + share, total);
    break;
  }
  if (begin >= end) return;
  auto seq_at = [&](int b) { return seq_of(kv_ld(p.cu + b), kv_ld(p.cu + b + 1), kv_ld(p.kv_len + b), false); };
  // the sequence that holds it, and where in that
  int b = b_first, in_seq = begin - before;
  const bool here = in_seq >= 0 && in_seq < mine;
  if (here) {
#pragma unroll 1
    for (; b + 1 < b_last; ++b) {
      int lo, hi;
      const int w = unit_weight_of(steps_of(seq_at(b), lo, hi)) * heads;
      if (in_seq < w) break;
      in_seq -= w;
    }
  }
  const int holder = __ffs(__ballot_sync(0xffffffffu, here)) - 1;
  b = __shfl_sync(0xffffffffu, b, holder);
  in_seq = __shfl_sync(0xffffffffu, in_seq, holder);

  unsigned char* const rings = kva_smem_raw + kva4_q_bytes(D, NR);
  const uint32_t ring_at = ptx::smem_addr(rings) + static_cast<uint32_t>(warp * DEPTH) * SLOT;
  const uint32_t q_at = ptx::smem_addr(kva_smem_raw) + lane * 16;
  // [two tokens][sk, sk, ok, ok], [two tokens][log2 sv, log2 sv, 1 / sv, 1 / sv], [token] ov + 8 sv
  const uint32_t f_at_warp = ptx::smem_addr(kva_smem_raw) + NR * KW * 512 + static_cast<uint32_t>(warp * STEP * 20);
  float* const merge = reinterpret_cast<float*>(rings);
  // This lane's places in a slot: of its pieces as they arrive, and of what it reads.  All of them repeat every eight tokens.
  constexpr int PIECES = ROW / 16;              // 16-byte pieces of a token
  constexpr int AT_ONCE = 32 / PIECES;          // tokens that a copy of the warp covers: 16, 8, 4
  const int c_tok = lane / PIECES, c_piece = lane % PIECES;
  uint32_t copy_to[D == 256 ? 2 : 1];           // (at 256 d a copy covers half a group)
#pragma unroll
  for (int i = 0; i < (D == 256 ? 2 : 1); ++i) {
    const int tok = c_tok + 4 * i;
    copy_to[i] = static_cast<uint32_t>((tok & 8) * ROW + row_at<D>(tok & 7) * ROW + piece_at<D>(tok & 7, c_piece) * 16);
  }
  uint32_t k_from[D == 256 ? 2 : 1], v_from[2];
#pragma unroll
  for (int i = 0; i < (D == 256 ? 2 : 1); ++i)
    k_from[i] = static_cast<uint32_t>(row_at<D>(g) * ROW + (D == 64 ? t * 8 : piece_at<D>(g, t + 4 * i) * 16));
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int tok = 2 * t + i;
    v_from[i] = static_cast<uint32_t>(V_AT + row_at<D>(tok) * ROW +
                                      (D == 64 ? g * 4 : D == 128 ? piece_at<D>(tok, g >> 1) * 16 + (g & 1) * 8 : piece_at<D>(tok, g) * 16));
  }

  bool first_piece = true;
#pragma unroll 1
  for (int at = begin; at < end; ++b) {
    const KvSeq s = seq_at(b);
    int lo = 0, hi = 0;
    const int unit_steps = steps_of(s, lo, hi);
    // count c of a unit: its c-th piece of per_count steps, or step c - COST of it
    const int unit_weight = unit_weight_of(unit_steps);
    if (in_seq >= unit_weight * heads) {
      in_seq -= unit_weight * heads;
      continue;
    }
    const int per_count = one_piece ? (unit_steps + unit_weight - 1) / unit_weight : 1;
    const int cost = one_piece ? 0 : COST;
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
      const int rows = min(ROWS, s.n * p.group);  // row = query * group + head in group
      const int per = max(0, s1 - s0 + KVA_WARPS - 1) / KVA_WARPS;
      const int w0 = min(s1, s0 + warp * per), w1 = min(s1, w0 + per);

      // ids of 32 pages at a time, one per lane, the next 32 on their way
      const int* const table = p.table + static_cast<long long>(b) * p.table_stride;
      const int last_page = (hi - 1) >> p.c.page_shift;  // (nothing visible: below every page)
      const int first_page = kv_first_seen(s.len - s.n, p.window) >> p.c.page_shift;
      int id_first = (lo + w0 * STEP) >> p.c.page_shift;
      auto load_ids = [&](int first) {
        return first + lane <= last_page && first + lane >= first_page ? kv_ld(table + first + lane) : -1;
      };
      int ids = load_ids(id_first);

      // q: piece (group of rows, word of K) i is converted by warp i % KVA_WARPS; its loads go out first
      float krow[NR], q_sum[NR];
      uint32_t q_bad = 0;  // bit n: row g of group n holds a NaN or an infinity
      uint32_t qx[NR][KW][4];
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        const int r = 8 * n + g, qi = r / p.group;
        const bool in = r < rows;
        const __half* const src = p.q + (static_cast<long long>(s.row0) + (in ? qi : 0)) * p.q_token_stride +
                                  (static_cast<long long>(head) * p.group + (in ? r - qi * p.group : 0)) * p.q_head_stride;
#pragma unroll
        for (int w = 0; w < KW; ++w) {  // word w holds these eight d
          const int d = D == 256 ? 32 * (t + (w & 4)) + 8 * (w & 3) : (D / 4) * t + 8 * w;
#pragma unroll
          for (int u = 0; u < 4; ++u) qx[n][w][u] = 0;
          if (in)
            asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(qx[n][w][0]), "=r"(qx[n][w][1]), "=r"(qx[n][w][2]), "=r"(qx[n][w][3])
                         : "l"(src + d) : "memory");
        }
      }
      int ids_next = load_ids(id_first + 32);

      // copies of one step, sixteen tokens (of one page) at a time
      int f_step = w0, f_slot = 0;
      uint32_t f_at = ring_at;
      auto fetch = [&]() {
        if (f_step < w1) {
#pragma unroll
          for (int h = 0; h < STEP / 16; ++h) {
            const int tok = lo + f_step * STEP + 16 * h;
            const int page = tok >> p.c.page_shift;
            if (page - id_first >= 32) {
              id_first += 32;
              ids = ids_next;
              ids_next = load_ids(id_first + 32);
            }
            const uint32_t found = static_cast<uint32_t>(__shfl_sync(0xffffffffu, ids, page - id_first));
            const bool ok = found < static_cast<uint32_t>(p.c.num_pages);
            if (!ok && page <= last_page && page >= first_page && lane == 0) kv_report(p.status);
            const int bytes = ok ? 16 : 0;  // (0: zeros)
            const uint64_t token = ok ? (static_cast<uint64_t>(found) * static_cast<uint32_t>(heads) + head) * p.c.page +
                                            static_cast<uint32_t>(tok & (p.c.page - 1))
                                      : 0;
            const uint8_t* const kb = p.c.codes[0] + token * ROW + lane * 16;
            const uint8_t* const vb = p.c.codes[1] + token * ROW + lane * 16;
            const uint32_t to = f_at + static_cast<uint32_t>(h * 16 * ROW);
            each<16 / AT_ONCE>([&](auto i) {
              // i-th copy: tokens AT_ONCE i ...; whole groups of eight lie one behind the other
              constexpr int group = AT_ONCE * i / 8 * 8 * ROW;
              const uint32_t at = to + copy_to[D == 256 ? i % 2 : 0];
              cp_async<group, i * 512, 16>(at, kb, bytes);
              cp_async<V_AT + group, i * 512, 16>(at, vb, bytes);
            });
            // scales and offsets: of K by the lower half of the warp, of V by the upper
            const __half2* const sb = (lane < 16 ? p.c.scales[0] : p.c.scales[1]) + token + (lane & 15);
            const uint32_t st = f_at + static_cast<uint32_t>(S_AT + (lane < 16 ? 0 : STEP * 4) + h * 64 + (lane & 15) * 4);
            cp_async<0, 0, 4>(st, sb, bytes / 4);
          }
          ++f_step;
          const bool wrap = ++f_slot == DEPTH;
          f_slot = wrap ? 0 : f_slot;
          f_at += wrap ? static_cast<uint32_t>(-(DEPTH - 1) * SLOT) : SLOT;
        }
        cp_async_commit();
      };
#pragma unroll 1
      for (int d = 0; d < DEPTH - 1; ++d) fetch();

      // q as 254 q1 + q2 times a scale per row: even d of a word, then odd ones
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        uint32_t top2 = 0;
#pragma unroll
        for (int w = 0; w < KW; ++w)
#pragma unroll
          for (int u = 0; u < 4; ++u) top2 = __vmaxu2(top2, qx[n][w][u] & 0x7fff7fffu);
        uint32_t top = max(top2 & 0xffffu, top2 >> 16);
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const float amax = __half2float(__ushort_as_half(static_cast<unsigned short>(top)));
        const float inv = amax > 0.0f ? __fdividef(127.0f, amax) : 0.0f;
        // (a row with an infinity or a NaN becomes NaN below, if it sees anything)
        q_bad |= top >= 0x7c00u ? 1u << n : 0u;
        krow[n] = p.scale_log2 * (top >= 0x7c00u ? 0.0f : amax * (1.0f / (127.0f * 254.0f)));
#pragma unroll
        for (int w = 0; w < KW; ++w)
          if (warp == (n * KW + w) % KVA_WARPS) {
            float2 e[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) e[u] = half2_of(qx[n][w][u]);
            uint32_t a0, a1, a2, a3;
            split_q(e[0].x * inv, e[1].x * inv, e[2].x * inv, e[3].x * inv, a0, a1);
            split_q(e[0].y * inv, e[1].y * inv, e[2].y * inv, e[3].y * inv, a2, a3);
            ptx::st_shared_v4(q_at + (n * KW + w) * 512, a0, a1, a2, a3);
          }
      }
      __syncthreads();
      uint32_t qf[NR][KW][4];
      each<NR * KW>([&](auto i) { lds_v4<i * 512>(q_at, qf[i / KW][i % KW]); });
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        int hi_sum = 0, lo_sum = 0;
#pragma unroll
        for (int w = 0; w < KW; ++w) {
          hi_sum = __dp4a(static_cast<int>(qf[n][w][0]), 0x01010101, __dp4a(static_cast<int>(qf[n][w][2]), 0x01010101, hi_sum));
          lo_sum = __dp4a(static_cast<int>(qf[n][w][1]), 0x01010101, __dp4a(static_cast<int>(qf[n][w][3]), 0x01010101, lo_sum));
        }
        int sum = hi_sum * 254 + lo_sum;
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        q_sum[n] = static_cast<float>(sum);
      }

      // O^T: o[n][i] = d (two per lane, see the exchange below) x rows 2t, 2t + 1 of group n; m, l and z (what the
      // offsets add) of row g of group n
      float o[NR][OT][4], mrow[NR], lrow[NR], zrow[NR];
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        mrow[n] = -INFINITY;
        lrow[n] = zrow[n] = 0.0f;
#pragma unroll
        for (int i = 0; i < OT; ++i)
#pragma unroll
          for (int v = 0; v < 4; ++v) o[n][i][v] = 0.0f;
      }
      // what every row of the tile sees
      const int base_pos = s.len - s.n;
      const int all_hi = base_pos;  // last token the first row sees
      const int all_lo = p.window > 0 ? base_pos + (rows - 1) / p.group - p.window + 1 : 0;

      uint32_t c_at = ring_at;
      int c_slot = 0;
#pragma unroll 1
      for (int st = w0; st < w1; ++st) {
        cp_async_wait<DEPTH - 2>();
        __syncwarp();  // (the lanes read one another's pieces; and have read those that the next copies replace)
        const uint32_t slot = c_at;
        const bool wrap = ++c_slot == DEPTH;
        c_slot = wrap ? 0 : c_slot;
        c_at += wrap ? static_cast<uint32_t>(-(DEPTH - 1) * SLOT) : SLOT;
        fetch();
        // ---- the tokens' factors, a lane for each.  A token whose scale or offset is not finite: NaN for the rows that see it, nothing
        // (-inf below, which such factors would turn into a NaN) for those that do not.
        bool down = false;  // the lane's token counts from its maximum
        each<(STEP + 31) / 32>([&](auto part) {
          if (STEP < 32 && lane >= STEP) return;
          const uint32_t k_word = kva4::lds<S_AT + part * 128>(slot + lane * 4), v_word = kva4::lds<S_AT + STEP * 4 + part * 128>(slot + lane * 4);
          auto finite = [](uint32_t w) { return (w & 0x7c00u) != 0x7c00u && (w & 0x7c000000u) != 0x7c000000u; };
          const bool good = finite(k_word) && finite(v_word);
          const float2 k = half2_of(k_word), x = half2_of(good ? v_word : 0x00003c00u);
          const float sv = kva_value_scale(fabsf(x.x));
          down = x.x < 0.0f;
          const uint32_t to = f_at_warp + part * 256 + (lane >> 1) * 16 + (lane & 1) * 4;
          auto put = [](uint32_t at, float v) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(v) : "memory"); };
          put(to, good ? k.x : __int_as_float(0x7fffffff));
          put(to + 8, good ? k.y : 0.0f);
          put(to + STEP * 8, __log2f(sv));
          put(to + STEP * 8 + 8, __fdividef(1.0f, sv));
          put(f_at_warp + STEP * 16 + part * 128 + lane * 4, fmaf(x.x < 0.0f ? 7.0f : 8.0f, x.x, x.y));
        });
        // ---- scores: 8 NR rows x STEP tokens, two exact integer sums each; this lane: row g of each
        // group, tokens 8 j + 2t, + 1
        float sc[NR][NT][2];
        each<NT>([&](auto j) {
          uint32_t kw[KW];
          if constexpr (D == 64) {
            lds_v2<j * 8 * ROW>(slot + k_from[0], kw[0], kw[1]);
          } else {
            each<KW / 4>([&](auto i) {
              uint32_t x[4];
              lds_v4<j * 8 * ROW>(slot + k_from[i], x);
#pragma unroll
              for (int u = 0; u < 4; ++u) kw[4 * i + u] = x[u];
            });
          }
          int sum[NR][4];
#pragma unroll
          for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int v = 0; v < 4; ++v) sum[n][v] = 0;
#pragma unroll
          for (int w = 0; w < KW; ++w) {
            const uint32_t even = kw[w] & 0x0f0f0f0fu, odd = (kw[w] >> 4) & 0x0f0f0f0fu;
#pragma unroll
            for (int n = 0; n < NR; ++n) mma_s8_m16n8k32(sum[n], qf[n][w][0], qf[n][w][1], qf[n][w][2], qf[n][w][3], even, odd);
          }
#pragma unroll
          for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int v = 0; v < 2; ++v)  // |254 q1 + q2| 15 D <= 32385 * 15 * 256 < 2^31
              sc[n][j][v] = static_cast<float>(sum[n][v] * 254 + sum[n][v + 2]);
        });
        if (__any_sync(0xffffffffu, down)) {  // (few caches have such tokens)
          if (down) {
            const uint32_t row = slot + V_AT + static_cast<uint32_t>((lane >> 3) * 8 * ROW + row_at<D>(lane & 7) * ROW);
#pragma unroll 1
            for (int i = 0; i < ROW; i += 16) {
              uint32_t w[4];
              ptx::ld_shared_v4(row + i, w[0], w[1], w[2], w[3]);
              ptx::st_shared_v4(row + i, ~w[0], ~w[1], ~w[2], ~w[3]);
            }
          }
        }
        __syncwarp();
        const int tok0 = lo + st * STEP;
        const uint32_t factors = f_at_warp + t * 16;
        float inv_sv[NT][2];
        each<NT>([&](auto j) {
          uint32_t k[4], v[4];
          lds_v4<j * 64>(factors, k);
          lds_v4<STEP * 8 + j * 64>(factors, v);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            inv_sv[j][i] = __uint_as_float(v[2 + i]);
#pragma unroll
            for (int n = 0; n < NR; ++n)
              sc[n][j][i] = fmaf(fmaf(__uint_as_float(k[2 + i]), q_sum[n], __uint_as_float(k[i]) * sc[n][j][i]), krow[n], __uint_as_float(v[i]));
          }
        });
        if (tok0 + STEP - 1 > all_hi || tok0 < all_lo) {
#pragma unroll
          for (int n = 0; n < NR; ++n) {
            const int pos = base_pos + (8 * n + g) / p.group;
            const int from = p.window > 0 ? pos - p.window + 1 : 0;
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
              for (int v = 0; v < 2; ++v) {
                const int tok = tok0 + 8 * j + 2 * t + v;
                if (tok > pos || tok < from) sc[n][j][v] = -INFINITY;
              }
          }
        }
        uint32_t pw[NR][NT];
        float mid[NT][2];
        each<NT>([&](auto j) {
          uint32_t a, b;
          lds_v2<STEP * 16 + j * 32>(f_at_warp + t * 8, a, b);
          mid[j][0] = __uint_as_float(a);
          mid[j][1] = __uint_as_float(b);
        });
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          float top = fmaxf(sc[n][0][0], sc[n][0][1]);
#pragma unroll
          for (int j = 1; j < NT; ++j) top = fmaxf(top, fmaxf(sc[n][j][0], sc[n][j][1]));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
          if (__any_sync(0xffffffffu, top > mrow[n] + 8.0f)) {
            const float now = fmaxf(mrow[n], top);
            const float f = now == -INFINITY ? 1.0f : exp2_approx(mrow[n] - now);
            mrow[n] = now;
            lrow[n] *= f;
            zrow[n] *= f;
            const float f0 = __shfl_sync(0xffffffffu, f, 8 * t), f1 = __shfl_sync(0xffffffffu, f, 8 * t + 4);
#pragma unroll
            for (int i = 0; i < OT; ++i) {
              o[n][i][0] *= f0;
              o[n][i][1] *= f1;
              o[n][i][2] *= f0;
              o[n][i][3] *= f1;
            }
          }
          const float at_ref = KVA_WEIGHT_BITS - (mrow[n] == -INFINITY ? 0.0f : mrow[n]);
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            const float e0 = exp2_approx(sc[n][j][0] + at_ref), e1 = exp2_approx(sc[n][j][1] + at_ref);
            pw[n][j] = pack_halves(e0, e1);
            const float u0 = e0 * inv_sv[j][0], u1 = e1 * inv_sv[j][1];
            lrow[n] += u0 + u1;
            zrow[n] = fmaf(u0, mid[j][0], fmaf(u1, mid[j][1], zrow[n]));
          }
        }
        // ---- O^T += V^T w^T, sixteen tokens at a time
        each<NT / 2>([&](auto h) {
          uint32_t vw[4][VW];  // words of tokens 2t, 2t + 1, 2t + 8, 2t + 9
          each<4>([&](auto i) {
            constexpr int off = (h * 16 + (i >> 1) * 8) * ROW;
            const uint32_t from = slot + v_from[i & 1];
            if constexpr (D == 64) {
              vw[i][0] = kva4::lds<off>(from);
            } else if constexpr (D == 128) {
              lds_v2<off>(from, vw[i][0], vw[i][1]);
            } else {
              lds_v4<off>(from, vw[i]);
            }
          });
#pragma unroll
          for (int w = 0; w < VW; ++w) {
            // codes of two tokens side by side, eight bits of each in a half: [tokens 2t / 2t + 8][d 0-3 / 4-7]
            uint32_t x[2][2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              x[i][0] = __byte_perm(vw[2 * i][w], vw[2 * i + 1][w], 0x5410);
              x[i][1] = __byte_perm(vw[2 * i][w], vw[2 * i + 1][w], 0x7632);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {  // d 2u and 2u + 1 of the word
              const uint32_t a = u & 1 ? x[0][u >> 1] >> 8 : x[0][u >> 1], bb = u & 1 ? x[1][u >> 1] >> 8 : x[1][u >> 1];
              const uint32_t a0 = low_codes(a), a1 = high_codes(a), a2 = low_codes(bb), a3 = high_codes(bb);
#pragma unroll
              for (int n = 0; n < NR; ++n) mma_f16_m16n8k16(o[n][4 * w + u], a0, a1, a2, a3, pw[n][2 * h], pw[n][2 * h + 1]);
            }
          }
        });
      }
      cp_async_wait<0>();

      // ---- join the warps: [warp][row][O, m, l, z]
      __syncthreads();  // every warp is done with its ring
      float* const mine_out = merge + warp * ROWS * PITCH;
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        lrow[n] += __shfl_xor_sync(0xffffffffu, lrow[n], 1);
        lrow[n] += __shfl_xor_sync(0xffffffffu, lrow[n], 2);
        zrow[n] += __shfl_xor_sync(0xffffffffu, zrow[n], 1);
        zrow[n] += __shfl_xor_sync(0xffffffffu, zrow[n], 2);
        if ((q_bad >> n & 1u) && base_pos + (8 * n + g) / p.group >= 0) lrow[n] = __int_as_float(0x7fffffff);
        if (t == 0) {
          *reinterpret_cast<float2*>(mine_out + (8 * n + g) * PITCH + D) = make_float2(mrow[n], lrow[n]);
          mine_out[(8 * n + g) * PITCH + D + 2] = zrow[n];
        }
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          if (8 * n + 2 * t + v >= rows) continue;
          float* const dst = mine_out + (8 * n + 2 * t + v) * PITCH + g * (D / 8);
          // tile i holds d = g D / 8 + 2 i and the one behind it
#pragma unroll
          for (int i = 0; i < OT; ++i)
            *reinterpret_cast<float2*>(dst + 2 * i) = make_float2(o[n][i][v] * 512.0f, o[n][i][v + 2] * 512.0f);
        }
      }
      __syncthreads();
      const bool whole = s0 == 0 && s1 == unit_steps;
      float* const part = p.partial + (2ll * blockIdx.x + (first_piece ? 0 : 1)) * PART;
      auto out_at = [&](int r) {
        const int qi = r / p.group;
        return p.out + (static_cast<long long>(s.row0) + qi) * p.out_token_stride +
               (static_cast<long long>(head) * p.group + (r - qi * p.group)) * D;
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
          const float4 mlz = *reinterpret_cast<const float4*>(src + w * ROWS * PITCH + D);
          const float2 x = *reinterpret_cast<const float2*>(src + w * ROWS * PITCH + d);
          const float f = exp2_approx(mlz.x - ref);
          a0 = fmaf(x.x + mlz.z, f, a0);
          a1 = fmaf(x.y + mlz.z, f, a1);
          l = fmaf(mlz.y, f, l);
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
        unsigned* const counter = p.arrived + static_cast<long long>(b) * heads + head;
        __threadfence();
        __syncthreads();
        if (tid == 0) s_last = atomicAdd(counter, 1u);
        __syncthreads();
        const int pieces = c_last - c_first + 1;
        if (s_last == static_cast<unsigned>(pieces - 1)) {
          __threadfence();
          if (tid == 0) *counter = 0;
          auto piece_of = [&](int c) {
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
                  ml[u] = __ldcg(reinterpret_cast<const float2*>(piece_of(first + lane + 32 * u) + ROWS * D + 2 * r));
                top = fmaxf(top, ml[u].x);
              }
#pragma unroll
              for (int x = 16; x; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
              const float ref = top == -INFINITY ? 0.0f : top;
              float l = 0.0f;
#pragma unroll
              for (int u = 0; u < JOIN / 32; ++u) {
                const float w = exp2_approx(ml[u].x - ref);
                weight[r * JOIN + lane + 32 * u] = w;
                l = fmaf(ml[u].y, w, l);
              }
#pragma unroll
              for (int x = 16; x; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
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
              auto add = [&](int from, auto batch) {
                float4 x[batch];
#pragma unroll
                for (int u = 0; u < batch; ++u)
                  x[u] = __ldcg(reinterpret_cast<const float4*>(piece_of(first + min(from + u, count - 1)) + r * D + d));
#pragma unroll
                for (int u = 0; u < batch; ++u) {
                  const float w = weight[r * JOIN + from + u];
                  acc[a].x = fmaf(x[u].x, w, acc[a].x);
                  acc[a].y = fmaf(x[u].y, w, acc[a].y);
                  acc[a].z = fmaf(x[u].z, w, acc[a].z);
                  acc[a].w = fmaf(x[u].w, w, acc[a].w);
                }
              };
              int from = 0;
#pragma unroll 1
              for (; count - from > 8; from += 16) add(from, Index<16>{});
              if (from < count) add(from, Index<8>{});
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

}  // namespace b200gemm
