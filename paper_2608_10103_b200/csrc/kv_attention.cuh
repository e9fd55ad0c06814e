// Attention over the INT8 cache for few query rows per KV head (decoding, verification of a few
// tokens), and the general path for everything else.
//
// Mathematics.  The rows that share a KV head (queries x heads of its group) form one tile of
// 16 MT rows, so the cache is read once for all of them.  With page scales sk, sv, codes K, V and
// weights relative to a running reference m,
//     t = c sk (q . K) + log2 sv,   w = 2^(t - m),   O = sum w V,   l = sum w / sv,   out = O / l,
// c = softmax_scale log2 e: the value scale is folded into the exponent, so that O needs one
// accumulator whatever the pages' scales are, w <= 1 whichever page dominates, and the softmax
// denominator takes it out again.  m, l, O and the scores are FP32; w is rounded to binary16 for the
// product with V (relative 2^-11 a weight, the rounding of the result itself).  Codes are exact in
// binary16.
//
// What bounds it: reading the codes once (2 D bytes a token and KV head).  So, as in few_rows.cuh, a
// thread fetches exactly the pieces its own fragments of mma.sync m16n8k16 need, by cp.async into a
// ring nobody else reads: no barrier, no bank conflict, and `depth` steps of 16 tokens in flight per
// warp.  The positions the instruction gives a thread are filled with whatever 16 bytes are contiguous: K's
// d order is permuted (Q is loaded in the same order), V's d order is permuted over the columns of the
// result.  An int8 code becomes binary16 by placing code ^ 0x80 under the exponent of 1024
// (prmt) and subtracting 1152 -- five instructions for four codes.
//
// Work split: the (sequence, row tile, head) units, laid end to end in steps of 16 tokens, are cut
// into equal contiguous shares, one per CTA, whatever the lengths are.  A CTA's warps share each
// piece; a piece that is not a whole unit leaves its m, l, O in scratch, and the CTA that finishes a
// unit last joins its pieces in their order (no second launch, and no dependence on who was last).
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

struct KvAttnParams {
  KvCacheView c;
  int batch;
  const int* cu;
  const int* kv_len;
  const int* table;
  int table_stride;
  int max_q;
  int group;  // query heads per KV head
  const __half* q;
  long long q_token_stride, q_head_stride;
  __half* out;
  long long out_token_stride;
  float scale_log2;  // softmax_scale * log2(e)
  int window;        // 0 = all
  int* status;
  int min_share;     // steps per CTA at least
  int depth;
  float* partial;    // [2 * grid][rows * (D + 2)]
  unsigned* arrived; // per unit, zero before and after
};

// A sequence's share of the work.
struct KvSeq {
  int row0, n, len;
};
__device__ __forceinline__ KvSeq kv_seq(const KvAttnParams& p, int b, bool report) {
  KvSeq s;
  s.row0 = kv_ld(p.cu + b);
  s.n = kv_ld(p.cu + b + 1) - s.row0;
  s.len = kv_ld(p.kv_len + b);
  const long long room = static_cast<long long>(p.table_stride) * p.c.page;
  bool bad = s.n < 0 || s.n > p.max_q || s.len < 0 || s.len > room || s.row0 < 0;
  if (s.row0 < 0 || s.n < 0) s.n = 0;
  if (s.n > p.max_q) s.n = p.max_q;
  if (s.len < 0) s.len = 0;
  if (s.len > room) s.len = static_cast<int>(room);
  if (bad && report) kv_report(p.status);
  return s;
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

__device__ __forceinline__ void cp_async_8(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_4(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
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
__device__ __forceinline__ uint32_t pack_halves(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

}  // namespace kva

// Bytes of one ring slot of a warp: 16 tokens of K and V, and each lane's copy of both scales.
__host__ __device__ constexpr int kva_slot_bytes(int dim) { return KVA_STEP * 2 * dim + 256; }
__host__ __device__ constexpr int kva_rows_floats(int rows, int dim) { return rows * (dim + 2); }
// Dynamic shared memory: the rings, reused for the warps' results; Q fragments where they are kept there.
__host__ __device__ constexpr bool kva_q_in_regs(int dim, int mt) { return dim * mt <= 128; }
__host__ __device__ constexpr int kva_q_bytes(int dim, int mt) {
  return kva_q_in_regs(dim, mt) ? 0 : mt * (dim / 16) * 512;
}
__host__ __device__ constexpr int kva_smem(int dim, int mt, int depth) {
  const int ring = KVA_WARPS * depth * kva_slot_bytes(dim);
  const int merge = KVA_WARPS * kva_rows_floats(16 * mt, dim) * 4;
  return (ring > merge ? ring : merge) + kva_q_bytes(dim, mt);
}

// CTAs an SM is meant to hold: what the rings leave room for.
__host__ __device__ constexpr int kva_ctas(int dim, int mt) { return mt * dim >= 256 ? 2 : mt * dim == 128 ? 3 : 4; }

template <int D, int MT>
__global__ void __launch_bounds__(KVA_THREADS, kva_ctas(D, MT)) kv_attention_kernel(const KvAttnParams p) {
  using namespace kva;
  using namespace warp_pieces;
  constexpr int ROWS = 16 * MT;
  constexpr int KP = 2 * (D / 64);                // 16-byte pieces of K per thread and step
  constexpr int VP = D >= 128 ? D / 128 : 1;      // pieces of V per token (8 bytes for D = 64)
  constexpr int NT = D / 8;                       // column tiles of the result
  constexpr int KS = D / 16;                      // MMA steps over d
  constexpr bool Q_REGS = kva_q_in_regs(D, MT);
  constexpr int SLOT = kva_slot_bytes(D);
  extern __shared__ __align__(16) unsigned char kva_smem_raw[];
  __shared__ long long s_scan[KVA_WARPS + 1];
  __shared__ int s_find[2];
  __shared__ long long s_before;
  __shared__ unsigned s_last;

  const int tid = static_cast<int>(threadIdx.x), lane = tid & 31, warp = tid >> 5;
  const int g = lane >> 2, t = lane & 3;
  if (tid == 0) ptx::grid_dep_launch_dependents();
  ptx::grid_dep_wait();

  // ---- this CTA's share: steps [begin, end) of all units laid end to end
  const int heads = p.c.heads;
  auto tiles_of = [&](const KvSeq& s) { return static_cast<int>((static_cast<long long>(s.n) * p.group + ROWS - 1) / ROWS); };
  auto tile_steps = [&](const KvSeq& s, int qt, int& lo, int& hi) {
    const int i0 = static_cast<int>(static_cast<long long>(qt) * ROWS / p.group);
    const int i1 = min(s.n, static_cast<int>((static_cast<long long>(qt + 1) * ROWS + p.group - 1) / p.group));
    kv_visible(p, s, i0, i1, lo, hi);
    return kv_steps(lo, hi);
  };
  auto seq_steps = [&](int b, bool report) {  // all heads and row tiles of a sequence
    const KvSeq s = kv_seq(p, b, report);
    const int tiles = tiles_of(s);
    long long sum = 0;
    for (int qt = 0; qt < tiles; ++qt) {
      int lo, hi;
      sum += tile_steps(s, qt, lo, hi);
    }
    return sum * heads;
  };
  long long total = 0;
  for (int b = tid; b < p.batch; b += KVA_THREADS) total += seq_steps(b, blockIdx.x == 0);
  for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  if (lane == 0) s_scan[warp] = total;
  __syncthreads();
  total = 0;
  for (int w = 0; w < KVA_WARPS; ++w) total += s_scan[w];
  long long share = (total + gridDim.x - 1) / gridDim.x;
  if (share < p.min_share) share = p.min_share;
  const long long begin = share * blockIdx.x;
  const long long end = begin + share < total ? begin + share : total;
  if (begin >= end) return;
  // the sequence that holds step `begin`
  long long seen = 0;
  int b = 0;
  long long in_seq = 0;  // step within that sequence
  for (int base = 0;; base += KVA_THREADS) {
    const int mine = base + tid;
    const long long steps = mine < p.batch ? seq_steps(mine, false) : 0;
    long long incl = steps;
    for (int o = 1; o < 32; o <<= 1) {
      const long long up = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += up;
    }
    __syncthreads();
    if (lane == 31) s_scan[warp] = incl;
    if (tid == 0) s_find[0] = -1;
    __syncthreads();
    long long before = seen;
    for (int w = 0; w < warp; ++w) before += s_scan[w];
    incl += before;
    if (begin >= incl - steps && begin < incl) {
      s_find[0] = mine;
      s_before = incl - steps;
    }
    for (int w = 0; w < KVA_WARPS; ++w) seen += s_scan[w];
    __syncthreads();
    if (s_find[0] >= 0) {
      b = s_find[0];
      in_seq = begin - s_before;
      break;
    }
    if (base + KVA_THREADS >= p.batch) return;  // (cannot happen: begin < total)
  }

  unsigned char* const ring = kva_smem_raw + kva_q_bytes(D, MT) + warp * p.depth * SLOT;
  const uint32_t ring_at = ptx::smem_addr(ring);
  const uint32_t q_at = ptx::smem_addr(kva_smem_raw) + lane * 16;
  float* const merge = reinterpret_cast<float*>(kva_smem_raw + kva_q_bytes(D, MT));

  long long at = begin;
  bool first_piece = true;
#pragma unroll 1
  for (; at < end; ++b, in_seq = 0) {
    const KvSeq s = kv_seq(p, b, false);
    const int tiles = tiles_of(s);
#pragma unroll 1
    for (int qt = 0; qt < tiles && at < end; ++qt) {
      int lo, hi;
      const int unit_steps = tile_steps(s, qt, lo, hi);
      const long long tile_total = static_cast<long long>(unit_steps) * heads;
      if (in_seq >= tile_total) {
        in_seq -= tile_total;
        continue;
      }
      int head = static_cast<int>(in_seq / unit_steps);
      int s0 = static_cast<int>(in_seq - static_cast<long long>(head) * unit_steps);
      in_seq = 0;
#pragma unroll 1
      for (; head < heads && at < end; ++head, s0 = 0) {
        const long long left = end - at;
        const int s1 = left < unit_steps - s0 ? s0 + static_cast<int>(left) : unit_steps;
        // ------------------------------------------------ piece: steps [s0, s1) of this unit
        const int row_first = qt * ROWS;  // row = query * group + head in group
        const int rows = min(ROWS, s.n * p.group - row_first);
        const int per = (s1 - s0 + KVA_WARPS - 1) / KVA_WARPS;
        const int w0 = min(s1, s0 + warp * per), w1 = min(s1, w0 + per);

        // copies: one step of 16 tokens = rows g, g + 8 of K and rows 2t, 2t+1, 2t+8, 2t+9 of V
        const int* const table = p.table + static_cast<long long>(b) * p.table_stride;
        int f_step = w0, f_slot = 0;
        int f_page = -1, f_id = 0;
        auto fetch = [&]() {
          if (f_step < w1) {
            const int tok = lo + f_step * KVA_STEP;
            const int page = tok >> p.c.page_shift;
            if (page != f_page && tok < hi) {
              f_page = page;
              f_id = kv_ld(table + page);
              if (f_id < 0 || f_id >= p.c.num_pages) {
                if (lane == 0) kv_report(p.status);
                f_id = -1;
              }
            }
            const bool ok = tok < hi && f_id >= 0;
            const long long ph = ok ? static_cast<long long>(f_id) * heads + head : 0;
            const long long row = ph * p.c.page + (tok & (p.c.page - 1));
            const uint32_t slot = ring_at + static_cast<uint32_t>(f_slot) * SLOT;
            const int bytes = ok ? 16 : 0;
            const uint8_t* const kb = reinterpret_cast<const uint8_t*>(p.c.codes[0]) + row * D;
            const uint8_t* const vb = reinterpret_cast<const uint8_t*>(p.c.codes[1]) + row * D;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int c = 0; c < D / 64; ++c)
                cp_async_16_cg(slot + (j * (D / 64) + c) * 512 + lane * 16,
                               kb + (g + 8 * j) * D + c * 64 + t * 16, bytes);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int tr = 2 * t + (j & 1) + 8 * (j >> 1);
              if constexpr (D == 64) {
                cp_async_8(slot + KP * 512 + j * 256 + lane * 8, vb + tr * D + g * 8, ok ? 8 : 0);
              } else {
#pragma unroll
                for (int c = 0; c < VP; ++c)
                  cp_async_16_cg(slot + KP * 512 + (j * VP + c) * 512 + lane * 16,
                                 vb + tr * D + c * 128 + g * 16, bytes);
              }
            }
            cp_async_4(slot + KVA_STEP * 2 * D + lane * 8, p.c.scales[0] + ph, ok ? 4 : 0);
            cp_async_4(slot + KVA_STEP * 2 * D + lane * 8 + 4, p.c.scales[1] + ph, ok ? 4 : 0);
            ++f_step;
            f_slot = f_slot + 1 == p.depth ? 0 : f_slot + 1;
          }
          cp_async_commit();
        };
#pragma unroll 1
        for (int d = 0; d < p.depth; ++d) fetch();

        // Q fragments, in the d order of K's pieces; rows beyond the tile read nothing
        uint32_t qf[Q_REGS ? MT * KS * 4 : 4];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
#pragma unroll
          for (int c = 0; c < D / 64; ++c) {
            uint4 x[2][2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int r = row_first + 16 * m + 8 * h + g;
              const int qi = r / p.group;
              x[h][0] = x[h][1] = make_uint4(0, 0, 0, 0);
              if (r - row_first < rows) {
                const __half* src = p.q + (static_cast<long long>(s.row0) + qi) * p.q_token_stride +
                                    (static_cast<long long>(head) * p.group + (r - qi * p.group)) * p.q_head_stride +
                                    c * 64 + t * 16;
                asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(x[h][0].x), "=r"(x[h][0].y), "=r"(x[h][0].z), "=r"(x[h][0].w)
                             : "l"(src) : "memory");
                asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(x[h][1].x), "=r"(x[h][1].y), "=r"(x[h][1].z), "=r"(x[h][1].w)
                             : "l"(src + 8) : "memory");
              }
            }
#pragma unroll
            for (int w = 0; w < 4; ++w) {  // 16 halves = 8 words: word w of K holds d 4w .. 4w+3
              const uint32_t a0 = word_of(x[0][w >> 1], 2 * (w & 1)), a2 = word_of(x[0][w >> 1], 2 * (w & 1) + 1);
              const uint32_t a1 = word_of(x[1][w >> 1], 2 * (w & 1)), a3 = word_of(x[1][w >> 1], 2 * (w & 1) + 1);
              const int ks = m * KS + c * 4 + w;
              if constexpr (Q_REGS) {
                qf[4 * ks] = a0; qf[4 * ks + 1] = a1; qf[4 * ks + 2] = a2; qf[4 * ks + 3] = a3;
              } else {
                if (warp == 0) ptx::st_shared_v4(q_at + ks * 512, a0, a1, a2, a3);
              }
            }
          }
        }
        if constexpr (!Q_REGS) __syncthreads();

        float o[MT][NT][4], mrow[MT][2], lrow[MT][2];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          mrow[m][0] = mrow[m][1] = -INFINITY;
          lrow[m][0] = lrow[m][1] = 0.0f;
#pragma unroll
          for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int v = 0; v < 4; ++v) o[m][i][v] = 0.0f;
        }
        // positions of this thread's rows, and what every row of the tile sees
        const int base_pos = s.len - s.n;
        int pos[MT][2];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int h = 0; h < 2; ++h) pos[m][h] = base_pos + (row_first + 16 * m + 8 * h + g) / p.group;
        const int all_hi = base_pos + row_first / p.group;  // last token the first row sees
        const int all_lo = p.window > 0 ? base_pos + (row_first + rows - 1) / p.group - p.window + 1 : 0;

        int c_slot = 0;
#pragma unroll 1
        for (int st = w0; st < w1; ++st) {
          cp_async_wait_all_but(p.depth - 1);
          const uint32_t slot = ring_at + static_cast<uint32_t>(c_slot) * SLOT;
          c_slot = c_slot + 1 == p.depth ? 0 : c_slot + 1;
          const int tok0 = lo + st * KVA_STEP;
          // ---- scores: rows x 16 tokens
          float sc[MT][2][4];
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int v = 0; v < 4; ++v) sc[m][j][v] = 0.0f;
#pragma unroll
          for (int c = 0; c < D / 64; ++c) {
            uint32_t kw[2][4];
#pragma unroll
            for (int j = 0; j < 2; ++j)
              ptx::ld_shared_v4(slot + (j * (D / 64) + c) * 512 + lane * 16, kw[j][0], kw[j][1], kw[j][2], kw[j][3]);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              uint32_t b0[2], b1[2];
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                const uint32_t u = kw[j][w] ^ 0x80808080u;
                b0[j] = lo_halves(u);
                b1[j] = hi_halves(u);
              }
#pragma unroll
              for (int m = 0; m < MT; ++m) {
                const int ks = m * KS + c * 4 + w;
                uint32_t a0, a1, a2, a3;
                if constexpr (Q_REGS) {
                  a0 = qf[4 * ks]; a1 = qf[4 * ks + 1]; a2 = qf[4 * ks + 2]; a3 = qf[4 * ks + 3];
                } else {
                  ptx::ld_shared_v4(q_at + ks * 512, a0, a1, a2, a3);
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) mma_f16_m16n8k16(sc[m][j], a0, a1, a2, a3, b0[j], b1[j]);
              }
            }
          }
          float sk, sv;
          asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(sk), "=f"(sv) : "r"(slot + KVA_STEP * 2 * D + lane * 8) : "memory");
          if (sv == 0.0f) sv = 1e-30f;  // a page of zeros: its codes are 0, its tokens still count in l
          const float kscale = p.scale_log2 * sk, lsv = __log2f(sv), inv_sv = __fdividef(1.0f, sv);
          const bool masked = tok0 + KVA_STEP - 1 > all_hi || tok0 < all_lo;
          uint32_t pw[MT][4];
#pragma unroll
          for (int m = 0; m < MT; ++m) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int v = 0; v < 4; ++v) {
                float x = fmaf(sc[m][j][v], kscale, lsv);
                if (masked) {
                  const int tok = tok0 + 8 * j + 2 * t + (v & 1), at_pos = pos[m][v >> 1];
                  if (tok > at_pos || (p.window > 0 && tok <= at_pos - p.window)) x = -INFINITY;
                }
                sc[m][j][v] = x;
              }
            float top[2], ref[2];
            bool grow = false;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              top[h] = fmaxf(fmaxf(sc[m][0][2 * h], sc[m][0][2 * h + 1]), fmaxf(sc[m][1][2 * h], sc[m][1][2 * h + 1]));
              top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], 1));
              top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], 2));
              top[h] = fmaxf(top[h], mrow[m][h]);
              grow |= top[h] > mrow[m][h];
              ref[h] = top[h] == -INFINITY ? 0.0f : top[h];
            }
            if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const float f = exp2_approx(mrow[m][h] - ref[h]);
                lrow[m][h] *= f;
                mrow[m][h] = top[h];
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                  o[m][i][2 * h] *= f;
                  o[m][i][2 * h + 1] *= f;
                }
              }
            }
            float sum[2] = {0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const float e0 = exp2_approx(sc[m][j][2 * h] - ref[h]), e1 = exp2_approx(sc[m][j][2 * h + 1] - ref[h]);
                sum[h] += e0 + e1;
                pw[m][2 * j + h] = pack_halves(e0, e1);
              }
            lrow[m][0] = fmaf(sum[0], inv_sv, lrow[m][0]);
            lrow[m][1] = fmaf(sum[1], inv_sv, lrow[m][1]);
          }
          // ---- O += w V
#pragma unroll
          for (int c = 0; c < VP; ++c) {
            uint32_t vw[4][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if constexpr (D == 64) {
                asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(vw[j][0]), "=r"(vw[j][1]) : "r"(slot + KP * 512 + j * 256 + lane * 8) : "memory");
              } else {
                ptx::ld_shared_v4(slot + KP * 512 + (j * VP + c) * 512 + lane * 16, vw[j][0], vw[j][1], vw[j][2], vw[j][3]);
              }
            }
#pragma unroll
            for (int w = 0; w < (D == 64 ? 2 : 4); ++w) {
              uint32_t pair[2][2];  // [tokens 2t,2t+1 / +8,+9][columns 0,1 / 2,3] bytes interleaved by token
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const uint32_t a = vw[2 * h][w] ^ 0x80808080u, bb = vw[2 * h + 1][w] ^ 0x80808080u;
                pair[h][0] = __byte_perm(a, bb, 0x5140);
                pair[h][1] = __byte_perm(a, bb, 0x7362);
              }
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint32_t b0 = (i & 1) ? hi_halves(pair[0][i >> 1]) : lo_halves(pair[0][i >> 1]);
                const uint32_t b1 = (i & 1) ? hi_halves(pair[1][i >> 1]) : lo_halves(pair[1][i >> 1]);
#pragma unroll
                for (int m = 0; m < MT; ++m)
                  mma_f16_m16n8k16(o[m][c * 16 + 4 * w + i], pw[m][0], pw[m][1], pw[m][2], pw[m][3], b0, b1);
              }
            }
          }
          fetch();
        }
        cp_async_wait<0>();

        // ---- join the warps: [warp][row][D + 2] (O, m, l)
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            lrow[m][h] += __shfl_xor_sync(0xffffffffu, lrow[m][h], 1);
            lrow[m][h] += __shfl_xor_sync(0xffffffffu, lrow[m][h], 2);
          }
        __syncthreads();  // every warp is done with its ring
        float* const mine = merge + warp * kva_rows_floats(ROWS, D);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int r = 16 * m + 8 * h + g;
            float* const dst = mine + r * (D + 2);
#pragma unroll
            for (int i = 0; i < NT; ++i) {
              // column tile i = 16 c + j of piece c: columns n of it are d = 128 c + 16 n + j (D = 64: 8 n + j)
              const int per_n = D == 64 ? 8 : 16, c = i / per_n, j = i % per_n;
              dst[c * 128 + per_n * (2 * t) + j] = o[m][i][2 * h];
              dst[c * 128 + per_n * (2 * t + 1) + j] = o[m][i][2 * h + 1];
            }
            if (t == 0) {
              dst[D] = mrow[m][h];
              dst[D + 1] = lrow[m][h];
            }
          }
        __syncthreads();
        const bool whole = s0 == 0 && s1 == unit_steps;
        float* const part = p.partial + (2 * static_cast<long long>(blockIdx.x) + (first_piece ? 0 : 1)) *
                                            kva_rows_floats(ROWS, D);
        auto out_at = [&](int r) {
          const int row = row_first + r, qi = row / p.group;
          return p.out + (static_cast<long long>(s.row0) + qi) * p.out_token_stride +
                 (static_cast<long long>(head) * p.group + (row - qi * p.group)) * D;
        };
        for (int idx = tid; idx < rows * (D / 2); idx += KVA_THREADS) {
          const int r = idx / (D / 2), d = idx % (D / 2) * 2;
          float top = -INFINITY;
#pragma unroll
          for (int w = 0; w < KVA_WARPS; ++w) top = fmaxf(top, merge[w * kva_rows_floats(ROWS, D) + r * (D + 2) + D]);
          const float ref = top == -INFINITY ? 0.0f : top;
          float a0 = 0.0f, a1 = 0.0f, l = 0.0f;
#pragma unroll
          for (int w = 0; w < KVA_WARPS; ++w) {
            const float* src = merge + w * kva_rows_floats(ROWS, D) + r * (D + 2);
            const float f = exp2_approx(src[D] - ref);
            a0 = fmaf(src[d], f, a0);
            a1 = fmaf(src[d + 1], f, a1);
            l = fmaf(src[D + 1], f, l);
          }
          if (whole) {
            const float inv = l == 0.0f ? 0.0f : __fdividef(1.0f, l);
            *reinterpret_cast<__half2*>(out_at(r) + d) = __floats2half2_rn(a0 * inv, a1 * inv);
          } else {
            float* dst = part + r * (D + 2);
            dst[d] = a0;
            dst[d + 1] = a1;
            if (d == 0) {
              dst[D] = top;
              dst[D + 1] = l;
            }
          }
        }
        if (!whole) {
          // ---- hand over; the last CTA of this unit joins
          const long long u_begin = at - s0, u_end = u_begin + unit_steps;
          const int c_first = static_cast<int>(u_begin / share), c_last = static_cast<int>((u_end - 1) / share);
          const long long tiles_max = (static_cast<long long>(p.max_q) * p.group + ROWS - 1) / ROWS;
          unsigned* const counter = p.arrived + (b * tiles_max + qt) * heads + head;
          __threadfence();
          __syncthreads();
          if (tid == 0) s_last = atomicAdd(counter, 1u);
          __syncthreads();
          if (s_last == static_cast<unsigned>(c_last - c_first)) {
            __threadfence();
            if (tid == 0) *counter = 0;
            for (int idx = tid; idx < rows * (D / 2); idx += KVA_THREADS) {
              const int r = idx / (D / 2), d = idx % (D / 2) * 2;
              float top = -INFINITY, a0 = 0.0f, a1 = 0.0f, l = 0.0f;
              for (int c = c_first; c <= c_last; ++c) {
                // the first CTA's piece of the unit is its last one unless the unit starts its share
                const int second = (c == c_first && u_begin > share * c) ? 1 : 0;
                const float* src = p.partial + (2ll * c + second) * kva_rows_floats(ROWS, D) + r * (D + 2);
                const float m = __ldcg(src + D);
                const float now = fmaxf(top, m);
                const float ref = now == -INFINITY ? 0.0f : now;
                const float f0 = exp2_approx(top - ref), f1 = exp2_approx(m - ref);
                const float2 x = __ldcg(reinterpret_cast<const float2*>(src + d));
                a0 = fmaf(x.x, f1, a0 * f0);
                a1 = fmaf(x.y, f1, a1 * f0);
                l = fmaf(__ldcg(src + D + 1), f1, l * f0);
                top = now;
              }
              const float inv = l == 0.0f ? 0.0f : __fdividef(1.0f, l);
              *reinterpret_cast<__half2*>(out_at(r) + d) = __floats2half2_rn(a0 * inv, a1 * inv);
            }
          }
        }
        __syncthreads();  // the results are read: the rings may be filled again
        first_piece = false;
        at += s1 - s0;
      }
    }
  }
}

}  // namespace b200gemm
