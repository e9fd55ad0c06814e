// Attention over the INT8 cache for many query rows per KV head (a chunk of a prompt): the two products
// on the 5th-generation tensor cores.  Same mathematics as kv_attention.cuh, except that q stays binary16.
//
// A CTA owns QT tiles of 128 rows (queries x heads of a group) of one KV head and walks its tokens in tiles of
// TN.  Per tile of rows and tokens: S = Q K^T (tcgen05.mma, operands in shared memory) into tensor memory; four warps,
// one thread per row, turn S into weights, rounded to binary16, in the same place; O += P V (A operand in tensor
// memory).  With two tiles of rows one is in its softmax while the tensor cores work on the other.
// K and V arrive as int8, by bulk copies of whole pages of a head; four warps convert them
// exactly to binary16 and write them as rows of 64 d in the 128-byte swizzle.  Such a tile is K-major for the
// first product and, read the other way round, MN-major for the second: no transpose anywhere.
// Page scales: a table of (c sk, log2 sv, 1 / sv) per 16 tokens, in a ring of its own.
// A page whose scale is not finite or below 0 gets harmless factors and raises a flag: the rows then look through the pages
// that they see themselves, at the end, and become NaN by their l (a test per tile of tokens costs 2 %).
//
// What bounds it: at 128 d, 1024 cycles of tensor pipe a tile pair of 128 x 128 against as many of exponentials
// (16 a cycle and SM); the conversion takes a tenth of the issue slots.  O is rescaled in tensor memory only
// when a row's maximum has grown by 2^8 (see kv_attention.cuh), so that it need not pass through registers.
// Tiles of rows are taken longest first.  With fewer of them than half the SMs the tokens are split too, and the
// CTA that finishes a row tile last joins the parts (4 x 64 queries over <= 8192 tokens: 150 -> 78 us).
// Measured: 2 x 2048 queries, 32 heads on 8, over <= 8192 tokens 326-331 us (0.55 of the cuBLAS bf16 rate), 4096
// queries over themselves 187 us.  A pair of row tiles takes 4140 cycles per 128 tokens where its products and its
// exponentials are 2048 each: per row tile scores -> maximum (600) -> weights (1580: the two row tiles share the
// exponential unit) -> both products (1400: the first takes shared memory's 128 bytes a cycle up by itself, the conversion
// wants some too) is a chain.  Slower: two buffers of 64 scores per row tile (421 against 358 us then), part of the
// exponentials as a polynomial (383-510), weights handed over in two or four parts (353, 369 against 331: the
// issuing thread waits in order and holds back the other row tile's products), weights without the maximum first,
// checked afterwards (338).
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

#include "bounded_wait.cuh"
#include "kv_attention.cuh"
#include "ptx.cuh"

namespace b200gemm {

template <int D>
struct KvTileShape {
  static constexpr int QT = D <= 128 ? 2 : 1;      // row tiles of 128 per CTA (O fills tensor memory beyond that)
  static constexpr int TN = D <= 128 ? 128 : 64;   // tokens per tile
  static constexpr int ROWS = 128 * QT;
  static constexpr int SOFTMAX_WARPS = 4 * QT;
  static constexpr int THREADS = 32 * (SOFTMAX_WARPS + 8);  // + 4 converting, MMA issuer, loader, two idle
  static constexpr int STAGES = 2;
  static constexpr int GROUPS = TN / 16;
  static constexpr int CHUNK = TN * 128;           // bytes of 64 d of a K or V tile
  static constexpr int Q_BYTES = QT * (D / 64) * 128 * 128;
  static constexpr int KV_BYTES = (D / 64) * CHUNK;
  static constexpr int K_OFFSET = Q_BYTES;
  static constexpr int V_OFFSET = K_OFFSET + STAGES * KV_BYTES;
  static constexpr int SCALES = 4;                 // ring of scale tables
  static constexpr int RAW_BYTES = TN * D;         // int8 codes of a K or V tile
  static constexpr int RAW_OFFSET = V_OFFSET + STAGES * KV_BYTES;  // K, V of one tile; then of the next
  static constexpr int SCALE_OFFSET = RAW_OFFSET + 2 * RAW_BYTES;
  static constexpr int BAR_OFFSET = SCALE_OFFSET + SCALES * GROUPS * 16;
  // q_full, k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], p_full[2], o_done[2], scale_full[4], drain,
  // raw_full[2], raw_empty[2] (K, V)
  static constexpr int BARS = 1 + 4 * STAGES + 6 + SCALES + 1 + 4;
  static constexpr int MISC_OFFSET = BAR_OFFSET + BARS * 8;
  static constexpr int DYN_BYTES = MISC_OFFSET + 16 + 1024;
  static constexpr uint32_t O_COLUMN = 256;        // S (and P) of tile q at 128 q, O behind both
  // O is summed in tensor memory over this many tiles of tokens at most, 16384 tokens: the accumulator cuts off what does
  // not fit, 1e-9 to 2e-9 of the result a token (6.4e-9 with values of one sign), always towards zero (131072 tokens in one sum: 1.3e-4 to 2.8e-4, as much
  // as the rounding to binary16).  Then the rows' threads add it to a sum in scratch.
  static constexpr int SUM_TILES = 16384 / TN;
  static_assert(DYN_BYTES <= 232448, "exceeds the 227 KB shared-memory limit per CTA");
  static_assert(O_COLUMN + QT * D <= 512, "tensor memory");
};

// The rank-th longest row tile of all sequences (sequence, tile), or (-1, 0) beyond the last: CTAs start in order,
// and a long one that starts last leaves the rest of the chip idle (2 x 2048 queries over 8192 and 3130 tokens:
// 358 -> 326 us).  A row tile's length is its number of token tiles (without a window; with one they are much
// alike).  By one warp, a lane per sequence, searching for the length that `rank` tiles exceed.
template <int ROWS, int TN>
__device__ __noinline__ int2 kvt_item(const KvAttnParams& p, int rank) {
  const int lane = static_cast<int>(threadIdx.x) & 31;
  auto tiles_of = [&](const KvSeq& s) { return s.n * p.group <= p.split_rows ? 0 : (s.n * p.group + ROWS - 1) / ROWS; };
  if (p.batch == 1) {  // its own order
    const int tiles = tiles_of(kv_seq(p, 0, rank == 0 && lane == 0));
    return rank < tiles ? make_int2(0, tiles - 1 - rank) : make_int2(-1, 0);
  }
  // row tiles of a sequence that are at least x token tiles long: their last query sees beyond (x - 1) TN
  auto long_tiles = [&](const KvSeq& s, int x) {
    const int all = tiles_of(s), need = (x - 1) * TN - (s.len - s.n);  // first query that sees so far
    if (x <= 0 || need <= 0) return all;
    return need < s.n ? all - static_cast<int>(static_cast<long long>(need) * p.group / ROWS) : 0;
  };
  int longest = 0, all = 0;
  for (int i = lane; i < p.batch; i += 32) {
    const KvSeq s = kv_seq(p, i, rank == 0);
    longest = max(longest, (s.len + TN - 1) / TN);
    all += tiles_of(s);
  }
  longest = static_cast<int>(__reduce_max_sync(0xffffffffu, static_cast<unsigned>(longest)));
  all = static_cast<int>(__reduce_add_sync(0xffffffffu, static_cast<unsigned>(all)));
  if (rank >= all) return make_int2(-1, 0);
  int x_lo = 0, x_hi = longest + 1, beyond = 0;  // more than rank tiles are x_lo long, `beyond` <= rank are x_hi long
#pragma unroll 1
  while (x_hi - x_lo > 1) {
    const int mid = (x_lo + x_hi) / 2;
    int c = 0;
    for (int i = lane; i < p.batch; i += 32) c += long_tiles(kv_seq(p, i, false), mid);
    c = static_cast<int>(__reduce_add_sync(0xffffffffu, static_cast<unsigned>(c)));
    if (c > rank) {
      x_lo = mid;
    } else {
      x_hi = mid;
      beyond = c;
    }
  }
  // the tiles of exactly that length, by sequence
  int left = rank - beyond;
#pragma unroll 1
  for (int i0 = 0; i0 < p.batch; i0 += 32) {
    int same = 0, qt = 0;
    if (i0 + lane < p.batch) {
      const KvSeq s = kv_seq(p, i0 + lane, false);
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
      return make_int2(i0 + from, __shfl_sync(0xffffffffu, qt - (left - (incl - same)), from));
    }
    left -= __shfl_sync(0xffffffffu, incl, 31);
  }
  return make_int2(-1, 0);  // (not reached: the tiles of that length are `rank - beyond` and more)
}

template <int D>
__global__ void __launch_bounds__(KvTileShape<D>::THREADS, 1)
kv_attention_tiles_kernel(const __grid_constant__ KvAttnParams p) {
  using namespace kva;
  using T = KvTileShape<D>;
  constexpr int QT = T::QT, TN = T::TN, GROUPS = T::GROUPS, STAGES = T::STAGES;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = ptx::smem_addr(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* const base_ptr = smem_raw + (base - raw);
  const uint32_t bar0 = base + T::BAR_OFFSET;
  const uint32_t q_full = bar0;
  auto k_full = [&](int s) { return bar0 + 8u * (1 + s); };
  auto k_empty = [&](int s) { return bar0 + 8u * (3 + s); };
  auto v_full = [&](int s) { return bar0 + 8u * (5 + s); };
  auto v_empty = [&](int s) { return bar0 + 8u * (7 + s); };
  auto s_full = [&](int q) { return bar0 + 8u * (9 + q); };
  auto p_full = [&](int q) { return bar0 + 8u * (11 + q); };
  auto o_done = [&](int q) { return bar0 + 8u * (13 + q); };
  auto scale_full = [&](int s) { return bar0 + 8u * (15 + s); };
  const uint32_t drain = bar0 + 8u * 19;
  auto raw_full = [&](int w) { return bar0 + 8u * (20 + w); };
  auto raw_empty = [&](int w) { return bar0 + 8u * (22 + w); };
  static_assert(T::BARS == 24, "barrier numbering");
  volatile uint32_t* const tmem_holder = reinterpret_cast<volatile uint32_t*>(base_ptr + T::MISC_OFFSET);
  volatile uint32_t* const abort_flag = tmem_holder + 1;
  volatile uint32_t* const poison_flag = tmem_holder + 2;  // a page of this CTA's tokens has a scale that is not finite
  const int tid = static_cast<int>(threadIdx.x), lane = tid & 31, warp = tid >> 5;
  if (tid == 0) ptx::grid_dep_launch_dependents();

  // ---- what this CTA works on
  ptx::grid_dep_wait();
  const int heads = p.c.heads;
  const int unit = static_cast<int>(blockIdx.x) / p.splits, split = static_cast<int>(blockIdx.x) - unit * p.splits;
  const int rank = unit / heads, head = unit - rank * heads;
  __shared__ int s_item[2];
  if (warp == 0) {
    const int2 item = kvt_item<T::ROWS, TN>(p, rank);
    if (lane == 0) {
      s_item[0] = item.x;
      s_item[1] = item.y;
    }
  }
  __syncthreads();
  const int b = s_item[0], qt = s_item[1];
  if (b < 0) return;
  const KvSeq s = kv_seq(p, b, false);
  const int all_rows = s.n * p.group;
  const int row_first = qt * T::ROWS, rows = min(T::ROWS, all_rows - row_first);
  const int active = QT == 2 && rows > 128 ? 2 : 1;  // row tiles with a row in them
  int lo, hi;
  kv_visible(p, s, row_first / p.group, (row_first + rows + p.group - 1) / p.group, lo, hi);
  const int visible_lo = lo;  // pages wholly in front of it are not looked at: their owners may have given them away
  lo = lo / TN * TN;
  int tiles = (hi - lo + TN - 1) / TN;  // 0: nothing is visible
  if (p.splits > 1) {  // this CTA's part of the tokens
    const int per = (tiles + p.splits - 1) / p.splits, first = min(tiles, split * per);
    tiles = min(tiles, first + per) - first;
    lo += first * TN;
    hi = min(hi, lo + tiles * TN);
  }

  __shared__ int s_slot;  // of the sums in scratch; -1 = none needed
  if (tid == 0) {
    s_slot = -1;
    if (p.long_sums && tiles > T::SUM_TILES) {
      // There are as many slots as CTAs at a time, so one is free at any time; which one may change while this looks
      // at them, hence the (limited) rounds.  The one that the SM's last CTA had is as a rule free at once.
      uint32_t sm;
      asm volatile("mov.u32 %0, %%smid;" : "=r"(sm));
      for (int i = 0; i < 1000 * p.slots && s_slot < 0; ++i) {
        const int slot = static_cast<int>((sm + static_cast<uint32_t>(i)) % static_cast<uint32_t>(p.slots));
        if (atomicCAS(p.taken + slot, 0u, 1u) == 0u) s_slot = slot;
      }
      __threadfence();
    }
    ptx::mbar_init(q_full, T::SOFTMAX_WARPS);
    for (int i = 0; i < STAGES; ++i) {
      ptx::mbar_init(k_full(i), 4);
      ptx::mbar_init(k_empty(i), 1);
      ptx::mbar_init(v_full(i), 4);
      ptx::mbar_init(v_empty(i), 1);
    }
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(s_full(i), 1);
      ptx::mbar_init(p_full(i), 4);
      ptx::mbar_init(o_done(i), 1);
    }
    for (int i = 0; i < T::SCALES; ++i) ptx::mbar_init(scale_full(i), 1);
    ptx::mbar_init(drain, 1);
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(raw_full(i), 1);
      ptx::mbar_init(raw_empty(i), 4);
    }
    *abort_flag = 0;
    *poison_flag = 0;
    ptx::fence_mbar_init();
  }
  if (warp == T::SOFTMAX_WARPS + 4) {
    ptx::tmem_alloc<1>(ptx::smem_addr(const_cast<uint32_t*>(tmem_holder)), 512);
    ptx::tmem_relinquish<1>();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  const uint32_t tmem = *tmem_holder;
  const int slot = s_slot;
  // the tile whose products start a new sum in tensor memory
  auto new_sum = [&](int j) { return j == 0 || (slot >= 0 && (j & (T::SUM_TILES - 1)) == 0); };

  if constexpr (QT == 2) {
    // Register shares of the four groups of four warps, which sum up to the 4 x 128 they were launched with:
    // the scores of a row stay in registers between the maximum and the weights.
    if (warp < T::SOFTMAX_WARPS) {
      asm volatile("setmaxnreg.inc.sync.aligned.u32 176;");
    } else if (warp < T::SOFTMAX_WARPS + 4) {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 96;");
    } else {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    }
  }
  if (warp < T::SOFTMAX_WARPS) {
    // ------------------------------------------------------------------ softmax, one thread per row
    const int q = warp >> 2;
    const int r = q * 128 + (warp & 3) * 32 + lane;  // row of the CTA
    const int row = row_first + r, qi = row / p.group, hq = head * p.group + (row - qi * p.group);
    const bool live = r < rows;
    const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_at = tmem + lane_base + static_cast<uint32_t>(q * 128);
    const uint32_t o_at = tmem + lane_base + T::O_COLUMN + static_cast<uint32_t>(q * D);
    uint32_t q_top = 0;  // two maxima of magnitude bits of the row
    if (q < active) {  // this row of Q, in the 128-byte swizzle
      const __half* const src = p.q + (static_cast<long long>(s.row0) + (live ? qi : 0)) * p.q_token_stride +
                                static_cast<long long>(live ? hq : 0) * p.q_head_stride;
      const uint32_t dst = base + static_cast<uint32_t>(q * (D / 64) * 16384 + (r & 127) * 128);
#pragma unroll 8
      for (int u = 0; u < D / 8; ++u) {
        uint4 x = make_uint4(0, 0, 0, 0);
        if (live) x = ptx::ld_global_stream_v4(src + u * 8);
        q_top = __vmaxu2(q_top, __vmaxu2(__vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu),
                                         __vmaxu2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu)));
        ptx::st_shared_v4(dst + static_cast<uint32_t>((u >> 3) * 16384 + (((u & 7) ^ (r & 7)) << 4)), x.x, x.y, x.z, x.w);
      }
      ptx::fence_proxy_async_smem();
    }
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(q_full);

    const int pos = s.len - s.n + qi;  // sees tokens from .. pos
    const int from = p.window > 0 ? pos - p.window + 1 : 0;
    const int all_hi = s.len - s.n + (row_first + q * 128) / p.group;
    const int all_lo = p.window > 0 ? s.len - s.n + (row_first + min(rows, q * 128 + 128) - 1) / p.group - p.window + 1 : 0;
    // A row with a NaN or an infinity is NaN if it sees anything, also where all its scores are -inf.
    const bool q_bad = max(q_top & 0xffffu, q_top >> 16) >= 0x7c00u && pos >= 0;
    float m = -INFINITY, l = q_bad ? __int_as_float(0x7fffffff) : 0.0f;
    float* const long_sum = p.long_sums + (static_cast<long long>(max(slot, 0)) * T::ROWS + r) * D;
    float long_m = -INFINITY;  // reference of the sum in scratch
    auto long_factor = [&]() { return long_m == -INFINITY ? 0.0f : exp2_approx(long_m - m); };
    bool ok = true;
    const int my_tiles = q < active ? tiles : 0;
#pragma unroll 1
    for (int j = 0; j < my_tiles; ++j) {
      ok = wait_bounded(scale_full(j & 3), (j >> 2) & 1, abort_flag, p.status, DEV_TIMEOUT_EPILOGUE) &&
           wait_bounded(s_full(q), j & 1, abort_flag, p.status, DEV_TIMEOUT_EPILOGUE);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      ptx::tc_fence_after_sync();
      const float4* const scale = reinterpret_cast<const float4*>(base_ptr + T::SCALE_OFFSET) + (j & 3) * GROUPS;
      const int tok0 = lo + j * TN;
      const bool masked = tok0 + TN - 1 > all_hi || tok0 < all_lo;
      uint32_t x[TN / 32][32];
#pragma unroll
      for (int h = 0; h < TN / 32; ++h) ptx::tmem_ld_32x32b_x32(s_at + h * 32, x[h]);
      ptx::tmem_wait_ld();
      if (masked) {
#pragma unroll
        for (int h = 0; h < TN / 32; ++h)
#pragma unroll
          for (int v = 0; v < 32; ++v) {
            const int tok = tok0 + h * 32 + v;
            if (tok > pos || tok < from) x[h][v] = 0xff800000u;  // -inf
          }
      }
      // the largest score of the row
      float top = -INFINITY;
#pragma unroll
      for (int g = 0; g < GROUPS; ++g) {
        float mx = __uint_as_float(x[g / 2][16 * (g & 1)]);
#pragma unroll
        for (int v = 1; v < 16; ++v) mx = fmaxf(mx, __uint_as_float(x[g / 2][16 * (g & 1) + v]));
        const float4 c = scale[g];
        top = fmaxf(top, fmaf(mx, c.x, c.y));
      }
      const bool grow = top > m + 8.0f;
      const bool move = j > 0 && new_sum(j);
      if (__any_sync(0xffffffffu, grow) || move) {
        const float now = grow ? top : m;
        const float f = now == -INFINITY ? 1.0f : exp2_approx(m - now);
        m = now;
        l *= f;
        if (j > 0) {  // O of the tiles before, once their products are done
          ok = wait_bounded(o_done(q), (j - 1) & 1, abort_flag, p.status, DEV_TIMEOUT_EPILOGUE);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          ptx::tc_fence_after_sync();
          const float of_old = long_factor();
#pragma unroll 1
          for (int c = 0; c < D; c += 16) {
            uint32_t y[16];  // (few registers: the scores are in the others)
            ptx::tmem_ld_32x32b_x16(o_at + c, y);
            ptx::tmem_wait_ld();
#pragma unroll
            for (int v = 0; v < 16; ++v) y[v] = __float_as_uint(__uint_as_float(y[v]) * f);
            if (move) {
#pragma unroll 1
              for (int v = 0; v < 16; ++v) {
                float sum = __uint_as_float(y[0]);
#pragma unroll
                for (int u = 0; u < 15; ++u) y[u] = y[u + 1];
                if (j > T::SUM_TILES) sum = fmaf(__ldcg(long_sum + c + v), of_old, sum);
                __stcg(long_sum + c + v, sum);
              }
            } else {
              ptx::tmem_st_32x32b_x16(o_at + c, y);
            }
          }
          if (move) long_m = m;
          ptx::tmem_wait_st();
        }
      }
      const float ref = (m == -INFINITY ? 0.0f : m) - KVA_WEIGHT_BITS;
      // weights, two per column, over the scores: 32 tokens take 16 columns
#pragma unroll
      for (int h = 0; h < TN / 32; ++h) {
        uint32_t w[16];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          const float4 c = scale[2 * h + g];
          const float at_ref = c.y - ref;
          float sum0 = 0.0f, sum1 = 0.0f;
#pragma unroll
          for (int v = 0; v < 16; v += 2) {
            const float e0 = exp2_approx(fmaf(__uint_as_float(x[h][16 * g + v]), c.x, at_ref));
            const float e1 = exp2_approx(fmaf(__uint_as_float(x[h][16 * g + v + 1]), c.x, at_ref));
            sum0 += e0;
            sum1 += e1;
            w[8 * g + v / 2] = pack_halves(e0, e1);
          }
          l = fmaf(sum0 + sum1, c.z, l);
        }
        ptx::tmem_st_32x32b_x16(s_at + h * 16, w);
      }
      ptx::tmem_wait_st();
      ptx::tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(p_full(q));
    }
    // ---- the rows' results
    if (q < active && ok) {
      if (tiles > 0) {
        ok = wait_bounded(o_done(q), (tiles - 1) & 1, abort_flag, p.status, DEV_TIMEOUT_EPILOGUE);
        ok = __all_sync(0xffffffffu, ok);
        ptx::tc_fence_after_sync();
      }
      if (*poison_flag && live) {  // (written in front of the scale_full arrivals this thread has waited for)
        const int* const table = p.table + static_cast<long long>(b) * p.table_stride;
        const int last = min(pos, hi - 1);
#pragma unroll 1
        for (int t = max(from, lo); t <= last; t = (t | (p.c.page - 1)) + 1) {
          const int id = kv_ld(table + (t >> p.c.page_shift));
          if (id < 0 || id >= p.c.num_pages) continue;
          const long long ph = static_cast<long long>(id) * heads + head;
          if (kva_no_scales(ptx::ld_global_f32(p.c.scales[0] + ph), ptx::ld_global_f32(p.c.scales[1] + ph)))
            l = __int_as_float(0x7fffffff);
        }
      }
      const float inv = l == 0.0f ? 0.0f : __fdividef(1.0f, l);
      float* const part = p.partial + (static_cast<long long>(blockIdx.x) * T::ROWS + r) * (D + 4);
      if (p.splits > 1 && live && ok) *reinterpret_cast<float2*>(part + D) = make_float2(m, l);
      __half* const dst = p.out + (static_cast<long long>(s.row0) + qi) * p.out_token_stride + static_cast<long long>(hq) * D;
#pragma unroll 1
      for (int c = 0; c < D && ok; c += 32) {
        uint32_t x[32];
        if (tiles > 0) {
          ptx::tmem_ld_32x32b_x32(o_at + c, x);
          ptx::tmem_wait_ld();
          if (slot >= 0) {
            const float of_old = long_factor();
#pragma unroll
            for (int v = 0; v < 32; ++v) x[v] = __float_as_uint(fmaf(__ldcg(long_sum + c + v), of_old, __uint_as_float(x[v])));
          }
        }
        if (!live) continue;
        if (p.splits > 1) {  // O as it stands, to be joined
#pragma unroll
          for (int v = 0; v < 8; ++v)
            *reinterpret_cast<uint4*>(part + c + 4 * v) =
                tiles > 0 ? make_uint4(x[4 * v], x[4 * v + 1], x[4 * v + 2], x[4 * v + 3]) : make_uint4(0, 0, 0, 0);
          continue;
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          uint32_t y[4];
#pragma unroll
          for (int u = 0; u < 4; ++u)
            y[u] = tiles > 0 ? pack_halves(__uint_as_float(x[8 * v + 2 * u]) * inv, __uint_as_float(x[8 * v + 2 * u + 1]) * inv) : 0u;
          *reinterpret_cast<uint4*>(dst + c + 8 * v) = make_uint4(y[0], y[1], y[2], y[3]);
        }
      }
    }
  } else if (warp < T::SOFTMAX_WARPS + 4) {
    // ------------------------------------------------------------------ K and V: int8 codes to binary16 tiles
    const int ct = tid - 32 * T::SOFTMAX_WARPS;       // 0 .. 127
    constexpr int PER_TOKEN = D / 16;                 // 16-byte pieces of a token
    constexpr int N = TN * PER_TOKEN / 128;           // pieces per thread and tile
    constexpr int TOKENS_AT_ONCE = 128 / PER_TOKEN;   // tokens the 128 threads cover together
    const int c = ct % PER_TOKEN, t0 = ct / PER_TOKEN;
    // the two 16-byte pieces of the 128-byte row; odd chunks of 64 d store them in the other order, which
    // keeps eight neighbouring lanes on different banks
    const uint32_t chunk_at = static_cast<uint32_t>((c >> 2) * T::CHUNK);
    const uint32_t unit = static_cast<uint32_t>((c & 3) * 2), flip = static_cast<uint32_t>((c >> 2) & 1);
    auto convert = [&](int which, uint32_t tile) {
      const uint32_t src = base + T::RAW_OFFSET + which * T::RAW_BYTES + static_cast<uint32_t>(ct * 16);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int tok = i * TOKENS_AT_ONCE + t0;
        uint32_t w[4];
        ptx::ld_shared_v4(src + i * 2048, w[0], w[1], w[2], w[3]);
#pragma unroll
        for (int v = 0; v < 4; ++v) w[v] ^= 0x80808080u;
        const uint32_t at = tile + chunk_at + static_cast<uint32_t>(tok * 128);
        const uint32_t sw = static_cast<uint32_t>(tok & 7);
        const uint32_t a0 = flip ? w[2] : w[0], a1 = flip ? w[3] : w[1];
        const uint32_t b0 = flip ? w[0] : w[2], b1 = flip ? w[1] : w[3];
        ptx::st_shared_v4(at + (((unit + flip) ^ sw) << 4), lo_halves(a0), hi_halves(a0), lo_halves(a1), hi_halves(a1));
        ptx::st_shared_v4(at + (((unit + (flip ^ 1u)) ^ sw) << 4), lo_halves(b0), hi_halves(b0), lo_halves(b1), hi_halves(b1));
      }
      ptx::fence_proxy_async_smem();
      __syncwarp();
    };
    bool ok = true;
#pragma unroll 1
    for (int j = 0; j < tiles; ++j) {
      const int st = j & 1;
      const uint32_t ph = ((j >> 1) & 1) ^ 1u;
      ok = wait_bounded(raw_full(0), j & 1, abort_flag, p.status, DEV_TIMEOUT_PRODUCER) &&
           wait_bounded(k_empty(st), ph, abort_flag, p.status, DEV_TIMEOUT_PRODUCER);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      convert(0, base + T::K_OFFSET + st * T::KV_BYTES);
      if (lane == 0) {
        ptx::mbar_arrive(k_full(st));
        ptx::mbar_arrive(raw_empty(0));
      }
      ok = wait_bounded(raw_full(1), j & 1, abort_flag, p.status, DEV_TIMEOUT_PRODUCER) &&
           wait_bounded(v_empty(st), ph, abort_flag, p.status, DEV_TIMEOUT_PRODUCER);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      convert(1, base + T::V_OFFSET + st * T::KV_BYTES);
      if (lane == 0) {
        ptx::mbar_arrive(v_full(st));
        ptx::mbar_arrive(raw_empty(1));
      }
    }
  } else if (warp == T::SOFTMAX_WARPS + 5) {
    // ------------------------------------------------------------------ loader: int8 pages and their scales
    // Lane g looks after the tile's g-th run of `run` tokens: one page, or half a tile's worth of a longer one.
    const int run = min(p.c.page, TN), runs = TN / run;
    const uint32_t run_bytes = static_cast<uint32_t>(run * D);
    const int* const table = p.table + static_cast<long long>(b) * p.table_stride;
    const uint64_t page_bytes = static_cast<uint64_t>(heads) * p.c.page * D;
    auto visible = [&](int j) {  // the lane's run of tile j, or a part of it
      const int tok = lo + j * TN + run * lane;
      return lane < runs && j < tiles && tok < hi && tok + run > visible_lo;
    };
    auto load_id = [&](int j) {  // its page, or -1
      return visible(j) ? kv_ld(table + ((lo + j * TN + run * lane) >> p.c.page_shift)) : -1;
    };
    bool ok = true;
    int id = load_id(0);
#pragma unroll 1
    for (int j = 0; j < tiles && ok; ++j) {
      const int id_next = load_id(j + 1);
      const bool in = visible(j);
      const bool good = in && id >= 0 && id < p.c.num_pages;
      if (in && !good) kv_report(p.status);
      const int tok = lo + j * TN + run * lane;
      const uint64_t off = good ? static_cast<uint64_t>(id) * page_bytes +
                                      static_cast<uint32_t>((head * p.c.page + (tok & (p.c.page - 1))) * D)
                                : 0;
      const uint32_t bytes = static_cast<uint32_t>(__popc(__ballot_sync(0xffffffffu, good))) * run_bytes;
      float sk = 0.0f, sv = 1.0f;
      if (good) {
        const long long ph = static_cast<long long>(id) * heads + head;
        sk = ptx::ld_global_f32(p.c.scales[0] + ph);
        sv = ptx::ld_global_f32(p.c.scales[1] + ph);
      }
#pragma unroll 1
      for (int which = 0; which < 2; ++which) {
        ok = wait_bounded(raw_empty(which), (j & 1) ^ 1, abort_flag, p.status, DEV_TIMEOUT_PRODUCER);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (lane == 0) ptx::mbar_arrive_expect_tx(raw_full(which), bytes);
        __syncwarp();
        // (runs that are left out keep what the buffer held: codes are finite, and their weights are 0)
        if (good)
          ptx::bulk_load(base + T::RAW_OFFSET + which * T::RAW_BYTES + lane * run_bytes,
                         (which ? p.c.codes[1] : p.c.codes[0]) + off, run_bytes, raw_full(which));
        if (which == 0) {
          // scales by groups of 16 tokens (a hidden token's -inf must stay one)
          const float v = kva_value_scale(sv), k = p.scale_log2 * sk;
          float4 c = make_float4(k == 0.0f ? 1e-30f : k, __log2f(v), __fdividef(1.0f, v), 0.0f);
          if (kva_no_scales(sk, sv)) {
            c = make_float4(1e-30f, 0.0f, 1.0f, 0.0f);
            *poison_flag = 1;
          }
          if (lane < runs)
            for (int g = 0; g < run / 16; ++g)
              reinterpret_cast<float4*>(base_ptr + T::SCALE_OFFSET)[(j & 3) * GROUPS + lane * (run / 16) + g] = c;
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(scale_full(j & 3));
        }
      }
      id = id_next;
    }
    if (!ok) {
      // Gave up: let the copies in flight land before the CTA exits.
      const uint64_t start = ptx::globaltimer_ns();
      while (ptx::globaltimer_ns() - start < 1000000ull) {
      }
    }
  } else if (warp == T::SOFTMAX_WARPS + 4) {
    // ------------------------------------------------------------------ MMA issuer
    const bool elected = ptx::elect_one();
    constexpr uint32_t idesc_qk = ptx::make_idesc<ptx::KIND_F16>(128, TN);
    constexpr uint32_t idesc_pv = ptx::make_idesc<ptx::KIND_F16>(128, D) | ptx::IDESC_B_MN_MAJOR;
    auto qk = [&](int q, int j) {
      if (elected) {
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          const uint32_t off = static_cast<uint32_t>((kk & 3) * 32);
          const uint64_t a = ptx::smem_desc_sw128(base + (q * (D / 64) + (kk >> 2)) * 16384 + off);
          const uint64_t k = ptx::smem_desc_sw128(base + T::K_OFFSET + (j & 1) * T::KV_BYTES + (kk >> 2) * T::CHUNK + off);
          ptx::mma_ss<ptx::KIND_F16, 1>(tmem + q * 128, a, k, idesc_qk, kk > 0);
        }
        ptx::mma_commit<1>(s_full(q));
      }
    };
    auto pv = [&](int q, int j) {
      if (elected) {
#pragma unroll
        for (int kk = 0; kk < TN / 16; ++kk) {
          const uint64_t v = ptx::smem_desc_sw128_mn(base + T::V_OFFSET + (j & 1) * T::KV_BYTES + kk * 2048, T::CHUNK);
          ptx::mma_f16_ts(tmem + T::O_COLUMN + q * D, tmem + q * 128 + kk * 8, v, idesc_pv, !new_sum(j) || kk > 0);
        }
        ptx::mma_commit<1>(o_done(q));
      }
    };
    bool ok = true;
    if (tiles > 0) {
      ok = wait_bounded(q_full, 0, abort_flag, p.status, DEV_TIMEOUT_MMA) &&
           wait_bounded(k_full(0), 0, abort_flag, p.status, DEV_TIMEOUT_MMA);
      if (ok) {
        ptx::tc_fence_after_sync();
        for (int q = 0; q < active; ++q) qk(q, 0);
        if (elected) ptx::mma_commit<1>(k_empty(0));
      }
    }
#pragma unroll 1
    for (int j = 0; j < tiles && ok; ++j) {
      ok = wait_bounded(v_full(j & 1), (j >> 1) & 1, abort_flag, p.status, DEV_TIMEOUT_MMA);
#pragma unroll 1
      for (int q = 0; q < active && ok; ++q) {
        ok = wait_bounded(p_full(q), j & 1, abort_flag, p.status, DEV_TIMEOUT_MMA);
        if (!ok) break;
        ptx::tc_fence_after_sync();
        pv(q, j);
        if (j + 1 < tiles) {  // (the scores go where the weights are: the MMAs of this thread run in order)
          if (q == 0) {
            ok = wait_bounded(k_full((j + 1) & 1), ((j + 1) >> 1) & 1, abort_flag, p.status, DEV_TIMEOUT_MMA);
            if (!ok) break;
            ptx::tc_fence_after_sync();
          }
          qk(q, j + 1);
        }
      }
      if (ok && elected) {
        ptx::mma_commit<1>(v_empty(j & 1));
        if (j + 1 < tiles) ptx::mma_commit<1>(k_empty((j + 1) & 1));
      }
    }
    if (!ok && elected) {
      // Gave up: wait for the MMAs already issued before tensor memory is released.
      ptx::mma_commit<1>(drain);
      const uint64_t start = ptx::globaltimer_ns();
      while (!ptx::mbar_try_wait(drain, 0) && ptx::globaltimer_ns() - start < WAIT_LIMIT_NS) {
      }
    }
    __syncwarp();
  }

  // Every role gets here: all waits are bounded, and the last products have been waited for above.
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (warp == T::SOFTMAX_WARPS + 4) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc<1>(tmem, 512);
  }
  if (tid == 0 && slot >= 0) {  // (the rows' threads are done with it)
    __threadfence();
    atomicExch(p.taken + slot, 0u);
  }
  if (p.splits > 1) {
    // ---- the CTA that finishes a row tile last joins its parts, in their order
    __threadfence();
    __syncthreads();
    __shared__ unsigned s_last;
    if (tid == 0) s_last = atomicAdd(p.arrived + unit, 1u);
    __syncthreads();
    if (s_last != static_cast<unsigned>(p.splits - 1)) return;
    __threadfence();
    if (tid == 0) p.arrived[unit] = 0;
    const float* const parts = p.partial + static_cast<long long>(unit) * p.splits * T::ROWS * (D + 4);
    for (int i = tid; i < rows * (D / 4); i += T::THREADS) {
      const int rr = i / (D / 4), d = i % (D / 4) * 4;
      const float* const mine = parts + rr * (D + 4);
      float top = -INFINITY, sum = 0.0f;
      float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      for (int k = 0; k < p.splits; ++k) {
        const float m = __ldcg(mine + static_cast<long long>(k) * T::ROWS * (D + 4) + D);
        top = m > top || m != m ? m : top;
      }
      const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll 4
      for (int k = 0; k < p.splits; ++k) {
        const float* const at = mine + static_cast<long long>(k) * T::ROWS * (D + 4);
        const float2 ml = __ldcg(reinterpret_cast<const float2*>(at + D));
        const float4 x = __ldcg(reinterpret_cast<const float4*>(at + d));
        const float f = exp2_approx(ml.x - ref);
        sum = fmaf(ml.y, f, sum);
        o.x = fmaf(x.x, f, o.x);
        o.y = fmaf(x.y, f, o.y);
        o.z = fmaf(x.z, f, o.z);
        o.w = fmaf(x.w, f, o.w);
      }
      const float inv = sum == 0.0f ? 0.0f : __fdividef(1.0f, sum);
      const int row = row_first + rr, qi = row / p.group;
      __half2* const dst = reinterpret_cast<__half2*>(
          p.out + (static_cast<long long>(s.row0) + qi) * p.out_token_stride +
          (static_cast<long long>(head) * p.group + (row - qi * p.group)) * D + d);
      dst[0] = __floats2half2_rn(o.x * inv, o.y * inv);
      dst[1] = __floats2half2_rn(o.z * inv, o.w * inv);
    }
  }
}

}  // namespace b200gemm
