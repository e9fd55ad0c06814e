// C-ABI of the 4-bit key/value cache (include/b200kv.h): argument checks and launches.
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/b200kv.h"
#include "attention_tiles.cuh"
#include "kv_attention_u4.cuh"
#include "kv_cache_u4.cuh"
#include "kv_host.cuh"
#include "shared_state.h"

namespace b200gemm {
namespace {

int check_cache(const kv_cache_u4_t* c, KvCacheU4View* v) {
  if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale) return GEMM_ERR_INVALID_ARG;
  if (c->num_pages <= 0 || c->kv_heads <= 0 || c->kv_heads > 65535) return GEMM_ERR_INVALID_ARG;
  int shift = 4;
  while (shift < 7 && (1 << shift) != c->page_size) ++shift;
  if ((1 << shift) != c->page_size) return GEMM_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return GEMM_ERR_INVALID_ARG;
  if (misaligned(c->k, 16) || misaligned(c->v, 16) || misaligned(c->k_scale, 16) || misaligned(c->v_scale, 16))
    return GEMM_ERR_MISALIGNED;
  v->codes[0] = c->k;
  v->codes[1] = c->v;
  v->scales[0] = static_cast<__half2*>(c->k_scale);
  v->scales[1] = static_cast<__half2*>(c->v_scale);
  v->num_pages = c->num_pages;
  v->heads = c->kv_heads;
  v->page = c->page_size;
  v->page_shift = shift;
  v->dim = c->head_dim;
  return GEMM_OK;
}

// Blocks of `tokens` tokens of every sequence; 0 = too many.
int blocks_of(int max_rows, int tokens, int batch, int* per_seq) {
  *per_seq = static_cast<int>((static_cast<long long>(max_rows) + tokens - 1) / tokens);
  const long long blocks = static_cast<long long>(*per_seq) * batch;
  return blocks > 0x7fffffffll ? 0 : static_cast<int>(blocks);
}

// Sequences with more than p.split_rows rows, on the tensor cores.
template <int D>
int launch_tiles(const SharedDevice& dev, AttnTilesParams p, cudaStream_t stream) {
  using T = AttnTileShape<D, true>;
  const int per_tile = 128 / p.group, per_cta = T::QT * per_tile;
  const int longest = p.max_q < p.rows ? p.max_q : p.rows;
  // row tiles: one more a sequence than its rows would fill, and no more than the longest allows
  const long long by_rows = static_cast<long long>(p.rows) / per_cta + p.batch;
  const long long by_longest = (static_cast<long long>(longest) + per_cta - 1) / per_cta * p.batch;
  const long long units = (by_rows < by_longest ? by_rows : by_longest) * p.heads;
  if (units > 0x3fffffffll) return GEMM_ERR_TOO_LARGE;
  p.units = static_cast<int>(units);
  CUtensorMap q;
  int rc = shared_row_map(&q, p.q, D, p.heads * p.group, p.rows, p.q_token_stride, p.q_head_stride, p.group, per_tile);
  if (rc != GEMM_OK) return rc;
  // Fewer row tiles than half the SMs: as many parts of their tokens as fill the chip, two token tiles each if
  // sequences are as long as their tables allow, sixteen at most (what is joined grows with them).
  p.splits = 1;
  if (2 * units <= dev.num_sms) {
    long long most = dev.num_sms / units;
    if (most > p.max_len / (2 * T::TN)) most = p.max_len / (2 * T::TN);
    if (most > 16) most = 16;
    if (most > 1) p.splits = static_cast<int>(most);
  }
  const long long items = units * p.splits;
  const int grid = items < dev.num_sms ? static_cast<int>(items) : dev.num_sms;
  if (p.splits == 1) return launch_attention_tiles<D, true>(dev, p.max_len, grid, stream, q, q, q, p);
  SharedLease lease;
  rc = shared_scratch(dev.device, stream, static_cast<size_t>(items) * T::ROWS * (D + 4) * 4,
                      (static_cast<size_t>(units) * 4 + 255) / 256 * 256, &lease);
  if (rc != GEMM_OK) return rc;
  p.arrived = static_cast<unsigned*>(lease.head);
  p.partial = static_cast<float*>(lease.data);
  rc = launch_attention_tiles<D, true>(dev, p.max_len, grid, stream, q, q, q, p);
  const int done = shared_scratch_done(dev.device, stream, lease);
  return rc != GEMM_OK ? rc : done;
}

// Sequences of up to p.split_rows rows.  D: head size, NR: groups of eight rows.
template <int D, int NR>
int launch_few_rows(const SharedDevice& dev, KvAttn4Params p, cudaStream_t stream) {
  static std::atomic<int> resident[MAX_DEV];
  // (1 KB of each CTA is the system's, a few bytes are static)
  constexpr int room = 228 * 1024 / kva4_ctas(D, NR) - 1024 - 64 - kva4_q_bytes(D, NR);
  constexpr int slots = room / (KVA_WARPS * kva4_slot_bytes(D));
  constexpr int depth = slots < 8 ? slots : 8;
  static_assert(depth >= 2, "the ring holds two steps at least");
  constexpr int smem = kva4_smem(D, NR, depth);
  auto kernel = kv_attention_u4_kernel<D, NR, depth>;
  int per_sm = resident[dev.device].load();
  if (per_sm == 0) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, KVA_THREADS, smem);
    if (e != cudaSuccess) return shared_cuda_fail(e);
    if (per_sm < 1) return shared_cuda_fail(cudaErrorLaunchOutOfResources);
    resident[dev.device].store(per_sm);
  }
  p.min_share = 4;
  const int grid = per_sm * dev.num_sms;
  const size_t counters = static_cast<size_t>(p.batch) * p.c.heads * 4;
  const size_t bytes = 2ull * grid * kva_rows_floats(8 * NR, D) * 4;
  SharedLease lease;
  int rc = shared_scratch(dev.device, stream, bytes, (counters + 255) / 256 * 256, &lease);
  if (rc != GEMM_OK) return rc;
  p.arrived = static_cast<unsigned*>(lease.head);
  p.partial = static_cast<float*>(lease.data);
  rc = launch(dev, kernel, dim3(grid), KVA_THREADS, smem, stream, p);
  const int done = shared_scratch_done(dev.device, stream, lease);
  return rc != GEMM_OK ? rc : done;
}

// Most rows of a sequence that the few-rows kernel takes, two groups of eight. The tile kernel gives each such sequence row tiles of 128
// rows by itself: 64 sequences of 4096 tokens with 9 to 16 rows for each of 8 KV heads take 73-75, 108-112 and 231-240 us (64, 128, 256 d) against
// 337, 405 and 569; one of 1000 tokens with 9 rows 13.8 against 23.9. There is no form of more than two groups: 17 rows cost what 127 do.
constexpr int FEW_ROWS = 16;

template <int D>
int attention(const SharedDevice& dev, AttnTilesParams& p, cudaStream_t stream) {
  const long long most = static_cast<long long>(p.max_q < p.rows ? p.max_q : p.rows) * p.group;
  p.split_rows = FEW_ROWS;
  // The few-rows kernel counts the steps of all sequences in 32 bits.
  const long long steps = static_cast<long long>(p.max_len) / kva4_step(D) + 1 + kva4_unit_cost(D);
  if (most + p.group + 512 >= (1ll << 31) || static_cast<long long>(p.batch) * p.heads >= (1ll << 30) / steps)
    return GEMM_ERR_TOO_LARGE;
  if (most > FEW_ROWS) {
    const int rc = launch_tiles<D>(dev, p, stream);
    if (rc != GEMM_OK || p.group > FEW_ROWS) return rc;
  }
  KvAttn4Params few = {};
  few.c = p.c;
  few.batch = p.batch;
  few.cu = p.cu;
  few.kv_len = p.kv_len;
  few.table = p.table;
  few.table_stride = p.table_stride;
  few.max_q = p.max_q;
  few.rows = p.rows;
  few.max_len = p.max_len;
  few.group = p.group;
  few.q = p.q;
  few.q_token_stride = p.q_token_stride;
  few.q_head_stride = p.q_head_stride;
  few.out = p.out;
  few.out_token_stride = p.out_token_stride;
  few.scale_log2 = p.scale_log2;
  few.window = p.window;
  few.split_rows = p.split_rows;
  few.status = p.status;
  // One group of eight rows where the call's bounds exclude a second, whose work would be done for nothing: 64 single tokens of 4 rows over up
  // to 8192 tokens 75 us with max_q = 1, 105 with max_q = 4 (140 and 235 at 256 d).
  return most <= 8 ? launch_few_rows<D, 1>(dev, few, stream) : launch_few_rows<D, 2>(dev, few, stream);
}

}  // namespace
}  // namespace b200gemm

using namespace b200gemm;

extern "C" {

int kv_append_u4(const kv_cache_u4_t* cache, int batch, const int* cu, const int* past,
                 const int* block_table, int table_stride, int max_new, const void* K,
                 const void* V, long long token_stride, long long head_stride, int rows,
                 gemm_stream_t stream) {
  KvAppendU4Params p = {};
  int rc = check_cache(cache, &p.c);
  if (rc == GEMM_OK) rc = check_batch(batch, cu, past, block_table, table_stride, max_new, rows, &p.b);
  if (rc != GEMM_OK) return rc;
  if (!K || !V || token_stride < 0 || head_stride < p.c.dim) return GEMM_ERR_INVALID_ARG;
  if (misaligned(K, 16) || misaligned(V, 16) || token_stride % 8 || head_stride % 8)
    return GEMM_ERR_MISALIGNED;
  const int blocks = blocks_of(max_new < rows ? max_new : rows, kv4_tokens(p.c.dim), batch, &p.blocks_per_seq);
  if (!blocks) return GEMM_ERR_TOO_LARGE;
  SharedDevice dev;
  rc = shared_device(&dev);
  if (rc != GEMM_OK) return rc;
  p.b.status = dev.status;
  p.x[0] = static_cast<const __half*>(K);
  p.x[1] = static_cast<const __half*>(V);
  p.token_stride = token_stride;
  p.head_stride = head_stride;
  const dim3 grid(static_cast<unsigned>(blocks), 2);
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  switch (p.c.dim) {
    case 64: return launch(dev, kv_append_u4_kernel<64>, grid, KV4_THREADS, 0, st, p);
    case 128: return launch(dev, kv_append_u4_kernel<128>, grid, KV4_THREADS, 0, st, p);
    default: return launch(dev, kv_append_u4_kernel<256>, grid, KV4_THREADS, 0, st, p);
  }
}

int kv_read_u4(const kv_cache_u4_t* cache, int batch, const int* cu, const int* first,
               const int* block_table, int table_stride, int max_read, void* K, void* V, int rows,
               gemm_stream_t stream) {
  KvReadU4Params p = {};
  int rc = check_cache(cache, &p.c);
  if (rc == GEMM_OK) rc = check_batch(batch, cu, first, block_table, table_stride, max_read, rows, &p.b);
  if (rc != GEMM_OK) return rc;
  if (!K && !V) return GEMM_ERR_INVALID_ARG;
  if (misaligned(K, 16) || misaligned(V, 16)) return GEMM_ERR_MISALIGNED;
  const int blocks = blocks_of(max_read < rows ? max_read : rows, kv4_tokens(p.c.dim), batch, &p.blocks_per_seq);
  if (!blocks) return GEMM_ERR_TOO_LARGE;
  SharedDevice dev;
  rc = shared_device(&dev);
  if (rc != GEMM_OK) return rc;
  p.b.status = dev.status;
  p.out[0] = static_cast<__half*>(K);
  p.out[1] = static_cast<__half*>(V);
  const dim3 grid(static_cast<unsigned>(blocks), 2);
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  switch (p.c.dim) {
    case 64: return launch(dev, kv_read_u4_kernel<64>, grid, KV4_THREADS, 0, st, p);
    case 128: return launch(dev, kv_read_u4_kernel<128>, grid, KV4_THREADS, 0, st, p);
    default: return launch(dev, kv_read_u4_kernel<256>, grid, KV4_THREADS, 0, st, p);
  }
}

int kv_attention_u4(const kv_cache_u4_t* cache, int batch, const int* cu, const int* kv_len,
                    const int* block_table, int table_stride, int max_q, int q_heads,
                    const void* Q, long long q_token_stride, long long q_head_stride,
                    float softmax_scale, int window, void* out, long long out_token_stride,
                    int rows, gemm_stream_t stream) {
  AttnTilesParams p = {};
  KvBatch b;
  int rc = check_cache(cache, &p.c);
  if (rc == GEMM_OK) rc = check_batch(batch, cu, kv_len, block_table, table_stride, max_q, rows, &b);
  if (rc != GEMM_OK) return rc;
  if (!Q || !out || q_heads <= 0 || q_heads % p.c.heads || window < 0 || q_token_stride < p.c.dim ||
      q_head_stride < p.c.dim || out_token_stride < static_cast<long long>(q_heads) * p.c.dim ||
      !(softmax_scale > 0.0f && softmax_scale < 1e30f))
    return GEMM_ERR_INVALID_ARG;
  if (misaligned(Q, 16) || misaligned(out, 16) || q_token_stride % 8 || q_head_stride % 8 ||
      out_token_stride % 8)
    return GEMM_ERR_MISALIGNED;
  p.group = q_heads / p.c.heads;
  constexpr long long FAR = 1ll << 38;  // (strides of tensor maps stay below 2^40 bytes)
  if (p.group > 128 || q_token_stride > FAR || q_head_stride > FAR || rows > 0x7fffffff - 1024) return GEMM_ERR_TOO_LARGE;
  SharedDevice dev;
  rc = shared_device(&dev);
  if (rc != GEMM_OK) return rc;
  p.batch = batch;
  p.cu = cu;
  p.kv_len = kv_len;
  p.table = block_table;
  p.table_stride = table_stride;
  p.max_q = max_q;
  p.rows = rows;
  p.heads = p.c.heads;
  p.q = static_cast<const __half*>(Q);
  p.q_token_stride = q_token_stride;
  p.q_head_stride = q_head_stride;
  p.out = static_cast<__half*>(out);
  p.out_token_stride = out_token_stride;
  p.scale_log2 = softmax_scale * 1.4426950408889634f;
  p.causal = 1;
  p.window = window;
  p.status = dev.status;
  const long long max_len = static_cast<long long>(table_stride) * p.c.page;
  p.max_len = max_len < 0x7fffffff - 256 ? static_cast<int>(max_len) : 0x7fffffff - 256;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  switch (p.c.dim) {
    case 64: return attention<64>(dev, p, st);
    case 128: return attention<128>(dev, p, st);
    default: return attention<256>(dev, p, st);
  }
}

}  // extern "C"
