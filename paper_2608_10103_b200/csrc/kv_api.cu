// C-ABI of the INT8 key/value cache (include/b200kv.h): argument checks and launches.
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/b200kv.h"
#include "kv_attention.cuh"
#include "kv_attention_tiles.cuh"
#include "kv_cache.cuh"
#include "shared_state.h"

namespace b200gemm {
namespace {

bool misaligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

int check_cache(const kv_cache_s8_t* c, KvCacheView* v) {
  if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale) return GEMM_ERR_INVALID_ARG;
  if (c->num_pages <= 0 || c->kv_heads <= 0 || c->kv_heads > 65535) return GEMM_ERR_INVALID_ARG;
  int shift = 4;
  while (shift < 7 && (1 << shift) != c->page_size) ++shift;
  if ((1 << shift) != c->page_size) return GEMM_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return GEMM_ERR_INVALID_ARG;
  if (misaligned(c->k, 16) || misaligned(c->v, 16) || misaligned(c->k_scale, 4) || misaligned(c->v_scale, 4))
    return GEMM_ERR_MISALIGNED;
  v->codes[0] = c->k;
  v->codes[1] = c->v;
  v->scales[0] = c->k_scale;
  v->scales[1] = c->v_scale;
  v->num_pages = c->num_pages;
  v->heads = c->kv_heads;
  v->page = c->page_size;
  v->page_shift = shift;
  v->dim = c->head_dim;
  return GEMM_OK;
}

int check_batch(int batch, const int* cu, const int* start, const int* table, int table_stride,
                int max_rows, int rows, KvBatch* b) {
  if (batch <= 0 || !cu || !start || !table || table_stride <= 0 || max_rows <= 0 || rows <= 0)
    return GEMM_ERR_INVALID_ARG;
  if (misaligned(cu, 4) || misaligned(start, 4) || misaligned(table, 4)) return GEMM_ERR_MISALIGNED;
  b->batch = batch;
  b->cu = cu;
  b->start = start;
  b->table = table;
  b->table_stride = table_stride;
  b->max_rows = max_rows;
  b->rows = rows;
  return GEMM_OK;
}

template <class Kernel, class Params>
int launch(const SharedDevice& dev, Kernel kernel, dim3 grid, int threads, size_t smem,
           cudaStream_t stream, const Params& p) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(static_cast<unsigned>(threads));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = dev.plain_order ? 0 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, p);
  return e == cudaSuccess ? GEMM_OK : shared_cuda_fail(e);
}

constexpr int MAX_DEV = 64;
constexpr int ANY_ROWS = 0x7fffffff;  // the entry points without a row count

// D: head size, NR: groups of eight rows per tile.
template <int D, int NR>
int launch_attention(const SharedDevice& dev, KvAttnParams& p, cudaStream_t stream) {
  static std::atomic<int> resident[MAX_DEV];
  constexpr int room = 227 * 1024 / kva_ctas(D, NR) - 2048 - kva_q_bytes(D, NR);
  constexpr int slots = room / (KVA_WARPS * kva_slot_bytes(D));
  constexpr int depth = slots < 8 ? slots : 8;
  static_assert(depth >= 2, "the ring holds two steps at least");
  constexpr int smem = kva_smem(D, NR, depth);
  auto kernel = kv_attention_kernel<D, NR, depth>;
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
  const int rows = 8 * NR;
  const long long most = static_cast<long long>(p.max_q) * p.group;
  const long long tiles = ((most < p.split_rows ? most : p.split_rows) + rows - 1) / rows;
  p.max_tiles = static_cast<int>(tiles);
  const size_t counters = static_cast<size_t>(p.batch) * tiles * p.c.heads * 4;
  const size_t bytes = 2ull * grid * kva_rows_floats(rows, D) * 4;
  SharedLease lease;
  int rc = shared_scratch(dev.device, stream, bytes, (counters + 255) / 256 * 256, &lease);
  if (rc != GEMM_OK) return rc;
  p.arrived = static_cast<unsigned*>(lease.head);
  p.partial = static_cast<float*>(lease.data);
  rc = launch(dev, kernel, dim3(grid), KVA_THREADS, smem, stream, p);
  const int done = shared_scratch_done(dev.device, stream, lease);
  return rc != GEMM_OK ? rc : done;
}

// Sequences with more than p.split_rows rows, on the tensor cores.
template <int D>
int launch_attention_tiles(const SharedDevice& dev, KvAttnParams p, cudaStream_t stream) {
  static std::atomic<bool> ready[MAX_DEV];
  using T = KvTileShape<D>;
  auto kernel = kv_attention_tiles_kernel<D>;
  if (!ready[dev.device].load()) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, T::DYN_BYTES);
    if (e != cudaSuccess) return shared_cuda_fail(e);
    ready[dev.device].store(true);
  }
  const long long tiles = (static_cast<long long>(p.max_q) * p.group + T::ROWS - 1) / T::ROWS;
  const long long blocks = tiles * p.c.heads * p.batch;
  if (blocks > 0x7fffffffll) return GEMM_ERR_TOO_LARGE;
  // Fewer row tiles than half the SMs: as many parts of their tokens as fill the chip, two token tiles each if
  // sequences are as long as their tables allow, sixteen at most (what is joined grows with them).
  p.splits = 1;
  if (2 * blocks <= dev.num_sms) {
    long long most = dev.num_sms / blocks;
    if (most > p.max_len / (2 * T::TN)) most = p.max_len / (2 * T::TN);
    if (most > 16) most = 16;
    if (most > 1) p.splits = static_cast<int>(most);
  }
  // Sums of long sequences: one CTA is resident per SM (its registers are all of them), so as many slots do.
  const bool long_sums = p.max_len > T::SUM_TILES * T::TN;
  if (p.splits == 1 && !long_sums)
    return launch(dev, kernel, dim3(static_cast<unsigned>(blocks)), T::THREADS, T::DYN_BYTES, stream, p);
  const size_t parts = p.splits > 1 ? static_cast<size_t>(blocks) * p.splits * T::ROWS * (D + 4) * 4 : 0;
  const size_t counters = p.splits > 1 ? static_cast<size_t>(blocks) : 0;
  p.slots = long_sums ? dev.num_sms : 0;
  SharedLease lease;
  const int rc = shared_scratch(dev.device, stream, parts + static_cast<size_t>(p.slots) * T::ROWS * D * 4,
                                ((counters + p.slots) * 4 + 255) / 256 * 256, &lease);
  if (rc != GEMM_OK) return rc;
  p.arrived = static_cast<unsigned*>(lease.head);
  p.partial = static_cast<float*>(lease.data);
  if (long_sums) {
    p.taken = p.arrived + counters;
    p.long_sums = p.partial + parts / 4;
  }
  const int launched = launch(dev, kernel, dim3(static_cast<unsigned>(blocks * p.splits)), T::THREADS, T::DYN_BYTES, stream, p);
  const int done = shared_scratch_done(dev.device, stream, lease);
  return launched != GEMM_OK ? launched : done;
}

template <int D, int MAX_NR>
int attention(const SharedDevice& dev, KvAttnParams& p, cudaStream_t stream) {
  const long long rows = static_cast<long long>(p.max_q) * p.group;
  p.split_rows = 8 * MAX_NR;
  KvAttnParams few = p;
  const long long bound = rows < p.split_rows ? rows : p.split_rows;
  // The few-rows kernel takes a sequence's rows as one tile (its width goes by this bound) and counts the steps of
  // 16 tokens of all of them in 32 bits.
  const long long steps = static_cast<long long>(p.max_len) / KVA_STEP + 1 + KVA_UNIT_COST;
  if (rows + p.group + 512 >= (1ll << 31) || static_cast<long long>(p.batch) * p.c.heads >= (1ll << 30) / steps)
    return GEMM_ERR_TOO_LARGE;
  if (rows > p.split_rows) {
    const int rc = launch_attention_tiles<D>(dev, p, stream);
    if (rc != GEMM_OK) return rc;
  }
  if (bound <= 8) return launch_attention<D, 1>(dev, few, stream);
  if (bound <= 16 || MAX_NR == 2) return launch_attention<D, 2>(dev, few, stream);
  return launch_attention<D, MAX_NR>(dev, few, stream);
}

}  // namespace
}  // namespace b200gemm

using namespace b200gemm;

extern "C" {

int kv_append_s8_rows(const kv_cache_s8_t* cache, int batch, const int* cu, const int* past,
                      const int* block_table, int table_stride, int max_new, const void* K,
                      const void* V, long long token_stride, long long head_stride, int rows,
                      gemm_stream_t stream) {
  KvAppendParams p = {};
  int rc = check_cache(cache, &p.c);
  if (rc == GEMM_OK) rc = check_batch(batch, cu, past, block_table, table_stride, max_new, rows, &p.b);
  if (rc != GEMM_OK) return rc;
  if (!K || !V || token_stride < 0 || head_stride < p.c.dim) return GEMM_ERR_INVALID_ARG;
  if (misaligned(K, 16) || misaligned(V, 16) || token_stride % 8 || head_stride % 8)
    return GEMM_ERR_MISALIGNED;
  SharedDevice dev;
  rc = shared_device(&dev);
  if (rc != GEMM_OK) return rc;
  p.b.status = dev.status;
  p.x[0] = static_cast<const __half*>(K);
  p.x[1] = static_cast<const __half*>(V);
  p.token_stride = token_stride;
  p.head_stride = head_stride;
  const long long pages = (static_cast<long long>(max_new) + p.c.page - 2) / p.c.page + 1;
  p.pages_per_seq = static_cast<int>(pages < table_stride ? pages : table_stride);
  const long long blocks = static_cast<long long>(p.pages_per_seq) * batch;
  if (blocks > 0x7fffffffll) return GEMM_ERR_TOO_LARGE;
  int threads = p.c.page * p.c.dim / (8 * KV_APPEND_PIECES);
  if (threads < 32) threads = 32;
  return launch(dev, kv_append_kernel, dim3(static_cast<unsigned>(blocks), p.c.heads, 2), threads, 0,
                reinterpret_cast<cudaStream_t>(stream), p);
}

int kv_append_s8(const kv_cache_s8_t* cache, int batch, const int* cu, const int* past,
                 const int* block_table, int table_stride, int max_new, const void* K,
                 const void* V, long long token_stride, long long head_stride,
                 gemm_stream_t stream) {
  return kv_append_s8_rows(cache, batch, cu, past, block_table, table_stride, max_new, K, V, token_stride,
                           head_stride, ANY_ROWS, stream);
}

int kv_read_s8_rows(const kv_cache_s8_t* cache, int batch, const int* cu, const int* first,
                    const int* block_table, int table_stride, int max_read, void* K, void* V,
                    int rows, gemm_stream_t stream) {
  KvReadParams p = {};
  int rc = check_cache(cache, &p.c);
  if (rc == GEMM_OK) rc = check_batch(batch, cu, first, block_table, table_stride, max_read, rows, &p.b);
  if (rc != GEMM_OK) return rc;
  if (!K && !V) return GEMM_ERR_INVALID_ARG;
  if (misaligned(K, 16) || misaligned(V, 16)) return GEMM_ERR_MISALIGNED;
  SharedDevice dev;
  rc = shared_device(&dev);
  if (rc != GEMM_OK) return rc;
  p.b.status = dev.status;
  p.out[0] = static_cast<__half*>(K);
  p.out[1] = static_cast<__half*>(V);
  p.blocks_per_seq = static_cast<int>((static_cast<long long>(max_read) + KV_READ_TOKENS - 1) / KV_READ_TOKENS);
  const long long blocks = static_cast<long long>(p.blocks_per_seq) * batch;
  if (blocks > 0x7fffffffll) return GEMM_ERR_TOO_LARGE;
  return launch(dev, kv_read_kernel, dim3(static_cast<unsigned>(blocks), 2), KV_READ_THREADS, 0,
                reinterpret_cast<cudaStream_t>(stream), p);
}

int kv_read_s8(const kv_cache_s8_t* cache, int batch, const int* cu, const int* first,
               const int* block_table, int table_stride, int max_read, void* K, void* V,
               gemm_stream_t stream) {
  return kv_read_s8_rows(cache, batch, cu, first, block_table, table_stride, max_read, K, V, ANY_ROWS, stream);
}

int kv_attention_s8_rows(const kv_cache_s8_t* cache, int batch, const int* cu, const int* kv_len,
                         const int* block_table, int table_stride, int max_q, int q_heads,
                         const void* Q, long long q_token_stride, long long q_head_stride,
                         float softmax_scale, int window, void* out, long long out_token_stride,
                         int rows, gemm_stream_t stream) {
  KvAttnParams p = {};
  KvBatch b;
  int rc = check_cache(cache, &p.c);
  if (rc == GEMM_OK) rc = check_batch(batch, cu, kv_len, block_table, table_stride, max_q, rows, &b);
  if (rc != GEMM_OK) return rc;
  if (!Q || !out || q_heads <= 0 || q_heads % p.c.heads || window < 0 || q_token_stride < 0 ||
      q_head_stride < p.c.dim || out_token_stride < static_cast<long long>(q_heads) * p.c.dim ||
      !(softmax_scale > 0.0f && softmax_scale < 1e30f))
    return GEMM_ERR_INVALID_ARG;
  if (misaligned(Q, 16) || misaligned(out, 16) || q_token_stride % 8 || q_head_stride % 8 ||
      out_token_stride % 8)
    return GEMM_ERR_MISALIGNED;
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
  p.group = q_heads / p.c.heads;
  p.q = static_cast<const __half*>(Q);
  p.q_token_stride = q_token_stride;
  p.q_head_stride = q_head_stride;
  p.out = static_cast<__half*>(out);
  p.out_token_stride = out_token_stride;
  p.scale_log2 = softmax_scale * 1.4426950408889634f;
  p.window = window;
  p.status = dev.status;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const long long max_len = static_cast<long long>(table_stride) * p.c.page;
  p.max_len = max_len < 0x7fffffff - 256 ? static_cast<int>(max_len) : 0x7fffffff - 256;
  switch (p.c.dim) {
    case 64: return attention<64, 4>(dev, p, st);
    case 128: return attention<128, 4>(dev, p, st);
    default: return attention<256, 2>(dev, p, st);
  }
}

int kv_attention_s8(const kv_cache_s8_t* cache, int batch, const int* cu, const int* kv_len,
                    const int* block_table, int table_stride, int max_q, int q_heads,
                    const void* Q, long long q_token_stride, long long q_head_stride,
                    float softmax_scale, int window, void* out, long long out_token_stride,
                    gemm_stream_t stream) {
  return kv_attention_s8_rows(cache, batch, cu, kv_len, block_table, table_stride, max_q, q_heads, Q,
                              q_token_stride, q_head_stride, softmax_scale, window, out, out_token_stride,
                              ANY_ROWS, stream);
}

}  // extern "C"
