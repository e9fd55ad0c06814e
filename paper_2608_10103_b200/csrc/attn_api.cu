// C-ABI of rotary positions and prompt attention (include/b200attn.h): argument checks and launches.
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/b200attn.h"
#include "attention_tiles.cuh"
#include "kv_host.cuh"
#include "rotary.cuh"
#include "shared_state.h"

namespace b200gemm {
namespace {

// Rows of one tensor; `least` is the smallest distance between heads.
int check_rotary_rows(const rotary_rows_t& r, int least) {
  if (!r.x || !r.y || r.heads <= 0 || r.x_head_stride < least || r.y_head_stride < least || r.x_token_stride < 0 ||
      r.y_token_stride < least)
    return GEMM_ERR_INVALID_ARG;
  if (r.x == r.y && (r.x_head_stride != r.y_head_stride || r.x_token_stride != r.y_token_stride)) return GEMM_ERR_INVALID_ARG;
  if (misaligned(r.x, 16) || misaligned(r.y, 16) || r.x_token_stride % 8 || r.x_head_stride % 8 || r.y_token_stride % 8 ||
      r.y_head_stride % 8)
    return GEMM_ERR_MISALIGNED;
  return GEMM_OK;
}

template <int D>
int launch_prompts(const SharedDevice& dev, AttnTilesParams& p, cudaStream_t stream) {
  using T = AttnTileShape<D, false>;
  const int per_tile = 128 / p.group, per_cta = T::QT * per_tile;
  const int longest = p.max_q < p.rows ? p.max_q : p.rows;
  // row tiles: one more a sequence than its rows would fill, and no more than the longest allows
  const long long by_rows = static_cast<long long>(p.rows) / per_cta + p.batch;
  const long long by_longest = (static_cast<long long>(longest) + per_cta - 1) / per_cta * p.batch;
  const long long items = (by_rows < by_longest ? by_rows : by_longest) * p.heads;
  if (items > 0x3fffffffll) return GEMM_ERR_TOO_LARGE;
  p.units = static_cast<int>(items);
  CUtensorMap q, k, v;
  int rc = shared_row_map(&q, p.q, D, p.heads * p.group, p.rows, p.q_token_stride, p.q_head_stride, p.group, per_tile);
  if (rc == GEMM_OK) rc = shared_row_map(&k, p.k, D, p.heads, p.rows, p.kv_token_stride, p.kv_head_stride, 1, T::TN);
  if (rc == GEMM_OK) rc = shared_row_map(&v, p.v, D, p.heads, p.rows, p.kv_token_stride, p.kv_head_stride, 1, T::TN);
  if (rc != GEMM_OK) return rc;
  const int grid = items < dev.num_sms ? static_cast<int>(items) : dev.num_sms;
  return launch_attention_tiles<D, false>(dev, longest, grid, stream, q, k, v, p);
}

}  // namespace
}  // namespace b200gemm

using namespace b200gemm;

extern "C" {

int rotary_fp16(int tokens, int head_dim, int rotary_dim, int pairs, const rotary_rows_t* q,
                const rotary_rows_t* k, const int* positions, int axes, long long axis_stride,
                const int* sections, const float* inv_freq, gemm_stream_t stream) {
  if (tokens <= 0 || head_dim <= 0 || head_dim > 1024 || rotary_dim <= 0 || rotary_dim > head_dim || (!q && !k) ||
      (pairs != ROTARY_HALVES && pairs != ROTARY_NEIGHBOURS) || axes < 1 || axes > ROTARY_AXES || !positions || !inv_freq ||
      (axes > 1 && (!sections || axis_stride < tokens)))
    return GEMM_ERR_INVALID_ARG;
  if (head_dim % 8 || rotary_dim % 16 || misaligned(positions, 4) || misaligned(inv_freq, 4)) return GEMM_ERR_MISALIGNED;
  RotaryParams p = {};
  long long sum = 0;
  for (int a = 0; a < ROTARY_AXES; ++a) {
    const int n = a >= axes ? 0 : axes == 1 && !sections ? rotary_dim / 2 : sections[a];
    if (n < 0) return GEMM_ERR_INVALID_ARG;
    sum += n;
    if (sum > rotary_dim / 2) return GEMM_ERR_INVALID_ARG;
    p.end[a] = static_cast<int>(sum);
  }
  if (sum != rotary_dim / 2) return GEMM_ERR_INVALID_ARG;
  long long heads = 0;
  for (int i = 0; i < 2; ++i) {
    const rotary_rows_t* const r = i ? k : q;
    if (!r) continue;
    const int rc = check_rotary_rows(*r, head_dim);
    if (rc != GEMM_OK) return rc;
    p.rows[i] = {static_cast<const __half*>(r->x), static_cast<__half*>(r->y), r->heads, r->x_token_stride, r->x_head_stride,
                 r->y_token_stride, r->y_head_stride};
    heads += r->heads;
  }
  // (a CTA counts its pieces in 32 bits, and tokens a little beyond the last)
  if (heads * head_dim > (1ll << 26) || tokens > 0x7fffffff - 1024) return GEMM_ERR_TOO_LARGE;
  SharedDevice dev;
  const int rc = shared_device(&dev);
  if (rc != GEMM_OK) return rc;
  p.tokens = tokens;
  p.dim = head_dim;
  p.rotary = rotary_dim;
  p.positions = positions;
  p.axis_stride = axis_stride;
  p.inv_freq = inv_freq;
  // Several tokens a CTA only where that leaves the chip full: one token is what a decoding batch has per SM.
  int per_cta = tokens / (8 * dev.num_sms);
  per_cta = per_cta < 1 ? 1 : per_cta > ROTARY_TOKENS ? ROTARY_TOKENS : per_cta;
  p.per_cta = per_cta;
  const dim3 grid((tokens + per_cta - 1) / per_cta);
  const size_t smem = static_cast<size_t>(per_cta) * rotary_dim * 4;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (pairs == ROTARY_HALVES) return launch(dev, rotary_kernel<true>, grid, ROTARY_THREADS, smem, st, p);
  return launch(dev, rotary_kernel<false>, grid, ROTARY_THREADS, smem, st, p);
}

int attention_fp16(int batch, const int* cu, int max_len, int rows, int q_heads, int kv_heads,
                   int head_dim, const void* Q, long long q_token_stride, long long q_head_stride,
                   const void* K, const void* V, long long kv_token_stride, long long kv_head_stride,
                   float softmax_scale, int causal, int window, void* out,
                   long long out_token_stride, gemm_stream_t stream) {
  if (batch <= 0 || !cu || max_len <= 0 || rows <= 0 || q_heads <= 0 || kv_heads <= 0 || q_heads % kv_heads ||
      (head_dim != 64 && head_dim != 128 && head_dim != 256) || !Q || !K || !V || !out || (causal != 0 && causal != 1) ||
      window < 0 || (window > 0 && !causal) || q_head_stride < head_dim || kv_head_stride < head_dim ||
      q_token_stride < head_dim || kv_token_stride < head_dim || out_token_stride < static_cast<long long>(q_heads) * head_dim ||
      !(softmax_scale > 0.0f && softmax_scale < 1e30f))
    return GEMM_ERR_INVALID_ARG;
  if (misaligned(cu, 4) || misaligned(Q, 16) || misaligned(K, 16) || misaligned(V, 16) || misaligned(out, 16) ||
      q_token_stride % 8 || q_head_stride % 8 || kv_token_stride % 8 || kv_head_stride % 8 || out_token_stride % 8)
    return GEMM_ERR_MISALIGNED;
  const int group = q_heads / kv_heads;
  constexpr long long FAR = 1ll << 38;  // (strides of tensor maps stay below 2^40 bytes)
  if (group > 128 || kv_heads > 65535 || q_token_stride > FAR || q_head_stride > FAR || kv_token_stride > FAR ||
      kv_head_stride > FAR || rows > 0x7fffffff - 1024)
    return GEMM_ERR_TOO_LARGE;
  SharedDevice dev;
  const int rc = shared_device(&dev);
  if (rc != GEMM_OK) return rc;
  AttnTilesParams p = {};
  p.batch = batch;
  p.cu = cu;
  p.max_q = max_len;
  p.rows = rows;
  p.group = group;
  p.heads = kv_heads;
  p.q = static_cast<const __half*>(Q);
  p.q_token_stride = q_token_stride;
  p.q_head_stride = q_head_stride;
  p.k = static_cast<const __half*>(K);
  p.v = static_cast<const __half*>(V);
  p.kv_token_stride = kv_token_stride;
  p.kv_head_stride = kv_head_stride;
  p.out = static_cast<__half*>(out);
  p.out_token_stride = out_token_stride;
  p.scale_log2 = softmax_scale * 1.4426950408889634f;
  p.causal = causal;
  p.window = window;
  p.status = dev.status;
  p.splits = 1;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  switch (head_dim) {
    case 64: return launch_prompts<64>(dev, p, st);
    case 128: return launch_prompts<128>(dev, p, st);
    default: return launch_prompts<256>(dev, p, st);
  }
}

}  // extern "C"
