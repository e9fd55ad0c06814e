// INT8 key/value cache: writing new tokens and reading tokens back (see include/b200kv.h for the
// layout and the definition of the scales).
//
// Writing.  One CTA owns one (page, head, K or V): it sees every new token of the page, so the
// page's scale needs no atomics and the result no order.  A thread keeps its pieces of eight values
// in registers between the maximum and the codes: a page is read once and written once.  Only the
// first page a call touches can hold older tokens; its old codes are fetched along with the new
// values (latency, not bytes, is what a single-token call is made of) and rewritten only if the
// scale grew.  Everything else is bound by 2 bytes read and 1 written per value.
//
// Reading back.  One thread per 16 codes: 16 bytes in, 32 out.
//
// Measured: 4 x 8192 tokens of 8 heads of 128 d written in 34 us and 4 x 9192 read back in 33 us, together 0.75 of the copy
// rate; 64 sequences of one token 5 us each way, which is a launch and three dependent loads.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

#include "ptx.cuh"

namespace b200gemm {

constexpr int DEV_BAD_INDEX = 6;  // status word: a length, count or page id outside its range

struct KvCacheView {
  int8_t* codes[2];  // K, V
  float* scales[2];
  int num_pages, heads, page, page_shift, dim;
};

struct KvBatch {
  int batch;
  const int* cu;       // rows of the packed arrays
  const int* start;    // past (append), first (read)
  const int* table;
  int table_stride;    // entries per sequence
  int max_rows;        // upper bound of rows per sequence
  int rows;            // rows of the packed arrays
  int* status;
};

__device__ __forceinline__ int kv_ld(const int* p) {  // may have been written by the grid in front
  int v;
  asm volatile("ld.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void kv_report(int* status) { atomicCAS(status, 0, DEV_BAD_INDEX); }

// Rows and positions of a sequence, cut to what the packed arrays, the table and the caller's bound allow.
struct KvRange {
  int row0;   // first row in the packed arrays
  int begin;  // first position
  int end;    // one past the last
};
__device__ __forceinline__ KvRange kv_range(const KvBatch& b, int seq, int page, bool report) {
  KvRange r;
  r.row0 = kv_ld(b.cu + seq);
  long long n = static_cast<long long>(kv_ld(b.cu + seq + 1)) - r.row0;
  long long first = kv_ld(b.start + seq);
  const long long room = min(static_cast<long long>(b.table_stride) * page, 0x7fffffffll);
  bool bad = n < 0 || n > b.max_rows || first < 0 || r.row0 < 0 || r.row0 + n > b.rows;
  n = min(n, min(static_cast<long long>(b.max_rows), static_cast<long long>(b.rows) - r.row0));
  if (n < 0 || first < 0 || r.row0 < 0) n = first = 0;
  if (n > 0 && first + n > room) {
    bad = true;
    n = room > first ? room - first : 0;
  }
  if (bad && report) kv_report(b.status);
  r.begin = static_cast<int>(first);
  r.end = static_cast<int>(first + n);
  return r;
}

struct KvAppendParams {
  KvCacheView c;
  KvBatch b;
  const __half* x[2];
  long long token_stride, head_stride;
  int pages_per_seq;  // upper bound of pages a sequence touches
};

constexpr int KV_APPEND_PIECES = 8;

// grid: (batch * pages_per_seq, heads, 2); threads: page * dim / 64 (at least 32).
__global__ void __launch_bounds__(512) kv_append_kernel(const KvAppendParams p) {
  __shared__ uint32_t warp_max[16];
  if (threadIdx.x == 0) ptx::grid_dep_launch_dependents();
  const int seq = static_cast<int>(blockIdx.x) / p.pages_per_seq;
  const int nth = static_cast<int>(blockIdx.x) % p.pages_per_seq;
  const int head = static_cast<int>(blockIdx.y), which = static_cast<int>(blockIdx.z);
  const bool lead = threadIdx.x == 0;
  ptx::grid_dep_wait();
  const KvRange r = kv_range(p.b, seq, p.c.page, lead && nth == 0 && head == 0 && which == 0);
  if (r.begin >= r.end) return;
  const int index = (r.begin >> p.c.page_shift) + nth;
  const int pos0 = index << p.c.page_shift;
  if (pos0 >= r.end) return;
  // the page's id is on its way while the new values are asked for, which do not need it
  const int slot = kv_ld(p.b.table + static_cast<long long>(seq) * p.b.table_stride + index);
  const int per_row = p.c.dim / 8, pieces = p.c.page * per_row;
  const __half* const src = (which ? p.x[1] : p.x[0]) +
                            (static_cast<long long>(r.row0) + (pos0 - r.begin)) * p.token_stride + head * p.head_stride;
  uint4 x[KV_APPEND_PIECES];  // eight new binary16 values, or in .x, .y eight old codes
  int pos[KV_APPEND_PIECES];  // token of the piece; -1 = none
#pragma unroll
  for (int i = 0; i < KV_APPEND_PIECES; ++i) {
    const int piece = static_cast<int>(threadIdx.x) + i * static_cast<int>(blockDim.x);
    const int row = piece / per_row;
    pos[i] = piece < pieces && pos0 + row < r.end ? pos0 + row : -1;
    x[i] = make_uint4(0, 0, 0, 0);
    if (pos[i] >= r.begin) x[i] = ptx::ld_global_stream_v4(src + row * p.token_stride + (piece - row * per_row) * 8);
  }
  if (slot < 0 || slot >= p.c.num_pages) {
    if (lead) kv_report(p.b.status);
    return;
  }
  const long long page_head = static_cast<long long>(slot) * p.c.heads + head;
  int8_t* const codes = (which ? p.c.codes[1] : p.c.codes[0]) + page_head * p.c.page * p.c.dim;
  float* const scale_at = (which ? p.c.scales[1] : p.c.scales[0]) + page_head;
  const bool has_old = pos0 < r.begin;
  const float was = has_old ? ptx::ld_global_f32(scale_at) : 0.0f;
  uint32_t m2 = 0;  // two maxima of magnitude bits: infinities and NaN compare above every finite value
#pragma unroll
  for (int i = 0; i < KV_APPEND_PIECES; ++i) {
    const int piece = static_cast<int>(threadIdx.x) + i * static_cast<int>(blockDim.x);
    if (has_old && pos[i] >= 0 && pos[i] < r.begin)
      asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(x[i].x), "=r"(x[i].y) : "l"(codes + piece * 8) : "memory");
  }
#pragma unroll
  for (int i = 0; i < KV_APPEND_PIECES; ++i)
    if (pos[i] >= r.begin)
      m2 = __vmaxu2(m2, __vmaxu2(__vmaxu2(x[i].x & 0x7fff7fffu, x[i].y & 0x7fff7fffu),
                                 __vmaxu2(x[i].z & 0x7fff7fffu, x[i].w & 0x7fff7fffu)));
  uint32_t m = __reduce_max_sync(0xffffffffu, max(m2 & 0xffffu, m2 >> 16));
  if (blockDim.x > 32) {
    if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = m;
    __syncthreads();
    const int warps = static_cast<int>(blockDim.x) >> 5;
    for (int w = 0; w < warps; ++w) m = max(m, warp_max[w]);
  }
  const float fresh = __fdiv_rn(__half2float(__ushort_as_half(static_cast<unsigned short>(m))), 127.0f);
  const float now = (fresh > was || fresh != fresh) ? fresh : was;  // a NaN on either side stays
  const float inverse = now == 0.0f ? 0.0f : __fdiv_rn(1.0f, now);
  const float ratio = was * inverse;
  const bool grew = has_old && !(now == was);
  // (every thread has read the old scale: a value that each used above or, with several warps, behind the barrier)
  if (blockDim.x > 32 && has_old) __syncthreads();
  if (lead) *scale_at = now;
#pragma unroll
  for (int i = 0; i < KV_APPEND_PIECES; ++i) {
    const int piece = static_cast<int>(threadIdx.x) + i * static_cast<int>(blockDim.x);
    if (pos[i] < 0 || (pos[i] < r.begin && !grew)) continue;
    float v[8];
    if (pos[i] >= r.begin) {
      const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
        v[2 * j] = f.x * inverse;
        v[2 * j + 1] = f.y * inverse;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        v[j] = static_cast<float>(static_cast<int8_t>((j < 4 ? x[i].x : x[i].y) >> (8 * (j & 3)))) * ratio;
    }
    uint2 out;
    uint32_t c[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) c[j] = static_cast<uint32_t>(__float2int_rn(v[j])) & 255u;
    out.x = c[0] | (c[1] << 8) | (c[2] << 16) | (c[3] << 24);
    out.y = c[4] | (c[5] << 8) | (c[6] << 16) | (c[7] << 24);
    *reinterpret_cast<uint2*>(codes + piece * 8) = out;
  }
}

struct KvReadParams {
  KvCacheView c;
  KvBatch b;
  __half* out[2];
  int blocks_per_seq;
};

constexpr int KV_READ_TOKENS = 16;  // tokens per CTA
constexpr int KV_READ_THREADS = 256;
constexpr int KV_READ_UNITS = 4;    // 16-byte pieces a thread has in flight

// grid: (batch * blocks_per_seq, 2)
__global__ void __launch_bounds__(KV_READ_THREADS) kv_read_kernel(const KvReadParams p) {
  if (threadIdx.x == 0) ptx::grid_dep_launch_dependents();
  const int seq = static_cast<int>(blockIdx.x) / p.blocks_per_seq;
  const int nth = static_cast<int>(blockIdx.x) % p.blocks_per_seq;
  const int which = static_cast<int>(blockIdx.y);
  ptx::grid_dep_wait();
  __half* const out = which ? p.out[1] : p.out[0];
  if (!out) return;
  const KvRange r = kv_range(p.b, seq, p.c.page, threadIdx.x == 0 && nth == 0);
  const int t0 = nth * KV_READ_TOKENS;
  const int tokens = min(KV_READ_TOKENS, r.end - r.begin - t0);
  if (tokens <= 0) return;
  const int per_head = p.c.dim / 16, per_token = p.c.heads * per_head;
  const int* const table = p.b.table + static_cast<long long>(seq) * p.b.table_stride;
  const int8_t* const codes = which ? p.c.codes[1] : p.c.codes[0];
  const float* const scales = which ? p.c.scales[1] : p.c.scales[0];
  const int units = tokens * per_token;
#pragma unroll 1
  for (int first = static_cast<int>(threadIdx.x); first < units; first += KV_READ_UNITS * KV_READ_THREADS) {
    // the ids of all pieces, then their codes and scales, then the results: three latencies for all
    int slot[KV_READ_UNITS], pos[KV_READ_UNITS], head[KV_READ_UNITS], rest[KV_READ_UNITS];
    uint4 q[KV_READ_UNITS];
    float s[KV_READ_UNITS];
#pragma unroll
    for (int i = 0; i < KV_READ_UNITS; ++i) {
      const int u = first + i * KV_READ_THREADS;
      const int t = u / per_token;
      rest[i] = u - t * per_token;
      head[i] = rest[i] / per_head;
      pos[i] = u < units ? t : -1;
      slot[i] = -1;
      if (u < units) slot[i] = kv_ld(table + ((r.begin + t0 + t) >> p.c.page_shift));
    }
#pragma unroll
    for (int i = 0; i < KV_READ_UNITS; ++i) {
      q[i] = make_uint4(0, 0, 0, 0);
      s[i] = 0.0f;
      if (slot[i] < 0 || slot[i] >= p.c.num_pages) {
        if (pos[i] >= 0) kv_report(p.b.status);
        continue;
      }
      const long long page_head = static_cast<long long>(slot[i]) * p.c.heads + head[i];
      q[i] = ptx::ld_global_stream_v4(codes + (page_head * p.c.page + ((r.begin + t0 + pos[i]) & (p.c.page - 1))) * p.c.dim +
                                      (rest[i] - head[i] * per_head) * 16);
      s[i] = ptx::ld_global_f32(scales + page_head);
    }
#pragma unroll
    for (int i = 0; i < KV_READ_UNITS; ++i) {
      if (pos[i] < 0) continue;
      const uint32_t w[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
      uint32_t h[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float a = static_cast<float>(static_cast<int8_t>(w[j / 2] >> (16 * (j & 1)))) * s[i];
        const float b = static_cast<float>(static_cast<int8_t>(w[j / 2] >> (16 * (j & 1) + 8))) * s[i];
        const __half2 x = __floats2half2_rn(a, b);
        h[j] = *reinterpret_cast<const uint32_t*>(&x);
      }
      // rows of a token are dense: heads x dim
      uint4* const dst = reinterpret_cast<uint4*>(
          out + ((static_cast<long long>(r.row0) + t0 + pos[i]) * per_token + rest[i]) * 16);
      dst[0] = make_uint4(h[0], h[1], h[2], h[3]);
      dst[1] = make_uint4(h[4], h[5], h[6], h[7]);
    }
  }
}

}  // namespace b200gemm
