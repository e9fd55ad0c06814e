// Key/value cache in 4 bits: writing new tokens and reading tokens back (see include/b200kv.h for the
// layout and the definition of scales and offsets).
//
// Every token and head has a scale and an offset of its own, so that writing looks at nothing that is there
// already, and what a token is held as does not depend on the call that brought it.
//
// Both kernels move 16 bytes of binary16 a lane, a row of head_dim values being 8 to 32 lanes side by side; the
// extrema of a row travel between them as one pair (max, -min), four or five shuffles. Bound by 2 bytes read and 0.53 written
// per value (reading back: the reverse), and in single-token calls by a launch and two dependent loads.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

#include "kv_common.cuh"
#include "ptx.cuh"

namespace b200gemm {

struct KvAppendU4Params {
  KvCacheU4View c;
  KvBatch b;
  const __half* x[2];
  long long token_stride, head_stride;
  int blocks_per_seq;
};

constexpr int KV4_THREADS = 256;
constexpr int KV4_TOKENS = 16;  // tokens per CTA
constexpr int KV4_UNITS = 4;    // 16-byte pieces a thread has in flight

// Two halves' larger one each, a NaN on either side staying.
__device__ __forceinline__ uint32_t kv4_max2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// grid: (batch * blocks_per_seq, 2)
__global__ void __launch_bounds__(KV4_THREADS) kv_append_u4_kernel(const KvAppendU4Params p) {
  if (threadIdx.x == 0) ptx::grid_dep_launch_dependents();
  const int seq = static_cast<int>(blockIdx.x) / p.blocks_per_seq;
  const int nth = static_cast<int>(blockIdx.x) % p.blocks_per_seq;
  const int which = static_cast<int>(blockIdx.y);
  ptx::grid_dep_wait();
  const KvRange r = kv_range(p.b, seq, p.c.page, threadIdx.x == 0 && nth == 0 && which == 0);
  const int t0 = nth * KV4_TOKENS;
  const int tokens = min(KV4_TOKENS, r.end - r.begin - t0);
  if (tokens <= 0) return;
  const int per_row = p.c.dim / 8;  // lanes of a row: 8, 16 or 32
  const int rows = tokens * p.c.heads, at_once = KV4_THREADS / per_row;
  const int lane = static_cast<int>(threadIdx.x) & (per_row - 1), first = static_cast<int>(threadIdx.x) / per_row;
  const __half* const x = (which ? p.x[1] : p.x[0]) + lane * 8;
  const int* const table = p.b.table + static_cast<long long>(seq) * p.b.table_stride;
  uint8_t* const codes = which ? p.c.codes[1] : p.c.codes[0];
  __half2* const scales = which ? p.c.scales[1] : p.c.scales[0];
#pragma unroll 1
  for (int row0 = 0; row0 < rows; row0 += KV4_UNITS * at_once) {
    uint4 v[KV4_UNITS];
    int slot[KV4_UNITS], head[KV4_UNITS], pos[KV4_UNITS];  // pos -1 = none
#pragma unroll
    for (int i = 0; i < KV4_UNITS; ++i) {
      const int row = row0 + first + i * at_once;
      const bool in = row < rows;
      const int t = in ? row / p.c.heads : 0;
      head[i] = in ? row - t * p.c.heads : 0;
      pos[i] = in ? r.begin + t0 + t : -1;
      v[i] = make_uint4(0, 0, 0, 0);
      slot[i] = -1;
      if (in) {
        slot[i] = kv_ld(table + (pos[i] >> p.c.page_shift));
        v[i] = ptx::ld_global_stream_v4(x + (static_cast<long long>(r.row0) + t0 + t) * p.token_stride + head[i] * p.head_stride);
      }
    }
#pragma unroll
    for (int i = 0; i < KV4_UNITS; ++i) {
      const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
      // (max, -min) of the row; the sign bit turned makes a minimum a maximum
      uint32_t most = kv4_max2(kv4_max2(w[0], w[1]), kv4_max2(w[2], w[3]));
      uint32_t least = kv4_max2(kv4_max2(w[0] ^ 0x80008000u, w[1] ^ 0x80008000u),
                                kv4_max2(w[2] ^ 0x80008000u, w[3] ^ 0x80008000u));
      uint32_t both = kv4_max2(__byte_perm(most, least, 0x5410), __byte_perm(most, least, 0x7632));
#pragma unroll
      for (int o = 16; o; o >>= 1)
        if (o < per_row) both = kv4_max2(both, __shfl_xor_sync(0xffffffffu, both, o));
      const __half hi = __ushort_as_half(static_cast<unsigned short>(both & 0xffffu));
      const __half lo = __ushort_as_half(static_cast<unsigned short>((both >> 16) ^ 0x8000u));
      const float low = __half2float(lo);
      // A row with a NaN or an infinity: scale NaN, which every value of it will be.
      const float range = __fsub_rn(__half2float(hi), low);
      const bool bad = !(fabsf(range) < INFINITY);
      __half step = bad ? __ushort_as_half(0x7fffu) : __float2half_rn(__fdiv_rn(range, 15.0f));
      // (the value of code 15 stays a binary16)
      if (low + 15.0f * __half2float(step) >= 65520.0f) step = __ushort_as_half(static_cast<unsigned short>(__half_as_ushort(step) - 1));
      const float s = __half2float(step);
      const float inverse = s > 0.0f ? __fdiv_rn(1.0f, s) : 0.0f;
      // Codes as whole FP32 numbers by adding 2^23 (rounded to even by the addition), four of them as one number below 2^16:
      // conversions to integers run at a quarter of the rate of all this.
      float four[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[2 * j]));
        const float2 g = __half22float2(*reinterpret_cast<const __half2*>(&w[2 * j + 1]));
        auto code = [&](float x) {  // (16 bits of scale may leave the largest value a little beyond 15)
          return __fadd_rn(__fadd_rn(fminf(__fmul_rn(__fsub_rn(x, low), inverse), 15.0f), 8388608.0f), -8388608.0f);
        };
        four[j] = fmaf(code(g.y), 4096.0f, fmaf(code(g.x), 256.0f, fmaf(code(f.y), 16.0f, code(f.x)))) + 8388608.0f;
      }
      const uint32_t word = bad ? 0u : __byte_perm(__float_as_uint(four[0]), __float_as_uint(four[1]), 0x5410);
      if (pos[i] < 0) continue;
      if (slot[i] < 0 || slot[i] >= p.c.num_pages) {
        if (lane == 0) kv_report(p.b.status);
        continue;
      }
      const long long token = (static_cast<long long>(slot[i]) * p.c.heads + head[i]) * p.c.page + (pos[i] & (p.c.page - 1));
      *reinterpret_cast<uint32_t*>(codes + token * (p.c.dim / 2) + lane * 4) = word;
      if (lane == 0) scales[token] = __halves2half2(step, lo);
    }
  }
}

struct KvReadU4Params {
  KvCacheU4View c;
  KvBatch b;
  __half* out[2];
  int blocks_per_seq;
};

// grid: (batch * blocks_per_seq, 2)
__global__ void __launch_bounds__(KV4_THREADS) kv_read_u4_kernel(const KvReadU4Params p) {
  if (threadIdx.x == 0) ptx::grid_dep_launch_dependents();
  const int seq = static_cast<int>(blockIdx.x) / p.blocks_per_seq;
  const int nth = static_cast<int>(blockIdx.x) % p.blocks_per_seq;
  const int which = static_cast<int>(blockIdx.y);
  ptx::grid_dep_wait();
  __half* const out = which ? p.out[1] : p.out[0];
  if (!out) return;
  const KvRange r = kv_range(p.b, seq, p.c.page, threadIdx.x == 0 && nth == 0);
  const int t0 = nth * KV4_TOKENS;
  const int tokens = min(KV4_TOKENS, r.end - r.begin - t0);
  if (tokens <= 0) return;
  const int per_row = p.c.dim / 8, per_token = p.c.heads * per_row;
  const int* const table = p.b.table + static_cast<long long>(seq) * p.b.table_stride;
  const uint8_t* const codes = which ? p.c.codes[1] : p.c.codes[0];
  const __half2* const scales = which ? p.c.scales[1] : p.c.scales[0];
  const int units = tokens * per_token;
#pragma unroll 1
  for (int first = static_cast<int>(threadIdx.x); first < units; first += KV4_UNITS * KV4_THREADS) {
    // the ids of all pieces, then their codes and scales, then the results: three latencies for all
    int slot[KV4_UNITS], pos[KV4_UNITS], rest[KV4_UNITS];
    uint32_t q[KV4_UNITS], s[KV4_UNITS];
#pragma unroll
    for (int i = 0; i < KV4_UNITS; ++i) {
      const int u = first + i * KV4_THREADS;
      const int t = u / per_token;
      rest[i] = u - t * per_token;
      pos[i] = u < units ? t : -1;
      slot[i] = u < units ? kv_ld(table + ((r.begin + t0 + t) >> p.c.page_shift)) : -1;
    }
#pragma unroll
    for (int i = 0; i < KV4_UNITS; ++i) {
      q[i] = s[i] = 0;
      if (slot[i] < 0 || slot[i] >= p.c.num_pages) {
        if (pos[i] >= 0) kv_report(p.b.status);
        continue;
      }
      const int head = rest[i] / per_row;
      const long long token = (static_cast<long long>(slot[i]) * p.c.heads + head) * p.c.page + ((r.begin + t0 + pos[i]) & (p.c.page - 1));
      asm volatile("ld.global.u32 %0, [%1];" : "=r"(q[i]) : "l"(codes + token * (p.c.dim / 2) + (rest[i] - head * per_row) * 4) : "memory");
      asm volatile("ld.global.u32 %0, [%1];" : "=r"(s[i]) : "l"(scales + token) : "memory");
    }
#pragma unroll
    for (int i = 0; i < KV4_UNITS; ++i) {
      if (pos[i] < 0) continue;
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&s[i]));
      uint32_t h[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // (a code under the exponent of 2^23; code times scale is exact in FP32, so that a fused product changes nothing)
        const float a = fmaf(__uint_as_float(0x4b000000u | ((q[i] >> (8 * j)) & 15u)) - 8388608.0f, f.x, f.y);
        const float b = fmaf(__uint_as_float(0x4b000000u | ((q[i] >> (8 * j + 4)) & 15u)) - 8388608.0f, f.x, f.y);
        const __half2 v = __floats2half2_rn(a, b);
        h[j] = *reinterpret_cast<const uint32_t*>(&v);
      }
      // rows of a token are dense: heads x dim
      *reinterpret_cast<uint4*>(out + ((static_cast<long long>(r.row0) + t0 + pos[i]) * per_token + rest[i]) * 8) =
          make_uint4(h[0], h[1], h[2], h[3]);
    }
  }
}

}  // namespace b200gemm
