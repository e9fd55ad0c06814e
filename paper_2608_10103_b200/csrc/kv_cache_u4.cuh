// Key/value cache in 4 bits: writing new tokens and reading tokens back (see include/b200kv.h for the
// layout and the definition of scales and offsets).
//
// Every token and head has a scale and an offset of its own, so that writing looks at nothing that is there
// already, and what a token is held as does not depend on the call that brought it.
//
// Eight lanes share a row (a token's head), head_dim / 64 pieces of eight values each: 16 bytes of binary16 or 4 of codes, side by
// side. The extrema of a row travel between them as one pair (max, -min), three shuffles. What a row costs besides its values
// (where it lies, two divisions) is a third of the instructions so, instead of two thirds with one piece per lane
// (4 x up to 8192 tokens of 8 heads of 128 written and 4 x up to 9192 read back: 104 -> 62 us; values by pairs, 62 -> 58: 0.75 of the copy rate, at
// 256 d 0.88). Bound by 2 bytes read and 0.53 written per value (reading back: the reverse) and by issuing some 9 (5) instructions
// for each, in single-token calls by a launch and two dependent loads.
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
// Tokens per CTA: at 8 heads two turns through its rows (4 x up to 8192 tokens written and 9192 read at 64 d: 16 tokens, which one turn
// takes, 47.4 us, 32 39.4, 64 41.0; at 128 d 8 tokens 69.7, 16 57.7, 32 57.9, 64 64.8).
__host__ __device__ constexpr int kv4_tokens(int dim) { return dim == 64 ? 32 : 16; }
constexpr int KV4_ROWS = KV4_THREADS / 8;  // rows a CTA works on at a time
// Rows a thread has in flight: four pieces of 16 bytes.
__host__ __device__ constexpr int kv4_units(int dim) { return 256 / dim; }

// Two halves' larger or smaller one each, a NaN on either side staying.
__device__ __forceinline__ uint32_t kv4_max2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t kv4_min2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// Rows in the order of tokens, then heads, KV4_ROWS apart: no division per row.
struct Kv4Row {
  int token, head, step_token, step_head, heads;
  __device__ Kv4Row(int first, int heads) : heads(heads) {
    token = first / heads;
    head = first - token * heads;
    step_token = KV4_ROWS / heads;
    step_head = KV4_ROWS - step_token * heads;
  }
  __device__ void next() {
    token += step_token;
    head += step_head;
    if (head >= heads) {
      head -= heads;
      ++token;
    }
  }
};

// grid: (batch * blocks_per_seq, 2)
// Six CTAs per SM: 64 single tokens written and 16 of each read 6.7 us, as against 7.3 with what the compiler takes by itself (five).
template <int D>
__global__ void __launch_bounds__(KV4_THREADS, 6) kv_append_u4_kernel(const KvAppendU4Params p) {
  constexpr int PIECES = D / 64, UNITS = kv4_units(D);
  if (threadIdx.x == 0) ptx::grid_dep_launch_dependents();
  const int seq = static_cast<int>(blockIdx.x) / p.blocks_per_seq;
  const int nth = static_cast<int>(blockIdx.x) % p.blocks_per_seq;
  const int which = static_cast<int>(blockIdx.y);
  ptx::grid_dep_wait();
  const KvRange r = kv_range(p.b, seq, p.c.page, threadIdx.x == 0 && nth == 0 && which == 0);
  const int t0 = nth * kv4_tokens(D);
  const int tokens = min(kv4_tokens(D), r.end - r.begin - t0);
  if (tokens <= 0) return;
  const int lane = static_cast<int>(threadIdx.x) & 7;
  const __half* const x = (which ? p.x[1] : p.x[0]) + (static_cast<long long>(r.row0) + t0) * p.token_stride + lane * 8;
  const int* const table = p.b.table + static_cast<long long>(seq) * p.b.table_stride;
  uint8_t* const codes = (which ? p.c.codes[1] : p.c.codes[0]) + lane * 4;
  __half2* const scales = which ? p.c.scales[1] : p.c.scales[0];
  Kv4Row row(static_cast<int>(threadIdx.x) >> 3, p.c.heads);
#pragma unroll 1
  for (int done = 0; done < tokens * p.c.heads; done += UNITS * KV4_ROWS) {
    uint4 v[UNITS][PIECES];
    int slot[UNITS], at[UNITS];  // page, place of the row in it; -1 = no row
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      at[i] = -1;
      slot[i] = -1;
#pragma unroll
      for (int k = 0; k < PIECES; ++k) v[i][k] = make_uint4(0, 0, 0, 0);
      if (row.token < tokens) {
        const int pos = r.begin + t0 + row.token;
        at[i] = row.head * p.c.page + (pos & (p.c.page - 1));
        slot[i] = kv_ld(table + (pos >> p.c.page_shift));
        const __half* const from = x + row.token * p.token_stride + row.head * p.head_stride;
#pragma unroll
        for (int k = 0; k < PIECES; ++k) v[i][k] = ptx::ld_global_stream_v4(from + k * 64);
      }
      row.next();
    }
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      // (max, -min) of the row
      uint32_t most = 0xfc00fc00u, least = 0x7c007c00u;
#pragma unroll
      for (int k = 0; k < PIECES; ++k) {
        const uint32_t w[4] = {v[i][k].x, v[i][k].y, v[i][k].z, v[i][k].w};
        most = kv4_max2(most, kv4_max2(kv4_max2(w[0], w[1]), kv4_max2(w[2], w[3])));
        least = kv4_min2(least, kv4_min2(kv4_min2(w[0], w[1]), kv4_min2(w[2], w[3])));
      }
      least ^= 0x80008000u;
      uint32_t both = kv4_max2(__byte_perm(most, least, 0x5410), __byte_perm(most, least, 0x7632));
#pragma unroll
      for (int o = 4; o; o >>= 1) both = kv4_max2(both, __shfl_xor_sync(0xffffffffu, both, o));
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
      if (at[i] < 0) continue;
      if (slot[i] < 0 || slot[i] >= p.c.num_pages) {
        if (lane == 0) kv_report(p.b.status);
        continue;
      }
      const long long token = static_cast<long long>(slot[i]) * (p.c.heads * p.c.page) + at[i];
      if (lane == 0) scales[token] = __halves2half2(step, lo);
      // The scale's rounding may leave the largest value beyond 15 scale: by 2^-12 of it, three times that where the scale was lowered,
      // or by 15 x 2^-25 where binary16 has steps of 2^-24. From 2^-20 up that is less than half a scale, so that code 15 is its all the same.
      const bool tiny = s < 0x1p-20f;
      const uint64_t minus_low = ptx::pair(-low, -low), inverse2 = ptx::pair(inverse, inverse);
#pragma unroll
      for (int k = 0; k < PIECES; ++k) {
        const uint32_t w[4] = {v[i][k].x, v[i][k].y, v[i][k].z, v[i][k].w};
        // Codes as whole FP32 numbers by adding 2^23 (rounded to even by the addition), four of them as one number below 2^16:
        // conversions to integers run at a quarter of the rate of all this, which goes by pairs.
        constexpr float WHOLE = 8388608.0f;
        uint64_t y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
          y[j] = ptx::mul2(ptx::add2(ptx::pair(f.x, f.y), minus_low), inverse2);
        }
        if (__builtin_expect(tiny, 0)) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 f = ptx::unpair(y[j]);
            y[j] = ptx::pair(fminf(f.x, 15.0f), fminf(f.y, 15.0f));
          }
        }
        float four[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          // (2^23 stays with the first code, so that the bits of the whole can be read off)
          const uint64_t a = ptx::add2(ptx::add2(y[2 * j], ptx::pair(WHOLE, WHOLE)), ptx::pair(0.0f, -WHOLE));
          const uint64_t b = ptx::add2(ptx::add2(y[2 * j + 1], ptx::pair(WHOLE, WHOLE)), ptx::pair(-WHOLE, -WHOLE));
          const float2 f = ptx::unpair(ptx::fma2(b, ptx::pair(256.0f, 256.0f), a));
          four[j] = fmaf(f.y, 16.0f, f.x);
        }
        const uint32_t word = bad ? 0u : __byte_perm(__float_as_uint(four[0]), __float_as_uint(four[1]), 0x5410);
        *reinterpret_cast<uint32_t*>(codes + token * (D / 2) + k * 32) = word;
      }
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
template <int D>
__global__ void __launch_bounds__(KV4_THREADS) kv_read_u4_kernel(const KvReadU4Params p) {
  constexpr int PIECES = D / 64, UNITS = 2 * kv4_units(D);
  if (threadIdx.x == 0) ptx::grid_dep_launch_dependents();
  const int seq = static_cast<int>(blockIdx.x) / p.blocks_per_seq;
  const int nth = static_cast<int>(blockIdx.x) % p.blocks_per_seq;
  const int which = static_cast<int>(blockIdx.y);
  ptx::grid_dep_wait();
  __half* const out = which ? p.out[1] : p.out[0];
  if (!out) return;
  const KvRange r = kv_range(p.b, seq, p.c.page, threadIdx.x == 0 && nth == 0);
  const int t0 = nth * kv4_tokens(D);
  const int tokens = min(kv4_tokens(D), r.end - r.begin - t0);
  if (tokens <= 0) return;
  const int lane = static_cast<int>(threadIdx.x) & 7;
  const int* const table = p.b.table + static_cast<long long>(seq) * p.b.table_stride;
  const uint8_t* const codes = (which ? p.c.codes[1] : p.c.codes[0]) + lane * 4;
  const __half2* const scales = which ? p.c.scales[1] : p.c.scales[0];
  // rows of a token are dense: heads x dim, and so are those of neighbouring tokens
  __half* to = out + ((static_cast<long long>(r.row0) + t0) * p.c.heads + (threadIdx.x >> 3)) * D + lane * 8;
  Kv4Row row(static_cast<int>(threadIdx.x) >> 3, p.c.heads);
#pragma unroll 1
  for (int done = 0; done < tokens * p.c.heads; done += UNITS * KV4_ROWS) {
    // the ids of all rows, then their codes and scales, then the results: three latencies for all
    int slot[UNITS], at[UNITS];
    uint32_t q[UNITS][PIECES], s[UNITS];
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      at[i] = slot[i] = -1;
      if (row.token < tokens) {
        const int pos = r.begin + t0 + row.token;
        at[i] = row.head * p.c.page + (pos & (p.c.page - 1));
        slot[i] = kv_ld(table + (pos >> p.c.page_shift));
      }
      row.next();
    }
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      s[i] = 0;
#pragma unroll
      for (int k = 0; k < PIECES; ++k) q[i][k] = 0;
      if (slot[i] < 0 || slot[i] >= p.c.num_pages) {
        if (at[i] >= 0) kv_report(p.b.status);
        continue;
      }
      const long long token = static_cast<long long>(slot[i]) * (p.c.heads * p.c.page) + at[i];
#pragma unroll
      for (int k = 0; k < PIECES; ++k)
        asm volatile("ld.global.u32 %0, [%1];" : "=r"(q[i][k]) : "l"(codes + token * (D / 2) + k * 32) : "memory");
      asm volatile("ld.global.u32 %0, [%1];" : "=r"(s[i]) : "l"(scales + token) : "memory");
    }
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      if (at[i] >= 0) {
        // Code times scale plus offset, rounded once.
        const __half2 pair = *reinterpret_cast<const __half2*>(&s[i]), scale = __low2half2(pair), offset = __high2half2(pair);
        auto value = [&](uint32_t code, uint32_t zero) {
          const __half2 c = __hsub2(*reinterpret_cast<const __half2*>(&code), *reinterpret_cast<const __half2*>(&zero));
          const __half2 y = __hfma2(c, scale, offset);
          return *reinterpret_cast<const uint32_t*>(&y);
        };
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
          // Codes under the exponent of 1024 or 64, from which they come off exactly: 0 and 4 of the eight, 1 and 5, 2 and 6, 3 and 7.
          const uint32_t q0 = q[i][k], q1 = q0 >> 8;
          const uint32_t h04 = value((q0 & 0x000f000fu) | 0x64006400u, 0x64006400u), h15 = value((q0 & 0x00f000f0u) | 0x54005400u, 0x54005400u);
          const uint32_t h26 = value((q1 & 0x000f000fu) | 0x64006400u, 0x64006400u), h37 = value((q1 & 0x00f000f0u) | 0x54005400u, 0x54005400u);
          *reinterpret_cast<uint4*>(to + k * 64) =
              make_uint4(__byte_perm(h04, h15, 0x5410), __byte_perm(h26, h37, 0x5410), __byte_perm(h04, h15, 0x7632), __byte_perm(h26, h37, 0x7632));
        }
      }
      to += KV4_ROWS * D;
    }
  }
}

}  // namespace b200gemm
