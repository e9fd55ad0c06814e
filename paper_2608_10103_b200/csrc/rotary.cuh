// Rotary positions of several axes (see include/b200attn.h).
//
//     (x_a, x_b) -> (x_a cos - x_b sin, x_b cos + x_a sin),   angle = position[axis(i)][token] * inv_freq[i]
//
// for the pair (a, b) = (i, i + rotary_dim / 2) or (2i, 2i + 1) of every head. Bound by 2 bytes read and 2 written
// per value: a CTA works the angles of its tokens out once for all heads, into shared memory, while its first values
// are on their way. An angle is reduced as turns in 64 bits, position * (inv_freq / 2 pi) minus the nearest whole number, so
// that a position of 2^31 still has its angle to 5e-7; cosine and sine, the products and their sum are FP32, rounded once.
// Measured: 16384 tokens, 40 heads of 128 and three axes 62 us, 0.84 of the copy rate (0.7 of the issue slots busy); 64 tokens 3.2 us.
// A thread's piece are two runs of eight values (halves) or one (neighbours), with its cosines and sines as whole
// 16-byte words that neighbouring lanes find on different banks.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

#include "kv_common.cuh"
#include "ptx.cuh"

namespace b200gemm {

constexpr int ROTARY_AXES = 4;
constexpr int ROTARY_THREADS = 256;
constexpr int ROTARY_TOKENS = 4;  // tokens per CTA at most
constexpr int ROTARY_UNITS = 2;   // pieces a thread has in flight

struct RotaryRows {
  const __half* x;
  __half* y;
  int heads;
  long long x_token, x_head, y_token, y_head;
};
struct RotaryParams {
  RotaryRows rows[2];
  int tokens, per_cta;
  int dim, rotary;
  int end[ROTARY_AXES];  // of the axes' frequencies
  const int* positions;
  long long axis_stride;
  const float* inv_freq;
};

// HALVES: pairs (i, i + rotary / 2), else (2i, 2i + 1).  Dynamic shared memory: per_cta * rotary floats.
template <bool HALVES>
__global__ void __launch_bounds__(ROTARY_THREADS) rotary_kernel(const RotaryParams p) {
  extern __shared__ float4 rotary_table[];
  if (threadIdx.x == 0) ptx::grid_dep_launch_dependents();
  const int token0 = static_cast<int>(blockIdx.x) * p.per_cta;
  const int tokens = min(p.per_cta, p.tokens - token0);
  const int tid = static_cast<int>(threadIdx.x);
  const int count = p.rotary / 2;
  constexpr int FREQS = HALVES ? 8 : 4;   // of a piece
  constexpr int WORDS = FREQS / 2;        // float4 of a piece: cosines, then sines
  const int turned = count / FREQS;       // pieces of a head that turn
  const int passed = (p.dim - p.rotary) / 8;  // runs of eight values that do not
  const int per_head = turned + passed, heads = p.rows[0].heads + p.rows[1].heads;
  const int per_token = heads * per_head, units = tokens * per_token;
  ptx::grid_dep_wait();

  struct Piece {
    uint4 a, b;
    __half* to;
    int table;  // first word of its cosines; -1: passed on, -2: none
  };
  auto load = [&](int u) {
    Piece w;
    w.table = -2;
    if (u >= units) return w;
    const int t = u / per_token, rest = u - t * per_token;
    int head = rest / per_head;
    const int piece = rest - head * per_head;
    const bool second = head >= p.rows[0].heads;
    const RotaryRows& r = p.rows[second];
    if (second) head -= p.rows[0].heads;
    const int d = piece < turned ? piece * 8 : p.rotary + (piece - turned) * 8;
    const __half* const from = r.x + (static_cast<long long>(token0) + t) * r.x_token + head * r.x_head + d;
    w.to = r.y + (static_cast<long long>(token0) + t) * r.y_token + head * r.y_head + d;
    w.table = piece < turned ? t * (WORDS * turned) + piece : -1;
    if (w.table < 0 && r.x == r.y) {
      w.table = -2;  // in place: nothing to do
      return w;
    }
    w.a = ptx::ld_global_stream_v4(from);
    if (HALVES && w.table >= 0) w.b = ptx::ld_global_stream_v4(from + count);
    return w;
  };
  Piece piece[ROTARY_UNITS];
#pragma unroll
  for (int i = 0; i < ROTARY_UNITS; ++i) piece[i] = load(tid + i * ROTARY_THREADS);

  float* const table = reinterpret_cast<float*>(rotary_table);
#pragma unroll 1
  for (int u = tid; u < tokens * count; u += ROTARY_THREADS) {
    const int t = u / count, i = u - t * count;
    int axis = 0;
#pragma unroll
    for (int a = 0; a < ROTARY_AXES - 1; ++a) axis += i >= p.end[a];
    const int pos = kv_ld(p.positions + axis * p.axis_stride + token0 + t);
    const double turns = static_cast<double>(pos) * (static_cast<double>(ptx::ld_global_f32(p.inv_freq + i)) * 0.15915494309189535);
    float sine, cosine;
    sincospif(static_cast<float>(2.0 * (turns - rint(turns))), &sine, &cosine);
    // [token][word][piece][4]
    const int at = ((t * WORDS + (i % FREQS) / 4) * turned + i / FREQS) * 4 + i % 4;
    table[at] = cosine;
    table[at + WORDS / 2 * turned * 4] = sine;
  }
  __syncthreads();

#pragma unroll 1
  for (int first = tid; first < units; first += ROTARY_UNITS * ROTARY_THREADS) {
#pragma unroll
    for (int i = 0; i < ROTARY_UNITS; ++i) {
      const Piece w = piece[i];
      piece[i] = load(first + (i + ROTARY_UNITS) * ROTARY_THREADS);
      if (w.table == -2) continue;
      if (w.table == -1) {
        *reinterpret_cast<uint4*>(w.to) = w.a;
        continue;
      }
      float c[FREQS], s[FREQS];
#pragma unroll
      for (int v = 0; v < WORDS / 2; ++v) {
        *reinterpret_cast<float4*>(c + 4 * v) = rotary_table[w.table + v * turned];
        *reinterpret_cast<float4*>(s + 4 * v) = rotary_table[w.table + (WORDS / 2 + v) * turned];
      }
      uint32_t a[4] = {w.a.x, w.a.y, w.a.z, w.a.w};
      if constexpr (HALVES) {
        uint32_t b[4] = {w.b.x, w.b.y, w.b.z, w.b.w};
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&a[v]));
          const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&b[v]));
          const __half2 lo = __floats2half2_rn(x.x * c[2 * v] - y.x * s[2 * v], x.y * c[2 * v + 1] - y.y * s[2 * v + 1]);
          const __half2 hi = __floats2half2_rn(y.x * c[2 * v] + x.x * s[2 * v], y.y * c[2 * v + 1] + x.y * s[2 * v + 1]);
          a[v] = *reinterpret_cast<const uint32_t*>(&lo);
          b[v] = *reinterpret_cast<const uint32_t*>(&hi);
        }
        *reinterpret_cast<uint4*>(w.to + count) = make_uint4(b[0], b[1], b[2], b[3]);
      } else {
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&a[v]));
          const __half2 r = __floats2half2_rn(x.x * c[v] - x.y * s[v], x.y * c[v] + x.x * s[v]);
          a[v] = *reinterpret_cast<const uint32_t*>(&r);
        }
      }
      *reinterpret_cast<uint4*>(w.to) = make_uint4(a[0], a[1], a[2], a[3]);
    }
  }
}

}  // namespace b200gemm
