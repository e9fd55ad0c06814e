// Epilogue of a linear layer, shared by every GEMM kernel:
//
//     y[i][j] = act(x[i][j] + bias[j]) + residual[i][j],   x = sum, or float(sum) * row_scale * col_scale
//
// all in FP32, rounded once when the result is binary16.  Where the kernel runs on exchanged
// operands its rows are the caller's columns: the bias then goes by kernel row, and the residual
// is read through the same transposed index as C.
//
// Activations.  SiLU is x * s(x) with s the logistic function; the tanh form of GELU is
// 0.5 x (1 + tanh z) = x * s(2 z), z = sqrt(2/pi) (x + 0.044715 x^3).  Both are therefore
// x * s(x (a + b x^2)), one body for two constants, with s from one exponential and one division
// (__expf, __fdividef): the exponential's relative error, about |u| 2^-22 + 2^-22 at argument u, is
// weighed by s (1 - s), which leaves an absolute error below 1e-6 |x| everywhere.  GELU proper uses erff.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

#include "ptx.cuh"

namespace b200gemm {

enum LinearAct { LIN_ACT_NONE = 0, LIN_ACT_RELU = 1, LIN_ACT_GATE = 2, LIN_ACT_ERF = 3 };

struct LinearEpilogue {
  const float* row_bias;  // indexed by the kernel's rows / columns; at most one of them is set
  const float* col_bias;
  const void* residual;   // element type of C, or null
  long long ldr;          // its row pitch in elements
  int r_vec_ok;           // 1: 16-byte loads along a row are aligned
  int act;                // LinearAct
  float gate_a, gate_b;   // LIN_ACT_GATE: x * s(x (a + b x^2))
};

__device__ __forceinline__ float lin_gate(float x, float a, float b) {
  const float u = x * fmaf(b * x, x, a);
  return __fdividef(x, 1.0f + __expf(-u));
}

__device__ __forceinline__ float lin_erf(float x) { return 0.5f * x * (1.0f + erff(x * 0.70710678118654752f)); }

__device__ __forceinline__ float lin_activate(float x, const LinearEpilogue& e) {
  switch (e.act) {
    case LIN_ACT_RELU: return x < 0.0f ? 0.0f : x;  // (a NaN stays one)
    case LIN_ACT_GATE: return lin_gate(x, e.gate_a, e.gate_b);
    case LIN_ACT_ERF: return lin_erf(x);
    default: return x;
  }
}

// The same for N values of a thread; the choice is the same for the whole grid.  (N = 16 in the tile
// kernels, in a rolled loop: an epilogue unrolled over 64 columns is some 2000 instructions that a CTA with
// one tile fetches cold, at about ten cycles each.)
template <int N>
__device__ __forceinline__ void lin_activate_all(float (&x)[N], const LinearEpilogue& e) {
  if (e.act == LIN_ACT_NONE) return;
  if (e.act == LIN_ACT_GATE) {
    const float a = e.gate_a, b = e.gate_b;
#pragma unroll
    for (int v = 0; v < N; ++v) x[v] = lin_gate(x[v], a, b);
  } else if (e.act == LIN_ACT_ERF) {
#pragma unroll
    for (int v = 0; v < N; ++v) x[v] = lin_erf(x[v]);
  } else {
#pragma unroll
    for (int v = 0; v < N; ++v) x[v] = x[v] < 0.0f ? 0.0f : x[v];
  }
}

// Scales (integer sums) and bias.  Lane v holds the factors of column v of the block.
template <int N>
__device__ __forceinline__ void lin_scale_bias(float (&x)[N], bool scaled, float row_scale,
                                               float col_scale_mine, float row_bias,
                                               float col_bias_mine, bool by_column) {
  if (scaled) {
#pragma unroll
    for (int v = 0; v < N; ++v) x[v] = x[v] * row_scale * __shfl_sync(0xffffffffu, col_scale_mine, v);
  }
  if (by_column) {
#pragma unroll
    for (int v = 0; v < N; ++v) x[v] += __shfl_sync(0xffffffffu, col_bias_mine, v);
  } else {
#pragma unroll
    for (int v = 0; v < N; ++v) x[v] += row_bias;  // 0 without a bias
  }
}

// Asks the tile's part of a residual row into L2 while the products are still being summed.
template <int BYTES, int COLS>
__device__ __forceinline__ void lin_prefetch_row(const LinearEpilogue& e, int row, int col0, int n) {
  const char* at = static_cast<const char*>(e.residual) +
                   (static_cast<long long>(row) * e.ldr + col0) * BYTES;
  const int bytes = min(COLS, n - col0) * BYTES;
  for (int b = 0; b < bytes; b += 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(at + b));
}

// Residual values of one row, columns col .. col + N - 1, as raw words (two halves or one float each).
// Rows and columns outside C read nothing and give zeros.  Ordinary loads: the values may come
// from the grid in front, whose end the caller has awaited.
template <int BYTES, int N>
__device__ __forceinline__ void lin_load_residual(const LinearEpilogue& e, int row, int col, int m,
                                                  int n, int transposed, uint32_t (&r)[BYTES * N / 4]) {
#pragma unroll
  for (int v = 0; v < BYTES * N / 4; ++v) r[v] = 0;
  if (row >= m) return;
  if (!transposed && e.r_vec_ok && col + N <= n) {
    const char* at = static_cast<const char*>(e.residual) +
                     (static_cast<long long>(row) * e.ldr + col) * BYTES;
#pragma unroll
    for (int v = 0; v < BYTES * N / 16; ++v)
      asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(r[4 * v]), "=r"(r[4 * v + 1]), "=r"(r[4 * v + 2]), "=r"(r[4 * v + 3])
                   : "l"(at + 16 * v)
                   : "memory");
    return;
  }
  const long long base = transposed ? row : static_cast<long long>(row) * e.ldr;
  const long long step = transposed ? e.ldr : 1;
#pragma unroll
  for (int v = 0; v < N; ++v) {
    if (col + v >= n) continue;
    const long long at = base + (col + v) * step;
    if constexpr (BYTES == 4) {
      asm volatile("ld.global.u32 %0, [%1];"
                   : "=r"(r[v])
                   : "l"(static_cast<const uint32_t*>(e.residual) + at)
                   : "memory");
    } else {
      uint16_t h;
      asm volatile("ld.global.u16 %0, [%1];"
                   : "=h"(h)
                   : "l"(static_cast<const uint16_t*>(e.residual) + at)
                   : "memory");
      r[v / 2] |= static_cast<uint32_t>(h) << (16 * (v & 1));
    }
  }
}

template <int BYTES, int N>
__device__ __forceinline__ void lin_add_residual(float (&x)[N], const uint32_t (&r)[BYTES * N / 4]) {
#pragma unroll
  for (int v = 0; v < N; ++v) {
    if constexpr (BYTES == 4) {
      x[v] += __uint_as_float(r[v]);
    } else {
      const __half h = __ushort_as_half(static_cast<unsigned short>(r[v / 2] >> (16 * (v & 1))));
      x[v] += __half2float(h);
    }
  }
}

}  // namespace b200gemm
