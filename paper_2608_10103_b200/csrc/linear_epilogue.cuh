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
// x * s(x (a + b x^2)), with b = 0 for SiLU (which leaves the term out: 0 * inf is a NaN), with s from one exponential and one division
// (ex2.approx, __fdividef): the exponential's relative error, about |u| 2^-22 + 2^-22 at argument u, is
// weighed by s (1 - s), which leaves an absolute error below 1e-6 |x| everywhere.  GELU proper takes
// erfc(z) = t (a1 + t (a2 + ... a5 t^3)) exp(-z^2), t = 1 / (1 + p z), for z >= 0 (Abramowitz and Stegun
// 7.1.26, error below 1.5e-7) on the side where it is small: 0.5 |x| times that error.
//
// In the tile kernels a call of this epilogue meets a chain of latencies, not a throughput: with one
// wave of tiles the whole of it lies behind the last product.  So it works on 16 columns at a time in a rolled loop
// (an epilogue unrolled over 64 columns is some 2000 instructions that a CTA with one tile fetches cold, at about
// ten cycles each), everything it reads is on its way one step ahead, and the residual arrives by the copy engine
// in the very staging buffer the result leaves from: the residual's block is fetched there, each thread
// reads its pieces, and writes the result over them.
//
// Measured: 4096 x 16384 x 4096 FP16 with bias and GELU 378-390 us (0.87 of the burst rate), 512 x 8192 x 8192 with bias, SiLU and
// residual 60.5 us, 333 x 1001 x 1096 FP32 with all stages 11.5 us; one row against 4096 x 4096 with bias and residual 7.1 us.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

#include "ptx.cuh"

namespace b200gemm {

enum LinearAct { LIN_ACT_NONE = 0, LIN_ACT_RELU = 1, LIN_ACT_GATE = 2, LIN_ACT_ERF = 3, LIN_ACT_SILU = 4 };

struct LinearEpilogue {
  const float* row_bias;  // indexed by the kernel's rows / columns; at most one of them is set
  const float* col_bias;
  const void* residual;   // element type of C, or null
  long long ldr;          // its row pitch in elements
  int r_vec_ok;           // 1: 16-byte loads along a row are aligned
  int r_tma;              // 1: the tile kernel fetches it by the copy engine (C goes out the same way)
  int act;                // LinearAct
  float gate_a, gate_b;   // LIN_ACT_GATE: x * s(x (a + b x^2)), LIN_ACT_SILU: x * s(a x); times log2 e
};

__device__ __forceinline__ float lin_exp2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float lin_gate(float x, float a, float b) {
  return __fdividef(x, 1.0f + lin_exp2(-x * fmaf(b * x, x, a)));
}

__device__ __forceinline__ float lin_silu(float x, float a) { return __fdividef(x, 1.0f + lin_exp2(-x * a)); }

__device__ __forceinline__ float lin_erf(float x) {
  const float z = fabsf(x) * 0.70710678118654752f;
  const float t = __fdividef(1.0f, fmaf(0.3275911f, z, 1.0f));
  float q = fmaf(t, 1.061405429f, -1.453152027f);
  q = fmaf(t, q, 1.421413741f);
  q = fmaf(t, q, -0.284496736f);
  q = fmaf(t, q, 0.254829592f);
  const float erfc = q * t * lin_exp2(-1.4426950408889634f * z * z);
  return 0.5f * x * (x < 0.0f ? erfc : 2.0f - erfc);
}

__device__ __forceinline__ float lin_activate(float x, const LinearEpilogue& e) {
  switch (e.act) {
    case LIN_ACT_RELU: return x < 0.0f ? 0.0f : x;  // (a NaN stays one)
    case LIN_ACT_GATE: return lin_gate(x, e.gate_a, e.gate_b);
    case LIN_ACT_ERF: return lin_erf(x);
    case LIN_ACT_SILU: return lin_silu(x, e.gate_a);
    default: return x;
  }
}

// The same for N values of a thread; the choice is the same for the whole grid.  (N = 8 or 16 in the tile
// kernels, in a rolled loop: an epilogue unrolled over 64 columns is some 2000 instructions that a CTA with
// one tile fetches cold, at about ten cycles each.)
template <int N>
__device__ __forceinline__ void lin_activate_all(float (&x)[N], const LinearEpilogue& e) {
  if (e.act == LIN_ACT_NONE) return;
  if (e.act == LIN_ACT_GATE) {
    const float a = e.gate_a, b = e.gate_b;
#pragma unroll
    for (int v = 0; v < N; ++v) x[v] = lin_gate(x[v], a, b);
  } else if (e.act == LIN_ACT_SILU) {
    const float a = e.gate_a;
#pragma unroll
    for (int v = 0; v < N; ++v) x[v] = lin_silu(x[v], a);
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

// Exchanged operands (lanes are consecutive elements of a row of C): the warp's 32 x COLS residual
// values, asked into L2 while the products are still being summed.
template <int BYTES, int COLS>
__device__ __forceinline__ void lin_prefetch_transposed(const LinearEpilogue& e, int row0, int col0, int m,
                                                        int n, int lane) {
  if (row0 < m)
    for (int c = col0 + lane; c < min(n, col0 + COLS); c += 32)
      asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const char*>(e.residual) +
                                                    (static_cast<long long>(c) * e.ldr + row0) * BYTES));
}
// A thread's part of a residual row, likewise.
template <int BYTES, int COLS>
__device__ __forceinline__ void lin_prefetch_row(const LinearEpilogue& e, int row, int col0, int n) {
  const char* at = static_cast<const char*>(e.residual) +
                   (static_cast<long long>(row) * e.ldr + col0) * BYTES;
  const int bytes = min(COLS, n - col0) * BYTES;
  for (int b = 0; b < bytes; b += 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(at + b));
}

// A value as it lies in memory: loaded without the conversion, which would wait for it.
template <int BYTES>
struct LinRaw;
template <>
struct LinRaw<4> {
  uint32_t bits = 0;
  __device__ __forceinline__ void load(const void* at) { asm volatile("ld.global.u32 %0, [%1];" : "=r"(bits) : "l"(at) : "memory"); }
  __device__ __forceinline__ float value() const { return __uint_as_float(bits); }
};
template <>
struct LinRaw<2> {
  uint16_t bits = 0;
  __device__ __forceinline__ void load(const void* at) { asm volatile("ld.global.u16 %0, [%1];" : "=h"(bits) : "l"(at) : "memory"); }
  __device__ __forceinline__ float value() const { return __half2float(__ushort_as_half(bits)); }
};
// N values of one lane of such a block.
template <int BYTES, int N>
__device__ __forceinline__ void lin_load_transposed(const LinearEpilogue& e, int row, int col, int m, int n,
                                                    LinRaw<BYTES> (&r)[N]) {
  const char* const base = static_cast<const char*>(e.residual) + static_cast<long long>(row) * BYTES;
#pragma unroll
  for (int v = 0; v < N; ++v) {
    r[v] = LinRaw<BYTES>();
    if (row < m && col + v < n) r[v].load(base + static_cast<long long>(col + v) * e.ldr * BYTES);
  }
}
template <int BYTES, int N>
__device__ __forceinline__ void lin_add_transposed(float (&x)[N], const LinRaw<BYTES> (&r)[N]) {
#pragma unroll
  for (int v = 0; v < N; ++v)
    x[v] += r[v].value();
}

// Where 16-byte pieces of rows are not aligned: a block of 32 rows x COLS elements between global memory
// and a staging buffer (rows of 128 bytes, 16-byte piece j of row r at j ^ (r & 7)), lanes along the rows.
template <int BYTES, int COLS, bool TO_GLOBAL>
__device__ __forceinline__ void lin_block_copy(uint32_t buf, void* global, long long pitch, int row0, int col0,
                                               int m, int n, int lane) {
  char* const base = static_cast<char*>(global);
#pragma unroll 8
  for (int r = 0; r < 32; ++r) {
#pragma unroll
    for (int h = 0; h < COLS / 32; ++h) {
      const int c = h * 32 + lane;
      if (row0 + r >= m || col0 + c >= n) continue;
      char* const at = base + (static_cast<long long>(row0 + r) * pitch + col0 + c) * BYTES;
      const uint32_t s = buf + static_cast<uint32_t>(r * 128 + (((c * BYTES / 16) ^ (r & 7)) << 4) + c * BYTES % 16);
      if constexpr (BYTES == 4) {
        uint32_t v;
        if constexpr (TO_GLOBAL) {
          asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(s) : "memory");
          *reinterpret_cast<uint32_t*>(at) = v;
        } else {
          asm volatile("ld.global.u32 %0, [%1];" : "=r"(v) : "l"(at) : "memory");
          asm volatile("st.shared.u32 [%0], %1;" ::"r"(s), "r"(v) : "memory");
        }
      } else {
        uint16_t v;
        if constexpr (TO_GLOBAL) {
          asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(s) : "memory");
          *reinterpret_cast<uint16_t*>(at) = v;
        } else {
          asm volatile("ld.global.u16 %0, [%1];" : "=h"(v) : "l"(at) : "memory");
          asm volatile("st.shared.u16 [%0], %1;" ::"r"(s), "h"(v) : "memory");
        }
      }
    }
  }
}

// Residual values of one row, columns col .. col + N - 1, as raw words (two halves or one float each).
// Rows and columns outside C read nothing and give zeros.  Ordinary loads: the values may come
// from the grid in front, whose end the caller has awaited.
template <int BYTES, int N>
__device__ __forceinline__ void lin_load_residual(const LinearEpilogue& e, int row, int col, int m,
                                                  int n, uint32_t (&r)[BYTES * N / 4]) {
#pragma unroll
  for (int v = 0; v < BYTES * N / 4; ++v) r[v] = 0;
  if (row >= m) return;
  if (e.r_vec_ok && col + N <= n) {
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
#pragma unroll
  for (int v = 0; v < N; ++v) {
    if (col + v >= n) continue;
    const long long at = static_cast<long long>(row) * e.ldr + col + v;
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
