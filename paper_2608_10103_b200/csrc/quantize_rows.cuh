// Row quantisation in front of an integer product: per row of X
//
//     amax = max_k |x[k]|,  scale = amax / T,  q[k] = rint(x[k] * (T / amax)),   T = 127 (INT8) or 7 (INT4)
//
// with IEEE divisions and round-half-even, so that the codes are a function of the inputs alone
// and |q| <= T without a clamp.  A row of zeros gives scale 0 and codes 0.  A row with an infinity
// or a NaN gives that as its scale and codes of 0 where x * (T / amax) is not a number, so that
// every result of the product that uses it is NaN rather than plausible: the maximum is taken over
// the magnitude bits, where infinities and NaN compare above every finite value.
//
// Bound by reading X once and writing the codes.  A row is kept in registers between its two
// passes (eight values per piece, QR_PIECES pieces per thread); what a very long row has beyond
// that is read again, from L2.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

#include "ptx.cuh"

namespace b200gemm {

constexpr int QR_PIECES = 4;    // pieces of eight values a thread keeps
constexpr int QR_THREADS = 256;

struct QuantRowsParams {
  const void* x;
  long long ldx;   // row pitch in elements
  uint8_t* q;      // rows of K (INT8) or K / 2 (INT4, low nibble first) bytes
  float* scale;
  int rows, K;     // K % 16 == 0
  int vec_ok;      // rows of x allow 16-byte loads
  int row_threads; // threads per row: 32, 64, 128 or 256
};

// Eight values as they are in memory.  Loading and converting are apart, so that all of a thread's loads are on their
// way before the first is waited for.
template <bool F16>
struct QrPiece {
  uint4 w[F16 ? 1 : 2];

  __device__ __forceinline__ void load(const QuantRowsParams& p, long long at) {
    if constexpr (F16) {
      const __half* x = static_cast<const __half*>(p.x) + at;
      if (p.vec_ok) {
        w[0] = ptx::ld_global_stream_v4(x);
      } else {
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const volatile uint16_t* h = reinterpret_cast<const volatile uint16_t*>(x) + 2 * i;
          u[i] = h[0] | (static_cast<uint32_t>(h[1]) << 16);
        }
        w[0] = make_uint4(u[0], u[1], u[2], u[3]);
      }
    } else {
      const float* x = static_cast<const float*>(p.x) + at;
      if (p.vec_ok) {
        w[0] = ptx::ld_global_stream_v4(x);
        w[1] = ptx::ld_global_stream_v4(x + 4);
      } else {
        uint32_t u[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = __float_as_uint(ptx::ld_global_f32(x + i));
        w[0] = make_uint4(u[0], u[1], u[2], u[3]);
        w[1] = make_uint4(u[4], u[5], u[6], u[7]);
      }
    }
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < (F16 ? 4 : 2); ++i) {
      if constexpr (F16) {
        const uint32_t u = i == 0 ? w[0].x : i == 1 ? w[0].y : i == 2 ? w[0].z : w[0].w;
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
      } else {
        v[4 * i] = __uint_as_float(w[i].x);
        v[4 * i + 1] = __uint_as_float(w[i].y);
        v[4 * i + 2] = __uint_as_float(w[i].z);
        v[4 * i + 3] = __uint_as_float(w[i].w);
      }
    }
  }
  // The larger of m and the magnitude bits (as FP32) of the eight values.
  __device__ __forceinline__ uint32_t max_bits(uint32_t m) const {
    float v[8];
    values(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    return m;
  }
};

template <bool S4, bool F16>
__device__ __forceinline__ void qr_store(const QuantRowsParams& p, int row, int piece, float inverse,
                                         const QrPiece<F16>& x) {
  float v[8];
  x.values(v);
  int c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = __float2int_rn(v[i] * inverse);
  if constexpr (S4) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) w |= (static_cast<uint32_t>(c[i]) & 15u) << (4 * i);
    *reinterpret_cast<uint32_t*>(p.q + static_cast<long long>(row) * (p.K / 2) + piece * 4) = w;
  } else {
    uint2 w;
    w.x = (c[0] & 255) | ((c[1] & 255) << 8) | ((c[2] & 255) << 16) | (static_cast<uint32_t>(c[3]) << 24);
    w.y = (c[4] & 255) | ((c[5] & 255) << 8) | ((c[6] & 255) << 16) | (static_cast<uint32_t>(c[7]) << 24);
    *reinterpret_cast<uint2*>(p.q + static_cast<long long>(row) * p.K + piece * 8) = w;
  }
}

template <bool F16, bool S4>
__global__ void __launch_bounds__(QR_THREADS) quantize_rows_kernel(const QuantRowsParams p) {
  __shared__ uint32_t warp_max[QR_THREADS / 32];
  if (threadIdx.x == 0) ptx::grid_dep_launch_dependents();
  const int t = static_cast<int>(threadIdx.x) & (p.row_threads - 1);
  const int rows_per_cta = QR_THREADS / p.row_threads;
  const int row = static_cast<int>(blockIdx.x) * rows_per_cta + static_cast<int>(threadIdx.x) / p.row_threads;
  const bool live = row < p.rows;
  const int pieces = live ? p.K / 8 : 0;
  const long long at = static_cast<long long>(live ? row : 0) * p.ldx;
  ptx::grid_dep_wait();  // x may come from the grid in front, which may also still read q
  QrPiece<F16> v[QR_PIECES] = {};  // (what is not loaded counts as zeros)
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < QR_PIECES; ++i) {
    const int piece = t + i * p.row_threads;
    if (piece < pieces) v[i].load(p, at + piece * 8);
  }
#pragma unroll
  for (int i = 0; i < QR_PIECES; ++i) m = v[i].max_bits(m);
  for (int piece = t + QR_PIECES * p.row_threads; piece < pieces; piece += p.row_threads) {
    QrPiece<F16> u;
    u.load(p, at + piece * 8);
    m = u.max_bits(m);
  }
  m = __reduce_max_sync(0xffffffffu, m);
  if (p.row_threads > 32) {
    const int warp = static_cast<int>(threadIdx.x) >> 5, per = p.row_threads >> 5;
    if ((threadIdx.x & 31) == 0) warp_max[warp] = m;
    __syncthreads();
    const int first = warp / per * per;
    for (int w = 0; w < per; ++w) m = max(m, warp_max[first + w]);
  }
  if (!live) return;
  constexpr float TOP = S4 ? 7.0f : 127.0f;
  const float amax = __uint_as_float(m);
  // (FP32 rows whose largest value is below 4e-37: the inverse stays finite, codes come out smaller)
  const float inverse = m == 0 ? 0.0f : fminf(__fdiv_rn(TOP, amax), 3.402823466e38f);
  if (t == 0) p.scale[row] = __fdiv_rn(amax, TOP);
#pragma unroll
  for (int i = 0; i < QR_PIECES; ++i) {
    const int piece = t + i * p.row_threads;
    if (piece < pieces) qr_store<S4>(p, row, piece, inverse, v[i]);
  }
  for (int piece = t + QR_PIECES * p.row_threads; piece < pieces; piece += p.row_threads) {
    QrPiece<F16> u;
    u.load(p, at + piece * 8);
    qr_store<S4>(p, row, piece, inverse, u);
  }
}

}  // namespace b200gemm
