// Row quantisation in front of an integer product: per row of X
//
//     amax = max_k |x[k]|,  scale = amax / T,  q[k] = rint(x[k] * (T / amax)),   T = 127 (INT8) or 7 (INT4)
//
// with IEEE divisions and round-half-even, so that the codes are a function of the inputs alone
// and |q| <= T without a clamp.  A row of zeros gives scale 0 and codes 0.  A row with an infinity
// or a NaN gives that as its scale and codes of 0 where x * (T / amax) is not a number, so that
// every result of the product that uses it is NaN rather than plausible: the maximum is taken over
// the magnitude bits, where infinities and NaN compare above every finite value.  FP32 rows below 2^-64, whose T / amax
// may leave the type, are multiplied by 2^64 first, which is exact.
//
// Bound by reading X once and writing the codes.  A row is kept in registers between its two
// passes (eight values per piece, QR_PIECES pieces per thread, as they are in memory: all loads are under way
// before the first is waited for); what a row of more than 32 K values has beyond that is read again, from L2.
// Measured: 8 x 8192 FP16 -> INT8 2.5 us, 2000 x 8192 11.2 us (4.4 TB/s), 8192 x 8192 41 us (4.9 TB/s), 2000 x 4096 FP32
// 8.1 us (5.1 TB/s).  32 values per thread: with 16, in CTAs twice as large, 2000 x 8192 took 19 us, with 64 (8 pieces)
// 8 rows took 3.5.  FP16 rows fit 48 registers, which puts 10 CTAs of 128 on an SM (64: 12.2 us); FP32 rows spill there.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

#include <type_traits>

#include "ptx.cuh"

namespace b200gemm {

constexpr int QR_PIECES = 4;    // pieces of eight values a thread keeps
constexpr int QR_THREADS = 128;       // of a CTA; a longer row takes one of up to QR_MAX_THREADS
constexpr int QR_MAX_THREADS = 1024;

struct QuantRowsParams {
  const void* x;
  long long ldx;   // row pitch in elements
  uint8_t* q;      // rows of K (INT8) or K / 2 (INT4, low nibble first) bytes
  float* scale;
  int rows, K;     // K % 16 == 0
  int vec_ok;      // rows of x allow 16-byte loads
  int row_threads; // threads per row: 32, 64, ... QR_MAX_THREADS
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
  // The larger of m and the magnitude bits of the eight values: FP32 in m, or binary16 in each half of m.
  __device__ __forceinline__ uint32_t max_bits(uint32_t m) const {
    const uint32_t u[8] = {w[0].x, w[0].y, w[0].z, w[0].w, w[F16 ? 0 : 1].x, w[F16 ? 0 : 1].y, w[F16 ? 0 : 1].z, w[F16 ? 0 : 1].w};
#pragma unroll
    for (int i = 0; i < (F16 ? 4 : 8); ++i)
      m = F16 ? __vmaxu2(m, u[i] & 0x7fff7fffu) : max(m, u[i] & 0x7fffffffu);
    return m;
  }
};

// The codes of a piece.  FINITE: |x * inverse| <= T for all of the row, and adding 1.5 * 2^23 in FP32 rounds to the nearest
// even integer and leaves it in the low bits (a conversion instruction per value runs at a quarter of the rate).  Rows that
// are not finite or are tiny go the other way, with a factor `lift` in front.
template <bool S4, bool FINITE, bool F16>
__device__ __forceinline__ void qr_store(const QuantRowsParams& p, int row, int piece, float lift, float inverse,
                                         const QrPiece<F16>& x) {
  float v[8];
  x.values(v);
  uint32_t c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    c[i] = FINITE ? __float_as_uint(__fadd_rn(__fmul_rn(v[i], inverse), 12582912.0f))
                  : static_cast<uint32_t>(__float2int_rn(__fmul_rn(__fmul_rn(v[i], lift), inverse)));
  if constexpr (S4) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) w |= (c[i] & 15u) << (4 * i);
    *reinterpret_cast<uint32_t*>(p.q + static_cast<long long>(row) * (p.K / 2) + piece * 4) = w;
  } else {
    uint2 w;
    w.x = __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
    w.y = __byte_perm(__byte_perm(c[4], c[5], 0x0040), __byte_perm(c[6], c[7], 0x0040), 0x5410);
    *reinterpret_cast<uint2*>(p.q + static_cast<long long>(row) * p.K + piece * 8) = w;
  }
}

template <bool F16, bool S4>
__global__ void __maxnreg__(F16 ? 48 : 64) quantize_rows_kernel(const QuantRowsParams p) {
  __shared__ uint32_t warp_max[QR_MAX_THREADS / 32];
  if (threadIdx.x == 0) ptx::grid_dep_launch_dependents();
  const int t = static_cast<int>(threadIdx.x) & (p.row_threads - 1);
  const int rows_per_cta = static_cast<int>(blockDim.x) / p.row_threads;
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
  for (int i = 0; i < QR_PIECES; ++i)
    if (i * p.row_threads < pieces) m = v[i].max_bits(m);
  for (int piece = t + QR_PIECES * p.row_threads; piece < pieces; piece += p.row_threads) {
    QrPiece<F16> u;
    u.load(p, at + piece * 8);
    m = u.max_bits(m);
  }
  if constexpr (F16) m = __float_as_uint(__half2float(__ushort_as_half(static_cast<unsigned short>(max(m & 0xffffu, m >> 16)))));
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
  const bool tiny = !F16 && m < 0x1f800000u;  // below 2^-64 (the least binary16 value is 2^-24)
  const float lift = tiny ? 0x1p64f : 1.0f;
  const float inverse = m == 0 ? 0.0f : __fdiv_rn(TOP, __fmul_rn(amax, lift));
  if (t == 0) p.scale[row] = __fdiv_rn(amax, TOP);
  auto store = [&](auto finite) {
    constexpr bool FINITE = decltype(finite)::value;
#pragma unroll
    for (int i = 0; i < QR_PIECES; ++i) {
      const int piece = t + i * p.row_threads;
      if (piece < pieces) qr_store<S4, FINITE>(p, row, piece, lift, inverse, v[i]);
    }
    for (int piece = t + QR_PIECES * p.row_threads; piece < pieces; piece += p.row_threads) {
      QrPiece<F16> u;
      u.load(p, at + piece * 8);
      qr_store<S4, FINITE>(p, row, piece, lift, inverse, u);
    }
  };
  if (m < 0x7f800000u && !tiny)
    store(std::true_type());
  else
    store(std::false_type());
}

}  // namespace b200gemm
