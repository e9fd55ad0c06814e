// Building blocks of the kernels whose threads fetch the pieces of their own MMA fragments: 16-byte
// asynchronous copies into a ring that is private to the thread, and the warp-level MMAs.
#pragma once

#include <stdint.h>

namespace b200gemm {

// Ring slots such a thread may have; the wait below takes its count as an immediate.
constexpr int FEW_ROWS_MAX_DEPTH = 8;

namespace warp_pieces {

// 16 bytes global -> shared, asynchronously; bytes = 0 writes zeros and reads nothing.
// cg: through L2 only (the long operand, read once); ca: kept in L1 too (the short operand,
// which every CTA of the SM reads again: a third of the kernel's requests).
__device__ __forceinline__ void cp_async_16_cg(uint32_t dst, const uint8_t* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes)
               : "memory");
}
__device__ __forceinline__ void cp_async_16_ca(uint32_t dst, const uint8_t* src, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes)
               : "memory");
}
// (The kernel may have been launched while the grid in front of it was still writing its
// operands -- programmatic dependent launch -- and reads nothing before griddepcontrol.wait.  The
// non-coherent path, ld.global.nc / __ldg, carries no order against that wait and promises
// nothing for data written during the kernel's lifetime: a version that fetched a step into
// registers with it returned a few hundred wrong sums per call for INT4 through gemm_host, whose
// int8 scratch is rewritten by the unpack kernel right in front.  Nothing here uses it.)
__device__ __forceinline__ void prefetch_l2(const uint8_t* p) {
  asm volatile("prefetch.global.L2 [%0];" ::"l"(p));
}
// Scale factors: an ordinary load, for the same reason.
__device__ __forceinline__ float ld_f32(const float* p) {
  float v;
  asm volatile("ld.global.f32 %0, [%1];" : "=f"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void cp_async_commit() {
  asm volatile("cp.async.commit_group;" ::: "memory");
}
template <int PENDING>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory");
}
// The instruction takes its count as an immediate; pending is 0 .. FEW_ROWS_MAX_DEPTH - 1 (0, a
// ring of one slot, is never launched but must not fall through to a wait that waits for less).
__device__ __forceinline__ void cp_async_wait_all_but(int pending) {
  switch (pending) {
    case 0: cp_async_wait<0>(); break;
    case 1: cp_async_wait<1>(); break;
    case 2: cp_async_wait<2>(); break;
    case 3: cp_async_wait<3>(); break;
    case 4: cp_async_wait<4>(); break;
    case 5: cp_async_wait<5>(); break;
    case 6: cp_async_wait<6>(); break;
    default: cp_async_wait<7>(); break;
  }
}

__device__ __forceinline__ void mma_s8_m16n8k32(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                                uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// FP16 operands: 16 rows x 16 values against 8 rows per instruction, FP32 accumulators; a 32-bit
// word holds two values, and words w, w + 1 of a thread's piece fill its K positions 2t, 2t + 1
// and 2t + 8, 2t + 9 on both sides.
__device__ __forceinline__ void mma_f16_m16n8k16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                                 uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t word_of(const uint4& v, int i) {
  return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
}

}  // namespace warp_pieces
}  // namespace b200gemm
