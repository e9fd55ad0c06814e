// Host side of the cache and attention entry points: argument checks they share, and the launch.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/b200gemm.h"
#include "kv_common.cuh"
#include "shared_state.h"

namespace b200gemm {
namespace {

constexpr int MAX_DEV = 64;

bool misaligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

int check_batch(int batch, const int* cu, const int* start, const int* table, int table_stride,
                int max_rows, int rows, KvBatch* b) {
  if (batch <= 0 || !cu || !start || !table || table_stride <= 0 || max_rows <= 0 || rows <= 0)
    return GEMM_ERR_INVALID_ARG;
  if (misaligned(cu, 4) || misaligned(start, 4) || misaligned(table, 4)) return GEMM_ERR_MISALIGNED;
  b->batch = batch;
  b->cu = cu;
  b->start = start;
  b->table = table;
  b->table_stride = table_stride;
  b->max_rows = max_rows;
  b->rows = rows;
  return GEMM_OK;
}

template <class Kernel, class... Params>
int launch(const SharedDevice& dev, Kernel kernel, dim3 grid, int threads, size_t smem,
           cudaStream_t stream, const Params&... p) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(static_cast<unsigned>(threads));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = dev.plain_order ? 0 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, p...);
  return e == cudaSuccess ? GEMM_OK : shared_cuda_fail(e);
}

// Dynamic shared memory beyond 48 KB, once per kernel and device.
template <auto Kernel>
int allow_smem(const SharedDevice& dev, int bytes) {
  static std::atomic<bool> ready[MAX_DEV];
  if (ready[dev.device].load()) return GEMM_OK;
  const cudaError_t e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != cudaSuccess) return shared_cuda_fail(e);
  ready[dev.device].store(true);
  return GEMM_OK;
}

}  // namespace
}  // namespace b200gemm
