// What the second translation unit (kv_api.cu) needs of the state that gemm_api.cu owns.
// Internal: not exported in any header of include/.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>

namespace b200gemm {

struct SharedDevice {
  int device;
  int num_sms;
  int* status;       // device status word
  bool plain_order;  // launches in plain stream order (gemm_set_l2_policy bit 32)
};
int shared_device(SharedDevice* out);

// Records the error for gemm_last_cuda_error and returns GEMM_ERR_CUDA.
int shared_cuda_fail(cudaError_t e);

// Scratch leased for the launches enqueued between the two calls: `head` bytes that are zero when
// first handed out and that every user leaves zero, then `need` bytes.
struct SharedLease {
  void* head;
  void* data;
  void* ptr;
  size_t bytes, head_bytes;
  int slot;
};
int shared_scratch(int device, cudaStream_t stream, size_t need, size_t head, SharedLease* out);
int shared_scratch_done(int device, cudaStream_t stream, const SharedLease& lease);

}  // namespace b200gemm
