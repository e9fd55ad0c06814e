// Barrier waits that give up, and the codes they leave in the device status word.
#pragma once

#include <stdint.h>

#include "ptx.cuh"

namespace b200gemm {

constexpr uint64_t WAIT_LIMIT_NS = 2000000000ull;  // every barrier wait gives up after 2 s

// Device status codes written to the status word when a wait gives up.
enum DeviceStatus {
  DEV_OK = 0,
  DEV_TIMEOUT_PRODUCER = 1,
  DEV_TIMEOUT_MMA = 2,
  DEV_TIMEOUT_EPILOGUE = 3,
  DEV_TIMEOUT_DRAIN = 4,
  DEV_TIMEOUT_UNPACK = 5,
};

// Bounded wait: polls the barrier; after the limit (or once another role has
// given up) records `code` and returns false.  The caller then leaves its loop.
template <bool BACKOFF = false>
__device__ __forceinline__ bool wait_bounded(uint32_t bar, uint32_t parity,
                                             volatile uint32_t* abort_flag, int* status, int code,
                                             uint32_t backoff_ns = 0) {
  auto done = [&]() { return ptx::mbar_try_wait(bar, parity); };
  if (done()) return true;
  uint64_t t0 = 0;
  uint32_t spins = 0;
  while (true) {
    if (done()) return true;
    if (BACKOFF && backoff_ns) __nanosleep(backoff_ns);
    if ((++spins & 255u) == 0) {
      if (*abort_flag) return false;
      uint64_t now = ptx::globaltimer_ns();
      if (t0 == 0) {
        t0 = now;
      } else if (now - t0 > WAIT_LIMIT_NS) {
        *abort_flag = 1;
        atomicCAS(status, 0, code);
        return false;
      }
    }
  }
}

}  // namespace b200gemm
