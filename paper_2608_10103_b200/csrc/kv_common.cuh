// What the kernels of the key/value caches share: views of cache and batch, and a sequence's range of rows.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

namespace b200gemm {

constexpr int DEV_BAD_INDEX = 6;  // status word: a length, count or page id outside its range

struct KvCacheView {
  int8_t* codes[2];  // K, V
  float* scales[2];
  int num_pages, heads, page, page_shift, dim;
};

struct KvCacheU4View {
  uint8_t* codes[2];  // K, V
  __half2* scales[2]; // (scale, offset) per token
  int num_pages, heads, page, page_shift, dim;
};

struct KvBatch {
  int batch;
  const int* cu;       // rows of the packed arrays
  const int* start;    // past (append), first (read)
  const int* table;
  int table_stride;    // entries per sequence
  int max_rows;        // upper bound of rows per sequence
  int rows;            // rows of the packed arrays
  int* status;
};

__device__ __forceinline__ int kv_ld(const int* p) {  // may have been written by the grid in front
  int v;
  asm volatile("ld.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void kv_report(int* status) { atomicCAS(status, 0, DEV_BAD_INDEX); }

// First token that a query at position `pos` sees (0 where it sees none); window 0: all.
__device__ __forceinline__ int kv_first_seen(int pos, int window) { return window > 0 && pos >= window ? pos - window + 1 : 0; }

// Rows and positions of a sequence, cut to what the packed arrays, the table and the caller's bound allow.
struct KvRange {
  int row0;   // first row in the packed arrays
  int begin;  // first position
  int end;    // one past the last
};
__device__ __forceinline__ KvRange kv_range(const KvBatch& b, int seq, int page, bool report) {
  KvRange r;
  r.row0 = kv_ld(b.cu + seq);
  long long n = static_cast<long long>(kv_ld(b.cu + seq + 1)) - r.row0;
  long long first = kv_ld(b.start + seq);
  const long long room = min(static_cast<long long>(b.table_stride) * page, 0x7fffffffll);
  bool bad = n < 0 || n > b.max_rows || first < 0 || r.row0 < 0 || r.row0 + n > b.rows;
  n = min(n, min(static_cast<long long>(b.max_rows), static_cast<long long>(b.rows) - r.row0));
  if (n < 0 || first < 0 || r.row0 < 0) n = first = 0;
  if (n > 0 && first + n > room) {
    bad = true;
    n = room > first ? room - first : 0;
  }
  if (bad && report) kv_report(b.status);
  r.begin = static_cast<int>(first);
  r.end = static_cast<int>(first + n);
  return r;
}

}  // namespace b200gemm
