// Where a sequence's rows lie in a call, from what its array says of them.  Apart from the kernels so that a test can compile it by itself.
// Internal: not part of the C ABI.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define LQ_KV_HD __host__ __device__ __forceinline__
#else
#define LQ_KV_HD inline
#endif

struct LqRowRange {
  int row, n;                            // first row, and how many
};
// Rows start .. end - 1, kept within the call's `rows`, whatever the array holds (an end below its start: none).
LQ_KV_HD LqRowRange lq_kv_rows(int32_t start, int32_t end, int rows) {
  const int first = start < 0 ? 0 : start < rows ? start : rows, last = end < first ? first : end < rows ? end : rows;
  return {first, last - first};
}
