// Cache of pages: what the kernels that serve from it share (tsfm_kv_pages of include/tsfm.h on the device).
#pragma once
#include "common.cuh"

namespace tsfm {

constexpr int BAD_ID = 1, BAD_LEN = 2, PAGES_TIMEOUT = 4;      // TSFM_PAGES_*

struct PagesDev {
  char *k, *v;
  long long page_stride, head_stride, slot_stride;               // bytes
  const int *table;
  int table_stride, n_pages, page_log, n_kv_heads;
  int capacity;                                                  // slots a series may use
  int *status;                                                   // or NULL
};

__device__ __forceinline__ void pages_report(const PagesDev &pg, int bits) {
  if (pg.status) atomicOr(pg.status, bits);
}

// A length read from the device, cut to [0, cap].
__device__ __forceinline__ int cut(int v, int cap) { return min(max(v, 0), cap); }

// Page that holds `slot` (0 <= slot < capacity) of the series whose table row is given; -1 for an id outside the pool.
__device__ __forceinline__ int page_of(const PagesDev &pg, const int *row, int slot) {
  const int id = __ldg(row + (slot >> pg.page_log));
  return (unsigned)id < (unsigned)pg.n_pages ? id : -1;
}
// Byte offset of a slot's row of one head inside k and v.  64 bits: pools of long caches pass 2^32 bytes.
__device__ __forceinline__ long long slot_offset(const PagesDev &pg, int page, int head, int slot) {
  return page * pg.page_stride + head * pg.head_stride + (slot & ((1 << pg.page_log) - 1)) * pg.slot_stride;
}

// 16 bytes as elements.
template <typename T> struct Pack16 {
  static constexpr int N = 16 / (int)sizeof(T);
  uint4 raw;
  __device__ __forceinline__ float get(int i) const { return to_f32(reinterpret_cast<const T *>(&raw)[i]); }
  __device__ __forceinline__ void set(int i, float v) { reinterpret_cast<T *>(&raw)[i] = from_f32<T>(v); }
};

}  // namespace tsfm
