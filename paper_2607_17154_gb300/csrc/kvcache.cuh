// What the calls on a paged cache share: its descriptor's checks and how a slot's row is found.
#pragma once

#include "common.cuh"

namespace om {

constexpr int kCacheMaxPage = 1024;

// Checks a descriptor before anything is enqueued; `what` begins the message.
int check_cache(const ordermoe_cache* c, const char* what);

// A cache as kernels take it. A sequence's slot i is row i % page of page table[s][i / page].
struct CacheView {
  uint16_t* k;
  uint16_t* v;
  int64_t pages;
  int page_log, heads, seqs, cap;  // cap: slots that a sequence's row of the table reaches
  const int32_t* table;
  int64_t ld_table;
  const int32_t* length;
  float* mass;
  int32_t* pos;

  // slots of sequence s that are read: a length outside [0, cap] is cut to it (and reported by the caller)
  __device__ __forceinline__ int slots(int s) const {
    const int n = length[s];
    return n < 0 ? 0 : n > cap ? cap : n;
  }
  __device__ __forceinline__ int32_t page_of(int s, int slot) const {
    return table[static_cast<int64_t>(s) * ld_table + (slot >> page_log)];
  }
  __device__ __forceinline__ bool good(int32_t p) const { return p >= 0 && p < pages; }
  // row of [pages * heads * page]; times the width it may pass 32 bits
  __device__ __forceinline__ int64_t row(int32_t p, int head, int slot) const {
    return ((static_cast<int64_t>(p) * heads + head) << page_log) + (slot & ((1 << page_log) - 1));
  }
  __device__ __forceinline__ int64_t side(int s, int head, int slot) const {  // in mass and pos
    return (static_cast<int64_t>(s) * heads + head) * cap + slot;
  }
};

CacheView cache_view(const ordermoe_cache* c);

}  // namespace om
