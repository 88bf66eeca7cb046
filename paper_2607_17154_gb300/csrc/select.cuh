// The selection tables as kernels read them: what the router kernels (route_select.cu) and the
// few-token layer (few_tokens.cu) share.
#pragma once

#include "common.cuh"

namespace om {

// The device error word of the translation unit that selects.
static __device__ unsigned long long g_err_route = 0;

// Byte layout of the tables buffer (documented in ordermoe.h).
constexpr int kTabMagic = 0x4f4d5442;
constexpr size_t kOffPmask = 64, kOffSubst = 320, kOffQtab = 832;
__host__ __device__ inline size_t off_cq(int E) { return kOffQtab + sizeof(float) * E * E; }
__host__ __device__ inline size_t off_a(int E) { return off_cq(E) + sizeof(float) * E * E; }
__host__ __device__ inline size_t tables_bytes(int E, int M) {
  size_t b = off_a(E) + sizeof(float) * (size_t)M * M * M;
  return (b + 255) & ~size_t(255);
}

// Selection tables staged in shared memory (one copy per CTA).
struct SelSmem {
  uint32_t pmask[64];
  int nsub[64];
  int kind[4];
  uint8_t sublist[64 * 64];
};

}  // namespace om
