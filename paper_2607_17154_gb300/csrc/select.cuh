// The selection tables as kernels read them, and Alg. 2's slots on eight lanes a
// token: what the router kernels (route_select.cu) and the few-token layer
// (few_tokens.cu) share.
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

// ---------------------------------------------------------------------------
// Selection tables staged in shared memory (one copy per CTA).
struct SelSmem {
  uint32_t pmask[64];
  int nsub[64];
  int kind[4];
  uint8_t sublist[64 * 64];
};

// Threads t0, t0 + nt (nt >= 64) ... of the block load the layer's tables
// into shared memory. The header, masks and the first E x E entries are
// loaded before any of them is used, so that their latencies overlap; the
// E x E tables are copied with 16-byte loads where sizes and addresses
// allow.
static __device__ bool load_tables_range(const uint8_t* __restrict__ tab, int E, SelSmem& sm, float* s_Q,
                                  float* s_Cq, int t0, int nt) {
  const float* gQ = reinterpret_cast<const float*>(tab + kOffQtab);
  const float* gCq = reinterpret_cast<const float*>(tab + off_cq(E));
  const int n = E * E;
  const bool vec = (n & 3) == 0 && ((reinterpret_cast<uintptr_t>(gQ) | reinterpret_cast<uintptr_t>(gCq) |
                                     reinterpret_cast<uintptr_t>(s_Q) | reinterpret_cast<uintptr_t>(s_Cq)) &
                                    15u) == 0;
  const int Eh = reinterpret_cast<const int32_t*>(tab)[1];
  const int M = reinterpret_cast<const int32_t*>(tab)[2];
  uint32_t pm = 0;
  unsigned long long sb = 0;
  if (t0 < 64) {
    pm = reinterpret_cast<const uint32_t*>(tab + kOffPmask)[t0];
    sb = reinterpret_cast<const unsigned long long*>(tab + kOffSubst)[t0];
  }
  constexpr int kFirst = 4;  // 16-byte chunks of each table a thread loads up front
  float4 q_first[kFirst], c_first[kFirst];
  if (vec) {
    const float4* q4 = reinterpret_cast<const float4*>(gQ);
    const float4* c4 = reinterpret_cast<const float4*>(gCq);
#pragma unroll
    for (int u = 0; u < kFirst; ++u) {
      const int i = t0 + u * nt;
      if (i < n / 4) {
        q_first[u] = __ldg(q4 + i);
        c_first[u] = __ldg(c4 + i);
      }
    }
  }
  if (Eh != E || M <= 0 || M > 32) {
    if (blockIdx.x == 0 && t0 == 0) report(&g_err_route, ORDERMOE_DEV_BAD_INDEX, -1);
    return false;
  }
  if (t0 < 64) {
    sm.pmask[t0] = pm;
    int cnt = 0;
    while (sb) {
      const int b = __ffsll(static_cast<long long>(sb)) - 1;
      sm.sublist[t0 * 64 + cnt++] = static_cast<uint8_t>(b);
      sb &= sb - 1;
    }
    sm.nsub[t0] = cnt;
  }
  if (vec) {
    const float4* q4 = reinterpret_cast<const float4*>(gQ);
    const float4* c4 = reinterpret_cast<const float4*>(gCq);
#pragma unroll
    for (int u = 0; u < kFirst; ++u) {
      const int i = t0 + u * nt;
      if (i < n / 4) {
        reinterpret_cast<float4*>(s_Q)[i] = q_first[u];
        reinterpret_cast<float4*>(s_Cq)[i] = c_first[u];
      }
    }
#pragma unroll 4
    for (int i = t0 + kFirst * nt; i < n / 4; i += nt) {
      const float4 x = __ldg(q4 + i), y = __ldg(c4 + i);
      reinterpret_cast<float4*>(s_Q)[i] = x;
      reinterpret_cast<float4*>(s_Cq)[i] = y;
    }
  } else {
#pragma unroll 4
    for (int i = t0; i < n; i += nt) {
      s_Q[i] = gQ[i];
      s_Cq[i] = gCq[i];
    }
  }
  for (int i = t0; i < 4; i += nt) sm.kind[i] = 0;
  return true;
}

__device__ __forceinline__ void flush_kind_counts(SelSmem& sm, const int (&kind_count)[4],
                                                  int32_t* counters) {
  if (counters == nullptr) return;
  for (int i = 0; i < 4; ++i)
    if (kind_count[i]) atomicAdd(&sm.kind[i], kind_count[i]);
}

// The slots of one token whose targets are idx, on eight lanes (sub 0 .. 7); Aas:
// its row A[a][s][.] of the delay table (valid when a, s < M). Every lane of the
// warp calls it (the butterflies need them all), inactive tokens (past T, a NaN
// token) write nothing.
__device__ __forceinline__ void select_slots(
    int t, bool active, int sub, const int (&idx)[ORDERMOE_MAX_TOPK], int E, int k, int M, float qbar,
    const float* Aas, const SelSmem& sm, const float* s_Q, const float* s_Cq, int a, int s, float q,
    uint8_t* __restrict__ loc, float* __restrict__ qhat, int32_t* __restrict__ chosen_expert,
    uint8_t* __restrict__ chosen_server, uint8_t* __restrict__ kind_out, int (&kind_count)[4]) {
  unsigned long long taken = 0;
#pragma unroll
  for (int j = 0; j < ORDERMOE_MAX_TOPK; ++j)
    if (j < k && active) {
      if (idx[j] < 0 || idx[j] >= E) active = false;
      else taken |= 1ull << idx[j];
    }
  if (active && (a >= M || s >= M)) {
    if (sub == 0) report(&g_err_route, ORDERMOE_DEV_BAD_INDEX, t);
    active = false;
  }
  int first_server = s;
#pragma unroll
  for (int j = 0; j < ORDERMOE_MAX_TOPK; ++j) {
    if (j >= k) break;  // k is the same for every lane
    const int r = idx[j];
    const int nsub = active ? sm.nsub[r] : -1;
    unsigned long long best = ~0ull;
    for (int ki = sub; ki <= nsub; ki += 8) {
      const int kk = (ki == 0) ? r : sm.sublist[r * 64 + ki - 1];
      const bool issub = (ki != 0);
      float cq = 0.0f;
      if (issub) {
        if ((taken >> kk) & 1ull) continue;
        if (!(__fadd_rn(q, s_Q[r * E + kk]) <= qbar)) continue;  // Eq. 40 budget
        cq = s_Cq[r * E + kk];
      }
      uint32_t pm = sm.pmask[kk];
      while (pm) {
        const int m = __ffs(pm) - 1;
        pm &= pm - 1;
        const float cost = __fadd_rn(Aas[m], cq);
        const unsigned long long key =
            (static_cast<unsigned long long>(__float_as_uint(cost)) << 32) |
            (static_cast<unsigned long long>(issub ? 1u : 0u) << 31) |
            (static_cast<unsigned long long>(m != s ? 1u : 0u) << 30) |
            (static_cast<unsigned long long>(m) << 8) | static_cast<unsigned long long>(kk);
        best = key < best ? key : best;
      }
    }
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) {
      const unsigned long long other = __shfl_xor_sync(0xffffffffu, best, o);
      best = other < best ? other : best;
    }
    if (!active) continue;
    int kstar, mstar, kd;
    if (best == ~0ull) {
      if (sub == 0) report(&g_err_route, ORDERMOE_DEV_NO_CANDIDATE, t);
      kstar = r; mstar = s; kd = 0;
    } else {
      kstar = static_cast<int>(best & 0xFFu);
      mstar = static_cast<int>((best >> 8) & 0xFFu);
      const int bsub = static_cast<int>((best >> 31) & 1u);
      const int away = static_cast<int>((best >> 30) & 1u);
      kd = 2 * away + bsub;
      if (bsub) {
        taken |= 1ull << kstar;
        q = __fadd_rn(q, s_Q[r * E + kstar]);
      }
    }
    if (j == 0) first_server = mstar;
    if (sub == 0) {
      chosen_expert[(size_t)t * k + j] = kstar;
      chosen_server[(size_t)t * k + j] = static_cast<uint8_t>(mstar);
      kind_out[(size_t)t * k + j] = static_cast<uint8_t>(kd);
      if (kd == 0) ++kind_count[0];  // constant indices: kind_count[] stays in registers
      else if (kd == 1) ++kind_count[1];
      else if (kd == 2) ++kind_count[2];
      else ++kind_count[3];
    }
  }
  if (active && sub == 0 && loc != nullptr) {
    loc[t] = static_cast<uint8_t>(first_server);
    qhat[t] = q;
  }
}

}  // namespace om
