// A whole MoE layer for a few tokens in one launch: router, softmax, top-k,
// selection (Alg. 2, H = 1), the chosen experts' SwiGLU FFN, the weighted
// combine and, on the residual map, the next layer's norm.
//
// At 1 to 16 tokens a layer is one pass over the chosen experts' weights: an
// expert's 6 d d_ff bytes meet at most 16 rows, so HBM bounds it and the tensor
// rate does not matter (mma.sync m16n8k16 with the weights as A and all tokens as
// the columns of B; a token's column of an expert it does not use is dropped).
// What a chain of launches costs beside that pass is their latency and the pauses
// of HBM between them, so one cooperative kernel of a CTA per SM runs it all:
//   route    every pair of CTAs computes all logits X W_r^T, half of K each, and both take
//            the same decisions (the router is small; a grid barrier would take longer);
//   gate/up  units of 16 columns of W1 and W3 of one expert over the whole K = d,
//            dealt out to the CTAs in turn: gate in rows 0-7 of a 16-row MMA tile
//            and up in rows 8-15, so that SwiGLU is in one lane's registers;
//   down     row tiles of 64 rows of W2 by all chosen experts' K = d_ff, cut
//            into one contiguous share of equal length per CTA. A share's partial
//            sums of a row tile go to the workspace;
//   finish   one CTA a token adds the partials of every row tile in CTA order and
//            writes y, or h + y and its norm.
// H, the SwiGLU activations, are handed on as the sum of two bf16 and the experts' outputs stay in
// fp32, so y is rounded once. Sums are fp32 in a fixed order: the same call gives the same bits.
// Two producer warps stream the weights and the tokens' K blocks through a ring of TMA
// boxes with the 128-byte swizzle; eight MMA warps take its slots in turn; an
// epilogue warp adds their eight partial accumulators. Between gate/up and down
// the producers fill the ring with W2 while the other CTAs finish H: the grid
// barrier there costs HBM no pause.
// In a CUDA graph: 16 tokens on 8 experts of d 4096, d_ff 14336 420 us = 6.4 TB/s of weights (0.95 of a
// copy's rate), 1 token 120 us (0.87); 1 token, top-6 of 64 experts of d 2048, d_ff 1408 38 us, of which the
// weights take 15: the rest is the latency of what comes one after the other.
#include <cstddef>
#include <type_traits>

#include "select.cuh"

namespace om {

int read_clear_err_few(unsigned long long* out) {
  unsigned long long zero = 0;
  OM_CUDA(cudaMemcpyFromSymbol(out, g_err_route, sizeof(*out)));
  OM_CUDA(cudaMemcpyToSymbol(g_err_route, &zero, sizeof(zero)));
  return ORDERMOE_OK;
}

namespace fw {

constexpr int TOKENS = ORDERMOE_FEW_TOKENS;
constexpr int MMA_WARPS = 8;
constexpr int PRODUCERS = 2;  // the warps behind the MMA warps; the last is the epilogue's
constexpr int THREADS = 32 * (MMA_WARPS + PRODUCERS + 1);
constexpr int KB_UP = 4, KB_DOWN = 2;  // 64-element K blocks a stage

// 16-row MMA tiles of a gate/up unit: with one, twice as many units share the SMs more evenly, but a
// token's rows are loaded for half the weights (1 token on 64 narrow experts, 528 units on 152 SMs, 37.8 us
// with two and 38.2 with one; 4 tokens 68.9 and 72.3; 4 on 8 wide experts 289 and 297).
constexpr int MT = 2;
// K blocks of a router stage, which holds rt tiles of 16 experts
__host__ __device__ constexpr int route_kb(int rt) { return 4 * MT / rt < 4 ? 4 * MT / rt : 4; }

// NT: 8-token column tiles.
template <int NT>
struct Cfg {
  static constexpr int W_BYTES = 8192 * MT;            // 16 MT rows x 256, or 32 MT x 128
  static constexpr int STAGE_BYTES = W_BYTES + 4096 * NT;  // and 8 NT tokens x 256
  static constexpr int DOWN_ROWS = 32 * MT;
  // partial accumulators of the MMA warps: two sets of a unit's, or one of a row tile's
  // (the router has up to four tiles, once)
  static constexpr int RED_FLOATS = MMA_WARPS * 2 * MT * NT * 128;
  static_assert(2 * MT >= 4, "tiles of 64 experts");
  // shared memory beside the ring: alignment, partials, the selection's Q and Cq
  static constexpr int other_bytes(int E) { return 1024 + RED_FLOATS * 4 + ((8 * E * E + 15) & ~15); }
};
constexpr int MAX_STAGES = 16;
constexpr int MAX_D = 32768;  // a row and its tiles' owners fit in the ring's memory

struct Smem {
  uint64_t full[MAX_STAGES], empty[MAX_STAGES];
  uint64_t red_full[3], red_empty[3];  // a unit's two sets; [2]: a row tile's
  int abort, zero;
  int tables_ok;                   // the header fits the layer
  uint8_t act[64];                 // their indices, ascending
  unsigned int mask[64];           // of an expert: the tokens that use it
  uint8_t slot[64][TOKENS];        // and the slot it is of each
  float logits[2][TOKENS][68];     // shares of K of either CTA
  alignas(16) float ex[TOKENS][68];  // exponentials of the softmax, read 16 bytes at a time
  float delay[TOKENS][ORDERMOE_MAX_SERVERS];  // A[home][location] of the tokens
  int32_t target[TOKENS * ORDERMOE_MAX_TOPK];
  float weight[TOKENS * ORDERMOE_MAX_TOPK];
  int32_t chosen[TOKENS * ORDERMOE_MAX_TOPK];
  uint8_t server[TOKENS * ORDERMOE_MAX_TOPK], kind[TOKENS * ORDERMOE_MAX_TOPK];
  uint8_t loc[TOKENS];             // location and loss, before and then after
  float qhat[TOKENS], qbar;
  int nan[TOKENS];                 // a logit is NaN
  int placed[TOKENS];              // home and location are servers
  int valid[TOKENS];               // decided: its outputs are written
  float sum[THREADS / 32];
};
static_assert(MAX_STAGES <= 32, "a lane a barrier");
static_assert(offsetof(Smem, ex) % 16 == 0 && alignof(Smem) == 16, "16-byte loads");
// A ring takes what the layer's tables leave of the 227 KB.
template <int NT>
constexpr int stages(int E) {
  const int left = 227 * 1024 - static_cast<int>(sizeof(Smem) + sizeof(SelSmem)) - 256 - Cfg<NT>::other_bytes(E);
  const int n = left / Cfg<NT>::STAGE_BYTES;
  return n < MAX_STAGES ? n : MAX_STAGES;
}
static_assert(stages<1>(64) >= 6 && stages<2>(64) >= 5, "ring");
static_assert(MAX_D / Cfg<1>::DOWN_ROWS * 4 + MAX_D * 2 <= 5 * Cfg<2>::STAGE_BYTES &&
                  Cfg<1>::STAGE_BYTES * 6 >= 5 * Cfg<2>::STAGE_BYTES, "finish");
static_assert(TOKENS * ORDERMOE_MAX_TOPK * 64 * 12 <= 5 * Cfg<2>::STAGE_BYTES, "candidates");

struct Maps {
  CUtensorMap Wr, Xr, X, W1, W3, W2, H;
};

struct Args {
  int T, E, d, dff, k, renorm;
  int stages;  // of the ring
  int given;  // the decisions are in target / weight / chosen (look-ahead): no routing
  const uint8_t* tab;
  const uint8_t* home;
  uint8_t* loc;
  float* qhat;
  const uint16_t* h;  // residual map, else null
  uint16_t* y;        // y, or h_out
  uint16_t* x_out;
  float eps;
  float* logits;
  int32_t* topk_idx;
  float* topk_w;
  int32_t* chosen;
  uint8_t* server;
  uint8_t* kind;
  int32_t* counters;
  unsigned int* sync;  // [0] gate/up done, [1] down done, [2] left: zero between launches
  uint16_t* H;         // [n_act][2][T][dff]: bf16 parts that add up to it
  float* part;         // [row tile + CTA][T][DOWN_ROWS]
  uint64_t limit_ns;
};

__device__ __forceinline__ void tma_load_3d(void* smem_dst, const CUtensorMap* map, uint64_t* bar,
                                            int row, int kb) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_u32(smem_dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(0), "r"(row), "r"(kb)
      : "memory");
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async;" ::: "memory"); }
__device__ __forceinline__ unsigned int load_acquire(const unsigned int* p) {
  unsigned int v;
  asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
// One thread: waits until the counter has reached n (bounded).
__device__ __forceinline__ bool grid_wait(const unsigned int* count, unsigned int n, uint64_t limit_ns,
                                          volatile int* abort) {
  if (load_acquire(count) >= n) return true;
  const uint64_t t0 = globaltimer();
  for (uint32_t i = 1;; ++i) {
    if (load_acquire(count) >= n) return true;
    if ((i & 15u) == 0 && (*abort || globaltimer() - t0 > limit_ns)) return false;
  }
}

// acc += the rows of a stage's weights times its token columns, KB blocks of 64.
// Rows 0-7 of MMA tile i start at w + i * tile_pitch, rows 8-15 hi bytes on; a K
// block's rows are kb_pitch bytes; its T token rows follow the block before's. Rows of
// 128 bytes, 16-byte chunk c of the row at 128 r at c ^ (r % 8): the eight rows that an
// ldmatrix phase reads are in different banks. Columns past T read the first
// token's row and are dropped later. (Boxes of 8 or 16 rows, zero-filled past T, took
// TMA's time for every row: it copies a row of 128 bytes in about 3 cycles.)
// PARTS 2: the tokens' rows are followed by T rows that are added to them (H in two parts).
template <int TILES, int NT, int KB, int PARTS = 1>
__device__ __forceinline__ void mma_stage(float (&acc)[TILES][NT][4], uint32_t w, uint32_t kb_pitch,
                                          uint32_t hi, uint32_t tile_pitch, uint32_t x, int T, int lane) {
  const uint32_t r = lane & 7;
  const uint32_t wr = w + ((lane >> 3) & 1) * hi + r * 128;
  uint32_t xr[PARTS][NT];  // the lane's token rows
#pragma unroll
  for (int p = 0; p < PARTS; ++p)
#pragma unroll
    for (int n = 0; n < NT; ++n) xr[p][n] = p * T + (static_cast<int>(n * 8 + r) < T ? n * 8 + r : 0);
  const uint32_t wc = lane >> 4, xc = lane >> 3;
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) {
    if (kb > 0)
#pragma unroll
      for (int p = 0; p < PARTS; ++p)
#pragma unroll
        for (int n = 0; n < NT; ++n) xr[p][n] += PARTS * T;
#pragma unroll
    for (int half = 0; half < 2; ++half) {  // 32 elements: two K steps of the MMA
      uint32_t b[PARTS][NT][4];
#pragma unroll
      for (int p = 0; p < PARTS; ++p)
#pragma unroll
        for (int n = 0; n < NT; ++n)
          ldmatrix4(b[p][n], x + xr[p][n] * 128 + (((half * 4 + xc) ^ (xr[p][n] & 7)) << 4));
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          uint32_t a[4];
          ldmatrix4(a, wr + kb * kb_pitch + i * tile_pitch + (((half * 4 + s * 2 + wc) ^ r) << 4));
#pragma unroll
          for (int p = 0; p < PARTS; ++p)
#pragma unroll
            for (int n = 0; n < NT; ++n) mma16816(acc[i][n], a, b[p][n][2 * s], b[p][n][2 * s + 1]);
        }
      }
    }
  }
}

__device__ __forceinline__ uint32_t cluster_ctas() {
  uint32_t n;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
  return n;
}
// A value to the same place in both CTAs of the pair.
__device__ __forceinline__ void store_both(float* p, uint32_t peer, float v) {
  *p = v;
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(mapa_shared(smem_u32(p), peer)), "f"(v) : "memory");
}

// The tables' header, the tokens' states and their delay rows into shared memory, by one warp
// while the router's products run.
__device__ __forceinline__ void load_states(Smem& s, const Args& a, int lane) {
  const int32_t* head = reinterpret_cast<const int32_t*>(a.tab);
  const int Eh = head[1], M = head[2];
  const float qbar = reinterpret_cast<const float*>(a.tab)[5];
  int home = 0, loc = 0;
  float q = 0.0f;
  if (lane < a.T) {
    home = a.home[lane];
    loc = a.loc != nullptr ? a.loc[lane] : home;  // no state given: first layer (Eq. 36)
    q = a.qhat != nullptr ? a.qhat[lane] : 0.0f;
  }
  const bool good = Eh == a.E && M > 0 && M <= ORDERMOE_MAX_SERVERS;
  if (lane == 0) {
    if (!good && blockIdx.x == 0) report(&g_err_route, ORDERMOE_DEV_BAD_INDEX, -1);
    s.tables_ok = good;
    s.qbar = qbar;
  }
  const bool placed = good && lane < a.T && home < M && loc < M;
  if (lane < TOKENS) {
    s.placed[lane] = placed;
    s.loc[lane] = static_cast<uint8_t>(loc);
    s.qhat[lane] = q;
  }
  const int row = placed ? (home * M + loc) * M : 0;
#pragma unroll 4
  for (int t = 0; t < a.T; ++t) {
    const int r = __shfl_sync(0xffffffffu, row, t);
    if (good && lane < M) s.delay[t][lane] = reinterpret_cast<const float*>(a.tab + off_a(a.E))[r + lane];
  }
}

// Qtab and Cq, one after the other in the tables and in shared memory, without a wait
// (copies_arrived); E odd: 8 bytes at the end.
__device__ __forceinline__ void copy_tables(const Args& a, float* s_Q, int t0, int nt) {
  const uint8_t* src = a.tab + kOffQtab;
  const uint32_t dst = smem_u32(s_Q);
  const int n = 8 * a.E * a.E;
  for (int i = t0 * 16; i + 16 <= n; i += nt * 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + i), "l"(src + i) : "memory");
  if (n % 16 != 0 && t0 == 0)
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst + n - 8), "l"(src + n - 8) : "memory");
}
__device__ __forceinline__ void copies_arrived() { asm volatile("cp.async.wait_all;" ::: "memory"); }

__device__ __forceinline__ void mma_warps_sync() {
  asm volatile("bar.sync 1, %0;" ::"n"(32 * MMA_WARPS) : "memory");
}

// The decisions in three steps on the MMA warps: the top-k, a warp a token; the candidates of
// every slot, whose costs hang on no other slot, eight lanes each; then the slots of a token in
// rank order on eight lanes, beside the gate weights in the other warps. What bounds it is the
// latency of dependent instructions at ten warps an SM.

// The k largest logits by (logit desc, index asc), as unsigned keys in their order, -0 as +0; 0 is
// below every key.
__device__ __forceinline__ void top_k(Smem& s, const Args& a, int t, int lane) {
  const float x0 = s.logits[0][t][lane] + s.logits[1][t][lane];
  const float x1 = s.logits[0][t][lane + 32] + s.logits[1][t][lane + 32];
  const bool nan = __any_sync(0xffffffffu, (lane < a.E && x0 != x0) || (lane + 32 < a.E && x1 != x1));
  auto key = [](float x) {
    const unsigned int u = __float_as_uint(x + 0.0f);
    return u >> 31 ? ~u : u | 0x80000000u;
  };
  unsigned int k0 = lane < a.E ? key(x0) : 0u, k1 = lane + 32 < a.E ? key(x1) : 0u;
  unsigned int lo = 0, hi = 0;
#pragma unroll 1
  for (int j = 0; j < a.k; ++j) {
    const unsigned int best = __reduce_max_sync(0xffffffffu, max(k0, k1));
    lo = __ballot_sync(0xffffffffu, k0 == best);
    hi = __ballot_sync(0xffffffffu, k1 == best);
    const int e = lo ? __ffs(lo) - 1 : __ffs(hi) + 31;
    if (lane == (e & 31)) {
      if (e < 32) k0 = 0u;
      else k1 = 0u;
      s.target[t * a.k + j] = e;
      s.weight[t * a.k + j] = e < 32 ? x0 : x1;  // the logit, until the weights are taken
    }
  }
  if (lane == 0) s.nan[t] = nan;
}

// A token's gate weights on eight lanes (sub): fp32 softmax over all E, summed in index order,
// the arithmetic of the router kernels, so the same logits give the same bits.
__device__ __forceinline__ void weigh(Smem& s, const Args& a, int t, int sub, int lane) {
  const int k = a.k;
  const bool in = t < a.T;  // (the others' rows hold nothing that is read)
  const float top = s.weight[t * k], mine = sub < k ? s.weight[t * k + sub] : 0.0f;
  __syncwarp();  // (read before the weights take the logits' place)
#pragma unroll 1
  for (int e = sub; e < a.E; e += 8) s.ex[t][e] = expf(s.logits[0][t][e] + s.logits[1][t][e] - top);
  if (a.E % 4 != 0 && sub == 0)
    for (int e = a.E; e % 4 != 0; ++e) s.ex[t][e] = 0.0f;
  __syncwarp();
  float denom = 0.0f;
#pragma unroll 4
  for (int c = 0; c < (a.E + 3) / 4; ++c) {  // past E: exact zeros
    const float4 x = *reinterpret_cast<const float4*>(&s.ex[t][4 * c]);
    denom += x.x;
    denom += x.y;
    denom += x.z;
    denom += x.w;
  }
  const float w = sub < k ? expf(mine - top) / denom : 0.0f;
  float sum = 0.0f;
#pragma unroll 1
  for (int j = 0; j < k; ++j) sum += __shfl_sync(0xffffffffu, w, (lane & 24) + j);
  if (in && sub < k) s.weight[t * k + sub] = s.nan[t] ? 0.0f : a.renorm ? w / sum : w;
}

// A candidate of a slot: the fp32 bits of its lowest cost over the servers that host it (none:
// all ones), then (substitute, away, server, expert) of it, and its loss.
struct Candidate {
  unsigned int cost, rest;
  float loss;
};

// The candidates of slot i = t k + j on eight lanes: the target, and its substitutes in turn.
__device__ __forceinline__ void candidates(const Smem& s, const SelSmem& sm, const Args& a, const float* s_Q,
                                           const float* s_Cq, Candidate* list, int i, int sub) {
  const int t = i / a.k, target = s.target[i], loc = s.loc[t], nsub = sm.nsub[target];
#pragma unroll 1
  for (int c = sub; c <= nsub; c += 8) {
    const int e = c == 0 ? target : sm.sublist[target * 64 + c - 1];
    const float loss = c == 0 ? 0.0f : s_Q[target * a.E + e], quality = c == 0 ? 0.0f : s_Cq[target * a.E + e];
    unsigned int best = ~0u, low = ~0u;
#pragma unroll 1
    for (uint32_t pm = sm.pmask[e]; pm; pm &= pm - 1) {
      const int m = __ffs(pm) - 1;
      const unsigned int cost = __float_as_uint(__fadd_rn(s.delay[t][m], quality));
      const unsigned int rest = (c != 0 ? 1u << 31 : 0u) | (m != loc ? 1u << 30 : 0u) |
                                static_cast<unsigned int>(m) << 8 | static_cast<unsigned int>(e);
      if (cost < best || (cost == best && rest < low)) {
        best = cost;
        low = rest;
      }
    }
    list[c] = Candidate{best, low, loss};
  }
}

// Alg. 2 of a token on eight lanes, slots in rank order: the costs, the order and the ties of
// select_slots. lists: the candidates of its slots.
__device__ __forceinline__ void decide(Smem& s, SelSmem& sm, const Args& a, const Candidate* lists, int t, int sub,
                                       int lane) {
  const int k = a.k;
  const bool in = t < a.T;
  if (!in) t = 0;
  const bool speaks = in && sub == 0 && blockIdx.x == 0, bad = s.nan[t] || !s.placed[t];
  if (speaks && bad) report(&g_err_route, s.nan[t] ? ORDERMOE_DEV_NAN_LOGIT : ORDERMOE_DEV_BAD_INDEX, t);
  const int mine = sub < k ? s.target[t * k + sub] : -1;
  unsigned long long taken = mine >= 0 ? 1ull << mine : 0ull;
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) taken |= __shfl_xor_sync(0xffffffffu, taken, o);
  const int loc = s.loc[t];
  const float qbar = s.qbar;
  float q = s.qhat[t];
  int first_server = loc;
#pragma unroll 1
  for (int j = 0; j < k; ++j) {
    const int target = __shfl_sync(0xffffffffu, mine, (lane & 24) + j), nsub = sm.nsub[target];
    unsigned long long best = ~0ull;
    float loss = 0.0f;
#pragma unroll 1
    for (int c = sub; c <= nsub; c += 8) {
      const Candidate v = lists[j * 64 + c];
      const unsigned long long key = static_cast<unsigned long long>(v.cost) << 32 | v.rest;
      const bool open = c == 0 || (!((taken >> (v.rest & 63u)) & 1ull) && __fadd_rn(q, v.loss) <= qbar);  // Eq. 40
      if (open && key < best) {
        best = key;
        loss = v.loss;
      }
    }
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) {
      const unsigned long long other = __shfl_xor_sync(0xffffffffu, best, o);
      const float its = __shfl_xor_sync(0xffffffffu, loss, o);
      if (other < best) {
        best = other;
        loss = its;
      }
    }
    const unsigned int rest = static_cast<unsigned int>(best);
    const bool none = best == ~0ull;
    const int issub = none ? 0 : rest >> 31;
    const int kd = none ? 0 : 2 * ((rest >> 30) & 1u) + issub;
    const int kstar = none ? target : rest & 0xFFu, mstar = none ? loc : (rest >> 8) & 0xFFu;
    if (issub) {
      taken |= 1ull << kstar;
      q = __fadd_rn(q, loss);
    }
    if (j == 0) first_server = mstar;
    if (speaks && !bad) {
      if (none) report(&g_err_route, ORDERMOE_DEV_NO_CANDIDATE, t);
      atomicAdd(&sm.kind[kd], 1);
    }
    if (in && sub == 0) {
      if (!bad) {
        atomicOr(&s.mask[kstar], 1u << t);
        s.slot[kstar][t] = static_cast<uint8_t>(j);
      }
      s.chosen[t * k + j] = bad ? -1 : kstar;
      s.server[t * k + j] = static_cast<uint8_t>(mstar);
      s.kind[t * k + j] = static_cast<uint8_t>(kd);
    }
  }
  if (in && sub == 0) s.valid[t] = !bad;
  if (in && sub == 0 && !bad) {
    s.loc[t] = static_cast<uint8_t>(first_server);
    s.qhat[t] = q;
  }
}

// The ring's position, the same walk in the producers and in the MMA warps. A slot belongs to one
// producer and to one MMA warp, which see its phases in order: a wait by parity tells only a
// phase from the next, and slots are not consumed in the order in which they are filled.
struct Ring {
  int slot = 0, stages;
  uint32_t phase = 0;
  __device__ __forceinline__ explicit Ring(int stages_) : stages(stages_) {}
  __device__ __forceinline__ void next() {
    if (++slot == stages) {
      slot = 0;
      phase ^= 1u;
    }
  }
};

// A CTA's contiguous share of the down stages: row tiles outer, chosen experts, then
// K stages. The first n CTAs have four stages or more each (a few MMA warps work at once and a
// row tile has fewer partials); stage i belongs to CTA ((i + 1) n - 1) / total.
struct Share {
  long long total, begin, end;
  int per_tile, per_expert, n;
  __device__ __forceinline__ Share(int d, int dff, int rows, int n_act, int c, int G) {
    per_expert = dff / (64 * KB_DOWN);
    per_tile = per_expert * n_act;
    total = static_cast<long long>(d / rows) * per_tile;
    n = total < 4ll * G ? static_cast<int>((total + 3) / 4) : G;
    begin = c < n ? total * c / n : total;
    end = c < n ? total * (c + 1) / n : total;
  }
  __device__ __forceinline__ int owner(long long i) const {
    return static_cast<int>(((i + 1) * n - 1) / total);
  }
};

// A walk over a share: row tile, chosen expert and K stage of the next one.
struct Walk {
  int tile, act, k;
  int left;  // stages: a share is at most 2^31 / G of them
  __device__ __forceinline__ explicit Walk(const Share& s) : tile(0), act(0), k(0) {
    left = static_cast<int>(s.end - s.begin);
    if (left > 0) {
      tile = static_cast<int>(s.begin / s.per_tile);
      const int r = static_cast<int>(s.begin - static_cast<long long>(tile) * s.per_tile);
      act = r / s.per_expert;
      k = r - act * s.per_expert;
    }
  }
  __device__ __forceinline__ void next(const Share& s, int n_act) {
    --left;
    if (++k == s.per_expert) {
      k = 0;
      if (++act == n_act) {
        act = 0;
        ++tile;
      }
    }
  }
};

template <int NT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1)
    few_tokens_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Args a) {
  using C = Cfg<NT>;
  const int STAGES = a.stages;
  extern __shared__ uint8_t smem_raw[];
  __shared__ Smem s;
  __shared__ SelSmem sm;
  uint8_t* ring = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  float* red = reinterpret_cast<float*>(ring + STAGES * C::STAGE_BYTES);
  float* s_Q = red + C::RED_FLOATS;
  float* s_Cq = s_Q + a.E * a.E;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int G = gridDim.x, cta = blockIdx.x;
  volatile int* abort = &s.abort;
  // The pair is the kernel's own, not only the launch's: without it the peer's shared memory is
  // no address. (A launch that a tool repeats may not carry every attribute.)
  if (cluster_ctas() != 2) {
    if (tid == 0) report(&g_err_route, ORDERMOE_DEV_BAD_INDEX, -3);
    return;
  }

  if (warp == MMA_WARPS + PRODUCERS && lane < static_cast<int>(sizeof(Maps) / sizeof(CUtensorMap)))
    tma_prefetch_map(reinterpret_cast<const CUtensorMap*>(&maps) + lane);
  if (warp == 0) {  // a barrier a lane
    if (lane < STAGES) {
      mbar_init(&s.full[lane], 1);
      mbar_init(&s.empty[lane], 1);
    }
    if (lane < 3) {
      mbar_init(&s.red_full[lane], MMA_WARPS);
      mbar_init(&s.red_empty[lane], 1);
    }
    if (lane < 4) sm.kind[lane] = 0;
    if (lane == 0) {
      s.abort = 0;
      s.zero = 0;
    }
    fence_mbar_init();
  }
  if (warp == 1) s.mask[lane] = s.mask[lane + 32] = 0;
  cluster_sync();  // both CTAs run: the peer's shared memory may be written

  Ring ring_at(STAGES);          // producer and MMA warps
  uint32_t units = 0, rows = 0;  // hand-overs to the epilogue warp so far: units, row tiles
  using MTc = std::integral_constant<int, MT>;        // MMA tiles of a unit
  using MT2c = std::integral_constant<int, 2 * MT>;   // and of a row tile
  uint32_t issued_mask = 0, last_phase_bits = 0;  // the producer's, for the drain after an abort
  const uint32_t ring0 = smem_u32(ring);
  const int k_up = a.d / (64 * KB_UP);

  // --- roles' steps
  auto timeout = [&](int where) {
    if (!*abort) report(&g_err_route, ORDERMOE_DEV_WAIT_TIMEOUT, where);
    *abort = 1;
  };
  // The producer walks the stages as a converged warp and one elected lane issues: a lane
  // walking alone took about 550 cycles a stage whatever its bytes (1 token on 8 wide
  // experts 190 us).
  // Two of them take the slots in turn: one issued a stage of two or three boxes in about 0.17
  // us, 8 KB of weights at the rate of HBM.
  const bool issuer = elect_one();
  const int producer = warp >= MMA_WARPS && warp < MMA_WARPS + PRODUCERS ? warp - MMA_WARPS : -1;
  auto mine = [&]() { return ring_at.slot % PRODUCERS == producer; };
  auto claim = [&](uint32_t bytes) {  // the next slot, its barrier set; false: give up
    if (!__all_sync(0xffffffffu, mbar_wait(&s.empty[ring_at.slot], ring_at.phase ^ 1u, a.limit_ns, abort))) {
      if (issuer) timeout(31);
      return false;
    }
    if (issuer) mbar_arrive_expect_tx(&s.full[ring_at.slot], bytes);
    issued_mask |= 1u << ring_at.slot;
    last_phase_bits = (last_phase_bits & ~(1u << ring_at.slot)) | (ring_at.phase << ring_at.slot);
    return true;
  };
  auto slot_ptr = [&](int slot) { return ring + slot * C::STAGE_BYTES; };
  // an MMA warp: its stage has arrived / has been read
  auto arrived = [&]() {
    const bool ok = __all_sync(0xffffffffu, mbar_wait(&s.full[ring_at.slot], ring_at.phase, a.limit_ns, abort));
    if (!ok && lane == 0) timeout(32);
    return ok;
  };
  auto release = [&]() {
    __syncwarp();
    if (lane == 0) mbar_arrive(&s.empty[ring_at.slot]);
  };
  // MMA warps hand a unit's accumulators (two sets in turn), or a row tile's (one set over
  // the same memory), to the epilogue warp. `n` such hand-overs came before.
  auto wait_empty = [&](int b, uint32_t parity) {
    const bool ok = __all_sync(0xffffffffu, mbar_wait(&s.red_empty[b], parity, a.limit_ns, abort));
    if (!ok && lane == 0) timeout(33);
    return ok;
  };
  auto put = [&](auto& acc, auto tiles, int set, int b) {
    constexpr int TILES = decltype(tiles)::value;
    float4* dst = reinterpret_cast<float4*>(red) + (set * MMA_WARPS + warp) * (TILES * NT * 32) + lane;
#pragma unroll
    for (int i = 0; i < TILES; ++i)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        dst[(i * NT + n) * 32] = make_float4(acc[i][n][0], acc[i][n][1], acc[i][n][2], acc[i][n][3]);
        acc[i][n][0] = acc[i][n][1] = acc[i][n][2] = acc[i][n][3] = 0.0f;
      }
    __syncwarp();
    if (lane == 0) mbar_arrive(&s.red_full[b]);
  };
  auto put_unit = [&](auto& acc) {
    const int b = units & 1;
    if (!wait_empty(b, ((units >> 1) & 1u) ^ 1u)) return false;
    put(acc, MTc{}, b, b);
    ++units;
    return true;
  };
  auto put_tile = [&](auto& acc) {
    if (rows == 0) {  // both of the units' sets have been read
      for (int b = 0; b < 2; ++b) {
        const uint32_t uses = (units + 1 - b) >> 1;
        if (uses > 0 && !wait_empty(b, (uses - 1) & 1u)) return false;
      }
    } else if (!wait_empty(2, (rows - 1) & 1u)) {
      return false;
    }
    put(acc, MT2c{}, 0, 2);
    ++rows;
    return true;
  };
  // the epilogue warp: body(i, n, sum over the MMA warps in warp order)
  auto take = [&](auto tiles, int set, int b, uint32_t parity, auto body) {
    constexpr int TILES = decltype(tiles)::value;
    const bool ok = __all_sync(0xffffffffu, mbar_wait(&s.red_full[b], parity, a.limit_ns, abort));
    if (!ok) {
      if (lane == 0) timeout(34);
      return false;
    }
    const float4* src = reinterpret_cast<const float4*>(red) + set * MMA_WARPS * (TILES * NT * 32) + lane;
#pragma unroll
    for (int i = 0; i < TILES; ++i)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float4 v = src[(i * NT + n) * 32];
#pragma unroll
        for (int w = 1; w < MMA_WARPS; ++w) {
          const float4 u = src[(w * TILES * NT + i * NT + n) * 32];
          v.x += u.x;
          v.y += u.y;
          v.z += u.z;
          v.w += u.w;
        }
        body(i, n, v);
      }
    __syncwarp();
    if (lane == 0) mbar_arrive(&s.red_empty[b]);
    return true;
  };
  auto take_unit = [&](auto body) {
    const int b = units & 1;
    const uint32_t parity = (units >> 1) & 1u;
    ++units;
    return take(MTc{}, b, b, parity, body);
  };
  auto take_tile = [&](auto body) {
    const uint32_t parity = rows & 1u;
    ++rows;
    return take(MT2c{}, 0, 2, parity, body);
  };
  // ---------------------------------------------------------------- route
  const uint32_t rank = cluster_ctarank();
  auto route = [&](auto row_tiles) {
    // stages of all experts' rows (RT tiles of 16) by KB blocks of K, the first half of them in
    // rank 0
    constexpr int RT = decltype(row_tiles)::value, KB = route_kb(RT);
    constexpr uint32_t W = RT * 2048 * KB;
    const int all = a.d / (64 * KB), half = (all + 1) / 2;
    const int s0 = rank == 0 ? 0 : half, s1 = rank == 0 ? half : all;
    if (producer >= 0) {
      bool ok = true;
      for (int i = s0; i < s1 && ok; ++i) {
        if (mine() && (ok = claim(W + a.T * KB * 128)) && issuer) {
          uint8_t* p = slot_ptr(ring_at.slot);
          tma_load_3d(p, &maps.Wr, &s.full[ring_at.slot], 0, i * KB);
          tma_load_3d(p + C::W_BYTES, &maps.Xr, &s.full[ring_at.slot], 0, i * KB);
        }
        ring_at.next();
      }
    } else if (warp < MMA_WARPS) {
      uint32_t pm = 0;
      unsigned long long sb = 0;
      if (tid < 64) {
        pm = reinterpret_cast<const uint32_t*>(a.tab + kOffPmask)[tid];
        sb = reinterpret_cast<const unsigned long long*>(a.tab + kOffSubst)[tid];
      }
      copy_tables(a, s_Q, tid, 32 * MMA_WARPS);
      float acc[RT][NT][4] = {};
      bool ok = true;
      for (int i = s0; i < s1; ++i) {
        if (ring_at.slot % MMA_WARPS == warp) {
          if (!(ok = arrived())) break;
          const uint32_t w = ring0 + ring_at.slot * C::STAGE_BYTES;
          mma_stage<RT, NT, KB>(acc, w, 2048 * RT, 1024, 2048, w + C::W_BYTES, a.T, lane);
          release();
        }
        ring_at.next();
      }
      if (ok) put(acc, row_tiles, 0, 0);
      ++units;
      if (tid < 64) {
        sm.pmask[tid] = pm;
        int n = 0;
#pragma unroll 1
        for (; sb; sb &= sb - 1) sm.sublist[tid * 64 + n++] = static_cast<uint8_t>(__ffsll(static_cast<long long>(sb)) - 1);
        sm.nsub[tid] = n;
      }
      copies_arrived();
    } else {
      load_states(s, a, lane);
      take(row_tiles, 0, 0, 0, [&](int m, int n, float4 v) {
        const int e = m * 16 + (lane >> 2), t = n * 8 + (lane & 3) * 2;
        float* p = &s.logits[rank][t][e];
        if (e < a.E) {
          store_both(p, rank ^ 1u, v.x);
          store_both(p + 68, rank ^ 1u, v.y);
        }
        if (e + 8 < a.E) {
          store_both(p + 8, rank ^ 1u, v.z);
          store_both(p + 68 + 8, rank ^ 1u, v.w);
        }
      });
      ++units;
    }
  };
  if (!a.given) {
    if (a.E <= 16) route(std::integral_constant<int, 1>{});
    else if (a.E <= 32) route(std::integral_constant<int, 2>{});
    else route(std::integral_constant<int, 4>{});
    cluster_sync();  // the peer's half of the logits is here
    if (warp < MMA_WARPS) {
      Candidate* lists = reinterpret_cast<Candidate*>(ring);  // [T * k][64]
      const int group = warp * 4 + (lane >> 3), sub = lane & 7;
#pragma unroll 1
      for (int t = warp; t < a.T; t += MMA_WARPS) top_k(s, a, t, lane);
      mma_warps_sync();
      const bool tables_ok = s.tables_ok;
      if (tables_ok)
#pragma unroll 1
        for (int i = group; i < a.T * a.k; i += 4 * MMA_WARPS)
          candidates(s, sm, a, s_Q, s_Cq, lists + i * 64, i, sub);
      mma_warps_sync();
      // four warps decide, four weigh: four tokens each
      static_assert(MMA_WARPS * 2 == TOKENS, "four tokens a warp");
      const int t = group % TOKENS;
      if (group >= TOKENS) weigh(s, a, t, sub, lane);
      else if (tables_ok) decide(s, sm, a, lists + (t < a.T ? t : 0) * a.k * 64, t, sub, lane);
      else if (t < a.T && sub < a.k) s.valid[t] = 0;
      fence_proxy_async();  // the ring's memory is TMA's again
    }
  } else if (tid < a.T) {  // decided by the look-ahead; a NaN token has no targets
    bool ok = a.topk_idx[tid * a.k] >= 0;
    for (int j = 0; j < a.k; ++j) {
      const int e = a.chosen[tid * a.k + j];
      ok = ok && e >= 0 && e < a.E;
      s.weight[tid * a.k + j] = a.topk_w[tid * a.k + j];
    }
    for (int j = 0; j < a.k && ok; ++j) {  // its experts are distinct
      const int e = a.chosen[tid * a.k + j];
      atomicOr(&s.mask[e], 1u << tid);
      s.slot[e][tid] = static_cast<uint8_t>(j);
    }
    s.valid[tid] = ok;
  }
  __syncthreads();
  // the chosen experts in ascending order, the same in every warp
  int n_act;
  {
    const bool lo = s.mask[lane] != 0, hi = s.mask[lane + 32] != 0;
    const unsigned int l = __ballot_sync(0xffffffffu, lo), h = __ballot_sync(0xffffffffu, hi);
    const unsigned int before = (1u << lane) - 1;
    if (lo) s.act[__popc(l & before)] = static_cast<uint8_t>(lane);
    if (hi) s.act[__popc(l) + __popc(h & before)] = static_cast<uint8_t>(lane + 32);
    n_act = *abort ? 0 : __popc(l) + __popc(h);
    __syncwarp();
  }

  // -------------------------------------------------------------- gate/up
  const int per = a.dff / (8 * MT);  // units of an expert
  const int n_units = n_act * per;
  const Share share(a.d, a.dff, C::DOWN_ROWS, n_act, cta, G);
  if (producer >= 0) {
    bool ok = true;
    for (int u = cta; u < n_units && ok; u += G) {
      const int row = s.act[u / per] * a.dff + (u % per) * 8 * MT;
      for (int kb = 0; kb < k_up && ok; ++kb) {
        if (mine() && (ok = claim(C::W_BYTES + a.T * KB_UP * 128)) && issuer) {
          uint8_t* p = slot_ptr(ring_at.slot);
          tma_load_3d(p, &maps.W1, &s.full[ring_at.slot], row, kb * KB_UP);
          tma_load_3d(p + C::W_BYTES / 2, &maps.W3, &s.full[ring_at.slot], row, kb * KB_UP);
          tma_load_3d(p + C::W_BYTES, &maps.X, &s.full[ring_at.slot], 0, kb * KB_UP);
        }
        ring_at.next();
      }
    }
    // down: the weights of a stage as soon as its slot is free, H behind the barrier
    // that every CTA's gate/up passes
    const uint32_t bytes = C::W_BYTES + 2 * a.T * KB_DOWN * 128;
    Walk w(share), hw(share);
    Ring first = ring_at;
    auto load_w = [&]() {
      if (issuer)
        tma_load_3d(slot_ptr(ring_at.slot), &maps.W2, &s.full[ring_at.slot],
                    s.act[w.act] * a.d + w.tile * C::DOWN_ROWS, w.k * KB_DOWN);
    };
    auto load_h = [&]() {
      if (issuer)
        tma_load_3d(slot_ptr(first.slot) + C::W_BYTES, &maps.H, &s.full[first.slot], hw.act * 2 * a.T,
                    hw.k * KB_DOWN);
    };
    auto next_w = [&]() {
      ring_at.next();
      w.next(share, n_act);
    };
    auto next_h = [&]() {
      first.next();
      hw.next(share, n_act);
    };
    while (ok && w.left > 0 && hw.left - w.left < STAGES) {
      if (mine()) {
        if (!(ok = claim(bytes))) break;
        load_w();
      }
      next_w();
    }
    if (ok) {
      const bool up = !issuer || grid_wait(&a.sync[0], G, a.limit_ns, abort);
      if (!up) timeout(35);
      ok = __all_sync(0xffffffffu, up);
    }
    fence_proxy_async();
    // (also after a failure: the barriers of the stages under way expect these bytes)
    while (hw.left > w.left) {
      if (first.slot % PRODUCERS == producer) load_h();
      next_h();
    }
    while (ok && w.left > 0) {
      if (mine()) {
        if (!(ok = claim(bytes))) break;
        load_w();
        load_h();
      }
      next_w();
      next_h();
    }
  } else if (warp < MMA_WARPS) {
    bool ok = true;
    {
      float acc[MT][NT][4] = {};
      for (int u = cta; u < n_units && ok; u += G) {
        for (int kb = 0; kb < k_up; ++kb) {
          if (ring_at.slot % MMA_WARPS == warp) {
            if (!(ok = arrived())) break;
            const uint32_t w = ring0 + ring_at.slot * C::STAGE_BYTES;
            mma_stage<MT, NT, KB_UP>(acc, w, 1024 * MT, 4096 * MT, 1024, w + C::W_BYTES, a.T, lane);
            release();
          }
          ring_at.next();
        }
        ok = ok && put_unit(acc);
      }
    }
    float acc[2 * MT][NT][4] = {}, tot[2 * MT][NT][4] = {};
    bool any = false;
    for (Walk w(share); w.left > 0 && ok;) {
      if (ring_at.slot % MMA_WARPS == warp) {
        if (!(ok = arrived())) break;
        const uint32_t p = ring0 + ring_at.slot * C::STAGE_BYTES;
        mma_stage<2 * MT, NT, KB_DOWN, 2>(acc, p, 4096 * MT, 1024, 2048, p + C::W_BYTES, a.T, lane);
        release();
        any = true;
      }
      ring_at.next();
      const int act = w.act, tile = w.tile;
      w.next(share, n_act);
      if (any && (w.k == 0 || w.left == 0)) {
        // the expert's sums to the tokens that use it
        const int e = s.act[act];
        const unsigned int m = s.mask[e];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const int t = n * 8 + (lane & 3) * 2;
          const bool u0 = (m >> t) & 1u, u1 = (m >> (t + 1)) & 1u;
          const float g0 = u0 ? s.weight[t * a.k + s.slot[e][t]] : 0.0f;
          const float g1 = u1 ? s.weight[(t + 1) * a.k + s.slot[e][t + 1]] : 0.0f;
#pragma unroll
          for (int j = 0; j < 2 * MT; ++j) {
            float (&c)[4] = acc[j][n];
            float (&o)[4] = tot[j][n];
            o[0] = u0 ? fmaf(g0, c[0], o[0]) : o[0];
            o[1] = u1 ? fmaf(g1, c[1], o[1]) : o[1];
            o[2] = u0 ? fmaf(g0, c[2], o[2]) : o[2];
            o[3] = u1 ? fmaf(g1, c[3], o[3]) : o[3];
            c[0] = c[1] = c[2] = c[3] = 0.0f;
          }
        }
        any = false;
      }
      if (w.tile != tile || w.left == 0) ok = put_tile(tot);
    }
  } else {
    if (cta == 0 && !a.given && !*abort) {  // one warp of the grid writes the decisions
      for (int i = lane; i < a.T * a.k; i += 32) {
        const bool ok = s.valid[i / a.k], nan = s.nan[i / a.k];
        a.topk_idx[i] = nan ? -1 : s.target[i];
        a.topk_w[i] = s.weight[i];
        if (ok) {
          a.chosen[i] = s.chosen[i];
          a.server[i] = s.server[i];
          a.kind[i] = s.kind[i];
        }
      }
      if (a.logits != nullptr)
        for (int t = 0; t < a.T; ++t)
          for (int e = lane; e < a.E; e += 32) a.logits[t * a.E + e] = s.logits[0][t][e] + s.logits[1][t][e];
      if (a.counters != nullptr && lane < 4 && sm.kind[lane]) atomicAdd(&a.counters[lane], sm.kind[lane]);
    }
    bool ok = true;
    for (int u = cta; u < n_units && ok; u += G) {
      const int e = u / per, f0 = (u - e * per) * 8 * MT + (lane >> 2);
      ok = take_unit([&](int m, int n, float4 v) {
        // rows 0-7 gate, 8-15 up: silu(g) u as the sum of two bf16 (16 bits: one bf16 would double
        // the error of y, and flip roundings of h_out that the next norm carries on; at a few
        // tokens the second part costs no time, HBM bounds it). The fast exponential is (2 + 1.2 |g|) 2^-23
        // off, below the two parts' 2^-16 for |g| < 100.
        const int t = n * 8 + (lane & 3) * 2;
        uint16_t* out = a.H + (static_cast<size_t>(e) * 2 * a.T + t) * a.dff + f0 + m * 8;
        const float h0 = v.x / (1.0f + __expf(-v.x)) * v.z, h1 = v.y / (1.0f + __expf(-v.y)) * v.w;
        const uint32_t hi = pack_bf16x2(h0, h1);
        const float r0 = h0 - bf16_lo(hi), r1 = h1 - bf16_hi(hi);
        // (an infinite part has no rest)
        const uint32_t lo = pack_bf16x2(isfinite(r0) ? r0 : 0.0f, isfinite(r1) ? r1 : 0.0f);
        const size_t rest = static_cast<size_t>(a.T) * a.dff;
        if (t < a.T) {
          out[0] = static_cast<uint16_t>(hi & 0xFFFFu);
          out[rest] = static_cast<uint16_t>(lo & 0xFFFFu);
        }
        if (t + 1 < a.T) {
          out[a.dff] = static_cast<uint16_t>(hi >> 16);
          out[rest + a.dff] = static_cast<uint16_t>(lo >> 16);
        }
      });
    }
    fence_proxy_async();  // H is read by the other CTAs' TMA loads
    __syncwarp();
    if (lane == 0) {
      __threadfence();
      atomicAdd(&a.sync[0], 1u);
    }
    long long i = share.begin;
    while (ok && i < share.end) {
      const int tile = static_cast<int>(i / share.per_tile);
      float* out = a.part + static_cast<size_t>(tile + cta) * a.T * C::DOWN_ROWS + (lane >> 2);
      ok = take_tile([&](int m, int n, float4 v) {
        const int t = n * 8 + (lane & 3) * 2;
        float* o = out + t * C::DOWN_ROWS + m * 16;
        if (t < a.T) {
          o[0] = v.x;
          o[8] = v.z;
        }
        if (t + 1 < a.T) {
          o[C::DOWN_ROWS] = v.y;
          o[C::DOWN_ROWS + 8] = v.w;
        }
      });
      i = static_cast<long long>(tile + 1) * share.per_tile;
    }
    __syncwarp();
    if (lane == 0) {
      __threadfence();
      atomicAdd(&a.sync[1], 1u);
    }
  }
  __syncthreads();

  // ---------------------------------------------------------------- finish
  // On the residual map a CTA a token (its norm is a sum over the row), otherwise every token's
  // columns over G / T CTAs.
  const int parts = a.h != nullptr ? 1 : max(1, G / a.T);
  // Thread 0 leaves the counters behind its CTA's last wait, not behind its last store; the answer is not
  // needed before the end (8 experts, d 256: 8 tokens 18.5 -> 17.8 us, 16 tokens 23.9 -> 22.8).
  unsigned int before = 0;
  if (tid == 0 && cta >= a.T * parts) before = atomicAdd(&a.sync[2], 1u);
  if (cta < a.T * parts) {
    const int tiles = a.d / C::DOWN_ROWS, part = cta / a.T;
    const int first_tile = tiles * part / parts, last_tile = tiles * (part + 1) / parts;
    // the first and last owner of every row tile, while the others finish (the ring is free)
    int16_t* own = reinterpret_cast<int16_t*>(ring);
    uint2* s_row = reinterpret_cast<uint2*>(ring + MAX_D / C::DOWN_ROWS * 4);  // the token's row of h_out
    if (share.total > 0)
      for (int i = first_tile + tid; i < last_tile; i += THREADS) {
        own[2 * i] = static_cast<int16_t>(share.owner(static_cast<long long>(i) * share.per_tile));
        own[2 * i + 1] = static_cast<int16_t>(share.owner(static_cast<long long>(i + 1) * share.per_tile - 1));
      }
    if (tid == 0) {
      if (!grid_wait(&a.sync[1], G, a.limit_ns, abort)) timeout(36);
      before = atomicAdd(&a.sync[2], 1u);
    }
    __syncthreads();
    for (int t = cta % a.T; t < a.T && !*abort; t += G) {
      if (!s.valid[t]) continue;
      float sq = 0.0f;
      const size_t row = static_cast<size_t>(t) * a.d, pitch = static_cast<size_t>(a.T) * C::DOWN_ROWS;
      const int end = last_tile * C::DOWN_ROWS;
      // four groups of columns a thread, four partials of each: sixteen loads under way
#pragma unroll 1
      for (int c = first_tile * C::DOWN_ROWS + tid * 4; c < end; c += 4 * THREADS * 4) {
        const float* p[4];
        int n[4];
        uint2 hv[4];
        float4 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int cj = c + j * THREADS * 4, tile = cj / C::DOWN_ROWS;
          int c0 = 0, c1 = -1;
          if (cj < end) {
            c0 = own[2 * tile];
            c1 = own[2 * tile + 1];
          }
          n[j] = c1 - c0 + 1;
          p[j] = a.part + (static_cast<size_t>(tile + c0) * a.T + t) * C::DOWN_ROWS + cj % C::DOWN_ROWS;
          hv[j] = make_uint2(0, 0);
          if (a.h != nullptr && cj < end) hv[j] = *reinterpret_cast<const uint2*>(a.h + row + cj);
          v[j] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
        const int most = max(max(n[0], n[1]), max(n[2], n[3]));
#pragma unroll 1
        for (int q = 0; q < most; q += 4) {
          float4 u[4][4];
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (q + i < n[j]) u[j][i] = __ldcg(reinterpret_cast<const float4*>(p[j] + (q + i) * pitch));
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (q + i < n[j]) {
                v[j].x += u[j][i].x;
                v[j].y += u[j][i].y;
                v[j].z += u[j][i].z;
                v[j].w += u[j][i].w;
              }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int cj = c + j * THREADS * 4;
          if (cj >= end) continue;
          v[j].x += bf16_lo(hv[j].x);
          v[j].y += bf16_hi(hv[j].x);
          v[j].z += bf16_lo(hv[j].y);
          v[j].w += bf16_hi(hv[j].y);
          const uint2 o = make_uint2(pack_bf16x2(v[j].x, v[j].y), pack_bf16x2(v[j].z, v[j].w));
          *reinterpret_cast<uint2*>(a.y + row + cj) = o;
          s_row[cj / 4] = o;
          const float f[4] = {bf16_lo(o.x), bf16_hi(o.x), bf16_lo(o.y), bf16_hi(o.y)};
#pragma unroll
          for (int i = 0; i < 4; ++i) sq = fmaf(f[i], f[i], sq);
        }
      }
      if (a.h == nullptr) continue;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
      __syncthreads();  // s.sum of the token before has been read
      if (lane == 0) s.sum[warp] = sq;
      __syncthreads();
      float total = 0.0f;
#pragma unroll
      for (int w = 0; w < THREADS / 32; ++w) total += s.sum[w];
      const float r = 1.0f / sqrtf(total / static_cast<float>(a.d) + a.eps);
      for (int c = tid * 4; c < a.d; c += THREADS * 4) {  // each thread's own columns again
        const uint2 o = s_row[c / 4];
        *reinterpret_cast<uint2*>(a.x_out + row + c) =
            make_uint2(pack_bf16x2(bf16_lo(o.x) * r, bf16_hi(o.x) * r),
                       pack_bf16x2(bf16_lo(o.y) * r, bf16_hi(o.y) * r));
      }
    }
    // the tokens' new state, once every CTA has read the old one
    if (cta == 0 && a.loc != nullptr && !a.given && !*abort && tid < a.T && s.valid[tid]) {
      a.loc[tid] = s.loc[tid];
      a.qhat[tid] = s.qhat[tid];
    }
  }
  __syncthreads();
  if (s.abort && producer >= 0 && issuer) {  // every copy that this CTA issued (bounded)
    volatile int* never = &s.zero;
    for (int i = 0; i < STAGES; ++i)
      if ((issued_mask >> i) & 1u) mbar_wait(&s.full[i], (last_phase_bits >> i) & 1u, a.limit_ns, never);
  }
  // the last CTA that left the counters sets them back (none accesses its peer's memory here)
  if (tid == 0 && before == static_cast<unsigned int>(G) - 1) a.sync[0] = a.sync[1] = a.sync[2] = 0;
}

}  // namespace fw

static size_t up256(size_t v) { return (v + 255) & ~size_t(255); }

// The workspace: counters, H, partial sums, and the decisions of a call that keeps none.
struct FewScratch {
  unsigned int* sync;
  uint16_t* H;
  float *part, *topk_w;
  int32_t *topk_idx, *chosen;
  uint8_t *server, *kind;
  size_t bytes;
};

// SMs at most: the partial sums have a place for every CTA of a launch.
constexpr int kFewMaxCtas = 256;

static FewScratch few_carve(uint8_t* base, int T, int E, int d, int dff, int k) {
  FewScratch s{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    uint8_t* p = base ? base + off : nullptr;
    off += up256(bytes);
    return p;
  };
  const size_t R = (size_t)T * k, act = R < (size_t)E ? R : (size_t)E;
  s.sync = reinterpret_cast<unsigned int*>(take(16));
  s.H = reinterpret_cast<uint16_t*>(take(act * 2 * T * dff * 2));
  // a row tile's partials, one for each CTA more
  constexpr int rows = fw::Cfg<1>::DOWN_ROWS;
  s.part = reinterpret_cast<float*>(take(((size_t)d / rows + kFewMaxCtas) * T * rows * 4));
  s.topk_w = reinterpret_cast<float*>(take(R * 4));
  s.topk_idx = reinterpret_cast<int32_t*>(take(R * 4));
  s.chosen = reinterpret_cast<int32_t*>(take(R * 4));
  s.server = take(R);
  s.kind = take(R);
  s.bytes = off;
  return s;
}

template <int NT>
static cudaError_t few_attr() {
  return cudaFuncSetAttribute(fw::few_tokens_kernel<NT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              227 * 1024 - static_cast<int>(sizeof(fw::Smem) + sizeof(SelSmem)) - 256);
}

template <int NT>
static int few_launch(const ordermoe_layer_desc* L, const uint16_t* X, fw::Args& a, cudaStream_t stream) {
  using C = fw::Cfg<NT>;
  static PerDevice cache;
  const cudaError_t ae = static_cast<cudaError_t>(per_device(cache, [] {
    return static_cast<int>(few_attr<NT>());
  }));
  if (ae != cudaSuccess) return cuda_fail(ae, "cudaFuncSetAttribute(few_tokens_kernel)");
  const int R = a.T * a.k, act = R < a.E ? R : a.E;
  fw::Maps m;
  int rc;
  const int rt = a.E <= 16 ? 1 : a.E <= 32 ? 2 : 4, kb = fw::route_kb(rt);  // as the kernel's route
  if ((rc = make_tmap_bf16_kb(&m.Wr, L->W_r, a.E, a.d, 16 * rt, kb))) return rc;
  if ((rc = make_tmap_bf16_kb(&m.Xr, X, a.T, a.d, a.T, kb))) return rc;
  if ((rc = make_tmap_bf16_kb(&m.X, X, a.T, a.d, a.T, fw::KB_UP))) return rc;
  if ((rc = make_tmap_bf16_kb(&m.W1, L->W1, (uint64_t)a.E * a.dff, a.d, 8 * fw::MT, fw::KB_UP))) return rc;
  if ((rc = make_tmap_bf16_kb(&m.W3, L->W3, (uint64_t)a.E * a.dff, a.d, 8 * fw::MT, fw::KB_UP))) return rc;
  if ((rc = make_tmap_bf16_kb(&m.W2, L->W2, (uint64_t)a.E * a.d, a.dff, C::DOWN_ROWS, fw::KB_DOWN))) return rc;
  if ((rc = make_tmap_bf16_kb(&m.H, a.H, (uint64_t)act * 2 * a.T, a.dff, 2 * a.T, fw::KB_DOWN))) return rc;
  a.stages = fw::stages<NT>(a.E);
  // a CTA per SM, fewer where there are not as many units of gate/up
  int grid = num_sms() < kFewMaxCtas ? num_sms() : kFewMaxCtas;
  const long long units = (long long)act * (a.dff / (8 * fw::MT));
  if (units < grid) grid = static_cast<int>(units);
  grid = (grid < a.T ? a.T : grid) / 2 * 2;  // pairs
  if (grid < 2) grid = 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid, 1, 1);
  cfg.blockDim = dim3(fw::THREADS, 1, 1);
  cfg.dynamicSmemBytes = a.stages * C::STAGE_BYTES + C::other_bytes(a.E);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeCooperative;  // the CTAs wait for one another: all or none run
  attr[0].val.cooperative = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, fw::few_tokens_kernel<NT>, m, a);
  if (e != cudaSuccess) return cuda_fail(e, "few_tokens_kernel");
  OM_LAUNCHED("few_tokens_kernel");
  return ORDERMOE_OK;
}

static int few_layer(const char* who, const ordermoe_layer_desc* L, int T, const uint16_t* X, const uint16_t* h,
                     const uint8_t* home, uint8_t* loc, float* qhat, float eps, uint16_t* y, uint16_t* x_out,
                     const ordermoe_few_out* out, void* workspace, size_t workspace_bytes,
                     cudaStream_t stream) {
  if (!L) return fail(ORDERMOE_ERR_INVALID_ARG, "%s: null layer", who);
  if (T < 0) return fail(ORDERMOE_ERR_INVALID_ARG, "%s: T < 0", who);
  if (T > ORDERMOE_FEW_TOKENS)
    return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "%s: at most %d tokens", who, ORDERMOE_FEW_TOKENS);
  if (L->E <= 0 || L->E > ORDERMOE_MAX_EXPERTS || L->k <= 0 || L->k > ORDERMOE_MAX_TOPK || L->k > L->E)
    return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "%s: need 1 <= k <= min(E, 8), E <= 64", who);
  if (L->d <= 0 || L->d % 256 != 0 || L->dff <= 0 || L->dff % 128 != 0)
    return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "%s: need d %% 256 == 0 and dff %% 128 == 0", who);
  if (L->d > fw::MAX_D) return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "%s: need d <= %d", who, fw::MAX_D);
  if ((long long)L->E * L->dff > INT32_MAX || (long long)L->E * L->d > INT32_MAX)
    return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "%s: sizes too large", who);
  if (L->lookahead_H > 4) return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "%s: look-ahead of at most 4 layers", who);
  if (L->lookahead_H > 1 &&
      (!L->P || L->tables_stride < om::tables_bytes(L->E, 1) || L->tables_stride % 16 != 0))
    return fail(ORDERMOE_ERR_INVALID_ARG, "%s: look-ahead needs P and a table stride of a multiple of 16", who);
  if (!L->W_r || !L->W1 || !L->W3 || !L->W2 || !L->tables)
    return fail(ORDERMOE_ERR_INVALID_ARG, "%s: null pointer in the layer", who);
  if (!aligned16(L->W_r) || !aligned16(L->W1) || !aligned16(L->W3) || !aligned16(L->W2) || !aligned16(L->tables))
    return fail(ORDERMOE_ERR_INVALID_ARG, "%s: weights and tables must be 16-byte aligned", who);
  if (L->tables_bytes < om::tables_bytes(L->E, 1))
    return fail(ORDERMOE_ERR_INVALID_ARG, "%s: tables buffer smaller than E needs", who);
  if (T == 0) return ORDERMOE_OK;
  const bool res = h != nullptr;
  if (!X || !home || !y) return fail(ORDERMOE_ERR_INVALID_ARG, "%s: null input or output", who);
  if (!aligned16(X) || !aligned16(y) || (res && (!aligned16(h) || !aligned16(x_out))))
    return fail(ORDERMOE_ERR_INVALID_ARG, "%s: rows of d must be 16-byte aligned", who);
  if ((loc == nullptr) != (qhat == nullptr))
    return fail(ORDERMOE_ERR_INVALID_ARG, "%s: give both loc and qhat, or neither", who);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 ||
      workspace_bytes < ordermoe_layer_few_workspace_bytes(T, L->E, L->d, L->dff, L->k))
    return fail(ORDERMOE_ERR_INVALID_ARG, "%s: workspace null, too small or not 256-byte aligned", who);
  const FewScratch s = few_carve(static_cast<uint8_t*>(workspace), T, L->E, L->d, L->dff, L->k);
  const ordermoe_few_out o = out ? *out : ordermoe_few_out{};
  fw::Args a{};
  a.T = T; a.E = L->E; a.d = L->d; a.dff = L->dff; a.k = L->k; a.renorm = L->renorm;
  a.tab = static_cast<const uint8_t*>(L->tables);
  a.home = home; a.loc = loc; a.qhat = qhat;
  a.h = h; a.y = y; a.x_out = x_out; a.eps = eps;
  a.logits = o.logits;
  a.topk_idx = o.topk_idx ? o.topk_idx : s.topk_idx;
  a.topk_w = o.topk_w ? o.topk_w : s.topk_w;
  a.chosen = o.chosen_expert ? o.chosen_expert : s.chosen;
  a.server = o.chosen_server ? o.chosen_server : s.server;
  a.kind = o.kind ? o.kind : s.kind;
  a.counters = o.counters;
  a.sync = s.sync; a.H = s.H; a.part = s.part;
  a.limit_ns = wait_limit_ns();
  if (L->lookahead_H > 1) {  // decided by the look-ahead's launches, the experts here
    // (it leaves an undecided token's experts unwritten: none is what is read here then)
    OM_CUDA(cudaMemsetAsync(a.chosen, 0xff, (size_t)T * a.k * 4, stream));
    const int rc = ordermoe_route_select_lookahead(X, L->W_r, nullptr, T, a.E, a.d, a.k, a.renorm, L->tables,
                                                   L->tables_stride, L->lookahead_H, L->P, home, loc, qhat,
                                                   o.logits, a.topk_idx, a.topk_w, a.chosen, a.server, a.kind,
                                                   o.counters, stream);
    if (rc) return rc;
    a.given = 1;
  }
  return T <= 8 ? few_launch<1>(L, X, a, stream) : few_launch<2>(L, X, a, stream);
}

}  // namespace om

using namespace om;

extern "C" size_t ordermoe_layer_few_workspace_bytes(int T, int E, int d, int dff, int k) {
  if (T <= 0 || T > ORDERMOE_FEW_TOKENS || E <= 0 || E > ORDERMOE_MAX_EXPERTS || d <= 0 || dff <= 0 || k <= 0 ||
      k > ORDERMOE_MAX_TOPK || k > E)
    return 0;
  return few_carve(nullptr, T, E, d, dff, k).bytes;
}

extern "C" int ordermoe_layer_few_init(void* workspace, size_t workspace_bytes, ordermoe_stream_t stream) {
  OM_TRACE();
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 || workspace_bytes < 256)
    return fail(ORDERMOE_ERR_INVALID_ARG, "layer_few_init: workspace null, too small or not 256-byte aligned");
  OM_CUDA(cudaMemsetAsync(workspace, 0, 256, stream));
  return ORDERMOE_OK;
}

extern "C" int ordermoe_layer_few(const ordermoe_layer_desc* layer, int T, const uint16_t* X, const uint8_t* home,
                                  uint8_t* loc, float* qhat, uint16_t* y, const ordermoe_few_out* out,
                                  void* workspace, size_t workspace_bytes, ordermoe_stream_t stream) {
  OM_TRACE();
  return few_layer("layer_few", layer, T, X, nullptr, home, loc, qhat, 1.0f, y, nullptr, out, workspace,
                   workspace_bytes, stream);
}

extern "C" int ordermoe_layer_few_residual(const ordermoe_layer_desc* layer, int T, const uint16_t* x,
                                           const uint16_t* h, const uint8_t* home, uint8_t* loc, float* qhat,
                                           float eps, uint16_t* h_out, uint16_t* x_out,
                                           const ordermoe_few_out* out, void* workspace,
                                           size_t workspace_bytes, ordermoe_stream_t stream) {
  OM_TRACE();
  if (T > 0 && (!h || !x_out)) return fail(ORDERMOE_ERR_INVALID_ARG, "layer_few_residual: null h or x_out");
  if (!(eps > 0.0f)) return fail(ORDERMOE_ERR_INVALID_ARG, "layer_few_residual: eps must be > 0");
  return few_layer("layer_few_residual", layer, T, x, h, home, loc, qhat, eps, h_out, x_out, out, workspace,
                   workspace_bytes, stream);
}
