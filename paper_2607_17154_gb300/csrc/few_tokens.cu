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
//   gate/up  units of 8 MT columns of W1 and W3 of one expert over the whole K = d,
//            dealt out to the CTAs in turn: gate in rows 0-7 of a 16-row MMA tile
//            and up in rows 8-15, so that SwiGLU is in one lane's registers;
//   down     row tiles of 32 MT rows of W2 by all chosen experts' K = d_ff, cut
//            into one contiguous share of equal length per CTA. A share's partial
//            sums of a row tile go to the workspace;
//   finish   one CTA a token adds the partials of every row tile in CTA order and
//            writes y, or h + y and its norm.
// Sums are fp32 in a fixed order: the same call gives the same bits.
// A producer warp streams the weights and the tokens' K blocks through a ring of TMA
// boxes with the 128-byte swizzle; eight MMA warps take its slots in turn; an
// epilogue warp adds their eight partial accumulators. Between gate/up and down
// the producer fills the ring with W2 while the other CTAs finish H: the grid
// barrier there costs HBM no pause.
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
constexpr int PRODUCER = MMA_WARPS;  // the last warp is the epilogue's
constexpr int THREADS = 32 * (MMA_WARPS + 2);
constexpr int KB_UP = 4, KB_DOWN = 2;  // 64-element K blocks a stage

// MT: 16-row MMA tiles of a gate/up unit; NT: 8-token column tiles.
template <int MT, int NT>
struct Cfg {
  static constexpr int W_BYTES = 8192 * MT;            // 16 MT rows x 256, or 32 MT x 128
  static constexpr int STAGE_BYTES = W_BYTES + 4096 * NT;  // and 8 NT tokens x 256
  static constexpr int DOWN_ROWS = 32 * MT;
  // partial accumulators of the MMA warps: two sets of a unit's, or one of a row tile's
  // (the router has up to four tiles, once)
  static constexpr int RED_FLOATS = MMA_WARPS * (MT == 1 ? 4 : 2 * MT) * NT * 128;
  // shared memory beside the ring: alignment, partials, the selection's Q and Cq
  static constexpr int other_bytes(int E) { return 1024 + RED_FLOATS * 4 + ((8 * E * E + 15) & ~15); }
};
constexpr int MAX_STAGES = 16;

struct Smem {
  uint64_t full[MAX_STAGES], empty[MAX_STAGES];
  uint64_t red_full[3], red_empty[3];  // a unit's two sets; [2]: a row tile's
  int abort, zero;
  int n_act;                       // chosen experts
  uint8_t act[64];                 // their indices, ascending
  unsigned int mask[64];           // of an expert: the tokens that use it
  float gate[64][TOKENS];          // and their gate weights
  float logits[2][TOKENS][68];     // shares of K of either CTA; [0] is -inf past E
  alignas(16) float ex[TOKENS][68];  // exponentials of the softmax, read 16 bytes at a time
  float delay[TOKENS][ORDERMOE_MAX_SERVERS];  // A[home][location] of the tokens
  int32_t target[TOKENS * ORDERMOE_MAX_TOPK];
  float weight[TOKENS * ORDERMOE_MAX_TOPK];
  int32_t chosen[TOKENS * ORDERMOE_MAX_TOPK];
  uint8_t server[TOKENS * ORDERMOE_MAX_TOPK], kind[TOKENS * ORDERMOE_MAX_TOPK];
  uint8_t loc[TOKENS];
  float qhat[TOKENS];
  int valid[TOKENS];               // decided: its outputs are written
  float sum[THREADS / 32];
};
static_assert(offsetof(Smem, ex) % 16 == 0 && alignof(Smem) == 16, "16-byte loads");
// A ring takes what the layer's tables leave of the 227 KB.
template <int MT, int NT>
constexpr int stages(int E) {
  const int left = 227 * 1024 - static_cast<int>(sizeof(Smem) + sizeof(SelSmem)) - 256 - Cfg<MT, NT>::other_bytes(E);
  const int n = left / Cfg<MT, NT>::STAGE_BYTES;
  return n < MAX_STAGES ? n : MAX_STAGES;
}
static_assert(stages<1, 1>(64) >= 12 && stages<2, 1>(64) >= 6 && stages<2, 2>(64) >= 5, "ring");

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
  uint16_t* H;         // [n_act][T][dff]
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
// block's rows are kb_pitch bytes, its tokens 1024 NT. Rows of 128 bytes,
// 16-byte chunk c of row r at c ^ (r % 8): the eight rows that an ldmatrix phase
// reads are in different banks.
template <int TILES, int NT, int KB>
__device__ __forceinline__ void mma_stage(float (&acc)[TILES][NT][4], uint32_t w, uint32_t kb_pitch,
                                          uint32_t hi, uint32_t tile_pitch, uint32_t x, int lane) {
  const uint32_t r = lane & 7;
  const uint32_t wr = w + ((lane >> 3) & 1) * hi + r * 128, xr = x + r * 128;
  const uint32_t wc = lane >> 4, xc = lane >> 3;
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {  // 32 elements: two K steps of the MMA
      uint32_t b[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n)
        ldmatrix4(b[n], xr + kb * (1024 * NT) + n * 1024 + (((half * 4 + xc) ^ r) << 4));
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          uint32_t a[4];
          ldmatrix4(a, wr + kb * kb_pitch + i * tile_pitch + (((half * 4 + s * 2 + wc) ^ r) << 4));
#pragma unroll
          for (int n = 0; n < NT; ++n) mma16816(acc[i][n], a, b[n][2 * s], b[n][2 * s + 1]);
        }
      }
    }
  }
}

// A value to the same place in both CTAs of the pair.
__device__ __forceinline__ void store_both(float* p, uint32_t peer, float v) {
  *p = v;
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(mapa_shared(smem_u32(p), peer)), "f"(v) : "memory");
}

// A token's state (eight lanes a token) and what the tables say of all tokens, loaded while
// the router's products run.
struct State {
  int home, loc, M;
  float q, qbar;
};
__device__ __forceinline__ State load_state(Smem& s, const Args& a, int t, int sub) {
  State st{0, 0, 0, 0.0f, 0.0f};
  st.M = reinterpret_cast<const int32_t*>(a.tab)[2];
  st.qbar = reinterpret_cast<const float*>(a.tab)[5];
  if (t < a.T) {
    st.home = a.home[t];
    st.loc = a.loc != nullptr ? a.loc[t] : st.home;  // no state given: first layer (Eq. 36)
    st.q = a.qhat != nullptr ? a.qhat[t] : 0.0f;
    if (st.M > 0 && st.M <= ORDERMOE_MAX_SERVERS && st.home < st.M && st.loc < st.M) {
      const float* A = reinterpret_cast<const float*>(a.tab + off_a(a.E)) + (st.home * st.M + st.loc) * st.M;
      for (int m = sub; m < st.M; m += 8) s.delay[t][m] = A[m];
    }
  }
  return st;
}

// Top-k by (logit desc, index asc) of a token on eight lanes; lane j keeps slot j
// (my_v, my_e), every lane the slots' experts. Lane `sub` holds the logits sub, sub + 8, ...
struct Top {
  float v[8], my_v, max;
  int my_e, idx[ORDERMOE_MAX_TOPK];
  bool nan;
};
__device__ __forceinline__ void top_k(Top& r, const Smem& s, int t, int sub, int lane, int E, int k) {
  r.nan = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    r.v[i] = s.logits[0][t][sub + 8 * i] + s.logits[1][t][sub + 8 * i];
    r.nan |= r.v[i] != r.v[i];
  }
  const unsigned group = 0xFFu << (lane & 24);  // the token's lanes
  r.nan = (__ballot_sync(0xffffffffu, r.nan) & group) != 0u;
  r.my_v = r.max = -INFINITY;
  r.my_e = 0;
  uint32_t used = 0;
#pragma unroll
  for (int j = 0; j < ORDERMOE_MAX_TOPK; ++j) {
    r.idx[j] = 0;
    if (j >= k) continue;  // the same for every lane
    float bv = -INFINITY;
    int be = 1 << 20, bi = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = sub + 8 * i;
      // an unused expert, a real one before the padding past E
      if (!((used >> i) & 1u) && e < E && (be == (1 << 20) || r.v[i] > bv)) {
        bv = r.v[i];
        be = e;
        bi = i;
      }
    }
    const int own = be;
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) {
      const float ov = __shfl_xor_sync(0xffffffffu, bv, o);
      const int oe = __shfl_xor_sync(0xffffffffu, be, o);
      if (oe != (1 << 20) && (be == (1 << 20) || ov > bv || (ov == bv && oe < be))) {
        bv = ov;
        be = oe;
      }
    }
    if (own == be && own != (1 << 20)) used |= 1u << bi;
    r.idx[j] = be < E ? be : 0;
    if (j == 0) r.max = bv;
    if (sub == j) {
      r.my_v = bv;
      r.my_e = be;
    }
  }
}

// The gate weights of four tokens (fp32 softmax over all E, summed in index order) and their
// targets: the arithmetic of the router kernels, so the same logits give the same bits.
__device__ void weigh(Smem& s, const Args& a, const Top& r, int t, int sub, int lane) {
  const int E = a.E, k = a.k;
#pragma unroll
  for (int i = 0; i < 8; ++i) s.ex[t][sub + 8 * i] = expf(r.v[i] - r.max);
  __syncwarp();
  float denom = 0.0f;
#pragma unroll 4
  for (int c = 0; c < (E + 3) / 4; ++c) {  // past E: exact zeros
    const float4 x = *reinterpret_cast<const float4*>(&s.ex[t][4 * c]);
    denom += x.x;
    denom += x.y;
    denom += x.z;
    denom += x.w;
  }
  const float wsel = sub < k ? expf(r.my_v - r.max) / denom : 0.0f;
  float ssel = 0.0f;
  for (int j = 0; j < k; ++j) ssel += __shfl_sync(0xffffffffu, wsel, (lane & 24) + j);
  if (sub < k) {
    const bool active = t < a.T && !r.nan;
    s.target[t * k + sub] = active ? r.my_e : -1;
    s.weight[t * k + sub] = active ? (a.renorm ? wsel / ssel : wsel) : 0.0f;
  }
}

// Alg. 2 of four tokens, eight lanes each.
__device__ void decide(Smem& s, SelSmem& sm, const Args& a, const Top& r, const State& st, const float* s_Q,
                       const float* s_Cq, int t, int sub) {
  const int k = a.k;
  const bool active = t < a.T && !r.nan;
  if (t < a.T && r.nan && sub == 0 && blockIdx.x == 0) report(&g_err_route, ORDERMOE_DEV_NAN_LOGIT, t);
  if (sub < k) {
    s.chosen[t * k + sub] = -1;
    s.server[t * k + sub] = 0;
    s.kind[t * k + sub] = 0;
  }
  if (sub == 0) {
    s.loc[t] = static_cast<uint8_t>(st.loc);
    s.qhat[t] = st.q;
  }
  __syncwarp();
  int kind_count[4] = {0, 0, 0, 0};
  select_slots(t, active, sub, r.idx, a.E, k, st.M, st.qbar, s.delay[t], sm, s_Q, s_Cq, st.home, st.loc, st.q,
               s.loc, s.qhat, s.chosen, s.server, s.kind, kind_count);
  if (blockIdx.x == 0) flush_kind_counts(sm, kind_count, a.counters);
}

// The ring's position, the same walk in the producer and in the MMA warps. A slot belongs to one
// MMA warp, which sees its phases in order: a wait by parity tells only a phase from the next.
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
// K stages. The first n CTAs have at least one stage each, stage i belongs to CTA
// ((i + 1) n - 1) / total.
struct Share {
  long long total, begin, end;
  int per_tile, per_expert, n;
  __device__ __forceinline__ Share(int d, int dff, int rows, int n_act, int c, int G) {
    per_expert = dff / (64 * KB_DOWN);
    per_tile = per_expert * n_act;
    total = static_cast<long long>(d / rows) * per_tile;
    n = total < G ? static_cast<int>(total) : G;
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

template <int MT, int NT>
__global__ void __launch_bounds__(THREADS, 1)
    few_tokens_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Args a) {
  using C = Cfg<MT, NT>;
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

  if (tid == 0) {
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(&s.full[i], 1);
      mbar_init(&s.empty[i], 1);
    }
    for (int i = 0; i < 3; ++i) {
      mbar_init(&s.red_full[i], MMA_WARPS);
      mbar_init(&s.red_empty[i], 1);
    }
    s.abort = 0;
    s.zero = 0;
    fence_mbar_init();
  }
  if (tid < 4) sm.kind[tid] = 0;
  for (int i = tid; i < TOKENS * 68; i += THREADS) {
    (&s.logits[0][0][0])[i] = -INFINITY;
    (&s.logits[1][0][0])[i] = 0.0f;
  }
  for (int i = tid; i < 64 * TOKENS; i += THREADS) (&s.gate[0][0])[i] = 0.0f;
  for (int i = tid; i < 64; i += THREADS) s.mask[i] = 0;
  cluster_sync();  // both CTAs run: the peer's shared memory may be written

  Ring ring_at(STAGES);          // producer and MMA warps
  uint32_t units = 0, rows = 0;  // hand-overs to the epilogue warp so far: units, row tiles
  using MTc = std::integral_constant<int, MT>;        // MMA tiles of a unit
  using MT2c = std::integral_constant<int, 2 * MT>;   // and of a row tile
  uint32_t issued_mask = 0, last_phase_bits = 0;  // the producer's, for the drain after an abort
  const uint32_t ring0 = smem_u32(ring);
  const int k_up = a.d / (64 * KB_UP);
  bool tables_ok = true;

  // --- roles' steps
  auto timeout = [&](int where) {
    if (!*abort) report(&g_err_route, ORDERMOE_DEV_WAIT_TIMEOUT, where);
    *abort = 1;
  };
  // The producer walks the stages as a converged warp and one elected lane issues: a lane
  // walking alone took about 550 cycles a stage whatever its bytes (1 token on 8 wide
  // experts 190 us).
  const bool issuer = elect_one();
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
  auto route = [&](auto row_tiles, State& st) {
    // stages of all experts' rows (RT tiles of 16) by KB blocks of K, the first half of them
    // in rank 0
    constexpr int RT = decltype(row_tiles)::value, KB = RT == 4 && MT == 1 ? 1 : 2;
    constexpr uint32_t W = RT * 2048 * KB;
    const int all = a.d / (64 * KB), half = (all + 1) / 2;
    const int s0 = rank == 0 ? 0 : half, s1 = rank == 0 ? half : all;
    if (warp == PRODUCER) {
      for (int i = s0; i < s1; ++i) {
        if (!claim(W + KB * 1024 * NT)) break;
        if (issuer) {
          uint8_t* p = slot_ptr(ring_at.slot);
          tma_load_3d(p, &maps.Wr, &s.full[ring_at.slot], 0, i * KB);
          tma_load_3d(p + C::W_BYTES, &maps.Xr, &s.full[ring_at.slot], 0, i * KB);
        }
        ring_at.next();
      }
    } else if (warp < MMA_WARPS) {
      if (warp < TOKENS / 4) st = load_state(s, a, warp * 4 + (lane >> 3), lane & 7);
      tables_ok = load_tables_range(a.tab, a.E, sm, s_Q, s_Cq, tid, 32 * MMA_WARPS);
      float acc[RT][NT][4] = {};
      bool ok = true;
      for (int i = s0; i < s1; ++i) {
        if (ring_at.slot % MMA_WARPS == warp) {
          if (!(ok = arrived())) break;
          const uint32_t w = ring0 + ring_at.slot * C::STAGE_BYTES;
          mma_stage<RT, NT, KB>(acc, w, 2048 * RT, 1024, 2048, w + C::W_BYTES, lane);
          release();
        }
        ring_at.next();
      }
      if (ok) put(acc, row_tiles, 0, 0);
      ++units;
    } else {
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
    State st{};
    if (a.E <= 16) route(std::integral_constant<int, 1>{}, st);
    else if (a.E <= 32) route(std::integral_constant<int, 2>{}, st);
    else route(std::integral_constant<int, 4>{}, st);
    cluster_sync();  // the peer's half of the logits is here
    if (warp < 2 * (TOKENS / 4)) {  // warps 0-3 decide, 4-7 weigh: four tokens each
      const int t = (warp % (TOKENS / 4)) * 4 + (lane >> 3), sub = lane & 7;
      Top r;
      top_k(r, s, t, sub, lane, a.E, a.k);
      if (warp >= TOKENS / 4) weigh(s, a, r, t, sub, lane);
      else if (tables_ok) decide(s, sm, a, r, st, s_Q, s_Cq, t, sub);  // the same for the block
      else if (sub < a.k) s.chosen[t * a.k + sub] = -1;
    }
  } else {
    for (int i = tid; i < a.T * a.k; i += THREADS) {
      s.target[i] = a.topk_idx[i];
      s.weight[i] = a.topk_w[i];
      s.chosen[i] = a.chosen[i];
    }
  }
  __syncthreads();
  // The chosen experts in ascending order, the tokens that use them and their gate weights. A
  // token counts when all of its slots were decided.
  if (tid < a.T) {
    bool ok = s.target[tid * a.k] >= 0;
    for (int j = 0; j < a.k; ++j) ok = ok && s.chosen[tid * a.k + j] >= 0 && s.chosen[tid * a.k + j] < a.E;
    s.valid[tid] = ok;
    if (ok)
      for (int j = 0; j < a.k; ++j) {  // a token's experts are distinct
        const int e = s.chosen[tid * a.k + j];
        atomicOr(&s.mask[e], 1u << tid);
        s.gate[e][tid] += s.weight[tid * a.k + j];
      }
  }
  __syncthreads();
  if (warp == 0) {
    const bool lo = s.mask[lane] != 0, hi = s.mask[lane + 32] != 0;
    const unsigned int l = __ballot_sync(0xffffffffu, lo), h = __ballot_sync(0xffffffffu, hi);
    const unsigned int before = (1u << lane) - 1;
    if (lo) s.act[__popc(l & before)] = static_cast<uint8_t>(lane);
    if (hi) s.act[__popc(l) + __popc(h & before)] = static_cast<uint8_t>(lane + 32);
    if (lane == 0) s.n_act = __popc(l) + __popc(h);
  }
  if (cta == 0 && !a.given && !*abort) {  // one CTA writes the decisions
    for (int i = tid; i < a.T * a.k; i += THREADS) {
      const bool ok = s.target[i] >= 0 && s.chosen[i] >= 0;
      a.topk_idx[i] = s.target[i];
      a.topk_w[i] = s.weight[i];
      if (ok) {
        a.chosen[i] = s.chosen[i];
        a.server[i] = s.server[i];
        a.kind[i] = s.kind[i];
      }
    }
    if (a.logits != nullptr)
      for (int i = tid; i < a.T * a.E; i += THREADS) {
        const int t = i / a.E, e = i - t * a.E;
        a.logits[i] = s.logits[0][t][e] + s.logits[1][t][e];
      }
    if (a.counters != nullptr && tid < 4 && sm.kind[tid]) atomicAdd(&a.counters[tid], sm.kind[tid]);
  }
  __syncthreads();

  // -------------------------------------------------------------- gate/up
  const int n_act = *abort ? 0 : s.n_act;
  const int per = a.dff / (8 * MT);  // units of an expert
  const int n_units = n_act * per;
  const Share share(a.d, a.dff, C::DOWN_ROWS, n_act, cta, G);
  if (warp == PRODUCER) {
    bool ok = true;
    for (int u = cta; u < n_units && ok; u += G) {
      const int row = s.act[u / per] * a.dff + (u % per) * 8 * MT;
      for (int kb = 0; kb < k_up; ++kb) {
        if (!(ok = claim(C::STAGE_BYTES))) break;
        if (issuer) {
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
    const uint32_t bytes = C::W_BYTES + 2048 * NT;
    Walk w(share), hw(share);
    Ring first = ring_at;
    auto load_w = [&]() {
      if (issuer)
        tma_load_3d(slot_ptr(ring_at.slot), &maps.W2, &s.full[ring_at.slot],
                    s.act[w.act] * a.d + w.tile * C::DOWN_ROWS, w.k * KB_DOWN);
      ring_at.next();
      w.next(share, n_act);
    };
    auto load_h = [&]() {
      if (issuer)
        tma_load_3d(slot_ptr(first.slot) + C::W_BYTES, &maps.H, &s.full[first.slot], hw.act * a.T,
                    hw.k * KB_DOWN);
      first.next();
      hw.next(share, n_act);
    };
    while (ok && w.left > 0 && hw.left - w.left < STAGES && (ok = claim(bytes))) load_w();
    if (ok) {
      const bool up = !issuer || grid_wait(&a.sync[0], G, a.limit_ns, abort);
      if (!up) timeout(35);
      ok = __all_sync(0xffffffffu, up);
    }
    fence_proxy_async();
    // (also after a failure: the barriers of the stages under way expect these bytes)
    while (hw.left > w.left) load_h();
    while (ok && w.left > 0 && (ok = claim(bytes))) {
      load_w();
      load_h();
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
            mma_stage<MT, NT, KB_UP>(acc, w, 1024 * MT, 4096 * MT, 1024, w + C::W_BYTES, lane);
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
        mma_stage<2 * MT, NT, KB_DOWN>(acc, p, 4096 * MT, 1024, 2048, p + C::W_BYTES, lane);
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
          const float g0 = s.gate[e][t], g1 = s.gate[e][t + 1];
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
    bool ok = true;
    for (int u = cta; u < n_units && ok; u += G) {
      const int e = u / per, f0 = (u - e * per) * 8 * MT + (lane >> 2);
      ok = take_unit([&](int m, int n, float4 v) {
        // rows 0-7 gate, 8-15 up: silu(g) u, rounded to bf16 as ordermoe_expert_ffn's H
        const int t = n * 8 + (lane & 3) * 2;
        uint16_t* out = a.H + (static_cast<size_t>(e) * a.T + t) * a.dff + f0 + m * 8;
        const uint32_t pk = pack_bf16x2(v.x / (1.0f + __expf(-v.x)) * v.z, v.y / (1.0f + __expf(-v.y)) * v.w);
        if (t < a.T) out[0] = static_cast<uint16_t>(pk & 0xFFFFu);
        if (t + 1 < a.T) out[a.dff] = static_cast<uint16_t>(pk >> 16);
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
  if (cta < a.T * parts) {
    const int tiles = a.d / C::DOWN_ROWS, part = cta / a.T;
    const int first_tile = tiles * part / parts, last_tile = tiles * (part + 1) / parts;
    // the first and last owner of every row tile, while the others finish (the ring is free)
    int16_t* own = reinterpret_cast<int16_t*>(ring);
    const int cap = STAGES * C::STAGE_BYTES / 4;  // tiles that fit
    const bool listed = tiles <= cap;
    auto owners = [&](int tile, int& c0, int& c1) {
      c0 = share.owner(static_cast<long long>(tile) * share.per_tile);
      c1 = share.owner(static_cast<long long>(tile + 1) * share.per_tile - 1);
    };
    if (listed && share.total > 0)
      for (int i = first_tile + tid; i < last_tile; i += THREADS) {
        int c0, c1;
        owners(i, c0, c1);
        own[2 * i] = static_cast<int16_t>(c0);
        own[2 * i + 1] = static_cast<int16_t>(c1);
      }
    if (tid == 0 && !grid_wait(&a.sync[1], G, a.limit_ns, abort)) timeout(36);
    __syncthreads();
    for (int t = cta % a.T; t < a.T && !*abort; t += G) {
      if (!s.valid[t]) continue;
      float sq = 0.0f;
      const size_t row = static_cast<size_t>(t) * a.d;
      for (int c = first_tile * C::DOWN_ROWS + tid * 4; c < last_tile * C::DOWN_ROWS; c += THREADS * 4) {
        const int tile = c / C::DOWN_ROWS;
        uint2 hv = make_uint2(0, 0);
        if (a.h != nullptr) hv = *reinterpret_cast<const uint2*>(a.h + row + c);
        int c0, c1;
        if (listed) {
          c0 = own[2 * tile];
          c1 = own[2 * tile + 1];
        } else {
          owners(tile, c0, c1);
        }
        const size_t pitch = static_cast<size_t>(a.T) * C::DOWN_ROWS;
        const float* p = a.part + (static_cast<size_t>(tile + c0) * a.T + t) * C::DOWN_ROWS + c % C::DOWN_ROWS;
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int q = c0; q <= c1; q += 4, p += 4 * pitch) {  // four loads under way
          float4 u[4];
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (q + j <= c1) u[j] = __ldcg(reinterpret_cast<const float4*>(p + j * pitch));
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (q + j <= c1) {
              v.x += u[j].x;
              v.y += u[j].y;
              v.z += u[j].z;
              v.w += u[j].w;
            }
        }
        v.x += bf16_lo(hv.x);
        v.y += bf16_hi(hv.x);
        v.z += bf16_lo(hv.y);
        v.w += bf16_hi(hv.y);
        const uint2 o = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
        *reinterpret_cast<uint2*>(a.y + row + c) = o;
        const float f[4] = {bf16_lo(o.x), bf16_hi(o.x), bf16_lo(o.y), bf16_hi(o.y)};
#pragma unroll
        for (int j = 0; j < 4; ++j) sq = fmaf(f[j], f[j], sq);
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
        const uint2 o = *reinterpret_cast<const uint2*>(a.y + row + c);
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
  if (s.abort && warp == PRODUCER && issuer) {  // every copy that this CTA issued (bounded)
    volatile int* never = &s.zero;
    for (int i = 0; i < STAGES; ++i)
      if ((issued_mask >> i) & 1u) mbar_wait(&s.full[i], (last_phase_bits >> i) & 1u, a.limit_ns, never);
  }
  cluster_sync();  // (no access to the peer is under way)
  // the last CTA to leave sets the counters back
  if (tid == 0) {
    __threadfence();
    if (atomicAdd(&a.sync[2], 1u) == static_cast<unsigned int>(G) - 1) {
      a.sync[0] = a.sync[1] = a.sync[2] = 0;
      __threadfence();
    }
  }
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
  s.H = reinterpret_cast<uint16_t*>(take(act * T * dff * 2));
  // rows of 32 (T <= 4) or 64 columns: a row tile's partials, one for each CTA more
  const size_t rows = T <= 4 ? 32 : 64;
  s.part = reinterpret_cast<float*>(take((d / rows + kFewMaxCtas) * T * rows * 4));
  s.topk_w = reinterpret_cast<float*>(take(R * 4));
  s.topk_idx = reinterpret_cast<int32_t*>(take(R * 4));
  s.chosen = reinterpret_cast<int32_t*>(take(R * 4));
  s.server = take(R);
  s.kind = take(R);
  s.bytes = off;
  return s;
}

template <int MT, int NT>
static cudaError_t few_attr() {
  return cudaFuncSetAttribute(fw::few_tokens_kernel<MT, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              227 * 1024 - static_cast<int>(sizeof(fw::Smem) + sizeof(SelSmem)) - 256);
}

template <int MT, int NT>
static int few_launch(const ordermoe_layer_desc* L, const uint16_t* X, fw::Args& a, cudaStream_t stream) {
  using C = fw::Cfg<MT, NT>;
  static PerDevice cache;
  const cudaError_t ae = static_cast<cudaError_t>(per_device(cache, [] {
    return static_cast<int>(few_attr<MT, NT>());
  }));
  if (ae != cudaSuccess) return cuda_fail(ae, "cudaFuncSetAttribute(few_tokens_kernel)");
  const int R = a.T * a.k, act = R < a.E ? R : a.E;
  fw::Maps m;
  int rc;
  const int rt = a.E <= 16 ? 1 : a.E <= 32 ? 2 : 4, kb = rt == 4 && MT == 1 ? 1 : 2;  // as the kernel's route
  if ((rc = make_tmap_bf16_kb(&m.Wr, L->W_r, a.E, a.d, 16 * rt, kb))) return rc;
  if ((rc = make_tmap_bf16_kb(&m.Xr, X, a.T, a.d, 8 * NT, kb))) return rc;
  if ((rc = make_tmap_bf16_kb(&m.X, X, a.T, a.d, 8 * NT, fw::KB_UP))) return rc;
  if ((rc = make_tmap_bf16_kb(&m.W1, L->W1, (uint64_t)a.E * a.dff, a.d, 8 * MT, fw::KB_UP))) return rc;
  if ((rc = make_tmap_bf16_kb(&m.W3, L->W3, (uint64_t)a.E * a.dff, a.d, 8 * MT, fw::KB_UP))) return rc;
  if ((rc = make_tmap_bf16_kb(&m.W2, L->W2, (uint64_t)a.E * a.d, a.dff, C::DOWN_ROWS, fw::KB_DOWN))) return rc;
  if ((rc = make_tmap_bf16_kb(&m.H, a.H, (uint64_t)act * a.T, a.dff, 8 * NT, fw::KB_DOWN))) return rc;
  a.stages = fw::stages<MT, NT>(a.E);
  // a CTA per SM, fewer where there are not as many units of gate/up
  int grid = num_sms() < kFewMaxCtas ? num_sms() : kFewMaxCtas;
  const long long units = (long long)act * (a.dff / (8 * MT));
  if (units < grid) grid = static_cast<int>(units);
  grid = (grid < a.T ? a.T : grid) / 2 * 2;  // pairs
  if (grid < 2) grid = 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid, 1, 1);
  cfg.blockDim = dim3(fw::THREADS, 1, 1);
  cfg.dynamicSmemBytes = a.stages * C::STAGE_BYTES + C::other_bytes(a.E);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeCooperative;  // the CTAs wait for one another: all or none run
  attr[0].val.cooperative = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 2;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, fw::few_tokens_kernel<MT, NT>, m, a);
  if (e != cudaSuccess) return cuda_fail(e, "few_tokens_kernel");
  OM_LAUNCHED("few_tokens_kernel");
  return ORDERMOE_OK;
}

// Variants by the number of tokens: up to 4 take units of one MMA tile (more units, an even
// share for every SM), more take two, so that a token's K block is loaded for twice
// the weights; past 8 tokens a second column tile.
static int few_dispatch(const ordermoe_layer_desc* L, const uint16_t* X, fw::Args& a, cudaStream_t stream) {
  if (a.T <= 4) return few_launch<1, 1>(L, X, a, stream);
  return a.T <= 8 ? few_launch<2, 1>(L, X, a, stream) : few_launch<2, 2>(L, X, a, stream);
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
  if ((long long)L->E * L->dff > INT32_MAX || (long long)L->E * L->d > INT32_MAX)
    return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "%s: sizes too large", who);
  if (L->lookahead_H > 4) return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "%s: look-ahead of at most 4 layers", who);
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
    const int rc = ordermoe_route_select_lookahead(X, L->W_r, nullptr, T, a.E, a.d, a.k, a.renorm, L->tables,
                                                   L->tables_stride, L->lookahead_H, L->P, home, loc, qhat,
                                                   o.logits, a.topk_idx, a.topk_w, a.chosen, a.server, a.kind,
                                                   o.counters, stream);
    if (rc) return rc;
    a.given = 1;
  }
  return few_dispatch(L, X, a, stream);
}

}  // namespace om

using namespace om;

extern "C" size_t ordermoe_layer_few_workspace_bytes(int T, int E, int d, int dff, int k) {
  if (T <= 0 || T > ORDERMOE_FEW_TOKENS || E <= 0 || E > ORDERMOE_MAX_EXPERTS || d <= 0 || dff <= 0 || k <= 0 ||
      k > ORDERMOE_MAX_TOPK || k > E)
    return 0;
  // fewer tokens take less, but for rows of partials: the largest of both variants
  const size_t n = few_carve(nullptr, T, E, d, dff, k).bytes;
  const size_t four = few_carve(nullptr, T < 4 ? T : 4, E, d, dff, k).bytes;
  return n > four ? n : four;
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
