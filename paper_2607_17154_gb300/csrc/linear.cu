// Matrix product with an epilogue: Y = act(X W^T + bias) + residual, X [M][K] and W [N][K]
// bf16 with row strides, fp32 sums on tcgen05, one rounding to Y (bf16) or none (f32).
//
// The weights are the MMA's M side and the rows of X its N side, as in the expert GEMMs: few
// rows waste little of the tensor pipe, and the accumulator is transposed (TMEM lane =
// output column).
//   linear_split_kernel: one tile of up to 128 columns x 128 rows a cluster of S CTAs, which
//     share its K and add their accumulators through distributed shared memory, every CTA the
//     rows of its own share in rank order (the same bits at every call), four columns a thread.
//     For few rows, whose weights are one pass over HBM: the tile's width and S are chosen so
//     that every SM streams the same share of them.
//   linear_pair_kernel: persistent CTA pairs, tiles of up to 256 columns x up to 256 rows with
//     cta_group::2 MMAs, two accumulators, so that a tile's epilogue overlaps the next tile's
//     main loop. For batches with a tile for most pairs, bound by the tensor cores (4096 x 14336 x
//     4096 274 us launched from the host or in a long loop of graphs, 1755 TFLOP/s, as a library product
//     there; 240 in the first few replays, before the chip's power cap). Its epilogue is bound by instructions and latency: sixteen
//     warps, eight rows of a column at a time from TMEM (eight warps, 32 rows through shared memory:
//     2048 x 4096 x 4096 with SiLU and residual 87 us for 47).
//   linear_pair_split_kernel: one tile of 256 columns x up to 256 rows a cluster of 2 or 4 CTA
//     pairs that share its K, the accumulators added as in the first kernel. For batches in between,
//     whose tiles are too few for the pairs but whose operands, in tiles of 128 x 128, take
//     longer from L2 than their products. (Sixteen warps in the epilogue for four: 300 x 4096 x
//     14336 with residual 44.3 -> 38.5 us, 512 x 2048 x 2048 16.2 -> 13.2.)
// The tensor cores truncate a running sum, an error that grows with K (2e-6 of the result at K = 2048).
// Where the sums leave in fp32 (F32), the epilogue warps therefore take the accumulator every 512 of K
// and add it to sums in registers: 4.7e-7 off in the 2-norm at K = 512, 4.8e-7 at 14336 (sums of fp32
// FMAs 1.6e-7 and 1.4e-6). bf16 results, rounded by 1.7e-3, do not see it.
// Rows and columns past M, N and K are zero-filled by TMA and not stored. Every wait is bounded; one that
// runs out reports ORDERMOE_DEV_WAIT_TIMEOUT, and the copies and MMAs under way are drained.
#include "common.cuh"

#include <type_traits>

namespace om {

static __device__ unsigned long long g_err_linear = 0;

int read_clear_err_linear(unsigned long long* out) {
  unsigned long long zero = 0;
  OM_CUDA(cudaMemcpyFromSymbol(out, g_err_linear, sizeof(*out)));
  OM_CUDA(cudaMemcpyToSymbol(g_err_linear, &zero, sizeof(zero)));
  return ORDERMOE_OK;
}

namespace ln {

constexpr int BK = 64;                 // K block: 128 bytes a row
constexpr int W_BYTES = 128 * BK * 2;  // 128 weight rows of a K block
constexpr int F32_BLOCKS = 8;          // K blocks that an fp32 result's accumulator sums up
constexpr int F32_ROWS = 64;           // rows of the split kernel's tiles then: sums in 64 registers
constexpr int F32_PAIR_ROWS = 128;     // and of the pair kernel's, over its groups of epilogue warps

struct Epilogue {
  int M, N;
  const uint16_t* bias;      // nullable
  const uint16_t* residual;  // nullable; may be Y
  void* Y;
  int64_t ldr, ldy;
  int act, f32;
  int vec_r, vec_y;          // 4 columns at a time: strides and addresses allow it
};

// An activation in fp32 of the product's sum; NaN stays NaN. A bf16 result takes the fast exponential and
// quotient (within 2^-14 in the tails, of its rounding's 2^-8; a few 2^-23 near zero): 301 x 1009 x 1999
// with SiLU 9.8 us, with the exact ones 10.8; 2048 x 4096 x 4096 48.6 and 51.0.
template <int ACT, bool FAST>
__device__ __forceinline__ float activate(float v) {
  if (ACT == ORDERMOE_ACT_RELU) return v < 0.0f ? 0.0f : v;
  // v Phi(v); erfc keeps the digits of a negative v's tail, which 1 + erf loses
  if (ACT == ORDERMOE_ACT_GELU) return 0.5f * v * erfcf(-0.70710678118654752f * v);
  // v sigmoid(s): s = v, or 2 sqrt(2/pi) (v + 0.044715 v^3), whose sigmoid is (1 + tanh) / 2 of half of it.
  // As v exp(-|s|) / (1 + exp(-|s|)) for a negative s: 1 / (1 + exp(-s)) is 0 where the result still is a normal
  // number (v = -89). The exponential as a square h h, last: one rounding where h h is below the normal numbers.
  const float s = ACT == ORDERMOE_ACT_SILU ? v : 1.5957691216057308f * fmaf(0.044715f * v * v, v, v);
  const float x = -0.5f * fabsf(s), h = FAST ? __expf(x) : expf(x);
  const float d = fmaf(h, h, 1.0f), q = FAST ? __fdividef(v, d) : v / d;
  return s < 0.0f ? q * h * h : q;
}

template <int N, bool FAST>
__device__ __forceinline__ void activate_all(float (&f)[N], int act) {
  auto all = [&](auto kind) {
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = activate<decltype(kind)::value, FAST>(f[j]);
  };
  if (act == ORDERMOE_ACT_RELU) all(std::integral_constant<int, ORDERMOE_ACT_RELU>{});
  else if (act == ORDERMOE_ACT_GELU) all(std::integral_constant<int, ORDERMOE_ACT_GELU>{});
  else if (act == ORDERMOE_ACT_GELU_TANH) all(std::integral_constant<int, ORDERMOE_ACT_GELU_TANH>{});
  else if (act == ORDERMOE_ACT_SILU) all(std::integral_constant<int, ORDERMOE_ACT_SILU>{});
}

// Not inlined: the epilogue of a few rows runs once and its instructions come from L2, so one copy of the five
// activations serves all four columns (inlined the same: 301 x 1009 x 1999 with SiLU 9.5 and 9.4 us).
template <bool FAST>
__device__ __noinline__ float4 activate4(float4 v, int act) {
  float f[4] = {v.x, v.y, v.z, v.w};
  activate_all<4, FAST>(f, act);
  return make_float4(f[0], f[1], f[2], f[3]);
}

__device__ __forceinline__ void load_bias4(float (&b)[4], const Epilogue& e, int n) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
    b[j] = e.bias != nullptr && n + j < e.N ? __uint_as_float(static_cast<uint32_t>(e.bias[n + j]) << 16) : 0.0f;
}

// Columns n .. n + 3 of the residual's row m (0 past N, or without one).
__device__ __forceinline__ float4 load_residual4(const Epilogue& e, int m, int n) {
  float f[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  if (e.residual != nullptr) {
    const uint16_t* r = e.residual + m * e.ldr + n;
    if (e.vec_r && n + 4 <= e.N) {
      const uint2 h = *reinterpret_cast<const uint2*>(r);
      f[0] = bf16_lo(h.x);
      f[1] = bf16_hi(h.x);
      f[2] = bf16_lo(h.y);
      f[3] = bf16_hi(h.y);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (n + j < e.N) f[j] = __uint_as_float(static_cast<uint32_t>(r[j]) << 16);
    }
  }
  return make_float4(f[0], f[1], f[2], f[3]);
}

// The line of the residual's row m that holds column n, into L2 while the sums are made (64 x 4096 x 4096
// 12.9 -> 12.3 us, 300 x 2048 x 2048 12.5 -> 12.0; 300 x 4096 x 14336, whose sums take long, the same).
__device__ __forceinline__ void prefetch_residual(const Epilogue& e, int m, int n) {
  asm volatile("prefetch.global.L2 [%0];" ::"l"(e.residual + m * e.ldr + n));
}

// Columns n .. n + 3 of row m from their sums v and their residual r.
__device__ __forceinline__ void finish4(const Epilogue& e, int m, int n, float4 v, const float (&b)[4], float4 r) {
  v = make_float4(v.x + b[0], v.y + b[1], v.z + b[2], v.w + b[3]);
  if (e.act != ORDERMOE_ACT_NONE) v = e.f32 ? activate4<false>(v, e.act) : activate4<true>(v, e.act);
  float f[4] = {v.x, v.y, v.z, v.w};
  if (e.residual != nullptr) {  // (without one -0 stays -0)
    f[0] += r.x;
    f[1] += r.y;
    f[2] += r.z;
    f[3] += r.w;
  }
  const bool whole = n + 4 <= e.N;
  if (e.f32) {
    float* y = static_cast<float*>(e.Y) + m * e.ldy + n;
    if (e.vec_y && whole) {
      *reinterpret_cast<float4*>(y) = make_float4(f[0], f[1], f[2], f[3]);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (n + j < e.N) y[j] = f[j];
    }
  } else {
    uint16_t* y = static_cast<uint16_t*>(e.Y) + m * e.ldy + n;
    const uint2 o = make_uint2(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]));
    if (e.vec_y && whole) {
      *reinterpret_cast<uint2*>(y) = o;
    } else {
      const uint32_t h[4] = {o.x & 0xFFFFu, o.x >> 16, o.y & 0xFFFFu, o.y >> 16};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (n + j < e.N) y[j] = static_cast<uint16_t>(h[j]);
    }
  }
}

// ------------------------------------------------------------ few rows: K over a cluster
constexpr int S_THREADS = 192;  // TMA warp, MMA warp, four epilogue warps; all of them reduce
constexpr int S_MAX_STAGES = 12;
constexpr int S_MAX_SPLIT = 8;
// An allocation of TMEM that has to wait holds up a cluster, or a kernel whose dependents already wait for it,
// and nothing bounds that wait. So none has to: a CTA takes 128 of the 512 columns at most, and shared memory
// for at most four on an SM (228 KB, 1 KB of it reserved for each), which does not fit beside a CTA that
// takes all columns (those, here and in the expert GEMMs, the logits and the similarity, hold 180 KB and more).
constexpr int S_MIN_SMEM = 48 * 1024, S_MAX_COLS = 128;
static_assert(5 * (S_MIN_SMEM + 1024) > 228 * 1024 && 4 * S_MAX_COLS <= 512, "TMEM of the CTAs of an SM");

struct SplitSmem {
  uint64_t full[S_MAX_STAGES], empty[S_MAX_STAGES];
  uint64_t tfull[2], tempty[2], drain;
  uint32_t tmem_base;
  int abort, zero;
};

struct SplitArgs {
  Epilogue e;
  int rows;      // of a tile: a multiple of 16, at most 128
  int cols;      // a multiple of 16, at most 128
  int row_tiles;
  int x_rows;    // rows that are loaded: all, or the M that there are
  int kblocks, split, stages, tmem_cols;
  uint64_t limit_ns;
};

// Four floats of the same place in a CTA of the cluster.
__device__ __forceinline__ float4 load_rank(const float* p, uint32_t rank) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(mapa_shared(smem_u32(p), rank))
               : "memory");
  return v;
}

template <bool F32>
__global__ void __launch_bounds__(S_THREADS, 2)
    linear_split_kernel(const __grid_constant__ CUtensorMap mapW, const __grid_constant__ CUtensorMap mapX,
                        const __grid_constant__ SplitArgs a) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ SplitSmem s;
  uint8_t* ring = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  float* sums = reinterpret_cast<float*>(ring);  // [rows][128], when the main loop is done
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_trigger();  // barriers, TMEM and tensor maps while the previous kernel finishes
  if (warp == 0 && lane == 0) {
    tma_prefetch_map(&mapW);
    tma_prefetch_map(&mapX);
  }
  if (tid == 0) {
    for (int i = 0; i < a.stages; ++i) {
      mbar_init(&s.full[i], 1);
      mbar_init(&s.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s.tfull[i], 1);
      mbar_init(&s.tempty[i], 4);  // every epilogue warp
    }
    mbar_init(&s.drain, 1);
    s.abort = 0;
    s.zero = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&s.tmem_base, a.tmem_cols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_wait();  // every thread: the previous kernel's outputs are visible
  const uint32_t tmem_base = s.tmem_base;
  volatile int* abort = &s.abort;
  const int rank = static_cast<int>(blockIdx.x % a.split), tile = static_cast<int>(blockIdx.x / a.split);
  const int n0 = tile / a.row_tiles * a.cols, m0 = tile % a.row_tiles * a.rows;
  const int kb0 = static_cast<int>(static_cast<long long>(a.kblocks) * rank / a.split);
  const int kb1 = static_cast<int>(static_cast<long long>(a.kblocks) * (rank + 1) / a.split);
  // The MMA's M side is 128 rows: past `cols` it reads what follows in shared memory, and its N side
  // past x_rows what an earlier stage left there; those sums are not stored.
  const int w_bytes = a.cols * BK * 2, stage_bytes = w_bytes + a.rows * BK * 2;
  uint32_t issued_mask = 0, last_phase_bits = 0;
  bool mma_issued = false, leader = false;
  const int part = F32 ? F32_BLOCKS : kb1 - kb0;  // K blocks of an accumulator, two in turn
  const int r0 = a.rows * rank / a.split, r1 = a.rows * (rank + 1) / a.split;  // rows that this CTA finishes

  if (warp == 0) {
    const bool issuer = elect_one();
    int slot = 0;
    uint32_t phase = 0;
    for (int kb = kb0; kb < kb1; ++kb) {
      if (!__all_sync(0xffffffffu, mbar_wait(&s.empty[slot], phase ^ 1u, a.limit_ns, abort))) {
        if (issuer && !*abort) report(&g_err_linear, ORDERMOE_DEV_WAIT_TIMEOUT, 41);
        *abort = 1;
        break;
      }
      if (issuer) {
        uint8_t* p = ring + slot * stage_bytes;
        mbar_arrive_expect_tx(&s.full[slot], w_bytes + a.x_rows * BK * 2);
        tma_load_2d(p, &mapW, &s.full[slot], kb * BK, n0);
        tma_load_2d(p + w_bytes, &mapX, &s.full[slot], kb * BK, m0);
      }
      issued_mask |= 1u << slot;
      last_phase_bits = (last_phase_bits & ~(1u << slot)) | (phase << slot);
      if (++slot == a.stages) {
        slot = 0;
        phase ^= 1u;
      }
    }
  } else if (warp == 1) {
    leader = elect_one();
    const uint64_t desc0 = sdesc_kmajor_sw128(smem_u32(ring));
    const uint32_t idesc = idesc_bf16_f32(128, a.rows);
    int slot = 0;
    uint32_t phase = 0;
    bool ok = true;
    int u = 0;
    for (int first = kb0; first < kb1 && ok; first += part, ++u) {
      const int end = min(first + part, kb1), b = u & 1;
      if (!__all_sync(0xffffffffu, mbar_wait(&s.tempty[b], ((u >> 1) & 1) ^ 1u, a.limit_ns, abort))) {
        if (leader && !*abort) report(&g_err_linear, ORDERMOE_DEV_WAIT_TIMEOUT, 44);
        *abort = 1;
        break;
      }
      tc_fence_after();
      for (int kb = first; kb < end; ++kb) {
        if (!__all_sync(0xffffffffu, mbar_wait(&s.full[slot], phase, a.limit_ns, abort))) {
          if (leader && !*abort) report(&g_err_linear, ORDERMOE_DEV_WAIT_TIMEOUT, 42);
          *abort = 1;
          ok = false;
          break;
        }
        tc_fence_after();
        const uint64_t dw = desc0 + static_cast<uint64_t>((slot * stage_bytes) >> 4);
        const uint64_t dx = dw + static_cast<uint64_t>(w_bytes >> 4);
        if (leader) {
#pragma unroll
          for (int kk = 0; kk < BK / 16; ++kk)  // 16 elements = 32 bytes on
            mma_bf16(tmem_base + b * (a.tmem_cols / 2), dw + 2 * kk, dx + 2 * kk, idesc,
                     kb != first || kk != 0 ? 1u : 0u);
          mma_commit(&s.empty[slot]);
        }
        mma_issued = true;
        if (++slot == a.stages) {
          slot = 0;
          phase ^= 1u;
        }
      }
      if (ok && leader) mma_commit(&s.tfull[b]);
      __syncwarp();
    }
  } else {
    const int q = warp & 3;
    if (a.e.residual != nullptr && lane * 4 < a.cols && n0 + lane * 4 < a.e.N)  // what this CTA finishes
      for (int r = r0 + q; r < min(r1, a.e.M - m0); r += 4) prefetch_residual(a.e, m0 + r, n0 + lane * 4);
    const uint32_t tb = tmem_base + (static_cast<uint32_t>(q * 32) << 16);
    float acc[F32 ? F32_ROWS / 32 : 1][32];
    bool ok = true;
    int u = 0;
    for (int first = kb0; first < kb1 && ok; first += part, ++u) {
      const int b = u & 1;
      ok = __all_sync(0xffffffffu, mbar_wait(&s.tfull[b], (u >> 1) & 1, a.limit_ns, abort));
      if (!ok) {
        if (lane == 0 && !*abort) report(&g_err_linear, ORDERMOE_DEV_WAIT_TIMEOUT, 43);
        *abort = 1;
        break;
      }
      tc_fence_after();
      if (F32) {
#pragma unroll
        for (int j = 0; j < F32_ROWS / 32; ++j) {
          if (j * 32 >= a.rows) continue;
          uint32_t v[32];
          tmem_ld32(tb + b * (a.tmem_cols / 2) + j * 32, v);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 32; ++i)
            acc[j][i] = first == kb0 ? __uint_as_float(v[i]) : acc[j][i] + __uint_as_float(v[i]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.tempty[b]);
      }
    }
    if (ok) {  // the ring's copies and MMAs are done: its memory takes the sums
      if (F32) {
#pragma unroll
        for (int j = 0; j < F32_ROWS / 32; ++j)
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (j * 32 + i < a.rows) sums[(j * 32 + i) * 128 + q * 32 + lane] = acc[j][i];
      } else {
#pragma unroll 1
        for (int c = 0; c < a.rows; c += 32) {
          uint32_t v[32];
          tmem_ld32(tb + c, v);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (c + i < a.rows) sums[(c + i) * 128 + q * 32 + lane] = __uint_as_float(v[i]);
        }
        tc_fence_before();
      }
    }
  }
  __syncthreads();
  if (s.abort) {
    volatile int* never = &s.zero;
    if (warp == 0 && lane == 0)
      for (int i = 0; i < a.stages; ++i)
        if ((issued_mask >> i) & 1u) mbar_wait(&s.full[i], (last_phase_bits >> i) & 1u, a.limit_ns, never);
    if (leader && mma_issued) {
      mma_commit(&s.drain);
      mbar_wait(&s.drain, 0, a.limit_ns, never);
    }
    __syncthreads();
  }
  cluster_sync();  // every CTA's sums are there
  {
    const int n = n0 + lane * 4;
    float b[4];
    load_bias4(b, a.e, n);
    const bool mine = lane * 4 < a.cols && n < a.e.N && !*abort;
    const int end = min(r1, a.e.M - m0);
#pragma unroll 1
    for (int r = r0 + warp; r < end; r += S_THREADS / 32) {
      float4 res = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (mine) res = load_residual4(a.e, m0 + r, n);
      float4 u[S_MAX_SPLIT];
#pragma unroll
      for (int j = 0; j < S_MAX_SPLIT; ++j)
        if (j < a.split) u[j] = load_rank(sums + r * 128 + lane * 4, j);
      float4 v = u[0];
#pragma unroll
      for (int j = 1; j < S_MAX_SPLIT; ++j)
        if (j < a.split) {
          v.x += u[j].x;
          v.y += u[j].y;
          v.z += u[j].z;
          v.w += u[j].w;
        }
      if (mine) finish4(a.e, m0 + r, n, v, b, res);
    }
  }
  cluster_sync();  // no CTA leaves while another reads its sums
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, a.tmem_cols);
  }
}

// ---------------------------------------------------------------- CTA pairs
constexpr int P_STAGES = 7;  // (six: 300 x 14336 x 4096 38.9 us for 36.4, 64 rows 26.3 for 25.6)
constexpr int P_STAGE_BYTES = 2 * W_BYTES;  // 128 weight rows and up to 128 rows of X a CTA
constexpr int P_GROUPS = 4;                 // of four epilogue warps, eight rows of a tile in turn
constexpr int P_THREADS = 64 + 128 * P_GROUPS;
constexpr int P_GROUP_ROWS = 16;            // row tiles that share a pass over the weights

struct PairSmem {
  uint64_t full[P_STAGES], empty[P_STAGES];
  uint64_t tfull[2], tempty[2], drain;
  uint32_t tmem_base;
  int abort, zero;
};
constexpr int P_SMEM = P_STAGES * P_STAGE_BYTES + 1024 + static_cast<int>(sizeof(PairSmem));
static_assert(P_SMEM <= 227 * 1024, "shared memory of the pair kernel");
static_assert(P_SMEM + S_MIN_SMEM > 226 * 1024, "no CTA of the split kernel beside its TMEM");

struct PairArgs {
  Epilogue e;
  int rows;  // of a tile: a multiple of 32, at most 256
  int cols;  // of a tile: a multiple of 16, at most 256. The MMA's rows past cols / 2 multiply what lies
             // in shared memory and are not stored (a row of A reaches its own lane alone)
  int row_tiles, col_tiles, kblocks;
  uint64_t limit_ns;
};

// Tiles in groups of P_GROUP_ROWS row tiles, in a group all row tiles of a column tile one after
// the other: pairs at work together share their weights and rows in L2.
__device__ __forceinline__ void pair_tile(int tile, const PairArgs& a, int& m0, int& n0) {
  const int per = P_GROUP_ROWS * a.col_tiles, g = tile / per, i = tile - g * per;
  const int in = min(P_GROUP_ROWS, a.row_tiles - g * P_GROUP_ROWS);
  const int ct = i / in;
  m0 = (g * P_GROUP_ROWS + i - ct * in) * a.rows;
  n0 = ct * a.cols;
}

// The even CTA's barrier, on which both CTAs' copies and arrivals count.
__device__ __forceinline__ uint32_t lead_barrier(uint64_t* bar) { return mapa_shared(smem_u32(bar), 0); }

// Eight columns of this warp's lanes.
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}

template <bool F32>
__global__ void __launch_bounds__(P_THREADS, 1)
    linear_pair_kernel(const __grid_constant__ CUtensorMap mapW, const __grid_constant__ CUtensorMap mapX,
                       const __grid_constant__ PairArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* ring = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  PairSmem& s = *reinterpret_cast<PairSmem*>(ring + P_STAGES * P_STAGE_BYTES);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = static_cast<int>(cluster_ctarank() & 1u);
  const bool even = rank == 0;
  pdl_trigger();
  if (warp == 0 && lane == 0) {
    tma_prefetch_map(&mapW);
    tma_prefetch_map(&mapX);
  }
  if (tid == 0) {
    for (int i = 0; i < P_STAGES; ++i) {
      mbar_init(&s.full[i], 1);
      mbar_init(&s.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s.tfull[i], 1);
      mbar_init(&s.tempty[i], 2 * 4 * P_GROUPS);  // every epilogue warp of both CTAs
    }
    mbar_init(&s.drain, 1);
    s.abort = 0;
    s.zero = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc_pair(&s.tmem_base, 512);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  cluster_sync();  // barriers of both CTAs initialised, TMEM allocated
  tc_fence_after();
  pdl_wait();  // every thread: the previous kernel's outputs are visible
  const uint32_t tmem_base = s.tmem_base;
  volatile int* abort = &s.abort;
  const int pair = blockIdx.x / 2, pairs = gridDim.x / 2;
  const int total = a.row_tiles * a.col_tiles;
  const int half = a.rows / 2, cols = a.cols / 2;  // rows of X and of W in a CTA's shared memory
  const int part = F32 ? F32_BLOCKS : a.kblocks;  // K blocks of an accumulator, two in turn
  uint32_t issued_mask = 0, last_phase_bits = 0;
  bool mma_issued = false, leader = false;

  if (warp == 0) {
    const bool issuer = elect_one();
    const uint32_t bytes = 2u * static_cast<uint32_t>((cols + half) * BK * 2);
    int slot = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int tile = pair; tile < total && ok; tile += pairs) {
      int m0, n0;
      pair_tile(tile, a, m0, n0);
      for (int kb = 0; kb < a.kblocks; ++kb) {
        if (!__all_sync(0xffffffffu, mbar_wait(&s.empty[slot], phase ^ 1u, a.limit_ns, abort))) {
          if (issuer && !*abort) report(&g_err_linear, ORDERMOE_DEV_WAIT_TIMEOUT, 51);
          *abort = 1;
          ok = false;
          break;
        }
        if (issuer) {
          uint8_t* p = ring + slot * P_STAGE_BYTES;
          if (even) mbar_arrive_expect_tx(&s.full[slot], bytes);
          const uint32_t full = lead_barrier(&s.full[slot]);
          tma_load_2d_pair(p, &mapW, full, kb * BK, n0 + rank * cols);
          tma_load_2d_pair(p + W_BYTES, &mapX, full, kb * BK, m0 + rank * half);
        }
        issued_mask |= 1u << slot;
        last_phase_bits = (last_phase_bits & ~(1u << slot)) | (phase << slot);
        if (++slot == P_STAGES) {
          slot = 0;
          phase ^= 1u;
        }
      }
    }
  } else if (warp == 1) {
    if (even) {
      leader = elect_one();
      const uint64_t desc0 = sdesc_kmajor_sw128(smem_u32(ring));
      const uint32_t idesc = idesc_bf16_f32(256, a.rows);
      int slot = 0, it = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int tile = pair; tile < total && ok; tile += pairs)
        for (int first = 0; first < a.kblocks && ok; first += part, ++it) {
          const int b = it & 1, end = min(first + part, a.kblocks);
          if (!__all_sync(0xffffffffu, mbar_wait(&s.tempty[b], ((it >> 1) & 1) ^ 1u, a.limit_ns, abort))) {
            if (leader && !*abort) report(&g_err_linear, ORDERMOE_DEV_WAIT_TIMEOUT, 52);
            *abort = 1;
            ok = false;
            break;
          }
          tc_fence_after();
          for (int kb = first; kb < end; ++kb) {
            if (!__all_sync(0xffffffffu, mbar_wait(&s.full[slot], phase, a.limit_ns, abort))) {
              if (leader && !*abort) report(&g_err_linear, ORDERMOE_DEV_WAIT_TIMEOUT, 53);
              *abort = 1;
              ok = false;
              break;
            }
            tc_fence_after();
            const uint64_t dw = desc0 + static_cast<uint64_t>((slot * P_STAGE_BYTES) >> 4), dx = dw + (W_BYTES >> 4);
            if (leader) {
#pragma unroll
              for (int kk = 0; kk < BK / 16; ++kk)  // 16 elements = 32 bytes on
                mma_bf16_pair(tmem_base + b * 256, dw + 2 * kk, dx + 2 * kk, idesc,
                              kb != first || kk != 0 ? 1u : 0u);
              mma_commit_pair(&s.empty[slot], 0x3);
            }
            mma_issued = true;
            if (++slot == P_STAGES) {
              slot = 0;
              phase ^= 1u;
            }
          }
          if (ok && leader) mma_commit_pair(&s.tfull[b], 0x3);
          __syncwarp();
        }
    }
  } else {
    // A thread's column of eight rows at a time, straight from TMEM: a warp writes 64 bytes of a row (128 in
    // fp32), whatever the strides.
    const int q = warp & 3, group = (warp - 2) >> 2, column = q * 32 + lane;
    int it = 0;
    bool go = true;
    auto arrived = [&]() {  // this unit's accumulator is there
      const bool ok = __all_sync(0xffffffffu, mbar_wait(&s.tfull[it & 1], (it >> 1) & 1, a.limit_ns, abort));
      if (!ok) {
        if (lane == 0 && !*abort) report(&g_err_linear, ORDERMOE_DEV_WAIT_TIMEOUT, 54);
        *abort = 1;
      }
      tc_fence_after();
      return ok;
    };
    auto taken = [&]() {  // its columns may be written again
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_remote(lead_barrier(&s.tempty[it & 1]));
      ++it;
    };
    for (int tile = pair; tile < total && go; tile += pairs) {
      int m0, n0;
      pair_tile(tile, a, m0, n0);
      const int rows = min(a.rows, a.e.M - m0), n = n0 + rank * cols + column;
      const bool mine = column < cols && n < a.e.N;
      const uint32_t tb = tmem_base + (static_cast<uint32_t>(q * 32) << 16);
      const float bias = mine && a.e.bias != nullptr ? bf16_lo(a.e.bias[n]) : 0.0f;
      const bool add = mine && a.e.residual != nullptr;
      uint32_t res[8], next[8];
      auto load_next = [&](int r) {  // the residual of rows r .. r + 7
        if (!add) return;
        const uint16_t* p = a.e.residual + (m0 + r) * a.e.ldr + n;
#pragma unroll
        for (int i = 0; i < 8; ++i, p += a.e.ldr)
          if (r + i < rows) next[i] = *p;
      };
      auto finish = [&](float (&v)[8], int r) {
        if (!mine) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += bias;
        activate_all<8, !F32>(v, a.e.act);
        if (add) {
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] += bf16_lo(res[i]);
        }
        if constexpr (F32) {
          float* y = static_cast<float*>(a.e.Y) + (m0 + r) * a.e.ldy + n;
#pragma unroll
          for (int i = 0; i < 8; ++i, y += a.e.ldy)
            if (r + i < rows) *y = v[i];
        } else {
          uint16_t* y = static_cast<uint16_t*>(a.e.Y) + (m0 + r) * a.e.ldy + n;
#pragma unroll
          for (int i = 0; i < 8; i += 2) {
            const uint32_t o = pack_bf16x2(v[i], v[i + 1]);
            if (r + i < rows) *y = static_cast<uint16_t>(o);
            y += a.e.ldy;
            if (r + i + 1 < rows) *y = static_cast<uint16_t>(o >> 16);
            y += a.e.ldy;
          }
        }
      };
      // (the first rows' residual while the sums are made, the others' one step ahead)
      load_next(group * 8);
      if constexpr (F32) {
        constexpr int BLOCKS = F32_PAIR_ROWS / 8 / P_GROUPS;
        float acc[BLOCKS][8];
        for (int first = 0; first < a.kblocks; first += part) {
          if (!(go = arrived())) break;
#pragma unroll
          for (int j = 0; j < BLOCKS; ++j) {
            const int r = (group + j * P_GROUPS) * 8;
            if (r >= rows) continue;
            uint32_t v[8];
            tmem_ld8(tb + (it & 1) * 256 + r, v);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 8; ++i)
              acc[j][i] = first == 0 ? __uint_as_float(v[i]) : acc[j][i] + __uint_as_float(v[i]);
          }
          taken();
        }
        if (!go) break;
#pragma unroll 1
        for (int j = 0; j < BLOCKS; ++j) {
          const int r = (group + j * P_GROUPS) * 8;
          if (r >= rows) break;
          float v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            v[i] = acc[0][i];
            res[i] = next[i];
#pragma unroll
            for (int b = 1; b < BLOCKS; ++b) v[i] = j == b ? acc[b][i] : v[i];
          }
          load_next(r + 8 * P_GROUPS);
          finish(v, r);
        }
      } else {
        if (!(go = arrived())) break;
#pragma unroll 1
        for (int r = group * 8; r < rows; r += 8 * P_GROUPS) {
          uint32_t u[8];
          tmem_ld8(tb + (it & 1) * 256 + r, u);  // TMEM column = row r + i of the tile
#pragma unroll
          for (int i = 0; i < 8; ++i) res[i] = next[i];
          load_next(r + 8 * P_GROUPS);
          tmem_ld_wait();
          float v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(u[i]);
          finish(v, r);
        }
        taken();
      }
    }
  }

  __syncthreads();
  if (s.abort) {
    volatile int* never = &s.zero;
    if (warp == 0 && lane == 0 && even)
      for (int i = 0; i < P_STAGES; ++i)
        if ((issued_mask >> i) & 1u) mbar_wait(&s.full[i], (last_phase_bits >> i) & 1u, a.limit_ns, never);
    if (leader && mma_issued) {
      mma_commit_pair(&s.drain, 0x1);
      mbar_wait(&s.drain, 0, a.limit_ns, never);
    }
  }
  tc_fence_before();
  cluster_sync();  // both CTAs finished: no more arrivals or copies into either
  tc_fence_after();
  if (warp == 1) tmem_dealloc_pair(tmem_base, 512);
}

// ------------------------------------------------------ CTA pairs, K over a cluster
constexpr int Q_STAGES = 6;
constexpr int Q_SMEM = Q_STAGES * P_STAGE_BYTES + 1024;
static_assert(Q_SMEM + S_MIN_SMEM > 226 * 1024, "no CTA of the split kernel beside its TMEM");
constexpr int Q_MAX_PAIRS = 4;
constexpr int Q_GROUPS = 4;  // of four epilogue warps
constexpr int Q_THREADS = 64 + 128 * Q_GROUPS;

struct PairSplitSmem {
  uint64_t full[Q_STAGES], empty[Q_STAGES];
  uint64_t tfull, drain;
  uint32_t tmem_base;
  int abort, zero;
};

struct PairSplitArgs {
  Epilogue e;
  int rows;  // of a tile: a multiple of 32, at most 256
  int row_tiles, kblocks, pairs;
  uint64_t limit_ns;
};

// The barrier of this pair's even CTA.
__device__ __forceinline__ uint32_t pair_barrier(uint64_t* bar, uint32_t lead) {
  return mapa_shared(smem_u32(bar), lead);
}

__global__ void __launch_bounds__(Q_THREADS, 1)
    linear_pair_split_kernel(const __grid_constant__ CUtensorMap mapW, const __grid_constant__ CUtensorMap mapX,
                             const __grid_constant__ PairSplitArgs a) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ PairSplitSmem s;
  uint8_t* ring = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  float* sums = reinterpret_cast<float*>(ring);  // [rows][128], when the main loop is done
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_ctarank(), lead = rank & ~1u;
  const int h = static_cast<int>(rank & 1u), pair = static_cast<int>(rank >> 1);
  const bool even = h == 0;
  pdl_trigger();
  if (warp == 0 && lane == 0) {
    tma_prefetch_map(&mapW);
    tma_prefetch_map(&mapX);
  }
  if (tid == 0) {
    for (int i = 0; i < Q_STAGES; ++i) {
      mbar_init(&s.full[i], 1);
      mbar_init(&s.empty[i], 1);
    }
    mbar_init(&s.tfull, 1);
    mbar_init(&s.drain, 1);
    s.abort = 0;
    s.zero = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc_pair(&s.tmem_base, 256);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  cluster_sync();  // every CTA's barriers are initialised, TMEM is allocated
  tc_fence_after();
  pdl_wait();  // every thread: the previous kernel's outputs are visible
  const uint32_t tmem_base = s.tmem_base;
  volatile int* abort = &s.abort;
  const int tile = static_cast<int>(blockIdx.x) / (2 * a.pairs);
  const int n0 = tile / a.row_tiles * 256 + h * 128, m0 = tile % a.row_tiles * a.rows;
  const int half = a.rows / 2;
  const int kb0 = static_cast<int>(static_cast<long long>(a.kblocks) * pair / a.pairs);
  const int kb1 = static_cast<int>(static_cast<long long>(a.kblocks) * (pair + 1) / a.pairs);
  const int r0 = a.rows * pair / a.pairs, r1 = a.rows * (pair + 1) / a.pairs;  // rows that this CTA finishes
  uint32_t issued_mask = 0, last_phase_bits = 0;
  bool mma_issued = false, leader = false;

  if (warp == 0) {
    const bool issuer = elect_one();
    const uint32_t bytes = 2u * static_cast<uint32_t>(W_BYTES + half * BK * 2);
    int slot = 0;
    uint32_t phase = 0;
    for (int kb = kb0; kb < kb1; ++kb) {
      if (!__all_sync(0xffffffffu, mbar_wait(&s.empty[slot], phase ^ 1u, a.limit_ns, abort))) {
        if (issuer && !*abort) report(&g_err_linear, ORDERMOE_DEV_WAIT_TIMEOUT, 61);
        *abort = 1;
        break;
      }
      if (issuer) {
        uint8_t* p = ring + slot * P_STAGE_BYTES;
        if (even) mbar_arrive_expect_tx(&s.full[slot], bytes);
        const uint32_t full = pair_barrier(&s.full[slot], lead);
        tma_load_2d_pair(p, &mapW, full, kb * BK, n0);
        tma_load_2d_pair(p + W_BYTES, &mapX, full, kb * BK, m0 + h * half);
      }
      issued_mask |= 1u << slot;
      last_phase_bits = (last_phase_bits & ~(1u << slot)) | (phase << slot);
      if (++slot == Q_STAGES) {
        slot = 0;
        phase ^= 1u;
      }
    }
  } else if (warp == 1) {
    if (even) {
      leader = elect_one();
      const uint64_t desc0 = sdesc_kmajor_sw128(smem_u32(ring));
      const uint32_t idesc = idesc_bf16_f32(256, a.rows);
      const uint16_t both = static_cast<uint16_t>(0x3u << lead);
      int slot = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!__all_sync(0xffffffffu, mbar_wait(&s.full[slot], phase, a.limit_ns, abort))) {
          if (leader && !*abort) report(&g_err_linear, ORDERMOE_DEV_WAIT_TIMEOUT, 62);
          *abort = 1;
          ok = false;
          break;
        }
        tc_fence_after();
        const uint64_t dw = desc0 + static_cast<uint64_t>((slot * P_STAGE_BYTES) >> 4), dx = dw + (W_BYTES >> 4);
        if (leader) {
#pragma unroll
          for (int kk = 0; kk < BK / 16; ++kk)  // 16 elements = 32 bytes on
            mma_bf16_pair(tmem_base, dw + 2 * kk, dx + 2 * kk, idesc, kb != kb0 || kk != 0 ? 1u : 0u);
          mma_commit_pair(&s.empty[slot], both);
        }
        mma_issued = true;
        if (++slot == Q_STAGES) {
          slot = 0;
          phase ^= 1u;
        }
      }
      if (ok && leader) mma_commit_pair(&s.tfull, both);
      __syncwarp();
    }
  } else {
    if (a.e.residual != nullptr && n0 + lane * 4 < a.e.N)
      for (int r = r0 + warp - 2; r < min(r1, a.e.M - m0); r += 4 * Q_GROUPS)
        prefetch_residual(a.e, m0 + r, n0 + lane * 4);
    const bool ok = __all_sync(0xffffffffu, mbar_wait(&s.tfull, 0, a.limit_ns, abort));
    if (!ok) {
      if (lane == 0 && !*abort) report(&g_err_linear, ORDERMOE_DEV_WAIT_TIMEOUT, 63);
      *abort = 1;
    } else {
      tc_fence_after();  // the pair's copies and MMAs are done: the ring's memory takes the sums
      const int q = warp & 3;
#pragma unroll 1
      for (int c = (warp - 2) / 4 * 32; c < a.rows; c += 32 * Q_GROUPS) {
        uint32_t v[32];
        tmem_ld32(tmem_base + (static_cast<uint32_t>(q * 32) << 16) + c, v);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 32; ++i) sums[(c + i) * 128 + q * 32 + lane] = __uint_as_float(v[i]);
      }
      tc_fence_before();
    }
  }
  __syncthreads();
  if (s.abort) {
    volatile int* never = &s.zero;
    if (warp == 0 && lane == 0 && even)
      for (int i = 0; i < Q_STAGES; ++i)
        if ((issued_mask >> i) & 1u) mbar_wait(&s.full[i], (last_phase_bits >> i) & 1u, a.limit_ns, never);
    if (leader && mma_issued) {
      mma_commit_pair(&s.drain, static_cast<uint16_t>(0x1u << lead));
      mbar_wait(&s.drain, 0, a.limit_ns, never);
    }
    __syncthreads();
  }
  cluster_sync();  // every CTA's sums are there
  {
    const int n = n0 + lane * 4, end = min(r1, a.e.M - m0);
    const bool mine = n < a.e.N && !*abort;
    float b[4];
    load_bias4(b, a.e, n);
#pragma unroll 1
    for (int r = r0 + warp; r < end; r += Q_THREADS / 32) {
      float4 res = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (mine) res = load_residual4(a.e, m0 + r, n);
      float4 u[Q_MAX_PAIRS];
#pragma unroll
      for (int j = 0; j < Q_MAX_PAIRS; ++j)
        if (j < a.pairs) u[j] = load_rank(sums + r * 128 + lane * 4, 2 * j + h);
      float4 v = u[0];
#pragma unroll
      for (int j = 1; j < Q_MAX_PAIRS; ++j)
        if (j < a.pairs) {
          v.x += u[j].x;
          v.y += u[j].y;
          v.z += u[j].z;
          v.w += u[j].w;
        }
      if (mine) finish4(a.e, m0 + r, n, v, b, res);
    }
  }
  tc_fence_before();
  cluster_sync();  // no CTA leaves while another reads its sums
  tc_fence_after();
  if (warp == 1) tmem_dealloc_pair(tmem_base, 256);
}

}  // namespace ln

// The pair kernel takes products of at least kLinearPairRows rows and kLinearPairTiles tiles of
// 256 x 256 (M x N x K in us, graph replays, bias and residual, pairs / split kernel: 64 x 14336 x 4096 (56
// tiles) 25.3 / 28.7, 128 rows 27.0 / 35.8, 256 rows 32.4 / 49.7; 768 x 4096 x 4096 (48) 23.4 / 42.2);
// and from kLinearPairLeast of them where the rows are kPairSplitRows or more (512 x 5120 x 5120
// (40) 27.0 / 46.2, 300 rows 22.6 / 28.6) or K is at most kLinearPairShort blocks (64 x 5120 x 1024 8.5 / 9.0,
// 128 rows 10.0 / 12.8; 128 x 5632 x 2048 13.3 / 15.6). Else the split kernel, whose CTAs stream the weights
// faster (128 x 5120 x 13824 44.5 / 37.4, 128 x 5120 x 5120 21.8 / 21.0; 64 x 4096 x 4096 (16) 16.5 / 12.2, 64 x
// 2048 x 8192 25.9 / 12.3; at 256 x 5120 x 5120 the pairs would be faster, 22.2 / 27.3).
constexpr int kLinearPairRows = 64, kLinearPairTiles = 48, kLinearPairLeast = 20, kLinearPairShort = 32;
// Below kLinearPairTiles, pairs share K from kPairSplitRows rows and kPairSplitBlocks K blocks (shared / split
// kernel: 160 x 4096 x 14336 35.1 / 31.4, 256 rows 37.2 / 37.7, 300 rows 38.7 / 51.3, 512 rows 46.7 / 59.8;
// 256 x 2048 x 2048 11.3 / 11.0, 300 rows 12.3 / 11.9, 512 rows 13.5 / 14.5), and from kPairSplitLong where there are
// kLinearPairLeast tiles (shared / pairs on their own: 300 x 4096 x 14336 38.9 / 47.2, 512 rows 46.9 / 47.3; 384 x
// 4096 x 8192 28.8 / 30.7, but 512 rows 33.2 / 30.6, 512 x 4096 x 6144 27.7 / 25.2; 384 x 4096 x 4096 20.1 / 19.3, 512
// rows 22.7 / 19.4; 768 x 2048 x 2048 15.4 / 13.3).
constexpr int kPairSplitRows = 257, kPairSplitBlocks = 32, kPairSplitLong = 96;

template <bool F32>
static cudaError_t linear_attr() {
  const cudaError_t e = cudaFuncSetAttribute(ln::linear_split_kernel<F32>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             227 * 1024 - static_cast<int>(sizeof(ln::SplitSmem)) - 256);
  if (e != cudaSuccess) return e;
  if (!F32) {
    const cudaError_t q = cudaFuncSetAttribute(ln::linear_pair_split_kernel,
                                               cudaFuncAttributeMaxDynamicSharedMemorySize, ln::Q_SMEM);
    if (q != cudaSuccess) return q;
  }
  return cudaFuncSetAttribute(ln::linear_pair_kernel<F32>, cudaFuncAttributeMaxDynamicSharedMemorySize, ln::P_SMEM);
}

static void cluster_config(cudaLaunchConfig_t& cfg, cudaLaunchAttribute* attr, int size, cudaStream_t stream) {
  cfg.stream = stream;
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = size;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // waits in the kernel
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl_on(stream) ? 2 : 1;
}

// CTA pairs that can be resident at once: the persistent grid never exceeds them.
static int linear_resident_pairs() {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  cluster_config(cfg, attr, 2, nullptr);
  cfg.numAttrs = 1;
  cfg.gridDim = dim3(2 * (num_sms() / 2), 1, 1);
  cfg.blockDim = dim3(ln::P_THREADS, 1, 1);
  cfg.dynamicSmemBytes = ln::P_SMEM;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, ln::linear_pair_kernel<false>, &cfg) != cudaSuccess || n <= 0) {
    cudaGetLastError();
    n = num_sms() / 2;
  }
  return n < num_sms() / 2 ? n : num_sms() / 2;
}

// Clusters of `pairs` (2 or 4) pairs that can be resident at once: a cluster stays within a GPC.
static int linear_resident_clusters(int pairs) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  cluster_config(cfg, attr, 2 * pairs, nullptr);
  cfg.numAttrs = 1;
  cfg.gridDim = dim3(num_sms() / (2 * pairs) * (2 * pairs), 1, 1);
  cfg.blockDim = dim3(ln::Q_THREADS, 1, 1);
  cfg.dynamicSmemBytes = ln::Q_SMEM;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, ln::linear_pair_split_kernel, &cfg) != cudaSuccess || n < 0) {
    cudaGetLastError();
    n = 0;
  }
  return n;
}

// What the choice of a kernel asks of a device: its SMs, and how many CTA pairs, clusters of two pairs and
// clusters of four are resident at once.
struct LinearDevice {
  int sms, pairs, clusters[2];
};

// The current device's, and the kernels' limits of shared memory: once per device (beyond the 64 that
// PerDevice keeps, at every call).
static cudaError_t linear_device(LinearDevice& dev) {
  static PerDevice cache;
  static LinearDevice devices[64];
  auto count = [](LinearDevice& to) {
    cudaError_t e = linear_attr<false>();
    if (e == cudaSuccess) e = linear_attr<true>();
    if (e == cudaSuccess)
      to = {num_sms(), linear_resident_pairs(), {linear_resident_clusters(2), linear_resident_clusters(4)}};
    return e;
  };
  int id = 0;
  const cudaError_t e = cudaGetDevice(&id);
  if (e != cudaSuccess) return e;
  if (id < 0 || id >= 64) return count(dev);
  const cudaError_t a =
      static_cast<cudaError_t>(per_device(cache, [&] { return static_cast<int>(count(devices[id])); }));
  if (a == cudaSuccess) dev = devices[id];  // (written before per_device returned)
  return a;
}

enum { LINEAR_SPLIT = 0, LINEAR_PAIR = 1, LINEAR_PAIR_SPLIT = 2 };
struct LinearPlan {
  int kernel;
  int rows, cols;  // of a tile
  int row_tiles, col_tiles;
  int split;       // CTAs (LINEAR_SPLIT) or pairs (LINEAR_PAIR_SPLIT) that share a tile's K
  int stages, x_rows, tmem_cols, smem;  // LINEAR_SPLIT
  int grid;
};

static long long div_up(long long x, long long y) { return (x + y - 1) / y; }

// The kernel of a product and its tiles; on the host alone. false: more tiles than 32 bits count.
static bool linear_plan(int M, int N, int K, bool f32, const LinearDevice& dev, LinearPlan& p) {
  using namespace ln;
  const int kblocks = static_cast<int>(div_up(K, BK));
  const long long p_tiles = div_up(M, 256) * div_up(N, 256);
  // pairs that share K: as many tiles as all clusters take at once, on most of the pairs
  if (!f32 && p_tiles < kLinearPairTiles && M >= kPairSplitRows &&
      kblocks >= (p_tiles < kLinearPairLeast ? kPairSplitBlocks : kPairSplitLong))
    for (int pairs = 2; pairs <= Q_MAX_PAIRS; pairs *= 2) {
      const long long ct = div_up(N, 256), cap = dev.clusters[pairs / 4];
      long long rt = cap / ct;  // row tiles of at most 256 rows and at least 64
      if (rt > div_up(M, 64)) rt = div_up(M, 64);
      if (rt < div_up(M, 256) || rt * ct * pairs * 4 < 3ll * (dev.sms / 2)) continue;
      p.kernel = LINEAR_PAIR_SPLIT;
      p.rows = static_cast<int>(div_up(div_up(M, rt), 32) * 32);
      p.cols = 256;
      p.row_tiles = static_cast<int>(div_up(M, p.rows));
      p.col_tiles = static_cast<int>(ct);
      p.split = pairs;
      p.grid = p.row_tiles * p.col_tiles * 2 * pairs;
      return true;
    }
  // pairs: even row tiles of at most 256 rows
  if (M >= kLinearPairRows &&
      (p_tiles >= kLinearPairTiles ||
       (p_tiles >= kLinearPairLeast && (M >= kPairSplitRows || kblocks <= kLinearPairShort)))) {
    p.kernel = LINEAR_PAIR;
    // Row tiles of 128 to 256 rows, by the rounds over the pairs that they take. A K block of a tile is taken
    // to cost the longer of its products, as rows, and its loads, 0.8 of (128 + rows / 2). (One round of N = 4096,
    // K = 14336 with start and epilogue: 256 rows 73 us, 224 67, 192 61, 160 55, 128 51, 96 46.) In tiles of up to
    // 256 rows / by this rule, N = 4096, K = 14336: 768 rows 70.7 / 57.3, 1500 rows 141 / 110, 2500 rows 220 / 172,
    // 4096 rows 322 / 285; 512 x 5632 x 2048 20.5 / 17.3. A gain of less than 3 % is left to the larger tiles, which
    // load less.
    const int most = dev.pairs;
    long long best = INT64_MAX;
    for (int rows = f32 ? F32_PAIR_ROWS : 256; rows >= 128; rows -= 32) {
      const long long rt = div_up(M, rows), even = div_up(div_up(M, rt), 32) * 32, loads = 102 + even * 2 / 5;
      const long long cost = div_up(rt * div_up(N, 256), most) * (even > loads ? even : loads);
      if (best == INT64_MAX || cost * 100 < best * 97) {
        best = cost;
        p.rows = static_cast<int>(even);
      }
    }
    p.row_tiles = static_cast<int>(div_up(M, p.rows));
    p.cols = 256;
    // One or two row tiles are bound by the weights' bytes: tiles as narrow as the same number of rounds
    // allows, so that every pair loads the same share (tiles of 256 columns / these: 64 x 32003 x 2048 28.1 / 27.5
    // us, 128 rows 30.1 / 29.9, 256 rows 35.7 / 35.9, 64 x 14336 x 4096 26.2 / 26.2). From three on, X's rows
    // loaded once more a column tile cost more (768 x 4096 x 14336 57.6 / 60.5, 1021 rows 81.5 / 83.3).
    if (p.row_tiles <= 2) {
      const long long rounds = div_up(p.row_tiles * div_up(N, 256), most);
      const long long even = div_up(div_up((long long)N * p.row_tiles, rounds * most), 16) * 16;
      if (even < 256 && p.row_tiles * div_up(N, even) <= rounds * most) p.cols = static_cast<int>(even);
    }
    p.col_tiles = static_cast<int>(div_up(N, p.cols));
    p.split = 1;
    if ((long long)p.row_tiles * p.col_tiles > INT32_MAX / 2) return false;
    const int tiles = p.row_tiles * p.col_tiles;
    p.grid = 2 * (tiles < most ? tiles : most);
    return true;
  }
  p.kernel = LINEAR_SPLIT;
  // Row tiles of 32 rows and more, as many as leave each tile four CTAs (or what K has for them) of two an
  // SM: the sums that a CTA exchanges and finishes are fewer (tiles of up to 128 rows / these, us:
  // 128 x 1024 x 2048 10.3 / 8.1, 128 x 2048 x 2048 10.9 / 9.0, 301 x 1009 x 1999 10.8 / 9.0, 64 x
  // 4096 x 4096 13.1 / 12.3, 1000 x 512 x 512 11.0 / 7.5). Without the four it loses (33 x 5632 x 2048 in
  // two row tiles 11.7 for 11.0).
  int want = 1;
  while (want < 4 && kblocks / (want * 2) >= 4) want *= 2;
  long long rt = 2ll * dev.sms / (div_up(N, 128) * want);
  if (rt > div_up(M, 32)) rt = div_up(M, 32);
  if (rt < div_up(M, f32 ? F32_ROWS : 128)) rt = div_up(M, f32 ? F32_ROWS : 128);
  p.rows = static_cast<int>(div_up(div_up(M, rt), 16) * 16);
  p.row_tiles = static_cast<int>(div_up(M, p.rows));
  long long tiles = p.row_tiles * div_up(N, 128);
  if (p.row_tiles * div_up(N, 80) > INT32_MAX / S_MAX_SPLIT) return false;
  // K over as many CTAs as two an SM leave room for, four K blocks each at least: two rings hide each
  // other's latency (1 x 4096 x 4096: 1, 2, 4, 8 CTAs a tile 18.0, 12.4, 11.3, 11.0 us;
  // 1 x 4096 x 14336: 48.6, 28.7, 24.7, 23.9)
  p.split = 1;
  while (p.split * 2 <= S_MAX_SPLIT && tiles * p.split * 2 <= 2ll * dev.sms && kblocks / (p.split * 2) >= 4) p.split *= 2;
  p.cols = 128;
  if (p.split <= 2 && tiles * p.split > dev.sms && tiles * p.split <= 2ll * dev.sms) {
    // narrower tiles where that gives every SM two CTAs (1 x 14336 x 4096: 128 columns 24.1 us, 96 23.7;
    // 128 x 10000 x 4096: 128 29.8, 80 28.6; 200 x 8100 x 2200: 128 26.9, 112 26.0). Wider clusters do not fill
    // the GPCs.
    const int even = static_cast<int>(div_up(div_up((long long)N * p.row_tiles * p.split, 2 * dev.sms), 16) * 16);
    p.cols = even < 80 ? 80 : even < 128 ? even : 128;
    if (p.row_tiles * div_up(N, p.cols) * p.split > 2ll * dev.sms) p.cols = 128;
    tiles = p.row_tiles * div_up(N, p.cols);
  }
  // One CTA an SM takes a ring of most of its shared memory, two half of it each. So do clusters of eight,
  // which do not fill the GPCs with one an SM (128 CTAs, 1 x 2048 x 8192: 18.0 us, two an SM 11.0, clusters of
  // four 12.6). Behind the ring what the MMA reads past the last stage's weights.
  const int stage = (p.cols + p.rows) * BK * 2, over = W_BYTES > stage ? W_BYTES - stage : 0;
  const int room = (tiles * p.split <= dev.sms && p.split < S_MAX_SPLIT ? 220 * 1024 : 108 * 1024) - over;
  const int share = (kblocks + p.split - 1) / p.split, need = (p.rows * 512 + stage - 1) / stage;
  p.stages = room / stage < S_MAX_STAGES ? room / stage : S_MAX_STAGES;
  if (p.stages > share) p.stages = share > need ? share : need;  // and the sums fit in it
  p.x_rows = M < p.rows ? M : p.rows;
  const int acc = p.rows <= 32 ? 32 : p.rows <= 64 ? 64 : 128;
  p.tmem_cols = f32 ? 2 * acc : acc;  // in turn, or the one of all K
  static_assert(2 * F32_ROWS <= S_MAX_COLS, "two accumulators");
  const int smem = p.stages * stage + over + 1024;
  p.smem = smem < S_MIN_SMEM ? S_MIN_SMEM : smem;
  p.col_tiles = static_cast<int>(tiles / p.row_tiles);
  p.grid = static_cast<int>(tiles * p.split);
  return true;
}

static int linear_launch(const uint16_t* X, int64_t ldx, const uint16_t* W, int64_t ldw, int M, int N, int K,
                         const ln::Epilogue& e, cudaStream_t stream) {
  using namespace ln;
  LinearDevice dev;
  const cudaError_t de = linear_device(dev);
  if (de != cudaSuccess) return cuda_fail(de, "cudaFuncSetAttribute(linear)");
  LinearPlan p{};
  if (!linear_plan(M, N, K, e.f32 != 0, dev, p))
    return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "linear: sizes too large");
  const int kblocks = static_cast<int>(div_up(K, BK));
  CUtensorMap mW, mX;
  int rc;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  cfg.gridDim = dim3(static_cast<unsigned>(p.grid), 1, 1);
  if (p.kernel == LINEAR_PAIR_SPLIT) {
    PairSplitArgs a{};
    a.e = e;
    a.rows = p.rows; a.row_tiles = p.row_tiles; a.kblocks = kblocks; a.pairs = p.split;
    a.limit_ns = wait_limit_ns();
    if ((rc = make_tmap_bf16_ld(&mW, W, N, K, ldw, 128))) return rc;
    if ((rc = make_tmap_bf16_ld(&mX, X, M, K, ldx, a.rows / 2))) return rc;
    cluster_config(cfg, attr, 2 * a.pairs, stream);
    cfg.blockDim = dim3(Q_THREADS, 1, 1);
    cfg.dynamicSmemBytes = Q_SMEM;
    const cudaError_t ce = cudaLaunchKernelEx(&cfg, linear_pair_split_kernel, mW, mX, a);
    if (ce != cudaSuccess) return cuda_fail(ce, "linear_pair_split_kernel");
    OM_LAUNCHED("linear_pair_split_kernel");
    return ORDERMOE_OK;
  }
  if (p.kernel == LINEAR_PAIR) {
    PairArgs a{};
    a.e = e;
    a.rows = p.rows; a.cols = p.cols; a.row_tiles = p.row_tiles; a.col_tiles = p.col_tiles; a.kblocks = kblocks;
    a.limit_ns = wait_limit_ns();
    if ((rc = make_tmap_bf16_ld(&mW, W, N, K, ldw, a.cols / 2))) return rc;
    if ((rc = make_tmap_bf16_ld(&mX, X, M, K, ldx, a.rows / 2))) return rc;
    cluster_config(cfg, attr, 2, stream);
    cfg.blockDim = dim3(P_THREADS, 1, 1);
    cfg.dynamicSmemBytes = P_SMEM;
    const cudaError_t ce = e.f32 ? cudaLaunchKernelEx(&cfg, linear_pair_kernel<true>, mW, mX, a)
                                 : cudaLaunchKernelEx(&cfg, linear_pair_kernel<false>, mW, mX, a);
    if (ce != cudaSuccess) return cuda_fail(ce, "linear_pair_kernel");
    OM_LAUNCHED("linear_pair_kernel");
    return ORDERMOE_OK;
  }
  SplitArgs a{};
  a.e = e;
  a.rows = p.rows; a.cols = p.cols; a.row_tiles = p.row_tiles; a.x_rows = p.x_rows; a.kblocks = kblocks;
  a.split = p.split; a.stages = p.stages; a.tmem_cols = p.tmem_cols;
  a.limit_ns = wait_limit_ns();
  if ((rc = make_tmap_bf16_ld(&mW, W, N, K, ldw, a.cols))) return rc;
  if ((rc = make_tmap_bf16_ld(&mX, X, M, K, ldx, a.x_rows))) return rc;
  cluster_config(cfg, attr, a.split, stream);
  cfg.blockDim = dim3(S_THREADS, 1, 1);
  cfg.dynamicSmemBytes = p.smem;
  const cudaError_t ce = e.f32 ? cudaLaunchKernelEx(&cfg, linear_split_kernel<true>, mW, mX, a)
                               : cudaLaunchKernelEx(&cfg, linear_split_kernel<false>, mW, mX, a);
  if (ce != cudaSuccess) return cuda_fail(ce, "linear_split_kernel");
  OM_LAUNCHED("linear_split_kernel");
  return ORDERMOE_OK;
}

}  // namespace om

using namespace om;

extern "C" int ordermoe_linear(const uint16_t* X, int64_t ldx, const uint16_t* W, int64_t ldw, const uint16_t* bias,
                               int act, const uint16_t* residual, int64_t ldr, int M, int N, int K, void* Y,
                               int64_t ldy, int f32, ordermoe_stream_t stream) {
  OM_TRACE();
  if (M < 0 || N <= 0 || K <= 0)
    return fail(ORDERMOE_ERR_INVALID_ARG, "linear: need M >= 0, N > 0 and K > 0");
  if (act < ORDERMOE_ACT_NONE || act > ORDERMOE_ACT_SILU)
    return fail(ORDERMOE_ERR_INVALID_ARG, "linear: unknown activation %d", act);
  if (ldx < K || ldw < K || ldy < N || (residual && ldr < N))
    return fail(ORDERMOE_ERR_INVALID_ARG, "linear: a row stride is shorter than the row");
  if (ldx % 8 != 0 || ldw % 8 != 0 || ldx >= (1ll << 38) || ldw >= (1ll << 38))
    return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "linear: ldx and ldw must be multiples of 8, below 2^38");
  constexpr int most = INT32_MAX - 512;  // indices of a tile's end stay in 32 bits
  if (M > most || N > most || K > most)
    return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "linear: need M, N and K of at most %d", most);
  if (M == 0) return ORDERMOE_OK;
  if (!X || !W || !Y) return fail(ORDERMOE_ERR_INVALID_ARG, "linear: null pointer");
  if (!aligned16(X) || !aligned16(W)) return fail(ORDERMOE_ERR_INVALID_ARG, "linear: X and W must be 16-byte aligned");
  const uintptr_t y = reinterpret_cast<uintptr_t>(Y), r = reinterpret_cast<uintptr_t>(residual);
  if (y % (f32 ? 4 : 2) != 0 || r % 2 != 0 || reinterpret_cast<uintptr_t>(bias) % 2 != 0)
    return fail(ORDERMOE_ERR_INVALID_ARG, "linear: Y, residual or bias is not aligned to its type");
  if (r == y && (f32 || (M > 1 && ldr != ldy)))
    return fail(ORDERMOE_ERR_INVALID_ARG, "linear: a Y that is the residual must have its type and stride");
  ln::Epilogue e{};
  e.M = M; e.N = N; e.bias = bias; e.residual = residual; e.Y = Y;
  e.ldr = ldr; e.ldy = ldy; e.act = act; e.f32 = f32 != 0;
  e.vec_r = ldr % 4 == 0 && r % 8 == 0;
  e.vec_y = ldy % 4 == 0 && y % (f32 ? 16 : 8) == 0;
  return linear_launch(X, ldx, W, ldw, M, N, K, e, stream);
}

extern "C" int ordermoe_selftest_linear_plan(int M, int N, int K, int f32, const int32_t* device, int32_t* plan) {
  OM_TRACE();
  if (M <= 0 || N <= 0 || K <= 0 || !plan)
    return fail(ORDERMOE_ERR_INVALID_ARG, "selftest_linear_plan: need M, N, K > 0 and a plan");
  LinearDevice dev;
  if (device) {
    dev = {device[0], device[1], {device[2], device[3]}};
    if (dev.sms < 2 || dev.pairs < 1 || dev.clusters[0] < 0 || dev.clusters[1] < 0)
      return fail(ORDERMOE_ERR_INVALID_ARG, "selftest_linear_plan: no such device");
  } else {
    const cudaError_t e = linear_device(dev);
    if (e != cudaSuccess) return cuda_fail(e, "cudaFuncSetAttribute(linear)");
  }
  LinearPlan p{};
  if (!linear_plan(M, N, K, f32 != 0, dev, p))
    return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "selftest_linear_plan: sizes too large");
  const int32_t v[8] = {p.kernel, p.rows, p.cols, p.row_tiles, p.col_tiles, p.split, p.stages, p.grid};
  for (int i = 0; i < 8; ++i) plan[i] = v[i];
  return ORDERMOE_OK;
}
