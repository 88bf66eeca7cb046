// Low-rank adapters of many requests beside a shared projection: Y[t] = residual[t] + scale_a B_a (A_a X[t]).
//
// Two products of R <= 128: H = A X^T by a first kernel (K shared out over CTAs, partial sums in fp32), B H by a second one.
// Both are bound by bytes (X, Y and the used adapters' weights), or with few tokens by latency. Tokens come in
// any order of adapters: a tile is 128 tokens, and a CTA takes the j-th distinct adapter among them with the tokens that
// have it, so an adapter's weights are read once a tile whatever the order.
#include "common.cuh"

namespace om {

static __device__ unsigned long long g_err_adapters = 0;

int read_clear_err_adapters(unsigned long long* out) {
  unsigned long long zero = 0;
  OM_CUDA(cudaMemcpyFromSymbol(out, g_err_adapters, sizeof(*out)));
  OM_CUDA(cudaMemcpyToSymbol(g_err_adapters, &zero, sizeof(zero)));
  return ORDERMOE_OK;
}

namespace ad {

constexpr int TILE = 128;      // tokens among which adapters are looked for
constexpr int THREADS = 256;
constexpr int MAX_R = 128;
constexpr int MAX_SPLIT = 32;  // CTAs that share K
constexpr int KB = 64;         // of K a step
constexpr int NB = 256;        // columns of a CTA of the second product

struct Args {
  const uint16_t* X; int64_t ldx;
  const uint16_t* A; int64_t stride_a, lda;
  const uint16_t* B; int64_t stride_b, ldb;
  const int32_t* ids;
  const int32_t* rank;
  const float* scale;
  const uint16_t* res; int64_t ldr;
  void* Y; int64_t ldy;
  int n, R, T, N, K, f32, split, share;  // share: steps of K of a CTA
  int vec_r, vec_y;                      // residual and Y may be moved 16 bytes at a time
  float* H;                              // [split][T][R]
};

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
               "{%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The tokens of a tile by adapter.
struct Groups {
  int id[TILE];       // adapter of each token, -1: none
  int leader[TILE];   // the first token of each distinct adapter, in order
  int row[TILE];      // tokens of the adapter in hand, in order
  int warp[4];
  int distinct, rows;
};

__device__ __forceinline__ void find_groups(const Args& a, Groups& s, int t0, bool tell) {
  const int tid = threadIdx.x, lane = tid % 32;
  if (tid < TILE) {
    int id = -1;
    if (t0 + tid < a.T) {
      id = a.ids[t0 + tid];
      if (id < -1 || id >= a.n) {
        if (tell) report(&g_err_adapters, ORDERMOE_DEV_BAD_INDEX, t0 + tid);
        id = -1;
      }
    }
    s.id[tid] = id;
  }
  __syncthreads();
  bool first = false;
  if (tid < TILE) {
    const int id = s.id[tid];
    first = id >= 0;
    for (int i = 0; i < tid && first; ++i) first = s.id[i] != id;
    const unsigned v = __ballot_sync(~0u, first);
    if (lane == 0) s.warp[tid / 32] = __popc(v);
  }
  __syncthreads();
  if (tid < TILE) {
    int at = 0;
    for (int i = 0; i < tid / 32; ++i) at += s.warp[i];
    const unsigned v = __ballot_sync(~0u, first);
    if (first) s.leader[at + __popc(v & ((1u << lane) - 1))] = tid;
    if (tid == TILE - 1) s.distinct = at + __popc(v);
  }
  __syncthreads();
}
// Lists the tokens with adapter `id` (tile's index, in order).
__device__ __forceinline__ void list_rows(Groups& s, int id) {
  const int tid = threadIdx.x, lane = tid % 32;
  __syncthreads();  // the rows before are done with
  bool on = false;
  unsigned v = 0;
  if (tid < TILE) {
    on = s.id[tid] == id;
    v = __ballot_sync(~0u, on);
    if (lane == 0) s.warp[tid / 32] = __popc(v);
  }
  __syncthreads();
  if (tid < TILE) {
    int at = 0;
    for (int i = 0; i < tid / 32; ++i) at += s.warp[i];
    if (on) s.row[at + __popc(v & ((1u << lane) - 1))] = tid;
    if (tid == TILE - 1) s.rows = at + __popc(v);
  }
  __syncthreads();
}
__device__ __forceinline__ int rank_of(const Args& a, int id, bool tell) {
  if (!a.rank) return a.R;
  const int r = a.rank[id];
  if (tell && (r < 0 || r > a.R) && threadIdx.x == 0) report(&g_err_adapters, ORDERMOE_DEV_BAD_INDEX, id);
  return r < 0 ? 0 : r > a.R ? a.R : r;
}

// 16-byte vectors of rows of 64 (8 vectors), exchanged by the row's lowest three bits.
__device__ __forceinline__ uint32_t at64(int row, int vec) { return (row * 8 + (vec ^ (row & 7))) * 16; }

// H[split][t][r] over a CTA's steps of K. A step has 64 of K of up to 128 tokens and all ranks in shared memory.
// Up to 16 tokens: the warps share the step's four products of 16 of K and halves of the ranks, and add up at the end;
// more: 16 tokens a warp.
constexpr int X_BYTES = TILE * KB * 2, A_BYTES = MAX_R * KB * 2, DOWN_STAGES = 3;
constexpr int DOWN_SMEM = DOWN_STAGES * (X_BYTES + A_BYTES);
__global__ void __launch_bounds__(THREADS) adapters_down_kernel(const Args a) {
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ Groups s;
  pdl_wait();
  pdl_trigger();
  const int t0 = blockIdx.x * TILE, tid = threadIdx.x, lane = tid % 32, w = tid / 32, g = lane / 4, q4 = lane % 4;
  const bool tell = blockIdx.y == 0 && blockIdx.z == 0;
  find_groups(a, s, t0, tell);
  const int k0 = blockIdx.z * a.share, steps_all = (a.K + KB - 1) / KB;
  const int k1 = min(k0 + a.share, steps_all);
  const uint32_t base = smem_u32(ring);
  for (int d = blockIdx.y; d < s.distinct; d += gridDim.y) {
    const int id = s.id[s.leader[d]];
    list_rows(s, id);
    const int rows = s.rows, r = rank_of(a, id, blockIdx.z == 0), rt = (r + 15) / 16 * 16;
    const int m16 = (rows + 15) / 16 * 16;
    const uint16_t* A = a.A + id * a.stride_a;
    auto fetch = [&](int kb, int stage) {
      const uint32_t xs = base + stage * (X_BYTES + A_BYTES), as = xs + X_BYTES;
      for (int i = tid; i < m16 * 8; i += THREADS) {
        const int row = i / 8, v = i % 8, k = kb * KB + v * 8;
        const int left = row < rows ? min(8, a.K - k) : 0;
        cp16(xs + at64(row, v), left > 0 ? a.X + (t0 + s.row[row]) * a.ldx + k : a.X, left > 0 ? left * 2 : 0);
      }
      for (int i = tid; i < rt * 8; i += THREADS) {
        const int row = i / 8, v = i % 8, k = kb * KB + v * 8;
        const int left = row < r ? min(8, a.K - k) : 0;
        cp16(as + at64(row, v), left > 0 ? A + row * a.lda + k : a.A, left > 0 ? left * 2 : 0);
      }
    };
    for (int i = 0; i < DOWN_STAGES - 1; ++i) {
      if (k0 + i < k1) fetch(k0 + i, i);
      cp_commit();
    }
    float acc[MAX_R / 8][4];
#pragma unroll
    for (int n = 0; n < MAX_R / 8; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.0f;
    const bool few = rows <= 16;
    for (int kb = k0; kb < k1; ++kb) {
      cp_wait<DOWN_STAGES - 2>();
      __syncthreads();
      const int next = kb + DOWN_STAGES - 1;
      if (next < k1) fetch(next, (next - k0) % DOWN_STAGES);
      cp_commit();
      const uint32_t xs = base + (kb - k0) % DOWN_STAGES * (X_BYTES + A_BYTES), as = xs + X_BYTES;
      const int m0 = few ? 0 : w * 16;
      if (m0 >= rows) continue;
#pragma unroll
      for (int k = 0; k < KB / 16; ++k) {
        if (few && k != (w & 3)) continue;
        uint32_t x[4], b[4];
        ldm4(x, xs + at64(m0 + (lane & 7) + (lane / 8 % 2) * 8, 2 * k + lane / 16));
#pragma unroll
        for (int n = 0; n < MAX_R / 8; n += 2) {
          if (n * 8 >= r || (few && (n / 2 & 1) != w / 4)) continue;
          ldm4(b, as + at64(n * 8 + (lane & 7) + lane / 16 * 8, 2 * k + lane / 8 % 2));
          mma(acc[n], x, b[0], b[1]);
          mma(acc[n + 1], x, b[2], b[3]);
        }
      }
    }
    cp_wait<0>();
    __syncthreads();
    float* H = a.H + (static_cast<int64_t>(blockIdx.z) * a.T + t0) * a.R;
    if (few) {  // four warps have sums of the same ranks
      float* part = reinterpret_cast<float*>(ring);  // [4][16][MAX_R]
#pragma unroll
      for (int n = 0; n < MAX_R / 8; ++n) {
        if (n * 8 >= r || (n / 2 & 1) != w / 4) continue;
        float* p = part + (w & 3) * 16 * MAX_R + n * 8 + q4 * 2;
        *reinterpret_cast<float2*>(p + g * MAX_R) = make_float2(acc[n][0], acc[n][1]);
        *reinterpret_cast<float2*>(p + (g + 8) * MAX_R) = make_float2(acc[n][2], acc[n][3]);
      }
      __syncthreads();
      for (int i = tid; i < rows * r; i += THREADS) {
        const int row = i / r, c = i % r;
        const float* p = part + row * MAX_R + c;
        H[static_cast<int64_t>(s.row[row]) * a.R + c] =
            (p[0] + p[16 * MAX_R]) + (p[2 * 16 * MAX_R] + p[3 * 16 * MAX_R]);
      }
    } else {
#pragma unroll
      for (int n = 0; n < MAX_R / 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = w * 16 + g + e / 2 * 8, c = n * 8 + q4 * 2 + e % 2;
          if (row < rows && c < r) H[static_cast<int64_t>(s.row[row]) * a.R + c] = acc[n][e];
        }
    }
    __syncthreads();
  }
}

// One token's part of Y: eight columns from c on, v their sums.
__device__ __forceinline__ void put8(const Args& a, int64_t t, int c, float* v) {
  const int left = min(8, a.N - c);
  if (left <= 0) return;
  if (a.res) {
    const uint16_t* r = a.res + t * a.ldr + c;
    if (a.vec_r && left == 8) {
      const uint4 u = *reinterpret_cast<const uint4*>(r);
      v[0] += bf16_lo(u.x); v[1] += bf16_hi(u.x); v[2] += bf16_lo(u.y); v[3] += bf16_hi(u.y);
      v[4] += bf16_lo(u.z); v[5] += bf16_hi(u.z); v[6] += bf16_lo(u.w); v[7] += bf16_hi(u.w);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < left) v[i] += bf16_lo(r[i]);
    }
  }
  if (a.f32) {
    float* y = static_cast<float*>(a.Y) + t * a.ldy + c;
    if (a.vec_y && left == 8) {
      *reinterpret_cast<float4*>(y) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4*>(y + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < left) y[i] = v[i];
    }
    return;
  }
  uint16_t* y = static_cast<uint16_t*>(a.Y) + t * a.ldy + c;
  if (a.vec_y && left == 8) {
    *reinterpret_cast<uint4*>(y) =
        make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) y[i] = static_cast<uint16_t>(pack_bf16x2(v[i], 0.0f));
  }
}

// Y = residual + scale B H, 256 columns of a tile's j-th distinct adapter. H's fp32 sums become two bf16 parts. The columns
// of four products of 8 are dealt out so that each thread holds eight in a row: column c of product j is
// 8 (c / 2) + 2 j + c % 2 of 32. Tokens without an adapter go with the first.
constexpr int ROW16 = MAX_R * 2;  // bytes of a row of H's parts and of B
constexpr int UP_SMEM = 2 * TILE * ROW16 + NB * ROW16;
__device__ __forceinline__ uint32_t at128(int row, int vec) { return row * ROW16 + (vec ^ (row & 7)) * 16; }
__global__ void __launch_bounds__(THREADS) adapters_up_kernel(const Args a) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ Groups s;
  pdl_wait();
  pdl_trigger();
  const int t0 = blockIdx.x * TILE, tid = threadIdx.x, lane = tid % 32, w = tid / 32, g = lane / 4, q4 = lane % 4;
  find_groups(a, s, t0, false);
  const int c0 = blockIdx.z * NB;
  if (blockIdx.y == 0)
    for (int i = tid; i < TILE * (NB / 8); i += THREADS) {
      const int row = i / (NB / 8), c = c0 + i % (NB / 8) * 8;
      if (t0 + row < a.T && s.id[row] < 0) {
        float v[8] = {};
        put8(a, t0 + row, c, v);
      }
    }
  const uint32_t hi = smem_u32(smem), lo = hi + TILE * ROW16, bs = lo + TILE * ROW16;
  for (int d = blockIdx.y; d < s.distinct; d += gridDim.y) {
    const int id = s.id[s.leader[d]];
    list_rows(s, id);
    const int rows = s.rows, r = rank_of(a, id, false), rv = (r + 15) / 16 * 2;  // vectors of 8 ranks, even
    const uint16_t* B = a.B + id * a.stride_b;
    for (int i = tid; i < NB * rv; i += THREADS) {
      const int row = i / rv, v = i % rv, left = c0 + row < a.N ? min(8, r - v * 8) : 0;
      cp16(bs + at128(row, v), left > 0 ? B + (c0 + row) * a.ldb + v * 8 : a.B, left > 0 ? left * 2 : 0);
    }
    cp_commit();
    const int m16 = (rows + 15) / 16 * 16;
    for (int i = tid; i < m16 * rv * 4; i += THREADS) {  // two ranks of a token
      const int row = i / (rv * 4), c = i % (rv * 4) * 2;
      float v[2] = {0.0f, 0.0f};
      if (row < rows)
        for (int p = 0; p < a.split; ++p) {
          const float* h = a.H + (static_cast<int64_t>(p) * a.T + t0 + s.row[row]) * a.R + c;
          if (c < r) v[0] += h[0];
          if (c + 1 < r) v[1] += h[1];
        }
      const uint32_t x = pack_bf16x2(v[0], v[1]);
      const uint32_t y = pack_bf16x2(v[0] - bf16_lo(x), v[1] - bf16_hi(x));
      const uint32_t at = at128(row, c / 8) + c % 8 * 2;
      *reinterpret_cast<uint32_t*>(smem + at) = x;
      *reinterpret_cast<uint32_t*>(smem + TILE * ROW16 + at) = y;
    }
    cp_wait<0>();
    __syncthreads();
    const float scale = a.scale ? a.scale[id] : 1.0f;
    const bool few = rows <= 16;  // 32 columns a warp, else 16 tokens a warp
    const int m0 = few ? 0 : w * 16;
    if (m0 < rows)
      for (int n0 = few ? w * 32 : 0; n0 < (few ? w * 32 + 32 : NB); n0 += 32) {
        float acc[4][4] = {};
        for (int k = 0; k < rv / 2; ++k) {
          uint32_t x[4], y[4], b[2][4];
          const int row = m0 + (lane & 7) + (lane / 8 % 2) * 8;
          ldm4(x, hi + at128(row, 2 * k + lane / 16));
          ldm4(y, lo + at128(row, 2 * k + lane / 16));
#pragma unroll
          for (int j = 0; j < 2; ++j) {  // products 2 j and 2 j + 1
            const int c = lane & 7, col = n0 + c / 2 * 8 + (2 * j + lane / 16) * 2 + c % 2;
            ldm4(b[j], bs + at128(col, 2 * k + lane / 8 % 2));
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            mma(acc[j], x, b[j / 2][j % 2 * 2], b[j / 2][j % 2 * 2 + 1]);
            mma(acc[j], y, b[j / 2][j % 2 * 2], b[j / 2][j % 2 * 2 + 1]);
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int row = m0 + g + h * 8;
          if (row >= rows) continue;
          float v[8];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            v[2 * j] = acc[j][2 * h] * scale;
            v[2 * j + 1] = acc[j][2 * h + 1] * scale;
          }
          put8(a, t0 + s.row[row], c0 + n0 + q4 * 8, v);
        }
      }
    __syncthreads();
  }
}

// How K is shared out: as many CTAs as fill the SMs twice with the tiles, four steps each at least.
struct Plan {
  int tiles, split, share;
};
static Plan plan(int T, int K) {
  Plan p{};
  p.tiles = (T + TILE - 1) / TILE;
  const int steps = (K + KB - 1) / KB;
  int want = 2 * 152 / p.tiles;
  if (want > MAX_SPLIT) want = MAX_SPLIT;
  if (want > steps / 4) want = steps / 4;
  if (want < 1) want = 1;
  p.share = (steps + want - 1) / want;
  p.split = (steps + p.share - 1) / p.share;
  return p;
}

static int adapters_attr() {
  cudaError_t e = cudaFuncSetAttribute(adapters_down_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, DOWN_SMEM);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(adapters_up_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, UP_SMEM);
  return static_cast<int>(e);
}

}  // namespace ad
}  // namespace om

using namespace om;

static bool sizes_ok(int T, int K, int N, int R) {
  return T >= 0 && K > 0 && N > 0 && T <= INT32_MAX - 512 && N <= INT32_MAX - 512 && K <= (1 << 30) && R >= 8 && R % 8 == 0 &&
         R <= ad::MAX_R;
}

extern "C" size_t ordermoe_adapters_workspace_bytes(int T, int K, int N, int R) {
  if (!sizes_ok(T, K, N, R) || T == 0) return 0;
  const ad::Plan p = ad::plan(T, K);
  return static_cast<size_t>(p.split) * T * R * 4;
}

extern "C" int ordermoe_adapters(const uint16_t* X, int64_t ldx, const uint16_t* A, int64_t stride_a, int64_t lda,
                                 const uint16_t* B, int64_t stride_b, int64_t ldb, const int32_t* ids,
                                 const int32_t* rank, const float* scale, int n, int R, const uint16_t* residual,
                                 int64_t ldr, int T, int N, int K, void* Y, int64_t ldy, int f32, void* workspace,
                                 size_t workspace_bytes, ordermoe_stream_t stream) {
  OM_TRACE();
  if (T < 0 || N <= 0 || K <= 0 || n <= 0)
    return fail(ORDERMOE_ERR_INVALID_ARG, "adapters: need T >= 0, N > 0, K > 0 and n > 0");
  if (!sizes_ok(T, K, N, R))
    return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "adapters: need R a multiple of 8, 8 to %d, and T, N and K within their limits",
                ad::MAX_R);
  if ((T > 1 && (ldx < K || ldy < N || (residual && ldr < N))) || lda < K || ldb < R ||
      (n > 1 && (stride_a < 0 || stride_b < 0)))
    return fail(ORDERMOE_ERR_INVALID_ARG, "adapters: a row stride is shorter than the row");
  const int64_t most = 1ll << 38;
  if ((T > 1 && ldx % 8 != 0) || lda % 8 != 0 || ldb % 8 != 0 || (n > 1 && (stride_a % 8 != 0 || stride_b % 8 != 0)) ||
      ldx >= most || lda >= most || ldb >= most || ldy >= most || ldr >= most)
    return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "adapters: the strides of X, A and B must be multiples of 8, below 2^38");
  if (T == 0) return ORDERMOE_OK;
  if (!X || !A || !B || !ids || !Y) return fail(ORDERMOE_ERR_INVALID_ARG, "adapters: null pointer");
  if (!aligned16(X) || !aligned16(A) || !aligned16(B))
    return fail(ORDERMOE_ERR_INVALID_ARG, "adapters: X, A and B must be 16-byte aligned");
  const uintptr_t y = reinterpret_cast<uintptr_t>(Y), r = reinterpret_cast<uintptr_t>(residual);
  if (y % (f32 ? 4 : 2) != 0 || r % 2 != 0 || reinterpret_cast<uintptr_t>(ids) % 4 != 0 ||
      reinterpret_cast<uintptr_t>(rank) % 4 != 0 || reinterpret_cast<uintptr_t>(scale) % 4 != 0)
    return fail(ORDERMOE_ERR_INVALID_ARG, "adapters: Y, residual, ids, rank or scale is not aligned to its type");
  if (r == y && (f32 || (T > 1 && ldr != ldy)))
    return fail(ORDERMOE_ERR_INVALID_ARG, "adapters: a Y that is the residual must have its type and stride");
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 != 0 ||
      workspace_bytes < ordermoe_adapters_workspace_bytes(T, K, N, R))
    return fail(ORDERMOE_ERR_INVALID_ARG, "adapters: workspace is null, too small or not 256-byte aligned");
  const int64_t slices = (static_cast<int64_t>(N) + ad::NB - 1) / ad::NB;
  if (slices > 65535) return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "adapters: need N of at most %d", 65535 * ad::NB);
  static PerDevice attr_;
  const int e = per_device(attr_, ad::adapters_attr);
  if (e != 0) return cuda_fail(static_cast<cudaError_t>(e), "cudaFuncSetAttribute(adapters)");
  const ad::Plan p = ad::plan(T, K);
  ad::Args a{};
  a.X = X; a.ldx = ldx; a.A = A; a.stride_a = stride_a; a.lda = lda; a.B = B; a.stride_b = stride_b; a.ldb = ldb;
  a.ids = ids; a.rank = rank; a.scale = scale; a.res = residual; a.ldr = ldr; a.Y = Y; a.ldy = ldy;
  a.n = n; a.R = R; a.T = T; a.N = N; a.K = K; a.f32 = f32 != 0; a.split = p.split; a.share = p.share;
  a.vec_r = ldr % 8 == 0 && r % 16 == 0;
  a.vec_y = ldy % (f32 ? 4 : 8) == 0 && y % 16 == 0;
  a.H = static_cast<float*>(workspace);
  // CTAs for a tile's distinct adapters: as many as it can have, while the grid is not many times the SMs
  const int distinct = T < n ? (T < ad::TILE ? T : ad::TILE) : (n < ad::TILE ? n : ad::TILE);
  auto side = [&](int64_t others) {
    const int64_t fill = 8ll * 152 / others + 1;
    return static_cast<unsigned>(fill < distinct ? fill : distinct);
  };
  OM_LAUNCH_PDL("adapters_down_kernel", ad::adapters_down_kernel,
                dim3(p.tiles, side(static_cast<int64_t>(p.tiles) * p.split), p.split), dim3(ad::THREADS),
                static_cast<size_t>(ad::DOWN_SMEM), stream, a);
  OM_LAUNCH_PDL("adapters_up_kernel", ad::adapters_up_kernel,
                dim3(p.tiles, side(p.tiles * slices), static_cast<unsigned>(slices)), dim3(ad::THREADS),
                static_cast<size_t>(ad::UP_SMEM), stream, a);
  return ORDERMOE_OK;
}
