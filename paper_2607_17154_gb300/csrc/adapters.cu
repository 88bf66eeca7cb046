// Low-rank adapters of many requests beside a shared projection: Y[t] = residual[t] + scale_a B_a (A_a X[t]).
//
// Two products of R <= 128: H = A X^T by a first kernel (K shared out over CTAs, partial sums in fp32), B H by a second one.
// What the operator cannot do without are bytes (X, Y, residual, the used adapters' weights); with few tokens latency is
// longer. Tokens come in any order of adapters: a tile is 128 tokens, and a CTA takes adapters of a tile with the tokens
// that have them, so an adapter's weights are read once a tile whatever the order (and from L2 by the later tiles). Both products run on
// mma.sync: the tokens of an adapter are its M side, 1 to 128 of them, in blocks of 16.
// Measured (both kernels, launched from the host): 1 token, K = N = 4096, R 16: 6.1 us; 128 tokens on 32 adapters, K 4096, N
// 6144, R 64: 16.0 us, floor 3.7; 4096 tokens on 8 adapters, K 4096, N 14336, R 64: 77 us = 3.7 TB/s, floor 42.6
// (the first kernel 15, the second 62: four products of 16 tokens x 32 columns a residual vector, 1.5 instructions a cycle
// and SM; its tensor pipe is busy for 25 us).
#include <type_traits>

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
constexpr int THREADS = 256, MAX_WARPS = 16;
constexpr int MAX_R = 128;
constexpr int MAX_SPLIT = 32;  // CTAs that share K
constexpr int KB = 64;         // of K a step
constexpr int NB = 128;        // columns of a slice of the second product

struct Args {
  const uint16_t* X; int64_t ldx;
  const uint16_t* A; int64_t stride_a, lda;
  const uint16_t* B; int64_t stride_b, ldb;
  const int32_t* ids;
  const int32_t* rank;
  const float* scale;
  const uint16_t* res; int64_t ldr;
  void* Y; int64_t ldy;
  int n, R, T, N, K, f32, split, ctas;   // the most parts of K, and the first kernel's CTAs of a tile
  int vec_r, vec_y;                      // residual and Y may be moved 16 bytes at a time
  int flat;                              // second kernel: all tiles' slices shared out evenly over the CTAs
  int rows, ranks;                       // of a tile, in steps of 16 (what shared memory is laid out for)
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
  alignas(16) int id[TILE];  // adapter of each token, -1: none, -2: no token
  int rank[TILE];            // its ranks in use and its scale
  float scale[TILE];
  int leader[TILE];          // the first token of each distinct adapter, in order
  uint8_t row[MAX_WARPS][TILE];  // tokens of the adapter in hand, in order; every warp has a list of its own
  int warp[TILE / 32];
  int distinct;
};

// Returns whether a token has no adapter.
__device__ __forceinline__ bool find_groups(const Args& a, Groups& s, int t0, bool tell) {
  const int tid = threadIdx.x, lane = tid % 32;
  int id = t0 + tid < a.T ? -1 : -2, rank = a.R;
  float scale = 1.0f;
  if (tid < TILE) {
    if (t0 + tid < a.T) {
      id = a.ids[t0 + tid];
      if (id < -1 || id >= a.n) {
        if (tell) report(&g_err_adapters, ORDERMOE_DEV_BAD_INDEX, t0 + tid);
        id = -1;
      }
    }
    s.id[tid] = id;
    if (id >= 0 && a.rank) rank = a.rank[id];
    if (id >= 0 && a.scale) scale = a.scale[id];
  }
  __syncthreads();
  bool first = false;
  if (tid < TILE) {
    const unsigned same = __match_any_sync(~0u, id);  // by every lane, with a token or without
    first = id >= 0 && (same & ((1u << lane) - 1)) == 0;
    bool seen = false;
    for (int i = 0; i < tid / 32 * 32; i += 4) {
      const int4 x = *reinterpret_cast<const int4*>(s.id + i);
      seen = seen || x.x == id || x.y == id || x.z == id || x.w == id;
    }
    first = first && !seen;
    const unsigned v = __ballot_sync(~0u, first);
    if (lane == 0) s.warp[tid / 32] = __popc(v);
    if (rank < 0 || rank > a.R) {
      if (tell && first) report(&g_err_adapters, ORDERMOE_DEV_BAD_INDEX, id);
      rank = rank < 0 ? 0 : a.R;
    }
    s.rank[tid] = rank;
    s.scale[tid] = scale;
  }
  __syncthreads();
  if (tid < TILE) {
    int at = 0;
    for (int i = 0; i < tid / 32; ++i) at += s.warp[i];
    const unsigned v = __ballot_sync(~0u, first);
    if (first) s.leader[at + __popc(v & ((1u << lane) - 1))] = tid;
    if (tid == TILE - 1) s.distinct = at + __popc(v);
  }
  return __syncthreads_or(tid < TILE && id == -1);
}
// Lists the tokens with adapter `id` (tile's index, in order) for this warp; their number.
__device__ __forceinline__ int list_rows(Groups& s, int id) {
  const int lane = threadIdx.x % 32, w = threadIdx.x / 32;
  int at = 0;
  __syncwarp();  // the list before is done with
#pragma unroll
  for (int i = 0; i < TILE; i += 32) {
    const bool on = s.id[i + lane] == id;
    const unsigned v = __ballot_sync(~0u, on);
    if (on) s.row[w][at + __popc(v & ((1u << lane) - 1))] = static_cast<uint8_t>(i + lane);
    at += __popc(v);
  }
  __syncwarp();
  return at;
}

// Into how many parts K goes for every adapter of a tile, so that its adapters use the tile's CTAs; `share`: steps of a part.
__device__ __forceinline__ int tile_split(const Args& a, int distinct, int& share) {
  const int steps = (a.K + KB - 1) / KB, want = distinct > 0 ? a.ctas / distinct : 1;
  share = (steps + a.split - 1) / a.split;
  if (want < a.split) share = want > 1 ? (steps + want - 1) / want : steps;
  return (steps + share - 1) / share;
}

// 16-byte vectors of rows of 64 (8 vectors), exchanged by the row's lowest three bits.
__device__ __forceinline__ uint32_t at64(int row, int vec) { return (row * 8 + (vec ^ (row & 7))) * 16; }

// H[split][t][r] over a CTA's part of K, in steps of 64 of K of up to 128 tokens and all ranks in shared memory, 16 tokens
// a warp. Up to 16 tokens: steps of 128, whose instructions are fewer (64: 51 us where 128 take 18, 9 tiles x 32 adapters of 4
// tokens, K 4431, R 16); the warps share a step's products of 16 of K and the ranks, and add up at the end.
constexpr int FEW_KB = 128, MANY_STAGES = 3;
constexpr int few_stages(int ranks) { return ranks <= 64 ? 4 : 3; }  // so that an SM has room for two CTAs
constexpr int SUMS = 4 * 16 * (MAX_R + 2) * 4;  // bytes of four warps' sums of 16 tokens
constexpr int down_smem(int rows, int ranks) {
  const int many = MANY_STAGES * (rows + ranks) * KB * 2, few = few_stages(ranks) * (16 + ranks) * FEW_KB * 2;
  const int ring = many > few && rows > 16 ? many : few;
  return ring > SUMS ? ring : SUMS;
}
__global__ void __launch_bounds__(THREADS, 2) adapters_down_kernel(const Args a) {
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ Groups s;
  pdl_wait();
  pdl_trigger();
  const int t0 = blockIdx.x * TILE, tid = threadIdx.x, lane = tid % 32, w = tid / 32, g = lane / 4, q4 = lane % 4;
  find_groups(a, s, t0, blockIdx.y == 0);
  int share;
  const int split = tile_split(a, s.distinct, share), part_of = blockIdx.y % split, dg = gridDim.y / split;
  const int k0 = part_of * share, k1 = min(k0 + share, (a.K + KB - 1) / KB);
  if (static_cast<int>(blockIdx.y) / split >= dg) return;
  const uint32_t base = smem_u32(ring);
  for (int d = blockIdx.y / split; d < s.distinct; d += dg) {
    const int lead = s.leader[d], id = s.id[lead], rows = list_rows(s, id), r = s.rank[lead], rt = (r + 15) / 16 * 16;
    const int m16 = (rows + 15) / 16 * 16;
    const uint16_t* A = a.A + id * a.stride_a;
    const bool few = rows <= 16;
    // Results of 32 bits: a sum of at most 512 of K at a time, added up in H by the thread that has it. The tensor
    // cores cut a running sum (K 14336 in parts of 1600: 4.0e-6 off in the 2-norm, the plain form in fp32 1.3e-6).
    const int chunk = a.f32 && few ? 512 / KB : k1 - k0;  // (many tokens: see flush)
    float* const H = a.H + (static_cast<int64_t>(part_of) * a.T + t0) * a.R;
    for (int kc0 = k0; kc0 < k1; kc0 += chunk) {
      float acc[MAX_R / 8][4];
#pragma unroll
      for (int n = 0; n < MAX_R / 8; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.0f;
      // `count` steps through a ring of `stages`: `fetch` fills a stage, `step` has its products.
      auto steps = [&](auto stages, int count, int stage_bytes, auto fetch, auto step) {
        constexpr int STAGES = decltype(stages)::value;
        for (int i = 0; i < STAGES - 1; ++i) {
          if (i < count) fetch(i, base + i * stage_bytes);
          cp_commit();
        }
        int stage = 0, free = STAGES - 1;
        for (int i = 0; i < count; ++i) {
          cp_wait<STAGES - 2>();
          __syncthreads();
          if (i + STAGES - 1 < count) fetch(i + STAGES - 1, base + free * stage_bytes);
          cp_commit();
          free = free + 1 == STAGES ? 0 : free + 1;
          step(base + stage * stage_bytes);
          stage = stage + 1 == STAGES ? 0 : stage + 1;
        }
      };
      bool held = false;  // H has a sum of this thread's
      auto flush = [&]() {  // more than 16 tokens: a warp's 16 of them
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int row = w * 16 + g + h * 8;
          if (row >= rows) continue;
          float* to = H + static_cast<int64_t>(s.row[w][row]) * a.R + q4 * 2;  // (a column behind the rank is not read)
#pragma unroll
          for (int n = 0; n < MAX_R / 8; ++n) {
            if (n * 8 + q4 * 2 >= r) continue;
            float2 v = make_float2(acc[n][2 * h], acc[n][2 * h + 1]);
            if (held) {
              const float2 was = *reinterpret_cast<const float2*>(to + n * 8);
              v = make_float2(was.x + v.x, was.y + v.y);
            }
            *reinterpret_cast<float2*>(to + n * 8) = v;
            acc[n][2 * h] = acc[n][2 * h + 1] = 0.0f;
          }
        }
        held = true;
      };
      const int kc1 = min(kc0 + chunk, k1), k_first = kc0 * KB, k_end = min(kc1 * KB, a.K);
      if (few) {  // steps of 128 of K: a row is 16 vectors, a thread's rows are tid / 16 and of A every 16th from there
        constexpr int X_BYTES = 16 * FEW_KB * 2;
        const int v = tid % 16, row = tid / 16;
        const uint16_t* xp = row < rows ? a.X + (t0 + s.row[w][row]) * a.ldx + k_first + v * 8 : nullptr;
        const uint16_t* ap = A + row * a.lda + k_first + v * 8;
        auto at = [](int r_, int v_) { return (r_ * 16 + (v_ ^ (r_ & 7))) * 16; };
        const uint32_t place = at(row, v);
        auto fetch = [&](int i, uint32_t stage) {
          const int left = k_end - k_first - i * FEW_KB - v * 8, bytes = left >= 8 ? 16 : left > 0 ? left * 2 : 0;
          const bool on = xp && bytes > 0;
          cp16(stage + place, on ? xp + i * FEW_KB : a.X, on ? bytes : 0);
#pragma unroll
          for (int e = 0; e < MAX_R / 16; ++e) {
            if (e * 16 >= rt) break;
            const bool ok = row + e * 16 < r && bytes > 0;
            cp16(stage + X_BYTES + place + e * X_BYTES, ok ? ap + e * 16 * a.lda + i * FEW_KB : a.A, ok ? bytes : 0);
          }
        };
        // warps w and w + 4 have products w % 4 and w % 4 + 4 of 16 of K, of every other 16 ranks
        auto step = [&](uint32_t xs) {
#pragma unroll
          for (int h = 0; h < FEW_KB / 64; ++h) {
            const int k = (w & 3) + 4 * h;
            uint32_t x[4], b[4];
            ldm4(x, xs + at((lane & 7) + (lane / 8 % 2) * 8, 2 * k + lane / 16));
#pragma unroll
            for (int n = 0; n < MAX_R / 8; n += 2) {
              if (n * 8 >= r) break;
              if ((n / 2 & 1) != w / 4) continue;
              ldm4(b, xs + X_BYTES + at(n * 8 + (lane & 7) + lane / 16 * 8, 2 * k + lane / 8 % 2));
              mma(acc[n], x, b[0], b[1]);
              mma(acc[n + 1], x, b[2], b[3]);
            }
          }
        };
        const int count = (k_end - k_first + FEW_KB - 1) / FEW_KB, bytes = (16 + a.ranks) * FEW_KB * 2;
        if (a.ranks <= 64) steps(std::integral_constant<int, few_stages(64)>{}, count, bytes, fetch, step);
        else steps(std::integral_constant<int, few_stages(MAX_R)>{}, count, bytes, fetch, step);
      } else {
        // a thread's rows are tid / 8 and every 32nd from there, of X and of A; its vector of a step is tid % 8
        const int v = tid % 8, x_bytes = a.rows * KB * 2;
        const uint16_t *xp[TILE / 32], *ap = A + (tid / 8) * a.lda + k_first + v * 8;
#pragma unroll
        for (int e = 0; e < TILE / 32; ++e)
          xp[e] = tid / 8 + e * 32 < rows ? a.X + (t0 + s.row[w][tid / 8 + e * 32]) * a.ldx + k_first + v * 8 : nullptr;
        const uint32_t place = at64(tid / 8, v);
        auto fetch = [&](int i, uint32_t stage) {
          const uint32_t xs = stage + place, as = xs + x_bytes;
          const int left = k_end - k_first - i * KB - v * 8, bytes = left >= 8 ? 16 : left > 0 ? left * 2 : 0;
#pragma unroll
          for (int e = 0; e < TILE / 32; ++e)
            if (tid / 8 + e * 32 < m16) {
              const bool ok = xp[e] && bytes > 0;
              cp16(xs + e * 32 * KB * 2, ok ? xp[e] + i * KB : a.X, ok ? bytes : 0);
            }
#pragma unroll
          for (int e = 0; e < MAX_R / 32; ++e)
            if (tid / 8 + e * 32 < rt) {
              const bool ok = tid / 8 + e * 32 < r && bytes > 0;
              cp16(as + e * 32 * KB * 2, ok ? ap + e * 32 * a.lda + i * KB : a.A, ok ? bytes : 0);
            }
        };
        int done = 0;
        auto step = [&](uint32_t xs) {
          if (w * 16 >= rows) return;
          if (a.f32 && done > 0 && done % (512 / KB) == 0) flush();
          ++done;
          const uint32_t as = xs + x_bytes;
          uint32_t x[KB / 16][4];
#pragma unroll
          for (int k = 0; k < KB / 16; ++k) ldm4(x[k], xs + at64(w * 16 + (lane & 7) + (lane / 8 % 2) * 8, 2 * k + lane / 16));
#pragma unroll
          for (int n = 0; n < MAX_R / 8; n += 2) {
            if (n * 8 >= r) break;
#pragma unroll
            for (int k = 0; k < KB / 16; ++k) {
              uint32_t b[4];
              ldm4(b, as + at64(n * 8 + (lane & 7) + lane / 16 * 8, 2 * k + lane / 8 % 2));
              mma(acc[n], x[k], b[0], b[1]);
              mma(acc[n + 1], x[k], b[2], b[3]);
            }
          }
        };
        steps(std::integral_constant<int, MANY_STAGES>{}, kc1 - kc0, x_bytes + a.ranks * KB * 2, fetch, step);
      }
      cp_wait<0>();
      __syncthreads();
      if (few) {  // four warps have sums of the same ranks
        float* part = reinterpret_cast<float*>(ring);  // [4][16][LD]
        constexpr int LD = MAX_R + 2;
#pragma unroll
        for (int n = 0; n < MAX_R / 8; ++n) {
          if (n * 8 >= r || (n / 2 & 1) != w / 4) continue;
          float* p = part + (w & 3) * 16 * LD + n * 8 + q4 * 2;
          *reinterpret_cast<float2*>(p + g * LD) = make_float2(acc[n][0], acc[n][1]);
          *reinterpret_cast<float2*>(p + (g + 8) * LD) = make_float2(acc[n][2], acc[n][3]);
        }
        __syncthreads();
        for (int i = tid; i < rows * r; i += THREADS) {
          const int row = i / r, c = i % r;
          const float* p = part + row * LD + c;
          float* h = H + static_cast<int64_t>(s.row[w][row]) * a.R + c;
          const float sum = (p[0] + p[16 * LD]) + (p[2 * 16 * LD] + p[3 * 16 * LD]);
          *h = kc0 == k0 ? sum : *h + sum;
        }
      } else {
        flush();
      }
      __syncthreads();
    }
  }
}

// Four of a token's ranks, c and on, from the first kernel's partial sums; zeros behind the rank.
__device__ __forceinline__ float4 sum_h(const Args& a, int split, int64_t t, int c, int r) {
  float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (c >= r) return v;
  const float* h = a.H + t * a.R + c;
#pragma unroll 8
  for (int p = 0; p < split; ++p, h += static_cast<int64_t>(a.T) * a.R) {
    const float4 x = *reinterpret_cast<const float4*>(h);
    v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
  }
  return make_float4(v.x, c + 1 < r ? v.y : 0.0f, c + 2 < r ? v.z : 0.0f, c + 3 < r ? v.w : 0.0f);
}
// Eight columns of a token's residual from c on, as they are.
__device__ __forceinline__ uint4 get8(const Args& a, int64_t t, int c) {
  const int left = a.N - c;
  uint4 u = make_uint4(0, 0, 0, 0);
  if (!a.res || left <= 0) return u;
  const uint16_t* r = a.res + t * a.ldr + c;
  if (a.vec_r && left >= 8) return *reinterpret_cast<const uint4*>(r);
  uint32_t x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = i < left ? r[i] : 0u;
  return make_uint4(x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16);
}
// One column of Y, u its residual's bits.
__device__ __forceinline__ void put1(const Args& a, int64_t t, int c, uint32_t u, float v) {
  v += bf16_lo(u);
  if (a.f32) static_cast<float*>(a.Y)[t * a.ldy + c] = v;
  else static_cast<uint16_t*>(a.Y)[t * a.ldy + c] = static_cast<uint16_t>(pack_bf16x2(v, 0.0f));
}
__device__ __forceinline__ uint4 pack8(const float* v) {
  return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}
// Y = u + v there.
__device__ __forceinline__ void put8(const Args& a, int64_t t, int c, const uint4& u, float* v) {
  const int left = a.N - c;
  if (left <= 0) return;
  v[0] += bf16_lo(u.x); v[1] += bf16_hi(u.x); v[2] += bf16_lo(u.y); v[3] += bf16_hi(u.y);
  v[4] += bf16_lo(u.z); v[5] += bf16_hi(u.z); v[6] += bf16_lo(u.w); v[7] += bf16_hi(u.w);
  if (a.f32) {
    float* y = static_cast<float*>(a.Y) + t * a.ldy + c;
    if (a.vec_y && left >= 8) {
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
  if (a.vec_y && left >= 8) {
    *reinterpret_cast<uint4*>(y) =
        make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) y[i] = static_cast<uint16_t>(pack_bf16x2(v[i], 0.0f));
  }
}

// Y = residual + scale B H for a tile's adapters, in slices of 128 columns, the next one's weights on their way while
// one is computed. H's fp32 sums, times the scale, become PARTS bf16 parts: two (16 bits) for results of 16 bits (with one
// Y would be off by as much again as its own rounding), three for those of 32. Warps share the blocks of 16 tokens and,
// where there are fewer of those, the slice's columns. The columns of four products of 8 are dealt out so that each thread
// holds eight in a row: column c of product j is 8 (c / 2) + 2 j + c % 2 of 32. What does not depend on H (weights,
// residual) is asked for before the first kernel has ended. Tokens without an adapter are a group of their own.
constexpr int up_row(int ranks) { return ranks * 2 + 16; }  // bytes of a row of H's parts and of B: no bank is met twice
// Threads of a CTA: two CTAs an SM, or one of as many warps where shared memory has no room for two; with few tokens
// registers (for weights) are worth more than warps.
constexpr bool up_pairs(int parts, int ranks) { return parts == 2 && ranks == 64; }
constexpr int up_threads(int parts, int ranks, bool few) { return few || up_pairs(parts, ranks) ? 256 : 512; }
constexpr int TURN = 16 * 33 * 4;  // bytes of 16 tokens x 32 columns, a warp
constexpr int up_smem(int rows, int ranks, int parts, bool few_tokens) {
  const int many = up_threads(parts, ranks, few_tokens) / 32 * TURN + (parts * rows + 2 * NB) * up_row(ranks);
  const int few = 16 * (MAX_R + 4) * 4;
  return rows > 16 && many > few ? many : few;  // 16 tokens at most: all adapters have few
}
template <int PARTS, int RANKS, bool FEW, bool PLAIN>
__global__ void __launch_bounds__(up_threads(PARTS, RANKS, FEW), up_pairs(PARTS, RANKS) ? 2 : 1)
    adapters_up_kernel(const Args a) {
  constexpr int THREADS = up_threads(PARTS, RANKS, FEW), WARPS = THREADS / 32;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ Groups s;
  __shared__ const uint16_t* res_of[PLAIN ? 1 : WARPS][16];  // a warp's rows
  __shared__ char* y_of[PLAIN ? 1 : WARPS][16];
  const int tid = threadIdx.x, lane = tid % 32, w = tid / 32, g = lane / 4, q4 = lane % 4;
  constexpr int ld = up_row(RANKS);
  float* const turn = reinterpret_cast<float*>(smem + w * TURN);
  uint8_t* const parts = smem + WARPS * TURN;
  const uint32_t hs = smem_u32(parts), bs = hs + PARTS * a.rows * ld;
  const int slices = (a.N + NB - 1) / NB;
  const long long all = static_cast<long long>(slices) * ((a.T - 1) / TILE + 1);
  const long long lo = all * blockIdx.x / gridDim.x, hi = all * (blockIdx.x + 1) / gridDim.x;  // flat: this CTA's slices
  const int tile0 = !FEW && a.flat ? static_cast<int>(lo / slices) : static_cast<int>(blockIdx.x);
  const int tile1 = !FEW && a.flat ? static_cast<int>((hi - 1) / slices) : tile0;
  bool waited = false;
  for (int tile = tile0; tile <= tile1; ++tile) {
    const int t0 = tile * TILE;
    const long long before = static_cast<long long>(tile) * slices;
    if (tile > tile0) __syncthreads();  // the groups before are done with
    const bool alone = find_groups(a, s, t0, false);
    // The tile's groups are its adapters, and the tokens without one. Few tokens an adapter: where the groups leave few of
    // the tile's CTAs idle each has as many for itself, which take every dz-th slice; else groups times slices are shared
    // out evenly, group after group. More tokens: a CTA has the same slices of every group, or of every dg-th where
    // there are more CTAs than slices, because groups of more tokens cost more (2001 tokens of runs of 466, R 128: 131 us,
    // groups apart 171).
    int share_k;
    const int split = tile_split(a, s.distinct, share_k);
    const int groups_of = s.distinct + (alone && a.res != a.Y ? 1 : 0), q = blockIdx.y, Q = gridDim.y;
    const bool apart = FEW && groups_of > 0 && groups_of <= Q && Q % groups_of <= Q / 16;
    const int dz = FEW ? (apart ? Q / groups_of : 1) : a.flat ? 1 : min(Q, slices), dg = FEW || a.flat ? 1 : Q / dz;
    int d0 = FEW || a.flat ? 0 : q / dz, d1 = !FEW && d0 >= dg ? 0 : groups_of;
    int z_first = a.flat ? static_cast<int>(max(lo - before, 0ll)) : q % dz, z_end = slices;
    long long u0 = 0, u1 = 0;
    if (!FEW && a.flat && hi - before < slices) z_end = static_cast<int>(hi - before);
    if (FEW && apart) {
      d0 = q / dz;
      d1 = min(d0 + 1, groups_of);
    } else if (FEW) {
      const long long units = static_cast<long long>(groups_of) * slices;
      u0 = units * q / Q;
      u1 = units * (q + 1) / Q;
      d0 = static_cast<int>(u0 / slices);
      d1 = static_cast<int>((u1 + slices - 1) / slices);
    }
    for (int d = d0; d < d1; d += dg) {
      if (FEW && apart) {
        z_first = q % dz;
      } else if (FEW) {
        const long long start = static_cast<long long>(d) * slices;
        z_first = static_cast<int>(max(u0 - start, 0ll));
        z_end = static_cast<int>(min(u1 - start, static_cast<long long>(slices)));
      }
      const int z0 = z_first, z1 = z_end;
      if (d == s.distinct) {  // tokens without an adapter: the residual as it is
        const int rows = list_rows(s, -1), mine = z1 > z0 ? (z1 - z0 + dz - 1) / dz : 0;
        const bool by8 = a.vec_y && (a.vec_r || !a.res) && a.N % 8 == 0;
        const int width = by8 ? NB / 8 : NB;
        for (int64_t i = tid; i < static_cast<int64_t>(mine) * rows * width; i += THREADS) {
          const int64_t t = t0 + s.row[w][i / width % rows];
          const int c = (z0 + static_cast<int>(i / (width * rows)) * dz) * NB + static_cast<int>(i % width) * (by8 ? 8 : 1);
          if (c >= a.N) continue;
          if (by8) {
            float v[8] = {};
            put8(a, t, c, get8(a, t, c), v);
          } else {
            put1(a, t, c, a.res ? a.res[t * a.ldr + c] : 0u, 0.0f);
          }
        }
        continue;
      }
      const int lead = s.leader[d], id = s.id[lead], rows = list_rows(s, id), r = s.rank[lead];
      const int rv = (r + 15) / 16 * 2;  // vectors of 8 ranks, even
      const uint16_t* B = a.B + id * a.stride_b;
      if (FEW && rows <= 16) {  // weights and H in registers, 32 columns a warp and turn
        float* sum = reinterpret_cast<float*>(smem);  // [16][LD] of H
        constexpr int LD = RANKS + 4;
        const int steps = (r + 31) / 32, groups = (a.N + 31) / 32;
        const float scale = s.scale[lead];
        int64_t tok[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) tok[h] = g + h * 8 < rows ? t0 + s.row[w][g + h * 8] : -1;
        // Within 32 ranks a thread has eight in a row, q4 * 8 and on: two products' shares, of weights and of H alike.
        uint4 b[4][RANKS / 32], u[2] = {};
        auto ask = [&](int n) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int col = n * 32 + g / 2 * 8 + j * 2 + g % 2;
            const uint16_t* from = B + col * a.ldb + q4 * 8;
#pragma unroll
            for (int k = 0; k < RANKS / 32; ++k) {
              b[j][k] = make_uint4(0, 0, 0, 0);
              if (col < a.N && k * 32 + q4 * 8 < r) b[j][k] = *reinterpret_cast<const uint4*>(from + k * 32);
            }
          }
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (tok[h] >= 0) u[h] = get8(a, tok[h], n * 32 + q4 * 8);
        };
        // eight times 32 columns a turn
        const int n0 = apart ? z0 * WARPS + w : z0 * (NB / 32) + w, dn = dz * WARPS;
        const int n1 = apart ? groups : min(z1 * (NB / 32), groups);
        if (n0 < n1) ask(n0);
        for (int n = n0 + dn; n < n1; n += dn)  // the turns behind it, as far as L2
          if (n * 32 + lane < a.N)
            for (int c = 0; c < r; c += 64)
              asm volatile("prefetch.global.L2 [%0];" ::"l"(B + (n * 32 + lane) * a.ldb + c));
        if (!waited) pdl_wait();
        waited = true;
        for (int i = tid; i < 16 * steps * 8; i += THREADS) {  // four ranks of a token
          const int row = i / (steps * 8), c = (i - row * steps * 8) * 4;
          const float4 v = row < rows ? sum_h(a, split, static_cast<int64_t>(t0) + s.row[w][row], c, r) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          *reinterpret_cast<float4*>(sum + row * LD + c) = v;
        }
        __syncthreads();
        for (int n = n0; n < n1; n += dn) {
          float acc[4][4] = {};
#pragma unroll
          for (int k = 0; k < RANKS / 32; ++k) {
            if (k >= steps) continue;
            if (k * 32 + 32 > r) {  // columns behind the rank say nothing, whatever they hold
              const int left = r - k * 32 - q4 * 8;
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                uint32_t* x = reinterpret_cast<uint32_t*>(&b[j][k]);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = 2 * e + 1 < left ? x[e] : 2 * e < left ? x[e] & 0xFFFFu : 0u;
              }
            }
            float h[2][8];
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
              for (int f = 0; f < 2; ++f)
                *reinterpret_cast<float4*>(&h[e][4 * f]) =
                    *reinterpret_cast<const float4*>(sum + (g + 8 * e) * LD + k * 32 + q4 * 8 + f * 4);
#pragma unroll
            for (int p = 0; p < PARTS; ++p)
#pragma unroll
              for (int half = 0; half < 2; ++half) {
                uint32_t x[4];  // rows g, g + 8 of ranks 4 half, + 1, then of + 2, + 3
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  float* v = &h[e & 1][4 * half + (e / 2) * 2];
                  x[e] = pack_bf16x2(v[0], v[1]);
                  v[0] -= bf16_lo(x[e]);
                  v[1] -= bf16_hi(x[e]);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
                  if (half == 0) mma(acc[j], x, b[j][k].x, b[j][k].y);
                  else mma(acc[j], x, b[j][k].z, b[j][k].w);
              }
          }
          const uint4 now[2] = {u[0], u[1]};
          if (n + dn < n1) ask(n + dn);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (tok[h] < 0) continue;
            float v[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              v[2 * j] = acc[j][2 * h] * scale;
              v[2 * j + 1] = acc[j][2 * h + 1] * scale;
            }
            put8(a, tok[h], n * 32 + q4 * 8, now[h], v);
          }
        }
        __syncthreads();
        continue;
      }
      constexpr int VECS = RANKS / 8, ROWS = THREADS / VECS;  // a thread's vector is tid % VECS, of every ROWS-th column
      const int fv = tid % VECS, fleft = min(8, r - fv * 8);
      const uint16_t* fp = B + (tid / VECS) * a.ldb + fv * 8;
      auto fetch = [&](int z, int buffer) {
        if (fv >= rv) return;
#pragma unroll
        for (int e = 0; e < NB / ROWS; ++e) {
          const int row = tid / VECS + e * ROWS, col = z * NB + row;
          const int at = (row & ~31) + (row % 8 / 2) * 8 + row % 32 / 8 * 2 + row % 2;  // column c of product j: 8 j + c
          const bool ok = col < a.N && fleft > 0;
          cp16(bs + (buffer * NB + at) * ld + fv * 16, ok ? fp + (z * NB + e * ROWS) * a.ldb : a.B, ok ? fleft * 2 : 0);
        }
      };
      if (z0 < z1) fetch(z0, 0);
      cp_commit();
      if (!waited) pdl_wait();
      waited = true;
      const int blocks = (rows + 15) / 16, m16 = blocks * 16;
      const float scale = s.scale[lead];
      for (int i = tid; i < m16 * rv * 2; i += THREADS) {  // four ranks of a token
        const int row = i / (rv * 2), c = (i - row * rv * 2) * 4;
        alignas(16) float v[4] = {};
        if (row < rows) *reinterpret_cast<float4*>(v) = sum_h(a, split, static_cast<int64_t>(t0) + s.row[w][row], c, r);
        v[0] *= scale; v[1] *= scale; v[2] *= scale; v[3] *= scale;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
          const uint32_t x = pack_bf16x2(v[0], v[1]), y = pack_bf16x2(v[2], v[3]);
          *reinterpret_cast<uint2*>(parts + (p * a.rows + row) * ld + c * 2) = make_uint2(x, y);
          v[0] -= bf16_lo(x); v[1] -= bf16_hi(x); v[2] -= bf16_lo(y); v[3] -= bf16_hi(y);
        }
      }
      constexpr int LEAST = WARPS / 8;
      const int share = blocks > 4 ? LEAST : blocks > 2 ? 2 * LEAST : 4;  // warps that share a block's columns
      const int m0 = w / share * 16, first = w % share;
      const bool busy = m0 < rows;
      int64_t tok[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) tok[h] = m0 + g + h * 8 < rows ? t0 + s.row[w][m0 + g + h * 8] : -1;
      const uint16_t* rp[2] = {nullptr, nullptr};
      uint16_t* yp[2] = {nullptr, nullptr};
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (PLAIN && tok[h] >= 0) {
          rp[h] = a.res + tok[h] * a.ldr + q4 * 8;
          yp[h] = static_cast<uint16_t*>(a.Y) + tok[h] * a.ldy + q4 * 8;
        }
      if constexpr (!PLAIN) {
        if (lane < 16) {
          const bool on = m0 + lane < rows;
          const int64_t t = on ? t0 + s.row[w][m0 + lane] : 0;
          res_of[w][lane] = on && a.res ? a.res + t * a.ldr : nullptr;
          y_of[w][lane] = on ? static_cast<char*>(a.Y) + t * a.ldy * (a.f32 ? 4 : 2) : nullptr;
        }
        __syncwarp();
      }
      const uint32_t xa = hs + (m0 + (lane & 7) + (lane / 8 % 2) * 8) * ld + lane / 16 * 16;
      const uint32_t ba = bs + (lane / 16 * 8 + (lane & 7)) * ld + (lane / 8 % 2) * 16;
      // The residual is asked for ahead. In vectors: that of a slice's n-th 32 columns of this warp, once the slice before
      // has used its own. Else a column a lane, of 16 tokens, two times 32 columns ahead.
      const int count = 4 / share;  // times 32 columns of a slice that this warp has
      uint4 u[PLAIN ? 4 : 1][2];
      uint16_t one[PLAIN ? 1 : 2][16];
      auto ask = [&](int set, int n, int z) {  // `set` is known when this is compiled: an index of registers
        const int c = z * NB + (first + n * share) * 32;
        if constexpr (PLAIN) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            u[set][h] = make_uint4(0, 0, 0, 0);
            if (busy && z < z1 && n < count && rp[h] && c + q4 * 8 < a.N) u[set][h] = *reinterpret_cast<const uint4*>(rp[h] + c);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            one[set][e] = 0;
            const uint16_t* from = res_of[w][e];
            if (from && z < z1 && n < count && c + lane < a.N) one[set][e] = from[c + lane];
          }
        }
      };
#pragma unroll
      for (int n = 0; n < (PLAIN ? 4 : 2); ++n) ask(n, n, z0);
      // H's parts stay in registers where two CTAs an SM leave room for them
      constexpr bool HELD = !FEW && PARTS * RANKS <= 128;
      uint32_t x[HELD ? RANKS / 16 : 1][PARTS][4];
      auto load_h = [&](int k, uint32_t (&v)[PARTS][4]) {
#pragma unroll
        for (int p = 0; p < PARTS; ++p) ldm4(v[p], xa + p * a.rows * ld + k * 32);
      };
      if constexpr (HELD) {
        __syncthreads();  // H is written
        if (busy)
#pragma unroll
          for (int k = 0; k < RANKS / 16; ++k)
            if (2 * k < rv) load_h(k, x[k]);
      }
      int buffer = 0;
      for (int z = z0; z < z1; z += dz, buffer ^= 1) {
        if (z + dz < z1) fetch(z + dz, buffer ^ 1);
        cp_commit();
        cp_wait<1>();
        __syncthreads();
        if (busy)
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            const int col = (first + n * share) * 32, c = z * NB + col;
            if (n >= count || c >= a.N) continue;  // behind the last column no slice follows
            float acc[4][4] = {};
            if constexpr (PLAIN)  // results of 16 bits: the residual may be the sums' beginning
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const uint32_t x[4] = {u[n][h].x, u[n][h].y, u[n][h].z, u[n][h].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  acc[j][2 * h] = bf16_lo(x[j]);
                  acc[j][2 * h + 1] = bf16_hi(x[j]);
                }
              }
            if constexpr (PLAIN) ask(n, n, z + dz);
            const uint32_t bb = ba + (buffer * NB + col) * ld;
#pragma unroll
            for (int k = 0; k < RANKS / 16; ++k) {
              if (2 * k >= rv) break;
              uint32_t b[2][4];
#pragma unroll
              for (int j = 0; j < 2; ++j) ldm4(b[j], bb + j * 16 * ld + k * 32);  // products 2 j and 2 j + 1
              if constexpr (!HELD) load_h(k, x[0]);
#pragma unroll
              for (int p = 0; p < PARTS; ++p)
#pragma unroll
                for (int j = 0; j < 4; ++j) mma(acc[j], x[HELD ? k : 0][p], b[j / 2][j % 2 * 2], b[j / 2][j % 2 * 2 + 1]);
            }
            if (PLAIN) {
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                if (tok[h] < 0 || c + q4 * 8 >= a.N) continue;
                float v[8];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  v[2 * j] = acc[j][2 * h];
                  v[2 * j + 1] = acc[j][2 * h + 1];
                }
                *reinterpret_cast<uint4*>(yp[h] + c) = pack8(v);
              }
            } else {  // through shared memory: a column a lane, token after token
              __syncwarp();
#pragma unroll
              for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) turn[(g + e / 2 * 8) * 33 + q4 * 8 + j * 2 + e % 2] = acc[j][e];
              __syncwarp();
              if (c + lane < a.N)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                  if (char* y = y_of[w][e]) {
                    const float v = turn[e * 33 + lane] + bf16_lo(one[n & 1][e]);
                    if (PARTS == 3) reinterpret_cast<float*>(y)[c + lane] = v;
                    else reinterpret_cast<uint16_t*>(y)[c + lane] = static_cast<uint16_t>(pack_bf16x2(v, 0.0f));
                  }
              const bool here = n + 2 < count;
              ask(n & 1, here ? n + 2 : count >= 2 ? n + 2 - count : 0, here ? z : z + dz);
            }
          }
        __syncthreads();  // the buffer is free
      }
      cp_wait<0>();
      __syncthreads();
    }
  }
  if (!waited) pdl_wait();  // never done before the first kernel
}

// Into how many parts K may go: two CTAs an SM with the tiles (less where a tile turns out to have many adapters, see
// tile_split); four steps each at least. (4096 tokens on 8 adapters, K 4096, N 14336, R 64, both kernels:
// one CTA an SM 105 us, two 93.) By a GB300's SMs whatever the device has: workspaces and the most parts of a sum are
// the same on all. Grids go by the device's own.
constexpr int SPLIT_SMS = 152;
struct Plan {
  int tiles, split;
};
// n = 0: the most that any number of adapters asks for (what a workspace holds).
static Plan plan(int T, int K, int R, int n) {
  Plan p{};
  p.tiles = T / TILE + (T % TILE != 0);
  const int steps = (K + KB - 1) / KB;
  int want = 2 * SPLIT_SMS / p.tiles;
  if (n > 0) {
    const int tokens = T < TILE ? T : TILE, distinct = p.tiles > 4 ? 1 : tokens < n ? tokens : n;
    // A step costs a CTA about what one more partial sum of 128 tokens and 64 ranks costs each CTA of the second
    // kernel (0.35 us): no more parts than make the two equal.
    const long long even = static_cast<long long>(steps) * (TILE * 64) * distinct / (static_cast<long long>(tokens) * R);
    while (want > 4 && static_cast<long long>(want) * want > even) --want;
  }
  if (want < 4) want = 4;
  if (want > MAX_SPLIT) want = MAX_SPLIT;
  if (want > steps / 4) want = steps / 4;
  if (want < 1) want = 1;
  const int share = (steps + want - 1) / want;
  p.split = (steps + share - 1) / share;
  return p;
}

using Up = void (*)(const Args);
// The second kernel's forms: parts of H, ranks, few tokens an adapter, rows of residual and Y in 16-byte vectors.
template <class F>
static void each_up(F f) {
  f(adapters_up_kernel<2, 64, false, true>, 2, 64, false, true);
  f(adapters_up_kernel<2, 64, true, true>, 2, 64, true, true);
  f(adapters_up_kernel<2, MAX_R, false, true>, 2, MAX_R, false, true);
  f(adapters_up_kernel<2, MAX_R, true, true>, 2, MAX_R, true, true);
  f(adapters_up_kernel<2, 64, false, false>, 2, 64, false, false);
  f(adapters_up_kernel<2, 64, true, false>, 2, 64, true, false);
  f(adapters_up_kernel<2, MAX_R, false, false>, 2, MAX_R, false, false);
  f(adapters_up_kernel<2, MAX_R, true, false>, 2, MAX_R, true, false);
  f(adapters_up_kernel<3, 64, false, false>, 3, 64, false, false);
  f(adapters_up_kernel<3, 64, true, false>, 3, 64, true, false);
  f(adapters_up_kernel<3, MAX_R, false, false>, 3, MAX_R, false, false);
  f(adapters_up_kernel<3, MAX_R, true, false>, 3, MAX_R, true, false);
}

static int adapters_attr() {
  const auto most = cudaFuncAttributeMaxDynamicSharedMemorySize;
  cudaError_t e = cudaFuncSetAttribute(adapters_down_kernel, most, down_smem(TILE, MAX_R));
  each_up([&](auto kernel, int parts, int ranks, bool few, bool) {
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, most, up_smem(TILE, ranks, parts, few));
  });
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
  const ad::Plan p = ad::plan(T, K, R, 0);
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
  static PerDevice attr_;
  const int e = per_device(attr_, ad::adapters_attr);
  if (e != 0) return cuda_fail(static_cast<cudaError_t>(e), "cudaFuncSetAttribute(adapters)");
  const ad::Plan p = ad::plan(T, K, R, n);
  ad::Args a{};
  a.X = X; a.ldx = ldx; a.A = A; a.stride_a = stride_a; a.lda = lda; a.B = B; a.stride_b = stride_b; a.ldb = ldb;
  a.ids = ids; a.rank = rank; a.scale = scale; a.res = residual; a.ldr = ldr; a.Y = Y; a.ldy = ldy;
  a.n = n; a.R = R; a.T = T; a.N = N; a.K = K; a.f32 = f32 != 0; a.split = p.split;
  a.vec_r = ldr % 8 == 0 && r % 16 == 0;
  a.vec_y = ldy % (f32 ? 4 : 8) == 0 && y % 16 == 0;
  a.H = static_cast<float*>(workspace);
  a.rows = T < ad::TILE ? (T + 15) / 16 * 16 : ad::TILE;
  a.ranks = (R + 15) / 16 * 16;
  // As many CTAs as run at once. With few tiles they go to the adapters that a tile can have before its columns; with
  // many a CTA takes a tile's adapters in turn (one that finds no adapter costs 1.5 us of its SM).
  const int64_t tokens = T < ad::TILE ? T : ad::TILE, distinct = tokens < n ? tokens : n;
  const bool low = a.ranks <= 64;
  const int64_t sms = num_sms(), room = p.tiles < 2 * sms ? 2 * sms / p.tiles : 1;
  auto at_most = [](int64_t v, int64_t most) { return static_cast<unsigned>(v < 1 ? 1 : v < most ? v : most); };
  a.ctas = static_cast<int>(at_most(room, distinct * p.split));
  OM_LAUNCH_PDL("adapters_down_kernel", ad::adapters_down_kernel, dim3(p.tiles, a.ctas), dim3(ad::THREADS),
                static_cast<size_t>(ad::down_smem(a.rows, a.ranks)), stream, a);
  const int parts = f32 ? 3 : 2;
  // Few tokens an adapter: up to 16 in the mean of all adapters that a tile can have; in batches of many tiles, where an
  // adapter's tokens mostly follow one another, up to 8 (4096 tokens, N 14336, 8 adapters in runs of 512: 85 us by the
  // form for few, 79 by the other; 2072 tokens, N 9512, 25 adapters in runs of 7: 71 and 119)
  const bool few = tokens <= (p.tiles > 4 ? 8 : 16) * distinct;
  const int64_t ctas = (ad::up_pairs(parts, low ? 64 : ad::MAX_R) ? 2 : 1) * sms;
  const int64_t slices = (static_cast<int64_t>(N) + ad::NB - 1) / ad::NB, mine = ctas / p.tiles;
  // Slices of a CTA where the tiles share the CTAs evenly, and where all tiles' slices do: then most CTAs meet two tiles
  // and sum up H twice, which costs as much as 1.5 slices (32 tiles, N 14336, R 64, 304 CTAs: 13 slices 82 us, 11.8 90).
  const int64_t z = at_most(mine, slices), rounds = (p.tiles * z + ctas - 1) / ctas * ((slices + z - 1) / z);
  a.flat = !few && p.tiles > 4 && 2 * rounds * ctas > 2 * p.tiles * slices + 3 * ctas;
  const int64_t turns = (distinct + 1) * (few ? (slices + 1) / 2 : slices);  // few: a turn has two slices
  const dim3 grid = a.flat ? dim3(at_most(ctas, p.tiles * slices)) : dim3(p.tiles, at_most(mine, turns));
  const size_t smem = static_cast<size_t>(ad::up_smem(a.rows, low ? 64 : ad::MAX_R, parts, few));
  const bool plain = !f32 && residual && a.vec_r && a.vec_y && N % 8 == 0;
  ad::Up up = nullptr;
  ad::each_up([&](ad::Up kernel, int p_, int ranks_, bool few_, bool plain_) {
    if (p_ == parts && (ranks_ == 64) == low && few_ == few && plain_ == plain) up = kernel;
  });
  OM_LAUNCH_PDL("adapters_up_kernel", up, grid, dim3(ad::up_threads(parts, low ? 64 : ad::MAX_R, few)), smem, stream, a);
  return ORDERMOE_OK;
}
