// Attention of one new token a sequence over a paged cache.
//
// For a cached head with G query heads: x_i = scale <q, k_i>, out = sum_i exp(x_i - m) v_i / sum_i exp(x_i - m). Every byte
// of the cache is used G times, so HBM bounds it (2 G operations a byte; from about 100 the tensor cores would). The
// slots of all sequences and heads, cut into units of 16, form one list that is shared out evenly over the warps of a grid
// of one CTA an SM, by the lengths on the device; a warp runs through its part with a running maximum and sum and a ring of
// its own in shared memory, filled STAGES - 1 units ahead by 16-byte asynchronous copies (two for heads of
// 128 and 256, five for 64: 128 KB on their way an SM, 160 for 64). Rows that warps of one CTA share are joined there, rows
// that CTAs share by a second kernel, in the order of their slots.
// Measured (launched from the host, 32 / 8 heads of 128): one sequence of 131071 slots 88 us = 6.1 TB/s, 0.91 of the measured
// rate; 128 sequences of 1 to 8191 slots 334 us = 6.4 TB/s, 0.95; with a partial result a warp and one join for all of them
// 143 and 386. 17 sequences of up to 4097 slots, 16 heads of 128, weights kept: 65 us, floor 43 (attention 50, the two
// kernels behind it and their starts 15). Pages of fewer than 8 slots look a page up for every row.
#include "kvcache.cuh"

namespace om {

static __device__ unsigned long long g_err_attention = 0;

int read_clear_err_attention(unsigned long long* out) {
  unsigned long long zero = 0;
  OM_CUDA(cudaMemcpyFromSymbol(out, g_err_attention, sizeof(*out)));
  OM_CUDA(cudaMemcpyToSymbol(g_err_attention, &zero, sizeof(zero)));
  return ORDERMOE_OK;
}

namespace at {

constexpr int UNIT = 16;        // slots of a unit: the K of one m16n8k16 product with V
constexpr int MAX_CTAS = 192;   // workspaces hold partial results of so many
constexpr int MAX_WARPS = 8;

template <int D>
struct Shape {
  static constexpr int WARPS = D == 256 ? 4 : 8;
  static constexpr int STAGES = D == 64 ? 6 : 3;
  static constexpr int HALF = UNIT * D * 2;  // bytes of a unit's keys
  static constexpr int SMEM = WARPS * STAGES * 2 * HALF;
};

struct Args {
  CacheView c;
  int Hq, G, GC, chunks;  // query heads, per cached head, per row, rows per cached head
  const uint16_t* q; int64_t ldq;
  uint16_t* out; int64_t ldo;
  float* lse;
  float scale2;   // scale * log2(e)
  int ctas;
  int by_row;     // a CTA a row
  int row_units;  // units of a row of as many slots as the table reaches
  float* part;    // [CTAs][2]: maxima, sums and outputs of the rows that other CTAs share
  float* early;   // [CTAs][warps]: the same of a row that ended early in a warp's part
  float* stat;    // weights: [rows][GP][2] maximum and 1 / sum
  float* score;   // weights: [rows][row_units][GC][16]
};

// Rows of tables that reach few slots, where there are no more of them than CTAs, have one CTA each: no sums over the
// lengths and no second kernel (one sequence of 100 slots, 4 heads of 64: 5.0 us, by the list, as a table that reaches more
// has it, 8.6; 16 sequences of 300 slots, 32 / 8 heads of 128: 8.5 and 15.1).
constexpr int ROW_SLOTS = 512;

// Units before each of the block's groups of sequences. Thread i has the sequences [i * per, (i + 1) * per).
template <int NT>
struct Units {
  long long before[NT + 1];
  long long warp_sum[NT / 32];
};
__device__ __forceinline__ int units_of(const Args& a, int s) { return (a.c.slots(s) + UNIT - 1) / UNIT; }

template <int NT>
__device__ __forceinline__ int count_units(const Args& a, Units<NT>& u) {
  const int per = (a.c.seqs + NT - 1) / NT, tid = threadIdx.x, lane = tid % 32;
  long long mine = 0;
  for (int s = tid * per; s < a.c.seqs && s < (tid + 1) * per; ++s) mine += units_of(a, s);
  long long upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long x = __shfl_up_sync(~0u, upto, o);
    if (lane >= o) upto += x;
  }
  if (lane == 31) u.warp_sum[tid / 32] = upto;
  __syncthreads();
  long long base = 0;
  for (int i = 0; i < tid / 32; ++i) base += u.warp_sum[i];
  u.before[tid] = base + upto - mine;
  if (tid == NT - 1) u.before[NT] = base + upto;
  __syncthreads();
  return per;
}

// The list is cut into W parts, one a warp: part w has the units [w U / W, (w + 1) U / W). A CTA has the next
// WARPS parts, so that it can join what its own warps share.
__device__ __forceinline__ long long first_unit(long long U, int w, int W) { return U * w / W; }
__device__ __forceinline__ int owner(long long U, long long unit, int W) {
  return static_cast<int>(((unit + 1) * W - 1) / U);
}
// All warps of as many CTAs as have a unit for each, and no part is empty.
__device__ __forceinline__ int parts(long long U, int ctas, int warps) {
  const long long most = static_cast<long long>(ctas) * warps;
  return static_cast<int>(U < most ? U : most);
}

// A unit's place: sequence, row (cached head and chunk of its query heads) and unit of the row.
struct Place {
  int s, r, j, nu, n;
};
template <int NT>
__device__ __forceinline__ Place find_place(const Args& a, const Units<NT>& u, int per, long long unit, int rows) {
  const long long t = unit / rows;
  int lo = 0, hi = NT;  // before[lo] <= t < before[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (u.before[mid] <= t) lo = mid;
    else hi = mid;
  }
  Place p;
  long long b = u.before[lo];
  p.s = lo * per;
  while (b + units_of(a, p.s) <= t) b += units_of(a, p.s++);
  p.n = a.c.slots(p.s);
  p.nu = (p.n + UNIT - 1) / UNIT;
  const long long rest = unit - b * rows;
  p.r = static_cast<int>(rest / p.nu);
  p.j = static_cast<int>(rest % p.nu);
  return p;
}
// By a whole warp: sequences without slots are skipped 32 at a time.
__device__ __forceinline__ void next_place(const Args& a, Place& p, int rows) {
  if (++p.j < p.nu) return;
  p.j = 0;
  if (++p.r < rows) return;
  p.r = 0;
  for (++p.s; p.s < a.c.seqs; p.s += 32) {
    const int s = p.s + static_cast<int>(threadIdx.x % 32);
    const int n = s < a.c.seqs ? a.c.slots(s) : 0;
    const unsigned held = __ballot_sync(~0u, n > 0);
    if (held == 0) continue;
    const int first = __ffs(held) - 1;
    p.n = __shfl_sync(~0u, n, first);
    p.s += first;
    break;
  }
  p.nu = (p.n + UNIT - 1) / UNIT;
}

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
__device__ __forceinline__ void ldm4t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
               "{%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Loads a unit's keys and values, rows of D with their 16-byte vectors exchanged by the row's lowest three
// bits (no bank is met twice by a matrix load). Rows behind the length, and pages that do not exist, are zeros.
template <int D>
__device__ __forceinline__ void load_unit(const Args& a, const Place& p, const int32_t (&page)[2], uint32_t stage) {
  constexpr int VECS = D / 8, HALF = Shape<D>::HALF, N = UNIT * VECS / 32;
  const int lane = threadIdx.x % 32, head = p.r / a.chunks, base = p.j * UNIT, left = p.n - base;
  if (a.c.page_log >= 4) {  // a unit lies in one page, row after row
    const bool good = a.c.good(page[0]);
    if (!good && lane == 0) report(&g_err_attention, ORDERMOE_DEV_BAD_INDEX, p.s);
    const int64_t at = good ? a.c.row(page[0], head, base) * D + lane * 8 : 0;
    const int end = good ? left : 0;
    const uint16_t *k = a.c.k + at, *v = a.c.v + at;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int x = i * 32 + lane, row = x / VECS, vec = x % VECS;
      const uint32_t dst = stage + (row * VECS + (vec ^ (row & 7))) * 16;
      const bool ok = row < end;
      cp16(dst, ok ? k + i * 256 : a.c.k, ok ? 16 : 0);
      cp16(dst + HALF, ok ? v + i * 256 : a.c.v, ok ? 16 : 0);
    }
    return;
  }
  if (a.c.page_log == 3) {  // in two
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int slot = base + 8 * h;
      const bool in = slot < p.n, good = in && a.c.good(page[h]);
      if (in && !good && lane == 0) report(&g_err_attention, ORDERMOE_DEV_BAD_INDEX, p.s);
      const int64_t at = good ? a.c.row(page[h], head, slot) * D + lane * 8 : 0;
      const int end = good ? left - 8 * h : 0;
      const uint16_t *k = a.c.k + at, *v = a.c.v + at;
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        const int x = i * 32 + lane, row = x / VECS, vec = x % VECS;
        const uint32_t dst = stage + ((row + 8 * h) * VECS + (vec ^ (row & 7))) * 16;
        const bool ok = row < end;
        cp16(dst, ok ? k + i * 256 : a.c.k, ok ? 16 : 0);
        cp16(dst + HALF, ok ? v + i * 256 : a.c.v, ok ? 16 : 0);
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int x = i * 32 + lane, row = x / VECS, vec = x % VECS, slot = base + row;
    const bool in = row < left;
    const int32_t pg = in ? a.c.page_of(p.s, slot) : 0;
    const bool ok = in && a.c.good(pg);
    if (in && !ok && vec == 0) report(&g_err_attention, ORDERMOE_DEV_BAD_INDEX, p.s);
    const int64_t at = ok ? a.c.row(pg, head, slot) * D + vec * 8 : 0;
    const uint32_t dst = stage + (row * VECS + (vec ^ (row & 7))) * 16;
    cp16(dst, a.c.k + at, ok ? 16 : 0);
    cp16(dst + HALF, a.c.v + at, ok ? 16 : 0);
  }
}

// A row: one cached head of a sequence and up to GP of its query heads, `first` and on.
struct Row {
  int s, r, head, first, heads;
};
__device__ __forceinline__ Row row_of(const Args& a, int s, int r) {
  Row x{s, r, r / a.chunks, (r % a.chunks) * a.GC, 0};
  x.heads = min(a.GC, a.G - x.first);
  return x;
}
__device__ __forceinline__ uint16_t* out_of(const Args& a, const Row& x, int y, int D) {
  return a.out + x.s * a.ldo + (static_cast<int64_t>(x.head) * a.G + x.first + y) * D;
}
__device__ __forceinline__ float inverse(float sum) { return sum == 0.0f ? 0.0f : 1.0f / sum; }
// Two outputs. Where nothing is attended they are 0, whatever the sums of p v became (0 times an infinity).
__device__ __forceinline__ uint32_t output2(float x, float y, float inv) {
  return inv == 0.0f ? 0u : pack_bf16x2(x * inv, y * inv);
}
// lse, and what the weights are computed from, of head y.
template <int GP, bool WEIGHTS>
__device__ __forceinline__ void put_sums(const Args& a, const Row& x, int y, float m, float sum, float inv, int rows) {
  if (a.lse)
    a.lse[static_cast<int64_t>(x.s) * a.Hq + x.head * a.G + x.first + y] =
        sum == 0.0f ? -INFINITY : (m + log2f(sum)) * 0.69314718055994531f;
  if constexpr (WEIGHTS)
    *reinterpret_cast<float2*>(a.stat + ((static_cast<int64_t>(x.s) * rows + x.r) * GP + y) * 2) = make_float2(m, inv);
}

// GP = 8 NG rows of the 16-row product hold query heads. With eight, the other eight rows carry the second bf16 part of
// p in the product with V; with sixteen a second product does. (One part, 8 bits, would add as much to out's error as its
// own rounding. With two, out is as far from 64 bits as with p in fp32, 1.6e-3 in the 2-norm for 131071 slots, and two in
// a thousand of its values are one step of bf16 from the nearest one; with fp32 two in ten thousand.) mma.sync is enough: a row has 1 to 16 queries, and 16 slots cost 32 products, a fifth of the time that
// their 8 KB take.
template <int D, int NG, bool WEIGHTS>
__global__ void __launch_bounds__(Shape<D>::WARPS * 32, 1) attend_kernel(const Args a) {
  constexpr int WARPS = Shape<D>::WARPS, NT = WARPS * 32, STAGES = Shape<D>::STAGES, HALF = Shape<D>::HALF;
  constexpr int GP = 8 * NG, PS = GP * (D + 2), KS = D / 16, VECS = D / 8;
  static_assert(WARPS * PS * 4 <= Shape<D>::SMEM, "a row's partial results a warp fit in the ring");
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ Units<NT> units;
  // The row that a warp's part begins inside of ([0]; where its results are, and whether it ends in the part), and the
  // one that begins in the part and goes on behind it ([1]). Sequence, -1: none.
  __shared__ int cut_s[WARPS][2], cut_r[WARPS][2], cut_ends[WARPS];
  __shared__ const float* cut_at[WARPS][2];
  pdl_wait();
  pdl_trigger();
  const int per = a.by_row ? 0 : count_units(a, units);
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, g = lane / 4, q4 = lane % 4;
  const int rows = a.c.heads * a.chunks;
  for (int s0 = (blockIdx.x * WARPS + warp) * 32; s0 < a.c.seqs; s0 += gridDim.x * NT) {  // bad lengths, and none
    const int mine = s0 + lane, n = mine < a.c.seqs ? a.c.slots(mine) : 1;
    if (mine < a.c.seqs && n != a.c.length[mine]) report(&g_err_attention, ORDERMOE_DEV_BAD_INDEX, mine);
    for (unsigned none = __ballot_sync(~0u, n == 0); none != 0; none &= none - 1) {
      const int s = s0 + __ffs(none) - 1;
      for (int i = lane; i < a.Hq * VECS; i += 32) reinterpret_cast<uint4*>(a.out + s * a.ldo)[i] = make_uint4(0, 0, 0, 0);
      if (a.lse)
        for (int i = lane; i < a.Hq; i += 32) a.lse[static_cast<int64_t>(s) * a.Hq + i] = -INFINITY;
    }
  }
  // all units, or those of this CTA's row
  const long long U = a.by_row ? units_of(a, blockIdx.x / rows) : units.before[NT] * rows;
  const int W = parts(U, a.by_row ? 1 : a.ctas, WARPS), w0 = a.by_row ? 0 : blockIdx.x * WARPS, w = w0 + warp;
  if (w0 >= W) return;
  const long long u0 = w < W ? first_unit(U, w, W) : 0;
  const int count = w < W ? static_cast<int>(first_unit(U, w + 1, W) - u0) : 0;
  if (lane < 2) cut_s[warp][lane] = -1;
  Place p{};
  int32_t page[2] = {0, 0};  // of the two halves of the unit that is loaded next
  auto find_pages = [&](const Place& at) {
    const int slot = at.j * UNIT;
    page[0] = a.c.page_of(at.s, slot);
    if (a.c.page_log == 3 && slot + 8 < at.n) page[1] = a.c.page_of(at.s, slot + 8);
  };
  if (count > 0) {
    if (a.by_row) {
      p.s = blockIdx.x / rows;
      p.r = blockIdx.x % rows;
      p.j = static_cast<int>(u0);
      p.nu = static_cast<int>(U);
      p.n = a.c.slots(p.s);
    } else {
      p = find_place(a, units, per, u0, rows);
    }
    find_pages(p);
  }
  const uint32_t mine = smem_u32(ring) + warp * STAGES * 2 * HALF;
  Place f = p;  // what is loaded next, and its stage
  int fetched = 0, fstage = 0;
  auto fetch = [&]() {
    if (fetched < count) {
      load_unit<D>(a, f, page, mine + fstage * 2 * HALF);
      fstage = fstage + 1 == STAGES ? 0 : fstage + 1;
      if (++fetched < count) {
        next_place(a, f, rows);
        find_pages(f);
      }
    }
    cp_commit();
  };
#pragma unroll
  for (int i = 0; i < STAGES - 1; ++i) fetch();

  uint32_t qa[KS][NG == 1 ? 2 : 4];
  float o[VECS][4], m[2], l[2];
  int j0 = 0, stage = 0;
  bool fresh = true;
  auto load_q = [&](const Row& x) {
    const uint16_t* q = a.q + x.s * a.ldq + (static_cast<int64_t>(x.head) * a.G + x.first) * D + q4 * 2;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int i = 0; i < NG; ++i) {
        const bool on = g + 8 * i < x.heads;
        const uint16_t* v = q + static_cast<int64_t>(on ? g + 8 * i : 0) * D + k * 16;
        const uint32_t lo = *reinterpret_cast<const uint32_t*>(v), hi = *reinterpret_cast<const uint32_t*>(v + 8);
        qa[k][i] = on ? lo : 0u;
        qa[k][NG + i] = on ? hi : 0u;
      }
  };
  // a head's sum over the lanes, and two of its outputs
  auto total = [&](int i) {
    const float s = l[i] + __shfl_xor_sync(~0u, l[i], 1);
    return s + __shfl_xor_sync(~0u, s, 2);
  };
  auto pair = [&](int n, int i) {
    return NG == 1 ? make_float2(o[n][0] + o[n][2], o[n][1] + o[n][3]) : make_float2(o[n][2 * i], o[n][2 * i + 1]);
  };
  auto park = [&](float* part) {  // maxima, sums and outputs of the row in hand
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const float sum = total(i);
      const int y = g + 8 * i;
      if (q4 == 0) {
        part[y] = m[i];
        part[GP + y] = sum;
      }
#pragma unroll
      for (int n = 0; n < VECS; ++n) *reinterpret_cast<float2*>(part + 2 * GP + y * D + n * 8 + q4 * 2) = pair(n, i);
    }
  };
  int open = -1;  // which of the cut rows is in the registers at the part's end
  for (int u = 0; u < count; ++u) {
    if (fresh) {  // a row begins in this part
      fresh = false;
      j0 = p.j;
      load_q(row_of(a, p.s, p.r));
#pragma unroll
      for (int n = 0; n < VECS; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.0f;
      m[0] = m[1] = -INFINITY;
      l[0] = l[1] = 0.0f;
    }
    cp_wait<STAGES - 2>();
    __syncwarp();
    fetch();  // into the stage that was read a unit ago
    const uint32_t kb = mine + stage * 2 * HALF, vb = kb + HALF;
    stage = stage + 1 == STAGES ? 0 : stage + 1;
    float x[2][4] = {};
    {
      const int row = (lane & 7) + (lane >= 16 ? 8 : 0), half = lane / 8 % 2;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        uint32_t b[4];
        ldm4(b, kb + (row * VECS + ((2 * k + half) ^ (row & 7))) * 16);
        if constexpr (NG == 1) {
          mma(x[0], qa[k][0], 0u, qa[k][1], 0u, b[0], b[1]);
          mma(x[1], qa[k][0], 0u, qa[k][1], 0u, b[2], b[3]);
        } else {
          mma(x[0], qa[k][0], qa[k][1], qa[k][2], qa[k][3], b[0], b[1]);
          mma(x[1], qa[k][0], qa[k][1], qa[k][2], qa[k][3], b[2], b[3]);
        }
      }
    }
    const int left = p.n - p.j * UNIT;  // slots from here to the length
    uint32_t hi[2][2], lo[2][2];  // p's parts: [slots 0-7, 8-15][heads g, g + 8]
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      float* y[2] = {&x[0][2 * i], &x[1][2 * i]};
      float top = -INFINITY;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          y[t][e] = t * 8 + q4 * 2 + e < left ? __fmul_rn(y[t][e], a.scale2) : -INFINITY;
          top = fmaxf(top, y[t][e]);
        }
      if constexpr (WEIGHTS) {
        if (g + 8 * i < a.GC) {
          float* sc = a.score + (((static_cast<int64_t>(p.s) * rows + p.r) * a.row_units + p.j) * a.GC + g + 8 * i) * UNIT + q4 * 2;
          *reinterpret_cast<float2*>(sc) = make_float2(y[0][0], y[0][1]);
          *reinterpret_cast<float2*>(sc + 8) = make_float2(y[1][0], y[1][1]);
        }
      }
      top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
      top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
      top = fmaxf(top, m[i]);
      const float ref = top == -INFINITY ? 0.0f : top;
      const float shrink = exp2f(m[i] - ref);
      m[i] = top;
      l[i] *= shrink;
      if (__any_sync(~0u, shrink != 1.0f)) {
#pragma unroll
        for (int n = 0; n < VECS; ++n) {
          o[n][2 * i] *= shrink;
          o[n][2 * i + 1] *= shrink;
          if constexpr (NG == 1) {
            o[n][2] *= shrink;
            o[n][3] *= shrink;
          }
        }
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const float e0 = exp2f(y[t][0] - ref), e1 = exp2f(y[t][1] - ref);
        l[i] += e0 + e1;
        hi[t][i] = pack_bf16x2(e0, e1);
        lo[t][i] = pack_bf16x2(e0 - bf16_lo(hi[t][i]), e1 - bf16_hi(hi[t][i]));
      }
    }
    {
      const int row = (lane & 7) + (lane / 8 % 2) * 8, next = lane / 16;
#pragma unroll
      for (int n = 0; n < VECS; n += 2) {
        uint32_t b[4];
        ldm4t(b, vb + (row * VECS + ((n + next) ^ (row & 7))) * 16);
        if constexpr (NG == 1) {
          mma(o[n], hi[0][0], lo[0][0], hi[1][0], lo[1][0], b[0], b[1]);
          mma(o[n + 1], hi[0][0], lo[0][0], hi[1][0], lo[1][0], b[2], b[3]);
        } else {
          mma(o[n], hi[0][0], hi[0][1], hi[1][0], hi[1][1], b[0], b[1]);
          mma(o[n + 1], hi[0][0], hi[0][1], hi[1][0], hi[1][1], b[2], b[3]);
          mma(o[n], lo[0][0], lo[0][1], lo[1][0], lo[1][1], b[0], b[1]);
          mma(o[n + 1], lo[0][0], lo[0][1], lo[1][0], lo[1][1], b[2], b[3]);
        }
      }
    }
    const bool ends = p.j + 1 == p.nu, last = u + 1 == count;
    if (ends || last) {  // the row ends, or the part
      fresh = true;
      if (ends && j0 == 0) {  // all of the row was here
        const Row x = row_of(a, p.s, p.r);
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          const float sum = total(i), inv = inverse(sum);
          const int y = g + 8 * i;
          if (y >= x.heads) continue;
          if (q4 == 0) put_sums<GP, WEIGHTS>(a, x, y, m[i], sum, inv, rows);
          uint16_t* out = out_of(a, x, y, D) + q4 * 2;
#pragma unroll
          for (int n = 0; n < VECS; ++n) {
            const float2 v = pair(n, i);
            *reinterpret_cast<uint32_t*>(out + n * 8) = output2(v.x, v.y, inv);
          }
        }
      } else {
        const int which = j0 == 0;
        float* at = last ? reinterpret_cast<float*>(ring) + warp * PS : a.early + static_cast<int64_t>(w) * PS;
        if (last) open = which;
        else park(at);  // the ring is in use
        if (lane == 0) {
          cut_s[warp][which] = p.s;
          cut_r[warp][which] = p.r;
          cut_at[warp][which] = at;
          if (which == 0) cut_ends[warp] = ends;
        }
      }
    }
    if (!last) next_place(a, p, rows);
  }
  cp_wait<0>();
  __syncthreads();  // the ring is free
  if (open >= 0) park(reinterpret_cast<float*>(ring) + warp * PS);
  __syncthreads();
  // Chains of parts that share a row: the one that reaches into this CTA from the one before, and those that begin in
  // it. Each is joined by all threads, four outputs of a head each, part after part.
  for (int c = -1; c < WARPS; ++c) {
    const int b = c < 0 ? 0 : c, side = c < 0 ? 0 : 1;
    if (cut_s[b][side] < 0) continue;
    const Row x = row_of(a, cut_s[b][side], cut_r[b][side]);
    int end = b + 1;  // parts [b, end) of this CTA, and whether the row ends with the last
    bool done = side == 0 && cut_ends[0];
    while (!done && end < WARPS && w0 + end < W) done = cut_ends[end++];
    const bool whole = side == 1 && done;
    float* part = a.part + (static_cast<int64_t>(blockIdx.x) * 2 + side) * PS;
    for (int i = threadIdx.x; i < x.heads * (D / 4); i += NT) {
      const int y = i / (D / 4), d = i % (D / 4) * 4;
      float top = -INFINITY, sum = 0.0f;
      for (int k = b; k < end; ++k) top = fmaxf(top, cut_at[k][k == b ? side : 0][y]);
      const float ref = top == -INFINITY ? 0.0f : top;
      float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      for (int k = b; k < end; ++k) {
        const float* from = cut_at[k][k == b ? side : 0];
        const float z = exp2f(from[y] - ref);
        const float4 e = *reinterpret_cast<const float4*>(from + 2 * GP + y * D + d);
        sum += z * from[GP + y];
        v.x += z * e.x; v.y += z * e.y; v.z += z * e.z; v.w += z * e.w;
      }
      if (whole) {
        const float inv = inverse(sum);
        if (d == 0) put_sums<GP, WEIGHTS>(a, x, y, top, sum, inv, rows);
        *reinterpret_cast<uint2*>(out_of(a, x, y, D) + d) =
            make_uint2(output2(v.x, v.y, inv), output2(v.z, v.w, inv));
      } else {
        if (d == 0) {
          part[y] = top;
          part[GP + y] = sum;
        }
        *reinterpret_cast<float4*>(part + 2 * GP + y * D + d) = v;
      }
    }
  }
}

// Joins the rows that CTAs share. CTA (b, y) has head y of the row in which CTA b's units end, if the row began there:
// its threads are D / 4 columns of four outputs, and groups that share the partial results, in order.
constexpr int JOIN_THREADS = 256;
template <int D, int GP, bool WEIGHTS>
__global__ void __launch_bounds__(JOIN_THREADS) attend_join_kernel(const Args a) {
  constexpr int PS = GP * (D + 2), WARPS = Shape<D>::WARPS, COLS = D / 4, GROUPS = JOIN_THREADS / COLS;
  __shared__ Units<JOIN_THREADS> units;
  __shared__ float tops[MAX_CTAS], lens[MAX_CTAS];
  __shared__ float4 sums[GROUPS][COLS];
  // lengths are the call's inputs: the row is looked for while the first kernel ends
  const int per = count_units(a, units), rows = a.c.heads * a.chunks, tid = threadIdx.x, y = blockIdx.y;
  const long long U = units.before[JOIN_THREADS] * rows;
  const int W = parts(U, a.ctas, WARPS), next = (static_cast<int>(blockIdx.x) + 1) * WARPS;
  Place p{};
  Row x{};
  int c0 = -1, c1 = -1;
  if (next < W) {
    const long long at = first_unit(U, next, W);
    p = find_place(a, units, per, at, rows);
    x = row_of(a, p.s, p.r);
    c0 = owner(U, at - p.j, W) / WARPS;
    c1 = owner(U, at - p.j + p.nu - 1, W) / WARPS;
  }
  pdl_wait();
  pdl_trigger();
  if (next >= W || p.j == 0 || c0 != static_cast<int>(blockIdx.x) || y >= x.heads) return;
  auto part = [&](int c) { return a.part + (static_cast<int64_t>(c) * 2 + (c == c0)) * PS; };
  const int n = c1 - c0 + 1;
  for (int i = tid; i < n; i += JOIN_THREADS) {
    tops[i] = part(c0 + i)[y];
    lens[i] = part(c0 + i)[GP + y];
  }
  __syncthreads();
  float top = -INFINITY, sum = 0.0f;
  for (int i = 0; i < n; ++i) top = fmaxf(top, tops[i]);
  const float ref = top == -INFINITY ? 0.0f : top;
  const int col = tid % COLS, group = tid / COLS;
  float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
  for (int i = group; i < n; i += GROUPS) {
    const float z = exp2f(tops[i] - ref);
    const float4 e = *reinterpret_cast<const float4*>(part(c0 + i) + 2 * GP + y * D + col * 4);
    v.x += z * e.x; v.y += z * e.y; v.z += z * e.z; v.w += z * e.w;
  }
  sums[group][col] = v;
  __syncthreads();
  if (tid >= COLS) return;
  for (int i = 0; i < n; ++i) sum += lens[i] * exp2f(tops[i] - ref);
  for (int i = 1; i < GROUPS; ++i) {
    const float4 e = sums[i][col];
    v.x += e.x; v.y += e.y; v.z += e.z; v.w += e.w;
  }
  const float inv = inverse(sum);
  if (tid == 0) put_sums<GP, WEIGHTS>(a, x, y, top, sum, inv, rows);
  *reinterpret_cast<uint2*>(out_of(a, x, y, D) + col * 4) =
      make_uint2(output2(v.x, v.y, inv), output2(v.z, v.w, inv));
}

// mass[s][h][i] += the sum of p_i over the query heads of head h, from the scores that were kept.
constexpr int MASS_THREADS = 128;
template <int GP>
__global__ void __launch_bounds__(MASS_THREADS) attend_mass_kernel(const Args a) {
  pdl_wait();
  pdl_trigger();
  const int rows = a.c.heads * a.chunks, s = blockIdx.x / a.c.heads, h = blockIdx.x % a.c.heads, n = a.c.slots(s);
  float* mass = a.c.mass + a.c.side(s, h, 0);
  for (int i = blockIdx.y * MASS_THREADS + threadIdx.x; i < n; i += gridDim.y * MASS_THREADS) {
    float sum = 0.0f;
    for (int c = 0; c < a.chunks; ++c) {
      const int heads = min(a.GC, a.G - c * a.GC);
      const int64_t row = static_cast<int64_t>(s) * rows + h * a.chunks + c;
      const float* sc = a.score + (row * a.row_units + i / UNIT) * a.GC * UNIT + i % UNIT;
      const float* st = a.stat + row * GP * 2;
#pragma unroll 4
      for (int y = 0; y < heads; ++y) {
        const float inv = st[2 * y + 1];
        sum += inv == 0.0f ? 0.0f : exp2f(sc[y * UNIT] - st[2 * y]) * inv;
      }
    }
    mass[i] += sum;
  }
}

// What a call's sizes decide: query heads of a row (8 or 16), rows a cached head, and the workspace.
struct Layout {
  int GP, GC, chunks;
  size_t part, early, stat, score;  // bytes
};
static Layout layout(int seqs, int G, int heads, int dim, int64_t seq_slots, bool weights) {
  Layout l{};
  // Sixteen heads a row halve the passes over the cache of wide groups; heads of 256 have no registers for them.
  l.GP = G > 8 && dim <= 128 ? 16 : 8;
  l.GC = G < l.GP ? G : l.GP;
  l.chunks = (G + l.GC - 1) / l.GC;
  auto up = [](size_t v) { return (v + 255) / 256 * 256; };
  const size_t partial = static_cast<size_t>(l.GP) * (dim + 2) * 4;
  l.part = up(MAX_CTAS * 2 * partial);
  l.early = up(MAX_CTAS * MAX_WARPS * partial);
  if (weights) {
    const size_t rows = static_cast<size_t>(seqs) * heads * l.chunks;
    l.stat = up(rows * l.GP * 8);
    l.score = up(rows * ((static_cast<size_t>(seq_slots) + UNIT - 1) / UNIT) * UNIT * l.GC * 4);
  }
  return l;
}

template <int D, int NG, bool WEIGHTS>
static int attend_attr() {
  return static_cast<int>(cudaFuncSetAttribute(attend_kernel<D, NG, WEIGHTS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               Shape<D>::SMEM));
}

template <int D, int NG, bool WEIGHTS>
static int launch(Args& a, cudaStream_t stream) {
  static PerDevice attr_;
  const int e = per_device(attr_, attend_attr<D, NG, WEIGHTS>);
  if (e != 0) return cuda_fail(static_cast<cudaError_t>(e), "cudaFuncSetAttribute(attend)");
  const int sms = num_sms();
  a.ctas = sms < MAX_CTAS ? sms : MAX_CTAS;
  const int64_t rows = static_cast<int64_t>(a.c.seqs) * a.c.heads;
  const int64_t units = rows * a.chunks * ((static_cast<int64_t>(a.c.cap) + UNIT - 1) / UNIT);
  const int64_t most = (units + Shape<D>::WARPS - 1) / Shape<D>::WARPS;  // CTAs that can have work
  if (units / a.ctas > INT32_MAX) return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "attention_paged: the table reaches too many slots");
  a.row_units = (a.c.cap + UNIT - 1) / UNIT;
  a.by_row = a.c.cap <= ROW_SLOTS && rows * a.chunks <= a.ctas;
  const int grid = a.by_row ? static_cast<int>(rows * a.chunks) : most < a.ctas ? static_cast<int>(most) : a.ctas;
  OM_LAUNCH_PDL("attend_kernel", attend_kernel<D, NG, WEIGHTS>, dim3(grid), dim3(Shape<D>::WARPS * 32),
                static_cast<size_t>(Shape<D>::SMEM), stream, a);
  if (grid > 1 && !a.by_row)
    OM_LAUNCH_PDL("attend_join_kernel", attend_join_kernel<D, 8 * NG, WEIGHTS>, dim3(grid - 1, a.GC), dim3(JOIN_THREADS), 0,
                  stream, a);
  if (WEIGHTS) {
    const int64_t fill = 16ll * sms / rows + 1, need = (a.c.cap + MASS_THREADS - 1) / MASS_THREADS;
    OM_LAUNCH_PDL("attend_mass_kernel", attend_mass_kernel<8 * NG>,
                  dim3(static_cast<unsigned>(rows), static_cast<unsigned>(fill < need ? fill : need)), dim3(MASS_THREADS), 0,
                  stream, a);
  }
  return ORDERMOE_OK;
}
template <int D, int NG>
static int launch(Args& a, bool weights, cudaStream_t stream) {
  return weights ? launch<D, NG, true>(a, stream) : launch<D, NG, false>(a, stream);
}

}  // namespace at
}  // namespace om

using namespace om;

extern "C" size_t ordermoe_attention_paged_workspace_bytes(int seqs, int q_heads, int heads, int dim, int64_t seq_slots,
                                                           int weights) {
  if (seqs < 0 || heads <= 0 || q_heads <= 0 || q_heads % heads != 0 || seq_slots <= 0 || seq_slots > (1 << 30) ||
      (dim != 64 && dim != 128 && dim != 256))
    return 0;
  const at::Layout l = at::layout(seqs, q_heads / heads, heads, dim, seq_slots, weights != 0);
  return l.part + l.early + l.stat + l.score;
}

extern "C" int ordermoe_attention_paged(const ordermoe_cache* cache, const uint16_t* q, int64_t ldq, int q_heads,
                                        float scale, uint16_t* out, int64_t ldo, float* lse, int weights,
                                        void* workspace, size_t workspace_bytes, ordermoe_stream_t stream) {
  OM_TRACE();
  const int rc = check_cache(cache, "attention_paged");
  if (rc) return rc;
  if (q_heads <= 0 || q_heads % cache->heads != 0 || q_heads > 4096)
    return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "attention_paged: need query heads that are a multiple of the cache's, at most 4096");
  if (!(scale > 0.0f) || scale > 1e30f) return fail(ORDERMOE_ERR_INVALID_ARG, "attention_paged: need a scale > 0");
  if (cache->seqs == 0) return ORDERMOE_OK;
  if (!q || !out || (weights && !cache->mass))
    return fail(ORDERMOE_ERR_INVALID_ARG, "attention_paged: null pointer (q, out, or a mass for the weights)");
  const int64_t width = static_cast<int64_t>(q_heads) * cache->dim;
  const bool many = cache->seqs > 1;
  if (!aligned16(q) || !aligned16(out) || reinterpret_cast<uintptr_t>(lse) % 4 != 0)
    return fail(ORDERMOE_ERR_INVALID_ARG, "attention_paged: q and out must be 16-byte aligned, lse to its type");
  if (many && (ldq < width || ldo < width || ldq % 8 != 0 || ldo % 8 != 0 || ldq >= (1ll << 38) || ldo >= (1ll << 38)))
    return fail(ORDERMOE_ERR_INVALID_ARG, "attention_paged: ldq and ldo must be multiples of 8, not shorter than a row");
  if (q == out && many && ldq != ldo)
    return fail(ORDERMOE_ERR_INVALID_ARG, "attention_paged: an out that is q must have its stride");
  const int64_t cap = static_cast<int64_t>(cache->seq_pages) * cache->page;
  const at::Layout l = at::layout(cache->seqs, q_heads / cache->heads, cache->heads, cache->dim, cap, weights != 0);
  if (static_cast<int64_t>(cache->seqs) * cache->heads * l.chunks > INT32_MAX / 32)
    return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "attention_paged: need fewer sequences times heads");
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 != 0 || workspace_bytes < l.part + l.early + l.stat + l.score)
    return fail(ORDERMOE_ERR_INVALID_ARG, "attention_paged: workspace is null, too small or not 256-byte aligned");
  at::Args a{};
  a.c = cache_view(cache);
  a.Hq = q_heads; a.G = q_heads / cache->heads; a.GC = l.GC; a.chunks = l.chunks;
  a.q = q; a.ldq = ldq; a.out = out; a.ldo = ldo; a.lse = lse;
  a.scale2 = scale * 1.4426950408889634f;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  a.part = reinterpret_cast<float*>(ws);
  a.early = reinterpret_cast<float*>(ws + l.part);
  a.stat = reinterpret_cast<float*>(ws + l.part + l.early);
  a.score = reinterpret_cast<float*>(ws + l.part + l.early + l.stat);
  const bool wt = weights != 0;
  if (cache->dim == 64) return l.GP == 8 ? at::launch<64, 1>(a, wt, stream) : at::launch<64, 2>(a, wt, stream);
  if (cache->dim == 128) return l.GP == 8 ? at::launch<128, 1>(a, wt, stream) : at::launch<128, 2>(a, wt, stream);
  return at::launch<256, 1>(a, wt, stream);
}
