// The paged cache of keys and values of one layer: appending new tokens with rotary positions, and
// cutting a sequence to a budget of slots by what its tokens were attended.
#include "kvcache.cuh"

namespace om {

static __device__ unsigned long long g_err_cache = 0;

int read_clear_err_cache(unsigned long long* out) {
  unsigned long long zero = 0;
  OM_CUDA(cudaMemcpyFromSymbol(out, g_err_cache, sizeof(*out)));
  OM_CUDA(cudaMemcpyToSymbol(g_err_cache, &zero, sizeof(zero)));
  return ORDERMOE_OK;
}

int check_cache(const ordermoe_cache* c, const char* what) {
  if (!c) return fail(ORDERMOE_ERR_INVALID_ARG, "%s: null cache", what);
  if (c->seqs < 0 || c->pages < 0 || c->seq_pages <= 0 || c->ld_table < c->seq_pages)
    return fail(ORDERMOE_ERR_INVALID_ARG, "%s: need seqs >= 0, pages >= 0 and 0 < seq_pages <= ld_table", what);
  if (c->dim != 64 && c->dim != 128 && c->dim != 256)
    return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "%s: need heads of 64, 128 or 256", what);
  if (c->page <= 0 || c->page > kCacheMaxPage || (c->page & (c->page - 1)) != 0)
    return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "%s: a page must hold a power of two of slots, at most %d", what,
                kCacheMaxPage);
  if (c->heads <= 0 || c->heads > 1024 || c->seqs > 65535)
    return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "%s: need 1 to 1024 heads and at most 65535 sequences", what);
  if (c->pages > INT32_MAX || static_cast<int64_t>(c->seq_pages) * c->page > (1 << 30))
    return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "%s: need at most 2^31 - 1 pages and 2^30 slots a sequence", what);
  if (c->seqs == 0) return ORDERMOE_OK;
  if (!c->k || !c->v || !c->table || !c->length) return fail(ORDERMOE_ERR_INVALID_ARG, "%s: null pointer in the cache", what);
  if (!aligned16(c->k) || !aligned16(c->v))
    return fail(ORDERMOE_ERR_INVALID_ARG, "%s: the cache's pages must be 16-byte aligned", what);
  const uintptr_t a = reinterpret_cast<uintptr_t>(c->table) | reinterpret_cast<uintptr_t>(c->length) |
                      reinterpret_cast<uintptr_t>(c->mass) | reinterpret_cast<uintptr_t>(c->pos);
  if (a % 4 != 0) return fail(ORDERMOE_ERR_INVALID_ARG, "%s: table, length, mass or pos is not aligned to its type", what);
  return ORDERMOE_OK;
}

CacheView cache_view(const ordermoe_cache* c) {
  CacheView v{};
  v.k = c->k; v.v = c->v;
  v.pages = c->pages;
  while ((1 << v.page_log) < c->page) ++v.page_log;
  v.heads = c->heads; v.seqs = c->seqs; v.cap = c->seq_pages * c->page;
  v.table = c->table; v.ld_table = c->ld_table; v.length = c->length;
  v.mass = c->mass; v.pos = c->pos;
  return v;
}

namespace kv {

// ------------------------------------------------------------------------- append
constexpr int APPEND_THREADS = 128;
constexpr int MAX_DIM = 256;

struct AppendArgs {
  CacheView c;
  int D, Hq, T;
  const uint16_t* k; int64_t ldk;
  const uint16_t* v; int64_t ldv;
  const uint16_t* q; int64_t ldq;
  uint16_t* q_out; int64_t ldqo;
  const int32_t* starts;
  const int32_t* position;
  const double* inv_freq;
  int rot;
};

__device__ __forceinline__ void unpack8(const uint4& u, float* f) {
  f[0] = bf16_lo(u.x); f[1] = bf16_hi(u.x); f[2] = bf16_lo(u.y); f[3] = bf16_hi(u.y);
  f[4] = bf16_lo(u.z); f[5] = bf16_hi(u.z); f[6] = bf16_lo(u.w); f[7] = bf16_hi(u.w);
}
__device__ __forceinline__ uint4 pack8(const float* f) {
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}

// One CTA a token. With R(pos) the rotation of the pairs (a, b) of a head by pos * inv_freq,
//   (a, b) -> (a cos - b sin, a sin + b cos),
// it writes R q, R k and v as they are. The angle is taken in turns in 64 bits and reduced to half a turn
// before it becomes 32 bits: far positions lose nothing. A thread holds 16 values of a head, the eight pairs
// of two vectors of 16 bytes half a rotation apart (next to each other a load would touch half of each sector: 24 us
// for 21). It is bound by bytes, or with few tokens by the chain sequence - length - page - store: a token's rows are read
// before that chain, which does not say where they are. (4094 tokens of 5 sequences, 32 / 8 heads of 128: 20.8 us = 4.9
// TB/s, 0.72 of the measured rate, floor 15: chains of 3 us, ten CTAs an SM, 2.7 waves of them; read behind the chain 40.
// One token 3.1 us.)
constexpr int APPEND_AHEAD = 3;      // items of a thread that are read first
constexpr int APPEND_SCAN = 1024;    // sequences whose starts the threads compare all at once
template <bool ADJACENT>
__global__ void __launch_bounds__(APPEND_THREADS) append_kernel(const AppendArgs a) {
  __shared__ float2 turn_of[MAX_DIM / 2 + MAX_DIM / 16];  // cos, sin; one entry left out after eight: no bank is met twice
  pdl_wait();
  pdl_trigger();
  const int t = blockIdx.x, D = a.D, H = a.c.heads, tid = threadIdx.x;
  const int log_pairs = D == 64 ? 2 : D == 128 ? 3 : 4, half = a.rot / 2;
  const int nq = a.q ? a.Hq : 0, items = (nq + 2 * H) << log_pairs;
  auto vectors = [&](int i, int& x, int& y) {  // of item i, in its head; true: to be turned
    const int head = i >> log_pairs, p = i & ((1 << log_pairs) - 1);
    const bool in = a.rot == 0 || p < a.rot / 16;
    x = in ? p * 8 : p * 16;
    y = in ? x + (a.rot == 0 ? D / 2 : half) : x + 8;
    return in && a.rot > 0 && head < nq + H;
  };
  auto source = [&](int i) {
    const int head = i >> log_pairs;
    return head < nq ? a.q + t * a.ldq + static_cast<int64_t>(head) * D
           : head < nq + H ? a.k + t * a.ldk + static_cast<int64_t>(head - nq) * D
                           : a.v + t * a.ldv + static_cast<int64_t>(head - nq - H) * D;
  };
  uint4 ahead[APPEND_AHEAD][2];
#pragma unroll
  for (int n = 0; n < APPEND_AHEAD; ++n) {
    const int i = tid + n * APPEND_THREADS;
    if (i < items) {
      int x, y;
      vectors(i, x, y);
      const uint16_t* src = source(i);
      ahead[n][0] = *reinterpret_cast<const uint4*>(src + x);
      ahead[n][1] = *reinterpret_cast<const uint4*>(src + y);
    }
  }
  auto turns = [&](int pos) {
    for (int i = tid; i < half; i += APPEND_THREADS) {
      double v = static_cast<double>(pos) * a.inv_freq[i] * 0.15915494309189533577;  // 1 / (2 pi)
      v -= rint(v);
      float2 c;
      sincospif(static_cast<float>(2.0 * v), &c.y, &c.x);
      turn_of[i + i / 8] = c;
    }
  };
  const int given = a.position ? a.position[t] : 0;
  if (a.position) turns(given);
  int s = t, first = t, count = 1;
  if (a.starts) {  // the last sequence that starts at t or before it
    if (t >= a.starts[a.c.seqs]) return;  // rows behind the last sequence
    if (a.c.seqs <= APPEND_SCAN) {
      int n = 0;
      for (int i = 0; i < a.c.seqs; i += APPEND_THREADS)
        n += __syncthreads_count(i + tid < a.c.seqs && a.starts[i + tid] <= t);
      s = n > 0 ? n - 1 : 0;
    } else {
      int lo = 0, hi = a.c.seqs;  // starts[lo] <= t < starts[hi]
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.starts[mid] <= t) lo = mid;
        else hi = mid;
      }
      s = lo;
    }
    first = a.starts[s];
    count = a.starts[s + 1] - first;
  }
  const int held = a.c.length[s];
  if (!a.starts && held == 0) return;  // an idle sequence of the batch
  const int64_t at = static_cast<int64_t>(held) - count + (t - first);
  const bool inside = at >= 0 && at < a.c.cap && t >= first && t - first < count;
  const int slot = inside ? static_cast<int>(at) : 0;
  const int32_t page = inside ? a.c.page_of(s, slot) : -1;
  if (!a.c.good(page)) {  // no such slot or page: the token is left out
    if (tid == 0) report(&g_err_cache, ORDERMOE_DEV_BAD_INDEX, t);
    return;
  }
  const int pos = a.position ? given : slot;
  if (!a.position) turns(pos);
  if (a.c.pos)
    for (int h = tid; h < H; h += APPEND_THREADS) a.c.pos[a.c.side(s, h, slot)] = pos;
  if (a.c.mass)
    for (int h = tid; h < H; h += APPEND_THREADS) a.c.mass[a.c.side(s, h, slot)] = 0.0f;
  __syncthreads();
  auto finish = [&](int i, const uint4& u, const uint4& w) {
    const int head = i >> log_pairs, p = i & ((1 << log_pairs) - 1);
    int x, y;
    const bool turn = vectors(i, x, y);
    uint16_t* dst = head < nq ? a.q_out + t * a.ldqo + static_cast<int64_t>(head) * D
                    : head < nq + H ? a.c.k + a.c.row(page, head - nq, slot) * D
                                    : a.c.v + a.c.row(page, head - nq - H, slot) * D;
    if (!turn) {
      *reinterpret_cast<uint4*>(dst + x) = u;
      *reinterpret_cast<uint4*>(dst + y) = w;
      return;
    }
    float m[16];
    unpack8(u, m);
    unpack8(w, m + 8);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      // pair j: (j, j + 8) of the two vectors, or neighbours in one of them
      const int f = ADJACENT ? p * 4 + j % 4 + j / 4 * (half / 2) : p * 8 + j;
      const float2 c = turn_of[f + f / 8];
      float &e = ADJACENT ? m[2 * j] : m[j], &o = ADJACENT ? m[2 * j + 1] : m[8 + j];
      const float turned = e * c.x - o * c.y;
      o = e * c.y + o * c.x;
      e = turned;
    }
    *reinterpret_cast<uint4*>(dst + x) = pack8(m);
    *reinterpret_cast<uint4*>(dst + y) = pack8(m + 8);
  };
#pragma unroll
  for (int n = 0; n < APPEND_AHEAD; ++n)
    if (tid + n * APPEND_THREADS < items) finish(tid + n * APPEND_THREADS, ahead[n][0], ahead[n][1]);
  for (int i = tid + APPEND_AHEAD * APPEND_THREADS; i < items; i += APPEND_THREADS) {
    int x, y;
    vectors(i, x, y);
    const uint16_t* src = source(i);
    finish(i, *reinterpret_cast<const uint4*>(src + x), *reinterpret_cast<const uint4*>(src + y));
  }
}

// -------------------------------------------------------------------------- evict
constexpr int EVICT_THREADS = 1024, EVICT_WARPS = 32;
constexpr int EVICT_KEYS = 49152;  // keys of a row that shared memory holds; longer rows are read again a round

struct EvictArgs {
  CacheView c;
  int budget, sinks, recent;
  const int32_t* newest;
  int32_t* length_out;
  int32_t* count;  // [rows] slots that move
  int32_t* moves;  // [rows][2][budget]: to, from
  int smem_keys;
};

// Larger keys stay. Protected tokens are above every weight; weights as ordered integers (-0 = 0, NaN as 0:
// not attended).
__device__ __forceinline__ uint32_t evict_key(const EvictArgs& a, float mass, int pos, int64_t old) {
  if (pos < a.sinks || pos > old) return 0xFFFFFFFFu;
  const uint32_t b = mass == mass && mass != 0.0f ? __float_as_uint(mass) : 0u;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Exclusive sums of one value a warp, and their total.
template <int WARPS>
__device__ __forceinline__ int block_before(int v, int* warp_sums, int* total) {
  const int w = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (lane == 0) warp_sums[w] = v;
  __syncthreads();
  const int x = lane < WARPS ? warp_sums[lane] : 0;  // every warp sums for itself
  const int before = __reduce_add_sync(~0u, lane < w ? x : 0);
  *total = __reduce_add_sync(~0u, x);
  __syncthreads();
  return before;
}

// One CTA a (sequence, head). The budget-th largest key, ties to the lower slot; then the freed slots below the
// budget and the kept ones behind it, each ascending: the i-th kept one moves into the i-th freed one. Order
// within the cache says nothing to attention, so only these rows move.
//
// The key is found two bits a round, by how many keys reach each of three candidates (histograms of eight bits met in
// few bins, weights being of a kind: 16383 slots 51 us), and as soon as a candidate is reached by exactly the budget
// no further. Rows of up to KEYS * NT slots have their keys in registers, key i in thread i % NT; longer ones in
// shared memory, or beyond that they are read again a round. Once the keys that a candidate can still part are one a
// thread at most, they alone are counted. (64 rows of 1500 to 16383 slots: 21 us, most of it instructions of 64 SMs, and 21 for
// the moves behind it, 100000 rows of 2 x 256 bytes; 256 rows of 1025 slots with their one move each: 10.3 us. 8 rows cut to
// 4096, both launches: of 16384 slots 27 us, of 32768 in shared memory 68, of 65536 and 131072 read again 345 and 658.)
constexpr int KEYS = 16;
template <int NT>
struct Select {
  static constexpr int WARPS = NT / 32;
  int hits[16][3];
  uint32_t near[NT];  // the keys that are still counted, once they are one a thread
  int n_near;
  int sums[WARPS];
  int block[KEYS * WARPS];  // of 32 slots each, in order
};

// Exclusive sums over the blocks of 32 slots; every entry may hold two counts of 16 bits.
template <int NT>
__device__ __forceinline__ int blocks_before(Select<NT>& s, int blocks) {
  constexpr int WARPS = NT / 32;
  static_assert(KEYS * WARPS <= NT, "a block a thread at most");
  const int tid = threadIdx.x, lane = tid % 32;
  __syncthreads();
  const int v = tid < blocks ? s.block[tid] : 0;
  int upto = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(~0u, upto, o);
    if (lane >= o) upto += x;
  }
  int total;
  const int base = block_before<WARPS>(__shfl_sync(~0u, upto, 31), s.sums, &total);
  if (tid < blocks) s.block[tid] = base + upto - v;
  __syncthreads();
  return total;
}

template <int NT>
__device__ __forceinline__ int select_held(const EvictArgs& a, Select<NT>& s, const float* mass, const int32_t* pos, int n,
                                           int64_t old, int32_t* to, int32_t* from) {
  constexpr int WARPS = NT / 32;
  const int tid = threadIdx.x, lane = tid % 32, w = tid / 32;
  const unsigned below = (1u << lane) - 1;
  uint32_t key[KEYS];
#pragma unroll
  for (int half = 0; half < KEYS; half += KEYS / 2) {  // eight loads of each kind on their way at a time
    float m[KEYS / 2];
    int p[KEYS / 2];
#pragma unroll
    for (int k = 0; k < KEYS / 2; ++k) {
      const int i = min((half + k) * NT + tid, n - 1);
      m[k] = (half + k) * NT < n ? mass[i] : 0.0f;
      p[k] = (half + k) * NT < n && pos ? pos[i] : i;
    }
#pragma unroll
    for (int k = 0; k < KEYS / 2; ++k)
      key[half + k] = (half + k) * NT + tid < n ? evict_key(a, m[k], p[k], old) : 0u;
  }
  if (tid < 48) s.hits[tid / 3][tid % 3] = 0;
  if (tid == 0) s.n_near = 0;
  __syncthreads();
  uint32_t known = 0, mine = key[0];
  int reach = n, upper = 0;  // keys that reach `known`, and the bound above it
  int base = 0;              // near: keys above the bound, which are counted no more
  bool exact = false, near = n <= NT;
  for (int round = 0; round < 16 && !exact; ++round) {
    const int shift = 30 - 2 * round;
    const uint32_t c1 = known | 1u << shift, c2 = known | 2u << shift, c3 = known | 3u << shift;
    uint32_t c = 0;  // three counts of ten bits: 512 a warp at most
    if (near) {
      c = (mine >= c1 ? 1u : 0u) + (mine >= c2 ? 1u << 10 : 0u) + (mine >= c3 ? 1u << 20 : 0u);
    } else {
#pragma unroll
      for (int k = 0; k < KEYS; ++k) {
        if (k * NT >= n) break;
        c += (key[k] >= c1 ? 1u : 0u) + (key[k] >= c2 ? 1u << 10 : 0u) + (key[k] >= c3 ? 1u << 20 : 0u);
      }
    }
    c = __reduce_add_sync(~0u, c);
    if (lane < 3 && c != 0) atomicAdd(&s.hits[round][lane], static_cast<int>(c >> (10 * lane) & 1023u));
    __syncthreads();
    int up = 0;
#pragma unroll
    for (int j = 0; j < 3; ++j) {
      const int h = s.hits[round][j] + base;
      if (h >= a.budget) {
        ++up;
        reach = h;
      } else if (up == j) {
        upper = h;
      }
      exact = exact || h == a.budget;
    }
    known |= static_cast<uint32_t>(up) << shift;
    if (near || reach - upper > NT) continue;
    // what lies in [known, known + 2^shift) is one a thread at most
    const uint32_t span = (1u << shift) - 1;
    int here = 0;
#pragma unroll
    for (int k = 0; k < KEYS; ++k) {
      if (k * NT >= n) break;
      here += __popc(__ballot_sync(~0u, k * NT + tid < n && key[k] - known <= span));
    }
    int at = lane == 0 ? atomicAdd(&s.n_near, here) : 0;
    at = __shfl_sync(~0u, at, 0);
#pragma unroll
    for (int k = 0; k < KEYS; ++k) {
      if (k * NT >= n) break;
      const bool in = k * NT + tid < n && key[k] - known <= span;
      const unsigned v = __ballot_sync(~0u, in);
      if (in) s.near[at + __popc(v & below)] = key[k];
      at += __popc(v);
    }
    __syncthreads();
    mine = tid < reach - upper ? s.near[tid] : 0u;
    base = upper;
    near = true;
  }
  // Kept: keys above `known`, and of those equal to it the first `left`. Exactly as many keys as the budget reach an exact one.
  int left = n, total = 0;
  if (!exact) {
    int above = 0;
#pragma unroll
    for (int k = 0; k < KEYS; ++k) {
      if (k * NT >= n) break;
      above += key[k] > known;
      const unsigned eq = __ballot_sync(~0u, k * NT + tid < n && key[k] == known);
      if (lane == 0) s.block[k * WARPS + w] = __popc(eq);
    }
    block_before<WARPS>(__reduce_add_sync(~0u, above), s.sums, &total);
    left = a.budget - total;
    blocks_before<NT>(s, (n + NT - 1) / NT * WARPS);
  }
  unsigned kept = 0;  // bit k: key k stays
#pragma unroll
  for (int k = 0; k < KEYS; ++k) {
    if (k * NT >= n) break;
    const bool in = k * NT + tid < n;
    const unsigned eq = __ballot_sync(~0u, in && key[k] == known);
    const int tie = (exact ? 0 : s.block[k * WARPS + w]) + __popc(eq & below);
    if (in && (key[k] > known || (key[k] == known && (exact || tie < left)))) kept |= 1u << k;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < KEYS; ++k) {
    if (k * NT >= n) break;
    const int i = k * NT + tid;
    const unsigned fr = __ballot_sync(~0u, i < n && i < a.budget && !(kept >> k & 1));
    const unsigned lt = __ballot_sync(~0u, i >= a.budget && (kept >> k & 1));
    if (lane == 0) s.block[k * WARPS + w] = __popc(fr) | __popc(lt) << 16;
  }
  total = blocks_before<NT>(s, (n + NT - 1) / NT * WARPS);
#pragma unroll
  for (int k = 0; k < KEYS; ++k) {
    if (k * NT >= n) break;
    const int i = k * NT + tid, at = s.block[k * WARPS + w];
    const bool freed = i < n && i < a.budget && !(kept >> k & 1), late = i >= a.budget && (kept >> k & 1);
    const unsigned fr = __ballot_sync(~0u, freed), lt = __ballot_sync(~0u, late);
    if (freed) to[(at & 0xFFFF) + __popc(fr & below)] = i;
    if (late) from[(at >> 16) + __popc(lt & below)] = i;
  }
  return total & 0xFFFF;  // as many late kept slots as freed ones
}

// Moves some of the listed rows of both halves of the cache with their weights and positions: threads that share a
// 16-byte vector of `AHEAD` rows at a time, rows first and on by `step`. Sources lie behind the budget and targets below it: no
// move reads what another one writes.
constexpr int MOVE_AHEAD = 2;  // (64 heads of 1500 to 16383 slots to 2048, both launches: 1 row 55 us, 2 48, 4 49, 8 56)
template <int D>
__device__ __forceinline__ void move_rows(const EvictArgs& a, int s, int h, const int32_t* to, const int32_t* from, int n,
                                          int first, int step) {
  constexpr int VECS = D / 8, PER = 2 * VECS, AHEAD = MOVE_AHEAD;  // vectors of a row, of both halves
  const int v = threadIdx.x % PER;
  uint16_t* half = (v < VECS ? a.c.k : a.c.v) + v % VECS * 8;
  uint32_t* beside = v == 0 ? reinterpret_cast<uint32_t*>(a.c.mass) : v == 1 ? reinterpret_cast<uint32_t*>(a.c.pos) : nullptr;
  if (beside) beside += a.c.side(s, h, 0);
  for (int m = first + static_cast<int>(threadIdx.x) / PER; m < n; m += AHEAD * step) {
    int x[AHEAD], y[AHEAD];
    int32_t px[AHEAD], py[AHEAD];
    uint4 u[AHEAD];
    uint32_t w[AHEAD];  // weight or position, by the threads of a row's first vectors
    bool ok[AHEAD];
#pragma unroll
    for (int e = 0; e < AHEAD; ++e) {
      const bool in = m + e * step < n;
      x[e] = in ? from[m + e * step] : -1;
      y[e] = in ? to[m + e * step] : 0;
    }
#pragma unroll
    for (int e = 0; e < AHEAD; ++e) {
      px[e] = x[e] >= 0 ? a.c.page_of(s, x[e]) : 0;
      py[e] = x[e] >= 0 ? a.c.page_of(s, y[e]) : 0;
    }
#pragma unroll
    for (int e = 0; e < AHEAD; ++e) {
      ok[e] = x[e] >= 0 && a.c.good(px[e]) && a.c.good(py[e]);
      if (ok[e]) {
        u[e] = *reinterpret_cast<const uint4*>(half + a.c.row(px[e], h, x[e]) * D);
        if (beside) w[e] = beside[x[e]];
      } else if (x[e] >= 0 && v == 0) report(&g_err_cache, ORDERMOE_DEV_BAD_INDEX, s);
    }
#pragma unroll
    for (int e = 0; e < AHEAD; ++e) {
      if (!ok[e]) continue;
      *reinterpret_cast<uint4*>(half + a.c.row(py[e], h, y[e]) * D) = u[e];
      if (beside) beside[y[e]] = w[e];
    }
  }
}

// What every CTA of a selection does first: the length out, bad lengths, and whether there is anything to cut.
struct Cut {
  int s, h, n;
  int64_t old;  // the newest position that no longer counts as recent; without a newest one and recent = 0 every one
  const float* mass;
  const int32_t* pos;
};
__device__ __forceinline__ bool begin_cut(const EvictArgs& a, Cut& c) {
  const int row = blockIdx.x;
  c.s = row / a.c.heads;
  c.h = row % a.c.heads;
  c.n = a.c.slots(c.s);
  if (threadIdx.x == 0) {
    if (c.n != a.c.length[c.s]) report(&g_err_cache, ORDERMOE_DEV_BAD_INDEX, c.s);
    if (c.h == 0) a.length_out[c.s] = c.n < a.budget ? c.n : a.budget;
    if (c.n <= a.budget) a.count[row] = 0;
  }
  if (c.n <= a.budget) return false;
  c.old = a.newest ? static_cast<int64_t>(a.newest[c.s]) - a.recent
                   : a.c.pos ? static_cast<int64_t>(INT32_MAX) : static_cast<int64_t>(c.n) - 1 - a.recent;
  c.mass = a.c.mass + a.c.side(c.s, c.h, 0);
  c.pos = a.c.pos ? a.c.pos + a.c.side(c.s, c.h, 0) : nullptr;
  return true;
}

// Rows of up to KEYS * NT slots. Where a row can have few moves only (MOVES: a cache that is cut at every step), its own
// CTA does them and there is no second launch.
template <int NT, int D, bool MOVES>
__global__ void __launch_bounds__(NT) evict_short_kernel(const EvictArgs a) {
  __shared__ Select<NT> s;
  pdl_wait();
  pdl_trigger();
  Cut c;
  if (!begin_cut(a, c)) return;
  int32_t* to = a.moves + static_cast<int64_t>(blockIdx.x) * 2 * a.budget;
  int32_t* from = to + a.budget;
  const int moves = select_held<NT>(a, s, c.mass, c.pos, c.n, c.old, to, from);
  if constexpr (MOVES) {
    __syncthreads();  // the lists are written
    move_rows<D>(a, c.s, c.h, to, from, moves, 0, NT / (D / 4));
  } else if (threadIdx.x == 0) {
    a.count[blockIdx.x] = moves;
  }
}

__global__ void __launch_bounds__(EVICT_THREADS) evict_select_kernel(const EvictArgs a) {
  extern __shared__ uint32_t keys[];
  __shared__ Select<EVICT_THREADS> held_s;
  __shared__ int counts[2][3][EVICT_WARPS];
  pdl_wait();
  pdl_trigger();
  Cut cut;
  if (!begin_cut(a, cut)) return;
  const int row = blockIdx.x, n = cut.n, tid = threadIdx.x, lane = tid % 32, w = tid / 32;
  int32_t* to = a.moves + static_cast<int64_t>(row) * 2 * a.budget;
  int32_t* from = to + a.budget;
  if (n <= KEYS * EVICT_THREADS) {
    const int moves = select_held<EVICT_THREADS>(a, held_s, cut.mass, cut.pos, n, cut.old, to, from);
    if (tid == 0) a.count[row] = moves;
    return;
  }
  int* sums = held_s.sums;
  const float* mass = cut.mass;
  const int32_t* pos = cut.pos;
  auto read = [&](int i) { return evict_key(a, mass[i], pos ? pos[i] : i, cut.old); };
  const bool held = n <= a.smem_keys;
  auto key = [&](int i) { return held ? keys[i] : read(i); };
  if (held)
    for (int i = tid; i < n; i += EVICT_THREADS) keys[i] = read(i);
  uint32_t known = 0;
  __syncthreads();
  for (int round = 0; round < 16; ++round) {
    const int shift = 30 - 2 * round;
    int c[3] = {0, 0, 0};
    for (int i = tid; i < n; i += EVICT_THREADS) {
      const uint32_t x = key(i);
#pragma unroll
      for (int j = 0; j < 3; ++j) c[j] += x >= (known | static_cast<uint32_t>(j + 1) << shift);
    }
    int(*hits)[EVICT_WARPS] = counts[round & 1];
#pragma unroll
    for (int j = 0; j < 3; ++j) {
      c[j] = __reduce_add_sync(~0u, c[j]);
      if (lane == 0) hits[j][w] = c[j];
    }
    __syncthreads();
    int up = 0;  // candidates that the budget-th largest reaches
#pragma unroll
    for (int j = 0; j < 3; ++j) up += __reduce_add_sync(~0u, hits[j][lane]) >= a.budget;
    known |= static_cast<uint32_t>(up) << shift;
  }
  // the keys above it all stay, and so many of its equals
  int above = 0, total;
  for (int i = tid; i < n; i += EVICT_THREADS) above += key(i) > known;
  block_before<EVICT_WARPS>(__reduce_add_sync(~0u, above), sums, &total);
  const int left = a.budget - total;
  // every warp has a range of slots, 32 at a time
  const int per = ((n + EVICT_WARPS - 1) / EVICT_WARPS + 31) / 32 * 32;
  const int b0 = min(w * per, n), b1 = min(b0 + per, n);
  int ties = 0;
  for (int i = b0; i < b1; i += 32) ties += __popc(__ballot_sync(~0u, i + lane < b1 && key(i + lane) == known));
  const int ties_before = block_before<EVICT_WARPS>(ties, sums, &total);
  const unsigned below_me = (1u << lane) - 1;
  // freed and late kept slots of 32 slots from i on, as votes
  auto votes = [&](int i, int& tie, unsigned& freed, unsigned& late) {
    const bool in = i + lane < b1;
    const uint32_t x = in ? key(i + lane) : 0u;
    const unsigned eq = __ballot_sync(~0u, in && x == known);
    const bool kept = in && (x > known || (x == known && tie + __popc(eq & below_me) < left));
    tie += __popc(eq);
    freed = __ballot_sync(~0u, in && !kept && i + lane < a.budget);
    late = __ballot_sync(~0u, kept && i + lane >= a.budget);
  };
  int tie = ties_before, n_freed = 0, n_late = 0;
  unsigned freed, late;
  for (int i = b0; i < b1; i += 32) {
    votes(i, tie, freed, late);
    n_freed += __popc(freed);
    n_late += __popc(late);
  }
  int at_to = block_before<EVICT_WARPS>(n_freed, sums, &total), at_from = block_before<EVICT_WARPS>(n_late, sums, &total);
  if (tid == 0) a.count[row] = total;  // as many late kept slots as freed ones
  tie = ties_before;
  for (int i = b0; i < b1; i += 32) {
    votes(i, tie, freed, late);
    if (freed >> lane & 1) to[at_to + __popc(freed & below_me)] = i + lane;
    if (late >> lane & 1) from[at_from + __popc(late & below_me)] = i + lane;
    at_to += __popc(freed);
    at_from += __popc(late);
  }
}

constexpr int MOVE_THREADS = 256, MOVE_SELF = 64;  // moves of a row that its selection does itself
template <int D>
__global__ void __launch_bounds__(MOVE_THREADS) evict_move_kernel(const EvictArgs a) {
  pdl_wait();
  pdl_trigger();
  const int row = blockIdx.x, n = a.count[row];
  constexpr int PER = MOVE_THREADS / (D / 4);  // rows of a CTA at a time
  const int32_t* to = a.moves + static_cast<int64_t>(row) * 2 * a.budget;
  move_rows<D>(a, row / a.c.heads, row % a.c.heads, to, to + a.budget, n, blockIdx.y * PER, gridDim.y * PER);
}

template <int D>
static int evict(const EvictArgs& a, cudaStream_t stream) {
  const int rows = a.c.seqs * a.c.heads;
  const int most = a.c.cap - a.budget < a.budget ? a.c.cap - a.budget : a.budget;  // moves of a row
  if (most <= 0) {  // no row can have more than the budget: lengths alone
    OM_LAUNCH_PDL("evict_short_kernel", evict_short_kernel<256, D, true>, dim3(rows), dim3(256), 0, stream, a);
    return ORDERMOE_OK;
  }
  if (a.c.cap <= KEYS * 256 && most <= MOVE_SELF) {
    OM_LAUNCH_PDL("evict_short_kernel", evict_short_kernel<256, D, true>, dim3(rows), dim3(256), 0, stream, a);
    return ORDERMOE_OK;
  }
  if (a.c.cap <= KEYS * 256)
    OM_LAUNCH_PDL("evict_short_kernel", evict_short_kernel<256, D, false>, dim3(rows), dim3(256), 0, stream, a);
  else if (a.c.cap <= KEYS * EVICT_THREADS)
    OM_LAUNCH_PDL("evict_short_kernel", evict_short_kernel<EVICT_THREADS, D, false>, dim3(rows), dim3(EVICT_THREADS), 0,
                  stream, a);
  else
    OM_LAUNCH_PDL("evict_select_kernel", evict_select_kernel, dim3(rows), dim3(EVICT_THREADS),
                  static_cast<size_t>(a.smem_keys) * 4, stream, a);
  int64_t y = (static_cast<int64_t>(most) * (D / 4) + MOVE_AHEAD * MOVE_THREADS - 1) / (MOVE_AHEAD * MOVE_THREADS);
  const int64_t fill = 48ll * num_sms() / rows + 1;
  y = y > fill ? fill : y;
  OM_LAUNCH_PDL("evict_move_kernel", evict_move_kernel<D>, dim3(rows, static_cast<unsigned>(y)), dim3(MOVE_THREADS), 0, stream, a);
  return ORDERMOE_OK;
}

}  // namespace kv
}  // namespace om

using namespace om;

static bool rows_ok(const void* p, int64_t ld, int64_t width, bool many) {
  return aligned16(p) && (!many || (ld >= width && ld % 8 == 0 && ld < (1ll << 38)));
}

extern "C" int ordermoe_cache_append(const ordermoe_cache* cache, const uint16_t* k, int64_t ldk, const uint16_t* v,
                                     int64_t ldv, const uint16_t* q, int64_t ldq, uint16_t* q_out, int64_t ldqo,
                                     int T, int q_heads, const int32_t* starts, const int32_t* position,
                                     const double* inv_freq, int rot_dim, int adjacent, ordermoe_stream_t stream) {
  OM_TRACE();
  const int rc = check_cache(cache, "cache_append");
  if (rc) return rc;
  if (T < 0 || (T > 0 && cache->seqs == 0) || (!starts && T != cache->seqs))
    return fail(ORDERMOE_ERR_INVALID_ARG, "cache_append: need T >= 0 tokens of the cache's sequences, one each without starts");
  if (!q != !q_out) return fail(ORDERMOE_ERR_INVALID_ARG, "cache_append: q and q_out go together");
  if (q && (q_heads <= 0 || q_heads > 4096))
    return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "cache_append: need 1 to 4096 query heads");
  if (rot_dim < 0 || rot_dim > cache->dim || rot_dim % 16 != 0)
    return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "cache_append: rot_dim must be a multiple of 16, at most the heads' width");
  if (T == 0) return ORDERMOE_OK;
  if (!k || !v || (rot_dim > 0 && !inv_freq)) return fail(ORDERMOE_ERR_INVALID_ARG, "cache_append: null pointer");
  const int64_t wk = static_cast<int64_t>(cache->heads) * cache->dim, wq = static_cast<int64_t>(q_heads) * cache->dim;
  if (!rows_ok(k, ldk, wk, T > 1) || !rows_ok(v, ldv, wk, T > 1) ||
      (q && (!rows_ok(q, ldq, wq, T > 1) || !rows_ok(q_out, ldqo, wq, T > 1))))
    return fail(ORDERMOE_ERR_INVALID_ARG,
                "cache_append: rows must start at multiples of 16 bytes and their strides may not be shorter than they are");
  if (q && q == q_out && T > 1 && ldq != ldqo)
    return fail(ORDERMOE_ERR_INVALID_ARG, "cache_append: a q_out that is q must have its stride");
  if (reinterpret_cast<uintptr_t>(starts) % 4 || reinterpret_cast<uintptr_t>(position) % 4 ||
      reinterpret_cast<uintptr_t>(inv_freq) % 8)
    return fail(ORDERMOE_ERR_INVALID_ARG, "cache_append: starts, position or inv_freq is not aligned to its type");
  kv::AppendArgs a{};
  a.c = cache_view(cache);
  a.D = cache->dim; a.Hq = q_heads; a.T = T;
  a.k = k; a.ldk = ldk; a.v = v; a.ldv = ldv; a.q = q; a.ldq = ldq; a.q_out = q_out; a.ldqo = ldqo;
  a.starts = starts; a.position = position; a.inv_freq = inv_freq; a.rot = rot_dim;
  const auto kernel = adjacent ? kv::append_kernel<true> : kv::append_kernel<false>;
  OM_LAUNCH_PDL("append_kernel", kernel, dim3(T), dim3(kv::APPEND_THREADS), 0, stream, a);
  return ORDERMOE_OK;
}

extern "C" size_t ordermoe_cache_evict_workspace_bytes(int seqs, int heads, int budget) {
  if (seqs < 0 || heads <= 0 || budget <= 0) return 0;
  const size_t rows = static_cast<size_t>(seqs) * heads;
  return (rows + 63) / 64 * 256 + rows * 8 * budget;
}

static int evict_attr() {
  return static_cast<int>(cudaFuncSetAttribute(kv::evict_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               kv::EVICT_KEYS * 4));
}

extern "C" int ordermoe_cache_evict(const ordermoe_cache* cache, int budget, int sinks, int recent,
                                    const int32_t* newest, int32_t* length_out, void* workspace,
                                    size_t workspace_bytes, ordermoe_stream_t stream) {
  OM_TRACE();
  const int rc = check_cache(cache, "cache_evict");
  if (rc) return rc;
  if (budget <= 0 || sinks < 0 || recent < 0 || static_cast<int64_t>(sinks) + recent > budget)
    return fail(ORDERMOE_ERR_INVALID_ARG, "cache_evict: need budget > 0, and sinks and recent >= 0 within it");
  if (budget > (1 << 30)) return fail(ORDERMOE_ERR_UNSUPPORTED_SHAPE, "cache_evict: need a budget of at most 2^30");
  if (cache->seqs == 0) return ORDERMOE_OK;
  if (!cache->mass || !length_out) return fail(ORDERMOE_ERR_INVALID_ARG, "cache_evict: null pointer (mass or length_out)");
  if (recent > 0 && cache->pos && !newest)
    return fail(ORDERMOE_ERR_INVALID_ARG, "cache_evict: recent positions need a pointer to the newest ones");
  // every head's CTA reads them, and one of them writes the new length
  auto meets = [&](const int32_t* p) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(length_out), b = reinterpret_cast<uintptr_t>(p);
    return p && (a < b ? b - a : a - b) < static_cast<uintptr_t>(cache->seqs) * 4;
  };
  if (meets(cache->length) || meets(newest))
    return fail(ORDERMOE_ERR_INVALID_ARG, "cache_evict: length_out may overlap neither the cache's length nor newest");
  if (reinterpret_cast<uintptr_t>(newest) % 4 || reinterpret_cast<uintptr_t>(length_out) % 4)
    return fail(ORDERMOE_ERR_INVALID_ARG, "cache_evict: newest or length_out is not aligned to its type");
  const int64_t cap = static_cast<int64_t>(cache->seq_pages) * cache->page;  // with a budget of as many nothing moves
  const int listed = static_cast<int>(budget < cap ? budget : cap);
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 != 0 ||
      workspace_bytes < ordermoe_cache_evict_workspace_bytes(cache->seqs, cache->heads, listed))
    return fail(ORDERMOE_ERR_INVALID_ARG, "cache_evict: workspace is null, too small or not 256-byte aligned");
  static PerDevice attr_;
  const int e = per_device(attr_, evict_attr);
  if (e != 0) return cuda_fail(static_cast<cudaError_t>(e), "cudaFuncSetAttribute(evict_select)");
  kv::EvictArgs a{};
  a.c = cache_view(cache);
  a.budget = budget; a.sinks = sinks; a.recent = recent; a.newest = newest; a.length_out = length_out;
  const int rows = cache->seqs * cache->heads;
  a.count = static_cast<int32_t*>(workspace);
  a.moves = a.count + (static_cast<size_t>(rows) + 63) / 64 * 64;
  a.smem_keys = a.c.cap < kv::EVICT_KEYS ? a.c.cap : kv::EVICT_KEYS;
  if (cache->dim == 64) return kv::evict<64>(a, stream);
  if (cache->dim == 128) return kv::evict<128>(a, stream);
  return kv::evict<256>(a, stream);
}
