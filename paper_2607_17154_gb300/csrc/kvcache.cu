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
constexpr int APPEND_THREADS = 256;
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
  int rot, adjacent;
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
// of two vectors of 16 bytes (adjacent pairs: the two next to each other; else half a rotation apart).
__global__ void __launch_bounds__(APPEND_THREADS) append_kernel(AppendArgs a) {
  __shared__ float cs[MAX_DIM / 2], sn[MAX_DIM / 2];
  pdl_wait();
  pdl_trigger();
  const int t = blockIdx.x, D = a.D, H = a.c.heads;
  int s = t, first = t, count = 1;
  if (a.starts) {  // the last sequence that starts at t or before it
    if (t >= a.starts[a.c.seqs]) return;  // rows behind the last sequence
    int lo = 0, hi = a.c.seqs;  // starts[lo] <= t < starts[hi] where the starts ascend
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (a.starts[mid] <= t) lo = mid;
      else hi = mid;
    }
    s = lo;
    first = a.starts[s];
    count = a.starts[s + 1] - first;
  }
  const int64_t at = static_cast<int64_t>(a.c.length[s]) - count + (t - first);
  const bool inside = at >= 0 && at < a.c.cap && t >= first && t - first < count;
  const int slot = inside ? static_cast<int>(at) : 0;
  const int32_t page = inside ? a.c.page_of(s, slot) : -1;
  if (!a.c.good(page)) {  // no such slot or page: the token is left out
    if (threadIdx.x == 0) report(&g_err_cache, ORDERMOE_DEV_BAD_INDEX, t);
    return;
  }
  const int pos = a.position ? a.position[t] : slot;
  const int half = a.rot / 2;
  for (int i = threadIdx.x; i < half; i += APPEND_THREADS) {
    double turns = static_cast<double>(pos) * a.inv_freq[i] * 0.15915494309189533577;  // 1 / (2 pi)
    turns -= rint(turns);
    sincospif(static_cast<float>(2.0 * turns), &sn[i], &cs[i]);
  }
  if (a.c.pos)
    for (int h = threadIdx.x; h < H; h += APPEND_THREADS) a.c.pos[a.c.side(s, h, slot)] = pos;
  if (a.c.mass)
    for (int h = threadIdx.x; h < H; h += APPEND_THREADS) a.c.mass[a.c.side(s, h, slot)] = 0.0f;
  __syncthreads();
  const int pairs = D / 16, nq = a.q ? a.Hq : 0;
  const int items = (nq + 2 * H) * pairs;
  for (int i = threadIdx.x; i < items; i += APPEND_THREADS) {
    const int head = i / pairs, p = i % pairs;
    const uint16_t* src;
    uint16_t* dst;
    bool turn = true;
    if (head < nq) {
      src = a.q + t * a.ldq + static_cast<int64_t>(head) * D;
      dst = a.q_out + t * a.ldqo + static_cast<int64_t>(head) * D;
    } else if (head < nq + H) {
      const int h = head - nq;
      src = a.k + t * a.ldk + static_cast<int64_t>(h) * D;
      dst = a.c.k + a.c.row(page, h, slot) * D;
    } else {
      const int h = head - nq - H;
      src = a.v + t * a.ldv + static_cast<int64_t>(h) * D;
      dst = a.c.v + a.c.row(page, h, slot) * D;
      turn = false;
    }
    // the two vectors of this thread, in the rotated part or behind it
    int x, y, f;
    if (a.adjacent || p >= a.rot / 16) {
      x = p * 16; y = x + 8; f = p * 8;
    } else {
      x = p * 8; y = x + half; f = p * 8;
    }
    const uint4 u = *reinterpret_cast<const uint4*>(src + x), w = *reinterpret_cast<const uint4*>(src + y);
    if (!turn || p >= a.rot / 16) {
      *reinterpret_cast<uint4*>(dst + x) = u;
      *reinterpret_cast<uint4*>(dst + y) = w;
      continue;
    }
    float m[16];
    unpack8(u, m);
    unpack8(w, m + 8);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float &e = a.adjacent ? m[2 * j] : m[j], &o = a.adjacent ? m[2 * j + 1] : m[8 + j];
      const float c = cs[f + j], z = sn[f + j], e2 = e * c - o * z;
      o = e * z + o * c;
      e = e2;
    }
    *reinterpret_cast<uint4*>(dst + x) = pack8(m);
    *reinterpret_cast<uint4*>(dst + y) = pack8(m + 8);
  }
}

// -------------------------------------------------------------------------- evict
constexpr int EVICT_THREADS = 1024, EVICT_WARPS = 32;
constexpr int EVICT_KEYS = 49152;  // keys of a row that shared memory holds; longer rows are read again a pass

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

__device__ __forceinline__ int block_before(int v, int* warp_sums, int* total) {  // exclusive sum of a value a warp
  const int w = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (lane == 0) warp_sums[w] = v;
  __syncthreads();
  const int x = warp_sums[lane];  // every warp sums for itself
  int before = lane < w ? x : 0, all = x;
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    before += __shfl_xor_sync(~0u, before, o);
    all += __shfl_xor_sync(~0u, all, o);
  }
  __syncthreads();
  *total = all;
  return before;
}

// One CTA a (sequence, head). The budget-th largest key by four passes over 8 bits of it, ties to the lower
// slot; then the freed slots below the budget and the kept ones behind it, each ascending: the i-th kept one
// moves into the i-th freed one. Order within the cache says nothing to attention, so only these rows move.
__global__ void __launch_bounds__(EVICT_THREADS) evict_select_kernel(EvictArgs a) {
  extern __shared__ uint32_t keys[];
  __shared__ int hist[256];
  __shared__ int sums[EVICT_WARPS];
  __shared__ int pick[2];
  pdl_wait();
  pdl_trigger();
  const int row = blockIdx.x, s = row / a.c.heads, h = row % a.c.heads;
  const int tid = threadIdx.x, lane = tid % 32, w = tid / 32;
  const int n = a.c.slots(s);
  if (tid == 0) {
    if (n != a.c.length[s]) report(&g_err_cache, ORDERMOE_DEV_BAD_INDEX, s);
    if (h == 0) a.length_out[s] = n < a.budget ? n : a.budget;
    if (n <= a.budget) a.count[row] = 0;
  }
  if (n <= a.budget) return;
  // the newest position that no longer counts as recent; without a newest one and recent = 0 every one
  const int64_t old = a.newest ? static_cast<int64_t>(a.newest[s]) - a.recent
                               : a.c.pos ? static_cast<int64_t>(INT32_MAX) : static_cast<int64_t>(n) - 1 - a.recent;
  const float* mass = a.c.mass + a.c.side(s, h, 0);
  const int32_t* pos = a.c.pos ? a.c.pos + a.c.side(s, h, 0) : nullptr;
  auto read = [&](int i) { return evict_key(a, mass[i], pos ? pos[i] : i, old); };
  const bool held = n <= a.smem_keys;
  auto key = [&](int i) { return held ? keys[i] : read(i); };
  if (held)
    for (int i = tid; i < n; i += EVICT_THREADS) keys[i] = read(i);
  uint32_t known = 0;
  int left = a.budget;  // of the keys whose higher bits are `known`, the left-th largest is looked for
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    const uint32_t mask = shift == 24 ? 0u : 0xFFFFFFFFu << (shift + 8);
    for (int i = tid; i < n; i += EVICT_THREADS) {
      const uint32_t x = key(i);
      if ((x & mask) == known) atomicAdd(&hist[(x >> shift) & 255], 1);
    }
    __syncthreads();
    if (w == 0) {  // bins from the largest: lane l has bins 255 - 8 l and the seven below it
      int mine = 0;
      for (int j = 0; j < 8; ++j) mine += hist[255 - 8 * lane - j];
      int upto = mine;
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(~0u, upto, o);
        if (lane >= o) upto += x;
      }
      const int above = upto - mine;
      if (above < left && left <= upto) {
        int b = 255 - 8 * lane, sum = above;
        while (sum + hist[b] < left) sum += hist[b--];
        pick[0] = b;
        pick[1] = left - sum;
      }
    }
    __syncthreads();
    known |= static_cast<uint32_t>(pick[0]) << shift;
    left = pick[1];
    __syncthreads();
  }
  // every warp has a range of slots, 32 at a time
  const int per = ((n + EVICT_WARPS - 1) / EVICT_WARPS + 31) / 32 * 32;
  const int b0 = min(w * per, n), b1 = min(b0 + per, n);
  int ties = 0, total;
  for (int i = b0; i < b1; i += 32) ties += __popc(__ballot_sync(~0u, i + lane < b1 && key(i + lane) == known));
  const int ties_before = block_before(ties, sums, &total);
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
  int at_to = block_before(n_freed, sums, &total), at_from = block_before(n_late, sums, &total);
  if (tid == 0) a.count[row] = total;  // as many late kept slots as freed ones
  int32_t* to = a.moves + static_cast<int64_t>(row) * 2 * a.budget;
  int32_t* from = to + a.budget;
  tie = ties_before;
  for (int i = b0; i < b1; i += 32) {
    votes(i, tie, freed, late);
    if (freed >> lane & 1) to[at_to + __popc(freed & below_me)] = i + lane;
    if (late >> lane & 1) from[at_from + __popc(late & below_me)] = i + lane;
    at_to += __popc(freed);
    at_from += __popc(late);
  }
}

// Moves the listed rows of both halves of the cache with their weights and positions. Sources lie behind
// the budget and targets below it: no move reads what another one writes.
constexpr int MOVE_THREADS = 256;
__global__ void __launch_bounds__(MOVE_THREADS) evict_move_kernel(EvictArgs a, int D) {
  pdl_wait();
  pdl_trigger();
  const int row = blockIdx.x, s = row / a.c.heads, h = row % a.c.heads;
  const int n = a.count[row], vecs = D / 8, per = 2 * vecs;  // 16-byte vectors of a row, of both halves
  const int32_t* to = a.moves + static_cast<int64_t>(row) * 2 * a.budget;
  const int32_t* from = to + a.budget;
  const int64_t items = static_cast<int64_t>(n) * per, step = static_cast<int64_t>(gridDim.y) * MOVE_THREADS;
  for (int64_t i = static_cast<int64_t>(blockIdx.y) * MOVE_THREADS + threadIdx.x; i < items; i += step) {
    const int m = static_cast<int>(i / per), v = static_cast<int>(i % per);
    const int x = from[m], y = to[m];
    const int32_t px = a.c.page_of(s, x), py = a.c.page_of(s, y);
    if (!a.c.good(px) || !a.c.good(py)) {
      if (v == 0) report(&g_err_cache, ORDERMOE_DEV_BAD_INDEX, s);
      continue;
    }
    uint16_t* half = v < vecs ? a.c.k : a.c.v;
    const int at = (v < vecs ? v : v - vecs) * 8;
    *reinterpret_cast<uint4*>(half + a.c.row(py, h, y) * D + at) =
        *reinterpret_cast<const uint4*>(half + a.c.row(px, h, x) * D + at);
    if (v == 0) a.c.mass[a.c.side(s, h, y)] = a.c.mass[a.c.side(s, h, x)];
    if (v == 1 && a.c.pos) a.c.pos[a.c.side(s, h, y)] = a.c.pos[a.c.side(s, h, x)];
  }
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
  a.starts = starts; a.position = position; a.inv_freq = inv_freq; a.rot = rot_dim; a.adjacent = adjacent != 0;
  OM_LAUNCH_PDL("append_kernel", kv::append_kernel, dim3(T), dim3(kv::APPEND_THREADS), 0, stream, a);
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
  if (length_out == cache->length)
    return fail(ORDERMOE_ERR_INVALID_ARG, "cache_evict: length_out may not be the cache's length");
  if (reinterpret_cast<uintptr_t>(newest) % 4 || reinterpret_cast<uintptr_t>(length_out) % 4)
    return fail(ORDERMOE_ERR_INVALID_ARG, "cache_evict: newest or length_out is not aligned to its type");
  if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 != 0 ||
      workspace_bytes < ordermoe_cache_evict_workspace_bytes(cache->seqs, cache->heads, budget))
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
  OM_LAUNCH_PDL("evict_select_kernel", kv::evict_select_kernel, dim3(rows), dim3(kv::EVICT_THREADS),
                static_cast<size_t>(a.smem_keys) * 4, stream, a);
  // rows of more than the budget's slots move at most so many
  const int64_t most = a.c.cap - static_cast<int64_t>(budget) < budget ? a.c.cap - static_cast<int64_t>(budget) : budget;
  int64_t y = (most * (cache->dim / 4) + 4 * kv::MOVE_THREADS - 1) / (4 * kv::MOVE_THREADS);
  const int64_t fill = 16ll * num_sms() / rows + 1;
  y = y < 1 ? 1 : y > fill ? fill : y;
  OM_LAUNCH_PDL("evict_move_kernel", kv::evict_move_kernel, dim3(rows, static_cast<unsigned>(y)), dim3(kv::MOVE_THREADS),
                0, stream, a, static_cast<int>(cache->dim));
  return ORDERMOE_OK;
}
