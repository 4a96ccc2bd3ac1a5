// Serving from a paged cache: rows in (append), rows out (eviction by accumulated attention weight), and the start
// of it, the state of rows that a compaction has written (admit).  The attention itself: cache_attention.hip.
#include <string.h>

#include "cache.h"

namespace cmp {

int cache_view(const compactor_cache_t *c, CacheNeed need, CacheView *view) {
  if (!c) return COMPACTOR_EINVAL;
  if (c->nreq < 1 || c->layers < 1 || c->kv_heads < 1) return COMPACTOR_EINVAL;
  if ((long long)c->layers * c->kv_heads > (1 << 20)) return COMPACTOR_EINVAL;
  if ((long long)c->nreq * c->layers * c->kv_heads > 0x7fffffffll) return COMPACTOR_EINVAL;
  if (c->head_dim != D) return COMPACTOR_EUNSUPPORTED;
  const compactor_page_pool_t &p = c->pool;
  if (p.page_size < 1 || p.num_pages < 1 || c->table_len < 1 || c->table_stride < c->table_len) return COMPACTOR_EINVAL;
  if ((long long)c->table_len * p.page_size > 0x7fffffffll - 64) return COMPACTOR_EINVAL;
  if (need != CACHE_SIZES) {
    if (!p.k_pages || !p.v_pages || !c->tables || !c->counts) return COMPACTOR_EINVAL;
    if (p.page_stride < 0 || p.layer_stride < 0 || p.head_stride < 0 || p.slot_stride < D) return COMPACTOR_EINVAL;
    if (c->count_stride_b < 0 || c->count_stride_l < 0) return COMPACTOR_EINVAL;
    if (c->state_page_stride < 0 || c->state_layer_stride < 0 || c->state_head_stride < 0) return COMPACTOR_EINVAL;
    const int state = (c->seen != nullptr) + (c->mass != nullptr) + (c->positions != nullptr);
    if (state != 3 && (state != 0 || need == CACHE_STATE)) return COMPACTOR_EINVAL;
    if (((reinterpret_cast<uintptr_t>(p.k_pages) | reinterpret_cast<uintptr_t>(p.v_pages)) & 15u) ||
        ((p.page_stride | p.layer_stride | p.head_stride | p.slot_stride) & 7) ||
        ((reinterpret_cast<uintptr_t>(c->tables) | reinterpret_cast<uintptr_t>(c->counts) |
          reinterpret_cast<uintptr_t>(c->seen) | reinterpret_cast<uintptr_t>(c->mass) |
          reinterpret_cast<uintptr_t>(c->positions)) & 3u))
      return COMPACTOR_EALIGN;
  }
  CacheView &v = *view;
  memset(&v, 0, sizeof(v));
  v.k = static_cast<uint16_t *>(p.k_pages);
  v.v = static_cast<uint16_t *>(p.v_pages);
  v.page_stride = p.page_stride; v.layer_stride = p.layer_stride;
  v.head_stride = p.head_stride; v.slot_stride = p.slot_stride;
  v.tables = c->tables; v.table_stride = c->table_stride;
  v.page_size = p.page_size; v.num_pages = p.num_pages;
  v.capacity = c->table_len * p.page_size;
  page_divisor(p.page_size, &v.div_mul, &v.div_shift);
  v.nreq = c->nreq; v.layers = c->layers; v.kv_heads = c->kv_heads;
  v.counts = c->counts; v.seen = c->seen;
  v.count_stride_b = c->count_stride_b; v.count_stride_l = c->count_stride_l;
  v.mass = c->mass; v.positions = c->positions;
  v.state_page_stride = c->state_page_stride; v.state_layer_stride = c->state_layer_stride;
  v.state_head_stride = c->state_head_stride;
  return COMPACTOR_OK;
}

// ------------------------------------------------------------------------------------------ append
// 16 lanes move the K and the V row of one token of one head, 16 bytes a lane, and note its state.  Bound by the
// latency of a chain of three: count, table entry, row.
struct NewRows {
  const uint16_t *k, *v;
  long long stride_b, stride_l, stride_t, stride_h;
  const int32_t *new_tokens;
  int tokens;
};

constexpr int APPEND_FEW = 8;        // rows of a head that one group of 16 lanes takes alone
constexpr int APPEND_ROWS = 64;      // else, rows of a head per workgroup

__device__ __forceinline__ void append_row(const CacheView &C, const NewRows &R, const HeadOf &w, const HeadPlace &p,
                                           int count, int seen, int t, int lane) {
  const long long src = w.b * R.stride_b + w.l * R.stride_l + t * R.stride_t + w.h * R.stride_h + 8 * lane;
  const uint4 k = *reinterpret_cast<const uint4 *>(R.k + src);
  const uint4 v = *reinterpret_cast<const uint4 *>(R.v + src);
  if (t >= C.capacity - count) return;
  const SlotPlace s = slot_place(C, p, count + t);
  if (!page_there(C, s.page)) return;
  const long long dst = row_at(C, p, s) + 8 * lane;
  *reinterpret_cast<uint4 *>(C.k + dst) = k;
  *reinterpret_cast<uint4 *>(C.v + dst) = v;
  if (C.mass != nullptr && lane == 0) {
    const long long at = state_at(C, p, s);
    C.mass[at] = 0.f;
    C.positions[at] = (int)((unsigned)seen + (unsigned)t);
  }
}
__device__ __forceinline__ void append_count(const CacheView &C, const HeadOf &w, int count, int seen, int n) {
  const long long at = count_at(C, w.b, w.l, w.h);
  C.counts[at] = n < C.capacity - count ? count + n : C.capacity;
  if (C.seen != nullptr) C.seen[at] = (int)((unsigned)seen + (unsigned)n);
}

// A group of 16 lanes per head takes all its rows and then moves its counts on.
__global__ __launch_bounds__(256) void append_few_kernel(const CacheView C, const NewRows R) {
  const unsigned g = blockIdx.x * 16u + (threadIdx.x >> 4);
  if (g >= (unsigned)C.nreq * (unsigned)C.layers * (unsigned)C.kv_heads) return;
  const int lane = threadIdx.x & 15;
  const HeadOf w = head_of(C, g);
  const HeadPlace p = head_place(C, w);
  const int n = tokens_new(R.new_tokens, w.b, R.tokens), count = held(C, w.b, w.l, w.h);
  const int seen = C.seen != nullptr ? C.seen[count_at(C, w.b, w.l, w.h)] : 0;
  for (int t = 0; t < n; ++t) append_row(C, R, w, p, count, seen, t, lane);
  if (lane == 0 && n > 0) append_count(C, w, count, seen, n);
}

// A workgroup per APPEND_ROWS rows of a head; where a head has several, another launch moves the counts on.
__global__ __launch_bounds__(256) void append_kernel(const CacheView C, const NewRows R, int parts) {
  const unsigned g = blockIdx.x / (unsigned)parts;
  const int part = (int)(blockIdx.x - g * (unsigned)parts), lane = threadIdx.x & 15;
  const HeadOf w = head_of(C, g);
  const HeadPlace p = head_place(C, w);
  const int n = tokens_new(R.new_tokens, w.b, R.tokens), count = held(C, w.b, w.l, w.h);
  const int seen = C.seen != nullptr ? C.seen[count_at(C, w.b, w.l, w.h)] : 0;
  const int t0 = part * APPEND_ROWS;
#pragma unroll
  for (int i = 0; i < APPEND_ROWS / 16; ++i) {
    const int t = t0 + 16 * i + (int)(threadIdx.x >> 4);
    if (t < n) append_row(C, R, w, p, count, seen, t, lane);
  }
  if (parts == 1) {
    __syncthreads();                   // every wave has read the count
    if (threadIdx.x == 0 && n > 0) append_count(C, w, count, seen, n);
  }
}
__global__ __launch_bounds__(256) void append_counts_kernel(const CacheView C, const NewRows R) {
  const unsigned g = blockIdx.x * 256u + threadIdx.x;
  if (g >= (unsigned)C.nreq * (unsigned)C.layers * (unsigned)C.kv_heads) return;
  const HeadOf w = head_of(C, g);
  const int n = tokens_new(R.new_tokens, w.b, R.tokens);
  const int seen = C.seen != nullptr ? C.seen[count_at(C, w.b, w.l, w.h)] : 0;
  if (n > 0) append_count(C, w, held(C, w.b, w.l, w.h), seen, n);
}

// ------------------------------------------------------------------------------------------ admit
// State of the rows of a compaction, in the order of kept_idx: a selection pool (one head, or the heads of a layer) is
// pool_heads * k_keep entries, ADMIT_ROWS of them per workgroup.
constexpr int ADMIT_ROWS = 1024;

__global__ __launch_bounds__(256) void admit_kernel(const SegTable T, const CacheView C, const int32_t *__restrict__ kept_idx,
                                                    const int32_t *__restrict__ kept_cnt, const float *__restrict__ scores) {
  int seg = 0;
  unsigned local = blockIdx.x, parts = 1;
  for (int i = 0; i < T.nseg; ++i) {
    const int nh = pool_heads(T, T.s[i]);
    parts = (unsigned)(((long long)nh * T.s[i].k_keep + ADMIT_ROWS - 1) / ADMIT_ROWS);
    const unsigned nb = parts * (unsigned)(T.s[i].head_count / nh);
    seg = i;
    if (local < nb || i == T.nseg - 1) break;
    local -= nb;
  }
  const Seg &s = T.s[seg];
  const int nh = pool_heads(T, s), pool = (int)(local / parts), part = (int)(local - (unsigned)pool * parts);
  const int head0 = s.head_begin + pool * nh;              // l * H + h of the pool's first head
  const long long entries = (long long)nh * s.k_keep, first = s.kept_off + (long long)head0 * s.k_keep;
  const int32_t *cnt = kept_cnt + s.ghead0 + head0;
  // what head j of the pool keeps, of the entries that are left
  auto kept = [&](int j, long long left) {
    if (!T.layer_scope) return (long long)s.k_keep;
    const long long c = cnt[j];
    return c < 0 ? 0 : (c < left ? c : left);
  };
  const long long e0 = (long long)part * ADMIT_ROWS, e1 = e0 + ADMIT_ROWS < entries ? e0 + ADMIT_ROWS : entries;
  long long base = 0;                                      // entries of the heads before
  for (int j = 0; j < nh && base < e1; ++j) {
    const long long c = kept(j, entries - base);
    const int l = (head0 + j) / s.H, h = (head0 + j) - l * s.H;
    const HeadOf w{s.req, l, h};
    const HeadPlace p = head_place(C, w);
    const long long room = c < C.capacity ? c : C.capacity;
    const long long lo = e0 > base ? e0 - base : 0, hi = e1 - base < room ? e1 - base : room;
    for (long long i = lo + threadIdx.x; i < hi; i += 256) {
      const int tok = kept_idx[first + base + i];
      const SlotPlace at = slot_place(C, p, (int)i);
      if (!page_there(C, at.page)) continue;
      const long long x = state_at(C, p, at);
      C.positions[x] = tok;
      C.mass[x] = scores != nullptr && tok >= 0 && tok < s.n ? scores[s.score_off + (long long)(head0 + j) * s.n + tok] : 0.f;
    }
    base += c;
  }
  if (part == 0) {
    if (!T.layer_scope) {
      if (threadIdx.x == 0) {
        const int l = head0 / s.H;
        const long long at = count_at(C, s.req, l, head0 - l * s.H);
        C.counts[at] = s.k_keep < C.capacity ? s.k_keep : C.capacity;
        C.seen[at] = s.n;
      }
    } else if (threadIdx.x == 0) {
      long long left = entries;
      for (int j = 0; j < nh; ++j) {
        const long long c = kept(j, left), at = count_at(C, s.req, head0 / s.H, j);
        left -= c;
        C.counts[at] = (int)(c < C.capacity ? c : C.capacity);
        C.seen[at] = s.n;
      }
    }
  }
}

hipError_t launch_cache_admit(const SegTable &T, const CacheView &C, const int32_t *kept_idx, const int32_t *kept_cnt,
                              const float *scores, hipStream_t st) {
  long long nb = 0;
  for (int i = 0; i < T.nseg; ++i) {
    const int nh = pool_heads(T, T.s[i]);
    nb += ((long long)nh * T.s[i].k_keep + ADMIT_ROWS - 1) / ADMIT_ROWS * (T.s[i].head_count / nh);
  }
  if (nb > 0x7fffffffll) return hipErrorInvalidValue;
  hipLaunchKernelGGL(admit_kernel, dim3((unsigned)nb), dim3(256), 0, st, T, C, kept_idx, kept_cnt, scores);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------ evict
// One workgroup per pool (a head, or the heads of a layer) finds the key of the last token that stays, by radix
// selection on an order-preserving key (12, 12 and 8 bits), counts what every head keeps and lists its moves: the holes
// below the new count and the retained tokens from it on, both ascending, as many of the one as of the other.  A second
// launch moves the rows.  Sources and destinations of a head are disjoint, so the moves need no order.
constexpr int EVICT_THREADS = 1024, EVICT_WAVES = EVICT_THREADS / 64;
constexpr uint32_t KEY_PROTECTED = 0xffffffffu;      // above the key of +inf (0xff800000)
constexpr int EVICT_BINS = 4096;

struct EvictPlan {
  int budget;
  const int32_t *budgets;
  int sink, recent;
  int pool_heads;              // 1 or kv_heads
  int most;                    // tokens of a head that the lists have room for
  int list;                    // ints from one head's lists to the next: `list / 2` destinations, then as many sources
  int *lists, *moves;          // moves[head]: how many
};

__device__ __forceinline__ uint32_t evict_key(const CacheView &C, const HeadPlace &p, int slot, const EvictPlan &E,
                                              long long recent_from) {
  const SlotPlace s = slot_place(C, p, slot);
  if (!page_there(C, s.page)) return 0u;
  const long long at = state_at(C, p, s);
  const int pos = C.positions[at];
  if (pos < E.sink || pos >= recent_from) return KEY_PROTECTED;
  return score_key(C.mass[at]);
}

struct EvictLds {
  int hist[EVICT_BINS];
  int wave[3][EVICT_WAVES];
  int bin, above;              // the bin that holds the last of the wanted, and how many lie in higher ones
};

// Sum over the workgroup, and over the waves before this one.
__device__ __forceinline__ int waves_before(const int *per_wave, int wave, int &total) {
  int before = 0;
  total = 0;
  for (int i = 0; i < EVICT_WAVES; ++i) {
    before += i < wave ? per_wave[i] : 0;
    total += per_wave[i];
  }
  return before;
}

__global__ __launch_bounds__(EVICT_THREADS) void evict_rank_kernel(const CacheView C, const EvictPlan E) {
  __shared__ EvictLds L;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int nh = E.pool_heads;
  const unsigned g0 = blockIdx.x * (unsigned)nh;
  const HeadOf w0 = head_of(C, g0);
  const int asked = E.budgets != nullptr ? E.budgets[w0.b] : E.budget;
  const long long want_all = (long long)nh * (asked > 0 ? asked : 0);
  long long total = 0;
  bool too_long = false;
  for (int j = 0; j < nh; ++j) {
    const int c = held(C, w0.b, w0.l, w0.h + j);
    total += c;
    too_long |= c > E.most;
  }
  if (total <= want_all || too_long) {                     // uniform
    for (int j = tid; j < nh; j += EVICT_THREADS) E.moves[g0 + j] = 0;
    return;
  }
  // the key of the last one that stays, and how many of its equals stay
  uint32_t prefix = 0, mask = 0;
  int want = (int)want_all;                                // < total < 2^31
  if (want > 0) {
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 20 : pass == 1 ? 8 : 0, bins = pass == 2 ? 256 : EVICT_BINS;
      for (int i = tid; i < EVICT_BINS; i += EVICT_THREADS) L.hist[i] = 0;
      __syncthreads();
      for (int j = 0; j < nh; ++j) {
        const HeadOf w{w0.b, w0.l, w0.h + j};
        const HeadPlace p = head_place(C, w);
        const int c = held(C, w.b, w.l, w.h);
        const long long from = (long long)C.seen[count_at(C, w.b, w.l, w.h)] - E.recent;
        for (int s = tid; s < c; s += EVICT_THREADS) {
          const uint32_t key = evict_key(C, p, s, E, from);
          if ((key & mask) == prefix) atomicAdd(&L.hist[key >> shift & (uint32_t)(bins - 1)], 1);
        }
      }
      __syncthreads();
      // bins from the top: thread t has bins top - 4 t .. top - 4 t - 3
      int mine[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        mine[i] = L.hist[EVICT_BINS - 1 - (4 * tid + i)];
        sum += mine[i];
      }
      int upto = sum;
      for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(upto, d);
        if (lane >= d) upto += o;
      }
      if (lane == 63) L.wave[0][wave] = upto;
      __syncthreads();
      int all;
      int before = waves_before(L.wave[0], wave, all) + upto - sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (before < want && want <= before + mine[i]) {
          L.bin = EVICT_BINS - 1 - (4 * tid + i);
          L.above = before;
        }
        before += mine[i];
      }
      __syncthreads();
      want -= L.above;
      prefix |= (uint32_t)L.bin << shift;
      mask |= (uint32_t)(bins - 1) << shift;
      __syncthreads();
    }
  }
  const bool none = want_all == 0;
  // head after head: a wave has a run of consecutive slots
  int ties = none ? 0 : want;                              // equals of `prefix` that stay, from here on
  for (int j = 0; j < nh; ++j) {
    const HeadOf w{w0.b, w0.l, w0.h + j};
    const HeadPlace p = head_place(C, w);
    const int c = held(C, w.b, w.l, w.h);
    const long long from = (long long)C.seen[count_at(C, w.b, w.l, w.h)] - E.recent;
    const int run = ((c + EVICT_WAVES - 1) / EVICT_WAVES + 63) / 64 * 64;
    const int s0 = min(wave * run, c), s1 = min(s0 + run, c);
    auto state_of = [&](int s) {                           // 0: goes, 1: equal, 2: stays
      if (s >= s1 || none) return 0;
      const uint32_t key = evict_key(C, p, s, E, from);
      return key > prefix ? 2 : (key == prefix ? 1 : 0);
    };
    int eq = 0, gt = 0;
    for (int s = s0; s < s1; s += 64) {
      const int st = state_of(s + lane);
      eq += __popcll(__ballot(st == 1));
      gt += __popcll(__ballot(st == 2));
    }
    if (lane == 0) {
      L.wave[0][wave] = eq;
      L.wave[1][wave] = gt;
    }
    __syncthreads();
    int eq_all, gt_all;
    const int eq_before = waves_before(L.wave[0], wave, eq_all);
    waves_before(L.wave[1], wave, gt_all);
    const int eq_stay = min(ties, eq_all), left = gt_all + eq_stay;
    __syncthreads();
    // pass 0 counts a wave's holes and late tokens, pass 1 lists them
    int hole_at = 0, late_at = 0;
    for (int pass = 0; pass < 2; ++pass) {
      int eq_seen = eq_before, holes = hole_at, late = late_at;
      for (int s = s0; s < s1; s += 64) {
        const int slot = s + lane, st = state_of(slot);
        const unsigned long long below = (1ull << lane) - 1, eqs = __ballot(st == 1);
        const bool stays = st == 2 || (st == 1 && eq_seen + __popcll(eqs & below) < eq_stay);
        const bool is_hole = slot < s1 && !stays && slot < left, is_late = stays && slot >= left;
        const unsigned long long hs = __ballot(is_hole), ls = __ballot(is_late);
        if (pass == 1) {
          int *list = E.lists + (long long)(g0 + j) * E.list;
          if (is_hole) list[holes + __popcll(hs & below)] = slot;
          if (is_late) list[E.list / 2 + late + __popcll(ls & below)] = slot;
        }
        eq_seen += __popcll(eqs);
        holes += __popcll(hs);
        late += __popcll(ls);
      }
      if (pass == 0) {
        if (lane == 0) {
          L.wave[0][wave] = holes;
          L.wave[1][wave] = late;
        }
        __syncthreads();
        int all;
        late_at = waves_before(L.wave[1], wave, all);
        hole_at = waves_before(L.wave[0], wave, all);
        if (tid == 0) E.moves[g0 + j] = all;
      }
    }
    if (tid == 0) C.counts[count_at(C, w.b, w.l, w.h)] = left;
    ties -= eq_stay;
    __syncthreads();
  }
}

constexpr int MOVE_THREADS = 256;

__global__ __launch_bounds__(MOVE_THREADS) void evict_move_kernel(const CacheView C, const EvictPlan E, int parts) {
  const unsigned g = blockIdx.x / (unsigned)parts;
  const int part = (int)(blockIdx.x - g * (unsigned)parts), lane = threadIdx.x & 15;
  const int moves = E.moves[g];
  const HeadPlace p = head_place(C, head_of(C, g));
  const int *list = E.lists + (long long)g * E.list;
  for (int i = part * (MOVE_THREADS / 16) + (int)(threadIdx.x >> 4); i < moves; i += parts * (MOVE_THREADS / 16)) {
    const SlotPlace to = slot_place(C, p, list[i]), from = slot_place(C, p, list[E.list / 2 + i]);
    if (!page_there(C, to.page) || !page_there(C, from.page)) continue;
    const long long src = row_at(C, p, from) + 8 * lane, dst = row_at(C, p, to) + 8 * lane;
    const uint4 k = *reinterpret_cast<const uint4 *>(C.k + src);
    const uint4 v = *reinterpret_cast<const uint4 *>(C.v + src);
    *reinterpret_cast<uint4 *>(C.k + dst) = k;
    *reinterpret_cast<uint4 *>(C.v + dst) = v;
    if (lane == 0) {
      const long long a = state_at(C, p, from), z = state_at(C, p, to);
      C.mass[z] = C.mass[a];
      C.positions[z] = C.positions[a];
    }
  }
}

// Lists of a head: it moves at most half of its tokens (one into a slot that another left).
static int evict_list_ints(int most) { return 2 * (most / 2 + 1); }

static size_t evict_bytes(const CacheView &C, int most) {
  const size_t heads = (size_t)C.nreq * C.layers * C.kv_heads;
  return (heads * ((size_t)evict_list_ints(most) + 1) * sizeof(int) + 255) / 256 * 256;
}

static int evict_most(const CacheView &C, const compactor_cache_evict_params_t *e) {
  return e->max_tokens > 0 && e->max_tokens < C.capacity ? e->max_tokens : C.capacity;
}

static int evict_check(const compactor_cache_evict_params_t *e, const CacheView &C) {
  if (!e) return COMPACTOR_EINVAL;
  if (e->sink < 0 || e->recent < 0 || e->max_tokens < 0) return COMPACTOR_EINVAL;
  if (e->scope != COMPACTOR_SCOPE_HEAD && e->scope != COMPACTOR_SCOPE_LAYER) return COMPACTOR_EINVAL;
  if (e->scope == COMPACTOR_SCOPE_LAYER && (long long)C.capacity * C.kv_heads > 0x7fffffffll - 64) return COMPACTOR_EINVAL;
  return COMPACTOR_OK;
}

}  // namespace cmp

using namespace cmp;

extern "C" {
#pragma GCC visibility push(default)

int compactor_cache_append(const compactor_cache_t *cache, const compactor_cache_rows_t *rows, void *stream) {
  CacheView C;
  const int rc = cache_view(cache, CACHE_ROWS, &C);
  if (rc) return rc;
  if (!rows || !rows->k || !rows->v || rows->tokens < 1) return COMPACTOR_EINVAL;
  if (rows->stride_b < 0 || rows->stride_l < 0 || rows->stride_t < 0 || rows->stride_h < 0) return COMPACTOR_EINVAL;
  if (((reinterpret_cast<uintptr_t>(rows->k) | reinterpret_cast<uintptr_t>(rows->v)) & 15u) ||
      ((rows->stride_b | rows->stride_l | rows->stride_t | rows->stride_h) & 7) ||
      (reinterpret_cast<uintptr_t>(rows->new_tokens) & 3u))
    return COMPACTOR_EALIGN;
  NewRows R{static_cast<const uint16_t *>(rows->k), static_cast<const uint16_t *>(rows->v), rows->stride_b,
            rows->stride_l, rows->stride_t, rows->stride_h, rows->new_tokens, rows->tokens};
  const long long heads = (long long)C.nreq * C.layers * C.kv_heads;
  const int parts = (int)(((long long)R.tokens + APPEND_ROWS - 1) / APPEND_ROWS);
  if (R.tokens > APPEND_FEW && heads * parts > 0x7fffffffll) return COMPACTOR_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();   // a leftover of earlier, unrelated HIP calls is not this call's error
  if (R.tokens <= APPEND_FEW) {
    hipLaunchKernelGGL(append_few_kernel, dim3((unsigned)((heads + 15) / 16)), dim3(256), 0, st, C, R);
  } else {
    hipLaunchKernelGGL(append_kernel, dim3((unsigned)(heads * parts)), dim3(256), 0, st, C, R, parts);
    if (parts > 1) {
      if (hipGetLastError() != hipSuccess) return COMPACTOR_EHIP;
      hipLaunchKernelGGL(append_counts_kernel, dim3((unsigned)((heads + 255) / 256)), dim3(256), 0, st, C, R);
    }
  }
  return hipGetLastError() == hipSuccess ? COMPACTOR_OK : COMPACTOR_EHIP;
}

int compactor_cache_evict_workspace_size(const compactor_cache_t *cache, const compactor_cache_evict_params_t *evict,
                                         size_t *bytes) {
  CacheView C;
  int rc = cache_view(cache, CACHE_SIZES, &C);
  if (rc) return rc;
  rc = evict_check(evict, C);
  if (rc) return rc;
  if (!bytes) return COMPACTOR_EINVAL;
  *bytes = evict_bytes(C, evict_most(C, evict));
  return COMPACTOR_OK;
}

int compactor_cache_evict(const compactor_cache_t *cache, const compactor_cache_evict_params_t *evict,
                          void *workspace, size_t workspace_bytes, void *stream) {
  CacheView C;
  int rc = cache_view(cache, CACHE_STATE, &C);
  if (rc) return rc;
  rc = evict_check(evict, C);
  if (rc) return rc;
  if (!evict->budgets && evict->budget < 0) return COMPACTOR_EINVAL;
  if (reinterpret_cast<uintptr_t>(evict->budgets) & 3u) return COMPACTOR_EALIGN;
  EvictPlan E;
  E.budget = evict->budget; E.budgets = evict->budgets;
  E.sink = evict->sink; E.recent = evict->recent;
  E.pool_heads = evict->scope == COMPACTOR_SCOPE_LAYER ? C.kv_heads : 1;
  E.most = evict_most(C, evict);
  E.list = evict_list_ints(E.most);
  if (!workspace || workspace_bytes < evict_bytes(C, E.most)) return COMPACTOR_EWORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return COMPACTOR_EALIGN;
  const long long heads = (long long)C.nreq * C.layers * C.kv_heads;
  E.moves = static_cast<int *>(workspace);
  E.lists = E.moves + heads;
  long long parts = 2048 / heads;
  parts = parts < 1 ? 1 : (parts > 128 ? 128 : parts);
  if (heads * parts > 0x7fffffffll) return COMPACTOR_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  hipLaunchKernelGGL(evict_rank_kernel, dim3((unsigned)(heads / E.pool_heads)), dim3(EVICT_THREADS), 0, st, C, E);
  if (hipGetLastError() != hipSuccess) return COMPACTOR_EHIP;
  hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)(heads * parts)), dim3(MOVE_THREADS), 0, st, C, E, (int)parts);
  return hipGetLastError() == hipSuccess ? COMPACTOR_OK : COMPACTOR_EHIP;
}

#pragma GCC visibility pop
}  // extern "C"
