// Serving from a paged cache: rows in (append), rows out (eviction by accumulated attention weight), and the start
// of it, the state of rows that a compaction has written (admit).  The attention itself: cache_attention.hip.
#include <string.h>

#include <algorithm>

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
  // (half a TB of rows of one head; sums of a slot and a launch's steps, and a tile's end, then fit)
  if ((long long)c->table_len * p.page_size > 1ll << 30) return COMPACTOR_EINVAL;
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
  invariant_divisor(p.page_size, &v.div_mul, &v.div_shift);
  invariant_divisor(c->layers * c->kv_heads, &v.req_mul, &v.req_shift);
  invariant_divisor(c->kv_heads, &v.layer_mul, &v.layer_shift);
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
// pool_heads * k_keep entries, ADMIT_ROWS of them per workgroup.  Bound by the latency of the chain index, score (table entry): a
// thread's four entries leave together.
constexpr int ADMIT_ROWS = 1024;

// Entries [lo, hi) of a head's list, at most ADMIT_ROWS of them.
__device__ __forceinline__ void admit_rows(const CacheView &C, const HeadPlace &p, const int32_t *kept_idx, const float *scores, int n, int lo, int hi) {
  constexpr int N = ADMIT_ROWS / 256;
  int tok[N], page[N], at[N];
  float mass[N];
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const int i = min(lo + 256 * u + (int)threadIdx.x, hi - 1);
    tok[u] = kept_idx[i];
    const SlotPlace s = slot_place(C, p, i);
    page[u] = s.page;
    at[u] = s.at;
  }
#pragma unroll
  for (int u = 0; u < N; ++u) mass[u] = scores != nullptr && (unsigned)tok[u] < (unsigned)n ? scores[tok[u]] : 0.f;
#pragma unroll
  for (int u = 0; u < N; ++u)
    if (lo + 256 * u + (int)threadIdx.x < hi && page_there(C, page[u])) {
      const long long x = state_at(C, p, SlotPlace{page[u], at[u]});
      C.positions[x] = tok[u];
      C.mass[x] = mass[u];
    }
}

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
  const int nh = pool_heads(T, s), pool = (int)(local / parts), part = (int)(local - (unsigned)pool * parts), lane = threadIdx.x & 63;
  const int head0 = s.head_begin + pool * nh, layer = head0 / s.H;       // l * H + h of the pool's first head
  const long long entries = (long long)nh * s.k_keep, first = s.kept_off + (long long)head0 * s.k_keep;
  const long long e0 = (long long)part * ADMIT_ROWS, e1 = e0 + ADMIT_ROWS < entries ? e0 + ADMIT_ROWS : entries;
  auto head = [&](int j, long long base, long long kept) {             // the pool's j-th head has entries [base, base + kept); uniform
    const HeadOf w{s.req, layer, head0 + j - layer * s.H};
    const int room = (int)(kept < C.capacity ? kept : C.capacity);
    const int lo = (int)(e0 > base ? e0 - base : 0), hi = (int)(e1 - base < room ? e1 - base : room);
    if (lo < hi)
      admit_rows(C, head_place(C, w), kept_idx + first + base,
                 scores == nullptr ? nullptr : scores + s.score_off + (long long)(head0 + j) * s.n, s.n, lo, hi);
  };
  auto note = [&](int j, long long kept) {
    const long long at = count_at(C, s.req, layer, head0 + j - layer * s.H);
    C.counts[at] = (int)(kept < C.capacity ? kept : C.capacity);
    C.seen[at] = s.n;
  };
  if (!T.layer_scope) {
    head(0, 0, s.k_keep);
    if (part == 0 && threadIdx.x == 0) note(0, s.k_keep);
    return;
  }
  // 64 heads at a time: a lane has one, and where its entries begin (a count that does not fit the layer's entries is cut to them)
  long long before = 0;
  for (int j0 = 0; j0 < nh && (before < e1 || part == 0); j0 += 64) {
    const int c = j0 + lane < nh ? kept_cnt[s.ghead0 + head0 + j0 + lane] : 0;
    long long upto = c < 0 ? 0 : c;
    for (int d = 1; d < 64; d <<= 1) {
      const long long o = __shfl_up(upto, d);
      if (lane >= d) upto += o;
    }
    upto = before + upto < entries ? before + upto : entries;
    long long base = __shfl_up(upto, 1);
    if (lane == 0) base = before;
    if (part == 0 && threadIdx.x < 64 && j0 + lane < nh) note(j0 + lane, upto - base);
    for (unsigned long long mine = __ballot(base < e1 && upto > e0 && j0 + lane < nh); mine != 0; mine &= mine - 1) {
      const int at = __builtin_ctzll(mine);
      const long long b = __shfl(base, at);
      head(j0 + at, b, __shfl(upto, at) - b);
    }
    before = __shfl(upto, 63);
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
// The slots of a pool (a head, or the heads of a layer) are ranked by an order-preserving 32-bit key; the key of the last one
// that stays and how many of its equals stay (the first ones) is all that the rest needs.  A head that keeps `left` of its
// tokens moves those in slots from `left` on into the holes below.  Both come out in order from the number `before` of retained
// tokens in front of a slot: slot s is hole number s - before, and the retained token in slot s >= left has left - 1 - before
// others behind it.  Sources and destinations of a head are disjoint, so the moves need no order.
//
// One workgroup does everything where a pool has up to 256 units of 64 slots (a head of 16384 tokens, 8 heads of 2048); its keys stay in
// registers.  More would keep one compute unit busy too long, so there the pool is cut into parts of PART_SLOTS slots and every part's
// workgroup does the same steps in a launch each: keys and the tally of their first 12 bits, the next 12, the last 8, the lists,
// the moves (us with the append in front, one workgroup / parts: one layer of 8 heads of 1700 tokens 26 / 33, 512 such layers 66 / 151).
// What bounds both is not the 8 bytes of state a slot but the chain of steps and the instructions of each: a compute unit issues
// one scalar instruction a cycle, and one vector instruction, for all its waves, and fetches what it runs for the first time (lists of 10 units a
// wave: 5.1 us, run a second time 2.9).  Parts of 8 waves with 8 units each: 8 heads of 26215
// tokens 35 us, 32 layers of 79000 tokens 52 (when the three were compared 36 and 57; 4 with 16 41 and 60, 16 with 4 35 and 71).
constexpr uint32_t KEY_PROTECTED = 0xffffffffu;      // above the key of +inf (0xff800000)
constexpr uint32_t KEY_NO_NUMBER = 2u;               // NaN; below the key of -inf (0x007fffff)
constexpr uint32_t KEY_NOT_THERE = 1u;               // the token's page is not there.  0: no token

struct EvictPlan {
  int budget;
  const int32_t *budgets;
  int sink, recent;
  int pool_heads;              // 1 or kv_heads
  int most;                    // tokens of a head that the launches reach
  // parts
  int parts;                   // of a head, at most
  unsigned parts_mul, parts_shift;        // workgroup / parts
  long long pitch;             // ints from one head's keys to the next
  int list;                    // and its lists: `list / 2` destinations, then as many sources
  int *hist1, *hist2, *hist3;  // [pool][4096], [pool][256]: tallies of the first, the next 12 and the last 8 bits
  int *moves;                  // [head]: how many
  int *left;                   // [head]: the new count, -1 where nothing changes
  int2 *state1, *state2;       // [pool]: 12 and 24 bits of the key, and how many of those that begin so stay
  int *above;                  // [head][part]: keys that begin with more
  int *last;                   // [head][part][256]: a part's own tally of the last 8 bits
  uint32_t *keys;
  int *lists;
};

__device__ __forceinline__ long long evict_budget(const EvictPlan &E, int b) {
  const int asked = E.budgets != nullptr ? E.budgets[b] : E.budget;
  return (long long)E.pool_heads * (asked > 0 ? asked : 0);
}

// The first position that is protected as recent (an int: positions are).
__device__ __forceinline__ int recent_from(const EvictPlan &E, int seen) {
  const long long from = (long long)seen - E.recent;
  return from < -0x80000000ll ? (int)-0x80000000ll : (int)from;
}

// Keys of the 64 slots from first + 64 i on, i < N, one a lane; 0 where there is no token.  count > 0.  `units`, uniform, of them hold
// any.  All table entries leave before the first is waited for, and so do the states.  Four units at a time and the last token's slot
// for what lies behind: code that runs once costs what its fetch takes.
template <int N>
__device__ __forceinline__ void evict_keys(const CacheView &C, const HeadPlace &p, const EvictPlan &E, int first, int units, int count, int recent,
                                           uint32_t (&key)[N]) {
  const int lane = threadIdx.x & 63;
  int page[N], at[N], pos[N];
  float mass[N];
#pragma unroll
  for (int i0 = 0; i0 < N; i0 += 4)
    if (i0 < units)
#pragma unroll
      for (int i = i0; i < i0 + 4; ++i) {
        const int slot = min(first + 64 * i + lane, count - 1), q = invariant_quotient((unsigned)slot, C.div_mul, C.div_shift);
        page[i] = p.table[(unsigned)q];
        at[i] = slot - q * C.page_size;
      }
#pragma unroll
  for (int i0 = 0; i0 < N; i0 += 4)
    if (i0 < units)
#pragma unroll
      for (int i = i0; i < i0 + 4; ++i) {
        const long long x = (page_there(C, page[i]) ? page[i] : 0) * C.state_page_stride + p.state + at[i];
        mass[i] = C.mass[x];
        pos[i] = C.positions[x];
      }
#pragma unroll
  for (int i0 = 0; i0 < N; i0 += 4) {
#pragma unroll
    for (int i = i0; i < i0 + 4; ++i) key[i] = 0u;
    if (i0 < units)
#pragma unroll
      for (int i = i0; i < i0 + 4; ++i) {
        const uint32_t rank = pos[i] < E.sink || pos[i] >= recent ? KEY_PROTECTED : score_key(mass[i]);
        key[i] = first + 64 * i + lane < count ? (page_there(C, page[i]) ? max(rank, KEY_NO_NUMBER) : KEY_NOT_THERE) : 0u;
      }
  }
}

// Sum of the waves before this one, and of all.
template <int WAVES>
__device__ __forceinline__ int waves_before(const int *per_wave, int wave, int &total) {
  const int upto = wave_scan((int)(threadIdx.x & 63) < WAVES ? per_wave[threadIdx.x & (WAVES - 1)] : 0);
  total = __builtin_amdgcn_readlane(upto, WAVES - 1);
  return wave == 0 ? 0 : __builtin_amdgcn_readlane(upto, wave - 1);
}

// Equals of `last` and larger ones among a wave's keys.  (last is some token's key, so never 0.)
template <int N>
__device__ __forceinline__ void count_keys(const uint32_t (&key)[N], int units, uint32_t last, int &equal, int &more) {
  equal = more = 0;
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i < units) {
      equal += __popcll(__ballot(key[i] == last));
      more += __popcll(__ballot(key[i] > last));
    }
}

__device__ __forceinline__ int lanes_before(unsigned long long mask, int start) {       // start + ones below the lane
  return (int)__builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, (unsigned)start));
}

// Which lanes' tokens stay, where `room` more equals may.
__device__ __forceinline__ unsigned long long who_stays(uint32_t key, uint32_t last, int room, int &equals) {
  const unsigned long long eqs = __ballot(key == last);
  unsigned long long stay = __ballot(key > last);
  equals = __popcll(eqs);
  if (equals <= room) stay |= eqs;
  else if (room > 0) stay |= eqs & __ballot(lanes_before(eqs, 0) < room);
  return stay;
}

// The places of a unit's tokens in the lists of their head: `before` of those that stay lie in front of it, `left` stay in all.  -> retained
// tokens in slots from `left` on.  (Scalar instructions count: a compute unit issues one a cycle for all its waves.)
__device__ __forceinline__ int list_unit(unsigned long long stay, int base, int before, int left, int *holes, int *late) {
  const int slot = base + (int)(threadIdx.x & 63), in_front = lanes_before(stay, before);
  if (base + 64 <= left) {
    if (__builtin_amdgcn_inverse_ballot_w64(~stay)) holes[slot - in_front] = slot;
    return 0;
  }
  const unsigned long long low = base < left ? (1ull << (left - base)) - 1 : 0ull;
  if (__builtin_amdgcn_inverse_ballot_w64(low & ~stay)) holes[slot - in_front] = slot;
  if (__builtin_amdgcn_inverse_ballot_w64(stay & ~low)) late[left - 1 - in_front] = slot;
  return __popcll(stay & ~low);
}

// A wave's units: `equal` equals and `more` larger ones lie in front of the wave, `ties` equals stay.
template <int N>
__device__ __forceinline__ int list_keys(const uint32_t (&key)[N], int first, int units, uint32_t last, int equal, int more, int ties, int left, int *holes,
                                         int *late) {
  int before = more + min(equal, ties), moves = 0;
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i < units) {
      int n;
      const unsigned long long stay = who_stays(key[i], last, ties - equal, n);
      moves += list_unit(stay, first + 64 * i, before, left, holes, late);
      equal += n;
      before += __popcll(stay);
    }
  return moves;
}

// The bin of hist[BINS] in which the want-th largest lies, and how many lie in higher ones; by all THREADS.  per_wave and found: LDS.
template <int BINS, int THREADS>
__device__ __forceinline__ void find_bin(const int *hist, int want, int *per_wave, int *found) {
  constexpr int EACH = (BINS + THREADS - 1) / THREADS;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int mine[EACH], sum = 0;
  if constexpr (EACH % 4 == 0) {
#pragma unroll
    for (int i = 0; i < EACH; i += 4) {
      const int4 x = *reinterpret_cast<const int4 *>(hist + BINS - 4 - (EACH * tid + i));
      mine[i] = x.w;
      mine[i + 1] = x.z;
      mine[i + 2] = x.y;
      mine[i + 3] = x.x;
    }
  } else {
#pragma unroll
    for (int i = 0; i < EACH; ++i) mine[i] = EACH * tid + i < BINS ? hist[BINS - 1 - (EACH * tid + i)] : 0;
  }
#pragma unroll
  for (int i = 0; i < EACH; ++i) sum += mine[i];
  const int upto = wave_scan(sum);
  if (lane == 63) per_wave[wave] = upto;
  __syncthreads();
  int all;
  int before = waves_before<THREADS / 64>(per_wave, wave, all) + upto - sum;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    if (before < want && want <= before + mine[i]) {
      found[0] = BINS - 1 - (EACH * tid + i);
      found[1] = before;
      found[2] = mine[i];
    }
    before += mine[i];
  }
  __syncthreads();
}

// Moves one row, its state with it, by 16 lanes.
__device__ __forceinline__ void move_row(const CacheView &C, const HeadPlace &p, int to, int from, int lane) {
  const SlotPlace z = slot_place(C, p, to), a = slot_place(C, p, from);
  if (!page_there(C, z.page) || !page_there(C, a.page)) return;
  const long long src = row_at(C, p, a) + 8 * lane, dst = row_at(C, p, z) + 8 * lane;
  const uint4 k = *reinterpret_cast<const uint4 *>(C.k + src);
  const uint4 v = *reinterpret_cast<const uint4 *>(C.v + src);
  *reinterpret_cast<uint4 *>(C.k + dst) = k;
  *reinterpret_cast<uint4 *>(C.v + dst) = v;
  if (lane == 0) {
    const long long x = state_at(C, p, a), y = state_at(C, p, z);
    C.mass[y] = C.mass[x];
    C.positions[y] = C.positions[x];
  }
}

// ---- one workgroup a head
constexpr int ALONE_THREADS = 1024, ALONE_WAVES = ALONE_THREADS / 64, ALONE_UNITS = 16;
constexpr int ALONE_SLOTS = ALONE_WAVES * ALONE_UNITS * 64;
constexpr int ALONE_BINS = 4096, ALONE_CANDS = 256;

struct AloneLds {
  alignas(16) int hist[ALONE_BINS];
  int late[ALONE_SLOTS / 2 + 1], holes[ALONE_SLOTS / 2 + 1];
  uint32_t cand[ALONE_CANDS];
  int wave[3][ALONE_WAVES];
  uint32_t top[2][ALONE_WAVES];
  int found[3], cands, moves;
  uint32_t key;
  int ties;
};

__device__ __forceinline__ void clear_hist(int (&hist)[ALONE_BINS]) {
  reinterpret_cast<int4 *>(hist)[threadIdx.x] = make_int4(0, 0, 0, 0);
}
static_assert(ALONE_BINS == 4 * ALONE_THREADS, "one store clears the tally");

// Key of the last token that stays: its bin among 4096 of equal width between the least and the largest key that are neither
// protected nor such as are ranked behind all, so that bins are even whatever the weights' range; then among the few keys of the bin, or 4096 bins within it.
// units of the wave hold keys, `left` tokens stay; L.hist is clear.  -> key of the last one that stays, and how many of its equals stay
__device__ __forceinline__ void find_last(AloneLds &L, const uint32_t (&key)[ALONE_UNITS], int units, int left, uint32_t &last, int &ties) {
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  int both = 0;                                            // protected tokens, and 2^16 times plain ones
  uint32_t most = 0, least = 0;                            // least: as ~key
#pragma unroll
  for (int i = 0; i < ALONE_UNITS; ++i)
    if (i < units) {
      const bool plain = key[i] > KEY_NO_NUMBER && key[i] != KEY_PROTECTED;
      both += plain ? 1 << 16 : (key[i] == KEY_PROTECTED ? 1 : 0);
      most = max(most, plain ? key[i] : 0u);
      least = max(least, plain ? ~key[i] : 0u);
    }
  both = wave_scan(both);
  most = wave_max_up(most);
  least = wave_max_up(least);
  if (lane == 63) {
    L.wave[0][wave] = both;
    L.top[0][wave] = most;
    L.top[1][wave] = least;
  }
  if (tid == 0) L.moves = 0;
  __syncthreads();
  waves_before<ALONE_WAVES>(L.wave[0], wave, both);
  const int kept = both & 0xffff, plain = both >> 16;
  most = __builtin_amdgcn_readlane(wave_max_up(L.top[0][lane & (ALONE_WAVES - 1)]), 63);
  least = __builtin_amdgcn_readlane(wave_max_up(L.top[1][lane & (ALONE_WAVES - 1)]), 63);
  if (left <= kept) {
    last = KEY_PROTECTED;
    ties = left;
  } else if (left - kept > plain) {
    int numberless = 0;                                    // all of those stay before a token that is not there does
#pragma unroll
    for (int i = 0; i < ALONE_UNITS; ++i)
      if (i < units) numberless += __popcll(__ballot(key[i] == KEY_NO_NUMBER));
    if (lane == 0) L.wave[2][wave] = numberless;
    __syncthreads();
    waves_before<ALONE_WAVES>(L.wave[2], wave, numberless);
    ties = left - kept - plain;
    last = ties <= numberless ? KEY_NO_NUMBER : KEY_NOT_THERE;
    if (ties > numberless) ties -= numberless;
  } else {
    uint32_t lo = ~least, hi = most;
    int want = left - kept;
    bool again = false;
    for (;;) {
      const int shift = hi - lo < (uint32_t)ALONE_BINS ? 0 : 32 - __builtin_clz((hi - lo) / ALONE_BINS);
      if (tid == 0) L.cands = 0;
      if (again) {
        clear_hist(L.hist);
        __syncthreads();
      }
      again = true;
#pragma unroll
      for (int i = 0; i < ALONE_UNITS; ++i)
        if (i < units && key[i] >= lo && key[i] <= hi) atomicAdd(&L.hist[(key[i] - lo) >> shift], 1);
      __syncthreads();
      find_bin<ALONE_BINS, ALONE_THREADS>(L.hist, want, L.wave[2], L.found);
      const int bin = L.found[0], in_bin = L.found[2];
      want -= L.found[1];
      lo += (uint32_t)bin << shift;
      const uint32_t end = lo + ((1u << shift) - 1u);
      hi = end < hi ? end : hi;
      if (shift == 0) {
        last = lo;
        ties = want;
        break;
      }
      if (in_bin <= ALONE_CANDS) {
#pragma unroll
        for (int i = 0; i < ALONE_UNITS; ++i)
          if (i < units && key[i] >= lo && key[i] <= hi) L.cand[atomicAdd(&L.cands, 1)] = key[i];
        __syncthreads();
        if (tid < in_bin) {
          const uint32_t mine = L.cand[tid];
          int more = 0, same = 0;
          for (int i = 0; i < in_bin; ++i) {
            const uint32_t o = L.cand[i];
            more += o > mine;
            same += o == mine;
          }
          if (more < want && want <= more + same) {        // equal candidates write the same
            L.key = mine;
            L.ties = want - more;
          }
        }
        __syncthreads();
        last = L.key;
        ties = L.ties;
        break;
      }
      __syncthreads();                                     // found has been read
    }
  }

}

__global__ __launch_bounds__(ALONE_THREADS) void evict_alone_kernel(const CacheView C, const EvictPlan E) {
  __shared__ AloneLds L;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const HeadOf w = head_of(C, blockIdx.x);
  const HeadPlace p = head_place(C, w);
  const long long here = count_at(C, w.b, w.l, w.h);
  const int seen = C.seen[here], c = clamp_to(C.counts[here], C.capacity);        // (leave together, with the budget)
  const long long budget = evict_budget(E, w.b);
  if (c <= budget || c > E.most) return;                   // uniform
  const int left = (int)budget;
  const int units = ((c + 63) / 64 + ALONE_WAVES - 1) / ALONE_WAVES, first = wave * units * 64;       // of every wave
  uint32_t key[ALONE_UNITS];
  clear_hist(L.hist);                                      // while the keys come
  evict_keys(C, p, E, first, units, c, recent_from(E, seen), key);

  uint32_t last;
  int ties;
  find_last(L, key, units, left, last, ties);
  int equal, more, all;
  count_keys(key, units, last, equal, more);
  if (lane == 0) L.wave[1][wave] = equal | more << 16;     // (a wave may still read wave[0])
  __syncthreads();
  const int front = waves_before<ALONE_WAVES>(L.wave[1], wave, all);
  const int late = list_keys(key, first, units, last, front & 0xffff, front >> 16, ties, left, L.holes, L.late);
  if (lane == 0 && late > 0) atomicAdd(&L.moves, late);
  __syncthreads();
  const int moves = L.moves;
  if (tid == 0) C.counts[here] = left;
  for (int i = tid >> 4; i < moves; i += ALONE_THREADS / 16) move_row(C, p, L.holes[i], L.late[moves - 1 - i], tid & 15);
}

// The same for the heads of a layer that share a budget: units of 64 slots, head after head, in equal numbers to the waves.
constexpr int POOL_UNITS = ALONE_WAVES * ALONE_UNITS;
struct PoolLds {
  AloneLds a;
  alignas(16) int before[POOL_UNITS + 4];                  // retained tokens of a unit; then, of all units before it
  int start[POOL_UNITS + 1], count[POOL_UNITS], seen[POOL_UNITS];        // of a head: its first unit, tokens now and ever
  int moves[POOL_UNITS], first_move[POOL_UNITS + 1];
};

__global__ __launch_bounds__(ALONE_THREADS) void evict_pool_kernel(const CacheView C, const EvictPlan E) {
  __shared__ PoolLds L;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, H = C.kv_heads;
  const HeadOf w0 = head_of(C, blockIdx.x * (unsigned)H);
  const long long budget = evict_budget(E, w0.b);
  int total = 0, longest = 0, units_all = 0;               // (every wave for itself)
  for (int h0 = 0; h0 < H; h0 += 64) {
    const int h = min(h0 + lane, H - 1);
    const long long at = count_at(C, w0.b, w0.l, h);
    const int seen = C.seen[at], c = h0 + lane < H ? clamp_to(C.counts[at], C.capacity) : 0;
    const int mine = (int)(((unsigned)c + 63) / 64), upto = units_all + wave_scan(min(mine, POOL_UNITS));
    total += __builtin_amdgcn_readlane(wave_scan(c), 63);
    longest = max(longest, (int)__builtin_amdgcn_readlane(wave_max_up((unsigned)c), 63));
    if (wave == 0 && h0 + lane < H) {
      L.start[h] = upto - mine;
      L.count[h] = c;
      L.seen[h] = seen;
      L.moves[h] = 0;
    }
    units_all = __builtin_amdgcn_readlane(upto, 63);
  }
  if (total <= budget || longest > E.most) return;         // uniform; from here on the units fit (the host has seen to it)
  if (tid == 0) L.start[H] = units_all;
  clear_hist(L.a.hist);
  __syncthreads();
  const int units = (units_all + ALONE_WAVES - 1) / ALONE_WAVES, unit0 = wave * units;
  // lane i: unit i of the wave
  const int mine = unit0 + lane;
  int head = 0;
  for (int h = 1; h < H; ++h) head += L.start[h] <= mine;
  const bool there = lane < units && mine < units_all;
  const int unit_count = there ? L.count[head] : 0, unit_base = there ? 64 * (mine - L.start[head]) : 0, unit_recent = recent_from(E, L.seen[head]);
  auto base = [&](int i) { return (int)__builtin_amdgcn_readlane(unit_base, i); };
  auto count = [&](int i) { return (int)__builtin_amdgcn_readlane(unit_count, i); };
  auto head_at = [&](int i) { return (int)__builtin_amdgcn_readlane(head, i); };

  uint32_t key[ALONE_UNITS];
  {
    const HeadPlace p = head_place(C, w0);
    int page[ALONE_UNITS], at[ALONE_UNITS], pos[ALONE_UNITS];
    float mass[ALONE_UNITS];
#pragma unroll
    for (int i = 0; i < ALONE_UNITS; ++i)
      if (i < units) {
        const int slot = max(min(base(i) + lane, count(i) - 1), 0), q = invariant_quotient((unsigned)slot, C.div_mul, C.div_shift);
        page[i] = p.table[(unsigned)q];
        at[i] = slot - q * C.page_size;
      }
#pragma unroll
    for (int i = 0; i < ALONE_UNITS; ++i)
      if (i < units) {
        const long long x = (page_there(C, page[i]) ? page[i] : 0) * C.state_page_stride + p.state + head_at(i) * C.state_head_stride + at[i];
        mass[i] = C.mass[x];
        pos[i] = C.positions[x];
      }
#pragma unroll
    for (int i = 0; i < ALONE_UNITS; ++i) {
      key[i] = 0u;
      if (i < units) {
        const uint32_t rank = pos[i] < E.sink || pos[i] >= (int)__builtin_amdgcn_readlane(unit_recent, i) ? KEY_PROTECTED : score_key(mass[i]);
        key[i] = base(i) + lane < count(i) ? (page_there(C, page[i]) ? max(rank, KEY_NO_NUMBER) : KEY_NOT_THERE) : 0u;
      }
    }
  }
  uint32_t last;
  int ties;
  find_last(L.a, key, units, (int)budget, last, ties);

  // equals in front, over all heads; then which slots of a unit stay
  int equal, more, all;
  count_keys(key, units, last, equal, more);
  if (lane == 0) L.a.wave[1][wave] = equal;
  __syncthreads();
  equal = waves_before<ALONE_WAVES>(L.a.wave[1], wave, all);
  unsigned long long unit_stay = 0ull;                     // lane i: of unit i
#pragma unroll
  for (int i = 0; i < ALONE_UNITS; ++i)
    if (i < units) {
      int n;
      const unsigned long long stay = who_stays(key[i], last, ties - equal, n);
      equal += n;
      if (lane == i) unit_stay = stay;
    }
  if (lane < units) L.before[mine] = __popcll(unit_stay);
  for (int u = units * ALONE_WAVES + tid; u < POOL_UNITS; u += ALONE_THREADS) L.before[u] = 0;
  __syncthreads();
  if (wave == 0) {                                         // sums over the units before each
    int4 x = *reinterpret_cast<const int4 *>(&L.before[4 * lane]);
    const int four = x.x + x.y + x.z + x.w, upto = wave_scan(four), b = upto - four;
    *reinterpret_cast<int4 *>(&L.before[4 * lane]) = make_int4(b, b + x.x, b + x.x + x.y, b + x.x + x.y + x.z);
    if (lane == 63) L.before[POOL_UNITS] = upto;
  }
  __syncthreads();
  // A head's lists have half as many places as its units have slots: it moves at most half of its tokens.  Lane i again has unit i of the wave.
  const int first_unit = L.start[head], front = L.before[first_unit], unit_left = L.before[L.start[head + 1]] - front;
  const int unit_front = L.before[min(mine, POOL_UNITS - 1)] - front;
#pragma unroll 1
  for (int i = 0; i < units; ++i) {
    const unsigned lo = __builtin_amdgcn_readlane((unsigned)unit_stay, i), hi = __builtin_amdgcn_readlane((unsigned)(unit_stay >> 32), i);
    const int list = 32 * __builtin_amdgcn_readlane(first_unit, i);
    if (unit0 + i >= units_all) break;
    const int late = list_unit((unsigned long long)hi << 32 | lo, base(i), __builtin_amdgcn_readlane(unit_front, i), __builtin_amdgcn_readlane(unit_left, i),
                               L.a.holes + list, L.a.late + list);
    if (lane == 0 && late > 0) atomicAdd(&L.moves[head_at(i)], late);
  }
  __syncthreads();
  int moves = 0;
  for (int h0 = 0; h0 < H; h0 += 64) {
    const int h = h0 + lane, n = h < H ? L.moves[h] : 0, upto = moves + wave_scan(n);
    if (wave == 0 && h < H) {
      L.first_move[h] = upto - n;
      C.counts[count_at(C, w0.b, w0.l, h)] = L.before[L.start[h + 1]] - L.before[L.start[h]];
    }
    moves = __builtin_amdgcn_readlane(upto, 63);
  }
  if (tid == 0) L.first_move[H] = moves;
  __syncthreads();
  int h = 0;
  for (int i = tid >> 4; i < moves; i += ALONE_THREADS / 16) {
    while (L.first_move[h + 1] <= i) ++h;                  // (first_move[H] > i)
    const int k = i - L.first_move[h], list = 32 * L.start[h];
    move_row(C, head_place(C, HeadOf{w0.b, w0.l, h}), L.a.holes[list + k], L.a.late[list + L.moves[h] - 1 - k], tid & 15);
  }
}

// ---- a workgroup a part
constexpr int PART_THREADS = 512, PART_WAVES = PART_THREADS / 64, PART_UNITS = 8;
constexpr int PART_SLOTS = PART_WAVES * PART_UNITS * 64;

__global__ __launch_bounds__(256) void evict_clear_kernel(int *zero, long long ints) {
  for (long long i = blockIdx.x * 256ll + threadIdx.x; i < ints; i += gridDim.x * 256ll) zero[i] = 0;
}

struct EvictPart {
  unsigned g, g0;              // head, and first head of its pool
  int pool, part, count, seen, first;        // tokens of the head now and ever, first slot of the part
  HeadOf w;
  long long want;
};
// -> false: nothing to do for this workgroup.  A head's first part is there even if it holds nothing, for its count.
__device__ __forceinline__ bool evict_part(const CacheView &C, const EvictPlan &E, EvictPart &P) {
  P.g = (unsigned)invariant_quotient(blockIdx.x, E.parts_mul, E.parts_shift);
  P.part = (int)(blockIdx.x - P.g * (unsigned)E.parts);
  P.pool = E.pool_heads == 1 ? (int)P.g : invariant_quotient(P.g, C.layer_mul, C.layer_shift);
  P.g0 = (unsigned)P.pool * (unsigned)E.pool_heads;
  P.w = head_of(C, P.g);
  P.first = P.part * PART_SLOTS;
  // one round trip for all that is asked
  const int lane = threadIdx.x & 63;
  const long long here = count_at(C, P.w.b, P.w.l, P.w.h), layer = count_at(C, P.w.b, P.w.l, 0);
  P.seen = C.seen[here];
  const int mine = C.counts[E.pool_heads == 1 ? here : layer + min(lane, E.pool_heads - 1)], own = C.counts[here];
  P.want = evict_budget(E, P.w.b);
  P.count = clamp_to(own, C.capacity);
  if (P.part > 0 && P.first >= P.count) return false;
  if (E.pool_heads == 1) return P.count > P.want && P.count <= E.most;
  int c = lane < E.pool_heads ? clamp_to(mine, C.capacity) : 0, longest = c;        // (a pool's sum fits: check_scope)
  for (int h = lane + 64; h < E.pool_heads; h += 64) {
    const int x = held(C, P.w.b, P.w.l, h);
    c += x;
    longest = max(longest, x);
  }
  c = __builtin_amdgcn_readlane(wave_scan(c), 63);
  longest = (int)__builtin_amdgcn_readlane(wave_max_up((unsigned)longest), 63);
  return c > P.want && longest <= E.most;
}

// Adds a part's tally to its pool's.
__device__ __forceinline__ void add_hist(const int *mine, int *pool) {
  for (int i = threadIdx.x; i < 4096; i += PART_THREADS)
    if (mine[i] != 0) atomicAdd(&pool[i], mine[i]);
}

// The part's keys, as every launch but the first finds them; 0 behind the end.
__device__ __forceinline__ void part_keys(const EvictPlan &E, const EvictPart &P, int first, uint32_t (&key)[PART_UNITS]) {
  const uint32_t *k = E.keys + (long long)P.g * E.pitch + first + (threadIdx.x & 63);
#pragma unroll
  for (int i = 0; i < PART_UNITS; ++i) key[i] = k[64 * i];         // (the pitch is whole parts)
}

__global__ __launch_bounds__(PART_THREADS) void evict_keys_kernel(const CacheView C, const EvictPlan E) {
  __shared__ int hist[4096];
  EvictPart P;
  if (!evict_part(C, E, P)) {
    if (threadIdx.x == 0 && P.part == 0) E.left[P.g] = -1;
    return;
  }
  for (int i = threadIdx.x; i < 4096; i += PART_THREADS) hist[i] = 0;
  const int first = P.first + (int)(threadIdx.x >> 6) * PART_UNITS * 64, lane = threadIdx.x & 63;
  uint32_t key[PART_UNITS];
  // (no units of an empty head)
  evict_keys(C, head_place(C, P.w), E, first, P.count > 0 ? PART_UNITS : 0, P.count, recent_from(E, P.seen), key);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PART_UNITS; ++i) {
    const int slot = first + 64 * i + lane;
    E.keys[(long long)P.g * E.pitch + slot] = key[i];
    if (slot < P.count) atomicAdd(&hist[key[i] >> 20], 1);
  }
  __syncthreads();
  add_hist(hist, E.hist1 + (long long)P.pool * 4096);
}

__global__ __launch_bounds__(PART_THREADS) void evict_next_kernel(const CacheView C, const EvictPlan E) {
  __shared__ int hist[4096], per_wave[PART_WAVES], found[3];
  EvictPart P;
  if (!evict_part(C, E, P) || P.want == 0) return;
  const int first = P.first + (int)(threadIdx.x >> 6) * PART_UNITS * 64, lane = threadIdx.x & 63;
  uint32_t key[PART_UNITS];
  part_keys(E, P, first, key);
  for (int i = threadIdx.x; i < 4096; i += PART_THREADS) hist[i] = 0;
  find_bin<4096, PART_THREADS>(E.hist1 + (long long)P.pool * 4096, (int)P.want, per_wave, found);
  const int bin = found[0];
  if (threadIdx.x == 0 && P.g == P.g0 && P.part == 0) E.state1[P.pool] = make_int2(bin, (int)P.want - found[1]);
#pragma unroll
  for (int i = 0; i < PART_UNITS; ++i)
    if (first + 64 * i + lane < P.count && (int)(key[i] >> 20) == bin) atomicAdd(&hist[key[i] >> 8 & 4095], 1);
  __syncthreads();
  add_hist(hist, E.hist2 + (long long)P.pool * 4096);
}

__global__ __launch_bounds__(PART_THREADS) void evict_last_kernel(const CacheView C, const EvictPlan E) {
  __shared__ int hist[256], per_wave[PART_WAVES], found[3];
  EvictPart P;
  if (!evict_part(C, E, P) || P.want == 0) return;
  const int first = P.first + (int)(threadIdx.x >> 6) * PART_UNITS * 64, lane = threadIdx.x & 63;
  uint32_t key[PART_UNITS];
  part_keys(E, P, first, key);
  const int2 one = E.state1[P.pool];
  if (threadIdx.x < 256) hist[threadIdx.x] = 0;
  find_bin<4096, PART_THREADS>(E.hist2 + (long long)P.pool * 4096, one.y, per_wave, found);
  const int begins = one.x << 12 | found[0];
  if (threadIdx.x == 0 && P.g == P.g0 && P.part == 0) E.state2[P.pool] = make_int2(begins, one.y - found[1]);
  int above = 0;
#pragma unroll
  for (int i = 0; i < PART_UNITS; ++i) {
    const bool in = first + 64 * i + lane < P.count;
    const int b = (int)(key[i] >> 8);
    above += __popcll(__ballot(in && b > begins));
    if (in && b == begins) atomicAdd(&hist[key[i] & 255u], 1);
  }
  if (lane == 0) per_wave[threadIdx.x >> 6] = above;
  __syncthreads();
  const long long at = (long long)P.g * E.parts + P.part;
  if (threadIdx.x < 256) {
    E.last[at * 256 + threadIdx.x] = hist[threadIdx.x];
    if (hist[threadIdx.x] != 0) atomicAdd(&E.hist3[(long long)P.pool * 256 + threadIdx.x], hist[threadIdx.x]);
  }
  int all;
  waves_before<PART_WAVES>(per_wave, 0, all);
  if (threadIdx.x == 0) E.above[at] = all;
}

// Sums over the workgroup, to all: every wave adds up the eight waves' of all N at once, eight lanes each.
template <int N>
__device__ __forceinline__ void part_sums(int (&x)[N], int (*per_wave)[PART_WAVES]) {
  static_assert(PART_WAVES == 8 && N <= 8, "eight lanes a sum");
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int upto = wave_scan(x[i]);
    if (lane == 63) per_wave[i][threadIdx.x >> 6] = upto;
  }
  __syncthreads();
  int all = lane < 8 * N ? per_wave[0][lane] : 0;
  all += __builtin_amdgcn_update_dpp(0, all, 0xb1, 0xf, 0xf, false);         // the neighbour's, the other pair's, the other four's
  all += __builtin_amdgcn_update_dpp(0, all, 0x4e, 0xf, 0xf, false);
  all += __builtin_amdgcn_update_dpp(0, all, 0x141, 0xf, 0xf, false);
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = __builtin_amdgcn_readlane(all, 8 * i);
}

__global__ __launch_bounds__(PART_THREADS) void evict_list_kernel(const CacheView C, const EvictPlan E) {
  __shared__ int per_wave[PART_WAVES], found[3], waves[PART_WAVES], sums[5][PART_WAVES];
  EvictPart P;
  if (!evict_part(C, E, P)) return;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  if (P.want == 0) {                                       // nothing stays, nothing moves
    if (tid == 0 && P.part == 0) E.left[P.g] = 0;
    return;
  }
  const int first = P.first + wave * PART_UNITS * 64;
  uint32_t key[PART_UNITS];
  part_keys(E, P, first, key);
  const int2 two = E.state2[P.pool];
  // the head's tallies of the last 8 bits, this thread's digit in every other part, in all of them and in those before this one
  const int parts = max(1, (int)(((long long)P.count + PART_SLOTS - 1) / PART_SLOTS)), d = tid & 255;
  int same = 0, same_front = 0, above = 0, above_front = 0;
#pragma unroll 1
  for (int q = tid >> 8; q < parts; q += PART_THREADS / 256) {
    const long long at = (long long)P.g * E.parts + q;
    const int x = E.last[at * 256 + d], a = d == 0 ? E.above[at] : 0;
    same += x;
    above += a;
    same_front += q < P.part ? x : 0;
    above_front += q < P.part ? a : 0;
  }
  find_bin<256, PART_THREADS>(E.hist3 + (long long)P.pool * 256, two.y, per_wave, found);
  const int digit = found[0], ties = two.y - found[1];
  const uint32_t last = (uint32_t)two.x << 8 | (uint32_t)digit;
  // equals in the heads before; equals and larger ones in the head, and in its parts before this one
  enum { EQ_HEADS, EQ_HEAD, EQ_FRONT, GT_HEAD, GT_FRONT };
  int sum[5] = {0, d == digit ? same : 0, d == digit ? same_front : 0, above + (d > digit ? same : 0), above_front + (d > digit ? same_front : 0)};
  if (found[2] > ties)                                     // else all equals stay
    for (long long i = tid; i < (long long)(P.g - P.g0) * E.parts; i += PART_THREADS) {
      const int h = (int)((unsigned long long)i / (unsigned)E.parts), q = (int)(i - (long long)h * E.parts);
      if (q == 0 || q * (long long)PART_SLOTS < held(C, P.w.b, P.w.l, h)) sum[EQ_HEADS] += E.last[((long long)P.g0 * E.parts + i) * 256 + digit];
    }
  part_sums(sum, sums);
  const int mine = min(max(ties - sum[EQ_HEADS], 0), sum[EQ_HEAD]), left = sum[GT_HEAD] + mine;      // equals that stay in the head, its new count
  if (tid == 0 && P.part == 0) E.left[P.g] = left;

  int equal, more, all;
  count_keys(key, PART_UNITS, last, equal, more);
  if (lane == 0) waves[wave] = equal | more << 16;
  __syncthreads();
  const int front = waves_before<PART_WAVES>(waves, wave, all);
  int *list = E.lists + (long long)P.g * E.list;
  const int late = list_keys(key, first, PART_UNITS, last, sum[EQ_FRONT] + (front & 0xffff), sum[GT_FRONT] + (front >> 16), mine, left, list,
                             list + E.list / 2);
  if (lane == 0 && late > 0) atomicAdd(&E.moves[P.g], late);
}

constexpr int MOVE_THREADS = 256;

__global__ __launch_bounds__(MOVE_THREADS) void evict_move_kernel(const CacheView C, const EvictPlan E, int parts) {
  const unsigned g = blockIdx.x / (unsigned)parts;
  const int part = (int)(blockIdx.x - g * (unsigned)parts);
  const int left = E.left[g];
  if (left < 0) return;
  const int moves = E.moves[g];
  const HeadOf w = head_of(C, g);
  if (part == 0 && threadIdx.x == 0) C.counts[count_at(C, w.b, w.l, w.h)] = left;
  const HeadPlace p = head_place(C, w);
  const int *list = E.lists + (long long)g * E.list;
  for (int i = part * (MOVE_THREADS / 16) + (int)(threadIdx.x >> 4); i < moves; i += parts * (MOVE_THREADS / 16))
    move_row(C, p, list[i], list[E.list / 2 + moves - 1 - i], threadIdx.x & 15);
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

// Whether one workgroup a pool does everything.
static bool evict_alone(const CacheView &C, const compactor_cache_evict_params_t *e) {
  const int most = evict_most(C, e);
  if (e->scope == COMPACTOR_SCOPE_HEAD || C.kv_heads == 1) return most <= ALONE_SLOTS;
  return (long long)C.kv_heads * ((most + 63) / 64) <= POOL_UNITS;
}

// Sizes and places of the parts' scratch in a workspace at `ws` (null: sizes only); returns its bytes.
static size_t evict_scratch(const CacheView &C, const compactor_cache_evict_params_t *e, unsigned char *ws, EvictPlan *E) {
  const size_t heads = (size_t)C.nreq * C.layers * C.kv_heads;
  const size_t pools = e->scope == COMPACTOR_SCOPE_LAYER ? heads / C.kv_heads : heads;
  E->most = evict_most(C, e);
  E->parts = (int)(((long long)E->most + PART_SLOTS - 1) / PART_SLOTS);
  invariant_divisor(E->parts, &E->parts_mul, &E->parts_shift);
  const size_t pitch = (size_t)E->parts * PART_SLOTS;
  E->list = 2 * (E->most / 2 + 1);               // a head moves at most half of its tokens (one into a slot that another left)
  size_t at = 0;
  auto take = [&](size_t ints) {
    unsigned char *x = ws == nullptr ? nullptr : ws + at;
    at += (ints * sizeof(int) + 255) / 256 * 256;
    return x;
  };
  // the first four are cleared before they are used
  E->hist1 = reinterpret_cast<int *>(take(pools * 4096));
  E->hist2 = reinterpret_cast<int *>(take(pools * 4096));
  E->hist3 = reinterpret_cast<int *>(take(pools * 256));
  E->moves = reinterpret_cast<int *>(take(heads));
  E->left = reinterpret_cast<int *>(take(heads));
  E->state1 = reinterpret_cast<int2 *>(take(2 * pools));
  E->state2 = reinterpret_cast<int2 *>(take(2 * pools));
  E->above = reinterpret_cast<int *>(take(heads * E->parts));
  E->last = reinterpret_cast<int *>(take(heads * E->parts * 256));
  E->keys = reinterpret_cast<uint32_t *>(take(heads * pitch));
  E->lists = reinterpret_cast<int *>(take(heads * E->list));
  E->pitch = (long long)pitch;
  return at;
}

static size_t evict_bytes(const CacheView &C, const compactor_cache_evict_params_t *e) {
  EvictPlan E;
  return evict_alone(C, e) ? 0 : evict_scratch(C, e, nullptr, &E);
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
  if (!launchable(R.tokens <= APPEND_FEW ? (heads + 15) / 16 : heads * parts, 256)) return COMPACTOR_EINVAL;
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
  *bytes = evict_bytes(C, evict);
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
  const long long heads = (long long)C.nreq * C.layers * C.kv_heads;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (evict_alone(C, evict)) {
    E.most = evict_most(C, evict);
    if (!launchable(heads / E.pool_heads, ALONE_THREADS)) return COMPACTOR_EINVAL;
    (void)hipGetLastError();
    if (E.pool_heads == 1)
      hipLaunchKernelGGL(evict_alone_kernel, dim3((unsigned)heads), dim3(ALONE_THREADS), 0, st, C, E);
    else
      hipLaunchKernelGGL(evict_pool_kernel, dim3((unsigned)(heads / C.kv_heads)), dim3(ALONE_THREADS), 0, st, C, E);
    return hipGetLastError() == hipSuccess ? COMPACTOR_OK : COMPACTOR_EHIP;
  }
  if (!workspace || workspace_bytes < evict_bytes(C, evict)) return COMPACTOR_EWORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return COMPACTOR_EALIGN;
  evict_scratch(C, evict, static_cast<unsigned char *>(workspace), &E);
  long long movers = 2048 / heads;
  movers = movers < 1 ? 1 : (movers > 128 ? 128 : movers);
  if (!launchable(heads * E.parts, PART_THREADS) || !launchable(heads * movers, MOVE_THREADS)) return COMPACTOR_EINVAL;
  const dim3 grid((unsigned)(heads * E.parts)), block(PART_THREADS);
  const long long clear = (reinterpret_cast<unsigned char *>(E.left) - reinterpret_cast<unsigned char *>(E.hist1)) / (long long)sizeof(int);
  const unsigned clear_wgs = (unsigned)std::min((clear + 1023) / 1024, 1024ll);
  (void)hipGetLastError();
  hipLaunchKernelGGL(evict_clear_kernel, dim3(clear_wgs), dim3(256), 0, st, E.hist1, clear);
  if (hipGetLastError() != hipSuccess) return COMPACTOR_EHIP;
  hipLaunchKernelGGL(evict_keys_kernel, grid, block, 0, st, C, E);
  if (hipGetLastError() != hipSuccess) return COMPACTOR_EHIP;
  hipLaunchKernelGGL(evict_next_kernel, grid, block, 0, st, C, E);
  if (hipGetLastError() != hipSuccess) return COMPACTOR_EHIP;
  hipLaunchKernelGGL(evict_last_kernel, grid, block, 0, st, C, E);
  if (hipGetLastError() != hipSuccess) return COMPACTOR_EHIP;
  hipLaunchKernelGGL(evict_list_kernel, grid, block, 0, st, C, E);
  if (hipGetLastError() != hipSuccess) return COMPACTOR_EHIP;
  hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)(heads * movers)), dim3(MOVE_THREADS), 0, st, C, E, (int)movers);
  return hipGetLastError() == hipSuccess ? COMPACTOR_OK : COMPACTOR_EHIP;
}

#pragma GCC visibility pop
}  // extern "C"
