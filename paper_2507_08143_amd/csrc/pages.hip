// Pages that caches share (see compactor_pages_reserve): which entries of the tables get one, fork, release, compaction, and the copies.
//
// Deciding is a few hundred to some ten thousand numbers, bound by the latency of its steps: one workgroup takes it, so that the steps
// are barriers and not launches.  Copies are bound by HBM.
#include <algorithm>
#include <initializer_list>
#include <utility>

#include "cache.h"

namespace cmp {

constexpr int PLAN_THREADS = 1024, PLAN_WAVES = PLAN_THREADS / 64;
constexpr int PAGES_MOST = 16384;            // requests
constexpr int POOL_MOST = 1 << 30;           // pages, so that a step beyond the last one fits 32 bits
constexpr long long ENTRIES_MOST = 0x7fffffffll - PLAN_THREADS;        // of all tables, likewise

__device__ __forceinline__ int pages_of(const CacheView &C, int tokens) {       // that hold them
  const int full = invariant_quotient((unsigned)tokens, C.div_mul, C.div_shift);
  return full + (tokens > full * C.page_size ? 1 : 0);
}

// Sums over the threads of the workgroup up to and with this one; *all: over all of them.  part: PLAN_WAVES numbers.
__device__ __forceinline__ int plan_scan(int x, int *part, int *all) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int upto = wave_scan(x);
  __syncthreads();                           // the numbers of the last sum have been read
  if (lane == 63) part[wave] = upto;
  __syncthreads();
  int before = 0, sum = 0;
#pragma unroll
  for (int i = 0; i < PLAN_WAVES; ++i) {
    const int y = part[i];
    before += i < wave ? y : 0;
    sum += y;
  }
  *all = sum;
  return before + upto;
}

// The most and the fewest tokens of a request's heads, by a workgroup of 256.
struct Most { int top, low; };
__device__ __forceinline__ Most most_of(const CacheView &C, int b, int2 *part) {
  int top = 0, low = C.capacity;
  const int heads = C.layers * C.kv_heads;
#pragma unroll 4
  for (int i = threadIdx.x; i < heads; i += 256) {
    const int l = invariant_quotient((unsigned)i, C.layer_mul, C.layer_shift);
    const int n = held(C, b, l, i - l * C.kv_heads);
    top = max(top, n);
    low = min(low, n);
  }
  for (int d = 32; d > 0; d >>= 1) {
    top = max(top, __shfl_xor(top, d));
    low = min(low, __shfl_xor(low, d));
  }
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = make_int2(top, low);
  __syncthreads();
  Most m{0, C.capacity};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m.top = max(m.top, part[i].x);
    m.low = min(m.low, part[i].y);
  }
  return m;
}

// ------------------------------------------------------------------------------------------ reserve
struct Reserve {
  int32_t *tables, *refs;
  const int32_t *new_tokens;
  int tokens, own_all, table_len;
  int2 *pairs;
  int32_t *done;
  // scratch
  int4 *spans;                 // [request]: entries from, to, those from here on are for new tokens, the first one's number of all
  int *entries, *kinds, *pages;        // of the entries of all spans, one after the other: place in the tables, what it wants, page that it names
  int *tally, *last;           // [page]: entries in spans that name it, the last of them
  int *free_pages;
};
enum EntryKind { WANTS_NONE, WANTS_PAGE, WANTS_COPY };

// Entries of a request from .. to, those from `holds` on are for new tokens.
__device__ __forceinline__ int4 span_of(const CacheView &C, const Reserve &R, int b, const Most &m) {
  const int n = tokens_new(R.new_tokens, b, R.tokens), holds = pages_of(C, m.top);
  const int need = pages_of(C, n < C.capacity - m.top ? m.top + n : C.capacity);
  const int first = R.own_all ? 0 : n > 0 ? invariant_quotient((unsigned)m.low, C.div_mul, C.div_shift) : holds;
  return make_int4(min(first, need), need, holds, 0);
}
__device__ __forceinline__ void reserve_done(const Reserve &R, int copies, int wants, int found) {
  if (threadIdx.x != 0) return;
  R.done[0] = copies;
  R.done[1] = max(wants - found, 0);
}
// Which of the pages p .. p + 3 are free.
__device__ __forceinline__ void four_free(const CacheView &C, const Reserve &R, int p, int (&is_free)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) is_free[i] = p + i < C.num_pages && R.refs[min(p + i, C.num_pages - 1)] == 0;
}
// A bit for each of the references of pages p .. p + 15 that is `so`; none for pages beyond the last.
template <class So>
__device__ __forceinline__ unsigned sixteen(const int32_t *refs, int pages, long long p, So so) {
  unsigned bits = 0;
  if (p + 16 <= pages) {
    int4 x[4];
    __builtin_memcpy(x, refs + p, sizeof(x));        // on 4 bytes
#pragma unroll
    for (int i = 0; i < 4; ++i)
      bits |= (unsigned)so(x[i].x) << (4 * i) | (unsigned)so(x[i].y) << (4 * i + 1) | (unsigned)so(x[i].z) << (4 * i + 2) | (unsigned)so(x[i].w) << (4 * i + 3);
  } else if (p < pages) {
#pragma unroll
    for (int i = 0; i < 16; ++i) bits |= (unsigned)(p + i < pages && so(refs[min(p + i, pages - 1ll)])) << i;
  }
  return bits;
}
// The first `wants` free pages, in order, or as many as there are; -> how many.  first: four_free(4 * threadIdx.x), which is enough for a small pool; behind
// those 16 a thread (us of a reserve where all but the last pages are in use, with 4 and with 16: of 5000 pages 7.6 and 8.6, of 20 000 13.1 and 8.7, of
// 100 000 48 and 17, of 400 000 180 and 50; with the next ones loaded before the scan 64 requests' step in a pool of 20 000 takes 9.1 us instead of 7.8).
__device__ __forceinline__ int find_free(const CacheView &C, const Reserve &R, int wants, const int (&first)[4], int *pages, int *part) {
  unsigned bits = (unsigned)first[0] | (unsigned)first[1] << 1 | (unsigned)first[2] << 2 | (unsigned)first[3] << 3;
  int found = 0, each = 4;
  for (long long p0 = 0; p0 < C.num_pages && found < wants;) {
    if (p0 > 0) {
      each = 16;
      bits = sixteen(R.refs, C.num_pages, p0 + 16 * (int)threadIdx.x, [](int refs) { return refs == 0; });
    }
    const int mine = __popc(bits);
    int all;
    int at = found + plan_scan(mine, part, &all) - mine;
    for (; bits != 0 && at < wants; bits &= bits - 1) pages[at++] = (int)p0 + each * (int)threadIdx.x + __ffs(bits) - 1;
    found += all;
    p0 += each * PLAN_THREADS;
  }
  __syncthreads();                           // they are listed, and no count of references is looked at any more
  return found;
}
__device__ __forceinline__ void give_page(const Reserve &R, int32_t *entry, int kind, int old, int page, int pair) {
  *entry = page;
  R.refs[page] = 1;
  if (kind == WANTS_COPY) {
    atomicAdd(&R.refs[old], -1);
    R.pairs[pair] = make_int2(old, page);
  }
}

__global__ __launch_bounds__(256) void reserve_spans_kernel(const CacheView C, const Reserve R) {
  __shared__ int2 part[4];
  const int b = (int)blockIdx.x;
  const Most m = most_of(C, b, part);
  if (threadIdx.x == 0) R.spans[b] = span_of(C, R, b, m);
}

// Numbers that atomics have made, past the cache of the compute unit.
__device__ __forceinline__ int atomic_read(const int *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Any number of entries, by way of the workspace; the spans are there, with their numbers.
__device__ __forceinline__ void reserve_many(const CacheView &C, const Reserve &R, int entries, const int (&first)[4], int *part) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  for (int b = wave; b < C.nreq; b += PLAN_WAVES) {
    const int4 s = R.spans[b];
    for (int i = s.x + lane; i < s.y; i += 64) {
      const int e = s.w + i - s.x;
      R.entries[e] = b * R.table_len + i;
      R.kinds[e] = i >= s.z ? WANTS_PAGE : WANTS_NONE;
    }
  }
  __syncthreads();
  auto entry_of = [&](int e) {
    const int at = R.entries[e], b = (int)((unsigned)at / (unsigned)R.table_len);
    return R.tables + b * C.table_stride + (at - b * R.table_len);
  };
  for (int e = tid; e < entries; e += PLAN_THREADS) {
    const int page = *entry_of(e);
    const bool there = page_there(C, page);
    const int kind = !there ? R.kinds[e] : R.refs[page] > 1 ? WANTS_COPY : WANTS_NONE;
    R.kinds[e] = kind;
    R.pages[e] = page;
    if (kind == WANTS_COPY) {
      R.tally[page] = 0;
      R.last[page] = -1;
    }
  }
  __threadfence();
  __syncthreads();
  for (int e = tid; e < entries; e += PLAN_THREADS)
    if (R.kinds[e] == WANTS_COPY) {
      atomicAdd(&R.tally[R.pages[e]], 1);
      atomicMax(&R.last[R.pages[e]], e);
    }
  __threadfence();
  __syncthreads();
  int wants = 0;
  for (int e = tid; e < entries; e += PLAN_THREADS) {
    int kind = R.kinds[e];
    if (kind == WANTS_COPY) {
      const int page = R.pages[e];
      if (atomic_read(&R.tally[page]) == R.refs[page] && atomic_read(&R.last[page]) == e) R.kinds[e] = kind = WANTS_NONE;      // keeps it
    }
    wants += kind != WANTS_NONE;
  }
  plan_scan(wants, part, &wants);
  const int found = find_free(C, R, wants, first, R.free_pages, part);
  int given = 0, copies = 0;
  for (int e0 = 0; e0 < entries && found >= wants && wants > 0; e0 += PLAN_THREADS) {
    const int e = e0 + tid, kind = e < entries ? R.kinds[e] : WANTS_NONE;
    int all;
    const int mine = (kind != WANTS_NONE) + ((kind == WANTS_COPY) << 16), before = plan_scan(mine, part, &all) - mine;
    if (kind != WANTS_NONE) give_page(R, entry_of(e), kind, R.pages[e], R.free_pages[given + (before & 0xffff)], copies + (before >> 16));
    given += all & 0xffff;
    copies += all >> 16;
  }
  reserve_done(R, copies, wants, found);
}

__global__ __launch_bounds__(PLAN_THREADS) void reserve_plan_kernel(const CacheView C, const Reserve R) {
  __shared__ int part[PLAN_WAVES];
  int first[4];
  four_free(C, R, 4 * (int)threadIdx.x, first);
  int entries = 0;
  for (int b0 = 0; b0 < C.nreq; b0 += PLAN_THREADS) {
    const int b = b0 + (int)threadIdx.x;
    const int4 s = b < C.nreq ? R.spans[b] : make_int4(0, 0, 0, 0);
    int all;
    const int upto = plan_scan(s.y - s.x, part, &all);
    if (b < C.nreq) R.spans[b].w = entries + upto - (s.y - s.x);
    entries += all;
  }
  __syncthreads();
  reserve_many(C, R, entries, first, part);
}

// Up to an entry a thread, which is a step that does not ask for the pages of whole contexts: all in registers and LDS, one launch, and three loads that wait for each other (counts,
// entry, references).  64 requests of which some need a page: 14.2 and 3.1 us in two launches by way of the workspace, 7.4 in this one.
// More entries go the other way, in time that grows with them (us of own_all, no page shared / eight contexts on the same pages: 48 contexts of 1640 pages 174 / 833, 64 of
// 2000 276 / 1353).
constexpr int FEW_REQUESTS = PLAN_THREADS;
constexpr long long FEW_COUNTS = 65536;
__global__ __launch_bounds__(PLAN_THREADS) void reserve_few_kernel(const CacheView C, const Reserve R) {
  __shared__ int part[PLAN_WAVES];
  __shared__ int4 spans[FEW_REQUESTS];
  __shared__ int4 named4[PLAN_THREADS / 4];              // pages that entries would have copies of, else -1
  __shared__ int free_pages[PLAN_THREADS];
  int *named = reinterpret_cast<int *>(named4);
  const int tid = threadIdx.x, row = tid >> 4, lane = tid & 15, heads = C.layers * C.kv_heads;
  int first[4];
  four_free(C, R, 4 * tid, first);
  for (int b0 = 0; b0 < C.nreq; b0 += PLAN_THREADS / 16) {
    const int b = b0 + row;
    int top = 0, low = C.capacity;
    if (b < C.nreq) {
      auto take = [&](int count) {
        const int n = clamp_to(count, C.capacity);
        top = max(top, n);
        low = min(low, n);
      };
      if (C.layers == 1 || C.count_stride_l == C.kv_heads) {             // a request's counts lie together
        const int32_t *counts = C.counts + b * C.count_stride_b;
#pragma unroll 16
        for (int i = lane; i < heads; i += 16) take(counts[i]);
      } else {
#pragma unroll 4
        for (int i = lane; i < heads; i += 16) {
          const int l = invariant_quotient((unsigned)i, C.layer_mul, C.layer_shift);
          take(C.counts[count_at(C, b, l, i - l * C.kv_heads)]);
        }
      }
    }
    for (int d = 8; d > 0; d >>= 1) {
      top = max(top, __shfl_xor(top, d));
      low = min(low, __shfl_xor(low, d));
    }
    if (lane == 0 && b < C.nreq) spans[b] = span_of(C, R, b, Most{top, low});
  }
  __syncthreads();
  int4 s = tid < C.nreq ? spans[tid] : make_int4(0, 0, 0, 0);
  int entries;
  const int upto = plan_scan(s.y - s.x, part, &entries);
  s.w = upto - (s.y - s.x);
  if (tid < C.nreq) {
    spans[tid].w = s.w;
    if (entries > PLAN_THREADS) R.spans[tid] = s;
  }
  __syncthreads();
  if (entries > PLAN_THREADS) {
    reserve_many(C, R, entries, first, part);
    return;
  }
  // the request of entry `tid`: the last whose first entry is not behind it
  int b = 0;
  for (int d = PLAN_THREADS / 2; d > 0; d >>= 1)
    if (b + d < C.nreq && spans[b + d].w <= tid) b += d;
  const bool is = tid < entries;
  s = spans[b];
  const int i = s.x + tid - s.w;
  int32_t *entry = R.tables + b * C.table_stride + i;
  const int page = is ? *entry : -1;
  const bool there = page_there(C, page);
  int kind = !is ? WANTS_NONE : !there ? (i >= s.z ? WANTS_PAGE : WANTS_NONE) : WANTS_NONE, refs = 0;
  if (there && (refs = R.refs[page]) > 1) kind = WANTS_COPY;
  named[tid] = kind == WANTS_COPY ? page : -1;
  if (__syncthreads_or(kind == WANTS_COPY)) {
    if (kind == WANTS_COPY) {
      int tally = 0, last = 0;
#pragma unroll 8
      for (int k = 0; k < (entries + 3) / 4; ++k) {
        const int4 x = named4[k];
        tally += (x.x == page) + (x.y == page) + (x.z == page) + (x.w == page);
        last = x.w == page ? 4 * k + 3 : x.z == page ? 4 * k + 2 : x.y == page ? 4 * k + 1 : x.x == page ? 4 * k : last;
      }
      if (tally == refs && last == tid) kind = WANTS_NONE;             // keeps it
    }
  }
  const int mine = (kind != WANTS_NONE) + ((kind == WANTS_COPY) << 16);
  int all;
  const int before = plan_scan(mine, part, &all) - mine, wants = all & 0xffff;
  const int found = find_free(C, R, wants, first, free_pages, part);
  if (found >= wants && kind != WANTS_NONE) give_page(R, entry, kind, page, free_pages[before & 0xffff], before >> 16);
  reserve_done(R, found >= wants ? all >> 16 : 0, wants, found);
}

// ------------------------------------------------------------------------------------------ fork
// A workgroup has a strip of columns of the tables, of counts or of seen: of all requests, so that it reads all of it before it writes.  Bound by the
// latency of its three loads and of the atomics behind them, so strips are of 1024 numbers, but 8 columns at least, part of a cache line: 64 tables of
// 2000 pages, beams of four, 4.0 us with 16 columns, 10.6 with 64.  Where many requests make even those large, strips get narrower so that they fit LDS.
struct Fork {
  int32_t *tables, *refs;
  const int32_t *parents;
  int table_len, width_log;    // of a strip
  int table_strips, head_strips;
};
constexpr int FORK_NUMBERS = 16384;          // of a strip, that LDS holds

__global__ __launch_bounds__(256) void fork_kernel(const CacheView C, const Fork F) {
  extern __shared__ int old[];
  const int which = (int)blockIdx.x < F.table_strips ? 0 : (int)blockIdx.x - F.table_strips < F.head_strips ? 1 : 2;
  const int strip = (int)blockIdx.x - (which > 0 ? F.table_strips : 0) - (which > 1 ? F.head_strips : 0);
  const int width = 1 << F.width_log, columns = which == 0 ? F.table_len : C.layers * C.kv_heads, all = C.nreq << F.width_log;
  auto at = [&](int i) {
    const int b = i >> F.width_log, c = strip * width + (i & (width - 1));
    if (which == 0) return F.tables + b * C.table_stride + c;
    const int l = invariant_quotient((unsigned)c, C.layer_mul, C.layer_shift);
    return (which == 1 ? C.counts : C.seen) + count_at(C, b, l, c - l * C.kv_heads);
  };
  auto there = [&](int i) { return strip * width + (i & (width - 1)) < columns; };
#pragma unroll 4
  for (int i = threadIdx.x; i < all; i += 256)
    if (there(i)) old[i] = *at(i);
  __syncthreads();
#pragma unroll 4
  for (int i = threadIdx.x; i < all; i += 256) {
    const int parent = F.parents[i >> F.width_log];
    if (!there(i) || (unsigned)parent >= (unsigned)C.nreq) continue;
    const int x = old[(parent << F.width_log) + (i & (width - 1))], was = old[i];
    if (x == was) continue;
    *at(i) = x;
    if (which == 0) {
      if (page_there(C, x)) atomicAdd(&F.refs[x], 1);
      if (page_there(C, was)) atomicAdd(&F.refs[was], -1);
    }
  }
}

// ------------------------------------------------------------------------------------------ release
__global__ __launch_bounds__(256) void release_kernel(const CacheView C, int32_t *tables, int table_len, int32_t *refs, const int32_t *finished) {
  __shared__ int2 part[4];
  const int b = (int)blockIdx.x;
  const bool ended = finished != nullptr && finished[b] != 0;
  int keep = 0;
  if (ended) {
    const int heads = C.layers * C.kv_heads;
    for (int i = threadIdx.x; i < heads; i += 256) {
      const int l = invariant_quotient((unsigned)i, C.layer_mul, C.layer_shift);
      const long long at = count_at(C, b, l, i - l * C.kv_heads);
      C.counts[at] = 0;
      if (C.seen != nullptr) C.seen[at] = 0;
    }
  } else {
    keep = pages_of(C, most_of(C, b, part).top);
  }
  int32_t *table = tables + b * C.table_stride;
#pragma unroll 4
  for (int i = keep + (int)threadIdx.x; i < table_len; i += 256) {
    const int page = table[i];
    if (!page_there(C, page)) continue;
    table[i] = -1;
    atomicAdd(&refs[page], -1);
  }
}

// ------------------------------------------------------------------------------------------ compact
struct Compact {
  int32_t *tables, *refs;
  int table_len;
  int2 *pairs;
  int32_t *done;
  int *to;                     // scratch, [page]: from the number of pages in use on, where a page goes; behind them that number
};

// Bound by the latency of its passes, one over all references and one in steps of 16 384 with the numbers in between (us with the tables' kernel, where nothing
// has to move; in brackets with 4 pages a thread and step: of 5000 pages 6.7 (6.9), of 20 000 7.7 (12.6), of 100 000 22 (45), of 400 000 77 (167)).
__global__ __launch_bounds__(PLAN_THREADS) void compact_plan_kernel(const CacheView C, const Compact K) {
  __shared__ int part[PLAN_WAVES];
  const int tid = threadIdx.x, N = C.num_pages;
  auto used = [&](long long p) { return sixteen(K.refs, N, p, [](int refs) { return refs > 0; }); };
  int n = 0, moves = 0;
#pragma unroll 4
  for (long long p = 16 * tid; p < N; p += 16 * PLAN_THREADS) n += __popc(used(p));
  plan_scan(n, part, &n);
  int before = 0;                            // pages in use so far
  for (long long p0 = 0; p0 < N; p0 += 16 * PLAN_THREADS) {
    const long long p = p0 + 16 * tid;
    const unsigned is_used = used(p);
    int all;
    const int at = before + plan_scan(__popc(is_used), part, &all) - __popc(is_used);
    before += all;
    if (p >= N) continue;
    const int low = clamp_to(n - p, 16);                                    // of the 16 are below n
    const unsigned below = (1u << low) - 1u;
    auto rank = [&](int i) { return at + __popc(is_used & ((1u << i) - 1u)); };             // pages in use before p + i
    for (unsigned bits = ~is_used & below; bits != 0; bits &= bits - 1, ++moves) {
      const int i = __ffs(bits) - 1;
      K.pairs[p + i - rank(i)].y = (int)p + i;
    }
    for (unsigned bits = is_used & ~below; bits != 0; bits &= bits - 1) {
      const int i = __ffs(bits) - 1;
      K.pairs[n - 1 - rank(i)].x = (int)p + i;
    }
    if (low == 16) continue;
    if (p + 16 <= N) {                       // (those below n are not looked at)
      const int q = (int)p;
#pragma unroll
      for (int i = 0; i < 16; i += 4) reinterpret_cast<int4 *>(K.to + q)[i >> 2] = make_int4(q + i, q + i + 1, q + i + 2, q + i + 3);
    } else {
      for (int i = 0; p + i < N; ++i) K.to[p + i] = (int)p + i;
    }
  }
  plan_scan(moves, part, &moves);
  __syncthreads();
  for (int i = tid; i < moves; i += PLAN_THREADS) {
    const int2 x = K.pairs[i];
    K.to[x.x] = x.y;
    K.refs[x.y] = K.refs[x.x];
    K.refs[x.x] = 0;
  }
  if (tid == 0) {
    K.to[N] = n;
    K.done[0] = moves;
    K.done[1] = n;
  }
}
__global__ __launch_bounds__(256) void compact_tables_kernel(const CacheView C, const Compact K) {
  const unsigned at = blockIdx.x * 256u + threadIdx.x;
  if (at >= (unsigned)C.nreq * (unsigned)K.table_len) return;
  const unsigned b = at / (unsigned)K.table_len;
  int32_t *entry = K.tables + b * C.table_stride + (at - b * (unsigned)K.table_len);
  const int page = *entry;
  if (!page_there(C, page) || page < K.to[C.num_pages]) return;
  const int to = K.to[page];
  if (to != page) *entry = to;
}

// ------------------------------------------------------------------------------------------ copy
// What a page consists of: runs of bytes that lie together, in up to three dimensions.
struct Runs {
  long long page;              // stride of pages, bytes
  int units;                   // of a page, of 16 (state: 4) bytes
  int run;                     // of a run
  unsigned run_mul, run_shift;
  int dims;
  int n[3];
  unsigned mul[3], shift[3];
  long long stride[3];         // bytes
};
struct Copy {
  const int2 *pairs;
  const int32_t *done;
  int most;
  char *rows[2];
  char *state[4];              // those that there are, in front
  int states;
  Runs row, word;
  int row_chunks, chunks;      // of K (V) of a page; of a page
};
// Written past the caches: what is read is often shared by several copies, and what is written nobody reads for a while.  us of 112 copies of 16 pages of all layers
// (477 MB in and out) with the reserve before them 65, with plain stores 75 at the same number of workgroups; 3570 pages of 0.27 MB (1.9 GB) with release and
// plan 427.  With 8 workgroups a unit 74 and 463, with 32 66 and 427; 8 units a thread 80 and 427.  Of the 427 the copy is 390, 4.8 TB/s.
constexpr int COPY_AT_ONCE = 4;              // units of a thread
constexpr int COPY_WORKGROUPS = 4;           // a compute unit
__device__ __forceinline__ void put(char *p, const uint4 &x) { store_stream16(p, x); }
__device__ __forceinline__ void put(char *p, unsigned x) { *reinterpret_cast<unsigned *>(p) = x; }

__device__ __forceinline__ long long unit_at(const Runs &R, int u, int bytes) {
  if (R.dims == 0) return (long long)u * bytes;
  int outer = invariant_quotient((unsigned)u, R.run_mul, R.run_shift);
  long long at = (long long)(u - outer * R.run) * bytes;
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (i < R.dims) {
      const int next = i + 1 < R.dims ? invariant_quotient((unsigned)outer, R.mul[i], R.shift[i]) : 0;
      at += (outer - next * R.n[i]) * R.stride[i];
      outer = next;
    }
  return at;
}
template <class T>
__device__ __forceinline__ void copy_chunk(char *base, const Runs &R, int2 pair, int chunk) {
  T x[COPY_AT_ONCE];
  long long at[COPY_AT_ONCE];
  const int u0 = chunk * 256 * COPY_AT_ONCE + (int)threadIdx.x;
#pragma unroll
  for (int i = 0; i < COPY_AT_ONCE; ++i)
    if (u0 + 256 * i < R.units) {
      at[i] = unit_at(R, u0 + 256 * i, sizeof(T));
      x[i] = *reinterpret_cast<const T *>(base + pair.x * R.page + at[i]);
    }
#pragma unroll
  for (int i = 0; i < COPY_AT_ONCE; ++i)
    if (u0 + 256 * i < R.units) put(base + pair.y * R.page + at[i], x[i]);
}
__global__ __launch_bounds__(256) void copy_kernel(const CacheView C, const Copy P) {
  const long long all = (long long)clamp_to(P.done[0], P.most) * P.chunks;
  for (long long w = blockIdx.x; w < all; w += gridDim.x) {
    const long long i = w / P.chunks;
    int chunk = (int)(w - i * P.chunks);
    const int2 pair = P.pairs[i];
    if (!page_there(C, pair.x) || !page_there(C, pair.y)) continue;
    if (chunk < 2 * P.row_chunks) {
      const bool v = chunk >= P.row_chunks;
      copy_chunk<uint4>(P.rows[v], P.row, pair, v ? chunk - P.row_chunks : chunk);
    } else {
      chunk -= 2 * P.row_chunks;
#pragma unroll
      for (int s = 0; s < 4; ++s)
        if (s < P.states) copy_chunk<unsigned>(P.state[s], P.word, pair, chunk);
    }
  }
}

// ------------------------------------------------------------------------------------------ calls
static bool runs_of(long long page, long long run, int unit, std::initializer_list<std::pair<int, long long>> dims, Runs *R) {
  std::pair<int, long long> d[3];
  int n = 0;
  for (const auto &x : dims)
    if (x.first > 1) d[n++] = x;
  std::sort(d, d + n, [](const auto &a, const auto &b) { return a.second < b.second; });
  int k = 0;
  while (k < n && d[k].second == run) run *= d[k++].first;
  *R = Runs{};
  R->page = page;
  R->run = (int)(run / unit);
  long long units = run / unit;
  for (; k < n; ++k, ++R->dims) {
    R->n[R->dims] = d[k].first;
    R->stride[R->dims] = d[k].second;
    invariant_divisor(d[k].first, &R->mul[R->dims], &R->shift[R->dims]);
    units *= d[k].first;
  }
  if (run / unit > 1 << 30 || units > 1 << 30) return false;               // (and a chunk beyond the last unit fits 32 bits)
  R->units = (int)units;
  invariant_divisor(R->run, &R->run_mul, &R->run_shift);
  return true;
}

static int copy_call(const CacheView &C, const int32_t *pairs, int max_pairs, const int32_t *done, void *stream) {
  if (!pairs || !done || max_pairs < 1) return COMPACTOR_EINVAL;
  if ((reinterpret_cast<uintptr_t>(pairs) & 7u) || (reinterpret_cast<uintptr_t>(done) & 3u)) return COMPACTOR_EALIGN;
  Copy P{};
  P.pairs = reinterpret_cast<const int2 *>(pairs);
  P.done = done;
  P.most = max_pairs;
  P.rows[0] = reinterpret_cast<char *>(C.k);
  P.rows[1] = reinterpret_cast<char *>(C.v);
  const bool fp4 = C.k_scales != nullptr;
  auto add = [&](void *p) { P.state[P.states++] = static_cast<char *>(p); };
  if (C.mass != nullptr) add(C.mass), add(C.positions);
  if (fp4) add(C.k_scales), add(C.v_scales);
  if (!runs_of(2 * C.page_stride, fp4 ? 2 * ROW4 : 2 * D, 16,
               {{C.page_size, 2 * C.slot_stride}, {C.kv_heads, 2 * C.head_stride}, {C.layers, 2 * C.layer_stride}}, &P.row))
    return COMPACTOR_EINVAL;
  if (!runs_of(4 * C.state_page_stride, 4ll * C.page_size, 4, {{C.kv_heads, 4 * C.state_head_stride}, {C.layers, 4 * C.state_layer_stride}}, &P.word))
    return COMPACTOR_EINVAL;
  constexpr int each = 256 * COPY_AT_ONCE;
  P.row_chunks = (int)(((long long)P.row.units + each - 1) / each);
  P.chunks = 2 * P.row_chunks + (P.states > 0 ? (int)(((long long)P.word.units + each - 1) / each) : 0);
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0)
    cus = 256;
  const unsigned blocks = (unsigned)std::min((long long)max_pairs * P.chunks, (long long)COPY_WORKGROUPS * cus);
  (void)hipGetLastError();   // a leftover of earlier, unrelated HIP calls is not this call's error
  hipLaunchKernelGGL(copy_kernel, dim3(blocks), dim3(256), 0, static_cast<hipStream_t>(stream), C, P);
  return hipGetLastError() == hipSuccess ? COMPACTOR_OK : COMPACTOR_EHIP;
}

// The view of a cache whose tables a call writes.
static int pages_view(const compactor_cache_t *cache, CacheNeed need, CacheView *C) {
  const int rc = cache_view(cache, need, C);
  if (rc) return rc;
  const bool fits = C->nreq <= PAGES_MOST && C->num_pages <= POOL_MOST && (long long)C->nreq * cache->table_len <= ENTRIES_MOST;
  return fits ? COMPACTOR_OK : COMPACTOR_EINVAL;
}

static size_t up(size_t x) { return (x + 255) / 256 * 256; }

// Workspace of a reserve; ws null: only its size.
static size_t reserve_scratch(const CacheView &C, int table_len, unsigned char *ws, Reserve *R) {
  size_t at = 0;
  auto take = [&](size_t bytes) {
    unsigned char *p = ws + at;
    at += up(bytes);
    return p;
  };
  const size_t entries = (size_t)C.nreq * table_len, pages = C.num_pages;
  R->spans = reinterpret_cast<int4 *>(take(C.nreq * sizeof(int4)));
  R->entries = reinterpret_cast<int *>(take(entries * 4));
  R->kinds = reinterpret_cast<int *>(take(entries * 4));
  R->pages = reinterpret_cast<int *>(take(entries * 4));
  R->tally = reinterpret_cast<int *>(take(pages * 4));
  R->last = reinterpret_cast<int *>(take(pages * 4));
  R->free_pages = reinterpret_cast<int *>(take(std::min(entries, pages) * 4));
  return at;
}

static bool on4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
static bool on8(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }

}  // namespace cmp

using namespace cmp;

extern "C" {
#pragma GCC visibility push(default)

int compactor_pages_reserve_workspace_size(const compactor_cache_t *cache, size_t *bytes) {
  CacheView C;
  const int rc = pages_view(cache, CACHE_SIZES, &C);
  if (rc) return rc;
  if (!bytes) return COMPACTOR_EINVAL;
  Reserve R;
  *bytes = reserve_scratch(C, cache->table_len, nullptr, &R);
  return COMPACTOR_OK;
}

int compactor_pages_reserve(const compactor_cache_t *cache, const compactor_pages_reserve_params_t *reserve, void *workspace, size_t workspace_bytes,
                            void *stream) {
  CacheView C;
  const int rc = pages_view(cache, CACHE_TABLES, &C);
  if (rc) return rc;
  if (!reserve || !reserve->refs || !reserve->pairs || !reserve->done || reserve->tokens < 0) return COMPACTOR_EINVAL;
  if (!on4(reserve->refs) || !on4(reserve->new_tokens) || !on8(reserve->pairs) || !on4(reserve->done)) return COMPACTOR_EALIGN;
  Reserve R;
  const size_t need = reserve_scratch(C, cache->table_len, static_cast<unsigned char *>(workspace), &R);
  if (!workspace || workspace_bytes < need) return COMPACTOR_EWORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return COMPACTOR_EALIGN;
  R.tables = const_cast<int32_t *>(cache->tables);
  R.refs = reserve->refs;
  R.new_tokens = reserve->new_tokens;
  R.tokens = reserve->tokens;
  R.own_all = reserve->own_all;
  R.table_len = cache->table_len;
  R.pairs = reinterpret_cast<int2 *>(reserve->pairs);
  R.done = reserve->done;
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();   // a leftover of earlier, unrelated HIP calls is not this call's error
  if (C.nreq <= FEW_REQUESTS && (long long)C.nreq * C.layers * C.kv_heads <= FEW_COUNTS) {
    hipLaunchKernelGGL(reserve_few_kernel, dim3(1), dim3(PLAN_THREADS), 0, st, C, R);
  } else {
    hipLaunchKernelGGL(reserve_spans_kernel, dim3((unsigned)C.nreq), dim3(256), 0, st, C, R);
    if (hipGetLastError() != hipSuccess) return COMPACTOR_EHIP;
    hipLaunchKernelGGL(reserve_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, st, C, R);
  }
  return hipGetLastError() == hipSuccess ? COMPACTOR_OK : COMPACTOR_EHIP;
}

int compactor_pages_copy(const compactor_cache_t *cache, const int32_t *pairs, int32_t max_pairs, const int32_t *done, void *stream) {
  CacheView C;
  const int rc = cache_view(cache, CACHE_ROWS, &C);
  return rc ? rc : copy_call(C, pairs, max_pairs, done, stream);
}

int compactor_mx_pages_copy(const compactor_mx_cache_t *cache, const int32_t *pairs, int32_t max_pairs, const int32_t *done, void *stream) {
  CacheView C;
  const int rc = cache_view(cache, CACHE_ROWS, &C);
  return rc ? rc : copy_call(C, pairs, max_pairs, done, stream);
}

int compactor_pages_fork(const compactor_cache_t *cache, int32_t *refs, const int32_t *parents, void *stream) {
  CacheView C;
  const int rc = pages_view(cache, CACHE_TABLES, &C);
  if (rc) return rc;
  if (!refs || !parents) return COMPACTOR_EINVAL;
  if (!on4(refs) || !on4(parents)) return COMPACTOR_EALIGN;
  Fork F{const_cast<int32_t *>(cache->tables), refs, parents, cache->table_len, 6, 0, 0};
  while (F.width_log > 0 && (C.nreq << F.width_log) > FORK_NUMBERS / (F.width_log > 3 ? 16 : 1)) --F.width_log;
  const int width = 1 << F.width_log, heads = C.layers * C.kv_heads;
  F.table_strips = (cache->table_len + width - 1) / width;
  F.head_strips = (heads + width - 1) / width;
  const long long blocks = F.table_strips + (long long)F.head_strips * (C.seen != nullptr ? 2 : 1);
  if (!launchable(blocks, 256)) return COMPACTOR_EINVAL;
  (void)hipGetLastError();   // a leftover of earlier, unrelated HIP calls is not this call's error
  hipLaunchKernelGGL(fork_kernel, dim3((unsigned)blocks), dim3(256), (size_t)(C.nreq << F.width_log) * 4, static_cast<hipStream_t>(stream), C, F);
  return hipGetLastError() == hipSuccess ? COMPACTOR_OK : COMPACTOR_EHIP;
}

int compactor_pages_release(const compactor_cache_t *cache, int32_t *refs, const int32_t *finished, void *stream) {
  CacheView C;
  const int rc = pages_view(cache, CACHE_TABLES, &C);
  if (rc) return rc;
  if (!refs) return COMPACTOR_EINVAL;
  if (!on4(refs) || !on4(finished)) return COMPACTOR_EALIGN;
  (void)hipGetLastError();   // a leftover of earlier, unrelated HIP calls is not this call's error
  hipLaunchKernelGGL(release_kernel, dim3((unsigned)C.nreq), dim3(256), 0, static_cast<hipStream_t>(stream), C, const_cast<int32_t *>(cache->tables),
                     cache->table_len, refs, finished);
  return hipGetLastError() == hipSuccess ? COMPACTOR_OK : COMPACTOR_EHIP;
}

int compactor_pages_compact_workspace_size(const compactor_cache_t *cache, size_t *bytes) {
  CacheView C;
  const int rc = pages_view(cache, CACHE_SIZES, &C);
  if (rc) return rc;
  if (!bytes) return COMPACTOR_EINVAL;
  *bytes = up(((size_t)C.num_pages + 1) * 4);
  return COMPACTOR_OK;
}

int compactor_pages_compact(const compactor_cache_t *cache, int32_t *refs, int32_t *pairs, int32_t *done, void *workspace, size_t workspace_bytes,
                            void *stream) {
  CacheView C;
  const int rc = pages_view(cache, CACHE_TABLES, &C);
  if (rc) return rc;
  if (!refs || !pairs || !done) return COMPACTOR_EINVAL;
  if (!on4(refs) || !on8(pairs) || !on4(done)) return COMPACTOR_EALIGN;
  if (!workspace || workspace_bytes < up(((size_t)C.num_pages + 1) * 4)) return COMPACTOR_EWORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return COMPACTOR_EALIGN;
  const Compact K{const_cast<int32_t *>(cache->tables), refs, cache->table_len, reinterpret_cast<int2 *>(pairs), done, static_cast<int *>(workspace)};
  const long long entries = (long long)C.nreq * cache->table_len;
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();   // a leftover of earlier, unrelated HIP calls is not this call's error
  hipLaunchKernelGGL(compact_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, st, C, K);
  if (hipGetLastError() != hipSuccess) return COMPACTOR_EHIP;
  hipLaunchKernelGGL(compact_tables_kernel, dim3((unsigned)((entries + 255) / 256)), dim3(256), 0, st, C, K);
  return hipGetLastError() == hipSuccess ? COMPACTOR_OK : COMPACTOR_EHIP;
}

#pragma GCC visibility pop
}  // extern "C"
