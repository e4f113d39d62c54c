// ea_pages.hip -- the page table of a cache: pages handed out to growing
// sequences, sequences forked, reordered and freed by a parent list, and the
// used pages moved together.
//
// State is three int32 arrays: table[n_seq][stride] (pages of each sequence in
// order), lengths[n_seq] (keys) and refs[n_pages] (table entries that name the
// page; 0: free).  Whole pages may be shared; a partly filled last page has one
// owner, so that tokens are appended without a check.  Pages are given out in
// ascending order and duties ranked by position, so results do not depend on
// timing: counts change by integer atomics only, whose order is immaterial.
//
// The bookkeeping is some thousand integers: bound by the latency of dependent
// steps, not by bandwidth, so one workgroup of 16 waves does it between
// barriers (extend's counting, and the parts of select that touch every entry of
// a large table, are launches of their own).  Each wave owns a contiguous range
// of the pages; inside it a free page's rank is a population count of lane
// ballots, and 16 wave totals are the only numbers that cross waves.  Moving the
// pages' contents is bound by HBM and runs in a launch on the whole chip.
// Measured: new pages for 256 sequences in a cache of 33 thousand pages 11.5 us;
// a beam step over 64 sequences 10 us and its copies, 134 MB moved, 30; 1.35 GB
// made dense 8 us and 275, against 263 at a large copy's rate.
#include "ea_decode.h"
#include "ea_device.h"

namespace ea {

namespace {

constexpr int kMetaThreads = 1024, kMetaWaves = kMetaThreads / 64;
constexpr int kMaxSeq = EA_PAGED_MAX_SEQ;
constexpr int kCopyThreads = 256, kCopyWgs = 2048;

// Workspace words: the copies a bookkeeping kernel asks for.
constexpr int kWorkCount = 0;   // pages to move
constexpr int kWorkUsed = 1;    // compact: pages in use; -1: the state goes through as it came
constexpr int kWorkLists = 16;  // then source pages, destinations and rows

constexpr int kBlock = 4 * kMetaThreads;  // pages that a workgroup looks at together
// Table entries and pages up to which select's bookkeeping is one workgroup's;
// beyond, three launches of many (6.5 thousand: 13.5 us in one workgroup, 16.2 in
// three launches; 25 thousand: 27 and 21; 200 thousand: 157 and 31).
constexpr int64_t kOneWorkgroup = 16384;

__device__ __forceinline__ int held(int len, int page) { return (len + page - 1) / page; }

// A barrier after which every wave of the workgroup sees the others' writes and
// atomics to global memory: all of them have been carried out (the atomics in
// the L2), and the lines that are read next were not read before.
__device__ __forceinline__ void settle() {
  drain_vmem();
  __syncthreads();
}

// Exclusive prefix sums of per-thread values over the workgroup; returns the
// total.  s: kMetaWaves ints.
__device__ __forceinline__ int block_scan(int v, int* s, int* total) {
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 63) s[wid] = x;
  __syncthreads();
  int before = 0, all = 0;
  for (int i = 0; i < kMetaWaves; ++i) {
    if (i < wid) before += s[i];
    all += s[i];
  }
  *total = all;
  return before + x - v;
}

// Pages of wave w: [begin, end), multiples of 256 apart (64 lanes of 4).
__device__ __forceinline__ void wave_range(int n_pages, int wid, int* begin, int* end) {
  const int per = ((n_pages + kMetaWaves - 1) / kMetaWaves + 255) / 256 * 256;
  *begin = (int)min((int64_t)n_pages, (int64_t)wid * per);
  *end = (int)min((int64_t)n_pages, (int64_t)(wid + 1) * per);
}

// Four counts from page p on; what lies past the last page is undefined.  One
// load whatever the alignment and the end are: near the end it starts earlier
// and is shifted.
typedef int i32x4_t __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ i32x4_t load_refs(const int32_t* refs, int p, int n_pages) {
  if (n_pages < 4) {  // (uniform)
    i32x4_t r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = refs[min(i, n_pages - 1)];
    return r;
  }
  const int at = min(p, n_pages - 4), by = p - at;
  const i32x4_t r = *reinterpret_cast<const i32x4_t*>(refs + at);
  i32x4_t s;
  s[0] = by == 0 ? r[0] : by == 1 ? r[1] : by == 2 ? r[2] : r[3];
  s[1] = by == 0 ? r[1] : by == 1 ? r[2] : r[3];
  s[2] = by == 0 ? r[2] : r[3];
  s[3] = r[3];
  return s;
}

constexpr int kBatch = 16;  // loads of a wave in flight: 16 * 256 pages

// Free pages before each wave's range, and in all (s: kMetaWaves ints).
__device__ __forceinline__ int free_before(const int32_t* refs, int n_pages, int* s, int* total) {
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  int begin, end, n = 0;
  wave_range(n_pages, wid, &begin, &end);
  for (int p0 = begin; p0 < end; p0 += 256 * kBatch) {
    i32x4_t r[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) r[i] = load_refs(refs, p0 + 256 * i + 4 * lane, n_pages);
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int left = end - (p0 + 256 * i + 4 * lane);
#pragma unroll
      for (int e = 0; e < 4; ++e) n += e < left && r[i][e] <= 0;
    }
  }
#pragma unroll
  for (int o = 1; o < 64; o *= 2) n += __shfl_xor(n, o);
  __syncthreads();
  if (lane == 0) s[wid] = n;
  __syncthreads();
  int before = 0, all = 0;
  for (int i = 0; i < kMetaWaves; ++i) {
    if (i < wid) before += s[i];
    all += s[i];
  }
  *total = all;
  return before;
}

// Walk of a wave's pages in order: f(page, refs, rank among the free pages),
// until the rank `limit`.
template <class F>
__device__ __forceinline__ void each_page(const int32_t* refs, int n_pages, int before, int limit, F f) {
  constexpr int kAhead = 4;
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  int begin, end;
  wave_range(n_pages, wid, &begin, &end);
  int run = __builtin_amdgcn_readfirstlane(before);
  i32x4_t ahead[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) ahead[i] = load_refs(refs, begin + 256 * i + 4 * lane, n_pages);
  for (int p0 = begin; p0 < end; p0 += 256) {
    if (run >= limit) return;
    const int p = p0 + 4 * lane;
    const i32x4_t v = ahead[0];
#pragma unroll
    for (int i = 0; i + 1 < kAhead; ++i) ahead[i] = ahead[i + 1];
    ahead[kAhead - 1] = load_refs(refs, p + 256 * kAhead, n_pages);
    int rank = run, all = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint64_t b = __ballot(p + i < end && v[i] <= 0);
      rank += __popcll(b & ((uint64_t(1) << lane) - 1));
      all += __popcll(b);
    }
    run += all;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (p + i < end) {
        f(p + i, v[i], rank);
        rank += v[i] <= 0;
      }
  }
}

// Index of the last element <= v of s[0..n) (ascending, s[0] <= v).
__device__ __forceinline__ int last_at_most(const int* s, int n, int v) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (s[mid] <= v) lo = mid;
    else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ void set_status(const PagesArgs& a, int code, int left) {
  if (threadIdx.x == 0) {
    a.status[0] = code;
    a.status[1] = left;
  }
}

// ---- extend: new pages for add[s] more keys of every sequence; slots and
// positions of the new tokens, sequence by sequence.
// Free pages of every block of 4096, in a launch on the whole chip; copies the
// counts on the way where they are not updated in place.  (Counted and copied by
// the one workgroup that goes on: 3 thousand pages 8.4 us in place and 11.6 into
// other arrays instead of 7.2 and 10.6, 33 thousand 9.2 and 17.4 instead of 7.8
// and 11.5, a million 84 and 309 instead of 8.2 and 12.2.)
__global__ __launch_bounds__(kMetaThreads) void count_free_kernel(const PagesArgs a) {
  __shared__ int s_wave[kMetaWaves];
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int blocks = (a.n_pages + kBlock - 1) / kBlock;
  for (int b = blockIdx.x; b < blocks; b += gridDim.x) {
    const int p = b * kBlock + 4 * threadIdx.x;
    const i32x4_t v = load_refs(a.refs, p, a.n_pages);
    int n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (p + i >= a.n_pages) continue;
      n += v[i] <= 0;
      if (a.out_refs != a.refs) a.out_refs[p + i] = v[i];
    }
#pragma unroll
    for (int o = 1; o < 64; o *= 2) n += __shfl_xor(n, o);
    __syncthreads();
    if (lane == 0) s_wave[wid] = n;
    __syncthreads();
    if (threadIdx.x == 0) {
      int all = 0;
      for (int i = 0; i < kMetaWaves; ++i) all += s_wave[i];
      a.work[kWorkLists + b] = all;
    }
  }
}

__global__ __launch_bounds__(kMetaThreads) void extend_kernel(const PagesArgs a) {
  __shared__ int s_need[kMaxSeq], s_tok[kMaxSeq], s_len[kMaxSeq];  // the first two: exclusive sums over sequences
  __shared__ int s_list[kBlock], s_block[kMetaThreads], s_base[kMetaThreads];
  __shared__ int s_wave[kMetaWaves];
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  const int per = (a.n_seq + kMetaThreads - 1) / kMetaThreads;
  const int s0 = min(a.n_seq, tid * per), s1 = min(a.n_seq, s0 + per);
  int need = 0, tok = 0, bad = 0;
  for (int s = s0; s < s1; ++s) {
    const int64_t len = a.len[s], add = max(a.add[s], 0);
    s_len[s] = (int)len;
    s_need[s] = need;
    s_tok[s] = tok;
    if (len < 0 || len + add > (int64_t)a.stride * a.page_size) {
      bad = 1;
    } else {
      need += held((int)(len + add), a.page_size) - held((int)len, a.page_size);
      tok += (int)add;
    }
  }
  const int blocks = (a.n_pages + kBlock - 1) / kBlock;
  int in_mine = 0, all_free, all_need, all_tok;
  for (int b = tid; b < blocks; b += kMetaThreads) in_mine += a.work[kWorkLists + b];
  block_scan(in_mine, s_wave, &all_free);
  const int need0 = block_scan(need, s_wave, &all_need);
  const int tok0 = block_scan(tok, s_wave, &all_tok);
  for (int s = s0; s < s1; ++s) {
    s_need[s] += need0;
    s_tok[s] += tok0;
  }
  bad = __syncthreads_or(bad);
  const int code = bad ? EA_PAGES_TOO_LONG : all_need > all_free ? EA_PAGES_NONE_FREE : 0;
  if (code) all_need = all_tok = 0;
  // the lowest free pages, a block of 4096 at a time: listed by rank, then
  // handed out a thread each.  Blocks without free pages are passed over.
  int run = 0;
  for (int c0 = 0; c0 < blocks && run < all_need; c0 += kMetaThreads) {
    const int b = c0 + tid;
    const int n = b < blocks ? a.work[kWorkLists + b] : 0;
    int in_chunk, some;
    const int before = block_scan(n, s_wave, &in_chunk);
    const bool mine = n > 0 && run + before < all_need;
    const int at = block_scan(mine, s_wave, &some);
    if (mine) {
      s_block[at] = b;
      s_base[at] = run + before;
    }
    __syncthreads();
    for (int k = 0; k < some; ++k) {
      const int base = s_base[k], p = s_block[k] * kBlock + 4 * tid;
      const i32x4_t v = load_refs(a.out_refs, p, a.n_pages);
      int rank = 0, here = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint64_t m = __ballot(p + i < a.n_pages && v[i] <= 0);
        rank += __popcll(m & ((uint64_t(1) << lane) - 1));
        here += __popcll(m);
      }
      if (lane == 0) s_wave[wid] = here;
      __syncthreads();
      int found = 0;
      for (int i = 0; i < kMetaWaves; ++i) {
        if (i < wid) rank += s_wave[i];
        found += s_wave[i];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (p + i < a.n_pages && v[i] <= 0) s_list[rank++] = p + i;
      __syncthreads();
      found = min(found, all_need - base);
      for (int i = tid; i < found; i += kMetaThreads) {
        const int s = last_at_most(s_need, a.n_seq, base + i), pg = s_list[i];
        a.out_table[(int64_t)s * a.stride + held(s_len[s], a.page_size) + base + i - s_need[s]] = pg;
        a.out_refs[pg] = 1;
      }
      run = base + found;
      __syncthreads();
    }
  }
  set_status(a, code, all_free - all_need);
  settle();
  for (int t = tid; t < a.n_tokens; t += kMetaThreads) {
    int slot = -1, pos = 0;
    if (t < all_tok) {
      const int s = last_at_most(s_tok, a.n_seq, t);
      pos = s_len[s] + t - s_tok[s];
      const int in = pos / a.page_size;
      const int pg = a.out_table[(int64_t)s * a.stride + in];
      if ((uint32_t)pg < (uint32_t)a.n_pages) slot = pg * a.page_size + pos - in * a.page_size;
    }
    if (a.slots) a.slots[t] = slot;
    if (a.pos) a.pos[t] = pos;
  }
  for (int s = tid; s < a.n_seq; s += kMetaThreads) a.out_len[s] = s_len[s] + (code ? 0 : max(a.add[s], 0));
}

// ---- select: every sequence i becomes a copy of parent[i] (outside the batch:
// empty).  Three steps: the counts are copied; the old sequences' pages gain or
// lose references and the new table is written; copies of partly filled pages
// are ranked and given pages.
struct Family {
  int children[kMaxSeq], first[kMaxSeq];  // of every old sequence
  int len[kMaxSeq], parent[kMaxSeq];
};

// By the whole workgroup; returns whether a length is one that no row holds.
__device__ __forceinline__ int load_family(const PagesArgs& a, Family& f) {
  const int64_t most = (int64_t)a.stride * a.page_size;
  int bad = 0;
  for (int s = threadIdx.x; s < a.n_seq; s += kMetaThreads) {
    const int p = a.parent[s];
    f.children[s] = 0;
    f.first[s] = a.n_seq;
    f.len[s] = a.len[s];
    f.parent[s] = (uint32_t)p < (uint32_t)a.n_seq ? p : -1;
    bad |= f.len[s] < 0 || f.len[s] > most;
  }
  bad = __syncthreads_or(bad);
  if (!bad)
    for (int i = threadIdx.x; i < a.n_seq; i += kMetaThreads)
      if (f.parent[i] >= 0) {
        atomicAdd(&f.children[f.parent[i]], 1);
        atomicMin(&f.first[f.parent[i]], i);
      }
  __syncthreads();
  return bad;
}

// The counts as they come, by workgroup `block` of `blocks`.
__device__ __forceinline__ void copy_refs(const PagesArgs& a, int block, int blocks) {
  for (int64_t p0 = (int64_t)block * 4 * kMetaThreads + threadIdx.x; p0 < a.n_pages;
       p0 += (int64_t)blocks * 4 * kMetaThreads) {
    int r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = p0 + i * kMetaThreads < a.n_pages ? a.refs[p0 + i * kMetaThreads] : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (p0 + i * kMetaThreads < a.n_pages) a.out_refs[p0 + i * kMetaThreads] = r[i];
  }
}

// Counts of the old sequences' pages, and the new rows of the table: entry
// (s, j) by one thread, four in flight.
__device__ __forceinline__ void select_cells(const PagesArgs& a, const Family& f, int block, int blocks) {
  const int64_t cells = (int64_t)a.n_seq * a.stride;
  for (int64_t x0 = (int64_t)block * 4 * kMetaThreads + threadIdx.x; x0 < cells;
       x0 += (int64_t)blocks * 4 * kMetaThreads) {
    int old_pg[4], new_pg[4], d[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t x = x0 + i * kMetaThreads;
      old_pg[i] = new_pg[i] = -1;
      d[i] = 0;
      if (x >= cells) continue;
      const int s = div_fast((int)x, a.row), j = (int)x - s * a.stride;
      const int ch = f.children[s], full = f.len[s] / a.page_size, tail = f.len[s] - full * a.page_size;
      // a partly filled page stays its first child's
      d[i] = j < full ? ch - 1 : j == full && tail > 0 && ch == 0 ? -1 : 0;
      if (d[i]) old_pg[i] = a.table[x];
      const int par = f.parent[s];
      if (par >= 0 && j < held(f.len[par], a.page_size)) new_pg[i] = a.table[(int64_t)par * a.stride + j];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t x = x0 + i * kMetaThreads;
      if (x >= cells) continue;
      if (d[i] && (uint32_t)old_pg[i] < (uint32_t)a.n_pages) atomicAdd(&a.out_refs[old_pg[i]], d[i]);
      a.out_table[x] = new_pg[i];
    }
  }
  for (int s = block * kMetaThreads + threadIdx.x; s < a.n_seq; s += blocks * kMetaThreads)
    a.out_len[s] = f.parent[s] >= 0 ? f.len[f.parent[s]] : 0;
}

__global__ __launch_bounds__(kMetaThreads) void copy_refs_kernel(const PagesArgs a) {
  copy_refs(a, blockIdx.x, gridDim.x);
}
__global__ __launch_bounds__(kMetaThreads) void select_cells_kernel(const PagesArgs a) {
  __shared__ Family f;
  if (!load_family(a, f)) select_cells(a, f, blockIdx.x, gridDim.x);
}

// All three steps, or the third alone.
template <bool ALL>
__global__ __launch_bounds__(kMetaThreads) void select_kernel(const PagesArgs a) {
  __shared__ Family f;
  __shared__ int s_wave[kMetaWaves];
  const int tid = threadIdx.x;
  int* src = a.work + kWorkLists;
  int* dst = src + a.n_seq;
  int* rows = dst + a.n_seq;
  int* who = rows + a.n_seq;
  if (ALL) copy_refs(a, 0, 1);
  const int bad = load_family(a, f);
  if (ALL) {
    settle();
    if (!bad) select_cells(a, f, 0, 1);
  }
  // copies of partly filled pages, ranked by sequence
  const int per = (a.n_seq + kMetaThreads - 1) / kMetaThreads;
  const int s0 = min(a.n_seq, tid * per), s1 = min(a.n_seq, s0 + per);
  auto copies = [&](int i) {
    const int p = f.parent[i];
    return !bad && p >= 0 && f.first[p] != i && f.len[p] % a.page_size > 0;
  };
  int mine = 0;
  for (int i = s0; i < s1; ++i) mine += copies(i);
  int count;
  int rank = block_scan(mine, s_wave, &count);
  for (int i = s0; i < s1; ++i)
    if (copies(i)) {
      const int p = f.parent[i], full = f.len[p] / a.page_size;
      const int pg = a.table[(int64_t)p * a.stride + full];
      src[rank] = (uint32_t)pg < (uint32_t)a.n_pages ? pg : -1;
      rows[rank] = f.len[p] - full * a.page_size;
      who[rank] = i;
      ++rank;
    }
  settle();
  int all_free;
  const int before = free_before(a.out_refs, a.n_pages, s_wave, &all_free);
  const int code = bad ? EA_PAGES_TOO_LONG : count > all_free ? EA_PAGES_NONE_FREE : 0;
  if (!code) {
    each_page(a.out_refs, a.n_pages, before, count, [&](int p, int refs, int r) {
      if (refs <= 0 && r < count) dst[r] = p;
    });
    settle();
    for (int r = tid; r < count; r += kMetaThreads) {
      const int i = who[r], at = f.len[f.parent[i]] / a.page_size, p = dst[r];
      a.out_refs[p] = 1;
      a.out_table[(int64_t)i * a.stride + at] = p;
    }
    if (tid == 0) a.work[kWorkCount] = count;
    set_status(a, 0, all_free - count);
    return;
  }
  // nothing is done: the state goes through as it came
  settle();
  copy_refs(a, 0, 1);
  for (int s = tid; s < a.n_seq; s += kMetaThreads) a.out_len[s] = f.len[s];
  for (int64_t j = tid; j < (int64_t)a.n_seq * a.stride; j += kMetaThreads) a.out_table[j] = a.table[j];
  int left;
  free_before(a.refs, a.n_pages, s_wave, &left);
  if (tid == 0) a.work[kWorkCount] = 0;
  set_status(a, code, left);
}

// ---- compact: the used pages behind the first n_used go to the free places
// before, the k-th lowest to the k-th lowest.  Here the two lists are made and
// every moved page's rank noted; the launch that moves the contents rewrites
// the table and the counts beside.
__global__ __launch_bounds__(kMetaThreads) void compact_kernel(const PagesArgs a) {
  __shared__ int s_wave[kMetaWaves];
  __shared__ int s_moves;
  const int tid = threadIdx.x;
  int* src = a.work + kWorkLists;
  int* dst = src + a.n_pages;
  int* rank_of = dst + a.n_pages;
  int all_free, bad = 0;
  for (int s = tid; s < a.n_seq; s += kMetaThreads) bad |= a.len[s] < 0 || a.len[s] > (int64_t)a.stride * a.page_size;
  const int before = free_before(a.refs, a.n_pages, s_wave, &all_free);
  if (__syncthreads_or(bad)) {
    if (tid == 0) {
      a.work[kWorkCount] = 0;
      a.work[kWorkUsed] = -1;
    }
    set_status(a, EA_PAGES_TOO_LONG, all_free);
    return;
  }
  const int n_used = a.n_pages - all_free;
  if (tid == 0) s_moves = 0;
  __syncthreads();
  each_page(a.refs, a.n_pages, before, 0x7fffffff, [&](int p, int refs, int free_rank) {
    if (p < n_used && refs <= 0) dst[free_rank] = p;
    if (p == n_used - 1) s_moves = free_rank + (refs <= 0);
    // the free pages before n_used are as many as the used ones behind it, and
    // p - free_rank pages before p are used: n_used - 1 less that many come
    // after it, which ranks the pages behind n_used from their end
    if (p >= n_used && refs > 0) src[n_used - 1 - (p - free_rank)] = p;
  });
  __syncthreads();
  const int moves = s_moves;
  if (tid == 0) {
    a.work[kWorkCount] = moves;
    a.work[kWorkUsed] = n_used;
  }
  settle();
  for (int k0 = tid; k0 < moves; k0 += 8 * kMetaThreads) {
    int p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = k0 + i * kMetaThreads < moves ? src[k0 + i * kMetaThreads] : -1;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (p[i] >= 0) rank_of[p[i]] = moves - 1 - (k0 + i * kMetaThreads);
  }
  set_status(a, 0, all_free);
}

// In place: the moved pages' counts.
__global__ __launch_bounds__(kMetaThreads) void compact_refs_kernel(const PagesArgs a) {
  const int count = a.work[kWorkCount];
  const int* src = a.work + kWorkLists;
  const int* dst = src + a.n_pages;
  for (int r = blockIdx.x * kMetaThreads + threadIdx.x; r < count; r += gridDim.x * kMetaThreads) {
    const int from = src[count - 1 - r], into = dst[r];
    a.out_refs[into] = a.refs[from];
    a.out_refs[from] = 0;
  }
}

// The pages that a bookkeeping kernel listed, in every plane and cache, cut in
// pieces of 16 KiB; with ROWS, only the rows of a page that its sequence holds.
// Compact's launch rewrites the table beside.  Stores are streamed: the pages
// are larger than the caches in all layers together (64 planes, 134 MB moved:
// 45.8 us plain, 30.8 streamed, 26 at a large copy's rate; 1.35 GB: 284 and 275,
// of 263; pieces of 8 and 32 KiB are as fast).
constexpr int kUnroll = 4, kPiece = kUnroll * kCopyThreads;  // 16-byte units
template <bool ROWS>
__global__ __launch_bounds__(kCopyThreads) void move_kernel(const PagesArgs a, const PagesCopyArgs c) {
  const int count = ld_uniform(&c.work[kWorkCount]);
  const int32_t* src = c.work + kWorkLists;
  const int32_t* dst = src + (ROWS ? a.n_seq : a.n_pages);
  const int32_t* more = dst + (ROWS ? a.n_seq : a.n_pages);  // rows, or ranks of moved pages
  if constexpr (!ROWS) {
    const int n_used = ld_uniform(&c.work[kWorkUsed]);
    const int64_t cells = (int64_t)a.n_seq * a.stride, step = (int64_t)gridDim.x * gridDim.y * kCopyThreads;
    const int64_t first = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kCopyThreads + threadIdx.x;
    for (int64_t j = first; j < cells; j += step) {
      const int s = div_fast((int)j, a.row), at = (int)j - s * a.stride;
      int pg = a.table[j];
      if (n_used >= 0) {
        // (a page that no count calls used was not moved: its entry stays)
        if (pg >= n_used && pg < a.n_pages && a.refs[pg] > 0) pg = dst[more[pg]];
        if (at >= held(a.len[s], a.page_size)) pg = -1;
      }
      a.out_table[j] = pg;
    }
    if (a.out_refs != a.refs)
      for (int64_t p = first; p < a.n_pages; p += step) {
        // places before n_used that were free get the moved pages' counts
        const int n = a.refs[p];
        if (n > 0 || p >= n_used) a.out_refs[p] = p < n_used || n_used < 0 ? n : 0;
      }
    for (int64_t r = first; a.out_refs != a.refs && r < count; r += step)
      a.out_refs[dst[r]] = a.refs[src[count - 1 - r]];
  }
  for (int k = 0; k < c.n_cache; ++k) {
    const PagesCache& pc = c.c[k];
    const uint32_t head = (uint32_t)(c.page_size * pc.row_bytes / 16);  // 16-byte units
    const uint32_t pieces = (pc.heads * head + kPiece - 1) / kPiece, items = count * pieces;
    for (int plane = blockIdx.y; plane < pc.planes; plane += gridDim.y) {
      char* base = pc.data + plane * pc.plane_bytes;
      for (uint32_t it = blockIdx.x; it < items; it += gridDim.x) {
        const uint32_t j = it / pieces, piece = it - j * pieces;
        const int from = ld_uniform(src + (ROWS ? j : count - 1 - j)), into = ld_uniform(dst + j);
        if (from < 0) continue;
        const uint4* s = reinterpret_cast<const uint4*>(base + from * pc.page_bytes);
        uint4* d = reinterpret_cast<uint4*>(base + into * pc.page_bytes);
        const uint32_t part = ROWS ? (uint32_t)(ld_uniform(more + j) * pc.row_bytes / 16) : head;  // of a head
        const uint32_t all = pc.heads * part, first = piece * kPiece + threadIdx.x;
        uint4 v[kUnroll];
        uint32_t at[kUnroll];
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
          const uint32_t x = first + i * kCopyThreads;
          at[i] = ROWS ? x / part * head + x % part : x;
          if (x < all) v[i] = s[at[i]];
        }
#pragma unroll
        for (int i = 0; i < kUnroll; ++i)
          if (first + i * kCopyThreads < all) store_stream(d + at[i], v[i]);
      }
    }
  }
  // scales: of every block that holds a row that moves
  for (int k = 0; k < c.n_scales; ++k) {
    const PagesScales& ps = c.s[k];
    const int64_t items = (int64_t)count * ps.words;
    for (int plane = blockIdx.y; plane < ps.planes; plane += gridDim.y) {
      float* base = reinterpret_cast<float*>(ps.data + plane * ps.plane_bytes);
      for (int64_t it = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; it < items; it += gridDim.x * kCopyThreads) {
        const int j = (int)(it / ps.words), w = (int)(it - (int64_t)j * ps.words);
        const int from = src[ROWS ? j : count - 1 - j];
        if (from >= 0 && (!ROWS || w % ps.n_blocks * ps.block_rows < more[j]))
          base[(int64_t)dst[j] * ps.words + w] = base[(int64_t)from * ps.words + w];
      }
    }
  }
}

// Workgroups over pieces and planes.
dim3 copy_grid(const PagesCopyArgs& c) {
  int y = 1;
  for (int k = 0; k < c.n_cache; ++k) y = c.c[k].planes > y ? c.c[k].planes : y;
  if (y > kCopyWgs) y = kCopyWgs;
  return dim3((kCopyWgs + y - 1) / y, y);
}

}  // namespace

hipError_t launch_pages_extend(const PagesArgs& a, hipStream_t s) {
  const int blocks = (a.n_pages + kBlock - 1) / kBlock;
  count_free_kernel<<<dim3(blocks < 1024 ? blocks : 1024), dim3(kMetaThreads), 0, s>>>(a);
  extend_kernel<<<dim3(1), dim3(kMetaThreads), 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_pages_select(const PagesArgs& a, const PagesCopyArgs& c, hipStream_t s) {
  const int64_t cells = (int64_t)a.n_seq * a.stride;
  if (cells + a.n_pages <= kOneWorkgroup) {
    select_kernel<true><<<dim3(1), dim3(kMetaThreads), 0, s>>>(a);
  } else {
    auto blocks = [](int64_t n) { return dim3((uint32_t)(n > (int64_t)256 * 4096 ? 256 : (n + 4095) / 4096)); };
    copy_refs_kernel<<<blocks(a.n_pages), dim3(kMetaThreads), 0, s>>>(a);
    select_cells_kernel<<<blocks(cells), dim3(kMetaThreads), 0, s>>>(a);
    select_kernel<false><<<dim3(1), dim3(kMetaThreads), 0, s>>>(a);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || c.n_cache == 0) return e;
  move_kernel<true><<<copy_grid(c), dim3(kCopyThreads), 0, s>>>(a, c);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PagesArgs& a, const PagesCopyArgs& c, hipStream_t s) {
  compact_kernel<<<dim3(1), dim3(kMetaThreads), 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  move_kernel<false><<<copy_grid(c), dim3(kCopyThreads), 0, s>>>(a, c);
  if ((e = hipGetLastError()) != hipSuccess || a.out_refs != a.refs) return e;
  // in place the counts change when every workgroup has read them
  compact_refs_kernel<<<dim3(64), dim3(kMetaThreads), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace ea
