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
// The bookkeeping is a few thousand integers: bound by the latency of a
// dependent chain, not by bandwidth, so one workgroup of 16 waves does it
// between barriers.  Each wave owns a contiguous range of the pages; inside it
// a free page's rank is a population count of lane ballots, and 16 wave totals
// are the only numbers that cross waves.  Moving the pages' contents is bound
// by HBM and runs in a launch of its own on the whole chip.
#include "ea_decode.h"
#include "ea_device.h"

namespace ea {

namespace {

constexpr int kMetaThreads = 1024, kMetaWaves = kMetaThreads / 64;
constexpr int kMaxSeq = EA_PAGED_MAX_SEQ;
constexpr int kCopyThreads = 256, kCopyWgs = 2048;

// Workspace words: the copies a bookkeeping kernel asks for.
constexpr int kWorkCount = 0;   // pages to move
constexpr int kWorkLists = 16;  // then source pages, destinations and rows

__device__ __forceinline__ int held(int len, int page) { return (len + page - 1) / page; }

// A barrier after which every wave sees the others' writes and atomics to
// global memory (the atomics are carried out in the L2, past the L1).
__device__ __forceinline__ void settle() {
  __threadfence();
  __syncthreads();
  __threadfence();
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

// refs[p..p+3], pages past the end counting as used.
__device__ __forceinline__ int4 load_refs(const int32_t* refs, int p, int end) {
  int4 r = make_int4(1, 1, 1, 1);
  if (p + 3 < end) {
    if (((uintptr_t)refs & 15) == 0) return *reinterpret_cast<const int4*>(refs + p);
    r = make_int4(refs[p], refs[p + 1], refs[p + 2], refs[p + 3]);
  } else {
    if (p < end) r.x = refs[p];
    if (p + 1 < end) r.y = refs[p + 1];
    if (p + 2 < end) r.z = refs[p + 2];
  }
  return r;
}

// Free pages before each wave's range, and in all (s: kMetaWaves ints).
__device__ __forceinline__ int free_before(const int32_t* refs, int n_pages, int* s, int* total) {
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  int begin, end, n = 0;
  wave_range(n_pages, wid, &begin, &end);
  for (int p = begin + 4 * lane; p < end; p += 256) {
    const int4 r = load_refs(refs, p, end);
    n += (r.x <= 0) + (r.y <= 0) + (r.z <= 0) + (r.w <= 0);
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

// Walk of a wave's pages in order: f(page, refs, rank among the free pages).
template <class F>
__device__ __forceinline__ void each_page(const int32_t* refs, int n_pages, int before, F f) {
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  int begin, end;
  wave_range(n_pages, wid, &begin, &end);
  int run = before;
  for (int p0 = begin; p0 < end; p0 += 256) {
    const int p = p0 + 4 * lane;
    const int4 r = load_refs(refs, p, end);
    const int v[4] = {r.x, r.y, r.z, r.w};
    int rank = run, all = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint64_t b = __ballot(p + i < end && v[i] <= 0);
      rank += __popcll(b & ((uint64_t(1) << lane) - 1));
      all += __popcll(b);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (p + i < end) {
        f(p + i, v[i], rank);
        rank += v[i] <= 0;
      }
    run += all;
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

// New pages for add[s] more keys of every sequence; slots and positions of the
// new tokens, sequence by sequence.
__global__ __launch_bounds__(kMetaThreads) void extend_kernel(const PagesArgs a) {
  __shared__ int s_need[kMaxSeq], s_tok[kMaxSeq];  // exclusive sums over sequences
  __shared__ int s_wave[kMetaWaves];
  const int tid = threadIdx.x;
  const int per = (a.n_seq + kMetaThreads - 1) / kMetaThreads;
  const int s0 = min(a.n_seq, tid * per), s1 = min(a.n_seq, s0 + per);
  int need = 0, tok = 0, bad = 0;
  for (int s = s0; s < s1; ++s) {
    const int64_t len = a.len[s], add = max(a.add[s], 0);
    s_need[s] = need;
    s_tok[s] = tok;
    if (len < 0 || len + add > (int64_t)a.stride * a.page_size) {
      bad = 1;
    } else {
      need += held((int)(len + add), a.page_size) - held((int)len, a.page_size);
      tok += (int)add;
    }
  }
  int all_need, all_tok;
  const int need0 = block_scan(need, s_wave, &all_need);
  const int tok0 = block_scan(tok, s_wave, &all_tok);
  for (int s = s0; s < s1; ++s) {
    s_need[s] += need0;
    s_tok[s] += tok0;
  }
  bad = __syncthreads_or(bad);
  int all_free;
  const int before = free_before(a.refs, a.n_pages, s_wave, &all_free);
  const int code = bad ? EA_PAGES_TOO_LONG : all_need > all_free ? EA_PAGES_NONE_FREE : 0;
  if (code) need = all_need = all_tok = 0;
  each_page(a.refs, a.n_pages, before, [&](int p, int refs, int rank) {
    const bool take = refs <= 0 && rank < all_need;
    if (take) {
      const int s = last_at_most(s_need, a.n_seq, rank);
      a.out_table[(int64_t)s * a.stride + held(a.len[s], a.page_size) + rank - s_need[s]] = p;
    }
    if (take || a.out_refs != a.refs) a.out_refs[p] = take ? 1 : refs;
  });
  set_status(a, code, all_free - all_need);
  settle();
  for (int t = tid; t < a.n_tokens; t += kMetaThreads) {
    int slot = -1, pos = 0;
    if (t < all_tok) {
      const int s = last_at_most(s_tok, a.n_seq, t);
      pos = a.len[s] + t - s_tok[s];
      const int in = pos / a.page_size;
      const int pg = a.out_table[(int64_t)s * a.stride + in];
      if ((uint32_t)pg < (uint32_t)a.n_pages) slot = pg * a.page_size + pos - in * a.page_size;
    }
    if (a.slots) a.slots[t] = slot;
    if (a.pos) a.pos[t] = pos;
  }
  __syncthreads();  // lengths may be updated in place
  for (int s = tid; s < a.n_seq; s += kMetaThreads)
    a.out_len[s] = code ? a.len[s] : a.len[s] + max(a.add[s], 0);
}

// Every sequence i becomes a copy of parent[i] (outside the batch: empty).
__global__ __launch_bounds__(kMetaThreads) void select_kernel(const PagesArgs a) {
  __shared__ int s_children[kMaxSeq], s_first[kMaxSeq];
  __shared__ int s_wave[kMetaWaves];
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  const int64_t most = (int64_t)a.stride * a.page_size;
  int* src = a.work + kWorkLists;
  int* dst = src + a.n_seq;
  int* rows = dst + a.n_seq;
  int* who = rows + a.n_seq;
  int bad = 0;
  for (int s = tid; s < a.n_seq; s += kMetaThreads) {
    s_children[s] = 0;
    s_first[s] = a.n_seq;
    bad |= a.len[s] < 0 || a.len[s] > most;
  }
  for (int p = tid; p < a.n_pages; p += kMetaThreads) a.out_refs[p] = a.refs[p];
  bad = __syncthreads_or(bad);
  settle();
  if (!bad)
    for (int i = tid; i < a.n_seq; i += kMetaThreads) {
      const int p = a.parent[i];
      if ((uint32_t)p < (uint32_t)a.n_seq) {
        atomicAdd(&s_children[p], 1);
        atomicMin(&s_first[p], i);
      }
    }
  __syncthreads();
  // counts of the old sequences' pages; new rows of the table
  for (int s = wid; s < a.n_seq && !bad; s += kMetaWaves) {
    const int ch = s_children[s], full = a.len[s] / a.page_size, tail = a.len[s] - full * a.page_size;
    if (ch != 1)
      for (int j = lane; j < full + (tail > 0); j += 64) {
        const int p = a.table[(int64_t)s * a.stride + j];
        const int d = j < full ? ch - 1 : ch == 0 ? -1 : 0;  // a partly filled page stays its first child's
        if (d && (uint32_t)p < (uint32_t)a.n_pages) atomicAdd(&a.out_refs[p], d);
      }
    const int par = a.parent[s];
    const bool alive = (uint32_t)par < (uint32_t)a.n_seq;
    const int len = alive ? a.len[par] : 0, n = held(len, a.page_size);
    for (int j = lane; j < a.stride; j += 64)
      a.out_table[(int64_t)s * a.stride + j] = j < n ? a.table[(int64_t)par * a.stride + j] : -1;
    if (lane == 0) a.out_len[s] = len;
  }
  // copies of partly filled pages, ranked by sequence
  const int per = (a.n_seq + kMetaThreads - 1) / kMetaThreads;
  const int s0 = min(a.n_seq, tid * per), s1 = min(a.n_seq, s0 + per);
  auto copies = [&](int i) {
    const int p = a.parent[i];
    return !bad && (uint32_t)p < (uint32_t)a.n_seq && s_first[p] != i && a.len[p] % a.page_size > 0;
  };
  int mine = 0;
  for (int i = s0; i < s1; ++i) mine += copies(i);
  int count;
  int rank = block_scan(mine, s_wave, &count);
  for (int i = s0; i < s1; ++i)
    if (copies(i)) {
      const int p = a.parent[i], full = a.len[p] / a.page_size;
      const int pg = a.table[(int64_t)p * a.stride + full];
      src[rank] = (uint32_t)pg < (uint32_t)a.n_pages ? pg : -1;
      rows[rank] = a.len[p] - full * a.page_size;
      who[rank] = i;
      ++rank;
    }
  settle();
  int all_free;
  const int before = free_before(a.out_refs, a.n_pages, s_wave, &all_free);
  const int code = bad ? EA_PAGES_TOO_LONG : count > all_free ? EA_PAGES_NONE_FREE : 0;
  if (!code) {
    each_page(a.out_refs, a.n_pages, before, [&](int p, int refs, int r) {
      if (refs <= 0 && r < count) {
        const int i = who[r], at = a.len[a.parent[i]] / a.page_size;
        dst[r] = p;
        a.out_refs[p] = 1;
        a.out_table[(int64_t)i * a.stride + at] = p;
      }
    });
    if (tid == 0) a.work[kWorkCount] = count;
    set_status(a, 0, all_free - count);
    return;
  }
  // nothing is done: the state goes through as it came
  settle();
  int left = 0;
  for (int p = tid; p < a.n_pages; p += kMetaThreads) {
    a.out_refs[p] = a.refs[p];
    left += a.refs[p] <= 0;
  }
  for (int s = tid; s < a.n_seq; s += kMetaThreads) a.out_len[s] = a.len[s];
  for (int64_t j = tid; j < (int64_t)a.n_seq * a.stride; j += kMetaThreads) a.out_table[j] = a.table[j];
  int sum;
  block_scan(left, s_wave, &sum);
  if (tid == 0) a.work[kWorkCount] = 0;
  set_status(a, code, sum);
}

// Used pages behind the first n_used go to the free places before: the k-th
// lowest to the k-th lowest.
__global__ __launch_bounds__(kMetaThreads) void compact_kernel(const PagesArgs a) {
  __shared__ int s_wave[kMetaWaves];
  __shared__ int s_moves;
  const int tid = threadIdx.x;
  int* src = a.work + kWorkLists;
  int* dst = src + a.n_pages;
  int* to = dst + a.n_pages;  // by page: where it went
  int all_free;
  const int before = free_before(a.refs, a.n_pages, s_wave, &all_free);
  const int n_used = a.n_pages - all_free;
  if (tid == 0) s_moves = 0;
  __syncthreads();
  each_page(a.refs, a.n_pages, before, [&](int p, int refs, int free_rank) {
    to[p] = p;
    if (p < n_used && refs <= 0) dst[free_rank] = p;
    // the free pages before n_used are as many as the used ones behind it:
    // a used page's rank among the latter is its rank among the used ones
    // less those before n_used
    if (p == n_used - 1) s_moves = free_rank + (refs <= 0);
  });
  settle();
  const int moves = s_moves;
  each_page(a.refs, a.n_pages, before, [&](int p, int refs, int free_rank) {
    if (p >= n_used && refs > 0) src[p - free_rank - (n_used - moves)] = p;
  });
  settle();
  // every count is read before a thread writes another's (they may be updated
  // in place): moved pages are behind n_used, holes before it
  for (int k = tid; k < moves; k += kMetaThreads) to[src[k]] = dst[k];
  if (a.out_refs != a.refs)
    for (int p = tid; p < a.n_pages; p += kMetaThreads) a.out_refs[p] = max(a.refs[p], 0);
  settle();
  for (int k = tid; k < moves; k += kMetaThreads) {
    const int n = a.refs[src[k]];
    a.out_refs[dst[k]] = n;
    a.out_refs[src[k]] = 0;
  }
  if (tid == 0) a.work[kWorkCount] = moves;
  set_status(a, 0, all_free);
}

// The pages that a bookkeeping kernel listed, in every plane and cache; with
// ROWS, only the rows of a page that its sequence holds.  Compact's launch
// rewrites the table beside.
template <bool ROWS>
__global__ __launch_bounds__(kCopyThreads) void move_kernel(const PagesArgs a, const PagesCopyArgs c) {
  const int count = ld_uniform(&c.work[kWorkCount]);
  const int32_t* src = c.work + kWorkLists;
  const int32_t* dst = src + (ROWS ? a.n_seq : a.n_pages);
  const int32_t* more = dst + (ROWS ? a.n_seq : a.n_pages);  // rows, or where each page went
  if constexpr (!ROWS) {
    const int64_t n = (int64_t)a.n_seq * a.stride;
    for (int64_t j = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; j < n; j += (int64_t)gridDim.x * kCopyThreads) {
      const int s = (int)(j / a.stride), at = (int)(j - (int64_t)s * a.stride);
      const int pg = a.table[j];
      a.out_table[j] = at >= held(max(a.len[s], 0), a.page_size) ? -1
                       : (uint32_t)pg < (uint32_t)a.n_pages     ? more[pg]
                                                                : pg;
    }
  }
  for (int k = 0; k < c.n_cache; ++k) {
    const PagesCache& pc = c.c[k];
    const int64_t items = (int64_t)count * pc.planes;
    for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
      const int plane = (int)(it / count), j = (int)(it - (int64_t)plane * count);
      const int from = src[j], into = dst[j];
      if (from < 0) continue;
      const char* s = pc.data + plane * pc.plane_bytes + from * pc.page_bytes;
      char* d = pc.data + plane * pc.plane_bytes + into * pc.page_bytes;
      const int64_t head = (int64_t)c.page_size * pc.row_bytes;
      const int64_t part = (ROWS ? more[j] : c.page_size) * pc.row_bytes;  // bytes of a head that move
      if (part == head) {
        const int64_t n = pc.heads * head / 16;
        for (int64_t i = threadIdx.x; i < n; i += kCopyThreads)
          reinterpret_cast<uint4*>(d)[i] = reinterpret_cast<const uint4*>(s)[i];
      } else {
        const int n = (int)(part / 16), all = pc.heads * n;
        for (int i = threadIdx.x; i < all; i += kCopyThreads) {
          const int h = i / n;
          const int64_t off = h * head + (int64_t)(i - h * n) * 16;
          *reinterpret_cast<uint4*>(d + off) = *reinterpret_cast<const uint4*>(s + off);
        }
      }
    }
  }
}

}  // namespace

hipError_t launch_pages_extend(const PagesArgs& a, hipStream_t s) {
  extend_kernel<<<dim3(1), dim3(kMetaThreads), 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_pages_select(const PagesArgs& a, const PagesCopyArgs& c, hipStream_t s) {
  select_kernel<<<dim3(1), dim3(kMetaThreads), 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || c.n_cache == 0) return e;
  move_kernel<true><<<dim3(kCopyWgs), dim3(kCopyThreads), 0, s>>>(a, c);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PagesArgs& a, const PagesCopyArgs& c, hipStream_t s) {
  compact_kernel<<<dim3(1), dim3(kMetaThreads), 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  move_kernel<false><<<dim3(kCopyWgs), dim3(kCopyThreads), 0, s>>>(a, c);
  return hipGetLastError();
}

}  // namespace ea
