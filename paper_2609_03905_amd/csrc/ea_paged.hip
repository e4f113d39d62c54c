// ea_paged.hip -- attention of a batch's newest tokens over a paged cache,
// the keys that a group of sequences shares read once for the whole group.
//
// For a query row q of a sequence (one head) and the keys j it sees,
//   O = sum_j 2^(s_j - m) v_j / sum_j 2^(s_j - m),   s_j = scale log2(e) q.k_j
// Any split of the keys gives partial (m, l, O) that join as
//   m = max(m1, m2), l = l1 2^(m1-m) + l2 2^(m2-m), O likewise
// (the aggregation of the block attention), so a row's shared prefix and its
// own keys, and chunks of either, are worked on apart and joined at the end.
//
// A call is a set of segments: a group's shared keys under all of its rows,
// and each sequence's own keys under its rows.  A segment's query columns
// (rows x query heads of one key-value head) are cut in tiles; the keys of each
// (segment, head, tile) are walked in steps.  All steps of a pass lie end to
// end, and workgroup w of n takes the w-th n-th part of them, so that the work
// is even whatever the lengths are: a workgroup's part may end one tile's walk
// and begin the next one's, and a tile's walk has as many partial results as
// parts touch it.  The i-th tile's result from part w is slot i + w (one of the
// two grows from piece to piece).  The lengths are read on the device, by every
// workgroup for itself (a scan over the segments, 2.5 us), so a captured launch
// serves batches that grow.  Parts that run on one XCD are neighbours: tiles
// over the same keys then share its L2.
//
// Few columns (up to 32 a tile) are bound by HBM: 16 of D = 128 need
// 4 * 128 * 16 operations on a key's 512 bytes, a tenth of what the matrix cores
// do while the bytes arrive.  So nothing is staged in shared memory: each wave
// walks its own 32 keys of a step of 128 and loads K and V from the pages
// straight into the registers of
//   S^T = K Q^T     (16x16x32: A = 16 keys x 32 d, B = 32 d x 16 columns)
//   O^T += V^T P^T  (A = 16 d x 32 keys, B = 32 keys x 16 columns)
// The B operand of the second product holds eight keys a lane, and the
// accumulators of two S^T tiles hold exactly eight keys of that lane's column:
// keys 4g + i and 16 + 4g + i (g = lane / 16).  A product may take its k index
// in any order, so V is loaded for those eight keys, 8 (or 4) neighbouring d a
// lane, and turned in registers: d index 16 m + j' becomes row m of tile j'.
// The addresses of a wave's 32 key rows come from the page table, one lane a
// key, through shared memory, so that pages may be of any size; a step's table
// entries are read a step ahead.
//
// Measured (bf16 or fp16, 32 query heads over 8, D = 128): 48 sequences of up to
// 8K keys 148 us, 5.4 TB/s (5.1 is a large copy's rate); 64 sequences that share
// 8K keys 42 + 8 us (walk, join), 32 that share 64K 91 + 8 us, where the bytes
// take 20 and 66; one sequence of 1000 keys 10.1 us.  With every column tile
// reading the shared keys for itself those of shared keys took 92 and 213 us.
#include "ea_decode.h"
#include "ea_device.h"

namespace ea {

namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr float kLazyMax = 8.0f;  // log2 of the largest P: the running max moves only past this
// Weights are held 2^7 times as large in fp16: the largest of a walk is then from
// 2^7 to 2^15, and half the smallest step, what a small one may lose, 2^-32 or less
// of it (beside a weight of 1, 2^-26 would be nothing).  The factor is in
// every partial result's O and l alike.
template <bool BF>
constexpr float kRaise = BF ? 0.0f : 7.0f;

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

template <bool BF>
__device__ __forceinline__ f32x4_t mfma16(const uint4& a, const uint4& b, const f32x4_t& c) {
  if constexpr (BF)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b),
                                                   c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c,
                                                  0, 0, 0);
}

template <bool BF>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  return BF ? pack_bf16x2(a, b) : (uint32_t)f32_to_f16(a) | ((uint32_t)f32_to_f16(b) << 16);
}

// Two weights for the product with V, each as two values of the cache's type:
// the weight rounded, and what that leaves, rounded.  The first alone is off by
// half a step of the type (2^-8 of the weight in bf16, 2^-11 in fp16), as much
// as the output's own store; the two by half a step of half a step (2^-16 and
// 2^-22; in fp16 also by half the smallest step, see kRaise).  The sum takes the
// weights as they are.  Twice the products with V: 64 sequences that share 8K
// keys 46 to 47.5 us, 32 that share 64K 90 to 98; without shared keys no change.
template <bool BF>
__device__ __forceinline__ void split_p(float a, float b, uint32_t& hi, uint32_t& lo) {
  hi = pack2<BF>(a, b);
  if constexpr (BF) lo = pack2<BF>(a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xffff0000u));
  else lo = pack2<BF>(a - f16_to_f32((uint16_t)hi), b - f16_to_f32((uint16_t)(hi >> 16)));
}

// 0 V is no number where V is not finite: a value that a column does not see, or
// whose weight's second part is zero, would reach it through the product.  So
// every step's values are looked through; those that are not finite are taken
// out of the product and added to the columns that see them.
// The top bit of a word's elements that are not finite (the exponent is all ones).
template <bool BF>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
  return ((w & (BF ? 0x7f807f80u : 0x7c007c00u)) + (BF ? 0x00800080u : 0x04000400u)) & 0x80008000u;
}
// The word with zeros in their place.
template <bool BF>
__device__ __forceinline__ uint32_t finite(uint32_t w) {
  const uint32_t top = not_finite<BF>(w);
  return w & ~(top | (top - (top >> 15)));
}
// What the others add to the sums lo and hi.
template <bool BF>
__device__ __forceinline__ void add_odd(uint32_t w, float& lo, float& hi) {
  const float a = BF ? __uint_as_float(w << 16) : f16_to_f32((uint16_t)w);
  const float b = BF ? __uint_as_float(w & 0xffff0000u) : f16_to_f32((uint16_t)(w >> 16));
  lo += __builtin_isfinite(a) ? 0.0f : a;
  hi += __builtin_isfinite(b) ? 0.0f : b;
}

// Part that workgroup b of n works on: XCD b mod 8 takes neighbouring parts.
__device__ __forceinline__ int xcd_part(int b, int n) {
  const int x = b & 7, per = n >> 3, more = n & 7;  // XCD x runs per workgroups, one more if x < more
  return x * per + min(x, more) + (b >> 3);
}

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return min(max(v, lo), hi); }

// First query row of sequence s (0 <= s <= n_seq).
__device__ __forceinline__ int first_row(const PagedArgs& a, int s) {
  return a.q_start ? clampi(a.q_start[s], 0, a.rows) : min(s, a.rows);
}

struct Segment {
  int r0, r1;  // query rows
  int k0, k1;  // keys
  int seq;     // whose table row lists the pages
};

// Keys that group g shares (no more than a table row holds).
__device__ __forceinline__ int shared_keys(const PagedArgs& a, int g) {
  return clampi(a.group_shared[g], 0, a.stride * a.page_size);
}

// The group that sequence s is in, or -1: groups are [group_start[i],
// group_start[i + 1]), ascending.
__device__ __forceinline__ int group_of(const PagedArgs& a, int s) {
  if (a.n_group == 0 || s < a.group_start[0] || s >= a.group_start[a.n_group]) return -1;
  int lo = 0, hi = a.n_group;  // group_start[lo] <= s < group_start[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.group_start[mid] <= s) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Segment i: the groups, then the sequences.
__device__ __forceinline__ Segment segment(const PagedArgs& a, int i) {
  Segment s;
  if (i < a.n_group) {
    const int s0 = clampi(a.group_start[i], 0, a.n_seq), s1 = clampi(a.group_start[i + 1], s0, a.n_seq);
    s.r0 = first_row(a, s0);
    s.r1 = max(first_row(a, s1), s.r0);
    s.k0 = 0;
    s.k1 = shared_keys(a, i);
    s.seq = min(s0, a.n_seq - 1);
  } else {
    const int seq = i - a.n_group, g = group_of(a, seq);
    s.r0 = first_row(a, seq);
    s.r1 = max(first_row(a, seq + 1), s.r0);
    s.k1 = clampi(a.len[seq], 0, a.stride * a.page_size);
    s.k0 = g >= 0 ? min(shared_keys(a, g), s.k1) : 0;
    s.seq = seq;
  }
  return s;
}

// Keys of a step of a walk over tiles of COLS columns.
template <int COLS>
__device__ __forceinline__ constexpr int step_keys() {
  return COLS <= 32 ? kPagedStep : kPagedWideStep;
}

// A segment as the walk needs it, kept in shared memory (one more at the end
// holds the totals).
struct Seg {
  int r0, rows;    // query rows
  int k0, k1;      // keys
  int step, tile;  // first step and first tile
  int seq;         // whose table row lists the pages
};

__device__ __forceinline__ int add_most(int a, int b) { return (int)min((int64_t)a + b, (int64_t)0x7fffffff); }

// Inclusive sums over a wave's lanes, no larger than 2^31 - 1.
__device__ __forceinline__ int wave_scan(int v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int u = __shfl_up(v, o);
    if (lane >= o) v = add_most(v, u);
  }
  return v;
}

__device__ __forceinline__ int steps_of(int k0, int k1, int keys) {
  return (int)(((int64_t)k1 - k0 + keys - 1) / keys);
}
__device__ __forceinline__ int tiles_of(int rows, int g, int cols) {
  return (int)(((int64_t)rows * g + cols - 1) / cols);
}

// Every segment's first step and tile, by the whole workgroup: the groups' (none
// where SHARED is 0) and the sequences', whose loads are one round trip.  *to and
// *ts: the steps of all; none where there are more tiles than the rows can have,
// that is, where the sequences' rows overlap.
template <int OWN, int SHARED>
__device__ __forceinline__ void schedule(const PagedArgs& a, const PagedPass& own, const PagedPass& shared, Seg* seg_o,
                                         Seg* seg_s, int* to, int* ts) {
  constexpr int N = SHARED ? 4 : 2;  // steps and tiles of the sequences, and of the groups
  __shared__ int s_wave[kWaves][N];
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  const int ng = SHARED ? shared.n : 0, n = ng + own.n;
  const int per = (n + kThreads - 1) / kThreads;
  const int i0 = min(n, tid * per), i1 = min(n, i0 + per);
  int mine[N] = {};
  for (int i = i0; i < i1; ++i) {
    const bool g = SHARED && i < ng;
    const Segment s = segment(a, i);
    const int keys = g ? step_keys<SHARED>() : step_keys<OWN>(), cols = g ? SHARED : OWN;
    const int steps = steps_of(s.k0, s.k1, keys);
    const int64_t tiles = steps ? (((int64_t)(s.r1 - s.r0) * a.g + cols - 1) / cols) * a.hkv : 0;
    Seg x;
    x.r0 = s.r0, x.rows = s.r1 - s.r0, x.k0 = s.k0, x.k1 = s.k1, x.seq = s.seq;
    x.step = g ? mine[N - 2] : mine[0];
    x.tile = g ? mine[N - 1] : mine[1];
    Seg* to_seg = g ? seg_s + i : seg_o + (i - ng);
    *to_seg = x;
    const int more_steps = (int)min(steps * tiles, (int64_t)0x7fffffff), more_tiles = (int)min(tiles, (int64_t)0x7fffffff);
    if (g) {
      mine[N - 2] = add_most(mine[N - 2], more_steps);
      mine[N - 1] = add_most(mine[N - 1], more_tiles);
    } else {
      mine[0] = add_most(mine[0], more_steps);
      mine[1] = add_most(mine[1], more_tiles);
    }
  }
  int sum[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    sum[k] = wave_scan(mine[k]);
    if (lane == 63) s_wave[wid][k] = sum[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k)
    for (int w = 0; w < wid; ++w) sum[k] = add_most(sum[k], s_wave[w][k]);
  if (tid == kThreads - 1) {
    seg_o[own.n].step = sum[0];
    seg_o[own.n].tile = sum[1];
    if (SHARED) {
      seg_s[ng].step = sum[N - 2];
      seg_s[ng].tile = sum[N - 1];
    }
  }
  for (int i = i0; i < i1; ++i) {
    const bool g = SHARED && i < ng;
    Seg* s = g ? seg_s + i : seg_o + (i - ng);
    s->step = add_most(s->step, g ? sum[N - 2] - mine[N - 2] : sum[0] - mine[0]);
    s->tile = add_most(s->tile, g ? sum[N - 1] - mine[N - 1] : sum[1] - mine[1]);
  }
  __syncthreads();
  *to = seg_o[own.n].tile > own.tiles ? 0 : seg_o[own.n].step;
  if (SHARED) *ts = seg_s[ng].tile > shared.tiles ? 0 : seg_s[ng].step;
}

// What the join needs of a pass's segments (by workgroup `block` of n).
template <int COLS, int KEYS>
__device__ __forceinline__ void publish(const PagedArgs& a, const PagedPass& ps, const Seg* seg, int total, int parts,
                                        int block, int n) {
  for (int i = block * kThreads + threadIdx.x; i < ps.n; i += n * kThreads) {
    const Seg s = seg[i];
    PagedSeg g;
    g.r0 = s.r0, g.r1 = s.r0 + s.rows, g.step = s.step, g.steps = total ? steps_of(s.k0, s.k1, KEYS) : 0;
    g.tile = s.tile, g.tiles = tiles_of(s.rows, a.g, COLS), g.total = total, g.parts = parts;
    g.group = ps.shared ? -1 : group_of(a, i);
    a.seg[ps.first + i] = g;
  }
}

// Zeros in the rows of sequences without keys, which no walk reaches.
template <int D>
__device__ __forceinline__ void clear_empty(const PagedArgs& a, const PagedPass& ps, const Seg* seg) {
  const int n = a.hkv * a.g * (D / 8);
  for (int i = blockIdx.x; i < ps.n; i += gridDim.x) {
    const Seg s = seg[i];
    if (s.k1 > 0) continue;
    for (int64_t j = threadIdx.x; j < (int64_t)s.rows * n; j += kThreads) {
      const int r = (int)(j / n), x = (int)(j - (int64_t)r * n);
      *reinterpret_cast<uint4*>(a.po + row_offset(a.o, s.r0 + r, x / (D / 8)) + x % (D / 8) * 16) =
          make_uint4(0, 0, 0, 0);
    }
  }
}

// The segment that step `at` belongs to (empty ones share a step).
__device__ __forceinline__ int find_segment(const Seg* seg, int n, int at) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (seg[mid].step <= at) lo = mid;
    else hi = mid;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Keys that query row `row`, the rr-th of segment s, sees.  In a group the
// row's own sequence says so: `own` are the sequences' segments.
__device__ __forceinline__ int limit_of(const PagedArgs& a, const Seg& s, const Seg* own, int row, int rr) {
  if (!own) return s.k1 - s.rows + rr + 1;
  int lo = s.seq, hi = a.n_seq;  // sequences' rows ascend
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (own[mid].r0 <= row) lo = mid;
    else hi = mid;
  }
  return own[lo].k1 - own[lo].rows + row - own[lo].r0 + 1;
}

// VE neighbouring elements of an output row, scaled.
template <int VE, bool BF>
__device__ __forceinline__ void store_row(char* dst, const float (&o)[VE], float scale) {
  uint32_t x[VE / 2];
#pragma unroll
  for (int j = 0; j < VE; j += 2) x[j / 2] = pack2<BF>(o[j] * scale, o[j + 1] * scale);
  if constexpr (VE == 8) *reinterpret_cast<uint4*>(dst) = make_uint4(x[0], x[1], x[2], x[3]);
  else *reinterpret_cast<uint2*>(dst) = make_uint2(x[0], x[1]);
}

// A stretch of one tile's walk.
struct Piece {
  Seg s;
  const int32_t* pages;
  int64_t head_off;
  int si, h, tile, it, n;  // segment, key-value head, tile of the head, tile of the segment, steps of its walk
  int ka, kb;              // keys
  bool whole;
};

// The part of n that takes step `at` of `total`: the last w with total w / n,
// rounded down, at or before it.  The quotient is below 2^10 and at least
// 2^-31 below the next whole number unless it is one, so that 53 bits do.
__device__ __forceinline__ int part_of(int64_t at, int64_t n, int total) {
  return (int)((double)((at + 1) * n - 1) / (double)total);
}

// Shared memory of the two walks.
template <int D>
struct __attribute__((aligned(16))) FewShared {
  int64_t off[kWaves][2][32];
  float o[kWaves][kPagedCols][D + 4];  // (four more: banks)
  float ml[kWaves][kPagedCols][2];
  int last;
};
template <int D>
struct __attribute__((aligned(1024))) ManyShared {
  uint16_t kv[2][2 * kPagedWideStep * D];  // two steps' buffers: K, then V
  int64_t off[2][kPagedWideStep];
  int odd[2][kWaves];   // whether a wave found values that are not finite in its rows of a step
};

template <int D, bool BF, int COLS>
__device__ __forceinline__ void walk_few(const PagedArgs& a, const PagedPass& ps, const Seg* seg, FewShared<D>& sh,
                                         int total, int parts, int block) {
  constexpr int NC = COLS / kPagedCols;
  constexpr int VE = D / 16;          // d elements a lane holds of a V row
  constexpr int KS = D / 32;          // k steps of the score product
  auto& s_off = sh.off;
  auto& s_o = sh.o;
  auto& s_ml = sh.ml;
  int& s_last = sh.last;

  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g4 = lane >> 4;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int w = xcd_part(block, parts);
  int at = (int)((int64_t)total * w / parts);
  const int end = (int)((int64_t)total * (w + 1) / parts);

  // ---- the tile that step `at` belongs to, and how far this part walks it
  auto next_piece = [&]() {
    Piece p;
    p.si = find_segment(seg, ps.n, at);
    p.s = seg[p.si];
    p.n = steps_of(p.s.k0, p.s.k1, kPagedStep);
    const int tiles = tiles_of(p.s.rows, a.g, COLS);
    const int local = at - p.s.step, step = local % p.n;
    p.it = local / p.n;
    p.h = p.it / tiles;
    p.tile = p.it - p.h * tiles;
    const int walk = min(p.n - step, end - at);
    // the only result of these columns: no join
    p.whole = walk == p.n && p.s.k0 == 0;
    p.ka = p.s.k0 + step * kPagedStep;
    p.kb = (int)min((int64_t)p.s.k1, (int64_t)p.ka + (int64_t)walk * kPagedStep);
    p.pages = a.table + (int64_t)p.s.seq * a.stride;
    p.head_off = (int64_t)p.h * a.page_size * D * 2;
    at += walk;
    return p;
  };
  // a wave's step is 32 keys; lane i (and i + 32) looks after key i
  const int kl = lane & 31;
  auto entry = [&](const Piece& p, int k) { return k + kl < p.kb ? p.pages[div_fast(k + kl, a.page)] : -1; };
  auto place = [&](const Piece& p, int slot, int k, int pg) {  // the rows' offsets, -1: no such row
    const int key = k + kl, in = key - div_fast(key, a.page) * a.page_size;
    const int64_t off = (uint32_t)pg < (uint32_t)a.n_pages ? pg * a.page_bytes + (int64_t)in * (D * 2) : -1;
    if (lane < 32) s_off[wid][slot][kl] = off;
    __builtin_amdgcn_wave_barrier();
  };
  uint4 kr[2][KS];
  uint32_t vr[8][VE / 2];
  auto load_k = [&](const Piece& pc, int slot) {
    const char* base = a.pk + pc.head_off + g4 * 16;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int64_t off = s_off[wid][slot][16 * t + c];
      const char* p = base + (off < 0 ? 0 : off);
#pragma unroll
      for (int i = 0; i < KS; ++i) kr[t][i] = *reinterpret_cast<const uint4*>(p + i * 64);
    }
  };
  auto load_v = [&](const Piece& pc, int slot) {
    const char* base = a.pv + pc.head_off + c * VE * 2;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t off = s_off[wid][slot][16 * (i >> 2) + 4 * g4 + (i & 3)];
      const char* p = base + (off < 0 ? 0 : off);
      if constexpr (VE == 8) {
        const uint4 x = *reinterpret_cast<const uint4*>(p);
        vr[i][0] = x.x, vr[i][1] = x.y, vr[i][2] = x.z, vr[i][3] = x.w;
      } else {
        const uint2 x = *reinterpret_cast<const uint2*>(p);
        vr[i][0] = x.x, vr[i][1] = x.y;
      }
    }
  };
  uint4 q[NC][KS];
  auto load_q = [&](const Piece& pc) {  // this lane's columns: query rows and heads
#pragma unroll
    for (int t = 0; t < NC; ++t) {
      const int cc = min(pc.tile * COLS + t * kPagedCols + c, pc.s.rows * a.g - 1);
      const int rr = div_fast(cc, a.gdiv);
      const char* p = a.pq + row_offset(a.q, pc.s.r0 + rr, pc.h * a.g + cc - rr * a.g) + g4 * 16;
#pragma unroll
      for (int i = 0; i < KS; ++i) q[t][i] = *reinterpret_cast<const uint4*>(p + i * 64);
    }
  };

  // The loads of a step are on their way while the step before is computed,
  // also from one piece to the next: `next` is known before the last step of
  // `cur`, and its first rows are fetched behind that step's products.
  Piece next = next_piece();
  int slot = 0, next_pg = entry(next, next.ka + wid * 32);
  load_q(next);
  place(next, 0, next.ka + wid * 32, next_pg);
  load_k(next, 0);
  load_v(next, 0);
  bool have = true;
  while (have) {
    const Piece cur = next;
    have = at < end;
    if (have) next = next_piece();
    const Seg s = cur.s;
    const int h = cur.h, tile = cur.tile, it = cur.it, n = cur.n, kb = cur.kb, slot_out = s.tile + it + w;
    const bool whole = cur.whole;

    // ---- the keys that this lane's columns see
    const int ncol = s.rows * a.g;
    int lim[NC], lim_min = 0x7fffffff;
#pragma unroll
    for (int t = 0; t < NC; ++t) {
      const int col = tile * COLS + t * kPagedCols + c, rr = div_fast(min(col, ncol - 1), a.gdiv);
      lim[t] = col < ncol ? limit_of(a, s, nullptr, s.r0 + rr, rr) : 0x7fffffff;  // (never stored: no mask)
      lim_min = min(lim_min, lim[t]);
    }
    lim_min = min(lim_min, __shfl_xor(lim_min, 1));
    lim_min = min(lim_min, __shfl_xor(lim_min, 2));
    lim_min = min(lim_min, __shfl_xor(lim_min, 4));
    lim_min = __builtin_amdgcn_readfirstlane(min(lim_min, __shfl_xor(lim_min, 8)));

    f32x4_t acc[NC][VE];
    float m[NC], l[NC];
#pragma unroll
    for (int t = 0; t < NC; ++t) {
      m[t] = -INFINITY;
      l[t] = 0.0f;
#pragma unroll
      for (int j = 0; j < VE; ++j) acc[t][j] = f32x4_t{};
    }
    // (a piece shorter than the waves before this one's rows: the step is
    // empty, its rows are masked, and the next piece's loads follow it)
    int k = cur.ka + wid * 32;
    next_pg = entry(cur, k + kPagedStep);
    for (bool again = true; again; k += kPagedStep) {
      again = k + kPagedStep < kb;
      // every key of the step has a row and is seen by every column
      const bool full = __all(s_off[wid][slot][kl] >= 0) && k + 32 <= lim_min;
      if (again) {
        place(cur, slot ^ 1, k + kPagedStep, next_pg);
        next_pg = entry(cur, k + 2 * kPagedStep);
      } else if (have) {
        place(next, slot ^ 1, next.ka + wid * 32, entry(next, next.ka + wid * 32));
      }
      f32x4_t sc[NC][2];
#pragma unroll
      for (int t = 0; t < NC; ++t) {
        sc[t][0] = sc[t][1] = f32x4_t{};
#pragma unroll
        for (int i = 0; i < KS; ++i) {
          sc[t][0] = mfma16<BF>(kr[0][i], q[t][i], sc[t][0]);
          sc[t][1] = mfma16<BF>(kr[1][i], q[t][i], sc[t][1]);
        }
      }
      if (again) load_k(cur, slot ^ 1);
      else if (have) load_k(next, slot ^ 1);
      if (!full) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int kk = 16 * (i >> 2) + 4 * g4 + (i & 3);
          const bool row_there = s_off[wid][slot][kk] >= 0;
#pragma unroll
          for (int t = 0; t < NC; ++t) {
            float& x = reinterpret_cast<float*>(&sc[t][i >> 2])[i & 3];
            x = row_there && k + kk < lim[t] ? x : -INFINITY;
          }
          // a row that is not there was read elsewhere: it may hold anything
#pragma unroll
          for (int j = 0; j < VE / 2; ++j) vr[i][j] = row_there ? vr[i][j] : 0u;
        }
      }
      uint4 p[NC], p2[NC];
#pragma unroll
      for (int t = 0; t < NC; ++t) {
        // online softmax in the log2 domain; the scale (> 0) is one FMA ahead of exp2
        float mx = sc[t][0][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) mx = fmaxf(mx, sc[t][i >> 2][i & 3]);
        mx = fmaxf(mx, other16(mx));
        mx = fmaxf(mx, other32(mx)) * a.scale;
        const float m_new = mx > m[t] + kLazyMax || m[t] == -INFINITY ? fmaxf(mx, m[t]) : m[t];
        const float m_use = m_new == -INFINITY ? 0.0f : m_new;
        if (__any(m_new != m[t])) {
          const float alpha = __builtin_amdgcn_exp2f(m[t] - m_use);
          l[t] *= alpha;
#pragma unroll
          for (int j = 0; j < VE; ++j) acc[t][j] *= alpha;
        }
        m[t] = m_new;
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_exp2f(fmaf(sc[t][i >> 2][i & 3], a.scale, kRaise<BF> - m_use));
        split_p<BF>(x[0], x[1], p[t].x, p2[t].x);
        split_p<BF>(x[2], x[3], p[t].y, p2[t].y);
        split_p<BF>(x[4], x[5], p[t].z, p2[t].z);
        split_p<BF>(x[6], x[7], p[t].w, p2[t].w);
        l[t] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
      }
      uint32_t odd = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < VE / 2; ++j) odd |= not_finite<BF>(vr[i][j]);
      if (__builtin_expect(__any(odd != 0), 0)) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int j = 0; j < VE / 2; ++j) vr[i][j] = finite<BF>(vr[i][j]);
      }
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;
        uint4 v;
        v.x = __builtin_amdgcn_perm(vr[1][j / 2], vr[0][j / 2], sel);
        v.y = __builtin_amdgcn_perm(vr[3][j / 2], vr[2][j / 2], sel);
        v.z = __builtin_amdgcn_perm(vr[5][j / 2], vr[4][j / 2], sel);
        v.w = __builtin_amdgcn_perm(vr[7][j / 2], vr[6][j / 2], sel);
#pragma unroll
        for (int t = 0; t < NC; ++t) {
          acc[t][j] = mfma16<BF>(v, p[t], acc[t][j]);
          acc[t][j] = mfma16<BF>(v, p2[t], acc[t][j]);
        }
      }
      if (__builtin_expect(__any(odd != 0), 0)) {
#pragma unroll 1
        for (int kk = 0; kk < 32; ++kk) {
          const int64_t off = s_off[wid][slot][kk];
          if (off < 0) continue;
          const char* row = a.pv + cur.head_off + off;
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < VE; j += 2) {
              const uint32_t v = *reinterpret_cast<const uint32_t*>(row + ((4 * g4 + i) * VE + j) * 2);
#pragma unroll
              for (int t = 0; t < NC; ++t) {
                float lo = acc[t][j][i], hi = acc[t][j + 1][i];
                if (k + kk < lim[t]) add_odd<BF>(v, lo, hi);
                acc[t][j][i] = lo, acc[t][j + 1][i] = hi;
              }
            }
        }
      }
      if (again) load_v(cur, slot ^ 1);
      else if (have) load_v(next, slot ^ 1);
      slot ^= 1;
    }
    if (have) load_q(next);
    // ---- join the four waves, 16 columns at a time.  Lane (g4, c) holds
    // d = (4 g4 + i) VE + j of its column: 4 VE neighbours.
#pragma unroll
    for (int t = 0; t < NC; ++t) {
      l[t] += other16(l[t]);
      l[t] += other32(l[t]);
      if (g4 == 0) {
        s_ml[wid][c][0] = m[t];
        s_ml[wid][c][1] = l[t];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < VE; j += 4)
          *reinterpret_cast<float4*>(&s_o[wid][c][(4 * g4 + i) * VE + j]) =
              make_float4(acc[t][j][i], acc[t][j + 1][i], acc[t][j + 2][i], acc[t][j + 3][i]);
      __syncthreads();
      const int jc = tid >> 4, part = tid & 15;  // column, and VE neighbouring d
      float mw[kWaves], top = -INFINITY;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        mw[i] = s_ml[i][jc][0];
        top = fmaxf(top, mw[i]);
      }
      const float use = top == -INFINITY ? 0.0f : top;
      float lt = 0.0f, o[VE] = {};
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        const float f = __builtin_amdgcn_exp2f(mw[i] - use);
        lt += s_ml[i][jc][1] * f;
#pragma unroll
        for (int j = 0; j < VE; ++j) o[j] += s_o[i][jc][part * VE + j] * f;
      }
      if (whole) {
        const int col = tile * COLS + t * kPagedCols + jc;
        if (col < ncol) {
          const int rr = div_fast(col, a.gdiv);
          const float inv = lt == 0.0f ? 0.0f : 1.0f / lt;
          store_row<VE, BF>(a.po + row_offset(a.o, s.r0 + rr, h * a.g + col - rr * a.g) + part * VE * 2, o, inv);
        }
      } else if (tile * COLS + t * kPagedCols + jc < ncol) {
        const int64_t to = (int64_t)slot_out * COLS + t * kPagedCols + jc;
        if (ps.fused) {  // read by another workgroup of this launch
          if (part == 0) store_agent2(ps.part_ml + 2 * to, top, lt);
#pragma unroll
          for (int j = 0; j < VE; j += 2) store_agent2(ps.part_o + to * D + part * VE + j, o[j], o[j + 1]);
        } else {
          if (part == 0) {
            ps.part_ml[2 * to] = top;
            ps.part_ml[2 * to + 1] = lt;
          }
#pragma unroll
          for (int j = 0; j < VE; j += 4)
            *reinterpret_cast<float4*>(ps.part_o + to * D + part * VE + j) =
                make_float4(o[j], o[j + 1], o[j + 2], o[j + 3]);
        }
      }
      __syncthreads();
    }
    if (!ps.fused || whole) continue;

    // ---- the last part of the tile to arrive joins them, in part order
    const int64_t from = s.step + (int64_t)it * n;
    const int w0 = part_of(from, parts, total), w1 = part_of(from + n - 1, parts, total);
    drain_vmem();
    __syncthreads();
    int32_t* counter = ps.counters + s.tile + it;
    if (tid == 0) {
      const bool last = arrive_agent(counter) == w1 - w0;
      if (last) reset_agent(counter);  // ready for the next call (stream-ordered)
      s_last = last;
    }
    __syncthreads();
    if (s_last) {
      const int jc = tid >> 4, part = tid & 15;
#pragma unroll
      for (int t = 0; t < NC; ++t) {
        const int col = tile * COLS + t * kPagedCols + jc;
        if (col >= ncol) continue;
        const int64_t first = (int64_t)(s.tile + it + w0) * COLS + t * kPagedCols + jc;
        float m_all = -INFINITY, l_all = 0.0f, o[VE] = {};
        for (int p0 = 0; p0 <= w1 - w0; p0 += 4) {  // four parts' loads at a time
          float2 ml[4], x[4][VE / 2];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int64_t to = first + (int64_t)min(p0 + i, w1 - w0) * COLS;
            ml[i] = load_agent2(ps.part_ml + 2 * to);
#pragma unroll
            for (int j = 0; j < VE; j += 2) x[i][j / 2] = load_agent2(ps.part_o + to * D + part * VE + j);
          }
          float top = m_all;
#pragma unroll
          for (int i = 0; i < 4; ++i) top = fmaxf(top, ml[i].x);
          const float use = top == -INFINITY ? 0.0f : top, keep = __builtin_amdgcn_exp2f(m_all - use);
          m_all = top;
          l_all *= keep;
#pragma unroll
          for (int j = 0; j < VE; ++j) o[j] *= keep;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (p0 + i > w1 - w0) break;
            const float f = __builtin_amdgcn_exp2f(ml[i].x - use);
            l_all = fmaf(ml[i].y, f, l_all);
#pragma unroll
            for (int j = 0; j < VE; j += 2) {
              o[j] = fmaf(x[i][j / 2].x, f, o[j]);
              o[j + 1] = fmaf(x[i][j / 2].y, f, o[j + 1]);
            }
          }
        }
        const int rr = div_fast(col, a.gdiv);
        store_row<VE, BF>(a.po + row_offset(a.o, s.r0 + rr, h * a.g + col - rr * a.g) + part * VE * 2, o,
                          l_all == 0.0f ? 0.0f : 1.0f / l_all);
      }
    }
    __syncthreads();
  }
}

// ---- the walk for many columns --------------------------------------------------
// A workgroup's tile is 32 CW columns, 32 a wave (CW 4), or, for up to 64, two
// waves of columns and two halves of every step's keys (CW 2).  With 64 columns
// and more the keys' bytes arrive faster than the matrix cores use them, so a
// step of 64 keys is fetched once for the workgroup, straight into shared
// memory (one instruction 1 KiB, a lane 16 bytes, each from its own key row),
// while the step before is computed; two workgroups share a CU, so that one's
// softmax runs beside the other's products.  (The schedule takes 28 bytes of
// shared memory a segment beside the 66 KiB of the walk at D = 128: from about
// 510 sequences and groups on only one fits.  Groups of 8 that share 2K keys: 504
// segments 4.0 TB/s, 513 segments 2.9.)
//   S^T = K Q^T on 32x32x16: a lane holds one column's scores of 16 keys in 32
//   O^T += V^T P^T: V^T through transposing reads; the product's k index 8 g + e
//   stands for key 16 hh + 4 g + e (e < 4) or 16 hh + 8 + 4 g + e - 4, as the
//   accumulators of S^T lie
// 16-byte pieces of a row are XOR-swizzled so that the 16 rows of a K read, and
// the 4 rows of a transposing V read, take different banks.
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));

template <bool BF>
__device__ __forceinline__ f32x16_t mfma32(const uint4& a, const uint4& b, const f32x16_t& c) {
  if constexpr (BF)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b),
                                                   c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c,
                                                  0, 0, 0);
}

template <int D>
__device__ __forceinline__ int swz_k(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
template <int D>
__device__ __forceinline__ int swz_v(int r) { return D == 128 ? (2 * (r & 3)) ^ (8 * (r & 1)) : 4 * ((r >> 1) & 1); }

// 16 bytes a lane from its own address to 1 KiB of shared memory at lds (wave
// uniform).  Written as asm, so that the compiler does not wait for it at every
// shared read; the kernel waits itself (vmcnt 0, then a barrier).
__device__ __forceinline__ void load_to_lds(const char* p, uint32_t lds) {
  const uint32_t to = __builtin_amdgcn_readfirstlane(lds);
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
  asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(p), "s"(to) : "memory", "m0");
#pragma clang diagnostic pop
}

template <int D, bool BF, int COLS>
__device__ __forceinline__ void walk_many(const PagedArgs& a, const PagedPass& ps, const Seg* seg, const Seg* own,
                                          ManyShared<D>& sh, int total, int parts, int block) {
  constexpr int CW = COLS / 32, KEYS = kPagedWideStep;
  constexpr int KT = CW / 2;          // 32-key tiles that a wave computes of a step
  constexpr int NS = D / 16, ND = D / 32;
  constexpr int CPR = D / 8;          // 16-byte pieces of a row
  constexpr int RPI = 64 / CPR;       // rows of one load
  constexpr int LPW = 16 / RPI;       // loads of a wave (16 rows) for K, and for V
  constexpr int BUF = 2 * KEYS * D;   // elements of a step: K, then V
  uint16_t* sKV = sh.kv[0];
  auto& s_off = sh.off;

  const int tid = threadIdx.x, lane = tid & 63, lq = lane & 31, g = lane >> 5;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wc = wid % CW, wk = wid / CW;  // the wave's columns, and its part of a step's keys
  const int w = xcd_part(block, parts);
  int at = (int)((int64_t)total * w / parts);
  const int end = (int)((int64_t)total * (w + 1) / parts);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint16_t*)sKV;

  while (at < end) {
    const int si = find_segment(seg, ps.n, at);
    const Seg s = seg[si];
    const int n = steps_of(s.k0, s.k1, KEYS), tiles = tiles_of(s.rows, a.g, COLS);
    const int local = at - s.step, it = local / n, step = local - it * n;
    const int h = it / tiles, tile = it - h * tiles;
    const int walk = min(n - step, end - at);
    const int slot_out = s.tile + it + w;
    const bool whole = !ps.shared && walk == n && s.k0 == 0;
    const int ka = s.k0 + step * KEYS;
    const int kb = (int)min((int64_t)s.k1, (int64_t)ka + (int64_t)walk * KEYS);
    at += walk;

    const int32_t* pages = a.table + (int64_t)s.seq * a.stride;
    const int64_t head_off = (int64_t)h * a.page_size * D * 2;
    const char* kbase = a.pk + head_off;
    const char* vbase = a.pv + head_off;
    // a wave fetches 16 of a step's rows; lane i (and i + 16, ...) looks after row i
    const int my = wid * 16 + (lane & 15);
    auto entry = [&](int k) { return k + my < kb ? pages[div_fast(k + my, a.page)] : -1; };
    auto place = [&](int b, int k, int pg) {  // the rows' offsets; -1: no such row
      const int key = k + my, in = key - div_fast(key, a.page) * a.page_size;
      const int64_t off = (uint32_t)pg < (uint32_t)a.n_pages ? pg * a.page_bytes + (int64_t)in * (D * 2) : -1;
      if (lane < 16) s_off[b][my] = off;
      __builtin_amdgcn_wave_barrier();
    };
    // one of a step's 2 LPW loads of this wave: i < LPW a K piece, else a V piece
    auto issue = [&](int b, int i) {
      const int inst = wid * LPW + i % LPW, r = inst * RPI + lane / CPR;
      const int64_t off = s_off[b][r];
      const int sw = i < LPW ? swz_k<D>(r) : swz_v<D>(r);
      const char* p = (i < LPW ? kbase : vbase) + (off < 0 ? 0 : off) + 16 * ((lane % CPR) ^ sw);
      load_to_lds(p, lds0 + (b * BUF + (i < LPW ? 0 : KEYS * D)) * 2 + inst * 1024);
    };
    // this wave's loads are there; zeros in the place of values whose rows do not
    // exist and of those that are not finite, which sh.odd tells of
    auto landed = [&](int b) {
      asm volatile("" ::: "memory");
      drain_vmem();
      asm volatile("" ::: "memory");
      uint4* at = reinterpret_cast<uint4*>(sKV + b * BUF + KEYS * D + wid * LPW * 512 + lane * 8);
      uint4 x[LPW];
      uint32_t gone[LPW], odd = 0, change = 0;
#pragma unroll
      for (int i = 0; i < LPW; ++i) {
        x[i] = at[i * 64];
        gone[i] = s_off[b][(wid * LPW + i) * RPI + lane / CPR] < 0;
      }
#pragma unroll
      for (int i = 0; i < LPW; ++i) {
        const uint32_t o = not_finite<BF>(x[i].x) | not_finite<BF>(x[i].y) | not_finite<BF>(x[i].z) | not_finite<BF>(x[i].w);
        odd |= gone[i] ? 0 : o;
        change |= gone[i] | o;
      }
      if (__builtin_expect(__any(change != 0), 0)) {
#pragma unroll
        for (int i = 0; i < LPW; ++i)
          at[i * 64] = gone[i] ? make_uint4(0, 0, 0, 0)
                               : make_uint4(finite<BF>(x[i].x), finite<BF>(x[i].y), finite<BF>(x[i].z), finite<BF>(x[i].w));
      }
      const bool any = __any(odd != 0);
      if (lane == 0) sh.odd[b][wid] = any;
    };
    int next_pg = entry(ka);
    place(0, ka, next_pg);
#pragma unroll
    for (int i = 0; i < 2 * LPW; ++i) issue(0, i);
    next_pg = entry(ka + KEYS);

    // ---- this lane's column
    const int ncol = s.rows * a.g, col = tile * COLS + wc * 32 + lq, cc = min(col, ncol - 1);
    const int rr = div_fast(cc, a.gdiv), row = s.r0 + rr, head = h * a.g + cc - rr * a.g;
    const int lim = col < ncol ? limit_of(a, s, own, row, rr) : 0x7fffffff;  // (never stored: no mask)
    const bool idle = tile * COLS + wc * 32 >= ncol;  // a wave without columns only fetches
    uint4 q[NS];
    {
      const char* p = a.pq + row_offset(a.q, row, head) + g * 16;
#pragma unroll
      for (int i = 0; i < NS; ++i) q[i] = *reinterpret_cast<const uint4*>(p + i * 32);
    }
    int lim_min = lim;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) lim_min = min(lim_min, __shfl_xor(lim_min, o));
    lim_min = __builtin_amdgcn_readfirstlane(lim_min);

    f32x16_t acc[ND];
#pragma unroll
    for (int i = 0; i < ND; ++i) acc[i] = f32x16_t{};
    float m = -INFINITY, l = 0.0f;

    auto compute = [&](int b, int k, bool full, auto&& load) {
      const uint16_t* sK = sKV + b * BUF;
      const uint16_t* sV = sK + KEYS * D;
      f32x16_t sc[KT];
#pragma unroll
      for (int t = 0; t < KT; ++t) sc[t] = f32x16_t{};
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        uint4 x[KT];
#pragma unroll
        for (int t = 0; t < KT; ++t) {
          const int r = 32 * (wk * KT + t) + lq;
          x[t] = *reinterpret_cast<const uint4*>(sK + r * D + 8 * ((2 * i + g) ^ swz_k<D>(r)));
        }
        load(i);
#pragma unroll
        for (int t = 0; t < KT; ++t) sc[t] = mfma32<BF>(x[t], q[i], sc[t]);
      }
      __builtin_amdgcn_s_setprio(0);
      if (!full) {
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int kk = 32 * (wk * KT + t) + 8 * (r >> 2) + 4 * g + (r & 3);
            sc[t][r] = s_off[b][kk] >= 0 && k + kk < lim ? sc[t][r] : -INFINITY;
          }
      }
      float mx = sc[0][0];
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[t][r]);
      mx = fmaxf(mx, other32(mx)) * a.scale;
      const float m_new = mx > m + kLazyMax || m == -INFINITY ? fmaxf(mx, m) : m;
      const float m_use = m_new == -INFINITY ? 0.0f : m_new;
      if (__any(m_new != m)) {
        const float alpha = __builtin_amdgcn_exp2f(m - m_use);
        l *= alpha;
#pragma unroll
        for (int i = 0; i < ND; ++i) acc[i] *= alpha;
      }
      m = m_new;
      const int gq = lane >> 4, li = lane & 15;
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[t][r] = __builtin_amdgcn_exp2f(fmaf(sc[t][r], a.scale, kRaise<BF> - m_use));
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          uint4 p, p2;
          split_p<BF>(sc[t][8 * hh], sc[t][8 * hh + 1], p.x, p2.x);
          split_p<BF>(sc[t][8 * hh + 2], sc[t][8 * hh + 3], p.y, p2.y);
          split_p<BF>(sc[t][8 * hh + 4], sc[t][8 * hh + 5], p.z, p2.z);
          split_p<BF>(sc[t][8 * hh + 6], sc[t][8 * hh + 7], p.w, p2.w);
#pragma unroll
          for (int i = 0; i < 8; ++i) l += sc[t][8 * hh + i];
          const int k0 = 32 * (wk * KT + t) + 16 * hh + 4 * (gq >> 1) + (li >> 2);
          uint4 x[ND];
#pragma unroll
          for (int i = 0; i < ND; ++i) {
            const int d = 32 * i + 16 * (gq & 1) + 4 * (li & 3);
            auto tr = [&](int r) {
              return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(
                  sV + r * D + 8 * ((d >> 3) ^ swz_v<D>(r)) + (d & 4)));
            };
            const s16x8_t v = __builtin_shufflevector(tr(k0), tr(k0 + 8), 0, 1, 2, 3, 4, 5, 6, 7);
            x[i] = __builtin_bit_cast(uint4, v);
            acc[i] = mfma32<BF>(x[i], p, acc[i]);
          }
#pragma unroll
          for (int i = 0; i < ND; ++i) acc[i] = mfma32<BF>(x[i], p2, acc[i]);
        }
      __builtin_amdgcn_s_setprio(0);
      if (__builtin_expect(sh.odd[b][0] | sh.odd[b][1] | sh.odd[b][2] | sh.odd[b][3], 0)) {
#pragma unroll 1
        for (int kk = 32 * wk * KT; kk < 32 * (wk + 1) * KT; ++kk) {
          const int64_t off = s_off[b][kk];
          if (off < 0) continue;
#pragma unroll
          for (int i = 0; i < ND; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const uint2 v = *reinterpret_cast<const uint2*>(vbase + off + (32 * i + 8 * r + 4 * g) * 2);
              float x[4] = {acc[i][4 * r], acc[i][4 * r + 1], acc[i][4 * r + 2], acc[i][4 * r + 3]};
              if (k + kk < lim) {
                add_odd<BF>(v.x, x[0], x[1]);
                add_odd<BF>(v.y, x[2], x[3]);
              }
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[i][4 * r + e] = x[e];
            }
        }
      }
    };

    landed(0);
    __syncthreads();
    int b = 0;
    for (int k = ka; k < kb; k += KEYS, b ^= 1) {
      const bool more = k + KEYS < kb;
      if (more) {
        place(b ^ 1, k + KEYS, next_pg);
        next_pg = entry(k + 2 * KEYS);
      }
      if (idle) {
#pragma unroll
        for (int i = 0; i < 2 * LPW; ++i)
          if (more) issue(b ^ 1, i);
      } else {
        const bool full = k + KEYS <= lim_min && __all(s_off[b][lane] >= 0);
        compute(b, k, full, [&](int i) {
          if (more) issue(b ^ 1, i);
        });
      }
      if (more) landed(b ^ 1);
      __syncthreads();
    }
    l += other32(l);

    // ---- CW 2: the halves of the keys meet in shared memory
    if (CW == 2) {
      float4* box = reinterpret_cast<float4*>(sKV) + wc * (ND * 4 + 1) * 64;
      if (wk == 1) {
#pragma unroll
        for (int i = 0; i < ND; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            box[(4 * i + r) * 64 + lane] =
                make_float4(acc[i][4 * r], acc[i][4 * r + 1], acc[i][4 * r + 2], acc[i][4 * r + 3]);
        box[ND * 4 * 64 + lane] = make_float4(m, l, 0.0f, 0.0f);
      }
      __syncthreads();
      if (wk == 0) {
        const float4 o = box[ND * 4 * 64 + lane];
        const float top = fmaxf(m, o.x), use = top == -INFINITY ? 0.0f : top;
        const float f0 = __builtin_amdgcn_exp2f(m - use), f1 = __builtin_amdgcn_exp2f(o.x - use);
        m = top;
        l = l * f0 + o.y * f1;
#pragma unroll
        for (int i = 0; i < ND; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float4 v = box[(4 * i + r) * 64 + lane];
            acc[i][4 * r] = acc[i][4 * r] * f0 + v.x * f1;
            acc[i][4 * r + 1] = acc[i][4 * r + 1] * f0 + v.y * f1;
            acc[i][4 * r + 2] = acc[i][4 * r + 2] * f0 + v.z * f1;
            acc[i][4 * r + 3] = acc[i][4 * r + 3] * f0 + v.w * f1;
          }
      }
      __syncthreads();
    }
    // acc[i][4 r + e] is d = 32 i + 8 r + 4 g + e of this lane's column
    if (col >= ncol || wk != 0) continue;
    if (whole) {
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;
      char* dst = a.po + row_offset(a.o, row, head) + g * 8;
#pragma unroll
      for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          *reinterpret_cast<uint2*>(dst + (32 * i + 8 * r) * 2) =
              make_uint2(pack2<BF>(acc[i][4 * r] * inv, acc[i][4 * r + 1] * inv),
                         pack2<BF>(acc[i][4 * r + 2] * inv, acc[i][4 * r + 3] * inv));
    } else {
      const int64_t to = (int64_t)slot_out * COLS + wc * 32 + lq;
      if (g == 0) {
        ps.part_ml[2 * to] = m;
        ps.part_ml[2 * to + 1] = l;
      }
      float* dst = ps.part_o + to * D + 4 * g;
#pragma unroll
      for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          *reinterpret_cast<float4*>(dst + 32 * i + 8 * r) =
              make_float4(acc[i][4 * r], acc[i][4 * r + 1], acc[i][4 * r + 2], acc[i][4 * r + 3]);
    }
  }
}

// Join of a row's partial results, shared keys first: W waves a (row, query
// head), D / 4 lanes a part, several parts at a time and eight loads of each in
// flight; what the lane groups (and waves) hold is joined at the end.
template <int D, bool BF, int W>
__global__ __launch_bounds__(W > kWaves ? W * 64 : kThreads) void paged_join_kernel(const PagedArgs a, const PagedPass sh,
                                                              const PagedPass own) {
  constexpr int LPP = D / 4, PPW = 64 / LPP, STRIDE = PPW * W;
  __shared__ float4 s_o[W][LPP];
  __shared__ float2 s_ml[W];
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, e4 = lane % LPP, sub = lane / LPP + (W > 1 ? wid * PPW : 0);
  const int hq = W > 1 ? blockIdx.y : blockIdx.y * kWaves + wid;
  if (hq >= a.hkv * a.g) return;
  const int h = div_fast(hq, a.gdiv), hg = hq - h * a.g;
  const PagedSeg q = a.seg[a.n_group + blockIdx.x];
  PagedSeg g = {};
  if (q.group >= 0) g = a.seg[q.group];
  for (int row = q.r0 + blockIdx.z; row < q.r1; row += gridDim.z) {
    // parts of a walk, and the column of the first one's slot; none where the
    // row is not the segment's (query rows that do not ascend, under a group)
    auto range = [&](const PagedSeg& s, const PagedPass& p, int64_t* at) {
      if (s.steps == 0 || row < s.r0 || row >= s.r1) return 0;
      const int col = (row - s.r0) * a.g + hg, tile = col / p.cols;
      const int it = h * s.tiles + tile;
      const int64_t n = s.parts, from = s.step + (int64_t)it * s.steps;
      const int w0 = part_of(from, n, s.total), w1 = part_of(from + s.steps - 1, n, s.total);
      *at = ((int64_t)s.tile + it + w0) * p.cols + (col - tile * p.cols);
      return w1 - w0 + 1;
    };
    int64_t at_g = 0, at_q = 0;
    const int n_g = range(g, sh, &at_g), n_q = range(q, own, &at_q);
    if (n_g == 0 && n_q == 1) continue;  // stored by the walk itself
    const int parts = n_g + n_q;
    float m = -INFINITY, l = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int p0 = sub; p0 < parts; p0 += 8 * STRIDE) {
      float2 ml[8];
      float4 x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int p = p0 + i * STRIDE;
        ml[i] = make_float2(-INFINITY, 0.0f);
        x[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (p < parts) {
          const bool in_g = p < n_g;
          const int64_t at = in_g ? at_g + (int64_t)p * sh.cols : at_q + (int64_t)(p - n_g) * own.cols;
          ml[i] = *reinterpret_cast<const float2*>((in_g ? sh.part_ml : own.part_ml) + 2 * at);
          x[i] = *reinterpret_cast<const float4*>((in_g ? sh.part_o : own.part_o) + at * D + 4 * e4);
        }
      }
      float top = m;
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, ml[i].x);
      const float use = top == -INFINITY ? 0.0f : top, keep = __builtin_amdgcn_exp2f(m - use);
      m = top;
      l *= keep;
      o.x *= keep, o.y *= keep, o.z *= keep, o.w *= keep;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float f = __builtin_amdgcn_exp2f(ml[i].x - use);
        l = fmaf(ml[i].y, f, l);
        o.x = fmaf(x[i].x, f, o.x), o.y = fmaf(x[i].y, f, o.y);
        o.z = fmaf(x[i].z, f, o.z), o.w = fmaf(x[i].w, f, o.w);
      }
    }
    float top = fmaxf(m, other32(m));
    if (PPW == 4) top = fmaxf(top, other16(top));
    const float f = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.0f : top));
    auto sum = [&](float v) {
      v *= f;
      v += other32(v);
      return PPW == 4 ? v + other16(v) : v;
    };
    l = sum(l);
    o = make_float4(sum(o.x), sum(o.y), sum(o.z), sum(o.w));
    if constexpr (W > 1) {
      if (lane < LPP) s_o[wid][lane] = o;
      if (lane == 0) s_ml[wid] = make_float2(top, l);
      __syncthreads();
      if (wid == 0) {
        float t2 = top;
#pragma unroll
        for (int i = 1; i < W; ++i) t2 = fmaxf(t2, s_ml[i].x);
        const float use = t2 == -INFINITY ? 0.0f : t2;
        l = 0.0f;
        o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < W; ++i) {
          const float2 ml = s_ml[i];
          const float4 x = s_o[i][e4];
          const float fi = __builtin_amdgcn_exp2f(ml.x - use);
          l = fmaf(ml.y, fi, l);
          o.x = fmaf(x.x, fi, o.x), o.y = fmaf(x.y, fi, o.y), o.z = fmaf(x.z, fi, o.z), o.w = fmaf(x.w, fi, o.w);
        }
      }
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    if (sub == 0)
      *reinterpret_cast<uint2*>(a.po + row_offset(a.o, row, hq) + e4 * 8) =
          make_uint2(pack2<BF>(o.x * inv, o.y * inv), pack2<BF>(o.z * inv, o.w * inv));
    if (W > 1) __syncthreads();  // the boxes are the next row's
  }
}

// The sequences' own keys alone.
template <int D, bool BF, int COLS>
__global__ __launch_bounds__(kThreads, COLS == 32 && D == 128 ? 1 : 2) void paged_kernel(const PagedArgs a, const PagedPass ps) {
  extern __shared__ __attribute__((aligned(16))) char dyn[];
  Seg* seg = reinterpret_cast<Seg*>(dyn);
  int total;
  schedule<COLS, 0>(a, ps, ps, seg, nullptr, &total, nullptr);
  const int parts = min(ps.grid, total);
  if (ps.fused) clear_empty<D>(a, ps, seg);
  else publish<COLS, step_keys<COLS>()>(a, ps, seg, total, parts, blockIdx.x, gridDim.x);
  if ((int)blockIdx.x >= parts) return;
  if constexpr (COLS <= 32) {
    __shared__ FewShared<D> sh;
    walk_few<D, BF, COLS>(a, ps, seg, sh, total, parts, blockIdx.x);
  } else {
    __shared__ ManyShared<D> sh;
    walk_many<D, BF, COLS>(a, ps, seg, nullptr, sh, total, parts, blockIdx.x);
  }
}

// Shared and own keys of a call with groups in one launch: as many workgroups
// as the chip holds at once, dealt to the two walks so that they end together.
template <int D, bool BF, int OWN, int SHARED>
__global__ __launch_bounds__(kThreads, 2) void paged_both_kernel(const PagedArgs a, const PagedPass own,
                                                                 const PagedPass shared) {
  extern __shared__ __attribute__((aligned(16))) char dyn[];
  Seg* seg_o = reinterpret_cast<Seg*>(dyn);
  Seg* seg_s = seg_o + own.n + 1;
  __shared__ union Both {
    __device__ Both() {}
    FewShared<D> few;
    ManyShared<D> many;
  } sh;
  constexpr int KO = step_keys<OWN>(), KS = step_keys<SHARED>();
  int to, ts;
  schedule<OWN, SHARED>(a, own, shared, seg_o, seg_s, &to, &ts);
  const int n = gridDim.x;
  // by the bytes that the walks read (with the measured times of their steps and
  // of beginning and ending a walk instead: 8K prefix 43 us against 40); in
  // multiples of eight, so that neighbouring parts stay on one XCD
  const double ws = (double)ts * KS, wo = (double)to * KO;
  const int ns = ts == 0 ? 0 : to == 0 ? n : min(max((int)(n * ws / (ws + wo) + 4.0) / 8 * 8, 8), n - 8);
  const int ps = min(ns, ts), po = min(n - ns, to);
  publish<OWN, KO>(a, own, seg_o, to, po, blockIdx.x, n);
  publish<SHARED, KS>(a, shared, seg_s, ts, ps, blockIdx.x, n);
  const int b = blockIdx.x;
  if (b < ns) {
    if (b >= ps) return;
    walk_many<D, BF, SHARED>(a, shared, seg_s, seg_o, sh.many, ts, ps, b);
  } else {
    if (b - ns >= po) return;
    if constexpr (OWN <= 32) walk_few<D, BF, OWN>(a, own, seg_o, sh.few, to, po, b - ns);
    else walk_many<D, BF, OWN>(a, own, seg_o, nullptr, sh.many, to, po, b - ns);
  }
}

template <int D, bool BF>
hipError_t run_own(const PagedArgs& a, const PagedPass& p, hipStream_t s) {
  const dim3 g(p.grid), b(kThreads);
  const size_t lds = (p.n + 1) * sizeof(Seg);
  if (p.cols == 16) {
    paged_kernel<D, BF, 16><<<g, b, lds, s>>>(a, p);
  } else if (p.cols == 32) {
    paged_kernel<D, BF, 32><<<g, b, lds, s>>>(a, p);
  } else if (p.cols == 64) {
    paged_kernel<D, BF, 64><<<g, b, lds, s>>>(a, p);
  } else {
    paged_kernel<D, BF, 128><<<g, b, lds, s>>>(a, p);
  }
  return hipGetLastError();
}
template <int D, bool BF, int OWN>
hipError_t run_both(const PagedArgs& a, const PagedPass& own, const PagedPass& sh, hipStream_t s) {
  const dim3 g(own.grid), b(kThreads);
  const size_t lds = (own.n + sh.n + 2) * sizeof(Seg);
  if (sh.cols == 64) paged_both_kernel<D, BF, OWN, 64><<<g, b, lds, s>>>(a, own, sh);
  else paged_both_kernel<D, BF, OWN, 128><<<g, b, lds, s>>>(a, own, sh);
  return hipGetLastError();
}

template <int D, bool BF>
hipError_t run_paged(const PagedArgs& a, const PagedPass& sh, const PagedPass& own, hipStream_t s) {
  hipError_t e = sh.n == 0         ? run_own<D, BF>(a, own, s)
                 : own.cols == 16  ? run_both<D, BF, 16>(a, own, sh, s)
                 : own.cols == 32  ? run_both<D, BF, D == 64 ? 32 : 16>(a, own, sh, s)
                 : own.cols == 64  ? run_both<D, BF, 64>(a, own, sh, s)
                                   : run_both<D, BF, 128>(a, own, sh, s);
  if (e != hipSuccess || own.fused) return e;
  const int64_t avg = (a.rows + (int64_t)a.n_seq - 1) / a.n_seq;
  const int heads = a.hkv * a.g;
  const uint32_t z = (uint32_t)(avg < 64 ? avg : 64);
  // the parts that a row may have: all the waves of a workgroup join many (one
  // wave a row, 4 and 16 of a workgroup: 16 sequences of 4K keys, 32 heads over 8,
  // 3 parts, 48.4, 49.0 and 51.3 us; 4 of 2K, 12 parts, 14.0, 13.8 and 14.4; 8 of
  // 32K, 4 over 1, 51 parts, 32.7, 29.9 and 30.4; 3 of 64K, 128 parts, 35.0, 27.1
  // and 27.0; one of 64K, 512 parts, 44.2, 21.3 and 17.9)
  const int parts = own.grid / (sh.n && sh.tiles < own.tiles ? sh.tiles : own.tiles);
  if (parts >= 128)
    paged_join_kernel<D, BF, 16><<<dim3(a.n_seq, heads, z), dim3(1024), 0, s>>>(a, sh, own);
  else if (parts >= 8)
    paged_join_kernel<D, BF, kWaves><<<dim3(a.n_seq, heads, z), dim3(kThreads), 0, s>>>(a, sh, own);
  else
    paged_join_kernel<D, BF, 1><<<dim3(a.n_seq, (heads + kWaves - 1) / kWaves, z), dim3(kThreads), 0, s>>>(a, sh, own);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged(const PagedArgs& a, const PagedPass& sh, const PagedPass& own, int32_t d, int32_t dt,
                        hipStream_t s) {
  if (d == 128) return dt == EA_BF16 ? run_paged<128, true>(a, sh, own, s) : run_paged<128, false>(a, sh, own, s);
  return dt == EA_BF16 ? run_paged<64, true>(a, sh, own, s) : run_paged<64, false>(a, sh, own, s);
}

}  // namespace ea
