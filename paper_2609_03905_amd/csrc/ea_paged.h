// ea_paged.h -- what the walks over a paged cache share, whatever their elements:
// the schedule of a call's steps, a column's limits, the products, and the join
// of partial results (ea_paged.hip says how a call is cut).
#pragma once

#include "ea_decode.h"
#include "ea_device.h"

namespace ea {

namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr float kLazyMax = 8.0f;  // log2 of the largest P: the running max moves only past this

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
  asm("" : "+v"(hi));  // (else a is rounded once more, alone, for what it leaves)
  if constexpr (BF) lo = pack2<BF>(a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xffff0000u));
  else lo = pack2<BF>(a - f16_to_f32((uint16_t)hi), b - f16_to_f32((uint16_t)(hi >> 16)));
}

// Part that workgroup b of n works on: XCD b mod 8 takes neighbouring parts.
__device__ __forceinline__ int xcd_part(int b, int n) {
  const int x = b & 7, per = n >> 3, more = n & 7;  // XCD x runs per workgroups, one more if x < more
  return x * per + min(x, more) + (b >> 3);
}

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return min(max(v, lo), hi); }

struct Segment {
  int r0, r1;  // query rows (of sequence s: q_start[s] to q_start[s + 1], or s)
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
  if (a.n_group == 0) return -1;
  const int first = a.group_start[0], last = a.group_start[a.n_group];
  if ((s < first) | (s >= last)) return -1;
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
    const int first = a.group_start[i], last = a.group_start[i + 1], keys = shared_keys(a, i);
    const int s0 = clampi(first, 0, a.n_seq), s1 = clampi(last, s0, a.n_seq);
    int r0 = s0, r1 = s1;
    if (a.q_start) r0 = a.q_start[s0], r1 = a.q_start[s1];
    s.r0 = clampi(r0, 0, a.rows);
    s.r1 = max(clampi(r1, 0, a.rows), s.r0);
    s.k0 = 0;
    s.k1 = keys;
    s.seq = min(s0, a.n_seq - 1);
  } else {
    // (loads that wait for none of the others first, so that they are one round trip)
    const int seq = i - a.n_group, len = a.len[seq];
    int r0 = seq, r1 = seq + 1;
    if (a.q_start) r0 = a.q_start[seq], r1 = a.q_start[seq + 1];
    const int g = group_of(a, seq);
    s.r0 = clampi(r0, 0, a.rows);
    s.r1 = max(clampi(r1, 0, a.rows), s.r0);
    s.k1 = clampi(len, 0, a.stride * a.page_size);
    s.k0 = g >= 0 ? min(shared_keys(a, g), s.k1) : 0;
    s.seq = seq;
  }
  return s;
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

// Inclusive sums over a wave's lanes, no larger than 2^31 - 1, of N values side by
// side: one's shuffles are on their way with the others'.
template <int N>
__device__ __forceinline__ void wave_scan(int (&v)[N]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    int u[N];
#pragma unroll
    for (int k = 0; k < N; ++k) u[k] = __shfl_up(v[k], o);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = lane >= o ? add_most(v[k], u[k]) : v[k];
  }
}

__device__ __forceinline__ int steps_of(int k0, int k1, int keys) {
  return (int)(((int64_t)k1 - k0 + keys - 1) / keys);
}
__device__ __forceinline__ int tiles_of(int rows, int g, int cols) {
  return (int)(((int64_t)rows * g + cols - 1) / cols);
}

// Every segment's first step and tile, by the whole workgroup: the groups' (none
// where SHARED is 0) and the sequences', whose loads are one round trip.  *to and
// *ts: the steps (of OWN_KEYS and SHARED_KEYS keys) of all; none where there are
// more tiles than the rows can have, that is, where the sequences' rows overlap.
template <int OWN, int OWN_KEYS, int SHARED, int SHARED_KEYS>
__device__ __forceinline__ void schedule(const PagedArgs& a, const PagedPass& own, const PagedPass& shared, Seg* seg_o,
                                         Seg* seg_s, int* to, int* ts) {
  constexpr int N = SHARED ? 4 : 2;  // steps and tiles of the sequences, and of the groups
  __shared__ int s_wave[kWaves][N];
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  const int ng = SHARED ? shared.n : 0, n = ng + own.n;
  // segments of a thread: the groups first, or, where there are few, by the last
  // threads, whose loads then wait beside the sequences' and not before them
  const int per = (n + kThreads - 1) / kThreads;
  int i0 = min(n, tid * per), i1 = min(n, i0 + per);
  if (SHARED && per == 1) {
    i0 = tid < own.n ? ng + tid : tid >= kThreads - ng ? tid - (kThreads - ng) : n;
    i1 = min(n, i0 + 1);
  }
  int mine[N] = {};
  for (int i = i0; i < i1; ++i) {
    const bool g = SHARED && i < ng;
    const Segment s = segment(a, i);
    const int keys = g ? SHARED_KEYS : OWN_KEYS, cols = g ? SHARED : OWN;
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
  for (int k = 0; k < N; ++k) sum[k] = mine[k];
  wave_scan(sum);
#pragma unroll
  for (int k = 0; k < N; ++k)
    if (lane == 63) s_wave[wid][k] = sum[k];
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves - 1; ++w)
#pragma unroll
    for (int k = 0; k < N; ++k) sum[k] = add_most(sum[k], w < wid ? s_wave[w][k] : 0);
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

// The end of a piece of a walk over few columns, by the whole workgroup: the
// waves' results joined and stored, to the output or (slot_out) for the join;
// fused, the last part of a tile to arrive joins the tile's.
template <int D, bool BF, int COLS, class Shared>
__device__ __forceinline__ void finish_few(const PagedArgs& a, const PagedPass& ps, const Piece& p, int slot_out,
                                           f32x4_t (&acc)[COLS / kPagedCols][D / 16],
                                           const float (&m)[COLS / kPagedCols], float (&l)[COLS / kPagedCols],
                                           Shared& sh, int total, int parts) {
  constexpr int NC = COLS / kPagedCols, VE = D / 16;
  auto& s_o = sh.o;
  auto& s_ml = sh.ml;
  int& s_last = sh.last;
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g4 = lane >> 4;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Seg& s = p.s;
  const int h = p.h, tile = p.tile, it = p.it, n = p.n, ncol = s.rows * a.g;
  const bool whole = p.whole;
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
  if (!ps.fused || whole) return;

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

}  // namespace

}  // namespace ea
