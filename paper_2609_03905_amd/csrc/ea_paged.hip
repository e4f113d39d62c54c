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
// (rows x query heads of one key-value head) are cut in tiles of 16 NC; the
// keys of each (segment, head, tile) are walked in steps of 128.  All steps of
// a launch lie end to end, and workgroup w of n takes the w-th n-th part of
// them, so that the work is even whatever the lengths are: a workgroup's part
// may end one tile's walk and begin the next one's, and a tile's walk has as
// many partial results as parts touch it.  The i-th tile's result from part w
// is slot i + w (one of the two grows from piece to piece).  The lengths are
// read on the device, by every workgroup for itself (a scan over the
// segments), so a captured launch serves batches that grow.  Parts that run on
// one XCD are neighbours: tiles over the same keys then share its L2.
//
// Bound by HBM: 16 columns of D = 128 need 4 * 128 * 16 operations on a key's
// 512 bytes, a tenth of what the matrix cores do while the bytes arrive.  So
// nothing is staged in shared memory: each wave walks its own 32 keys of a
// step and loads K and V from the pages straight into the registers of
//   S^T = K Q^T     (16x16x32: A = 16 keys x 32 d, B = 32 d x 16 columns)
//   O^T += V^T P^T  (A = 16 d x 32 keys, B = 32 keys x 16 columns)
// The B operand of the second product holds eight keys a lane, and the
// accumulators of two S^T tiles hold exactly eight keys of that lane's column:
// keys 4g + i and 16 + 4g + i (g = lane / 16).  A product may take its k index
// in any order, so V is loaded for those eight keys, 8 (or 4) neighbouring d a
// lane, and turned in registers: d index 16 m + j' becomes row m of tile j'.
// The addresses of a wave's 32 key rows come from the page table, one lane a
// key, through shared memory; a step's table entries are read a step ahead.
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

// Two weights rounded to the cache's type, and the same two as floats.  A
// rounding is off by at most half a step of the type relative to the weight
// (2^-8 in bf16, 2^-11 in fp16), no more than the output's own store; the sum
// takes the rounded weights too, so that an error common to numerator and
// denominator cancels.
template <bool BF>
__device__ __forceinline__ uint32_t pack_p(float a, float b, float& sum) {
  if constexpr (BF) {
    const uint32_t w = pack_bf16x2(a, b);
    sum += __uint_as_float(w << 16) + __uint_as_float(w & 0xffff0000u);
    return w;
  } else {
    const uint16_t x = f32_to_f16(a), y = f32_to_f16(b);
    sum += f16_to_f32(x) + f16_to_f32(y);
    return (uint32_t)x | ((uint32_t)y << 16);
  }
}

template <bool BF>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  return BF ? pack_bf16x2(a, b) : (uint32_t)f32_to_f16(a) | ((uint32_t)f32_to_f16(b) << 16);
}

// Part that workgroup b of n works on: XCD b mod 8 takes neighbouring parts.
__device__ __forceinline__ int xcd_part(int b, int n) {
  const int x = b & 7, per = n >> 3, more = n & 7;  // XCD x runs per workgroups, one more if x < more
  return x * per + min(x, more) + (b >> 3);
}

constexpr int64_t kMost = 0x7fffffff;

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return min(max(v, lo), hi); }

// First query row of sequence s (0 <= s <= n_seq).
__device__ __forceinline__ int first_row(const PagedArgs& a, int s) {
  return a.q_start ? clampi(a.q_start[s], 0, a.rows) : min(s, a.rows);
}

struct Segment {
  int r0, r1;  // query rows
  int k0, k1;  // keys
  int seq;     // whose table row lists the pages
  int group;   // own keys: the sequence's group or -1
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

__device__ __forceinline__ Segment segment(const PagedArgs& a, int i) {
  Segment s;
  if (i < a.n_group) {
    const int s0 = clampi(a.group_start[i], 0, a.n_seq), s1 = clampi(a.group_start[i + 1], s0, a.n_seq);
    s.seq = min(s0, a.n_seq - 1);
    s.r0 = first_row(a, s0);
    s.r1 = max(first_row(a, s1), s.r0);
    s.k0 = 0;
    s.k1 = shared_keys(a, i);
    s.group = -1;
  } else {
    s.seq = i - a.n_group;
    s.r0 = first_row(a, s.seq);
    s.r1 = max(first_row(a, s.seq + 1), s.r0);
    s.k1 = clampi(a.len[s.seq], 0, a.stride * a.page_size);
    s.group = group_of(a, s.seq);
    s.k0 = s.group >= 0 ? min(shared_keys(a, s.group), s.k1) : 0;
  }
  return s;
}

__device__ __forceinline__ int tiles_of(const PagedArgs& a, const Segment& s, int cols) {
  return (int)(((int64_t)(s.r1 - s.r0) * a.g + cols - 1) / cols);
}
__device__ __forceinline__ int steps_of(const Segment& s) { return (s.k1 - s.k0 + kPagedStep - 1) / kPagedStep; }

template <int D, bool BF, int NC>
__global__ __launch_bounds__(kThreads, NC > 1 ? 1 : 2) void paged_kernel(const PagedArgs a, const PagedPass ps) {
  constexpr int VE = D / 16;          // d elements a lane holds of a V row
  constexpr int KS = D / 32;          // k steps of the score product
  constexpr int PITCH = D + 4;        // of a column in the waves' join (banks)
  constexpr int COLS = kPagedCols * NC;
  __shared__ int s_step[kPagedMaxSeg + 1];  // first step of every segment
  __shared__ int s_tile[kPagedMaxSeg + 1];  // and its first tile
  __shared__ int64_t s_off[kWaves][2][32];
  __shared__ __attribute__((aligned(16))) float s_o[kWaves][kPagedCols][PITCH];
  __shared__ float s_ml[kWaves][kPagedCols][2];
  __shared__ int64_t s_sum[kThreads][2];

  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g4 = lane >> 4;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nseg = ps.n;
  const int per = (nseg + kThreads - 1) / kThreads;

  // ---- the schedule: every segment's first step and tile
  int64_t steps = 0, ntile = 0;
  for (int i = tid * per; i < min(nseg, (tid + 1) * per); ++i) {
    const Segment s = segment(a, ps.first + i);
    const int n = steps_of(s), t = n ? tiles_of(a, s, COLS) * a.hkv : 0;
    s_step[i] = (int)min(steps, kMost);
    s_tile[i] = (int)min(ntile, kMost);
    steps = min(steps + (int64_t)n * t, kMost);
    ntile = min(ntile + t, kMost);
  }
  s_sum[tid][0] = steps;
  s_sum[tid][1] = ntile;
  __syncthreads();
  for (int o = 1; o < kThreads && o < nseg; o *= 2) {
    const int64_t x = tid >= o ? s_sum[tid - o][0] : 0, y = tid >= o ? s_sum[tid - o][1] : 0;
    __syncthreads();
    s_sum[tid][0] = min(s_sum[tid][0] + x, kMost);
    s_sum[tid][1] = min(s_sum[tid][1] + y, kMost);
    __syncthreads();
  }
  const int64_t step0 = tid ? s_sum[tid - 1][0] : 0, tile0 = tid ? s_sum[tid - 1][1] : 0;
  for (int i = tid * per; i < min(nseg, (tid + 1) * per); ++i) {
    s_step[i] = (int)min(s_step[i] + step0, kMost);
    s_tile[i] = (int)min(s_tile[i] + tile0, kMost);
  }
  // with fewer segments than threads the scan stops early: the last one has all
  const int last = min(kThreads, (nseg + per - 1) / per) - 1;
  if (tid == 0) {
    s_step[nseg] = (int)s_sum[last][0];
    s_tile[nseg] = (int)s_sum[last][1];
  }
  __syncthreads();
  const int total = s_step[nseg];
  const int parts = min((int)gridDim.x, total);
  if (blockIdx.x == 0) {  // for the join
    for (int i = tid; i < nseg; i += kThreads) {
      const Segment s = segment(a, ps.first + i);
      PagedSeg g;
      g.r0 = s.r0, g.r1 = s.r1, g.step = s_step[i], g.steps = steps_of(s), g.tile = s_tile[i];
      g.tiles = tiles_of(a, s, COLS), g.group = s.group, g.total = total;
      a.seg[ps.first + i] = g;
    }
  }
  // part w of `parts` for this workgroup: neighbours on one XCD (workgroup b
  // runs on XCD b mod 8)
  if ((int)blockIdx.x >= parts) return;
  const int w = xcd_part(blockIdx.x, parts);
  int at = (int)((int64_t)total * w / parts);
  const int end = (int)((int64_t)total * (w + 1) / parts);

  while (at < end) {
    // ---- which tile, and how far this part walks it
    int lo = 0, hi = nseg;  // s_step[lo] <= at < s_step[hi]; empty segments share a step
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s_step[mid] <= at) lo = mid;
      else hi = mid;
    }
    const int si = __builtin_amdgcn_readfirstlane(lo);
    const Segment s = segment(a, ps.first + si);
    const bool shared = ps.first + si < a.n_group;
    const int n = steps_of(s), tiles = tiles_of(a, s, COLS);
    const int local = at - s_step[si], it = local / n, step = local - it * n;
    const int h = it / tiles, tile = it - h * tiles;
    const int walk = min(n - step, end - at);
    const int slot_out = s_tile[si] + it + w;
    // the only result of these columns: no join
    const bool whole = !shared && walk == n && (s.group < 0 || s.k0 == 0);
    const int ka = s.k0 + step * kPagedStep;
    const int kb = (int)min((int64_t)s.k1, (int64_t)ka + (int64_t)walk * kPagedStep);
    at += walk;

    // ---- this lane's columns: query rows and heads, and the keys they see
    const int ncol = (s.r1 - s.r0) * a.g;
    int lim[NC], lim_min = 0x7fffffff;
    uint4 q[NC][KS];
#pragma unroll
    for (int t = 0; t < NC; ++t) {
      const int col = tile * COLS + t * kPagedCols + c;
      const int cc = min(col, ncol - 1);
      const int rr = div_fast(cc, a.gdiv), row = s.r0 + rr, head = h * a.g + cc - rr * a.g;
      if (!shared) {
        lim[t] = s.k1 - (s.r1 - s.r0) + rr + 1;
      } else {  // the row's own sequence says how far it sees
        int l2 = clampi(a.group_start[si], 0, a.n_seq), h2 = clampi(a.group_start[si + 1], l2, a.n_seq);
        while (h2 - l2 > 1) {
          const int mid = (l2 + h2) >> 1;
          if (first_row(a, mid) <= row) l2 = mid;
          else h2 = mid;
        }
        l2 = min(l2, a.n_seq - 1);
        const int ln = clampi(a.len[l2], 0, a.stride * a.page_size);
        lim[t] = ln - (first_row(a, l2 + 1) - row) + 1;
      }
      if (col >= ncol) lim[t] = 0x7fffffff;  // never stored: no mask
      lim_min = min(lim_min, lim[t]);
      const char* p = a.pq + row_offset(a.q, row, head) + g4 * 16;
#pragma unroll
      for (int i = 0; i < KS; ++i) q[t][i] = *reinterpret_cast<const uint4*>(p + i * 64);
    }
    lim_min = min(lim_min, __shfl_xor(lim_min, 1));
    lim_min = min(lim_min, __shfl_xor(lim_min, 2));
    lim_min = min(lim_min, __shfl_xor(lim_min, 4));
    lim_min = __builtin_amdgcn_readfirstlane(min(lim_min, __shfl_xor(lim_min, 8)));

    const int32_t* pages = a.table + (int64_t)s.seq * a.stride;
    const int64_t head_off = (int64_t)h * a.page_size * D * 2;
    const char* kbase = a.pk + head_off + g4 * 16;
    const char* vbase = a.pv + head_off + c * VE * 2;

    f32x4_t acc[NC][VE];
    float m[NC], l[NC];
#pragma unroll
    for (int t = 0; t < NC; ++t) {
      m[t] = -INFINITY;
      l[t] = 0.0f;
#pragma unroll
      for (int j = 0; j < VE; ++j) acc[t][j] = f32x4_t{};
    }

    // a wave's step is 32 keys; lane i (and i + 32) looks after key i
    const int kl = lane & 31;
    auto entry = [&](int k) { return k + kl < kb ? pages[div_fast(k + kl, a.page)] : -1; };
    auto offset = [&](int k, int pg) -> int64_t {  // of the key's row, -1: no such row
      if ((uint32_t)pg >= (uint32_t)a.n_pages) return -1;
      const int key = k + kl, in = key - div_fast(key, a.page) * a.page_size;
      return pg * a.page_bytes + (int64_t)in * (D * 2);
    };
    uint4 kr[2][KS];
    uint32_t vr[8][VE / 2];
    auto load_k = [&](int slot) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int64_t off = s_off[wid][slot][16 * t + c];
        const char* p = kbase + (off < 0 ? 0 : off);
#pragma unroll
        for (int i = 0; i < KS; ++i) kr[t][i] = *reinterpret_cast<const uint4*>(p + i * 64);
      }
    };
    auto load_v = [&](int slot) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t off = s_off[wid][slot][16 * (i >> 2) + 4 * g4 + (i & 3)];
        const char* p = vbase + (off < 0 ? 0 : off);
        if constexpr (VE == 8) {
          const uint4 x = *reinterpret_cast<const uint4*>(p);
          vr[i][0] = x.x, vr[i][1] = x.y, vr[i][2] = x.z, vr[i][3] = x.w;
        } else {
          const uint2 x = *reinterpret_cast<const uint2*>(p);
          vr[i][0] = x.x, vr[i][1] = x.y;
        }
      }
    };
    int k = ka + wid * 32;
    bool full = false;  // every key of the step has a row and is seen by every column
    int next_pg = 0;
    if (k < kb) {
      const int64_t off = offset(k, entry(k));
      if (lane < 32) s_off[wid][0][kl] = off;
      full = __all(off >= 0) && k + 32 <= lim_min;
      next_pg = entry(k + kPagedStep);
      __builtin_amdgcn_wave_barrier();
      load_k(0);
      load_v(0);
    }
    int slot = 0;
    for (; k < kb; k += kPagedStep) {
      const bool more = k + kPagedStep < kb;
      bool full_next = false;
      if (more) {
        const int64_t off = offset(k + kPagedStep, next_pg);
        if (lane < 32) s_off[wid][slot ^ 1][kl] = off;
        full_next = __all(off >= 0) && k + kPagedStep + 32 <= lim_min;
        next_pg = entry(k + 2 * kPagedStep);
        __builtin_amdgcn_wave_barrier();
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
      if (more) load_k(slot ^ 1);
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
      uint4 p[NC];
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
        for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_exp2f(fmaf(sc[t][i >> 2][i & 3], a.scale, -m_use));
        p[t].x = pack_p<BF>(x[0], x[1], l[t]);
        p[t].y = pack_p<BF>(x[2], x[3], l[t]);
        p[t].z = pack_p<BF>(x[4], x[5], l[t]);
        p[t].w = pack_p<BF>(x[6], x[7], l[t]);
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
        for (int t = 0; t < NC; ++t) acc[t][j] = mfma16<BF>(v, p[t], acc[t][j]);
      }
      if (more) load_v(slot ^ 1);
      slot ^= 1;
      full = full_next;
    }
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
          char* dst = a.po + row_offset(a.o, s.r0 + rr, h * a.g + col - rr * a.g) + part * VE * 2;
          uint32_t x[VE / 2];
#pragma unroll
          for (int j = 0; j < VE; j += 2) x[j / 2] = pack2<BF>(o[j] * inv, o[j + 1] * inv);
          if constexpr (VE == 8) *reinterpret_cast<uint4*>(dst) = make_uint4(x[0], x[1], x[2], x[3]);
          else *reinterpret_cast<uint2*>(dst) = make_uint2(x[0], x[1]);
        }
      } else if (slot_out < ps.slots) {
        const int64_t to = (int64_t)slot_out * COLS + t * kPagedCols + jc;
        if (part == 0) {
          ps.part_ml[2 * to] = top;
          ps.part_ml[2 * to + 1] = lt;
        }
#pragma unroll
        for (int j = 0; j < VE; j += 4)
          *reinterpret_cast<float4*>(ps.part_o + to * D + part * VE + j) =
              make_float4(o[j], o[j + 1], o[j + 2], o[j + 3]);
      }
      __syncthreads();
    }
  }
}

// Join of a row's partial results: one wave a (row, query head), its parts in
// order (shared keys, then own).
template <int D, bool BF>
__global__ __launch_bounds__(kThreads) void paged_join_kernel(const PagedArgs a, const PagedPass sh,
                                                              const PagedPass own) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hq = blockIdx.y * kWaves + wid;
  if (hq >= a.hkv * a.g) return;
  const int h = div_fast(hq, a.gdiv), hg = hq - h * a.g;
  const PagedSeg q = a.seg[a.n_group + blockIdx.x];
  PagedSeg g = {};
  if (q.group >= 0) g = a.seg[q.group];
  for (int row = q.r0 + blockIdx.z; row < q.r1; row += gridDim.z) {
    // parts [first, first + n) of a walk, and the column of slot `first`
    auto range = [&](const PagedSeg& s, const PagedPass& p, int64_t* at) {
      if (s.steps == 0) return 0;
      const int col = (row - s.r0) * a.g + hg, tile = col / p.cols;
      const int it = h * s.tiles + tile;
      const int64_t n = min(p.grid, s.total), from = s.step + (int64_t)it * s.steps;
      const int w0 = (int)(((from + 1) * n - 1) / s.total), w1 = (int)(((from + s.steps) * n - 1) / s.total);
      *at = ((int64_t)s.tile + it + w0) * p.cols + (col - tile * p.cols);
      return min(w1 - w0 + 1, max(0, p.slots - (s.tile + it + w0)));
    };
    int64_t at_g = 0, at_q = 0;
    const int n_g = range(g, sh, &at_g), n_q = range(q, own, &at_q);
    if (n_g == 0 && n_q == 1) continue;  // stored by the walk itself
    auto ml_of = [&](int p) {
      return p < n_g ? sh.part_ml + 2 * (at_g + (int64_t)p * sh.cols)
                     : own.part_ml + 2 * (at_q + (int64_t)(p - n_g) * own.cols);
    };
    const int parts = n_g + n_q;
    float top = -INFINITY;
    for (int p = lane; p < parts; p += 64) top = fmaxf(top, *ml_of(p));
    top = wave_max(top);
    const float use = top == -INFINITY ? 0.0f : top;
    float l = 0.0f, o[E] = {};
    for (int p0 = 0; p0 < parts; p0 += 64) {
      const int n = min(64, parts - p0);
      float f = 0.0f, lp = 0.0f;
      if (lane < n) {
        const float* ml = ml_of(p0 + lane);
        f = __builtin_amdgcn_exp2f(ml[0] - use);
        lp = ml[1] * f;
      }
      l += wave_sum(lp);
      for (int i0 = 0; i0 < n; i0 += 8) {  // eight parts' loads at a time
        float x[8][E];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int p = p0 + min(i0 + i, n - 1);
          const float* src = (p < n_g ? sh.part_o + (at_g + (int64_t)p * sh.cols) * D
                                      : own.part_o + (at_q + (int64_t)(p - n_g) * own.cols) * D) + lane * E;
#pragma unroll
          for (int e = 0; e < E; ++e) x[i][e] = src[e];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float fi = __shfl(f, min(i0 + i, n - 1));
#pragma unroll
          for (int e = 0; e < E; ++e) o[e] = i0 + i < n ? fmaf(x[i][e], fi, o[e]) : o[e];
        }
      }
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    char* dst = a.po + row_offset(a.o, row, hq) + lane * E * 2;
    if constexpr (E == 2) *reinterpret_cast<uint32_t*>(dst) = pack2<BF>(o[0] * inv, o[1] * inv);
    else *reinterpret_cast<uint16_t*>(dst) = BF ? f32_to_bf16(o[0] * inv) : f32_to_f16(o[0] * inv);
  }
}

template <int D, bool BF>
hipError_t run_pass(const PagedArgs& a, const PagedPass& p, hipStream_t s) {
  const dim3 g(p.grid), b(kThreads);
  if (p.cols == 16) paged_kernel<D, BF, 1><<<g, b, 0, s>>>(a, p);
  else if (p.cols == 32) paged_kernel<D, BF, 2><<<g, b, 0, s>>>(a, p);
  else paged_kernel<D, BF, 4><<<g, b, 0, s>>>(a, p);
  return hipGetLastError();
}

template <int D, bool BF>
hipError_t run_paged(const PagedArgs& a, const PagedPass& sh, const PagedPass& own, hipStream_t s) {
  hipError_t e;
  if (sh.n && (e = run_pass<D, BF>(a, sh, s)) != hipSuccess) return e;
  if ((e = run_pass<D, BF>(a, own, s)) != hipSuccess) return e;
  const int64_t avg = (a.rows + (int64_t)a.n_seq - 1) / a.n_seq;
  const dim3 jg(a.n_seq, (a.hkv * a.g + kWaves - 1) / kWaves, (uint32_t)(avg < 64 ? avg : 64));
  paged_join_kernel<D, BF><<<jg, dim3(kThreads), 0, s>>>(a, sh, own);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged(const PagedArgs& a, const PagedPass& sh, const PagedPass& own, int32_t d, int32_t dt,
                        hipStream_t s) {
  if (d == 128) return dt == EA_BF16 ? run_paged<128, true>(a, sh, own, s) : run_paged<128, false>(a, sh, own, s);
  return dt == EA_BF16 ? run_paged<64, true>(a, sh, own, s) : run_paged<64, false>(a, sh, own, s);
}

}  // namespace ea
