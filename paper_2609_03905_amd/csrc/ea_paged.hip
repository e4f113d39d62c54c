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
// (rows x query heads of one key-value head) are cut in tiles of 16, its keys
// in chunks of a power of two times 128, long enough that about 4096 units
// (chunk, tile, key-value head) result.  The lengths are read on the device,
// by every workgroup for itself (a scan over the segments), so a captured
// launch serves batches that grow.
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

__device__ __forceinline__ int tiles_of(const PagedArgs& a, const Segment& s) {
  return (int)(((int64_t)(s.r1 - s.r0) * a.g + kPagedCols - 1) / kPagedCols);
}
__device__ __forceinline__ int chunks_of(const Segment& s, int shift) {  // chunk: 128 << shift keys
  return (int)(((int64_t)(s.k1 - s.k0) + (kPagedStep << shift) - 1) >> (7 + shift));
}
// Unit `local` of a segment: eight (chunk, head) streams, then the tiles, then
// the next eight streams.  Workgroup w works on units w, w + 8 n, ...: all
// tiles of a stream run on one XCD, whose L2 holds the keys they share.
__device__ __forceinline__ int unit_of(int base, int tiles, int stream, int tile) {
  return base + ((stream >> 3) * tiles + tile) * 8 + (stream & 7);
}

template <int D, bool BF>
__global__ __launch_bounds__(kThreads, 2) void paged_kernel(const PagedArgs a) {
  constexpr int VE = D / 16;          // d elements a lane holds of a V row
  constexpr int KS = D / 32;          // k steps of the score product
  constexpr int PITCH = D + 4;        // of a column in the waves' join (banks)
  __shared__ int s_base[kPagedMaxSeg + 1];
  __shared__ int64_t s_off[kWaves][2][32];
  __shared__ __attribute__((aligned(16))) float s_o[kWaves][kPagedCols][PITCH];
  __shared__ float s_ml[kWaves][kPagedCols][2];
  __shared__ unsigned long long s_work;
  __shared__ int s_sum[kThreads];

  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g4 = lane >> 4;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nseg = a.n_group + a.n_seq;
  const int per = (nseg + kThreads - 1) / kThreads;

  // ---- the schedule: chunk length, then every segment's first unit
  if (tid == 0) s_work = 0;
  __syncthreads();
  unsigned long long w = 0;
  for (int i = tid * per; i < min(nseg, (tid + 1) * per); ++i) {
    const Segment s = segment(a, i);
    w += (unsigned long long)tiles_of(a, s) * chunks_of(s, 0) * a.hkv;
  }
  if (w) atomicAdd(&s_work, w);
  __syncthreads();
  int shift = 0;
  while (shift < 20 && (s_work >> shift) > kPagedTarget) ++shift;
  int sum = 0;
  for (int i = tid * per; i < min(nseg, (tid + 1) * per); ++i) {
    const Segment s = segment(a, i);
    const int64_t n = (int64_t)tiles_of(a, s) * (((int64_t)chunks_of(s, shift) * a.hkv + 7) / 8 * 8);
    s_base[i] = sum;
    sum = (int)min((int64_t)a.cap, sum + n);
  }
  s_sum[tid] = sum;
  __syncthreads();
  for (int o = 1; o < kThreads; o *= 2) {
    const int v = tid >= o ? s_sum[tid - o] : 0;
    __syncthreads();
    s_sum[tid] = min(a.cap, s_sum[tid] + v);
    __syncthreads();
  }
  const int before = tid ? s_sum[tid - 1] : 0;
  for (int i = tid * per; i < min(nseg, (tid + 1) * per); ++i) s_base[i] = min(a.cap, s_base[i] + before);
  if (tid == 0) s_base[nseg] = s_sum[kThreads - 1];
  __syncthreads();
  const int total = s_base[nseg];
  if (blockIdx.x == 0) {  // for the join
    for (int i = tid; i < nseg; i += kThreads) {
      const Segment s = segment(a, i);
      if (i < a.n_group) {
        PagedGroup g;
        g.r0 = s.r0, g.base = s_base[i], g.chunks = chunks_of(s, shift), g.tiles = tiles_of(a, s);
        a.group[i] = g;
      } else {
        PagedSeq q = {};
        q.r0 = s.r0, q.r1 = s.r1, q.base = s_base[i], q.chunks = chunks_of(s, shift), q.group = s.group;
        a.seq[s.seq] = q;
      }
    }
  }

  for (int u = blockIdx.x; u < total; u += gridDim.x) {
    // ---- which unit
    int lo = 0, hi = nseg;  // s_base[lo] <= u < s_base[hi]; empty segments share a base
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s_base[mid] <= u) lo = mid;
      else hi = mid;
    }
    const int si = __builtin_amdgcn_readfirstlane(lo);
    const Segment s = segment(a, si);
    const int tiles = tiles_of(a, s), chunks = chunks_of(s, shift);
    const int local = u - s_base[si];
    const int eight = local >> 3, block = eight / tiles, tile = eight - block * tiles;
    const int stream = block * 8 + (local & 7);
    if (stream >= chunks * a.hkv) continue;  // the padding of the last eight
    const int chunk = stream / a.hkv, h = stream - chunk * a.hkv;
    const int ka = s.k0 + (int)((int64_t)chunk << (7 + shift));
    const int kb = (int)min((int64_t)s.k1, (int64_t)ka + ((int64_t)kPagedStep << shift));

    // ---- this lane's column: a query row and head, and the keys it sees
    const int ncol = (s.r1 - s.r0) * a.g;
    const int col = tile * kPagedCols + c;
    const int cc = min(col, ncol - 1);
    const int rr = div_fast(cc, a.gdiv), row = s.r0 + rr, head = h * a.g + cc - rr * a.g;
    int lim;
    if (si >= a.n_group) {
      lim = s.k1 - (s.r1 - s.r0) + rr + 1;
    } else {  // the row's own sequence says how far it sees
      int l2 = clampi(a.group_start[si], 0, a.n_seq), h2 = clampi(a.group_start[si + 1], l2, a.n_seq);
      while (h2 - l2 > 1) {
        const int mid = (l2 + h2) >> 1;
        if (first_row(a, mid) <= row) l2 = mid;
        else h2 = mid;
      }
      l2 = min(l2, a.n_seq - 1);
      const int ln = clampi(a.len[l2], 0, a.stride * a.page_size);
      lim = ln - (first_row(a, l2 + 1) - row) + 1;
    }
    if (col >= ncol) lim = 0x7fffffff;  // never stored: no mask
    int lim_min = lim;
    lim_min = min(lim_min, __shfl_xor(lim_min, 1));
    lim_min = min(lim_min, __shfl_xor(lim_min, 2));
    lim_min = min(lim_min, __shfl_xor(lim_min, 4));
    lim_min = __builtin_amdgcn_readfirstlane(min(lim_min, __shfl_xor(lim_min, 8)));

    uint4 q[KS];
    {
      const char* p = a.pq + row_offset(a.q, row, head) + g4 * 16;
#pragma unroll
      for (int i = 0; i < KS; ++i) q[i] = *reinterpret_cast<const uint4*>(p + i * 64);
    }
    const int32_t* pages = a.table + (int64_t)s.seq * a.stride;
    const int64_t head_off = (int64_t)h * a.page_size * D * 2;
    const char* kbase = a.pk + head_off + g4 * 16;
    const char* vbase = a.pv + head_off + c * VE * 2;

    f32x4_t acc[VE];
#pragma unroll
    for (int j = 0; j < VE; ++j) acc[j] = f32x4_t{};
    float m = -INFINITY, l = 0.0f;

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
      f32x4_t sc[2] = {};
#pragma unroll
      for (int i = 0; i < KS; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t) sc[t] = mfma16<BF>(kr[t][i], q[i], sc[t]);
      if (more) load_k(slot ^ 1);
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = sc[i >> 2][i & 3] * a.scale;
      if (!full) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int kk = 16 * (i >> 2) + 4 * g4 + (i & 3);
          const bool row_there = s_off[wid][slot][kk] >= 0;
          x[i] = row_there && k + kk < lim ? x[i] : -INFINITY;
          // a row that is not there was read elsewhere: it may hold anything
#pragma unroll
          for (int j = 0; j < VE / 2; ++j) vr[i][j] = row_there ? vr[i][j] : 0u;
        }
      }
      float mx = x[0];
#pragma unroll
      for (int i = 1; i < 8; ++i) mx = fmaxf(mx, x[i]);
      mx = fmaxf(mx, other16(mx));
      mx = fmaxf(mx, other32(mx));
      const float m_new = mx > m + kLazyMax || m == -INFINITY ? fmaxf(mx, m) : m;
      const float m_use = m_new == -INFINITY ? 0.0f : m_new;
      if (__any(m_new != m)) {
        const float alpha = __builtin_amdgcn_exp2f(m - m_use);
        l *= alpha;
#pragma unroll
        for (int j = 0; j < VE; ++j) acc[j] *= alpha;
      }
      m = m_new;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __builtin_amdgcn_exp2f(x[i] - m_use);
      uint4 p;
      p.x = pack_p<BF>(x[0], x[1], l);
      p.y = pack_p<BF>(x[2], x[3], l);
      p.z = pack_p<BF>(x[4], x[5], l);
      p.w = pack_p<BF>(x[6], x[7], l);
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;
        uint4 v;
        v.x = __builtin_amdgcn_perm(vr[1][j / 2], vr[0][j / 2], sel);
        v.y = __builtin_amdgcn_perm(vr[3][j / 2], vr[2][j / 2], sel);
        v.z = __builtin_amdgcn_perm(vr[5][j / 2], vr[4][j / 2], sel);
        v.w = __builtin_amdgcn_perm(vr[7][j / 2], vr[6][j / 2], sel);
        acc[j] = mfma16<BF>(v, p, acc[j]);
      }
      if (more) load_v(slot ^ 1);
      slot ^= 1;
      full = full_next;
    }
    l += other16(l);
    l += other32(l);

    // ---- join the four waves.  Lane (g4, c) holds d = (4 g4 + i) VE + j of
    // its column: 4 VE neighbours.
    if (g4 == 0) {
      s_ml[wid][c][0] = m;
      s_ml[wid][c][1] = l;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < VE; j += 4)
        *reinterpret_cast<float4*>(&s_o[wid][c][(4 * g4 + i) * VE + j]) =
            make_float4(acc[j][i], acc[j + 1][i], acc[j + 2][i], acc[j + 3][i]);
    __syncthreads();
    {
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
      const int64_t at = (int64_t)u * kPagedCols + jc;
      if (part == 0) {
        a.part_ml[2 * at] = top;
        a.part_ml[2 * at + 1] = lt;
      }
#pragma unroll
      for (int j = 0; j < VE; j += 4)
        *reinterpret_cast<float4*>(a.part_o + at * D + part * VE + j) = make_float4(o[j], o[j + 1], o[j + 2], o[j + 3]);
    }
    __syncthreads();
  }
}

// Join of a row's partial results: one wave a (row, query head), its parts in
// order (shared chunks, then own chunks).
template <int D, bool BF>
__global__ __launch_bounds__(kThreads) void paged_join_kernel(const PagedArgs a) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int seq = blockIdx.x, hq = blockIdx.y * kWaves + wid;
  if (hq >= a.hkv * a.g) return;
  const int h = div_fast(hq, a.gdiv), hg = hq - h * a.g;
  const PagedSeq q = a.seq[seq];
  PagedGroup g = {};
  if (q.group >= 0) g = a.group[q.group];
  const int own_tiles = (int)(((int64_t)(q.r1 - q.r0) * a.g + kPagedCols - 1) / kPagedCols);
  const int parts = g.chunks + q.chunks;
  for (int row = q.r0 + blockIdx.z; row < q.r1; row += gridDim.z) {
    auto place = [&](int p) -> int64_t {  // the part's column in the workspace
      int u, col;
      if (p < g.chunks) {
        col = (row - g.r0) * a.g + hg;
        u = unit_of(g.base, g.tiles, p * a.hkv + h, col / kPagedCols);
      } else {
        col = (row - q.r0) * a.g + hg;
        u = unit_of(q.base, own_tiles, (p - g.chunks) * a.hkv + h, col / kPagedCols);
      }
      u = min(u, a.cap - 1);
      return (int64_t)u * kPagedCols + col % kPagedCols;
    };
    float top = -INFINITY;
    for (int p = lane; p < parts; p += 64) top = fmaxf(top, a.part_ml[2 * place(p)]);
    top = wave_max(top);
    const float use = top == -INFINITY ? 0.0f : top;
    float l = 0.0f, o[E] = {};
    for (int p0 = 0; p0 < parts; p0 += 64) {
      const int p = p0 + lane;
      int64_t at = 0;
      float f = 0.0f, lp = 0.0f;
      if (p < parts) {
        at = place(p);
        f = __builtin_amdgcn_exp2f(a.part_ml[2 * at] - use);
        lp = a.part_ml[2 * at + 1] * f;
      }
      l += wave_sum(lp);
      const int n = min(64, parts - p0);
      for (int i0 = 0; i0 < n; i0 += 4) {  // four parts' loads at a time
        float x[4][E];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float* src = a.part_o + __shfl(at, min(i0 + i, n - 1)) * D + lane * E;
#pragma unroll
          for (int e = 0; e < E; ++e) x[i][e] = src[e];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float fi = __shfl(f, min(i0 + i, n - 1));
#pragma unroll
          for (int e = 0; e < E; ++e) o[e] = i0 + i < n ? fmaf(x[i][e], fi, o[e]) : o[e];
        }
      }
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    char* dst = a.po + row_offset(a.o, row, hq) + lane * E * 2;
    if constexpr (E == 2) {
      const float x = o[0] * inv, y = o[1] * inv;
      *reinterpret_cast<uint32_t*>(dst) =
          BF ? pack_bf16x2(x, y) : (uint32_t)f32_to_f16(x) | ((uint32_t)f32_to_f16(y) << 16);
    } else {
      const float x = o[0] * inv;
      *reinterpret_cast<uint16_t*>(dst) = BF ? f32_to_bf16(x) : f32_to_f16(x);
    }
  }
}

template <int D, bool BF>
hipError_t run_paged(const PagedArgs& a, hipStream_t s) {
  // two workgroups a CU; fewer where the workspace holds fewer units
  const int grid = a.cap < 512 ? a.cap : 512;
  paged_kernel<D, BF><<<dim3(grid), dim3(kThreads), 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t avg = (a.rows + (int64_t)a.n_seq - 1) / a.n_seq;
  const dim3 jg(a.n_seq, (a.hkv * a.g + kWaves - 1) / kWaves, (uint32_t)(avg < 64 ? avg : 64));
  paged_join_kernel<D, BF><<<jg, dim3(kThreads), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged(const PagedArgs& a, int32_t d, int32_t dt, hipStream_t s) {
  if (d == 128) return dt == EA_BF16 ? run_paged<128, true>(a, s) : run_paged<128, false>(a, s);
  return dt == EA_BF16 ? run_paged<64, true>(a, s) : run_paged<64, false>(a, s);
}

}  // namespace ea
