// ea_cache8.hip -- a paged cache in 8 bits: rows quantised as they are written,
// and read back.
//
// A cache's codes c stand for c s, s the scale of the code's head and block of B
// neighbouring rows of a page.  For the rows x that a write puts into a block, K
// and V and every head apart,
//   a = max |x| over the finite ones,   e = the least whole number with a <= M 2^e
// (M the largest code, 448 or 57344; e in [-120, 120]), and the block's scale is
// 2^e, or the one it has if that is larger and the block holds rows of earlier
// calls; where the scale is another one then, their codes become round(c s_old / s).  Then
// c = round(x / s).  Scales being powers of two, both quotients are exact in 32
// bits, so that a code is off by its own rounding alone, and one that is rounded
// again changes only where it falls below the code's normal range.
//
// Rows of a block are neighbours both in the call and in the page, so a block's
// head is one wave's: the rows stay in registers between the maximum and the
// codes.  What bounds both calls, and what was measured, stands at the kernels.
#include "ea_decode.h"
#include "ea_device.h"

namespace ea {

namespace {

constexpr int kThreads = 256, kWaves = 4;

// Eight elements of a row.
template <int DT>
struct Eight {
  uint4 v[DT == EA_F32 ? 2 : 1];
  __device__ __forceinline__ void load(const char* p) {
    v[0] = *reinterpret_cast<const uint4*>(p);
    if constexpr (DT == EA_F32) v[1] = *reinterpret_cast<const uint4*>(p + 16);
  }
  __device__ __forceinline__ void values(float (&x)[8]) const {
    const uint32_t w[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
    if constexpr (DT == EA_F32) {
      const uint32_t u[4] = {v[1].x, v[1].y, v[1].z, v[1].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]), x[4 + i] = __uint_as_float(u[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = DT == EA_BF16 ? __uint_as_float(w[i] << 16) : f16_to_f32((uint16_t)w[i]);
        x[2 * i + 1] = DT == EA_BF16 ? __uint_as_float(w[i] & 0xffff0000u) : f16_to_f32((uint16_t)(w[i] >> 16));
      }
    }
  }
};

// The largest |x| of several, as bits, which are ordered as the values are (NaN
// above infinity): two halves of a word each, or a word.
template <int DT>
struct Largest {
  uint32_t bits = 0;
  __device__ __forceinline__ void one(uint32_t w) {
    if constexpr (DT == EA_F32) {
      bits = max(bits, w & 0x7fffffffu);
    } else {
      typedef unsigned short v2 __attribute__((ext_vector_type(2)));
      bits = __builtin_bit_cast(
          uint32_t, __builtin_elementwise_max(__builtin_bit_cast(v2, bits), __builtin_bit_cast(v2, w & 0x7fff7fffu)));
    }
  }
  __device__ __forceinline__ void add(const Eight<DT>& e) {
#pragma unroll
    for (const uint4& w : e.v) one(w.x), one(w.y), one(w.z), one(w.w);
  }
  __device__ __forceinline__ float value() const {  // infinity or NaN if one was not finite
    if constexpr (DT == EA_F32) return __uint_as_float(bits);
    const uint32_t w = max(bits & 0xffffu, bits >> 16);
    return DT == EA_BF16 ? __uint_as_float(w << 16) : f16_to_f32((uint16_t)w);
  }
};

// x / f (a power of two) rounded to codes, to nearest, ties to even; what is not
// finite has the code that stands for it (e4m3 has none for an infinity: NaN).
typedef short s16x2_t __attribute__((ext_vector_type(2)));
template <bool E5>
__device__ __forceinline__ uint2 encode(const float (&x)[8], float f) {
  s16x2_t w[2] = {};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (E5) {
      w[i] = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(w[i], x[4 * i], x[4 * i + 1], f, false);
      w[i] = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(w[i], x[4 * i + 2], x[4 * i + 3], f, true);
    } else {
      w[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w[i], x[4 * i], x[4 * i + 1], f, false);
      w[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w[i], x[4 * i + 2], x[4 * i + 3], f, true);
    }
  }
  return make_uint2(__builtin_bit_cast(uint32_t, w[0]), __builtin_bit_cast(uint32_t, w[1]));
}
// Two elements of 16 bits of a word each.
template <int DT, bool E5>
__device__ __forceinline__ uint32_t encode4(uint32_t a, uint32_t b, float f) {
  s16x2_t w = {};
  if constexpr (DT == EA_BF16) {
    typedef __bf16 v2 __attribute__((ext_vector_type(2)));
    const v2 x = __builtin_bit_cast(v2, a), y = __builtin_bit_cast(v2, b);
    if constexpr (E5) {
      w = __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(w, x, f, false);
      w = __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(w, y, f, true);
    } else {
      w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, x, f, false);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, y, f, true);
    }
  } else {
    typedef _Float16 v2 __attribute__((ext_vector_type(2)));
    const v2 x = __builtin_bit_cast(v2, a), y = __builtin_bit_cast(v2, b);
    if constexpr (E5) {
      w = __builtin_amdgcn_cvt_scalef32_pk_bf8_f16(w, x, f, false);
      w = __builtin_amdgcn_cvt_scalef32_pk_bf8_f16(w, y, f, true);
    } else {
      w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(w, x, f, false);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(w, y, f, true);
    }
  }
  return __builtin_bit_cast(uint32_t, w);
}

typedef float f32x2_t __attribute__((ext_vector_type(2)));
template <bool E5>
__device__ __forceinline__ void decode4(uint32_t w, float* x) {
  f32x2_t a, b;
  if constexpr (E5) {
    a = __builtin_amdgcn_cvt_pk_f32_bf8(w, false);
    b = __builtin_amdgcn_cvt_pk_f32_bf8(w, true);
  } else {
    a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
    b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  }
  x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1];
}

// The exponent of the least scale under which a (finite, not negative) has a code.
template <bool E5>
__device__ __forceinline__ int least_exponent(float a) {
  const int bits = __float_as_int(a);
  const int e = (bits >> 23) - 127 - (E5 ? 15 : 8) + ((bits & 0x7fffff) > 0x600000);  // M is 1.75 2^15, or 2^8
  return min(max(e, -kScaleExp), kScaleExp);
}
__device__ __forceinline__ float power(int e) { return __int_as_float((e + 127) << 23); }

// c f, where it is no 32-bit number the neighbour whose last bit is set, so that
// rounding it to fewer bits is one rounding of the product (28 bits: exact in 64).
__device__ __forceinline__ float product_to_odd(float c, float f) {
  const double exact = (double)c * (double)f;
  const float p = (float)exact;
  const int bits = __float_as_int(p);
  if ((double)p == exact || !(fabsf(p) < INFINITY) || (bits & 1)) return p;
  return __int_as_float(bits + (fabs(exact) > fabs((double)p) ? 1 : -1));
}

__device__ __forceinline__ int first_row(const Cache8Args& a, int s) { return min(max(a.q_start[s], 0), a.rows); }

// Where row t of the call lies in the cache.
struct Place {
  int page, in, at;  // page (-1: the row has none), row of the page, position
  bool mine;         // the row is a sequence's
};

// q_start's first rows in shared memory: all threads of the workgroup take part.
__device__ __forceinline__ void load_starts(const Cache8Args& a, int* starts) {
  if (a.q_start)
    for (int i = threadIdx.x; i <= a.n_seq; i += kThreads) starts[i] = first_row(a, i);
  __syncthreads();
}

__device__ __forceinline__ Place place_of(const Cache8Args& a, const int* starts, int t) {
  Place p = {-1, 0, 0, false};
  int s = t, r0 = t, r1 = t + 1;
  if (a.q_start) {
    int hi = a.n_seq;  // starts[s] <= t < starts[hi], if they ascend and t is a sequence's
    s = 0;
    while (hi - s > 1) {
      const int mid = (s + hi) >> 1;
      if (starts[mid] <= t) s = mid;
      else hi = mid;
    }
    r0 = starts[s], r1 = starts[s + 1];
  }
  if (s >= a.n_seq || t < r0 || t >= r1 || t >= a.rows) return p;
  p.mine = true;
  if (a.slots && a.slots[r0] < 0) return p;
  p.at = min(max(a.len[s], 0), a.stride * a.page_size) - r1 + t;
  if (p.at < 0) return p;
  const int i = div_fast(p.at, a.page);
  p.in = p.at - i * a.page_size;
  const int pg = a.table[(int64_t)s * a.stride + i];
  p.page = (uint32_t)pg < (uint32_t)a.n_pages ? pg : -1;
  return p;
}

// What a workgroup of the write knows of a sequence.
struct Span {
  int begun;       // blocks that the sequences before it write to
  int r1;          // behind its last row
  int first, end;  // positions of its first new row and behind its last
};

template <class T>
__device__ __forceinline__ T wave_scan(T v) {  // inclusive sums over the lanes
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const T u = __shfl_up(v, o);
    if ((int)(threadIdx.x & 63) >= o) v += u;
  }
  return v;
}

// Every sequence's span, by the whole workgroup; returns the blocks of all (none
// where there are more rows than the call has, that is, where they overlap).
__device__ __forceinline__ int schedule_write(const Cache8Args& a, Span* spans) {
  __shared__ int64_t s_wave[2][kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  const int per = (a.n_seq + kThreads - 1) / kThreads;
  const int i0 = min(a.n_seq, tid * per), i1 = min(a.n_seq, i0 + per);
  int64_t blocks = 0, rows = 0;
  for (int i = i0; i < i1; ++i) {
    const int r0 = a.q_start ? first_row(a, i) : i, r1 = a.q_start ? max(first_row(a, i + 1), r0) : i + 1;
    Span s;
    s.begun = (int)min(blocks, (int64_t)0x7fffffff);
    s.r1 = r1;
    s.end = min(max(a.len[i], 0), a.stride * a.page_size);
    s.first = max(s.end - (r1 - r0), 0);
    if (a.slots && r1 > r0 && r0 < a.rows && a.slots[r0] < 0) s.first = s.end;  // (its length counts no such rows)
    spans[i] = s;
    if (s.end > s.first) blocks += div_fast(s.end - 1, a.block) - div_fast(s.first, a.block) + 1;
    rows += r1 - r0;
  }
  const int64_t upto = wave_scan(blocks), upto_rows = wave_scan(rows);
  if (lane == 63) s_wave[0][wid] = upto, s_wave[1][wid] = upto_rows;
  __syncthreads();
  int64_t before = upto - blocks, total = 0, n = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wid) before += s_wave[0][w];
    total += s_wave[0][w];
    n += s_wave[1][w];
  }
  for (int i = i0; i < i1; ++i) spans[i].begun += (int)before;
  __syncthreads();
  return n > a.rows ? 0 : (int)total;
}

// A unit is a block's head, of K or of V: one wave's.  Units lie block by block and
// every wave takes an equal stretch, so that it looks a block up once for its heads;
// it fetches the rows of a unit while it works on the one before.  HELD: passes over
// a unit's rows that stay in registers between the maximum and the codes (others are
// read twice): 4 and two units at a time, or 16 (f32 8) of one unit for long blocks.
// Bound by HBM: 65 thousand tokens of 32 sequences, 8 heads of 128, blocks of 16,
// bf16, in 88 us, 4.6 TB/s (one unit at a time, rows dealt to workgroups by position,
// 150 us); 8192 tokens of one sequence, blocks of 64, in 14.2 us, 3.5 TB/s, of which
// 7 are the launch and the first rows' round trips; 64 sequences of one token each
// are 6.7 us, a chain of three round trips (schedule, table, rows).
template <int DT, bool E5, int HELD>
__global__ __launch_bounds__(kThreads) void cache8_write_kernel(const Cache8Args a) {
  extern __shared__ __attribute__((aligned(16))) char dyn[];
  Span* spans = reinterpret_cast<Span*>(dyn);
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lpr = a.d / 8, rows_pass = 64 / lpr;  // lanes of a row, rows of a pass
  const int r = lane / lpr, el = lane - r * lpr, sides = 2 * a.hkv;
  constexpr int ES = DT == EA_F32 ? 4 : 2;
  const int64_t units = (int64_t)__builtin_amdgcn_readfirstlane(schedule_write(a, spans)) * sides;
  const int w = blockIdx.x * kWaves + wid, waves = gridDim.x * kWaves;
  const int end = (int)(units * (w + 1) / waves);
  int u = (int)(units * w / waves);
  if (u >= end) return;

  struct Block {
    int n, before, passes;  // new rows, rows before them, passes over them
    int page, blk, t0;
  };
  struct Unit {
    Block b;
    int h;
    bool v, one;
    int64_t first, pitch;
    Eight<DT> held[HELD];
  };
  auto block_of = [&](int lead) {
    Block z;
    int s = 0, hi = a.n_seq;
    while (hi - s > 1) {
      const int mid = (s + hi) >> 1;
      if (spans[mid].begun <= lead) s = mid;
      else hi = mid;
    }
    s = __builtin_amdgcn_readfirstlane(s);
    const int r1 = __builtin_amdgcn_readfirstlane(spans[s].r1), begun = __builtin_amdgcn_readfirstlane(spans[s].begun);
    const int first = __builtin_amdgcn_readfirstlane(spans[s].first), last = __builtin_amdgcn_readfirstlane(spans[s].end);
    const int begin = (div_fast(first, a.block) + lead - begun) * a.block_rows, at = max(first, begin);
    z.n = min(begin + a.block_rows, last) - at;
    z.before = at - begin;
    z.t0 = r1 - (last - at);
    const int page = div_fast(at, a.page);
    z.blk = div_fast(begin - page * a.page_size, a.block);
    z.page = ld_uniform(a.table + (int64_t)s * a.stride + page);
    z.passes = (z.n + rows_pass - 1) / rows_pass;
    return z;
  };
  auto load = [&](const Unit& z, int p, Eight<DT>& e) {  // (lanes without a row take the last one's)
    const int i = min(p * rows_pass + r, z.b.n - 1);
    e.load((z.v ? a.pxv : a.pxk) + (z.one ? z.first + i * z.pitch : row_offset(z.v ? a.xv : a.xk, z.b.t0 + i, z.h)) +
           el * 8 * ES);
  };
  auto fetch = [&](const Block& b, int x, Unit& z) {
    z.b = b;
    z.v = x >= a.hkv;
    z.h = z.v ? x - a.hkv : x;
    // neighbouring rows of the relation's one block lie a pitch apart
    const RowMap map = z.v ? a.xv : a.xk;
    const int tb = div_fast(b.t0, map.tdiv), hb = div_fast(z.h, map.hdiv);
    z.one = b.t0 + b.n <= (tb + 1) * (int64_t)map.tb;
    z.first = row_offset(map, b.t0, z.h);
    z.pitch = map.row_bytes * (map.head_major ? 1 : min(map.hb, map.h - hb * map.hb));
#pragma unroll
    for (int p = 0; p < HELD; ++p)
      if (p < b.passes) load(z, p, z.held[p]);
  };
  auto work = [&](Unit& z) {
    if ((uint32_t)z.b.page >= (uint32_t)a.n_pages) return;
    float* scale = (z.v ? a.vs : a.ks) + ((int64_t)z.b.page * a.hkv + z.h) * a.n_blocks + z.b.blk;
    char* dst = (z.v ? a.pv : a.pk) + z.b.page * a.page_bytes +
                ((int64_t)z.h * a.page_size + z.b.blk * a.block_rows) * a.d + el * 8;
    const float old = z.b.before ? *scale : 0.0f;
    Largest<DT> largest;
#pragma unroll
    for (int p = 0; p < HELD; ++p)
      if (p < z.b.passes) largest.add(z.held[p]);
    for (int p = HELD; p < z.b.passes; ++p) {
      Eight<DT> x;
      load(z, p, x);
      largest.add(x);
    }
    float top = largest.value();
    if (__builtin_expect(__any(!(top < INFINITY)), 0)) {  // of the finite ones, then
      top = 0.0f;
#pragma unroll 1
      for (int p = 0; p < z.b.passes; ++p) {
        Eight<DT> x;
        load(z, p, x);
        float y[8];
        x.values(y);
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(y[j]) < INFINITY ? fabsf(y[j]) : 0.0f);
      }
    }
    int e = least_exponent<E5>(wave_max(top));
    if (old > 0.0f && old < INFINITY) {
      // (a scale that another program left may be no power of two: the next one; or
      // past 2^120, which then holds whatever the codes stood for: a 32-bit number's
      // code is below 256 under it)
      const int bits = __float_as_int(old);
      e = max(e, min(max((bits >> 23) - 127 + ((bits & 0x7fffff) != 0), -kScaleExp), kScaleExp));
      const float ratio = old * power(-e);
      if (ratio != 1.0f)
#pragma unroll 1
        for (int b = r; b < z.b.before && r < rows_pass; b += rows_pass) {
          uint2* at = reinterpret_cast<uint2*>(dst + (int64_t)b * a.d);
          const uint2 c = *at;
          float y[8];
          decode4<E5>(c.x, y);
          decode4<E5>(c.y, y + 4);
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = product_to_odd(y[j], ratio);
          *at = encode<E5>(y, 1.0f);
        }
    }
    const float s = power(e);
    auto store = [&](int p, const Eight<DT>& x) {
      const int i = p * rows_pass + r;
      if (r >= rows_pass || i >= z.b.n) return;
      uint2 c;
      if constexpr (DT == EA_F32) {
        float y[8];
        x.values(y);
        c = encode<E5>(y, s);
      } else {
        c = make_uint2(encode4<DT, E5>(x.v[0].x, x.v[0].y, s), encode4<DT, E5>(x.v[0].z, x.v[0].w, s));
      }
      store_stream(dst + (int64_t)(z.b.before + i) * a.d, c);
    };
#pragma unroll
    for (int p = 0; p < HELD; ++p)
      if (p < z.b.passes) store(p, z.held[p]);
    for (int p = HELD; p < z.b.passes; ++p) {
      Eight<DT> x;
      load(z, p, x);
      store(p, x);
    }
    if (lane == 0) *scale = s;
  };

  int lead = u / sides, x = u - lead * sides;
  Block b = block_of(lead);
  Unit z0;
  fetch(b, x, z0);
  auto next = [&](Unit& z) {
    if (++u >= end) return false;
    if (++x == sides) {
      x = 0;
      b = block_of(++lead);
    }
    fetch(b, x, z);
    return true;
  };
  if constexpr (HELD > 4) {  // (enough on their way in one)
    do work(z0);
    while (next(z0));
  } else {
    Unit z1;
    while (true) {
      const bool one = next(z1);
      work(z0);
      if (!one) break;
      const bool two = next(z0);
      work(z1);
      if (!two) break;
    }
  }
}

// ---- reading back -----------------------------------------------------------------
// Pieces of 8 codes, a thread each and UNROLL in flight; stores are whole lines.
// Bound by HBM: 196 thousand rows of 48 sequences, 8 heads of 128, to bf16 in 220 us,
// 5.5 TB/s (places looked up by every thread, a row a wave: 268 us; loads guarded by
// branches, so that they wait one for another: 281).  One sequence of 1000 rows in
// 7.0 us, a chain of four round trips: first rows, table, codes and scale, store.
constexpr int kReadRows = 16;

// Where a row lies, in the cache and in the call.
struct ReadRow {
  int64_t code, scale;       // head 0's (code -1: none)
  int64_t out[2], pitch[2];  // K's and V's head 0, and from head to head
  int mine;                  // the row is a sequence's
};

template <int DT, bool E5, int UNROLL>
__global__ __launch_bounds__(kThreads) void cache8_read_kernel(const Cache8Args a, int chunk_rows) {
  extern __shared__ int starts[];
  __shared__ ReadRow s_rows[kReadRows];
  constexpr int ES = DT == EA_F32 ? 4 : 2;
  const int tid = threadIdx.x;
  const int ppr = a.d / 8, sides = 2 * a.hkv, items = chunk_rows * sides * ppr;
  const int64_t head = (int64_t)a.page_size * a.d;
  // heads a pitch apart: of one block, or a block each
  const bool even = (a.xk.hb == 1 || a.xk.hb >= a.hkv) && (a.xv.hb == 1 || a.xv.hb >= a.hkv);
  load_starts(a, starts);
  for (int64_t first = blockIdx.x * (int64_t)chunk_rows; first < a.rows; first += gridDim.x * (int64_t)chunk_rows) {
    const int t0 = (int)first;
    if (tid < chunk_rows) {
      const Place p = place_of(a, starts, t0 + tid);
      ReadRow z;
      z.code = p.page < 0 ? -1 : p.page * a.page_bytes + (int64_t)p.in * a.d;
      z.scale = p.page < 0 ? 0 : (int64_t)p.page * a.hkv * a.n_blocks + div_fast(p.in, a.block);
      z.mine = p.mine;
      if (p.mine) {
        z.out[0] = row_offset(a.xk, t0 + tid, 0);
        z.out[1] = row_offset(a.xv, t0 + tid, 0);
        z.pitch[0] = a.hkv > 1 ? row_offset(a.xk, t0 + tid, 1) - z.out[0] : 0;
        z.pitch[1] = a.hkv > 1 ? row_offset(a.xv, t0 + tid, 1) - z.out[1] : 0;
      }
      s_rows[tid] = z;
    }
    __syncthreads();
    for (int i0 = tid; i0 < items; i0 += kThreads * UNROLL) {
      uint2 c[UNROLL];
      float f[UNROLL];
      char* to[UNROLL];
#pragma unroll
      for (int k = 0; k < UNROLL; ++k) {
        const int i = min(i0 + k * kThreads, items - 1);
        const int rx = div_fast(i, a.pieces), piece = i - rx * ppr, rr = div_fast(rx, a.sides), x = rx - rr * sides;
        const bool v = x >= a.hkv;
        const int h = v ? x - a.hkv : x;
        const ReadRow& z = s_rows[rr];
        const int64_t code = z.code;
        c[k] = make_uint2(0, 0);
        f[k] = 0.0f;
        if (code >= 0) {
          c[k] = *reinterpret_cast<const uint2*>((v ? a.pv : a.pk) + code + (h * head + piece * 8));
          f[k] = (v ? a.vs : a.ks)[z.scale + (int64_t)h * a.n_blocks];
        }
        const int64_t at = even ? z.out[v] + h * z.pitch[v] : row_offset(v ? a.xv : a.xk, min(t0 + rr, a.rows - 1), h);
        to[k] = z.mine && i0 + k * kThreads < items ? const_cast<char*>(v ? a.pxv : a.pxk) + at + piece * 8 * ES : nullptr;
      }
#pragma unroll
      for (int k = 0; k < UNROLL; ++k) {
        if (!to[k]) continue;
        float y[8];
        decode4<E5>(c[k].x, y);
        decode4<E5>(c[k].y, y + 4);
        // (the product with a power of two is exact; another's is rounded once, as
        // the output)
        if (DT != EA_F32 && __builtin_expect((__float_as_uint(f[k]) & 0x7fffffu) != 0, 0)) {
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = product_to_odd(y[j], f[k]);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] *= f[k];
        }
        if constexpr (DT == EA_F32) {
#pragma unroll
          for (int j = 0; j < 2; ++j)
            reinterpret_cast<float4*>(to[k])[j] = make_float4(y[4 * j], y[4 * j + 1], y[4 * j + 2], y[4 * j + 3]);
        } else {
          uint32_t w[4];
#pragma unroll
          for (int j = 0; j < 4; ++j)
            w[j] = DT == EA_BF16 ? pack_bf16x2(y[2 * j], y[2 * j + 1])
                                 : (uint32_t)f32_to_f16(y[2 * j]) | ((uint32_t)f32_to_f16(y[2 * j + 1]) << 16);
          store_stream(to[k], make_uint4(w[0], w[1], w[2], w[3]));
        }
      }
    }
    __syncthreads();  // the places are the next chunk's
  }
}

template <int DT, bool E5>
hipError_t run(const Cache8Args& a, bool write, hipStream_t s) {
  if (write) {
    // the blocks that the rows can lie in, a wave for each head of K and of V
    const int64_t blocks = a.rows / a.block_rows + 2 * (int64_t)a.n_seq;
    const int64_t units = (blocks < a.rows ? blocks : a.rows) * 2 * a.hkv, wgs = (units + kWaves - 1) / kWaves;
    // passes over a whole block; as many workgroups as the chip holds of them
    const bool few = a.block_rows <= 4 * (64 / (a.d / 8));
    const int64_t most = few && DT != EA_F32 ? 1536 : 1024;
    const dim3 grid(wgs < most ? wgs : most);
    const size_t lds = a.n_seq * sizeof(Span);
    if (few)
      cache8_write_kernel<DT, E5, 4><<<grid, dim3(kThreads), lds, s>>>(a);
    else
      cache8_write_kernel<DT, E5, DT == EA_F32 ? 8 : 16><<<grid, dim3(kThreads), lds, s>>>(a);
  } else {
    const size_t lds = a.q_start ? (a.n_seq + 1) * sizeof(int) : 0;
    // few rows a workgroup where there are few: one sequence of 1000 rows, 8 heads
    // of 128, 7.7 us with 1 and 9.2 with 16
    const int chunk_rows = a.rows >= kReadRows * 1024 ? kReadRows : a.rows / 1024 > 1 ? a.rows / 1024 : 1;
    const int chunks = (a.rows + chunk_rows - 1) / chunk_rows;
    const dim3 grid(chunks < 65536 ? chunks : 65536);
    if (chunk_rows * 2 * (int64_t)a.hkv * (a.d / 8) <= kThreads)
      cache8_read_kernel<DT, E5, 1><<<grid, dim3(kThreads), lds, s>>>(a, chunk_rows);
    else
      cache8_read_kernel<DT, E5, 8><<<grid, dim3(kThreads), lds, s>>>(a, chunk_rows);
  }
  return hipGetLastError();
}

template <int DT>
hipError_t run_code(const Cache8Args& a, int32_t code, bool write, hipStream_t s) {
  return code == EA_E5M2 ? run<DT, true>(a, write, s) : run<DT, false>(a, write, s);
}

}  // namespace

hipError_t launch_cache8(const Cache8Args& a, int32_t dtype, int32_t code, bool write, hipStream_t s) {
  if (dtype == EA_F32) return run_code<EA_F32>(a, code, write, s);
  return dtype == EA_BF16 ? run_code<EA_BF16>(a, code, write, s) : run_code<EA_F16>(a, code, write, s);
}

}  // namespace ea
