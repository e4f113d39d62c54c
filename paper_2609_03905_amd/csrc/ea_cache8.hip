// ea_cache8.hip -- a paged cache in 8 bits: rows quantised as they are written,
// and read back.
//
// A cache's codes c stand for c s, s the scale of the code's head and block of B
// neighbouring rows of a page.  For the rows x that a write puts into a block, K
// and V and every head apart,
//   a = max |x| over the finite ones,   e = the least whole number with a <= M 2^e
// (M the largest code, 448 or 57344; e in [-120, 120]), and the block's scale is
// 2^e, or the one it has if that is larger and the block holds rows of earlier
// calls; where the scale grows, their codes become round(c s_old / s).  Then
// c = round(x / s).  Scales being powers of two, both quotients are exact in 32
// bits, so that a code is off by its own rounding alone, and one that is rounded
// again changes only where it falls below the code's normal range.
//
// Rows of a block are neighbours both in the call and in the page, so a block's
// head is one wave's: the rows stay in registers between the maximum and the
// codes.  The wave that the block's first new row falls to takes it.
#include "ea_decode.h"
#include "ea_device.h"

namespace ea {

namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr int kChunk = 64;  // rows whose places a workgroup of the write looks up
constexpr int kHold = 8;    // passes over rows that a wave keeps in registers

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

// x f rounded to codes, to nearest, ties to even; what is not finite has the
// code that stands for it (e4m3 has none for an infinity: NaN).
template <bool E5>
__device__ __forceinline__ uint2 encode(const float (&x)[8], float f) {
  int w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (E5) {
      w[i] = __builtin_amdgcn_cvt_pk_bf8_f32(x[4 * i] * f, x[4 * i + 1] * f, 0, false);
      w[i] = __builtin_amdgcn_cvt_pk_bf8_f32(x[4 * i + 2] * f, x[4 * i + 3] * f, w[i], true);
    } else {
      w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * f, x[4 * i + 1] * f, 0, false);
      w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * f, x[4 * i + 3] * f, w[i], true);
    }
  }
  return make_uint2(w[0], w[1]);
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
// rounding it to a code (of far fewer bits) is one rounding of the product.
__device__ __forceinline__ float product_to_odd(float c, float f) {
  const float p = c * f, rest = fmaf(c, f, -p);
  const int bits = __float_as_int(p);
  if (rest == 0.0f || !(fabsf(p) < INFINITY) || (bits & 1)) return p;
  return __int_as_float(bits + ((rest > 0.0f) == (p > 0.0f) ? 1 : -1));
}

__device__ __forceinline__ int first_row(const Cache8Args& a, int s) { return min(max(a.q_start[s], 0), a.rows); }

// Where row t of the call lies in the cache.
struct Place {
  int page, in, at;  // page (-1: the row has none), row of the page, position
  int first, end;    // positions of the sequence's first new row and behind its last
  bool mine;         // the row is a sequence's
};

// q_start's first rows in shared memory: all threads of the workgroup take part.
__device__ __forceinline__ void load_starts(const Cache8Args& a, int* starts) {
  if (a.q_start)
    for (int i = threadIdx.x; i <= a.n_seq; i += kThreads) starts[i] = first_row(a, i);
  __syncthreads();
}

__device__ __forceinline__ Place place_of(const Cache8Args& a, const int* starts, int t) {
  Place p = {-1, 0, 0, 0, 0, false};
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
  p.end = min(max(a.len[s], 0), a.stride * a.page_size);
  p.first = max(p.end - (r1 - r0), 0);
  p.at = p.end - r1 + t;
  if (p.at < 0) return p;
  const int i = div_fast(p.at, a.page);
  p.in = p.at - i * a.page_size;
  const int pg = a.table[(int64_t)s * a.stride + i];
  p.page = (uint32_t)pg < (uint32_t)a.n_pages ? pg : -1;
  return p;
}

template <int DT, bool E5>
__global__ __launch_bounds__(kThreads) void cache8_write_kernel(const Cache8Args a) {
  extern __shared__ int starts[];
  __shared__ int s_row[kChunk], s_page[kChunk], s_in[kChunk], s_count[kChunk], s_n;
  const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  load_starts(a, starts);
  const int chunks = (a.rows + kChunk - 1) / kChunk;
  for (int chunk = blockIdx.x; chunk < chunks; chunk += gridDim.x) {
  if (wid == 0) {
    const int t = chunk * kChunk + lane;
    const Place p = place_of(a, starts, t);
    const int b = p.in - div_fast(p.in, a.block) * a.block_rows;  // row of the block
    const bool lead = p.page >= 0 && (b == 0 || p.at == p.first);
    const uint64_t leads = __ballot(lead);
    if (lead) {
      const int i = __popcll(leads & ((uint64_t(1) << lane) - 1));
      s_row[i] = t;
      s_page[i] = p.page;
      s_in[i] = p.in;
      s_count[i] = min(a.block_rows - b, p.end - p.at);
    }
    if (lane == 0) s_n = __popcll(leads);
  }
  __syncthreads();

  const int lpr = a.d / 8, rows_pass = 64 / lpr;  // lanes of a row, rows of a pass
  const int r = lane / lpr, el = lane - r * lpr;
  const int sides = 2 * a.hkv, units = s_n * sides;
  constexpr int ES = DT == EA_F32 ? 4 : 2;
  for (int u = blockIdx.y * kWaves + wid; u < units; u += gridDim.y * kWaves) {
    const int i = u / sides, x = u - i * sides;
    const bool v = x >= a.hkv;
    const int h = v ? x - a.hkv : x;
    const int t0 = s_row[i], in = s_in[i], n = s_count[i];
    const int blk = div_fast(in, a.block), before = in - blk * a.block_rows;
    const RowMap& map = v ? a.xv : a.xk;
    const char* src = v ? a.pxv : a.pxk;
    float* scale = (v ? a.vs : a.ks) + ((int64_t)s_page[i] * a.hkv + h) * a.n_blocks + blk;
    char* dst = (v ? a.pv : a.pk) + s_page[i] * a.page_bytes + ((int64_t)h * a.page_size + blk * a.block_rows) * a.d + el * 8;
    const int passes = (n + rows_pass - 1) / rows_pass;
    auto row = [&](int p) { return p * rows_pass + r; };
    auto there = [&](int p) { return r < rows_pass && row(p) < n; };
    auto load = [&](int p, Eight<DT>& e) { e.load(src + row_offset(map, t0 + row(p), h) + el * 8 * ES); };

    const float old = before ? *scale : 0.0f;
    Eight<DT> held[kHold];
    float top = 0.0f;
    auto look = [&](const Eight<DT>& e) {
      float y[8];
      e.values(y);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float z = fabsf(y[j]);
        top = fmaxf(top, z < INFINITY ? z : 0.0f);
      }
    };
#pragma unroll
    for (int p = 0; p < kHold; ++p)
      if (there(p)) load(p, held[p]);
#pragma unroll
    for (int p = 0; p < kHold; ++p)
      if (there(p)) look(held[p]);
    for (int p = kHold; p < passes; ++p)
      if (there(p)) {
        Eight<DT> e;
        load(p, e);
        look(e);
      }
    int e = least_exponent<E5>(wave_max(top));
    if (old > 0.0f && old < INFINITY) {
      // (a scale that another program left may be no power of two: the next one)
      const int bits = __float_as_int(old);
      e = max(e, min(max((bits >> 23) - 127 + ((bits & 0x7fffff) != 0), -kScaleExp), 126));
      const float ratio = old * power(-e);
      if (ratio != 1.0f)
        for (int b = r; b < before && r < rows_pass; b += rows_pass) {
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
    const float inv = power(-e);
    auto store = [&](int p, const Eight<DT>& z) {
      float y[8];
      z.values(y);
      *reinterpret_cast<uint2*>(dst + (int64_t)(before + row(p)) * a.d) = encode<E5>(y, inv);
    };
#pragma unroll
    for (int p = 0; p < kHold; ++p)
      if (there(p)) store(p, held[p]);
    for (int p = kHold; p < passes; ++p)
      if (there(p)) {
        Eight<DT> z;
        load(p, z);
        store(p, z);
      }
    if (lane == 0) *scale = power(e);
  }
  __syncthreads();  // the lists are the next chunk's
  }
}

// ---- reading back -----------------------------------------------------------------
// Pieces of 16 codes, a thread each and four in flight: bound by HBM.
constexpr int kReadRows = 16, kReadUnroll = 4;

template <int DT, bool E5>
__global__ __launch_bounds__(kThreads) void cache8_read_kernel(const Cache8Args a) {
  extern __shared__ int starts[];
  __shared__ int64_t s_off[kReadRows], s_scale[kReadRows];
  __shared__ int s_mine[kReadRows];
  const int tid = threadIdx.x, chunks = (a.rows + kReadRows - 1) / kReadRows;
  load_starts(a, starts);
  for (int chunk = blockIdx.x; chunk < chunks; chunk += gridDim.x) {
  const int t0 = chunk * kReadRows;
  if (tid < kReadRows) {
    const Place p = place_of(a, starts, t0 + tid);
    const int b = div_fast(p.in, a.block);
    s_off[tid] = p.page < 0 ? -1 : p.page * a.page_bytes + (int64_t)p.in * a.d;
    s_scale[tid] = p.page < 0 ? 0 : (int64_t)p.page * a.hkv * a.n_blocks + b;
    s_mine[tid] = p.mine;
  }
  __syncthreads();
  constexpr int ES = DT == EA_F32 ? 4 : 2;
  const int ppr = a.d / 16, row_items = 2 * a.hkv * ppr, items = kReadRows * row_items;
  for (int i0 = tid; i0 < items; i0 += kThreads * kReadUnroll) {
    uint4 c[kReadUnroll];
    float f[kReadUnroll];
    char* to[kReadUnroll];
#pragma unroll
    for (int k = 0; k < kReadUnroll; ++k) {
      const int i = i0 + k * kThreads;
      to[k] = nullptr;
      if (i >= items) continue;
      const int side = i / (items / 2), j = i - side * (items / 2);
      const int rh = j / ppr, piece = j - rh * ppr, rr = rh / a.hkv, h = rh - rr * a.hkv;
      if (!s_mine[rr]) continue;
      const int64_t off = s_off[rr];
      c[k] = make_uint4(0, 0, 0, 0);
      f[k] = 0.0f;
      if (off >= 0) {
        c[k] = *reinterpret_cast<const uint4*>((side ? a.pv : a.pk) + off + ((int64_t)h * a.page_size * a.d + piece * 16));
        f[k] = (side ? a.vs : a.ks)[s_scale[rr] + (int64_t)h * a.n_blocks];
      }
      to[k] = const_cast<char*>(side ? a.pxv : a.pxk) + row_offset(side ? a.xv : a.xk, t0 + rr, h) + piece * 16 * ES;
    }
#pragma unroll
    for (int k = 0; k < kReadUnroll; ++k) {
      if (!to[k]) continue;
      float y[16];
      decode4<E5>(c[k].x, y);
      decode4<E5>(c[k].y, y + 4);
      decode4<E5>(c[k].z, y + 8);
      decode4<E5>(c[k].w, y + 12);
#pragma unroll
      for (int j = 0; j < 16; ++j) y[j] *= f[k];
      uint4* out = reinterpret_cast<uint4*>(to[k]);
      if constexpr (DT == EA_F32) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          out[j] = make_uint4(__float_as_uint(y[4 * j]), __float_as_uint(y[4 * j + 1]), __float_as_uint(y[4 * j + 2]),
                              __float_as_uint(y[4 * j + 3]));
      } else {
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
          w[j] = DT == EA_BF16 ? pack_bf16x2(y[2 * j], y[2 * j + 1])
                               : (uint32_t)f32_to_f16(y[2 * j]) | ((uint32_t)f32_to_f16(y[2 * j + 1]) << 16);
        out[0] = make_uint4(w[0], w[1], w[2], w[3]);
        out[1] = make_uint4(w[4], w[5], w[6], w[7]);
      }
    }
  }
  __syncthreads();  // the places are the next chunk's
  }
}

template <int DT, bool E5>
hipError_t run(const Cache8Args& a, bool write, hipStream_t s) {
  const size_t lds = a.q_start ? (a.n_seq + 1) * sizeof(int) : 0;
  if (write) {
    const int chunks = (a.rows + kChunk - 1) / kChunk;
    // blocks that a chunk's rows begin or go on with, on the average
    const int64_t begun = (int64_t)a.rows / a.block_rows + 2 * (int64_t)a.n_seq;
    const int64_t leads = (begun + chunks - 1) / chunks;
    const int64_t units = (leads < kChunk ? leads : kChunk) * 2 * a.hkv;
    const int64_t y = (units + kWaves - 1) / kWaves;
    cache8_write_kernel<DT, E5><<<dim3(chunks < 65536 ? chunks : 65536, y < 1024 ? y : 1024), dim3(kThreads), lds, s>>>(a);
  } else {
    const int chunks = (a.rows + kReadRows - 1) / kReadRows;
    cache8_read_kernel<DT, E5><<<dim3(chunks < 65536 ? chunks : 65536), dim3(kThreads), lds, s>>>(a);
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
