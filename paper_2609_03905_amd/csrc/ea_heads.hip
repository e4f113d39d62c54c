// ea_heads.hip -- the head rows of a QKV activation: per-head RMSNorm of
// queries and keys, the position rotation and the move to where attention
// reads them (per-head rows, or the pages of a cache), in one pass; and its
// gradient.
//
// A head row u of d elements at position p becomes
//   n = w u r,  r = 1 / sqrt(mean(u^2) + eps)
//   (n_i, n_j) -> (n_i cos a - n_j sin a, n_j cos a + n_i sin a),  a = p f_i
// over pairs (i, i + rot/2) or (2i, 2i+1) of its first rot elements.  The
// rotation is orthogonal, so its gradient is the rotation by -a: with g the
// rotated-back gradient, dw = sum g u r and, with s = w g,
//   du = r (s - u r mean(s u r)).
//
// Bound by memory: each element is read once and written once, about 10
// operations on it.  A head row is held by d/8 lanes (16 bytes each in bf16),
// so the mean is a few lane exchanges, and the other half of a rotated pair is
// read again by the lane that needs it, which the L1 answers.  A wave walks
// several groups of heads of one row, because the angles are the costly part:
// p f_i / 2 pi is taken to its fraction in 64 bits (positions of a million
// cost 32-bit products all of their angle) and sine and cosine follow in 32.
#include "ea_decode.h"
#include "ea_device.h"

namespace ea {

namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr int64_t kHeadsMaxWg = 1 << 20;  // of a launch; more rows go round again

// Eight elements of a row as they are stored.
template <int DT>
struct Raw {
  uint4 v[DT == EA_F32 ? 2 : 1];
};
template <int DT>
__device__ __forceinline__ Raw<DT> load_raw(const char* p) {
  Raw<DT> r;
  r.v[0] = *reinterpret_cast<const uint4*>(p);
  if constexpr (DT == EA_F32) r.v[1] = *reinterpret_cast<const uint4*>(p + 16);
  return r;
}
template <int DT>
__device__ __forceinline__ void store_raw(char* p, const Raw<DT>& r) {
  *reinterpret_cast<uint4*>(p) = r.v[0];
  if constexpr (DT == EA_F32) *reinterpret_cast<uint4*>(p + 16) = r.v[1];
}
template <int DT>
__device__ __forceinline__ void widen(const Raw<DT>& r, float (&f)[8]) {
  if constexpr (DT == EA_F32) {
    const float4 a = __builtin_bit_cast(float4, r.v[0]), b = __builtin_bit_cast(float4, r.v[1]);
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
  } else {
    const uint32_t w[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (DT == EA_BF16) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      } else {
        f[2 * i] = f16_to_f32((uint16_t)w[i]);
        f[2 * i + 1] = f16_to_f32((uint16_t)(w[i] >> 16));
      }
    }
  }
}
template <int DT>
__device__ __forceinline__ Raw<DT> narrow(const float (&f)[8]) {
  Raw<DT> r;
  if constexpr (DT == EA_F32) {
    r.v[0] = __builtin_bit_cast(uint4, make_float4(f[0], f[1], f[2], f[3]));
    r.v[1] = __builtin_bit_cast(uint4, make_float4(f[4], f[5], f[6], f[7]));
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = DT == EA_BF16 ? pack_bf16x2(f[2 * i], f[2 * i + 1])
                           : (uint32_t)f32_to_f16(f[2 * i]) | ((uint32_t)f32_to_f16(f[2 * i + 1]) << 16);
    r.v[0] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return r;
}

// Sum over the LPH lanes of a head row (LPH a power of two from 8 to 64).
template <int LPH>
__device__ __forceinline__ float row_sum(float v) {
  v += dpp_f<0xB1>(v);
  v += dpp_f<0x4E>(v);
  v += dpp_f<0x141>(v);
  if constexpr (LPH >= 16) v += dpp_f<0x140>(v);
  if constexpr (LPH >= 32) v += other16(v);
  if constexpr (LPH >= 64) v += other32(v);
  return v;
}

// How the partner of an element is reached: in the lane's own eight (pairs of
// neighbours), as another eight (halves, rot/2 a multiple of 8), or one by one.
enum { PAIR_NONE, PAIR_OWN, PAIR_CHUNK, PAIR_ELEM };
__device__ __forceinline__ int pair_mode(int rot, int inter) {
  return rot == 0 ? PAIR_NONE : inter ? PAIR_OWN : (rot / 2) % 8 == 0 ? PAIR_CHUNK : PAIR_ELEM;
}
// Index of element i's partner (i < rot, halves).
__device__ __forceinline__ int partner_of(int i, int half) { return i < half ? i + half : i - half; }

// cos and signed sin of the lane's eight elements at one position; elements
// past the rotated part get (1, 0).
__device__ __forceinline__ void angles(const float* freq, int pos, int c, int rot, int inter, bool active,
                                       float (&cs)[8], float (&sn)[8]) {
  const int half = rot / 2;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int i = 8 * c + e;
    cs[e] = 1.0f;
    sn[e] = 0.0f;
    if (active && i < rot) {
      const int f = inter ? i >> 1 : (i < half ? i : i - half);
      const bool first = inter ? !(i & 1) : i < half;
      const double turns = (double)pos * (double)freq[f] * 0.15915494309189535;  // 1 / (2 pi)
      const float part = (float)(turns - rint(turns));
      float s, co;
      sincospif(2.0f * part, &s, &co);
      cs[e] = co;
      sn[e] = first ? -s : s;
    }
  }
}

// The partner values of the lane's eight elements of the row at `row`, in
// their stored order (own: its own eight).
template <int DT>
__device__ __forceinline__ void partners(const char* row, int mode, int c, int rot, const float (&own)[8],
                                         float (&p)[8]) {
  const int half = rot / 2;
  if (mode == PAIR_CHUNK) {
    if (8 * c < rot) {
      widen<DT>(load_raw<DT>(row + (int64_t)partner_of(8 * c, half) * (DT == EA_F32 ? 4 : 2)), p);
      return;
    }
  } else if (mode == PAIR_ELEM) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = 8 * c + e;
      p[e] = i < rot ? ld_elem(row, partner_of(i, half), DT) : 0.0f;
    }
    return;
  } else if (mode == PAIR_OWN) {
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = 8 * c + e < rot ? own[e ^ 1] : 0.0f;
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) p[e] = 0.0f;
}

// Norm weights of the lane's eight elements and of their partners.
__device__ __forceinline__ void weights(const char* w, int dt, int mode, int c, int rot, bool active, float (&own)[8],
                                        float (&par)[8]) {
  const int half = rot / 2;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int i = 8 * c + e;
    own[e] = w && active ? ld_elem(w, i, dt) : 1.0f;
    const int j = mode == PAIR_OWN ? i ^ 1 : partner_of(i, half);
    par[e] = w && active && i < rot ? ld_elem(w, j, dt) : 1.0f;
  }
}

template <int LPH, int DT>
__global__ __launch_bounds__(kThreads) void heads_kernel(const HeadsArgs a) {
  constexpr int RPW = 64 / LPH;  // head rows that a wave holds at once
  const int lane = threadIdx.x & 63, sub = lane / LPH, c = lane % LPH;
  const int heads = a.hq + 2 * a.hkv, groups = (heads + RPW - 1) / RPW;
  const int parts = (groups + a.groups_per_wave - 1) / a.groups_per_wave;
  const int64_t items = (int64_t)a.t * parts;
  const bool active = 8 * c < a.d;
  const int mode = pair_mode(a.rot, a.inter);
  float wq[8], wqp[8], wk[8], wkp[8];
  weights(a.wq, a.wq_dt, mode, c, a.rot, active, wq, wqp);
  weights(a.wk, a.wk_dt, mode, c, a.rot, active, wk, wkp);
  for (int64_t it = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); it < items;
       it += (int64_t)gridDim.x * kWaves) {
  const int t = (int)(it / parts), part = (int)(it - (int64_t)t * parts);
  float cs[8], sn[8];
  angles(a.freq, a.pos ? a.pos[t] : t, c, a.rot, a.inter, active, cs, sn);
  // a row's place in the cache; none: its key and value rows go nowhere
  int slot = 0;
  int64_t page_off = 0;
  int in_page = 0;
  if (a.slots) {
    slot = a.slots[t];
    if (slot < 0 || slot >= a.n_slots) slot = -1;
    const int pg = div_fast(max(slot, 0), a.page);
    in_page = max(slot, 0) - pg * a.page_size;
    page_off = pg * a.page_bytes;
  }
  const int g1 = min(groups, (part + 1) * a.groups_per_wave);
  constexpr int ES = DT == EA_F32 ? 4 : 2;
  for (int gi = part * a.groups_per_wave; gi < g1; ++gi) {
    const int h = gi * RPW + sub;
    const bool on = active && h < heads;
    const bool is_q = h < a.hq, is_k = !is_q && h < a.hq + a.hkv, is_v = !is_q && !is_k;
    const char* row = a.px + row_offset(a.x, t, min(h, heads - 1));
    float u[8], p[8];
    if (on) {
      widen<DT>(load_raw<DT>(row + c * 8 * ES), u);
      partners<DT>(row, mode, c, a.rot, u, p);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) u[e] = p[e] = 0.0f;
    }
    const char* w = is_q ? a.wq : a.wk;
    float ss = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(u[e], u[e], ss);
    ss = row_sum<LPH>(ss);
    const float r = w && !is_v ? 1.0f / sqrtf(ss / (float)a.d + a.eps) : 1.0f;
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float n = u[e] * r * (is_q ? wq[e] : wk[e]);
      const float m = p[e] * r * (is_q ? wqp[e] : wkp[e]);
      y[e] = is_v ? u[e] : fmaf(n, cs[e], m * sn[e]);
    }
    if (!on) continue;
    char* dst;
    if (is_q) {
      dst = a.pq + row_offset(a.q, t, h);
    } else {
      const int hh = h - a.hq - (is_k ? 0 : a.hkv);
      dst = is_k ? a.pk : a.pv;
      if (a.slots) {
        if (slot < 0) continue;
        dst += page_off + ((int64_t)hh * a.page_size + in_page) * a.d * ES;
      } else {
        dst += row_offset(is_k ? a.k : a.v, t, hh);
      }
    }
    store_raw<DT>(dst + c * 8 * ES, narrow<DT>(y));
  }
  }
}

template <int LPH, int DT>
__global__ __launch_bounds__(kThreads) void heads_grad_kernel(const HeadsGradArgs a) {
  constexpr int RPW = 64 / LPH;
  constexpr int ES = DT == EA_F32 ? 4 : 2;
  __shared__ float s_dw[kWaves][2][LPH * 8];
  const int lane = threadIdx.x & 63, sub = lane / LPH, c = lane % LPH;
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int heads = a.hq + 2 * a.hkv, groups = (heads + RPW - 1) / RPW;
  const int parts = (groups + a.groups_per_wave - 1) / a.groups_per_wave;
  const bool active = 8 * c < a.d;
  const int mode = pair_mode(a.rot, a.inter);
  float wq[8], wk[8], unused[8], dwq[8] = {}, dwk[8] = {};
  weights(a.wq, a.wq_dt, mode, c, a.rot, active, wq, unused);
  weights(a.wk, a.wk_dt, mode, c, a.rot, active, wk, unused);
  const int64_t items = (int64_t)a.t * parts;
  for (int64_t it = (int64_t)blockIdx.x * kWaves + wid; it < items; it += (int64_t)gridDim.x * kWaves) {
    const int t = (int)(it / parts), part = (int)(it - (int64_t)t * parts);
    float cs[8], sn[8];
    angles(a.freq, a.pos ? a.pos[t] : t, c, a.rot, a.inter, active, cs, sn);
    const int g1 = min(groups, (part + 1) * a.groups_per_wave);
    for (int gi = part * a.groups_per_wave; gi < g1; ++gi) {
      const int h = gi * RPW + sub;
      const bool on = active && h < heads;
      const bool is_q = h < a.hq, is_k = !is_q && h < a.hq + a.hkv, is_v = !is_q && !is_k;
      const int hh = is_q ? h : h - a.hq - (is_k ? 0 : a.hkv);
      const int64_t xoff = row_offset(a.x, t, min(h, heads - 1));
      float u[8] = {}, dy[8] = {}, p[8] = {};
      const char* w = is_q ? a.wq : a.wk;
      if (on) {
        const char* row = is_q ? a.pdq + row_offset(a.q, t, hh)
                               : is_k ? a.pdk + row_offset(a.k, t, hh) : a.pdv + row_offset(a.v, t, hh);
        widen<DT>(load_raw<DT>(row + c * 8 * ES), dy);
        if (!is_v) {
          partners<DT>(row, mode, c, a.rot, dy, p);
          if (w) widen<DT>(load_raw<DT>(a.px + xoff + c * 8 * ES), u);
        }
      }
      float ss = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(u[e], u[e], ss);
      ss = row_sum<LPH>(ss);
      const bool normed = w && !is_v;
      const float r = normed ? 1.0f / sqrtf(ss / (float)a.d + a.eps) : 1.0f;
      float g[8], n[8], dot = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        g[e] = is_v ? dy[e] : fmaf(dy[e], cs[e], -p[e] * sn[e]);  // rotated by -a
        n[e] = u[e] * r;
        const float gn = g[e] * n[e];
        dwq[e] += is_q && on ? gn : 0.0f;
        dwk[e] += is_k && on ? gn : 0.0f;
        g[e] *= normed ? (is_q ? wq[e] : wk[e]) : 1.0f;
        dot = fmaf(g[e], n[e], dot);
      }
      const float mean = row_sum<LPH>(dot) / (float)a.d;
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] = normed ? r * fmaf(-n[e], mean, g[e]) : g[e];
      if (on) store_raw<DT>(a.pdx + xoff + c * 8 * ES, narrow<DT>(g));
    }
  }
  if (!a.part) return;
  // over the wave's head rows, then over the workgroup's waves, in a fixed order
#pragma unroll
  for (int e = 0; e < 8; ++e) {
#pragma unroll
    for (int o = LPH; o < 64; o *= 2) {
      dwq[e] += __shfl_xor(dwq[e], o);
      dwk[e] += __shfl_xor(dwk[e], o);
    }
    if (sub == 0) {
      s_dw[wid][0][8 * c + e] = dwq[e];
      s_dw[wid][1][8 * c + e] = dwk[e];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * a.d; i += kThreads) {
    const int kind = i >= a.d, col = i - kind * a.d;
    float v = s_dw[0][kind][col];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v += s_dw[w][kind][col];
    a.part[((int64_t)blockIdx.x * 2 + kind) * a.d + col] = v;
  }
}

// Sums of the workgroups' parts: 16 columns and 16 strips of workgroups each.
__global__ __launch_bounds__(kThreads) void heads_dw_kernel(const HeadsGradArgs a) {
  __shared__ float s[16][16];
  const int per = (a.d + 15) / 16;
  const int kind = blockIdx.x / per, col = (blockIdx.x % per) * 16 + (threadIdx.x & 15);
  const int strip = threadIdx.x >> 4;
  float v = 0.0f;
  if (col < a.d)
#pragma unroll 4
    for (int w = strip; w < a.n_wg; w += 16) v += a.part[((int64_t)w * 2 + kind) * a.d + col];
  s[strip][threadIdx.x & 15] = v;
  __syncthreads();
  char* out = kind ? a.dwk : a.dwq;
  if (strip == 0 && col < a.d && out) {
    for (int i = 1; i < 16; ++i) v += s[i][threadIdx.x];
    st_elem(out, col, kind ? a.dwk_dt : a.dwq_dt, v);
  }
}

template <int LPH>
hipError_t run_heads(const HeadsArgs& a, int32_t dt, int64_t grid, hipStream_t s) {
  const dim3 g((uint32_t)grid), b(kThreads);
  if (dt == EA_F32) heads_kernel<LPH, EA_F32><<<g, b, 0, s>>>(a);
  else if (dt == EA_BF16) heads_kernel<LPH, EA_BF16><<<g, b, 0, s>>>(a);
  else heads_kernel<LPH, EA_F16><<<g, b, 0, s>>>(a);
  return hipGetLastError();
}
template <int LPH>
hipError_t run_heads_grad(const HeadsGradArgs& a, int32_t dt, hipStream_t s) {
  const dim3 g((uint32_t)a.n_wg), b(kThreads);
  if (dt == EA_F32) heads_grad_kernel<LPH, EA_F32><<<g, b, 0, s>>>(a);
  else if (dt == EA_BF16) heads_grad_kernel<LPH, EA_BF16><<<g, b, 0, s>>>(a);
  else heads_grad_kernel<LPH, EA_F16><<<g, b, 0, s>>>(a);
  return hipGetLastError();
}

// Lanes of a head row: 8 elements each, a power of two from 8 up.
int lanes_of(int d) {
  int n = 8;
  while (n * 8 < d) n *= 2;
  return n;
}

}  // namespace

hipError_t launch_heads(const HeadsArgs& a0, int32_t dt, hipStream_t s) {
  HeadsArgs a = a0;
  const int lph = lanes_of(a.d), rpw = 64 / lph;
  const int groups = (a.hq + 2 * a.hkv + rpw - 1) / rpw;
  // As many groups a wave as leave eight waves a CU to hide the loads.
  int64_t gpw = (int64_t)a.t * groups / (8 * 256);
  a.groups_per_wave = (int32_t)(gpw < 1 ? 1 : gpw > groups ? groups : gpw);
  const int64_t parts = (groups + a.groups_per_wave - 1) / a.groups_per_wave;
  const int64_t wgs = ((int64_t)a.t * parts + kWaves - 1) / kWaves;
  const int64_t grid = wgs < kHeadsMaxWg ? wgs : kHeadsMaxWg;
  switch (lph) {
    case 8: return run_heads<8>(a, dt, grid, s);
    case 16: return run_heads<16>(a, dt, grid, s);
    case 32: return run_heads<32>(a, dt, grid, s);
    default: return run_heads<64>(a, dt, grid, s);
  }
}

hipError_t launch_heads_grad(const HeadsGradArgs& a0, int32_t dt, hipStream_t s) {
  HeadsGradArgs a = a0;
  const int lph = lanes_of(a.d), rpw = 64 / lph;
  const int groups = (a.hq + 2 * a.hkv + rpw - 1) / rpw;
  int64_t gpw = (int64_t)a.t * groups / (8 * 256);
  a.groups_per_wave = (int32_t)(gpw < 1 ? 1 : gpw > groups ? groups : gpw);
  const int64_t parts = (groups + a.groups_per_wave - 1) / a.groups_per_wave;
  const int64_t wgs = ((int64_t)a.t * parts + kWaves - 1) / kWaves;
  a.n_wg = (int32_t)(wgs < kHeadsGradMaxWg ? wgs : kHeadsGradMaxWg);
  hipError_t e;
  switch (lph) {
    case 8: e = run_heads_grad<8>(a, dt, s); break;
    case 16: e = run_heads_grad<16>(a, dt, s); break;
    case 32: e = run_heads_grad<32>(a, dt, s); break;
    default: e = run_heads_grad<64>(a, dt, s); break;
  }
  if (e != hipSuccess || !a.part) return e;
  heads_dw_kernel<<<dim3(2 * ((a.d + 15) / 16)), dim3(kThreads), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace ea
