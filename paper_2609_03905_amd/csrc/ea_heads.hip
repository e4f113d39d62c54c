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
// operations on it.  A lane holds 16 elements of a row (two loads of 16 bytes
// in bf16), the two halves of 8 rotated pairs, so no element is read twice and
// the mean takes few lane exchanges.  A wave holds 64 / LPH rows at once, heads
// of one token, and walks the token's heads with the next rows' loads in
// flight.  The angles are the costly part: p f_i / 2 pi is taken to its
// fraction in 64 bits (at a position of a million a 32-bit product has lost the
// angle), sine and cosine follow in 32; the wave's lanes share that work, each
// pair once a token, and hand the results round through shared memory, where
// the norm weights are kept too.
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

// Sum over the LPH lanes of a head row (LPH a power of two from 4 to 32).
template <int LPH>
__device__ __forceinline__ float row_sum(float v) {
  v += dpp_f<0xB1>(v);
  v += dpp_f<0x4E>(v);
  if constexpr (LPH >= 8) v += dpp_f<0x141>(v);
  if constexpr (LPH >= 16) v += dpp_f<0x140>(v);
  if constexpr (LPH >= 32) v += other16(v);
  return v;
}

// Which 16 elements of a row lane l holds, as two eights, and how they pair:
//   HALVES  eights (l, l + rot/16) of the rotated part, element e of one with
//           element e of the other; then the rest of the row, eight by eight
//   NEIGHBOURS  eights (2l, 2l + 1), pairs of neighbours
//   APART   as NEIGHBOURS, but halves that no eight divides (rot/2 no multiple
//           of 8): partners are read one by one
enum { HALVES, NEIGHBOURS, APART };
template <int MODE>
__device__ __forceinline__ int eight_of(int l, int which, int rot) {
  if (MODE == HALVES) return l < rot / 16 ? l + which * (rot / 16) : 2 * l + which;
  return 2 * l + which;
}

// Shared memory of a workgroup: the norm weights as f32 (1 where there are
// none) and every wave's cos and sin of its token's angles.
template <int LPH>
struct HeadsShared {
  __attribute__((aligned(16))) float w[2][LPH * 16];
  __attribute__((aligned(16))) float2 turn[kWaves][LPH * 8];
};

template <int LPH, class A>
__device__ __forceinline__ void stage_weights(const A& a, HeadsShared<LPH>& s) {
  for (int i = threadIdx.x; i < 2 * LPH * 16; i += kThreads) {
    const int kind = i >= LPH * 16, col = i - kind * LPH * 16;
    const char* w = kind ? a.wk : a.wq;
    s.w[kind][col] = w && col < a.d ? ld_elem(w, col, kind ? a.wk_dt : a.wq_dt) : 1.0f;
  }
  __syncthreads();
}

// cos and sin of the token's rot/2 angles, one lane a pair.
__device__ __forceinline__ void turn_table(const float* freq, int pos, int pairs, int lane, float2* out) {
  for (int i = lane; i < pairs; i += 64) {
    const double turns = (double)pos * (double)freq[i] * 0.15915494309189535;  // 1 / (2 pi)
    const float part = (float)(turns - rint(turns));
    float s, c;
    sincospif(2.0f * part, &s, &c);
    out[i] = make_float2(c, s);
  }
  __builtin_amdgcn_wave_barrier();
}

// The lane's eight (cos, sin) of its pairs; (1, 0) past the rotated part.
template <int MODE>
__device__ __forceinline__ void my_turns(const float2* t, int l, int pairs, float (&cs)[8], float (&sn)[8]) {
  if (MODE == APART) return;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    float4 v = make_float4(1.0f, 0.0f, 1.0f, 0.0f);
    if (8 * l + e + 1 < pairs) v = *reinterpret_cast<const float4*>(t + 8 * l + e);
    else if (8 * l + e < pairs) v.x = t[8 * l + e].x, v.y = t[8 * l + e].y;
    cs[e] = v.x, sn[e] = v.y, cs[e + 1] = v.z, sn[e + 1] = v.w;
  }
}

// The lane's first n pairs rotated by its angles (sign -1: back); the others
// stay, whatever their neighbours hold.  a, b: its two eights.
template <int MODE>
__device__ __forceinline__ void turn(float (&a)[8], float (&b)[8], const float (&cs)[8], const float (&sn)[8],
                                     float sign, int n) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float c = cs[e], s = sign * sn[e];
    float& x = MODE == HALVES ? a[e] : (e < 4 ? a : b)[2 * (e & 3)];
    float& y = MODE == HALVES ? b[e] : (e < 4 ? a : b)[2 * (e & 3) + 1];
    const float p = fmaf(x, c, -y * s), q = fmaf(y, c, x * s);
    x = e < n ? p : x;
    y = e < n ? q : y;
  }
}

// APART: the eight v (elements 8 q ..) rotated with partners read one by one
// from the stored row, scaled by r and the weights w (null: none).
template <int DT>
__device__ __forceinline__ void turn_apart(float (&v)[8], const char* row, int q, int rot, const float2* t, float r,
                                           const float* w, float sign) {
  const int half = rot / 2;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int i = 8 * q + e;
    if (i < rot) {
      const bool first = i < half;
      const int j = first ? i + half : i - half;
      const float2 cs = t[first ? i : j];
      const float other = ld_elem(row, j, DT) * r * (w ? w[j] : 1.0f), s = sign * cs.y;
      v[e] = fmaf(v[e], cs.x, first ? -other * s : other * s);
    }
  }
}

// A lane's two eights as stored; zeros where the row has none.
template <int DT>
struct Pair {
  Raw<DT> a, b;
};
template <int DT>
__device__ __forceinline__ Pair<DT> load_pair(const char* row, bool ona, bool onb, int qa, int qb) {
  constexpr int ES = DT == EA_F32 ? 4 : 2;
  Pair<DT> p{};
  if (ona) p.a = load_raw<DT>(row + qa * 8 * ES);
  if (onb) p.b = load_raw<DT>(row + qb * 8 * ES);
  return p;
}

template <int LPH, int DT, int MODE>
__global__ __launch_bounds__(kThreads) void heads_kernel(const HeadsArgs a) {
  constexpr int RPW = 64 / LPH;  // head rows that a wave holds at once
  constexpr int ES = DT == EA_F32 ? 4 : 2;
  __shared__ HeadsShared<LPH> sh;
  const int lane = threadIdx.x & 63, sub = lane / LPH, l = lane % LPH;
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int heads = a.hq + 2 * a.hkv, groups = (heads + RPW - 1) / RPW, pairs = a.rot / 2;
  const int parts = (groups + a.groups_per_wave - 1) / a.groups_per_wave;
  const int64_t items = (int64_t)a.t * parts;
  const int qa = eight_of<MODE>(l, 0, a.rot), qb = eight_of<MODE>(l, 1, a.rot);
  const bool in_a = 8 * qa < a.d, in_b = 8 * qb < a.d;
  auto row_of = [&](int t, int gi) { return a.px + row_offset(a.x, t, min(gi * RPW + sub, heads - 1)); };
  auto load = [&](int t, int gi) {
    const bool on = gi * RPW + sub < heads;
    return load_pair<DT>(row_of(t, gi), on && in_a, on && in_b, qa, qb);
  };
  int64_t it = (int64_t)blockIdx.x * kWaves + wid;
  // the first rows are on their way while the weights are staged
  Pair<DT> next{};
  int t = 0, part = 0, pos = 0;
  auto begin = [&]() {
    if (it >= items) return;
    t = (int)(it / parts);
    part = (int)(it - (int64_t)t * parts);
    next = load(t, part * a.groups_per_wave);
    pos = a.pos ? a.pos[t] : t;
  };
  begin();
  stage_weights<LPH>(a, sh);
  while (it < items) {
    const int g0 = part * a.groups_per_wave, g1 = min(groups, g0 + a.groups_per_wave);
    // the row's place in the cache; none: its keys and values go nowhere
    int slot = 0, in_page = 0;
    int64_t page_off = 0;
    if (a.slots) {
      slot = a.slots[t];
      if (slot < 0 || slot >= a.n_slots) slot = -1;
      const int pg = div_fast(max(slot, 0), a.page);
      in_page = max(slot, 0) - pg * a.page_size;
      page_off = pg * a.page_bytes;
    }
    float cs[8], sn[8];
    turn_table(a.freq, pos, pairs, lane, sh.turn[wid]);
    my_turns<MODE>(sh.turn[wid], l, pairs, cs, sn);
    for (int gi = g0; gi < g1; ++gi) {
      const Pair<DT> cur = next;
      if (gi + 1 < g1) next = load(t, gi + 1);
      const int h = gi * RPW + sub;
      const bool is_q = h < a.hq, is_v = h >= a.hq + a.hkv;
      Pair<DT> out = cur;
      if (__any(!is_v)) {
        float u[8], v[8];
        widen<DT>(cur.a, u);
        widen<DT>(cur.b, v);
        float r = 1.0f;
        const float* w = sh.w[is_q ? 0 : 1];
        if (a.wq) {
          float ss = 0.0f;
#pragma unroll
          for (int e = 0; e < 8; ++e) ss = fmaf(v[e], v[e], fmaf(u[e], u[e], ss));
          r = 1.0f / sqrtf(row_sum<LPH>(ss) / (float)a.d + a.eps);
#pragma unroll
          for (int e = 0; e < 8; e += 4) {
            const float4 x = *reinterpret_cast<const float4*>(w + 8 * min(qa, LPH * 2 - 1) + e);
            const float4 y = *reinterpret_cast<const float4*>(w + 8 * min(qb, LPH * 2 - 1) + e);
            u[e] *= r * x.x, u[e + 1] *= r * x.y, u[e + 2] *= r * x.z, u[e + 3] *= r * x.w;
            v[e] *= r * y.x, v[e + 1] *= r * y.y, v[e + 2] *= r * y.z, v[e + 3] *= r * y.w;
          }
        }
        if (MODE == APART) {
          if (h < heads && !is_v) {
            turn_apart<DT>(u, row_of(t, gi), qa, a.rot, sh.turn[wid], r, w, 1.0f);
            turn_apart<DT>(v, row_of(t, gi), qb, a.rot, sh.turn[wid], r, w, 1.0f);
          }
        } else {
          turn<MODE>(u, v, cs, sn, 1.0f, pairs - 8 * l);
        }
        if (!is_v) {
          out.a = narrow<DT>(u);
          out.b = narrow<DT>(v);
        }
      }
      if (h >= heads) continue;
      char* dst;
      if (is_q) {
        dst = a.pq + row_offset(a.q, t, h);
      } else {
        const int hh = h - a.hq - (is_v ? a.hkv : 0);
        dst = is_v ? a.pv : a.pk;
        if (a.slots) {
          if (slot < 0) continue;
          dst += page_off + ((int64_t)hh * a.page_size + in_page) * a.d * ES;
        } else {
          dst += row_offset(is_v ? a.v : a.k, t, hh);
        }
      }
      if (in_a) store_raw<DT>(dst + qa * 8 * ES, out.a);
      if (in_b) store_raw<DT>(dst + qb * 8 * ES, out.b);
    }
    __builtin_amdgcn_wave_barrier();  // the table is the next token's from here
    it += (int64_t)gridDim.x * kWaves;
    begin();
  }
}

template <int LPH, int DT, int MODE>
__global__ __launch_bounds__(kThreads, DT == EA_F32 ? 2 : 3) void heads_grad_kernel(const HeadsGradArgs a) {
  constexpr int RPW = 64 / LPH;
  constexpr int ES = DT == EA_F32 ? 4 : 2;
  __shared__ HeadsShared<LPH> sh;
  __shared__ float s_dw[kWaves][2][LPH * 16];
  const int lane = threadIdx.x & 63, sub = lane / LPH, l = lane % LPH;
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int heads = a.hq + 2 * a.hkv, groups = (heads + RPW - 1) / RPW, pairs = a.rot / 2;
  const int parts = (groups + a.groups_per_wave - 1) / a.groups_per_wave;
  const int64_t items = (int64_t)a.t * parts;
  const int qa = eight_of<MODE>(l, 0, a.rot), qb = eight_of<MODE>(l, 1, a.rot);
  const bool in_a = 8 * qa < a.d, in_b = 8 * qb < a.d;
  float dwq[16] = {}, dwk[16] = {};
  auto dy_of = [&](int t, int gi) {
    const int h = min(gi * RPW + sub, heads - 1);
    return h < a.hq             ? a.pdq + row_offset(a.q, t, h)
           : h < a.hq + a.hkv ? a.pdk + row_offset(a.k, t, h - a.hq)
                              : a.pdv + row_offset(a.v, t, h - a.hq - a.hkv);
  };
  auto load_dy = [&](int t, int gi) {
    const bool on = gi * RPW + sub < heads;
    return load_pair<DT>(dy_of(t, gi), on && in_a, on && in_b, qa, qb);
  };
  auto load_x = [&](int t, int gi) {
    const int h = gi * RPW + sub;
    const bool on = h < a.hq + a.hkv && a.wq;  // the values' rows are not needed
    return load_pair<DT>(a.px + row_offset(a.x, t, min(h, heads - 1)), on && in_a, on && in_b, qa, qb);
  };
  int64_t it = (int64_t)blockIdx.x * kWaves + wid;
  Pair<DT> dy_next{}, x_next{};
  int t = 0, part = 0, pos = 0;
  auto begin = [&]() {
    if (it >= items) return;
    t = (int)(it / parts);
    part = (int)(it - (int64_t)t * parts);
    dy_next = load_dy(t, part * a.groups_per_wave);
    x_next = load_x(t, part * a.groups_per_wave);
    pos = a.pos ? a.pos[t] : t;
  };
  begin();
  stage_weights<LPH>(a, sh);
  while (it < items) {
    const int g0 = part * a.groups_per_wave, g1 = min(groups, g0 + a.groups_per_wave);
    float cs[8], sn[8];
    turn_table(a.freq, pos, pairs, lane, sh.turn[wid]);
    my_turns<MODE>(sh.turn[wid], l, pairs, cs, sn);
    for (int gi = g0; gi < g1; ++gi) {
      const Pair<DT> dy = dy_next, x = x_next;
      if (gi + 1 < g1) {
        dy_next = load_dy(t, gi + 1);
        x_next = load_x(t, gi + 1);
      }
      const int h = gi * RPW + sub;
      const bool is_q = h < a.hq, is_v = h >= a.hq + a.hkv;
      Pair<DT> out = dy;
      if (__any(!is_v)) {
        float g[8], k[8];
        widen<DT>(dy.a, g);
        widen<DT>(dy.b, k);
        if (MODE == APART) {
          if (!is_v) {
            turn_apart<DT>(g, dy_of(t, gi), qa, a.rot, sh.turn[wid], 1.0f, nullptr, -1.0f);
            turn_apart<DT>(k, dy_of(t, gi), qb, a.rot, sh.turn[wid], 1.0f, nullptr, -1.0f);
          }
        } else {
          turn<MODE>(g, k, cs, sn, -1.0f, pairs - 8 * l);
        }
        if (a.wq) {
          float u[8], v[8];
          widen<DT>(x.a, u);
          widen<DT>(x.b, v);
          float ss = 0.0f;
#pragma unroll
          for (int e = 0; e < 8; ++e) ss = fmaf(v[e], v[e], fmaf(u[e], u[e], ss));
          const float r = 1.0f / sqrtf(row_sum<LPH>(ss) / (float)a.d + a.eps);
          const float* w = sh.w[is_q ? 0 : 1];
          const bool is_k = !is_q && !is_v;
          float dot = 0.0f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            u[e] *= r;
            v[e] *= r;
            const float gu = g[e] * u[e], kv = k[e] * v[e];
            dwq[e] = is_q ? dwq[e] + gu : dwq[e];
            dwq[8 + e] = is_q ? dwq[8 + e] + kv : dwq[8 + e];
            dwk[e] = is_k ? dwk[e] + gu : dwk[e];
            dwk[8 + e] = is_k ? dwk[8 + e] + kv : dwk[8 + e];
          }
#pragma unroll
          for (int e = 0; e < 8; e += 4) {
            const float4 p = *reinterpret_cast<const float4*>(w + 8 * min(qa, LPH * 2 - 1) + e);
            const float4 q = *reinterpret_cast<const float4*>(w + 8 * min(qb, LPH * 2 - 1) + e);
            g[e] *= p.x, g[e + 1] *= p.y, g[e + 2] *= p.z, g[e + 3] *= p.w;
            k[e] *= q.x, k[e + 1] *= q.y, k[e + 2] *= q.z, k[e + 3] *= q.w;
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) dot = fmaf(k[e], v[e], fmaf(g[e], u[e], dot));
          const float mean = row_sum<LPH>(dot) / (float)a.d;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            g[e] = r * fmaf(-u[e], mean, g[e]);
            k[e] = r * fmaf(-v[e], mean, k[e]);
          }
        }
        if (!is_v) {
          out.a = narrow<DT>(g);
          out.b = narrow<DT>(k);
        }
      }
      if (h >= heads) continue;
      char* dst = a.pdx + row_offset(a.x, t, h);
      if (in_a) store_raw<DT>(dst + qa * 8 * ES, out.a);
      if (in_b) store_raw<DT>(dst + qb * 8 * ES, out.b);
    }
    __builtin_amdgcn_wave_barrier();
    it += (int64_t)gridDim.x * kWaves;
    begin();
  }
  if (!a.part) return;
  // over the wave's head rows, then over the workgroup's waves, in a fixed order
#pragma unroll
  for (int e = 0; e < 16; ++e) {
#pragma unroll
    for (int o = LPH; o < 64; o *= 2) {
      dwq[e] += __shfl_xor(dwq[e], o);
      dwk[e] += __shfl_xor(dwk[e], o);
    }
    const int q = e < 8 ? qa : qb;
    if (sub == 0 && 8 * q < a.d) {
      s_dw[wid][0][8 * q + (e & 7)] = dwq[e];
      s_dw[wid][1][8 * q + (e & 7)] = dwk[e];
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

// Sums of the workgroups' parts: 8 columns and 32 strips of workgroups each.
__global__ __launch_bounds__(kThreads) void heads_dw_kernel(const HeadsGradArgs a) {
  __shared__ float s[32][8];
  const int per = a.d / 8;
  const int kind = blockIdx.x / per, col = (blockIdx.x % per) * 8 + (threadIdx.x & 7);
  const int strip = threadIdx.x >> 3;
  float v = 0.0f;
  for (int w0 = strip; w0 < a.n_wg; w0 += 32 * 8) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = w0 + 32 * i < a.n_wg ? a.part[((int64_t)(w0 + 32 * i) * 2 + kind) * a.d + col] : 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v += x[i];
  }
  s[strip][threadIdx.x & 7] = v;
  __syncthreads();
  char* out = kind ? a.dwk : a.dwq;
  if (strip == 0 && out) {
    for (int i = 1; i < 32; ++i) v += s[i][threadIdx.x];
    st_elem(out, col, kind ? a.dwk_dt : a.dwq_dt, v);
  }
}

template <int LPH, int MODE>
hipError_t run_heads(const HeadsArgs& a, int32_t dt, int64_t grid, hipStream_t s) {
  const dim3 g((uint32_t)grid), b(kThreads);
  if (dt == EA_F32) heads_kernel<LPH, EA_F32, MODE><<<g, b, 0, s>>>(a);
  else if (dt == EA_BF16) heads_kernel<LPH, EA_BF16, MODE><<<g, b, 0, s>>>(a);
  else heads_kernel<LPH, EA_F16, MODE><<<g, b, 0, s>>>(a);
  return hipGetLastError();
}
template <int LPH, int MODE>
hipError_t run_heads(const HeadsGradArgs& a, int32_t dt, int64_t grid, hipStream_t s) {
  const dim3 g((uint32_t)grid), b(kThreads);
  if (dt == EA_F32) heads_grad_kernel<LPH, EA_F32, MODE><<<g, b, 0, s>>>(a);
  else if (dt == EA_BF16) heads_grad_kernel<LPH, EA_BF16, MODE><<<g, b, 0, s>>>(a);
  else heads_grad_kernel<LPH, EA_F16, MODE><<<g, b, 0, s>>>(a);
  return hipGetLastError();
}

// Lanes of a head row: 16 elements each, a power of two from 4 up.
int lanes_of(int d) {
  int n = 4;
  while (n * 16 < d) n *= 2;
  return n;
}

// Workgroups of a launch, and the groups of heads that a wave walks for one
// token: so many that the launch is one round of the `waves` a CU that its
// registers admit, up to all of a token's.
template <class A>
int64_t split(A* a, int waves) {
  const int rpw = 64 / lanes_of(a->d), groups = (a->hq + 2 * a->hkv + rpw - 1) / rpw;
  const int64_t gpw = ((int64_t)a->t * groups + waves * 256 - 1) / (waves * 256);
  a->groups_per_wave = (int32_t)(gpw > groups ? groups : gpw);
  const int64_t parts = (groups + a->groups_per_wave - 1) / a->groups_per_wave;
  return ((int64_t)a->t * parts + kWaves - 1) / kWaves;
}

template <int LPH, class A>
hipError_t run_mode(const A& a, int32_t dt, int64_t grid, hipStream_t s) {
  if (a.inter || a.rot == 0) return run_heads<LPH, NEIGHBOURS>(a, dt, grid, s);
  if ((a.rot / 2) % 8) return run_heads<LPH, APART>(a, dt, grid, s);
  return run_heads<LPH, HALVES>(a, dt, grid, s);
}
template <class A>
hipError_t run_any(const A& a, int32_t dt, int64_t grid, hipStream_t s) {
  switch (lanes_of(a.d)) {
    case 4: return run_mode<4>(a, dt, grid, s);
    case 8: return run_mode<8>(a, dt, grid, s);
    case 16: return run_mode<16>(a, dt, grid, s);
    default: return run_mode<32>(a, dt, grid, s);
  }
}

}  // namespace

hipError_t launch_heads(const HeadsArgs& a0, int32_t dt, hipStream_t s) {
  HeadsArgs a = a0;
  const int64_t wgs = split(&a, 16);
  return run_any(a, dt, wgs < kHeadsMaxWg ? wgs : kHeadsMaxWg, s);
}

hipError_t launch_heads_grad(const HeadsGradArgs& a0, int32_t dt, hipStream_t s) {
  HeadsGradArgs a = a0;
  // its registers admit three workgroups a CU (two in f32): more would wait
  // for a second round and leave the chip half empty
  const int64_t most = dt == EA_F32 ? 512 : kHeadsGradMaxWg;
  const int64_t wgs = split(&a, dt == EA_F32 ? 8 : 12);
  a.n_wg = (int32_t)(wgs < most ? wgs : most);
  const hipError_t e = run_any(a, dt, a.n_wg, s);
  if (e != hipSuccess || !a.part) return e;
  heads_dw_kernel<<<dim3(2 * (a.d / 8)), dim3(kThreads), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace ea
