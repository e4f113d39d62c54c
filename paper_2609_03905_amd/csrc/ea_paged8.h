// ea_paged8.h -- attention over a paged cache in 8 bits (the call is cut as in
// ea_paged.hip).  With codes c and scales k_j, v_j of a key's blocks,
//   O = sum_j w_j v_j cv_j / sum_j w_j,   w_j = 2^(s_j - m),
//   s_j = scale log2(e) k_j q.ck_j
// Codes are widened on their way to the matrix cores, K's to q's type, V's to bf16.
// A scale is a power of two, and a code has at most four significant bits: c s is
// exact in bf16 from 2^-133 to below 2^128, so that there the widening instruction
// applies the scale.  (e5m2's least codes are below under scales of 2^-118 and less,
// codes of 2^8 and more above under 2^120: V's are taken out, see below.)  Where it
// does not, the scales enter in f32: k_j a score (fp16 queries), v_j a weight (the
// walk over few columns, which widens the codes of two keys at once).  The weights,
// whose exponents may be as far apart as f32's, go to the product with V as two bf16
// values.
#pragma once

#include "ea_paged.h"

namespace ea {

namespace {

typedef float f32x2_t __attribute__((ext_vector_type(2)));

// Two codes of a word, the lower or the upper, times a power of two, as two values
// of a type.  (The instruction takes the scale's exponent alone; NaN gives NaN.
// Every code times every power from 2^-120 to 2^120 was compared: exact where bf16
// has the number, its subnormal ones among them, which the matrix cores take as they
// are; below them rounded, above them an infinity.)
template <bool BF, bool E5, bool UP>
__device__ __forceinline__ uint32_t widen2(uint32_t w, float s) {
  if constexpr (BF && E5) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, s, UP));
  else if constexpr (BF) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, UP));
  else if constexpr (E5) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(w, s, UP));
  else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, s, UP));
}
template <bool BF, bool E5>
__device__ __forceinline__ uint4 widen8(uint32_t a, uint32_t b, float s) {
  return make_uint4(widen2<BF, E5, false>(a, s), widen2<BF, E5, true>(a, s), widen2<BF, E5, false>(b, s),
                    widen2<BF, E5, true>(b, s));
}

// A scale, NaN where it is no power of two of its range: what such a scale stands
// for shows in every row that sees it.
__device__ __forceinline__ float power_of_two(float s) {
  const uint32_t b = __float_as_uint(s);
  return (b & 0x807fffffu) == 0 && b - 0x00800000u < 0x7f000000u ? s : NAN;
}

// 0 V is no number where V is not finite, and a column that does not see a value
// gives it the weight 0: codes that stand for no number, or for one past bf16's (and
// f32's) range, are taken out of the product and added to the columns that see them.
// Those are a scale's codes from one on, the signs aside: e4m3's NaN 0x7f, e5m2's
// infinity 0x7c, or 2^k with 2^k times the scale 2^128.
template <bool E5>
__device__ __forceinline__ uint32_t odd_from(float scale) {  // 128 less the first, in every byte
  // (2^k is the code 8 (k + 7), or 4 (k + 15))
  const int k = 255 - (int)(__float_as_uint(scale) >> 23);
  return 0x01010101u * (uint32_t)(128 - (E5 ? min(0x7c, 4 * (k + 15)) : min(0x7f, 8 * (k + 7))));
}
// The top bit of the word's codes that are such.
template <bool E5>
__device__ __forceinline__ uint32_t odd_codes(uint32_t w, uint32_t from = odd_from<E5>(1.0f)) {
  return ((w & 0x7f7f7f7fu) + from) & 0x80808080u;
}
// The word with zeros in their place.
template <bool E5>
__device__ __forceinline__ uint32_t even_codes(uint32_t w, uint32_t from = odd_from<E5>(1.0f)) {
  const uint32_t top = odd_codes<E5>(w, from);
  return w & ~(top | (top - (top >> 7)));
}
// What such codes, times a scale, add to the sums x.
template <bool E5>
__device__ __forceinline__ void add_odd4(uint32_t w, float scale, float (&x)[4]) {
  f32x2_t lo, hi;
  if constexpr (E5) lo = __builtin_amdgcn_cvt_pk_f32_bf8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_bf8(w, true);
  else lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  const float v[4] = {lo[0] * scale, lo[1] * scale, hi[0] * scale, hi[1] * scale};
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] += __builtin_isfinite(v[i]) ? 0.0f : v[i];
}

// Shared memory of the two walks.
template <int D>
struct __attribute__((aligned(16))) Few8Shared {
  int64_t off[kWaves][2][kPaged8Step / kWaves];
  float scale[kWaves][2][kPaged8Step / kWaves];  // of a step's keys: K's, V's
  float o[kWaves][kPagedCols][D + 4];
  float ml[kWaves][kPagedCols][2];
  int last;
};
template <int D>
struct __attribute__((aligned(1024))) Many8Shared {
  uint16_t kv[2][2 * kPagedWideStep * D];  // two steps' buffers: K, then V
  int64_t off[3][kPagedWideStep];
  float ks[2][kPagedWideStep];   // K's scales (fp16 queries)
  float vs[2][kPagedWideStep];   // V's, NaN for none
  int odd[2][kWaves];            // whether a wave found such a scale, or odd codes
  int lim[kWaves];               // the keys that every column of a wave sees
};

// Few columns: each wave walks its own 64 keys of a step of 256, codes from the
// pages to registers.
//   S^T = K Q^T     (16x16x32: A = 16 keys x 32 d, B = 32 d x 16 columns)
//   O^T += V^T P^T  (A = 16 d x 32 keys, B = 32 keys x 16 columns)
// A lane's 16 bytes of a K row are two steps' k indices, Q's are taken alike.  A V
// row's lane has D / 16 neighbouring codes of each of the sixteen keys whose
// scores its column's accumulators hold; a byte permutation puts two keys' codes of
// one d side by side, and widening them gives the operand.  Bound by HBM where there
// is work for the chip: 48 ragged sequences of up to 8K keys, 4 heads over each of 8,
// 85.5 us, 4.7 TB/s (a wave's step of 32 keys, its scales as f32 factors: 96); one
// sequence alone by the chain of its round trips (1000 keys 10.0 us, over 16 bits 9.4).
// Two waves a SIMD: their registers hold the step's codes.
template <int D, bool BF, bool E5, int COLS>
__device__ __forceinline__ void walk_few8(const PagedArgs& a, const PagedPass& ps, const Seg* seg, Few8Shared<D>& sh,
                                          int total, int parts, int block) {
  constexpr int NC = COLS / kPagedCols;
  constexpr int VE = D / 16;                // codes a lane holds of a V row
  constexpr int KL = D / 64;                // loads of 16 codes of a K row
  constexpr int NK = kPaged8Step / kWaves;  // keys of a wave's step
  constexpr int NT = NK / 16;               // and tiles of 16 of them

  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g4 = lane >> 4;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int w = xcd_part(block, parts);
  int at = (int)((int64_t)total * w / parts);
  const int end = (int)((int64_t)total * (w + 1) / parts);
  static_assert(NK == 64, "a lane a key");

  auto next_piece = [&]() {
    Piece p;
    p.si = find_segment(seg, ps.n, at);
    p.s = seg[p.si];
    p.n = steps_of(p.s.k0, p.s.k1, kPaged8Step);
    const int tiles = tiles_of(p.s.rows, a.g, COLS);
    const int local = at - p.s.step, step = local % p.n;
    p.it = local / p.n;
    p.h = p.it / tiles;
    p.tile = p.it - p.h * tiles;
    const int walk = min(p.n - step, end - at);
    p.whole = walk == p.n && p.s.k0 == 0;
    p.ka = p.s.k0 + step * kPaged8Step;
    p.kb = (int)min((int64_t)p.s.k1, (int64_t)p.ka + (int64_t)walk * kPaged8Step);
    p.pages = a.table + (int64_t)p.s.seq * a.stride;
    p.head_off = (int64_t)p.h * a.page_size * D;
    at += walk;
    return p;
  };
  // What a step's lane knows of its key: the row's place goes to shared memory
  // (any row's, if the key has none), the scales follow a step later.
  struct Keys {
    uint64_t there;  // keys that have a row
    float ks, vs;    // this lane's key's scales
  };
  auto entry = [&](const Piece& p, int k) { return k + lane < p.kb ? p.pages[div_fast(k + lane, a.page)] : -1; };
  auto place = [&](const Piece& p, int slot, int k, int pg) {
    const int key = k + lane, in = key - div_fast(key, a.page) * a.page_size;
    const bool there = (uint32_t)pg < (uint32_t)a.n_pages;
    sh.off[wid][slot][lane] = there ? pg * a.page_bytes + (int64_t)in * D : 0;
    __builtin_amdgcn_wave_barrier();
    const int64_t i = there ? ((int64_t)pg * a.hkv + p.h) * a.n_blocks + div_fast(in, a.block) : 0;
    return Keys{__ballot(there), a.ks[i], a.vs[i]};
  };
  uint4 kr[NT][KL];
  uint32_t vr[4 * NT][VE / 4];
  auto load_k = [&](const Piece& pc, int slot) {
    const char* base = a.pk + pc.head_off + g4 * 16;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const char* p = base + sh.off[wid][slot][16 * t + c];
#pragma unroll
      for (int i = 0; i < KL; ++i) kr[t][i] = *reinterpret_cast<const uint4*>(p + i * 64);
    }
  };
  auto load_v = [&](const Piece& pc, int slot) {
    const char* base = a.pv + pc.head_off + c * VE;
#pragma unroll
    for (int i = 0; i < 4 * NT; ++i) {
      const char* p = base + sh.off[wid][slot][16 * (i >> 2) + 4 * g4 + (i & 3)];
      if constexpr (VE == 8) {
        const uint2 x = *reinterpret_cast<const uint2*>(p);
        vr[i][0] = x.x, vr[i][1] = x.y;
      } else {
        vr[i][0] = *reinterpret_cast<const uint32_t*>(p);
      }
    }
  };
  uint4 q[NC][2 * KL];
  auto load_q = [&](const Piece& pc) {  // this lane's columns: query rows and heads
#pragma unroll
    for (int t = 0; t < NC; ++t) {
      const int cc = min(pc.tile * COLS + t * kPagedCols + c, pc.s.rows * a.g - 1);
      const int rr = div_fast(cc, a.gdiv);
      const char* p = a.pq + row_offset(a.q, pc.s.r0 + rr, pc.h * a.g + cc - rr * a.g) + g4 * 32;
#pragma unroll
      for (int i = 0; i < 2 * KL; ++i) q[t][i] = *reinterpret_cast<const uint4*>(p + (i >> 1) * 128 + (i & 1) * 16);
    }
  };

  // The loads of a step are on their way while the step before is computed, also
  // from one piece to the next.
  Piece next = next_piece();
  int slot = 0, next_pg = entry(next, next.ka + wid * NK);
  load_q(next);
  Keys keys = place(next, 0, next.ka + wid * NK, next_pg);
  load_k(next, 0);
  load_v(next, 0);
  bool have = true;
  while (have) {
    const Piece cur = next;
    have = at < end;
    int first_pg = -1;
    if (have) {
      next = next_piece();
      first_pg = entry(next, next.ka + wid * NK);
    }
    const Seg s = cur.s;
    const int tile = cur.tile, kb = cur.kb, slot_out = s.tile + cur.it + w;

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
    int k = cur.ka + wid * NK;
    next_pg = entry(cur, k + kPaged8Step);
    for (bool again = true; again; k += kPaged8Step) {
      again = k + kPaged8Step < kb;
      const uint64_t there = keys.there;
      // every key of the step has a row and is seen by every column
      const bool full = there == ~uint64_t(0) && k + NK <= lim_min;
      sh.scale[wid][0][lane] = power_of_two(keys.ks);
      sh.scale[wid][1][lane] = power_of_two(keys.vs);
      __builtin_amdgcn_wave_barrier();
      if (again) {
        keys = place(cur, slot ^ 1, k + kPaged8Step, next_pg);
        next_pg = entry(cur, k + 2 * kPaged8Step);
      } else if (have) {
        keys = place(next, slot ^ 1, next.ka + wid * NK, first_pg);
      }
      f32x4_t sc[NC][NT];
#pragma unroll
      for (int u = 0; u < NT; ++u) {
#pragma unroll
        for (int t = 0; t < NC; ++t) sc[t][u] = f32x4_t{};
        const float ks = BF ? sh.scale[wid][0][16 * u + c] : 1.0f;
#pragma unroll
        for (int i = 0; i < KL; ++i) {
          const uint4 k0 = widen8<BF, E5>(kr[u][i].x, kr[u][i].y, ks), k1 = widen8<BF, E5>(kr[u][i].z, kr[u][i].w, ks);
#pragma unroll
          for (int t = 0; t < NC; ++t) {
            sc[t][u] = mfma16<BF>(k0, q[t][2 * i], sc[t][u]);
            sc[t][u] = mfma16<BF>(k1, q[t][2 * i + 1], sc[t][u]);
          }
        }
      }
      if (again) load_k(cur, slot ^ 1);
      else if (have) load_k(next, slot ^ 1);
      if constexpr (!BF) {  // (a scaled code may be out of fp16's reach)
#pragma unroll
        for (int u = 0; u < NT; ++u) {
          const f32x4_t ks = *reinterpret_cast<const f32x4_t*>(&sh.scale[wid][0][16 * u + 4 * g4]);
#pragma unroll
          for (int t = 0; t < NC; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[t][u][i] *= ks[i];
        }
      }
      uint32_t odd = 0;
      if (__builtin_expect(!full, 0)) {
        asm volatile("" ::: "memory");
        const uint64_t mine = there >> (4 * g4);
#pragma unroll
        for (int i = 0; i < 4 * NT; ++i) {
          const bool row_there = mine >> (16 * (i >> 2) + (i & 3)) & 1;
#pragma unroll
          for (int t = 0; t < NC; ++t) {
            const float x = sc[t][i >> 2][i & 3];
            sc[t][i >> 2][i & 3] = row_there && k + 16 * (i >> 2) + 4 * g4 + (i & 3) < lim[t] ? x : -INFINITY;
          }
          // a row that is not there was read elsewhere: it may hold anything
#pragma unroll
          for (int j = 0; j < VE / 4; ++j) vr[i][j] = row_there ? vr[i][j] : 0u;
        }
      }
      // (where every column sees every key, NaN times its weight is right as it
      // is, but an infinity's second weight may be 0)
      if (E5 || !full) {
#pragma unroll
        for (int i = 0; i < 4 * NT; ++i)
#pragma unroll
          for (int j = 0; j < VE / 4; ++j) odd |= odd_codes<E5>(vr[i][j]);
        if (__builtin_expect(__any(odd != 0), 0)) {
#pragma unroll
          for (int i = 0; i < 4 * NT; ++i)
#pragma unroll
            for (int j = 0; j < VE / 4; ++j) vr[i][j] = even_codes<E5>(vr[i][j]);
        }
      }
      uint4 p[NC][NT / 2], p2[NC][NT / 2];
#pragma unroll
      for (int t = 0; t < NC; ++t) {
        float mx = sc[t][0][0];
#pragma unroll
        for (int i = 1; i < 4 * NT; ++i) mx = fmaxf(mx, sc[t][i >> 2][i & 3]);
        mx = fmaxf(mx, other16(mx));
        mx = fmaxf(mx, other32(mx)) * a.scale;
        const float m_new = mx > m[t] + kLazyMax || m[t] == -INFINITY ? fmaxf(mx, m[t]) : m[t];
        const float m_use = m_new == -INFINITY ? 0.0f : m_new;
        if (__any(m_new != m[t])) {
          asm volatile("" ::: "memory");
          const float alpha = __builtin_amdgcn_exp2f(m[t] - m_use);
          l[t] *= alpha;
#pragma unroll
          for (int j = 0; j < VE; ++j) acc[t][j] *= alpha;
        }
        m[t] = m_new;
        float x[4 * NT];
#pragma unroll
        for (int i = 0; i < 4 * NT; ++i)
          x[i] = __builtin_amdgcn_exp2f(fmaf(sc[t][i >> 2][i & 3], a.scale, -m_use));
#pragma unroll
        for (int i = 0; i < 4 * NT; i += 4) l[t] += (x[i] + x[i + 1]) + (x[i + 2] + x[i + 3]);
#pragma unroll
        for (int u = 0; u < NT; ++u) {
          const f32x4_t vs = *reinterpret_cast<const f32x4_t*>(&sh.scale[wid][1][16 * u + 4 * g4]);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[4 * u + i] *= vs[i];
        }
        if (!full) {  // (the scale of a key that is not seen may be anything)
#pragma unroll
          for (int i = 0; i < 4 * NT; ++i) x[i] = sc[t][i >> 2][i & 3] == -INFINITY ? 0.0f : x[i];
        }
#pragma unroll
        for (int u = 0; u < NT / 2; ++u) {
          split_p<true>(x[8 * u], x[8 * u + 1], p[t][u].x, p2[t][u].x);
          split_p<true>(x[8 * u + 2], x[8 * u + 3], p[t][u].y, p2[t][u].y);
          split_p<true>(x[8 * u + 4], x[8 * u + 5], p[t][u].z, p2[t][u].z);
          split_p<true>(x[8 * u + 6], x[8 * u + 7], p[t][u].w, p2[t][u].w);
        }
      }
#pragma unroll
      for (int j = 0; j < VE; j += 2)
#pragma unroll
        for (int u = 0; u < NT / 2; ++u) {
          // d j and j + 1 of two keys a word
          const uint32_t sel = j & 2 ? 0x07030602u : 0x05010400u;
          uint32_t x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            x[i] = __builtin_amdgcn_perm(vr[8 * u + 2 * i + 1][j / 4], vr[8 * u + 2 * i][j / 4], sel);
          const uint4 v0 = make_uint4(widen2<true, E5, false>(x[0], 1.0f), widen2<true, E5, false>(x[1], 1.0f),
                                      widen2<true, E5, false>(x[2], 1.0f), widen2<true, E5, false>(x[3], 1.0f));
          const uint4 v1 = make_uint4(widen2<true, E5, true>(x[0], 1.0f), widen2<true, E5, true>(x[1], 1.0f),
                                      widen2<true, E5, true>(x[2], 1.0f), widen2<true, E5, true>(x[3], 1.0f));
#pragma unroll
          for (int t = 0; t < NC; ++t) {
            acc[t][j] = mfma16<true>(v0, p[t][u], acc[t][j]);
            acc[t][j + 1] = mfma16<true>(v1, p[t][u], acc[t][j + 1]);
            acc[t][j] = mfma16<true>(v0, p2[t][u], acc[t][j]);
            acc[t][j + 1] = mfma16<true>(v1, p2[t][u], acc[t][j + 1]);
          }
        }
      if (__builtin_expect(__any(odd != 0), 0)) {
#pragma unroll 1
        for (int kk = 0; kk < NK; ++kk) {
          if (!(there >> kk & 1)) continue;
          const char* row = a.pv + cur.head_off + sh.off[wid][slot][kk];
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < VE; j += 4) {
              const uint32_t v = *reinterpret_cast<const uint32_t*>(row + (4 * g4 + i) * VE + j);
#pragma unroll
              for (int t = 0; t < NC; ++t) {
                float x[4] = {acc[t][j][i], acc[t][j + 1][i], acc[t][j + 2][i], acc[t][j + 3][i]};
                if (k + kk < lim[t]) add_odd4<E5>(v, 1.0f, x);
                acc[t][j][i] = x[0], acc[t][j + 1][i] = x[1], acc[t][j + 2][i] = x[2], acc[t][j + 3][i] = x[3];
              }
            }
        }
      }
      if (again) load_v(cur, slot ^ 1);
      else if (have) load_v(next, slot ^ 1);
      slot ^= 1;
    }
    if (have) load_q(next);
    finish_few<D, BF, COLS>(a, ps, cur, slot_out, acc, m, l, sh, total, parts);
  }
}

// Many columns: steps of 64 keys, widened on the way to shared memory by the
// thread that fetched them (a wave's column tiles share the work), one step ahead
// of the products; tiles and products as for a cache in 16 bits.  Bound by the
// vector instructions and products of a step, about half and a third of its clocks:
// 32 sequences that share 64K keys, 4 heads over each of 8, 92 us (over 16 bits 96),
// whose bytes are twice as many (scales as f32 factors 107).  Without a gain: widening
// between the products of the step before (102), weights of sixteen keys computed
// under the products of the sixteen before (98; one product and six instructions in
// turn, forced, 116).  One fp16 weight instead of two bf16 values needs V relative to
// a largest scale, which a key that a mask hides may set: small values would go.
template <int D, bool BF, bool E5, int COLS>
__device__ __forceinline__ void walk_many8(const PagedArgs& a, const PagedPass& ps, const Seg* seg, const Seg* own,
                                           Many8Shared<D>& sh, int total, int parts, int block) {
  constexpr int CW = COLS / 32, KEYS = kPagedWideStep;
  constexpr int KT = CW / 2;         // 32-key tiles that a wave computes of a step
  constexpr int NS = D / 16, ND = D / 32;
  constexpr int LPR = D / 16;        // lanes of a row: 16 codes each
  constexpr int RPI = 64 / LPR;      // rows of one load
  constexpr int LPW = 16 / RPI;      // loads of a wave (16 rows) for K, and for V
  constexpr int BUF = 2 * KEYS * D;  // elements of a step: K, then V
  uint16_t* sKV = sh.kv[0];
  auto& s_off = sh.off;

  // (one by one in scalar registers: they are too many to stay there, and the
  // arguments' come back from a spill in eights)
  FastDiv dpage = a.page, dblock = a.block;
  int page_size = a.page_size, n_pages = a.n_pages;
  int64_t page_bytes = a.page_bytes, page_scales = (int64_t)a.hkv * a.n_blocks;
  asm("" : "+s"(dpage.d), "+s"(dpage.m), "+s"(dpage.s), "+s"(dblock.d), "+s"(dblock.m), "+s"(dblock.s));
  asm("" : "+s"(page_size), "+s"(n_pages), "+s"(page_bytes), "+s"(page_scales));

  const int tid = threadIdx.x, lane = tid & 63, lq = lane & 31, g = lane >> 5;
  const int wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wc = wid % CW, wk = wid / CW;  // the wave's columns, and its part of a step's keys
  const int w = xcd_part(block, parts);
  int at = (int)((int64_t)total * w / parts);
  const int end = (int)((int64_t)total * (w + 1) / parts);

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
    const int64_t head_off = (int64_t)h * a.page_size * D;
    const char* kbase = a.pk + head_off + (lane % LPR) * 16;
    const char* vbase = a.pv + head_off + (lane % LPR) * 16;
    // a wave fetches 16 of a step's rows; lane i (and i + 16, ...) looks after row
    // i, the first 16 after K's scale, the next after V's
    const int my = wid * 16 + (lane & 15);
    const float* scales = (lane & 16 ? a.vs : a.ks) + (int64_t)h * a.n_blocks;
    auto entry = [&](int k) { return k + my < kb ? pages[div_fast(k + my, dpage)] : -1; };
    bool lacking;                                // some of the wave's rows do not exist
    auto place = [&](int slot, int k, int pg) {  // the rows' offsets, -1: no such row; the scale
      const int key = k + my, in = key - div_fast(key, dpage) * page_size;
      const bool there = (uint32_t)pg < (uint32_t)n_pages;
      const int64_t off = there ? pg * page_bytes + (int64_t)in * D : -1;
      if (lane < 16) s_off[slot][my] = off;
      lacking = __ballot(!there) != 0;
      __builtin_amdgcn_wave_barrier();
      return there ? scales[pg * page_scales + div_fast(in, dblock)] : 1.0f;
    };
    uint4 kr[LPW], vr[LPW];
    float scale;
    auto fetch = [&](int slot) {
#pragma unroll
      for (int i = 0; i < LPW; ++i) {
        const int64_t off = s_off[slot][(wid * LPW + i) * RPI + lane / LPR];
        kr[i] = *reinterpret_cast<const uint4*>(kbase + (off < 0 ? 0 : off));
        vr[i] = *reinterpret_cast<const uint4*>(vbase + (off < 0 ? 0 : off));
      }
    };
    int lim_all = 0;  // the keys that every column of the workgroup sees
    // Widened to buffer b.  Zeros in the place of values whose rows do not exist, and
    // of odd codes where some column may not see them, which sh.odd tells of.  (Where
    // all columns see all of the step's rows, e4m3's NaN is right as it is; an
    // infinity's second weight may be 0.  Without the checks 64K prefix 99 us to 97.)
    auto land = [&](int b, int slot, int k) {
      uint16_t* sK = sKV + b * BUF;
      uint16_t* sV = sK + KEYS * D;
      scale = power_of_two(scale);
      const bool none = scale != scale;
      // (a scale under which every finite code is a number in bf16)
      const bool care = E5 || lacking || k + KEYS > lim_all || __any(!(scale < 0x1p120f));
      if (!BF && lane < 16) sh.ks[b][my] = scale;
      if (lane >= 16 && lane < 32) sh.vs[b][my] = scale;
      bool any = false;
      uint4 v[LPW];
      float vs[LPW];
#pragma unroll
      for (int i = 0; i < LPW; ++i) {
        const int row = i * RPI + lane / LPR, r = wid * 16 + row, pc = 2 * (lane % LPR);
        const float ks = BF ? __shfl(scale, row) : 1.0f;
        vs[i] = __shfl(scale, 16 + row);
        uint4* tk = reinterpret_cast<uint4*>(sK + r * D);
        tk[pc ^ swz_k<D>(r)] = widen8<BF, E5>(kr[i].x, kr[i].y, ks);
        tk[(pc + 1) ^ swz_k<D>(r)] = widen8<BF, E5>(kr[i].z, kr[i].w, ks);
        v[i] = vr[i];
      }
      if (care) {
        asm volatile("" ::: "memory");  // a branch
        uint32_t odd = none && lane >= 16 && lane < 32;
#pragma unroll
        for (int i = 0; i < LPW; ++i) {
          if (s_off[slot][wid * 16 + i * RPI + lane / LPR] < 0 || vs[i] != vs[i]) v[i] = make_uint4(0, 0, 0, 0);
          const uint32_t f = odd_from<E5>(vs[i]);
          odd |= odd_codes<E5>(v[i].x, f) | odd_codes<E5>(v[i].y, f) | odd_codes<E5>(v[i].z, f) | odd_codes<E5>(v[i].w, f);
        }
        any = __any(odd != 0);
        if (__builtin_expect(any, 0)) {
#pragma unroll
          for (int i = 0; i < LPW; ++i) {
            const uint32_t f = odd_from<E5>(vs[i]);
            v[i] = make_uint4(even_codes<E5>(v[i].x, f), even_codes<E5>(v[i].y, f), even_codes<E5>(v[i].z, f),
                              even_codes<E5>(v[i].w, f));
            if (vs[i] != vs[i]) vs[i] = 1.0f;
          }
        }
      }
#pragma unroll
      for (int i = 0; i < LPW; ++i) {
        const int r = wid * 16 + i * RPI + lane / LPR, pc = 2 * (lane % LPR);
        uint4* tv = reinterpret_cast<uint4*>(sV + r * D);
        tv[pc ^ swz_v<D>(r)] = widen8<true, E5>(v[i].x, v[i].y, vs[i]);
        tv[(pc + 1) ^ swz_v<D>(r)] = widen8<true, E5>(v[i].z, v[i].w, vs[i]);
      }
      if (lane == 0) sh.odd[b][wid] = any;
    };
    scale = place(0, ka, entry(ka));
    fetch(0);
    int next_pg = entry(ka + KEYS);

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
    if (lane == 0) sh.lim[wid] = lim_min;

    f32x16_t acc[ND];
#pragma unroll
    for (int i = 0; i < ND; ++i) acc[i] = f32x16_t{};
    float m = -INFINITY, l = 0.0f;

    auto compute = [&](int b, int slot, int k) {
      // every key of the step has a row and is seen by every column of the wave
      const uint64_t there = __ballot(s_off[slot][lane] >= 0);
      const bool full = there == ~uint64_t(0) && k + KEYS <= lim_min;
      const uint16_t* sK = sKV + b * BUF;
      const uint16_t* sV = sK + KEYS * D;
      f32x16_t sc[KT];
#pragma unroll
      for (int t = 0; t < KT; ++t) sc[t] = f32x16_t{};
      __builtin_amdgcn_s_setprio(1);
      uint4 x[2][KT];
      auto read_k = [&](int i) {
#pragma unroll
        for (int t = 0; t < KT; ++t) {
          const int r = 32 * (wk * KT + t) + lq;
          x[i & 1][t] = *reinterpret_cast<const uint4*>(sK + r * D + 8 * ((2 * i + g) ^ swz_k<D>(r)));
        }
      };
      read_k(0);
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        if (i + 1 < NS) read_k(i + 1);
        __builtin_amdgcn_sched_barrier(0);  // (the next operand on its way before this one's products)
#pragma unroll
        for (int t = 0; t < KT; ++t) sc[t] = mfma32<BF>(x[i & 1][t], q[i], sc[t]);
      }
      __builtin_amdgcn_s_setprio(0);
      if constexpr (!BF) {  // (a scaled code may be out of fp16's reach)
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const f32x4_t ks = *reinterpret_cast<const f32x4_t*>(&sh.ks[b][32 * (wk * KT + t) + 8 * r + 4 * g]);
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[t][4 * r + e] *= ks[e];
          }
      }
      if (__builtin_expect(!full, 0)) {
        asm volatile("" ::: "memory");  // a branch: the masks would be a third of a step's instructions
        const uint64_t mine = there >> (32 * wk * KT + 4 * g);
        const int seen = lim - k - 32 * wk * KT - 4 * g;
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int kk = 32 * t + 8 * (r >> 2) + (r & 3);
            sc[t][r] = (mine >> kk & 1) && kk < seen ? sc[t][r] : -INFINITY;
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
        asm volatile("" ::: "memory");  // a branch: most steps leave the maximum where it is
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
        for (int r = 0; r < 16; ++r) sc[t][r] = __builtin_amdgcn_exp2f(fmaf(sc[t][r], a.scale, -m_use));
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          uint4 p, p2;
          split_p<true>(sc[t][8 * hh], sc[t][8 * hh + 1], p.x, p2.x);
          split_p<true>(sc[t][8 * hh + 2], sc[t][8 * hh + 3], p.y, p2.y);
          split_p<true>(sc[t][8 * hh + 4], sc[t][8 * hh + 5], p.z, p2.z);
          split_p<true>(sc[t][8 * hh + 6], sc[t][8 * hh + 7], p.w, p2.w);
#pragma unroll
          for (int i = 0; i < 8; ++i) l += sc[t][8 * hh + i];
          const int k0 = 32 * (wk * KT + t) + 16 * hh + 4 * (gq >> 1) + (li >> 2);
          uint4 y[ND];
#pragma unroll
          for (int i = 0; i < ND; ++i) {
            const int d = 32 * i + 16 * (gq & 1) + 4 * (li & 3);
            auto tr = [&](int r) {
              return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(
                  sV + r * D + 8 * ((d >> 3) ^ swz_v<D>(r)) + (d & 4)));
            };
            const s16x8_t v = __builtin_shufflevector(tr(k0), tr(k0 + 8), 0, 1, 2, 3, 4, 5, 6, 7);
            y[i] = __builtin_bit_cast(uint4, v);
            acc[i] = mfma32<true>(y[i], p, acc[i]);
          }
#pragma unroll
          for (int i = 0; i < ND; ++i) acc[i] = mfma32<true>(y[i], p2, acc[i]);
        }
      __builtin_amdgcn_s_setprio(0);
      if (__builtin_expect(sh.odd[b][0] | sh.odd[b][1] | sh.odd[b][2] | sh.odd[b][3], 0)) {
#pragma unroll 1
        for (int kk = 32 * wk * KT; kk < 32 * (wk + 1) * KT; ++kk) {
          const int64_t off = s_off[slot][kk];
          if (off < 0) continue;
          const char* vrow = a.pv + head_off + off + 4 * g;
          const float vs = sh.vs[b][kk];  // (NaN: in all of the row)
#pragma unroll
          for (int i = 0; i < ND; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const uint32_t v = *reinterpret_cast<const uint32_t*>(vrow + 32 * i + 8 * r);
              float x[4] = {acc[i][4 * r], acc[i][4 * r + 1], acc[i][4 * r + 2], acc[i][4 * r + 3]};
              if (k + kk < lim) add_odd4<E5>(vs != vs ? 0x7f7f7f7fu : v, vs != vs ? 1.0f : vs, x);
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[i][4 * r + e] = x[e];
            }
        }
      }
    };

    // A step's codes are fetched two steps ahead and land, widened, one step ahead,
    // before the products of the step between: their loads had a whole step's time.
    land(0, 0, ka);
    if (ka + KEYS < kb) {
      scale = place(1, ka + KEYS, next_pg);
      next_pg = entry(ka + 2 * KEYS);
      fetch(1);
    }
    __syncthreads();
    lim_all = __builtin_amdgcn_readfirstlane(min(min(sh.lim[0], sh.lim[1]), min(sh.lim[2], sh.lim[3])));
    int b = 0, slot = 0;
    for (int k = ka; k < kb; k += KEYS, b ^= 1) {
      const int slot1 = slot == 2 ? 0 : slot + 1, slot2 = slot1 == 2 ? 0 : slot1 + 1;
      if (k + KEYS < kb) {
        land(b ^ 1, slot1, k + KEYS);
        if (k + 2 * KEYS < kb) {
          scale = place(slot2, k + 2 * KEYS, next_pg);
          next_pg = entry(k + 3 * KEYS);
          fetch(slot2);
        }
      }
      if (!idle) compute(b, slot, k);
      slot = slot1;
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

// Keys of a step of a walk over tiles of COLS columns.
template <int COLS>
__device__ __forceinline__ constexpr int step_keys() {
  return COLS <= 32 ? kPaged8Step : kPagedWideStep;
}

// The sequences' own keys alone.
template <int D, bool BF, bool E5, int COLS>
__global__ __launch_bounds__(kThreads, COLS == 32 && D == 128 ? 1 : 2) void paged8_kernel(const PagedArgs a,
                                                                                           const PagedPass ps) {
  extern __shared__ __attribute__((aligned(16))) char dyn[];
  Seg* seg = reinterpret_cast<Seg*>(dyn);
  int total;
  schedule<COLS, step_keys<COLS>(), 0, 1>(a, ps, ps, seg, nullptr, &total, nullptr);
  const int parts = min(ps.grid, total);
  if (ps.fused) clear_empty<D>(a, ps, seg);
  else publish<COLS, step_keys<COLS>()>(a, ps, seg, total, parts, blockIdx.x, gridDim.x);
  if ((int)blockIdx.x >= parts) return;
  if constexpr (COLS <= 32) {
    __shared__ Few8Shared<D> sh;
    walk_few8<D, BF, E5, COLS>(a, ps, seg, sh, total, parts, blockIdx.x);
  } else {
    __shared__ Many8Shared<D> sh;
    walk_many8<D, BF, E5, COLS>(a, ps, seg, nullptr, sh, total, parts, blockIdx.x);
  }
}

// Shared and own keys of a call with groups in one launch.
template <int D, bool BF, bool E5, int OWN, int SHARED>
__global__ __launch_bounds__(kThreads, 2) void paged8_both_kernel(const PagedArgs a, const PagedPass own,
                                                                  const PagedPass shared) {
  extern __shared__ __attribute__((aligned(16))) char dyn[];
  Seg* seg_o = reinterpret_cast<Seg*>(dyn);
  Seg* seg_s = seg_o + own.n + 1;
  __shared__ union Both {
    __device__ Both() {}
    Few8Shared<D> few;
    Many8Shared<D> many;
  } sh;
  constexpr int KO = step_keys<OWN>(), KS = step_keys<SHARED>();
  int to, ts;
  schedule<OWN, KO, SHARED, KS>(a, own, shared, seg_o, seg_s, &to, &ts);
  const int n = gridDim.x;
  // Workgroups are dealt to the walks by the bytes they read.  (Own keys weighted
  // more, up to 12 times: slower.  An equal part of both walks for every workgroup,
  // neighbours beginning with different ones: 8K prefix 47.6 us to 60.5.)
  const double ws = (double)ts * KS, wo = (double)to * KO;
  const int ns = ts == 0 ? 0 : to == 0 ? n : min(max((int)(n * ws / (ws + wo) + 4.0) / 8 * 8, 8), n - 8);
  const int ps = min(ns, ts), po = min(n - ns, to);
  publish<OWN, KO>(a, own, seg_o, to, po, blockIdx.x, n);
  publish<SHARED, KS>(a, shared, seg_s, ts, ps, blockIdx.x, n);
  const int b = blockIdx.x;
  if (b < ns) {
    if (b >= ps) return;
    walk_many8<D, BF, E5, SHARED>(a, shared, seg_s, seg_o, sh.many, ts, ps, b);
  } else {
    if (b - ns >= po) return;
    if constexpr (OWN <= 32) walk_few8<D, BF, E5, OWN>(a, own, seg_o, sh.few, to, po, b - ns);
    else walk_many8<D, BF, E5, OWN>(a, own, seg_o, nullptr, sh.many, to, po, b - ns);
  }
}

template <int D, bool BF, bool E5>
hipError_t run_own8(const PagedArgs& a, const PagedPass& p, hipStream_t s) {
  const dim3 g(p.grid), b(kThreads);
  const size_t lds = (p.n + 1) * sizeof(Seg);
  if (p.cols == 16) paged8_kernel<D, BF, E5, 16><<<g, b, lds, s>>>(a, p);
  else if (p.cols == 32) paged8_kernel<D, BF, E5, 32><<<g, b, lds, s>>>(a, p);
  else if (p.cols == 64) paged8_kernel<D, BF, E5, 64><<<g, b, lds, s>>>(a, p);
  else paged8_kernel<D, BF, E5, 128><<<g, b, lds, s>>>(a, p);
  return hipGetLastError();
}
template <int D, bool BF, bool E5, int OWN>
hipError_t run_both8(const PagedArgs& a, const PagedPass& own, const PagedPass& sh, hipStream_t s) {
  const dim3 g(own.grid), b(kThreads);
  const size_t lds = (own.n + sh.n + 2) * sizeof(Seg);
  if (sh.cols == 64) paged8_both_kernel<D, BF, E5, OWN, 64><<<g, b, lds, s>>>(a, own, sh);
  else paged8_both_kernel<D, BF, E5, OWN, 128><<<g, b, lds, s>>>(a, own, sh);
  return hipGetLastError();
}

template <int D, bool BF, bool E5>
hipError_t run_paged8(const PagedArgs& a, const PagedPass& sh, const PagedPass& own, hipStream_t s) {
  const hipError_t e = sh.n == 0         ? run_own8<D, BF, E5>(a, own, s)
                       : own.cols == 16  ? run_both8<D, BF, E5, 16>(a, own, sh, s)
                       : own.cols == 32  ? run_both8<D, BF, E5, D == 64 ? 32 : 16>(a, own, sh, s)
                       : own.cols == 64  ? run_both8<D, BF, E5, 64>(a, own, sh, s)
                                         : run_both8<D, BF, E5, 128>(a, own, sh, s);
  if (e != hipSuccess || own.fused) return e;
  return launch_paged_join(a, sh, own, D, BF ? EA_BF16 : EA_F16, s);
}

template <bool E5>
hipError_t run_code(const PagedArgs& a, const PagedPass& sh, const PagedPass& own, int32_t d, int32_t dt,
                    hipStream_t s) {
  if (d == 128) return dt == EA_BF16 ? run_paged8<128, true, E5>(a, sh, own, s) : run_paged8<128, false, E5>(a, sh, own, s);
  return dt == EA_BF16 ? run_paged8<64, true, E5>(a, sh, own, s) : run_paged8<64, false, E5>(a, sh, own, s);
}

}  // namespace

}  // namespace ea
