// ea_decode.h -- what the decoding operators (head rows, paged attention, the
// page table) share: addresses of head rows inside block-partitioned
// relations, and the argument blocks of their kernels.
#pragma once

#include "ea_internal.h"

namespace ea {

// n / d for 0 <= n < 2^31 and d >= 1 by one high multiply: m = ceil(2^(31+s) / d)
// with s = ceil(log2 d) exceeds the true reciprocal by less than 2^s / d <= 1
// units of 2^-(31+s) per n, so the quotient's floor is exact below 2^31.
struct FastDiv {
  uint32_t d = 1, m = 0, s = 0;
};
inline FastDiv fast_div(uint32_t d) {
  FastDiv f;
  f.d = d;
  if (d > 1) {
    uint32_t l = 0;
    while ((uint64_t(1) << l) < d) ++l;
    f.m = (uint32_t)(((uint64_t(1) << (31 + l)) + d - 1) / d);
    f.s = l - 1;
  }
  return f;
}
#if defined(__HIPCC__)
__device__ __forceinline__ int32_t div_fast(int32_t n, const FastDiv& f) {
  return f.d == 1 ? n : (int32_t)(__umulhi((uint32_t)n, f.m) >> f.s);
}
#endif

// Where head h of row t lies: the d elements are contiguous.  Two forms, both
// over a partition of equal blocks whose last one may be shorter:
//   token-major [T, H d]: blocks of tb rows and hb heads, rows outermost;
//   head-major [H, T, d]: blocks of hb heads and tb rows, heads outermost.
// Blocks start at multiples of 256 bytes, so a shorter block changes the
// pitch of its own row (or head) of blocks only.
struct RowMap {
  int32_t t = 0, h = 0, head_major = 0;
  int32_t tb = 1, hb = 1;
  FastDiv tdiv, hdiv;
  int64_t row_bytes = 0;  // bytes of one head row
  int64_t outer = 0;      // bytes of a full outermost stretch of blocks
};
#if defined(__HIPCC__)
__device__ __forceinline__ int64_t row_offset(const RowMap& m, int32_t t, int32_t h) {
  const int32_t bt = div_fast(t, m.tdiv), bh = div_fast(h, m.hdiv);
  const int32_t rt = t - bt * m.tb, rh = h - bh * m.hb;
  const int32_t rows = min(m.tb, m.t - bt * m.tb), heads = min(m.hb, m.h - bh * m.hb);
  const int64_t r = m.row_bytes;
  if (m.head_major)
    return bh * m.outer + bt * ((((int64_t)heads * m.tb) * r + 255) & ~(int64_t)255) + ((int64_t)rh * rows + rt) * r;
  return bt * m.outer + bh * ((((int64_t)rows * m.hb) * r + 255) & ~(int64_t)255) + ((int64_t)rt * heads + rh) * r;
}
#endif

// ---- head rows ---------------------------------------------------------------
struct HeadsArgs {
  RowMap x, q, k, v;  // v, k: unused fields where slots is set
  const char* px;
  char *pq, *pk, *pv;
  const char *wq, *wk;       // norm weights or null
  int32_t wq_dt, wk_dt;
  const float* freq;         // rot / 2 frequencies
  const int32_t* pos;        // or null: the row index
  const int32_t* slots;      // or null: k and v are addressed by their maps
  FastDiv page;
  int32_t page_size, n_slots;
  int64_t page_bytes;        // from page to page
  int32_t t, hq, hkv, d, rot, inter;
  float eps;
  int32_t groups_per_wave;   // groups of heads that a wave walks for one row
};
hipError_t launch_heads(const HeadsArgs& a, int32_t dtype, hipStream_t s);

struct HeadsGradArgs {
  RowMap x, q, k, v;         // x and dx share their map
  const char *px, *pdq, *pdk, *pdv;
  char* pdx;
  const char *wq, *wk;
  char *dwq, *dwk;
  int32_t wq_dt, wk_dt, dwq_dt, dwk_dt;
  const float* freq;
  const int32_t* pos;
  float* part;               // [workgroups][2][d] sums of dw
  int32_t t, hq, hkv, d, rot, inter;
  float eps;
  int32_t groups_per_wave, n_wg;
};
constexpr int kHeadsGradMaxWg = 768;
hipError_t launch_heads_grad(const HeadsGradArgs& a, int32_t dtype, hipStream_t s);

// ---- attention over pages ------------------------------------------------------
constexpr int kPagedCols = 16;      // query columns of a matrix tile
constexpr int kPagedStep = 128;     // keys that a workgroup takes at a time
constexpr int kPagedWideStep = 64;  // and with many columns
constexpr int kPaged8Step = 256;    // a cache in 8 bits, few columns

struct PagedSeg {  // what the join needs of a segment
  int32_t r0, r1;       // query rows
  int32_t step, steps;  // first step of its first tile's walk; steps of a walk
  int32_t tile, tiles;  // first tile; tiles of a head
  int32_t group;        // own keys: the sequence's group or -1
  int32_t total, parts; // steps of the pass, and parts they are cut in
};

// One launch of the walk: the groups' shared keys, or the sequences' own.
struct PagedPass {
  int32_t first, n;  // segments
  int32_t shared;    // the groups' pass
  int32_t grid;      // workgroups
  int32_t cols;      // query columns of a tile: 16, 32, 64 or 128
  int32_t fused;     // the walk joins its results itself (no groups)
  int32_t* counters; // fused: arrivals at every tile, zero between calls
  int32_t tiles;     // the most that ascending query rows can have
  float* part_ml;    // [tiles + grid][cols][2]
  float* part_o;     // [tiles + grid][cols][D]
};

struct PagedArgs {
  RowMap q, o;
  const char *pq, *pk, *pv;
  char* po;
  const int32_t *q_start, *len, *table, *group_start, *group_shared;
  int32_t n_seq, n_group, stride, n_pages, page_size, rows, hkv, g;
  FastDiv page, gdiv;
  int64_t page_bytes;
  float scale;       // of the scores, log2 domain
  PagedSeg* seg;     // groups, then sequences
  // a cache in 8 bits: scales [pages][heads][blocks of a page]
  const float *ks, *vs;
  FastDiv block;     // by rows of a scale's block
  int32_t n_blocks;
};
hipError_t launch_paged(const PagedArgs& a, const PagedPass& shared, const PagedPass& own, int32_t d, int32_t dtype,
                        hipStream_t s);
// The same over codes; dtype is that of q and out.
hipError_t launch_paged8_e4m3(const PagedArgs& a, const PagedPass& shared, const PagedPass& own, int32_t d,
                              int32_t dtype, hipStream_t s);
hipError_t launch_paged8_e5m2(const PagedArgs& a, const PagedPass& shared, const PagedPass& own, int32_t d,
                              int32_t dtype, hipStream_t s);
// The join of a call's partial results, where the walk does not do it itself.
hipError_t launch_paged_join(const PagedArgs& a, const PagedPass& shared, const PagedPass& own, int32_t d,
                             int32_t dtype, hipStream_t s);

// ---- a cache in 8 bits ---------------------------------------------------------
constexpr int kScaleExp = 120;  // scales that a write gives are 2^-120 to 2^120

struct Cache8Args {
  RowMap xk, xv;              // rows
  const char *pxk, *pxv;      // read by the write, written by the read
  char *pk, *pv;              // codes
  float *ks, *vs;             // scales [pages][heads][blocks of a page]
  const int32_t *q_start, *len, *table, *slots;
  int32_t n_seq, stride, n_pages, page_size, rows, hkv, d;
  int32_t block_rows, n_blocks;  // rows of a scale's block, blocks of a page
  FastDiv page, block;
  FastDiv pieces, sides;  // by 8-code pieces of a row, by K's and V's heads
  int64_t page_bytes;
};
hipError_t launch_cache8(const Cache8Args& a, int32_t dtype, int32_t code, bool write, hipStream_t s);

// ---- the page table -------------------------------------------------------------
struct PagesArgs {
  int32_t n_seq, stride, n_pages, page_size;
  FastDiv row;  // by stride
  const int32_t *table, *len, *refs;
  int32_t *out_table, *out_len, *out_refs, *status;
  // extend
  const int32_t* add;
  int32_t *slots, *pos;
  int32_t n_tokens;
  // select
  const int32_t* parent;
  int32_t* work;  // workspace behind the counter area
};
constexpr int kPagesMaxCaches = EA_MAX_INPUTS;
struct PagesCache {
  char* data;
  int64_t plane_bytes, page_bytes, row_bytes;  // row: one head's one token
  int32_t planes, heads;
};
struct PagesScales {  // of a cache in 8 bits: [planes][pages][words]
  char* data;
  int64_t plane_bytes;
  int32_t planes, words;         // words of a page: heads times its blocks
  int32_t n_blocks, block_rows;  // blocks of a page, rows of a block
};
struct PagesCopyArgs {
  PagesCache c[kPagesMaxCaches];
  PagesScales s[kPagesMaxCaches];
  int32_t n_cache, n_scales, page_size;
  const int32_t* work;
};
hipError_t launch_pages_extend(const PagesArgs& a, hipStream_t s);
hipError_t launch_pages_select(const PagesArgs& a, const PagesCopyArgs& c, hipStream_t s);
hipError_t launch_pages_compact(const PagesArgs& a, const PagesCopyArgs& c, hipStream_t s);

}  // namespace ea
