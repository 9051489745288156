// What the kernels of the paged cache share (a2d_cache in a2d.h): the formats, where a token's rows lie, and their launchers.
#pragma once
#include "a2d_mfma.hpp"

namespace a2d {

// Bytes of n values (a multiple of 8) in a format
template <int FMT>
__host__ __device__ constexpr int code_bytes(int n) {
  return FMT == A2D_CACHE_BF16 ? 2 * n : FMT == A2D_CACHE_E4M3 ? n : n / 2;
}
constexpr int CACHE_BLOCK = 32;       // values that share a scale
constexpr int CACHE_LOWEST = -100;    // smallest exponent of a scale: what it stands for is a normal bf16 number

// A scale byte as a number: 2^(byte - 127).  255, the mark of a block with a NaN or an infinity, as the conversions' scale makes NaN of every code.
__device__ __forceinline__ float scale_number(unsigned byte) { return __builtin_bit_cast(float, byte << 23); }

// Codes times their scale as bf16 numbers, which hold them exactly (e4m3: 3 bits behind the point, e2m1: 1).
template <int FMT>
__device__ __forceinline__ bf16x8 decode8(unsigned w0, unsigned w1, float scale);
template <>
__device__ __forceinline__ bf16x8 decode8<A2D_CACHE_E4M3>(unsigned w0, unsigned w1, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
template <>
__device__ __forceinline__ bf16x8 decode8<A2D_CACHE_E2M1>(unsigned w, unsigned, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The cache as kernels take it.  Rows are counted in units of 16, which never cross a page: unit (page * kv_heads + head) * page_units + n.
struct CacheView {
  char *K, *V;
  char *Ks, *Vs;               // 4 bytes a row
  const int32_t* table;
  int kv_heads, page_units, pages, max_pages;
  unsigned inverse;            // floor((2^32 - 1) / page_units)
};
constexpr unsigned NO_UNIT = 0xFFFFFFFFu;
// The place of tile `tile` (16 tokens) of sequence b in the table and in its page; the page's number is then asked for, and unit() takes it.
// (Two steps without a branch, so that other requests can go out in between.)
struct Place {
  int page, rest;              // the table's entry; -1: there is none
  __device__ __forceinline__ void ask(const CacheView& c, int b, int tile, bool wanted = true) {
    int at = (int)__umulhi((unsigned)tile, c.inverse);             // (one too few at the most)
    rest = tile - at * c.page_units;
    if (rest >= c.page_units) {
      ++at;
      rest -= c.page_units;
    }
    const bool there = wanted && (unsigned)at < (unsigned)c.max_pages && tile >= 0;
    const int entry = c.table[(int64_t)b * c.max_pages + (there ? at : 0)];
    rest = there ? rest : -1;
    page = entry;
  }
  // of head h; NO_UNIT where the table names no page of the cache
  __device__ __forceinline__ unsigned unit(const CacheView& c, int h) const {
    return rest >= 0 && (unsigned)page < (unsigned)c.pages ? ((unsigned)page * c.kv_heads + h) * c.page_units + rest : NO_UNIT;
  }
};
__device__ __forceinline__ unsigned unit_of(const CacheView& c, int b, int h, int tile) {
  Place p;
  p.ask(c, b, tile);
  return p.unit(c, h);
}

struct BatchLayout {           // elements between sequences, heads, rows
  int64_t sequence, head, row;
};
__host__ __device__ inline int64_t at_row(const BatchLayout& l, int64_t b, int64_t h, int64_t i) {
  return b * l.sequence + h * l.head + i * l.row;
}

struct CacheRows {             // of a write or a read
  CacheView c;
  int sequences, rows, count;  // rows of K and V; of these written for each sequence (read: the same)
  int first;                   // read
  const int32_t *starts, *index;   // write: starts, read: lens
  const char *K, *V;
  BatchLayout lk, lv;
};
hipError_t launch_cache_write(int format, int hdim, int dtype, const CacheRows& a, hipStream_t s);
hipError_t launch_cache_read(int format, int hdim, int dtype, const CacheRows& a, hipStream_t s);
hipError_t launch_tree_masks(int sequences, int rows, const int32_t* parents, const int32_t* lens, uint64_t* masks, int32_t* positions,
                             hipStream_t s);

// Attention of rows against the cache and the drafted rows beside it (a2d_cached_fwd.hpp).
struct CachedArgs {
  CacheView c;
  int sequences, heads, group, rows;   // group: query heads of a key/value head
  int max_tokens, words, norm;         // words: of a row's mask
  float c2;                            // scale log2(e)
  const int32_t* lens;
  const uint64_t* masks;
  const char *Q, *K, *V;               // K, V: drafted rows, or NULL
  BatchLayout lq, lk, lv, lo;
  void* out0;
  float *out1, *out2;
  // how the call goes out (plan_cached)
  int blocks;                          // row blocks of a key/value head, `tiles` tiles of 16 rows each
  int tiles, shift;                    // a step has 2^shift keys
  int workers;                         // workgroups that share all steps; 0: one for each block
  float* parts;                        // two results of a block for each worker
  int2* cuts;                          // of each walk: the first worker that has steps of it, and how many have
};
struct CachedPlan {
  int tiles, shift, blocks, workers;
  size_t part_bytes, bytes;            // of a.parts; with a.cuts behind them
};
constexpr int64_t MAX_THREADS = (int64_t)1 << 32;      // a launch has fewer
inline int cached_threads(int tiles) { return 64 * (tiles == 16 ? 8 : 4); }       // of a workgroup
// workspace: whether there may be one
CachedPlan plan_cached(int format, int hdim, const CachedArgs& a, int cus, bool workspace);
hipError_t launch_cached(Phase ph, int format, int hdim, const CachedArgs& a, hipStream_t s);
hipError_t launch_cached_generic(int format, int hdim, const CachedArgs& a, hipStream_t s);
// the kernels of one format (a translation unit each)
hipError_t launch_cached_bf16(Phase ph, int hdim, const CachedArgs& a, hipStream_t s);
hipError_t launch_cached_e4m3(Phase ph, int hdim, const CachedArgs& a, hipStream_t s);
hipError_t launch_cached_e2m1(Phase ph, int hdim, const CachedArgs& a, hipStream_t s);

}  // namespace a2d
