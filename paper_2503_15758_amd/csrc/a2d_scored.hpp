// What the kernels of attention under score rules share (a2d_score_rules in a2d.h): the rules as they take them, the run
// of keys that a query row sees, and their launchers.
#pragma once
#include "a2d_common.hpp"

namespace a2d {

struct ScoreRules {
  float cap;            // 0: none
  int step;
  int heads_per_set;    // query heads of a set of ranges
  int group;            // query heads per key/value head
  int row_shift;        // causal: row i sees the keys k <= i + row_shift = floor((q_off - kv_off) / step) + i
  int acc, norm;        // as in SegList
  int64_t rel, kv_off;  // tokens: of row 0 behind key 0; of key 0
  const float* slopes;
  const int2* ranges;
};

// keys [lo, lo + n) that a row sees; none: n = 0
struct Run {
  int lo, n;
};

__device__ __forceinline__ int64_t floor_div(int64_t a, int b) {
  const int64_t q = a / b;
  return q - (a - q * b < 0);
}

// of row i of query head `head`
__device__ __forceinline__ Run visible_run(const a2d_tile_desc& d, const ScoreRules& r, int head, int i) {
  int lo = 0, hi = d.nkv;
  if (d.causal) {
    const int64_t h = (int64_t)i + r.row_shift + 1;
    hi = h < 0 ? 0 : h < hi ? (int)h : hi;
  }
  if (r.ranges) {
    const int2 t = r.ranges[(int64_t)(head / r.heads_per_set) * d.nq + i];
    int64_t a = (int64_t)t.x - r.kv_off, b = (int64_t)t.y - r.kv_off;      // first key: token >= t.x, so rounded up
    if (r.step != 1) {
      a = -floor_div(-a, r.step);
      b = -floor_div(-b, r.step);
    }
    lo = a < 0 ? 0 : a < d.nkv ? (int)a : d.nkv;
    hi = b < 0 ? 0 : b < hi ? (int)b : hi;
  }
  return Run{lo, hi > lo ? hi - lo : 0};
}

// one row or key in a workgroup, vector ALU (a2d_scored_generic.hip): both types, every shape
hipError_t launch_scored_fwd_generic(const a2d_tile_desc& d, const ScoreRules& r, const void* Q, const void* K, const void* V,
                                     void* out0, float* out1, float* out2, hipStream_t s);
hipError_t launch_scored_bwd_generic(const a2d_tile_desc& d, const ScoreRules& r, const void* Q, const void* K, const void* V,
                                     const void* O, const void* dO, const float* lse, float* delta, void* dQ, void* dK,
                                     void* dV, hipStream_t s);

hipError_t launch_document_ranges(int documents, const int32_t* starts, const int32_t* prefix, int causal, int64_t first, int step,
                                  int rows, int32_t* ranges, hipStream_t s);

// a2d_rotary, its layouts filled in
hipError_t launch_rotary(const a2d_rotary_desc& d, int n, const a2d_rotary_tensor* x, int cus, hipStream_t s);

}  // namespace a2d
