// What the kernels of attention under score rules share (a2d_score_rules in a2d.h): the rules as they take them, the run
// of keys that a query row sees, and their launchers.
#pragma once
#include "a2d_common.hpp"
#include "a2d_grid.hpp"

namespace a2d {

// The cap in log2 units, y = cap log2(e) tanh(scale z / cap) of a raw dot product z: up to |z| = small (half of cap / scale) an odd polynomial
// z (c0 + .. + c3 z^6), fitted to tanh with 5e-7 of it; beyond, top (1 - 2 / (1 + 2^(rate z))), whose error, some 2^-22 of top, is relative to
// a y of 0.46 top and more.  (That form alone would be off by 2^-22 of the cap everywhere: as much as y itself for a wide cap.)
// fine: one coefficient more (1e-8 and the roundings), for fp32 inputs.
// lift: a power of two that the kernels' Q (dK / dV: K) comes multiplied with, where the coefficients, up to (scale / cap)^9, or z^2 would leave
// fp32's range otherwise (a scale of 1e-8 under a cap of 30); all of these are of that z then.  1: as it is.
struct CapArgs {
  float small, rate, top, c[4], fine[5], lift;
};
struct ScoreRules {
  float cap;            // 0: none
  CapArgs capped;
  int step;
  int heads_per_set;    // query heads of a set of ranges
  int group;            // query heads per key/value head
  int row_shift;        // causal: row i sees the keys k <= i + row_shift = floor((q_off - kv_off) / step) + i
  int acc, norm;        // as in SegList
  int64_t rel, kv_off;  // tokens: of row 0 behind key 0; of key 0
  float steps[6];       // step times 1, 2, 3, 16, 32, 48: between the scores that a lane holds
  float all_steps[16];  // step times 16 (e / 4) + e % 4: of score e behind a lane's first
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

// Distance of score i of tile t (16 rows or keys each) of a lane whose first one is `first` tokens off: each of its additions takes
// its step from a scalar register (as a multiply-add by a constant it needs a vector register for each constant).
template <int SIGN>
__device__ __forceinline__ float distance(const ScoreRules& r, float first, int t, int i) {
  const float f = t == 0 ? first : SIGN > 0 ? first + r.steps[2 + t] : first - r.steps[2 + t];
  return i == 0 ? f : SIGN > 0 ? f + r.steps[i - 1] : f - r.steps[i - 1];
}

// z -> (factor of z: y = z * factor), for |z| <= small
__device__ __forceinline__ float cap_factor(const CapArgs& a, float z) {
  const float u = z * z;
  return fmaf(u, fmaf(u, fmaf(u, a.c[3], a.c[2]), a.c[1]), a.c[0]);
}
__device__ __forceinline__ float cap_beyond(const CapArgs& a, float z) {
  return a.top * fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + fast_exp2(z * a.rate)), 1.f);
}
// any z (NaN: beyond, which is NaN too)
__device__ __forceinline__ float cap_log2(const CapArgs& a, float z) {
  return fabsf(z) <= a.small ? z * cap_factor(a, z) : cap_beyond(a, z);
}
__device__ __forceinline__ float cap_log2_f32(const CapArgs& a, float z) {
  const float u = z * z;
  const float y = z * fmaf(u, fmaf(u, fmaf(u, fmaf(u, a.fine[4], a.fine[3]), a.fine[2]), a.fine[1]), a.fine[0]);
  return fabsf(z) <= a.small ? y : cap_beyond(a, z);
}

// Ranges that the host cannot see: one set for all heads is taken for documents, which see a part of the keys each, where a head's rows are
// more than a workgroup's.  Fewer (new tokens against a cache) lie in one document or two, and the set may as well be a cache's
// filled length, which they see all of.  One sequence's 16384 keys, heads of 128, planned for all of them and for documents: 100 rows of 32 / 8
// heads 41 us and 63, their gradients 127 and 142; those of a token of 8 heads 56 and 429.
inline bool taken_for_documents(const a2d_tile_desc& d, const ScoreRules& r) { return r.ranges && r.heads_per_set == d.heads && d.nq > 128; }

// keys of a row's walk, on average and at most, as far as sizes and the causal mask tell
struct WalkKeys {
  double mean, most;
};
inline WalkKeys walk_keys(const a2d_tile_desc& d, const ScoreRules& r) {
  if (!d.causal) return WalkKeys{(double)d.nkv, (double)d.nkv};
  const auto seen = [&](double x) { return x < 0 ? 0.0 : x > d.nkv ? (double)d.nkv : x; };
  const double most = seen((double)d.nq + r.row_shift);
  return WalkKeys{0.5 * (seen(1.0 + r.row_shift) + most), most};
}

// bf16 forward on the matrix units (a2d_scored_fwd.hip).  How a call goes out: the form of its workgroups, and how many
// share a walk of the keys (their partials [parts][heads][nq] in place of the outputs, to be merged): `cap` at most, one without `scratch`.
struct ScoredPlan {
  int form, parts;
  bool fine;             // 32 rows: P as two bf16 numbers
};
enum { SCORED_256, SCORED_LANES, SCORED_PAIRS, SCORED_32 };   // 256 rows; 128 rows in two key lanes; 128 rows in four wavefronts, two
                                                              // workgroups a compute unit; 32 rows in eight key lanes
ScoredPlan plan_scored_fwd(const a2d_tile_desc& d, const ScoreRules& r, int cus, int cap, bool scratch);
hipError_t launch_scored_fwd(Phase ph, const a2d_tile_desc& d, const ScoreRules& r, const ScoredPlan& plan, const void* Q, const void* K,
                             const void* V, float* out0, float* out1, float* out2, const FwdInput& in, hipStream_t s);

// bf16 backward (a2d_scored_bwd.hip).  ws: scored_bwd_bytes(d); more: scored_bwd_scratch(...) bytes for the fp32 partials of blocks that
// workgroups share.  r.norm writes bf16, r.acc adds to dQ.
struct ScoredBwdPlan {
  int lanes;             // key lanes of a dQ workgroup (1: 256 rows, 2: 128)
  int q, kv;             // fp32: workgroups that share a walk; bf16: workgroups of a query head for dQ, of a key/value head for dK / dV
  bool share_q, share_kv;  // bf16: shared out in proportion to the blocks' walks (Cut in a2d_scored_rows.hpp); else evenly
};
constexpr int SCORED_MOST_BITS = 16384;              // bytes: a bit a step of 64 rows of each query head of a group, group * nq <= 2^22
size_t scored_bwd_bytes(const a2d_tile_desc& d);
ScoredBwdPlan plan_scored_bwd(const a2d_tile_desc& d, const ScoreRules& r, int cus, size_t most_bytes);  // most_bytes: of a result's partials
size_t scored_bwd_scratch(const a2d_tile_desc& d, const ScoreRules& r, const ScoredBwdPlan& plan);
hipError_t launch_scored_bwd(Phase ph, const a2d_tile_desc& d, const ScoreRules& r, const ScoredBwdPlan& plan, const void* Q, const void* K,
                             const void* V, const void* O, const void* dO, const float* lse, void* ws, void* more, void* dQ, void* dK,
                             void* dV, hipStream_t s);

// what a call's plan makes of it (kernels and launches of these files alone)
void route_scored_fwd(const a2d_tile_desc& d, const ScoreRules& r, const ScoredPlan& plan, ScoredRoute* out);
void route_scored_bwd(const a2d_tile_desc& d, const ScoreRules& r, const ScoredBwdPlan& plan, ScoredRoute* out);
void route_scored_fwd_f32(const a2d_tile_desc& d, const ScoreRules& r, const ScoredPlan& plan, ScoredRoute* out);
void route_scored_bwd_f32(const a2d_tile_desc& d, const ScoreRules& r, const ScoredBwdPlan& plan, ScoredRoute* out);

// the same for fp32 (a2d_scored_f32.hip; plan.form: 1 or 2 tiles of 16 rows a workgroup)
ScoredPlan plan_scored_fwd_f32(const a2d_tile_desc& d, const ScoreRules& r, int cus, int cap);
hipError_t launch_scored_fwd_f32(Phase ph, const a2d_tile_desc& d, const ScoreRules& r, const ScoredPlan& plan, const void* Q, const void* K,
                                 const void* V, float* out0, float* out1, float* out2, const FwdInput& in, hipStream_t s);
ScoredBwdPlan plan_scored_bwd_f32(const a2d_tile_desc& d, const ScoreRules& r, int cus, int cap_q, int cap_kv);
hipError_t launch_scored_bwd_f32(Phase ph, const a2d_tile_desc& d, const ScoreRules& r, const ScoredBwdPlan& plan, const void* Q,
                                 const void* K, const void* V, const void* O, const void* dO, const float* lse, void* ws, float* dQ,
                                 float* dK, float* dV, hipStream_t s);

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
