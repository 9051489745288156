// How the steps of a batch's walks are dealt to the workgroups of a cached call (a2d_cached_fwd.hpp), found alike by the workgroups
// that walk and by those that merge.
#pragma once
#include "a2d_cache.hpp"

namespace a2d {

// The walk of a block of rows: steps of 32 keys, those of the cached tokens first, then those of the drafted rows.  Sequence b has
// kv_heads * blocks such walks of the same length; all walks, one after another, are a line of steps, cut into equal runs, one for each
// worker, whatever the lengths are (which the host does not know).
constexpr int STEP = 32;
__device__ __forceinline__ int cached_tokens(const CachedArgs& a, int b) { return min(max(a.lens[b], 0), a.max_tokens); }
__device__ __forceinline__ int draft_steps(const CachedArgs& a) { return a.K ? (a.rows + STEP - 1) / STEP : 0; }
// (a walk of nothing is one step all the same: its results have to be written)
__device__ __forceinline__ int walk_steps(const CachedArgs& a, int b) {
  return max(1, (cached_tokens(a, b) + STEP - 1) / STEP + draft_steps(a));
}

// sum over the lanes up to this one
__device__ __forceinline__ unsigned lanes_sum(unsigned x, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const unsigned y = __shfl_up(x, d);
    x += lane >= d ? y : 0;
  }
  return x;
}

struct Cut {
  unsigned total, each, more;          // steps; of a worker; the first `more` workers have one more
  unsigned workers;
  __device__ __forceinline__ unsigned begin(unsigned w) const { return w * each + min(w, more); }
  __device__ __forceinline__ unsigned worker_of(unsigned step) const {
    const unsigned far = more * (each + 1);
    return step < far ? step / (each + 1) : more + (step - far) / each;
  }
};

constexpr unsigned LEAST_STEPS = 8;    // of a worker: two for each wavefront

// steps of all walks of sequences first .. first + 63, the lane's and those in front of it; 0 behind the last
__device__ __forceinline__ unsigned sequence_sum(const CachedArgs& a, int first, int lane) {
  const int b = first + lane;
  return lanes_sum(b < a.sequences ? (unsigned)walk_steps(a, b) * (unsigned)(a.c.kv_heads * a.blocks) : 0, lane);
}
// (before: steps of the sequences in front of b)
__device__ __forceinline__ Cut make_cut(const CachedArgs& a, int lane, int b = 0, unsigned* before = nullptr) {
  Cut c;
  c.total = 0;
  for (int first = 0; first < a.sequences; first += 64) {
    const unsigned sum = sequence_sum(a, first, lane);
    if (before && b >= first && b < first + 64) *before = c.total + (b > first ? (unsigned)__builtin_amdgcn_readlane((int)sum, b - first - 1) : 0);
    c.total += (unsigned)__builtin_amdgcn_readlane((int)sum, 63);
  }
  c.workers = min((unsigned)a.workers, max(1u, c.total / LEAST_STEPS));
  c.each = c.total / c.workers;
  c.more = c.total - c.each * c.workers;
  return c;
}

// Results that are parts of a block's: m (log2 units), l, N of `rows` = 16 * tiles rows; a worker leaves at most one of a walk that
// began before it (slot 2 w) and one of a walk that goes on behind it (slot 2 w + 1).
__host__ __device__ inline size_t part_floats(int rows, int hdim) { return (size_t)rows * (hdim + 2); }

// Columns 4 quad .. + 3 of row i of query head `head` of sequence b, from N, l relative to m = top (log2 units; l = 0: an empty row)
__device__ __forceinline__ void finish(const CachedArgs& a, int b, int head, int i, int hdim, int quad, f32x4 o, float top, float l) {
  constexpr float kLn2 = 0.69314718055994531f;
  const int64_t row = ((int64_t)b * a.heads + head) * a.rows + i;
  if (a.norm) {
    const float inverse = l == 0.f ? 0.f : 1.f / l;
    bf16x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (bf16_t)(o[e] * inverse);
    *reinterpret_cast<bf16x4*>(static_cast<bf16_t*>(a.out0) + at_row(a.lo, b, head, i) + 4 * quad) = y;
    if (quad == 0) a.out1[row] = l == 0.f ? -INFINITY : fmaf(top, kLn2, logf(l));
  } else {
    *reinterpret_cast<f32x4*>(static_cast<float*>(a.out0) + row * hdim + 4 * quad) = o;
    if (quad == 0) {
      a.out1[row] = top * kLn2;
      a.out2[row] = l;
    }
  }
}

}  // namespace a2d
