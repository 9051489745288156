// How the steps of a batch's walks are dealt to the workgroups of a cached call (a2d_cached_fwd.hpp).
#pragma once
#include "a2d_cache.hpp"

namespace a2d {

// Brings the kernel's arguments into the scalar cache in one go: read line after line as the prologue comes to them, a cold one is half a
// microsecond each time.
__device__ __forceinline__ void warm_cached() {
  constexpr int last = ((int)sizeof(CachedArgs) - 1) / 64;
  static_assert(last <= 5, "lines to touch");
  int v[6];
  asm volatile(
      "s_load_dword %0, %6, 0x0\n\ts_load_dword %1, %6, 0x40\n\ts_load_dword %2, %6, 0x80\n\ts_load_dword %3, %6, 0xc0\n\t"
      "s_load_dword %4, %6, %7\n\ts_load_dword %5, %6, %8\n\ts_waitcnt lgkmcnt(0)"
      : "=&s"(v[0]), "=&s"(v[1]), "=&s"(v[2]), "=&s"(v[3]), "=&s"(v[4]), "=&s"(v[5])
      : "s"(__builtin_amdgcn_kernarg_segment_ptr()), "i"(64 * (last < 4 ? last : 4)), "i"(64 * last));
}

// The walk of a block of rows: steps of 32 keys (`shift` 5; in the form of many rows 64), those of the drafted rows first, which need no table, then
// those of the cached tokens.  Sequence b has kv_heads * blocks such walks of the same length.  All walks, one after another, are a line that is
// cut into equal runs, one for each worker, whatever the lengths are (which the host does not know).  On the line a walk takes start_of() places
// more than its steps: what it costs besides (Q, the table, the first codes, the join of the wavefronts).  With 0 / 8 places a call on 8 sequences,
// one of them of a single token, took 61 / 41 us; with 8 / 16 one on 32 sequences 27.1 / 26.2.
__device__ __forceinline__ unsigned least_of(const CachedArgs& a) { return a.shift == 6 ? 6 : 12; }       // places of a worker
__device__ __forceinline__ unsigned start_of(const CachedArgs& a) { return a.shift == 6 ? 4 : 16; }
__device__ __forceinline__ int steps_for(const CachedArgs& a, int keys) { return (keys + (1 << a.shift) - 1) >> a.shift; }
__device__ __forceinline__ int draft_steps(const CachedArgs& a) { return a.K ? steps_for(a, a.rows) : 0; }
__device__ __forceinline__ int tokens_of(const CachedArgs& a, int length) { return min(max(length, 0), a.max_tokens); }
// (a walk of nothing is one step all the same: its results have to be written)
__device__ __forceinline__ int steps_of(const CachedArgs& a, int tokens) { return max(1, steps_for(a, tokens) + draft_steps(a)); }

// sum over the lanes up to this one
__device__ __forceinline__ unsigned lanes_sum(unsigned x) {
  const auto add = [&](auto C, auto R) {
    x += (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, decltype(C)::value, decltype(R)::value, 0xF, false);
  };
  using std::integral_constant;
  add(integral_constant<int, 0x111>{}, integral_constant<int, 0xF>{});    // within 16 lanes: shifted by 1, 2, 4, 8
  add(integral_constant<int, 0x112>{}, integral_constant<int, 0xF>{});
  add(integral_constant<int, 0x114>{}, integral_constant<int, 0xF>{});
  add(integral_constant<int, 0x118>{}, integral_constant<int, 0xF>{});
  add(integral_constant<int, 0x142>{}, integral_constant<int, 0xA>{});    // the last of 16 lanes to the next 16
  add(integral_constant<int, 0x143>{}, integral_constant<int, 0xC>{});    // lane 31 to the upper half
  return x;
}

// 64 sequences of the batch: a lane's tokens, and the places of the walks of the sequences up to it (behind the last: no more)
struct Batch {
  int first;
  int tokens;
  unsigned sum;
  __device__ __forceinline__ void set(const CachedArgs& a, int from, int lane, int length) {
    first = from;
    const int b = from + lane;
    tokens = b < a.sequences ? tokens_of(a, length) : 0;
    sum = lanes_sum(b < a.sequences ? (steps_of(a, tokens) + start_of(a)) * (unsigned)(a.c.kv_heads * a.blocks) : 0);
  }
  __device__ __forceinline__ void look(const CachedArgs& a, int from, int lane) {
    set(a, from, lane, a.lens[min(from + lane, a.sequences - 1)]);
  }
  __device__ __forceinline__ int tokens_at(int b) const { return __builtin_amdgcn_readlane(tokens, b - first); }
  __device__ __forceinline__ unsigned before(int b) const { return b > first ? (unsigned)__builtin_amdgcn_readlane((int)sum, b - first - 1) : 0; }
  __device__ __forceinline__ unsigned all() const { return (unsigned)__builtin_amdgcn_readlane((int)sum, 63); }
};

// All sequences, 64 at a time, the last ones first; f(batch) for each.  (256 lengths are asked for at once.)
template <class F>
__device__ __forceinline__ void all_batches(const CachedArgs& a, int lane, Batch& batch, F&& f) {
  for (int from = (a.sequences - 1) & ~255; from >= 0; from -= 256) {
    int length[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) length[i] = a.lens[min(from + 64 * i + lane, a.sequences - 1)];
#pragma unroll
    for (int i = 3; i >= 0; --i) {
      if (from + 64 * i >= a.sequences) continue;
      batch.set(a, from + 64 * i, lane, length[i]);
      f();
    }
  }
}

struct Cut {
  unsigned total, each, more;          // places; of a worker; the first `more` workers have one more
  unsigned workers;
  __device__ __forceinline__ void make(const CachedArgs& a, unsigned places) {
    total = places;
    workers = min((unsigned)a.workers, max(1u, total / least_of(a)));
    each = total / workers;
    more = total - each * workers;
  }
  __device__ __forceinline__ unsigned begin(unsigned w) const { return w * each + min(w, more); }
  __device__ __forceinline__ unsigned worker_of(unsigned place) const {
    const unsigned far = more * (each + 1);
    return place < far ? place / (each + 1) : more + (place - far) / each;
  }
};

// What a worker does next: steps s0 .. s1 - 1 of the walk of block `block` of head h of sequence b
struct Run {
  int b, h, block, s0, s1, steps, tokens;
};
// A workgroup's run of the line
struct Runs {
  Batch batch;
  Cut cut;
  int b, unit, worker;
  unsigned at, left;                                 // within the walk; of the run
  unsigned walk0;                                    // the walk's first place on the line
  // false: there is none
  __device__ __forceinline__ bool begin(const CachedArgs& a, int lane) {
    const int per_sequence = a.c.kv_heads * a.blocks;
    worker = -1;
    if (a.workers == 0) {
      b = blockIdx.x / per_sequence;
      unit = blockIdx.x - b * per_sequence;
      batch.look(a, b, lane);
      at = 0;
      left = start_of(a) + steps_of(a, batch.tokens_at(b));
      return true;
    }
    unsigned places = 0;
    all_batches(a, lane, batch, [&] { places += batch.all(); });     // (ends with the first 64)
    cut.make(a, places);
    // neighbours on the line, which share keys where a head has several blocks, to one XCD
    const unsigned per = (cut.workers + 7) / 8, n = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= per || n >= cut.workers) return false;
    worker = (int)n;
    at = walk0 = cut.begin(n);
    left = cut.begin(n + 1) - at;
    while (at >= batch.all() && batch.first + 64 < a.sequences) {
      at -= batch.all();
      batch.look(a, batch.first + 64, lane);
    }
    b = batch.first + __popcll(__ballot(batch.sum <= at));
    at -= batch.before(b);
    const unsigned walk = start_of(a) + steps_of(a, batch.tokens_at(b));
    unit = at / walk;
    at -= unit * walk;
    walk0 -= at;
    return true;
  }
  __device__ __forceinline__ bool next(const CachedArgs& a, int lane, Run& r) {
    if (left == 0) return false;
    if (b >= batch.first + 64) batch.look(a, b, lane);
    const unsigned start = start_of(a);
    r.b = b;
    r.tokens = batch.tokens_at(b);
    r.steps = steps_of(a, r.tokens);
    const mfma::Split sp = mfma::split_by(unit, a.blocks);
    r.h = sp.q;
    r.block = sp.r;
    const unsigned to = min(start + r.steps, at + left);
    r.s0 = at > start ? at - start : 0;
    r.s1 = to > start ? to - start : 0;
    if (worker >= 0 && r.s0 == 0 && r.s1 > 0 && threadIdx.x == 0)      // (every walk has one worker with its first step)
      a.cuts[b * (a.c.kv_heads * a.blocks) + unit] = int2{worker, r.s1 == r.steps ? 1 : (int)cut.worker_of(walk0 + start + r.steps - 1) - worker + 1};
    left -= to - at;
    at = 0;
    walk0 += start + r.steps;
    if (++unit == a.c.kv_heads * a.blocks) {
      unit = 0;
      ++b;
    }
    return r.s1 > 0;                                 // (else the run ends in front of the walk's first step)
  }
};
inline unsigned cached_grid(const CachedArgs& a) {
  return a.workers ? (unsigned)((a.workers + 7) / 8 * 8) : (unsigned)(a.sequences * a.c.kv_heads * a.blocks);
}

// Results that are parts of a block's: m (log2 units), l, N of `rows` = 16 * tiles rows; a worker leaves at most one of a walk that
// began before it (slot 2 w) and one of a walk that goes on behind it (slot 2 w + 1).
__host__ __device__ inline size_t part_floats(int rows, int hdim) { return (size_t)rows * (hdim + 2); }

// Columns 4 quad .. + 3 of row i of query head `head` of sequence b, from N, l relative to m = top (log2 units; l = 0: an empty row).
// A NaN among the row's scores is in l and N, but in no maximum: m is NaN with l, since merges leave out what has m = -inf.
__device__ __forceinline__ void finish(const CachedArgs& a, int b, int head, int i, int hdim, int quad, f32x4 o, float top, float l) {
  constexpr float kLn2 = 0.69314718055994531f;
  const int64_t row = ((int64_t)b * a.heads + head) * a.rows + i;
  if (a.norm) {
    const float inverse = l == 0.f ? 0.f : 1.f / l;
    bf16x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (bf16_t)(o[e] * inverse);
    *reinterpret_cast<bf16x4*>(static_cast<bf16_t*>(a.out0) + at_row(a.lo, b, head, i) + 4 * quad) = y;
    if (quad == 0) a.out1[row] = l == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * kLn2;      // (log2)
  } else {
    *reinterpret_cast<f32x4*>(static_cast<float*>(a.out0) + row * hdim + 4 * quad) = o;
    if (quad == 0) {
      a.out1[row] = l != l ? l : top * kLn2;
      a.out2[row] = l;
    }
  }
}

}  // namespace a2d
