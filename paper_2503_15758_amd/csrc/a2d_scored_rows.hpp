// Query rows and steps as the matrix-unit kernels under score rules take them (a2d_scored_fwd.hip, a2d_scored_bwd.hip, a2d_scored_f32.hip).
#pragma once
#include <limits.h>

#include "a2d_mfma.hpp"
#include "a2d_scored.hpp"

namespace a2d {

// Where the rows of a launch lie: `sub` runs of `rows` query rows for a key/value head, cut into blocks
struct RowMap {
  int sub, rows;         // packed: 1, group * nq; else group, nq
  int by_size;           // blocks in order of size (see xcd_map): BY_ROWS late ones first, the causal mask crosses the tile; BY_RANK
  int parts;
};
enum { BY_ROWS = 1, BY_RANK = 2 };

// Blocks by the length of their walks, longest first, where ranges of tokens say it (of one set, for all heads alike): what the host
// cannot know, every workgroup finds out for itself.  weight[i] of block i (n <= MAX_RANKED) -> order[rank].
constexpr int MAX_RANKED = 512;
struct Ranks {
  int weight[MAX_RANKED];
  unsigned short order[MAX_RANKED];
};
__device__ __forceinline__ void rank_blocks(Ranks& r, int n, int threads) {
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += threads) {
    const int w = r.weight[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += r.weight[j] > w || (r.weight[j] == w && j > i);
    r.order[rank] = (unsigned short)i;
  }
  __syncthreads();
}
// of bm query rows each: by the steps of 64 keys in the hull of a block's first and last row
__device__ __forceinline__ void weigh_rows(Ranks& ranks, const a2d_tile_desc& d, const ScoreRules& r, int rows, int bm, int threads) {
  const int n = (rows + bm - 1) / bm;
  for (int i = threadIdx.x; i < n; i += threads) {
    const Run a = visible_run(d, r, 0, i * bm), b = visible_run(d, r, 0, min((i + 1) * bm, rows) - 1);
    const int lo = min(a.n ? a.lo : INT_MAX, b.n ? b.lo : INT_MAX), hi = max(a.lo + a.n, b.lo + b.n);
    ranks.weight[i] = lo < hi ? (hi - lo + 63) / 64 : 0;
  }
}
__device__ __forceinline__ void rank_rows(Ranks& ranks, const a2d_tile_desc& d, const ScoreRules& r, int rows, int bm, int threads) {
  weigh_rows(ranks, d, r, rows, bm, threads);
  rank_blocks(ranks, (rows + bm - 1) / bm, threads);
}

// How the blocks of a head (row blocks of dQ, key blocks of dK / dV) are cut into units, a workgroup each: uniform, every block into
// `parts`; or (parts = 0) in proportion to the blocks' walks, which again the workgroups find out for themselves: a causal mask
// and documents leave walks of any length, and what an even cut of them costs is the traffic of the short ones' partials.
struct Cut {
  int blocks, units;     // a head; units: at most, where they are shared out
  int parts;             // 0: shared out
  int least;             // weight of the smallest unit that is worth its partial (shared out)
};
// a unit: one of the `parts` of a block, whose partials stand from `slot` on (of the head's)
struct Share {
  int block, part, parts, slot;
};
struct Shares {
  Ranks ranks;
  int each[8], wave[8];
  Share mine;
};
// Unit u where they are shared out: a unit takes `each` of the blocks' weights at most, blocks of at least one unit, the heaviest blocks'
// units first; the least `each` of eight, a wavefront each, that makes no more than cut.units of them.  They lie between W / units, which no
// cut can undercut, and W / (units - blocks) + 1, which always does: sum_b max(1, ceil(w_b / each)) < W / each + blocks.
// parts = 0: there are fewer units.  ranks.weight is set; 512 threads, cut.blocks <= MAX_RANKED
__device__ __forceinline__ Share share_out(Shares& s, const Cut& cut, int u) {
  const int i = threadIdx.x, n = cut.blocks, lane = i & 63;
  const auto units = [](int w, int each) { return max(1, (int)(((unsigned)w + each - 1) / (unsigned)each)); };
  const auto sum = [](int x) {
#pragma unroll
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o, 64);
    return x;
  };
  __syncthreads();
  int each = INT_MAX;
  if (cut.units > n) {
    int total = 0, made = 0;
    for (int b = lane; b < n; b += 64) total += s.ranks.weight[b];
    total = sum(total);
    const int lo = total / cut.units, hi = total / (cut.units - n) + 1;
    each = max(cut.least, lo + (int)((int64_t)(hi - lo) * ((i >> 6) + 1) / 8));
    for (int b = lane; b < n; b += 64) made += units(s.ranks.weight[b], each);
    if (sum(made) > cut.units) each = INT_MAX;
  }
  if (lane == 0) s.each[i >> 6] = each;
  if (i == 0) s.mine = Share{0, 0, 0, 0};
  rank_blocks(s.ranks, n, 512);
#pragma unroll
  for (int x = 0; x < 8; ++x) each = min(each, s.each[x]);
  const int block = i < n ? s.ranks.order[i] : 0;
  const int parts = i < n ? units(s.ranks.weight[block], each) : 0;
  int upto = parts;                                  // of this rank and those before it
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(upto, o, 64);
    if (lane >= o) upto += x;
  }
  if (lane == 63) s.wave[i >> 6] = upto;
  __syncthreads();
  for (int x = 0; x < i >> 6; ++x) upto += s.wave[x];
  if (u < upto && u >= upto - parts) s.mine = Share{block, u - (upto - parts), parts, upto - parts};
  __syncthreads();
  return Share{__builtin_amdgcn_readfirstlane(s.mine.block), __builtin_amdgcn_readfirstlane(s.mine.part),
               __builtin_amdgcn_readfirstlane(s.mine.parts), __builtin_amdgcn_readfirstlane(s.mine.slot)};
}
// the same where every block is cut alike; the last block first
__device__ __forceinline__ Share share_evenly(const Cut& cut, int u, bool last_first) {
  const mfma::Split at = mfma::split_by(u, cut.parts);
  const int block = last_first ? cut.blocks - 1 - at.q : at.q;
  return Share{block, at.r, cut.parts, block * cut.parts};
}

// what a wavefront knows of its NT tiles of 16 rows; of the lane's row in each
template <int NT>
struct RowState {
  int64_t q_at[NT];       // its place in Q, from the key/value head's first
  Run run[NT];
  float at[NT], slope[NT]; // tokens behind key 0; slope in log2 units
  int lo, hi;            // hull of the wavefront's runs; lo > hi: nothing seen
  int all_lo, all_hi;    // keys that all of its rows see
  int nearest, farthest; // `at` of its rows, the least and the most
};

// (exact: a power of two)
__device__ __forceinline__ void lift(bf16x8& v, float by) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (bf16_t)((float)v[e] * by);
}

// min or max over the 16 lanes of a lane's tile (every 16 lanes hold the same rows)
template <class F>
__device__ __forceinline__ int over16(int x, F&& f) {
#pragma unroll
  for (int o = 8; o; o >>= 1) x = f(x, __shfl_xor(x, o, 64));
  return __builtin_amdgcn_readfirstlane(x);
}

// rows w0 .. w0 + 16 NT - 1 of the run of map.rows rows that starts at row 0 of query head `head`
template <int NT, bool BIAS>
__device__ __forceinline__ void look_up_rows(RowState<NT>& rs, const a2d_tile_desc& d, const ScoreRules& r, const RowMap& map, int head, int w0,
                                             int lane) {
  const auto least = [](int a, int b) { return min(a, b); };
  const auto most = [](int a, int b) { return max(a, b); };
  int lo = INT_MAX, hi = 0, all_lo = 0, all_hi = INT_MAX, nearest = INT_MAX, farthest = INT_MIN;
#pragma unroll
  for (int q = 0; q < NT; ++q) {
    const int row = w0 + 16 * q + (lane & 15), in = min(row, map.rows - 1);
    const mfma::Split hd = map.sub == 1 ? mfma::Split{in / d.nq, in - in / d.nq * d.nq} : mfma::Split{0, in};
    rs.q_at[q] = hd.q * d.lq.head + hd.r * d.lq.row;
    rs.run[q] = visible_run(d, r, head + hd.q, hd.r);
    if constexpr (BIAS) {
      const int at = (int)(r.rel + (int64_t)hd.r * r.step);
      rs.at[q] = (float)at;
      nearest = min(nearest, at);
      farthest = max(farthest, at);
      rs.slope[q] = r.slopes[head + hd.q] * kLog2e;
    }
    if (row >= map.rows) rs.run[q] = Run{0, 0};                // (never stored; asks for nothing)
    if (rs.run[q].n > 0) {
      lo = min(lo, rs.run[q].lo);
      hi = max(hi, rs.run[q].lo + rs.run[q].n);
    }
    if (row < map.rows) {
      all_lo = max(all_lo, rs.run[q].lo);
      all_hi = min(all_hi, rs.run[q].lo + rs.run[q].n);
    }
  }
  rs.lo = over16(lo, least);
  rs.hi = over16(hi, most);
  rs.all_lo = over16(all_lo, most);
  rs.all_hi = over16(all_hi, least);
  rs.nearest = BIAS ? over16(nearest, least) : 0;
  rs.farthest = BIAS ? over16(farthest, most) : 0;
}

// how the blocks of a tile are ordered, of which there are n a head
inline int blocks_by_size(const a2d_tile_desc& d, const ScoreRules& r, int n) {
  if (r.ranges) return r.heads_per_set == d.heads && n > 1 && n <= MAX_RANKED ? BY_RANK : 0;
  return d.causal && r.row_shift < d.nkv && (int64_t)d.nq + r.row_shift > 0 && d.nq > 1 ? BY_ROWS : 0;
}
// for workgroups of bm rows
inline RowMap row_map(const a2d_tile_desc& d, const ScoreRules& r, int bm, int parts) {
  const bool packed = r.group > 1 && d.nq < bm;
  return RowMap{packed ? 1 : r.group, packed ? r.group * d.nq : d.nq, packed ? 0 : blocks_by_size(d, r, (d.nq + bm - 1) / bm), parts};
}

// what the dQ kernel leaves of the rows, [heads][padded]: padded = nq up to the next multiple of 64
struct RowTile {
  int lo, hi;            // hull of the runs (none: lo > hi)
  int all_lo, all_hi;    // keys that all rows see that see any
  unsigned live;         // bit i: row i sees something
  int pad[3];
};
struct RowTable {
  int padded;
  float *from, *delta;   // bf16: lse in log2 units, with a cap; without one -lse in units of raw products: what the scores start from; fp32: lse.  -(dO . O)
  int *lo, *n;           // run of keys
  RowTile* tiles;        // [heads][padded / 32]
};

// (of one tile's rows and keys: the table in `ws`, see scored_bwd_bytes)
inline RowTable row_table(const a2d_tile_desc& d, void* ws) {
  RowTable t;
  t.padded = (d.nq + 63) / 64 * 64;
  const int64_t n = (int64_t)d.heads * t.padded;
  t.from = static_cast<float*>(ws);
  t.delta = t.from + n;
  t.lo = reinterpret_cast<int*>(t.delta + n);
  t.n = t.lo + n;
  t.tiles = reinterpret_cast<RowTile*>(t.n + n);
  return t;
}

// The set bits of a map in LDS, one after another, by all lanes of a wavefront alike
struct StepWalk {
  const uint64_t* bits;
  int words, at;
  uint64_t left;
  __device__ __forceinline__ uint64_t word(int w) const {
    const uint64_t b = bits[w];
    return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(b >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)b);
  }
  __device__ __forceinline__ int open(const uint64_t* map, int n) {     // returns how many there are; n >= 1
    bits = map;
    words = n;
    at = 0;
    int total = 0;
    for (int w = 0; w < n; ++w) total += __builtin_popcountll(word(w));
    left = word(0);
    return total;
  }
  __device__ __forceinline__ void skip(int n) {                         // fewer than are left, or all
    while (n > 0) {
      const int here = __builtin_popcountll(left);
      if (here <= n) {
        n -= here;
        left = 0;
        if (++at >= words) { at = words - 1; return; }
        left = word(at);
      } else {
        for (; n > 0; --n) left &= left - 1;
      }
    }
  }
  __device__ __forceinline__ int next() {                               // there is one left
    while (left == 0 && at + 1 < words) left = word(++at);
    const int s = 64 * at + __builtin_ctzll(left);
    left &= left - 1;
    return s;
  }
};

}  // namespace a2d
