// fp32 tiles under score rules (a2d_score_rules in a2d.h) on the fp32 matrix units, H = 128, 96, 80 and 64: fp32 throughout.
//
// Tiles of 16 rows in LDS of a wavefront's own, fragments, contractions and the merge of the four key lanes as in
// a2d_f32_mfma.hip; masks, hulls and the row table as in a2d_scored_fwd.hip and a2d_scored_bwd.hip.  A step of 16 x 16 scores is
// H / 4 matrix instructions of 32 cycles for each contraction and four scores a lane, so the rules are branches of the one kernel that all
// lanes take alike: their few vector instructions a score are a small part of a step.  Scores are kept in log2 units.  In the backward a bias
// and lse, which may be thousands where their difference is a few units, meet in natural units in one multiply-add, rounded once.
//
// Bound by the fp32 matrix rate where there are many rows, by the chip's idle units, first loads and launches where there are few: backward of
// 8 heads of 96, 700 x 900, causal, 78 us (matrix units busy 30 % of the time, one wavefront a SIMD); forward of 2 x 128 x 128 7 us.
#include "a2d_f32.hpp"
#include "a2d_scored_rows.hpp"

namespace a2d {
namespace {

using namespace f32;
using mfma::row_max;
using mfma::row_sum;
using mfma::uniform_gptr;
using mfma::xcd_grid;
using mfma::xcd_map;

// log2 units of four raw products of a lane, the score i of which is `far` + (a row, -1 a key) i steps off; slope in log2 units
template <int SIGN>
__device__ __forceinline__ void to_scores(f32x4& s, const ScoreRules& r, float raw, float slope, float far) {
  if (r.cap != 0.f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = cap_log2_f32(r.capped, s[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] *= raw;
  }
  if (r.slopes) {
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = fmaf(-slope, fabsf(distance<SIGN>(r, far, 0, i)), s[i]);
  }
}

// rows of a query head's Q: as Nat<H>::load, at byte `off`
template <int H>
__device__ __forceinline__ void load_at(Nat<H>& x, gptr_t base, unsigned off, int g4) {
#pragma unroll
  for (int y = 0; y < H / 16; ++y) x.v[y] = gload<f32x4>(base, off + 16 * g4 + 64 * y);
}

// (see CapArgs)
template <int H>
__device__ __forceinline__ void lift(Nat<H>& x, const ScoreRules& r) {
  if (r.cap != 0.f && A2D_SELDOM(r.capped.lift != 1.f)) {
#pragma unroll
    for (int y = 0; y < H / 16; ++y) x.v[y] *= r.capped.lift;
  }
}

// ------------------------------------------------------------------------------------------- forward
// 16 RT rows a workgroup of four key lanes, 16 keys a step (as fwd_f32_kernel)
// (out0, out1, out2 are not __restrict__: an accumulating call's `in` is the same memory)
template <int H, int RT>
__global__ __launch_bounds__(64 * KL, 2) void scored_fwd_f32_kernel(
    a2d_tile_desc d, ScoreRules r, RowMap map, const float* __restrict__ Q, const float* __restrict__ K,
    const float* __restrict__ V, float* out0, float* out1, float* out2, FwdInput in) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  constexpr int BM = BLK * RT;
  const int nqb = (map.rows + BM - 1) / BM;
  int unit, blk;
  if (!xcd_map(blockIdx.x, d.heads / r.group * map.parts, map.sub * nqb, map.by_size != 0, unit, blk)) return;
  const mfma::Split up = mfma::split_by(unit, map.parts), in_group = mfma::query_head(blk, map.sub, nqb, map.by_size != 0);
  const int kvh = up.q, part = up.r, head = kvh * r.group + in_group.r, q0 = (nqb - 1 - in_group.q) * BM;
  const int kl = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int l15 = lane & 15, g4 = lane >> 4;
  const gptr_t kb = uniform_gptr(K + (int64_t)kvh * d.lk.head), vb = uniform_gptr(V + (int64_t)kvh * d.lv.head);
  const gptr_t qb = uniform_gptr(Q + (int64_t)head * d.lq.head);
  const unsigned k_row = (unsigned)d.lk.row * 4, v_row = (unsigned)d.lv.row * 4;
  const float raw = d.scale * kLog2e;
  const int64_t row0 = (int64_t)head * d.nq;

  RowState<RT> rs;
  if (r.slopes) look_up_rows<RT, true>(rs, d, r, map, head, q0, lane);
  else look_up_rows<RT, false>(rs, d, r, map, head, q0, lane);
  Nat<H> qf[RT];
  Out<H> o[RT];
  float m_lane[RT], m_ref[RT], l_run[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    load_at<H>(qf[t], qb, (unsigned)rs.q_at[t] * 4, g4);
    lift(qf[t], r);
    o[t].zero();
    m_lane[t] = -INFINITY;
    l_run[t] = 0.f;
    const int row = q0 + BLK * t + l15;
    if (r.acc && kl == 0 && part == 0 && row < map.rows) {      // continue from the triple given
      o[t].load(in.N + (row0 + row) * H, g4);
      m_lane[t] = in.m[row0 + row] * kLog2e;       // -inf stays -inf
      l_run[t] = g4 == 0 ? in.l[row0 + row] : 0.f;
    }
    m_ref[t] = m_lane[t];
  }
  const int lo = rs.lo, hi = rs.hi, end = hi > lo ? (hi + BLK - 1) / BLK : 0, lanes = KL * map.parts;
  int j = (hi > lo ? lo / BLK : 0) + part * KL + kl;

  // K through LDS, the next block's as soon as the scores are there; V by columns into registers, the next block's as soon as the
  // products are through.  Keys outside the hull: its first or last.
  Blocks<H> kt;
  kt.init((lds_t)smem + kl * Blocks<H>::BYTES, l15, g4);
  Cols<H> vt[4];
  constexpr int V_LOADS = 4 * (Cols<H>::N4 + (Cols<H>::REST != 0));
  const auto within = [&](int key) { return (unsigned)min(max(key, lo), hi - 1); };
  auto load_k = [&](int b) { kt.load(kb, __umul24(within(b * BLK + (lane >> 2)), k_row) + Blocks<H>::chunk(lane)); };
  auto load_v = [&](int b) {
#pragma unroll
    for (int i = 0; i < 4; ++i) vt[i].load(vb, within(b * BLK + 4 * g4 + i), v_row, l15);
  };
  if (j < end) {
    load_k(j);
    load_v(j);
  }
  while (j < end) {
    const int k0 = j * BLK;
    f32x4 p[RT];
    mfma::wait_dma<V_LOADS>();
    __builtin_amdgcn_sched_barrier(0);
    dot_rows<H, RT>(p, kt, qf);
    j += lanes;
    mfma::wait_vmem_all();                            // V: the products would wait for the next block's K too
    reads_done();
    if (j < end) load_k(j);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      to_scores<-1>(p[t], r, raw, r.slopes ? rs.slope[t] : 0.f, r.slopes ? fmaf((float)-(k0 + 4 * g4), r.steps[0], rs.at[t]) : 0.f);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[t][i] = (unsigned)(k0 + 4 * g4 + i - rs.run[t].lo) < (unsigned)rs.run[t].n ? p[t][i] : -INFINITY;
        m_lane[t] = fmaxf(m_lane[t], p[t][i]);
      }
      // (m_lane - m_ref) is +inf on the first visible block, NaN (-> false) while nothing is visible
      const bool grow = m_lane[t] - m_ref[t] > kRescaleThreshold;
      if (__builtin_amdgcn_ballot_w64(grow) != 0) {
        const float m_row = row_max(m_lane[t]);
        const float alpha = m_ref[t] == -INFINITY ? 0.f : fast_exp2(m_ref[t] - m_row);
        m_ref[t] = m_row;
        l_run[t] *= alpha;
        o[t].scale(alpha);
      }
      const float mr = m_ref[t] == -INFINITY ? 0.f : m_ref[t];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[t][i] = fast_exp2(p[t][i] - mr);
        l_run[t] += p[t][i];
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < RT; ++t) o[t].contract(vt[i], p[t][i]);
    __builtin_amdgcn_sched_barrier(0);
    if (j < end) load_v(j);
  }
  mfma::wait_vmem_all();

  // ---- to the true row maximum over all key lanes, then the sums over the lanes
  float m_all[RT];
  float* stat = reinterpret_cast<float*>(smem);      // [kl][t][16]
#pragma unroll
  for (int t = 0; t < RT; ++t) m_all[t] = row_max(m_lane[t]);
  __syncthreads();                                   // (the tiles are written over)
#pragma unroll
  for (int t = 0; t < RT; ++t)
    if (g4 == 0) stat[(kl * RT + t) * 16 + l15] = m_all[t];
  __syncthreads();
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int x = 0; x < KL; ++x) m_all[t] = fmaxf(m_all[t], stat[(x * RT + t) * 16 + l15]);
  f32x4 lsum[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const float f = m_ref[t] == -INFINITY ? 0.f : fast_exp2(m_ref[t] - m_all[t]);
    o[t].scale(f);
    lsum[t] = f32x4{row_sum(l_run[t]) * f, 0.f, 0.f, 0.f};
  }
  merge_lanes<RT * (H / 16 + 1)>(reinterpret_cast<f32x4*>(smem), kl, lane, [&](int i) -> f32x4& {
    return i < RT ? lsum[i] : o[(i - RT) / (H / 16)].acc[(i - RT) % (H / 16)];
  });
  if (kl != 0) return;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int row = q0 + BLK * t + l15;
    if (row >= map.rows) continue;
    const int64_t at = (int64_t)part * d.heads * d.nq + row0 + row;
    const float l = lsum[t][0];
    if (r.norm && map.parts == 1) {
      o[t].store(out0 + at * H, g4, l > 0.f ? 1.0f / l : 0.f);
      if (g4 == 0) out1[at] = l > 0.f ? m_all[t] / kLog2e + logf(l) : -INFINITY;
    } else {
      o[t].store(out0 + at * H, g4, 1.0f);
      if (g4 == 0) { out1[at] = m_all[t] / kLog2e; out2[at] = l; }
    }
  }
}

// ------------------------------------------------------------------------------------------------ dQ
// 32 rows a workgroup: two pairs of wavefronts with 16 rows each, two key lanes.  It also leaves the row table.
// (Two lanes of each 16 rows, where the plain kernel has four of 16 rows: the table is by 32.)
template <int H>
__global__ __launch_bounds__(64 * KL, 2) void scored_dq_f32_kernel(
    a2d_tile_desc d, ScoreRules r, int by_size, int parts, RowTable tab, const float* __restrict__ Q, const float* __restrict__ K,
    const float* __restrict__ V, const float* __restrict__ O, const float* __restrict__ dO, const float* __restrict__ lse,
    float* dQ) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  __shared__ RowTile half[2];
  constexpr int BM = 2 * BLK;
  const int nqb = (d.nq + BM - 1) / BM;
  int unit, blk;
  if (!xcd_map(blockIdx.x, d.heads / r.group * parts, r.group * nqb, by_size != 0, unit, blk)) return;
  const mfma::Split up = mfma::split_by(unit, parts), in_group = mfma::query_head(blk, r.group, nqb, by_size != 0);
  const int kvh = up.q, part = up.r, head = kvh * r.group + in_group.r, q0 = (nqb - 1 - in_group.q) * BM;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int rg = wave & 1, kl = wave >> 1, lanes = 2 * parts;    // row group, key lane
  const int l15 = lane & 15, g4 = lane >> 4;
  const gptr_t kb = uniform_gptr(K + (int64_t)kvh * d.lk.head), vb = uniform_gptr(V + (int64_t)kvh * d.lv.head);
  const unsigned k_row = (unsigned)d.lk.row * 4, v_row = (unsigned)d.lv.row * 4;
  const float raw = d.scale * kLog2e, inv_top = r.cap != 0.f ? 1.f / r.capped.top : 0.f;
  const int row = q0 + BLK * rg + l15, in = min(row, d.nq - 1);

  Nat<H> qf, gf, of;
  qf.load(uniform_gptr(Q + (int64_t)head * d.lq.head), in, (unsigned)d.lq.row * 4, g4);
  gf.load(uniform_gptr(dO + (int64_t)head * d.ldo.head), in, (unsigned)d.ldo.row * 4, g4);
  of.load(uniform_gptr(O + (int64_t)head * d.lo.head), in, (unsigned)d.lo.row * 4, g4);       // for delta only
  const float L = lse[(int64_t)head * d.nq + in];
  Run run = visible_run(d, r, head, in);
  if (row >= d.nq || L == -INFINITY) run.n = 0;
  const bool live = run.n > 0;
  float del = 0.f;
#pragma unroll
  for (int y = 0; y < H / 16; ++y)
#pragma unroll
    for (int e = 0; e < 4; ++e) del = fmaf(gf.v[y][e], of.v[y][e], del);
  del = live ? row_sum(del) : 0.f;
  if (!live) {
#pragma unroll
    for (int y = 0; y < H / 16; ++y) qf.v[y] = gf.v[y] = zero4();
  }
  lift(qf, r);
  const float from = live ? L : INFINITY;             // +inf: P = 0
  const float slope = r.slopes ? r.slopes[head] : 0.f;
  const float at = (float)(int)(r.rel + (int64_t)in * r.step);
  const auto least = [](int a, int b) { return min(a, b); };
  const auto most = [](int a, int b) { return max(a, b); };
  const int lo = over16(live ? run.lo : INT_MAX, least), hi = over16(live ? run.lo + run.n : 0, most);
  const int all_lo = over16(live ? run.lo : 0, most), all_hi = over16(live ? run.lo + run.n : INT_MAX, least);
  const unsigned rows = (unsigned)__builtin_amdgcn_ballot_w64(live) & 0xFFFFu;
  if (part == 0 && kl == 0) {
    if (g4 == 0 && row < tab.padded) {
      const int64_t to = (int64_t)head * tab.padded + row;
      tab.from[to] = from;
      tab.delta[to] = -del;
      tab.lo[to] = run.lo;
      tab.n[to] = run.n;
    }
    if (lane == 0) half[rg] = RowTile{lo, hi, all_lo, all_hi, rows, {0, 0, 0}};
  }
  __syncthreads();
  if (part == 0 && threadIdx.x == 0)
    tab.tiles[((int64_t)head * tab.padded + q0) / 32] =
        RowTile{min(half[0].lo, half[1].lo), max(half[0].hi, half[1].hi), max(half[0].all_lo, half[1].all_lo),
                min(half[0].all_hi, half[1].all_hi), half[0].live | half[1].live << 16, {0, 0, 0}};
  // (heads whose rows end in the first half of the last 64: the rest of the table)
  if (part == 0 && q0 + BM >= d.nq && q0 + BM < tab.padded) {
    const int64_t to = (int64_t)head * tab.padded + q0 + BM;
    if (threadIdx.x < 32) {
      tab.from[to + threadIdx.x] = INFINITY;
      tab.delta[to + threadIdx.x] = 0.f;
      tab.lo[to + threadIdx.x] = tab.n[to + threadIdx.x] = 0;
    }
    if (threadIdx.x == 0) tab.tiles[to / 32] = RowTile{INT_MAX, 0, 0, INT_MAX, 0, {0, 0, 0}};
  }

  Out<H> dq;
  dq.zero();
  Blocks<H> kt, vt;
  kt.init((lds_t)smem + 2 * wave * Blocks<H>::BYTES, l15, g4);
  vt.init((lds_t)smem + (2 * wave + 1) * Blocks<H>::BYTES, l15, g4);
  const int end = hi > lo ? (hi + BLK - 1) / BLK : 0;
  int j = (hi > lo ? lo / BLK : 0) + part * 2 + kl;
  const auto load = [&](const Blocks<H>& to, gptr_t base, unsigned row_bytes, int b) {
    to.load(base, __umul24((unsigned)min(max(b * BLK + (lane >> 2), lo), hi - 1), row_bytes) + Blocks<H>::chunk(lane));
  };
  if (j < end) {
    load(kt, kb, k_row, j);
    load(vt, vb, v_row, j);
  }
  Cols<H> ring[2];
  while (j < end) {
    const int k0 = j * BLK;
    f32x4 p, ds;
    mfma::wait_dma();
    dot_two<H>(p, ds, kt, qf, vt, gf, [] {}, [&](auto Y) {
      constexpr int y = decltype(Y)::value;
      if constexpr (y >= H / 16 - 2) kt.cols(ring[y - (H / 16 - 2)], y - (H / 16 - 2));
    });
    reads_done();
    j += lanes;
    const bool more = j < end;
    if (more) load(vt, vb, v_row, j);
    f32x4 y = p;
    if (r.cap != 0.f) {
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = cap_log2_f32(r.capped, p[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = p[i] * raw;
    }
    const float far = fmaf((float)-(k0 + 4 * g4), r.steps[0], at);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float less = r.slopes ? fmaf(slope, fabsf(distance<-1>(r, far, 0, i)), from) : from, t = y[i] * inv_top;
      ds[i] = fast_exp2(fmaf(-less, kLog2e, y[i])) * (ds[i] - del) * fmaf(-t, t, 1.f);
      ds[i] = (unsigned)(k0 + 4 * g4 + i - run.lo) < (unsigned)run.n ? ds[i] : 0.f;
    }
    static_for<0, 4>([&](auto R) {
      constexpr int i = decltype(R)::value;
      dq.contract(ring[i & 1], ds[i]);
      if constexpr (i < 2) kt.cols(ring[i & 1], i + 2);
      if constexpr (i == 2) {
        reads_done();
        if (more) load(kt, kb, k_row, j);
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  }
  // key lane 1's sums to lane 0's wavefront of the same rows
  f32x4* const xch = reinterpret_cast<f32x4*>(smem) + rg * (H / 16) * 64 + lane;
  __syncthreads();
  if (kl == 1) {
#pragma unroll
    for (int t = 0; t < H / 16; ++t) xch[64 * t] = dq.acc[t];
  }
  __syncthreads();
  if (kl == 1 || row >= d.nq) return;
#pragma unroll
  for (int t = 0; t < H / 16; ++t) {
    const f32x4 v = xch[64 * t];
    dq.acc[t][0] += v[0]; dq.acc[t][1] += v[1]; dq.acc[t][2] += v[2]; dq.acc[t][3] += v[3];
  }
  dq.store(dQ + (((int64_t)part * d.heads + head) * d.nq + row) * H, g4, d.scale, parts == 1 && r.acc != 0);
}

// -------------------------------------------------------------------------------------------- dK, dV
// 16 keys a workgroup; its key lanes take every fourth of the tiles of 32 rows that see one of them, 16 rows a step.
template <int H>
__global__ __launch_bounds__(64 * KL, 2) void scored_dkdv_f32_kernel(
    a2d_tile_desc d, ScoreRules r, int by_size, int parts, RowTable tab, int bits_at, const float* __restrict__ Q,
    const float* __restrict__ K, const float* __restrict__ V, const float* __restrict__ dO, float* __restrict__ dK,
    float* __restrict__ dV) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  int head, blk;                                      // key/value head
  if (!xcd_map(blockIdx.x, d.heads / r.group * parts, (d.nkv + BLK - 1) / BLK, by_size != 0, head, blk)) return;
  const mfma::Split up = mfma::split_by(head, parts);
  head = up.q;
  const int part = up.r, qh0 = head * r.group;
  const int kl = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int l15 = lane & 15, g4 = lane >> 4;
  const int k0 = blk * BLK, key = k0 + l15, k_ld = min(key, d.nkv - 1);
  const gptr_t qb = uniform_gptr(Q + (int64_t)qh0 * d.lq.head), gb = uniform_gptr(dO + (int64_t)qh0 * d.ldo.head);
  const unsigned q_row = (unsigned)d.lq.row * 4, g_row = (unsigned)d.ldo.row * 4;
  const unsigned q_head = (unsigned)d.lq.head * 4, g_head = (unsigned)d.ldo.head * 4;
  const float raw = d.scale * kLog2e, inv_top = r.cap != 0.f ? 1.f / r.capped.top : 0.f;

  // ---- a bit for each tile of 32 rows, of all query heads, that sees a key of the workgroup
  const int ntiles = tab.padded / 32, all = ntiles * r.group, words = (all + 63) / 64;
  uint64_t* const bits = reinterpret_cast<uint64_t*>(smem + bits_at);
  const RowTile* const tiles = tab.tiles + (int64_t)qh0 * ntiles;
  for (int w = kl; w < words; w += KL) {
    const int t = 64 * w + lane;
    bool seen = false;
    if (t < all) {
      const int lo = tiles[t].lo, hi = tiles[t].hi;
      seen = lo < hi && lo < k0 + BLK && hi > k0;
    }
    const uint64_t m = __builtin_amdgcn_ballot_w64(seen);
    if (lane == 0) bits[w] = m;
  }
  Nat<H> kf, vf;
  kf.load(uniform_gptr(K + (int64_t)head * d.lk.head), k_ld, (unsigned)d.lk.row * 4, g4);
  vf.load(uniform_gptr(V + (int64_t)head * d.lv.head), k_ld, (unsigned)d.lv.row * 4, g4);
  lift(kf, r);
  Out<H> dk, dv;
  dk.zero();
  dv.zero();
  Blocks<H> qt, gt;
  qt.init((lds_t)smem + 2 * kl * Blocks<H>::BYTES, l15, g4);
  gt.init((lds_t)smem + (2 * kl + 1) * Blocks<H>::BYTES, l15, g4);
  __syncthreads();
  StepWalk walk;
  const int lanes = KL * parts, first = part * KL + kl;
  int left = walk.open(bits, words) - first;          // of the set bits, this lane's first among them
  left = left > 0 ? (left + lanes - 1) / lanes : 0;   // tiles that it takes
  if (left > 0) walk.skip(first);

  // position of the next step to be loaded: tile, half of it
  int tile = 0, h = 0, qh = 0, i0 = 0;
  unsigned live = 0;
  f32x4 from, del;
  u32x4 lo, n;
  float slope = 0.f;
  const auto place = [&]() {                          // what a tile's steps need
    tile = walk.next();
    walk.skip(lanes - 1);
    qh = tile / ntiles;
    live = tiles[tile].live;
    live = __builtin_amdgcn_readfirstlane(live);
  };
  const auto load_rows = [&](const Blocks<H>& to, gptr_t base, unsigned head_bytes, unsigned row_bytes) {
    const int ln = mfma::lane_again();
    if (live >> (16 * h + (ln >> 2)) & 1) {
      to.load(base, qh * head_bytes + __umul24((unsigned)((tile - qh * ntiles) * 32 + 16 * h + (ln >> 2)), row_bytes) + Blocks<H>::chunk(ln));
    } else {
#pragma unroll
      for (int y = 0; y < H / 16; ++y) lstore(to.base + y * Blocks<H>::STRIDE + 16 * ln, zero4());      // (rows that see nothing)
    }
  };
  const auto load_table = [&]() {
    const int64_t at = ((int64_t)qh0 * ntiles + tile) * 32 + 16 * h + 4 * g4;
    from = *reinterpret_cast<const f32x4*>(tab.from + at);
    del = *reinterpret_cast<const f32x4*>(tab.delta + at);
    lo = *reinterpret_cast<const u32x4*>(tab.lo + at);
    n = *reinterpret_cast<const u32x4*>(tab.n + at);
  };
  bool more = left > 0;
  if (more) {
    place();
    load_table();
    load_rows(qt, qb, q_head, q_row);
    load_rows(gt, gb, g_head, g_row);
  }
  Cols<H> ring[2];
  while (more) {
    i0 = (tile - qh * ntiles) * 32 + 16 * h;
    if (r.slopes) slope = r.slopes[qh0 + qh];
    f32x4 p, ds;
    mfma::wait_dma();
    reads_done();                                     // (zeros written in place of rows)
    const f32x4 fr = from, de = del;
    const u32x4 ll = lo, nn = n;
    dot_two<H>(p, ds, qt, kf, gt, vf, [] {}, [&](auto Y) {
      constexpr int y = decltype(Y)::value;
      if constexpr (y >= H / 16 - 2) qt.cols(ring[y - (H / 16 - 2)], y - (H / 16 - 2));
    });
    // ---- the next step
    if (h == 0) {
      h = 1;
    } else {
      h = 0;
      more = --left > 0;
      if (more) place();
    }
    if (more) load_table();
    const float far = (float)(int)(r.rel + (int64_t)(i0 + 4 * g4 - key) * r.step);
    f32x4 y = p;
    if (r.cap != 0.f) {
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = cap_log2_f32(r.capped, p[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = p[i] * raw;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool vis = (unsigned)key - ll[i] < nn[i];
      const float less = r.slopes ? fmaf(slope, fabsf(distance<1>(r, far, 0, i)), fr[i]) : fr[i];
      const float t = y[i] * inv_top, e = fast_exp2(fmaf(-less, kLog2e, y[i]));
      p[i] = vis ? e : 0.f;
      ds[i] = vis ? e * (ds[i] + de[i]) * fmaf(-t, t, 1.f) : 0.f;
    }
    static_for<0, 8>([&](auto R) {                    // dK, dV; the next tiles as soon as the last read of these is through
      constexpr int i = decltype(R)::value, next = i + 2;
      if constexpr (i < 4) dk.contract(ring[i & 1], ds[i]); else dv.contract(ring[i & 1], p[i - 4]);
      if constexpr (i == 2 || i == 6) {
        reads_done();
        if (more) {
          if constexpr (i == 2) load_rows(qt, qb, q_head, q_row); else load_rows(gt, gb, g_head, g_row);
        }
      }
      if constexpr (next < 8) (next < 4 ? qt : gt).cols(ring[i & 1], next & 3);
      __builtin_amdgcn_sched_barrier(0);
    });
  }
  mfma::wait_vmem_all();
  merge_lanes<H / 8>(reinterpret_cast<f32x4*>(smem), kl, lane, [&](int i) -> f32x4& {
    return i < H / 16 ? dk.acc[i] : dv.acc[i - H / 16];
  });
  if (kl != 0 || key >= d.nkv) return;
  const int64_t row = ((int64_t)part * (d.heads / r.group) + head) * d.nkv + key;
  dk.store(dK + row * H, g4, d.scale);
  dv.store(dV + row * H, g4, 1.0f);
}

constexpr int most(int a, int b) { return a > b ? a : b; }
template <int H, int RT>
constexpr int fwd_lds() { return most(KL * Blocks<H>::BYTES, KL / 2 * RT * (H / 16 + 1) * 1024); }
template <int H>
constexpr int bwd_lds() { return most(2 * KL * Blocks<H>::BYTES, KL / 2 * (H / 8) * 1024); }
constexpr int MOST_BITS = 2 * SCORED_MOST_BITS;      // (by 32 rows)

template <int H, int RT>
hipError_t fwd(Phase ph, const a2d_tile_desc& d, const ScoreRules& r, int parts, const void* Q, const void* K, const void* V, float* out0,
               float* out1, float* out2, const FwdInput& in, hipStream_t s) {
  constexpr int lds = fwd_lds<H, RT>(), bm = BLK * RT;
  if (ph == PREPARE) return ensure_dynamic_lds(reinterpret_cast<const void*>(scored_fwd_f32_kernel<H, RT>), lds);
  RowMap map = row_map(d, r, bm, parts);
  if (map.by_size == BY_RANK) map.by_size = 0;
  A2D_LAUNCH((scored_fwd_f32_kernel<H, RT>), dim3(xcd_grid(d.heads / r.group * parts, map.sub * ((map.rows + bm - 1) / bm))), dim3(64 * KL), lds,
             s, d, r, map, (const float*)Q, (const float*)K, (const float*)V, out0, out1, out2, in);
  return hipGetLastError();
}

template <int H>
hipError_t bwd(Phase ph, const a2d_tile_desc& d, const ScoreRules& r, const ScoredBwdPlan& plan, const void* Q, const void* K, const void* V,
               const void* O, const void* dO, const float* lse, void* ws, float* dQ, float* dK, float* dV, hipStream_t s) {
  constexpr int lds = bwd_lds<H>();
  if (ph == PREPARE) {
    const hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void*>(scored_dq_f32_kernel<H>), lds);
    return e != hipSuccess ? e : ensure_dynamic_lds(reinterpret_cast<const void*>(scored_dkdv_f32_kernel<H>), lds + MOST_BITS);
  }
  const RowTable tab = row_table(d, ws);
  const int by_size = blocks_by_size(d, r, 1) != 0, kvh = d.heads / r.group, words = (tab.padded / 32 * r.group + 63) / 64;
  A2D_LAUNCH((scored_dq_f32_kernel<H>), dim3(xcd_grid(kvh * plan.q, r.group * ((d.nq + 31) / 32))), dim3(64 * KL), lds, s, d, r, by_size,
             plan.q, tab, (const float*)Q, (const float*)K, (const float*)V, (const float*)O, (const float*)dO, lse, dQ);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  A2D_LAUNCH((scored_dkdv_f32_kernel<H>), dim3(xcd_grid(kvh * plan.kv, (d.nkv + BLK - 1) / BLK)), dim3(64 * KL), lds + 8 * words, s, d, r,
             by_size, plan.kv, tab, lds, (const float*)Q, (const float*)K, (const float*)V, (const float*)dO, dK, dV);
  return hipGetLastError();
}

int head_index(int hdim) { return hdim > 96 ? 3 : hdim > 80 ? 2 : hdim > 64 ? 1 : 0; }

}  // namespace

ScoredPlan plan_scored_fwd_f32(const a2d_tile_desc& d, const ScoreRules& r, int cus, int cap) {
  const auto blocks = [&](int bm) {
    const RowMap map = row_map(d, r, bm, 1);
    return (int64_t)(d.heads / r.group) * map.sub * ((map.rows + bm - 1) / bm);
  };
  if (blocks(32) >= 4 * (int64_t)cus) return ScoredPlan{2, 1, false};
  constexpr double kStep[4] = {0.93, 1.11, 1.49, 1.99};
  const WalkKeys w = walk_keys(d, r);
  const WalkModel m{blocks(16), 2 * cus, w.mean / (BLK * KL) + 0.2, w.most / (BLK * KL) + 0.2, kStep[head_index(d.hdim)], 2.4, 0, 0, nullptr, 0, 0.5};
  return ScoredPlan{1, best_parts(m, cap, 5.0, (double)d.heads * d.nq * (d.hdim + 2) * 8 / 4.6e6, nullptr), false};
}

ScoredBwdPlan plan_scored_bwd_f32(const a2d_tile_desc& d, const ScoreRules& r, int cus, int cap_q, int cap_kv) {
  constexpr double kRow[4] = {0.95, 1.21, 1.87, 2.88}, kKey[4] = {1.69, 2.06, 3.05, 4.28};
  const int h = head_index(d.hdim);
  const WalkKeys w = walk_keys(d, r);
  const double rows = (double)d.nq * r.group;
  const WalkModel q{(int64_t)d.heads * ((d.nq + 31) / 32), 2 * cus, w.mean / (2 * BLK) + 0.2, w.most / (2 * BLK) + 0.2, kRow[h], 3.6, 0, 0, nullptr, 0, 0.5};
  const WalkModel k{(int64_t)(d.heads / r.group) * ((d.nkv + BLK - 1) / BLK), 2 * cus, rows * (w.mean / d.nkv) / (BLK * KL) + 0.2,
                    rows / (BLK * KL) + 0.2, kKey[h], 1.7, 0, 0, nullptr, 0, 0.5};
  return ScoredBwdPlan{1, best_parts(q, cap_q, 4.6, (double)d.heads * d.nq * d.hdim * 8 / 4.9e6, nullptr),
                       best_parts(k, cap_kv, 4.6, (double)(d.heads / r.group) * d.nkv * d.hdim * 16 / 4.9e6, nullptr)};
}

void route_scored_fwd_f32(const a2d_tile_desc& d, const ScoreRules& r, const ScoredPlan& plan, ScoredRoute* out) {
  const int bm = BLK * plan.form;
  const RowMap map = row_map(d, r, bm, plan.parts);
  *out = ScoredRoute{};
  out->kernel[out->kernels++] = "scored_fwd_f32_kernel";
  out->rows = bm;
  out->lanes = out->waves = KL;
  out->order = map.by_size ? BY_ROWS : 0;
  out->blocks_q = map.sub * ((map.rows + bm - 1) / bm);
  out->units_q = out->blocks_q * plan.parts;
}
void route_scored_bwd_f32(const a2d_tile_desc& d, const ScoreRules&, const ScoredBwdPlan& plan, ScoredRoute* out) {
  *out = ScoredRoute{};
  for (const char* k : {"scored_dq_f32_kernel", "scored_dkdv_f32_kernel"}) out->kernel[out->kernels++] = k;
  out->rows = 2 * BLK;
  out->lanes = 2;
  out->waves = KL;
  out->blocks_q = (d.nq + 31) / 32;
  out->units_q = out->blocks_q * plan.q;
  out->blocks_kv = (d.nkv + BLK - 1) / BLK;
  out->units_kv = out->blocks_kv * plan.kv;
  if (plan.q > 1 || plan.kv > 1) out->kernel[out->kernels++] = "sum_parts_kernel";
}

#define A2D_HEADS(CALL)              \
  switch (d.hdim) {                  \
    case 128: return CALL(128);      \
    case 96: return CALL(96);        \
    case 80: return CALL(80);        \
    default: return CALL(64);        \
  }
hipError_t launch_scored_fwd_f32(Phase ph, const a2d_tile_desc& d, const ScoreRules& r, const ScoredPlan& plan, const void* Q, const void* K,
                                 const void* V, float* out0, float* out1, float* out2, const FwdInput& in, hipStream_t s) {
#define A2D_CALL(H)                                                                              \
  plan.form == 2 ? fwd<H, 2>(ph, d, r, plan.parts, Q, K, V, out0, out1, out2, in, s)              \
                 : fwd<H, 1>(ph, d, r, plan.parts, Q, K, V, out0, out1, out2, in, s)
  A2D_HEADS(A2D_CALL)
#undef A2D_CALL
}
hipError_t launch_scored_bwd_f32(Phase ph, const a2d_tile_desc& d, const ScoreRules& r, const ScoredBwdPlan& plan, const void* Q,
                                 const void* K, const void* V, const void* O, const void* dO, const float* lse, void* ws, float* dQ,
                                 float* dK, float* dV, hipStream_t s) {
#define A2D_CALL(H) bwd<H>(ph, d, r, plan, Q, K, V, O, dO, lse, ws, dQ, dK, dV, s)
  A2D_HEADS(A2D_CALL)
#undef A2D_CALL
}

}  // namespace a2d
