// bf16 forward tile under score rules (a2d_score_rules in a2d.h) on the matrix units, H = 128, 96, 80 and 64.
//
// The contractions are those of fwd_mfma_kernel and fwd_small_kernel: S^T = K Q^T with a lane holding four keys of one query
// row in each tile of 16 x 16, and P^T as it stands as an operand of O^T += V^T P^T.  Between them the scores are brought into log2
// units (z -> cap -> minus the bias) relative to the row's reference, so that 2^x follows directly.  The rules cost vector instructions a
// score: the cap 4.5 (a polynomial, see CapArgs; where some score of a wavefront's block is beyond its range 12, two of them of a quarter of the
// rate), the bias 1, near the diagonal 2.3.  Bound: the vector instructions (of 64 keys and 32 rows of a wavefront at H = 64, 512 clocks of
// exponentials and 600 to 900 of others stand beside 512 of matrix instructions), which the two (H = 64: up to three) wavefronts of a SIMD share;
// 32 / 8 heads of 128, 4096 x 4096, causal under a cap: vector instructions 58 % of the time, matrix instructions 35 %.  Documents end with
// their longest walk instead: six of 8192 tokens, H = 64, 53 % and 22 %, up to 50 steps where an even share were 30.  16 heads of 64,
// 8192 x 8192, not causal: 295 us without rules, 326 with a bias, 390 with a cap; 32 / 8 of 128, 4096 x 4096, causal: 139, 132, 155.
//
// Masks: whatever they are made of, a query row sees one run of keys (visible_run).  A workgroup walks the hull of
// its rows' runs; a wavefront leaves out the blocks that none of its rows sees, and compares keys only in blocks that some row does not see
// whole.  Keys outside the hull are not read (rows of a block beyond it re-read the hull's first or last key), so
// that a cache's unused slots may hold anything.
//
// Rows: the query rows of the heads that share a key/value head follow one another (packed) where a head has fewer rows
// than a workgroup: a token of each of the group's heads reads the keys once.
#include "a2d_fwd.hpp"
#include "a2d_scored_rows.hpp"

namespace a2d {
namespace {

using namespace mfma;

constexpr float kRescaleThreshold = 8.0f;            // log2 units (as in a2d_fwd_mfma.hip)
constexpr float kFarReference = 64.0f;               // (see Softmax::follow)

// ---- Scores in log2 units, relative to the row's reference from the start: the multiply-add that ends the cap or takes in the raw product takes
// the reference too, so that 2^x follows directly (a subtraction of its own was a tenth of the vector instructions).
// Score e of a lane's: tile of 16 keys e >> 2, key e & 3 of its four.  raw: log2 units of a raw product.  from: distance of the lane's first
// key.  BEYOND: products beyond the polynomial's range too.  ASIDE: the keys stand on one side of the row, all of them ASIDE_STEPS off at
// least, so that the bias is linear (slope < 0: keys ahead) and its multiply-add takes in the reference: start = -ref - slope from.  (What
// `start` is rounded by is 2^-24 of ref and of the first key's bias, which is 3 times the score's own at most.)
constexpr int ASIDE_STEPS = 32;
template <bool CAP, bool BIAS, bool BEYOND, bool ASIDE>
__device__ __forceinline__ float to_score(float z, float ref, const ScoreRules& r, float raw, float slope, float from, float start, int e) {
  const float less = ASIDE ? (e == 0 ? start : fmaf(slope, r.all_steps[e], start)) : -ref;
  float x;
  if constexpr (CAP) x = BEYOND ? cap_log2(r.capped, z) + less : fmaf(z, cap_factor(r.capped, z), less);
  else x = fmaf(z, raw, less);
  if constexpr (BIAS && !ASIDE) x = fmaf(-slope, fabsf(from - r.all_steps[e]), x);
  return x;
}
// whether some score of the wavefront's is beyond the polynomial's range (a NaN is left out, and comes through it as NaN)
template <int NT>
__device__ __forceinline__ bool some_beyond(const f32x4 (&s)[NT][2], const CapArgs& a) {
  float big = 0.f;
#pragma unroll
  for (int q = 0; q < 2; ++q)
#pragma unroll
    for (int e = 0; e < 4 * NT; ++e) big = fmaxf(big, fabsf(s[e >> 2][q][e & 3]));
  return __builtin_amdgcn_ballot_w64(big > a.small) != 0;
}
// Distance of a lane's first key of the tiles from k0 on (whole numbers below 2^24: exact)
template <bool BIAS>
__device__ __forceinline__ float first_distance(const ScoreRules& r, const RowState<2>& rs, int q, int k0, int grp) {
  return BIAS ? fmaf((float)-(k0 + 4 * grp), r.steps[0], rs.at[q]) : 0.f;
}

// What a wavefront's softmax keeps of the lane's row in each of its two tiles
struct Softmax {
  float m_lane[2];       // maximum of the lane's scores so far, relative to ref; -inf: none
  float ref[2];          // reference of the row's scores (the same in its four lanes); 0 until it sees something
  float l[2];            // the lane's share of the row sum, relative to ref
  __device__ __forceinline__ void start(int q, float m) {                // m: stored maximum, natural units
    m_lane[q] = m == -INFINITY ? m : 0.f;
    ref[q] = m == -INFINITY ? 0.f : m * kLog2e;
  }
  // the row's maximum in log2 units, and what N and l are multiplied with to be relative to it
  __device__ __forceinline__ void finish(int q, float& m_row, float& f) const {
    m_row = row_max(m_lane[q]);
    const bool none = m_row == -INFINITY;
    f = none ? 0.f : fast_exp2(-m_row);
    if (!none) m_row += ref[q];
  }
  // take: the maxima of new scores.  The reference follows the running maximum only when a score exceeds it by more than 2^8, or
  // with the first keys that a lane sees (as in fwd_softmax): a rare branch, and the only place where the lanes of a row talk.
  // follow is true where a row left a reference far behind: its scores are rounded to 2^-24 of their distance from that, which may be many
  // times their own size (a steep bias, met far keys first), so they are made again, from the products, and taken.  Up to 2^64, whose
  // logarithm's rounding is 4e-6 of a probability, a thousandth of its own to bf16, they stay: rows that saw but a few keys
  // of their first block leave its reference often (32 / 8 heads of 128, 4096 x 4096, capped: 178 us with every one made again, 153 with these).
  template <int NT>
  __device__ __forceinline__ bool take(const f32x4 (&s)[NT][2], float (&was)[2]) {       // whether the reference is to follow
    bool grow = false;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      float mx = was[q] = m_lane[q];
#pragma unroll
      for (int e = 0; e < 4 * NT; ++e) mx = fmaxf(mx, s[e >> 2][q][e & 3]);
      m_lane[q] = mx;
      grow |= mx > kRescaleThreshold || (was[q] == -INFINITY && mx > -INFINITY);         // (NaN: false)
    }
    return __builtin_amdgcn_ballot_w64(grow) != 0;
  }
  template <int NT, int HT>
  __device__ __forceinline__ bool follow(f32x4 (&s)[NT][2], f32x4 (&o)[HT][2], const float (&was)[2]) {
    bool left = false;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const float m_row = row_max(m_lane[q]);
      const bool held = row_max(was[q]) > -INFINITY;
      const float next = m_row == -INFINITY ? ref[q] : ref[q] + m_row, by = next - ref[q];
      const float alpha = held ? fast_exp2(-by) : 0.f;
      const bool made = held && by > kFarReference;
      left |= made;
      ref[q] = next;
      m_lane[q] = made ? was[q] - by : m_lane[q] - by;
      l[q] *= alpha;
#pragma unroll
      for (int e = 0; e < 4 * NT; ++e) s[e >> 2][q][e & 3] -= by;
#pragma unroll
      for (int t = 0; t < HT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[t][q][e] *= alpha;
    }
    return __builtin_amdgcn_ballot_w64(left) != 0;
  }
  // P^T in bf16 (nearest-even, for the contraction); the sums take the probabilities before their rounding.  O is off by 1.41 times what its
  // own rounding does: two roundings of one size.  Two numbers, as below, would double the contraction with V: 32 / 8 heads of
  // 128, 4096 x 4096, capped 205 us for 154, six documents of 8192 tokens 96 for 75, 16384 x 16384 652 for 482.
  template <int NT>
  __device__ __forceinline__ void probabilities(const f32x4 (&s)[NT][2], bf16x8 (&pb)[NT / 2][2]) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 4 * NT; ++e) {
        const float p = fast_exp2(s[e >> 2][q][e & 3]);
        sum += p;
        pb[e >> 3][q][e & 7] = (bf16_t)p;
      }
      l[q] += sum;
    }
  }
  // P^T as the sum of two bf16 numbers, 2^-17 of it off
  template <int NT>
  __device__ __forceinline__ void probabilities(const f32x4 (&s)[NT][2], bf16x8 (&pb)[NT / 2][2], bf16x8 (&rest)[NT / 2][2]) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 4 * NT; ++e) {
        const float p = fast_exp2(s[e >> 2][q][e & 3]);
        sum += p;
        pb[e >> 3][q][e & 7] = (bf16_t)p;
        rest[e >> 3][q][e & 7] = (bf16_t)(p - (float)pb[e >> 3][q][e & 7]);
      }
      l[q] += sum;
    }
  }
};

// Raw products of NT tiles of 16 keys from k0 on -> scores
// (ONE_WAY: of whatever size and place, which every product may go)
template <int NT, bool CAP, bool BIAS, bool ONE_WAY = false>
__device__ __forceinline__ void to_scores(f32x4 (&s)[NT][2], const Softmax& sm, const ScoreRules& r, const RowState<2>& rs, bool masked, int k0,
                                          int grp, float raw) {
  const auto all = [&](auto beyond, auto aside, bool ahead) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const float from = first_distance<BIAS>(r, rs, q, k0, grp), slope = !BIAS ? 0.f : ahead ? -rs.slope[q] : rs.slope[q], start = fmaf(-slope, from, -sm.ref[q]);
#pragma unroll
      for (int e = 0; e < 4 * NT; ++e)
        s[e >> 2][q][e & 3] =
            to_score<CAP, BIAS, decltype(beyond)::value, decltype(aside)::value>(s[e >> 2][q][e & 3], sm.ref[q], r, raw, slope, from, start, e);
    }
  };
  const bool ahead = BIAS && rs.farthest <= (k0 - ASIDE_STEPS) * r.step;
  if constexpr (ONE_WAY) {
    all(std::true_type{}, std::false_type{}, false);
  } else if (CAP && A2D_SELDOM(some_beyond(s, r.capped))) {
    asm volatile("" ::: "memory");                   // keep this a branch
    all(std::true_type{}, std::false_type{}, false);
  } else if (BIAS && A2D_SELDOM(!ahead && rs.nearest < (k0 + 16 * NT - 1 + ASIDE_STEPS) * r.step)) {
    asm volatile("" ::: "memory");
    all(std::false_type{}, std::false_type{}, false);
  } else {
    all(std::false_type{}, std::bool_constant<BIAS>{}, ahead);
  }
  if (A2D_SELDOM(masked)) {
    asm volatile("" ::: "memory");                   // keep this a branch
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int e = 0; e < 4 * NT; ++e) {
        const int key = k0 + 16 * (e >> 2) + 4 * grp + (e & 3) - rs.run[q].lo;
        s[e >> 2][q][e & 3] = (unsigned)key < (unsigned)rs.run[q].n ? s[e >> 2][q][e & 3] : -INFINITY;
      }
  }
}

template <int WAVES, int HR, int KL, bool CAP, bool BIAS>
__device__ __forceinline__ void scored_fwd_rows(
    int id, char* const lds_all, int* const hull, const Ranks& ranks, const a2d_tile_desc& d, const ScoreRules& r, const RowMap& map,
    const bf16_t* __restrict__ Q, const bf16_t* __restrict__ K, const bf16_t* __restrict__ V, float* out0, float* out1, float* out2,
    const FwdInput& in) {
  constexpr int RW = WAVES / KL, BM = 32 * RW, kThreads = 64 * RW;
  constexpr int HD = padded_head(HR), H = HR, KS = HD / 32, HT = HR / 16, BUF_BYTES = buf_bytes(HD);
  const int kl = KL == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x / kThreads);
  char* const lds = lds_all + kl * lds_bytes(HD);
  const unsigned lds_base = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds;

  const int nqb = (map.rows + BM - 1) / BM;
  int unit, blk;
  if (!xcd_map(id, d.heads / r.group * map.parts, map.sub * nqb, map.by_size != 0, unit, blk, kXcdCus * 8 / WAVES)) return;
  const Split up = split_by(unit, map.parts);
  const int kvh = up.q, part = up.r;
  const Split in_group = query_head(blk, map.sub, nqb, map.by_size != 0);
  const int head = kvh * r.group + in_group.r;
  // longest walks first, as far as they are known (late rows)
  const int q0 = (map.by_size == BY_RANK ? __builtin_amdgcn_readfirstlane((int)ranks.order[in_group.q]) : nqb - 1 - in_group.q) * BM;
  const int tid = (int)threadIdx.x - kl * kThreads;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, grp = lane >> 4;
  Q += (int64_t)head * d.lq.head;
  K += (int64_t)kvh * d.lk.head;
  V += (int64_t)kvh * d.lv.head;
  if (map.parts > 1) {
    const int64_t slot = (int64_t)part * d.heads * d.nq;
    out0 += slot * H;
    out1 += slot;
    out2 += slot;
  }
  const int64_t row0 = (int64_t)head * d.nq;          // of the run of rows, in the outputs
  const float raw = uniform(d.scale * kLog2e);

  RowState<2> rs;
  look_up_rows<2, BIAS>(rs, d, r, map, head, q0 + wave * 32, lane);
  bf16x8 qf[KS][2];
#pragma unroll
  for (int q = 0; q < 2; ++q)
#pragma unroll
    for (int x = 0; x < KS; ++x) {
      const int at = 32 * x + 8 * grp;
      qf[x][q] = *reinterpret_cast<const bf16x8*>(Q + rs.q_at[q] + min(at, H - 8));
      if (32 * x + 32 > H && at >= H) qf[x][q] = bf16x8{};
    }
  if (CAP && A2D_SELDOM(r.capped.lift != 1.f)) {
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int x = 0; x < KS; ++x) lift(qf[x][q], r.capped.lift);
  }
  if ((KL == 1 || kl == 0) && lane == 0) {
    hull[2 * wave] = rs.lo;
    hull[2 * wave + 1] = rs.hi;
  }
  if constexpr (H != HD) {
    // the K tiles' columns past the head size are zero for good (those of V are not read)
    for (int i = tid; i < 2 * BN * (HD - H) / 8; i += kThreads) {
      const int row = i % BN, x = i / BN, buf = x / ((HD - H) / 8), ch = H % 32 / 8 + x % ((HD - H) / 8);
      *reinterpret_cast<u32x4*>(lds + buf * BUF_BYTES + ((row >> 4) * KS + H / 32) * BLOCK + (row & 15) * 64 +
                                16 * (ch ^ block_swap((row & 15) >> 2))) = u32x4{0, 0, 0, 0};
    }
  }
  f32x4 o[HT][2];
#pragma unroll
  for (int t = 0; t < HT; ++t) o[t][0] = o[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
  Softmax sm;
  float m_in[2] = {-INFINITY, -INFINITY};
  sm.l[0] = sm.l[1] = 0.f;
  if (r.acc && part == 0 && kl == 0) {
    // continues the stored partial: N into the accumulators, m as the exponent's reference, l into one of the four lanes of a row
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int row = q0 + wave * 32 + 16 * q + (lane & 15);
      if (row >= map.rows) continue;
      m_in[q] = in.m[row0 + row];
      sm.l[q] = grp == 0 ? in.l[row0 + row] : 0.f;
#pragma unroll
      for (int t = 0; t < HT; ++t) o[t][q] = *reinterpret_cast<const f32x4*>(in.N + (row0 + row) * H + 16 * t + 4 * grp);
    }
  }
  __syncthreads();
  int lo = INT_MAX, hi = 0;
#pragma unroll
  for (int w = 0; w < RW; ++w) {
    lo = min(lo, hull[2 * w]);
    hi = max(hi, hull[2 * w + 1]);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(hi);
  const int first = hi > lo ? lo / BN : 1, end = hi > lo ? (hi + BN - 1) / BN : 1;     // key blocks of the walk

  // ---- staging, straight into LDS: of eight wavefronts 0 .. 3 load a row tile of K each and 4 .. 7 one of V, each of four
  // one of both.  Rows outside the hull re-read its first or last key.
  constexpr int LD_N = RW == 8 ? 1 : 2;
  const int ld_first = RW == 8 ? wave >> 2 : 0, ld_tile = wave & 3, ld_row = 16 * ld_tile + (lane >> 2);
  const int ld_chunk = (lane & 3) ^ block_swap(lane >> 4);
  const char* ld_base[LD_N];
  unsigned ld_row_bytes[LD_N];
#pragma unroll
  for (int x = 0; x < LD_N; ++x) {
    const bool v = ld_first + x != 0;
    ld_base[x] = reinterpret_cast<const char*>(v ? V : K);
    ld_row_bytes[x] = __builtin_amdgcn_readfirstlane((unsigned)(v ? d.lv.row : d.lk.row) * 2);
  }
  auto load_tile = [&](int j, int boff) {
    const int from = max(j * BN, lo), row = min(max(j * BN + ld_row, lo), hi - 1) - from;
#pragma unroll
    for (int x = 0; x < LD_N; ++x)
      dma_blocks<KS, H>(lds_base + boff + (4 * (ld_first + x) + ld_tile) * KS * BLOCK,
                        uniform_gptr(ld_base[x] + (unsigned)from * ld_row_bytes[x]), __umul24(row, ld_row_bytes[x]) + 16 * ld_chunk, ld_chunk);
  };
  Blocks16 rd;
  rd.init(lane, lds_base);
  // Under a bias the nearest keys score highest, and met last they would move a row's reference again and again: from the block of the
  // last row's own token down, then up from there (16 heads of 64, 8192 x 8192: causal 225 us from the first block up, 177 down; not
  // causal 410 from the last block down, 317 from the row's own)
  int turn = end - 1;
  if constexpr (BIAS) {
    const int64_t key = floor_div(r.rel + (int64_t)((map.rows > d.nq ? d.nq : min(q0 + BM, d.nq)) - 1) * r.step, r.step);
    turn = max(min(turn, (int)(max(key, (int64_t)0) / BN)), first);
  }
  const auto block_at = [&](int i) { return i <= turn - first ? turn - i : first + i; };
  const int blocks = end - first, stride = KL * map.parts;
  int lead = part * KL, i = lead + kl, j = block_at(i);      // key lane 0's place in the walk; this lane's, and its block
  if (i < blocks) load_tile(j, 0);
  wait_vmem_all();                                    // (the Q rows and the first tiles together)
#pragma unroll
  for (int q = 0; q < 2; ++q) sm.start(q, m_in[q]);
  __syncthreads();

  int boff = 0;
  for (; lead < blocks; lead += stride) {
    const int next = block_at(i + stride), k0 = j * BN;
    if (A2D_OFTEN(i + stride < blocks)) load_tile(next, BUF_BYTES - boff);
    if (i < blocks && k0 + BN > rs.lo && k0 < rs.hi) {
      Scores s;
      Ring kr, vr;
      bf16x8 pb[2][2];
      fwd_first_keys<HR>(kr, rd, boff);
      fwd_scores<HR>(s, kr, qf, rd, boff);
      const bool masked = k0 < rs.all_lo || k0 + BN > rs.all_hi;
      to_scores<4, CAP, BIAS>(s, sm, r, rs, masked, k0, grp, raw);
      float was[2];
      if (A2D_SELDOM(sm.take(s, was))) {
        asm volatile("" ::: "memory");               // keep this a branch
        if (sm.follow(s, o, was)) {
          fwd_first_keys<HR>(kr, rd, boff);
          fwd_scores<HR>(s, kr, qf, rd, boff);
          to_scores<4, CAP, BIAS, true>(s, sm, r, rs, masked, k0, grp, raw);
          sm.take(s, was);
        }
      }
      fwd_first_values<HR>(vr, rd, boff);
      sm.probabilities(s, pb);
      __builtin_amdgcn_sched_barrier(0);
      fwd_products<HR>(o, pb, vr, rd, boff);
    }
    wait_vmem_all();
    __syncthreads();
    i += stride;
    j = next;
    boff = BUF_BYTES - boff;
  }

  // ---- epilogue: N and l to the true row maximum
  float m_row[2], f[2], l_tot[2];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    sm.finish(q, m_row[q], f[q]);
    l_tot[q] = row_sum(sm.l[q]) * f[q];
  }
  if constexpr (KL == 2) {
    // key lane 1 hands its (N, m, l) to lane 0 through LDS, which merges them as two partials (Alg. 2)
    constexpr int NV = HT * 8 + 4;
    static_assert(RW * NV * 256 <= KL * lds_bytes(HD), "the exchange area must fit the tile buffers");
    float* xch = reinterpret_cast<float*>(lds_all) + wave * NV * 64 + lane;
    if (kl == 1) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
#pragma unroll
        for (int t = 0; t < HT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) xch[(8 * t + 4 * q + e) * 64] = o[t][q][e] * f[q];
        xch[(HT * 8 + 2 * q) * 64] = m_row[q];
        xch[(HT * 8 + 2 * q + 1) * 64] = l_tot[q];
      }
    }
    __syncthreads();
    if (kl == 1) return;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const float m1 = xch[(HT * 8 + 2 * q) * 64], l1 = xch[(HT * 8 + 2 * q + 1) * 64];
      const float m_new = fmaxf(m_row[q], m1);
      const float a0 = (m_row[q] == -INFINITY) ? 0.f : f[q] * fast_exp2(m_row[q] - m_new);
      const float a1 = (m1 == -INFINITY) ? 0.f : fast_exp2(m1 - m_new);
#pragma unroll
      for (int t = 0; t < HT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[t][q][e] = o[t][q][e] * a0 + xch[(8 * t + 4 * q + e) * 64] * a1;
      l_tot[q] = (m_row[q] == -INFINITY ? 0.f : l_tot[q] * fast_exp2(m_row[q] - m_new)) + l1 * a1;
      m_row[q] = m_new;
      f[q] = 1.f;
    }
  }
  // (KL = 2: inside what this wavefront has read of the exchange)
  char* const area = lds_all + wave * (KL == 2 ? (HT * 8 + 4) * 256 : acc_area(HT));
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int row = q0 + wave * 32 + 16 * q, n = map.rows - row;
    const bool stat = grp == 0 && (lane & 15) < n;
    const int64_t at = row0 + row;
    if (r.norm && map.parts == 1) {
      store_acc16(reinterpret_cast<bf16_t*>(out0) + at * H, H, n, area, o, q, lane, l_tot[q] > 0.f ? f[q] / l_tot[q] : 0.f);
      if (stat) out1[at + (lane & 15)] = l_tot[q] > 0.f ? m_row[q] / kLog2e + logf(l_tot[q]) : -INFINITY;
    } else {
      store_acc16(out0 + at * H, H, n, area, o, q, lane, f[q]);
      if (stat) {
        out1[at + (lane & 15)] = m_row[q] / kLog2e;         // -inf stays -inf
        out2[at + (lane & 15)] = l_tot[q];
      }
    }
  }
}

// (pairs of workgroups at H = 64 are three, with 168 registers, where the rules leave room for that: 8192 x 8192, 16 heads, causal, 165 us under
// a bias and 205 under a cap; 189 and 216 as two)
template <int WAVES, int HR, int KL, bool CAP, bool BIAS>
__global__ __launch_bounds__(64 * WAVES, WAVES == 4 && HR == 64 && !(CAP && BIAS) ? 3 : 8 / WAVES) void scored_fwd_kernel(
    a2d_tile_desc d, ScoreRules r, RowMap map, const bf16_t* __restrict__ Q, const bf16_t* __restrict__ K,
    const bf16_t* __restrict__ V, float* out0, float* out1, float* out2, FwdInput in) {
  extern __shared__ __attribute__((aligned(1024))) char lds_all[];
  __shared__ int hull[2 * WAVES];
  __shared__ Ranks ranks;
  constexpr int BM = 32 * WAVES / KL;
  if (map.by_size == BY_RANK) rank_rows(ranks, d, r, map.rows, BM, 64 * WAVES);
  scored_fwd_rows<WAVES, HR, KL, CAP, BIAS>(blockIdx.x, lds_all, hull, ranks, d, r, map, Q, K, V, out0, out1, out2, in);
}

// ---- 32 rows and eight key lanes: for few rows.  Every wavefront holds the same rows and takes every eighth slab of 32 keys,
// which it stages in LDS of its own, without a barrier in the walk (as fwd_small_kernel); the eight (N, m, l) are merged at the end.  Single
// tokens against a long cache are bound by reading it: a compute unit keeps up to 96 KiB (H = 128) of requests in flight.
constexpr int SB = 32;
constexpr int STAT = 8 * 16 * 1024;                  // (slabs, at the end every wavefront's results) | m, l of every wavefront's rows
constexpr int SMALL_LDS = STAT + 2 * 8 * SB * 4;

//
// FINE: both halves of P are contracted, as two bf16 numbers (2^-17 off).  A row of few keys' weight shows the rounding of one: a token
// against 1133 keys is off by 1.49 times what rounding the output alone does, and by 1.0 with two; the walk waits for memory meanwhile
// (256 / 64 heads of 128 against up to 16384 keys: 67 us with either).
template <int HR, bool CAP, bool BIAS, bool FINE>
__global__ __launch_bounds__(512, 1) void scored_fwd_small_kernel(
    a2d_tile_desc d, ScoreRules r, RowMap map, const bf16_t* __restrict__ Q, const bf16_t* __restrict__ K,
    const bf16_t* __restrict__ V, float* out0, float* out1, float* out2, FwdInput in) {
  constexpr int HD = padded_head(HR), H = HR, KS = HD / 32, HT = HR / 16, WAVES = 8, BM = 32;
  constexpr int V_AT = 2 * KS * BLOCK, SLAB_BYTES = 2 * V_AT;
  static_assert(WAVES * SLAB_BYTES <= STAT && HT * 2 <= 16, "slabs and results must fit");
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const unsigned lds_base = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int grp = lane >> 4;

  const int nqb = (map.rows + BM - 1) / BM;
  int unit, blk;
  if (!xcd_map(blockIdx.x, d.heads / r.group * map.parts, map.sub * nqb, map.by_size != 0, unit, blk, kXcdCus)) return;
  const Split up = split_by(unit, map.parts);
  const int kvh = up.q, part = up.r;
  const Split in_group = query_head(blk, map.sub, nqb, map.by_size != 0);
  const int head = kvh * r.group + in_group.r;
  const int q0 = (nqb - 1 - in_group.q) * BM;         // (late ones first)
  Q += (int64_t)head * d.lq.head;
  K += (int64_t)kvh * d.lk.head;
  V += (int64_t)kvh * d.lv.head;
  if (map.parts > 1) {
    const int64_t slot = (int64_t)part * d.heads * d.nq;
    out0 += slot * H;
    out1 += slot;
    out2 += slot;
  }
  const int64_t row0 = (int64_t)head * d.nq;
  const float raw = uniform(d.scale * kLog2e);

  RowState<2> rs;
  look_up_rows<2, BIAS>(rs, d, r, map, head, q0, lane);
  bf16x8 qf[KS][2];
#pragma unroll
  for (int q = 0; q < 2; ++q)
#pragma unroll
    for (int x = 0; x < KS; ++x) {
      const int at = 32 * x + 8 * grp;
      qf[x][q] = *reinterpret_cast<const bf16x8*>(Q + rs.q_at[q] + min(at, H - 8));
      if (32 * x + 32 > H && at >= H) qf[x][q] = bf16x8{};
    }
  if (CAP && A2D_SELDOM(r.capped.lift != 1.f)) {
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int x = 0; x < KS; ++x) lift(qf[x][q], r.capped.lift);
  }
  const int lo = rs.lo, hi = rs.hi;
  const int first = hi > lo ? lo / SB : 1, end = hi > lo ? (hi + SB - 1) / SB : 1;

  const unsigned k_row_bytes = __builtin_amdgcn_readfirstlane((unsigned)d.lk.row * 2);
  const unsigned v_row_bytes = __builtin_amdgcn_readfirstlane((unsigned)d.lv.row * 2);
  const unsigned slab = lds_base + wave * SLAB_BYTES;
  const int ld_chunk = (lane & 3) ^ block_swap(lane >> 4);
  constexpr int LOADS = 2 * KS;                      // of a K or V slab
  auto load = [&](bool v, int j) {
    const unsigned row_bytes = v ? v_row_bytes : k_row_bytes;
    const int from = max(j * SB, lo);
    const gptr_t base = uniform_gptr(reinterpret_cast<const char*>(v ? V : K) + (unsigned)from * row_bytes);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int row = min(max(j * SB + 16 * t + (lane >> 2), lo), hi - 1) - from;
      dma_blocks<KS, H>(slab + (v ? V_AT : 0) + t * KS * BLOCK, base, __umul24(row, row_bytes) + 16 * ld_chunk, ld_chunk);
    }
  };
  if constexpr (H != HD) {
    // the columns of the K slabs past the head size are zero for good (those of V are not read)
    for (int i = lane; i < SB * (HD - H) / 8; i += 64) {
      const int row = i % SB, ch = H % 32 / 8 + i / SB;
      *reinterpret_cast<u32x4*>(lds + wave * SLAB_BYTES + ((row >> 4) * KS + H / 32) * BLOCK + (row & 15) * 64 +
                                16 * (ch ^ block_swap((row & 15) >> 2))) = u32x4{0, 0, 0, 0};
    }
  }
  Blocks16 rd;
  rd.init(lane, slab);

  f32x4 o[HT][2];
#pragma unroll
  for (int t = 0; t < HT; ++t) o[t][0] = o[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
  Softmax sm;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    sm.start(q, -INFINITY);
    sm.l[q] = 0.f;
  }
  if (r.acc && part == 0 && wave == 0) {
    // the first wavefront continues the stored partial
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int row = q0 + 16 * q + (lane & 15);
      if (row >= map.rows) continue;
      sm.start(q, in.m[row0 + row]);
      sm.l[q] = grp == 0 ? in.l[row0 + row] : 0.f;
#pragma unroll
      for (int t = 0; t < HT; ++t) o[t][q] = *reinterpret_cast<const f32x4*>(in.N + (row0 + row) * H + 16 * t + 4 * grp);
    }
  }
  wait_vmem_all();                                   // (Q, and what an accumulating call starts from: the waits below count slabs alone)
  const int stride = WAVES * map.parts;
  int j = end - 1 - part * WAVES - wave;             // (from the last block down, as scored_fwd_rows)
  if (j >= first) {
    load(false, j);
    load(true, j);
    wait_dma<LOADS>();                               // (K)
  }
  // the next K goes where the last one was read from while the exponentials and V P^T are under way, the next V behind those
  for (; j >= first; j -= stride) {
    const bool more = j - stride >= first;
    const int k0 = j * SB;
    f32x4 s[2][2];
#pragma unroll
    for (int k = 0; k < 2; ++k) s[k][0] = s[k][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < KS; ++x)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const bf16x8 a = lds_load_b128(rd.nat + (k * KS + x) * BLOCK);
#pragma unroll
        for (int q = 0; q < 2; ++q) s[k][q] = mma16(a, qf[x][q], s[k][q]);
      }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more) load(false, j - stride);
    const f32x4 z[2][2] = {{s[0][0], s[0][1]}, {s[1][0], s[1][1]}};
    const bool masked = k0 < rs.all_lo || k0 + SB > rs.all_hi;
    to_scores<2, CAP, BIAS>(s, sm, r, rs, masked, k0, grp, raw);
    float was[2];
    if (A2D_SELDOM(sm.take(s, was))) {
      asm volatile("" ::: "memory");                 // keep this a branch
      if (sm.follow(s, o, was)) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int q = 0; q < 2; ++q) s[k][q] = z[k][q];
        to_scores<2, CAP, BIAS, true>(s, sm, r, rs, masked, k0, grp, raw);
        sm.take(s, was);
      }
    }
    bf16x8 pb[1][2], rest[1][2];
    if constexpr (FINE) sm.probabilities(s, pb, rest);
    else sm.probabilities(s, pb);
    __builtin_amdgcn_sched_barrier(0);
    if (more) wait_dma<LOADS>(); else wait_dma();    // V has arrived
#pragma unroll
    for (int t = 0; t < HT; ++t) {
      const unsigned at = (t & 1 ? rd.tr_o : rd.tr_e) + V_AT + (t >> 1) * BLOCK;
      const bf16x8 a = lds_load_tr(at, at + KS * BLOCK);
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        o[t][q] = mma16(a, pb[0][q], o[t][q]);
        if constexpr (FINE) o[t][q] = mma16(a, rest[0][q], o[t][q]);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more) {
      load(true, j - stride);
      wait_dma<LOADS>();
    }
  }

  // ---- the wavefronts' (N, m, l) become one (Alg. 2)
  float* const xm = reinterpret_cast<float*>(lds + STAT) + (lane & 31);
  float* const xl = xm + WAVES * 32;
  float m_row[2], l_row[2], f[2];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    sm.finish(q, m_row[q], f[q]);
    l_row[q] = row_sum(sm.l[q]) * f[q];
  }
  if (lane < 32) {                                   // (lanes 0 .. 15 hold tile 0's rows, 16 .. 31 tile 1's)
    xm[wave * 32] = m_row[grp & 1];
    xl[wave * 32] = l_row[grp & 1];
  }
  __syncthreads();
  f32x4* const x = reinterpret_cast<f32x4*>(lds);
  const bool norm = r.norm && map.parts == 1;
  float m_new = -INFINITY, l_tot = 0.f, use[2], fn[2] = {0.f, 0.f};
#pragma unroll
  for (int k = 0; k < WAVES; ++k) m_new = fmaxf(m_new, xm[k * 32]);
  const float m_use = m_new == -INFINITY ? 0.f : m_new;
  row_pair(m_use, use);
  if (norm || wave == 0) {
#pragma unroll
    for (int k = 0; k < WAVES; ++k) l_tot += xl[k * 32] * fast_exp2(xm[k * 32] - m_use);
    row_pair(l_tot > 0.f ? 1.0f / l_tot : 0.f, fn);
  }
  if (wave == 0 && lane < 32 && q0 + lane < map.rows) {
    const int64_t row = row0 + q0 + lane;
    if (norm) out1[row] = l_tot > 0.f ? m_new / kLog2e + logf(l_tot) : -INFINITY;
    else {
      out1[row] = m_new / kLog2e;
      out2[row] = l_tot;
    }
  }
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const float a = f[q] * fast_exp2(m_row[q] - use[q]);
    // every wavefront leaves its pieces of four columns, [wavefront][piece][lane], and adds up and stores two of them
#pragma unroll
    for (int t = 0; t < HT; ++t)
      x[(wave * 16 + 2 * t + q) * 64 + lane] = f32x4{o[t][q][0] * a, o[t][q][1] * a, o[t][q][2] * a, o[t][q][3] * a};
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int piece = wave + WAVES * i, q = piece & 1, col = 16 * (piece >> 1) + 4 * grp, row = q0 + 16 * q + (lane & 15);
    if (piece >= 2 * HT || row >= map.rows) continue;
    f32x4 v = x[piece * 64 + lane];
#pragma unroll
    for (int k = 1; k < WAVES; ++k) {
      const f32x4 w = x[(k * 16 + piece) * 64 + lane];
      v[0] += w[0]; v[1] += w[1]; v[2] += w[2]; v[3] += w[3];
    }
    const int64_t at = (row0 + row) * H + col;
    if (norm) {
      const float by = q ? fn[1] : fn[0];
      bf16x4 b;
#pragma unroll
      for (int e = 0; e < 4; ++e) b[e] = (bf16_t)(v[e] * by);
      *reinterpret_cast<bf16x4*>(reinterpret_cast<bf16_t*>(out0) + at) = b;
    } else {
      *reinterpret_cast<f32x4*>(out0 + at) = v;
    }
  }
}

constexpr int kRows[4] = {256, 128, 128, 32};

template <int HR, bool CAP, bool BIAS>
hipError_t go(Phase ph, const a2d_tile_desc& d, const ScoreRules& r, const ScoredPlan& plan, const void* Q, const void* K, const void* V,
              float* out0, float* out1, float* out2, const FwdInput& in, hipStream_t s) {
  const int bm = kRows[plan.form];
  const RowMap map = row_map(d, r, bm, plan.parts);
  const int waves = plan.form == SCORED_PAIRS ? 4 : 8;
  const int bytes = plan.form == SCORED_32 ? SMALL_LDS : fwd_lds(waves, padded_head(HR), plan.form == SCORED_LANES ? 2 : 1);
  const auto run = [&](auto* kernel) {
    if (ph == PREPARE) return ensure_dynamic_lds(reinterpret_cast<const void*>(kernel), bytes);
    const int units = d.heads / r.group * map.parts, blocks = map.sub * ((map.rows + bm - 1) / bm);
    const dim3 grid(xcd_grid(units, blocks));
    A2D_LAUNCH(kernel, grid, dim3(64 * waves), bytes, s, d, r, map, (const bf16_t*)Q, (const bf16_t*)K, (const bf16_t*)V, out0, out1, out2, in);
    return hipGetLastError();
  };
  return plan.form == SCORED_256     ? run(scored_fwd_kernel<8, HR, 1, CAP, BIAS>)
         : plan.form == SCORED_LANES ? run(scored_fwd_kernel<8, HR, 2, CAP, BIAS>)
         : plan.form == SCORED_PAIRS ? run(scored_fwd_kernel<4, HR, 1, CAP, BIAS>)
         : plan.fine                 ? run(scored_fwd_small_kernel<HR, CAP, BIAS, true>)
                                     : run(scored_fwd_small_kernel<HR, CAP, BIAS, false>);
}

}  // namespace

// Every form's time from its turns of the chip (walk_time), the quickest.  Steps in us, of 64 keys (of 128 and 256 in the forms with key
// lanes), by head size and rules, fitted to 40 calls timed in every form.  What they choose between, measured: 8192 x 8192 rows of
// 16 heads of 64 in six documents 76 us in pairs, 90 with 256 rows (the pairs' turns are half as long), 102 in two key lanes; 16384 x 16384, 8
// heads of 128: 491 with 256 rows, 512 in pairs; 13611 x 14346, 4 of 80, causal: 156 in two key lanes, 207 in pairs, 273 with 256 rows;
// a token of 256 / 64 heads of 64 against up to 16384 keys: 30 with 32 rows in four parts, 67 in one, 196 with 256.  Ranges that the
// host cannot see: one set for all heads is taken for documents, which see a part of the keys each (749 x 9939: 13 us in one part, 21 where
// a plan for whole walks split them; see taken_for_documents); one a sequence for its filled length.
static ScoredPlan best_form(const a2d_tile_desc& d, const ScoreRules& r, int cus, int cap, bool rows_of_32) {
  constexpr struct {
    double step, by_head, fixed, pair;                // pair: both workgroups of a compute unit, of one's time
    int keys;
  } kForms[4] = {{0.95, 0.95, 4.0, 0, 64}, {0.9, 1.15, 7.5, 0, 128}, {0.5, 0.95, 4.0, 1.4, 64}, {1.0, 0.8, 3.7, 0, 256}};
  const int kv_heads = d.heads / r.group;
  const WalkKeys walk = walk_keys(d, r);
  const double part_us = (double)d.heads * d.nq * (d.hdim + 2) * 8 / 4.5e6;
  double least = 0;
  ScoredPlan best{SCORED_32, 1, false};
  const int only = rows_of_32 ? SCORED_32 : SCORED_256;
  for (int f = only; f < 4; ++f) {
    const auto& form = kForms[f];
    const int bm = kRows[f];
    const bool packed = r.group > 1 && d.nq < bm;
    const int64_t blocks = packed ? (int64_t)kv_heads * (((int64_t)r.group * d.nq + bm - 1) / bm)
                                  : (int64_t)d.heads * ((d.nq + bm - 1) / bm);
    double most = walk.most, mean = packed ? most : walk.mean;
    if (taken_for_documents(d, r) && !packed) {
      most *= 0.35;
      mean *= 0.25;
    }
    const double step = form.step + form.by_head * d.hdim / 128 + 0.2 * ((r.cap != 0.f) + (r.slopes != nullptr));
    const WalkModel m{blocks, cus, mean / form.keys + 0.2, most / form.keys + 0.2, step, form.fixed, form.pair * step,
                      form.pair != 0 ? form.fixed : 0, nullptr, 0, 0.4};
    double t;
    const int parts = best_parts(m, cap, 4.5, part_us, &t);
    if (f == only || t < least) {
      least = t;
      best = ScoredPlan{f, parts, false};
    }
  }
  return best;
}

// How P is rounded is a matter of the call, not of the memory that there happens to be: fine are calls of few rows - a workgroup's 32 for
// a key/value head, whatever is quickest - and those that go to 32 rows with memory for their parts.
ScoredPlan plan_scored_fwd(const a2d_tile_desc& d, const ScoreRules& r, int cus, int cap, bool scratch) {
  const bool few = (r.group > 1 ? (int64_t)r.group * d.nq : d.nq) <= kRows[SCORED_32];
  ScoredPlan plan = best_form(d, r, cus, cap, few);
  plan.fine = plan.form == SCORED_32;
  if (scratch || plan.parts == 1) return plan;
  ScoredPlan whole = best_form(d, r, cus, 1, plan.fine);
  whole.fine = plan.fine;
  return whole;
}

void route_scored_fwd(const a2d_tile_desc& d, const ScoreRules& r, const ScoredPlan& plan, ScoredRoute* out) {
  const int bm = kRows[plan.form];
  const RowMap map = row_map(d, r, bm, plan.parts);
  *out = ScoredRoute{};
  out->kernel[out->kernels++] = plan.form == SCORED_32 ? "scored_fwd_small_kernel" : "scored_fwd_kernel";
  out->rows = bm;
  out->lanes = plan.form == SCORED_32 ? 8 : plan.form == SCORED_LANES ? 2 : 1;
  out->waves = plan.form == SCORED_PAIRS ? 4 : 8;
  out->order = plan.form == SCORED_32 && map.by_size ? BY_ROWS : map.by_size;
  out->blocks_q = map.sub * ((map.rows + bm - 1) / bm);
  out->units_q = out->blocks_q * plan.parts;
  out->fine = plan.fine;
}

hipError_t launch_scored_fwd(Phase ph, const a2d_tile_desc& d, const ScoreRules& r, const ScoredPlan& plan, const void* Q, const void* K,
                             const void* V, float* out0, float* out1, float* out2, const FwdInput& in, hipStream_t s) {
#define A2D_RULES(HR)                                                                                  \
  return r.cap != 0.f ? (r.slopes ? go<HR, true, true>(ph, d, r, plan, Q, K, V, out0, out1, out2, in, s)   \
                                  : go<HR, true, false>(ph, d, r, plan, Q, K, V, out0, out1, out2, in, s)) \
                      : (r.slopes ? go<HR, false, true>(ph, d, r, plan, Q, K, V, out0, out1, out2, in, s)  \
                                  : go<HR, false, false>(ph, d, r, plan, Q, K, V, out0, out1, out2, in, s))
  if (d.hdim == 128) { A2D_RULES(128); }
  if (d.hdim == 96) { A2D_RULES(96); }
  if (d.hdim == 80) { A2D_RULES(80); }
  A2D_RULES(64);
#undef A2D_RULES
}

}  // namespace a2d
