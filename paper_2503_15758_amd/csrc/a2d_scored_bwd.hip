// bf16 backward tile under score rules (a2d_score_rules in a2d.h) on the matrix units, H = 128, 96, 80 and 64.
//
// P = 2^(y - bias - lse) and dP as ever; with t = tanh(z / cap), the gradient of a raw product is dZ = P (1 - t^2) (dP - delta), so a
// cap costs the polynomial again (see CapArgs) and three vector instructions.  Two kernels, both recomputing S and dP (7 contractions for
// the 5 of the definition): scored_dq_kernel, whose wavefronts own 32 query rows and walk the keys of their hull, and
// scored_dkdv_kernel, whose wavefronts own 32 keys and walk the query rows.  (Structure, fragments and staging: dq_rows and dkdv_wide.)
//
// Masks.  The dQ kernel looks up what each row sees and leaves it for the other one: per row its run of keys, lse and delta in the
// units that are used (a row that sees nothing: lse = +inf, so that its P is 0), per 32 rows the hull of their runs and the keys that
// all of them see.  From the hulls a dK / dV workgroup makes a bit for every step of 64 query rows, and walks the set ones: documents cost
// nothing but their own scores, wherever they lie.  Rows that see nothing are zeros in front of every product, so they may hold anything;
// so may keys that no row sees: dQ reads none outside a block's hull, dK / dV hold those of every block (asked for before the steps that see
// one are known) and leave out what an unseen one would take part in.
//
// Bound: of 4096 x 4096, 32 / 8 of 128, causal under a cap, 535 us, vector and matrix instructions of two wavefronts a SIMD that share its issue
// (matrix units busy 43 % of dQ's time and 38 % of dK / dV's, vector ALUs 62 % and 48 %).  Documents, by their longest walk: 8192 x 8192, 16 heads of
// 128 in four, 347 us (660 TFLOP/s of the five contractions; 41 % and 35 %, 31 % and 27 %; 1.6 wavefronts a SIMD: up to 66 steps where an even
// share were 51); below some hundred million scores also by what a workgroup costs besides, and launches: 2999 x 2999, 12 / 4 of
// 80 in four documents 76.
#include "a2d_bwd.hpp"
#include "a2d_scored_rows.hpp"

namespace a2d {
namespace {

using namespace mfma;

// z -> y in log2 units, of 2 x 2 tiles
__device__ __forceinline__ void cap_in_place(f32x4 (&s)[2][2], const CapArgs& a) {
  float big = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) big = fmaxf(big, fabsf(s[e >> 3][(e >> 2) & 1][e & 3]));
  if (A2D_SELDOM(__builtin_amdgcn_ballot_w64(big > a.small) != 0)) {
    asm volatile("" ::: "memory");                   // keep this a branch
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e >> 3][(e >> 2) & 1][e & 3] = cap_log2(a, s[e >> 3][(e >> 2) & 1][e & 3]);
      if (e & 1) __builtin_amdgcn_sched_barrier(0);  // (more at a time takes registers that dK and dV need)
    }
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e >> 3][(e >> 2) & 1][e & 3] *= cap_factor(a, s[e >> 3][(e >> 2) & 1][e & 3]);
      if ((e & 3) == 3) __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// ------------------------------------------------------------------------------------------------ dQ

constexpr int BKS = 64;                              // keys per step
__host__ __device__ constexpr int dq_buf(int hd) { return 2 * BKS * 2 * hd; }      // { K tile, V tile }, in blocks
__host__ __device__ constexpr int dq_launch_lds(int hd, int kl) {
  return kl * 2 * dq_buf(hd) > 8 * acc_area(hd / 16) ? kl * 2 * dq_buf(hd) : 8 * acc_area(hd / 16);
}
__host__ __device__ constexpr int dq_ring(int hd) { return hd == 64 ? 4 : 2; }

// KL = 1: 256 rows, KL = 2: 128 rows in two key lanes (see scored_fwd_kernel)
template <int HR, int KL, bool CAP, bool BIAS, bool FINE>
__device__ __forceinline__ void scored_dq_rows(
    int id, char* const lds_all, int* const hull, Shares& shares, const a2d_tile_desc& d, const ScoreRules& r, const Cut& cut, int in_order,
    const RowTable& tab, const bf16_t* __restrict__ Q, const bf16_t* __restrict__ K, const bf16_t* __restrict__ V,
    const bf16_t* __restrict__ O, const bf16_t* __restrict__ dO, const float* __restrict__ lse, void* dQ, float* __restrict__ more,
    int2* __restrict__ table) {
  constexpr int WAVES = 8, RW = WAVES / KL, BM = 32 * RW, kThreads = 64 * RW;
  constexpr int HD = padded_head(HR), H = HR, KS = HD / 32, HT = HR / 16, DQ_BUF = dq_buf(HD), RING = dq_ring(HD);
  const int kl = KL == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x / kThreads);
  char* const lds = lds_all + kl * (2 * DQ_BUF);
  const unsigned lds_base = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  int kvh, at_unit;
  if (!xcd_map(id, d.heads / r.group, r.group * cut.units, in_order, kvh, at_unit, kXcdCus)) return;
  const Split in_group = query_head(at_unit, r.group, cut.units, in_order);
  const int head = kvh * r.group + in_group.r;
  // longest walks first, as far as they are known (late rows)
  if (cut.parts == 0) weigh_rows(shares.ranks, d, r, d.nq, BM, 512);
  const Share mine = cut.parts == 0 ? share_out(shares, cut, in_group.q) : share_evenly(cut, in_group.q, true);
  if (mine.parts == 0) return;
  const int q0 = mine.block * BM, part = mine.part, parts = mine.parts;
  if (table && head == 0 && part == 0 && threadIdx.x == 0) table[mine.block] = int2{mine.slot, parts};
  const int tid = (int)threadIdx.x - kl * kThreads;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, grp = lane >> 4;
  Q += (int64_t)head * d.lq.head;
  O += (int64_t)head * d.lo.head;
  dO += (int64_t)head * d.ldo.head;
  K += (int64_t)kvh * d.lk.head;
  V += (int64_t)kvh * d.lv.head;
  const float raw = uniform(d.scale * kLog2e), inv_top = CAP ? 1.f / r.capped.top : 0.f;
  const float slope = BIAS ? uniform(r.slopes[head] * kLog2e) : 0.f;

  // ---- the rows: fragments, delta, what they see
  const int w0 = q0 + wave * 32;
  bf16x8 qf[KS][2], gf[KS][2];
  f32x4 start[2];                                      // -delta: what dP starts from
  float lse2[2], from[2];
  Run run[2];
  int lo = INT_MAX, hi = 0, all_lo = 0, all_hi = INT_MAX;
  unsigned live_rows = 0;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int row = w0 + 16 * q + (lane & 15), in = min(row, d.nq - 1);
    bf16x8 of[KS];
#pragma unroll
    for (int x = 0; x < KS; ++x) {
      const int at = 32 * x + 8 * grp, ld = min(at, H - 8);
      qf[x][q] = *reinterpret_cast<const bf16x8*>(Q + (int64_t)in * d.lq.row + ld);
      gf[x][q] = *reinterpret_cast<const bf16x8*>(dO + (int64_t)in * d.ldo.row + ld);
      of[x] = *reinterpret_cast<const bf16x8*>(O + (int64_t)in * d.lo.row + ld);
      if (32 * x + 32 > H && at >= H) qf[x][q] = gf[x][q] = of[x] = bf16x8{};
    }
    const float L = lse[(int64_t)head * d.nq + in];
    run[q] = visible_run(d, r, head, in);
    if (row >= d.nq || L == -INFINITY) run[q].n = 0;
    const bool live = run[q].n > 0;
    live_rows |= ((unsigned)__builtin_amdgcn_ballot_w64(live) & 0xFFFFu) << (16 * q);
    float del = 0.f;
#pragma unroll
    for (int x = 0; x < KS; ++x) del = dot8(__builtin_bit_cast(u32x4, of[x]), __builtin_bit_cast(u32x4, gf[x][q]), del);
    del = row_sum(del);
    if (!live) del = 0.f;
    lse2[q] = live ? L * kLog2e : INFINITY;            // +inf: P = 0
    if (!live) {
#pragma unroll
      for (int x = 0; x < KS; ++x) qf[x][q] = gf[x][q] = bf16x8{};
    }
    if (CAP && A2D_SELDOM(r.capped.lift != 1.f)) {
#pragma unroll
      for (int x = 0; x < KS; ++x) lift(qf[x][q], r.capped.lift);
    }
    start[q] = f32x4{-del, -del, -del, -del};
    if (BIAS) from[q] = (float)(int)(r.rel + (int64_t)in * r.step);
    if (live) {
      lo = min(lo, run[q].lo);
      hi = max(hi, run[q].lo + run[q].n);
      all_lo = max(all_lo, run[q].lo);
      all_hi = min(all_hi, run[q].lo + run[q].n);
    }
    if (part == 0 && kl == 0 && grp == 0 && row < tab.padded) {
      const int64_t at = (int64_t)head * tab.padded + row;
      tab.from[at] = CAP ? lse2[q] : live ? -L / d.scale : -INFINITY;
      tab.delta[at] = -del;
      tab.lo[at] = run[q].lo;
      tab.n[at] = run[q].n;
    }
  }
  const auto least = [](int a, int b) { return min(a, b); };
  const auto most = [](int a, int b) { return max(a, b); };
  lo = over16(lo, least);
  hi = over16(hi, most);
  all_lo = over16(all_lo, most);
  all_hi = over16(all_hi, least);
  if (kl == 0 && lane == 0) {
    if (part == 0 && w0 < tab.padded) tab.tiles[((int64_t)head * tab.padded + w0) / 32] = RowTile{lo, hi, all_lo, all_hi, live_rows, {0, 0, 0}};
    hull[2 * wave] = lo;
    hull[2 * wave + 1] = hi;
  }
  if constexpr (H != HD) {                             // columns past the head size are zero for good
    for (int i = tid; i < 4 * BKS * (HD - H) / 8; i += kThreads) {
      const int row = i % BKS, x = i / BKS, tile = x / ((HD - H) / 8), ch = H % 32 / 8 + x % ((HD - H) / 8);
      *reinterpret_cast<u32x4*>(lds + tile * (DQ_BUF / 2) + ((row >> 4) * KS + H / 32) * BLOCK + (row & 15) * 64 +
                                16 * (ch ^ block_swap((row & 15) >> 2))) = u32x4{0, 0, 0, 0};
    }
  }
  __syncthreads();
  int wg_lo = INT_MAX, wg_hi = 0;
#pragma unroll
  for (int w = 0; w < RW; ++w) {
    wg_lo = min(wg_lo, hull[2 * w]);
    wg_hi = max(wg_hi, hull[2 * w + 1]);
  }
  wg_lo = __builtin_amdgcn_readfirstlane(wg_lo);
  wg_hi = __builtin_amdgcn_readfirstlane(wg_hi);
  const bool some = wg_hi > wg_lo;
  const int first = some ? wg_lo / BKS : 0, end = some ? (wg_hi + BKS - 1) / BKS : 0;

  f32x4 dq[HT][2];
#pragma unroll
  for (int t = 0; t < HT; ++t) dq[t][0] = dq[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
  Blocks16 ka;                                         // K tile of the current buffer (V's stands DQ_BUF / 2 behind it)
  ka.init(lane, lds_base);

  // ---- staging (as in scored_fwd_kernel)
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
    const int at = max(j * BKS, wg_lo), row = min(max(j * BKS + ld_row, wg_lo), wg_hi - 1) - at;
#pragma unroll
    for (int x = 0; x < LD_N; ++x)
      dma_blocks<KS, H>(lds_base + boff + (4 * (ld_first + x) + ld_tile) * KS * BLOCK,
                        uniform_gptr(ld_base[x] + (unsigned)at * ld_row_bytes[x]), __umul24(row, ld_row_bytes[x]) + 16 * ld_chunk, ld_chunk);
  };

  // one 32-key x 32-query piece, half T of the step at key0 - 32 T (as dq_piece): S^T and dP^T in tiles of 16 keys (k) x 16 queries (q)
  auto piece = [&](auto TT, int key0) {
    constexpr int T = decltype(TT)::value, N = 2 * KS, RB = T * 2 * KS * BLOCK, VT = DQ_BUF / 2;
    bf16x8 kr[RING], vr[RING], kt[RING];
    auto ld1 = [&](auto X) {
      constexpr int x = decltype(X)::value;
      const unsigned at = ka.nat + RB + ((x & 1) * KS + (x >> 1)) * BLOCK;
      kr[x % RING] = lds_load_b128(at);
      vr[x % RING] = lds_load_b128(at + VT);
      __builtin_amdgcn_sched_barrier(0);
    };
    auto ld2 = [&](auto I) {
      constexpr int i = decltype(I)::value;
      const unsigned at = (i & 1 ? ka.tr_o : ka.tr_e) + RB + (i >> 1) * BLOCK;
      kt[i % RING] = lds_load_tr(at, at + KS * BLOCK);
      __builtin_amdgcn_sched_barrier(0);
    };
    static_for<0, RING>(ld1);
    f32x4 s[2][2], dp[2][2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int q = 0; q < 2; ++q) { s[k][q] = f32x4{0.f, 0.f, 0.f, 0.f}; dp[k][q] = start[q]; }
    static_for<0, N>([&](auto X) {
      constexpr int x = decltype(X)::value, k = x & 1;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        s[k][q] = mma16(kr[x % RING], qf[x >> 1][q], s[k][q]);
        dp[k][q] = mma16(vr[x % RING], gf[x >> 1][q], dp[k][q]);
      }
      if constexpr (x + RING < N) ld1(std::integral_constant<int, x + RING>{});
      else ld2(std::integral_constant<int, x + RING - N>{});
    });
    if constexpr (CAP) cap_in_place(s, r.capped);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const float base = BIAS ? fmaf((float)-(key0 + 4 * grp), r.steps[0], from[q]) : 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y = s[e >> 2][q][e & 3];
        float x = CAP ? y - lse2[q] : fmaf(y, raw, -lse2[q]);
        if constexpr (BIAS) x = fmaf(-slope, fabsf(distance<-1>(r, base, e >> 2, e & 3)), x);
        float p = fast_exp2(x);
        if constexpr (CAP) {
          const float t = y * inv_top;
          p = fmaf(-p * t, t, p);
        }
        s[e >> 2][q][e & 3] = p * dp[e >> 2][q][e & 3];
      }
    }
    if (A2D_SELDOM(key0 < all_lo || key0 + 32 > all_hi)) {
      asm volatile("" ::: "memory");                   // keep this a branch
#pragma unroll
      for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int key = key0 + 16 * (e >> 2) + 4 * grp + (e & 3) - run[q].lo;
          s[e >> 2][q][e & 3] = (unsigned)key < (unsigned)run[q].n ? s[e >> 2][q][e & 3] : 0.f;
        }
    }
    bf16x8 dsb[2], rest[2];                            // dZ is rounded to the inputs' type, as P is (FINE: see fine_call)
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        dsb[q][e] = (bf16_t)s[e >> 2][q][e & 3];
        if constexpr (FINE) rest[q][e] = (bf16_t)(s[e >> 2][q][e & 3] - (float)dsb[q][e]);
      }
    __builtin_amdgcn_sched_barrier(0);
    static_for<0, HT>([&](auto I) {
      constexpr int i = decltype(I)::value;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        dq[i][q] = mma16(kt[i % RING], dsb[q], dq[i][q]);
        if constexpr (FINE) dq[i][q] = mma16(kt[i % RING], rest[q], dq[i][q]);
      }
      if constexpr (i + RING < HT) ld2(std::integral_constant<int, i + RING>{});
    });
  };

  const int stride = KL * parts;
  int lead = first + part * KL, j = lead + kl;
  if (j < end) load_tile(j, 0);
  wait_vmem_all();
  __syncthreads();
  int boff = 0;
  for (; lead < end; lead += stride) {
    if (A2D_OFTEN(j + stride < end)) load_tile(j + stride, DQ_BUF - boff);
    const int k0 = j * BKS;
    if (j < end && k0 + 32 > lo && k0 < hi) piece(std::integral_constant<int, 0>{}, k0);
    if (j < end && k0 + 64 > lo && k0 + 32 < hi) piece(std::integral_constant<int, 1>{}, k0 + 32);
    const int tog = boff ? -DQ_BUF : DQ_BUF;
    ka.nat += tog; ka.tr_e += tog; ka.tr_o += tog;
    boff = DQ_BUF - boff;
    wait_vmem_all();
    __syncthreads();
    j += stride;
  }
  if constexpr (KL == 2) {
    // lane 1 hands its sums to lane 0 through LDS
    static_assert(RW * HT * 8 * 256 <= KL * 2 * DQ_BUF, "the exchange area must fit the tile buffers");
    float* xch = reinterpret_cast<float*>(lds_all) + wave * (HT * 8 * 64) + lane;
    if (kl == 1) {
#pragma unroll
      for (int t = 0; t < HT; ++t)
#pragma unroll
        for (int e = 0; e < 8; ++e) xch[(8 * t + e) * 64] = dq[t][e >> 2][e & 3];
    }
    __syncthreads();
    if (kl == 1) return;
#pragma unroll
    for (int t = 0; t < HT; ++t)
#pragma unroll
      for (int e = 0; e < 8; ++e) dq[t][e >> 2][e & 3] += xch[(8 * t + e) * 64];
  }
  char* const area = lds_all + wave * (KL == 2 ? HT * 8 * 256 : acc_area(HT));
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const int row = w0 + 16 * q;
    const int64_t at = ((int64_t)head * d.nq + row) * H;
    if (parts > 1) store_acc16(more + (((int64_t)head * cut.units + mine.slot + part) * BM + row - q0) * H, H, d.nq - row, area, dq, q, lane, d.scale);
    else if (r.norm) store_acc16(static_cast<bf16_t*>(dQ) + at, H, d.nq - row, area, dq, q, lane, d.scale);
    else store_acc16(static_cast<float*>(dQ) + at, H, d.nq - row, area, dq, q, lane, d.scale, r.acc != 0);
  }
}

template <int HR, int KL, bool CAP, bool BIAS, bool FINE>
__global__ __launch_bounds__(512, 1) void scored_dq_kernel(
    a2d_tile_desc d, ScoreRules r, Cut cut, int in_order, RowTable tab, const bf16_t* __restrict__ Q, const bf16_t* __restrict__ K,
    const bf16_t* __restrict__ V, const bf16_t* __restrict__ O, const bf16_t* __restrict__ dO, const float* __restrict__ lse,
    void* dQ, float* __restrict__ more, int2* __restrict__ table) {
  extern __shared__ __attribute__((aligned(1024))) char lds_all[];
  __shared__ int hull[16];
  __shared__ Shares shares;
  scored_dq_rows<HR, KL, CAP, BIAS, FINE>(blockIdx.x, lds_all, hull, shares, d, r, cut, in_order, tab, Q, K, V, O, dO, lse, dQ, more, table);
}

// --------------------------------------------------------------------------------------------- dK, dV

constexpr int WK_KEYS = 256, WK_THREADS = 512, WK_ROWS = 64;
__host__ __device__ constexpr int wk_tile(int hd) { return WK_ROWS * 2 * hd; }
// LDS: two buffers { Q tile, dO tile } in blocks | two of { from [64], -delta [64], lo [64], n [64] } | two of two RowTiles | bits
// (64-bit words) of the steps.  (At the end 16 keys of every wavefront go out at a time.)
constexpr int WK_STAT = 4 * WK_ROWS * 4, WK_TILES = 2 * sizeof(RowTile);
__host__ __device__ constexpr int wk_stat(int hd) { return 4 * wk_tile(hd); }
__host__ __device__ constexpr int wk_bits(int hd) {
  const int walk = wk_stat(hd) + 2 * WK_STAT + 2 * WK_TILES, rows = 8 * acc_area(hd / 16);
  return walk > rows ? walk : rows;
}

// slices of H whose K^T and V^T fragments wait in LDS, behind the bits
__host__ __device__ constexpr int wk_park(int hd) { return hd == 128 ? 1 : 0; }
__host__ __device__ constexpr int wk_lds(int hd) { return wk_bits(hd) + SCORED_MOST_BITS + wk_park(hd) * 8 * 4 * BLOCK; }

// weights of the key blocks (the same for all heads): row tiles that see one, +1 at the first block of a tile's hull, -1 behind its last, summed up
__device__ __forceinline__ void weigh_keys(Ranks& ranks, const ScoreRules& r, const Cut& cut, const RowTable& tab) {
  const int tid = threadIdx.x;
  for (int i = tid; i < cut.blocks; i += WK_THREADS) ranks.weight[i] = 0;
  __syncthreads();
  for (int i = tid; i < tab.padded / 32; i += WK_THREADS) {
    const int lo = tab.tiles[i].lo, hi = tab.tiles[i].hi;
    if (lo >= hi) continue;
    atomicAdd(&ranks.weight[lo / WK_KEYS], r.group);
    if ((hi - 1) / WK_KEYS + 1 < cut.blocks) atomicAdd(&ranks.weight[(hi - 1) / WK_KEYS + 1], -r.group);
  }
  __syncthreads();
  int sum = 0;
  if (tid < cut.blocks)
    for (int j = 0; j <= tid; ++j) sum += ranks.weight[j];
  __syncthreads();
  if (tid < cut.blocks) ranks.weight[tid] = sum;
}

template <int HR, bool CAP, bool BIAS, bool FINE>
__device__ __forceinline__ void scored_dkdv_keys(
    int id, char* const lds, Shares& shares, const a2d_tile_desc& d, const ScoreRules& r, const Cut& cut, int in_order, const RowTable& tab,
    const bf16_t* __restrict__ Q, const bf16_t* __restrict__ K, const bf16_t* __restrict__ V, const bf16_t* __restrict__ dO,
    void* __restrict__ dK, void* __restrict__ dV, float* __restrict__ more, int2* __restrict__ table) {
  const unsigned lds_base = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  constexpr int HD = padded_head(HR), H = HR, TILE = wk_tile(HD), BUF = 2 * TILE;
  constexpr int KS = HD / 32, HT = HR / 16;
  constexpr bool TIGHT = HD == 128;                  // registers (see dkdv_wide)
  const int kv_heads = d.heads / r.group;
  int head, at_unit;
  if (!xcd_map(id, kv_heads, cut.units, in_order, head, at_unit)) return;
  if (cut.parts == 0) weigh_keys(shares.ranks, r, cut, tab);
  const Share mine = cut.parts == 0 ? share_out(shares, cut, at_unit) : share_evenly(cut, at_unit, false);
  if (mine.parts == 0) return;
  const int part = mine.part, parts = mine.parts, qh0 = head * r.group;
  const int k0 = mine.block * WK_KEYS;
  if (table && head == 0 && part == 0 && threadIdx.x == 0) table[mine.block] = int2{mine.slot, parts};
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int l16 = lane & 15, grp = lane >> 4;
  Q += (int64_t)qh0 * d.lq.head;
  dO += (int64_t)qh0 * d.ldo.head;
  K += (int64_t)head * d.lk.head;
  V += (int64_t)head * d.lv.head;
  const float raw = uniform(d.scale * kLog2e), inv_top = CAP ? uniform(1.f / r.capped.top) : 0.f;

  // ---- the steps of 64 query rows, of all query heads one after another, that see a key of the workgroup: a bit each
  const int nsteps = tab.padded / WK_ROWS, all_steps = nsteps * r.group, words = (all_steps + 63) / 64;
  uint64_t* const bits = reinterpret_cast<uint64_t*>(lds + wk_bits(HD));
  const RowTile* const tiles = tab.tiles + (int64_t)qh0 * (tab.padded / 32);
  for (int w = wave; w < words; w += 8) {
    const int s = 64 * w + lane;
    bool seen = false;
    if (s < all_steps) {
      const RowTile &a = tiles[2 * s], &b = tiles[2 * s + 1];    // (a head's tiles follow the one before's: 2 a step)
      const int al = a.lo, ah = a.hi, bl = b.lo, bh = b.hi;
      seen = (al < ah && al < k0 + WK_KEYS && ah > k0) || (bl < bh && bl < k0 + WK_KEYS && bh > k0);
    }
    const uint64_t m = __builtin_amdgcn_ballot_w64(seen);
    if (lane == 0) bits[w] = m;
  }

  // ---- K^T and V^T fragments of the wavefront's 32 keys, two tiles of 16: lane = key.  Keys beyond nkv re-read the last one; no
  // row's run holds them.  (Columns past the head size are zero.)
  const int wk = k0 + wave * 32, key = wk + l16;     // (of tile 0)
  // Where registers are tight the first slice of both stays in LDS instead (PARK): it is read where a contraction begins, when
  // its results' registers are still free.
  constexpr int PARK = wk_park(HD);
  const unsigned park = lds_base + wk_bits(HD) + SCORED_MOST_BITS + wave * 4 * BLOCK;
  bf16x8 kf[KS - PARK][2], vf[KS - PARK][2];
#pragma unroll
  for (int kt = 0; kt < 2; ++kt) {
    const int64_t at_row = min(key + 16 * kt, d.nkv - 1);
#pragma unroll
    for (int x = 0; x < KS; ++x) {
      const int at = 32 * x + 8 * grp, ld = min(at, H - 8);
      bf16x8 kx = *reinterpret_cast<const bf16x8*>(K + at_row * d.lk.row + ld);
      bf16x8 vx = *reinterpret_cast<const bf16x8*>(V + at_row * d.lv.row + ld);
      if (32 * x + 32 > H && at >= H) kx = vx = bf16x8{};
      if (CAP && A2D_SELDOM(r.capped.lift != 1.f)) lift(kx, r.capped.lift);
      if (x < PARK) {
        auto* const p = reinterpret_cast<__attribute__((address_space(3))) bf16x8*>((uintptr_t)(park + 16 * lane));
        p[64 * kt] = kx;
        p[64 * (2 + kt)] = vx;
      } else {
        kf[x - PARK][kt] = kx;
        vf[x - PARK][kt] = vx;
      }
    }
  }
  f32x4 dk[HT][2], dv[HT][2];
#pragma unroll
  for (int x = 0; x < HT; ++x)
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) dk[x][kt] = dv[x][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
  if constexpr (H != HD) {                           // columns past the head size are zero for good
    for (int i = tid; i < 4 * WK_ROWS * (HD - H) / 8; i += WK_THREADS) {
      const int row = i % WK_ROWS, x = i / WK_ROWS, tile = x / ((HD - H) / 8), ch = H % 32 / 8 + x % ((HD - H) / 8);
      *reinterpret_cast<u32x4*>(lds + tile * TILE + ((row >> 4) * KS + H / 32) * BLOCK + (row & 15) * 64 +
                                16 * (ch ^ block_swap((row & 15) >> 2))) = u32x4{0, 0, 0, 0};
    }
  }
  __syncthreads();
  // this part's share of the set bits: `total` of them
  StepWalk walk;
  int total = walk.open(bits, words);
  if (parts > 1) {
    const int skip = (int)((int64_t)part * total / parts);
    total = (int)((int64_t)(part + 1) * total / parts) - skip;
    walk.skip(skip);
  }
  // ---- staging, straight into LDS: wavefronts 0 .. 3 load a row tile of Q each, 4 .. 7 of dO; 0 .. 3 also bring one of the row
  // tables each, 4 the tiles' records.  The next step is requested while one is computed.  Rows that see nothing are
  // zeros (what they see has been asked for a step earlier: live).
  const bool is_g = wave >= 4;
  const int ld_tile = 16 * (wave & 3);
  const bf16_t* const ld_base = is_g ? dO : Q;
  const int64_t ld_head = is_g ? d.ldo.head : d.lq.head;
  const unsigned ld_row_bytes = __builtin_amdgcn_readfirstlane((unsigned)(is_g ? d.ldo.row : d.lq.row) * 2);
  const int* const ld_table = wave == 0   ? reinterpret_cast<const int*>(tab.from)
                              : wave == 1 ? reinterpret_cast<const int*>(tab.delta)
                              : wave == 2 ? tab.lo
                                          : tab.n;
  struct Step {
    int head, i0;                                    // of the group; first row
  };
  const auto place = [&](int s) {
    const int h = s / nsteps;
    return Step{h, (s - h * nsteps) * WK_ROWS};
  };
  // which of the 16 rows that this wavefront loads see anything (a scalar load: the table is an earlier kernel's)
  const auto ask_live = [&](Step st) -> unsigned {
    const int64_t at = (((int64_t)qh0 + st.head) * tab.padded + st.i0 + ld_tile) / 32;
    const auto* p = reinterpret_cast<const __attribute__((address_space(4))) RowTile*>(reinterpret_cast<uint64_t>(tab.tiles + at));
    return p->live >> (ld_tile & 16) & 0xFFFFu;
  };
  const auto load_step = [&](Step st, unsigned live, int buf) {
    const int ln = TIGHT ? lane_again() : lane, ch = (ln & 3) ^ block_swap(ln >> 4);
    const unsigned at = lds_base + buf * BUF + wave * KS * BLOCK;
    const gptr_t base = uniform_gptr(reinterpret_cast<const char*>(ld_base + st.head * ld_head) + (int64_t)(st.i0 + ld_tile) * ld_row_bytes);
    const unsigned off = __umul24(ln >> 2, ld_row_bytes) + 16 * ch;
    if (A2D_OFTEN(live == 0xFFFFu)) {
      dma_blocks<KS, H>(at, base, off, ch);
    } else if (live >> (ln >> 2) & 1) {
      dma_blocks<KS, H>(at, base, off, ch);
    } else {
#pragma unroll
      for (int x = 0; x < KS; ++x)
        *reinterpret_cast<__attribute__((address_space(3))) u32x4*>((uintptr_t)(at + x * BLOCK + 16 * ln)) = u32x4{0, 0, 0, 0};
    }
    const int64_t row = ((int64_t)qh0 + st.head) * tab.padded + st.i0;
    const unsigned stat = lds_base + wk_stat(HD);
    if (wave < 4) {
      dma_b32<0>(stat + buf * WK_STAT + wave * (4 * WK_ROWS), uniform_gptr(ld_table + row), 4 * ln);
    } else if (wave == 4) {
      if (ln < WK_TILES / 4) dma_b32<0>(stat + 2 * WK_STAT + buf * WK_TILES, uniform_gptr(tab.tiles + row / 32), 4 * ln);
    }
  };
  Step now{0, 0}, then{0, 0};
  unsigned live = 0;
  if (total > 0) {
    now = place(walk.next());
    load_step(now, ask_live(now), 0);
    if (total > 1) {
      then = place(walk.next());
      live = ask_live(then);
    }
  }
  wait_dma();
  __syncthreads();

  Blocks16 da;
  da.init(lane, lds_base);
  unsigned st_addr = lds_base + wk_stat(HD) + 16 * grp;

  // Half a step: S and dP of 32 rows in tiles of 16 rows (t) x 16 keys (kt), lane = key, registers = rows 16 t + 4 grp + 0..3 (see
  // dkdv_wide).  i0: its first row
  constexpr int N1 = 2 * KS, N2 = 4 * KS, N3 = N2 + HT, N4 = N3 + HT, RING = TIGHT || N4 % 4 != 0 ? 2 : 4;
  auto compute = [&](int i0, float slope, bool masked) {
    bf16x8 a[RING];
    auto ld = [&](auto I) {
      constexpr int i = decltype(I)::value;
      if constexpr (i < N2) a[i % RING] = lds_load_b128(da.nat + (i < N1 ? 0 : TILE) + ((i & 1) * KS + (i % N1 >> 1)) * BLOCK);
      else if constexpr (i < N4) {
        constexpr int y = i < N3 ? i - N2 : i - N3;
        const unsigned at = (y & 1 ? da.tr_e ^ 32 : da.tr_e) + (i < N3 ? TILE : 0) + (y >> 1) * BLOCK;
        a[i % RING] = lds_load_tr(at, at + KS * BLOCK);
      }
    };
    bf16x8 first[2];                                   // (parked)
    const auto fetch = [&](int v) {
      const unsigned at = park + 16 * (TIGHT ? lane_again() : lane) + 2 * BLOCK * v;
      first[0] = lds_load_b128(at);
      first[1] = lds_load_b128(at + BLOCK);
    };
    if constexpr (PARK) fetch(0);
    static_for<0, RING>(ld);
    f32x4 s[2][2], dp[2][2];
#pragma unroll
    for (int t = 0; t < 2; ++t) s[t][0] = s[t][1] = CAP ? f32x4{0.f, 0.f, 0.f, 0.f} : lds_load_f32x4(st_addr + 64 * t);
    __builtin_amdgcn_sched_barrier(0);
    static_for<0, N1>([&](auto I) {
      constexpr int i = decltype(I)::value, x = i >> 1, t = i & 1;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) s[t][kt] = mma16(a[i % RING], x < PARK ? first[kt] : kf[x < PARK ? 0 : x - PARK][kt], s[t][kt]);
      ld(std::integral_constant<int, i + RING>{});
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (CAP) cap_in_place(s, r.capped);
    if constexpr (PARK) fetch(1);
    f32x4 l2[2];                                       // (with a cap)
    if constexpr (CAP) l2[0] = lds_load_f32x4(st_addr);
#pragma unroll
    for (int t = 0; t < 2; ++t) dp[t][0] = dp[t][1] = lds_load_f32x4(st_addr + WK_ROWS * 4 + 64 * t);
    float base[2] = {0.f, 0.f};
    if constexpr (BIAS) {
      const int ln = TIGHT ? lane_again() : lane;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
        base[kt] = (float)(int)(r.rel + (int64_t)(i0 + 4 * (ln >> 4) - (wk + (ln & 15) + 16 * kt)) * r.step);
    }
    bf16x8 pb[2], sb[2], p_rest[2], s_rest[2];
    // score e of the lane's 16: row tile e >> 3, key tile (e >> 2) & 1, row e & 3 of the lane's four.  P to pb, P (1 - t^2) stays in s
    auto prob = [&](int e) {
      const int t = e >> 3, kt = (e >> 2) & 1, i = e & 3;
      const float y = s[t][kt][i];
      float x = CAP ? y - l2[t][i] : y * raw;
      if constexpr (BIAS) x = fmaf(-slope, fabsf(distance<1>(r, base[kt], t, i)), x);
      const float p = fast_exp2(x);
      pb[kt][4 * t + i] = (bf16_t)p;
      if constexpr (FINE) p_rest[kt][4 * t + i] = (bf16_t)(p - (float)pb[kt][4 * t + i]);
      if constexpr (CAP) {
        const float u = y * inv_top;
        s[t][kt][i] = fmaf(-p * u, u, p);
      } else {
        s[t][kt][i] = p;
      }
    };
    // (hidden pairs: their products may have overflowed, so they are taken out of the scores themselves.  HIDDEN: 2^x of it is 0; with
    // a cap its square, times 0, must be 0 too)
    auto mask = [&]() {
      if (A2D_SELDOM(masked)) {
        asm volatile("" ::: "memory");
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const u32x4 lo = __builtin_bit_cast(u32x4, lds_load_f32x4(st_addr + 2 * WK_ROWS * 4 + 64 * t));
          const u32x4 n = __builtin_bit_cast(u32x4, lds_load_f32x4(st_addr + 3 * WK_ROWS * 4 + 64 * t));
          const int ln = TIGHT ? lane_again() : lane;
          float HIDDEN = CAP ? -1e30f : -INFINITY;
          asm volatile("" : "+v"(HIDDEN));             // (it would be kept in a register for all steps)
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              s[t][kt][i] = (unsigned)(wk + (ln & 15) + 16 * kt) - lo[i] < n[i] ? s[t][kt][i] : HIDDEN;
        }
      }
    };
    auto dscore = [&](int e) {
      const int t = e >> 3, kt = (e >> 2) & 1, i = e & 3;
      const float z = s[t][kt][i] * dp[t][kt][i];
      sb[kt][4 * t + i] = (bf16_t)z;
      if constexpr (FINE) s_rest[kt][4 * t + i] = (bf16_t)(z - (float)sb[kt][4 * t + i]);
    };
    mask();
    static_for<0, N1>([&](auto I) {
      constexpr int i = decltype(I)::value, x = i >> 1, t = i & 1;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) dp[t][kt] = mma16(a[(N1 + i) % RING], x < PARK ? first[kt] : vf[x < PARK ? 0 : x - PARK][kt], dp[t][kt]);
      if constexpr (CAP && i == N1 / 2 - 1) l2[1] = lds_load_f32x4(st_addr + 64);
#pragma unroll
      for (int e = 16 * i / N1; e < 16 * (i + 1) / N1; ++e) prob(e);
      ld(std::integral_constant<int, N1 + i + RING>{});
      __builtin_amdgcn_sched_barrier(0);
    });
    if (A2D_SELDOM(masked)) {
      // (0 times the product of a dO with what an unseen key's V holds)
      asm volatile("" ::: "memory");
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int t = (e >> 2) & 1, kt = e >> 3, i = e & 3;
        dp[t][kt][i] = s[t][kt][i] == 0.f ? 0.f : dp[t][kt][i];
      }
    }
    static_for<0, HT>([&](auto Y) {
      constexpr int y = decltype(Y)::value;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        dv[y][kt] = mma16(a[(N2 + y) % RING], pb[kt], dv[y][kt]);
        if constexpr (FINE) dv[y][kt] = mma16(a[(N2 + y) % RING], p_rest[kt], dv[y][kt]);
      }
#pragma unroll
      for (int e = 16 * y / HT; e < 16 * (y + 1) / HT; ++e) dscore(e);
      ld(std::integral_constant<int, N2 + y + RING>{});
      __builtin_amdgcn_sched_barrier(0);
    });
    static_for<0, HT>([&](auto Y) {
      constexpr int y = decltype(Y)::value;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        dk[y][kt] = mma16(a[(N3 + y) % RING], sb[kt], dk[y][kt]);
        if constexpr (FINE) dk[y][kt] = mma16(a[(N3 + y) % RING], s_rest[kt], dk[y][kt]);
      }
      ld(std::integral_constant<int, N3 + y + RING>{});
      __builtin_amdgcn_sched_barrier(0);
    });
  };

  constexpr int HALF = 2 * KS * BLOCK;               // of a tile
  int buf = 0;
#pragma nounroll
  for (int n = 0; n < total; ++n) {
    const Step cur = now;
    if (n + 1 < total) {
      load_step(then, live, buf ^ 1);
      now = then;
      if (n + 2 < total) {
        then = place(walk.next());
        live = ask_live(then);
      }
    }
    const float slope = BIAS ? uniform(r.slopes[qh0 + cur.head] * kLog2e) : 0.f;
#pragma nounroll
    for (int h = 0; h < 2; ++h) {
      const u32x4 rec = __builtin_bit_cast(u32x4, lds_load_f32x4(lds_base + wk_stat(HD) + 2 * WK_STAT + buf * WK_TILES + (int)sizeof(RowTile) * h));
      const int lo = __builtin_amdgcn_readfirstlane(rec[0]), hi = __builtin_amdgcn_readfirstlane(rec[1]);
      const int all_lo = __builtin_amdgcn_readfirstlane(rec[2]), all_hi = __builtin_amdgcn_readfirstlane(rec[3]);
      if (lo < wk + 32 && hi > wk) compute(cur.i0 + 32 * h, slope, all_lo > wk || all_hi < wk + 32);
      const int go = h == 0 ? HALF : buf ? -BUF - HALF : BUF - HALF;
      da.nat += go; da.tr_e += go;
      st_addr += h == 0 ? 32 * 4 : buf ? -WK_STAT - 32 * 4 : WK_STAT - 32 * 4;
    }
    buf ^= 1;
    wait_dma();
    __syncthreads();
  }

  char* const area = lds + wave * acc_area(HT);
  const int ln = TIGHT ? lane_again() : lane;
#pragma unroll
  for (int kt = 0; kt < 2; ++kt) {
    const int first = wk + 16 * kt, n = d.nkv - first;
    const int64_t at = ((int64_t)head * d.nkv + first) * H;
    if (parts > 1) {
      float* const to = more + (((int64_t)head * cut.units + mine.slot + part) * WK_KEYS + first - k0) * H;
      store_acc16(to + (int64_t)kv_heads * cut.units * WK_KEYS * H, H, n, area, dv, kt, ln, 1.0f);
      store_acc16(to, H, n, area, dk, kt, ln, d.scale);
    } else if (r.norm) {
      store_acc16(static_cast<bf16_t*>(dV) + at, H, n, area, dv, kt, ln, 1.0f);
      store_acc16(static_cast<bf16_t*>(dK) + at, H, n, area, dk, kt, ln, d.scale);
    } else {
      store_acc16(static_cast<float*>(dV) + at, H, n, area, dv, kt, ln, 1.0f);
      store_acc16(static_cast<float*>(dK) + at, H, n, area, dk, kt, ln, d.scale);
    }
  }
}

template <int HR, bool CAP, bool BIAS, bool FINE>
__global__ __launch_bounds__(WK_THREADS) void scored_dkdv_kernel(
    a2d_tile_desc d, ScoreRules r, Cut cut, int in_order, RowTable tab, const bf16_t* __restrict__ Q, const bf16_t* __restrict__ K,
    const bf16_t* __restrict__ V, const bf16_t* __restrict__ dO, void* __restrict__ dK, void* __restrict__ dV, float* __restrict__ more,
    int2* __restrict__ table) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  __shared__ Shares shares;
  scored_dkdv_keys<HR, CAP, BIAS, FINE>(blockIdx.x, lds, shares, d, r, cut, in_order, tab, Q, K, V, dO, dK, dV, more, table);
}
static_assert(MAX_RANKED <= WK_THREADS, "a thread a block");

// ---- sums of the partials, blocks of one part left out (theirs are written already): four floats a thread, the parts in their order
struct SumOf {
  const float* p;        // [heads][cut.units][bm][hdim]
  void* out;             // [heads][rows][hdim]
  const int2* table;     // shared out: slot and parts of each block
  Cut cut;
  int heads, rows, bm;
};
struct SumsOf {
  SumOf s[3];
};
template <bool ROUNDED>
__global__ __launch_bounds__(256) void scored_sum_kernel(SumsOf sums, int hdim, int add) {
  const SumOf& s = sums.s[blockIdx.z];               // (dK, dV, dQ: the last is added to)
  const int per = s.bm * hdim / 1024;                // workgroups a block: bm is 128 or 256, hdim a multiple of 16
  if ((int)blockIdx.x >= s.cut.blocks * per || (int)blockIdx.y >= s.heads) return;
  const int block = blockIdx.x / per, in = (blockIdx.x - block * per) * 1024 + 4 * threadIdx.x;
  const int2 at = s.table ? s.table[block] : int2{block * s.cut.parts, s.cut.parts};
  const int64_t to = ((int64_t)blockIdx.y * s.rows + (int64_t)block * s.bm) * hdim + in;
  if (at.y == 1 || in >= (s.rows - block * s.bm) * hdim) return;
  const int64_t part = (int64_t)s.bm * hdim;
  const float* p = s.p + ((int64_t)blockIdx.y * s.cut.units + at.x) * part + in;
  f32x4 acc{0.f, 0.f, 0.f, 0.f};
  if (!ROUNDED && add && blockIdx.z == 2) acc = *reinterpret_cast<const f32x4*>(static_cast<float*>(s.out) + to);
  int z = 0;
  for (; z + 4 <= at.y; z += 4) {
    f32x4 v[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) v[x] = *reinterpret_cast<const f32x4*>(p + (z + x) * part);
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += v[x][e];
  }
  for (; z < at.y; ++z) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(p + z * part);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += v[e];
  }
  if constexpr (ROUNDED) *reinterpret_cast<bf16x4*>(static_cast<bf16_t*>(s.out) + to) = bf16x4{(bf16_t)acc[0], (bf16_t)acc[1], (bf16_t)acc[2], (bf16_t)acc[3]};
  else *reinterpret_cast<f32x4*>(static_cast<float*>(s.out) + to) = acc;
}

constexpr int LEAST_Q = 1, LEAST_KV = 2;             // a step: 64 keys; two tiles of 32 rows
// in_order: heaviest blocks first over all heads (see xcd_map)
Cut cut_of(const a2d_tile_desc& d, const ScoreRules& r, int n, int units, bool share, int least, int* in_order) {
  *in_order = share || blocks_by_size(d, r, n) == BY_ROWS;
  return share ? Cut{n, units, 0, least} : Cut{n, units / n * n, units / n, least};
}
struct BwdCuts {
  Cut q, kv;
  int bm, q_in_order, kv_in_order;
  int64_t q_floats, kv_floats;                       // of partials, each result's
  BwdCuts(const a2d_tile_desc& d, const ScoreRules& r, const ScoredBwdPlan& plan) : bm(256 / plan.lanes) {
    q = cut_of(d, r, (d.nq + bm - 1) / bm, plan.q, plan.share_q, LEAST_Q, &q_in_order);
    kv = cut_of(d, r, (d.nkv + WK_KEYS - 1) / WK_KEYS, plan.kv, plan.share_kv, LEAST_KV, &kv_in_order);
    q_floats = q.units > q.blocks ? (int64_t)d.heads * q.units * bm * d.hdim : 0;
    kv_floats = kv.units > kv.blocks ? (int64_t)(d.heads / r.group) * kv.units * WK_KEYS * d.hdim : 0;
  }
};

template <int HR, bool CAP, bool BIAS, bool FINE>
hipError_t go(Phase ph, const a2d_tile_desc& d, const ScoreRules& r, const ScoredBwdPlan& plan, const void* Q, const void* K, const void* V,
              const void* O, const void* dO, const float* lse, void* ws, void* more, void* dQ, void* dK, void* dV, hipStream_t s) {
  constexpr int HD = padded_head(HR);
  const RowTable tab = row_table(d, ws);
  const BwdCuts c(d, r, plan);
  const int kvh = d.heads / r.group, dq_bytes = dq_launch_lds(HD, plan.lanes);
  const int words = (tab.padded / WK_ROWS * r.group + 63) / 64, wk_bytes = wk_park(HD) ? wk_lds(HD) : wk_bits(HD) + 8 * words;
  float* const q_more = static_cast<float*>(more);
  float* const kv_more = q_more + c.q_floats;
  int2* const q_table = reinterpret_cast<int2*>(kv_more + 2 * c.kv_floats);
  int2* const kv_table = q_table + c.q.blocks;
  const bool q_shared = c.q_floats && c.q.parts == 0, kv_shared = c.kv_floats && c.kv.parts == 0;
  const auto dq = [&](auto* kernel) {
    if (ph == PREPARE) return ensure_dynamic_lds(reinterpret_cast<const void*>(kernel), dq_bytes);
    A2D_LAUNCH(kernel, dim3(xcd_grid(kvh, r.group * c.q.units)), dim3(512), dq_bytes, s, d, r, c.q, c.q_in_order, tab, (const bf16_t*)Q,
               (const bf16_t*)K, (const bf16_t*)V, (const bf16_t*)O, (const bf16_t*)dO, lse, dQ, q_more, q_shared ? q_table : nullptr);
    return hipGetLastError();
  };
  hipError_t e = plan.lanes == 2 ? dq(scored_dq_kernel<HR, 2, CAP, BIAS, FINE>) : dq(scored_dq_kernel<HR, 1, CAP, BIAS, FINE>);
  if (e != hipSuccess) return e;
  // (the most a call can ask for: ensure_dynamic_lds is asked once for a kernel)
  if (ph == PREPARE) return ensure_dynamic_lds(reinterpret_cast<const void*>(scored_dkdv_kernel<HR, CAP, BIAS, FINE>), wk_lds(HD));
  A2D_LAUNCH((scored_dkdv_kernel<HR, CAP, BIAS, FINE>), dim3(xcd_grid(kvh, c.kv.units)), dim3(WK_THREADS), wk_bytes, s, d, r, c.kv, c.kv_in_order, tab,
             (const bf16_t*)Q, (const bf16_t*)K, (const bf16_t*)V, (const bf16_t*)dO, dK, dV, kv_more, kv_shared ? kv_table : nullptr);
  if ((e = hipGetLastError()) != hipSuccess || c.q_floats + c.kv_floats == 0) return e;
  Cut none{};
  const SumsOf sums{{{kv_more, dK, kv_shared ? kv_table : nullptr, c.kv_floats ? c.kv : none, kvh, d.nkv, WK_KEYS},
                     {kv_more + c.kv_floats, dV, kv_shared ? kv_table : nullptr, c.kv_floats ? c.kv : none, kvh, d.nkv, WK_KEYS},
                     {q_more, dQ, q_shared ? q_table : nullptr, c.q_floats ? c.q : none, d.heads, d.nq, c.bm}}};
  int wide = 0;
  for (const SumOf& x : sums.s) wide = std::max(wide, x.cut.blocks * (x.bm * d.hdim / 1024));
  const dim3 grid(wide, c.q_floats ? d.heads : kvh, c.q_floats ? 3 : 2);
  if (r.norm) A2D_LAUNCH(scored_sum_kernel<true>, grid, dim3(256), 0, s, sums, d.hdim, 0);
  else A2D_LAUNCH(scored_sum_kernel<false>, grid, dim3(256), 0, s, sums, d.hdim, (int)r.acc);
  return hipGetLastError();
}

}  // namespace

size_t scored_bwd_bytes(const a2d_tile_desc& d) {
  const size_t n = (size_t)d.heads * ((d.nq + 63) / 64 * 64);
  return 16 * n + n / 32 * sizeof(RowTile);
}

size_t scored_bwd_scratch(const a2d_tile_desc& d, const ScoreRules& r, const ScoredBwdPlan& plan) {
  const BwdCuts c(d, r, plan);
  if (c.q_floats + c.kv_floats == 0) return 0;
  return (size_t)(c.q_floats + 2 * c.kv_floats) * sizeof(float) + (size_t)(c.q.blocks + c.kv.blocks) * sizeof(int2);
}

// Every way's time from its turns of the chip, the quickest; one launch sums up every result that is cut.  Steps in us, fitted to 45 calls
// timed in each of 120 ways.  Documents, which the host cannot see, are taken to have their tokens in the rows and the keys alike and for
// walks of a third of them.  What it chooses between, measured: 4096 x 4096, 32 / 8 heads of 128, causal under a cap: dK / dV of four
// parts a block 532 us, of one 1169 (128 workgroups, of any length); 8192 x 8192, 16 of 128 in documents: whole blocks, the longest first 343,
// in their own order 427, dK / dV in four parts besides 520; of the fit's calls, as they were timed for it: 427 x 5532, 16 / 4 of 64 in documents,
// dK / dV of three units a block on average, shared out, 43, of four even parts 56; 746 x 895, 4 / 1 of 64, shared out 28, even 22
// (finding out the shares takes some 3 us).
ScoredBwdPlan plan_scored_bwd(const a2d_tile_desc& d, const ScoreRules& r, int cus, size_t most_bytes) {
  constexpr double kFindOut = 4.0, kSum = 5.0, kBytes = 6e6;             // us; bytes of partials a us, out and back
  const bool documents = taken_for_documents(d, r);
  const int rules = (r.cap != 0.f) + (r.slopes != nullptr), kvh = d.heads / r.group;
  const double by_head = d.hdim / 128.0, all_rows = (double)d.nq * r.group, alike = std::min(1.0, (double)d.nkv / d.nq);
  const WalkKeys w = walk_keys(d, r);
  struct Walks {
    double mean, most;
  } keys{w.mean, w.most}, rows{all_rows * (w.mean / d.nkv), all_rows};
  if (documents) {
    const double part = std::sqrt(std::min(1.0, (double)d.nq / d.nkv));
    keys = Walks{0.35 * part * keys.mean, 0.65 * part * keys.most};
    rows = Walks{0.35 * alike * rows.mean, 0.65 * alike * rows.most};
  }
  struct Way {
    int units;
    bool share;
    double us;
  };
  // n blocks of `bm` rows or keys of each of `heads` heads, which walk in steps of `of` keys or rows
  const auto cut = [&](int n, int heads, int bm, int results, Walks walks, int of, double step, double fixed, bool split) {
    const double mean = walks.mean / of + 0.2, most = walks.most / of + 0.2, unit_us = bm * d.hdim * 8.0 * results / kBytes;
    const double blind = documents ? 1.2 : 1.0;                          // walks in no order
    const int64_t room = split ? (int64_t)(most_bytes / ((size_t)heads * bm * d.hdim * sizeof(float))) : 0;
    const bool uneven = n > 1 && n <= MAX_RANKED && (documents || !r.ranges) && blocks_by_size(d, r, n) != 0;
    const WalkModel whole{(int64_t)heads * n, cus, mean, most, step, fixed, 0, 0, nullptr, 0, 0.1};
    Way best{n, false, walk_time(whole, 1) * blind};
    for (int x = 4; x <= 128; x += x < 8 ? 1 : x < 32 ? 4 : 16) {        // quarters of n
      const int u = (int)((int64_t)n * x / 4);
      if (u > n && u > room) break;
      if (u > n && x % 4 == 0) {
        const double us = walk_time(whole, x / 4) * blind + (double)heads * u * unit_us;
        if (us < best.us) best = Way{u, false, us};
      }
      if (uneven) {
        const double each = u > n ? std::max(1.0, n * mean / (u - 0.5 * n)) : most, made = u > n ? std::min<double>(u, 0.5 * n + n * mean / each) : n;
        const double one = std::min(each, most) * step + fixed + kFindOut;
        const double even = heads * (n * mean * step + made * (fixed + kFindOut)) / cus + 0.15 * one;
        const double turns = u > n ? std::ceil(heads * made / cus) : 1;
        const double us = std::max(turns * one, even) + (u > n ? heads * made * unit_us : 0);
        if (us < best.us) best = Way{u, true, us};
      }
    }
    return best;
  };
  const auto plan = [&](bool split, double* us) {
    const Way one = cut((d.nq + 255) / 256, d.heads, 256, 1, keys, 64, 0.35 + 1.4 * by_head + 0.2 * rules, 3.6, split);
    const Way two = cut((d.nq + 127) / 128, d.heads, 128, 1, keys, 128, 0.75 + 1.4 * by_head + 0.1 * rules, 5.3, split);
    const Way kv = cut((d.nkv + WK_KEYS - 1) / WK_KEYS, kvh, WK_KEYS, 2, rows, WK_ROWS, 1.3 + 1.1 * by_head + 0.55 * rules, 7.5, split);
    const Way& q = two.us < one.us ? two : one;
    *us = q.us + kv.us + (split ? kSum : 0);
    return ScoredBwdPlan{two.us < one.us ? 2 : 1, q.units, kv.units, q.share, kv.share};
  };
  double whole_us, split_us;
  const ScoredBwdPlan whole = plan(false, &whole_us), split = plan(true, &split_us);
  return split_us < whole_us ? split : whole;
}

// Calls of few scores contract P and dZ as two bf16 numbers each (hi + lo, 2^-17 off).  One rounding to bf16 leaves gradients off by 1.41
// times what the rounding of the outputs alone does - two roundings of one size -, however long the sums are (4096 rows in documents of 2 to
// 4096 tokens: 1.25 to 1.43), where few scores make the result by chance more (349 x 193, 4 / 1 heads of 80: 1.47).  Up to 2^22 scores the
// second number is nearly free, as calls wait for launches and first loads: 637 x 260, 4 / 2 of 96, 31 -> 33 us.  Beyond it is not: 4619 x 543, 2
// of 80, 41 -> 46; 2999 x 2999, 12 / 4 of 80 in documents 76 -> 89; 4096 x 4096, 32 / 8 of 128 under a cap 532 -> 667.
static bool fine_call(const a2d_tile_desc& d) { return (int64_t)d.heads * d.nq * d.nkv <= (int64_t)1 << 22; }

void route_scored_bwd(const a2d_tile_desc& d, const ScoreRules& r, const ScoredBwdPlan& plan, ScoredRoute* out) {
  const BwdCuts c(d, r, plan);
  *out = ScoredRoute{};
  for (const char* k : {"scored_dq_kernel", "scored_dkdv_kernel"}) out->kernel[out->kernels++] = k;
  if (c.q_floats + c.kv_floats) out->kernel[out->kernels++] = "scored_sum_kernel";
  out->rows = c.bm;
  out->lanes = plan.lanes;
  out->waves = 8;
  out->blocks_q = c.q.blocks;
  out->units_q = c.q.units;
  out->blocks_kv = c.kv.blocks;
  out->units_kv = c.kv.units;
  out->shared_q = plan.share_q;
  out->shared_kv = plan.share_kv;
  out->fine = fine_call(d);
}

hipError_t launch_scored_bwd(Phase ph, const a2d_tile_desc& d, const ScoreRules& r, const ScoredBwdPlan& plan, const void* Q, const void* K,
                             const void* V, const void* O, const void* dO, const float* lse, void* ws, void* more, void* dQ, void* dK,
                             void* dV, hipStream_t s) {
  const bool fine = fine_call(d);
#define A2D_FINE(HR, CAP, BIAS)                                                                              \
  (fine ? go<HR, CAP, BIAS, true>(ph, d, r, plan, Q, K, V, O, dO, lse, ws, more, dQ, dK, dV, s)                \
        : go<HR, CAP, BIAS, false>(ph, d, r, plan, Q, K, V, O, dO, lse, ws, more, dQ, dK, dV, s))
#define A2D_RULES(HR)                                                                                        \
  return r.cap != 0.f ? (r.slopes ? A2D_FINE(HR, true, true) : A2D_FINE(HR, true, false))                     \
                      : (r.slopes ? A2D_FINE(HR, false, true) : A2D_FINE(HR, false, false))
  if (d.hdim == 128) { A2D_RULES(128); }
  if (d.hdim == 96) { A2D_RULES(96); }
  if (d.hdim == 80) { A2D_RULES(80); }
  A2D_RULES(64);
#undef A2D_RULES
#undef A2D_FINE
}

}  // namespace a2d
