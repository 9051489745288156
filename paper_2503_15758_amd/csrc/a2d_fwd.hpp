// What the bf16 forward kernels of many rows share: the state of a wavefront's 32 query rows and the MFMAs of a 64-key block
// (see a2d_fwd_mfma.hip for the kernel that they were made for).
#pragma once
#include "a2d_mfma.hpp"

namespace a2d {
namespace mfma {

constexpr int BN = 64;             // keys per step
__host__ __device__ constexpr int buf_bytes(int hd) { return 2 * BN * 2 * hd; }   // { K tile, V tile }, in blocks
__host__ __device__ constexpr int lds_bytes(int hd) { return 2 * buf_bytes(hd); }          // of a key lane
// of a launch: 16 rows of every wavefront come in (accumulating calls) and go out at a time
__host__ __device__ constexpr int fwd_lds(int waves, int hd, int kl) {
  const int tiles = kl * lds_bytes(hd), rows = waves / kl * acc_area(hd / 16);
  return tiles > rows ? tiles : rows;
}

template <int HR>
struct FwdState {
  f32x4 o[HR / 16][2];   // column tiles x the wavefront's two tiles of 16 query rows
  // of the lane's row in each tile:
  float m_lane[2];       // true running max of this lane's raw dot products
  float m_ref[2];        // reference the exponentials are taken against (raw units, same in the four lanes of a row)
  float l_run[2];        // this lane's share of the row sum, relative to m_ref
};

// A 64-key block for one wavefront, in three pieces; at: its buffer's offset from the addresses in rd.  S^T in tiles of 16 keys (k) x 16
// queries (q): lane = query, registers = keys 16 k + 4 grp + 0..3; the registers of two key tiles are the eight contraction indices of a
// lane in O^T += V^T P^T.
// Fragments of K and V go through rings four deep: each is requested four slots of two MFMAs before its use (the scheduling fences
// keep the compiler from sinking the requests back to their uses), the first ones before the piece that uses them.
using Scores = f32x4[4][2];
using Ring = bf16x8[4];
template <int HR, int I>                           // slot I of the scores: key tile I & 3, slice I >> 2 of H, both query tiles
__device__ __forceinline__ void fwd_key(Ring& kr, const Blocks16& rd, unsigned at) {
  kr[I & 3] = lds_load_b128(rd.nat + at + ((I & 3) * (padded_head(HR) / 32) + (I >> 2)) * BLOCK);
}
template <int HR, int I>                           // step I of the products: 32-key group I / HT, column tile I % HT
__device__ __forceinline__ void fwd_value(Ring& vr, const Blocks16& rd, unsigned at) {
  constexpr int KS = padded_head(HR) / 32, HT = HR / 16, K_BYTES = buf_bytes(padded_head(HR)) / 2;
  const unsigned a = (I % HT & 1 ? rd.tr_o : rd.tr_e) + at + K_BYTES + ((I / HT) * 2 * KS + (I % HT >> 1)) * BLOCK;
  vr[I & 3] = lds_load_tr(a, a + KS * BLOCK);
}
template <int HR>
__device__ __forceinline__ void fwd_first_keys(Ring& kr, const Blocks16& rd, unsigned at) {
  static_for<0, 4>([&](auto I) { fwd_key<HR, decltype(I)::value>(kr, rd, at); });
  __builtin_amdgcn_sched_barrier(0);
}
template <int HR>
__device__ __forceinline__ void fwd_first_values(Ring& vr, const Blocks16& rd, unsigned at) {
  static_for<0, 4>([&](auto I) { fwd_value<HR, decltype(I)::value>(vr, rd, at); });
  __builtin_amdgcn_sched_barrier(0);
}

template <int HR>
__device__ __forceinline__ void fwd_scores(Scores& s, Ring& kr, const bf16x8 (&qf)[padded_head(HR) / 32][2], const Blocks16& rd, unsigned at) {
  constexpr int KS = padded_head(HR) / 32;
#pragma unroll
  for (int k = 0; k < 4; ++k) s[k][0] = s[k][1] = f32x4{0.f, 0.f, 0.f, 0.f};
  static_for<0, 4 * KS>([&](auto I) {
    constexpr int i = decltype(I)::value;
#pragma unroll
    for (int q = 0; q < 2; ++q) s[i & 3][q] = mma16(kr[i & 3], qf[i >> 2][q], s[i & 3][q]);
    if constexpr (i + 4 < 4 * KS) fwd_key<HR, i + 4>(kr, rd, at);
    __builtin_amdgcn_sched_barrier(0);
  });
}

// O^T += V^T P^T
template <int HR>
__device__ __forceinline__ void fwd_products(f32x4 (&o)[HR / 16][2], const bf16x8 (&pb)[2][2], Ring& vr, const Blocks16& rd, unsigned at) {
  constexpr int HT = HR / 16;
  static_for<0, 2 * HT>([&](auto I) {
    constexpr int i = decltype(I)::value;
#pragma unroll
    for (int q = 0; q < 2; ++q) o[i % HT][q] = mma16(vr[i & 3], pb[i / HT][q], o[i % HT][q]);
    if constexpr (i + 4 < 2 * HT) fwd_value<HR, i + 4>(vr, rd, at);
    __builtin_amdgcn_sched_barrier(0);
  });
}

}  // namespace mfma
}  // namespace a2d
