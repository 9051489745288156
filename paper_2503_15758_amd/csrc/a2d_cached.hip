// Attention over the paged cache: how a call goes out, the merge of walks that several workgroups share, and the plain kernel.
#include <algorithm>

#include "a2d_cached_cut.hpp"

namespace a2d {
namespace {

// Joins the parts of the blocks whose walk was cut: M = max m, N = sum 2^(m_k - M) N_k, l likewise.  SHARED: a workgroup has one row, whose
// parts its eight groups of 32 lanes take in turn (they are joined in order); else each group has a row of its own.
// Bound: HBM and the last-level cache, each part read once; short calls: the launch.
template <int H, bool SHARED>
__global__ __launch_bounds__(256) void cached_merge_kernel(CachedArgs a, int groups) {
  constexpr int QUADS = H / 4;
  __shared__ f32x4 sums[8][QUADS];
  __shared__ float ms[8], ls[8];
  warm_cached();
  const int group = threadIdx.x >> 5, quad = threadIdx.x & 31;
  const int u = blockIdx.x / groups, at = blockIdx.x - u * groups, per_sequence = a.c.kv_heads * a.blocks;
  const int b = u / per_sequence, unit = u - b * per_sequence;
  const int2 cut = a.cuts[u];                          // (as the workers found it)
  const unsigned w0 = cut.x, parts = cut.y;
  if (parts == 1) return;
  const int rows = 16 * a.tiles, h = unit / a.blocks, block = unit - h * a.blocks;
  const int r = SHARED ? at : 8 * at + group, index = block * rows + r;
  const bool there = r < rows && index < a.group * a.rows;
  if (SHARED && !there) return;
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  if (there) {
#pragma unroll 4
    for (unsigned k = SHARED ? group : 0; k < parts; k += SHARED ? 8 : 1) {
      const float* part = a.parts + (size_t)(2 * (w0 + k) + (k == 0)) * part_floats(rows, H);
      const float pm = part[r], pl = part[rows + r];
      f32x4 x = {0.f, 0.f, 0.f, 0.f};
      if (quad < QUADS) x = *reinterpret_cast<const f32x4*>(part + 2 * rows + (size_t)r * H + 4 * quad);
      const float top = fmaxf(m, pm);
      const float f = top == -INFINITY ? 0.f : fast_exp2(m - top), g = top == -INFINITY ? 0.f : fast_exp2(pm - top);
      m = top;
      l = l * f + pl * g;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = o[e] * f + x[e] * g;
    }
  }
  if constexpr (SHARED) {
    if (quad < QUADS) sums[group][quad] = o;
    if (quad == 0) {
      ms[group] = m;
      ls[group] = l;
    }
    __syncthreads();
    if (threadIdx.x >= QUADS) return;
    m = -INFINITY;
#pragma unroll
    for (int k = 0; k < 8; ++k) m = fmaxf(m, ms[k]);
    l = 0.f;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float f = m == -INFINITY ? 0.f : fast_exp2(ms[k] - m);
      const f32x4 x = sums[k][quad];
      l += ls[k] * f;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += x[e] * f;
    }
  }
  if (!there || quad >= QUADS) return;
  const int g = index / a.rows;
  finish(a, b, h * a.group + g, index - g * a.rows, H, quad, o, m, l);
}

// The plain form, on the vector ALU: a wavefront for each row of each query head; a lane has one of 64 keys for the scores, and two columns of O.
template <int FMT>
__device__ __forceinline__ float cached_value(const char* codes, const char* scales, int64_t row, int hdim, int c) {
  const char* p = codes + row * code_bytes<FMT>(8) * (hdim / 8);
  if constexpr (FMT == A2D_CACHE_BF16) {
    return (float)reinterpret_cast<const bf16_t*>(p)[c];
  } else {
    const float scale = scale_number((unsigned char)scales[row * 4 + c / CACHE_BLOCK]);
    if constexpr (FMT == A2D_CACHE_E4M3)
      return (float)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned char)p[c], scale, false)[0];
    else
      return (float)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((unsigned char)p[c / 2] >> (4 * (c & 1)) & 15, scale, 0)[0];
  }
}
template <int FMT>
__global__ __launch_bounds__(64) void cached_generic_kernel(CachedArgs a, int hdim) {
  __shared__ float q[128], p[64];
  __shared__ int64_t at[64];
  const int lane = threadIdx.x;
  const int64_t x = blockIdx.x;
  const int i = (int)(x % a.rows), head = (int)(x / a.rows % a.heads), b = (int)(x / a.rows / a.heads), h = head / a.group;
  for (int c = lane; c < hdim; c += 64) q[c] = (float)(reinterpret_cast<const bf16_t*>(a.Q) + at_row(a.lq, b, head, i))[c];
  const bool token = !a.masks || (a.masks[((int64_t)b * a.rows + i) * a.words + (i >> 6)] >> (i & 63) & 1);
  const int tokens = token ? tokens_of(a, a.lens[b]) : 0, drafts = token && a.K ? a.rows : 0;
  float m = -INFINITY, l = 0.f, o[2] = {0.f, 0.f};
  const int64_t cached = (tokens + 63) / 64, all = cached + (drafts + 63) / 64;
  for (int64_t s = 0; s < all; ++s) {
    __syncthreads();
    const bool draft = s >= cached;
    const int key = (int)(64 * (draft ? s - cached : s)) + lane;
    bool see;
    int64_t row = 0;
    if (draft) {
      see = key < drafts && (a.masks ? a.masks[((int64_t)b * a.rows + i) * a.words + (key >> 6)] >> (key & 63) & 1 : key <= i);
      row = see ? key : -1;
    } else {
      see = key < tokens;
      const unsigned unit = see ? unit_of(a.c, b, h, key >> 4) : NO_UNIT;
      see = unit != NO_UNIT;
      row = see ? (int64_t)unit * 16 + (key & 15) : -1;
    }
    at[lane] = row;
    float z = 0.f;
    if (see)
      for (int c = 0; c < hdim; ++c)
        z += q[c] * (draft ? (float)(reinterpret_cast<const bf16_t*>(a.K) + at_row(a.lk, b, h, row))[c]
                           : cached_value<FMT>(a.c.K, a.c.Ks, row, hdim, c));
    z = see ? z * a.c2 : -INFINITY;
    float top = z;
    for (int d = 32; d > 0; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
    top = fmaxf(top, m);
    const float f = m == top ? 1.f : fast_exp2(m - top);
    const float w = z == -INFINITY ? 0.f : fast_exp2(z - top);         // (NaN: NaN, whatever the others are)
    p[lane] = w;
    m = top;
    l = l * f + w;
    o[0] *= f;
    o[1] *= f;
    __syncthreads();
    for (int k = 0; k < 64; ++k) {
      if (at[k] < 0) continue;
      for (int e = 0; e < 2; ++e) {
        const int c = lane + 64 * e;
        if (c < hdim)
          o[e] += p[k] * (draft ? (float)(reinterpret_cast<const bf16_t*>(a.V) + at_row(a.lv, b, h, at[k]))[c]
                                : cached_value<FMT>(a.c.V, a.c.Vs, at[k], hdim, c));
      }
    }
  }
  for (int d = 32; d > 0; d /= 2) l += __shfl_xor(l, d);
  __syncthreads();
  for (int e = 0; e < 2; ++e)
    if (lane + 64 * e < hdim) q[lane + 64 * e] = o[e];
  __syncthreads();
  if (lane < hdim / 4) finish(a, b, head, i, hdim, lane, *reinterpret_cast<const f32x4*>(q + 4 * lane), l == 0.f ? -INFINITY : m, l);
}

// How the rows of `walks` blocks are merged: `groups` workgroups for each
struct Merge {
  bool shared;
  int groups;
  Merge(int64_t walks, int64_t rows_of_head, int tiles) {
    const int rows = (int)std::min<int64_t>(rows_of_head, 16 * tiles);
    // Few rows are of long walks in many parts, which the eight groups of lanes of a row's workgroup take side by side; of many rows that is eight times
    // the workgroups for parts that are few.  us of a call with a workgroup for each row / for eight, 128 columns, e4m3: 4 rows of a walk of 60000 tokens
    // 16.0 / 30.4, 64 rows of 8 walks 20.8 / 26.6, 512 rows 56.2 / 56.2, 4096 rows 54.3 / 53.4, 8192 rows 60.4 / 58.6, 12800 rows 76.4 / 72.2.
    shared = walks * rows <= 4096;
    groups = shared ? rows : (rows + 7) / 8;
  }
};
template <int H>
void go_merge(const CachedArgs& a, hipStream_t s) {
  const int64_t walks = (int64_t)a.sequences * a.c.kv_heads * a.blocks;
  const Merge m(walks, (int64_t)a.group * a.rows, a.tiles);
  const dim3 grid((unsigned)(walks * m.groups));
  if (m.shared) A2D_LAUNCH((cached_merge_kernel<H, true>), grid, dim3(256), 0, s, a, m.groups);
  else A2D_LAUNCH((cached_merge_kernel<H, false>), grid, dim3(256), 0, s, a, m.groups);
}

}  // namespace

CachedPlan plan_cached(int format, int hdim, const CachedArgs& a, int cus, bool workspace) {
  CachedPlan p{};
  const int64_t rows = (int64_t)a.group * a.rows;
  const auto padded = [&](int n) { return (rows + n - 1) / n * n; };
  // Up to 32 rows: blocks of 16 or 32, a wavefront has them all.  More: workgroups of 128 or 256, whichever leaves fewer rows empty.
  // us of blocks of 32 / 128 / 256, 8 sequences of 8192 tokens, 8 heads of 128, e4m3: 40 rows 60.9 / 53.8 / 61.2, 100 rows 87 / 58 / 62, 160 rows
  // 116 / 92 / 78, 256 rows 142 / 98 / 91; 4 sequences, 300 rows of 4 heads of 64, bf16 50 / 35 / 39.
  // Calls of short walks that leave most of the chip idle take blocks of 16 up to 32 rows: 28 rows of 2 heads of 64, 307 keys 8.7 -> 7.6 us, of 16 heads
  // 9.5 -> 9.1 (elsewhere two blocks that read the same keys: 8 sequences of 8192 tokens, 28 rows of 8 heads 39.6, not 49.9).
  const int64_t keys = (int64_t)a.max_tokens + (a.K ? a.rows : 0), walks = (int64_t)a.sequences * a.c.kv_heads;
  const bool idle = keys <= 512 && 2 * walks <= mfma::kXcds * mfma::kXcdCus;
  p.tiles = rows <= 16 || (rows <= 32 && idle) ? 1 : rows <= 32 ? 2 : padded(256) <= padded(128) ? 16 : 8;
  p.shift = p.tiles > 2 ? 6 : 5;
  p.blocks = (int)((rows + 16 * p.tiles - 1) / (16 * p.tiles));
  // (walks whose merge one launch could not hold are many times what fills the chip)
  if (!workspace || keys <= 512 || walks * p.blocks * Merge(walks * p.blocks, rows, p.tiles).groups * 256 >= MAX_THREADS) return p;
  p.workers = (p.tiles == 16 ? 1 : 2) * cus;
  p.part_bytes = 2 * (size_t)p.workers * part_floats(16 * p.tiles, hdim) * sizeof(float);
  p.bytes = p.part_bytes + (size_t)(walks * p.blocks) * sizeof(int2);
  return p;
}

hipError_t launch_cached(Phase ph, int format, int hdim, const CachedArgs& a, hipStream_t s) {
  const hipError_t e = format == A2D_CACHE_BF16 ? launch_cached_bf16(ph, hdim, a, s)
                       : format == A2D_CACHE_E4M3 ? launch_cached_e4m3(ph, hdim, a, s)
                                                  : launch_cached_e2m1(ph, hdim, a, s);
  if (e != hipSuccess || ph == PREPARE || a.workers == 0) return e;
  if (hdim == 64) go_merge<64>(a, s);
  else if (hdim == 80) go_merge<80>(a, s);
  else if (hdim == 96) go_merge<96>(a, s);
  else go_merge<128>(a, s);
  return hipGetLastError();
}

hipError_t launch_cached_generic(int format, int hdim, const CachedArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)a.sequences * a.heads * a.rows));
  if (format == A2D_CACHE_BF16) A2D_LAUNCH((cached_generic_kernel<A2D_CACHE_BF16>), grid, dim3(64), 0, s, a, hdim);
  else if (format == A2D_CACHE_E4M3) A2D_LAUNCH((cached_generic_kernel<A2D_CACHE_E4M3>), grid, dim3(64), 0, s, a, hdim);
  else A2D_LAUNCH((cached_generic_kernel<A2D_CACHE_E2M1>), grid, dim3(64), 0, s, a, hdim);
  return hipGetLastError();
}

}  // namespace a2d
