// Attention under score rules, the plain form of it: fp32 arithmetic on the vector ALUs, one wavefront a query row (forward,
// dQ) or a key (dK, dV), 64 scores at a time, lane = key or row.  Both input types, any nq / nkv.  Bound by its operand
// loads (every row reads all of K and V from the caches) far from any peak; the debug switch a2d_debug_force_generic
// routes calls here, to tell a kernel's mistake from a caller's.
#include "a2d_scored.hpp"

namespace a2d {
namespace {

constexpr int LANES = 64, CH = 128 / LANES;        // columns of a lane: lane, lane + 64 (H <= 128)

template <class F>
__device__ __forceinline__ float all_lanes(float x, F&& f) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x = f(x, __shfl_xor(x, o, 64));
  return x;
}
__device__ __forceinline__ float max_of(float x) { return all_lanes(x, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float sum_of(float x) { return all_lanes(x, [](float a, float b) { return a + b; }); }

template <typename T>
__device__ __forceinline__ float dot(const T* a, const T* b, int n) {
  float s = 0.f;
  for (int j = 0; j < n; ++j) s = fmaf(to_f32(a[j]), to_f32(b[j]), s);
  return s;
}
// y and dy / dz of z
__device__ __forceinline__ void capped(float cap, float z, float& y, float& dy) {
  y = z;
  dy = 1.f;
  if (cap != 0.f) {
    const float t = tanhf(z / cap);
    y = cap * t;
    dy = 1.f - t * t;
  }
}
__device__ __forceinline__ float tokens_apart(const ScoreRules& r, int i, int k) {
  const int64_t far = r.rel + (int64_t)(i - k) * r.step;
  return (float)(far < 0 ? -far : far);
}
__device__ __forceinline__ float slope_of(const ScoreRules& r, int head) { return r.slopes ? r.slopes[head] : 0.f; }

template <typename T>
__device__ __forceinline__ void put(void* out, int64_t at, float x, bool rounded) {
  if (rounded) static_cast<T*>(out)[at] = (T)x;
  else static_cast<float*>(out)[at] = x;
}

template <typename T>
__global__ __launch_bounds__(LANES) void scored_fwd_generic_kernel(a2d_tile_desc d, ScoreRules r, const T* Q, const T* K,
                                                                   const T* V, void* out0, float* out1, float* out2) {
  const int head = blockIdx.y, i = blockIdx.x, lane = threadIdx.x, H = d.hdim;
  const int64_t row = (int64_t)head * d.nq + i;
  Q += head * d.lq.head + i * d.lq.row;
  K += head / r.group * d.lk.head;
  V += head / r.group * d.lv.head;
  const Run run = visible_run(d, r, head, i);
  const float slope = slope_of(r, head);
  float m = -INFINITY, l = 0.f, n[CH] = {0.f, 0.f};
  if (r.acc) {
    m = out1[row];
    l = out2[row];
    for (int c = 0; c < CH; ++c)
      if (lane + LANES * c < H) n[c] = static_cast<const float*>(out0)[row * H + lane + LANES * c];
  }
  for (int k0 = run.lo; k0 < run.lo + run.n; k0 += LANES) {
    const int k = k0 + lane, keys = min(LANES, run.lo + run.n - k0);
    float s = -INFINITY, dy;
    if (lane < keys) {
      capped(r.cap, d.scale * dot(Q, K + k * d.lk.row, H), s, dy);
      s = fmaf(-slope, tokens_apart(r, i, k), s);
    }
    const float m_new = fmaxf(m, max_of(s)), use = m_new == -INFINITY ? 0.f : m_new;
    const float p = expf(s - use), alpha = expf(m - use);
    m = m_new;
    l = l * alpha + sum_of(p);
    for (int c = 0; c < CH; ++c) n[c] *= alpha;
    for (int j = 0; j < keys; ++j) {
      const float pj = __shfl(p, j, 64);
      for (int c = 0; c < CH; ++c)
        if (lane + LANES * c < H) n[c] = fmaf(pj, to_f32(V[(k0 + j) * d.lv.row + lane + LANES * c]), n[c]);
    }
  }
  for (int c = 0; c < CH; ++c)
    if (lane + LANES * c < H) put<T>(out0, row * H + lane + LANES * c, r.norm ? (l > 0.f ? n[c] / l : 0.f) : n[c], r.norm != 0);
  if (lane == 0) {
    out1[row] = !r.norm ? m : l > 0.f ? m + logf(l) : -INFINITY;
    if (!r.norm) out2[row] = l;
  }
}

// P and dZ of one score
template <typename T>
__device__ __forceinline__ void gradient(const a2d_tile_desc& d, const ScoreRules& r, const T* q, const T* k, const T* g, const T* v,
                                         float lse, float delta, float slope, int i, int key, float& p, float& dz) {
  float y, dy;
  capped(r.cap, d.scale * dot(q, k, d.hdim), y, dy);
  p = expf(y - fmaf(slope, tokens_apart(r, i, key), lse));      // (bias and lse may be thousands where their difference is a few units)
  dz = p * (dot(g, v, d.hdim) - delta) * dy;
}

template <typename T>
__global__ __launch_bounds__(LANES) void scored_dq_generic_kernel(a2d_tile_desc d, ScoreRules r, const T* Q, const T* K,
                                                                  const T* V, const T* O, const T* dO, const float* lse,
                                                                  float* delta, void* dQ) {
  const int head = blockIdx.y, i = blockIdx.x, lane = threadIdx.x, H = d.hdim;
  const int64_t row = (int64_t)head * d.nq + i;
  const T *q = Q + head * d.lq.head + i * d.lq.row, *g = dO + head * d.ldo.head + i * d.ldo.row, *o = O + head * d.lo.head + i * d.lo.row;
  K += head / r.group * d.lk.head;
  V += head / r.group * d.lv.head;
  const Run run = visible_run(d, r, head, i);
  const float slope = slope_of(r, head);
  float del = 0.f, acc[CH] = {0.f, 0.f};
  for (int c = 0; c < CH; ++c)
    if (lane + LANES * c < H) del = fmaf(to_f32(o[lane + LANES * c]), to_f32(g[lane + LANES * c]), del);
  del = sum_of(del);
  const float L = lse[row];
  if (lane == 0) delta[row] = del;
  for (int k0 = run.lo; L != -INFINITY && k0 < run.lo + run.n; k0 += LANES) {
    const int k = k0 + lane, keys = min(LANES, run.lo + run.n - k0);
    float p, dz = 0.f;
    if (lane < keys) gradient(d, r, q, K + k * d.lk.row, g, V + k * d.lv.row, L, del, slope, i, k, p, dz);
    for (int j = 0; j < keys; ++j) {
      const float z = __shfl(dz, j, 64);
      for (int c = 0; c < CH; ++c)
        if (lane + LANES * c < H) acc[c] = fmaf(z, to_f32(K[(k0 + j) * d.lk.row + lane + LANES * c]), acc[c]);
    }
  }
  for (int c = 0; c < CH; ++c) {
    if (lane + LANES * c >= H) continue;
    const int64_t at = row * H + lane + LANES * c;
    put<T>(dQ, at, acc[c] * d.scale + (r.acc ? static_cast<float*>(dQ)[at] : 0.f), r.norm != 0);
  }
}

template <typename T>
__global__ __launch_bounds__(LANES) void scored_dkdv_generic_kernel(a2d_tile_desc d, ScoreRules r, const T* Q, const T* K,
                                                                    const T* V, const T* dO, const float* lse,
                                                                    const float* delta, void* dK, void* dV) {
  const int kvh = blockIdx.y, key = blockIdx.x, lane = threadIdx.x, H = d.hdim;
  const int64_t row = (int64_t)kvh * d.nkv + key;
  const T *k = K + kvh * d.lk.head + key * d.lk.row, *v = V + kvh * d.lv.head + key * d.lv.row;
  float dk[CH] = {0.f, 0.f}, dv[CH] = {0.f, 0.f};
  for (int head = kvh * r.group; head < (kvh + 1) * r.group; ++head) {
    const T *q = Q + head * d.lq.head, *g = dO + head * d.ldo.head;
    const float slope = slope_of(r, head);
    for (int i0 = 0; i0 < d.nq; i0 += LANES) {
      const int i = i0 + lane;
      float p = 0.f, dz = 0.f;
      bool sees = false;
      if (i < d.nq) {
        const Run run = visible_run(d, r, head, i);
        const float L = lse[(int64_t)head * d.nq + i];
        sees = (unsigned)(key - run.lo) < (unsigned)run.n && L != -INFINITY;
        if (sees) gradient(d, r, q + i * d.lq.row, k, g + i * d.ldo.row, v, L, delta[(int64_t)head * d.nq + i], slope, i, key, p, dz);
      }
      for (uint64_t left = __ballot(sees); left; left &= left - 1) {
        const int j = __builtin_ctzll(left);
        const float pj = __shfl(p, j, 64), zj = __shfl(dz, j, 64);
        for (int c = 0; c < CH; ++c) {
          if (lane + LANES * c >= H) continue;
          dv[c] = fmaf(pj, to_f32(g[(i0 + j) * d.ldo.row + lane + LANES * c]), dv[c]);
          dk[c] = fmaf(zj, to_f32(q[(i0 + j) * d.lq.row + lane + LANES * c]), dk[c]);
        }
      }
    }
  }
  for (int c = 0; c < CH; ++c) {
    if (lane + LANES * c >= H) continue;
    put<T>(dK, row * H + lane + LANES * c, dk[c] * d.scale, r.norm != 0);
    put<T>(dV, row * H + lane + LANES * c, dv[c], r.norm != 0);
  }
}

template <typename T>
hipError_t fwd(const a2d_tile_desc& d, const ScoreRules& r, const void* Q, const void* K, const void* V, void* out0, float* out1,
               float* out2, hipStream_t s) {
  A2D_LAUNCH((scored_fwd_generic_kernel<T>), dim3(d.nq, d.heads), dim3(LANES), 0, s, d, r, (const T*)Q,
             (const T*)K, (const T*)V, out0, out1, out2);
  return hipGetLastError();
}
template <typename T>
hipError_t bwd(const a2d_tile_desc& d, const ScoreRules& r, const void* Q, const void* K, const void* V, const void* O,
               const void* dO, const float* lse, float* delta, void* dQ, void* dK, void* dV, hipStream_t s) {
  A2D_LAUNCH((scored_dq_generic_kernel<T>), dim3(d.nq, d.heads), dim3(LANES), 0, s, d, r, (const T*)Q,
             (const T*)K, (const T*)V, (const T*)O, (const T*)dO, lse, delta, dQ);
  A2D_LAUNCH((scored_dkdv_generic_kernel<T>), dim3(d.nkv, d.heads / r.group), dim3(LANES), 0, s, d, r,
             (const T*)Q, (const T*)K, (const T*)V, (const T*)dO, lse, (const float*)delta, dK, dV);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_scored_fwd_generic(const a2d_tile_desc& d, const ScoreRules& r, const void* Q, const void* K, const void* V,
                                     void* out0, float* out1, float* out2, hipStream_t s) {
  return d.dtype == A2D_F32 ? fwd<float>(d, r, Q, K, V, out0, out1, out2, s) : fwd<bf16_t>(d, r, Q, K, V, out0, out1, out2, s);
}
hipError_t launch_scored_bwd_generic(const a2d_tile_desc& d, const ScoreRules& r, const void* Q, const void* K, const void* V,
                                     const void* O, const void* dO, const float* lse, float* delta, void* dQ, void* dK,
                                     void* dV, hipStream_t s) {
  return d.dtype == A2D_F32 ? bwd<float>(d, r, Q, K, V, O, dO, lse, delta, dQ, dK, dV, s)
                            : bwd<bf16_t>(d, r, Q, K, V, O, dO, lse, delta, dQ, dK, dV, s);
}

// ---- ranges of packed documents: a thread a row, a binary search of its document.  A few thousand rows: bound by the launch.
namespace {
__global__ __launch_bounds__(256) void document_ranges_kernel(int documents, const int32_t* __restrict__ starts,
                                                              const int32_t* __restrict__ prefix, int causal, int64_t first,
                                                              int step, int rows, int2* __restrict__ ranges) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= rows) return;
  const int64_t t = first + (int64_t)i * step;
  int a = 0, b = documents + 1;                    // starts[0 .. a) <= t < starts[b ..)
  while (a < b) {
    const int mid = (a + b) >> 1;
    if (starts[mid] <= t) a = mid + 1; else b = mid;
  }
  int2 out = {0, 0};
  if (a >= 1 && a <= documents) {                  // (of empty documents that start where this one does, the last is left out)
    const int from = starts[a - 1], to = starts[a];
    int64_t end = to;
    if (causal) {
      end = t + 1;
      if (prefix && (int64_t)from + prefix[a - 1] > end) end = (int64_t)from + prefix[a - 1];
      if (end > to) end = to;
    }
    out = int2{from, (int)end};
  }
  ranges[i] = out;
}
}  // namespace

hipError_t launch_document_ranges(int documents, const int32_t* starts, const int32_t* prefix, int causal, int64_t first, int step,
                                  int rows, int32_t* ranges, hipStream_t s) {
  A2D_LAUNCH(document_ranges_kernel, dim3((rows + 255) / 256), dim3(256), 0, s, documents, starts, prefix, causal, first, step, rows,
             reinterpret_cast<int2*>(ranges));
  return hipGetLastError();
}

}  // namespace a2d
