// What the kernels on the fp32 matrix units share: tiles of 16 rows in LDS, the fragments read from them, contractions and the merge of
// key lanes (see a2d_f32_mfma.hip for their layouts and what they measured).
#pragma once
#include "a2d_mfma.hpp"

namespace a2d {
namespace f32 {

using mfma::gptr_t;
using mfma::static_for;

constexpr int BLK = 16;                      // rows of one step of a walk
constexpr int KL = 4;                        // key lanes (wavefronts) of a workgroup
constexpr float kRescaleThreshold = 8.0f;    // log2 units (lazy rescaling, as in the bf16 forward)

__device__ __forceinline__ f32x4 mma4(float a, float b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 zero4() { return f32x4{0.f, 0.f, 0.f, 0.f}; }
template <typename T>
__device__ __forceinline__ T gload(gptr_t base, unsigned byte_off) {
  return *reinterpret_cast<const __attribute__((address_space(1))) T*>(base + byte_off);
}

// Natural rows: H / 16 pieces of 16 bytes per lane
template <int H>
struct Nat {
  f32x4 v[H / 16];
  __device__ __forceinline__ void load(gptr_t base, unsigned row, unsigned row_bytes, int g4) {
    const unsigned off = __umul24(row, row_bytes) + 16 * g4;
#pragma unroll
    for (int y = 0; y < H / 16; ++y) v[y] = gload<f32x4>(base, off + 64 * y);
  }
};

// Column groups of a row for the transposed operand: H / 64 groups of 64 columns (4 per lane) and a
// rest of 32 (2 per lane) or 16 (1 per lane); T = tile index 0 .. H / 16 - 1
template <int H>
struct Cols {
  static constexpr int N4 = H / 64, REST = H % 64;
  f32x4 a[N4];
  f32x4 b;                                   // 1, 2 of it used when there is a rest
  __device__ __forceinline__ void load(gptr_t base, unsigned row, unsigned row_bytes, int l15) {
    const unsigned off = __umul24(row, row_bytes);
#pragma unroll
    for (int G = 0; G < N4; ++G) a[G] = gload<f32x4>(base, off + 256 * G + 16 * l15);
    if constexpr (REST == 32) {
      const f32x2 w = gload<f32x2>(base, off + 256 * N4 + 8 * l15);
      b[0] = w[0]; b[1] = w[1];
    }
    if constexpr (REST == 16) b[0] = gload<float>(base, off + 256 * N4 + 4 * l15);
  }
  template <int T>
  __device__ __forceinline__ float get() const {
    if constexpr (T < 4 * N4) return a[T / 4][T % 4]; else return b[T - 4 * N4];
  }
};

typedef __attribute__((address_space(3))) char* lds_t;
template <typename T>
__device__ __forceinline__ T lload(lds_t p) { return *reinterpret_cast<__attribute__((address_space(3))) T*>(p); }
template <typename T>
__device__ __forceinline__ void lstore(lds_t p, T v) { *reinterpret_cast<__attribute__((address_space(3))) T*>(p) = v; }

// A wavefront's tile of 16 rows that is loaded straight into LDS (see mfma::Blocks16: here a block is 16 rows x 16 columns).
// Blocks lie 64 bytes more than their size apart, so that the columns' reads, which take 64 bytes of four blocks at a time,
// meet every bank once too.  (Not so those of the last 32 columns at H = 96, which meet half of the banks twice, and of the last 16 at
// H = 80, a quarter four times: 10 % of the kernel's LDS cycles at H = 96.)
template <int H>
struct Blocks {
  static constexpr int N = H / 16, N4 = Cols<H>::N4, REST = Cols<H>::REST, STRIDE = mfma::BLOCK + 64, BYTES = N * STRIDE;
  lds_t base, nat, col, rest;                // + this lane's place for natural rows, for columns (row 4 g), for the last ones
  __device__ __forceinline__ void init(lds_t b, int l15, int g4) {
    const int swap = mfma::block_swap(g4);
    base = b;
    nat = b + l15 * 64 + 16 * (g4 ^ mfma::block_swap(l15 >> 2));
    col = b + (l15 >> 2) * STRIDE + 256 * g4 + 16 * ((l15 & 3) ^ swap);
    rest = b + 4 * N4 * STRIDE + 256 * g4 +
           (REST == 32 ? (l15 >> 3) * STRIDE + 16 * ((l15 >> 1 & 3) ^ swap) + 8 * (l15 & 1) : 16 * ((l15 >> 2) ^ swap) + 4 * (l15 & 3));
  }
  // lane i's row i >> 2 of the tile is at byte `off` of from; + chunk(i)
  static __device__ __forceinline__ unsigned chunk(int lane) { return 16 * ((lane & 3) ^ mfma::block_swap(lane >> 4)); }
  __device__ __forceinline__ void load(gptr_t from, unsigned off) const {
    static_for<0, N>([&](auto Y) {
      constexpr int y = decltype(Y)::value;
      mfma::dma_b128<64 * y>((unsigned)(uintptr_t)base + y * STRIDE, from, off);
    });
  }
  __device__ __forceinline__ f32x4 row(int y) const { return lload<f32x4>(nat + y * STRIDE); }
  // what this lane has loaded
  __device__ __forceinline__ f32x4 own(int y, int lane) const { return lload<f32x4>(base + y * STRIDE + 16 * lane); }
  __device__ __forceinline__ void cols(Cols<H>& c, int r) const {
#pragma unroll
    for (int G = 0; G < N4; ++G) c.a[G] = lload<f32x4>(col + 64 * r + 4 * G * STRIDE);
    if constexpr (REST == 32) {
      const f32x2 w = lload<f32x2>(rest + 64 * r);
      c.b[0] = w[0]; c.b[1] = w[1];
    }
    if constexpr (REST == 16) c.b[0] = lload<float>(rest + 64 * r);
  }
};
// before a load into a tile that has been read
__device__ __forceinline__ void reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// D layout of the transposed results: acc[T][r] is column col<T>(g, r) of the lane's row (l15)
template <int H>
struct Out {
  f32x4 acc[H / 16];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int t = 0; t < H / 16; ++t) acc[t] = zero4();
  }
  __device__ __forceinline__ void scale(float f) {
#pragma unroll
    for (int t = 0; t < H / 16; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[t][r] *= f;
  }
  // The 16-byte pieces of the lane's row: f(column, four places (t, r) of the accumulators)
  template <class F>
  __device__ __forceinline__ void pieces(int g4, F&& f) {
    constexpr int N4 = Cols<H>::N4, REST = Cols<H>::REST;
#pragma unroll
    for (int G = 0; G < N4; ++G)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        f(64 * G + 16 * g4 + 4 * r, [=](int e) { return 4 * G + e; }, [=](int) { return r; });
    if constexpr (REST == 32) {
#pragma unroll
      for (int r = 0; r < 4; r += 2)
        f(64 * N4 + 8 * g4 + 2 * r, [=](int e) { return 4 * N4 + (e & 1); }, [=](int e) { return r + (e >> 1); });
    }
    if constexpr (REST == 16) f(64 * N4 + 4 * g4, [=](int) { return 4 * N4; }, [=](int e) { return e; });
  }
  __device__ __forceinline__ void store(float* row, int g4, float mul, bool add = false) {
    pieces(g4, [&](int col, auto t, auto r) {
      f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = acc[t(e)][r(e)] * mul;
      if (add) {
        const f32x4 o = *reinterpret_cast<const f32x4*>(row + col);
        v[0] += o[0]; v[1] += o[1]; v[2] += o[2]; v[3] += o[3];
      }
      *reinterpret_cast<f32x4*>(row + col) = v;
    });
  }
  __device__ __forceinline__ void load(const float* row, int g4) {
    pieces(g4, [&](int col, auto t, auto r) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(row + col);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[t(e)][r(e)] = v[e];
    });
  }
  // acc += rows^T * b over the 4 rows (one per group) `c` holds
  __device__ __forceinline__ void contract(const Cols<H>& c, float b) {
    static_for<0, H / 16>([&](auto T) {
      constexpr int t = decltype(T)::value;
      acc[t] = mma4(c.template get<t>(), b, acc[t]);
    });
  }
};

// 16 x 16 results of contractions over H of a tile's rows with RT sets of rows in registers (two
// accumulators each).  The tile's pieces are requested one ahead of their use.
template <int H, int RT>
__device__ __forceinline__ void dot_rows(f32x4 (&out)[RT], const Blocks<H>& a, const Nat<H> (&b)[RT]) {
  constexpr int N = H / 16;
  f32x4 s1[RT], ring[2];
#pragma unroll
  for (int t = 0; t < RT; ++t) { out[t] = zero4(); s1[t] = zero4(); }
  ring[0] = a.row(0);
  ring[1] = a.row(1);
  __builtin_amdgcn_sched_barrier(0);
  static_for<0, N>([&](auto Y) {
    constexpr int y = decltype(Y)::value;
    const f32x4 v = ring[y & 1];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      out[t] = mma4(v[0], b[t].v[y][0], out[t]);
      s1[t] = mma4(v[1], b[t].v[y][1], s1[t]);
      out[t] = mma4(v[2], b[t].v[y][2], out[t]);
      s1[t] = mma4(v[3], b[t].v[y][3], s1[t]);
    }
    if constexpr (y + 2 < N) ring[y & 1] = a.row(y + 2);
    __builtin_amdgcn_sched_barrier(0);
  });
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) out[t][r] += s1[t][r];
}

// The backward's two contractions over H of a step, s = rows of `a` . fa and d = rows of `b` . fb, as one stream of MFMAs: the
// tiles' pieces are requested two ahead of their use across the seam (`seam()`: before b's first), and what `between(y)` does
// behind the MFMAs of d's piece y (s is complete from y = 1 on) runs while they do.
template <int H, class S, class F>
__device__ __forceinline__ void dot_two(f32x4& s, f32x4& d, const Blocks<H>& a, const Nat<H>& fa, const Blocks<H>& b,
                                        const Nat<H>& fb, S&& seam, F&& between) {
  constexpr int N = H / 16;
  f32x4 acc[2][2] = {{zero4(), zero4()}, {zero4(), zero4()}}, ring[2] = {a.row(0), a.row(1)};
  __builtin_amdgcn_sched_barrier(0);
  static_for<0, 2 * N>([&](auto I) {
    constexpr int i = decltype(I)::value, of = i / N, y = i % N, next = i + 2;
    const f32x4 v = ring[i & 1];
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[of][e & 1] = mma4(v[e], (of ? fb : fa).v[y][e], acc[of][e & 1]);
    if constexpr (next == N) seam();
    if constexpr (next < 2 * N) ring[i & 1] = next < N ? a.row(next) : b.row(next - N);
    if constexpr (i == N + 1) {
#pragma unroll
      for (int r = 0; r < 4; ++r) s[r] = acc[0][0][r] + acc[0][1][r];
    }
    if constexpr (of == 1) between(std::integral_constant<int, y>{});
    __builtin_amdgcn_sched_barrier(0);
  });
#pragma unroll
  for (int r = 0; r < 4; ++r) d[r] = acc[1][0][r] + acc[1][1][r];
}

// Sum of N results over the KL wavefronts of the workgroup, by halves: the upper half writes, the
// lower half adds; wavefront 0 ends up with the total.  xch: KL / 2 areas of N * 64 16-byte pieces.
template <int N, class Get>
__device__ __forceinline__ void merge_lanes(f32x4* xch, int kl, int lane, Get&& get) {
#pragma unroll
  for (int half = KL / 2; half >= 1; half /= 2) {
    __syncthreads();
    if (kl >= half && kl < 2 * half) {
#pragma unroll
      for (int i = 0; i < N; ++i) xch[((kl - half) * N + i) * 64 + lane] = get(i);
    }
    __syncthreads();
    if (kl < half) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const f32x4 v = xch[(kl * N + i) * 64 + lane];
        f32x4& a = get(i);
        a[0] += v[0]; a[1] += v[1]; a[2] += v[2]; a[3] += v[3];
      }
    }
  }
}

}  // namespace f32
}  // namespace a2d
