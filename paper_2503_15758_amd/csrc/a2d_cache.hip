// The paged cache: rows of K and V written into it in 16, 8 or 4 bits, read back, and the ancestors of drafted tokens.
//
// Codes.  32 values of a row share a scale 2^s, s the smallest integer from -100 on with max |x| <= M 2^s (M = 448 for e4m3, 6 for e2m1: the
// largest numbers that the codes have), so that nothing saturates; a code is x / 2^s to the nearest, ties to even.  The division by a power of
// two is exact, so the codes follow from the values alone.  A scale that is no power of two would gain nothing in e4m3, whose steps are
// relative, and cost a multiplication with a rounding in every reader: here the conversions of the matrix operands take it for nothing.
#include "a2d_cache.hpp"

namespace a2d {
namespace {

using mfma::lane_swap;

__device__ __forceinline__ void load_values(const bf16_t* p, float (&v)[8]) {
  const bf16x8 b = *reinterpret_cast<const bf16x8*>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)b[i];
}
__device__ __forceinline__ void load_values(const float* p, float (&v)[8]) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
}

// largest of four lanes
__device__ __forceinline__ unsigned quad_max(unsigned x) {
  const auto swap = [](unsigned u, auto C) {
    return __builtin_bit_cast(unsigned, lane_swap<decltype(C)::value>(__builtin_bit_cast(float, u)));
  };
  x = max(x, swap(x, std::integral_constant<int, 0xB1>{}));     // quad_perm 1 0 3 2
  return max(x, swap(x, std::integral_constant<int, 0x4E>{}));  // 2 3 0 1
}

// The scale byte of a block whose largest |x| has these bits
template <int FMT>
__device__ __forceinline__ unsigned scale_byte(unsigned top) {
  if (top >= 0x7F800000u) return 255;                            // a NaN or an infinity among them
  constexpr int power = FMT == A2D_CACHE_E4M3 ? 8 : 2;           // M = 1.75 2^8, 1.5 2^2
  constexpr unsigned fraction = FMT == A2D_CACHE_E4M3 ? 0x600000u : 0x400000u;
  const int s = (int)(top >> 23) - power + ((top & 0x7FFFFFu) > fraction);        // + 127
  return (unsigned)max(s, CACHE_LOWEST + 127);
}

template <int FMT>
__device__ __forceinline__ void store_codes(char* p, const float (&v)[8], float scale) {
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  if constexpr (FMT == A2D_CACHE_E4M3) {
    u32x2 w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s16x2 c = {0, 0};
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, v[4 * i], v[4 * i + 1], scale, false);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, v[4 * i + 2], v[4 * i + 3], scale, true);
      w[i] = __builtin_bit_cast(unsigned, c);
    }
    *reinterpret_cast<u32x2*>(p) = w;
  } else {
    unsigned w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
    *reinterpret_cast<unsigned*>(p) = w;
  }
}

// Lanes of a row: one for each eight values, in whole fours (a block each)
__host__ __device__ constexpr int row_lanes(int h) { return (h + CACHE_BLOCK - 1) / CACHE_BLOCK * 4; }

// A thread has eight values of K and the same eight of V; blockIdx: rows, head, sequence.
// Bound: HBM, each value read once and its code written once: 8 heads of 128, 16384 tokens from a packed projection 23.8 us, 4.3 TB/s, where a copy of
// as many bytes takes 19.5 (three inputs in turn, of which the last-level cache holds a part, 21.3 us); a token of 64 sequences 3.5 us, its call 6.
template <int H, int FMT, typename T>
__global__ __launch_bounds__(256) void cache_write_kernel(CacheRows a) {
  constexpr int LANES = row_lanes(H), ROW = code_bytes<FMT>(H);
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int j = (int)(t / LANES), chunk = (int)(t % LANES);
  const int h = blockIdx.y, b = blockIdx.z;
  if (j >= a.count) return;                                      // (whole fours of lanes)
  const int src = a.index ? a.index[(int64_t)b * a.count + j] : j;
  const int64_t token = (int64_t)a.starts[b] + j;
  if ((unsigned)src >= (unsigned)a.rows || token < 0 || token > 0x7FFFFFFF) return;
  const unsigned unit = unit_of(a.c, b, h, (int)(token >> 4));
  if (unit == NO_UNIT) return;
  const int64_t row = (int64_t)unit * 16 + (token & 15);
  const bool live = 8 * chunk < H;                               // (H = 80: the last block has two chunks)
  const T* k = reinterpret_cast<const T*>(a.K) + at_row(a.lk, b, h, src) + 8 * chunk;
  const T* v = reinterpret_cast<const T*>(a.V) + at_row(a.lv, b, h, src) + 8 * chunk;
  char *ko = a.c.K + row * ROW + code_bytes<FMT>(8) * chunk, *vo = a.c.V + row * ROW + code_bytes<FMT>(8) * chunk;
  float x[2][8] = {};
  if (live) {
    load_values(k, x[0]);
    load_values(v, x[1]);
  }
  if constexpr (FMT == A2D_CACHE_BF16) {
    if (!live) return;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      bf16x8 y;
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = (bf16_t)x[w][i];
      *reinterpret_cast<bf16x8*>(w ? vo : ko) = y;
    }
  } else {
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      unsigned top = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __builtin_bit_cast(unsigned, x[w][i]) & 0x7FFFFFFFu);
      const unsigned byte = scale_byte<FMT>(quad_max(top));
      if (byte == 255)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[w][i] = 0.f;
      if (live) store_codes<FMT>(w ? vo : ko, x[w], scale_number(byte == 255 ? 127 : byte));
      if ((chunk & 3) == 0) (w ? a.c.Vs : a.c.Ks)[row * 4 + (chunk >> 2)] = (char)byte;
    }
  }
}

// Values of a token that a thread reads: as many as make a store of 16 bytes, so that neighbours' stores are one run, which may leave
// non-temporal.  Bound: HBM, mostly writes; codes that the last-level cache still holds come from there.  8 heads of 128, 16384 tokens to bf16:
// 23.6 us, 4.3 TB/s of reads and writes, where a copy of as many bytes takes 19.5; caches of 34 MB, three in turn, 17.1 us, 5.9 TB/s (through the L2s
// 18.0).  5 sequences, 12 heads of 80, 4135 tokens to fp32, behind the write of 40 rows: 36.0 us, 4.6 TB/s, up to 16 caches in turn 30.6 (through
// the L2s 38.5, two stores of every second 16 bytes 40.4).
template <typename T>
struct Piece;
template <>
struct Piece<bf16_t> {
  static constexpr int N = 8;
  bf16x8 v;
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (bf16_t)0.f;
  }
  template <int FMT>
  __device__ __forceinline__ void read(const char* p, unsigned byte) {
    if constexpr (FMT == A2D_CACHE_BF16) {
      v = *reinterpret_cast<const bf16x8*>(p);
    } else if constexpr (FMT == A2D_CACHE_E4M3) {
      const u32x2 w = *reinterpret_cast<const u32x2*>(p);
      v = decode8<FMT>(w[0], w[1], scale_number(byte));
    } else {
      v = decode8<A2D_CACHE_E2M1>(*reinterpret_cast<const unsigned*>(p), 0, scale_number(byte));
    }
  }
  __device__ __forceinline__ void store(bf16_t* p) const { __builtin_nontemporal_store(v, reinterpret_cast<bf16x8*>(p)); }
};
template <>
struct Piece<float> {
  static constexpr int N = 4;
  f32x4 v;
  __device__ __forceinline__ void clear() { v = f32x4{0.f, 0.f, 0.f, 0.f}; }
  template <int FMT>
  __device__ __forceinline__ void read(const char* p, unsigned byte) {
    if constexpr (FMT == A2D_CACHE_BF16) {
      const bf16x4 b = *reinterpret_cast<const bf16x4*>(p);
      v = f32x4{(float)b[0], (float)b[1], (float)b[2], (float)b[3]};
    } else {
      const unsigned w = FMT == A2D_CACHE_E4M3 ? *reinterpret_cast<const unsigned*>(p) : *reinterpret_cast<const unsigned short*>(p);
      const bf16x8 b = decode8<FMT>(w, 0, scale_number(byte));
      v = f32x4{(float)b[0], (float)b[1], (float)b[2], (float)b[3]};
    }
  }
  __device__ __forceinline__ void store(float* p) const { __builtin_nontemporal_store(v, reinterpret_cast<f32x4*>(p)); }
};

template <int H, int FMT, typename T>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheRows a) {
  constexpr int N = Piece<T>::N, CHUNKS = H / N, ROW = code_bytes<FMT>(H);
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int j = (int)(t / CHUNKS), chunk = (int)(t % CHUNKS);
  const int h = blockIdx.y, b = blockIdx.z;
  if (j >= a.rows) return;
  const int64_t token = (int64_t)a.first + j;
  Piece<T> k, v;
  k.clear();
  v.clear();
  if (token < a.starts[b]) {
    const unsigned unit = unit_of(a.c, b, h, (int)(token >> 4));
    if (unit != NO_UNIT) {
      const int64_t row = (int64_t)unit * 16 + (token & 15), at = row * ROW + code_bytes<FMT>(8) * N / 8 * chunk;
      unsigned ks = 0, vs = 0;
      if constexpr (FMT != A2D_CACHE_BF16) {
        ks = (unsigned char)a.c.Ks[row * 4 + chunk * N / CACHE_BLOCK];
        vs = (unsigned char)a.c.Vs[row * 4 + chunk * N / CACHE_BLOCK];
      }
      k.template read<FMT>(a.c.K + at, ks);
      v.template read<FMT>(a.c.V + at, vs);
    }
  }
  k.store(const_cast<T*>(reinterpret_cast<const T*>(a.K)) + at_row(a.lk, b, h, j) + N * chunk);
  v.store(const_cast<T*>(reinterpret_cast<const T*>(a.V)) + at_row(a.lv, b, h, j) + N * chunk);
}

template <int H, int FMT, typename T>
void go_rows(bool write, const CacheRows& a, hipStream_t s) {
  const int64_t threads = write ? (int64_t)a.count * row_lanes(H) : (int64_t)a.rows * (H / Piece<T>::N);
  const dim3 grid((unsigned)((threads + 255) / 256), (unsigned)a.c.kv_heads, (unsigned)a.sequences);
  if (write) A2D_LAUNCH((cache_write_kernel<H, FMT, T>), grid, dim3(256), 0, s, a);
  else A2D_LAUNCH((cache_read_kernel<H, FMT, T>), grid, dim3(256), 0, s, a);
}
template <int FMT, typename T>
void go_head(bool write, int hdim, const CacheRows& a, hipStream_t s) {
  if (hdim == 64) go_rows<64, FMT, T>(write, a, s);
  else if (hdim == 80) go_rows<80, FMT, T>(write, a, s);
  else if (hdim == 96) go_rows<96, FMT, T>(write, a, s);
  else go_rows<128, FMT, T>(write, a, s);
}
template <typename T>
hipError_t go_format(bool write, int format, int hdim, const CacheRows& a, hipStream_t s) {
  if (format == A2D_CACHE_BF16) go_head<A2D_CACHE_BF16, T>(write, hdim, a, s);
  else if (format == A2D_CACHE_E4M3) go_head<A2D_CACHE_E4M3, T>(write, hdim, a, s);
  else go_head<A2D_CACHE_E2M1, T>(write, hdim, a, s);
  return hipGetLastError();
}

// Ancestors: round k lets every row take what the row 2^k steps up has, so a chain of 256 rows takes eight rounds.  up: a row before it,
// -1: the text, -2: no token (padding, and what follows padding), which is handed down.  Bound: the launch: one sequence of 7 rows 1.8 us, 64 of 250
// 3.9.
constexpr int TREE_ROWS = A2D_TREE_MAX_ROWS, TREE_WORDS = TREE_ROWS / 64;
__global__ __launch_bounds__(TREE_ROWS) void tree_masks_kernel(int rows, int words, const int32_t* parents, const int32_t* lens, uint64_t* masks,
                                                               int32_t* positions) {
  __shared__ uint64_t seen[2][TREE_WORDS][TREE_ROWS];
  __shared__ int above[2][TREE_ROWS];
  const int i = threadIdx.x, b = blockIdx.x;
  uint64_t mine[TREE_WORDS];
#pragma unroll
  for (int w = 0; w < TREE_WORDS; ++w) mine[w] = i >> 6 == w ? (uint64_t)1 << (i & 63) : 0;
  int up = -2;
  if (i < rows) {
    up = parents[(int64_t)b * rows + i];
    if (up < -1 || up >= i) up = -2;
  }
  int side = 0;
  for (int reach = 1; reach < rows; reach *= 2, side ^= 1) {
#pragma unroll
    for (int w = 0; w < TREE_WORDS; ++w) seen[side][w][i] = mine[w];
    above[side][i] = up;
    __syncthreads();
    if (up >= 0) {
#pragma unroll
      for (int w = 0; w < TREE_WORDS; ++w) mine[w] |= seen[side][w][up];
      up = above[side][up];
    }
  }
  if (i >= rows) return;
  const bool token = up == -1;
  int depth = -1;
#pragma unroll
  for (int w = 0; w < TREE_WORDS; ++w) {
    if (w < words) masks[((int64_t)b * rows + i) * words + w] = token ? mine[w] : 0;
    depth += __popcll(mine[w]);
  }
  positions[(int64_t)b * rows + i] = token ? (lens ? max(lens[b], 0) : 0) + depth : 0;
}

}  // namespace

hipError_t launch_cache_write(int format, int hdim, int dtype, const CacheRows& a, hipStream_t s) {
  return dtype == A2D_F32 ? go_format<float>(true, format, hdim, a, s) : go_format<bf16_t>(true, format, hdim, a, s);
}
hipError_t launch_cache_read(int format, int hdim, int dtype, const CacheRows& a, hipStream_t s) {
  return dtype == A2D_F32 ? go_format<float>(false, format, hdim, a, s) : go_format<bf16_t>(false, format, hdim, a, s);
}
hipError_t launch_tree_masks(int sequences, int rows, const int32_t* parents, const int32_t* lens, uint64_t* masks, int32_t* positions,
                             hipStream_t s) {
  A2D_LAUNCH(tree_masks_kernel, dim3((unsigned)sequences), dim3(TREE_ROWS), 0, s, rows, (rows + 63) / 64, parents, lens, masks, positions);
  return hipGetLastError();
}

}  // namespace a2d
