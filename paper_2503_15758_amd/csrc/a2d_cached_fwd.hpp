// Attention of a few rows of each sequence - new tokens, a tree of drafted ones - against the paged cache, bf16 on the matrix units.
//
//   s = scale <q, k>;  row i sees all cached tokens of its sequence and the drafted rows j whose bit is set in its mask (no masks: j <= i);
//   N = sum 2^(s' - m') v, l = sum 2^(s' - m') in log2 units, one pass over the keys.
//
// A workgroup has a block of 16 or 32 rows (query heads of a group and rows of a sequence, numbered through) of one key/value head, and
// a run of its keys in steps of 32, dealt in turn to its four wavefronts.  Each wavefront keeps (N, m, l) of all the block's rows to itself: no
// barrier on the walk, the four are joined through LDS at its end.
//  - S^T = K Q^T: a lane's part of K comes straight from memory, 16 values in a piece (16 bytes of e4m3): the order in which the columns
//    are contracted is the one in which pieces lie (half a row apart they fill whole lines), and Q is held in the same.
//  - O^T += V^T P^T: V goes through LDS of the wavefront's own, decoded, for the transposing reads.
//  - Codes are decoded with their scales by the conversion itself, exactly (a2d_cache.hpp); so only P is rounded, to two bf16
//    numbers (2^-17): these calls wait for memory.
//  - Pages: 64 page numbers at a time are in the lanes of a register, and a step's two are read from there as scalars.
// Bound: HBM for long texts.  A token of 8 sequences, 32 / 8 heads of 128, 73622 tokens in e4m3: 28 us, 5.5 TB/s (with the merge and the second launch
// 37).  Short ones: what a walk costs besides its steps, some 5 us of dependent requests and of instructions that are fetched for the first time
// (7 rows over 300 tokens, 8 / 2 heads of 64: 6.9 us a call).
#pragma once
#include "a2d_cached_cut.hpp"

namespace a2d {
namespace cached {

using namespace mfma;

constexpr int WAVES = 4, STEP = 32;
constexpr float LOW = -0x1.fffffep127f;              // a reference that no score is below
// References (log2 units) from which on a score's product with the scale is rounded before the reference is taken off, as the reference is: a row's
// largest exponent is then 0.  Taken from the unrounded product it is the reference's rounding, up to half a step, which is 1/2 below 2^24 (and all of
// a row's probabilities have that factor), but passes the range of the exponential from 2^31 on.  Below, the unrounded product is the
// more exact one: keys next to each other differ by their scores alone.
constexpr float ROUNDED = 0x1p24f;
// (keeps a branch one whose scores stay where they are: as selects of all of them it takes a register more for each)
__device__ __forceinline__ float in_place(float x) {
  asm volatile("" : "+v"(x));
  return x;
}
// what a wavefront's part of a row is to be multiplied with to be relative to the row's largest score, top = m * c2
__device__ __forceinline__ float part_factor(float ref, float top) {
#pragma clang fp contract(off)                       // (not from the unrounded product, which the reference may be)
  return fast_exp2(ref - top);
}

template <int N>
struct Words { unsigned w[N]; };
// N = 1, 2, 4, 8 dwords
template <int N>
__device__ __forceinline__ Words<N> load_words(gptr_t base, unsigned off) {
  Words<N> r;
  if constexpr (N == 1) {
    r.w[0] = *reinterpret_cast<const __attribute__((address_space(1))) unsigned*>(base + off);
  } else if constexpr (N == 2) {
    const u32x2 x = *reinterpret_cast<const __attribute__((address_space(1))) u32x2*>(base + off);
    r.w[0] = x[0];
    r.w[1] = x[1];
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const u32x4 x = gload_b128(base, off + 16 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) r.w[4 * i + e] = x[e];
    }
  }
  return r;
}

// How a head size's columns fall into a lane's pieces.  Lane group g = lane / 16 has the columns 64 j + 16 g .. + 15 (slices 2 j and
// 2 j + 1 of the contraction) and, of the rest, 64 JF + 8 g .. + 7 (the last slice; H = 80: groups 0 and 1).
template <int H>
struct Head {
  static constexpr int HD = padded_head(H), KS = HD / 32, HT = H / 16, JF = H / 64, REST = (H % 64) / 8;
  static constexpr int PIECES = H / 16, NV = (PIECES + 3) / 4;             // of a row of V; loads of a tile
  static constexpr int AREA = 2 * KS * BLOCK;                              // of a wavefront in LDS
};

// a lane's codes of 16 keys as they come from memory
template <int H, int FMT>
struct Codes {
  using G = Head<H>;
  static constexpr int W = code_bytes<FMT>(16) / 4;
  Words<W> k[G::JF], v[G::NV];
  Words<(W + 1) / 2> rest;
  unsigned ks, vs;
};

// Where a lane's pieces lie in a tile of 16 rows: of row lane & 15, of K as above, of V the pieces 4 n + g.  (16 lanes that write into LDS together
// then meet every bank once; with a row's pieces side by side they met a quarter of them, four times: 64 rows, 8 sequences 140 us, so 137.)
template <int H>
struct Lane {
  using G = Head<H>;
  int row, g;
  unsigned lds;                // of its first piece in the blocks of a tile of V
  bool has_rest;
  __device__ __forceinline__ void init(int lane) {
    row = lane & 15;
    g = lane >> 4;
    has_rest = g < G::REST;
    lds = (g >> 1) * BLOCK + row * 64 + 16 * ((2 * (g & 1)) ^ block_swap(row >> 2));
  }
  __device__ __forceinline__ bool live(int n) const { return 4 * n + 4 <= G::PIECES || 4 * n + g < G::PIECES; }
  // (pieces that there are none of: the row's first)
  __device__ __forceinline__ int piece(int n) const { return live(n) ? 4 * n + g : 0; }
};

// The codes of one unit of the cache
template <int H, int FMT>
__device__ __forceinline__ void load_unit(Codes<H, FMT>& c, const CacheView& view, unsigned unit, const Lane<H>& l) {
  using G = Head<H>;
  constexpr int ROW = code_bytes<FMT>(H), W = Codes<H, FMT>::W;
  const gptr_t k = uniform_gptr(view.K + (uint64_t)unit * (16 * ROW)), v = uniform_gptr(view.V + (uint64_t)unit * (16 * ROW));
#pragma unroll
  for (int j = 0; j < G::JF; ++j) c.k[j] = load_words<W>(k, l.row * ROW + l.g * code_bytes<FMT>(16) + j * code_bytes<FMT>(64));
  if constexpr (G::REST)       // (lanes without columns there take the row's first)
    c.rest = load_words<(W + 1) / 2>(k, l.row * ROW + (l.has_rest ? code_bytes<FMT>(64) * G::JF + l.g * code_bytes<FMT>(8) : 0));
#pragma unroll
  for (int n = 0; n < G::NV; ++n) c.v[n] = load_words<W>(v, l.row * ROW + l.piece(n) * code_bytes<FMT>(16));
  if constexpr (FMT != A2D_CACHE_BF16) {
    const gptr_t ks = uniform_gptr(view.Ks + (uint64_t)unit * 64), vs = uniform_gptr(view.Vs + (uint64_t)unit * 64);
    c.ks = load_words<1>(ks, l.row * 4).w[0];
    c.vs = load_words<1>(vs, l.row * 4).w[0];
  }
}

// 16 drafted rows from `first` on (the last row in place of those behind it)
template <int H>
__device__ __forceinline__ void load_drafts(Codes<H, A2D_CACHE_BF16>& c, const CachedArgs& a, int b, int h, int first, const Lane<H>& l) {
  using G = Head<H>;
  const gptr_t k = uniform_gptr(a.K + 2 * at_row(a.lk, b, h, 0)), v = uniform_gptr(a.V + 2 * at_row(a.lv, b, h, 0));
  const unsigned kr = (unsigned)min(first + l.row, a.rows - 1) * (unsigned)(2 * a.lk.row);
#pragma unroll
  for (int j = 0; j < G::JF; ++j) c.k[j] = load_words<8>(k, kr + l.g * 32 + j * 128);
  if constexpr (G::REST) c.rest = load_words<4>(k, kr + (l.has_rest ? 128 * G::JF + l.g * 16 : 0));
#pragma unroll
  for (int n = 0; n < G::NV; ++n)
    c.v[n] = load_words<8>(v, (unsigned)min(first + l.row, a.rows - 1) * (unsigned)(2 * a.lv.row) + l.piece(n) * 32);
}

template <int FMT, int N>
__device__ __forceinline__ bf16x8 decode_half(const Words<N>& w, int half, float scale) {
  if constexpr (FMT == A2D_CACHE_BF16) {
    return __builtin_bit_cast(bf16x8, u32x4{w.w[4 * half], w.w[4 * half + 1], w.w[4 * half + 2], w.w[4 * half + 3]});
  } else if constexpr (FMT == A2D_CACHE_E4M3) {
    return decode8<FMT>(w.w[2 * half], w.w[2 * half + 1], scale);
  } else {
    return decode8<FMT>(w.w[half], 0, scale);
  }
}
__device__ __forceinline__ void lds_store(unsigned at, bf16x8 x) {
  *reinterpret_cast<__attribute__((address_space(3))) bf16x8*>((uintptr_t)at) = x;
}
// Columns 16 h + 4 g .. + 3 of row r of a tile, which begins at `row` in the tile's first block
__device__ __forceinline__ unsigned quad_at(unsigned row, int r, int h, int g) {
  return row + (h >> 1) * BLOCK + 16 * ((2 * (h & 1) + (g >> 1)) ^ block_swap(r >> 2)) + 8 * (g & 1);
}
__device__ __forceinline__ bf16x4 lds_quad(unsigned at) {
  return *reinterpret_cast<const __attribute__((address_space(3))) bf16x4*>((uintptr_t)at);
}
__device__ __forceinline__ bf16x8 zero8() { return __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0}); }

// K of a tile as fragments
template <int H, int FMT>
__device__ __forceinline__ void decode_keys(bf16x8 (&kf)[Head<H>::KS], const Codes<H, FMT>& c, const Lane<H>& l) {
  using G = Head<H>;
#pragma unroll
  for (int j = 0; j < G::JF; ++j) {
    float scale = 1.f;
    if constexpr (FMT != A2D_CACHE_BF16) scale = scale_number(c.ks >> (16 * j + 8 * (l.g >> 1)) & 255);
    kf[2 * j] = decode_half<FMT>(c.k[j], 0, scale);
    kf[2 * j + 1] = decode_half<FMT>(c.k[j], 1, scale);
  }
  if constexpr (G::REST) {
    float scale = 1.f;
    if constexpr (FMT != A2D_CACHE_BF16) scale = scale_number(c.ks >> (16 * G::JF) & 255);
    kf[2 * G::JF] = decode_half<FMT>(c.rest, 0, scale);
    if (G::REST < 4 && !l.has_rest) kf[2 * G::JF] = zero8();
  }
}
// V of it into LDS at `at` (of the tile's blocks), rows whose bit in `vis` is not set as zeros
template <int H, int FMT>
__device__ __forceinline__ void decode_values(const Codes<H, FMT>& c, const Lane<H>& l, unsigned at, unsigned vis) {
  using G = Head<H>;
#pragma unroll
  for (int n = 0; n < G::NV; ++n) {
    float scale = 1.f;
    if constexpr (FMT != A2D_CACHE_BF16) scale = scale_number(c.vs >> (8 * (2 * n + (l.g >> 1))) & 255);
    bf16x8 x = decode_half<FMT>(c.v[n], 0, scale), y = decode_half<FMT>(c.v[n], 1, scale);
    if (A2D_SELDOM(vis != 0xFFFFu)) {
      const bool keep = vis >> l.row & 1;
      x = keep ? x : zero8();
      y = keep ? y : zero8();
    }
    if (l.live(n)) {
      lds_store(at + l.lds + 2 * n * BLOCK, x);
      lds_store(at + (l.lds ^ 16) + 2 * n * BLOCK, y);
    }
  }
}

// What a wavefront keeps of RT tiles of 16 rows; a lane: row lane & 15 of each, of which it has a quarter of the keys and of O's columns
template <int H, int RT>
struct State {
  f32x4 o[Head<H>::HT][RT];
  float m[RT];          // largest score the lane has seen, as it comes from the matrix unit
  float ref[RT];        // log2 units: what the exponentials are relative to, the same in the four lanes of a row
  float l[RT];
  bool far;             // some reference is ROUNDED or more, up or down
  __device__ __forceinline__ void clear() {
    far = false;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      m[t] = -INFINITY;
      ref[t] = LOW;
      l[t] = 0.f;
#pragma unroll
      for (int h = 0; h < Head<H>::HT; ++h) o[h][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
};

// Scores to probabilities: s becomes P
template <int H, int RT>
__device__ __forceinline__ void soften(State<H, RT>& st, f32x4 (&s)[2][RT], float c2) {
  float top[RT];
  bool far = false;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    float x = fmaxf(s[0][t][0], s[1][t][0]);
#pragma unroll
    for (int i = 1; i < 4; ++i) x = fmaxf(x, fmaxf(s[0][t][i], s[1][t][i]));
    top[t] = x;
    st.m[t] = fmaxf(st.m[t], x);
    far |= x * c2 > st.ref[t] + 8.f;
  }
  float by[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) by[t] = c2;
  if (A2D_SELDOM(__any(far || st.far))) {
    if (__any(far)) {                                // a reference is only moved by more than 2^8
      far = false;
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const float x = row_max(top[t]) * c2, ref = x > st.ref[t] + 8.f ? x : st.ref[t];    // (each row by its own scores alone)
        const float f = ref == st.ref[t] ? 1.f : fast_exp2(st.ref[t] - ref);
        far |= ref != LOW && fabsf(ref) >= ROUNDED;
        st.ref[t] = ref;
        st.l[t] *= f;
#pragma unroll
        for (int h = 0; h < Head<H>::HT; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) st.o[h][t][i] *= f;
      }
      st.far |= __any(far) != 0;
    }
    if (A2D_SELDOM(st.far)) {
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const bool rounded = fabsf(st.ref[t]) >= ROUNDED;
        by[t] = rounded ? 1.f : c2;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[k][t][i] = in_place(s[k][t][i] * (rounded ? c2 : 1.f));
      }
    }
  }
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[k][t][i] = fast_exp2(fmaf(s[k][t][i], by[t], -st.ref[t]));
        st.l[t] += s[k][t][i];
      }
}

template <int H, int RT>
__device__ __forceinline__ void products(State<H, RT>& st, const f32x4 (&s)[2][RT], const Blocks16& rd) {
  using G = Head<H>;
  bf16x8 hi[RT], lo[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float p = s[e >> 2][t][e & 3];
      hi[t][e] = (bf16_t)p;
      lo[t][e] = (bf16_t)(p - (float)hi[t][e]);
    }
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int h = 0; h < G::HT; ++h) {
    const unsigned at = (h & 1 ? rd.tr_o : rd.tr_e) + (h >> 1) * BLOCK;
    const bf16x8 v = lds_load_tr(at, at + G::KS * BLOCK);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      st.o[h][t] = mma16(v, hi[t], st.o[h][t]);
      st.o[h][t] = mma16(v, lo[t], st.o[h][t]);
    }
  }
}

// of the 16 keys of a tile
template <int H, int RT>
__device__ __forceinline__ void scores(f32x4 (&s)[RT], const bf16x8 (&kf)[Head<H>::KS], const bf16x8 (&qf)[Head<H>::KS][RT]) {
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < Head<H>::KS; ++x) s[t] = mma16(kf[x], qf[x][t], s[t]);
  }
}

// Is any of the 16 numbers a NaN or an infinity?  (Their products with 0, two at a time, are 0 or NaN.)
__device__ __forceinline__ bool not_finite(const Words<8>& w) {
  float x = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) x = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w.w[i]), bf16x2{(bf16_t)0.f, (bf16_t)0.f}, x, false);
  return !(x == 0.f);
}

// May a value of a cached V be infinite?  (of 8 and 4 bits, by its scale: 448 2^119 is not)
constexpr float LARGE_SCALE = 0x1p120f;
template <int FMT, int N>
__device__ __forceinline__ bool maybe_infinite(const Words<N>& w, float scale) {
  if constexpr (FMT == A2D_CACHE_BF16) return not_finite(w);
  else return scale >= LARGE_SCALE;
}

// with zeros in place of NaN and infinities
__device__ __forceinline__ bf16x8 finite_part(bf16x8 x) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (float)x[i] - (float)x[i] == 0.f ? x[i] : (bf16_t)0.f;
  return x;
}

// rows of a tile some lane of which is set
__device__ __forceinline__ unsigned rows_of(uint64_t lanes) {
  const unsigned x = (unsigned)lanes | (unsigned)(lanes >> 32);
  return (x | x >> 16) & 0xFFFF;
}

// of the 16 lanes 0 .. 15 (which 16 .. 31 and so on repeat)
__device__ __forceinline__ unsigned or16(unsigned x) {
  const auto with = [&](auto C) { x |= __builtin_bit_cast(unsigned, lane_swap<decltype(C)::value>(__builtin_bit_cast(float, x))); };
  with(std::integral_constant<int, 0xB1>{});         // lanes 1, 2 off, then those of the other half of 8, of 16
  with(std::integral_constant<int, 0x4E>{});
  with(std::integral_constant<int, 0x141>{});
  with(std::integral_constant<int, 0x140>{});
  return (unsigned)__builtin_amdgcn_readfirstlane((int)x);
}

// bits of 32 drafted rows from 32 * step on that row i of sequence b sees (own: the word of its mask with its own bit)
__device__ __forceinline__ unsigned seen_rows(const CachedArgs& a, int b, int i, int step, uint64_t own) {
  if (a.masks) {
    const uint64_t w = a.words == 1 ? own : a.masks[((int64_t)b * a.rows + i) * a.words + (step >> 1)];
    const unsigned x = (unsigned)(w >> (32 * (step & 1)));
    const int left = a.rows - STEP * step;            // (bits of no row)
    return left < 32 ? x & ((1u << left) - 1) : x;
  }
  const int n = i - STEP * step;
  return n < 0 ? 0 : n >= 31 ? ~0u : (2u << n) - 1;
}
template <int H, int FMT, int RT>
struct Walk {
  using G = Head<H>;
  const CachedArgs& a;
  const Lane<H>& ln;
  const Blocks16& rd;
  unsigned area;                                     // LDS: the wavefront's V
  int lane, wave;
  State<H, RT> st;
  bf16x8 qf[G::KS][RT];
  int row_of[RT];                                    // the lane's row of a tile within its sequence; -1: there is none
  uint64_t own[RT];                                  // the word of its mask with its own bit
  unsigned units;
  uint64_t some, good;                               // bits of the lanes whose tile is there; is there, all of it

  // steps s0 .. s1 - 1 of block `block` of head h of sequence b, which has `tokens` cached ones
  __device__ __forceinline__ void run(int b, int h, int block, int s0, int s1, int tokens) {
    const int rows = a.group * a.rows, drafts = draft_steps(a);
    int s = s0 + wave;                               // the wavefront's steps: s, s + WAVES, ..
    const int first = s < drafts ? s + (drafts - s + WAVES - 1) / WAVES * WAVES : s;       // the first one of cached tokens
    // requests go out before any is waited for: pages, drafted rows, masks, Q
    Place place;
    look_up(place, b, first - drafts, tokens, first < s1);
    Codes<H, A2D_CACHE_BF16> drafted;
    if (s < min(s1, drafts)) {
      Lane<H> ln;
      ln.init(lane_again());
      load_drafts<H>(drafted, a, b, h, STEP * s, ln);
    }
    {
      Lane<H> ln;
      ln.init(lane_again());
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const int at = (block * RT + t) * 16 + ln.row, r = min(at, rows - 1);
        const int head = a.rows == 1 ? r : r / a.rows, i = r - head * a.rows;
        row_of[t] = at < rows ? i : -1;
        own[t] = a.masks ? a.masks[((int64_t)b * a.rows + i) * a.words + (i >> 6)] : ~(uint64_t)0;
        const bf16_t* q = reinterpret_cast<const bf16_t*>(a.Q) + at_row(a.lq, b, h * a.group + head, i);
#pragma unroll
        for (int x = 0; x < 2 * G::JF; ++x) qf[x][t] = *reinterpret_cast<const bf16x8*>(q + 64 * (x >> 1) + 16 * ln.g + 8 * (x & 1));
        if constexpr (G::REST) {
          qf[2 * G::JF][t] = *reinterpret_cast<const bf16x8*>(q + (ln.has_rest ? 64 * G::JF + 8 * ln.g : 0));
          if (G::REST < 4 && !ln.has_rest) qf[2 * G::JF][t] = zero8();
        }
      }
    }
    st.clear();
    take(place, h, first - drafts, tokens);
    // (of one row tile the first codes are asked for before the drafted rows are worked on; two leave no registers for that)
    constexpr bool EARLY = RT == 1;
    const int from = first - drafts, last = min(s1 - drafts, (tokens + STEP - 1) / STEP);
    Codes<H, FMT> c[2];
    unsigned vis = 0;
    if (EARLY && from < last) vis = load(c, 0, from, tokens);
    for (bool again = false; s < min(s1, drafts); s += WAVES, again = true) draft_step(b, h, s, drafted, again);
    if (from < last) {
      if (!EARLY) vis = load(c, 0, from, tokens);
      cache_steps(c, vis, b, h, from, last, tokens);
    }
  }
  // does the lane's row of tile t exist, and is it a token (its own bit is set)?
  __device__ __forceinline__ bool live(int t) const { return row_of[t] >= 0 && (own[t] >> (row_of[t] & 63) & 1); }

  // the units of tile lane & 1 of the wavefront's step lane >> 1 of 32 from s on
  __device__ __forceinline__ void look_up(Place& p, int b, int s, int tokens, bool wanted = true) const {
    const int tile = 2 * (s + WAVES * (lane >> 1)) + (lane & 1);
    p.ask(a.c, b, tile, wanted && tile < (tokens + 15) / 16);
  }

  __device__ __forceinline__ void take(const Place& p, int h, int s, int tokens) {
    units = p.unit(a.c, h);
    some = __ballot(units != NO_UNIT);
    good = some & __ballot(16 * (2 * (s + WAVES * (lane >> 1)) + (lane & 1)) + 16 <= tokens);
    if (units == NO_UNIT) units = 0;                 // (some tile, whose keys are not seen)
  }
  // keys of step s, the wavefront's n-th, that are there
  __device__ __forceinline__ unsigned there(int n, int s, int tokens) const {
    const int at = 2 * (n & 31);
    if (A2D_OFTEN(((unsigned)(good >> at) & 3) == 3)) return ~0u;
    unsigned vis = 0;
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (some >> (at + k) & 1) vis |= ((1u << min(max(tokens - STEP * s - 16 * k, 0), 16)) - 1) << (16 * k);
    return vis;
  }

  // asks for the codes of the wavefront's n-th step, s; returns the keys of it that are there
  __device__ __forceinline__ unsigned load(Codes<H, FMT> (&c)[2], int n, int s, int tokens) const {
#pragma unroll
    for (int k = 0; k < 2; ++k) load_unit<H, FMT>(c[k], a.c, __builtin_amdgcn_readlane((int)units, 2 * (n & 31) + k), ln);
    return there(n, s, tokens);
  }
  __device__ __forceinline__ void cache_steps(Codes<H, FMT> (&c)[2], unsigned vis, int b, int h, int first, int last, int tokens) {
    Place place;                                     // (asked for a step before it is taken)
    for (int s = first, n = 0; s < last; s += WAVES, ++n) {
      f32x4 sc[2][RT];
      const unsigned now = vis;
      uint64_t large[2];                             // lanes that have a value of V that may be infinite
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        bf16x8 kf[G::KS];
        bool some_large = false;
#pragma unroll
        for (int x = 0; x < G::NV; ++x) some_large |= maybe_infinite<FMT>(c[k].v[x], scale_number(c[k].vs >> (8 * (2 * x + (ln.g >> 1))) & 255));
        large[k] = __ballot(some_large);
        decode_values<H, FMT>(c[k], ln, area + k * G::KS * BLOCK, k ? now >> 16 : now & 0xFFFF);
        decode_keys<H, FMT>(kf, c[k], ln);
        scores<H, RT>(sc[k], kf, qf);
      }
      __builtin_amdgcn_sched_barrier(0);
      // the next step's codes, while this one is worked on (behind the last: the last again)
      const bool more = s + WAVES < last;
      if (A2D_SELDOM((n & 31) == 30)) look_up(place, b, s + 2 * WAVES, tokens);
      if (A2D_SELDOM((n & 31) == 31)) take(place, h, s + WAVES, tokens);
      vis = load(c, more ? n + 1 : n, more ? s + WAVES : s, tokens);
      if (A2D_SELDOM(now != ~0u)) {
        const unsigned mine = now >> (4 * ln.g);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[k][t][i] = mine >> (16 * k + i) & 1 ? sc[k][t][i] : -INFINITY;
      }
      soften<H, RT>(st, sc, a.c2);
      if (A2D_SELDOM((large[0] | large[1]) != 0)) {  // (P's second number, 0 or below, would make NaN of infinities)
        unsigned all[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) all[t] = ~0u;
        apart(sc, all, rows_of(large[0]) | rows_of(large[1]) << 16);
      }
      products<H, RT>(st, sc, rd);
    }
  }

  // (the lane's places are computed anew: kept beside the walk over the cache, they would take its registers)
  // (c: the codes of its first tile, asked for already where it is not a further step)
  __device__ __forceinline__ void draft_step(int b, int h, int step, Codes<H, A2D_CACHE_BF16>& c, bool further) {
    Lane<H> ln;
    ln.init(lane_again());
    unsigned seen[RT], all = 0;
    if (further) load_drafts<H>(c, a, b, h, STEP * step, ln);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      seen[t] = live(t) ? seen_rows(a, b, row_of[t], step, own[t]) : 0;
      all |= seen[t];
    }
    all = or16(all);
    if (all == 0) return;
    f32x4 sc[2][RT];
    unsigned bad = 0;                                // drafted rows of the step whose V is not finite
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (k == 1 && all >> 16 == 0) {                // (no second tile: zeros, since P = 0 meets them)
#pragma unroll
        for (int n = 0; n < G::NV; ++n)
          if (ln.live(n)) {
            lds_store(area + (G::KS + 2 * n) * BLOCK + ln.lds, zero8());
            lds_store(area + (G::KS + 2 * n) * BLOCK + (ln.lds ^ 16), zero8());
          }
#pragma unroll
        for (int t = 0; t < RT; ++t) sc[1][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        break;
      }
      if (k) load_drafts<H>(c, a, b, h, STEP * step + 16, ln);
#pragma unroll
      for (int n = 0; n < G::NV; ++n)
        if ((all >> (16 * k + ln.row) & 1) && not_finite(c.v[n])) bad |= 1u << (16 * k + ln.row);
      // (rows that none of the block's rows see are zeros: they may hold anything)
      decode_values<H, A2D_CACHE_BF16>(c, ln, area + k * G::KS * BLOCK, all >> (16 * k) & 0xFFFF);
      bf16x8 kf[G::KS];
      decode_keys<H, A2D_CACHE_BF16>(kf, c, ln);
      scores<H, RT>(sc[k], kf, qf);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[k][t][i] = seen[t] >> (16 * k + 4 * ln.g + i) & 1 ? sc[k][t][i] : -INFINITY;
    soften<H, RT>(st, sc, a.c2);
    if (A2D_SELDOM(__any(bad != 0))) {
#pragma unroll
      for (int d = 1; d < 64; d *= 2) bad |= (unsigned)__shfl_xor((int)bad, d);
      apart(sc, seen, __builtin_amdgcn_readfirstlane((int)bad));
    }
    products<H, RT>(st, sc, rd);
  }

  // A NaN or an infinity in a drafted row's V may be added to those rows only that see it, and its product with P = 0, or with P's second
  // number, is not 0: such numbers, also those of a cached V, are added one at a time and become zeros in LDS.  bad: keys of the step that may have any.
  __device__ __forceinline__ void apart(const f32x4 (&sc)[2][RT], const unsigned (&seen)[RT], unsigned bad) {
    const int lane = lane_again();
    while (bad) {
      const int key = __builtin_ctz(bad), k = key >> 4, r = key & 15;
      bad &= bad - 1;
      const unsigned row = area + k * G::KS * BLOCK + r * 64;
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        float p = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) p = 4 * (e >> 2) + (e & 3) == 4 * k + (r & 3) ? sc[e >> 2][t][e & 3] : p;
        p = __shfl(p, 16 * (r >> 2) + (lane & 15));
        if (!(seen[t] >> key & 1)) continue;
#pragma unroll
        for (int h = 0; h < G::HT; ++h) {
          const bf16x4 v4 = lds_quad(quad_at(row, r, h, lane >> 4));
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float v = (float)v4[i];
            st.o[h][t][i] = in_place(v - v == 0.f ? st.o[h][t][i] : fmaf(p, v, st.o[h][t][i]));
          }
        }
      }
      const unsigned at = row + (lane >> 2) * BLOCK + 16 * ((lane & 3) ^ block_swap(r >> 2));
      if (lane < H / 8) lds_store(at, finite_part(lds_load_b128(at)));
    }
  }
};

template <int H, int FMT, int RT>
__global__ __launch_bounds__(64 * WAVES, 2) void cached_kernel(CachedArgs a) {
  using G = Head<H>;
  constexpr int ROWS = 16 * RT, QUADS = H / 4;
  __shared__ __align__(1024) char area[WAVES][G::AREA];
  __shared__ f32x4 stat[WAVES][ROWS];                // m (log2 units), ref, l of a wavefront's row; whether it is a token's
  __shared__ f32x2 joined[ROWS];                     // m, l of all four
  warm_cached();
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Lane<H> ln;
  ln.init(lane);
  Blocks16 rd;
  const unsigned mine = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)area[wave];
  rd.init(lane, mine);
  Walk<H, FMT, RT> w{a, ln, rd, mine, lane, wave};

  Runs runs;
  if (!runs.begin(a, lane)) return;
  Run run;
  while (runs.next(a, lane, run)) {
    const int block = run.block;
    w.run(run.b, run.h, block, run.s0, run.s1, run.tokens);

    // the four wavefronts' results become one, 16 rows at a time
    const int lane = lane_again(), thread = 64 * wave + lane;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const float l = row_reduce(w.st.l[t], [](float x, float y) { return x + y; });
      const float m = row_max(w.st.m[t]) * a.c2;
      if (lane < 16) stat[wave][16 * t + lane] = f32x4{m, w.st.ref[t], w.live(t) ? l : 0.f, w.live(t) ? 1.f : 0.f};
    }
    __syncthreads();
    const bool whole = run.s0 == 0 && run.s1 == run.steps;
    float* part = whole ? nullptr : a.parts + (size_t)(2 * runs.worker + (run.s0 == 0)) * part_floats(ROWS, H);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      {
        const int r = 16 * t + (lane & 15);
        f32x4 of[WAVES];
        float top = -INFINITY, l = 0.f;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) {
          of[v] = stat[v][r];
          top = fmaxf(top, of[v][0]);
        }
        const bool any = top != -INFINITY;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) l += of[v][2] * (any ? fast_exp2(of[v][1] - top) : 0.f);      // (any or not: NaN stays NaN)
        if (wave == 0 && lane < 16) {
          const bool empty = of[0][3] == 0.f || l == 0.f;
          joined[r] = f32x2{empty ? -INFINITY : top, empty ? 0.f : l};
        }
        const float f = any ? fast_exp2(w.st.ref[t] - top) : 0.f;
#pragma unroll
        for (int x = 0; x < G::HT; ++x) {
          f32x4 o = w.st.o[x][t];
#pragma unroll
          for (int i = 0; i < 4; ++i) o[i] *= f;
          *reinterpret_cast<f32x4*>(area[wave] + 4 * H * (lane & 15) + 16 * ((4 * x + (lane >> 4)) ^ (lane & 3))) = o;
        }
      }
      __syncthreads();
      for (int at = thread; at < 16 * QUADS; at += 64 * WAVES) {
        const int row = at / QUADS, quad = at - row * QUADS, r = 16 * t + row;
        const int index = (block * RT + t) * 16 + row;
        if (index >= a.group * a.rows) continue;
        const f32x2 of = joined[r];
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < WAVES; ++v) {
          const f32x4 x = *reinterpret_cast<const f32x4*>(area[v] + 4 * H * row + 16 * (quad ^ (row & 3)));
#pragma unroll
          for (int i = 0; i < 4; ++i) o[i] += x[i];
        }
        if (of[1] == 0.f) o = f32x4{0.f, 0.f, 0.f, 0.f};
        if (whole) {
          const Split sp = split_by(index, a.rows);
          finish(a, run.b, run.h * a.group + (a.rows == 1 ? index : sp.q), a.rows == 1 ? 0 : sp.r, H, quad, o, of[0], of[1]);
        } else {
          *reinterpret_cast<f32x4*>(part + 2 * ROWS + (size_t)r * H + 4 * quad) = o;
          if (quad == 0) {
            part[r] = of[0];
            part[ROWS + r] = of[1];
          }
        }
      }
      __syncthreads();
    }
  }
}

template <int H, int FMT>
hipError_t go_tiles(Phase ph, const CachedArgs& a, hipStream_t s) {
  if (ph == PREPARE) return hipSuccess;              // (no dynamic LDS)
  const dim3 grid(cached_grid(a));
  if (a.tiles == 1) A2D_LAUNCH((cached_kernel<H, FMT, 1>), grid, dim3(64 * WAVES), 0, s, a);
  else A2D_LAUNCH((cached_kernel<H, FMT, 2>), grid, dim3(64 * WAVES), 0, s, a);
  return hipGetLastError();
}
template <int FMT>
hipError_t go_format(Phase ph, int hdim, const CachedArgs& a, hipStream_t s) {
  return hdim == 64 ? go_tiles<64, FMT>(ph, a, s) : hdim == 80 ? go_tiles<80, FMT>(ph, a, s) : hdim == 96 ? go_tiles<96, FMT>(ph, a, s)
                                                                                              : go_tiles<128, FMT>(ph, a, s);
}

}  // namespace cached
}  // namespace a2d
