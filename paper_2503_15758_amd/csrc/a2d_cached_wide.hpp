// Attention of many rows - large trees, several heads of a group - against the paged cache: the form of a2d_cached_fwd.hpp for more rows than
// a wavefront can hold (the formulas and the line of walks are the same).
//
// A workgroup has 32 rows for each of its wavefronts, which share the keys: 64 a step, decoded once into LDS as bf16 by all wavefronts together
// (a piece of 16 values a lane), two buffers, one barrier a step.  A step's codes are asked for a step before they are decoded and are decoded a step
// before they are used.  The contractions are those of the bf16 forward (a2d_fwd.hpp).  Bound: power, and the vector ALU beside
// the matrix units.  64 rows of 8 sequences, 32 / 8 heads of 128, 9001 to 16384 tokens in e4m3: calls that follow one another 141 us, 860 TFLOP/s with the
// merge of the parts; this kernel by itself under the profiler 158 us, 765 TFLOP/s, at 1.93 GHz, MFMA busy 38 %, vector ALU 46 % of the cycles.
#pragma once
#include "a2d_cached_fwd.hpp"
#include "a2d_fwd.hpp"

namespace a2d {
namespace cached {

template <int H, int FMT, int W, bool FINE>
struct WideWalk {
  using G = Head<H>;
  static constexpr int HD = padded_head(H), KS = HD / 32, HT = H / 16;
  static constexpr int BUF = buf_bytes(HD), K_BYTES = BUF / 2;
  static constexpr int LOADS = 8 * G::NV, PER = (LOADS + W - 1) / W;       // of K and V of a step: of a wavefront
  static constexpr int WORDS = code_bytes<FMT>(16) / 4;
  static_assert(LOADS % W == 0 && W % G::NV == 0, "a wavefront's loads are of one half of their tiles");
  const CachedArgs& a;
  const Blocks16& rd;
  unsigned area;                                     // LDS: two buffers
  unsigned* bad;                                     // LDS: drafted rows of a step whose V is not finite (64 bits); of each buffer, LARGE where a
                                                     // cached V in it may be infinite (FINE; never cleared beforehand, which would take a barrier:
                                                     // the same number found there by chance changes no result)
  static constexpr unsigned LARGE = 0x1A26E1A2;
  int lane, wave;
  // the lane's place in the tiles that its wavefront loads
  int prow, ppiece;            // (pieces that there are none of: the row's first)
  bool plive;
  unsigned plds;
  // rows
  f32x4 o[HT][2];
  float m[2], ref[2], l[2];
  bool far;                                          // some reference is ROUNDED or more, up or down
  bf16x8 qf[KS][2];
  unsigned units;                                    // of tile lane & 3 of step lane >> 2 of 16
  uint64_t some, good;                               // bits of the lanes whose tile is there; is there, all of it
  Words<WORDS> code[PER];
  unsigned scale[PER];

  __device__ __forceinline__ void init() {
    const int n = wave % G::NV;
    Lane<H> ln;
    ln.init(lane);
    plive = ln.live(n);
    prow = ln.row;
    ppiece = ln.piece(n);
    plds = ln.lds + 2 * n * BLOCK;
    if constexpr (H % 32 != 0) {                     // K's columns behind the last: they meet zeros of Q, and must be numbers
      static_assert(H % 32 == 16, "two chunks of a row");
      for (int x = 64 * wave + lane; x < 2 * 4 * 16 * 2; x += 64 * W) {
        const int c = 2 + (x & 1), row = x >> 1 & 15, tile = x >> 5 & 3, buf = x >> 7;
        lds_store(area + buf * BUF + (tile * KS + KS - 1) * BLOCK + row * 64 + 16 * (c ^ block_swap(row >> 2)), zero8());
      }
    }
  }
  // the wavefront's n-th load of a step: K or V, of which tile
  __device__ __forceinline__ int tile_of(int n) const { return (wave + W * n) / G::NV & 3; }
  // (known beforehand where the wavefronts' loads of K end together, but for one form whose registers spill then; a partial of 25 rows in
  // e4m3 takes 31.9 us so, 33.0 otherwise)
  static constexpr bool APART = LOADS / 2 % W == 0 && !(FINE && FMT == A2D_CACHE_BF16 && H == 128 && W == 4);
  __device__ __forceinline__ bool is_value(int n) const { return (APART ? 0 : wave) + W * n >= LOADS / 2; }

  __device__ __forceinline__ void look_up(Place& p, int b, int s, int tokens, bool wanted = true) const {
    const int tile = 4 * s + lane;
    p.ask(a.c, b, tile, wanted && tile < (tokens + 15) / 16);
  }
  __device__ __forceinline__ void take(const Place& p, int h, int s, int tokens) {
    units = p.unit(a.c, h);
    some = __ballot(units != NO_UNIT);
    good = some & __ballot(16 * (4 * s + lane) + 16 <= tokens);
    if (units == NO_UNIT) units = 0;                 // (some tile, whose keys are not seen)
  }
  // keys of step s, the n-th of the walk, that are there
  __device__ __forceinline__ uint64_t there(int n, int s, int tokens) const {
    const int at = 4 * (n & 15);
    if (A2D_OFTEN(((unsigned)(good >> at) & 15) == 15)) return ~(uint64_t)0;
    uint64_t vis = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (some >> (at + t) & 1) vis |= (uint64_t)((1u << min(max(tokens - 64 * s - 16 * t, 0), 16)) - 1) << (16 * t);
    return vis;
  }
  // asks for the codes of the walk's n-th step
  __device__ __forceinline__ void load(int n) {
    constexpr int ROW = code_bytes<FMT>(H);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int t = tile_of(i);
      const unsigned unit = __builtin_amdgcn_readlane((int)units, 4 * (n & 15) + t);
      const gptr_t p = uniform_gptr((is_value(i) ? a.c.V : a.c.K) + (uint64_t)unit * (16 * ROW));
      code[i] = load_words<WORDS>(p, prow * ROW + ppiece * code_bytes<FMT>(16));
      if constexpr (FMT != A2D_CACHE_BF16)
        scale[i] = load_words<1>(uniform_gptr((is_value(i) ? a.c.Vs : a.c.Ks) + (uint64_t)unit * 64), prow * 4).w[0];
    }
  }
  // the codes that have come become bf16 in a buffer; V of keys that are not there: zeros
  __device__ __forceinline__ void decode(int buf, uint64_t vis) {
    bool large = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      float f = 1.f;
      if constexpr (FMT != A2D_CACHE_BF16) f = scale_number(scale[i] >> (8 * (ppiece >> 1)) & 255);
      bf16x8 x = decode_half<FMT>(code[i], 0, f), y = decode_half<FMT>(code[i], 1, f);
      if constexpr (FINE)
        if (is_value(i)) large |= maybe_infinite<FMT>(code[i], f);
      const int t = tile_of(i);
      if (A2D_SELDOM(vis != ~(uint64_t)0)) {
        const bool keep = !is_value(i) || (vis >> (16 * t + prow) & 1);
        x = keep ? x : zero8();
        y = keep ? y : zero8();
      }
      const unsigned at = area + buf * BUF + (is_value(i) ? K_BYTES : 0) + t * KS * BLOCK + plds;
      if (4 * G::NV == G::PIECES || plive) {
        lds_store(at, x);
        lds_store(at ^ 16, y);
      }
    }
    if (FINE && A2D_SELDOM(__any(large)) && lane == 0) bad[2 + buf] = LARGE;
  }
  // a buffer's V with zeros in place of infinities (which P's second number, 0 or below, would make NaN of), the flag taken back; for all
  // wavefronts between the products of P's first number and those of its second
  __device__ __forceinline__ void finite_values(int buf) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const unsigned at = area + buf * BUF + K_BYTES + tile_of(i) * KS * BLOCK + plds;
      if (is_value(i) && (4 * G::NV == G::PIECES || plive)) {
        lds_store(at, finite_part(lds_load_b128(at)));
        lds_store(at ^ 16, finite_part(lds_load_b128(at ^ 16)));
      }
    }
    if (wave == 0 && lane == 0) bad[2 + buf] = 0;
    __syncthreads();
  }

  __device__ __forceinline__ void soften(Scores& s) {
    float top[2];
    bool far = false;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      float x = s[0][q][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) x = fmaxf(x, s[e >> 2][q][e & 3]);
      top[q] = x;
      m[q] = fmaxf(m[q], x);
      far |= x * a.c2 > ref[q] + 8.f;
    }
    float by[2] = {a.c2, a.c2};
    if (A2D_SELDOM(__any(far || this->far))) {
      if (__any(far)) {
        far = false;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const float x = row_max(top[q]) * a.c2, to = x > ref[q] + 8.f ? x : ref[q];       // (each row by its own scores alone)
          const float f = to == ref[q] ? 1.f : fast_exp2(ref[q] - to);
          ref[q] = to;
          far |= to != LOW && fabsf(to) >= ROUNDED;
          l[q] *= f;
#pragma unroll
          for (int h = 0; h < HT; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[h][q][i] *= f;
        }
        this->far |= __any(far) != 0;
      }
      if (A2D_SELDOM(this->far)) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const bool rounded = fabsf(ref[q]) >= ROUNDED;
          by[q] = rounded ? 1.f : a.c2;
#pragma unroll
          for (int e = 0; e < 16; ++e) s[e >> 2][q][e & 3] = in_place(s[e >> 2][q][e & 3] * (rounded ? a.c2 : 1.f));
        }
      }
    }
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[e >> 2][q][e & 3] = fast_exp2(fmaf(s[e >> 2][q][e & 3], by[q], -ref[q]));
        l[q] += s[e >> 2][q][e & 3];
      }
  }
  // P as one bf16 number, or two
  struct Weights {
    bf16x8 p[2][2], rest[FINE ? 2 : 1][2];
    __device__ __forceinline__ void set(const Scores& s) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float x = s[2 * k + (e >> 2)][q][e & 3];
            p[k][q][e] = (bf16_t)x;
            if constexpr (FINE) rest[k][q][e] = (bf16_t)(x - (float)p[k][q][e]);
          }
    }
  };
  __device__ __forceinline__ void rest_products(const Weights& w, Ring& vr, unsigned at) {
    if constexpr (FINE) {
      fwd_first_values<H>(vr, rd, at);
      fwd_products<H>(o, w.rest, vr, rd, at);
    }
  }

  __device__ __forceinline__ void run(int b, int h, int block, int s0, int s1, int tokens) {
    const int drafts = draft_steps(a), first = max(s0 - drafts, 0), last = min(s1 - drafts, (tokens + 63) / 64);
    const bool any_row = (block * W + wave) * 32 < a.group * a.rows;      // of the wavefront's
    Place place;
    look_up(place, b, first, tokens, first < last);
    const int ln = lane_again();
    far = false;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const Row r = row(b, h, block, q);
      const bf16_t* p = reinterpret_cast<const bf16_t*>(a.Q) + at_row(a.lq, b, r.head, r.i);
#pragma unroll
      for (int x = 0; x < KS; ++x) {
        const int c = 32 * x + 8 * (ln >> 4);
        qf[x][q] = *reinterpret_cast<const bf16x8*>(p + min(c, H - 8));
        if (32 * x + 32 > H && c >= H) qf[x][q] = zero8();
      }
      m[q] = -INFINITY;
      ref[q] = LOW;
      l[q] = 0.f;
#pragma unroll
      for (int x = 0; x < HT; ++x) o[x][q] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    take(place, h, first, tokens);
    for (int s = s0; s < min(s1, drafts); ++s) draft_step(b, h, block, s);
    if (first < last) {
      uint64_t now = there(0, first, tokens), next = 0;
      load(0);
      decode(0, now);
      if (first + 1 < last) {
        next = there(1, first + 1, tokens);
        load(1);
      }
      __syncthreads();
      for (int s = first, n = 0; s < last; ++s, ++n) {
        uint64_t after = 0;
        if (s + 1 < last) {
          decode((n + 1) & 1, next);
          if (A2D_SELDOM((n & 15) == 14)) {
            Place p;
            look_up(p, b, s + 2, tokens);
            take(p, h, s + 2, tokens);
          }
          if (s + 2 < last) after = there(n + 2, s + 2, tokens);
          load(n + 2);                               // (behind the last step: nothing that is used)
        }
        const unsigned at = (n & 1) * BUF;
        const unsigned large = FINE ? bad[2 + (n & 1)] : 0;      // (asked for here, looked at behind the products)
        Weights w;
        Ring ring;
        if (any_row) {
          Scores sc;
          fwd_first_keys<H>(ring, rd, at);
          fwd_scores<H>(sc, ring, qf, rd, at);
          if (A2D_SELDOM(now != ~(uint64_t)0)) {
            const uint64_t mine = now >> (4 * (lane >> 4));
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
              for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int i = 0; i < 4; ++i) sc[k][q][i] = mine >> (16 * k + i) & 1 ? sc[k][q][i] : -INFINITY;
          }
          fwd_first_values<H>(ring, rd, at);
          soften(sc);
          w.set(sc);
          fwd_products<H>(o, w.p, ring, rd, at);
        }
        if constexpr (FINE) {
          if (A2D_SELDOM(__builtin_amdgcn_readfirstlane((int)large) == LARGE)) finite_values(n & 1);
          if (any_row) rest_products(w, ring, at);
        }
        __syncthreads();
        now = next;
        next = after;
      }
    }
  }
  // the lane's row of tile q (the block's last one in place of those behind it); made again where it is needed, not kept on the walk
  struct Row {
    int head, i;
    bool there, token;                               // token: and its own bit is set
    uint64_t own;                                    // the word with it
  };
  __device__ __forceinline__ Row row(int b, int h, int block, int q) const {
    const int at = ((block * W + wave) * 2 + q) * 16 + (lane_again() & 15), rows = a.group * a.rows, r = min(at, rows - 1);
    Row x;
    x.head = r / a.rows;
    x.i = r - x.head * a.rows;
    x.head += h * a.group;
    x.there = at < rows;
    x.own = a.masks ? a.masks[((int64_t)b * a.rows + x.i) * a.words + (x.i >> 6)] : ~(uint64_t)0;
    x.token = x.there && (x.own >> (x.i & 63) & 1);
    return x;
  }

  // 64 drafted rows, in the first buffer
  __device__ __forceinline__ void draft_step(int b, int h, int block, int step) {
    if (!a.masks) {
      // (a chain's rows see none behind themselves: the last row of a block that has rows of one head alone)
      const int from = block * W * 32, to = min(from + W * 32, a.group * a.rows) - 1;
      if (from / a.rows == to / a.rows && 64 * step > to % a.rows) return;
    }
    if (wave == 0 && lane < 2) bad[lane] = 0;
    __syncthreads();
    const gptr_t base[2] = {uniform_gptr(a.K + 2 * at_row(a.lk, b, h, 0)), uniform_gptr(a.V + 2 * at_row(a.lv, b, h, 0))};
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int t = tile_of(i), key = 16 * t + prow, r = min(64 * step + key, a.rows - 1);
      const bool value = is_value(i);
      const Words<8> w = load_words<8>(value ? base[1] : base[0], (unsigned)r * (unsigned)(2 * (value ? a.lv.row : a.lk.row)) + ppiece * 32);
      const bf16x8 x = decode_half<A2D_CACHE_BF16>(w, 0, 1.f), y = decode_half<A2D_CACHE_BF16>(w, 1, 1.f);
      if (4 * G::NV == G::PIECES || plive) {
        const unsigned at = area + (value ? K_BYTES : 0) + t * KS * BLOCK + plds;
        lds_store(at, x);
        lds_store(at ^ 16, y);
        if (value && not_finite(w)) atomicOr(&bad[key >> 5], 1u << (key & 31));
      }
    }
    __syncthreads();
    const unsigned odd0 = (unsigned)__builtin_amdgcn_readfirstlane((int)bad[0]), odd1 = (unsigned)__builtin_amdgcn_readfirstlane((int)bad[1]);
    const uint64_t odd = (uint64_t)odd1 << 32 | odd0;
    Scores sc;
    Ring ring;
    fwd_first_keys<H>(ring, rd, 0);
    fwd_scores<H>(sc, ring, qf, rd, 0);
    uint64_t seen[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      seen[q] = 0;
      const Row r = row(b, h, block, q);
      if (r.token)
        seen[q] = seen_rows(a, b, r.i, 2 * step, r.own) | (uint64_t)(64 * step + 32 < a.rows ? seen_rows(a, b, r.i, 2 * step + 1, r.own) : 0) << 32;
      const uint64_t mine = seen[q] >> (4 * (lane >> 4));
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[k][q][i] = mine >> (16 * k + i) & 1 ? sc[k][q][i] : -INFINITY;
    }
    soften(sc);
    if (A2D_SELDOM(odd != 0)) apart(sc, seen, odd);
    fwd_first_values<H>(ring, rd, 0);
    Weights w;
    w.set(sc);
    fwd_products<H>(o, w.p, ring, rd, 0);
    rest_products(w, ring, 0);
    __syncthreads();
  }

  // as in the form of few rows: numbers of V that are not finite go to the rows that see them, one at a time, and become zeros
  __device__ __forceinline__ void apart(const Scores& sc, const uint64_t (&seen)[2], uint64_t odd) {
    const int ln = lane_again();
    for (uint64_t left = odd; left; left &= left - 1) {
      const int key = __builtin_ctzll(left), r = key & 15;
      const unsigned row = area + K_BYTES + (key >> 4) * KS * BLOCK + r * 64;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        float p = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) p = 4 * (e >> 2) + (e & 3) == 4 * (key >> 4) + (r & 3) ? sc[e >> 2][q][e & 3] : p;
        p = __shfl(p, 16 * (r >> 2) + (ln & 15));
        if (!(seen[q] >> key & 1)) continue;
#pragma unroll
        for (int x = 0; x < HT; ++x) {
          const bf16x4 v4 = lds_quad(quad_at(row, r, x, ln >> 4));
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float v = (float)v4[i];
            o[x][q][i] = v - v == 0.f ? o[x][q][i] : fmaf(p, v, o[x][q][i]);
          }
        }
      }
    }
    __syncthreads();
    for (uint64_t left = odd; left; left &= left - 1) {
      const int key = __builtin_ctzll(left), r = key & 15;
      const unsigned row = area + K_BYTES + (key >> 4) * KS * BLOCK + r * 64;
      const unsigned at = row + (ln >> 2) * BLOCK + 16 * ((ln & 3) ^ block_swap(r >> 2));
      if (wave == 0 && ln < H / 8) lds_store(at, finite_part(lds_load_b128(at)));
    }
    __syncthreads();
  }
};

template <int H>
__host__ __device__ constexpr int wide_lds() { return 2 * buf_bytes(padded_head(H)) + 16; }

template <int H, int FMT, int W, bool FINE>
__global__ __launch_bounds__(64 * W, 2) void cached_wide_kernel(CachedArgs a) {
  extern __shared__ __align__(1024) char lds[];
  constexpr int ROWS = 32 * W;
  warm_cached();
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned area = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  Blocks16 rd;
  rd.init(lane, area);
  WideWalk<H, FMT, W, FINE> w{a, rd, area, reinterpret_cast<unsigned*>(lds + 2 * buf_bytes(padded_head(H))), lane, wave};
  w.init();
  Runs runs;
  if (!runs.begin(a, lane)) return;
  Run run;
  while (runs.next(a, lane, run)) {
    w.run(run.b, run.h, run.block, run.s0, run.s1, run.tokens);
    const bool whole = run.s0 == 0 && run.s1 == run.steps;
    float* const part = whole ? nullptr : a.parts + (size_t)(2 * runs.worker + (run.s0 == 0)) * part_floats(ROWS, H);
    const int ln = lane_again();
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      float l = row_sum(w.l[q]), top = row_max(w.m[q]) * a.c2;
      float f = top == -INFINITY ? 0.f : part_factor(w.ref[q], top);
      l *= f;
      const auto row = w.row(run.b, run.h, run.block, q);
      const bool empty = !row.token || l == 0.f;
      if (empty) {
        top = -INFINITY;
        l = 0.f;
      }
      if (!row.there) continue;
      const int r = 32 * wave + 16 * q + (ln & 15);
#pragma unroll
      for (int x = 0; x < H / 16; ++x) {
        f32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = empty ? 0.f : w.o[x][q][i] * f;
        const int quad = 4 * x + (ln >> 4);
        if (whole) {
          finish(a, run.b, row.head, row.i, H, quad, v, top, l);
        } else {
          *reinterpret_cast<f32x4*>(part + 2 * ROWS + (size_t)r * H + 4 * quad) = v;
          if (quad == 0) {
            part[r] = top;
            part[ROWS + r] = l;
          }
        }
      }
    }
  }
}

template <int H, int FMT, int W, bool FINE>
hipError_t go_wide(Phase ph, const CachedArgs& a, hipStream_t s) {
  const auto kernel = &cached_wide_kernel<H, FMT, W, FINE>;
  if (ph == PREPARE) return ensure_dynamic_lds(reinterpret_cast<const void*>(kernel), wide_lds<H>());
  A2D_LAUNCH((cached_wide_kernel<H, FMT, W, FINE>), dim3(cached_grid(a)), dim3(64 * W), wide_lds<H>(), s, a);
  return hipGetLastError();
}
template <int H, int FMT>
hipError_t go_wide_form(Phase ph, const CachedArgs& a, hipStream_t s) {
  // (fp32 partials take P as two bf16 numbers)
  if (a.tiles == 16) return a.norm ? go_wide<H, FMT, 8, false>(ph, a, s) : go_wide<H, FMT, 8, true>(ph, a, s);
  return a.norm ? go_wide<H, FMT, 4, false>(ph, a, s) : go_wide<H, FMT, 4, true>(ph, a, s);
}
template <int FMT>
hipError_t go_wide_head(Phase ph, int hdim, const CachedArgs& a, hipStream_t s) {
  return hdim == 64 ? go_wide_form<64, FMT>(ph, a, s) : hdim == 80 ? go_wide_form<80, FMT>(ph, a, s) : hdim == 96 ? go_wide_form<96, FMT>(ph, a, s)
                                                                                              : go_wide_form<128, FMT>(ph, a, s);
}

}  // namespace cached
}  // namespace a2d
