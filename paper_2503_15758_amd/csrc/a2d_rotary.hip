// Rotary positions with several axes: (x, y) -> (x cos - y sin, x sin + y cos) of the pairs of columns of Q and K.
//
// The angle of a pair is a position times a frequency.  Taken as a part of a turn it needs only what is left of the product
// behind its whole turns, so the frequency comes as a 64-bit fixed-point part of a turn (2^-64 units, made on the host)
// and the product is formed modulo 2^64: one wrapping multiplication, no reduction, and a position of 2^31 is off by
// 2^-33 turns at most.  Of the product, what is left of the nearest quarter turn becomes an fp32 number, so that it loses 2^-24 of
// itself, wherever the angle is: a sine near half a turn is as good as one near none.  Sine and cosine of up to an eighth
// of a turn are the first terms of their series (see sine_cosine).
//
// Bound: HBM, each value read and written once.  A thread owns eight pairs of a row (two 16-byte pieces a head in bf16):
// it makes their sines and cosines once and walks over heads, as many as still leave the chip full of wavefronts.  32 + 8 heads of 128, 16384
// rows, packed: 70 us, 4.8 TB/s; 24 + 24 of 80, 2999 rows, fp32 to bf16: 14.9 us, 4.6 TB/s; a token of 256 + 64 heads: 3.3 us, host 6.2 to
// 7.2.  (With the hardware's sine and cosine, some 2^-20 of a whole one off, where a low frequency's is 2^-13: 69.6 and 14.7.)
#include "a2d_scored.hpp"

namespace a2d {
namespace {

constexpr int MAX_PAIRS = 128;
struct Turns {
  uint64_t step[MAX_PAIRS];      // part of a turn for a position, 2^-64 units
  uint8_t axis[MAX_PAIRS];
};
struct RotaryArgs {
  int rows, chunks;              // chunks of eight pairs of a row (hdim / 16)
  int half;                      // hdim / 2
  int pairs, axes, inverse;
  int runs, per;                 // runs of heads of a set, `per` heads each
  int heads[2];                  // of a set
  const int32_t* positions;
  const void* x[2];
  void* y[2];
  a2d_layout lx[2], ly[2];
};

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]);
template <>
__device__ __forceinline__ void load8<bf16_t>(const bf16_t* p, float (&v)[8]) {
  const bf16x8 b = *reinterpret_cast<const bf16x8*>(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)b[i];
}
template <>
__device__ __forceinline__ void load8<float>(const float* p, float (&v)[8]) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
}
__device__ __forceinline__ void store8(bf16_t* p, const float (&v)[8]) {
  bf16x8 b;
#pragma unroll
  for (int i = 0; i < 8; ++i) b[i] = (bf16_t)v[i];
  *reinterpret_cast<bf16x8*>(p) = b;
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}

// Sine and cosine of `part` 2^-64 turns: a number of quarter turns, and t = -pi/4 .. pi/4 beyond, as fp32.  The series end at t^9 / 9! and
// t^10 / 10!: what is left off is 2^-28 of the sine and 2^-32 of the cosine at the most; with the roundings 4 half steps of either.
__device__ __forceinline__ void sine_cosine(uint64_t part, float& sn, float& cs) {
  const unsigned quarter = (unsigned)((part + ((uint64_t)1 << 61)) >> 62);
  const float t = (float)(int64_t)(part - ((uint64_t)quarter << 62)) * 0x1.921fb6p-62f, u = t * t;     // 2 pi 2^-64
  const float s = fmaf(t * u, fmaf(u, fmaf(u, fmaf(u, 1 / 362880.f, -1 / 5040.f), 1 / 120.f), -1 / 6.f), t);
  const float c = fmaf(u, fmaf(u, fmaf(u, fmaf(u, fmaf(u, -1 / 3628800.f, 1 / 40320.f), -1 / 720.f), 1 / 24.f), -0.5f), 1.f);
  sn = quarter & 1 ? c : s;
  cs = quarter & 1 ? s : c;
  if (quarter & 2) sn = -sn;
  if ((quarter + 1) & 2) cs = -cs;
}

// (x and y may be the same memory: a thread reads its pieces of a head before it writes them, and no other thread touches them)
template <typename TI, typename TO, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a, Turns turns) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int row = (int)(t / a.chunks), chunk = (int)(t - (int64_t)row * a.chunks);
  if (row >= a.rows) return;
  const int set = blockIdx.y / a.runs, run = blockIdx.y - set * a.runs;
  const int32_t* pos = a.positions + (int64_t)set * a.axes * a.rows + row;
  float cs[8], sn[8];
  const int p0 = 8 * chunk, live = min(max(a.pairs - p0, 0), 8);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int p = min(p0 + i, a.pairs - 1);
    const int64_t at = pos[(int64_t)turns.axis[p] * a.rows];
    sine_cosine((uint64_t)at * turns.step[p], sn[i], cs[i]);
    if (a.inverse) sn[i] = -sn[i];
  }
  const int at0 = INTERLEAVED ? 2 * p0 : p0, at1 = INTERLEAVED ? 2 * p0 + 8 : p0 + a.half;
  const int end = min((run + 1) * a.per, a.heads[0] + a.heads[1]);
  for (int h = run * a.per; h < end; ++h) {
    const int which = h >= a.heads[0], head = set * a.heads[which] + h - (which ? a.heads[0] : 0);
    const TI* x = static_cast<const TI*>(a.x[which]) + head * a.lx[which].head + row * a.lx[which].row;
    TO* y = static_cast<TO*>(a.y[which]) + head * a.ly[which].head + row * a.ly[which].row;
    float u[8], v[8], ou[8], ov[8];
    load8<TI>(x + at0, u);
    load8<TI>(x + at1, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // pair i: columns (u[i], v[i]), or (w[2 i], w[2 i + 1]) of the sixteen w = u, v
      float& px = INTERLEAVED ? (i < 4 ? u[2 * i] : v[2 * i - 8]) : u[i];
      float& py = INTERLEAVED ? (i < 4 ? u[2 * i + 1] : v[2 * i - 7]) : v[i];
      float& qx = INTERLEAVED ? (i < 4 ? ou[2 * i] : ov[2 * i - 8]) : ou[i];
      float& qy = INTERLEAVED ? (i < 4 ? ou[2 * i + 1] : ov[2 * i - 7]) : ov[i];
      qx = i < live ? px * cs[i] - py * sn[i] : px;      // (columns of no pair: not even times 1, plus 0 times the other)
      qy = i < live ? px * sn[i] + py * cs[i] : py;
    }
    store8(y + at0, ou);
    store8(y + at1, ov);
  }
}

template <typename TI, typename TO>
hipError_t go(const RotaryArgs& a, const Turns& t, dim3 grid, bool interleaved, hipStream_t s) {
  if (interleaved) A2D_LAUNCH((rotary_kernel<TI, TO, true>), grid, dim3(256), 0, s, a, t);
  else A2D_LAUNCH((rotary_kernel<TI, TO, false>), grid, dim3(256), 0, s, a, t);
  return hipGetLastError();
}

// freq / (2 pi) modulo 1, in 2^-64 units: the product of freq's 53 bits and the first 128 of 1 / (2 pi) behind the point, in integers (a call
// makes one for each pair: as divisions and floors of 80-bit numbers they took 8.7 us of the host's time for 64 pairs).
// |freq| < 2^64: beyond, 128 bits do not reach the fraction.
uint64_t part_of_turn(double freq) {
  constexpr uint64_t kHi = 0x28BE60DB9391054Aull, kLo = 0x7F09D5F47D4D3770ull;
  uint64_t bits;
  __builtin_memcpy(&bits, &freq, sizeof(bits));
  const int biased = (int)(bits >> 52) & 0x7FF, e = biased ? biased - 1075 : -1074;        // |freq| = m 2^e
  const uint64_t m = (bits & (((uint64_t)1 << 52) - 1)) | (biased ? (uint64_t)1 << 52 : 0);
  const int shift = 64 - e;                                              // of m / (2 pi) in 2^-128 units, down
  if (shift >= 192) return 0;
  const unsigned __int128 low = (unsigned __int128)m * kLo, high = (unsigned __int128)m * kHi + (uint64_t)(low >> 64);
  const uint64_t w[4] = {(uint64_t)low, (uint64_t)high, (uint64_t)(high >> 64), 0};
  const int at = shift / 64, by = shift % 64;
  const uint64_t part = by ? w[at] >> by | w[at + 1] << (64 - by) : w[at];
  return bits >> 63 ? 0 - part : part;
}

}  // namespace

hipError_t launch_rotary(const a2d_rotary_desc& d, int n, const a2d_rotary_tensor* x, int cus, hipStream_t s) {
  RotaryArgs a{};
  Turns t{};
  a.rows = d.rows;
  a.chunks = d.hdim / 16;
  a.half = d.hdim / 2;
  a.pairs = d.pairs;
  a.axes = d.axes;
  a.inverse = d.inverse;
  a.positions = d.positions;
  for (int i = 0; i < n; ++i) {
    a.heads[i] = x[i].heads / d.sets;
    a.x[i] = x[i].x;
    a.y[i] = x[i].y;
    a.lx[i] = x[i].lx;
    a.ly[i] = x[i].ly;
  }
  for (int p = 0; p < d.pairs; ++p) {
    t.step[p] = part_of_turn(d.freqs[p]);
    t.axis[p] = d.axis ? d.axis[p] : 0;
  }
  const int heads = a.heads[0] + a.heads[1];
  const int64_t blocks = ((int64_t)d.rows * a.chunks + 255) / 256;
  // heads of a thread: as many as leave eight workgroups for each compute unit, at least one
  int64_t runs = (8 * cus + blocks * d.sets - 1) / (blocks * d.sets);
  if (runs > heads) runs = heads;
  if (runs > 65535 / d.sets) runs = 65535 / d.sets;                     // (a launch's second dimension)
  if (runs < 1) runs = 1;
  a.per = (heads + (int)runs - 1) / (int)runs;
  a.runs = (heads + a.per - 1) / a.per;
  const dim3 grid((unsigned)blocks, (unsigned)(a.runs * d.sets));
  const bool f = d.in_dtype == A2D_F32;
  return f && d.out_dtype == A2D_F32 ? go<float, float>(a, t, grid, d.interleaved != 0, s)
         : f                         ? go<float, bf16_t>(a, t, grid, d.interleaved != 0, s)
                                     : go<bf16_t, bf16_t>(a, t, grid, d.interleaved != 0, s);
}

}  // namespace a2d
