// Rotary positions (rest_rotary), and the rows of a step rotated and written into a cache in pages in one
// launch: 16-bit pages (rest_paged_kv_append) or e4m3 pages with scales (rest_paged_kv_append_scaled).
// Not in the paper, which takes the verifier as given; the position ids are rest_draft's.
//
// Pair f of a row at position p turns by the angle t = p * inv_freq[f]:
//   y1 = a (x1 cos t - x2 sin t), y2 = a (x2 cos t + x1 sin t).
// t is a product in 64 bits (exact up to p = 2^29): in 32 bits the angle of position 10^6 would be 0.03 off.  For queries
// and 16-bit keys whole quarter turns are taken off it in 64 bits; the rest's sine and cosine and the rotation are in 32 bits,
// rounded once: below 2^-22 of |x1| + |x2|, where half a step of 16 bits is 2^-11 or 2^-8.  (Rows of 32 bits are up to four
// half steps off by it, in the same kernel.)  Keys that become codes are rotated in 64 bits throughout: the border between two
// codes decides a whole step of 2^-4, so that a result a rounding off would now and then be a code off.
//
// Pages with scales: the 16 rows of a block share a scale per head, the smallest power of two that holds the largest new
// value, and never less than before where the block has older rows; those are requantised when it grows
// (by a power of two, so they change only where they fall below the smallest code).
//
// A thread block takes new rows of one context that fall into one block of 16 rows.  A row is D / 16 lanes, 16
// elements each (a pair's halves sit in the same lane, unless half the head is no multiple of 8); a lane stays with its
// row, keeps its sines and cosines in registers and steps through the heads, four of them on their way at a time.  One
// head's keys or values of a block of codes are a warp's, which holds all its rows while it looks for the largest value;
// the angles of its thread block's rows are computed once, into shared memory.
//
// What bounds it, for few rows: the launch and the chain length -> table -> page (one row: 4.1 to 4.6 us with codes or without).
// For many, measured with 128 x up to 64 rows, D = 128, 32 heads of queries and 8 of keys and values: the rotation of 64 rows
// of queries alone takes 28 us (4.8 TB/s, 73 % of the copy rate; 1024 equal blocks for 444 that are resident leave the last
// wave a third full); the append with codes 45 us, 20 of them for the queries and 21 for K and V alone: a warp's chain of
// rows, angles, products, scale and codes at 16 warps an SM (issue 41 %, conversions 32 %, 64-bit pipe 9 %, HBM 12 %).  With
// 61 pairs, half the head apart, 60 us and 95 us: shifting the partners into place is bound by the instructions it takes, and
// codes of 128 elements spill 460 to 520 bytes a thread there.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "common.cuh"
#include "e4m3.cuh"
#include "paged_pool.cuh"
#include "rest.h"

namespace {

using namespace rest_pool;
using namespace rest_e4m3;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMostRows = 1 << 30;                      // of a context in a call (sums with it stay below 2^31)
constexpr double kQuarterTurns = 0.63661977236758134308, kQuarterHigh = 0x1.921fb54400000p+0,    // 2 / pi; pi / 2 in two parts
                 kQuarterLow = 0x1.0b4611a626331p-34;
enum Where { kNowhere, kPages16, kPagesScaled };        // where keys and values go

struct Args {
  Pool c;                                               // strides in vectors of 16 bytes
  float *k_scales, *v_scales;
  const void *q, *k_new, *v_new;
  void* q_out;
  int64_t q_b, q_n, q_h, o_b, o_n, o_h, n_b, n_n, n_h;  // in elements
  const int32_t *kv_len, *n_nodes, *pos;
  const float* inv_freq;
  int N, H, H_kv, D, half, groups, interleaved, parts, code_parts;
  float amplitude;
};

// eight elements as they lie in memory
template <typename T> struct Eight {
  uint4 v[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = reinterpret_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(p)[i] = v[i];
  }
  __device__ __forceinline__ void to(float* x) const {
    const uint32_t w[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[sizeof(T) / 2 - 1].x, v[sizeof(T) / 2 - 1].y,
                           v[sizeof(T) / 2 - 1].z, v[sizeof(T) / 2 - 1].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) {
        x[2 * i] = __uint_as_float(w[2 * i]);
        x[2 * i + 1] = __uint_as_float(w[2 * i + 1]);
      } else {
        float2 f;
        if constexpr (__is_same(T, __half)) f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        else f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w[i]));
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
      }
    }
  }
};
template <typename T> __device__ __forceinline__ Eight<T> packed(const float* x) {
  Eight<T> e;
  if constexpr (sizeof(T) == 4) {
    e.v[0] = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    e.v[1] = make_uint4(__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7]));
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (__is_same(T, __half)) {
        const __half2 h = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
      } else {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
      }
    }
    e.v[0] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return e;
}
// y's elements from `live` on, an even number, are x's, bit for bit.
template <typename T> __device__ __forceinline__ void keep(Eight<T>& y, const Eight<T>& x, int live) {
  constexpr int kPerWord = 4 / (int)sizeof(T);
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
    if (kPerWord * (4 * i) >= live) y.v[i].x = x.v[i].x;
    if (kPerWord * (4 * i + 1) >= live) y.v[i].y = x.v[i].y;
    if (kPerWord * (4 * i + 2) >= live) y.v[i].z = x.v[i].z;
    if (kPerWord * (4 * i + 3) >= live) y.v[i].w = x.v[i].w;
  }
}
// Elements s .. s + 7 of the 16 in a and b.
template <typename T> __device__ __forceinline__ Eight<T> shifted(const Eight<T>& a, const Eight<T>& b, int s) {
  constexpr int kWords = 2 * (int)sizeof(T), kPerWord = 4 / (int)sizeof(T);
  uint32_t w[2 * kWords];
#pragma unroll
  for (int i = 0; i < kWords / 4; ++i) {
    w[4 * i] = a.v[i].x, w[4 * i + 1] = a.v[i].y, w[4 * i + 2] = a.v[i].z, w[4 * i + 3] = a.v[i].w;
    w[kWords + 4 * i] = b.v[i].x, w[kWords + 4 * i + 1] = b.v[i].y, w[kWords + 4 * i + 2] = b.v[i].z, w[kWords + 4 * i + 3] = b.v[i].w;
  }
#pragma unroll
  for (int by = kWords / 2; by > 0; by >>= 1)
#pragma unroll
    for (int i = 0; i + by < 2 * kWords; ++i) w[i] = (s / kPerWord) & by ? w[i + by] : w[i];
  if constexpr (kPerWord == 2) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16 * (s & 1));
  }
  Eight<T> out;
#pragma unroll
  for (int i = 0; i < kWords / 4; ++i) out.v[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  return out;
}

// A lane's 16 elements of a row, in two runs of 8 from at[0] and at[1].  kPairs: a pair's halves lie in the same place
// of both runs (half the head apart); kNeighbours: pairs are neighbours (where their number is no multiple of 8, only the
// first of them may turn); kStill: nothing turns; kLoose: half the head is no multiple of 8, so that runs of 8 do not meet
// their partners (class Loose).
enum Kind { kPairs, kNeighbours, kStill, kLoose };
struct Lane { Kind kind; int at[2], first; };           // first: of kPairs and kNeighbours, the first pair's number
__device__ __forceinline__ Lane lane_of(const Args& a, int chunk) {
  const int at = 16 * chunk, pairs = a.half >> 3;
  if (a.interleaved || (a.half & 7)) return {at >= 2 * a.half ? kStill : a.interleaved ? kNeighbours : kLoose, {at, at + 8}, 8 * chunk};
  return chunk < pairs ? Lane{kPairs, {8 * chunk, a.half + 8 * chunk}, 8 * chunk} : Lane{kStill, {at, at + 8}, 0};
}
// What a lane of kLoose does with element j of its 16, at + j of the row: y = x cos + partner sin, the sine's sign being
// that of its half of the pair.
struct Loose {
  int at, half;
  __device__ __forceinline__ Loose(const Args& a, const Lane& l) : at(l.at[0]), half(a.half) {}
  __device__ __forceinline__ bool turns(int j) const { return at + j < 2 * half; }
  __device__ __forceinline__ bool second(int j) const { return at + j >= half; }
  __device__ __forceinline__ int pair(int j) const { return at + j - (second(j) ? half : 0); }
  // The partners of run k (0 or 1), half the head away: aligned loads on both sides, shifted.  Two sets where the run
  // holds the end of the first half.
  template <typename T> __device__ __forceinline__ void partners(const T* row, int k, int D, float (&p)[8]) const {
    const int e = at + 8 * k;
    run(row, e + (e >= half ? -half : half), D, p);
    if (e < half && e + 8 > half) {
      float x[8];
      run(row, e - half, D, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) p[j] = e + j >= half ? x[j] : p[j];
    }
  }
  // elements from .. from + 7 of a row, 0 outside of it
  template <typename T> static __device__ __forceinline__ void run(const T* row, int from, int D, float (&x)[8]) {
    const int base = from & ~7;
    Eight<T> lo = {}, hi = {};
    if (base >= 0 && base < D) lo.load(row + base);
    if (base + 8 >= 0 && base + 8 < D) hi.load(row + base + 8);
    shifted(lo, hi, from & 7).to(x);
  }
};
// What is left of the angle t without whole quarter turns, in 64 bits (the reduction of Cody and Waite): pi / 2 in two parts,
// the first of 33 bits, so that its multiples up to 2^20 are exact; beyond them the multiply-add rounds once, what is left of t.
__device__ __forceinline__ double reduced(double t, double& whole) {
  whole = rint(t * kQuarterTurns);
  return fma(-whole, kQuarterLow, fma(-whole, kQuarterHigh, t));
}
// Cosine and sine of pair f of a row at position p, times the amplitude, in 32 bits: whole quarter turns are taken off in
// 64, and what is left, |x| <= pi / 4, goes through the Taylor series, whose next terms are below 2^-29 (x^11 / 11!,
// x^12 / 12!).
__device__ __forceinline__ float2 turn_of(const Args& a, double p, int f) {
  double whole;
  const float x = (float)reduced(p * (double)a.inv_freq[f], whole), z = x * x;
  const float s = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), x);
  const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const int q = (int)(long long)whole;
  const float cq = q & 1 ? s : c, sq = q & 1 ? c : s;
  return make_float2(a.amplitude * ((q + 1) & 2 ? -cq : cq), a.amplitude * (q & 2 ? -sq : sq));
}
// The same in 64 bits, from the angle t: the Taylor series up to terms below 2^-54 (x^17 / 17!, x^18 / 18!).
__device__ __forceinline__ double2 turn64(double t, double amplitude) {
  double whole;
  const double x = reduced(t, whole), z = x * x;
  double s = -1.0 / 1307674368000.0, c = 1.0 / 20922789888000.0;
  s = fma(s, z, 1.0 / 6227020800.0);
  c = fma(c, z, -1.0 / 87178291200.0);
  s = fma(s, z, -1.0 / 39916800.0);
  c = fma(c, z, 1.0 / 479001600.0);
  s = fma(s, z, 1.0 / 362880.0);
  c = fma(c, z, -1.0 / 3628800.0);
  s = fma(s, z, -1.0 / 5040.0);
  c = fma(c, z, 1.0 / 40320.0);
  s = fma(s, z, 1.0 / 120.0);
  c = fma(c, z, -1.0 / 720.0);
  s = fma(s, z, -1.0 / 6.0);
  c = fma(c, z, 1.0 / 24.0);
  s = fma(s * z, x, x);
  c = fma(c, z, -0.5);
  c = fma(c, z, 1.0);
  const int q = (int)(long long)whole;
  const double cq = q & 1 ? s : c, sq = q & 1 ? c : s;
  return make_double2(amplitude * ((q + 1) & 2 ? -cq : cq), amplitude * (q & 2 ? -sq : sq));
}
// Where pair f of row r has its cosine and sine (64 bits).  Lanes next to one another read pairs 8 apart, so of each eight the
// twos are laid out apart: 16-byte reads without bank conflicts.
__device__ __forceinline__ int table_at(const Args& a, int r, int f) {
  const int eighths = a.half >> 3;
  return r * a.half + ((a.half & 7) ? f : ((((f >> 1) & 3) * eighths + (f >> 3)) << 1 | (f & 1)));
}

// cosines and sines of a lane's eight pairs
template <typename F> struct Angles { F c[8], s[8]; };
// The rotated elements y of a lane from x; `round` makes what is stored of each.
template <bool NEIGHBOURS, typename F, typename R>
__device__ __forceinline__ void rotate(const Angles<F>& t, const float (&x)[16], float (&y)[16], R round) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    constexpr int kApart = NEIGHBOURS ? 1 : 8, kStep = NEIGHBOURS ? 2 : 1;
    const F c = t.c[j], s = t.s[j], x1 = x[kStep * j], x2 = x[kStep * j + kApart];
    y[kStep * j] = round(fma(x1, c, -(x2 * s)));
    y[kStep * j + kApart] = round(fma(x2, c, x1 * s));
  }
}
// A lane's 16 elements of a new row as they become codes: rotated in 64 bits, rounded to 32.
template <bool LOOSE, typename T, typename R>
__device__ __forceinline__ void code_values(const Args& a, const Eight<T> (&e)[2], const T* row, const Lane& l, const double2* table,
                                            int r, float (&y)[16], R round) {
  float x[16];
  e[0].to(x);
  e[1].to(x + 8);
  if (l.kind == kStill) {
#pragma unroll
    for (int j = 0; j < 16; ++j) y[j] = x[j];
  } else if (LOOSE && l.kind == kLoose) {
    const Loose o(a, l);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float p[8];
      o.partners(row, k, a.D, p);
#pragma unroll
      for (int j = 8 * k; j < 8 * k + 8; ++j) {
        y[j] = x[j];
        if (o.turns(j)) {
          const double2 cs = table[table_at(a, r, o.pair(j))];
          y[j] = round(fma((double)x[j], cs.x, (double)p[j & 7] * (o.second(j) ? cs.y : -cs.y)));
        }
      }
    }
  } else {
    Angles<double> t;
    if (LOOSE) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const double2 cs = table[table_at(a, r, min(l.first + j, a.half - 1))];
        t.c[j] = cs.x;
        t.s[j] = cs.y;
      }
      rotate<true>(t, x, y, round);
#pragma unroll
      for (int j = 0; j < 16; ++j) y[j] = l.at[0] + j < 2 * a.half ? y[j] : x[j];
      return;
    }
    const double2* twos = table + table_at(a, r, l.first);
    const int apart = a.half >> 2;                      // (see table_at)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const double2 cs = twos[(j >> 1) * apart + (j & 1)];
      t.c[j] = cs.x;
      t.s[j] = cs.y;
    }
    if (l.kind == kPairs) rotate<false>(t, x, y, round);
    else rotate<true>(t, x, y, round);
  }
}
// 64 bits rounded to 32; what is finite stays so.
__device__ __forceinline__ float finite_float(double v) {
  const float f = __double2float_rn(v);
  return fabsf(f) < INFINITY ? f : __double2float_rz(v);
}
// The largest finite magnitude of a lane's values, those in 64 bits rounded up; only asked for where it matters (below).
template <typename T, int D, bool LOOSE>
__device__ __noinline__ float largest_rounded_up(const Args& a, const T* row, bool turn, const double2* table, int rows) {
  constexpr int kLanes = D / 16, kRows = 32 / kLanes;
  const int lane = threadIdx.x & 31, sub = lane / kLanes, chunk = lane % kLanes;
  const Lane l = turn ? lane_of(a, chunk) : Lane{kStill, {16 * chunk, 16 * chunk + 8}, 0};
  float most = 0.f, y[16];
  for (int r = sub; r < rows; r += kRows) {
    Eight<T> e[2];
    e[0].load(row + r * a.n_n + l.at[0]);
    e[1].load(row + r * a.n_n + l.at[1]);
    code_values<LOOSE>(a, e, row + r * a.n_n, l, table, r, y, [&](double v) {
      const float up = __double2float_ru(fabs(v));
      most = fmaxf(most, up < INFINITY ? up : 0.f);
      return finite_float(v);
    });
#pragma unroll
    for (int j = 0; j < 16; ++j) most = fmaxf(most, fabsf(y[j]) < INFINITY ? fabsf(y[j]) : 0.f);
  }
  return most;
}
// A lane's 16 values, times `inverse`, as codes of a row.
__device__ __forceinline__ void put_codes(float (&y)[16], float inverse, unsigned char* row, const Lane& l) {
#pragma unroll
  for (int j = 0; j < 16; ++j) y[j] *= inverse;
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = pack2(y[4 * j], y[4 * j + 1]) | pack2(y[4 * j + 2], y[4 * j + 3]) << 16;
  *reinterpret_cast<uint2*>(row + l.at[0]) = make_uint2(w[0], w[1]);
  *reinterpret_cast<uint2*>(row + l.at[1]) = make_uint2(w[2], w[3]);
}
// The codes of a block's new rows (`codes`: the first one's) where a value is beyond 32 bits: what is finite stays so, the rest is NaN.
template <typename T, int D, bool LOOSE>
__device__ __noinline__ void write_finite(const Args& a, const T* row, bool turn, const double2* table, int rows, float inverse,
                                          unsigned char* codes, int64_t code_row) {
  constexpr int kLanes = D / 16, kRows = 32 / kLanes;
  const int lane = threadIdx.x & 31, sub = lane / kLanes, chunk = lane % kLanes;
  const Lane l = turn ? lane_of(a, chunk) : Lane{kStill, {16 * chunk, 16 * chunk + 8}, 0};
  for (int r = sub; r < rows; r += kRows) {
    Eight<T> e[2];
    float y[16];
    e[0].load(row + r * a.n_n + l.at[0]);
    e[1].load(row + r * a.n_n + l.at[1]);
    code_values<LOOSE>(a, e, row + r * a.n_n, l, table, r, y, [](double v) { return finite_float(v); });
#pragma unroll
    for (int j = 0; j < 16; ++j) y[j] = fabsf(y[j]) < INFINITY ? y[j] : NAN;
    put_codes(y, inverse, codes + r * code_row, l);
  }
}

// One head's keys or values of a block of 16 rows: a warp.  Rows lo .. lo + m - 1 of the block are new, `row` is the first
// of them in memory; codes and scale: the block's in the pool.
template <typename T, int D> struct Rows {
  const T* row;
  bool turn;
  unsigned char* codes;
  float* scale;
  Lane l;
  float old;
  // looks up head u of K, then of V
  __device__ __forceinline__ void load(const Args& a, int u, int64_t new_row, int64_t page_row, int64_t cell, int lo) {
    const int chunk = (threadIdx.x & 31) % (D / 16);
    const bool v = u >= a.H_kv;
    const int h = v ? u - a.H_kv : u;
    row = static_cast<const T*>(v ? a.v_new : a.k_new) + new_row + h * a.n_h;
    turn = !v && a.half > 0;
    codes = reinterpret_cast<unsigned char*>((v ? a.c.v : a.c.k) + page_row + h * a.c.s_head);
    scale = (v ? a.v_scales : a.k_scales) + cell + (int64_t)h * (1 << (a.c.page_log - 4));
    l = turn ? lane_of(a, chunk) : Lane{kStill, {16 * chunk, 16 * chunk + 8}, 0};
    old = lo > 0 ? *scale : 0.f;
  }
};
template <typename T, int D, bool LOOSE>
__device__ __forceinline__ void write_codes(const Args& a, const Rows<T, D>& x, const double2* table, int lo, int m, int64_t code_row) {
  constexpr int kLanes = D / 16, kRows = 32 / kLanes, kSteps = 16 / kRows;
  const int lane = threadIdx.x & 31, sub = lane / kLanes, chunk = lane % kLanes, hi = lo + m;
  const Lane l = x.l;
  unsigned char* codes = x.codes;
  const float old = lo > 0 ? within_limits(x.old) : 0.f;
  // Rows are kept as they come and rotated twice, for the largest value and for the codes: 32 registers instead of 64 that
  // do not fit (128 x 64 rows: 47 us, once 51).  LOOSE: once (95 us, twice 110).
  Eight<T> e[LOOSE ? 1 : kSteps][2];
  float kept[LOOSE ? kSteps : 1][16], most = 0.f;
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int r = i * kRows + sub;
    if (!LOOSE && lo + r < hi) {
      e[LOOSE ? 0 : i][0].load(x.row + r * a.n_n + l.at[0]);
      e[LOOSE ? 0 : i][1].load(x.row + r * a.n_n + l.at[1]);
    }
  }
  auto values = [&](int i, float (&y)[16]) {
    const int r = i * kRows + sub;
    if (LOOSE) {
      e[0][0].load(x.row + r * a.n_n + l.at[0]);
      e[0][1].load(x.row + r * a.n_n + l.at[1]);
    }
    code_values<LOOSE>(a, e[LOOSE ? 0 : i], x.row + r * a.n_n, l, table, r, y, [](double v) { return __double2float_rn(v); });
  };
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int r = i * kRows + sub;
    if (lo + r < hi) {
      float(&y)[16] = kept[LOOSE ? i : 0];
      values(i, y);
#pragma unroll
      for (int j = 0; j < 16; j += 2) most = fmaxf(most, fmaxf(fabsf(y[j]), fabsf(y[j + 1])));      // (NaN is passed over)
    }
  }
  most = warp_max(most);
  // An infinity has no part in the scale, a finite value that 32 bits do not hold has one; and 64 bits just above 448 times a
  // power of two, which round to it, count as more.
  const bool infinite = most == INFINITY;
  if (infinite || (x.turn && (__float_as_uint(most) & 0x7FFFFFu) == 0x600000u))
    most = warp_max(largest_rounded_up<T, D, LOOSE>(a, x.row, x.turn, table, m));
  const float need = fitting_scale(most), s = fmaxf(need, old);
  const float inverse = 1.f / s;                        // (a power of two, and the products exact, unless an older scale was none:
                                                        // then a product 2^-23 off may be a code off)
  if (lo > 0 && s != old) {                             // older rows: the scale grew
    const float ratio = old / s;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int r = i * kRows + sub;
      if (r < lo) {
        uint4* p = reinterpret_cast<uint4*>(codes + r * code_row + 16 * chunk);
        *p = rescale16(*p, ratio);
      }
    }
  }
  if (infinite) {
    write_finite<T, D, LOOSE>(a, x.row, x.turn, table, m, inverse, codes + lo * code_row, code_row);
  } else {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int r = lo + i * kRows + sub;
      if (r < hi) {
        float(&y)[16] = kept[LOOSE ? i : 0];
        if (!LOOSE) values(i, y);
        put_codes(y, inverse, codes + r * code_row, l);
      }
    }
  }
  __syncwarp();                                         // (every lane has read the old scale)
  if (lane == 0) *x.scale = s;
}

// (LOOSE: the number of pairs is no multiple of 8.  A kernel of its own: in one, the others lose registers, and 128 x 64
// rows of 32 heads take 35 us instead of 28.)
template <typename T, Where W, int D_SCALED, bool LOOSE>
__global__ void __launch_bounds__(kThreads, W == kPagesScaled || LOOSE ? 2 : 3) rest_kv_append_kernel(const __grid_constant__ Args a) {
  grid_wait();
  extern __shared__ __align__(16) unsigned char smem[];
  const int all_groups = gridDim.x / a.parts, part = blockIdx.x / all_groups, b = blockIdx.x % all_groups / a.groups,
            group = blockIdx.x % all_groups % a.groups;
  const int n = a.n_nodes ? min(max(a.n_nodes[b], 0), a.N) : a.N;
  const int L = W == kNowhere ? 0 : a.kv_len[b];
  // new rows i0 .. i1 - 1 are rows lo ... of the block that starts at row `first`
  const uint32_t first = ((uint32_t)max(L, 0) & ~15u) + 16u * group;
  const int i0 = max((int)(first - (uint32_t)max(L, 0)), 0), lo = group == 0 ? max(L, 0) & 15 : 0;
  const int m = min(n - i0, 16 - lo);
  if (m <= 0) return;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t page_row = W == kNowhere || L < 0 || first > 0x7FFFFFFFu ? -1 : row_offset(a.c, b, (int)first);
  if constexpr (W == kPagesScaled) {
    if (part < a.code_parts) {                          // some blocks write codes, the others rows
      if (page_row < 0) return;
      const int p = a.c.table[b * a.c.table_stride + (first >> a.c.page_log)];
      const int64_t cell = (int64_t)p * a.H_kv * (1 << (a.c.page_log - 4)) + ((first & ((1u << a.c.page_log) - 1)) >> 4);
      const int64_t new_row = b * a.n_b + i0 * a.n_n;
      int u = part * kWarps + warp;
      Rows<T, D_SCALED> x;
      if (u < 2 * a.H_kv) x.load(a, u, new_row, page_row, cell, lo);
      double2* table = reinterpret_cast<double2*>(smem);
      if (part * kWarps < a.H_kv && a.half > 0) {       // (else no keys)
        for (int e = threadIdx.x; e < m * a.half; e += kThreads) {
          const int r = e / a.half, f = e - r * a.half;
          table[table_at(a, r, f)] = turn64((double)a.pos[(int64_t)b * a.N + i0 + r] * (double)a.inv_freq[f], a.amplitude);
        }
        __syncthreads();
      }
      while (u < 2 * a.H_kv) {
        write_codes<T, D_SCALED, LOOSE>(a, x, table, lo, m, a.c.s_row * 16);
        u += a.code_parts * kWarps;
        if (u < 2 * a.H_kv) x.load(a, u, new_row, page_row, cell, lo);
      }
      return;
    }
  }

  // rows of 16-bit (or 32-bit) results: D / 16 lanes a row; a lane stays with its row and steps through the heads
  const int lanes = a.D >> 4, rows = 32 / lanes, sub = lane / lanes, chunk = lane % lanes;
  if (sub >= rows) return;                              // (D / 16 need not divide 32)
  const int me = warp * rows + sub, all = kWarps * rows;
  const int together = all >= m ? all / m : 1;          // heads at a time
  if (all >= m && me >= together * m) return;
  const Lane l = lane_of(a, chunk);
  const int moving = min(lanes, (2 * a.half + 15) >> 4);        // lanes of a row of loose pairs that hold some
  const int parts = a.parts - a.code_parts, h0 = (all >= m ? me / m : 0) + (part - a.code_parts) * together, step = together * parts;
  for (int r = all >= m ? me % m : me; r < m; r += all >= m ? m : all) {
    Angles<float> t;
    float c[LOOSE ? 16 : 1], s[LOOSE ? 16 : 1];         // of kLoose, for each element
    bool known = false;
    // one row in `count` heads; the first heads are on their way while the angles are worked out
    auto heads = [&](const T* from, int64_t from_h, T* to, int64_t to_h, int count, Kind kind) {
      if constexpr (LOOSE) {
        if (kind == kLoose) {
          const Loose o(a, l);
          if (!known) {
            const double p = a.pos[(int64_t)b * a.N + i0 + r];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const float2 cs = o.turns(j) ? turn_of(a, p, o.pair(j)) : make_float2(1.f, 0.f);
              c[j] = cs.x;
              s[j] = o.second(j) ? cs.y : -cs.y;
            }
            known = true;
          }
          for (int h = h0; h < count; h += step) {
            const T* x0 = from + h * from_h;
            Eight<T> e[2];
            float other[2][8];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              e[k].load(x0 + l.at[k]);
              o.partners(x0, k, a.D, other[k]);
            }
            // a row may be rotated in place: all its lanes have loaded before the first stores
            __syncwarp(((moving == 32 ? 0u : 1u << moving) - 1u) << (sub * lanes));
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              float x[8], y[8];
              e[k].to(x);
#pragma unroll
              for (int j = 0; j < 8; ++j) y[j] = fmaf(x[j], c[8 * k + j], other[k][j] * s[8 * k + j]);
              Eight<T> out = packed<T>(y);
              keep(out, e[k], 2 * a.half - l.at[k]);
              out.store(to + h * to_h + l.at[k]);
            }
          }
          return;
        }
      }
      constexpr int kAtOnce = sizeof(T) == 4 || W == kPages16 ? 2 : 4;      // heads on their way
      from += h0 * from_h;
      to += h0 * to_h;
      from_h *= step;
      to_h *= step;
      for (int left = h0 < count ? (count - h0 + step - 1) / step : 0; left > 0; left -= kAtOnce, from += kAtOnce * from_h, to += kAtOnce * to_h) {
        Eight<T> e[kAtOnce][2];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
          if (i < left) {
            e[i][0].load(from + i * from_h + l.at[0]);
            e[i][1].load(from + i * from_h + l.at[1]);
          }
        if (kind != kStill && !known) {
          const double p = a.pos[(int64_t)b * a.N + i0 + r];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float2 cs = turn_of(a, p, LOOSE ? min(l.first + j, a.half - 1) : l.first + j);
            t.c[j] = cs.x;
            t.s[j] = cs.y;
          }
          known = true;
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
          if (i < left) {
            T* y0 = to + i * to_h;
            if (kind == kStill) {
              e[i][0].store(y0 + l.at[0]);
              e[i][1].store(y0 + l.at[1]);
            } else {
              float x[16], y[16];
              e[i][0].to(x);
              e[i][1].to(x + 8);
              auto same = [](float v) { return v; };
              if (kind == kPairs) rotate<false>(t, x, y, same);
              else rotate<true>(t, x, y, same);
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                Eight<T> out = packed<T>(y + 8 * k);
                if (LOOSE) keep(out, e[i][k], 2 * a.half - l.at[k]);
                out.store(y0 + l.at[k]);
              }
            }
          }
      }
    };
    if (a.H > 0)
      heads(static_cast<const T*>(a.q) + b * a.q_b + (i0 + r) * a.q_n, a.q_h,
            static_cast<T*>(a.q_out) + b * a.o_b + (i0 + r) * a.o_n, a.o_h, a.H, l.kind);
    if (W == kPages16 && page_row >= 0) {
      const int64_t new_row = b * a.n_b + (i0 + r) * a.n_n, to = page_row + (lo + r) * a.c.s_row;
      heads(static_cast<const T*>(a.k_new) + new_row, a.n_h, reinterpret_cast<T*>(a.c.k + to), a.c.s_head * 8, a.H_kv, l.kind);
      heads(static_cast<const T*>(a.v_new) + new_row, a.n_h, reinterpret_cast<T*>(a.c.v + to), a.c.s_head * 8, a.H_kv, kStill);
    }
  }
}

template <typename T, Where W, int D>
rest_status run(const Args& a, int B, void* stream) {
  // Few rows: their heads are shared out until a warp has one task or there are eight blocks an SM (of which three are
  // resident, two with codes).  Many: still two blocks of codes (K and V, which needs no angles) and two of rows for
  // each group of 16, so that the last wave is short.
  const int64_t blocks = (int64_t)B * a.groups;
  const int sms = rest::sm_count(), most = min(a.N, 16), rows = 32 / (a.D / 16);
  const int64_t wanted = 8 * (int64_t)(sms > 0 ? sms : 148) / (blocks > 0 ? blocks : 1), each = W == kPagesScaled ? wanted / 2 : wanted;
  auto tasks = [](int warps) { return (warps + kWarps - 1) / kWarps; };
  auto parts = [&](int tasks_) { return (int)(tasks_ < 2 || tasks_ < each ? tasks_ : each < 2 ? 2 : each); };
  // Many rows: the queries in a launch of their own, at three blocks an SM instead of the two that codes allow
  // (128 x up to 64 rows, 32/8 heads, before rows were rotated twice: 49 us in two, 52 in one).
  const bool two = W == kPagesScaled && a.H > 0 && each < 2;
  Args args = a;
  if (two) args.H = 0;
  args.code_parts = W == kPagesScaled ? parts(tasks(2 * a.H_kv)) : 0;
  args.parts = args.code_parts + parts(tasks(((W == kPages16 ? a.H + 2 * a.H_kv : args.H) * most + rows - 1) / rows));
  if (blocks * args.parts > 0x7FFFFFFFll) return REST_UNSUPPORTED;      // (before the first launch)
  if (two) {
    Args queries = a;
    queries.groups = (a.N + 15) / 16;
    if (rest_status st = run<T, kNowhere, 0>(queries, B, stream)) return st;
  }
  const size_t smem = W == kPagesScaled ? (size_t)16 * a.half * sizeof(double2) : 0;
  REST_CUDA_TRY(launch(a.half & 7 ? rest_kv_append_kernel<T, W, D, true> : rest_kv_append_kernel<T, W, D, false>, dim3((unsigned)(blocks * args.parts)), kThreads, smem, stream, args));
  return REST_OK;
}

bool rows_ok(const int64_t* s, int64_t B, int64_t N, int64_t H, int D, int per_vec) {
  const int64_t extent[3] = {B, N, H};
  for (int i = 0; i < 3; ++i)
    if (extent[i] > 1 && s[i] < D) return false;
  return stride_ok(s, 3, per_vec);
}

// the rotation's arguments, for all three calls
rest_status fill_turn(Args& a, const int32_t* pos, const float* inv_freq, int32_t pairs, int32_t interleaved, float amplitude,
                      int32_t D) {
  if (pairs < 0 || 2 * (int64_t)pairs > D || (pairs > 0 && (!pos || !inv_freq))) return REST_INVALID_ARG;
  if (!(fabsf(amplitude) < INFINITY)) return REST_INVALID_ARG;
  a.pos = pos; a.inv_freq = inv_freq; a.half = pairs; a.interleaved = interleaved != 0; a.amplitude = amplitude; a.D = D;
  return REST_OK;
}
rest_status fill_q(Args& a, const void* q, const int64_t* qs, void* out, const int64_t* os, int64_t B, int64_t N, int64_t H,
                   int per_vec) {
  if (!q || !out || !qs || !os || !aligned16(q, out)) return REST_INVALID_ARG;
  if (!rows_ok(qs, B, N, H, a.D, per_vec) || !rows_ok(os, B, N, H, a.D, per_vec)) return REST_INVALID_ARG;
  a.q = q; a.q_out = out;
  a.q_b = qs[0]; a.q_n = qs[1]; a.q_h = qs[2];
  a.o_b = os[0]; a.o_n = os[1]; a.o_h = os[2];
  return REST_OK;
}

rest_status append(void* d_k_pages, void* d_v_pages, const int64_t* page_strides, float* d_k_scales, float* d_v_scales, int32_t P,
                   int32_t page, const int32_t* d_table, int64_t table_stride, int32_t table_cols, const int32_t* d_kv_len,
                   const void* d_k_new, const void* d_v_new, const int64_t* new_strides, const int32_t* d_n_nodes, int32_t dtype,
                   const int32_t* d_pos, const float* d_inv_freq, int32_t pairs, int32_t interleaved, float amplitude,
                   const void* d_q, const int64_t* q_strides, void* d_q_out, const int64_t* out_strides, int32_t H, int32_t B,
                   int32_t H_kv, int32_t N, int32_t D, bool scaled, void* stream) {
  if (B < 0 || H_kv < 1 || N < 0 || H < 0 || !new_strides || (dtype != REST_BF16 && dtype != REST_FP16)) return REST_INVALID_ARG;
  if (B == 0 || N == 0) return REST_OK;
  if (!d_kv_len || !d_k_new || !d_v_new || !table_ok(d_table, table_stride, table_cols)) return REST_INVALID_ARG;
  if (scaled && (!d_k_scales || !d_v_scales)) return REST_INVALID_ARG;
  Args a = {};
  if (rest_status st = fill_pool(a.c, d_k_pages, d_v_pages, page_strides, d_table, table_stride, table_cols, P, H_kv, page, D,
                                 scaled ? 16 : 8))
    return st;
  if (H > 65536 || H_kv > 65536 || N > kMostRows) return REST_UNSUPPORTED;
  if (rest_status st = fill_turn(a, d_pos, d_inv_freq, pairs, interleaved, amplitude, D)) return st;
  if (!rows_ok(new_strides, B, N, H_kv, D, 8) || !aligned16(d_k_new, d_v_new)) return REST_INVALID_ARG;
  if (H > 0)
    if (rest_status st = fill_q(a, d_q, q_strides, d_q_out, out_strides, B, N, H, 8)) return st;
  a.k_scales = d_k_scales; a.v_scales = d_v_scales;
  a.k_new = d_k_new; a.v_new = d_v_new;
  a.n_b = new_strides[0]; a.n_n = new_strides[1]; a.n_h = new_strides[2];
  a.kv_len = d_kv_len; a.n_nodes = d_n_nodes;
  a.N = N; a.H = H; a.H_kv = H_kv;
  a.groups = (N + 30) / 16;                             // blocks of 16 rows that N rows can touch
  const bool bf16 = dtype == REST_BF16;
  if (!scaled) return bf16 ? run<__nv_bfloat16, kPages16, 0>(a, B, stream) : run<__half, kPages16, 0>(a, B, stream);
  if (D == 128)
    return bf16 ? run<__nv_bfloat16, kPagesScaled, 128>(a, B, stream) : run<__half, kPagesScaled, 128>(a, B, stream);
  return bf16 ? run<__nv_bfloat16, kPagesScaled, 64>(a, B, stream) : run<__half, kPagesScaled, 64>(a, B, stream);
}

}  // namespace

extern "C" rest_status rest_rotary(const void* d_x, const int64_t* x_strides, int32_t dtype, const int32_t* d_pos,
                                   const float* d_inv_freq, int32_t pairs, int32_t interleaved, float amplitude,
                                   const int32_t* d_n_nodes, int32_t B, int32_t H, int32_t N, int32_t D, void* d_out,
                                   const int64_t* out_strides, void* stream) {
  if (B < 0 || H < 1 || N < 0 || D < 1 || (dtype != REST_BF16 && dtype != REST_FP16 && dtype != REST_FP32)) return REST_INVALID_ARG;
  if (B == 0 || N == 0) return REST_OK;
  if (D > 512 || (D % 16) != 0 || H > 65536 || N > kMostRows) return REST_UNSUPPORTED;
  Args a = {};
  if (rest_status st = fill_turn(a, d_pos, d_inv_freq, pairs, interleaved, amplitude, D)) return st;
  if (rest_status st = fill_q(a, d_x, x_strides, d_out, out_strides, B, N, H, dtype == REST_FP32 ? 4 : 8)) return st;
  a.n_nodes = d_n_nodes;
  a.N = N; a.H = H;
  a.groups = (N + 15) / 16;
  if (dtype == REST_FP32) return run<float, kNowhere, 0>(a, B, stream);
  return dtype == REST_BF16 ? run<__nv_bfloat16, kNowhere, 0>(a, B, stream) : run<__half, kNowhere, 0>(a, B, stream);
}

extern "C" rest_status rest_paged_kv_append(void* d_k_pages, void* d_v_pages, const int64_t* page_strides, int32_t P,
                                            int32_t page, const int32_t* d_table, int64_t table_stride, int32_t table_cols,
                                            const int32_t* d_kv_len, const void* d_k_new, const void* d_v_new,
                                            const int64_t* new_strides, const int32_t* d_n_nodes, int32_t dtype,
                                            const int32_t* d_pos, const float* d_inv_freq, int32_t pairs, int32_t interleaved,
                                            float amplitude, const void* d_q, const int64_t* q_strides, void* d_q_out,
                                            const int64_t* out_strides, int32_t H, int32_t B, int32_t H_kv, int32_t N,
                                            int32_t D, void* stream) {
  return append(d_k_pages, d_v_pages, page_strides, nullptr, nullptr, P, page, d_table, table_stride, table_cols, d_kv_len,
                d_k_new, d_v_new, new_strides, d_n_nodes, dtype, d_pos, d_inv_freq, pairs, interleaved, amplitude, d_q,
                q_strides, d_q_out, out_strides, H, B, H_kv, N, D, false, stream);
}

extern "C" rest_status rest_paged_kv_append_scaled(void* d_k_pages, void* d_v_pages, const int64_t* page_strides,
                                                   float* d_k_scales, float* d_v_scales, int32_t P, int32_t page,
                                                   const int32_t* d_table, int64_t table_stride, int32_t table_cols,
                                                   const int32_t* d_kv_len, const void* d_k_new, const void* d_v_new,
                                                   const int64_t* new_strides, const int32_t* d_n_nodes, int32_t dtype,
                                                   const int32_t* d_pos, const float* d_inv_freq, int32_t pairs,
                                                   int32_t interleaved, float amplitude, const void* d_q,
                                                   const int64_t* q_strides, void* d_q_out, const int64_t* out_strides,
                                                   int32_t H, int32_t B, int32_t H_kv, int32_t N, int32_t D, void* stream) {
  return append(d_k_pages, d_v_pages, page_strides, d_k_scales, d_v_scales, P, page, d_table, table_stride, table_cols, d_kv_len,
                d_k_new, d_v_new, new_strides, d_n_nodes, dtype, d_pos, d_inv_freq, pairs, interleaved, amplitude, d_q,
                q_strides, d_q_out, out_strides, H, B, H_kv, N, D, true, stream);
}
