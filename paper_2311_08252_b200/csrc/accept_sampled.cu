// rest_accept_sampled: draft acceptance against the verifier's probabilities (Sec. 4.1 "Sampling
// strategies": temperature, nucleus).
//
// One block works on one row of logits at a time and says where a walk that reaches that row goes:
// to a child, or to an end with a drawn token.  Its steps:
//   1. the row's largest logit;
//   2. every token's weight, kept in shared memory (rows beyond 51200 tokens: computed again whenever it is
//      looked at), their sum, and the sums of bins of a sixteenth of an octave - for tokens heavy enough to
//      be in the nucleus: those below (1 - top_p) / V of the largest are not, whatever else the row holds;
//   3. with a nucleus: the bin in which the running sum reaches its target; the tokens of that bin (some
//      hundred) are ordered against one another;
//   4. the children of the row's node in index order;
//   5. if none is accepted: the drawn token, by sums over the tokens in order.
// A weight is a float that holds a whole number of 2^-44 of the largest, so all sums are sums of integers:
// exact, and the same for any order of addition and any number of threads.  It is off by 2^-24 of itself,
// either way alike: plain 32-bit arithmetic (the product of a far logit and 1 / temperature alone: 1e-6)
// would move the borders between tokens often enough to be seen in a large batch.
//
// A walk visits 1 + accepted rows of N + 1.  Either one block per context walks, a row after the
// other, reading only those rows; or, when the rows of all contexts are few enough to run at once,
// every row gets a block of its own and a second small kernel follows the outcomes.  Bound: instructions
// (about 35 a token for the weights, more time than the row's bytes take), and a walk is a chain of rows.
// Measured (B200, vocabulary 32000, temperature 0.8, top_p 0.95): one context, 65 rows of bf16, a block each,
// 30 us with the second kernel; 128 contexts, fp32, a block walks each, 115 to 130 us (the longest walk decides).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "common.cuh"
#include "rest.h"

namespace {

typedef unsigned long long u64;
constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr uint32_t kOneBits = 0x55800000u;      // 2^44 as a float: the weight of a row's largest logit
constexpr int kBins = 16 * 46;                  // 16 to an octave, from [2^44, 2^45) down
constexpr int kList = 512;                      // tokens of one bin that are ordered pairwise
constexpr int kKeptTokens = 51200;              // rows whose weights stay in shared memory (200 KB)

struct Args {
  const void* logits;
  int64_t s_ctx, s_row;
  const int32_t *tokens, *parents, *n_nodes;
  const float *uniforms, *temperature, *top_p;
  int32_t *accept_len, *accept_nodes, *out_tokens;
  int2* outcome;                                // [B][N + 1] {child or -1, token} when every row has a block
  int V, N, max_depth;
};

__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// order-preserving integer of a logit (-0 counts as 0); NaN and -infinity are 0 (impossible)
__device__ __forceinline__ uint32_t key_of(float x) {
  if (!(x > -INFINITY)) return 0u;
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) {
  return k == 0 ? -INFINITY : __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}

struct Shared {
  float2 pow16[16];                             // 2^(44 + j/16) as a float and what it leaves
  u64 sum[32], left, above, over, seg_before, cut, cut_mass;   // (a warp looks at all 32: those of no warp stay as they began)
  ulonglong2 list[kList];                       // {order: key, then ~index; weight}
  uint32_t bin_lo[kBins], bin_hi[kBins];        // sums of the low and high 12 bits of the weights' mantissas
  uint32_t red[32], red2[32];
  int32_t tok[REST_MAX_N], par[REST_MAX_N];
  int cut_tie, bin, n_list, child, n_refused, refused[REST_MAX_N], token, seg;
};

// A row's scale: 16 log2 of a token's weight = (x - top) * c16, with c16 as a sum of two floats (held
// below 1e30, where any two different logits are worlds apart); differences beyond `least` weigh nothing.
// Rows of greedy walks and rows with an infinite logit (flat): the largest weigh 1, all others 0.
struct Row {
  float top, c16_hi, c16_lo, least;
  bool flat;
};

// The weight of logit x: 2^44 2^((x - top) c16 / 16), rounded to 24 bits and to a whole number; no
// branches.  With y the product, k its nearest integer and f the rest: a table gives 2^(j/16), j = k % 16,
// q = 2^(f/16) - 1 comes from its Taylor series (|q| < 0.022, the fifth power is 4e-11), k / 16 goes into
// the exponent.  y is kept to 48 bits (its rounding error, the low half of c16, for fp32 logits the
// rounding of the difference too): f is off by some 1e-8, where a plain product of a far logit would be
// off by 4e-5.  32-bit arithmetic throughout: 64-bit instructions issue at half the rate.
template <typename T>
__device__ __forceinline__ float smooth_weight(const Shared& sh, const Row& r, float x) {
  constexpr float kMagic = 12582912.f;          // 1.5 * 2^23: adding it rounds to an integer
  constexpr double l = 0.6931471805599453 / 16.0;
  constexpr float a1 = (float)l, a2 = (float)(l * l / 2), a3 = (float)(l * l * l / 6), a4 = (float)(l * l * l * l / 24);
  const float raw = __fsub_rn(x, r.top), d = fmaxf(raw, r.least), y = __fmul_rn(d, r.c16_hi);   // NaN: least
  float rest = fmaf(d, r.c16_lo, fmaf(d, r.c16_hi, -y));
  if (sizeof(T) == 4) {
    const float b = __fsub_rn(raw, x), e = __fsub_rn(__fsub_rn(x, __fsub_rn(raw, b)), __fadd_rn(r.top, b));
    rest = fmaf(raw > r.least ? e : 0.f, r.c16_hi, rest);
  }
  const float t = __fadd_rn(y, kMagic), f = __fadd_rn(__fsub_rn(y, __fsub_rn(t, kMagic)), rest);
  const float q = f * fmaf(f, fmaf(f, fmaf(f, a4, a3), a2), a1);
  const uint32_t k = __float_as_uint(t);        // (the magic's low bits are 0)
  const float2 p = sh.pow16[k & 15u];
  const float w = __uint_as_float(__float_as_uint(__fadd_rn(p.x, fmaf(p.x, q, p.y))) + ((k & ~15u) << 19));
  const float whole = __fsub_rn(__fadd_rn(w, 8388608.f), 8388608.f);       // below 2^23: rounds to a whole number
  return w < 8388608.f ? whole : w;
}
__device__ __forceinline__ u64 whole(float w) {            // a weight as an integer
  const uint32_t b = __float_as_uint(w);
  const int e = (int)(b >> 23) - 150;
  const u64 m = (b & 0x7FFFFFu) | 0x800000u;
  return b == 0u ? 0ull : e >= 0 ? m << e : m >> -e;
}
template <typename T>
__device__ __forceinline__ float weight(const Shared& sh, const Row& r, float x) {
  return r.flat ? (x == r.top ? __uint_as_float(kOneBits) : 0.f) : smooth_weight<T>(sh, r, x);
}
// Sum of weights in two 32-bit integers: units of 2^22 (rounded; 512 of 2^22 at most a thread) and the rest,
// both read off the low bits of a float to which 2^23 or 1.5 * 2^23 was added.
struct Sum {
  uint32_t high = 0, low = 0;
  __device__ __forceinline__ void add(float w) {
    const float t = fmaf(w, 0x1p-22f, 8388608.f), rest = fmaf(__fsub_rn(t, 8388608.f), -0x1p22f, w);
    high += __float_as_uint(t) - 0x4B000000u;
    low += __float_as_uint(__fadd_rn(rest, 12582912.f)) - 0x4B400000u;
  }
  __device__ __forceinline__ u64 total() const { return ((u64)high << 22) + (u64)(long long)(int)low; }
};
// How far apart the weights of two tokens may be for the one with the larger logit to have the smaller
// weight: before they are rounded, weights are off by less than 5e-9 of themselves (the series' products,
// 2^-24 of |q| < 0.022, and the table), so after it by one step of 2^-23 more, or by one whole number where
// that is more.  Here 16 steps.
__device__ __forceinline__ float slack_of(float w) { return fmaf(w, 0x1p-19f, 1.f); }
__device__ __forceinline__ int bin_of(float w) { return (int)((kOneBits + 0x7FFFFFu - __float_as_uint(w)) >> 19); }

__device__ __forceinline__ u64 warp_sum(u64 x) {
#pragma unroll
  for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
  return x;
}
__device__ __forceinline__ u64 warp_scan(u64 x) {     // inclusive
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const u64 y = __shfl_up_sync(0xFFFFFFFFu, x, d);
    if ((int)(threadIdx.x & 31) >= d) x += y;
  }
  return x;
}
__device__ __forceinline__ u64 block_sum(Shared& sh, u64 x) {
  x = warp_sum(x);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh.sum[threadIdx.x >> 5] = x;
  __syncthreads();
  return warp_sum(sh.sum[threadIdx.x & 31]);
}
// inclusive prefix sum over the block's threads
__device__ __forceinline__ u64 block_scan(Shared& sh, u64 x) {
  x = warp_scan(x);
  __syncthreads();
  if ((threadIdx.x & 31) == 31) sh.sum[threadIdx.x >> 5] = x;
  __syncthreads();
  const u64 upto = warp_scan(sh.sum[threadIdx.x & 31]);
  const int warp = threadIdx.x >> 5;
  const u64 before = __shfl_sync(0xFFFFFFFFu, upto, warp ? warp - 1 : 0);
  return x + (warp ? before : 0);
}
__device__ __forceinline__ double uniform(const float* u, int s) {
  return u[s] > 0.f ? (double)fminf(u[s], 0.99999994f) : 0.0;
}

// The outcome of row `cur` (-1: the root's) of context b: an accepted child, or -1 and the drawn token
// (-1: nothing can be drawn).  depth: nodes accepted on the way, -1: to be counted here; a walk that is as
// deep as allowed only draws.
template <typename T, bool KEPT>
__device__ int2 row_outcome(const Args& a, Shared& sh, float* s_w, int b, int cur, int depth) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int nn = min(max(a.n_nodes[b], 0), a.N);
  const float* uni = a.uniforms + (int64_t)b * (a.N + 1);
  const float temp = a.temperature[b], top_p = a.top_p[b];
  const T* row = static_cast<const T*>(a.logits) + b * a.s_ctx + (int64_t)(cur + 1) * a.s_row;
  const int V = a.V;
  // The row is read in 16-byte vectors; positions before and behind it in its first and last vector hold
  // -infinity.  KEPT: weights stand in shared memory by position; otherwise that memory is one bit per
  // token: refused at this node.
  constexpr int kPer = 16 / sizeof(T);
  const int shift = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
  const int vecs = (shift + V + kPer - 1) / kPer;
  const uint4* src = reinterpret_cast<const uint4*>(row - shift);
  uint32_t* s_gone = reinterpret_cast<uint32_t*>(s_w);
  auto load = [&](int i) -> uint4 {                       // whole vectors inside the row; its ends one by one
    if (i * kPer >= shift && (i + 1) * kPer <= shift + V) return __ldg(src + i);
    uint4 x;
    T* e = reinterpret_cast<T*>(&x);
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int v = i * kPer + k - shift;
      e[k] = v >= 0 && v < V ? row[v] : (T)(-INFINITY);
    }
    return x;
  };

  // ---- 1. the largest logit; the tree
  float most = -INFINITY;
  __syncthreads();                              // the row before it is done with
  for (int i = tid; i < a.N; i += kThreads) {
    sh.tok[i] = a.tokens[(int64_t)b * a.N + i];
    sh.par[i] = a.parents[(int64_t)b * a.N + i];
  }
  for (int i0 = tid; i0 < vecs; i0 += 8 * kThreads) {
    uint4 x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (i0 + j * kThreads < vecs) x[j] = load(i0 + j * kThreads);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (i0 + j * kThreads < vecs) {
        const T* e = reinterpret_cast<const T*>(&x[j]);
#pragma unroll
        for (int k = 0; k < kPer; ++k) most = fmaxf(most, (float)e[k]);    // (passes NaN over)
      }
  }
  if (!KEPT)
    for (int w = tid; w < (V + 31) / 32; w += kThreads) s_gone[w] = 0u;
  for (int i = tid; i < kBins; i += kThreads) sh.bin_lo[i] = sh.bin_hi[i] = 0u;
  uint32_t top = __reduce_max_sync(0xFFFFFFFFu, key_of(most));
  if (lane == 0) sh.red[warp] = top;
  if (tid == 0) { sh.cut_tie = 0x7FFFFFFF; sh.bin = -1; sh.n_list = 0; sh.over = 0ull; }
  __syncthreads();
  top = __reduce_max_sync(0xFFFFFFFFu, sh.red[lane]);
  if (top == 0) return make_int2(-1, -1);
  Row r;
  r.top = of_key(top);
  const bool greedy = !(temp > 0.f);
  r.flat = greedy || r.top == INFINITY;
  const double c16 = r.flat ? 1.0 : 16.0 * 1.4426950408889634 / fmax((double)fminf(temp, 1e30f), 1e-29);
  r.c16_hi = (float)c16;
  r.c16_lo = (float)(c16 - (double)r.c16_hi);
  r.least = (float)(-760.0 / c16);              // 2^-47.5: rounds to nothing

  // ---- 2. weights, their sum, and the bins' if there will be a cut
  const bool cut = greedy || top_p < 1.f;
  // the lightest weight that can be in the nucleus, and a little less
  const float lightest = cut ? (!greedy && top_p > 0.f ? fmaxf((1.f - top_p) / (float)V * 1.5e13f, 1.f) : __uint_as_float(kOneBits)) : INFINITY;
  Sum all;
  uint4 next = tid < vecs ? load(tid) : make_uint4(0u, 0u, 0u, 0u);
  for (int i = tid; i < vecs; i += kThreads) {
    const uint4 x = next;
    if (i + kThreads < vecs) next = load(i + kThreads);
    const T* e = reinterpret_cast<const T*>(&x);
    float w[kPer];
    if (r.flat) {
#pragma unroll
      for (int k = 0; k < kPer; ++k) w[k] = (float)e[k] == r.top ? __uint_as_float(kOneBits) : 0.f;
    } else {
#pragma unroll
      for (int k = 0; k < kPer; ++k) w[k] = smooth_weight<T>(sh, r, (float)e[k]);
    }
    float heaviest = 0.f;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      all.add(w[k]);
      heaviest = fmaxf(heaviest, w[k]);
    }
    if (heaviest >= lightest) {
#pragma unroll
      for (int k = 0; k < kPer; ++k)
        if (w[k] >= lightest) {
          const uint32_t bits = __float_as_uint(w[k]);
          atomicAdd(&sh.bin_lo[bin_of(w[k])], bits & 0xFFFu);
          atomicAdd(&sh.bin_hi[bin_of(w[k])], (bits >> 12 & 0x7FFu) | 0x800u);
        }
    }
    if (KEPT) {
#pragma unroll
      for (int k = 0; k < kPer; k += 4)
        *reinterpret_cast<float4*>(s_w + i * kPer + k) = make_float4(w[k], w[k + 1], w[k + 2], w[k + 3]);
    }
  }
  u64 mass = block_sum(sh, all.total());        // (its barriers put the weights and the bins in place, too)

  auto weight_at = [&](int v) -> float { return KEPT ? s_w[shift + v] : weight<T>(sh, r, (float)row[v]); };
  // fn(token, its weight and those of the three after it) for the positions' fours [from, to), `step` apart
  auto each = [&](int from, int to, int step, auto fn) {
#pragma unroll 2
    for (int i = from; i < to; i += step) {
      float w[4];
      if (KEPT) {
        const float4 x = *reinterpret_cast<const float4*>(s_w + i * 4);
        w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int v = i * 4 + k - shift;
          w[k] = v >= 0 && v < V ? weight_at(v) : 0.f;
        }
      }
      fn(i * 4 - shift, w);
    }
  };
  const int fours = (shift + V + 3) / 4;

  // ---- 3. the nucleus: the tokens from (cut_key, cut_tie) up: those of weight above cut_w, and of those at
  // cut_w the ones that their logits put there.  Rounding may give the smaller of two logits that are next to
  // one another the larger weight; where it did so to the cut (rare), logits decide for all weights near cut_w
  // (see slack_of).  (Always deciding so took 8 % more for 128 rows of 32000 fp32 logits.)
  float cut_w = 0.f;
  bool turned = false;
  uint32_t cut_key = 0;
  int cut_tie = 0x7FFFFFFF;
  if (cut) {
    u64 target = 1;
    if (!greedy && top_p > 0.f) target = max((u64)1, (u64)ceil((double)top_p * (double)mass));
    {
      static_assert(2 * kThreads >= kBins, "two bins a thread");
      auto bin_mass = [&](int i) -> u64 {
        if (i >= kBins) return 0ull;
        const int e = 44 - 23 - (i >> 4);                 // what the bin's mantissas of 24 bits count
        const u64 m = (u64)sh.bin_lo[i] + ((u64)sh.bin_hi[i] << 12);
        return e >= 0 ? m << e : m >> -e;
      };
      const u64 m0 = bin_mass(2 * tid), m1 = bin_mass(2 * tid + 1);
      const u64 upto = block_scan(sh, m0 + m1);
      if (upto >= target && upto - m0 - m1 < target) {
        const bool second = upto - m1 < target;
        sh.bin = 2 * tid + second;
        sh.above = upto - m1 - (second ? 0ull : m0);
      }
      __syncthreads();
    }
    // fn(token, weight) for the tokens of the bin (weights in [low, high)) and for those that may be in
    // another one by rounding alone: any token above them all has a larger logit than any in the bin, any
    // below a smaller one
    const uint32_t low_bits = kOneBits + 0x780000u - ((uint32_t)sh.bin << 19);
    const float low = __uint_as_float(low_bits), high = __uint_as_float(low_bits + 0x80000u);
    const uint32_t first = __float_as_uint(fmaxf(low - slack_of(low), 1.f)), width = __float_as_uint(high + slack_of(high)) - first;
    auto in_bin = [&](auto fn) {
      each(tid, fours, kThreads, [&](int v, const float (&w)[4]) {
        bool is[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) is[k] = __float_as_uint(w[k]) - first < width;
        if (is[0] || is[1] || is[2] || is[3]) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (is[k]) fn(v + k, w[k]);
        }
      });
    };
    in_bin([&](int v, float w) {
      const int at = atomicAdd(&sh.n_list, 1);
      if (at < kList) sh.list[at] = make_ulonglong2((u64)key_of((float)row[v]) << 32 | (uint32_t)~v, whole(w));
      if (w >= high) atomicAdd(&sh.over, whole(w));
    });
    __syncthreads();
    const int n = sh.n_list;
    const u64 above = sh.above - sh.over;       // mass of the tokens that are above all of these
    if (n <= kList) {
      // the mass before each token of the bin; several lanes share a token when there are few
      int parts = 1;
      while (parts < 32 && n * parts * 2 <= kThreads) parts *= 2;
      const int e = tid / parts, part = tid % parts;
      const ulonglong2 mine = e < n ? sh.list[e] : make_ulonglong2(~0ull, 0ull);
      u64 before = 0;
#pragma unroll 8
      for (int j = part; j < n; j += parts) {
        const ulonglong2 other = sh.list[j];
        before += other.x > mine.x ? other.y : 0ull;
      }
      for (int d = 1; d < parts; d <<= 1) before += __shfl_xor_sync(0xFFFFFFFFu, before, d);
      before += above;
      if (e < n && part == 0 && before < target && before + mine.y >= target) {
        sh.cut = mine.x;
        sh.cut_mass = mine.y;
        sh.left = before + mine.y;
      }
      __syncthreads();
      turned = __syncthreads_or(e < n && (mine.x > sh.cut ? mine.y < sh.cut_mass : mine.x < sh.cut && mine.y > sh.cut_mass));
      cut_key = (uint32_t)(sh.cut >> 32);
      cut_tie = (int)~(uint32_t)sh.cut;
      mass = sh.left;
    } else {
      // a crowd in one bin (flat rows): the largest key whose tokens and all above reach the target, by
      // bisection, then how many of its tokens stay, lowest index first
      uint32_t kmin = 0xFFFFFFFFu, kmax = 0;
      in_bin([&](int v, float) { const uint32_t k = key_of((float)row[v]); kmin = min(kmin, k); kmax = max(kmax, k); });
      kmin = __reduce_min_sync(0xFFFFFFFFu, kmin);
      kmax = __reduce_max_sync(0xFFFFFFFFu, kmax);
      __syncthreads();
      if (lane == 0) { sh.red[warp] = kmin; sh.red2[warp] = kmax; }
      __syncthreads();
      uint32_t lo = __reduce_min_sync(0xFFFFFFFFu, lane < kWarps ? sh.red[lane] : 0xFFFFFFFFu), hi = __reduce_max_sync(0xFFFFFFFFu, sh.red2[lane]);
      auto mass_from = [&](uint32_t key) -> u64 {         // of the bin's tokens with that key and above
        Sum part;
        in_bin([&](int v, float w) { if (key_of((float)row[v]) >= key) part.add(w); });
        return block_sum(sh, part.total());
      };
      while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2 + 1;
        if (above + mass_from(mid) >= target) lo = mid; else hi = mid - 1;
      }
      cut_key = lo;
      const u64 over = lo == 0xFFFFFFFFu ? 0ull : mass_from(lo + 1);
      const u64 one = whole(weight<T>(sh, r, of_key(lo))), ties = (target - above - over + one - 1) / one;
      // every warp counts in a run of its own; the warp whose run holds the last one finds it
      const int per = (V + kThreads - 1) / kThreads * 32, v0 = min(V, warp * per), v1 = min(V, v0 + per);
      u64 count = 0;
      for (int v = v0 + lane; v < v1; v += 32) count += key_of((float)row[v]) == lo;
      count = warp_sum(count);
      __syncthreads();
      if (lane == 0) sh.sum[warp] = count;
      __syncthreads();
      const u64 counts = warp_scan(sh.sum[lane]);
      const u64 upto = __shfl_sync(0xFFFFFFFFu, counts, warp);
      if (upto >= ties && upto - count < ties) {          // (one warp)
        u64 seen = upto - count;
        for (int base = v0; base < v1; base += 32) {
          const bool is = base + lane < v1 && key_of((float)row[base + lane]) == lo;
          const unsigned bal = __ballot_sync(0xFFFFFFFFu, is);
          if (seen + __popc(bal) >= ties) {
            if (is && seen + __popc(bal & ((2u << lane) - 1u)) == ties) sh.cut_tie = base + lane;
            break;
          }
          seen += __popc(bal);
        }
      }
      __syncthreads();
      cut_tie = sh.cut_tie;
      mass = above + over + ties * one;
      turned = true;                            // (nobody looked)
    }
    cut_w = weight<T>(sh, r, of_key(cut_key));
  }
  auto kept = [&](int v, float w) -> bool {
    if (w != cut_w && !(turned && fabsf(w - cut_w) <= slack_of(cut_w))) return w > cut_w;
    if (!cut) return false;                     // (weight 0)
    const uint32_t key = key_of((float)row[v]);
    return key > cut_key || (key == cut_key && v <= cut_tie);
  };

  // ---- 4. children, in index order
  if (warp == 0) {
    int child = -1, n_refused = 0;
    u64 left = mass;
    if (depth < 0) {                            // (as far as it matters; no walk gets to deeper rows)
      depth = 0;
      for (int i = cur; i >= 0 && i < a.N && depth <= a.max_depth; i = sh.par[i]) ++depth;
    }
    const bool children = depth < a.max_depth;
    for (int base = 0; children && base < nn && child < 0; base += 32) {
      const int i = base + lane;
      const bool is = i < nn && sh.par[i] == cur;
      const int t = is ? sh.tok[i] : -1;
      u64 w = 0;
      double u = 0.0;
      if (is && t >= 0 && t < V) {
        const float x = weight_at(t);
        w = kept(t, x) ? whole(x) : 0ull;
        u = uniform(uni, i + 1);
        for (int j = 0; j < n_refused; ++j)
          if (sh.refused[j] == t) w = 0;
      }
      unsigned todo = __ballot_sync(0xFFFFFFFFu, w != 0);
      while (todo) {
        const int l = __ffs(todo) - 1;
        todo &= todo - 1;
        const u64 wl = __shfl_sync(0xFFFFFFFFu, w, l);
        const double ul = __shfl_sync(0xFFFFFFFFu, u, l);
        const int tl = __shfl_sync(0xFFFFFFFFu, t, l);
        if (wl == 0) continue;                  // its token was refused before
        if (ul * (double)left < (double)wl) { child = base + l; break; }
        left -= wl;
        if (lane == 0) sh.refused[n_refused] = tl;
        __syncwarp();
        ++n_refused;
        if (t == tl) w = 0;
      }
    }
    if (lane == 0) { sh.child = child; sh.left = left; sh.n_refused = n_refused; sh.token = -1; sh.seg = kWarps - 1; sh.seg_before = 0; }
  }
  __syncthreads();
  if (sh.child >= 0) return make_int2(sh.child, sh.tok[sh.child]);

  // ---- 5. the drawn token, from what the refused children leave: first the 1/16 of the row that holds
  // it (a warp's share), then the token in it
  for (int j = tid; j < sh.n_refused; j += kThreads) {
    if (KEPT) s_w[shift + sh.refused[j]] = 0.f;
    else atomicOr(&s_gone[sh.refused[j] >> 5], 1u << (sh.refused[j] & 31));
  }
  __syncthreads();
  auto there = [&](int v, float w) -> bool {
    if (!KEPT && w > 0.f && ((s_gone[v >> 5] >> (v & 31)) & 1u)) return false;
    return kept(v, w);
  };
  const int per = (fours + kWarps - 1) / kWarps, f0 = min(fours, warp * per), f1 = min(fours, f0 + per);
  Sum part;
  each(f0 + lane, f1, 32, [&](int v, const float (&w)[4]) {
    bool tie = false;
#pragma unroll
    for (int k = 0; k < 4; ++k) tie = tie || w[k] == cut_w;
    if (KEPT && !turned && (!tie || !cut)) {                          // nobody needs a closer look
#pragma unroll
      for (int k = 0; k < 4; ++k) part.add(w[k] > cut_w ? w[k] : 0.f);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) part.add(w[k] > 0.f && there(v + k, w[k]) ? w[k] : 0.f);
    }
  });
  const u64 sum = warp_sum(part.total());
  if (lane == 0) sh.sum[warp] = sum;
  __syncthreads();
  const double goal = uniform(uni, 0) * (double)sh.left;
  if (warp == 0) {
    const u64 mine = sh.sum[lane], upto = warp_scan(mine);
    if ((double)upto > goal && !((double)(upto - mine) > goal)) { sh.seg = lane; sh.seg_before = upto - mine; }
  }
  __syncthreads();
  const int g0 = min(fours, sh.seg * per), g1 = min(fours, g0 + per);
  const int s0 = max(g0 * 4 - shift, 0), s1 = min(V, g1 * 4 - shift);
  u64 before = sh.seg_before;
  for (int base = s0; base < s1; base += kThreads) {      // (more than one round for more than 8192 tokens)
    const int v = base + tid;
    const float w = v < s1 ? weight_at(v) : 0.f;
    const u64 mine = v < s1 && there(v, w) ? whole(w) : 0ull;
    const u64 upto = before + block_scan(sh, mine);
    if ((double)upto > goal && !((double)(upto - mine) > goal)) sh.token = v;
    if (tid == kThreads - 1) sh.above = upto;
    __syncthreads();
    before = sh.above;
  }
  return make_int2(-1, sh.token);
}

__device__ __forceinline__ void fill_table(Shared& sh) {
  if (threadIdx.x < 32) { sh.sum[threadIdx.x] = 0ull; sh.red[threadIdx.x] = 0u; sh.red2[threadIdx.x] = 0u; }
  if (threadIdx.x < 16) {
    const double p = exp2(44.0 + (double)threadIdx.x / 16.0);
    const float hi = (float)p;
    sh.pow16[threadIdx.x] = make_float2(hi, (float)(p - (double)hi));
  }
}

// One block per context walks.
template <typename T, bool KEPT>
__global__ void __launch_bounds__(kThreads, 1) rest_accept_sampled_walk_kernel(const __grid_constant__ Args a) {
  extern __shared__ __align__(16) float s_w[];
  __shared__ Shared sh;
  fill_table(sh);
  grid_wait();
  const int b = blockIdx.x, tid = threadIdx.x;
  int32_t *an = a.accept_nodes + (int64_t)b * a.max_depth, *ot = a.out_tokens + (int64_t)b * (a.max_depth + 1);
  int cur = -1, len = 0;
  for (;;) {
    const int2 o = row_outcome<T, KEPT>(a, sh, s_w, b, cur, len);
    if (tid == 0) ot[len] = o.y;
    if (o.x < 0) break;
    if (tid == 0) an[len] = o.x;
    cur = o.x;
    ++len;
  }
  if (tid == 0) a.accept_len[b] = len;
  for (int d = len + tid; d < a.max_depth; d += kThreads) { an[d] = -1; ot[d + 1] = -1; }
}

// Every row has a block; blockIdx.x = row, blockIdx.y = context.
template <typename T, bool KEPT>
__global__ void __launch_bounds__(kThreads, 1) rest_accept_sampled_rows_kernel(const __grid_constant__ Args a) {
  extern __shared__ __align__(16) float s_w[];
  __shared__ Shared sh;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  fill_table(sh);
  grid_wait();
  const int b = blockIdx.y, cur = (int)blockIdx.x - 1, tid = threadIdx.x;
  if (cur >= min(max(a.n_nodes[b], 0), a.N)) return;
  const int2 o = row_outcome<T, KEPT>(a, sh, s_w, b, cur, -1);
  if (tid == 0) a.outcome[(int64_t)b * (a.N + 1) + cur + 1] = o;
}

__global__ void __launch_bounds__(128) rest_accept_sampled_follow_kernel(const __grid_constant__ Args a) {
  __shared__ int2 s[REST_MAX_N + 1];
  grid_wait();
  const int b = blockIdx.x, tid = threadIdx.x;
  const int rows = min(max(a.n_nodes[b], 0), a.N) + 1;
  for (int i = tid; i < rows; i += 128) s[i] = a.outcome[(int64_t)b * (a.N + 1) + i];
  __syncthreads();
  int32_t *an = a.accept_nodes + (int64_t)b * a.max_depth, *ot = a.out_tokens + (int64_t)b * (a.max_depth + 1);
  int cur = -1, len = 0;
  for (;;) {                                    // every thread walks; a row at full depth has no child
    const int2 o = s[cur + 1];
    if (tid == 0) ot[len] = o.y;
    if (o.x < 0 || len == a.max_depth) break;
    if (tid == 0) an[len] = o.x;
    cur = o.x;
    ++len;
  }
  if (tid == 0) a.accept_len[b] = len;
  for (int d = len + tid; d < a.max_depth; d += 128) { an[d] = -1; ot[d + 1] = -1; }
}

// Every row of its own block pays when all of them run in about two rounds of one block an SM: a walk
// is rarely shorter than three rows, one after the other.
bool every_row(int B, int N) {
  const int sms = rest::sm_count();
  return (int64_t)B * (N + 1) <= 2 * (sms > 0 ? sms : 148);
}

template <typename T, bool KEPT>
rest_status run(const Args& a, int B, size_t smem, int smem_slot, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (a.outcome) {
    REST_CUDA_TRY(rest::ensure_dynamic_smem(reinterpret_cast<const void*>(rest_accept_sampled_rows_kernel<T, KEPT>), smem_slot, smem));
    cfg.gridDim = dim3((unsigned)(a.N + 1), (unsigned)B, 1);
    REST_CUDA_TRY(cudaLaunchKernelEx(&cfg, rest_accept_sampled_rows_kernel<T, KEPT>, a));
    rest::count_launch();
    cfg.gridDim = dim3((unsigned)B, 1, 1);
    cfg.blockDim = dim3(128, 1, 1);
    cfg.dynamicSmemBytes = 0;
    REST_CUDA_TRY(cudaLaunchKernelEx(&cfg, rest_accept_sampled_follow_kernel, a));
  } else {
    REST_CUDA_TRY(rest::ensure_dynamic_smem(reinterpret_cast<const void*>(rest_accept_sampled_walk_kernel<T, KEPT>), smem_slot + 1, smem));
    cfg.gridDim = dim3((unsigned)B, 1, 1);
    REST_CUDA_TRY(cudaLaunchKernelEx(&cfg, rest_accept_sampled_walk_kernel<T, KEPT>, a));
  }
  rest::count_launch();
  return REST_OK;
}

template <typename T>
rest_status pick(const Args& a, int B, int smem_slot, cudaStream_t st) {
  if (a.V <= kKeptTokens) return run<T, true>(a, B, ((size_t)a.V + 16) * sizeof(float), smem_slot, st);   // and its ends
  return run<T, false>(a, B, 4 * (((size_t)a.V + 31) / 32), smem_slot + 2, st);
}

}  // namespace

extern "C" size_t rest_accept_sampled_workspace_bytes(int32_t B, int32_t N) {
  if (B <= 0 || N <= 0 || N > REST_MAX_N) return 0;
  return every_row(B, N) ? sizeof(int2) * (size_t)B * (N + 1) : 0;
}

extern "C" rest_status rest_accept_sampled(const void* d_logits, int32_t dtype, int64_t ctx_stride, int64_t row_stride,
                                           int32_t V, const int32_t* d_tokens, const int32_t* d_parents,
                                           const int32_t* d_n_nodes, const float* d_uniforms,
                                           const float* d_temperature, const float* d_top_p, int32_t B, int32_t N,
                                           int32_t max_depth, int32_t* d_accept_len, int32_t* d_accept_nodes,
                                           int32_t* d_out_tokens, void* d_ws, size_t ws_bytes, void* stream) {
  if (B < 0 || N < 1 || max_depth < 1 || V < 1 || ctx_stride < 0 || row_stride < 0) return REST_INVALID_ARG;
  if (dtype != REST_BF16 && dtype != REST_FP16 && dtype != REST_FP32) return REST_INVALID_ARG;
  if (B == 0) return REST_OK;
  if (!d_logits || !d_tokens || !d_parents || !d_n_nodes || !d_uniforms || !d_temperature || !d_top_p ||
      !d_accept_len || !d_accept_nodes || !d_out_tokens)
    return REST_INVALID_ARG;
  if (V > REST_MAX_VOCAB_SAMPLED || max_depth > REST_MAX_M || N > REST_MAX_N) return REST_UNSUPPORTED;
  if (reinterpret_cast<uintptr_t>(d_logits) % (dtype == REST_FP32 ? 4 : 2)) return REST_INVALID_ARG;
  Args a;
  a.logits = d_logits; a.s_ctx = ctx_stride; a.s_row = row_stride;
  a.tokens = d_tokens; a.parents = d_parents; a.n_nodes = d_n_nodes;
  a.uniforms = d_uniforms; a.temperature = d_temperature; a.top_p = d_top_p;
  a.accept_len = d_accept_len; a.accept_nodes = d_accept_nodes; a.out_tokens = d_out_tokens;
  a.V = V; a.N = N; a.max_depth = max_depth;
  a.outcome = nullptr;
  // without the scratch the contexts walk: slower for few contexts, the same results
  if (every_row(B, N) && d_ws && ws_bytes >= rest_accept_sampled_workspace_bytes(B, N)) {
    if (reinterpret_cast<uintptr_t>(d_ws) & 7) return REST_INVALID_ARG;
    a.outcome = static_cast<int2*>(d_ws);
  }
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dtype == REST_BF16) return pick<__nv_bfloat16>(a, B, rest::kSmemSlotAccept, st);
  if (dtype == REST_FP16) return pick<__half>(a, B, rest::kSmemSlotAccept + 4, st);
  return pick<float>(a, B, rest::kSmemSlotAccept + 8, st);
}
