// rest_accept_sampled: draft acceptance against the verifier's probabilities (Sec. 4.1 "Sampling
// strategies": temperature, nucleus).
//
// One block works on one row of logits at a time and says where a walk that reaches that row goes:
// to a child, or to an end with a drawn token.  Its steps:
//   1. the row into shared memory (larger ones are read again from L2), and its largest logit;
//   2. every token's weight as an integer of 2^-44 of the largest (rounded to 27 bits), their sum, and
//      the sums of bins of 1/16 in log2 - for tokens heavy enough to be in the nucleus: those below
//      (1 - top_p) / V of the largest are not, whatever the rest of the row holds;
//   3. with a nucleus: the bin in which the running sum reaches its target; the tokens of that bin (some
//      hundred) are ordered against one another;
//   4. the children of the row's node in index order;
//   5. if none is accepted: the drawn token, by sums over the tokens in order.
// Integer sums are exact, so the result depends neither on the order of addition nor on the number of
// threads.  A weight is off by 2^-27 of itself at most, either way alike: plain 32-bit arithmetic (the
// product of a far logit and 1 / temperature alone: 1e-6) would move the borders between tokens often
// enough to be seen in a large batch.
//
// A walk visits 1 + accepted rows of N + 1.  Either one block per context walks, a row after the
// other, reading only those rows; or, when the rows of all contexts are few enough to run at once,
// every row gets a block of its own and a second small kernel follows the outcomes.  Bound: instructions
// (about 30 a token for the sums, more time than the row's bytes take), and a walk is a chain of rows.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "common.cuh"
#include "rest.h"

namespace {

typedef unsigned long long u64;
constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr u64 kOne = 1ull << 44;                // the weight of a row's largest logit
constexpr int kBins = 45 * 16 + 1;              // bins of 1/16 in log2, down to 2^-45
constexpr int kList = 1024;                     // tokens of one bin that are ordered pairwise
constexpr size_t kRowBytes = 200 * 1024;        // longest row kept in shared memory

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
  uint2 pow16[16];                              // 2^(26 + j/16) as a float and as an integer
  u64 sum[kWarps], left, above, seg_before, cut;
  ulonglong2 list[kList];                       // {order: key, then ~index; weight}, largest order first
  uint32_t bin_lo[kBins], bin_hi[kBins];        // sums of the low 14 and the higher bits of 27-bit weights
  uint32_t red[kWarps], red2[kWarps];
  int32_t tok[REST_MAX_N], par[REST_MAX_N];
  int cut_tie, bin, n_list, child, n_refused, refused[REST_MAX_N], token, seg;
};

// A row's scale: 16 log2 of a token's weight = (x - top) * c16, with c16 as a sum of two floats (held
// below 1e30, where any two different logits are worlds apart); differences beyond `least` weigh nothing
struct Row {
  float top, c16_hi, c16_lo, least;
  double c16;
  bool greedy, inf;
};

// log2 weight in sixteenths, rounded (monotonic in x), and the rest f, |f| <= 1/2; no branches.  The
// product is kept to 48 bits (its rounding error, the low half of c16, for fp32 logits the rounding of the
// difference too): f is off by some 1e-8, where a plain product of a far logit would be off by 4e-5.
// 32-bit arithmetic throughout: 64-bit instructions issue at half the rate.
template <typename T>
__device__ __forceinline__ void split(const Row& r, float x, int& k, float& f) {
  constexpr float kMagic = 12582912.f;          // 1.5 * 2^23: adding it rounds to an integer
  const float raw = __fsub_rn(x, r.top), d = fmaxf(raw, r.least), y = __fmul_rn(d, r.c16_hi);   // NaN: least
  float rest = fmaf(d, r.c16_lo, fmaf(d, r.c16_hi, -y));
  if (sizeof(T) == 4) {
    const float b = __fsub_rn(raw, x), e = __fsub_rn(__fsub_rn(x, __fsub_rn(raw, b)), __fadd_rn(r.top, b));
    rest = fmaf(raw > r.least ? e : 0.f, r.c16_hi, rest);
  }
  const float t = __fadd_rn(y, kMagic);
  k = __float_as_int(t) - 0x4B400000;
  f = __fadd_rn(__fsub_rn(y, __fsub_rn(t, kMagic)), rest);
}
// The weight 2^((k + f)/16) in units of 2^-44, of 27 bits at most (see up).  From a table of 2^(j/16) and
// q = 2^(f/16) - 1 by its Taylor series (|q| < 0.022, the fifth power is 4e-11): q is off by 2^-24 of
// itself, so the product of 27 bits by less than one.
__device__ __forceinline__ u64 weight_of(const Shared& sh, int k, float f) {
  constexpr double l = 0.6931471805599453 / 16.0;
  constexpr float a1 = (float)l, a2 = (float)(l * l / 2), a3 = (float)(l * l * l / 6), a4 = (float)(l * l * l * l / 24);
  const float q = f * fmaf(f, fmaf(f, fmaf(f, a4, a3), a2), a1);
  const uint2 t = sh.pow16[k & 15];
  const uint32_t m = t.y + (__float_as_uint(fmaf(__uint_as_float(t.x), q, 12582912.f)) - 0x4B400000u);
  return ((u64)m << 18) >> -(k >> 4);
}
// zero bits at the end of such a weight
__device__ __forceinline__ int up(int k) { return max(18 + (k >> 4), 0); }
// weight before the nucleus cut (see Row): an infinite logit takes all of the mass
template <typename T>
__device__ __forceinline__ u64 weight(const Shared& sh, const Row& r, float x) {
  if (r.inf || r.greedy) return x == r.top ? kOne : 0ull;
  int k;
  float f;
  split<T>(r, x, k, f);
  return weight_of(sh, k, f);
}

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
__device__ int2 row_outcome(const Args& a, Shared& sh, unsigned char* s_row, int b, int cur, int depth) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int nn = min(max(a.n_nodes[b], 0), a.N);
  const int32_t *tok = a.tokens + (int64_t)b * a.N, *par = a.parents + (int64_t)b * a.N;
  const float* uni = a.uniforms + (int64_t)b * (a.N + 1);
  const float temp = a.temperature[b], top_p = a.top_p[b];
  const T* row = static_cast<const T*>(a.logits) + b * a.s_ctx + (int64_t)(cur + 1) * a.s_row;
  const int V = a.V;
  // KEPT: the row's 16-byte vectors, at the same offset from a 16-byte border as in memory, padded with
  // -infinity on both sides.  Otherwise this memory is one bit per token: refused at this node.
  constexpr int kPer = 16 / sizeof(T);
  const int shift = KEPT ? (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T)) : 0;
  const int vecs = (shift + V + kPer - 1) / kPer;
  T* s_val = reinterpret_cast<T*>(s_row) + shift;
  uint32_t* s_gone = reinterpret_cast<uint32_t*>(s_row);
  auto get = [&](int v) -> float { return KEPT ? (float)s_val[v] : (float)row[v]; };
  // fn(token, logit) for all tokens, or for those of vectors / tokens [from, to) by this thread and those
  // `step` on
  auto each = [&](int from, int to, int step, auto fn) {
    if (KEPT) {
      for (int i = from; i < to; i += step) {
        const uint4 x = reinterpret_cast<const uint4*>(s_row)[i];
        const T* e = reinterpret_cast<const T*>(&x);
#pragma unroll
        for (int k = 0; k < kPer; ++k) fn(i * kPer + k - shift, (float)e[k]);
      }
    } else {
#pragma unroll 4
      for (int v = from; v < to; v += step) fn(v, (float)row[v]);
    }
  };
  const int units = KEPT ? vecs : V;

  // ---- 1. the row and its largest logit; the tree
  uint32_t top = 0;
  __syncthreads();                              // the row before it is done with
  for (int i = tid; i < a.N; i += kThreads) { sh.tok[i] = tok[i]; sh.par[i] = par[i]; }
  if (KEPT) {
    const T* base = row - shift;                // whole vectors inside the row; its ragged ends one by one
    const int first = shift ? 1 : 0, last = (shift + V) / kPer;
    for (int i0 = first + tid; i0 < last; i0 += 8 * kThreads) {
      uint4 x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (i0 + j * kThreads < last) x[j] = __ldcs(reinterpret_cast<const uint4*>(base) + i0 + j * kThreads);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (i0 + j * kThreads < last) {
          reinterpret_cast<uint4*>(s_row)[i0 + j * kThreads] = x[j];
          const T* e = reinterpret_cast<const T*>(&x[j]);
          float most = -INFINITY;               // (fmaxf passes NaN over)
#pragma unroll
          for (int k = 0; k < kPer; ++k) most = fmaxf(most, (float)e[k]);
          top = max(top, key_of(most));
        }
    }
    if (tid < 2 * kPer) {
      const int at = tid < kPer ? tid : (vecs - 1) * kPer + tid - kPer, v = at - shift;
      const bool ragged = tid < kPer ? first == 1 : last < vecs && (vecs > 1 || first == 0);
      if (ragged) {
        const T x = v >= 0 && v < V ? row[v] : (T)(-INFINITY);
        reinterpret_cast<T*>(s_row)[at] = x;
        top = max(top, key_of((float)x));
      }
    }
  } else {
    for (int w = tid; w < (V + 31) / 32; w += kThreads) s_gone[w] = 0u;
    each(tid, units, kThreads, [&](int, float x) { top = max(top, key_of(x)); });
  }
  for (int i = tid; i < kBins; i += kThreads) sh.bin_lo[i] = sh.bin_hi[i] = 0u;
  top = __reduce_max_sync(0xFFFFFFFFu, top);
  if (lane == 0) sh.red[warp] = top;
  if (tid == 0) { sh.cut_tie = 0x7FFFFFFF; sh.bin = -1; sh.n_list = 0; }
  __syncthreads();
  top = __reduce_max_sync(0xFFFFFFFFu, sh.red[lane]);
  if (top == 0) return make_int2(-1, -1);
  Row r;
  r.top = of_key(top);
  r.greedy = !(temp > 0.f);
  r.inf = r.top == INFINITY;
  r.c16 = r.greedy ? 0.0 : 16.0 * 1.4426950408889634 / fmax((double)fminf(temp, 1e30f), 1e-29);
  r.c16_hi = (float)r.c16;
  r.c16_lo = (float)(r.c16 - (double)r.c16_hi);
  r.least = r.greedy ? 0.f : (float)(-760.0 / r.c16);     // 2^-47.5: rounds to nothing
  const bool smooth = !r.greedy && !r.inf;      // weights between 0 and 1

  // ---- 2. the mass, and the bins' if there will be a cut
  const bool cut = r.greedy || top_p < 1.f;
  u64 mass = 0;
  if (smooth) {
    // the last bin that can be in the nucleus: 16 log2(V / (1 - top_p)), and two more for its roundings
    const int bins = cut ? (top_p > 0.f ? min(kBins, (int)(16.f * (log2f((float)V) - log2f(1.f - top_p))) + 3) : 1) : 0;
    each(tid, units, kThreads, [&](int, float x) {
      int k;
      float f;
      split<T>(r, x, k, f);
      const u64 w = weight_of(sh, k, f);
      mass += w;
      if (-k < bins) {
        const uint32_t m = (uint32_t)(w >> up(k));
        atomicAdd(&sh.bin_lo[-k], m & 0x3FFFu);
        atomicAdd(&sh.bin_hi[-k], m >> 14);
      }
    });
  } else {
    each(tid, units, kThreads, [&](int, float x) { mass += x == r.top ? kOne : 0ull; });
  }
  mass = block_sum(sh, mass);

  // ---- 3. the nucleus: tokens from (cut_key, cut_tie) up
  uint32_t cut_key = 0;
  int cut_tie = 0x7FFFFFFF;
  if (cut) {
    u64 target = 1;
    if (!r.greedy && top_p > 0.f) target = max((u64)1, (u64)ceil((double)top_p * (double)mass));
    u64 above = 0;                              // mass of the bins that are surely kept
    bool ordered = false;
    uint32_t lo = top, hi = top;                // keys among which the cut lies, if it is not found by order
    float x_lo = 0.f, x_hi = 0.f;               // logits of the bin lie between them
    if (smooth) {
      const u64 mine = tid < kBins ? (u64)sh.bin_lo[tid] + ((u64)sh.bin_hi[tid] << 14) << up(-tid) : 0ull;
      const u64 upto = block_scan(sh, mine);
      if (upto >= target && upto - mine < target) { sh.bin = tid; sh.above = upto - mine; }
      __syncthreads();
      const int bin = sh.bin;
      above = sh.above;
      // a little wider than half a bin on both sides, so that only few tokens are looked at closely
      x_hi = (float)((double)r.top - ((double)bin - 0.51) / r.c16);
      x_lo = (float)((double)r.top - ((double)bin + 0.51) / r.c16);
      x_hi += fabsf(x_hi) * 1e-6f;
      x_lo -= fabsf(x_lo) * 1e-6f;
      each(tid, units, kThreads, [&](int v, float x) {
        int k;
        float f;
        if (!(x >= x_lo && x <= x_hi)) return;
        split<T>(r, x, k, f);
        if (-k == bin) {
          const int at = atomicAdd(&sh.n_list, 1);
          if (at < kList) sh.list[at] = make_ulonglong2((u64)key_of(x) << 32 | (uint32_t)~v, weight_of(sh, k, f));
        }
      });
      __syncthreads();
      const int n = sh.n_list;
      if (n <= kList) {
        ordered = true;
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
          sh.left = before + mine.y;
        }
        __syncthreads();
        cut_key = (uint32_t)(sh.cut >> 32);
        cut_tie = (int)~(uint32_t)sh.cut;
        mass = sh.left;
      } else {                                  // a crowd in one bin (flat rows): bisect its keys
        uint32_t kmin = 0xFFFFFFFFu, kmax = 0;
        each(tid, units, kThreads, [&](int, float x) {
          int k;
          float f;
          if (!(x >= x_lo && x <= x_hi)) return;
          split<T>(r, x, k, f);
          if (-k == sh.bin) { kmin = min(kmin, key_of(x)); kmax = max(kmax, key_of(x)); }
        });
        kmin = __reduce_min_sync(0xFFFFFFFFu, kmin);
        kmax = __reduce_max_sync(0xFFFFFFFFu, kmax);
        __syncthreads();
        if (lane == 0) { sh.red[warp] = kmin; sh.red2[warp] = kmax; }
        __syncthreads();
        lo = __reduce_min_sync(0xFFFFFFFFu, sh.red[lane]);
        hi = __reduce_max_sync(0xFFFFFFFFu, sh.red2[lane]);
      }
    }
    if (!ordered) {
      // the largest key that reaches the target, then how many of its tokens stay, lowest index first
      const u64 base = above;
      while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2 + 1;
        u64 more = 0;
        each(tid, units, kThreads, [&](int, float x) {
          int k;
          float f;
          if (!(x >= x_lo && x <= x_hi && key_of(x) >= mid)) return;
          split<T>(r, x, k, f);
          if (-k == sh.bin) more += weight_of(sh, k, f);
        });
        if (base + block_sum(sh, more) >= target) lo = mid; else hi = mid - 1;
      }
      cut_key = lo;
      u64 over = 0;
      if (smooth)
        each(tid, units, kThreads, [&](int, float x) {
          int k;
          float f;
          if (!(x >= x_lo && x <= x_hi && key_of(x) > cut_key)) return;
          split<T>(r, x, k, f);
          if (-k == sh.bin) over += weight_of(sh, k, f);
        });
      over = block_sum(sh, over);
      const u64 one = weight<T>(sh, r, of_key(cut_key)), ties = (target - base - over + one - 1) / one;
      // every warp counts in a run of its own; the warp whose run holds the last one finds it
      const int per = (units + kWarps - 1) / kWarps, u0 = min(units, warp * per), u1 = min(units, u0 + per);
      u64 mine = 0;
      each(u0 + lane, u1, 32, [&](int, float x) { mine += key_of(x) == cut_key; });
      mine = warp_sum(mine);
      __syncthreads();
      if (lane == 0) sh.sum[warp] = mine;
      __syncthreads();
      const u64 counts = warp_scan(sh.sum[lane]);
      const u64 upto = __shfl_sync(0xFFFFFFFFu, counts, warp);
      if (upto >= ties && upto - mine < ties) {           // (one warp)
        u64 n = upto - mine;
        const int v0 = max(KEPT ? u0 * kPer - shift : u0, 0), v1 = min(V, KEPT ? u1 * kPer - shift : u1);
        for (int base_v = v0; base_v < v1; base_v += 32) {
          const bool is = base_v + lane < v1 && key_of(get(base_v + lane)) == cut_key;
          const unsigned bal = __ballot_sync(0xFFFFFFFFu, is);
          if (n + __popc(bal) >= ties) {
            if (is && n + __popc(bal & ((2u << lane) - 1u)) == ties) sh.cut_tie = base_v + lane;
            break;
          }
          n += __popc(bal);
        }
      }
      __syncthreads();
      cut_tie = sh.cut_tie;
      mass = base + over + ties * one;
    }
  }
  auto kept_weight = [&](float x, int v) -> u64 {
    const uint32_t key = key_of(x);
    if (key < cut_key || (key == cut_key && v > cut_tie)) return 0ull;
    return weight<T>(sh, r, x);
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
        w = kept_weight(get(t), t);
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

  // ---- 5. the drawn token, from what the refused children leave: first the 1/32 of the row that holds
  // it (a warp's share), then the token in it
  for (int j = tid; j < sh.n_refused; j += kThreads) {
    if (KEPT) s_val[sh.refused[j]] = (T)(-INFINITY);
    else atomicOr(&s_gone[sh.refused[j] >> 5], 1u << (sh.refused[j] & 31));
  }
  __syncthreads();
  auto rest_weight = [&](int v, float x) -> u64 {
    if (!KEPT && ((s_gone[v >> 5] >> (v & 31)) & 1u)) return 0ull;
    return kept_weight(x, v);
  };
  const int per = (units + kWarps - 1) / kWarps, u0 = min(units, warp * per), u1 = min(units, u0 + per);
  u64 sum = 0;
  each(u0 + lane, u1, 32, [&](int v, float x) { sum += rest_weight(v, x); });
  sum = warp_sum(sum);
  if (lane == 0) sh.sum[warp] = sum;
  __syncthreads();
  const double goal = uniform(uni, 0) * (double)sh.left;
  if (warp == 0) {
    const u64 mine = sh.sum[lane], upto = warp_scan(mine);
    if ((double)upto > goal && !((double)(upto - mine) > goal)) { sh.seg = lane; sh.seg_before = upto - mine; }
  }
  __syncthreads();
  const int g0 = min(units, sh.seg * per), g1 = min(units, g0 + per);
  const int s0 = max(KEPT ? g0 * kPer - shift : g0, 0), s1 = min(V, KEPT ? g1 * kPer - shift : g1);
  u64 before = sh.seg_before;
  for (int base = s0; base < s1; base += kThreads) {      // (more than one round for more than 32768 tokens)
    const u64 mine = base + tid < s1 ? rest_weight(base + tid, get(base + tid)) : 0ull;
    const u64 upto = before + block_scan(sh, mine);
    if ((double)upto > goal && !((double)(upto - mine) > goal)) sh.token = base + tid;
    if (tid == kThreads - 1) sh.above = upto;
    __syncthreads();
    before = sh.above;
  }
  return make_int2(-1, sh.token);
}

__device__ __forceinline__ void fill_table(Shared& sh) {
  if (threadIdx.x < 16) {
    const double p = exp2(26.0 + (double)threadIdx.x / 16.0);
    sh.pow16[threadIdx.x] = make_uint2(__float_as_uint((float)p), (uint32_t)(p + 0.5));
  }
}

// One block per context walks.
template <typename T, bool KEPT>
__global__ void __launch_bounds__(kThreads, 1) rest_accept_sampled_walk_kernel(const __grid_constant__ Args a) {
  extern __shared__ __align__(16) unsigned char s_row[];
  __shared__ Shared sh;
  fill_table(sh);
  grid_wait();
  const int b = blockIdx.x, tid = threadIdx.x;
  int32_t *an = a.accept_nodes + (int64_t)b * a.max_depth, *ot = a.out_tokens + (int64_t)b * (a.max_depth + 1);
  int cur = -1, len = 0;
  for (;;) {
    const int2 o = row_outcome<T, KEPT>(a, sh, s_row, b, cur, len);
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
  extern __shared__ __align__(16) unsigned char s_row[];
  __shared__ Shared sh;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  fill_table(sh);
  grid_wait();
  const int b = blockIdx.y, cur = (int)blockIdx.x - 1, tid = threadIdx.x;
  if (cur >= min(max(a.n_nodes[b], 0), a.N)) return;
  const int2 o = row_outcome<T, KEPT>(a, sh, s_row, b, cur, -1);
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
  const size_t row = ((size_t)a.V * sizeof(T) + 31) / 16 * 16;
  if (row <= kRowBytes) return run<T, true>(a, B, row, smem_slot, st);
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
