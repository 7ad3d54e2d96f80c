// rest_paged_attention_scaled: the attention of rest_paged_attention over pages of e4m3 codes with a scale for every
// 16 rows of a head.  K/V are half the bytes of a 16-bit cache.
//
// Scales never touch the codes.  With x = scale log2(e) (q . k codes) ks the score in log2 units, the weight of a key is
//   2^(x + log2 vs - m) = p vs 2^-m,
// V's scale rides in the exponent: O += weight * (v codes), and the row's sum takes weight / vs, once for the 16 keys that
// share it.  The reference m is a whole number (a rescaling of O and the sum is exact) and stays 2^7 below what
// would make the largest weight 1, so that fp16 weights reach 2^-31 of it.  Weights and V are fp16 operands (a code is
// exact in fp16), K's codes go in as they are or as fp16; sums are in 32 bits.  A weight is rounded to fp16 because that is
// what a matrix product takes: half a step is 2^-11 of it, as much as the output's own rounding in fp16 and an eighth of that in
// bf16, and roundings of many keys cancel; the rest of its bits would be a second product of the same size.
//
// Two kernels, by the rows of a KV head, R = N H / H_kv: up to 16, warps on their own (below); more, the 128-row tiles of
// the 16-bit call with K's codes as operands of kind f8f6f4 next to Q as a sum of e4m3 terms (both operands of a product have 8
// bits or both 16, and K widened as V is cost more: 338 and 930 us as terms, 382 and 1239 widened, for the two cases of
// trees below as they were then), V widened to fp16 by four more warps.  Both go by the same shares of the flat tile list, and
// the same second kernel joins cut units.
//
// Measured (B200; copy rate 6568 GB/s, bf16 matrix rate 1658 TFLOP/s; captured in a graph, back to back): 1 token x 2048 keys,
// 32/8 heads 12.5 us (two dependent launches; 16-bit pages 16.6); 256 tokens x 4096 keys 262 us = 94 % of the copy rate;
// 256 tokens, window 2048, D = 64, fp16 135 us (4.1 TB/s; 16-bit pages 198); 61 ragged trees of 64 nodes x 4096 283 us
// (246); 16 trees of 128 nodes x 16384, 640 rows a KV head, 771 us = 900 TFLOP/s (686).  The last two are no
// quicker than with 16-bit pages: both are bound by the chain from S to P, and here S takes two products (three with fp16) of
// half the depth, and V's widening its share of shared-memory reads.  What they give is the room.
// The border, 64 contexts x 4096: 4, 8, 16 rows 78, 80, 115 us by warps, 183, 185, 189 us by tiles; from 17 rows on O no
// longer fits a warp's registers, and 20 rows take 187 us by tiles.  Beside 16-bit pages, 64 x 4096 keys of full contexts,
// bf16: 1, 4, 8, 16 rows 94, 98, 101, 131 us (171, 179, 175, 179); 17, 20, 32, 64, 128, 256 rows 217, 221, 221, 234, 250, 386 us
// (182, 185, 189, 201, 230, 358); fp16, with three terms of Q, 233, 231, 233, 246, 265, 418 us (184, 188, 189, 201, 231, 360).
// One stream's tree over 2048 keys, 32/8 heads: 16 nodes 22 us (20), 64 nodes 32 us (32).  D = 64 by warps is bound by
// instructions: half as many bytes go with each softmax.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "common.cuh"
#include "paged_attention.cuh"
#include "rest.h"

namespace {

// ------------------------------------------------------------------------- up to 16 rows a KV head
// Few rows make the K/V stream all that counts, and 128-row matrix instructions would read a tile of Q that is nearly
// empty from shared memory for every 64 keys.  Here two warps fetch key tiles by TMA into a ring (128 to 192 KB of
// keys on their way), and the others take 16 keys at a time (one scale of K and one of V), four warps a tile: they widen the
// codes in registers and feed them to m16n8k16 instructions as the operand with 16 rows, S^T = K Q^T and O^T = V^T P^T,
// with 8 query rows (or 16, two columns of tiles) as the other one.  Each has maxima, sums and O of its own; they
// meet at the end of a piece only, where their rows are joined while the ring fills with the next piece.
//
// The order of elements inside a dot product is free as long as both sides have the same one, and so is the order of O's
// columns: lane (g, c) = (lane / 4, lane % 4) takes elements 32 c ... 32 c + 31 (D = 128) of keys g and g + 8 as its
// part of K, and columns 16 g ... 16 g + 15 of keys 2c, 2c + 1, 2c + 8, 2c + 9 as its part of V, all in 16-byte
// reads without bank conflicts (D = 64: half of either, 8-byte reads of V in twos).
template <int D, int NB> struct Few {
  static constexpr int kWarps = NB == 1 ? 12 : 8, kTeams = kWarps / 4, kThreads = 32 * (kWarps + 2), kRows = 8 * NB;
  static constexpr int kTile = 64 * D, kStage = 2 * kTile;                // bytes of 64 keys of K, and of K and V
  // A stage belongs to one team (a multiple of the teams): whoever waits for a stage's next tile has seen the one before, so
  // that the parity of its barrier says which of the two has landed.
  static constexpr int kStages = D == 64 ? (NB == 1 ? 18 : 16) : NB == 1 ? 12 : 10;
  static_assert(kStages % kTeams == 0, "a stage belongs to one team");
  static constexpr int kRing = kStages * kStage;
  // O's copies in the join: D = 64 has room for every warp's at once; with D = 128 half of the warps leave theirs for the
  // others to add to, and the ring keeps its length (256 tokens x 4096 keys: 261 us; all at once and a ring of 9: 303 us)
  static constexpr int kCopies = D == 64 ? kWarps : kWarps / 2;
  static constexpr int kRowStride = D + 8;                                // floats: rows two apart meet different banks
  static constexpr int kMerge = kRing, kMl = kMerge + kCopies * kRows * kRowStride * 4;    // [2][kWarps][kRows] float2
  static constexpr int kScale = kMl + 2 * kWarps * kRows * 8;         // [kStages] {K's of 16 keys each, V's}
  static constexpr int kFull = kScale + kStages * 32, kFree = kFull + kStages * 8;
  static constexpr int kCtl = (kFree + kStages * 8 + 15) / 16 * 16;
  static constexpr int kScanAt = 512;                                     // of the control words: a sum of each warp
  static constexpr int kSmem = kCtl + 512 + 8 * (kWarps + 2);
};

__device__ __forceinline__ void mma_16x8x16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {            // of an 8 x 8 matrix of 16-bit elements
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void halves(uint32_t codes, uint32_t& lo, uint32_t& hi) {    // four codes as fp16
  asm("{.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;}" : "=r"(lo), "=r"(hi) : "r"(codes));
}
__device__ __forceinline__ void lds128(uint32_t at, uint32_t (&w)[4]) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void lds64(uint32_t at, uint32_t (&w)[2]) {
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at) : "memory");
}
// NaN codes become 0; whether there were any
__device__ __forceinline__ bool without_nan(uint32_t& w) {
  const uint32_t nan = ((w & 0x7F7F7F7Fu) + 0x01010101u & 0x80808080u) >> 7;
  w &= ~(nan * 0xFFu);
  return nan != 0;
}
// Whether packed row r sees key `key` (bit 0) and key + 8 (bit 1).  No more than 16 rows means no more than 16 nodes, so one
// word of the mask says what it sees of them; only where a path may be longer than the window have they positions of
// their own.  (A call: inside the loop its values would push others out of the registers.)
__device__ __noinline__ uint32_t sees(const Args& a, Ctx ctx, int b, int rows, int r, int key) {
  const int node = node_of(a, min(r, rows - 1));
  const uint32_t word = (a.mask ? __ldg(a.mask + (int64_t)b * a.N + node) : (2u << node) - 1u) & ((1u << a.N) - 1u);
  uint32_t seen;
  if (a.window > 0 && a.window < a.N) {
    const int key0 = key & ~63;
    const u64 v = visible(a, ctx, b, node, node_depth(a, b, node), word, key0) >> (key - key0);
    seen = (uint32_t)(v & 1u) | (uint32_t)(v >> 8 & 1u) << 1;
  } else {
    const int from = a.window > 0 ? max(ctx.L + max(__popc(word), 1) - a.window, 0) : 0;   // first position in its window
    auto one = [&](int k) -> uint32_t {
      const bool before = k >= from || k < a.sinks, node_seen = k < ctx.L + ctx.n && (word >> (k - ctx.L & 31) & 1u);
      return k < ctx.L ? before : node_seen;
    };
    seen = one(key) | one(key + 8) << 1;
  }
  return r < rows ? seen : 0u;
}

template <typename T, int D, int NB>
__global__ void __launch_bounds__(Few<D, NB>::kThreads, 1)
paged_attention_few_kernel(const __grid_constant__ Args a, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v) {
  using F = Few<D, NB>;
  constexpr int W = F::kWarps, S = F::kStages, TEAMS = F::kTeams, kWords = D / 32;           // words of V's four codes that a lane has of a key
  extern __shared__ __align__(1024) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0), g = lane >> 2, c = lane & 3;
  const uint32_t sbase = smem_u32(smem), ring = sbase, full = sbase + F::kFull, free_ = sbase + F::kFree, scales = sbase + F::kScale;
  unsigned char* ctl = smem + F::kCtl;
  volatile uint32_t* abort_word = reinterpret_cast<volatile uint32_t*>(ctl + kAbort);
  volatile int* s_bad = reinterpret_cast<volatile int*>(ctl + kBad);
  const Rows where{0, (int)blockIdx.x, a.teams_last, 1};

  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if ((sbase & 1023u) != 0) {                           // swizzled tiles need it (uniform over the grid)
    if (tid == 0) {
      atomicOr(&g_paged_error, 2u);
      asm volatile("griddepcontrol.wait;" ::: "memory");
      a.meta[blockIdx.x] = make_int4(0, 0, 0, 0);
    }
    return;
  }
  if (tid == 0) {
    for (int i = 0; i < S; ++i) {
      mbar_init(full + 8 * i, 2 + 2 * (64 >> min(a.page_log, 6)));        // two tiles' bytes, and each box's scales
      mbar_init(free_ + 8 * i, 4);
    }
    *abort_word = 0u;
    for (int i = 0; i < 8; ++i) s_bad[i] = 0;
  }
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const Share share = find_share<64, 1, F::kThreads>(a, where, 0, ctl, ctl + F::kScanAt);
  __syncthreads();
  Walk<64, 128> walk(a, *reinterpret_cast<int*>(ctl + kStartB), *reinterpret_cast<long long*>(ctl + kStartOff),
                     share.x0 < share.x1 ? *reinterpret_cast<long long*>(ctl + kStartLeft) : 0ll, 0);

  Piece p;
  if (warp >= W) {
    // ------------------------------------------------------------------ K's and V's fetching warps
    // A lane has a box (a page, or 64 rows of a larger one) and its scales, so a warp works out the addresses of 8 to 32
    // tiles at once; then it goes through them, and only waits and starts copies.
    const bool is_v = warp > W;
    const CUtensorMap* map = is_v ? &tm_v : &tm_k;
    const uint32_t my_ring = ring + (is_v ? F::kTile : 0), my_scale = scales + (is_v ? 16 : 0);
    const int box_log = min(a.page_log, 6), boxes_log = 6 - box_log, mine = lane >> boxes_log, at_once = 32 >> boxes_log;
    const int box0 = (lane & ((1 << boxes_log) - 1)) << box_log;          // the box's first row in its tile
    int slot = 0, filled = 0;
    uint32_t parity = 1;                                // a fresh ring's slots count as free
    bool ok = true;
    while (ok && walk.next(p)) {
      for (int it0 = 0; ok && it0 < p.len; it0 += at_once) {
        const int row = tile_key<64>(p.c, p.t0 + min(it0 + mine, p.len - 1)) + box0, col = row >> a.page_log;
        int page = col < a.table_cols ? __ldg(a.table + p.b * a.table_stride + col) : -1;
        if (page < 0 || page >= a.P) page = a.P;        // outside the map: reads as zeros
        const int in_page = row & ((1 << a.page_log) - 1);
        const int c1 = a.slot[0] == 1 ? in_page : a.slot[1] == 1 ? p.hk : page, c2 = a.slot[0] == 2 ? in_page : a.slot[1] == 2 ? p.hk : page,
                  c3 = a.slot[0] == 3 ? in_page : a.slot[1] == 3 ? p.hk : page;
        // (without a page 0, which counts as the least scale)
        const float* from = is_v ? a.v_scales : a.k_scales;
        const int bytes = page < a.P ? 1 << (box_log - 2) : 0;
        if (bytes) from += (((int64_t)page * a.H_kv + p.hk) << (a.page_log - 4)) + (in_page >> 4);
        const int n = min(at_once, p.len - it0);
        for (int j = 0; j < n; ++j) {
          if (filled >= S) ok = wait_warp(free_ + slot * 8, parity, abort_word);
          if (!ok) break;
          if (mine == j) {
            const uint32_t bar = full + slot * 8, to = my_scale + slot * 32 + (box0 >> 2);
            if (box0 == 0) mbar_expect_tx(bar, (uint32_t)F::kTile);
            asm volatile(
                "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                ::"r"(my_ring + slot * F::kStage + box0 * D), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(0), "r"(c1), "r"(c2), "r"(c3)
                : "memory");
            copy_scales(box_log, to, from, bytes);
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
          }
          __syncwarp();
          ++filled;
          if (++slot == S) { slot = 0; parity ^= 1; }
        }
      }
    }
    if (*abort_word != 0u) {                            // giving up: let the copies in flight land before this block goes away
      asm volatile("cp.async.wait_all;" ::: "memory");
      for (int i = max(0, filled - S); i < filled; ++i) mbar_wait(full + (i % S) * 8, (uint32_t)((i / S) & 1));
    }
    if (is_v && lane == 0 && share.x0 < share.x1) leave_unfinished<64, 1>(a, share, where.team, 0, ctl);
    return;
  }

  // -------------------------------------------------------------------- the others
  const int team = warp >> 2, sub = warp & 3;           // every TEAMS-th tile, keys 16 sub ... of it
  auto meet = [&]() {                                   // (counts threads, not warps: lanes need not come together)
    __syncwarp();
    asm volatile("barrier.sync 1, %0;" ::"n"(32 * W) : "memory");
  };
  uint32_t base = 0;                                    // tiles before this piece
  bool dead = false;                                    // a wait gave up; the barriers of the block are still kept
  // a piece's rows of Q as they lie in memory (this lane's D / 4 elements of rows g, g + 8)
  uint4 raw[NB][D / 32];
  auto look = [&]() {
#pragma unroll
    for (int t = 0; t < NB; ++t) {
      const int r = t * 8 + g;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) raw[t][i] = make_uint4(0u, 0u, 0u, 0u);
      if (r < p.rows) {
        const int node = node_of(a, r);
        const T* from = static_cast<const T*>(a.q) + p.b * a.q_b + node * a.q_n + (int64_t)(p.hk * a.G + r - node * a.G) * a.q_h + c * (D / 4);
#pragma unroll
        for (int i = 0; i < D / 32; ++i) raw[t][i] = __ldg(reinterpret_cast<const uint4*>(from) + i);
      }
    }
  };
  int piece = 0;
  while (walk.next(p)) {
    ++piece;
    look();
    // ---- Q as the second operand: fp16 under a power of two for each row (bf16 has fewer bits and more range)
    uint32_t q[NB][2 * kWords][2];                      // [.][k step][.]
    float mult[NB][2];                                  // what makes log2 units of a row's raw scores, but for K's scale
#pragma unroll
    for (int t = 0; t < NB; ++t) {
      float x[D / 4], most = 0.f;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        const uint32_t w[4] = {raw[t][i].x, raw[t][i].y, raw[t][i].z, raw[t][i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 f = Type<T>::unpack(w[j]);
          x[8 * i + 2 * j] = f.x;
          x[8 * i + 2 * j + 1] = f.y;
        }
      }
      float up = 1.f, own = a.scale_log2;
      if constexpr (!__is_same(T, __half)) {
#pragma unroll
        for (int i = 0; i < D / 4; ++i) most = fmaxf(most, fabsf(x[i]) < INFINITY ? fabsf(x[i]) : 0.f);
        most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
        // the largest to [2^14, 2^15): elements down to 2^-31 of it are exact
        const int e = most > 0.f ? min(max(14 - ((int)(__float_as_uint(most) >> 23) - 127), -100), 100) : 0;
        up = __uint_as_float((uint32_t)(e + 127) << 23);
        own *= __uint_as_float((uint32_t)(127 - e) << 23);
      }
#pragma unroll
      for (int s = 0; s < 2 * kWords; ++s) {
        q[t][s][0] = Type<__half>::pack(x[4 * s] * up, x[4 * s + 1] * up);
        q[t][s][1] = Type<__half>::pack(x[4 * s + 2] * up, x[4 * s + 3] * up);
      }
      mult[t][0] = __shfl_sync(0xFFFFFFFFu, own, 8 * c);
      mult[t][1] = __shfl_sync(0xFFFFFFFFu, own, 8 * c + 4);
    }
    float o[NB][D / 16][4], m[NB][2], l[NB][2];
#pragma unroll
    for (int t = 0; t < NB; ++t) {
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[t][i][j] = 0.f;
      m[t][0] = m[t][1] = -INFINITY;
      l[t][0] = l[t][1] = 0.f;
    }
    int clear0, clear1;
    clear_tiles<64>(a, p, clear0, clear1);
    const int end = p.c.L + p.c.n;
    // (by the tile's number among all that the block has fetched, so that a stage stays with its team from piece to piece)
    const uint32_t start = (team + TEAMS - base % TEAMS) % TEAMS;
    uint32_t slot = (base + start) % S, parity = (base + start) / S & 1;
    base += p.len;
#pragma unroll 1
    for (int it = start; it < p.len; it += TEAMS) {
      const int key0 = tile_key<64>(p.c, p.t0 + it) + sub * 16;
      if (!dead && !wait_warp(full + 8 * slot, parity, abort_word)) dead = true;
      if (dead) break;
      const uint32_t sK = ring + slot * F::kStage + sub * (16 * D), sV = sK + F::kTile, at_scale = scales + slot * 32 + sub * 4,
                     bar = free_ + 8 * slot;
      slot += TEAMS;
      if (slot >= S) { slot -= S; parity ^= 1; }
      if (key0 >= end) {                                // no such keys
        if (lane == 0) mbar_arrive(bar);
        __syncwarp();
        continue;
      }
      // ---- S^T: 16 keys x 8 rows, even and odd steps apart (half the chain of dependent products)
      float s2[NB][2][4];
#pragma unroll
      for (int t = 0; t < NB; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) s2[t][0][j] = s2[t][1][j] = 0.f;
#pragma unroll
      for (int j = 0; j < D / 64; ++j) {
        uint32_t lo[4], hi[4];                          // of keys g and g + 8
        if constexpr (D == 128) {
          lds128(sK + g * 128 + ((2 * c + j ^ g) << 4), lo);
          lds128(sK + (g + 8) * 128 + ((2 * c + j ^ g) << 4), hi);
        } else {
          lds128(sK + g * 64 + ((c ^ (g >> 1)) << 4), lo);
          lds128(sK + (g + 8) * 64 + ((c ^ (g >> 1)) << 4), hi);
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          uint32_t k[4];
          halves(lo[w], k[0], k[2]);
          halves(hi[w], k[1], k[3]);
#pragma unroll
          for (int t = 0; t < NB; ++t) mma_16x8x16(s2[t][w & 1], k, q[t][4 * j + w][0], q[t][4 * j + w][1]);
        }
      }
      float sk, sv;
      sk = lds1(at_scale);
      sv = lds1(at_scale + 16);
      uint32_t v[4][kWords];                            // keys 2c, 2c + 1, 2c + 8, 2c + 9
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = 2 * c + (j & 1) + (j >> 1) * 8;
        if constexpr (D == 128) lds128(sV + key * 128 + ((g ^ (key & 7)) << 4), v[j]);
        else lds64(sV + key * 64 + ((g >> 1 ^ (key >> 1 & 3)) << 4) + (g & 1) * 8, v[j]);
      }
      __syncwarp();                                     // the tile's part is read
      if (lane == 0) mbar_arrive(bar);
      __syncwarp();
      // ---- probabilities: the scale of V rides in the exponent
      sk = rest_e4m3::within_limits(sk);
      float log_v;
      asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(log_v) : "f"(rest_e4m3::within_limits(sv)));
      const float inv_v = ex2(-log_v);
      float y[NB][4];                                   // raw scores: keys g, g, g + 8, g + 8, rows 2c, 2c + 1 in turn
      float ka[NB][2];
#pragma unroll
      for (int t = 0; t < NB; ++t) {
#pragma unroll
        for (int j = 0; j < 2; ++j) ka[t][j] = fminf(fmaxf(sk * mult[t][j], 0x1p-126f), 0x1p127f);
#pragma unroll
        for (int j = 0; j < 4; ++j) y[t][j] = s2[t][0][j] + s2[t][1][j];
      }
      if (!(it >= clear0 && it < clear1)) {             // not every row sees every key
#pragma unroll
        for (int t = 0; t < NB; ++t)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const uint32_t seen = sees(a, p.c, p.b, p.rows, t * 8 + 2 * c + j, key0 + g);
            if (!(seen & 1u)) y[t][j] = -INFINITY;
            if (!(seen & 2u)) y[t][2 + j] = -INFINITY;
          }
        bool found = false;                             // NaN would reach rows that do not see its key (0 x NaN)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          bool any = false;
#pragma unroll
          for (int w = 0; w < kWords; ++w) any |= without_nan(v[j][w]);
          found |= any && key0 + 2 * c + (j & 1) + (j >> 1) * 8 < end;
        }
        if (found) s_bad[piece & 7] = piece + 1;
        __syncwarp();                                   // (what follows is for the whole warp)
      }
      bool over = false;
#pragma unroll
      for (int t = 0; t < NB; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) over |= fmaf(y[t][j], ka[t][j & 1], log_v) > m[t][j & 1] + (kRescaleStep + kShift);
      if (__builtin_expect(__any_sync(0xFFFFFFFFu, over), 0)) {
#pragma unroll
        for (int t = 0; t < NB; ++t)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float mx = fmaf(fmaxf(y[t][j], y[t][2 + j]), ka[t][j], log_v);
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, d));
            const float m_new = fmaxf(m[t][j], ceilf(mx) - kShift);
            const float alpha = m_new == -INFINITY ? 1.f : ex2(m[t][j] - m_new);
            l[t][j] *= alpha;
            m[t][j] = m_new;
#pragma unroll
            for (int e = 0; e < D / 16; ++e) { o[t][e][j] *= alpha; o[t][e][2 + j] *= alpha; }
          }
      }
      uint32_t pb[NB][2];
#pragma unroll
      for (int t = 0; t < NB; ++t) {
        float e[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) e[j] = ex2(fmaf(y[t][j], ka[t][j & 1], log_v - (m[t][j & 1] == -INFINITY ? 0.f : m[t][j & 1])));
        l[t][0] = fmaf(e[0] + e[2], inv_v, l[t][0]);
        l[t][1] = fmaf(e[1] + e[3], inv_v, l[t][1]);
        pb[t][0] = transposed(Type<__half>::pack(e[0], e[1]));
        pb[t][1] = transposed(Type<__half>::pack(e[2], e[3]));
      }
      // ---- O^T += V^T P^T: columns 4 w ... 4 w + 3 of this lane's from word w, two to a product
#pragma unroll
      for (int w = 0; w < kWords; ++w) {
        const uint32_t ab = __byte_perm(v[0][w], v[1][w], 0x5140), cd = __byte_perm(v[2][w], v[3][w], 0x5140),
                       ef = __byte_perm(v[0][w], v[1][w], 0x7362), gh = __byte_perm(v[2][w], v[3][w], 0x7362);
        uint32_t x[4], z[4];
        halves(ab, x[0], x[1]);
        halves(cd, x[2], x[3]);
        halves(ef, z[0], z[1]);
        halves(gh, z[2], z[3]);
#pragma unroll
        for (int t = 0; t < NB; ++t) {
          mma_16x8x16(o[t][2 * w], x, pb[t][0], pb[t][1]);
          mma_16x8x16(o[t][2 * w + 1], z, pb[t][0], pb[t][1]);
        }
      }
    }

    // ---- the warps' rows are joined: maxima and sums (in turns of two: a warp may be a piece ahead), then O
    float2* ml = reinterpret_cast<float2*>(smem + F::kMl) + (piece & 1) * W * F::kRows;
#pragma unroll
    for (int t = 0; t < NB; ++t)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l[t][j] += __shfl_xor_sync(0xFFFFFFFFu, l[t][j], d);
        if (g == 0) ml[warp * F::kRows + t * 8 + 2 * c + j] = make_float2(m[t][j], l[t][j]);
      }
    meet();                                             // (all are done with the O's of the join before, too)
    // where every warp's O has room it is left as it is; else both halves weigh theirs and the second adds to the first
    constexpr bool kAll = F::kCopies == W;
#pragma unroll
    for (int round = 0; round < (kAll ? 1 : 2); ++round) {
      if (kAll || (warp >= F::kCopies) == (round == 0)) {
#pragma unroll
        for (int t = 0; t < NB; ++t)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int r = t * 8 + 2 * c + j;
            float weight = 1.f;
            if (!kAll) {
              float top = -INFINITY;
#pragma unroll
              for (int w = 0; w < W; ++w) top = fmaxf(top, ml[w * F::kRows + r].x);
              weight = m[t][j] == -INFINITY ? 0.f : ex2(m[t][j] - top);
            }
            // columns 2e, 2e + 1 of this lane's D / 8 stand at e * 16 + 2 g
            float* to = reinterpret_cast<float*>(smem + F::kMerge) + (warp % F::kCopies * F::kRows + r) * F::kRowStride + 2 * g;
#pragma unroll
            for (int e = 0; e < D / 16; ++e) {
              float2 v = make_float2(o[t][e][j] * weight, o[t][e][2 + j] * weight);
              if (round == 1) {
                const float2 other = *reinterpret_cast<const float2*>(to + e * 16);
                v.x += other.x;
                v.y += other.y;
              }
              *reinterpret_cast<float2*>(to + e * 16) = v;
            }
          }
      }
      meet();
    }
    const int64_t w0 = ((int64_t)blockIdx.x * 2 + (p.t0 == 0 ? 1 : 0)) * a.rows;
    for (int r = warp; r < p.rows; r += W) {
      const int gg = lane & 7, part = lane >> 3;        // columns (D / 8) gg + (D / 32) part ...
      float top = -INFINITY, sum = 0.f, y[D / 32];
#pragma unroll
      for (int e = 0; e < D / 32; ++e) y[e] = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) top = fmaxf(top, ml[w * F::kRows + r].x);
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float2 v = ml[w * F::kRows + r];          // (a maximum passes NaN over; the sum says so)
        const float weight = v.x == -INFINITY ? 0.f : ex2(v.x - top);
        sum = fmaf(v.y, weight, sum);
        if (w >= F::kCopies) continue;
        const float* from = reinterpret_cast<const float*>(smem + F::kMerge) + (w * F::kRows + r) * F::kRowStride + 2 * gg;
#pragma unroll
        for (int e = 0; e < D / 64; ++e) {
          const float2 f = *reinterpret_cast<const float2*>(from + (part * (D / 64) + e) * 16);
          // (a warp without keys has weight 0 and an O of 0)
          y[2 * e] = fmaf(f.x, kAll ? weight : 1.f, y[2 * e]);
          y[2 * e + 1] = fmaf(f.y, kAll ? weight : 1.f, y[2 * e + 1]);
        }
      }
      const int node = node_of(a, r), head = p.hk * a.G + r - node * a.G, col = gg * (D / 8) + part * (D / 32);
      if (p.whole) {
        const float inv = sum != 0.f ? 1.f / sum : 0.f;
        uint32_t* to = reinterpret_cast<uint32_t*>(static_cast<T*>(a.out) + p.b * a.o_b + node * a.o_n + head * a.o_h + col);
        uint32_t v[D / 64];
#pragma unroll
        for (int e = 0; e < D / 64; ++e) v[e] = sum != 0.f ? Type<T>::pack(y[2 * e] * inv, y[2 * e + 1] * inv) : 0u;
        if constexpr (D == 128) *reinterpret_cast<uint2*>(to) = make_uint2(v[0], v[1]);
        else *to = v[0];
        if (a.lse && lane == 0) a.lse[((int64_t)p.b * a.H + head) * a.N + node] = sum != 0.f ? (top + log2f(sum)) * kLn2 : -INFINITY;
      } else {
        float* to = a.ws_o + (w0 + r) * D + col;
        if constexpr (D == 128) *reinterpret_cast<float4*>(to) = make_float4(y[0], y[1], y[2], y[3]);
        else *reinterpret_cast<float2*>(to) = make_float2(y[0], y[1]);
        if (lane == 0) *reinterpret_cast<float2*>(a.ws_ml + (w0 + r) * 2) = make_float2(top, sum);
      }
    }
    if (__builtin_expect(s_bad[piece & 7] == piece + 1, 0)) {             // (behind a barrier: all threads see the same)
      meet();
      if (warp == 0) {
        const int r = lane;
        bool live = r < p.rows;
        const int node = live ? node_of(a, r) : 0, head = p.hk * a.G + (live ? r - node * a.G : 0);
        u64 mask0 = 0;
        float sum = 0.f;
        if (live) {
          for (int w = 0; w < W; ++w) sum += ml[w * F::kRows + r].y;
          if (a.mask) {
            const uint32_t* mp = a.mask + ((int64_t)p.b * a.N + node) * a.Wm;
            mask0 = __ldg(mp);
            if (a.Wm > 1) mask0 |= (u64)__ldg(mp + 1) << 32;
          }
        }
        live = live && sum == sum;                      // (a row whose sum is NaN is NaN throughout)
        write_not_finite<T, D, 64, true>(a, p, live, node, live && a.window > 0 ? node_depth(a, p.b, node) : 1, mask0,
                                         p.whole ? p.b * a.o_b + node * a.o_n + head * a.o_h : (w0 + r) * D);
      }
    }
  }
  if (dead && lane == 0) atomicOr(&g_paged_error, 1u);
}

template <typename T, int D, int NB>
rest_status run_few(const Args& a, const CUtensorMap& tm_k, const CUtensorMap& tm_v, int slot, cudaStream_t st) {
  using F = Few<D, NB>;
  static_assert(F::kSmem <= 232448, "shared memory of a block");
  REST_CUDA_TRY(rest::ensure_dynamic_smem(reinterpret_cast<const void*>(paged_attention_few_kernel<T, D, NB>), slot, F::kSmem));
  return launch_and_join<T, D>(paged_attention_few_kernel<T, D, NB>, a, tm_k, tm_v, F::kThreads, F::kSmem, st);
}

template <typename T, int D>
rest_status pick_scaled(const Args& a, const CUtensorMap& tm_k, const CUtensorMap& tm_v, const Plan& pl, int slot, cudaStream_t st) {
  slot += rest::kSmemSlotScaled;
  if (pl.few) return pl.rows > 8 ? run_few<T, D, 2>(a, tm_k, tm_v, slot + 3, st) : run_few<T, D, 1>(a, tm_k, tm_v, slot + 2, st);
  return run<T, D, 2, 1, true>(a, tm_k, tm_v, slot, st);
}

}  // namespace

rest_status rest::take_scaled_error_flags(uint32_t* h_flags) { return take_error_flags(h_flags); }

extern "C" rest_status rest_paged_attention_scaled(const void* d_q, const void* d_k_pages, const void* d_v_pages,
                                                   const int64_t* strides, const float* d_k_scales, const float* d_v_scales,
                                                   int32_t dtype, int32_t P, int32_t page, const int32_t* d_table,
                                                   int64_t table_stride, int32_t table_cols, const int32_t* d_kv_len,
                                                   const int32_t* d_n_nodes, const uint32_t* d_mask, int32_t B, int32_t H,
                                                   int32_t H_kv, int32_t N, int32_t D, int32_t window, int32_t sinks,
                                                   float scale, void* d_out, float* d_lse, void* d_ws, size_t ws_bytes,
                                                   void* stream) {
  return attend<true>(d_q, d_k_pages, d_v_pages, strides, d_k_scales, d_v_scales, dtype, P, page, d_table, table_stride,
                      table_cols, d_kv_len, d_n_nodes, d_mask, B, H, H_kv, N, D, window, sinks, scale, d_out, d_lse, d_ws,
                      ws_bytes, stream);
}
