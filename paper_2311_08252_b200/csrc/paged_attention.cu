// rest_paged_attention: attention of draft rows (or single tokens) over a KV cache in pages, with
// an optional sliding window and first tokens that stay visible.
//
// The G = H / H_kv query heads of a KV head times the n nodes of a context give R = G n rows that
// all read the same keys, so the rows (node-major, r = i G + g) are packed into 128-row tiles of
// tcgen05.mma: S = Q K^T, then O += P V.
//
// Work.  The key tiles of all (context, KV head) units stand in one flat list, and every thread
// block takes an equal, contiguous share of it, by cost: uneven lengths, windows, one long context or
// hundreds of short ones all give the same even load in a single wave, and the shares follow from
// the lengths on the device alone.  A unit that a share's border cuts leaves partial rows
// (unnormalised O, maximum, sum) in the caller's scratch, which a second small kernel joins.  When R
// needs several row blocks of 256 rows, each has a list and blocks of its own (see plan).  With a
// window the tiles between the sinks and the earliest visible position are not in the list at all.
//
// Two kernel shapes, picked by R (rows per KV head):
//   R <= 128  one 128-row tile, two blocks per SM: bound by the K/V stream, so what counts is bytes
//             in flight (5 tiles of 16 KB a block) and a second block that fills the first one's gaps.
//   R > 128   two 128-row tiles that share each 64-key K/V tile (read once for 256 rows), one block
//             per SM: bound by the chain from S to P (exponentials half of it) and the tensor core.
// S has two buffers in TMEM for each row tile, so the tensor core runs a key tile ahead of the softmax
// warps and neither waits for the other's round trip (one 128-key buffer per row tile instead, which
// spends a fifth less tensor time, needed 5500 cycles per 128 keys and 256 rows).
// P is written back over S in TMEM and is the A operand of P V from there: no shared-memory round
// trip for it.
// O stays in TMEM and accumulates; its reference maximum is only raised when a tile exceeds it by
// 2^8, and only then is the O row rescaled.
//
// K and V tiles arrive by TMA, one box per page (or per 64-key slice of a larger page) and
// 64-element half of the head, in the 128-byte-swizzled operand layout; a page index that is out
// of range reads as zeros.  Every wait is bounded (see rest_device_error_flags).
//
// Precision: scores, maxima, sums and O in 32 bits; P is rounded to the cache's type for the
// tensor core (half a step, 2^-9 of each probability in bf16 - the output is rounded as much), the
// sum takes the unrounded values, so lse carries none of it.
//
// Measured (B200, join included; the copy rate is 6536 GB/s, the bf16 matrix rate 1669 TFLOP/s): calls back to back
// (the large ones then run into the board's power limit, at 1500 to 1700 of 1965 MHz; captured in a graph they take
// the same), and in brackets one at a time at the full clock with a cold L2.  64 nodes x 2048 keys, 32 KV
// heads, 24.4 us (latency); 61 ragged trees x 4096 keys, 32/8 heads, page 16, 277 us (252: 595 TFLOP/s); 16 trees of
// 128 nodes x 16384 keys, 40/8 heads, 800 us (674: 1030 TFLOP/s); 64 trees of 33 nodes, window 4096, 250 us (226: 4.9
// TB/s); 256 tokens, window 2048, D = 64, fp16, 240 us (211: 5.3 TB/s).  1 token x 2048 keys, 32/8 heads: 21 us a call, of
// which the GPU needs 15 (captured).  Of the fourth, with half the keys, a profile shows no pipe full (tensor core
// 46 %, exponentials 49 %, issue 37 %, DRAM 32 %): two softmax warps a scheduler, each with its chain of S
// out of TMEM, maximum, exponentials and P back, do not fill each other's waits.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "common.cuh"
#include "rest.h"
#include "tensor_core.cuh"

namespace {

using namespace rest_tc;
typedef unsigned long long u64;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kRescaleStep = 8.f;                     // log2 units

struct Args {
  const void* q;
  void* out;
  float* lse;
  const void *k, *v;                                    // only read again for non-finite values
  const int32_t *table, *kv_len, *n_nodes;
  const uint32_t* mask;
  int4* meta;                                           // per block: unit it starts and leaves unfinished
  float *ws_o, *ws_ml;                                  // partial rows [block][2][rows][D], [..][2]
  int64_t q_b, q_n, q_h, p_p, p_h, p_r, o_b, o_n, o_h, table_stride;
  int B, H, H_kv, G, N, Wm, P, page_log, table_cols, window, sinks, RB, rows;
  int teams, teams_last;                                // blocks of each row block, and of the last one
  uint32_t g_inverse;                                   // ceil(2^32 / G), G > 1
  int slot[3];                                          // tensor-map coordinate (1..3) of row, head, page
  float scale_log2;
};

// packed row r = node * G + head within the group (r * G < 2^32: the product's error stays below 1)
__device__ __forceinline__ int node_of(const Args& a, int r) {
  return a.G == 1 ? r : (int)__umulhi((uint32_t)r, a.g_inverse);
}
// n / d; most are small, and a 64-bit division takes some hundred instructions
__device__ __forceinline__ long long divide(long long n, long long d) {
  return ((n | d) >> 32) == 0 ? (long long)((uint32_t)n / (uint32_t)d) : n / d;
}
// Blocks of a row block lie `apart` blocks from one another: the last one's stand behind those of all others,
// which take turns (they read the same tiles at about the same time).
struct Rows { int rb, team, teams, apart; };
__device__ __forceinline__ Rows rows_of(const Args& a, int x, int teams, int teams_last) {
  const int others = teams * (a.RB - 1);
  if (x >= others) return {a.RB - 1, x - others, teams_last, 1};
  return {x % (a.RB - 1), x / (a.RB - 1), teams, a.RB - 1};
}
// A block of two row tiles is quicker with a key tile when one row tile would hold all rows (the two take turns
// then), so its share holds more of them.  Costs 1 : 1, 4 : 3, 3 : 2, 2 : 1 took 270, 218, 217, 221 us for 64 windows
// of 4096 keys with 68 to 132 rows, and 242, 242, 238, 291 us for 61 contexts of 2048 to 4096 keys with 128 to 256.
constexpr int kBoth = 3, kTurns = 2;
__device__ __forceinline__ long long tiles_for(long long cost, int of_one) {          // rounded up
  return of_one == 1 ? cost : divide(cost + of_one - 1, of_one);
}
// One context's keys and its list of visible tiles: the first ns tiles hold the sinks, the others
// run from tile w0 to the end.
struct Ctx { int L, n, w0, ns, cost; long long nt; };   // cost: of one of its tiles
template <int BN, int TILES>
__device__ __forceinline__ Ctx context(const Args& a, int b, int row0) {    // (no tiles without rows from row0 on)
  Ctx c;
  const int cap = a.table_cols << a.page_log;           // a longer length has no pages behind it
  c.L = min(max(a.kv_len[b], 0), cap);
  c.n = a.n_nodes ? min(max(a.n_nodes[b], 0), a.N) : a.N;
  c.w0 = c.ns = 0;
  c.cost = TILES == 1 ? 1 : a.G * c.n - row0 > 128 ? kBoth : kTurns;
  const int first = c.L - a.window + 1;                 // earliest position in any node's window
  if (a.window > 0 && first > 0) {
    c.w0 = first / BN;
    c.ns = min((min(a.sinks, c.L) + BN - 1) / BN, c.w0);
  }
  c.nt = a.G * c.n <= row0 ? 0 : c.ns + (c.L + c.n + BN - 1) / BN - c.w0;
  return c;
}
template <int BN>
__device__ __forceinline__ int tile_key(const Ctx& c, int t) { return (t < c.ns ? t : t - c.ns + c.w0) * BN; }

// A block's share of the flat tile list, piece by piece; every role of the block walks it alike.
struct Piece { Ctx c; int b, hk, t0, len, rows; bool whole; };
template <int BN, int ROWS>
struct Walk {                                           // left: cost up to the end of the share
  const Args& a;
  int b, rb;
  long long off, left;
  __device__ Walk(const Args& a_, int b_, long long off_, long long left_, int rb_)
      : a(a_), b(b_), rb(rb_), off(off_), left(left_) {}
  __device__ __forceinline__ bool next(Piece& p) {
    while (left > 0) {
      p.c = context<BN, ROWS / 128>(a, b, rb * ROWS);
      if (off >= a.H_kv * p.c.nt) { off -= a.H_kv * p.c.nt; ++b; continue; }
      p.b = b;
      p.hk = (int)divide(off, p.c.nt);
      p.t0 = (int)(off - p.hk * p.c.nt);
      p.len = (int)min(p.c.nt - (long long)p.t0, tiles_for(left, p.c.cost));
      p.whole = p.len == (int)p.c.nt;
      off += p.len;
      left -= (long long)p.len * p.c.cost;
      p.rows = min(a.G * p.c.n - rb * ROWS, ROWS);
      return true;
    }
    return false;
  }
};

template <typename T> struct Type;
template <> struct Type<__nv_bfloat16> {
  static constexpr uint32_t format = 1, exponent = 0x7F80u;
  __device__ static uint32_t pack(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
  }
  __device__ static float2 unpack(uint32_t x) { return __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&x)); }
};
template <> struct Type<__half> {
  static constexpr uint32_t format = 0, exponent = 0x7C00u;
  __device__ static uint32_t pack(float lo, float hi) {
    __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
  }
  __device__ static float2 unpack(uint32_t x) { return __half22float2(*reinterpret_cast<__half2*>(&x)); }
};

// instruction descriptor: T x T -> fp32, M = 128, A K-major, B K-major (0) or MN-major (1)
template <typename T>
__device__ __forceinline__ constexpr uint32_t idesc(int N, int b_mn_major) {
  return (1u << 4) | (Type<T>::format << 7) | (Type<T>::format << 10) | ((uint32_t)b_mn_major << 16) |
         ((uint32_t)(N >> 3) << 17) | ((128u >> 4) << 24);
}
__device__ __forceinline__ uint32_t elect_one() {       // true in one lane of a converged warp
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.b32 %0, 1, 0, p;\n\t}\n" : "=r"(p));
  return p;
}
// A from TMEM
__device__ __forceinline__ void umma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc_,
                                            uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, {%5, %5, %5, %5}, p;\n\t}\n"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc_), "r"(accumulate), "r"(0u)
      : "memory");
}

__device__ __forceinline__ void tmem_st_32x8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};\n"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
      : "memory");
}
// 16 TMEM columns from taddr of the thread's lane into registers: tmem_issue starts, tmem_wait_ld waits for
// all that was started, and tmem_named keeps whatever uses the values from moving ahead of that wait.
// (Values are kept in arrays of 16, indexed by constants only: anything else lands in local memory.)
__device__ __forceinline__ void tmem_issue(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]),
        "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
        "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_named(uint32_t (&r)[16]) {
  asm volatile(""
      : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]),
        "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]),
        "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
      :
      : "memory");
}
__device__ __forceinline__ void tmem_load(uint32_t taddr, uint32_t (&r)[16]) {
  tmem_issue(taddr, r);
  tmem_wait_ld();
  tmem_named(r);
}
__device__ __forceinline__ void tmem_st_32x16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};\n"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

__device__ unsigned int g_paged_error;                  // bit 0: wait gave up, bit 1: smem misaligned

template <int D, int NT> struct Shape {
  static constexpr int BN = 64;                         // keys per step
  static constexpr int kHalves = D / 64;
  static constexpr int kRows = 128 * NT;
  static constexpr int kQTile = 128 * D * 2, kTile = BN * D * 2;
  static constexpr int KS = NT == 1 && D == 128 ? 2 : 4, VS = NT == 1 && D == 128 ? 3 : 6;      // ring stages
  static constexpr int kBars = NT * kQTile + (KS + VS) * kTile;           // barriers behind the tiles
  static constexpr int kSmem = kBars + 512;
  static constexpr int kSoftmax = 4 * NT;               // softmax warps; then K loader, V loader, MMA warps
  static constexpr int kThreads = 32 * (kSoftmax + 2 + NT);
  static constexpr uint32_t kTmem = NT == 1 ? 256 : 512;
  static constexpr uint32_t kColO = 2 * NT * BN;        // behind two S buffers for each row tile
};
// byte offsets behind kBars
enum {
  kKFull = 0, kKFree = 32, kVFull = 64, kVFree = 112, kSFull = 160, kPFull = 192, kOFull = 224, kQFull = 240, kQFree = 248,
  kTmemSlot = 256, kAbort = 260, kBad = 264 /* 8 x 4 */, kStartB = 296, kStartOff = 304, kTotal = 312,
  kScan = 320 /* 12 x 8 */, kJoin = 416, kTurn = 424 /* 8 x 8 */, kStartLeft = 488
};

// Bounded wait of a whole warp, with one result for all lanes (TMEM accesses and elected lanes need
// them together).  The first look comes without the clock and the abort word: most barriers are ready.
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, volatile uint32_t* abort_word) {
  uint32_t ready;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.b32 %0, 1, 0, p;\n\t}\n"
      : "=r"(ready)
      : "r"(bar), "r"(parity)
      : "memory");
  if (__builtin_expect(__all_sync(0xFFFFFFFFu, ready != 0), 1)) return true;
  return __all_sync(0xFFFFFFFFu, mbar_wait_abortable(bar, parity, abort_word) ? 1 : 0) != 0;
}

// one 64-element x box-rows box of the pool -> shared memory
__device__ __forceinline__ void tma_page(uint32_t dst, const CUtensorMap* map, int c0, int row, int head, int page,
                                         const int (&slot)[3], uint32_t bar) {
  const int c1 = slot[0] == 1 ? row : slot[1] == 1 ? head : page;
  const int c2 = slot[0] == 2 ? row : slot[1] == 2 ? head : page;
  const int c3 = slot[0] == 3 ? row : slot[1] == 3 ? head : page;
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5, %6}], [%2];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
      : "memory");
}

// bits [lo, hi) of a 64-bit word, clipped to it
__device__ __forceinline__ u64 bits_between(int lo, int hi) {
  lo = max(lo, 0);
  hi = min(hi, 64);
  if (hi <= lo) return 0ull;
  return (hi == 64 ? ~0ull : (1ull << hi) - 1ull) & ~((1ull << lo) - 1ull);
}
__device__ __forceinline__ int node_depth(const Args& a, int b, int i) {
  if (!a.mask) return i + 1;
  const uint32_t* m = a.mask + ((int64_t)b * a.N + i) * a.Wm;
  int d = 0;
  for (int w = 0; w < a.Wm; ++w) {
    const uint32_t x = __ldg(m + w);
    d += __popc(32 * w + 32 <= a.N ? x : x & ((1u << (a.N & 31)) - 1u));         // (no bits behind node N - 1)
  }
  return d;
}
// one position behind the last that a node can stand at: a mask row may hold bits of nodes that do not exist
__device__ __forceinline__ int end_of(const Args& a, const Ctx& c) { return c.L + (a.mask ? a.N : c.n); }
// every row of the block sees every key of the tile at key0 (tiles of the sinks count as masked)
template <int BN>
__device__ __forceinline__ bool all_see(const Args& a, const Ctx& c, int key0) {
  return key0 + BN <= c.L && (a.window == 0 || key0 > end_of(a, c) - 1 - a.window);
}
// which of the keys k0 .. k0 + 63 node i (of depth `depth`) of context b sees; first: words 0 and 1 of its
// mask row
__device__ __noinline__ u64 visible(const Args& a, Ctx c, int b, int i, int depth, u64 first, int k0) {
  const int pos = c.L + max(depth, 1) - 1;
  u64 v;
  if (a.window == 0)
    v = bits_between(0, c.L - k0);
  else
    v = bits_between(0, min(a.sinks, c.L) - k0) | bits_between(max(pos - a.window + 1, 0) - k0, c.L - k0);
  if (k0 + 64 > c.L) {
    u64 m[4] = {0ull, 0ull, 0ull, 0ull};
    if (a.mask) {
      const uint32_t* mp = a.mask + ((int64_t)b * a.N + i) * a.Wm;
#pragma unroll
      for (int w = 2; w < 8; ++w)
        if (w < a.Wm) m[w >> 1] |= (u64)__ldg(mp + w) << (32 * (w & 1));
      m[0] = first;
    } else {
#pragma unroll
      for (int w = 0; w < 4; ++w) m[w] = bits_between(0, i + 1 - 64 * w);
    }
    const int shift = k0 - c.L;
    u64 t = mask_window(m, shift) & bits_between(-shift, c.n - shift);
    if (a.window > 0 && a.window < a.N) {               // only then can a path be longer than the window
      for (u64 rest_ = t; rest_; rest_ &= rest_ - 1) {
        const int bit = __ffsll((long long)rest_) - 1;
        const int at = c.L + max(node_depth(a, b, shift + bit), 1) - 1;
        if (!(at < a.sinks || at > pos - a.window)) t &= ~(1ull << bit);
      }
    }
    v |= t;
  }
  return v;
}

// Values of V that are not finite, at keys that a row sees, decide their columns of the row alone: +infinity,
// -infinity, or NaN where there is a NaN or both.  The products do not say so (they were taken out of masked
// tiles, and a probability that is 0, by rounding or because the key belongs to another copy, makes NaN of
// them), so such columns of a piece's rows, at `mine` of the output or the scratch, are written once more.
// For whole warps, a row (`live`) a lane: the lanes read a key each, then every row looks at those that hold
// something.  Rare, and far from free: with an infinity in every context the 61 trees x 4096 keys take 1.2 instead of
// 0.27 ms, the 16 x 16384 keys 6.7 instead of 0.76 (other warps' bounded waits have to outlast one piece's search).
template <typename T, int D, int BN>
__device__ __noinline__ void write_not_finite(const Args& a, Piece p, bool live, int node, int depth, u64 mask0,
                                              long long mine) {
  const int lane = threadIdx.x & 31;
  constexpr uint32_t inf = Type<T>::exponent;
  constexpr int kGroups = 4;      // 64 columns at a time (all of 128 at once took registers from the caller's loop)
  for (int d0 = 0; d0 < D; d0 += 64) {
    uint32_t found[kGroups];      // of columns d0 + 16 c ...: bit j +infinity or NaN in the j-th, 16 + j -infinity or NaN
#pragma unroll
    for (int c = 0; c < kGroups; ++c) found[c] = 0;
    for (int it = 0; it < p.len; ++it) {
      const int first = tile_key<BN>(p.c, p.t0 + it);
      u64 vis = 0ull;
      bool asked = false;
      for (int h = 0; h < BN; h += 32) {
        const int key = first + h + lane, col = key >> a.page_log;
        const int page = key < p.c.L + p.c.n && col < a.table_cols ? a.table[p.b * a.table_stride + col] : -1;
        uint32_t odd[kGroups], any = 0;
#pragma unroll
        for (int c = 0; c < kGroups; ++c) odd[c] = 0;
        if (page >= 0 && page < a.P) {
          const uint4* v = reinterpret_cast<const uint4*>(static_cast<const T*>(a.v) + page * a.p_p + p.hk * a.p_h +
                                                          (key & ((1 << a.page_log) - 1)) * a.p_r + d0);
#pragma unroll
          for (int c = 0; c < kGroups; ++c) {
            const uint4 x = v[2 * c], y = v[2 * c + 1];
            const uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const uint32_t e = w[j >> 1] >> (16 * (j & 1)) & 0xFFFFu;
              if ((e & 0x7FFFu) >= inf) odd[c] |= (e != (inf | 0x8000u) ? 1u << j : 0u) | (e != inf ? 0x10000u << j : 0u);
            }
            any |= odd[c];
          }
        }
        for (unsigned which = __ballot_sync(0xFFFFFFFFu, any != 0); which; which &= which - 1) {
          const int l = __ffs(which) - 1;
          if (!asked) vis = !live ? 0ull : all_see<BN>(a, p.c, first) ? ~0ull : visible(a, p.c, p.b, node, depth, mask0, first);
          asked = true;
          const bool sees = (vis >> (h + l)) & 1u;
#pragma unroll
          for (int c = 0; c < kGroups; ++c) {
            const uint32_t there = __shfl_sync(0xFFFFFFFFu, odd[c], l);
            if (sees) found[c] |= there;
          }
        }
      }
    }
#pragma unroll
    for (int c = 0; c < kGroups; ++c) {
      for (uint32_t left = (found[c] | found[c] >> 16) & 0xFFFFu; left; left &= left - 1) {
        const int j = __ffs(left) - 1;
        const bool plus = found[c] >> j & 1u, minus = found[c] >> (16 + j) & 1u;
        const long long to = mine + d0 + c * 16 + j;
        if (p.whole)
          static_cast<uint16_t*>(a.out)[to] = (uint16_t)(plus && minus ? 0x7FFFu : minus ? inf | 0x8000u : inf);
        else
          a.ws_o[to] = __uint_as_float(plus && minus ? 0x7FFFFFFFu : minus ? 0xFF800000u : 0x7F800000u);
      }
    }
  }
}
// a partial O, weighed: what is not finite stays so under a weight that rounds to 0
__device__ __forceinline__ float weighed(float o, float w) { return fabsf(o) < INFINITY ? o * w : o; }

template <typename T, int D, int NT, int C>
__global__ void __launch_bounds__(Shape<D, NT>::kThreads, NT == 1 ? 2 : 1)
paged_attention_kernel(const __grid_constant__ Args a, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v) {
  using S_ = Shape<D, NT>;
  constexpr int BN = S_::BN, KS = S_::KS, VS = S_::VS, kHalves = S_::kHalves;
  extern __shared__ __align__(1024) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);
  const uint32_t sbase = smem_u32(smem);
  const uint32_t sQ = sbase, sK = sQ + NT * S_::kQTile, sV = sK + KS * S_::kTile;
  const uint32_t bars = sbase + S_::kBars;
  unsigned char* ctl = smem + S_::kBars;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ctl + kTmemSlot);
  volatile uint32_t* abort_word = reinterpret_cast<volatile uint32_t*>(ctl + kAbort);
  volatile int* s_bad = reinterpret_cast<volatile int*>(ctl + kBad);       // [piece % 8]: piece + 1
  const Rows where = NT == 1 ? Rows{0, (int)blockIdx.x, a.teams_last, 1}      // one row tile: one row block
                             : rows_of(a, blockIdx.x, a.teams, a.teams_last);
  const int team = where.team, rb = where.rb, row0 = rb * S_::kRows;

  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if ((sbase & 1023u) != 0) {   // the swizzled operand layout needs a 1024-byte aligned base
    if (tid == 0) {
      atomicOr(&g_paged_error, 2u);
      asm volatile("griddepcontrol.wait;" ::: "memory");
      a.meta[blockIdx.x] = make_int4(0, 0, 0, 0);       // nothing to join
    }
    return;                     // uniform over the grid: every block sees the same offset
  }
  if (tid == 0) {
    for (int i = 0; i < KS; ++i) { mbar_init(bars + kKFull + 8 * i, 1); mbar_init(bars + kKFree + 8 * i, NT); }
    for (int i = 0; i < VS; ++i) { mbar_init(bars + kVFull + 8 * i, 1); mbar_init(bars + kVFree + 8 * i, NT); }
    for (int i = 0; i < 4; ++i) {
      mbar_init(bars + kSFull + 8 * i, 1);
      mbar_init(bars + kPFull + 8 * i, 4);              // one arrival per softmax warp
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bars + kOFull + 8 * i, 1);
    }
    mbar_init(bars + kQFull, 1);
    mbar_init(bars + kQFree, NT);                       // one arrival per row tile
    mbar_init(bars + kJoin, S_::kSoftmax);
    for (int i = 0; i < 8; ++i) { s_bad[i] = 0; mbar_init(bars + kTurn + 8 * i, 1); }
    *abort_word = 0u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                 "r"(S_::kTmem)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // everything above is independent of the inputs; from here on global memory is read
  asm volatile("griddepcontrol.wait;" ::: "memory");

  // ---- this team's share of the flat tile list: the tiles that start in [x0, x1), and the first one's context
  long long x0, x1;
  int teams;
  {
    const int per = (a.B + S_::kThreads - 1) / S_::kThreads;
    long long mine = 0;
    for (int i = 0; i < per; ++i)
      if (tid * per + i < a.B) {
        const Ctx c = context<BN, NT>(a, tid * per + i, row0);
        mine += a.H_kv * c.nt * c.cost;
      }
    long long inc = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long y = __shfl_up_sync(0xFFFFFFFFu, inc, d);
      if (lane >= d) inc += y;
    }
    long long* s_scan = reinterpret_cast<long long*>(ctl + kScan);
    if (lane == 31) s_scan[warp] = inc;
    __syncthreads();
    long long before = 0, total = 0;
    for (int w = 0; w < S_::kThreads / 32; ++w) {
      if (w == warp) before = total;
      total += s_scan[w];
    }
    // fewer tiles than teams: one each, the rest idle (no share is shorter than a tile)
    teams = (int)min((long long)where.teams, NT == 1 ? total : max(total / kBoth, 1ll));
    // no more than 64 pieces of a unit: joining 296 pieces of one KV head took longer than the keys
    // (32768 keys, one KV head: 51 us; in 128 pieces 27 us)
    teams = min((long long)teams, 64ll * a.B * a.H_kv);
    // one context: its units are alike, and with the same number of teams each no share crosses a border
    if (a.B == 1 && teams > a.H_kv) teams -= teams % a.H_kv;
    x0 = team < teams ? divide(total * team, teams) : total;
    x1 = team < teams ? divide(total * (team + 1), teams) : total;
    long long at = before + inc - mine;
    if (x0 < x1 && at <= x0 && x0 < at + mine) {        // one thread
      int b = tid * per;
      for (;; ++b) {
        const Ctx c = context<BN, NT>(a, b, row0);
        const long long n = a.H_kv * c.nt * c.cost;
        if (x0 < at + n) {
          const long long skip = tiles_for(x0 - at, c.cost);
          *reinterpret_cast<long long*>(ctl + kStartOff) = skip;
          *reinterpret_cast<long long*>(ctl + kStartLeft) = x1 - at - skip * c.cost;
          break;
        }
        at += n;
      }
      *reinterpret_cast<int*>(ctl + kStartB) = b;
    }
    if (tid == 0) {
      if (x0 >= x1) a.meta[blockIdx.x] = make_int4(0, 0, 0, 0);      // else the V loader writes it
      *reinterpret_cast<long long*>(ctl + kTotal) = total;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, *tmem_slot, 0);
  Walk<BN, S_::kRows> walk(a, *reinterpret_cast<int*>(ctl + kStartB), *reinterpret_cast<long long*>(ctl + kStartOff),
                           x0 < x1 ? *reinterpret_cast<long long*>(ctl + kStartLeft) : 0ll, rb);
  Piece p;

  if (warp == S_::kSoftmax || warp == S_::kSoftmax + 1) {
    // ------------------------------------------------------------------ K loader, V loader
    const bool is_v = warp == S_::kSoftmax + 1;
    const int stages = is_v ? VS : KS;
    const uint32_t ring = is_v ? sV : sK, full = bars + (is_v ? kVFull : kKFull), free_ = bars + (is_v ? kVFree : kKFree);
    const CUtensorMap* map = is_v ? &tm_v : &tm_k;
    const int box = min(1 << a.page_log, BN);           // rows of one box
    const int pg = lane / kHalves, half = lane % kHalves;
    const bool active = pg * box < BN;
    int slot = 0, filled = 0;
    uint32_t parity = 1;                                // a fresh ring's slots count as free
    bool ok = true;
    uint32_t pieces = 0;
    while (ok && walk.next(p)) {
      const int32_t* table = a.table + p.b * a.table_stride;
      // the page of this lane's box, looked up a tile ahead
      auto find = [&](int it, int& row) -> int {
        row = tile_key<BN>(p.c, p.t0 + it) + pg * box;
        const int col = row >> a.page_log;
        return active && col < a.table_cols ? __ldg(table + col) : -1;
      };
      int row, page = find(0, row);
      if (is_v) {
        // Q rows of the piece -> shared memory, K-major 128-byte-swizzled, each for every copy of its row.
        // Rows past the last one keep whatever is there: their scores are never looked at.  This warp gets
        // here while the softmax warps are still busy with the piece before, so the copies (thousands of
        // cycles behind the key tiles in flight) are under way by the time that Q is free for them.
        if (pieces > 0) ok = wait_warp(bars + kQFree, (pieces - 1) & 1, abort_word);
        if (!ok) break;
        ++pieces;
        const bool turns = NT == 2 && p.rows <= 128;
        constexpr int kChunks = D / 8, kRowsAtOnce = 32 / kChunks;
        const int chunk = lane % kChunks;
        const T* q = static_cast<const T*>(a.q) + p.b * a.q_b + (int64_t)p.hk * a.G * a.q_h + chunk * 8;
        for (int row32 = 0; row32 < p.rows; row32 += 32) {
          const int r = rb * S_::kRows + row32 + lane, node = node_of(a, r);
          const long long mine = node * a.q_n + (r - node * a.G) * a.q_h;  // where this lane's row starts
#pragma unroll 4
          for (int j = 0; j < kChunks; ++j) {
            const int row = row32 + j * kRowsAtOnce + lane / kChunks;
            const long long at = __shfl_sync(0xFFFFFFFFu, mine, row & 31);
            if (row < p.rows) {
#pragma unroll
              for (int c = 0; c < (NT == 2 ? 2 : C); ++c) {
                if (NT == 2 && c == 1 && !turns) break;
                const int to = (row & 127) + (NT == 2 ? 0 : c * (128 / C));
                const uint32_t dst = sQ + (NT == 2 ? (row >> 7) + c : 0) * S_::kQTile + (chunk >> 3) * (128 * 128) +
                                     (to >> 3) * 1024 + (to & 7) * 128 + (((chunk & 7) ^ (to & 7)) << 4);
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(q + at) : "memory");
              }
            }
          }
        }
      }
      for (int it = 0; it < p.len; ++it) {
        int next_row = row;
        const int next_page = it + 1 < p.len ? find(it + 1, next_row) : page;
        if (page < 0 || page >= a.P) page = a.P;        // outside the map: reads as zeros
        if (filled >= stages)
          ok = wait_warp(free_ + slot * 8, parity, abort_word);
        if (!ok) break;
        if (lane == 0) mbar_expect_tx(full + slot * 8, (uint32_t)S_::kTile);
        __syncwarp();
        if (active)
          tma_page(ring + slot * S_::kTile + half * (BN * 128) + pg * (box * 128), map, half * 64,
                   row & ((1 << a.page_log) - 1), p.hk, page, a.slot, full + slot * 8);
        row = next_row;
        page = next_page;
        if (is_v && it == 0) {                          // the first V tile is on its way; now Q has to be there
          asm volatile("cp.async.wait_all;" ::: "memory");
          fence_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(bars + kQFull);
        }
        ++filled;
        if (++slot == stages) { slot = 0; parity ^= 1; }
      }
    }
    if (*abort_word != 0u) {
      // giving up: let the copies in flight land before this block goes away
      asm volatile("cp.async.wait_all;" ::: "memory");
      for (int i = max(0, filled - stages); i < filled; ++i)
        mbar_wait(full + (i % stages) * 8, (uint32_t)((i / stages) & 1));
    }
    if (is_v && lane == 0 && x0 < x1) {
      // The unit that this share starts but does not finish (if any) goes to the joining kernel:
      // {pieces, context, KV head}.  Its later pieces are the first pieces of the blocks that follow.
      int4 m = make_int4(0, 0, 0, 0);
      // step over whole contexts to the last tile of the share
      long long off = *reinterpret_cast<long long*>(ctl + kStartOff), left = *reinterpret_cast<long long*>(ctl + kStartLeft);
      int b = *reinterpret_cast<int*>(ctl + kStartB);
      Ctx c;
      long long count;
      for (;;) {
        c = context<BN, NT>(a, b, row0);
        count = tiles_for(left, c.cost);
        if (off + count <= a.H_kv * c.nt) break;
        left -= (a.H_kv * c.nt - off) * c.cost;
        off = 0;
        ++b;
      }
      const long long end = off + count, u0 = (end - 1) / c.nt * c.nt, u1 = u0 + c.nt;      // its unit
      const long long base = x1 - left - off * c.cost;                  // where context b starts
      if (u1 > end && base + u0 * c.cost >= x0) {
        const long long total = *reinterpret_cast<long long*>(ctl + kTotal), last = base + (u1 - 1) * c.cost;
        int to = team + 1;
        while (total * (to + 1) / teams <= last) ++to;
        m = make_int4(to - team + 1, b, (int)(u0 / c.nt), 0);
      }
      a.meta[blockIdx.x] = m;
    }
  } else if (warp >= S_::kSoftmax + 2) {
    // ------------------------------------------------------------- MMA issuers, one per row tile
    // The whole warp walks the loop, so that descriptors and addresses stay in uniform registers, and one
    // elected lane issues (a loop in one lane moved them there before every instruction: about 100 cycles
    // each, three times what the tensor core needs).  With two row tiles, one's waits are filled by the
    // other's instructions.
    const int s = warp - (S_::kSoftmax + 2);
    const uint32_t leader = elect_one();
    constexpr uint32_t idesc_s = idesc<T>(BN, 0), idesc_o = idesc<T>(D, 1);
    const uint64_t dq = umma_desc(sQ + s * S_::kQTile, 16, 1024), dk = umma_desc(sK, 16, 1024),
                   dv = umma_desc(sV, BN * 128, 1024);
    const uint32_t t_s = tmem + 2 * s * BN, t_o = tmem + S_::kColO + s * 128;
    const uint32_t b_s = bars + kSFull + 16 * s, b_p = bars + kPFull + 16 * s, b_o = bars + kOFull + 8 * s;
    uint32_t base = 0, n_s = 0, n_p = 0, n_q = 0;       // key tiles before this piece; S issued, P and Q taken
    bool ok = true;
    while (ok && walk.next(p)) {
      // one row tile's rows only: the two row tiles take the key tiles in turn
      const bool turns = NT == 2 && p.rows <= 128;
      const int step = turns ? 2 : 1;
      auto qk = [&](int it) {                           // S of key tile `it`
        const uint32_t g = base + it, slot = g % KS, buf = n_s++ & 1;
        ok = ok && wait_warp(bars + kKFull + slot * 8, (g / KS) & 1, abort_word);
        if (!ok) return;
        tc_fence_after();
        if (leader) {
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            const uint32_t qoff = (uint32_t)((ks >> 2) * (128 * 128) + (ks & 3) * 32);
            const uint32_t koff = (uint32_t)((ks >> 2) * (BN * 128) + (ks & 3) * 32);
            umma_f16(t_s + buf * BN, dq + (qoff >> 4), dk + ((slot * S_::kTile + koff) >> 4), idesc_s, ks > 0);
          }
          umma_commit(b_s + buf * 8);
          umma_commit(bars + kKFree + slot * 8);
          if (turns) umma_commit(bars + kKFree + slot * 8);      // for both row tiles
          if (C == 1 && !turns && it + 1 == p.len) umma_commit(bars + kQFree);
        }
        __syncwarp();
      };
      int it = turns ? s : 0;
      ok = wait_warp(bars + kQFull, n_q++ & 1, abort_word);
      // (a piece of one tile does not need the second row tile: it tells that it has seen the piece's Q)
      if (ok && turns && s == 1 && leader) mbar_arrive(bars + kQFree);
      if (ok && it < p.len) qk(it);
      if (ok && it + step < p.len) qk(it + step);
      for (bool fresh = true; ok && it < p.len; it += step, fresh = false) {
        const uint32_t g = base + it, slot = g % VS, buf = n_p & 1;
        ok = wait_warp(bars + kVFull + slot * 8, (g / VS) & 1, abort_word) &&
             wait_warp(b_p + buf * 8, (n_p >> 1) & 1, abort_word);
        if (!ok) break;
        ++n_p;
        tc_fence_after();
        if (leader) {
#pragma unroll
          for (int kk = 0; kk < BN / 16; ++kk)
            umma_f16_ts(t_o, t_s + buf * BN + kk * 8, dv + ((slot * S_::kTile + kk * 2048) >> 4), idesc_o,
                        (fresh && kk == 0) ? 0u : 1u);
          umma_commit(b_o);
          umma_commit(bars + kVFree + slot * 8);
          if (turns) umma_commit(bars + kVFree + slot * 8);
        }
        __syncwarp();
        // S two tiles on goes over this P: the tensor core works in order of issue, so P V is done with it
        if (it + 2 * step < p.len) qk(it + 2 * step);
      }
      base += p.len;
    }
  } else {
    // ----------------------------------------------------------------------- softmax warps
    // A thread owns one row of its row tile.  With C copies (few rows) the tile holds the same 128 / C
    // packed rows C times and copy ci takes the ci-th 64 / C keys of every key tile, so that all four
    // warps work; the P of its other keys is zero.  Two row tiles that take the key tiles in turn are
    // two copies as well.  Copies have maxima, sums and O of their own and are joined at the end.
    constexpr int kCopyRows = 128 / C, KP = BN / C;     // rows of a copy, keys of a thread per key tile
    const int s = warp >> 2, t = tid & 127;             // which row tile, row inside it
    const int ci = t / kCopyRows, tr = t % kCopyRows;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t o_col = tmem + lanes + S_::kColO + s * 128;
    auto wait = [&](uint32_t bar, uint32_t parity) -> bool { return wait_warp(bar, parity, abort_word); };
    uint32_t n = 0, base = 0, joins = 0, e_n = 0;
    int piece = 0;
    bool ok = true;
    for (; ok && walk.next(p); base += p.len) {
      ++piece;
      const bool turns = NT == 2 && p.rows <= 128;
      const int step = turns ? 2 : 1;
      const int r0 = rb * S_::kRows + (turns ? 0 : s * 128);               // first packed row of this tile
      const int rows = min(kCopyRows, p.rows - (turns ? 0 : s * 128));
      const bool warp_live = tr - lane < rows, live = tr < rows;
      const int node = live ? node_of(a, r0 + tr) : 0, head = p.hk * a.G + (live ? r0 + tr - node * a.G : 0);
      const int depth = live && a.window > 0 ? node_depth(a, p.b, node) : 1;   // (only windows need it)
      u64 mask0 = 0;                                    // (asked for now, needed in the last tiles)
      if (live && a.mask) {
        const uint32_t* mp = a.mask + ((int64_t)p.b * a.N + node) * a.Wm;
        mask0 = __ldg(mp);
        if (a.Wm > 1) mask0 |= (u64)__ldg(mp + 1) << 32;
      }
      float m_used = -INFINITY, l_run = 0.f;
      // tiles [clear0, clear1) of the piece are those that all rows see whole (see all_see)
      const int at0 = p.c.ns - p.c.w0 - p.t0;
      const int clear0 = a.window == 0 ? 0 : at0 + (max(end_of(a, p.c) - a.window, 0) + BN - 1) / BN, clear1 = at0 + p.c.L / BN;
      int it = turns ? s : 0;
      constexpr int kParts = KP / 16;
      // Two row tiles of the same piece work on the same key tiles, and each scheduler has one warp of either.
      // Left alone they fall into step, both at their exponentials and then both at everything else; taking
      // turns at the exponentials (the first tile before the second, the second before the first's next)
      // keeps the special function unit fed.  A turn ends half way: the second half fills the other's start
      // (768 us at the end, 748 us half way, 845 us after a quarter, for 16 x 16384 keys and 640 rows).
      const bool paired = NT == 2 && !turns && (warp & 3) * 32 + 128 < p.rows;
      const uint32_t my_turn = bars + kTurn + 8 * (warp & 7), other_turn = bars + kTurn + 8 * ((warp & 7) ^ 4);
      for (bool fresh = true; it < p.len; it += step, fresh = false) {
        const uint32_t buf = 2 * s + (n & 1);
        const bool plain = it >= clear0 && it < clear1;
        if (__builtin_expect(!plain, 0)) {
          const int key0 = tile_key<BN>(p.c, p.t0 + it);
          // Values of V that are not finite would reach rows that do not see their key (0 x NaN): take
          // them out of the tile, and remember the piece if the key exists (the epilogue puts in what they
          // come to; where all rows see the whole tile, they are left in it and show in O).  Both row
          // tiles do it when both use the tile, each before its own P V; the piece is remembered before a
          // value is cleared, so whoever finds it cleared finds it remembered.  (One row tile is never
          // more than six key tiles ahead of the other, so eight pieces are told apart.)
          const uint32_t g = base + it, slot = g % VS;
          if (!wait(bars + kVFull + slot * 8, (g / VS) & 1)) { ok = false; break; }
#pragma unroll 4
          for (int j = 0; j < S_::kTile / 16 / 128; ++j) {
            const uint32_t at = (uint32_t)((j * 128 + t) * 16);
            const uint32_t src = sV + slot * S_::kTile + at;
            uint32_t w[4];
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(src) : "memory");
            // an exponent of all ones carries into the bit above when a one is added at its end
            constexpr uint32_t lo = Type<T>::exponent, hi = lo << 16, one = lo & (0u - lo);
            uint32_t any = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) any |= (w[e] & (lo | hi)) + (one | one << 16);
            if (any & 0x80008000u) {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                if ((w[e] & lo) == lo) w[e] &= 0xFFFF0000u;
                if ((w[e] & hi) == hi) w[e] &= 0x0000FFFFu;
              }
              if (key0 + (int)((at % (BN * 128)) >> 7) < p.c.L + p.c.n) { s_bad[piece & 7] = piece + 1; __threadfence_block(); }
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(src), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
            }
          }
          fence_async_smem();
        }
        if (__builtin_expect(!wait(bars + kSFull + buf * 8, (n >> 1) & 1), 0)) { ok = false; break; }
        tc_fence_after();
        if (warp_live) {
          const uint32_t s_col = tmem + lanes + buf * BN;
          uint32_t x[kParts][16];
#pragma unroll
          for (int c = 0; c < kParts; ++c) tmem_issue(s_col + ci * KP + c * 16, x[c]);
          tmem_wait_ld();
#pragma unroll
          for (int c = 0; c < kParts; ++c) tmem_named(x[c]);
          if (__builtin_expect(!plain, 0)) {
            const int key0 = tile_key<BN>(p.c, p.t0 + it);
            const u64 vis = live ? visible(a, p.c, p.b, node, depth, mask0, key0) >> (ci * KP) : 0ull;
            const uint32_t lo = (uint32_t)vis, hi = (uint32_t)(vis >> 32);
#pragma unroll
            for (int j = 0; j < KP; ++j)
              if (!(((j < 32 ? lo : hi) >> (j & 31)) & 1u)) x[j / 16][j % 16] = 0xFF800000u;       // -inf
          }
          // maximum of the raw scores (the scale is positive, so it commutes with max); the scale
          // is applied inside the exponent's multiply-add
          float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int j = 0; j < KP / 2; ++j)
            mx4[j & 3] = max3(mx4[j & 3], __uint_as_float(x[j / 8][2 * (j % 8)]), __uint_as_float(x[j / 8][2 * (j % 8) + 1]));
          const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * a.scale_log2;
          if (__builtin_expect(__any_sync(0xFFFFFFFFu, live && mx > m_used + kRescaleStep), 0)) {
            const float m_new = fmaxf(m_used, mx);
            const float alpha = m_new == -INFINITY ? 1.f : ex2(m_used - m_new);   // m_used = -inf gives 0
            if (!fresh) {
              if (!wait(bars + kOFull + s * 8, (n - 1) & 1)) { ok = false; break; }
              tc_fence_after();
#pragma unroll 1
              for (int c = 0; c < D / 16; ++c) {
                uint32_t o[16];
                tmem_load(o_col + c * 16, o);
#pragma unroll
                for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * alpha);
                tmem_st_32x16(o_col + c * 16, o);
              }
            }
            l_run *= alpha;
            m_used = m_new;
          }
          const float neg = m_used == -INFINITY ? 0.f : -m_used;
          float ps[4] = {0.f, 0.f, 0.f, 0.f};
          if (paired) {
            if ((s == 1 || e_n > 0) && !wait(other_turn, (s == 1 ? e_n : e_n - 1) & 1)) { ok = false; break; }
            ++e_n;
          }
          // P: 64 keys in 32 packed columns over S's first half, eight columns (16 keys) at a time
#pragma unroll
          for (int c = 0; c < kParts; ++c) {
            uint32_t pk[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              float e0, e1;
              fma2(e0, e1, __uint_as_float(x[c][2 * j]), __uint_as_float(x[c][2 * j + 1]), a.scale_log2, neg);
              e0 = ex2(e0);
              e1 = ex2(e1);
              add2(ps[(j & 1) * 2], ps[(j & 1) * 2 + 1], e0, e1);
              pk[j] = Type<T>::pack(e0, e1);
            }
            tmem_st_32x8(s_col + (ci * kParts + c) * 8, pk);
            if (c == 1 && paired && lane == 0) mbar_arrive(my_turn);
          }
          if (C > 1) {                                  // the other copies' keys
            const uint32_t zero[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
#pragma unroll
            for (int c = 0; c < 4; ++c)
              if (c / kParts != ci) tmem_st_32x8(s_col + c * 8, zero);     // (warp-uniform)
          }
          l_run += (ps[0] + ps[1]) + (ps[2] + ps[3]);
          tmem_wait_st();
        }
        // The parity below cannot tell "P V(n) is done" from "P V(n - 1) is not": the last tile but one is
        // waited for while the last one's P is still held back.  (Its S tells of P V(n - 2) only.)
        if (it + step >= p.len && !fresh && !wait(bars + kOFull + s * 8, (n - 1) & 1)) { ok = false; break; }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bars + kPFull + buf * 8);
        ++n;
      }
      if (!ok) break;
      if ((turns ? s : 0) < p.len && !wait(bars + kOFull + s * 8, (n - 1) & 1)) { ok = false; break; }
      tc_fence_after();
      // ---- epilogue: a finished unit's rows go to the output, others to the scratch
      // scratch slot 1: the unit's first piece; 0: a later one (then it is the block's first piece)
      const int64_t w0 = ((int64_t)blockIdx.x * 2 + (p.t0 == 0 ? 1 : 0)) * a.rows + (turns ? 0 : s * 128);
      const long long mine = p.whole ? p.b * a.o_b + node * a.o_n + head * a.o_h : (w0 + tr) * D;
      float odd = 0.f;                                  // NaN when something in this row of O is not finite
      if (C == 1 && !turns) {                           // no copies: every thread writes its row
        const float w = p.whole ? (l_run != 0.f ? 1.f / l_run : 0.f) : 1.f;
        if (warp_live) {
#pragma unroll 1
          for (int c = 0; c < D / 16; ++c) {
            uint32_t o[16];
            __syncwarp();
            tmem_load(o_col + c * 16, o);
            if (!live) continue;
#pragma unroll
            for (int j = 0; j < 16; ++j) odd = fmaf(__uint_as_float(o[j]), 0.f, odd);
#pragma unroll
            for (int j = 0; j < 16; ++j) o[j] = w == 0.f ? 0u : __float_as_uint(__uint_as_float(o[j]) * w);
            if (p.whole) {
              T* op = static_cast<T*>(a.out) + mine + c * 16;
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                uint32_t v[4];
#pragma unroll
                for (int f = 0; f < 4; ++f)
                  v[f] = Type<T>::pack(__uint_as_float(o[8 * e + 2 * f]), __uint_as_float(o[8 * e + 2 * f + 1]));
                *reinterpret_cast<uint4*>(op + e * 8) = make_uint4(v[0], v[1], v[2], v[3]);
              }
            } else {
              float* wo = a.ws_o + mine + c * 16;
#pragma unroll
              for (int e = 0; e < 2; ++e)
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(wo + 8 * e), "r"(o[8 * e]),
                             "r"(o[8 * e + 1]), "r"(o[8 * e + 2]), "r"(o[8 * e + 3]), "r"(o[8 * e + 4]), "r"(o[8 * e + 5]),
                             "r"(o[8 * e + 6]), "r"(o[8 * e + 7])
                             : "memory");
            }
          }
          // (a row whose sum is NaN is NaN throughout)
          const bool bad = s_bad[piece & 7] == piece + 1;
          const bool ask = live && l_run == l_run && (bad || odd != 0.f);
          if (__builtin_expect(__any_sync(0xFFFFFFFFu, ask), 0))
            write_not_finite<T, D, BN>(a, p, ask, node, depth, mask0, mine);
        }
        if (live) {
          if (!p.whole)
            *reinterpret_cast<float2*>(a.ws_ml + (w0 + t) * 2) = make_float2(m_used, l_run);
          else if (a.lse)
            a.lse[((int64_t)p.b * a.H + head) * a.N + node] = l_run != 0.f ? (m_used + log2f(l_run)) * kLn2 : -INFINITY;
        }
        tc_fence_before();                              // O is read: the next piece's P V may overwrite it
        continue;
      }
      // Copies are joined through the memory of the Q tiles, as many columns at a time as fit (all of them
      // for few rows): their last reader, this piece's last S, is done, and the next Q is let in behind
      // the join.
      constexpr int kAll = 128 * NT, copies = NT == 2 ? 2 : C, apart = NT == 2 ? 128 : kCopyRows;
      constexpr int kStage = NT * S_::kQTile - kAll * 8;
      const int me = NT == 2 ? s : ci;                  // this thread's copy
      float w, top, sum;
      auto sync = [&]() -> bool {                       // of the warps that share rows, with a bounded wait
        __syncwarp();
        if (lane == 0) mbar_arrive(bars + kJoin);
        ok = wait(bars + kJoin, joins++ & 1);
        return ok;
      };
      {                                                 // the copies' maxima and sums
        float2* s_ml = reinterpret_cast<float2*>(smem + kStage);                   // [kAll]
        if (!sync()) break;                             // (NT = 2: the other tile's last S is done too)
        s_ml[tid] = make_float2(m_used, l_run);
        if (!sync()) break;
        top = -INFINITY;
        sum = 0.f;
#pragma unroll
        for (int c = 0; c < copies; ++c) top = fmaxf(top, s_ml[tr + c * apart].x);
#pragma unroll
        for (int c = 0; c < copies; ++c) {              // (a maximum passes NaN over: with it alone it stays at
          const float2 ml = s_ml[tr + c * apart];       // -infinity, and the sum, 0 otherwise, says so)
          sum += ml.y * (ml.x == -INFINITY ? 0.f : ex2(ml.x - top));
        }
        w = m_used == -INFINITY ? 0.f : ex2(m_used - top);
      }
      if (p.whole) w *= sum != 0.f ? 1.f / sum : 0.f;
      int cols = D;
      while (rows * copies * cols * 4 > kStage) cols >>= 1;                        // (16 at least)
      const int vecs = cols >> 2, together = 32 / vecs, col = lane & (vecs - 1);   // lanes of a row, rows of a warp
      auto stage = [&](int copy, int row, int vec) -> unsigned char* {
        return smem + ((copy * rows + row) * vecs + (vec ^ (row & 7 & (vecs - 1)))) * 16;
      };
#pragma unroll 1
      for (int c = 0; c < D; c += cols) {
        if (warp_live) {
#pragma unroll 1
          for (int d = 0; d < cols; d += 16) {
            uint32_t o[16];
            __syncwarp();
            tmem_load(o_col + c + d, o);
            if (!live) continue;
#pragma unroll
            for (int j = 0; j < 16; ++j) odd = fmaf(__uint_as_float(o[j]), 0.f, odd);
#pragma unroll
            for (int j = 0; j < 16; ++j) o[j] = w == 0.f ? 0u : __float_as_uint(__uint_as_float(o[j]) * w);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              *reinterpret_cast<uint4*>(stage(me, tr, (d >> 2) + e)) = make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
          }
        }
        // (one of two row tiles in turn may have no tile: then O is what was there before)
        if (live && odd != 0.f && l_run == l_run && (!turns || s < p.len)) s_bad[piece & 7] = piece + 1;
        if (!sync()) break;
        // the warps that hold copies of the same 32 rows share them out again
#pragma unroll 2
        for (int j = me * together; j < min(32, rows - tr + lane); j += copies * together) {
          const int row = j + lane / vecs;              // of this warp's 32
          const long long at = __shfl_sync(0xFFFFFFFFu, mine, row) + c + col * 4;
          if (tr - lane + row >= rows) continue;
          float4 y = *reinterpret_cast<const float4*>(stage(0, tr - lane + row, col));
#pragma unroll
          for (int k = 1; k < copies; ++k) {
            const float4 z = *reinterpret_cast<const float4*>(stage(k, tr - lane + row, col));
            y.x += z.x; y.y += z.y; y.z += z.z; y.w += z.w;
          }
          if (p.whole)
            *reinterpret_cast<uint2*>(static_cast<T*>(a.out) + at) = make_uint2(Type<T>::pack(y.x, y.y), Type<T>::pack(y.z, y.w));
          else
            *reinterpret_cast<float4*>(a.ws_o + at) = y;
        }
        if (!sync()) break;                             // the stage is free again
      }
      if (!ok) break;
      // looked at behind barriers that all copies come to with their tiles checked and their O seen: in turns,
      // one row tile's last tile may be checked later than the other one's last product is done
      if (me == 0 && warp_live && __builtin_expect(__any_sync(0xFFFFFFFFu, s_bad[piece & 7] == piece + 1), 0))
        write_not_finite<T, D, BN>(a, p, live && sum == sum, node, depth, mask0, mine);
      if (tid == 0) mbar_arrive(bars + kQFree);
      if (live && me == 0) {
        if (!p.whole)
          *reinterpret_cast<float2*>(a.ws_ml + (w0 + tr) * 2) = make_float2(top, sum);
        else if (a.lse)
          a.lse[((int64_t)p.b * a.H + head) * a.N + node] = sum != 0.f ? (top + log2f(sum)) * kLn2 : -INFINITY;
      }
      tc_fence_before();                                // O is read: the next piece's P V may overwrite it
    }
  }
  tc_fence_before();
  __syncthreads();
  if (*abort_word != 0u && tid == 0) atomicOr(&g_paged_error, 1u);
  if (warp == 0)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S_::kTmem) : "memory");
}

// Joins the pieces of the units that shares' borders cut.  Block x = (n-th such unit, row block); the
// n-th unit is found by counting the shares that left one, unless there may be one for every share.
// Blocks y take eight rows in turn, a warp each, or - for units cut into more than 16 pieces - one row
// in turn, a warp for each of eight ranges of its pieces, added in a fixed order.
template <typename T, int D>
__global__ void __launch_bounds__(256) paged_attention_join_kernel(const __grid_constant__ Args a) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  __shared__ float s_m[8], s_l[8], s_o[8][D];
  __shared__ int s_team, s_count[8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long units = (long long)a.B * a.H_kv;
  const Rows mine = rows_of(a, blockIdx.x, (int)min(units, (long long)a.teams), (int)min(units, (long long)a.teams_last));
  const int rb = mine.rb, teams = rb + 1 == a.RB ? a.teams_last : a.teams;
  const int block0 = rb + 1 == a.RB ? a.teams * (a.RB - 1) : rb;   // (all scratch rows count to less than 2^31)
  int team = mine.team;
  if (units < teams) {
    const int nth = team;
    if (threadIdx.x == 0) s_team = -1;
    int before = 0;
    for (int base = 0; base < teams; base += 256) {   // (teams <= two blocks an SM: one or two rounds)
      const int i = base + threadIdx.x;
      const bool has = i < teams && a.meta[block0 + i * mine.apart].x != 0;
      const unsigned bal = __ballot_sync(0xFFFFFFFFu, has);
      __syncthreads();
      if (lane == 0) s_count[warp] = __popc(bal);
      __syncthreads();
      int nr = before + __popc(bal & ((1u << lane) - 1u));
      for (int w = 0; w < 8; ++w) { if (w < warp) nr += s_count[w]; before += s_count[w]; }
      if (has && nr == nth) s_team = i;
    }
    __syncthreads();
    team = s_team;
    if (team < 0) return;
  }
  const int block = block0 + team * mine.apart;
  const int4 meta = a.meta[block];
  const int np = meta.x, b = meta.y, hk = meta.z;
  if (np == 0) return;
  const int n = a.n_nodes ? min(max(a.n_nodes[b], 0), a.N) : a.N;
  const int r0 = rb * a.rows, rows = min(a.G * n - r0, a.rows);
  constexpr int E = D / 32;
  const bool wide = np > 16;
  const int lo = wide ? np * warp / 8 : 0, hi = wide ? np * (warp + 1) / 8 : np;
  for (int row0 = wide ? blockIdx.y : blockIdx.y * 8; row0 < rows; row0 += gridDim.y * (wide ? 1 : 8)) {
    const int row = wide ? row0 : row0 + warp;
    float m = -INFINITY, l = 0.f, o[E];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.f;
    if (row < rows) {
      const int first = block * 2 * a.rows + row, step = mine.apart * 2 * a.rows;
      auto at = [&](int i) -> int64_t {                 // piece i: slot 1 of the first block, slot 0 of the others
        return first + i * step + (i == 0 ? a.rows : 0);
      };
      for (int i0 = lo; i0 < hi; i0 += 32) {            // 32 pieces at a time, a lane for each one's maximum and sum
        float2 ml = make_float2(-INFINITY, 0.f);
        if (i0 + lane < hi) ml = *reinterpret_cast<const float2*>(a.ws_ml + at(i0 + lane) * 2);
        float top = fmaxf(m, ml.x);
#pragma unroll
        for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
        const float w = ml.x == -INFINITY ? 0.f : ex2(ml.x - top), old = m == -INFINITY ? 0.f : ex2(m - top);
        float sum = ml.y * w;
#pragma unroll
        for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
        l = l * old + sum;
        m = top;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = weighed(o[e], old);
        const int count = min(32, hi - i0);
#pragma unroll 8
        for (int i = 0; i < count; ++i) {
          const int64_t x = at(i0 + i);
          float v[E];
          if constexpr (E == 4) *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(a.ws_o + x * D + lane * E);
          else *reinterpret_cast<float2*>(v) = *reinterpret_cast<const float2*>(a.ws_o + x * D + lane * E);
          const float wi = __shfl_sync(0xFFFFFFFFu, w, i);
#pragma unroll
          for (int e = 0; e < E; ++e) o[e] += weighed(v[e], wi);
        }
      }
    }
    if (wide) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < E; ++e) s_o[warp][lane * E + e] = o[e];
      if (lane == 0) { s_m[warp] = m; s_l[warp] = l; }
      __syncthreads();
      if (warp != 0) continue;
      m = -INFINITY;
      l = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll
      for (int w = 0; w < 8; ++w) m = fmaxf(m, s_m[w]);
#pragma unroll
      for (int w = 0; w < 8; ++w) {
        const float c = s_m[w] == -INFINITY ? 0.f : ex2(s_m[w] - m);
        l += s_l[w] * c;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] += weighed(s_o[w][lane * E + e], c);
      }
    }
    if (row >= rows) continue;
    const int node = node_of(a, r0 + row), head = hk * a.G + r0 + row - node * a.G;
    const float inv = l != 0.f ? 1.f / l : 0.f;
    uint32_t* op = reinterpret_cast<uint32_t*>(static_cast<T*>(a.out) + b * a.o_b + node * a.o_n + head * a.o_h + lane * E);
#pragma unroll
    for (int e = 0; e < E / 2; ++e) op[e] = Type<T>::pack(o[2 * e] * inv, o[2 * e + 1] * inv);
    if (a.lse && lane == 0)
      a.lse[((int64_t)b * a.H + head) * a.N + node] = l != 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
  }
}

// ------------------------------------------------------------------------------------- host
using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                   const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                   CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_tiled_fn() {
  static EncodeTiledFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult st;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &st) != cudaSuccess ||
        st != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiledFn>(p);
  }();
  return fn;
}

// Map of a pool (d, rows of a page, heads, pages), outer dimensions in order of increasing stride.
bool encode_pool(CUtensorMap* map, const void* base, int dtype, int D, int page, int H_kv, int P, const int64_t* strides,
                 int box_rows, int (&slot)[3]) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const int64_t size[3] = {page, H_kv, P}, stride[3] = {strides[2], strides[1], strides[0]};
  int order[3] = {0, 1, 2};
  auto key = [&](int i) { return size[i] > 1 ? stride[i] : (int64_t)1 << 60; };   // extent 1: stride unused, last
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (key(order[j]) < key(order[i])) { const int t = order[i]; order[i] = order[j]; order[j] = t; }
  cuuint64_t dims[4] = {(cuuint64_t)D, 1, 1, 1}, bytes[3] = {0, 0, 0}, prev = (cuuint64_t)D * 2;
  cuuint32_t box[4] = {64, 1, 1, 1};
  const cuuint32_t step[4] = {1, 1, 1, 1};
  for (int i = 0; i < 3; ++i) {
    const int which = order[i];
    slot[which] = i + 1;
    dims[i + 1] = (cuuint64_t)size[which];
    cuuint64_t st = size[which] > 1 ? (cuuint64_t)stride[which] * 2 : prev;
    if (st < prev) st = prev;
    bytes[i] = prev = st;
    if (which == 0) box[i + 1] = (cuuint32_t)box_rows;
  }
  return fn(map, dtype == REST_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4,
            const_cast<void*>(base), dims, bytes, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Plan { int NT, RB, teams, teams_last, rows; };
Plan plan(int H, int H_kv, int N) {
  Plan p;
  const int64_t R = (int64_t)(H / H_kv) * N;
  p.NT = R > 128 ? 2 : 1;
  p.RB = (int)((R + 128 * p.NT - 1) / (128 * p.NT));
  const int sms = rest::sm_count(), blocks = (p.NT == 1 ? 2 : 1) * (sms > 0 ? sms : 148);
  // A last row block of one row tile's height is quicker with its key tiles (its two row tiles take turns at
  // them), so it gets 0.6 of the blocks that another one has (16 x 16384 keys, 640 rows: 740 us with as many,
  // 750 us with 0.5, 686 us with 0.6, 702 us with 0.65, 716 us with 0.75).
  const bool half = p.NT == 2 && p.RB > 1 && R - (int64_t)(p.RB - 1) * 256 <= 128;
  p.teams = half ? blocks * 20 / (20 * (p.RB - 1) + 12) : blocks / p.RB;
  p.teams = p.teams > 0 ? p.teams : 1;
  p.teams_last = blocks - p.teams * (p.RB - 1);
  p.teams_last = p.teams_last > 0 ? p.teams_last : 1;
  p.rows = R < 128 * p.NT ? (int)R : 128 * p.NT;
  return p;
}
size_t blocks_of(const Plan& p) { return (size_t)p.teams * (p.RB - 1) + p.teams_last; }
size_t workspace_bytes(const Plan& p, int D) {
  const size_t blocks = blocks_of(p);
  return 32 + (blocks + 1) / 2 * 2 * sizeof(int4) + blocks * 2 * p.rows * (D + 2) * sizeof(float);
}

template <typename T, int D, int NT, int C>
rest_status run(const Args& a, const CUtensorMap& tm_k, const CUtensorMap& tm_v, int smem_slot, cudaStream_t st) {
  using S_ = Shape<D, NT>;
  REST_CUDA_TRY(rest::ensure_dynamic_smem(reinterpret_cast<const void*>(paged_attention_kernel<T, D, NT, C>), smem_slot, S_::kSmem));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.teams * (a.RB - 1) + a.teams_last), 1, 1);
  cfg.blockDim = dim3((unsigned)S_::kThreads, 1, 1);
  cfg.dynamicSmemBytes = S_::kSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  REST_CUDA_TRY(cudaLaunchKernelEx(&cfg, paged_attention_kernel<T, D, NT, C>, a, tm_k, tm_v));
  rest::count_launch();
  // never more cut units than shares or units; about eight blocks per SM in all, eight rows each at least
  // (one where units may be cut into more than 16 pieces)
  const int64_t units = (int64_t)a.B * a.H_kv;
  auto cut = [&](int teams) { return units < teams ? (int)units : teams; };
  const int joins = cut(a.teams) * (a.RB - 1) + cut(a.teams_last), per = 8 * 148 / joins;
  const int most = (a.RB > 1 && a.teams > a.teams_last ? a.teams : a.teams_last) > 16 * units ? a.rows : (a.rows + 7) / 8;
  cfg.gridDim = dim3((unsigned)joins, (unsigned)(per < 1 ? 1 : per > most ? most : per), 1);
  cfg.blockDim = dim3(256, 1, 1);
  cfg.dynamicSmemBytes = 0;
  REST_CUDA_TRY(cudaLaunchKernelEx(&cfg, paged_attention_join_kernel<T, D>, a));
  rest::count_launch();
  return REST_OK;
}

template <typename T, int D>
rest_status pick(const Args& a, const CUtensorMap& tm_k, const CUtensorMap& tm_v, const Plan& pl, int slot, cudaStream_t st) {
  slot += rest::kSmemSlotPaged;
  if (pl.NT == 2) return run<T, D, 2, 1>(a, tm_k, tm_v, slot, st);
  if (pl.rows > 64) return run<T, D, 1, 1>(a, tm_k, tm_v, slot + 1, st);
  if (pl.rows > 32) return run<T, D, 1, 2>(a, tm_k, tm_v, slot + 2, st);
  return run<T, D, 1, 4>(a, tm_k, tm_v, slot + 3, st);
}

}  // namespace

// error bits of this file's kernels, read and cleared (see rest_device_error_flags)
rest_status rest::take_paged_error_flags(uint32_t* h_flags) {
  unsigned int v = 0, zero = 0;
  REST_CUDA_TRY(cudaMemcpyFromSymbol(&v, g_paged_error, sizeof(v)));
  if (v != 0) REST_CUDA_TRY(cudaMemcpyToSymbol(g_paged_error, &zero, sizeof(zero)));
  *h_flags = v;
  return REST_OK;
}

extern "C" size_t rest_paged_attention_workspace_bytes(int32_t B, int32_t H, int32_t H_kv, int32_t N, int32_t D) {
  if (B <= 0 || H <= 0 || H_kv <= 0 || N <= 0 || N > REST_MAX_N || (D != 64 && D != 128) || H % H_kv) return 0;
  return workspace_bytes(plan(H, H_kv, N), D);
}

extern "C" rest_status rest_paged_attention(const void* d_q, const void* d_k_pages, const void* d_v_pages,
                                            const int64_t* strides, int32_t dtype, int32_t P, int32_t page,
                                            const int32_t* d_table, int64_t table_stride, int32_t table_cols,
                                            const int32_t* d_kv_len, const int32_t* d_n_nodes,
                                            const uint32_t* d_mask, int32_t B, int32_t H, int32_t H_kv, int32_t N,
                                            int32_t D, int32_t window, int32_t sinks, float scale, void* d_out,
                                            float* d_lse, void* d_ws, size_t ws_bytes, void* stream) {
  if (B < 0 || H < 1 || H_kv < 1 || N < 1 || !strides || window < 0 || sinks < 0 || P < 1) return REST_INVALID_ARG;
  if (dtype != REST_BF16 && dtype != REST_FP16) return REST_INVALID_ARG;
  if (B == 0) return REST_OK;
  if (!d_q || !d_k_pages || !d_v_pages || !d_table || !d_kv_len || !d_out) return REST_INVALID_ARG;
  if (table_cols < 1 || table_stride < table_cols) return REST_INVALID_ARG;
  if (!(scale > 0.f) || !(scale < INFINITY)) return REST_INVALID_ARG;
  if ((D != 64 && D != 128) || N > REST_MAX_N || (H % H_kv) != 0) return REST_UNSUPPORTED;
  if (page < 16 || page > 256 || (page & (page - 1)) != 0 || (int64_t)table_cols * page > 0x7FFF0000ll ||
      H > 65536 || H / H_kv > 1024)
    return REST_UNSUPPORTED;
  const int64_t extent[9] = {B, N, H, P, H_kv, page, B, N, H};
  for (int i = 0; i < 9; ++i) {
    if (strides[i] < 0 || (strides[i] % 8) != 0) return REST_INVALID_ARG;
    if (extent[i] > 1 && strides[i] < D) return REST_INVALID_ARG;
  }
  if ((reinterpret_cast<uintptr_t>(d_q) | reinterpret_cast<uintptr_t>(d_k_pages) |
       reinterpret_cast<uintptr_t>(d_v_pages) | reinterpret_cast<uintptr_t>(d_out) | reinterpret_cast<uintptr_t>(d_ws)) & 15)
    return REST_INVALID_ARG;
  const Plan pl = plan(H, H_kv, N);
  if (!d_ws) return REST_INVALID_ARG;
  if (ws_bytes < workspace_bytes(pl, D)) return REST_WORKSPACE_TOO_SMALL;
  Args a;
  a.q = d_q; a.k = d_k_pages; a.v = d_v_pages; a.out = d_out; a.lse = d_lse;
  a.table = d_table; a.kv_len = d_kv_len; a.n_nodes = d_n_nodes; a.mask = d_mask;
  a.q_b = strides[0]; a.q_n = strides[1]; a.q_h = strides[2];
  a.p_p = strides[3]; a.p_h = strides[4]; a.p_r = strides[5];
  a.o_b = strides[6]; a.o_n = strides[7]; a.o_h = strides[8];
  a.table_stride = table_stride;
  a.B = B; a.H = H; a.H_kv = H_kv; a.G = H / H_kv; a.N = N; a.Wm = (N + 31) / 32; a.P = P; a.table_cols = table_cols;
  a.window = window; a.sinks = sinks; a.teams = pl.teams; a.teams_last = pl.teams_last; a.RB = pl.RB; a.rows = pl.rows;
  a.g_inverse = (uint32_t)((((u64)1 << 32) + a.G - 1) / a.G);
  a.scale_log2 = scale * kLog2e;
  a.page_log = 4;
  while ((1 << a.page_log) < page) ++a.page_log;
  const size_t blocks = blocks_of(pl);
  a.meta = reinterpret_cast<int4*>((reinterpret_cast<uintptr_t>(d_ws) + 31) & ~(uintptr_t)31);     // 32-byte stores
  a.ws_o = reinterpret_cast<float*>(a.meta + (blocks + 1) / 2 * 2);
  a.ws_ml = a.ws_o + blocks * 2 * pl.rows * D;
  const int bn = 64;                                    // keys per tile
  CUtensorMap tm_k, tm_v;
  if (!encode_pool(&tm_k, d_k_pages, dtype, D, page, H_kv, P, strides + 3, page < bn ? page : bn, a.slot) ||
      !encode_pool(&tm_v, d_v_pages, dtype, D, page, H_kv, P, strides + 3, page < bn ? page : bn, a.slot))
    return rest::note_cuda_error(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool bf16 = dtype == REST_BF16;
  if (D == 128) return bf16 ? pick<__nv_bfloat16, 128>(a, tm_k, tm_v, pl, 0, st) : pick<__half, 128>(a, tm_k, tm_v, pl, 4, st);
  return bf16 ? pick<__nv_bfloat16, 64>(a, tm_k, tm_v, pl, 8, st) : pick<__half, 64>(a, tm_k, tm_v, pl, 12, st);
}
