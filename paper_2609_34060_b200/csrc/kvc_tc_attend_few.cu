// kvc_attend for few rows a request and KV head (single tokens, short drafts): the keys are the long side, so they take
// the long side of the products.
//
//     S^T = K Q^T   (128 tokens x rows) ,   O^T += V^T P^T   (d x rows) ,
// a tile of 128 tokens lies in the 128 lanes of tensor memory, a softmax thread owns one token and holds its logits of
// all rows.  Bound: the bytes of K and V.  The tiles go from HBM to shared memory by TMA and straight into the tensor
// cores; registers only see rows x 128 logits a tile.
//
// Work: all (request, KV head) pairs one after the other form one line of key tiles, of which every SM's block takes an
// equal part (ragged batches balance to a tile, whatever their lengths).  A block finishes the pairs that lie inside its
// part; of a pair cut by its borders it leaves a float32 partial result (at most two a block), and a second kernel joins
// those in a fixed order.
//
// Two groups of four softmax warps take the tiles in turn, each with running maxima, sums and accumulators of its own (a
// tile's way from logits to probabilities is a chain of latencies, longer than a tile's bytes take); a pair's two halves
// are put together like the pieces of a split.
//
// Softmax: the running maximum of a row moves only when a logit exceeds it by 2^kLazy (one vote a tile, no reduction
// otherwise); the sum is kept per thread and added up at the end.
//
// 8-bit caches are not converted: the tensor cores take the codes.  A query row is split into two e4m3 parts,
//     q 2^-b = t1 + t2 / 16   (b the row's exponent; bf16 has 8 significant bits, each part 4: exact but for channels
//                              below 2^-15 of the row's largest, which are off by at most 2^-22 of it) ,
// as separate columns of one product, K's scale multiplies the finished logit (a token's scale is its thread's), and
// V's scale e_v goes into the probability before that is split into three parts 16 apart,
//     64 2^(s + e_v - Z) = t1 + t2 / 16 + t3 / 256   (s the logit to base 2, Z the row's largest s + e_v so far) ,
// 12 bits and a step of 2^-24 of the row's largest term p 2^e_v.  The reference is the product's, not the largest exponent
// alone: a large value row that a row of queries does not see, or hardly looks at, costs the others no bits.  The sum of
// the probabilities has its own reference, the largest s, and its own exponentials (eight requests of 32K: 113.8 us, 113.4
// with one exponential for both).
// Sums and joins are float32.  Over bf16 caches P is rounded to bf16 as in the chunk kernel.
//
// Measured: 64 requests of 4K (lognormal), 32 / 8 heads, bf16 pages of 16: 202-206 us = 6.3 TB/s of 6.55 copied; eight
// requests of 32K, 64 / 8 heads, 8-bit pages of 16: 110-114 us (100 with pages of 128: the copies of 2 KB boxes then bound it,
// and 12 us are start and join); one request of 777 keys: 11 us, of which 2 are the join's; one of 30K, 8 / 1 heads: 25 us
// (31 with the join loading a piece's sums after its weights, eight at a time).
//
// Warps: 0-3 and 4-7 softmax (0-3 epilogue), 8 first products, 9 second products, 10 queries of the next pair, 12-15
// loads: keys and values of even and odd tiles, with the exponents of 8-bit rows (a 16-token page is one small box, and
// one or two warps issuing them all were the bound: 8-bit batch at 32K 120 us with two).  Every wait is bounded.
#include <cuda_runtime.h>

#include "kvc_launch.h"
#include "kvc_tc.h"
#include "kvc_tc_attend.cuh"
#include "kvc_tc_attend_few.h"

namespace kvc {
namespace {

using namespace tc;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct FewLaunch {
  AttendLaunch a;
  TileGeo g;
  int32_t blocks;              // of the main kernel
  float* part;                 // [blocks][2][RC][D], then [blocks][2][RC][2]
};

// tiles of a (request, head) pair; 0: the request is not this kernel's
__device__ __forceinline__ int few_tiles(const AttendLaunch& a, int rc, int nq, int kv) {
  const int64_t rows = (int64_t)nq * a.G;
  return rows == 0 || rows > rc ? 0 : kv <= 0 ? 1 : (kv + 127) >> 7;
}

struct Piece {
  int b, h, q0, nq, kv, nt, t0, t1;
};

// A position on the line of tiles: request, head, tile, and how many tiles the walk still takes; the numbers of the
// request looked at last (`known`) stay with it.
struct Walk {
  int64_t left;
  int b, h, t;
  int known, q0, nq, kv, nt;
  __device__ __forceinline__ bool next(const AttendLaunch& a, int rc, Piece& x) {
    if (left <= 0) return false;
    for (;; ++b) {
      if (b >= a.req.n) return false;
      if (b != known) {
        request_span(a.req, b, nullptr, q0, nq, kv);
        nt = few_tiles(a, rc, nq, kv);
        known = b;
      }
      if (nt > 0) break;
    }
    x.b = b;
    x.h = h;
    x.q0 = q0;
    x.nq = nq;
    x.kv = kv;
    x.nt = nt;
    x.t0 = t;
    x.t1 = (int64_t)(nt - t) < left ? nt : t + (int)left;
    left -= x.t1 - x.t0;
    t = 0;
    if (++h == a.H) {
      h = 0;
      ++b;
    }
    return true;
  }
};

__device__ __forceinline__ int64_t warp_scan(int64_t v, int lane) {   // inclusive
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  return v;
}
// tiles of requests [0, n) (whole warp)
__device__ __forceinline__ int64_t line_length(const AttendLaunch& a, int rc, int lane, int n) {
  int64_t mine = 0;
  for (int b = lane; b < n; b += 32) {
    int q0, nq, kv;
    request_span(a.req, b, nullptr, q0, nq, kv);
    mine += (int64_t)few_tiles(a, rc, nq, kv) * a.H;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
  return mine;
}

// Where block c's part of a line of `total` tiles begins; with fewer tiles than blocks, the first `total` blocks take one each.
__device__ __forceinline__ int64_t line_cut(int64_t total, int c, int blocks) {
  if (total <= blocks) return c < total ? c : total;
  if (total < ((int64_t)1 << 31) / blocks) return (uint32_t)total * (uint32_t)c / (uint32_t)blocks;
  return total * c / blocks;
}

// The start of block c's part (whole warp): up to 32 requests are read once.
__device__ __forceinline__ Walk line_start(const AttendLaunch& a, int rc, int lane, int c, int blocks) {
  const int n = a.req.n;
  int q0 = 0, nq = 0, kv = 0, nt = 0;
  if (lane < n) {
    request_span(a.req, lane, c == 0 ? a.status : nullptr, q0, nq, kv);
    nt = few_tiles(a, rc, nq, kv);
  }
  int64_t incl = warp_scan((int64_t)nt * a.H, lane), total = __shfl_sync(0xffffffffu, incl, 31);
  for (int b0 = 32; b0 < n; b0 += 32) {
    int64_t mine = 0;
    if (b0 + lane < n) {
      int x, y, z;
      request_span(a.req, b0 + lane, c == 0 ? a.status : nullptr, x, y, z);
      mine = (int64_t)few_tiles(a, rc, y, z) * a.H;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
    total += mine;
  }
  const int64_t lo = line_cut(total, c, blocks), hi = line_cut(total, c + 1, blocks);
  Walk w{hi - lo, 0, 0, 0, -1, 0, 0, 0, 0};
  if (hi <= lo) return w;
  int64_t before = 0;
  for (int b0 = 0; b0 < n; b0 += 32) {
    if (b0 > 0) {
      q0 = nq = kv = nt = 0;
      if (b0 + lane < n) {
        request_span(a.req, b0 + lane, nullptr, q0, nq, kv);
        nt = few_tiles(a, rc, nq, kv);
      }
      incl = warp_scan((int64_t)nt * a.H, lane);
    }
    const unsigned hit = __ballot_sync(0xffffffffu, before + incl > lo);
    if (hit) {
      const int l = __ffs(hit) - 1;
      w.b = w.known = b0 + l;
      w.q0 = __shfl_sync(0xffffffffu, q0, l);
      w.nq = __shfl_sync(0xffffffffu, nq, l);
      w.kv = __shfl_sync(0xffffffffu, kv, l);
      w.nt = __shfl_sync(0xffffffffu, nt, l);
      const int64_t off = lo - before - (__shfl_sync(0xffffffffu, incl, l) - (int64_t)w.nt * a.H);   // below H nt
      w.h = off < ((int64_t)1 << 31) ? (int)((uint32_t)off / (uint32_t)w.nt) : (int)(off / w.nt);
      w.t = (int)(off - (int64_t)w.h * w.nt);
      return w;
    }
    before += __shfl_sync(0xffffffffu, incl, 31);
  }
  return w;
}

template <int D, bool Q8, int RC>
struct Few {
  static constexpr int E = Q8 ? 1 : 2;
  static constexpr int kRows = RC;
  static constexpr int kTile = 128 * D * E;
  static constexpr int kSlots = kTile == 32768 ? 6 : Q8 && D == 128 && RC > 8 ? 10 : 12;
  static constexpr int kQRows = Q8 ? 2 * RC : RC < 16 ? 16 : RC;   // rows of the query operand: N of the first product
  static constexpr int kQ = kQRows * D * E;
  static constexpr int kPCols = Q8 ? (RC == 8 ? 32 : 3 * RC) : RC < 16 ? 16 : RC;   // N of the second product
  static constexpr int kLogits = Q8 ? 2 * RC : RC;             // columns of logits that are read
  static constexpr int kPRow = Q8 ? (RC == 8 ? 32 : RC == 16 ? 64 : 128) : RC < 16 ? 32 : 2 * RC;   // bytes of a token's probabilities
  static constexpr uint32_t kPSwizzle = kPRow == 32 ? 6 : kPRow == 64 ? 4 : 2;
  static constexpr uint32_t kRowSwizzle = Q8 && D == 64 ? 4 : 2;
  static constexpr int kP = 128 * kPRow;
  static constexpr int kThreads = 512;
  static constexpr int kExpRing = Q8 ? 8 : 2;
  static constexpr int kQAlign = (kQ + 1023) / 1024 * 1024;
  static constexpr int kSmem = 1024 + kSlots * kTile + 2 * kQAlign + 2 * kP + (Q8 ? kExpRing * 1024 : 0);
  // logits of kSBufs tiles (the first products run kSBufs - 1 tiles ahead), then accumulators of (pair parity, group)
  static constexpr int kSBufs = Q8 && RC == 32 ? 2 : 4;
  static constexpr uint32_t kOCol = kSBufs * kQRows;
  static constexpr uint32_t kTmem = kOCol + 4 * kPCols <= 128 ? 128 : kOCol + 4 * kPCols <= 256 ? 256 : 512;
  static_assert(kOCol + 4 * kPCols <= 512, "tensor memory");
  // p <= 2^kLazy; with 8-bit values 64 2^(s + e_v - Z) <= 64 2^kLazyZ has to stay below 448
  static constexpr float kLazy = 8.f, kLazyZ = 2.f;
};

// 8-bit caches: maxima of s + e_v; a warp's copy of Z - 6 (0 while there is none) and of what a new Z does to the sums;
// group 1's Z - 6 of a finished piece
template <bool Q8, int RC>
struct FewScales {};
template <int RC>
struct alignas(16) FewScales<true, RC> {
  float z[2][4][RC], z_keep[2][4][RC], red_z[2][4][RC], half_z[RC];
};
template <typename F>
struct FewBars : FewScales<F::E == 1, F::kRows> {
  uint64_t full[F::kSlots], empty[F::kSlots], s_full[F::kSBufs], s_free[F::kSBufs], p_ready[2], pv_done[2], q_full[2], q_empty[2], o_free[2];
  uint64_t e_full[F::kExpRing], e_empty[F::kExpRing];
  Walk start;
  uint32_t tmem;
  int abort_flag;
  int64_t row_at[F::kRows];         // where a row of the finished pair goes
  float red[2][4][F::kRows];
  float qs[2][F::E == 1 ? F::kRows : 1];   // scales of the query rows (8-bit caches)
  float half[2][F::kRows];          // group 1's sums and maxima of a finished piece; then the weights of the two halves
  int fail[2][4];
};

template <int N>
__device__ __forceinline__ void tmem_ld(uint32_t taddr, float* v) {
  static_assert(N % 8 == 0, "columns");
#pragma unroll
  for (int k = 0; k < N; k += 8) tmem_ld8(taddr + k, v + k);
}
// largest of a warp's values (NaN does not count)
__device__ __forceinline__ float warp_max(float v) {
  float m;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(v));
  return m;
}
// 16-byte chunk of a token's row of probabilities under the row's swizzle
template <int ROW>
__device__ __forceinline__ int p_chunk(int chunk, int tok) {
  return ROW == 32 ? chunk ^ ((tok >> 2) & 1) : ROW == 64 ? chunk ^ ((tok >> 1) & 3) : chunk ^ (tok & 7);
}

static_assert(sizeof(FewBars<Few<128, false, 32>>) + Few<128, false, 32>::kSmem <= 232448, "shared memory");
static_assert(sizeof(FewBars<Few<128, false, 16>>) + Few<128, false, 16>::kSmem <= 232448, "shared memory");
static_assert(sizeof(FewBars<Few<128, true, 8>>) + Few<128, true, 8>::kSmem <= 232448, "shared memory");
static_assert(sizeof(FewBars<Few<128, true, 16>>) + Few<128, true, 16>::kSmem <= 232448, "shared memory");
static_assert(sizeof(FewBars<Few<128, true, 32>>) + Few<128, true, 32>::kSmem <= 232448, "shared memory");

// kTree: a request's new tokens (at most RC, so that a row's mask is one word) form a tree; a row sees the context and those
// new tokens whose bits are set in its mask.
template <int D, bool Q8, int RC, bool kTree>
__global__ void __launch_bounds__(Few<D, Q8, RC>::kThreads, 1)
attend_few_kernel(const __grid_constant__ FewLaunch p, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  using F = Few<D, Q8, RC>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ FewBars<F> bars;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* skv = smem;
  uint8_t* sq = skv + F::kSlots * F::kTile;
  uint8_t* sp = sq + 2 * F::kQAlign;
  float* sexp = reinterpret_cast<float*>(sp + 2 * F::kP);          // [kExpRing][2][128]
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  volatile int* abort_flag = &bars.abort_flag;
  const uint32_t full = smem_u32(bars.full), empty = smem_u32(bars.empty), s_full = smem_u32(bars.s_full), s_free = smem_u32(bars.s_free), p_ready = smem_u32(bars.p_ready);
  const uint32_t pv_done = smem_u32(bars.pv_done), q_full = smem_u32(bars.q_full), q_empty = smem_u32(bars.q_empty);
  const uint32_t o_free = smem_u32(bars.o_free), e_full = smem_u32(bars.e_full), e_empty = smem_u32(bars.e_empty);
  if (tid == 0) {
    for (int s = 0; s < F::kSlots; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(empty + 8 * s, 1);
    }
    for (int s = 0; s < F::kSBufs; ++s) {
      mbar_init(s_full + 8 * s, 1);
      mbar_init(s_free + 8 * s, 4);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(p_ready + 8 * s, 128);
      mbar_init(pv_done + 8 * s, 1);
      mbar_init(q_full + 8 * s, 32);
      mbar_init(q_empty + 8 * s, 1 + 8);                             // the products and the eight softmax warps
      mbar_init(o_free + 8 * s, 128);
    }
    for (int s = 0; s < F::kExpRing; ++s) {
      mbar_init(e_full + 8 * s, 64);                                 // the tile's two loading warps
      mbar_init(e_empty + 8 * s, 128);
    }
    bars.abort_flag = 0;
    fence_barrier_init();
  }
  if (tid == 32) {
    prefetch_map(&map_k);
    prefetch_map(&map_v);
  }
  if (warp == 9) {
    tmem_alloc(smem_u32(&bars.tmem), F::kTmem);
    tmem_relinquish();
  }
  grid_dependency_wait();          // what follows reads what earlier kernels wrote
  if (warp == 11) {
    const Walk w = line_start(p.a, RC, lane, (int)blockIdx.x, p.blocks);
    if (lane == 0) bars.start = w;
  }
  grid_dependents_launch();        // the join's blocks may take the SMs that finish first
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars.tmem;
  Walk walk = bars.start;
  Piece x;
  const uint32_t gs = (uint32_t)p.g.gs, ps = (uint32_t)p.g.ps;

  if (warp < 8) {
    regs_inc<184>();
    const int wg = warp >> 2, tid4 = tid & 127, w4 = warp & 3;
    const uint32_t lane_at = tmem + ((uint32_t)(w4 * 32) << 16);
    const float minus_inf = __uint_as_float(0xff800000u);
    const float c = p.a.scale * kLog2e;
    int g = 0, piece = 0;
    // a failed wait (ok) becomes a decision of the group's four warps (stop) at the vote of its next tile: a warp that
    // left alone would leave the others at a barrier.  The groups meet at one barrier a piece, which both always reach.
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity) { ok = ok && wait_all(bar, parity, abort_flag); };
    while (walk.next(p.a, RC, x)) {
      const int R = x.nq * p.a.G;
      const uint32_t o_at = lane_at + F::kOCol + ((piece & 1) * 2 + wg) * F::kPCols;
      float m[RC], l[RC];
      uint32_t mask_lane = 0;                                       // kTree: mask of row `lane`
      if (kTree && lane < R) mask_lane = __ldg(p.a.mask + (int64_t)(x.q0 + lane / p.a.G) * p.a.words);
      float z_lane = minus_inf;                                     // 8-bit values: Z - 6 of row `lane`, under which its sums are held
#pragma unroll
      for (int r = 0; r < RC; ++r) {
        m[r] = minus_inf;
        l[r] = 0.f;
      }
      if constexpr (Q8) {
        if (lane < RC) bars.z[wg][w4][lane] = 0.f;
        __syncwarp();
      }
      wait(q_full + 8 * (piece & 1), (piece >> 1) & 1);
      const int g0 = g, g1 = g + x.t1 - x.t0;                       // the piece's tiles in the block's count
      const int first = g0 + ((g0 ^ wg) & 1);                       // this group's first
      bool stop = false;
      for (g = first; g < g1; g += 2) {
        const int i = x.t0 + g - g0;
        const int tok = i * 128 + tid4;
        const uint32_t use = (uint32_t)(g >> 1) & 1u;               // of buffer wg
        float ek = 1.f, ev = 0.f;
        if (Q8) {
          const int es = g % F::kExpRing;
          wait(e_full + 8 * es, (g / F::kExpRing) & 1);
          ek = sexp[es * 256 + tid4];
          ev = sexp[es * 256 + 128 + tid4];
          mbar_arrive(e_empty + 8 * es);
        }
        const int sb = g % F::kSBufs;
        wait(s_full + 8 * sb, (g / F::kSBufs) & 1);
        tc_fence_after();
        float s[F::kLogits];
        tmem_ld<F::kLogits>(lane_at + sb * F::kQRows, s);
        tmem_ld_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(s_free + 8 * sb);
#pragma unroll
        for (int r = 0; r < RC; ++r) s[r] = Q8 ? fmaf(s[(Q8 ? RC : 0) + r], 0.0625f, s[r]) * (bars.qs[piece & 1][Q8 ? r : 0] * ek) : s[r] * c;
        if (x.kv - x.nq < i * 128 + 128) {                          // the last keys, or some that early rows do not see
          const int lim = p.a.causal ? x.kv - x.nq : x.kv - 1;
#pragma unroll
          for (int r = 0; r < RC; ++r)
            if (tok > lim + (p.a.causal ? r / p.a.G : 0) || r >= R) s[r] = minus_inf;
          if (kTree) {
            const int fresh = tok - lim;                            // the key's place among the new tokens
#pragma unroll
            for (int r = 0; r < RC; ++r) {
              const uint32_t mask = __shfl_sync(0xffffffffu, mask_lane, r);
              if (fresh >= 0 && !((mask >> (fresh & 31)) & 1u)) s[r] = minus_inf;
            }
          }
        }
        bool grow = false;
#pragma unroll
        for (int r = 0; r < RC; ++r) grow |= s[r] - m[r] > F::kLazy;
        if constexpr (Q8) {
#pragma unroll
          for (int r = 0; r < RC; r += 4) {
            const float4 z = *reinterpret_cast<const float4*>(&bars.z[wg][w4][r]);
            grow |= s[r] + (ev - z.x) > F::kLazyZ + 6.f || s[r + 1] + (ev - z.y) > F::kLazyZ + 6.f;
            grow |= s[r + 2] + (ev - z.z) > F::kLazyZ + 6.f || s[r + 3] + (ev - z.w) > F::kLazyZ + 6.f;
          }
        }
        if (named_bar_or(1 + wg, 128, grow || !ok)) {
          float keep[RC];
#pragma unroll
          for (int r = 0; r < RC; ++r) {
            const float v = warp_max(s[r]);
            if (lane == 0) bars.red[wg][w4][r] = v;
            if constexpr (Q8) {
              const float z = warp_max(s[r] + ev);
              if (lane == 0) bars.red_z[wg][w4][r] = z;
            }
          }
          if (lane == 0) bars.fail[wg][w4] = !ok;
          named_bar_sync(1 + wg, 128);
          if (bars.fail[wg][0] | bars.fail[wg][1] | bars.fail[wg][2] | bars.fail[wg][3]) {
            stop = true;
            break;
          }
          if constexpr (Q8) {
            // a lane a row, in every warp alike
            if (lane < RC) {
              const int r = lane;
              const float top = fmaxf(z_lane, fmaxf(fmaxf(bars.red_z[wg][0][r], bars.red_z[wg][1][r]), fmaxf(bars.red_z[wg][2][r], bars.red_z[wg][3][r])) - 6.f);
              bars.z_keep[wg][w4][r] = top == z_lane || z_lane == minus_inf ? 1.f : exp2_fast(z_lane - top);
              bars.z[wg][w4][r] = top == minus_inf ? 0.f : top;
              z_lane = top;
            }
            __syncwarp();
          }
#pragma unroll
          for (int r = 0; r < RC; ++r) {
            const float top = fmaxf(m[r], fmaxf(fmaxf(bars.red[wg][0][r], bars.red[wg][1][r]), fmaxf(bars.red[wg][2][r], bars.red[wg][3][r])));
            keep[r] = top == m[r] ? 1.f : exp2_fast(m[r] - top);
            m[r] = top;
            l[r] *= keep[r];
          }
          if (g > first) {
            // the sums so far, once the product that wrote them last is done
            wait(pv_done + 8 * wg, use ^ 1);
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < (Q8 ? 3 * RC : RC); k += 8) {
              float o[8];
              tmem_ld8(o_at + k, o);
              tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                if constexpr (Q8)
                  o[j] *= bars.z_keep[wg][w4][(k + j) % RC];
                else
                  o[j] *= keep[(k + j) % RC];
              }
              tmem_st8(o_at + k, reinterpret_cast<const uint32_t*>(o));
            }
            tmem_st_wait();
          }
        }
        // probabilities; the buffer is free once the product that read it last is done
        wait(pv_done + 8 * wg, use ^ 1);
        uint8_t* row = sp + wg * F::kP + tid4 * F::kPRow;
        uint32_t w[F::kPRow / 4];
#pragma unroll
        for (int r = 0; r < RC; r += Q8 ? 4 : 2) {
          float e[4];
#pragma unroll
          for (int j = 0; j < (Q8 ? 4 : 2); ++j) {
            e[j] = exp2_fast(s[r + j] - (m[r + j] == minus_inf ? 0.f : m[r + j]));
            l[r + j] += e[j];
          }
          if constexpr (Q8) {
            const float4 z = *reinterpret_cast<const float4*>(&bars.z[wg][w4][r]);
            e[0] = exp2_fast(s[r] + (ev - z.x));
            e[1] = exp2_fast(s[r + 1] + (ev - z.y));
            e[2] = exp2_fast(s[r + 2] + (ev - z.z));
            e[3] = exp2_fast(s[r + 3] + (ev - z.w));
#pragma unroll
            for (int term = 0; term < 3; ++term) {
              const uint32_t lo = e4m3x2(e[0], e[1]), hi = e4m3x2(e[2], e[3]);
              w[(term * RC + r) / 4] = lo | (hi << 16);
              const float2 a = e4m3x2_to_float2(lo), b = e4m3x2_to_float2(hi);
              e[0] = (e[0] - a.x) * 16.f;
              e[1] = (e[1] - a.y) * 16.f;
              e[2] = (e[2] - b.x) * 16.f;
              e[3] = (e[3] - b.y) * 16.f;
            }
          } else {
            w[r / 2] = pack2(e[0], e[1]);
          }
        }
#pragma unroll
        for (int k = (Q8 ? 3 * RC : 2 * RC) / 4; k < F::kPRow / 4; ++k) w[k] = 0;
#pragma unroll
        for (int k = 0; k < F::kPRow / 16; ++k)
          *reinterpret_cast<uint4*>(row + (p_chunk<F::kPRow>(k, tid4) << 4)) = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
        if (x.kv < i * 128 + 128) {
          // stale rows behind the last key: P is zero there, but zero times a stale NaN would not be
          const int vs = (2 * g + 1) % F::kSlots;
          wait(full + 8 * vs, ((2 * g + 1) / F::kSlots) & 1);
          if (tok >= x.kv) {
            uint8_t* v = skv + vs * F::kTile + (tid4 >> 3) * gs + (tid4 & 7) * (Q8 ? D : 128);
#pragma unroll
            for (int k = 0; k < D * F::E / 16; ++k) *reinterpret_cast<uint4*>(v + (Q8 ? k << 4 : (k >> 3) * ps + ((k & 7) << 4))) = make_uint4(0, 0, 0, 0);
          }
        }
        fence_proxy_async();
        tc_fence_before();
        mbar_arrive(p_ready + 8 * wg);
      }
      g = g1;
      const int last = g1 - 1 - (((g1 - 1) ^ wg) & 1);              // this group's last tile; before g0: it had none
      if (last >= g0 && !stop) wait(pv_done + 8 * wg, (uint32_t)(last >> 1) & 1u);
      tc_fence_after();
      // sums of the rows over the group's threads
      named_bar_sync(1 + wg, 128);                                  // everyone is done with red
#pragma unroll
      for (int r = 0; r < RC; ++r) {
        float v = l[r];
#pragma unroll
        for (int k = 16; k > 0; k >>= 1) v += __shfl_xor_sync(0xffffffffu, v, k);
        if (lane == 0) bars.red[wg][w4][r] = v;
      }
      named_bar_sync(1 + wg, 128);
      if (wg == 1) {
        named_bar_sync(4, 256);                                     // group 0 has read the last piece's half
        if (tid4 < RC) bars.half[0][tid4] = last >= g0 ? (bars.red[1][0][tid4] + bars.red[1][1][tid4]) + (bars.red[1][2][tid4] + bars.red[1][3][tid4]) : 0.f;
        if (tid4 == 0) {
#pragma unroll
          for (int r = 0; r < RC; ++r) bars.half[1][r] = m[r];
        }
        if constexpr (Q8)
          if (tid4 < RC) bars.half_z[tid4] = z_lane;                // warp 0: lane r has row r's
        tc_fence_before();                                          // group 0 reads this group's accumulators
        named_bar_sync(3, 256);
      } else {
        named_bar_sync(4, 256);
        named_bar_sync(3, 256);
        tc_fence_after();
        const bool had0 = last >= g0, had1 = g1 - g0 > 1 || !had0;  // which groups had tiles
        const uint32_t o0 = o_at, o1 = o_at + F::kPCols;
        const bool whole = x.t0 == 0 && x.t1 == x.nt;
        const int64_t slot = ((int64_t)blockIdx.x * 2 + (x.t0 > 0 ? 0 : 1)) * RC;
        // a thread a row: weights of the halves, place of the result
        if (tid4 < R) {
          const int r = tid4;
          float mr = minus_inf;
#pragma unroll
          for (int k = 0; k < RC; ++k) mr = k == r ? m[k] : mr;
          const float l0 = (bars.red[0][0][r] + bars.red[0][1][r]) + (bars.red[0][2][r] + bars.red[0][3][r]), l1 = bars.half[0][r], m1 = bars.half[1][r];
          // a half that saw no key of the row (l = 0) gets no weight, whatever its accumulators hold
          const float top = l1 == 0.f ? mr : l0 == 0.f ? m1 : fmaxf(mr, m1);
          float w0 = l0 == 0.f ? 0.f : exp2_fast(mr - top), w1 = l1 == 0.f ? 0.f : exp2_fast(m1 - top);
          const float sum = w0 * l0 + w1 * l1;
          const bool dead = sum == 0.f;
          const float scale = whole ? (dead ? 0.f : 1.f / sum) : 1.f;
          if constexpr (Q8) {
            // sums of codes are held under 2^(Z - 6): 2^(Z - 6 - 127 - top), whose exponent alone may leave float32's range
            const float h0 = exp2_fast(0.5f * (z_lane - 127.f - top)), h1 = exp2_fast(0.5f * (bars.half_z[r] - 127.f - top));
            w0 = h0 * scale * h0;
            w1 = h1 * scale * h1;
          } else {
            w0 *= scale;
            w1 *= scale;
          }
          bars.half[0][r] = had0 && l0 != 0.f ? w0 : 0.f;
          bars.half[1][r] = had1 && l1 != 0.f ? w1 : 0.f;
          if (whole) {
            const int64_t at = x.q0 + r / p.a.G;
            const int head = x.h * p.a.G + r % p.a.G;
            bars.row_at[r] = at * p.a.out.s_row + (int64_t)head * p.a.out.s_head;
            if (p.a.lse && ok) p.a.lse[at * (p.a.H * p.a.G) + head] = dead ? minus_inf : (top + log2f(sum)) * kLn2;
          } else if (ok) {
            *reinterpret_cast<float2*>(p.part + (int64_t)p.blocks * 2 * RC * D + (slot + r) * 2) = make_float2(top, sum);
          }
        }
        named_bar_sync(1, 128);
#pragma unroll
        for (int rb = 0; rb < RC; rb += 8) {
          if (rb >= R) continue;
          float v0[8], v1[8];
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            float* v = half ? v1 : v0;
            const uint32_t at = half ? o1 : o0;
            tmem_ld8(at + rb, v);                                   // of a half without tiles: stale, weight zero
            if (Q8) {
              float a[8], b[8];
              tmem_ld8(at + (Q8 ? RC : 0) + rb, a);
              tmem_ld8(at + (Q8 ? 2 * RC : 0) + rb, b);
              tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 8; ++j) v[j] = fmaf(fmaf(b[j], 0.0625f, a[j]), 0.0625f, v[j]);
            } else {
              tmem_ld_wait();
            }
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int r = rb + j;
            if (r >= R || !ok) continue;
            const float w0 = bars.half[0][r], w1 = bars.half[1][r];
            const float v = (w0 == 0.f ? 0.f : v0[j] * w0) + (w1 == 0.f ? 0.f : v1[j] * w1);
            if (tid4 < D) {
              if (whole)
                p.a.out.p[bars.row_at[r] + tid4] = __float2bfloat16(v);
              else
                p.part[(slot + r) * D + tid4] = v;
            }
          }
        }
        tc_fence_before();
        mbar_arrive(o_free + 8 * (piece & 1));
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(q_empty + 8 * (piece & 1));
      ++piece;
    }
  } else {
    regs_dec<72>();
    if (warp >= 12) {
      // ---- loads: keys (12, 13) or values (14, 15) of every other tile.  A slot's earlier use was consumed before the
      // warp's last load but one could be issued, so a slot's phase is never more than one ahead of the wait.
      const uint32_t ring = smem_u32(skv);
      const int is_v = warp >= 14, odd = warp & 1;
      const CUtensorMap* map = is_v ? &map_v : &map_k;
      const uint8_t* ex = is_v ? p.a.e.v : p.a.e.k;
      int g = 0;
      bool ok = true;
      // exponents, four tokens a lane, handed on one load later than they were asked for
      int held = -1;
      uint32_t bytes[4] = {0, 0, 0, 0};
      bool live[4] = {false, false, false, false};
      auto hand_on = [&]() {
        if (held < 0 || !ok) return;
        const int es = held % F::kExpRing;
        ok = wait_all(e_empty + 8 * es, ((held / F::kExpRing) & 1) ^ 1, abort_flag);
        if (!ok) return;
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = is_v ? (!live[j] ? 0.f : bytes[j] == 255u ? __uint_as_float(0x7fc00000u) : (float)bytes[j]) : live[j] ? exponent_up(bytes[j]) : 1.f;
        *reinterpret_cast<float4*>(sexp + es * 256 + is_v * 128 + lane * 4) = make_float4(v[0], v[1], v[2], v[3]);
        mbar_arrive(e_full + 8 * es);
      };
      while (ok && walk.next(p.a, RC, x)) {
        const int g0 = g, n = x.t1 - x.t0;
        g += n;
        int k = (g0 ^ odd) & 1;                                     // this warp's first tile of the piece
        auto rows_of = [&](int k) { return max(0, min(128, x.kv - (x.t0 + k) * 128)); };
        // page ids a load ahead: nobody waits for the look-up
        int ahead = k < n ? tile_entry(p.a, p.g, x.b, (x.t0 + k) * 128, rows_of(k), lane) : 0;
        for (; k < n; k += 2) {
          const int t0 = (x.t0 + k) * 128, rows = rows_of(k), entry = ahead;
          if (k + 2 < n) ahead = tile_entry(p.a, p.g, x.b, t0 + 256, rows_of(k + 2), lane);
          uint32_t next[4] = {0, 0, 0, 0};
          bool nlive[4] = {false, false, false, false};
          if (Q8) {
            const int tok = t0 + lane * 4;
            int64_t at = (int64_t)p.a.layer * p.a.e.s_layer + (int64_t)x.h * p.a.e.s_head;
            bool good = true;
            if (p.g.paged) {
              const int page = __shfl_sync(0xffffffffu, entry, (lane * 4) >> p.g.box_shift);
              good = (unsigned)page < (unsigned)p.a.c.n_phys;
              at += (int64_t)page * p.a.e.s_page + (int64_t)(tok & p.a.c.page_mask) * p.a.e.s_tok;
            } else {
              at += (int64_t)tok * p.a.e.s_tok;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              nlive[j] = good && tok + j < x.kv;
              if (nlive[j]) next[j] = ex[at + j * p.a.e.s_tok];
            }
          }
          const int use = 2 * (g0 + k) + is_v, slot = use % F::kSlots;
          if (!wait_all(empty + 8 * slot, ((use / F::kSlots) & 1) ^ 1, abort_flag)) {
            ok = false;
            break;
          }
          tile_load<Q8 || D == 64>(map, p.a, p.g, ring + slot * F::kTile, full + 8 * slot, t0, rows, x.h, entry, lane);
          if (Q8) {
            hand_on();
            held = g0 + k;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              bytes[j] = next[j];
              live[j] = nlive[j];
            }
          }
        }
      }
      if (Q8) hand_on();
    } else if (warp == 8 || warp == 9) {
      // ---- products: warp 8 the logits, warp 9 the values
      // descriptors differ in their start address alone (its 18 bits / 16 are the low word); d = 64: the upper 64 rows of
      // the values' product repeat the lower (no distance between the blocks)
      bool ok = true;
      auto wait = [&](uint32_t bar, uint32_t parity) {
        if (ok) ok = wait_all(bar, parity, abort_flag);
        return ok;
      };
      int g = 0, piece = 0, slot = warp == 8 ? 0 : 1;
      uint32_t phase = 0;
      if (warp == 8) {
        constexpr uint32_t idesc = Q8 ? idesc_e4m3(128, F::kQRows, 0, 0) : idesc_bf16(128, F::kQRows, 0, 0);
        constexpr int kSteps = Q8 ? D / 32 : D / 16;
        const uint64_t k_desc = operand_desc(smem_u32(skv), 16, gs, F::kRowSwizzle);
        const uint64_t q_desc = operand_desc(smem_u32(sq), 16, Q8 ? 8 * D : 1024, F::kRowSwizzle);
        const uint32_t k_part = ps >> 4;
        for (; ok && walk.next(p.a, RC, x); ++piece) {
          if (!wait(q_full + 8 * (piece & 1), (piece >> 1) & 1)) break;
          for (int i = x.t0; i < x.t1; ++i, ++g) {
            const int sb = g % F::kSBufs;
            if (!wait(s_free + 8 * sb, ((g / F::kSBufs) & 1) ^ 1) || !wait(full + 8 * slot, phase)) break;
            tc_fence_after();
            const uint64_t kd = k_desc + (uint32_t)(slot * (F::kTile >> 4)), qd = q_desc + (uint32_t)((piece & 1) * (F::kQAlign >> 4));
            const uint32_t to = tmem + sb * F::kQRows;
            const bool end = i + 1 == x.t1;
            if (elect_one()) {
#pragma unroll
              for (int k = 0; k < kSteps; ++k) {
                if (Q8)
                  umma_f8(to, kd + k * 2, qd + k * 2, idesc, k > 0);
                else
                  umma_bf16(to, kd + ((k >> 2) * k_part + (k & 3) * 2), qd + ((k >> 2) * (F::kQRows * 8) + (k & 3) * 2), idesc, k > 0);
              }
              umma_commit(s_full + 8 * sb);
              umma_commit(empty + 8 * slot);
              if (end) umma_commit(q_empty + 8 * (piece & 1));
            }
            slot += 2;
            if (slot >= F::kSlots) {
              slot -= F::kSlots;
              phase ^= 1;
            }
          }
        }
      } else {
        constexpr uint32_t idesc = Q8 ? idesc_e4m3(128, F::kPCols, 1, 1) : idesc_bf16(128, F::kPCols, 1, 1);
        constexpr int kSteps = Q8 ? 4 : 8;
        const uint64_t v_desc = operand_desc(smem_u32(skv), D == 128 && !Q8 ? ps : 0u, gs, F::kRowSwizzle);
        const uint64_t p_desc = operand_desc(smem_u32(sp), 0, 8 * F::kPRow, F::kPSwizzle);
        const uint32_t v_step = ((Q8 ? 4 : 2) * gs) >> 4;
        for (; ok && walk.next(p.a, RC, x); ++piece) {
          if (!wait(o_free + 8 * (piece & 1), ((piece >> 1) & 1) ^ 1)) break;
          for (int i = x.t0; i < x.t1; ++i, ++g) {
            if (!wait(full + 8 * slot, phase) || !wait(p_ready + 8 * (g & 1), (g >> 1) & 1)) break;
            tc_fence_after();
            const uint64_t vd = v_desc + (uint32_t)(slot * (F::kTile >> 4)), pd = p_desc + (uint32_t)((g & 1) * (F::kP >> 4));
            const uint32_t oa = tmem + F::kOCol + ((piece & 1) * 2 + (g & 1)) * F::kPCols;
            const bool acc = i >= x.t0 + 2;                         // the group's first tile of the piece starts its sums
            if (elect_one()) {
#pragma unroll
              for (int k = 0; k < kSteps; ++k) {
                if (Q8)
                  umma_f8(oa, vd + k * v_step, pd + k * (32 * F::kPRow / 16), idesc, acc || k > 0);
                else
                  umma_bf16(oa, vd + k * v_step, pd + k * (16 * F::kPRow / 16), idesc, acc || k > 0);
              }
              umma_commit(pv_done + 8 * (g & 1));
              umma_commit(empty + 8 * slot);
            }
            slot += 2;
            if (slot >= F::kSlots) {
              slot -= F::kSlots;
              phase ^= 1;
            }
          }
        }
      }
    } else if (warp == 10) {
      // ---- queries of the pairs, one pair ahead
      constexpr int LPR = D / 8, RPP = 32 / LPR;
      const int ch = lane % LPR;
      const float c = p.a.scale * kLog2e;
      int piece = 0;
      while (walk.next(p.a, RC, x)) {
        if (!wait_all(q_empty + 8 * (piece & 1), ((piece >> 1) & 1) ^ 1, abort_flag)) break;
        uint8_t* dst = sq + (piece & 1) * F::kQAlign;
        const int R = x.nq * p.a.G;
#pragma unroll 4
        for (int r0 = 0; r0 < (Q8 ? RC : F::kQRows); r0 += RPP) {
          const int r = r0 + lane / LPR;
          uint4 raw = make_uint4(0, 0, 0, 0);
          if (r < R)
            raw = __ldg(reinterpret_cast<const uint4*>(p.a.q.p + (int64_t)(x.q0 + r / p.a.G) * p.a.q.s_row + (int64_t)(x.h * p.a.G + r % p.a.G) * p.a.q.s_head + ch * 8));
          if (!Q8) {
            *reinterpret_cast<uint4*>(dst + (ch >> 3) * (F::kQRows * 128) + (r >> 3) * 1024 + (r & 7) * 128 + (((ch & 7) ^ (r & 7)) << 4)) = raw;
          } else {
            float v[8];
            unpack8(raw, v);
            float top = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(v[j]));
#pragma unroll
            for (int o = LPR / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            const bool finite = top < __uint_as_float(0x7f800000u);
            const uint32_t b = finite ? row_exponent(top) : 127u;
            const float down = exponent_down(b);
#pragma unroll
            for (int term = 0; term < 2; ++term) {
              uint2 code;
              uint32_t w[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                float lo = v[2 * j], hi = v[2 * j + 1];
                if (term == 0) {
                  lo *= down;
                  hi *= down;
                  if (!(fabsf(lo) < __uint_as_float(0x7f800000u))) lo = __uint_as_float(0x7fc00000u);   // infinities give NaN logits
                  if (!(fabsf(hi) < __uint_as_float(0x7f800000u))) hi = __uint_as_float(0x7fc00000u);
                }
                w[j] = e4m3x2(lo, hi);
                const float2 f = e4m3x2_to_float2(w[j]);
                v[2 * j] = (lo - f.x) * 16.f;
                v[2 * j + 1] = (hi - f.y) * 16.f;
              }
              code.x = w[0] | (w[1] << 16);
              code.y = w[2] | (w[3] << 16);
              const int rr = term * RC + r;
              const int chunk = D == 128 ? (ch >> 1) ^ (rr & 7) : (ch >> 1) ^ ((rr >> 1) & 3);
              *reinterpret_cast<uint2*>(dst + rr * D + (chunk << 4) + (ch & 1) * 8) = code;
            }
            if (ch == 0) bars.qs[piece & 1][Q8 ? r : 0] = exponent_up(b) * c;
          }
        }
        fence_proxy_async();
        mbar_arrive(q_full + 8 * (piece & 1));
        ++piece;
      }
    }
  }
  __syncthreads();
  if (*abort_flag) {
    // copies may still be in flight: give them time to land before the block's memory is handed on
    const long long t0 = clock64();
    while (clock64() - t0 < kWaitLimitCycles / 8) {
    }
    if (tid == 0) atomicOr(p.a.status, KVC_FLAG_WAIT_EXPIRED);
    __syncthreads();
  }
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem, F::kTmem);
  }
}

// ---- join of the pieces of a pair that block borders cut; grid: x = (request, head) pairs, y = groups of 4 rows
constexpr int kJoinPieces = 160;   // pieces whose weights are kept at a time
template <int D, int RC>
__global__ void __launch_bounds__(4 * D) attend_few_join_kernel(const __grid_constant__ FewLaunch p) {
  __shared__ int64_t s_total, s_before;
  __shared__ float s_w[4][kJoinPieces], s_m[4], s_l[4];
  const int b = (int)(blockIdx.x / p.a.H), h = (int)(blockIdx.x % p.a.H);
  const int rr = threadIdx.x / D, r = (int)blockIdx.y * 4 + rr, ch = threadIdx.x % D;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  grid_dependents_launch();
  int q0, nq, kv;
  request_span(p.a.req, b, nullptr, q0, nq, kv);
  const int nt = few_tiles(p.a, RC, nq, kv), R = nq * p.a.G;
  const bool none = nt == 0 || (int)blockIdx.y * 4 >= R;
  if (!none && warp < 2) {
    const int64_t sum = line_length(p.a, RC, lane, warp ? p.a.req.n : b);
    if (lane == 0) (warp ? s_total : s_before) = sum;
  }
  // launched while the main kernel ends: its results are there after this wait.  Every block waits, also those with
  // nothing to join: this kernel's end must not come before the main kernel's.
  grid_dependency_wait();
  if (none) return;
  __syncthreads();
  const int64_t total = s_total, w0 = s_before + (int64_t)h * nt, w1 = w0 + nt;
  const int C = (int)(total < p.blocks ? total : p.blocks);
  int c0 = (int)(((w0 + 1) * C + total - 1) / total) - 1, c1 = (int)((w1 * C + total - 1) / total) - 1;   // blocks of the first and last tile
  if (c0 == c1) return;
  const float minus_inf = __uint_as_float(0xff800000u);
  const float* ml = p.part + (int64_t)p.blocks * 2 * RC * D;
  // where block c left its piece: slot 1 holds a piece that begins with the pair, slot 0 one cut in front
  auto place = [&](int c) { return ((int64_t)c * 2 + (c == c0 ? 1 : 0)) * RC; };
  // sums of the first pieces are under way before their weights are known, and always kAtOnce of them
  constexpr int kAtOnce = 16;
  const int pieces = c1 + 1 - c0;
  float x[kAtOnce];
  auto load = [&](int i0) {
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) x[k] = r < R && i0 + k < pieces ? p.part[(place(c0 + i0 + k) + r) * D + ch] : 0.f;
  };
  load(0);
  // maxima and weights: a warp a row, the first pieces' kept
  const int mine = (int)blockIdx.y * 4 + warp;
  auto held = [&](int i) {
    return warp < 4 && mine < R && i < pieces ? *reinterpret_cast<const float2*>(ml + 2 * (place(c0 + i) + mine)) : make_float2(0.f, 0.f);
  };
  float2 v[kJoinPieces / 32];
  float m = minus_inf;
  for (int i0 = (pieces - 1) / kJoinPieces * kJoinPieces; i0 >= 0; i0 -= kJoinPieces) {
#pragma unroll
    for (int k = 0; k < kJoinPieces / 32; ++k) v[k] = held(i0 + k * 32 + lane);
#pragma unroll
    for (int k = 0; k < kJoinPieces / 32; ++k)
      if (v[k].y != 0.f) m = fmaxf(m, v[k].x);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  float acc = 0.f, all = 0.f;
  for (int i0 = 0; i0 < pieces; i0 += kJoinPieces) {
    const int n = min(kJoinPieces, pieces - i0);
    __syncthreads();
    if (warp < 4) {
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < kJoinPieces / 32; ++k) {
        if (i0 > 0) v[k] = held(i0 + k * 32 + lane);
        const float w = v[k].y == 0.f ? 0.f : exp2f(v[k].x - m);
        s_w[warp][k * 32 + lane] = w;
        sum += w * v[k].y;
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      all += sum;
      if (lane == 0) {
        s_m[warp] = m;
        s_l[warp] = all;
      }
    }
    __syncthreads();
    for (int k0 = 0; k0 < n; k0 += kAtOnce) {
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) acc += s_w[rr][k0 + k] * x[k];      // behind the last piece both are 0
      if (i0 + k0 + kAtOnce < pieces) load(i0 + k0 + kAtOnce);
    }
  }
  if (r >= R) return;
  const float l = s_l[rr];
  const bool dead = l == 0.f;
  const int64_t row = q0 + r / p.a.G;
  const int head = h * p.a.G + r % p.a.G;
  p.a.out.p[row * p.a.out.s_row + (int64_t)head * p.a.out.s_head + ch] = __float2bfloat16(dead ? 0.f : acc / l);
  if (p.a.lse && ch == 0) p.a.lse[row * (p.a.H * p.a.G) + head] = dead ? minus_inf : (s_m[rr] + log2f(l)) * kLn2;
}

template <int D, bool Q8, int RC, bool kTree>
cudaError_t launch(const FewLaunch& p, const CUtensorMap& mk, const CUtensorMap& mv, cudaStream_t s) {
  using F = Few<D, Q8, RC>;
  static DeviceOnce once;
  int dev;
  if (once.pending(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(attend_few_kernel<D, Q8, RC, kTree>, cudaFuncAttributeMaxDynamicSharedMemorySize, F::kSmem);
    if (e != cudaSuccess) return e;
    once.mark(dev);
  }
  const cudaError_t e = launch_after(attend_few_kernel<D, Q8, RC, kTree>, dim3((unsigned)p.blocks), F::kThreads, F::kSmem, s, p, mk, mv);
  if (e != cudaSuccess) return e;
  const int64_t rows = (int64_t)p.a.req.max_q * p.a.G;
  const dim3 g((unsigned)((int64_t)p.a.req.n * p.a.H), (unsigned)(((rows < RC ? rows : RC) + 3) / 4));
  return launch_after(attend_few_join_kernel<D, RC>, g, 4 * D, 0, s, p);
}

}  // namespace

// rows the kernel is built for, from the rows a request may have (0: more than it takes)
int few_capacity(int64_t rows) { return rows <= 8 ? 8 : rows <= 16 ? 16 : rows <= 32 ? 32 : 0; }

int few_blocks(int n, int max_kv, int H) {
  const int64_t tiles = (int64_t)n * H * (max_kv <= 0 ? 1 : (max_kv + 127) / 128);
  const int sms = device_sm_count();
  return (int)(tiles < sms ? tiles : sms);
}

size_t few_workspace_bytes(int n, int max_kv, int H, int d, int rc) { return (size_t)few_blocks(n, max_kv, H) * 2 * rc * (d + 2) * 4; }

cudaError_t launch_attend_few(const AttendLaunch& a, const tc::TileGeo& g, const CUtensorMap& mk, const CUtensorMap& mv, int rc, int d, float* part,
                              cudaStream_t s) {
  FewLaunch p;
  p.a = a;
  p.g = g;
  p.blocks = few_blocks(a.req.n, a.req.max_kv, a.H);
  p.part = part;
  const bool q8 = a.e.k != nullptr;
  if (p.blocks <= 0) return cudaErrorInvalidConfiguration;
#define KVC_FEW(D, Q, R) \
  if (d == D && q8 == Q && rc == R) return a.mask ? launch<D, Q, R, true>(p, mk, mv, s) : launch<D, Q, R, false>(p, mk, mv, s);
  KVC_FEW(128, false, 8) KVC_FEW(64, false, 8) KVC_FEW(128, false, 16) KVC_FEW(128, false, 32) KVC_FEW(64, false, 16) KVC_FEW(64, false, 32)
  KVC_FEW(128, true, 8) KVC_FEW(128, true, 16) KVC_FEW(128, true, 32) KVC_FEW(64, true, 8) KVC_FEW(64, true, 16) KVC_FEW(64, true, 32)
#undef KVC_FEW
  return cudaErrorInvalidValue;
}

}  // namespace kvc
