// kvc_attend for chunks of new tokens: tiles of 2 x 128 query rows against tiles of 128 keys on the tensor cores.
//
//     S = Q K^T  (tcgen05, f32 in tensor memory) ,  P = exp2(c S - c m) ,  O += P V  (P bf16 in tensor memory) ,
// c = scale log2 e, m a running row maximum.  The rows of a request and KV head are packed as token * G + query head, so
// the G heads that share K and V share the tile, and a few tokens fill it.
//
// Bound: 4 d flops a (row, key) pair on the tensor cores and one exponential; at d = 128 a 128 x 128 tile costs 1024
// cycles of either.  So one block keeps two row tiles going: while the softmax warps of one work, the tensor cores run
// the other's products.  One warp issues both tiles' in turn (two warps let the tiles fall into step, and then either the
// softmax warps or the tensor cores wait: 314 us against 256 on 2K tokens behind 8K at that time).  P lies over S in
// tensor memory (2 x 128 columns of S, 2 x d of O: all 512), and A operands come from there: P never passes through
// shared memory.  It is handed over in two parts (96 and 32 keys), so that most of the second product runs while the rest
// is still being computed.
//
// Measured, 2048 tokens behind 8K, 32 / 8 heads of 128 (240 GFLOP): 212 us (1.13 PFLOP/s) in a short run, 245 us
// once the power cap has set the clock.  What bounds it: a row tile's own chain, softmax (about 1750 cycles), the second
// product's tail, the next first product, and the hand-overs between them (about 3200 a tile of keys, in which the tensor
// cores need 2048 for both row tiles; over the whole launch, start, epilogues and join included, they are busy 53 %).  A
// second S of 128 columns finds no room; two of 64 would (P takes the lower half of S's columns), and are not tried.
// Local memory would cost more than anything else (shared
// memory takes all of L1: with 100 bytes of spills in the loop the kernel ran 310 us), and so does code that the
// instruction cache does not hold (8-bit conversion unrolled whole: 277 us on the image context, in rounds 233).
//
// Exponentials stay on the special-function units (16 a cycle and SM, a tile's time of the tensor cores).  Moving a
// quarter or half of them to the FMA pipe (rounding to a whole exponent and a degree-5 polynomial) made the kernel
// slower, 234 -> 274 and 297 us on 2K tokens behind 8K: the chain above got longer.
//
// m is a maximum of earlier tiles: a tile's own maximum is taken beside its exponentials, off the way from logits to
// probabilities.  Exponentials above 1 cost no precision (bf16 and float32 have the same range), but P V is summed in
// float32, and a sum that overflowed stays infinite whatever it is scaled by later: where one would pass 2^kJump the tile
// is done over with its own maximum.  A maximum grown by more than 2^kLazy becomes m at the next tile: sums and
// accumulators are then rescaled, which the softmax warps do.  (kJump = kLazy = 8, always done over: 250 us on 2K tokens
// behind 8K, 244 so; 64 let values from 2^63 on overflow.)
//
// Rounding: P to bf16 (2^-8 of each term: what the tensor cores take), everything else float32.
//
// Work: the key tiles of all (request, KV head, 256-row unit) triples form one line, of which every block takes an equal
// part; ragged and causal batches balance to a tile.  Of a unit cut by its borders a block leaves a float32 partial
// result (at most two a block); a second kernel joins those in a fixed order.
//
// Warps: 0-3 and 4-7 softmax and epilogue of the row tiles (a thread a row; two threads a row with sixteen warps were no
// faster, 235 us), 8 and 10 loads of keys and values, 9 products, 11 walks the block's part of the line and hands its
// pieces to the others through shared memory (their registers are for the work itself); 8-bit caches: 12-15 turn raw
// tiles into bf16 ones (code * 2^e, exact).  Every wait is bounded; on expiry the CTA records KVC_FLAG_WAIT_EXPIRED and
// returns.
#include <cuda_runtime.h>

#include "kvc_launch.h"
#include "kvc_tc.h"
#include "kvc_tc_attend.cuh"
#include "kvc_tc_attend_few.h"

namespace kvc {
namespace {

using namespace tc;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLazy = 8.f, kJump = 16.f; // log2 of the growth of a row's maximum that is let pass, and that a tile bears
constexpr int kUnitRows = 256;

struct alignas(16) UnitStart {             // where a block's part of the line begins; b < 0: it has none
  int32_t b, h, u, t;
};

struct ChunkLaunch {
  AttendLaunch a;
  TileGeo g;                               // of the raw tile
  int32_t blocks;
  int32_t min_rows;                        // requests with fewer rows belong to the other kernel
  bool fine;                               // few units in many pieces: the join's small blocks
  UnitStart* starts;                       // [blocks]
  float* ml;                               // [blocks][2][256][2] maximum and sum of the rows of a block's two cut units
  float* part;                             // [blocks][2][256][d] their sums
};

template <int D, bool Q8>
struct Shape {
  static constexpr int kTile = 128 * D * 2;                       // bytes of a bf16 tile
  static constexpr int kRaw = 128 * D;
  static constexpr int kSlots = Q8 ? 4 : (D == 128 ? 5 : 8);
  static constexpr int kRawSlots = Q8 ? 2 : 1;
  static constexpr int kThreads = Q8 ? 512 : 384;
  static constexpr int kRegs = Q8 ? 184 : 208;                    // of the softmax warps; the others keep 72 or 88
  static constexpr int kSmem = 1024 + 2 * kTile + kSlots * kTile + (Q8 ? kRawSlots * kRaw : 0);
};

// Key tiles of unit u of a request (at least one, so that rows without keys are answered too), and of its two row tiles.
struct UnitTiles {
  int row[2], all;
};
__device__ __forceinline__ UnitTiles unit_tiles(const AttendLaunch& a, int nq, int kv, int rows, int u) {
  UnitTiles x;
  x.all = 1;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int first = u * kUnitRows + t * 128, last = min(first + 128, rows) - 1;
    const int keys = first >= rows ? 0 : a.causal ? max(0, kv - nq + last / a.G + 1) : kv;
    x.row[t] = (keys + 127) >> 7;
    x.all = max(x.all, x.row[t]);
  }
  return x;
}
__device__ __forceinline__ int units_of(const ChunkLaunch& p, int nq) {
  const int rows = nq * p.a.G;
  return rows < p.min_rows ? 0 : (rows + kUnitRows - 1) / kUnitRows;
}

// A block's piece of a unit; b < 0: there are no more.
struct alignas(16) Piece {
  int b, h, u, q0;
  int nq, kv, rows, whole;
  int t0, n_all, n[2];                     // first key tile, key tiles of the piece and of either row tile
};
constexpr int kPieces = 4;                 // pieces on their way

struct Walk {
  int64_t left;
  int b, h, u, t;
  int known, q0, nq, kv, units;
  __device__ __forceinline__ bool next(const ChunkLaunch& p, Piece& x) {
    if (left <= 0) return false;
    for (;; ++b) {
      if (b >= p.a.req.n) return false;
      if (b != known) {
        request_span(p.a.req, b, nullptr, q0, nq, kv);
        units = units_of(p, nq);
        known = b;
      }
      if (units > 0) break;
    }
    x.b = b;
    x.h = h;
    x.u = u;
    x.q0 = q0;
    x.nq = nq;
    x.kv = kv;
    x.rows = nq * p.a.G;
    const UnitTiles c = unit_tiles(p.a, nq, kv, x.rows, u);
    const int t1 = (int64_t)(c.all - t) < left ? c.all : t + (int)left;
    x.whole = t == 0 && t1 == c.all;
    x.t0 = t;
    x.n[0] = max(0, min(c.row[0], t1) - t);
    x.n[1] = max(0, min(c.row[1], t1) - t);
    x.n_all = max(x.n[0], x.n[1]);
    left -= t1 - t;
    t = 0;
    if (++u == units) {
      u = 0;
      if (++h == p.a.H) {
        h = 0;
        ++b;
      }
    }
    return true;
  }
};

__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {
  return (a | b) < ((int64_t)1 << 31) ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}
__device__ __forceinline__ int64_t warp_scan(int64_t v, int lane) {   // inclusive
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  return v;
}
// Key tiles of one head of 32 requests, each lane with a request of its own (whole warp): a lane adds up its request's
// units, or, where few requests have many, the warp does, a lane a unit.
__device__ __forceinline__ int64_t head_tiles(const ChunkLaunch& p, int nq, int kv, int lane) {
  const int units = units_of(p, nq);
  int64_t sum = 0;
  unsigned left = __ballot_sync(0xffffffffu, units > 0);
  if (__reduce_max_sync(0xffffffffu, units) <= min(8, __popc(left))) {
    for (int u = 0; u < units; ++u) sum += unit_tiles(p.a, nq, kv, nq * p.a.G, u).all;
    return sum;
  }
  while (left) {
    const int o = __ffs(left) - 1;
    left &= left - 1;
    const int nq_o = __shfl_sync(0xffffffffu, nq, o), kv_o = __shfl_sync(0xffffffffu, kv, o), units_o = __shfl_sync(0xffffffffu, units, o);
    int64_t mine = 0;
    for (int u = lane; u < units_o; u += 32) mine += unit_tiles(p.a, nq_o, kv_o, nq_o * p.a.G, u).all;
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, k);
    if (lane == o) sum = mine;
  }
  return sum;
}
// The start of block c's part of the line (whole warp); up to 32 requests are looked at once.
__device__ __forceinline__ Walk line_start(const ChunkLaunch& p, int lane, int c) {
  const int n = p.a.req.n;
  int q0 = 0, nq = 0, kv = 0;
  int64_t each = 0, incl = 0, total = 0;
  auto look = [&](int b0, uint32_t* status) {                     // requests b0 .. b0 + 31
    q0 = nq = kv = 0;
    if (b0 + lane < n) request_span(p.a.req, b0 + lane, status, q0, nq, kv);
    each = head_tiles(p, nq, kv, lane);
    incl = warp_scan(each * p.a.H, lane);
  };
  for (int b0 = 0; b0 < n; b0 += 32) {
    look(b0, c == 0 ? p.a.status : nullptr);
    total += __shfl_sync(0xffffffffu, incl, 31);
  }
  const int64_t blocks = total < p.blocks ? total : p.blocks;
  Walk w{0, 0, 0, 0, 0, -1, 0, 0, 0, 0};
  if (c >= blocks) return w;
  const int64_t lo = divide(total * c, blocks);
  int64_t before = 0;
  for (int b0 = 0; b0 < n; b0 += 32) {
    if (n > 32) look(b0, nullptr);
    const unsigned hit = __ballot_sync(0xffffffffu, before + incl > lo);
    if (!hit) {
      before += __shfl_sync(0xffffffffu, incl, 31);
      continue;
    }
    const int l = __ffs(hit) - 1;
    w.b = w.known = b0 + l;
    w.q0 = __shfl_sync(0xffffffffu, q0, l);
    w.nq = __shfl_sync(0xffffffffu, nq, l);
    w.kv = __shfl_sync(0xffffffffu, kv, l);
    w.units = units_of(p, w.nq);
    const int64_t head = __shfl_sync(0xffffffffu, each, l);
    int64_t off = lo - before - (__shfl_sync(0xffffffffu, incl, l) - head * p.a.H);
    w.h = (int)divide(off, head);
    off -= w.h * head;
    for (int u0 = 0; u0 < w.units; u0 += 32) {
      const int mine = u0 + lane < w.units ? unit_tiles(p.a, w.nq, w.kv, w.nq * p.a.G, u0 + lane).all : 0;
      const int sum = (int)warp_scan(mine, lane);
      const unsigned in = __ballot_sync(0xffffffffu, (int64_t)sum > off);
      if (in) {
        const int k = __ffs(in) - 1;
        w.u = u0 + k;
        w.t = (int)(off - __shfl_sync(0xffffffffu, sum - mine, k));
        w.left = divide(total * (c + 1), blocks) - lo;
        return w;
      }
      off -= __shfl_sync(0xffffffffu, sum, 31);
    }
    return w;                                                     // not reached: the tile lies in one of the units
  }
  return w;
}

template <int NS, int NR>
struct Bars {
  uint64_t q_full[2], s_full[2], p_ready[2][2], o_done[2];
  uint64_t full[NS], empty[NS], raw_full[NR], raw_empty[NR], piece_full[kPieces], piece_empty[kPieces];
  Piece piece[kPieces];
  uint32_t tmem;
  int abort_flag;
};

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// 32 bytes of a row in one store where they are aligned (a thread's rows are far apart: each store costs a sector a row)
__device__ __forceinline__ void store32(__nv_bfloat16* at, const uint4& a, const uint4& b) {
  if ((reinterpret_cast<uintptr_t>(at) & 31) == 0) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(at), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y),
                 "r"(b.z), "r"(b.w)
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(at)[0] = a;
    reinterpret_cast<uint4*>(at)[1] = b;
  }
}

// Four e4m3 codes -> channels (0, 2) and (1, 3) as bf16 pairs, before the scale: sign, exponent and mantissa moved to
// their places read 2^-120 of the code's value, subnormals included (bias 7 against 127).
__device__ __forceinline__ void spread_codes(uint32_t w, uint32_t& even, uint32_t& odd) {
  even = ((w << 8) & 0x80008000u) | ((w << 4) & 0x07f007f0u);
  odd = (w & 0x80008000u) | ((w >> 4) & 0x07f007f0u);
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

template <int D, bool Q8>
__global__ void __launch_bounds__(Shape<D, Q8>::kThreads, 1)
attend_chunk_kernel(const __grid_constant__ ChunkLaunch p, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  using SH = Shape<D, Q8>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ Bars<SH::kSlots, SH::kRawSlots> bars;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* sq = smem;                                             // [2][part][128 rows][128 B]
  uint8_t* skv = smem + 2 * SH::kTile;
  uint8_t* sraw = skv + SH::kSlots * SH::kTile;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  volatile int* abort_flag = &bars.abort_flag;
  const uint32_t q_full = smem_u32(bars.q_full), s_full = smem_u32(bars.s_full), p_ready = smem_u32(bars.p_ready), o_done = smem_u32(bars.o_done);
  const uint32_t full = smem_u32(bars.full), empty = smem_u32(bars.empty), rfull = smem_u32(bars.raw_full), rempty = smem_u32(bars.raw_empty);
  const uint32_t piece_full = smem_u32(bars.piece_full), piece_empty = smem_u32(bars.piece_empty);
  if (tid == 0) {
    for (int t = 0; t < 2; ++t) {
      mbar_init(q_full + 8 * t, 128);
      mbar_init(s_full + 8 * t, 1);
      mbar_init(p_ready + 16 * t, 128);
      mbar_init(p_ready + 16 * t + 8, 128);
      mbar_init(o_done + 8 * t, 1);
    }
    for (int s = 0; s < SH::kSlots; ++s) {
      mbar_init(full + 8 * s, Q8 ? 128 : 1);
      mbar_init(empty + 8 * s, 1);
    }
    for (int s = 0; s < SH::kRawSlots; ++s) {
      mbar_init(rfull + 8 * s, 1);
      mbar_init(rempty + 8 * s, 128);
    }
    for (int s = 0; s < kPieces; ++s) {
      mbar_init(piece_full + 8 * s, 1);
      mbar_init(piece_empty + 8 * s, SH::kThreads / 32 - 1);      // a lane of every warp but the walking one
    }
    bars.abort_flag = 0;
    fence_barrier_init();
  }
  if (tid == 32) {
    prefetch_map(&map_k);
    prefetch_map(&map_v);
  }
  if (warp == 9) {
    tmem_alloc(smem_u32(&bars.tmem), 512);
    tmem_relinquish();
  }
  grid_dependency_wait();                                         // what follows reads what earlier kernels wrote
  grid_dependents_launch();                                       // the join's blocks may take the SMs that finish first
  Walk walk;                                                      // warp 11: the block's part of the line
  if (warp == 11) walk = line_start(p, lane, (int)blockIdx.x);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars.tmem;
  // a warp's view of the pieces: wait for number `i`, give it back
  auto piece_wait = [&](int i) { return wait_all(piece_full + 8 * (i % kPieces), (i / kPieces) & 1, abort_flag); };
  auto piece_done = [&](int i) {
    __syncwarp();
    if (lane == 0) mbar_arrive(piece_empty + 8 * (i % kPieces));
  };
  // the tile's strides as the tensor cores see it
  const uint32_t gs = Q8 ? 1024u : (uint32_t)p.g.gs, ps = Q8 ? 16384u : (uint32_t)p.g.ps;

  if (warp < 8) {
    regs_inc<SH::kRegs>();
    const int t = warp >> 2, row = tid & 127;
    const float c = p.a.scale * kLog2e, minus_inf = __uint_as_float(0xff800000u);
    const uint32_t lane_at = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t s_at = lane_at + t * 128, o_at = lane_at + 256 + t * D;
    const uint32_t pr = p_ready + 16 * t;
    int count = 0;                                                // products of this row tile so far
    int g = 0;                                                    // key tiles of the block so far
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity) { return ok = ok && wait_all(bar, parity, abort_flag); };
    // queries of a piece's row tile, a thread its row, all loads in flight at once; 8-bit caches: channels 1 and 2 of
    // every four change places, as their keys do
    auto load_q = [&](const Piece& y) {
      const int r = y.u * kUnitRows + t * 128 + row, tok = r / p.a.G;
      const bool live = r < y.rows;
      const uint4* src = reinterpret_cast<const uint4*>(p.a.q.p + (live ? (int64_t)(y.q0 + tok) * p.a.q.s_row + (int64_t)(y.h * p.a.G + r - tok * p.a.G) * p.a.q.s_head : 0));
      uint8_t* dst = sq + t * SH::kTile + (row >> 3) * 1024 + (row & 7) * 128;
      uint4 v[D / 8];
#pragma unroll
      for (int j = 0; j < D / 8; ++j) v[j] = live ? __ldg(src + j) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int j = 0; j < D / 8; ++j) {
        if (Q8) v[j] = make_uint4(__byte_perm(v[j].x, v[j].y, 0x5410), __byte_perm(v[j].x, v[j].y, 0x7632), __byte_perm(v[j].z, v[j].w, 0x5410), __byte_perm(v[j].z, v[j].w, 0x7632));
        *reinterpret_cast<uint4*>(dst + (j >> 3) * 16384 + (((j & 7) ^ (row & 7)) << 4)) = v[j];
      }
      fence_proxy_async();
      mbar_arrive(q_full + 8 * t);
    };
    auto next_piece = [&](int i) {                                // the queries of piece i, if there is one
      if (!ok || !(ok = piece_wait(i))) return false;
      const Piece& y = bars.piece[i % kPieces];
      if (y.b < 0) return false;
      if (y.n[t] > 0) load_q(y);                                  // only then: the products wait for no others
      return true;
    };
    bool more = next_piece(0);
    for (int piece = 0; more; ++piece) {
      const Piece& y = bars.piece[piece % kPieces];
      const int n = y.n[t], kv = y.kv, first = y.t0 * 128;
      int lim = -1;
      {
        const int r = y.u * kUnitRows + t * 128 + row;
        if (r < y.rows) lim = p.a.causal ? kv - y.nq + r / p.a.G : kv - 1;
      }
      const int lowest = __reduce_min_sync(0xffffffffu, lim);     // of the warp's rows
      float m = minus_inf, l = 0.f;
      float late = minus_inf;                                     // a maximum that m is to follow
      for (int it = 0; it < n; ++it) {
        const uint32_t par = (uint32_t)(count + it) & 1u;
        if (!wait(s_full + 8 * t, par)) break;
        tc_fence_after();
        float s[128];
#pragma unroll
        for (int k = 0; k < 4; ++k) tmem_ld32(s_at + 32 * k, s + 32 * k);
        tmem_ld_wait();
        const int t0 = first + it * 128;
        if (lowest < t0 + 127) {
#pragma unroll
          for (int k = 0; k < 128; ++k) s[k] = t0 + k <= lim ? s[k] : minus_inf;
        }
        const f32x2 c2 = f2_pack(c, c);
        f32x2 mc2, sum2[2];
        float mx[4];
        // 32 probabilities
        auto quarter = [&](int at0) {
          uint32_t w[16];
          f32x2 e[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) e[k] = f2_fma(f2_pack(s[at0 + 2 * k], s[at0 + 2 * k + 1]), c2, mc2);
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            float a, b;
            f2_unpack(e[k], a, b);
            e[k] = f2_pack(exp2_fast(a), exp2_fast(b));
          }
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            sum2[k & 1] = f2_add(sum2[k & 1], e[k]);
            w[k] = f2_to_bf16x2(e[k]);
          }
          tmem_st16(s_at + at0 / 2, w);
        };
        // one copy of each step (the instruction cache holds the loop): first round with the maximum of earlier tiles, a
        // second where the tile's own is too far above it (a piece's first tile among them: m = -inf)
        bool grow = late > m;
        float to = late, top;
#pragma unroll 1
        for (;;) {
          if (__any_sync(0xffffffffu, grow)) {
            // O and l to the new m, once the product that wrote O last is done
            const float keep = grow ? exp2_fast((m - to) * c) : 1.f;
            if (it > 0) {
              wait(o_done + 8 * t, par ^ 1);
              tc_fence_after();
#pragma unroll 1
              for (int k = 0; k < D; k += 16) {
                float o[16];
                tmem_ld16(o_at + k, o);
                tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 16; ++j) o[j] *= keep;
                tmem_st16(o_at + k, reinterpret_cast<const uint32_t*>(o));
              }
              tmem_st_wait();
            }
            if (grow) {
              l *= keep;
              m = to;
            }
          }
          const float mc = m == minus_inf ? 0.f : m * c;
          mc2 = f2_pack(-mc, -mc);
          sum2[0] = sum2[1] = f2_pack(0.f, 0.f);
#pragma unroll
          for (int j = 0; j < 4; ++j) mx[j] = s[j];
#pragma unroll
          for (int k = 4; k < 124; k += 8) {
#pragma unroll
            for (int j = 0; j < 4; ++j) mx[j] = max3(mx[j], s[k + 2 * j], s[k + 2 * j + 1]);
          }
          mx[0] = max3(mx[0], s[124], s[125]);
          mx[1] = max3(mx[1], s[126], s[127]);
          quarter(0);
          quarter(32);
          quarter(64);
          top = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]);
          grow = (top - m) * c > kJump;
          to = top;
          if (!__any_sync(0xffffffffu, grow)) break;
        }
        late = (top - m) * c > kLazy ? top : minus_inf;
        // stale value rows behind the last key: P is zero there, but zero times a stale NaN would not be
        if (!Q8 && kv < t0 + 128) {
          const int use = 2 * (g + it) + 1, vs = use % SH::kSlots;
          if (wait(full + 8 * vs, (use / SH::kSlots) & 1) && t0 + row >= kv) {
            uint8_t* v = skv + vs * SH::kTile + (row >> 3) * gs + (row & 7) * 128;
#pragma unroll
            for (int ch = 0; ch < D / 8; ++ch) *reinterpret_cast<uint4*>(v + (ch >> 3) * ps + ((ch & 7) << 4)) = make_uint4(0, 0, 0, 0);
          }
          fence_proxy_async();
        }
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive(pr);
        quarter(96);
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive(pr + 8);
        float a, b;
        f2_unpack(f2_add(sum2[0], sum2[1]), a, b);
        l += a + b;
      }
      // the next piece's queries go in while the last products run: this tile's logits are all there
      g += y.n_all;
      count += n;
      more = next_piece(piece + 1);
      if (n > 0) wait(o_done + 8 * t, (uint32_t)(count - 1) & 1u);
      tc_fence_after();
      const int r = y.u * kUnitRows + t * 128 + row;
      const bool live = r < y.rows;
      const int tok = r / p.a.G, head = y.h * p.a.G + r - tok * p.a.G;
      // no key seen: decided by the sum, which a NaN logit makes NaN (maxima pass over NaN: m may still be minus infinity)
      const bool dead = l == 0.f;
      const bool whole = y.whole;
      const int64_t slot = ((int64_t)blockIdx.x * 2 + (y.t0 > 0 ? 0 : 1)) * kUnitRows + t * 128 + row;
      const float inv = whole ? (dead ? 0.f : 1.f / l) : 1.f;
      __nv_bfloat16* dst = p.a.out.p + (int64_t)(y.q0 + tok) * p.a.out.s_row + (int64_t)head * p.a.out.s_head;
      // partial sums lie channel by channel: a warp's rows are neighbours
      float* pdst = p.part + (slot - row - t * 128) * D + t * 128 + row;
#pragma unroll 1
      for (int k = 0; k < D; k += 16) {
        float o[16];
        if (n > 0) {
          tmem_ld16(o_at + k, o);
          tmem_ld_wait();
        }
        if (!live || !ok) continue;
#pragma unroll
        for (int j = 0; j < 16; ++j) o[j] = dead ? 0.f : o[j] * inv;
        if (Q8) {                                                 // channels back in their places
#pragma unroll
          for (int j = 0; j < 16; j += 4) {
            const float v = o[j + 1];
            o[j + 1] = o[j + 2];
            o[j + 2] = v;
          }
        }
        if (whole) {
          store32(dst + k, pack8(o), pack8(o + 8));
        } else if (n > 0) {
#pragma unroll
          for (int j = 0; j < 16; ++j) pdst[(k + j) * kUnitRows] = o[j];
        }
      }
      if (live && ok) {
        if (!whole)
          *reinterpret_cast<float2*>(p.ml + 2 * slot) = make_float2(m, l);
        else if (p.a.lse)
          p.a.lse[(int64_t)(y.q0 + tok) * (p.a.H * p.a.G) + head] = dead ? minus_inf : m * p.a.scale + log2f(l) * kLn2;
      }
      tc_fence_before();
      piece_done(piece);
    }
  } else {
    regs_dec<Q8 ? 72 : 88>();
    bool ok = true;
    if (warp == 11) {
      // ---- the block's part of the line
      if (lane == 0) p.starts[blockIdx.x] = walk.left > 0 ? UnitStart{walk.b, walk.h, walk.u, walk.t} : UnitStart{-1, 0, 0, 0};
      for (int i = 0; ok; ++i) {
        ok = wait_all(piece_empty + 8 * (i % kPieces), ((i / kPieces) & 1) ^ 1, abort_flag);
        Piece x;
        const bool more = walk.next(p, x);
        if (!more) x.b = -1;
        if (ok && lane == 0) {
          bars.piece[i % kPieces] = x;
          mbar_arrive(piece_full + 8 * (i % kPieces));
        }
        if (!more) break;
      }
    } else if (warp == 8 || warp == 10) {
      // ---- loads of the keys (8) and the values (10); the ring's slots alternate between them.  (A 16-token page is a box
      // of its own, about 140 cycles each: one warp for both was the bound.)
      const uint32_t ring = smem_u32(Q8 ? sraw : skv);
      const uint32_t bytes = Q8 ? SH::kRaw : SH::kTile;
      constexpr int NS = Q8 ? SH::kRawSlots : SH::kSlots;
      const uint32_t fb = Q8 ? rfull : full, eb = Q8 ? rempty : empty;
      const CUtensorMap* map = warp == 8 ? &map_k : &map_v;
      int use = warp == 8 ? 0 : 1;
      for (int i = 0; ok && (ok = piece_wait(i)); ++i) {
        const Piece x = bars.piece[i % kPieces];
        piece_done(i);
        if (x.b < 0) break;
        const int n = x.n_all;
        int ahead = n > 0 ? tile_entry(p.a, p.g, x.b, x.t0 * 128, min(128, x.kv - x.t0 * 128), lane) : 0;
        for (int it = 0; it < n; ++it, use += 2) {
          const int t0 = (x.t0 + it) * 128, rows = min(128, x.kv - t0), entry = ahead;
          if (it + 1 < n) ahead = tile_entry(p.a, p.g, x.b, t0 + 128, min(128, x.kv - t0 - 128), lane);
          const int slot = use % NS;
          ok = wait_all(eb + 8 * slot, ((use / NS) & 1) ^ 1, abort_flag);
          if (!ok) break;
          tile_load<Q8 || D == 64>(map, p.a, p.g, ring + slot * bytes, fb + 8 * slot, t0, rows, x.h, entry, lane);
        }
      }
    } else if (warp == 9) {
      // ---- products
      constexpr uint32_t idesc_s = idesc_bf16(128, 128, 0, 0), idesc_o = idesc_bf16(128, D, 0, 1);
      // descriptors differ in their start address alone (its 18 bits / 16 are the low word)
      const uint64_t q_desc = operand_desc(smem_u32(sq), 16, 1024, 2), k_desc = operand_desc(smem_u32(skv), 16, gs, 2);
      const uint64_t v_desc = operand_desc(smem_u32(skv), ps, gs, 2);
      const uint32_t k_part = ps >> 4, v_step = (2 * gs) >> 4;
      auto wait = [&](uint32_t bar, uint32_t parity) { return ok = ok && wait_all(bar, parity, abort_flag); };
      int slot = 0, count[2] = {0, 0}, queries[2] = {0, 0};
      uint32_t phase = 0;
      auto next = [&]() {
        if (++slot == SH::kSlots) {
          slot = 0;
          phase ^= 1;
        }
      };
      auto release = [&](int slot) {
        if (elect_one()) umma_commit(empty + 8 * slot);
      };
      auto score = [&](int t, int slot) {                         // S_t = Q_t K^T
        tc_fence_after();
        const uint64_t kd = k_desc + (uint32_t)(slot * (SH::kTile >> 4)), qd = q_desc + (uint32_t)(t * (SH::kTile >> 4));
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
            umma_bf16(tmem + t * 128, qd + ((k >> 2) * 1024 + (k & 3) * 2), kd + ((k >> 2) * k_part + (k & 3) * 2), idesc_s, k > 0);
          umma_commit(s_full + 8 * t);
        }
      };
      for (int piece = 0; ok && (ok = piece_wait(piece)); ++piece) {
        const Piece& y = bars.piece[piece % kPieces];
        const int b = y.b, n_all = y.n_all, n[2] = {y.n[0], y.n[1]};
        piece_done(piece);
        if (b < 0) break;
        if (n_all > 0) {
          wait(full + 8 * slot, phase);
#pragma unroll
          for (int t = 0; t < 2; ++t)
            if (n[t] > 0 && wait(q_full + 8 * t, (uint32_t)queries[t]++ & 1u)) score(t, slot);
          release(slot);
          next();
        }
        for (int it = 0; it < n_all && ok; ++it) {
          const int vs = slot, ks = slot + 1 == SH::kSlots ? 0 : slot + 1;
          const uint32_t vphase = phase, kphase = ks == 0 ? phase ^ 1 : phase;
          const bool more = it + 1 < n_all;
          if (!wait(full + 8 * vs, vphase)) break;
          if (more && !wait(full + 8 * ks, kphase)) break;
          const uint64_t vd = v_desc + (uint32_t)(vs * (SH::kTile >> 4)), kd = k_desc + (uint32_t)(ks * (SH::kTile >> 4));
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (!ok || it >= n[t]) continue;
            const uint32_t par = (uint32_t)(count[t] + it) & 1u;
            const bool again = it + 1 < n[t];
            const uint64_t qd = q_desc + (uint32_t)(t * (SH::kTile >> 4));
            if (!wait(p_ready + 16 * t, par)) break;
            tc_fence_after();
            if (elect_one()) {                                    // O_t += P_t V, keys 0 .. 95
#pragma unroll
              for (int k = 0; k < 6; ++k) umma_bf16_ts(tmem + 256 + t * D, tmem + t * 128 + 8 * k, vd + k * v_step, idesc_o, it > 0 || k > 0);
            }
            if (!wait(p_ready + 16 * t + 8, par)) break;
            tc_fence_after();
            if (elect_one()) {                                    // keys 96 .. 127, then the next S_t over them
#pragma unroll
              for (int k = 6; k < 8; ++k) umma_bf16_ts(tmem + 256 + t * D, tmem + t * 128 + 8 * k, vd + k * v_step, idesc_o, 1);
              umma_commit(o_done + 8 * t);
              if (again) {
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                  umma_bf16(tmem + t * 128, qd + ((k >> 2) * 1024 + (k & 3) * 2), kd + ((k >> 2) * k_part + (k & 3) * 2), idesc_s, k > 0);
                umma_commit(s_full + 8 * t);
              }
            }
          }
          if (!ok) break;
          release(vs);
          next();
          if (more) {
            release(ks);
            next();
          }
        }
        count[0] += n[0];
        count[1] += n[1];
      }
    } else if (Q8 && warp >= 12) {
      // ---- 8-bit tiles to bf16: a thread a token row, channels in the order (0, 2, 1, 3) of every four
      const int r = tid & 127;
      constexpr int CH = D / 16;                                  // 16-byte chunks of a raw row
      const uint32_t sw = D == 128 ? (uint32_t)(r & 7) : (uint32_t)((r >> 1) & 3);
      int rs = 0, rphase = 0, slot = 0, phase = 0;
      Piece x{};
      auto exponents = [&](int tt, uint32_t& ek, uint32_t& ev) {
        ek = ev = 127;
        if (tt >= x.kv) return;
        int64_t o = (int64_t)p.a.layer * p.a.e.s_layer + (int64_t)x.h * p.a.e.s_head;
        if (p.g.paged) {
          const int page = request_page(p.a.req, p.a.c, x.b, tt, nullptr);
          if (page < 0) return;
          o += (int64_t)page * p.a.e.s_page + (int64_t)(tt & p.a.c.page_mask) * p.a.e.s_tok;
        } else {
          o += (int64_t)tt * p.a.e.s_tok;
        }
        ek = p.a.e.k[o];
        ev = p.a.e.v[o];
      };
      for (int i = 0; ok && (ok = piece_wait(i)); ++i) {
        x = bars.piece[i % kPieces];
        piece_done(i);
        if (x.b < 0) break;
        const int n = x.n_all;
        uint32_t ek, ev, nk, nv;
        exponents(x.t0 * 128 + r, ek, ev);
        for (int it = 0; it < n && ok; ++it) {
          const int tt = (x.t0 + it) * 128 + r;
          exponents(it + 1 < n ? tt + 128 : x.kv, nk, nv);
          const bool valid = tt < x.kv;
#pragma unroll 1
          for (int kv = 0; kv < 2; ++kv) {
            ok = wait_all(rfull + 8 * rs, rphase, abort_flag) && wait_all(empty + 8 * slot, phase ^ 1, abort_flag);
            if (!ok) break;
            const uint8_t* in = sraw + rs * SH::kRaw + r * D;
            uint8_t* out = skv + slot * SH::kTile + (r >> 3) * 1024 + (r & 7) * 128;
            // 2^120 2^(e - 127), in one factor where bf16 holds it; exponent 255 reads as NaN
            const uint32_t e = kv ? ev : ek;
            const uint32_t f1 = e == 255u ? 0x7fc0u : e > 134u ? 254u << 7 : (e + 120u) << 7;
            const uint32_t scale = f1 | (f1 << 16);
            uint32_t nan = 0;
            // two chunks a round, the next round's on their way: unrolled whole, this code and the softmax's displace each
            // other in the instruction cache
            uint4 raw[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) raw[j] = *reinterpret_cast<const uint4*>(in + ((j ^ sw) << 4));
#pragma unroll 1
            for (int c0 = 0; c0 < CH; c0 += 2) {
             const uint4 now[2] = {raw[0], raw[1]};
             if (c0 + 2 < CH) {
#pragma unroll
               for (int j = 0; j < 2; ++j) raw[j] = *reinterpret_cast<const uint4*>(in + (((c0 + 2 + j) ^ sw) << 4));
             }
#pragma unroll
             for (int jj = 0; jj < 2; ++jj) {
              const int ch = c0 + jj;
              const uint32_t w[4] = {valid ? now[jj].x : 0u, valid ? now[jj].y : 0u, valid ? now[jj].z : 0u, valid ? now[jj].w : 0u};
              uint32_t o[8];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                spread_codes(w[j], o[2 * j], o[2 * j + 1]);
                nan |= (w[j] & 0x7f7f7f7fu) + 0x01010101u;
              }
#pragma unroll
              for (int j = 0; j < 8; ++j) o[j] = mul_bf16x2(o[j], scale);
              uint8_t* q = out + (ch >> 2) * 16384;
              const int j0 = (2 * ch) & 7;
              *reinterpret_cast<uint4*>(q + ((j0 ^ (r & 7)) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
              *reinterpret_cast<uint4*>(q + (((j0 + 1) ^ (r & 7)) << 4)) = make_uint4(o[4], o[5], o[6], o[7]);
             }
            }
            if (((nan & 0x80808080u) != 0 || e > 134u) && valid) {
              // a NaN code in the row, or a scale beyond one factor: the plain way
              const float s = exponent_up(e);
#pragma unroll 1
              for (int ch = 0; ch < CH; ++ch) {
                const uint4 v = *reinterpret_cast<const uint4*>(in + ((ch ^ sw) << 4));
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
                for (int j = 0; j < 4; ++j) {
                  const float2 lo = e4m3x2_to_float2(w[j] & 0xffffu), hi = e4m3x2_to_float2(w[j] >> 16);
                  const int at = 2 * ch + (j >> 1);
                  *reinterpret_cast<uint2*>(out + (at >> 3) * 16384 + (((at & 7) ^ (r & 7)) << 4) + (j & 1) * 8) =
                      make_uint2(pack2(lo.x * s, hi.x * s), pack2(lo.y * s, hi.y * s));
                }
              }
            }
            fence_proxy_async();
            mbar_arrive(full + 8 * slot);
            mbar_arrive(rempty + 8 * rs);
            if (++rs == SH::kRawSlots) {
              rs = 0;
              rphase ^= 1;
            }
            if (++slot == SH::kSlots) {
              slot = 0;
              phase ^= 1;
            }
          }
          ek = nk;
          ev = nv;
        }
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
    tmem_dealloc(tmem, 512);
  }
}

// ---- join of the units that block borders cut; grid: x = border in front of block x + 1 (CH = 4: a unit), y = 32 rows (a
// lane a row) and 8 CH channels (CH a warp).  The first border inside a unit does its work: the pieces are slot 1 of the
// block before it and slot 0 of the blocks whose parts begin inside the unit.  The warps share the pieces' weights, and the loads of
// several pieces are in flight at once.  Few units in many pieces (four a unit and more) take more and smaller blocks, CH = 4:
// 427 rows over 3133 keys, 25 pieces a unit: 19 us in all, 40 with a thread a row and piece after piece.  Many
// units in two or three pieces each take CH = D / 8 (2K tokens behind 8K 212 us, by small blocks 217).
template <int D, int CH>
__global__ void __launch_bounds__(256) attend_chunk_join_kernel(const __grid_constant__ ChunkLaunch p) {
  constexpr int kJoinPieces = CH == 4 ? 64 : 16;                  // weights held at once
  __shared__ float s_w[kJoinPieces][32], s_part[8][32];
  grid_dependents_launch();
  grid_dependency_wait();                                         // in every block, also those with nothing to join
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int row = (int)(blockIdx.y & 7) * 32 + lane, ch = ((int)(blockIdx.y >> 3) * 8 + warp) * CH;
  UnitStart me;
  int j, pieces;                                                  // blocks j - 1, j, ...
  if constexpr (CH == 4) {                                        // x is a unit: the borders that lie inside it
    const int units = (int)(((int64_t)p.a.req.max_q * p.a.G + kUnitRows - 1) / kUnitRows), bh = (int)blockIdx.x / units;
    me = UnitStart{bh / p.a.H, bh % p.a.H, (int)blockIdx.x % units, 1};
    j = p.blocks;
    pieces = 1;
    for (int k = 1 + lane; k < p.blocks + lane; k += 32) {
      const UnitStart o = k < p.blocks ? p.starts[k] : UnitStart{-1, 0, 0, 0};
      const unsigned in = __ballot_sync(0xffffffffu, o.b == me.b && o.h == me.h && o.u == me.u && o.t > 0);
      if (in && j == p.blocks) j = k - lane + __ffs(in) - 1;
      pieces += __popc(in);
    }
    if (pieces == 1) return;
  } else {
    j = (int)blockIdx.x + 1;
    me = p.starts[j];
    const UnitStart before = p.starts[j - 1];
    if (me.b < 0 || me.t == 0) return;
    auto same = [&](const UnitStart& o) { return o.b == me.b && o.h == me.h && o.u == me.u && o.t > 0; };
    if (same(before)) return;
    pieces = 2;
    for (bool go = true; go; pieces += 32) {
      const int k = j + pieces - 1 + lane;
      const bool in = k < p.blocks && same(p.starts[k]);
      const unsigned out = ~__ballot_sync(0xffffffffu, in);
      if (out) {
        pieces += __ffs(out) - 1 - 32;
        go = false;
      }
    }
  }
  int q0, nq, kv;
  request_span(p.a.req, me.b, nullptr, q0, nq, kv);
  const int r = me.u * kUnitRows + row, rows = nq * p.a.G;
  if (r - lane >= rows) return;
  const float c = p.a.scale * kLog2e, minus_inf = __uint_as_float(0xff800000u);
  auto place = [&](int i) { return ((int64_t)(j - 1 + i) * 2 + (i == 0 ? 1 : 0)) * kUnitRows; };
  auto held = [&](int i) { return *reinterpret_cast<const float2*>(p.ml + 2 * (place(i) + row)); };
  constexpr int kAtOnce = CH == 4 ? 8 : 16 / CH;                                // pieces whose sums are in flight: before their weights are known
  float x[kAtOnce][CH];
  auto load = [&](int i0) {
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const float* o = p.part + place(i0 + k) * D + row + ch * kUnitRows;
#pragma unroll
      for (int q = 0; q < CH; ++q) x[k][q] = i0 + k < pieces ? o[q * kUnitRows] : 0.f;
    }
  };
  load(0);
  float m = minus_inf;
  float2 v[kJoinPieces / 8];
  for (int i0 = (pieces - 1) / kJoinPieces * kJoinPieces; i0 >= 0; i0 -= kJoinPieces) {   // the first ones stay in v
#pragma unroll
    for (int k = 0; k < kJoinPieces / 8; ++k) v[k] = i0 + k * 8 + warp < pieces ? held(i0 + k * 8 + warp) : make_float2(0.f, 0.f);
#pragma unroll
    for (int k = 0; k < kJoinPieces / 8; ++k)
      if (v[k].y != 0.f) m = fmaxf(m, v[k].x);
  }
  s_part[warp][lane] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) m = fmaxf(m, s_part[w][lane]);
  float sum = 0.f, acc[CH];
#pragma unroll
  for (int q = 0; q < CH; ++q) acc[q] = 0.f;
  for (int i0 = 0; i0 < pieces; i0 += kJoinPieces) {
    const int n = min(kJoinPieces, pieces - i0);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kJoinPieces / 8; ++k) {
      const int i = k * 8 + warp;
      if (i >= n) break;
      if (i0 > 0) v[k] = held(i0 + i);
      const bool none = v[k].y == 0.f;                            // a piece that saw no key of the row wrote no sums of it (one of NaN did)
      const float w = none ? -1.f : exp2f((v[k].x - m) * c);
      s_w[i][lane] = w;
      if (!none) sum += w * v[k].y;
    }
    __syncthreads();
    for (int i = 0; i < n; i += kAtOnce) {
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const float w = i + k < n ? s_w[i + k][lane] : -1.f;
#pragma unroll
        for (int q = 0; q < CH; ++q) acc[q] = w < 0.f ? acc[q] : fmaf(w, x[k][q], acc[q]);
      }
      if (i0 + i + kAtOnce < pieces) load(i0 + i + kAtOnce);
    }
  }
  __syncthreads();
  s_part[warp][lane] = sum;
  __syncthreads();
  if (r >= rows) return;
  float l = 0.f;
#pragma unroll
  for (int w = 0; w < 8; ++w) l += s_part[w][lane];
  const bool dead = l == 0.f;
  const float inv = dead ? 0.f : 1.f / l;
  const int64_t tok = q0 + r / p.a.G;
  const int head = me.h * p.a.G + r % p.a.G;
  __nv_bfloat16* dst = p.a.out.p + tok * p.a.out.s_row + (int64_t)head * p.a.out.s_head + ch;
#pragma unroll
  for (int q = 0; q < CH; ++q) acc[q] = dead ? 0.f : acc[q] * inv;
  if constexpr (CH == 4)
    *reinterpret_cast<uint2*>(dst) = make_uint2(pack2(acc[0], acc[1]), pack2(acc[2], acc[3]));
  else
#pragma unroll
    for (int q = 0; q < CH; q += 8) *reinterpret_cast<uint4*>(dst + q) = pack8(acc + q);
  if (p.a.lse && ch == 0) p.a.lse[tok * (p.a.H * p.a.G) + head] = dead ? minus_inf : m * p.a.scale + log2f(l) * kLn2;
}

int64_t chunk_units(int n, int max_q, int G, int H) { return (int64_t)n * H * (((int64_t)max_q * G + kUnitRows - 1) / kUnitRows); }
int64_t chunk_blocks(int n, int max_q, int max_kv, int G, int H) {
  const int64_t tiles = chunk_units(n, max_q, G, H) * (max_kv <= 0 ? 1 : (max_kv + 127) / 128);
  const int sms = device_sm_count();
  return tiles < sms ? tiles : sms;
}
size_t chunk_starts_bytes(int64_t blocks) { return ((size_t)blocks * sizeof(UnitStart) + 255) / 256 * 256; }

template <int D, bool Q8>
cudaError_t launch_chunk(const ChunkLaunch& p, const CUtensorMap& mk, const CUtensorMap& mv, cudaStream_t s) {
  using SH = Shape<D, Q8>;
  static DeviceOnce once;
  int dev;
  if (once.pending(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(attend_chunk_kernel<D, Q8>, cudaFuncAttributeMaxDynamicSharedMemorySize, SH::kSmem);
    if (e != cudaSuccess) return e;
    once.mark(dev);
  }
  const cudaError_t e = launch_after(attend_chunk_kernel<D, Q8>, dim3((unsigned)p.blocks), SH::kThreads, SH::kSmem, s, p, mk, mv);
  if (e != cudaSuccess || p.blocks < 2) return e;
  if (p.fine) return launch_after(attend_chunk_join_kernel<D, 4>, dim3((unsigned)chunk_units(p.a.req.n, p.a.req.max_q, p.a.G, p.a.H), 8 * (D / 32)), 256, 0, s, p);
  return launch_after(attend_chunk_join_kernel<D, D / 8>, dim3((unsigned)p.blocks - 1, 8), 256, 0, s, p);
}

}  // namespace

// Which kernels a call launches: requests of up to `rc` rows a KV head go to the few-rows kernel (rc = 0: none), the
// others to this one (chunk = false: there are none).  Decided from the bounds alone: all requests within the few-rows
// kernel's 32 rows take it; a batch of several requests with longer ones among them is served by both, single tokens by
// the few-rows kernel; one long request by this kernel.  Both cost two more launches one behind the other, about 10 us,
// and a tile of a single token costs this kernel about twice the other's time.  The host knows the longest request only,
// so batches that could hold up to kBothTiles key tiles by the bounds stay with this kernel alone.  Measured, this kernel
// alone and both, us, 4 query heads of 128 per KV head, lengths to twice their mean, the rest single tokens:
//     tiles by the bounds                     1152   1536   2304    4096    4608    8192    16384   32256
//     bf16, one request in ten of 50-400 rows 43 56  46 56  60 76   83 94   92 92   138 121 243 194 370 304
//     bf16, one in two                        54 60  66 79  97 102  130 140 168 171 209 215 392 381 735 697
//     8 bits, one in ten                      41 51  44 52  62 69   88 86   108 98  164 125 302 206 496 295
//     8 bits, one in two                      61 68  80 90  111 112 161 165 193 193 267 261 508 454 848 737
// The lines cross at about 4500 tiles; a batch between 2048 and 4096 is up to 16 us slower by both.
constexpr int64_t kBothTiles = 2048;
struct Plan {
  int rc;
  bool chunk;
};
static Plan attend_plan(int n, int max_q, int max_kv, int G, int H) {
  const int64_t rows = (int64_t)max_q * G;
  if (const int rc = few_capacity(rows)) return {rc, false};
  const bool both = n > 1 && (int64_t)n * H * ((max_kv + 127) / 128) > kBothTiles;
  return {both ? few_capacity(G) : 0, true};
}

size_t tc_attend_workspace_bytes(int n, int max_q, int max_kv, int G, int H, int d) {
  const Plan p = attend_plan(n, max_q, max_kv, G, H);
  size_t bytes = p.rc ? (few_workspace_bytes(n, max_kv, H, d, p.rc) + 255) / 256 * 256 : 0;
  if (p.chunk) {
    const int64_t blocks = chunk_blocks(n, max_q, max_kv, G, H);
    bytes += chunk_starts_bytes(blocks) + (size_t)(blocks * 2 * kUnitRows * (d + 2) * 4);
  }
  return bytes;
}

int tc_attend(const AttendLaunch& a, int L, int d, cudaStream_t s) {
  (void)L;
  const bool q8 = a.e.k != nullptr;
  const Plan plan = attend_plan(a.req.n, a.req.max_q, a.req.max_kv, a.G, a.H);
  ChunkLaunch p;
  p.a = a;
  p.min_rows = plan.rc + 1;
  p.blocks = (int)chunk_blocks(a.req.n, a.req.max_q, a.req.max_kv, a.G, a.H);
  if (p.blocks <= 0) return KVC_E_CUDA;
  p.fine = 4 * chunk_units(a.req.n, a.req.max_q, a.G, a.H) <= p.blocks;
  CUtensorMap mk, mv;
  bool ok;
  if (q8)
    ok = encode_attend_tile(&mk, &p.g, a.c, reinterpret_cast<const uint8_t*>(a.c.k), a.layer, a.H, d) &&
         encode_attend_tile(&mv, &p.g, a.c, reinterpret_cast<const uint8_t*>(a.c.v), a.layer, a.H, d);
  else
    ok = encode_attend_tile(&mk, &p.g, a.c, a.c.k, a.layer, a.H, d) && encode_attend_tile(&mv, &p.g, a.c, a.c.v, a.layer, a.H, d);
  if (!ok) return KVC_E_UNSUPPORTED;
  uint8_t* ws = reinterpret_cast<uint8_t*>(a.part);
  if (plan.rc) {
    if (launch_attend_few(a, p.g, mk, mv, plan.rc, d, a.part, s) != cudaSuccess) return KVC_E_CUDA;
    ws += (few_workspace_bytes(a.req.n, a.req.max_kv, a.H, d, plan.rc) + 255) / 256 * 256;
  }
  if (!plan.chunk) return KVC_OK;
  p.starts = reinterpret_cast<UnitStart*>(ws);
  p.ml = reinterpret_cast<float*>(ws + chunk_starts_bytes(p.blocks));
  p.part = p.ml + (int64_t)p.blocks * 2 * kUnitRows * 2;
  cudaError_t e;
  if (d == 128)
    e = q8 ? launch_chunk<128, true>(p, mk, mv, s) : launch_chunk<128, false>(p, mk, mv, s);
  else
    e = q8 ? launch_chunk<64, true>(p, mk, mv, s) : launch_chunk<64, false>(p, mk, mv, s);
  return e == cudaSuccess ? KVC_OK : KVC_E_CUDA;
}

}  // namespace kvc
