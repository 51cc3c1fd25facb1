// kvc_attend for chunks of new tokens: tiles of 2 x 128 query rows against tiles of 128 keys on the tensor cores.
//
//     S = Q K^T  (tcgen05, f32 in tensor memory) ,  P = exp2(c S - c m) ,  O += P V  (P bf16 in tensor memory) ,
// c = scale log2 e, m a running row maximum.  The rows of a request and KV head are packed as token * G + query head, so
// the G heads that share K and V share the tile, and a few tokens fill it.
//
// Bound: 4 d flops a (row, key) pair on the tensor cores and one exponential; at d = 128 a 128 x 128 tile costs 1024
// cycles of either.  So one block keeps two row tiles going: while the softmax warps of one work, the tensor cores run
// the other's products.  P lies over S in tensor memory (2 x 128 columns of S, 2 x d of O: all 512), and A operands come
// from there: P never passes through shared memory.
//
// m moves lazily: only when a row's maximum grows by more than 2^8 are its sum and its accumulators rescaled (exact in
// float32 up to rounding; exponentials then reach 2^8, far inside every range).  Rescaling is rare after the first
// tiles, so the softmax warps do it themselves.
//
// Rounding: P to bf16 (2^-8 of each term: what the tensor cores take), everything else float32.
//
// Warps: 0-3 and 4-7 softmax and epilogue of the row tiles (a thread a row), 8 TMA producer, 9 MMA issue (one thread),
// 8-bit caches: 12-15 turn raw tiles into bf16 ones (code * 2^e, exact).  Every wait is bounded; on expiry the CTA
// records KVC_FLAG_WAIT_EXPIRED and returns.
//
// Few rows against many keys leave SMs idle: the keys are then split over `nsplit` blocks, whose float32 partial results
// (unnormalised sums, maximum and sum of each row) a second kernel joins in a fixed order.
#include <cuda_runtime.h>

#include "kvc_launch.h"
#include "kvc_tc.h"
#include "kvc_tc_attend.cuh"
#include "kvc_tc_attend_few.h"

namespace kvc {
namespace {

using namespace tc;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLazy = 8.f;               // log2 of the growth of a row's maximum that is let pass
constexpr int kUnitRows = 256;

struct ChunkLaunch {
  AttendLaunch a;
  TileGeo g;                               // of the raw tile
  int32_t nsplit, units_u;                 // key splits; row units a request may have
  int32_t min_rows;                        // requests with fewer rows belong to the other kernel
};

template <int D, bool Q8>
struct Shape {
  static constexpr int kTile = 128 * D * 2;                       // bytes of a bf16 tile
  static constexpr int kRaw = 128 * D;
  static constexpr int kSlots = Q8 ? 3 : (D == 128 ? 5 : 8);
  static constexpr int kRawSlots = Q8 ? 3 : 0;
  static constexpr int kThreads = Q8 ? 512 : 384;
  static constexpr int kSmem = 1024 + 2 * kTile + kSlots * kTile + kRawSlots * kRaw + 512;
};

struct Bars {
  uint64_t q_full[2], s_full[2], p_ready[2], o_done[2], v_clean;
  uint64_t full[8], empty[8], raw_full[4], raw_empty[4];
  uint32_t tmem;
  int abort_flag;
};

// the row unit of this block
struct Unit {
  int b, h, u, split, q0, nq, kv, rows, tiles0, tiles[2], n[2];   // first key tile, end tile and count of each row tile
  __device__ __forceinline__ bool decode(const ChunkLaunch& p, bool flag) {
    int x = blockIdx.x;
    split = x % p.nsplit;
    x /= p.nsplit;
    h = x % p.a.H;
    x /= p.a.H;
    b = x % p.a.req.n;
    u = p.units_u - 1 - x / p.a.req.n;                            // the longest units of a causal chunk first
    request_span(p.a.req, b, flag && u == 0 && h == 0 && split == 0 ? p.a.status : nullptr, q0, nq, kv);
    rows = nq * p.a.G;
    if (rows < p.min_rows || u * kUnitRows >= rows) return false;
    int all = 0;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int first = u * kUnitRows + t * 128, last = min(first + 128, rows) - 1;
      int keys = 0;
      if (first < rows) keys = p.a.causal ? max(0, kv - nq + last / p.a.G + 1) : kv;
      tiles[t] = (keys + 127) >> 7;
      all = max(all, tiles[t]);
    }
    const int per = (all + p.nsplit - 1) / p.nsplit;
    tiles0 = min(split * per, all);
    const int end = min(tiles0 + per, all);
#pragma unroll
    for (int t = 0; t < 2; ++t) n[t] = max(0, min(tiles[t], end) - tiles0);
    return true;
  }
  __device__ __forceinline__ int count() const { return max(n[0], n[1]); }
};

template <int D, bool Q8>
__global__ void __launch_bounds__(Shape<D, Q8>::kThreads, 1)
attend_chunk_kernel(const __grid_constant__ ChunkLaunch p, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  using SH = Shape<D, Q8>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ Bars bars;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* sq = smem;                                             // [2][NP][128 rows][128 B]
  uint8_t* skv = smem + 2 * SH::kTile;
  uint8_t* sraw = skv + SH::kSlots * SH::kTile;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  Unit un;
  if (!un.decode(p, tid == 0)) return;                            // the same for the whole block
  volatile int* abort_flag = &bars.abort_flag;
  const uint32_t q_full = smem_u32(bars.q_full), s_full = smem_u32(bars.s_full), p_ready = smem_u32(bars.p_ready), o_done = smem_u32(bars.o_done);
  const uint32_t full = smem_u32(bars.full), empty = smem_u32(bars.empty), rfull = smem_u32(bars.raw_full), rempty = smem_u32(bars.raw_empty);
  const uint32_t v_clean = smem_u32(&bars.v_clean);
  if (tid == 0) {
    for (int t = 0; t < 2; ++t) {
      mbar_init(q_full + 8 * t, 128);
      mbar_init(s_full + 8 * t, 1);
      mbar_init(p_ready + 8 * t, 128);
      mbar_init(o_done + 8 * t, 1);
    }
    mbar_init(v_clean, 32);
    for (int s = 0; s < SH::kSlots; ++s) {
      mbar_init(full + 8 * s, Q8 ? 128 : 1);
      mbar_init(empty + 8 * s, 1);
    }
    for (int s = 0; s < SH::kRawSlots; ++s) {
      mbar_init(rfull + 8 * s, 1);
      mbar_init(rempty + 8 * s, 128);
    }
    bars.abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == 9) {
    tmem_alloc(smem_u32(&bars.tmem), 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars.tmem;
  const int n_all = un.count();
  // the tile's strides as the tensor cores see it
  const uint32_t gs = Q8 ? 1024u : (uint32_t)p.g.gs, ps = Q8 ? 16384u : (uint32_t)p.g.ps;
  const int tail = un.kv - (un.tiles0 + n_all - 1) * 128;         // valid rows of the last tile of this block
  const bool clean = !Q8 && n_all > 0 && tail < 128;              // stale rows behind them: values must be zeroed

  if (warp < 8) {
    regs_inc<Q8 ? 184 : 216>();
    const int t = warp >> 2, row = (tid & 127);
    const int r = un.u * kUnitRows + t * 128 + row;
    const bool live = r < un.rows;
    const int tok = r / p.a.G, head = un.h * p.a.G + r % p.a.G;
    const int n = un.n[t];
    const int lim = !live ? -1 : p.a.causal ? un.kv - un.nq + tok : un.kv - 1;
    const float c = p.a.scale * kLog2e;
    const float minus_inf = __uint_as_float(0xff800000u);
    float m = minus_inf, l = 0.f;
    if (n > 0) {
      uint8_t* dst = sq + t * SH::kTile + (row >> 3) * 1024 + (row & 7) * 128;
      const __nv_bfloat16* src = p.a.q.p + (int64_t)(un.q0 + tok) * p.a.q.s_row + (int64_t)head * p.a.q.s_head;
#pragma unroll
      for (int j = 0; j < D / 8; ++j) {
        const uint4 x = live ? *reinterpret_cast<const uint4*>(src + 8 * j) : make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>(dst + (j >> 3) * 16384 + (((j & 7) ^ (row & 7)) << 4)) = x;
      }
      fence_proxy_async();
      mbar_arrive(q_full + 8 * t);
    }
    const uint32_t lane_at = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t s_at = lane_at + t * 128, o_at = lane_at + 256 + t * D;
    bool ok = true;
    for (int it = 0; it < n; ++it) {
      if (!wait_all(s_full + 8 * t, it & 1, abort_flag)) {
        ok = false;
        break;
      }
      tc_fence_after();
      float s[128];
#pragma unroll
      for (int k = 0; k < 4; ++k) tmem_ld32(s_at + 32 * k, s + 32 * k);
      tmem_ld_wait();
      const int t0 = (un.tiles0 + it) * 128;
      if (__any_sync(0xffffffffu, lim < t0 + 127)) {
#pragma unroll
        for (int k = 0; k < 128; ++k) s[k] = t0 + k <= lim ? s[k] : minus_inf;
      }
      float mx0 = s[0], mx1 = s[1], mx2 = s[2], mx3 = s[3];
#pragma unroll
      for (int k = 4; k < 128; k += 4) {
        mx0 = fmaxf(mx0, s[k]);
        mx1 = fmaxf(mx1, s[k + 1]);
        mx2 = fmaxf(mx2, s[k + 2]);
        mx3 = fmaxf(mx3, s[k + 3]);
      }
      const float top = fmaxf(m, fmaxf(fmaxf(mx0, mx1), fmaxf(mx2, mx3)));
      const bool grow = (top - m) * c > kLazy;                    // a first finite maximum too (m = -inf)
      if (__any_sync(0xffffffffu, grow)) {
        const float keep = grow ? exp2_fast((m - top) * c) : 1.f;
        if (it > 0) {
          if (!wait_all(o_done + 8 * t, (it - 1) & 1, abort_flag)) {
            ok = false;
            break;
          }
          tc_fence_after();
#pragma unroll
          for (int k = 0; k < D; k += 32) {
            float o[32];
            tmem_ld32(o_at + k, o);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] *= keep;
            tmem_st32(o_at + k, reinterpret_cast<const uint32_t*>(o));
          }
          tmem_st_wait();
        }
        if (grow) {
          l *= keep;
          m = top;
        }
      }
      const float mc = m == minus_inf ? 0.f : m * c;
      const f32x2 c2 = f2_pack(c, c), mc2 = f2_pack(-mc, -mc);
      f32x2 sum2 = f2_pack(0.f, 0.f);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        uint32_t w[32];
#pragma unroll
        for (int k = 0; k < 32; ++k) {
          float a, b;
          f2_unpack(f2_fma(f2_pack(s[half * 64 + 2 * k], s[half * 64 + 2 * k + 1]), c2, mc2), a, b);
          const f32x2 e = f2_pack(exp2_fast(a), exp2_fast(b));
          sum2 = f2_add(sum2, e);
          w[k] = f2_to_bf16x2(e);
        }
        tmem_st32(s_at + 32 * half, w);
      }
      float sa, sb;
      f2_unpack(sum2, sa, sb);
      l += sa + sb;
      tmem_st_wait();
      tc_fence_before();
      mbar_arrive(p_ready + 8 * t);
    }
    if (ok && n > 0) ok = wait_all(o_done + 8 * t, (n - 1) & 1, abort_flag);
    tc_fence_after();
    const bool dead = l == 0.f;                                   // no key seen
    if (p.nsplit == 1) {
      const float inv = dead ? 0.f : 1.f / l;
      __nv_bfloat16* dst = p.a.out.p + (int64_t)(un.q0 + tok) * p.a.out.s_row + (int64_t)head * p.a.out.s_head;
#pragma unroll
      for (int k = 0; k < D; k += 32) {
        float o[32];
        if (n > 0) {
          tmem_ld32(o_at + k, o);
          tmem_ld_wait();
        }
        if (live && ok) {
#pragma unroll
          for (int j = 0; j < 32; ++j) o[j] = dead ? 0.f : o[j] * inv;
#pragma unroll
          for (int j = 0; j < 32; j += 8) *reinterpret_cast<uint4*>(dst + k + j) = pack8(o + j);
        }
      }
      if (live && ok && p.a.lse) p.a.lse[(int64_t)(un.q0 + tok) * (p.a.H * p.a.G) + head] = dead ? minus_inf : m * p.a.scale + log2f(l) * kLn2;
    } else {
      const int64_t slot = ((((int64_t)un.b * p.a.H + un.h) * p.units_u + un.u) * p.nsplit + un.split) * kUnitRows + t * 128 + row;
      const int64_t slots = (int64_t)p.a.req.n * p.a.H * p.units_u * p.nsplit * kUnitRows;
      float* dst = p.a.part + 2 * slots + slot * D;
#pragma unroll
      for (int k = 0; k < D; k += 32) {
        float o[32];
        if (n > 0) {
          tmem_ld32(o_at + k, o);
          tmem_ld_wait();
        }
        if (live && ok && n > 0) {
#pragma unroll
          for (int j = 0; j < 32; j += 4) *reinterpret_cast<float4*>(dst + k + j) = make_float4(o[j], o[j + 1], o[j + 2], o[j + 3]);
        }
      }
      if (live) {
        p.a.part[2 * slot] = m;
        p.a.part[2 * slot + 1] = ok ? l : 0.f;
      }
    }
    tc_fence_before();
  } else {
    regs_dec<72>();
    if (warp == 8) {
      // ---- producer: K, V tiles in the order in which the products take them
      const uint32_t ring = smem_u32(Q8 ? sraw : skv);
      const uint32_t bytes = Q8 ? SH::kRaw : SH::kTile;
      constexpr int NS = Q8 ? SH::kRawSlots : SH::kSlots;
      const uint32_t fb = Q8 ? rfull : full, eb = Q8 ? rempty : empty;
      int slot = 0, phase = 0;
      bool ok = true;
      int ahead = n_all > 0 ? tile_entry(p.a, p.g, un.b, un.tiles0 * 128, min(128, un.kv - un.tiles0 * 128), lane) : 0;
      for (int it = 0; it < n_all && ok; ++it) {
        const int t0 = (un.tiles0 + it) * 128, rows = min(128, un.kv - t0);
        const int page = ahead;
        if (it + 1 < n_all) ahead = tile_entry(p.a, p.g, un.b, t0 + 128, min(128, un.kv - t0 - 128), lane);
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          if (!wait_all(eb + 8 * slot, phase ^ 1, abort_flag)) {
            ok = false;
            break;
          }
          tile_load(kv ? &map_v : &map_k, p.a, p.g, ring + slot * bytes, fb + 8 * slot, t0, rows, un.h, page, lane);
          if (clean && kv && it == n_all - 1) {
            // stale rows behind the last key: P is zero there, but zero times a stale NaN would not be
            if (mbar_wait(fb + 8 * slot, phase, abort_flag)) {
              uint8_t* v = skv + slot * SH::kTile;
              for (int x = lane; x < (128 - rows) * (D / 8); x += 32) {
                const int rr = rows + x / (D / 8), ch = x % (D / 8);
                *reinterpret_cast<uint4*>(v + (rr >> 3) * gs + (ch >> 3) * ps + (rr & 7) * 128 + ((ch & 7) << 4)) = make_uint4(0, 0, 0, 0);
              }
              fence_proxy_async();
            }
            mbar_arrive(v_clean);
          }
          if (++slot == NS) {
            slot = 0;
            phase ^= 1;
          }
        }
      }
    } else if (warp == 9) {
      if (n_all > 0) {
        constexpr uint32_t idesc_s = idesc_bf16(128, 128, 0, 0), idesc_o = idesc_bf16(128, D, 0, 1);
        const uint32_t kv0 = smem_u32(skv);
        bool ok = true;
        auto wait = [&](uint32_t bar, uint32_t parity) {
          if (ok) ok = wait_all(bar, parity, abort_flag);
          return ok;
        };
        // descriptors differ in their start address alone (its 18 bits / 16 are the low word)
        const uint64_t q_desc = operand_desc(smem_u32(sq), 16, 1024, 2), k_desc = operand_desc(kv0, 16, gs, 2), v_desc = operand_desc(kv0, ps, gs, 2);
        const uint32_t k_part = ps >> 4, v_step = (2 * gs) >> 4;
        auto score = [&](int t, int slot) {                       // S_t = Q_t K^T
          const uint64_t qd = q_desc + (uint32_t)(t * (SH::kTile >> 4)), kd = k_desc + (uint32_t)(slot * (SH::kTile >> 4));
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
              umma_bf16(tmem + t * 128, qd + ((k >> 2) * 1024 + (k & 3) * 2), kd + ((k >> 2) * k_part + (k & 3) * 2), idesc_s, k > 0);
            umma_commit(s_full + 8 * t);
          }
        };
        auto values = [&](int t, int slot, bool acc) {            // O_t += P_t V
          const uint64_t vd = v_desc + (uint32_t)(slot * (SH::kTile >> 4));
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
              umma_bf16_ts(tmem + 256 + t * D, tmem + t * 128 + 8 * k, vd + k * v_step, idesc_o, acc || k > 0);
            umma_commit(o_done + 8 * t);
          }
        };
        auto release = [&](int slot) {
          if (elect_one()) umma_commit(empty + 8 * slot);
        };
        int slot = 0, phase = 0;
        auto next = [&]() {
          if (++slot == SH::kSlots) {
            slot = 0;
            phase ^= 1;
          }
        };
        if (wait(full, 0)) {
          for (int t = 0; t < 2; ++t)
            if (un.n[t] > 0 && wait(q_full + 8 * t, 0)) {
              tc_fence_after();
              score(t, 0);
            }
          release(0);
          next();
        }
        for (int it = 0; it < n_all && ok; ++it) {
          const int vs = slot, vphase = phase;
          next();
          const int ks = slot, kphase = phase;
          const bool more = it + 1 < n_all;
          if (!wait(full + 8 * vs, vphase)) break;
          if (clean && !more && !wait(v_clean, 0)) break;
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (!ok || it >= un.n[t]) continue;
            if (!wait(p_ready + 8 * t, it & 1)) break;
            tc_fence_after();
            values(t, vs, it > 0);
            if (it + 1 < un.n[t]) {
              if (!wait(full + 8 * ks, kphase)) break;
              tc_fence_after();
              score(t, ks);
            }
          }
          if (!ok) break;
          release(vs);
          if (more) {
            release(ks);
            next();
          }
        }
      }
    } else if (Q8 && warp >= 12) {
      // ---- 8-bit tiles to bf16: a thread a token row
      const int r = tid & 127;
      constexpr int CH = D / 16;                                  // 16-byte chunks of a raw row
      const uint32_t sw = D == 128 ? (uint32_t)(r & 7) : (uint32_t)((r >> 1) & 3);
      int rs = 0, rphase = 0, slot = 0, phase = 0;
      bool ok = true;
      auto exponents = [&](int it, float& ek, float& ev) {
        ek = ev = 1.f;
        const int tt = (un.tiles0 + it) * 128 + r;
        if (it >= n_all || tt >= un.kv) return;
        int64_t o = (int64_t)p.a.layer * p.a.e.s_layer + (int64_t)un.h * p.a.e.s_head;
        if (p.g.paged) {
          const int page = request_page(p.a.req, p.a.c, un.b, tt, nullptr);
          if (page < 0) return;
          o += (int64_t)page * p.a.e.s_page + (int64_t)(tt & p.a.c.page_mask) * p.a.e.s_tok;
        } else {
          o += (int64_t)tt * p.a.e.s_tok;
        }
        ek = exponent_up(p.a.e.k[o]);
        ev = exponent_up(p.a.e.v[o]);
      };
      float ek, ev;
      exponents(0, ek, ev);
      for (int it = 0; it < n_all && ok; ++it) {
        float nk, nv;
        exponents(it + 1, nk, nv);
        const bool valid = (un.tiles0 + it) * 128 + r < un.kv;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          if (!mbar_wait(rfull + 8 * rs, rphase, abort_flag) || !mbar_wait(empty + 8 * slot, phase ^ 1, abort_flag)) {
            ok = false;
            break;
          }
          const uint8_t* in = sraw + rs * SH::kRaw + r * D;
          uint8_t* out = skv + slot * SH::kTile + (r >> 3) * 1024 + (r & 7) * 128;
          const float e = kv ? ev : ek;
#pragma unroll
          for (int ch = 0; ch < CH; ++ch) {
            const uint4 raw = *reinterpret_cast<const uint4*>(in + ((ch ^ sw) << 4));
            const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
            uint32_t o[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float2 lo = e4m3x2_to_float2(w[j] & 0xffffu), hi = e4m3x2_to_float2(w[j] >> 16);
              o[2 * j] = valid ? pack2(lo.x * e, lo.y * e) : 0u;
              o[2 * j + 1] = valid ? pack2(hi.x * e, hi.y * e) : 0u;
            }
            uint8_t* q = out + (ch >> 2) * 16384;
            const int j0 = (2 * ch) & 7;
            *reinterpret_cast<uint4*>(q + ((j0 ^ (r & 7)) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
            *reinterpret_cast<uint4*>(q + (((j0 + 1) ^ (r & 7)) << 4)) = make_uint4(o[4], o[5], o[6], o[7]);
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
  grid_dependents_launch();
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

// ---- join of the key splits: a warp a row
template <int D>
__global__ void __launch_bounds__(256) attend_chunk_join_kernel(const __grid_constant__ ChunkLaunch p) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int units = p.units_u * p.a.H;
  const int b = blockIdx.y, u = (int)(blockIdx.x % p.units_u), h = (int)(blockIdx.x / p.units_u) % p.a.H, seg = (int)(blockIdx.x / units);
  int q0, nq, kv;
  request_span(p.a.req, b, nullptr, q0, nq, kv);
  const int rows = nq * p.a.G;
  grid_dependency_wait();                                         // in every block, also those with nothing to join
  if (rows < p.min_rows) return;
  const int64_t slots = (int64_t)p.a.req.n * units * p.nsplit * kUnitRows;
  const int64_t base = (((int64_t)b * p.a.H + h) * p.units_u + u) * p.nsplit;
  for (int k = 0; k < 4; ++k) {
    const int row = seg * 32 + warp * 4 + k, r = u * kUnitRows + row;
    if (r >= rows) return;
    const float c = p.a.scale * kLog2e, minus_inf = __uint_as_float(0xff800000u);
    float m = minus_inf;
    for (int s = 0; s < p.nsplit; ++s) {
      const int64_t slot = (base + s) * kUnitRows + row;
      if (p.a.part[2 * slot + 1] != 0.f) m = fmaxf(m, p.a.part[2 * slot]);
    }
    float l = 0.f, acc[D / 32];
#pragma unroll
    for (int j = 0; j < D / 32; ++j) acc[j] = 0.f;
    for (int s = 0; s < p.nsplit; ++s) {
      const int64_t slot = (base + s) * kUnitRows + row;
      const float ls = p.a.part[2 * slot + 1];
      if (ls == 0.f) continue;                                    // a split that saw no key wrote no sums
      const float w = exp2f((p.a.part[2 * slot] - m) * c);
      l += w * ls;
      const float* o = p.a.part + 2 * slots + slot * D;
#pragma unroll
      for (int j = 0; j < D / 32; ++j) acc[j] += w * o[j * 32 + lane];
    }
    const bool dead = l == 0.f;
    const float inv = dead ? 0.f : 1.f / l;
    const int64_t tok = q0 + r / p.a.G;
    const int head = h * p.a.G + r % p.a.G;
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
      p.a.out.p[tok * p.a.out.s_row + (int64_t)head * p.a.out.s_head + j * 32 + lane] = __float2bfloat16(dead ? 0.f : acc[j] * inv);
    if (p.a.lse && lane == 0) p.a.lse[tok * (p.a.H * p.a.G) + head] = dead ? minus_inf : m * p.a.scale + log2f(l) * kLn2;
  }
}

int chunk_units(int max_q, int G) { return (int)(((int64_t)max_q * G + kUnitRows - 1) / kUnitRows); }

// Key splits: as many as idle SMs allow, at least four tiles (512 keys) each, so that a block's fixed costs stay small.
int chunk_splits(int64_t units, int max_kv) {
  const int sms = device_sm_count();
  const int tiles = (max_kv + 127) / 128;
  int64_t s = sms > 0 && units > 0 ? sms / units : 1;
  if (s > tiles / 4) s = tiles / 4;
  return s < 1 ? 1 : (int)s;
}

template <int D, bool Q8>
cudaError_t launch_chunk(const ChunkLaunch& p, const CUtensorMap& mk, const CUtensorMap& mv, int64_t blocks, cudaStream_t s) {
  using SH = Shape<D, Q8>;
  static DeviceOnce once;
  int dev;
  if (once.pending(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(attend_chunk_kernel<D, Q8>, cudaFuncAttributeMaxDynamicSharedMemorySize, SH::kSmem);
    if (e != cudaSuccess) return e;
    once.mark(dev);
  }
  attend_chunk_kernel<D, Q8><<<(unsigned)blocks, SH::kThreads, SH::kSmem, s>>>(p, mk, mv);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || p.nsplit == 1) return e;
  const dim3 g((unsigned)(p.units_u * p.a.H * (kUnitRows / 32)), (unsigned)p.a.req.n);
  return launch_after(attend_chunk_join_kernel<D>, g, 256, s, p);
}

}  // namespace

// Which kernels a call launches: requests of up to `rc` rows a KV head go to the few-rows kernel (rc = 0: none), the
// others to this one (chunk = false: there are none).  Decided from the bounds alone: all requests within the few-rows
// kernel's 32 rows take it; a batch of several requests with longer ones among them is served by both, single tokens by
// the few-rows kernel; one long request by this kernel.
struct Plan {
  int rc;
  bool chunk;
};
static Plan attend_plan(int n, int max_q, int G) {
  const int64_t rows = (int64_t)max_q * G;
  if (const int rc = few_capacity(rows)) return {rc, false};
  return {n > 1 ? few_capacity(G) : 0, true};
}

size_t tc_attend_workspace_bytes(int n, int max_q, int max_kv, int G, int H, int d) {
  const Plan p = attend_plan(n, max_q, G);
  size_t bytes = p.rc ? (few_workspace_bytes(n, max_kv, H, d, p.rc) + 255) / 256 * 256 : 0;
  if (p.chunk) {
    const int64_t units = (int64_t)n * H * chunk_units(max_q, G);
    const int ns = chunk_splits(units, max_kv);
    if (ns > 1) bytes += (size_t)(units * ns * kUnitRows * (d + 2) * 4);
  }
  return bytes;
}

int tc_attend(const AttendLaunch& a, int L, int d, cudaStream_t s) {
  (void)L;
  const bool q8 = a.e.k != nullptr;
  const Plan plan = attend_plan(a.req.n, a.req.max_q, a.G);
  ChunkLaunch p;
  p.a = a;
  p.units_u = chunk_units(a.req.max_q, a.G);
  p.min_rows = plan.rc + 1;
  const int64_t units = (int64_t)a.req.n * a.H * p.units_u;
  p.nsplit = chunk_splits(units, a.req.max_kv);
  if (units * p.nsplit >= (int64_t)1 << 31 || a.req.n > 65535) return KVC_E_UNSUPPORTED;
  CUtensorMap mk, mv;
  bool ok;
  if (q8)
    ok = encode_attend_tile(&mk, &p.g, a.c, reinterpret_cast<const uint8_t*>(a.c.k), a.layer, a.H, d) &&
         encode_attend_tile(&mv, &p.g, a.c, reinterpret_cast<const uint8_t*>(a.c.v), a.layer, a.H, d);
  else
    ok = encode_attend_tile(&mk, &p.g, a.c, a.c.k, a.layer, a.H, d) && encode_attend_tile(&mv, &p.g, a.c, a.c.v, a.layer, a.H, d);
  if (!ok) return KVC_E_UNSUPPORTED;
  if (plan.rc) {
    if (launch_attend_few(a, p.g, mk, mv, plan.rc, d, a.part, s) != cudaSuccess) return KVC_E_CUDA;
    p.a.part = a.part + (few_workspace_bytes(a.req.n, a.req.max_kv, a.H, d, plan.rc) + 255) / 256 * 64;
  }
  if (!plan.chunk) return KVC_OK;
  cudaError_t e;
  if (d == 128)
    e = q8 ? launch_chunk<128, true>(p, mk, mv, units * p.nsplit, s) : launch_chunk<128, false>(p, mk, mv, units * p.nsplit, s);
  else
    e = q8 ? launch_chunk<64, true>(p, mk, mv, units * p.nsplit, s) : launch_chunk<64, false>(p, mk, mv, units * p.nsplit, s);
  return e == cudaSuccess ? KVC_OK : KVC_E_CUDA;
}

}  // namespace kvc
