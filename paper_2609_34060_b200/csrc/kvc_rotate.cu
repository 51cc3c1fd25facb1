// kvc_append_rotated: queries and keys of the new tokens turned to their positions, keys and values written into the cache.
//
//     (x, y) -> a (x cos - y sin, x sin + y cos) ,  angle = p f_k ,
// over the first `rot` channels of a head.  Bound: the bytes of the rows, read once and written once.  A block has all
// heads of a token, or of eight: they share the angles, which its threads work out while the first rows are on their way.
// An angle is p f_k / 2 pi turns, less the whole ones, in float64 (position 2^20: off by 2e-10 of a turn), cos and sin of
// the rest in float32.
//
// Measured: five prompts of 1500-2500 tokens, 28 / 4 heads of 128 into bf16 pages (167 MB): 33 us, 5.1 TB/s of 6.5 copied
// (a block a token 36, four 37, 32 tokens 57; streaming loads and stores no better); 32 trees of 9-63 drafts 6.8 us, 64
// single tokens into 8-bit pages 3.2 us, where launch and the chain lists -> pages -> rows bound it.
//
// Layout of the work: d / 16 neighbouring lanes hold one row, 16 channels each: two 16-byte chunks that hold pairs, half a
// rotated width apart (KVC_ROPE_HALF) or side by side.  Eight bits: the row's largest magnitude over its lanes, exponents
// and codes as in kvc_quantize, from the float32 products (rounded once).
#include <cuda_runtime.h>

#include "kvc_draft.h"
#include "kvc_launch.h"
#include "kvc_tc_attend.cuh"

namespace kvc {
namespace {

// 16 values of a row -> 16 codes and the row's exponent (the same in all LPR lanes of the row)
template <int LPR>
__device__ __forceinline__ void encode16(float* x, uint32_t& b, uint2& lo, uint2& hi) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint32_t m = __float_as_uint(x[i]) & 0x7fffffffu;
    if (m < 0x7f800000u)
      top = max(top, m);
    else
      x[i] = __uint_as_float(0x7fc00000u);                        // infinities become NaN, neither counts towards the scale
  }
#pragma unroll
  for (int o = LPR / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  b = row_exponent(__uint_as_float(top));
  const float s = exponent_down(b);
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] *= s;
  if (b >= 247u) {                                                // 256 * 2^120 is no finite bf16
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (fabsf(x[i]) > 240.f) x[i] = copysignf(240.f, x[i]);
  }
  lo = make_uint2(e4m3x2(x[0], x[1]) | (e4m3x2(x[2], x[3]) << 16), e4m3x2(x[4], x[5]) | (e4m3x2(x[6], x[7]) << 16));
  hi = make_uint2(e4m3x2(x[8], x[9]) | (e4m3x2(x[10], x[11]) << 16), e4m3x2(x[12], x[13]) | (e4m3x2(x[14], x[15]) << 16));
}

constexpr int kUnroll = 2;
constexpr int64_t kManyTokens = 7000;

// grid: x = tiles of TOKENS tokens of a request, y = requests (strided)
template <int D, bool Q8, int TOKENS>
__global__ void __launch_bounds__(256) append_rotated_kernel(const __grid_constant__ RotateLaunch p) {
  constexpr int LPR = D / 16;
  __shared__ alignas(16) float s_cos[TOKENS][kMaxHalfD], s_sin[TOKENS][kMaxHalfD];
  __shared__ int64_t s_off[TOKENS], s_exp[TOKENS];        // of the tokens' rows in the layer, head 0; -1: none
  tc::grid_dependency_wait();
  tc::grid_dependents_launch();
  const int tid = threadIdx.x, step = (int)blockDim.x, j0 = (int)blockIdx.x * TOKENS;
  const int heads = p.Hq + 2 * p.H, half = p.rot / 2;
  // r / heads for a row r of the tile: quotients below 8 with steps of at least 2^-18 between them, off by less than 2^-20
  const float each = 1.f / (float)heads;
  auto token_of = [&](int r) { return TOKENS == 1 ? 0 : (int)(((float)r + 0.5f) * each); };
  for (int b = blockIdx.y; b < p.req.n; b += gridDim.y) {
    int q0, nq, kv;
    request_span(p.req, b, tid == 0 && j0 == 0 ? p.status : nullptr, q0, nq, kv);
    if (j0 >= nq) continue;
    const int nt = min(TOKENS, nq - j0), items = nt * heads * LPR, lane = tid % LPR;   // step is a multiple of LPR
    // 16 channels of a row a lane, in two chunks
    const bool turns = lane * 16 < p.rot, far = turns && p.pairing == KVC_ROPE_HALF;
    const int ch0 = far ? 8 * lane : 16 * lane, ch1 = far ? half + 8 * lane : 16 * lane + 8;
    uint4 lo[kUnroll], hi[kUnroll];
    auto load = [&](int i0) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int i = i0 + u * step + tid, r = i / LPR, tk = token_of(r), head = r - tk * heads;
        lo[u] = hi[u] = make_uint4(0, 0, 0, 0);
        if (i >= items) continue;
        const bool is_q = head < p.Hq, is_k = head < p.Hq + p.H;
        const DevHeads& src = is_q ? p.q : is_k ? p.kn : p.vn;
        const __nv_bfloat16* x = src.p + (int64_t)(q0 + j0 + tk) * src.s_row + (int64_t)(head - (is_q ? 0 : is_k ? p.Hq : p.Hq + p.H)) * src.s_head;
        lo[u] = *reinterpret_cast<const uint4*>(x + ch0);
        hi[u] = *reinterpret_cast<const uint4*>(x + ch1);
      }
    };
    load(0);
    // while the first rows are on their way: angles, and where the tokens' rows go
    for (int i = tid; i < nt * half; i += step) {
      const int tk = TOKENS == 1 ? 0 : i / half, k = i - tk * half, j = j0 + tk;
      const double pos = (double)((int64_t)(p.pos_begin ? p.pos_begin[b] : 0) + (kv - nq) + (p.depth ? p.depth[q0 + j] : j));
      const double rounds = pos * p.turns[k];
      float sn, cs;
      sincospif((float)(2.0 * (rounds - rint(rounds))), &sn, &cs);
      s_cos[tk][k] = cs * p.amplitude;
      s_sin[tk][k] = sn * p.amplitude;
    }
    if (tid < nt) {
      const int at = kv - nq + j0 + tid;
      int page = at < 0 ? -1 : 0;
      if (at < 0) atomicOr(p.status, KVC_FLAG_BAD_LENGTH);
      if (at >= 0 && is_paged(p.dst)) page = request_page(p.req, p.dst, b, at, p.status);
      s_off[tid] = page < 0 ? -1 : row_off(p.dst, p.layer, 0, at, page);
      if (Q8) s_exp[tid] = page < 0 ? -1 : exp_off(p.e, p.dst, p.layer, 0, at, page);
    }
    __syncthreads();
    for (int i0 = 0; i0 < items; i0 += kUnroll * step) {
      if (i0 > 0) load(i0);
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int i = i0 + u * step + tid, r = i / LPR, tk = min(token_of(r), nt - 1), head = i < items ? r - tk * heads : -1;
        const bool is_q = head < p.Hq, is_v = head >= p.Hq + p.H;
        float x[16];
        unpack8(lo[u], x);
        unpack8(hi[u], x + 8);
        if (turns && !is_v) {
          float cs[8], sn[8];
          *reinterpret_cast<float4*>(cs) = *reinterpret_cast<const float4*>(&s_cos[tk][8 * lane]);
          *reinterpret_cast<float4*>(cs + 4) = *reinterpret_cast<const float4*>(&s_cos[tk][8 * lane + 4]);
          *reinterpret_cast<float4*>(sn) = *reinterpret_cast<const float4*>(&s_sin[tk][8 * lane]);
          *reinterpret_cast<float4*>(sn + 4) = *reinterpret_cast<const float4*>(&s_sin[tk][8 * lane + 4]);
          rope16(x, cs, sn, p.pairing);
          if (!Q8 || is_q) {
            lo[u] = pack8(x);
            hi[u] = pack8(x + 8);
          }
        }
        if (head >= 0 && is_q) {
          __nv_bfloat16* y = p.qo.p + (int64_t)(q0 + j0 + tk) * p.qo.s_row + (int64_t)head * p.qo.s_head;
          *reinterpret_cast<uint4*>(y + ch0) = lo[u];
          *reinterpret_cast<uint4*>(y + ch1) = hi[u];
        }
        const int64_t off = s_off[tk];
        const bool write = head >= 0 && !is_q && off >= 0;
        const int h = head - (is_v ? p.Hq + p.H : p.Hq);          // of the cache
        if constexpr (Q8) {
          if (!__any_sync(0xffffffffu, write)) continue;
          uint32_t e;
          uint2 first, second;
          encode16<LPR>(x, e, first, second);                     // every lane takes part in the shuffles
          if (!write) continue;
          uint8_t* y = reinterpret_cast<uint8_t*>(is_v ? p.dst.v : p.dst.k) + off + (int64_t)h * p.dst.s_head;
          *reinterpret_cast<uint2*>(y + ch0) = first;
          *reinterpret_cast<uint2*>(y + ch1) = second;
          if (lane == 0) (is_v ? p.e.v : p.e.k)[s_exp[tk] + (int64_t)h * p.e.s_head] = (uint8_t)e;
        } else if (write) {
          __nv_bfloat16* y = (is_v ? p.dst.v : p.dst.k) + off + (int64_t)h * p.dst.s_head;
          *reinterpret_cast<uint4*>(y + ch0) = lo[u];
          *reinterpret_cast<uint4*>(y + ch1) = hi[u];
        }
      }
    }
    __syncthreads();                                              // before the next request's angles
  }
}

}  // namespace

cudaError_t launch_append_rotated(const RotateLaunch& r, int d, cudaStream_t s) {
  // Where the bounds allow 7000 tokens and more, eight a block, whose rows stream behind one set of angles; otherwise one, as
  // many threads as it has work (eight would leave SMs without a block).  Measured, us, one token a block and eight, heads of
  // 128, tokens in all:
  //                  64        2100       4000       6000       8000       32000
  //     32 / 8 bf16  3.0  7.8  13.0 14.7  22.2 20.8  30.8 34.4  40.0 37.9  145 129
  //     32 / 8 8-bit 3.1  9.6  15.2 17.7  25.7 29.9  36.1 34.5  47.0 46.1  174 149
  //     8 / 1 bf16   2.9  4.3  4.8  5.3   7.5  7.8   10.8 12.8  14.7 15.3  47  46
  // and 64 single tokens under bounds of 2000 each 141 and 32: most blocks find nothing.
  const int tokens = (int64_t)r.req.n * r.req.max_q >= kManyTokens ? 8 : 1;
  const int64_t each = ((int64_t)tokens * (r.Hq + 2 * r.H) * (d / 16) + kUnroll - 1) / kUnroll;
  const int threads = each < kMaxHalfD ? kMaxHalfD : each > 256 ? 256 : (int)((each + 31) / 32 * 32);
  const dim3 g((unsigned)(((int64_t)r.req.max_q + tokens - 1) / tokens), (unsigned)(r.req.n < 65535 ? r.req.n : 65535));
  const bool q8 = r.e.k != nullptr;
#define KVC_ROTATE(D, Q, T) \
  if (d == D && q8 == Q && tokens == T) return tc::launch_after(append_rotated_kernel<D, Q, T>, g, threads, 0, s, r);
  KVC_ROTATE(128, false, 1) KVC_ROTATE(128, true, 1) KVC_ROTATE(64, false, 1) KVC_ROTATE(64, true, 1)
  KVC_ROTATE(128, false, 8) KVC_ROTATE(128, true, 8) KVC_ROTATE(64, false, 8) KVC_ROTATE(64, true, 8)
#undef KVC_ROTATE
  return cudaErrorInvalidValue;
}

}  // namespace kvc
