// kvc_append_rotated: queries and keys of the new tokens turned to their positions, keys and values written into the cache.
//
//     (x, y) -> a (x cos - y sin, x sin + y cos) ,  angle = p f_k ,
// over the first `rot` channels of a head.  Bound: the bytes of the rows, read once and written once.  A block has one
// token, all of its heads: they share the angles, of which rot / 2 threads work out one each while the rows are on their
// way.  An angle is p f_k / 2 pi turns, less the whole ones, in float64 (position 2^20: off by 2e-10 of a turn), cos and
// sin of the rest in float32.
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

constexpr int kMaxThreads = 512, kUnroll = 2;

// grid: x = tokens of a request, y = requests (strided)
template <int D, bool Q8>
__global__ void __launch_bounds__(kMaxThreads) append_rotated_kernel(const __grid_constant__ RotateLaunch p) {
  constexpr int LPR = D / 16;
  __shared__ float s_cos[kMaxHalfD], s_sin[kMaxHalfD];
  tc::grid_dependency_wait();
  tc::grid_dependents_launch();
  const int tid = threadIdx.x, step = (int)blockDim.x, j = (int)blockIdx.x;
  const int items = (p.Hq + 2 * p.H) * LPR;
  for (int b = blockIdx.y; b < p.req.n; b += gridDim.y) {
    int q0, nq, kv;
    request_span(p.req, b, tid == 0 && j == 0 ? p.status : nullptr, q0, nq, kv);
    if (j >= nq) continue;
    const int row = q0 + j, at = kv - nq + j;
    const int ahead = p.depth ? p.depth[row] : j, begin = p.pos_begin ? p.pos_begin[b] : 0;
    int page = at < 0 ? -1 : 0;
    if (at >= 0 && is_paged(p.dst)) page = request_page(p.req, p.dst, b, at, p.status);
    if (at < 0 && tid == 0) atomicOr(p.status, KVC_FLAG_BAD_LENGTH);
    bool angles = false;
    for (int i0 = 0; i0 < items; i0 += kUnroll * step) {
      uint4 lo[kUnroll], hi[kUnroll];
      int head[kUnroll], a[kUnroll], c[kUnroll];                  // head among q, k, v; channels of the two chunks
      bool turn[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int i = i0 + u * step + tid, lane = i % LPR;
        head[u] = i < items ? i / LPR : -1;
        turn[u] = lane * 16 < p.rot && head[u] < p.Hq + p.H;
        const bool half = lane * 16 < p.rot && p.pairing == KVC_ROPE_HALF;
        a[u] = half ? 8 * lane : 16 * lane;
        c[u] = half ? p.rot / 2 + 8 * lane : 16 * lane + 8;
        lo[u] = hi[u] = make_uint4(0, 0, 0, 0);
        if (head[u] < 0) continue;
        const bool is_q = head[u] < p.Hq, is_k = head[u] < p.Hq + p.H;
        const DevHeads& src = is_q ? p.q : is_k ? p.kn : p.vn;
        const __nv_bfloat16* x = src.p + (int64_t)row * src.s_row + (int64_t)(head[u] - (is_q ? 0 : is_k ? p.Hq : p.Hq + p.H)) * src.s_head;
        lo[u] = *reinterpret_cast<const uint4*>(x + a[u]);
        hi[u] = *reinterpret_cast<const uint4*>(x + c[u]);
      }
      if (!angles) {
        const double pos = (double)((int64_t)begin + (kv - nq) + ahead);
        if (tid < p.rot / 2) {
          const double turns = pos * p.turns[tid];
          float sn, cs;
          sincospif((float)(2.0 * (turns - rint(turns))), &sn, &cs);
          s_cos[tid] = cs * p.amplitude;
          s_sin[tid] = sn * p.amplitude;
        }
        __syncthreads();
        angles = true;
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int lane = (i0 + u * step + tid) % LPR;
        float x[16];
        unpack8(lo[u], x);
        unpack8(hi[u], x + 8);
        if (turn[u]) rope16(x, s_cos + 8 * lane, s_sin + 8 * lane, p.pairing);
        const bool is_q = head[u] < p.Hq, is_v = head[u] >= p.Hq + p.H;
        const int h = head[u] - (is_v ? p.Hq + p.H : p.Hq);       // of the cache
        const bool write = head[u] >= 0 && !is_q && page >= 0;
        if (head[u] >= 0 && is_q) {
          __nv_bfloat16* y = p.qo.p + (int64_t)row * p.qo.s_row + (int64_t)head[u] * p.qo.s_head;
          *reinterpret_cast<uint4*>(y + a[u]) = turn[u] ? pack8(x) : lo[u];
          *reinterpret_cast<uint4*>(y + c[u]) = turn[u] ? pack8(x + 8) : hi[u];
        }
        if constexpr (Q8) {
          if (!__any_sync(0xffffffffu, write)) continue;
          uint32_t e;
          uint2 first, second;
          encode16<LPR>(x, e, first, second);                     // every lane takes part in the shuffles
          if (!write) continue;
          uint8_t* y = reinterpret_cast<uint8_t*>(is_v ? p.dst.v : p.dst.k) + row_off(p.dst, p.layer, h, at, page);
          *reinterpret_cast<uint2*>(y + a[u]) = first;
          *reinterpret_cast<uint2*>(y + c[u]) = second;
          if (lane == 0) (is_v ? p.e.v : p.e.k)[exp_off(p.e, p.dst, p.layer, h, at, page)] = (uint8_t)e;
        } else if (write) {
          __nv_bfloat16* y = (is_v ? p.dst.v : p.dst.k) + row_off(p.dst, p.layer, h, at, page);
          *reinterpret_cast<uint4*>(y + a[u]) = turn[u] ? pack8(x) : lo[u];
          *reinterpret_cast<uint4*>(y + c[u]) = turn[u] ? pack8(x + 8) : hi[u];
        }
      }
    }
    __syncthreads();                                              // before the next request's angles
  }
}

}  // namespace

cudaError_t launch_append_rotated(const RotateLaunch& r, int d, cudaStream_t s) {
  const int64_t items = (int64_t)(r.Hq + 2 * r.H) * (d / 16);
  const int64_t each = (items + kUnroll - 1) / kUnroll;
  const int threads = each < kMaxHalfD ? kMaxHalfD : each > kMaxThreads ? kMaxThreads : (int)((each + 31) / 32 * 32);
  const dim3 g((unsigned)r.req.max_q, (unsigned)(r.req.n < 65535 ? r.req.n : 65535));
  const bool q8 = r.e.k != nullptr;
#define KVC_ROTATE(D, Q) \
  if (d == D && q8 == Q) return tc::launch_after(append_rotated_kernel<D, Q>, g, threads, 0, s, r);
  KVC_ROTATE(128, false) KVC_ROTATE(128, true) KVC_ROTATE(64, false) KVC_ROTATE(64, true)
#undef KVC_ROTATE
  return cudaErrorInvalidValue;
}

}  // namespace kvc
