// kvc_attend on the CUDA cores: any shape the checks let through, one pass over the keys with the running maximum and sum
// of the softmax.  The tensor-core kernels serve nearly every call; this one serves the layouts their tensor maps cannot
// describe, and is what they are compared with.
//
// Rows of a request and KV head are packed as token * G + query head: 16 rows a block, 4 a warp.  Tiles of 32 keys and
// values are staged as float32; a lane scores one key against the warp's rows, then owns d / 32 channels of the outputs.
#include <cuda_runtime.h>

#include "kvc_attend.h"
#include "kvc_launch.h"

namespace kvc {
namespace {

constexpr int kRows = 16, kKeys = 32;

template <int D, bool Q8>
__global__ void __launch_bounds__(128) attend_generic_kernel(const __grid_constant__ AttendLaunch p) {
  constexpr int C = D / 32;                 // output channels a lane owns
  __shared__ float ks[kKeys][D + 1];
  __shared__ float vs[kKeys][D];
  __shared__ float qs[kRows][D];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int h = blockIdx.y;
  for (int b = blockIdx.z; b < p.req.n; b += gridDim.z) {
    int q0, nq, kv;
    request_span(p.req, b, threadIdx.x == 0 ? p.status : nullptr, q0, nq, kv);
    const int rows = nq * p.G;
    for (int rb = blockIdx.x * kRows; rb < rows; rb += gridDim.x * kRows) {
      __syncthreads();
      for (int i = threadIdx.x; i < kRows * D; i += 128) {
        const int r = rb + i / D;
        qs[i / D][i % D] = r < rows ? __bfloat162float(p.q.p[(int64_t)(q0 + r / p.G) * p.q.s_row + (int64_t)(h * p.G + r % p.G) * p.q.s_head + i % D]) : 0.f;
      }
      float m[4], l[4], acc[4][C];
      int lim[4];
      const float minus_inf = __uint_as_float(0xff800000u);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int r = rb + warp * 4 + k;
        m[k] = minus_inf;
        l[k] = 0.f;
        lim[k] = r >= rows ? -1 : p.causal ? kv - nq + r / p.G : kv - 1;
#pragma unroll
        for (int c = 0; c < C; ++c) acc[k][c] = 0.f;
      }
      const int last = min(rb + kRows, rows) - 1;
      const int end = p.causal ? kv - nq + last / p.G + 1 : kv;   // keys any row of the block sees
      for (int t0 = 0; t0 < end; t0 += kKeys) {
        __syncthreads();
        {
          const int kr = threadIdx.x >> 2, part = threadIdx.x & 3, t = t0 + kr;
          bool live = t < kv;
          int page = 0;
          if (live && is_paged(p.c)) {
            page = request_page(p.req, p.c, b, t, p.status);
            live = page >= 0;
          }
          const int64_t base = (int64_t)p.layer * p.c.s_layer + (int64_t)h * p.c.s_head +
                               (is_paged(p.c) ? (int64_t)page * p.c.s_page + (int64_t)(t & p.c.page_mask) * p.c.s_tok : (int64_t)t * p.c.s_tok);
          float sk = 1.f, sv = 1.f;
          if (Q8 && live) {
            const int64_t eo = (int64_t)p.layer * p.e.s_layer + (int64_t)h * p.e.s_head +
                               (is_paged(p.c) ? (int64_t)page * p.e.s_page + (int64_t)(t & p.c.page_mask) * p.e.s_tok : (int64_t)t * p.e.s_tok);
            sk = exponent_up(p.e.k[eo]);
            sv = exponent_up(p.e.v[eo]);
          }
#pragma unroll 4
          for (int c = part * (D / 4); c < (part + 1) * (D / 4); c += 2) {
            float2 a = make_float2(0.f, 0.f), v = a;
            if (live) {
              if (Q8) {
                a = e4m3x2_to_float2(*reinterpret_cast<const uint16_t*>(reinterpret_cast<const uint8_t*>(p.c.k) + base + c));
                v = e4m3x2_to_float2(*reinterpret_cast<const uint16_t*>(reinterpret_cast<const uint8_t*>(p.c.v) + base + c));
              } else {
                a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(p.c.k + base + c));
                v = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(p.c.v + base + c));
              }
            }
            ks[kr][c] = a.x * sk;
            ks[kr][c + 1] = a.y * sk;
            vs[kr][c] = v.x * sv;
            vs[kr][c + 1] = v.y * sv;
          }
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (lim[k] < t0) continue;             // the same for the whole warp
          float s = 0.f;
#pragma unroll 8
          for (int c = 0; c < D; ++c) s = fmaf(qs[warp * 4 + k][c], ks[lane][c], s);
          s = t0 + lane <= lim[k] ? s * p.scale : minus_inf;
          float mx = s;
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
          mx = fmaxf(mx, m[k]);
          const float base = mx == minus_inf ? 0.f : mx;   // nothing finite seen yet
          const float e = expf(s - base), keep = expf(m[k] - base);
          m[k] = mx;
          float sum = e;
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
          l[k] = l[k] * keep + sum;
#pragma unroll
          for (int c = 0; c < C; ++c) acc[k][c] *= keep;
          const int n = min(kKeys, lim[k] - t0 + 1);       // a hidden key's value is not touched, whatever it holds
          for (int j = 0; j < n; ++j) {
            const float w = __shfl_sync(0xffffffffu, e, j);
#pragma unroll
            for (int c = 0; c < C; ++c) acc[k][c] = fmaf(w, vs[j][c * 32 + lane], acc[k][c]);
          }
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int r = rb + warp * 4 + k;
        if (r >= rows) continue;
        const int64_t row = q0 + r / p.G;
        const int head = h * p.G + r % p.G;
        const float inv = l[k] > 0.f ? 1.f / l[k] : l[k] == 0.f ? 0.f : l[k];   // a NaN sum stays one
#pragma unroll
        for (int c = 0; c < C; ++c)
          p.out.p[row * p.out.s_row + (int64_t)head * p.out.s_head + c * 32 + lane] = __float2bfloat16(l[k] == 0.f ? 0.f : acc[k][c] * inv);
        if (p.lse && lane == 0) p.lse[row * (p.H * p.G) + head] = l[k] == 0.f ? minus_inf : m[k] + logf(l[k]);
      }
    }
  }
}

}  // namespace

cudaError_t launch_attend_generic(const AttendLaunch& a, int d, cudaStream_t s) {
  const int64_t blocks = ((int64_t)a.req.max_q * a.G + kRows - 1) / kRows;
  const dim3 g((unsigned)(blocks < (1 << 20) ? blocks : 1 << 20), (unsigned)a.H, (unsigned)(a.req.n < 65535 ? a.req.n : 65535));
  const bool q8 = a.e.k != nullptr;
  if (d == 128)
    q8 ? attend_generic_kernel<128, true><<<g, 128, 0, s>>>(a) : attend_generic_kernel<128, false><<<g, 128, 0, s>>>(a);
  else
    q8 ? attend_generic_kernel<64, true><<<g, 128, 0, s>>>(a) : attend_generic_kernel<64, false><<<g, 128, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace kvc
