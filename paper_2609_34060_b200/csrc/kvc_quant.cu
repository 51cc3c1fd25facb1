// Caches in 8 bits: kvc_quantize, kvc_dequantize (whole caches, every layer) and kvc_append, kvc_append_q8 (the new
// tokens of a step, one layer).
//
// A row is the d channels of one (token, layer, head), keys or values.  With amax its largest finite magnitude,
//     e = min { integer e >= -127 : amax <= 448 * 2^e } ,  code = rn_e4m3(x * 2^-e) ,  value = code * 2^e .
// Multiplying by a power of two is exact, so the only rounding is the one to e4m3 (to nearest even), and decoding is
// exact in bf16 (at e = 120, where 256 * 2^e would leave its range, magnitudes stop at 240 * 2^e).  All of it is bound by the bytes moved: 3 d + 1 a row to convert, 4 d or 3 d + 1 to append.
//
// Layout of the work: d / 16 neighbouring lanes hold one row, 16 channels each (two 16-byte loads of bf16, one 16-byte
// store of codes).  The row's maximum is taken on the bit patterns (magnitudes of bf16 order like integers), two at a
// time, then a butterfly over the row's lanes.
#include <cuda_runtime.h>

#include "kvc_attend.h"
#include "kvc_launch.h"

namespace kvc {
namespace {

// 16 values of a row -> 16 codes and the row's exponent (the same in all LPR lanes of the row)
template <int LPR>
__device__ __forceinline__ uint4 encode16(const uint4& lo, const uint4& hi, uint32_t& b) {
  uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
  uint32_t m = w[0] & 0x7fff7fffu;
#pragma unroll
  for (int i = 1; i < 8; ++i) m = __vmaxu2(m, w[i] & 0x7fff7fffu);
#pragma unroll
  for (int o = LPR / 2; o > 0; o >>= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, o));
  uint32_t top = max(m & 0xffffu, m >> 16);
  const bool odd = top >= 0x7f00u;             // near the end of the range, or an infinity or NaN in the row (the same in all its lanes)
  if (__any_sync(0xffffffffu, odd)) {
    // infinities become NaN too (e4m3 has none, and 448 would be a plausible number); neither counts towards the scale
    uint32_t f = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t a = w[i] & 0x7fffu, c = (w[i] >> 16) & 0x7fffu;
      if (a < 0x7f80u) f = max(f, a);
      if (c < 0x7f80u) f = max(f, c);
      if (a >= 0x7f80u) w[i] |= 0x7fffu;
      if (c >= 0x7f80u) w[i] |= 0x7fff0000u;
    }
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) f = max(f, __shfl_xor_sync(0xffffffffu, f, o));
    top = f;
  }
  b = row_exponent(__uint_as_float(top << 16));
  const float s = exponent_down(b);
  float x[16];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16) * s;
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u) * s;
  }
  if (b == 247u) {                             // the next code, 256 * 2^120 = 2^128, is no finite bf16
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (fabsf(x[i]) > 240.f) x[i] = copysignf(240.f, x[i]);
  }
  uint32_t c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) c[i] = e4m3x2(x[4 * i], x[4 * i + 1]) | (e4m3x2(x[4 * i + 2], x[4 * i + 3]) << 16);
  return make_uint4(c[0], c[1], c[2], c[3]);
}

__device__ __forceinline__ void decode16(const uint4& c, uint32_t b, uint4& lo, uint4& hi) {
  const float s = exponent_up(b);
  const uint32_t w[4] = {c.x, c.y, c.z, c.w};
  uint32_t o[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = e4m3x2_to_float2(w[i] & 0xffffu), g = e4m3x2_to_float2(w[i] >> 16);
    o[2 * i] = pack2(f.x * s, f.y * s);
    o[2 * i + 1] = pack2(g.x * s, g.y * s);
  }
  lo = make_uint4(o[0], o[1], o[2], o[3]);
  hi = make_uint4(o[4], o[5], o[6], o[7]);
}

// element offset of row (l, h, t); -1 when the table names no page
__device__ __forceinline__ int64_t row_off(const DevCache& c, int l, int h, int t, int page) {
  const int64_t o = (int64_t)l * c.s_layer + (int64_t)h * c.s_head;
  return is_paged(c) ? o + (int64_t)page * c.s_page + (int64_t)(t & c.page_mask) * c.s_tok : o + (int64_t)t * c.s_tok;
}
__device__ __forceinline__ int64_t exp_off(const DevScale& e, const DevCache& c, int l, int h, int t, int page) {
  const int64_t o = (int64_t)l * e.s_layer + (int64_t)h * e.s_head;
  return is_paged(c) ? o + (int64_t)page * e.s_page + (int64_t)(t & c.page_mask) * e.s_tok : o + (int64_t)t * e.s_tok;
}
__device__ __forceinline__ int own_page(const DevCache& c, int t, uint32_t* status) {
  if (!is_paged(c)) return 0;
  const int p = c.page_table[t >> c.page_shift];
  if ((unsigned)p < (unsigned)c.n_phys) return p;
  atomicOr(status, KVC_FLAG_BAD_PAGE);
  return -1;
}

constexpr int kThreads = 256;

// grid: x = token blocks, y = head x (K|V), z = layers (strided).  A thread keeps kUnroll rows in flight: two to quantise
// (one: 296 us, four: 333), one to read back (two: 247), on the 8K and the 16K cache.  Measured: 264 us = 6.1 TB/s to
// quantise the 8K cache (32 layers; 253 us alone and cold under a profiler), 240 us = 5.9 TB/s to read back the 16K one,
// of 6.55 TB/s copied.
template <int D, bool TO8, int kUnroll>
__global__ void __launch_bounds__(kThreads) convert_kernel(const __grid_constant__ ConvertLaunch p) {
  constexpr int LPR = D / 16, RPP = kThreads / LPR;
  const int lane = threadIdx.x % LPR, row = threadIdx.x / LPR;
  const int h = blockIdx.y >> 1, is_v = blockIdx.y & 1;
  const int t0 = blockIdx.x * (RPP * kUnroll);
  __nv_bfloat16* bf = (is_v ? p.bf.v : p.bf.k) + lane * 16;
  uint8_t* q8 = reinterpret_cast<uint8_t*>(is_v ? p.q8.v : p.q8.k) + lane * 16;
  uint8_t* ex = is_v ? p.e.v : p.e.k;
  int pb[kUnroll], pq[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int t = t0 + u * RPP + row;
    pb[u] = t < p.T ? own_page(p.bf, t, p.status) : -1;
    pq[u] = t < p.T ? own_page(p.q8, t, p.status) : -1;
  }
  for (int l = blockIdx.z; l < p.L; l += gridDim.z) {
    if (TO8) {
      uint4 lo[kUnroll], hi[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        lo[u] = hi[u] = make_uint4(0, 0, 0, 0);
        if (pb[u] < 0 || pq[u] < 0) continue;
        const uint4* src = reinterpret_cast<const uint4*>(bf + row_off(p.bf, l, h, t0 + u * RPP + row, pb[u]));
        lo[u] = __ldcs(src);
        hi[u] = __ldcs(src + 1);
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        uint32_t b;
        const uint4 c = encode16<LPR>(lo[u], hi[u], b);   // every lane takes part in the shuffles
        if (pb[u] < 0 || pq[u] < 0) continue;
        const int t = t0 + u * RPP + row;
        __stcs(reinterpret_cast<uint4*>(q8 + row_off(p.q8, l, h, t, pq[u])), c);
        if (lane == 0) ex[exp_off(p.e, p.q8, l, h, t, pq[u])] = (uint8_t)b;
      }
    } else {
      uint4 c[kUnroll];
      uint32_t b[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        c[u] = make_uint4(0, 0, 0, 0);
        b[u] = 0;
        if (pb[u] < 0 || pq[u] < 0) continue;
        const int t = t0 + u * RPP + row;
        c[u] = __ldcs(reinterpret_cast<const uint4*>(q8 + row_off(p.q8, l, h, t, pq[u])));
        b[u] = ex[exp_off(p.e, p.q8, l, h, t, pq[u])];
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (pb[u] < 0 || pq[u] < 0) continue;
        uint4 lo, hi;
        decode16(c[u], b[u], lo, hi);
        uint4* dst = reinterpret_cast<uint4*>(bf + row_off(p.bf, l, h, t0 + u * RPP + row, pb[u]));
        __stcs(dst, lo);
        __stcs(dst + 1, hi);
      }
    }
  }
}

// grid: x = blocks of (token, head, K|V) rows of one request, y = requests (strided)
template <int D, bool TO8, int kUnroll>
__global__ void __launch_bounds__(kThreads) append_kernel(const __grid_constant__ AppendLaunch p) {
  constexpr int LPR = D / 16, RPP = kThreads / LPR;
  const int lane = threadIdx.x % LPR;
  for (int b = blockIdx.y; b < p.req.n; b += gridDim.y) {
    int q0, nq, kv;
    request_span(p.req, b, threadIdx.x == 0 && blockIdx.x == 0 ? p.status : nullptr, q0, nq, kv);
    const uint32_t items = (uint32_t)nq * (uint32_t)p.H * 2u;      // the host checked that this fits
    if (blockIdx.x * (uint32_t)(RPP * kUnroll) >= items) continue;
    uint4 lo[kUnroll], hi[kUnroll];
    int64_t at[kUnroll], eat[kUnroll];
    bool isv[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const uint32_t item = blockIdx.x * (uint32_t)(RPP * kUnroll) + u * RPP + threadIdx.x / LPR;
      const int j = (int)(item / (2u * p.H)), rest = (int)(item - (uint32_t)j * (2u * p.H));
      const int is_v = rest >= p.H, h = is_v ? rest - p.H : rest;
      const int pos = kv - nq + j;
      lo[u] = hi[u] = make_uint4(0, 0, 0, 0);
      at[u] = -1;
      isv[u] = is_v;
      if (item >= items) continue;
      if (pos < 0) {
        if (lane == 0) atomicOr(p.status, KVC_FLAG_BAD_LENGTH);
        continue;
      }
      const int page = is_paged(p.dst) ? request_page(p.req, p.dst, b, pos, p.status) : 0;
      if (page < 0) continue;
      at[u] = row_off(p.dst, p.layer, h, pos, page) + lane * 16;
      if (TO8) eat[u] = exp_off(p.e, p.dst, p.layer, h, pos, page);
      const DevHeads& src = is_v ? p.vn : p.kn;
      const uint4* x = reinterpret_cast<const uint4*>(src.p + (int64_t)(q0 + j) * src.s_row + (int64_t)h * src.s_head + lane * 16);
      lo[u] = x[0];
      hi[u] = x[1];
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (TO8) {
        uint32_t e;
        const uint4 c = encode16<LPR>(lo[u], hi[u], e);
        if (at[u] < 0) continue;
        *reinterpret_cast<uint4*>(reinterpret_cast<uint8_t*>(isv[u] ? p.dst.v : p.dst.k) + at[u]) = c;
        if (lane == 0) (isv[u] ? p.e.v : p.e.k)[eat[u]] = (uint8_t)e;
      } else if (at[u] >= 0) {
        uint4* dst = reinterpret_cast<uint4*>((isv[u] ? p.dst.v : p.dst.k) + at[u]);
        dst[0] = lo[u];
        dst[1] = hi[u];
      }
    }
  }
}

template <int D, bool TO8>
void convert(const ConvertLaunch& c, cudaStream_t s) {
  constexpr int U = TO8 ? 2 : 1, rows = kThreads / (D / 16) * U;
  const dim3 g((unsigned)((c.T + rows - 1) / rows), (unsigned)(2 * c.H), (unsigned)(c.L < 65535 ? c.L : 65535));
  convert_kernel<D, TO8, U><<<g, kThreads, 0, s>>>(c);
}

template <int D, bool TO8>
void append(const AppendLaunch& a, cudaStream_t s) {
  constexpr int U = 2, rows = kThreads / (D / 16) * U;
  const int64_t items = (int64_t)a.req.max_q * a.H * 2;
  const dim3 g((unsigned)((items + rows - 1) / rows), (unsigned)(a.req.n < 65535 ? a.req.n : 65535));
  append_kernel<D, TO8, U><<<g, kThreads, 0, s>>>(a);
}

}  // namespace

cudaError_t launch_convert(const ConvertLaunch& c, int d, cudaStream_t s) {
  if (d == 128)
    c.to8 ? convert<128, true>(c, s) : convert<128, false>(c, s);
  else
    c.to8 ? convert<64, true>(c, s) : convert<64, false>(c, s);
  return cudaGetLastError();
}

cudaError_t launch_append(const AppendLaunch& a, int d, cudaStream_t s) {
  const bool q8 = a.e.k != nullptr;
  if (d == 128)
    q8 ? append<128, true>(a, s) : append<128, false>(a, s);
  else
    q8 ? append<64, true>(a, s) : append<64, false>(a, s);
  return cudaGetLastError();
}

}  // namespace kvc
