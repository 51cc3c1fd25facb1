// Caches in 8 bits: kvc_quantize, kvc_dequantize (whole caches, every layer) and kvc_append, kvc_append_q8 (the new
// tokens of a step, one layer).
//
// A row is the d channels of one (token, layer, head), keys or values.  With amax its largest finite magnitude,
//     e = min { integer e >= -127 : amax <= 448 * 2^e } ,  code = rn_e4m3(x * 2^-e) ,  value = code * 2^e .
// Multiplying by a power of two is exact, so the only rounding is the one to e4m3 (to nearest even), and decoding is
// exact in bf16 (at e = 120, where 256 * 2^e would leave its range, magnitudes stop at 240 * 2^e).  All of it is bound by the bytes moved: 3 d + 1 a row to convert, 4 d or 3 d + 1 to append.
//
// Layout of the work: d / 8 neighbouring lanes hold one row (a 16-byte load of 8 bf16 values a lane, an 8-byte store of
// 8 codes), the row's maximum is a butterfly over those lanes.
#include <cuda_runtime.h>

#include "kvc_attend.h"
#include "kvc_launch.h"

namespace kvc {
namespace {

// 8 values of a row -> 8 codes and the row's exponent (the same in all LPR lanes of the row)
template <int LPR>
__device__ __forceinline__ uint2 encode8(const uint4& raw, uint32_t& b) {
  float x[8];
  unpack8(raw, x);
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = fabsf(x[i]);
    if (a < __uint_as_float(0x7f800000u))
      m = fmaxf(m, a);
    else
      x[i] = __uint_as_float(0x7fc00000u);   // infinities too: e4m3 has none, and 448 would be a plausible number
  }
#pragma unroll
  for (int o = LPR / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  b = row_exponent(m);
  const float s = exponent_down(b);
  if (b == 247u) {                           // the next code, 256 * 2^120 = 2^128, is no finite bf16
    const float top = 240.f * exponent_up(b);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (fabsf(x[i]) > top) x[i] = copysignf(top, x[i]);
  }
  uint2 c;
  c.x = e4m3x2(x[0] * s, x[1] * s) | (e4m3x2(x[2] * s, x[3] * s) << 16);
  c.y = e4m3x2(x[4] * s, x[5] * s) | (e4m3x2(x[6] * s, x[7] * s) << 16);
  return c;
}

__device__ __forceinline__ uint4 decode8(const uint2& c, uint32_t b) {
  const float s = exponent_up(b);
  float x[8];
  const uint32_t w[4] = {c.x & 0xffffu, c.x >> 16, c.y & 0xffffu, c.y >> 16};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = e4m3x2_to_float2(w[i]);
    x[2 * i] = f.x * s;
    x[2 * i + 1] = f.y * s;
  }
  return pack8(x);
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
constexpr int kUnroll = 4;

// grid: x = token blocks, y = head x (K|V), z = layers (strided)
template <int D, bool TO8>
__global__ void __launch_bounds__(kThreads) convert_kernel(const __grid_constant__ ConvertLaunch p) {
  constexpr int LPR = D / 8, RPP = kThreads / LPR;
  const int lane = threadIdx.x % LPR, row = threadIdx.x / LPR;
  const int h = blockIdx.y >> 1, is_v = blockIdx.y & 1;
  const int t0 = blockIdx.x * (RPP * kUnroll);
  __nv_bfloat16* bf = is_v ? p.bf.v : p.bf.k;
  uint8_t* q8 = reinterpret_cast<uint8_t*>(is_v ? p.q8.v : p.q8.k);
  uint8_t* ex = is_v ? p.e.v : p.e.k;
  for (int l = blockIdx.z; l < p.L; l += gridDim.z) {
    int64_t ob[kUnroll], oq[kUnroll], oe[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int t = t0 + u * RPP + row;
      ob[u] = oq[u] = oe[u] = -1;
      if (t < p.T) {
        const int pb = own_page(p.bf, t, p.status), pq = own_page(p.q8, t, p.status);
        if (pb >= 0 && pq >= 0) {
          ob[u] = row_off(p.bf, l, h, t, pb) + lane * 8;
          oq[u] = row_off(p.q8, l, h, t, pq) + lane * 8;
          oe[u] = exp_off(p.e, p.q8, l, h, t, pq);
        }
      }
    }
    if (TO8) {
      uint4 raw[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) raw[u] = ob[u] >= 0 ? __ldcs(reinterpret_cast<const uint4*>(bf + ob[u])) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        uint32_t b;
        const uint2 c = encode8<LPR>(raw[u], b);   // every lane takes part in the shuffles
        if (ob[u] >= 0) {
          *reinterpret_cast<uint2*>(q8 + oq[u]) = c;
          if (lane == 0) ex[oe[u]] = (uint8_t)b;
        }
      }
    } else {
      uint2 c[kUnroll];
      uint32_t b[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        c[u] = ob[u] >= 0 ? __ldcs(reinterpret_cast<const uint2*>(q8 + oq[u])) : make_uint2(0, 0);
        b[u] = ob[u] >= 0 ? ex[oe[u]] : 0;
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        if (ob[u] >= 0) *reinterpret_cast<uint4*>(bf + ob[u]) = decode8(c[u], b[u]);
    }
  }
}

// grid: x = blocks of (token, head, K|V) rows of one request, y = requests (strided)
template <int D, bool TO8>
__global__ void __launch_bounds__(kThreads) append_kernel(const __grid_constant__ AppendLaunch p) {
  constexpr int LPR = D / 8, RPP = kThreads / LPR;
  const int lane = threadIdx.x % LPR;
  const int64_t item = (int64_t)blockIdx.x * RPP + threadIdx.x / LPR;
  for (int b = blockIdx.y; b < p.req.n; b += gridDim.y) {
    int q0, nq, kv;
    request_span(p.req, b, threadIdx.x == 0 && blockIdx.x == 0 ? p.status : nullptr, q0, nq, kv);
    const int j = (int)(item / (2 * p.H)), rest = (int)(item % (2 * p.H));
    const int is_v = rest & 1, h = rest >> 1;
    const int pos = kv - nq + j;
    bool live = j < nq;
    if (live && pos < 0) {
      if (lane == 0) atomicOr(p.status, KVC_FLAG_BAD_LENGTH);
      live = false;
    }
    int page = 0;
    if (live && is_paged(p.dst)) {
      page = request_page(p.req, p.dst, b, pos, p.status);
      live = page >= 0;
    }
    uint4 raw = make_uint4(0, 0, 0, 0);
    if (live) {
      const DevHeads& src = is_v ? p.vn : p.kn;
      raw = *reinterpret_cast<const uint4*>(src.p + (int64_t)(q0 + j) * src.s_row + (int64_t)h * src.s_head + lane * 8);
    }
    if (TO8) {
      uint32_t e;
      const uint2 c = encode8<LPR>(raw, e);
      if (live) {
        uint8_t* q8 = reinterpret_cast<uint8_t*>(is_v ? p.dst.v : p.dst.k);
        *reinterpret_cast<uint2*>(q8 + row_off(p.dst, p.layer, h, pos, page) + lane * 8) = c;
        if (lane == 0) (is_v ? p.e.v : p.e.k)[exp_off(p.e, p.dst, p.layer, h, pos, page)] = (uint8_t)e;
      }
    } else if (live) {
      *reinterpret_cast<uint4*>((is_v ? p.dst.v : p.dst.k) + row_off(p.dst, p.layer, h, pos, page) + lane * 8) = raw;
    }
  }
}

}  // namespace

cudaError_t launch_convert(const ConvertLaunch& c, int d, cudaStream_t s) {
  const int rows = kThreads / (d / 8) * kUnroll;
  const dim3 g((unsigned)((c.T + rows - 1) / rows), (unsigned)(2 * c.H), (unsigned)(c.L < 65535 ? c.L : 65535));
  if (d == 128)
    c.to8 ? convert_kernel<128, true><<<g, kThreads, 0, s>>>(c) : convert_kernel<128, false><<<g, kThreads, 0, s>>>(c);
  else
    c.to8 ? convert_kernel<64, true><<<g, kThreads, 0, s>>>(c) : convert_kernel<64, false><<<g, kThreads, 0, s>>>(c);
  return cudaGetLastError();
}

cudaError_t launch_append(const AppendLaunch& a, int d, cudaStream_t s) {
  const int64_t items = (int64_t)a.req.max_q * a.H * 2, rows = kThreads / (d / 8);
  const dim3 g((unsigned)((items + rows - 1) / rows), (unsigned)(a.req.n < 65535 ? a.req.n : 65535));
  const bool q8 = a.e.k != nullptr;
  if (d == 128)
    q8 ? append_kernel<128, true><<<g, kThreads, 0, s>>>(a) : append_kernel<128, false><<<g, kThreads, 0, s>>>(a);
  else
    q8 ? append_kernel<64, true><<<g, kThreads, 0, s>>>(a) : append_kernel<64, false><<<g, kThreads, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace kvc
