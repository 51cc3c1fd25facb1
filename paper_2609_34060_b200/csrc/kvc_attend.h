// Requests, packed rows and 8-bit caches as the kernels of kvc_append, kvc_attend, kvc_quantize and kvc_dequantize see
// them, and the launch interface between their translation units.
#pragma once
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/kvc.h"
#include "kvc_dev.cuh"

namespace kvc {

struct DevRequests {
  const int32_t* q_begin;
  const int32_t* kv_len;
  const int32_t* table;        // nullptr: every request uses the cache's own table (or contiguous rows)
  int64_t table_stride;
  int32_t n, max_q, max_kv, n_rows;
};

struct DevHeads {
  __nv_bfloat16* p;
  int64_t s_row, s_head;
};

// exponent bytes of an 8-bit cache; k == nullptr: the cache is bf16
struct DevScale {
  uint8_t* k;
  uint8_t* v;
  int64_t s_layer, s_page, s_head, s_tok;
};

struct AppendLaunch {
  DevRequests req;
  DevHeads kn, vn;
  DevCache dst;
  DevScale e;
  int32_t H, layer;
  uint32_t* status;
};

struct ConvertLaunch {         // quantize (to8) or dequantize
  DevCache bf, q8;
  DevScale e;
  int32_t L, H, T, to8;
  uint32_t* status;
};

struct AttendLaunch {
  DevRequests req;
  DevHeads q, out;
  float* lse;
  DevCache c;                  // bf16, or codes when e.k is set
  DevScale e;
  int32_t H, G, layer, causal; // G query heads per KV head
  float scale;
  uint32_t* status;
  float* part;                 // workspace
  const uint32_t* mask;        // trees of drafted tokens: [n_rows, words], else nullptr (causal is set with it)
  int32_t words;
};

// Request b's packed rows and cache length; false (and the flag) when its numbers break the bounds the launch was sized by.
__device__ __forceinline__ bool request_span(const DevRequests& r, int b, uint32_t* status, int& q0, int& nq, int& kv) {
  const int a = r.q_begin[b], e = r.q_begin[b + 1];
  kv = r.kv_len[b];
  q0 = a;
  nq = e - a;
  const bool ok = a >= 0 && e >= a && e <= r.n_rows && nq <= r.max_q && kv >= 0 && kv <= r.max_kv;
  if (!ok) {
    if (status) atomicOr(status, KVC_FLAG_BAD_LENGTH);
    nq = 0;
    kv = 0;
  }
  return ok;
}

// Physical page of request b's token t (paged caches), -1 and the flag when the table names none.
__device__ __forceinline__ int request_page(const DevRequests& r, const DevCache& c, int b, int t, uint32_t* status) {
  const int32_t* tab = r.table ? r.table + (int64_t)b * r.table_stride : c.page_table;
  const int p = tab[t >> c.page_shift];
  if ((unsigned)p < (unsigned)c.n_phys) return p;
  if (status) atomicOr(status, KVC_FLAG_BAD_PAGE);
  return -1;
}
// whether a cache is paged (the table itself may come from the requests)
__host__ __device__ __forceinline__ bool is_paged(const DevCache& c) { return c.n_phys > 0; }

// element offset of row (l, h, t)
__device__ __forceinline__ int64_t row_off(const DevCache& c, int l, int h, int t, int page) {
  const int64_t o = (int64_t)l * c.s_layer + (int64_t)h * c.s_head;
  return is_paged(c) ? o + (int64_t)page * c.s_page + (int64_t)(t & c.page_mask) * c.s_tok : o + (int64_t)t * c.s_tok;
}
__device__ __forceinline__ int64_t exp_off(const DevScale& e, const DevCache& c, int l, int h, int t, int page) {
  const int64_t o = (int64_t)l * e.s_layer + (int64_t)h * e.s_head;
  return is_paged(c) ? o + (int64_t)page * e.s_page + (int64_t)(t & c.page_mask) * e.s_tok : o + (int64_t)t * e.s_tok;
}

// 32 bits of a row's mask over the request's new tokens, from new token `rel` on; tokens of the context (rel < 0) are seen.
// `row`: the row's words, nullptr: nothing seen.
__device__ __forceinline__ uint32_t seen_word(const uint32_t* row, int words, int i) {
  return row == nullptr ? 0u : i < 0 ? 0xffffffffu : i < words ? __ldg(row + i) : 0u;
}

// ---- e4m3 rows under a power-of-two scale
// Exponent byte of a row from its largest finite magnitude: the smallest b with amax <= 448 * 2^(b - 127), at least 0.
// amax = 1.f * 2^(E-127), 448 = 1.75 * 2^8: b = E - 8, one more when 1.f > 1.75.
__device__ __forceinline__ uint32_t row_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int b = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)(b < 0 ? 0 : b);
}
__device__ __forceinline__ float exponent_down(uint32_t b) { return __uint_as_float((254u - b) << 23); }   // 2^(127 - b)
__device__ __forceinline__ float exponent_up(uint32_t b) {                                                  // 2^(b - 127)
  return b == 0 ? __uint_as_float(0x00400000u) : b == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float(b << 23);
}
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float2 e4m3x2_to_float2(uint32_t two) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// argument resolution shared by the C entry points (kvc_api.cu)
int resolve_cache(const kvc_cache* c, DevCache* out);
int path_force();
void set_last_path(int path);

cudaError_t launch_append(const AppendLaunch& a, int d, cudaStream_t s);
cudaError_t launch_convert(const ConvertLaunch& c, int d, cudaStream_t s);
cudaError_t launch_attend_generic(const AttendLaunch& a, int d, cudaStream_t s);

}  // namespace kvc
