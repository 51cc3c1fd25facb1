// Trees of drafted tokens: kvc_tree_build (masks and depths from parents) and kvc_keep (accepted rows moved together).
#include <cuda_runtime.h>

#include "kvc_draft.h"
#include "kvc_launch.h"
#include "kvc_tc_attend.cuh"

namespace kvc {
namespace {

using tc::grid_dependency_wait;
using tc::grid_dependents_launch;
using tc::launch_after;

// A block a request, a thread a row: the row's ancestors one after the other, parents in shared memory.  A parent comes
// before its child, so a walk ends after at most max_q steps and meets the words of the mask from the last to the first:
// each is written once, complete.  Bound: launch and the chain lengths -> parents -> walk (a tree of 24 drafts 1.8 us, 192 of
// 40-200 drafts 4.5 us).
__global__ void __launch_bounds__(256) tree_build_kernel(const __grid_constant__ TreeLaunch p) {
  __shared__ int16_t parent[KVC_TREE_MAX_Q];
  grid_dependency_wait();
  grid_dependents_launch();
  int q0, nq, kv;
  request_span(p.req, (int)blockIdx.x, threadIdx.x == 0 ? p.status : nullptr, q0, nq, kv);
  for (int j = threadIdx.x; j < nq; j += blockDim.x) {
    int a = p.parent[q0 + j];
    if (a < -1 || a >= j) {
      atomicOr(p.status, KVC_FLAG_BAD_TREE);
      a = -1;
    }
    parent[j] = (int16_t)a;
  }
  __syncthreads();
  for (int j = threadIdx.x; j < nq; j += blockDim.x) {
    uint32_t* out = p.mask + (int64_t)(q0 + j) * p.words;
    int w = p.words - 1, depth = -1;
    uint32_t bits = 0;
    for (int a = j; a >= 0; a = parent[a]) {
      for (; w > a >> 5; --w) {
        out[w] = bits;
        bits = 0;
      }
      bits |= 1u << (a & 31);
      ++depth;
    }
    for (; w >= 0; --w) {
      out[w] = bits;
      bits = 0;
    }
    p.depth[q0 + j] = depth;
  }
}

constexpr int kKeepThreads = 128, kRowsAtOnce = 32, kInFlight = 4;

// A thread owns 16 bytes of a row in one (layer, head, K|V) and moves them for the request's accepted rows in their order,
// kInFlight loads and then as many stores.  Places are ascending, so a row's new place is never one that a later row is
// still to be read from, and nobody else touches these bytes.  Bound: bytes for many requests, for one the chain of
// dependent reads (lengths, page ids, rows).  Measured, 32 layers, 8 heads of 128: 64 requests in 8 bits, 38 MB moved, 7.8 us
// from L2, 11.6 from HBM (eight rows in flight 12.3: registers; 256 threads a block 9); one request 2.6 us.
// grid: x = (layer, K|V, head, 16-byte chunk), y = requests (strided)
template <int D, bool Q8>
__global__ void __launch_bounds__(kKeepThreads) keep_kernel(const __grid_constant__ KeepLaunch p) {
  constexpr int CH = D * (Q8 ? 1 : 2) / 16;
  __shared__ int64_t s_src[kRowsAtOnce], s_dst[kRowsAtOnce], s_esrc[kRowsAtOnce], s_edst[kRowsAtOnce];   // of the rows that move
  __shared__ int s_n;
  grid_dependency_wait();
  grid_dependents_launch();
  const int tid = threadIdx.x;
  const uint32_t item = blockIdx.x * (uint32_t)kKeepThreads + tid, items = (uint32_t)p.L * p.H * 2 * CH;
  const int chunk = item % CH;
  uint32_t rest = item / CH;
  const int h = rest % p.H;
  rest /= p.H;
  const int is_v = rest & 1, l = (int)(rest >> 1);
  const bool live = item < items, exponent = Q8 && chunk == 0;
  uint8_t* rows = reinterpret_cast<uint8_t*>(is_v ? p.c.v : p.c.k) + ((int64_t)l * p.c.s_layer + (int64_t)h * p.c.s_head) * (Q8 ? 1 : 2) + chunk * 16;
  uint8_t* exps = (is_v ? p.e.v : p.e.k) + ((int64_t)l * p.e.s_layer + (int64_t)h * p.e.s_head);
  for (int b = blockIdx.y; b < p.req.n; b += gridDim.y) {
    const int32_t* kept = p.kept + (int64_t)b * p.stride;
    const bool first_block = blockIdx.x == 0 && tid == 0;
    const int nk = p.n_kept[b];
    // the first places and the ones before them, asked for before the lengths are there
    const int place = tid < p.req.max_q ? kept[tid] : 0, place_before = tid > 0 && tid < p.req.max_q ? kept[tid - 1] : -1;
    int q0, nq, kv;
    const bool valid = request_span(p.req, b, first_block ? p.status : nullptr, q0, nq, kv);
    const int first = kv - nq;
    bool bad = nk < 0 || nk > nq || first < 0;                   // kv_out would be negative, whatever is kept
    if (!bad) {
      for (int j = tid; j < nk; j += kKeepThreads) {
        const int a = j == tid ? place : kept[j];
        bad |= a >= nq || a <= (j == tid ? place_before : kept[j - 1]);
      }
    }
    bad = __syncthreads_or(bad);
    if (first_block && valid) {
      if (bad) atomicOr(p.status, KVC_FLAG_BAD_TREE);
      if (p.kv_out) p.kv_out[b] = bad ? kv : first + nk;
    }
    if (bad || !valid) continue;
    for (int j0 = 0; j0 < nk; j0 += kRowsAtOnce) {
      if (j0 > 0) __syncthreads();
      if (tid < kRowsAtOnce) {                                   // one warp
        const int j = j0 + tid, a = j >= nk ? j : j0 == 0 ? place : kept[j];
        int ps = -1, pd = -1;
        if (a != j) {
          ps = is_paged(p.c) ? request_page(p.req, p.c, b, first + a, p.status) : 0;
          pd = is_paged(p.c) ? request_page(p.req, p.c, b, first + j, p.status) : 0;
        }
        const bool moves = ps >= 0 && pd >= 0;
        const unsigned all = __ballot_sync(0xffffffffu, moves);
        if (moves) {
          const int at = __popc(all & ((1u << tid) - 1u));
          s_src[at] = row_off(p.c, 0, 0, first + a, ps);
          s_dst[at] = row_off(p.c, 0, 0, first + j, pd);
          if (Q8) {
            s_esrc[at] = exp_off(p.e, p.c, 0, 0, first + a, ps);
            s_edst[at] = exp_off(p.e, p.c, 0, 0, first + j, pd);
          }
        }
        if (tid == 0) s_n = __popc(all);
      }
      __syncthreads();
      const int n = s_n;
      if (live) {
        for (int k0 = 0; k0 < n; k0 += kInFlight) {
          uint4 x[kInFlight];
          uint8_t e[kInFlight];
#pragma unroll
          for (int k = 0; k < kInFlight; ++k) {
            if (k0 + k >= n) continue;
            x[k] = *reinterpret_cast<const uint4*>(rows + s_src[k0 + k] * (Q8 ? 1 : 2));
            if (exponent) e[k] = exps[s_esrc[k0 + k]];
          }
#pragma unroll
          for (int k = 0; k < kInFlight; ++k) {
            if (k0 + k >= n) continue;
            *reinterpret_cast<uint4*>(rows + s_dst[k0 + k] * (Q8 ? 1 : 2)) = x[k];
            if (exponent) exps[s_edst[k0 + k]] = e[k];
          }
        }
      }
    }
    __syncthreads();                                             // before the next request's places
  }
}

}  // namespace

cudaError_t launch_tree_build(const TreeLaunch& t, cudaStream_t s) {
  const int rows = t.req.max_q < 256 ? (t.req.max_q + 31) / 32 * 32 : 256;
  return launch_after(tree_build_kernel, dim3((unsigned)t.req.n), rows, 0, s, t);
}

cudaError_t launch_keep(const KeepLaunch& k, int d, cudaStream_t s) {
  const bool q8 = k.e.k != nullptr;
  const int64_t items = (int64_t)k.L * k.H * 2 * (d * (q8 ? 1 : 2) / 16);
  const dim3 g((unsigned)((items + kKeepThreads - 1) / kKeepThreads), (unsigned)(k.req.n < 65535 ? k.req.n : 65535));
#define KVC_KEEP(D, Q) \
  if (d == D && q8 == Q) return launch_after(keep_kernel<D, Q>, g, kKeepThreads, 0, s, k);
  KVC_KEEP(128, false) KVC_KEEP(128, true) KVC_KEEP(64, false) KVC_KEEP(64, true)
#undef KVC_KEEP
  return cudaErrorInvalidValue;
}

}  // namespace kvc
