// kvc_verify: which drafted tokens stay, and the next token, by rejection sampling from given random numbers.
//
// With P the distribution at the current node (the target's at first) and q the one its children were drawn from, child c
// with token x stays where u q(x) < P(x); otherwise P <- max(P - q, 0) / Z.  After any number of rejections
//     P = max(A p - B q, 0) ,   A = B = 1 and divided by Z, B one more at each ( max(max(a, 0) / Z - q, 0) = max(a / Z - q, 0) ) ,
// so nothing of a distribution is stored: a sum or a draw is one pass over p and q.  A rejection alone needs no pass; a
// further sibling needs Z, and the draw at the end one pass more for the sum (its last part is read twice, from L2).
//
// Bound: the bytes of the distributions that are passed over (V values each), and for few requests the chain lists -> gathers
// -> pass -> draw.  The gathers of all rows, p and q at their tokens, are made at once before the walk.
//
// A cluster of blocks shares a request.  Every block walks the tree by itself (all of them come to the same decisions from
// the same numbers), sums its part of the vocabulary, and the parts' sums meet in distributed shared memory.  Blocks, warps
// and lanes hold ascending parts, so the draw finds its place from prefix sums: block, warp, then a run of entries a thread
// over the warp's part.
// Sums are float64, in a fixed order.
//
// Measured on the device, inputs that change from call to call: 64 trees of 8-16 drafts over 128000 entries, up to five passes
// a request, 40 us (66 MB from HBM, a fifth of its rate: the longest chain of passes bounds it, and a pass the latency of the
// few loads that 64 registers let fly); nothing rejected, or one draft, 17-18 us; one chain of five drafts over 32000 entries 6 us:
// launch, lists, gathers, two cluster barriers, draw.  Those trees' distributions have their small entries cut off, and the
// lists of what is left (kList) hold it: 43 us without lists.  Distributions that keep their tails overflow them, which costs
// more than it gives: 49 us, 45 without lists (of flatter ones 51 and 46; 4 and 16 trees 13 / 18 us cut, 16 / 23 whole, by
// no lists 15 / 20 and 15 / 22).
// Chosen drafts: every entry is compared with every sibling rejected at the node, so a wide node costs vocabulary times
// siblings: 64 requests with 10 rejected 63 us, 16 with 64 209 us, one with 300 1.3 ms, one with 1000 9.7 ms.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include "kvc_draft.h"
#include "kvc_launch.h"
#include "kvc_tc_attend.cuh"

namespace kvc {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 256, kWarps = kThreads / 32, kMaxCluster = 16;
constexpr int kRowBytes = 24;              // of shared memory for a row of the request
constexpr int kStep = 128;                 // entries a warp takes at a time
constexpr int kList = 512;                 // entries of a warp's part that are kept from one pass over a node to the next

// A float below kTooLarge, not negative, as a double, by moving its bits: the conversion unit takes 16 a cycle and SM, four
// times fewer than the integer pipe (64 trees over 128000 entries 47 us with it for subnormal numbers alone).  2^24 first, so
// that subnormal numbers are normal ones.  (0 comes out as 2^-151: the callers look at that before.)
constexpr float kTooLarge = 0x1p104f;
__device__ __forceinline__ double widen(float x) {
  const uint32_t u = __float_as_uint(x * 0x1p24f);
  return __hiloint2double((int)((u >> 3) + 0x36800000u), (int)(u << 29));
}
// P(x) from the node's two distributions; NaN and negative entries count as 0
__device__ __forceinline__ double residual(float p, float q, double A, double B) {
  const double v = widen(p) * A - (q > 0.f ? widen(q) : 0.0) * B;
  return p > 0.f && v > 0.0 ? v : 0.0;
}

struct Node {                              // where the walk is
  int node, asked, gone;                   // the node's row, the row tried last, rejected tokens (drafts chosen)
  bool listed;                             // the node's entries with P > 0 are in shared memory
  bool spent;                              // no residual left: no further child, the draw is from p itself
  bool normal;                             // A and B hold the last rejection's division
  double A, B, left;
};

template <bool kDraft, bool kWide>
__global__ void __launch_bounds__(kThreads, 4) verify_kernel(const __grid_constant__ VerifyLaunch p) {
  extern __shared__ float s_p[];           // [max_q] each: p and q of the drafted tokens, u, tokens, rejected tokens, parents, path
  float* s_q = s_p + p.req.max_q;
  float* s_u = s_q + p.req.max_q;
  int* s_token = reinterpret_cast<int*>(s_u + p.req.max_q);
  int* s_gone = s_token + p.req.max_q;
  int16_t* s_parent = reinterpret_cast<int16_t*>(s_gone + p.req.max_q);
  int16_t* s_path = s_parent + p.req.max_q;
  // entries (p, q) with P > 0 of every warp's part, where they fit: P > 0 never comes back, so the passes behind a node's
  // first rejection go over these alone
  float2* s_list = reinterpret_cast<float2*>(s_p + (p.req.max_q * kRowBytes / 4 + 3) / 4 * 4) + (threadIdx.x >> 5) * kList;
  __shared__ int s_count[kWarps];          // of them; -1: too many
  __shared__ double s_warp[kWarps], s_block[2][kMaxCluster];
  __shared__ Node s_at;
  __shared__ int s_more, s_kept;
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), blocks = (int)cluster.num_blocks();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int b = (int)(blockIdx.x / blocks);
  tc::grid_dependency_wait();
  tc::grid_dependents_launch();
  const float u_next = p.u_next[b];
  int q0, nq, kv;
  request_span(p.req, b, tid == 0 && rank == 0 ? p.status : nullptr, q0, nq, kv);
  if (nq == 0) {
    if (rank == 0) {
      for (int j = tid; j < p.req.max_q; j += kThreads) p.kept[(int64_t)b * p.stride + j] = -1;
      if (tid == 0) {
        p.n_kept[b] = 0;
        p.next[b] = -1;
      }
    }
    return;                                // the same for the whole cluster
  }
  // what the walk may ask for
  for (int j = tid; j < nq; j += kThreads) {
    int a = j == 0 ? -1 : p.parent[q0 + j];
    const int x = j == 0 ? 0 : p.token[q0 + j];
    s_u[j] = j == 0 ? 0.f : p.u[q0 + j];
    const bool known = (unsigned)x < (unsigned)p.vocab;
    if (a < -1 || a >= j || !known) {
      if (rank == 0) atomicOr(p.status, KVC_FLAG_BAD_TREE);
      a = -1;
    }
    s_parent[j] = (int16_t)a;
    s_token[j] = x;
    s_p[j] = a >= 0 ? p.target[(int64_t)(q0 + a) * p.s_target + x] : 0.f;
    if (kDraft) s_q[j] = a >= 0 ? p.draft[(int64_t)(q0 + a) * p.s_draft + x] : 0.f;
  }
  if (tid == 0) {
    s_at = Node{0, 0, 0, false, false, true, 1.0, 0.0, 1.0};
    s_path[0] = 0;
    s_kept = 1;
  }
  cluster.sync();                          // every block of the cluster runs: its shared memory may be written

  // the vocabulary: blocks, warps, steps of 128 entries
  const int64_t per_block = (((int64_t)p.vocab + blocks - 1) / blocks + kStep - 1) / kStep * kStep;
  const int64_t lo_block = per_block * rank, hi_block = min((int64_t)p.vocab, lo_block + per_block);
  const int per_warp = (int)((per_block + kWarps * kStep - 1) / (kWarps * kStep) * kStep);
  auto warp_range = [&](int w, int64_t& lo, int64_t& hi) {
    lo = lo_block + (int64_t)w * per_warp;
    hi = min(hi_block, lo + per_warp);
  };
  // four entries of P from `at` on (at a multiple of 4; behind hi: 0)
  struct Four {
    float p[4], q[4];
  };
  auto fetch = [&](const float* pt, const float* pd, int64_t at, int64_t hi, Four& x) {   // pd == nullptr: P is p's
    x.q[0] = x.q[1] = x.q[2] = x.q[3] = 0.f;
    if (kWide && at + 4 <= hi) {
      const float4 v = __ldg(reinterpret_cast<const float4*>(pt + at));
      x.p[0] = v.x, x.p[1] = v.y, x.p[2] = v.z, x.p[3] = v.w;
      if (kDraft && pd) {
        const float4 w = __ldg(reinterpret_cast<const float4*>(pd + at));
        x.q[0] = w.x, x.q[1] = w.y, x.q[2] = w.z, x.q[3] = w.w;
      }
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x.p[k] = at + k < hi ? __ldg(pt + at + k) : 0.f;
        if (kDraft && pd) x.q[k] = at + k < hi ? __ldg(pd + at + k) : 0.f;
      }
    }
  };
  auto value = [&](const Four& x, int k, int64_t at, double A, double B, int gone) {
    if (!kDraft) {
      for (int g = 0; g < gone; ++g)
        if (s_gone[g] == at + k) return 0.0;
    }
    if (!kDraft) return x.p[k] > 0.f ? widen(x.p[k]) : 0.0;
    return residual(x.p[k], x.q[k], A, B);
  };
  int passes = 0;
  // sum of P over the vocabulary, the same in all threads of the cluster; list: fill the lists, or go over them (listed)
  auto sum_all = [&](int node, double A, double B, int gone, bool list, bool listed) {
    const float* pt = p.target + (int64_t)(q0 + node) * p.s_target;
    const float* pd = kDraft && B != 0.0 ? p.draft + (int64_t)(q0 + node) * p.s_draft : nullptr;
    int64_t lo, hi;
    warp_range(warp, lo, hi);
    double sum = 0.0;
    float top = 0.f;
    if (kDraft && listed && s_count[warp] >= 0) {
      const int n = s_count[warp];
      for (int i = lane; i < n; i += 32) sum += residual(s_list[i].x, s_list[i].y, A, B);
    } else if (kDraft && list) {
      int n = 0;
      for (int64_t base = lo; base < hi; base += 2 * kStep) {
        Four x[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) fetch(pt, pd, base + i * kStep + lane * 4, hi, x[i]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const double v = residual(x[i].p[k], x[i].q[k], A, B);
            sum += v;
            top = fmaxf(top, x[i].p[k]);
            const unsigned some = __ballot_sync(0xffffffffu, v > 0.0);
            const int at = n + __popc(some & ((1u << lane) - 1u));
            if (v > 0.0 && at < kList) s_list[at] = make_float2(x[i].p[k], x[i].q[k]);
            n += __popc(some);
          }
        }
      }
      if (lane == 0) s_count[warp] = n <= kList ? n : -1;
      __syncwarp();
    } else {
      constexpr int kAhead = kDraft ? 2 : 4;   // loads in flight (two rows, or one)
      for (int64_t at = lo + lane * 4; at < hi; at += kAhead * kStep) {
        Four x[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) fetch(pt, pd, at + i * kStep, hi, x[i]);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          double s = 0.0;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            s += value(x[i], k, at + i * kStep, A, B, gone);
            top = fmaxf(top, x[i].p[k]);
          }
          sum += s;
        }
      }
    }
    if (top >= kTooLarge) sum = __longlong_as_double(0x7ff0000000000000ll);   // no sum with an infinity in it
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    __syncthreads();                       // s_warp of the pass before has been read
    if (lane == 0) s_warp[warp] = sum;
    __syncthreads();
    double* mine = s_block[passes & 1];
    ++passes;
    if (tid < blocks) {
      double all = 0.0;
      for (int w = 0; w < kWarps; ++w) all += s_warp[w];
      *cluster.map_shared_rank(mine + rank, tid) = all;
    }
    cluster.sync();                        // the parts lie in two buffers in turn: nobody writes one that is still read
    double total = 0.0;
    for (int c = 0; c < blocks; ++c) total += mine[c];
    return total;
  };

  for (;;) {
    if (warp == 0) {
      Node n = s_at;
      int kept = s_kept;
      bool more = false;                   // a sibling waits for the sum
      for (int c0 = n.asked + 1; c0 < nq && !n.spent;) {
        const int c = c0 + lane;
        const unsigned hit = __ballot_sync(0xffffffffu, c < nq && s_parent[c] == n.node);
        if (!hit) {
          c0 += 32;
          continue;
        }
        const int child = c0 + __ffs(hit) - 1;
        if (!n.normal) {
          more = true;
          break;
        }
        n.asked = child;
        c0 = child + 1;
        bool yes;
        bool fresh = true;
        const double px = (double)s_p[child];
        if (kDraft) {
          const double qx = (double)fmaxf(s_q[child], 0.f);       // u q is not below a P of 0, nor below one that is negative
          yes = (double)s_u[child] * qx < px * n.A - qx * n.B;
        } else {
          for (int g = 0; g < n.gone; ++g) fresh = fresh && s_gone[g] != s_token[child];
          yes = fresh && (double)s_u[child] * n.left < px;
        }
        if (yes) {
          if (lane == 0) s_path[kept] = (int16_t)child;
          ++kept;
          n.node = child;
          n.A = 1.0;
          n.B = 0.0;
          n.left = 1.0;
          n.gone = 0;
          n.listed = false;
        } else if (kDraft) {
          n.B += 1.0;
          n.normal = false;
        } else if (fresh) {
          n.left -= fmax(px, 0.0);
          __syncwarp();
          if (lane == 0) s_gone[n.gone] = s_token[child];
          __syncwarp();
          ++n.gone;
        }
      }
      if (lane == 0) {
        s_at = n;
        s_kept = kept;
        s_more = more;
      }
    }
    __syncthreads();
    if (!s_more) break;
    const Node n = s_at;
    const double z = sum_all(n.node, n.A, n.B, n.gone, !n.listed, n.listed);
    __syncthreads();
    if (tid == 0) {
      const bool some = z > 0.0 && z < __longlong_as_double(0x7ff0000000000000ll);
      s_at.spent = !some;
      s_at.listed = true;
      s_at.normal = true;
      s_at.A = some ? n.A / z : 1.0;
      s_at.B = some ? n.B / z : 0.0;
    }
    __syncthreads();
  }

  Node n = s_at;
  const double infinite = __longlong_as_double(0x7ff0000000000000ll);
  double total = sum_all(n.node, n.A, n.B, n.gone, false, n.listed && n.B != 0.0);
  if (!(total > 0.0 && total < infinite) && (n.B != 0.0 || n.gone > 0)) {
    n.A = 1.0;
    n.B = 0.0;
    n.gone = 0;
    total = sum_all(n.node, n.A, n.B, n.gone, false, false);
  }
  if (rank == 0) {
    const int kept = s_kept;
    for (int j = tid; j < p.req.max_q; j += kThreads) p.kept[(int64_t)b * p.stride + j] = j < kept ? s_path[j] : -1;
    if (tid == 0) p.n_kept[b] = kept;
  }
  if (!(total > 0.0 && total < infinite)) {
    if (rank == 0 && tid == 0) {
      p.next[b] = -1;
      atomicOr(p.status, KVC_FLAG_BAD_PROB);
    }
    return;
  }
  // the draw: the first part whose end lies beyond the threshold; where rounding leaves none, the last that has anything
  const double threshold = (double)u_next * total;
  auto find = [&](const double* parts, int count, double& before) {
    double run = before;
    int last = -1;
    double at_last = before;
    for (int i = 0; i < count; ++i) {
      if (parts[i] > 0.0) {
        last = i;
        at_last = run;
      }
      run += parts[i];
      if (run > threshold && last == i) break;
    }
    before = at_last;
    return last;
  };
  double before = 0.0;
  const int block = find(s_block[(passes - 1) & 1], blocks, before);
  if (block != rank) return;
  // the warp's part once more, by the whole block: a thread a run of entries, one scan over the threads
  const int part = find(s_warp, kWarps, before);
  const float* pt = p.target + (int64_t)(q0 + n.node) * p.s_target;
  const float* pd = kDraft && n.B != 0.0 ? p.draft + (int64_t)(q0 + n.node) * p.s_draft : nullptr;
  int64_t lo, hi;
  warp_range(part, lo, hi);
  const int run = (per_warp + 4 * kThreads - 1) / (4 * kThreads) * 4;
  const int64_t begin = lo + (int64_t)tid * run, end = min(hi, begin + run);
  double own = 0.0;
  for (int64_t at = begin; at < end; at += 4) {
    Four x;
    fetch(pt, pd, at, end, x);
#pragma unroll
    for (int k = 0; k < 4; ++k) own += value(x, k, at, n.A, n.B, n.gone);
  }
  double incl = own;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const double t = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += t;
  }
  __syncthreads();                         // s_warp has been read
  if (lane == 31) s_warp[warp] = incl;
  if (tid == 0) {
    s_more = kThreads;                     // the first thread whose run ends beyond the threshold
    s_kept = -1;                           // the last one with anything
  }
  __syncthreads();
  for (int w = 0; w < warp; ++w) before += s_warp[w];
  if (own > 0.0) {
    if (before + incl > threshold) atomicMin(&s_more, tid);
    atomicMax(&s_kept, tid);
  }
  __syncthreads();
  if (tid != (s_more < kThreads ? s_more : s_kept)) return;
  double sum = before + (incl - own);
  int64_t next = -1;
  for (int64_t at = begin; at < end && !(next >= 0 && sum > threshold); at += 4) {
    Four x;
    fetch(pt, pd, at, end, x);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const double v = value(x, k, at, n.A, n.B, n.gone);
      if (v > 0.0 && !(next >= 0 && sum > threshold)) {
        next = at + k;
        sum += v;
      }
    }
  }
  p.next[b] = (int)next;
}

int dynamic_bytes(int max_q, bool draft) { return (max_q * kRowBytes + 15) / 16 * 16 + 16 + (draft ? kWarps * kList * 8 : 0); }

template <bool kDraft, bool kWide>
cudaError_t launch(const VerifyLaunch& v, cudaStream_t s) {
  // A small vocabulary is one block's.  Else eight blocks a request (four fit on an SM: 74 requests at once), or, while all
  // requests are resident with them, sixteen: 4 / 16 trees over 128000 entries 20 / 27 us with eight, 15 / 20 with sixteen;
  // 64 trees 42 and 45 (all without lists).  Lists of 1024 entries would leave room for three blocks on an SM.
  const int blocks = v.vocab <= 4096 ? 1 : v.req.n <= 32 ? kMaxCluster : kMaxCluster / 2;
  static DeviceOnce once;
  int dev;
  if (once.pending(&dev)) {
    cudaError_t e = cudaFuncSetAttribute(verify_kernel<kDraft, kWide>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(verify_kernel<kDraft, kWide>, cudaFuncAttributeMaxDynamicSharedMemorySize, dynamic_bytes(KVC_TREE_MAX_Q, kDraft));
    if (e != cudaSuccess) return e;
    once.mark(dev);
  }
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim = {(unsigned)blocks, 1, 1};
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((int64_t)v.req.n * blocks));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = (size_t)dynamic_bytes(v.req.max_q, kDraft);
  cfg.stream = s;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, verify_kernel<kDraft, kWide>, v);
}

}  // namespace

cudaError_t launch_verify(const VerifyLaunch& v, cudaStream_t s) {
  // 16-byte loads where every row begins on 16 bytes
  const bool wide = ((reinterpret_cast<uintptr_t>(v.target) | (uintptr_t)(v.s_target * 4)) & 15) == 0 &&
                    (!v.draft || ((reinterpret_cast<uintptr_t>(v.draft) | (uintptr_t)(v.s_draft * 4)) & 15) == 0);
  if (v.draft) return wide ? launch<true, true>(v, s) : launch<true, false>(v, s);
  return wide ? launch<false, true>(v, s) : launch<false, false>(v, s);
}

}  // namespace kvc
