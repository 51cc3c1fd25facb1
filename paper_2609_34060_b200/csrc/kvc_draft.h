// Launch interface of the operators on drafted tokens: kvc_tree_build, kvc_append_rotated, kvc_verify, kvc_keep.
#pragma once
#include "kvc_attend.h"

namespace kvc {

struct TreeLaunch {
  DevRequests req;
  const int32_t* parent;
  uint32_t* mask;
  int32_t* depth;
  int32_t words;
  uint32_t* status;
};

struct RotateLaunch {
  DevRequests req;
  DevHeads q, qo, kn, vn;
  DevCache dst;
  DevScale e;
  int32_t Hq, H, layer, rot, pairing;
  float amplitude;
  const int32_t* depth;
  const int32_t* pos_begin;
  uint32_t* status;
  double turns[kMaxHalfD];     // f_k / 2 pi
};

struct VerifyLaunch {
  DevRequests req;
  const int32_t* parent;
  const int32_t* token;
  const float* target;
  const float* draft;          // nullptr: the drafts were chosen
  int64_t s_target, s_draft;
  int32_t vocab, stride;       // of kept
  const float* u;
  const float* u_next;
  int32_t* kept;
  int32_t* n_kept;
  int32_t* next;
  uint32_t* status;
};

struct KeepLaunch {
  DevRequests req;
  DevCache c;
  DevScale e;
  int32_t L, H, stride;
  const int32_t* kept;
  const int32_t* n_kept;
  int32_t* kv_out;
  uint32_t* status;
};

// A call's arguments in one piece, as the Python binding hands them over (one argument costs it a third of nine).
struct AppendRotatedCall {
  const kvc_requests* req;
  const kvc_rotary* rot;
  void* cache;                 // kvc_cache or, with q8, kvc_qcache
  int64_t q8;
  void* stream;
  kvc_heads q, q_out, k_new, v_new;
  int32_t layer, has_q;
  int32_t n_depth, n_pos;      // entries that depth and pos_begin hold; -1: there are none
};
struct AttendTreeCall {
  const kvc_requests* req;
  const kvc_tree* tree;
  const void* cache;
  int64_t q8;
  float* lse;
  void* workspace;
  uint64_t workspace_bytes;
  void* stream;
  double scale;
  kvc_heads q, out;
  int64_t layer;
};
struct VerifyCall {
  const kvc_requests* req;
  kvc_probs target, draft;
  const int32_t* parent;
  const int32_t* token;
  const float* u;
  const float* u_next;
  int32_t* kept;
  int64_t stride;              // of kept
  int32_t* n_kept;
  int32_t* next;
  void* stream;
  int64_t has_draft;
};
struct KeepCall {
  const kvc_requests* req;
  const int32_t* kept;
  int64_t stride;
  const int32_t* n_kept;
  void* cache;
  int64_t q8;
  int32_t* kv_out;
  void* stream;
};

cudaError_t launch_tree_build(const TreeLaunch& t, cudaStream_t s);
cudaError_t launch_append_rotated(const RotateLaunch& r, int d, cudaStream_t s);
cudaError_t launch_verify(const VerifyLaunch& v, cudaStream_t s);
cudaError_t launch_keep(const KeepLaunch& k, int d, cudaStream_t s);

}  // namespace kvc
