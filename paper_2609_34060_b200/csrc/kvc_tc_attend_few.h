// Host interface of the few-rows kernel of kvc_attend (kvc_tc_attend_few.cu).
#pragma once
#include "kvc_tc_attend.cuh"

namespace kvc {

int few_capacity(int64_t rows);
size_t few_workspace_bytes(int n, int max_kv, int H, int d, int rc);
cudaError_t launch_attend_few(const AttendLaunch& a, const tc::TileGeo& g, const CUtensorMap& mk, const CUtensorMap& mv, int rc, int d, float* part,
                              cudaStream_t s);

}  // namespace kvc
