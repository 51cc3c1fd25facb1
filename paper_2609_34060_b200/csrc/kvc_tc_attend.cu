// Tensor-core kernels of kvc_attend: none yet, every call runs on the CUDA cores (kvc_attend_generic.cu).
#include "kvc_attend.h"
#include "kvc_tc.h"

namespace kvc {
size_t tc_attend_workspace_bytes(int, int, int, int, int, int) { return 0; }
int tc_attend(const AttendLaunch&, int, int, cudaStream_t) { return KVC_E_UNSUPPORTED; }
}  // namespace kvc
