// The linear layers of many experts, each with the rows that a plan gives it, on the tensor cores: see mx_tc.cuh, MODE 2.
#include "mx_tc.cuh"

namespace aiq {

aiq_status_t launch_mx_linear_experts(const MxProduct& p, void* workspace, cudaStream_t s) {
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  bool done;
  if (aiq_status_t st = launch_mx_few(p, s, &done)) return st;
  if (done) return AIQ_OK;
  MxExpireOnce once;
  switch (p.dtype) {
    case AIQ_DTYPE_F32: return launch_kind<1, float, 2>(p, ws, s);
    case AIQ_DTYPE_F16: return launch_kind<1, __half, 2>(p, ws, s);
    default: return launch_kind<1, __nv_bfloat16, 2>(p, ws, s);
  }
}

}  // namespace aiq
