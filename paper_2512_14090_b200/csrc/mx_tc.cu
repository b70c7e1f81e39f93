// The plain products on the tensor cores: see mx_tc.cuh.
#include "mx_tc.cuh"

namespace aiq {
namespace {
thread_local long long mx_expire = 0;          // cycles: the next product of this thread holds an arrival back, 0: none does
}

size_t mx_tc_workspace_bytes(int K, int M, int dtype) {
  return align_up((size_t)mx_pieces(dtype) * M * (size_t)(mx_plane_row(K) + mx_scale_row_bytes(K)), 16);
}

void mx_tc_expire_next(int64_t limit_cycles) { mx_expire = limit_cycles; }
long long mx_tc_expire_cycles() { return mx_expire; }

aiq_status_t launch_mx_product_tc(const MxProduct& p, void* workspace, cudaStream_t s) {
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  MxExpireOnce once;
  switch (p.dtype) {
    case AIQ_DTYPE_F32: return p.x ? launch_kind<1, float, 0>(p, ws, s) : launch_kind<0, float, 0>(p, ws, s);
    case AIQ_DTYPE_F16: return p.x ? launch_kind<1, __half, 0>(p, ws, s) : launch_kind<0, __half, 0>(p, ws, s);
    default: return p.x ? launch_kind<1, __nv_bfloat16, 0>(p, ws, s) : launch_kind<0, __nv_bfloat16, 0>(p, ws, s);
  }
}

}  // namespace aiq
