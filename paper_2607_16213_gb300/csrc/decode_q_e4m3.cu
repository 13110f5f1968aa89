// The e4m3 kernels of decode_q.cuh.
#include "decode_q.cuh"

namespace selkv {
cudaError_t launch_decode_q_e4m3(const QDecodeArgs& a, cudaStream_t st) { return launch_type<SELKV_Q_E4M3>(a, st); }
}  // namespace selkv
