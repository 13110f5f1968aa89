// The int8 kernels of decode_q.cuh.
#include "decode_q.cuh"

namespace selkv {
cudaError_t launch_decode_q_int8(const QDecodeArgs& a, cudaStream_t st) { return launch_type<SELKV_Q_INT8>(a, st); }
}  // namespace selkv
