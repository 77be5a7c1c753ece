// linattn_bf16.cu — linear attention's chunked kernels for bf16 values.
#include "linattn.cuh"

namespace qnn {
template qnn_status launch_linear_chunks<__nv_bfloat16>(const LinearArgs &, cudaStream_t);
}  // namespace qnn
