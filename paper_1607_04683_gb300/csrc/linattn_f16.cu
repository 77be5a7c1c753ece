// linattn_f16.cu — linear attention's chunked kernels for f16 values.
#include "linattn.cuh"

namespace qnn {
template qnn_status launch_linear_chunks<__half>(const LinearArgs &, cudaStream_t);
}  // namespace qnn
