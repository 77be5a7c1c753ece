// linattn_f32.cu — linear attention's chunked kernels for f32 values.
#include "linattn.cuh"

namespace qnn {
template qnn_status launch_linear_chunks<float>(const LinearArgs &, cudaStream_t);
}  // namespace qnn
