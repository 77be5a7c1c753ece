// linattn.h — linear attention with a decay for each head: arguments of its kernels, and the launches by type.
#pragma once

#include "qnn_host.h"

namespace qnn {

struct LinearArgs {
    const void *q, *k, *v;
    void *y;
    const float *log_decay, *state_in;
    float *state_out, *partial;  // partial: [B H][parts][dk][dv], what each part but the last ends with from zeros, then what each begins with
    const int32_t *lengths;
    int64_t q_seq, q_frame, k_seq, k_frame, v_seq, v_frame, y_seq, y_frame, B, T;
    int64_t per;  // frames of a part
    int H, q_share, k_share, v_share, dk, dv;  // heads that share one of q, k, v
    int parts, tiles;                          // parts of a sequence, tiles of a head's columns
    int q_copy, k_copy, v_copy, y_copy;        // bytes of an asynchronous copy: 16, 8 or 4, or 0 where values lie apart from those
    float scale;
    bool pairs;  // y takes pairs of values
};

// Whole sequences by chunks of frames (the parts' states first, where there are parts).
template <typename T>
qnn_status launch_linear_chunks(const LinearArgs &a, cudaStream_t st);
// bf16 sequences on the tcgen05 tensor cores, without parts: whether it takes the sizes and places, and its launch.
bool linear_tc_fits(const LinearArgs &a);
qnn_status launch_linear_tc(const LinearArgs &a, cudaStream_t st);
// Frames of a chunk.
int linear_chunk(int dtype, int dk);

}  // namespace qnn
