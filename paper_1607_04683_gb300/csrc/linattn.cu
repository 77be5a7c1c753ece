// linattn.cu — linear attention with a decay for each head on sm_103a: the call, and its recurrent kernel for few frames.
#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <cstring>

#include "elem.cuh"
#include "linattn.h"
#include "qnn_device.cuh"
#include "qnn_host.h"

namespace qnn {
namespace {

constexpr int kMostDim = 256;

// Few frames: the states are most of the traffic, in and out. A block takes 32 columns of one head's state, whose rows lie in
// runs of 128 bytes; a warp four rows of them at a time, kRows times in flight. A row's part in the outputs is added over the
// warp's rows by shuffles and over the block's warps in shared memory. Bound: HBM for the states; 256 sequences x 16 heads x 128 x 128, one
// frame, 541 MB: 79.5 us, 6.8 TB/s (the copy's rate).
constexpr int kStepFrames = 8, kStepThreads = 128, kStepCols = 32, kRows = 8, kBlockRows = kRows * kStepThreads / 8;
template <typename T, bool VEC, int FRAMES>
__global__ void __launch_bounds__(kStepThreads) linear_step_kernel(const LinearArgs a) {
    __shared__ float qk[2][FRAMES][kMostDim];
    __shared__ float parts[kStepThreads / 32][FRAMES][kStepCols];
    int64_t at = blockIdx.x;
    const int tile = (int)(at % a.tiles);
    const int64_t unit = at / a.tiles, b = unit / a.H;
    const int h = (int)(unit % a.H), warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int n = frames_of(a.lengths, b, a.T);
    const float g = __ldg(a.log_decay + h);
    const float decay = expf(g > 0.0f ? 0.0f : g);
    // a lane's four columns: neighbours, or every eighth where runs are not aligned
    int col[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) col[c] = tile * kStepCols + (VEC ? lane % 8 * 4 + c : lane % 8 + 8 * c);
    const int64_t size = (int64_t)a.dk * a.dv;
    const float *in = a.state_in ? a.state_in + unit * size : nullptr;
    float *out = a.state_out ? a.state_out + unit * size : nullptr;
    const int row0 = threadIdx.x / 8;  // rows row0 + 16 i
    float S[kRows][4];
    auto load = [&](int r0) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int r = r0 + row0 + i * (kStepThreads / 8);
            if constexpr (VEC) {
                const bool there = in && r < a.dk && col[0] < a.dv;
                const float4 v = there ? __ldcs(reinterpret_cast<const float4 *>(in + (int64_t)r * a.dv + col[0])) : make_float4(0, 0, 0, 0);
                S[i][0] = v.x, S[i][1] = v.y, S[i][2] = v.z, S[i][3] = v.w;
            } else {
#pragma unroll
                for (int c = 0; c < 4; ++c) S[i][c] = in && r < a.dk && col[c] < a.dv ? __ldcs(in + (int64_t)r * a.dv + col[c]) : 0.0f;
            }
        }
    };
    load(0);
    const T *q = static_cast<const T *>(a.q) + b * a.q_seq + (int64_t)(h / a.q_share) * a.dk;
    const T *k = static_cast<const T *>(a.k) + b * a.k_seq + (int64_t)(h / a.k_share) * a.dk;
    const T *v = static_cast<const T *>(a.v) + b * a.v_seq + (int64_t)(h / a.v_share) * a.dv;
    float vt[FRAMES][4], y[FRAMES][4];
#pragma unroll
    for (int f = 0; f < FRAMES; ++f)
        if (f < n) {
            for (int i = threadIdx.x; i < a.dk; i += kStepThreads) {
                qk[0][f][i] = to_f32(q[f * a.q_frame + i]);
                qk[1][f][i] = to_f32(k[f * a.k_frame + i]);
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) vt[f][c] = col[c] < a.dv ? to_f32(v[f * a.v_frame + col[c]]) : 0.0f, y[f][c] = 0.0f;
        }
    __syncthreads();
    for (int r0 = 0; r0 < a.dk; r0 += kBlockRows) {
        if (r0) load(r0);
#pragma unroll
        for (int f = 0; f < FRAMES; ++f)
            if (f < n) {
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    const int r = r0 + row0 + i * (kStepThreads / 8);
                    if (r < a.dk) {
                        const float qr = qk[0][f][r], kr = qk[1][f][r];
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            S[i][c] = __fmaf_rn(kr, vt[f][c], __fmul_rn(S[i][c], decay));
                            y[f][c] = __fmaf_rn(qr, S[i][c], y[f][c]);
                        }
                    }
                }
            }
        if (out)
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const int r = r0 + row0 + i * (kStepThreads / 8);
                if constexpr (VEC) {
                    if (r < a.dk && col[0] < a.dv)
                        __stcs(reinterpret_cast<float4 *>(out + (int64_t)r * a.dv + col[0]), make_float4(S[i][0], S[i][1], S[i][2], S[i][3]));
                } else {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (r < a.dk && col[c] < a.dv) __stcs(out + (int64_t)r * a.dv + col[c], S[i][c]);
                }
            }
    }
#pragma unroll
    for (int f = 0; f < FRAMES; ++f)
        if (f < n) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float s = y[f][c];
                s = __fadd_rn(s, __shfl_xor_sync(0xffffffffu, s, 8));
                s = __fadd_rn(s, __shfl_xor_sync(0xffffffffu, s, 16));
                if (lane < 8) parts[warp][f][col[c] - tile * kStepCols] = s;
            }
        }
    __syncthreads();
    for (int i = threadIdx.x; i < n * kStepCols; i += kStepThreads) {
        const int f = i / kStepCols, c = i % kStepCols;
        if (tile * kStepCols + c < a.dv) {
            float s = parts[0][f][c];
#pragma unroll
            for (int w = 1; w < kStepThreads / 32; ++w) s = __fadd_rn(s, parts[w][f][c]);
            static_cast<T *>(a.y)[b * a.y_seq + f * a.y_frame + (int64_t)h * a.dv + tile * kStepCols + c] = from_f32<T>(__fmul_rn(s, a.scale));
        }
    }
}

template <typename T, int FRAMES>
qnn_status launch_step(const LinearArgs &a, bool vec, cudaStream_t st) {
    const int64_t blocks = a.B * a.H * a.tiles;
    if (blocks > INT32_MAX) return QNN_FAIL(QNN_ERR_INVALID_ARG);
    if (vec) linear_step_kernel<T, true, FRAMES><<<(unsigned)blocks, kStepThreads, 0, st>>>(a);
    else linear_step_kernel<T, false, FRAMES><<<(unsigned)blocks, kStepThreads, 0, st>>>(a);
    return QNN_OK;
}
template <typename T>
qnn_status launch_step(const LinearArgs &a, bool vec, cudaStream_t st) {
    return a.T <= 1 ? launch_step<T, 1>(a, vec, st) : a.T <= 4 ? launch_step<T, 4>(a, vec, st) : launch_step<T, kStepFrames>(a, vec, st);
}

// Bytes of an asynchronous copy from which rows of [B][T][heads][width] can be put together.
int copy_unit(const void *p, int64_t B, int64_t T, int64_t heads, int64_t width, int64_t seq, int64_t frame, int e) {
    uintptr_t bits = reinterpret_cast<uintptr_t>(p);
    if (B > 1) bits |= (uintptr_t)(seq * e);
    if (T > 1) bits |= (uintptr_t)(frame * e);
    if (heads > 1) bits |= (uintptr_t)(width * e);
    return bits % 16 == 0 ? 16 : bits % 8 == 0 ? 8 : bits % 4 == 0 ? 4 : 0;
}

// Which of the two kernels takes a bf16 sequence, by what they took (us): the tcgen05 one a chunk of 128 frames in 3.3 and a unit in
// 1.7 more, one block an SM; the other a chunk of 64 frames in 4.4 or 5.8, or with the sequence in parts both passes of a part's chunks, that take
// longer with more blocks an SM, and 9 or 13 for the call. Sequences x frames x heads x dk: 1 x 16 x 8 x 64 10.4 / 8.3, 1 x 128 x 8 x 64 10.4 / 12.6, 1 x 300
// x 4 x 64 16.6 / 12.6, 8 x 300 x 8 x 64 16.6 / 19.8, 1 x 1000 x 8 x 64 33 / 16.6, 8 x 1000 x 8 x 64 33 / 39; 1 x 500 x 4 x 128 20.6 / 18.8, 1 x 1000 x 16 x 128 33.1 /
// 33.4, 2 x 1000 x 16 x 128 35 / 56, 1 x 2000 x 16 x 128 60 / 53, 1 x 4000 x 16 x 128 112 / 83, 16 x 1000 x 16 x 128 138 / 238.
// Frames are T for every sequence (lengths lie on the device); batches of a third to all of T were not fitted, but keep to it: 8 x 300 x 8 x 64 15.5 /
// 18.9, 2 x 1000 x 16 x 128 35 / 56, 16 x 1000 x 16 x 128 97 / 183.
bool prefers_tc(const LinearArgs &a, int chunk, int64_t chunks) {
    if (const char *e = std::getenv("QNN_LINEAR")) {  // one of them always (tests)
        if (std::strcmp(e, "tc") == 0) return true;
        if (std::strcmp(e, "chunks") == 0) return false;
    }
    const double units = (double)(a.B * a.H * a.tiles), sms = sm_count(), full = units * a.parts / sms;
    const double tc = 5.5 + (1.7 + 3.3 * (double)((a.T + 127) / 128)) * std::ceil(units / sms);
    const bool wide = a.dk > 64;
    if (a.parts > 1) return tc < (wide ? 13.0 : 9.0) + (double)(a.per / chunk) * (wide ? 5.5 + 2.6 * full : 4.5 + 2.4 * full);
    return tc < (wide ? 3.0 : 4.0) + (wide ? 5.8 : 4.4) * (double)chunks * std::ceil(full / (wide ? 2.0 : 3.0));
}

}  // namespace

int linear_chunk(int dtype, int dk) { return (dtype == QNN_BF16 ? 64 : 32) / (dk > 128 ? 2 : 1); }

}  // namespace qnn

using namespace qnn;

extern "C" qnn_status qnn_linear_attention(const qnn_linear_args *args, void *stream) {
    if (!args) return QNN_ERR_INVALID_ARG;
    const qnn_linear_args &p = *args;
    if (!dtype_ok(p.dtype) || p.B < 0 || p.T < 0 || p.T > (1 << 30) || p.B > INT32_MAX || p.H < 1 || p.H > 65536 || p.q_heads < 1 ||
        p.H % p.q_heads || p.k_heads < 1 || p.H % p.k_heads || p.v_heads < 1 || p.H % p.v_heads || p.dk < 1 || p.dk > kMostDim ||
        p.dv < 1 || p.dv > kMostDim || !(p.scale > -INFINITY && p.scale < INFINITY) || !reach_ok(p.T, p.B * p.H * kMostDim))
        return QNN_ERR_INVALID_ARG;
    const int e = dtype_size(p.dtype);
    const int64_t B = p.B, T = p.T, wq = (int64_t)p.q_heads * p.dk, wk = (int64_t)p.k_heads * p.dk, wv = (int64_t)p.v_heads * p.dv,
                  wy = (int64_t)p.H * p.dv;
    if (!frames_ok(p.q, B, T, p.q_seq, p.q_frame, e) || !frames_ok(p.k, B, T, p.k_seq, p.k_frame, e) ||
        !frames_ok(p.v, B, T, p.v_seq, p.v_frame, e) || !frames_ok(p.y, B, T, p.y_seq, p.y_frame, e) ||
        !apart(B, T, wy, p.y_seq, p.y_frame) || !aligned4(p.log_decay) || !aligned4(p.state_in) || !aligned4(p.state_out) ||
        !aligned4(p.lengths))
        return QNN_ERR_INVALID_ARG;
    if (B == 0 || (T == 0 && !p.state_out)) return QNN_OK;
    if ((T > 0 && (!is_local_ptr(p.q) || !is_local_ptr(p.k) || !is_local_ptr(p.v) || !is_local_ptr(p.y))) ||
        !is_local_ptr(p.log_decay) || !local_or_null(p.state_in) || !local_or_null(p.state_out) || !local_or_null(p.lengths))
        return QNN_ERR_INVALID_ARG;
    const int64_t states = B * p.H * p.dk * p.dv;
    const Span in[6] = {frames_span(p.q, B, T, wq, p.q_seq, p.q_frame, e), frames_span(p.k, B, T, wk, p.k_seq, p.k_frame, e),
                        frames_span(p.v, B, T, wv, p.v_seq, p.v_frame, e), Span(p.log_decay, 4 * p.H), Span(p.lengths, 4 * B),
                        Span(p.state_in, 4 * states)};
    const Span ys = frames_span(p.y, B, T, wy, p.y_seq, p.y_frame, e), so(p.state_out, 4 * states);
    if (ys.meets(so)) return QNN_ERR_INVALID_ARG;
    for (int i = 0; i < 6; ++i)
        if (ys.meets(in[i]) || (so.meets(in[i]) && !(i == 5 && p.state_in == p.state_out))) return QNN_ERR_INVALID_ARG;
    LinearArgs a = {};
    a.q = p.q, a.k = p.k, a.v = p.v, a.y = p.y, a.log_decay = p.log_decay, a.state_in = p.state_in, a.state_out = p.state_out;
    a.lengths = p.lengths, a.q_seq = p.q_seq, a.q_frame = p.q_frame, a.k_seq = p.k_seq, a.k_frame = p.k_frame, a.v_seq = p.v_seq;
    a.v_frame = p.v_frame, a.y_seq = p.y_seq, a.y_frame = p.y_frame, a.B = B, a.T = T, a.H = p.H, a.dk = p.dk, a.dv = p.dv;
    a.q_share = p.H / p.q_heads, a.k_share = p.H / p.k_heads, a.v_share = p.H / p.v_heads, a.scale = p.scale, a.parts = 1;
    cudaStream_t st = as_stream(stream);
    if (T <= kStepFrames) {
        a.tiles = (p.dv + kStepCols - 1) / kStepCols;
        auto at16 = [](const void *q) { return reinterpret_cast<uintptr_t>(q) % 16 == 0; };
        const bool vec = p.dv % 4 == 0 && at16(p.state_in) && at16(p.state_out);
        ProfScope prof("linear_step", st);
        QNN_TRY(with_type(p.dtype, [&](auto t) { return launch_step<decltype(t)>(a, vec, st); }));
        QNN_CUDA_TRY(cudaGetLastError());
        return QNN_OK;
    }
    a.tiles = (p.dv + 63) / 64;
    a.q_copy = copy_unit(p.q, B, T, p.q_heads, p.dk, p.q_seq, p.q_frame, e);
    a.k_copy = copy_unit(p.k, B, T, p.k_heads, p.dk, p.k_seq, p.k_frame, e);
    a.v_copy = copy_unit(p.v, B, T, p.v_heads, p.dv, p.v_seq, p.v_frame, e);
    a.y_copy = copy_unit(p.y, B, T, p.H, p.dv, p.y_seq, p.y_frame, e);
    const uintptr_t ybits = reinterpret_cast<uintptr_t>(p.y) | (uintptr_t)((B > 1 ? p.y_seq * e : 0) | p.y_frame * e | (int64_t)p.dv * e);
    a.pairs = ybits % (2 * e) == 0;
    // Parts of a sequence: as many as the SMs hold blocks of at once, of a chunk at least, where both passes take less than one: a
    // chunk c us (3.5 to 6.5) and 2 more, in parts 13 and 1.7 c a chunk. fp32 8 x 200 x 8 x 64 by 1, 2, 3, 4, 7 parts 33, 45, 37, 30,
    // 22 us; 1 x 1000 x 8 x 64 by 16 and 32 27 and 19; 1 x 4000 x 8 x 64 by 32, 42, 63 47, 40, 41; 1 x 1000 x 16 x 128 by 8, 16, 32 60, 64, 75;
    // 10 x 1000 x 16 x 64 by 1 and 2 173 and 168, of fp16 124 and 141.
    const int chunk = linear_chunk(p.dtype, p.dk), held = p.dk > 64 ? 2 : 3;
    const int64_t units = B * p.H * a.tiles, chunks = (T + chunk - 1) / chunk;
    int64_t parts = std::max<int64_t>(1, std::min<int64_t>({held * (int64_t)sm_count() / units, chunks, 64}));
    int64_t per = (chunks + parts - 1) / parts;
    if (5 * per + 8 > 3 * chunks || (p.dk <= 64 && parts < 3)) per = chunks;
    a.parts = (int)((chunks + per - 1) / per);
    a.per = per * chunk;
    if (p.dtype == QNN_BF16 && linear_tc_fits(a) && prefers_tc(a, chunk, chunks)) {
        ProfScope prof("linear_attention", st);
        return launch_linear_tc(a, st);
    }
    Scratch scratch;
    if (a.parts > 1) {
        QNN_TRY(scratch.take((size_t)(B * p.H * a.parts) * p.dk * p.dv * sizeof(float), st));
        a.partial = static_cast<float *>(scratch.ptr());
    }
    ProfScope prof("linear_attention", st);
    return with_type(p.dtype, [&](auto t) { return launch_linear_chunks<decltype(t)>(a, st); });
}
