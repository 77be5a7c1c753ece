// ssm.cu — the recurrent half of a selective state-space layer on sm_103a: a short causal convolution per channel and the
// selective scan, for whole sequences and for single frames with carried states.
#include <algorithm>

#include "elem.cuh"
#include "qnn_device.cuh"
#include "qnn_host.h"

namespace qnn {
namespace {

__device__ __forceinline__ float silu(float v) { return __fdiv_rn(v, __fadd_rn(1.0f, expf(-v))); }

// Frames of sequence b.
__device__ __forceinline__ int64_t frames_of(const int32_t *lengths, int64_t b, int64_t T) {
    if (!lengths) return T;
    const int64_t n = __ldg(lengths + b);
    return n < 0 ? 0 : n > T ? T : n;
}

struct ConvArgs {
    const void *x, *state_in;
    void *state_out, *y;
    const float *w, *bias;
    const int32_t *lengths;
    int64_t x_seq, x_frame, y_seq, y_frame, B, T, D;
    int W, silu;
};

// A thread a channel of a sequence, all its frames in turn; it alone reads and writes the channel's state.
constexpr int kMostTaps = 8;
template <typename T>
__global__ void __launch_bounds__(128) causal_conv_plain_kernel(const ConvArgs a) {
    const int64_t at = (int64_t)blockIdx.x * 128 + threadIdx.x, b = at / a.D, d = at % a.D;
    if (b >= a.B) return;
    const int64_t n = frames_of(a.lengths, b, a.T);
    const int W = a.W;
    const T *x = static_cast<const T *>(a.x) + b * a.x_seq + d;
    T *y = static_cast<T *>(a.y) + b * a.y_seq + d;
    const T *in = static_cast<const T *>(a.state_in) + (b * (W - 1)) * a.D + d;
    T *out = static_cast<T *>(a.state_out) + (b * (W - 1)) * a.D + d;
    T taps[kMostTaps];  // the last W inputs, taps[W - 1] the newest
    float w[kMostTaps];
    for (int j = 0; j < W; ++j) w[j] = __ldg(a.w + d * W + j);
    for (int j = 0; j + 1 < W; ++j) taps[j + 1] = a.state_in ? in[j * a.D] : from_f32<T>(0.0f);
    const float bias = a.bias ? __ldg(a.bias + d) : 0.0f;
    for (int64_t t = 0; t < n; ++t) {
        for (int j = 0; j + 1 < W; ++j) taps[j] = taps[j + 1];
        taps[W - 1] = x[t * a.x_frame];
        float v = bias;
        for (int j = 0; j < W; ++j) v = __fmaf_rn(w[j], to_f32(taps[j]), v);
        y[t * a.y_frame] = from_f32<T>(a.silu ? silu(v) : v);
    }
    if (a.state_out)
        for (int j = 0; j + 1 < W; ++j) out[j * a.D] = taps[j + 1];
}

constexpr int kMostStates = 128;

// A warp a channel of a sequence, a lane every 32nd state.
template <typename T>
__global__ void __launch_bounds__(128) ssm_scan_plain_kernel(const qnn_ssm_args a) {
    const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5), b = at / a.D, d = at % a.D;
    const int lane = threadIdx.x & 31;
    if (b >= a.B) return;
    const int64_t frames = frames_of(a.lengths, b, a.T), g = d / (a.D / a.groups);
    float h[4], A[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int n = lane + 32 * i;
        h[i] = n < a.N && a.state_in ? a.state_in[(b * a.D + d) * a.N + n] : 0.0f;
        A[i] = n < a.N ? a.A[d * a.N + n] : 0.0f;
    }
    const float skip = a.skip ? a.skip[d] : 0.0f, bias = a.dt_bias ? a.dt_bias[d] : 0.0f;
    for (int64_t t = 0; t < frames; ++t) {
        const float u = to_f32(static_cast<const T *>(a.u)[b * a.u_seq + t * a.u_frame + d]);
        float s = __fadd_rn(to_f32(static_cast<const T *>(a.dt)[b * a.dt_seq + t * a.dt_frame + d]), bias);
        if (a.softplus && s <= 20.0f) s = log1pf(expf(s));
        const T *Bm = static_cast<const T *>(a.Bm) + b * a.Bm_seq + t * a.Bm_frame + g * a.N;
        const T *Cm = static_cast<const T *>(a.Cm) + b * a.Cm_seq + t * a.Cm_frame + g * a.N;
        float y = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = lane + 32 * i;
            if (n < a.N) {
                h[i] = __fmaf_rn(expf(__fmul_rn(s, A[i])), h[i], __fmul_rn(__fmul_rn(s, u), to_f32(Bm[n])));
                y = __fmaf_rn(to_f32(Cm[n]), h[i], y);
            }
        }
        y = __fmaf_rn(skip, u, warp_sum_f(y));
        if (a.z) y = __fmul_rn(y, silu(to_f32(static_cast<const T *>(a.z)[b * a.z_seq + t * a.z_frame + d])));
        if (lane == 0) static_cast<T *>(a.y)[b * a.y_seq + t * a.y_frame + d] = from_f32<T>(y);
    }
    if (a.state_out)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (lane + 32 * i < a.N) a.state_out[(b * a.D + d) * a.N + lane + 32 * i] = h[i];
}

constexpr int64_t kMostStride = (int64_t)1 << 40, kMostCount = (int64_t)1 << 40;

// A [B][T][width] array: its strides are in range, its first element aligned to its type.
bool frames_ok(const void *p, int64_t seq, int64_t frame, int e) {
    return seq >= 0 && frame >= 0 && seq <= kMostStride && frame <= kMostStride && (reinterpret_cast<uintptr_t>(p) & (e - 1)) == 0;
}
// No frame of an output overlaps another: sequences apart and frames apart within one, or the other way round.
bool apart(int64_t B, int64_t T, int64_t width, int64_t seq, int64_t frame) {
    const bool inner = T <= 1 || frame >= width, outer = B <= 1 || seq >= width;
    return inner && outer && (B <= 1 || T <= 1 || seq >= (T - 1) * frame + width || frame >= (B - 1) * seq + width);
}
Span frames_span(const void *p, int64_t B, int64_t T, int64_t width, int64_t seq, int64_t frame, int e) {
    return T > 0 ? Span(p, ((B - 1) * seq + (T - 1) * frame + width) * e) : Span();
}
bool sizes_ok(int64_t B, int64_t T, int64_t D) {
    return B >= 0 && T >= 0 && D >= 1 && T <= INT32_MAX && D <= INT32_MAX && B <= INT32_MAX && B * D <= kMostCount;
}
bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }
bool local_or_null(const void *p) { return !p || is_local_ptr(p); }

}  // namespace
}  // namespace qnn

using namespace qnn;

extern "C" qnn_status qnn_causal_conv(const void *x, int64_t x_seq, int64_t x_frame, int dtype, int64_t B, int64_t T, int64_t D,
                                      const float *w, int32_t W, const float *bias, int silu, const void *state_in,
                                      void *state_out, const int32_t *lengths, void *y, int64_t y_seq, int64_t y_frame,
                                      void *stream) {
    if (!dtype_ok(dtype) || !sizes_ok(B, T, D) || W < 1 || W > kMostTaps) return QNN_ERR_INVALID_ARG;
    const int e = dtype_size(dtype);
    if (!frames_ok(x, x_seq, x_frame, e) || !frames_ok(y, y_seq, y_frame, e) || !apart(B, T, D, y_seq, y_frame) ||
        !frames_ok(state_in, 0, 0, e) || !frames_ok(state_out, 0, 0, e) || !aligned4(w) || !aligned4(bias) || !aligned4(lengths))
        return QNN_ERR_INVALID_ARG;
    if (B == 0 || (T == 0 && !state_out)) return QNN_OK;
    if ((T > 0 && (!is_local_ptr(x) || !is_local_ptr(y))) || !is_local_ptr(w) || !local_or_null(bias) || !local_or_null(state_in) ||
        !local_or_null(state_out) || !local_or_null(lengths))
        return QNN_ERR_INVALID_ARG;
    const int64_t state = B * (W - 1) * D * e;
    const Span in[5] = {frames_span(x, B, T, D, x_seq, x_frame, e), Span(w, 4 * D * W), Span(bias, 4 * D), Span(lengths, 4 * B),
                        Span(state_in, state)};
    const Span ys = frames_span(y, B, T, D, y_seq, y_frame, e), so(state_out, state);
    if (ys.meets(so)) return QNN_ERR_INVALID_ARG;
    for (int i = 0; i < 5; ++i)
        if (ys.meets(in[i]) || (so.meets(in[i]) && !(i == 4 && state_in == state_out))) return QNN_ERR_INVALID_ARG;
    ConvArgs a;
    a.x = x, a.state_in = state_in, a.state_out = state_out, a.y = y, a.w = w, a.bias = bias, a.lengths = lengths;
    a.x_seq = x_seq, a.x_frame = x_frame, a.y_seq = y_seq, a.y_frame = y_frame, a.B = B, a.T = T, a.D = D, a.W = W, a.silu = silu != 0;
    const int64_t blocks = (B * D + 127) / 128;
    if (blocks > INT32_MAX) return QNN_ERR_INVALID_ARG;
    cudaStream_t st = as_stream(stream);
    ProfScope prof("causal_conv", st);
    with_type(dtype, [&](auto t) { causal_conv_plain_kernel<decltype(t)><<<(unsigned)blocks, 128, 0, st>>>(a); });
    QNN_CUDA_TRY(cudaGetLastError());
    return QNN_OK;
}

extern "C" qnn_status qnn_ssm_scan(const qnn_ssm_args *args, void *stream) {
    if (!args) return QNN_ERR_INVALID_ARG;
    const qnn_ssm_args &a = *args;
    if (!dtype_ok(a.dtype) || !sizes_ok(a.B, a.T, a.D) || a.N < 1 || a.N > kMostStates || a.groups < 1 || a.D % a.groups)
        return QNN_ERR_INVALID_ARG;
    const int e = dtype_size(a.dtype);
    const int64_t gn = (int64_t)a.groups * a.N;
    if (!frames_ok(a.u, a.u_seq, a.u_frame, e) || !frames_ok(a.dt, a.dt_seq, a.dt_frame, e) ||
        !frames_ok(a.Bm, a.Bm_seq, a.Bm_frame, e) || !frames_ok(a.Cm, a.Cm_seq, a.Cm_frame, e) ||
        (a.z && !frames_ok(a.z, a.z_seq, a.z_frame, e)) || !frames_ok(a.y, a.y_seq, a.y_frame, e) ||
        !apart(a.B, a.T, a.D, a.y_seq, a.y_frame) || !aligned4(a.A) || !aligned4(a.skip) || !aligned4(a.dt_bias) ||
        !aligned4(a.state_in) || !aligned4(a.state_out) || !aligned4(a.lengths))
        return QNN_ERR_INVALID_ARG;
    if (a.B == 0 || (a.T == 0 && !a.state_out)) return QNN_OK;
    if ((a.T > 0 && (!is_local_ptr(a.u) || !is_local_ptr(a.dt) || !is_local_ptr(a.Bm) || !is_local_ptr(a.Cm) || !is_local_ptr(a.y) ||
                     !local_or_null(a.z))) ||
        !is_local_ptr(a.A) || !local_or_null(a.skip) || !local_or_null(a.dt_bias) || !local_or_null(a.state_in) ||
        !local_or_null(a.state_out) || !local_or_null(a.lengths))
        return QNN_ERR_INVALID_ARG;
    const int64_t state = 4 * a.B * a.D * a.N;
    const Span in[10] = {frames_span(a.u, a.B, a.T, a.D, a.u_seq, a.u_frame, e),
                         frames_span(a.dt, a.B, a.T, a.D, a.dt_seq, a.dt_frame, e),
                         frames_span(a.Bm, a.B, a.T, gn, a.Bm_seq, a.Bm_frame, e),
                         frames_span(a.Cm, a.B, a.T, gn, a.Cm_seq, a.Cm_frame, e),
                         a.z ? frames_span(a.z, a.B, a.T, a.D, a.z_seq, a.z_frame, e) : Span(),
                         Span(a.A, 4 * a.D * a.N),
                         Span(a.skip, 4 * a.D),
                         Span(a.dt_bias, 4 * a.D),
                         Span(a.lengths, 4 * a.B),
                         Span(a.state_in, state)};
    const Span ys = frames_span(a.y, a.B, a.T, a.D, a.y_seq, a.y_frame, e), so(a.state_out, state);
    if (ys.meets(so)) return QNN_ERR_INVALID_ARG;
    for (int i = 0; i < 10; ++i)
        if (ys.meets(in[i]) || (so.meets(in[i]) && !(i == 9 && a.state_in == a.state_out))) return QNN_ERR_INVALID_ARG;
    const int64_t blocks = (a.B * a.D + 3) / 4;
    if (blocks > INT32_MAX) return QNN_ERR_INVALID_ARG;
    cudaStream_t st = as_stream(stream);
    ProfScope prof("ssm_scan", st);
    with_type(a.dtype, [&](auto t) { ssm_scan_plain_kernel<decltype(t)><<<(unsigned)blocks, 128, 0, st>>>(a); });
    QNN_CUDA_TRY(cudaGetLastError());
    return QNN_OK;
}
