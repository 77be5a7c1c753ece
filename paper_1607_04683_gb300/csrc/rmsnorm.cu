// rmsnorm.cu — residual addition, root-mean-square norm and the on-the-fly quantizer (Sec. 3, eq. 2) on sm_103a:
// h = x + r; s = 1 / sqrt(mean h^2 + eps); v = (h s) w; one 8-bit unit per row of v.
//
// Every code of a row goes by the last bit of s, so s must not depend on how the sum is split: the squares are summed in
// pairs of fp32 (value and remainder, about 2^-46 relative), the root is taken of the pair and rounded once.
#include <cfloat>

#include "elem.cuh"
#include "qnn_device.cuh"
#include "qnn_host.h"

namespace qnn {
namespace {

// An unevaluated sum of two fp32 numbers. add(): Knuth's exact addition (the rounding error of hi + v, whatever their
// order of size, goes to lo); add_square(): v^2 is p + e exactly by a fused multiply-add (while e is above the least
// subnormal; what is lost below lies 2^-80 under eps).
struct Pair {
    float hi = 0.0f, lo = 0.0f;
    __device__ __forceinline__ void add(float v, float rest) {
        const float s = __fadd_rn(hi, v);
        const float b = __fsub_rn(s, hi);
        const float err = __fadd_rn(__fsub_rn(hi, __fsub_rn(s, b)), __fsub_rn(v, b));
        hi = s;
        lo = __fadd_rn(lo, __fadd_rn(err, rest));
    }
    __device__ __forceinline__ void add_square(float v) {
        const float p = __fmul_rn(v, v);
        add(p, __fmaf_rn(v, v, -p));
    }
    __device__ __forceinline__ void add(const Pair &o) { add(o.hi, o.lo); }
};

__device__ __forceinline__ Pair warp_sum_pair(Pair a) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        Pair b;
        b.hi = __shfl_xor_sync(0xffffffffu, a.hi, o);
        b.lo = __shfl_xor_sync(0xffffffffu, a.lo, o);
        a.add(b);
    }
    return a;
}

// 1 / sqrt(sum / n + eps) rounded once, for sum and eps as pairs: the hardware root r (two ulp) and the next two terms of
// its series in e = 1 - m r^2, which is formed exactly up to 2^-48: r (1 + e/2 + 3/8 e^2).
__device__ __forceinline__ float inverse_rms(const Pair &sum, float n, float eps_hi, float eps_lo) {
    Pair m;
    m.hi = __fdiv_rn(sum.hi, n);
    m.lo = __fdiv_rn(__fadd_rn(__fmaf_rn(-m.hi, n, sum.hi), sum.lo), n);
    m.add(eps_hi, eps_lo);
    const float mh = __fadd_rn(m.hi, m.lo), ml = __fadd_rn(__fsub_rn(m.hi, mh), m.lo);
    // a power of four out of m, so that the root's square and the products stay far from the ends of the range
    const int half = ((__float_as_int(mh) >> 23) - 127) >> 1;
    const float down = __int_as_float((127 - half) << 23);
    const float a = __fmul_rn(__fmul_rn(mh, down), down), b = __fmul_rn(__fmul_rn(ml, down), down);
    const float r = rsqrtf(a);
    const float t = __fmul_rn(r, r), te = __fmaf_rn(r, r, -t);
    const float p = __fmul_rn(a, t), pe = __fmaf_rn(a, t, -p);
    const float e = __fsub_rn(__fsub_rn(__fsub_rn(__fsub_rn(1.0f, p), pe), __fmul_rn(a, te)), __fmul_rn(b, t));
    const float c = __fmul_rn(__fmaf_rn(0.375f, __fmul_rn(e, e), __fmul_rn(0.5f, e)), r);
    return __fmul_rn(__fadd_rn(r, c), down);
}

// Rows whose squares overflow are summed again at this scale.
constexpr float kDown = 0x1p-80f;

struct NormArgs {
    const void *x, *r;
    void *h;
    const float *w;
    int64_t rows, ldx, ldr, ldh, ldc, ldv;
    int cols;
    float eps_hi, eps_lo, eps_down_hi;
    uint8_t *codes;
    qnn_qparams *params;
    int32_t *sums;
    float *values;
    int *status;
};

// A row a block, three passes over it (sum of squares, range, codes), h formed again in each: every element is read and
// written by one thread, so h may take the place of x or r.
constexpr int kThreads = 256, kWarps = kThreads / 32;
template <typename T>
__global__ void __launch_bounds__(kThreads) rmsnorm_long_rows_kernel(const NormArgs a) {
    __shared__ Pair s_sum[kWarps];
    __shared__ float s_mn[kWarps], s_mx[kWarps];
    __shared__ int s_bad[kWarps], s_cnt[kWarps];
    const int64_t row = blockIdx.x;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const T *x = static_cast<const T *>(a.x) + row * a.ldx;
    const T *r = a.r ? static_cast<const T *>(a.r) + row * a.ldr : nullptr;
    auto h_at = [&](int k) { return r ? __fadd_rn(to_f32(x[k]), to_f32(r[k])) : to_f32(x[k]); };
    auto total = [&](float scale) {
        Pair p;
        for (int k = threadIdx.x; k < a.cols; k += kThreads) p.add_square(__fmul_rn(h_at(k), scale));
        p = warp_sum_pair(p);
        __syncthreads();
        if (lane == 0) s_sum[warp] = p;
        __syncthreads();
        p = s_sum[0];
        for (int w = 1; w < kWarps; ++w) p.add(s_sum[w]);
        return p;
    };
    Pair sum = total(1.0f);
    float s;
    if (sum.hi <= 0x1p126f)
        s = inverse_rms(sum, (float)a.cols, a.eps_hi, a.eps_lo);
    else
        s = __fmul_rn(inverse_rms(total(kDown), (float)a.cols, a.eps_down_hi, 0.0f), kDown);
    float mn = FLT_MAX, mx = -FLT_MAX, bad = 0.0f;
    auto v_at = [&](float h, int k) { return __fmul_rn(__fmul_rn(h, s), __ldg(a.w + k)); };
    for (int k = threadIdx.x; k < a.cols; k += kThreads) {
        const float v = v_at(h_at(k), k);
        mn = fminf(mn, v);
        mx = fmaxf(mx, v);
        bad = __fmaf_rn(v, 0.0f, bad);
    }
    mn = warp_min(mn);
    mx = warp_max(mx);
    const int ok = __all_sync(0xffffffffu, bad == 0.0f);
    if (lane == 0) s_mn[warp] = mn, s_mx[warp] = mx, s_bad[warp] = !ok;
    __syncthreads();
    int any = 0;
    for (int w = 0; w < kWarps; ++w) mn = fminf(mn, s_mn[w]), mx = fmaxf(mx, s_mx[w]), any |= s_bad[w];
    if (any) {
        if (threadIdx.x == 0) record_status(a.status, QNN_ERR_NONFINITE);
        mn = mx = 0.0f;
    }
    const qnn_qparams p = params_from_range(mn, mx);
    const UnitCoder unit(p.Q, p.z);
    int cnt = 0;
    for (int k = threadIdx.x; k < a.cols; k += kThreads) {
        const float h = h_at(k);
        const uint32_t c = unit.code(v_at(h, k));
        cnt += (int)c;
        a.codes[row * a.ldc + k] = (uint8_t)c;
        if (a.h) static_cast<T *>(a.h)[row * a.ldh + k] = from_f32<T>(h);
        if (a.values) a.values[row * a.ldv + k] = __fdiv_rn((float)((int)c + p.z), p.Q);
    }
    cnt = warp_sum(cnt);
    if (lane == 0) s_cnt[warp] = cnt;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kWarps; ++w) cnt += s_cnt[w];
        a.params[row] = p;
        if (a.sums) a.sums[row] = cnt;
    }
}

}  // namespace
}  // namespace qnn

using namespace qnn;

extern "C" qnn_status qnn_rmsnorm_quantize(const void *x, int64_t ldx, const void *residual, int64_t ldr, int dtype,
                                           const float *weight, double eps, int64_t rows, int64_t cols, void *residual_out,
                                           int64_t ldh, uint8_t *codes, int64_t ldc, qnn_qparams *params,
                                           int32_t *code_sums, float *values, int64_t ldv, void *stream) {
    constexpr int64_t kMostCols = 1 << 24, kMostRows = INT32_MAX, kMostLd = (int64_t)1 << 40;
    if (!dtype_ok(dtype) || rows < 0 || rows > kMostRows || cols < 1 || cols > kMostCols || !(eps >= 1e-20 && eps <= 1e20) ||
        ldx < cols || ldx > kMostLd || ldc < cols || ldc > kMostLd || (residual && (ldr < cols || ldr > kMostLd)) ||
        (residual_out && (ldh < cols || ldh > kMostLd)) || (values && (ldv < cols || ldv > kMostLd)))
        return QNN_ERR_INVALID_ARG;
    if (rows == 0) return QNN_OK;
    if (!is_local_ptr(x) || !is_local_ptr(weight) || !is_local_ptr(codes) || !is_local_ptr(params) ||
        (residual && !is_local_ptr(residual)) || (residual_out && !is_local_ptr(residual_out)) ||
        (code_sums && !is_local_ptr(code_sums)) || (values && !is_local_ptr(values)))
        return QNN_ERR_INVALID_ARG;
    const int e = dtype_size(dtype);
    auto aligned = [](const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; };
    if (!aligned(x, e) || !aligned(residual, e) || !aligned(residual_out, e) || !aligned(weight, 4) || !aligned(params, 4) ||
        !aligned(code_sums, 4) || !aligned(values, 4))
        return QNN_ERR_INVALID_ARG;
    auto matrix = [&](const void *p, int64_t ld, int64_t size) { return Span(p, ((rows - 1) * ld + cols) * size); };
    const Span in[3] = {matrix(x, ldx, e), matrix(residual, ldr, e), Span(weight, 4 * cols)};
    const Span out[5] = {matrix(residual_out, ldh, e), matrix(codes, ldc, 1), Span(params, 16 * rows), Span(code_sums, 4 * rows),
                         matrix(values, ldv, 4)};
    for (int o = 0; o < 5; ++o) {
        for (int i = 0; i < 3; ++i) {
            const bool same = o == 0 && ((i == 0 && residual_out == x && ldh == ldx) || (i == 1 && residual_out == residual && ldh == ldr));
            if (!same && out[o].meets(in[i])) return QNN_ERR_INVALID_ARG;
        }
        for (int q = 0; q < o; ++q)
            if (out[o].meets(out[q])) return QNN_ERR_INVALID_ARG;
    }
    NormArgs a;
    a.x = x, a.r = residual, a.h = residual_out, a.w = weight;
    a.rows = rows, a.ldx = ldx, a.ldr = ldr, a.ldh = ldh, a.ldc = ldc, a.ldv = ldv, a.cols = (int)cols;
    a.eps_hi = (float)eps, a.eps_lo = (float)(eps - (double)a.eps_hi), a.eps_down_hi = (float)(eps * 0x1p-160);
    a.codes = codes, a.params = params, a.sums = code_sums, a.values = values;
    QNN_TRY(status_word(&a.status));
    cudaStream_t st = as_stream(stream);
    ProfScope prof("rmsnorm_quantize", st);
    with_type(dtype, [&](auto t) {
        rmsnorm_long_rows_kernel<decltype(t)><<<(unsigned)rows, kThreads, 0, st>>>(a);
    });
    QNN_CUDA_TRY(cudaGetLastError());
    return QNN_OK;
}
