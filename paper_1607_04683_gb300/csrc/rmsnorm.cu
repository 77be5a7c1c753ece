// rmsnorm.cu — residual addition, root-mean-square norm and the on-the-fly quantizer (Sec. 3, eq. 2) on sm_103a:
// h = x + r; s = 1 / sqrt(mean h^2 + eps); v = (h s) w; one 8-bit unit per row of v.
//
// Every code of a row goes by the last bit of s, so s should hardly ever depend on how the sum is split: the squares are summed
// in pairs of fp32 (value and remainder, to about 2^-44 relative), the root is taken of the pair and rounded once.
//
// Bound: HBM in fp32 (16384 x 2048 with the residual's sum and the recovered values, 571 MB: 89.7 us, 6.4 TB/s; 128000 x 500 161 us,
// 6.8 TB/s), the instructions in 16 bits (bf16, 369 MB, 80 us: some 70 instructions a value, ten of them the exact sum, half
// the bytes).
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
    // The same sum with a remainder of at most half a step of hi. (Additions leave what they round off in lo, which is rounded
    // itself: relative to a sum of n squares by up to n^2 2^-53, so that no more than 16 or 32 are added without this.)
    __device__ __forceinline__ void settle() {
        const float s = __fadd_rn(hi, lo);
        lo = __fsub_rn(lo, __fsub_rn(s, hi));
        hi = s;
    }
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

// The row's scale: s, or s found again at a smaller scale where squares overflow. total(f): the sum of the squares of f h.
template <typename F>
__device__ __forceinline__ float row_scale(const NormArgs &a, F total) {
    const Pair sum = total(1.0f);
    if (sum.hi <= 0x1p126f) return inverse_rms(sum, (float)a.cols, a.eps_hi, a.eps_lo);
    return __fmul_rn(inverse_rms(total(kDown), (float)a.cols, a.eps_down_hi, 0.0f), kDown);
}

// Sums, ranges and counts over the warps of a block, by every warp from shared memory, each on arrays of its own (again: the
// sum's are used for a second time).
struct BlockShare {
    float2 sum[32];
    float mn[32], mx[32];
    int ok[32], count[32];
};
__device__ __forceinline__ Pair block_sum(Pair p, BlockShare &sh, int warps, bool again) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    p = warp_sum_pair(p);
    if (again) __syncthreads();
    if (lane == 0) sh.sum[warp] = make_float2(p.hi, p.lo);
    __syncthreads();
    Pair q;
    if (lane < warps) q.hi = sh.sum[lane].x, q.lo = sh.sum[lane].y;
    return warp_sum_pair(q);
}
// The range over the block; false if a value was not finite.
__device__ __forceinline__ bool block_range(float &mn, float &mx, bool ok, BlockShare &sh, int warps) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    mn = warp_min(mn);
    mx = warp_max(mx);
    ok = __all_sync(0xffffffffu, ok);
    if (lane == 0) sh.mn[warp] = mn, sh.mx[warp] = mx, sh.ok[warp] = ok;
    __syncthreads();
    const int w = lane < warps ? lane : 0;
    mn = warp_min(sh.mn[w]);
    mx = warp_max(sh.mx[w]);
    return __all_sync(0xffffffffu, sh.ok[w] != 0);
}

// Rows held in registers: R runs of V neighbouring values a thread (16 bytes of x each), a warp a row (ROWWARP, several
// rows a block) or a block a row. Every value is read once; the row's two reductions lie between the loads and the stores.
// VEC: all of the call's rows begin on whole runs; otherwise the runs are single values, as many.
constexpr int kNormWarps = 4;  // rows a block, ROWWARP
template <typename T, int RUNS, bool ROWWARP, bool VEC>
__global__ void __launch_bounds__(ROWWARP ? 32 * kNormWarps : 1024) rmsnorm_rows_kernel(const NormArgs a) {
    constexpr int V = VEC ? 16 / (int)sizeof(T) : 1, R = VEC ? RUNS : RUNS * 16 / (int)sizeof(T);
    __shared__ BlockShare sh;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = ROWWARP ? 1 : blockDim.x >> 5;
    const int64_t row = ROWWARP ? (int64_t)blockIdx.x * kNormWarps + warp : blockIdx.x;
    if (row >= a.rows) return;
    const int first = V * (ROWWARP ? lane : (int)threadIdx.x), step = V * 32 * warps;
    auto left = [&](int j) { return a.cols - (first + j * step); };
    float h[R][V], w[R][V];
    {
        const T *x = static_cast<const T *>(a.x) + row * a.ldx + first;
        const T *r = static_cast<const T *>(a.r) + (a.r ? row * a.ldr + first : 0);
        Run<T, V> rx[R], rr[R];
        Run<float, V> rw[R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            if (VEC && left(j) >= V) {
                rx[j].load(x + j * step);
                if (a.r) rr[j].load(r + j * step);
                rw[j].load(a.w + first + j * step);
            } else {
                rx[j].load_some(x + j * step, left(j));
                if (a.r) rr[j].load_some(r + j * step, left(j));
                rw[j].load_some(a.w + first + j * step, left(j));
            }
        }
#pragma unroll
        for (int j = 0; j < R; ++j)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                h[j][v] = rx[j].get(v);
                if (a.r) h[j][v] = __fadd_rn(h[j][v], rr[j].get(v));
                w[j][v] = rw[j].get(v);
            }
    }
    if (a.h) {
        T *out = static_cast<T *>(a.h) + row * a.ldh + first;
#pragma unroll
        for (int j = 0; j < R; ++j) {
            Run<T, V> o;
            o.set(h[j]);
            if (VEC && left(j) >= V)
                o.store(out + j * step);
            else
                o.store_some(out + j * step, left(j));
        }
    }
    const float s = row_scale(a, [&](float scale) {
        Pair p;  // (values past the row's end are 0)
#pragma unroll
        for (int j = 0; j < R; ++j)
#pragma unroll
            for (int v = 0; v < V; ++v) p.add_square(__fmul_rn(h[j][v], scale));
        return ROWWARP ? warp_sum_pair(p) : block_sum(p, sh, warps, scale != 1.0f);
    });
    float mn = FLT_MAX, mx = -FLT_MAX, bad = 0.0f;
#pragma unroll
    for (int j = 0; j < R; ++j)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            h[j][v] = __fmul_rn(__fmul_rn(h[j][v], s), w[j][v]);
            if (v < left(j)) {
                mn = fminf(mn, h[j][v]);
                mx = fmaxf(mx, h[j][v]);
                bad = __fmaf_rn(h[j][v], 0.0f, bad);
            }
        }
    bool ok = bad == 0.0f;
    if (ROWWARP)
        mn = warp_min(mn), mx = warp_max(mx), ok = __all_sync(0xffffffffu, ok);
    else
        ok = block_range(mn, mx, ok, sh, warps);
    if (!ok) {
        if (first == 0) record_status(a.status, QNN_ERR_NONFINITE);
        mn = mx = 0.0f;
    }
    const qnn_qparams p = params_from_range(mn, mx);
    const UnitCoder unit(p.Q, p.z);
    const bool quick = p.Q >= 0x1p-60f && p.Q <= 0x1p60f;  // quotients by the reciprocal, correctly rounded all the same
    const float inv = quick ? rcp_rn(p.Q) : 0.0f;
    int count = 0;
    uint8_t *codes = a.codes + row * a.ldc + first;
    float *values = a.values + (a.values ? row * a.ldv + first : 0);
#pragma unroll
    for (int j = 0; j < R; ++j) {
        uint32_t c[V];
        float q[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            c[v] = unit.code(h[j][v]);
            if (v < left(j)) count += (int)c[v];
        }
        if (VEC && left(j) >= V) {
            uint32_t word[(V + 3) / 4];
#pragma unroll
            for (int k = 0; k < V / 4; ++k) word[k] = c[4 * k] | (c[4 * k + 1] << 8) | (c[4 * k + 2] << 16) | (c[4 * k + 3] << 24);
            if constexpr (V == 8)
                *reinterpret_cast<uint2 *>(codes + j * step) = make_uint2(word[0], word[1]);
            else
                *reinterpret_cast<uint32_t *>(codes + j * step) = word[0];
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (v < left(j)) codes[j * step + v] = (uint8_t)c[v];
        }
        if (a.values) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float k = (float)((int)c[v] + p.z);
                q[v] = quick ? div_by_recip(k, p.Q, inv) : __fdiv_rn(k, p.Q);
            }
            Run<float, V> o;
            o.set(q);
            if (VEC && left(j) >= V)
                o.store(values + j * step);
            else
                o.store_some(values + j * step, left(j));
        }
    }
    count = warp_sum(count);
    if (!ROWWARP) {
        if (lane == 0) sh.count[warp] = count;
        __syncthreads();
        if (warp == 0) count = warp_sum(lane < warps ? sh.count[lane] : 0);
    }
    if (first == 0) {
        a.params[row] = p;
        if (a.sums) a.sums[row] = count;
    }
}

// Rows too long for registers: a row a block, three passes over it (sum of squares, range, codes), h formed again in each.
// Every element is read and written by one thread, and h only in the last pass, so it may take the place of x or r. 300 x 40000
// fp32 36 us, 64 x 2^20 729.
constexpr int kThreads = 1024;
template <typename T>
__global__ void __launch_bounds__(kThreads) rmsnorm_long_rows_kernel(const NormArgs a) {
    __shared__ BlockShare sh;
    const int64_t row = blockIdx.x;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const T *x = static_cast<const T *>(a.x) + row * a.ldx;
    const T *r = a.r ? static_cast<const T *>(a.r) + row * a.ldr : nullptr;
    auto h_at = [&](int k) { return r ? __fadd_rn(to_f32(x[k]), to_f32(r[k])) : to_f32(x[k]); };
    const float s = row_scale(a, [&](float scale) {
        // a thread's squares (up to 2^14) in sums of 16, of 32 of those, of 32 of those: in one sum, of 2^14 equal ones, up to
        // 2^-25 were lost, so 2^-44
        Pair p, p32;
        auto take = [](Pair &to, Pair &from) {
            to.add(from);
            to.settle();
            from = Pair();
        };
        int k = threadIdx.x;
        Pair p16;
        for (int i = 1; k + 15 * kThreads < a.cols; ++i) {
#pragma unroll
            for (int j = 0; j < 16; ++j, k += kThreads) p16.add_square(__fmul_rn(h_at(k), scale));
            take(p32, p16);
            if (i % 32 == 0) take(p, p32);
        }
        for (; k < a.cols; k += kThreads) p16.add_square(__fmul_rn(h_at(k), scale));
        take(p32, p16);
        take(p, p32);
        return block_sum(p, sh, kThreads / 32, scale != 1.0f);
    });
    float mn = FLT_MAX, mx = -FLT_MAX, bad = 0.0f;
    auto v_at = [&](float h, int k) { return __fmul_rn(__fmul_rn(h, s), __ldg(a.w + k)); };
    for (int k = threadIdx.x; k < a.cols; k += kThreads) {
        const float v = v_at(h_at(k), k);
        mn = fminf(mn, v);
        mx = fmaxf(mx, v);
        bad = __fmaf_rn(v, 0.0f, bad);
    }
    if (!block_range(mn, mx, bad == 0.0f, sh, kThreads / 32)) {
        if (threadIdx.x == 0) record_status(a.status, QNN_ERR_NONFINITE);
        mn = mx = 0.0f;
    }
    const qnn_qparams p = params_from_range(mn, mx);
    const UnitCoder unit(p.Q, p.z);
    int count = 0;
    for (int k = threadIdx.x; k < a.cols; k += kThreads) {
        const float h = h_at(k);
        const uint32_t c = unit.code(v_at(h, k));
        count += (int)c;
        a.codes[row * a.ldc + k] = (uint8_t)c;
        if (a.h) static_cast<T *>(a.h)[row * a.ldh + k] = from_f32<T>(h);
        if (a.values) a.values[row * a.ldv + k] = __fdiv_rn((float)((int)c + p.z), p.Q);
    }
    count = warp_sum(count);
    if (lane == 0) sh.count[warp] = count;
    __syncthreads();
    if (warp == 0) count = warp_sum(sh.count[lane]);
    if (threadIdx.x == 0) {
        a.params[row] = p;
        if (a.sums) a.sums[row] = count;
    }
}

template <typename T, int R, bool ROWWARP>
void launch_rows(const NormArgs &a, bool vec, unsigned blocks, int threads, cudaStream_t st) {
    if (vec)
        rmsnorm_rows_kernel<T, R, ROWWARP, true><<<blocks, threads, 0, st>>>(a);
    else
        rmsnorm_rows_kernel<T, R, ROWWARP, false><<<blocks, threads, 0, st>>>(a);
}

template <typename T>
void launch_norm(const NormArgs &a, cudaStream_t st) {
    constexpr int V = 16 / (int)sizeof(T), kMost = 16 / V;  // runs a thread: 16 values
    auto whole = [](const void *p, int64_t ld, int64_t size, uintptr_t bytes) {
        return !p || (reinterpret_cast<uintptr_t>(p) % bytes == 0 && ld * size % (int64_t)bytes == 0);
    };
    const int64_t one = a.rows == 1 ? 0 : 1;  // (a single row has no next one)
    const bool vec = whole(a.x, one * a.ldx, sizeof(T), 16) && whole(a.r, one * a.ldr, sizeof(T), 16) && whole(a.h, one * a.ldh, sizeof(T), 16) &&
                     whole(a.w, 0, 4, 16) && whole(a.codes, one * a.ldc, 1, V) && whole(a.values, one * a.ldv, 4, 16);
    const int runs = (a.cols + V - 1) / V;
    if (runs <= 32 * kMost && a.rows > sm_count() / 2) {
        const unsigned blocks = (unsigned)((a.rows + kNormWarps - 1) / kNormWarps);
        if (runs <= 32)
            launch_rows<T, 1, true>(a, vec, blocks, 32 * kNormWarps, st);
        else if (runs <= 64)
            launch_rows<T, 2, true>(a, vec, blocks, 32 * kNormWarps, st);
        else
            launch_rows<T, kMost, true>(a, vec, blocks, 32 * kNormWarps, st);
    } else if (runs <= 1024 && a.rows <= sm_count()) {  // few rows: as many threads as runs
        launch_rows<T, 1, false>(a, vec, (unsigned)a.rows, (runs + 31) / 32 * 32, st);
    } else if (runs <= 1024 * kMost) {
        launch_rows<T, kMost, false>(a, vec, (unsigned)a.rows, ((runs + kMost - 1) / kMost + 31) / 32 * 32, st);
    } else {
        rmsnorm_long_rows_kernel<T><<<(unsigned)a.rows, kThreads, 0, st>>>(a);
    }
}

}  // namespace
}  // namespace qnn

using namespace qnn;

extern "C" qnn_status qnn_rmsnorm_quantize(const void *x, int64_t ldx, const void *residual, int64_t ldr, int dtype,
                                           const float *weight, double eps, int64_t rows, int64_t cols, void *residual_out,
                                           int64_t ldh, uint8_t *codes, int64_t ldc, qnn_qparams *params,
                                           int32_t *code_sums, float *values, int64_t ldv, void *stream) {
    constexpr int64_t kMostCols = 1 << 24, kMostRows = INT32_MAX, kMostSummed = INT32_MAX / 255;  // (sums of codes are 32 bits)
    auto bad = [&](int64_t ld) { return ld < cols || !reach_ok(rows, ld); };
    if (!dtype_ok(dtype) || rows < 0 || rows > kMostRows || cols < 1 || cols > (code_sums ? kMostSummed : kMostCols) || !(eps >= 1e-20 && eps <= 1e20) ||
        bad(ldx) || bad(ldc) || (residual && bad(ldr)) || (residual_out && bad(ldh)) || (values && bad(ldv)))
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
    with_type(dtype, [&](auto t) { launch_norm<decltype(t)>(a, st); });
    QNN_CUDA_TRY(cudaGetLastError());
    return QNN_OK;
}
