// qgemm4.cu — 4-bit weights in units of `group` columns of a row (Sec. 3.1's sub-matrices, eq. 2 with S = 15) and their
// product with rows of 8-bit activation codes, recovered to fp32 (eq. 1, eq. 3) on sm_103a.
#include <algorithm>

#include "qnn_device.cuh"
#include "qnn_host.h"

namespace qnn {
namespace {

constexpr int kTileRows = 16, kTileCols = 128, kTileBytes = 1024;

__device__ __forceinline__ float unit_scale(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
__device__ __forceinline__ float unit_offset(uint32_t u) { return __uint_as_float(u << 16); }

// A positive fp32 value rounded up to bf16, at least 2^-126.
__device__ __forceinline__ float bf16_up(float v) {
    const uint32_t b = (__float_as_uint(v) + 0xffffu) & 0xffff0000u;
    return __uint_as_float(b < 0x00800000u ? 0x00800000u : b);
}

// A warp a row, 128 columns a step, four columns a lane: the lanes of a group (8, 16 or 32) find its range by shuffles, a
// lane and its neighbour make the 32-bit word of their eight codes. Runs once per weight matrix: 5 bytes read or written a
// weight, short of what memory could do.
template <int GROUP>
__global__ void __launch_bounds__(256) quantize4_kernel(const float *__restrict__ w, int64_t N, int K, int64_t ldw,
                                                        int64_t ktiles, uint8_t *__restrict__ codes, uint32_t *__restrict__ units,
                                                        float *__restrict__ row_sums, int *status) {
    const int64_t n = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), ntile = n / kTileRows;
    const int lane = threadIdx.x & 31, r = (int)(n % kTileRows);
    if (ntile >= (N + kTileRows - 1) / kTileRows) return;
    double sum = 0.0;
    bool bad = false;
    for (int64_t kt = 0; kt < ktiles; ++kt) {
        const int k0 = (int)kt * kTileCols + 4 * lane;
        float v[4], mn = 0.0f, mx = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = n < N && k0 + i < K ? __ldg(w + n * ldw + k0 + i) : 0.0f;
            mn = fminf(mn, v[i]);
            mx = fmaxf(mx, v[i]);
            bad |= !isfinite(v[i]);
        }
#pragma unroll
        for (int o = GROUP / 8; o > 0; o >>= 1) {
            mn = fminf(mn, __shfl_xor_sync(0xffffffffu, mn, o));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        }
        const bool zero = !(mx > mn);
        const float s = zero ? 0.0f : bf16_up(__fsub_rn(__fdiv_rn(mx, 15.0f), __fdiv_rn(mn, 15.0f)));
        const float z = zero ? 0.0f : rintf(__fdiv_rn(mn, s));
        uint32_t word = 0;
        int total = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float q = zero ? 0.0f : fminf(fmaxf(__fsub_rn(rintf(__fdiv_rn(v[i], s)), z), 0.0f), 15.0f);
            const uint32_t c = n < N && k0 + i < K ? (uint32_t)q : 0u;
            if (n < N && k0 + i < K) total += (int)c + (int)z;
            const int e = (4 * lane + i) & 7;  // place of column e of eight: 0 2 4 6 1 3 5 7
            word |= c << (4 * (e / 2 + 4 * (e & 1)));
        }
        word |= __shfl_xor_sync(0xffffffffu, word, 1);
        const int64_t tile = ntile * ktiles + kt;
        if ((lane & 1) == 0)
            *reinterpret_cast<uint32_t *>(codes + tile * kTileBytes + 64 * r + 16 * ((lane & 7) >> 1) + 4 * (lane >> 3)) = word;
        if (4 * lane % GROUP == 0) {
            const uint32_t u = (__float_as_uint(s) & 0xffff0000u) | (__float_as_uint(z == 0.0f ? 0.0f : z) >> 16);
            units[(tile * kTileRows + r) * (kTileCols / GROUP) + 4 * lane / GROUP] = u;
        }
        sum += (double)((float)total * s);  // exact: at most 11 + 8 bits
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0 && n < N) row_sums[n] = (float)sum;
    if (bad) record_status(status, QNN_ERR_NONFINITE);
}

struct Mm4Args {
    const uint8_t *A, *codes;
    const qnn_qparams *pa;
    const uint32_t *units;
    const float *row_sums, *bias;
    float *Y;
    int64_t lda, ldy, M, N;
    int K, ktiles, per_row;
};

// y from the sum t1 over centered codes c = a' - 128: sum (a' + za) w^ = t1 + (128 + za) sum w^, over Qa, plus the bias.
__device__ __forceinline__ float recover4(float t1, const qnn_qparams &p, float row_sum, float bias) {
    return __fadd_rn(__fdiv_rn(__fmaf_rn(__fadd_rn(128.0f, (float)p.z), row_sum, t1), p.Q), bias);
}

// A warp an output, a lane eight columns of every second tile.
template <int GROUP>
__global__ void __launch_bounds__(256) qmatmul4_plain_kernel(const Mm4Args a) {
    const int64_t n = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31, j = (lane >> 2) & 3, t = lane & 3;
    if (n >= a.N) return;
    for (int64_t m = blockIdx.y; m < a.M; m += gridDim.y) {
        float acc = 0.0f;
        for (int kt = lane >> 4; kt < a.ktiles; kt += 2) {
            const int64_t tile = n / kTileRows * a.ktiles + kt;
            const int r = (int)(n % kTileRows);
            const uint32_t word = __ldg(reinterpret_cast<const uint32_t *>(a.codes + tile * kTileBytes + 64 * r + 16 * t + 4 * j));
            const uint32_t u = __ldg(a.units + (tile * kTileRows + r) * (kTileCols / GROUP) + 32 * j / GROUP);
            int p = 0, sum = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int k = kt * kTileCols + 32 * j + 8 * t + e;
                const int c = k < a.K ? (int)__ldg(a.A + m * a.lda + k) - 128 : 0;
                p += c * (int)((word >> (4 * (e / 2 + 4 * (e & 1)))) & 15u);
                sum += c;
            }
            acc = __fmaf_rn(unit_scale(u), __fmaf_rn(unit_offset(u), (float)sum, (float)p), acc);
        }
        acc = warp_sum_f(acc);
        if (lane == 0)
            a.Y[m * a.ldy + n] = recover4(acc, a.pa[a.per_row ? m : 0], a.row_sums[n], a.bias ? a.bias[n] : 0.0f);
    }
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }
bool group_ok(int g) { return g == 32 || g == 64 || g == 128; }

constexpr int64_t kMostN = INT32_MAX / 2, kMostLd = (int64_t)1 << 40;
int64_t tiles_of(int64_t N, int64_t K) { return (N + kTileRows - 1) / kTileRows * ((K + kTileCols - 1) / kTileCols); }

}  // namespace
}  // namespace qnn

using namespace qnn;

extern "C" qnn_status qnn_quantize4(const float *w, int64_t N, int64_t K, int64_t ldw, int32_t group, uint8_t *codes,
                                    uint32_t *units, float *row_sums, void *stream) {
    if (N < 1 || N > kMostN || K < 1 || ldw < K || ldw > kMostLd || !group_ok(group)) return QNN_ERR_INVALID_ARG;
    if (K > QNN_K_MAX) return QNN_ERR_K_TOO_LARGE;
    if (!is_local_ptr(w) || !is_local_ptr(codes) || !is_local_ptr(units) || !is_local_ptr(row_sums) || !aligned4(w) ||
        !aligned16(codes) || !aligned16(units) || !aligned16(row_sums))
        return QNN_ERR_INVALID_ARG;
    const int64_t tiles = tiles_of(N, K);
    const Span in(w, 4 * ((N - 1) * ldw + K));
    const Span out[3] = {Span(codes, tiles * kTileBytes), Span(units, tiles * (kTileRows * kTileCols / group) * 4),
                         Span(row_sums, 4 * N)};
    for (int o = 0; o < 3; ++o) {
        if (out[o].meets(in)) return QNN_ERR_INVALID_ARG;
        for (int q = 0; q < o; ++q)
            if (out[o].meets(out[q])) return QNN_ERR_INVALID_ARG;
    }
    int *status = nullptr;
    QNN_TRY(status_word(&status));
    cudaStream_t st = as_stream(stream);
    ProfScope prof("quantize4", st);
    const auto kern = group == 32 ? quantize4_kernel<32> : group == 64 ? quantize4_kernel<64> : quantize4_kernel<128>;
    const int64_t ntiles = (N + kTileRows - 1) / kTileRows;
    kern<<<(unsigned)(2 * ntiles), 256, 0, st>>>(w, N, (int)K, ldw, (K + kTileCols - 1) / kTileCols, codes, units, row_sums, status);
    QNN_CUDA_TRY(cudaGetLastError());
    return QNN_OK;
}

extern "C" qnn_status qnn_qmatmul4(const uint8_t *A, int64_t lda, const qnn_qparams *pa, int ga, int64_t M, int64_t K,
                                   const uint8_t *codes, const uint32_t *units, int32_t group, const float *row_sums,
                                   int64_t N, const float *bias, float *Y, int64_t ldy, void *stream) {
    if (M < 0 || M > INT32_MAX || N < 1 || N > kMostN || K < 1 || lda < K || lda > kMostLd || ldy < N || ldy > kMostLd ||
        !group_ok(group) || (ga != QNN_PER_MATRIX && ga != QNN_PER_ROW))
        return QNN_ERR_INVALID_ARG;
    if (K > QNN_K_MAX) return QNN_ERR_K_TOO_LARGE;
    if (M == 0) return QNN_OK;
    if (!is_local_ptr(A) || !is_local_ptr(pa) || !is_local_ptr(codes) || !is_local_ptr(units) || !is_local_ptr(row_sums) ||
        (bias && !is_local_ptr(bias)) || !is_local_ptr(Y) || !aligned4(pa) || !aligned16(codes) || !aligned16(units) ||
        !aligned4(row_sums) || !aligned4(bias) || !aligned4(Y))
        return QNN_ERR_INVALID_ARG;
    const int64_t tiles = tiles_of(N, K);
    const Span y(Y, 4 * ((M - 1) * ldy + N));
    if (y.meets(Span(A, (M - 1) * lda + K)) || y.meets(Span(pa, 16 * (ga == QNN_PER_ROW ? M : 1))) ||
        y.meets(Span(codes, tiles * kTileBytes)) || y.meets(Span(units, tiles * (kTileRows * kTileCols / group) * 4)) ||
        y.meets(Span(row_sums, 4 * N)) || y.meets(Span(bias, 4 * N)))
        return QNN_ERR_INVALID_ARG;
    Mm4Args a;
    a.A = A, a.codes = codes, a.pa = pa, a.units = units, a.row_sums = row_sums, a.bias = bias, a.Y = Y;
    a.lda = lda, a.ldy = ldy, a.M = M, a.N = N, a.K = (int)K, a.ktiles = (int)((K + kTileCols - 1) / kTileCols);
    a.per_row = ga == QNN_PER_ROW;
    cudaStream_t st = as_stream(stream);
    ProfScope prof("qmatmul4", st);
    const auto kern = group == 32 ? qmatmul4_plain_kernel<32> : group == 64 ? qmatmul4_plain_kernel<64> : qmatmul4_plain_kernel<128>;
    kern<<<dim3((unsigned)((N + 7) / 8), (unsigned)std::min<int64_t>(M, 65535)), 256, 0, st>>>(a);
    QNN_CUDA_TRY(cudaGetLastError());
    return QNN_OK;
}
