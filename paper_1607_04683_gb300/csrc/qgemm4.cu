// qgemm4.cu — 4-bit weights in units of `group` columns of a row (Sec. 3.1's sub-matrices, eq. 2 with S = 15) and their
// product with rows of 8-bit activation codes, recovered to fp32 (eq. 1, eq. 3) on sm_103a.
#include <algorithm>

#include <cuda_fp16.h>

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
    int segments;     // warps that share a row tile's columns; the block's other warps take other row tiles
    int64_t items;    // blocks' shares of row tiles
    int chunk, stride;  // column tiles of A in shared memory at once, bytes of a row of them
    int align;        // of A's rows, 16, 4 or 1
};

// y from the sum t1 over centered codes c = a' - 128: sum (a' + za) w^ = t1 + (128 + za) sum w^, over Qa, plus the bias.
__device__ __forceinline__ float recover4(float t1, float Q, float z, float row_sum, float bias) {
    return __fadd_rn(__fdiv_rn(__fmaf_rn(__fadd_rn(128.0f, z), row_sum, t1), Q), bias);
}

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Two fp16 values x m + c.
__device__ __forceinline__ uint32_t hfma2_bits(uint32_t x, uint32_t m, uint32_t c) {
    uint32_t d;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(x), "r"(m), "r"(c));
    return d;
}
__device__ __forceinline__ uint32_t both(float v) { return __half_as_ushort(__float2half_rn(v)) * 0x10001u; }

// The products run on the fp16 tensor-core instruction, exactly, on codes that cost next to nothing to convert:
//   - a 4-bit code masked out of its word in place is a subnormal fp16 number, code 2^-24 in a half's lowest four bits and
//     16 code 2^-24 in the next four (0x000f000f and 0x00f000f0 give two of a word's eight columns each; one shift gives the
//     other four);
//   - an 8-bit code b under the byte 0x64 is the fp16 number 1024 + b, from which one multiply-add makes 16 (b - 128) for
//     columns whose weights count once and b - 128 for those that count 16 times.
// So every product is (b - 128) code 2^-20, and a group's sum, below 2^24 of that unit, is exact in fp32. The sum of a
// group starts from offset x (sum of b - 128) and is taken into the output's sum by its scale, in fp32.
//
// A block's 16 warps split the columns of its row tiles (each of the `segments` a part of every stretch of as many tiles, so
// that a block reads long contiguous stretches) and add up through shared memory at the end, in a fixed order. RT row tiles
// a warp share the converted activations. Bound: the weights' bytes; the loads of the next column tile are in flight
// while one is worked on.
constexpr int kMmThreads = 512, kMmWarps = kMmThreads / 32, kRedStride = 20;
constexpr float kUnit = 0x1p-20f, kPerUnit = 0x1p20f;

template <int GROUP>
struct Units {  // of a row's 128 columns
    static constexpr int kCount = kTileCols / GROUP;
    uint32_t u[kCount];
    __device__ __forceinline__ void load(const uint32_t *p) {
        if constexpr (kCount == 4) {
            const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p));
            u[0] = v.x, u[1] = v.y, u[2] = v.z, u[3] = v.w;
        } else if constexpr (kCount == 2) {
            const uint2 v = __ldg(reinterpret_cast<const uint2 *>(p));
            u[0] = v.x, u[1] = v.y;
        } else {
            u[0] = __ldg(p);
        }
    }
};

template <int GROUP, int NT, int RT>
__global__ void __launch_bounds__(kMmThreads, 1) qmatmul4_kernel(const Mm4Args a) {
    extern __shared__ __align__(16) uint8_t smem[];
    constexpr int kRows = 8 * NT, kGroups = kTileCols / GROUP;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int64_t m0 = (int64_t)blockIdx.y * kRows;
    const int rows = (int)min((int64_t)kRows, a.M - m0);
    uint8_t *sA = smem;                                              // [rows][stride]
    float *sR = reinterpret_cast<float *>(sA + rows * a.stride);     // [chunk groups][kRows]: group sums of b - 128
    float *red = sR + a.chunk * kGroups * kRows;                     // [warps][RT][kRows][kRedStride]
    const int seg = warp % a.segments, tile_group = warp / a.segments, tile_groups = kMmWarps / a.segments;
    const int64_t ntiles = (a.N + kTileRows - 1) / kTileRows;
    const int chunks = (a.ktiles + a.chunk - 1) / a.chunk;

    struct Tile {
        uint4 w[RT][2];
        Units<GROUP> u[RT][2];
    };
    for (int64_t item = blockIdx.x; item < a.items; item += gridDim.x) {
        const int64_t tile0 = (item * tile_groups + tile_group) * RT;
        auto load = [&](Tile &x, int kt, int end) {
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                if (kt < end && tile0 + r < ntiles) {
                    const int64_t at = (tile0 + r) * a.ktiles + kt;
                    const uint4 *p = reinterpret_cast<const uint4 *>(a.codes + at * kTileBytes) + lane;
                    x.w[r][0] = __ldg(p), x.w[r][1] = __ldg(p + 32);
                    const uint32_t *q = a.units + (at * kTileRows + g) * kGroups;
                    x.u[r][0].load(q), x.u[r][1].load(q + 8 * kGroups);
                }
            }
        };
        float acc[RT][NT][4] = {};
        for (int chunk = 0; chunk < chunks; ++chunk) {
            const int kt0 = chunk * a.chunk, kt1 = min(a.ktiles, kt0 + a.chunk);
            Tile next;
            load(next, kt0 + seg, kt1);
            if (chunks > 1 || item == blockIdx.x) {
                if (chunk > 0 || item != blockIdx.x) __syncthreads();  // all warps are done with what was there
                // A's codes, 16 a step; past K, 128, which counts 0
                const int blocks = (kt1 - kt0) * (kTileCols / 16);
                for (int i = tid; i < rows * blocks; i += kMmThreads) {
                    const int m = i / blocks, k = kt0 * kTileCols + 16 * (i % blocks);
                    const uint8_t *p = a.A + (m0 + m) * a.lda + k;
                    uint32_t v[4];
                    if (a.align == 16 && k + 16 <= a.K) {
                        const uint4 x = __ldg(reinterpret_cast<const uint4 *>(p));
                        v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if (a.align >= 4 && k + 4 * j + 4 <= a.K) {
                                v[j] = __ldg(reinterpret_cast<const uint32_t *>(p + 4 * j));
                            } else {
                                v[j] = 0;
#pragma unroll
                                for (int e = 0; e < 4; ++e) v[j] |= (uint32_t)(k + 4 * j + e < a.K ? __ldg(p + 4 * j + e) : 128) << (8 * e);
                            }
                        }
                    }
                    *reinterpret_cast<uint4 *>(sA + m * a.stride + 16 * (i % blocks)) = make_uint4(v[0], v[1], v[2], v[3]);
                }
                __syncthreads();
                const int groups = (kt1 - kt0) * kGroups;
                for (int i = tid; i < kRows * groups; i += kMmThreads) {
                    const int m = i / groups, q = i % groups;
                    int sum = 0;
                    if (m < rows) {
                        const uint4 *p = reinterpret_cast<const uint4 *>(sA + m * a.stride + q * GROUP);
#pragma unroll
                        for (int j = 0; j < GROUP / 16; ++j) {
                            const uint4 v = p[j];
                            sum = (int)__dp4a(v.x, 0x01010101u, (uint32_t)sum), sum = (int)__dp4a(v.y, 0x01010101u, (uint32_t)sum);
                            sum = (int)__dp4a(v.z, 0x01010101u, (uint32_t)sum), sum = (int)__dp4a(v.w, 0x01010101u, (uint32_t)sum);
                        }
                        sum -= 128 * GROUP;
                    }
                    sR[q * kRows + m] = (float)sum * kUnit;
                }
                __syncthreads();
            }
            const uint8_t *pa = sA + g * a.stride + 8 * t;
            for (int kt = kt0 + seg; kt < kt1; kt += a.segments) {
                const Tile now = next;
                load(next, kt + a.segments, kt1);
                float sum[RT][NT][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (j * 32 % GROUP == 0) {  // a group begins: offset x (sum of its b - 128)
                        const float2 *R = reinterpret_cast<const float2 *>(sR + ((kt - kt0) * kGroups + j * 32 / GROUP) * kRows) + t;
#pragma unroll
                        for (int c = 0; c < NT; ++c) {
                            const float2 v = R[4 * c];
#pragma unroll
                            for (int r = 0; r < RT; ++r) {
                                const float z0 = unit_offset(now.u[r][0].u[j * 32 / GROUP]), z1 = unit_offset(now.u[r][1].u[j * 32 / GROUP]);
                                sum[r][c][0] = __fmul_rn(z0, v.x), sum[r][c][1] = __fmul_rn(z0, v.y);
                                sum[r][c][2] = __fmul_rn(z1, v.x), sum[r][c][3] = __fmul_rn(z1, v.y);
                            }
                        }
                    }
                    uint32_t wa[RT][4], wb[RT][4];
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        const uint32_t *w0 = &now.w[r][0].x, *w1 = &now.w[r][1].x;
                        const uint32_t x = w0[j], y = w1[j], x8 = x >> 8, y8 = y >> 8;
                        wa[r][0] = x & 0x000f000fu, wa[r][1] = y & 0x000f000fu, wa[r][2] = x & 0x00f000f0u, wa[r][3] = y & 0x00f000f0u;
                        wb[r][0] = x8 & 0x000f000fu, wb[r][1] = y8 & 0x000f000fu, wb[r][2] = x8 & 0x00f000f0u, wb[r][3] = y8 & 0x00f000f0u;
                    }
#pragma unroll
                    for (int c = 0; c < NT; ++c) {
                        uint2 v = make_uint2(0x80808080u, 0x80808080u);
                        if (8 * c + g < rows)
                            v = *reinterpret_cast<const uint2 *>(pa + 8 * c * a.stride + (kt - kt0) * kTileCols + 32 * j);
                        const uint32_t one = both(1.0f), six = both(16.0f), cone = both(-1152.0f), csix = both(-18432.0f);
                        const uint32_t b0 = hfma2_bits(__byte_perm(v.x, 0x64646464u, 0x4140), six, csix);
                        const uint32_t b1 = hfma2_bits(__byte_perm(v.x, 0x64646464u, 0x4342), one, cone);
                        const uint32_t b2 = hfma2_bits(__byte_perm(v.y, 0x64646464u, 0x4140), six, csix);
                        const uint32_t b3 = hfma2_bits(__byte_perm(v.y, 0x64646464u, 0x4342), one, cone);
#pragma unroll
                        for (int r = 0; r < RT; ++r) {
                            mma_f16(sum[r][c], wa[r], b0, b1);
                            mma_f16(sum[r][c], wb[r], b2, b3);
                        }
                    }
                    if ((j + 1) * 32 % GROUP == 0) {  // and ends
#pragma unroll
                        for (int r = 0; r < RT; ++r) {
                            const float s0 = unit_scale(now.u[r][0].u[j * 32 / GROUP]), s1 = unit_scale(now.u[r][1].u[j * 32 / GROUP]);
#pragma unroll
                            for (int c = 0; c < NT; ++c) {
                                acc[r][c][0] = __fmaf_rn(s0, sum[r][c][0], acc[r][c][0]);
                                acc[r][c][1] = __fmaf_rn(s0, sum[r][c][1], acc[r][c][1]);
                                acc[r][c][2] = __fmaf_rn(s1, sum[r][c][2], acc[r][c][2]);
                                acc[r][c][3] = __fmaf_rn(s1, sum[r][c][3], acc[r][c][3]);
                            }
                        }
                    }
                }
            }
        }
        // the segments' sums, in order
        if (item != blockIdx.x) __syncthreads();  // the item before is out
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                float *p = red + ((warp * RT + r) * kRows + 8 * c + 2 * t) * kRedStride + g;
                p[0] = acc[r][c][0], p[kRedStride] = acc[r][c][1];
                p[8] = acc[r][c][2], p[kRedStride + 8] = acc[r][c][3];
            }
        __syncthreads();
        const int wide = tile_groups * RT * kTileRows;
        for (int i = tid; i < wide * rows; i += kMmThreads) {
            const int m = i / wide, col = i % wide, tg = col / (RT * kTileRows), r = col / kTileRows % RT, row = col % kTileRows;
            const int64_t n = item * wide + col;
            if (n >= a.N) continue;
            const qnn_qparams p = a.pa[a.per_row ? m0 + m : 0];
            const float row_sum = __ldg(a.row_sums + n), bias = a.bias ? __ldg(a.bias + n) : 0.0f;
            float sum = 0.0f;
            for (int k = 0; k < a.segments; ++k)
                sum = __fadd_rn(sum, red[(((tg * a.segments + k) * RT + r) * kRows + m) * kRedStride + row]);
            a.Y[(m0 + m) * a.ldy + n] = recover4(__fmul_rn(sum, kPerUnit), p.Q, (float)p.z, row_sum, bias);
        }
    }
}

template <int GROUP, int NT, int RT>
qnn_status launch_mm4(Mm4Args a, cudaStream_t st) {
    constexpr int kRows = 8 * NT;
    const int64_t ntiles = (a.N + kTileRows - 1) / kTileRows;
    a.segments = 1;
    while (a.segments < kMmWarps && a.segments < a.ktiles) a.segments *= 2;
    const int64_t per_item = (int64_t)kMmWarps / a.segments * RT;
    a.items = (ntiles + per_item - 1) / per_item;
    // shared memory: the sums of all warps, and as many column tiles of A (codes and group sums) as fit beside them
    constexpr size_t kMost = 220 * 1024, kRed = (size_t)kMmWarps * RT * kRows * kRedStride * 4;
    const int rows = (int)std::min<int64_t>(kRows, a.M);
    const size_t per_tile = (size_t)rows * kTileCols + (size_t)(kTileCols / GROUP) * kRows * 4;
    a.chunk = (int)std::min<int64_t>(a.ktiles, (int64_t)((kMost - kRed - (size_t)rows * 32) / per_tile));
    a.stride = a.chunk * kTileCols + 32;
    const size_t bytes = kRed + (size_t)rows * a.stride + (size_t)a.chunk * (kTileCols / GROUP) * kRows * 4;
    const auto kern = qmatmul4_kernel<GROUP, NT, RT>;
    if (bytes > 48 * 1024) QNN_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    const int64_t mblocks = (a.M + kRows - 1) / kRows;
    if (mblocks > 65535) return QNN_FAIL(QNN_ERR_INVALID_ARG);
    kern<<<dim3((unsigned)std::min<int64_t>(a.items, sm_count()), (unsigned)mblocks), kMmThreads, bytes, st>>>(a);
    QNN_CUDA_TRY(cudaGetLastError());
    return QNN_OK;
}

template <int GROUP>
qnn_status launch_mm4(const Mm4Args &a, cudaStream_t st) {
    const int64_t ntiles = (a.N + kTileRows - 1) / kTileRows;
    const bool two = ntiles > sm_count();
    if (a.M <= 8) return two ? launch_mm4<GROUP, 1, 2>(a, st) : launch_mm4<GROUP, 1, 1>(a, st);
    if (a.M <= 16) return two ? launch_mm4<GROUP, 2, 2>(a, st) : launch_mm4<GROUP, 2, 1>(a, st);
    return launch_mm4<GROUP, 4, 1>(a, st);  // (two row tiles a warp do not fit its registers)
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
    a.align = (reinterpret_cast<uintptr_t>(A) | (uintptr_t)lda) % 16 == 0 ? 16 : (reinterpret_cast<uintptr_t>(A) | (uintptr_t)lda) % 4 == 0 ? 4 : 1;
    return group == 32 ? launch_mm4<32>(a, st) : group == 64 ? launch_mm4<64>(a, st) : launch_mm4<128>(a, st);
}
