// linattn.cuh — linear attention with a decay for each head over whole sequences on sm_103a, by chunks of frames.
//
// With d = exp(min(log_decay, 0)) and S the state before a chunk's first frame, frames i of the chunk give
//   y_i = scale (d^(i+1) q_i S + sum_{j <= i} d^(i-j) (q_i . k_j) v_j),    S' = d^C S + sum_j d^(C-1-j) k_j v_j^T,
// four matrix products a chunk: scores q k^T, their product with v, q S, and k^T of the scaled v. A block takes 64 columns of v of
// one head and goes over the frames of its part of the sequence chunk by chunk, a warp 16 columns; the next chunk is
// copied while this one is multiplied. The state never leaves the registers: its transpose S^T [16 columns][dk] is the
// accumulator of the last product, and lies in a lane as the first operand of q S wants it.
//
// Numbers. bf16 inputs are operands of bf16 products as they are, and what is held in fp32 is put in as a sum of bf16 pieces of 8
// bits: scores and state in two (2^-17 of each, far below the output's rounding), the scaled v in three (2^-25: the state is kept
// in fp32 and is an output). fp16 and fp32 inputs take products of tf32 (11 bits), where an fp16 value is one piece and an fp32
// one is two, high and low; low times low (2^-22) is left out. All sums are fp32.
#pragma once

#include <algorithm>
#include <type_traits>

#include "elem.cuh"
#include "linattn.h"
#include "tc_ptx.cuh"

namespace qnn {
namespace {

constexpr int kLinThreads = 128, kLinCols = 64;

__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_tf32(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ld_matrix(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr));
}
__device__ __forceinline__ void ld_matrix_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr));
}
// `bytes` of N from global memory, zeros behind them.
template <int N>
__device__ __forceinline__ void copy_async(uint32_t dst, const void *src, int bytes) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(N), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }

// The high halves of two floats as a pair of bf16 (cut off, so that a large value stays finite), and what is left of them.
__device__ __forceinline__ uint32_t high_halves(float x, float y) { return __byte_perm(__float_as_uint(x), __float_as_uint(y), 0x7632); }
__device__ __forceinline__ float below_high(float x) { return __fsub_rn(x, __uint_as_float(__float_as_uint(x) & 0xffff0000u)); }
__device__ __forceinline__ uint32_t rounded_pair(float x, float y) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t *>(&p);
}
__device__ __forceinline__ void pieces2(float x, float y, uint32_t &hi, uint32_t &lo) {
    hi = high_halves(x, y);
    lo = rounded_pair(below_high(x), below_high(y));
}
__device__ __forceinline__ void pieces3(float x, float y, uint32_t &hi, uint32_t &mid, uint32_t &lo) {
    hi = high_halves(x, y);
    const float rx = below_high(x), ry = below_high(y);
    mid = high_halves(rx, ry);
    lo = rounded_pair(below_high(rx), below_high(ry));
}
__device__ __forceinline__ uint32_t tf32_of(float x) {
    uint32_t r;
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(r) : "f"(x));
    return r;
}
// An operand in tf32: the value itself where it is exact, else its two pieces.
struct Tf {
    uint32_t hi, lo;
};
__device__ __forceinline__ Tf tf_split(float x) {
    Tf r;
    r.hi = tf32_of(x);
    r.lo = tf32_of(__fsub_rn(x, __uint_as_float(r.hi)));
    return r;
}
template <bool EXACT>
__device__ __forceinline__ Tf tf_in(float x) {
    if constexpr (EXACT) return {__float_as_uint(x), 0};
    else return tf_split(x);
}

__device__ __forceinline__ float2 two(const float *p) { return *reinterpret_cast<const float2 *>(p); }
__device__ __forceinline__ float2 two(const __half *p) { return __half22float2(*reinterpret_cast<const __half2 *>(p)); }

// exp(rate n), rate <= 0: the product's rounding is put back in. (No arithmetic in 64 bits: this part's units for it are few, and a
// table of these by exp() in 64 bits took 20 us of a launch.)
__device__ __forceinline__ float power(float rate, float n) {
    const float x = __fmul_rn(rate, n), e = expf(x);
    return __fmaf_rn(e, __fmaf_rn(rate, n, -x), e);
}
__device__ __forceinline__ float head_rate(const float *log_decay, int h) {
    const float g = __ldg(log_decay + h);
    // (rates below -200 leave nothing of a state after one frame, as infinite ones do; a NaN stays one)
    return g > 0.0f ? 0.0f : g < -200.0f ? -200.0f : g;
}

template <typename T, int DKP, int C, bool STATES>
struct ChunkShape {
    static constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
    static constexpr int E = sizeof(T), QS = DKP + 8, VS = kLinCols + 8, PS = kBf16 ? C + 8 : C + 4;
    static constexpr int kStage = (C * QS * (STATES ? 1 : 2) + C * VS) * E;
    static constexpr int kScores = STATES ? 0 : kBf16 ? 2 * C * PS * 2 : C * PS * 4;
    static constexpr int kBytes = 2 * kStage + kScores + (C + 1) * 4;
};

// `rows` rows of `cols` values from global memory into rows of WIDTH in shared memory, zeros beyond both.
template <typename T, int C, int WIDTH, int STRIDE, int U>
__device__ __forceinline__ void copy_rows(T *dst, const T *src, int64_t frame, int rows, int cols) {
    constexpr int kPieces = WIDTH * (int)sizeof(T) / U, kValues = U / (int)sizeof(T);
    const uint32_t base = su32(dst);
#pragma unroll 4
    for (int i = threadIdx.x; i < C * kPieces; i += kLinThreads) {
        const int r = i / kPieces, c = i % kPieces * kValues;
        const int some = r < rows ? (cols - c) * (int)sizeof(T) : 0, bytes = some < 0 ? 0 : some > U ? U : some;
        copy_async<U>(base + (r * STRIDE + c) * (int)sizeof(T), bytes ? src + r * frame + c : src, bytes);
    }
}
template <typename T, int C, int WIDTH, int STRIDE>
__device__ __forceinline__ void copy_rows(T *dst, const T *src, int64_t frame, int rows, int cols, int unit) {
    if (unit == 16) {
        copy_rows<T, C, WIDTH, STRIDE, 16>(dst, src, frame, rows, cols);
    } else if (unit == 8) {
        copy_rows<T, C, WIDTH, STRIDE, 8>(dst, src, frame, rows, cols);
    } else if (unit == 4) {
        copy_rows<T, C, WIDTH, STRIDE, 4>(dst, src, frame, rows, cols);
    } else {
        for (int i = threadIdx.x; i < C * WIDTH; i += kLinThreads) {
            const int r = i / WIDTH, c = i % WIDTH;
            dst[r * STRIDE + c] = r < rows && c < cols ? src[r * frame + c] : from_f32<T>(0.0f);
        }
    }
}

template <typename T, int DKP, int C, bool STATES>
__global__ void __launch_bounds__(kLinThreads) linear_chunk_kernel(const LinearArgs a) {
    using Sh = ChunkShape<T, DKP, C, STATES>;
    constexpr bool BF = Sh::kBf16, EXACT = sizeof(T) == 2;
    constexpr int QS = Sh::QS, VS = Sh::VS, PS = Sh::PS, MT = C / 16;
    extern __shared__ __align__(16) unsigned char smem[];
    T *const stage0 = reinterpret_cast<T *>(smem);
    unsigned char *const scores = smem + 2 * Sh::kStage;
    float *const powers = reinterpret_cast<float *>(scores + Sh::kScores);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;

    int64_t at = blockIdx.x;
    const int tile = (int)(at % a.tiles);
    at /= a.tiles;
    const int nparts = STATES ? a.parts - 1 : a.parts;
    const int part = (int)(at % nparts);
    const int64_t unit = at / nparts, b = unit / a.H;
    const int h = (int)(unit % a.H);
    const int64_t n = frames_of(a.lengths, b, a.T), lo = part * a.per, hi = lo + a.per < n ? lo + a.per : n;
    // (a part's state is needed by those behind it that have frames; a part without frames has nothing to do but part 0)
    if (STATES ? lo + a.per >= n : part > 0 && lo >= n) return;
    const float rate = head_rate(a.log_decay, h);
    for (int i = threadIdx.x; i <= C; i += kLinThreads) powers[i] = power(rate, (float)i);

    const int col0 = tile * kLinCols, cols = a.dv - col0 < kLinCols ? a.dv - col0 : kLinCols, wcol = warp * 16;
    const bool works = wcol < cols;
    const T *const q = static_cast<const T *>(a.q) + b * a.q_seq + (int64_t)(h / a.q_share) * a.dk;
    const T *const k = static_cast<const T *>(a.k) + b * a.k_seq + (int64_t)(h / a.k_share) * a.dk;
    const T *const v = static_cast<const T *>(a.v) + b * a.v_seq + (int64_t)(h / a.v_share) * a.dv + col0;

    auto qs = [&](int s) { return stage0 + s * (Sh::kStage / Sh::E); };
    auto ks = [&](int s) { return qs(s) + (STATES ? 0 : C * QS); };
    auto vs = [&](int s) { return ks(s) + C * QS; };
    auto fetch = [&](int64_t at, int s) {
        const int rows = hi - at < C ? (int)(hi - at) : C;
        if constexpr (!STATES) copy_rows<T, C, DKP, QS>(qs(s), q + at * a.q_frame, a.q_frame, rows, a.dk, a.q_copy);
        copy_rows<T, C, DKP, QS>(ks(s), k + at * a.k_frame, a.k_frame, rows, a.dk, a.k_copy);
        copy_rows<T, C, kLinCols, VS>(vs(s), v + at * a.v_frame, a.v_frame, rows, cols, a.v_copy);
        copy_commit();
    };
    if (lo < hi) fetch(lo, 0);

    // S^T: rows (columns of v) g and g + 8, values of dk 8 j + 2 t and the next
    float S[DKP / 8][4];
    auto each_state = [&](auto f) {
#pragma unroll
        for (int j = 0; j < DKP / 8; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = 8 * j + 2 * t + (e & 1), c = wcol + g + 8 * (e >> 1);
                if (r < a.dk && c < cols) f(S[j][e], (int64_t)r * a.dv + col0 + c);
            }
    };
#pragma unroll
    for (int j = 0; j < DKP / 8; ++j) S[j][0] = S[j][1] = S[j][2] = S[j][3] = 0.0f;
    const int64_t size = (int64_t)a.dk * a.dv;
    if constexpr (!STATES) {
        // (another part may write state_out, which may be state_in: only a sequence of one part reads that here)
        const float *p = n > a.per ? a.partial + unit * a.parts * size : a.state_in ? a.state_in + unit * size : nullptr;
        if (p) each_state([&](float &s, int64_t i) { s = p[i]; });
        if (part > 0) {
            const float over = power(rate, (float)a.per);
            for (int j = 0; j < part; ++j) {
                p += size;
                each_state([&](float &s, int64_t i) { s = __fmaf_rn(s, over, p[i]); });
            }
        }
    } else if (part == 0) {
        float *p = a.partial + unit * a.parts * size;
        const float *in = a.state_in + unit * size;
        each_state([&](float &, int64_t i) { p[i] = a.state_in ? in[i] : 0.0f; });
    }

    int s = 0;
    for (int64_t base = lo; base < hi; base += C, s ^= 1) {
        copy_wait();
        __syncthreads();
        if (base + C < hi) fetch(base + C, s ^ 1);
        const int rows = hi - base < C ? (int)(hi - base) : C;
        const T *const Q = qs(s), *const K = ks(s), *const V = vs(s);
        const uint32_t Qa = su32(Q), Ka = su32(K), Va = su32(V);

        // scores of pairs of 16 frames, those of later frames on earlier ones 0, times the decay between them
        if constexpr (!STATES) {
            for (int block = warp; block < MT * (MT + 1) / 2; block += kLinThreads / 32) {
                int r0 = 0, c0 = block;
                while (c0 > r0) c0 -= ++r0;
                r0 *= 16, c0 *= 16;
                float acc[2][4] = {}, rest[2][4] = {};
                if constexpr (BF) {
#pragma unroll
                    for (int k0 = 0; k0 < DKP; k0 += 16) {
                        if (k0 < a.dk) {
                            uint32_t x[4], y[4];
                            ld_matrix(x, Qa + ((r0 + lane % 16) * QS + k0 + lane / 16 * 8) * 2);
                            ld_matrix(y, Ka + ((c0 + lane % 8 + lane / 16 * 8) * QS + k0 + lane / 8 % 2 * 8) * 2);
                            mma_bf16(acc[0], x, y[0], y[1]);
                            mma_bf16(acc[1], x, y[2], y[3]);
                        }
                    }
                } else {
#pragma unroll 4
                    for (int k0 = 0; k0 < DKP; k0 += 8) {
                        if (k0 < a.dk) {
                            const float2 x0 = two(Q + (r0 + g) * QS + k0 + 2 * t), x1 = two(Q + (r0 + g + 8) * QS + k0 + 2 * t);
                            const Tf a0 = tf_in<EXACT>(x0.x), a1 = tf_in<EXACT>(x1.x), a2 = tf_in<EXACT>(x0.y), a3 = tf_in<EXACT>(x1.y);
                            const uint32_t hi4[4] = {a0.hi, a1.hi, a2.hi, a3.hi}, lo4[4] = {a0.lo, a1.lo, a2.lo, a3.lo};
#pragma unroll
                            for (int nt = 0; nt < 2; ++nt) {
                                const float2 y = two(K + (c0 + nt * 8 + g) * QS + k0 + 2 * t);
                                const Tf b0 = tf_in<EXACT>(y.x), b1 = tf_in<EXACT>(y.y);
                                if constexpr (!EXACT) {
                                    mma_tf32(rest[nt], lo4, b0.hi, b1.hi);
                                    mma_tf32(rest[nt], hi4, b0.lo, b1.lo);
                                }
                                mma_tf32(acc[nt], hi4, b0.hi, b1.hi);
                            }
                        }
                    }
                }
                if constexpr (!EXACT) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[i / 4][i % 4] = __fadd_rn(acc[i / 4][i % 4], rest[i / 4][i % 4]);
                }
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int i = r0 + g + 8 * half, j = c0 + nt * 8 + 2 * t;
                        const float x = i >= j ? __fmul_rn(acc[nt][2 * half], powers[i >= j ? i - j : 0]) : 0.0f;
                        const float y = i > j ? __fmul_rn(acc[nt][2 * half + 1], powers[i > j ? i - j - 1 : 0]) : 0.0f;
                        if constexpr (BF) {
                            uint32_t *hi = reinterpret_cast<uint32_t *>(scores) + (i * PS + j) / 2, *lo = hi + C * PS / 2;
                            pieces2(x, y, *hi, *lo);
                        } else {
                            *reinterpret_cast<float2 *>(reinterpret_cast<float *>(scores) + i * PS + j) = make_float2(x, y);
                        }
                    }
            }
            __syncthreads();
        }
        if (!works) continue;

        // the warp's columns of v, a pair of frames of one column a register (bf16)
        uint32_t vf[MT][4];
        bool finite = true;
        if constexpr (BF) {
            uint32_t zero = 0;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                ld_matrix_t(vf[m], Va + ((m * 16 + lane % 16) * VS + wcol + lane / 16 * 8) * 2);
#pragma unroll
                for (int e = 0; e < 4; ++e) asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(zero) : "r"(vf[m][e]), "r"(0u));
            }
            finite = (zero & 0x7fff7fffu) == 0;
        } else {
            float zero = 0.0f;
            for (int i = lane; i < C * 16; i += 32) zero = __fmaf_rn(to_f32(V[i / 16 * VS + wcol + i % 16]), 0.0f, zero);
            finite = zero == 0.0f;
        }
        finite = __all_sync(0xffffffffu, finite);

        if constexpr (!STATES) {
            float y[MT][2][4] = {}, rest[MT][2][4] = {};  // (fp32: products with low pieces apart, see the state)
            // q S
            if constexpr (BF) {
#pragma unroll
                for (int k0 = 0; k0 < DKP; k0 += 16) {
                    if (k0 < a.dk) {
                        const int j = k0 / 8;
                        uint32_t hi[4], lo[4];
                        pieces2(S[j][0], S[j][1], hi[0], lo[0]);
                        pieces2(S[j + 1][0], S[j + 1][1], hi[1], lo[1]);
                        pieces2(S[j][2], S[j][3], hi[2], lo[2]);
                        pieces2(S[j + 1][2], S[j + 1][3], hi[3], lo[3]);
#pragma unroll
                        for (int m = 0; m < MT; ++m) {
                            uint32_t x[4];
                            ld_matrix(x, Qa + ((m * 16 + lane % 16) * QS + k0 + lane / 16 * 8) * 2);
                            mma_bf16(y[m][0], x, lo[0], lo[1]);
                            mma_bf16(y[m][1], x, lo[2], lo[3]);
                            mma_bf16(y[m][0], x, hi[0], hi[1]);
                            mma_bf16(y[m][1], x, hi[2], hi[3]);
                        }
                    }
                }
            } else {
#pragma unroll
                for (int k0 = 0; k0 < DKP; k0 += 8) {
                    if (k0 < a.dk) {
                        Tf sp[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) sp[e] = tf_split(S[k0 / 8][e]);
#pragma unroll
                        for (int m = 0; m < MT; ++m) {
                            const float2 x0 = two(Q + (m * 16 + g) * QS + k0 + 2 * t), x1 = two(Q + (m * 16 + g + 8) * QS + k0 + 2 * t);
                            const Tf a0 = tf_in<EXACT>(x0.x), a1 = tf_in<EXACT>(x1.x), a2 = tf_in<EXACT>(x0.y), a3 = tf_in<EXACT>(x1.y);
                            const uint32_t hi4[4] = {a0.hi, a1.hi, a2.hi, a3.hi}, lo4[4] = {a0.lo, a1.lo, a2.lo, a3.lo};
#pragma unroll
                            for (int nt = 0; nt < 2; ++nt) {
                                if constexpr (!EXACT) mma_tf32(rest[m][nt], lo4, sp[2 * nt].hi, sp[2 * nt + 1].hi);
                                mma_tf32(EXACT ? y[m][nt] : rest[m][nt], hi4, sp[2 * nt].lo, sp[2 * nt + 1].lo);
                                mma_tf32(y[m][nt], hi4, sp[2 * nt].hi, sp[2 * nt + 1].hi);
                            }
                        }
                    }
                }
            }
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (!EXACT) y[m][nt][e] = __fadd_rn(y[m][nt][e], rest[m][nt][e]), rest[m][nt][e] = 0.0f;
                        y[m][nt][e] = __fmul_rn(y[m][nt][e], powers[m * 16 + g + 8 * (e >> 1) + 1]);
                    }
            // scores v. A later frame's score is 0, whose product with an infinity would be a NaN in an earlier frame's output:
            // where a column holds one, the sums are formed frame by frame.
            if (!finite) {
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int i = m * 16 + g + 8 * (e >> 1), c = wcol + nt * 8 + 2 * t + (e & 1);
                            float sum = y[m][nt][e];
                            for (int j = 0; j <= i; ++j) {
                                float p;
                                if constexpr (BF) {
                                    const __nv_bfloat16 *hi = reinterpret_cast<const __nv_bfloat16 *>(scores) + i * PS + j;
                                    p = __fadd_rn(to_f32(hi[0]), to_f32(hi[C * PS]));
                                } else {
                                    p = reinterpret_cast<const float *>(scores)[i * PS + j];
                                }
                                sum = __fmaf_rn(p, to_f32(V[j * VS + c]), sum);
                            }
                            y[m][nt][e] = sum;
                        }
            } else if constexpr (BF) {
                const uint32_t P = su32(scores);
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int j = 0; j <= m; ++j) {
                        uint32_t hi[4], lo[4];
                        const uint32_t p = P + ((m * 16 + lane % 16) * PS + j * 16 + lane / 16 * 8) * 2;
                        ld_matrix(lo, p + C * PS * 2);
                        ld_matrix(hi, p);
                        mma_bf16(y[m][0], lo, vf[j][0], vf[j][1]);
                        mma_bf16(y[m][1], lo, vf[j][2], vf[j][3]);
                        mma_bf16(y[m][0], hi, vf[j][0], vf[j][1]);
                        mma_bf16(y[m][1], hi, vf[j][2], vf[j][3]);
                    }
            } else {
                const float *P = reinterpret_cast<const float *>(scores);
#pragma unroll
                for (int j = 0; j < C; j += 8) {
                    Tf vp[2][2];
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) vp[nt][e] = tf_in<EXACT>(to_f32(V[(j + t + 4 * e) * VS + wcol + nt * 8 + g]));
#pragma unroll
                    for (int m = j / 16; m < MT; ++m) {
                        const float *p = P + (m * 16 + g) * PS + j + t;
                        const Tf a0 = tf_split(p[0]), a1 = tf_split(p[8 * PS]), a2 = tf_split(p[4]), a3 = tf_split(p[8 * PS + 4]);
                        const uint32_t hi4[4] = {a0.hi, a1.hi, a2.hi, a3.hi}, lo4[4] = {a0.lo, a1.lo, a2.lo, a3.lo};
#pragma unroll
                        for (int nt = 0; nt < 2; ++nt) {
                            mma_tf32(EXACT ? y[m][nt] : rest[m][nt], lo4, vp[nt][0].hi, vp[nt][1].hi);
                            if constexpr (!EXACT) mma_tf32(rest[m][nt], hi4, vp[nt][0].lo, vp[nt][1].lo);
                            mma_tf32(y[m][nt], hi4, vp[nt][0].hi, vp[nt][1].hi);
                        }
                    }
                }
                if constexpr (!EXACT) {
#pragma unroll
                    for (int i = 0; i < MT * 8; ++i) y[i / 8][i / 4 % 2][i % 4] = __fadd_rn(y[i / 8][i / 4 % 2][i % 4], rest[i / 8][i / 4 % 2][i % 4]);
                }
            }
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int i = m * 16 + g + 8 * half;
                    if (i < rows) {
                        T *out = static_cast<T *>(a.y) + b * a.y_seq + (base + i) * a.y_frame + (int64_t)h * a.dv + col0;
#pragma unroll
                        for (int nt = 0; nt < 2; ++nt) {
                            const int c = wcol + nt * 8 + 2 * t;
                            const float f[2] = {__fmul_rn(y[m][nt][2 * half], a.scale), __fmul_rn(y[m][nt][2 * half + 1], a.scale)};
                            if (a.pairs && c + 1 < cols) {
                                Run<T, 2> o;
                                o.set(f);
                                o.store(out + c);
                            } else {
                                if (c < cols) out[c] = from_f32<T>(f[0]);
                                if (c + 1 < cols) out[c + 1] = from_f32<T>(f[1]);
                            }
                        }
                    }
                }
        }

        // The state after the chunk. A chunk's products are added up from zero and then to the state: the matrix instruction cuts its
        // sums off (2^-24 of the largest term, always downwards), and a state that went through all of them as their accumulator
        // came out 1e-6 low.
        const float decay = powers[rows];
        auto weight = [&](int frame) { return powers[rows - 1 - frame > 0 ? rows - 1 - frame : 0]; };  // (frames past the last are zeros)
        auto add = [&](int j, const float (&sum)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e) S[j][e] = __fmaf_rn(S[j][e], decay, sum[e]);
        };
        if constexpr (BF) {
            uint32_t hi[MT][4], mid[MT][4], lo[MT][4];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) {  // registers 0 .. 3: frames 2 t, 2 t + 8, and again for 8 columns on
                    const int frame = m * 16 + 2 * t + 8 * (e & 1);
                    const float x = __fmul_rn(__uint_as_float(vf[m][e] << 16), weight(frame));
                    const float z = __fmul_rn(__uint_as_float(vf[m][e] & 0xffff0000u), weight(frame + 1));
                    const int to = e == 1 ? 2 : e == 2 ? 1 : e;  // (operand order: columns before frames)
                    pieces3(x, z, hi[m][to], mid[m][to], lo[m][to]);
                }
#pragma unroll
            for (int n0 = 0; n0 < DKP; n0 += 16) {
                if (n0 < a.dk) {
                    float sum[2][4] = {};
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        uint32_t x[4];
                        ld_matrix_t(x, Ka + ((m * 16 + lane % 16) * QS + n0 + lane / 16 * 8) * 2);
                        mma_bf16(sum[0], lo[m], x[0], x[1]);
                        mma_bf16(sum[1], lo[m], x[2], x[3]);
                        mma_bf16(sum[0], mid[m], x[0], x[1]);
                        mma_bf16(sum[1], mid[m], x[2], x[3]);
                        mma_bf16(sum[0], hi[m], x[0], x[1]);
                        mma_bf16(sum[1], hi[m], x[2], x[3]);
                    }
                    add(n0 / 8, sum[0]);
                    add(n0 / 8 + 1, sum[1]);
                }
            }
        } else {
            Tf x[C / 8][4];
#pragma unroll
            for (int j = 0; j < C; j += 8) {
                const T *p = V + (j + t) * VS + wcol + g;
                const float w0 = weight(j + t), w1 = weight(j + t + 4);
                x[j / 8][0] = tf_split(__fmul_rn(to_f32(p[0]), w0)), x[j / 8][1] = tf_split(__fmul_rn(to_f32(p[8]), w0));
                x[j / 8][2] = tf_split(__fmul_rn(to_f32(p[4 * VS]), w1)), x[j / 8][3] = tf_split(__fmul_rn(to_f32(p[4 * VS + 8]), w1));
            }
#pragma unroll
            for (int n0 = 0; n0 < DKP; n0 += 8) {
                if (n0 < a.dk) {
                    float sum[4] = {}, rest[4] = {};
#pragma unroll
                    for (int j = 0; j < C; j += 8) {
                        const Tf(&v4)[4] = x[j / 8];
                        const uint32_t hi4[4] = {v4[0].hi, v4[1].hi, v4[2].hi, v4[3].hi}, lo4[4] = {v4[0].lo, v4[1].lo, v4[2].lo, v4[3].lo};
                        const Tf b0 = tf_in<EXACT>(to_f32(K[(j + t) * QS + n0 + g])), b1 = tf_in<EXACT>(to_f32(K[(j + t + 4) * QS + n0 + g]));
                        mma_tf32(rest, lo4, b0.hi, b1.hi);
                        if constexpr (!EXACT) mma_tf32(rest, hi4, b0.lo, b1.lo);
                        mma_tf32(sum, hi4, b0.hi, b1.hi);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[e] = __fadd_rn(sum[e], rest[e]);
                    add(n0 / 8, sum);
                }
            }
        }
    }
    if constexpr (STATES) {
        float *p = a.partial + (unit * a.parts + part + 1) * size;
        each_state([&](float &s, int64_t i) { p[i] = s; });
    } else {
        // the part with the sequence's last frame (the first one, for none) has its state
        if (a.state_out && (hi == n || n == 0)) each_state([&](float &s, int64_t i) { a.state_out[unit * size + i] = s; });
    }
}

template <typename T, int DKP, int C, bool STATES>
qnn_status launch_chunk(const LinearArgs &a, cudaStream_t st) {
    using Sh = ChunkShape<T, DKP, C, STATES>;
    static_assert(Sh::kBytes <= 227 * 1024);
    const auto kern = linear_chunk_kernel<T, DKP, C, STATES>;
    QNN_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::kBytes));
    const int64_t blocks = a.B * a.H * a.tiles * (STATES ? a.parts - 1 : a.parts);
    if (blocks > INT32_MAX) return QNN_FAIL(QNN_ERR_INVALID_ARG);
    kern<<<(unsigned)blocks, kLinThreads, Sh::kBytes, st>>>(a);
    QNN_CUDA_TRY(cudaGetLastError());
    return QNN_OK;
}

template <typename T, int DKP, int C>
qnn_status launch_parts(const LinearArgs &a, cudaStream_t st) {
    if (a.parts > 1) QNN_TRY((launch_chunk<T, DKP, C, true>(a, st)));
    return launch_chunk<T, DKP, C, false>(a, st);
}

}  // namespace

template <typename T>
qnn_status launch_linear_chunks(const LinearArgs &a, cudaStream_t st) {
    constexpr int C = sizeof(T) == 4 ? 32 : 64;
    if (a.dk <= 64) return launch_parts<T, 64, C>(a, st);
    if (a.dk <= 128) return launch_parts<T, 128, C>(a, st);
    return launch_parts<T, 256, C / 2>(a, st);
}

}  // namespace qnn
