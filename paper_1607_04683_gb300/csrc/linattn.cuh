// linattn.cuh — linear attention with a decay for each head over whole sequences on sm_103a, by chunks of frames.
//
// With d = exp(min(log_decay, 0)) and S the state before a chunk's first frame, frames i of the chunk give
//   y_i = scale (d^(i+1) q_i S + sum_{j <= i} d^(i-j) (q_i . k_j) v_j),    S' = d^C S + sum_j d^(C-1-j) k_j v_j^T,
// four matrix products a chunk: scores q k^T, their product with v, q S, and k^T of the scaled v. A block takes 64 columns of v of
// one head and goes over the frames of its part of the sequence chunk by chunk, a warp 16 columns; the next chunk is
// copied while this one is multiplied. The state never leaves the registers: its transpose S^T [16 columns][dk] is the
// accumulator of the last product, and lies in a lane as the first operand of q S wants it.
//
// Numbers. All products are of bf16 pieces of 8 bits with fp32 sums: a bf16 input is one piece, an fp16 input two, an fp32 input
// three (all exact). What is formed in fp32 is put in as a sum of such pieces: scores and state in two (2^-16 of each, below a
// 16-bit output's rounding; fp32: three), the scaled v in three, all of its 24 bits (the state is kept in fp32 and is an output). Of the products of
// pieces those are taken that the shorter of the two sides' precisions needs: one to three for bf16, four or five for fp16, six for fp32
// (2^-23). (tf32 instructions for fp16 and fp32 took as many, and three times the instructions around them to split operands in
// every warp: 1 x 4000 x 8 x 64 fp32 125 us.)
//
// Bound: a warp's instructions, of which the products are a tenth, and their way into the caches. 1 x 4000 x 8 x 64 fp32, three chunks a part
// and pass: 39 us (states 16, prefix 10, outputs 31 one by one with cold caches); 1 x 1000 x 8 x 64, a chunk a part, 19 us; 16 x 1000 x 16 x 128
// 510 us, fp16 375, bf16 238. Eight warps a block, each half of dk, took 43 us for the first and 690 for the last: v's pieces are made twice.
#pragma once

#include <algorithm>
#include <type_traits>

#include "elem.cuh"
#include "linattn.h"
#include "qnn_device.cuh"
#include "tc_ptx.cuh"

namespace qnn {
namespace {

constexpr int kLinThreads = 128, kLinCols = 64;

__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
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
// Two values as N pieces each, a pair of the first, second, ... of them a word; the last piece is rounded.
template <int N>
__device__ __forceinline__ void split_pair(float x, float y, uint32_t (&p)[N]) {
#pragma unroll
    for (int i = 0; i + 1 < N; ++i) {
        p[i] = high_halves(x, y);
        x = below_high(x), y = below_high(y);
    }
    p[N - 1] = rounded_pair(x, y);
}
__device__ __forceinline__ float low_of(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_of(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// The products (i, j) of A's and B's pieces that count, the smallest first: i + j below the larger number of pieces, and all four of
// two and two (a second piece is up to 2^-7 of its value: without the last product fp16 outputs were up to 2^-14 of their terms off).
template <int A, int B, typename F>
__device__ __forceinline__ void each_product(F f) {
    constexpr int kMost = A == 2 && B == 2 ? 3 : A > B ? A : B;
#pragma unroll
    for (int sum = kMost - 1; sum >= 0; --sum)
#pragma unroll
        for (int i = 0; i <= sum; ++i)
            if (i < A && sum - i < B) f(i, sum - i);
}

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
    static constexpr int kPieces = std::is_same<T, __nv_bfloat16>::value ? 1 : sizeof(T) == 2 ? 2 : 3;
    static constexpr int kHeld = kPieces == 3 ? 3 : 2;  // of a score and of the state
    static constexpr int QS = DKP + 8, VS = kLinCols + 8, PS = C + 8;
    static constexpr int kRows = STATES ? 1 : 2;                                   // q and k, or k
    static constexpr int kPlane = C * (QS * kRows + VS) * 2;                       // a piece of q, k and v
    static constexpr int kRaw = kPieces == 1 ? 0 : C * (DKP * kRows + kLinCols) * (int)sizeof(T);  // them as they were loaded
    static constexpr int kOperands = kPieces == 1 ? 2 * kPlane : kPieces * kPlane + kRaw;
    static constexpr int kScores = STATES ? 0 : kHeld * C * PS * 2;
    static constexpr int kBytes = kOperands + kScores + (C + 1) * 4;
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
// Rows of WIDTH loaded values to N planes of pieces.
template <typename T, int C, int WIDTH, int STRIDE, int N>
__device__ __forceinline__ void split_rows(const T *raw, __nv_bfloat16 *planes, int plane) {
#pragma unroll 2
    for (int i = threadIdx.x; i < C * WIDTH / 8; i += kLinThreads) {
        Run<T, 8> v;
        v.load(raw + i * 8);
        uint32_t w[N][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t p[N];
            split_pair<N>(v.get(2 * e), v.get(2 * e + 1), p);
#pragma unroll
            for (int n = 0; n < N; ++n) w[n][e] = p[n];
        }
        const int to = i * 8 / WIDTH * STRIDE + i * 8 % WIDTH;
#pragma unroll
        for (int n = 0; n < N; ++n) *reinterpret_cast<uint4 *>(planes + n * plane + to) = make_uint4(w[n][0], w[n][1], w[n][2], w[n][3]);
    }
}

template <typename T, int DKP, int C, bool STATES>
__global__ void __launch_bounds__(kLinThreads, DKP == 64 ? 4 : DKP == 128 ? 2 : 1) linear_chunk_kernel(const LinearArgs a) {
    using Sh = ChunkShape<T, DKP, C, STATES>;
    using P16 = __nv_bfloat16;
    constexpr int NP = Sh::kPieces, NH = Sh::kHeld;
    constexpr int QS = Sh::QS, VS = Sh::VS, PS = Sh::PS, MT = C / 16, PLANE = Sh::kPlane / 2;
    extern __shared__ __align__(16) unsigned char smem[];
    P16 *const planes = reinterpret_cast<P16 *>(smem);
    unsigned char *const scores = smem + Sh::kOperands;
    float *const powers = reinterpret_cast<float *>(scores + Sh::kScores);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
    grid_dependents_launch();  // (what follows in the call waits for all of this before it reads any of it)

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

    const int col0 = tile * kLinCols, cols = a.dv - col0 < kLinCols ? a.dv - col0 : kLinCols, wcol = warp * 16;
    const bool works = wcol < cols;
    const T *const q = static_cast<const T *>(a.q) + b * a.q_seq + (int64_t)(h / a.q_share) * a.dk;
    const T *const k = static_cast<const T *>(a.k) + b * a.k_seq + (int64_t)(h / a.k_share) * a.dk;
    const T *const v = static_cast<const T *>(a.v) + b * a.v_seq + (int64_t)(h / a.v_share) * a.dv + col0;

    // bf16: two stages of operands, copied as they are; others: one stage of what was loaded, from which the pieces are made
    constexpr int kVRow = Sh::kRows * C * QS;  // of a plane
    auto fetch = [&](int64_t at, int s) {
        const int rows = hi - at < C ? (int)(hi - at) : C;
        if constexpr (NP == 1) {
            P16 *to = planes + s * PLANE;
            if constexpr (!STATES) copy_rows<T, C, DKP, QS>(to, q + at * a.q_frame, a.q_frame, rows, a.dk, a.q_copy);
            copy_rows<T, C, DKP, QS>(to + (STATES ? 0 : C * QS), k + at * a.k_frame, a.k_frame, rows, a.dk, a.k_copy);
            copy_rows<T, C, kLinCols, VS>(to + kVRow, v + at * a.v_frame, a.v_frame, rows, cols, a.v_copy);
        } else {
            T *to = reinterpret_cast<T *>(smem + NP * Sh::kPlane);
            if constexpr (!STATES) copy_rows<T, C, DKP, DKP>(to, q + at * a.q_frame, a.q_frame, rows, a.dk, a.q_copy);
            copy_rows<T, C, DKP, DKP>(to + (STATES ? 0 : C * DKP), k + at * a.k_frame, a.k_frame, rows, a.dk, a.k_copy);
            copy_rows<T, C, kLinCols, kLinCols>(to + Sh::kRows * C * DKP, v + at * a.v_frame, a.v_frame, rows, cols, a.v_copy);
        }
        copy_commit();
    };
    if (lo < hi) fetch(lo, 0);
    const float rate = head_rate(a.log_decay, h);
    for (int i = threadIdx.x; i <= C; i += kLinThreads) powers[i] = power(rate, (float)i);

    // S^T: rows (columns of v) g and g + 8, values of dk 8 j + 2 t and the next
    float S[DKP / 8][4];
    auto each_state = [&](auto f) {
#pragma unroll
        for (int j = 0; j < DKP / 8; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = 8 * j + 2 * t + (e & 1), c = wcol + g + 8 * (e >> 1);
                if (r < a.dk && c < cols) f(S[j][e], r * a.dv + col0 + c);
            }
    };
#pragma unroll
    for (int j = 0; j < DKP / 8; ++j) S[j][0] = S[j][1] = S[j][2] = S[j][3] = 0.0f;
    const int64_t size = (int64_t)a.dk * a.dv;
    if constexpr (!STATES) {
        // (with parts, the state each begins with: another part may write state_out, which may be state_in)
        if (a.parts > 1) grid_dependency_wait();
        const float *p = a.parts > 1 ? a.partial + (unit * a.parts + part) * size : a.state_in ? a.state_in + unit * size : nullptr;
        if (p) each_state([&](float &s, int i) { s = p[i]; });
    }

    const bool keeps = a.state_out && hi == n;
    int s = 0;
    for (int64_t base = lo; base < hi; base += C, s ^= NP == 1) {
        copy_wait();
        __syncthreads();
        if constexpr (NP == 1) {
            if (base + C < hi) fetch(base + C, s ^ 1);
        } else {
            const T *raw = reinterpret_cast<const T *>(smem + NP * Sh::kPlane);
            split_rows<T, C * Sh::kRows, DKP, QS, NP>(raw, planes, PLANE);
            split_rows<T, C, kLinCols, VS, NP>(raw + Sh::kRows * C * DKP, planes + kVRow, PLANE);
            __syncthreads();
            if (base + C < hi) fetch(base + C, 0);
        }
        const int rows = hi - base < C ? (int)(hi - base) : C;
        const P16 *const Qp = planes + (NP == 1 ? s * PLANE : 0), *const Kp = Qp + (STATES ? 0 : C * QS), *const Vp = Qp + kVRow;
        const uint32_t Qa = su32(Qp), Ka = su32(Kp), Va = su32(Vp);

        // scores of pairs of 16 frames, those of later frames on earlier ones 0, times the decay between them
        if constexpr (!STATES) {
            for (int block = warp; block < MT * (MT + 1) / 2; block += kLinThreads / 32) {
                int r0 = 0, c0 = block;
                while (c0 > r0) c0 -= ++r0;
                r0 *= 16, c0 *= 16;
                float acc[2][2][4] = {};  // (two sums of each, of every other step: a sum's instructions wait for one another)
                const uint32_t qa = Qa + ((r0 + lane % 16) * QS + lane / 16 * 8) * 2;
                const uint32_t ka = Ka + ((c0 + lane % 8 + lane / 16 * 8) * QS + lane / 8 % 2 * 8) * 2;
#pragma unroll
                for (int k0 = 0; k0 < DKP; k0 += 16) {
                    if (k0 < a.dk) {
                        uint32_t x[NP][4], y[NP][4];
#pragma unroll
                        for (int p = 0; p < NP; ++p) {
                            ld_matrix(x[p], qa + (p * PLANE + k0) * 2);
                            ld_matrix(y[p], ka + (p * PLANE + k0) * 2);
                        }
                        each_product<NP, NP>([&](int i, int j) {
                            float(&to)[2][4] = acc[NP == 1 ? k0 / 16 & 1 : i + j > 0];
                            mma_bf16(to[0], x[i], y[j][0], y[j][1]);
                            mma_bf16(to[1], x[i], y[j][2], y[j][3]);
                        });
                    }
                }
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int i = r0 + g + 8 * half, j = c0 + nt * 8 + 2 * t;
                        const float u = __fadd_rn(acc[0][nt][2 * half], acc[1][nt][2 * half]);
                        const float w = __fadd_rn(acc[0][nt][2 * half + 1], acc[1][nt][2 * half + 1]);
                        const float x = i >= j ? __fmul_rn(u, powers[i >= j ? i - j : 0]) : 0.0f;
                        const float y = i > j ? __fmul_rn(w, powers[i > j ? i - j - 1 : 0]) : 0.0f;
                        uint32_t p[NH];
                        split_pair<NH>(x, y, p);
                        uint32_t *to = reinterpret_cast<uint32_t *>(scores) + (i * PS + j) / 2;
#pragma unroll
                        for (int m = 0; m < NH; ++m) to[m * (C * PS / 2)] = p[m];
                    }
            }
            __syncthreads();
        }
        if (!works) continue;

        // the warp's columns of v: registers 0 .. 3 of frames 2 t, 2 t + 8 (pairs), and again for 8 columns on
        uint32_t vf[NP][MT][4];
        uint32_t zero = 0;
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                ld_matrix_t(vf[p][m], Va + (p * PLANE + (m * 16 + lane % 16) * VS + wcol + lane / 16 * 8) * 2);
#pragma unroll
                for (int e = 0; e < 4; ++e) asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(zero) : "r"(vf[p][m][e]), "r"(0u));
            }
        const bool finite = __all_sync(0xffffffffu, (zero & 0x7fff7fffu) == 0);

        if constexpr (!STATES) {
            float y[MT][2][4] = {}, rest[NP == 3 ? MT : 1][2][4] = {};  // (fp32: products of second and third pieces apart, see the state)
            // q S
            const uint32_t qa = Qa + (lane % 16 * QS + lane / 16 * 8) * 2;
#pragma unroll
            for (int k0 = 0; k0 < DKP; k0 += 16) {
                if (k0 < a.dk) {
                    const int j = k0 / 8;
                    uint32_t sp[4][NH], x[MT][NP][4];
                    split_pair<NH>(S[j][0], S[j][1], sp[0]);
                    split_pair<NH>(S[j + 1][0], S[j + 1][1], sp[1]);
                    split_pair<NH>(S[j][2], S[j][3], sp[2]);
                    split_pair<NH>(S[j + 1][2], S[j + 1][3], sp[3]);
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int p = 0; p < NP; ++p) ld_matrix(x[m][p], qa + (p * PLANE + m * 16 * QS + k0) * 2);
                    each_product<NP, NH>([&](int i, int j) {
#pragma unroll
                        for (int m = 0; m < MT; ++m) {
                            float(&to)[2][4] = NP == 3 && i + j > 0 ? rest[NP == 3 ? m : 0] : y[m];
                            mma_bf16(to[0], x[m][i], sp[0][j], sp[1][j]);
                            mma_bf16(to[1], x[m][i], sp[2][j], sp[3][j]);
                        }
                    });
                }
            }
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (NP == 3) y[m][nt][e] = __fadd_rn(y[m][nt][e], rest[m][nt][e]), rest[m][nt][e] = 0.0f;
                        y[m][nt][e] = __fmul_rn(y[m][nt][e], powers[m * 16 + g + 8 * (e >> 1) + 1]);
                    }
            // scores v. A later frame's score is 0, whose product with an infinity would be a NaN in an earlier frame's output:
            // where a column holds one, the sums are formed frame by frame.
            if (!finite) {
                const P16 *p = reinterpret_cast<const P16 *>(scores);
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int i = m * 16 + g + 8 * (e >> 1), c = wcol + nt * 8 + 2 * t + (e & 1);
                            float sum = y[m][nt][e];
                            for (int j = 0; j <= i; ++j) {
                                float u = 0.0f, w = 0.0f;
                                for (int r = NH - 1; r >= 0; --r) u = __fadd_rn(u, to_f32(p[r * C * PS + i * PS + j]));
                                for (int r = NP - 1; r >= 0; --r) w = __fadd_rn(w, to_f32(Vp[r * PLANE + j * VS + c]));
                                sum = __fmaf_rn(u, w, sum);
                            }
                            y[m][nt][e] = sum;
                        }
            } else {
                const uint32_t pa = su32(scores) + (lane % 16 * PS + lane / 16 * 8) * 2;
#pragma unroll
                for (int j = 0; j < MT; ++j) {
                    uint32_t x[MT][NH][4];
#pragma unroll
                    for (int m = j; m < MT; ++m)
#pragma unroll
                        for (int p = 0; p < NH; ++p) ld_matrix(x[m][p], pa + (p * C * PS + m * 16 * PS + j * 16) * 2);
                    each_product<NH, NP>([&](int i, int p) {
#pragma unroll
                        for (int m = j; m < MT; ++m) {
                            float(&to)[2][4] = NP == 3 && i + p > 0 ? rest[NP == 3 ? m : 0] : y[m];
                            mma_bf16(to[0], x[m][i], vf[p][j][0], vf[p][j][1]);
                            mma_bf16(to[1], x[m][i], vf[p][j][2], vf[p][j][3]);
                        }
                    });
                }
                if constexpr (NP == 3) {
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[m][e / 4][e % 4] = __fadd_rn(y[m][e / 4][e % 4], rest[m][e / 4][e % 4]);
                }
            }
            T *const out = static_cast<T *>(a.y) + b * a.y_seq + (base + g) * a.y_frame + (int64_t)h * a.dv + col0;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int i = m * 16 + 8 * half;
                    if (i + g < rows) {
                        T *o = out + i * a.y_frame;
#pragma unroll
                        for (int nt = 0; nt < 2; ++nt) {
                            const int c = wcol + nt * 8 + 2 * t;
                            const float f[2] = {__fmul_rn(y[m][nt][2 * half], a.scale), __fmul_rn(y[m][nt][2 * half + 1], a.scale)};
                            if (a.pairs && c + 1 < cols) {
                                Run<T, 2> r;
                                r.set(f);
                                r.store(o + c);
                            } else {
                                if (c < cols) o[c] = from_f32<T>(f[0]);
                                if (c + 1 < cols) o[c + 1] = from_f32<T>(f[1]);
                            }
                        }
                    }
                }
        }

        if (!STATES && base + C >= hi && !keeps) break;  // (a part's last state is another's first, which the prefix has formed)

        // The state after the chunk. A chunk's products are added up from zero and then to the state: the matrix instruction cuts its
        // sums off (2^-24 of the largest term, always downwards), and a state that went through all of them as their accumulator
        // came out 1e-6 low. For the same reason products of small pieces have a sum of their own.
        const float decay = powers[rows];
        auto weight = [&](int frame) { return powers[rows - 1 - frame > 0 ? rows - 1 - frame : 0]; };  // (frames past the last are zeros)
        uint32_t vp[MT][3][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int frame = m * 16 + 2 * t + 8 * (e & 1);
                float x = low_of(vf[NP - 1][m][e]), z = high_of(vf[NP - 1][m][e]);
#pragma unroll
                for (int p = NP - 2; p >= 0; --p) x = __fadd_rn(x, low_of(vf[p][m][e])), z = __fadd_rn(z, high_of(vf[p][m][e]));
                uint32_t p3[3];
                split_pair<3>(__fmul_rn(x, weight(frame)), __fmul_rn(z, weight(frame + 1)), p3);
                const int to = e == 1 ? 2 : e == 2 ? 1 : e;  // (operand order: columns before frames)
                vp[m][0][to] = p3[0], vp[m][1][to] = p3[1], vp[m][2][to] = p3[2];
            }
        const uint32_t ka = Ka + (lane % 16 * QS + lane / 16 * 8) * 2;
#pragma unroll
        for (int n0 = 0; n0 < DKP; n0 += 32) {
            if (n0 < a.dk) {
                float sum[4][4] = {}, rest[NP > 1 ? 4 : 1][4] = {};
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    uint32_t x[NP][2][4];
#pragma unroll
                    for (int p = 0; p < NP; ++p) {
                        ld_matrix_t(x[p][0], ka + (p * PLANE + m * 16 * QS + n0) * 2);
                        ld_matrix_t(x[p][1], ka + (p * PLANE + m * 16 * QS + n0 + 16) * 2);
                    }
                    each_product<3, NP>([&](int i, int p) {
                        const bool small = NP > 1 && i + p > 0;
                        mma_bf16(small ? rest[0] : sum[0], vp[m][i], x[p][0][0], x[p][0][1]);
                        mma_bf16(small ? rest[NP > 1 ? 1 : 0] : sum[1], vp[m][i], x[p][0][2], x[p][0][3]);
                        mma_bf16(small ? rest[NP > 1 ? 2 : 0] : sum[2], vp[m][i], x[p][1][0], x[p][1][1]);
                        mma_bf16(small ? rest[NP > 1 ? 3 : 0] : sum[3], vp[m][i], x[p][1][2], x[p][1][3]);
                    });
                }
                if constexpr (NP > 1) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) sum[e / 4][e % 4] = __fadd_rn(sum[e / 4][e % 4], rest[e / 4][e % 4]);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) S[n0 / 8 + j][e] = __fmaf_rn(S[n0 / 8 + j][e], decay, sum[j][e]);
            }
        }
    }
    if constexpr (STATES) {
        float *p = a.partial + (unit * a.parts + part) * size;
        each_state([&](float &s, int i) { p[i] = s; });
    } else {
        // the part with the sequence's last frame (the first one, for none) has its state
        if (keeps || (a.state_out && n == 0)) {
            float *p = a.state_out + unit * size;
            each_state([&](float &s, int i) { p[i] = s; });
        }
    }
}

// From the states that the parts of a sequence end with from zeros, those that they begin with, in their place: a thread an element,
// kAhead parts loaded at a time (42 parts of 8 states of 64 x 64: 7.5 to 10 us). (Of parts without frames nothing is used.)
constexpr int kPrefixThreads = 256, kAhead = 16;
__global__ void __launch_bounds__(kPrefixThreads) linear_prefix_kernel(const LinearArgs a) {
    grid_dependents_launch();
    const int64_t size = (int64_t)a.dk * a.dv;
    const Split at = split((int64_t)blockIdx.x * kPrefixThreads + threadIdx.x, size);
    const int64_t unit = at.quot;
    if (unit >= a.B * a.H) return;
    const float over = power(head_rate(a.log_decay, (int)(unit % a.H)), (float)a.per);
    float run = a.state_in ? a.state_in[unit * size + at.rem] : 0.0f;
    float *p = a.partial + unit * a.parts * size + at.rem;
    grid_dependency_wait();
    for (int j0 = 0; j0 < a.parts; j0 += kAhead) {
        float v[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) v[j] = j0 + j + 1 < a.parts ? p[(j0 + j) * size] : 0.0f;
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (j0 + j < a.parts) {
                p[(j0 + j) * size] = run;
                run = __fmaf_rn(run, over, v[j]);
            }
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
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(kLinThreads);
    cfg.dynamicSmemBytes = Sh::kBytes;
    cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = !STATES && a.parts > 1 ? 1 : 0;
    QNN_CUDA_TRY(cudaLaunchKernelEx(&cfg, kern, a));
    return QNN_OK;
}

template <typename T, int DKP, int C>
qnn_status launch_parts(const LinearArgs &a, cudaStream_t st) {
    if (a.parts > 1) {
        QNN_TRY((launch_chunk<T, DKP, C, true>(a, st)));
        const int64_t blocks = (a.B * a.H * a.dk * a.dv + kPrefixThreads - 1) / kPrefixThreads;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)blocks);
        cfg.blockDim = dim3(kPrefixThreads);
        cfg.stream = st;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr.val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        QNN_CUDA_TRY(cudaLaunchKernelEx(&cfg, linear_prefix_kernel, a));
    }
    return launch_chunk<T, DKP, C, false>(a, st);
}

}  // namespace

template <typename T>
qnn_status launch_linear_chunks(const LinearArgs &a, cudaStream_t st) {
    constexpr int C = std::is_same<T, __nv_bfloat16>::value ? 64 : 32;
    if (a.dk <= 64) return launch_parts<T, 64, C>(a, st);
    if (a.dk <= 128) return launch_parts<T, 128, C>(a, st);
    return launch_parts<T, 256, C / 2>(a, st);
}

}  // namespace qnn
