// linattn_tc.cu — linear attention with a decay for each head over long bf16 sequences, on the tcgen05 tensor cores.
//
// The chunk's products of linattn.cuh with chunks of 128 frames, for 64 columns of v of one head:
//   QK: scores = q k^T;  KV: D = k^T (v scaled);  PV: A = scores v;  QS: B = q S;  y_i = scale (A_i + d^(i+1) B_i),  S' = d^128 S + D.
// One block an SM goes through (sequence, head, columns) after another as one stream of chunks; its warps have parts of their own:
//   warps 0 - 7    scores from tensor memory, times their decays, back into it as pairs of bf16 pieces; outputs;
//   warps 8 - 11   the state, a row of 64 columns a thread in registers, and its two bf16 pieces for QS;
//   warps 12 - 15  v times its decays in three pieces (two buffers: the last piece first, and the middle one in its place);
//   warp 16        issues the products, in the order KV, PV, QS and the next chunk's QK;
//   warp 17        one thread has the operands copied (TMA, two stages).
// While KV runs, scores are worked on; while PV and QS do, the state and the next v; outputs behind the next scores.
// k, v, the scaled v and the state lie in rows of 64 values (128 bytes, swizzled): read along rows they are one operand's layout, across
// rows the other's, so nothing is transposed.
//
// Numbers. q, k and v are operands as they are. Scores and state go in as two pieces (2^-16 of each), the scaled v as three,
// which hold all of its 24 bits (two left the states 2.4e-6 off). The state's sums are fp32 in registers, a chunk's products in tensor memory.
//
// Bound: the products' issue and the warps' work between them, not bytes: the 52 to 64 products of a chunk, of 64 or 128 columns, take 45 to
// 70 cycles each, 3.3 us a chunk or more in all. 16 x 1000 frames x 16 heads x 128: 138 us (512 units of 8 chunks on 152 SMs, 1.9
// TB/s), with sequences of a third to all of that 97 us; the kernel of linattn.cuh takes 238 and 183 us.
#include <algorithm>

#include "linattn.cuh"
#include "tc_gemm.h"

namespace qnn {
namespace {

// Registers: 96 a thread at launch; the issuing warps (and the copying ones) leave some of theirs to the state's, which hold 64 values each.
constexpr int kChunk = 128, kTcThreads = 20 * 32, kRegs = 96, kRegsScores = 112, kRegsState = 136, kRegsCopy = 72, kRegsIssue = 48;
static_assert(2 * kRegsScores + kRegsState + kRegsCopy + kRegsIssue <= 5 * kRegs);
constexpr unsigned long long kTcWaitNs = 2000000000ull;
constexpr int kPanel = kChunk * 128;                        // bytes of 128 rows of 64 values
constexpr int kSc = 0, kO = 128, kD = 384;  // columns of tensor memory: scores (then their pieces), A and B of two chunks, D in two parts

constexpr int kSorted = 256;
struct TcShared {  // behind the operands
    float powers[2][kChunk + 32];  // d^0 .. from 32 on (what lies before is read for later frames, and not used)
    int bad[4][kLinCols];  // first frame of a chunk at which a column of v is not finite
    uint64_t full[2], unit[2], k_free[2], qv_free[2], vp, vp2, v_ready, low_done, sc_full, d_full, pv_done, p_ready, s_ready, d_free, end, o_full[2],
        o_free[2];
    uint8_t order[kSorted];
    uint32_t tmem;
    int abort;
};
template <int KP>
struct TcLayout {  // byte offsets: k, q, v, scaled v (two pieces), state (two pieces)
    static constexpr int kK = 0, kQ = 2 * KP * kPanel, kV = kQ + 2 * KP * kPanel, kVs = kV + 2 * kPanel, kS = kVs + 2 * kPanel,
                         kRest = kS + 2 * kPanel, kBytes = kRest + (int)sizeof(TcShared);
};

// Low word of the descriptor of an operand in shared memory with 128-byte swizzle; rows of 64 values 128 bytes apart, eight of them
// 1024. Read across rows, the next 64 values lie `panel` bytes on. (Byte offsets / 16 are added to it; the high word is kSmemDescHi.)
__device__ __forceinline__ uint32_t operand(uint32_t addr, uint32_t panel) { return ((addr & 0x3ffff) >> 4) | (panel >> 4) << 16; }
// kind::f16 with bf16 operands and fp32 sums: M = 128 rows, N columns; a, b: read across rows.
__host__ __device__ constexpr uint32_t idesc(int N, bool a, bool b) {
    return 1u << 4 | 1u << 7 | 1u << 10 | (uint32_t)a << 15 | (uint32_t)b << 16 | (uint32_t)(N >> 3) << 17 | (uint32_t)(128 >> 4) << 24;
}
// Issued by one elected thread of a warp that goes through the program as a whole: operands then stay in uniform registers. (A
// program of one thread moved them there for every product, 100 to 190 cycles each.)
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t desc, uint32_t add) {
    asm volatile(
        "{\n .reg .pred p, q;\n .reg .b64 a, b;\n setp.ne.b32 p, %4, 0;\n elect.sync _|q, 0xffffffff;\n mov.b64 a, {%1, %5};\n mov.b64 b, {%2, %5};\n"
        " @q tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}" ::"r"(d),
        "r"(a), "r"(b), "r"(desc), "r"(add), "n"(kSmemDescHi)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t desc, uint32_t add) {
    asm volatile(
        "{\n .reg .pred p, q;\n .reg .b64 b;\n setp.ne.b32 p, %4, 0;\n elect.sync _|q, 0xffffffff;\n mov.b64 b, {%2, %5};\n"
        " @q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n}" ::"r"(d),
        "r"(a), "r"(b), "r"(desc), "r"(add), "n"(kSmemDescHi)
        : "memory");
}
__device__ __forceinline__ void commit_elected(uint32_t bar) {
    asm volatile(
        "{\n .reg .pred q;\n elect.sync _|q, 0xffffffff;\n"
        " @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar)
        : "memory");
}
// Steps of 16: along rows 32 bytes, and the next panel after four; across rows 16 rows of 128 bytes.
constexpr uint32_t kAcross = 16 * 128 / 16;
__device__ __forceinline__ uint32_t next_along(uint32_t x, int i) { return x + ((i & 3) == 3 ? (kPanel - 96) / 16 : 2); }
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
                 "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// A (sequence, head, columns) of the block's list. The list goes over the sequences from the longest to the shortest (of up to
// kSorted of them with lengths of their own), back and forth over the blocks: 16 x 16 heads x 128 with sequences of a third to all of 1000
// frames 6 us less than in the order that they are given, 97.
struct Unit {
    int64_t bh, b;
    int round, h, tile, n, chunks;
    bool live, valid;  // the list goes on; this entry is one
    __device__ __forceinline__ void set(const LinearArgs &a, const uint8_t *order, int to) {
        round = to;
        const int64_t all = a.B * a.H * a.tiles, first = (int64_t)round * gridDim.x;
        const int64_t at = first + ((round & 1) ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
        live = first < all, valid = at < all;
        const Split t = split(valid ? at : 0, a.tiles), x = split(t.quot, a.H);
        tile = (int)t.rem, h = (int)x.rem, b = a.lengths && a.B <= kSorted ? order[x.quot] : x.quot, bh = b * a.H + h;
        n = valid ? frames_of(a.lengths, b, a.T) : 0;
        chunks = (n + kChunk - 1) / kChunk;
    }
};

template <int KP>
__global__ void __launch_bounds__(kTcThreads, 1) linear_tc_kernel(const LinearArgs a, int *status, const __grid_constant__ CUtensorMap qm, const __grid_constant__ CUtensorMap km,
                     const __grid_constant__ CUtensorMap vm) {
    using L = TcLayout<KP>;
    extern __shared__ __align__(1024) unsigned char tc_smem[];
    unsigned char *const smem = tc_smem;
    TcShared &sh = *reinterpret_cast<TcShared *>(smem + L::kRest);
    const uint32_t base = su32(smem);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    if (base & 1023) {  // (swizzled rows and descriptors count on it)
        record_status(status, QNN_ERR_CUDA);
        return;
    }
    if (threadIdx.x == 0) {
        sh.abort = 0;
        for (int i = 0; i < 2; ++i) mb_init(su32(&sh.full[i]), 1), mb_init(su32(&sh.unit[i]), 4), mb_init(su32(&sh.k_free[i]), 1), mb_init(su32(&sh.qv_free[i]), 1);
        mb_init(su32(&sh.vp), 4), mb_init(su32(&sh.vp2), 4), mb_init(su32(&sh.v_ready), 4), mb_init(su32(&sh.low_done), 1);
        mb_init(su32(&sh.sc_full), 1), mb_init(su32(&sh.d_full), 1), mb_init(su32(&sh.pv_done), 1);
        mb_init(su32(&sh.p_ready), 8), mb_init(su32(&sh.s_ready), 4), mb_init(su32(&sh.d_free), 4), mb_init(su32(&sh.end), 1);
        for (int i = 0; i < 2; ++i) mb_init(su32(&sh.o_full[i]), 1), mb_init(su32(&sh.o_free[i]), 8);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_smem();
    }
    if (warp == 16) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(su32(&sh.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (a.lengths && a.B <= kSorted) {
        int *const frames = &sh.bad[0][0];
        static_assert(sizeof(sh.bad) >= kSorted * sizeof(int));
        const int t = threadIdx.x, B = (int)a.B;
        if (t < B) frames[t] = frames_of(a.lengths, t, a.T);
        __syncthreads();
        if (t < B) {
            int longer = 0;
            for (int j = 0; j < B; ++j) longer += frames[j] > frames[t] || (frames[j] == frames[t] && j < t);
            sh.order[longer] = (uint8_t)t;
        }
    }
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = sh.tmem;
    const uint8_t *const list = sh.order;
    const uint32_t full0 = su32(&sh.full[0]), unit0 = su32(&sh.unit[0]), k_free0 = su32(&sh.k_free[0]), qv_free0 = su32(&sh.qv_free[0]), vp = su32(&sh.vp), vp2 = su32(&sh.vp2), v_ready = su32(&sh.v_ready), low_done = su32(&sh.low_done),
                   sc_full = su32(&sh.sc_full), d_full = su32(&sh.d_full), o_full0 = su32(&sh.o_full[0]), pv_done = su32(&sh.pv_done),
                   p_ready = su32(&sh.p_ready), s_ready = su32(&sh.s_ready), d_free = su32(&sh.d_free), o_free0 = su32(&sh.o_free[0]);
    // waits are bounded; after one gave up the block's other loops end too
    auto wait = [&](uint32_t bar, unsigned parity) {
        if (mbar_try(bar, parity)) return true;
        if (!*reinterpret_cast<volatile int *>(&sh.abort) && mbar_wait_bounded(bar, parity, status, kTcWaitNs)) return true;
        *reinterpret_cast<volatile int *>(&sh.abort) = 1;
        return false;
    };
    auto all_wait = [&](uint32_t bar, unsigned parity) { return __all_sync(0xffffffffu, wait(bar, parity)) != 0; };
    auto arrive = [&](uint32_t bar) {  // of the warp, once its threads are done
        __syncwarp();
        if (lane == 0) mb_arrive(bar);
    };
    Unit u;

    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsScores));
        const int quarter = warp & 3, half = warp >> 2, i = quarter * 32 + lane;
        const uint32_t tm = tmem + ((uint32_t)(quarter * 32) << 16);
        unsigned c = 0, order = 0;
        // the outputs of a chunk are taken behind the next one's scores
        float over = 0.0f, last_over = 0.0f;
        __nv_bfloat16 *last = nullptr;
        int last_cols = 0;
        bool last_there = false;
        auto outputs = [&](unsigned c) {
            if (!all_wait(o_full0 + 8 * (c & 1), (c >> 1) & 1)) return false;
            tc_after();
            const volatile int *bad = &sh.bad[c & 3][half * 32];
            const bool some = __any_sync(0xffffffffu, bad[lane] < kChunk);
            uint32_t r[32], x[32];
            tmem_ld32_nowait(tm + kO + (c & 1) * 128 + half * 32, r);
            tmem_ld32_nowait(tm + kO + (c & 1) * 128 + 64 + half * 32, x);
            tmem_wait_ld();
#pragma unroll
            for (int j = 0; j < 32; ++j) asm volatile("" : "+r"(r[j]), "+r"(x[j]));  // (no use of them goes before the wait)
            tc_before();
            arrive(o_free0 + 8 * (c & 1));
#pragma unroll
            for (int j = 0; j < 32; ++j)
                r[j] = __float_as_uint(__fmul_rn(__fmaf_rn(__uint_as_float(x[j]), last_over, __uint_as_float(r[j])), a.scale));
            if (some) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (i >= bad[j]) r[j] = 0x7fffffffu;
            }
            if (last_there) {
#pragma unroll
                for (int j = 0; j < 32; j += 8)
                    if (j < last_cols) {
                        uint32_t w[4];
#pragma unroll
                        for (int q = 0; q < 4; ++q) w[q] = rounded_pair(__uint_as_float(r[j + 2 * q]), __uint_as_float(r[j + 2 * q + 1]));
                        *reinterpret_cast<uint4 *>(last + j) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
            }
            return true;
        };
        const float *powers = nullptr;
        __nv_bfloat16 *out = nullptr;
        int cols = 0, k = 0;
        u.set(a, list, 0);
        // (each part once in the code: five programs share the instruction caches)
        for (;; ++c) {
            while (u.live && k == u.chunks) u.set(a, list, u.round + 1), k = 0;
            const bool more = u.live;
            if (more) {
                if (k == 0) {
                    powers = sh.powers[order & 1] + 32;
                    if (!all_wait(unit0 + 8 * (order & 1), (order >> 1) & 1)) goto done;
                    ++order;
                    over = power(head_rate(a.log_decay, u.h), (float)(i + 1));
                    out = static_cast<__nv_bfloat16 *>(a.y) + u.b * a.y_seq + (int64_t)i * a.y_frame + (int64_t)u.h * a.dv + u.tile * kLinCols +
                          half * 32;
                    cols = a.dv - u.tile * kLinCols - half * 32;
                }
                if (!all_wait(sc_full, c & 1)) goto done;
                tc_after();
                uint32_t r[2][16];
                const int end = quarter * 32 + 32;  // columns of the warp's rows
                if (half * 64 < end) tmem_ld16_nowait(tm + kSc + half * 64, r[0]);
#pragma unroll 1
                for (int col = half * 64; col < half * 64 + 64; col += 32) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int at = col + 16 * e, left = i - at;  // columns 0 .. left are of frames up to the row's
                        uint32_t hi[8], lo[8];
                        if (at < end) {
                            tmem_wait_ld();
#pragma unroll
                            for (int j = 0; j < 16; ++j) asm volatile("" : "+r"(r[e][j]));  // (no use before the wait)
                            if (at + 16 < end && at + 16 < half * 64 + 64) tmem_ld16_nowait(tm + kSc + at + 16, r[e ^ 1]);
                            const float *p = powers + left;  // d^(i - j)
#pragma unroll
                            for (int j = 0; j < 16; j += 2) {
                                const float f = j <= left ? __fmul_rn(__uint_as_float(r[e][j]), p[-j]) : 0.0f;
                                const float g = j < left ? __fmul_rn(__uint_as_float(r[e][j + 1]), p[-j - 1]) : 0.0f;
                                uint32_t w[2];
                                split_pair<2>(f, g, w);
                                hi[j / 2] = w[0], lo[j / 2] = w[1];
                            }
                        } else {
#pragma unroll
                            for (int j = 0; j < 8; ++j) hi[j] = lo[j] = 0;
                        }
                        tmem_st8(tm + kSc + at, hi);
                        tmem_st8(tm + kSc + at + 8, lo);
                    }
                }
                tmem_wait_st();
                tc_before();
                __syncwarp();
                if (lane == 0) mb_arrive(p_ready);
            }
            if (c > 0 && !outputs(c - 1)) goto done;
            if (!more) break;
            last = out, last_over = over, last_cols = cols, last_there = k * kChunk + i < u.n;
            out += kChunk * a.y_frame;
            ++k;
        }
    } else if (warp < 12) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsState));
        const int r = (warp & 3) * 32 + lane;  // row of the state
        const uint32_t tm = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t row = base + L::kS + r * 128;
        unsigned c = 0;
        float S[kLinCols];
        auto pieces = [&] {
            if (r < KP * 64) {
#pragma unroll
                for (int j = 0; j < kLinCols; j += 8) {
                    uint32_t hi[4], lo[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t w[2];
                        split_pair<2>(S[j + 2 * e], S[j + 2 * e + 1], w);
                        hi[e] = w[0], lo[e] = w[1];
                    }
                    const uint32_t to = row + (((j / 8) ^ (r & 7)) << 4);
                    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(to), "r"(hi[0]), "r"(hi[1]), "r"(hi[2]), "r"(hi[3]) : "memory");
                    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(to + kPanel), "r"(lo[0]), "r"(lo[1]), "r"(lo[2]), "r"(lo[3])
                                 : "memory");
                }
            }
            fence_async_smem();
            arrive(s_ready);
        };
        for (u.set(a, list, 0); u.live; u.set(a, list, u.round + 1)) {
            const int col0 = u.tile * kLinCols, cols = a.dv - col0 < kLinCols ? a.dv - col0 : kLinCols;
            const int64_t at = (u.bh * a.dk + r) * a.dv + col0;
            const bool in = a.state_in && r < a.dk && u.valid;
#pragma unroll
            for (int j = 0; j < kLinCols; j += 4) {
                float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (in && j < cols) v = *reinterpret_cast<const float4 *>(a.state_in + at + j);
                S[j] = v.x, S[j + 1] = v.y, S[j + 2] = v.z, S[j + 3] = v.w;
            }
            const float rate = head_rate(a.log_decay, u.h);
            for (int k = 0; k < u.chunks; ++k, ++c) {
                const int rows = u.n - k * kChunk < kChunk ? u.n - k * kChunk : kChunk;
                const float decay = power(rate, (float)rows);
                if (c > 0) {  // (the products with the state before, of another unit perhaps, are done)
                    if (!all_wait(o_full0 + 8 * ((c - 1) & 1), ((c - 1) >> 1) & 1)) goto done;
                    if (threadIdx.x == 8 * 32) mb_arrive(qv_free0 + 8 * ((c - 1) & 1));
                }
                pieces();
                if (!all_wait(d_full, c & 1)) goto done;
                tc_after();
                if (threadIdx.x == 8 * 32) mb_arrive(k_free0 + 8 * (c & 1));
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    uint32_t d[16], e[16];
                    tmem_ld16(tm + kD + p * 16, d);
                    tmem_ld16(tm + kD + 64 + p * 16, e);
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        S[p * 16 + j] = __fmaf_rn(S[p * 16 + j], decay, __fadd_rn(__uint_as_float(d[j]), __uint_as_float(e[j])));
                }
                tc_before();
                arrive(d_free);
            }
            if (a.state_out && r < a.dk && u.valid)
#pragma unroll
                for (int j = 0; j < kLinCols; j += 4)
                    if (j < cols) *reinterpret_cast<float4 *>(a.state_out + at + j) = make_float4(S[j], S[j + 1], S[j + 2], S[j + 3]);
        }
    } else if (warp < 16) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsCopy));
        // (after a wait gave up these warps go on, as they meet at a barrier)
        const int t = threadIdx.x - 12 * 32;
        const uint32_t at = (t >> 3) * 128 + (((t & 7) ^ ((t >> 3) & 7)) << 4);  // a thread's 16 bytes of rows t / 8 + 16 e
        unsigned c = 0, order = 0;
        for (u.set(a, list, 0); u.live; u.set(a, list, u.round + 1)) {
            if (u.chunks == 0) continue;
            float *const powers = sh.powers[order & 1] + 32;
            const float rate = head_rate(a.log_decay, u.h);
            for (int k = 0; k < u.chunks; ++k, ++c) {
                const uint32_t s = c & 1;
                const int rows = u.n - k * kChunk < kChunk ? u.n - k * kChunk : kChunk;
                wait(full0 + 8 * s, (c >> 1) & 1);
                if (k == 0) {  // (the table of the unit before last: its scores are done, as these operands came after outputs behind it)
                    for (int i = t; i < kChunk; i += 128) powers[i] = power(rate, (float)i);
                    arrive(unit0 + 8 * (order & 1));
                    ++order;
                }
                if (t < kLinCols) sh.bad[c & 3][t] = kChunk;
                asm volatile("bar.sync 1, 128;" ::: "memory");
                const uint32_t vrow = base + L::kV + s * kPanel + at, to = base + L::kVs + at;
                auto load = [](uint32_t from, uint32_t (&v)[4]) {
                    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(from));
                };
                auto store = [](uint32_t to, const uint32_t (&v)[4]) {
                    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
                };
                if (rows < kChunk) {
                    // frames behind the sequence's end, which another may have written anything into: zeros
                    const uint32_t none[4] = {0, 0, 0, 0};
#pragma unroll 1
                    for (int e = 0; e < 8; ++e)
                        if ((t >> 3) + 16 * e >= rows) {
                            store(vrow + e * 2048, none);
                            for (int p = 0; p < KP; ++p) store(base + L::kK + (s * KP + p) * kPanel + at + e * 2048, none);
                        }
                }
                auto weight = [&](int e) {
                    const int left = rows - 1 - ((t >> 3) + 16 * e);
                    return powers[left > 0 ? left : 0];
                };
                // pieces of the scaled v into two buffers: the first and, in turn, the last and the middle one (v and its rounding again:
                // unrolled, with the middle pieces kept, the code's way into the caches took longer)
                if (c > 0) wait(d_full, (c - 1) & 1);
                uint32_t zero = 0;
#pragma unroll 1
                for (int e = 0; e < 8; ++e) {
                    const float w = weight(e);
                    uint32_t v[4], hi[4], lo[4];
                    load(vrow + e * 2048, v);
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(zero) : "r"(v[x]), "r"(0u));
                        float f = __fmul_rn(low_of(v[x]), w), g = __fmul_rn(high_of(v[x]), w);
                        hi[x] = rounded_pair(f, g);
                        f = __fsub_rn(f, low_of(hi[x])), g = __fsub_rn(g, high_of(hi[x]));
                        lo[x] = rounded_pair(f, g);
                        lo[x] = rounded_pair(__fsub_rn(f, low_of(lo[x])), __fsub_rn(g, high_of(lo[x])));
                    }
                    store(to + e * 2048, hi);
                    store(to + kPanel + e * 2048, lo);
                }
                fence_async_smem();
                arrive(vp);
                const bool finite = __all_sync(0xffffffffu, (zero & 0x7fff7fffu) == 0);
                if (finite && lane == 0) mb_arrive(v_ready);
                wait(low_done, c & 1);
#pragma unroll 1
                for (int e = 0; e < 8; ++e) {
                    const float w = weight(e);
                    uint32_t v[4], mid[4];
                    load(vrow + e * 2048, v);
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const float f = __fmul_rn(low_of(v[x]), w), g = __fmul_rn(high_of(v[x]), w);
                        const uint32_t hi = rounded_pair(f, g);
                        mid[x] = rounded_pair(__fsub_rn(f, low_of(hi)), __fsub_rn(g, high_of(hi)));
                    }
                    store(to + kPanel + e * 2048, mid);
                }
                if (!finite) {
                    // a value that is not finite: 0 for PV (whose scores of earlier frames are 0), and outputs from its frame on are NaNs
#pragma unroll 1
                    for (int e = 0; e < 8; ++e) {
                        uint32_t v[4];
                        load(vrow + e * 2048, v);
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            if ((v[x] & 0x7f80u) == 0x7f80u) {
                                v[x] &= 0xffff0000u;
                                atomicMin(&sh.bad[c & 3][(t & 7) * 8 + 2 * x], (t >> 3) + 16 * e);
                            }
                            if ((v[x] & 0x7f800000u) == 0x7f800000u) {
                                v[x] &= 0xffffu;
                                atomicMin(&sh.bad[c & 3][(t & 7) * 8 + 2 * x + 1], (t >> 3) + 16 * e);
                            }
                        }
                        store(vrow + e * 2048, v);
                    }
                    fence_async_smem();
                    arrive(v_ready);
                }
                fence_async_smem();
                arrive(vp2);
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsIssue));
        if (warp == 17 && lane == 0) {
            unsigned c = 0;
            bool go = true;
            for (u.set(a, list, 0); go && u.live; u.set(a, list, u.round + 1))
                for (int k = 0; go && k < u.chunks; ++k, ++c) {
                    const uint32_t s = c & 1, bar = full0 + 8 * s;
                    const int frame = k * kChunk, b = (int)u.b, hk = u.h / a.k_share, hq = u.h / a.q_share, hv = u.h / a.v_share;
                    // a stage is free once the products of the chunk before last are done with it: KV first, of k
                    // (after a wait gave up, the copies that the barrier counts on are made all the same, and no more)
                    if (c > 1 && !wait(k_free0 + 8 * s, ((c >> 1) - 1) & 1)) go = false;
                    mb_expect(bar, (2 * KP + 1) * kPanel);
                    for (int p = 0; p < KP; ++p) tma_load_4d(base + L::kK + (s * KP + p) * kPanel, &km, bar, p * 64, hk, frame, b);
                    if (c > 1 && !wait(qv_free0 + 8 * s, ((c >> 1) - 1) & 1)) go = false;
                    for (int p = 0; p < KP; ++p) tma_load_4d(base + L::kQ + (s * KP + p) * kPanel, &qm, bar, p * 64, hq, frame, b);
                    tma_load_4d(base + L::kV + s * kPanel, &vm, bar, u.tile * kLinCols, hv, frame, b);
                }
            // (every copy has landed when the block ends)
            for (unsigned i = c > 1 ? c - 2 : 0; i < c; ++i)
                mbar_wait_bounded(full0 + 8 * (i & 1), (i >> 1) & 1, status, kTcWaitNs);
            goto done;
        }
        if (warp > 16) goto done;
        const uint32_t vs = operand(base + L::kVs, 1024), st = operand(base + L::kS, 1024);
        u.set(a, list, 0);
        int k = -1;  // chunk of the unit that QK is issued for
        auto next_chunk = [&] {
            if (++k < u.chunks) return true;
            k = 0;
            do u.set(a, list, u.round + 1);
            while (u.live && u.chunks == 0);
            return u.live;
        };
        // (the first round has QK alone, the last all but it)
        bool more = u.live && next_chunk();
        for (unsigned x = 0; more || x > 0; ++x) {
            const uint32_t s = (x - 1) & 1, n = x & 1;  // stages of this chunk, x - 1, and of the next
            const uint32_t kc = operand(base + L::kK + s * KP * kPanel, KP == 2 ? kPanel : 1024), vv = operand(base + L::kV + s * kPanel, 1024);
            const uint32_t o = tmem + kO + s * 128, q = operand(base + L::kQ + s * KP * kPanel, 1024);
            constexpr uint32_t kv = idesc(64, true, true), pv = idesc(64, false, true), qk = idesc(128, false, false);
            if (x > 0) {
                const unsigned c = x - 1;
                if (!all_wait(vp, c & 1) || (c > 0 && !all_wait(d_free, (c - 1) & 1))) goto issued;
                tc_after();
                uint32_t x0 = kc, x1 = vs;
#pragma unroll 2
                for (int i = 0; i < 8; ++i) {  // the first pieces, the last pieces
                    mma_ss(tmem + kD, x0, x1, kv, i > 0);
                    mma_ss(tmem + kD + 64, x0, x1 + (kPanel >> 4), kv, i > 0);
                    x0 += kAcross, x1 += kAcross;
                }
                commit_elected(low_done);
                if (!all_wait(v_ready, c & 1) || (c > 1 && !all_wait(o_free0 + 8 * s, ((c >> 1) - 1) & 1)) || !all_wait(p_ready, c & 1)) goto issued;
                tc_after();
                x0 = tmem + kSc, x1 = vv;
#pragma unroll 2
                for (int i = 0; i < 8; ++i) {
                    mma_ts(o, x0 + 8, x1, pv, i > 0);
                    mma_ts(o, x0, x1, pv, 1);
                    x0 += 16, x1 += kAcross;
                }
                commit_elected(pv_done);
                if (!all_wait(s_ready, c & 1) || !all_wait(vp2, c & 1)) goto issued;
                tc_after();
                x0 = kc, x1 = vs + (kPanel >> 4);
                uint32_t x2 = q, x3 = st + (kPanel >> 4);
#pragma unroll 4
                for (int i = 0; i < 8; ++i) {  // the middle pieces, in turn with QS of the second ones
                    mma_ss(tmem + kD + 64, x0, x1, kv, 1);
                    x0 += kAcross, x1 += kAcross;
                    if (i < 4 * KP) {
                        mma_ss(o + 64, x2, x3, pv, i > 0);
                        x2 = next_along(x2, i), x3 += kAcross;
                    }
                }
                commit_elected(d_full);
            }
            // QK of the next chunk, in turn with QS of the first pieces
            if (more) {
                if (!all_wait(full0 + 8 * n, (x >> 1) & 1) || (x > 0 && !all_wait(pv_done, (x - 1) & 1))) goto issued;  // (the scores' place)
                tc_after();
            }
            {
                uint32_t x0 = operand(base + L::kQ + n * KP * kPanel, 1024), x1 = operand(base + L::kK + n * KP * kPanel, 1024), x2 = q, x3 = st;
                if (more && x > 0) {
#pragma unroll 4
                    for (int i = 0; i < 4 * KP; ++i) {
                        mma_ss(tmem + kSc, x0, x1, qk, i > 0);
                        mma_ss(o + 64, x2, x3, pv, 1);
                        x0 = next_along(x0, i), x1 = next_along(x1, i), x2 = next_along(x2, i), x3 += kAcross;
                    }
                } else {
#pragma unroll 1
                    for (int i = 0; i < 4 * KP; ++i) {
                        if (more) mma_ss(tmem + kSc, x0, x1, qk, i > 0);
                        else mma_ss(o + 64, x2, x3, pv, 1);
                        x0 = next_along(x0, i), x1 = next_along(x1, i), x2 = next_along(x2, i), x3 += kAcross;
                    }
                }
                if (more) commit_elected(sc_full);
                if (x > 0) commit_elected(o_full0 + 8 * s);
            }
            if (!more) break;
            more = next_chunk();
        }
    issued:
        // (no product is in flight when the tensor memory is given back, after a wait that gave up neither)
        commit_elected(su32(&sh.end));
        mbar_wait_bounded(su32(&sh.end), 0, status, kTcWaitNs);
    }
done:
    tc_before();
    __syncthreads();
    if (warp == 16) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

template <int KP>
qnn_status launch_tc(const LinearArgs &a, cudaStream_t st) {
    using L = TcLayout<KP>;
    static_assert(L::kBytes <= 227 * 1024);
    int *status = nullptr;
    QNN_TRY(status_word(&status));
    CUtensorMap qm, km, vm;
    QNN_TRY(tc_map_heads(&qm, a.q, a.dk, a.H / a.q_share, a.T, a.B, a.q_frame, a.q_seq, kChunk));
    QNN_TRY(tc_map_heads(&km, a.k, a.dk, a.H / a.k_share, a.T, a.B, a.k_frame, a.k_seq, kChunk));
    QNN_TRY(tc_map_heads(&vm, a.v, a.dv, a.H / a.v_share, a.T, a.B, a.v_frame, a.v_seq, kChunk));
    QNN_CUDA_TRY(cudaFuncSetAttribute(linear_tc_kernel<KP>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kBytes));
    const int64_t blocks = std::min<int64_t>(a.B * a.H * a.tiles, sm_count());
    linear_tc_kernel<KP><<<(unsigned)blocks, kTcThreads, L::kBytes, st>>>(a, status, qm, km, vm);
    QNN_CUDA_TRY(cudaGetLastError());
    return QNN_OK;
}

}  // namespace

// (Tensor maps take no strides of zero, which are the inputs of one sequence or frame for all, nor any of 2^40 bytes.)
bool linear_tc_fits(const LinearArgs &a) {
    const uintptr_t states = reinterpret_cast<uintptr_t>(a.state_in) | reinterpret_cast<uintptr_t>(a.state_out);
    const int64_t strides[8] = {a.q_frame, a.k_frame, a.v_frame, a.y_frame, a.q_seq, a.k_seq, a.v_seq, a.y_seq};
    for (int i = 0; i < (a.B > 1 ? 8 : 4); ++i)
        if (strides[i] <= 0 || strides[i] >= (int64_t)1 << 39) return false;
    return a.dk <= 128 && a.dv % 8 == 0 && states % 16 == 0 && a.q_copy == 16 && a.k_copy == 16 && a.v_copy == 16 && a.y_copy == 16;
}
qnn_status launch_linear_tc(const LinearArgs &a, cudaStream_t st) { return a.dk <= 64 ? launch_tc<1>(a, st) : launch_tc<2>(a, st); }

}  // namespace qnn
