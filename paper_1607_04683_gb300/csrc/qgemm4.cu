// qgemm4.cu — 4-bit weights in units of `group` columns of a row (Sec. 3.1's sub-matrices, eq. 2 with S = 15) and their
// product with rows of 8-bit activation codes, recovered to fp32 (eq. 1, eq. 3) on sm_103a.
#include <algorithm>
#include <atomic>

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
    int seg_shift;    // 2^seg_shift warps share a row tile's columns; the block's other warps take other row tiles
    int blocks, span; // of a cluster, which share the columns of its row tiles, and the column tiles of one
    int64_t items;    // clusters' shares of row tiles
    int chunks, chunk, stride;  // column tiles of A in shared memory at once, how often, and bytes of a row of them
    uint32_t per_row_magic;     // ceil(2^32 / (8 chunk)): divides by the steps of a row of a whole chunk
    int align;        // of A's rows, 16, 4 or 1
};

// y from the sum t1 over centered codes c = a' - 128: sum (a' + za) w^ = t1 + (128 + za) sum w^, over Qa, plus the bias.
// `unit`: Qa, 128 + za.
__device__ __forceinline__ float recover4(float t1, float2 unit, float row_sum, float bias) {
    return __fadd_rn(__fdiv_rn(__fmaf_rn(unit.y, row_sum, t1), unit.x), bias);
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

// The first two and the last two of four 8-bit codes b as 16 (b - 128) and as b - 128.
__device__ __forceinline__ uint32_t codes_x16(uint32_t v) {
    return hfma2_bits(__byte_perm(v, 0x64646464u, 0x4140), both(16.0f), both(-18432.0f));
}
__device__ __forceinline__ uint32_t codes_x1(uint32_t v) {
    return hfma2_bits(__byte_perm(v, 0x64646464u, 0x4342), both(1.0f), both(-1152.0f));
}

// The products run on the fp16 tensor-core instruction, exactly, on codes that cost next to nothing to convert:
//   - a 4-bit code masked out of its word in place is a subnormal fp16 number, code 2^-24 in a half's lowest four bits and
//     16 code 2^-24 in the next four (0x000f000f and 0x00f000f0 give two of a word's eight columns each; one shift gives the
//     other four);
//   - an 8-bit code b under the byte 0x64 is the fp16 number 1024 + b, from which one multiply-add makes 16 (b - 128) for
//     columns whose weights count once and b - 128 for those that count 16 times.
// So every product is (b - 128) code 2^-20, and a group's sum, below 2^24 of that unit, is exact in fp32. The sum of a
// group starts from offset x (sum of b - 128) and is taken into the output's sum by its scale, in fp32, 2^4 times as large: a
// scale is a multiple of 2^-133 (eight bits from 2^-126 on), so products with it are multiples of 2^-149, as every fp32 number is,
// and none loses bits below the range's end; at its other end they overflow no earlier than the whole sum.
//
// A block's 16 warps split the columns of its row tiles (`segments` of them, tile by tile in turn, so that a block reads long
// contiguous stretches) and add up through shared memory at the end, in a fixed order. Bound: the weights' bytes. Each
// warp streams its own column tiles through kStages slots of shared memory by asynchronous copies, across row tiles, so that
// 16 kStages KB a block are in flight at any time; a slot is read into registers and filled again before its products.
// Measured (weights from HBM): 1 x 8192 x 8192 in groups of 32, 42 MB, 11.2 to 11.8 us (3.7 TB/s; 175 instructions a cell of 16
// rows x 128 columns), of 128 10.2; 8 rows in groups of 128 10.9 to 11.4; 16 rows 13.2 to 13.3; 1 x 2048 x 2048 3.2 us, of which
// 1.1 are a launch with one load and one store. Clock stamps, 16 rows: 1.6 us until A's loads and the first copies are out, 1.3 for
// A's way into shared memory, 7.8 the products (16 cells a warp, 234 cycles each and scheduler, 128 of them the tensor pipe's), 0.6
// the barrier, 1.1 the sums and 0.7 the last barrier. Four or five slots a warp, where three took 13.2: 13.3 and 13.6 us.
constexpr int kMmThreads = 512, kMmWarps = kMmThreads / 32, kRedStride = 20, kMostBlocks = 4;
constexpr float kUnit = 0x1p-20f, kUp = 0x1p4f, kPerUnit = 0x1p16f;

__device__ __forceinline__ void copy16_async(uint32_t to, const void *from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {  // until all but the last N groups are there
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

template <int GROUP>
struct Units {  // of a row's 128 columns
    static constexpr int kCount = kTileCols / GROUP;
    uint32_t u[kCount];
    __device__ __forceinline__ void load(const uint32_t *p) {
        if constexpr (kCount == 4) {
            const uint4 v = *reinterpret_cast<const uint4 *>(p);
            u[0] = v.x, u[1] = v.y, u[2] = v.z, u[3] = v.w;
        } else if constexpr (kCount == 2) {
            const uint2 v = *reinterpret_cast<const uint2 *>(p);
            u[0] = v.x, u[1] = v.y;
        } else {
            u[0] = *p;
        }
    }
};

// All threads of the block, or of the cluster, and what they wrote to shared memory.
__device__ __forceinline__ void all_here(bool cluster) {
    if (cluster)
        asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");
    else
        __syncthreads();
}
// A shared variable of a block of the cluster, written before all_here. (No order against other loads: several are in flight.)
__device__ __forceinline__ float peer_load(const float *p, int rank) {
    uint32_t at;
    float v;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at));
    return v;
}

template <int GROUP, int NT>
struct Mm4Plan {
    static constexpr int kRows = 8 * NT, kGroups = kTileCols / GROUP;
    static constexpr int kStages = NT <= 2 ? 3 : 2;
    static constexpr int kUnitBytes = kTileRows * kGroups * 4, kSlot = kTileBytes + kUnitBytes;
    static constexpr int kRing = kMmWarps * kStages * kSlot;
    static constexpr int kReds = NT == 1 ? 2 : 1, kRed = kMmWarps * kRows * kRedStride * 4;  // two: one barrier a row tile
    // shared memory: the slots, the warps' sums, A's codes, their group sums
};

template <int GROUP, int NT>
__global__ void __launch_bounds__(kMmThreads, 1) qmatmul4_kernel(const Mm4Args a) {
    using P = Mm4Plan<GROUP, NT>;
    constexpr int kRows = P::kRows, kGroups = P::kGroups;
    extern __shared__ __align__(16) uint8_t smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int64_t m0 = (int64_t)blockIdx.y * kRows;
    const int rows = (int)min((int64_t)kRows, a.M - m0);
    uint8_t *ring = smem + warp * P::kStages * P::kSlot;
    float *reds = reinterpret_cast<float *>(smem + P::kRing);        // [kReds][warps][kRows][kRedStride]
    uint8_t *sA = smem + P::kRing + P::kReds * P::kRed;              // [rows][stride]
    float *sR = reinterpret_cast<float *>(sA + rows * a.stride);     // [chunk groups][kRows]: group sums of b - 128
    float2 *sP = reinterpret_cast<float2 *>(sR + a.chunk * kGroups * kRows);  // [rows]: Qa, 128 + za
    const int segments = 1 << a.seg_shift, seg = warp & (segments - 1), tile_group = warp >> a.seg_shift;
    const int tile_groups = kMmWarps >> a.seg_shift;
    const int rank = a.blocks > 1 ? (int)(blockIdx.x & (a.blocks - 1)) : 0;  // (of the cluster: its size divides the grid)
    const int64_t first_item = blockIdx.x / a.blocks, item_step = gridDim.x / a.blocks;
    const int kt_begin = rank * a.span, kt_end = min(a.ktiles, kt_begin + a.span);
    const int64_t ntiles = (a.N + kTileRows - 1) / kTileRows;

    // the copies' place: the next of `left` column tiles of this warp's row tile of item_next
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring) + 16 * lane;
    const int steps = (max(kt_end - kt_begin - seg, 0) + segments - 1) >> a.seg_shift;
    int64_t item_next = first_item;
    int left = 0;
    const uint8_t *code_next = nullptr, *unit_next = nullptr;
    auto seek = [&]() {
        const int64_t tile = item_next * tile_groups + tile_group, at = tile * a.ktiles + kt_begin + seg;
        left = item_next < a.items && tile < ntiles ? steps : 0;
        code_next = a.codes + at * kTileBytes + 16 * lane;
        unit_next = reinterpret_cast<const uint8_t *>(a.units) + at * P::kUnitBytes + 16 * lane;
    };
    seek();
    auto issue = [&](int slot) {
        if (left > 0) {
            const uint32_t to = ring_at + slot * P::kSlot;
            copy16_async(to, code_next);
            copy16_async(to + 512, code_next + 512);
            if (16 * lane < P::kUnitBytes) copy16_async(to + kTileBytes, unit_next);
            code_next += kTileBytes << a.seg_shift;
            unit_next += P::kUnitBytes << a.seg_shift;
            if (--left == 0) {
                item_next += item_step;
                seek();
            }
        }
        copies_commit();
    };
    // A's codes of column tiles kt0 .. kt1, 16 a thread and step (past K: 128, which counts 0), kAtOnce steps at a time: loaded,
    // and put into shared memory as fp16 values and their sums by groups, over 2 to 8 lanes
    constexpr int kAtOnce = NT == 1 ? 2 : 4;
    const int per_row = a.chunk * (kTileCols / 16), total = rows * per_row;
    uint32_t v[kAtOnce][4];
    auto load_A = [&](int i0, int kt0) {
#pragma unroll
        for (int s = 0; s < kAtOnce; ++s) {
            const int i = i0 + s * kMmThreads + tid, m = (int)__umulhi((uint32_t)i, a.per_row_magic), k = kt0 * kTileCols + 16 * (i - m * per_row);
            v[s][0] = v[s][1] = v[s][2] = v[s][3] = 0x80808080u;
            if (i >= total || k >= a.K) continue;
            const uint8_t *p = a.A + (m0 + m) * a.lda + k;
            if (a.align == 16 && k + 16 <= a.K) {
                const uint4 x = __ldg(reinterpret_cast<const uint4 *>(p));
                v[s][0] = x.x, v[s][1] = x.y, v[s][2] = x.z, v[s][3] = x.w;
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (a.align >= 4 && k + 4 * j + 4 <= a.K) {
                        v[s][j] = __ldg(reinterpret_cast<const uint32_t *>(p + 4 * j));
                    } else if (k + 4 * j < a.K) {
                        v[s][j] = 0;
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[s][j] |= (uint32_t)(k + 4 * j + e < a.K ? __ldg(p + 4 * j + e) : 128) << (8 * e);
                    }
                }
            }
        }
    };
    auto put_A = [&](int i0, int there) {  // of a row's steps
#pragma unroll
        for (int s = 0; s < kAtOnce; ++s) {
            const int i = i0 + s * kMmThreads + tid, m = (int)__umulhi((uint32_t)i, a.per_row_magic), blk = i - m * per_row;
            uint32_t sum = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) sum = __dp4a(v[s][j], 0x01010101u, sum);
#pragma unroll
            for (int o = 1; o < GROUP / 16; o *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (i >= total || blk >= there) continue;
            uint4 *to = reinterpret_cast<uint4 *>(sA + m * a.stride + 32 * blk);
            to[0] = make_uint4(codes_x16(v[s][0]), codes_x1(v[s][0]), codes_x16(v[s][1]), codes_x1(v[s][1]));
            to[1] = make_uint4(codes_x16(v[s][2]), codes_x1(v[s][2]), codes_x16(v[s][3]), codes_x1(v[s][3]));
            if (blk % (GROUP / 16) == 0) sR[blk / (GROUP / 16) * kRows + m] = (float)((int)sum - 128 * GROUP) * kUnit;
        }
    };
    auto stage = [&](int kt0, int kt1, bool loaded) {
        for (int i0 = 0; i0 < total; i0 += kAtOnce * kMmThreads) {
            if (i0 > 0 || !loaded) load_A(i0, kt0);
            put_A(i0, (kt1 - kt0) * (kTileCols / 16));
        }
    };
    // (A before the weights: behind 16 kStages KB a block of them its first codes came 2.4 us later)
    load_A(0, kt_begin);
#pragma unroll
    for (int i = 0; i < P::kStages; ++i) issue(i);
    stage(kt_begin, min(kt_end, kt_begin + a.chunk), true);
    int slot = 0, red_at = 0;
    if (tid < rows) {
        const qnn_qparams p = a.pa[a.per_row ? m0 + tid : 0];
        sP[tid] = make_float2(p.Q, __fadd_rn(128.0f, (float)p.z));
    }
    const int wide_shift = 8 - a.seg_shift, wide = 1 << wide_shift;  // columns of an item: 16 a tile group
    const int share = wide * rows / a.blocks, first_out = rank * share;  // this block's outputs of them
    const int col = (first_out + tid) & (wide - 1);  // this thread's column, of all its outputs: kMmThreads is a multiple of wide
    __syncthreads();

    for (int64_t item = first_item; item < a.items; item += item_step) {
        float2 acc[NT][2] = {};  // by row; its two columns
        float row_sum = 0.0f, bias = 0.0f;
        const int64_t n = item * wide + col;
        if (tid < share && n < a.N) {  // what its outputs need is loaded ahead
            row_sum = __ldg(a.row_sums + n);
            if (a.bias) bias = __ldg(a.bias + n);
        }
        for (int chunk = 0; chunk < a.chunks; ++chunk) {
            const int kt0 = min(kt_end, kt_begin + chunk * a.chunk), kt1 = min(kt_end, kt0 + a.chunk);
            if (a.chunks > 1 && (chunk > 0 || item != first_item)) {
                __syncthreads();  // all warps are done with what was there
                stage(kt0, kt1, false);
                __syncthreads();
            }
            const uint8_t *pa[NT];  // (columns past the rows there are repeat the last: their sums go nowhere)
#pragma unroll
            for (int c = 0; c < NT; ++c) pa[c] = sA + min(8 * c + g, rows - 1) * a.stride + 16 * t;
            for (int kt = kt0 + seg; kt < kt1; kt += segments) {
                copies_wait<P::kStages - 1>();
                __syncwarp();
                const uint8_t *at = ring + slot * P::kSlot;
                const uint4 w0v = *reinterpret_cast<const uint4 *>(at + 16 * lane), w1v = *reinterpret_cast<const uint4 *>(at + 512 + 16 * lane);
                Units<GROUP> u0, u1;
                u0.load(reinterpret_cast<const uint32_t *>(at + kTileBytes) + g * kGroups);
                u1.load(reinterpret_cast<const uint32_t *>(at + kTileBytes) + (g + 8) * kGroups);
                __syncwarp();
                issue(slot);
                slot = slot + 1 == P::kStages ? 0 : slot + 1;
                const uint32_t w0[4] = {w0v.x, w0v.y, w0v.z, w0v.w}, w1[4] = {w1v.x, w1v.y, w1v.z, w1v.w};
                float sum[NT][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int q = j * 32 / GROUP;
                    if (j * 32 % GROUP == 0) {  // a group begins: offset x (sum of its b - 128)
                        const float2 *R = reinterpret_cast<const float2 *>(sR + ((kt - kt0) * kGroups + q) * kRows) + t;
                        const float2 z0 = f2(unit_offset(u0.u[q])), z1 = f2(unit_offset(u1.u[q]));
#pragma unroll
                        for (int c = 0; c < NT; ++c) {
                            const float2 v = R[4 * c], s0 = fmul2_rn(z0, v), s1 = fmul2_rn(z1, v);
                            sum[c][0] = s0.x, sum[c][1] = s0.y, sum[c][2] = s1.x, sum[c][3] = s1.y;
                        }
                    }
                    const uint32_t x = w0[j], y = w1[j], x8 = x >> 8, y8 = y >> 8;
                    const uint32_t wa[4] = {x & 0x000f000fu, y & 0x000f000fu, x & 0x00f000f0u, y & 0x00f000f0u};
                    const uint32_t wb[4] = {x8 & 0x000f000fu, y8 & 0x000f000fu, x8 & 0x00f000f0u, y8 & 0x00f000f0u};
#pragma unroll
                    for (int c = 0; c < NT; ++c) {
                        const uint4 v = *reinterpret_cast<const uint4 *>(pa[c] + 2 * ((kt - kt0) * kTileCols + 32 * j));
                        mma_f16(sum[c], wa, v.x, v.y);
                        mma_f16(sum[c], wb, v.z, v.w);
                    }
                    if ((j + 1) * 32 % GROUP == 0) {  // and ends
                        const float2 s0 = f2(unit_scale(u0.u[q])), s1 = f2(unit_scale(u1.u[q]));
#pragma unroll
                        for (int c = 0; c < NT; ++c) {
                            acc[c][0] = ffma2_rn(s0, fmul2_rn(make_float2(sum[c][0], sum[c][1]), f2(kUp)), acc[c][0]);
                            acc[c][1] = ffma2_rn(s1, fmul2_rn(make_float2(sum[c][2], sum[c][3]), f2(kUp)), acc[c][1]);
                        }
                    }
                }
            }
        }
        // the segments' sums, in order, and those of the cluster's blocks
        float *red = reds + red_at * (P::kRed / 4);
        if (P::kReds == 1 && item != first_item) all_here(a.blocks > 1);  // the item before is out
        if (P::kReds == 2) red_at ^= 1;
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            float *p = red + (warp * kRows + 8 * c + 2 * t) * kRedStride + g;
            p[0] = acc[c][0].x, p[kRedStride] = acc[c][0].y;
            p[8] = acc[c][1].x, p[kRedStride + 8] = acc[c][1].y;
        }
        all_here(a.blocks > 1);
        for (int i = n < a.N ? tid : share; i < share; i += kMmThreads) {
            const int m = (first_out + i) >> wide_shift, tg = col / kTileRows, row = col % kTileRows;
            float sum = 0.0f;
            const float *at = red + ((tg << a.seg_shift) * kRows + m) * kRedStride + row;
            if (a.blocks == 1) {
                for (int k = 0; k < segments; ++k) sum = __fadd_rn(sum, at[k * (kRows * kRedStride)]);
            } else {  // four loads in flight: one takes as long as the barrier
                const int all = a.blocks << a.seg_shift;
                for (int j = 0; j < all; j += 4) {
                    float part[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int k = j + e;
                        part[e] = k < all ? peer_load(at + (k & (segments - 1)) * (kRows * kRedStride), k >> a.seg_shift) : 0.0f;
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum = __fadd_rn(sum, part[e]);
                }
            }
            a.Y[(m0 + m) * a.ldy + n] = recover4(__fmul_rn(sum, kPerUnit), sP[m], row_sum, bias);
        }
    }
    if (a.blocks > 1) all_here(true);  // the others may still read this block's sums
    copies_wait<0>();
}

template <int GROUP, int NT>
qnn_status launch_mm4(Mm4Args a, cudaStream_t st) {
    using P = Mm4Plan<GROUP, NT>;
    const int64_t ntiles = (a.N + kTileRows - 1) / kTileRows;
    // A in shared memory: as many column tiles (fp16 values and group sums) as fit beside the slots and sums
    constexpr size_t kMost = 227 * 1024 - 64, kFixed = P::kRing + P::kReds * P::kRed;
    const int rows = (int)std::min<int64_t>(P::kRows, a.M), sms = sm_count();
    const size_t sums = (size_t)P::kGroups * P::kRows * 4;  // a column tile's group sums
    const int fit = (int)((kMost - kFixed - (size_t)rows * (64 + sizeof(float2))) / ((size_t)rows * 2 * kTileCols + sums));
    // Blocks that share a row tile's columns: kMostBlocks where A has more than kMostCells cells (a row's column tile) to convert
    // or does not fit, and, where row tiles are few, as many as give half of the SMs one (a column tile each at least).
    // (16 x 8192 x 8192: A in two parts through one block 16.7 us, two blocks 14.5, four 13.2; 8 x 8192 x 8192, 512 cells, one 12.4,
    // two 11.5, four 10.9; 16 x 2048 x 8192, 256 cells, one 6.7, four 7.7.)
    constexpr int kMostCells = 256;
    a.blocks = 1;
    while (a.blocks < kMostBlocks && (a.blocks * fit < a.ktiles || rows * a.ktiles > kMostCells ||
                                      (2 * ntiles * a.blocks <= sms && 2 * a.blocks <= a.ktiles)))
        a.blocks *= 2;
    a.span = (a.ktiles + a.blocks - 1) / a.blocks;
    // as many warps on a row tile as leave every SM a block, and as have a column tile each
    a.seg_shift = 4;
    while (a.seg_shift > 0 && ((1 << a.seg_shift) >= 2 * a.span || (ntiles * a.blocks << a.seg_shift) > (int64_t)kMmWarps * sms)) --a.seg_shift;
    const int segments = 1 << a.seg_shift;
    a.items = (ntiles * segments + kMmWarps - 1) / kMmWarps;
    // parts of A that do not fit at once are even, and whole rounds of the warps
    a.chunk = a.span, a.chunks = 1;
    if (fit < a.span) {
        const int whole = fit / segments * segments;
        a.chunks = (a.span + whole - 1) / whole;
        a.chunk = ((a.span + a.chunks - 1) / a.chunks + segments - 1) / segments * segments;
    }
    a.stride = a.chunk * 2 * kTileCols + 64;  // (so that the two rows of a quarter of a load lie in different banks)
    const uint32_t steps = (uint32_t)a.chunk * (kTileCols / 16);
    a.per_row_magic = (uint32_t)((((uint64_t)1 << 32) + steps - 1) / steps);  // (exact: at most 32 rows of 2072 steps)
    const size_t bytes = kFixed + (size_t)rows * (a.stride + sizeof(float2)) + (size_t)a.chunk * sums;
    const auto kern = qmatmul4_kernel<GROUP, NT>;
    static std::atomic<bool> allowed[64];  // by device: the attribute costs a microsecond a call
    int dev = 0;
    QNN_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64) return QNN_FAIL(QNN_ERR_CUDA);
    if (!allowed[dev].load(std::memory_order_acquire)) {
        QNN_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMost));
        allowed[dev].store(true, std::memory_order_release);
    }
    const int64_t mblocks = (a.M + P::kRows - 1) / P::kRows;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.blocks, (unsigned)mblocks);
    cfg.blockDim = dim3(kMmThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)a.blocks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = a.blocks > 1 ? 1 : 0;
    // As many clusters as the device holds at once, asked once: less than its SMs by four, as the SMs of a part of it need not
    // divide by four. (Here 36 of 38: 16 x 8192 x 9216 13.8 us; by 33 clusters, two row tiles each, 23.2. 16 x 8192 x 9728 by 36 23.2,
    // by 38, two of which wait, 25.5.)
    int64_t most = sms;
    if (a.blocks > 1) {
        static std::atomic<int> room[kMostBlocks + 1][64];
        int clusters = room[a.blocks][dev].load(std::memory_order_acquire);
        if (clusters == 0) {
            if (cudaOccupancyMaxActiveClusters(&clusters, kern, &cfg) != cudaSuccess || clusters < 1) {
                cudaGetLastError();
                clusters = std::max(1, sms / a.blocks);
            }
            room[a.blocks][dev].store(clusters, std::memory_order_release);
        }
        most = clusters;
    }
    cfg.gridDim.x = (unsigned)(std::min(a.items, most) * a.blocks);
    QNN_CUDA_TRY(cudaLaunchKernelEx(&cfg, kern, a));
    return QNN_OK;
}

template <int GROUP>
qnn_status launch_mm4(const Mm4Args &a, cudaStream_t st) {
    if (a.M <= 8) return launch_mm4<GROUP, 1>(a, st);
    if (a.M <= 16) return launch_mm4<GROUP, 2>(a, st);
    return launch_mm4<GROUP, 4>(a, st);
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }
bool group_ok(int g) { return g == 32 || g == 64 || g == 128; }

constexpr int64_t kMostN = INT32_MAX / 2, kMostM = 65535 * 8;  // (grid rows of 8 rows at least)
int64_t tiles_of(int64_t N, int64_t K) { return (N + kTileRows - 1) / kTileRows * ((K + kTileCols - 1) / kTileCols); }

}  // namespace
}  // namespace qnn

using namespace qnn;

extern "C" qnn_status qnn_quantize4(const float *w, int64_t N, int64_t K, int64_t ldw, int32_t group, uint8_t *codes,
                                    uint32_t *units, float *row_sums, void *stream) {
    if (N < 1 || N > kMostN || K < 1 || ldw < K || !reach_ok(N, ldw) || !group_ok(group)) return QNN_ERR_INVALID_ARG;
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
    if (M < 0 || M > kMostM || N < 1 || N > kMostN || K < 1 || lda < K || !reach_ok(M, lda) || ldy < N || !reach_ok(M, ldy) ||
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
