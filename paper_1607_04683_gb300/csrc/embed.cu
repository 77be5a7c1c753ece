// embed.cu — embedding lookup with scaling, and its gradient by sorted labels, on sm_103a.
#include <algorithm>

#include "elem.cuh"
#include "qnn_device.cuh"
#include "qnn_host.h"
#include "tc_ptx.cuh"

namespace qnn {
namespace {

bool runs_ok(const void *p, int64_t ld, int e, int v) { return reinterpret_cast<uintptr_t>(p) % (v * e) == 0 && ld % v == 0; }

// ------------------------------------------------------------------------------------------------
// Lookup
// ------------------------------------------------------------------------------------------------

struct EmbedArgs {
    const void *ids, *table;
    void *out;
    int64_t n, V, D, ldt, ldo, items;
    float scale;
    int *status;
    int shares;  // of a row
};

constexpr int kEmbedThreads = 128, kEmbedRuns = 4;

// A warp takes a share of a row, 32 kEmbedRuns runs of W values whose loads are in flight together, and loads the label of the next
// meanwhile. Bound: HBM for the output; rows that come again are read from L2. 16000 x 2048 bf16: 12.4 us, with nothing in L2 17.5 (94 MB).
template <typename T, typename O, typename I, int W>
__global__ void __launch_bounds__(kEmbedThreads) embed_kernel(const EmbedArgs a) {
    const int lane = threadIdx.x % 32;
    const int64_t all = (int64_t)gridDim.x * (kEmbedThreads / 32);
    int64_t at = (int64_t)blockIdx.x * (kEmbedThreads / 32) + threadIdx.x / 32;
    const uint32_t shares = (uint32_t)a.shares;
    auto of = [&](int64_t item) { return shares == 1 ? Split{item, 0} : split(item, shares); };
    Split s = of(at);
    int64_t id = at < a.items ? (int64_t)__ldg(static_cast<const I *>(a.ids) + s.quot) : -1;
    while (at < a.items) {
        const bool there = id >= 0 && id < a.V;
        if (id >= a.V && s.rem == 0 && lane == 0) record_status(a.status, QNN_ERR_INVALID_ARG);
        const int64_t col = (s.rem * (32 * kEmbedRuns) + lane) * W;
        const T *from = static_cast<const T *>(a.table) + (there ? id : 0) * a.ldt + col;
        O *to = static_cast<O *>(a.out) + s.quot * a.ldo + col;
        Run<T, W> v[kEmbedRuns];
#pragma unroll
        for (int i = 0; i < kEmbedRuns; ++i)
            if (there && col + i * 32 * W < a.D) v[i].load(from + i * 32 * W);
        at += all;
        if (at < a.items) {
            s = of(at);
            id = (int64_t)__ldg(static_cast<const I *>(a.ids) + s.quot);
        }
#pragma unroll
        for (int i = 0; i < kEmbedRuns; ++i)
            if (col + i * 32 * W < a.D) {
                float f[W];
#pragma unroll
                for (int e = 0; e < W; ++e) f[e] = there ? __fmul_rn(v[i].get(e), a.scale) : 0.0f;
                Run<O, W> o;
                o.set(f);
                o.store(to + i * 32 * W);
            }
    }
}

template <typename T, typename O, typename I, int W>
qnn_status launch_embed(EmbedArgs a, cudaStream_t st) {
    a.shares = (int)((a.D / W + 32 * kEmbedRuns - 1) / (32 * kEmbedRuns));
    a.items = a.n * a.shares;
    constexpr int kWarps = kEmbedThreads / 32;
    const int64_t blocks = std::min<int64_t>((a.items + kWarps - 1) / kWarps, 10 * (int64_t)sm_count());
    embed_kernel<T, O, I, W><<<(unsigned)blocks, kEmbedThreads, 0, st>>>(a);
    return QNN_OK;
}

template <typename T, typename O, typename I>
qnn_status launch_embed(const EmbedArgs &a, cudaStream_t st) {
    const int t = sizeof(T), o = sizeof(O);
    auto whole = [&](int v) { return a.D % v == 0 && runs_ok(a.table, a.ldt, t, v) && runs_ok(a.out, a.ldo, o, v); };
    if constexpr (sizeof(T) == 2) {
        if (whole(8)) return launch_embed<T, O, I, 8>(a, st);
    }
    if (whole(4)) return launch_embed<T, O, I, 4>(a, st);
    return launch_embed<T, O, I, 1>(a, st);
}

// ------------------------------------------------------------------------------------------------
// Labels in order
// ------------------------------------------------------------------------------------------------

// A stable sort of positions by label, digit by digit from the lowest (a radix sort): a tile of the positions a block, a
// segment of the tile a warp. A warp counts its segment's digits 32 positions at a time, lanes of one digit found by votes over
// its bits; a position's place is then the number of smaller digits, plus those of its own in the tiles, the warps' segments
// and the lanes before it. The next digit's counts by tile are whole numbers added in global memory as places are known, so that no order
// shows. Labels outside the table count as V and come last.
constexpr int kSortThreads = 256, kSortWarps = kSortThreads / 32, kMostBits = 9, kMostBins = 1 << kMostBits;
// Rows of bytes to be cleared by the blocks behind a sort's own, which few blocks of the device take part in: the gradient's rows, most
// of which no position may have. (The others are written again. 16000 labels of 8192 rows of 8 KB: 74 us with the
// absent rows cleared by the sums' kernel, 14 of them by blocks that looked for each row among the labels.)
struct ClearArgs {
    char *p;
    int64_t rows, row, pitch;  // bytes of a row and from one to the next
    int width;                 // bytes of a store: 16, 4 or 2
    int blocks;                // that clear
};
template <typename W>
__device__ __forceinline__ void clear_words(const ClearArgs &c, int64_t warp, int64_t warps, W zero) {
    const int64_t words = c.row / (int64_t)sizeof(W);
    if (c.pitch == c.row) {  // one piece
        const int64_t all = c.rows * words;
        for (int64_t i = warp * 32 + threadIdx.x % 32; i < all; i += warps * 32) reinterpret_cast<W *>(c.p)[i] = zero;
        return;
    }
    for (int64_t r = warp; r < c.rows; r += warps)
        for (int64_t i = threadIdx.x % 32; i < words; i += 32) reinterpret_cast<W *>(c.p + r * c.pitch)[i] = zero;
}
__device__ __forceinline__ void clear_rows(const ClearArgs &c, int64_t block) {
    const int64_t per = blockDim.x / 32, warp = block * per + threadIdx.x / 32, warps = c.blocks * per;
    if (c.width == 16) clear_words(c, warp, warps, make_uint4(0, 0, 0, 0));
    else if (c.width == 4) clear_words(c, warp, warps, 0u);
    else clear_words(c, warp, warps, (unsigned short)0);
}

struct SortArgs {
    const void *ids;  // of the first digit
    const uint32_t *id_in, *pos_in;
    uint32_t *id_out, *pos_out;
    uint32_t *counts, *next;  // [tiles][bins] of this digit and the next
    int64_t n, V, clear;      // clear: words of later digits' counts behind the first's
    int shift, bits, next_shift, next_bits, tile, tiles;
    ClearArgs rows;
};

template <typename I>
__device__ __forceinline__ uint32_t label(const void *ids, int64_t i, int64_t V) {
    const int64_t id = (int64_t)__ldg(static_cast<const I *>(ids) + i);
    return id >= 0 && id < V ? (uint32_t)id : (uint32_t)V;
}

// Lanes of one digit, among those in `active`: what all its bits' votes leave. (match.any takes 85 cycles of an SM a warp; the votes of
// seven bits 20 issue slots.)
__device__ __forceinline__ unsigned alike(unsigned active, uint32_t digit, int bits) {
    unsigned same = active;
    for (int i = 0; i < bits; ++i) {
        const bool set = (digit >> i) & 1;
        const unsigned votes = __ballot_sync(0xffffffffu, set);
        same &= set ? votes : ~votes;
    }
    return same;
}

template <typename I>
__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(const SortArgs a) {
    __shared__ uint32_t count[kMostBins];
    const int bins = 1 << a.bits;
    grid_dependents_launch();
    for (int i = threadIdx.x; i < bins; i += kSortThreads) count[i] = 0;
    for (int64_t i = (int64_t)blockIdx.x * kSortThreads + threadIdx.x; i < a.clear; i += (int64_t)gridDim.x * kSortThreads) a.next[i] = 0;
    __syncthreads();
    const int64_t lo = (int64_t)blockIdx.x * a.tile, hi = lo + a.tile < a.n ? lo + a.tile : a.n;
    for (int64_t i = lo + threadIdx.x; i < hi; i += kSortThreads)
        atomicAdd(&count[label<I>(a.ids, i, a.V) & (bins - 1)], 1u);
    __syncthreads();
    for (int i = threadIdx.x; i < bins; i += kSortThreads) a.counts[(int64_t)blockIdx.x * bins + i] = count[i];
}

template <typename I, bool FIRST>
__global__ void __launch_bounds__(kSortThreads) sort_place_kernel(const SortArgs a) {
    __shared__ uint32_t place[kSortWarps][kMostBins];
    __shared__ uint32_t warp_total[kSortWarps];
    const int bins = 1 << a.bits, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    grid_dependents_launch();
    if ((int)blockIdx.x >= a.tiles) return clear_rows(a.rows, (int)blockIdx.x - a.tiles);
    for (int i = threadIdx.x; i < kSortWarps * bins; i += kSortThreads) place[i / bins][i % bins] = 0;
    grid_dependency_wait();
    __syncthreads();
    const int64_t seg = a.tile / kSortWarps, lo = (int64_t)blockIdx.x * a.tile + warp * seg;
    const int64_t hi = lo + seg < a.n ? lo + seg : a.n;
    auto digit = [&](int64_t i, uint32_t &id, uint32_t &pos) {
        id = FIRST ? label<I>(a.ids, i, a.V) : a.id_in[i];
        pos = FIRST ? (uint32_t)i : a.pos_in[i];
        return (id >> a.shift) & (uint32_t)(bins - 1);
    };
    for (int64_t base = lo; base < hi; base += 32) {
        const int64_t i = base + lane;
        const unsigned active = __ballot_sync(0xffffffffu, i < hi);
        uint32_t id, pos, d = 0;
        if (i < hi) d = digit(i, id, pos);
        const unsigned same = alike(active, d, a.bits);
        if (i < hi && (same & ((1u << lane) - 1)) == 0) place[warp][d] += __popc(same);
        __syncwarp();
    }
    __syncthreads();
    // a run of bins a thread: all of the digit, those of tiles before this one, and the exclusive sum of the first over the bins
    constexpr int kRun = kMostBins / kSortThreads;
    uint32_t total[kRun], earlier[kRun], sum = 0;
#pragma unroll
    for (int r = 0; r < kRun; ++r) {
        const int d = threadIdx.x * kRun + r;
        total[r] = earlier[r] = 0;
        if (d < bins)
            for (int t = 0; t < a.tiles; ++t) {
                const uint32_t c = a.counts[(int64_t)t * bins + d];
                total[r] += c;
                if (t < (int)blockIdx.x) earlier[r] += c;
            }
        sum += total[r];
    }
    uint32_t before = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(0xffffffffu, before, o);
        if (lane >= o) before += v;
    }
    if (lane == 31) warp_total[warp] = before;
    __syncthreads();
    before -= sum;
    for (int w = 0; w < warp; ++w) before += warp_total[w];
#pragma unroll
    for (int r = 0; r < kRun; ++r) {
        const int d = threadIdx.x * kRun + r;
        if (d < bins) {
            uint32_t at = before + earlier[r];
            for (int w = 0; w < kSortWarps; ++w) {
                const uint32_t c = place[w][d];
                place[w][d] = at;
                at += c;
            }
        }
        before += total[r];
    }
    __syncthreads();
    for (int64_t base = lo; base < hi; base += 32) {
        const int64_t i = base + lane;
        const unsigned active = __ballot_sync(0xffffffffu, i < hi);
        uint32_t id, pos, d = 0;
        if (i < hi) d = digit(i, id, pos);
        const unsigned same = alike(active, d, a.bits);
        const uint32_t first = place[warp][d];
        __syncwarp();
        if (i < hi) {
            const uint32_t to = first + __popc(same & ((1u << lane) - 1));
            if ((same & ((1u << lane) - 1)) == 0) place[warp][d] = first + __popc(same);
            a.id_out[to] = id;
            a.pos_out[to] = pos;
            if (a.next_bits)
                atomicAdd(&a.next[(int64_t)(to / (uint32_t)a.tile) * (1 << a.next_bits) + ((id >> a.next_shift) & ((1u << a.next_bits) - 1))], 1u);
        }
        __syncwarp();
    }
}

// The same in one launch, by a cluster of blocks, for what their shared memory holds: every block keeps its tile's labels and positions
// in registers from counting to placing; counts are read and places written across the cluster. 16000 labels of 14 bits: 8 us, by
// the kernels above 23 us (one block alone: 38 us).
constexpr int kOneThreads = 512, kOneWarps = kOneThreads / 32, kOneEach = 8, kOneTile = kOneThreads * kOneEach, kOneBlocks = 8;
constexpr int64_t kOneMost = (int64_t)kOneTile * kOneBlocks;
struct OneShared {
    uint32_t id[2][kOneTile], pos[2][kOneTile];
    uint32_t count[kMostBins];  // this tile's labels of a digit
    uint16_t place[kOneWarps][kMostBins];
    uint32_t first[kMostBins], warp_total[kOneWarps];
};
__device__ __forceinline__ uint32_t load_remote(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void store_remote(uint32_t addr, uint32_t v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
template <typename I>
__global__ void __launch_bounds__(kOneThreads, 1) sort_cluster_kernel(const SortArgs a, int passes) {
    extern __shared__ __align__(16) unsigned char raw[];
    OneShared &s = *reinterpret_cast<OneShared *>(raw);
    grid_dependents_launch();
    const int bins = 1 << a.bits, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int rank = (int)cluster_rank(), blocks = a.tiles, tile = a.tile;
    if ((int)blockIdx.x >= blocks) return clear_rows(a.rows, (int)blockIdx.x - blocks);  // (whole clusters)
    const int64_t left = a.n - (int64_t)rank * tile;
    const int n = left < tile ? (int)left : tile;  // of this block
    const int rounds = (tile + kOneThreads - 1) / kOneThreads, lo = warp * rounds * 32;
    uint32_t id[kOneEach], pos[kOneEach], earlier[kOneEach];
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = pass * a.bits, now = pass & 1;
        for (int i = lane; i < bins; i += 32) s.place[warp][i] = 0;
        __syncwarp();
#pragma unroll
        for (int r = 0; r < kOneEach; ++r) {
            const int i = lo + r * 32 + lane;
            if (r < rounds && i < n) {
                id[r] = pass == 0 ? label<I>(a.ids, (int64_t)rank * tile + i, a.V) : s.id[now][i];
                pos[r] = pass == 0 ? (uint32_t)(rank * tile + i) : s.pos[now][i];
            }
        }
#pragma unroll
        for (int r = 0; r < kOneEach; ++r) {
            const int i = lo + r * 32 + lane;
            if (r < rounds) {
                const unsigned active = __ballot_sync(0xffffffffu, i < n);
                const uint32_t d = i < n ? (id[r] >> shift) & (uint32_t)(bins - 1) : 0;
                const unsigned same = alike(active, d, a.bits), before = same & ((1u << lane) - 1);
                const uint32_t first = s.place[warp][d];
                __syncwarp();
                earlier[r] = first + __popc(before);
                if (i < n && before == 0) s.place[warp][d] = (uint16_t)(first + __popc(same));
                __syncwarp();
            }
        }
        __syncthreads();
        for (int d = threadIdx.x; d < bins; d += kOneThreads) {
            uint32_t sum = 0;
#pragma unroll
            for (int w = 0; w < kOneWarps; ++w) {
                const uint32_t c = s.place[w][d];
                s.place[w][d] = (uint16_t)sum;
                sum += c;
            }
            s.count[d] = sum;
        }
        __syncwarp();
        cluster_sync();
        // a bin a thread: its labels in all blocks and in those before this one, and the sum of the first over smaller bins
        uint32_t total = 0, mine = 0;
        if ((int)threadIdx.x < bins) {
            const uint32_t at = su32(&s.count[threadIdx.x]);
#pragma unroll
            for (int k = 0; k < kOneBlocks; ++k)
                if (k < blocks) {
                    const uint32_t c = load_remote(cluster_addr(at, (uint32_t)k));
                    total += c;
                    if (k < rank) mine += c;
                }
        }
        uint32_t before = total;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t v = __shfl_up_sync(0xffffffffu, before, o);
            if (lane >= o) before += v;
        }
        if (lane == 31) s.warp_total[warp] = before;
        __syncthreads();
        before += mine - total;
        if ((int)threadIdx.x < bins) {
            for (int w = 0; w < warp; ++w) before += s.warp_total[w];
            s.first[threadIdx.x] = before;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kOneEach; ++r)
            if (r < rounds && lo + r * 32 + lane < n) {
                const uint32_t d = (id[r] >> shift) & (uint32_t)(bins - 1), to = s.first[d] + s.place[warp][d] + earlier[r];
                if (pass + 1 < passes) {
                    const uint32_t block = to / (uint32_t)tile, i = to % (uint32_t)tile;
                    store_remote(cluster_addr(su32(&s.id[now ^ 1][i]), block), id[r]);
                    store_remote(cluster_addr(su32(&s.pos[now ^ 1][i]), block), pos[r]);
                } else {
                    a.id_out[to] = id[r], a.pos_out[to] = pos[r];
                }
            }
        __syncwarp();
        cluster_sync();  // (the last one: no block leaves while another may still read its counts)
    }
}

// ------------------------------------------------------------------------------------------------
// Gradient
// ------------------------------------------------------------------------------------------------

struct GradArgs {
    const void *grad;
    const uint32_t *id, *pos;  // [n], by label
    void *out;
    float *head, *tail;  // [chunks][D]: sums of runs that began before a chunk, and that go on behind it
    int64_t n, V, D, ldg, ldo, chunks, cols;  // cols: tiles of 32 lanes' runs
    float scale;
    int rounds;  // of 32 positions a chunk
    bool add;
};

constexpr int kGradThreads = 128, kJoinWarps = 8;

template <typename O, int W>
__device__ __forceinline__ void put(const GradArgs &a, int64_t row, int64_t col, const float (&sum)[W]) {
    O *p = static_cast<O *>(a.out) + row * a.ldo + col;
    Run<O, W> o;
    float f[W];
#pragma unroll
    for (int e = 0; e < W; ++e) f[e] = __fmul_rn(sum[e], a.scale);
    if (a.add) {
        o.load(p);
#pragma unroll
        for (int e = 0; e < W; ++e) f[e] = __fadd_rn(o.get(e), f[e]);
    }
    o.set(f);
    o.store(p);
}

// First of the n ascending labels that is not below (UPPER: that is above) id, by a whole warp: 32 probes a step.
template <bool UPPER>
__device__ __forceinline__ int64_t bound(const uint32_t *ids, int64_t lo, int64_t hi, uint32_t id) {
    const int lane = threadIdx.x % 32;
    while (lo < hi) {
        const int64_t step = (hi - lo + 31) / 32, at = lo + (lane + 1) * step - 1;  // last of the lane's share
        const bool under = at < hi && (UPPER ? ids[at] <= id : ids[at] < id);
        const int k = __popc(__ballot_sync(0xffffffffu, under));
        const int64_t a = lo + k * step, b = lo + (k + 1) * step;
        lo = a < hi ? a : hi;
        hi = b - 1 < hi ? (b - 1 > lo ? b - 1 : lo) : hi;
        if (step == 1) break;
    }
    return lo;
}

// A warp adds the rows of a chunk of sorted positions, 32 lanes' columns of them, in the order of the positions, kRows loads in
// flight. A run of one label that lies within the chunk is written out; what began before it or goes on behind it is kept for the
// second kernel. Rows that no position has were cleared while the labels were sorted. Bound: memory's latency, with few warps (1200 x 500:
// 13 us by itself), and its rate: 16000 x 2048 bf16 18 us.
constexpr int kRows = 4;  // (the whole call by 2, 4, 8, 16: 16000 x 2048 bf16 44, 41, 47, 46 us; 60000 x 512 fp32 81, 74, 75, 85)
template <typename T, typename O, int W>
__global__ void __launch_bounds__(kGradThreads) grad_sum_kernel(const GradArgs a) {
    const int lane = threadIdx.x % 32;
    grid_dependents_launch();  // (each kernel of the call waits for all of the one before)
    grid_dependency_wait();
    const int64_t warp = (int64_t)blockIdx.x * (kGradThreads / 32) + threadIdx.x / 32;
    const Split s = split(warp, a.cols);
    if (s.quot >= a.chunks) return;
    const int64_t lo = s.quot * 32 * a.rounds, hi = lo + 32 * a.rounds < a.n ? lo + 32 * a.rounds : a.n;
    const int64_t col = (s.rem * 32 + lane) * W;
    const bool mine = col < a.D;
    const uint32_t before = lo > 0 ? a.id[lo - 1] : 0xffffffffu, after = hi < a.n ? a.id[hi] : 0xffffffffu;
    float sum[W];
#pragma unroll
    for (int e = 0; e < W; ++e) sum[e] = 0.0f;
    bool first = true;  // the run that reaches the chunk's beginning
    uint32_t run = a.id[lo];
    auto end_run = [&](bool goes_on) {
        if (run < (uint32_t)a.V && mine) {
            const bool began = first && run == before;
            if (began || goes_on) {
                float *p = (began ? a.head : a.tail) + s.quot * a.D + col;
                Run<float, W> o;
                o.set(sum);
                o.store(p);
            } else {
                put<O, W>(a, run, col, sum);
            }
        }
        first = false;
#pragma unroll
        for (int e = 0; e < W; ++e) sum[e] = 0.0f;
    };
    for (int64_t base = lo; base < hi; base += 32) {
        const int count = hi - base < 32 ? (int)(hi - base) : 32;
        const uint32_t id = lane < count ? a.id[base + lane] : (uint32_t)a.V, pos = lane < count ? a.pos[base + lane] : 0;
        for (int j0 = 0; j0 < count; j0 += kRows) {
            Run<T, W> v[kRows];
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                const uint32_t i = __shfl_sync(0xffffffffu, id, j0 + j), p = __shfl_sync(0xffffffffu, pos, j0 + j);
                if (mine && i < (uint32_t)a.V) v[j].load(static_cast<const T *>(a.grad) + (int64_t)p * a.ldg + col);
                else v[j].clear();
            }
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                const uint32_t i = __shfl_sync(0xffffffffu, id, j0 + j);
                if (j0 + j < count) {
                    if (i != run) end_run(false), run = i;
#pragma unroll
                    for (int e = 0; e < W; ++e) sum[e] = __fadd_rn(sum[e], v[j].get(e));
                }
            }
        }
    }
    end_run(run == after);
}

// Runs over several chunks. A warp looks at one chunk (and 32 lanes' columns): where a run begins in it and goes on, it adds the sums
// of the chunks that hold the rest, in order. Runs over more than kLongRun chunks are left to all of the block's warps, which
// add a share of the chunks each, then the shares in order. 16000 x 2048: 12 us by itself, the search for a run's end and the sums of up to
// kLongRun chunks in turn.
constexpr int kLongRun = 32;
template <int W>
__device__ __forceinline__ void add_heads(const GradArgs &a, int64_t from, int64_t to, int64_t col, float (&sum)[W]) {
    for (int64_t i0 = from; i0 < to; i0 += 8) {
        Run<float, W> v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (i0 + j < to) v[j].load(a.head + (i0 + j) * a.D + col);
            else v[j].clear();
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int e = 0; e < W; ++e) sum[e] = __fadd_rn(sum[e], v[j].get(e));
    }
}
template <typename O, int W>
__global__ void __launch_bounds__(32 * kJoinWarps) grad_join_kernel(const GradArgs a) {
    __shared__ float share[kJoinWarps][32][W + 1];
    __shared__ int64_t more[kJoinWarps];  // further chunks of a warp's run, 0 where it has added them
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    grid_dependency_wait();
    const Split s = split((int64_t)blockIdx.x, a.cols);
    const int64_t chunk0 = s.quot * kJoinWarps, step = 32 * a.rounds;
    const int64_t col = (s.rem * 32 + lane) * W;
    const bool mine = col < a.D;
    {
        const int64_t chunk = chunk0 + warp, lo = chunk * step, hi = lo + step;
        int64_t left = 0;
        if (hi < a.n) {
            const uint32_t run = a.id[hi], last = a.id[hi - 1], first = a.id[lo], before = lo > 0 ? a.id[lo - 1] : 0xffffffffu;
            if (run < (uint32_t)a.V && last == run && !(first == run && before == run)) {
                left = (bound<true>(a.id, hi, a.n, run) - 1) / step - chunk;
                if (left <= kLongRun) {
                    if (mine) {
                        Run<float, W> v;
                        float sum[W];
                        v.load(a.tail + chunk * a.D + col);
#pragma unroll
                        for (int e = 0; e < W; ++e) sum[e] = v.get(e);
                        add_heads<W>(a, chunk + 1, chunk + 1 + left, col, sum);
                        put<O, W>(a, run, col, sum);
                    }
                    left = 0;
                }
            }
        }
        if (lane == 0) more[warp] = left;
    }
    __syncthreads();
    for (int w = 0; w < kJoinWarps; ++w) {
        const int64_t left = more[w], chunk = chunk0 + w;
        if (left == 0) continue;  // (of the block)
        float sum[W];
#pragma unroll
        for (int e = 0; e < W; ++e) sum[e] = 0.0f;
        if (mine) add_heads<W>(a, chunk + 1 + left * warp / kJoinWarps, chunk + 1 + left * (warp + 1) / kJoinWarps, col, sum);
#pragma unroll
        for (int e = 0; e < W; ++e) share[warp][lane][e] = sum[e];
        __syncthreads();
        if (warp == 0 && mine) {
            Run<float, W> v;
            v.load(a.tail + chunk * a.D + col);
#pragma unroll
            for (int e = 0; e < W; ++e) {
                sum[e] = v.get(e);
                for (int i = 0; i < kJoinWarps; ++i) sum[e] = __fadd_rn(sum[e], share[i][lane][e]);
            }
            put<O, W>(a, a.id[(chunk + 1) * step], col, sum);
        }
        __syncthreads();
    }
}

template <typename F>
cudaLaunchConfig_t after(F grid, int threads, cudaStream_t st, cudaLaunchAttribute *attr) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = st;
    attr->id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr->val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cfg;
}

struct SortPlan {
    int passes, bits, tile, tiles;
    bool one;       // by one cluster
    int64_t words;  // of 32 bits: labels and positions twice, counts of every digit
};
SortPlan sort_plan(int64_t n, int64_t V) {
    SortPlan p;
    int bits = 1;
    while ((V >> bits) != 0) ++bits;  // labels 0 .. V
    p.passes = (bits + kMostBits - 1) / kMostBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    const int64_t most = sm_count();  // tiles: every block reads all tiles' counts
    p.one = n <= kOneMost;
    p.tile = 1024;
    while ((n + p.tile - 1) / p.tile > (p.one ? kOneBlocks : most)) p.tile *= 2;
    p.tiles = (int)((n + p.tile - 1) / p.tile);
    p.words = 4 * n + (int64_t)p.passes * p.tiles * (1 << p.bits);
    return p;
}

// Leaves the labels in order and their positions in id, pos.
template <typename I>
qnn_status launch_sort(const void *ids, int64_t n, int64_t V, const SortPlan &p, const ClearArgs &rows, uint32_t *work,
                       const uint32_t **id, const uint32_t **pos, cudaStream_t st) {
    uint32_t *buf[2][2] = {{work, work + n}, {work + 2 * n, work + 3 * n}}, *counts = work + 4 * n;
    const int64_t each = (int64_t)p.tiles << p.bits;
    SortArgs a = {};
    a.ids = ids, a.n = n, a.V = V, a.tile = p.tile, a.tiles = p.tiles, a.bits = p.bits;
    a.counts = counts, a.next = counts + each, a.clear = (p.passes - 1) * each;
    a.rows = rows;
    if (p.one) {
        a.rows.blocks = (rows.blocks + p.tiles - 1) / p.tiles * p.tiles;
        a.id_out = buf[0][0], a.pos_out = buf[0][1];
        static_assert(sizeof(OneShared) <= 227 * 1024);
        QNN_CUDA_TRY(cudaFuncSetAttribute(sort_cluster_kernel<I>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(OneShared)));
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = (unsigned)p.tiles, attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cfg.gridDim = dim3((unsigned)(p.tiles + a.rows.blocks));
        cfg.blockDim = dim3(kOneThreads);
        cfg.dynamicSmemBytes = sizeof(OneShared);
        cfg.stream = st;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        QNN_CUDA_TRY(cudaLaunchKernelEx(&cfg, sort_cluster_kernel<I>, a, p.passes));
        *id = buf[0][0], *pos = buf[0][1];
        return QNN_OK;
    }
    sort_count_kernel<I><<<(unsigned)p.tiles, kSortThreads, 0, st>>>(a);
    QNN_CUDA_TRY(cudaGetLastError());
    for (int i = 0; i < p.passes; ++i) {
        a.counts = counts + i * each, a.next = a.counts + each;
        a.shift = i * p.bits, a.next_shift = a.shift + p.bits, a.next_bits = i + 1 < p.passes ? p.bits : 0;
        a.id_in = buf[i & 1][0], a.pos_in = buf[i & 1][1];
        a.id_out = buf[(i + 1) & 1][0], a.pos_out = buf[(i + 1) & 1][1];
        cudaLaunchAttribute attr;
        const cudaLaunchConfig_t cfg = after(p.tiles + (i == 0 ? rows.blocks : 0), kSortThreads, st, &attr);
        QNN_CUDA_TRY(i == 0 ? cudaLaunchKernelEx(&cfg, sort_place_kernel<I, true>, a) : cudaLaunchKernelEx(&cfg, sort_place_kernel<I, false>, a));
    }
    *id = buf[p.passes & 1][0], *pos = buf[p.passes & 1][1];
    return QNN_OK;
}

template <typename T, typename O, int W>
qnn_status launch_grad(GradArgs a, cudaStream_t st) {
    constexpr int kWarps = kGradThreads / 32;
    a.cols = (a.D / W + 31) / 32;
    const int64_t sums = (a.chunks * a.cols + kWarps - 1) / kWarps;
    cudaLaunchAttribute attr;
    cudaLaunchConfig_t cfg = after(sums, kGradThreads, st, &attr);
    QNN_CUDA_TRY(cudaLaunchKernelEx(&cfg, grad_sum_kernel<T, O, W>, a));
    if (a.chunks > 1) {
        cfg = after((a.chunks + kJoinWarps - 1) / kJoinWarps * a.cols, 32 * kJoinWarps, st, &attr);
        QNN_CUDA_TRY(cudaLaunchKernelEx(&cfg, grad_join_kernel<O, W>, a));
    }
    return QNN_OK;
}

template <typename T, typename O>
qnn_status launch_grad(const GradArgs &a, cudaStream_t st) {
    const int t = sizeof(T), o = sizeof(O);
    auto whole = [&](int v) { return a.D % v == 0 && runs_ok(a.grad, a.ldg, t, v) && runs_ok(a.out, a.ldo, o, v); };
    if constexpr (sizeof(T) == 2) {
        // (16 bytes a load where warps are many all the same: 16000 x 2048 43 us, so 50, 8000 x 1024 27 and 29, 2000 x 2048 29 and 28)
        if (whole(8) && a.chunks * (a.D / 256) >= 4 * (int64_t)sm_count()) return launch_grad<T, O, 8>(a, st);
    }
    if (whole(4)) return launch_grad<T, O, 4>(a, st);
    return launch_grad<T, O, 1>(a, st);
}

constexpr int64_t kMostIds = 1 << 30, kMostRows = INT32_MAX - 1;
bool rows_ok(const void *p, int64_t rows, int64_t D, int64_t ld, int e) {
    return ld >= D && reach_ok(rows, ld) && (reinterpret_cast<uintptr_t>(p) & (e - 1)) == 0;
}
Span rows_span(const void *p, int64_t rows, int64_t D, int64_t ld, int e) { return rows > 0 ? Span(p, ((rows - 1) * ld + D) * e) : Span(); }

}  // namespace
}  // namespace qnn

using namespace qnn;

extern "C" qnn_status qnn_embedding(const void *ids, int id_bytes, int64_t n, const void *table, int64_t ldt, int dtype, int64_t V,
                                    int64_t D, float scale, void *out, int64_t ldo, int out_dtype, void *stream) {
    if (!dtype_ok(dtype) || !dtype_ok(out_dtype) || (id_bytes != 4 && id_bytes != 8) || n < 0 || n > kMostIds || V < 1 ||
        V > kMostRows || D < 1 || D > INT32_MAX)
        return QNN_ERR_INVALID_ARG;
    const int e = dtype_size(dtype), eo = dtype_size(out_dtype);
    if (!rows_ok(table, V, D, ldt, e) || !rows_ok(out, n, D, ldo, eo) || (reinterpret_cast<uintptr_t>(ids) & (id_bytes - 1)))
        return QNN_ERR_INVALID_ARG;
    if (n == 0) return QNN_OK;
    if (!is_local_ptr(ids) || !is_local_ptr(table) || !is_local_ptr(out)) return QNN_ERR_INVALID_ARG;
    const Span os = rows_span(out, n, D, ldo, eo);
    if (os.meets(Span(ids, n * id_bytes)) || os.meets(rows_span(table, V, D, ldt, e))) return QNN_ERR_INVALID_ARG;
    EmbedArgs a = {};
    a.ids = ids, a.table = table, a.out = out, a.n = n, a.V = V, a.D = D, a.ldt = ldt, a.ldo = ldo, a.scale = scale;
    QNN_TRY(status_word(&a.status));
    cudaStream_t st = as_stream(stream);
    ProfScope prof("embedding", st);
    QNN_TRY(with_type(dtype, [&](auto t) {
        return with_type(out_dtype, [&](auto o) {
            return id_bytes == 4 ? launch_embed<decltype(t), decltype(o), int32_t>(a, st)
                                 : launch_embed<decltype(t), decltype(o), int64_t>(a, st);
        });
    }));
    QNN_CUDA_TRY(cudaGetLastError());
    return QNN_OK;
}

extern "C" qnn_status qnn_embedding_grad(const void *grad, int64_t ldg, int dtype, const void *ids, int id_bytes, int64_t n,
                                         int64_t V, int64_t D, float scale, int add, void *out, int64_t ldo, int out_dtype,
                                         void *stream) {
    if (!dtype_ok(dtype) || !dtype_ok(out_dtype) || (id_bytes != 4 && id_bytes != 8) || n < 0 || n > kMostIds || V < 1 ||
        V > kMostRows || D < 1 || D > INT32_MAX)
        return QNN_ERR_INVALID_ARG;
    const int e = dtype_size(dtype), eo = dtype_size(out_dtype);
    if (!rows_ok(grad, n, D, ldg, e) || !rows_ok(out, V, D, ldo, eo) || (reinterpret_cast<uintptr_t>(ids) & (id_bytes - 1)))
        return QNN_ERR_INVALID_ARG;
    if ((n > 0 && (!is_local_ptr(ids) || !is_local_ptr(grad))) || !is_local_ptr(out)) return QNN_ERR_INVALID_ARG;
    const Span os = rows_span(out, V, D, ldo, eo);
    if (n > 0 && (os.meets(Span(ids, n * id_bytes)) || os.meets(rows_span(grad, n, D, ldg, e)))) return QNN_ERR_INVALID_ARG;
    GradArgs a = {};
    a.grad = grad, a.out = out, a.n = n, a.V = V, a.D = D, a.ldg = ldg, a.ldo = ldo, a.scale = scale, a.add = add != 0;
    // chunks of 32 positions, of 128 from 2^17 on: a label that most positions have leaves that many sums to join
    a.rounds = n < 1 << 17 ? 1 : 4;
    a.chunks = (n + 32 * a.rounds - 1) / (32 * a.rounds);
    if (a.chunks > INT32_MAX / ((D + 31) / 32)) return QNN_ERR_INVALID_ARG;
    cudaStream_t st = as_stream(stream);
    ClearArgs clear = {};
    if (!add) {
        const uintptr_t bits = reinterpret_cast<uintptr_t>(out) | (uintptr_t)(D * eo) | (uintptr_t)(ldo * eo);
        clear.p = static_cast<char *>(out), clear.rows = V, clear.row = D * eo, clear.pitch = ldo * eo;
        clear.width = bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : 2;
        clear.blocks = (int)std::min<int64_t>((V * D * eo + 16383) / 16384, 2 * (int64_t)sm_count());
    }
    if (n == 0) {
        if (!add) QNN_CUDA_TRY(cudaMemset2DAsync(out, (size_t)clear.pitch, 0, (size_t)clear.row, (size_t)V, st));
        return QNN_OK;
    }
    Scratch scratch;
    {
        const SortPlan p = sort_plan(n, V);
        const size_t sums = (size_t)a.chunks * D * sizeof(float), sort = ((size_t)p.words * 4 + 255) / 256 * 256;
        const size_t half = (sums + 255) / 256 * 256;
        QNN_TRY(scratch.take(sort + 2 * half, st));
        char *base = static_cast<char *>(scratch.ptr());
        a.head = reinterpret_cast<float *>(base + sort), a.tail = reinterpret_cast<float *>(base + sort + half);
        ProfScope prof("embedding_sort", st);
        uint32_t *work = reinterpret_cast<uint32_t *>(base);
        QNN_TRY(id_bytes == 4 ? launch_sort<int32_t>(ids, n, V, p, clear, work, &a.id, &a.pos, st)
                              : launch_sort<int64_t>(ids, n, V, p, clear, work, &a.id, &a.pos, st));
    }
    ProfScope prof("embedding_grad", st);
    QNN_TRY(with_type(dtype, [&](auto t) {
        return with_type(out_dtype, [&](auto o) { return launch_grad<decltype(t), decltype(o)>(a, st); });
    }));
    QNN_CUDA_TRY(cudaGetLastError());
    return QNN_OK;
}
