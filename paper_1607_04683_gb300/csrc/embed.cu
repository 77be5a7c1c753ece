// embed.cu — embedding lookup with scaling, and its gradient by sorted labels, on sm_103a.
#include <algorithm>

#include "elem.cuh"
#include "qnn_device.cuh"
#include "qnn_host.h"

namespace qnn {
namespace {

bool runs_ok(const void *p, int64_t ld, int e, int v) { return reinterpret_cast<uintptr_t>(p) % (v * e) == 0 && ld % v == 0; }

// ------------------------------------------------------------------------------------------------
// Lookup
// ------------------------------------------------------------------------------------------------

struct EmbedArgs {
    const void *ids, *table;
    void *out;
    int64_t n, V, D, ldt, ldo, runs, items;
    float scale;
    int *status;
};

constexpr int kEmbedThreads = 128, kEmbedItems = 4;

// A thread takes kEmbedItems runs of W values of different rows, their loads in flight together.
// Bound: HBM for the output; rows that come again are read from L2.
template <typename T, typename O, typename I, int W>
__global__ void __launch_bounds__(kEmbedThreads) embed_kernel(const EmbedArgs a) {
    const int64_t all = (int64_t)gridDim.x * kEmbedThreads;
    for (int64_t at = (int64_t)blockIdx.x * kEmbedThreads + threadIdx.x; at < a.items; at += all * kEmbedItems) {
        Run<T, W> v[kEmbedItems];
        Split s[kEmbedItems];
        bool there[kEmbedItems];
#pragma unroll
        for (int i = 0; i < kEmbedItems; ++i) {
            const int64_t item = at + i * all;
            there[i] = false;
            if (item < a.items) {
                s[i] = split(item, a.runs);
                const int64_t id = (int64_t)__ldg(static_cast<const I *>(a.ids) + s[i].quot);
                there[i] = id >= 0 && id < a.V;
                if (id >= a.V && s[i].rem == 0) record_status(a.status, QNN_ERR_INVALID_ARG);
                if (there[i])
                    v[i].load(static_cast<const T *>(a.table) + id * a.ldt + s[i].rem * W);
                else
                    v[i].clear();
            }
        }
#pragma unroll
        for (int i = 0; i < kEmbedItems; ++i)
            if (at + i * all < a.items) {
                float f[W];
#pragma unroll
                for (int e = 0; e < W; ++e) f[e] = there[i] ? __fmul_rn(v[i].get(e), a.scale) : 0.0f;
                Run<O, W> o;
                o.set(f);
                o.store(static_cast<O *>(a.out) + s[i].quot * a.ldo + s[i].rem * W);
            }
    }
}

template <typename T, typename O, typename I, int W>
qnn_status launch_embed(EmbedArgs a, cudaStream_t st) {
    a.runs = a.D / W;
    a.items = a.n * a.runs;
    const int64_t per = kEmbedThreads * kEmbedItems;
    // (blocks of one item a thread while that leaves SMs without one)
    int64_t blocks = (a.items + per - 1) / per;
    if (blocks < 2 * (int64_t)sm_count()) blocks = (a.items + kEmbedThreads - 1) / kEmbedThreads;
    embed_kernel<T, O, I, W><<<(unsigned)std::min<int64_t>(blocks, 1 << 30), kEmbedThreads, 0, st>>>(a);
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
// segment of the tile a warp. A warp counts its segment's digits 32 positions at a time, lanes of one digit found by a match across
// the warp; a position's place is then the number of smaller digits, plus those of its own in the tiles, the warps' segments
// and the lanes before it. The next digit's counts by tile are whole numbers added in global memory as places are known, so that no order
// shows. Labels outside the table count as V and come last.
constexpr int kSortThreads = 256, kSortWarps = kSortThreads / 32, kMostBits = 9, kMostBins = 1 << kMostBits;
struct SortArgs {
    const void *ids;  // of the first digit
    const uint32_t *id_in, *pos_in;
    uint32_t *id_out, *pos_out;
    uint32_t *counts, *next;  // [tiles][bins] of this digit and the next
    int64_t n, V, clear;      // clear: words of later digits' counts behind the first's
    int shift, bits, next_shift, next_bits, tile, tiles;
};

template <typename I>
__device__ __forceinline__ uint32_t label(const void *ids, int64_t i, int64_t V) {
    const int64_t id = (int64_t)__ldg(static_cast<const I *>(ids) + i);
    return id >= 0 && id < V ? (uint32_t)id : (uint32_t)V;
}

template <typename I>
__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(const SortArgs a) {
    __shared__ uint32_t count[kMostBins];
    const int bins = 1 << a.bits;
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
        if (i < hi) {
            uint32_t id, pos;
            const uint32_t d = digit(i, id, pos);
            const unsigned same = __match_any_sync(active, d);
            if ((same & ((1u << lane) - 1)) == 0) place[warp][d] += __popc(same);
        }
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
        if (i < hi) {
            uint32_t id, pos;
            const uint32_t d = digit(i, id, pos);
            const unsigned same = __match_any_sync(active, d);
            const uint32_t first = place[warp][d];
            __syncwarp(active);
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

// ------------------------------------------------------------------------------------------------
// Gradient
// ------------------------------------------------------------------------------------------------

struct GradArgs {
    const void *grad;
    const uint32_t *id, *pos;  // [n], by label
    void *out;
    float *head, *tail;  // [chunks][D]: sums of runs that began before a chunk, and that go on behind it
    int64_t n, V, D, ldg, ldo, chunks, cols, sums;  // cols: tiles of 32 lanes' runs; sums: blocks that add, the others clear
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

// A warp adds the rows of a chunk of sorted positions, 32 lanes' columns of them, in the order of the positions, eight loads in
// flight. A run of one label that lies within the chunk is written out; what began before it or goes on behind it is kept for the
// second kernel. The blocks behind write zeros where no position has the label.
template <typename T, typename O, int W>
__global__ void __launch_bounds__(kGradThreads) grad_sum_kernel(const GradArgs a) {
    const int lane = threadIdx.x % 32;
    grid_dependency_wait();
    const int64_t warp = ((int64_t)blockIdx.x - (blockIdx.x < a.sums ? 0 : a.sums)) * (kGradThreads / 32) + threadIdx.x / 32;
    if (blockIdx.x >= a.sums) {
        const int64_t row0 = warp * 32;
        if (row0 >= a.V) return;
        const int64_t row = row0 + lane;
        bool absent = false;
        if (row < a.V) {
            int64_t lo = 0, hi = a.n;
            while (lo < hi) {
                const int64_t mid = (lo + hi) / 2;
                if (a.id[mid] < (uint32_t)row) lo = mid + 1;
                else hi = mid;
            }
            absent = lo == a.n || a.id[lo] != (uint32_t)row;
        }
        unsigned rows = __ballot_sync(0xffffffffu, absent);
        Run<O, W> zero;
        zero.clear();
        while (rows) {
            const int r = __ffs(rows) - 1;
            rows &= rows - 1;
            for (int64_t c = lane; c < a.D / W; c += 32) zero.store(static_cast<O *>(a.out) + (row0 + r) * a.ldo + c * W);
        }
        return;
    }
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
        for (int j0 = 0; j0 < count; j0 += 8) {
            Run<T, W> v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t i = __shfl_sync(0xffffffffu, id, j0 + j), p = __shfl_sync(0xffffffffu, pos, j0 + j);
                if (mine && i < (uint32_t)a.V) v[j].load(static_cast<const T *>(a.grad) + (int64_t)p * a.ldg + col);
                else v[j].clear();
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
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

// Runs over several chunks: a block for each chunk (and 32 lanes' columns) in which one begins. Its warps add the chunks' sums in
// kJoinWarps shares, then the shares are added, in the order of the positions.
template <typename O, int W>
__global__ void __launch_bounds__(32 * kJoinWarps) grad_join_kernel(const GradArgs a) {
    __shared__ float share[kJoinWarps][32][W + 1];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    grid_dependency_wait();
    const Split s = split((int64_t)blockIdx.x, a.cols);
    const int64_t chunk = s.quot, step = 32 * a.rounds, lo = chunk * step, hi = lo + step;
    if (hi >= a.n) return;
    const uint32_t run = a.id[hi];
    if (run >= (uint32_t)a.V || a.id[hi - 1] != run || (a.id[lo] == run && lo > 0 && a.id[lo - 1] == run)) return;
    const int64_t end = bound<true>(a.id, hi, a.n, run);  // first position behind the run
    const int64_t chunks = (end - 1) / step - chunk;      // further chunks that hold some of it
    const int64_t col = (s.rem * 32 + lane) * W;
    const bool mine = col < a.D;
    const int64_t from = chunks * warp / kJoinWarps, to = chunks * (warp + 1) / kJoinWarps;
    float sum[W];
#pragma unroll
    for (int e = 0; e < W; ++e) sum[e] = 0.0f;
    if (mine) {
        for (int64_t i0 = from; i0 < to; i0 += 8) {
            Run<float, W> v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (i0 + j < to) v[j].load(a.head + (chunk + 1 + i0 + j) * a.D + col);
                else v[j].clear();
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int e = 0; e < W; ++e) sum[e] = __fadd_rn(sum[e], v[j].get(e));
        }
    }
#pragma unroll
    for (int e = 0; e < W; ++e) share[warp][lane][e] = sum[e];
    __syncthreads();
    if (warp || !mine) return;
    Run<float, W> v;
    v.load(a.tail + chunk * a.D + col);
#pragma unroll
    for (int e = 0; e < W; ++e) {
        sum[e] = v.get(e);
        for (int w = 0; w < kJoinWarps; ++w) sum[e] = __fadd_rn(sum[e], share[w][lane][e]);
    }
    put<O, W>(a, run, col, sum);
}

// No positions: zeros.
template <typename O, int W>
__global__ void __launch_bounds__(kGradThreads) grad_clear_kernel(const GradArgs a) {
    Run<O, W> zero;
    zero.clear();
    const int64_t runs = a.D / W, all = a.V * runs;
    for (int64_t i = (int64_t)blockIdx.x * kGradThreads + threadIdx.x; i < all; i += (int64_t)gridDim.x * kGradThreads) {
        const Split s = split(i, runs);
        zero.store(static_cast<O *>(a.out) + s.quot * a.ldo + s.rem * W);
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
    int64_t words;  // of 32 bits: labels and positions twice, counts of every digit
};
SortPlan sort_plan(int64_t n, int64_t V) {
    SortPlan p;
    int bits = 1;
    while ((V >> bits) != 0) ++bits;  // labels 0 .. V
    p.passes = (bits + kMostBits - 1) / kMostBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    const int64_t most = sm_count();  // tiles: every block reads all tiles' counts
    p.tile = 1024;
    while ((n + p.tile - 1) / p.tile > most) p.tile *= 2;
    p.tiles = (int)((n + p.tile - 1) / p.tile);
    p.words = 4 * n + (int64_t)p.passes * p.tiles * (1 << p.bits);
    return p;
}

// Leaves the labels in order and their positions in id, pos.
template <typename I>
qnn_status launch_sort(const void *ids, int64_t n, int64_t V, const SortPlan &p, uint32_t *work, const uint32_t **id,
                       const uint32_t **pos, cudaStream_t st) {
    uint32_t *buf[2][2] = {{work, work + n}, {work + 2 * n, work + 3 * n}}, *counts = work + 4 * n;
    const int64_t each = (int64_t)p.tiles << p.bits;
    SortArgs a = {};
    a.ids = ids, a.n = n, a.V = V, a.tile = p.tile, a.tiles = p.tiles, a.bits = p.bits;
    a.counts = counts, a.next = counts + each, a.clear = (p.passes - 1) * each;
    sort_count_kernel<I><<<(unsigned)p.tiles, kSortThreads, 0, st>>>(a);
    QNN_CUDA_TRY(cudaGetLastError());
    for (int i = 0; i < p.passes; ++i) {
        a.counts = counts + i * each, a.next = a.counts + each;
        a.shift = i * p.bits, a.next_shift = a.shift + p.bits, a.next_bits = i + 1 < p.passes ? p.bits : 0;
        a.id_in = buf[i & 1][0], a.pos_in = buf[i & 1][1];
        a.id_out = buf[(i + 1) & 1][0], a.pos_out = buf[(i + 1) & 1][1];
        cudaLaunchAttribute attr;
        const cudaLaunchConfig_t cfg = after(p.tiles, kSortThreads, st, &attr);
        QNN_CUDA_TRY(i == 0 ? cudaLaunchKernelEx(&cfg, sort_place_kernel<I, true>, a) : cudaLaunchKernelEx(&cfg, sort_place_kernel<I, false>, a));
    }
    *id = buf[p.passes & 1][0], *pos = buf[p.passes & 1][1];
    return QNN_OK;
}

template <typename T, typename O, int W>
qnn_status launch_grad(GradArgs a, cudaStream_t st) {
    if (a.n == 0) {
        const int64_t blocks = std::min<int64_t>((a.V * (a.D / W) + kGradThreads - 1) / kGradThreads, 16 * (int64_t)sm_count());
        if (!a.add) grad_clear_kernel<O, W><<<(unsigned)blocks, kGradThreads, 0, st>>>(a);
        return QNN_OK;
    }
    constexpr int kWarps = kGradThreads / 32;
    a.cols = (a.D / W + 31) / 32;
    a.sums = (a.chunks * a.cols + kWarps - 1) / kWarps;
    const int64_t clears = a.add ? 0 : ((a.V + 31) / 32 + kWarps - 1) / kWarps;
    if (a.sums + clears > INT32_MAX || a.chunks * a.cols > INT32_MAX) return QNN_FAIL(QNN_ERR_INVALID_ARG);
    cudaLaunchAttribute attr;
    cudaLaunchConfig_t cfg = after(a.sums + clears, kGradThreads, st, &attr);
    QNN_CUDA_TRY(cudaLaunchKernelEx(&cfg, grad_sum_kernel<T, O, W>, a));
    if (a.chunks > 1) {
        cfg = after(a.chunks * a.cols, 32 * kJoinWarps, st, &attr);
        QNN_CUDA_TRY(cudaLaunchKernelEx(&cfg, grad_join_kernel<O, W>, a));
    }
    return QNN_OK;
}

template <typename T, typename O>
qnn_status launch_grad(const GradArgs &a, cudaStream_t st) {
    const int t = sizeof(T), o = sizeof(O);
    auto whole = [&](int v) { return a.D % v == 0 && runs_ok(a.grad, a.ldg, t, v) && runs_ok(a.out, a.ldo, o, v); };
    if constexpr (sizeof(T) == 2) {
        if (whole(8)) return launch_grad<T, O, 8>(a, st);
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
    cudaStream_t st = as_stream(stream);
    Scratch scratch;
    if (n > 0) {
        const SortPlan p = sort_plan(n, V);
        const size_t sums = (size_t)a.chunks * D * sizeof(float), sort = ((size_t)p.words * 4 + 255) / 256 * 256;
        const size_t half = (sums + 255) / 256 * 256;
        QNN_TRY(scratch.take(sort + 2 * half, st));
        char *base = static_cast<char *>(scratch.ptr());
        a.head = reinterpret_cast<float *>(base + sort), a.tail = reinterpret_cast<float *>(base + sort + half);
        ProfScope prof("embedding_sort", st);
        uint32_t *work = reinterpret_cast<uint32_t *>(base);
        QNN_TRY(id_bytes == 4 ? launch_sort<int32_t>(ids, n, V, p, work, &a.id, &a.pos, st)
                              : launch_sort<int64_t>(ids, n, V, p, work, &a.id, &a.pos, st));
    }
    ProfScope prof("embedding_grad", st);
    QNN_TRY(with_type(dtype, [&](auto t) {
        return with_type(out_dtype, [&](auto o) { return launch_grad<decltype(t), decltype(o)>(a, st); });
    }));
    QNN_CUDA_TRY(cudaGetLastError());
    return QNN_OK;
}
