// beam.cu — one step of a beam search on sm_103a: the best continuations over beams and classes, and the carried states
// of the beams that were kept.
#include <algorithm>
#include <cfloat>

#include "elem.cuh"
#include "qnn_device.cuh"
#include "qnn_host.h"

namespace qnn {
namespace {

constexpr int kMostKept = 128, kMostBeams = 128;

// ------------------------------------------------------------------------------------------------
// The n best of what a block's threads hold
// ------------------------------------------------------------------------------------------------

// A candidate: larger ones first, 0 none. The value in an order-preserving form, above it the index's complement, so that
// of equal values the lowest index is the largest candidate and no two are equal.
using Logit = unsigned long long;  // 32 bits of a logit, 32 of ~index
struct Cand {                      // a score in 64 bits
    unsigned long long v;
    unsigned index;
};
__device__ __forceinline__ bool before(Logit a, Logit b) { return a > b; }
__device__ __forceinline__ bool before(const Cand &a, const Cand &b) { return a.v > b.v || (a.v == b.v && a.index < b.index); }
__device__ __forceinline__ bool some(Logit a) { return a != 0; }
__device__ __forceinline__ bool some(const Cand &a) { return a.v != 0; }
__device__ __forceinline__ Logit none_of(Logit) { return 0; }
__device__ __forceinline__ Cand none_of(Cand) { return {0, 0xffffffffu}; }

__device__ __forceinline__ Logit logit_key(float v, unsigned index) {
    const uint32_t b = __float_as_uint(__fadd_rn(v, 0.0f));  // (-0 is 0)
    const uint32_t o = b ^ ((int32_t)b < 0 ? 0xffffffffu : 0x80000000u);
    return v > -INFINITY ? (Logit)o << 32 | (uint32_t)~index : 0;  // (a NaN is none either)
}
__device__ __forceinline__ float logit_of(Logit k) {
    const uint32_t o = (uint32_t)(k >> 32);
    return __uint_as_float(o ^ ((int32_t)o < 0 ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ Cand cand_key(double v, unsigned index) {
    if (!(v > -INFINITY)) return none_of(Cand());
    const unsigned long long b = (unsigned long long)__double_as_longlong(v + 0.0);
    return {b ^ ((long long)b < 0 ? ~0ull : 1ull << 63), index};
}
__device__ __forceinline__ double cand_of(const Cand &c) {
    return __longlong_as_double((long long)(c.v ^ ((long long)c.v < 0 ? 1ull << 63 : ~0ull)));
}

// The n best candidates so far, best first. A block of kThreads threads brings kEach candidates a thread at a time. Only those
// better than the n-th best so far count, and where more than n threads have one, those no worse than the n-th best of the
// threads' bests: n threads at most, so that n kEach + n are ever ranked. A candidate's rank is the number of better ones,
// counted by one thread: no order of arrival shows in the result.
constexpr int kThreads = 256, kEach = 8;
template <typename K>
struct Best {
    K list[kMostKept * (kEach + 1)];
    K ranked[kMostKept];
    K bests[kThreads];
    K last;  // the n-th best, or none
    K least;
    int count, held;

    __device__ __forceinline__ void start() {
        if (threadIdx.x == 0) count = 0, held = 0, last = none_of(K());
        __syncthreads();
    }
    // mine: the best of key[]. All threads call it; ends behind a barrier.
    __device__ __forceinline__ void take(const K (&key)[kEach], const K &mine, int n) {
        const K bar = last;
        const bool pass = before(mine, bar);
        const int threads = __syncthreads_count(pass);
        if (threads == 0) return;
        K from = bar;
        bool with = false;  // `from` itself counts
        if (threads > n) {
            bests[threadIdx.x] = pass ? mine : none_of(K());
            __syncthreads();
            if (pass) {
                int better = 0;
#pragma unroll 8
                for (int i = 0; i < kThreads; ++i) better += before(bests[i], mine);
                if (better == n - 1) least = mine;
            }
            __syncthreads();
            from = least, with = true;
        }
        if (pass && (with ? !before(from, mine) : true)) {
#pragma unroll
            for (int e = 0; e < kEach; ++e)
                if (some(key[e]) && (with ? !before(from, key[e]) : before(key[e], from))) list[atomicAdd(&count, 1)] = key[e];
        }
        __syncthreads();
        const int m = count;
        for (int i = threadIdx.x; i < m; i += kThreads) {
            const K k = list[i];
            int better = 0;
#pragma unroll 4
            for (int j = 0; j < m; ++j) better += before(list[j], k);
            if (better < n) ranked[better] = k;
        }
        __syncthreads();
        const int h = m < n ? m : n;
        for (int i = threadIdx.x; i < h; i += kThreads) list[i] = ranked[i];
        if (threadIdx.x == 0) {
            count = held = h;
            if (h == n) last = ranked[n - 1];
        }
        __syncthreads();
    }
};

// ------------------------------------------------------------------------------------------------
// Selection
// ------------------------------------------------------------------------------------------------

// Of a part of a row: its largest value and the sum of exp(value - largest) as a whole number of 2^-32 (exact sums
// of the threads' fp32 ones, in any order; ~0: not a number).
struct RowPart {
    unsigned long long sum;
    float most;
    int held;
};

struct SelectArgs {
    const void *logits;
    int64_t ldl;
    const float *scores;
    const uint8_t *finished;
    float *scores_out;
    int32_t *parents, *tokens;
    Logit *keys;     // [rows][parts][n]
    RowPart *parts_of;  // [rows][parts]
    int64_t K, V, per;  // per: classes of a part
    int n, parts, eos;
};

// exp(d) for d <= 0 by the hardware's exponential, its argument's product with log2(e) in two terms: log2(e) rounded to 24
// bits alone moves exp(-8) by 1e-7, always the same way. kBias takes out the instruction's own (it lies low by about 2e-8), so that
// sums of many terms are right to about 1e-8 and two beams' continuations that close are still told apart.
constexpr float kLog2eRest = 1.925963033500e-08f, kBias = 2e-8f;
__device__ __forceinline__ float exp_term(float d) { return exp2_hw(__fmaf_rn(d, kLog2eRest, __fmaf_rn(d, kLog2e, kBias))); }

template <typename T, bool VEC>
__device__ __forceinline__ void load_tile(const T *row, int64_t base, int64_t end, float (&v)[kEach]) {
    if constexpr (VEC) {
        const int64_t at = base + (int64_t)threadIdx.x * kEach;
        Run<T, kEach> r;
        if (at + kEach <= end) {
            r.load(row + at);
        } else {
            r.load_some(row + at, at < end ? (int)(end - at) : 0);
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e) v[e] = at + e < end ? r.get(e) : -INFINITY;
    } else {
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int64_t at = base + threadIdx.x + (int64_t)e * kThreads;
            v[e] = at < end ? to_f32(row[at]) : -INFINITY;
        }
    }
}

// One part of a beam's row: its sum of exponentials and its n best classes in one pass over it, each thread's running maximum
// and sum in registers. Within a beam the order of the logits is that of the scores, so that no score is formed here.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) beam_rows_kernel(const SelectArgs a) {
    __shared__ Best<Logit> best;
    __shared__ float warp_most[kThreads / 32];
    __shared__ unsigned long long warp_sum[kThreads / 32];
    const int64_t row = blockIdx.x / (unsigned)a.parts;
    const int part = blockIdx.x % (unsigned)a.parts;
    RowPart *out = a.parts_of + row * a.parts + part;
    const float score = a.scores[row];
    if ((a.finished && a.finished[row]) || !(score > -INFINITY)) return;  // (nothing of this row is looked at)
    const T *x = static_cast<const T *>(a.logits) + row * a.ldl;
    const int64_t lo = part * a.per, hi = lo + a.per < a.V ? lo + a.per : a.V;
    float v[kEach], most = -INFINITY, sum = 0.0f;
    load_tile<T, VEC>(x, lo, hi, v);
    best.start();
    for (int64_t base = lo; base < hi; base += kThreads * kEach) {
        float next[kEach];
        if (base + kThreads * kEach < hi) load_tile<T, VEC>(x, base + kThreads * kEach, hi, next);
        float top = v[0];
#pragma unroll
        for (int e = 1; e < kEach; ++e) top = fmaxf(top, v[e]);
        if (top > most) sum = __fmul_rn(sum, exp_term(__fsub_rn(most, top))), most = top;
        const float from = most > -INFINITY ? most : 0.0f;
#pragma unroll
        for (int e = 0; e < kEach; ++e) sum = __fadd_rn(sum, exp_term(__fsub_rn(v[e], from)));
        Logit key[kEach], mine = 0;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            key[e] = logit_key(v[e], (unsigned)(VEC ? base + threadIdx.x * kEach + e : base + threadIdx.x + e * kThreads));
            mine = key[e] > mine ? key[e] : mine;
        }
        best.take(key, mine, a.n);
#pragma unroll
        for (int e = 0; e < kEach; ++e) v[e] = next[e];
    }
    // the block's maximum, then the sums' parts of it
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    float m = warp_max(most);
    if (lane == 0) warp_most[warp] = m;
    __syncthreads();
    m = warp_most[0];
#pragma unroll
    for (int i = 1; i < kThreads / 32; ++i) m = fmaxf(m, warp_most[i]);
    const float share = most > -INFINITY ? __fmul_rn(sum, exp_term(__fsub_rn(most, m))) : sum;  // (NaNs pass through)
    const bool bad = !(share >= 0.0f && share < INFINITY);
    unsigned long long s = bad ? 0 : __float2ull_rn(__fmul_rn(share, 4294967296.0f));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) warp_sum[warp] = s;
    const int any_bad = __syncthreads_or(bad);
    const int held = best.held;
    Logit *keys = a.keys + (row * a.parts + part) * a.n;
    for (int i = threadIdx.x; i < held; i += kThreads) keys[i] = best.list[i];
    if (threadIdx.x == 0) {
        s = 0;
        for (int i = 0; i < kThreads / 32; ++i) s += warp_sum[i];
        *out = {any_bad ? ~0ull : s, m, held};
    }
    grid_dependents_launch();
}

// A batch row's continuations: each beam's log of its sum in 64 bits from its parts, then the n best of the parts' lists.
__global__ void __launch_bounds__(kThreads) beam_merge_kernel(const SelectArgs a) {
    __shared__ Best<Cand> best;
    __shared__ double lse[kMostBeams];
    __shared__ unsigned char state[kMostBeams];  // 0: no candidates, 1: its parts' lists, 2: finished
    __shared__ float score[kMostBeams];
    const int64_t b = blockIdx.x;
    const int K = (int)a.K;
    grid_dependency_wait();
    for (int k = threadIdx.x; k < K; k += kThreads) {
        const int64_t row = b * K + k;
        const float sc = a.scores[row];
        int st = 0;
        double l = 0.0;
        if (sc > -INFINITY) {
            if (a.finished && a.finished[row]) {
                st = 2;
            } else {
                const RowPart *p = a.parts_of + row * a.parts;
                float m = -INFINITY;
                bool bad = false;
                for (int i = 0; i < a.parts; ++i) m = fmaxf(m, p[i].most), bad |= p[i].sum == ~0ull;
                double s = 0.0;
                if (!bad && m > -INFINITY && m < INFINITY) {
                    for (int i = 0; i < a.parts; ++i) {
                        const double share = (double)p[i].sum * 0x1p-32;
                        if (p[i].most > -INFINITY) s += p[i].most == m ? share : share * exp((double)p[i].most - (double)m);
                    }
                    l = (double)m + log(s);
                    st = 1;
                }
            }
        }
        lse[k] = l, state[k] = (unsigned char)st, score[k] = sc;
    }
    best.start();
    const int64_t lists = (int64_t)K * a.parts, total = lists * a.n;
    for (int64_t base = 0; base < total; base += kThreads * kEach) {
        Cand key[kEach], mine = none_of(Cand());
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int64_t at = base + threadIdx.x + (int64_t)e * kThreads;
            key[e] = none_of(Cand());
            if (at < total) {
                const unsigned list = (unsigned)at / (unsigned)a.n, i = (unsigned)at % (unsigned)a.n;
                const int k = (int)(list / (unsigned)a.parts), part = (int)(list % (unsigned)a.parts);
                const int64_t row = b * K + k;
                if (state[k] == 2) {
                    if (part == 0 && i == 0) key[e] = cand_key((double)score[k], (unsigned)(k * a.V + a.eos));
                } else if (state[k] == 1 && (int)i < a.parts_of[row * a.parts + part].held) {
                    const Logit l = a.keys[(row * a.parts + part) * a.n + i];
                    key[e] = cand_key((double)score[k] + ((double)logit_of(l) - lse[k]), (unsigned)(k * a.V + (unsigned)~(uint32_t)l));
                }
            }
            if (before(key[e], mine)) mine = key[e];
        }
        best.take(key, mine, a.n);
    }
    const int held = best.held;
    for (int i = threadIdx.x; i < a.n; i += kThreads) {
        const int64_t o = b * a.n + i;
        if (i < held) {
            const Cand c = best.list[i];
            a.scores_out[o] = (float)cand_of(c);
            a.parents[o] = (int32_t)(c.index / (unsigned)a.V);
            a.tokens[o] = (int32_t)(c.index % (unsigned)a.V);
        } else {
            a.scores_out[o] = -INFINITY;
            a.parents[o] = 0;
            a.tokens[o] = a.eos;
        }
    }
}

template <typename T>
qnn_status launch_select(SelectArgs a, int64_t rows, int64_t B, cudaStream_t st) {
    const bool vec = reinterpret_cast<uintptr_t>(a.logits) % 16 == 0 && a.ldl * (int64_t)sizeof(T) % 16 == 0;
    const auto kern = vec ? beam_rows_kernel<T, true> : beam_rows_kernel<T, false>;
    kern<<<(unsigned)(rows * a.parts), kThreads, 0, st>>>(a);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)B);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    QNN_CUDA_TRY(cudaGetLastError());
    QNN_CUDA_TRY(cudaLaunchKernelEx(&cfg, beam_merge_kernel, a));
    return QNN_OK;
}

// ------------------------------------------------------------------------------------------------
// Reordering
// ------------------------------------------------------------------------------------------------

constexpr int kStatesALaunch = 16, kReorderThreads = 128;
struct ReorderState {
    const char *in;
    char *out;
    int64_t words;  // of a row, in the launch's words
    int64_t items;  // outer * B * words before this state's, of the launch
};
struct ReorderArgs {
    ReorderState s[kStatesALaunch];
    const int32_t *parents;
    int64_t B, K, n, items;
    int count;
    int *status;
};

// A thread takes one word of every beam of a batch row: it has loaded all that it needs of up to NB beams before it stores
// the first of them, so that states may be reordered in place (n <= NB then). A beam that is its own parent in place is left alone.
template <typename W, int NB>
__global__ void __launch_bounds__(kReorderThreads) beam_reorder_kernel(const ReorderArgs a) {
    for (int64_t item = (int64_t)blockIdx.x * kReorderThreads + threadIdx.x; item < a.items; item += (int64_t)gridDim.x * kReorderThreads) {
        int i = 0;
        while (i + 1 < a.count && item >= a.s[i + 1].items) ++i;
        const ReorderState &s = a.s[i];
        const Split at = split(item - s.items, s.words), ob = split(at.quot, a.B);  // (of outer * B + b: ob.quot outer, ob.rem b)
        const W *in = reinterpret_cast<const W *>(s.in) + at.quot * a.K * s.words + at.rem;
        W *out = reinterpret_cast<W *>(s.out) + at.quot * a.n * s.words + at.rem;
        const int32_t *parents = a.parents + ob.rem * a.n;
        const bool same = s.in == s.out;
        for (int64_t j0 = 0; j0 < a.n; j0 += NB) {
            W v[NB];
            bool moved[NB];
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                moved[j] = false;
                if (j0 + j < a.n) {
                    const int p = __ldg(parents + j0 + j);
                    if (p >= 0 && p < a.K) {
                        moved[j] = !(same && p == j0 + j);
                        if (moved[j]) v[j] = in[p * s.words];
                    } else if (at.rem == 0) {
                        record_status(a.status, QNN_ERR_INVALID_ARG);
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < NB; ++j)
                if (moved[j]) out[(j0 + j) * s.words] = v[j];
        }
    }
}

template <typename W, int NB>
qnn_status launch_reorder(const ReorderArgs &a, cudaStream_t st) {
    const int64_t blocks = std::min<int64_t>((a.items + kReorderThreads - 1) / kReorderThreads, 64 * (int64_t)sm_count());
    beam_reorder_kernel<W, NB><<<(unsigned)blocks, kReorderThreads, 0, st>>>(a);
    return QNN_OK;
}

template <typename W>
qnn_status launch_reorder(const ReorderArgs &a, bool in_place, cudaStream_t st) {
    if (a.n <= 4) return launch_reorder<W, 4>(a, st);
    if (a.n <= 8 || !in_place) return launch_reorder<W, 8>(a, st);
    if (a.n <= 16) return launch_reorder<W, 16>(a, st);
    return QNN_ERR_INVALID_ARG;  // (the caller took narrower words)
}

}  // namespace
}  // namespace qnn

using namespace qnn;

extern "C" qnn_status qnn_beam_select(const void *logits, int64_t ldl, int dtype, const float *scores, const uint8_t *finished,
                                      int64_t B, int64_t K, int64_t V, int32_t n, int32_t eos, float *scores_out,
                                      int32_t *parents, int32_t *tokens, void *stream) {
    if (!dtype_ok(dtype) || B < 0 || K < 1 || K > kMostBeams || V < 1 || V > INT32_MAX / K || n < 1 || n > kMostKept || eos < 0 ||
        eos >= V || ldl < V || B > INT32_MAX / K || !reach_ok(B * K, ldl))
        return QNN_ERR_INVALID_ARG;
    const int e = dtype_size(dtype);
    if ((reinterpret_cast<uintptr_t>(logits) & (e - 1)) || !aligned4(scores) || !aligned4(scores_out) || !aligned4(parents) ||
        !aligned4(tokens))
        return QNN_ERR_INVALID_ARG;
    if (B == 0) return QNN_OK;
    if (!is_local_ptr(logits) || !is_local_ptr(scores) || !local_or_null(finished) || !is_local_ptr(scores_out) ||
        !is_local_ptr(parents) || !is_local_ptr(tokens))
        return QNN_ERR_INVALID_ARG;
    const Span in[3] = {Span(logits, ((B * K - 1) * ldl + V) * e), Span(finished, B * K), Span(scores, 4 * B * K)};
    const Span out[3] = {Span(scores_out, 4 * B * n), Span(parents, 4 * B * n), Span(tokens, 4 * B * n)};
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < 3; ++j)  // (a batch row's scores are read before its own are written)
            if (out[i].meets(in[j]) && !(i == 0 && j == 2 && scores_out == scores && n == K)) return QNN_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (out[i].meets(out[j])) return QNN_ERR_INVALID_ARG;
    }
    SelectArgs a;
    a.logits = logits, a.ldl = ldl, a.scores = scores, a.finished = finished, a.scores_out = scores_out, a.parents = parents;
    a.tokens = tokens, a.K = K, a.V = V, a.n = n, a.eos = eos;
    // parts of a row: two tiles or more, while the SMs have fewer than four blocks each
    const int64_t rows = B * K, tile = kThreads * kEach, tiles = (V + tile - 1) / tile;
    int64_t parts = std::max<int64_t>(1, std::min<int64_t>({4 * (int64_t)sm_count() / rows, (tiles + 1) / 2, 32}));
    const int64_t per = (tiles + parts - 1) / parts;
    parts = (tiles + per - 1) / per;
    if (rows * parts > INT32_MAX) return QNN_ERR_INVALID_ARG;
    a.parts = (int)parts, a.per = per * tile;
    cudaStream_t st = as_stream(stream);
    Scratch scratch;
    const size_t keys = (size_t)(rows * parts * n) * sizeof(Logit);
    QNN_TRY(scratch.take(keys + (size_t)(rows * parts) * sizeof(RowPart), st));
    a.keys = static_cast<Logit *>(scratch.ptr());
    a.parts_of = reinterpret_cast<RowPart *>(static_cast<char *>(scratch.ptr()) + keys);
    ProfScope prof("beam_select", st);
    QNN_TRY(with_type(dtype, [&](auto t) { return launch_select<decltype(t)>(a, rows, B, st); }));
    QNN_CUDA_TRY(cudaGetLastError());
    return QNN_OK;
}

extern "C" qnn_status qnn_beam_reorder(const qnn_beam_state *states, int32_t count, const int32_t *parents, int64_t B, int64_t K,
                                       int64_t n, void *stream) {
    if (count < 0 || (count > 0 && !states) || B < 0 || K < 1 || K > kMostBeams || n < 1 || n > kMostBeams || B > INT32_MAX / kMostBeams ||
        !aligned4(parents))
        return QNN_ERR_INVALID_ARG;
    const int64_t most = (int64_t)1 << 46;
    for (int32_t i = 0; i < count; ++i) {
        const qnn_beam_state &s = states[i];
        if (s.outer < 0 || s.row_bytes < 0 || (s.outer && s.row_bytes && s.in == s.out && n != K)) return QNN_ERR_INVALID_ARG;
        if (s.outer && s.row_bytes && B && (s.outer > most / (B * kMostBeams) || s.row_bytes > most / (s.outer * B * kMostBeams)))
            return QNN_ERR_INVALID_ARG;
    }
    if (B == 0) return QNN_OK;
    if (count > 0 && !is_local_ptr(parents)) return QNN_ERR_INVALID_ARG;
    const Span ps(parents, 4 * B * n);
    for (int32_t i = 0; i < count; ++i) {
        const qnn_beam_state &s = states[i];
        if (s.outer * s.row_bytes == 0) continue;
        if (!is_local_ptr(s.in) || !is_local_ptr(s.out)) return QNN_ERR_INVALID_ARG;
        const Span o(s.out, s.outer * B * n * s.row_bytes);
        if (o.meets(ps)) return QNN_ERR_INVALID_ARG;
        for (int32_t j = 0; j < count; ++j) {
            const qnn_beam_state &t = states[j];
            if (t.outer * t.row_bytes == 0) continue;
            if (o.meets(Span(t.in, t.outer * B * K * t.row_bytes)) && !(i == j && s.in == s.out)) return QNN_ERR_INVALID_ARG;
            if (j < i && o.meets(Span(t.out, t.outer * B * n * t.row_bytes))) return QNN_ERR_INVALID_ARG;
        }
    }
    cudaStream_t st = as_stream(stream);
    ProfScope prof("beam_reorder", st);
    // launches of up to kStatesALaunch states whose words are of one width: 16 bytes where rows and addresses allow it, else
    // 4, 2 or 1; more than 16 beams in place take words of 4 bytes at most, which a thread can hold 128 of
    ReorderArgs a;
    a.parents = parents, a.B = B, a.K = K, a.n = n;
    QNN_TRY(status_word(&a.status));
    for (int in_place = 0; in_place < 2; ++in_place)
        for (int width = 16; width >= 1; width = width == 16 ? 4 : width / 2) {
            a.count = 0, a.items = 0;
            for (int32_t i = 0; i <= count; ++i) {
                if (i < count) {
                    const qnn_beam_state &s = states[i];
                    if (s.outer * s.row_bytes == 0 || (s.in == s.out) != (in_place != 0)) continue;
                    const uintptr_t bits = reinterpret_cast<uintptr_t>(s.in) | reinterpret_cast<uintptr_t>(s.out) | (uintptr_t)s.row_bytes;
                    const int w = bits % 16 == 0 && (!in_place || n <= 16) ? 16 : bits % 4 == 0 ? 4 : bits % 2 == 0 ? 2 : 1;
                    if (w != width) continue;
                    a.s[a.count++] = {static_cast<const char *>(s.in), static_cast<char *>(s.out), s.row_bytes / w, a.items};
                    a.items += s.outer * B * (s.row_bytes / w);
                }
                if (a.count == kStatesALaunch || (i == count && a.count > 0)) {
                    if (in_place && n > 16) {
                        if (width == 4) QNN_TRY((launch_reorder<uint32_t, 128>(a, st)));
                        else if (width == 2) QNN_TRY((launch_reorder<uint16_t, 128>(a, st)));
                        else QNN_TRY((launch_reorder<uint8_t, 128>(a, st)));
                    } else if (width == 16) {
                        QNN_TRY(launch_reorder<uint4>(a, in_place != 0, st));
                    } else if (width == 4) {
                        QNN_TRY(launch_reorder<uint32_t>(a, in_place != 0, st));
                    } else if (width == 2) {
                        QNN_TRY(launch_reorder<uint16_t>(a, in_place != 0, st));
                    } else {
                        QNN_TRY(launch_reorder<uint8_t>(a, in_place != 0, st));
                    }
                    QNN_CUDA_TRY(cudaGetLastError());
                    a.count = 0, a.items = 0;
                }
            }
        }
    return QNN_OK;
}
