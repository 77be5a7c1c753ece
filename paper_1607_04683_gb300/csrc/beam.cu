// beam.cu — one step of a beam search on sm_103a: the best continuations over beams and classes, and the carried states
// of the beams that were kept.
#include <algorithm>
#include <cfloat>
#include <cmath>

#include "elem.cuh"
#include "qnn_device.cuh"
#include "qnn_host.h"
#include "tc_ptx.cuh"

namespace qnn {
namespace {

constexpr int kMostKept = 128, kMostBeams = 128;

// ------------------------------------------------------------------------------------------------
// The n best of what a block's threads hold
// ------------------------------------------------------------------------------------------------

// A candidate: larger ones first, 0 none. The value in an order-preserving form, above it the index's complement, so that
// of equal values the lowest index is the largest candidate and no two are equal.
using Logit = unsigned long long;  // 32 bits of a logit, 32 of ~index
struct Cand {                      // a score in two fp32 terms, 32 bits each
    unsigned long long v;
    unsigned index;
};
__device__ __forceinline__ bool before(Logit a, Logit b) { return a > b; }
__device__ __forceinline__ bool before(const Cand &a, const Cand &b) { return a.v > b.v || (a.v == b.v && a.index < b.index); }
__device__ __forceinline__ bool some(Logit a) { return a != 0; }
__device__ __forceinline__ bool some(const Cand &a) { return a.v != 0; }
__device__ __forceinline__ Logit none_of(Logit) { return 0; }
__device__ __forceinline__ Cand none_of(Cand) { return {0, 0xffffffffu}; }
__device__ __forceinline__ Logit from_lane(Logit a, int lane) { return __shfl_sync(0xffffffffu, a, lane); }
__device__ __forceinline__ Cand from_lane(const Cand &a, int lane) {
    return {__shfl_sync(0xffffffffu, a.v, lane), __shfl_sync(0xffffffffu, a.index, lane)};
}
__device__ __forceinline__ Logit across(Logit a, int mask) { return __shfl_xor_sync(0xffffffffu, a, mask); }
__device__ __forceinline__ Cand across(const Cand &a, int mask) {
    return {__shfl_xor_sync(0xffffffffu, a.v, mask), __shfl_xor_sync(0xffffffffu, a.index, mask)};
}

__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t b = __float_as_uint(__fadd_rn(v, 0.0f));  // (-0 is 0)
    return b ^ ((int32_t)b < 0 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t o) { return __uint_as_float(o ^ ((int32_t)o < 0 ? 0x80000000u : 0xffffffffu)); }
__device__ __forceinline__ Logit logit_key(float v, unsigned index) {
    return v > -INFINITY ? (Logit)ordered(v) << 32 | (uint32_t)~index : 0;  // (a NaN is none either)
}

// A value as the sum of two fp32 terms, hi the sum rounded: 48 bits or so. (This part's units for 64 bits are few: a logarithm and
// some sums in 64 bits took a block 15 us.)
struct Two {
    float hi, lo;
};
__device__ __forceinline__ Two two_sum(float a, float b) {
    const float s = __fadd_rn(a, b), t = __fsub_rn(s, a);
    return {s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t))};
}
__device__ __forceinline__ Two add(Two a, Two b) {
    Two s = two_sum(a.hi, b.hi);
    s.lo = __fadd_rn(s.lo, __fadd_rn(a.lo, b.lo));
    return two_sum(s.hi, s.lo);
}
__device__ __forceinline__ Two mul(Two a, Two b) {
    const float p = __fmul_rn(a.hi, b.hi), e = __fmaf_rn(a.hi, b.hi, -p);
    return two_sum(p, __fmaf_rn(a.hi, b.lo, __fmaf_rn(a.lo, b.hi, e)));
}
// ln 2 in parts of 15 bits (whose product with an exponent is exact), 24, and the rest.
constexpr float kLn2Head = 0.693145751953125f, kLn2Mid = 1.428606765330187e-06f, kLn2Rest = 5.497923e-14f;
// exp(x), |x| <= 80, to 2^-34 (2^-39 on average): x = n ln 2 + 8 r, exp(r) - 1 = r + r^2 / 2 + r^3 / 6 + ... (the first two terms in two fp32 terms
// each; r^3 <= 10^-4), its square taken three times by p -> 2 p + p^2.
__device__ __forceinline__ Two exp_two(Two x) {
    const float n = rintf(__fmul_rn(x.hi, kLog2e));
    Two r = two_sum(__fmaf_rn(-n, kLn2Head, x.hi), __fmul_rn(-n, kLn2Mid));
    r.lo = __fadd_rn(r.lo, __fadd_rn(__fmaf_rn(-n, kLn2Mid, -__fmul_rn(-n, kLn2Mid)), __fmaf_rn(-n, kLn2Rest, x.lo)));
    r = two_sum(__fmul_rn(r.hi, 0.125f), __fmul_rn(r.lo, 0.125f));
    const Two q = mul(r, r);
    float c = __fmaf_rn(r.hi, 1.0f / 720, 1.0f / 120);
    c = __fmaf_rn(c, r.hi, 1.0f / 24);
    c = __fmaf_rn(c, r.hi, 1.0f / 6);
    Two p = add(r, {__fmul_rn(q.hi, 0.5f), __fmaf_rn(__fmul_rn(q.hi, r.hi), c, __fmul_rn(q.lo, 0.5f))});
#pragma unroll
    for (int i = 0; i < 3; ++i) p = add({__fmul_rn(2.0f, p.hi), __fmul_rn(2.0f, p.lo)}, mul(p, p));
    p = add({1.0f, 0.0f}, p);
    const float scale = __int_as_float((int)(n + 127.0f) << 23);
    return {__fmul_rn(p.hi, scale), __fmul_rn(p.lo, scale)};
}
// log(x), 2^-10 <= x < 2^64, off by 2^-35 at most (2^-39 on average): a first value in fp32, and the logarithm of what x exp(-value) is off 1.
__device__ __forceinline__ Two log_two(Two x) {
    const float y = logf(x.hi);
    const Two e = exp_two({-y, 0.0f});
    const Two d = add(mul(x, e), {-1.0f, 0.0f});
    return two_sum(y, __fmaf_rn(__fmul_rn(-0.5f, d.hi), d.hi, __fadd_rn(d.hi, d.lo)));
}
// score + (logit - lse), none where that is minus infinity or not a number.
__device__ __forceinline__ Cand cand_key(float score, float logit, Two lse, unsigned index) {
    const Two a = two_sum(logit, -lse.hi), b = two_sum(score, a.hi);
    Two s = two_sum(b.hi, __fadd_rn(b.lo, __fsub_rn(a.lo, lse.lo)));
    if (!(fabsf(b.hi) < INFINITY)) s = {b.hi, 0.0f};
    if (!(s.hi > -INFINITY)) return none_of(Cand());
    return {(unsigned long long)ordered(s.hi) << 32 | ordered(s.lo), index};
}

// The n best candidates so far, best first. A block of kThreads threads brings EACH candidates a thread at a time. Only those
// better than the n-th best so far count, and of them those no worse than the n-th best of the bests of G groups of threads, G >= 2 n:
// of candidates in no order 1.4 n at most are expected, n groups' at worst. A candidate's rank is the number of better
// ones, counted by one thread: no order of arrival shows in the result.
constexpr int kThreads = 256, kWarps = kThreads / 32;
template <typename K, int EACH>
struct Best {
    static constexpr int kMost = kThreads * EACH / 2 + kMostKept;
    K list[kMost];
    K ranked[kMostKept];
    K bests[kThreads];
    K last;  // the n-th best, or none
    int count, held, wanted;

    __device__ __forceinline__ void start() {
        if (threadIdx.x == 0) count = 0, held = 0, last = none_of(K());
        __syncthreads();
    }
    // What is in list[0 .. count), ranked: the best n of it, in order. Ends behind a barrier.
    __device__ __forceinline__ void rank(int n) {
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
    // key(e), e < EACH: the thread's candidates, mine the best of them. All threads call it; ends behind a barrier.
    template <typename F>
    __device__ __forceinline__ void take(F key, K mine, int n) {
        const K bar = last;
        if (!before(mine, bar)) mine = none_of(K());
        if (__syncthreads_or(some(mine)) == 0) return;
        // the groups' bests, and of them the n-th: every warp for itself
        const int lane = threadIdx.x % 32, groups = n <= 16 ? 32 : n <= 32 ? 64 : n <= 64 ? 128 : 256, size = kThreads / groups;
        K top = mine;
        for (int m = 1; m < size; m <<= 1) {
            const K other = across(top, m);
            if (before(other, top)) top = other;
        }
        if (threadIdx.x % size == 0) bests[threadIdx.x / size] = top;
        __syncthreads();
        K from = none_of(K());
        for (int i = lane; i < groups; i += 32) {
            const K k = bests[i];
            int better = 0;
#pragma unroll 8
            for (int j = 0; j < groups; ++j) better += before(bests[j], k);
            const unsigned hit = __ballot_sync(0xffffffffu, some(k) && better == n - 1);
            if (hit) from = from_lane(k, __ffs(hit) - 1);
        }
        if (some(mine) && !before(from, mine)) {
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                const K k = key(e);
                if (before(k, bar) && !before(from, k)) list[atomicAdd(&count, 1)] = k;
            }
        }
        __syncthreads();
        rank(n);
    }
};

// ------------------------------------------------------------------------------------------------
// Selection
// ------------------------------------------------------------------------------------------------

// Of a part of a row: its largest value and the sum of exp(value - largest) as a whole number of the call's units (exact sums
// of the threads' ones, in any order; ~0: not a number).
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
    float units, unit;  // of RowPart::sum: how many are 1, a power of two by which `per` has 62 bits, and what one is
    int n, parts, eos;
};

// exp(d) for d <= 0 by the hardware's exponential, whose argument, the product with log2(e) in two terms, is rounded once. kBias takes
// out what the instruction is off on average (it lies low by 5e-8, 7e-8 ln 2; that of 0 stays 1).
//
// How far a row's log sum exp is off, in 2^-24: a term's difference d from the part's largest value is rounded (|d|), as is its argument (|d| too,
// for a factor ln 2 of log2(e) |d|), the instruction is 2^-22 off at most (4) and the bias 5e-8 (1). A tile's terms of a thread are added in
// pairs (5 roundings for 32), tiles and threads without loss (two fp32 terms, then whole numbers). In all 10 + 2 D, D the mean of |d| by the classes'
// probabilities, which is the entropy at most; up to 2.1 in 1700 rows of 97 to 262144 classes. (Terms added one after another into one fp32 sum: up to
// 380 for 262144 classes of two values, as every term's rounding goes the same way. 320 x 65536 fp32 30.8 us, so 27.4; 128 x 8 x 8192 as before.)
constexpr float kLog2eRest = 1.925963033500e-08f, kBias = 7e-8f;
__device__ __forceinline__ float exp_term(float d) { return exp2_hw(__fmaf_rn(d, kLog2e, __fmaf_rn(d, kLog2eRest, kBias))); }
// The sum of exp(v - from) over N values, in pairs.
template <int N>
__device__ __forceinline__ float exp_terms(const float *v, float from) {
    if constexpr (N == 1) return exp_term(__fsub_rn(*v, from));
    else return __fadd_rn(exp_terms<N / 2>(v, from), exp_terms<N / 2>(v + N / 2, from));
}

// A tile of a row: with VEC runs of eight values a thread, else neighbouring values by neighbouring threads.
constexpr int kRun = 8;
template <bool VEC>
__device__ __forceinline__ int64_t place(int64_t base, int e) {
    return base + (VEC ? (e / kRun * kThreads + (int)threadIdx.x) * kRun + e % kRun : e * kThreads + (int)threadIdx.x);
}
template <typename T, bool VEC, int EACH>
__device__ __forceinline__ void load_tile(const T *row, int64_t base, int64_t end, float (&v)[EACH]) {
    if (base + kThreads * EACH <= end) {  // whole
        if constexpr (VEC) {
#pragma unroll
            for (int r = 0; r < EACH / kRun; ++r) {
                Run<T, kRun> x;
                x.load(row + place<VEC>(base, r * kRun));
#pragma unroll
                for (int e = 0; e < kRun; ++e) v[r * kRun + e] = x.get(e);
            }
        } else {
#pragma unroll
            for (int e = 0; e < EACH; ++e) v[e] = to_f32(row[place<VEC>(base, e)]);
        }
    } else if constexpr (VEC) {
#pragma unroll
        for (int r = 0; r < EACH / kRun; ++r) {
            const int64_t at = place<VEC>(base, r * kRun);
            Run<T, kRun> x;
            if (at + kRun <= end) x.load(row + at);
            else x.load_some(row + at, at < end ? (int)(end - at) : 0);
#pragma unroll
            for (int e = 0; e < kRun; ++e) v[r * kRun + e] = at + e < end ? x.get(e) : -INFINITY;
        }
    } else {
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int64_t at = place<VEC>(base, e);
            v[e] = at < end ? to_f32(row[at]) : -INFINITY;
        }
    }
}

// Best::take for a tile of a row, by values alone: candidates are those no less than the n-th best of the groups' largest values (and
// above the n-th best so far, which comes from lower classes). False, with nothing taken, where so many are equal to it that
// they need to be told apart by their classes first. One 32-bit comparison a value instead of keys of 64: 128 x 8 x 8192
// bf16 11 us less. `also` is called once by every thread on the way, with the tile's largest value, or minus infinity where that is
// no larger than those before.
constexpr int kFewCands = 512;
template <bool VEC, int EACH, typename F>
__device__ __forceinline__ bool take_values(Best<Logit, EACH> &s, const float (&v)[EACH], float top, int64_t base, int n, F also) {
    const float bar = s.held == n ? unordered((uint32_t)(s.last >> 32)) : -INFINITY;
    const bool pass = top > bar;
    if (__syncthreads_or(pass) == 0) {
        also(-INFINITY);
        return true;
    }
    const int lane = threadIdx.x % 32, groups = n <= 16 ? 32 : n <= 32 ? 64 : n <= 64 ? 128 : 256, size = kThreads / groups;
    float most = pass ? top : -INFINITY;
    for (int m = 1; m < size; m <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, m));
    float *bests = reinterpret_cast<float *>(s.bests);
    if (threadIdx.x % size == 0) bests[threadIdx.x / size] = most;
    if (threadIdx.x == 0) s.wanted = s.held;
    __syncthreads();
    float from = -INFINITY, largest = -INFINITY;  // the n-th largest, if there are as many
    for (int i = lane; i < groups; i += 32) {
        const float mine = bests[i];
        largest = fmaxf(largest, mine);
        int better = 0;
#pragma unroll 8
        for (int j = 0; j < groups; ++j) better += bests[j] > mine;
        // (of equal ones all have the same count: the n-th has less than n better ones, and n or more with its equals)
        float least = better < n ? mine : INFINITY;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) least = fminf(least, __shfl_xor_sync(0xffffffffu, least, o));
        from = i == lane ? least : fminf(from, least);
    }
    // (one comparison a value: those no less than the n-th, or than the next value above the bar)
    const float least = from > bar ? from : unordered(ordered(bar) + 1);
    if (pass && top >= least)
#pragma unroll
        for (int e = 0; e < EACH; ++e)
            if (v[e] >= least) {
                const int at = atomicAdd(&s.wanted, 1);
                if (at < kFewCands) s.list[at] = logit_key(v[e], (unsigned)place<VEC>(base, e));
            }
    also(warp_max(largest));
    __syncthreads();
    if (s.wanted > kFewCands) return false;
    if (threadIdx.x == 0) s.count = s.wanted;
    __syncthreads();
    s.rank(n);
    return true;
}

// One part of a beam's row: its sum of exponentials and its n best classes in one pass over it, tiles of kThreads EACH values
// in registers. Within a beam the order of the logits is that of the scores, so that no score is formed here. The classes lie in
// best.list. Bound: instructions, 770 a warp for 8192 classes (exponentials 5 a class), and the block's meetings: 128 x 8 x 8192 bf16 14 us
// for all rows, so 1.2 TB/s.
template <int EACH>
struct RowShared {
    Best<Logit, EACH> best;
    unsigned long long warp_sum[kWarps];
};
template <typename T, bool VEC, int EACH>
__device__ __forceinline__ RowPart look_at(const T *x, int64_t lo, int64_t hi, int n, float units, RowShared<EACH> &sh) {
    float v[EACH], most = -INFINITY;  // most: of the block's values so far, which the sum's terms go by
    Two sum = {0.0f, 0.0f};
    load_tile<T, VEC, EACH>(x, lo, hi, v);
    sh.best.start();
    for (int64_t base = lo; base < hi; base += kThreads * EACH) {
        if (base > lo) load_tile<T, VEC, EACH>(x, base, hi, v);
        float top = v[0];
#pragma unroll
        for (int e = 1; e < EACH; ++e) top = fmaxf(top, v[e]);
        auto add_up = [&](float largest) {
            if (largest > most) {  // (NaNs stay NaNs)
                const Two d = two_sum(most, -largest);
                if (most > -INFINITY) sum = mul(sum, d.hi < -80.0f ? Two{0.0f, 0.0f} : exp_two(d));
                most = largest;
            }
            const Two s = two_sum(sum.hi, exp_terms<EACH>(v, most > -INFINITY ? most : 0.0f));
            sum = {s.hi, __fadd_rn(sum.lo, s.lo)};
        };
        if (!take_values<VEC, EACH>(sh.best, v, top, base, n, add_up)) {
            unsigned first = 0;
#pragma unroll
            for (int e = EACH - 1; e >= 0; --e)
                if (v[e] == top) first = (unsigned)place<VEC>(base, e);
            sh.best.take([&](int e) { return logit_key(v[e], (unsigned)place<VEC>(base, e)); }, logit_key(top, first), n);
        }
    }
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const bool bad = !(sum.hi >= 0.0f && sum.hi < INFINITY);
    unsigned long long s =
        bad ? 0 : __float2ull_rn(__fmul_rn(sum.hi, units)) + (unsigned long long)__float2ll_rn(__fmul_rn(sum.lo, units));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) sh.warp_sum[warp] = s;
    const int any_bad = __syncthreads_or(bad);
    s = 0;
    for (int i = 0; i < kWarps; ++i) s += sh.warp_sum[i];
    return {any_bad ? ~0ull : s, most, sh.best.held};
}
// A beam that is not finished and not lost has its logits looked at.
__device__ __forceinline__ bool looked_at(const SelectArgs &a, int64_t row) {
    return !(a.finished && a.finished[row]) && a.scores[row] > -INFINITY;
}

template <typename T, bool VEC, int EACH>
__global__ void __launch_bounds__(kThreads, 4) beam_rows_kernel(const SelectArgs a) {
    __shared__ RowShared<EACH> sh;
    grid_dependents_launch();  // (the merge waits for all of this before it reads any of it)
    const int64_t row = blockIdx.x / (unsigned)a.parts;
    const int part = blockIdx.x % (unsigned)a.parts;
    if (!looked_at(a, row)) return;
    const int64_t lo = part * a.per, hi = lo + a.per < a.V ? lo + a.per : a.V;
    const RowPart of = look_at<T, VEC, EACH>(static_cast<const T *>(a.logits) + row * a.ldl, lo, hi, a.n, a.units, sh);
    Logit *keys = a.keys + (row * a.parts + part) * a.n;
    for (int i = threadIdx.x; i < of.held; i += kThreads) keys[i] = sh.best.list[i];
    if (threadIdx.x == 0) a.parts_of[row * a.parts + part] = of;
}

// A batch row's beams: each one's score and the log of its sum from its parts.
struct Beams {
    Two lse[kMostBeams];
    unsigned char state[kMostBeams];  // 0: no candidates, 1: its parts' lists, 2: finished
    float score[kMostBeams];

    // parts: those of the batch row's first beam, then of its next (whatever is in memory for a row that nothing was looked for in).
    // By thread k for beam k; seen behind a barrier.
    __device__ __forceinline__ void set(const SelectArgs &a, int64_t b, const RowPart *parts) {
        for (int k = threadIdx.x; k < a.K; k += kThreads) {
            const int64_t row = b * a.K + k;
            const float sc = a.scores[row];
            const RowPart *p = parts + (int64_t)k * a.parts, part0 = p[0];
            int st = 0;
            Two l = {0.0f, 0.0f};
            if (sc > -INFINITY) {
                if (a.finished && a.finished[row]) {
                    st = 2;
                } else {
                    float m = part0.most;
                    bool bad = part0.sum == ~0ull;
                    for (int i = 1; i < a.parts; ++i) m = fmaxf(m, p[i].most), bad |= p[i].sum == ~0ull;
                    if (!bad && m > -INFINITY && m < INFINITY) {
                        Two s = {0.0f, 0.0f};
                        for (int i = 0; i < a.parts; ++i) {
                            const RowPart of = i == 0 ? part0 : p[i];
                            const float d = __fsub_rn(of.most, m);  // (below -80 a part counts for nothing)
                            if (d < -80.0f) continue;
                            const unsigned long long whole = of.sum;
                            const float hi = __ull2float_rn(whole);
                            const Two share = {__fmul_rn(hi, a.unit),
                                               __fmul_rn(__ll2float_rn((long long)(whole - (unsigned long long)hi)), a.unit)};
                            s = add(s, d == 0.0f ? share : mul(share, exp_two(two_sum(of.most, -m))));
                        }
                        l = add({m, 0.0f}, log_two(s));
                        st = 1;
                    }
                }
            }
            lse[k] = l, state[k] = (unsigned char)st, score[k] = sc;
        }
    }
    // The candidate of beam k's logit l (0: none, and the finished beam's own for its first).
    __device__ __forceinline__ Cand scored(const SelectArgs &a, int k, Logit l, bool first) const {
        if (state[k] == 2 && first) return cand_key(score[k], 0.0f, {0.0f, 0.0f}, (unsigned)(k * a.V + a.eos));
        if (state[k] == 1 && l) return cand_key(score[k], unordered((uint32_t)(l >> 32)), lse[k], (unsigned)(k * a.V + (unsigned)~(uint32_t)l));
        return none_of(Cand());
    }
};
__device__ __forceinline__ void put_selected(const SelectArgs &a, int64_t b, const Cand *best, int held) {
    for (int i = threadIdx.x; i < a.n; i += kThreads) {
        const int64_t o = b * a.n + i;
        if (i < held) {
            const Cand c = best[i];
            a.scores_out[o] = unordered((uint32_t)(c.v >> 32));
            a.parents[o] = (int32_t)(c.index / (unsigned)a.V);
            a.tokens[o] = (int32_t)(c.index % (unsigned)a.V);
        } else {
            a.scores_out[o] = -INFINITY;
            a.parents[o] = 0;
            a.tokens[o] = a.eos;
        }
    }
}
// A batch row's candidate `at`: the beam and, where its list has one, its logit. True for the beam's first.
__device__ __forceinline__ bool candidate(const SelectArgs &a, const RowPart *parts, const Logit *keys, unsigned at, int &k, Logit &logit) {
    const unsigned list = at / (unsigned)a.n, i = at % (unsigned)a.n;
    k = (int)(list / (unsigned)a.parts);
    const int held = parts[list].held;
    logit = keys[at];
    if ((int)i >= held) logit = 0;
    return list == (unsigned)k * (unsigned)a.parts && i == 0;
}

// A batch row's continuations, where a block's threads hold all candidates one each: a candidate's rank is counted over all of
// them by as many threads as there are for it; a list's candidates lie in order and lists by beam and classes, so that of equal scores the
// first is the one with the lowest index. (Code that is not in a cache yet is most of a short kernel's time.)
struct FewShared {
    Beams beams;
    Cand all[kThreads], ranked[kMostKept];
};
__device__ __forceinline__ void select_of_few(const SelectArgs &a, int64_t b, const RowPart *parts, const Logit *keys, FewShared &sh) {
    const int total = (int)a.K * a.parts * a.n;
    int k = 0;
    Logit logit = 0;
    bool first = false;
    if ((int)threadIdx.x < total) first = candidate(a, parts, keys, threadIdx.x, k, logit);
    sh.beams.set(a, b, parts);
    __syncthreads();
    sh.all[threadIdx.x] = (int)threadIdx.x < total ? sh.beams.scored(a, k, logit, first) : none_of(Cand());
    int share = 1;  // threads a candidate
    while (share < 32 && 2 * share * total <= kThreads) share *= 2;
    __syncthreads();
    const int i = threadIdx.x / share, part = threadIdx.x % share;
    const unsigned long long mine = i < total ? sh.all[i].v : 0;
    int better = 0;
#pragma unroll 4
    for (int j = part; j < total; j += share) better += sh.all[j].v >= mine + (j >= i);
    for (int m = 1; m < share; m <<= 1) better += __shfl_xor_sync(0xffffffffu, better, m);
    const int there = __syncthreads_count(part == 0 && mine);
    if (part == 0 && mine && better < a.n) sh.ranked[better] = sh.all[i];
    __syncthreads();
    put_selected(a, b, sh.ranked, there < a.n ? there : a.n);
}

// The merge of what rows' blocks left in memory. EACH: 1 as above, else a thread takes 8 candidates at a time.
template <int EACH>
__global__ void __launch_bounds__(kThreads) beam_merge_kernel(const SelectArgs a) {
    const int64_t b = blockIdx.x, list0 = b * a.K * a.parts;
    const RowPart *const parts = a.parts_of + list0;
    const Logit *const keys = a.keys + list0 * a.n;
    grid_dependency_wait();
    if constexpr (EACH == 1) {
        __shared__ FewShared sh;
        select_of_few(a, b, parts, keys, sh);
    } else {
        __shared__ Best<Cand, EACH> best;
        __shared__ Beams beams;
        const int64_t total = a.K * a.parts * a.n;
        beams.set(a, b, parts);
        best.start();
        for (int64_t base = 0; base < total; base += kThreads * EACH) {
            Cand key[EACH], mine = none_of(Cand());
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                const int64_t at = base + threadIdx.x + (int64_t)e * kThreads;
                key[e] = none_of(Cand());
                if (at < total) {
                    int k;
                    Logit l;
                    const bool first = candidate(a, parts, keys, (unsigned)at, k, l);
                    key[e] = beams.scored(a, k, l, first);
                }
                if (before(key[e], mine)) mine = key[e];
            }
            best.take([&](int e) { return key[e]; }, mine, a.n);
        }
        put_selected(a, b, best.list, best.held);
    }
}

// Both in one launch where a batch row's parts are a cluster of blocks and the candidates few: lists and sums go to the
// first block's shared memory. 128 x 8 x 8192 bf16 20.5 us a call, by two launches 27; 1 x 4 x 2000 fp32 18.5 and 22 (most of it
// the call on the host).
constexpr int kMostCluster = 8;
template <int EACH>
struct ClusterShared {
    RowShared<EACH> row;
    FewShared few;
    Logit keys[kThreads];
    RowPart parts[kMostCluster];
};
__device__ __forceinline__ void store_remote64(uint32_t addr, unsigned long long v) {
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.aligned;" ::: "memory"); }
template <typename T, bool VEC, int EACH>
__global__ void __launch_bounds__(kThreads, 4) beam_cluster_kernel(const SelectArgs a) {
    extern __shared__ __align__(16) unsigned char raw[];
    ClusterShared<EACH> &sh = *reinterpret_cast<ClusterShared<EACH> *>(raw);
    const unsigned blocks = (unsigned)a.K * (unsigned)a.parts, rank = blockIdx.x % blocks, part = rank % (unsigned)a.parts;
    const int64_t b = blockIdx.x / blocks, row = b * a.K + rank / (unsigned)a.parts;
    cluster_arrive();  // (the first block has to run before the others write into its memory)
    const bool there = looked_at(a, row);
    RowPart of;
    if (there) {
        const int64_t lo = part * a.per, hi = lo + a.per < a.V ? lo + a.per : a.V;
        of = look_at<T, VEC, EACH>(static_cast<const T *>(a.logits) + row * a.ldl, lo, hi, a.n, a.units, sh.row);
    }
    __syncwarp();
    cluster_wait();
    if (there) {
        const uint32_t keys = cluster_addr(su32(&sh.keys[rank * a.n]), 0), to = cluster_addr(su32(&sh.parts[rank]), 0);
        for (int i = threadIdx.x; i < of.held; i += kThreads) store_remote64(keys + 8 * i, sh.row.best.list[i]);
        if (threadIdx.x == 0) {
            store_remote64(to, of.sum);
            store_remote64(to + 8, (unsigned long long)(uint32_t)of.held << 32 | __float_as_uint(of.most));
        }
    }
    __syncwarp();
    cluster_sync();
    if (rank == 0) select_of_few(a, b, sh.parts, sh.keys, sh.few);
}

bool in_cluster(const SelectArgs &a) { return a.K * a.parts <= kMostCluster && a.K * a.parts * a.n <= kThreads; }

template <typename T, int EACH>
qnn_status launch_select(const SelectArgs &a, bool vec, int64_t B, cudaStream_t st) {
    const int64_t blocks = B * a.K * a.parts;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr;
    cfg.attrs = &attr;
    if (in_cluster(a)) {
        const auto kern = vec ? beam_cluster_kernel<T, true, EACH> : beam_cluster_kernel<T, false, EACH>;
        cfg.dynamicSmemBytes = sizeof(ClusterShared<EACH>);
        static_assert(sizeof(ClusterShared<EACH>) <= 48 * 1024);  // (what a launch has without asking)
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = (unsigned)(a.K * a.parts), attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cfg.numAttrs = 1;
        QNN_CUDA_TRY(cudaLaunchKernelEx(&cfg, kern, a));
        return QNN_OK;
    }
    QNN_CUDA_TRY(vec ? cudaLaunchKernelEx(&cfg, beam_rows_kernel<T, true, EACH>, a) : cudaLaunchKernelEx(&cfg, beam_rows_kernel<T, false, EACH>, a));
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)B);
    cfg.numAttrs = 1;
    QNN_CUDA_TRY(a.K * a.parts * a.n <= kThreads ? cudaLaunchKernelEx(&cfg, beam_merge_kernel<1>, a) : cudaLaunchKernelEx(&cfg, beam_merge_kernel<8>, a));
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
// Bound: HBM or L2; 64 x 8 beams, states of 5 x 2048 and 5 x 512 values, 54 MB: 9.4 us, 5.7 TB/s. Over 16 beams in place: registers, as a
// thread holds 128 words of 4 bytes (452 bytes of them spilled) whatever n is; 30 x 17, 16 x 32, 8 x 64 and 4 x 128 beams of the same states 139, 108, 86
// and 105 us, into other tensors 11, 12, 17 and 30.
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
    SelectArgs a = {};
    a.logits = logits, a.ldl = ldl, a.scores = scores, a.finished = finished, a.scores_out = scores_out, a.parents = parents;
    a.tokens = tokens, a.K = K, a.V = V, a.n = n, a.eos = eos;
    // Tiles of 8192 classes where those alone give the SMs two blocks each, else of 2048; a part of a row is as many tiles as leave
    // four blocks an SM (one, while there are fewer).
    const int64_t rows = B * K;
    const int each = rows * (V / (32 * kThreads)) >= 2 * (int64_t)sm_count() ? 32 : 8;
    const int64_t tile = each * kThreads, tiles = (V + tile - 1) / tile;
    int64_t parts = std::max<int64_t>(1, std::min<int64_t>({4 * (int64_t)sm_count() / rows, tiles, 32}));
    const int64_t per = (tiles + parts - 1) / parts;
    parts = (tiles + per - 1) / per;
    if (rows * parts > INT32_MAX) return QNN_ERR_INVALID_ARG;
    a.parts = (int)parts, a.per = per * tile;
    a.units = std::ldexp(1.0f, 61 - std::ilogb((double)a.per)), a.unit = 1.0f / a.units;  // (a term is 1 at most)
    cudaStream_t st = as_stream(stream);
    Scratch scratch;
    if (!in_cluster(a)) {
        const size_t keys = (size_t)(rows * parts * n) * sizeof(Logit);
        QNN_TRY(scratch.take(keys + (size_t)(rows * parts) * sizeof(RowPart), st));
        a.keys = static_cast<Logit *>(scratch.ptr());
        a.parts_of = reinterpret_cast<RowPart *>(static_cast<char *>(scratch.ptr()) + keys);
    }
    const bool vec = reinterpret_cast<uintptr_t>(logits) % 16 == 0 && ldl * e % 16 == 0;
    ProfScope prof("beam_select", st);
    return with_type(dtype, [&](auto t) {
        return each == 8 ? launch_select<decltype(t), 8>(a, vec, B, st) : launch_select<decltype(t), 32>(a, vec, B, st);
    });
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
