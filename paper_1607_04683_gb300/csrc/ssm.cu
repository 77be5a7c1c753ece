// ssm.cu — the recurrent half of a selective state-space layer on sm_103a: a short causal convolution per channel and the
// selective scan, for whole sequences and for single frames with carried states.
#include <algorithm>
#include <atomic>
#include <cfloat>

#include "elem.cuh"
#include "qnn_device.cuh"
#include "qnn_host.h"

namespace qnn {
namespace {

// Frames of sequence b.
__device__ __forceinline__ int frames_of(const int32_t *lengths, int64_t b, int64_t T) {
    if (!lengths) return (int)T;
    const int n = __ldg(lengths + b);
    return n < 0 ? 0 : n > T ? (int)T : n;
}

// i / n and i % n. 64-bit divisions take a hundred instructions; most indices need 32.
struct Split {
    int64_t quot, rem;
};
__device__ __forceinline__ Split split(int64_t i, int64_t n) {
    if (((i | n) >> 32) == 0) {
        const uint32_t q = (uint32_t)i / (uint32_t)n;
        return {(int64_t)q, (int64_t)((uint32_t)i - q * (uint32_t)n)};
    }
    return {i / n, i % n};
}

// ------------------------------------------------------------------------------------------------
// Convolution
// ------------------------------------------------------------------------------------------------

struct ConvArgs {
    const void *x, *state_in;
    void *state_out, *y;
    const float *w, *bias;
    const int32_t *lengths;
    int64_t x_seq, x_frame, y_seq, y_frame, B, T, D, runs, chunks;
    int silu, chunk;
};

// A thread takes V neighbouring channels of a sequence over a chunk of its frames in rounds of kAhead, the last W - 1 inputs
// in registers and the next round's loads in flight. The first chunk's thread alone reads and writes the channels' state: it
// has read the old state before it writes the new one, and later chunks (at least W - 1 frames on) never look at it. A kernel for
// each number of taps: in one for more of them the missing ones would be products of 0 with older inputs, NaN where those
// are not finite.
//
// Bound: HBM. 16 x 1000 x 2048, 4 taps: fp32 42 to 44 us (6.1 TB/s), bf16 27 to 29 (4.7 TB/s; without SiLU 25.9, a plain copy of
// as many bytes 22.9). Tried for bf16 and no faster: two channels a thread at twice the warps, 16 and 24 frames ahead, chunks of 24
// to 112 frames. Other numbers of taps, bf16: one 24.5, seven 32.7, eight 54 (fp32 61).
constexpr int kMostTaps = 8, kConvThreads = 128;
template <typename T, int W, int V, int kAhead>
__global__ void __launch_bounds__(kConvThreads) causal_conv_kernel(const ConvArgs a) {
    const int64_t at = (int64_t)blockIdx.x * kConvThreads + threadIdx.x;
    const Split of_runs = split(at, a.runs), of_chunks = split(of_runs.quot, a.chunks);
    const int64_t run = of_runs.rem, chunk = of_chunks.rem, b = of_chunks.quot;
    if (b >= a.B) return;
    const int n = frames_of(a.lengths, b, a.T), t0 = (int)chunk * a.chunk, t1 = min(n, t0 + a.chunk);
    if (chunk > 0 && t0 >= n) return;
    const int64_t d = run * V;
    const T *x = static_cast<const T *>(a.x) + b * a.x_seq + d;
    T *y = static_cast<T *>(a.y) + b * a.y_seq + d;
    const T *s_in = static_cast<const T *>(a.state_in) + b * (W - 1) * a.D + d;
    T *s_out = static_cast<T *>(a.state_out) + b * (W - 1) * a.D + d;
    auto unpack = [](const Run<T, V> &r, float (&to)[V]) {
#pragma unroll
        for (int v = 0; v < V; ++v) to[v] = r.get(v);
    };
    float in[W - 1 + kAhead][V];  // the W - 1 inputs before a round of kAhead frames, and the round's
    {
        Run<T, V> r[W];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {  // before the chunk: W - 1 - j frames back of t0
            const int t = t0 - (W - 1) + j;
            r[j].clear();
            if (chunk > 0)
                r[j].load(x + t * a.x_frame);
            else if (a.state_in)
                r[j].load(s_in + (t + W - 1) * a.D);
        }
#pragma unroll
        for (int j = 0; j < W - 1; ++j) unpack(r[j], in[j]);
    }
    if (t0 < t1) {
        Run<T, V> next[kAhead];
        const T *from = x + t0 * a.x_frame;
        T *to = y + t0 * a.y_frame;
        auto fetch = [&](int left) {  // the next round's frames, of `left` there are
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (i < left) next[i].load(from);
                from += a.x_frame;
            }
        };
        fetch(t1 - t0);
        float w[W][V], bias[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            bias[v] = a.bias ? __ldg(a.bias + d + v) : 0.0f;
            if constexpr (W == 4 && V > 1) {  // (V channels' taps lie side by side: whole loads; one by one, a load's 32 lanes
                                               // touch as many lines)
                const float4 q = __ldg(reinterpret_cast<const float4 *>(a.w + (d + v) * 4));
                w[0][v] = q.x, w[1][v] = q.y, w[2][v] = q.z, w[3][v] = q.w;
            } else {
#pragma unroll
                for (int j = 0; j < W; ++j) w[j][v] = __ldg(a.w + (d + v) * W + j);
            }
        }
        auto frame = [&](int i) {  // the i-th of the round
            float o[V];
            if constexpr (V > 1) {
#pragma unroll
                for (int v = 0; v < V; v += 2) {
                    float2 f = make_float2(bias[v], bias[v + 1]);
#pragma unroll
                    for (int j = 0; j < W; ++j) f = ffma2_rn(make_float2(w[j][v], w[j][v + 1]), make_float2(in[i + j][v], in[i + j][v + 1]), f);
                    if (a.silu) f = silu2(f);
                    o[v] = f.x, o[v + 1] = f.y;
                }
            } else {
                o[0] = bias[0];
#pragma unroll
                for (int j = 0; j < W; ++j) o[0] = __fmaf_rn(w[j][0], in[i + j][0], o[0]);
                if (a.silu) o[0] = silu(o[0]);
            }
            Run<T, V> out;
            out.set(o);
            out.store(to);
            to += a.y_frame;
        };
        int t = t0;
        for (; t + kAhead <= t1; t += kAhead) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) unpack(next[i], in[W - 1 + i]);
            fetch(t1 - t - kAhead);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) frame(i);
#pragma unroll
            for (int j = 0; j < W - 1; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) in[j][v] = in[j + kAhead][v];
        }
#pragma unroll
        for (int i = 0; i < kAhead - 1; ++i) {  // the frames of a last, shorter round
            if (t + i >= t1) break;
            unpack(next[i], in[W - 1]);
            frame(0);
#pragma unroll
            for (int j = 0; j < W - 1; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) in[j][v] = in[j + 1][v];
        }
    }
    if (chunk > 0 || !a.state_out) return;
    // the last W - 1 of old state and n frames. Where the chunk holds all frames they are at hand
    if (n <= a.chunk) {
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            Run<T, V> last;
            last.set(in[j]);
            last.store(s_out + j * a.D);
        }
    } else {
        for (int j = 0; j < W - 1; ++j) {
            Run<T, V> last;
            last.load(x + (int64_t)(n - (W - 1) + j) * a.x_frame);
            last.store(s_out + j * a.D);
        }
    }
}

// ------------------------------------------------------------------------------------------------
// Scan
// ------------------------------------------------------------------------------------------------

constexpr int kMostStates = 128;

// The hardware's exponential lies low: by 0.5 to 0.8e-8 on average for arguments of -2^-14 .. -2^-8, 1.6 to 2.7e-8 for -2^-8 .. -2^-2
// (relative; its rounding noise is 3e-8). Over a state's memory of 1/(s A) frames noise grows as the root and bias as itself, so
// arguments are taken kBias higher, by the multiply-add that forms them: -1.3 to 0.8e-8 are left (a state after 100 frames
// 2.0e-6 off without, 0.9e-6 with). A step of 0 still has a factor of 1, as exp2(kBias) rounds to it.
constexpr float kBias = 2e-8f;
// A log2(e), as a number: a frame that is not there has a step of 0, whose product with an infinity would be a NaN. (Steps
// of 2^-120 and more have factors of 0 by minus FLT_MAX as by minus infinity.)
__device__ __forceinline__ float rate(float A) {
    const float v = __fmul_rn(A, kLog2e);
    return isinf(v) ? copysignf(FLT_MAX, v) : v;
}
__device__ __forceinline__ float factor(float s, float A) { return exp2_hw(__fmaf_rn(s, A, kBias)); }

struct ScanArgs : qnn_ssm_args {
    bool vec;             // (few frames) runs of four states are loaded and stored whole
    int64_t group_chans;  // D / groups
    int64_t units;        // warps' shares of channels, of all sequences
    int group_blocks;     // of them a group
    int parts;            // warps that share a unit's frames
};

// Few frames: states are most of the traffic (8 N bytes a channel, in and out). A lane holds four states of a channel, L lanes a
// channel, and takes NB sequences at a time: lane q forms the steps and gates of sequence q of them and passes them on by
// shuffles, so that each is formed once. It goes on to further sequences of its channel, whose states and inputs are loaded
// one round ahead; what depends on the channel alone is read once. (256 x 1 x 2048 x 16 fp32: a sequence a thread 29 us, 350
// instructions each; four, once, 22 us.)
constexpr int kStepFrames = 4, kStepThreads = 128;
template <typename T, int L, bool VEC>
__global__ void __launch_bounds__(kStepThreads, 4) ssm_step_kernel(const ScanArgs a) {
    constexpr int NB = L < 4 ? L : 4;
    const int64_t at = (int64_t)blockIdx.x * kStepThreads + threadIdx.x;
    const int q = (int)(at % L), n0 = 4 * q, lane = threadIdx.x & 31, mine = q % NB;  // mine: this lane's sequence
    const bool chan = at / L < a.D;
    const int64_t d = chan ? at / L : a.D - 1, g = a.groups == 1 ? 0 : split(d, a.group_chans).quot;
    const int count = chan ? max(min(a.N - n0, 4), 0) : 0;  // states
    float A[4];
    {
        Run<float, 4> r;
        r.clear();
        if (!VEC)
            r.load_some(a.A + d * a.N + n0, count);
        else if (count)
            r.load(a.A + d * a.N + n0);
#pragma unroll
        for (int k = 0; k < 4; ++k) A[k] = rate(r.get(k));
    }
    const float skip = a.skip ? __ldg(a.skip + d) : 0.0f, bias = a.dt_bias ? __ldg(a.dt_bias + d) : 0.0f;

    const int64_t step = (int64_t)gridDim.y * NB, row = a.D * a.N;  // sequences from a round to the next, states of one
    int64_t b0 = (int64_t)blockIdx.y * NB;
    const float *p_in = a.state_in + (a.state_in ? b0 * row + d * a.N + n0 : 0);
    float *p_out = a.state_out + (a.state_out ? b0 * row + d * a.N + n0 : 0);
    const T *pu = static_cast<const T *>(a.u) + (b0 + mine) * a.u_seq + d, *pd = static_cast<const T *>(a.dt) + (b0 + mine) * a.dt_seq + d;
    const T *pz = static_cast<const T *>(a.z) + (b0 + mine) * a.z_seq + d;
    T *py = static_cast<T *>(a.y) + (b0 + mine) * a.y_seq + d;
    const T *pB = static_cast<const T *>(a.Bm) + b0 * a.Bm_seq + g * a.N + n0, *pC = static_cast<const T *>(a.Cm) + b0 * a.Cm_seq + g * a.N + n0;

    Run<float, 4> next[NB];
    Run<T, 1> nu, nd, nz;
    int n_frames = 0;
    auto fetch = [&](int64_t b) {  // the states of the round from sequence b on, and their first frame's inputs
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            next[i].clear();
            if (a.state_in && b + i < a.B) {
                if (!VEC)
                    next[i].load_some(p_in + i * row, count);
                else if (count)
                    next[i].load(p_in + i * row);
            }
        }
        p_in += step * row;
        n_frames = chan && b + mine < a.B ? frames_of(a.lengths, b + mine, a.T) : 0;
        nu.clear(), nd.clear(), nz.clear();
        if (n_frames > 0) {
            nu.load(pu), nd.load(pd);
            if (a.z) nz.load(pz);
        }
    };
    fetch(b0);
    for (; b0 < a.B; b0 += step) {
        float h[NB][4];
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) h[i][k] = next[i].get(k);
        float u = nu.get(0), s = nd.get(0), gate = nz.get(0);
        const int frames = n_frames;
        const T *qu = pu, *qd = pd, *qz = pz;  // (further frames)
        pu += step * a.u_seq, pd += step * a.dt_seq, pz += step * a.z_seq;
        fetch(b0 + step);
        T *qy = py;
        const T *qB = pB, *qC = pC;
        for (int t = 0; t < a.T; ++t) {  // (sequences differ in frames: all lanes take part in the shuffles)
            const bool on = t < frames;
            if (t > 0 && on) {
                qu += a.u_frame, qd += a.dt_frame, qz += a.z_frame;
                u = to_f32(*qu), s = to_f32(*qd);
                if (a.z) gate = to_f32(*qz);
            }
            const unsigned group_on = __ballot_sync(0xffffffffu, on) >> (lane - q);  // bit i: sequence i has this frame
            Run<T, 4> rB[NB], rC[NB];
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const int some = group_on >> i & 1 ? count : 0;
                if (!VEC) {
                    rB[i].load_some(qB + i * a.Bm_seq, some), rC[i].load_some(qC + i * a.Cm_seq, some);
                } else {
                    rB[i].clear(), rC[i].clear();
                    if (some) rB[i].load(qB + i * a.Bm_seq), rC[i].load(qC + i * a.Cm_seq);
                }
            }
            qB += a.Bm_frame, qC += a.Cm_frame;
            s = __fadd_rn(s, bias);
            if (a.softplus) s = softplus(s);
            if (!on) s = 0.0f;  // (a frame that is not there has a step of 0 and no Bm: the state stays as it is)
            const float su = on ? __fmul_rn(s, u) : 0.0f;
            float y[NB];
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const float si = __shfl_sync(0xffffffffu, s, lane - q + i), sui = __shfl_sync(0xffffffffu, su, lane - q + i);
                y[i] = 0.0f;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    h[i][k] = __fmaf_rn(factor(si, A[k]), h[i][k], __fmul_rn(sui, rB[i].get(k)));
                    y[i] = __fmaf_rn(rC[i].get(k), h[i][k], y[i]);
                }
            }
            // NB sums over L lanes: whole sums where there are more lanes than sequences, then halved, until lane q has its own
#pragma unroll
            for (int o = L / 2; o >= NB && o > 0; o >>= 1)
#pragma unroll
                for (int i = 0; i < NB; ++i) y[i] = __fadd_rn(y[i], __shfl_xor_sync(0xffffffffu, y[i], o));
#pragma unroll
            for (int o = NB / 2; o > 0; o >>= 1)
#pragma unroll
                for (int i = 0; i < o; ++i) {
                    const float send = q & o ? y[i] : y[i + o], keep = q & o ? y[i + o] : y[i];
                    y[i] = __fadd_rn(keep, __shfl_xor_sync(0xffffffffu, send, o));
                }
            if (on && q < NB) {
                float o = __fmaf_rn(skip, u, y[0]);
                if (a.z) o = __fmul_rn(o, silu(gate));
                *qy = from_f32<T>(o);
            }
            qy += a.y_frame;
        }
        if (a.state_out) {
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                if (b0 + i >= a.B) continue;
                Run<float, 4> o;
                o.set(h[i]);
                if (!VEC)
                    o.store_some(p_out + i * row, count);
                else if (count)
                    o.store(p_out + i * row);
            }
            p_out += step * row;
        }
        py += step * a.y_seq, pB += step * a.Bm_seq, pC += step * a.Cm_seq;
    }
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
// The address of a shared variable in another block of the cluster, and a load from it.
__device__ __forceinline__ uint32_t peer_address(const void *p, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ float peer_load(uint32_t at) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
    return v;
}

// Whole sequences, a warp by itself: 32 / L channels of one group over a part of a sequence's frames, tile by tile of kTile
// frames. Its lanes load u, dt (and z) in runs of channels, form s = softplus(dt) and s u, and leave them in shared memory
// beside the tile's Bm and Cm; then L lanes a channel, NS states each (or 2 L lanes two channels, half as many), carry the
// states over the tile's frames; then the lanes that loaded u and z finish the outputs. The next tile's loads are in flight
// meanwhile. No block-wide barriers: the phases of a block's warps overlap.
//
// Where sequences are few, `parts` warps (of a block, or of a cluster of blocks) share each one's frames. The recurrence is
// linear: over a part, h' = exp(A S) h + r, with S the sum of its steps and r what it reaches from h = 0. Each warp first
// finds S and r of its part (no Cm, z or outputs), reads those of the parts before its own from shared memory, composes its
// first state from them, and then goes over its part once more with it. Where that state is not finite, the factor of a part
// (exp(A S) with A S > 0) or what it reached alone may have overflowed although the state does not: the warp then goes over all
// frames from the first on, without their outputs before its part, and has what the formula gives (1 x 4000 x 1000 x 16 fp32 with a NaN
// in each channel's first frame 333 us, without 43).
//
// Bound: instructions. A frame of 16 channels x 16 states takes a warp 57 of them (16 states x 2: a product each for the
// exponent and the input, a multiply-add each for the state and the sum, the exponential), 103 cycles alone for the steps and 68
// for loading and finishing; three or four warps a scheduler overlap to 0.57 instructions a cycle, shared memory's port
// 0.61 busy, the multiply-add units 0.46, the exponential's 0.42. 16 x 1000 x 2048 x 16: bf16 197 us, fp32 197 (2.7 TB/s); padded to a
// third, bf16 128. One sequence, 4000 x 1000 x 16 fp32 in 16 parts: 45 us. (Forming the next tile's steps between the frames'
// products: 257 us and 52; sixteen states a lane: 240 and 74.)
constexpr int kTile = 16;
template <int NS, int L>
struct ScanWarp {
    static constexpr int kChans = 32 / L;                // of a warp
    static constexpr int kStates = NS * L;               // of a channel, padded
    static constexpr int kSide = L < 4 ? 1 : 2;          // channels side by side in a lane
    static constexpr int kMine = NS / kSide, kLanes = kSide * L;  // states a lane holds of each, lanes of such a set
    static constexpr int kEach = kTile / L;              // values a lane loads of each array
    static constexpr int V = kEach < 4 ? kEach : 4, kRuns = kEach / V;
    static constexpr int kRowLanes = kChans / V, kRows = 32 / kRowLanes;  // lanes a frame, frames a load
    static constexpr int kBCEach = (kTile * kStates / 4 + 31) / 32;       // runs of four a lane loads of Bm and Cm
    static constexpr bool kBCAhead = kBCEach <= 4;       // a tile ahead, while registers allow it
    static constexpr int kBlockWarps = kStates <= 64 ? 4 : 2;  // (48 KB of shared memory a block)

    alignas(16) float2 s[kTile][kChans];  // steps s and s u
    alignas(16) float B[kTile][kStates], C[kTile][kStates];
    struct Part {
        float part[NS][32], sum[kSide][32];   // r and S
    } own;                                // of this warp's part
    float start[NS][32];                  // the states that a part starts from, where it is the first
};

// A frame's factors exp2(s A), its step h <- f h + su B and the sum of C h, for M states in pairs: one instruction for two
// results.
template <int M>
__device__ __forceinline__ void factors(float2 (&f)[M / 2], const float2 (&A)[M / 2], float s) {
    const float2 s2 = make_float2(s, s);
#pragma unroll
    for (int i = 0; i < M / 2; ++i) {
        const float2 x = ffma2_rn(s2, A[i], f2(kBias));
        f[i] = make_float2(exp2_hw(x.x), exp2_hw(x.y));
    }
}
template <int M>
__device__ __forceinline__ void load_pairs(float2 (&to)[M / 2], const float *from) {
#pragma unroll
    for (int i = 0; i < M / 2; i += 2) {
        const float4 v = *reinterpret_cast<const float4 *>(from + 2 * i);
        to[i] = make_float2(v.x, v.y), to[i + 1] = make_float2(v.z, v.w);
    }
}
// The steps s and s u of channels side by side.
__device__ __forceinline__ void load_steps(float2 (&to)[1], const float2 *from) { to[0] = *from; }
__device__ __forceinline__ void load_steps(float2 (&to)[2], const float2 *from) {
    const float4 v = *reinterpret_cast<const float4 *>(from);
    to[0] = make_float2(v.x, v.y), to[1] = make_float2(v.z, v.w);
}
template <int M>
__device__ __forceinline__ void advance(float2 (&h)[M / 2], const float2 (&f)[M / 2], float su, const float2 (&B)[M / 2]) {
    const float2 su2 = make_float2(su, su);
#pragma unroll
    for (int i = 0; i < M / 2; ++i) h[i] = ffma2_rn(f[i], h[i], fmul2_rn(su2, B[i]));
}
template <int M>
__device__ __forceinline__ float dot(const float2 (&h)[M / 2], const float2 (&C)[M / 2]) {
    float2 y = fmul2_rn(h[0], C[0]);
#pragma unroll
    for (int i = 1; i < M / 2; ++i) y = ffma2_rn(h[i], C[i], y);
    return __fadd_rn(y.x, y.y);
}

template <typename T, int NS, int L, bool VEC>
__global__ void __launch_bounds__(32 * ScanWarp<NS, L>::kBlockWarps, sizeof(T) == 4 ? 2 : 3) ssm_scan_kernel(const ScanArgs a) {
    using Sh = ScanWarp<NS, L>;
    constexpr int V = Sh::V, R = Sh::kRuns, W = Sh::kBlockWarps, BC = Sh::kBCEach, X = Sh::kSide, M = Sh::kMine, Q = Sh::kLanes;
    __shared__ Sh all[W];
    __shared__ typename Sh::Part whole;  // of the block's parts together
    __shared__ __align__(16) float all_y[W][kTile][Sh::kChans];  // sums over the states (apart: nothing else may be waited for with them)
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Sh &sh = all[warp];
    float(&yw)[kTile][Sh::kChans] = all_y[warp];
    const int64_t at = (int64_t)blockIdx.x * W + warp;
    const int rank = (int)at & (a.parts - 1);  // (parts is a power of two)
    int64_t unit = at >> (31 - __clz(a.parts));
    const bool there = unit < a.units;  // (a warp without work still takes part in the barriers)
    if (!there) unit = 0;
    const Split of_blocks = split(unit, a.group_blocks), of_groups = split(of_blocks.quot, a.groups);
    const int blk = (int)of_blocks.rem, g = (int)of_groups.rem;
    const int64_t b = of_groups.quot, d0 = g * a.group_chans + (int64_t)blk * Sh::kChans;
    const int chans = (int)min((int64_t)Sh::kChans, (g + 1) * a.group_chans - d0);
    const int n = there ? frames_of(a.lengths, b, a.T) : 0;
    const int tiles = (n + kTile - 1) / kTile, each = (tiles + a.parts - 1) / a.parts * kTile;
    const int first = min(n, rank * each), last = min(n, first + each);

    // this lane's place in the loads and stores: frames row + j kRows of the tile, channels run .. run + V
    const int row = lane / Sh::kRowLanes, run = V * (lane % Sh::kRowLanes), left = chans - run;
    float bias[V], skip[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        bias[v] = a.dt_bias && v < left ? __ldg(a.dt_bias + d0 + run + v) : 0.0f;
        skip[v] = a.skip && v < left ? __ldg(a.skip + d0 + run + v) : 0.0f;
    }
    // the next tile's values, and where they lie
    Run<T, V> ru[R], rd[R], rz[R];
    Run<T, 4> rB[BC], rC[BC];
    Run<T, V> cu[R];  // u of the tile at work, for its outputs
    const T *pu, *pd, *pz, *pB, *pC;
    auto seek = [&](int t0) {
        auto at = [&](const void *p, int64_t seq, int64_t frame, int t, int64_t i) {
            return static_cast<const T *>(p) + b * seq + t * frame + i;
        };
        pu = at(a.u, a.u_seq, a.u_frame, t0 + row, d0 + run);
        pd = at(a.dt, a.dt_seq, a.dt_frame, t0 + row, d0 + run);
        pz = at(a.z, a.z_seq, a.z_frame, t0 + row, d0 + run);
        pB = at(a.Bm, a.Bm_seq, a.Bm_frame, t0, (int64_t)g * a.N);
        pC = at(a.Cm, a.Cm_seq, a.Cm_frame, t0, (int64_t)g * a.N);
    };
    auto fetch_bc = [&](int t0, Run<T, 4> *r, const T *&p, int64_t frame) {
#pragma unroll
        for (int i = 0; i < BC; ++i) {
            const int e = 4 * (lane + 32 * i), t = e / Sh::kStates, k = e % Sh::kStates;
            const int count = t0 + t < last && e < kTile * Sh::kStates ? a.N - k : 0;
            if constexpr (VEC) {
                r[i].clear();
                if (count > 0) r[i].load(p + t * frame + k);
            } else {
                r[i].load_some(p + t * frame + k, count);
            }
        }
        p += kTile * frame;
    };
    auto get = [&](int t0, Run<T, V> *r, const T *&p, int64_t frame) {  // reads tile t0, where p stands, and moves p on
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int count = t0 + row + j * Sh::kRows < last ? left : 0;
            if constexpr (VEC) {
                r[j].clear();
                if (count > 0) r[j].load(p + j * Sh::kRows * frame);
            } else {
                r[j].load_some(p + j * Sh::kRows * frame, count);
            }
        }
        p += kTile * frame;
    };
    auto fetch = [&](int t0, bool final) {
        get(t0, ru, pu, a.u_frame);
        get(t0, rd, pd, a.dt_frame);
        if constexpr (Sh::kBCAhead) {
            fetch_bc(t0, rB, pB, a.Bm_frame);
            if (final) fetch_bc(t0, rC, pC, a.Cm_frame);
        }
    };
    seek(first);
    fetch(first, a.parts == 1);
    // and in the recurrence: channels c .. c + X, states n0 .. n0 + M of each. (Two channels side by side share the reads of Bm
    // and Cm, but have twice the sums to exchange: 16 x 500 x 2048 x 32 bf16 227 us by one, 177 by two; 16 x 1000 x 2048 x 16 198 and
    // 207.)
    const int c = lane / Q * X, q = lane % Q, n0 = q * M;
    float2 A[X][M / 2], h[X][M / 2];
    const bool start = there && rank == 0 && a.state_in;
    auto state_at = [&](int x, int i) { return (b * a.D + d0 + c + x) * a.N + n0 + i; };
#pragma unroll
    for (int x = 0; x < X; ++x)
#pragma unroll
        for (int i = 0; i < M; ++i) {
            const bool ok = c + x < chans && n0 + i < a.N;
            const float v = ok ? rate(__ldg(a.A + (d0 + c + x) * a.N + n0 + i)) : 0.0f;
            const float s = ok && start ? a.state_in[state_at(x, i)] : 0.0f;
            if (i & 1)
                A[x][i / 2].y = v, h[x][i / 2].y = s;
            else
                A[x][i / 2].x = v, h[x][i / 2].x = s;
        }
    auto put = [&](float (&to)[NS][32]) {
#pragma unroll
        for (int i = 0; i < NS; ++i) to[i][lane] = i & 1 ? h[i / M][i % M / 2].y : h[i / M][i % M / 2].x;
    };
    auto take = [&](const float (&from)[NS][32]) {
#pragma unroll
        for (int i = 0; i < NS; i += 2) h[i / M][i % M / 2] = make_float2(from[i][lane], from[i + 1][lane]);
    };
    auto stage = [&](int t0, bool final) {  // a frame that is not there has a step of 0, which leaves the states as they are
        if constexpr (!Sh::kBCAhead) {
            fetch_bc(t0, rB, pB, a.Bm_frame);
            if (final) fetch_bc(t0, rC, pC, a.Cm_frame);
        }
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int r = row + j * Sh::kRows;
            const bool on = t0 + r < last;
#pragma unroll
            for (int v = 0; v < V; v += 2) {
                const int w = v + 1 < V ? v + 1 : v;
                const float2 u = make_float2(ru[j].get(v), ru[j].get(w));
                float2 s = fadd2_rn(make_float2(rd[j].get(v), rd[j].get(w)), make_float2(bias[v], bias[w]));
                if (a.softplus) s = softplus2(s);
                if (!on) s = make_float2(0.0f, 0.0f);
                const float2 su = fmul2_rn(s, u);
                if constexpr (V > 1)
                    *reinterpret_cast<float4 *>(&sh.s[r][run + v]) = make_float4(s.x, su.x, s.y, su.y);
                else
                    sh.s[r][run] = make_float2(s.x, su.x);
            }
        }
#pragma unroll
        for (int i = 0; i < BC; ++i) {
            const int e = 4 * (lane + 32 * i);
            if (e < kTile * Sh::kStates) {
                *reinterpret_cast<float4 *>(&sh.B[0][0] + e) = make_float4(rB[i].get(0), rB[i].get(1), rB[i].get(2), rB[i].get(3));
                if (final)
                    *reinterpret_cast<float4 *>(&sh.C[0][0] + e) = make_float4(rC[i].get(0), rC[i].get(1), rC[i].get(2), rC[i].get(3));
            }
        }
    };

    int begin = first;  // of the frames that this warp goes over for its outputs
    if (a.parts > 1) {
        put(sh.start);
        float sum[X] = {};
        for (int t0 = first; t0 < last; t0 += kTile) {
            stage(t0, false);
            __syncwarp();
            fetch(t0 + kTile, false);
#pragma unroll 4
            for (int t = 0; t < kTile; ++t) {
                float2 s[X], Bt[M / 2];
                load_steps(s, &sh.s[t][c]);
                load_pairs<M>(Bt, &sh.B[t][n0]);
#pragma unroll
                for (int x = 0; x < X; ++x) {
                    float2 f[M / 2];
                    sum[x] = __fadd_rn(sum[x], s[x].x);
                    factors<M>(f, A[x], s[x].x);
                    advance<M>(h[x], f, s[x].y, Bt);
                }
            }
            __syncwarp();
        }
        put(sh.own.part);
#pragma unroll
        for (int x = 0; x < X; ++x) sh.own.sum[x][lane] = sum[x];
        seek(first);  // the second pass's first loads are in flight meanwhile
        fetch(first, true);
        // The parts of a block, then those of the blocks before it, which the last warp of each has put together. `first_part`
        // takes r as it is: nothing lies before it.
        const bool cluster = a.parts > W;
        const int w0 = cluster ? 0 : warp - rank;  // the first part's warp in this block
        auto compose = [&](const float (&s)[X], const float (&r)[NS], bool first_part) {
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                float &to = i & 1 ? h[i / M][i % M / 2].y : h[i / M][i % M / 2].x;
                const float Ai = i & 1 ? A[i / M][i % M / 2].y : A[i / M][i % M / 2].x;
                to = first_part ? r[i] : __fmaf_rn(factor(s[i / M], Ai), to, r[i]);
            }
        };
        auto compose_warps = [&](float (&total)[X], int end, bool first_part) {  // and the sum of their steps
#pragma unroll
            for (int x = 0; x < X; ++x) total[x] = 0.0f;
            for (int w = w0; w < end; ++w) {
                float r[NS];
#pragma unroll
                for (int k = 0; k < NS; ++k) r[k] = all[w].own.part[k][lane];
                float s[X];
#pragma unroll
                for (int x = 0; x < X; ++x) {
                    s[x] = all[w].own.sum[x][lane];
                    total[x] = __fadd_rn(total[x], s[x]);
                }
                compose(s, r, first_part && w == w0);
            }
        };
        float total[X];
        __syncthreads();
        if (cluster) {
            const int block = rank / W;
            if (warp == W - 1) {
                compose_warps(total, W, true);
                put(whole.part);
#pragma unroll
                for (int x = 0; x < X; ++x) whole.sum[x][lane] = total[x];
            }
            cluster_arrive();
            cluster_wait();
            take(sh.start);
            constexpr int kAtOnce = 4;  // blocks whose values are loaded together
            for (int p0 = 0; p0 < block; p0 += kAtOnce) {
                float s[kAtOnce][X], r[kAtOnce][NS];
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) {
                    if (p0 + i >= block) break;
#pragma unroll
                    for (int x = 0; x < X; ++x) s[i][x] = peer_load(peer_address(&whole.sum[x][lane], p0 + i));
#pragma unroll
                    for (int k = 0; k < NS; ++k) r[i][k] = peer_load(peer_address(&whole.part[k][lane], p0 + i));
                }
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) {
                    if (p0 + i >= block) break;
                    compose(s[i], r[i], p0 + i == 0);
                }
            }
            compose_warps(total, warp, block == 0);
        } else {
            take(sh.start);
            compose_warps(total, warp, true);
        }
        float2 odd = f2(0.0f);
#pragma unroll
        for (int i = 0; i < NS; i += 2) odd = ffma2_rn(h[i / M][i % M / 2], f2(0.0f), odd);
        if (__any_sync(0xffffffffu, !(odd.x == 0.0f && odd.y == 0.0f))) {  // from the sequence's first frame on
            begin = 0;
            seek(0);
            fetch(0, true);
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                const float *at = &all[w0].start[i][lane];
                const float v = cluster ? peer_load(peer_address(at, 0)) : *at;
                if (i & 1)
                    h[i / M][i % M / 2].y = v;
                else
                    h[i / M][i % M / 2].x = v;
            }
        }
        if (cluster) cluster_arrive();  // waited for at the end: the others may still read this block's
    }

    constexpr int kSteps = 8;  // frames between stores: their loads and products overlap
    T *py = static_cast<T *>(a.y) + b * a.y_seq + (begin + row) * a.y_frame + d0 + run;
    for (int t0 = begin; t0 < last; t0 += kTile) {
        stage(t0, true);
#pragma unroll
        for (int j = 0; j < R; ++j) cu[j] = ru[j];
        if (a.z) get(t0, rz, pz, a.z_frame);  // for the outputs, after the steps
        __syncwarp();
        fetch(t0 + kTile, true);
#pragma unroll 1
        for (int tb = 0; tb < kTile; tb += kSteps) {
            float y[X * kSteps];  // by frame and channel
            float2 f[X][M / 2];   // a frame's factors are formed beside the products of the one before
            float2 s[X];
            load_steps(s, &sh.s[tb][c]);
#pragma unroll
            for (int x = 0; x < X; ++x) factors<M>(f[x], A[x], s[x].x);
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                float2 f1[X][M / 2], Bt[M / 2], Ct[M / 2], s1[X];
                load_pairs<M>(Bt, &sh.B[tb + i][n0]);
                load_steps(s1, &sh.s[i + 1 < kSteps ? tb + i + 1 : tb][c]);
                if (i + 1 < kSteps)
#pragma unroll
                    for (int x = 0; x < X; ++x) factors<M>(f1[x], A[x], s1[x].x);
#pragma unroll
                for (int x = 0; x < X; ++x) advance<M>(h[x], f[x], s[x].y, Bt);
                load_pairs<M>(Ct, &sh.C[tb + i][n0]);
#pragma unroll
                for (int x = 0; x < X; ++x) y[X * i + x] = dot<M>(h[x], Ct);
                if (i + 1 < kSteps)
#pragma unroll
                    for (int x = 0; x < X; ++x) {
                        s[x] = s1[x];
#pragma unroll
                        for (int k = 0; k < M / 2; ++k) f[x][k] = f1[x][k];
                    }
            }
            // The sums of as many frames and channels as lanes at a time: each exchange halves the values that a lane holds, until
            // lane q has the q-th of them. (More lanes than values: whole sums over the lanes beyond first.)
            constexpr int kAtOnce = Q < X * kSteps ? Q : X * kSteps;
            if constexpr (Q > kAtOnce)
#pragma unroll
                for (int i = 0; i < X * kSteps; ++i) y[i] = __fadd_rn(y[i], __shfl_xor_sync(0xffffffffu, y[i], kAtOnce));
#pragma unroll
            for (int r = 0; r < X * kSteps; r += kAtOnce) {
#pragma unroll
                for (int o = kAtOnce / 2; o > 0; o >>= 1)
#pragma unroll
                    for (int i = 0; i < o; ++i) {
                        const float send = q & o ? y[r + i] : y[r + i + o], keep = q & o ? y[r + i + o] : y[r + i];
                        y[r + i] = __fadd_rn(keep, __shfl_xor_sync(0xffffffffu, send, o));
                    }
                const int at = r + (q & (kAtOnce - 1));
                if (Q <= kAtOnce || q < kAtOnce) yw[tb + at / X][c + at % X] = y[r];
            }
        }
        __syncwarp();
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int r = row + j * Sh::kRows;
            if (t0 + r < last && t0 >= first) {
                float o[V];
#pragma unroll
                for (int v = 0; v < V; v += 2) {
                    const int w = v + 1 < V ? v + 1 : v;
                    float2 y = ffma2_rn(make_float2(skip[v], skip[w]), make_float2(cu[j].get(v), cu[j].get(w)),
                                        make_float2(yw[r][run + v], yw[r][run + w]));
                    if (a.z) y = fmul2_rn(y, silu2(make_float2(rz[j].get(v), rz[j].get(w))));
                    o[v] = y.x;
                    if (w > v) o[w] = y.y;
                }
                Run<T, V> out;
                out.set(o);
                if constexpr (VEC) {
                    if (left > 0) out.store(py + j * Sh::kRows * a.y_frame);
                } else {
                    out.store_some(py + j * Sh::kRows * a.y_frame, left);
                }
            }
        }
        py += kTile * a.y_frame;
    }
    if (there && a.state_out && rank == a.parts - 1) {
#pragma unroll
        for (int x = 0; x < X; ++x)
#pragma unroll
            for (int i = 0; i < M; ++i)
                if (c + x < chans && n0 + i < a.N) a.state_out[state_at(x, i)] = i & 1 ? h[x][i / 2].y : h[x][i / 2].x;
    }
    if (a.parts > W) cluster_wait();
}

bool aligned_to(const void *p, int64_t seq, int64_t frame, int e, int bytes) {
    return reinterpret_cast<uintptr_t>(p) % bytes == 0 && seq * e % bytes == 0 && frame * e % bytes == 0;
}

template <typename T, int L>
qnn_status launch_step(const ScanArgs &a, cudaStream_t st) {
    constexpr int NB = L < 4 ? L : 4;
    // two waves of blocks, each on a part of the channels and every so many of the sequences
    const int64_t chans = (a.D * L + kStepThreads - 1) / kStepThreads, rounds = (a.B + NB - 1) / NB;
    if (chans > INT32_MAX) return QNN_FAIL(QNN_ERR_INVALID_ARG);
    const int64_t shares = std::min<int64_t>({rounds, std::max<int64_t>(1, 8 * (int64_t)sm_count() / chans), 65535});
    const dim3 grid((unsigned)chans, (unsigned)shares);
    if (a.vec)
        ssm_step_kernel<T, L, true><<<grid, kStepThreads, 0, st>>>(a);
    else
        ssm_step_kernel<T, L, false><<<grid, kStepThreads, 0, st>>>(a);
    return QNN_OK;
}

template <typename T, int NS, int L>
qnn_status launch_tiles(ScanArgs a, cudaStream_t st) {
    using Sh = ScanWarp<NS, L>;
    constexpr int W = Sh::kBlockWarps;
    const int e = sizeof(T);
    // runs of channels and of states are loaded and stored whole where every one of them is aligned and full
    auto whole = [&](const void *p, int64_t seq, int64_t frame, int values) { return !p || aligned_to(p, seq, frame, e, values * e); };
    const bool vec = a.group_chans % Sh::V == 0 && a.N % 4 == 0 && whole(a.u, a.u_seq, a.u_frame, Sh::V) &&
                     whole(a.dt, a.dt_seq, a.dt_frame, Sh::V) && whole(a.z, a.z_seq, a.z_frame, Sh::V) &&
                     whole(a.y, a.y_seq, a.y_frame, Sh::V) && whole(a.Bm, a.Bm_seq, a.Bm_frame, 4) && whole(a.Cm, a.Cm_seq, a.Cm_frame, 4);
    const int64_t blocks_g = (a.group_chans + Sh::kChans - 1) / Sh::kChans;
    a.units = a.B * a.groups * blocks_g;
    a.group_blocks = (int)blocks_g;
    // parts: while the SMs have fewer than four warps each, but no fewer than two tiles a part
    const int64_t tiles = (a.T + kTile - 1) / kTile;
    int parts = 1;
    while (parts < 16 * W && a.units * parts < 4 * (int64_t)sm_count() && 4 * parts <= tiles) parts *= 2;
    const auto kern = vec ? ssm_scan_kernel<T, NS, L, true> : ssm_scan_kernel<T, NS, L, false>;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.blockDim = dim3(32 * W);
    cfg.stream = st;
    cfg.attrs = attr;
    auto shared_by = [&](int n) {  // a cluster of as many blocks a unit
        const int cluster = std::max(1, n / W);
        a.parts = n;
        attr[0].val.clusterDim.x = (unsigned)cluster;
        cfg.numAttrs = cluster > 1 ? 1 : 0;
        cfg.gridDim = dim3((unsigned)std::min<int64_t>((a.units * n + W - 1) / W, UINT32_MAX));
    };
    shared_by(parts);
    if (parts > 8 * W) {  // a device need not have room for more than eight (it is asked once)
        static std::atomic<int> room[2][64];
        int dev = 0;
        QNN_CUDA_TRY(cudaGetDevice(&dev));
        if (dev < 0 || dev >= 64) return QNN_FAIL(QNN_ERR_CUDA);
        int known = room[vec][dev].load(std::memory_order_acquire);
        if (!known) {
            int clusters = 0;
            if (cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
                cudaOccupancyMaxActiveClusters(&clusters, kern, &cfg) != cudaSuccess)
                cudaGetLastError();
            known = clusters > 0 ? 1 : -1;
            room[vec][dev].store(known, std::memory_order_release);
        }
        if (known < 0) shared_by(8 * W);
    }
    if (cfg.gridDim.x > INT32_MAX) return QNN_FAIL(QNN_ERR_INVALID_ARG);
    QNN_CUDA_TRY(cudaLaunchKernelEx(&cfg, kern, a));
    return QNN_OK;
}

template <typename T>
qnn_status launch_scan(ScanArgs &a, cudaStream_t st) {
    const int e = sizeof(T);
    a.group_chans = a.D / a.groups;
    a.parts = 1;
    a.vec = false;
    if (a.T <= kStepFrames) {
        auto at16 = [](const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
        a.vec = a.N % 4 == 0 && at16(a.A) && at16(a.state_in) && at16(a.state_out) &&
                (a.T == 0 || (aligned_to(a.Bm, a.Bm_seq, a.Bm_frame, e, 4 * e) && aligned_to(a.Cm, a.Cm_seq, a.Cm_frame, e, 4 * e)));
        if (a.N <= 4) return launch_step<T, 1>(a, st);
        if (a.N <= 8) return launch_step<T, 2>(a, st);
        if (a.N <= 16) return launch_step<T, 4>(a, st);
        if (a.N <= 32) return launch_step<T, 8>(a, st);
        if (a.N <= 64) return launch_step<T, 16>(a, st);
        return launch_step<T, 32>(a, st);
    }
    if (a.N <= 4) return launch_tiles<T, 4, 1>(a, st);
    if (a.N <= 8) return launch_tiles<T, 8, 1>(a, st);
    if (a.N <= 16) return launch_tiles<T, 8, 2>(a, st);
    if (a.N <= 32) return launch_tiles<T, 8, 4>(a, st);
    if (a.N <= 64) return launch_tiles<T, 8, 8>(a, st);
    return launch_tiles<T, 8, 16>(a, st);
}

template <typename T, int W>
qnn_status launch_conv(ConvArgs a, cudaStream_t st) {
    constexpr int V = 4;  // (eight 16-bit values a thread: 26 us where four take 22)
    const int e = sizeof(T);
    auto whole = [](const void *p, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; };
    const bool vec = a.D % V == 0 && whole(a.state_in, V * e) && whole(a.state_out, V * e) && whole(a.w, 16) &&
                     (a.T == 0 || (aligned_to(a.x, a.x_seq, a.x_frame, e, V * e) && aligned_to(a.y, a.y_seq, a.y_frame, e, V * e)));
    a.runs = vec ? a.D / V : a.D;
    // Frames a thread: 40, or 16 while that leaves the SMs less than two waves of blocks (1 x 300 x 2048 bf16 5.8 us with 32 and
    // 4.3 so). A few frames take a round of one (a kernel of half the registers: 256 x 1 x 2048 fp32 6.3 us with eight).
    const bool few = a.T <= 4;
    a.chunk = few || a.B * a.runs * ((a.T + 39) / 40) < 8 * kConvThreads * (int64_t)sm_count() ? 16 : 40;
    a.chunks = std::max<int64_t>(1, (a.T + a.chunk - 1) / a.chunk);
    const int64_t blocks = (a.B * a.runs * a.chunks + kConvThreads - 1) / kConvThreads;
    if (blocks > INT32_MAX) return QNN_FAIL(QNN_ERR_INVALID_ARG);
    const auto kern = vec ? (few ? causal_conv_kernel<T, W, V, 1> : causal_conv_kernel<T, W, V, 8>)
                          : (few ? causal_conv_kernel<T, W, 1, 1> : causal_conv_kernel<T, W, 1, 8>);
    kern<<<(unsigned)blocks, kConvThreads, 0, st>>>(a);
    return QNN_OK;
}

template <typename T>
qnn_status launch_conv(const ConvArgs &a, int W, cudaStream_t st) {
    static_assert(kMostTaps == 8);
    switch (W) {
        case 1: return launch_conv<T, 1>(a, st);
        case 2: return launch_conv<T, 2>(a, st);
        case 3: return launch_conv<T, 3>(a, st);
        case 4: return launch_conv<T, 4>(a, st);
        case 5: return launch_conv<T, 5>(a, st);
        case 6: return launch_conv<T, 6>(a, st);
        case 7: return launch_conv<T, 7>(a, st);
        default: return launch_conv<T, 8>(a, st);
    }
}

constexpr int64_t kMostCount = (int64_t)1 << 40, kMostFrames = 1 << 30;

// A [B][T][width] array: its strides are in range, its first element aligned to its type.
bool frames_ok(const void *p, int64_t B, int64_t T, int64_t seq, int64_t frame, int e) {
    return reach_ok(B, seq) && reach_ok(T, frame) && (reinterpret_cast<uintptr_t>(p) & (e - 1)) == 0;
}
// No frame of an output overlaps another: sequences apart and frames apart within one, or the other way round.
bool apart(int64_t B, int64_t T, int64_t width, int64_t seq, int64_t frame) {
    const bool inner = T <= 1 || frame >= width, outer = B <= 1 || seq >= width;
    return inner && outer && (B <= 1 || T <= 1 || seq >= (T - 1) * frame + width || frame >= (B - 1) * seq + width);
}
Span frames_span(const void *p, int64_t B, int64_t T, int64_t width, int64_t seq, int64_t frame, int e) {
    return T > 0 ? Span(p, ((B - 1) * seq + (T - 1) * frame + width) * e) : Span();
}
bool sizes_ok(int64_t B, int64_t T, int64_t D) {
    return B >= 0 && T >= 0 && D >= 1 && T <= kMostFrames && D <= INT32_MAX && B <= INT32_MAX && B * D <= kMostCount && reach_ok(T, B * D);
}
bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }
bool local_or_null(const void *p) { return !p || is_local_ptr(p); }

}  // namespace
}  // namespace qnn

using namespace qnn;

extern "C" qnn_status qnn_causal_conv(const void *x, int64_t x_seq, int64_t x_frame, int dtype, int64_t B, int64_t T, int64_t D,
                                      const float *w, int32_t W, const float *bias, int silu, const void *state_in,
                                      void *state_out, const int32_t *lengths, void *y, int64_t y_seq, int64_t y_frame,
                                      void *stream) {
    if (!dtype_ok(dtype) || !sizes_ok(B, T, D) || W < 1 || W > kMostTaps) return QNN_ERR_INVALID_ARG;
    const int e = dtype_size(dtype);
    if (!frames_ok(x, B, T, x_seq, x_frame, e) || !frames_ok(y, B, T, y_seq, y_frame, e) || !apart(B, T, D, y_seq, y_frame) ||
        !frames_ok(state_in, 0, 0, 0, 0, e) || !frames_ok(state_out, 0, 0, 0, 0, e) || !aligned4(w) || !aligned4(bias) || !aligned4(lengths))
        return QNN_ERR_INVALID_ARG;
    if (B == 0 || (T == 0 && !state_out)) return QNN_OK;
    if ((T > 0 && (!is_local_ptr(x) || !is_local_ptr(y))) || !is_local_ptr(w) || !local_or_null(bias) || !local_or_null(state_in) ||
        !local_or_null(state_out) || !local_or_null(lengths))
        return QNN_ERR_INVALID_ARG;
    const int64_t state = B * (W - 1) * D * e;
    const Span in[5] = {frames_span(x, B, T, D, x_seq, x_frame, e), Span(w, 4 * D * W), Span(bias, 4 * D), Span(lengths, 4 * B),
                        Span(state_in, state)};
    const Span ys = frames_span(y, B, T, D, y_seq, y_frame, e), so(state_out, state);
    if (ys.meets(so)) return QNN_ERR_INVALID_ARG;
    for (int i = 0; i < 5; ++i)
        if (ys.meets(in[i]) || (so.meets(in[i]) && !(i == 4 && state_in == state_out))) return QNN_ERR_INVALID_ARG;
    ConvArgs a;
    a.x = x, a.state_in = state_in, a.state_out = state_out, a.y = y, a.w = w, a.bias = bias, a.lengths = lengths;
    a.x_seq = x_seq, a.x_frame = x_frame, a.y_seq = y_seq, a.y_frame = y_frame, a.B = B, a.T = T, a.D = D, a.silu = silu != 0;
    cudaStream_t st = as_stream(stream);
    ProfScope prof("causal_conv", st);
    QNN_TRY(with_type(dtype, [&](auto t) { return launch_conv<decltype(t)>(a, W, st); }));
    QNN_CUDA_TRY(cudaGetLastError());
    return QNN_OK;
}

extern "C" qnn_status qnn_ssm_scan(const qnn_ssm_args *args, void *stream) {
    if (!args) return QNN_ERR_INVALID_ARG;
    const qnn_ssm_args &a = *args;
    if (!dtype_ok(a.dtype) || !sizes_ok(a.B, a.T, a.D) || a.N < 1 || a.N > kMostStates || a.groups < 1 || a.D % a.groups)
        return QNN_ERR_INVALID_ARG;
    const int e = dtype_size(a.dtype);
    const int64_t gn = (int64_t)a.groups * a.N;
    if (!frames_ok(a.u, a.B, a.T, a.u_seq, a.u_frame, e) || !frames_ok(a.dt, a.B, a.T, a.dt_seq, a.dt_frame, e) ||
        !frames_ok(a.Bm, a.B, a.T, a.Bm_seq, a.Bm_frame, e) || !frames_ok(a.Cm, a.B, a.T, a.Cm_seq, a.Cm_frame, e) ||
        (a.z && !frames_ok(a.z, a.B, a.T, a.z_seq, a.z_frame, e)) || !frames_ok(a.y, a.B, a.T, a.y_seq, a.y_frame, e) ||
        !apart(a.B, a.T, a.D, a.y_seq, a.y_frame) || !aligned4(a.A) || !aligned4(a.skip) || !aligned4(a.dt_bias) ||
        !aligned4(a.state_in) || !aligned4(a.state_out) || !aligned4(a.lengths))
        return QNN_ERR_INVALID_ARG;
    if (a.B == 0 || (a.T == 0 && !a.state_out)) return QNN_OK;
    if ((a.T > 0 && (!is_local_ptr(a.u) || !is_local_ptr(a.dt) || !is_local_ptr(a.Bm) || !is_local_ptr(a.Cm) || !is_local_ptr(a.y) ||
                     !local_or_null(a.z))) ||
        !is_local_ptr(a.A) || !local_or_null(a.skip) || !local_or_null(a.dt_bias) || !local_or_null(a.state_in) ||
        !local_or_null(a.state_out) || !local_or_null(a.lengths))
        return QNN_ERR_INVALID_ARG;
    const int64_t state = 4 * a.B * a.D * a.N;
    const Span in[10] = {frames_span(a.u, a.B, a.T, a.D, a.u_seq, a.u_frame, e),
                         frames_span(a.dt, a.B, a.T, a.D, a.dt_seq, a.dt_frame, e),
                         frames_span(a.Bm, a.B, a.T, gn, a.Bm_seq, a.Bm_frame, e),
                         frames_span(a.Cm, a.B, a.T, gn, a.Cm_seq, a.Cm_frame, e),
                         a.z ? frames_span(a.z, a.B, a.T, a.D, a.z_seq, a.z_frame, e) : Span(),
                         Span(a.A, 4 * a.D * a.N),
                         Span(a.skip, 4 * a.D),
                         Span(a.dt_bias, 4 * a.D),
                         Span(a.lengths, 4 * a.B),
                         Span(a.state_in, state)};
    const Span ys = frames_span(a.y, a.B, a.T, a.D, a.y_seq, a.y_frame, e), so(a.state_out, state);
    if (ys.meets(so)) return QNN_ERR_INVALID_ARG;
    for (int i = 0; i < 10; ++i)
        if (ys.meets(in[i]) || (so.meets(in[i]) && !(i == 9 && a.state_in == a.state_out))) return QNN_ERR_INVALID_ARG;
    ScanArgs k;
    static_cast<qnn_ssm_args &>(k) = a;
    cudaStream_t st = as_stream(stream);
    ProfScope prof("ssm_scan", st);
    QNN_TRY(with_type(a.dtype, [&](auto t) { return launch_scan<decltype(t)>(k, st); }));
    QNN_CUDA_TRY(cudaGetLastError());
    return QNN_OK;
}
