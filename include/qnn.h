/*
 * qnn.h — C ABI of libqnn: 8-bit quantized LSTM acoustic-model inference on one GB300 (sm_103a).
 *
 * The method is the one of Alvarez, Prabhavalkar and Bakhtin, "On the efficient representation
 * and execution of deep acoustic models" (INTERSPEECH 2016):
 *   - a uniform linear quantizer to 8 bits, S = 255, Q = S / (Vmax - Vmin), with the offset
 *     rounded consistently: V' = round(Q V) - round(Q Vmin)          (Sec. 3, eq. 2);
 *   - products of independently quantized matrices in 8-bit integers with 32-bit accumulators,
 *     recovered as (V_a'' V_b'') / (Q_a Q_b), V'' = V' + round(Q Vmin)  (Sec. 3.1, eq. 1, eq. 3);
 *   - layers that take fp32 in and give fp32 out: inputs quantized on the fly, weights offline,
 *     recovered products plus bias through the activation function (Sec. 3.1, Fig. 1);
 *   - one quantization unit per weight matrix, e.g. per LSTM gate (Sec. 3.1, last paragraph).
 *
 * Conventions for every call:
 *   - Matrices are row-major with an explicit leading dimension in elements.
 *   - Unless a call says otherwise, pointers are DEVICE pointers on the current CUDA device, and
 *     the caller owns them. A host pointer where a device pointer is required is rejected with
 *     QNN_ERR_INVALID_ARG.
 *   - `stream` is a cudaStream_t (NULL = the legacy default stream). Calls are asynchronous on it:
 *     argument errors are returned at once; errors found by the GPU (non-finite inputs, a
 *     persistent-kernel wait that timed out) are recorded in a device status word and returned
 *     by qnn_device_status().
 *   - There is no CPU fallback: without a usable CUDA device every compute call returns
 *     QNN_ERR_CUDA.
 */
#ifndef QNN_H
#define QNN_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    QNN_OK = 0,
    QNN_ERR_INVALID_ARG = 1,  /* bad size, stride, pointer kind or enum value */
    QNN_ERR_NONFINITE = 2,    /* a quantization unit held NaN or +-Inf (no range exists, Sec. 3) */
    QNN_ERR_K_TOO_LARGE = 3,  /* K > 33025: K * 255^2 would overflow the 32-bit accumulator */
    QNN_ERR_CUDA = 4,         /* a CUDA runtime call failed, or no device */
    QNN_ERR_TIMEOUT = 5,      /* a grid-wide wait in a persistent kernel gave up (bounded spin) */
    QNN_ERR_NO_COOP = 6,      /* the persistent grid cannot be co-resident on this device */
    QNN_ERR_NO_MEMORY = 7,    /* device allocation failed */
} qnn_status;

typedef enum { QNN_PER_MATRIX = 0, QNN_PER_ROW = 1 } qnn_granularity;

/* Output layer of an LSTM model: none (the top layer's outputs are returned), 8-bit
 * ("quant-all" of Sec. 5), or float ("quant" of Sec. 5: all layers but the softmax quantized). */
typedef enum { QNN_OUT_NONE = 0, QNN_OUT_QUANT = 1, QNN_OUT_FLOAT = 2 } qnn_output_mode;

/* Largest reduction length for which 8-bit codes cannot overflow a 32-bit accumulator:
 * K * 255 * 255 <= 2^31 - 1. */
#define QNN_K_MAX 33025

/* Quantization parameters of one unit (16 bytes). vmin/vmax: the exact fp32 range of the unit;
 * Q: the fp32 scale S / (vmax - vmin), S = 255 (Sec. 3); z: round(Q vmin), the rounded offset of
 * eq. (2). Code of v: clamp(round(Q v) - z, 0, 255). Recovery (eq. 3): (code + z) / Q.
 * Readings where the paper is silent: Q is raised by single ulps until the range maximum reaches
 * code 255; codes are clamped to [0, 255]; a unit with vmax == vmin, or with |Q vmin| or
 * |Q vmax| >= 2^22, uses Q = 255 / max(|vmin|, |vmax|) (Q = 1 if all values are 0). Where that
 * overflows (a maximum below about 7.5e-37) Q is infinite; the conversions to integers saturate (NaN to
 * 0) and the difference wraps, so that a unit's codes are all 0, or, if its least value is 0, 255 for
 * every other value; products recover 0 from it. That rule
 * takes the place of a range error: no call fails on a unit without a usable range (an all-zero
 * initial state, a constant row); only non-finite values are errors (QNN_ERR_NONFINITE). */
typedef struct {
    float vmin;
    float vmax;
    float Q;
    int32_t z;
} qnn_qparams;

/* Human-readable name of a status code (static string). */
const char *qnn_status_string(qnn_status s);

/* Waits for `stream`, then returns and clears the device status word of the current device:
 * QNN_OK, QNN_ERR_NONFINITE or QNN_ERR_TIMEOUT (the first error recorded since the last call), or
 * QNN_ERR_CUDA if the stream itself failed. */
qnn_status qnn_device_status(void *stream);

/*
 * qnn_quantize — Sec. 3 "Quantizing" and eq. (2): fp32 -> 8-bit codes, on the fly.
 *   x          [rows x cols] fp32, leading dimension ldx >= cols.
 *   granularity QNN_PER_MATRIX: one unit for the whole matrix (one params entry);
 *              QNN_PER_ROW: one unit per row (rows params entries).
 *   codes      [rows x cols] uint8 out, leading dimension ldc >= cols.
 *   params     out: 1 or `rows` entries.
 *   code_sums  out, nullable: [rows] int32, sum of each row's codes (used by the offset terms of
 *              eq. 1).
 * Non-finite values: the unit's codes are unspecified and QNN_ERR_NONFINITE is recorded.
 * Per-matrix quantization allocates a small library-owned scratch buffer on first use; calls on different
 * streams have parts of their own.
 */
qnn_status qnn_quantize(const float *x, int64_t rows, int64_t cols, int64_t ldx, int granularity,
                        uint8_t *codes, int64_t ldc, qnn_qparams *params, int32_t *code_sums, void *stream);

/*
 * qnn_qmatmul — eq. (1) with eq. (2)'s offsets, recovered to fp32 (Fig. 1: y = R(Mult(Q(X), W')) + B).
 *   A     [M x K] uint8 activation codes (lda >= K); pa: 1 (ga = QNN_PER_MATRIX) or M
 *         (ga = QNN_PER_ROW) params; rsA [M] int32 row code sums of A.
 *   W     [N x K] uint8 weight codes (ldw >= K): the rows split into n_blocks equal blocks
 *         (N % n_blocks == 0), block b quantized with pw[b] (e.g. one block per LSTM gate);
 *         csW [N] int32 row code sums of W.
 *   bias  [N] fp32, nullable.
 *   Y     [M x N] fp32 out (ldy >= N): Y[m,n] = S / (Qa Qw) + bias[n], with the exact integer
 *         S = sum_k (A[m,k] + za)(W[n,k] + zw) = acc + zw*rsA[m] + za*csW[n] + K*za*zw and
 *         the fp32 operations (float)S, Qa*Qw, divide, add, each rounded once.
 *   acc_out [M x N] int32 out, nullable: acc[m,n] = sum_k A[m,k] W[n,k] (the 32-bit accumulator).
 * 1 <= K <= QNN_K_MAX. Large products take scratch for centered copies of both operands, 2 (M + N)
 * (K rounded up to 64) bytes, from a pool of the library's on `stream`, so that calls on different streams
 * never share it. The pool keeps the largest request so far, or 1 GiB, for later calls.
 */
qnn_status qnn_qmatmul(const uint8_t *A, int64_t lda, const qnn_qparams *pa, int ga, const int32_t *rsA,
                       int64_t M, int64_t K, const uint8_t *W, int64_t ldw, const qnn_qparams *pw,
                       int64_t n_blocks, const int32_t *csW, int64_t N, const float *bias, float *Y,
                       int64_t ldy, int32_t *acc_out, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Quantized LSTM / LSTMP stack (Sec. 4 model family) with an optional softmax output layer.
 * ------------------------------------------------------------------------------------------- */

typedef struct {
    int32_t num_layers;  /* L >= 1 */
    int32_t input_dim;   /* I, features per frame */
    int32_t hidden;      /* H, LSTM cells per layer */
    int32_t proj;        /* P, recurrent projection units after each layer; 0 = none */
    int32_t num_classes; /* C, softmax outputs; 0 = no output layer */
    int32_t output_mode; /* qnn_output_mode; must be QNN_OUT_NONE iff num_classes == 0 */
    int32_t stack;        /* Sec. 4 frontend: frames stacked into one network input (the frame and
                             stack - 1 frames of right context; the paper uses 8); 0 or 1 = none.
                             The first layer then takes I * stack features. */
    int32_t stack_stride; /* only every stack_stride-th stacked frame is presented (the paper: 3);
                             0 or 1 = every frame */
    int32_t weight_blocks; /* Sec. 3.1 granularity: every weight matrix (each gate's Wx and Wh, Wp,
                              Wo) is quantized as this many equal blocks of rows (sub-matrices), each
                              its own unit; 0 or 1 = one unit per matrix, the paper's setting. H, P
                              and (quantized output layer) C must be multiples of it. */
} qnn_lstm_desc;

typedef struct qnn_lstm_model qnn_lstm_model;

/* Number of fp32 values in the packed parameter buffer. Layout, layer by layer, with
 * Ik = I * max(stack, 1) for the first layer and R = (P > 0 ? P : H) otherwise, gates in the order
 * [i, f, g, o]:
 *   Wx[4][H][Ik], Wh[4][H][R], b[4][H], then Wp[P][H] if P > 0;
 * after the last layer, if C > 0: Wo[C][R], bo[C]. Returns -1 on an invalid descriptor. */
int64_t qnn_lstm_param_count(const qnn_lstm_desc *d);

/* Quantizes the weights offline (Sec. 3.1: one unit per gate matrix, per projection and per
 * output matrix, or weight_blocks units per matrix) and keeps device copies in the model. `params` (host or device) is read during
 * the call only. The call is synchronous. *out receives the model (destroy with
 * qnn_lstm_model_destroy). */
qnn_status qnn_lstm_model_create(const qnn_lstm_desc *d, const float *params, qnn_lstm_model **out);

void qnn_lstm_model_destroy(qnn_lstm_model *m);

/* Copies the model's weight codes (host buffer, qnn_lstm_param_count bytes; the packed layout
 * with every bias slot zero) and the parameters of each unit in order (4 Wx, 4 Wh, Wp per layer,
 * then Wo, each matrix's blocks in row order; host buffer of at least S (9 L + 1) entries,
 * S = max(weight_blocks, 1)) and their count. Synchronous. */
qnn_status qnn_lstm_model_weights(const qnn_lstm_model *m, uint8_t *codes_host, qnn_qparams *params_host,
                                  int64_t *n_units);

/*
 * qnn_lstm_forward — inference over B independent sequences of T frames.
 *   x        [B][T][I] fp32 frames. With frame stacking (desc.stack, desc.stack_stride) the
 *            network runs on T' = ceil(T / stride) stacked inputs, formed as qnn_stack_frames does
 *            within this call (frames past the end of x repeat its last frame); every output
 *            below then has T' frames instead of T.
 *   y        [B][T][C] softmax outputs if the model has an output layer, else [B][T][R] top-layer
 *            outputs.
 *   h_state  [L][B][R], c_state [L][B][H], nullable: initial state in, final state out (a
 *            stream can therefore be processed in chunks); NULL means a zero initial state and
 *            the final state is not returned.
 *   h_all    [L][B][T][R], nullable: every layer's output at every frame (diagnostics).
 * x, y, h_state, c_state and h_all may each be host or device memory: host buffers are copied
 * to or from device memory on `stream` inside the call (pinned host memory keeps the copies
 * asynchronous). Posteriors (num_classes > 0) for a y in pinned host memory are written there
 * by the softmax kernel itself, or, when the output layer runs beside the recurrence (below),
 * staged chunk by chunk in two device buffers of the workspace and copied by the copy engines.
 * With any host buffer the results are complete once `stream` has been synchronized.
 * Activations are quantized per row (one frame of one sequence), weights per gate matrix.
 * Large batches of a multi-layer model run their layers as a wavefront: the call may place its
 * work on streams and events the model owns (one stream per layer, one for the output layer and
 * one for its copies to the host), which start after everything queued on `stream` before the
 * call, and `stream` waits for all of them before anything queued after it, so the call stays
 * ordered on `stream` as a single launch would be. The model keeps a device workspace sized for
 * the largest B*T seen; calls on one model must not overlap in time.
 */
qnn_status qnn_lstm_forward(qnn_lstm_model *m, const float *x, int64_t B, int64_t T, float *y, float *h_state,
                            float *c_state, float *h_all, void *stream);

/*
 * qnn_lstm_forward_logits — qnn_lstm_forward that also returns the output layer's values before
 * the softmax (Sec. 5: "quant-all" takes the softmax layer's product in 8 bits, "quant" in float).
 *   logits   [B][T][C] fp32, host or device memory, caller-owned, nullable (NULL: the call is
 *            qnn_lstm_forward). logits[b][t][c] is exactly the value the softmax receives: with
 *            QNN_OUT_QUANT the recovered product of the top layer's quantized outputs with the
 *            output weights, eq. (1) and eq. (3), plus the output bias (Fig. 1); with QNN_OUT_FLOAT
 *            the fp32 product plus the bias. With frame stacking T is the stacked length T'.
 * Other arguments and behaviour as for qnn_lstm_forward. QNN_ERR_INVALID_ARG if logits is given
 * for a model without an output layer (num_classes == 0). The copy is made on `stream` after the
 * output product; a host buffer is complete once the stream has been synchronized.
 */
qnn_status qnn_lstm_forward_logits(qnn_lstm_model *m, const float *x, int64_t B, int64_t T, float *y, float *logits,
                                   float *h_state, float *c_state, float *h_all, void *stream);

/*
 * Streaming server mode — frame-at-a-time inference with a resident kernel (the embedded,
 * frame-by-frame setting of Sec. 1 and Sec. 3.1, where inputs are quantized on the fly as they
 * arrive). One launch of the batch-of-few dataflow kernel stays resident for `chunk` frames and
 * takes each frame as soon as the host has written it into host-mapped memory; the output blocks
 * finish the softmax in the kernel and write each frame's posteriors straight to host-mapped
 * memory, flagging the frame when it is complete. The next chunk's launch is queued when its
 * first frame is pushed, with the state (h, c) carried from the previous launch on the device,
 * so the results equal qnn_lstm_forward on the whole sequence (the recurrence bit for bit; the
 * posteriors to within the rounding of the softmax's sum order).
 *
 * qnn_lstm_stream_open — B sequences (1 <= B <= 4) of model m (no projection, H <= 512, R and I
 *   <= 512, output layer absent or quantized; the model's frame stacking is not applied: push
 *   network input rows of m's input width). chunk: frames per launch (1 .. 65536). idle_seconds
 *   (0.001 .. 3600): every wait of the kernel gives up after this long, so a stream left without
 *   input for longer ends with QNN_ERR_TIMEOUT (reopen it to continue). Allocates pinned
 *   host-mapped buffers of 2 chunk B (8 I + 4 out) bytes and device buffers on the current
 *   device, and creates its own CUDA stream. Errors: QNN_ERR_INVALID_ARG (a size or the model out
 *   of range), QNN_ERR_NO_COOP (the kernel's clusters cannot all be resident), QNN_ERR_CUDA.
 *   The model must outlive the session.
 * qnn_lstm_stream_push — appends n frames of every sequence: x is host memory [B][n][I]
 *   (sequence-major, as for qnn_lstm_forward), read during the call only. At most `chunk` frames
 *   may be pushed ahead of those pulled (QNN_ERR_INVALID_ARG otherwise, nothing pushed). Returns
 *   without waiting for the GPU.
 * qnn_lstm_stream_pull — waits (at most timeout_seconds) for the next n frames and copies them
 *   into y, host memory [B][n][C] posteriors (or [B][n][R] top-layer outputs without an output
 *   layer). n must not exceed the frames pushed and not yet pulled (QNN_ERR_INVALID_ARG).
 *   QNN_ERR_TIMEOUT if the frames are not ready in time or the kernel gave up (see idle_seconds);
 *   the session is then unusable except for qnn_lstm_stream_close.
 * qnn_lstm_stream_close — completes the current launch with zero frames (their outputs are
 *   dropped), waits for it, frees the session and returns the first error the kernel recorded
 *   (QNN_ERR_NONFINITE for a non-finite input, QNN_ERR_TIMEOUT) or QNN_OK.
 * A session's calls must not overlap in time (one host thread at a time).
 */
typedef struct qnn_lstm_stream qnn_lstm_stream;
qnn_status qnn_lstm_stream_open(qnn_lstm_model *m, int64_t B, int64_t chunk, double idle_seconds,
                                qnn_lstm_stream **out);
qnn_status qnn_lstm_stream_push(qnn_lstm_stream *s, const float *x, int64_t n);
qnn_status qnn_lstm_stream_pull(qnn_lstm_stream *s, float *y, int64_t n, double timeout_seconds);
qnn_status qnn_lstm_stream_close(qnn_lstm_stream *s);

/*
 * qnn_stack_frames — the frontend of Sec. 4: features of n consecutive frames are stacked (the frame
 * and n - 1 frames of right context) and only every stride-th stacked frame is kept.
 *   x   [B][T][I] fp32, device memory, caller-owned.
 *   out [B][T'][n I] fp32, T' = ceil(T / stride), device memory, caller-owned: out[b][t'] is frames
 *       stride t' .. stride t' + n - 1 of sequence b, concatenated; a frame past the end of the
 *       sequence is replaced by its last frame (the paper does not say).
 * QNN_ERR_INVALID_ARG for B < 0, T < 1, I < 1, n < 1, stride < 1 or non-device pointers (B > 0).
 * Asynchronous on `stream`.
 */
qnn_status qnn_stack_frames(const float *x, int64_t B, int64_t T, int64_t I, int32_t n, int32_t stride, float *out,
                            void *stream);

/*
 * qnn_quantize_matrix_static — qnn_quantize with QNN_PER_MATRIX, allocating nothing.
 * The paper has no counterpart: this is an interface for callers that cannot allocate device
 * memory inside a library call (a fixed pre-reserved memory budget, device memory owned by the
 * caller's own allocator or pool, or a latency-critical stream where the device-wide
 * synchronization of cudaMalloc/cudaFree is not acceptable). Same results as qnn_quantize with
 * QNN_PER_MATRIX (codes, params[0], code_sums) for finite inputs.
 *   x, codes, params, code_sums: as for qnn_quantize (device memory, caller-owned); params has
 *     one entry.
 *   status   device int, nullable, caller-owned: QNN_ERR_NONFINITE is written into it (if it is
 *     still 0) when the matrix holds NaN or +-Inf; the codes are then unspecified.
 *   A pointer that is not device memory of the current device (x, codes, params, and code_sums or
 *   status when given) returns QNN_ERR_INVALID_ARG before anything runs.
 * Limits: rows <= 524288 (its scratch holds one partial range per 32 rows); larger inputs return
 * QNN_ERR_INVALID_ARG before anything runs.
 * Scratch: a 128 KiB + 256 B static device array inside the library, held on every GPU that loads
 * the library until the process exits and shared by all calls. Calls that overlap in time on the
 * GPU (unordered streams) race on it; ordered calls are safe (each call clears the completion
 * counter on its stream before its kernels run). The first call on each device resolves the
 * array's device address (cudaGetSymbolAddress) with that device current; make that first call
 * before any stream capture. Calls no cudaMalloc or cudaFree.
 */
qnn_status qnn_quantize_matrix_static(const float *x, int64_t rows, int64_t cols, int64_t ldx, uint8_t *codes,
                                      int64_t ldc, qnn_qparams *params, int32_t *code_sums, int *status,
                                      void *stream);

/* ---------------------------------------------------------------------------------------------
 * Selective state-space layers on 8-bit activations. The paper's layers are fully connected and LSTM ones; these calls
 * apply its quantization scheme (activations on the fly, one unit per row; weights offline, in units of sub-matrices) to a
 * layer whose state update is element-wise:
 *   qnn_rmsnorm_quantize -> qnn_qmatmul4 (or qnn_qmatmul) -> qnn_causal_conv -> qnn_ssm_scan -> qnn_quantize -> a product.
 * For these calls device pointers have to belong to the current device (or be managed memory), and an output may not
 * overlap an input unless a call allows it; QNN_ERR_INVALID_ARG otherwise, before anything runs. Overlap goes by the
 * range from an argument's first byte to its last. Rows (sequences, frames) times their stride may not pass 2^48 elements.
 * The calls take no scratch, so any number may run at once, and may be captured into a graph after a first call on the device
 * (which allocates the device status word).
 * ------------------------------------------------------------------------------------------- */

/* Types of the values that pass between layers. All arithmetic is fp32 or wider, each output rounded once. */
typedef enum { QNN_F32 = 0, QNN_BF16 = 1, QNN_F16 = 2 } qnn_dtype;

/*
 * qnn_rmsnorm_quantize — residual addition, root-mean-square norm and the on-the-fly quantizer (Sec. 3, eq. 2) in one pass.
 *   x, residual   [rows x cols] of `dtype` (leading dimensions ldx, ldr >= cols); residual nullable.
 *   residual_out  [rows x cols] of `dtype` (ldh >= cols), nullable: h = x + residual (fp32), rounded once. It may be x or
 *                 residual itself (same pointer and leading dimension).
 *   weight        [cols] fp32. eps: 1e-20 .. 1e20.
 *   codes, params, code_sums  as qnn_quantize with QNN_PER_ROW gives them for the fp32 rows
 *                 v = (h s) weight, s = 1 / sqrt(sum h^2 / cols + eps); code_sums nullable.
 *   values        [rows x cols] fp32 (ldv >= cols), nullable: the values that the codes stand for, (code + z) / Q (eq. 3),
 *                 for consumers in float (the "quant" output layer of Sec. 5).
 * The codes are defined to the bit: the norm is taken of h before it is rounded to `dtype`; s is computed to about 2^-44
 * relative and rounded once to fp32; h s and its product with the weight are each rounded once to fp32.
 * 1 <= cols <= 2^24, and 8421504 with code_sums, which a row of more could take past 2^31 - 1. A row with a value of v that is
 * not finite: its codes and values are unspecified and QNN_ERR_NONFINITE is recorded, as for qnn_quantize (h is stored all the
 * same).
 */
qnn_status qnn_rmsnorm_quantize(const void *x, int64_t ldx, const void *residual, int64_t ldr, int dtype,
                                const float *weight, double eps, int64_t rows, int64_t cols, void *residual_out,
                                int64_t ldh, uint8_t *codes, int64_t ldc, qnn_qparams *params, int32_t *code_sums,
                                float *values, int64_t ldv, void *stream);

/*
 * qnn_quantize4 — weights to 4-bit codes, offline: eq. (2) with S = 15 on sub-matrices (Sec. 3.1) of `group` (32, 64 or
 * 128) consecutive weights of a row, the last of a row perhaps shorter.
 *   w          [N x K] fp32, leading dimension ldw >= K.
 *   Per unit, the range taken to include 0: scale = (max / 15 - min / 15) rounded up to bf16, offset = round(min / scale)
 *   (-15 .. 0), code = clamp(round(w / scale) - offset, 0, 15); a code stands for (code + offset) scale, at most half a
 *   scale from w. A unit of zeros has scale 0. The least scale is 2^-126.
 *   codes      [ceil(N/16)][ceil(K/128)][1024] bytes: tiles of 16 rows x 128 columns. Row 8 h + g and column
 *              32 j + 8 t + e of a tile are in the four bytes from 512 h + 64 g + 16 t + 4 j on, whose eight halves,
 *              low ones first, hold e = 0 2 4 6 1 3 5 7. Rows and columns past the matrix have code 0.
 *   units      [ceil(N/16)][ceil(K/128)][16][128 / group] entries: bf16 offset in the low half, bf16 scale in the high
 *              half; 0 past the matrix.
 *   row_sums   [N] fp32: the sum of the values that the row's codes stand for.
 * The three are 16-byte aligned. 1 <= N, 1 <= K <= QNN_K_MAX (QNN_ERR_K_TOO_LARGE). A unit with a value that is not finite:
 * unspecified codes, QNN_ERR_NONFINITE is recorded.
 */
qnn_status qnn_quantize4(const float *w, int64_t N, int64_t K, int64_t ldw, int32_t group, uint8_t *codes, uint32_t *units,
                         float *row_sums, void *stream);

/*
 * qnn_qmatmul4 — the recovered product of Fig. 1 with 4-bit weights of qnn_quantize4, for few rows (each 32 of them read
 * the weights once).
 *   A, lda, pa, ga  [M x K] uint8 activation codes and their units, as for qnn_qmatmul; M <= 524280.
 *   codes, units, group, row_sums  of a matrix [N x K].
 *   bias [N] fp32, nullable; Y [M x N] fp32 out (ldy >= N):
 *     Y[m,n] = (1 / Qa) sum_groups scale sum_{k in group} (A[m,k] + za)(code[n,k] + offset) + bias[n].
 *   The sums of a group's codes are exact; the groups' terms are added in fp32, in an order that depends on the sizes and the
 *   device only. Codes past K are not read as products whatever A holds there.
 */
qnn_status qnn_qmatmul4(const uint8_t *A, int64_t lda, const qnn_qparams *pa, int ga, int64_t M, int64_t K,
                        const uint8_t *codes, const uint32_t *units, int32_t group, const float *row_sums, int64_t N,
                        const float *bias, float *Y, int64_t ldy, void *stream);

/*
 * qnn_causal_conv — short causal convolution of each channel over time, optionally through SiLU:
 *   y[b][t][d] = f(bias[d] + sum_{j < W} w[d][j] x[b][t - W + 1 + j][d]),  f(v) = v / (1 + exp(-v)) or v.
 *   x, y   [B][T][D] of `dtype`: frame t of sequence b at b * seq + t * frame elements (strides in elements, channels
 *          contiguous). Outputs of different frames must not overlap.
 *   w [D][W] fp32 (1 <= W <= 8), bias [D] fp32, nullable.
 *   state_in, state_out  [B][W - 1][D] of `dtype`, nullable: the W - 1 inputs before the first frame, oldest first (NULL:
 *          zeros), and the last W - 1 inputs after the last one. They may be the same buffer, for streaming.
 *   lengths [B] int32, nullable: frames of each sequence (values outside 0 .. T count as the nearer of them). Frames behind a
 *          sequence's end are not read for it and their outputs are left as they are.
 * One frame of many sequences (T = 1 with states) is the serving form; T = 0 only carries the states over. T <= 2^30.
 */
qnn_status qnn_causal_conv(const void *x, int64_t x_seq, int64_t x_frame, int dtype, int64_t B, int64_t T, int64_t D,
                           const float *w, int32_t W, const float *bias, int silu, const void *state_in, void *state_out,
                           const int32_t *lengths, void *y, int64_t y_seq, int64_t y_frame, void *stream);

/* Arguments of qnn_ssm_scan. Strides in elements: frame t of sequence b at b * seq + t * frame, its channels contiguous. */
typedef struct {
    int64_t B, T, D;  /* sequences, frames, channels */
    int32_t N;        /* states of a channel, 1 .. 128 */
    int32_t groups;   /* groups of D / groups channels that share Bm and Cm; divides D */
    int32_t dtype;    /* of u, dt, Bm, Cm, z and y */
    int32_t softplus; /* 1: the step is log(1 + exp(dt + dt_bias)); 0: dt + dt_bias */
    const void *u;    /* [B][T][D] inputs */
    int64_t u_seq, u_frame;
    const void *dt;   /* [B][T][D] steps, before dt_bias and softplus */
    int64_t dt_seq, dt_frame;
    const void *Bm;   /* [B][T][groups * N] */
    int64_t Bm_seq, Bm_frame;
    const void *Cm;   /* [B][T][groups * N] */
    int64_t Cm_seq, Cm_frame;
    const void *z;    /* [B][T][D] gates, nullable */
    int64_t z_seq, z_frame;
    void *y;          /* [B][T][D] out */
    int64_t y_seq, y_frame;
    const float *A;       /* [D][N] */
    const float *skip;    /* [D], nullable */
    const float *dt_bias; /* [D], nullable */
    const float *state_in; /* [B][D][N], nullable: zeros */
    float *state_out;      /* [B][D][N], nullable; may be state_in */
    const int32_t *lengths; /* [B], nullable */
} qnn_ssm_args;

/*
 * qnn_ssm_scan — selective scan over time, every channel d of every sequence b with N states h of its own:
 *   s = softplus(dt[t][d] + dt_bias[d]);  h[n] = exp(s A[d][n]) h[n] + s u[t][d] Bm[t][g][n];
 *   y[t][d] = (sum_n Cm[t][g][n] h[n] + skip[d] u[t][d]) * z / (1 + exp(-z)),  z = z[t][d],
 * with the last factor only where z is given and g = d / (D / groups). States and sums are fp32. lengths, frames behind a
 * sequence's end and T = 0 as for qnn_causal_conv; state_out is the state after each sequence's last frame, and
 * the states of a sequence do not depend on the others. One frame of many sequences is the serving form.
 * Long sequences are taken in parts whose states are put together by their factors over a part, unless that is not finite: it
 * may overflow where states grow (A s > 0) although no state does, and the frames before a part are then gone over one by one.
 * An A whose product with log2(e) is infinite counts as the last with a finite one, so that a step of 0 leaves its state as it is.
 * Other non-finite inputs give non-finite outputs (infinities or NaN), in their own channel and sequence (group, for Bm and Cm).
 */
qnn_status qnn_ssm_scan(const qnn_ssm_args *args, void *stream);

/* Arguments of qnn_linear_attention. Strides in elements: frame t of sequence b at b * seq + t * frame, its heads and their
 * values contiguous. q, k and v have any number of heads that divides H: head h of the H uses head h / (H / heads) of each. */
typedef struct {
    int64_t B, T;     /* sequences, frames */
    int32_t H;        /* heads of the output and the states */
    int32_t q_heads, k_heads, v_heads;
    int32_t dk, dv;   /* 1 .. 256 */
    int32_t dtype;    /* of q, k, v and y */
    float scale;
    const void *q;    /* [B][T][q_heads][dk] */
    int64_t q_seq, q_frame;
    const void *k;    /* [B][T][k_heads][dk] */
    int64_t k_seq, k_frame;
    const void *v;    /* [B][T][v_heads][dv] */
    int64_t v_seq, v_frame;
    void *y;          /* [B][T][H][dv] out */
    int64_t y_seq, y_frame;
    const float *log_decay; /* [H] */
    const float *state_in;  /* [B][H][dk][dv], nullable: zeros */
    float *state_out;       /* [B][H][dk][dv], nullable; may be state_in */
    const int32_t *lengths; /* [B], nullable */
} qnn_linear_args;

/*
 * qnn_linear_attention — linear attention with a decay for each head, every head h of every sequence with a state S of its own:
 *   S = exp(min(log_decay[h], 0)) S + k_t v_t^T;  y_t = scale q_t S.
 * States and sums are fp32. Where T is more than 8, scores (q_t k_s times the decay between them) and states enter their products
 * rounded to 2^-16 of each with bf16 and fp16 inputs, and such terms to 2^-20 with fp32 ones: where an output's terms cancel, it is that
 * far off beside them, not beside itself. The states that are carried are not rounded so. A score q_t k_s is formed ahead of its
 * product with v_s and has to lie in fp32's range, as k_s v_s does. Whole sequences are taken by chunks of frames (and long ones of few
 * sequences in parts whose states are put together by their decays), a few frames one by one: a prompt and the frames after it may be
 * given in any division, and one frame of many sequences is the serving form. lengths, frames behind a sequence's end and T = 0 as for
 * qnn_causal_conv; state_out is the state after each sequence's last frame. A decay above 1 counts as 1, one below exp(-200) as 0.
 * Inputs that are not finite give outputs that are not (infinities or NaN) from their frame on, in the heads that use them: v in
 * its own column, k in all of them; q in its own frame only.
 */
qnn_status qnn_linear_attention(const qnn_linear_args *args, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Label-synchronous decoding: selection over beams and classes, the kept beams' states, labels' rows.
 * As for the calls above, device pointers belong to the current device and outputs overlap nothing unless a call allows it; any
 * number of calls may run at once, and be captured into a graph, a first call on the device too. The same holds for
 * qnn_linear_attention.
 * ------------------------------------------------------------------------------------------- */

/*
 * qnn_beam_select — the n best continuations of each of B utterances' K beams over V classes.
 *   logits   [B * K x V] of `dtype` (ldl >= V), row b * K + k of utterance b's beam k.
 *   scores   [B][K] fp32: log probabilities of the beams. finished [B][K], nullable: non-zero for beams that have ended.
 *   A candidate (k, v) has the score scores[k] + logits[k][v] - log(sum_v exp(logits[k][v])); a finished beam has one candidate
 *   (k, eos) of its own score, its logits are not read. A candidate whose score is minus infinity or not a number is none (a
 *   class masked by minus infinity, a beam of score minus infinity); a beam with a NaN or plus infinity among its logits, or with
 *   minus infinity alone, has none.
 *   scores_out, parents, tokens  [B][n] out, best first: score, beam and class. Of equal scores the lowest beam, then the lowest
 *   class comes first; a slot without a candidate has score minus infinity, beam 0 and class eos. scores_out may be
 *   scores if n = K.
 * Scores are formed and compared as two fp32 terms (48 bits) and rounded once for scores_out. The sums of exponentials are of fp32
 * terms: a row's log(sum exp) is off by (10 + 2 D) 2^-24 at most, where D is the mean distance of a class's logit from the row's
 * largest, by the classes' probabilities (at most their entropy, log V). 2.1 2^-24 is the most that was seen of rows of 97 to 262144
 * classes, 2^-29 where thousands of random logits count. Each row of a call is summed in the same order, so that equal rows have equal
 * sums. Candidates of different beams whose scores are closer than two rows' errors may come in either order. Within a beam the n
 * best are those of the logits, in their order as far as the scores differ.
 * 1 <= K, n <= 128; K V < 2^31; 0 <= eos < V.
 */
qnn_status qnn_beam_select(const void *logits, int64_t ldl, int dtype, const float *scores, const uint8_t *finished, int64_t B,
                           int64_t K, int64_t V, int32_t n, int32_t eos, float *scores_out, int32_t *parents, int32_t *tokens,
                           void *stream);

/* A carried state: in [outer][B * K] rows of row_bytes, out [outer][B * n]. out may be in if n = K; otherwise outputs overlap
 * nothing. */
typedef struct {
    const void *in;
    void *out;
    int64_t outer, row_bytes;
} qnn_beam_state;

/*
 * qnn_beam_reorder — states of the beams that were kept: row b * n + j of out is row b * K + parents[b][j] of in, for each of
 * `count` states (a host array, read before the call returns) of any types. parents [B][n] int32, as qnn_beam_select gives them. A
 * row whose parent is outside 0 .. K - 1 is left as it is and QNN_ERR_INVALID_ARG is recorded. 1 <= K, n <= 128.
 */
qnn_status qnn_beam_reorder(const qnn_beam_state *states, int32_t count, const int32_t *parents, int64_t B, int64_t K, int64_t n,
                            void *stream);

/*
 * qnn_embedding — rows of a table by label: out[i] = scale table[ids[i]] in fp32, rounded to out_dtype.
 *   ids [n] int32 or int64 (id_bytes 4 or 8); table [V x D] of `dtype` (ldt >= D); out [n x D] (ldo >= D).
 *   A label below 0 is padding: a row of zeros. One of V or more is that too, and QNN_ERR_INVALID_ARG is recorded.
 */
qnn_status qnn_embedding(const void *ids, int id_bytes, int64_t n, const void *table, int64_t ldt, int dtype, int64_t V, int64_t D,
                         float scale, void *out, int64_t ldo, int out_dtype, void *stream);

/*
 * qnn_embedding_grad — its gradient: out[r] = scale sum of grad[i] over the i with ids[i] = r (plus out[r] where `add` is not 0), in
 * fp32, rounded once to out_dtype.
 *   grad [n x D] of `dtype` (ldg >= D), out [V x D] (ldo >= D). Labels outside 0 .. V - 1 have no part in it.
 *   The sums are taken in an order that depends on the sizes and labels only (positions sorted by label), so that the same inputs
 *   give the same bits. Takes scratch of about 16 n + n D / 4 bytes. n <= 2^30.
 */
qnn_status qnn_embedding_grad(const void *grad, int64_t ldg, int dtype, const void *ids, int id_bytes, int64_t n, int64_t V,
                              int64_t D, float scale, int add, void *out, int64_t ldo, int out_dtype, void *stream);

/* ---------------------------------------------------------------------------------------------
 * Kernel timing (diagnostics and benchmarks; no counterpart in the paper).
 * ------------------------------------------------------------------------------------------- */

/* While enabled, every kernel launch the library makes is bracketed by two CUDA events on the
 * launching stream (process-wide switch, off by default). */
qnn_status qnn_profile_enable(int on);

/* Waits for the recorded events, then returns per kernel name (static strings) the number of
 * launches and their summed device time in milliseconds since the last read, and resets the
 * totals. Up to `capacity` entries are written to the (nullable) host arrays; *count receives
 * the number of distinct kernels. */
qnn_status qnn_profile_read(int capacity, const char **names, double *total_ms, int64_t *launches, int *count);

/* Measures the peak rate of an integer datapath on the current device, in tera-operations per
 * second (a multiply-add counts as two operations): kind 0 = the warp-level integer tensor-core
 * MMA (mma.sync m16n8k32 u8 x u8 -> s32) the products use, kind 1 = dp4a on the CUDA cores.
 * Register-only loops on every SM; synchronous; the best of three timed runs. */
qnn_status qnn_measure_peak(int kind, double *tops);

/* Measures the latency floor of the batch-of-few recurrence (no counterpart in the paper): the
 * time per round, in microseconds, of that kernel's per-frame synchronisation skeleton with all
 * arithmetic removed, on one cluster of cluster_size (1 .. 16) blocks: product warps wait for the
 * cluster-wide exchange of the previous frame's outputs (distributed shared memory stores completing
 * on a transaction-count barrier) and hand over to the epilogue warps, which send their values to
 * every block of the cluster. A layer of that kernel cannot take less per frame. rounds: 1 ..
 * 10^6 rounds per launch; synchronous; best of three launches; QNN_ERR_NO_COOP if the cluster
 * cannot be launched, QNN_ERR_TIMEOUT if a (bounded) wait gave up. */
qnn_status qnn_measure_exchange_floor(int32_t cluster_size, int32_t rounds, double *us_per_round);

/* Diagnostic (no counterpart in the paper): out[i] = in[i] rounded to the nearest fp32 value, ties
 * to even, by the conversion the recovery of eq. (3) uses on the device for the exact int64 sums
 * S of eq. (1). in [n] int64 and out [n] float are device buffers owned by the caller; errors:
 * QNN_ERR_INVALID_ARG for n < 0 or null/host pointers with n > 0. Asynchronous on `stream`. */
qnn_status qnn_selftest_s64_to_f32(const int64_t *in, float *out, int64_t n, void *stream);

/* Diagnostic (no counterpart in the paper): the recurrent kernels evaluate sigma, tanh and the cell
 * update (on one cell or two at once) and the recovery's quotient through a reciprocal of their own
 * and, for moderate arguments, without clamps; this runs those forms and the same operations with
 * IEEE divides on the pairs (in[2i], in[2i+1]) and writes into *mismatches (device, caller-owned) the
 * number of pairs where any result differs in any bit (0 is required for bit-exact parity). in
 * [2 npairs] fp32, device memory. Errors: QNN_ERR_INVALID_ARG for npairs < 0 or null/host pointers.
 * Asynchronous on `stream`. */
qnn_status qnn_selftest_pair_functions(const float *in, int64_t npairs, unsigned long long *mismatches, void *stream);

/* Diagnostic (no counterpart in the paper): runs one warp that waits, through the bounded wait of
 * the tensor-core kernels, on a barrier nothing completes, for limit_ns (1 us .. 1 s). The wait
 * gives up and records QNN_ERR_TIMEOUT in the device status word (read it with qnn_device_status);
 * the context stays usable. Synchronous on `stream`. Returns QNN_OK when the wait gave up as
 * designed, QNN_ERR_INVALID_ARG for a limit out of range. */
qnn_status qnn_selftest_wait_timeout(int64_t limit_ns, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* QNN_H */
