/* agq - the W4A8 / W4A4 quantized linear layer of Agile-Quant (arxiv 2312.05693)
 * and its log2-quantized softmax x V path, with the paged 8-bit key/value cache
 * (its pages shared and compacted too), the attentions that serving needs and the
 * log probabilities of its answers, as HIP kernels for gfx950 (MI355X).
 *
 * C ABI.  Conventions that hold for every call unless a comment says otherwise:
 *   - every tensor pointer is a DEVICE pointer owned by the caller; the library
 *     allocates nothing and keeps no tensor state between calls.  What it does
 *     keep, per process and device, are facts looked up once: the device's number
 *     of compute units, a raised LDS limit of its own kernels, and the address of
 *     agq_gemm_w4a8_static's array.  Each is set up, thread-safely, by the first
 *     call that needs it on that device;
 *   - tensors are row-major, leading dimensions are in elements;
 *   - work is enqueued asynchronously on `stream` (a hipStream_t passed as
 *     void*, NULL = the default stream); the caller synchronises;
 *   - the return value is an agq_status: 0 on success, negative on error.
 *     Argument errors (AGQ_EINVAL, AGQ_ESIZE) are found on the host before any
 *     HIP call is made; AGQ_EHIP reports a failed launch.  Nothing is printed,
 *     thrown or aborted;
 *   - fp16 inputs must not hold NaN (a NaN yields an unspecified code inside
 *     the grid); +-Inf saturate.
 */
#ifndef AGQ_H
#define AGQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum agq_status {
    AGQ_OK = 0,
    AGQ_EINVAL = -1, /* bad argument (null pointer, size, granularity, range) */
    AGQ_ESIZE = -2,  /* workspace too small                                    */
    AGQ_EHIP = -3,   /* the HIP runtime refused a launch                       */
    AGQ_ETIMEOUT = -4 /* agq_gemm_chain_status: a wait inside a chain launch ran
                         out of time (see there)                                */
};

/* what `x` of the GEMM calls holds */
enum agq_x_kind {
    AGQ_X_F16 = 0, /* fp16 [M,K]; Eq.2 is applied inside the call            */
    AGQ_X_Q = 1,   /* codes written by agq_quantize_act with the same
                      bits / e / zp: int8 [M,K] (8 bit) or nibbles [M,K/2]   */
    AGQ_X_F16_DOT = 2 /* as AGQ_X_F16, for M == 1 and zp == 0 only: the product runs
                      on the vector ALU (v_dot4_i32_i8 / v_dot8_i32_i4, the
                      chip's counterpart of the paper's 4-bit multiplier,
                      Section 4.4 and the appendix) with Eq.2 applied in
                      registers, no LDS staging and no matrix core.  Same
                      results bit for bit; which form is faster is a
                      measurement (the library itself never picks this one).
                      Not accepted by the _trip and chain calls.             */
};

/* range of the activation exponent e (scale s = 2^e) accepted everywhere */
#define AGQ_E_MIN (-40)
#define AGQ_E_MAX 40

const char *agq_status_string(int status);
int agq_version(void);

/* Layer-wise power-of-two activation scale (Section 4.4: all channels share one
 * set of quantization parameters; the scale is read as a power of two).
 * Writes to *e_dev (device int32) the smallest e with max|x| <= qmax * 2^e,
 * qmax = 2^(bits-1)-1; 0 for an all-zero tensor; +-Inf/NaN count as 2^16.
 * x_f16: fp16 [M,K], ldx >= K.  bits in {4,8}.  M*K may be 0 (e = 0).        */
int agq_calibrate_act_exp(const void *x_f16, int64_t M, int64_t K, int64_t ldx,
                          int bits, int32_t *e_dev, void *stream);

/* Uniform quantizer, Section 4.1 Eq.2, with s = 2^e and round-half-to-even:
 *   q = CLIP(round(x / 2^e) + zp, lo, hi)
 * zp == 0 selects the signed grid of Eq.1, [-2^(b-1), 2^(b-1)-1]; zp > 0 the
 * unsigned grid [0, 2^b-1] of Eq.2 as printed.  bits in {4,8}.
 * x_f16 : fp16 [M,K], ldx >= K, ldx % 8 == 0, 16-byte aligned; K % 8 == 0.
 * xq_out: bits=8: one byte per code, [M,K] contiguous (int8, or uint8 if zp>0);
 *         bits=4: two codes per byte, [M,K/2] contiguous, low nibble = even k,
 *         signed codes in two's complement.
 * M == 0 is a no-op.                                                          */
int agq_quantize_act(const void *x_f16, int64_t M, int64_t K, int64_t ldx,
                     int bits, int e, int zp, void *xq_out, void *stream);

/* 4-bit weight storage (Section 4.4 stores two 4-bit weights per byte).  The
 * order of nibbles inside `packed` is private to the library: it is laid out
 * for 64-lane coalesced loads and the int8 MFMA operand order, followed by the
 * sum of each output channel's weights (used by the unsigned activation grid).
 * Only agq_unpack_w4(agq_pack_w4(W)) == W is contractual.
 * wq     : int8 [N,K], K contiguous, values in [-8,7]; K % 128 == 0, N >= 1.
 *          Values outside [-8,7] are saturated and counted into *bad_count_dev
 *          (device int32, may be NULL; the caller zeroes it and reads it after
 *          synchronising).
 * packed : agq_pack_w4_bytes(N,K) bytes, 16-byte aligned (0 = invalid N,K).   */
size_t agq_pack_w4_bytes(int64_t N, int64_t K);
int agq_pack_w4(const int8_t *wq, int64_t N, int64_t K, void *packed,
                int32_t *bad_count_dev, void *stream);
int agq_unpack_w4(const void *packed, int64_t N, int64_t K, int8_t *wq_out,
                  void *stream);

/* The quantized linear layer (Sections 4.2 and 4.4): the activation on the
 * b-bit grid of Eq.2 with the layer-wise scale 2^e, times the 4-bit weights,
 * accumulated in int32, dequantized per output channel:
 *   acc[m,n] = sum_k (q[m,k] - zp) * Wq[n,k]       (int32, exact)
 *   y[m,n]   = fp16( float(acc[m,n]) * (2^e * sw[n]) )
 * agq_gemm_w4a8 uses b = 8, agq_gemm_w4a4 b = 4 (codes widened to int8 for the
 * MFMA; CDNA4 has no 4-bit matrix instruction).
 * x        : see agq_x_kind.  fp16: ldx % 8 == 0; codes: ldx in code units,
 *            ldx % 16 == 0 (8 bit) or ldx % 32 == 0 (4 bit); 16-byte aligned.
 *            w_packed, w_scale_f16 and y_f16 are 16-byte aligned too.
 * zp       : 0 = the signed grid of Eq.1 (the measured configuration); 1 .. 2^b-1 =
 *            the unsigned grid of Eq.2 with that zero point.  Inside the kernels
 *            the unsigned code travels as q - 2^(b-1), which the int8 matrix
 *            instruction takes, and sum_k (q - zp) w = sum_k (q - 2^(b-1)) w +
 *            (2^(b-1) - zp) * sum_k w, the last sum precomputed by agq_pack_w4.
 * w_packed : output of agq_pack_w4 for [N,K].   w_scale_f16: fp16 [N].
 * y_f16    : fp16 [M,N], ldy >= N.   acc_out: optional int32 [M,N] contiguous
 *            copy of the accumulators (NULL to skip).
 * workspace: agq_gemm_workspace_bytes(M,N,K) bytes, 16-byte aligned, may be
 *            NULL when that is 0.  Holds the quantized activation when M is
 *            large enough for the tiled kernel, and behind it, when the call
 *            has few output tiles and a long K, room for the int32 partial tiles
 *            of a split of K over workgroups (taken when the split is the fastest
 *            way for the call's sizes); contents are scratch.  A workspace of
 *            agq_gemm_workspace_bytes(M,0,K) bytes (the activation only) is
 *            accepted too: K is then not split, which costs time where it
 *            applies and changes no result; a smaller one is AGQ_ESIZE.
 * K % 128 == 0, K <= 65536 (keeps every partial sum inside int32), M >= 0.
 * Which kernel runs is the library's choice and does not change a result: up to 16
 * rows the weight-streaming kernel; 17..256 rows of fp16 input the same kernel with
 * sixteen rows (and two channel tiles) per workgroup while re-reading the weights per row group is cheaper
 * than the tiled path (a measured rule on the sizes); else the layout pre-pass and
 * the tiled kernel: with tiles of 32, 64 or 128 tokens x 64 to 256 channels, K shared
 * by one or two groups of wavefronts, or with K split over workgroups (few tiles, a
 * long K, and the workspace has the room), whichever a measured cost model puts first.
 * Graph capture: the calls enqueue kernels only and may be captured.  (The first
 * weight-streaming call on a device also raises the LDS limit of the library's
 * kernels there: a host-side setting, not a stream operation, made once per
 * device whatever the shape of that first call.)                              */
size_t agq_gemm_workspace_bytes(int64_t M, int64_t N, int64_t K);
int agq_gemm_w4a8(const void *x, int x_kind, int64_t M, int64_t K, int64_t ldx,
                  int e, int zp, const void *w_packed, const void *w_scale_f16,
                  int64_t N, void *y_f16, int64_t ldy, int32_t *acc_out,
                  void *workspace, size_t workspace_bytes, void *stream);
int agq_gemm_w4a4(const void *x, int x_kind, int64_t M, int64_t K, int64_t ldx,
                  int e, int zp, const void *w_packed, const void *w_scale_f16,
                  int64_t N, void *y_f16, int64_t ldy, int32_t *acc_out,
                  void *workspace, size_t workspace_bytes, void *stream);

/* For callers that cannot allocate device memory (code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc): agq_gemm_w4a8 without the
 * workspace arguments.  The quantized activation of the tiled path, and the partial
 * tiles of a K split behind it, live in a fixed array of
 * AGQ_STATIC_WORKSPACE_BYTES inside the library's device image (one copy on every
 * GPU the library is used on, held until the process ends); the call makes no
 * hipMalloc / hipFree and calls no allocating routine.  The array's address is
 * looked up once per device, on the first call made with that device current.
 * Same arguments, checks, kernels and results as agq_gemm_w4a8.  A call whose
 * activation codes alone (M rounded up to 128, times K bytes; nothing for M <= 16)
 * exceed the array returns AGQ_ESIZE before any HIP call; every configuration up
 * to 2048 x 11008 fits.  When the codes fit but the partial tiles do not, K is
 * not split (slower for few output tiles, same result).
 * All calls on one GPU share the array: two calls that overlap in time on one GPU
 * (different streams or threads) race and give wrong results; calls on one stream
 * are safe.  Nothing in the array needs clearing between calls.                */
#define AGQ_STATIC_WORKSPACE_BYTES ((size_t)32 << 20)
int agq_gemm_w4a8_static(const void *x, int x_kind, int64_t M, int64_t K, int64_t ldx,
                         int e, int zp, const void *w_packed, const void *w_scale_f16,
                         int64_t N, void *y_f16, int64_t ldy, int32_t *acc_out,
                         void *stream);

/* Several projections of the same activation in one call (q/k/v, gate/up of a
 * transformer block; Section 4.2's pipeline quantizes such an activation once).
 * Same computation as `count` calls of agq_gemm_w4a8 / agq_gemm_w4a4 with the
 * same x, M, K, e: Eq.2 (or the layout pre-pass) runs once, and all projections
 * run as one kernel launch: what a launch-bound decode step needs, and for many
 * rows one grid over the tiles of all projections fills the chip better.  projs: HOST array of `count` descriptors (1 <= count <=
 * AGQ_MAX_PROJ), read before the call returns.  workspace:
 * agq_gemm_workspace_bytes(M, N, K) with N = the widths of the projections added
 * up (any smaller N down to 0 is accepted, see above).  Other arguments and errors as
 * for the single calls.                                                       */
#define AGQ_MAX_PROJ 4
typedef struct agq_proj {
    const void *w_packed;    /* agq_pack_w4 output for [N,K]            */
    const void *w_scale_f16; /* fp16 [N]                                */
    int64_t N;
    void *y_f16;             /* fp16 [M,N]                              */
    int64_t ldy;
    int32_t *acc_out;        /* optional int32 [M,N] contiguous, or NULL */
} agq_proj;
int agq_gemm_w4a8_multi(const void *x, int x_kind, int64_t M, int64_t K, int64_t ldx,
                        int e, int zp, const agq_proj *projs, int count,
                        void *workspace, size_t workspace_bytes, void *stream);
int agq_gemm_w4a4_multi(const void *x, int x_kind, int64_t M, int64_t K, int64_t ldx,
                        int e, int zp, const agq_proj *projs, int count,
                        void *workspace, size_t workspace_bytes, void *stream);

/* A chain of linear layers for a few tokens in ONE kernel launch: the decode
 * regime, where a step of the model is a sequence of layers that each read
 * 8-45 MB of 4-bit weights once (Section 3.3: the matrix products are the
 * workload; Section 4.4: layer-wise activation parameters, so every stage has its
 * own static exponent).  Stage s computes what agq_gemm_w4a8_multi /
 * agq_gemm_w4a4_multi computes (zp = 0, fp16 input, Eq.2 inside, per-channel
 * dequantization, fp16 outputs written to the caller's tensors), on
 *   - a caller tensor x_f16 [M,K] (ldx % 8 == 0, 16-byte aligned), or
 *   - x_f16 == NULL: the fp16 output of projection `src_proj` of stage s-1, whose
 *     width must equal this stage's K (never allowed for stage 0).
 * Results are those of the single calls, bit for bit.  One persistent workgroup
 * per compute unit walks through the stages; the weights of the next stage are
 * requested while the outputs of the current one travel between the compute
 * units (through records in the workspace that carry their own epoch), which a
 * launch per layer cannot do.
 *
 * M: 1..AGQ_CHAIN_MAX_M.  Per stage: K % 128 == 0, 128 <= K <= 16384; bits 8 or 4;
 * 1 <= count <= AGQ_MAX_PROJ; every N % 16 == 0, ldy even; pointers as for
 * agq_gemm_w4a8 (acc_out, if given, 8-byte aligned).  n_stages <=
 * AGQ_CHAIN_MAX_STAGES.  stages is a HOST array.
 *
 * agq_gemm_chain_prepare: checks everything on the host, then writes the stage
 * table and zeroes the records in `workspace` (agq_gemm_chain_workspace_bytes,
 * 0 = invalid arguments; 256-byte aligned) and WAITS for `stream`: set-up work,
 * not capturable.  The pointers inside the stages are baked into the workspace.
 * agq_gemm_chain_run: enqueues the one kernel on a prepared workspace; allocates
 * nothing and may be captured and replayed any number of times.  Runs of one
 * workspace must not overlap in time, and the device must not be busy with other
 * kernels of comparable length while a chain runs: the workgroups wait for each
 * other, so all of them have to be resident at once (one per compute unit).
 * Every wait inside the kernel is bounded (20 ms): if one runs out, all workgroups
 * leave, outputs are incomplete, and the workspace is marked; later runs on it
 * return at once.  agq_gemm_chain_status waits for `stream` and returns AGQ_OK or
 * AGQ_ETIMEOUT for the runs so far; after a time-out prepare the workspace again. */
#define AGQ_CHAIN_MAX_M 4
#define AGQ_CHAIN_MAX_STAGES 1024
typedef struct agq_chain_stage {
    const void *x_f16;          /* caller input, or NULL: output of the stage before */
    int64_t ldx;                /* elements; ignored when x_f16 == NULL               */
    int src_proj;               /* which projection of stage s-1 (x_f16 == NULL)      */
    int bits;                   /* activation grid: 8 or 4                            */
    int e;                      /* activation scale 2^e of this stage                 */
    int64_t K;
    int count;
    agq_proj projs[AGQ_MAX_PROJ];
} agq_chain_stage;
size_t agq_gemm_chain_workspace_bytes(const agq_chain_stage *stages, int n_stages, int64_t M);
int agq_gemm_chain_prepare(const agq_chain_stage *stages, int n_stages, int64_t M,
                           void *workspace, size_t workspace_bytes, void *stream);
int agq_gemm_chain_run(void *workspace, void *stream);
int agq_gemm_chain_status(const void *workspace, void *stream);

/* TRIP: per-channel power-of-two factors on top of the layer-wise step
 * (Section 4.3, Eq.5-8) and the matrix product that carries them on the weight
 * rows (Section 4.4, "efficient TRIP matrix multiplication").
 *
 * Eq.5 quantizes input channel k with the step 2^(e + alpha[k]), alpha[k] in
 * 0..AGQ_TRIP_MAX_FACTOR, grid and rounding as in Eq.2:
 *   q[m,k]   = CLIP(round(x[m,k] / 2^(e + alpha[k])) + zp, lo, hi)
 *   acc[m,n] = sum_k (q[m,k] - zp) * 2^alpha[k] * Wq[n,k]      (int32, exact)
 *   y[m,n]   = fp16( float(acc[m,n]) * (2^e * sw[n]) )
 * e is the base (finest) step: Eq.6 is read as the layer-wise step divided by
 * 2^kmax, i.e. e = agq_calibrate_act_exp's result minus kmax.
 *
 * agq_trip_search (Eq.8): alpha[k] = the factor in 0..kmax with the smallest
 * squared error || x[:,k] - dequant(quant(x[:,k])) ||^2 over the M tokens, the
 * quantizer being Eq.5 with its clip; equal errors give the smaller factor.
 * Errors are summed in float64 in token order, so the result is reproducible
 * bit for bit.  x_f16: fp16 [M,K], ldx >= K; alpha_dev: device int8 [K].
 * M == 0 gives all zeros.  A calibration-time call, not tuned for speed.
 *
 * The weight blob for a set of factors: channels with alpha > 0 are served by
 * extra 128-wide chunks (at most AGQ_TRIP_MAX_EXTRA of them, each holding
 * channels of one factor), the other channels by the ordinary chunks.
 * alpha_host is a HOST array int8 [K] (copy agq_trip_search's result back: packing
 * is set-up work).  agq_trip_extra_chunks returns the number of extra chunks
 * (>= 0) these factors need, or AGQ_EINVAL (a factor outside 0..4, more chunks
 * than the maximum, bad K).  agq_pack_w4_trip_bytes(N, K, n_extra) is the blob
 * size (0 = invalid arguments).  agq_pack_w4_trip copies small tables to the
 * device and WAITS for `stream` before it launches its kernels (not capturable).
 * agq_unpack_w4_trip(agq_pack_w4_trip(W)) == W (after saturation to [-8,7]).
 * K % 128 == 0, K <= 32768 (keeps every partial sum inside int32).
 *
 * agq_gemm_w4a8_trip / agq_gemm_w4a4_trip: the layer above with b = 8 / 4.
 * x_f16 is fp16 [M,K] (ldx % 8 == 0, 16-byte aligned): the quantizer runs inside
 * the call.  n_extra: as returned by agq_trip_extra_chunks for the factors the
 * blob was packed with.  workspace: agq_gemm_trip_workspace_bytes(M,N,K,n_extra)
 * (with N = 0: the activation alone, accepted too, as for agq_gemm_w4a8).
 * Other arguments, alignment and errors as for agq_gemm_w4a8.                 */
#define AGQ_TRIP_MAX_FACTOR 4
#define AGQ_TRIP_MAX_EXTRA 16
int agq_trip_search(const void *x_f16, int64_t M, int64_t K, int64_t ldx, int bits,
                    int e, int zp, int kmax, int8_t *alpha_dev, void *stream);
int agq_trip_extra_chunks(const int8_t *alpha_host, int64_t K);
size_t agq_pack_w4_trip_bytes(int64_t N, int64_t K, int n_extra);
int agq_pack_w4_trip(const int8_t *wq, int64_t N, int64_t K, const int8_t *alpha_host,
                     void *packed, int32_t *bad_count_dev, void *stream);
int agq_unpack_w4_trip(const void *packed, int64_t N, int64_t K, int n_extra,
                       int8_t *wq_out, void *stream);
size_t agq_gemm_trip_workspace_bytes(int64_t M, int64_t N, int64_t K, int n_extra);
int agq_gemm_w4a8_trip(const void *x_f16, int64_t M, int64_t K, int64_t ldx, int e, int zp,
                       const void *w_packed, int n_extra, const void *w_scale_f16,
                       int64_t N, void *y_f16, int64_t ldy, int32_t *acc_out,
                       void *workspace, size_t workspace_bytes, void *stream);
int agq_gemm_w4a4_trip(const void *x_f16, int64_t M, int64_t K, int64_t ldx, int e, int zp,
                       const void *w_packed, int n_extra, const void *w_scale_f16,
                       int64_t N, void *y_f16, int64_t ldy, int32_t *acc_out,
                       void *workspace, size_t workspace_bytes, void *stream);
/* Several projections of one activation with TRIP (the factors belong to the
 * activation, so q/k/v or gate/up share them): every blob packed with the same
 * factors, n_extra theirs.  One quantize-and-gather pass, one launch.  projs as for
 * agq_gemm_w4a8_multi; workspace: agq_gemm_trip_workspace_bytes(M, N, K, n_extra)
 * with N = the widths added up.                                                  */
int agq_gemm_w4a8_trip_multi(const void *x_f16, int64_t M, int64_t K, int64_t ldx, int e, int zp,
                             const agq_proj *projs, int count, int n_extra, void *workspace,
                             size_t workspace_bytes, void *stream);
int agq_gemm_w4a4_trip_multi(const void *x_f16, int64_t M, int64_t K, int64_t ldx, int e, int zp,
                             const agq_proj *projs, int count, int n_extra, void *workspace,
                             size_t workspace_bytes, void *stream);

/* Log2 quantizer on softmax probabilities (Section 4.1 Eq.3 with max|X| = 1,
 * used for the softmax output per Section 5.1) fused with the product with the
 * int8 value matrix, plus the token importance of Section 4.3 (attention paid
 * to the first token):
 *   c[h,i,j]  = CLIP(round(-log2 p[h,i,j]), 0, qmax)            (p = 0 -> qmax)
 *   o[i,h*D+d]= fp16( 2^(e_v-qmax) * sum_j 2^(qmax-c[h,i,j]) * v_q[h,j,d] )
 *   score[i]  = sum_h p[h,i,0] * 2^24                           (exact integer)
 * p_f16   : fp16 [H,S,S] in [0,1], row i = query i; causal != 0 reads j <= i only.
 * qmax    : 15 (all four bits carry magnitude) or 7 (Eq.3's 2^(b-1)-1, b = 4).
 * v_q     : int8 [H,S,D], scale 2^e_v;  D % 16 == 0, D <= 256;  S % 8 == 0,
 *           S <= 32768.
 * o_f16   : fp16 [S, H*D].   codes_out: optional [H,S,S/2] bytes, two codes per
 *           byte, low nibble = even j, entries above the diagonal carry qmax.
 * score_out: optional int32 [S]; needs H <= 127.
 * Precondition: rows are softmax outputs (values in [0,1], sum <= ~1), which
 * keeps the integer sum below 2^24; a value above 1 gives an unspecified
 * result, and arbitrary inputs may lose low bits.                           */
int agq_log2_quant_softmax(const void *p_f16, int64_t H, int64_t S, int64_t D,
                           int causal, int qmax, const int8_t *v_q, int e_v,
                           void *o_f16, void *codes_out, int32_t *score_out,
                           void *stream);

/* Attention from quantized Q and K in one call: the integer product Q K^T
 * (Section 4.2 lists QK among the quantized products), softmax in floating point
 * (Section 3.3), Eq.3 on the probabilities, the product with the int8 value
 * matrix, and the token importance of Section 4.3 read on the quantized map.
 * The probabilities are never written to memory.
 *   s[h,i,j]  = sum_d q_q[h,i,d] * k_q[h,j,d]                    (int32, exact)
 *   p[h,i,:]  = softmax_j( s * 2^(e_q+e_k) / sqrt(D) )           (j <= i if causal)
 *   c[h,i,j]  = CLIP(round(-log2 p[h,i,j]), 0, qmax)
 *   o[i,h*D+d]= fp16( 2^(e_v-qmax) * sum_j 2^(qmax-c[h,i,j]) * v_q[h,j,d] )
 *   score[i] += sum_h 2^(qmax - c[h,i,0])
 * -log2 p is evaluated in fp32 as log2(sum_j 2^(kappa s_j)) - kappa s, kappa =
 * 2^(e_q+e_k) log2(e) / sqrt(D), with the hardware's exp2 / log2: a code may differ
 * from an exact evaluation where -log2 p lies within about 1e-5 of a rounding
 * boundary, to which 2^-22 times the row's largest |kappa s| is added for kappa
 * <= 1 (6e-5 at 256; beyond kappa = 1 differences of scores are scaled instead);
 * o and score follow exactly from the codes.
 * q_q, k_q, v_q : int8 [H,S,D] on the signed grid of Eq.2 with scales 2^e_q,
 *           2^e_k, 2^e_v.  D = 64 or 128; S % 128 == 0, S <= 32768.
 * qmax    : 15 or 7.   o_f16: fp16 [S, H*D].
 * codes_out : optional [H,S,S/2] bytes as for agq_log2_quant_softmax.
 * score_out : optional int32 [S], ACCUMULATED with atomic adds: the caller
 *           zeroes it before the call.
 * All pointers 16-byte aligned.                                               */
int agq_qk_log2_softmax(const int8_t *q_q, const int8_t *k_q, int64_t H, int64_t S,
                        int64_t D, int causal, int qmax, int e_q, int e_k,
                        const int8_t *v_q, int e_v, void *o_f16, void *codes_out,
                        int32_t *score_out, void *stream);

/* Token pruning, Section 4.3 Eq.4: keep the n_keep tokens with the largest
 * score (equal scores: lower index first), in their original order.
 * score  : int32 [S], S <= 8192.   x_f16: fp16 [S,d] contiguous, d % 8 == 0.
 * idx_out: int32 [n_keep] ascending.  x_out_f16: fp16 [n_keep,d].
 * 0 <= n_keep <= S.                                                           */
int agq_prune_tokens(const int32_t *score, int64_t S, int64_t n_keep,
                     const void *x_f16, int64_t d, int32_t *idx_out,
                     void *x_out_f16, void *stream);

/* One block of the quantized model: the activation quantization pipeline of
 * Section 4.2 (Figure 3: every matrix product takes quantized operands, the
 * non-linear operators in between stay in fp16) with the activation-aware token
 * pruning of Section 4.3 right after attention, for a LLaMA block (RMSNorm,
 * rotary embedding, SwiGLU).  With x fp16 [S,d], positions pos[S]:
 *   h1        = RMSNorm(x; g_attn)
 *   q,k,v     = W4A8(h1)        one Eq.2 pass (step 2^e_attn_in) serves all three
 *   Q,K,V     = Eq.2 to int8 of rope(q), rope(k), v   (steps 2^e_q, 2^e_k, 2^e_v)
 *   o, score  = agq_qk_log2_softmax(Q, K, V), causal
 *   idx       = the n_keep tokens with the largest score (agq_prune_tokens' rule)
 *   x1        = x[idx] + W4A8-or-W4A4(o[idx])           (step 2^e_attn_out;
 *               Section 4.2 allows 4-bit activations after self-attention)
 *   h2        = RMSNorm(x1; g_mlp)
 *   a         = silu(gate) * up,  gate, up = W4A8(h2)   (one Eq.2 pass, 2^e_mlp_in)
 *   x_out     = x1 + W4A8(a)                            (step 2^e_mlp_act)
 * RMSNorm: y = x g / sqrt(mean(x^2) + rms_eps).  rope: inside a head of width D the
 * pair (i, i + D/2) is rotated by the angle whose cosine and sine are
 * rope_cos[pos, i], rope_sin[pos, i].  Every fp16 operator returns what float64
 * arithmetic gives, rounded once to fp16.  All activation grids are signed (zp = 0).
 *
 * d = H*D with D = 64 or 128; d % 128 == 0, F % 128 == 0; 1 <= n_keep <= S
 * (n_keep == S: nothing is pruned); S <= 8192 when tokens are pruned, else
 * S <= 32768.  Eq.9's cascade is a sequence of such calls whose n_keep follow
 * agq_cascade_keep (agq_stack_forward runs such a sequence in one call).
 * All pointers are device pointers, 16-byte aligned; weights are agq_pack_w4 blobs
 * ([d,d] for q, k, v, o; [F,d] for gate, up; [d,F] for down) with fp16 scales.   */
typedef struct agq_block {
    int64_t d, H, F;
    int qmax;               /* 15 or 7, as for agq_qk_log2_softmax                */
    int bits_attn_out;      /* 4 or 8: activation grid of the projection after attention */
    double rms_eps;
    const void *g_attn_f16, *g_mlp_f16;                /* fp16 [d]               */
    const void *w_q, *w_k, *w_v, *w_o, *w_gate, *w_up, *w_down;
    const void *s_q, *s_k, *s_v, *s_o, *s_gate, *s_up, *s_down;
    /* static exponents of the seven quantizers (post-training calibration)       */
    int e_attn_in, e_q, e_k, e_v, e_attn_out, e_mlp_in, e_mlp_act;
    /* TRIP (Section 4.3) at the four activations that feed projections: -1 = the
     * projections of that activation are agq_pack_w4 blobs and Eq.2 is used; n >= 0 =
     * they are agq_pack_w4_trip blobs, all packed with the same factors, n =
     * agq_trip_extra_chunks of those factors, and the site's exponent is Eq.6's base
     * step.  (attn_in: q, k, v; attn_out: o; mlp_in: gate, up; mlp_act: down.)
     * Needs d, F <= 32768.  Factors come from agq_trip_search on the site's tensor of
     * a calibration pass (h1, o_kept, h2, act in the workspace).                  */
    int trip_attn_in, trip_attn_out, trip_mlp_in, trip_mlp_act;
} agq_block;

/* Where every intermediate tensor of a call lives inside the workspace (byte
 * offsets; fp16 unless noted).  Shapes: h1, q, k, v [S,d]; q_q, k_q, v_q int8
 * [H,S_pad,D] (rows from S on are zero); o [S_pad,d]; score int32 [S_pad]; idx int32
 * [n_keep]; o_kept, attn_out, x1, h2, down [n_keep,d] (o_kept == o when nothing is
 * pruned); gate, up, act [n_keep,F]; q_rot, k_rot [S,d] (written by
 * agq_block_calibrate only).  total = the workspace size a call needs.           */
typedef struct agq_block_layout {
    int64_t S_pad;          /* S rounded up to a multiple of 128                   */
    size_t h1, q, k, v, q_q, k_q, v_q, o, score, idx, o_kept, attn_out, x1, h2, gate, up, act, down, q_rot, k_rot,
        gemm_ws, total;
} agq_block_layout;
int agq_block_layout_of(const agq_block *blk, int64_t S, int64_t n_keep, agq_block_layout *out);

/* The fp16 operators of the block as calls of their own (Section 4.2 keeps them in
 * fp16; other block shapes can be wired from these and the products above).  Each
 * returns what float64 arithmetic gives, rounded once to fp16 (values for which fewer
 * bits tell that are computed in fewer).  fp16 tensors are contiguous
 * (leading dimension = row width) and 16-byte aligned.
 *
 * agq_rmsnorm: y[r,:] = t[r,:] * g / sqrt(mean(t[r,:]^2) + eps).  res_f16 == NULL:
 * t = x.  Otherwise t[r,:] = fp16(res[idx[r],:] + x[r,:]) (idx == NULL: row r
 * itself), also written to sum_out_f16 [rows,d]: the residual addition, and the row
 * gather after pruning, fused into the normalisation that follows them.
 * d % 8 == 0, d <= 65536; idx values must be valid rows of res.
 *
 * agq_rope_quantize: rotary embedding of q and k (pairs (i, i + D/2) of every head,
 * angle tables float32 [P, D/2] read at row pos[t], positions clamped into the
 * table), then Eq.2 to int8 (signed grid, steps 2^e_q, 2^e_k, 2^e_v) of the rotated
 * q, k and of v, written per head: int8 [H, S_pad, D] with zero rows from S on
 * (S_pad >= S; agq_qk_log2_softmax wants a multiple of 128).  q, k, v: fp16
 * [S, H*D]; D % 16 == 0.
 *
 * agq_swiglu: out = silu(gate) * up, silu(z) = z / (1 + exp(-z)); n elements,
 * n % 8 == 0.   agq_residual_add: out = fp16(a + b); n % 8 == 0.                  */
int agq_rmsnorm(const void *x_f16, const void *res_f16, const int32_t *idx, const void *g_f16,
                int64_t rows, int64_t d, double eps, void *sum_out_f16, void *y_f16, void *stream);
int agq_rope_quantize(const void *q_f16, const void *k_f16, const void *v_f16, int64_t S, int64_t H,
                      int64_t D, const int32_t *pos, const float *rope_cos, const float *rope_sin,
                      int64_t P, int e_q, int e_k, int e_v, int64_t S_pad, int8_t *q_q, int8_t *k_q,
                      int8_t *v_q, void *stream);
int agq_swiglu(const void *gate_f16, const void *up_f16, void *out_f16, int64_t n, void *stream);
int agq_residual_add(const void *a_f16, const void *b_f16, void *out_f16, int64_t n, void *stream);

/* x_f16 [S,d]; pos int32 [S], every value in [0, P); rope_cos, rope_sin float32
 * [P, D/2] (a position outside the table is clamped into it).  x_out_f16
 * [n_keep,d]; pos_out int32 [n_keep] = pos[idx] (may be NULL).  workspace: `total`
 * bytes of agq_block_layout_of, 256-byte aligned.  Enqueues kernels only.        */
int agq_block_forward(const agq_block *blk, const void *x_f16, const int32_t *pos, const float *rope_cos,
                      const float *rope_sin, int64_t P, int64_t S, int64_t n_keep, void *x_out_f16,
                      int32_t *pos_out, void *workspace, size_t workspace_bytes, void *stream);

/* The same pass with every exponent derived on the way from this input
 * (agq_calibrate_act_exp on the tensor each quantizer reads) and written back to
 * *blk: the post-training calibration step.  Waits for `stream` several times; not
 * capturable.  All four trip_* fields must be -1 (plain blobs).                   */
int agq_block_calibrate(agq_block *blk, const void *x_f16, const int32_t *pos, const float *rope_cos,
                        const float *rope_sin, int64_t P, int64_t S, int64_t n_keep, void *x_out_f16,
                        int32_t *pos_out, void *workspace, size_t workspace_bytes, void *stream);

/* A stack of blocks with the cascade pruning of Section 5.2: block l receives the
 * tokens block l-1 kept and keeps keep[l] of them (keep[l] equal to what it
 * receives: that block prunes nothing); Eq.9's schedule prunes in m of the blocks
 * with the counts of agq_cascade_keep.  blocks: HOST array of n_blocks descriptors
 * with the same d (read before the call returns); keep: HOST int64 [n_blocks],
 * non-increasing, keep[0] <= S.  x_out_f16 [keep[n_blocks-1], d]; pos_out as for a
 * block.  workspace: agq_stack_workspace_bytes (0 = invalid arguments), 256-byte
 * aligned; after the call it holds the intermediates of the last block only.
 * Enqueues kernels only.  Same result as n_blocks calls of agq_block_forward.    */
size_t agq_stack_workspace_bytes(const agq_block *blocks, int n_blocks, int64_t S, const int64_t *keep);
int agq_stack_forward(const agq_block *blocks, int n_blocks, const int64_t *keep, const void *x_f16,
                      const int32_t *pos, const float *rope_cos, const float *rope_sin, int64_t P,
                      int64_t S, void *x_out_f16, int32_t *pos_out, void *workspace,
                      size_t workspace_bytes, void *stream);

/* Section 5.2, Eq.9: m pruning stages share the progressive ratio
 * gamma = 1 - (1 - beta)^(1/m), so that a fraction beta is gone after the last one;
 * a stage that receives S tokens keeps S - floor(S * gamma).  keep_out (HOST int64
 * [m]) receives the tokens left after each stage.  0 <= beta < 1, 1 <= m <= 1024.  */
int agq_cascade_keep(int64_t S, double beta, int m, int64_t *keep_out);

/* ---- Serving: a paged key/value cache in 8 bits, and attention for prompts and for generated tokens.
 *
 * The projections of generation read every weight once per step (agq_gemm_w4a8 and the others with few rows); these
 * calls are what lies between them.  A step is: agq_kv_map (which pages and slots the step's new tokens get), per layer
 * agq_kv_append (rotary embedding, keys and values into the cache on Eq.2's 8-bit grid, the step's exponent per page and
 * head instead of per layer), then agq_attn_packed for prompts (fp16 keys and values as they came from the projections)
 * or agq_attn_kv for generated tokens (everything from the cache).
 *
 * Conventions of these calls: fp16 tensors are [tokens, heads, D] with a leading dimension ("ld", elements, a multiple
 * of 8, at least heads * D) between tokens, so q, k and v may be parts of one projection's output; fp16 tensors,
 * caches, rope tables and workspaces are 16-byte aligned, int32 arrays 4-byte.  D = 64 or 128.  Hq % Hkv == 0: query
 * head h reads key head h / (Hq / Hkv).  page = tokens of a page: 16, 32, 64 or 128.  `cu` arrays hold B + 1 offsets in
 * ascending order; sequence b is tokens cu[b] .. cu[b+1] - 1 of the packed tensor, and rows that belong to no sequence
 * (padding behind the last one) are neither read nor written.  Offsets, lengths, page numbers and slots live on the
 * device and are never trusted with an address: whatever lies outside the tensors is left out.  Every call enqueues
 * kernels only, may be captured, and needs nothing cleared.  Outputs overlap neither inputs nor each other unless a call
 * says so.  A call with no tokens is a no-op (agq_kv_map: it still gives back pages).                                */

/* The cache of one layer.  Entry (token, d) of page p and head h is the code k[p, h, token, d] with the scale
 * 2^k_exp[p, h]; values lie transposed inside a page, v[p, h, d, token], scale 2^v_exp[p, h].  agq_kv_append makes
 * exponents of -30 .. 10; agq_attn_kv reads any, those beyond -64 .. 64 as the nearer of the two.  All pages of a cache
 * lie in one allocation; n_pages * page < 2^31.  HOST struct, read before a call returns.                            */
typedef struct agq_kv_cache {
    int8_t *k;              /* int8 [n_pages, Hkv, page, D]                          */
    int8_t *v;              /* int8 [n_pages, Hkv, D, page]                          */
    int8_t *k_exp, *v_exp;  /* int8 [n_pages, Hkv]                                   */
    int64_t n_pages, Hkv, D, page;
} agq_kv_cache;

/* Pages, slots and positions of one step from the requests' lengths, on the device in one launch.
 * kv_len [B]: tokens that request b has in the cache; n_new [B]: tokens that it gets in this step, or -1: it is
 * finished, its pages go back and its length becomes 0.  block_table [B, max_pages] (updated): the page numbers of
 * request b, entry j for its tokens j * page .. (j+1) * page - 1; entries behind its pages mean nothing.
 * The free pages are a ring: free_ring [n_pages] (updated) and free_state = {head, count}; pages are taken at head, in
 * the order of requests and tokens, and given back behind the last one in the same order.  To begin with: free_ring =
 * 0 .. n_pages - 1 in any order, free_state = {0, n_pages}, kv_len = 0.
 * Out: kv_len_out [B] (the lengths after the step), cu_new [B+1] (offsets of the requests' new tokens, finished
 * requests have none), pos [T], slot [T] (token t goes to token slot % page of page slot / page; T >= the sum of the
 * new tokens; rows behind them get pos 0, slot -1), free_state_out, and *status: 0; or the number of free pages that
 * are missing; or -1 (a negative length, n_new < -1, a request longer than max_pages * page, more than T tokens, an
 * impossible free_state).  With a status other than 0 the step is left out: lengths, table, ring and state stay as they
 * are, cu_new is all 0 and every slot -1, so that calls which follow do nothing.
 * kv_len_out and free_state_out must not overlap kv_len and free_state (AGQ_EINVAL): a loop swaps two of each.  Between
 * steps a program may lower a length (a draft's tokens that were not taken) as far as the request keeps its pages;
 * pages behind that would be lost, as nothing gives them back.  n_new = -1 gives pages back without a look at other requests
 * that hold them: where pages are shared (agq_kv_fork, below) a request is ended by agq_kv_fork alone.
 * B <= 2^20; max_pages * page < 2^31; pos and slot may be NULL when T == 0.                                          */
int agq_kv_map(const int32_t *kv_len, const int32_t *n_new, int64_t B, int64_t page, int32_t *block_table,
               int64_t max_pages, int32_t *free_ring, int64_t n_pages, const int32_t *free_state, int64_t T,
               int32_t *kv_len_out, int32_t *cu_new, int32_t *pos, int32_t *slot, int32_t *free_state_out,
               int32_t *status, void *stream);

/* A step's keys and values into the cache, with the rotary embedding on the way (as in agq_rope_quantize: pairs
 * (i, i + D/2), float64 arithmetic, rounded once to fp16; positions are clamped into the tables).
 * slot [T]: as agq_kv_map writes it.  A token whose slot is negative or not in the cache is left out: nothing of it is
 * read or written.  Codes: Eq.2 on the signed 8-bit grid with the step 2^e, e that of the page and head:
 *   e = the smallest e with max|x| <= 127 * 2^e over the tokens that this call writes there (infinities count as 2^16, a
 *       NaN as nothing, all zeros as 2^-30's e), but not below the page's present e if earlier tokens lie in front of
 *       them (slot % page of the first one > 0); the codes of those are then divided by 2^(e - present e), halves to the
 *       even code.
 * Tokens of the call in one page have to be consecutive, in the order of their slots, and no slot twice, as agq_kv_map
 * makes them; otherwise the contents of that page (of no other memory) are unspecified.  Bytes of the page behind them
 * stay as they are.
 * k, v: fp16 [T, Hkv, D].  q (may be NULL with q_out NULL, Hq = 0): fp16 [T, Hq, D], rotated into q_out.  k_out (may be
 * NULL): the rotated keys in fp16, for agq_attn_packed.  q_out and k_out may be q and k themselves.
 * rope_cos, rope_sin [P, D/2] float32 and pos [T]; all three NULL: no rotation (q and k_out must be NULL then).
 * T * D / 16 <= (2^31 - 1) / max(Hq, 2 Hkv) - 4096.                                                                    */
int agq_kv_append(const agq_kv_cache *cache, const void *k_f16, int64_t ldk, const void *v_f16, int64_t ldv, int64_t T,
                  const int32_t *slot, const void *q_f16, int64_t ldq, int64_t Hq, const int32_t *pos,
                  const float *rope_cos, const float *rope_sin, int64_t P, void *q_out_f16, int64_t ldqo,
                  void *k_out_f16, int64_t ldko, void *stream);

/* Attention over packed prompts, fp16 in and out, in one pass over the keys:
 *   o[i,h] = sum_j softmax_j( scale * q[i,h] . k[j,h'] ) v[j,h'],   h' = h / (Hq / Hkv)
 * over the keys j of the query's own sequence; causal != 0: query i of n sees keys j <= i + (m - n) of m, so the last
 * query sees the last key (n < m: the queries are the later part of the prompt; n > m: the first queries see nothing).
 * A row that sees no key is 0, one that sees keys with scores of -infinity only is NaN.  Keys and values that a row does
 * not see do not reach it, infinities and NaN included; an infinity or NaN among the values that it sees makes their
 * column of it infinite or NaN.
 * q, o: fp16 [Tq, Hq, D]; k, v: fp16 [Tk, Hkv, D], ldk and ldv at most 2^24; cu_q, cu_k [B+1].
 * 2^-60 <= scale <= 2^24, usually 1 / sqrt(D); B <= 2^20; Hq * (Tq / 128 + B) < 2^24 (a launch's workgroups).
 * workspace: agq_attn_packed_workspace_bytes (0, and NULL, unless there are few queries and many keys): partial results
 * where workgroups share the keys of a tile of queries; contents are scratch.
 * Scores, maxima, sums and the accumulated output are fp32; a probability is rounded to fp16 (by 2^-11 of it at
 * most) for the product with v; the output is rounded once.                                                            */
size_t agq_attn_packed_workspace_bytes(int64_t Tq, int64_t Hq, int64_t Tk, int64_t Hkv, int64_t D, int64_t B);
int agq_attn_packed(const void *q_f16, int64_t ldq, int64_t Tq, int64_t Hq, const void *k_f16, int64_t ldk,
                    const void *v_f16, int64_t ldv, int64_t Tk, int64_t Hkv, int64_t D, const int32_t *cu_q,
                    const int32_t *cu_k, int64_t B, int causal, float scale, void *o_f16, int64_t ldo, void *workspace,
                    size_t workspace_bytes, void *stream);

/* Attention of each request's newest tokens over its pages: the same sum over the cache, for the n = cu_q[b+1] -
 * cu_q[b] tokens that are the last of the request's kv_len[b] (kv_len counts them: agq_kv_append comes first; it is
 * agq_kv_map's kv_len_out).  Always causal: token i of n sees the first kv_len - n + i + 1 tokens.  n = 1 is plain
 * generation; a few tokens (a draft to be checked) share one pass over the cache; a prompt's part works as well.
 * max_q, max_kv: the largest n and kv_len as the program knows them.  They choose how the work is dealt out (and so the
 * workspace); larger lengths are computed all the same.  Lengths beyond max_pages * page are cut to it, and tokens of a
 * page number outside the cache are left out.
 * q, o: fp16 [T, Hq, D].  workspace: agq_attn_kv_workspace_bytes (may be 0; NULL then): partial results where the keys
 * of a request are shared by several workgroups; contents are scratch.  scale as in agq_attn_packed; Hq / Hkv <= 1024;
 * B <= 65535; max_pages * page, max_q and max_kv at most 2^30.
 * Codes are exact in fp16; scores, maxima, sums and the accumulated output are fp32.  (A key enters its score's sum 128
 * steps larger, which are taken out again: the sum's roundings are those of 128 * 2^k_exp * |q|_1 in size, as if every
 * code of the page were that large.)  For the product with v, and for it alone, a probability times its page's scale of
 * v is rounded to fp16: by 2^-11 of it at most, down to 2^-29 of the row's largest such product, and by 2^-40 of that
 * one below.                                                                                                         */
size_t agq_attn_kv_workspace_bytes(int64_t T, int64_t Hq, int64_t Hkv, int64_t D, int64_t B, int64_t max_q, int64_t max_kv);
int agq_attn_kv(const agq_kv_cache *cache, const void *q_f16, int64_t ldq, int64_t T, int64_t Hq, const int32_t *cu_q,
                const int32_t *kv_len, int64_t B, const int32_t *block_table, int64_t max_pages, int64_t max_q,
                int64_t max_kv, float scale, void *o_f16, int64_t ldo, void *workspace, size_t workspace_bytes,
                void *stream);

/* agq_kv_append for models that normalise their queries and keys per head: before the rotation
 *   y[i] = x[i] * g[i] / sqrt(mean(x^2) + eps)        over the D values of each head of q and of k, not of v,
 * and y is rotated and rounded once: float64 arithmetic from the fp16 input to the fp16 result.
 * g_q, g_k: fp16, 16-byte aligned, [D] for all heads (ldgq, ldgk = 0) or [heads, D] with ldg elements between heads (a
 * multiple of 8, at least D).  g_q is NULL where q is.  eps >= 0.  q, q_out and k_out may be given without tables (pos,
 * rope_cos, rope_sin NULL: no rotation).  Everything else as in agq_kv_append.                                          */
int agq_kv_append_norm(const agq_kv_cache *cache, const void *k_f16, int64_t ldk, const void *v_f16, int64_t ldv, int64_t T,
                       const int32_t *slot, const void *q_f16, int64_t ldq, int64_t Hq, const void *g_q_f16, int64_t ldgq,
                       const void *g_k_f16, int64_t ldgk, double eps, const int32_t *pos, const float *rope_cos,
                       const float *rope_sin, int64_t P, void *q_out_f16, int64_t ldqo, void *k_out_f16, int64_t ldko, void *stream);

/* The same normalisation and rotation without a cache, fp16 to fp16, for texts that are only scored (agq_attn_packed reads
 * the results).  q: fp16 [T, Hq, D], k: [T, Hkv, D]; either may be absent (NULL, with its output, and 0 heads).  A gain that
 * is NULL: that tensor is not normalised.  No tables (all three NULL): no rotation; one of the two has to be there.  q_out
 * and k_out may be q and k themselves.  T * (Hq + Hkv) * D < 2^35.                                                        */
int agq_qk_norm_rope(const void *q_f16, int64_t ldq, int64_t Hq, const void *k_f16, int64_t ldk, int64_t Hkv, int64_t T, int64_t D,
                     const void *g_q_f16, int64_t ldgq, const void *g_k_f16, int64_t ldgk, double eps, const int32_t *pos,
                     const float *rope_cos, const float *rope_sin, int64_t P, void *q_out_f16, int64_t ldqo, void *k_out_f16,
                     int64_t ldko, void *stream);

/* ---- Pages that several requests hold, requests that go on as copies of others, and requests that lose tokens.
 *
 * shared [n_pages] counts the requests that hold a page beyond the first one: 0 for a free page and for one with a single
 * holder (a count below 0 is taken as 0).  To begin with all are 0; agq_kv_map neither needs nor changes them, as the pages
 * that it takes are free.  But it gives pages back without looking: with shared pages around, requests are ended by
 * agq_kv_fork.  A request writes only into the page that its length ends in, so full pages can be shared; agq_kv_fork and
 * agq_kv_compact leave every partly filled page that a request would write into to that request alone.  A length that a
 * program lowers by itself must therefore stay within the last page if that one is not shared; agq_kv_compact takes any.
 * Both calls work from the old lengths, table, counts and ring state to new ones (a loop swaps two of each), on the device, in
 * one launch or three; the ring alone is updated in place, behind the free pages.  No output, the ring and moves among them, may
 * overlap an input, parents, stay and listed tokens among them, or another output (AGQ_EINVAL).
 * Pages are taken at the ring's head in the order of requests and entries, as in agq_kv_map; pages that lost their last
 * holder are given back in ascending order, and are not taken again by the same call.  Entries of block_table_out behind a
 * request's pages are left as they are.  *status: 0; or the number of free pages that are missing; or -1 (an impossible
 * free_state, a length that is negative or beyond max_pages * page, more pages to be given back than are not free, and what each
 * call adds).  With a status other than 0 nothing happens: the outputs are copies of the inputs, and the calls that follow do
 * nothing (where too many pages were to be given back, ring entries that are not free and table entries behind a request's pages
 * are unspecified; they mean nothing).
 * 0 <= B <= AGQ_KV_MAX_FORK.  Everything is captured and replayed like the other calls.                                 */
#define AGQ_KV_MAX_FORK 4096

/* After the call request b is what request parent[b] was before it: itself (parent[b] == b), a copy of another one, or
 * nothing (-1: length 0).  A request that is nobody's parent has ended.  Full pages are held by every copy; a partly filled
 * last page goes to the first copy (the lowest b; to none if the page is shared), and the others get a free page each that
 * it has to be copied into: copy_src[b] to copy_dst[b], -1 where nothing is to be copied.  agq_kv_copy_pages does that, in
 * every layer, before anything else is written into the cache.  status -1 also for a parent outside -1 .. B - 1.          */
int agq_kv_fork(const int32_t *kv_len, const int32_t *parent, int64_t B, int64_t page, const int32_t *block_table,
                int64_t max_pages, const int32_t *shared, int32_t *free_ring, int64_t n_pages, const int32_t *free_state,
                int32_t *kv_len_out, int32_t *block_table_out, int32_t *shared_out, int32_t *copy_src, int32_t *copy_dst,
                int32_t *free_state_out, int32_t *status, void *stream);

/* Pages src[i] to dst[i], codes and exponents, whole, in each of the caches (HOST array, n_caches <= 65536, read before the
 * call returns; all of one n_pages, Hkv, D and page).  An i whose src or dst is not in the cache is left out.  No page may
 * be written twice or be both read and written (unspecified contents of those pages).  0 <= n <= 2^20.                    */
int agq_kv_copy_pages(const agq_kv_cache *caches, int n_caches, const int32_t *src, const int32_t *dst, int64_t n, void *stream);

/* Request b keeps its first stay[b] tokens (all of them if it has no more) and of the others those that are listed:
 * keep[cu_keep[b]] .. keep[cu_keep[b+1] - 1], in ascending order, each at least stay[b] and below kv_len[b].  They move
 * together: token i of the request is token i as before for i < stay[b], else keep[cu_keep[b] + i - stay[b]].  With no
 * listed tokens the request is cut to its first stay[b]; with those all kept as well it stays as it is.
 * Pages in front of stay[b] / page stay; where tokens are listed the pages from there on are new ones, else all remaining
 * pages stay, but a partly filled last page that is shared and is now to be written into becomes a new one.  The old pages
 * are let go.  moves [agq_kv_moves_ints(N, B, page)], 16-byte aligned: the new pages, for agq_kv_move; its contents are the library's.
 * Keys keep the rotation of their old positions, while agq_kv_map counts a request's next position from its new length: a
 * program that wants the old count adds the difference to pos.
 * status -1 also for a stay below 0, cu_keep that descends or leaves 0 .. N, and listed tokens that are not as said.
 * 0 <= N < 2^30.                                                                                                         */
size_t agq_kv_moves_ints(int64_t N, int64_t B, int64_t page);
int agq_kv_compact(const int32_t *kv_len, const int32_t *stay, const int32_t *cu_keep, const int32_t *keep, int64_t N, int64_t B,
                   int64_t page, const int32_t *block_table, int64_t max_pages, const int32_t *shared, int32_t *free_ring,
                   int64_t n_pages, const int32_t *free_state, int32_t *kv_len_out, int32_t *block_table_out,
                   int32_t *shared_out, int32_t *moves, int32_t *free_state_out, int32_t *status, void *stream);

/* The tokens of agq_kv_compact's new pages, in each of the caches (as in agq_kv_copy_pages), from the pages that held them:
 * block_table, stay, cu_keep and keep are those that agq_kv_compact was given.  It comes before anything else is written
 * into the cache, as the old pages are free by then.  A new page's exponent is the largest of its tokens' old ones; codes of
 * the others are divided by what it grew by, halves to the even code.  Entries of a new page behind its tokens are 0.      */
int agq_kv_move(const agq_kv_cache *caches, int n_caches, const int32_t *moves, const int32_t *block_table, int64_t max_pages,
                const int32_t *stay, const int32_t *cu_keep, const int32_t *keep, int64_t N, int64_t B, void *stream);

/* ---- What a model answers: log probabilities of given tokens, entropy, and the likeliest tokens of each row of logits.
 *   p[t,:] = softmax(scale * x[t,:]),   logprob[t] = log p[t, tokens[t]],   entropy[t] = - sum_v p log p,
 *   top_idx[t, 0..n_top-1] = the tokens with the largest x[t,v], equal ones by their index, top_logprob their log p.
 * logits: [T, V], fp16 or float32 (kind), ld >= V elements between rows, aligned to its type; agq_gemm_w4a8's output is such
 * a tensor.  tokens int32 [T]; a token outside 0 .. V - 1 (no token is given) has logprob NaN.  scale: 1 / temperature.
 * logprob, entropy float32 [T]; top_idx int32, top_logprob float32 [T, n_top] contiguous.  tokens and logprob, entropy, and
 * both of top_* (n_top == 0 then) may be NULL.
 * Logits of -infinity are tokens that are ruled out: p = 0, log p = -infinity, 0 in the entropy; as alternatives they come
 * last.  A row without a distribution (a NaN or +infinity among its logits, or -infinity only) has NaN for logprob, entropy
 * and top_logprob, and -1 for top_idx.
 * 1 <= V <= 2^24, 0 <= T <= 2^22, 0 <= n_top <= min(V, AGQ_MAX_TOP), 2^-24 <= scale <= 2^24, ld <= 2^30; float32 logits times
 * scale have to be finite (a log probability below float32's range is -infinity).  workspace: agq_logprobs_workspace_bytes, 16-byte aligned; contents are scratch.
 * Exponents and results are float32, sums float32 for a few values and float64 beyond, in a fixed order.  With d = 2^-24, D the
 * mean and Q the mean square of scale (max x - x) under p, a log probability l is off by at most d (|l| + 8 D + 32), an entropy H by
 * d (H + 128 + 128 D + 16 Q), whatever V; 1 to 2 d of the result are usual.                                               */
enum agq_logit_kind { AGQ_LOGITS_F16 = 0, AGQ_LOGITS_F32 = 1 };
#define AGQ_MAX_TOP 64
size_t agq_logprobs_workspace_bytes(int64_t T, int64_t V, int kind, int64_t n_top);
int agq_logprobs(const void *logits, int kind, int64_t T, int64_t V, int64_t ld, float scale, const int32_t *tokens,
                 int64_t n_top, float *logprob, float *entropy, int32_t *top_idx, float *top_logprob, void *workspace,
                 size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* AGQ_H */
