/*
 * hif8.h -- C ABI of the B200 (sm_100a) HiFloat8 conversion library.
 *
 * HiFloat8 (HiF8) is the 8-bit tapered floating-point format of "Ascend HiFloat8 Format for Deep
 * Learning" (arXiv 2409.16626), Section 2.1: one byte = sign | dot field (prefix code, Table 2) |
 * sign-magnitude exponent with implicit leading 1 (Table 3) | 3/2/1-bit mantissa; normal values follow
 * Eq. 1, the denormal extension follows Eq. 2; 0x00 is the single zero, 0x80 is NaN, 0x6F / 0xEF are
 * +-Inf (Table 4).
 *
 * Conventions for every entry point
 *   - All data pointers are DEVICE pointers owned by the caller (any CUDA allocation); the library
 *     never allocates, frees or copies to the host, and never synchronises.  All work is enqueued on
 *     `stream` (a cudaStream_t; NULL = the legacy default stream) of the current device.
 *   - Tensors are contiguous, element count `n`.  Any byte alignment is accepted; 16-byte aligned
 *     pointers take the vectorised path, others a slower scalar kernel with identical results.
 *   - Return value: HIF8_OK or an error code (see hif8_status_string).  Argument errors are detected
 *     before anything is launched and leave all outputs untouched.  NaN / Inf inputs are data.
 *   - A conversion whose source and destination byte ranges intersect is rejected with HIF8_ERR_OVERLAP
 *     (host-side range test; the kernels read and write in an order that makes no promise for aliased data).
 *   - `scale_exp` is the exponent E of a power-of-two scale 2^E (Section 4.2: scale factors are
 *     integer powers of two, so scaling only adds to the exponent), limited to [-126, 126].
 *   - The library needs a CUDA device of compute capability 10.0 and fails with HIF8_ERR_CUDA elsewhere.
 */
#ifndef HIF8_H
#define HIF8_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct CUstream_st* hif8_stream_t; /* same type as cudaStream_t */

/* element formats of the high-precision side (Section 3: FP32, FP16 and BF16 sources) */
typedef enum { HIF8_F32 = 0, HIF8_BF16 = 1, HIF8_F16 = 2 } hif8_dtype_t;

/* rounding methods of Section 3 */
typedef enum {
    HIF8_RND_TA = 0,  /* Section 3.1: round half away from zero (the default everywhere)               */
    HIF8_RND_HR = 1,  /* Eq. 3: hybrid -- TA if |E| < 4, simplified stochastic rounding if |E| >= 4    */
    HIF8_RND_SSR = 2, /* Section 3.2 simplified SR for every E: SR14 (FP32 source), SR2 (FP16 / BF16)  */
    HIF8_RND_TE = 3,  /* Section 3.1: round half to even                                               */
    HIF8_RND_SR = 4   /* Section 3.2 standard SR; thresholds from Philox4x32-10 keyed by `seed`         */
} hif8_round_t;

/* the two options of Section 3 */
enum {
    HIF8_FLAG_SATURATE = 1u,   /* overflow (and a source +-Inf) gives +-2^15 instead of +-Inf */
    HIF8_FLAG_NAN_TO_ZERO = 2u /* a source NaN gives 0x00 instead of 0x80                     */
};

enum {
    HIF8_OK = 0,
    HIF8_ERR_NULL = 1,        /* a required pointer is NULL                         */
    HIF8_ERR_DTYPE = 2,       /* unknown element format                             */
    HIF8_ERR_ROUND = 3,       /* unknown rounding method                            */
    HIF8_ERR_FLAGS = 4,       /* unknown option bits                                */
    HIF8_ERR_SCALE_RANGE = 5, /* scale or target exponent outside [-126, 126]       */
    HIF8_ERR_SHAPE = 6,       /* negative or unsupported extent / leading dimension */
    HIF8_ERR_ALIGN = 7,       /* GEMM operand not 16-byte aligned                   */
    HIF8_ERR_WORKSPACE = 8,   /* workspace missing or too small                     */
    HIF8_ERR_CUDA = 9,        /* a CUDA call failed (launch error, wrong device)    */
    HIF8_ERR_DEVICE_TIMEOUT = 10, /* a bounded device-side wait gave up            */
    HIF8_ERR_OVERLAP = 11     /* source and destination share bytes (Section 3: a conversion reads one tensor and
                                 writes another; only hif8_fake_quant may run in place, dst == src exactly)   */
};

/* which call a workspace size is asked for */
enum { HIF8_WS_AMAX_SCALE_ENCODE = 0, HIF8_WS_FAKE_QUANT = 1, HIF8_WS_GEMM = 2 };

/*
 * High-precision tensor -> HiF8 bytes (Section 3: rounding of FP32 / FP16 / BF16 data into the format).
 *   dst[i] = To_HiF8_<rnd>( src[i] * 2^scale_exp )
 * The scaled value is rounded as if 1.5*2^15 were representable; a result of that magnitude or more is
 * +-Inf (or +-2^15 with HIF8_FLAG_SATURATE).  Magnitudes that round to zero give 0x00 for either sign.
 * src: n elements of `src_dtype`; dst: n bytes; they must not overlap (HIF8_ERR_OVERLAP).  `seed` is used by HIF8_RND_SR only:
 * element i takes word (i mod 4) of Philox4x32-10 with counter (i/4, 0, 0) and key `seed`; its top 24 bits
 * (FP32 source) or 16 bits (16-bit sources) are the threshold T of Section 3.2.
 */
int hif8_encode(const void* src, int src_dtype, uint8_t* dst, size_t n, int scale_exp, int rnd,
                unsigned flags, uint64_t seed, hif8_stream_t stream);

/*
 * hif8_encode of a source that is generated instead of read: element i is the FP32 value whose encoding is
 * first_pattern + i (modulo 2^32), i = 0 .. n-1, n <= 2^32.  This is the exhaustive sweep over FP32 inputs (every
 * exponent including the denormal extension of Eq. 2, underflow to the single zero, overflow, Inf and NaN patterns of
 * Section 2.1 / Table 4) without a 4-byte-per-element source tensor: the call only writes, one byte per element.
 * HIF8_RND_SR draws the word of index i.  Arguments and errors otherwise as hif8_encode.
 */
int hif8_encode_f32_patterns(uint32_t first_pattern, uint8_t* dst, size_t n, int scale_exp, int rnd, unsigned flags,
                             uint64_t seed, hif8_stream_t stream);

/*
 * HiF8 bytes -> high-precision tensor (Eq. 1, Eq. 2, Table 4 specials), with the descale of
 * Algorithm 1 ("Restore"):   dst[i] = value(src[i]) * 2^(-scale_exp)
 * rounded to nearest-even into `dst_dtype` when not representable (only possible at the far ends of the
 * scale range, or for FP16 destinations).  0x80 gives the canonical quiet NaN, 0x6F / 0xEF give +-Inf.
 * src: n bytes; dst: n elements; no overlap (HIF8_ERR_OVERLAP).
 */
int hif8_decode(const uint8_t* src, void* dst, int dst_dtype, size_t n, int scale_exp,
                hif8_stream_t stream);

/*
 * Per-tensor scaled conversion (Section 5.1 "Per-Tensor Scaling"; Algorithm 1 "Scale & Cast").
 *   d_scale_exp_in == NULL  (just-in-time):  amax = max |src[i]| over finite elements;
 *        scale_exp = clamp(target_exp - floor(log2 amax), -126, 126)  (0 if amax is 0), so that
 *        amax * 2^scale_exp lies in [2^target_exp, 2^(target_exp+1)); then dst = To_HiF8(src * 2^scale_exp).
 *        One to three kernels, by size and alignment; the scale never leaves the device.
 *   d_scale_exp_in != NULL  (delayed scaling: Section 5.1 measures amax once per ten iterations): the scale exponent
 *        is read from that device int; amax of this tensor is still produced for the next update.  One pass.
 * Outputs (device scalars, each may be NULL): d_amax_out (float, exact), d_scale_exp_out (int, the exponent
 * used), d_scale_out (float 2^scale_exp).  workspace: hif8_workspace_bytes(HIF8_WS_AMAX_SCALE_ENCODE, n)
 * bytes of device memory, 256-byte aligned, contents irrelevant on entry and undefined on return.
 * target_exp in [-22, 15]; 14 keeps amax just below the largest finite value 2^15.
 */
int hif8_amax_scale_encode(const void* src, int src_dtype, uint8_t* dst, size_t n, int target_exp, int rnd,
                           unsigned flags, uint64_t seed, const int* d_scale_exp_in, float* d_amax_out,
                           int* d_scale_exp_out, float* d_scale_out, void* workspace,
                           size_t workspace_bytes, hif8_stream_t stream);

/*
 * Amax alone (Section 5.1, per-tensor scaling: the largest magnitude of each GEMM input tensor is measured at a fixed
 * cadence of iterations and the tensor's scale follows from it):
 *   *d_amax_out = max |src[i]| over the finite elements (0 if there is none), as an exact float.
 * One read of the tensor.  workspace as for hif8_amax_scale_encode.  The caller derives the next scale exponent
 * from it (or lets hif8_amax_scale_encode do both in one call).
 */
int hif8_amax(const void* src, int src_dtype, size_t n, float* d_amax_out, void* workspace, size_t workspace_bytes,
              hif8_stream_t stream);

/*
 * The second half of the just-in-time form on its own: the scale exponent is derived on the device from an amax the
 * caller already has in device memory, scale_exp = clamp(target_exp - floor(log2 *d_amax), -126, 126) (0 if it is 0),
 * then dst = To_HiF8_<rnd>(src * 2^scale_exp).  *d_amax must be a non-negative float.  Together with hif8_amax this
 * splits hif8_amax_scale_encode where a tensor is sharded over several GPUs: each rank reduces its shard, the ranks
 * combine the 4-byte values with a max all-reduce, and each converts its shard with the common exponent (Section 5.1:
 * one scale factor per GEMM input tensor).  Optional outputs as in hif8_amax_scale_encode.  No workspace.
 */
int hif8_encode_from_amax(const void* src, int src_dtype, uint8_t* dst, size_t n, int target_exp, int rnd, unsigned flags,
                          uint64_t seed, const float* d_amax, int* d_scale_exp_out, float* d_scale_out,
                          hif8_stream_t stream);

/*
 * hif8_amax_scale_encode without a caller-supplied workspace.  (The paper has no counterpart: this entry
 * point exists for the benefit of the calling environment only.)
 *
 * Who needs it: code that must not, or cannot, obtain device memory at the point of the call -- a plug-in that
 * runs inside another framework's memory pool and may not allocate behind its back, a call site inside a
 * real-time or fault-handling path where cudaMalloc's implicit synchronisation and possible failure are not
 * acceptable, or a process whose memory budget was handed out completely at start-up.  Such callers still pass
 * their input and output tensors; the few bytes of scratch the amax reduction needs come from a
 * HIF8_STATIC_SCRATCH_BYTES-byte array inside the library image, resident on every device that loads the
 * library until the process exits.
 *
 * Same arguments, results and errors as hif8_amax_scale_encode minus the workspace pair, plus:
 *   - n > HIF8_STATIC_MAX_ELEMENTS is rejected with HIF8_ERR_SHAPE before anything is launched.
 *   - No cudaMalloc / cudaFree / allocating library routine is called, now or later.
 *   - The first call on each device looks up the array's device address (cudaGetSymbolAddress); make that
 *     first call outside any stream capture.
 *   - All calls on a device share the one array.  A call may overwrite all of it and writes what it reads there
 *     itself first, on `stream`, so back-to-back calls on one stream are safe; two calls that can overlap on the GPU
 *     (different streams, no dependency) race on it and give wrong scales -- serialise them, or use
 *     hif8_amax_scale_encode with separate workspaces.
 */
#define HIF8_STATIC_SCRATCH_BYTES 256
#define HIF8_STATIC_MAX_ELEMENTS ((size_t)1 << 32)
int hif8_amax_scale_encode_static(const void* src, int src_dtype, uint8_t* dst, size_t n, int target_exp, int rnd,
                                  unsigned flags, uint64_t seed, const int* d_scale_exp_in, float* d_amax_out,
                                  int* d_scale_exp_out, float* d_scale_out, hif8_stream_t stream);

/*
 * Per-channel scaled conversion of a weight matrix (Section 4.2 and the closing remarks of Section 5 and Section 6 name
 * the combination of one scale per activation tensor with one scale per weight channel).  W is [rows, cols] row-major and
 * contiguous; every output channel has its own power-of-two scale:
 *   channel_axis = 0: channel = row    (weights stored [N,K]);   channel_axis = 1: channel = column (stored [K,N]).
 *   d_scale_exp_in == NULL: per channel, amax over the channel's finite elements and
 *        scale_exp = clamp(target_exp - floor(log2 amax), -126, 126) (0 for an all-zero channel), the per-tensor rule
 *        of hif8_amax_scale_encode applied to the channel alone; d_amax [channels] receives the amax values (it is also
 *        the accumulator of the reduction and must not be NULL).
 *   d_scale_exp_in != NULL: the exponents are read from that device array [channels]; d_amax is not touched.
 *   dst[r, c] = To_HiF8_<rnd>( W[r, c] * 2^scale_exp[channel(r, c)] ), same layout as W, one byte per element.
 * d_scale_exp_out [channels] (may be NULL; may equal d_scale_exp_in): the exponents used, ready for
 * hif8_gemm_channel_scaled.  HIF8_RND_SR draws the word of flat index r * cols + c, as hif8_encode would.
 * Needs no workspace.  The fast path wants 16-byte aligned pointers and rows (cols * element size a multiple of 16);
 * anything else takes a slower element-wise path with identical results.
 */
int hif8_channel_amax_scale_encode(const void* W, int src_dtype, uint8_t* dst, int64_t rows, int64_t cols,
                                   int channel_axis, int target_exp, int rnd, unsigned flags, uint64_t seed,
                                   const int* d_scale_exp_in, float* d_amax, int* d_scale_exp_out,
                                   hif8_stream_t stream);

/*
 * The every-N-iterations cadence of per-tensor scaling in training (Section 5.1: scale factors start at 1; once per ten
 * iterations the amax of each tensor is measured and its scale updated; the scale in force is applied in every
 * iteration, updated or not).  The paper does not give the update rule; this library keeps, per tensor, the exponent
 * in force and a ring of the last `hist_len` measured amax values, and after a measurement sets
 *   scale_exp = clamp(target_exp - floor(log2 max(ring)), -126, 126)      (0 while every entry is 0)
 * which takes effect from the next conversion on.  The state lives in HIF8_SCALE_STATE_BYTES of device memory
 * (256-byte aligned) owned by the caller; nothing returns to the host.
 *   hif8_scale_state_init:      exponent 0, empty ring of hist_len entries (1..HIF8_SCALE_HISTORY_MAX).
 *   hif8_delayed_scale_encode:  dst = To_HiF8_<rnd>(src * 2^(exponent in force)) in one pass over src.  With
 *        measure != 0 (the caller's "iteration % N == 0") the same pass also reduces amax of src, and the last
 *        thread block to finish pushes it into the ring and updates the exponent (one kernel launch either way).  The first int of the state is the exponent
 *        in force (readable as the d_scale_exp_a / d_scale_exp_w of hif8_gemm), the float at byte 16 the last amax.
 */
#define HIF8_SCALE_STATE_BYTES 1024
#define HIF8_SCALE_HISTORY_MAX 32
int hif8_scale_state_init(void* d_state, int hist_len, hif8_stream_t stream);
int hif8_delayed_scale_encode(const void* src, int src_dtype, uint8_t* dst, size_t n, int rnd, unsigned flags,
                              uint64_t seed, void* d_state, int measure, int target_exp, hif8_stream_t stream);

/*
 * Adaptive loss scaling (Section 5.1, "Adaptive Loss-Scaling (ALS)"), resident on the device.
 * The loss scale is 2^scale_exp.  After each backward pass: hif8_check_finite over the (scaled) gradient tensors ORs
 * "holds an Inf or NaN" into *d_found_inf (a device int the caller zeroes once; hif8_als_update clears it again), then
 * hif8_als_update advances the controller:
 *   overflow          -> scale / 2, clean-iteration count = 0
 *   no overflow       -> count + 1; when it reaches the scale window -> scale * 2, count = 0
 *   scale window      : walks the list {1, 20, 50, 100, 200, 500, 1000}: three increases of the scale since the last
 *                       window change move it up one entry; three decreases not interrupted by an increase move it
 *                       down one entry; a window change clears both counts; it stops at the ends of the list.
 * The paper starts from scale 2^32 and window 20 (init_scale_exp = 32, init_window_index = 1).
 * State: HIF8_ALS_STATE_BYTES of device memory, 16-byte aligned, eight ints the caller may read at any time:
 *   [0] scale_exp  [1] window  [2] window index  [3] clean iterations  [4] increases counted  [5] decreases in a row
 *   [6] iterations seen  [7] iterations that overflowed.
 * The optimizer step of an overflowed iteration is the caller's to skip (it can test the flag on the device before
 * hif8_als_update clears it).  Nothing here returns to the host or synchronises.
 */
#define HIF8_ALS_STATE_BYTES 64
int hif8_als_state_init(void* d_state, int init_scale_exp, int init_window_index, hif8_stream_t stream);
int hif8_als_update(void* d_state, int* d_found_inf, hif8_stream_t stream);
/* *d_found_inf |= (some src[i] is +-Inf or NaN); one read of the tensor; src must be aligned to its element size */
int hif8_check_finite(const void* src, int dtype, size_t n, int* d_found_inf, hif8_stream_t stream);

/*
 * Quantize-dequantize in the source format (Section 4: the paper's experiments simulate the format by replacing every
 * value with its nearest HiF8-representable one):   dst[i] = value( To_HiF8_<rnd>(src[i] * 2^e) ) * 2^(-e)   in `dtype`.
 *   use_amax == 0: e = scale_or_target_exp.  No workspace needed (may be NULL).
 *   use_amax == 1: e derived from the tensor's amax with target exponent scale_or_target_exp, as in
 *                  hif8_amax_scale_encode (one to three kernels, by size); workspace as for HIF8_WS_FAKE_QUANT.
 * dst may be the same pointer as src (in place); any other overlap is rejected with HIF8_ERR_OVERLAP.
 * d_amax_out / d_scale_exp_out: optional device scalars as above.
 */
int hif8_fake_quant(const void* src, void* dst, int dtype, size_t n, int use_amax, int scale_or_target_exp,
                    int rnd, unsigned flags, uint64_t seed, float* d_amax_out, int* d_scale_exp_out,
                    void* workspace, size_t workspace_bytes, hif8_stream_t stream);

/*
 * GEMM with HiF8 operands decoded in-kernel (Algorithm 1, "MatMul & Restore"; Section 4.1: only the GEMM
 * inputs are HiF8):   C[m,n] = 2^-(sa+sw) * sum_k value(Aq[m,k]) * value(Wq[k,n])
 * Decoded values are exact in BF16; products are accumulated in FP32 on the tensor cores.
 *   Aq: [M,K] row-major bytes, leading dimension lda.  Wq: [K,N] (w_is_nk = 0) or [N,K] (w_is_nk = 1)
 *   row-major bytes, leading dimension ldw.  C: [M,N] row-major, `c_dtype` HIF8_BF16 or HIF8_F32, ldc.
 *   d_scale_exp_a / d_scale_exp_w: device ints sa, sw (NULL = 0).
 * Pointers and leading dimensions (in bytes) must be multiples of 16 (HIF8_ERR_ALIGN); K must be a positive
 * multiple of 16 (HIF8_ERR_SHAPE).  NaN / Inf codes propagate as in IEEE arithmetic.
 * workspace: at least hif8_workspace_bytes(HIF8_WS_GEMM, 0) = 256 bytes, 16-byte aligned; its first int is a device
 * status word that the call clears and the kernel sets if one of its bounded waits ever gives up (see
 * hif8_gemm_status).  With only that, the kernels decode both byte operands themselves.
 * With hif8_workspace_bytes(HIF8_WS_GEMM, M*K + K*N) bytes, 256-byte aligned, and contiguous operands (lda = K,
 * ldw = row length of Wq), each operand byte is instead decoded once into the workspace (BF16, exact) and the
 * tensor-core kernel streams BF16 tiles: several times faster for compute-bound shapes, same results.
 * In between -- hif8_workspace_bytes(HIF8_WS_GEMM, M*K) bytes or more, 256-byte aligned, A contiguous -- A alone is
 * expanded into the workspace and the kernel decodes only the W tiles (any ldw): for when the weight's BF16 copy does
 * not fit but the activation's does; same results.  A workspace with room for both operands takes this form too while
 * the product is too small to win the pass over W back (see hif8_gemm_path_policy).
 * Products of few rows and a small weight take one launch in which every warp decodes its share of both operands, whatever
 * the workspace.  Others with at most 64 rows of A (and A given as [M,K]) take a weight-streaming kernel; with the workspace
 * size above it first expands the few rows of A to BF16 there (one small launch more, A contiguous).  Products of few tiles
 * take A as bytes even when the workspace has room for it, where that is faster.
 * Where several SMs share the sum of an output (K split among them), the parts are added in a fixed order: results are
 * reproducible run to run; how K is split depends on the sizes, the device and the workspace.
 */
int hif8_gemm(const uint8_t* Aq, int64_t lda, const uint8_t* Wq, int64_t ldw, int w_is_nk, void* C,
              int64_t ldc, int c_dtype, int M, int N, int K, const int* d_scale_exp_a,
              const int* d_scale_exp_w, void* workspace, size_t workspace_bytes, hif8_stream_t stream);

/*
 * hif8_gemm with one weight exponent per output channel (per-tensor activation scale, per-channel weight scales):
 *   C[m,n] = 2^-(sa + sw[n]) * sum_k value(Aq[m,k]) * value(Wq[k,n]),   d_scale_exp_w_channel: device int [N], not NULL.
 * Everything else as hif8_gemm.
 */
int hif8_gemm_channel_scaled(const uint8_t* Aq, int64_t lda, const uint8_t* Wq, int64_t ldw, int w_is_nk, void* C,
                             int64_t ldc, int c_dtype, int M, int N, int K, const int* d_scale_exp_a,
                             const int* d_scale_exp_w_channel, void* workspace, size_t workspace_bytes,
                             hif8_stream_t stream);

/*
 * The general form of the HiF8 GEMM, covering the backward pass of Y = X W (Section 3: the activation gradient is
 * converted with TA or hybrid rounding; Section 4.1: activation, weight and activation gradient are the GEMM inputs):
 *   dgrad  dX[M,K'] = dY[M,N'] W^T :  Aq = dYq [M,N'],           Wq = the forward weight bytes [K',N'], w_is_nk = 1
 *   wgrad  dW[K',N'] = X^T dY      :  Aq = Xq [M',K'], a_is_km = 1 (A is read as [K,M] = [M',K']), Wq = dYq [M',N'], w_is_nk = 0
 * so neither backward GEMM needs a transposed copy of a byte tensor.
 *   C[m,n] (+)= 2^-(sa + sw_n) * sum_k value(A(m,k)) * value(W(k,n))
 *   a_is_km = 0: Aq is [M,K] row-major (lda >= K);  a_is_km = 1: Aq is [K,M] row-major (lda >= M).
 *   w_is_nk as in hif8_gemm.  sw_n = d_scale_exp_w_channel[n] if that pointer is given, else *d_scale_exp_w (or 0).
 *   accumulate != 0: the product is added to the existing contents of C (FP32 C: one rounding per element per call;
 *   BF16 C: sum formed in FP32, then rounded to nearest even) -- gradient accumulation over micro-batches.
 * Alignment, K, workspace and status conventions as in hif8_gemm (the decode-once path needs contiguous operands).
 */
int hif8_gemm_ex(const uint8_t* Aq, int64_t lda, int a_is_km, const uint8_t* Wq, int64_t ldw, int w_is_nk, void* C,
                 int64_t ldc, int c_dtype, int M, int N, int K, const int* d_scale_exp_a, const int* d_scale_exp_w,
                 const int* d_scale_exp_w_channel, int accumulate, void* workspace, size_t workspace_bytes,
                 hif8_stream_t stream);

/*
 * Conversion with transposed store: dst[c, r] = To_HiF8_<rnd>( src[r, c] * 2^e ), src [rows, cols] row-major of
 * `src_dtype`, dst [cols, rows] bytes.  For frameworks that keep a second, transposed byte copy of a GEMM operand
 * (the backward GEMMs contract over the other dimension); hif8_gemm_ex does not need it.
 *   e = *d_scale_exp if that device pointer is given (delayed scaling), else scale_exp.
 *   HIF8_RND_SR draws the word of the SOURCE flat index r * cols + c, so the codes equal those of hif8_encode, moved.
 * The fast path wants 16-byte aligned pointers, cols a multiple of the 16-byte vector (4 FP32 / 8 16-bit elements) and
 * rows a multiple of 16; anything else takes an element-wise path with identical results.
 */
int hif8_encode_transpose(const void* src, int src_dtype, uint8_t* dst, int64_t rows, int64_t cols, int scale_exp,
                          const int* d_scale_exp, int rnd, unsigned flags, uint64_t seed, hif8_stream_t stream);

/*
 * Host-side query of the status word of a finished hif8_gemm: copies it from `workspace`, SYNCHRONISES `stream`,
 * and returns HIF8_OK or HIF8_ERR_DEVICE_TIMEOUT (the output tile of the CTA that gave up is then undefined).
 * The only entry point that blocks the host.
 */
int hif8_gemm_status(const void* workspace, hif8_stream_t stream);

/*
 * Which kernel takes a product.  HIF8_GEMM_PATH_AUTO (the default): the one that is expected to be fastest, by the sizes, the
 * layouts and what the workspace has room for; with room for both operands W is expanded too only when the product is large
 * enough to win that pass back.  The other settings are for measurements and tests of one kernel on products that another
 * one would take:
 *   HIF8_GEMM_PATH_EXPAND_BOTH  both operands expanded whenever the workspace has room
 *   HIF8_GEMM_PATH_EXPAND_A     A expanded whenever the workspace has room, W decoded in the kernel
 *   HIF8_GEMM_PATH_NO_WARP      as AUTO, without the kernel for few rows and a small weight (nor do the two above take it)
 *   HIF8_GEMM_PATH_WARP         that kernel; HIF8_ERR_SHAPE for a product that it cannot take (K too long for its registers, far
 *                               too large a product, [K,N] weights with N no multiple of four)
 * Products of block-scaled operands (hif8_gemm_block) go by the same setting where the kernel can take them and the workspace has room, and are not refused otherwise.
 * Up to 64 rows of A given as [M,K] take the weight-streaming kernel under the first three.  Process-wide; returns the
 * previous setting, or HIF8_ERR_FLAGS (4, which is no setting) for an unknown one.  What it computes does not depend on it,
 * only the order of the FP32 sums does.
 */
enum {
    HIF8_GEMM_PATH_AUTO = 0, HIF8_GEMM_PATH_EXPAND_BOTH = 1, HIF8_GEMM_PATH_NO_WARP = 2, HIF8_GEMM_PATH_EXPAND_A = 3,
    HIF8_GEMM_PATH_WARP = 5
};
int hif8_gemm_path_policy(int policy);

/*
 * Status of the most recent GEMM-class call (hif8_gemm, hif8_gemm_ex, hif8_gemm_channel_scaled, hif8_pts_search,
 * hif8_selftest_wait_timeout) enqueued on `stream` of the current device, without the caller naming the workspace:
 * the library remembers, per stream, where that call's status word lives.  SYNCHRONISES `stream`, then returns HIF8_OK,
 * HIF8_ERR_DEVICE_TIMEOUT, or HIF8_ERR_CUDA (read failed, or another device is current).  HIF8_OK when no such call was
 * made on the stream.  The workspace of that call must still be allocated.  (Algorithm 1 has no counterpart; this is
 * the host-side end of the bounded device-side waits.)
 */
int hif8_last_device_status(hif8_stream_t stream);

/*
 * Self-test of the host-side caches (no device needed): the once-per-device set-up record and the tensor-map cache are
 * driven with synthetic keys; returns HIF8_OK, or HIF8_ERR_SHAPE with the number of the failed check in *failed_check.
 */
int hif8_selftest_host_caches(int* failed_check);

/*
 * Self-test of the device-side failure detection: launches one warp that waits, with a limit of `limit_ms`
 * milliseconds (1..1000), on a barrier that is never completed.  The wait gives up, the kernel records the status
 * word in `workspace` (first int, cleared by the call) and ends normally; hif8_gemm_status(workspace, stream) then
 * returns HIF8_ERR_DEVICE_TIMEOUT and the device stays usable.  No fault, trap or unbounded loop is involved.
 */
int hif8_selftest_wait_timeout(void* workspace, unsigned limit_ms, hif8_stream_t stream);

/*
 * Per-layer search of Algorithm 1 ("HiF8 Calibration with Per-Tensor Scaling"): for every (Ea, Ew) with both
 * exponents in [e_min, e_max] (the paper searches [-4, 5]):
 *     A_q = To_HiF8_TA(A * 2^Ea), W_q = To_HiF8_TA(W * 2^Ew);  O_q = (A_q x W_q) * 2^-(Ea+Ew);
 *     d_err[(Ea - e_min) * n + (Ew - e_min)] = MSE(O_q, O_ref) over all M*N outputs      (n = e_max - e_min + 1 <= 16)
 * and d_best[0], d_best[1] = the (Ea, Ew) of the smallest error (first one in that order on exact ties).
 * A: [M,K] row-major; W: [K,N] (w_is_nk = 0) or [N,K]; both contiguous, of `dtype`; O_ref: the layer's high-precision
 * output [M,N] as float, leading dimension ldo.  K and the row length of W must be multiples of 16.
 * All device memory; 2n encodes, n*n GEMMs with FP32 output and n*n reductions are enqueued on `stream`, nothing
 * returns to the host.  workspace: hif8_pts_workspace_bytes(M, N, K, n) bytes, 256-byte aligned; its first int is a
 * device status word as for hif8_gemm (hif8_pts_status reads it, synchronising the stream).
 */
int hif8_pts_search(const void* A, const void* W, int dtype, int w_is_nk, const float* O_ref, int64_t ldo, int M, int N,
                    int K, int e_min, int e_max, float* d_err, int* d_best, void* workspace, size_t workspace_bytes,
                    hif8_stream_t stream);
size_t hif8_pts_workspace_bytes(int M, int N, int K, int n_exp);
int hif8_pts_status(const void* workspace, hif8_stream_t stream);

/*
 * Key/value cache in HiF8, paged.  (Section 4.1 keeps to GEMM inputs; the keys and values of attention are the other tensors of
 * inference that are read again and again, here with one power-of-two scale for each block of tokens and head.)
 *
 * A cache is device memory of the caller's:
 *   k_pages, v_pages  [n_pages][kv_heads][page_tokens][head_dim] bytes, 16-byte aligned
 *   k_exp, v_exp      [n_pages][kv_heads] ints: the scale exponent e of each block (one page's tokens of one head); a code stands for
 *                     value(code) * 2^-e.  Exponents are taken within [-HIF8_CACHE_EXP_MAX, HIF8_CACHE_EXP_MAX].
 *   page_table        ints, row s (of table_stride entries) lists the pages of sequence s in order: token t lies in slot t % page_tokens
 *                     of page page_table[s * table_stride + t / page_tokens].
 * page_tokens: 16, 32, 64 or 128; head_dim: 64, 128 or 256; kv_heads: 1 .. HIF8_CACHE_MAX_HEADS; up to HIF8_CACHE_MAX_SEQS sequences a call
 * (HIF8_ERR_SHAPE otherwise).  Lengths are taken within what a row can name (table_stride * page_tokens tokens, at most 2^30) and starts within the
 * number of tokens given.  An entry that is no page number (negative, n_pages or more) names no page: its tokens are not written, not
 * attended to, and read back as zeros.  Sequences may share pages that no call of append writes to.
 * A ragged batch of tokens (new ones, queries, ones to read) lies sequence by sequence; d_*_start [n_seqs + 1] says where each begins,
 * in ascending order, and the last entry where the last one ends.  Tokens and heads of such a batch are token_stride and head_stride elements
 * apart, those of a head contiguous.  What a call writes must not overlap what else it writes or reads (HIF8_ERR_OVERLAP); rows of K and of V may be slices of one tensor.  16-byte aligned pointers and strides take the vectorised path, others a slower one with identical results.
 */
#define HIF8_CACHE_MAX_SEQS 2048
#define HIF8_CACHE_MAX_HEADS 128
#define HIF8_CACHE_MAX_GROUP 64
#define HIF8_CACHE_EXP_MAX 48

/*
 * New tokens into the cache: those of sequence s take the positions from d_lengths[s] (the tokens it has) on.
 *   A block whose first slot is written by the call gets its exponent from the largest finite magnitude among the tokens of the call that it
 *   receives: clamp(target_exp - floor(log2 amax)), 0 for zeros.  A block that has tokens keeps its exponent.  target_exp in [-22, 15]: 3 puts the values
 *   from amax down to amax / 128 where the format has three mantissa bits, and leaves later tokens of the block 2^12 times that before they overflow.
 *   code = To_HiF8_<rnd>(x * 2^e), rnd one of HIF8_RND_TA, _HR, _SSR, _TE (HIF8_ERR_ROUND for _SR: what a cache holds does not depend on draws).
 * k, v: [n_new tokens][kv_heads][head_dim] of src_dtype.  The pages and exponents of the tokens are written, nothing else; d_lengths stays as it is.
 * No page may receive tokens of two sequences, or of two places of a row, of the same call.
 */
int hif8_cache_append(const void* k, const void* v, int src_dtype, int64_t token_stride, int64_t head_stride, const int* d_new_start,
                      const int* d_lengths, int n_seqs, int n_new, uint8_t* k_pages, uint8_t* v_pages, int* k_exp, int* v_exp, int n_pages,
                      int kv_heads, int page_tokens, int head_dim, const int* page_table, int64_t table_stride, int target_exp, int rnd,
                      unsigned flags, hif8_stream_t stream);

/*
 * Tokens out of the cache: those of sequence s from position d_first[s] on, d_out_start[s + 1] - d_out_start[s] of them, as
 * value(code) * 2^-e rounded to nearest-even in dst_dtype, to k, v [n_out tokens][kv_heads][head_dim] (rows must not share elements: HIF8_ERR_SHAPE, those of
 * k with those of v: HIF8_ERR_OVERLAP).
 */
int hif8_cache_read(const uint8_t* k_pages, const uint8_t* v_pages, const int* k_exp, const int* v_exp, int n_pages, int kv_heads,
                    int page_tokens, int head_dim, const int* page_table, int64_t table_stride, const int* d_first, const int* d_out_start,
                    int n_seqs, int n_out, void* k, void* v, int dst_dtype, int64_t token_stride, int64_t head_stride, hif8_stream_t stream);

/*
 * Attention of queries over the cache: q [n_q queries][heads][head_dim] of `dtype` (HIF8_BF16 or HIF8_F16), out likewise, lse [n_q][heads] floats or NULL.
 * Query head h looks at key head h / (heads / kv_heads); heads is a multiple of kv_heads, up to HIF8_CACHE_MAX_GROUP times as many (HIF8_ERR_SHAPE).
 *   s_ij = softmax_scale * sum_d q_i[d] k_j[d],  out_i = sum_j softmax_j(s_ij) v_j,  lse_i = ln sum_j exp(s_ij)
 * d_lengths[s]: tokens of sequence s in the cache, those of its own queries among them (append first).  The n queries of a sequence stand at its last n
 * positions: query i at p_i = d_lengths[s] - n + i.  It looks at the cached tokens j
 *   causal != 0: j <= p_i;  causal == 0: all;   window > 0: only j > p_i - window (window == 0: no such limit).
 * A query that sees no token (an empty cache, with causal a position below 0) gives zeros and lse = -Inf, and so does one whose scores are all -Inf.  Tokens that a query does not see never
 * reach its result, Inf and NaN among them, nor do slots behind a sequence's length.  Inf and NaN of queries and keys propagate through the scores as
 * in IEEE arithmetic.  Inf and NaN among the values that a query sees reach that element of its result whatever the tokens' weights are (also none): Inf of its sign, NaN of a NaN or of both signs.
 * Products of codes are exact and sums are FP32; the weights of the softmax are rounded to FP16 as they multiply codes: w_j = exp(s_ij) 2^-e, e the exponent of the
 * block of v_j (of 16 tokens whose values are all zero: HIF8_CACHE_EXP_MAX).  Down to 2^-18 of the largest w_j that a query sees they have 11 bits, below that
 * steps of 2^-28 of it (fewer than 64 query rows of a key head: 2^-22, 2^-32): where blocks of very different exponents meet, elements in which the larger one is zero have fewer bits.
 * softmax_scale: positive and finite (HIF8_ERR_SCALE_RANGE).
 * The pool must have a page and less than 2^31 rows (n_pages * kv_heads * page_tokens), and n_q * heads / kv_heads must stay below 2^30 (HIF8_ERR_SHAPE).
 * One of two kernels takes all sequences of a call, chosen by max_q * heads / kv_heads: single tokens beside a chunk of 64 query rows of a key head or more are better a call of
 * their own (64 of up to 4096 tokens and a chunk of 512, 32/8 heads of 128: 422 us and 1.1 GB of workspace in one call, 76 + 67 us and 62 MB in two).
 * max_q and max_length: upper bounds of a sequence's queries and tokens, known to the host.  They have to hold (where they do not, results may be wrong, but no
 * memory beside the arguments' is touched).
 * workspace: hif8_cache_attention_workspace_bytes(...) bytes of the same arguments, 256-byte aligned, contents irrelevant on entry and
 * undefined on return, for one call at a time (two captured graphs that may run at the same time need one each).  Its first int is a device status word as for hif8_gemm
 * (hif8_gemm_status, hif8_last_device_status).  From 64 query rows of a key head on (max_q * heads / kv_heads) the size has room for FP16 tiles of what is looked
 * at, up to 16 GiB; a smaller workspace, down to the size for max_q = 1, gives results within the same bounds more slowly.  Where the sum over a sequence's tokens is shared, the parts are added in a fixed order: results are reproducible.
 */
int hif8_cache_attention(const void* q, int dtype, int64_t q_token_stride, int64_t q_head_stride, const int* d_q_start, const int* d_lengths,
                         int n_seqs, int n_q, int max_q, int max_length, const uint8_t* k_pages, const uint8_t* v_pages, const int* k_exp,
                         const int* v_exp, int n_pages, int kv_heads, int page_tokens, int head_dim, const int* page_table, int64_t table_stride,
                         int heads, float softmax_scale, int causal, int window, void* out, int64_t out_token_stride, int64_t out_head_stride,
                         float* lse, void* workspace, size_t workspace_bytes, hif8_stream_t stream);
size_t hif8_cache_attention_workspace_bytes(int n_seqs, int n_q, int max_q, int max_length, int heads, int kv_heads, int head_dim);

/*
 * Sequences that continue from others' pages (beam search, several samples of a prompt): row i of table_out (n_children rows, table_out_stride entries
 * apart) becomes row d_parent[i] of page_table as far as that sequence has tokens, -1 behind, and d_lengths_out[i] its length.  Where the last page is
 * partly filled and d_new_page[i] is a page, its contents and exponents are copied there and the child's row names the copy; full pages are shared, and so
 * is the last one where d_new_page[i] is none (or d_new_page NULL): for the child that keeps it.  Of children that name the same new page the first gets it.
 * New pages must be free: no page of a row.  (The rows go to a table of their own so that any child may continue any parent.)  A parent that is none (outside 0 .. n_seqs - 1) gives an empty child.  A length beyond table_out_stride pages is cut there.
 */
int hif8_cache_fork(uint8_t* k_pages, uint8_t* v_pages, int* k_exp, int* v_exp, int n_pages, int kv_heads, int page_tokens, int head_dim,
                    const int* page_table, int64_t table_stride, const int* d_lengths, int n_seqs, const int* d_parent, const int* d_new_page,
                    int n_children, int* table_out, int64_t table_out_stride, int* d_lengths_out, hif8_stream_t stream);

/*
 * The pages in use, and the others.  A page is live when a row names it within its sequence's length (a sequence is freed by setting its length to 0; a
 * page that several rows name is live until the last of them goes).  *d_n_live: the number of live pages.
 *   move != 0: live pages with numbers from *d_n_live on move (contents and exponents) to the free ones below, the lowest to the lowest, and the rows name their
 *              new places; pages 0 .. *d_n_live - 1 are then the live ones.  Contents of pages left behind stay as they are.
 *   move == 0: nothing moves.
 * d_free_pages [n_pages]: the free pages (after the move) in ascending order, -1 behind them.
 * workspace: hif8_cache_compact_workspace_bytes(n_pages) bytes, 256-byte aligned, contents irrelevant on entry and undefined on return.
 */
int hif8_cache_compact(uint8_t* k_pages, uint8_t* v_pages, int* k_exp, int* v_exp, int n_pages, int kv_heads, int page_tokens, int head_dim,
                       int* page_table, int64_t table_stride, const int* d_lengths, int n_seqs, int move, int* d_n_live, int* d_free_pages,
                       void* workspace, size_t workspace_bytes, hif8_stream_t stream);
size_t hif8_cache_compact_workspace_bytes(int n_pages);


/*
 * Block-scaled matrices: one power-of-two scale for each block of 128 (the finest of the scalings that Sections 5 and 6 name is a channel's).
 *
 * A matrix [rows, cols] of codes, rows ld bytes apart, has an exponent e for each block of block_rows x HIF8_BLOCK elements (block_rows 1, for activations
 * and their gradients, or HIF8_BLOCK, for weights): d_exp[(r / block_rows) * exp_stride + c / HIF8_BLOCK], exp_stride >= ceil(cols / HIF8_BLOCK).  A code
 * stands for value(code) * 2^-e.  Exponents lie, and are taken, within [-HIF8_BLOCK_EXP_MAX, HIF8_BLOCK_EXP_MAX]: within them what a code stands for is exact in BF16.
 * Matrices of values have rows ld elements apart.  Rows must not overlap one another, nor what a call writes anything else that it writes or reads
 * (HIF8_ERR_OVERLAP) but for what a call names.  Pointers are aligned to their elements (HIF8_ERR_ALIGN); rows on 16-byte boundaries (of codes: 8) take the vectorised path, others a slower one with identical
 * results but for the order in which a norm adds its row (see hif8_rmsnorm_encode).  Each call says how large a matrix may be (HIF8_ERR_SHAPE beyond).
 */
#define HIF8_BLOCK 128
#define HIF8_BLOCK_EXP_MAX 96

/*
 * Values -> block-scaled codes, one pass:
 *   e = clamp(target_exp - floor(log2 amax)) with the block's largest finite magnitude, 0 for zeros;  dst = To_HiF8_<rnd>(src * 2^e)
 * target_exp in [-22, 15]: 3 puts what lies from amax down to amax / 128 where the format has three mantissa bits.
 * HIF8_RND_SR draws the word of index r * cols + c, as hif8_encode does.  At most 2^31 - 1 blocks.
 */
int hif8_block_encode(const void* src, int src_dtype, int64_t ld_src, int64_t rows, int64_t cols, int block_rows, uint8_t* dst, int64_t ld_dst, int* d_exp,
                      int64_t exp_stride, int target_exp, int rnd, unsigned flags, uint64_t seed, hif8_stream_t stream);

/* Block-scaled codes -> values: value(src) * 2^-e, rounded to nearest-even in dst_dtype (only FP16 needs it).  At most 2^31 - 1 groups of sixteen columns (rows * ceil(cols / 16)). */
int hif8_block_decode(const uint8_t* src, int64_t ld_src, const int* d_exp, int64_t exp_stride, int64_t rows, int64_t cols, int block_rows, void* dst, int dst_dtype,
                      int64_t ld_dst, hif8_stream_t stream);

/*
 * Root-mean-square norm with the residual's addition, its result in block-scaled codes (blocks of 1 x 128): what stands in front of a product.
 *   h = x + residual, rounded to dtype (residual NULL: h = x);  r = 1 / sqrt(mean_c h^2 + eps);  dst, d_exp = the codes of h * r * weight (see hif8_block_encode)
 * x, residual, h (may be NULL; may be x or residual itself, with the same ld) [rows, cols], weight [cols]: all of `dtype`.  d_rstd [rows] (may be NULL): r, for the gradient.
 * cols at most HIF8_NORM_MAX_COLS, rows at most 32 * (2^31 - 1) (HIF8_ERR_SHAPE); eps >= 0 and finite (HIF8_ERR_SCALE_RANGE).  Squares are added in FP32, products are FP32 and rounded once, to the codes.
 * The order in which a row's squares are added depends on its alignment and, from 513 to 8192 columns, on whether the call has more than 148 rows: r then differs in its last bits, and a code whose
 * value lies on the border of two.  Within one call all rows are added alike.  A row whose squares add up to more than FP32 holds has r 0; squares below FP32 count as 0.
 * rnd one of HIF8_RND_TA, _HR, _SSR, _TE (HIF8_ERR_ROUND for _SR).  Inf and NaN propagate within their row as in IEEE arithmetic.
 */
#define HIF8_NORM_MAX_COLS 32768
int hif8_rmsnorm_encode(const void* x, int64_t ld_x, const void* residual, int64_t ld_residual, int dtype, const void* weight, float eps, int64_t rows, int64_t cols,
                        void* h, int64_t ld_h, float* d_rstd, uint8_t* dst, int64_t ld_dst, int* d_exp, int64_t exp_stride, int target_exp, int rnd, unsigned flags,
                        hif8_stream_t stream);

/*
 * Its gradient (the rounding to codes passes it on as it is):  with u = h * r
 *   dx = r * (weight * dy - u * mean_c(weight * dy * u)) + dh      the gradient of x and of residual; dh (NULL: 0): that of h from behind
 *   d_weight_grad[c] (+)= sum over rows of dy * u                  FP32, added to what is there when accumulate != 0; NULL: not wanted
 * dy, h, dh, dx [rows, cols] of dtype; dx may be dy or dh itself, with the same ld.  Sums are FP32 in a fixed order: results are reproducible.
 * workspace (for d_weight_grad): hif8_rmsnorm_backward_workspace_bytes(rows, cols) bytes, 256-byte aligned, contents irrelevant on entry and undefined on return, for one call at a time.
 */
int hif8_rmsnorm_backward(const void* dy, int64_t ld_dy, const void* h, int64_t ld_h, const void* dh, int64_t ld_dh, int dtype, const void* weight, const float* d_rstd,
                          int64_t rows, int64_t cols, void* dx, int64_t ld_dx, float* d_weight_grad, int accumulate, void* workspace, size_t workspace_bytes,
                          hif8_stream_t stream);
size_t hif8_rmsnorm_backward_workspace_bytes(int64_t rows, int64_t cols);

/*
 * The product of block-scaled operands, and with it the gradients' products:
 *   C[m,n] (+)= sum_k value(A(m,k)) 2^-ea * value(W(k,n)) 2^-ew
 * Aq is stored [M,K] (a_is_km = 0) or [K,M], Wq [K,N] (w_is_nk = 0) or [N,K]; either operand's blocks (a_block_rows, w_block_rows: 1 or HIF8_BLOCK) lie on the
 * matrix as it is stored, so what one call made of a tensor serves all its products:
 *   forward  Y[T,N'] = X W^T:   A = X [T,K'] (1),  W = [N',K'] (128), w_is_nk = 1
 *   dX[T,K'] = dY W:            A = dY [T,N'] (1), the same W, w_is_nk = 0
 *   dW[N',K'] += dY^T X:        A = dY, a_is_km = 1, W = X [T,K'] (1), w_is_nk = 0, accumulate = 1
 * M, N and K are any numbers from 1 to 2^31 - 4096 (0: nothing is done for M or N, HIF8_ERR_SHAPE for K).  An operand that is expanded in any case has at most 2^30 - 2^20 groups of sixteen
 * columns: weights with scales for each 1 x 128 (as [N,K]: N up to the next multiple of eight), and A but where it is [K,M] beside weights with scales for each 128 x 128 (HIF8_ERR_SHAPE).  All three matrices are 16-byte aligned with rows a multiple of 16 bytes apart (HIF8_ERR_ALIGN).  C [M,N] of HIF8_BF16 or HIF8_F32; what lies
 * behind column N of a row stays as it is.  Products are exact in FP32 unless they leave its range (beyond it Inf, below 2^-126 possibly 0); sums are FP32, in a fixed order.
 * NaN and Inf codes propagate as in IEEE arithmetic.  accumulate as in hif8_gemm_ex.  Which kernel takes a product, and with it the order of its sums, depends on M, N and K.
 * Codes are read in whole pieces of 16 bytes: of the last one of a row the bytes behind its end too, whatever they hold (they have no effect, and lie in the same aligned 16 bytes as the row's end).
 * workspace: hif8_gemm_block_workspace_bytes(...) bytes of the same arguments, 256-byte aligned, contents irrelevant on entry and undefined on return, for one call at a time; its first int is a device status
 * word as for hif8_gemm (hif8_gemm_status, hif8_last_device_status).
 */
int hif8_gemm_block(const uint8_t* Aq, int64_t lda, int a_is_km, const int* d_exp_a, int64_t exp_stride_a, int a_block_rows, const uint8_t* Wq, int64_t ldw,
                    int w_is_nk, const int* d_exp_w, int64_t exp_stride_w, int w_block_rows, void* C, int64_t ldc, int c_dtype, int M, int N, int K, int accumulate,
                    void* workspace, size_t workspace_bytes, hif8_stream_t stream);
size_t hif8_gemm_block_workspace_bytes(int M, int N, int K, int a_is_km, int w_is_nk, int w_block_rows);

/*
 * The global norm of all gradients and clipping, behind a backward pass under a loss scale of 2^s (Section 5.1, ALS):
 *   *d_norm = sqrt(sum g^2) * 2^-s over all elements of all tensors;  dst = g * (2^-s * min(1, max_norm / norm))
 * A list of tensors in device memory: d_src [n_tensors] addresses, d_dst the same for the results (NULL, or equal entries: in place; otherwise no result may overlap a
 * gradient), d_dtype [n_tensors] element formats, d_start [n_tensors + 1] running sums of the tensors' numbers of elements, from 0 to n_elements.  (They have to be right: the library
 * cannot check them.  A tensor of no known format, or at an address that is 0 or not aligned to its elements, is left out.)  No two tensors of the list may
 * overlap.  16-byte aligned addresses take the vectorised path.
 *   d_scale_exp: device int s, the first int of the state of hif8_als_state_init, for instance (NULL: 0);  max_norm > 0, +Inf for no clipping (HIF8_ERR_SCALE_RANGE).
 *   A norm beyond FP32 is stored as +Inf and clipped to all the same.  Gradients that are not all finite: nothing is written to dst, *d_norm = +Inf and *d_found_inf |= 1 (as hif8_check_finite; either pointer may be NULL).
 * Squares are added in FP32 within 16 bytes of a tensor and in FP64 from there on, in a fixed order: results are reproducible, and the norm is within 5 * 2^-24 of the exact one.  The factor is rounded to FP32,
 * its product with g to FP32 too, and for 16-bit tensors once more to their type.  workspace: hif8_grad_clip_workspace_bytes() bytes, 256-byte aligned, for one call at a time.
 */
int hif8_grad_clip(const uint64_t* d_src, const uint64_t* d_dst, const int* d_dtype, const int64_t* d_start, int n_tensors, int64_t n_elements, const int* d_scale_exp,
                   float max_norm, float* d_norm, int* d_found_inf, void* workspace, size_t workspace_bytes, hif8_stream_t stream);
size_t hif8_grad_clip_workspace_bytes(void);

/* bytes of device workspace a call needs (which = HIF8_WS_*; n = element count; for HIF8_WS_GEMM: 0 for the
 * minimum, or M*K + K*N for the decode-once path) */
size_t hif8_workspace_bytes(int which, size_t n);

/* static, NUL-terminated description of a status code */
const char* hif8_status_string(int status);

/*
 * Number of kernels the library has launched from this process since it was loaded (all entry points,
 * all streams).  Host-side counter for tests and benchmarks.
 */
uint64_t hif8_launch_count(void);

#ifdef __cplusplus
}
#endif
#endif /* HIF8_H */
