/*
 * eqat.h - C ABI of the B200 (sm_100a) library for the group-wise low-bit
 * quantised linear layer of EfficientQAT (arXiv 2407.11062).
 *
 * The layer is the one both training phases of the paper run through:
 *   Block-AP (Sec. 3.2): the weight is fake-quantised in the graph,
 *       W_int = clamp(round(W / s) + z, 0, 2^N - 1)          (Eq. 1)
 *       W_hat = (W_int - z) * s                              (Eq. 2)
 *     and W, s, z receive straight-through gradients (appendix "Gradient of
 *     Trainable Parameters in Block-AP", Eqs. 3-5).
 *   E2E-QP (Sec. 3.3): W_int is frozen and stored in N bits, only Eq. 2 runs,
 *     and the step size s is trained with d w_hat / d s = w_q - z.
 *
 * Conventions shared by every entry point
 *   - W is [out_features, in_features] row-major, as in Y = X * W^T.  A
 *     quantisation group is `group` consecutive elements along in_features
 *     inside one row; s and z are [out_features, in_features / group]
 *     row-major.  X is [tokens, in_features], Y and dY are [tokens,
 *     out_features], all row-major and dense (no padding, no strides).
 *   - bf16 / fp16 values are passed as their 16-bit patterns.
 *   - Every tensor pointer is a DEVICE pointer owned by the caller unless its
 *     name starts with `h_` (host).  The library allocates no memory and keeps
 *     no pointer after a call returns.  Device base pointers must be 16-byte
 *     aligned; nothing more is required (where a kernel has a faster path for
 *     32-byte aligned data it picks it from the pointer).
 *   - `stream` is a cudaStream_t passed as void* (NULL = the default stream).
 *     Calls enqueue work on `stream` and return without waiting for it.
 *   - Return value: EQAT_OK, or a negative eqat_status decided on the host
 *     BEFORE anything is launched (outputs untouched), or EQAT_ERR_CUDA if the
 *     runtime rejected a launch.  A kernel that gives up a bounded wait records
 *     it in a device status word read by eqat_device_status().
 *   - Gradients are overwritten, never accumulated.  No bias term (the
 *     quantised layers of the paper have none).
 *   - Tensor contents are not inspected: s <= 0, NaN or Inf give undefined
 *     values (never out-of-bounds accesses).
 *
 * Supported geometry: bits in {2,3,4}; group in {32,64,128,256} or a larger
 * multiple of 32 dividing in_features (e.g. group == in_features, one group
 * per row) for the element-wise and codec entry points; in_features a
 * multiple of 128.  The GEMM entry points also need out_features a multiple
 * of 64; tokens may be any positive number.  The packed-weight GEMMs take
 * group in {32,64,128,256} or group == in_features (channel-wise).
 */
#ifndef EQAT_H_
#define EQAT_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef uint16_t eqat_bf16;   /* bfloat16 bit pattern */
typedef uint16_t eqat_fp16;   /* IEEE binary16 bit pattern */

typedef enum {
  EQAT_OK = 0,
  EQAT_ERR_NULL = -1,         /* a required pointer is NULL                          */
  EQAT_ERR_SHAPE = -2,        /* a size is non-positive or violates a divisibility   */
  EQAT_ERR_ALIGN = -3,        /* a device pointer is not 16-byte aligned             */
  EQAT_ERR_UNSUPPORTED = -4,  /* bits / group / mode outside the supported set       */
  EQAT_ERR_WORKSPACE = -5,    /* workspace missing, misaligned or too small          */
  EQAT_ERR_CUDA = -6,         /* the CUDA runtime or driver reported an error        */
  EQAT_ERR_TIMEOUT = -7       /* a kernel gave up a bounded wait (device status)     */
} eqat_status;

/* Problem descriptor: plain data, read during the call, never retained. */
typedef struct {
  int32_t bits;               /* N: 2, 3 or 4                                         */
  int32_t group;              /* g: elements per quantisation group along in_features */
  int32_t out_features;
  int32_t in_features;
  int64_t tokens;             /* rows of X / dY (ignored by weight-only entry points) */
  int32_t dz_mode;            /* clamped-branch value of d w_hat / d z:
                                 0 = -s (derivative of Eq. 2 at a saturated code),
                                 1 = -1 (Eq. 4 as printed)                            */
  int32_t zero_point_format;  /* how the packed-weight (E2E-QP) entry points read their
                                 zero points: EQAT_ZP_U8 or EQAT_ZP_FP16; must be
                                 EQAT_ZP_U8 (0) for every other entry point           */
} eqat_desc;

/* Zero points of the packed-weight entry points.  EQAT_ZP_U8: one byte per group,
 * the frozen N-bit integers of the hand-off.  EQAT_ZP_FP16: one fp16 value per
 * group, used as it is (not rounded): the variant of Sec. 3.3 that also trains z
 * and therefore keeps it in FP16 (2 + 32/64 = 2.50 bits per weight at w2g64 in
 * the paper's table of E2E-QP variants). */
enum { EQAT_ZP_U8 = 0, EQAT_ZP_FP16 = 1 };

/* Operations that need caller-provided scratch memory (eqat_workspace_bytes). */
enum { EQAT_OP_FAKEQUANT_BWD = 1, EQAT_OP_PACKED_BWD_DS = 2,
       EQAT_OP_PACKED_GATED_FWD = 3, EQAT_OP_PACKED_GATED_BWD = 4 };

const char* eqat_status_string(int status);
int eqat_version(void);

/* Bytes of device scratch the given operation needs for this problem (0 if none,
 * (size_t)-1 if desc/op is invalid).  The workspace must be 256-byte aligned. */
size_t eqat_workspace_bytes(const eqat_desc* desc, int op);

/* Reads and clears the device status word of the current device (synchronises
 * the device).  *h_status receives EQAT_OK or EQAT_ERR_TIMEOUT; *h_detail (may be
 * NULL) a code naming the wait that was abandoned. */
int eqat_device_status(int* h_status, int* h_detail);

/* Diagnostic of the bounded waits (no counterpart in the paper).  Every wait of
 * a kernel on a barrier has a time limit, after which the kernel records
 * EQAT_ERR_TIMEOUT in the device status word, abandons its work and returns
 * normally.  This call enqueues one warp that waits, with a limit of 1 ms, on a
 * barrier that nothing ever signals, through the very wait routine of the GEMM
 * kernels (which = 0), of the streaming kernels (1), of the matrix-vector forward
 * (2), of the forward on weight-row tiles (3) or on pairs of them (4), or of the
 * attention over the cache for few rows (5) or prompts (6); afterwards
 * eqat_device_status() must report EQAT_ERR_TIMEOUT once and EQAT_OK from then
 * on.  It touches no tensor. */
int eqat_selftest_wait_expiry(int which, void* stream);

/* ------------------------------------------------------------------ helpers */

/* Round-to-nearest initialisation of the quantisation parameters from each
 * group's range (the paper does not describe its initialisation; this is the
 * min/max rule):  s = max((max - min) / (2^N - 1), 2^-14),
 * z = clamp(-round(min / s), 0, 2^N - 1), evaluated in binary32.
 *   W [out,in] bf16 (in)   s, z [out,in/g] fp32 (out; z is integer valued) */
int eqat_minmax_init(const eqat_desc* desc, const eqat_bf16* W, float* s, float* z, void* stream);

/* ------------------------------------------------------------------ Block-AP */

/* Eq. 1 followed by Eq. 2: W_hat = (clamp(round(W/s) + round(z), 0, 2^N-1) - round(z)) * s.
 * The quotient W/s is an IEEE binary32 division, rounded half-to-even.  Zeros of
 * W_hat may carry either sign.
 *   W [out,in] bf16, s, z [out,in/g] fp32 (in)   W_hat [out,in] bf16 (out) */
int eqat_fakequant_weight(const eqat_desc* desc, const eqat_bf16* W, const float* s, const float* z,
                          eqat_bf16* W_hat, void* stream);

/* Block-AP forward (Sec. 3.2): W_hat as above, then Y = X * W_hat^T with fp32
 * accumulation.  Two forms, same Y bit for bit:
 *   - W_hat != NULL: W_hat is computed once by a streaming kernel and written out
 *     (the backward pass can then read it); the faster form.
 *   - W_hat == NULL: nothing is stored; every tile of W is fake-quantised inside
 *     the GEMM after it has been copied to shared memory (Eq. 1-2 "integrated
 *     within the computation graph" taken literally).  It saves out*in*2 bytes of
 *     memory and costs more time, because each tile of W is quantised once per
 *     512 tokens instead of once.  Needs group <= 256 or group == in_features.
 *   X [T,in] bf16, W, s, z (in)   Y [T,out] bf16, W_hat [out,in] bf16 (out, optional) */
int qlinear_fakequant_fwd(const eqat_desc* desc, const eqat_bf16* X, const eqat_bf16* W, const float* s,
                          const float* z, eqat_bf16* Y, eqat_bf16* W_hat, void* stream);

/* Straight-through backward of the fake quantiser (Eqs. 3-5, upper bound read
 * as 2^N - 1 as in Eq. 1, bounds inclusive).  With p = round(w/s) + round(z):
 *   dW      = dW_hat            if 0 <= p <= 2^N-1, else 0
 *   ds[o,g] = sum over the group of dW_hat * (round(w/s) - w/s | -z | 2^N-1-z)
 *   dz[o,g] = sum over the group of dW_hat * (0 | -s | -s)      (dz_mode 1: -1)
 *   dW_hat, W [out,in] bf16, s, z fp32 (in)   dW bf16, ds, dz fp32 (out)
 * dz may be NULL (not computed). */
int eqat_ste_bwd(const eqat_desc* desc, const eqat_bf16* dW_hat, const eqat_bf16* W, const float* s,
                 const float* z, eqat_bf16* dW, float* ds, float* dz, void* stream);

/* Block-AP backward: dX = dY * W_hat, dW_hat = dY^T * X, then Eqs. 3-5 as in
 * eqat_ste_bwd.  W_hat is the array qlinear_fakequant_fwd stored, or NULL, in
 * which case the dX GEMM fake-quantises W tile by tile itself (same dX; same
 * restriction on the group as in the forward).  With groups of up to 256 elements Eqs. 3-5 are applied to the
 * fp32 accumulators of dW_hat inside the same kernel and dW_hat is never
 * stored; longer groups (channel-wise) keep dW_hat in bf16 in the workspace and
 * run eqat_ste_bwd on it.  Needs eqat_workspace_bytes(desc,
 * EQAT_OP_FAKEQUANT_BWD) bytes of scratch: 0 for groups of up to 256 elements
 * (workspace may then be NULL), out*in*2 bytes for longer ones.
 *   X [T,in], dY [T,out], W, W_hat [out,in] bf16, s, z (in)
 *   dX [T,in] bf16, dW [out,in] bf16, ds, dz [out,in/g] fp32 (out) */
int qlinear_fakequant_bwd(const eqat_desc* desc, const eqat_bf16* X, const eqat_bf16* dY, const eqat_bf16* W,
                          const float* s, const float* z, const eqat_bf16* W_hat,
                          eqat_bf16* dX, eqat_bf16* dW, float* ds, float* dz,
                          void* workspace, size_t workspace_bytes, void* stream);

/* The same computation as qlinear_fakequant_bwd, for callers that cannot
 * allocate device memory (no counterpart in the paper: it is a deployment
 * convenience of this library).  Typical cases: the process's device memory is
 * already owned by another framework's pool, or the caller sits in a section
 * where the device-wide synchronisation that cudaMalloc / cudaFree may imply is
 * not acceptable.  The out*in bf16 values of scratch live in a fixed array
 * inside the library, so
 *   - out_features * in_features must not exceed EQAT_NOALLOC_MAX_WEIGHT_ELEMS
 *     (8 MiB of bf16); larger problems return EQAT_ERR_WORKSPACE and launch
 *     nothing.  Every GPU that loads the library holds those 8 MiB until exit;
 *   - the first call on each device looks the array's address up (a runtime
 *     call that is not stream work).  With CUDA's lazy module loading that
 *     look-up is also the moment the device actually sets the 8 MiB aside, so
 *     make that first call (any small valid problem will do) early: before
 *     another framework claims the rest of the device's memory, and before any
 *     stream capture begins on that device.  EQAT_ERR_CUDA from a first call
 *     means the array could not be reserved;
 *   - all calls on a device share the one array.  Its previous contents do not
 *     matter (every value read is written earlier in the same call), but two
 *     calls whose kernels overlap on the GPU (different streams) race on it:
 *     serialise them;
 *   - it calls no cudaMalloc, cudaFree or other allocating routine.
 * Arguments, outputs and status codes are otherwise those of
 * qlinear_fakequant_bwd. */
#define EQAT_NOALLOC_MAX_WEIGHT_ELEMS (4u << 20)
int qlinear_fakequant_bwd_noalloc(const eqat_desc* desc, const eqat_bf16* X, const eqat_bf16* dY,
                                  const eqat_bf16* W, const float* s, const float* z, const eqat_bf16* W_hat,
                                  eqat_bf16* dX, eqat_bf16* dW, float* ds, float* dz, void* stream);

/* ------------------------------------------------------------------ storage format */
/* The paper stores W_int and z in N bits and s in fp16 (Sec. 3.2, last
 * paragraph; N + (N+16)/g bits per parameter, appendix "Size of Quantized
 * Models") but gives no bit order.  This library's: each row of W_int is a
 * dense little-endian bit stream, code j in stream bits [N*j, N*j+N), stream
 * bit b = bit (b % 8) of byte (b / 8); row pitch in*N/8 bytes. */

/* Hand-off from Block-AP to E2E-QP: codes of Eq. 1 packed, zero points as
 * bytes, step sizes rounded to fp16.
 *   W, s, z (in)   Wq_packed [out, in*N/8] u8, z8 [out,in/g] u8, s16 [out,in/g] fp16 (out) */
int eqat_quantize_pack(const eqat_desc* desc, const eqat_bf16* W, const float* s, const float* z,
                       uint8_t* Wq_packed, uint8_t* z8, eqat_fp16* s16, void* stream);

/* codes [out,in] u8 (each < 2^N) <-> Wq_packed [out, in*N/8]. */
int eqat_pack(const eqat_desc* desc, const uint8_t* codes, uint8_t* Wq_packed, void* stream);
int eqat_unpack(const eqat_desc* desc, const uint8_t* Wq_packed, uint8_t* codes, void* stream);

/* Zero points for storage: z8 [out*in/g] u8 <-> one flat N-bit stream of
 * out*in/g*N/8 bytes with the same bit rule (the count must be a multiple of 8). */
int eqat_pack_zeros(const eqat_desc* desc, const uint8_t* z8, uint8_t* z_packed, void* stream);
int eqat_unpack_zeros(const eqat_desc* desc, const uint8_t* z_packed, uint8_t* z8, void* stream);

/* ------------------------------------------------------------------ E2E-QP */

/* In the three calls below `z` is [out,in/g] uint8, or [out,in/g] fp16 when
 * desc->zero_point_format is EQAT_ZP_FP16. */

/* Y = X * ((W_int - z) * s)^T, the packed codes expanded tile by tile in
 * shared or tensor memory inside the GEMM (Eq. 2; Sec. 3.3).  With few tokens (decoding),
 * up to 64, the codes enter the products as exact integers and the step sizes
 * multiply fp32 sums, so (W_int - z) * s is not rounded to bf16: a matrix-vector
 * kernel of up to eight tokens per launch for the smallest batches (groups of at
 * least 64; a token's result does not depend on how the tokens were sliced into
 * launches), a kernel on tiles of 128 weight rows otherwise.  (Rows of more than
 * 57344 columns may not fit either; they are then treated like larger batches,
 * where (W_int - z) * s is rounded to bf16.)
 *
 * Repeated calls give the same bits on one device.  The bits of a token may
 * depend on the batch around it: which kernel runs, and in which order it adds up
 * K, follow the number of tokens, and above 64 tokens also the number of thread
 * block clusters that the device keeps resident, so a token can differ in the
 * last bits between batches of 7 and 8 tokens, between prefill chunks of 256 and
 * 512, and between devices.  They do not depend on it where every batch of up to
 * 16 tokens takes the matrix-vector kernel: weights of less than 3,000,000 bytes
 * of codes (out*in*N/8), in_features from 1024 to 4096, groups of at least 64.
 *   X [T,in] bf16, Wq_packed, s16, z (in)   Y [T,out] bf16 (out) */
int qlinear_packed_fwd(const eqat_desc* desc, const eqat_bf16* X, const uint8_t* Wq_packed,
                       const eqat_fp16* s16, const void* z, eqat_bf16* Y, void* stream);

/* Which kernel qlinear_packed_fwd takes for a problem, decided on the host from
 * the descriptor alone (a diagnostic; no counterpart in the paper).  `sms`: the
 * number of SMs to decide for, 0 for the current device.  Returns one of the
 * EQAT_ROUTE_* values or a negative eqat_status.  h_plan (may be NULL) receives
 * three numbers: launches or token tiles, tokens of each, and the split of K
 * over a cluster (0, 0, 1 for the tiled kernel).  Where a prompt goes out as two
 * launches the split is the first one's (eqat_packed_fwd_rest has the other). */
enum {
  EQAT_ROUTE_MATRIX_VECTOR = 1,     /* a few tokens: up to eight per pass over the weight   */
  EQAT_ROUTE_WEIGHT_ROWS = 2,       /* up to 64 tokens: tiles of 128 weight rows            */
  EQAT_ROUTE_WEIGHT_ROW_PAIRS = 3,  /* prompts: tiles of 256 weight rows                    */
  EQAT_ROUTE_TILED = 4              /* large batches: tiles of 512 or 256 tokens            */
};
int eqat_packed_fwd_route(const eqat_desc* desc, int sms, int* h_plan);

/* The second launch of a prompt on pairs of weight-row tiles: its weight rows, the
 * last ones of the weight, whose K is split over larger clusters than that of the
 * rows before them.  The token tiles are the same.  Same arguments as above (a
 * diagnostic); h_rest receives the number of those rows and their split, or 0 and 0
 * where one launch takes all rows. */
int eqat_packed_fwd_rest(const eqat_desc* desc, int sms, int* h_rest);

/* The output tiles of a contraction, decided on the host from the descriptor alone
 * (a diagnostic; no counterpart in the paper).  `sms` as in eqat_packed_fwd_route;
 * h_tile receives three numbers: rows of a tile per CTA, its columns, and the CTAs
 * that share it (1 or 2; two CTAs have rows of their own).  EQAT_GEMM_PACKED_Y is
 * the tiled kernel, whether or not qlinear_packed_fwd takes it. */
enum {
  EQAT_GEMM_Y = 0,                  /* qlinear_fakequant_fwd, W_hat stored                  */
  EQAT_GEMM_DX = 1,                 /* qlinear_fakequant_bwd: dX, W_hat stored              */
  EQAT_GEMM_DW = 2,                 /* qlinear_fakequant_bwd: the weight gradient           */
  EQAT_GEMM_LATENT_Y = 3,           /* as 0 and 1 with W_hat == NULL                        */
  EQAT_GEMM_LATENT_DX = 4,
  EQAT_GEMM_PACKED_Y = 5,           /* qlinear_packed_fwd, bwd_dx and bwd_ds                */
  EQAT_GEMM_PACKED_DX = 6,
  EQAT_GEMM_PACKED_DS = 7
};
int eqat_gemm_tile(const eqat_desc* desc, int contraction, int sms, int* h_tile);

/* dX = dY * ((W_int - z) * s).
 *   dY [T,out] bf16, Wq_packed, s16, z (in)   dX [T,in] bf16 (out) */
int qlinear_packed_bwd_dx(const eqat_desc* desc, const eqat_bf16* dY, const uint8_t* Wq_packed,
                          const eqat_fp16* s16, const void* z, eqat_bf16* dX, void* stream);

/* Step-size gradient (Sec. 3.3, d w_hat/d s = w_q - z):
 *   ds[o,g] = sum_{j in g} (sum_t dY[t,o] X[t,j]) * (W_int[o,j] - z[o,g]),
 * reduced in the epilogue of the weight-gradient GEMM; the [out,in] weight
 * gradient is never written to memory.  If dz is not NULL it also receives the
 * zero-point gradient of the same layer (the Sec. 3.3 variant that trains z),
 * dz[o,g] = -s[o,g] * sum_{j in g} G[o,j]; s16 is then required, else it may be
 * NULL.  Needs eqat_workspace_bytes(desc, EQAT_OP_PACKED_BWD_DS) bytes of
 * scratch: 0 for groups of up to 256 elements (workspace may then be NULL);
 * with one group per row the sums of the 256-column tiles of a row pass through
 * it and are added up in a fixed order.
 *   X [T,in], dY [T,out] bf16, Wq_packed, z (in)   ds [out,in/g] fp32 (out) */
int qlinear_packed_bwd_ds(const eqat_desc* desc, const eqat_bf16* X, const eqat_bf16* dY,
                          const uint8_t* Wq_packed, const void* z, const eqat_fp16* s16,
                          float* ds, float* dz, void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------ key/value cache */

/* The keys and values of the tokens before, held in 4 bits and in pages, and the
 * attention over them (no counterpart in the paper, which quantises weights only:
 * a block whose linears run through qlinear_packed_fwd spends its memory and its
 * decoding time on them).  The quantiser is that of Eqs. 1-2 with the parameters
 * of each group's range, as in eqat_minmax_init, except that the zero point is the
 * real number -m/s: a group of a cache need not contain 0.  A group x_1..x_g of
 * bf16 numbers (consecutive elements of a head of one token) with the minimum m
 * and the maximum M is held as
 *     s   = bf16((M - m) * (1/15)), 0 where that is below 2^-126,
 *     q_i = clamp(round((x_i - m) * (1/s)), 0, 15), 0 where s = 0,
 * evaluated in binary32 (1/15 and 1/s rounded to it; half to even), and stands
 * for q_i * s + m.  m is exact.  A group with a NaN, an infinity or a range
 * beyond binary32 stands for NaN.
 *
 * A pool holds `pages` pages, each `page_size` tokens of every key/value head:
 *     codes  [pages, kv_heads, page_size, head_dim/2]      u8, two codes a byte, the
 *            even element in the low half (the dense stream of eqat_pack)
 *     params [pages, kv_heads, page_size, head_dim/group, 2] bf16, s then m
 * for the keys and for the values.  Sequence b owns the pages in row b of
 * page_table [sequences, max_pages]: its token at position p is token p %
 * page_size of page page_table[b][p / page_size].
 *
 * A call works on `rows` rows, the new tokens of all sequences one after the
 * other: rows row_offsets[b] up to row_offsets[b+1] belong to sequence b
 * (row_offsets [sequences+1] starts at 0 and does not fall; a sequence may have
 * none), which holds lengths[b] tokens WITH them, so that its n rows stand at
 * positions lengths[b]-n .. lengths[b]-1.  The three arrays are int32 in device
 * memory; the host knows upper bounds only, so a captured call serves every
 * batch within them.  Rows from row_offsets[sequences] on belong to nobody:
 * nothing is read or written for them.
 * Contents of the arrays are not checked on the host: offsets are limited to
 * rows and lengths to max_pages * page_size; a position below 0 or a page number
 * outside the pool is not written, reads as zero, and as a key the latter gives
 * undefined values; no access leaves the tensors.  Table entries behind a
 * sequence's length may hold anything.
 *
 * X, Q, O, K, V are [rows, heads, head_dim] with heads and elements dense; the
 * pitch of a row, in elements, is a multiple of 8 (a slice of a fused projection
 * can be passed as it is).
 *
 * Geometry: bits 4; head_dim 64, 128 or 256; group 32, 64 or 128, at most
 * head_dim; page_size a multiple of 16; page_size * max_pages at most 2^30; at most
 * 2^37 bytes of codes for the keys (and as many for the values). */
typedef struct {
  int32_t bits;               /* 4                                                    */
  int32_t group;              /* elements per group along head_dim                    */
  int32_t head_dim;
  int32_t kv_heads;
  int32_t page_size;          /* tokens in a page                                     */
  int32_t pages;              /* pages in the pool                                    */
  int32_t sequences;
  int32_t max_pages;          /* columns of page_table                                */
  int64_t rows;               /* rows of the row tensors                              */
} eqat_cache_desc;

typedef struct {              /* the pool: device pointers, each 16-byte aligned */
  uint8_t* k_codes;
  eqat_bf16* k_params;
  uint8_t* v_codes;
  eqat_bf16* v_params;
} eqat_cache;

/* Quantises K and V of the rows and writes them to their places.  K_hat, V_hat
 * [rows, kv_heads, head_dim] dense (both or neither may be NULL) receive, in
 * bf16, what the cache now holds for them, as W_hat of qlinear_fakequant_fwd: a
 * prompt's own attention can use the values that later tokens will see.  Two rows
 * that name the same place leave it with bytes of either. */
int eqat_cache_append(const eqat_cache_desc* desc, const eqat_bf16* K, int64_t k_pitch, const eqat_bf16* V,
                      int64_t v_pitch, const int32_t* row_offsets, const int32_t* lengths,
                      const int32_t* page_table, const eqat_cache* cache, eqat_bf16* K_hat, eqat_bf16* V_hat,
                      void* stream);

/* The values that the cache holds for the rows' positions, in bf16: the last
 * row_offsets[b+1] - row_offsets[b] tokens of each sequence.
 *   K_hat, V_hat [rows, kv_heads, head_dim] dense (out) */
int eqat_cache_read(const eqat_cache_desc* desc, const int32_t* row_offsets, const int32_t* lengths,
                    const int32_t* page_table, const eqat_cache* cache, eqat_bf16* K_hat, eqat_bf16* V_hat,
                    void* stream);

typedef struct {
  int32_t q_heads;            /* a multiple of kv_heads; query head h reads kv head h / (q_heads/kv_heads) */
  int32_t max_new;            /* no sequence has more rows in this call (rows beyond are left out)         */
  float scale;                /* of the scores, e.g. head_dim^-1/2                                         */
  int32_t window;             /* a row at position p sees keys p-window+1 .. p; 0: 0 .. p                  */
} eqat_attention_desc;

/* Bytes of scratch eqat_cache_attention needs on the current device, 256-byte
 * aligned ((size_t)-1 if a descriptor is invalid).  Its contents do not matter and
 * are overwritten: calls that may overlap (streams, graphs replayed side by
 * side) need a workspace each. */
size_t eqat_cache_workspace_bytes(const eqat_cache_desc* desc, const eqat_attention_desc* attn);

/* How eqat_cache_attention divides a call, decided on the host from the descriptors
 * alone (a diagnostic).  `sms` as in eqat_packed_fwd_route (0 where there is no
 * device: 148, as eqat_cache_workspace_bytes assumes there); h_plan receives two
 * numbers: the query rows (new tokens x query heads of a key/value head) for which
 * the kernel for few rows reads a tile of the cache, and the number of rows from
 * which on a sequence goes to the kernel for prompts (0: none does; so for heads of
 * 256 and where the page table has room for more than 2^25 tokens of a sequence). */
int eqat_cache_attention_plan(const eqat_cache_desc* desc, const eqat_attention_desc* attn, int sms, int* h_plan);

/* Causal attention of the rows' queries over the cache, which already holds the
 * rows' own keys and values (eqat_cache_append):
 *     z_j = scale * sum_d Q_d K_jd,   O = sum_j softmax(z)_j V_j,
 * over the keys j that a row sees.  A row that sees none gets zeros, and lse
 * -infinity.  A query row whose largest element is below 2^-100 loses bits.
 * lse [rows, q_heads] fp32 dense (may be NULL): log of sum_j exp(z_j).
 * Few rows (decoding, drafted tokens): codes enter the products as exact integers,
 * steps and minima multiply the sums, and the weights of the values (softmax times
 * step) are integers of up to 23 bits, the largest of a row at least 2^20, rounded up
 * or down by a fixed sequence over the positions so that they are right in the mean:
 * an output's error is about sqrt(tokens) * 2^-20 of the row's largest product of
 * softmax, step and 15, besides the output's own rounding to bf16.
 * Many rows (eqat_cache_attention_plan): values and softmax weights are rounded to
 * bf16, values as eqat_cache_read gives them, keys to fp16 in steps of 2^-11 of
 * themselves or 2^-19 of the key's largest element; an infinite query element makes
 * its row NaN, and so do products of keys and the row brought to [1, 2) that pass
 * fp32's range; a row that sees a group of values that is NaN, or that bf16 cannot
 * hold, becomes NaN as a whole.  Softmax statistics and outputs are held in 32 bits
 * until the final rounding.  What a row does not see does not reach it, NaN or not.
 * Repeated calls give the same bits on one device; the order in which a long
 * sequence is added up depends on the lengths of the whole batch.
 *   Q [rows, q_heads, head_dim] bf16 (in)   O [rows, q_heads, head_dim] bf16 (out) */
int eqat_cache_attention(const eqat_cache_desc* desc, const eqat_attention_desc* attn, const eqat_bf16* Q,
                         int64_t q_pitch, const int32_t* row_offsets, const int32_t* lengths,
                         const int32_t* page_table, const eqat_cache* cache, eqat_bf16* O, int64_t o_pitch,
                         float* lse, void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------ between the linears of a block */

/* What a decoder block computes between its linears (no counterpart in the paper,
 * which trains whole blocks of such models): the norm of the residual stream, the
 * positions of queries and keys, and the gated product of two projections, each
 * with its backward pass.  Sizes are on the host; nothing is allocated, and calls
 * can be captured.  Statistics, angles and sums are held in 32 bits or more and
 * every output is rounded once, where nothing else is said.  In place means the
 * very same array and, with more than one row, the same pitch (EQAT_ERR_SHAPE
 * otherwise); arrays that overlap in any other way give undefined values. */

/* ---- root-mean-square norm of the residual stream
 *
 * A row of the stream, with what a linear adds to it:
 *     h = bf16(x + r),   c = (mean(h^2) + eps)^(-1/2),   y = bf16((h * w) * c).
 * The norm is that of h as it is stored.  Optionally the result is held in 8 bits,
 * every `group` consecutive elements with a scale of their own: with
 * t = fl(h * w) and a = max |t| over the group, both binary32,
 *     EQAT_CODES_INT8:  q = rint(fl(t * fl(127 / a)))    scale = a * c / 127
 *     EQAT_CODES_E4M3:  q = e4m3(fl(t * fl(448 / a)))    scale = a * c / 448
 * (half to even; a < 2^-110: q = 0, scale = 0).  c is left out of the decision, so
 * codes do not depend on the order in which squares are added up.  y is then
 * bf16(q * scale), what the codes stand for, as K_hat of eqat_cache_append.  A row
 * with a NaN gives NaN in y and the scales, one with an infinity NaN where it
 * stands (its group) and zeros elsewhere; codes of such groups may be anything.  A
 * row whose sum of squares passes binary32 gives zeros (NaN where h * w passes it
 * too), with eps = 0 a row of zeros gives NaN, and one whose root mean square is
 * below 2^-66 loses bits with its squares.
 *
 * features: a multiple of 8, at most 32768.  group (with codes): 32, 64, 128 or 256
 * dividing features, or features itself; 0 without codes. */
enum { EQAT_CODES_NONE = 0, EQAT_CODES_INT8 = 1, EQAT_CODES_E4M3 = 2 };

typedef struct {
  int64_t rows;
  int32_t features;
  int32_t codes;              /* EQAT_CODES_*                                         */
  int32_t group;              /* elements per scale                                   */
  float eps;                  /* finite, not negative                                 */
} eqat_norm_desc;

/*   X [rows, features], W [features] bf16 (in); R [rows, features] bf16 (in) or NULL: h = x
 *   H [rows, features] bf16 (out), may be NULL; may be X or R
 *   Y [rows, features] bf16 (out), may be NULL with codes
 *   codes [rows, features] u8 or s8, scales [rows, features/group] fp32 (out): both, or both NULL
 *   with EQAT_CODES_NONE */
int eqat_rms_norm_fwd(const eqat_norm_desc* desc, const eqat_bf16* X, const eqat_bf16* R, const eqat_bf16* W,
                      eqat_bf16* H, eqat_bf16* Y, void* codes, float* scales, void* stream);

/* Bytes of scratch eqat_rms_norm_bwd needs for dW on the current device, 256-byte
 * aligned ((size_t)-1 if the descriptor is invalid).  Calls that may overlap need a
 * workspace each. */
size_t eqat_rms_norm_workspace_bytes(const eqat_norm_desc* desc);

/* With v = dy * w:
 *     dx = dr + c * (v - h * c^2 * mean(v * h)),   dw = sum over the rows of dy * h * c.
 * dx is the gradient of h, so of x and of r; dr what reaches h from the stream behind
 * it.  (Codes pass it through: the descriptor's are not looked at.)  dw is added up
 * in an order that depends on the device and the shape alone.
 *   dY, H [rows, features], W [features] bf16 (in); dR [rows, features] bf16 (in) or NULL
 *   dX [rows, features] bf16 (out), may be dR or dY
 *   dW [features] fp32 (out), may be NULL: then no workspace is needed */
int eqat_rms_norm_bwd(const eqat_norm_desc* desc, const eqat_bf16* dY, const eqat_bf16* H, const eqat_bf16* W,
                      const eqat_bf16* dR, eqat_bf16* dX, float* dW, void* workspace, size_t workspace_bytes,
                      void* stream);

/* ---- rotary positions
 *
 * The first rotary_dim elements of a head, as pairs (a, b): elements i and
 * i + rotary_dim/2 (EQAT_ROTARY_HALVES) or 2i and 2i + 1 (EQAT_ROTARY_PAIRS).  At
 * position p, with the frequency f_i of the pair,
 *     (a cos pf - b sin pf, b cos pf + a sin pf) * amplitude.
 * The other elements are handed on.  Frequencies are given as fractions of a turn
 * per position, in units of 2^-64: turns[i] = round(2^64 f_i / 2 pi) mod 2^64, so
 * that p * turns[i] mod 2^64 is the angle whatever the position; that is rounded to
 * 2^-32 of a turn, between -1/2 and 1/2, and then to binary32: together at most
 * 2^-26 + 2^-33 of a turn, 1e-7 radians, for any position. */
enum { EQAT_ROTARY_HALVES = 0, EQAT_ROTARY_PAIRS = 1 };

typedef struct {
  int64_t rows;
  int32_t q_heads;            /* 1 .. 16384                                           */
  int32_t kv_heads;           /* 0 .. 16384; 0: no keys                               */
  int32_t head_dim;           /* a multiple of 8, at most 512                         */
  int32_t rotary_dim;         /* even, 2 .. head_dim                                  */
  int32_t layout;             /* EQAT_ROTARY_HALVES or _PAIRS                         */
  int32_t sequences;          /* with row_offsets; 0 with positions                   */
  float amplitude;            /* finite; 1 without scaling                            */
} eqat_rotary_desc;

/* Frequencies of a model made for texts of some length, and for longer ones
 * (`factor` times as long).  With f_i = base^(-2i/rotary_dim):
 *   EQAT_ROTARY_PLAIN   f_i
 *   EQAT_ROTARY_LINEAR  f_i / factor: positions interpolated
 *   EQAT_ROTARY_BASE    f_i of the base * factor^(rotary_dim/(rotary_dim - 2)): the fastest pair
 *                       as it was, the slowest divided by factor
 *   EQAT_ROTARY_RAMP    by the turns t_i = length * f_i / 2 pi that a pair makes in the length the
 *                       model was made for: f_i where t_i >= high, f_i / factor where t_i <= low,
 *                       in between k f_i + (1 - k) f_i / factor with k = (t_i - low)/(high - low)
 * (arXiv 2306.15595 and 2309.00071 describe them.) */
enum { EQAT_ROTARY_PLAIN = 0, EQAT_ROTARY_LINEAR = 1, EQAT_ROTARY_BASE = 2, EQAT_ROTARY_RAMP = 3 };

typedef struct {
  int32_t kind;               /* EQAT_ROTARY_PLAIN ...                                */
  int32_t rotary_dim;
  double base;                /* > 0                                                  */
  double factor;              /* > 0; not looked at by PLAIN                          */
  double low, high, length;   /* RAMP: 0 <= low < high, length > 0                    */
} eqat_rotary_scaling;

/* h_turns receives rotary_dim/2 numbers, on the host; eqat_rotary_turns_of takes
 * frequencies of the caller's own, radians per position (finite). */
int eqat_rotary_turns(const eqat_rotary_scaling* scaling, uint64_t* h_turns);
int eqat_rotary_turns_of(const double* h_frequencies, int count, uint64_t* h_turns);

/* Positions are given either way:
 *   - positions [rows] int32, of any sign; row_offsets and lengths NULL;
 *   - positions NULL, row_offsets [sequences+1] and lengths [sequences] int32 as in
 *     the calls of the cache: the n rows of sequence b stand at lengths[b]-n ..
 *     lengths[b]-1; rows of no sequence are left as they were.
 * Q, K, Q_out, K_out [rows, heads, head_dim] bf16, heads and elements dense, the
 * pitch of a row in elements a multiple of 8; K and K_out are not looked at without
 * keys.  Q_out may be Q, K_out K, with the same pitch.  The backward pass, gradients
 * in and out, is the transposed rotation, the same amplitude.
 *   turns [rotary_dim/2] (in, device) */
int eqat_rotary_fwd(const eqat_rotary_desc* desc, const eqat_bf16* Q, int64_t q_pitch, const eqat_bf16* K, int64_t k_pitch,
                    const uint64_t* turns, const int32_t* positions, const int32_t* row_offsets,
                    const int32_t* lengths, eqat_bf16* Q_out, int64_t q_out_pitch, eqat_bf16* K_out,
                    int64_t k_out_pitch, void* stream);
int eqat_rotary_bwd(const eqat_rotary_desc* desc, const eqat_bf16* dQ, int64_t q_pitch, const eqat_bf16* dK, int64_t k_pitch,
                    const uint64_t* turns, const int32_t* positions, const int32_t* row_offsets,
                    const int32_t* lengths, eqat_bf16* dQ_out, int64_t q_out_pitch, eqat_bf16* dK_out,
                    int64_t k_out_pitch, void* stream);

/* ---- gated product
 *
 *     H = act(G) * U,   dG = dH * U * act'(G),   dU = dH * act(G),
 * with act(g) = g / (1 + e^-g) (EQAT_ACT_SILU), g Phi(g) with the normal
 * distribution's Phi (EQAT_ACT_GELU), or g / (1 + e^(-2z)), z = (2/pi)^(1/2)
 * (g + 0.044715 g^3) (EQAT_ACT_GELU_TANH).  Values of act below 2^-110 may be 0. */
enum { EQAT_ACT_SILU = 0, EQAT_ACT_GELU = 1, EQAT_ACT_GELU_TANH = 2 };

typedef struct {
  int64_t rows;
  int32_t features;           /* a multiple of 8                                      */
  int32_t activation;         /* EQAT_ACT_*                                           */
} eqat_gated_desc;

/* For projections that stand already (qlinear_fakequant_fwd, or one linear for both).
 * Rows of G, U, dG, dU have a pitch in elements, a multiple of 8 and at least
 * features (the halves of one tensor can be passed as they are); H and dH are dense.
 * H may be G or U where those are dense; dG and dU may be G, U (with their pitch) or dH. */
int eqat_gated_fwd(const eqat_gated_desc* desc, const eqat_bf16* G, int64_t g_pitch, const eqat_bf16* U, int64_t u_pitch,
                   eqat_bf16* H, void* stream);
int eqat_gated_bwd(const eqat_gated_desc* desc, const eqat_bf16* dH, const eqat_bf16* G, int64_t g_pitch, const eqat_bf16* U,
                   int64_t u_pitch, eqat_bf16* dG, int64_t dg_pitch, eqat_bf16* dU, int64_t du_pitch, void* stream);

typedef struct {              /* a weight as qlinear_packed_fwd takes it: device pointers */
  const uint8_t* Wq_packed;   /* [out, in*N/8]                                        */
  const eqat_fp16* s16;       /* [out, in/g]                                          */
  const void* z;              /* [out, in/g] uint8 or fp16 (desc.zero_point_format)   */
} eqat_packed_weight;

/* Both projections of a feed-forward block and their product, the weights packed:
 *     G = X * W_gate^T,   U = X * W_up^T,   H = act(G) * U
 * for two weights of one descriptor (out_features of each).  The kernel is the one
 * that qlinear_packed_fwd takes for a weight of 2*out_features rows, with tiles that
 * hold both projections of their features: one pass over both weights, in which G
 * and U leave the kernel only if they are wanted (for the backward pass), and H is
 * that of the sums before they are rounded.  The exception are prompts for which
 * eqat_packed_gated_route says EQAT_ROUTE_WEIGHT_ROW_PAIRS: two calls of
 * qlinear_packed_fwd and one of eqat_gated_fwd, through G and U or, where these are
 * NULL, through the workspace; H is then that of G and U as they are rounded.  What
 * is said of qlinear_packed_fwd, of how weights enter the products and of bits, holds.
 * So H of random numbers is off, in relative norm, by its own rounding where codes
 * enter as integers (1.7e-3, up to 64 tokens), by the rounding of both weights too on
 * EQAT_ROUTE_TILED (2.9e-3), and by that of G and U besides on
 * EQAT_ROUTE_WEIGHT_ROW_PAIRS (3.8e-3).
 * Without G and U it needs eqat_workspace_bytes(desc, EQAT_OP_PACKED_GATED_FWD) bytes
 * of scratch on the current device (0: workspace may be NULL; with G and U it always
 * may).  Calls that may overlap need a workspace each, here and in the backward pass.
 *   X [T,in] bf16, gate, up (in)   H [T,out] bf16 (out)
 *   G, U [T,out] bf16 (out): both, or both NULL */
int qlinear_packed_gated_fwd(const eqat_desc* desc, int activation, const eqat_bf16* X, const eqat_packed_weight* gate,
                             const eqat_packed_weight* up, eqat_bf16* H, eqat_bf16* G, eqat_bf16* U, void* workspace,
                             size_t workspace_bytes, void* stream);

/* The kernel that the call goes to, EQAT_ROUTE_* (a diagnostic): that of the 2*out_features
 * rows, or EQAT_ROUTE_TILED in the place of EQAT_ROUTE_WEIGHT_ROW_PAIRS where it is
 * expected to be faster than two projections.  `sms` as in eqat_packed_fwd_route. */
int eqat_packed_gated_route(const eqat_desc* desc, int sms);

/* The output tiles of both weights' contractions (a diagnostic): `op` is
 * EQAT_OP_PACKED_GATED_FWD, for the tiled kernel, whether or not the call takes it, or
 * EQAT_OP_PACKED_GATED_BWD.  h_tile receives the three numbers of eqat_gemm_tile (columns
 * of a forward tile: half of them of either weight) and the parts that the contraction is
 * split into, whose sums pass through the workspace where there is more than one.  `sms`
 * as in eqat_packed_fwd_route. */
int eqat_packed_gated_tile(const eqat_desc* desc, int op, int sms, int* h_tile);

/* dG and dU as in eqat_gated_bwd, and
 *     dX = dG * W_gate + dU * W_up
 * of them as they are stored, one contraction over the features of both.  The step
 * sizes' gradients are qlinear_packed_bwd_ds of X with dG, and with dU.
 * Few tokens split the contraction over the chip and add its parts up in a fixed
 * order, through eqat_workspace_bytes(desc, EQAT_OP_PACKED_GATED_BWD) bytes of scratch.
 *   dH, G, U [T,out] bf16, gate, up (in)   dX [T,in], dG, dU [T,out] bf16 (out); dG and dU may
 *   be G, U or dH */
int qlinear_packed_gated_bwd(const eqat_desc* desc, int activation, const eqat_bf16* dH, const eqat_bf16* G,
                             const eqat_bf16* U, const eqat_packed_weight* gate, const eqat_packed_weight* up,
                             eqat_bf16* dX, eqat_bf16* dG, eqat_bf16* dU, void* workspace, size_t workspace_bytes,
                             void* stream);

/* ------------------------------------------------------------------ whole blocks */

/* Both phases of the paper work on one transformer block at a time (Block-AP,
 * Sec. 3.2: "training of all parameters" of a block; E2E-QP, Sec. 3.3: every
 * quantised linear of the network with frozen codes), so a training step calls
 * the layer entry points above once per linear of the block (seven in a Llama
 * decoder block).  The two calls below take the block's linears as a HOST array
 * and do exactly that, in array order, on one stream:
 *   eqat_block_ap_step : qlinear_fakequant_fwd, then qlinear_fakequant_bwd
 *   eqat_e2e_qp_step   : qlinear_packed_fwd, qlinear_packed_bwd_dx,
 *                        qlinear_packed_bwd_ds
 * Every linear is validated on the host before the first launch: on an error
 * nothing has been enqueued, the status is that of the first offending linear
 * and *h_failed (may be NULL) receives its index.  The fields have the meaning
 * of the same-named arguments of the layer entry points (W_hat, dz, workspace
 * optional as there).  The arrays are read during the call and not retained. */
typedef struct {
  eqat_desc desc;
  const eqat_bf16* X;         /* [T,in]                          */
  const eqat_bf16* dY;        /* [T,out]                         */
  const eqat_bf16* W;         /* [out,in] latent weight          */
  const float* s;             /* [out,in/g]                      */
  const float* z;             /* [out,in/g]                      */
  eqat_bf16* Y;               /* [T,out]   (out)                 */
  eqat_bf16* W_hat;           /* [out,in]  (out, may be NULL)    */
  eqat_bf16* dX;              /* [T,in]    (out)                 */
  eqat_bf16* dW;              /* [out,in]  (out)                 */
  float* ds;                  /* [out,in/g] (out)                */
  float* dz;                  /* [out,in/g] (out, may be NULL)   */
  void* workspace;            /* eqat_workspace_bytes(EQAT_OP_FAKEQUANT_BWD), may be NULL if 0 */
  size_t workspace_bytes;
} eqat_block_ap_linear;

typedef struct {
  eqat_desc desc;
  const eqat_bf16* X;         /* [T,in]                          */
  const eqat_bf16* dY;        /* [T,out]                         */
  const uint8_t* Wq_packed;   /* [out, in*N/8]                   */
  const eqat_fp16* s16;       /* [out,in/g]                      */
  const void* z;              /* [out,in/g] uint8 or fp16 (desc.zero_point_format) */
  eqat_bf16* Y;               /* [T,out]   (out)                 */
  eqat_bf16* dX;              /* [T,in]    (out)                 */
  float* ds;                  /* [out,in/g] (out)                */
  float* dz;                  /* [out,in/g] (out, may be NULL)   */
  void* workspace;            /* eqat_workspace_bytes(EQAT_OP_PACKED_BWD_DS), may be NULL if 0 */
  size_t workspace_bytes;
} eqat_e2e_qp_linear;

int eqat_block_ap_step(const eqat_block_ap_linear* h_linears, int count, int* h_failed, void* stream);
int eqat_e2e_qp_step(const eqat_e2e_qp_linear* h_linears, int count, int* h_failed, void* stream);

#ifdef __cplusplus
}
#endif
#endif  /* EQAT_H_ */
