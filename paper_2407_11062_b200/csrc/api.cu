// C ABI (include/eqat.h): argument validation on the host, then launches.
#include <stdint.h>

#include <cmath>

#include "attention.cuh"
#include "between.cuh"
#include "cache.cuh"
#include "common.cuh"
#include "elementwise.cuh"
#include "gemm.cuh"
#include "gemv.cuh"
#include "slim.cuh"
#include "wide.cuh"

namespace {

using namespace eqat;

constexpr int kMaxFusedSteGroup = 256;   // longest group the weight-gradient epilogue reduces by itself

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool is_pow2(int v) { return v > 0 && (v & (v - 1)) == 0; }

// Geometry every entry point shares.
int check_weight_desc(const eqat_desc* d) {
  if (d == nullptr) return EQAT_ERR_NULL;
  if (d->zero_point_format != EQAT_ZP_U8 && d->zero_point_format != EQAT_ZP_FP16) return EQAT_ERR_UNSUPPORTED;
  if (d->bits < 2 || d->bits > 4) return EQAT_ERR_UNSUPPORTED;
  if (d->dz_mode != 0 && d->dz_mode != 1) return EQAT_ERR_UNSUPPORTED;
  if (d->out_features <= 0 || d->in_features <= 0 || d->group <= 0) return EQAT_ERR_SHAPE;
  if (d->in_features % 128 != 0) return EQAT_ERR_SHAPE;
  if (d->group % 32 != 0 || d->in_features % d->group != 0) return EQAT_ERR_SHAPE;
  if (d->group <= 256 && !is_pow2(d->group)) return EQAT_ERR_UNSUPPORTED;
  if (d->group > 32768) return EQAT_ERR_UNSUPPORTED;
  if ((int64_t)d->out_features * d->in_features > ((int64_t)1 << 34)) return EQAT_ERR_SHAPE;
  return EQAT_OK;
}

// Entry points that read no packed zero points take the default format only.
int check_plain_desc(const eqat_desc* d) {
  const int rc = check_weight_desc(d);
  if (rc != EQAT_OK) return rc;
  return d->zero_point_format == EQAT_ZP_U8 ? EQAT_OK : EQAT_ERR_UNSUPPORTED;
}

int check_gemm_desc(const eqat_desc* d, bool packed) {
  const int rc = packed ? check_weight_desc(d) : check_plain_desc(d);
  if (rc != EQAT_OK) return rc;
  if (d->tokens <= 0 || d->tokens > (int64_t)1 << 30) return EQAT_ERR_SHAPE;
  if (d->out_features % 64 != 0) return EQAT_ERR_SHAPE;
  // packed kernels: a group is a power of two up to 256, or the whole row
  if (packed && d->group > 256 && d->group != d->in_features) return EQAT_ERR_UNSUPPORTED;
  return EQAT_OK;
}

// The kernels that fake-quantise the latent weight tile by tile index groups with a shift, or not at all.
inline bool latent_group_ok(const eqat_desc* d) { return d->group <= 256 || d->group == d->in_features; }

template <typename... P>
int check_ptrs(P... ptrs) {
  const void* v[] = {static_cast<const void*>(ptrs)...};
  for (const void* p : v)
    if (p == nullptr) return EQAT_ERR_NULL;
  for (const void* p : v)
    if (!aligned16(p)) return EQAT_ERR_ALIGN;
  return EQAT_OK;
}

inline cudaStream_t as_stream(void* s) { return static_cast<cudaStream_t>(s); }

// Host-side validation of the layer entry points, one function each, so that the block-level calls can check
// every linear before the first launch.
int v_fakequant_fwd(const eqat_desc* d, const eqat_bf16* X, const eqat_bf16* W, const float* s, const float* z,
                    const eqat_bf16* Y, const eqat_bf16* W_hat) {
  int rc = check_gemm_desc(d, false);
  if (rc != EQAT_OK) return rc;
  if ((rc = check_ptrs(X, W, s, z, Y)) != EQAT_OK) return rc;
  if (W_hat == nullptr) return latent_group_ok(d) ? EQAT_OK : EQAT_ERR_UNSUPPORTED;
  return aligned16(W_hat) ? EQAT_OK : EQAT_ERR_ALIGN;
}

int v_fakequant_bwd(const eqat_desc* d, const eqat_bf16* X, const eqat_bf16* dY, const eqat_bf16* W, const float* s,
                    const float* z, const eqat_bf16* W_hat, const eqat_bf16* dX, const eqat_bf16* dW, const float* ds,
                    const float* dz, const void* workspace, size_t workspace_bytes) {
  int rc = check_gemm_desc(d, false);
  if (rc != EQAT_OK) return rc;
  if ((rc = check_ptrs(X, dY, W, s, z, dX, dW, ds)) != EQAT_OK) return rc;
  if (dz != nullptr && !aligned16(dz)) return EQAT_ERR_ALIGN;
  if (W_hat != nullptr && !aligned16(W_hat)) return EQAT_ERR_ALIGN;
  if (W_hat == nullptr && !latent_group_ok(d)) return EQAT_ERR_UNSUPPORTED;
  if (d->group > kMaxFusedSteGroup) {
    const size_t need = (size_t)d->out_features * d->in_features * sizeof(eqat_bf16);
    if (workspace == nullptr || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0)
      return EQAT_ERR_WORKSPACE;
  }
  return EQAT_OK;
}

int v_packed_fwd(const eqat_desc* d, const eqat_bf16* X, const uint8_t* Wq, const eqat_fp16* s16, const void* z,
                 const eqat_bf16* Y) {
  const int rc = check_gemm_desc(d, true);
  return rc != EQAT_OK ? rc : check_ptrs(X, Wq, s16, z, Y);
}

int v_packed_bwd_ds(const eqat_desc* d, const eqat_bf16* X, const eqat_bf16* dY, const uint8_t* Wq, const void* z,
                    const eqat_fp16* s16, const float* ds, const float* dz, const void* workspace,
                    size_t workspace_bytes) {
  int rc = check_gemm_desc(d, true);
  if (rc != EQAT_OK) return rc;
  if ((rc = check_ptrs(X, dY, Wq, z, ds)) != EQAT_OK) return rc;
  if (dz != nullptr && (rc = check_ptrs(dz, s16)) != EQAT_OK) return rc;
  const size_t need = packed_ds_workspace_bytes(*d);
  if (need != 0 && (workspace == nullptr || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0))
    return EQAT_ERR_WORKSPACE;
  return EQAT_OK;
}

int check_cache_desc(const eqat_cache_desc* d) {
  if (d == nullptr) return EQAT_ERR_NULL;
  if (d->bits != 4) return EQAT_ERR_UNSUPPORTED;
  if (d->head_dim != 64 && d->head_dim != 128 && d->head_dim != 256) return EQAT_ERR_UNSUPPORTED;
  if (d->group != 32 && d->group != 64 && d->group != 128) return EQAT_ERR_UNSUPPORTED;
  if (d->group > d->head_dim || d->kv_heads <= 0 || d->kv_heads > 65536) return EQAT_ERR_SHAPE;
  if (d->page_size <= 0 || d->page_size % 16 != 0 || d->pages <= 0 || d->sequences <= 0 || d->max_pages <= 0) return EQAT_ERR_SHAPE;
  if (d->sequences > 1 << 20 || d->rows <= 0 || d->rows > (int64_t)1 << 30) return EQAT_ERR_SHAPE;
  if ((int64_t)d->page_size * d->max_pages > (int64_t)1 << 30) return EQAT_ERR_SHAPE;
  // lines of 128 bytes of codes are counted in 30 bits; in steps, since the whole product may pass 64
  const int64_t page = (int64_t)d->kv_heads * d->page_size * (d->head_dim / 2);
  if (page > (int64_t)1 << 37 || page * d->pages > (int64_t)1 << 37) return EQAT_ERR_SHAPE;
  return EQAT_OK;
}

int check_cache_ptrs(const int32_t* row_offsets, const int32_t* lengths, const int32_t* page_table, const eqat_cache* c) {
  if (c == nullptr) return EQAT_ERR_NULL;
  return check_ptrs(row_offsets, lengths, page_table, c->k_codes, c->k_params, c->v_codes, c->v_params);
}

inline bool pitch_ok(int64_t pitch, int64_t heads, int64_t head_dim) {
  return pitch >= heads * head_dim && pitch % 8 == 0 && pitch < (int64_t)1 << 40;
}

int check_attention_desc(const eqat_cache_desc* d, const eqat_attention_desc* a) {
  const int rc = check_cache_desc(d);
  if (rc != EQAT_OK) return rc;
  if (a == nullptr) return EQAT_ERR_NULL;
  if (a->q_heads <= 0 || a->q_heads > 65536 || a->q_heads % d->kv_heads != 0) return EQAT_ERR_SHAPE;
  if (a->max_new <= 0 || a->window < 0) return EQAT_ERR_SHAPE;
  if (d->rows * a->q_heads > (int64_t)1 << 30) return EQAT_ERR_SHAPE;      // rows x heads are counted in 32 bits
  if (!(a->scale > -1e30f && a->scale < 1e30f)) return EQAT_ERR_UNSUPPORTED;
  return EQAT_OK;
}

inline bool workspace_ok(const void* workspace, size_t bytes, size_t need) {
  return need == 0 || (workspace != nullptr && bytes >= need && (reinterpret_cast<uintptr_t>(workspace) & 255u) == 0);
}

// An output in place of an input keeps its pitch; with another one rows would overwrite rows that are still to be read.
inline bool overwrites_rows(int64_t rows, const eqat_bf16* in, int64_t in_pitch, const eqat_bf16* out, int64_t out_pitch) {
  return rows > 1 && in == out && in_pitch != out_pitch;
}

int check_norm_desc(const eqat_norm_desc* d) {
  if (d == nullptr) return EQAT_ERR_NULL;
  if (d->rows <= 0 || d->rows > (int64_t)1 << 30) return EQAT_ERR_SHAPE;
  if (d->features <= 0 || d->features % 8 != 0 || d->features > 32768) return EQAT_ERR_SHAPE;
  if (!(d->eps >= 0.0f && d->eps < 1e30f)) return EQAT_ERR_UNSUPPORTED;
  if (d->codes != EQAT_CODES_NONE && d->codes != EQAT_CODES_INT8 && d->codes != EQAT_CODES_E4M3) return EQAT_ERR_UNSUPPORTED;
  if (d->codes == EQAT_CODES_NONE) return d->group == 0 ? EQAT_OK : EQAT_ERR_SHAPE;
  if (d->group == d->features) return EQAT_OK;
  if (d->group != 32 && d->group != 64 && d->group != 128 && d->group != 256) return EQAT_ERR_UNSUPPORTED;
  return d->features % d->group == 0 ? EQAT_OK : EQAT_ERR_SHAPE;
}

int check_rotary_desc(const eqat_rotary_desc* d) {
  if (d == nullptr) return EQAT_ERR_NULL;
  if (d->rows <= 0 || d->rows > (int64_t)1 << 30) return EQAT_ERR_SHAPE;
  if (d->q_heads <= 0 || d->q_heads > kMaxRotaryHeads || d->kv_heads < 0 || d->kv_heads > kMaxRotaryHeads) return EQAT_ERR_SHAPE;
  if (d->head_dim <= 0 || d->head_dim % 8 != 0 || d->head_dim > kMaxRotaryHeadDim) return EQAT_ERR_SHAPE;
  if (d->rotary_dim <= 0 || d->rotary_dim % 2 != 0 || d->rotary_dim > d->head_dim) return EQAT_ERR_SHAPE;
  if (d->layout != EQAT_ROTARY_HALVES && d->layout != EQAT_ROTARY_PAIRS) return EQAT_ERR_UNSUPPORTED;
  if (d->sequences < 0 || d->sequences > 1 << 20) return EQAT_ERR_SHAPE;
  return std::isfinite(d->amplitude) ? EQAT_OK : EQAT_ERR_UNSUPPORTED;
}

int check_gated_desc(const eqat_gated_desc* d) {
  if (d == nullptr) return EQAT_ERR_NULL;
  if (d->rows <= 0 || d->rows > (int64_t)1 << 30) return EQAT_ERR_SHAPE;
  if (d->features <= 0 || d->features % 8 != 0) return EQAT_ERR_SHAPE;
  return d->activation >= EQAT_ACT_SILU && d->activation <= EQAT_ACT_GELU_TANH ? EQAT_OK : EQAT_ERR_UNSUPPORTED;
}

int rotary(const eqat_rotary_desc* d, const RotaryRows& r, bool backward, void* stream) {
  int rc = check_rotary_desc(d);
  if (rc != EQAT_OK) return rc;
  if (!pitch_ok(r.q_pitch, d->q_heads, d->head_dim) || !pitch_ok(r.q_out_pitch, d->q_heads, d->head_dim)) return EQAT_ERR_SHAPE;
  if ((rc = check_ptrs(r.q, r.q_out, r.turns)) != EQAT_OK) return rc;
  if (d->kv_heads > 0) {
    if (!pitch_ok(r.k_pitch, d->kv_heads, d->head_dim) || !pitch_ok(r.k_out_pitch, d->kv_heads, d->head_dim)) return EQAT_ERR_SHAPE;
    if ((rc = check_ptrs(r.k, r.k_out)) != EQAT_OK) return rc;
    if (overwrites_rows(d->rows, r.k, r.k_pitch, r.k_out, r.k_out_pitch)) return EQAT_ERR_SHAPE;
  }
  if (overwrites_rows(d->rows, r.q, r.q_pitch, r.q_out, r.q_out_pitch)) return EQAT_ERR_SHAPE;
  // one of the two ways to give positions
  if (r.positions != nullptr) {
    if (r.row_offsets != nullptr || r.lengths != nullptr) return EQAT_ERR_UNSUPPORTED;
    if (!aligned16(r.positions)) return EQAT_ERR_ALIGN;
  } else {
    if (d->sequences <= 0) return EQAT_ERR_SHAPE;
    if ((rc = check_ptrs(r.row_offsets, r.lengths)) != EQAT_OK) return rc;
  }
  return launch_rotary(*d, r, backward, static_cast<cudaStream_t>(stream));
}

// A fraction of a turn per position, in units of 2^-64 (the extended type has the 64 bits).
uint64_t turns_of(long double radians) {
  const long double turn = radians / 6.283185307179586476925286766559005768L;
  const long double scaled = std::rint((turn - std::floor(turn)) * 18446744073709551616.0L);
  return scaled >= 18446744073709551616.0L ? 0 : (uint64_t)scaled;
}

// The kernel that takes a packed forward.
struct PackedRoute {
  int kernel;                            // EQAT_ROUTE_*
  SlimPlan slim;
  WidePlan wide;
};

// On the current device (sms = 0), or as on a device of `sms` SMs.
PackedRoute packed_route(const eqat_desc& d, int sms) {
  PackedRoute r{};
  if (slim_fwd_applies(d, sms > 0 ? sms : sm_count(), r.slim)) r.kernel = EQAT_ROUTE_WEIGHT_ROWS;
  // a handful of tokens (decoding): one pass over the packed weight instead of near-empty tensor-core tiles
  else if (packed_gemv_applies(d)) r.kernel = EQAT_ROUTE_MATRIX_VECTOR;
  else if (wide_fwd_applies(d, sms, r.wide)) r.kernel = EQAT_ROUTE_WEIGHT_ROW_PAIRS;
  else r.kernel = EQAT_ROUTE_TILED;
  return r;
}

// How a gated feed-forward block's projections are taken: by the kernel of a weight with the rows of both.  The kernel on pairs of
// weight-row tiles has no tiles of two weights: there the projections go through memory, one weight after the other, or the
// tiled kernel takes both, whichever is expected to be faster.  Over 28 calls of 65 to 700 tokens (2 x 1408 x 2048 to 2 x 28672 x
// 8192) the choice is wrong in one, by 3 %.  11008 x 4096, 2 bits, 128 / 333 / 640 tokens: 49, 82, 115 us through memory, 71,
// 95, 141 us in one kernel; 1408 x 2048, 512 tokens: 28 and 22 us.  Through memory both projections are rounded to bf16 before the
// activation and the product: H is off by 0.0038 in relative norm where one kernel leaves 0.0028, most of it the weights' rounding.
struct GatedRoute {
  eqat_desc both;
  PackedRoute packed;
  int kernel;                            // EQAT_ROUTE_*; EQAT_ROUTE_WEIGHT_ROW_PAIRS: through memory
  // one projection in the workspace
  size_t bytes() const { return ((size_t)both.tokens * (both.out_features / 2) * sizeof(eqat_bf16) + 255) & ~(size_t)255; }
};
// SMs of the current device; without one, as of one of 148.
int sms_or_148() {
  const int n = sm_count();
  return n > 0 ? n : 148;
}
GatedRoute gated_route(const eqat_desc& d, int sms) {
  if (sms == 0 && sm_count() <= 0) sms = 148;
  GatedRoute r{d, {}, 0};
  r.both.out_features = 2 * d.out_features;
  r.packed = packed_route(r.both, sms);
  r.kernel = r.packed.kernel;
  if (r.kernel == EQAT_ROUTE_WEIGHT_ROW_PAIRS) {
    const int n = sms > 0 ? sms : sm_count();
    const PackedRoute one = packed_route(d, sms);
    const double us = one.kernel == EQAT_ROUTE_WEIGHT_ROW_PAIRS ? one.wide.us : packed_tiled_us(d, n);
    const double product = 3.0 + (double)d.tokens * d.out_features * 6.0 / 5.5e6;          // of the element-wise kernel
    if (2.0 * us + product >= packed_tiled_us(r.both, n)) r.kernel = EQAT_ROUTE_TILED;
  }
  return r;
}

size_t gated_fwd_workspace(const eqat_desc& d) {
  const GatedRoute r = gated_route(d, 0);
  return r.kernel == EQAT_ROUTE_WEIGHT_ROW_PAIRS ? 2 * r.bytes() : 0;
}

int check_gated_desc(const eqat_desc* d) {
  const int rc = check_gemm_desc(d, true);
  if (rc != EQAT_OK) return rc;
  return d->out_features <= 1 << 29 ? EQAT_OK : EQAT_ERR_SHAPE;          // the rows of both are counted in 32 bits
}

int check_gated_weights(const eqat_desc* d, int activation, const eqat_packed_weight* gate, const eqat_packed_weight* up) {
  const int rc = check_gated_desc(d);
  if (rc != EQAT_OK) return rc;
  if (activation < EQAT_ACT_SILU || activation > EQAT_ACT_GELU_TANH) return EQAT_ERR_UNSUPPORTED;
  if (gate == nullptr || up == nullptr) return EQAT_ERR_NULL;
  return check_ptrs(gate->Wq_packed, gate->s16, gate->z, up->Wq_packed, up->s16, up->z);
}

#define EQAT_TRY(expr)            \
  do {                            \
    const int rc__ = (expr);      \
    if (rc__ != EQAT_OK) return rc__; \
  } while (0)

}  // namespace

extern "C" {

const char* eqat_status_string(int status) {
  switch (status) {
    case EQAT_OK: return "ok";
    case EQAT_ERR_NULL: return "null pointer";
    case EQAT_ERR_SHAPE: return "invalid shape";
    case EQAT_ERR_ALIGN: return "pointer not 16-byte aligned";
    case EQAT_ERR_UNSUPPORTED: return "unsupported bits/group/mode";
    case EQAT_ERR_WORKSPACE: return "workspace missing, misaligned or too small";
    case EQAT_ERR_CUDA: return "CUDA error";
    case EQAT_ERR_TIMEOUT: return "a kernel abandoned a bounded wait";
    default: return "unknown status";
  }
}

int eqat_version(void) { return 100; }

size_t eqat_workspace_bytes(const eqat_desc* d, int op) {
  if (op == EQAT_OP_FAKEQUANT_BWD) {
    if (check_gemm_desc(d, false) != EQAT_OK) return (size_t)-1;
    // groups that fit an output tile are reduced inside the weight-gradient GEMM: nothing to store
    if (d->group <= kMaxFusedSteGroup) return 0;
    return (size_t)d->out_features * d->in_features * sizeof(eqat_bf16);   // dW_hat in bf16
  }
  if (op == EQAT_OP_PACKED_BWD_DS) {
    if (check_gemm_desc(d, true) != EQAT_OK) return (size_t)-1;
    return packed_ds_workspace_bytes(*d);
  }
  if (op == EQAT_OP_PACKED_GATED_FWD || op == EQAT_OP_PACKED_GATED_BWD) {
    if (check_gated_desc(d) != EQAT_OK) return (size_t)-1;
    return op == EQAT_OP_PACKED_GATED_FWD ? gated_fwd_workspace(*d) : packed_gated_dx_workspace(*d, sms_or_148());
  }
  return (size_t)-1;
}

int eqat_device_status(int* h_status, int* h_detail) {
  if (h_status == nullptr) return EQAT_ERR_NULL;
  int st[7] = {0, 0, 0, 0, 0, 0, 0}, det[7] = {0, 0, 0, 0, 0, 0, 0};
  EQAT_TRY(read_device_status(&st[0], &det[0]));      // GEMM kernels
  EQAT_TRY(read_stream_status(&st[1], &det[1]));      // staged streaming kernels
  EQAT_TRY(read_gemv_status(&st[2], &det[2]));        // matrix-vector kernels
  EQAT_TRY(read_slim_status(&st[3], &det[3]));        // weight-row kernels: few tokens,
  EQAT_TRY(read_wide_status(&st[4], &det[4]));        // prompts
  EQAT_TRY(read_attention_status(&st[5], &det[5]));   // attention over the cache: few rows,
  EQAT_TRY(read_prompt_status(&st[6], &det[6]));      // prompts
  int k = 0;
  while (k < 6 && st[k] == EQAT_OK) ++k;
  *h_status = st[k];
  if (h_detail != nullptr) *h_detail = det[k];
  return EQAT_OK;
}

int eqat_selftest_wait_expiry(int which, void* stream) {
  if (which == 0) return launch_wait_expiry_gemm(as_stream(stream));
  if (which == 1) return launch_wait_expiry_stream(as_stream(stream));
  if (which == 2) return launch_wait_expiry_gemv(as_stream(stream));
  if (which == 3) return launch_wait_expiry_slim(as_stream(stream));
  if (which == 4) return launch_wait_expiry_wide(as_stream(stream));
  if (which == 5) return launch_wait_expiry_attention(as_stream(stream));
  if (which == 6) return launch_wait_expiry_prompt(as_stream(stream));
  return EQAT_ERR_UNSUPPORTED;
}

int eqat_minmax_init(const eqat_desc* d, const eqat_bf16* W, float* s, float* z, void* stream) {
  EQAT_TRY(check_plain_desc(d));
  EQAT_TRY(check_ptrs(W, s, z));
  return launch_minmax(*d, W, s, z, as_stream(stream));
}

int eqat_fakequant_weight(const eqat_desc* d, const eqat_bf16* W, const float* s, const float* z, eqat_bf16* W_hat,
                          void* stream) {
  EQAT_TRY(check_plain_desc(d));
  EQAT_TRY(check_ptrs(W, s, z, W_hat));
  return launch_fakequant(*d, W, s, z, W_hat, as_stream(stream));
}

int qlinear_fakequant_fwd(const eqat_desc* d, const eqat_bf16* X, const eqat_bf16* W, const float* s, const float* z,
                          eqat_bf16* Y, eqat_bf16* W_hat, void* stream) {
  EQAT_TRY(v_fakequant_fwd(d, X, W, s, z, Y, W_hat));
  // W_hat not wanted: fake-quantise each tile of W inside the GEMM, after it has reached shared memory
  if (W_hat == nullptr) return launch_latent_fwd(*d, X, W, s, z, Y, as_stream(stream));
  EQAT_TRY(launch_fakequant(*d, W, s, z, W_hat, as_stream(stream)));
  return launch_dense_fwd(*d, X, W_hat, Y, as_stream(stream));
}

int eqat_ste_bwd(const eqat_desc* d, const eqat_bf16* dW_hat, const eqat_bf16* W, const float* s, const float* z,
                 eqat_bf16* dW, float* ds, float* dz, void* stream) {
  EQAT_TRY(check_plain_desc(d));
  EQAT_TRY(check_ptrs(dW_hat, W, s, z, dW, ds));
  if (dz != nullptr && !aligned16(dz)) return EQAT_ERR_ALIGN;
  return launch_ste_bwd(*d, dW_hat, W, s, z, dW, ds, dz, as_stream(stream));
}

int qlinear_fakequant_bwd(const eqat_desc* d, const eqat_bf16* X, const eqat_bf16* dY, const eqat_bf16* W,
                          const float* s, const float* z, const eqat_bf16* W_hat, eqat_bf16* dX, eqat_bf16* dW,
                          float* ds, float* dz, void* workspace, size_t workspace_bytes, void* stream) {
  EQAT_TRY(v_fakequant_bwd(d, X, dY, W, s, z, W_hat, dX, dW, ds, dz, workspace, workspace_bytes));
  // A group that fits inside one output tile is reduced in the weight-gradient GEMM's epilogue and needs no
  // scratch; a longer one (channel-wise quantisation) spans tiles, so its gradient goes through the workspace
  // and a second kernel.
  const bool fused = d->group <= kMaxFusedSteGroup;
  eqat_bf16* dW_hat = static_cast<eqat_bf16*>(workspace);
  cudaStream_t st = as_stream(stream);
  if (W_hat != nullptr) EQAT_TRY(launch_dense_dx(*d, dY, W_hat, dX, st));
  else EQAT_TRY(launch_latent_dx(*d, dY, W, s, z, dX, st));      // no stored W_hat: Eq. 1-2 inside the dX GEMM
  if (fused) return launch_dense_dw_ste(*d, dY, X, W, s, z, dW, ds, dz, st);
  EQAT_TRY(launch_dense_dw(*d, dY, X, dW_hat, st));
  return launch_ste_bwd(*d, dW_hat, W, s, z, dW, ds, dz, st);
}

int eqat_quantize_pack(const eqat_desc* d, const eqat_bf16* W, const float* s, const float* z, uint8_t* Wq_packed,
                       uint8_t* z8, eqat_fp16* s16, void* stream) {
  EQAT_TRY(check_plain_desc(d));
  EQAT_TRY(check_ptrs(W, s, z, Wq_packed, z8, s16));
  return launch_quantize_pack(*d, W, s, z, Wq_packed, z8, s16, as_stream(stream));
}

int eqat_pack(const eqat_desc* d, const uint8_t* codes, uint8_t* Wq_packed, void* stream) {
  EQAT_TRY(check_plain_desc(d));
  EQAT_TRY(check_ptrs(codes, Wq_packed));
  return launch_pack(*d, codes, Wq_packed, as_stream(stream));
}

int eqat_unpack(const eqat_desc* d, const uint8_t* Wq_packed, uint8_t* codes, void* stream) {
  EQAT_TRY(check_plain_desc(d));
  EQAT_TRY(check_ptrs(Wq_packed, codes));
  return launch_unpack(*d, Wq_packed, codes, as_stream(stream));
}

int eqat_pack_zeros(const eqat_desc* d, const uint8_t* z8, uint8_t* z_packed, void* stream) {
  EQAT_TRY(check_plain_desc(d));
  EQAT_TRY(check_ptrs(z8, z_packed));
  if (((int64_t)d->out_features * d->in_features / d->group) % 8 != 0) return EQAT_ERR_SHAPE;
  return launch_pack_zeros(*d, z8, z_packed, as_stream(stream));
}

int eqat_unpack_zeros(const eqat_desc* d, const uint8_t* z_packed, uint8_t* z8, void* stream) {
  EQAT_TRY(check_plain_desc(d));
  EQAT_TRY(check_ptrs(z_packed, z8));
  if (((int64_t)d->out_features * d->in_features / d->group) % 8 != 0) return EQAT_ERR_SHAPE;
  return launch_unpack_zeros(*d, z_packed, z8, as_stream(stream));
}

int qlinear_packed_fwd(const eqat_desc* d, const eqat_bf16* X, const uint8_t* Wq_packed, const eqat_fp16* s16,
                       const void* z, eqat_bf16* Y, void* stream) {
  EQAT_TRY(v_packed_fwd(d, X, Wq_packed, s16, z, Y));
  const PackedRoute r = packed_route(*d, 0);
  switch (r.kernel) {
    case EQAT_ROUTE_WEIGHT_ROWS: return launch_slim_fwd(*d, X, Wq_packed, s16, z, Y, r.slim, as_stream(stream));
    case EQAT_ROUTE_MATRIX_VECTOR: return launch_packed_gemv(*d, X, Wq_packed, s16, z, Y, as_stream(stream));
    case EQAT_ROUTE_WEIGHT_ROW_PAIRS: return launch_wide_fwd(*d, X, Wq_packed, s16, z, Y, r.wide, as_stream(stream));
    default: return launch_packed_fwd(*d, X, Wq_packed, s16, z, Y, as_stream(stream));
  }
}

int eqat_packed_fwd_route(const eqat_desc* d, int sms, int* h_plan) {
  EQAT_TRY(check_gemm_desc(d, true));
  if (sms < 0) return EQAT_ERR_SHAPE;
  const PackedRoute r = packed_route(*d, sms);
  if (h_plan != nullptr) {
    const FewTokenPlan gemv = packed_gemv_plan(*d);
    const bool mv = r.kernel == EQAT_ROUTE_MATRIX_VECTOR, rows = r.kernel == EQAT_ROUTE_WEIGHT_ROWS;
    const bool pairs = r.kernel == EQAT_ROUTE_WEIGHT_ROW_PAIRS;
    h_plan[0] = mv ? gemv.launches : (rows ? r.slim.token_tiles : (pairs ? r.wide.token_tiles : 0));
    h_plan[1] = mv ? gemv.slice : (rows ? 16 * r.slim.nt : (pairs ? r.wide.tn : 0));
    h_plan[2] = rows ? r.slim.split : (pairs ? r.wide.split : 1);
  }
  return r.kernel;
}

int eqat_packed_fwd_rest(const eqat_desc* d, int sms, int* h_rest) {
  EQAT_TRY(check_gemm_desc(d, true));
  if (h_rest == nullptr) return EQAT_ERR_NULL;
  if (sms < 0) return EQAT_ERR_SHAPE;
  const PackedRoute r = packed_route(*d, sms);
  const int rows = r.kernel == EQAT_ROUTE_WEIGHT_ROW_PAIRS ? d->out_features - 256 * r.wide.first_pairs : 0;
  h_rest[0] = rows > 0 ? rows : 0;
  h_rest[1] = rows > 0 ? r.wide.rest_split : 0;
  return EQAT_OK;
}

int eqat_gemm_tile(const eqat_desc* d, int contraction, int sms, int* h_tile) {
  if (contraction < EQAT_GEMM_Y || contraction > EQAT_GEMM_PACKED_DS) return EQAT_ERR_UNSUPPORTED;
  EQAT_TRY(check_gemm_desc(d, contraction >= EQAT_GEMM_PACKED_Y));
  if (h_tile == nullptr) return EQAT_ERR_NULL;
  if (sms < 0) return EQAT_ERR_SHAPE;
  const TileShape t = contraction_shape(*d, contraction, sms > 0 ? sms : sm_count());
  h_tile[0] = 128 * t.mt;
  h_tile[1] = t.bn;
  h_tile[2] = t.pair ? 2 : 1;
  return EQAT_OK;
}

int qlinear_packed_bwd_dx(const eqat_desc* d, const eqat_bf16* dY, const uint8_t* Wq_packed, const eqat_fp16* s16,
                          const void* z, eqat_bf16* dX, void* stream) {
  EQAT_TRY(v_packed_fwd(d, dY, Wq_packed, s16, z, dX));          // same shape of check: one activation in, one out
  return launch_packed_dx(*d, dY, Wq_packed, s16, z, dX, as_stream(stream));
}

int qlinear_packed_bwd_ds(const eqat_desc* d, const eqat_bf16* X, const eqat_bf16* dY, const uint8_t* Wq_packed,
                          const void* z, const eqat_fp16* s16, float* ds, float* dz, void* workspace,
                          size_t workspace_bytes, void* stream) {
  EQAT_TRY(v_packed_bwd_ds(d, X, dY, Wq_packed, z, s16, ds, dz, workspace, workspace_bytes));
  return launch_packed_ds(*d, X, dY, Wq_packed, z, s16, ds, dz, workspace, as_stream(stream));
}

int eqat_cache_append(const eqat_cache_desc* d, const eqat_bf16* K, int64_t k_pitch, const eqat_bf16* V, int64_t v_pitch,
                      const int32_t* row_offsets, const int32_t* lengths, const int32_t* page_table, const eqat_cache* cache,
                      eqat_bf16* K_hat, eqat_bf16* V_hat, void* stream) {
  EQAT_TRY(check_cache_desc(d));
  if (!pitch_ok(k_pitch, d->kv_heads, d->head_dim) || !pitch_ok(v_pitch, d->kv_heads, d->head_dim)) return EQAT_ERR_SHAPE;
  EQAT_TRY(check_ptrs(K, V));
  EQAT_TRY(check_cache_ptrs(row_offsets, lengths, page_table, cache));
  if ((K_hat == nullptr) != (V_hat == nullptr)) return EQAT_ERR_NULL;
  if (!aligned16(K_hat) || !aligned16(V_hat)) return EQAT_ERR_ALIGN;
  return launch_cache_append(*d, K, k_pitch, V, v_pitch, cache_view(*d, row_offsets, lengths, page_table, *cache), K_hat, V_hat,
                             as_stream(stream));
}

int eqat_cache_read(const eqat_cache_desc* d, const int32_t* row_offsets, const int32_t* lengths, const int32_t* page_table,
                    const eqat_cache* cache, eqat_bf16* K_hat, eqat_bf16* V_hat, void* stream) {
  EQAT_TRY(check_cache_desc(d));
  EQAT_TRY(check_cache_ptrs(row_offsets, lengths, page_table, cache));
  EQAT_TRY(check_ptrs(K_hat, V_hat));
  return launch_cache_read(*d, cache_view(*d, row_offsets, lengths, page_table, *cache), K_hat, V_hat, as_stream(stream));
}

size_t eqat_cache_workspace_bytes(const eqat_cache_desc* d, const eqat_attention_desc* a) {
  return check_attention_desc(d, a) == EQAT_OK ? cache_attention_workspace(*d, *a) : (size_t)-1;
}

int eqat_cache_attention_plan(const eqat_cache_desc* d, const eqat_attention_desc* a, int sms, int* h_plan) {
  EQAT_TRY(check_attention_desc(d, a));
  if (h_plan == nullptr) return EQAT_ERR_NULL;
  if (sms < 0) return EQAT_ERR_SHAPE;
  if (sms == 0) sms = sm_count();
  if (sms <= 0) sms = 148;                                               // no device: as for the workspace
  cache_attention_plan(*d, *a, sms, h_plan);
  return EQAT_OK;
}

int eqat_cache_attention(const eqat_cache_desc* d, const eqat_attention_desc* a, const eqat_bf16* Q, int64_t q_pitch,
                         const int32_t* row_offsets, const int32_t* lengths, const int32_t* page_table,
                         const eqat_cache* cache, eqat_bf16* O, int64_t o_pitch, float* lse, void* workspace,
                         size_t workspace_bytes, void* stream) {
  EQAT_TRY(check_attention_desc(d, a));
  if (!pitch_ok(q_pitch, a->q_heads, d->head_dim) || !pitch_ok(o_pitch, a->q_heads, d->head_dim)) return EQAT_ERR_SHAPE;
  EQAT_TRY(check_ptrs(Q, O));
  EQAT_TRY(check_cache_ptrs(row_offsets, lengths, page_table, cache));
  if (!aligned16(lse)) return EQAT_ERR_ALIGN;
  const size_t need = cache_attention_workspace(*d, *a);
  if (need != 0 && (workspace == nullptr || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0))
    return EQAT_ERR_WORKSPACE;
  return launch_cache_attention(*d, *a, Q, q_pitch, cache_view(*d, row_offsets, lengths, page_table, *cache), O, o_pitch, lse,
                                workspace, as_stream(stream));
}

int eqat_rms_norm_fwd(const eqat_norm_desc* d, const eqat_bf16* X, const eqat_bf16* R, const eqat_bf16* W, eqat_bf16* H,
                      eqat_bf16* Y, void* codes, float* scales, void* stream) {
  EQAT_TRY(check_norm_desc(d));
  EQAT_TRY(check_ptrs(X, W));
  if (d->codes == EQAT_CODES_NONE) {
    if (codes != nullptr || scales != nullptr) return EQAT_ERR_UNSUPPORTED;
    EQAT_TRY(check_ptrs(Y));
  } else {
    EQAT_TRY(check_ptrs(codes, scales));
    if (!aligned16(Y)) return EQAT_ERR_ALIGN;
  }
  if (!aligned16(R) || !aligned16(H)) return EQAT_ERR_ALIGN;
  return launch_norm_fwd(*d, X, R, W, H, Y, codes, scales, as_stream(stream));
}

size_t eqat_rms_norm_workspace_bytes(const eqat_norm_desc* d) {
  if (check_norm_desc(d) != EQAT_OK) return (size_t)-1;
  return norm_workspace(*d, sms_or_148());
}

int eqat_rms_norm_bwd(const eqat_norm_desc* d, const eqat_bf16* dY, const eqat_bf16* H, const eqat_bf16* W, const eqat_bf16* dR,
                      eqat_bf16* dX, float* dW, void* workspace, size_t workspace_bytes, void* stream) {
  EQAT_TRY(check_norm_desc(d));
  EQAT_TRY(check_ptrs(dY, H, W, dX));
  if (!aligned16(dR) || !aligned16(dW)) return EQAT_ERR_ALIGN;
  if (dW != nullptr && !workspace_ok(workspace, workspace_bytes, eqat_rms_norm_workspace_bytes(d))) return EQAT_ERR_WORKSPACE;
  return launch_norm_bwd(*d, dY, H, W, dR, dX, dW, workspace, as_stream(stream));
}

int eqat_rotary_turns(const eqat_rotary_scaling* s, uint64_t* h_turns) {
  if (s == nullptr || h_turns == nullptr) return EQAT_ERR_NULL;
  if (s->rotary_dim <= 0 || s->rotary_dim % 2 != 0 || s->rotary_dim > 512) return EQAT_ERR_SHAPE;
  if (s->kind < EQAT_ROTARY_PLAIN || s->kind > EQAT_ROTARY_RAMP) return EQAT_ERR_UNSUPPORTED;
  if (!(std::isfinite(s->base) && s->base > 0.0)) return EQAT_ERR_UNSUPPORTED;
  if (s->kind != EQAT_ROTARY_PLAIN && !(std::isfinite(s->factor) && s->factor > 0.0)) return EQAT_ERR_UNSUPPORTED;
  if (s->kind == EQAT_ROTARY_RAMP &&
      !(std::isfinite(s->high) && s->low >= 0.0 && s->low < s->high && std::isfinite(s->length) && s->length > 0.0))
    return EQAT_ERR_UNSUPPORTED;
  const int n = s->rotary_dim / 2;
  long double base = s->base;
  if (s->kind == EQAT_ROTARY_BASE && n > 1) base *= std::pow((long double)s->factor, (long double)n / (n - 1));
  for (int i = 0; i < n; ++i) {
    long double f = std::pow(base, -(long double)i / n);
    if (!std::isfinite(f)) return EQAT_ERR_UNSUPPORTED;
    if (s->kind == EQAT_ROTARY_LINEAR) f /= s->factor;
    if (s->kind == EQAT_ROTARY_RAMP) {
      const long double t = s->length * f / 6.283185307179586476925286766559005768L;
      long double k = (t - s->low) / ((long double)s->high - s->low);
      k = k < 0.0L ? 0.0L : k > 1.0L ? 1.0L : k;
      f = k * f + (1.0L - k) * f / s->factor;
    }
    h_turns[i] = turns_of(f);
  }
  return EQAT_OK;
}

int eqat_rotary_turns_of(const double* h_frequencies, int count, uint64_t* h_turns) {
  if (h_frequencies == nullptr || h_turns == nullptr) return EQAT_ERR_NULL;
  if (count <= 0) return EQAT_ERR_SHAPE;
  for (int i = 0; i < count; ++i)
    if (!std::isfinite(h_frequencies[i])) return EQAT_ERR_UNSUPPORTED;
  for (int i = 0; i < count; ++i) h_turns[i] = turns_of(h_frequencies[i]);
  return EQAT_OK;
}

int eqat_rotary_fwd(const eqat_rotary_desc* d, const eqat_bf16* Q, int64_t q_pitch, const eqat_bf16* K, int64_t k_pitch,
                    const uint64_t* turns, const int32_t* positions, const int32_t* row_offsets, const int32_t* lengths,
                    eqat_bf16* Q_out, int64_t q_out_pitch, eqat_bf16* K_out, int64_t k_out_pitch, void* stream) {
  return rotary(d, RotaryRows{Q, K, q_pitch, k_pitch, Q_out, K_out, q_out_pitch, k_out_pitch, turns, positions, row_offsets, lengths},
                false, stream);
}

int eqat_rotary_bwd(const eqat_rotary_desc* d, const eqat_bf16* dQ, int64_t q_pitch, const eqat_bf16* dK, int64_t k_pitch,
                    const uint64_t* turns, const int32_t* positions, const int32_t* row_offsets, const int32_t* lengths,
                    eqat_bf16* dQ_out, int64_t q_out_pitch, eqat_bf16* dK_out, int64_t k_out_pitch, void* stream) {
  return rotary(d, RotaryRows{dQ, dK, q_pitch, k_pitch, dQ_out, dK_out, q_out_pitch, k_out_pitch, turns, positions, row_offsets, lengths},
                true, stream);
}

int eqat_gated_fwd(const eqat_gated_desc* d, const eqat_bf16* G, int64_t g_pitch, const eqat_bf16* U, int64_t u_pitch,
                   eqat_bf16* H, void* stream) {
  EQAT_TRY(check_gated_desc(d));
  if (!pitch_ok(g_pitch, 1, d->features) || !pitch_ok(u_pitch, 1, d->features)) return EQAT_ERR_SHAPE;
  EQAT_TRY(check_ptrs(G, U, H));
  if (overwrites_rows(d->rows, G, g_pitch, H, d->features) || overwrites_rows(d->rows, U, u_pitch, H, d->features)) return EQAT_ERR_SHAPE;
  return launch_gated_fwd(*d, G, g_pitch, U, u_pitch, H, as_stream(stream));
}

int eqat_gated_bwd(const eqat_gated_desc* d, const eqat_bf16* dH, const eqat_bf16* G, int64_t g_pitch, const eqat_bf16* U,
                   int64_t u_pitch, eqat_bf16* dG, int64_t dg_pitch, eqat_bf16* dU, int64_t du_pitch, void* stream) {
  EQAT_TRY(check_gated_desc(d));
  if (!pitch_ok(g_pitch, 1, d->features) || !pitch_ok(u_pitch, 1, d->features)) return EQAT_ERR_SHAPE;
  if (!pitch_ok(dg_pitch, 1, d->features) || !pitch_ok(du_pitch, 1, d->features)) return EQAT_ERR_SHAPE;
  EQAT_TRY(check_ptrs(dH, G, U, dG, dU));
  const struct { const eqat_bf16* at; int64_t pitch; } in[] = {{dH, d->features}, {G, g_pitch}, {U, u_pitch}};
  for (const auto& i : in)
    if (overwrites_rows(d->rows, i.at, i.pitch, dG, dg_pitch) || overwrites_rows(d->rows, i.at, i.pitch, dU, du_pitch)) return EQAT_ERR_SHAPE;
  return launch_gated_bwd(*d, dH, G, g_pitch, U, u_pitch, dG, dg_pitch, dU, du_pitch, as_stream(stream));
}

int eqat_packed_gated_route(const eqat_desc* d, int sms) {
  EQAT_TRY(check_gated_desc(d));
  if (sms < 0) return EQAT_ERR_SHAPE;
  return gated_route(*d, sms).kernel;
}

int eqat_packed_gated_tile(const eqat_desc* d, int op, int sms, int* h_tile) {
  if (op != EQAT_OP_PACKED_GATED_FWD && op != EQAT_OP_PACKED_GATED_BWD) return EQAT_ERR_UNSUPPORTED;
  EQAT_TRY(check_gated_desc(d));
  if (h_tile == nullptr) return EQAT_ERR_NULL;
  if (sms < 0) return EQAT_ERR_SHAPE;
  if (sms == 0) sms = sms_or_148();
  const JointPlan t = op == EQAT_OP_PACKED_GATED_BWD ? joint_plan(*d, sms) : JointPlan{packed_shape((int)d->tokens, 2 * d->out_features, sms), 1};
  h_tile[0] = 128 * t.shape.mt;
  h_tile[1] = t.shape.bn;
  h_tile[2] = t.shape.pair ? 2 : 1;
  h_tile[3] = t.split;
  return EQAT_OK;
}

int qlinear_packed_gated_fwd(const eqat_desc* d, int activation, const eqat_bf16* X, const eqat_packed_weight* gate,
                             const eqat_packed_weight* up, eqat_bf16* H, eqat_bf16* G, eqat_bf16* U, void* workspace,
                             size_t workspace_bytes, void* stream) {
  EQAT_TRY(check_gated_weights(d, activation, gate, up));
  EQAT_TRY(check_ptrs(X, H));
  if ((G == nullptr) != (U == nullptr)) return EQAT_ERR_NULL;
  if (!aligned16(G) || !aligned16(U)) return EQAT_ERR_ALIGN;
  const GatedRoute r = gated_route(*d, 0);
  cudaStream_t st = as_stream(stream);
  switch (r.kernel) {
    case EQAT_ROUTE_WEIGHT_ROWS: return launch_slim_gated(*d, activation, X, *gate, *up, H, G, U, r.packed.slim, st);
    case EQAT_ROUTE_MATRIX_VECTOR: return launch_gemv_gated(*d, r.both, activation, X, *gate, *up, H, G, U, st);
    case EQAT_ROUTE_TILED: return launch_packed_gated(*d, activation, X, *gate, *up, H, G, U, st);
    default: break;
  }
  if (G == nullptr) {
    if (!workspace_ok(workspace, workspace_bytes, 2 * r.bytes())) return EQAT_ERR_WORKSPACE;
    G = static_cast<eqat_bf16*>(workspace);
    U = reinterpret_cast<eqat_bf16*>(static_cast<uint8_t*>(workspace) + r.bytes());
  }
  EQAT_TRY(qlinear_packed_fwd(d, X, gate->Wq_packed, gate->s16, gate->z, G, stream));
  EQAT_TRY(qlinear_packed_fwd(d, X, up->Wq_packed, up->s16, up->z, U, stream));
  const eqat_gated_desc g{d->tokens, d->out_features, activation};
  return launch_gated_fwd(g, G, d->out_features, U, d->out_features, H, st);
}

int qlinear_packed_gated_bwd(const eqat_desc* d, int activation, const eqat_bf16* dH, const eqat_bf16* G, const eqat_bf16* U,
                             const eqat_packed_weight* gate, const eqat_packed_weight* up, eqat_bf16* dX, eqat_bf16* dG,
                             eqat_bf16* dU, void* workspace, size_t workspace_bytes, void* stream) {
  EQAT_TRY(check_gated_weights(d, activation, gate, up));
  EQAT_TRY(check_ptrs(dH, G, U, dX, dG, dU));
  if (!workspace_ok(workspace, workspace_bytes, packed_gated_dx_workspace(*d, sms_or_148()))) return EQAT_ERR_WORKSPACE;
  const eqat_gated_desc g{d->tokens, d->out_features, activation};
  const int64_t pitch = d->out_features;
  EQAT_TRY(launch_gated_bwd(g, dH, G, pitch, U, pitch, dG, pitch, dU, pitch, as_stream(stream)));
  return launch_packed_gated_dx(*d, dG, dU, *gate, *up, dX, workspace, as_stream(stream));
}

int eqat_block_ap_step(const eqat_block_ap_linear* L, int count, int* h_failed, void* stream) {
  if (h_failed != nullptr) *h_failed = -1;
  if (L == nullptr) return EQAT_ERR_NULL;
  if (count <= 0) return EQAT_ERR_SHAPE;
  for (int i = 0; i < count; ++i) {                         // everything is checked before anything is launched
    int rc = v_fakequant_fwd(&L[i].desc, L[i].X, L[i].W, L[i].s, L[i].z, L[i].Y, L[i].W_hat);
    if (rc == EQAT_OK)
      rc = v_fakequant_bwd(&L[i].desc, L[i].X, L[i].dY, L[i].W, L[i].s, L[i].z, L[i].W_hat, L[i].dX, L[i].dW, L[i].ds,
                           L[i].dz, L[i].workspace, L[i].workspace_bytes);
    if (rc != EQAT_OK) {
      if (h_failed != nullptr) *h_failed = i;
      return rc;
    }
  }
  for (int i = 0; i < count; ++i) {
    int rc = qlinear_fakequant_fwd(&L[i].desc, L[i].X, L[i].W, L[i].s, L[i].z, L[i].Y, L[i].W_hat, stream);
    if (rc == EQAT_OK)
      rc = qlinear_fakequant_bwd(&L[i].desc, L[i].X, L[i].dY, L[i].W, L[i].s, L[i].z, L[i].W_hat, L[i].dX, L[i].dW,
                                 L[i].ds, L[i].dz, L[i].workspace, L[i].workspace_bytes, stream);
    if (rc != EQAT_OK) {                                    // only the runtime can still refuse (EQAT_ERR_CUDA)
      if (h_failed != nullptr) *h_failed = i;
      return rc;
    }
  }
  return EQAT_OK;
}

int eqat_e2e_qp_step(const eqat_e2e_qp_linear* L, int count, int* h_failed, void* stream) {
  if (h_failed != nullptr) *h_failed = -1;
  if (L == nullptr) return EQAT_ERR_NULL;
  if (count <= 0) return EQAT_ERR_SHAPE;
  for (int i = 0; i < count; ++i) {
    int rc = v_packed_fwd(&L[i].desc, L[i].X, L[i].Wq_packed, L[i].s16, L[i].z, L[i].Y);
    if (rc == EQAT_OK) rc = v_packed_fwd(&L[i].desc, L[i].dY, L[i].Wq_packed, L[i].s16, L[i].z, L[i].dX);
    if (rc == EQAT_OK)
      rc = v_packed_bwd_ds(&L[i].desc, L[i].X, L[i].dY, L[i].Wq_packed, L[i].z, L[i].s16, L[i].ds, L[i].dz,
                           L[i].workspace, L[i].workspace_bytes);
    if (rc != EQAT_OK) {
      if (h_failed != nullptr) *h_failed = i;
      return rc;
    }
  }
  for (int i = 0; i < count; ++i) {
    int rc = qlinear_packed_fwd(&L[i].desc, L[i].X, L[i].Wq_packed, L[i].s16, L[i].z, L[i].Y, stream);
    if (rc == EQAT_OK) rc = qlinear_packed_bwd_dx(&L[i].desc, L[i].dY, L[i].Wq_packed, L[i].s16, L[i].z, L[i].dX, stream);
    if (rc == EQAT_OK)
      rc = qlinear_packed_bwd_ds(&L[i].desc, L[i].X, L[i].dY, L[i].Wq_packed, L[i].z, L[i].s16, L[i].ds, L[i].dz,
                                 L[i].workspace, L[i].workspace_bytes, stream);
    if (rc != EQAT_OK) {
      if (h_failed != nullptr) *h_failed = i;
      return rc;
    }
  }
  return EQAT_OK;
}

}  // extern "C"
