// extern "C" entry points of the token-wise operators: argument checking, launch order.
#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "layer.cuh"

using namespace sparsp;

#define SPARSP_TRY(x)             \
  do {                            \
    int rc__ = (x);               \
    if (rc__ != SPARSP_OK) return rc__; \
  } while (0)

namespace {

#define SPARSP_REFUSE(code, ...) \
  do {                           \
    set_error(__VA_ARGS__);      \
    return code;                 \
  } while (0)

int need(const void* p, const char* name, size_t align) {
  if (!p) SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "%s is NULL", name);
  if ((uintptr_t)p % align) SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "%s must be %zu-byte aligned", name, align);
  return SPARSP_OK;
}
int optional(const void* p, const char* name, size_t align) { return p ? need(p, name, align) : SPARSP_OK; }

// ---- rotary ----
int check_rotary(const sparsp_rotary* r) {
  if (!r) SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "rotary is NULL");
  if (r->dtype < SPARSP_BF16 || r->dtype > SPARSP_FP32)
    SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "unknown dtype %d", r->dtype);
  if (r->pairing != SPARSP_PAIRS_INTERLEAVED && r->pairing != SPARSP_PAIRS_HALF)
    SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "unknown pairing %d", r->pairing);
  const int32_t pairs[3] = {r->pairs_t, r->pairs_h, r->pairs_w}, len[3] = {r->len_t, r->len_h, r->len_w};
  int64_t all = 0;
  for (int a = 0; a < 3; ++a) {
    if (pairs[a] < 0 || (pairs[a] > 0 && len[a] < 1))
      SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "coordinate %d has %d pairs and %d positions", a, pairs[a], len[a]);
    all += pairs[a];
  }
  if (all < 1) SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "no channel pairs to rotate");
  if (r->rot_begin < 0 || r->rot_begin + 2 * all > kMaxRotaryHeadDim)
    SPARSP_REFUSE(SPARSP_ERR_UNSUPPORTED, "rotated channels %d .. %lld outside 0 .. %d", r->rot_begin,
                  (long long)(r->rot_begin + 2 * all), kMaxRotaryHeadDim);
  return SPARSP_OK;
}

// ---- layer norm ----
int check_norm(const sparsp_norm* n) {
  if (!n) SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "norm is NULL");
  if (n->dtype < SPARSP_BF16 || n->dtype > SPARSP_FP32)
    SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "unknown dtype %d", n->dtype);
  if (n->weight_dtype != n->dtype && n->weight_dtype != SPARSP_FP32)
    SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "weight_dtype %d is neither dtype nor fp32", n->weight_dtype);
  if (n->rows < 0 || n->rows_per_group < 0 || n->dim < 1)
    SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "rows, rows_per_group or dim is negative or zero");
  if (n->dim > kMaxNormDim) SPARSP_REFUSE(SPARSP_ERR_UNSUPPORTED, "dim %d above %d", n->dim, kMaxNormDim);
  if (n->stride_x < n->dim || n->stride_y < n->dim)
    SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "row strides must be at least dim");
  if (!(n->eps >= 0.0f) || std::isinf(n->eps)) SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "eps must be finite and >= 0");
  if (n->rows > (1LL << 37)) SPARSP_REFUSE(SPARSP_ERR_UNSUPPORTED, "%lld rows are too many", (long long)n->rows);
  if (norm_groups(*n) * ((n->dim + 7) / 8) > 0x7fffffffLL)
    SPARSP_REFUSE(SPARSP_ERR_UNSUPPORTED, "%lld groups of rows are too many", (long long)norm_groups(*n));
  return SPARSP_OK;
}

// ---- gated feed-forward ----
// Tiles of the outputs are written while others of the inputs are still to be read.
int apart(std::initializer_list<const void*> outputs, std::initializer_list<const void*> inputs) {
  for (auto o = outputs.begin(); o != outputs.end(); ++o) {
    if (*o == nullptr) continue;
    if (std::find(inputs.begin(), inputs.end(), *o) != inputs.end() || std::find(o + 1, outputs.end(), *o) != outputs.end())
      SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "an output may not be an input or another output");
  }
  return SPARSP_OK;
}

int check_ffn(const sparsp_ffn* f) {
  if (!f) SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "ffn is NULL");
  if (f->dtype != SPARSP_BF16 && f->dtype != SPARSP_FP16)
    SPARSP_REFUSE(SPARSP_ERR_UNSUPPORTED, "dtype %d unsupported (bf16 or fp16)", f->dtype);
  if (f->activation < SPARSP_ACT_SILU || f->activation > SPARSP_ACT_GELU)
    SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "unknown activation %d", f->activation);
  if (f->tokens < 0 || f->dim < 1 || f->hidden < 1)
    SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "tokens, dim or hidden is negative or zero");
  if (f->tokens > 0x7fffff00LL) SPARSP_REFUSE(SPARSP_ERR_UNSUPPORTED, "%lld tokens are too many", (long long)f->tokens);
  if (f->dim % 8 || f->hidden % 8)
    SPARSP_REFUSE(SPARSP_ERR_UNSUPPORTED, "dim %d and hidden %d must be multiples of 8", f->dim, f->hidden);
  if (f->hidden > (1 << 28) || f->dim > (1 << 28)) SPARSP_REFUSE(SPARSP_ERR_UNSUPPORTED, "dim or hidden above 2^28");
  if (f->stride_x < f->dim || f->stride_h < f->hidden || f->stride_w < f->dim || f->stride_x % 8 || f->stride_h % 8 ||
      f->stride_w % 8)
    SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "row strides must be multiples of 8 elements and not less than a row");
  const int64_t most = 1LL << 38;  // bytes of a stride that a tensor map holds: 2^40
  if (f->stride_x > most || f->stride_h > most || f->stride_w > most)
    SPARSP_REFUSE(SPARSP_ERR_UNSUPPORTED, "a row stride is above 2^38 elements");
  return SPARSP_OK;
}

}  // namespace

extern "C" {

int sparsp_rotary_frequencies(int32_t n_pairs, double theta, int32_t scaling, double factor, double original_length,
                              double beta_fast, double beta_slow, double* inv_freq, double* amplitude) {
  if (n_pairs < 0 || (n_pairs > 0 && !inv_freq)) SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "bad n_pairs or NULL inv_freq");
  if (!(theta > 1.0) || std::isinf(theta)) SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "theta %g must be above 1", theta);
  if (scaling < SPARSP_SCALING_NONE || scaling > SPARSP_SCALING_YARN)
    SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "unknown scaling %d", scaling);
  const bool yarn = scaling == SPARSP_SCALING_YARN;
  if (scaling != SPARSP_SCALING_NONE && (!(factor >= 1.0) || std::isinf(factor)))
    SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "factor %g must be at least 1", factor);
  if (yarn && (!(original_length >= 1.0) || std::isinf(original_length)))
    SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "original_length %g must be at least 1", original_length);
  if (yarn && (!(beta_slow > 0.0) || !(beta_fast > beta_slow) || std::isinf(beta_fast)))
    SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "beta_fast %g must be above beta_slow %g, and that above 0", beta_fast,
                  beta_slow);
  const int n = n_pairs;
  double base = theta, low = 0.0, high = 0.0;
  if (scaling == SPARSP_SCALING_NTK && n > 1) base = theta * std::pow(factor, (double)n / (n - 1));
  if (yarn) {
    const double tau = 6.283185307179586476925286766559;
    auto at = [&](double beta) { return n * std::log(original_length / (tau * beta)) / std::log(theta); };
    low = std::max(std::floor(at(beta_fast)), 0.0);
    // the limit is the head's last rotated channel, not its last pair, as published: it matters where even the slowest
    // pair turns more than beta_slow times, and pairs past the last are then part of the ramp
    high = std::min(std::ceil(at(beta_slow)), 2.0 * n - 1.0);
  }
  for (int i = 0; i < n; ++i) {
    double f = std::pow(base, -(double)i / n);
    if (scaling == SPARSP_SCALING_LINEAR) f /= factor;
    if (yarn) {
      const double past = std::min(std::max((i - low) / std::max(high - low, 0.001), 0.0), 1.0);
      f = f * (1.0 - past) + f / factor * past;
    }
    inv_freq[i] = f;
  }
  if (amplitude) *amplitude = yarn ? 0.1 * std::log(factor) + 1.0 : 1.0;
  return SPARSP_OK;
}

int sparsp_rotary_table_bytes(const sparsp_rotary* rotary, int64_t* bytes) {
  SPARSP_TRY(check_rotary(rotary));
  if (!bytes) SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = 0;
  const int32_t pairs[3] = {rotary->pairs_t, rotary->pairs_h, rotary->pairs_w};
  const int32_t len[3] = {rotary->len_t, rotary->len_h, rotary->len_w};
  for (int a = 0; a < 3; ++a) *bytes += pairs[a] > 0 ? (int64_t)pairs[a] * len[a] * 8 : 0;
  return SPARSP_OK;
}

int sparsp_rotary_table(const sparsp_rotary* rotary, const double* inv_freq, double amplitude, float* table,
                        void* stream) {
  SPARSP_TRY(check_rotary(rotary));
  SPARSP_TRY(need(inv_freq, "inv_freq", 8));
  SPARSP_TRY(need(table, "table", 16));
  if (!std::isfinite(amplitude)) SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "amplitude is not finite");
  return launch_rotary_table(*rotary, inv_freq, amplitude, table, (cudaStream_t)stream);
}

int sparsp_rotary_apply(const sparsp_shape* shape, const sparsp_rotary* rotary, const float* table,
                        const int32_t* positions, int64_t positions_stride_batch, int32_t origin_t, int32_t origin_h,
                        int32_t origin_w, const void* Q, const void* K, void* Q_out, void* K_out, int32_t inverse,
                        void* workspace, void* stream) {
  SPARSP_TRY(check_rotary(rotary));
  if (!shape) SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "shape is NULL");
  const sparsp_shape& s = *shape;
  if (s.batch < 1 || s.heads < 1 || s.head_dim < 1 || s.grid_t < 1 || s.grid_h < 1 || s.grid_w < 1 || s.n_text < 0)
    SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "shape has a non-positive dimension");
  if (s.head_dim % 8 || s.head_dim > kMaxRotaryHeadDim)
    SPARSP_REFUSE(SPARSP_ERR_UNSUPPORTED, "head_dim %d unsupported (a multiple of 8 up to %d)", s.head_dim,
                  kMaxRotaryHeadDim);
  // each factor is below 2^31 and the product of two below 2^62
  const int64_t frame = (int64_t)s.grid_h * s.grid_w;
  if (frame > 0x7fffffffLL || frame * s.grid_t + s.n_text > 0x7fffffffLL ||
      (frame * s.grid_t + s.n_text) * s.batch > 0x7fffffffLL)
    SPARSP_REFUSE(SPARSP_ERR_UNSUPPORTED, "batch * tokens must be below 2^31");
  if (s.stride_token < s.head_dim || s.stride_token % 8 || s.stride_head % 8 || s.stride_batch % 8 ||
      (s.heads > 1 && s.stride_head < 1) || (s.batch > 1 && s.stride_batch < 1))
    SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG,
                  "strides must be positive multiples of 8 elements with stride_token >= head_dim");
  const int32_t pairs[3] = {rotary->pairs_t, rotary->pairs_h, rotary->pairs_w};
  const int32_t len[3] = {rotary->len_t, rotary->len_h, rotary->len_w};
  const int32_t grid[3] = {s.grid_t, s.grid_h, s.grid_w}, origin[3] = {origin_t, origin_h, origin_w};
  if (rotary->rot_begin + 2 * (pairs[0] + pairs[1] + pairs[2]) > s.head_dim)
    SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "%d pairs from channel %d do not fit head_dim %d",
                  pairs[0] + pairs[1] + pairs[2], rotary->rot_begin, s.head_dim);
  SPARSP_TRY(need(table, "table", 16));
  SPARSP_TRY(need(Q, "Q", 16));
  SPARSP_TRY(need(Q_out, "Q_out", 16));
  if ((K == nullptr) != (K_out == nullptr)) SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "K and K_out go together");
  SPARSP_TRY(optional(K, "K", 16));
  SPARSP_TRY(optional(K_out, "K_out", 16));
  SPARSP_TRY(optional(positions, "positions", 4));
  SPARSP_TRY(optional(workspace, "workspace", 256));
  if (positions) {
    SPARSP_TRY(need(workspace, "workspace", 256));
    if (positions_stride_batch < 0) SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "positions_stride_batch is negative");
  } else {
    for (int a = 0; a < 3; ++a)
      if (pairs[a] > 0 && (origin[a] < 0 || (int64_t)origin[a] + grid[a] > len[a]))
        SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "coordinate %d: positions %d .. %lld are not in the table's 0 .. %d", a,
                      origin[a], (long long)origin[a] + grid[a] - 1, len[a] - 1);
  }
  return launch_rotary(s, *rotary, table, positions, positions_stride_batch, origin, Q, K, Q_out, K_out, inverse != 0,
                       (int32_t*)workspace, (cudaStream_t)stream);
}

int sparsp_layer_norm_fwd(const sparsp_norm* norm, const void* X, const void* weight, const void* bias, void* Y,
                          float* mean, float* rstd, void* stream) {
  SPARSP_TRY(check_norm(norm));
  if ((mean == nullptr) != (rstd == nullptr)) SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "mean and rstd go together");
  if (norm->rows == 0) return SPARSP_OK;
  const size_t e = element_bytes(norm->dtype), ew = element_bytes(norm->weight_dtype);
  SPARSP_TRY(need(X, "X", e));
  SPARSP_TRY(need(Y, "Y", e));
  if (X == Y && norm->stride_x != norm->stride_y)
    SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "Y may be X only when the strides are equal");
  SPARSP_TRY(optional(weight, "weight", ew));
  SPARSP_TRY(optional(bias, "bias", ew));
  SPARSP_TRY(optional(mean, "mean", 4));
  SPARSP_TRY(optional(rstd, "rstd", 4));
  return launch_norm_fwd(*norm, X, weight, bias, Y, mean, rstd, (cudaStream_t)stream);
}

int sparsp_layer_norm_workspace_bytes(const sparsp_norm* norm, int64_t* bytes) {
  SPARSP_TRY(check_norm(norm));
  if (!bytes) SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = norm_workspace_bytes(*norm);
  return SPARSP_OK;
}

int sparsp_layer_norm_bwd(const sparsp_norm* norm, const void* dY, const void* X, const void* weight,
                          const float* mean, const float* rstd, void* dX, void* dweight, void* dbias, void* workspace,
                          void* stream) {
  SPARSP_TRY(check_norm(norm));
  const size_t e = element_bytes(norm->dtype), ew = element_bytes(norm->weight_dtype);
  if (norm->rows > 0) {
    SPARSP_TRY(need(dY, "dY", e));
    SPARSP_TRY(need(X, "X", e));
    SPARSP_TRY(need(dX, "dX", e));
    SPARSP_TRY(need(mean, "mean", 4));
    SPARSP_TRY(need(rstd, "rstd", 4));
    if (dX == dY && norm->stride_x != norm->stride_y)
      SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "dX may be dY only when the strides are equal");
    if (dX == X) SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "dX may not be X");
  }
  SPARSP_TRY(optional(weight, "weight", ew));
  SPARSP_TRY(optional(dweight, "dweight", ew));
  SPARSP_TRY(optional(dbias, "dbias", ew));
  if (dweight || dbias) SPARSP_TRY(need(workspace, "workspace", 256));
  return launch_norm_bwd(*norm, dY, X, weight, mean, rstd, dX, dweight, dbias, (char*)workspace,
                         (cudaStream_t)stream);
}

int sparsp_gated_ffn_workspace_bytes(const sparsp_ffn* ffn, int32_t backward, int64_t* bytes) {
  SPARSP_TRY(check_ffn(ffn));
  if (!bytes) SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = ffn_workspace_bytes(*ffn, backward != 0);
  return SPARSP_OK;
}

int sparsp_gated_ffn_fwd(const sparsp_ffn* ffn, const void* X, const void* Wgate, const void* Wup, void* H, void* gate,
                         void* up, void* workspace, void* stream) {
  SPARSP_TRY(check_ffn(ffn));
  if ((gate == nullptr) != (up == nullptr)) SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "gate and up go together");
  if (ffn->tokens == 0) return SPARSP_OK;
  SPARSP_TRY(need(X, "X", 16));
  SPARSP_TRY(need(Wgate, "Wgate", 16));
  SPARSP_TRY(need(Wup, "Wup", 16));
  SPARSP_TRY(need(H, "H", 16));
  SPARSP_TRY(optional(gate, "gate", 16));
  SPARSP_TRY(optional(up, "up", 16));
  SPARSP_TRY(apart({H, gate, up}, {X, Wgate, Wup}));
  SPARSP_TRY(need(workspace, "workspace", 256));
  return launch_ffn_fwd(*ffn, X, Wgate, Wup, H, gate, up, (char*)workspace, (cudaStream_t)stream);
}

int sparsp_gated_ffn_bwd(const sparsp_ffn* ffn, const void* dH, const void* X, const void* Wgate, const void* Wup,
                         const void* gate, const void* up, void* dX, void* dWgate, void* dWup, void* workspace,
                         void* stream) {
  SPARSP_TRY(check_ffn(ffn));
  if ((dWgate == nullptr) != (dWup == nullptr)) SPARSP_REFUSE(SPARSP_ERR_INVALID_ARG, "dWgate and dWup go together");
  SPARSP_TRY(optional(dWgate, "dWgate", 16));
  SPARSP_TRY(optional(dWup, "dWup", 16));
  if (ffn->tokens > 0 && (dX || dWgate)) {
    SPARSP_TRY(need(dH, "dH", 16));
    SPARSP_TRY(need(gate, "gate", 16));
    SPARSP_TRY(need(up, "up", 16));
    SPARSP_TRY(need(workspace, "workspace", 256));
    if (dX) {
      SPARSP_TRY(need(dX, "dX", 16));
      SPARSP_TRY(need(Wgate, "Wgate", 16));
      SPARSP_TRY(need(Wup, "Wup", 16));
    }
    if (dWgate) SPARSP_TRY(need(X, "X", 16));
    SPARSP_TRY(apart({dX, dWgate, dWup}, {dWgate ? X : nullptr, dX ? Wgate : nullptr, dX ? Wup : nullptr}));
  }
  return launch_ffn_bwd(*ffn, dH, X, Wgate, Wup, gate, up, dX, dWgate, dWup, (char*)workspace, (cudaStream_t)stream);
}

}  // extern "C"
