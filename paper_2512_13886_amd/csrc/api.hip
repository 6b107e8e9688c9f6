// extern "C" entry points of liboptima.so: argument validation, then the
// launch sequences in the other sources.
#include "common.h"

namespace optima {
size_t hessian_workspace_bytes(int64_t n_tok, int64_t d, int dtype);
optima_status hessian_accumulate(const void* X, int dtype, int64_t n_tok, int64_t d, float* H,
                                 int accumulate, void* ws, hipStream_t s);
optima_status hessian_damp(float* H, int64_t d, float rel, float* lambda_out, hipStream_t s);
optima_status hessian_jacobi(float* H, int64_t d, float* D, hipStream_t s);
size_t spectral_norm_workspace_bytes(int64_t d, int block);
optima_status spectral_norm(const float* H, int64_t d, const float* V0, int block, int max_iters,
                            float tol, void* ws, float* lambda_max, int32_t* iters,
                            hipStream_t s);
optima_status spectral_norm_noalloc(const float* H, int64_t d, const float* V0, int block,
                                    int max_iters, float tol, float* lambda_max, int32_t* iters,
                                    hipStream_t s);
size_t spectral_lanczos_workspace_bytes(int64_t d, int max_steps);
optima_status spectral_lanczos(const float* H, int64_t d, const float* v0, int max_steps,
                               float tol, void* ws, float* lambda_max, int32_t* steps,
                               hipStream_t s);
optima_status wanda_mask(const float* W0, int64_t n_cols, int64_t d, const void* col_sq,
                         int col_dtype, int64_t col_stride, int pattern, double sparsity,
                         uint8_t* mask, hipStream_t s);
size_t qp_workspace_bytes(int64_t d, int64_t n_cols);
size_t linear_forward_workspace_bytes(int64_t n_tok, int64_t d_in, int64_t d_out);
optima_status linear_forward(const void* X, int64_t n_tok, int64_t d_in, const float* W,
                             int64_t d_out, int act, void* Y, int y_dtype, const float* Y_ref,
                             double* err_out, void* ws, hipStream_t s);
optima_status qp_solve(const float* H, int64_t d, const float* lambda_max, const float* W0,
                       const uint8_t* mask, int64_t n_cols, const optima_solver_opts& o, void* ws,
                       float* W_out, const optima_solve_stats& stats, optima_solve_info* info,
                       hipStream_t s);
optima_status rms_norm(const void* X, int64_t ldx, const void* R, int64_t ldr, int dtype, int64_t n,
                       int64_t d, const void* w, int w_dtype, float eps, void* S, int64_t lds,
                       void* Y, int64_t ldy, int y_dtype, float* scales, int64_t group,
                       hipStream_t s);
size_t rms_norm_backward_workspace_bytes(int64_t n, int64_t d);
optima_status rms_norm_backward(const void* S, int64_t lds, const void* w, int w_dtype,
                                const void* dY, int64_t lddy, const void* dS, int64_t ldds,
                                int dtype, int64_t n, int64_t d, float eps, void* dX, int64_t lddx,
                                float* dweight, int accumulate, void* ws, hipStream_t s);
size_t gated_forward_workspace_bytes(int64_t n_tok, int64_t d, int64_t ff);
optima_status gated_forward(const void* X, int64_t ldx, int64_t n_tok, int64_t d, const void* Wg,
                            const void* Wu, int64_t ff, int act, void* H, int64_t ldh, int h_dtype,
                            void* G, int64_t ldg, void* U, int64_t ldu, void* ws, hipStream_t s);
size_t gated_backward_workspace_bytes(int64_t n_tok, int64_t d, int64_t ff);
optima_status gated_backward(const void* X, int64_t ldx, int64_t n_tok, int64_t d, const void* Wg,
                             const void* Wu, int64_t ff, int act, const void* G, int64_t ldg,
                             const void* U, int64_t ldu, const void* dH, int64_t lddh, void* dX,
                             int64_t lddx, int dx_dtype, void* dWg, void* dWu, int dw_dtype,
                             const uint8_t* mask_g, const uint8_t* mask_u, int accumulate, void* ws,
                             hipStream_t s);
optima_status w4_pack(const void* W, int dtype, int64_t n, int64_t d, int64_t group, void* Q,
                      void* scales, hipStream_t s);
optima_status w4_linear(const void* X, int64_t ldx, const float* x_scales, int64_t x_group,
                        int64_t n_tok, int64_t d, const void* Q, const void* sc, const void* Q2,
                        const void* sc2, int64_t group, int64_t d_out, int act, void* Y,
                        int64_t ldy, int y_dtype, void* ws, hipStream_t s);
size_t w4_workspace_bytes(int64_t n_tok, int64_t d, int64_t d_out, int mats);
size_t mx4_row_bytes(int64_t d);
size_t mx4_scale_bytes(int64_t d);
optima_status mx4_pack(const void* X, int64_t ldx, int dtype, int64_t n, int64_t d, void* Q,
                       void* scales, hipStream_t s);
optima_status mx4_unpack(const void* Q, const void* scales, int64_t n, int64_t d, void* Y,
                         int64_t ldy, int dtype, hipStream_t s);
size_t mx4_workspace_bytes(int64_t n_tok, int64_t d, int64_t d_out);
optima_status mx4_linear(const void* X, int64_t ldx, const void* x_scales, int64_t n_tok, int64_t d,
                         const void* Q, const void* scales, int64_t d_out, void* Y, int64_t ldy,
                         int y_dtype, void* ws, hipStream_t s);
size_t token_logprobs_workspace_bytes(int64_t n, int64_t vocab, int64_t k);
optima_status token_logprobs(const void* X, int64_t ldx, int dtype, int64_t n, int64_t vocab,
                             const int64_t* tokens, float scale, float* logp, float* lse,
                             float* entropy, int64_t k, int64_t* top_index, float* top_logp,
                             void* ws, hipStream_t s);
optima_status token_logprobs_backward(const void* X, int64_t ldx, int dtype, int64_t n,
                                      int64_t vocab, const int64_t* tokens, float scale,
                                      const float* lse, const float* entropy, const float* dlogp,
                                      const float* dentropy, const float* dlse, void* dX,
                                      int64_t lddx, hipStream_t s);
}  // namespace optima

namespace {
// Sizes are kept within 32-bit tile and row indices.
constexpr int64_t kMaxDim = int64_t(1) << 20;
constexpr int64_t kMaxCols = int64_t(1) << 24;

bool overlaps(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

// A token matrix or another array as a call sees it: `rows` rows of `cols`
// elements of `esz` bytes, `ld` elements apart.
struct Span {
  const void* p;
  int64_t rows, cols, ld;
  int64_t esz;
  size_t bytes() const {
    return !p || rows < 1 ? 0 : (size_t(rows - 1) * size_t(ld) + size_t(cols)) * size_t(esz);
  }
  bool aligned() const { return reinterpret_cast<uintptr_t>(p) % size_t(esz) == 0; }
  // A pointer where there are rows, elements aligned, and rows that do not overlap.
  bool good() const {
    return ld >= cols && ld < (int64_t(1) << 31) && (rows < 1 || p) && aligned();
  }
  // Whether any element is in both. Rows of one pitch may lie between each other's, as the
  // halves of one buffer's columns do; of different pitches the whole extents count.
  bool meets(const Span& o) const {
    if (!bytes() || !o.bytes() || !overlaps(p, bytes(), o.p, o.bytes())) return false;
    const int64_t pitch = (rows > 1 ? ld * esz : o.ld * o.esz), a = cols * esz, b = o.cols * o.esz;
    if ((o.rows > 1 && o.ld * o.esz != pitch) || a > pitch || b > pitch) return true;
    const int64_t apart = int64_t(reinterpret_cast<uintptr_t>(o.p) - reinterpret_cast<uintptr_t>(p));
    const int64_t down = apart >= 0 ? apart / pitch : -((pitch - 1 - apart) / pitch);
    // o's first row begins `rest` bytes into the pitch of row `down`. Its rows reach into
    // those of row `down` from there and into row down + 1 from before it.
    const int64_t rest = apart - down * pitch;
    auto rows_apart = [&](int64_t k) { return k < rows && -k < o.rows; };
    return (rest < a && rows_apart(down)) || (pitch - rest < b && rows_apart(down + 1));
  }
  // The same elements in the same places: a kernel that reads a row before it
  // writes it may work in place.
  bool same(const Span& o) const { return p == o.p && ld == o.ld && esz == o.esz; }
};

constexpr int64_t kMaxTok = (int64_t(1) << 31) - 1;

int64_t esize(int dtype) {
  return dtype == OPTIMA_DTYPE_F32 ? 4 : dtype == OPTIMA_DTYPE_BF16 ? 2 : 1;
}
bool f32_or_bf16(int dtype) { return dtype == OPTIMA_DTYPE_F32 || dtype == OPTIMA_DTYPE_BF16; }
bool group_ok(int64_t group) { return group == 32 || group == 64 || group == 128; }

// Sizes of the gated product: the largest launch, which copies rows in blocks of 256
// threads, two for 64 x 64 values, stays below 2^32 threads.
bool gated_sizes(int64_t n_tok, int64_t d_in, int64_t d_ff) {
  auto tiles = [](int64_t a, int64_t b) { return (a / 64 + 1) * (b / 64 + 1); };
  return n_tok >= 0 && n_tok <= kMaxTok && d_in >= 1 && d_in <= kMaxDim && d_ff >= 1 &&
         d_ff <= kMaxDim &&
         2 * tiles(n_tok, std::max(d_in, d_ff)) + 4 * tiles(d_in, d_ff) < (int64_t(1) << 24);
}

optima_status w4_call(const void* X, int64_t ldx, int x_dtype, const float* x_scales,
                      int64_t x_group, int64_t n_tok, int64_t d, const void* Q, const void* scales,
                      const void* Q2, const void* scales2, int64_t group, int64_t d_out, int act,
                      void* Y, int64_t ldy, int y_dtype, void* ws, size_t ws_bytes,
                      hipStream_t stream) {
  if (x_dtype != OPTIMA_DTYPE_BF16 && x_dtype != OPTIMA_DTYPE_I8) return OPTIMA_E_UNSUPPORTED;
  if (!f32_or_bf16(y_dtype)) return OPTIMA_E_UNSUPPORTED;
  if (n_tok < 0 || n_tok > (int64_t(1) << 21) || d < 1 || d > kMaxDim || d_out < 1 ||
      d_out > kMaxCols || !group_ok(group))
    return OPTIMA_E_INVAL;
  const bool i8 = x_dtype == OPTIMA_DTYPE_I8;
  if (i8 ? x_group != 0 && x_group != group : x_group != 0 || x_scales) return OPTIMA_E_INVAL;
  if (!Q || !scales || !optima::aligned16(Q) || !optima::aligned16(Q2)) return OPTIMA_E_INVAL;
  const int64_t groups = (d + group - 1) / group, x_groups = x_group ? groups : 1;
  const Span x{X, n_tok, d, ldx, esize(x_dtype)}, y{Y, n_tok, d_out, ldy, esize(y_dtype)};
  const Span xs{x_scales, n_tok, x_groups, x_groups, 4};
  if (!x.good() || !y.good() || (i8 && !xs.good())) return OPTIMA_E_INVAL;
  const int64_t row = int64_t(optima_w4_row_bytes(d));
  for (int k = 0; k < 2; ++k) {
    const Span q{k ? Q2 : Q, d_out, row, row, 1};
    const Span sc{k ? scales2 : scales, d_out, groups, groups, 2};
    if (!sc.aligned() || y.meets(q) || y.meets(sc)) return OPTIMA_E_INVAL;
  }
  if (y.meets(x) || (i8 && y.meets(xs))) return OPTIMA_E_INVAL;
  const size_t need = optima::w4_workspace_bytes(n_tok, d, d_out, Q2 ? 2 : 1);
  if (need && (!ws || !optima::aligned16(ws) || ws_bytes < need)) return OPTIMA_E_WORKSPACE;
  if (n_tok == 0) return OPTIMA_OK;
  return optima::w4_linear(X, ldx, i8 ? x_scales : nullptr, x_group, n_tok, d, Q, scales, Q2,
                           scales2, group, d_out, act, Y, ldy, y_dtype, ws, stream);
}

// Rows in pieces of 256 values, 32 threads each, and 64 x 64 tiles of outputs of 256 threads: a launch
// has fewer than 2^32 threads.
bool mx4_rows(int64_t n, int64_t d) {
  return n >= 0 && n < (int64_t(1) << 27) && d >= 1 && d <= kMaxDim &&
         n * ((d + 255) / 256) <= (int64_t(1) << 27) - 8;
}
bool mx4_sizes(int64_t n_tok, int64_t d, int64_t d_out) {
  return n_tok >= 0 && n_tok <= (int64_t(1) << 21) && d >= 1 && d <= kMaxDim && d_out >= 1 &&
         d_out <= kMaxCols && ((n_tok + 63) / 64) * ((d_out + 63) / 64) < (int64_t(1) << 24) - 8;
}
// Codes and scales of n rows.
Span mx4_codes(const void* Q, int64_t n, int64_t d) {
  const int64_t row = int64_t(optima::mx4_row_bytes(d));
  return {Q, n, row, row, 1};
}
Span mx4_scales(const void* scales, int64_t n, int64_t d) {
  const int64_t row = int64_t(optima::mx4_scale_bytes(d)) / 4;
  return {scales, n, row, row, 4};
}
bool logprob_sizes(int64_t n, int64_t vocab) {
  return n >= 0 && n <= kMaxTok && vocab >= 1 && vocab <= kMaxDim;
}
bool positive(float v) { return v > 0.f && v < __builtin_inff(); }
}  // namespace

extern "C" {

const char* optima_status_string(optima_status status) {
  switch (status) {
    case OPTIMA_OK: return "OPTIMA_OK";
    case OPTIMA_E_INVAL: return "OPTIMA_E_INVAL: invalid argument";
    case OPTIMA_E_HIP: return "OPTIMA_E_HIP: HIP runtime error";
    case OPTIMA_E_NONFINITE: return "OPTIMA_E_NONFINITE: NaN or Inf in the input";
    case OPTIMA_E_WORKSPACE: return "OPTIMA_E_WORKSPACE: workspace missing or too small";
    case OPTIMA_E_UNSUPPORTED: return "OPTIMA_E_UNSUPPORTED: unsupported dtype or device";
    default: return "OPTIMA: unknown status";
  }
}

int optima_abi_version(void) { return 13; }

size_t optima_hessian_workspace_bytes(int64_t n_tok, int64_t d, int dtype) {
  if (n_tok < 0 || d < 1 || d > kMaxDim) return 0;
  if (dtype != OPTIMA_DTYPE_F32 && dtype != OPTIMA_DTYPE_BF16) return 0;
  return optima::hessian_workspace_bytes(n_tok, d, dtype);
}

optima_status optima_hessian_accumulate(const void* X, int dtype, int64_t n_tok, int64_t d,
                                        float* H, int accumulate, void* ws, size_t ws_bytes,
                                        hipStream_t stream) {
  if (dtype != OPTIMA_DTYPE_F32 && dtype != OPTIMA_DTYPE_BF16) return OPTIMA_E_UNSUPPORTED;
  if (!H || n_tok < 0 || d < 1 || d > kMaxDim) return OPTIMA_E_INVAL;
  if (n_tok > 0 && !X) return OPTIMA_E_INVAL;
  const size_t esz = dtype == OPTIMA_DTYPE_BF16 ? 2 : 4;
  if (n_tok > 0 && !optima::aligned16(X)) return OPTIMA_E_INVAL;
  if (X && overlaps(X, size_t(n_tok) * size_t(d) * esz, H, size_t(d) * size_t(d) * 4))
    return OPTIMA_E_INVAL;
  if (n_tok > 0) {
    const size_t need = optima::hessian_workspace_bytes(n_tok, d, dtype);
    if (!ws || ws_bytes < need) return OPTIMA_E_WORKSPACE;
  }
  return optima::hessian_accumulate(X, dtype, n_tok, d, H, accumulate ? 1 : 0, ws, stream);
}

optima_status optima_hessian_damp(float* H, int64_t d, float rel_damp, float* lambda_out,
                                  hipStream_t stream) {
  if (!H || !lambda_out || d < 1 || d > kMaxDim) return OPTIMA_E_INVAL;
  if (!(rel_damp >= 0.f)) return OPTIMA_E_INVAL;
  return optima::hessian_damp(H, d, rel_damp, lambda_out, stream);
}

optima_status optima_hessian_jacobi(float* H, int64_t d, float* scale_out, hipStream_t stream) {
  if (!H || !scale_out || d < 1 || d > kMaxDim) return OPTIMA_E_INVAL;
  if ((reinterpret_cast<uintptr_t>(H) & 3) || (reinterpret_cast<uintptr_t>(scale_out) & 3))
    return OPTIMA_E_INVAL;
  if (overlaps(H, size_t(d) * size_t(d) * 4, scale_out, size_t(d) * 4)) return OPTIMA_E_INVAL;
  return optima::hessian_jacobi(H, d, scale_out, stream);
}

size_t optima_spectral_norm_workspace_bytes(int64_t d, int block) {
  if (d < 1 || d > kMaxDim || block < 1 || block > OPTIMA_SPECTRAL_MAX_BLOCK) return 0;
  return optima::spectral_norm_workspace_bytes(d, block);
}

optima_status optima_spectral_norm(const float* H, int64_t d, const float* V0, int block,
                                   int max_iters, float tol, void* ws, size_t ws_bytes,
                                   float* lambda_max, int32_t* iters, hipStream_t stream) {
  if (!H || !V0 || !lambda_max || d < 1 || d > kMaxDim || max_iters < 1 || !(tol >= 0.f))
    return OPTIMA_E_INVAL;
  if (block < 1 || block > OPTIMA_SPECTRAL_MAX_BLOCK) return OPTIMA_E_INVAL;
  if ((reinterpret_cast<uintptr_t>(V0) & 3) || (reinterpret_cast<uintptr_t>(H) & 3))
    return OPTIMA_E_INVAL;
  if (!ws || ws_bytes < optima::spectral_norm_workspace_bytes(d, block))
    return OPTIMA_E_WORKSPACE;
  return optima::spectral_norm(H, d, V0, block, max_iters, tol, ws, lambda_max, iters, stream);
}

optima_status optima_spectral_norm_noalloc(const float* H, int64_t d, const float* V0, int block,
                                           int max_iters, float tol, float* lambda_max,
                                           int32_t* iters, hipStream_t stream) {
  if (!H || !V0 || !lambda_max || d < 1 || d > kMaxDim || max_iters < 1 || !(tol >= 0.f))
    return OPTIMA_E_INVAL;
  if (block < 1 || block > OPTIMA_SPECTRAL_MAX_BLOCK) return OPTIMA_E_INVAL;
  if ((reinterpret_cast<uintptr_t>(V0) & 3) || (reinterpret_cast<uintptr_t>(H) & 3))
    return OPTIMA_E_INVAL;
  if (d > OPTIMA_SPECTRAL_NOALLOC_MAX_DIM) return OPTIMA_E_WORKSPACE;
  return optima::spectral_norm_noalloc(H, d, V0, block, max_iters, tol, lambda_max, iters,
                                       stream);
}

size_t optima_spectral_lanczos_workspace_bytes(int64_t d, int max_steps) {
  if (d < 1 || d > kMaxDim || max_steps < 1 || max_steps > OPTIMA_LANCZOS_MAX_STEPS) return 0;
  return optima::spectral_lanczos_workspace_bytes(d, max_steps);
}

optima_status optima_spectral_lanczos(const float* H, int64_t d, const float* v0, int max_steps,
                                      float tol, void* ws, size_t ws_bytes, float* lambda_max,
                                      int32_t* steps, hipStream_t stream) {
  if (!H || !v0 || !lambda_max || d < 1 || d > kMaxDim || !(tol >= 0.f)) return OPTIMA_E_INVAL;
  if (max_steps < 1 || max_steps > OPTIMA_LANCZOS_MAX_STEPS) return OPTIMA_E_INVAL;
  if ((reinterpret_cast<uintptr_t>(v0) & 3) || (reinterpret_cast<uintptr_t>(H) & 3))
    return OPTIMA_E_INVAL;
  if (!ws || ws_bytes < optima::spectral_lanczos_workspace_bytes(d, max_steps))
    return OPTIMA_E_WORKSPACE;
  return optima::spectral_lanczos(H, d, v0, max_steps, tol, ws, lambda_max, steps, stream);
}

optima_status optima_wanda_mask(const float* W0, int64_t n_cols, int64_t d, const void* col_sq,
                                int col_sq_dtype, int64_t col_sq_stride, int pattern,
                                double sparsity, uint8_t* mask, hipStream_t stream) {
  if (d < 1 || d > kMaxDim || n_cols < 0 || n_cols > kMaxCols) return OPTIMA_E_INVAL;
  if (n_cols == 0) return OPTIMA_OK;
  if (!W0 || !col_sq || !mask || col_sq_stride < 1) return OPTIMA_E_INVAL;
  if (col_sq_dtype != OPTIMA_DTYPE_F32 && col_sq_dtype != OPTIMA_DTYPE_F64)
    return OPTIMA_E_UNSUPPORTED;
  const size_t csz = col_sq_dtype == OPTIMA_DTYPE_F64 ? 8 : 4;
  if ((reinterpret_cast<uintptr_t>(W0) & 3) || (reinterpret_cast<uintptr_t>(mask) & 3) ||
      (reinterpret_cast<uintptr_t>(col_sq) % csz))
    return OPTIMA_E_INVAL;
  if (pattern == OPTIMA_MASK_2TO4) {
    if (d % 4) return OPTIMA_E_INVAL;
  } else if (pattern == OPTIMA_MASK_UNSTRUCTURED) {
    if (!(sparsity >= 0.0 && sparsity <= 1.0)) return OPTIMA_E_INVAL;
  } else {
    return OPTIMA_E_INVAL;
  }
  const size_t mbytes = size_t(n_cols) * size_t(d);
  if (overlaps(mask, mbytes, W0, mbytes * 4) ||
      overlaps(mask, mbytes, col_sq, (size_t(d - 1) * size_t(col_sq_stride) + 1) * csz))
    return OPTIMA_E_INVAL;
  return optima::wanda_mask(W0, n_cols, d, col_sq, col_sq_dtype, col_sq_stride, pattern,
                            sparsity, mask, stream);
}

size_t optima_linear_forward_workspace_bytes(int64_t n_tok, int64_t d_in, int64_t d_out) {
  if (n_tok < 0 || d_in < 64 || d_in > kMaxDim || d_in % 64 || d_out < 4 || d_out > kMaxDim ||
      d_out % 4)
    return 0;
  // one workgroup per 128 x 128 output tile; the grid stays below 2^31
  if ((n_tok + 127) / 128 * ((d_out + 127) / 128) >= (int64_t(1) << 31)) return 0;
  return optima::linear_forward_workspace_bytes(n_tok, d_in, d_out);
}

optima_status optima_linear_forward(const void* X, int64_t n_tok, int64_t d_in, const float* W,
                                    int64_t d_out, int act, void* Y, int y_dtype,
                                    const float* Y_ref, double* err_out, void* ws,
                                    size_t ws_bytes, hipStream_t stream) {
  const size_t need = optima_linear_forward_workspace_bytes(n_tok, d_in, d_out);
  if (!need) return OPTIMA_E_INVAL;
  // Nothing to do without Y or err_out; an error needs its reference (no
  // pointer is read when n_tok == 0).
  if (!W || (n_tok > 0 && !X) || (!Y && !err_out)) return OPTIMA_E_INVAL;
  if ((Y_ref && !err_out) || (err_out && n_tok > 0 && !Y_ref)) return OPTIMA_E_INVAL;
  if (act != OPTIMA_ACT_NONE && act != OPTIMA_ACT_SILU) return OPTIMA_E_INVAL;
  if (Y && y_dtype != OPTIMA_DTYPE_BF16 && y_dtype != OPTIMA_DTYPE_F32) return OPTIMA_E_INVAL;
  if ((X && !optima::aligned16(X)) || (reinterpret_cast<uintptr_t>(W) & 3)) return OPTIMA_E_INVAL;
  if (Y && (reinterpret_cast<uintptr_t>(Y) & (y_dtype == OPTIMA_DTYPE_F32 ? 15 : 7)))
    return OPTIMA_E_INVAL;
  if (Y_ref && !optima::aligned16(Y_ref)) return OPTIMA_E_INVAL;
  if (err_out && (reinterpret_cast<uintptr_t>(err_out) & 7)) return OPTIMA_E_INVAL;
  const size_t ybytes = size_t(n_tok) * size_t(d_out) * (Y && y_dtype == OPTIMA_DTYPE_BF16 ? 2 : 4);
  if (Y && (overlaps(Y, ybytes, X, size_t(n_tok) * size_t(d_in) * 2) ||
            overlaps(Y, ybytes, W, size_t(d_out) * size_t(d_in) * 4) ||
            (Y_ref && overlaps(Y, ybytes, Y_ref, size_t(n_tok) * size_t(d_out) * 4))))
    return OPTIMA_E_INVAL;
  if (!ws || ws_bytes < need) return OPTIMA_E_WORKSPACE;
  return optima::linear_forward(X, n_tok, d_in, W, d_out, act, Y, y_dtype, Y_ref, err_out, ws,
                                stream);
}

void optima_solver_opts_default(optima_solver_opts* o) {
  if (!o) return;
  o->max_iters = 100000;
  o->check_every = 64;
  o->fixed_iters = 0;
  o->eps_rel = 0.01f;
  o->eps_abs = 0.01f;
  o->beta_sufficient = 0.2f;
  o->beta_necessary = 0.8f;
  o->beta_artificial = 0.36f;
  o->step_safety = 1e-3f;
  o->restarts = 1;
  o->precision = OPTIMA_PREC_BF16X3;
  o->method = OPTIMA_METHOD_RAPDHG;
  o->col_scale = nullptr;
  o->sparse = 1;
  o->cooperative = 1;
}

size_t optima_qp_workspace_bytes(int64_t d, int64_t n_cols) {
  if (d < 1 || d > kMaxDim || n_cols < 0 || n_cols > kMaxCols) return 0;
  return optima::qp_workspace_bytes(d, n_cols);
}

optima_status optima_qp_solve_batched(const float* H, int64_t d, const float* lambda_max,
                                      const float* W0, const uint8_t* mask, int64_t n_cols,
                                      const optima_solver_opts* opts, void* ws, size_t ws_bytes,
                                      float* W_out, const optima_solve_stats* stats,
                                      optima_solve_info* info, hipStream_t stream) {
  if (!opts || d < 1 || d > kMaxDim || n_cols < 0 || n_cols > kMaxCols) return OPTIMA_E_INVAL;
  if (info) *info = optima_solve_info{};
  if (n_cols == 0) return OPTIMA_OK;
  if (opts->method != OPTIMA_METHOD_RAPDHG && opts->method != OPTIMA_METHOD_CG)
    return OPTIMA_E_INVAL;
  if (!H || !W0 || !mask || !W_out) return OPTIMA_E_INVAL;
  if (!lambda_max && opts->method == OPTIMA_METHOD_RAPDHG) return OPTIMA_E_INVAL;
  if (!optima::aligned16(H) || (reinterpret_cast<uintptr_t>(W0) & 3) ||
      (reinterpret_cast<uintptr_t>(W_out) & 3) ||
      (reinterpret_cast<uintptr_t>(opts->col_scale) & 3))
    return OPTIMA_E_INVAL;
  const size_t wbytes = size_t(n_cols) * size_t(d) * sizeof(float);
  if (overlaps(W0, wbytes, W_out, wbytes) || overlaps(H, size_t(d) * d * 4, W_out, wbytes) ||
      overlaps(mask, size_t(n_cols) * d, W_out, wbytes))
    return OPTIMA_E_INVAL;
  const optima_solver_opts& o = *opts;
  if (o.max_iters < 0 || o.check_every < 1) return OPTIMA_E_INVAL;
  if (o.sparse != 0 && o.sparse != 1) return OPTIMA_E_INVAL;
  if (o.cooperative != 0 && o.cooperative != 1) return OPTIMA_E_INVAL;
  if (o.precision != OPTIMA_PREC_FP32 && o.precision != OPTIMA_PREC_BF16X3)
    return OPTIMA_E_UNSUPPORTED;
  if (!(o.eps_rel >= 0.f) || !(o.eps_abs >= 0.f) || !(o.step_safety >= 0.f) ||
      !(o.beta_sufficient >= 0.f) || !(o.beta_necessary >= 0.f) || !(o.beta_artificial >= 0.f))
    return OPTIMA_E_INVAL;
  if (!ws || ws_bytes < optima::qp_workspace_bytes(d, n_cols)) return OPTIMA_E_WORKSPACE;
  optima_solve_stats st{};
  if (stats) st = *stats;
  return optima::qp_solve(H, d, lambda_max, W0, mask, n_cols, o, ws, W_out, st, info, stream);
}

optima_status optima_rms_norm(const void* X, int64_t ldx, const void* R, int64_t ldr, int dtype,
                              int64_t n_tok, int64_t d, const void* weight, int w_dtype,
                              float eps, void* S, int64_t lds, void* Y, int64_t ldy, int y_dtype,
                              float* scales, int64_t group, hipStream_t stream) {
  if (!f32_or_bf16(dtype) || !f32_or_bf16(w_dtype)) return OPTIMA_E_UNSUPPORTED;
  const bool i8 = y_dtype == OPTIMA_DTYPE_I8;
  if (!i8 && !f32_or_bf16(y_dtype)) return OPTIMA_E_UNSUPPORTED;
  if (n_tok < 0 || n_tok > kMaxTok || d < 1 || !(eps > 0.f) || !weight) return OPTIMA_E_INVAL;
  if (d > OPTIMA_NORM_MAX_DIM) return OPTIMA_E_UNSUPPORTED;
  if (i8 ? group != 0 && !group_ok(group) : group != 0 || scales) return OPTIMA_E_INVAL;
  const int64_t e = esize(dtype), groups = group ? (d + group - 1) / group : 1;
  const Span x{X, n_tok, d, ldx, e}, r{R, n_tok, d, ldr, e}, w{weight, 1, d, d, esize(w_dtype)};
  const Span s{S, n_tok, d, lds, e}, y{Y, n_tok, d, ldy, esize(y_dtype)};
  const Span sc{scales, n_tok, groups, groups, 4};
  if (!x.good() || !y.good() || !w.aligned() || (R && !r.good()) || (S && !s.good()) ||
      (i8 && !sc.good()))
    return OPTIMA_E_INVAL;
  for (const Span& o : {s, y}) {
    if ((o.meets(x) && !o.same(x)) || (o.meets(r) && !o.same(r)) || o.meets(w)) return OPTIMA_E_INVAL;
    if (sc.meets(o)) return OPTIMA_E_INVAL;
  }
  if (s.meets(y) || sc.meets(x) || sc.meets(r) || sc.meets(w)) return OPTIMA_E_INVAL;
  if (n_tok == 0) return OPTIMA_OK;
  return optima::rms_norm(X, ldx, R, ldr, dtype, n_tok, d, weight, w_dtype, eps, S, lds, Y, ldy,
                          y_dtype, scales, group, stream);
}

size_t optima_rms_norm_backward_workspace_bytes(int64_t n_tok, int64_t d) {
  if (n_tok < 0 || n_tok > kMaxTok || d < 1 || d > OPTIMA_NORM_MAX_DIM) return 0;
  return optima::rms_norm_backward_workspace_bytes(n_tok, d);
}

optima_status optima_rms_norm_backward(const void* S, int64_t lds, const void* weight, int w_dtype,
                                       const void* dY, int64_t lddy, const void* dS, int64_t ldds,
                                       int dtype, int64_t n_tok, int64_t d, float eps, void* dX,
                                       int64_t lddx, float* dweight, int accumulate, void* ws,
                                       size_t ws_bytes, hipStream_t stream) {
  if (!f32_or_bf16(dtype) || !f32_or_bf16(w_dtype)) return OPTIMA_E_UNSUPPORTED;
  if (n_tok < 0 || n_tok > kMaxTok || d < 1 || !(eps > 0.f) || !weight) return OPTIMA_E_INVAL;
  if (d > OPTIMA_NORM_MAX_DIM) return OPTIMA_E_UNSUPPORTED;
  const int64_t e = esize(dtype);
  const Span s{S, n_tok, d, lds, e}, dy{dY, n_tok, d, lddy, e}, ds{dS, n_tok, d, ldds, e};
  const Span dx{dX, n_tok, d, lddx, e}, w{weight, 1, d, d, esize(w_dtype)}, dw{dweight, 1, d, d, 4};
  if (!s.good() || !dy.good() || !dx.good() || (dS && !ds.good()) || !w.aligned() || !dw.aligned())
    return OPTIMA_E_INVAL;
  if (dx.meets(s) || dx.meets(w) || (dx.meets(dy) && !dx.same(dy)) || (dx.meets(ds) && !dx.same(ds)))
    return OPTIMA_E_INVAL;
  for (const Span& o : {s, dy, ds, dx, w})
    if (dw.meets(o)) return OPTIMA_E_INVAL;
  if (dweight && n_tok > 0 &&
      (!ws || (reinterpret_cast<uintptr_t>(ws) & 3) ||
       ws_bytes < optima::rms_norm_backward_workspace_bytes(n_tok, d)))
    return OPTIMA_E_WORKSPACE;
  return optima::rms_norm_backward(S, lds, weight, w_dtype, dY, lddy, dS, ldds, dtype, n_tok, d, eps,
                                   dX, lddx, dweight, accumulate ? 1 : 0, ws, stream);
}

size_t optima_gated_forward_workspace_bytes(int64_t n_tok, int64_t d_in, int64_t d_ff) {
  if (!gated_sizes(n_tok, d_in, d_ff)) return 0;
  return optima::gated_forward_workspace_bytes(n_tok, d_in, d_ff);
}

optima_status optima_gated_forward(const void* X, int64_t ldx, int64_t n_tok, int64_t d_in,
                                   const void* Wg, const void* Wu, int64_t d_ff, int act, void* H,
                                   int64_t ldh, int h_dtype, void* G, int64_t ldg, void* U,
                                   int64_t ldu, void* ws, size_t ws_bytes, hipStream_t stream) {
  if (!gated_sizes(n_tok, d_in, d_ff) || !Wg || !Wu) return OPTIMA_E_INVAL;
  if (act != OPTIMA_ACT_NONE && act != OPTIMA_ACT_SILU) return OPTIMA_E_INVAL;
  if (!f32_or_bf16(h_dtype)) return OPTIMA_E_UNSUPPORTED;
  const Span x{X, n_tok, d_in, ldx, 2}, wg{Wg, d_ff, d_in, d_in, 2}, wu{Wu, d_ff, d_in, d_in, 2};
  const Span h{H, n_tok, d_ff, ldh, esize(h_dtype)}, g{G, n_tok, d_ff, ldg, 2};
  const Span u{U, n_tok, d_ff, ldu, 2};
  if (!x.good() || !wg.good() || !wu.good() || !h.good() || (G && !g.good()) || (U && !u.good()))
    return OPTIMA_E_INVAL;
  if (d_in % 8 == 0 && (!optima::aligned16(Wg) || !optima::aligned16(Wu))) return OPTIMA_E_INVAL;
  for (const Span& o : {h, g, u})
    if (o.meets(x) || o.meets(wg) || o.meets(wu)) return OPTIMA_E_INVAL;
  if (h.meets(g) || h.meets(u) || g.meets(u)) return OPTIMA_E_INVAL;
  const size_t need = optima::gated_forward_workspace_bytes(n_tok, d_in, d_ff);
  if (need && (!ws || !optima::aligned16(ws) || ws_bytes < need)) return OPTIMA_E_WORKSPACE;
  if (n_tok == 0) return OPTIMA_OK;
  return optima::gated_forward(X, ldx, n_tok, d_in, Wg, Wu, d_ff, act, H, ldh, h_dtype, G, ldg, U,
                               ldu, ws, stream);
}

size_t optima_gated_backward_workspace_bytes(int64_t n_tok, int64_t d_in, int64_t d_ff) {
  if (!gated_sizes(n_tok, d_in, d_ff)) return 0;
  return optima::gated_backward_workspace_bytes(n_tok, d_in, d_ff);
}

optima_status optima_gated_backward(const void* X, int64_t ldx, int64_t n_tok, int64_t d_in,
                                    const void* Wg, const void* Wu, int64_t d_ff, int act,
                                    const void* G, int64_t ldg, const void* U, int64_t ldu,
                                    const void* dH, int64_t lddh, void* dX, int64_t lddx,
                                    int dx_dtype, void* dWg, void* dWu, int dw_dtype,
                                    const uint8_t* mask_g, const uint8_t* mask_u, int accumulate,
                                    void* ws, size_t ws_bytes, hipStream_t stream) {
  if (!gated_sizes(n_tok, d_in, d_ff) || !Wg || !Wu) return OPTIMA_E_INVAL;
  if (act != OPTIMA_ACT_NONE && act != OPTIMA_ACT_SILU) return OPTIMA_E_INVAL;
  if ((!dX && !dWg) || !dWg != !dWu || ((mask_g || mask_u) && !dWg)) return OPTIMA_E_INVAL;
  if ((dX && !f32_or_bf16(dx_dtype)) || (dWg && !f32_or_bf16(dw_dtype)))
    return OPTIMA_E_UNSUPPORTED;
  const Span x{X, n_tok, d_in, ldx, 2}, wg{Wg, d_ff, d_in, d_in, 2}, wu{Wu, d_ff, d_in, d_in, 2};
  const Span g{G, n_tok, d_ff, ldg, 2}, u{U, n_tok, d_ff, ldu, 2}, dh{dH, n_tok, d_ff, lddh, 2};
  const Span dx{dX, n_tok, d_in, lddx, esize(dx_dtype)};
  const Span dwg{dWg, d_ff, d_in, d_in, esize(dw_dtype)}, dwu{dWu, d_ff, d_in, d_in, esize(dw_dtype)};
  const Span mg{mask_g, d_ff, d_in, d_in, 1}, mu{mask_u, d_ff, d_in, d_in, 1};
  for (const Span& i : {x, wg, wu, g, u, dh})
    if (!i.good()) return OPTIMA_E_INVAL;
  if (d_in % 8 == 0 && (!optima::aligned16(Wg) || !optima::aligned16(Wu))) return OPTIMA_E_INVAL;
  if ((dX && !dx.good()) || (dWg && (!dwg.good() || !dwu.good()))) return OPTIMA_E_INVAL;
  for (const Span& o : {dx, dwg, dwu})
    for (const Span& i : {x, wg, wu, g, u, dh, mg, mu})
      if (o.meets(i)) return OPTIMA_E_INVAL;
  if (dx.meets(dwg) || dx.meets(dwu) || dwg.meets(dwu)) return OPTIMA_E_INVAL;
  const size_t need = optima::gated_backward_workspace_bytes(n_tok, d_in, d_ff);
  if (!ws || !optima::aligned16(ws) || ws_bytes < need) return OPTIMA_E_WORKSPACE;
  return optima::gated_backward(X, ldx, n_tok, d_in, Wg, Wu, d_ff, act, G, ldg, U, ldu, dH, lddh, dX,
                                lddx, dx_dtype, dWg, dWu, dw_dtype, mask_g, mask_u,
                                accumulate ? 1 : 0, ws, stream);
}

size_t optima_w4_row_bytes(int64_t d) {
  return d < 1 || d > kMaxDim ? 0 : size_t((d + 127) / 128) * 64;
}

optima_status optima_w4_pack(const void* W, int dtype, int64_t n, int64_t d, int64_t group,
                             void* Q, void* scales, hipStream_t stream) {
  if (!f32_or_bf16(dtype)) return OPTIMA_E_UNSUPPORTED;
  if (n < 0 || n > kMaxCols || d < 1 || d > kMaxDim || !group_ok(group)) return OPTIMA_E_INVAL;
  const int64_t groups = (d + group - 1) / group, row = int64_t(optima_w4_row_bytes(d));
  // 16 threads a chunk, in blocks of 256: a launch has fewer than 2^32 threads.
  if ((n * (row / 64) + 15) / 16 >= int64_t(1) << 24) return OPTIMA_E_INVAL;
  const Span w{W, n, d, d, esize(dtype)}, q{Q, n, row, row, 1}, sc{scales, n, groups, groups, 2};
  if (!w.good() || !q.good() || !sc.good() || !optima::aligned16(Q)) return OPTIMA_E_INVAL;
  if (q.meets(w) || sc.meets(w) || q.meets(sc)) return OPTIMA_E_INVAL;
  if (n == 0) return OPTIMA_OK;
  return optima::w4_pack(W, dtype, n, d, group, Q, scales, stream);
}

size_t optima_w4_workspace_bytes(int64_t n_tok, int64_t d, int64_t d_out, int n_mats) {
  if (n_tok < 0 || n_tok > (int64_t(1) << 21) || d < 1 || d > kMaxDim || d_out < 1 ||
      d_out > kMaxCols || (n_mats != 1 && n_mats != 2))
    return 0;
  return optima::w4_workspace_bytes(n_tok, d, d_out, n_mats);
}

optima_status optima_w4_linear(const void* X, int64_t ldx, int x_dtype, const float* x_scales,
                               int64_t x_group, int64_t n_tok, int64_t d, const void* Q,
                               const void* scales, int64_t group, int64_t d_out, void* Y,
                               int64_t ldy, int y_dtype, void* ws, size_t ws_bytes,
                               hipStream_t stream) {
  return w4_call(X, ldx, x_dtype, x_scales, x_group, n_tok, d, Q, scales, nullptr, nullptr, group,
                 d_out, OPTIMA_ACT_NONE, Y, ldy, y_dtype, ws, ws_bytes, stream);
}

optima_status optima_w4_gated(const void* X, int64_t ldx, int x_dtype, const float* x_scales,
                              int64_t x_group, int64_t n_tok, int64_t d, const void* Qg,
                              const void* scales_g, const void* Qu, const void* scales_u,
                              int64_t group, int64_t d_ff, int act, void* H, int64_t ldh,
                              int h_dtype, void* ws, size_t ws_bytes, hipStream_t stream) {
  if (!Qu || !scales_u || (act != OPTIMA_ACT_NONE && act != OPTIMA_ACT_SILU)) return OPTIMA_E_INVAL;
  return w4_call(X, ldx, x_dtype, x_scales, x_group, n_tok, d, Qg, scales_g, Qu, scales_u, group,
                 d_ff, act, H, ldh, h_dtype, ws, ws_bytes, stream);
}

size_t optima_mx4_row_bytes(int64_t d) {
  return d < 1 || d > kMaxDim ? 0 : optima::mx4_row_bytes(d);
}
size_t optima_mx4_scale_bytes(int64_t d) {
  return d < 1 || d > kMaxDim ? 0 : optima::mx4_scale_bytes(d);
}

optima_status optima_mx4_pack(const void* X, int64_t ldx, int dtype, int64_t n, int64_t d, void* Q,
                              void* scales, hipStream_t stream) {
  if (!f32_or_bf16(dtype)) return OPTIMA_E_UNSUPPORTED;
  if (!mx4_rows(n, d)) return OPTIMA_E_INVAL;
  const Span x{X, n, d, ldx, esize(dtype)}, q = mx4_codes(Q, n, d), sc = mx4_scales(scales, n, d);
  if (!x.good() || !q.good() || !sc.good() || !optima::aligned16(Q)) return OPTIMA_E_INVAL;
  if (q.meets(x) || sc.meets(x) || q.meets(sc)) return OPTIMA_E_INVAL;
  if (n == 0) return OPTIMA_OK;
  return optima::mx4_pack(X, ldx, dtype, n, d, Q, scales, stream);
}

optima_status optima_mx4_unpack(const void* Q, const void* scales, int64_t n, int64_t d, void* Y,
                                int64_t ldy, int dtype, hipStream_t stream) {
  if (!f32_or_bf16(dtype)) return OPTIMA_E_UNSUPPORTED;
  if (!mx4_rows(n, d)) return OPTIMA_E_INVAL;
  const Span y{Y, n, d, ldy, esize(dtype)}, q = mx4_codes(Q, n, d), sc = mx4_scales(scales, n, d);
  if (!y.good() || !q.good() || !sc.good() || !optima::aligned16(Q)) return OPTIMA_E_INVAL;
  if (y.meets(q) || y.meets(sc)) return OPTIMA_E_INVAL;
  if (n == 0) return OPTIMA_OK;
  return optima::mx4_unpack(Q, scales, n, d, Y, ldy, dtype, stream);
}

size_t optima_mx4_workspace_bytes(int64_t n_tok, int64_t d, int64_t d_out) {
  return mx4_sizes(n_tok, d, d_out) ? optima::mx4_workspace_bytes(n_tok, d, d_out) : 0;
}

optima_status optima_mx4_linear(const void* X, int64_t ldx, int x_dtype, const void* x_scales,
                                int64_t n_tok, int64_t d, const void* Q, const void* scales,
                                int64_t d_out, void* Y, int64_t ldy, int y_dtype, void* ws,
                                size_t ws_bytes, hipStream_t stream) {
  const bool packed = x_dtype == OPTIMA_DTYPE_MX4;
  if ((!packed && x_dtype != OPTIMA_DTYPE_BF16) || !f32_or_bf16(y_dtype))
    return OPTIMA_E_UNSUPPORTED;
  if (!mx4_sizes(n_tok, d, d_out) || (!packed && x_scales)) return OPTIMA_E_INVAL;
  const Span x = packed ? mx4_codes(X, n_tok, d) : Span{X, n_tok, d, ldx, 2};
  const Span xs = mx4_scales(packed ? x_scales : nullptr, n_tok, d);
  const Span q = mx4_codes(Q, d_out, d), sc = mx4_scales(scales, d_out, d);
  const Span y{Y, n_tok, d_out, ldy, esize(y_dtype)};
  if (!x.good() || (packed && (!xs.good() || !optima::aligned16(X))) || !q.good() || !sc.good() ||
      !optima::aligned16(Q) || !y.good())
    return OPTIMA_E_INVAL;
  for (const Span& i : {x, xs, q, sc})
    if (y.meets(i)) return OPTIMA_E_INVAL;
  const size_t need = optima::mx4_workspace_bytes(n_tok, d, d_out);
  if (need && (!ws || !optima::aligned16(ws) || ws_bytes < need)) return OPTIMA_E_WORKSPACE;
  if (n_tok == 0) return OPTIMA_OK;
  return optima::mx4_linear(X, ldx, packed ? x_scales : nullptr, n_tok, d, Q, scales, d_out, Y, ldy,
                            y_dtype, ws, stream);
}

size_t optima_token_logprobs_workspace_bytes(int64_t n, int64_t vocab, int64_t k) {
  if (!logprob_sizes(n, vocab) || k < 0 || k > std::min<int64_t>(vocab, OPTIMA_TOP_MAX)) return 0;
  return optima::token_logprobs_workspace_bytes(n, vocab, k);
}

optima_status optima_token_logprobs(const void* X, int64_t ldx, int dtype, int64_t n, int64_t vocab,
                                    const int64_t* tokens, float scale, float* logp, float* lse,
                                    float* entropy, int64_t k, int64_t* top_index, float* top_logp,
                                    void* ws, size_t ws_bytes, hipStream_t stream) {
  if (!f32_or_bf16(dtype)) return OPTIMA_E_UNSUPPORTED;
  if (!logprob_sizes(n, vocab) || !positive(scale) || k < 0 || k > vocab) return OPTIMA_E_INVAL;
  if (k > OPTIMA_TOP_MAX) return OPTIMA_E_UNSUPPORTED;
  const bool top = top_index || top_logp;
  if (n > 0 && (top != (k > 0) || (!logp && !lse && !entropy && !top) || (logp && !tokens)))
    return OPTIMA_E_INVAL;
  const Span x{X, n, vocab, ldx, esize(dtype)}, t{tokens, 1, n, n, 8};
  const Span out[5] = {{logp, 1, n, n, 4}, {lse, 1, n, n, 4}, {entropy, 1, n, n, 4},
                       {top_index, 1, n * k, n * k, 8}, {top_logp, 1, n * k, n * k, 4}};
  if (!x.good() || !t.aligned()) return OPTIMA_E_INVAL;
  for (const Span& o : out) {
    if (!o.aligned() || o.meets(x) || o.meets(t)) return OPTIMA_E_INVAL;
    for (const Span& p : out)
      if (&p != &o && o.meets(p)) return OPTIMA_E_INVAL;
  }
  const size_t need = optima::token_logprobs_workspace_bytes(n, vocab, k);
  if (need && (!ws || (reinterpret_cast<uintptr_t>(ws) & 7) || ws_bytes < need))
    return OPTIMA_E_WORKSPACE;
  if (n == 0) return OPTIMA_OK;
  return optima::token_logprobs(X, ldx, dtype, n, vocab, tokens, scale, logp, lse, entropy, k,
                                top_index, top_logp, ws, stream);
}

optima_status optima_token_logprobs_backward(const void* X, int64_t ldx, int dtype, int64_t n,
                                             int64_t vocab, const int64_t* tokens, float scale,
                                             const float* lse, const float* entropy,
                                             const float* dlogp, const float* dentropy,
                                             const float* dlse, void* dX, int64_t lddx,
                                             hipStream_t stream) {
  if (!f32_or_bf16(dtype)) return OPTIMA_E_UNSUPPORTED;
  if (!logprob_sizes(n, vocab) || !positive(scale)) return OPTIMA_E_INVAL;
  if (n > 0 && (!lse || (!dlogp && !dentropy && !dlse) || (dlogp && !tokens) ||
                (dentropy && !entropy)))
    return OPTIMA_E_INVAL;
  const Span x{X, n, vocab, ldx, esize(dtype)}, dx{dX, n, vocab, lddx, esize(dtype)};
  if (!x.good() || !dx.good() || (dx.meets(x) && !dx.same(x))) return OPTIMA_E_INVAL;
  const Span t{tokens, 1, n, n, 8};
  if (!t.aligned() || dx.meets(t)) return OPTIMA_E_INVAL;
  for (const float* p : {lse, entropy, dlogp, dentropy, dlse}) {
    const Span i{p, 1, n, n, 4};
    if (!i.aligned() || dx.meets(i)) return OPTIMA_E_INVAL;
  }
  if (n == 0) return OPTIMA_OK;
  return optima::token_logprobs_backward(X, ldx, dtype, n, vocab, tokens, scale, lse, entropy, dlogp,
                                         dentropy, dlse, dX, lddx, stream);
}

}  // extern "C"
