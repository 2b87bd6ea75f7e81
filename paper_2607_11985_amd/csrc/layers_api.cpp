// layers_api.cpp -- the layers' entry points of include/vqc.h: argument checks and launches.
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <string>

#include "layers.h"
#include "vqc.h"
#include "vqc_internal.h"

namespace {

using vqc::element_bytes;

constexpr int64_t kMost = (int64_t)1 << 40;  // rows, columns and their products

int invalid(const std::string& msg) { return vqc::set_error(VQC_ERR_INVALID_ARG, msg); }

int hip_status(const char* what, int rc) {
  if (!rc) return VQC_OK;
  // a launch that failed leaves its error with the runtime: clear it, the status carries it
  (void)hipGetLastError();
  if (rc == (int)hipErrorInvalidConfiguration)
    return vqc::set_error(VQC_ERR_TOO_LARGE, std::string(what) + ": grid too large");
  return vqc::set_error(VQC_ERR_HIP, std::string(what) + " launch failed: " +
                                         hipGetErrorString((hipError_t)rc));
}

bool known_dtype(int32_t t) { return t == VQC_F32 || t == VQC_F16 || t == VQC_BF16; }

int check_size(const char* name, int64_t v, int64_t least) {
  if (v < least) return invalid(std::string(name) + " must be at least " + std::to_string(least));
  if (v > kMost) return vqc::set_error(VQC_ERR_TOO_LARGE, std::string(name) + " beyond 2^40");
  return VQC_OK;
}

int check_area(int64_t a, int64_t b) {
  if (a > 0 && b > kMost / a)
    return vqc::set_error(VQC_ERR_TOO_LARGE, "rows times columns beyond 2^40");
  return VQC_OK;
}

// A vector of `bytes`-byte elements; null where it may be.
int check_pointer(const char* name, const void* p, size_t bytes, bool optional) {
  if (!p) return optional ? VQC_OK : invalid(std::string(name) + " is NULL");
  if (reinterpret_cast<uintptr_t>(p) % bytes)
    return invalid(std::string(name) + " is not aligned to its elements");
  return VQC_OK;
}

// Rows of `cols` elements; strides of read arrays may be 0 or overlap.
int check_rows(const char* name, const void* p, int64_t ld, int64_t rows, int64_t cols,
               size_t bytes, bool written, bool optional) {
  if (rows == 0 || cols == 0) return VQC_OK;
  if (int rc = check_pointer(name, p, bytes, optional)) return rc;
  if (!p) return VQC_OK;
  if (ld < 0) return invalid(std::string("the row stride of ") + name + " is negative");
  if (written && rows > 1 && ld < cols)
    return invalid(std::string("the row stride of ") + name + " is below its width");
  if (rows > 1 && ld > (INT64_MAX / 16 - cols) / (rows - 1))
    return vqc::set_error(VQC_ERR_TOO_LARGE,
                          std::string("the rows of ") + name + " exceed 64-bit offsets");
  return VQC_OK;
}

int check_ws(const void* ws, size_t bytes, size_t need, const char* what) {
  if (need == 0) return VQC_OK;
  if (!ws || bytes < need)
    return vqc::set_error(VQC_ERR_WORKSPACE, std::string("workspace smaller than ") + what);
  if (reinterpret_cast<uintptr_t>(ws) % 256)
    return vqc::set_error(VQC_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  return VQC_OK;
}

// Nothing may be thrown through the C boundary (a message's allocation can).
template <typename F>
int guarded(F&& f) noexcept {
  try {
    return f();
  } catch (...) {
    return VQC_ERR_OOM;
  }
}

size_t norm_workspace(int64_t rows, int64_t cols) {
  return (size_t)vqc::norm_parts(rows, cols) * 2 * (size_t)cols * 4;
}

bool linear_sizes_ok(int64_t rows, int64_t n_in, int64_t n_out) {
  return rows >= 0 && n_in >= 0 && n_out >= 0 && rows <= kMost && n_in <= kMost &&
         n_out <= kMost && (rows == 0 || (n_in <= kMost / rows && n_out <= kMost / rows)) &&
         (n_in == 0 || n_out <= kMost / n_in);
}

int check_linear_sizes(int64_t rows, int64_t n_in, int64_t n_out) {
  int rc;
  if ((rc = check_size("rows", rows, 0)) || (rc = check_size("n_in", n_in, 0)) ||
      (rc = check_size("n_out", n_out, 0)) || (rc = check_area(rows, n_in)) ||
      (rc = check_area(rows, n_out)) || (rc = check_area(n_out, n_in)))
    return rc;
  return VQC_OK;
}

// A sequence's rows: drafts + 1 of the target and as many drafts'.
bool verify_sizes_ok(int64_t sequences, int64_t drafts, int64_t cols) {
  if (sequences < 0 || drafts < 0 || cols < 1 || sequences > kMost || drafts > kMost ||
      cols > kMost)
    return false;
  const int64_t rows = 2 * drafts + 1;
  return sequences == 0 || (rows <= kMost / sequences && cols <= kMost / (rows * sequences));
}

}  // namespace

extern "C" {

int vqc_layer_norm(int32_t dtype, int64_t rows, int64_t cols, const void* x, int64_t ldx,
                   const void* weight, const void* bias, float eps, void* y, int64_t ldy,
                   float* mean, float* rstd, void* stream) {
  return guarded([&]() -> int {
    if (!known_dtype(dtype)) return invalid("unknown element type");
    int rc;
    if ((rc = check_size("rows", rows, 0)) || (rc = check_size("cols", cols, 1)) ||
        (rc = check_area(rows, cols)))
      return rc;
    if (!(eps >= 0.f) || !std::isfinite(eps)) return invalid("eps must be finite and >= 0");
    if (rows == 0) return VQC_OK;
    const size_t b = element_bytes(dtype);
    if ((rc = check_rows("x", x, ldx, rows, cols, b, false, false)) ||
        (rc = check_rows("y", y, ldy, rows, cols, b, true, false)) ||
        (rc = check_pointer("weight", weight, b, true)) ||
        (rc = check_pointer("bias", bias, b, true)) ||
        (rc = check_pointer("mean", mean, 4, true)) || (rc = check_pointer("rstd", rstd, 4, true)))
      return rc;
    if (!mean != !rstd) return invalid("mean and rstd must both be given or both be NULL");
    vqc::NormArgs a{};
    a.rows = rows;
    a.cols = cols;
    a.x = x;
    a.ldx = ldx;
    a.weight = weight;
    a.bias = bias;
    a.eps = eps;
    a.y = y;
    a.ldy = ldy;
    a.mean = mean;
    a.rstd = rstd;
    return hip_status("layer norm", vqc::launch_layer_norm(dtype, a, stream));
  });
}

size_t vqc_layer_norm_workspace_bytes(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 1 || rows > kMost || cols > kMost || (rows && cols > kMost / rows))
    return (size_t)-1;
  return norm_workspace(rows, cols);
}

int vqc_layer_norm_backward(int32_t dtype, int64_t rows, int64_t cols, const void* x, int64_t ldx,
                            const void* weight, const float* mean, const float* rstd,
                            const void* dy, int64_t lddy, void* dx, int64_t lddx, void* dweight,
                            void* dbias, void* workspace, size_t workspace_bytes, void* stream) {
  return guarded([&]() -> int {
    if (!known_dtype(dtype)) return invalid("unknown element type");
    int rc;
    if ((rc = check_size("rows", rows, 0)) || (rc = check_size("cols", cols, 1)) ||
        (rc = check_area(rows, cols)))
      return rc;
    const size_t b = element_bytes(dtype);
    if ((rc = check_rows("x", x, ldx, rows, cols, b, false, false)) ||
        (rc = check_rows("dy", dy, lddy, rows, cols, b, false, false)) ||
        (rc = check_rows("dx", dx, lddx, rows, cols, b, true, true)) ||
        (rc = check_pointer("weight", weight, b, true)) ||
        (rc = check_pointer("mean", mean, 4, rows == 0)) ||
        (rc = check_pointer("rstd", rstd, 4, rows == 0)) ||
        (rc = check_pointer("dweight", dweight, b, true)) ||
        (rc = check_pointer("dbias", dbias, b, true)))
      return rc;
    if (!dx && !dweight && !dbias) return VQC_OK;
    if (rows == 0 && !dweight && !dbias) return VQC_OK;
    // the partial sums alone need it
    if ((dweight || dbias) &&
        (rc = check_ws(workspace, workspace_bytes, norm_workspace(rows, cols),
                       "vqc_layer_norm_workspace_bytes(rows, cols)")))
      return rc;
    vqc::NormArgs a{};
    a.rows = rows;
    a.cols = cols;
    a.x = x;
    a.ldx = ldx;
    a.weight = weight;
    a.mean_in = mean;
    a.rstd_in = rstd;
    a.dy = dy;
    a.lddy = lddy;
    a.dx = dx;
    a.lddx = lddx;
    a.dweight = dweight;
    a.dbias = dbias;
    a.partial = static_cast<float*>(workspace);
    return hip_status("layer norm backward", vqc::launch_layer_norm_backward(dtype, a, stream));
  });
}

size_t vqc_linear_workspace_bytes(int32_t dtype, int64_t rows, int64_t n_in, int64_t n_out,
                                  int32_t training) {
  if (!known_dtype(dtype) || training < 0 || training > 1 || !linear_sizes_ok(rows, n_in, n_out))
    return (size_t)-1;
  return vqc::linear_workspace(dtype, rows, n_in, n_out, training != 0);
}

int vqc_linear(int32_t dtype, int64_t rows, int64_t n_in, int64_t n_out, const void* x,
               int64_t ldx, const void* weight, int64_t ldw, const void* bias, int32_t act,
               const void* residual, int64_t ldr, void* y, int64_t ldy, float* pre,
               void* workspace, size_t workspace_bytes, void* stream) {
  return guarded([&]() -> int {
    if (!known_dtype(dtype)) return invalid("unknown element type");
    if (act < VQC_ACT_NONE || act > VQC_ACT_TANH) return invalid("unknown activation");
    int rc;
    if ((rc = check_linear_sizes(rows, n_in, n_out))) return rc;
    if (rows == 0 || n_out == 0) return VQC_OK;
    const size_t b = element_bytes(dtype);
    if ((rc = check_rows("x", x, ldx, rows, n_in, b, false, false)) ||
        (rc = check_rows("weight", weight, ldw, n_out, n_in, b, false, false)) ||
        (rc = check_rows("residual", residual, ldr, rows, n_out, b, false, true)) ||
        (rc = check_rows("y", y, ldy, rows, n_out, b, true, false)) ||
        (rc = check_pointer("bias", bias, b, true)) || (rc = check_pointer("pre", pre, 4, true)))
      return rc;
    if ((rc = check_ws(workspace, workspace_bytes,
                       vqc::linear_workspace(dtype, rows, n_in, n_out, false),
                       "vqc_linear_workspace_bytes(dtype, rows, n_in, n_out, 0)")))
      return rc;
    vqc::LinearArgs a{};
    a.rows = rows;
    a.n_in = n_in;
    a.n_out = n_out;
    a.x = x;
    a.ldx = ldx;
    a.weight = weight;
    a.ldw = ldw;
    a.bias = bias;
    a.act = act;
    a.residual = residual;
    a.ldr = ldr;
    a.y = y;
    a.ldy = ldy;
    a.pre = pre;
    a.ws = static_cast<unsigned char*>(workspace);
    return hip_status("linear", vqc::launch_linear(dtype, a, stream));
  });
}

int vqc_linear_backward(int32_t dtype, int64_t rows, int64_t n_in, int64_t n_out, const void* x,
                        int64_t ldx, const void* weight, int64_t ldw, int32_t act,
                        const float* pre, const void* dy, int64_t lddy, void* dx, int64_t lddx,
                        void* dweight, int64_t lddw, void* dbias, void* workspace,
                        size_t workspace_bytes, void* stream) {
  return guarded([&]() -> int {
    if (!known_dtype(dtype)) return invalid("unknown element type");
    if (act < VQC_ACT_NONE || act > VQC_ACT_TANH) return invalid("unknown activation");
    int rc;
    if ((rc = check_linear_sizes(rows, n_in, n_out))) return rc;
    if (!dx && !dweight && !dbias) return VQC_OK;
    const size_t b = element_bytes(dtype);
    if ((rc = check_rows("x", x, ldx, rows, n_in, b, false, !dweight)) ||
        (rc = check_rows("weight", weight, ldw, n_out, n_in, b, false, !dx)) ||
        (rc = check_rows("dy", dy, lddy, rows, n_out, b, false, false)) ||
        (rc = check_rows("dx", dx, lddx, rows, n_in, b, true, true)) ||
        (rc = check_rows("dweight", dweight, lddw, n_out, n_in, b, true, true)) ||
        (rc = check_pointer("dbias", dbias, b, true)) ||
        (rc = check_pointer("pre", pre, 4, act == VQC_ACT_NONE || rows == 0 || n_out == 0)))
      return rc;
    if ((rc = check_ws(workspace, workspace_bytes,
                       vqc::linear_workspace(dtype, rows, n_in, n_out, true),
                       "vqc_linear_workspace_bytes(dtype, rows, n_in, n_out, 1)")))
      return rc;
    vqc::LinearArgs a{};
    a.rows = rows;
    a.n_in = n_in;
    a.n_out = n_out;
    a.x = x;
    a.ldx = ldx;
    a.weight = weight;
    a.ldw = ldw;
    a.act = act;
    a.pre_in = pre;
    a.dy = dy;
    a.lddy = lddy;
    a.dx = dx;
    a.lddx = lddx;
    a.dweight = dweight;
    a.lddw = lddw;
    a.dbias = dbias;
    a.ws = static_cast<unsigned char*>(workspace);
    return hip_status("linear backward", vqc::launch_linear_backward(dtype, a, stream));
  });
}

int vqc_quantize(int32_t dtype, int64_t rows, int64_t cols, const void* x, int64_t ldx, int8_t* q,
                 int64_t ldq, float* scales, void* stream) {
  return guarded([&]() -> int {
    if (!known_dtype(dtype)) return invalid("unknown element type");
    int rc;
    if ((rc = check_size("rows", rows, 0)) || (rc = check_size("cols", cols, 0)) ||
        (rc = check_area(rows, cols)))
      return rc;
    if (rows == 0) return VQC_OK;
    if ((rc = check_rows("x", x, ldx, rows, cols, element_bytes(dtype), false, false)) ||
        (rc = check_rows("q", q, ldq, rows, cols, 1, true, false)) ||
        (rc = check_pointer("scales", scales, 4, false)))
      return rc;
    vqc::QuantizeArgs a{};
    a.rows = rows;
    a.cols = cols;
    a.x = x;
    a.ldx = ldx;
    a.q = q;
    a.ldq = ldq;
    a.scales = scales;
    a.width = cols;
    return hip_status("quantize", vqc::launch_quantize(dtype, a, stream));
  });
}

size_t vqc_linear_quantized_workspace_bytes(int64_t rows, int64_t n_in, int64_t n_out,
                                            int32_t integers) {
  if (integers < 0 || integers > 1 || !linear_sizes_ok(rows, n_in, n_out)) return (size_t)-1;
  return vqc::linear_quantized_workspace(rows, n_in, n_out, integers != 0);
}

int vqc_linear_quantized(int32_t dtype, int64_t rows, int64_t n_in, int64_t n_out, const void* x,
                         int64_t ldx, const float* x_scales, const int8_t* weight, int64_t ldw,
                         const float* weight_scales, const void* bias, int32_t act,
                         const void* residual, int64_t ldr, void* y, int64_t ldy, void* workspace,
                         size_t workspace_bytes, void* stream) {
  return guarded([&]() -> int {
    if (!known_dtype(dtype)) return invalid("unknown element type");
    if (act < VQC_ACT_NONE || act > VQC_ACT_TANH) return invalid("unknown activation");
    int rc;
    if ((rc = check_linear_sizes(rows, n_in, n_out))) return rc;
    if (rows == 0 || n_out == 0) return VQC_OK;
    const size_t b = element_bytes(dtype);
    if ((rc = check_rows("x", x, ldx, rows, n_in, x_scales ? 1 : b, false, false)) ||
        (rc = check_pointer("x_scales", x_scales, 4, true)) ||
        (rc = check_rows("weight", weight, ldw, n_out, n_in, 1, false, false)) ||
        (rc = check_pointer("weight_scales", weight_scales, 4, false)) ||
        (rc = check_rows("residual", residual, ldr, rows, n_out, b, false, true)) ||
        (rc = check_rows("y", y, ldy, rows, n_out, b, true, false)) ||
        (rc = check_pointer("bias", bias, b, true)))
      return rc;
    if ((rc = check_ws(workspace, workspace_bytes,
                       vqc::linear_quantized_workspace(rows, n_in, n_out, x_scales != nullptr),
                       "vqc_linear_quantized_workspace_bytes(rows, n_in, n_out, integers)")))
      return rc;
    vqc::QuantizedArgs a{};
    a.rows = rows;
    a.n_in = n_in;
    a.n_out = n_out;
    a.x = x;
    a.ldx = ldx;
    a.x_scales = x_scales;
    a.weight = weight;
    a.ldw = ldw;
    a.w_scales = weight_scales;
    a.bias = bias;
    a.act = act;
    a.residual = residual;
    a.ldr = ldr;
    a.y = y;
    a.ldy = ldy;
    a.ws = static_cast<unsigned char*>(workspace);
    return hip_status("quantized linear", vqc::launch_linear_quantized(dtype, a, stream));
  });
}

size_t vqc_log_probs_workspace_bytes(int64_t rows, int64_t cols, int32_t n_top) {
  if (rows < 0 || cols < 1 || rows > kMost || cols > kMost || (rows && cols > kMost / rows) ||
      n_top < 0 || n_top > VQC_MAX_TOP || n_top > cols)
    return (size_t)-1;
  return vqc::log_probs_workspace(rows, cols, n_top);
}

int vqc_log_probs(int32_t kind, int32_t dtype, int64_t rows, int64_t cols, const void* scores,
                  int64_t lds, float inv_temperature, const int64_t* targets, int64_t n_targets,
                  float* logp, float* entropy, int32_t n_top, float* top_logp,
                  int64_t* top_index, float* stats, void* workspace, size_t workspace_bytes,
                  void* stream) {
  return guarded([&]() -> int {
    if (kind != VQC_SCORES_LOGITS && kind != VQC_SCORES_WEIGHTS)
      return invalid("unknown kind of scores");
    if (!known_dtype(dtype)) return invalid("unknown element type");
    int rc;
    if ((rc = check_size("rows", rows, 0)) || (rc = check_size("cols", cols, 1)) ||
        (rc = check_area(rows, cols)) || (rc = check_size("n_targets", n_targets, 0)) ||
        (rc = check_area(rows, n_targets)))
      return rc;
    if (!(inv_temperature > 0.f) || !std::isfinite(inv_temperature))
      return invalid("inv_temperature must be finite and > 0");
    if (kind == VQC_SCORES_WEIGHTS && inv_temperature != 1.f)
      return invalid("weights have no temperature: inv_temperature must be 1");
    if (n_top < 0 || n_top > VQC_MAX_TOP || n_top > cols)
      return invalid("n_top must be in [0, min(cols, " + std::to_string(VQC_MAX_TOP) + ")]");
    if (n_top > 0 && cols > INT32_MAX)
      return vqc::set_error(VQC_ERR_TOO_LARGE, "the most probable of over 2^31 outcomes");
    if (rows == 0) return VQC_OK;
    if ((rc = check_rows("scores", scores, lds, rows, cols, element_bytes(dtype), false, false)) ||
        (rc = check_pointer("targets", targets, 8, n_targets == 0)) ||
        (rc = check_pointer("logp", logp, 4, n_targets == 0)) ||
        (rc = check_pointer("entropy", entropy, 4, true)) ||
        (rc = check_pointer("top_logp", top_logp, 4, n_top == 0)) ||
        (rc = check_pointer("top_index", top_index, 8, n_top == 0)) ||
        (rc = check_pointer("stats", stats, 4, true)))
      return rc;
    if ((rc = check_ws(workspace, workspace_bytes, vqc::log_probs_workspace(rows, cols, n_top),
                       "vqc_log_probs_workspace_bytes(rows, cols, n_top)")))
      return rc;
    vqc::ScoreArgs a{};
    a.rows = rows;
    a.cols = cols;
    a.scores = scores;
    a.lds = lds;
    a.inv_t = inv_temperature;
    a.targets = targets;
    a.n_targets = n_targets;
    a.logp = logp;
    a.entropy = entropy;
    a.n_top = n_top;
    a.top_logp = top_logp;
    a.top_index = top_index;
    a.stats = stats;
    a.ws = static_cast<unsigned char*>(workspace);
    return hip_status("log probabilities", vqc::launch_log_probs(kind, dtype, a, stream));
  });
}

int vqc_log_probs_backward(int32_t dtype, int64_t rows, int64_t cols, const void* scores,
                           int64_t lds, float inv_temperature, const int64_t* targets,
                           int64_t n_targets, const float* stats, const float* entropy,
                           const float* dlogp, const float* dentropy, void* dscores,
                           int64_t ldds, void* stream) {
  return guarded([&]() -> int {
    if (!known_dtype(dtype)) return invalid("unknown element type");
    int rc;
    if ((rc = check_size("rows", rows, 0)) || (rc = check_size("cols", cols, 1)) ||
        (rc = check_area(rows, cols)) || (rc = check_size("n_targets", n_targets, 0)) ||
        (rc = check_area(rows, n_targets)))
      return rc;
    if (!(inv_temperature > 0.f) || !std::isfinite(inv_temperature))
      return invalid("inv_temperature must be finite and > 0");
    if (rows == 0) return VQC_OK;
    const size_t b = element_bytes(dtype);
    const bool picks = dlogp && n_targets > 0;
    if ((rc = check_rows("scores", scores, lds, rows, cols, b, false, false)) ||
        (rc = check_rows("dscores", dscores, ldds, rows, cols, b, true, false)) ||
        (rc = check_pointer("targets", targets, 8, !picks)) ||
        (rc = check_pointer("stats", stats, 4, false)) ||
        (rc = check_pointer("entropy", entropy, 4, !dentropy)) ||
        (rc = check_pointer("dlogp", dlogp, 4, true)) ||
        (rc = check_pointer("dentropy", dentropy, 4, true)))
      return rc;
    vqc::ScoreArgs a{};
    a.rows = rows;
    a.cols = cols;
    a.scores = scores;
    a.lds = lds;
    a.inv_t = inv_temperature;
    a.targets = targets;
    a.n_targets = n_targets;
    a.stats_in = stats;
    a.entropy_in = entropy;
    a.dlogp = picks ? dlogp : nullptr;
    a.dentropy = dentropy;
    a.dscores = dscores;
    a.ldds = ldds;
    return hip_status("log probabilities backward",
                      vqc::launch_log_probs_backward(dtype, a, stream));
  });
}

size_t vqc_verify_drafts_workspace_bytes(int32_t dtype, int64_t sequences, int64_t drafts,
                                         int64_t cols, int32_t has_draft) {
  if (!known_dtype(dtype) || has_draft < 0 || has_draft > 1 ||
      !verify_sizes_ok(sequences, drafts, cols))
    return (size_t)-1;
  return sequences ? vqc::verify_workspace(dtype, sequences, drafts, cols, has_draft != 0) : 0;
}

int vqc_verify_drafts(int32_t kind, int32_t dtype, int64_t sequences, int64_t drafts, int64_t cols,
                      const void* target, int64_t ldt, const void* draft, int64_t ldd,
                      double inv_temperature, const int64_t* drafted, const double* uniforms,
                      int64_t* outcomes, int64_t* accepted, void* workspace,
                      size_t workspace_bytes, void* stream) {
  return guarded([&]() -> int {
    if (kind != VQC_SCORES_LOGITS && kind != VQC_SCORES_WEIGHTS)
      return invalid("unknown kind of scores");
    if (!known_dtype(dtype)) return invalid("unknown element type");
    int rc;
    if ((rc = check_size("sequences", sequences, 0)) || (rc = check_size("drafts", drafts, 0)) ||
        (rc = check_size("cols", cols, 1)))
      return rc;
    if (!verify_sizes_ok(sequences, drafts, cols))
      return vqc::set_error(VQC_ERR_TOO_LARGE, "rows times columns beyond 2^40");
    if (!(inv_temperature > 0.) || !std::isfinite(inv_temperature))
      return invalid("inv_temperature must be finite and > 0");
    if (kind == VQC_SCORES_WEIGHTS && inv_temperature != 1.)
      return invalid("weights have no temperature: inv_temperature must be 1");
    if (sequences == 0) return VQC_OK;
    const size_t b = element_bytes(dtype);
    if ((rc = check_rows("target", target, ldt, sequences * (drafts + 1), cols, b, false,
                         false)) ||
        (rc = check_rows("draft", draft, ldd, sequences * drafts, cols, b, false, true)) ||
        (rc = check_pointer("drafted", drafted, 8, drafts == 0)) ||
        (rc = check_pointer("uniforms", uniforms, 8, false)) ||
        (rc = check_pointer("outcomes", outcomes, 8, false)) ||
        (rc = check_pointer("accepted", accepted, 8, false)))
      return rc;
    if (drafts == 0) draft = nullptr;
    if ((rc = check_ws(workspace, workspace_bytes,
                       vqc::verify_workspace(dtype, sequences, drafts, cols, draft != nullptr),
                       "vqc_verify_drafts_workspace_bytes(dtype, sequences, drafts, cols, "
                       "has_draft)")))
      return rc;
    vqc::VerifyArgs a{};
    a.sequences = sequences;
    a.drafts = drafts;
    a.cols = cols;
    a.target = target;
    a.ldt = ldt;
    a.draft = draft;
    a.ldd = ldd;
    a.scale = inv_temperature;
    a.drafted = drafted;
    a.uniforms = uniforms;
    a.outcomes = outcomes;
    a.accepted = accepted;
    a.ws = static_cast<unsigned char*>(workspace);
    return hip_status("verification of drafts", vqc::launch_verify(kind, dtype, a, stream));
  });
}

}  // extern "C"
