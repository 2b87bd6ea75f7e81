// layers.h -- the layers around a circuit: argument records and launchers of the
// kernels in layer_norm.hip, linear.hip, linear_quantized.hip, log_probs.hip and
// verify.hip (host interface), and what the entry points in layers_api.cpp need to
// size their workspaces.
#pragma once

#include <cstddef>
#include <cstdint>

namespace vqc {

inline size_t element_bytes(int dtype) { return dtype == 0 ? 4 : 2; }
// Parts of a workspace start on 256 bytes.
inline size_t round256(size_t v) { return (v + 255) / 256 * 256; }

struct NormArgs {
  int64_t rows, cols;
  const void *x, *weight, *bias, *dy;
  void *y, *dx, *dweight, *dbias;
  int64_t ldx, ldy, lddy, lddx;
  float eps;
  float *mean, *rstd;              // written by the forward
  const float *mean_in, *rstd_in;  // read by the backward
  float* partial;                  // workspace: [parts][2][cols]
};
// Workgroups of the backward that keep partial sums, for any element type.
int64_t norm_parts(int64_t rows, int64_t cols);
// Launchers return 0 or a hipError_t value.
int launch_layer_norm(int dtype, const NormArgs& a, void* stream);
int launch_layer_norm_backward(int dtype, const NormArgs& a, void* stream);

struct LinearArgs {
  int64_t rows, n_in, n_out;
  const void *x, *weight, *bias, *residual, *dy;
  int64_t ldx, ldw, ldr, ldy, lddy, lddx, lddw;
  int act;
  void *y, *dx, *dweight, *dbias;
  float* pre;            // forward
  const float* pre_in;   // backward
  unsigned char* ws;
};
size_t linear_workspace(int dtype, int64_t rows, int64_t n_in, int64_t n_out, bool training);
int launch_linear(int dtype, const LinearArgs& a, void* stream);
int launch_linear_backward(int dtype, const LinearArgs& a, void* stream);

struct QuantizeArgs {
  int64_t rows, cols, ldx, ldq;
  int64_t width;  // q is 0 from cols to here
  const void* x;
  int8_t* q;
  float* scales;
};
int launch_quantize(int dtype, const QuantizeArgs& a, void* stream);

struct QuantizedArgs {
  int64_t rows, n_in, n_out;
  const void* x;            // integers where x_scales is given, else of the element type
  const float* x_scales;
  const int8_t* weight;
  const float* w_scales;
  const void *bias, *residual;
  int64_t ldx, ldw, ldr, ldy;
  int act;
  void* y;
  unsigned char* ws;
};
size_t linear_quantized_workspace(int64_t rows, int64_t n_in, int64_t n_out, bool integers);
int launch_linear_quantized(int dtype, const QuantizedArgs& a, void* stream);

struct ScoreArgs {
  int64_t rows, cols, lds, ldds;
  const void* scores;
  float inv_t;
  const int64_t* targets;
  int64_t n_targets;
  float *logp, *entropy;
  int n_top;
  float* top_logp;
  int64_t* top_index;
  float* stats;
  // backward
  const float *stats_in, *entropy_in, *dlogp, *dentropy;
  void* dscores;
  unsigned char* ws;
};
size_t log_probs_workspace(int64_t rows, int64_t cols, int n_top);
int launch_log_probs(int kind, int dtype, const ScoreArgs& a, void* stream);
int launch_log_probs_backward(int dtype, const ScoreArgs& a, void* stream);

struct VerifyArgs {
  int64_t sequences, drafts, cols, ldt, ldd;
  const void *target, *draft;  // draft: null where the drafts are certain
  double scale;                // 1 / T
  const int64_t* drafted;
  const double* uniforms;
  int64_t *outcomes, *accepted;
  unsigned char* ws;
};
size_t verify_workspace(int dtype, int64_t sequences, int64_t drafts, int64_t cols,
                        bool has_draft);
int launch_verify(int kind, int dtype, const VerifyArgs& a, void* stream);

}  // namespace vqc
