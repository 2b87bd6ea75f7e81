// layers.h -- the layers around a circuit: argument records and launchers of the
// kernels in layer_norm.hip, linear.hip and log_probs.hip (host interface), and
// what the entry points in layers_api.cpp need to size their workspaces.
#pragma once

#include <cstddef>
#include <cstdint>

namespace vqc {

inline size_t element_bytes(int dtype) { return dtype == 0 ? 4 : 2; }

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

}  // namespace vqc
