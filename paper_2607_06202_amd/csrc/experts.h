// Arguments and launchers of the router, the experts' products and combine's gradient (host side).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace epl {

// Row strides (…_ld) are in bytes, expert_stride in elements. cap: packed rows, the bound on expert_off.
struct ForwardArgs {
  const char* a;
  const float* a_scale;  // fp8: [rows][K / 128]
  const char *w, *w2;    // [E] matrices [N][K]; w2: the up projection (gated)
  const float *w_scale, *w2_scale;  // fp8: [E][N]
  const char* bias;      // [E][N] bf16 or null
  const char* residual;  // rows of N bf16 or null
  char* out;
  char* pre;  // null, or [rows][N] ([rows][2N] gated) bf16
  const int32_t* expert_off;
  int64_t a_ld, out_ld, res_ld, expert_stride;
  int E, cap, N, K, act;
};

struct RowGradArgs {
  const char* d;  // [rows][parts * N] bf16
  const char *w, *w2;
  char* dx;
  const int32_t* expert_off;
  int64_t dx_ld, expert_stride;
  int E, cap, N, K, parts;
};

struct WeightGradArgs {
  const char* d;  // [rows][parts * N] bf16
  const char* x;
  char *dw, *dw2;  // [E][N][K] bf16
  const int32_t* expert_off;
  int64_t x_ld;
  int E, cap, N, K, parts;
};

hipError_t launch_forward(const ForwardArgs& p, bool fp8, bool gated, hipStream_t stream);
hipError_t launch_row_grad(const RowGradArgs& p, hipStream_t stream);
hipError_t launch_weight_grad(const WeightGradArgs& p, hipStream_t stream);
hipError_t launch_gated_pre_grad(const void* dh, const void* pre, void* dpre, const int32_t* expert_off, int E,
                                 int cap, int I, int act, hipStream_t stream);
hipError_t launch_pre_grad(const void* dy, const void* pre, void* dpre, const int32_t* expert_off, int E, int cap,
                           int N, int act, hipStream_t stream);
hipError_t launch_bias_grad(const void* dy, const void* pre, void* dbias, const int32_t* expert_off, int E, int cap,
                            int N, int act, hipStream_t stream);

struct RouteArgs {
  const void* logits;  // [T][E] fp32 or bf16
  const float* bias;   // [E] or null
  const float* dw;     // backward: [T][k]
  int32_t* idx;        // [T][k] (read by the backward pass)
  float* w;            // forward: [T][k]
  void* dlogits;       // backward: [T][E], type of logits
  int64_t T;
  int E, k;
  bool bf16, sigmoid, normalize;
  float scale;
};
hipError_t launch_route(const RouteArgs& p, hipStream_t stream);
hipError_t launch_route_backward(const RouteArgs& p, hipStream_t stream);

hipError_t launch_combine_grad(const void* dout, const void* y, const float* w, const int32_t* pair_row, void* dy,
                               float* dw, int64_t T, int k, int H, int pitch, int64_t cap, hipStream_t stream);

}  // namespace epl
