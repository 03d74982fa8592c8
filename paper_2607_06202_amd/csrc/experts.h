// Arguments and launchers of the router, the experts' products and combine's gradient (host side).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

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
  const char* d;  // rows of parts * N bf16
  const char *w, *w2;
  char* dx;
  const int32_t* expert_off;
  int64_t d_ld, dx_ld, expert_stride;
  int E, cap, N, K, parts;
};

struct WeightGradArgs {
  const char* d;  // rows of parts * N bf16
  const char* x;
  char *dw, *dw2;  // [E][N][K] bf16
  const int32_t* expert_off;
  int64_t d_ld, x_ld;
  int E, cap, N, K, parts;
};

// The kernels' choice by the rows that there can be (cap = T*k) over E experts.
//
// few_rows: the split reduction of experts_few.hip against 128 x 256 tiles, us, 128 experts, top-8. 2048 to 2 x 768: 8
// rows 16.0 / 32.3, 16 rows 29.3 / 33.8, 32 rows 43.5 / 36.8, 128 rows 108 / 105; 768 to 2048: 8 rows 14.5 / 15.4, 32 rows
// 27 / 21.
inline bool few_rows(int64_t cap) { return cap <= 16; }
// short_rows (fp8): 64 x 256 tiles against 128 x 256, us, 64 experts, 7168 to 2 x 2048: 8 rows each 351 / 494, 128 rows 728
// / 897, 256 rows 1170 / 1136.
inline bool short_rows(int64_t cap, int E) { return cap / E < 256; }
// many_rows: 256 x 256 tiles against 128 x 256 (the smaller tile first), us, two runs of each, 32 experts. 7168 to 2 x
// 2048: 256 rows each 714-768 / 750-778, 512 rows 1131-1147 / 1143-1159, 1024 rows 1991-1993 / 1935-2008, 2048 rows
// 3784-3786 / 3578-3585; 2048 to 7168: 589 / 598-610 at 512 rows, 1053-1071 / 1039-1047 at 1024, 2004-2008 / 1921-1938
// at 2048.
inline bool many_rows(int64_t cap, int E) { return cap / E >= 1024; }
hipError_t launch_forward_few(const ForwardArgs& p, bool fp8, bool gated, hipStream_t stream);
hipError_t launch_forward(const ForwardArgs& p, bool fp8, bool gated, hipStream_t stream);
hipError_t launch_row_grad(const RowGradArgs& p, hipStream_t stream);
hipError_t launch_weight_grad(const WeightGradArgs& p, hipStream_t stream);
hipError_t launch_gated_pre_grad(const void* dh, const void* pre, void* dpre, const int32_t* expert_off, int E,
                                 int cap, int I, int act, hipStream_t stream);
// dpre (with an activation) and, unless dbias is null, dbias. dy rows dy_ld bytes apart.
hipError_t launch_pre_grad(const void* dy, int64_t dy_ld, const void* pre, void* dpre, void* dbias,
                           const int32_t* expert_off, int E, int cap, int N, int act, hipStream_t stream);

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
