// Arguments and launchers of the router, the experts' products, combine's gradient, dispatch with weights and the rows in
// int8 (host side).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

namespace epl {

// Elements of the products' operands. Int8 ones go through everything as bf16 ones twice as long do: 64 bytes of a row are
// one matrix instruction either way, and only the instruction and the type of its sums (32-bit integers, exact) differ.
enum class Elem { kBf16, kE4m3, kInt8 };
constexpr int elem_bytes(Elem t) { return t == Elem::kBf16 ? 2 : 1; }

// Row strides (…_ld) are in bytes, expert_stride in elements. cap: packed rows, the bound on expert_off.
struct ForwardArgs {
  const char* a;
  const float* a_scale;  // fp8: [rows][K / 128]; int8: [rows]
  const char *w, *w2;    // [E] matrices [N][K]; w2: the up projection (gated)
  const float *w_scale, *w2_scale;  // fp8, int8: [E][N]
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
// Int8. few_rows against 64 x 256 tiles: 2048 to 2 x 768 of 128 experts, 8 rows 9.3 / 16.8, 16 rows 16.0 / 18.6; 1408 to 5120
// of 160 experts, 8 rows 18.4 / 16.8, 16 rows 27.4 / 34.5 (kernel times).
// int8_few_each and int8_many_each were measured with two tiles a compute unit or more; with fewer, a shape that makes more of
// them may be faster, which the rules do not look at.
// int8_few_each: 64 x 256 tiles against 128 x 256, us. 1408 to 5120, 160 experts: 6 rows each 228 / 245, 26 rows 216 / 235,
// 51 rows 221 / 238, 64 rows 258 / 246; 7168 to 2 x 2048, 256 experts: 16 rows 1232 / 1241, 48 rows 1285 / 1280, 64 rows
// 1409 / 1287. (32 x 256, before the loads were spread: as 64 x 256 up to 25 rows, slower beyond.)
inline bool int8_few_each(int64_t cap, int E) { return cap / E < 56; }
// int8_many_each: 256 x 256 tiles against 128 x 256, us. 7168 to 2 x 2048, 32 experts: 96 rows each 227 / 175, 128 rows 219 /
// 216, 160 rows 221 / 254, 256 rows 315 / 321, 512 rows 487 / 542, 1024 rows 884 / 991, 2048 rows 1608 / 1881; 2048 to 7168
// with a residual, 64 experts: 128 rows 265 / 260, 160 rows 265 / 309, 256 rows 345 / 363, 512 rows 592 / 656, 1024 rows 1104
// / 1237.
inline bool int8_many_each(int64_t cap, int E) { return cap / E >= 144; }
hipError_t launch_forward_few(const ForwardArgs& p, Elem type, bool gated, hipStream_t stream);
hipError_t launch_forward(const ForwardArgs& p, Elem type, bool gated, hipStream_t stream);
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

// recv rows pitch elements apart; w [T][k].
hipError_t launch_dispatch_weighted(const void* x, const float* w, const int32_t* pair_row, void* recv, int64_t T, int k,
                                    int H, int pitch, int64_t cap, hipStream_t stream);
hipError_t launch_dispatch_grad(const void* d, const void* x, const float* w, const int32_t* pair_row, void* dx, float* dw,
                                int64_t T, int k, int H, int pitch, int64_t cap, hipStream_t stream);

// w: [T][k] or null. recv rows pitch bytes apart.
hipError_t launch_dispatch_int8(const void* x, const float* w, const int32_t* pair_row, void* recv, float* scale, int64_t T,
                                int k, int H, int pitch, int64_t cap, hipStream_t stream);
// The first count[0] of `rows` rows, or with count null all of them. Strides in 16-byte pieces.
hipError_t launch_quantize_rows(const void* a, void* q, float* scale, const int32_t* count, int64_t rows, int K, int64_t a_ld,
                                int64_t q_ld, hipStream_t stream);

}  // namespace epl
