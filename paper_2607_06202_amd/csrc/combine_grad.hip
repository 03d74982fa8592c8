// Gradient of combine: for token g with valid choices j in packed rows r,
//   dy[r] = topk_w[g][j] * dout[g],   dtopk_w[g][j] = <dout[g], y[r]>.
//
// One workgroup per token. Its threads keep their part of dout in registers and walk the token's rows: each
// row of y is read once, each row of dy written once, dout read once. The products are summed in fp32, a thread's
// own columns first, then a fixed tree over the wave and the waves in order, so the result does not depend on
// timing. HBM traffic bounds it.
#include "epl_internal.h"
#include "experts.h"

namespace epl {

constexpr int kGradThreads = 256;
constexpr int kGradWaves = kGradThreads / kWave;

// KMAX: choices held in registers (k <= KMAX).
template <int KMAX>
__global__ void __launch_bounds__(kGradThreads)
    combine_grad_kernel(const u32x4* __restrict__ dout, const u32x4* y, const float* __restrict__ w,
                        const int32_t* __restrict__ pair_row, u32x4* dy, float* __restrict__ dw, int64_t T, int k,
                        int nv, int pv, int cap) {
  __shared__ float part[kGradWaves][EPL_MAX_TOPK];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  for (int64_t g = blockIdx.x; g < T; g += gridDim.x) {
    float acc[KMAX];
#pragma unroll
    for (int j = 0; j < KMAX; ++j) acc[j] = 0.0f;
    for (int c = threadIdx.x; c < nv; c += kGradThreads) {
      const u32x4 dv = __builtin_nontemporal_load(dout + g * nv + c);
      float d[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        d[2 * i] = bf16lo_to_f32(dv[i]);
        d[2 * i + 1] = bf16hi_to_f32(dv[i]);
      }
      constexpr int kGroup = KMAX < 8 ? KMAX : 8;  // rows loaded before any is consumed
#pragma unroll
      for (int j0 = 0; j0 < KMAX; j0 += kGroup) {
        u32x4 buf[kGroup];
        int row[kGroup];
#pragma unroll
        for (int jj = 0; jj < kGroup; ++jj) {
          const int j = j0 + jj;
          row[jj] = j < k ? __builtin_amdgcn_readfirstlane(pair_row[g * k + j]) : -1;
          if (row[jj] >= cap) row[jj] = -1;
          if (row[jj] >= 0) buf[jj] = __builtin_nontemporal_load(y + (int64_t)row[jj] * pv + c);
        }
#pragma unroll
        for (int jj = 0; jj < kGroup; ++jj) {
          if (row[jj] < 0) continue;
          const float wj = w[g * k + j0 + jj];
          u32x4 o;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            acc[j0 + jj] = fmaf(d[2 * i], bf16lo_to_f32(buf[jj][i]), acc[j0 + jj]);
            acc[j0 + jj] = fmaf(d[2 * i + 1], bf16hi_to_f32(buf[jj][i]), acc[j0 + jj]);
            o[i] = f32x2_to_bf16x2(wj * d[2 * i], wj * d[2 * i + 1]);
          }
          __builtin_nontemporal_store(o, dy + (int64_t)row[jj] * pv + c);
        }
      }
    }
    __syncthreads();  // the previous token's sums have been read
#pragma unroll
    for (int j = 0; j < KMAX; ++j) {
      float v = acc[j];
#pragma unroll
      for (int off = kWave / 2; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
      if (lane == 0 && j < k) part[wave][j] = v;
    }
    __syncthreads();
    if (threadIdx.x < k) {
      float v = 0.0f;
#pragma unroll
      for (int i = 0; i < kGradWaves; ++i) v += part[i][threadIdx.x];
      dw[g * k + threadIdx.x] = v;
    }
  }
}

hipError_t launch_combine_grad(const void* dout, const void* y, const float* w, const int32_t* pair_row, void* dy,
                               float* dw, int64_t T, int k, int H, int pitch, int64_t cap, hipStream_t stream) {
  if (T == 0) return hipSuccess;
  const dim3 grid((unsigned)std::min<int64_t>(T, 1 << 20));
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kGradThreads), 0, stream, static_cast<const u32x4*>(dout),
                       static_cast<const u32x4*>(y), w, pair_row, static_cast<u32x4*>(dy), dw, T, k, H / 8, pitch / 8,
                       (int)std::min<int64_t>(cap, INT_MAX));
  };
  if (k <= 8)
    launch(combine_grad_kernel<8>);
  else
    launch(combine_grad_kernel<EPL_MAX_TOPK>);
  return hipGetLastError();
}

}  // namespace epl
