// Dispatch with the gate weights applied, and its gradient: for token g with valid choices j in packed rows r,
//   recv[r] = w[g][j] x[g];   dx[g] = sum_j w[g][j] drecv[r],   dw[g][j] = <x[g], drecv[r]>.
// HBM traffic bounds both.
#include "experts.h"
#include "rows_body.h"

namespace epl {

// As the plain bf16 dispatch: one (token, 1 KiB column chunk) a wave, two waves a workgroup, held at 4 waves per SIMD (6 with
// one or two choices). 8192 tokens of 7168 columns to 8 rows each: 191 us (without the weights 190); not held 198, held at 2 / 3
// / 5 / 6 228 / 193 / 192 / 195; with default stores 214, with streaming ones 194.
template <bool FEW>
__global__ void __launch_bounds__(kPlainThreads) __attribute__((amdgpu_waves_per_eu(FEW ? 6 : 4, FEW ? 6 : 4)))
    dispatch_weighted_kernel(const u32x4* __restrict__ x, const float* __restrict__ w, const int32_t* __restrict__ pair_row,
                             u32x4* __restrict__ recv, int64_t T, int k, int nv, int pv, int chunks, int64_t cap) {
  const int lane = threadIdx.x % kWave;
  const int64_t units = T * chunks;
  for (int64_t u = (int64_t)blockIdx.x * kPlainWaves + threadIdx.x / kWave; u < units;
       u += (int64_t)gridDim.x * kPlainWaves) {
    const int64_t g = u / chunks;
    const int v = (int)(u - g * chunks) * kWave + lane;
    const u32x4 buf = x[g * nv + std::min(v, nv - 1)];
    const int my_row = lane < k ? pair_row[g * k + lane] : -1;
    const float my_w = lane < k ? w[g * k + lane] : 0.0f;
    for (int j = 0; j < k; ++j) {
      const int row = __builtin_amdgcn_readlane(my_row, j);
      if (row < 0 || row >= cap) continue;
      const float wj = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(my_w), j));
      u32x4 o;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = f32x2_to_bf16x2(wj * bf16lo_to_f32(buf[i]), wj * bf16hi_to_f32(buf[i]));
      if (v < nv) store_row_policy<kCachePolicySc1>(o, recv + (int64_t)row * pv, nv, v);
    }
  }
}

// One workgroup a token. A thread's products are summed in fp32 over its own columns, then over the wave and the waves in a
// fixed order. dx may be x: a thread reads its columns before it writes them. 8192 tokens of 7168 columns with 8 rows each:
// 205 us (5.7 TB/s) with 448 threads held at 4 waves per SIMD, 211 not held, 258 at 3; stores with the default policy cost 5%.
// grad_threads: as many as the vectors need in the fewest equal passes of at most 256, or of at most 512 where those make
// workgroups of seven or eight waves: two of them take 14 or all of a compute unit's 16 places, two of five or six 10 or 12.
// us with at most 512 / 256, of seven or eight waves: 8 choices, 512 vectors 205 / 218, 832 215 / 224, 896 216 / 224, 1024 217 /
// 226, 1280 218 / 228, 1536 221 / 229, 2048 223 / 228; 4 choices, 512 251 / 248, 832 246 / 259, 1024 239 / 260, 1536 246 / 265,
// 2048 251 / 265. Of five or six: 8 choices, 640 231 / 220, 768 221 / 222, 1152 219 / 226. Rows of one pass: 448 230 / 217.
// Fewer choices have too little to load: 3, 512 295 / 269, 896 288 / 282, 1024 272 / 279. The instance for more is seldom faster
// for it: 16, 512 206 / 205, 896 215 / 213, 1024 203 / 211; 32, 512 231 / 219, 896 242 / 214, 1024 223 / 214.
// KMAX: choices held in registers (k <= KMAX).
constexpr int kDispatchGradThreads = 512;
constexpr int kDispatchGradWaves = kDispatchGradThreads / kWave;
template <int KMAX>
__global__ void __launch_bounds__(kDispatchGradThreads) __attribute__((amdgpu_waves_per_eu(KMAX <= 8 ? 4 : 2, 4)))
    dispatch_grad_kernel(const u32x4* __restrict__ d, const u32x4* x, const float* __restrict__ w,
                         const int32_t* __restrict__ pair_row, u32x4* dx, float* __restrict__ dw, int64_t T, int k, int nv,
                         int pv, int64_t cap) {
  __shared__ float part[kDispatchGradWaves][EPL_MAX_TOPK];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, threads = blockDim.x;
  constexpr int kGroup = KMAX < 8 ? KMAX : 8;  // rows loaded before any is consumed
  for (int64_t g = blockIdx.x; g < T; g += gridDim.x) {
    float acc[KMAX];
#pragma unroll
    for (int j = 0; j < KMAX; ++j) acc[j] = 0.0f;
    for (int c = threadIdx.x; c < nv; c += threads) {
      const u32x4 xv = __builtin_nontemporal_load(x + g * nv + c);
      float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
      for (int j0 = 0; j0 < KMAX; j0 += kGroup) {
        u32x4 buf[kGroup];
        int row[kGroup];
#pragma unroll
        for (int jj = 0; jj < kGroup; ++jj) {
          const int j = j0 + jj;
          row[jj] = j < k ? __builtin_amdgcn_readfirstlane(pair_row[g * k + j]) : -1;
          if (row[jj] >= cap) row[jj] = -1;
          if (row[jj] >= 0) buf[jj] = __builtin_nontemporal_load(d + (int64_t)row[jj] * pv + c);
        }
#pragma unroll
        for (int jj = 0; jj < kGroup; ++jj) {
          if (row[jj] < 0) continue;
          const float wj = w[g * k + j0 + jj];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float lo = bf16lo_to_f32(buf[jj][i]), hi = bf16hi_to_f32(buf[jj][i]);
            acc[j0 + jj] = fmaf(bf16lo_to_f32(xv[i]), lo, acc[j0 + jj]);
            acc[j0 + jj] = fmaf(bf16hi_to_f32(xv[i]), hi, acc[j0 + jj]);
            sum[2 * i] = fmaf(wj, lo, sum[2 * i]);
            sum[2 * i + 1] = fmaf(wj, hi, sum[2 * i + 1]);
          }
        }
      }
      u32x4 o;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = f32x2_to_bf16x2(sum[2 * i], sum[2 * i + 1]);
      store_row_policy<kCachePolicySc1Nt>(o, dx + g * nv, nv, c);
    }
    __syncthreads();  // the previous token's sums have been read
#pragma unroll
    for (int j = 0; j < KMAX; ++j) {
      if (j >= k) continue;
      float v = acc[j];
#pragma unroll
      for (int off = kWave / 2; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
      if (lane == 0) part[wave][j] = v;
    }
    __syncthreads();
    if (threadIdx.x < k) {
      float v = 0.0f;
      for (int i = 0; i < threads / kWave; ++i) v += part[i][threadIdx.x];
      dw[g * k + threadIdx.x] = v;
    }
  }
}

hipError_t launch_dispatch_weighted(const void* x, const float* w, const int32_t* pair_row, void* recv, int64_t T, int k,
                                    int H, int pitch, int64_t cap, hipStream_t stream) {
  if (T == 0) return hipSuccess;
  const int nv = H / 8, chunks = (nv + kWave - 1) / kWave;
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(unit_grid(T * chunks, kPlainWaves, kPlainThreads)), dim3(kPlainThreads), 0, stream,
                       static_cast<const u32x4*>(x), w, pair_row, static_cast<u32x4*>(recv), T, k, nv, pitch / 8, chunks,
                       cap);
  };
  if (k <= kFewChoices)
    launch(dispatch_weighted_kernel<true>);
  else
    launch(dispatch_weighted_kernel<false>);
  return hipGetLastError();
}

static int grad_threads(int nv, int k) {
  const auto equal = [&](int most) {
    const int passes = (nv + most - 1) / most;
    return ((nv + passes - 1) / passes + kWave - 1) / kWave * kWave;
  };
  const int wide = equal(kDispatchGradThreads);
  return k >= 4 && k <= 8 && nv >= kDispatchGradThreads && wide / kWave >= 7 ? wide : equal(256);
}

hipError_t launch_dispatch_grad(const void* d, const void* x, const float* w, const int32_t* pair_row, void* dx, float* dw,
                                int64_t T, int k, int H, int pitch, int64_t cap, hipStream_t stream) {
  if (T == 0) return hipSuccess;
  const int nv = H / 8, threads = grad_threads(nv, k);
  const dim3 grid((unsigned)std::min<int64_t>(T, 1 << 20));
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, stream, static_cast<const u32x4*>(d),
                       static_cast<const u32x4*>(x), w, pair_row, static_cast<u32x4*>(dx), dw, T, k, nv, pitch / 8, cap);
  };
  if (k <= 8)
    launch(dispatch_grad_kernel<8>);
  else
    launch(dispatch_grad_kernel<EPL_MAX_TOPK>);
  return hipGetLastError();
}

}  // namespace epl
