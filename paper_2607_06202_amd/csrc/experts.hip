// The experts' products on the packed rows: forward, input gradient and weight gradient, one tile loop
// (gemm_tile.h) with three ways of reading the operands and the work of each call fused into its end.
#include "gemm_tile.h"
#include "experts.h"

namespace epl {

constexpr int kCus = 256;  // compute units of an MI355X

// The steps of one tile: stage s+1 is loaded while stage s is multiplied; one barrier per step.
template <class S, class P, class A, class B>
__device__ __forceinline__ void run_steps(const P& prod, A& a, B& b, int steps, uint32_t lds, int wave,
                                          f32x4 (&acc)[S::MF][S::NF]) {
  uint32_t cur = lds, nxt = lds + S::kStage;
  a.load(cur, wave);
  b.load(cur + A::kBytes, wave);
  for (int s = 0; s < steps; ++s) {
    wait_tiles();
    if (s + 1 < steps) {
      a.load(nxt, wave);
      b.load(nxt + A::kBytes, wave);
    }
    prod.step(cur, acc, nullptr);
    const uint32_t t = cur;
    cur = nxt;
    nxt = t;
  }
}

template <class S>
__device__ __forceinline__ void clear(f32x4 (&acc)[S::MF][S::NF]) {
#pragma unroll
  for (int m = 0; m < S::MF; ++m)
#pragma unroll
    for (int n = 0; n < S::NF; ++n) acc[m][n] = f32x4{0, 0, 0, 0};
}

__device__ __forceinline__ u32x4 pack8(const float (&v)[8]) {
  return u32x4{f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]), f32x2_to_bf16x2(v[4], v[5]),
               f32x2_to_bf16x2(v[6], v[7])};
}
__device__ __forceinline__ void unpack8(u32x4 w, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = bf16lo_to_f32(w[i]);
    v[2 * i + 1] = bf16hi_to_f32(w[i]);
  }
}

// ---------------------------------------------------------------- forward
// GATED: B tile = BN/2 gate rows and BN/2 up rows; BN/2 output columns.
template <class S, bool FP8, bool GATED>
__global__ void __launch_bounds__(S::kThreads) forward_kernel(ForwardArgs p) {
  __shared__ __attribute__((aligned(1024))) char tiles[2 * S::kStage];
  __shared__ int mt[EPL_MAX_EXPERTS + 1];
  constexpr int kCols = GATED ? S::BN / 2 : S::BN;  // output columns of a tile
  const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int rho = lane & 15, q = lane >> 4;
  const int esize = FP8 ? 1 : 2;
  count_row_tiles<S::BM>(p.expert_off, p.E, p.cap, mt);
  Products<S, false, false, FP8, GATED> prod;
  prod.init(wave, lane);
  Operand<false, S::BM, S::kWaves, false> a;
  Operand<false, S::BN, S::kWaves, true, GATED> b;
  const int nt = (p.N + kCols - 1) / kCols;
  const int64_t total = (int64_t)mt[p.E] * nt;
  const int steps = (p.K * esize + kStepBytes - 1) / kStepBytes;
  const uint32_t lds = lds_addr(tiles);
  const int slot = xcd_slot(blockIdx.x, gridDim.x);
  for (int64_t t = slot; t < total; t += gridDim.x) {
    const int e = uniform(quaternary_find(mt, p.E, t / nt));
    int beg, end, m, n;
    expert_rows(p.expert_off, e, p.cap, beg, end);
    beg = uniform(beg);
    end = uniform(end);
    const int m0 = uniform(mt[e]);
    band_tile(t - (int64_t)m0 * nt, uniform(mt[e + 1]) - m0, nt, 8, m, n);
    const int row0 = beg + m * S::BM, rows = end - row0;
    const int col0 = n * kCols, cols = p.N - col0;
    if (m < 0 || rows <= 0) continue;
    const int64_t ldb = (int64_t)p.K * esize;
    const int64_t boff = e * p.expert_stride * esize + col0 * ldb;
    a.lanes(rows, p.a_ld, wave, lane);
    b.lanes(cols, ldb, wave, lane);
    a.start_rows(p.a + row0 * p.a_ld, nullptr, std::min(rows, S::BM), p.a_ld, p.K * esize);
    b.start_rows(p.w + boff, p.w2 + boff, std::min(cols, kCols), ldb, p.K * esize);
    f32x4 acc[S::MF][S::NF];
    clear<S>(acc);
    const int wm0 = (wave / S::WN) * S::MF * 16, wn0 = (wave % S::WN) * S::NF * 16 / (GATED ? 2 : 1);
    wait_tiles();  // the previous tile's reads are done
    if constexpr (!FP8) {
      run_steps<S>(prod, a, b, steps, lds, wave, acc);
    } else {
      // Row scales one step ahead; touched right after the wait for the step's tiles, where they have arrived.
      float sc[S::MF], sn[S::MF];
      const float* sp[S::MF];
#pragma unroll
      for (int f = 0; f < S::MF; ++f) {
        sp[f] = p.a_scale + (int64_t)std::min(row0 + wm0 + f * 16 + rho, end - 1) * (p.K / 128);
        sn[f] = sp[f][0];
      }
      uint32_t cur = lds, nxt = lds + S::kStage;
      a.load(cur, wave);
      b.load(cur + S::BM * kStepBytes, wave);
      for (int s = 0; s < steps; ++s) {
        wait_tiles();
#pragma unroll
        for (int f = 0; f < S::MF; ++f) {
          asm volatile("" : "+v"(sn[f]));
          sc[f] = sn[f];
        }
        if (s + 1 < steps) {
#pragma unroll
          for (int f = 0; f < S::MF; ++f) sn[f] = sp[f][s + 1];
          a.load(nxt, wave);
          b.load(nxt + S::BM * kStepBytes, wave);
        }
        prod.step(cur, acc, sc);
        const uint32_t u = cur;
        cur = nxt;
        nxt = u;
      }
    }
    // Lane: rows m0 + rho of each row fragment, eight consecutive columns of each pair of column fragments.
    constexpr int kPairs = (GATED ? S::NF / 2 : S::NF) / 2;
#pragma unroll
    for (int g = 0; g < kPairs; ++g) {
      const int c = col0 + wn0 + g * 32 + q * 8;
      if (c >= p.N) continue;
      float s1[8], s2[8], bias[8];
      if constexpr (FP8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          s1[i] = p.w_scale[(int64_t)e * p.N + c + i];
          if constexpr (GATED) s2[i] = p.w2_scale[(int64_t)e * p.N + c + i];
        }
      }
      if constexpr (!GATED) {
        if (p.bias) unpack8(*(const u32x4*)(p.bias + ((int64_t)e * p.N + c) * 2), bias);
      }
#pragma unroll
      for (int f = 0; f < S::MF; ++f) {
        const int64_t row = row0 + wm0 + f * 16 + rho;
        if (row >= end) continue;
        float v[8], u[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          v[i] = acc[f][g * 2 + i / 4][i % 4];
          if constexpr (FP8) v[i] *= s1[i];
          if constexpr (GATED) {
            u[i] = acc[f][S::NF / 2 + g * 2 + i / 4][i % 4];
            if constexpr (FP8) u[i] *= s2[i];
          } else if (p.bias) {
            v[i] += bias[i];
          }
        }
        if (p.pre) {
          if constexpr (GATED) {
            *(u32x4*)(p.pre + (row * 2 * p.N + c) * 2) = pack8(v);
            *(u32x4*)(p.pre + (row * 2 * p.N + p.N + c) * 2) = pack8(u);
          } else {
            *(u32x4*)(p.pre + (row * p.N + c) * 2) = pack8(v);
          }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          v[i] = activate(p.act, v[i]);
          if constexpr (GATED) v[i] *= u[i];
        }
        if constexpr (!GATED) {
          if (p.residual) {
            float r[8];
            unpack8(*(const u32x4*)(p.residual + row * p.res_ld + c * 2), r);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += r[i];
          }
        }
        *(u32x4*)(p.out + row * p.out_ld + c * 2) = pack8(v);
      }
    }
  }
}

// ---------------------------------------------------------------- gradient of the rows
// dx[r] = sum over parts and n of d[r][part * N + n] w_part[e][n]: the reduction runs over the weights' rows.
template <class S>
__global__ void __launch_bounds__(S::kThreads) row_grad_kernel(RowGradArgs p) {
  __shared__ __attribute__((aligned(1024))) char tiles[2 * S::kStage];
  __shared__ int mt[EPL_MAX_EXPERTS + 1];
  const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int rho = lane & 15, q = lane >> 4;
  count_row_tiles<S::BM>(p.expert_off, p.E, p.cap, mt);
  Products<S, false, true, false> prod;
  prod.init(wave, lane);
  Operand<false, S::BM, S::kWaves, false> a;
  Operand<true, S::BN, S::kWaves, true> b;
  const int nt = (p.K + S::BN - 1) / S::BN;
  const int64_t total = (int64_t)mt[p.E] * nt;
  const int part_steps = (p.N + kTileK - 1) / kTileK;
  const int steps = part_steps * p.parts;
  const uint32_t lds = lds_addr(tiles);
  const int64_t lda = (int64_t)p.N * p.parts * 2, ldb = (int64_t)p.K * 2;
  for (int64_t t = xcd_slot(blockIdx.x, gridDim.x); t < total; t += gridDim.x) {
    const int e = uniform(quaternary_find(mt, p.E, t / nt));
    int beg, end, m, n;
    expert_rows(p.expert_off, e, p.cap, beg, end);
    beg = uniform(beg);
    end = uniform(end);
    const int m0 = uniform(mt[e]);
    band_tile(t - (int64_t)m0 * nt, uniform(mt[e + 1]) - m0, nt, 8, m, n);
    const int row0 = beg + m * S::BM, rows = end - row0;
    const int col0 = n * S::BN, cols = std::min(p.K - col0, S::BN);
    if (m < 0 || rows <= 0) continue;
    a.lanes(rows, lda, wave, lane);
    b.lanes(cols, ldb, wave, lane);
    const int64_t boff = (e * p.expert_stride + col0) * 2;
    f32x4 acc[S::MF][S::NF];
    clear<S>(acc);
    uint32_t cur = lds, nxt = lds + S::kStage;
    int at = 0;  // steps loaded
    auto load = [&](uint32_t stage) {
      if (at == 0 || at == part_steps) {
        const int part = at == 0 ? 0 : 1;
        a.start_rows(p.d + row0 * lda + (int64_t)part * p.N * 2, nullptr, std::min(rows, S::BM), lda, p.N * 2);
        b.start_cols((part ? p.w2 : p.w) + boff, p.N, cols, ldb);
      }
      a.load(stage, wave);
      b.load(stage + S::BM * kStepBytes, wave);
      ++at;
    };
    wait_tiles();
    load(cur);
    for (int s = 0; s < steps; ++s) {
      wait_tiles();
      if (s + 1 < steps) load(nxt);
      prod.step(cur, acc, nullptr);
      const uint32_t u = cur;
      cur = nxt;
      nxt = u;
    }
    const int wm0 = (wave / S::WN) * S::MF * 16, wn0 = (wave % S::WN) * S::NF * 16;
#pragma unroll
    for (int g = 0; g < S::NF / 2; ++g) {
      const int c = col0 + wn0 + g * 32 + q * 8;
      if (c >= p.K) continue;
#pragma unroll
      for (int f = 0; f < S::MF; ++f) {
        const int64_t row = row0 + wm0 + f * 16 + rho;
        if (row >= end) continue;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = acc[f][g * 2 + i / 4][i % 4];
        *(u32x4*)(p.dx + row * p.dx_ld + c * 2) = pack8(v);
      }
    }
  }
}

// ---------------------------------------------------------------- gradient of the weights
// dw_part[e][n][k] = sum over the expert's rows r of d[r][part * N + n] x[r][k]: the reduction runs over the rows,
// which an expert without any leaves at zero.
template <class S>
__global__ void __launch_bounds__(S::kThreads) weight_grad_kernel(WeightGradArgs p) {
  __shared__ __attribute__((aligned(1024))) char tiles[2 * S::kStage];
  const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int rho = lane & 15, q = lane >> 4;
  Products<S, true, true, false> prod;
  prod.init(wave, lane);
  Operand<true, S::BM, S::kWaves, false> a;
  Operand<true, S::BN, S::kWaves, true> b;
  const int mt = (p.N + S::BM - 1) / S::BM * p.parts, nt = (p.K + S::BN - 1) / S::BN;
  const int64_t per = (int64_t)mt * nt;
  const int64_t total = per * p.E;
  const uint32_t lds = lds_addr(tiles);
  const int64_t lda = (int64_t)p.N * p.parts * 2;
  for (int64_t t = xcd_slot(blockIdx.x, gridDim.x); t < total; t += gridDim.x) {
    const int e = uniform((int)(t / per));
    int beg, end, mi, n;
    expert_rows(p.expert_off, e, p.cap, beg, end);
    beg = uniform(beg);
    end = uniform(end);
    band_tile(t - e * per, mt, nt, 8, mi, n);
    const int part = mi / (mt / p.parts), m0 = (mi % (mt / p.parts)) * S::BM;
    const int mrows = std::min(p.N - m0, S::BM);
    const int col0 = n * S::BN, cols = std::min(p.K - col0, S::BN);
    a.lanes(mrows, lda, wave, lane);
    b.lanes(cols, p.x_ld, wave, lane);
    a.start_cols(p.d + beg * lda + ((int64_t)part * p.N + m0) * 2, end - beg, mrows, lda);
    b.start_cols(p.x + beg * p.x_ld + col0 * 2, end - beg, cols, p.x_ld);
    f32x4 acc[S::MF][S::NF];
    clear<S>(acc);
    const int steps = (end - beg + kTileK - 1) / kTileK;
    wait_tiles();
    if (steps > 0) run_steps<S>(prod, a, b, steps, lds, wave, acc);
    char* dw = (part ? p.dw2 : p.dw) + (int64_t)e * p.N * p.K * 2;
    const int wm0 = (wave / S::WN) * S::MF * 16, wn0 = (wave % S::WN) * S::NF * 16;
#pragma unroll
    for (int g = 0; g < S::NF / 2; ++g) {
      const int c = col0 + wn0 + g * 32 + q * 8;
      if (c >= p.K) continue;
#pragma unroll
      for (int f = 0; f < S::MF; ++f) {
        const int r = m0 + wm0 + f * 16 + rho;
        if (r >= p.N) continue;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = acc[f][g * 2 + i / 4][i % 4];
        *(u32x4*)(dw + ((int64_t)r * p.K + c) * 2) = pack8(v);
      }
    }
  }
}

// ---------------------------------------------------------------- gradients through the activation
// Gated: dpre = (dh u act'(g), dh act(g)) from the kept projections, both rounded to bf16: they are operands of
// the two bf16 products that follow. dpre may be pre: a thread reads its values before it writes them.
__global__ void __launch_bounds__(256) gated_pre_grad_kernel(const char* dh, const char* pre, char* dpre,
                                                             const int32_t* expert_off, int E, int cap, int I,
                                                             int act) {
  const int64_t nv = I / 8;
  const int64_t n = std::min(std::max(expert_off[E], 0), cap) * nv;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / nv, c = i - r * nv;
    float d[8], g[8], u[8];
    unpack8(((const u32x4*)dh)[i], d);
    unpack8(((const u32x4*)pre)[r * 2 * nv + c], g);
    unpack8(((const u32x4*)pre)[r * 2 * nv + nv + c], u);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float a = activate(act, g[j]), ag = activate_grad(act, g[j]);
      g[j] = d[j] * u[j] * ag;
      u[j] = d[j] * a;
    }
    ((u32x4*)dpre)[r * 2 * nv + c] = pack8(g);
    ((u32x4*)dpre)[r * 2 * nv + nv + c] = pack8(u);
  }
}

// Linear: dpre = dy act'(pre) in bf16.
__global__ void __launch_bounds__(256) pre_grad_kernel(const char* dy, const char* pre, char* dpre,
                                                       const int32_t* expert_off, int E, int cap, int N, int act) {
  const int64_t n = std::min(std::max(expert_off[E], 0), cap) * (int64_t)(N / 8);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    float d[8], v[8];
    unpack8(((const u32x4*)dy)[i], d);
    unpack8(((const u32x4*)pre)[i], v);
#pragma unroll
    for (int j = 0; j < 8; ++j) d[j] *= activate_grad(act, v[j]);
    ((u32x4*)dpre)[i] = pack8(d);
  }
}

// dbias[e][n] = sum over the expert's rows of dy act'(pre), unrounded terms summed in fp32 in a fixed order:
// 8 row lanes of a workgroup take every eighth row of 256 columns, then are added in order.
__global__ void __launch_bounds__(256) bias_grad_kernel(const char* dy, const char* pre, char* dbias,
                                                        const int32_t* expert_off, int cap, int N, int act) {
  __shared__ float part[8][32][8 + 1];
  const int e = blockIdx.y, cv = threadIdx.x % 32, rl = threadIdx.x / 32;
  const int c = blockIdx.x * 32 + cv;  // 8-column vector
  int beg, end;
  expert_rows(expert_off, e, cap, beg, end);
  float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (c * 8 < N) {
    for (int64_t r = beg + rl; r < end; r += 8) {
      float d[8], v[8];
      unpack8(*(const u32x4*)(dy + (r * N + c * 8) * 2), d);
      if (act != EPL_ACT_NONE) {
        unpack8(*(const u32x4*)(pre + (r * N + c * 8) * 2), v);
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] *= activate_grad(act, v[j]);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] += d[j];
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) part[rl][cv][j] = s[j];
  __syncthreads();
  if (rl == 0 && c * 8 < N) {
    for (int k = 1; k < 8; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] += part[k][cv][j];
    *(u32x4*)(dbias + ((int64_t)e * N + c * 8) * 2) = pack8(s);
  }
}

// ---------------------------------------------------------------- launches
using Mid = Shape<128, 128, 2, 2>;

static unsigned persistent_grid(int64_t tiles, int per_cu) {
  return (unsigned)std::min<int64_t>(tiles, (int64_t)kCus * per_cu);
}

// Row tiles of BM over at most `rows` rows of E experts.
static int64_t row_tiles(int64_t rows, int E, int BM) { return rows / BM + std::min<int64_t>(E, rows); }

template <class S, bool FP8, bool GATED>
static hipError_t forward_as(const ForwardArgs& p, hipStream_t stream) {
  const int cols = GATED ? S::BN / 2 : S::BN;
  const int64_t tiles = row_tiles(p.cap, p.E, S::BM) * ((p.N + cols - 1) / cols);
  hipLaunchKernelGGL((forward_kernel<S, FP8, GATED>), dim3(persistent_grid(tiles, 2)), dim3(S::kThreads), 0, stream,
                     p);
  return hipGetLastError();
}

hipError_t launch_forward(const ForwardArgs& p, bool fp8, bool gated, hipStream_t stream) {
  if (p.cap == 0) return hipSuccess;
  if (fp8) return gated ? forward_as<Mid, true, true>(p, stream) : forward_as<Mid, true, false>(p, stream);
  return gated ? forward_as<Mid, false, true>(p, stream) : forward_as<Mid, false, false>(p, stream);
}

hipError_t launch_row_grad(const RowGradArgs& p, hipStream_t stream) {
  if (p.cap == 0) return hipSuccess;
  using S = Mid;
  const int64_t tiles = row_tiles(p.cap, p.E, S::BM) * ((p.K + S::BN - 1) / S::BN);
  hipLaunchKernelGGL((row_grad_kernel<S>), dim3(persistent_grid(tiles, 2)), dim3(S::kThreads), 0, stream, p);
  return hipGetLastError();
}

hipError_t launch_weight_grad(const WeightGradArgs& p, hipStream_t stream) {
  using S = Mid;
  const int64_t tiles =
      (int64_t)p.E * p.parts * ((p.N + S::BM - 1) / S::BM) * ((p.K + S::BN - 1) / S::BN);
  hipLaunchKernelGGL((weight_grad_kernel<S>), dim3(persistent_grid(tiles, 2)), dim3(S::kThreads), 0, stream, p);
  return hipGetLastError();
}

static unsigned elementwise_grid(int64_t n) {
  return (unsigned)std::max<int64_t>(1, std::min<int64_t>((n + 255) / 256, kCus * 16));
}

hipError_t launch_gated_pre_grad(const void* dh, const void* pre, void* dpre, const int32_t* expert_off, int E,
                                 int cap, int I, int act, hipStream_t stream) {
  if (cap == 0) return hipSuccess;
  hipLaunchKernelGGL(gated_pre_grad_kernel, dim3(elementwise_grid((int64_t)cap * (I / 8))), dim3(256), 0, stream,
                     (const char*)dh, (const char*)pre, (char*)dpre, expert_off, E, cap, I, act);
  return hipGetLastError();
}

hipError_t launch_pre_grad(const void* dy, const void* pre, void* dpre, const int32_t* expert_off, int E, int cap,
                           int N, int act, hipStream_t stream) {
  if (cap == 0) return hipSuccess;
  hipLaunchKernelGGL(pre_grad_kernel, dim3(elementwise_grid((int64_t)cap * (N / 8))), dim3(256), 0, stream,
                     (const char*)dy, (const char*)pre, (char*)dpre, expert_off, E, cap, N, act);
  return hipGetLastError();
}

hipError_t launch_bias_grad(const void* dy, const void* pre, void* dbias, const int32_t* expert_off, int E, int cap,
                            int N, int act, hipStream_t stream) {
  hipLaunchKernelGGL(bias_grad_kernel, dim3((unsigned)((N + 255) / 256), (unsigned)E), dim3(256), 0, stream,
                     (const char*)dy, (const char*)pre, (char*)dbias, expert_off, cap, N, act);
  return hipGetLastError();
}

}  // namespace epl
