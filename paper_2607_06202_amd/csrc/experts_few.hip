// The experts' forward product for a handful of rows: one token, a few sequences decoding.
//
// Reading the weights once is all there is to do, and a tile's start and end would cost as much as its middle. So a
// workgroup takes 16 * NF weight rows of one expert, its four waves each take every fourth 128-byte step of the
// reduction, and the four partial sums are joined through LDS in a fixed order. A wave's fragments come straight from
// memory, kDepth steps ahead: 2 * (NF + 1) KiB a step in flight.
//
// For at most 16 packed rows in all (few_rows): an expert's rows are one fragment.
//
// Workgroup i takes the i-th expert that has rows, which it finds from the offsets by itself; the grid is for
// as many experts as there can be.
#include "gemm_tile.h"
#include "experts.h"

namespace epl {

constexpr int kFewWaves = 4, kDepth = 4;

// The i-th expert with rows (E if there are not that many). Wave-uniform.
__device__ __forceinline__ int nth_expert(const int32_t* expert_off, int E, int cap, int i, int lane) {
  for (int e0 = 0; e0 < E; e0 += kWave) {
    const int e = e0 + lane;
    bool has = false;
    if (e < E) {
      const int beg = std::min(std::max(expert_off[e], 0), cap), end = std::min(std::max(expert_off[e + 1], beg), cap);
      has = end > beg;
    }
    const uint64_t m = __ballot(has);
    const int n = __builtin_popcountll(m);
    if (i < n) {
      // The bit with i set bits below it.
      const uint64_t mine = __ballot(has && rank_in_mask(m) == i);
      return e0 + __builtin_ctzll(mine);
    }
    i -= n;
  }
  return E;
}

template <int NF, bool FP8, bool GATED>
__global__ void __launch_bounds__(kFewWaves* kWave, 2) few_rows_kernel(ForwardArgs p) {
  constexpr int kCols = 16 * NF / (GATED ? 2 : 1), kEsize = FP8 ? 1 : 2;
  constexpr int kUnits = kCols / 32;  // groups of 32 output columns
  __shared__ f32x4 part[kFewWaves][NF][kWave];
  const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int rho = lane & 15, q = lane >> 4;
  const int nt = (p.N + kCols - 1) / kCols;
  const int which = blockIdx.x / nt, col0 = (blockIdx.x - which * nt) * kCols;
  const int e = uniform(nth_expert(p.expert_off, p.E, p.cap, which, lane));
  if (e == p.E) return;
  const int beg = uniform(std::min(std::max(p.expert_off[e], 0), p.cap));
  const int rows = uniform(std::min(std::max(p.expert_off[e + 1], beg), p.cap)) - beg;  // 1 to 16
  const int cols = std::min(p.N - col0, kCols);
  const int kbytes = p.K * kEsize, steps = (kbytes + 127) / 128, nb = p.K / 128;
  const int64_t ldb = kbytes;
  const int64_t boff = e * p.expert_stride * kEsize + col0 * ldb;
  const auto rsrc = [](const char* base, int64_t bytes) {
    const uint64_t at = (uint64_t)base;
    const uint64_t uni = (uint64_t)(uint32_t)uniform((int)(uint32_t)at) | (uint64_t)(uint32_t)uniform((int)(at >> 32)) << 32;
    return __builtin_amdgcn_make_buffer_rsrc((void*)uni, 0, uniform((int)std::min<int64_t>(bytes, INT_MAX)),
                                             kBufferRsrcWord3);
  };
  const __amdgpu_buffer_rsrc_t rb = rsrc(p.w + boff, (cols - 1) * ldb + kbytes);
  const __amdgpu_buffer_rsrc_t rb2 = GATED ? rsrc(p.w2 + boff, (cols - 1) * ldb + kbytes) : rb;
  // Offsets of the lane's weight rows; those past the last one are out of range.
  int vb[NF];
#pragma unroll
  for (int n = 0; n < NF; ++n) {
    const int f = GATED ? n % (NF / 2) : n;
    const int r = (f >> 1) * 32 + (rho >> 2) * 8 + (f & 1) * 4 + (rho & 3);
    vb[n] = r < cols ? r * (int)ldb + q * 16 : kOutOfRange;
  }
  const __amdgpu_buffer_rsrc_t ra = rsrc(p.a + beg * p.a_ld, (rows - 1) * p.a_ld + kbytes);
  const int va = rho < rows ? rho * (int)p.a_ld + q * 16 : kOutOfRange;
  const float* sp = FP8 ? p.a_scale + (int64_t)(beg + std::min(rho, rows - 1)) * nb : nullptr;
  u32x4 a[kDepth][2], b[kDepth][NF][2];
  float sc[kDepth];
  const auto load = [&](int d, int s) EPL_INLINE {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = std::min(s * 128 + h * 64, kbytes);  // the range check subtracts it from the descriptor's size
      const bool in = at + q * 16 < kbytes;               // false past the last step too
#pragma unroll
      for (int n = 0; n < NF; ++n)
        b[d][n][h] = __builtin_amdgcn_raw_buffer_load_b128(GATED && n >= NF / 2 ? rb2 : rb, in ? vb[n] : kOutOfRange,
                                                           at, kCachePolicyNt);
      a[d][h] = __builtin_amdgcn_raw_buffer_load_b128(ra, in ? va : kOutOfRange, at, 0);
    }
    if constexpr (FP8) sc[d] = sp[std::min(s, nb - 1)];
  };
  f32x4 acc[NF];
#pragma unroll
  for (int n = 0; n < NF; ++n) acc[n] = f32x4{0, 0, 0, 0};
#pragma unroll
  for (int d = 0; d < kDepth; ++d) load(d, wave + d * kFewWaves);
  for (int s = wave; s < steps; s += kDepth * kFewWaves) {
#pragma unroll
    for (int d = 0; d < kDepth; ++d) {
      // Steps past the last one multiply zeros.
      if constexpr (!FP8) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int n = 0; n < NF; ++n)
            acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b[d][n][h]),
                                                             __builtin_bit_cast(bf16x8, a[d][h]), acc[n], 0, 0, 0);
      } else {
        // As in run_tiles: a block's product joins the sum scaled, the instruction's own scales are one.
        const auto join = [](const u32x4(&h)[2]) EPL_INLINE {
          return __builtin_shufflevector(__builtin_bit_cast(i32x4, h[0]), __builtin_bit_cast(i32x4, h[1]), 0, 1, 2, 3,
                                         4, 5, 6, 7);
        };
#pragma unroll
        for (int n = 0; n < NF; ++n) {
          const f32x4 t = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
              join(b[d][n]), join(a[d]), f32x4{0, 0, 0, 0}, 0, 0, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[n][i] = fmaf(sc[d], t[i], acc[n][i]);
        }
      }
      load(d, s + (d + kDepth) * kFewWaves);
    }
  }
#pragma unroll
  for (int n = 0; n < NF; ++n) part[wave][n][lane] = acc[n];
  __syncthreads();
  // Column group `wave`: eight consecutive columns of row rho.
  const int c = col0 + wave * 32 + q * 8;
  if (wave < kUnits && c < p.N && rho < rows) {
    float v[8], u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = u[i] = 0.0f;
#pragma unroll
      for (int w = 0; w < kFewWaves; ++w) {
        v[i] += part[w][wave * 2 + i / 4][lane][i % 4];
        if constexpr (GATED) u[i] += part[w][NF / 2 + wave * 2 + i / 4][lane][i % 4];
      }
    }
    const int64_t cc = (int64_t)e * p.N + c, row = beg + rho;
    if constexpr (FP8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[i] *= p.w_scale[cc + i];
        if constexpr (GATED) u[i] *= p.w2_scale[cc + i];
      }
    }
    if constexpr (!GATED) {
      if (p.bias) {
        float d[8];
        unpack8(*(const u32x4*)(p.bias + cc * 2), d);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += d[i];
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
    with_activation(p.act, [&](auto act) EPL_INLINE {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[i] = activate<act>(v[i]);
        if constexpr (GATED) v[i] *= u[i];
      }
    });
    if constexpr (!GATED) {
      if (p.residual) {
        float d[8];
        unpack8(*(const u32x4*)(p.residual + row * p.res_ld + c * 2ll), d);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += d[i];
      }
    }
    *(u32x4*)(p.out + row * p.out_ld + c * 2ll) = pack8(v);
  }
}

template <int NF, bool FP8, bool GATED>
static hipError_t launch_as(const ForwardArgs& p, hipStream_t stream) {
  constexpr int kCols = 16 * NF / (GATED ? 2 : 1);
  const int64_t grid = (int64_t)((p.N + kCols - 1) / kCols) * std::min(p.E, p.cap);
  hipLaunchKernelGGL((few_rows_kernel<NF, FP8, GATED>), dim3((unsigned)grid), dim3(kFewWaves * kWave), 0,
                     stream, p);
  return hipGetLastError();
}

hipError_t launch_forward_few(const ForwardArgs& p, bool fp8, bool gated, hipStream_t stream) {
  if (gated) return fp8 ? launch_as<4, true, true>(p, stream) : launch_as<4, false, true>(p, stream);
  return fp8 ? launch_as<2, true, false>(p, stream) : launch_as<2, false, false>(p, stream);
}

}  // namespace epl
