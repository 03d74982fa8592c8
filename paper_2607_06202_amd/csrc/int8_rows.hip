// Rows of bf16 to int8 with one scale a row: in dispatch (into the packed receive rows) and of rows where they are.
//
//   A = max|x|,  s = A / 127,  q = the integer nearest to 127 x / A, halves to even.
//
// The nearest integer is decided on the exact quotient, at the price of a multiplication. x and A have 8-bit mantissas, so
// a quotient that is no half (n + 1/2) is at least 1.5e-5 of itself away from one: 254 X 2^a - (2 n + 1) A' 2^b is a whole
// multiple of the smaller power of two, over 2 A'. x * (127 / A) in fp32 is off by 2^-23 of itself at most; rounded to
// 20 bits (another 2^-20 = 9.5e-7 at most) a half comes out as that half and nothing else does. Adding 1.5 * 2^23 then
// rounds to the nearest even integer and leaves it in the low byte. 127 / A is finite for every bf16 A but those below
// 2^-121; x and A are taken times 2^100 where A is below 2^-100.
//
// HBM traffic bounds both. A row is read once: it stays in registers between the maximum and the conversion, of a wave (or,
// where it stays in place, of a part of one) up to 2048 elements, so that no workgroup waits, and of a workgroup beyond.
//   * Rows where they are, 65536 of 2048: a workgroup of 256 for each row 192 us, of a wave for each 71, with streaming loads
//     and stores 68 (5.9 TB/s).
//   * Dispatch, 8192 tokens of 7168 to 8 rows each: 118 us (5.0 TB/s), as the E4M3 dispatch of the same tokens (120), and
//     within 3% whatever the threads a row (64 to 448), the waves held at once and the stores' policy: what the scattered
//     writes of 7 KiB rows take.
#include <type_traits>

#include "experts.h"
#include "rows_body.h"

namespace epl {

constexpr int kInt8Threads = 256;
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// A row of n pieces of 16 elements in the registers of `group` threads, UNITS pieces each; longer rows in passes.
// STREAM: streaming loads, for rows that are read this once (past 32768 elements twice).
template <int UNITS, bool STREAM>
struct Int8Row {
  u32x4 v[UNITS][2];
  const u32x4* row;
  int n, t, group;
  // Pieces past the last one are the last one again.
  __device__ __forceinline__ void load(int first) {
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int u = std::min(first + i * group + t, n - 1);
#pragma unroll
      for (int h = 0; h < 2; ++h) v[i][h] = STREAM ? __builtin_nontemporal_load(row + 2 * u + h) : row[2 * u + h];
    }
  }
  // The larger of m and the magnitudes' bits, by halves.
  __device__ __forceinline__ u16x2 top(u16x2 m) const {
#pragma unroll
    for (int i = 0; i < UNITS; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, v[i][j / 4][j % 4] & 0x7FFF7FFFu));
    return m;
  }
};

// What a row's largest magnitude (bf16 bits) makes of it.
struct Int8Scale {
  float s, pre, mul;  // the row's scale; x * pre * mul is the quotient
  bool zero;          // q is 0 whatever x is
  __device__ __forceinline__ explicit Int8Scale(uint32_t bits) {
    const float a = __uint_as_float(bits << 16);
    zero = bits == 0 || bits >= 0x7F80u;
    s = bits >= 0x7F80u ? __uint_as_float(0x7FC00000u) : a / 127.0f;
    pre = a < 0x1p-100f ? 0x1p100f : 1.0f;
    mul = 127.0f / (a * pre);
  }
  // The low byte is q.
  __device__ __forceinline__ uint32_t one(float x) const {
    const uint32_t t = __float_as_uint(x * pre * mul);
    return __float_as_uint(__uint_as_float((t + 8u) & ~15u) + 12582912.0f);
  }
  __device__ __forceinline__ uint32_t four(uint32_t lo, uint32_t hi) const {
    const uint32_t a = one(bf16lo_to_f32(lo)), b = one(bf16hi_to_f32(lo)), c = one(bf16lo_to_f32(hi)), d = one(bf16hi_to_f32(hi));
    return __builtin_amdgcn_perm(b, a, 0x0C0C0400u) | __builtin_amdgcn_perm(d, c, 0x04000C0Cu);
  }
  __device__ __forceinline__ u32x4 sixteen(const u32x4 (&v)[2]) const {
    if (zero) return u32x4{0, 0, 0, 0};
    return u32x4{four(v[0][0], v[0][1]), four(v[0][2], v[0][3]), four(v[1][0], v[1][1]), four(v[1][2], v[1][3])};
  }
};

// The largest over a row's threads: GROUP of a wave, or (0) the workgroup, every thread of which is here.
template <int GROUP>
__device__ __forceinline__ uint32_t group_max(u16x2 m) {
  uint32_t v = std::max<uint32_t>(m[0], m[1]);
#pragma unroll
  for (int off = (GROUP ? GROUP : kWave) / 2; off > 0; off >>= 1) v = std::max(v, (uint32_t)__shfl_xor((int)v, off, kWave));
  if constexpr (GROUP == 0) {
    __shared__ uint32_t part[kInt8Threads / kWave];
    __syncthreads();  // the last row's have been read
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
    __syncthreads();
    for (int i = 0; i < (int)blockDim.x / kWave; ++i) v = std::max(v, part[i]);
  }
  return GROUP == 0 || GROUP == kWave ? (uint32_t)__builtin_amdgcn_readfirstlane((int)v) : v;
}

// One row: put(piece, its 16 values) of every piece and put_scale(s) once.
template <int GROUP, int UNITS, bool STREAM, class Put, class PutScale>
__device__ __forceinline__ void quantise_row(const u32x4* row, int n, int t, Put&& put, PutScale&& put_scale) {
  const int group = GROUP ? GROUP : (int)blockDim.x, pass = group * UNITS;
  Int8Row<UNITS, STREAM> r;
  r.row = row;
  r.n = n;
  r.t = t;
  r.group = group;
  u16x2 m = {0, 0};
  for (int first = 0; first < n; first += pass) {
    r.load(first);
    m = r.top(m);
  }
  const Int8Scale scale(group_max<GROUP>(m));
  put_scale(scale.s);
  for (int first = 0; first < n; first += pass) {
    if (n > pass) r.load(first);
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      const int u = first + i * group + t;
      if (u < n) put(u, scale.sixteen(r.v[i]));
    }
  }
}

// Row `which` of those of a workgroup, thread t of the row's.
template <int GROUP>
struct Place {
  static constexpr int kPer = GROUP ? kInt8Threads / GROUP : 1;
  int which = GROUP ? threadIdx.x / (GROUP ? GROUP : 1) : 0, t = GROUP ? threadIdx.x % (GROUP ? GROUP : 1) : threadIdx.x;
};

template <int GROUP, int UNITS>
__global__ void __launch_bounds__(kInt8Threads)
    quantize_rows_kernel(const u32x4* a, u32x4* q, float* scale, const int32_t* count, int64_t rows, int n, int64_t a_ld,
                         int64_t q_ld) {
  const Place<GROUP> at{};
  if (count) rows = std::min<int64_t>(std::max(*count, 0), rows);
  for (int64_t r = (int64_t)blockIdx.x * at.kPer + at.which; r < rows; r += (int64_t)gridDim.x * at.kPer)
    quantise_row<GROUP, UNITS, true>(
        a + r * a_ld, n, at.t, [&](int u, u32x4 v) EPL_INLINE { __builtin_nontemporal_store(v, q + r * q_ld + u); },
        [&](float s) EPL_INLINE {
          if (at.t == 0) scale[r] = s;
        });
}

template <int GROUP, int UNITS>
__global__ void __launch_bounds__(kInt8Threads)
    dispatch_int8_kernel(const u32x4* x, const float* w, const int32_t* pair_row, u32x4* recv, float* scale, int64_t T,
                         int k, int n, int64_t ld, int64_t cap) {
  static_assert(GROUP == 0 || GROUP == kWave, "a token's packed rows are a wave's");
  const Place<GROUP> at{};
  const int lane = threadIdx.x % kWave;
  for (int64_t g = (int64_t)blockIdx.x * at.kPer + at.which; g < T; g += (int64_t)gridDim.x * at.kPer) {
    int mine = lane < k ? pair_row[g * k + lane] : -1;
    if (mine >= cap) mine = -1;
    quantise_row<GROUP, UNITS, false>(
        x + g * 2 * n, n, at.t,
        [&](int u, u32x4 v) EPL_INLINE {
          for (int j = 0; j < k; ++j) {
            const int row = __builtin_amdgcn_readlane(mine, j);
            if (row >= 0) store_row_policy<kCachePolicySc1Nt>(v, recv + row * ld, n, u);
          }
        },
        [&](float s) EPL_INLINE {
          if (at.t < kWave && mine >= 0) scale[mine] = w ? s * w[g * k + lane] : s;
        });
  }
}

// f(threads of a wave to a row or 0: the workgroup, pieces a thread, threads a workgroup) for rows of n pieces. A workgroup to
// a row has as many threads as the row needs (65536 rows of 2064 82 us, with 256 threads 93; 16384 of 8208 80 / 91).
template <class F>
static void with_shape(int n, F&& f) {
  using std::integral_constant;
  using Whole = integral_constant<int, 0>;
  using Wave = integral_constant<int, kWave>;
  const auto threads = [&](int units) { return std::min(((n + units - 1) / units + kWave - 1) / kWave * kWave, kInt8Threads); };
  if (n > 4 * kInt8Threads)
    f(Whole{}, integral_constant<int, 8>{}, threads(8));
  else if (n > 2 * kInt8Threads)
    f(Whole{}, integral_constant<int, 4>{}, threads(4));
  else if (n > kInt8Threads)
    f(Whole{}, integral_constant<int, 2>{}, threads(2));
  else if (n > 2 * kWave)
    f(Whole{}, integral_constant<int, 1>{}, threads(1));
  else if (n > kWave)
    f(Wave{}, integral_constant<int, 2>{}, kInt8Threads);
  else
    f(Wave{}, integral_constant<int, 1>{}, kInt8Threads);
}

hipError_t launch_quantize_rows(const void* a, void* q, float* scale, const int32_t* count, int64_t rows, int K,
                                int64_t a_ld, int64_t q_ld, hipStream_t stream) {
  if (rows == 0) return hipSuccess;
  const int n = K / 16;
  const auto launch = [&](auto group, auto units, int threads) {
    const dim3 grid(unit_grid(rows, Place<group>::kPer, threads));
    hipLaunchKernelGGL((quantize_rows_kernel<group, units>), grid, dim3(threads), 0, stream,
                       static_cast<const u32x4*>(a), static_cast<u32x4*>(q), scale, count, rows, n, a_ld, q_ld);
  };
  // 65536 rows of 128 / 256 / 512 with a wave to each: 24.5 / 25.8 / 27.0 us, with a part of one 9.5 / 12.6 / 20.8.
  if (n <= 16)
    launch(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{}, kInt8Threads);
  else if (n <= 32)
    launch(std::integral_constant<int, 32>{}, std::integral_constant<int, 1>{}, kInt8Threads);
  else
    with_shape(n, launch);
  return hipGetLastError();
}

hipError_t launch_dispatch_int8(const void* x, const float* w, const int32_t* pair_row, void* recv, float* scale, int64_t T,
                                int k, int H, int pitch, int64_t cap, hipStream_t stream) {
  if (T == 0) return hipSuccess;
  with_shape(H / 16, [&](auto group, auto units, int threads) {
    const dim3 grid(unit_grid(T, Place<group>::kPer, threads));
    hipLaunchKernelGGL((dispatch_int8_kernel<group, units>), grid, dim3(threads), 0, stream,
                       static_cast<const u32x4*>(x), w, pair_row, static_cast<u32x4*>(recv), scale, T, k, H / 16,
                       (int64_t)pitch / 16, cap);
  });
  return hipGetLastError();
}

}  // namespace epl
