// Matrix-instruction tile shared by the experts' products (device only).
//
// A workgroup computes a BM x BN tile of D = A * B^T with 64-wide waves in a WM x WN arrangement. Both
// operands pass through LDS in steps of 128 bytes of the reduction (64 bf16 or 128 E4M3 elements), and each may
// be stored either way round in memory:
//   * reduction-contiguous ("rows"): LDS holds [rows][128 bytes]; a lane reads 16 bytes of its row;
//   * reduction-major ("columns"):   LDS holds [64 reduction rows][columns]; a lane reads two 4x16 blocks that
//     the transposing LDS read turns to its own column (ds_read_b64_tr_b16).
// Either way a lane ends up with the same eight reduction elements of one row, so the two mix freely: forward
// (rows x rows), input gradient (rows x columns) and weight gradient (columns x columns) are one loop.
//
// Global memory goes to LDS directly (buffer loads with the lds bit, 16 bytes a lane, no registers), bounded by
// the buffer descriptor: what lies past an operand's last row or column arrives as zero. A wave's load fills 1 KiB
// of consecutive LDS, so the bank swizzle is applied to the global addresses: 16-byte piece c of row r sits in
// slot c ^ key(r).
//
// The matrix instruction gets B's fragment as its first operand, so that a lane's four results are four
// consecutive output columns of one row, and B's rows are dealt to fragments so that two neighbouring fragments
// give eight: one 16-byte bf16 store per lane.
#pragma once

#include "epl_internal.h"

namespace epl {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kStepBytes = 128;       // reduction bytes of a row per step
constexpr int kTileK = 64;            // bf16 reduction elements per step
constexpr int kOutOfRange = INT_MIN;  // as an unsigned offset, past every descriptor below 2 GiB

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// LDS byte address of a pointer into shared memory.
__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

__device__ __forceinline__ u32x4 make_rsrc(uint64_t base, int64_t bytes) {
  const int n = bytes <= 0 ? 0 : (int)std::min<int64_t>(bytes, INT_MAX);
  return u32x4{(uint32_t)uniform((int)(uint32_t)base), (uint32_t)uniform((int)(base >> 32)), (uint32_t)uniform(n),
               (uint32_t)kBufferRsrcWord3};
}

// 64 lanes x 16 bytes from the descriptor to consecutive LDS bytes at lds. Outside the compiler's view of
// outstanding loads: wait_tiles() is what waits for it. (The builtin makes the compiler wait for every such load
// before any LDS read, which would end the overlap of a step's loads with the previous step's products.)
__device__ __forceinline__ void load_to_lds(u32x4 rsrc, uint32_t lds, int voff) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "buffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(uniform((int)lds)),
      "v"(voff), "s"(rsrc)
      : "memory");
}

// All of this wave's loads have landed and its LDS reads are done; then every wave of the workgroup is here.
__device__ __forceinline__ void wait_tiles() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// One operand's stream of steps. Wave-uniform except the lane's offsets.
//   COLS: reduction-major in memory (reduction rows ld bytes apart, columns contiguous);
//   ROWS: rows (columns) of the tile; NW waves share its loads; B: the B operand's swizzle key.
// A second base serves a tile whose second half of rows comes from another matrix (gate and up projections).
template <bool COLS, int ROWS, int NW, bool B, bool SPLIT = false>
struct Operand {
  static constexpr int kLoads = ROWS * kStepBytes / 1024 / NW;  // per wave and step
  static_assert(kLoads >= 1 && kLoads * NW * 1024 == ROWS * kStepBytes, "tile not a whole number of loads");
  static constexpr int kBytes = ROWS * kStepBytes;

  uint64_t base, base2;
  int64_t bytes;
  int64_t step;
  int left;  // rows: reduction bytes left
  int voff[kLoads];
  int piece[2];  // rows: byte offset of the lane's piece, for even and odd loads

  // rows: `n` valid rows ld bytes apart, kbytes reduction bytes. columns: `n` valid columns (of 2 bytes),
  // reduction rows ld bytes apart.
  __device__ __forceinline__ void lanes(int n, int64_t ld, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int ii = wave * kLoads + i;
      if constexpr (!COLS) {
        const int r8 = lane >> 3;
        const int key = B ? (r8 & 3) | ((ii & 1) << 2) : r8;
        int row = ii * 8 + r8;
        const int pc = ((lane & 7) ^ key) * 16;
        piece[i & 1] = pc;
        if constexpr (SPLIT) row = row >= ROWS / 2 ? row - ROWS / 2 : row;
        voff[i] = row < n ? (int)(row * ld) + pc : kOutOfRange;
      } else {
        constexpr int kPer = ROWS / 8;  // 16-byte pieces per reduction row
        const int p = ii * 64 + lane;
        const int kr = p / kPer, slot = p % kPer;
        const int c = slot ^ ((kr & 3) * (B ? 4 : 2));
        voff[i] = c * 8 < n ? (int)(kr * ld) + c * 16 : kOutOfRange;
      }
    }
  }
  __device__ __forceinline__ void start_rows(const void* p, const void* p2, int n, int64_t ld, int kbytes) {
    base = (uint64_t)p;
    base2 = (uint64_t)p2;
    bytes = n <= 0 ? 0 : (n - 1) * ld + kbytes;
    step = kStepBytes;
    left = kbytes;
  }
  // k reduction rows, n columns
  __device__ __forceinline__ void start_cols(const void* p, int64_t k, int n, int64_t ld) {
    base = (uint64_t)p;
    base2 = 0;
    bytes = k <= 0 ? 0 : (k - 1) * ld + n * 2;
    step = kTileK * ld;
    left = 0;
  }
  // Issue the loads of the next step into the tile at lds and move on.
  __device__ __forceinline__ void load(uint32_t lds, int wave) {
    const u32x4 r = make_rsrc(base, bytes);
    u32x4 r2 = r;
    if constexpr (SPLIT) r2 = make_rsrc(base2, bytes);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      int v = voff[i];
      if constexpr (!COLS) v = piece[i & 1] < left ? v : kOutOfRange;
      const bool second = SPLIT && wave * kLoads + i >= ROWS / 16;
      load_to_lds(second ? r2 : r, lds + (wave * kLoads + i) * 1024, v);
    }
    base += step;
    if constexpr (SPLIT) base2 += step;
    bytes -= step;
    left -= kStepBytes;
  }
};

// Eight reduction elements (bf16) of fragment rows from LDS. `rho` = lane % 16, `q` = lane / 16.
// rows: address of the lane's row at piece q ^ (rho & 7); the second half of the step is 64 bytes away by XOR.
__device__ __forceinline__ i32x4 read_rows(uint32_t addr) {
  return *(const __attribute__((address_space(3))) i32x4*)(uintptr_t)addr;
}
__device__ __forceinline__ i32x4 read_cols(uint32_t addr, int row_bytes) {
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)addr);
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4*)(uintptr_t)(addr + 4 * row_bytes));
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  const i32x2 a = __builtin_bit_cast(i32x2, lo), b = __builtin_bit_cast(i32x2, hi);
  return i32x4{a[0], a[1], b[0], b[1]};
}

// BM x BN tile by WM x WN waves. MF x NF fragments of 16 x 16 per wave.
template <int BM_, int BN_, int WM_, int WN_>
struct Shape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
  static constexpr int kWaves = WM * WN, kThreads = kWaves * kWave;
  static constexpr int MF = BM / WM / 16, NF = BN / WN / 16;
  static constexpr int kStage = (BM + BN) * kStepBytes;
  static_assert(NF % 2 == 0, "fragments of B come in pairs");
};

// Fragment addresses of one wave inside a stage (A tile first, then B), and the products of one step.
//   SPLIT: the B tile's first half of rows are gate rows and its second half up rows; a wave takes the same
//   columns of both: fragments 0..NF/2-1 are gate, the rest up.
template <class S, bool ACOLS, bool BCOLS, bool FP8, bool SPLIT = false>
struct Products {
  uint32_t a[ACOLS ? 4 : 1];
  uint32_t b[BCOLS ? (S::NF >= 4 ? 2 : 1) : 1];
  __device__ __forceinline__ void init(int wave, int lane) {
    const int rho = lane & 15, q = lane >> 4;
    const int wm = wave / S::WN, wn = wave % S::WN;
    const int m0 = wm * S::MF * 16;
    if constexpr (!ACOLS) {
      a[0] = (m0 + rho) * kStepBytes + ((q ^ (rho & 7)) * 16);
    } else {
      const int kr = q * 8 + (rho >> 2);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        a[i] = kr * S::BM * 2 + (((m0 / 8 + i * 2 + ((rho & 3) >> 1)) ^ ((rho >> 2) * 2)) * 16) + (rho & 1) * 8;
    }
    const int n0 = wn * S::NF * 16 / (SPLIT ? 2 : 1);
    const uint32_t bt = S::BM * kStepBytes;
    if constexpr (!BCOLS) {
      b[0] = bt + (n0 + (rho >> 2) * 8 + (rho & 3)) * kStepBytes + ((q ^ (rho & 7)) * 16);
    } else {
      const int kr = q * 8 + (rho >> 2);
#pragma unroll
      for (int i = 0; i < (S::NF >= 4 ? 2 : 1); ++i)
        b[i] = bt + kr * S::BN * 2 + (((n0 / 8 + i * 4 + (rho & 3)) ^ ((rho >> 2) * 4)) * 16);
    }
  }
  __device__ __forceinline__ i32x4 a_frag(uint32_t stage, int mf, int kk) const {
    if constexpr (!ACOLS)
      return read_rows(stage + (a[0] ^ (kk * 64)) + mf * 16 * kStepBytes);
    else  // four fragments are 128 bytes; further ones repeat the pattern
      return read_cols(stage + a[mf & 3] + (mf >> 2) * 128 + kk * 32 * S::BM * 2, S::BM * 2);
  }
  __device__ __forceinline__ i32x4 b_frag(uint32_t stage, int nf, int kk) const {
    const int half = SPLIT ? nf / (S::NF / 2) : 0;
    const int f = SPLIT ? nf % (S::NF / 2) : nf;
    if constexpr (!BCOLS)
      return read_rows(stage + (b[0] ^ (kk * 64)) + ((f >> 1) * 32 + (f & 1) * 4 + half * (S::BN / 2)) * kStepBytes);
    else
      return read_cols(stage + b[(f >> 1) & 1] + (f >> 2) * 128 + (f & 1) * 8 + kk * 32 * S::BN * 2, S::BN * 2);
  }
  __device__ __forceinline__ void step(uint32_t stage, f32x4 (&acc)[S::MF][S::NF], const float* row_scale) const {
    if constexpr (!FP8) {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        i32x4 fb[S::NF];
#pragma unroll
        for (int n = 0; n < S::NF; ++n) fb[n] = b_frag(stage, n, kk);
#pragma unroll
        for (int m = 0; m < S::MF; ++m) {
          const bf16x8 fa = __builtin_bit_cast(bf16x8, a_frag(stage, m, kk));
#pragma unroll
          for (int n = 0; n < S::NF; ++n)
            acc[m][n] =
                __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fb[n]), fa, acc[m][n], 0, 0, 0);
        }
      }
    } else {
      // The step is one 128-element block of the row's scale: the block's product starts at zero and joins the
      // sum scaled, in 32 bits. The instruction's own block scales stay at one (exponent 127).
      i32x8 fb[S::NF];
#pragma unroll
      for (int n = 0; n < S::NF; ++n) {
        const i32x4 lo = b_frag(stage, n, 0), hi = b_frag(stage, n, 1);
        fb[n] = i32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      }
#pragma unroll
      for (int m = 0; m < S::MF; ++m) {
        const i32x4 lo = a_frag(stage, m, 0), hi = a_frag(stage, m, 1);
        const i32x8 fa = i32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
#pragma unroll
        for (int n = 0; n < S::NF; ++n) {
          const f32x4 p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[n], fa, f32x4{0, 0, 0, 0}, 0, 0, 0,
                                                                           0x7f7f7f7f, 0, 0x7f7f7f7f);
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[m][n][i] = fmaf(row_scale[m], p[i], acc[m][n][i]);
        }
      }
    }
  }
};

// ---------------------------------------------------------------- tiles over the experts' rows
// Rows [beg, end) of expert e in the packed buffer. The offsets are clipped to the buffer, so that whatever they
// hold, no access leaves it.
__device__ __forceinline__ void expert_rows(const int32_t* expert_off, int e, int cap, int& beg, int& end) {
  beg = std::min(std::max(expert_off[e], 0), cap);
  end = std::min(std::max(expert_off[e + 1], beg), cap);
}

// mt[e] = row tiles of the experts before e, in LDS; returns after a barrier.
template <int BM>
__device__ __forceinline__ void count_row_tiles(const int32_t* expert_off, int E, int cap, int* mt) {
  if (threadIdx.x < kWave) {
    const int lane = threadIdx.x;
    int carry = 0;
    for (int e0 = 0; e0 < E; e0 += kWave) {
      const int e = e0 + lane;
      int n = 0;
      if (e < E) {
        int beg, end;
        expert_rows(expert_off, e, cap, beg, end);
        n = (end - beg + BM - 1) / BM;
      }
      const int inc = wave_inclusive_sum(n) + carry;
      if (e < E) mt[e + 1] = inc;
      carry = __shfl(inc, kWave - 1, kWave);
    }
    if (lane == 0) mt[0] = 0;
  }
  __syncthreads();
}

// Workgroup -> slot in the current round of tiles: consecutive slots share operands, and consecutive workgroups
// go to different XCDs, so each XCD (its own L2) takes a run of gridDim / 8 slots.
__device__ __forceinline__ int xcd_slot(int wg, int grid) {
  return grid % 8 == 0 ? (wg % 8) * (grid / 8) + wg / 8 : wg;
}

// Tile j of a grid of mt x nt tiles in bands of `band` columns: a run of tiles is nearly square.
__device__ __forceinline__ void band_tile(int64_t j, int64_t mt, int nt, int band, int& m, int& n) {
  const int64_t per = mt * band;
  const int64_t bi = j / per;
  const int w = (int)std::min<int64_t>(band, nt - bi * band);
  const int64_t r = j - bi * per;
  m = (int)(r / w);
  n = (int)(bi * band + (r - (int64_t)m * w));
}

// ---------------------------------------------------------------- activations (fp32)
__device__ __forceinline__ float activate(int act, float v) {
  switch (act) {
    case EPL_ACT_SILU:
      return v / (1.0f + expf(-v));
    case EPL_ACT_GELU:
      return 0.5f * v * (1.0f + erff(v * 0.70710678118654752f));
    case EPL_ACT_RELU:
      return v < 0.0f ? 0.0f : v;
    default:
      return v;
  }
}
__device__ __forceinline__ float activate_grad(int act, float v) {
  switch (act) {
    case EPL_ACT_SILU: {
      const float s = 1.0f / (1.0f + expf(-v));
      return s * (1.0f + v * (1.0f - s));
    }
    case EPL_ACT_GELU:
      return 0.5f * (1.0f + erff(v * 0.70710678118654752f)) + v * 0.39894228040143268f * expf(-0.5f * v * v);
    case EPL_ACT_RELU:
      return v > 0.0f ? 1.0f : 0.0f;
    default:
      return 1.0f;
  }
}

}  // namespace epl
