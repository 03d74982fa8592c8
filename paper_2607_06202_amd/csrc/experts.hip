// The experts' products on the packed rows: forward, input gradient and weight gradient, one tile loop
// (gemm_tile.h) with three ways of reading the operands and the work of each call fused into its end.
#include "gemm_tile.h"
#include "experts.h"

namespace epl {

constexpr int kCus = 256;  // compute units of an MI355X

// The lane's place in a tile's results: rows row + 16 f, and eight columns from col + 32 g of each pair of column
// fragments.
template <class S, bool SPLIT = false>
struct LanePlace {
  int row, col;
  __device__ __forceinline__ LanePlace(int wave, int lane)
      : row((wave / S::WN) * S::MF * 16 + (lane & 15)),
        col((wave % S::WN) * S::NF * 16 / (SPLIT ? 2 : 1) + (lane >> 4) * 8) {}
};

// Stores of a tile's results, bounded by the descriptor: every lane issues every store, so that the number of them is
// known (run_tiles counts on it), and those past the last row or column are dropped.
struct TileOut {
  __amdgpu_buffer_rsrc_t rs;
  int ld, cols;
  __device__ __forceinline__ TileOut(char* base, int64_t row0, int64_t ld_, int col0, int rows, int cols_)
      : ld((int)ld_), cols(cols_) {
    const uint64_t at = (uint64_t)(base + row0 * ld_ + (int64_t)col0 * 2);
    const uint64_t uni = (uint64_t)(uint32_t)uniform((int)(uint32_t)at) | (uint64_t)(uint32_t)uniform((int)(at >> 32)) << 32;
    rs = __builtin_amdgcn_make_buffer_rsrc((void*)uni, 0, uniform((rows - 1) * (int)ld_ + cols_ * 2), kBufferRsrcWord3);
  }
  // Streamed: results that stayed in L2 would push out the operands (8% of a gated tile of 16 steps).
  __device__ __forceinline__ void put(int r, int c, u32x4 v) const {
    __builtin_amdgcn_raw_buffer_store_b128(v, rs, c < cols ? r * ld + c * 2 : kOutOfRange, 0, kCachePolicyNt);
  }
  __device__ __forceinline__ void store(int r, int c, const float (&v)[8]) const { put(r, c, pack8(v)); }
  // Columns c.. and c + 32.. of row r from every lane, as whole 128-byte lines: lanes rho and rho + 8 of a row of 16
  // exchange halves, so that one store takes rows 0..7 of the fragment and the other rows 8..15.
  __device__ __forceinline__ void store2(int r, int c, const float (&v0)[8], const float (&v1)[8]) const {
    const bool low = (r & 8) == 0;
    const u32x4 p0 = pack8(v0), p1 = pack8(v1);
    u32x4 mine, other;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      mine[i] = low ? p0[i] : p1[i];
      other[i] = (uint32_t)__builtin_amdgcn_mov_dpp((int)(low ? p1[i] : p0[i]), 0x128, 0xf, 0xf, false);  // row_ror:8
    }
    const int cc = low ? c : c + 32;
    put(r & ~8, cc, low ? mine : other);
    put(r | 8, cc, low ? other : mine);
  }
};

template <class S>
__device__ __forceinline__ void store_tile(const TileOut& out, int row, int col, f32x4 (&acc)[S::MF][S::NF]) {
#pragma unroll
  for (int g = 0; g < S::NF / 4; ++g)
#pragma unroll
    for (int f = 0; f < S::MF; ++f) {
      float v[2][8];
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i / 8][i % 8] = acc[f][g * 4 + i / 4][i % 4];
      out.store2(row + f * 16, col + g * 64, v[0], v[1]);
    }
}

// ---------------------------------------------------------------- forward
// GATED: B tile = BN/2 gate rows and BN/2 up rows; BN/2 output columns.
template <class S, bool FP8, bool GATED>
struct ForwardJob {
  static constexpr int kCols = GATED ? S::BN / 2 : S::BN;  // output columns of a tile
  static constexpr int kPairs = kCols / S::WN / 32;        // pairs of column fragments of a wave
  static constexpr int kEsize = FP8 ? 1 : 2;
  struct Tile {
    int64_t t;
    RowTile at;
    int e, row0, rows, col0, steps;
  };
  const ForwardArgs& p;
  int wave, lane, nt, steps;
  LanePlace<S, GATED> at;
  __device__ __forceinline__ ForwardJob(const ForwardArgs& p_, int wave_, int lane_)
      : p(p_), wave(wave_), lane(lane_), at(wave_, lane_) {
    nt = (p.N + kCols - 1) / kCols;
    steps = S::steps(p.K * kEsize, FP8);
  }
  __device__ __forceinline__ bool place(Tile& t) const {
    if (!t.at.template find<S::BM>(p.expert_off, p.E, p.cap, t.t / nt, lane)) return false;
    int m, n;
    t.e = t.at.e;
    band_tile(t.t - t.at.before * nt, t.at.count, nt, 8, m, n);
    t.row0 = t.at.beg + m * S::BM;
    t.rows = std::min(t.at.end - t.row0, S::BM);
    t.col0 = n * kCols;
    t.steps = steps;
    return true;
  }
  __device__ __forceinline__ bool first(Tile& t) const {
    t = Tile{};
    t.t = xcd_slot(blockIdx.x, gridDim.x);
    return place(t);
  }
  __device__ __forceinline__ bool next(Tile& t) const {
    t.t += gridDim.x;
    return place(t);
  }
  template <class A, class B>
  __device__ __forceinline__ void begin(const Tile& t, A& a, B& b) const {
    const int64_t ldb = (int64_t)p.K * kEsize;
    const int64_t boff = t.e * p.expert_stride * kEsize + t.col0 * ldb;
    const int cols = std::min(p.N - t.col0, kCols);
    a.lanes(t.rows, p.a_ld, wave, lane);
    b.lanes(cols, ldb, wave, lane);
    a.start_rows(p.a + t.row0 * p.a_ld, nullptr, t.rows, p.a_ld, p.K * kEsize);
    b.start_rows(p.w + boff, p.w2 + boff, cols, ldb, p.K * kEsize);
  }
  template <class A, class B>
  __device__ __forceinline__ void turn(const Tile&, int, A&, B&) const {}
  // One scale per lane for 64 rows; a tile has at most 256, and waves beyond its rows load some again.
  __device__ __forceinline__ void load_scales(const Tile& t, int step, uint32_t lds) const {
    constexpr int kSpans = S::BM / kWave;
    const int span = wave % kSpans * kWave, nb = p.K / 128;
    const int64_t bytes = step < nb ? ((int64_t)(t.rows - 1) * nb + 1) * 4 : 0;
    const u32x4 rs = make_rsrc((uint64_t)(p.a_scale + (int64_t)t.row0 * nb + step), bytes);
    load_words_to_lds(rs, lds + span * 4, (span + lane) * nb * 4);
  }
  template <int N>
  __device__ __forceinline__ void wait(bool stored) const {
    constexpr int kEach = kPairs * S::MF;
    if (!stored)
      wait_tiles<N>();
    else if (!p.pre)
      wait_tiles<std::min(63, N + kEach)>();
    else
      wait_tiles<std::min(63, N + kEach * (GATED ? 3 : 2))>();
  }
  __device__ __forceinline__ void finish(const Tile& t, f32x4 (&acc)[S::MF][S::NF]) const {
    const int cols = std::min(p.N - t.col0, kCols);
    const TileOut out(p.out, t.row0, p.out_ld, t.col0, t.rows, cols);
    const int64_t pre_ld = (int64_t)p.N * (GATED ? 4 : 2);
    const TileOut pre(p.pre, t.row0, pre_ld, t.col0, t.rows, cols);
    const TileOut pre2(p.pre, t.row0, pre_ld, t.col0 + p.N, t.rows, cols);
    constexpr int kTake = kPairs % 2 ? 1 : 2;  // groups of 32 columns stored together
#pragma unroll
    for (int g0 = 0; g0 < kPairs; g0 += kTake) {
      const int c0 = at.col + g0 * 32;
      float s1[kTake][8], s2[kTake][8], bias[kTake][8];
#pragma unroll
      for (int k = 0; k < kTake; ++k) {
        // In range for the lanes past the last column.
        const int64_t cc = (int64_t)t.e * p.N + t.col0 + std::min(c0 + k * 32, cols - 8);
        if constexpr (FP8) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            s1[k][i] = p.w_scale[cc + i];
            if constexpr (GATED) s2[k][i] = p.w2_scale[cc + i];
          }
        }
        if constexpr (!GATED) {
          if (p.bias) unpack8(*(const u32x4*)(p.bias + cc * 2), bias[k]);
        }
      }
#pragma unroll
      for (int f = 0; f < S::MF; ++f) {
        const int r = at.row + f * 16;
        float v[kTake][8], u[kTake][8];
#pragma unroll
        for (int j = 0; j < kTake * 8; ++j) {
          const int k = j / 8, i = j % 8, at_n = (g0 + k) * 2 + i / 4;
          v[k][i] = acc[f][at_n][i % 4];
          if constexpr (FP8) v[k][i] *= s1[k][i];
          if constexpr (GATED) {
            u[k][i] = acc[f][S::NF / 2 + at_n][i % 4];
            if constexpr (FP8) u[k][i] *= s2[k][i];
          } else if (p.bias) {
            v[k][i] += bias[k][i];
          }
        }
        if (p.pre) {
          store<kTake>(pre, r, c0, v);
          if constexpr (GATED) store<kTake>(pre2, r, c0, u);
        }
        with_activation(p.act, [&](auto act) EPL_INLINE {
#pragma unroll
          for (int j = 0; j < kTake * 8; ++j) {
            v[j / 8][j % 8] = activate<act>(v[j / 8][j % 8]);
            if constexpr (GATED) v[j / 8][j % 8] *= u[j / 8][j % 8];
          }
        });
        if constexpr (!GATED) {
          if (p.residual) {
            const char* res = p.residual + (t.row0 + std::min(r, t.rows - 1)) * p.res_ld;
#pragma unroll
            for (int k = 0; k < kTake; ++k) {
              float d[8];
              unpack8(*(const u32x4*)(res + (t.col0 + std::min(c0 + k * 32, cols - 8)) * 2ll), d);
#pragma unroll
              for (int i = 0; i < 8; ++i) v[k][i] += d[i];
            }
          }
        }
        store<kTake>(out, r, c0, v);
      }
    }
  }
  template <int TAKE>
  static __device__ __forceinline__ void store(const TileOut& o, int r, int c, const float (&v)[TAKE][8]) {
    if constexpr (TAKE == 2)
      o.store2(r, c, v[0], v[1]);
    else
      o.store(r, c, v[0]);
  }
};

template <class S, bool FP8, bool GATED>
__global__ void __launch_bounds__(S::kThreads) forward_kernel(ForwardArgs p) {
  __shared__ __attribute__((aligned(1024))) char tiles[S::lds(FP8)];
  const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  ForwardJob<S, FP8, GATED> job(p, wave, lane);
  run_tiles<S, false, false, FP8, GATED>(job, lds_addr(tiles), wave, lane);
}

// ---------------------------------------------------------------- gradient of the rows
// dx[r] = sum over parts and n of d[r][part * N + n] w_part[e][n]: the reduction runs over the weights' rows.
template <class S>
struct RowGradJob {
  static_assert(!S::RING, "turn() sets both operands up for one step");
  struct Tile {
    int64_t t;
    RowTile at;
    int e, row0, rows, col0, steps;
  };
  const RowGradArgs& p;
  int wave, lane, nt, part_steps;
  LanePlace<S> at;
  __device__ __forceinline__ RowGradJob(const RowGradArgs& p_, int wave_, int lane_)
      : p(p_), wave(wave_), lane(lane_), at(wave_, lane_) {
    nt = (p.K + S::BN - 1) / S::BN;
    part_steps = (p.N * 2 + kStepBytes - 1) / kStepBytes;
  }
  __device__ __forceinline__ bool place(Tile& t) const {
    if (!t.at.template find<S::BM>(p.expert_off, p.E, p.cap, t.t / nt, lane)) return false;
    int m, n;
    t.e = t.at.e;
    band_tile(t.t - t.at.before * nt, t.at.count, nt, 8, m, n);
    t.row0 = t.at.beg + m * S::BM;
    t.rows = std::min(t.at.end - t.row0, S::BM);
    t.col0 = n * S::BN;
    t.steps = S::steps((int64_t)part_steps * p.parts * kStepBytes, false);
    return true;
  }
  __device__ __forceinline__ bool first(Tile& t) const {
    t = Tile{};
    t.t = xcd_slot(blockIdx.x, gridDim.x);
    return place(t);
  }
  __device__ __forceinline__ bool next(Tile& t) const {
    t.t += gridDim.x;
    return place(t);
  }
  template <class A, class B>
  __device__ __forceinline__ void begin(const Tile& t, A& a, B& b) const {
    a.lanes(t.rows, p.d_ld, wave, lane);
    b.lanes(std::min(p.K - t.col0, S::BN), (int64_t)p.K * 2, wave, lane);
    start(t, 0, p.w, a, b);
  }
  template <class A, class B>
  __device__ __forceinline__ void start(const Tile& t, int part, const char* w, A& a, B& b) const {
    const int64_t ldb = (int64_t)p.K * 2;
    a.start_rows(p.d + t.row0 * p.d_ld + (int64_t)part * p.N * 2, nullptr, t.rows, p.d_ld, p.N * 2);
    b.start_cols(w + (t.e * p.expert_stride + t.col0) * 2, p.N, std::min(p.K - t.col0, S::BN), ldb);
  }
  // The second part's first step. (An only part's padded step may have that number too.)
  template <class A, class B>
  __device__ __forceinline__ void turn(const Tile& t, int step, A& a, B& b) const {
    if (p.parts == 2 && step == part_steps) start(t, 1, p.w2, a, b);
  }
  template <int N>
  __device__ __forceinline__ void wait(bool stored) const {
    if (stored)
      wait_tiles<std::min(63, N + S::NF / 2 * S::MF)>();
    else
      wait_tiles<N>();
  }
  __device__ __forceinline__ void finish(const Tile& t, f32x4 (&acc)[S::MF][S::NF]) const {
    const TileOut out(p.dx, t.row0, p.dx_ld, t.col0, t.rows, std::min(p.K - t.col0, S::BN));
    store_tile<S>(out, at.row, at.col, acc);
  }
};

template <class S>
__global__ void __launch_bounds__(S::kThreads) row_grad_kernel(RowGradArgs p) {
  __shared__ __attribute__((aligned(1024))) char tiles[S::lds(false)];
  const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  RowGradJob<S> job(p, wave, lane);
  run_tiles<S, false, true, false, false>(job, lds_addr(tiles), wave, lane);
}

// ---------------------------------------------------------------- gradient of the weights
// dw_part[e][n][k] = sum over the expert's rows r of d[r][part * N + n] x[r][k]: the reduction runs over the rows. An
// expert without rows takes one step of zeros.
template <class S>
struct WeightGradJob {
  struct Tile {
    int64_t t;
    int e, part, m0, col0, beg, rows, steps;
  };
  const WeightGradArgs& p;
  int wave, lane, mt, nt;
  LanePlace<S> at;
  __device__ __forceinline__ WeightGradJob(const WeightGradArgs& p_, int wave_, int lane_)
      : p(p_), wave(wave_), lane(lane_), at(wave_, lane_) {
    mt = (p.N + S::BM - 1) / S::BM;
    nt = (p.K + S::BN - 1) / S::BN;
  }
  __device__ __forceinline__ bool place(Tile& t) const {
    const int64_t per = (int64_t)mt * p.parts * nt;
    if (t.t >= per * p.E) return false;
    int m, n;
    t.e = (int)(t.t / per);
    const int beg = std::min(std::max(p.expert_off[t.e], 0), p.cap);
    t.beg = uniform(beg);
    t.rows = uniform(std::min(std::max(p.expert_off[t.e + 1], beg), p.cap)) - t.beg;
    band_tile(t.t - t.e * per, mt * p.parts, nt, 8, m, n);
    t.part = m >= mt;
    t.m0 = (t.part ? m - mt : m) * S::BM;
    t.col0 = n * S::BN;
    t.steps = S::steps(t.rows * 2ll, false);
    return true;
  }
  __device__ __forceinline__ bool first(Tile& t) const {
    t = Tile{};
    t.t = xcd_slot(blockIdx.x, gridDim.x);
    return place(t);
  }
  __device__ __forceinline__ bool next(Tile& t) const {
    t.t += gridDim.x;
    return place(t);
  }
  template <class A, class B>
  __device__ __forceinline__ void turn(const Tile&, int, A&, B&) const {}
  template <class A, class B>
  __device__ __forceinline__ void begin(const Tile& t, A& a, B& b) const {
    const int m = std::min(p.N - t.m0, S::BM), cols = std::min(p.K - t.col0, S::BN);
    a.lanes(m, p.d_ld, wave, lane);
    b.lanes(cols, p.x_ld, wave, lane);
    a.start_cols(p.d + t.beg * p.d_ld + ((int64_t)t.part * p.N + t.m0) * 2, t.rows, m, p.d_ld);
    b.start_cols(p.x + t.beg * p.x_ld + t.col0 * 2ll, t.rows, cols, p.x_ld);
  }
  template <int N>
  __device__ __forceinline__ void wait(bool stored) const {
    if (stored)
      wait_tiles<std::min(63, N + S::NF / 2 * S::MF)>();
    else
      wait_tiles<N>();
  }
  __device__ __forceinline__ void finish(const Tile& t, f32x4 (&acc)[S::MF][S::NF]) const {
    char* dw = (t.part ? p.dw2 : p.dw) + (int64_t)t.e * p.N * p.K * 2;
    const TileOut out(dw, t.m0, (int64_t)p.K * 2, t.col0, std::min(p.N - t.m0, S::BM), std::min(p.K - t.col0, S::BN));
    store_tile<S>(out, at.row, at.col, acc);
  }
};

template <class S>
__global__ void __launch_bounds__(S::kThreads) weight_grad_kernel(WeightGradArgs p) {
  __shared__ __attribute__((aligned(1024))) char tiles[S::lds(false)];
  const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  WeightGradJob<S> job(p, wave, lane);
  run_tiles<S, true, true, false, false>(job, lds_addr(tiles), wave, lane);
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
    with_activation(act, [&](auto act_) EPL_INLINE {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float a = activate<act_>(g[j]), ag = activate_grad<act_>(g[j]);
        g[j] = d[j] * u[j] * ag;
        u[j] = d[j] * a;
      }
    });
    ((u32x4*)dpre)[r * 2 * nv + c] = pack8(g);
    ((u32x4*)dpre)[r * 2 * nv + nv + c] = pack8(u);
  }
}

// Linear: dpre = dy act'(pre) in bf16; dy rows dy_ld bytes apart.
__global__ void __launch_bounds__(256) pre_grad_kernel(const char* dy, int64_t dy_ld, const char* pre, char* dpre,
                                                       const int32_t* expert_off, int E, int cap, int N, int act) {
  const int64_t nv = N / 8;
  const int64_t n = std::min(std::max(expert_off[E], 0), cap) * nv;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / nv;
    float d[8], v[8];
    unpack8(*(const u32x4*)(dy + r * dy_ld + (i - r * nv) * 16), d);
    unpack8(((const u32x4*)pre)[i], v);
    with_activation(act, [&](auto act_) EPL_INLINE {
#pragma unroll
      for (int j = 0; j < 8; ++j) d[j] *= activate_grad<act_>(v[j]);
    });
    ((u32x4*)dpre)[i] = pack8(d);
  }
}

// The same with dbias[e][n] = the sum of the unrounded dpre over the expert's rows, in one pass over dy and pre (without
// an activation there is no dpre to write). A workgroup takes 64 columns of one expert: 8 lanes of 8 columns, 32 row
// lanes that take every 32nd row, two at a time; fp32 sums, added over the row lanes in order.
__global__ void __launch_bounds__(256) pre_bias_grad_kernel(const char* dy, int64_t dy_ld, const char* pre, char* dpre,
                                                            char* dbias, const int32_t* expert_off, int cap, int N,
                                                            int act) {
  constexpr int kLanes = 32;
  __shared__ float part[kLanes][8][8 + 1];
  const int cv = threadIdx.x % 8, rl = threadIdx.x / 8;
  const int e = blockIdx.y, c = blockIdx.x * 64 + cv * 8;
  const int beg = std::min(std::max(expert_off[e], 0), cap);
  const int end = std::min(std::max(expert_off[e + 1], beg), cap);
  float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (c < N) {
    for (int64_t r0 = beg + rl; r0 < end; r0 += 2 * kLanes) {
      u32x4 dw[2], vw[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int64_t r = std::min<int64_t>(r0 + k * kLanes, end - 1);
        dw[k] = *(const u32x4*)(dy + r * dy_ld + c * 2);
        if (act != EPL_ACT_NONE) vw[k] = *(const u32x4*)(pre + (r * N + c) * 2);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int64_t r = r0 + k * kLanes;
        if (r >= end) continue;
        float d[8], v[8];
        unpack8(dw[k], d);
        if (act != EPL_ACT_NONE) {
          unpack8(vw[k], v);
          with_activation(act, [&](auto act_) EPL_INLINE {
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] *= activate_grad<act_>(v[j]);
          });
          *(u32x4*)(dpre + (r * N + c) * 2) = pack8(d);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] += d[j];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) part[rl][cv][j] = s[j];
  __syncthreads();
  if (rl == 0 && c < N) {
    for (int k = 1; k < kLanes; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] += part[k][cv][j];
    *(u32x4*)(dbias + ((int64_t)e * N + c) * 2) = pack8(s);
  }
}

// ---------------------------------------------------------------- launches
using Big = Shape<256, 256, 2, 4, 2, true>;
using Mid = Shape<128, 256, 2, 4, 3>;
using Short = Shape<64, 256, 1, 4, 3>;

static unsigned persistent_grid(int64_t tiles, int per_cu) {
  return (unsigned)std::min<int64_t>(tiles, (int64_t)kCus * per_cu);
}

// Row tiles of BM over at most `rows` rows of E experts.
static int64_t row_tiles(int64_t rows, int E, int BM) { return rows / BM + std::min<int64_t>(E, rows); }

template <class S, bool FP8, bool GATED>
static hipError_t forward_as(const ForwardArgs& p, hipStream_t stream) {
  const int cols = GATED ? S::BN / 2 : S::BN;
  const int64_t tiles = row_tiles(p.cap, p.E, S::BM) * ((p.N + cols - 1) / cols);
  hipLaunchKernelGGL((forward_kernel<S, FP8, GATED>), dim3(persistent_grid(tiles, 1)), dim3(S::kThreads), 0, stream,
                     p);
  return hipGetLastError();
}

hipError_t launch_forward(const ForwardArgs& p, bool fp8, bool gated, hipStream_t stream) {
  if (p.cap == 0) return hipSuccess;
  if (few_rows(p.cap)) return launch_forward_few(p, fp8, gated, stream);
  if (fp8 && short_rows(p.cap, p.E))
    return gated ? forward_as<Short, true, true>(p, stream) : forward_as<Short, true, false>(p, stream);
  if (fp8) return gated ? forward_as<Mid, true, true>(p, stream) : forward_as<Mid, true, false>(p, stream);
  if (many_rows(p.cap, p.E))
    return gated ? forward_as<Big, false, true>(p, stream) : forward_as<Big, false, false>(p, stream);
  return gated ? forward_as<Mid, false, true>(p, stream) : forward_as<Mid, false, false>(p, stream);
}

hipError_t launch_row_grad(const RowGradArgs& p, hipStream_t stream) {
  if (p.cap == 0) return hipSuccess;
  using S = Mid;
  const int64_t tiles = row_tiles(p.cap, p.E, S::BM) * ((p.K + S::BN - 1) / S::BN);
  hipLaunchKernelGGL((row_grad_kernel<S>), dim3(persistent_grid(tiles, 1)), dim3(S::kThreads), 0, stream, p);
  return hipGetLastError();
}

hipError_t launch_weight_grad(const WeightGradArgs& p, hipStream_t stream) {
  using S = Mid;
  const int64_t tiles =
      (int64_t)p.E * p.parts * ((p.N + S::BM - 1) / S::BM) * ((p.K + S::BN - 1) / S::BN);
  hipLaunchKernelGGL((weight_grad_kernel<S>), dim3(persistent_grid(tiles, 1)), dim3(S::kThreads), 0, stream, p);
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

hipError_t launch_pre_grad(const void* dy, int64_t dy_ld, const void* pre, void* dpre, void* dbias,
                           const int32_t* expert_off, int E, int cap, int N, int act, hipStream_t stream) {
  if (dbias)
    hipLaunchKernelGGL(pre_bias_grad_kernel, dim3((unsigned)((N + 63) / 64), E), dim3(256), 0, stream, (const char*)dy,
                       dy_ld, (const char*)pre, (char*)dpre, (char*)dbias, expert_off, cap, N, act);
  else if (act != EPL_ACT_NONE && cap > 0)
    hipLaunchKernelGGL(pre_grad_kernel, dim3(elementwise_grid((int64_t)cap * (N / 8))), dim3(256), 0, stream,
                       (const char*)dy, dy_ld, (const char*)pre, (char*)dpre, expert_off, E, cap, N, act);
  return hipGetLastError();
}

}  // namespace epl
