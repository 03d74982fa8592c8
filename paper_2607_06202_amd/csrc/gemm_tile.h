// Matrix-instruction tile shared by the experts' products (device only).
//
// A workgroup computes a BM x BN tile of D = A * B^T with 64-wide waves in a WM x WN arrangement. Both
// operands pass through LDS in steps of 128 bytes of the reduction (64 bf16 or 128 E4M3 or int8 elements), and each may be
// stored either way round in memory:
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

#include <type_traits>

#include "epl_internal.h"
#include "experts.h"

namespace epl {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// A lane's four sums.
template <Elem T>
using AccOf = std::conditional_t<T == Elem::kInt8, i32x4, f32x4>;

constexpr int kStepBytes = 128;       // reduction bytes of a row per step: 64 bf16 or 128 E4M3 or int8 elements
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
// outstanding loads: wait_tiles is what waits for it. (The builtin makes the compiler wait for every such load
// before any LDS read, which would end the overlap of a step's loads with the previous step's products.)
// The compiler does not see that a memory instruction is in here either, so its distance from the vector instructions
// that may have just written the descriptor is kept here: five wait states, one of s_mov and four of s_nop.
__device__ __forceinline__ void load_to_lds(u32x4 rsrc, uint32_t lds, int voff) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 3\n\t"
      "buffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(uniform((int)lds)),
      "v"(voff), "s"(rsrc)
      : "memory", "m0");
}

// 64 lanes x 4 bytes, the same way.
__device__ __forceinline__ void load_words_to_lds(u32x4 rsrc, uint32_t lds, int voff) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 3\n\t"
      "buffer_load_dword %1, %2, 0 offen lds" ::"s"(uniform((int)lds)),
      "v"(voff), "s"(rsrc)
      : "memory", "m0");
}

// One operand's stream of steps. Wave-uniform except the lane's offsets.
//   COLS: reduction-major in memory (reduction rows ld bytes apart, columns contiguous);
//   ROWS: rows (columns) of the tile; NW waves share its loads; B: the B operand's swizzle key.
// A second base serves a tile whose second half of rows comes from another matrix (gate and up projections).
template <bool COLS, int ROWS, int NW, bool B, bool SPLIT = false>
struct Operand {
  static constexpr int kBytes = ROWS * kStepBytes;
  static constexpr int kLoads = kBytes / 1024 / NW;  // per wave and step
  static_assert(kLoads >= 1 && kLoads * NW * 1024 == kBytes, "tile not a whole number of loads");
  static constexpr int kRowsPerLoad = 1024 / kStepBytes, kSlots = kStepBytes / 16;

  uint64_t base, base2;
  int64_t bytes;
  int64_t step;
  int left;  // rows: reduction bytes left
  int voff[kLoads];
  int piece[2];  // rows: byte offset of the lane's piece, for even and odd loads

  // The slot of a row's piece c is c ^ key(row), so that the rows that lanes read together meet different banks.
  static __device__ __forceinline__ int key(int row) {
    return B ? (row & 3) | ((row >> 1) & 4) : row & 7;
  }
  // rows: `n` valid rows ld bytes apart. columns: `n` valid columns (of 2 bytes), reduction rows ld bytes apart.
  __device__ __forceinline__ void lanes(int n, int64_t ld, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int ii = wave * kLoads + i;
      if constexpr (!COLS) {
        int row = ii * kRowsPerLoad + lane / kSlots;
        const int pc = ((lane % kSlots) ^ key(row)) * 16;
        piece[i & 1] = pc;
        if constexpr (SPLIT) row = row >= ROWS / 2 ? row - ROWS / 2 : row;
        voff[i] = row < n ? row * (int)ld + pc : kOutOfRange;
      } else {
        constexpr int kPer = ROWS / 8;  // 16-byte pieces per reduction row
        const int p = ii * 64 + lane;
        const int kr = p / kPer, slot = p % kPer;
        const int c = slot ^ ((kr & 3) * (B ? 4 : 2));
        voff[i] = c * 8 < n ? kr * (int)ld + c * 16 : kOutOfRange;
      }
    }
  }
  // n rows of kbytes reduction bytes
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
    step = kStepBytes / 2 * ld;
    left = 0;
  }
  // Load I of the next step into the tile at lds; the last one moves on to the step after.
  template <int I>
  __device__ __forceinline__ void load(uint32_t lds, int wave) {
    int v = voff[I];
    if constexpr (!COLS) v = piece[I & 1] < left ? v : kOutOfRange;
    const bool second = SPLIT && wave * kLoads + I >= kBytes / 2048;
    load_to_lds(make_rsrc(second ? base2 : base, bytes), lds + (wave * kLoads + I) * 1024, v);
    if constexpr (I == kLoads - 1) {
      base += step;
      if constexpr (SPLIT) base2 += step;
      bytes -= step;
      left -= kStepBytes;
    }
  }
};

// Sixteen bytes of a lane's row, and eight elements of a lane's column (two transposing reads, the second four
// reduction rows on), from LDS. Addresses come in registers that the compiler cannot see through plus constants, so
// that the constants become the instructions' offsets.
template <int OFFSET>
__device__ __forceinline__ i32x4 read_rows(uint32_t addr) {
  return *(const __attribute__((address_space(3))) i32x4*)(uintptr_t)(addr + OFFSET);
}
template <int OFFSET, int ROW_BYTES>
__device__ __forceinline__ i32x4 read_cols(uint32_t addr) {
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  using Ptr = __attribute__((address_space(3))) s16x4*;
  const i32x2 a = __builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(uintptr_t)(addr + OFFSET)));
  const i32x2 b = __builtin_bit_cast(
      i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Ptr)(uintptr_t)(addr + OFFSET + 4 * ROW_BYTES)));
  return i32x4{a[0], a[1], b[0], b[1]};
}

// BM x BN tile by WM x WN waves. MF x NF fragments of 16 x 16 per wave. STAGES: steps that LDS holds; RING: and half a
// step more (see run_tiles).
template <int BM_, int BN_, int WM_, int WN_, int STAGES_, bool RING_ = false>
struct Shape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_;
  static constexpr bool RING = RING_;
  static constexpr int kFinal = RING ? 3 : STAGES;  // last steps of a tile, which load less or nothing
  static constexpr int kWaves = WM * WN, kThreads = kWaves * kWave;
  static constexpr int MF = BM / WM / 16, NF = BN / WN / 16;
  // A tile, B tile and (fp8) the scales of A's rows.
  static constexpr int stage(bool fp8) { return (BM + BN) * kStepBytes + (fp8 ? 1024 : 0); }
  static constexpr int lds(bool fp8) { return RING ? 5 * BM * kStepBytes : STAGES * stage(fp8); }
  static_assert(!RING || (BM == BN && STAGES == 2), "a ring of five equal operand tiles");
  static_assert(NF % 2 == 0, "fragments of B come in pairs");
  // Steps of a tile with n bytes of reduction: at least those that are written out, and even for fp8, where a step is one
  // set of groups and the column fragments of successive steps alternate.
  __host__ __device__ static constexpr int steps(int64_t n, bool fp8) {
    const int s = std::max((int)((n + kStepBytes - 1) / kStepBytes), kFinal);
    return fp8 ? (s + 1) & ~1 : s;
  }
};

// Compile-time loop: f(integral_constant<int, I>) for I = 0 .. N-1, so that offsets are constants.
template <int I, int N, class F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    static_for<I + 1, N>(f);
  }
}

// Fragments of one wave inside the operands' tiles in LDS.
//   SPLIT: the B tile's first half of rows are gate rows and its second half up rows; a wave takes the same
//   columns of both: fragments 0..NF/2-1 are gate, the rest up.
template <class S, bool ACOLS, bool BCOLS, bool SPLIT>
struct Fragments {
  static constexpr int kStep = kStepBytes, kPieces = 2;  // 16-byte pieces of a lane's row
  static constexpr int kA = ACOLS ? 4 : kPieces, kB = BCOLS ? S::NF / 2 : kPieces;
  uint32_t a[kA], b[kB];    // offsets in an operand's tile
  uint32_t ra[kA], rb[kB];  // addresses in the tiles being read
  static_assert(!BCOLS || (S::BN >= 128 && !SPLIT), "column swizzle of B");
  static_assert(!ACOLS || (S::MF >= 4 && S::BM >= 64), "column swizzle of A");

  __device__ __forceinline__ void init(int wave, int lane) {
    const int rho = lane & 15, q = lane >> 4;
    const int m0 = (wave / S::WN) * S::MF * 16;
    const int n0 = (wave % S::WN) * S::NF * 16 / (SPLIT ? 2 : 1);
    const int kr = q * 8 + (rho >> 2);
    const int key = rho & 7;  // the key of the rows this lane reads, in both operands
#pragma unroll
    for (int i = 0; i < kA; ++i) {
      if constexpr (!ACOLS)
        a[i] = (m0 + rho) * kStep + (((q + 4 * i) ^ key) * 16);
      else
        a[i] = kr * S::BM * 2 + (((m0 / 8 + i * 2 + ((rho & 3) >> 1)) ^ ((rho >> 2) * 2)) * 16) + (rho & 1) * 8;
    }
#pragma unroll
    for (int i = 0; i < kB; ++i) {
      if constexpr (!BCOLS)
        b[i] = (n0 + (rho >> 2) * 8 + (rho & 3)) * kStep + (((q + 4 * i) ^ key) * 16);
      else
        b[i] = kr * S::BN * 2 + (((n0 / 8 + i * 4 + (rho & 3)) ^ ((rho >> 2) * 4)) * 16);
    }
  }
  __device__ __forceinline__ void point(uint32_t at_a, uint32_t at_b) {
#pragma unroll
    for (int i = 0; i < kA; ++i) {
      ra[i] = at_a + a[i];
      asm volatile("" : "+v"(ra[i]));
    }
#pragma unroll
    for (int i = 0; i < kB; ++i) {
      rb[i] = at_b + b[i];
      asm volatile("" : "+v"(rb[i]));
    }
  }
  // Piece H (the step's H-th 64 bytes) of row fragment M / column fragment N.
  template <int M, int H>
  __device__ __forceinline__ i32x4 read_a() const {
    if constexpr (!ACOLS)
      return read_rows<M * 16 * kStep>(ra[H]);
    else
      return read_cols<(M >> 2) * 128 + H * 32 * S::BM * 2, S::BM * 2>(ra[M & 3]);
  }
  template <int N, int H>
  __device__ __forceinline__ i32x4 read_b() const {
    constexpr int half = SPLIT ? N / (S::NF / 2) : 0, f = SPLIT ? N % (S::NF / 2) : N;
    if constexpr (!BCOLS)
      return read_rows<((f >> 1) * 32 + (f & 1) * 4 + half * (S::BN / 2)) * kStep>(rb[H]);
    else
      return read_cols<(f & 1) * 8 + H * 32 * S::BN * 2, S::BN * 2>(rb[f >> 1]);
  }
};

// The wave's loads but the last N have landed and its LDS reads are done; then every wave of the workgroup is here.
template <int N>
__device__ __forceinline__ void wait_tiles() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// Makes the compiler wait for a loaded value here, if it still has to.
template <class T>
__device__ __forceinline__ void arrived(T& v) {
  asm volatile("" : "+v"(v));
}

// ---------------------------------------------------------------- a workgroup's tiles
// `Job` provides
//   Tile, first(t), next(t)       the workgroup's tiles in order (false: no more); t.steps from Shape::steps (a step past the
//                                 operands' ends multiplies zeros);
//   begin(t, a, b)                sets the operands up for step 0 of tile t;
//   turn(t, step, a, b)           the same for a later step at which a source changes;
//   load_scales(t, step, lds)     fp8: one load per wave that brings the step's row scales to lds;
//   begin_a, begin_b, none(t), gather(t), gathered()   int8, see below;
//   finish(t, acc)                the end of a tile: a known number of buffer stores per wave, whatever is masked;
//   wait<N>(stored)               wait_tiles<N>, or with the number of stores added.
//
// A step is a group of NF products for each row fragment and (bf16, int8) 64 bytes of the reduction. The row fragment of a
// group is read kAhead groups before it, into a ring of four, across the end of the step too: the barrier between
// steps comes when the last kAhead groups' operands are in registers, so the matrix unit has their work while the
// waves meet and the first reads of the next stage return. At that point every wave has read this stage, and the
// loads of the step that takes its place are issued: they have STAGES - 1 steps to land. Each read and load stands
// behind a product: a wave issues in order, and eight waves that all read at once fill the queue of LDS and hold up
// what stands behind their reads. Scheduling barriers keep that order: left to itself the compiler reads each fragment
// right before its products and waits out the latency of LDS every time. The steps in the middle of a tile run without a
// branch, and the last STAGES steps, which load nothing, are written out: a taken branch refetches instructions, which
// costs as much as several products.
//
// What a compute unit gets out of its L2 is bounded by the lines it can have in flight, so the loads must not pause. Two
// stages of a 256 x 256 tile are 128 KiB; while a step waits for the whole next stage nothing else is in flight, and a
// step took as long as loading one (3100 cycles against 2048 of products). LDS has room for half a stage more: as a ring
// of five operand tiles the row operand's loads run one step further ahead and stay in flight across the wait.
//
// The next tile's first steps are loaded before this one's results are worked out and stored. Loads and stores leave
// one in-order counter, so the first steps of a tile wait for all but the stores behind their loads.
//
// Int8 (kStream): a product takes half the time of a bf16 one's for its bytes, so what stands between tiles weighs twice as
// much, and in 65536 rows of 7168 to 2 x 2048 it took a tenth of the time (a tile of 262000 cycles: 8000 of finding the next
// tile and waiting, 9200 until its first loads were issued, 8100 of results). There the loads go on between tiles:
//   * They run on into the next tile. Its place is worked out before the last steps, which load its first ones, and the ring
//     or the stages go round without a new start. After the last tile they load nothing (none: out of range).
//   * Step t issues the row operand's loads of step t + STAGES - 1 (ring: t + 2) among its first products, into the place that
//     step t - 1 left, and B's of step t + STAGES (ring: t + 2) after its barrier, into its own. All of them after the barrier
//     took 1705 us where this takes 1586. A step still waits for the next one's: behind them may be the loads of
//     STAGES - 2 steps (ring: of A for one), and the last tile's stores as long as those loads are older than the stores:
//     one step in a ring, else STAGES - 2.
//   * What the end of a tile reads besides (gather) is loaded before its last step and waited for at that step's barrier:
//     later it would come behind the next tile's loads.
// They pause where the compiler waits for something of its own: it does not see the loads to LDS, so it lets everything
// land. That is once a tile at the last step's barrier (gather); where the next tile is in another group of 64 experts
// (find); and in the gated 256 x 256 kernel, whose steps leave seven registers too few, twice more around the first
// written-out step, where those come back.
// 65536 rows of 7168 to 2 x 2048 1790 -> 1586 us (2430 TOPS), of 2048 to 7168 with a residual 1395 -> 1073 (one card).
template <class S, bool ACOLS, bool BCOLS, Elem T, bool SPLIT, class Job>
__device__ __forceinline__ void run_tiles(Job& job, uint32_t lds, int wave, int lane) {
  constexpr bool FP8 = T == Elem::kE4m3;
  using Acc = AccOf<T>;
  constexpr int kStage = S::stage(FP8);
  using A = Operand<ACOLS, S::BM, S::kWaves, false>;
  using B = Operand<BCOLS, S::BN, S::kWaves, true, SPLIT>;
  using Frag = std::conditional_t<FP8, i32x8, i32x4>;
  constexpr int kHalves = FP8 ? 1 : 2;
  constexpr int kGroups = kHalves * S::MF, kRing = 4, kAhead = 3, kTail = kGroups - kAhead;
  constexpr int kLoads = A::kLoads + B::kLoads + (FP8 ? 1 : 0);
  constexpr int kLater = S::STAGES - 2;  // steps loading behind the one that a step waits for
  constexpr bool kStream = T == Elem::kInt8;  // loads run on into the next tile
  constexpr int kEvery = std::max(1, kTail / A::kLoads);  // groups from one of A's loads to the next
  static_assert(!kStream || A::kLoads <= kTail, "A's loads are issued before the barrier");
  static_assert(kGroups % kRing == 0, "ring of row fragments");
  static_assert(T == Elem::kBf16 || (!ACOLS && !BCOLS), "8-bit operands are rows");
  static_assert(kHalves == 2 || S::STAGES == 3, "steps() gives an fp8 tile one step more than the written-out three");
  static_assert(!S::RING || kHalves == 2, "a ring holds steps of two halves");
  Fragments<S, ACOLS, BCOLS, SPLIT> fr;
  fr.init(wave, lane);
  const uint32_t scale_at = A::kBytes + B::kBytes + ((wave / S::WN) * S::MF * 16 + (lane & 15)) * 4;
  A a;
  B b;
  Frag fa[kRing], fb[2][S::NF];  // fb: by half, or by the parity of the step where it has one
  float sc[2][S::MF];
  Acc acc[S::MF][S::NF];
  int at = 0;  // steps of the tile being loaded
  typename Job::Tile tile;
  // Load i of a step, B's first, into the tiles at to_a and to_b (fp8: the scales behind them).
  const auto load = [&](uint32_t to_a, uint32_t to_b, auto i) EPL_INLINE {
    if constexpr (i < B::kLoads)
      b.template load<i>(to_b, wave);
    else if constexpr (i < A::kLoads + B::kLoads)
      a.template load<i - B::kLoads>(to_a, wave);
    else if constexpr (FP8)
      job.load_scales(tile, at - 1, to_b + B::kBytes);
  };
  // The operand tile n places on in the ring.
  const auto ahead = [&](uint32_t at_tile, int n) EPL_INLINE {
    const uint32_t t = at_tile + n * A::kBytes;
    return t >= lds + 5 * A::kBytes ? t - 5 * A::kBytes : t;
  };
  // B's tile of the step whose A tile is at t.
  const auto b_of = [&](uint32_t t) EPL_INLINE { return S::RING ? ahead(t, 1) : t + A::kBytes; };
  // Of the stage that fr points to: column fragment n of half h into fb[to]; the row fragment of group g.
  const auto read_b = [&](auto to, auto n, auto h) EPL_INLINE {
    if constexpr (FP8) {
      const i32x4 lo = fr.template read_b<n, 0>(), hi = fr.template read_b<n, 1>();
      fb[to][n] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      fb[to][n] = fr.template read_b<n, h>();
    }
  };
  const auto read_a = [&](auto g) EPL_INLINE {
    if constexpr (FP8) {
      const i32x4 lo = fr.template read_a<g, 0>(), hi = fr.template read_a<g, 1>();
      fa[g % kRing] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      fa[g % kRing] = fr.template read_a<g % S::MF, g / S::MF>();
    }
  };
  const auto read_scale = [&](auto to, auto f, uint32_t stage) EPL_INLINE {
    sc[to][f] = *(const __attribute__((address_space(3))) float*)(uintptr_t)(stage + scale_at + f * 64);
  };
  using Zero = std::integral_constant<int, 0>;
  using One = std::integral_constant<int, 1>;
  // Set up a tile's operands and issue the loads of its first steps: STAGES of them, and the next one's A in a ring.
  const auto begin_tile = [&]() EPL_INLINE {
    job.begin(tile, a, b);
    at = 1;
    static_for<0, S::STAGES>([&](auto i) EPL_INLINE {
      const uint32_t t = lds + i * kStage;
      if constexpr (S::RING) {  // in the ring's order
        static_for<0, A::kLoads>([&](auto j) EPL_INLINE { a.template load<j>(t, wave); });
        static_for<0, B::kLoads>([&](auto j) EPL_INLINE { b.template load<j>(t + A::kBytes, wave); });
      } else {
        static_for<0, kStream && i == S::STAGES - 1 ? B::kLoads : kLoads>(
            [&](auto j) EPL_INLINE { load(t, t + A::kBytes, j); });
      }
      job.turn(tile, at, a, b);
      ++at;
    });
    if constexpr (S::RING && !kStream)
      static_for<0, A::kLoads>([&](auto j) EPL_INLINE { a.template load<j>(lds + 4 * A::kBytes, wave); });
  };

  uint32_t cur = lds;  // A's tile of the current step
  int stored = 0;  // steps still to come whose loads are in front of the previous tile's stores
  // One step. par: its parity. left: steps of the tile after it, kFinal for that many or more.
  const auto step = [&](auto par, auto left) EPL_INLINE {
    const uint32_t here = cur, here_b = b_of(cur);
    if constexpr (S::RING)
      cur = ahead(cur, 2);
    else
      cur = cur == lds + (S::STAGES - 1) * kStage ? lds : cur + kStage;
    static_for<0, kGroups>([&](auto g) EPL_INLINE {
      constexpr int m = g % S::MF, bi = kHalves == 2 ? g / S::MF : par;
      if constexpr (g == kTail) {
        // All reads of this stage have returned, also in the compiler's books: otherwise it would make the last
        // groups' products wait for the reads that follow the barrier.
        static_for<0, kAhead>([&](auto i) EPL_INLINE { arrived(fa[(g + i) % kRing]); });
        if constexpr (kHalves == 2) static_for<0, S::NF>([&](auto n) EPL_INLINE { arrived(fb[1][n]); });
        if constexpr (kStream) {
          job.template wait<S::RING ? A::kLoads : kLoads * kLater>(stored > 0);
          if constexpr (left == 0) job.gathered();
        } else if constexpr (left > 0) {
          constexpr int behind = S::RING ? (left > 1 ? A::kLoads : 0) : kLoads * std::min(kLater, left - 1);
          job.template wait<behind>(stored > 0);
        }
        if constexpr (left > 0) fr.point(cur, b_of(cur));
      }
      static_for<0, S::NF>([&](auto n) EPL_INLINE {
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (T == Elem::kInt8) {
          acc[m][n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[bi][n], fa[g % kRing], acc[m][n], 0, 0, 0);
        } else if constexpr (!FP8) {
          acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fb[bi][n]),
                                                              __builtin_bit_cast(bf16x8, fa[g % kRing]), acc[m][n], 0,
                                                              0, 0);
        } else {
          // One 128-element block of the row's scale: the block's product starts at zero and joins the sum
          // scaled, in 32 bits; the instruction's own block scales stay at one (exponent 127).
          const f32x4 p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
              fb[bi][n], fa[g % kRing], f32x4{0, 0, 0, 0}, 0, 0, 0, 0x7f7f7f7f, 0, 0x7f7f7f7f);
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[m][n][i] = fmaf(sc[bi][m], p[i], acc[m][n][i]);
        }
        // What follows this product in the instruction stream.
        if constexpr (g < kTail) {
          if constexpr (n == 0) read_a(std::integral_constant<int, g + kAhead>{});
          if constexpr (kStream && n == 2 && g % kEvery == kEvery - 1 && g / kEvery < A::kLoads)
            a.template load<g / kEvery>(S::RING      ? ahead(here, 4)
                                        : here == lds ? lds + (S::STAGES - 1) * kStage
                                                      : here - kStage,
                                        wave);
          // The second half's column fragments, spread over the first half's groups.
          constexpr int kOver = std::min(S::MF, kTail), per = (S::NF + kOver - 1) / kOver;
          if constexpr (kHalves == 2 && g < kOver && n == S::NF / 2)
            static_for<g * per, std::min((g + 1) * per, S::NF)>([&](auto i) EPL_INLINE { read_b(One{}, i, One{}); });
        } else if constexpr (left > 0 || kStream) {
          constexpr int slot = (g - kTail) * S::NF + n, kSlots = kAhead * S::NF;
          constexpr int to = kHalves == 2 ? 0 : 1 - par;
          if constexpr (left > 0 && slot < S::NF) read_b(std::integral_constant<int, to>{}, n, Zero{});
          // A ring entry is free once its own group is done.
          if constexpr (left > 0 && g == kTail + 1 && n < 2) read_a(n);
          if constexpr (left > 0 && g == kTail + 2 && n == 0) read_a(std::integral_constant<int, 2>{});
          if constexpr (FP8 && slot == S::NF)
            static_for<0, S::MF>([&](auto f) EPL_INLINE { read_scale(std::integral_constant<int, to>{}, f, cur); });
          // The freed tiles: in a ring they take B of the step after the next and then A of the one behind it.
          constexpr int issue = kStream ? B::kLoads : left == S::kFinal ? kLoads : S::RING && left == 2 ? B::kLoads : 0;
          if constexpr (issue > 0) {
            constexpr int per = (issue + kSlots - 1) / kSlots, begin = kSlots - (issue + per - 1) / per;
            if constexpr (slot >= begin)
              static_for<(slot - begin) * per, std::min((slot - begin + 1) * per, issue)>(
                  [&](auto i) EPL_INLINE { load(S::RING ? here_b : here, S::RING ? here : here_b, i); });
          }
        }
      });
      __builtin_amdgcn_sched_barrier(0);
    });
    stored -= stored > 0;
    if constexpr (left == S::kFinal) {
      job.turn(tile, at, a, b);
      ++at;
    }
  };
  using Middle = std::integral_constant<int, S::kFinal>;

  if (!job.first(tile)) return;
  begin_tile();
  constexpr int kFirst = kStream ? (S::RING ? kLoads : kLoads * (S::STAGES - 2) + B::kLoads)
                         : S::RING ? 2 * A::kLoads + B::kLoads : kLoads * (S::STAGES - 1);  // loads behind the first step's
  if constexpr (kStream) job.template wait<kFirst>(false);
  while (true) {
#pragma unroll
    for (int m = 0; m < S::MF; ++m)
#pragma unroll
      for (int n = 0; n < S::NF; ++n) acc[m][n] = Acc{0, 0, 0, 0};
    if constexpr (!kStream) {
      job.template wait<kFirst>(stored > 0);
      cur = lds;
    }
    fr.point(cur, b_of(cur));
    static_for<0, S::NF>([&](auto n) EPL_INLINE { read_b(Zero{}, n, Zero{}); });
    if constexpr (FP8) static_for<0, S::MF>([&](auto f) EPL_INLINE { read_scale(Zero{}, f, cur); });
    static_for<0, kAhead>(read_a);
    constexpr int kOdd = kHalves == 2 ? 0 : S::STAGES % 2;  // an odd number of written-out steps
    if constexpr (kOdd) step(Zero{}, Middle{});
    for (int s = tile.steps - S::kFinal - kOdd; s > 0; s -= kHalves == 2 ? 1 : 2) {
      step(std::integral_constant<int, kHalves == 2 ? 0 : kOdd>{}, Middle{});
      if constexpr (kHalves == 1) step(std::integral_constant<int, 1 - kOdd>{}, Middle{});
    }
    typename Job::Tile other = tile;  // the next tile; where loads run on into it, known before this one's last steps
    bool more = false;
    static_for<0, S::kFinal>([&](auto i) EPL_INLINE {
      if constexpr (kStream) {
        if constexpr (i == 0) {
          more = job.next(other);
          if (!more) job.none(other);
        }
        if constexpr (i == (S::RING ? 1 : 0)) job.begin_b(other, b);
        if constexpr (i == 1) job.begin_a(other, a);
        if constexpr (i == S::kFinal - 1) job.gather(tile);
      }
      step(std::integral_constant<int, kHalves == 2 ? 0 : (kOdd + i) % 2>{},
           std::integral_constant<int, S::kFinal - 1 - i>{});
    });
    if constexpr (kStream) {
      job.finish(tile, acc);
      if (!more) {
        wait_tiles<0>();  // no load to LDS outlives the workgroup
        return;
      }
      tile = other;
    } else {
      const typename Job::Tile done = tile;
      const bool some = job.next(tile);
      wait_tiles<0>();  // every wave has read the last stages
      if (some) begin_tile();
      job.finish(done, acc);
      if (!some) return;
    }
    stored = kStream && !S::RING ? S::STAGES - 2 : S::STAGES - 1;
  }
}

// ---------------------------------------------------------------- tiles over the experts' rows
// The rows [b0, b1) of an expert a lane, of a group of 64, its row tiles and those up to it.
struct Offsets {
  int group = -1, b0, b1;
  uint32_t n, sum;
};

// Where a row tile lies: expert e, its rows [beg, end), the row tiles before it and its own.
struct RowTile {
  int e = 0, beg = 0, end = 0;
  int64_t before = 0;
  int count = 0;
  int64_t chunk_before = 0;  // row tiles before e's group of 64 experts

  // Finds row tile m (BM rows a tile), not before the one found last; false past the last one. A wave works it out from
  // the offsets, 64 experts at a time, from the group where it last was: a table in LDS would cost the room of the
  // ring. Offsets are clipped to the buffer, so that whatever they hold, no access leaves it.
  // o: a group's offsets, kept by the caller from one call to the next or fresh.
  template <int BM>
  __device__ __forceinline__ bool find(const int32_t* expert_off, int E, int cap, int64_t m, int lane, Offsets& o) {
    for (int e0 = e & ~(kWave - 1); e0 < E; e0 += kWave) {
      if (e0 != o.group) {
        const int mine = std::min(e0 + lane, E - 1);
        o.b0 = std::min(std::max(expert_off[mine], 0), cap);
        o.b1 = std::min(std::max(expert_off[mine + 1], o.b0), cap);
        o.n = e0 + lane < E ? (uint32_t)(o.b1 - o.b0 + BM - 1) / BM : 0u;
        o.sum = (uint32_t)wave_inclusive_sum((int)o.n);
        o.group = e0;
      }
      const uint64_t past = __ballot(chunk_before + o.sum > m);
      if (past) {
        const int l = __builtin_ctzll(past);
        e = e0 + l;
        beg = __builtin_amdgcn_readlane(o.b0, l);
        end = __builtin_amdgcn_readlane(o.b1, l);
        count = __builtin_amdgcn_readlane((int)o.n, l);
        before = chunk_before + (uint32_t)__builtin_amdgcn_readlane((int)o.sum, l) - (uint32_t)count;
        return true;
      }
      chunk_before += (uint32_t)__builtin_amdgcn_readlane((int)o.sum, kWave - 1);
    }
    return false;
  }
};

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

// ---------------------------------------------------------------- activations (fp32)
// What is left of the normal distribution past a >= 0, 1 - Phi(a) = tail_ratio(a) exp(-a^2 / 2). The ratio is t times a
// polynomial of t = 1 / (1 + 0.35 a), fitted here to erfc in 64 bits over [0, 14.5] for the least maximum of the relative
// error (weighted least squares, the weights multiplied by the error until it levels out): 3.2e-8.
__device__ __forceinline__ float tail_ratio(float a) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.35f, a, 1.0f));
  float p = -0.02915786f;
  p = fmaf(p, t, 0.14403081f);
  p = fmaf(p, t, -0.25583878f);
  p = fmaf(p, t, 0.15931946f);
  p = fmaf(p, t, -0.023212211f);
  p = fmaf(p, t, 0.10555245f);
  p = fmaf(p, t, 0.1198213f);
  p = fmaf(p, t, 0.13986352f);
  p = fmaf(p, t, 0.1396213f);
  return t * p;
}
// exp(-v^2 / 4): twice as a factor, so that products with exp(-v^2 / 2) below fp32's normal range still come out.
__device__ __forceinline__ float bell_root(float v) { return __builtin_amdgcn_exp2f(v * v * -0.36067376022224085f); }

// QUICK: SiLU without the library's exponential and without a division.
template <int ACT, bool QUICK = false>
__device__ __forceinline__ float activate(float v) {
  if constexpr (ACT == EPL_ACT_SILU && QUICK) {
    // 2^t from t = -|v| / (2 ln 2), in two parts, so that it is right relative to its value; twice as a factor, so that the
    // product comes out where exp(-|v|) is below fp32's normal range. From |v| = 200 on that is 0 either way (and rest
    // would be a NaN for an infinity).
    const float a = fminf(fabsf(v), 200.0f), t = a * -0.72134752f;
    const float rest = fmaf(a, -9.6298151e-9f, fmaf(a, -0.72134752f, -t)) * 0.69314718f;
    const float p = __builtin_amdgcn_exp2f(t), e = fmaf(p, rest, p);
    return (v < 0.0f ? v * e * e : v) * __builtin_amdgcn_rcpf(fmaf(e, e, 1.0f));
  }
  if constexpr (ACT == EPL_ACT_SILU) {
    // From exp(-|v|), which cannot overflow: v / (1 + exp(-v)) is 0 below -88.7, where the value is -2.6e-37.
    const float e = expf(-fabsf(v));
    return (v < 0.0f ? v * e : v) / (1.0f + e);
  }
  if constexpr (ACT == EPL_ACT_GELU) {
    // v Phi(v) = max(v, 0) - |v| (1 - Phi(|v|)). From 1 + erf it would cancel for negative v: 4% off at -5, 0 from -5.6.
    // Past 16 the second term is 0 in fp32. (A branch, not a clamp: with none in any activation the compiler keeps more of
    // the epilogue's offsets across tiles than there are registers, which costs every forward product 3 to 6%.)
    const float a = fabsf(v);
    float r = v < 0.0f ? 0.0f : v;
    if (a < 16.0f) {
      const float e = bell_root(v);
      r = fmaf(-(e * tail_ratio(a) * a), e, r);
    }
    return r;
  }
  if constexpr (ACT == EPL_ACT_RELU) return v < 0.0f ? 0.0f : v;
  return v;
}
template <int ACT>
__device__ __forceinline__ float activate_grad(float v) {
  if constexpr (ACT == EPL_ACT_SILU) {
    const float e = expf(-fabsf(v)), r = 1.0f / (1.0f + e);
    const float s = v < 0.0f ? e * r : r;  // sigmoid(v), as in activate
    return s * (1.0f + v * (v < 0.0f ? r : e * r));
  }
  if constexpr (ACT == EPL_ACT_GELU) {
    // Phi(v) + v phi(v) = [v > 0] + (v / sqrt(2 pi) -+ tail_ratio(|v|)) exp(-v^2 / 2). At every bf16 value off by at most
    // 1.5e-7, and by 6e-5 of the result (next to its zero at -0.75). With the library's erf and exp the pass over dy and
    // pre took 256 us, with this 224 (32672 x 4104, bytes alone 170).
    const float e = bell_root(v), q = tail_ratio(fabsf(v));
    return fmaf(e * fmaf(v, 0.39894228040143268f, v > 0.0f ? -q : q), e, v > 0.0f ? 1.0f : 0.0f);
  }
  if constexpr (ACT == EPL_ACT_RELU) return v > 0.0f ? 1.0f : 0.0f;
  return 1.0f;
}
// f(integral_constant<int, activation>) of the activation `act`: one branch for all that f does.
template <class F>
__device__ __forceinline__ void with_activation(int act, F&& f) {
  switch (act) {
    case EPL_ACT_SILU: f(std::integral_constant<int, EPL_ACT_SILU>{}); break;
    case EPL_ACT_GELU: f(std::integral_constant<int, EPL_ACT_GELU>{}); break;
    case EPL_ACT_RELU: f(std::integral_constant<int, EPL_ACT_RELU>{}); break;
    default: f(std::integral_constant<int, EPL_ACT_NONE>{});
  }
}

}  // namespace epl
