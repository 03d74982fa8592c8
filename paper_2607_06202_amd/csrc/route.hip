// The router: scores of a token's experts, its top-k choices with their gate weights, and the way back.
//
// One wave per token; lane l holds experts l, l + 64, ... The choices are taken one by one: a wave maximum over
// order-preserving integer keys (a key of 0 is an expert that cannot be chosen), then the lowest expert index
// among the lanes that hold the maximum.
//
// With a selection bias the order is that of score + bias, which fp32 arithmetic can get wrong where two experts
// nearly tie. So the fp32 keys choose only where every gap between one choice and the next best exceeds what the
// rounding can make of it; the rare other tokens are chosen again from fp64 scores.
#include <type_traits>

#include "epl_internal.h"
#include "experts.h"

namespace epl {

constexpr int kRouteWaves = 4;
// Most workgroups of a launch. 131072 tokens, 256 experts, us with 2048 / 4096 / 8192 / 16384: biased choice 126 / 120 /
// 117 / 114, gradient 95 / 90 / 83 / 82; one token to a wave, without the next token's loads in flight: 135 and 111.
constexpr int kRouteGrid = 16384;

__device__ __forceinline__ uint32_t order_key(float v) {
  const uint32_t u = __float_as_uint(v + 0.0f);  // -0 counts as 0
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ uint64_t order_key(double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v + 0.0);
  return u ^ ((uint64_t)((int64_t)u >> 63) | 0x8000000000000000ull);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

template <int CTRL, int ROW_MASK>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {  // lanes without a source take 0, the least key
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROW_MASK, 0xf, true);
  return v > o ? v : o;
}
// Maximum over the wave, uniform. Row shifts by 1, 2, 4, 8, then the broadcasts of lane 15 and lane 31.
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = dpp_max<0x111, 0xf>(v);
  v = dpp_max<0x112, 0xf>(v);
  v = dpp_max<0x114, 0xf>(v);
  v = dpp_max<0x118, 0xf>(v);
  v = dpp_max<0x142, 0xa>(v);
  v = dpp_max<0x143, 0xc>(v);
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    const uint64_t o = __shfl_xor((unsigned long long)v, off, kWave);
    v = v > o ? v : o;
  }
  return v;
}
__device__ __forceinline__ double wave_total(double v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
  return v;
}
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, ROW_MASK, 0xf, false));
}
// Sum over the wave in a fixed tree, uniform. Lanes without a source add 0.
__device__ __forceinline__ float wave_total(float v) {
  v = dpp_add<0x111, 0xf>(v);
  v = dpp_add<0x112, 0xf>(v);
  v = dpp_add<0x114, 0xf>(v);
  v = dpp_add<0x118, 0xf>(v);
  v = dpp_add<0x142, 0xa>(v);
  v = dpp_add<0x143, 0xc>(v);
  return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}

template <bool BF16>
__device__ __forceinline__ float load_logit(const void* logits, int64_t i) {
  if constexpr (BF16)
    return __uint_as_float((uint32_t)((const uint16_t*)logits)[i] << 16);
  else
    return ((const float*)logits)[i];
}
__device__ __forceinline__ bool can_choose(float l) { return l > -INFINITY; }  // false for NaN

// exp(l - m) for l <= m, 1 where they are equal (also where both are infinite).
// In fp32 from 2^t, t = x log2 e, with what the rounding of t left out put back to first order (log2 e in two parts): a
// unit or two in the last place, as expf, without its handling of results below fp32's normal range, which are 0 here.
// Past -150 the argument is clipped, also -inf under a maximum of +inf. Gradient of 131072 x 256 logits, same card: 74 us,
// with expf 83, with expf and cached stores 84 to 87.
__device__ __forceinline__ float exp_below(float l, float m) {
  constexpr float kLog2e = 1.44269502f, kLog2eRest = 1.92596303e-8f, kLn2 = 0.693147181f;
  const float x = fmaxf(l - m, -150.0f);
  const float t = x * kLog2e;
  const float rest = fmaf(x, kLog2eRest, fmaf(x, kLog2e, -t));
  const float e = __builtin_amdgcn_exp2f(t);
  return l == m ? 1.0f : fmaf(e, rest * kLn2, e);
}
__device__ __forceinline__ double exp_below(double l, double m) { return l == m ? 1.0 : exp(l - m); }
template <class F>
__device__ __forceinline__ F sigmoid(F l) {
  if constexpr (sizeof(F) == 8)
    return 1.0 / (1.0 + exp(-l));
  else
    return 1.0f / (1.0f + expf(-l));
}

// The same from the hardware's exponential and reciprocal (one unit in the last place each), for keys whose error is
// bounded below and for nothing that is returned.
__device__ __forceinline__ float exp_near(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504089f); }
__device__ __forceinline__ float sigmoid_near(float l) { return __builtin_amdgcn_rcpf(1.0f + exp_near(-l)); }

// Takes the k largest keys in order; lane j ends up with choice j (or -1). NEXT: also the largest key left.
template <int SLOTS, bool NEXT, class K>
__device__ __forceinline__ int take_top(K (&key)[SLOTS], int k, int lane, K* picked, K* next) {
  int mine = -1;
  K mine_key = 0;
  K best = 0;
  // A lane's keys in descending order, the lower slot first among equals (neighbours exchanged, so stable), with
  // their slots: a choice then only moves its lane's keys up. Sorting costs less than looking for the lane's
  // largest at every choice up to four slots.
  constexpr bool kSorted = SLOTS <= 4;
  uint32_t order = 0x03020100u;  // the sorted keys' slots, a byte each
  if constexpr (kSorted) {
    uint32_t slots[SLOTS];
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) slots[s] = s;
#pragma unroll
    for (int n = SLOTS - 1; n > 0; --n)
#pragma unroll
      for (int s = 0; s < n; ++s) {
        const bool swap = key[s] < key[s + 1];
        const K hi = swap ? key[s + 1] : key[s], lo = swap ? key[s] : key[s + 1];
        const uint32_t hs = swap ? slots[s + 1] : slots[s], ls = swap ? slots[s] : slots[s + 1];
        key[s] = hi;
        key[s + 1] = lo;
        slots[s] = hs;
        slots[s + 1] = ls;
      }
    order = 0;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) order |= slots[s] << (8 * s);
  }
  for (int j = 0; j < k + (NEXT ? 1 : 0); ++j) {
    K b = key[0];
    int bs = kSorted ? (int)(order & 255u) : 0;
    if constexpr (!kSorted) {
#pragma unroll
      for (int s = 1; s < SLOTS; ++s) {
        if (key[s] > b) {  // strictly: the lowest slot among equals
          b = key[s];
          bs = s;
        }
      }
    }
    best = wave_max(b);
    if (j == k || best == 0) break;
    // Lowest expert among the holders: lowest slot first, then lowest lane.
    const bool holds = b == best;
    uint64_t who = __ballot(holds);
    if (who & (who - 1)) {
#pragma unroll
      for (int s = 0; s < SLOTS; ++s) {
        const uint64_t at = __ballot(holds && bs == s);
        if (at) {
          who = at;
          break;
        }
      }
    }
    const int owner = __builtin_ctzll(who);
    const int slot = __builtin_amdgcn_readlane(bs, owner);
    if (lane == j) {
      mine = slot * kWave + owner;
      mine_key = best;
    }
    if constexpr (kSorted) {
      const bool move = lane == owner;
#pragma unroll
      for (int s = 0; s + 1 < SLOTS; ++s) key[s] = move ? key[s + 1] : key[s];
      key[SLOTS - 1] = move ? 0 : key[SLOTS - 1];
      order = move ? order >> 8 : order;
    } else {
#pragma unroll
      for (int s = 0; s < SLOTS; ++s)
        if (lane == owner && s == slot) key[s] = 0;
    }
  }
  *picked = mine_key;
  *next = best;
  return mine;
}

// fp64 scores and keys, for a token whose fp32 keys cannot be told apart.
template <int SLOTS>
__device__ __forceinline__ int take_top_wide(const float (&l)[SLOTS], const float* bias, float m, int E,
                                                       int k, bool sig, int lane) {
  double z[SLOTS], sum = 0.0;
#pragma unroll
  for (int s = 0; s < SLOTS; ++s) {
    z[s] = sig ? sigmoid((double)l[s]) : (can_choose(l[s]) ? exp_below((double)l[s], (double)m) : 0.0);
    sum += z[s];
  }
  sum = wave_total(sum);
  uint64_t key[SLOTS], a, b;
#pragma unroll
  for (int s = 0; s < SLOTS; ++s) {
    const int e = s * kWave + lane;
    key[s] = 0;
    if (e < E && can_choose(l[s])) {
      const double v = (sig ? z[s] : z[s] / sum) + (double)bias[e];
      if (v > -INFINITY) key[s] = order_key(v);
    }
  }
  return take_top<SLOTS, false, uint64_t>(key, k, lane, &a, &b);
}

// Weight of each chosen logit among the choices, p_j / sum of the chosen p, from scores scaled so that the largest
// stays in range: exp(l - m) for the softmax (its own sum cancels), exp(l - m) / (1 + exp(l)) for sigmoids that
// are all below one half, m the largest chosen logit. Zero where 64-bit sigmoids vanish.
__device__ __forceinline__ float share(float l, bool valid, bool sig) {
  constexpr float kVanish = -709.7827f;  // 1 / (1 + exp(-l)) is 0 in fp64 below
  const float m = key_value(wave_max(valid ? order_key(l) : 0u));
  float s = 0.0f;
  if (valid) {
    if (!sig)
      s = exp_below(l, m);
    else if (m >= 0.0f)
      s = sigmoid(l);
    else
      s = m < kVanish ? 0.0f : exp_below(l, m) / (1.0f + expf(l));
  }
  const float total = wave_total(s);
  return total > 0.0f ? s / total : 0.0f;
}

// A token's logits: experts lane, lane + 64, ...; -inf past the last expert.
template <int SLOTS, bool BF16>
__device__ __forceinline__ void load_row(const void* logits, int64_t g, int E, int lane, float (&l)[SLOTS]) {
#pragma unroll
  for (int s = 0; s < SLOTS; ++s) {
    const int e = s * kWave + lane;
    const float v = load_logit<BF16>(logits, g * E + std::min(e, E - 1));  // no branch for the last lanes
    l[s] = e < E ? v : -INFINITY;
  }
}
// Expert e's logit, of a row in registers; e differs from lane to lane.
template <int SLOTS>
__device__ __forceinline__ float pick_logit(const float (&l)[SLOTS], int e) {
  float v = -INFINITY;
#pragma unroll
  for (int s = 0; s < SLOTS; ++s) {
    const float o = __shfl(l[s], e & (kWave - 1), kWave);
    v = (e >> 6) == s ? o : v;
  }
  return v;
}

// The next token's logits load while a token is worked on. What bounds it is vector instructions, not the 128 MiB of
// logits: with four slots 22 for each choice and one more round for the certificate, and the scores, the sort and the
// weights around them.
template <int SLOTS, bool BF16, bool SIGMOID, bool BIASED>
__global__ void __launch_bounds__(kRouteWaves* kWave) route_kernel(RouteArgs p) {
  const int lane = threadIdx.x % kWave;
  const int E = p.E, k = p.k;
  const int64_t stride = (int64_t)gridDim.x * kRouteWaves;
  int64_t g = (int64_t)blockIdx.x * kRouteWaves + threadIdx.x / kWave;
  float coming[SLOTS], bias[SLOTS];
  if (g < p.T) load_row<SLOTS, BF16>(p.logits, g, E, lane, coming);
  if constexpr (BIASED) load_row<SLOTS, false>(p.bias, 0, E, lane, bias);
  const bool need_sum = !SIGMOID && (!p.normalize || BIASED);
  for (; g < p.T; g += stride) {
    float l[SLOTS];
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) l[s] = coming[s];
    if (g + stride < p.T) load_row<SLOTS, BF16>(p.logits, g + stride, E, lane, coming);
    // For the softmax scores, the largest logit and the sum.
    float m = 0.0f, sum = 1.0f, inv = 1.0f;
    if (need_sum) {
      uint32_t top = 0;
#pragma unroll
      for (int s = 0; s < SLOTS; ++s) top = can_choose(l[s]) ? std::max(top, order_key(l[s])) : top;
      m = key_value(wave_max(top));
      sum = 0.0f;
#pragma unroll
      for (int s = 0; s < SLOTS; ++s) sum += can_choose(l[s]) ? exp_below(l[s], m) : 0.0f;
      sum = wave_total(sum);
      inv = __builtin_amdgcn_rcpf(sum);
    }
    uint32_t key[SLOTS], picked, next;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      float v = l[s];
      if constexpr (BIASED)
        v = (SIGMOID ? sigmoid_near(l[s]) : (l[s] == m ? 1.0f : exp_near(l[s] - m)) * inv) + bias[s];
      const uint32_t kv = order_key(v);
      key[s] = can_choose(l[s]) && v > -INFINITY ? kv : 0u;
    }
    int e = take_top<SLOTS, BIASED, uint32_t>(key, k, lane, &picked, &next);
    if constexpr (BIASED) {
      // Error of an fp32 key: the exponential's argument x (rounded twice and multiplied by log2 e, 2e-7 |x| e^x
      // <= 1e-7), the exponential and the reciprocal 2.4e-7, the sum of up to 1024 terms (16 per lane, then a tree of
      // 6) and its own exponentials 1.5e-6, the multiplication 6e-8, all relative to a score of at most 1, and half a
      // unit of the final sum. Two keys further apart than twice that are in the right order.
      uint32_t after = (uint32_t)__shfl_down((int)picked, 1, kWave);
      if (lane == k - 1) after = next;
      const float a = key_value(picked), b = key_value(after);
      const bool near = lane < k && picked && after && !(a - b > 4e-6f + 2.4e-7f * (fabsf(a) + fabsf(b)));
      if (__ballot(near)) e = take_top_wide<SLOTS>(l, p.bias, m, E, k, SIGMOID, lane);
    }
    // Lane j: the score and weight of choice j.
    const bool valid = lane < k && e >= 0;
    const float chosen = pick_logit<SLOTS>(l, valid ? e : 0);
    const float le = valid ? chosen : -INFINITY;
    float sc = 0.0f;
    if (p.normalize)
      sc = share(le, valid, SIGMOID);
    else if (valid)
      sc = SIGMOID ? sigmoid(le) : exp_below(le, m) / sum;
    if (lane < k) {
      p.idx[g * k + lane] = e;
      p.w[g * k + lane] = sc * p.scale;
    }
  }
}

// Gradient of the logits. With p the scores, d_j = scale dw_j for choice j of expert e_j:
//   softmax               dl = p (dp - sum p dp), dp_e the sum of d_j over the choices of e
//   sigmoid               dl = dp p (1 - p)
//   renormalised softmax  dl_e = sum of w_j (d_j - sum_i w_i d_i) over the choices of e, w as in the forward pass:
//                         the row's own sum drops out
//   renormalised sigmoid  the same terms times (1 - p)
// Choices outside [0, E) count for nothing, and neither does a chosen expert that is masked.
template <int SLOTS, bool BF16>
__global__ void __launch_bounds__(kRouteWaves* kWave) route_backward_kernel(RouteArgs p) {
  const int lane = threadIdx.x % kWave;
  const int E = p.E, k = p.k;
  const bool need_row = !p.sigmoid && !p.normalize;
  const int64_t stride = (int64_t)gridDim.x * kRouteWaves;
  int64_t g = (int64_t)blockIdx.x * kRouteWaves + threadIdx.x / kWave;
  // The next token's choices, gradients and (where the whole row counts) logits load while a token is worked on.
  int coming_e = -1;
  float coming_dw = 0.0f, coming[SLOTS];
  const auto load = [&](int64_t t) __attribute__((always_inline)) {
    if (lane < k) {
      coming_e = p.idx[t * k + lane];
      coming_dw = p.dw[t * k + lane];
    }
    if (need_row) load_row<SLOTS, BF16>(p.logits, t, E, lane, coming);
  };
  if (g < p.T) load(g);
  for (; g < p.T; g += stride) {
    const int e = coming_e;
    float dw = coming_dw;
    const bool in = e >= 0 && e < E;
    float le;
    float p_row[SLOTS], m = 0.0f, sum = 1.0f;  // p_row: exp(l - m), 0 for a masked expert
    if (need_row) {
      float l[SLOTS];
      uint32_t top = 0;
#pragma unroll
      for (int s = 0; s < SLOTS; ++s) {
        l[s] = coming[s];
        top = can_choose(l[s]) ? std::max(top, order_key(l[s])) : top;
      }
      if (g + stride < p.T) load(g + stride);
      m = key_value(wave_max(top));
      sum = 0.0f;
#pragma unroll
      for (int s = 0; s < SLOTS; ++s) {
        p_row[s] = can_choose(l[s]) ? exp_below(l[s], m) : 0.0f;
        sum += p_row[s];
      }
      sum = wave_total(sum);
      le = pick_logit<SLOTS>(l, in ? e : 0);
    } else {
      le = in ? load_logit<BF16>(p.logits, g * E + e) : -INFINITY;
      if (g + stride < p.T) load(g + stride);
    }
    const bool valid = in && can_choose(le);
    dw = valid ? dw * p.scale : 0.0f;
    // What each choice adds to its expert's logit.
    float sc;
    if (p.normalize) {
      sc = share(le, valid, p.sigmoid);
      dw -= wave_total(dw * sc);
    } else {
      sc = !valid ? 0.0f : p.sigmoid ? sigmoid(le) : exp_below(le, m) / sum;
    }
    float add = valid ? dw * sc : 0.0f;
    if (p.sigmoid && valid) add *= sigmoid(-le);
    const float all = need_row && sum > 0.0f ? wave_total(add) / sum : 0.0f;
    float d[SLOTS];
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) d[s] = need_row ? -p_row[s] * all : 0.0f;
    for (int j = 0; j < k; ++j) {
      const int ej = __builtin_amdgcn_readlane(valid ? e : -1, j);
      const float aj = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(add), j));
#pragma unroll
      for (int s = 0; s < SLOTS; ++s)
        if (ej == s * kWave + lane) d[s] += aj;
    }
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      const int ee = s * kWave + lane;
      if (ee >= E) continue;
      if constexpr (BF16)
        ((uint16_t*)p.dlogits)[g * E + ee] = (uint16_t)f32x2_to_bf16x2(d[s], 0.0f);
      else
        __builtin_nontemporal_store(d[s], (float*)p.dlogits + g * E + ee);
    }
  }
}

template <int SLOTS>
static void launch_slots(const RouteArgs& p, bool back, dim3 grid, hipStream_t s) {
  const dim3 block(kRouteWaves * kWave);
  if (back) {
    if (p.bf16)
      hipLaunchKernelGGL((route_backward_kernel<SLOTS, true>), grid, block, 0, s, p);
    else
      hipLaunchKernelGGL((route_backward_kernel<SLOTS, false>), grid, block, 0, s, p);
  } else {
    const auto score = [&](auto bf16, auto sigmoid) {
      if (p.bias)
        hipLaunchKernelGGL((route_kernel<SLOTS, bf16, sigmoid, true>), grid, block, 0, s, p);
      else
        hipLaunchKernelGGL((route_kernel<SLOTS, bf16, sigmoid, false>), grid, block, 0, s, p);
    };
    const auto type = [&](auto bf16) {
      if (p.sigmoid)
        score(bf16, std::true_type{});
      else
        score(bf16, std::false_type{});
    };
    if (p.bf16)
      type(std::true_type{});
    else
      type(std::false_type{});
  }
}

static hipError_t launch(const RouteArgs& p, bool back, hipStream_t s) {
  if (p.T == 0) return hipSuccess;
  const dim3 grid((unsigned)std::min<int64_t>((p.T + kRouteWaves - 1) / kRouteWaves, kRouteGrid));
  if (p.E <= 64)
    launch_slots<1>(p, back, grid, s);
  else if (p.E <= 128)
    launch_slots<2>(p, back, grid, s);
  else if (p.E <= 256)
    launch_slots<4>(p, back, grid, s);
  else if (p.E <= 512)
    launch_slots<8>(p, back, grid, s);
  else
    launch_slots<16>(p, back, grid, s);
  return hipGetLastError();
}

hipError_t launch_route(const RouteArgs& p, hipStream_t s) { return launch(p, false, s); }
hipError_t launch_route_backward(const RouteArgs& p, hipStream_t s) { return launch(p, true, s); }

}  // namespace epl
