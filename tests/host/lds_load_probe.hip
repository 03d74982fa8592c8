// The loads to LDS of the product tiles right behind vector instructions that set their descriptor, for a look at the
// assembly. Compiled, never run.
#include "gemm_tile.h"

extern "C" __global__ void probe_pieces(const char* const* p, uint32_t at) {
  const uint64_t base = (uint64_t)p[threadIdx.x];
  const uint32_t lo = (uint32_t)epl::uniform((int)base), hi = (uint32_t)epl::uniform((int)(base >> 32));
  epl::load_to_lds(epl::u32x4{lo, hi, 4096u, (uint32_t)epl::kBufferRsrcWord3}, at, threadIdx.x * 16);
}

extern "C" __global__ void probe_words(const char* const* p, uint32_t at) {
  const uint64_t base = (uint64_t)p[threadIdx.x];
  const uint32_t lo = (uint32_t)epl::uniform((int)base), hi = (uint32_t)epl::uniform((int)(base >> 32));
  epl::load_words_to_lds(epl::u32x4{lo, hi, 4096u, (uint32_t)epl::kBufferRsrcWord3}, at, threadIdx.x * 4);
}
