// What the kernels on CTA pairs over the paged 8-bit and 4-bit caches share.
#pragma once

#include "attn_paged8.cuh"

namespace lca {

__device__ __forceinline__ void umma_f8_pair_elected(uint32_t leader, uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                                     uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(leader) : "memory");
}
// Offsets of the keys (weight_offset), read four at a time by whole warps.  Offsets for every row of a sequence would not fit; windows
// of 128 of them that start anywhere are as evenly spread, so a tile takes one of 1024 windows, in an order in which any number
// of successive ones is even as well.
constexpr int WINDOWS = 1024, WINDOW_ORDER = 613;
struct OffsetTable {
  float v[4 * WINDOWS + 128];
  constexpr OffsetTable() : v() {
    for (int i = 0; i < 4 * WINDOWS + 128; ++i) v[i] = (float)(int32_t)((uint32_t)i * GOLDEN) * 0x1p-41f;
  }
};
__constant__ const OffsetTable g_offsets{};

// bits [0, n) of a word of 64; n may be anything
__device__ __forceinline__ uint64_t low_bits(int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1ull; }

}  // namespace lca
