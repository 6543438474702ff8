// What the two tensor-core kernels over the paged 4-bit cache share.
#pragma once

#include "attn_paged8.cuh"
#include "fp4_common.cuh"

namespace lca {

struct Paged4Params {
  Paged8Params b;             // without the tensor maps and the scales
  const uint8_t* sem; const uint8_t* pos;
  const uint8_t* shift_sem; const uint8_t* shift_pos;
  const uint8_t* exp_k; const uint8_t* exp_v;
};

// whether the phase is complete, at once (try_wait may suspend the thread while the other barrier that it looks at completes)
__device__ __forceinline__ bool phase_done(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  return done != 0;
}

// 16 bytes that are read once
__device__ __forceinline__ uint4 load_stream(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

int attn_paged4_pair_launch(Paged4Params& P, cudaStream_t stream);      // MLA shape, blocks of 128 rows on CTA pairs
int attn_paged4_pair_take_status();

}  // namespace lca
