// What the two kernels over the paged 4-bit cache share.
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

static constexpr float T4_MAX = 8.75f;                       // log2 of the largest weight: e4m3 ends at 448
static constexpr float LO4_GAIN = 16.f;                      // of the second term, which has columns of O of its own

int attn_paged4_few_launch(const lca_params* p, Paged4Params& P, cudaStream_t stream);      // GQA, few query rows a KV head

}  // namespace lca
