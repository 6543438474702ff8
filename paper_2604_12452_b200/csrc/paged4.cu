// The paged 4-bit cache around its attention: the quantising write, reading rows back and the online condensation of a group.  The
// format is described in fp4_common.cuh and lca.h.
#include "fp4_common.cuh"
#include "paged_update.cuh"

namespace lca {

// ------------------------------------------------------------------------------------------------- write, read back
// Rows do not depend on one another (the exponent is the row's own), so there are no runs and no order to keep: a lane takes eight
// values (16 bytes in, 4 out), four lanes a block.  HBM-bound.
struct Paged4Rows {
  bf16* sem; bf16* pos;                                      // [n_rows, Hkv, d]: in (write), out (read)
  const int32_t* slots;
  uint32_t* pages_sem; uint32_t* pages_pos; uint8_t* shift_sem; uint8_t* shift_pos; uint8_t* exp_sem; uint8_t* exp_pos;
  long long n_rows, n_slots;
  int Hkv, page_log2;
};
// Row of the pool for slot s and KV head hk.
__device__ __forceinline__ size_t pool_row(const Paged4Rows& a, int s, int hk) {
  return (((size_t)(s >> a.page_log2) * a.Hkv + hk) << a.page_log2) + (size_t)(s & ((1 << a.page_log2) - 1));
}
// Largest finite |x| of eight bf16 values as bf16 bits; nan: whether one of them is NaN.
__device__ __forceinline__ uint32_t top8(const uint4& v, bool& nan) {
  uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
  uint32_t top = max(m & 0xffffu, m >> 16);
  nan = top > 0x7f80u;
  if (top >= 0x7f80u) {
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
    top = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t lo = u[k] & 0x7fffu, hi = (u[k] >> 16) & 0x7fffu;
      top = max(top, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
    }
  }
  return top;
}
__device__ __forceinline__ uint32_t pack8(const uint4& v, int e) {
  const float f = exp2_int(-e);                              // -108 <= e <= 126; the products are exact
  const uint32_t u[4] = {v.x, v.y, v.z, v.w};
  float x[8];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    x[2 * k] = __uint_as_float(u[k] << 16) * f;
    x[2 * k + 1] = __uint_as_float(u[k] & 0xffff0000u) * f;
  }
  return paged4_pack(x);
}
__device__ __forceinline__ uint4 unpack8(uint32_t w, int shift, float f, const uint2* s_table) {
  const uint2 c = paged4_expand(w, s_table[shift]);
  const float4 a = e4m3x4_to_float4(c.x), b = e4m3x4_to_float4(c.y);
  return make_uint4(tc::pack_bf16x2(a.x * f, a.y * f), tc::pack_bf16x2(a.z * f, a.w * f),
                    tc::pack_bf16x2(b.x * f, b.y * f), tc::pack_bf16x2(b.z * f, b.w * f));
}

static const int ROW_THREADS = 256, ROW_WARPS = ROW_THREADS / 32;

// MLA: a warp per row.  Units of eight values: lane and lane + 32 of the latent (512 wide; 128 wide: lanes 0..15), lanes 0..7 the key.
template <int D_SEM>
__global__ void __launch_bounds__(ROW_THREADS) paged4_write_mla_kernel(Paged4Rows a) {
  constexpr int D_POS = 64, NS = D_SEM / 256 > 0 ? D_SEM / 256 : 1, US = D_SEM / 8;
  const int lane = threadIdx.x & 31;
  const long long warps = (long long)gridDim.x * ROW_WARPS;
  chain_wait();
  chain_next();
#pragma unroll 2
  for (long long i = (long long)blockIdx.x * ROW_WARPS + (threadIdx.x >> 5); i < a.n_rows; i += warps) {
    const int slot = a.slots[i];
    if (slot < 0 || slot >= a.n_slots) continue;
    uint4 v[NS + 1];
#pragma unroll
    for (int q = 0; q < NS; ++q)
      v[q] = lane + 32 * q < US ? __ldcs(reinterpret_cast<const uint4*>(a.sem + (size_t)i * D_SEM) + lane + 32 * q) : make_uint4(0u, 0u, 0u, 0u);
    v[NS] = lane < D_POS / 8 ? __ldcs(reinterpret_cast<const uint4*>(a.pos + (size_t)i * D_POS) + lane) : make_uint4(0u, 0u, 0u, 0u);
    uint32_t top[NS + 1], all = 0;
    unsigned nan = 0;
#pragma unroll
    for (int q = 0; q <= NS; ++q) {
      bool n;
      uint32_t t = top8(v[q], n);
      t = max(t, __shfl_xor_sync(0xffffffffu, t, 1));
      t = max(t, __shfl_xor_sync(0xffffffffu, t, 2));
      const unsigned b = __ballot_sync(0xffffffffu, n);
      nan |= ((b >> (lane & ~3)) & 15u) ? 1u << q : 0u;
      top[q] = t; all = max(all, t);
    }
    all = __reduce_max_sync(0xffffffffu, all);
    const int E = max(paged4_block_exponent(all), PAGED4_MIN_EXP);
    const size_t row = pool_row(a, slot, 0);
#pragma unroll
    for (int q = 0; q <= NS; ++q) {
      const int shift = min(E - paged4_block_exponent(top[q]), PAGED4_MAX_SHIFT), s = (nan >> q) & 1u ? PAGED4_NAN_SHIFT : shift;
      const uint32_t w = pack8(v[q], E - shift);
      const int next = __shfl_down_sync(0xffffffffu, s, 4);
      if (q < NS && lane + 32 * q < US) {
        a.pages_sem[row * (D_SEM / 8) + lane + 32 * q] = w;
        if ((lane & 7) == 0) a.shift_sem[row * (D_SEM / 64) + (lane + 32 * q) / 8] = (uint8_t)(s | next << 4);
      }
      if (q == NS && lane < D_POS / 8) {
        a.pages_pos[row * (D_POS / 8) + lane] = w;
        if (lane == 0) a.shift_pos[row] = (uint8_t)(s | next << 4);
      }
    }
    if (lane == 0) a.exp_sem[row] = (uint8_t)(E + PAGED4_EXP_BIAS);
  }
}

// GQA: a warp takes a row's keys or values, or up to 16 KV heads of them (blockIdx.y: the two parts, then groups of heads), D / 8 lanes
// a vector and a KV head.  All its loads are under way before the first is used.
template <int D>
struct GqaRow {
  static constexpr int U = D / 8, HEADS = 32 / U;            // lanes of a vector; KV heads of a step
  static constexpr int STEPS = 16 / HEADS;
};
template <int D>
__global__ void __launch_bounds__(ROW_THREADS) paged4_write_gqa_kernel(Paged4Rows a) {
  using G = GqaRow<D>;
  const bool pos = blockIdx.y & 1;
  const int hk0 = (int)(blockIdx.y >> 1) * 16, lane = threadIdx.x & 31, u = lane % G::U;
  const uint4* src = reinterpret_cast<const uint4*>(pos ? a.pos : a.sem);
  uint32_t* pages = pos ? a.pages_pos : a.pages_sem;
  uint8_t* shifts = pos ? a.shift_pos : a.shift_sem;
  uint8_t* exps = pos ? a.exp_pos : a.exp_sem;
  const long long warps = (long long)gridDim.x * ROW_WARPS;
  chain_wait();
  chain_next();
  for (long long i = (long long)blockIdx.x * ROW_WARPS + (threadIdx.x >> 5); i < a.n_rows; i += warps) {
    const int slot = a.slots[i];
    if (slot < 0 || slot >= a.n_slots) continue;
    const uint4* row_src = src + ((size_t)i * a.Hkv + hk0) * G::U + lane;
    uint4 v[G::STEPS];
#pragma unroll
    for (int k = 0; k < G::STEPS; ++k)
      if (hk0 + k * G::HEADS < a.Hkv) v[k] = hk0 + k * G::HEADS + lane / G::U < a.Hkv ? __ldcs(row_src + k * 32) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int k = 0; k < G::STEPS; ++k) {
      if (hk0 + k * G::HEADS >= a.Hkv) break;                // the same in every lane
      bool n;
      uint32_t top = top8(v[k], n);
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const bool nan = (__ballot_sync(0xffffffffu, n) >> (lane & ~3)) & 15u;
      uint32_t all = max(top, __shfl_xor_sync(0xffffffffu, top, 4));
      if (G::U == 16) all = max(all, __shfl_xor_sync(0xffffffffu, all, 8));
      const int E = max(paged4_block_exponent(all), PAGED4_MIN_EXP);
      const int shift = min(E - paged4_block_exponent(top), PAGED4_MAX_SHIFT), s = nan ? PAGED4_NAN_SHIFT : shift;
      const uint32_t w = pack8(v[k], E - shift);
      const int next = __shfl_down_sync(0xffffffffu, s, 4), hk = hk0 + k * G::HEADS + lane / G::U;
      if (hk < a.Hkv) {
        const size_t row = pool_row(a, slot, hk);
        pages[row * G::U + u] = w;
        if (u % 8 == 0) shifts[row * (D / 64) + u / 8] = (uint8_t)(s | next << 4);
        if (u == 0) exps[row] = (uint8_t)(E + PAGED4_EXP_BIAS);
      }
    }
  }
}

template <int D_SEM>
__global__ void __launch_bounds__(ROW_THREADS) paged4_read_mla_kernel(Paged4Rows a) {
  constexpr int D_POS = 64, NS = D_SEM / 256 > 0 ? D_SEM / 256 : 1, US = D_SEM / 8;
  __shared__ uint2 s_table[16];
  const int lane = threadIdx.x & 31;
  const long long warps = (long long)gridDim.x * ROW_WARPS;
  paged4_table_load(s_table, threadIdx.x);
  __syncthreads();
  chain_wait();
  chain_next();
#pragma unroll 2
  for (long long i = (long long)blockIdx.x * ROW_WARPS + (threadIdx.x >> 5); i < a.n_rows; i += warps) {
    const int slot = a.slots[i];
    if (slot < 0 || slot >= a.n_slots) continue;
    const size_t row = pool_row(a, slot, 0);
    uint32_t w[NS + 1];
    int s[NS + 1];
#pragma unroll
    for (int q = 0; q < NS; ++q) {
      const int u = lane + 32 * q;
      w[q] = u < US ? __ldcs(a.pages_sem + row * US + u) : 0u;
      s[q] = u < US ? a.shift_sem[row * (D_SEM / 64) + u / 8] >> (u & 4) & 15 : 0;
    }
    w[NS] = lane < D_POS / 8 ? __ldcs(a.pages_pos + row * (D_POS / 8) + lane) : 0u;
    s[NS] = lane < D_POS / 8 ? a.shift_pos[row] >> (lane & 4) & 15 : 0;
    const float f = paged4_factor(a.exp_sem[row]);
#pragma unroll
    for (int q = 0; q < NS; ++q)
      if (lane + 32 * q < US) __stcs(reinterpret_cast<uint4*>(a.sem + (size_t)i * D_SEM) + lane + 32 * q, unpack8(w[q], s[q], f, s_table));
    if (lane < D_POS / 8) __stcs(reinterpret_cast<uint4*>(a.pos + (size_t)i * D_POS) + lane, unpack8(w[NS], s[NS], f, s_table));
  }
}

template <int D>
__global__ void __launch_bounds__(ROW_THREADS) paged4_read_gqa_kernel(Paged4Rows a) {
  using G = GqaRow<D>;
  __shared__ uint2 s_table[16];
  const bool pos = blockIdx.y & 1;
  const int hk0 = (int)(blockIdx.y >> 1) * 16, lane = threadIdx.x & 31, u = lane % G::U;
  uint4* dst = reinterpret_cast<uint4*>(pos ? a.pos : a.sem);
  const uint32_t* pages = pos ? a.pages_pos : a.pages_sem;
  const uint8_t* shifts = pos ? a.shift_pos : a.shift_sem;
  const uint8_t* exps = pos ? a.exp_pos : a.exp_sem;
  const long long warps = (long long)gridDim.x * ROW_WARPS;
  paged4_table_load(s_table, threadIdx.x);
  __syncthreads();
  chain_wait();
  chain_next();
  for (long long i = (long long)blockIdx.x * ROW_WARPS + (threadIdx.x >> 5); i < a.n_rows; i += warps) {
    const int slot = a.slots[i];
    if (slot < 0 || slot >= a.n_slots) continue;
    uint32_t w[G::STEPS];
    int s[G::STEPS], e[G::STEPS];
#pragma unroll
    for (int k = 0; k < G::STEPS; ++k) {
      const int hk = hk0 + k * G::HEADS + lane / G::U;
      w[k] = 0; s[k] = 0; e[k] = 0;
      if (hk < a.Hkv) {
        const size_t row = pool_row(a, slot, hk);
        w[k] = __ldcs(pages + row * G::U + u);
        s[k] = shifts[row * (D / 64) + u / 8];
        e[k] = exps[row];
      }
    }
    uint4* row_dst = dst + ((size_t)i * a.Hkv + hk0) * G::U + lane;
#pragma unroll
    for (int k = 0; k < G::STEPS; ++k)
      if (hk0 + k * G::HEADS + lane / G::U < a.Hkv) __stcs(row_dst + k * 32, unpack8(w[k], s[k] >> (u & 4) & 15, paged4_factor(e[k]), s_table));
  }
}

int paged4_rows_launch(const lca_params* p, const lca_paged4* c, bool write, const void* rows_sem, const void* rows_pos,
                       const int32_t* slot_map, long long n_rows, cudaStream_t stream) {
  const bool mla = p->variant == LCA_VARIANT_MLA;
  Paged4Rows a = {(bf16*)rows_sem, (bf16*)rows_pos, slot_map, (uint32_t*)c->pages_sem, (uint32_t*)c->pages_pos, c->shift_sem, c->shift_pos,
                  c->exp_sem, c->exp_pos, n_rows, (long long)c->n_pages * c->page_size, p->n_kv_heads,
                  c->page_size == 16 ? 4 : c->page_size == 32 ? 5 : c->page_size == 64 ? 6 : 7};
  const long long most = 148 * 8 * 8;                        // eight waves of all CTAs that are resident
  if (mla) {
    const long long want = (n_rows + ROW_WARPS - 1) / ROW_WARPS;
    const dim3 grid((unsigned)(want < most ? want : most), 1);
    auto kern = write ? (p->d_sem == 512 ? paged4_write_mla_kernel<512> : paged4_write_mla_kernel<128>)
                      : (p->d_sem == 512 ? paged4_read_mla_kernel<512> : paged4_read_mla_kernel<128>);
    return launch_chained(kern, grid, ROW_THREADS, 0, stream, 1, a);
  }
  const long long want = (n_rows + ROW_WARPS - 1) / ROW_WARPS, parts = 2 * ((p->n_kv_heads + 15) / 16);
  if (parts > 65535) return LCA_ERR_UNSUPPORTED_SHAPE;
  const dim3 grid((unsigned)(want < most ? want : most), (unsigned)parts);
  auto kern = write ? (p->d_sem == 128 ? paged4_write_gqa_kernel<128> : paged4_write_gqa_kernel<64>)
                    : (p->d_sem == 128 ? paged4_read_gqa_kernel<128> : paged4_read_gqa_kernel<64>);
  return launch_chained(kern, grid, ROW_THREADS, 0, stream, 1, a);
}

// ------------------------------------------------------------------------------------------------------------ update
int paged4_update_launch(const lca_params* p, const lca_paged4* c, const float* qbar_f, const double* qbar_d, const int32_t* n_rep,
                         const int32_t* n_tok, int32_t* n_rep_new, void* rep_sem, void* rep_pos, int32_t* anchor_out,
                         cudaStream_t stream) {
  const PagedRows4 rows = {(const uint8_t*)c->pages_sem, (const uint8_t*)c->pages_pos, c->shift_sem, c->shift_pos, c->exp_sem, c->exp_pos};
  return paged_update_shapes(p, c, rows, qbar_f, qbar_d, n_rep, n_tok, n_rep_new, rep_sem, rep_pos, anchor_out, stream);
}

}  // namespace lca
