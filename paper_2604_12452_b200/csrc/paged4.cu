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
// Largest finite |x| of eight bf16 values as bf16 bits; nan: whether one of them is NaN.  Every lane of the warp calls it.
__device__ __forceinline__ uint32_t top8(const uint4& v, bool& nan) {
  const uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
  uint32_t top = max(m & 0xffffu, m >> 16);
  nan = top > 0x7f80u;
  if (__any_sync(0xffffffffu, top >= 0x7f80u)) {
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
      const uint32_t w = paged4_pack(v[q], exp2_int(shift - E));
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

// GQA: a warp takes a row's keys or values, up to eight KV heads of them (blockIdx.y: the two parts, then groups of heads), D / 8 lanes
// a vector and a KV head.  All its loads are under way before the first is used; heads lie a page's rows apart in the pool.
template <int D>
struct GqaRow {
  static constexpr int U = D / 8, HEADS = 32 / U, STEPS = 8 / HEADS;         // lanes of a vector; KV heads of a step; steps
};
template <int D>
__global__ void __launch_bounds__(ROW_THREADS) paged4_write_gqa_kernel(Paged4Rows a) {
  using G = GqaRow<D>;
  const bool pos = blockIdx.y & 1;
  const int lane = threadIdx.x & 31, u = lane % G::U, hk = (int)(blockIdx.y >> 1) * 8 + lane / G::U, left = a.Hkv - hk;
  const uint4* src = reinterpret_cast<const uint4*>(pos ? a.pos : a.sem) + (size_t)(hk - lane / G::U) * G::U + lane;
  uint32_t* pages = (pos ? a.pages_pos : a.pages_sem) + u;
  uint8_t* shifts = (pos ? a.shift_pos : a.shift_sem) + u / 8;
  uint8_t* exps = pos ? a.exp_pos : a.exp_sem;
  const long long warps = (long long)gridDim.x * ROW_WARPS;
  const int apart = G::HEADS << a.page_log2;                 // rows of the pool from one step's head to the next one's
  chain_wait();
  chain_next();
  for (long long i = (long long)blockIdx.x * ROW_WARPS + (threadIdx.x >> 5); i < a.n_rows; i += warps) {
    const int slot = a.slots[i];
    if (slot < 0 || slot >= a.n_slots) continue;
    const uint4* row_src = src + (size_t)i * a.Hkv * G::U;
    uint4 v[G::STEPS];
#pragma unroll
    for (int k = 0; k < G::STEPS; ++k) v[k] = k * G::HEADS < left ? __ldcs(row_src + k * 32) : make_uint4(0u, 0u, 0u, 0u);
    const size_t row0 = pool_row(a, slot, hk);
    uint32_t* to = pages + row0 * G::U;
    uint8_t* to_shift = shifts + row0 * (D / 64);
    uint8_t* to_exp = exps + row0;
#pragma unroll
    for (int k = 0; k < G::STEPS; ++k) {
      bool n;
      uint32_t top = top8(v[k], n);
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      uint32_t all = max(top, __shfl_xor_sync(0xffffffffu, top, 4));
      if (G::U == 16) all = max(all, __shfl_xor_sync(0xffffffffu, all, 8));
      const int E = max(paged4_block_exponent(all), PAGED4_MIN_EXP);
      const int shift = min(E - paged4_block_exponent(top), PAGED4_MAX_SHIFT);
      const int s = (__ballot_sync(0xffffffffu, n) >> (lane & ~3)) & 15u ? PAGED4_NAN_SHIFT : shift;
      const uint32_t w = paged4_pack(v[k], exp2_int(shift - E));
      const int next = __shfl_down_sync(0xffffffffu, s, 4);
      if (k * G::HEADS < left) {
        *to = w;
        if (u % 8 == 0) *to_shift = (uint8_t)(s | next << 4);
        if (u == 0) *to_exp = (uint8_t)(E + PAGED4_EXP_BIAS);
      }
      to += (size_t)apart * G::U; to_shift += (size_t)apart * (D / 64); to_exp += apart;
    }
  }
}

template <int D_SEM>
__global__ void __launch_bounds__(ROW_THREADS) paged4_read_mla_kernel(Paged4Rows a) {
  constexpr int D_POS = 64, NS = D_SEM / 256 > 0 ? D_SEM / 256 : 1, US = D_SEM / 8;
  const int lane = threadIdx.x & 31;
  const long long warps = (long long)gridDim.x * ROW_WARPS;
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
    const int e = a.exp_sem[row];
#pragma unroll
    for (int q = 0; q < NS; ++q)
      if (lane + 32 * q < US) __stcs(reinterpret_cast<uint4*>(a.sem + (size_t)i * D_SEM) + lane + 32 * q, paged4_unpack(w[q], paged4_scale(e, s[q])));
    if (lane < D_POS / 8) __stcs(reinterpret_cast<uint4*>(a.pos + (size_t)i * D_POS) + lane, paged4_unpack(w[NS], paged4_scale(e, s[NS])));
  }
}

template <int D>
__global__ void __launch_bounds__(ROW_THREADS) paged4_read_gqa_kernel(Paged4Rows a) {
  using G = GqaRow<D>;
  const bool pos = blockIdx.y & 1;
  const int lane = threadIdx.x & 31, u = lane % G::U, hk = (int)(blockIdx.y >> 1) * 8 + lane / G::U, left = a.Hkv - hk;
  uint4* dst = reinterpret_cast<uint4*>(pos ? a.pos : a.sem) + (size_t)(hk - lane / G::U) * G::U + lane;
  const uint32_t* pages = (pos ? a.pages_pos : a.pages_sem) + u;
  const uint8_t* shifts = (pos ? a.shift_pos : a.shift_sem) + u / 8;
  const uint8_t* exps = pos ? a.exp_pos : a.exp_sem;
  const long long warps = (long long)gridDim.x * ROW_WARPS;
  const int apart = G::HEADS << a.page_log2;
  chain_wait();
  chain_next();
  for (long long i = (long long)blockIdx.x * ROW_WARPS + (threadIdx.x >> 5); i < a.n_rows; i += warps) {
    const int slot = a.slots[i];
    if (slot < 0 || slot >= a.n_slots) continue;
    const size_t row0 = pool_row(a, slot, hk);
    const uint32_t* from = pages + row0 * G::U;
    const uint8_t* from_shift = shifts + row0 * (D / 64);
    const uint8_t* from_exp = exps + row0;
    uint32_t w[G::STEPS];
    int s[G::STEPS], e[G::STEPS];
#pragma unroll
    for (int k = 0; k < G::STEPS; ++k) {
      const bool in = k * G::HEADS < left;
      w[k] = in ? __ldcs(from) : 0u;
      s[k] = in ? *from_shift : 0;
      e[k] = in ? *from_exp : 0;
      from += (size_t)apart * G::U; from_shift += (size_t)apart * (D / 64); from_exp += apart;
    }
    uint4* row_dst = dst + (size_t)i * a.Hkv * G::U;
#pragma unroll
    for (int k = 0; k < G::STEPS; ++k)
      if (k * G::HEADS < left) __stcs(row_dst + k * 32, paged4_unpack(w[k], paged4_scale(e[k], s[k] >> (u & 4) & 15)));
  }
}

int paged4_rows_launch(const lca_params* p, const lca_paged4* c, bool write, const void* rows_sem, const void* rows_pos,
                       const int32_t* slot_map, long long n_rows, cudaStream_t stream) {
  const bool mla = p->variant == LCA_VARIANT_MLA;
  Paged4Rows a = {(bf16*)rows_sem, (bf16*)rows_pos, slot_map, (uint32_t*)c->pages_sem, (uint32_t*)c->pages_pos, c->shift_sem, c->shift_pos,
                  c->exp_sem, c->exp_pos, n_rows, (long long)c->n_pages * c->page_size, p->n_kv_heads,
                  c->page_size == 16 ? 4 : c->page_size == 32 ? 5 : c->page_size == 64 ? 6 : 7};
  const long long most = 148 * 8 * 8;                        // a few waves of all CTAs that are resident
  if (mla) {
    const long long want = (n_rows + ROW_WARPS - 1) / ROW_WARPS;
    const dim3 grid((unsigned)(want < most ? want : most), 1);
    auto kern = write ? (p->d_sem == 512 ? paged4_write_mla_kernel<512> : paged4_write_mla_kernel<128>)
                      : (p->d_sem == 512 ? paged4_read_mla_kernel<512> : paged4_read_mla_kernel<128>);
    return launch_chained(kern, grid, ROW_THREADS, 0, stream, 1, a);
  }
  const long long want = (n_rows + ROW_WARPS - 1) / ROW_WARPS, parts = 2 * ((p->n_kv_heads + 7) / 8);
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
