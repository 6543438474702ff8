// The paged 4-bit cache around its attention: the quantising write, reading rows back and the online condensation of a group.  The
// format is described in fp4_common.cuh and lca.h.
#include "fp4_common.cuh"
#include "paged_update.cuh"

namespace lca {

// ------------------------------------------------------------------------------------------------- write, read back
// Rows do not depend on one another (the exponent is the row's own), so there are no runs and no order to keep: a lane takes eight
// values (16 bytes in, 4 out), four lanes a block.  Before HBM the integer instructions bound a write (74 % of their peak with a
// row at a time and idle lanes), so that a warp takes vectors as they lie in the input, whatever rows they belong to, and no lane is idle: MLA four rows
// at a time, their rope keys in one step of 32 lanes; GQA eight vectors of one KV head each.
struct Paged4Rows {
  bf16* sem; bf16* pos;                                      // [n_rows, Hkv, d]: in (write), out (read)
  const int32_t* slots;
  uint32_t* pages_sem; uint32_t* pages_pos; uint8_t* shift_sem; uint8_t* shift_pos; uint8_t* exp_sem; uint8_t* exp_pos;
  long long n_rows, n_slots;
  int Hkv, page_log2;
  uint32_t by_Hkv;                                           // 2^32 / Hkv, rounded up: quotients of numbers below 2^16
};
// Row of the pool for slot s and KV head hk.
__device__ __forceinline__ size_t pool_row(const Paged4Rows& a, int s, int hk) {
  return (((size_t)(s >> a.page_log2) * a.Hkv + hk) << a.page_log2) + (size_t)(s & ((1 << a.page_log2) - 1));
}
// Largest |x| of eight bf16 values as bf16 bits: above 0x7f80 with a NaN among them.
__device__ __forceinline__ uint32_t top8(const uint4& v) {
  uint32_t m, n;
  asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(v.x), "r"(v.y));
  asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(n) : "r"(v.z), "r"(v.w));
  asm("max.NaN.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(n));
  return max(m & 0x7fffu, (m >> 16) & 0x7fffu);
}
// The same of the finite ones among them.
__device__ __noinline__ uint32_t finite_top8(uint4 v) {
  const uint32_t u[4] = {v.x, v.y, v.z, v.w};
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t lo = u[k] & 0x7fffu, hi = (u[k] >> 16) & 0x7fffu;
    top = max(top, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
  }
  return top;
}
// Tops of N vectors a lane, over each block's four lanes; nan: bit q where a block of vector q has one.
template <int N>
__device__ __forceinline__ uint32_t block_tops(const uint4 (&v)[N], uint32_t (&top)[N]) {
  uint32_t all = 0, nan = 0;
#pragma unroll
  for (int q = 0; q < N; ++q) { top[q] = top8(v[q]); all = max(all, top[q]); }
  if (__any_sync(0xffffffffu, all >= 0x7f80u)) {             // infinities and NaN do not count
#pragma unroll
    for (int q = 0; q < N; ++q) {
      const unsigned b = __ballot_sync(0xffffffffu, top[q] > 0x7f80u);
      nan |= (b >> (threadIdx.x & 28)) & 15u ? 1u << q : 0u;
      if (top[q] >= 0x7f80u) top[q] = finite_top8(v[q]);
    }
  }
#pragma unroll
  for (int q = 0; q < N; ++q) {
    top[q] = max(top[q], __shfl_xor_sync(0xffffffffu, top[q], 1));
    top[q] = max(top[q], __shfl_xor_sync(0xffffffffu, top[q], 2));
  }
  return nan;
}
// One vector of a row with exponent E: its codes, and the shift of its block with that of the next block above it.
__device__ __forceinline__ uint32_t encode8(const uint4& v, uint32_t top, bool nan, int E, uint32_t& shifts) {
  const int shift = min(E - paged4_block_exponent(top), PAGED4_MAX_SHIFT);
  const uint32_t s = nan ? (uint32_t)PAGED4_NAN_SHIFT : (uint32_t)shift;
  shifts = s | __shfl_down_sync(0xffffffffu, s, 4) << 4;
  return paged4_pack(v, exp2_int(shift - E));
}

static const int ROW_THREADS = 256, ROW_WARPS = ROW_THREADS / 32;
// Up to here a warp takes one MLA row (128 + 64: two), for its fewer instructions; beyond, four, for their smaller number in all.  One row a warp
// and four, us: 512 + 64 written, 256 rows 1.7 / 2.4, 2048 rows 2.1 / 2.7, 4096 rows 3.2 / 2.9, 4800 rows 3.1 / 3.4, 8192 rows 4.1 / 4.5, 9600 rows 4.8 / 4.6,
// 20000 rows 8.2 / 6.8, 323584 rows 132 / 83; read back 1.7 / 2.1, 2.0 / 2.3, 2.7 / 2.3, 2.8 / 3.0, 3.6 / 3.8, 3.9 / 3.9, 6.5 / 5.6.  Two rows and four, 128 + 64
// written, 256 rows 1.5 / 1.7, 4096 rows 2.4 / 2.2, 8192 rows 2.9 / 2.4, 20000 rows 4.3 / 3.9; read back 1.5 / 1.5, 2.0 / 1.8, 2.7 / 2.0, 3.6 / 3.2.  Between
// 3000 and 9600 rows neither is ahead by more than 0.5 us, and which one is changes with the waves that the rows make.
static const long long FEW_ROWS = 4096;

// MLA, ROWS rows: step q < S takes units 32 q + lane of their latents (US of a row), step S units lane % 8 of their keys.
template <int D_SEM, int ROWS>
struct MlaRows {
  static constexpr int US = D_SEM / 8, S = ROWS * US / 32;
  static __device__ __forceinline__ int row(int q, int lane) { return q == S ? lane >> 3 : US == 64 ? q / 2 : 2 * q + (lane >> 4); }
  static __device__ __forceinline__ int unit(int q, int lane) { return q == S ? lane & 7 : US == 64 ? (q & 1) * 32 + lane : lane & 15; }
};
template <int D_SEM, int ROWS>
__global__ void __launch_bounds__(ROW_THREADS) paged4_write_mla_kernel(Paged4Rows a) {
  using M = MlaRows<D_SEM, ROWS>;
  constexpr int S = M::S;
  const int lane = threadIdx.x & 31;
  const long long warps = (long long)gridDim.x * ROW_WARPS, groups = (a.n_rows + ROWS - 1) / ROWS;
  chain_wait();
  chain_next();
  for (long long g = (long long)blockIdx.x * ROW_WARPS + (threadIdx.x >> 5); g < groups; g += warps) {
    const int left = (int)min(a.n_rows - ROWS * g, (long long)ROWS);
    int slot = lane < left ? a.slots[ROWS * g + lane] : -1;  // lane r < ROWS: of row r
    if (slot >= a.n_slots) slot = -1;
    uint4 v[S + 1];
#pragma unroll
    for (int q = 0; q <= S; ++q) {
      const uint4* src = q == S ? reinterpret_cast<const uint4*>(a.pos) + g * (8 * ROWS) + lane : reinterpret_cast<const uint4*>(a.sem) + g * (ROWS * M::US) + 32 * q + lane;
      v[q] = M::row(q, lane) < left ? __ldcs(src) : make_uint4(0u, 0u, 0u, 0u);
    }
    uint32_t top[S + 1];
    const uint32_t nan = block_tops(v, top);
    // exponents of the rows: E[r], and of the key's row in this lane
    const uint32_t key = max(top[S], __shfl_xor_sync(0xffffffffu, top[S], 4));
    int E[S], Ek;
    if constexpr (M::US == 64) {
      int e[ROWS];
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        const uint32_t t = __reduce_max_sync(0xffffffffu, max(max(top[2 * r], top[2 * r + 1]), (lane >> 3) == r ? key : 0u));
        e[r] = max(paged4_block_exponent(t), PAGED4_MIN_EXP);
        E[2 * r] = E[2 * r + 1] = e[r];
      }
      Ek = e[0];
#pragma unroll
      for (int r = 1; r < ROWS; ++r) Ek = (lane >> 3) == r ? e[r] : Ek;
    } else {
      uint32_t t[S];
#pragma unroll
      for (int q = 0; q < S; ++q) {
        t[q] = max(top[q], __shfl_xor_sync(0xffffffffu, top[q], 4));
        t[q] = max(t[q], __shfl_xor_sync(0xffffffffu, t[q], 8));
        t[q] = max(t[q], __shfl_sync(0xffffffffu, key, 8 * M::row(q, lane)));
        E[q] = max(paged4_block_exponent(t[q]), PAGED4_MIN_EXP);
      }
#pragma unroll
      for (int q = 0; q < S; ++q) { const int e = __shfl_sync(0xffffffffu, E[q], (lane & 8) * 2); Ek = (lane >> 4) == q || q == 0 ? e : Ek; }
    }
#pragma unroll
    for (int q = 0; q <= S; ++q) {
      uint32_t shifts;
      const int Eq = q < S ? E[q < S ? q : 0] : Ek, u = M::unit(q, lane);
      const uint32_t w = encode8(v[q], top[q], (nan >> q) & 1u, Eq, shifts);
      const int to = __shfl_sync(0xffffffffu, slot, M::row(q, lane));      // (-1 behind the last row)
      if (to < 0) continue;                                  // (a slot is its row in the pool: there is one KV head)
      if (q < S) {
        a.pages_sem[(size_t)to * M::US + u] = w;
        if ((lane & 7) == 0) a.shift_sem[(size_t)to * (D_SEM / 64) + u / 8] = (uint8_t)shifts;
      } else {
        a.pages_pos[(size_t)to * 8 + u] = w;
        if ((lane & 7) == 0) { a.shift_pos[to] = (uint8_t)shifts; a.exp_sem[to] = (uint8_t)(Eq + PAGED4_EXP_BIAS); }
      }
    }
  }
}

// GQA: eight vectors of one row and KV head each, in the order of the input (blockIdx.y: keys or values), D / 8 lanes a vector.
template <int D>
struct GqaRows {
  static constexpr int U = D / 8, HEADS = 32 / U, STEPS = 8 / HEADS;         // lanes of a vector; vectors of a step; steps
};
// Where a warp stands in the input: KV head `rem` of row `row`.
struct GqaWalk {
  long long row, rows_on;
  int rem, rem_on;
  __device__ __forceinline__ GqaWalk(const Paged4Rows& a) {
    const long long first = 8 * ((long long)blockIdx.x * ROW_WARPS + (threadIdx.x >> 5)), on = 8ll * gridDim.x * ROW_WARPS;
    row = first / a.Hkv; rem = (int)(first - row * a.Hkv);
    rows_on = on / a.Hkv; rem_on = (int)(on - rows_on * a.Hkv);
  }
  __device__ __forceinline__ void next(int Hkv) {
    row += rows_on; rem += rem_on;
    if (rem >= Hkv) { rem -= Hkv; ++row; }
  }
  // row and head `ahead` vectors on
  __device__ __forceinline__ long long at(const Paged4Rows& a, int ahead, int& hk) const {
    const uint32_t j = (uint32_t)(rem + ahead), d = a.Hkv == 1 ? j : __umulhi(j, a.by_Hkv);
    hk = (int)(j - d * (uint32_t)a.Hkv);
    return row + d;
  }
};
template <int D>
__global__ void __launch_bounds__(ROW_THREADS) paged4_write_gqa_kernel(Paged4Rows a) {
  using G = GqaRows<D>;
  const bool pos = blockIdx.y & 1;
  const int lane = threadIdx.x & 31, u = lane % G::U;
  const uint4* src = reinterpret_cast<const uint4*>(pos ? a.pos : a.sem) + lane;
  uint32_t* pages = (pos ? a.pages_pos : a.pages_sem) + u;
  uint8_t* shifts = (pos ? a.shift_pos : a.shift_sem) + u / 8;
  uint8_t* exps = pos ? a.exp_pos : a.exp_sem;
  chain_wait();
  chain_next();
  for (GqaWalk at(a); at.row < a.n_rows; at.next(a.Hkv)) {
    const uint4* here = src + ((size_t)at.row * a.Hkv + at.rem) * G::U;
    uint4 v[G::STEPS];
    long long to[G::STEPS];                                  // row of the pool, or none
#pragma unroll
    for (int k = 0; k < G::STEPS; ++k) {
      int hk;
      const long long i = at.at(a, k * G::HEADS + lane / G::U, hk);
      const bool in = i < a.n_rows;
      v[k] = in ? __ldcs(here + k * 32) : make_uint4(0u, 0u, 0u, 0u);
      const int slot = in ? a.slots[i] : -1;
      to[k] = slot >= 0 && slot < a.n_slots ? (long long)pool_row(a, slot, hk) : -1ll;
    }
    uint32_t top[G::STEPS];
    const uint32_t nan = block_tops(v, top);
#pragma unroll
    for (int k = 0; k < G::STEPS; ++k) {
      uint32_t all = max(top[k], __shfl_xor_sync(0xffffffffu, top[k], 4)), s;
      if (G::U == 16) all = max(all, __shfl_xor_sync(0xffffffffu, all, 8));
      const int E = max(paged4_block_exponent(all), PAGED4_MIN_EXP);
      const uint32_t w = encode8(v[k], top[k], (nan >> k) & 1u, E, s);
      if (to[k] < 0) continue;
      pages[to[k] * G::U] = w;
      if (u % 8 == 0) shifts[to[k] * (D / 64)] = (uint8_t)s;
      if (u == 0) exps[to[k]] = (uint8_t)(E + PAGED4_EXP_BIAS);
    }
  }
}

template <int D_SEM, int ROWS>
__global__ void __launch_bounds__(ROW_THREADS) paged4_read_mla_kernel(Paged4Rows a) {
  using M = MlaRows<D_SEM, ROWS>;
  constexpr int S = M::S;
  const int lane = threadIdx.x & 31;
  const long long warps = (long long)gridDim.x * ROW_WARPS, groups = (a.n_rows + ROWS - 1) / ROWS;
  chain_wait();
  chain_next();
  for (long long g = (long long)blockIdx.x * ROW_WARPS + (threadIdx.x >> 5); g < groups; g += warps) {
    const int left = (int)min(a.n_rows - ROWS * g, (long long)ROWS);
    int slot = lane < left ? a.slots[ROWS * g + lane] : -1;
    if (slot >= a.n_slots) slot = -1;
    uint32_t w[S + 1];
    int s[S + 1], e[S + 1], from[S + 1];
#pragma unroll
    for (int q = 0; q <= S; ++q) {
      const int u = M::unit(q, lane);
      from[q] = __shfl_sync(0xffffffffu, slot, M::row(q, lane));
      const size_t row = (size_t)max(from[q], 0);            // (of slot 0 where there is none: not written)
      w[q] = __ldcs(q < S ? a.pages_sem + row * M::US + u : a.pages_pos + row * 8 + u);
      s[q] = q < S ? a.shift_sem[row * (D_SEM / 64) + u / 8] : a.shift_pos[row];
      e[q] = a.exp_sem[row];
    }
#pragma unroll
    for (int q = 0; q <= S; ++q) {
      if (from[q] < 0) continue;
      uint4* dst = q == S ? reinterpret_cast<uint4*>(a.pos) + g * (8 * ROWS) + lane : reinterpret_cast<uint4*>(a.sem) + g * (ROWS * M::US) + 32 * q + lane;
      __stcs(dst, paged4_unpack(w[q], paged4_scale(e[q], s[q] >> (M::unit(q, lane) & 4) & 15)));
    }
  }
}

template <int D>
__global__ void __launch_bounds__(ROW_THREADS) paged4_read_gqa_kernel(Paged4Rows a) {
  using G = GqaRows<D>;
  const bool pos = blockIdx.y & 1;
  const int lane = threadIdx.x & 31, u = lane % G::U;
  uint4* dst = reinterpret_cast<uint4*>(pos ? a.pos : a.sem) + lane;
  const uint32_t* pages = (pos ? a.pages_pos : a.pages_sem) + u;
  const uint8_t* shifts = (pos ? a.shift_pos : a.shift_sem) + u / 8;
  const uint8_t* exps = pos ? a.exp_pos : a.exp_sem;
  chain_wait();
  chain_next();
  for (GqaWalk at(a); at.row < a.n_rows; at.next(a.Hkv)) {
    uint4* here = dst + ((size_t)at.row * a.Hkv + at.rem) * G::U;
    long long from[G::STEPS];
    uint32_t w[G::STEPS];
    int s[G::STEPS], e[G::STEPS];
#pragma unroll
    for (int k = 0; k < G::STEPS; ++k) {
      int hk;
      const long long i = at.at(a, k * G::HEADS + lane / G::U, hk);
      const int slot = i < a.n_rows ? a.slots[i] : -1;
      from[k] = slot >= 0 && slot < a.n_slots ? (long long)pool_row(a, slot, hk) : -1ll;
    }
#pragma unroll
    for (int k = 0; k < G::STEPS; ++k) {
      const bool in = from[k] >= 0;
      w[k] = in ? __ldcs(pages + from[k] * G::U) : 0u;
      s[k] = in ? shifts[from[k] * (D / 64)] : 0;
      e[k] = in ? exps[from[k]] : 0;
    }
#pragma unroll
    for (int k = 0; k < G::STEPS; ++k)
      if (from[k] >= 0) __stcs(here + k * 32, paged4_unpack(w[k], paged4_scale(e[k], s[k] >> (u & 4) & 15)));
  }
}

// The same where Hkv is a multiple of eight: a warp takes eight KV heads of a row (blockIdx.y: the two parts, then groups of heads), one look-up
// and one step through the pool for all (29000 rows of 8 KV heads of 128: written 34 us, one by one 41; read 26 and 30.  2 KV heads,
// 100000 rows, a warp a row: 99 and 40; one by one 35 and 27).
template <int D>
__global__ void __launch_bounds__(ROW_THREADS) paged4_write_gqa8_kernel(Paged4Rows a) {
  using G = GqaRows<D>;
  const bool pos = blockIdx.y & 1;
  const int lane = threadIdx.x & 31, u = lane % G::U, hk = (int)(blockIdx.y >> 1) * 8 + lane / G::U;
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
    for (int k = 0; k < G::STEPS; ++k) v[k] = __ldcs(row_src + k * 32);
    const size_t row0 = pool_row(a, slot, hk);
    uint32_t* to = pages + row0 * G::U;
    uint8_t* to_shift = shifts + row0 * (D / 64);
    uint8_t* to_exp = exps + row0;
    uint32_t top[G::STEPS];
    const uint32_t nan = block_tops(v, top);
#pragma unroll
    for (int k = 0; k < G::STEPS; ++k) {
      uint32_t all = max(top[k], __shfl_xor_sync(0xffffffffu, top[k], 4)), s;
      if (G::U == 16) all = max(all, __shfl_xor_sync(0xffffffffu, all, 8));
      const int E = max(paged4_block_exponent(all), PAGED4_MIN_EXP);
      *to = encode8(v[k], top[k], (nan >> k) & 1u, E, s);
      if (u % 8 == 0) *to_shift = (uint8_t)s;
      if (u == 0) *to_exp = (uint8_t)(E + PAGED4_EXP_BIAS);
      to += (size_t)apart * G::U; to_shift += (size_t)apart * (D / 64); to_exp += apart;
    }
  }
}

template <int D>
__global__ void __launch_bounds__(ROW_THREADS) paged4_read_gqa8_kernel(Paged4Rows a) {
  using G = GqaRows<D>;
  const bool pos = blockIdx.y & 1;
  const int lane = threadIdx.x & 31, u = lane % G::U, hk = (int)(blockIdx.y >> 1) * 8 + lane / G::U;
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
      w[k] = __ldcs(from);
      s[k] = *from_shift;
      e[k] = *from_exp;
      from += (size_t)apart * G::U; from_shift += (size_t)apart * (D / 64); from_exp += apart;
    }
    uint4* row_dst = dst + (size_t)i * a.Hkv * G::U;
#pragma unroll
    for (int k = 0; k < G::STEPS; ++k)
      __stcs(row_dst + k * 32, paged4_unpack(w[k], paged4_scale(e[k], s[k] >> (u & 4) & 15)));
  }
}

int paged4_rows_launch(const lca_params* p, const lca_paged4* c, bool write, const void* rows_sem, const void* rows_pos,
                       const int32_t* slot_map, long long n_rows, cudaStream_t stream) {
  const bool mla = p->variant == LCA_VARIANT_MLA;
  Paged4Rows a = {(bf16*)rows_sem, (bf16*)rows_pos, slot_map, (uint32_t*)c->pages_sem, (uint32_t*)c->pages_pos, c->shift_sem, c->shift_pos,
                  c->exp_sem, c->exp_pos, n_rows, (long long)c->n_pages * c->page_size, p->n_kv_heads,
                  c->page_size == 16 ? 4 : c->page_size == 32 ? 5 : c->page_size == 64 ? 6 : 7,
                  (uint32_t)(((1ull << 32) + p->n_kv_heads - 1) / p->n_kv_heads)};
  if (p->n_kv_heads >= 1 << 15) return LCA_ERR_UNSUPPORTED_SHAPE;      // by_Hkv
  // A few waves of all CTAs that are resident, a warp the least that it can take ...
  const bool eight = p->n_kv_heads % 8 == 0, few = n_rows <= FEW_ROWS;
  const long long most = 148 * 8 * 8;
  const int mla_rows = few ? (p->d_sem == 512 ? 1 : 2) : 4;
  const long long items = mla ? (n_rows + mla_rows - 1) / mla_rows : eight ? n_rows : (n_rows * p->n_kv_heads + 7) / 8;
  const long long want = (items + ROW_WARPS - 1) / ROW_WARPS;
  const dim3 grid((unsigned)(want < most ? want : most), mla ? 1 : eight ? (unsigned)(p->n_kv_heads / 4) : 2);
  auto go = [&](auto kern) { return launch_chained(kern, grid, ROW_THREADS, 0, stream, 1, a); };
  if (mla) {
    if (p->d_sem == 512) {
      if (few) return write ? go(paged4_write_mla_kernel<512, 1>) : go(paged4_read_mla_kernel<512, 1>);
      return write ? go(paged4_write_mla_kernel<512, 4>) : go(paged4_read_mla_kernel<512, 4>);
    }
    if (few) return write ? go(paged4_write_mla_kernel<128, 2>) : go(paged4_read_mla_kernel<128, 2>);
    return write ? go(paged4_write_mla_kernel<128, 4>) : go(paged4_read_mla_kernel<128, 4>);
  }
  if (eight) {
    if (p->d_sem == 128) return write ? go(paged4_write_gqa8_kernel<128>) : go(paged4_read_gqa8_kernel<128>);
    return write ? go(paged4_write_gqa8_kernel<64>) : go(paged4_read_gqa8_kernel<64>);
  }
  if (p->d_sem == 128) return write ? go(paged4_write_gqa_kernel<128>) : go(paged4_read_gqa_kernel<128>);
  return write ? go(paged4_write_gqa_kernel<64>) : go(paged4_read_gqa_kernel<64>);
}

// ------------------------------------------------------------------------------------------------------------ update
int paged4_update_launch(const lca_params* p, const lca_paged4* c, const float* qbar_f, const double* qbar_d, const int32_t* n_rep,
                         const int32_t* n_tok, int32_t* n_rep_new, void* rep_sem, void* rep_pos, int32_t* anchor_out,
                         cudaStream_t stream) {
  const PagedRows4 rows = {(const uint8_t*)c->pages_sem, (const uint8_t*)c->pages_pos, c->shift_sem, c->shift_pos, c->exp_sem, c->exp_pos};
  return paged_update_shapes(p, c, rows, qbar_f, qbar_d, n_rep, n_tok, n_rep_new, rep_sem, rep_pos, anchor_out, stream);
}

}  // namespace lca
