// Decode attention over the paged 4-bit cache for the MLA shape and many heads, on CTA pairs.  The mathematics is that of attn_paged4.cu; the
// weights are those of attn_paged8_pair.cu (first term e5m2, both in the same columns of O; its comment has the errors), and so are
// the products: cta_group::2, 128 query rows on two SMs, each CTA holds 64 rows of Q and P, half of the keys of a tile for S = Q K^T
// and half of the value columns for O += T V.
//
// What a block of 32 query rows on one CTA pays for a tile (attn_paged4.cu) is its expansion, 72 K values for 32 rows.  Here a CTA
// expands its own 64 keys only, 36 K values for 64 rows.  The values of the keys are the same codes: the 64 x 128 bytes of a
// latent chunk are, swizzle included, one half of the 128 x 128 bytes of the value chunk that the product reads, in the CTA that
// has those columns.  So they go there as they are by bulk copies of 8 KB from shared memory to shared memory, two within the CTA and two
// to the other one, on the reader's barrier.
//   softmax    8 warps: thread = row and a quarter of the keys (TMEM lane = row and half of them)
//   expansion  8 warps: packed rows from HBM to registers one tile ahead, to e4m3 in the operand's image
//   a warp each for products (even CTA; odd CTA: forwarding of its weights and queries), page table and exponents, copies, forwarding of
//   expanded keys and copied values
// An expanded tile's buffer is free once its product and the copies from it, at both ends, are done.  Signals from one CTA to the
// other go through one thread, as in attn_paged8_pair.cu.
// 64 x 5056 rows, 128 heads: 125 us (blocks of 32 rows on single CTAs: 228; the 8-bit cache, which expands nothing: 92).  A tile takes 5700
// clocks: S 2000 and O 1100 (36 x 32 + 16 x 64 if nothing else used the port of shared memory), between them the softmax's
// chain of 4400, which waits for neither.  Its instructions once did not fit the instruction cache (39 % of the stalls, products issued by
// unrolled code, keys and values expanded by warps of their own).  Values expanded a second time in place of the copies: 154 us;
// sixteen softmax warps with half the keys each: 131; maxima raised by a bound of 2^11 in place of 2^12, by all warps: 128.
#include <cstring>

#include "attn_paged4.cuh"
#include "attn_paged_pair.cuh"

namespace lca {
using namespace tc;

static __device__ int g_paged4_pair_status = 0;

namespace p4pair {
constexpr int ROWS = 128, DS = 512, DP = 64;
constexpr int SW = 8, EW = 8, W_EXP = SW, W_MMA = W_EXP + EW, W_LOOK = W_MMA + 1, W_COPY = W_LOOK + 1, W_FWD = W_COPY + 1, THREADS = 32 * (W_FWD + 1);
constexpr int Q_TERM = 4 * 64 * 128 + 64 * 64;               // 36 KB: four latent chunks and the rope chunk of 64 rows
constexpr int K_CHUNK = 64 * 128, K_BUF = 4 * K_CHUNK + 64 * 64;      // the same of 64 keys
constexpr int V_CHUNK = 128 * 128, V_BUF = 2 * V_CHUNK;      // 128 keys x 128 columns, twice
constexpr int P_TERM = 64 * 128;
constexpr int OFF_Q = 0, OFF_K = 2 * Q_TERM, OFF_V = OFF_K + 2 * K_BUF, OFF_P = OFF_V + 2 * V_BUF, OFF_MISC = OFF_P + 2 * P_TERM;
constexpr int FACTS = 4;
// Facts of a tile: factors of its rows as bf16, per 16 rows h (below) and the group of rows in the pool, what is present
constexpr int F_H = 256, F_GROUP = F_H + 32, F_SPAN = F_GROUP + 32, FACT = F_SPAN + 16;
constexpr int OFF_BAR = OFF_MISC, OFF_SCALAR = OFF_BAR + 224, OFF_TABLE = OFF_SCALAR + 32, OFF_QS = OFF_TABLE + 128, OFF_RED = OFF_QS + 64 * 4;
constexpr int OFF_FACT = OFF_RED + 256 * 4, SMEM_BYTES = OFF_FACT + FACTS * FACT;
constexpr int TM_S = 256, TM_COLS = 512;                     // O in columns 0..255, S in 256..319 and 320..383
constexpr float T_BITS = paged8_t_bits(ROWS);
constexpr float T_MAX = 12.f;                                // log2 of the largest weight: e5m2 has steps of 2^9 below, and leaves at most 2^8 of it to e4m3
static_assert(SMEM_BYTES <= 232448, "shared memory of one SM");
static_assert(OFF_FACT % 16 == 0 && FACT % 16 == 0 && OFF_TABLE % 16 == 0, "alignment");
}  // namespace p4pair

// 8 KB of shared memory to shared memory of a CTA of this cluster
__device__ __forceinline__ void smem_copy(uint32_t dst_cluster, uint32_t src, uint32_t bytes, uint32_t bar_cluster) {
  asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst_cluster), "r"(src), "r"(bytes), "r"(bar_cluster) : "memory");
}
// all softmax warps; the four of them that share 32 rows
__device__ __forceinline__ void softmax_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
__device__ __forceinline__ void rows_sync(int half) { asm volatile("bar.sync %0, 128;" ::"r"(half + 2) : "memory"); }
__device__ __forceinline__ bool rows_or(int half, bool v) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(r) : "r"((uint32_t)v), "r"(half + 2) : "memory");
  return r != 0;
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(p4pair::THREADS, 1)
attn_paged4_pair_kernel(const __grid_constant__ Paged4Params a) {
  using namespace p4pair;
  const Paged8Params& p = a.b;
  extern __shared__ __align__(1024) unsigned char smem[];
  const uint32_t base = smem_u32(smem);
  const uint32_t bars = base + OFF_BAR;
  const uint32_t QFULL = bars, PFULL = bars + 8, PVDONE = bars + 16, QLOCAL = bars + 24, PLOCAL = bars + 32;
  auto SFULL = [&](uint32_t i) { return bars + 40 + 8 * i; };
  auto KLOCAL = [&](uint32_t i) { return bars + 56 + 8 * i; };           // keys expanded, this CTA's
  auto KFULL = [&](uint32_t i) { return bars + 72 + 8 * i; };            // even CTA: both CTAs'
  auto KEMPTY = [&](uint32_t i) { return bars + 88 + 8 * i; };
  auto VFULL = [&](uint32_t i) { return bars + 104 + 8 * i; };           // values copied, this CTA's
  auto VPEER = [&](uint32_t i) { return bars + 120 + 8 * i; };           // even CTA: the odd CTA's
  auto VEMPTY = [&](uint32_t i) { return bars + 136 + 8 * i; };
  auto FFULL = [&](uint32_t i) { return bars + 152 + 8 * i; };
  auto FEMPTY = [&](uint32_t i) { return bars + 184 + 8 * i; };
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem + OFF_SCALAR);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + OFF_SCALAR + 4);
  int* s_b = reinterpret_cast<int*>(smem + OFF_SCALAR + 8);
  volatile uint32_t* s_sixteen = reinterpret_cast<volatile uint32_t*>(smem + OFF_SCALAR + 12);
  long long* s_off = reinterpret_cast<long long*>(smem + OFF_SCALAR + 16);
  uint2* s_table = reinterpret_cast<uint2*>(smem + OFF_TABLE);
  float* s_qs = reinterpret_cast<float*>(smem + OFF_QS);
  float* s_red = reinterpret_cast<float*>(smem + OFF_RED);
  unsigned char* s_fact = smem + OFF_FACT;
  long long* s_warp = reinterpret_cast<long long*>(smem + OFF_P);        // totals of the warps, and as many words; before the weights
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair_id = (int)(blockIdx.x >> 1);
  auto fail = [&](int code) { atomicCAS(&g_paged4_pair_status, 0, code); *abort_flag = 1; };

  if (threadIdx.x == 0) {
    mbar_init(QFULL, 32 * SW + 1); mbar_init(PFULL, 32 * SW + 1);        // the even CTA's threads and the odd CTA's forwarder
    mbar_init(PVDONE, 1); mbar_init(QLOCAL, 32 * SW); mbar_init(PLOCAL, 32 * SW);
    for (int i = 0; i < 2; ++i) {
      mbar_init(SFULL(i), 1); mbar_init(KLOCAL(i), EW); mbar_init(KFULL(i), 2); mbar_init(KEMPTY(i), 3);     // product, copies at both ends
      mbar_init(VFULL(i), 1); mbar_init(VPEER(i), 1); mbar_init(VEMPTY(i), 1);
    }
    for (int i = 0; i < FACTS; ++i) { mbar_init(FFULL(i), 1); mbar_init(FEMPTY(i), SW + EW); }
    *s_sixteen = 16u;
    *abort_flag = 0;
    fence_mbar_init();
    if (base & 1023u) fail(100);                             // the operands' images need it
  }
  if (warp == W_MMA) { tmem_alloc_pair(smem_u32((const void*)tmem_slot), TM_COLS); tmem_relinquish_pair(); }
  paged4_table_load(s_table, threadIdx.x);
  chain_wait();
  chain_next();                                              // the whole grid is resident: nothing is displaced
  paged8_range<THREADS>(p, pair_id, s_warp, s_b, s_off);
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                                        // both CTAs' barriers are initialised
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  Walk w;
  w.b = *s_b; w.off = s_off[0]; w.left = s_off[1]; w.fresh = true; w.n = 0;
  const uint32_t n_tiles = (uint32_t)min(s_off[1], 0x7fffffffll);

  if (warp == W_LOOK) {
    // ------------------------------------------------------------------------------------------------- look-ups
    // As in attn_paged4.cu.  Lane i < 8: the page of rows [16 i, 16 i + 16); every lane: the exponents of four rows.
    bool ok = !*abort_flag;
    int j = 0;
    bool more = w.next(p);
    struct Tile { int page, lo, mid, hi; bool any; };        // lo, mid, hi: PagedSpan from the tile's first row
    auto look = [&](Tile& y) {
      y.any = more;
      if (!more) return;
      const PagedSpan sp = w.t.s;
      const int row0 = w.t.row0(w.t0 + j), x = row0 + 16 * (lane & 7);
      y.lo = sp.n_rep - row0; y.mid = sp.tok0 - row0; y.hi = sp.n_tok - row0;
      y.page = -1;
      if (sp.any(x, 16) && (x >> p.page_log2) < p.width) y.page = p.table[(size_t)w.b * p.width + (x >> p.page_log2)];
      if (++j == w.n) { j = 0; more = w.next(p); }
    };
    auto group_of = [&](const Tile& y) {                     // the pool's group of 16 rows, ~0: none
      return y.any && (unsigned)y.page < (unsigned)p.n_pages
                 ? ((uint32_t)y.page << (p.page_log2 - 4)) + (uint32_t)(lane & ((p.page >> 4) - 1)) : ~0u;
    };
    auto exponents = [&](uint32_t group) {
      const uint32_t gr = __shfl_sync(0xffffffffu, group, lane >> 2);
      return gr == ~0u ? 0u : __ldg(reinterpret_cast<const uint32_t*>(a.exp_v) + (size_t)gr * 4 + (lane & 3));
    };
    Tile t0, t1;
    look(t0);
    look(t1);
    uint32_t g0 = group_of(t0), e0 = exponents(g0);
    uint32_t f = 0, phase = 0;
    while (ok && t0.any) {
      const uint32_t g1 = group_of(t1), e1 = exponents(g1);
      Tile t2;
      look(t2);
      const uint32_t here = __shfl_sync(0xffffffffu, g0, lane >> 2);
      uint32_t code[4];
      int most = -1000, least = 1000;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 4 * lane + i;
        const bool present = here != ~0u && (r < t0.lo || (r >= t0.mid && r < t0.hi));
        const int e = present ? paged4_log2_factor((int)(e0 >> (8 * i)) & 255) : 0;
        code[i] = (uint32_t)(e + 127) << 7;
        if (present) { most = max(most, e); least = min(least, e); }
      }
      // A weight is 2^y f, its part of the row sum 2^y: both are multiples of 2^(y + h), with h half of what is in the middle of the 16 rows'
      // log2 f, so that neither is lost below 2^-126 where the exponents of a sequence span more than fp32 does.
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) {
        most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
        least = min(least, __shfl_xor_sync(0xffffffffu, least, o));
      }
      const bool all = (__ballot_sync(0xffffffffu, g0 != ~0u) & 0xffu) == 0xffu && (t0.lo >= 128 || (t0.mid <= 0 && t0.hi >= 128));
      ok = mbar_wait(FEMPTY(f), phase ^ 1, abort_flag);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) { if (lane == 0) fail(ERR_WAIT_KV_EMPTY); break; }
      unsigned char* fact = s_fact + f * FACT;
      *reinterpret_cast<uint2*>(fact + 8 * lane) = make_uint2(code[0] | code[1] << 16, code[2] | code[3] << 16);
      if ((lane & 3) == 0) {                                 // h, and log2 t - z at most: as bf16 (integers below 2^8)
        const int h = most < least ? 0 : (most + least) >> 2, bound = most < least ? 0 : most - h + (int)T_BITS;
        reinterpret_cast<uint32_t*>(fact + F_H)[lane >> 2] = pack_bf16x2((float)h, (float)bound);
      }
      if (lane < 8) reinterpret_cast<uint32_t*>(fact + F_GROUP)[lane] = g0;
      if (lane == 8) *reinterpret_cast<int4*>(fact + F_SPAN) = make_int4(all, t0.lo, t0.mid, t0.hi);
      __syncwarp();
      if (lane == 0) mbar_arrive(FFULL(f));
      if (++f == FACTS) { f = 0; phase ^= 1; }
      t0 = t1; t1 = t2; g0 = g1; e0 = e1;
    }
  } else if (warp >= W_EXP && warp < W_MMA) {
    // ----------------------------------------------------------------------------------------------- expansion
    // Thread: row et / 4 of this CTA's 64, unit et % 4 (32 values) of each latent chunk and 16 values of the rope key.  Eight
    // neighbouring lanes write two rows, so that their units fall on all banks of the swizzled image.
    const int et = (int)threadIdx.x - 32 * W_EXP, row = et >> 2, u = et & 3, r = 64 * (int)rank + row;
    const uint32_t sixteen = *s_sixteen;
    bool ok = !*abort_flag;
    auto wait = [&](uint32_t bar, uint32_t ph, int code) {
      if (ok && !mbar_wait(bar, ph, abort_flag)) { fail(code); ok = false; }
      ok = __all_sync(0xffffffffu, ok);
      return ok;
    };
    uint4 sem[4];
    uint2 pos = make_uint2(0u, 0u), shift = pos;
    uint32_t shift_pos = 0, f = 0, fphase = 0;
#pragma unroll
    for (int c = 0; c < 4; ++c) sem[c] = make_uint4(0u, 0u, 0u, 0u);
    auto load = [&]() {
      if (!wait(FFULL(f), fphase, ERR_WAIT_KV_FULL)) return;
      const unsigned char* fact = s_fact + f * FACT;
      const int4 y = *reinterpret_cast<const int4*>(fact + F_SPAN);
      const uint32_t gr = reinterpret_cast<const uint32_t*>(fact + F_GROUP)[r >> 4];
      if (gr != ~0u && (y.x || r < y.y || (r >= y.z && r < y.w))) {
        const size_t at = (size_t)gr * 16 + (r & 15);
#pragma unroll
        for (int c = 0; c < 4; ++c) sem[c] = load_stream(a.sem + at * (DS / 2) + (4 * c + u) * 16);
        pos = __ldg(reinterpret_cast<const uint2*>(a.pos + at * (DP / 2) + 8 * u));
        shift = __ldg(reinterpret_cast<const uint2*>(a.shift_sem + at * (DS / 64)));
        shift_pos = a.shift_pos[at];
      } else {                                               // what absent rows hold is left alone
#pragma unroll
        for (int c = 0; c < 4; ++c) sem[c] = make_uint4(0u, 0u, 0u, 0u);
        pos = shift = make_uint2(0u, 0u);
        shift_pos = 0;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(FEMPTY(f));
      if (++f == FACTS) { f = 0; fphase ^= 1; }
    };
    const uint32_t sem_to = OFF_K + swz<128>(row, 2 * u), pos_to = OFF_K + 4 * K_CHUNK + swz<64>(row, u);
    if (n_tiles > 0) load();
#pragma unroll 1
    for (uint32_t t = 0; t < n_tiles && ok; ++t) {
      const uint32_t buf = t & 1, to = buf * K_BUF;
      if (t > 1 && !wait(KEMPTY(buf), ((t >> 1) - 1) & 1, ERR_WAIT_KV_EMPTY)) break;
      uint2 tab[5];                                          // block 4 c + u of the row, two shifts a byte
#pragma unroll
      for (int c = 0; c < 4; ++c) tab[c] = s_table[((c < 2 ? shift.x : shift.y) >> (16 * (c & 1) + 4 * u)) & 15];
      tab[4] = s_table[(shift_pos >> (4 * (u >> 1))) & 15];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const uint2 x0 = paged4_expand(sem[c].x, tab[c], sixteen), x1 = paged4_expand(sem[c].y, tab[c], sixteen),
                    x2 = paged4_expand(sem[c].z, tab[c], sixteen), x3 = paged4_expand(sem[c].w, tab[c], sixteen);
        *reinterpret_cast<uint4*>(smem + to + c * K_CHUNK + sem_to) = make_uint4(x0.x, x0.y, x1.x, x1.y);
        *reinterpret_cast<uint4*>(smem + to + c * K_CHUNK + (sem_to ^ 16u)) = make_uint4(x2.x, x2.y, x3.x, x3.y);
      }
      {
        const uint2 x0 = paged4_expand(pos.x, tab[4], sixteen), x1 = paged4_expand(pos.y, tab[4], sixteen);
        *reinterpret_cast<uint4*>(smem + to + pos_to) = make_uint4(x0.x, x0.y, x1.x, x1.y);
      }
      // the fence waits for loads under way too: those of the next tile come behind it
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(KLOCAL(buf));
      if (t + 1 < n_tiles) load();
    }
  } else if (warp == W_COPY) {
    // ------------------------------------------------------------------------------- keys are there: on to the values
    if (lane == 0 && !*abort_flag) {
#pragma unroll 1
      for (uint32_t t = 0; t < n_tiles; ++t) {
        const uint32_t buf = t & 1;
        if (!mbar_wait(KLOCAL(buf), (t >> 1) & 1, abort_flag)) { fail(ERR_WAIT_KV_FULL); break; }
        // (both CTAs' values of the tile before the last one have been read: one signal to both)
        if (t > 1 && !mbar_wait(VEMPTY(buf), ((t >> 1) - 1) & 1, abort_flag)) { fail(ERR_WAIT_O_DONE); break; }
        mbar_expect_tx(VFULL(buf), V_BUF);                   // two copies of this CTA and two of the other one
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {                   // the other CTA's columns first
          const uint32_t to = (i >> 1) ^ rank ^ 1u, n2 = i & 1;
          smem_copy(mapa_u32(base + OFF_V + buf * V_BUF + n2 * V_CHUNK + rank * K_CHUNK, to), base + OFF_K + buf * K_BUF + (2 * n2 + to) * K_CHUNK, K_CHUNK,
                    mapa_u32(VFULL(buf), to));
        }
      }
    }
  } else if (warp == W_FWD) {
    // ------------------------------------------- keys are there: the product may start; values are there: so it may, and a keys' buffer is free
    if (lane == 0 && !*abort_flag) {
      uint32_t k = 0, v = 0;
      long long since = clock64();
      uint32_t tries = 0;
#pragma unroll 1
      while (v < n_tiles) {
        bool idle = true;
        if (k < n_tiles && phase_done(KLOCAL(k & 1), (k >> 1) & 1)) { mbar_arrive_cluster_cta(mapa_u32(KFULL(k & 1), 0)); ++k; idle = false; }
        if (phase_done(VFULL(v & 1), (v >> 1) & 1)) {
          mbar_arrive_cluster_cta(mapa_u32(KEMPTY(v & 1), 0));
          mbar_arrive_cluster_cta(mapa_u32(KEMPTY(v & 1), 1));
          if (rank == 1) mbar_arrive_cluster_cta(mapa_u32(VPEER(v & 1), 0));
          ++v;
          idle = false;
        }
        if (!idle) { since = clock64(); tries = 0; }
        else if ((++tries & 63u) == 0 && (*abort_flag || clock64() - since > WAIT_TIMEOUT_CYCLES)) { fail(ERR_WAIT_KV_FULL); break; }
      }
    }
  } else if (warp == W_MMA && rank == 0) {
    // --------------------------------------------------------------------------------------------- MMA (even CTA)
    const uint32_t leader = elect_one();
    constexpr uint32_t ID_S = umma_idesc_f8(128, 128, 0, false, false);
    constexpr uint32_t ID_LO = umma_idesc_f8(128, 256, 0, false, true), ID_HI = ID_LO | (1u << 7);       // A: e4m3 / e5m2
    const uint64_t q_hi = desc_rows(base + OFF_Q, 128, 16), qp_hi = desc_rows(base + OFF_Q + 4 * 8192, 64, 16);
    const uint64_t k0 = desc_rows(base + OFF_K, 128, 16), kp0 = desc_rows(base + OFF_K + 4 * K_CHUNK, 64, 16);
    const uint64_t p_hi = desc_rows(base + OFF_P, 128, 16), v0 = desc_rows(base + OFF_V, 128, 16);
    uint32_t g = 0, seg = 0;
    bool ok = !*abort_flag;
    auto wait = [&](uint32_t bar, uint32_t ph, int code) {
      ok = ok && mbar_wait(bar, ph, abort_flag);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok && lane == 0) fail(code);
      return ok;
    };
    auto issue_s = [&](uint32_t t) {
      const uint32_t buf = t & 1, d = tmem + TM_S + 64 * buf, off = buf * (K_BUF / 16);
      tc_fence_after();
      // (rolled up, for the instructions of all these roles to be near: fetching them bound the kernel)
#pragma unroll 1
      for (int c = 0; c < 4; ++c)
#pragma unroll 1
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int h = 0; h < 2; ++h)
            umma_f8_pair_elected(leader, d, desc_add(q_hi, (h * Q_TERM + c * 8192 + k * 32) >> 4), desc_add(k0, off + ((c * K_CHUNK + k * 32) >> 4)), ID_S,
                                 (c > 0 || k > 0 || h > 0) ? 1u : 0u);
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) umma_f8_pair_elected(leader, d, desc_add(qp_hi, (h * Q_TERM + k * 32) >> 4), desc_add(kp0, off + 2 * k), ID_S, 1u);
      umma_commit_pair_elected(leader, KEMPTY(buf), 3);
      umma_commit_pair_elected(leader, SFULL(buf), 3);
    };
    auto issue_o = [&](uint32_t t, bool first) {
      const uint32_t buf = t & 1, off = buf * (V_BUF / 16);
      tc_fence_after();
#pragma unroll 1
      for (int n2 = 0; n2 < 2; ++n2)
#pragma unroll 1
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int h = 0; h < 2; ++h)
            umma_f8_pair_elected(leader, tmem + n2 * 128, desc_add(p_hi, (h * P_TERM + k * 32) >> 4), desc_add(v0, off + ((n2 * V_CHUNK + k * 4096) >> 4)),
                                 h ? ID_LO : ID_HI, (!first || k > 0 || h > 0) ? 1u : 0u);
      umma_commit_pair_elected(leader, VEMPTY(buf), 3);
      umma_commit_pair_elected(leader, PVDONE, 3);
    };
    while (ok && w.next(p)) {
      if (!wait(QFULL, seg & 1, ERR_WAIT_Q)) break;
      ++seg;
      tc_fence_after();
      // of the next S and the next O whichever can go first; S of a tile takes the columns of the last but one, whose S was
      // read before its weights were written and its O issued
      uint32_t js = 0, jo = 0, jv = 0;                       // jv: values that are there
      const uint32_t n = (uint32_t)w.n;
      long long since = clock64();
      uint32_t tries = 0;
#pragma unroll 1
      while (jo < n && ok) {
        bool idle = true;
        if (js < n && js < jo + 2 && __all_sync(0xffffffffu, phase_done(KFULL((g + js) & 1), ((g + js) >> 1) & 1))) { issue_s(g + js); ++js; idle = false; }
        if (jv == jo) {
          const uint32_t t = g + jv;
          if (__all_sync(0xffffffffu, phase_done(VFULL(t & 1), (t >> 1) & 1) && phase_done(VPEER(t & 1), (t >> 1) & 1))) ++jv;
        }
        if (jo < js && jo < jv && __all_sync(0xffffffffu, phase_done(PFULL, (g + jo) & 1))) { issue_o(g + jo, jo == 0); ++jo; idle = false; }
        if (!idle) { since = clock64(); tries = 0; }
        else if ((++tries & 63u) == 0 && (*abort_flag || clock64() - since > WAIT_TIMEOUT_CYCLES)) { if (lane == 0) fail(ERR_WAIT_P_FULL); ok = false; }
        ok = __all_sync(0xffffffffu, ok);
      }
      g += n;
    }
  } else if (warp == W_MMA) {
    // ------------------------------------------------------------------------ forwarding of the odd CTA's signals
    if (lane == 0 && !*abort_flag) {
      const uint32_t q_bar = mapa_u32(QFULL, 0), p_bar = mapa_u32(PFULL, 0);
      uint32_t g = 0, seg = 0;
      bool ok = true;
      while (ok && w.next(p)) {
        if (!mbar_wait(QLOCAL, seg & 1, abort_flag)) { fail(ERR_WAIT_Q); break; }
        mbar_arrive_cluster_cta(q_bar);
        ++seg;
        for (int j = 0; j < w.n; ++j, ++g) {
          if (!mbar_wait(PLOCAL, g & 1, abort_flag)) { fail(ERR_WAIT_P_FULL); ok = false; break; }
          mbar_arrive_cluster_cta(p_bar);
        }
      }
    }
  } else {
    // ---------------------------------------------------------------------------------------- softmax, epilogue
    // TMEM lane ln: row rl of this CTA, half half_no of a tile's keys / of each value chunk's columns; cg: which half of those
    const int quad = warp & 3, cg = warp >> 2, ln = quad * 32 + lane, rl = ln & 63, half_no = ln >> 6, key0 = 64 * half_no + 32 * cg;
    const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
    const uint32_t q_bar = rank == 0 ? QFULL : QLOCAL, p_bar = rank == 0 ? PFULL : PLOCAL;
    uint32_t g = 0;
    bool ok = true, first_piece = true;
    auto load_q = [&](const Walk& u) {
      const int valid = min(max(p.q_len * p.rep - u.blk * ROWS - 64 * (int)rank, 0), 64);      // rows of this CTA
#pragma unroll 2
      for (int r = warp; r < 64; r += SW) {
        const int gr = u.blk * ROWS + 64 * (int)rank + r, qt = gr / p.rep;
        const size_t row = ((size_t)u.b * p.q_len + qt) * p.Hq + (gr - qt * p.rep);
        uint4 v[3];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 3; ++i) {
          const int c = lane + 32 * i;
          v[i] = make_uint4(0u, 0u, 0u, 0u);
          if (r < valid && c < 72) v[i] = *reinterpret_cast<const uint4*>(c < 64 ? p.q_sem + row * DS + 8 * c : p.q_pos + row * DP + 8 * (c - 64));
        }
#pragma unroll
        for (int i = 0; i < 3; ++i) top = max(top, max_abs_bf16(v[i]));
        top = __reduce_max_sync(0xffffffffu, top);
        const int e = query_exponent(top);
#pragma unroll
        for (int i = 0; i < 3; ++i) {
          const int c = lane + 32 * i;
          if (c >= 72) continue;
          uint32_t hi[2], lo[2];
          split_e4m3(v[i], exp2_int(e), hi, lo);
          const uint32_t o = (c < 64 ? (c / 16) * 8192 + swz<128>(r, (c % 16) / 2) : 4 * 8192 + swz<64>(r, (c - 64) / 2)) + 8 * (c & 1);
          *reinterpret_cast<uint2*>(smem + OFF_Q + o) = make_uint2(hi[0], hi[1]);
          *reinterpret_cast<uint2*>(smem + OFF_Q + Q_TERM + o) = make_uint2(lo[0], lo[1]);
        }
        // a row with an infinity or a NaN has no finite logit
        if (lane == 0) s_qs[r] = top >= 0x7f80u ? __int_as_float(0x7fffffff) : exp2_int(-e);
      }
      fence_proxy_async_smem();
      mbar_arrive(q_bar);
      softmax_sync();
    };
    bool more = w.next(p);
    if (more) load_q(w);
    while (more) {
      const PagedSpan sp = w.t.s;
      const int gr = w.blk * ROWS + 64 * (int)rank + rl, qt = gr / p.rep;
      const bool row_valid = gr < p.q_len * p.rep;
      const int lim = sp.n_tok - p.q_len + 1 + (row_valid ? qt : 0), lim_all = sp.n_tok - p.q_len + 1;
      const float qs = row_valid ? s_qs[rl] * p.scale_log2 : 0.f;
      float m = row_valid ? 0.f : 3.0e38f, l = 0.f;          // rows behind the last one never have weight
      bool unset = row_valid;                                // no key seen yet
#pragma unroll 1
      for (int j = 0; j < w.n; ++j, ++g) {
        const int row0 = w.t.row0(w.t0 + j), x0 = row0 + key0;
        const uint32_t fr = g % FACTS;
        ok = mbar_wait(FFULL(fr), (g / FACTS) & 1, abort_flag);
        if (!ok) fail(ERR_WAIT_KV_FULL);
        __syncwarp();
        const unsigned char* fact = s_fact + fr * FACT;
        const uint2 hw = *reinterpret_cast<const uint2*>(fact + F_H + key0 / 4), groups = *reinterpret_cast<const uint2*>(fact + F_GROUP + key0 / 4);
        const float h[2] = {__uint_as_float(hw.x << 16), __uint_as_float(hw.y << 16)};
        // factors of four pairs of this thread's keys, bf16
        auto factors = [&](int i) { return *reinterpret_cast<const uint4*>(fact + 2 * key0 + 16 * i); };
        // keys this row may see and representatives, as bits; most tiles are all keys and no bias
        const bool tile_reps = row0 < sp.n_rep && p.bias_log2 != 0.f;
        const bool whole_tile = row0 + 128 <= min(sp.n_tok, lim_all) && (row0 >= sp.tok0 || row0 + 128 <= sp.n_rep);
        const bool special = !whole_tile || tile_reps || groups.x == ~0u || groups.y == ~0u;
        ok = mbar_wait(SFULL(g & 1), (g >> 1) & 1, abort_flag);
        if (!ok) fail(ERR_WAIT_S_FULL);
        __syncwarp();
        tc_fence_after();
        uint64_t z[16];                                      // log2 of e = 2^(y - m + h), in pairs of keys
        {
          uint32_t s[32];
          tmem_ld32(tmem + lane_base + TM_S + 64 * (g & 1) + 32 * cg, s);
          tmem_wait_ld();
          const uint64_t qs2 = pack_f32x2(qs, qs);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint4 kf = factors(i);
            const uint32_t f[4] = {kf.x, kf.y, kf.z, kf.w};
            const float c = h[i >> 1] - m;
#pragma unroll
            for (int k = 0; k < 4; ++k)
              z[4 * i + k] = fma_f32x2(join(s[8 * i + 2 * k], s[8 * i + 2 * k + 1]), mul_f32x2(join(f[k] << 16, f[k] & 0xffff0000u), qs2), pack_f32x2(c, c));
          }
        }
        if (special) {
          uint32_t see = (uint32_t)((low_bits(sp.n_rep - x0) | (low_bits(sp.n_tok - x0) & ~low_bits(sp.tok0 - x0))) & low_bits(lim - x0));
          const uint32_t reps = (uint32_t)low_bits(sp.n_rep - x0);
          if (groups.x == ~0u) see &= 0xffff0000u;
          if (groups.y == ~0u) see &= 0x0000ffffu;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float z0, z1;
            unpack_f32x2(z[i], z0, z1);
            z0 = (see >> (2 * i)) & 1 ? z0 + ((reps >> (2 * i)) & 1 ? p.bias_log2 : 0.f) : -INFINITY;
            z1 = (see >> (2 * i + 1)) & 1 ? z1 + ((reps >> (2 * i + 1)) & 1 ? p.bias_log2 : 0.f) : -INFINITY;
            z[i] = pack_f32x2(z0, z1);
          }
        }
        // The maximum is raised where a weight could come out too large: first a bound, with the largest factor of every 16 keys
        float top = -INFINITY;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          float most = -INFINITY;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            float z0, z1;
            unpack_f32x2(z[8 * q + i], z0, z1);
            most = max3(most, z0, z1);
          }
          top = fmaxf(top, most + __uint_as_float((q ? hw.y : hw.x) & 0xffff0000u));
        }
        float factor = 1.f;
        if (rows_or(quad & 1, unset || top > T_MAX)) {
          top = -INFINITY;                                   // largest log2 t of this row's keys
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint4 kf = factors(i);
            const uint32_t f[4] = {kf.x, kf.y, kf.z, kf.w};
            const float c = T_BITS - 127.f - h[i >> 1];      // (an exponent's bits below those of 2^23 are that many more: exact)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              float z0, z1;
              unpack_f32x2(z[4 * i + k], z0, z1);
              const float e0 = __uint_as_float(0x4b000000u | (f[k] >> 7 & 255u)) - 0x1p23f, e1 = __uint_as_float(0x4b000000u | f[k] >> 23) - 0x1p23f;
              top = max3(top, z0 + (e0 + c), z1 + (e1 + c));
            }
          }
          s_red[cg * 128 + ln] = top;
          rows_sync(quad & 1);
          top = fmaxf(fmaxf(s_red[rl], s_red[64 + rl]), fmaxf(s_red[128 + rl], s_red[192 + rl]));
          const bool raise = unset ? top > -INFINITY : top > T_MAX;
          const float d = raise ? top - T_BITS : 0.f;
          factor = raise && !unset ? ex2(-d) : 1.f;          // nothing has been added under an unset maximum
          m += d;
          l *= factor;
          unset = unset && !raise;
          const uint64_t d2 = pack_f32x2(-d, -d);
#pragma unroll
          for (int i = 0; i < 16; ++i) z[i] = add_f32x2(z[i], d2);
        }
        // The weights depend on S and the maximum only: they are packed while O of the previous tile is still running
        uint32_t wh[8], wl[8];
        const float4* offsets = reinterpret_cast<const float4*>(g_offsets.v + 4 * ((uint32_t)(row0 >> 7) * WINDOW_ORDER % WINDOWS) + key0);
        const uint64_t neg2 = pack_f32x2(-1.f, -1.f);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const float gain = ex2(T_BITS - h[q]);
          const uint64_t g2 = pack_f32x2(gain, gain);
          uint64_t sum2 = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint2 kf = *reinterpret_cast<const uint2*>(fact + 2 * key0 + 32 * q + 8 * i);
            uint64_t tt[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const uint32_t f = k ? kf.y : kf.x;
              float z0, z1;
              unpack_f32x2(z[8 * q + 2 * i + k], z0, z1);
              const uint64_t e = pack_f32x2(ex2(z0), ex2(z1));
              tt[k] = mul_f32x2(e, mul_f32x2(join(f << 16, f & 0xffff0000u), g2));
              sum2 = add_f32x2(sum2, e);
            }
            float t[4], h4[4], r[4];
            unpack_f32x2(tt[0], t[0], t[1]);
            unpack_f32x2(tt[1], t[2], t[3]);
            const uint32_t x = e5m2x4_from_float(t[0], t[1], t[2], t[3]);
            e5m2x4_to_float(x, h4);
            const float4 off = offsets[4 * q + i];
            // what the first term leaves (exactly) plus the key's offset
            unpack_f32x2(add_f32x2(fma_f32x2(pack_f32x2(h4[0], h4[1]), neg2, tt[0]), pack_f32x2(off.x, off.y)), r[0], r[1]);
            unpack_f32x2(add_f32x2(fma_f32x2(pack_f32x2(h4[2], h4[3]), neg2, tt[1]), pack_f32x2(off.z, off.w)), r[2], r[3]);
            wh[4 * q + i] = x;
            wl[4 * q + i] = e4m3x4_from_float(r[0], r[1], r[2], r[3]);
          }
          float s0, s1;
          unpack_f32x2(sum2, s0, s1);
          l = fmaf(s0 + s1, gain, l);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(FEMPTY(fr));
        if (j > 0) {                                         // O is complete up to the previous tile, its weights have been read
          ok = mbar_wait(PVDONE, (g - 1) & 1, abort_flag);
          if (!ok) fail(ERR_WAIT_O_DONE);
          __syncwarp();
          if (__any_sync(0xffffffffu, factor != 1.f)) {
            tc_fence_after();
#pragma unroll 1
            for (int q = 4 * cg; q < 4 * cg + 4; ++q) {
              uint32_t o[32];
              tmem_ld32(tmem + lane_base + q * 32, o);
              tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * factor);
              tmem_st32(tmem + lane_base + q * 32, o);
            }
            tmem_wait_st();
          }
        }
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          unsigned char* dst = smem + OFF_P + swz<128>(rl, 4 * half_no + 2 * cg + q);
          *reinterpret_cast<uint4*>(dst) = make_uint4(wh[4 * q], wh[4 * q + 1], wh[4 * q + 2], wh[4 * q + 3]);
          *reinterpret_cast<uint4*>(dst + P_TERM) = make_uint4(wl[4 * q], wl[4 * q + 1], wl[4 * q + 2], wl[4 * q + 3]);
        }
        fence_proxy_async_smem();
        tc_fence_before();
        mbar_arrive(p_bar);
      }
      // ---- the piece is done: its sum, the next unit's queries (S of this piece is complete), then O
      const bool whole = w.n == w.t.n;
      const size_t part = (size_t)2 * pair_id + (first_piece ? 0 : 1);
      const size_t row = ((size_t)w.b * p.q_len + qt) * p.Hq + (gr - qt * p.rep);
      const int rg = 64 * (int)rank + rl;
      first_piece = false;
      softmax_sync();                                        // every maximum has been read
      s_red[cg * 128 + ln] = l;
      softmax_sync();
      l = (s_red[rl] + s_red[64 + rl]) + (s_red[128 + rl] + s_red[192 + rl]);
      more = w.next(p);
      if (more) load_q(w);
      ok = mbar_wait(PVDONE, (g - 1) & 1, abort_flag);
      if (!ok) fail(ERR_WAIT_O_DONE);
      __syncwarp();
      tc_fence_after();
      const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll 1
      for (int q = 4 * cg; q < 4 * cg + 4; ++q) {
        uint32_t o[32];
        tmem_ld32(tmem + lane_base + q * 32, o);
        tmem_wait_ld();
        // columns 0..127 of O: 128 half + c, columns 128..255: 256 + 128 half + c - 128
        const int col = (q >> 2) * 256 + 128 * half_no + (q & 3) * 32;
        if (!whole) {
          float* dst = p.part + (part * ROWS + rg) * DS + col;
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const uint32_t x[8] = {o[8 * v], o[8 * v + 1], o[8 * v + 2], o[8 * v + 3], o[8 * v + 4], o[8 * v + 5], o[8 * v + 6], o[8 * v + 7]};
            st_global_32B(dst + 8 * v, x, true);             // part is 32-byte aligned
          }
        } else if (row_valid) {
          bf16* dst = p.out + row * DS + col;
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            uint32_t x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)                      // no key: O may be 0 * NaN
              x[e] = l == 0.f ? 0u : pack_bf16x2(__uint_as_float(o[16 * v + 2 * e]) * inv, __uint_as_float(o[16 * v + 2 * e + 1]) * inv);
            st_global_32B(dst + 16 * v, x, p.out_wide != 0);
          }
        }
      }
      if (half_no == 0 && cg == 0) {
        if (!whole) {
          float* ml = p.part + (size_t)2 * p.grid * ROWS * DS + part * 2 * ROWS;
          ml[rg] = unset ? -INFINITY : m; ml[ROWS + rg] = l;
        } else if (p.lse && row_valid) {
          p.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l) - T_BITS) * 0.6931471805599453f;
        }
      }
      tc_fence_before();                                     // O is overwritten once all threads have signalled the next piece's first weights
    }
  }
  // ---- free TMEM, once the peer is done with this CTA's memory.  Behind the first barrier no warp gives up any more; if one did, straggling
  // copies land before the second one
  __syncthreads();
  if (*abort_flag && warp == W_MMA) {
    const long long t0c = clock64();
    while (clock64() - t0c < 2000000ll) __nanosleep(1000);
    __syncwarp();
  }
  cluster_sync_all();
  if (warp == W_MMA) { tc_fence_after(); tmem_dealloc_pair(tmem, TM_COLS); }
}

int attn_paged4_pair_launch(Paged4Params& P, cudaStream_t stream) {
  using namespace p4pair;
  if (cudaFuncSetAttribute(attn_paged4_pair_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BYTES) != cudaSuccess) return LCA_ERR_CUDA;
  const int st = launch_chained(attn_paged4_pair_kernel, 2 * (unsigned)P.b.grid, THREADS, SMEM_BYTES, stream, 1, P);      // (clusters of two by declaration)
  if (st != LCA_OK) return st;
  return paged8_combine_launch<DS, ROWS>(P.b, stream);
}

int attn_paged4_pair_take_status() {
  int st = 0;
  if (cudaMemcpyFromSymbol(&st, g_paged4_pair_status, sizeof(int)) != cudaSuccess) return -1;
  if (st != 0) {
    int zero = 0;
    cudaMemcpyToSymbol(g_paged4_pair_status, &zero, sizeof(int));
  }
  return st;
}

}  // namespace lca
