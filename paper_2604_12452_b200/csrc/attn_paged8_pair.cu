// Decode attention over the paged 8-bit cache for the MLA shape and many heads, on CTA pairs.  The mathematics is that of
// attn_paged8.cu (two-term e4m3 queries, two-term weights, one scale per page); the layout is the other way round.
//
// Both terms of a weight are added up in the same columns here, O takes them all, so the second one cannot be scaled.  The first
// term is e5m2 instead: three significant bits (relative error of a weight 2^-8), but down to 2^-16.  What it leaves has steps of 2^-9,
// with the largest weight at 2^8 when its maximum is set (2^11 before it is raised): 2^-17 of it, with offsets spread as there.
// (Offsets that repeat every 64 rows and a largest weight of 2^5: 20000 rows with a period of 32 behind one large logit were off by 0.057.)
//
// With 64 rows or more the transposed tiles of attn_paged8.cu are bound by the 128 bytes per clock of shared memory: every
// product reads both operands from it, 2688 clocks for 64 rows x 128 keys, and the copies of the tile are written through
// the same port (4200 clocks a tile measured; 64 x 5056 rows of 128 heads: 128 us, here 92).  Here two CTAs share 128 query rows (cta_group::2, M = 128): each holds 64
// rows of Q and P, half of the keys for S = Q K^T (N = 128 split by keys) and half of the value columns for O += T V
// (N = 256, twice, split by columns), so that a product reads half the bytes per SM:
//   tensor core   S 36 x 32 + O 16 x 64 clocks = 2176 for 128 rows x 128 keys on two SMs
//   shared memory 36 x 32 + 16 x 48 for operands + 544 for copies + ~200 for the softmax = 2660
// Rows of S and O are TMEM lanes (64 rows, two key halves / two column halves): a softmax thread owns one row and 64 keys;
// the scale of a page is the same for at least 16 of them.
//   warp 0 keys (TMA), warp 1 MMA (even CTA) / forwarding of the odd CTA's signals, warps 2-5 softmax and epilogue,
//   warp 6 values (TMA), warp 7 page table and scales, four tiles at a time
// Signals from the odd to the even CTA ("Q written", "P written") go through one thread that has acquired the writers'
// arrivals and arrives at the even CTA's barrier with a release within its own CTA.  The data never leaves the odd SM: its
// threads write it, each with a fence towards the async proxy before its arrival, and its own tensor core reads it once the
// even CTA has issued the product.  A release across the cluster would order the same writes for readers on other SMs, and
// costs its thread over a thousand clocks (119 us instead of 91).  The tests compare repeated runs bit for bit.
#include <cstring>

#include "attn_paged8.cuh"

namespace lca {
using namespace tc;

static __device__ int g_paged8_pair_status = 0;

namespace p8pair {
constexpr int ROWS = 128, DS = 512, DP = 64;
constexpr int Q_TERM = 4 * 64 * 128 + 64 * 64;              // 36 KB: four latent chunks and the rope chunk of 64 rows
constexpr int K_BUF = 4 * 64 * 128 + 64 * 64;               // the same of 64 keys
constexpr int V_CHUNK = 128 * 128, V_BUF = 2 * V_CHUNK;     // 128 keys x 128 columns, twice
constexpr int P_TERM = 64 * 128;
constexpr int OFF_Q = 0, OFF_K = 2 * Q_TERM, OFF_V = OFF_K + 2 * K_BUF, OFF_P = OFF_V + 2 * V_BUF, OFF_MISC = OFF_P + 2 * P_TERM;
constexpr int BATCHES = 2;                                   // of four tiles of page facts
constexpr int OFF_BAR = OFF_MISC, OFF_SCALAR = OFF_MISC + 192, OFF_RED = OFF_SCALAR + 128, OFF_FACT = OFF_RED + 2 * 128 * 4;
constexpr int OFF_PAGE = OFF_FACT + BATCHES * 32 * 16, OFF_QS = OFF_PAGE + BATCHES * 32 * 4;
constexpr int SMEM_BYTES = OFF_QS + 64 * 4;
constexpr int TM_S = 256, TM_COLS = 512;                     // O in columns 0..255, S in 256..319 and 320..383
constexpr int THREADS = 256;
constexpr float T_BITS = paged8_t_bits(ROWS);
constexpr float T_MAX = 11.f;                                // log2 of the largest weight: e5m2 leaves at most 2^8 of it to e4m3
static_assert(SMEM_BYTES <= 232448, "shared memory of one SM");
static_assert(OFF_QS % 16 == 0 && OFF_FACT % 16 == 0, "alignment");
}  // namespace p8pair

__device__ __forceinline__ void umma_f8_pair_elected(uint32_t leader, uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                                     uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(leader) : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t smem_dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(smem_dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
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

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(p8pair::THREADS, 1)
attn_paged8_pair_kernel(const __grid_constant__ Paged8Params p) {
  using namespace p8pair;
  extern __shared__ __align__(1024) unsigned char smem[];
  const uint32_t base = smem_u32(smem);
  const uint32_t bars = base + OFF_BAR;
  const uint32_t QFULL = bars, PFULL = bars + 8, PVDONE = bars + 16, QLOCAL = bars + 24, PLOCAL = bars + 32;
  auto SFULL = [&](uint32_t i) { return bars + 48 + 8 * i; };
  auto KFULL = [&](uint32_t i) { return bars + 64 + 8 * i; };
  auto KEMPTY = [&](uint32_t i) { return bars + 80 + 8 * i; };
  auto VFULL = [&](uint32_t i) { return bars + 96 + 8 * i; };
  auto VEMPTY = [&](uint32_t i) { return bars + 112 + 8 * i; };
  auto GFULL = [&](uint32_t i) { return bars + 128 + 8 * i; };
  auto GEMPTY = [&](uint32_t i) { return bars + 144 + 8 * i; };
  auto VLOCAL = [&](uint32_t i) { return bars + 160 + 8 * i; };          // odd CTA, values of a tile present in part, per buffer
  const uint32_t QRAW = bars + 176, QDONE = bars + 184;      // queries landed as bf16; ... split, the value buffers are free again
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem + OFF_SCALAR);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + OFF_SCALAR + 4);
  int* s_b = reinterpret_cast<int*>(smem + OFF_SCALAR + 8);
  long long* s_off = reinterpret_cast<long long*>(smem + OFF_SCALAR + 16);
  long long* s_warp = reinterpret_cast<long long*>(smem + OFF_SCALAR + 32);          // 8, and 8 words
  float* s_red = reinterpret_cast<float*>(smem + OFF_RED);                             // [2][128] maxima of even / odd tiles; sums
  float4* s_fact = reinterpret_cast<float4*>(smem + OFF_FACT);                         // per 16 rows: key factor (-1: no page), half, f_t, f_l
  int* s_page = reinterpret_cast<int*>(smem + OFF_PAGE);
  float* s_qs = reinterpret_cast<float*>(smem + OFF_QS);
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair_id = (int)(blockIdx.x >> 1);

  if (threadIdx.x == 0) {
    mbar_init(QFULL, 129); mbar_init(PFULL, 129);            // 128 threads of the even CTA and the odd CTA's forwarder
    mbar_init(PVDONE, 1); mbar_init(QLOCAL, 128); mbar_init(PLOCAL, 128); mbar_init(QRAW, 1); mbar_init(QDONE, 128);
    for (int i = 0; i < 2; ++i) {
      mbar_init(SFULL(i), 1); mbar_init(KFULL(i), 1); mbar_init(KEMPTY(i), 1); mbar_init(VFULL(i), 1); mbar_init(VEMPTY(i), 1); mbar_init(VLOCAL(i), 1);
    }
    for (int i = 0; i < BATCHES; ++i) { mbar_init(GFULL(i), 32); mbar_init(GEMPTY(i), 6); }      // softmax warps, two loaders
    *abort_flag = (base & 1023u) ? 1 : 0;
    fence_mbar_init();
  }
  if (warp == 1) { tmem_alloc_pair(smem_u32((const void*)tmem_slot), TM_COLS); tmem_relinquish_pair(); }
  chain_wait();
  chain_next();
  paged8_range<THREADS>(p, pair_id, s_warp, s_b, s_off);
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                                        // both CTAs' barriers are initialised
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  auto fail = [&](int code) { atomicCAS(&g_paged8_pair_status, 0, code); *abort_flag = 1; };
  if (threadIdx.x == 0 && (base & 1023u)) atomicCAS(&g_paged8_pair_status, 0, 100);
  Walk w;
  w.b = *s_b; w.off = s_off[0]; w.left = s_off[1]; w.fresh = true; w.n = 0;

  // A tile whose pages are present in part (the rows behind the last representative or token of a sequence): what lies there
  // may be anything, and 0 * NaN is not 0, so each CTA zeroes those rows of its own values.  The odd CTA's copies of such a
  // tile complete on a barrier of its own, for it cannot see the even CTA's.
  auto partial = [&](const Walk& u, int j) {
    const int mask = p.page - 1, row0 = u.t.row0(u.t0 + j), r = u.t.s.n_rep, t = u.t.s.n_tok;
    return ((r & mask) && (unsigned)((r & ~mask) - row0) < 128u) || ((t & mask) && (unsigned)((t & ~mask) - row0) < 128u);
  };

  if (warp == 0 || warp == 6) {
    // ------------------------------------------------------------------------ loads: keys (warp 0), values (warp 6)
    const bool keys = warp == 0;
    const int box = min(p.page, 64);                                                   // rows of a request
    const int n_req = (keys ? 64 : 128) / box;                                         // per chunk
    uint32_t g = 0, bat0 = 0, seg = 0;
    bool ok = !*abort_flag;
    while (ok && w.next(p)) {
      if (!keys) {                                           // the queries of the piece pass through the value buffers
        ok = mbar_wait(QDONE, seg & 1, abort_flag);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) { if (lane == 0) fail(ERR_WAIT_Q); break; }
        ++seg;
      }
      for (int j = 0; j < w.n && ok; ++j, ++g) {
        const uint32_t bat = bat0 + (uint32_t)(j >> 2), ring = bat % BATCHES, buf = g & 1;
        if ((j & 3) == 0) ok = mbar_wait(GFULL(ring), (bat / BATCHES) & 1, abort_flag);
        if (ok) ok = mbar_wait(keys ? KEMPTY(buf) : VEMPTY(buf), ((g >> 1) & 1) ^ 1, abort_flag);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) { if (lane == 0) fail(ERR_WAIT_KV_EMPTY); break; }
        // request `lane` of a chunk: rows [first, first + box) of the tile
        const int first = (keys ? 64 * (int)rank : 0) + lane * box;
        const int z = lane < n_req ? s_page[ring * 32 + (j & 3) * 8 + (first >> 4)] : 0, y = (first & (p.page - 1));
        if (keys) {
          if (lane == 0 && rank == 0) mbar_expect_tx(KFULL(buf), 2 * K_BUF);
          const uint32_t bar = mapa_u32(KFULL(buf), 0), dst = base + OFF_K + buf * K_BUF;
          if (lane < n_req) {
#pragma unroll
            for (int c = 0; c < 4; ++c) tma_load_3d_pair(dst + c * 8192 + lane * box * 128, &p.sem, c * 128, y, z, bar);
            tma_load_3d_pair(dst + 4 * 8192 + lane * box * 64, &p.pos, 0, y, z, bar);
          }
        } else {
          const bool own_bar = rank == 1 && partial(w, j);
          uint32_t bar;
          if (own_bar) {
            if (lane == 0) mbar_expect_tx(VLOCAL(buf), V_BUF);
            bar = mapa_u32(VLOCAL(buf), 1);
          } else {
            if (lane == 0 && rank == 0) mbar_expect_tx(VFULL(buf), (partial(w, j) ? 1 : 2) * V_BUF);
            bar = mapa_u32(VFULL(buf), 0);
          }
          const uint32_t dst = base + OFF_V + buf * V_BUF;
          __syncwarp();
          if (lane < n_req) {
#pragma unroll
            for (int c = 0; c < 2; ++c) tma_load_3d_pair(dst + c * V_CHUNK + lane * box * 128, &p.sem, 256 * c + 128 * (int)rank, y, z, bar);
          }
        }
        __syncwarp();
        if (lane == 0 && ((j & 3) == 3 || j + 1 == w.n)) mbar_arrive(GEMPTY(ring));
      }
      bat0 += (uint32_t)(w.n + 3) >> 2;
    }
  } else if (warp == 7) {
    // ------------------------------------------------------------------ page facts: a lane per 16 rows, four tiles at a time
    uint32_t i = 0;
    bool ok = !*abort_flag;
    while (ok && w.next(p)) {
      const PagedSpan sp = w.t.s;
      const int32_t* table = p.table + (size_t)w.b * p.width;
#pragma unroll 1
      for (int j0 = 0; j0 < w.n && ok; j0 += 4, ++i) {
        const int j = j0 + (lane >> 3), x = j < w.n ? w.t.row0(w.t0 + j) + (lane & 7) * 16 : 0, first = x & ~(p.page - 1);
        int z = p.n_pages;                                   // one past the end: filled with zeros
        float4 f = make_float4(-1.f, 0.f, 1.f, 1.f);
        if (j < w.n && sp.any(first, p.page) && (x >> p.page_log2) < p.width) {
          const int pg = table[x >> p.page_log2];
          if (pg >= 0 && pg < p.n_pages) {
            z = pg;
            const float ks = p.scale_k[z], vs = fmaxf(ks, exp2_int(PAGED8_MIN_EXP));
            // The row sum needs 2^(y - M), the weight t = 2^(y - M + log2 vs + T): both are multiples of e = 2^(y - M + half), half
            // way between them, so that neither is lost below 2^-126 where the scales span more than fp32 does.
            const float half = 0.5f * (lg2(vs) + T_BITS);
            f = make_float4(ks * p.scale_log2, half, ex2(half), ex2(T_BITS - half));
          }
        }
        ok = mbar_wait(GEMPTY(i % BATCHES), ((i / BATCHES) & 1) ^ 1, abort_flag);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) { if (lane == 0) fail(ERR_WAIT_PEER); break; }
        s_fact[(i % BATCHES) * 32 + lane] = f;
        s_page[(i % BATCHES) * 32 + lane] = z;
        mbar_arrive(GFULL(i % BATCHES));
      }
    }
  } else if (warp == 1 && rank == 0) {
    // --------------------------------------------------------------------------------------------- MMA (even CTA)
    const uint32_t leader = elect_one();
    constexpr uint32_t ID_S = umma_idesc_f8(128, 128, 0, false, false);
    constexpr uint32_t ID_LO = umma_idesc_f8(128, 256, 0, false, true), ID_HI = ID_LO | (1u << 7);       // A: e4m3 / e5m2
    const uint64_t q_hi = desc_rows(base + OFF_Q, 128, 16), qp_hi = desc_rows(base + OFF_Q + 4 * 8192, 64, 16);
    const uint64_t k0 = desc_rows(base + OFF_K, 128, 16), kp0 = desc_rows(base + OFF_K + 4 * 8192, 64, 16);
    const uint64_t p_hi = desc_rows(base + OFF_P, 128, 16), v0 = desc_rows(base + OFF_V, 128, 16);
    uint32_t g = 0, seg = 0;
    bool ok = !*abort_flag;
    auto issue_s = [&](uint32_t t) {
      const uint32_t buf = t & 1, d = tmem + TM_S + 64 * buf, off = buf * (K_BUF / 16);
      ok = mbar_wait(KFULL(buf), (t >> 1) & 1, abort_flag);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) { if (lane == 0) fail(ERR_WAIT_KV_FULL); return; }
      tc_fence_after();
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int h = 0; h < 2; ++h)
            umma_f8_pair_elected(leader, d, desc_add(q_hi, (h * Q_TERM + c * 8192 + k * 32) >> 4), desc_add(k0, off + ((c * 8192 + k * 32) >> 4)), ID_S,
                                 (c > 0 || k > 0 || h > 0) ? 1u : 0u);
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) umma_f8_pair_elected(leader, d, desc_add(qp_hi, (h * Q_TERM + k * 32) >> 4), desc_add(kp0, off + 2 * k), ID_S, 1u);
      umma_commit_pair_elected(leader, KEMPTY(buf), 3);
      umma_commit_pair_elected(leader, SFULL(buf), 3);
    };
    while (ok && w.next(p)) {
      ok = mbar_wait(QFULL, seg & 1, abort_flag);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) { if (lane == 0) fail(ERR_WAIT_Q); break; }
      ++seg;
      tc_fence_after();
      issue_s(g);
      for (int j = 0; j < w.n && ok; ++j, ++g) {
        if (j + 1 < w.n) issue_s(g + 1);
        if (!ok) break;
        const uint32_t buf = g & 1, off = buf * (V_BUF / 16);
        ok = mbar_wait(VFULL(buf), (g >> 1) & 1, abort_flag);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) { if (lane == 0) fail(ERR_WAIT_KV_FULL); break; }
        ok = mbar_wait(PFULL, g & 1, abort_flag);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) { if (lane == 0) fail(ERR_WAIT_P_FULL); break; }
        tc_fence_after();
#pragma unroll
        for (int n2 = 0; n2 < 2; ++n2)
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h)
              umma_f8_pair_elected(leader, tmem + n2 * 128, desc_add(p_hi, (h * P_TERM + k * 32) >> 4), desc_add(v0, off + ((n2 * V_CHUNK + k * 4096) >> 4)),
                                   h ? ID_LO : ID_HI, (j > 0 || k > 0 || h > 0) ? 1u : 0u);
        umma_commit_pair_elected(leader, VEMPTY(buf), 3);
        umma_commit_pair_elected(leader, PVDONE, 3);
      }
    }
  } else if (warp == 1) {
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
    const int quad = warp & 3, ln = quad * 32 + lane, rl = ln & 63, half_no = ln >> 6;   // TMEM lane; row of this CTA, key half
    const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
    const uint32_t q_bar = rank == 0 ? QFULL : QLOCAL, p_bar = rank == 0 ? PFULL : PLOCAL;
    uint32_t g = 0, bat0 = 0, v_phase = 0, seg = 0;          // v_phase: phase of VLOCAL(0), VLOCAL(1) in bits 0, 1
    bool ok = true, first_piece = true;
    // The queries of a piece come as bf16 rows by bulk copies into the value and weight buffers, which nothing uses between two
    // pieces, and are split from there: the loop that splits them is then short (loaded straight into registers, several rows
    // at a time to cover the latency, its unrolled code had to be fetched once per launch and took 14000 clocks).
    auto start_q = [&](const Walk& u) {
      const int valid = min(max(p.q_len * p.rep - u.blk * ROWS - 64 * (int)rank, 0), 64);      // rows of this CTA
      if (ln == 0) mbar_expect_tx(QRAW, valid * (DS + DP) * 2);
      if (rl < valid) {
        const int gr = u.blk * ROWS + 64 * (int)rank + rl, qt = gr / p.rep;
        const size_t row = ((size_t)u.b * p.q_len + qt) * p.Hq + (gr - qt * p.rep);
        if (half_no == 0) bulk_load(base + OFF_V + rl * 1024, p.q_sem + row * DS, 1024, QRAW);
        else bulk_load(base + OFF_V + 65536 + rl * 128, p.q_pos + row * DP, 128, QRAW);
      }
    };
    auto finish_q = [&](const Walk& u) {
      const int valid = min(max(p.q_len * p.rep - u.blk * ROWS - 64 * (int)rank, 0), 64);
      ok = mbar_wait(QRAW, seg & 1, abort_flag);
      if (!ok) fail(ERR_WAIT_Q);
      __syncwarp();
#pragma unroll 1
      for (int r = quad; r < 64; r += 4) {
        uint4 v[3];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 3; ++i) {
          const int c = lane + 32 * i;
          v[i] = make_uint4(0u, 0u, 0u, 0u);
          if (r < valid && c < 72) v[i] = *reinterpret_cast<const uint4*>(smem + OFF_V + (c < 64 ? r * 1024 + 16 * c : 65536 + r * 128 + 16 * (c - 64)));
          top = max(top, max_abs_bf16(v[i]));
        }
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
      mbar_arrive(QDONE);
      asm volatile("bar.sync 1, 128;" ::: "memory");
      ++seg;
    };
    bool more = w.next(p);
    if (more) start_q(w);
    while (more) {
      finish_q(w);
      const PagedSpan sp = w.t.s;
      const int gr = w.blk * ROWS + 64 * (int)rank + rl, qt = gr / p.rep;
      const bool row_valid = gr < p.q_len * p.rep;
      const int lim = sp.n_tok - p.q_len + 1 + (row_valid ? qt : 0), lim_all = sp.n_tok - p.q_len + 1;
      const float qs = row_valid ? s_qs[rl] : 0.f;
      float m = row_valid ? 0.f : 3.0e38f, l = 0.f;          // rows behind the last one never have weight
      bool unset = row_valid;                                // no key seen yet
#pragma unroll 1
      for (int j = 0; j < w.n; ++j, ++g) {
        const uint32_t bat = bat0 + (uint32_t)(j >> 2), ring = bat % BATCHES;
        const int row0 = w.t.row0(w.t0 + j), x0 = row0 + 64 * half_no;
        if ((j & 3) == 0) {
          ok = mbar_wait(GFULL(ring), (bat / BATCHES) & 1, abort_flag);
          if (!ok) fail(ERR_WAIT_PEER);
        }
        const float4* fact = s_fact + ring * 32 + (j & 3) * 8 + 4 * half_no;
        ok = mbar_wait(SFULL(g & 1), (g >> 1) & 1, abort_flag);
        if (!ok) fail(ERR_WAIT_S_FULL);
        __syncwarp();
        tc_fence_after();
        uint64_t z[32];                                      // log2 of e, in pairs of keys
        {
          uint32_t s[2][32];
          tmem_ld32(tmem + lane_base + TM_S + 64 * (g & 1), s[0]);
          tmem_ld32(tmem + lane_base + TM_S + 64 * (g & 1) + 32, s[1]);
          tmem_wait_ld();
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float4 f = fact[q];
            const float wk = f.x * qs, c = f.y - m;
            const uint64_t w2 = pack_f32x2(wk, wk), c2 = pack_f32x2(c, c);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int e = (q & 1) * 16 + 2 * i;
              z[8 * q + i] = fma_f32x2(join(s[q >> 1][e], s[q >> 1][e + 1]), w2, c2);
            }
          }
        }
        // present keys, keys this row may see and representatives, as bits; most tiles are all keys and no bias
        const bool tile_reps = row0 < sp.n_rep && p.bias_log2 != 0.f;
        const bool whole_tile = row0 + 128 <= min(sp.n_tok, lim_all) && (row0 >= sp.tok0 || row0 + 128 <= sp.n_rep);
        const bool pages = fact[0].x >= 0.f && fact[1].x >= 0.f && fact[2].x >= 0.f && fact[3].x >= 0.f;
        if (!whole_tile || tile_reps || !pages) {
          uint64_t see = (low_bits(sp.n_rep - x0) | (low_bits(sp.n_tok - x0) & ~low_bits(sp.tok0 - x0))) & low_bits(lim - x0);
          const uint64_t reps = low_bits(sp.n_rep - x0);
#pragma unroll
          for (int q = 0; q < 4; ++q) if (fact[q].x < 0.f) see &= ~(0xffffull << (16 * q));
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            float z0, z1;
            unpack_f32x2(z[i], z0, z1);
            z0 = (see >> (2 * i)) & 1 ? z0 + ((reps >> (2 * i)) & 1 ? p.bias_log2 : 0.f) : -INFINITY;
            z1 = (see >> (2 * i + 1)) & 1 ? z1 + ((reps >> (2 * i + 1)) & 1 ? p.bias_log2 : 0.f) : -INFINITY;
            z[i] = pack_f32x2(z0, z1);
          }
        }
        float top = -INFINITY;                               // largest log2 t of this row's half
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float a = -INFINITY, b = -INFINITY;
#pragma unroll
          for (int i = 0; i < 8; i += 2) {
            float z0, z1, z2, z3;
            unpack_f32x2(z[8 * q + i], z0, z1);
            unpack_f32x2(z[8 * q + i + 1], z2, z3);
            a = max3(a, z0, z1); b = max3(b, z2, z3);
          }
          top = fmaxf(top, fmaxf(a, b) + fact[q].y);
        }
        s_red[(g & 1) * 128 + ln] = top;
        asm volatile("bar.sync 1, 128;" ::: "memory");
        top = fmaxf(top, s_red[(g & 1) * 128 + (ln ^ 64)]);
        const bool raise = unset ? top > -INFINITY : top > T_MAX;
        const float d = raise ? top - T_BITS : 0.f, factor = raise && !unset ? ex2(-d) : 1.f;
        m += d;
        l *= factor;
        unset = unset && !raise;
        // The weights depend on S and the maximum only: they are packed while O of the previous tile is still running
        uint32_t wh[16], wl[16];
        const uint64_t d2 = pack_f32x2(-d, -d), neg2 = pack_f32x2(-1.f, -1.f);
        const float4* offsets = reinterpret_cast<const float4*>(g_offsets.v + 4 * ((uint32_t)(row0 >> 7) * WINDOW_ORDER % WINDOWS) + 64 * half_no);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float4 f = fact[q];
          const uint64_t ft2 = pack_f32x2(f.z, f.z);
          uint64_t sum2 = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint64_t tt[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              float z0, z1;
              unpack_f32x2(add_f32x2(z[8 * q + 2 * i + k], d2), z0, z1);
              const uint64_t e = pack_f32x2(ex2(z0), ex2(z1));
              tt[k] = mul_f32x2(e, ft2);
              sum2 = add_f32x2(sum2, e);
            }
            float t[4], h[4], r[4];
            unpack_f32x2(tt[0], t[0], t[1]);
            unpack_f32x2(tt[1], t[2], t[3]);
            const uint32_t w = e5m2x4_from_float(t[0], t[1], t[2], t[3]);
            e5m2x4_to_float(w, h);
            const float4 off = offsets[4 * q + i];
            // what the first term leaves (exactly) plus the key's offset
            unpack_f32x2(add_f32x2(fma_f32x2(pack_f32x2(h[0], h[1]), neg2, tt[0]), pack_f32x2(off.x, off.y)), r[0], r[1]);
            unpack_f32x2(add_f32x2(fma_f32x2(pack_f32x2(h[2], h[3]), neg2, tt[1]), pack_f32x2(off.z, off.w)), r[2], r[3]);
            wh[4 * q + i] = w;
            wl[4 * q + i] = e4m3x4_from_float(r[0], r[1], r[2], r[3]);
          }
          float a, b;
          unpack_f32x2(sum2, a, b);
          l = fmaf(a + b, f.w, l);
        }
        if (j > 0) {                                         // O is complete up to the previous tile, its weights have been read
          ok = mbar_wait(PVDONE, (g - 1) & 1, abort_flag);
          if (!ok) fail(ERR_WAIT_O_DONE);
          __syncwarp();
          if (__any_sync(0xffffffffu, factor != 1.f)) {
            tc_fence_after();
#pragma unroll 1
            for (int q = 0; q < 8; ++q) {
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
        for (int q = 0; q < 4; ++q) {
          unsigned char* dst = smem + OFF_P + swz<128>(rl, 4 * half_no + q);
          *reinterpret_cast<uint4*>(dst) = make_uint4(wh[4 * q], wh[4 * q + 1], wh[4 * q + 2], wh[4 * q + 3]);
          *reinterpret_cast<uint4*>(dst + P_TERM) = make_uint4(wl[4 * q], wl[4 * q + 1], wl[4 * q + 2], wl[4 * q + 3]);
        }
        if (partial(w, j)) {
          ok = rank == 0 ? mbar_wait(VFULL(g & 1), (g >> 1) & 1, abort_flag) : mbar_wait(VLOCAL(g & 1), (v_phase >> (g & 1)) & 1, abort_flag);
          if (!ok) fail(ERR_WAIT_KV_FULL);
          v_phase ^= 1u << (g & 1);
          if (!sp.has(row0 + ln)) {                          // this thread: row ln of the tile
#pragma unroll
            for (int i = 0; i < 16; ++i)
              *reinterpret_cast<uint4*>(smem + OFF_V + (g & 1) * V_BUF + (i >> 3) * V_CHUNK + ln * 128 + (i & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
          __syncwarp();
        }
        fence_proxy_async_smem();
        tc_fence_before();
        mbar_arrive(p_bar);
        __syncwarp();
        if (lane == 0 && ((j & 3) == 3 || j + 1 == w.n)) mbar_arrive(GEMPTY(ring));
      }
      bat0 += (uint32_t)(w.n + 3) >> 2;
      // ---- the piece is done: its sum, the next unit's queries on their way, then O
      const bool whole = w.n == w.t.n;
      const size_t part = (size_t)2 * pair_id + (first_piece ? 0 : 1);
      const size_t row = ((size_t)w.b * p.q_len + qt) * p.Hq + (gr - qt * p.rep);
      const int rg = 64 * (int)rank + rl;
      first_piece = false;
      asm volatile("bar.sync 1, 128;" ::: "memory");         // every maximum has been read
      s_red[ln] = l;
      asm volatile("bar.sync 1, 128;" ::: "memory");
      l += s_red[ln ^ 64];
      asm volatile("bar.sync 1, 128;" ::: "memory");
      ok = mbar_wait(PVDONE, (g - 1) & 1, abort_flag);
      if (!ok) fail(ERR_WAIT_O_DONE);
      __syncwarp();
      more = w.next(p);
      if (more) start_q(w);
      tc_fence_after();
      const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll 1
      for (int q = 0; q < 8; ++q) {
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
      if (half_no == 0) {
        if (!whole) {
          float* ml = p.part + (size_t)2 * p.grid * ROWS * DS + part * 2 * ROWS;
          ml[rg] = unset ? -INFINITY : m; ml[ROWS + rg] = l;
        } else if (p.lse && row_valid) {
          p.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l) - T_BITS) * 0.6931471805599453f;
        }
      }
      tc_fence_before();
    }
  }
  // ---- let straggling copies land if the CTA gave up; the peer is done with this CTA's memory; free TMEM
  if (*abort_flag && (warp == 0 || warp == 6) && lane == 0) {
    const long long t0c = clock64();
    while (clock64() - t0c < 2000000ll) __nanosleep(1000);
  }
  __syncthreads();
  cluster_sync_all();
  if (warp == 1) { tc_fence_after(); tmem_dealloc_pair(tmem, TM_COLS); }
}

int attn_paged8_pair_launch(Paged8Params& P, cudaStream_t stream) {
  using namespace p8pair;
  if (cudaFuncSetAttribute(attn_paged8_pair_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BYTES) != cudaSuccess) return LCA_ERR_CUDA;
  const int st = launch_chained(attn_paged8_pair_kernel, 2 * (unsigned)P.grid, THREADS, SMEM_BYTES, stream, 1, P);      // (clusters of two by declaration)
  if (st != LCA_OK) return st;
  return paged8_combine_launch<DS, ROWS>(P, stream);
}

int attn_paged8_pair_take_status() {
  int st = 0;
  if (cudaMemcpyFromSymbol(&st, g_paged8_pair_status, sizeof(int)) != cudaSuccess) return -1;
  if (st != 0) {
    int zero = 0;
    cudaMemcpyToSymbol(g_paged8_pair_status, &zero, sizeof(int));
  }
  return st;
}

}  // namespace lca
