// Decode attention over the paged 4-bit cache (Sec. 4.3 over the layout of lca_paged4).
//
// Mathematics.  For a query row h and the present rows i of its sequence and KV head
//     y_i = log2(e) (scale * f_k(i) * sum_c q_c k_ic + bias_i),   out = sum_i 2^y_i f_v(i) v_i / sum_i 2^y_i
// where k, v are the cached rows expanded to e4m3 codes (exactly: fp4_common.cuh) and f one power of two for each row and KV head.
// Queries and weights are sums of two e4m3 terms, as in attn_paged8.cu, which derives their errors: a query element is off by at
// most 2^-17 of its row's largest, a weight t_i = 2^(y_i + log2 f_v(i) - M + 5) by 2^-9 of itself or by a step of 2^-18 of the largest,
// the step rounded with an offset of the key's own.  M is the running maximum of y + log2 f_v over a split, raised when a weight
// would exceed 2^8.75; the row sum adds the weights without f_v in fp32, unrounded.
//
// Transposed products, the key tile as the 128-row operand: S^T [128 keys x 2 NH] = K [Q_hi | Q_lo]^T, O^T [d x 2 NH] += V^T [T_hi | T_lo]^T.
//   softmax    GROUPS groups of four warps, each for ROWS of the query rows: thread = key = TMEM lane; epilogue: thread = output column
//   expansion  4 warps, or 8: 32 values (16 bytes of codes) at a time to e4m3, into the operands' swizzled images
//   + a warp each for page look-ups and exponents, for bulk copies of codes (STAGED), for the products and TMEM
// Tiles flow through the pieces of a CTA without a pause: look-ups, copies and expansion run ahead of the piece that the softmax
// warps are at.  There are two buffers of S and of weights; of the next S and the next O the product warp issues whichever can go first, so
// that a tile's softmax only waits for O of the tile before the last one, unless it has to raise a maximum.
// Codes: where two tiles of them fit into shared memory beside the expanded tiles (all shapes but MLA 512 + 64) they come by bulk copies, one for
// each page and part; else the expansion warps load them to registers a tile ahead, behind the fence that ends a tile (in front of it the
// fence waits for them).  GQA, 64 x 5056 rows of 8 KV heads, when either was built for it, before the steps to today's 121 us: 131 us by copies, 145
// by registers.
// Work: as in attn_paged8.cu, one line of tiles cut into equal ranges, pieces merged by paged8_combine_kernel.
// What bounds it: not HBM (64 x 5056 rows, GQA 32 heads on 8: 348 MB in 121 us, 2.9 TB/s; MLA 16 heads: 97 MB in 55 us) but the chain of a tile -
// expansion (seven instructions at half rate for eight values, 2000 warp instructions a tile for MLA 512 + 64, and 72 KB written through the port of
// shared memory that feeds the products), S, softmax, weights, O, each handed on at 300 to 400 clocks - about 3000 clocks a tile and CTA for
// GQA (two CTAs an SM), 3800 for MLA with 16 rows, 4800 with 32, and 22 us of launch, ranges, queries and merging.
#include <cstring>

#include "attn_paged4.cuh"

namespace lca {
using namespace tc;

static __device__ int g_paged4_status = 0;

static constexpr float T4_MAX = 8.75f;                       // log2 of the largest weight: e4m3 ends at 448
static constexpr float LO4_GAIN = 16.f;                      // of the second term, which has columns of O of its own

// --------------------------------------------------------------------------------------------------- scalar kernel
// One warp per query row, keys one by one, fp32: the cross-check of the tensor-core kernel (lca_set_attention_impl(1)).
template <int D_SEM, int D_POS, bool MLA>
__global__ void __launch_bounds__(128) attn_paged4_simt_kernel(const __grid_constant__ Paged4Params q, float scale, float bias, long long n_rows) {
  constexpr int PS = D_SEM / 64, PP = D_POS / 64;            // element pairs per lane: 2 lane + 64 i
  __shared__ uint2 s_table[16];
  const Paged8Params& p = q.b;
  const int lane = threadIdx.x & 31;
  paged4_table_load(s_table, threadIdx.x);
  __syncthreads();
  const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (row >= n_rows) return;
  const int h = (int)(row % p.Hq), t = (int)((row / p.Hq) % p.q_len), b = (int)(row / ((long long)p.Hq * p.q_len));
  const int hk = h / p.rep;
  float2 qs[PS], qp[PP], acc[PS];
#pragma unroll
  for (int i = 0; i < PS; ++i) {
    acc[i] = make_float2(0.f, 0.f);
    if (MLA) qs[i] = __bfloat1622float2(reinterpret_cast<const bf162*>(p.q_sem + (size_t)row * D_SEM)[lane + 32 * i]);
  }
#pragma unroll
  for (int i = 0; i < PP; ++i) qp[i] = __bfloat1622float2(reinterpret_cast<const bf162*>(p.q_pos + (size_t)row * D_POS)[lane + 32 * i]);
  // columns 2 lane, 2 lane + 1 of the 64 from 64 i on: in word 8 i + lane / 4, block 2 i + lane / 16
  auto pair = [&](const uint8_t* codes, const uint8_t* shifts, int i) {
    const uint32_t w = reinterpret_cast<const uint32_t*>(codes)[8 * i + (lane >> 2)];
    const uint2 c = paged4_expand(w, s_table[(shifts[i] >> ((lane >> 4) * 4)) & 15]);
    const float4 f = e4m3x4_to_float4(((lane & 2) ? c.y : c.x) >> ((lane & 1) * 16));
    return make_float2(f.x, f.y);
  };
  const PagedSpan sp = paged_span(p.n_rep, p.n_tok, b, p.g, p.width * p.page);
  const int last = sp.n_tok - p.q_len + 1 + t;               // rows below it are seen
  float mx = -INFINITY, l = 0.f;
  bool any = false;
  for (int x = 0; x < last; ++x) {
    if (x == sp.n_rep && x < sp.tok0) x = sp.tok0;
    if (x >= last) break;
    const int pg = p.table[(size_t)b * p.width + x / p.page];
    if (pg < 0 || pg >= p.n_pages) continue;
    const size_t r = ((size_t)pg * p.Hkv + hk) * p.page + x % p.page;
    const float fv = paged4_factor(q.exp_v[r]), fk = paged4_factor(q.exp_k[r]);
    float2 v[PS];
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < PS; ++i) {
      v[i] = pair(q.sem + r * (D_SEM / 2), q.shift_sem + r * (D_SEM / 64), i);
      if (MLA) s += qs[i].x * v[i].x + qs[i].y * v[i].y;
    }
#pragma unroll
    for (int i = 0; i < PP; ++i) {
      const float2 k = pair(q.pos + r * (D_POS / 2), q.shift_pos + r * (D_POS / 64), i);
      s += qp[i].x * k.x + qp[i].y * k.y;
    }
    s = warp_sum(s) * fk * scale + (x < sp.n_rep ? bias : 0.f);
    any = true;
    const float mn = fmaxf(mx, s), corr = expf(mx - mn), w = expf(s - mn);
    l = l * corr + w;
#pragma unroll
    for (int i = 0; i < PS; ++i) {
      acc[i].x = acc[i].x * corr + w * (v[i].x * fv);
      acc[i].y = acc[i].y * corr + w * (v[i].y * fv);
    }
    mx = mn;
  }
  const float inv = any ? 1.f / l : 0.f;
#pragma unroll
  for (int i = 0; i < PS; ++i)
    reinterpret_cast<bf162*>(p.out + (size_t)row * D_SEM)[lane + 32 * i] = __floats2bfloat162_rn(acc[i].x * inv, acc[i].y * inv);
  if (p.lse && lane == 0) p.lse[row] = any ? mx + logf(l) : -INFINITY;
}

// ---------------------------------------------------------------------------------------------- tensor-core kernel
template <bool MLA_, int DS_, int DP_, int NH_, int GROUPS_, int ROWS_>
struct Paged4Plan {
  static constexpr bool MLA = MLA_;
  static constexpr int DS = DS_, DP = DP_, NH = NH_, GROUPS = GROUPS_, ROWS = ROWS_;        // GROUPS * ROWS of the NH rows exist
  static constexpr int KSEM = MLA ? DS / 128 : 0;            // latent chunks of the key product; then the pos chunk (64 or 128 columns)
  static constexpr int NV = DS >= 128 ? DS / 128 : 1, VW = DS >= 128 ? 128 : DS;
  static constexpr int K_BYTES = 128 * (KSEM * 128 + DP), V_BYTES = MLA ? 0 : 16384, TILE = K_BYTES + V_BYTES;        // expanded
  static constexpr int Q_BYTES = 2 * NH * (KSEM * 128 + DP);
  static constexpr int P_BYTES = 128 * 2 * NH;               // per key the first terms of all rows, then the second ones
  static constexpr int TM_S = 2 * NV * NH, TM_USED = TM_S + 4 * NH;
  static constexpr int TM_COLS = TM_USED <= 64 ? 64 : TM_USED <= 128 ? 128 : TM_USED <= 256 ? 256 : 512;
  static constexpr int CTAS = (MLA && DS == 512) || NH == 32 ? 1 : 2;        // per SM
  // Packed rows come by bulk copies into shared memory where there is room for it, else straight to the registers of the threads that
  // expand them.
  static constexpr bool STAGED = !(MLA && DS == 512);
  // Expansion warps.  More of them hide more latency, fewer leave more registers and issue slots to the others: with 4 and 8, 64 x 5056 rows,
  // GQA 128 with 4 / 16 / 32 rows a KV head 121 / 157 / 206 and 121 / 173 / 208 us, GQA 64 90 and 101, MLA 128 + 64 with 4 / 16 / 32 rows 25 / 33 / 38 and 26 / 38 / 39;
  // MLA 512 + 64 with 16 rows 60 and 55.
  static constexpr int EW = STAGED ? 4 : 8, SOFTMAX_WARPS = 4 * GROUPS, W_EXP = SOFTMAX_WARPS, W_MMA = W_EXP + EW, W_LOOK = W_MMA + 1, W_LOAD = W_LOOK + (STAGED ? 1 : 0);
  static constexpr int THREADS = 32 * (W_LOAD + 1);
  static constexpr int STAGE = STAGED ? 128 * (DS + DP) / 2 : 0, ST_POS = 128 * DS / 2;      // codes of a tile: latents or V, keys
  // 32 values at a time: a thread's share of a tile, latents (V) and keys
  static constexpr int U_SEM = DS * 128 / 32 / (32 * EW), U_POS = DP * 128 / 32 / (32 * EW);
  // per tile: exponents of values and of keys, where its rows are, STAGED: shifts
  static constexpr int FACTS = 4, F_GROUP = 256, F_SPAN = 288, F_SHS = 304, F_SHP = F_SHS + (STAGED ? 2 * DS : 0), FACT = F_SHP + (STAGED ? 2 * DP : 0);
  // words: qs, M, d, factor, lim [NH]; wmax / sums [4][NH]; output rows [2][NH].  Barriers and scalars first, then the table.
  static constexpr int MISC_BYTES = 512 + 128 + 4 * (5 * NH + 4 * NH + 2 * NH) + FACTS * FACT;
  static constexpr int ROOM = CTAS == 1 ? 227 * 1024 : 113 * 1024;
  static constexpr int BUFS = CTAS == 1 && STAGED ? 3 : 2;   // expanded tiles
  static constexpr int STAGES_FIT = STAGED ? (ROOM - BUFS * TILE - Q_BYTES - 2 * P_BYTES - MISC_BYTES) / (STAGED ? STAGE : 1) : 0;
  static constexpr int STAGES = STAGES_FIT > 4 ? 4 : STAGES_FIT;
  static constexpr int OFF_Q = BUFS * TILE, OFF_P = OFF_Q + Q_BYTES, OFF_STAGE = OFF_P + 2 * P_BYTES, OFF_MISC = OFF_STAGE + STAGES * STAGE;
  static constexpr int SMEM = OFF_MISC + MISC_BYTES;
  static_assert((!STAGED || STAGES >= 2) && SMEM <= ROOM && OFF_MISC % 16 == 0 && OFF_Q % 1024 == 0 && FACT % 16 == 0, "one tile is expanded while another is used");
  static_assert(THREADS <= 32 * 28, "72 registers a thread");
};

// one group of softmax warps (128 threads)
__device__ __forceinline__ void group_sync(int grp) { asm volatile("bar.sync %0, 128;" ::"r"(grp + 1) : "memory"); }
__device__ __forceinline__ bool group_or(int grp, bool v) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(r) : "r"((uint32_t)v), "r"(grp + 1) : "memory");
  return r != 0;
}
// N consecutive 32-bit columns of this warp's lanes
template <int N>
__device__ __forceinline__ void tmem_ld(uint32_t at, uint32_t (&r)[N]) {
  if constexpr (N == 4)
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
  else
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(at) : "memory");
}
template <int N>
__device__ __forceinline__ void tmem_st(uint32_t at, const uint32_t (&r)[N]) {
  if constexpr (N == 4)
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
  else
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ void bulk_copy(uint32_t smem_dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(smem_dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
template <class PL>
__global__ void __launch_bounds__(PL::THREADS, PL::CTAS) attn_paged4_kernel(const __grid_constant__ Paged4Params a) {
  constexpr int NH = PL::NH, NV = PL::NV, DS = PL::DS, DP = PL::DP, ROWS = PL::ROWS;
  constexpr int W_EXP = PL::W_EXP, W_MMA = PL::W_MMA, W_LOOK = PL::W_LOOK, W_LOAD = PL::W_LOAD;
  const Paged8Params& p = a.b;
  extern __shared__ __align__(1024) unsigned char smem_p4[];
  unsigned char* base_ptr = smem_p4;
  const uint32_t base = smem_u32(smem_p4);
  const uint32_t bars = base + PL::OFF_MISC;
  // two buffers of each: S complete, weights written, O complete
  auto SFULL = [&](uint32_t i) { return bars + 8 * i; };
  auto PFULL = [&](uint32_t i) { return bars + 16 + 8 * i; };
  auto PVDONE = [&](uint32_t i) { return bars + 32 + 8 * i; };
  // BUFS of each: keys / values expanded, read by the products (MLA: latents are both, KFULL and VEMPTY)
  auto KFULL = [&](uint32_t i) { return bars + 48 + 8 * i; };
  auto VFULL = [&](uint32_t i) { return bars + 128 + 8 * i; };
  auto KEMPTY = [&](uint32_t i) { return bars + 152 + 8 * i; };
  auto VEMPTY = [&](uint32_t i) { return bars + 176 + 8 * i; };
  auto FFULL = [&](uint32_t i) { return bars + 240 + 8 * i; };          // facts of a tile written, read
  auto FEMPTY = [&](uint32_t i) { return bars + 272 + 8 * i; };
  auto GFULL = [&](uint32_t i) { return bars + 304 + 8 * i; };          // packed tile landed, read
  auto GEMPTY = [&](uint32_t i) { return bars + 336 + 8 * i; };
  const uint32_t QFULL = bars + 368;
  unsigned char* misc = base_ptr + PL::OFF_MISC;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(misc + 384);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 388);
  int* s_b = reinterpret_cast<int*>(misc + 392);
  long long* s_off = reinterpret_cast<long long*>(misc + 400);          // offset inside sequence s_b, tiles of this CTA
  uint2* s_table = reinterpret_cast<uint2*>(misc + 512);
  float* s_qs = reinterpret_cast<float*>(misc + 640);
  float* s_m = s_qs + NH; float* s_d = s_m + NH; float* s_f = s_d + NH;
  int* s_lim = reinterpret_cast<int*>(s_f + NH);
  float* s_wmax = reinterpret_cast<float*>(s_lim + NH);      // also the sums of the four warps of a group
  int* s_row = reinterpret_cast<int*>(s_wmax + 4 * NH);      // output row of each query row, of this piece and of the next one
  unsigned char* s_fact = reinterpret_cast<unsigned char*>(s_row + 2 * NH);
  long long* s_warp = reinterpret_cast<long long*>(base_ptr + PL::OFF_P);      // totals of the warps, and as many words; before the weights
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, tid = threadIdx.x;
  auto fail = [&](int code) { atomicCAS(&g_paged4_status, 0, code); *abort_flag = 1; };

  if (tid == 0) {
    *abort_flag = 0;
    *reinterpret_cast<uint32_t*>(misc + 416) = 16u;
    for (int i = 0; i < 2; ++i) { mbar_init(SFULL(i), 1); mbar_init(PFULL(i), 32 * PL::SOFTMAX_WARPS); mbar_init(PVDONE(i), 1); }
    for (int i = 0; i < PL::BUFS; ++i) {
      mbar_init(KFULL(i), PL::EW); mbar_init(VFULL(i), PL::EW); mbar_init(KEMPTY(i), 1); mbar_init(VEMPTY(i), 1);
    }
    for (int i = 0; i < 4; ++i) { mbar_init(GFULL(i), 1); mbar_init(GEMPTY(i), PL::EW); }
    for (int i = 0; i < PL::FACTS; ++i) { mbar_init(FFULL(i), 1); mbar_init(FEMPTY(i), PL::SOFTMAX_WARPS + PL::EW + (PL::STAGED ? 1 : 0)); }
    mbar_init(QFULL, 32 * PL::SOFTMAX_WARPS);
    fence_mbar_init();
    if (base & 1023u) fail(100);                             // the operands' images need it
  }
  if (warp == W_MMA) { tmem_alloc(smem_u32((const void*)tmem_slot), PL::TM_COLS); tmem_relinquish(); }
  paged4_table_load(s_table, tid);
  chain_wait();
  chain_next();                                              // the whole grid is resident: nothing is displaced
  paged8_range<PL::THREADS>(p, (int)blockIdx.x, s_warp, s_b, s_off);
  __syncthreads();
  if (PL::GROUPS * ROWS < NH) {                              // weights of rows that do not exist: 0
    for (int i = tid; i < 2 * PL::P_BYTES / 16; i += PL::THREADS) reinterpret_cast<uint4*>(base_ptr + PL::OFF_P)[i] = make_uint4(0u, 0u, 0u, 0u);
    fence_proxy_async_smem();
    __syncthreads();
  }
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  Walk w;
  w.b = *s_b; w.off = s_off[0]; w.left = s_off[1]; w.fresh = true; w.n = 0;

  if (warp == W_LOOK) {
    // ------------------------------------------------------------------------------------------------- look-ups
    // Where the rows of a tile are and what their exponents are, for all other warps: lane i < 8 the page of rows [16 i, 16 i + 16),
    // every lane the exponents of four rows.  Three tiles are under way, one step each: page, exponents, written.
    bool ok = !*abort_flag;
    int j = 0;
    bool more = w.next(p);
    struct Tile { int page, hk, lo, mid, hi; bool any; };    // page: of this lane's rows; lo, mid, hi: PagedSpan from the tile's first row
    auto look = [&](Tile& y) {
      y.any = more;
      if (!more) return;
      const PagedSpan sp = w.t.s;
      const int row0 = w.t.row0(w.t0 + j), x = row0 + 16 * (lane & 7);
      y.lo = sp.n_rep - row0; y.mid = sp.tok0 - row0; y.hi = sp.n_tok - row0; y.hk = w.hk;
      y.page = -1;
      if (sp.any(x, 16) && (x >> p.page_log2) < p.width) y.page = p.table[(size_t)w.b * p.width + (x >> p.page_log2)];
      if (++j == w.n) { j = 0; more = w.next(p); }
    };
    // The pool's group of 16 rows, ~0: none.  (A group takes 512 bytes at least: 32 bits count those of more memory than there is.)
    auto group_of = [&](const Tile& y) {
      return y.any && (unsigned)y.page < (unsigned)p.n_pages
                 ? (((uint32_t)y.page * (uint32_t)p.Hkv + (uint32_t)y.hk) << (p.page_log2 - 4)) + (uint32_t)(lane & ((p.page >> 4) - 1)) : ~0u;
    };
    // exponents of this lane's four rows, and their shifts: DS / 64 (DP / 64) bytes a row
    constexpr int WS = PL::STAGED ? DS / 64 : 1, WP = PL::STAGED ? DP / 64 : 1;
    struct Scales { uint32_t v, k, ss[WS], sp[WP]; };
    auto scales_of = [&](uint32_t group, Scales& y) {
      const uint32_t gr = __shfl_sync(0xffffffffu, group, lane >> 2);
      y.v = y.k = 0;
#pragma unroll
      for (int i = 0; i < WS; ++i) y.ss[i] = 0;
#pragma unroll
      for (int i = 0; i < WP; ++i) y.sp[i] = 0;
      if (gr == ~0u) return;
      const size_t at = (size_t)gr * 4 + (lane & 3);
      y.v = __ldg(reinterpret_cast<const uint32_t*>(a.exp_v) + at);
      if (!PL::MLA) y.k = __ldg(reinterpret_cast<const uint32_t*>(a.exp_k) + at);
      if (PL::STAGED) {
#pragma unroll
        for (int i = 0; i < WS; ++i) y.ss[i] = __ldg(reinterpret_cast<const uint32_t*>(a.shift_sem) + at * WS + i);
#pragma unroll
        for (int i = 0; i < WP; ++i) y.sp[i] = __ldg(reinterpret_cast<const uint32_t*>(a.shift_pos) + at * WP + i);
      }
    };
    Tile t0, t1;
    uint32_t g0;
    Scales s0, s1;
    look(t0);
    look(t1);
    g0 = group_of(t0);
    scales_of(g0, s0);
    uint32_t f = 0, phase = 0;
    while (ok && t0.any) {
      const uint32_t g1 = group_of(t1);
      scales_of(g1, s1);
      Tile t2;
      look(t2);
      ok = mbar_wait(FEMPTY(f), phase ^ 1, abort_flag);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) { if (lane == 0) fail(ERR_WAIT_KV_EMPTY); break; }
      unsigned char* fact = s_fact + f * PL::FACT;
      const bool all = (__ballot_sync(0xffffffffu, g0 != ~0u) & 0xffu) == 0xffu && (t0.lo >= 128 || (t0.mid <= 0 && t0.hi >= 128));
      reinterpret_cast<uint32_t*>(fact)[lane] = s0.v;
      if (!PL::MLA) reinterpret_cast<uint32_t*>(fact + 128)[lane] = s0.k;
      if (lane < 8) reinterpret_cast<uint32_t*>(fact + PL::F_GROUP)[lane] = g0;
      if (lane == 8) *reinterpret_cast<int4*>(fact + PL::F_SPAN) = make_int4(all, t0.lo, t0.mid, t0.hi);
      if (PL::STAGED) {                                      // of absent rows: whatever they hold must be no NaN
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) { const int r = 4 * lane + i; m |= all || r < t0.lo || (r >= t0.mid && r < t0.hi) ? 0xffu << (8 * i) : 0u; }
        // a row's bytes: one (WS = 1), or two, which lie in one half of a word
#pragma unroll
        for (int i = 0; i < WS; ++i) reinterpret_cast<uint32_t*>(fact + PL::F_SHS)[lane * WS + i] = s0.ss[i] & (WS == 1 ? m : __byte_perm(m, 0u, i ? 0x3322 : 0x1100));
#pragma unroll
        for (int i = 0; i < WP; ++i) reinterpret_cast<uint32_t*>(fact + PL::F_SHP)[lane * WP + i] = s0.sp[i] & (WP == 1 ? m : __byte_perm(m, 0u, i ? 0x3322 : 0x1100));
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(FFULL(f));
      if (++f == PL::FACTS) { f = 0; phase ^= 1; }
      t0 = t1; t1 = t2; g0 = g1; s0 = s1;
    }
  } else if (PL::STAGED && warp == W_LOAD) {
    // --------------------------------------------------------------------------------------------- loads
    // A request for each page (or the 128 rows of it that belong to the tile) and part; a lane's requests are issued one after the other,
    // 200 clocks each, so the small arrays come another way (with the look-ups).
    const int n_tiles = (int)min(s_off[1], 0x7fffffffll);
    bool ok = !*abort_flag;
    uint32_t f = 0, fphase = 0, stage = 0, phase = 0;
    const int per = p.page >> 4;                             // groups of 16 rows to a request
#pragma unroll 1
    for (int t = 0; t < n_tiles && ok; ++t) {
      ok = mbar_wait(FFULL(f), fphase, abort_flag);
      if (ok) ok = mbar_wait(GEMPTY(stage), phase ^ 1, abort_flag);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) { if (lane == 0) fail(ERR_WAIT_KV_EMPTY); break; }
      // lane: request + 8 * part
      const uint32_t* groups = reinterpret_cast<const uint32_t*>(s_fact + f * PL::FACT + PL::F_GROUP);
      const int first = (lane & 7) * per;
      uint32_t gr = ~0u;
      // a page that is present in part: groups without a present row are not looked up, the page starts at its first one that is
      if (first < 8)
        for (int i = 0; i < per; ++i) { const uint32_t y = groups[first + i]; if (gr == ~0u && y != ~0u) gr = y - i; }
      const unsigned there = __popc(__ballot_sync(0xffffffffu, gr != ~0u) & 0xffu);
      if (lane == 0) mbar_expect_tx(GFULL(stage), there * p.page * ((DS + DP) / 2));
      __syncwarp();
      if (lane == 0) mbar_arrive(FEMPTY(f));
      const uint32_t at = base + PL::OFF_STAGE + stage * PL::STAGE;
      if (gr != ~0u && lane < 16) {
        if (lane < 8) bulk_copy(at + first * 16 * (DS / 2), a.sem + (size_t)gr * (16 * (DS / 2)), p.page * (DS / 2), GFULL(stage));
        else bulk_copy(at + PL::ST_POS + first * 16 * (DP / 2), a.pos + (size_t)gr * (16 * (DP / 2)), p.page * (DP / 2), GFULL(stage));
      }
      __syncwarp();
      if (++f == PL::FACTS) { f = 0; fphase ^= 1; }
      if (++stage == PL::STAGES) { stage = 0; phase ^= 1; }
    }
  } else if (warp >= W_EXP && warp < W_MMA) {
    // ----------------------------------------------------------------------------------------------- expansion
    // A thread takes 32 values (16 bytes of codes) of a row at a time, STAGED: from the copies in shared memory, else from HBM to registers
    // while it expands those of the tile before.  Eight neighbouring lanes write two rows, so that their units fall on all banks of the
    // swizzled image.
    const int et = tid - 32 * W_EXP;
    const int n_tiles = (int)min(s_off[1], 0x7fffffffll);
    bool ok = !*abort_flag;
    const uint32_t sixteen = *reinterpret_cast<const volatile uint32_t*>(misc + 416);
    auto wait = [&](uint32_t bar, uint32_t ph, int code) {
      if (ok && !mbar_wait(bar, ph, abort_flag)) { fail(code); ok = false; }
      ok = __all_sync(0xffffffffu, ok);
      return ok;
    };
    // STAGED: goes on after a failure too (nothing that it would read from then on is an address)
    auto hold = [&](uint32_t bar, uint32_t ph, int code) { if (!mbar_wait(bar, ph, abort_flag)) fail(code); };
    auto signal = [&](uint32_t bar) {
      __syncwarp();
      if (lane == 0) mbar_arrive(bar);
    };
    constexpr bool LATENT = PL::MLA && DS == 512;
    constexpr int US = PL::VW / 32, UP = DP / 32, STEP = 32 * PL::EW, PER_CHUNK = US * 128 / STEP;
    // unit i of this thread: row and unit in the row, place in the expanded tile
    // (512 latents: PER_CHUNK of each chunk), neighbouring threads neighbouring units
    auto sem_row = [&](int i) { return (et + STEP * (LATENT ? i % PER_CHUNK : i)) / US; };
    const int sem_u = et % US, pos_u = et % UP;
    auto pos_row = [&](int i) { return (et + STEP * i) / UP; };
    const uint32_t sem_to = (PL::MLA ? 0 : PL::K_BYTES) + swz<PL::VW>(sem_row(0), 2 * sem_u);
    const uint32_t pos_to = PL::KSEM * 16384 + swz<DP>(pos_row(0), 2 * pos_u);
    struct Facts { bool all; int lo, mid, hi; const uint32_t* group; };
    auto has = [&](const Facts& f, int r) { return f.all || r < f.lo || (r >= f.mid && r < f.hi); };
    struct Unit { uint4 v; uint32_t s; };
    // N units of the next tile on their way (a tile without absent rows takes the short path)
    auto load = [&](auto count, Unit* x, int i0, const Facts& f, auto row_of, const uint8_t* codes, const uint8_t* shifts, int d, int u) {
      constexpr int N = decltype(count)::value;
      uint32_t gr[N];
#pragma unroll
      for (int i = 0; i < N; ++i) gr[i] = f.group[row_of(i0 + i) >> 4];
      codes += u * 16; shifts += u >> 1;
      if (f.all) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const size_t row = (size_t)gr[i] * 16 + (row_of(i0 + i) & 15);
          x[i].v = load_stream(codes + row * (d / 2));
          x[i].s = (uint32_t)__ldg(shifts + row * (d / 64));
        }
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int r = row_of(i0 + i);
          x[i].v = make_uint4(0u, 0u, 0u, 0u);
          x[i].s = 0;
          if (gr[i] != ~0u && has(f, r)) {                   // what absent rows hold is left alone
            const size_t row = (size_t)gr[i] * 16 + (r & 15);
            x[i].v = load_stream(codes + row * (d / 2));
            x[i].s = (uint32_t)__ldg(shifts + row * (d / 64));
          }
        }
      }
    };
    // N units expanded; dst: from the start of shared memory, `step` from one to the next
    auto put = [&](auto count, const Unit* x, int u, uint32_t dst, uint32_t step) {
      constexpr int N = decltype(count)::value;
      uint2 t[N];
#pragma unroll
      for (int i = 0; i < N; ++i) t[i] = s_table[(x[i].s >> (4 * (u & 1))) & 15];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const uint2 x0 = paged4_expand(x[i].v.x, t[i], sixteen), x1 = paged4_expand(x[i].v.y, t[i], sixteen), x2 = paged4_expand(x[i].v.z, t[i], sixteen),
                    x3 = paged4_expand(x[i].v.w, t[i], sixteen);
        *reinterpret_cast<uint4*>(base_ptr + dst + i * step) = make_uint4(x0.x, x0.y, x1.x, x1.y);
        *reinterpret_cast<uint4*>(base_ptr + (dst ^ 16u) + i * step) = make_uint4(x2.x, x2.y, x3.x, x3.y);
      }
    };
    constexpr int BATCH = LATENT ? PER_CHUNK : PL::U_SEM;
    using CP = std::integral_constant<int, PL::U_POS>;
    using CS = std::integral_constant<int, BATCH>;
    auto load_sem = [&](Unit* x, const Facts& f, int i0) { load(CS(), x, i0, f, sem_row, a.sem, a.shift_sem, DS, sem_u + (LATENT ? US * (i0 / PER_CHUNK) : 0)); };
    auto load_pos = [&](Unit* x, const Facts& f) { load(CP(), x, 0, f, pos_row, a.pos, a.shift_pos, DP, pos_u); };
    uint32_t ff = 0, fphase = 0;
    auto facts = [&](Facts& f, bool any) {                   // of the next tile; its groups are read until `signal`
      if (!any) return;
      if (!wait(FFULL(ff), fphase, ERR_WAIT_KV_FULL)) return;
      const unsigned char* fact = s_fact + ff * PL::FACT;
      const int4 y = *reinterpret_cast<const int4*>(fact + PL::F_SPAN);
      f = Facts{y.x != 0, y.y, y.z, y.w, reinterpret_cast<const uint32_t*>(fact + PL::F_GROUP)};
    };
    auto facts_done = [&](bool any) {
      if (!any) return;
      signal(FEMPTY(ff));
      if (++ff == PL::FACTS) { ff = 0; fphase ^= 1; }
    };
    uint32_t buf = 0, use = 0;                               // use: how often the buffer has been filled before
    Unit sem[PL::U_SEM], pos[PL::U_POS];
    Facts fx = {};
    constexpr uint32_t SEM_APART = STEP / US * PL::VW, POS_APART = (STEP / UP) * DP;
    if constexpr (!PL::STAGED) {
      facts(fx, n_tiles > 0);
      if (n_tiles > 0 && ok) {
        load_pos(pos, fx);
#pragma unroll
        for (int i = 0; i < PL::U_SEM; i += BATCH) load_sem(sem + i, fx, i);
        facts_done(true);
      }
#pragma unroll 1
      for (int t = 0; t < n_tiles && ok; ++t) {
        const bool any = t + 1 < n_tiles;
        const uint32_t tile = buf * PL::TILE;
        if (!wait(VEMPTY(buf), (use & 1) ^ 1, ERR_WAIT_O_DONE)) break;
        put(CP(), pos, pos_u, tile + pos_to, POS_APART);
#pragma unroll
        for (int c = 0; c < NV; ++c) put(CS(), sem + BATCH * c, sem_u, tile + sem_to + c * 16384, SEM_APART);
        // the fence waits for loads under way too: those of the next tile come behind it
        fence_proxy_async_smem();
        signal(KFULL(buf));
        facts(fx, any);
        if (any) {
          load_pos(pos, fx);
#pragma unroll
          for (int c = 0; c < NV; ++c) load_sem(sem + BATCH * c, fx, BATCH * c);
        }
        facts_done(any);
        if (++buf == PL::BUFS) { buf = 0; ++use; }
      }
    } else {
      uint32_t stage = 0, phase = 0;
#pragma unroll 1
      for (int t = 0; t < n_tiles; ++t) {
        const uint32_t tile = buf * PL::TILE;
        hold(GFULL(stage), phase, ERR_WAIT_KV_FULL);         // (and so the facts are there: the loading warp has waited for them)
        const unsigned char* fact = s_fact + ff * PL::FACT;
        const unsigned char* st = base_ptr + PL::OFF_STAGE + stage * PL::STAGE;
#pragma unroll
        for (int i = 0; i < PL::U_POS; ++i) {
          pos[i].v = *reinterpret_cast<const uint4*>(st + PL::ST_POS + (et + STEP * i) * 16);
          pos[i].s = fact[PL::F_SHP + pos_row(i) * (DP / 64) + (pos_u >> 1)];
        }
#pragma unroll
        for (int i = 0; i < PL::U_SEM; ++i) {
          sem[i].v = *reinterpret_cast<const uint4*>(st + (et + STEP * i) * 16);
          sem[i].s = fact[PL::F_SHS + sem_row(i) * (DS / 64) + (sem_u >> 1)];
        }
        __syncwarp();
        if (lane == 0) { mbar_arrive(GEMPTY(stage)); mbar_arrive(FEMPTY(ff)); }
        if (++ff == PL::FACTS) ff = 0;
        if (++stage == PL::STAGES) { stage = 0; phase ^= 1; }
        hold(PL::MLA ? VEMPTY(buf) : KEMPTY(buf), (use & 1) ^ 1, ERR_WAIT_O_DONE);
        put(CP(), pos, pos_u, tile + pos_to, POS_APART);
        if constexpr (!PL::MLA) {
          fence_proxy_async_smem();
          signal(KFULL(buf));
          hold(VEMPTY(buf), (use & 1) ^ 1, ERR_WAIT_O_DONE);
        }
        put(CS(), sem, sem_u, tile + sem_to, SEM_APART);
        fence_proxy_async_smem();
        signal(PL::MLA ? KFULL(buf) : VFULL(buf));
        if (++buf == PL::BUFS) { buf = 0; ++use; }
      }
    }
  } else if (warp == W_MMA) {
    // ----------------------------------------------------------------------------------------------------- MMA
    const uint32_t leader = elect_one();
    constexpr uint32_t ID_S = umma_idesc_f8(128, 2 * NH, 0, false, false);
    constexpr uint32_t ID_O = umma_idesc_f8(128, 2 * NH, 0, true, true);
    uint32_t g = 0, seg = 0;
    bool ok = !*abort_flag;
    struct Ring { uint32_t buf, phase; __device__ __forceinline__ void next() { if (++buf == PL::BUFS) { buf = 0; phase ^= 1; } } };
    Ring sb = {0, 0}, ob = {0, 0};                           // expanded tiles whose S and O come next
    auto wait = [&](uint32_t bar, uint32_t ph, int code) {
      ok = ok && mbar_wait(bar, ph, abort_flag);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok && lane == 0) fail(code);
      return ok;
    };
    auto issue_s = [&](uint32_t t) {
      const uint32_t buf = t & 1, d = tmem + PL::TM_S + buf * 2 * NH, tile = base + sb.buf * PL::TILE;
      tc_fence_after();
      uint32_t acc = 0;
#pragma unroll 1
      for (int c = 0; c < PL::KSEM; ++c) {
        const uint64_t ad = desc_rows(tile + c * 16384, 128, 16), bd = desc_rows(base + PL::OFF_Q + c * 2 * NH * 128, 128, 16);
#pragma unroll
        for (int k = 0; k < 4; ++k) { umma_f8_elected(leader, d, desc_add(ad, 2 * k), desc_add(bd, 2 * k), ID_S, acc); acc = 1; }
      }
      const uint64_t ad = desc_rows(tile + PL::KSEM * 16384, DP, 16), bd = desc_rows(base + PL::OFF_Q + PL::KSEM * 2 * NH * 128, DP, 16);
#pragma unroll
      for (int k = 0; k < DP / 32; ++k) { umma_f8_elected(leader, d, desc_add(ad, 2 * k), desc_add(bd, 2 * k), ID_S, acc); acc = 1; }
      umma_commit_elected(leader, SFULL(buf));
      if (!PL::MLA) umma_commit_elected(leader, KEMPTY(sb.buf));
      sb.next();
    };
    auto issue_o = [&](uint32_t t, bool first) {
      const uint32_t buf = t & 1;
      if (!PL::MLA && !wait(VFULL(ob.buf), ob.phase, ERR_WAIT_KV_FULL)) return;
      tc_fence_after();
      const uint64_t pd = desc_rows(base + PL::OFF_P + buf * PL::P_BYTES, 2 * NH, 128);
#pragma unroll 1
      for (int c = 0; c < NV; ++c) {
        // 64-wide values: M stays 128, the second half of the operand is the unused half of their 16 KB and the output
        // lanes it feeds are never read
        const uint64_t ad = desc_rows(base + ob.buf * PL::TILE + (PL::MLA ? c * 16384 : PL::K_BYTES), PL::VW, 8192);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          umma_f8_elected(leader, tmem + c * 2 * NH, desc_add(ad, k * 2 * PL::VW), desc_add(pd, k * 4 * NH), ID_O, (!first || k > 0) ? 1u : 0u);
      }
      umma_commit_elected(leader, PVDONE(buf));
      umma_commit_elected(leader, VEMPTY(ob.buf));
      ob.next();
    };
    while (ok && w.next(p)) {
      if (!wait(QFULL, seg & 1, ERR_WAIT_Q)) break;
      ++seg;
      tc_fence_after();
      // Each kind in order; of the next S and the next O whichever can go first.  S of a tile takes the columns of the last but one,
      // whose weights have been written (and S read) before its O is issued.
      uint32_t js = 0, jo = 0;
      const uint32_t n = (uint32_t)w.n;
      long long since = clock64();
      uint32_t tries = 0;
#pragma unroll 1
      while (jo < n && ok) {
        bool idle = true;
        if (js < n && js < jo + 2 && __all_sync(0xffffffffu, phase_done(KFULL(sb.buf), sb.phase))) { issue_s(g + js); ++js; idle = false; }
        if (jo < js && ok && __all_sync(0xffffffffu, phase_done(PFULL((g + jo) & 1), ((g + jo) >> 1) & 1))) { issue_o(g + jo, jo == 0); ++jo; idle = false; }
        if (!idle) { since = clock64(); tries = 0; }
        else if ((++tries & 63u) == 0 && (*abort_flag || clock64() - since > WAIT_TIMEOUT_CYCLES)) { if (lane == 0) fail(ERR_WAIT_P_FULL); ok = false; }
        ok = __all_sync(0xffffffffu, ok);
      }
      g += n;
    }
  } else {
    // ------------------------------------------------------------------------------------- softmax, epilogue
    const int grp = warp >> 2, quad = warp & 3, t = tid & 127, hb = ROWS * grp;    // this thread: key t of a tile, rows hb .. hb + ROWS - 1
    const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
    uint32_t g = 0, seg = 0;
    bool ok = !*abort_flag;
    float l[ROWS];
    // splits this group's query rows of a unit into e4m3 terms and writes them where S reads them
    auto load_q = [&](const Walk& u, uint32_t which) {
      constexpr int VS = PL::KSEM * 16, VQ = VS + DP / 8, NL = (VQ + 31) / 32;   // 8-element vectors of a row
      const int n_rows = p.q_len * p.rep - u.blk * NH;
#pragma unroll 2
      for (int r = hb + quad; r < hb + ROWS; r += 4) {
        const int gr = u.blk * NH + r, qt = gr / p.rep;
        const int row = ((int)(u.b * p.q_len) + qt) * p.Hq + u.hk * p.rep + (gr - qt * p.rep);
        uint4 v[NL];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          const int c = lane + 32 * i;
          v[i] = make_uint4(0u, 0u, 0u, 0u);
          if (r < n_rows && c < VQ)
            v[i] = *reinterpret_cast<const uint4*>(c < VS ? p.q_sem + (size_t)row * DS + 8 * c : p.q_pos + (size_t)row * DP + 8 * (c - VS));
        }
#pragma unroll
        for (int i = 0; i < NL; ++i) top = max(top, max_abs_bf16(v[i]));
        top = __reduce_max_sync(0xffffffffu, top);
        const int e = query_exponent(top);
        const float f = exp2_int(e);
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          const int c = lane + 32 * i;
          if (c >= VQ) continue;
          uint32_t hi[2], lo[2];
          split_e4m3(v[i], f, hi, lo);
          const bool sem = c < VS;
          const int chunk = sem ? c / 16 : PL::KSEM, u16 = (sem ? c % 16 : c - VS) / 2, half = c & 1;
          unsigned char* q = base_ptr + PL::OFF_Q + chunk * 2 * NH * 128 + 8 * half;
          const uint32_t oh = sem ? swz<128>(r, u16) : swz<DP>(r, u16), ol = sem ? swz<128>(NH + r, u16) : swz<DP>(NH + r, u16);
          *reinterpret_cast<uint2*>(q + oh) = make_uint2(hi[0], hi[1]);
          *reinterpret_cast<uint2*>(q + ol) = make_uint2(lo[0], lo[1]);
        }
        // a row with an infinity or a NaN has no finite logit; rows behind the last one never have weight
        if (lane == 0) {
          s_qs[r] = r < n_rows ? (top >= 0x7f80u ? __int_as_float(0x7fffffff) : exp2_int(-e)) : 0.f;
          s_m[r] = r < n_rows ? 0.f : 3.0e38f;
          s_lim[r] = u.t.s.n_tok - p.q_len + 1 + qt;
          s_row[(which & 1) * NH + r] = r < n_rows ? row : -1;
        }
      }
      fence_proxy_async_smem();
      mbar_arrive(QFULL);
      group_sync(grp);
    };
    bool more = w.next(p);
    if (more) load_q(w, 0);
    while (more) {
      const PagedSpan sp = w.t.s;
      const int* rows = s_row + (seg & 1) * NH + hb;
      bool unset = t < ROWS && rows[t % ROWS] >= 0;          // thread h of the group: its row has no maximum yet
#pragma unroll
      for (int i = 0; i < ROWS; ++i) l[i] = 0.f;
#pragma unroll 1
      for (int j = 0; j < w.n; ++j, ++g) {
        const int row0 = w.t.row0(w.t0 + j), x = row0 + t;
        const uint32_t buf = g & 1;
        ok = mbar_wait(FFULL(g % PL::FACTS), (g / PL::FACTS) & 1, abort_flag);
        if (!ok) fail(ERR_WAIT_KV_FULL);
        __syncwarp();
        const unsigned char* fact = s_fact + (g % PL::FACTS) * PL::FACT;
        const int ve = fact[t], ke = PL::MLA ? ve : fact[128 + t];
        const bool valid = reinterpret_cast<const uint32_t*>(fact + PL::F_GROUP)[t >> 4] != ~0u && sp.has(x);
        __syncwarp();
        if (lane == 0) mbar_arrive(FEMPTY(g % PL::FACTS));
        // The row sum needs 2^(y - M), the weight t = 2^(y - M + log2 f_v + T): both are multiples of e = 2^(y - M + half), half way
        // between them, so that neither is lost below 2^-126 where the factors of a sequence span more than fp32 does.
        const float half = 0.5f * ((float)paged4_log2_factor(ve) + paged8_t_bits(NH)), f_t = ex2(half), f_l = ex2(paged8_t_bits(NH) - half);
        const float kf = paged4_factor(ke) * p.scale_log2, cb = half + (x < sp.n_rep ? p.bias_log2 : 0.f);
        const float offset = weight_offset(x);
        const bool limited = row0 + 127 >= sp.n_tok - p.q_len + 1;      // some query may not see some row of this tile

        ok = mbar_wait(SFULL(buf), (g >> 1) & 1, abort_flag);
        if (!ok) fail(ERR_WAIT_S_FULL);
        __syncwarp();
        tc_fence_after();
        float z[ROWS];
        float zmax = -INFINITY;
        {
          uint32_t hi[ROWS], lo[ROWS];
          const uint32_t at = tmem + lane_base + PL::TM_S + buf * 2 * NH + hb;
          tmem_ld<ROWS>(at, hi);
          tmem_ld<ROWS>(at + NH, lo);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < ROWS; i += 4) {
            const float4 q4 = *reinterpret_cast<const float4*>(s_qs + hb + i), m4 = *reinterpret_cast<const float4*>(s_m + hb + i);
            const float qq[4] = {q4.x, q4.y, q4.z, q4.w}, mm[4] = {m4.x, m4.y, m4.z, m4.w};
#pragma unroll
            for (int k = 0; k < 4; ++k)
              z[i + k] = fmaf(__uint_as_float(hi[i + k]) + __uint_as_float(lo[i + k]), kf * qq[k], cb - mm[k]);
          }
        }
        if (limited || !__all_sync(0xffffffffu, valid)) {
#pragma unroll
          for (int i = 0; i < ROWS; ++i) z[i] = valid && (!limited || x < s_lim[hb + i]) ? z[i] : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < ROWS; i += 2) zmax = max3(zmax, z[i], z[i + 1]);
        const bool raise = group_or(grp, zmax + half > T4_MAX || unset);
        if (raise) {
          // raise the maxima: per row the largest log2 t of the tile
#pragma unroll
          for (int i = 0; i < ROWS; ++i) {
            const float m = warp_max_f32(z[i] + half);
            if (lane == i) s_wmax[quad * NH + hb + i] = m;
          }
          group_sync(grp);
          if (t < ROWS) {
            const int h = hb + t;
            const float m = fmaxf(fmaxf(s_wmax[h], s_wmax[NH + h]), fmaxf(s_wmax[2 * NH + h], s_wmax[3 * NH + h]));
            float d = 0.f, f = 1.f;
            if (unset ? m > -INFINITY : m > paged8_t_bits(NH)) {
              d = m - paged8_t_bits(NH);
              f = unset ? 1.f : ex2(-d);                     // nothing has been added under an unset maximum
              s_m[h] += d;
              unset = false;
            }
            s_d[h] = d; s_f[h] = f;
          }
          group_sync(grp);
#pragma unroll
          for (int i = 0; i < ROWS; ++i) { z[i] -= s_d[hb + i]; l[i] *= s_f[hb + i]; }
        }
        if (g > 1) {                                         // the weights of the tile before the last one have been read
          ok = mbar_wait(PVDONE(buf), ((g >> 1) - 1) & 1, abort_flag);
          if (!ok) fail(ERR_WAIT_O_DONE);
        }
        if (raise && j > 0) {                                // O is complete up to the last tile
          ok = mbar_wait(PVDONE(buf ^ 1), ((g - 1) >> 1) & 1, abort_flag);
          if (!ok) fail(ERR_WAIT_O_DONE);
          __syncwarp();
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < 2 * NV; ++c) {
            uint32_t o[ROWS];
            tmem_ld<ROWS>(tmem + lane_base + c * NH + hb, o);
            tmem_wait_ld();
#pragma unroll
            for (int k = 0; k < ROWS; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * s_f[hb + k]);
            tmem_st<ROWS>(tmem + lane_base + c * NH + hb, o);
          }
          tmem_wait_st();
        }
        {
          unsigned char* ph = base_ptr + PL::OFF_P + buf * PL::P_BYTES;
          uint32_t wh[ROWS / 4], wl[ROWS / 4];
#pragma unroll
          for (int i = 0; i < ROWS / 4; ++i) {
            float tt[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float e = ex2(z[4 * i + k]);
              tt[k] = e * f_t;
              l[4 * i + k] = fmaf(e, f_l, l[4 * i + k]);
            }
            wh[i] = e4m3x4_from_float(tt[0], tt[1], tt[2], tt[3]);
            const float4 h = e4m3x4_to_float4(wh[i]);        // what the first term leaves is exact: at most 2^4, times the gain 2^8
            wl[i] = e4m3x4_from_float(fmaf(tt[0] - h.x, LO4_GAIN, offset), fmaf(tt[1] - h.y, LO4_GAIN, offset),
                                      fmaf(tt[2] - h.z, LO4_GAIN, offset), fmaf(tt[3] - h.w, LO4_GAIN, offset));
          }
          const uint32_t oh = swz<2 * NH>(t, hb / 16) + hb % 16, ol = swz<2 * NH>(t, (NH + hb) / 16) + hb % 16;
          if constexpr (ROWS == 8) {
            *reinterpret_cast<uint2*>(ph + oh) = make_uint2(wh[0], wh[1]);
            *reinterpret_cast<uint2*>(ph + ol) = make_uint2(wl[0], wl[1]);
          } else {
            *reinterpret_cast<uint32_t*>(ph + oh) = wh[0];
            *reinterpret_cast<uint32_t*>(ph + ol) = wl[0];
          }
        }
        fence_proxy_async_smem();
        tc_fence_before();
        mbar_arrive(PFULL(buf));
      }
      // ---- this piece is done: its sums and maxima, then the next unit's queries (S of this piece is complete), then O
      const bool whole = w.n == w.t.n;
      const size_t part = (size_t)2 * blockIdx.x + (seg == 0 ? 0 : 1);
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        float v = l[i];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (lane == i) s_wmax[quad * NH + hb + i] = v;
      }
      group_sync(grp);
      if (t < ROWS) {
        const int h = hb + t;
        const float sum = (s_wmax[h] + s_wmax[NH + h]) + (s_wmax[2 * NH + h] + s_wmax[3 * NH + h]);
        if (!whole) {
          float* ml = p.part + (size_t)2 * p.grid * NH * DS + part * 2 * NH;
          ml[h] = unset ? -INFINITY : s_m[h]; ml[NH + h] = sum;
        } else if (p.lse && rows[t] >= 0) {
          p.lse[rows[t]] = sum == 0.f ? -INFINITY : (s_m[h] + log2f(sum) - paged8_t_bits(NH)) * 0.6931471805599453f;
        }
        s_f[h] = whole ? (sum == 0.f ? 0.f : 1.f / sum) : 1.f;
      }
      group_sync(grp);
      more = w.next(p);
      if (more) load_q(w, seg + 1);
      ok = mbar_wait(PVDONE((g - 1) & 1), ((g - 1) >> 1) & 1, abort_flag);
      if (!ok) fail(ERR_WAIT_O_DONE);
      __syncwarp();
      tc_fence_after();
#pragma unroll 1
      for (int c = 0; c < NV; ++c) {
        uint32_t o[ROWS], o2[ROWS];
        tmem_ld<ROWS>(tmem + lane_base + c * 2 * NH + hb, o);
        tmem_ld<ROWS>(tmem + lane_base + c * 2 * NH + NH + hb, o2);
        tmem_wait_ld();
#pragma unroll
        for (int k = 0; k < ROWS; ++k) o[k] = __float_as_uint(fmaf(__uint_as_float(o2[k]), 1.f / LO4_GAIN, __uint_as_float(o[k])));
        const int d = c * 128 + t;
        if (DS >= 128 || t < DS) {
          if (whole) {
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
              const float f = s_f[hb + k];
              const int row = rows[k];
              if (row >= 0) p.out[(size_t)row * DS + d] = __float2bfloat16_rn(f == 0.f ? 0.f : __uint_as_float(o[k]) * f);   // no key: O may be 0 * NaN
            }
          } else {
            float* dst = p.part + part * NH * DS + (size_t)hb * DS + d;
#pragma unroll
            for (int k = 0; k < ROWS; ++k) dst[(size_t)k * DS] = __uint_as_float(o[k]);
          }
        }
      }
      tc_fence_before();
      ++seg;
      group_sync(grp);                                       // s_f is written again by the next piece
    }
  }
  // ---- free TMEM.  Behind the barrier no warp gives up any more; if one did, this one keeps the CTA's memory until straggling copies have landed
  __syncthreads();
  if (warp == W_MMA) {
    if (*abort_flag) {
      const long long t0c = clock64();
      while (clock64() - t0c < 2000000ll) __nanosleep(1000);
      __syncwarp();
    }
    tc_fence_after();
    tmem_dealloc(tmem, PL::TM_COLS);
  }
}

// ------------------------------------------------------------------------------------------------------------- host
// Query rows that share a tile of keys: 16 or 32, the smaller one that holds all rows of a KV head (16 rows of GQA, 64 x 5056: 157 us, with
// room for 32: 202; MLA 512 + 64: 55 / 69), else blocks of 32.  Every block expands all tiles again: 64 x 5056 rows, GQA 128 on 8 KV heads with
// 32 / 33 / 64 / 112 / 128 rows a KV head 206 / 384 / 396 / 775 / 780 us, GQA 64 with 32 / 64 / 128 184 / 351 / 687, MLA 128 + 64 with 32 / 64 / 128 / 512
// 38 / 56 / 100 / 362.  MLA 512 + 64 with more than 64 rows: blocks of 128 on CTA pairs, whatever the lengths (which the host does not know),
// although single CTAs are faster where the tiles are few (66 rows: columns two and three, level in the fourth; 128 rows: the third).  Blocks of 32 on single CTAs against pairs:
//                 64 x 5056 rows   20 x up to 5056   1 x 2528   12 x up to 9001   100 x 5056   4 x 60000
//   40 rows           119 / 120 us      42 / 54        21 / 25       44 / 57       178 / 188     91 / 104
//   64 rows           120 / 123         43 / 56        21 / 26       44 / 57       184 / 198     90 / 103
//   66 rows           173 / 123         53 / 56        21 / 26       55 / 57       251 / 198    124 / 104
//   128 rows          228 / 125         66 / 59        21 / 26       66 / 58       347 / 213    158 / 104
static int paged4_rows_per_tile(const lca_params* p, int q_len) {
  const long long rows = (long long)q_len * (p->n_q_heads / p->n_kv_heads);
  if (p->d_sem == 512 && rows > 64) return 128;
  return rows <= 16 ? 16 : 32;
}
// CTAs (or pairs) that share the work: all that are resident at once.
static int paged4_grid(const lca_params* p, int nh) { return nh == 128 ? 74 : p->d_sem == 512 || nh == 32 ? 148 : 2 * 148; }
size_t attn_paged4_workspace_bytes(const lca_params* p, int q_len) {
  const int nh = paged4_rows_per_tile(p, q_len), grid = paged4_grid(p, nh);
  return (size_t)2 * grid * (nh * (size_t)p->d_sem + 2 * nh) * sizeof(float) + ((size_t)p->batch + 2) * sizeof(long long) + 64;
}

template <class PL>
static int paged4_launch(Paged4Params& P, cudaStream_t stream) {
  auto kern = attn_paged4_kernel<PL>;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, PL::SMEM) != cudaSuccess) return LCA_ERR_CUDA;
  const int st = launch_chained(kern, (unsigned)P.b.grid, PL::THREADS, PL::SMEM, stream, 1, P);
  if (st != LCA_OK) return st;
  return paged8_combine_launch<PL::DS, PL::NH>(P.b, stream);
}
template <bool MLA, int DS, int DP>
static int paged4_launch_rows(Paged4Params& P, int nh, cudaStream_t stream) {
  const long long rows = (long long)P.b.q_len * P.b.rep;
  if constexpr (DS == 512) if (nh == 128) return attn_paged4_pair_launch(P, stream);
  // Groups of softmax warps and rows a thread: what exists is computed, no more (GQA 128, 64 x 5056 rows: 4 rows 121 us, as 8 rows 134, as 16 152; 8 rows 135,
  // as 16 155; GQA 64, 4 rows: 90, 98, 123).
  if (nh == 32) return paged4_launch<Paged4Plan<MLA, DS, DP, 32, 4, 8>>(P, stream);
  if (rows <= 4) return paged4_launch<Paged4Plan<MLA, DS, DP, 16, 1, 4>>(P, stream);
  if (rows <= 8) return paged4_launch<Paged4Plan<MLA, DS, DP, 16, 1, 8>>(P, stream);
  return paged4_launch<Paged4Plan<MLA, DS, DP, 16, 2, 8>>(P, stream);
}

static void paged4_params(const Paged4Attn& q, Paged4Params& P) {
  const lca_params* p = q.p;
  const lca_paged4* c = q.c;
  const bool mla = p->variant == LCA_VARIANT_MLA;
  memset(&P, 0, sizeof(P));
  P.sem = (const uint8_t*)c->pages_sem; P.pos = (const uint8_t*)c->pages_pos;
  P.shift_sem = c->shift_sem; P.shift_pos = c->shift_pos;
  P.exp_v = c->exp_sem; P.exp_k = mla ? c->exp_sem : c->exp_pos;
  Paged8Params& b = P.b;
  b.q_sem = (const bf16*)q.q_sem; b.q_pos = (const bf16*)q.q_pos; b.table = c->block_table;
  b.n_rep = q.n_rep; b.n_tok = q.n_tok; b.out = (bf16*)q.out; b.lse = q.lse;
  b.out_wide = (reinterpret_cast<uintptr_t>(q.out) & 31u) == 0;
  b.B = p->batch; b.Hq = p->n_q_heads; b.Hkv = p->n_kv_heads; b.q_len = q.q_len; b.g = q.n_rep ? p->group_size : 1;
  b.page = c->page_size; b.page_log2 = c->page_size == 16 ? 4 : c->page_size == 32 ? 5 : c->page_size == 64 ? 6 : 7;
  b.n_pages = c->n_pages; b.width = c->table_width; b.rep = b.Hq / b.Hkv;
  b.scale_log2 = p->softmax_scale * 1.4426950408889634f; b.bias_log2 = p->rep_logit_bias * 1.4426950408889634f;
}

int attn_paged4_simt_launch(const Paged4Attn& q) {
  const lca_params* p = q.p;
  Paged4Params P;
  paged4_params(q, P);
  const long long n_rows = (long long)p->batch * q.q_len * p->n_q_heads;
  const unsigned grid = (unsigned)((n_rows + 3) / 4);
  const float scale = p->softmax_scale, bias = p->rep_logit_bias;
  if (p->variant == LCA_VARIANT_MLA) {
    if (p->d_sem == 512) attn_paged4_simt_kernel<512, 64, true><<<grid, 128, 0, q.stream>>>(P, scale, bias, n_rows);
    else attn_paged4_simt_kernel<128, 64, true><<<grid, 128, 0, q.stream>>>(P, scale, bias, n_rows);
  } else if (p->d_sem == 128) attn_paged4_simt_kernel<128, 128, false><<<grid, 128, 0, q.stream>>>(P, scale, bias, n_rows);
  else attn_paged4_simt_kernel<64, 64, false><<<grid, 128, 0, q.stream>>>(P, scale, bias, n_rows);
  note_launch();
  return cudaGetLastError() == cudaSuccess ? LCA_OK : LCA_ERR_CUDA;
}

int attn_paged4_launch(const Paged4Attn& q) {
  const lca_params* p = q.p;
  Paged4Params P;
  paged4_params(q, P);
  Paged8Params& b = P.b;
  const int nh = paged4_rows_per_tile(p, q.q_len);
  b.n_blk = (int)(((long long)b.q_len * b.rep + nh - 1) / nh);
  b.grid = paged4_grid(p, nh);
  b.part = reinterpret_cast<float*>((reinterpret_cast<uintptr_t>(q.ws) + 31) & ~(uintptr_t)31);
  const size_t part_bytes = (size_t)2 * b.grid * (nh * (size_t)p->d_sem + 2 * nh) * sizeof(float);
  b.prefix = reinterpret_cast<long long*>(reinterpret_cast<char*>(b.part) + (part_bytes + 15) / 16 * 16);
  if ((long long)b.B * b.Hkv * b.n_blk * ((long long)nh * p->d_sem / 512) > 0x7fffffffll) return LCA_ERR_UNSUPPORTED_SHAPE;
  if (p->variant == LCA_VARIANT_MLA) return p->d_sem == 512 ? paged4_launch_rows<true, 512, 64>(P, nh, q.stream)
                                                            : paged4_launch_rows<true, 128, 64>(P, nh, q.stream);
  return p->d_sem == 128 ? paged4_launch_rows<false, 128, 128>(P, nh, q.stream) : paged4_launch_rows<false, 64, 64>(P, nh, q.stream);
}

int attn_paged4_take_status() {
  int st = 0;
  if (cudaMemcpyFromSymbol(&st, g_paged4_status, sizeof(int)) != cudaSuccess) return -1;
  if (st != 0) {
    int zero = 0;
    cudaMemcpyToSymbol(g_paged4_status, &zero, sizeof(int));
  }
  const int pair = attn_paged4_pair_take_status();
  return pair != 0 ? pair : st;
}

}  // namespace lca
