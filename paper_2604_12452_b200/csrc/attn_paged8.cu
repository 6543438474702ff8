// Decode attention over the paged 8-bit cache (Sec. 4.3 over the layout of lca_paged8).
//
// Mathematics.  For a query row h and the present rows i of its sequence and KV head
//     y_i = log2(e) (scale * s_k(i) * sum_c q_c k_ic + bias_i),   out = sum_i 2^y_i s_v(i) v_i / sum_i 2^y_i
// with e4m3 codes k, v and one scale for each page and KV head.  Everything is multiplied as 8-bit numbers:
//   * q f = q_hi + q_lo, two e4m3 terms, f the power of two that brings the row's largest element into [128, 256).
//     Four significant bits each: exact for every element above 2^-9 of the largest, otherwise off by 2^-17 of the largest.
//   * t_i = 2^(y_i + log2 s_v(i) - M + 5) = t_hi + 2^-4 t_lo, two e4m3 terms again: relative error 2^-9 (a bf16 weight has 2^-8).
//     t_hi is the nearest e4m3 value down to the format's smallest step (2^-9), so that what it leaves, times 2^4, is below e4m3's
//     normal range wherever t is: there weights are held in steps of 2^-13, i.e. 2^-18 of the largest weight.  Such a step would round
//     a long flat tail all the same way, so every key adds its own offset within the step before the rounding, its row times
//     the golden ratio modulo 1: keys of every residue modulo anything small get evenly spread offsets, and a tail keeps its
//     weight under values of whatever period, to a few dozen steps in all.  (Offsets that repeat every 32 rows hand the tail to a
//     fixed subset of the keys: 20000 rows with +1 and -1 in turn behind one large logit, 0.38 instead of 0.)
//   M is the running maximum of y + log2 s_v over a split; it is raised only when a weight would exceed 2^8.75.  The row
//   sum adds the weights without s_v in fp32, unrounded.
#include <cstring>

#include "attn_paged8.cuh"

namespace lca {
using namespace tc;

static __device__ int g_paged8_status = 0;

// --------------------------------------------------------------------------------------------------- scalar kernel
// One warp per query row, keys one by one, fp32: the cross-check of the tensor-core kernel (lca_set_attention_impl(1)).
struct Paged8SimtArgs {
  const bf16* q_sem; const bf16* q_pos;
  const uint8_t* pages_sem; const uint8_t* pages_pos; const float* scale_sem; const float* scale_pos; const int32_t* table;
  const int32_t* n_rep; const int32_t* n_tok;
  bf16* out; float* lse;
  int Hq, Hkv, q_len, g, page, n_pages, width;
  float scale, bias;
  long long n_rows;
};

template <int D_SEM, int D_POS, bool MLA>
__global__ void __launch_bounds__(128) attn_paged8_simt_kernel(Paged8SimtArgs a) {
  constexpr int PS = D_SEM / 64, PP = D_POS / 64;            // element pairs per lane
  const int lane = threadIdx.x & 31;
  const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (row >= a.n_rows) return;
  const int h = (int)(row % a.Hq), t = (int)((row / a.Hq) % a.q_len), b = (int)(row / ((long long)a.Hq * a.q_len));
  const int hk = h / (a.Hq / a.Hkv);
  float2 qs[PS], qp[PP], acc[PS];
#pragma unroll
  for (int i = 0; i < PS; ++i) {
    acc[i] = make_float2(0.f, 0.f);
    if (MLA) qs[i] = __bfloat1622float2(reinterpret_cast<const bf162*>(a.q_sem + (size_t)row * D_SEM)[lane + 32 * i]);
  }
#pragma unroll
  for (int i = 0; i < PP; ++i) qp[i] = __bfloat1622float2(reinterpret_cast<const bf162*>(a.q_pos + (size_t)row * D_POS)[lane + 32 * i]);
  const PagedSpan sp = paged_span(a.n_rep, a.n_tok, b, a.g, a.width * a.page);
  const int last = sp.n_tok - a.q_len + 1 + t;               // rows below it are seen
  float mx = -INFINITY, l = 0.f;
  bool any = false;
  for (int x = 0; x < last; ++x) {
    if (x == sp.n_rep && x < sp.tok0) x = sp.tok0;
    if (x >= last) break;
    const int pg = a.table[(size_t)b * a.width + x / a.page];
    if (pg < 0 || pg >= a.n_pages) continue;
    const size_t block = (size_t)pg * a.Hkv + hk, r = block * a.page + x % a.page;
    const float fv = fmaxf(a.scale_sem[block], exp2_int(PAGED8_MIN_EXP)), fk = MLA ? a.scale_sem[block] : a.scale_pos[block];
    const uint16_t* vs = reinterpret_cast<const uint16_t*>(a.pages_sem + r * D_SEM);
    const uint16_t* ks = reinterpret_cast<const uint16_t*>(a.pages_pos + r * D_POS);
    float2 v[PS];
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < PS; ++i) {
      const float4 f = e4m3x4_to_float4(vs[lane + 32 * i]);
      v[i] = make_float2(f.x, f.y);
      if (MLA) s += qs[i].x * f.x + qs[i].y * f.y;
    }
#pragma unroll
    for (int i = 0; i < PP; ++i) {
      const float4 f = e4m3x4_to_float4(ks[lane + 32 * i]);
      s += qp[i].x * f.x + qp[i].y * f.y;
    }
    s = warp_sum(s) * fk * a.scale + (x < sp.n_rep ? a.bias : 0.f);
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
    reinterpret_cast<bf162*>(a.out + (size_t)row * D_SEM)[lane + 32 * i] = __floats2bfloat162_rn(acc[i].x * inv, acc[i].y * inv);
  if (a.lse && lane == 0) a.lse[row] = any ? mx + logf(l) : -INFINITY;
}

int attn_paged8_simt_launch(const Paged8Attn& q) {
  const lca_params* p = q.p;
  const lca_paged8* c = q.c;
  Paged8SimtArgs a = {(const bf16*)q.q_sem, (const bf16*)q.q_pos, (const uint8_t*)c->pages_sem, (const uint8_t*)c->pages_pos, c->scale_sem,
                      c->scale_pos, c->block_table, q.n_rep, q.n_tok, (bf16*)q.out, q.lse, p->n_q_heads, p->n_kv_heads, q.q_len,
                      q.n_rep ? p->group_size : 1, c->page_size, c->n_pages, c->table_width, p->softmax_scale, p->rep_logit_bias,
                      (long long)p->batch * q.q_len * p->n_q_heads};
  const unsigned grid = (unsigned)((a.n_rows + 3) / 4);
  if (p->variant == LCA_VARIANT_MLA) {
    if (p->d_sem == 512) attn_paged8_simt_kernel<512, 64, true><<<grid, 128, 0, q.stream>>>(a);
    else attn_paged8_simt_kernel<128, 64, true><<<grid, 128, 0, q.stream>>>(a);
  } else if (p->d_sem == 128) attn_paged8_simt_kernel<128, 128, false><<<grid, 128, 0, q.stream>>>(a);
  else attn_paged8_simt_kernel<64, 64, false><<<grid, 128, 0, q.stream>>>(a);
  note_launch();
  return cudaGetLastError() == cudaSuccess ? LCA_OK : LCA_ERR_CUDA;
}

// ---------------------------------------------------------------------------------------------- tensor-core kernel
// Transposed products: S^T [128 keys x 2 NH] = K [Q_hi | Q_lo]^T and O^T [d x 2 NH] += V^T [T_hi | T_lo]^T, so that the key
// tile is the 128-row operand whatever the number of heads, a row of K or V is read by the tensor core as it lies in the
// page (K-major for S, MN-major for O: no transposition, no conversion) and a softmax thread owns one key: scale, mask and
// bias are one value per thread.  NH (16, 32 or 64) query rows of one KV head share a tile.
//   softmax    NH / 16 groups of four warps, each for 16 of the rows: thread = key = TMEM lane; epilogue: thread = output
//              column d.  Sixteen rows a thread keep the unrolled code within the instruction cache (one group of 64 rows spent
//              most of its time fetching instructions: 64 x 5056 rows of 128 heads took 243 us instead of 150).
//   + 1 warp   TMA: 128-byte-wide chunks (16 KB) of the 128 rows of a tile, one request per page
//   + 1 warp   MMA issue and TMEM
// S of tile j+1 is issued before O of tile j.  GQA: one ring of slots, filled in the order of use, K(0) K(1) V(0) K(2)
// V(1) ...  MLA: the latent chunks are keys and values; they stay in their slots from S to O (two tiles at a time are in the
// ring, a third one is arriving), which saves the second copy: the tensor core reads its operands over the same 128 bytes
// per clock of shared memory that the copies are written through (NH = 16: 720 clocks of operands for S, 640 for O, 576 of
// copies; with a second copy of the values 1088).
// What bounds it.  GQA with one token: HBM (64 x 5056 rows, 32 heads on 8: 663 MB in 115 us, 5.8 TB/s).  MLA and several tokens: neither
// HBM nor that port, but the chain of a tile, S, softmax, weights, O, with one group of warps and one buffer of weights for 16
// rows; a tile's weights are stored once O of the tile before is complete.  64 x 5056 rows of 16 MLA heads, 17 tiles a CTA: 55 us, 3.1 us
// or about 6000 clocks a tile where the port would take 1936; 32 heads 65 us; 12 sequences of up to 9001 rows and 4 tokens, GQA: 42 us.
// Work: all tiles of all (sequence, KV head, block of NH rows) units form one line that is cut into equal ranges, one per
// CTA; a unit that is cut leaves (O, M, l) of its pieces in the workspace, merged by paged8_combine_kernel.
template <bool MLA_, int DS_, int DP_, int NH_>
struct Paged8Plan {
  static constexpr bool MLA = MLA_;
  static constexpr int DS = DS_, DP = DP_, NH = NH_;
  static constexpr int KSEM = MLA ? DS / 128 : 0;            // latent chunks of the key product
  static constexpr int NK = KSEM + 1;                        // + the pos chunk (64 or 128 bytes wide)
  static constexpr int NV = DS >= 128 ? DS / 128 : 1, VW = DS >= 128 ? 128 : DS;
  static constexpr bool SHARED = MLA;                        // a latent chunk stays from S to O
  static constexpr int PER_TILE = SHARED ? NK : NK + NV;     // slots a tile passes through
  static constexpr int SLOT = 16384;
  static constexpr int Q_BYTES = 2 * NH * (KSEM * 128 + DP);
  static constexpr int P_BYTES = 128 * 2 * NH;               // per key the first terms of all rows, then the second ones
  static constexpr int TM_S = 2 * NV * NH, TM_USED = TM_S + 4 * NH;        // O: for each 128 columns the two terms' sums side by side
  static constexpr int TM_COLS = TM_USED <= 64 ? 64 : TM_USED <= 128 ? 128 : TM_USED <= 256 ? 256 : 512;
  static constexpr int CTAS = (MLA && DS == 512) || TM_COLS == 512 ? 1 : 2;        // per SM
  static constexpr int GROUPS = NH / 16, SOFTMAX_WARPS = 4 * GROUPS, THREADS = 32 * (SOFTMAX_WARPS + 2);
  // words: qs, M, d, factor, lim [NH]; wmax / sums [4][NH]; output rows [2][NH].  Barriers first.
  static constexpr int MISC_BYTES = 512 + 4 * (5 * NH + 4 * NH + 2 * NH);
  static constexpr int BUDGET = (CTAS == 1 ? 227 * 1024 : 113 * 1024) - 1024;      // 1 KB to align the base
  static constexpr int SLOTS_FIT = (BUDGET - Q_BYTES - P_BYTES - MISC_BYTES) / SLOT;
  static constexpr int SLOTS = SLOTS_FIT > 12 ? 12 : SLOTS_FIT;
  static constexpr int OFF_Q = SLOTS * SLOT, OFF_P = OFF_Q + Q_BYTES, OFF_MISC = OFF_P + P_BYTES;
  static constexpr int SMEM = OFF_MISC + MISC_BYTES + 1024;
  static_assert(SLOTS >= (SHARED ? 2 * NK : NV + 1) && SMEM <= 227 * 1024, "the tiles that S and O work on fit the ring");
};

// one group of softmax warps (128 threads)
__device__ __forceinline__ void group_barrier(int grp) { asm volatile("bar.sync %0, 128;" ::"r"(grp + 1) : "memory"); }
__device__ __forceinline__ bool group_any(int grp, bool v) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(r) : "r"((uint32_t)v), "r"(grp + 1) : "memory");
  return r != 0;
}

static constexpr float T_MAX = 8.75f;                        // log2 of the largest weight: e4m3 ends at 448
static constexpr float LO_GAIN = 16.f;                       // of the second term, which has columns of O of its own

template <class PL>
__global__ void __launch_bounds__(PL::THREADS, PL::CTAS) attn_paged8_kernel(const __grid_constant__ Paged8Params p) {
  constexpr int NH = PL::NH, NK = PL::NK, NV = PL::NV, DS = PL::DS, DP = PL::DP, W_TMA = PL::SOFTMAX_WARPS, W_MMA = W_TMA + 1;
  extern __shared__ unsigned char smem_dyn[];
  const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  unsigned char* base_ptr = smem_dyn + (base - smem_u32(smem_dyn));
  const uint32_t bars = base + PL::OFF_MISC;
  auto FULL = [&](int s) { return bars + 8 * s; };
  auto EMPTY = [&](int s) { return bars + 8 * (PL::SLOTS + s); };
  const uint32_t SFULL = bars + 8 * (2 * PL::SLOTS), PFULL = SFULL + 16, PVDONE = SFULL + 24, QFULL = SFULL + 32;
  unsigned char* misc = base_ptr + PL::OFF_MISC;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(misc + 256);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 260);
  int* s_b = reinterpret_cast<int*>(misc + 264);
  long long* s_off = reinterpret_cast<long long*>(misc + 272);          // offset inside sequence s_b, tiles of this CTA
  long long* s_warp = reinterpret_cast<long long*>(misc + 288);         // totals of up to 18 warps, and 18 words
  float* s_qs = reinterpret_cast<float*>(misc + 512);
  float* s_m = s_qs + NH; float* s_d = s_m + NH; float* s_f = s_d + NH;
  int* s_lim = reinterpret_cast<int*>(s_f + NH);
  float* s_wmax = reinterpret_cast<float*>(s_lim + NH);      // also the sums of the four warps of a group
  int* s_row = reinterpret_cast<int*>(s_wmax + 4 * NH);      // output row of each query row, of this piece and of the next one
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, tid = threadIdx.x;

  if (tid == 0) {
    for (int s = 0; s < PL::SLOTS; ++s) { mbar_init(FULL(s), 1); mbar_init(EMPTY(s), 1); }
    mbar_init(SFULL, 1); mbar_init(SFULL + 8, 1); mbar_init(PFULL, 32 * W_TMA); mbar_init(PVDONE, 1); mbar_init(QFULL, 32 * W_TMA);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == W_MMA) { tmem_alloc(smem_u32((const void*)tmem_slot), PL::TM_COLS); tmem_relinquish(); }
  if (warp == W_TMA && lane == 0) { prefetch_tmap(&p.sem); prefetch_tmap(&p.pos); }
  chain_wait();
  chain_next();                                              // the whole grid is resident: nothing is displaced
  paged8_range<PL::THREADS>(p, (int)blockIdx.x, s_warp, s_b, s_off);
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  Walk w;
  w.b = *s_b; w.off = s_off[0]; w.left = s_off[1]; w.fresh = true; w.n = 0;
  auto fail = [&](int code) { atomicCAS(&g_paged8_status, 0, code); *abort_flag = 1; };

  if (warp == W_TMA) {
    // ------------------------------------------------------------------------------------------------ producer
    int slot = 0;
    uint32_t phase = 0;
    bool ok = true;
    const int npp = 128 / p.page;
    while (ok && w.next(p)) {
      const PagedSpan sp = w.t.s;
      const int32_t* table = p.table + (size_t)w.b * p.width;
      // third coordinate of this lane's page; one past the end (filled with zeros) where no row is present
      auto look = [&](int i) {
        const int nowhere = p.n_pages * p.Hkv;
        if (i >= w.n || lane >= npp) return nowhere;
        const int x = w.t.row0(w.t0 + i) + lane * p.page;
        if (!sp.any(x, p.page) || (x >> p.page_log2) >= p.width) return nowhere;
        const int pg = table[x >> p.page_log2];
        return pg >= 0 && pg < p.n_pages ? pg * p.Hkv + w.hk : nowhere;
      };
      auto load = [&](const CUtensorMap* map, int x, int width, int z) {
        if (!ok) return;
        if (!mbar_wait(EMPTY(slot), phase ^ 1, abort_flag)) { ok = false; }
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) { if (lane == 0) fail(ERR_WAIT_KV_EMPTY); return; }
        if (lane == 0) mbar_expect_tx(FULL(slot), 128 * width);
        __syncwarp();
        if (lane < npp) tma_load_3d(base + slot * PL::SLOT + lane * p.page * width, map, x, 0, z, FULL(slot));
        if (++slot == PL::SLOTS) { slot = 0; phase ^= 1; }
      };
      auto load_k = [&](int z) {
#pragma unroll
        for (int c = 0; c < PL::KSEM; ++c) load(&p.sem, c * 128, 128, z);
        load(&p.pos, 0, DP, z);
      };
      int z0 = look(0), z1 = look(1);
      load_k(z0);
      for (int j = 0; j < w.n && ok; ++j) {
        const int z2 = look(j + 2);
        if (j + 1 < w.n) load_k(z1);
        if (!PL::SHARED)
#pragma unroll
          for (int c = 0; c < NV; ++c) load(&p.sem, c * 128, PL::VW, z0);
        z0 = z1; z1 = z2;
      }
    }
  } else if (warp == W_MMA) {
    // ----------------------------------------------------------------------------------------------------- MMA
    const uint32_t leader = elect_one();
    constexpr uint32_t ID_S = umma_idesc_f8(128, 2 * NH, 0, false, false);
    constexpr uint32_t ID_O = umma_idesc_f8(128, 2 * NH, 0, true, true);
    int slot = 0;
    uint32_t phase = 0, g = 0, seg = 0;
    bool ok = true;
    int v_slot = 0;                                          // shared chunks: first slot of the tile whose O comes next
    auto wait_slot = [&]() {
      ok = ok && mbar_wait(FULL(slot), phase, abort_flag);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok && lane == 0) fail(ERR_WAIT_KV_FULL);
      return ok;
    };
    auto next_slot = [&]() { if (++slot == PL::SLOTS) { slot = 0; phase ^= 1; } };
    auto issue_s = [&](uint32_t buf) {
      const uint32_t d = tmem + PL::TM_S + buf * 2 * NH;
      uint32_t acc = 0;
#pragma unroll
      for (int c = 0; c < NK; ++c) {
        if (!wait_slot()) return;
        tc_fence_after();
        const int width = c < PL::KSEM ? 128 : DP;
        const uint64_t ad = desc_rows(base + slot * PL::SLOT, width, 16);
        const uint64_t bd = desc_rows(base + PL::OFF_Q + c * 2 * NH * 128, width, 16);
#pragma unroll
        for (int k = 0; k < width / 32; ++k) { umma_f8_elected(leader, d, desc_add(ad, 2 * k), desc_add(bd, 2 * k), ID_S, acc); acc = 1; }
        if (!PL::SHARED || c == PL::KSEM) umma_commit_elected(leader, EMPTY(slot));
        next_slot();
      }
      umma_commit_elected(leader, SFULL + 8 * buf);
    };
    const uint64_t pd = desc_rows(base + PL::OFF_P, 2 * NH, 128);
    while (ok && w.next(p)) {
      ok = mbar_wait(QFULL, seg & 1, abort_flag);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) { if (lane == 0) fail(ERR_WAIT_Q); break; }
      ++seg;
      tc_fence_after();
      issue_s(g & 1);
      for (int j = 0; j < w.n && ok; ++j, ++g) {
        if (j + 1 < w.n) issue_s((g + 1) & 1);
        if (!ok) break;
        ok = mbar_wait(PFULL, g & 1, abort_flag);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) { if (lane == 0) fail(ERR_WAIT_P_FULL); break; }
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < NV; ++c) {
          if (!PL::SHARED && !wait_slot()) break;
          if (!PL::SHARED) tc_fence_after();
          const int vs = PL::SHARED ? v_slot : slot;
          // 64-wide values: M stays 128, the second half of the operand is the unused half of the slot and the output
          // lanes it feeds are never read
          const uint64_t ad = desc_rows(base + vs * PL::SLOT, PL::VW, 8192);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            umma_f8_elected(leader, tmem + c * 2 * NH, desc_add(ad, k * 2 * PL::VW), desc_add(pd, k * 4 * NH), ID_O, (j > 0 || k > 0) ? 1u : 0u);
          umma_commit_elected(leader, EMPTY(vs));
          if (PL::SHARED) { if (++v_slot == PL::SLOTS) v_slot = 0; }
          else next_slot();
        }
        if (PL::SHARED && ++v_slot == PL::SLOTS) v_slot = 0; // the pos chunk's slot
        umma_commit_elected(leader, PVDONE);
      }
    }
  } else {
    // ------------------------------------------------------------------------------------- softmax, epilogue
    const int grp = warp >> 2, quad = warp & 3, t = tid & 127, hb = 16 * grp;      // this thread: key t of a tile, rows hb .. hb + 15
    const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
    uint32_t g = 0, seg = 0, seg_chunks = 0;
    bool ok = true;
    float l[16];
    int pg0 = -1, pg1 = -1;                                  // page of this thread's key in the current tile and in the next one
    float ks = 0.f, vs = 1.f;                                // scales of pg0
    auto page_of = [&](const Walk& u, int j) {               // -1: none
      if (j >= u.n) return -1;
      const int x = u.t.row0(u.t0 + j) + t;
      if (!u.t.s.has(x)) return -1;                          // has() implies x below the table's end
      const int pg = p.table[(size_t)u.b * p.width + (x >> p.page_log2)];
      return pg >= 0 && pg < p.n_pages ? pg : -1;
    };
    // splits this group's query rows of a unit into e4m3 terms and writes them where S reads them; the first lookups of the
    // piece run underneath
    auto load_q = [&](const Walk& u, uint32_t which) {
      pg0 = page_of(u, 0); pg1 = page_of(u, 1);
      constexpr int VS = PL::KSEM * 16, VQ = VS + DP / 8, NL = (VQ + 31) / 32;   // 8-element vectors of a row
      const int n_rows = p.q_len * p.rep - u.blk * NH;
#pragma unroll 2
      for (int r = hb + quad; r < hb + 16; r += 4) {
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
      ks = 0.f; vs = 1.f;
      if (pg0 >= 0) { ks = p.scale_k[(size_t)pg0 * p.Hkv + u.hk]; vs = p.scale_v[(size_t)pg0 * p.Hkv + u.hk]; }
      fence_proxy_async_smem();
      mbar_arrive(QFULL);
      group_barrier(grp);
    };
    bool more = w.next(p);
    if (more) load_q(w, 0);
    while (more) {
      const PagedSpan sp = w.t.s;
      const int* rows = s_row + (seg & 1) * NH + hb;
      bool unset = t < 16 && rows[t & 15] >= 0;              // thread h of the group: its row has no maximum yet
#pragma unroll
      for (int i = 0; i < 16; ++i) l[i] = 0.f;
      // first rows of the (at most two) pages that are present in part; one past every row where there is none
      const int none = 0x7fffffff, mask = p.page - 1;
      const int part_r = (sp.n_rep & mask) ? sp.n_rep & ~mask : none, part_t = (sp.n_tok & mask) ? sp.n_tok & ~mask : none;
#pragma unroll 1
      for (int j = 0; j < w.n; ++j, ++g) {
        const int row0 = w.t.row0(w.t0 + j), x = row0 + t;
        const bool valid = pg0 >= 0;
        // the next tile's scales and the page after that are on their way while this tile is worked on
        float ks1 = 0.f, vs1 = 1.f;
        if (pg1 >= 0) { ks1 = p.scale_k[(size_t)pg1 * p.Hkv + w.hk]; vs1 = p.scale_v[(size_t)pg1 * p.Hkv + w.hk]; }
        const int pg2 = page_of(w, j + 2);
        vs = fmaxf(vs, exp2_int(PAGED8_MIN_EXP));
        // The row sum needs 2^(y - M), the weight t = 2^(y - M + log2 vs + 5): both are multiples of e = 2^(y - M + half), half way
        // between them, so that neither is lost below 2^-126 where the scales of a sequence span more than fp32 does.
        const float half = 0.5f * (lg2(vs) + paged8_t_bits(NH)), f_t = ex2(half), f_l = ex2(paged8_t_bits(NH) - half);
        const float kf = ks * p.scale_log2, cb = half + (x < sp.n_rep ? p.bias_log2 : 0.f);
        const float offset = weight_offset(x);
        const bool limited = row0 + 127 >= sp.n_tok - p.q_len + 1;      // some query may not see some row of this tile

        ok = mbar_wait(SFULL + 8 * (g & 1), (g >> 1) & 1, abort_flag);
        if (!ok) fail(ERR_WAIT_S_FULL);
        __syncwarp();
        tc_fence_after();
        float z[16];
        float zmax = -INFINITY;
        {
          uint32_t hi[16], lo[16];
          const uint32_t at = tmem + lane_base + PL::TM_S + (g & 1) * 2 * NH + hb;
          tmem_ld16(at, hi);
          tmem_ld16(at + NH, lo);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            const float4 q4 = *reinterpret_cast<const float4*>(s_qs + hb + i), m4 = *reinterpret_cast<const float4*>(s_m + hb + i);
            const float qq[4] = {q4.x, q4.y, q4.z, q4.w}, mm[4] = {m4.x, m4.y, m4.z, m4.w};
#pragma unroll
            for (int k = 0; k < 4; ++k)
              z[i + k] = fmaf(__uint_as_float(hi[i + k]) + __uint_as_float(lo[i + k]), kf * qq[k], cb - mm[k]);
          }
        }
        if (limited || !__all_sync(0xffffffffu, valid)) {
#pragma unroll
          for (int i = 0; i < 16; ++i) z[i] = valid && (!limited || x < s_lim[hb + i]) ? z[i] : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < 16; i += 2) zmax = max3(zmax, z[i], z[i + 1]);
        const bool raise = group_any(grp, zmax + half > T_MAX || unset);
        if (raise) {
          // raise the maxima: per row the largest log2 t of the tile
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float m = warp_max_f32(z[i] + half);
            if (lane == i) s_wmax[quad * NH + hb + i] = m;
          }
          group_barrier(grp);
          if (t < 16) {
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
          group_barrier(grp);
#pragma unroll
          for (int i = 0; i < 16; ++i) { z[i] -= s_d[hb + i]; l[i] *= s_f[hb + i]; }
        }
        if (j > 0) {                                         // the weights of the previous tile have been read, O is complete up to it
          ok = mbar_wait(PVDONE, (g - 1) & 1, abort_flag);
          if (!ok) fail(ERR_WAIT_O_DONE);
          __syncwarp();
          if (raise) {
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < 2 * NV; ++c) {
              uint32_t o[16];
              tmem_ld16(tmem + lane_base + c * NH + hb, o);
              tmem_wait_ld();
#pragma unroll
              for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * s_f[hb + k]);
              tmem_st16(tmem + lane_base + c * NH + hb, o);
            }
            tmem_wait_st();
          }
        }
        {
          uint32_t wh[4], wl[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float tt[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float e = ex2(z[4 * i + k]);
              tt[k] = e * f_t;
              l[4 * i + k] = fmaf(e, f_l, l[4 * i + k]);
            }
            wh[i] = e4m3x4_from_float(tt[0], tt[1], tt[2], tt[3]);
            const float4 h = e4m3x4_to_float4(wh[i]);        // what the first term leaves is exact: at most 2^4, times LO_GAIN 2^8
            wl[i] = e4m3x4_from_float(fmaf(tt[0] - h.x, LO_GAIN, offset), fmaf(tt[1] - h.y, LO_GAIN, offset),
                                      fmaf(tt[2] - h.z, LO_GAIN, offset), fmaf(tt[3] - h.w, LO_GAIN, offset));
          }
          unsigned char* ph = base_ptr + PL::OFF_P;
          *reinterpret_cast<uint4*>(ph + swz<2 * NH>(t, grp)) = make_uint4(wh[0], wh[1], wh[2], wh[3]);
          *reinterpret_cast<uint4*>(ph + swz<2 * NH>(t, PL::GROUPS + grp)) = make_uint4(wl[0], wl[1], wl[2], wl[3]);
        }
        // Rows that were fetched with a page but are not present may hold anything; their weight is 0 and 0 * NaN is not.
        if (grp == 0 && ((unsigned)(part_r - row0) < 128u || (unsigned)(part_t - row0) < 128u)) {
#pragma unroll 1
          for (int c = 0; c < NV; ++c) {
            const uint32_t at = seg_chunks + (PL::SHARED ? (uint32_t)j * NK : (uint32_t)min(j + 2, w.n) * NK + (uint32_t)j * NV) + c;      // place in the order of loads
            const int s = (int)(at % PL::SLOTS);
            ok = mbar_wait(FULL(s), (at / PL::SLOTS) & 1, abort_flag);
            if (!ok) fail(ERR_WAIT_KV_FULL);
            if (!valid) {
              uint4* row = reinterpret_cast<uint4*>(base_ptr + s * PL::SLOT + t * PL::VW);
#pragma unroll
              for (int i = 0; i < PL::VW / 16; ++i) row[i] = make_uint4(0u, 0u, 0u, 0u);
            }
          }
          __syncwarp();
        }
        fence_proxy_async_smem();
        tc_fence_before();
        mbar_arrive(PFULL);
        pg0 = pg1; pg1 = pg2; ks = ks1; vs = vs1;
      }
      seg_chunks += (uint32_t)w.n * PL::PER_TILE;
      // ---- this piece is done: its sums and maxima, then the next unit's queries (S of this piece is complete), then O
      const bool whole = w.n == w.t.n;
      const size_t part = (size_t)2 * blockIdx.x + (seg == 0 ? 0 : 1);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float v = l[i];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (lane == i) s_wmax[quad * NH + hb + i] = v;
      }
      group_barrier(grp);
      if (t < 16) {
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
      group_barrier(grp);
      more = w.next(p);
      if (more) load_q(w, seg + 1);
      ok = mbar_wait(PVDONE, (g - 1) & 1, abort_flag);
      if (!ok) fail(ERR_WAIT_O_DONE);
      __syncwarp();
      tc_fence_after();
#pragma unroll 1
      for (int c = 0; c < NV; ++c) {
        uint32_t o[16], o2[16];
        tmem_ld16(tmem + lane_base + c * 2 * NH + hb, o);
        tmem_ld16(tmem + lane_base + c * 2 * NH + NH + hb, o2);
        tmem_wait_ld();
#pragma unroll
        for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(fmaf(__uint_as_float(o2[k]), 1.f / LO_GAIN, __uint_as_float(o[k])));
        const int d = c * 128 + t;
        if (DS >= 128 || t < DS) {
          if (whole) {
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              const float f = s_f[hb + k];
              const int row = rows[k];
              if (row >= 0) p.out[(size_t)row * DS + d] = __float2bfloat16_rn(f == 0.f ? 0.f : __uint_as_float(o[k]) * f);   // no key: O may be 0 * NaN
            }
          } else {
            float* dst = p.part + part * NH * DS + (size_t)hb * DS + d;
#pragma unroll
            for (int k = 0; k < 16; ++k) dst[(size_t)k * DS] = __uint_as_float(o[k]);
          }
        }
      }
      tc_fence_before();
      ++seg;
      group_barrier(grp);                                    // s_f is written again by the next piece
    }
  }
  // ---- let straggling copies land if the CTA gave up, then free TMEM
  if (*abort_flag && warp == 0 && lane == 0) {
    const long long t0c = clock64();
    while (clock64() - t0c < 2000000ll) __nanosleep(1000);
  }
  __syncthreads();
  if (warp == W_MMA) { tc_fence_after(); tmem_dealloc(tmem, PL::TM_COLS); }
}

// ------------------------------------------------------------------------------------------------------------- host
bool make_tensor_map_pages(CUtensorMap* map, const void* ptr, int d, int page, long long blocks, int box_d, int box_rows);   // attn_tc.cu

// Query rows that share a tile of keys.  The tile is padded to that number, so it is the smallest one that holds all rows of
// a KV head (the softmax threads compute an exponential per padded row and key); at most 64.  The MLA shape has columns of TMEM for
// 32 (O takes d / 128 * 2 NH of 512, S 4 NH): 33 to 64 rows are two such blocks, more go to CTA pairs in blocks of 128.  Single CTAs
// against pairs, MLA 512 + 64:
//                                     64 x 5056 rows   20 x 2500 .. 5056   1 x 2528   12 x up to 9001
//   34 rows (two blocks)                 89 / 89 us          46 / 55        17 / 26       40 / 51
//   64 rows (two blocks)                 92 / 92             48 / 57        17 / 26       43 / 52       (100 x 5056: 155 / 150)
//   65 rows (three blocks)              143 / 92             56 / 57        17 / 26       47 / 52       (4 x 60000: 104 / 83)
//   128 rows (four blocks)              187 / 95             69 / 62        18 / 27       56 / 54
static int paged8_rows_per_tile(const lca_params* p, int q_len) {
  const long long rows = (long long)q_len * (p->n_q_heads / p->n_kv_heads);
  if (p->d_sem == 512) return rows <= 16 ? 16 : rows <= 64 ? 32 : 128;
  return rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
}
// CTAs (or pairs) that share the work: all that are resident at once.
static int paged8_grid(const lca_params* p, int nh) {
  return nh == 128 ? 74 : (p->d_sem == 512 || nh == 64) ? 148 : 2 * 148;
}
size_t attn_paged8_workspace_bytes(const lca_params* p, int q_len) {
  const int nh = paged8_rows_per_tile(p, q_len), grid = paged8_grid(p, nh);
  return (size_t)2 * grid * (nh * (size_t)p->d_sem + 2 * nh) * sizeof(float) + ((size_t)p->batch + 2) * sizeof(long long) + 64;
}

template <class PL>
static int paged8_launch(Paged8Params& P, cudaStream_t stream) {
  auto kern = attn_paged8_kernel<PL>;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, PL::SMEM) != cudaSuccess) return LCA_ERR_CUDA;
  const int st = launch_chained(kern, (unsigned)P.grid, PL::THREADS, PL::SMEM, stream, 1, P);
  if (st != LCA_OK) return st;
  return paged8_combine_launch<PL::DS, PL::NH>(P, stream);
}
template <bool MLA, int DS, int DP>
static int paged8_launch_rows(Paged8Params& P, int nh, cudaStream_t stream) {
  if (nh == 16) return paged8_launch<Paged8Plan<MLA, DS, DP, 16>>(P, stream);
  if (nh == 32) return paged8_launch<Paged8Plan<MLA, DS, DP, 32>>(P, stream);
  if constexpr (DS == 512) return attn_paged8_pair_launch(P, stream);
  else return paged8_launch<Paged8Plan<MLA, DS, DP, 64>>(P, stream);
}

int attn_paged8_launch(const Paged8Attn& a) {
  const lca_params* p = a.p;
  const lca_paged8* c = a.c;
  const bool mla = p->variant == LCA_VARIANT_MLA;
  Paged8Params P;
  memset(&P, 0, sizeof(P));
  const long long blocks = (long long)c->n_pages * p->n_kv_heads;
  const int nh = paged8_rows_per_tile(p, a.q_len);
  // a request brings a whole page; on pairs, where a CTA takes 64 of a tile's keys, at most 64 rows
  const int box = nh == 128 && c->page_size > 64 ? 64 : c->page_size;
  if (!make_tensor_map_pages(&P.sem, c->pages_sem, p->d_sem, c->page_size, blocks, p->d_sem >= 128 ? 128 : p->d_sem, box) ||
      !make_tensor_map_pages(&P.pos, c->pages_pos, p->d_pos, c->page_size, blocks, p->d_pos, box))
    return LCA_ERR_CUDA;
  P.q_sem = (const bf16*)a.q_sem; P.q_pos = (const bf16*)a.q_pos;
  P.scale_v = c->scale_sem; P.scale_k = mla ? c->scale_sem : c->scale_pos; P.table = c->block_table;
  P.n_rep = a.n_rep; P.n_tok = a.n_tok; P.out = (bf16*)a.out; P.lse = a.lse;
  P.B = p->batch; P.Hq = p->n_q_heads; P.Hkv = p->n_kv_heads; P.q_len = a.q_len; P.g = a.n_rep ? p->group_size : 1;
  P.page = c->page_size; P.page_log2 = c->page_size == 16 ? 4 : c->page_size == 32 ? 5 : c->page_size == 64 ? 6 : 7; P.n_pages = c->n_pages; P.width = c->table_width; P.rep = P.Hq / P.Hkv;
  P.n_blk = (int)(((long long)P.q_len * P.rep + nh - 1) / nh);
  P.grid = paged8_grid(p, nh);
  P.scale_log2 = p->softmax_scale * 1.4426950408889634f; P.bias_log2 = p->rep_logit_bias * 1.4426950408889634f;
  P.part = reinterpret_cast<float*>((reinterpret_cast<uintptr_t>(a.ws) + 31) & ~(uintptr_t)31);
  P.out_wide = (reinterpret_cast<uintptr_t>(a.out) & 31u) == 0;
  const size_t part_bytes = (size_t)2 * P.grid * (nh * (size_t)p->d_sem + 2 * nh) * sizeof(float);
  P.prefix = reinterpret_cast<long long*>(reinterpret_cast<char*>(P.part) + (part_bytes + 15) / 16 * 16);
  if ((long long)P.B * P.Hkv * P.n_blk * ((long long)nh * p->d_sem / 512) > 0x7fffffffll) return LCA_ERR_UNSUPPORTED_SHAPE;
  if (mla) return p->d_sem == 512 ? paged8_launch_rows<true, 512, 64>(P, nh, a.stream) : paged8_launch_rows<true, 128, 64>(P, nh, a.stream);
  return p->d_sem == 128 ? paged8_launch_rows<false, 128, 128>(P, nh, a.stream) : paged8_launch_rows<false, 64, 64>(P, nh, a.stream);
}

int attn_paged8_take_status() {
  int st = 0;
  if (cudaMemcpyFromSymbol(&st, g_paged8_status, sizeof(int)) != cudaSuccess) return -1;
  if (st != 0) {
    int zero = 0;
    cudaMemcpyToSymbol(g_paged8_status, &zero, sizeof(int));
  }
  const int pair = attn_paged8_pair_take_status();
  return pair != 0 ? pair : st;
}

}  // namespace lca
