// The paged 8-bit cache around its attention: page tables and slot maps from request lengths, the quantising write and
// the online condensation of a group.  The row space, the pages and the scales are described in lca.h.
#include "lca_common.cuh"
#include "fp8_common.cuh"
#include "tc_common.cuh"

namespace lca {

// ------------------------------------------------------------------------------------------------ page tables, slots
// One cluster does everything, so that a decode step costs one launch: (1) every CTA sums pages to give back, pages to take
// and new rows over all sequences (a few hundred bytes to a few hundred KB from L2) and decides whether the update is
// possible; (2) pages that no present row needs are pushed on the free stack; (3) pages are popped into the tables; (4) the
// slot of every new row is looked up.  A sequence's share of each list starts at an exclusive prefix sum, so the result does
// not depend on how the work is spread.  Bound by latency (dependent passes over the counters and cluster barriers), not by
// its bytes: one CTA for a decode step (64 sequences: 4 us), sixteen for prompts (64 prompts of 5056 rows grown and given
// back: 19 us for both calls; one CTA took 100).
struct PageArgs {
  const int32_t* n_rep; const int32_t* n_tok;
  int32_t* held_rep; int32_t* held_tok;
  int32_t* table; int32_t* free_pages; int32_t* n_free; int32_t* slot_map; int32_t* row_offsets; int32_t* status;
  int B, g, page_log2, width, n_pages, n_rows, per_seq;
};

// What one sequence gives back and takes: up to three ranges of table entries each, ascending and disjoint.
struct PageDelta {
  int rel_lo[3], rel_hi[3], need_lo[3], need_hi[3];
  int r0, r1, tok_first, n_tok;     // new rows: [r0, r1) and [tok_first, n_tok)
  bool valid;
  __device__ __forceinline__ int n_rel() const { int s = 0;
#pragma unroll
    for (int i = 0; i < 3; ++i) s += max(rel_hi[i] - rel_lo[i], 0);
    return s; }
  __device__ __forceinline__ int n_need() const { int s = 0;
#pragma unroll
    for (int i = 0; i < 3; ++i) s += max(need_hi[i] - need_lo[i], 0);
    return s; }
  __device__ __forceinline__ int n_rows() const { return max(r1 - r0, 0) + max(n_tok - tok_first, 0); }
};

__device__ __forceinline__ PageDelta page_delta(const PageArgs& a, int b) {
  PageDelta d;
  const long long r0 = a.n_rep ? a.held_rep[b] : 0, r1 = a.n_rep ? a.n_rep[b] : 0, t0 = a.held_tok[b], t1 = a.n_tok[b];
  const int lg = a.page_log2, up = (1 << lg) - 1;
  const long long cap = (long long)a.width << lg, g0 = r0 * a.g, g1 = r1 * a.g;
  d.valid = r0 >= 0 && r1 >= 0 && g0 <= t0 && g1 <= t1 && t0 <= cap && t1 <= cap && (r1 >= r0 || t1 == 0);
  if (!d.valid) {
#pragma unroll
    for (int i = 0; i < 3; ++i) d.rel_lo[i] = d.rel_hi[i] = d.need_lo[i] = d.need_hi[i] = 0;
    d.r0 = d.r1 = d.tok_first = d.n_tok = 0;
    return d;
  }
  // pages held [0, a0) and [b0, c0), wanted [0, a1) and [b1, c1); a <= b <= c because representatives need no more pages
  // than the tokens they stand for (page | group).  All of them below 2^31.
  const int a0 = (int)((r0 + up) >> lg), b0 = (int)(g0 >> lg), c0 = (int)((t0 + up) >> lg);
  const int a1 = (int)((r1 + up) >> lg), b1 = (int)(g1 >> lg), c1 = (int)((t1 + up) >> lg);
  d.rel_lo[0] = a1;                          d.rel_hi[0] = a0;              // end of a request
  d.rel_lo[1] = max(b0, a1);                 d.rel_hi[1] = min(c0, b1);     // tokens condensed meanwhile
  d.rel_lo[2] = max(max(b0, c1), max(b1, a1)); d.rel_hi[2] = c0;            // tokens taken back
  d.need_lo[0] = a0;                         d.need_hi[0] = min(a1, b0);    // representatives in front of the held tokens
  d.need_lo[1] = max(a0, c0);                d.need_hi[1] = a1;             // ... and behind them
  d.need_lo[2] = max(b1, c0);                d.need_hi[2] = c1;             // new tokens
  d.r0 = (int)r0; d.r1 = (int)r1;
  d.tok_first = (int)max(t0, g1); d.n_tok = (int)t1;
  return d;
}

static const int PAGE_THREADS = 512, PAGE_WARPS = PAGE_THREADS / 32;
// Entries that a thread moves for its sequence one after the other; where a sequence has more a warp moves them, 32 at a time.
// Half of taking and giving back, a thread against a warp: 64 sequences of 1, 8, 16 and 32 entries 3.1, 3.4, 5.8 and 10.4 against 6.0,
// 5.5, 5.8 and 5.9 us; one sequence of 16, 128 and 2000 entries 4.2, 12.2 and 132 against 3.5, 4.1 and 14 us.
static const int FEW_ENTRIES = 8;

// Exclusive prefix sums over the CTA of pages (given back in the low, taken in the high half: each total is below 2^31, the
// tables have fewer entries) and of rows; totals in tot.
__device__ __forceinline__ void scan2(const unsigned long long (&v)[2], unsigned long long (&excl)[2], unsigned long long (&tot)[2],
                                      unsigned long long (*sums)[2]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned long long inc[2] = {v[0], v[1]};
#pragma unroll
  for (int o = 1; o < 32; o <<= 1)
#pragma unroll
    for (int k = 0; k < 2; ++k) { const unsigned long long y = __shfl_up_sync(0xffffffffu, inc[k], o); if (lane >= o) inc[k] += y; }
  if (lane == 31) { sums[warp][0] = inc[0]; sums[warp][1] = inc[1]; }
  __syncthreads();
  // lane w of every warp: total of warp w
  unsigned long long s[2] = {lane < PAGE_WARPS ? sums[lane][0] : 0ull, lane < PAGE_WARPS ? sums[lane][1] : 0ull};
#pragma unroll
  for (int o = 1; o < PAGE_WARPS; o <<= 1)
#pragma unroll
    for (int k = 0; k < 2; ++k) { const unsigned long long y = __shfl_up_sync(0xffffffffu, s[k], o); if (lane >= o) s[k] += y; }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    tot[k] = __shfl_sync(0xffffffffu, s[k], PAGE_WARPS - 1);
    const unsigned long long before = __shfl_sync(0xffffffffu, s[k], max(warp - 1, 0));
    excl[k] = (warp ? before : 0ull) + inc[k] - v[k];
  }
  __syncthreads();
}

__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

__global__ void __launch_bounds__(PAGE_THREADS) page_update_kernel(PageArgs a) {
  __shared__ unsigned long long sums[PAGE_WARPS][2];
  __shared__ unsigned s_flags[PAGE_WARPS];
  __shared__ unsigned s_rel[PAGE_THREADS];                   // first rank of each sequence of a chunk
  __shared__ int s_own[PAGE_THREADS];                        // entries that each moves
  // up to PAGE_THREADS sequences: first packed row of each, then its new rows: first and number of representatives, first
  // token, number in all
  __shared__ int s_row[PAGE_THREADS + 1], s_rep0[PAGE_THREADS], s_reps[PAGE_THREADS], s_tok0[PAGE_THREADS], s_rows[PAGE_THREADS];
  const int cta = blockIdx.x, n_cta = gridDim.x;            // the grid is one cluster
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool single = a.B <= PAGE_THREADS;                   // one sequence per thread: its delta stays in registers
  chain_wait();
  chain_next();
  const long long n_free = a.n_free[0];
  // (1) totals
  unsigned long long tot[2], ex[2];
  PageDelta mine;
  unsigned flags = 0;                                        // 1: not valid, 2: more rows than places, 4: a sequence moves many entries
  {
    unsigned long long v[2] = {0, 0};
#pragma unroll 1
    for (int b = tid; b < a.B; b += PAGE_THREADS) {
      mine = page_delta(a, b);
      const int nr = mine.n_rows();
      flags |= (mine.valid ? 0u : 1u) | (a.per_seq > 0 && a.slot_map && nr > a.per_seq ? 2u : 0u) |
               (max(mine.n_rel(), mine.n_need()) > FEW_ENTRIES ? 4u : 0u);
      v[0] += (unsigned long long)(unsigned)mine.n_rel() | (unsigned long long)(unsigned)mine.n_need() << 32;
      v[1] += (unsigned long long)nr;
    }
    flags = __reduce_or_sync(0xffffffffu, flags);
    if (lane == 0) s_flags[warp] = flags;
    scan2(v, ex, tot, sums);                                 // its barriers are those of s_flags too
    flags = __reduce_or_sync(0xffffffffu, s_flags[lane % PAGE_WARPS]);
    if (single && tid < a.B) {
      s_row[tid] = (int)min(ex[1], 0x7fffffffull);
      s_rep0[tid] = mine.r0; s_reps[tid] = max(mine.r1 - mine.r0, 0); s_tok0[tid] = mine.tok_first; s_rows[tid] = mine.n_rows();
      if (tid == 0) s_row[a.B] = (int)min(tot[1], 0x7fffffffull);
    }
  }
  const long long n_rel = (long long)(tot[0] & 0xffffffffull), n_need = (long long)(tot[0] >> 32), have = n_free + n_rel;
  int status = 0;
  if ((flags & 1u) || n_free < 0 || have > a.n_pages) status = -1;
  else if ((flags & 2u) || (a.slot_map && a.per_seq == 0 && (long long)tot[1] > a.n_rows)) status = -2;
  else if (n_need > have) status = (int)min(n_need - have, 0x7fffffffll);
  const long long gtid = (long long)cta * PAGE_THREADS + tid, gthreads = (long long)n_cta * PAGE_THREADS;
  if (status != 0) {                                         // nothing changes
    for (long long i = gtid; i < a.n_rows; i += gthreads) a.slot_map[i] = -1;
    if (a.row_offsets) for (long long i = gtid; i <= a.B; i += gthreads) a.row_offsets[i] = 0;
    if (gtid == 0) a.status[0] = status;
    return;                                                  // every CTA takes this branch or none
  }
  // (2) and (3)
  auto move_warp = [&](int c0, int i, int phase) {           // the entries of sequence c0 + i, 32 at a time
    const PageDelta d = page_delta(a, c0 + i);
    int32_t* row = a.table + (size_t)(c0 + i) * a.width;
    long long at = have - 1 - s_rel[i];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const int lo = phase == 0 ? d.rel_lo[k] : d.need_lo[k], hi = phase == 0 ? d.rel_hi[k] : d.need_hi[k];
#pragma unroll 4
      for (int e = lo + lane; e < hi; e += 32) {
        if (phase == 0) { a.free_pages[at - (e - lo)] = row[e]; row[e] = -1; }
        else row[e] = a.free_pages[at - (e - lo)];
      }
      at -= max(hi - lo, 0);
    }
  };
#pragma unroll 1
  for (int phase = 0; phase < 2; ++phase) {
    const long long work = phase == 0 ? n_rel : n_need;
    unsigned long long base[2] = {0, 0};
    if (work > 0 || (phase == 0 && a.row_offsets))
#pragma unroll 1
      for (int c0 = 0; c0 < a.B; c0 += PAGE_THREADS) {
        const int b = c0 + tid;
        if (!single) {                                       // (one chunk: the sums of (1) are its prefix sums)
          unsigned long long v[2] = {0, 0}, chunk[2];
          if (b < a.B) {
            mine = page_delta(a, b);
            v[0] = (unsigned long long)(unsigned)mine.n_rel() | (unsigned long long)(unsigned)mine.n_need() << 32;
            v[1] = (unsigned long long)mine.n_rows();
          }
          scan2(v, ex, chunk, sums);
          ex[0] += base[0]; ex[1] += base[1];
          base[0] += chunk[0]; base[1] += chunk[1];
        }
        if (phase == 0 && cta == 0 && a.row_offsets && b < a.B) {
          if (b == 0) a.row_offsets[0] = 0;
          a.row_offsets[b + 1] = (int32_t)min((long long)ex[1] + mine.n_rows(), 0x7fffffffll);
        }
        if (work == 0) continue;
        const unsigned first = phase == 0 ? (unsigned)ex[0] : (unsigned)(ex[0] >> 32);
        if (work <= 4 * PAGE_THREADS) {                      // a few entries, in CTA 0: every thread its own sequence's
          if (cta != 0) continue;
          const int n_own = b >= a.B ? 0 : phase == 0 ? mine.n_rel() : mine.n_need();
          if (n_own > 0 && n_own <= FEW_ENTRIES) {
            int32_t* row = a.table + (size_t)b * a.width;
            long long at = have - 1 - first;
#pragma unroll
            for (int k = 0; k < 3; ++k)
#pragma unroll 1
              for (int e = phase == 0 ? mine.rel_lo[k] : mine.need_lo[k]; e < (phase == 0 ? mine.rel_hi[k] : mine.need_hi[k]); ++e, --at) {
                if (phase == 0) { a.free_pages[at] = row[e]; row[e] = -1; }
                else row[e] = a.free_pages[at];
              }
          }
          if (flags & 4u) {                                  // ... or a warp for a sequence that has more: warp + 16 lane
            s_rel[tid] = first; s_own[tid] = n_own;
            __syncthreads();
#pragma unroll 1
            for (unsigned m = __ballot_sync(0xffffffffu, s_own[warp + PAGE_WARPS * lane] > FEW_ENTRIES); m; m &= m - 1)
              move_warp(c0, warp + PAGE_WARPS * (__ffs((int)m) - 1), phase);
            __syncthreads();
          }
          continue;
        }
        // many: a warp of the cluster for every sequence of the chunk
        s_rel[tid] = first;
        __syncthreads();
#pragma unroll 1
        for (int i = cta * PAGE_WARPS + warp; i < PAGE_THREADS && c0 + i < a.B; i += n_cta * PAGE_WARPS) move_warp(c0, i, phase);
        __syncthreads();
      }
    if (n_cta > 1) cluster_barrier(); else __syncthreads();
  }
  // (4) slots.  Packed: a warp takes 256 rows at a time, finds the sequence of the first and walks on from there.
  if (a.slot_map && single) {
    const int up = (1 << a.page_log2) - 1;
    auto slot_at = [&](int pg, int x) { return pg >= 0 && pg < a.n_pages ? (pg << a.page_log2) | (x & up) : -1; };
    auto row_of = [&](int b, int k) { const int reps = s_reps[b]; return k < reps ? s_rep0[b] + k : s_tok0[b] + (k - reps); };
    auto page_of = [&](int b, int x) { return a.table[(size_t)b * a.width + (x >> a.page_log2)]; };
    const int R = s_row[a.B];
    auto seq_at = [&](long long i) {                         // packed, i < R: the last sequence that starts at or before row i
      int lo = 0, hi = a.B;
      while (lo + 1 < hi) { const int mid = (lo + hi) >> 1; if (s_row[mid] <= i) lo = mid; else hi = mid; }
      return lo;
    };
    if (a.per_seq > 0 || a.n_rows <= gthreads) {             // a row per thread
      for (long long i = gtid; i < a.n_rows; i += gthreads) {
        int b = 0, k = 0x7fffffff, slot = -1;
        if (a.per_seq > 0) { b = (int)i / a.per_seq; k = (int)i - b * a.per_seq; }
        else if (i < R) { b = seq_at(i); k = (int)i - s_row[b]; }
        if (k < s_rows[b]) { const int x = row_of(b, k); slot = slot_at(page_of(b, x), x); }
        a.slot_map[i] = slot;
      }
    } else {
      // Many: a warp takes 256 rows at a time, a thread twice four neighbours, which lie on two pages at most unless a sequence
      // or its representatives end among them (a row at a time, the index arithmetic of sixteen SMs takes 10 us for 324000 rows).
      const bool wide = (reinterpret_cast<uintptr_t>(a.slot_map) & 15u) == 0;
#pragma unroll 1
      for (long long i0 = ((long long)cta * PAGE_WARPS + warp) * 256; i0 < a.n_rows; i0 += (long long)n_cta * PAGE_WARPS * 256) {
        int b = i0 < R ? seq_at(i0) : 0;
        int x[2], p0[2], p1[2], seq[2];
        bool plain[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const long long i = i0 + 128 * u + 4 * lane;
          plain[u] = false; x[u] = 0; p0[u] = p1[u] = -1;
          if (i < R) {
            while (i >= s_row[b + 1]) ++b;
            const int k = (int)i - s_row[b], reps = s_reps[b];
            plain[u] = k + 3 < s_rows[b] && (k >= reps || k + 3 < reps);
            if (plain[u]) { x[u] = row_of(b, k); p0[u] = page_of(b, x[u]); p1[u] = page_of(b, x[u] + 3); }
          }
          seq[u] = b;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const long long i = i0 + 128 * u + 4 * lane;
          int slot[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) slot[r] = slot_at((x[u] & up) + r <= up ? p0[u] : p1[u], x[u] + r);
          if (!plain[u] && i < R) {
            int c = seq[u];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              slot[r] = -1;
              if (i + r < R) {
                while (i + r >= s_row[c + 1]) ++c;
                const int y = row_of(c, (int)(i + r) - s_row[c]);
                slot[r] = slot_at(page_of(c, y), y);
              }
            }
          }
          if (wide && i + 3 < a.n_rows) *reinterpret_cast<int4*>(a.slot_map + i) = make_int4(slot[0], slot[1], slot[2], slot[3]);
          else
#pragma unroll
            for (int r = 0; r < 4; ++r) if (i + r < a.n_rows) a.slot_map[i + r] = slot[r];
        }
      }
    }
  } else if (a.slot_map) {
    auto slot_of = [&](int b, long long k, long long rows) {
      if (k >= rows) return -1;
      const int r0 = a.n_rep ? a.held_rep[b] : 0, r1 = a.n_rep ? a.n_rep[b] : 0, reps = max(r1 - r0, 0);
      const int first = (int)max((long long)a.held_tok[b], (long long)r1 * a.g);
      const int x = k < reps ? r0 + (int)k : first + (int)(k - reps);
      const int page = a.table[(size_t)b * a.width + (x >> a.page_log2)];
      return page >= 0 && page < a.n_pages ? (page << a.page_log2) | (x & ((1 << a.page_log2) - 1)) : -1;
    };
    if (a.per_seq > 0) {
      for (long long i = gtid; i < a.n_rows; i += gthreads) {
        const int b = (int)i / a.per_seq;
        const int r0 = a.n_rep ? a.held_rep[b] : 0, r1 = a.n_rep ? a.n_rep[b] : 0;
        const long long first = max((long long)a.held_tok[b], (long long)r1 * a.g);
        a.slot_map[i] = slot_of(b, (int)i - b * a.per_seq, max(r1 - r0, 0) + max((long long)a.n_tok[b] - first, 0ll));
      }
    } else {
      const long long R = (long long)tot[1];
#pragma unroll 1
      for (long long i0 = ((long long)cta * PAGE_WARPS + warp) * 256; i0 < a.n_rows; i0 += (long long)n_cta * PAGE_WARPS * 256) {
        int b = i0 < R ? seq_of(a.row_offsets, a.B, i0) : 0;
        long long lo = i0 < R ? a.row_offsets[b] : 0, hi = i0 < R ? a.row_offsets[b + 1] : 0;
#pragma unroll 2
        for (int u = 0; u < 8; ++u) {
          const long long i = i0 + 32 * u + lane;
          if (i >= a.n_rows) break;
          int slot = -1;
          if (i < R) {
            while (i >= hi) { ++b; lo = hi; hi = a.row_offsets[b + 1]; }
            slot = slot_of(b, i - lo, hi - lo);
          }
          a.slot_map[i] = slot;
        }
      }
    }
  }
  if (n_cta > 1) cluster_barrier(); else __syncthreads();    // the held state is read until here
  for (long long b = gtid; b < a.B; b += gthreads) {
    a.held_tok[b] = a.n_tok[b];
    if (a.n_rep) a.held_rep[b] = a.n_rep[b];
  }
  if (gtid == 0) { a.n_free[0] = (int32_t)(have - n_need); a.status[0] = 0; }
}

int page_update_launch(const lca_params* p, const lca_paged8* c, const int32_t* n_rep, const int32_t* n_tok, int32_t* held_rep,
                       int32_t* held_tok, int32_t* free_pages, int32_t* n_free, int32_t* slot_map, int n_rows, int rows_per_seq,
                       int32_t* row_offsets, int32_t* status, cudaStream_t stream) {
  const int lg = c->page_size == 16 ? 4 : c->page_size == 32 ? 5 : c->page_size == 64 ? 6 : 7;
  PageArgs a = {n_rep, n_tok, held_rep, held_tok, c->block_table, free_pages, n_free, slot_map, row_offsets, status,
                p->batch, n_rep ? p->group_size : 1, lg, c->table_width, c->n_pages, slot_map ? n_rows : 0, rows_per_seq};
  // The host does not know how many pages change hands.  Slots for many rows, or many tables that may be given back, want
  // many threads; otherwise the barriers of a cluster cost more than its threads bring.
  const long long entries = (long long)p->batch * c->table_width;
  const bool big = p->batch > PAGE_THREADS || a.n_rows > 8192 || (!slot_map && entries > 8192);
  if (big && cudaFuncSetAttribute(page_update_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return LCA_ERR_CUDA;
  return launch_chained(page_update_kernel, big ? 16 : 1, PAGE_THREADS, 0, stream, big ? 16 : 1, a);
}

// ------------------------------------------------------------------------------------------------------------- write
// A run (rows of one page in one call) and a block (GQA: K or V of one KV head; MLA: latent and rope key together) at a time.
// The rows of a run stay in registers between the maximum and the rounding, so the input is read once.  HBM-bound: 2 bytes
// in, 1 byte out per element (323584 rows of the MLA shape: 559 MB in 96 us, 5.8 TB/s; 29000 rows of 8 KV heads: 178 MB in
// 31 us, 5.7 TB/s).  A decode step of 64 rows is one launch's latency, 3 us.
struct WriteArgs {
  const bf16* rows_sem; const bf16* rows_pos; const int32_t* slots;
  uint8_t* pages_sem; uint8_t* pages_pos; float* scale_sem; float* scale_pos;
  long long n_rows, n_slots;
  int Hkv, window;           // rows whose runs are handled together
};

// log2 of the scale for a block whose largest finite |x| has these bf16 bits: smallest e with |x| <= 448 * 2^e
__device__ __forceinline__ int scale_exponent(uint32_t bits) {
  const int E = (int)(bits >> 7), M = (int)(bits & 0x7f);
  const int e = E - 127 - 8 + (M > 96 ? 1 : 0);              // 448 = 1.75 * 2^8, 1.75 = 1 + 96 / 128
  return max(E == 0 ? -1000 : e, PAGED8_MIN_EXP);
}

// The runs that start in rows [i0, i0 + window): a row starts one unless it follows its predecessor inside the same page.
// Bit k of the result: row i0 + 32 c + k (every lane of the warp gets the word of chunk c).
template <int P>
__device__ __forceinline__ unsigned run_heads(const WriteArgs& a, long long i0, int c) {
  const int k = 32 * c + (int)(threadIdx.x & 31);
  const long long i = i0 + k;
  bool head = false;
  if (k < a.window && i < a.n_rows) {
    const int s = a.slots[i], prev = i > 0 ? a.slots[i - 1] : -1;
    head = s >= 0 && s < a.n_slots && !(prev >= 0 && s == prev + 1 && s % P != 0);
  }
  return __ballot_sync(0xffffffffu, head);
}
// Rows of the run that starts at row i with this slot (every lane of the warp).
template <int P>
__device__ __forceinline__ int run_length(const WriteArgs& a, long long i, int slot) {
  const int room = P - slot % P;
  int n = 0;
#pragma unroll 1
  for (int k = 0; k < P; k += 32) {
    const int j = k + (int)(threadIdx.x & 31);
    const bool in = j < room && i + j < a.n_rows && a.slots[i + j] == slot + j;
    const unsigned ok = __ballot_sync(0xffffffffu, in);
    if (ok != 0xffffffffu) return n + __ffs((int)~ok) - 1;
    n += 32;
  }
  return n;
}
// Largest finite |x| of vectors of 8 bf16 values, as bf16 bits: two at a time, and again element by element where that finds
// an infinity or a NaN.
template <int N>
__device__ __forceinline__ uint32_t max_finite(const uint4 (&v)[N]) {
  uint32_t m = 0;
#pragma unroll
  for (int q = 0; q < N; ++q) {
    m = __vmaxu2(m, v[q].x & 0x7fff7fffu); m = __vmaxu2(m, v[q].y & 0x7fff7fffu);
    m = __vmaxu2(m, v[q].z & 0x7fff7fffu); m = __vmaxu2(m, v[q].w & 0x7fff7fffu);
  }
  uint32_t top = max(m & 0xffffu, m >> 16);
  if (top >= 0x7f80u) {
    top = 0;
#pragma unroll
    for (int q = 0; q < N; ++q) {
      const uint32_t u[4] = {v[q].x, v[q].y, v[q].z, v[q].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t lo = u[k] & 0x7fffu, hi = (u[k] >> 16) & 0x7fffu;
        top = max(top, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
      }
    }
  }
  return top;
}
__device__ __forceinline__ uint2 quantise8(const uint4& v, float inv) {
  return make_uint2(e4m3x4_from_bf16(v.x, v.y, inv), e4m3x4_from_bf16(v.z, v.w, inv));
}
// Rows [0, n16) units of 16 codes, times f, rounded again: thread `t` of `nt`.
__device__ __forceinline__ void rescale_codes(uint8_t* codes, int n16, float f, int t, int nt) {
#pragma unroll 1
  for (int x = t; x < n16; x += nt) {
    uint4* q = reinterpret_cast<uint4*>(codes) + x;
    uint4 w = *q;
    w.x = e4m3x4_scale(w.x, f); w.y = e4m3x4_scale(w.y, f); w.z = e4m3x4_scale(w.z, f); w.w = e4m3x4_scale(w.w, f);
    *q = w;
  }
}

// MLA: one CTA per run; with one KV head the rows of a run are contiguous in the input and in the page.
template <int D_SEM, int P>
struct WriteMla {
  static constexpr int NT = D_SEM == 512 && P >= 64 ? 512 : 256;
  static constexpr int NS = (P * D_SEM / 8 + NT - 1) / NT, NP = (P * 8 + NT - 1) / NT;       // vectors of a thread
  static constexpr int CTAS = NS + NP > 12 ? 1 : NT == 512 ? 2 : 4;
};
template <int D_SEM, int P>
__global__ void __launch_bounds__(WriteMla<D_SEM, P>::NT, WriteMla<D_SEM, P>::CTAS) paged8_write_mla_kernel(WriteArgs a) {
  constexpr int NT = WriteMla<D_SEM, P>::NT, NS = WriteMla<D_SEM, P>::NS, NP = WriteMla<D_SEM, P>::NP, D_POS = 64;
  __shared__ uint32_t s_red[NT / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long i0 = (long long)blockIdx.x * a.window;
  chain_wait();
  chain_next();
#pragma unroll 1
  for (int c = 0; 32 * c < a.window; ++c)
#pragma unroll 1
    for (unsigned heads = run_heads<P>(a, i0, c); heads; heads &= heads - 1) {        // the same in every warp
      const long long i = i0 + 32 * c + __ffs((int)heads) - 1;
      const int slot = a.slots[i], page = slot / P, off = slot % P, n = run_length<P>(a, i, slot);
      const float old = off > 0 ? a.scale_sem[page] : 0.f;
      const uint4* src_s = reinterpret_cast<const uint4*>(a.rows_sem + (size_t)i * D_SEM);
      const uint4* src_p = reinterpret_cast<const uint4*>(a.rows_pos + (size_t)i * D_POS);
      uint4 vs[NS], vp[NP];
#pragma unroll
      for (int q = 0; q < NS; ++q) vs[q] = q * NT + tid < n * (D_SEM / 8) ? __ldcs(src_s + q * NT + tid) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int q = 0; q < NP; ++q) vp[q] = q * NT + tid < n * (D_POS / 8) ? __ldcs(src_p + q * NT + tid) : make_uint4(0u, 0u, 0u, 0u);
      uint32_t top = __reduce_max_sync(0xffffffffu, max(max_finite(vs), max_finite(vp)));
      if (lane == 0) s_red[warp] = top;
      __syncthreads();                                        // also: every thread has read the block's old scale
#pragma unroll
      for (int k = 0; k < NT / 32; ++k) top = max(top, s_red[k]);
      const float want = exp2_int(scale_exponent(top)), now = off > 0 ? fmaxf(want, old) : want;
      uint8_t* dst_s = a.pages_sem + (size_t)page * P * D_SEM;
      uint8_t* dst_p = a.pages_pos + (size_t)page * P * D_POS;
      if (off > 0 && now > old) {                             // the block's scale grows: its rows are rounded again
        rescale_codes(dst_s, off * (D_SEM / 16), old / now, tid, NT);
        rescale_codes(dst_p, off * (D_POS / 16), old / now, tid, NT);
      }
      const float inv = 1.f / now;                            // exact: a power of two (unless `old` came from elsewhere)
      uint2* out_s = reinterpret_cast<uint2*>(dst_s + (size_t)off * D_SEM);
      uint2* out_p = reinterpret_cast<uint2*>(dst_p + (size_t)off * D_POS);
#pragma unroll
      for (int q = 0; q < NS; ++q) if (q * NT + tid < n * (D_SEM / 8)) out_s[q * NT + tid] = quantise8(vs[q], inv);
#pragma unroll
      for (int q = 0; q < NP; ++q) if (q * NT + tid < n * (D_POS / 8)) out_p[q * NT + tid] = quantise8(vp[q], inv);
      if (tid == 0) a.scale_sem[page] = now;
      __syncthreads();                                        // s_red is used again by the next run
    }
}

// GQA: a block is one KV head's keys or values of a page, at most 16 KB of input: one warp for 32 rows of it (two or four
// warps for larger pages), eight warps with neighbouring heads in a CTA.  No barrier but those warps' own.
template <int D, int P>
__global__ void __launch_bounds__(256, 2) paged8_write_gqa_kernel(WriteArgs a) {
  constexpr int WPB = P <= 32 ? 1 : P / 32, NT = 32 * WPB, V8 = D / 8, NV = P * V8 / NT;
  __shared__ uint32_t s_red[8];
  const int tid = threadIdx.x, warp = tid >> 5, group = warp / WPB, t = tid % NT;
  const long long item = (long long)blockIdx.x * (8 / WPB) + group;
  const int hk = (int)(item % a.Hkv), part = (int)((item / a.Hkv) & 1);
  const long long i0 = item / a.Hkv / 2 * a.window;
  chain_wait();
  chain_next();
  if (i0 >= a.n_rows) return;
  const bf16* src0 = part ? a.rows_pos : a.rows_sem;
  uint8_t* pages = part ? a.pages_pos : a.pages_sem;
  float* scale = part ? a.scale_pos : a.scale_sem;
  auto group_barrier = [&]() {
    if (WPB == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(NT) : "memory");
  };
#pragma unroll 1
  for (int c = 0; 32 * c < a.window; ++c)
#pragma unroll 1
    for (unsigned heads = run_heads<P>(a, i0, c); heads; heads &= heads - 1) {
      const long long i = i0 + 32 * c + __ffs((int)heads) - 1;
      const int slot = a.slots[i], page = slot / P, off = slot % P, n = run_length<P>(a, i, slot);
      const size_t block = (size_t)page * a.Hkv + hk;
      const float old = off > 0 ? scale[block] : 0.f;
      const uint4* src = reinterpret_cast<const uint4*>(src0 + ((size_t)i * a.Hkv + hk) * D);
      uint4 v[NV];
#pragma unroll
      for (int q = 0; q < NV; ++q) {
        const int x = q * NT + t, r = x / V8;
        v[q] = r < n ? __ldcs(src + (size_t)r * a.Hkv * V8 + x % V8) : make_uint4(0u, 0u, 0u, 0u);
      }
      uint32_t top = __reduce_max_sync(0xffffffffu, max_finite(v));
      if (WPB > 1) {
        if ((tid & 31) == 0) s_red[warp] = top;
        group_barrier();                                      // also: every thread has read the block's old scale
#pragma unroll
        for (int k = 0; k < WPB; ++k) top = max(top, s_red[group * WPB + k]);
      }
      const float want = exp2_int(scale_exponent(top)), now = off > 0 ? fmaxf(want, old) : want;
      uint8_t* dst = pages + block * P * D;
      if (off > 0 && now > old) rescale_codes(dst, off * (D / 16), old / now, t, NT);        // the block's scale grows
      const float inv = 1.f / now;
      uint2* out = reinterpret_cast<uint2*>(dst + (size_t)off * D);
#pragma unroll
      for (int q = 0; q < NV; ++q) if (q * NT + t < n * V8) out[q * NT + t] = quantise8(v[q], inv);
      group_barrier();                                        // the old scale has been read, s_red is used again
      if (t == 0) scale[block] = now;
    }
}

template <int D_SEM, bool MLA, int P>
static int write_launch(const WriteArgs& a, long long windows, cudaStream_t stream) {
  long long grid;
  if constexpr (MLA) {
    grid = windows;
    if (grid <= 0x7fffffffll) return launch_chained(paged8_write_mla_kernel<D_SEM, P>, (unsigned)grid, WriteMla<D_SEM, P>::NT, 0, stream, 1, a);
  } else {
    constexpr int PER = 8 / (P <= 32 ? 1 : P / 32);
    grid = (windows * a.Hkv * 2 + PER - 1) / PER;
    if (grid <= 0x7fffffffll) return launch_chained(paged8_write_gqa_kernel<D_SEM, P>, (unsigned)grid, 256, 0, stream, 1, a);
  }
  return LCA_ERR_UNSUPPORTED_SHAPE;
}
template <int D_SEM, bool MLA>
static int write_page_size(const WriteArgs& a, int page, long long windows, cudaStream_t stream) {
  switch (page) {
    case 16: return write_launch<D_SEM, MLA, 16>(a, windows, stream);
    case 32: return write_launch<D_SEM, MLA, 32>(a, windows, stream);
    case 64: return write_launch<D_SEM, MLA, 64>(a, windows, stream);
    default: return write_launch<D_SEM, MLA, 128>(a, windows, stream);
  }
}

int paged8_write_launch(const lca_params* p, const lca_paged8* c, const void* rows_sem, const void* rows_pos,
                        const int32_t* slot_map, long long n_rows, cudaStream_t stream) {
  const bool mla = p->variant == LCA_VARIANT_MLA;
  WriteArgs a = {(const bf16*)rows_sem, (const bf16*)rows_pos, slot_map, (uint8_t*)c->pages_sem, (uint8_t*)c->pages_pos, c->scale_sem,
                 c->scale_pos, n_rows, (long long)c->n_pages * c->page_size, p->n_kv_heads, 1};
  // A decode step brings one row per page: a CTA (a warp) per row, or it would handle its runs one after the other.  A prompt
  // brings whole pages: one per page of rows, or most would find no run to start.  In between: what fills the GPU twice.
  const long long per = n_rows * (mla ? 1 : 2 * p->n_kv_heads) / (mla ? 148 * 8 : 148 * 64);
  a.window = (int)(per < 1 ? 1 : (per > c->page_size ? c->page_size : per));
  const long long windows = (n_rows + a.window - 1) / a.window;
  if (mla) return p->d_sem == 512 ? write_page_size<512, true>(a, c->page_size, windows, stream)
                                  : write_page_size<128, true>(a, c->page_size, windows, stream);
  return p->d_sem == 128 ? write_page_size<128, false>(a, c->page_size, windows, stream)
                         : write_page_size<64, false>(a, c->page_size, windows, stream);
}

// ------------------------------------------------------------------------------------------------------------ update
// Condensation of the earliest group of every sequence that is due (Sec. 4.2 / 4.3) from the 8-bit values: fp64 scores,
// arg-max on them (lowest index on ties), fp32 softmax and pooling, one rounding to bf16.  One CTA per (sequence, KV
// head), a launch of a few dozen CTAs that read 37 KB each (g = 64, 576 wide): bound by the latency of what depends on each
// other, counters, table, codes.  A warp therefore takes whole rows: it looks up their pages itself, keeps its lanes' share
// of the query in registers and multiplies the codes as they arrive; shared memory only carries them to the pooling, for
// which the rows are split over all threads.  (With the group brought to shared memory first, the query read from there
// and a thread per four columns in the pooling: 10.5 us instead of 8.5 for 64 sequences of the MLA shape, 8.5
// instead of 6.2 for 48 sequences with 8 KV heads.)
struct Update8Args {
  const uint8_t* pages_sem; const uint8_t* pages_pos; const float* scale_sem; const float* scale_pos; const int32_t* table;
  const float* qbar_f; const double* qbar_d;
  const int32_t* n_rep; const int32_t* n_tok; int32_t* n_rep_new;
  bf16* rep_sem; bf16* rep_pos; int32_t* anchor;
  int Hkv, g, w, page_log2, n_pages, width;
  double scale;
};
static const int UPD_THREADS = 512, UPD_WARPS = UPD_THREADS / 32;

// N consecutive codes (2, 4 or 16) as words; two codes in the low half of one
template <int N>
struct Codes {
  uint32_t w[(N + 3) / 4];
  __device__ __forceinline__ void load(const uint8_t* p) {
    if constexpr (N == 2) w[0] = *reinterpret_cast<const uint16_t*>(p);
    else if constexpr (N == 4) w[0] = *reinterpret_cast<const uint32_t*>(p);
    else { const uint4 v = *reinterpret_cast<const uint4*>(p); w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
  }
  __device__ __forceinline__ void store(uint8_t* p) const {
    if constexpr (N == 2) *reinterpret_cast<uint16_t*>(p) = (uint16_t)w[0];
    else if constexpr (N == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
    else *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ double dot(const double (&q)[N], float scale, double acc) const {
#pragma unroll
    for (int k = 0; k < N; k += 4) {
      const float4 f = e4m3x4_to_float4(w[k / 4]);
      acc = fma(q[k], (double)(f.x * scale), acc); acc = fma(q[k + 1], (double)(f.y * scale), acc);
      if constexpr (N > 2) { acc = fma(q[k + 2], (double)(f.z * scale), acc); acc = fma(q[k + 3], (double)(f.w * scale), acc); }
    }
    return acc;
  }
};

template <bool MLA, int DS, int DP>
__global__ void __launch_bounds__(UPD_THREADS) paged8_update_kernel(Update8Args a) {
  constexpr int NS = DS / 32, NP = DP / 32, SEM_Q = MLA ? DS : 0, DK = SEM_Q + DP;
  constexpr int COLS = DS / 4, GROUPS = UPD_THREADS / COLS;   // pooling: threads across a row, groups of rows
  constexpr int ROWS = 4;                                     // rows whose loads a warp has in flight
  extern __shared__ __align__(16) unsigned char smem_raw[];
  float4* s_part = reinterpret_cast<float4*>(smem_raw);       // [GROUPS][COLS]
  const int g = a.g;                                          // a multiple of 16
  double* s_s = reinterpret_cast<double*>(s_part + UPD_THREADS);
  float* s_a = reinterpret_cast<float*>(s_s + g);
  float* s_fs = s_a + g;                                      // scale of each row's sem / pos codes
  float* s_fp = s_fs + g;
  uint8_t* t_sem = reinterpret_cast<uint8_t*>(s_fp + g);
  uint8_t* t_pos = t_sem + (size_t)g * DS;
  __shared__ int s_anchor;
  const int hk = (int)(blockIdx.x % a.Hkv), b = (int)(blockIdx.x / a.Hkv);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  chain_wait();
  chain_next();
  const int nr = a.n_rep[b], nt = a.n_tok[b];
  const long long first = (long long)nr * g, cap = (long long)a.width << a.page_log2;
  const bool due = nr >= 0 && nt >= 0 && nt <= cap && (long long)nt - first >= (long long)a.w + g;
  int missing = 0;
  if (due) {
    const size_t q0 = ((size_t)b * a.Hkv + hk) * DK;
    double qs[MLA ? NS : 1], qp[NP];
    if constexpr (MLA)
#pragma unroll
      for (int k = 0; k < NS; ++k) qs[k] = a.qbar_f ? (double)a.qbar_f[q0 + lane * NS + k] : a.qbar_d[q0 + lane * NS + k];
#pragma unroll
    for (int k = 0; k < NP; ++k) qp[k] = a.qbar_f ? (double)a.qbar_f[q0 + SEM_Q + lane * NP + k] : a.qbar_d[q0 + SEM_Q + lane * NP + k];
#pragma unroll 1
    for (int i0 = warp; i0 < g; i0 += ROWS * UPD_WARPS) {
      Codes<NS> cs[ROWS];
      Codes<NP> cp[ROWS];
      float fs[ROWS], fp[ROWS];
      int page[ROWS];
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        const int i = i0 + r * UPD_WARPS;
        page[r] = i < g ? a.table[(size_t)b * a.width + ((first + i) >> a.page_log2)] : 0;
        if (page[r] < 0 || page[r] >= a.n_pages) { missing = 1; page[r] = 0; }       // any page: nothing is made of it
      }
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        const int i = i0 + r * UPD_WARPS;
        if (i < g) {
          const size_t block = (size_t)page[r] * a.Hkv + hk, row = (block << a.page_log2) + (size_t)((first + i) & ((1 << a.page_log2) - 1));
          cs[r].load(a.pages_sem + row * DS + lane * NS);
          cp[r].load(a.pages_pos + row * DP + lane * NP);
          fs[r] = a.scale_sem[block];
          fp[r] = a.scale_pos ? a.scale_pos[block] : fs[r];
        }
      }
      double acc[ROWS];
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        const int i = i0 + r * UPD_WARPS;
        acc[r] = 0.0;
        if (i < g) {
          cs[r].store(t_sem + (size_t)i * DS + lane * NS);
          cp[r].store(t_pos + (size_t)i * DP + lane * NP);
          if constexpr (MLA) acc[r] = cs[r].dot(qs, fs[r], 0.0);
          acc[r] = cp[r].dot(qp, fp[r], acc[r]);
        }
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int r = 0; r < ROWS; ++r) acc[r] += __shfl_xor_sync(0xffffffffu, acc[r], o);
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        const int i = i0 + r * UPD_WARPS;
        if (lane == 0 && i < g) { s_s[i] = acc[r] * a.scale; s_fs[i] = fs[r]; s_fp[i] = fp[r]; }
      }
    }
  }
  const bool done = !__syncthreads_or(missing) && due;
  if (hk == 0 && tid == 0) a.n_rep_new[b] = nr + (done ? 1 : 0);
  if (!done) {
    if (tid == 0) a.anchor[b * a.Hkv + hk] = -1;
    return;
  }
  if (warp == 0) {
    double best = -INFINITY;
    int besti = 0x7fffffff;
    for (int i = lane; i < g; i += 32) { const double v = s_s[i]; if (v > best) { best = v; besti = i; } }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const double ob = __shfl_xor_sync(0xffffffffu, best, o);
      const int oi = __shfl_xor_sync(0xffffffffu, besti, o);
      if (ob > best || (ob == best && oi < besti)) { best = ob; besti = oi; }
    }
    float z = 0.f;
    for (int i = lane; i < g; i += 32) { const float e = expf((float)(s_s[i] - best)); s_a[i] = e; z += e; }
    z = warp_sum(z);
    const float inv = 1.f / z;
    for (int i = lane; i < g; i += 32) s_a[i] *= inv;
    if (lane == 0) s_anchor = min(besti, g - 1);              // no finite score at all (NaN): the last token
  }
  __syncthreads();
  const size_t o = (size_t)b * a.Hkv + hk;
  {
    const int c = tid % COLS, grp = tid / COLS;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int i = grp; i < g; i += GROUPS) {
      const float4 f = e4m3x4_to_float4(*reinterpret_cast<const uint32_t*>(t_sem + (size_t)i * DS + 4 * c));
      const float fs = s_fs[i], w = s_a[i];
      acc.x = fmaf(w, f.x * fs, acc.x); acc.y = fmaf(w, f.y * fs, acc.y); acc.z = fmaf(w, f.z * fs, acc.z); acc.w = fmaf(w, f.w * fs, acc.w);
    }
    s_part[tid] = acc;
  }
  __syncthreads();
  if (tid < COLS) {
    float4 acc = s_part[tid];
#pragma unroll
    for (int k = 1; k < GROUPS; ++k) {
      const float4 v = s_part[k * COLS + tid];
      acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
    }
    *reinterpret_cast<uint2*>(a.rep_sem + o * DS + 4 * tid) = make_uint2(tc::pack_bf16x2(acc.x, acc.y), tc::pack_bf16x2(acc.z, acc.w));
  } else if (tid >= UPD_THREADS - DP / 4) {
    const int ia = s_anchor, c = 4 * (tid - (UPD_THREADS - DP / 4));
    const float4 f = e4m3x4_to_float4(*reinterpret_cast<const uint32_t*>(t_pos + (size_t)ia * DP + c));
    const float fp = s_fp[ia];
    *reinterpret_cast<uint2*>(a.rep_pos + o * DP + c) = make_uint2(tc::pack_bf16x2(f.x * fp, f.y * fp), tc::pack_bf16x2(f.z * fp, f.w * fp));
  }
  if (tid == 0) a.anchor[o] = s_anchor;
}

size_t paged8_update_smem_bytes(const lca_params* p) {
  const size_t g = (size_t)p->group_size;
  return UPD_THREADS * sizeof(float4) + g * (sizeof(double) + 3 * sizeof(float)) + g * (size_t)(p->d_sem + p->d_pos);
}

template <bool MLA, int DS, int DP>
static int update8_launch(const Update8Args& a, long long grid, size_t smem, cudaStream_t stream) {
  auto kern = paged8_update_kernel<MLA, DS, DP>;
  // The limit belongs to the kernel, not to the call: every call sets the same one, so that another thread's call with a smaller
  // group does not lower it before this one's launch.
  if (smem > 48 * 1024 && cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, PAGED8_UPDATE_SMEM) != cudaSuccess)
    return LCA_ERR_CUDA;
  return launch_chained(kern, (unsigned)grid, UPD_THREADS, smem, stream, 1, a);
}

int paged8_update_launch(const lca_params* p, const lca_paged8* c, const float* qbar_f, const double* qbar_d, const int32_t* n_rep,
                         const int32_t* n_tok, int32_t* n_rep_new, void* rep_sem, void* rep_pos, int32_t* anchor_out,
                         cudaStream_t stream) {
  const int lg = c->page_size == 16 ? 4 : c->page_size == 32 ? 5 : c->page_size == 64 ? 6 : 7;
  Update8Args a = {(const uint8_t*)c->pages_sem, (const uint8_t*)c->pages_pos, c->scale_sem, c->scale_pos, c->block_table, qbar_f, qbar_d,
                   n_rep, n_tok, n_rep_new, (bf16*)rep_sem, (bf16*)rep_pos, anchor_out, p->n_kv_heads, p->group_size,
                   p->window, lg, c->n_pages, c->table_width, (double)p->softmax_scale};
  const long long grid = (long long)p->batch * p->n_kv_heads;
  if (grid > 0x7fffffffll) return LCA_ERR_UNSUPPORTED_SHAPE;
  const size_t smem = paged8_update_smem_bytes(p);
  if (p->variant == LCA_VARIANT_MLA) return p->d_sem == 512 ? update8_launch<true, 512, 64>(a, grid, smem, stream)
                                                            : update8_launch<true, 128, 64>(a, grid, smem, stream);
  return p->d_sem == 128 ? update8_launch<false, 128, 128>(a, grid, smem, stream) : update8_launch<false, 64, 64>(a, grid, smem, stream);
}

}  // namespace lca
