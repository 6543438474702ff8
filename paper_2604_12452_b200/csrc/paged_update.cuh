// The online condensation of a group from a paged cache of 8-bit or 4-bit rows.
#pragma once

#include <type_traits>

#include "fp4_common.cuh"
#include "lca_common.cuh"
#include "tc_common.cuh"

namespace lca {

// ------------------------------------------------------------------------------------------------------------ update
// Condensation of the earliest group of every sequence that is due (Sec. 4.2 / 4.3) from the cached values: fp64 scores,
// arg-max on them (lowest index on ties), fp32 softmax and pooling, one rounding to bf16.  One CTA per (sequence, KV
// head), a launch of a few dozen CTAs that read 37 KB each (g = 64, 576 wide): bound by the latency of what depends on each
// other, counters, table, codes.  A warp therefore takes whole rows: it looks up their pages itself, keeps its lanes' share
// of the query in registers and multiplies the codes as they arrive; shared memory only carries them to the pooling, for
// which the rows are split over all threads.  (With the group brought to shared memory first, the query read from there
// and a thread per four columns in the pooling: 10.5 us instead of 8.5 for 64 sequences of the MLA shape, 8.5
// instead of 6.2 for 48 sequences with 8 KV heads.)
// The group is held as e4m3 codes with a factor for each row: the 8-bit cache as it stands (PagedRows8), the 4-bit cache expanded
// (PagedRows4).
struct PagedRows8 { const uint8_t* pages_sem; const uint8_t* pages_pos; const float* scale_sem; const float* scale_pos; };
struct PagedRows4 {
  const uint8_t* pages_sem; const uint8_t* pages_pos; const uint8_t* shift_sem; const uint8_t* shift_pos;
  const uint8_t* exp_sem; const uint8_t* exp_pos;
};
template <class Rows>
struct PagedUpdateArgs {
  Rows rows;
  const int32_t* table;
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
  // the same columns [N lane, N lane + N) from 4-bit codes and their blocks' shifts
  __device__ __forceinline__ void load4(const uint8_t* codes, const uint8_t* shifts, int lane, const uint2* s_table) {
    const int block = lane * N / 32;
    const uint2 table = s_table[(shifts[block >> 1] >> (4 * (block & 1))) & 15];
    const uint32_t* words = reinterpret_cast<const uint32_t*>(codes);
    if constexpr (N == 16) {
      const uint2 v = reinterpret_cast<const uint2*>(words)[lane], a = paged4_expand(v.x, table), b = paged4_expand(v.y, table);
      w[0] = a.x; w[1] = a.y; w[2] = b.x; w[3] = b.y;
    } else {
      const uint2 a = paged4_expand(words[lane * N / 8], table);
      const uint32_t half = (lane * N) & 4 ? a.y : a.x;
      w[0] = N == 4 ? half : (half >> (8 * ((lane * N) & 2))) & 0xffffu;
    }
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

// Row `row` of the pool, in block (page, KV head) `block`: this lane's codes and the factors of both parts.
template <int NS, int NP, int DS, int DP>
__device__ __forceinline__ void load_row(const PagedRows8& r, size_t block, size_t row, int lane, const uint2*, Codes<NS>& cs, Codes<NP>& cp,
                                         float& fs, float& fp) {
  cs.load(r.pages_sem + row * DS + lane * NS);
  cp.load(r.pages_pos + row * DP + lane * NP);
  fs = r.scale_sem[block];
  fp = r.scale_pos ? r.scale_pos[block] : fs;
}
template <int NS, int NP, int DS, int DP>
__device__ __forceinline__ void load_row(const PagedRows4& r, size_t, size_t row, int lane, const uint2* s_table, Codes<NS>& cs, Codes<NP>& cp,
                                         float& fs, float& fp) {
  cs.load4(r.pages_sem + row * (DS / 2), r.shift_sem + row * (DS / 64), lane, s_table);
  cp.load4(r.pages_pos + row * (DP / 2), r.shift_pos + row * (DP / 64), lane, s_table);
  fs = paged4_factor(r.exp_sem[row]);
  fp = r.exp_pos ? paged4_factor(r.exp_pos[row]) : fs;
}

template <class Rows, bool MLA, int DS, int DP>
__global__ void __launch_bounds__(UPD_THREADS) paged_update_kernel(PagedUpdateArgs<Rows> a) {
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
  __shared__ uint2 s_table[16];
  const int hk = (int)(blockIdx.x % a.Hkv), b = (int)(blockIdx.x / a.Hkv);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if constexpr (std::is_same<Rows, PagedRows4>::value) {
    paged4_table_load(s_table, tid);
    __syncthreads();
  }
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
          load_row<NS, NP, DS, DP>(a.rows, block, row, lane, s_table, cs[r], cp[r], fs[r], fp[r]);
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

inline size_t paged_update_smem_bytes(const lca_params* p) {
  const size_t g = (size_t)p->group_size;
  return UPD_THREADS * sizeof(float4) + g * (sizeof(double) + 3 * sizeof(float)) + g * (size_t)(p->d_sem + p->d_pos);
}

template <class Rows, bool MLA, int DS, int DP>
int paged_update_launch(const PagedUpdateArgs<Rows>& a, long long grid, size_t smem, cudaStream_t stream) {
  auto kern = paged_update_kernel<Rows, MLA, DS, DP>;
  // The limit belongs to the kernel, not to the call: every call sets the same one, so that another thread's call with a smaller
  // group does not lower it before this one's launch.
  if (smem > 48 * 1024 && cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, PAGED8_UPDATE_SMEM) != cudaSuccess)
    return LCA_ERR_CUDA;
  return launch_chained(kern, (unsigned)grid, UPD_THREADS, smem, stream, 1, a);
}

template <class Rows, class Cache>
int paged_update_shapes(const lca_params* p, const Cache* c, const Rows& rows, const float* qbar_f, const double* qbar_d, const int32_t* n_rep,
                        const int32_t* n_tok, int32_t* n_rep_new, void* rep_sem, void* rep_pos, int32_t* anchor_out, cudaStream_t stream) {
  const int lg = c->page_size == 16 ? 4 : c->page_size == 32 ? 5 : c->page_size == 64 ? 6 : 7;
  PagedUpdateArgs<Rows> a = {rows, c->block_table, qbar_f, qbar_d, n_rep, n_tok, n_rep_new, (bf16*)rep_sem, (bf16*)rep_pos, anchor_out,
                             p->n_kv_heads, p->group_size, p->window, lg, c->n_pages, c->table_width, (double)p->softmax_scale};
  const long long grid = (long long)p->batch * p->n_kv_heads;
  if (grid > 0x7fffffffll) return LCA_ERR_UNSUPPORTED_SHAPE;
  const size_t smem = paged_update_smem_bytes(p);
  if (p->variant == LCA_VARIANT_MLA) return p->d_sem == 512 ? paged_update_launch<Rows, true, 512, 64>(a, grid, smem, stream)
                                                            : paged_update_launch<Rows, true, 128, 64>(a, grid, smem, stream);
  return p->d_sem == 128 ? paged_update_launch<Rows, false, 128, 128>(a, grid, smem, stream)
                         : paged_update_launch<Rows, false, 64, 64>(a, grid, smem, stream);
}

}  // namespace lca
