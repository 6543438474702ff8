// What the two tensor-core kernels over the paged 8-bit cache share: the line of tiles and its ranges, operand splitting,
// instruction and shared-memory descriptors, and the kernel that merges the pieces.
#pragma once

#include "fp8_common.cuh"
#include "lca_common.cuh"
#include "tc_common.cuh"

namespace lca {
using namespace tc;

// A raised maximum puts the largest weight at 2^5 (pairs, blocks of 128 rows: 2^8); it may grow until its leading term is as large as
// its format allows before the maximum is raised again.
__host__ __device__ constexpr float paged8_t_bits(int rows) { return rows == 128 ? 8.f : 5.f; }

// Offset of a key before the second term of its weight is rounded, in [-1/2, 1/2] of the smallest e4m3 step (2^-9): the row times the
// golden ratio, modulo 1.  At either end a weight of 0 still rounds to 0 (a tie, to even).
static constexpr uint32_t GOLDEN = 0x9E3779B9u;              // 2^32 / golden ratio
__device__ __forceinline__ float weight_offset(int row) { return (float)(int)((uint32_t)row * GOLDEN) * 0x1p-41f; }

struct Paged8Params {
  CUtensorMap sem, pos;       // [n_pages * Hkv, page, d] codes; boxes of one page x 128 (or 64) bytes
  const bf16* q_sem; const bf16* q_pos;
  const float* scale_k; const float* scale_v; const int32_t* table;
  const int32_t* n_rep; const int32_t* n_tok;
  bf16* out; float* lse;
  float* part;                // [2 * grid][NH][DS] partial O, then [2 * grid][2][NH] M and l
  long long* prefix;          // [B + 2] tiles before each sequence (all units), then 1 where every unit has a CTA; for B > MERGE_B, written by CTA 0
  int B, Hq, Hkv, q_len, g, page, page_log2, n_pages, width, rep, n_blk, grid;   // grid: CTAs (pairs of them) that share the line
  int out_wide;               // out is 32-byte aligned
  float scale_log2, bias_log2;
};

// Tiles of 128 rows of a sequence: those with representatives, then those with tokens.
struct TileSpan {
  PagedSpan s;
  int n_a, b0, n;
  __device__ __forceinline__ int row0(int i) const { return (i < n_a ? i : b0 + (i - n_a)) * 128; }
};
__device__ __forceinline__ TileSpan tile_span(const Paged8Params& p, int b) {
  TileSpan t;
  t.s = paged_span(p.n_rep, p.n_tok, b, p.g, p.width * p.page);
  t.n_a = (t.s.n_rep + 127) >> 7;
  t.b0 = max(t.s.tok0 >> 7, t.n_a);
  t.n = t.n_a + (t.s.n_tok > t.s.tok0 ? max(((t.s.n_tok + 127) >> 7) - t.b0, 0) : 0);
  return t;
}
// The line of T tiles is cut into G ranges: CTA c takes tiles [start(c), start(c + 1)), the first `rest` of them one tile more.
// At least two tiles for a CTA that works (a range of one tile costs a partial result that another CTA has to merge).  The
// numbers fit 32 bits except in absurd cases; a 64-bit division costs several hundred clocks of a launch's first microseconds.
struct Cut {
  long long per;
  int G, rest;
  __device__ __forceinline__ Cut(long long T, int grid) {
    const long long half = (T + 1) >> 1;
    G = half < grid ? max((int)half, 1) : grid;
    if (T >> 32) { per = T / G; rest = (int)(T % G); }
    else { per = (unsigned)T / (unsigned)G; rest = (int)((unsigned)T % (unsigned)G); }
  }
  __device__ __forceinline__ long long start(int c) const { return c * per + min(c, rest); }
  __device__ __forceinline__ int owner(long long x) const {              // the CTA whose range holds tile x
    const long long big = rest * (per + 1);
    if (x < big) return (int)(big >> 32 ? x / (per + 1) : (unsigned)x / (unsigned)(per + 1));
    return rest + (int)((x - big) >> 32 || per >> 32 ? (x - big) / per : (unsigned)(x - big) / (unsigned)per);
  }
};

// The pieces of units in one CTA's range of the line.
struct Walk {
  int b;
  long long off, left;        // position inside sequence b's part of the line; tiles left in this CTA's range
  TileSpan t;
  int hk, blk, t0, n;         // current piece: tiles [t0, t0 + n) of unit (b, hk, blk)
  bool fresh;
  __device__ __forceinline__ bool next(const Paged8Params& p) {
    if (!fresh) off += n;
    while (left > 0) {
      if (b >= p.B) return false;
      t = tile_span(p, b);
      if (off < (long long)t.n * p.Hkv * p.n_blk) break;
      off -= (long long)t.n * p.Hkv * p.n_blk;
      ++b;
    }
    if (left <= 0) return false;
    const int u = off >> 32 ? (int)(off / t.n) : (int)((unsigned)off / (unsigned)t.n);
    t0 = (int)(off - (long long)u * t.n);
    if (p.n_blk == 1) { hk = u; blk = 0; }
    else { hk = u / p.n_blk; blk = u - hk * p.n_blk; }
    n = (int)min((long long)(t.n - t0), left);
    left -= n;
    fresh = false;
    return true;
  }
};

// The range of CTA (or CTA pair) `id` (s_warp: room for 12 bytes a warp): thread i sums the tiles of sequences [i q, (i + 1) q); every thread of the CTA calls it.
// Leaves the first sequence in *s_b, the offset inside it and the tiles of the range in s_off[0 .. 1]; ends with a barrier
// still to come.  CTA 0 of the grid writes the prefix sums for the merging kernel, which finds those of few sequences itself.
// Where there are no more units than CTAs and the longest is at most WHOLE_SLACK tiles above the mean of all CTAs, every unit
// has a CTA of its own: a cut costs a second query load, a partial result and its merging, about as much as that many tiles.
static constexpr int WHOLE_SLACK = 8, MERGE_B = 256;
__device__ __forceinline__ bool units_whole(const Paged8Params& p, long long upu, int longest, long long T) {
  return p.B * upu <= p.grid && (long long)(longest - WHOLE_SLACK) * p.grid <= T;
}
template <int THREADS>
__device__ __forceinline__ void paged8_range(const Paged8Params& p, int id, long long* s_warp, int* s_b, long long* s_off) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long upu = (long long)p.Hkv * p.n_blk;
  const int q = (p.B + THREADS - 1) / THREADS, lo = min(tid * q, p.B), hi = min(lo + q, p.B);
  long long sum = 0;
  int longest = 0, n_only = 0;                               // n_only: tiles of the thread's only sequence (q = 1)
#pragma unroll 1
  for (int b = lo; b < hi; ++b) { n_only = tile_span(p, b).n; sum += n_only * upu; longest = max(longest, n_only); }
  long long inc = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const long long y = __shfl_up_sync(0xffffffffu, inc, o); if (lane >= o) inc += y; }
  longest = __reduce_max_sync(0xffffffffu, longest);
  int* s_longest = reinterpret_cast<int*>(s_warp + THREADS / 32);
  if (lane == 31) { s_warp[warp] = inc; s_longest[warp] = longest; }
  __syncthreads();
  long long T = 0, before = inc - sum;
  longest = 0;
#pragma unroll 1
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < warp) before += s_warp[w];
    T += s_warp[w];
    longest = max(longest, s_longest[w]);
  }
  const bool own = units_whole(p, upu, longest, T);
  if (blockIdx.x == 0 && p.B > MERGE_B) {
    long long at = before;
#pragma unroll 1
    for (int b = lo; b < hi; ++b) { p.prefix[b] = at; at += (q == 1 ? n_only : tile_span(p, b).n) * upu; }
    if (tid == 0) { p.prefix[p.B] = T; p.prefix[p.B + 1] = own; }
  }
  if (own) {
    if (tid == 0) {
      const int b = min(id / (int)upu, p.B - 1), n = id < p.B * upu ? tile_span(p, b).n : 0;
      *s_b = b; s_off[0] = (long long)(id % (int)upu) * n; s_off[1] = n;
    }
    return;
  }
  const Cut cut(T, p.grid);
  const long long s0 = id < cut.G ? cut.start(id) : 0, s1 = id < cut.G ? cut.start(id + 1) : 0;
  if (s1 > s0 && s0 >= before && s0 < before + sum) {        // exactly one thread
    long long at = before;
    int b = lo;
#pragma unroll 1
    while (q > 1) {
      const long long n = tile_span(p, b).n * upu;
      if (s0 < at + n) break;
      at += n; ++b;
    }
    *s_b = b; s_off[0] = s0 - at; s_off[1] = s1 - s0;
  }
  if (tid == 0 && s1 <= s0) { *s_b = 0; s_off[0] = 0; s_off[1] = 0; }
}

// Splits the 8 bf16 values of `v` times f into two e4m3 terms.  By way of f16, which holds the products (below 2^8, eight
// significant bits, nothing lost above 2^-24), the first term and what it leaves exactly.
__device__ __forceinline__ void split_e4m3(const uint4& v, float f, uint32_t (&hi)[2], uint32_t (&lo)[2]) {
  const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    uint32_t h = 0, l = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t w = x[2 * k + i];
      const __half2 a = __floats2half2_rn(__uint_as_float(w << 16) * f, __uint_as_float(w & 0xffff0000u) * f);
      const uint32_t hc = e4m3x2_from_half2(a), lc = e4m3x2_from_half2(__hsub2(a, half2_from_e4m3x2(hc)));
      h |= hc << (16 * i); l |= lc << (16 * i);
    }
    hi[k] = h; lo[k] = l;
  }
}
__device__ __forceinline__ uint32_t max_abs_bf16(const uint4& v) {
  uint32_t top = 0;
  const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) top = max(top, max(x[k] & 0x7fffu, (x[k] >> 16) & 0x7fffu));
  return top;
}
// Exponent that brings a row whose largest |element| has these bf16 bits into [128, 256).
__device__ __forceinline__ int query_exponent(uint32_t bits) { return min(max(134 - (int)(bits >> 7), -119), 120); }

__device__ __forceinline__ void umma_f8_elected(uint32_t leader, uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                                uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(leader) : "memory");
}
// kind::f8f6f4, fp32 accumulator, A e4m3, B e4m3 (0) or e5m2 (1)
__host__ __device__ constexpr uint32_t umma_idesc_f8(int M, int N, int b_format, bool a_mn_major, bool b_mn_major) {
  return (1u << 4) | ((uint32_t)b_format << 10) | ((a_mn_major ? 1u : 0u) << 15) | ((b_mn_major ? 1u : 0u) << 16) |
         ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// Shared-memory descriptor for rows of `width` bytes with the swizzle of that width (16: none).  K-major: 8 rows (one
// group) are 8 * width bytes apart.  MN-major: the same picture with the rows along K.  `lbo`: distance of the next block
// of `width` bytes along the contiguous dimension (only used where the operand is wider than one block).
__device__ __forceinline__ uint64_t desc_rows(uint32_t addr, int width, uint32_t lbo) {
  const uint64_t layout = width == 128 ? 2 : width == 64 ? 4 : width == 32 ? 6 : 0;
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)((lbo >> 4) & 0x3FFFu) << 16) |
         ((uint64_t)(((uint32_t)width * 8 >> 4) & 0x3FFFu) << 32) | (1ull << 46) | (layout << 61);
}
// Byte offset of 16-byte unit `u` of row `r` in such an image.
template <int WIDTH>
__device__ __forceinline__ uint32_t swz(int r, int u) {
  if (WIDTH == 128) return (uint32_t)(r * 128 + ((u ^ (r & 7)) << 4));
  if (WIDTH == 64) return (uint32_t)(r * 64 + ((u ^ ((r >> 1) & 3)) << 4));
  if (WIDTH == 32) return (uint32_t)(r * 32 + ((u ^ ((r >> 2) & 1)) << 4));
  return (uint32_t)(r * 16);
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ float warp_max_f32(float v) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ uint64_t mul_f32x2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t join(uint32_t lo, uint32_t hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
  return r;
}
__device__ __forceinline__ float ex2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float lg2(float x) { float r; asm("lg2.approx.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
// Merges the pieces of the units that were cut, in the order of their tiles, and writes the rows of sequences that have
// no tile at all.  One warp: 32 * VEC outputs of one row; lane i holds the maximum and the sum of piece i, so that their loads
// and the loads of the pieces' outputs are two round trips, not one per piece (64 x 5056 rows, 128 heads: 128 us for the call
// instead of 135).  Its CTAs are in place before the attention kernel ends and know by then what they have to merge: for
// up to MERGE_B sequences they sum the tiles themselves, from counters that the attention kernel has waited for already.
template <int DS, int NH, int VEC>
__global__ void __launch_bounds__(256) paged8_combine_kernel(const __grid_constant__ Paged8Params p) {
  constexpr int SPLIT = NH * DS / (256 * VEC);
  __shared__ int s_sum[3][8], s_n;
  const int lane = threadIdx.x & 31;
  const long long unit = blockIdx.x / SPLIT;
  const int x = ((int)(blockIdx.x % SPLIT) * 256 + (int)threadIdx.x) * VEC, h = x / DS, d = x % DS;      // h: one per warp
  const int per = p.Hkv * p.n_blk, b = (int)(unit / per), u = (int)(unit % per), hk = u / p.n_blk, blk = u % p.n_blk;
  const int gr = blk * NH + h;
  long long T = 0, seq = 0, n = 0;
  bool own = false;
  if (p.B <= MERGE_B) {                                      // thread i: sequence i
    const int i = threadIdx.x, tiles = i < p.B ? tile_span(p, i).n : 0;
    const int all = __reduce_add_sync(0xffffffffu, tiles), before = __reduce_add_sync(0xffffffffu, i < b ? tiles : 0);
    const int longest = __reduce_max_sync(0xffffffffu, tiles);
    if (lane == 0) { s_sum[0][i >> 5] = all; s_sum[1][i >> 5] = before; s_sum[2][i >> 5] = longest; }
    if (i == b) s_n = tiles;
    __syncthreads();
    int most = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) { T += s_sum[0][k]; seq += s_sum[1][k]; most = max(most, s_sum[2][k]); }
    T *= per; seq *= per; n = s_n;
    own = units_whole(p, per, most, T);
  }
  chain_wait();
  chain_next();
  if (gr >= p.q_len * p.rep) return;
  if (p.B > MERGE_B) {
    T = p.prefix[p.B]; seq = p.prefix[b]; own = p.prefix[p.B + 1];
    const long long n_all = p.prefix[b + 1] - seq;
    n = n_all >> 32 ? n_all / per : (unsigned)n_all / (unsigned)per;
  }
  const size_t row = ((size_t)b * p.q_len + gr / p.rep) * p.Hq + (size_t)hk * p.rep + gr % p.rep;
  float o[VEC] = {};
  float m = -INFINITY, l = 0.f;
  if (n > 0) {
    if (own) return;                                         // not cut: written by the CTA that worked on it
    const Cut cut(T, p.grid);
    const long long u0 = seq + u * n, u1 = u0 + n;
    const int c0 = cut.owner(u0), np = cut.owner(u1 - 1) - c0 + 1;
    if (np == 1) return;
    const float* ml = p.part + (size_t)2 * p.grid * NH * DS;
    const int first = cut.start(c0) == u0 ? 0 : 1;           // the CTA's first piece, or a later one
    for (int i = lane; i < np; i += 32) m = fmaxf(m, ml[(size_t)(2 * (c0 + i) + (i == 0 ? first : 0)) * 2 * NH + h]);
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, k));
    for (int i0 = 0; i0 < np; i0 += 32) {
      const int i = i0 + lane;
      float f = 0.f, lj = 0.f;
      if (i < np) {
        const float* q = ml + (size_t)(2 * (c0 + i) + (i == 0 ? first : 0)) * 2 * NH + h;
        lj = q[NH];
        // applied twice: M contains the scales, the square may be below fp32.  A piece without a seen key has no weight
        f = lj == 0.f ? 0.f : exp2f(0.5f * (q[0] - m));
      }
      l += warp_sum(f * lj * f);
      const int cnt = min(np - i0, 32);
#pragma unroll 8
      for (int k = 0; k < cnt; ++k) {
        const float w = __shfl_sync(0xffffffffu, f, k);
        const float* src = p.part + (size_t)(2 * (c0 + i0 + k) + (i0 + k == 0 ? first : 0)) * NH * DS + x;
        float v[VEC];
        if constexpr (VEC == 4) *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(src);
        else if constexpr (VEC == 2) *reinterpret_cast<float2*>(v) = *reinterpret_cast<const float2*>(src);
        else v[0] = *src;
#pragma unroll
        for (int e = 0; e < VEC; ++e) o[e] = w == 0.f ? o[e] : fmaf(w * v[e], w, o[e]);        // without weight: may be 0 * NaN
      }
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if constexpr (VEC == 1) p.out[row * DS + d] = __float2bfloat16_rn(o[0] * inv);
  else {
    uint32_t* dst = reinterpret_cast<uint32_t*>(p.out + row * DS + d);
#pragma unroll
    for (int k = 0; k < VEC / 2; ++k) dst[k] = pack_bf16x2(o[2 * k] * inv, o[2 * k + 1] * inv);
  }
  if (p.lse && d == 0) p.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l) - paged8_t_bits(NH)) * 0.6931471805599453f;
}

// Where VEC outputs a thread would fill less than one CTA an SM, a thread takes one: more warps have their pieces' loads under way, and the
// sums are the same.  The whole call over the 4-bit cache, 1 x 9000 / 1 x 30000 rows: MLA 128 heads 37 / 58 us with 4, 31 / 43 with 1;
// 16 heads and 4 tokens 34 / 54 and 29 / 39; 64 x 5056 rows (many CTAs): 126 with 4, 136 with 2.
template <int DS, int NH>
int paged8_combine_launch(const Paged8Params& P, cudaStream_t stream) {
  constexpr int VEC = DS >= 128 ? 4 : 2, FEW = 1;
  const long long units = (long long)P.B * P.Hkv * P.n_blk, ctas = units * (NH * DS / (256 * VEC));
  if (ctas <= 148) return launch_chained(paged8_combine_kernel<DS, NH, FEW>, (unsigned)(units * (NH * DS / (256 * FEW))), 256, 0, stream, 1, P);
  return launch_chained(paged8_combine_kernel<DS, NH, VEC>, (unsigned)ctas, 256, 0, stream, 1, P);
}

int attn_paged8_pair_launch(Paged8Params& P, cudaStream_t stream);      // MLA shape, blocks of 128 rows on CTA pairs
int attn_paged8_pair_take_status();

}  // namespace lca
