// Decode attention over the paged 4-bit cache for GQA with up to eight query rows a KV head (one token of a usual head layout).
//
// The mathematics is that of attn_paged4.cu: rows expanded exactly to e4m3, two-term queries and weights, a running maximum that is
// raised lazily.  With so few rows the cost is the expansion itself (seven integer instructions for eight values, on a pipe that takes
// two a clock per SM), so everything around it has to go: no expanded image in shared memory, no hand-over between warps, no barrier.
// Each warp works on 32 keys at a time by itself, with the operands of its products in registers:
//   S = K Q^T     m16n8k32, rows = keys.  Lane (g, t) = (lane / 4, lane % 4) expands its quarter (t) of the rows g and g + 8; which column is
//                 which k does not matter as long as the queries follow, so the quarter is what lies together in the page.
//                 Columns are (row, term) of the queries: a lane gets both terms' sums of one row in neighbouring registers.
//   O^T = V^T T   m16n8k32, rows = columns of V, k = keys.  A lane takes an eighth (g) of the rows 2 t + h + 8 j, h < 2, j < 4, and transposes
//                 4 x 4 bytes; in that order of the keys the weights it needs for B are two words that one other lane has packed.
// tcgen05 needs the expanded rows in shared memory, written by other warps than those that wait for the products: 64 x 5056 rows, 32 heads
// on 8 of 128, took 130 us that way and FIGURE us here.  What bounds it now: FIGURE.
#include "attn_paged4.cuh"

namespace lca {
using namespace tc;

static constexpr int FEW_THREADS = 256, FEW_WARPS = 8;

__device__ __forceinline__ void mma_e4m3(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// N words that are read once
template <int N>
__device__ __forceinline__ void load_words(uint32_t (&v)[N], const uint8_t* p) {
  if constexpr (N == 4) asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "l"(p));
  else if constexpr (N == 2) asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(v[0]), "=r"(v[1]) : "l"(p));
  else asm volatile("ld.global.nc.L1::no_allocate.u32 %0, [%1];" : "=r"(v[0]) : "l"(p));
}
// v[k] = byte k of (x0, x1, x2, x3)
__device__ __forceinline__ void transpose4(uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3, uint32_t (&v)[4]) {
  const uint32_t p = __byte_perm(x0, x1, 0x5140), q = __byte_perm(x2, x3, 0x5140);        // bytes 0 and 1 of both
  const uint32_t r = __byte_perm(x0, x1, 0x7362), s = __byte_perm(x2, x3, 0x7362);
  v[0] = __byte_perm(p, q, 0x5410); v[1] = __byte_perm(p, q, 0x7632);
  v[2] = __byte_perm(r, s, 0x5410); v[3] = __byte_perm(r, s, 0x7632);
}

template <int D, int NT>
__global__ void __launch_bounds__(FEW_THREADS, 2) attn_paged4_few_kernel(const __grid_constant__ Paged4Params a) {
  constexpr int WK = D / 32, WV = D / 64, EV = 2 * WV, MT = D / 16, ROWS = 4 * NT, NH = 16;      // NH: row count of the partial results' layout
  const Paged8Params& p = a.b;
  // facts of a warp's keys
  __shared__ float4 s_fa[FEW_WARPS][32];                     // logit factor, bias + half, half, f_t
  __shared__ float2 s_fb[FEW_WARPS][32];                     // rounding offset, f_l
  __shared__ uint32_t s_sh[FEW_WARPS][32];                   // shifts: K, V in the upper half
  __shared__ uint2 s_table[16];
  __shared__ __align__(16) float s_o[FEW_WARPS][ROWS][D];
  __shared__ float s_ml[FEW_WARPS][ROWS][2];
  __shared__ long long s_warp[2 * FEW_WARPS], s_off[2];
  __shared__ int s_b;
  __shared__ Walk s_walk;                                    // thread 0 moves it on; the piece that all work on
  __shared__ int s_more;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), g = lane >> 2, t = lane & 3;
  paged4_table_load(s_table, tid);
  chain_wait();
  chain_next();
  paged8_range<FEW_THREADS>(p, (int)blockIdx.x, s_warp, &s_b, s_off);
  __syncthreads();
  const int mask = p.page - 1, n_rows = p.q_len * p.rep;
  uint32_t seg = 0;
#pragma unroll 1
  for (;; ++seg) {
    if (tid == 0) {
      Walk x;
      if (seg == 0) { x.b = s_b; x.off = s_off[0]; x.left = s_off[1]; x.fresh = true; x.n = 0; }
      else x = s_walk;
      s_more = x.next(p);
      s_walk = x;
    }
    __syncthreads();
    if (!s_more) break;
    const volatile Walk& w = s_walk;
    const int n_tok = w.t.s.n_tok, n_rep = w.t.s.n_rep, tok0 = w.t.s.tok0, subs = 4 * w.n, hk = w.hk;
    const PagedSpan sp = {n_rep, tok0, n_tok};
    const int32_t* table = p.table + (size_t)w.b * p.width;
    const int tile0 = w.t0, n_a = w.t.n_a, skip = w.t.b0 - w.t.n_a;
    auto row_of = [&](int s) { const int i = tile0 + (s >> 2); return (i < n_a ? i : i + skip) * 128 + 32 * (s & 3); };        // first row of 32 keys
    // The pool's 16-row groups that the two halves of 32 keys are, ~0: no such page.  (A group takes 512 bytes at least, 32 bits
    // count those of more memory than there is.)
    struct Base { uint32_t r[2]; };
    struct Pages { int pg[2]; };
    auto look = [&](int s) {
      Pages y;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        y.pg[i] = -1;
        if (s < subs) {
          const int x = row_of(s) + 16 * i;
          if (sp.any(x, 16) && (x >> p.page_log2) < p.width) y.pg[i] = table[x >> p.page_log2];
        }
      }
      return y;
    };
    auto base_of = [&](const Pages& y, int s) {
      Base z;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        z.r[i] = (unsigned)y.pg[i] < (unsigned)p.n_pages
                     ? (((uint32_t)y.pg[i] * (uint32_t)p.Hkv + (uint32_t)hk) << (p.page_log2 - 4)) + (uint32_t)(((row_of(s) + 16 * i) & mask) >> 4) : ~0u;
      return z;
    };
    uint32_t kd[4][WK], vd[8][WV];                           // keys g + 8 m; values 2 t + h + 8 j at [4 h + j]
    uint32_t raw_sh = 0, raw_e = 0;                          // shifts and exponents of key `lane`
    auto load_k = [&](const Base& z) {
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        if (z.r[m >> 1] != ~0u) load_words<WK>(kd[m], a.pos + (size_t)z.r[m >> 1] * (8 * D) + (g + 8 * (m & 1)) * (D / 2) + t * (D / 8));
        else
#pragma unroll
          for (int k = 0; k < WK; ++k) kd[m][k] = 0u;
      }
    };
    auto load_v = [&](const Base& z) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (z.r[j >> 1] != ~0u) load_words<WV>(vd[4 * h + j], a.sem + (size_t)z.r[j >> 1] * (8 * D) + (2 * t + h + 8 * (j & 1)) * (D / 2) + g * (D / 16));
          else
#pragma unroll
            for (int k = 0; k < WV; ++k) vd[4 * h + j][k] = 0u;
        }
    };
    auto load_facts = [&](const Base& z, int s) {
      const uint32_t r = lane < 16 ? z.r[0] : z.r[1];
      raw_sh = 0; raw_e = 0x10000u;                          // bit 16: absent
      if (r != ~0u && sp.has(row_of(s) + lane)) {
        const size_t y = (size_t)r * 16 + (lane & 15);
        if constexpr (D == 128)
          raw_sh = (uint32_t)reinterpret_cast<const uint16_t*>(a.shift_pos)[y] | (uint32_t)reinterpret_cast<const uint16_t*>(a.shift_sem)[y] << 16;
        else raw_sh = (uint32_t)a.shift_pos[y] | (uint32_t)a.shift_sem[y] << 16;
        raw_e = (uint32_t)a.exp_k[y] | (uint32_t)a.exp_v[y] << 8;
      }
    };
    Pages nx = look(warp);
    if (warp < subs) { const Base z = base_of(nx, warp); load_k(z); load_facts(z, warp); load_v(z); }
    nx = look(warp + FEW_WARPS);
    // queries: column g of tile n is (row 4 n + g / 2, term g % 2), this lane's quarter of it
    uint32_t qd[NT][2 * WK];
    float qs[NT], m_run[NT], l[NT];
    int lim[NT], out_row[NT];
    bool unset[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      auto row_at = [&](int r) { const int qt = r / p.rep; return ((int)(w.b * p.q_len) + qt) * p.Hq + hk * p.rep + (r - qt * p.rep); };
      const int r = 4 * n + (g >> 1);
      uint4 v[D / 32];
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        v[i] = r < n_rows ? *reinterpret_cast<const uint4*>(p.q_pos + (size_t)row_at(r) * D + t * (D / 4) + 8 * i) : make_uint4(0u, 0u, 0u, 0u);
        top = max(top, max_abs_bf16(v[i]));
      }
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const int e = query_exponent(top);
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        uint32_t hi[2], lo[2];
        split_e4m3(v[i], exp2_int(e), hi, lo);
        qd[n][2 * i] = (g & 1) ? lo[0] : hi[0]; qd[n][2 * i + 1] = (g & 1) ? lo[1] : hi[1];
      }
      // a row with an infinity or a NaN has no finite logit; rows behind the last one never have weight
      const float back = r < n_rows ? (top >= 0x7f80u ? __int_as_float(0x7fffffff) : exp2_int(-e)) : 0.f;
      qs[n] = __shfl_sync(0xffffffffu, back, 8 * t);         // of row 4 n + t
      const int mine = 4 * n + t;
      unset[n] = mine < n_rows;
      m_run[n] = mine < n_rows ? 0.f : 3.0e38f;
      l[n] = 0.f;
      lim[n] = sp.n_tok - p.q_len + 1 + mine / p.rep;
      out_row[n] = mine < n_rows ? row_at(mine) : -1;
    }
    float acc[NT][MT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[n][i][k] = 0.f;

#pragma unroll 1
    for (int s = warp; s < subs; s += FEW_WARPS) {
      const int x0 = row_of(s);
      const bool more = s + FEW_WARPS < subs;
      const Base z1 = base_of(nx, s + FEW_WARPS);
      nx = look(s + 2 * FEW_WARPS);
      // ---- facts of key `lane`, for all lanes
      {
        const int ek = (int)(raw_e & 0xffu), ev = (int)((raw_e >> 8) & 0xffu), x = x0 + lane;
        // The row sum needs 2^(y - M), the weight t = 2^(y - M + log2 f_v + T): both are multiples of 2^(y - M + half), half way
        // between them, so that neither is lost below 2^-126 where the factors of a sequence span more than fp32 does.
        const float half = 0.5f * ((float)paged4_log2_factor(ev) + paged8_t_bits(NH));
        __syncwarp();                                        // the facts of the keys before have been read
        s_fa[warp][lane] = make_float4(paged4_factor(ek) * p.scale_log2, (raw_e >> 16) ? -INFINITY : half + (x < sp.n_rep ? p.bias_log2 : 0.f), half, ex2(half));
        s_fb[warp][lane] = make_float2(weight_offset(x), ex2(paged8_t_bits(NH) - half));
        s_sh[warp][lane] = raw_sh;
        __syncwarp();
        if (more) load_facts(z1, s + FEW_WARPS);
      }
      // ---- S
      float sc[2][NT][4];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int k = 0; k < 4; ++k) sc[u][n][k] = 0.f;
        const int block = D == 128 ? t : t >> 1;
        const uint2 t0 = s_table[(s_sh[warp][16 * u + g] >> (4 * block)) & 15], t1 = s_table[(s_sh[warp][16 * u + 8 + g] >> (4 * block)) & 15];
#pragma unroll
        for (int k = 0; k < WK; ++k) {
          const uint2 e0 = paged4_expand(kd[2 * u][k], t0), e1 = paged4_expand(kd[2 * u + 1][k], t1);
#pragma unroll
          for (int n = 0; n < NT; ++n) mma_e4m3(sc[u][n], e0.x, e1.x, e0.y, e1.y, qd[n][2 * k], qd[n][2 * k + 1]);
        }
      }
      if (more) load_k(z1);
      // ---- weights: keys g + 8 m of rows t, 4 + t
      float4 fa[4];
      float2 fb[4];
#pragma unroll
      for (int m = 0; m < 4; ++m) { fa[m] = s_fa[warp][g + 8 * m]; fb[m] = s_fb[warp][g + 8 * m]; }
      float zz[NT][4];
      bool over = false;
      const bool limited = x0 + 31 >= sp.n_tok - p.q_len + 1;      // some query may not see some of these rows
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          zz[n][m] = fmaf(sc[m >> 1][n][2 * (m & 1)] + sc[m >> 1][n][2 * (m & 1) + 1], fa[m].x * qs[n], fa[m].y - m_run[n]);
          if (limited && x0 + g + 8 * m >= lim[n]) zz[n][m] = -INFINITY;
          over = over || zz[n][m] + fa[m].z > T4_MAX;
        }
        over = over || unset[n];
      }
      if (__any_sync(0xffffffffu, over)) {
        // raise the maxima: per row the largest log2 t of these keys
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float m = fmaxf(fmaxf(zz[n][0] + fa[0].z, zz[n][1] + fa[1].z), fmaxf(zz[n][2] + fa[2].z, zz[n][3] + fa[3].z));
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
          if (unset[n] ? m > -INFINITY : m > paged8_t_bits(NH)) {
            const float d = m - paged8_t_bits(NH), f = unset[n] ? 1.f : ex2(-d);       // nothing has been added under an unset maximum
            m_run[n] += d;
            unset[n] = false;
            l[n] *= f;
#pragma unroll
            for (int k = 0; k < 4; ++k) zz[n][k] -= d;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
              for (int k = 0; k < 4; ++k) acc[n][i][k] *= f;
          }
        }
      }
      uint32_t b0[NT], b1[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float tt[4], sum = 0.f;
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const float e = ex2(zz[n][m]);
          tt[m] = e * fa[m].w;
          sum = fmaf(e, fb[m].y, sum);
        }
        l[n] += sum;
        const uint32_t hi = e4m3x4_from_float(tt[0], tt[1], tt[2], tt[3]);
        const float4 h = e4m3x4_to_float4(hi);               // what the first term leaves is exact: at most 2^4, times the gain 2^8
        const uint32_t lo = e4m3x4_from_float(fmaf(tt[0] - h.x, LO4_GAIN, fb[0].x), fmaf(tt[1] - h.y, LO4_GAIN, fb[1].x),
                                              fmaf(tt[2] - h.z, LO4_GAIN, fb[2].x), fmaf(tt[3] - h.w, LO4_GAIN, fb[3].x));
        // column g = (row g / 2, term g % 2), keys 2 t + 8 j and 2 t + 1 + 8 j: of lanes (2 t, g / 2) and (2 t + 1, g / 2)
        const int from = 8 * t + (g >> 1);
        const uint32_t h0 = __shfl_sync(0xffffffffu, hi, from), h1 = __shfl_sync(0xffffffffu, hi, from + 4);
        const uint32_t l0 = __shfl_sync(0xffffffffu, lo, from), l1 = __shfl_sync(0xffffffffu, lo, from + 4);
        b0[n] = (g & 1) ? l0 : h0; b1[n] = (g & 1) ? l1 : h1;
      }
      // ---- O
      {
        uint32_t ex[8][EV];
        const int block = 16 + 4 * (D == 128 ? g >> 1 : g >> 2);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint2 sh = *reinterpret_cast<const uint2*>(&s_sh[warp][2 * t + 8 * j]);
          const uint2 ta = s_table[(sh.x >> block) & 15], tb = s_table[(sh.y >> block) & 15];
#pragma unroll
          for (int k = 0; k < WV; ++k) {
            const uint2 ea = paged4_expand(vd[j][k], ta), eb = paged4_expand(vd[4 + j][k], tb);
            ex[j][2 * k] = ea.x; ex[j][2 * k + 1] = ea.y; ex[4 + j][2 * k] = eb.x; ex[4 + j][2 * k + 1] = eb.y;
          }
        }
        if (more) load_v(z1);
#pragma unroll
        for (int q = 0; q < EV / 2; ++q) {
          uint32_t a0[4], a1[4], a2[4], a3[4];
          transpose4(ex[0][q], ex[1][q], ex[2][q], ex[3][q], a0);
          transpose4(ex[0][EV / 2 + q], ex[1][EV / 2 + q], ex[2][EV / 2 + q], ex[3][EV / 2 + q], a1);
          transpose4(ex[4][q], ex[5][q], ex[6][q], ex[7][q], a2);
          transpose4(ex[4][EV / 2 + q], ex[5][EV / 2 + q], ex[6][EV / 2 + q], ex[7][EV / 2 + q], a3);
#pragma unroll
          for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_e4m3(acc[n][4 * q + b], a0[b], a1[b], a2[b], a3[b], b0[n], b1[n]);
        }
      }
    }
    // ---- the warps' results together: this lane has columns [D / 8 g, D / 8 (g + 1)) of rows t, 4 + t
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) l[n] += __shfl_xor_sync(0xffffffffu, l[n], o);
      if (g == 0) { s_ml[warp][4 * n + t][0] = unset[n] ? -INFINITY : m_run[n]; s_ml[warp][4 * n + t][1] = l[n]; }
      float* dst = &s_o[warp][4 * n + t][g * (D / 8)];
#pragma unroll
      for (int i = 0; i < MT; i += 4) {
        float x[4], y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          x[k] = fmaf(acc[n][i + k][1], 1.f / LO4_GAIN, acc[n][i + k][0]);
          y[k] = fmaf(acc[n][i + k][3], 1.f / LO4_GAIN, acc[n][i + k][2]);
        }
        *reinterpret_cast<float4*>(dst + i) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4*>(dst + MT + i) = make_float4(y[0], y[1], y[2], y[3]);
      }
    }
    __syncthreads();
    const bool whole = w.n == w.t.n;
    const size_t part = (size_t)2 * blockIdx.x + (seg == 0 ? 0 : 1);
#pragma unroll 1
    for (int i = tid; i < min(n_rows, ROWS) * D; i += FEW_THREADS) {
      const int r = i / D, d = i % D;
      float m = -INFINITY, sum = 0.f, o = 0.f;
#pragma unroll
      for (int k = 0; k < FEW_WARPS; ++k) m = fmaxf(m, s_ml[k][r][0]);
#pragma unroll
      for (int k = 0; k < FEW_WARPS; ++k) {
        const float lk = s_ml[k][r][1];
        if (lk == 0.f) continue;                             // no key with weight: o may be 0 * NaN
        const float f = ex2(0.5f * (s_ml[k][r][0] - m));     // applied twice: M contains the factors, the square may be below fp32
        sum += f * lk * f;
        o = fmaf(f * s_o[k][r][d], f, o);
      }
      if (whole) {
        const int qt = r / p.rep;
        const size_t row = ((size_t)w.b * p.q_len + qt) * p.Hq + (size_t)hk * p.rep + (r - qt * p.rep);
        p.out[row * D + d] = __float2bfloat16_rn(sum == 0.f ? 0.f : o / sum);
        if (p.lse && d == 0) p.lse[row] = sum == 0.f ? -INFINITY : (m + log2f(sum) - paged8_t_bits(NH)) * 0.6931471805599453f;
      } else {
        p.part[part * NH * D + (size_t)r * D + d] = o;
        if (d == 0) {
          float* ml = p.part + (size_t)2 * p.grid * NH * D + part * 2 * NH;
          ml[r] = m; ml[NH + r] = sum;
        }
      }
    }
    __syncthreads();
  }
}

template <int D, int NT>
static int few_launch(Paged4Params& P, cudaStream_t stream) {
  const int st = launch_chained(attn_paged4_few_kernel<D, NT>, (unsigned)P.b.grid, FEW_THREADS, 0, stream, 1, P);
  return st != LCA_OK ? st : paged8_combine_launch<D, 16>(P.b, stream);
}
int attn_paged4_few_launch(const lca_params* p, Paged4Params& P, cudaStream_t stream) {
  const bool four = (long long)P.b.q_len * P.b.rep <= 4;
  if (p->d_sem == 128) return four ? few_launch<128, 1>(P, stream) : few_launch<128, 2>(P, stream);
  return four ? few_launch<64, 1>(P, stream) : few_launch<64, 2>(P, stream);
}

}  // namespace lca
