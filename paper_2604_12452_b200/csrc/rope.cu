// Rotary positions: y = factor R(+-p f) x for pairs of columns of queries and keys, in the layouts that projections leave them in.
//
// A pair (a, b) becomes (a cos - b sin, a sin + b cos) of the angle p f_i.  The angle of a far position does not fit 32 bits (position
// 10^6 times a frequency of 1, rounded to fp32, is off by 0.03), so the product and its whole turns are taken in 64 bits and only the
// rest of less than half a turn goes on in 32, where sincospi is off by an ulp or two.  That is 64-bit work for each (token, pair), not
// for each head: a CTA computes the cosines and sines of its tokens once, in shared memory, and applies them to all the heads
// that it takes.  HBM-bound: 2 bytes in and 2 out per element; 32768 tokens x 40 heads of 128 columns 116 us, 5.8 TB/s.
#include <type_traits>

#include "lca_common.cuh"
#include "tc_common.cuh"

namespace lca {

struct RopePart { const void* x; void* y; long long x_token, x_head, y_token, y_head; int heads; };
struct RopeKernelArgs {
  RopePart part[2];          // queries, keys
  const int32_t* positions; const double* freqs;
  long long n_tokens;
  int d, rot, tokens, heads; // tokens of a CTA; heads (of both parts) of a CTA
  float factor, sign;
};

static const int ROPE_THREADS = 256, ROPE_TABLE = 4096;      // (token, pair)s that a CTA has room for

template <class T> struct Vec8 { uint4 v[sizeof(T) / 2]; };
template <class T>
__device__ __forceinline__ void unpack_vec(const Vec8<T>& v, float (&f)[8]) {
  if constexpr (sizeof(T) == 2) {
    const uint32_t u[4] = {v.v[0].x, v.v[0].y, v.v[0].z, v.v[0].w};
#pragma unroll
    for (int k = 0; k < 4; ++k) { f[2 * k] = __uint_as_float(u[k] << 16); f[2 * k + 1] = __uint_as_float(u[k] & 0xffff0000u); }
  } else {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      f[4 * k] = __uint_as_float(v.v[k].x); f[4 * k + 1] = __uint_as_float(v.v[k].y);
      f[4 * k + 2] = __uint_as_float(v.v[k].z); f[4 * k + 3] = __uint_as_float(v.v[k].w);
    }
  }
}
template <class T>
__device__ __forceinline__ Vec8<T> pack_vec(const float (&f)[8]) {
  Vec8<T> v;
  if constexpr (sizeof(T) == 2) v.v[0] = make_uint4(tc::pack_bf16x2(f[0], f[1]), tc::pack_bf16x2(f[2], f[3]), tc::pack_bf16x2(f[4], f[5]), tc::pack_bf16x2(f[6], f[7]));
  else
#pragma unroll
    for (int k = 0; k < 2; ++k)
      v.v[k] = make_uint4(__float_as_uint(f[4 * k]), __float_as_uint(f[4 * k + 1]), __float_as_uint(f[4 * k + 2]), __float_as_uint(f[4 * k + 3]));
  return v;
}
template <class T>
__device__ __forceinline__ Vec8<T> load_vec(const T* p) {
  Vec8<T> v;
#pragma unroll
  for (int k = 0; k < (int)sizeof(T) / 2; ++k) v.v[k] = reinterpret_cast<const uint4*>(p)[k];
  return v;
}
template <class T>
__device__ __forceinline__ void store_vec(T* p, const Vec8<T>& v) {
#pragma unroll
  for (int k = 0; k < (int)sizeof(T) / 2; ++k) reinterpret_cast<uint4*>(p)[k] = v.v[k];
}
__device__ __forceinline__ void turn(float& a, float& b, const float2& cs) {
  const float x = a, y = b;
  a = x * cs.x - y * cs.y;
  b = x * cs.y + y * cs.x;
}
template <class T> __device__ __forceinline__ float to_f(T v) { if constexpr (sizeof(T) == 2) return __bfloat162float(v); else return v; }
template <class T> __device__ __forceinline__ T from_f(float v) { if constexpr (sizeof(T) == 2) return __float2bfloat16_rn(v); else return v; }

// VEC: eight neighbouring columns at a time (rows 16-byte aligned, rot a multiple of 16, d of 8); otherwise a pair, or a column
// behind the rotated ones (the same 32768 tokens: 354 us).
template <class T, bool INTERLEAVED, bool VEC>
__global__ void __launch_bounds__(ROPE_THREADS) rope_kernel(const __grid_constant__ RopeKernelArgs a) {
  __shared__ float2 s_cs[ROPE_TABLE];
  const long long t0 = (long long)blockIdx.x * a.tokens;
  const int n_tok = (int)min((long long)a.tokens, a.n_tokens - t0), pairs = a.rot / 2;
  chain_wait();
  chain_next();
  for (int i = threadIdx.x; i < n_tok * pairs; i += ROPE_THREADS) {
    const int t = i / pairs, k = i - t * pairs;
    const double turns = (double)a.positions[t0 + t] * a.freqs[k] * 0.15915494309189533577;           // 1 / (2 pi)
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    s_cs[i] = make_float2(c * a.factor, s * a.factor * a.sign);
  }
  __syncthreads();
  // units of a head: VEC half layout: two vectors that face one another, then single ones; interleaved: vectors; otherwise pairs,
  // then columns
  const int rot_units = VEC ? (INTERLEAVED ? a.rot / 8 : a.rot / 16) : pairs;
  const int units = rot_units + (VEC ? (a.d - a.rot) / 8 : a.d - a.rot);
  const int h0 = (int)blockIdx.y * a.heads, n_heads = min(a.heads, a.part[0].heads + a.part[1].heads - h0);
  const unsigned total = (unsigned)n_tok * n_heads * units;
#pragma unroll 4
  for (unsigned x = threadIdx.x; x < total; x += ROPE_THREADS) {
    const unsigned th = x / (unsigned)units, t = th / (unsigned)n_heads;
    const int u = (int)(x - th * units);
    int h = h0 + (int)(th - t * n_heads);
    const bool key = h >= a.part[0].heads;
    const RopePart& q = a.part[key];
    if (key) h -= a.part[0].heads;
    const T* src = (const T*)q.x + (t0 + t) * q.x_token + h * q.x_head;
    T* dst = (T*)q.y + (t0 + t) * q.y_token + h * q.y_head;
    const float2* cs = s_cs + t * pairs;
    if constexpr (VEC) {
      if (u >= rot_units) {                                  // behind the rotated columns
        const int c = a.rot + 8 * (u - rot_units);
        if (src != dst) store_vec<T>(dst + c, load_vec<T>(src + c));
      } else if constexpr (INTERLEAVED) {
        float f[8];
        unpack_vec<T>(load_vec<T>(src + 8 * u), f);
#pragma unroll
        for (int k = 0; k < 4; ++k) turn(f[2 * k], f[2 * k + 1], cs[4 * u + k]);
        store_vec<T>(dst + 8 * u, pack_vec<T>(f));
      } else {
        float f[8], g[8];
        const Vec8<T> lo = load_vec<T>(src + 8 * u), hi = load_vec<T>(src + pairs + 8 * u);
        unpack_vec<T>(lo, f);
        unpack_vec<T>(hi, g);
#pragma unroll
        for (int k = 0; k < 8; ++k) turn(f[k], g[k], cs[8 * u + k]);
        store_vec<T>(dst + 8 * u, pack_vec<T>(f));
        store_vec<T>(dst + pairs + 8 * u, pack_vec<T>(g));
      }
    } else {
      if (u >= rot_units) {
        const int c = a.rot + u - rot_units;
        if (src != dst) dst[c] = src[c];
      } else {
        const int i = INTERLEAVED ? 2 * u : u, j = INTERLEAVED ? 2 * u + 1 : pairs + u;
        float f = to_f<T>(src[i]), g = to_f<T>(src[j]);
        turn(f, g, cs[u]);
        dst[i] = from_f<T>(f);
        dst[j] = from_f<T>(g);
      }
    }
  }
}

int rope_launch(const lca_rope_args* r, cudaStream_t stream) {
  const int size = r->dtype == LCA_DTYPE_BF16 ? 2 : 4, per16 = 16 / size;
  RopeKernelArgs a = {{{r->q, r->q_out, r->q_token_stride, r->q_head_stride, r->q_out_token_stride, r->q_out_head_stride, r->q ? r->n_q_heads : 0},
                       {r->k, r->k_out, r->k_token_stride, r->k_head_stride, r->k_out_token_stride, r->k_out_head_stride, r->k ? r->n_k_heads : 0}},
                      r->positions, r->freqs, r->n_tokens, r->head_dim, r->rot_dim, 1, 0, r->factor, r->inverse ? -1.f : 1.f};
  bool vec = r->rot_dim % 16 == 0 && r->head_dim % 8 == 0;
  for (const RopePart& q : a.part)
    if (q.heads)
      vec = vec && ((reinterpret_cast<uintptr_t>(q.x) | reinterpret_cast<uintptr_t>(q.y)) & 15u) == 0 && q.x_token % per16 == 0 &&
            q.x_head % per16 == 0 && q.y_token % per16 == 0 && q.y_head % per16 == 0;
  // A CTA takes about 4096 vectors, or fewer, down to 256, where the SMs would have less than eight CTAs each; the table bounds its tokens.
  // 32768 tokens x 40 heads of 128 with 256 / 1024 / 4096 / 16384: 258 / 152 / 116 / 123 us; 256 tokens x 129 heads of 64: 4.0 / 5.1 / 6.7 / 25.
  const int heads = a.part[0].heads + a.part[1].heads, units = vec ? r->head_dim / 8 : r->head_dim / 2 + 1;
  const long long all = r->n_tokens * heads * units;
  long long per = all / (8 * 148);
  per = per > 4096 ? 4096 : per < 256 ? 256 : per;
  const int pairs = r->rot_dim / 2, most = ROPE_TABLE / pairs;
  long long tokens = per / ((long long)heads * units);
  if (tokens < 1) tokens = 1;
  a.tokens = (int)(tokens < most ? tokens : most);
  a.heads = heads;
  if (per < (long long)heads * units) a.heads = (int)((per + units - 1) / units);
  const long long gx = (r->n_tokens + a.tokens - 1) / a.tokens;
  long long gy = (heads + a.heads - 1) / a.heads;
  if (gy > 65535) { a.heads = (heads + 65534) / 65535; gy = (heads + a.heads - 1) / a.heads; }
  if (gx > 0x7fffffffll || (long long)a.tokens * a.heads * r->head_dim > 0x7fffffffll) return LCA_ERR_UNSUPPORTED_SHAPE;
  const dim3 grid((unsigned)gx, (unsigned)gy);
  auto go = [&](auto kern) { return launch_chained(kern, grid, ROPE_THREADS, 0, stream, 1, a); };
  if (size == 2) {
    if (r->interleaved) return vec ? go(rope_kernel<bf16, true, true>) : go(rope_kernel<bf16, true, false>);
    return vec ? go(rope_kernel<bf16, false, true>) : go(rope_kernel<bf16, false, false>);
  }
  if (r->interleaved) return vec ? go(rope_kernel<float, true, true>) : go(rope_kernel<float, true, false>);
  return vec ? go(rope_kernel<float, false, true>) : go(rope_kernel<float, false, false>);
}

}  // namespace lca
