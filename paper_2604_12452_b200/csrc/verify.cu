// Verification of drafted tokens: which of a request's drafts the target accepts, and the token that follows them.
//
// Draft i is accepted while u_i q_i(x_i) < p_i(x_i) (a product of two fp32 numbers, exact in 64 bits).  After the first rejection, at i,
// the next token is drawn from max(p_i - q_i, 0), after the last accepted draft from p: the smallest token whose cumulative sum
// exceeds u times the whole.  Sums are 64-bit: with 32 the sum of 10^5 probabilities is off by more than many of them, and the
// token would depend on the order.
// Only what decides is read: two numbers for each draft, then one row of p and one of q.  A cluster takes a request, so that its CTAs
// share the row; each sums its part warp by warp; the CTA whose part holds the crossing finds the warp, spreads that warp's few
// hundred tokens over all its warps (from L2) and goes through the last few dozen.  Bound by the chain of
// four dependent trips to memory, for many requests by HBM and by conversions to 64 bits too (64 x 128000 fp32 tokens: 21 us, 3.1 TB/s).
#include "lca_common.cuh"
#include "tc_common.cuh"

namespace lca {

static const int VERIFY_THREADS = 256, VERIFY_WARPS = VERIFY_THREADS / 32, VERIFY_MOST_CTAS = 16;

struct VerifyArgs {
  const void* target; const void* draft; const int32_t* tokens; const float* u_accept; const float* u_sample;
  const int32_t* n_draft; const int32_t* n_tok;
  int32_t* accepted; int32_t* out; int32_t* n_tok_out;
  int B, K, V;
};

template <class T> __device__ __forceinline__ float prob(const T* p) {
  if constexpr (sizeof(T) == 2) return __bfloat162float(*p); else return *p;
}
template <class T>
__device__ __forceinline__ float4 vec4(const T* p) {
  if constexpr (sizeof(T) == 2) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u));
  } else return *reinterpret_cast<const float4*>(p);
}
// Values [x, x + 4) of a row (zero behind V), one vector where the row allows it.
template <class T>
__device__ __forceinline__ float4 four(const T* row, int x, int V, bool wide) {
  if (wide && x + 4 <= V) return vec4(row + x);
  return make_float4(x < V ? prob(row + x) : 0.f, x + 1 < V ? prob(row + x + 1) : 0.f, x + 2 < V ? prob(row + x + 2) : 0.f,
                     x + 3 < V ? prob(row + x + 3) : 0.f);
}
// Mass of a token, max(p - q, 0).  Its sign does not need 64 bits (a difference of two fp32 numbers is not rounded to 0), and what is no
// positive finite number has none; compared in 64 bits, the comparisons were half of the kernel's instructions.
__device__ __forceinline__ double mass(float p, float q) {
  const float r = p - q;
  const bool some = r > 0.f && r < INFINITY;
  return (double)(some ? p : 0.f) - (double)(some ? q : 0.f);
}

template <class T>
__global__ void __launch_bounds__(VERIFY_THREADS) verify_kernel(VerifyArgs a) {
  __shared__ double s_warp[VERIFY_WARPS], s_sub[VERIFY_WARPS], s_cta[VERIFY_MOST_CTAS];
  __shared__ int s_taken;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)tc::cluster_ctarank(), C = (int)(gridDim.x / a.B), b = (int)(blockIdx.x / C);
  // The CTAs write to one another's shared memory, which each may do once all have started: the other half of this barrier stands before
  // the first of those writes, so that the wait lies behind the reads up to there.
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  chain_wait();
  chain_next();
  const int K = a.K, V = a.V;
  const int n = a.n_draft ? min(max(a.n_draft[b], 0), K) : K;
  const T* target = (const T*)a.target + (size_t)b * (K + 1) * V;
  const T* draft = a.draft ? (const T*)a.draft + (size_t)b * K * V : nullptr;
  const float u_sample = a.u_sample[b];
  // (1) accepted drafts; every CTA of the cluster looks for itself
  if (warp == 0) {
    int taken = n;
    for (int i0 = 0; i0 < n; i0 += 32) {
      const int i = i0 + lane;
      bool bad = false;
      if (i < n) {
        const int x = a.tokens[(size_t)b * K + i];
        bad = true;                                          // a token outside the vocabulary has no probability
        if (x >= 0 && x < V) {
          const float p = prob(target + (size_t)i * V + x), q = draft ? prob(draft + (size_t)i * V + x) : 1.f;
          bad = !((double)a.u_accept[(size_t)b * K + i] * (double)q < (double)p);
        }
      }
      const unsigned m = __ballot_sync(0xffffffffu, bad);
      if (m) { taken = i0 + __ffs((int)m) - 1; break; }
    }
    if (lane == 0) s_taken = taken;
  }
  __syncthreads();
  const int taken = s_taken;
  const T* p = target + (size_t)taken * V;
  const T* q = taken < n && draft ? draft + (size_t)taken * V : nullptr;
  const int gone = taken < n && !draft ? a.tokens[(size_t)b * K + taken] : -1;      // the one token of a drafter without probabilities
  const uintptr_t mask = 4 * sizeof(T) - 1;
  const bool p_wide = (reinterpret_cast<uintptr_t>(p) & mask) == 0, q_wide = (reinterpret_cast<uintptr_t>(q) & mask) == 0;
  // (2) this warp's part of the row: whole vectors of four tokens for 32 lanes
  const int span = (int)(((long long)V + C * VERIFY_WARPS * 128 - 1) / (C * VERIFY_WARPS * 128)) * 128;
  const long long begin = (long long)(rank * VERIFY_WARPS + warp) * span;
  const int lo = (int)min(begin, (long long)V), hi = (int)min(begin + span, (long long)V);
  // nothing is left of a rejected row only where p <= q everywhere: then p itself
#pragma unroll 1
  for (int attempt = 0; attempt < 2; ++attempt) {
    const bool residual = attempt == 0;
    double sum = 0.0;
    const bool with_q = residual && q;
    const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
    auto mass4 = [&](const float4& f, const float4& g) { return (mass(f.x, g.x) + mass(f.y, g.y)) + (mass(f.z, g.z) + mass(f.w, g.w)); };
    int x = lo + 4 * lane;
    const bool skip = residual && gone >= lo && gone < hi;   // the one token that a certain drafter proposed and the target rejected
    if (p_wide && (!with_q || q_wide) && !skip) {
      const int stop = min(hi, V & ~3);                      // eight whole vectors on their way
      for (; x + 7 * 128 < stop; x += 8 * 128) {
        float4 f[8], g[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) { f[k] = vec4(p + x + 128 * k); g[k] = with_q ? vec4(q + x + 128 * k) : zero; }
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += mass4(f[k], g[k]);
      }
    }
    for (; x < hi; x += 128) {
      float4 f = four(p, x, V, p_wide);
      if (skip && (unsigned)(gone - x) < 4u) { if (gone == x) f.x = 0.f; else if (gone == x + 1) f.y = 0.f; else if (gone == x + 2) f.z = 0.f; else f.w = 0.f; }
      sum += mass4(f, with_q ? four(q, x, V, q_wide) : zero);
    }
    sum = warp_sum(sum);
    if (lane == 0) s_warp[warp] = sum;
    __syncthreads();
    if (attempt == 0) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");      // all CTAs have started
    if (warp == 0) {                                         // the CTA's sum to every CTA of the cluster
      double s = lane < VERIFY_WARPS ? s_warp[lane] : 0.0;
      s = warp_sum(s);
      if (lane < C) {
        const uint32_t at = tc::mapa_u32(tc::smem_u32(&s_cta[rank]), (uint32_t)lane);
        asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(at), "d"(s) : "memory");
      }
    }
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    double total = 0.0;
    for (int c = 0; c < C; ++c) total += s_cta[c];
    if (total > 0.0) {
      const double want = (double)u_sample * total;
      // the CTA: the first whose sums reach beyond `want`, or the last one with mass where rounding leaves none
      double before = 0.0;
      int cta = -1;
      double at = 0.0;
      for (int c = 0; c < C; ++c) {
        if (s_cta[c] > 0.0) { cta = c; at = before; }
        before += s_cta[c];
        if (s_cta[c] > 0.0 && before > want) break;
      }
      if (rank == cta) {                                     // the same for every thread of the CTA
        int w = -1;
        before = at;
        for (int k = 0; k < VERIFY_WARPS; ++k) {
          if (s_warp[k] > 0.0) { w = k; at = before; }
          before += s_warp[k];
          if (s_warp[k] > 0.0 && before > want) break;
        }
        // that warp's part again, split over all warps: their sums, then the tokens of the one with the crossing, 32 at a time
        const long long first = (long long)(rank * VERIFY_WARPS + w) * span;
        const int sub = (span / VERIFY_WARPS + 31) / 32 * 32;
        const int end = (int)min(first + span, (long long)V);
        auto range = [&](int k, int& a0, int& a1) { a0 = (int)min(first + (long long)k * sub, (long long)end); a1 = min(a0 + sub, end); };
        auto one = [&](int x) {
          const float f = prob(p + x), g = residual && q ? prob(q + x) : 0.f;
          return residual && x == gone ? 0.0 : mass(f, g);
        };
        int a0, a1;
        range(warp, a0, a1);
        double part = 0.0;
#pragma unroll 4
        for (int x = a0 + lane; x < a1; x += 32) part += one(x);
        part = warp_sum(part);
        if (lane == 0) s_sub[warp] = part;
        __syncthreads();
        if (warp == 0) {
          int k0 = -1;
          before = at;
          for (int k = 0; k < VERIFY_WARPS; ++k) {
            if (s_sub[k] > 0.0) { k0 = k; at = before; }
            before += s_sub[k];
            if (s_sub[k] > 0.0 && before > want) break;
          }
          range(k0, a0, a1);
          double run = at;                                   // sum of all tokens before this step's
          int token = -1;
          for (int x0 = a0; x0 < a1; x0 += 32) {
            const double mine = x0 + lane < a1 ? one(x0 + lane) : 0.0;
            double inc = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const double y = __shfl_up_sync(0xffffffffu, inc, o); if (lane >= o) inc += y; }
            const unsigned some = __ballot_sync(0xffffffffu, mine > 0.0), hit = __ballot_sync(0xffffffffu, mine > 0.0 && run + inc > want);
            if (some) token = x0 + 31 - __clz((int)some);    // the last one with mass, should rounding leave none
            if (hit) { token = x0 + __ffs((int)hit) - 1; break; }
            run += __shfl_sync(0xffffffffu, inc, 31);
          }
          if (lane == 0) a.out[(size_t)b * (K + 1) + taken] = token;
        }
      }
      break;                                                 // every CTA of the cluster, and every thread, alike
    }
    if (attempt == 1 || !(q || gone >= 0)) {                 // no mass at all
      if (rank == 0 && tid == 0) a.out[(size_t)b * (K + 1) + taken] = -1;
      break;
    }
    // s_warp and s_cta are written again
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  // (3) the tokens around it
  if (rank == 0) {
    for (int i = tid; i <= K; i += VERIFY_THREADS)
      if (i != taken) a.out[(size_t)b * (K + 1) + i] = i < taken ? a.tokens[(size_t)b * K + i] : -1;
    if (tid == 0) {
      a.accepted[b] = taken;
      if (a.n_tok_out) a.n_tok_out[b] = a.n_tok[b] - (n - taken);
    }
  }
  // a CTA stays until the others have written to its shared memory: they have, before the barrier that this one has passed
}

int verify_launch(const lca_verify_args* v, cudaStream_t stream) {
  VerifyArgs a = {v->target_probs, v->draft_probs, v->draft_tokens, v->u_accept, v->u_sample, v->n_draft, v->n_tok, v->accepted, v->tokens_out,
                  v->n_tok_out, v->batch, v->n_drafts, v->vocab};
  // CTAs of a request: as many as are resident at once, and not so many that a warp has nothing to read.  With 1 / 4 / 8 / 16: 1 request,
  // 32001 tokens bf16 34 / 12 / 7.7 / 5.9 us; 8000 tokens 7.6 / 5.1 / 4.6 / 4.9; 64 requests, 128000 tokens 83 / 23 / 21 / 21; 256 requests,
  // 32000 tokens 26 / 20 / 28 / 42.
  int c = 1;
  while (c < VERIFY_MOST_CTAS && (long long)v->batch * 2 * c <= 5 * 148 && (long long)v->vocab > (long long)c * VERIFY_WARPS * 128) c *= 2;
  if ((long long)v->batch * c > 0x7fffffffll) return LCA_ERR_UNSUPPORTED_SHAPE;
  const bool bf = v->dtype == LCA_DTYPE_BF16;
  auto kern = bf ? verify_kernel<bf16> : verify_kernel<float>;
  if (c > 8 && cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return LCA_ERR_CUDA;
  return launch_chained(kern, (unsigned)(v->batch * c), VERIFY_THREADS, 0, stream, (unsigned)c, a);
}

}  // namespace lca
