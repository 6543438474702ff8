// The 4-bit format of the paged cache: value = code * 2^(exponent of its row - shift of its block of 32 columns).
//
// Codes have a sign and one of the magnitudes 0, 1/2, 1, 3/2, 2, 3, 4, 6.  Eight fill a 32-bit word; value i has its magnitude's
// index in bits 4 i .. 4 i + 2, so that a nibble without its top bit selects a byte of a table of eight (one byte permutation for
// four values), and its sign in bit 8 i + 7 (i < 4) or 8 (i - 4) + 3, where the four of one permutation are the top bits of its
// four bytes, as they stand or after one shift.  Seven instructions make eight e4m3 codes.
//
// A block is expanded to e4m3 relative to its row: code * 2^(6 - shift), from 2^-9 (shift 14) to 384, all of them e4m3 values.  So
// the expansion is exact and what remains is one power of two per row, 2^(exponent - 6).
#pragma once

#include <cuda_bf16.h>

#include "fp8_common.cuh"

namespace lca {

static constexpr int PAGED4_MAX_SHIFT = 14, PAGED4_NAN_SHIFT = 15;
static constexpr int PAGED4_MIN_EXP = PAGED8_MIN_EXP + 6;    // of a row of zeros: the factor of its expansion is then 2^PAGED8_MIN_EXP
static constexpr int PAGED4_EXP_BIAS = 127;

// log2 of the factor of an expanded row
__host__ __device__ constexpr int paged4_log2_factor(int exp_byte) {
  return (exp_byte > PAGED4_MIN_EXP + PAGED4_EXP_BIAS ? exp_byte : PAGED4_MIN_EXP + PAGED4_EXP_BIAS) - PAGED4_EXP_BIAS - 6;
}
__device__ __forceinline__ float paged4_factor(int exp_byte) { return exp2_int(paged4_log2_factor(exp_byte)); }

// e4m3 code of magnitude m times 2^(6 - shift)
constexpr uint32_t paged4_code(int m, int shift) {
  if (shift > PAGED4_MAX_SHIFT) return 0x7f;                 // NaN
  if (m == 0) return 0;
  const int lead = m == 1 ? -1 : m / 2 - 1, half = m >= 2 ? m & 1 : 0;       // magnitude = 2^lead (1 + half / 2)
  const int e = lead + 6 - shift;
  if (e >= -6) return (uint32_t)((e + 7) << 3 | half << 2);
  return (uint32_t)((2 + half) << (e + 9) >> 1);             // steps of 2^-9
}
struct Paged4Table {
  uint2 v[16];
  constexpr Paged4Table() : v() {
    for (int s = 0; s < 16; ++s) {
      v[s].x = paged4_code(0, s) | paged4_code(1, s) << 8 | paged4_code(2, s) << 16 | paged4_code(3, s) << 24;
      v[s].y = paged4_code(4, s) | paged4_code(5, s) << 8 | paged4_code(6, s) << 16 | paged4_code(7, s) << 24;
    }
  }
};
static __constant__ const Paged4Table g_paged4_table{};

// The table in shared memory (lanes read different entries); a barrier follows.
__device__ __forceinline__ void paged4_table_load(uint2* s_table, int t) { if (t < 16) s_table[t] = g_paged4_table.v[t]; }

// eight values as e4m3 codes, in order
__device__ __forceinline__ uint2 paged4_expand(uint32_t w, const uint2& table) {
  const uint32_t m = w & 0x77777777u;
  return make_uint2(__byte_perm(table.x, table.y, m) | (w & 0x80808080u),
                    __byte_perm(table.x, table.y, m >> 16) | ((w << 4) & 0x80808080u));
}

// The same with the two shifts as multiplications, on the pipe that the permutations and masks leave idle; `sixteen` is 16, which the
// compiler must not know.
__device__ __forceinline__ uint2 paged4_expand(uint32_t w, const uint2& table, uint32_t sixteen) {
  const uint32_t m = w & 0x77777777u;
  uint32_t up, hi;
  asm("mul.lo.u32 %0, %1, %2;" : "=r"(up) : "r"(w), "r"(sixteen));
  asm("mul.hi.u32 %0, %1, %2;" : "=r"(hi) : "r"(m), "r"(sixteen << 12));
  return make_uint2(__byte_perm(table.x, table.y, m) | (w & 0x80808080u), __byte_perm(table.x, table.y, hi) | (up & 0x80808080u));
}

// Eight bf16 values (two a word) times f to a word of codes: nearest magnitude, ties to the even index; infinities become 6.
__device__ __forceinline__ uint32_t paged4_pack(const uint4& v, float f) {
  const uint32_t u[4] = {v.x, v.y, v.z, v.w};
  float x[8];
#pragma unroll
  for (int k = 0; k < 4; ++k) { x[2 * k] = __uint_as_float(u[k] << 16) * f; x[2 * k + 1] = __uint_as_float(u[k] & 0xffff0000u) * f; }
  uint32_t w;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(w) : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
  // nibble i: magnitude and sign of value i.  The signs go where the expansion wants them; they are the top bits of the values' halves
  const uint32_t lo = __byte_perm(v.x, v.y, 0x7531), hi = __byte_perm(v.z, v.w, 0x7531);
  return (w & 0x77777777u) | (lo & 0x80808080u) | ((hi >> 4) & 0x08080808u);
}
// Eight codes to bf16 values, two a word, times a power of two (or NaN): exact.  Both bytes of a magnitude come from a table.
__device__ __forceinline__ uint4 paged4_unpack(uint32_t w, __nv_bfloat162 scale) {
  const uint32_t m = w & 0x77777777u, n = m >> 16, up = w << 4;
  // 0, 0.5, 1, 1.5 / 2, 3, 4, 6 are 0000 3f00 3f80 3fc0 / 4000 4040 4080 40c0
  const uint32_t l0 = __byte_perm(0xc0800000u, 0xc0804000u, m), h0 = __byte_perm(0x3f3f3f00u, 0x40404040u, m) | (w & 0x80808080u);
  const uint32_t l1 = __byte_perm(0xc0800000u, 0xc0804000u, n), h1 = __byte_perm(0x3f3f3f00u, 0x40404040u, n) | (up & 0x80808080u);
  uint4 r = make_uint4(__byte_perm(l0, h0, 0x5140), __byte_perm(l0, h0, 0x7362), __byte_perm(l1, h1, 0x5140), __byte_perm(l1, h1, 0x7362));
  uint32_t* q = &r.x;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const __nv_bfloat162 x = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(q + k), scale);
    q[k] = *reinterpret_cast<const uint32_t*>(&x);
  }
  return r;
}
// the power of two of a block, NaN for a NaN block
__device__ __forceinline__ __nv_bfloat162 paged4_scale(int exp_byte, int shift) {
  const int e = (exp_byte > PAGED4_MIN_EXP + PAGED4_EXP_BIAS ? exp_byte : PAGED4_MIN_EXP + PAGED4_EXP_BIAS) - shift;       // 19 .. 255, biased
  const uint32_t bits = shift == PAGED4_NAN_SHIFT ? 0x7fffu : (uint32_t)e << 7, two = bits | bits << 16;
  return *reinterpret_cast<const __nv_bfloat162*>(&two);
}

// log2 of the scale of a block whose largest finite |x| has these bf16 bits: smallest e with |x| <= 6 * 2^e.  6 = 1.5 * 2^2, and a
// significand above 1.5 = 1 + 64 / 128 carries into the exponent.  (Zero and subnormal numbers: far below PAGED4_MIN_EXP.)
__device__ __forceinline__ int paged4_block_exponent(uint32_t bits) { return (int)((bits + 63u) >> 7) - 129; }

}  // namespace lca
