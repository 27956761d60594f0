// INT2 records as fp16 rows for the tensor cores (cache read-back, chunk
// attention).
//
// Word w of a slot's 32 code bytes holds the codes of channels 32 g + 4 w + r
// at bits 8 g + 2 r (include/optr.h), so its two 16-bit halves carry the same
// fields of groups g and g + 2, and one packed operation dequantizes both.  A
// row therefore comes out in the order
//   k = 16 w + 8 (g & 1) + 2 r + (g >> 1)   <->   channel 32 g + 4 w + r
// (row_channel), which the other operand of its product takes too: the rows
// and columns of a product's inner dimension may be permuted together.
#pragma once

#include "optr_internal.cuh"

namespace optr {

// Channel at place k of a dequantized row.
__host__ __device__ constexpr int row_channel(int k) {
  return 32 * (((k >> 3) & 1) + 2 * (k & 1)) + 4 * (k >> 4) + ((k >> 1) & 3);
}

// A slot's {scale, min} pairs as packed operands: groups (0, 2) and (1, 3).
struct SlotMeta {
  uint32_t s02, m02, s13, m13;
};

__device__ __forceinline__ uint32_t lo_halves(uint32_t a, uint32_t b) { return __byte_perm(a, b, 0x5410); }
__device__ __forceinline__ uint32_t hi_halves(uint32_t a, uint32_t b) { return __byte_perm(a, b, 0x7632); }

// From the four groups' words (scale low, min high).
__device__ __forceinline__ SlotMeta slot_meta(uint32_t g0, uint32_t g1, uint32_t g2, uint32_t g3) {
  return SlotMeta{lo_halves(g0, g2), hi_halves(g0, g2), lo_halves(g1, g3), hi_halves(g1, g3)};
}

__device__ __forceinline__ uint32_t hfma2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}

// Keeps in `past` whether a slot had a group with an end past fp16's range (codes 0
// and 3: min, itself fp16, and 3 scale + min), whose row comes out as infinities:
// zero times the upper end is a NaN then, which stays.  Four operations a row: the
// chunk attention takes 1% longer for them, 2% with a test of each row.
__device__ __forceinline__ void note_range(const SlotMeta& m, uint32_t& past) {
  constexpr uint32_t kThree = 0x42004200u;
  past = hfma2(hfma2(m.s02, kThree, m.m02), 0u, past);
  past = hfma2(hfma2(m.s13, kThree, m.m13), 0u, past);
}
__device__ __forceinline__ bool any_past_range(uint32_t past) { return (past & 0x7fff7fffu) != 0; }

// The field at bit kPos (4, 6 or 8) of each half of x as the exact fp16 code:
// one LOP3 puts it into the mantissa of 1024 (1024 + code 2^kPos), one HFMA2
// takes the offset off again.
template <int kPos>
__device__ __forceinline__ uint32_t code_f16x2(uint32_t x) {
  uint32_t y;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;"  // (a & b) | c
      : "=r"(y) : "r"(x), "n"(0x00030003u << kPos), "r"(0x64006400u));
  constexpr uint32_t kScale = (uint32_t)(15 - kPos) << 10;             // 2^-kPos
  constexpr uint32_t kShift = 0x8000u | (uint32_t)(25 - kPos) << 10;   // -2^(10 - kPos)
  return hfma2(y, kScale * 0x10001u, kShift * 0x10001u);
}

// Word w of a slot's codes as the 16 values at places 16 w .. 16 w + 15 of the
// row: code * scale + min, rounded once to fp16 (codes, scales and minima are
// exact in fp16, so this is within 2^-11 of the value the record stands for).
__device__ __forceinline__ void dequant_word(uint32_t x, const SlotMeta& m, uint32_t (&out)[8]) {
  const uint32_t xl = x << 4, xr = x >> 6;
  out[0] = hfma2(code_f16x2<4>(xl), m.s02, m.m02);
  out[1] = hfma2(code_f16x2<6>(xl), m.s02, m.m02);
  out[2] = hfma2(code_f16x2<4>(x), m.s02, m.m02);
  out[3] = hfma2(code_f16x2<6>(x), m.s02, m.m02);
  out[4] = hfma2(code_f16x2<8>(x), m.s13, m.m13);
  out[5] = hfma2(code_f16x2<4>(xr), m.s13, m.m13);
  out[6] = hfma2(code_f16x2<6>(xr), m.s13, m.m13);
  out[7] = hfma2(code_f16x2<8>(xr), m.s13, m.m13);
}

}  // namespace optr
