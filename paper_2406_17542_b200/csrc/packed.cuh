// The packed layout of a solved layer's codes, and what the kernels that read it share.
//
// A code takes CW = 2, 3, 4 or 8 bits (1 and 2 bits: 2; 3: 3; 4: 4; 5 to 8: 8).  The layer is cut into blocks of 16 columns (j) x
// 128 inputs (i), padded with zero codes, stored one after the other, all blocks of 16 columns before those of the next 16:
//   block (jt, ib) at ((jt * nib) + ib) * 256 * CW bytes, nib = ceil(d_in / 128).
// A piece holds the 32 codes of one column whose i = 128 ib + 32 c + 8 q + e (c = 0..3, e = 0..7) share q = 0..3: what one lane of a
// 16 x 8 x 16 matrix instruction needs of a row of its left operand, and a run of 8 inputs for every 32, so that groups that are multiples of
// 32 end between two instructions.  A block is plane 0, [q][16 columns][P0 bytes], then plane 1, [q][16][P1]:
// P0 = 8, 8, 16, 16 and P1 = 0, 4, 0, 16 bytes for CW = 2, 3, 4, 8.
// Codes are stored in pairs (2p, 2p + 1), p = 4 c + e / 2 = 0..15, the first in the low half of a word and the second at the same place of the
// high half, so that a shift and one three-input logic operation make a pair of bf16 numbers of 128 + code:
//   CW 2: word p / 8, bit 2 (p % 8);  CW 4: word p / 4, bit 4 (p % 4);  CW 8: word p / 2, bit 8 (p % 2);
//   CW 3: word p / 5, bit 3 (p % 5) for p < 15, and of pair 15 bit v at bit 15 of word v.
#pragma once

#include <cuda_bf16.h>

#include "common.cuh"

namespace cdq {

inline int packed_width(int bits) { return bits <= 2 ? 2 : bits == 3 ? 3 : bits == 4 ? 4 : 8; }
inline long long packed_blocks(long long d) { return (d + 127) / 128; }
inline long long packed_tiles(long long d) { return (d + 15) / 16; }
inline size_t packed_bytes_of(int bits, long long d_in, long long d_out) {
  return (size_t)packed_blocks(d_in) * packed_tiles(d_out) * 256 * packed_width(bits);
}

template <int CW> struct Piece {
  static constexpr int P0 = CW == 2 || CW == 3 ? 8 : 16;
  static constexpr int P1 = CW == 3 ? 4 : CW == 8 ? 16 : 0;
  static constexpr int WORDS = (P0 + P1) / 4;
  static constexpr int BLOCK = 256 * CW;
};

// The layer as the kernels see it.
struct PackedView {
  const unsigned char* codes;
  const float* scale;   // [ng, d_out]
  const float* zero;
  long long d_in, d_out;
  int g, ng;            // group size (d_in per channel), groups
  int nib;              // blocks of 128 inputs
  int njt;              // tiles of 16 columns
  int z;                // 2^(bits - 1): the kernels multiply by code - z, an integer of at most eight bits, exact in bf16
  uint32_t sub;         // bf16 pair of what is taken from the number that a code's bits make: 128 + z, or 256 for 8 bits (see dequant_pair)
};

// Makes code - z of the pair in `v` (codes in the low bits of both halves, everything else zero).  A bf16 number has seven stored
// mantissa bits, so 0x4300 with the code in them is 128 + code, exactly.  Eight-bit codes put their top bit aside: 128 + (code & 127) minus 128 where
// the top bit is set and 256 where it is not is code - 128 (z = 128); with fewer bits the top bit is zero and `sub` is 128 + z.
template <int CW>
__device__ __forceinline__ uint32_t centre_pair(uint32_t v, uint32_t sub) {
  uint32_t m, s = sub, r;
  if (CW == 8) {
    m = (v & 0x007f007fu) | 0x43004300u;
    s = sub ^ (v & 0x00800080u);
  } else {
    m = v | 0x43004300u;
  }
  asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(m), "r"(s));
  return r;
}

// Pair p (0..15, known at compile time once the loops are unrolled) of a piece.
template <int CW>
__device__ __forceinline__ uint32_t code_pair(const uint32_t* w, int p) {
  if (CW == 2) return (w[p >> 3] >> (2 * (p & 7))) & 0x00030003u;
  if (CW == 4) return (w[p >> 2] >> (4 * (p & 3))) & 0x000f000fu;
  if (CW == 8) return (w[p >> 1] >> (8 * (p & 1))) & 0x00ff00ffu;
  if (p < 15) return (w[p / 5] >> (3 * (p % 5))) & 0x00070007u;
  return ((w[0] >> 15) & 0x00010001u) | ((w[1] >> 14) & 0x00020002u) | ((w[2] >> 13) & 0x00040004u);
}

template <int CW>
__device__ __forceinline__ uint32_t dequant_pair(const uint32_t* w, int p, uint32_t sub) {
  return centre_pair<CW>(code_pair<CW>(w, p), sub);
}

// One piece: quarter q of column `row` (0..15) of a block.  The codes are read once per pass: they need no place in L1.
template <int CW>
__device__ __forceinline__ void load_piece(const unsigned char* block, int q, int row, uint32_t* w) {
  const unsigned char* a = block + (q * 16 + row) * Piece<CW>::P0;
  if (Piece<CW>::P0 == 16) {
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(a));
  } else {
    asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(a));
  }
  const unsigned char* b = block + 64 * Piece<CW>::P0 + (q * 16 + row) * Piece<CW>::P1;
  if (CW == 3) asm volatile("ld.global.nc.L1::no_allocate.u32 %0, [%1];" : "=r"(w[2]) : "l"(b));
  if (CW == 8)
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(b));
}

// fp32 = hi + mid + lo exactly, each a bf16 number: the upper 8, the next 8 and the last 8 bits of the mantissa, by truncation, so that nothing
// overflows (rounding 3.4e38 to bf16 would).  What is not finite stays in `hi` alone.
__device__ __forceinline__ void split3(float x, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
  const uint32_t b = __float_as_uint(x);
  hi = b >> 16;
  if ((b & 0x7f800000u) == 0x7f800000u) {
    if (b & 0x007fffffu) hi |= 0x40u;   // a NaN whose payload lies in the lower half stays one
    mid = lo = 0;
    return;
  }
  const float r1 = x - __uint_as_float(b & 0xffff0000u);
  const uint32_t b1 = __float_as_uint(r1);
  mid = b1 >> 16;
  lo = __float_as_uint(r1 - __uint_as_float(b1 & 0xffff0000u)) >> 16;
}

// ---- activations -------------------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ float act_of(float z, int act) {
  switch (act) {
    case CDQ_ACT_RELU: return z < 0.f ? 0.f : z;   // a NaN stays
    case CDQ_ACT_SILU: return __fdividef(z, 1.f + __expf(-z));
    case CDQ_ACT_GELU: return 0.5f * z * (1.f + erff(z * 0.70710678f));
    case CDQ_ACT_GELU_TANH: {
      // 0.5 (1 + tanh u) = 1 / (1 + exp(-2 u))
      const float u = 0.79788456f * (z + 0.044715f * z * z * z);
      return __fdividef(z, 1.f + __expf(-2.f * u));
    }
  }
  return z;
}
__device__ __forceinline__ float act_slope(float z, int act) {
  switch (act) {
    case CDQ_ACT_RELU: return z > 0.f ? 1.f : 0.f;
    case CDQ_ACT_SILU: {
      const float s = __fdividef(1.f, 1.f + __expf(-z));
      return s * (1.f + z * (1.f - s));
    }
    case CDQ_ACT_GELU: return 0.5f * (1.f + erff(z * 0.70710678f)) + z * 0.39894228f * __expf(-0.5f * z * z);
    case CDQ_ACT_GELU_TANH: {
      const float u = 0.79788456f * (z + 0.044715f * z * z * z);
      const float s = __fdividef(1.f, 1.f + __expf(-2.f * u));
      return s + z * s * (1.f - s) * 2.f * 0.79788456f * (1.f + 0.134145f * z * z);
    }
  }
  return 1.f;
}

__device__ __forceinline__ float load_x(const void* X, cdq_dtype t, long long i) {
  return t == CDQ_BF16 ? __bfloat162float(((const __nv_bfloat16*)X)[i]) : ((const float*)X)[i];
}
__device__ __forceinline__ void store_y(void* Y, cdq_dtype t, long long i, float v) {
  if (t == CDQ_BF16) ((__nv_bfloat16*)Y)[i] = __float2bfloat16_rn(v);
  else ((float*)Y)[i] = v;
}

// What follows the product: y = act(z + bias) + residual, the pre-activation kept for the backward pass where it is asked for.
struct Epilogue {
  const float* bias;      // [d_out], may be NULL
  const void* residual;   // [n, ldr], may be NULL; may be Y itself (every element is read by the thread that writes it)
  void* Y;
  void* Z;                // [n, ldz], may be NULL
  long long ldr, ldy, ldz;
  int act;
  cdq_dtype xt;
};
__device__ __forceinline__ void write_out(const Epilogue& e, long long tok, long long j, float z) {
  if (e.bias) z += e.bias[j];
  if (e.Z) store_y(e.Z, e.xt, tok * e.ldz + j, z);
  float y = act_of(z, e.act);
  if (e.residual) y += load_x(e.residual, e.xt, tok * e.ldr + j);
  store_y(e.Y, e.xt, tok * e.ldy + j, y);
}

}  // namespace cdq
