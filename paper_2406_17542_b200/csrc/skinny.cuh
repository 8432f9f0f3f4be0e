// Few rows times packed codes: the 16 x 8 x 16 matrix instruction with the codes as its left operand (16 columns of the layer), the rows of X as
// its right one, as used by linear_skinny.cu and moe.cu.
#pragma once

#include "packed.cuh"

namespace cdq {

__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Codes requested ahead by a warp, in blocks: as many as hide the latency of DRAM (2 to 4 KB per warp) in about 32 registers.
template <int CW> struct Ahead { static constexpr int D = CW == 2 ? 6 : CW == 3 ? 5 : CW == 4 ? 4 : 2; };

// The lane's part of a block: rows lane / 4 and lane / 4 + 8 of quarter lane % 4.
template <int CW>
__device__ __forceinline__ void load_block(const unsigned char* block, int lane, uint32_t* w) {
  load_piece<CW>(block, lane & 3, lane >> 2, w);
  load_piece<CW>(block, lane & 3, (lane >> 2) + 8, w + Piece<CW>::WORDS);
}

// P += codes of 32 inputs (chunk c of the block) x rows, S += the sums of the rows (the same instruction with ones on the left, so that they lie where P
// lies).  xs: row 0 of the staged rows at the chunk's first input, plus 8 (lane % 4); tok: the lane's row of every tile of eight.
template <int CW, int NT, int TERMS>
__device__ __forceinline__ void mma_chunk(const uint32_t* w, int c, uint32_t sub, const __nv_bfloat16* xs, const int (&row_at)[NT], int term_at,
                                          float (&P)[NT][4], float (&S)[NT][4]) {
  constexpr int W = Piece<CW>::WORDS;
  uint32_t a[4], b[4];
#pragma unroll
  for (int p = 0; p < 4; ++p) { a[p] = dequant_pair<CW>(w, 4 * c + p, sub); b[p] = dequant_pair<CW>(w + W, 4 * c + p, sub); }
  constexpr uint32_t ONES = 0x3f803f80u;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int m = 0; m < TERMS; ++m) {
      const uint4 x = *reinterpret_cast<const uint4*>(xs + row_at[t] + m * term_at);
      mma_16816(P[t], a[0], b[0], a[1], b[1], x.x, x.y);
      mma_16816(S[t], ONES, ONES, ONES, ONES, x.x, x.y);
      mma_16816(P[t], a[2], b[2], a[3], b[3], x.z, x.w);
      mma_16816(S[t], ONES, ONES, ONES, ONES, x.z, x.w);
    }
}

// acc += a P + (b + z a) S for the group's scales and zeros of the lane's two columns; P and S start anew.
template <int NT>
__device__ __forceinline__ void promote(float a0, float b0, float a1, float b1, float z, float (&P)[NT][4], float (&S)[NT][4], float (&acc)[NT][4]) {
  b0 = fmaf(z, a0, b0);
  b1 = fmaf(z, a1, b1);
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    acc[t][0] = fmaf(a0, P[t][0], fmaf(b0, S[t][0], acc[t][0]));
    acc[t][1] = fmaf(a0, P[t][1], fmaf(b0, S[t][1], acc[t][1]));
    acc[t][2] = fmaf(a1, P[t][2], fmaf(b1, S[t][2], acc[t][2]));
    acc[t][3] = fmaf(a1, P[t][3], fmaf(b1, S[t][3], acc[t][3]));
#pragma unroll
    for (int v = 0; v < 4; ++v) P[t][v] = S[t][v] = 0.f;
  }
}

// Stages inputs [i0, i0 + len) of `rows` rows into shared memory as bf16 (fp32 as three terms), zeros past d_in; len is a multiple of 8.
// Row r of term m starts at m * term_at + r * pitch.
template <int TERMS>
__device__ __forceinline__ void stage_rows(__nv_bfloat16* xs, int pitch, int term_at, const void* X, long long ldx, long long d_in, int rows,
                                           long long i0, int len, bool vec) {
  const int per = len / 8;
  for (int v = threadIdx.x; v < rows * per; v += blockDim.x) {
    const int r = v / per, c = (v - r * per) * 8;
    const long long i = i0 + c;
    uint32_t x[TERMS][4];
    if (TERMS == 1) {
      const __nv_bfloat16* src = (const __nv_bfloat16*)X + r * ldx + i;
      if (vec && i + 8 <= d_in) {
        const uint4 y = *reinterpret_cast<const uint4*>(src);
        x[0][0] = y.x; x[0][1] = y.y; x[0][2] = y.z; x[0][3] = y.w;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t lo = i + 2 * e < d_in ? __bfloat16_as_ushort(src[2 * e]) : 0, hi = i + 2 * e + 1 < d_in ? __bfloat16_as_ushort(src[2 * e + 1]) : 0;
          x[0][e] = lo | hi << 16;
        }
      }
    } else {
      const float* src = (const float*)X + r * ldx + i;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        uint32_t t[2][3];
#pragma unroll
        for (int h = 0; h < 2; ++h) split3(i + 2 * e + h < d_in ? src[2 * e + h] : 0.f, t[h][0], t[h][1], t[h][2]);
#pragma unroll
        for (int m = 0; m < TERMS; ++m) x[m][e] = t[0][m] | t[1][m] << 16;
      }
    }
#pragma unroll
    for (int m = 0; m < TERMS; ++m)
      *reinterpret_cast<uint4*>(xs + m * term_at + r * pitch + c) = make_uint4(x[m][0], x[m][1], x[m][2], x[m][3]);
  }
}

}  // namespace cdq
