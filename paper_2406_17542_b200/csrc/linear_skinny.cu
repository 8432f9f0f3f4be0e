// Y = act(X W_hat + bias) + residual for up to 16 rows of X: the layer while tokens are generated.
//
//   z[n, j] = sum_t a_t,j P_t[n, j] + (b_t,j + z a_t,j) S_t[n],   P_t = X_t (Q_t - z),   S_t[n] = sum_{i in t} X[n, i]
//
// P_t comes from bf16 matrix instructions whose operands are exact: Q - z is an integer of at most eight bits, X is bf16 (or fp32 as three bf16 terms).
// Scales meet the fp32 sums, once per group, so the result is that of the fp32 formula.
//
// Bound by the bytes of the codes.  Every warp owns tiles of 16 columns x 128 inputs (256 CW bytes in a row of DRAM, read by 8- or 16-byte loads
// straight into the operand's registers, a few blocks ahead); WJ x WK = 8 warps of a block take WJ tiles of columns and every WK-th block of
// inputs, and a cluster of CK thread blocks shares a long column.  The sums of warps and blocks are added in a fixed order, through shared memory
// and the cluster's shared memory: no workspace, no atomics, one launch.
#include <cooperative_groups.h>

#include "linear.cuh"
#include "skinny.cuh"

namespace cdq {
namespace {

namespace cg = cooperative_groups;

struct Params {
  PackedView w;
  const void* X;
  long long ldx;
  Epilogue ep;
  int n, wj, wk, ck, slab, vec;
};

// GM: where a group can end -- 0 nowhere (one group), 1 at blocks of 128 inputs, 2 at chunks of 32.
template <int CW, int NT, int TERMS, int GM>
__global__ void __launch_bounds__(256) linear_skinny_kernel(const __grid_constant__ Params p) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int W = Piece<CW>::WORDS, D = Ahead<CW>::D, BLOCK = Piece<CW>::BLOCK;
  const PackedView& w = p.w;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wj = warp % p.wj, wk = warp / p.wj;
  const int rank = (int)(blockIdx.x % p.ck), jt = (int)(blockIdx.x / p.ck) * p.wj + wj;
  const int ib0 = (int)((long long)w.nib * rank / p.ck), ib1 = (int)((long long)w.nib * (rank + 1) / p.ck);
  const bool on = jt < w.njt;
  const int pitch = p.slab * 128 + 32, term_at = p.n * pitch;   // rows 64 bytes apart modulo 128: eight lanes' vectors fill the banks
  __nv_bfloat16* xs = reinterpret_cast<__nv_bfloat16*>(smem);
  float* red = reinterpret_cast<float*>(smem + (size_t)TERMS * term_at * 2);

  const unsigned char* tile = w.codes + (long long)(on ? jt : 0) * w.nib * BLOCK;
  uint32_t ring[D][2 * W];
#pragma unroll
  for (int d = 0; d < D; ++d) {
    const int ib = ib0 + wk + d * p.wk;
    if (on && ib < ib1) load_block<CW>(tile + (long long)ib * BLOCK, lane, ring[d]);
  }
  // the lane's two columns (clamped: what lies past the last column is not stored)
  const long long j0 = min((long long)jt * 16 + (lane >> 2), w.d_out - 1), j1 = min((long long)jt * 16 + (lane >> 2) + 8, w.d_out - 1);
  float acc[NT][4] = {}, P[NT][4] = {}, S[NT][4] = {};
  int row_at[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) row_at[t] = min(t * 8 + (lane >> 2), p.n - 1) * pitch;
  const float zf = (float)w.z;
  auto scales = [&](long long i, float& a0, float& b0, float& a1, float& b1) {
    const long long t = GM == 0 ? 0 : i / w.g;
    a0 = __ldg(w.scale + t * w.d_out + j0); b0 = __ldg(w.zero + t * w.d_out + j0);
    a1 = __ldg(w.scale + t * w.d_out + j1); b1 = __ldg(w.zero + t * w.d_out + j1);
  };
  for (int s0 = ib0; s0 < ib1; s0 += p.slab) {
    const int s1 = min(s0 + p.slab, ib1);
    if (s0 > ib0) __syncthreads();
    stage_rows<TERMS>(xs, pitch, term_at, p.X, p.ldx, w.d_in, p.n, (long long)s0 * 128, (s1 - s0) * 128, p.vec);
    __syncthreads();
    for (int b = s0 + wk; b < s1; b += D * p.wk) {   // a slab is a multiple of D x WK blocks: ring[d] is always the block at hand
#pragma unroll
      for (int d = 0; d < D; ++d) {
        const int ib = b + d * p.wk;
        if (on && ib < s1) {
          float a0, b0, a1, b1;
          if (GM == 1) scales((long long)ib * 128, a0, b0, a1, b1);
          const __nv_bfloat16* x = xs + (ib - s0) * 128 + 8 * (lane & 3);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const long long i = (long long)ib * 128 + 32 * c;
            if (GM == 2) {
              if (i >= w.d_in) break;
              scales(i, a0, b0, a1, b1);
            }
            mma_chunk<CW, NT, TERMS>(ring[d], c, w.sub, x + 32 * c, row_at, term_at, P, S);
            if (GM == 2) promote<NT>(a0, b0, a1, b1, zf, P, S, acc);
          }
          if (GM == 1) promote<NT>(a0, b0, a1, b1, zf, P, S, acc);
        }
        const int next = ib + D * p.wk;
        if (on && next < ib1) load_block<CW>(tile + (long long)next * BLOCK, lane, ring[d]);
      }
    }
  }
  if (GM == 0) {
    float a0, b0, a1, b1;
    scales(0, a0, b0, a1, b1);
    promote<NT>(a0, b0, a1, b1, zf, P, S, acc);
  }
  // sums of the warps that share columns, then of the cluster's blocks, both in ascending order of the inputs' share
  const int cols = p.wj * 16, outs = cols * p.n;
  float* mine = red + (size_t)wk * outs;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int tok = t * 8 + 2 * (lane & 3) + (v & 1), col = wj * 16 + (lane >> 2) + 8 * (v >> 1);
      if (tok < p.n) mine[tok * cols + col] = acc[t][v];
    }
  __syncthreads();
  const long long jb = (long long)(blockIdx.x / p.ck) * cols;
  if (p.ck == 1) {
    for (int o = threadIdx.x; o < outs; o += 256) {
      float s = red[o];
      for (int k = 1; k < p.wk; ++k) s += red[(size_t)k * outs + o];
      const int tok = o / cols;
      const long long j = jb + (o - tok * cols);
      if (j < w.d_out) write_out(p.ep, tok, j, s);
    }
  } else {
    cg::cluster_group cluster = cg::this_cluster();
    for (int o = threadIdx.x; o < outs; o += 256) {
      float s = red[o];
      for (int k = 1; k < p.wk; ++k) s += red[(size_t)k * outs + o];
      red[o] = s;   // read by this thread alone so far
    }
    cluster.sync();
    for (int o = rank * 256 + threadIdx.x; o < outs; o += p.ck * 256) {
      float s = 0.f;
      for (int r = 0; r < p.ck; ++r) s += *cluster.map_shared_rank(red + o, r);
      const int tok = o / cols;
      const long long j = jb + (o - tok * cols);
      if (j < w.d_out) write_out(p.ep, tok, j, s);
    }
    cluster.sync();   // no block's shared memory goes while another reads it
  }
}

template <int CW, int NT, int TERMS, int GM>
cudaError_t launch(const Params& p, int blocks, size_t bytes, cudaStream_t st) {
  auto kern = linear_skinny_kernel<CW, NT, TERMS, GM>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(256);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)p.ck;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, kern, p);
  count_launch();
  return e;
}

template <int CW, int NT, int TERMS>
cudaError_t launch_gm(const Params& p, int blocks, size_t bytes, cudaStream_t st) {
  if (p.w.ng == 1) return launch<CW, NT, TERMS, 0>(p, blocks, bytes, st);
  return p.w.g % 128 == 0 ? launch<CW, NT, TERMS, 1>(p, blocks, bytes, st) : launch<CW, NT, TERMS, 2>(p, blocks, bytes, st);
}

template <int CW>
cudaError_t launch_cw(const Params& p, bool f32, int blocks, size_t bytes, cudaStream_t st) {
  if (p.n <= 8) return f32 ? launch_gm<CW, 1, 3>(p, blocks, bytes, st) : launch_gm<CW, 1, 1>(p, blocks, bytes, st);
  return f32 ? launch_gm<CW, 2, 3>(p, blocks, bytes, st) : launch_gm<CW, 2, 1>(p, blocks, bytes, st);
}

}  // namespace

bool linear_skinny_takes(const PackedView& w, long long n) { return n <= 16 && (w.ng == 1 || w.g % 32 == 0); }

cudaError_t launch_linear_skinny(const PackedView& w, int cw, const void* X, long long n, long long ldx, const Epilogue& ep, cudaStream_t st) {
  Params p{};
  p.w = w; p.X = X; p.ldx = ldx; p.ep = ep; p.n = (int)n;
  const bool f32 = ep.xt == CDQ_F32;
  p.vec = !f32 && ldx % 8 == 0 && aligned16(X);
  const int D = cw == 2 ? 6 : cw == 3 ? 5 : cw == 4 ? 4 : 2, terms = f32 ? 3 : 1;
  p.wj = 2; p.wk = 4; p.ck = 1;
  while (p.ck < 8 && (long long)((w.njt + p.wj - 1) / p.wj) * p.ck < 296 && w.nib >= 2 * p.ck * p.wk) p.ck *= 2;
#ifdef CDQ_TUNE
  if (const char* e = getenv("CDQ_SKINNY")) sscanf(e, "%d,%d,%d", &p.wj, &p.wk, &p.ck);
#endif
  // a slab holds at least what the rings do: many rows in fp32 take fewer warps along the inputs and more along the columns
  while (p.wk > 1 && (long long)2 * terms * n * (D * p.wk * 128 + 32) > 163840) { p.wk /= 2; p.wj *= 2; }
  // inputs staged at a time: all of the block's share if they take at most 64 KB, else a multiple of what the warps' rings hold
  const int share = (w.nib + p.ck - 1) / p.ck, unit = D * p.wk;
  const long long fit = (65536 / (2 * terms * n) - 32) / 128;
  p.slab = share <= fit ? share : (int)(fit / unit > 0 ? fit / unit * unit : unit);
  const size_t bytes = (size_t)terms * n * (p.slab * 128 + 32) * 2 + (size_t)p.wk * p.wj * 16 * n * sizeof(float);
  const int blocks = (w.njt + p.wj - 1) / p.wj * p.ck;
  switch (cw) {
    case 2: return launch_cw<2>(p, f32, blocks, bytes, st);
    case 3: return launch_cw<3>(p, f32, blocks, bytes, st);
    case 4: return launch_cw<4>(p, f32, blocks, bytes, st);
  }
  return launch_cw<8>(p, f32, blocks, bytes, st);
}

}  // namespace cdq
