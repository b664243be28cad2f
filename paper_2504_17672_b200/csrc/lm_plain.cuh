// Products of any strides and sizes: fp32 on the CUDA cores.
// Taken where rows do not start on 16-byte boundaries, which TMA and 16-byte loads need.
// C[m][n] = sum over sources s < S and k < K of A_s(m, k) * B_s(n, k), 64 x 64 tiles.
#pragma once

#include "lm_common.cuh"

namespace cocodc_lm_impl {

template <typename T> struct Operand {
  const T* p;
  long long outer, k;     // element strides of the row (m or n) and of k
};
constexpr int kTile = 64, kDepth = 16;

template <typename T>
__device__ __forceinline__ void load_tile(float (*dst)[kTile + 1], const Operand<T>& o, long long r0, long long rows,
                                          long long k0, long long K) {
  for (int i = threadIdx.x; i < kTile * kDepth; i += 256) {
    // consecutive threads along the contiguous axis
    const int r = o.k == 1 ? i / kDepth : i % kTile, k = o.k == 1 ? i % kDepth : i / kTile;
    const bool in = r0 + r < rows && k0 + k < K;
    dst[k][r] = in ? to_f32(o.p[(r0 + r) * o.outer + (k0 + k) * o.k]) : 0.f;
  }
}

template <typename T>
__device__ __forceinline__ void accumulate(float (&c)[4][4], const Operand<T>& A, const Operand<T>& B, long long m0,
                                           long long M, long long n0, long long N, long long K,
                                           float (*sa)[kTile + 1], float (*sb)[kTile + 1]) {
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  for (long long k0 = 0; k0 < K; k0 += kDepth) {
    load_tile(sa, A, m0, M, k0, K);
    load_tile(sb, B, n0, N, k0, K);
    __syncthreads();
    for (int k = 0; k < kDepth; ++k)
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) c[i][j] = fmaf(sa[k][ty * 4 + i], sb[k][tx * 4 + j], c[i][j]);
    __syncthreads();
  }
}

}  // namespace cocodc_lm_impl
