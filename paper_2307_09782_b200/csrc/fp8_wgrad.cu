// Weight gradient from an 8-bit activation checkpoint: dW[n, k] = sum_m G[m, n] * (code[m, k] * s[k / 128, m]).
//
// Plain tiled kernel on the CUDA cores: 64 x 64 outputs per CTA, 16 tokens at a time through shared memory,
// 4 x 4 outputs per thread.
#include "fp8_block.cuh"

namespace zq {
namespace fp8b {
namespace {

constexpr int kT = 64, kTok = 16;

__global__ void __launch_bounds__(256)
wgrad_simple_kernel(const __nv_bfloat16* __restrict__ g, int64_t ldg, int64_t g_stride, const uint8_t* __restrict__ q,
                    const float* __restrict__ s, int64_t M, int64_t N, int64_t K, void* __restrict__ dw, int dwdt) {
  __shared__ float s_g[kTok][kT], s_x[kTok][kT];
  const int64_t n0 = static_cast<int64_t>(blockIdx.y) * kT, k0 = static_cast<int64_t>(blockIdx.x) * kT;
  g += blockIdx.z * g_stride;
  const int tn = threadIdx.x >> 4, tk = threadIdx.x & 15;
  float acc[4][4] = {};
  for (int64_t m0 = 0; m0 < M; m0 += kTok) {
    for (int i = threadIdx.x; i < kTok * kT; i += 256) {
      const int r = i / kT, c = i % kT;
      const int64_t m = m0 + r;
      s_g[r][c] = m < M && n0 + c < N ? __bfloat162float(g[m * ldg + n0 + c]) : 0.0f;
      float v = 0.0f;
      if (m < M && k0 + c < K)
        v = __bfloat162float(__float2bfloat16_rn(decode2(q[m * K + k0 + c]).x * s[((k0 + c) / kBlk) * M + m]));
      s_x[r][c] = v;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kTok; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(s_g[r][tn * 4 + i], s_x[r][tk * 4 + j], acc[i][j]);
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int64_t n = n0 + tn * 4 + i, k = k0 + tk * 4 + j;
      if (n < N && k < K) {
        const int64_t o = (blockIdx.z * N + n) * K + k;
        if (dwdt == ZQ_OUT_F32)
          static_cast<float*>(dw)[o] = acc[i][j];
        else
          static_cast<__nv_bfloat16*>(dw)[o] = __float2bfloat16_rn(acc[i][j]);
      }
    }
}

}  // namespace

int launch_wgrad(const WgradArgs& a, cudaStream_t st) {
  const dim3 grid(static_cast<unsigned>((a.K + kT - 1) / kT), static_cast<unsigned>((a.N + kT - 1) / kT),
                  static_cast<unsigned>(a.parts));
  if (grid.y > 65535) return ZQ_ERR_SHAPE;
  wgrad_simple_kernel<<<grid, 256, 0, st>>>(static_cast<const __nv_bfloat16*>(a.g), a.ldg, a.g_stride, a.q, a.s, a.M,
                                            a.N, a.K, a.dw, a.dwdt);
  count_launch();
  return cudaGetLastError() == cudaSuccess ? ZQ_OK : ZQ_ERR_CUDA;
}

}  // namespace fp8b
}  // namespace zq
