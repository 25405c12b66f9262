// Quantizers of the FP8 operators with block scales: activations (one scale per row and 128 input features),
// weights (one per 128 x 128), and the transposed copy of quantized weights that gradients read.
//
// What they move: 3 bytes per element for activations (2 read, 1 written, plus 1/32 for the scale), 5 for weights, 2 for the
// transposition; the latter two run once per weight, or once per optimizer step.  Measured, us, caches cold, with the launch
// (about 6): activations 1 x 4096 6.1, 2048 x 4096 12.3, 8192 x 7168 42 (4.2 TB/s), 8192 x 28672 139 (5.1 TB/s, 0.78 of the copy
// rate); weights 11008 x 4096 48 (4.7 TB/s), 28672 x 7168 167 (6.2 TB/s, 0.94); transposition 11008 x 4096 36, 28672 x 7168 123
// (3.3 TB/s, 0.51: 16-byte stores, each lane to another row).
#include "fp8_block.cuh"

namespace zq {
namespace fp8b {
namespace {

constexpr int kQuantThreads = 256;
constexpr int kQuantGroups = kQuantThreads / 16;

// 16 lanes take one block: 16 bytes of x per lane, the maximum by four shuffles, 8 codes per lane.  A group takes U
// neighbouring blocks of its row with all loads in flight before the first reduction; neighbouring groups take
// neighbouring rows, so that their scales (stored with the row index innermost) share sectors.
template <int U>
__global__ void __launch_bounds__(kQuantThreads)
quantize_block_kernel(const __nv_bfloat16* x, int M, int K, int64_t ldx, int kblocks, bool pow2, uint8_t* q, float* s) {
  pdl_launch_dependents();
  const int64_t task = static_cast<int64_t>(blockIdx.x) * kQuantGroups + (threadIdx.x >> 4);
  const int lane = threadIdx.x & 15;
  const int64_t m = task % M;
  const int kb0 = static_cast<int>(task / M) * U;
  const bool row_ok = kb0 < kblocks;  // m < M always
  const __nv_bfloat16* xr = x + m * ldx;
  uint4 v[U];
  pdl_wait();
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int k = (kb0 + u) * kBlk + lane * 8;
    v[u] = make_uint4(0u, 0u, 0u, 0u);
    if (row_ok && k < K) v[u] = load_chained(reinterpret_cast<const uint4*>(xr + k));
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
    uint32_t a = 0u;  // the bf16 pattern in the upper half: comparing with the sign off orders like the values
#pragma unroll
    for (int i = 0; i < 4; ++i) a = max(a, max((w[i] << 16) & 0x7FFF0000u, w[i] & 0x7FFF0000u));
#pragma unroll
    for (int o = 8; o; o >>= 1) a = max(a, __shfl_xor_sync(0xFFFFFFFFu, a, o));
    const float sc = block_scale(a, pow2), inv = block_inv(sc);
    const int kb = kb0 + u, k = kb * kBlk + lane * 8;
    if (row_ok && k < K) *reinterpret_cast<uint2*>(q + m * K + k) = cast8(v[u], inv);
    if (row_ok && kb < kblocks && lane == 0) s[static_cast<int64_t>(kb) * M + m] = sc;
  }
}

// One CTA per 128 x 128 block, kept in registers between the maximum and the cast.
__global__ void __launch_bounds__(256)
quantize_weight_block_kernel(const float* __restrict__ w, int64_t N, int64_t K, int64_t kblocks, bool pow2,
                             uint8_t* __restrict__ q, float* __restrict__ s) {
  __shared__ uint32_t s_max[8];
  const int64_t nb = blockIdx.x / kblocks, kb = blockIdx.x % kblocks;
  const int row = threadIdx.x >> 5, lane = threadIdx.x & 31;  // a warp takes a row of 128, 8 rows at a time
  const int64_t k = kb * kBlk + lane * 4;
  float4 v[16];
  uint32_t a = 0u;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int64_t n = nb * kBlk + i * 8 + row;
    v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (n < N && k < K) v[i] = __ldg(reinterpret_cast<const float4*>(w + n * K + k));
    a = max(a, max(max(abs_bits(v[i].x), abs_bits(v[i].y)), max(abs_bits(v[i].z), abs_bits(v[i].w))));
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) a = max(a, __shfl_xor_sync(0xFFFFFFFFu, a, o));
  if (lane == 0) s_max[row] = a;
  __syncthreads();
  a = s_max[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) a = max(a, s_max[i]);
  const float sc = block_scale(a, pow2), inv = block_inv(sc);
  if (threadIdx.x == 0) s[blockIdx.x] = sc;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int64_t n = nb * kBlk + i * 8 + row;
    if (n < N && k < K) *reinterpret_cast<uint32_t*>(q + n * K + k) = cast4(v[i].x, v[i].y, v[i].z, v[i].w, inv);
  }
}

// 128 x 128 tile through shared memory: 16-byte loads along K, 16-byte stores along N.
__global__ void __launch_bounds__(256)
transpose_weight_block_kernel(const uint8_t* __restrict__ q, const float* __restrict__ s, int64_t N, int64_t K,
                              int64_t nblocks, int64_t kblocks, uint8_t* __restrict__ qt, float* __restrict__ st) {
  __shared__ uint8_t t[kBlk][kBlk + 4];
  const int64_t nb = blockIdx.x / kblocks, kb = blockIdx.x % kblocks;
  if (threadIdx.x == 0) st[kb * nblocks + nb] = s[blockIdx.x];
  for (int i = threadIdx.x; i < kBlk * 8; i += 256) {
    const int r = i >> 3, c = (i & 7) * 16;
    const int64_t n = nb * kBlk + r, k = kb * kBlk + c;
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (n < N && k < K) v = __ldg(reinterpret_cast<const uint4*>(q + n * K + k));
    uint32_t* d = reinterpret_cast<uint32_t*>(&t[r][c]);
    d[0] = v.x;
    d[1] = v.y;
    d[2] = v.z;
    d[3] = v.w;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < kBlk * 8; i += 256) {
    const int c = i & (kBlk - 1), r = (i >> 7) * 16;  // output row k = c, 16 consecutive n from r on
    const int64_t k = kb * kBlk + c, n = nb * kBlk + r;
    if (k < K && n < N) {  // N is a multiple of 16: the 16 are inside or outside together
      uint32_t o[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        o[j] = t[r + 4 * j][c] | (t[r + 4 * j + 1][c] << 8) | (t[r + 4 * j + 2][c] << 16) |
               (static_cast<uint32_t>(t[r + 4 * j + 3][c]) << 24);
      *reinterpret_cast<uint4*>(qt + k * N + n) = make_uint4(o[0], o[1], o[2], o[3]);
    }
  }
}

inline int launched(cudaError_t e) {
  count_launch();
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? ZQ_OK : ZQ_ERR_CUDA;
}

}  // namespace

int launch_quantize_block(const void* x, int64_t M, int64_t K, int64_t ldx, int mode, uint8_t* q, float* s,
                          cudaStream_t st) {
  const int64_t kb = blocks_of(K);
  // four blocks per group once every SM has work that way, one below
  const bool wide = M * kb >= 4 * static_cast<int64_t>(kQuantGroups) * sm_count() * 2;
  const int u = wide ? 4 : 1;
  const int64_t tasks = M * ((kb + u - 1) / u), ctas = (tasks + kQuantGroups - 1) / kQuantGroups;
  if (ctas > 0x7FFFFFFF) return ZQ_ERR_SHAPE;
  return launched(launch_chained(wide ? quantize_block_kernel<4> : quantize_block_kernel<1>,
                                 dim3(static_cast<unsigned>(ctas)), dim3(kQuantThreads), 0, st, false,
                                 static_cast<const __nv_bfloat16*>(x), static_cast<int>(M), static_cast<int>(K), ldx,
                                 static_cast<int>(kb), mode == ZQ_SCALE_M1, q, s));
}

int launch_quantize_weight_block(const float* w, int64_t N, int64_t K, int mode, uint8_t* q, float* s, cudaStream_t st) {
  const int64_t kb = blocks_of(K), ctas = blocks_of(N) * kb;
  if (ctas > 0x7FFFFFFF) return ZQ_ERR_SHAPE;
  quantize_weight_block_kernel<<<static_cast<unsigned>(ctas), 256, 0, st>>>(w, N, K, kb, mode == ZQ_SCALE_M1, q, s);
  return launched(cudaSuccess);
}

int launch_transpose_weight_block(const uint8_t* q, const float* s, int64_t N, int64_t K, uint8_t* qt, float* st_,
                                  cudaStream_t st) {
  const int64_t nb = blocks_of(N), kb = blocks_of(K);
  if (nb * kb > 0x7FFFFFFF) return ZQ_ERR_SHAPE;
  transpose_weight_block_kernel<<<static_cast<unsigned>(nb * kb), 256, 0, st>>>(q, s, N, K, nb, kb, qt, st_);
  return launched(cudaSuccess);
}

}  // namespace fp8b
}  // namespace zq
