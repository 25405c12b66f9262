// Norms of queries and keys for each head with the position rotation in the same pass, and its backward pass.
//   n = x / sqrt(mean(x^2) + eps);  z = n w;  y = R(p) z      (R rotates pairs of features by the position's angles)
//   backward:  g = R(-p) dy;  dw = sum g n;  dx = (g w - n mean(g w n)) / sqrt(mean(x^2) + eps)
//
// Bound by memory: 4 bytes per element forward (6 backward).  A lane holds 16 bytes (8 features) of a head, so a warp takes 2
// heads of 128 features (4 of 64) at a time and kSteps of them in flight; cosines, sines and weights of the lane's features
// stay in its registers for all of them.  The sum of squares takes shuffles over the head's lanes; the partner of a feature is
// in the lane itself (neighbours) or in one other lane (halves).  All arithmetic in FP32, one rounding to bf16 at the end.
#include "kv_cache.cuh"

namespace zq {
namespace kv {
namespace {

constexpr int kWarps = 8;
constexpr int kSteps = 4;

struct P {
  const __nv_bfloat16 *x[2], *dy[2];
  __nv_bfloat16* out[2];
  int64_t ldx[2], lddy[2], ldo[2];
  int heads[2], chunks[2];  // of queries and keys; chunks of kSteps x heads-per-warp
  const float* w[2];
  const float* table;
  const int* positions;
  int64_t far, units;
  int rot, neighbours;
  float eps;
  float* partial;
};

__device__ __forceinline__ void unpack8(uint4 v, float* f) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = bf16_lo(w[i]);
    f[2 * i + 1] = bf16_hi(w[i]);
  }
}
__device__ __forceinline__ uint4 pack8(const float* f) {
  return make_uint4(fp8b::pack_bf16(f[0], f[1]), fp8b::pack_bf16(f[2], f[3]), fp8b::pack_bf16(f[4], f[5]), fp8b::pack_bf16(f[6], f[7]));
}
__device__ __forceinline__ void load8(const float* p, float* f) {
  const float4 a = load_chained(reinterpret_cast<const float4*>(p)), b = load_chained(reinterpret_cast<const float4*>(p) + 1);
  f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
}
template <int LANES>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
  for (int o = LANES / 2; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}

// The angles of a lane's 8 features at a token's position.
struct Angles {
  float c[8], s[8];  // halves: of the 8 features; neighbours: of the 4 pairs
  int partner;       // halves: the lane with the other features of the pairs (itself where nothing is rotated)
  bool rotated;
};
template <int LANES>
__device__ __forceinline__ void load_angles(const P& p, int64_t t, int l, int lane, Angles& a) {
  const int pos = load_chained(p.positions + t);
  const bool known = pos >= 0 && pos < p.far;
  const int half = p.rot >> 1;
  a.rotated = l * 8 < p.rot;
  a.partner = lane;
#pragma unroll
  for (int i = 0; i < 8; ++i) a.c[i] = a.s[i] = __uint_as_float(0x7FC00000u);  // a position the table lacks: no angle
  if (!a.rotated) return;
  const float* row = p.table + static_cast<int64_t>(known ? pos : 0) * p.rot;
  if (p.neighbours) {
    if (known) {
      const float4 c = load_chained(reinterpret_cast<const float4*>(row + l * 4));
      const float4 s = load_chained(reinterpret_cast<const float4*>(row + half + l * 4));
      a.c[0] = c.x, a.c[1] = c.y, a.c[2] = c.z, a.c[3] = c.w;
      a.s[0] = s.x, a.s[1] = s.y, a.s[2] = s.z, a.s[3] = s.w;
    }
    return;
  }
  const int hl = half >> 3;  // lanes of half a pair
  const bool second = l >= hl;
  a.partner = second ? lane - hl : lane + hl;
  if (known) {
    load8(row + (second ? l - hl : l) * 8, a.c);
    load8(row + half + (second ? l - hl : l) * 8, a.s);
  }
  if (!second) {
#pragma unroll
    for (int i = 0; i < 8; ++i) a.s[i] = -a.s[i];  // y_a = z_a cos - z_b sin, y_b = z_b cos + z_a sin
  }
}
// Rotation by the angles, or back.  All lanes of the warp take part.
template <bool BACK>
__device__ __forceinline__ void rotate(const P& p, const Angles& a, float* z) {
  if (p.neighbours) {
    if (!a.rotated) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float u = z[2 * i], v = z[2 * i + 1], s = BACK ? -a.s[i] : a.s[i];
      z[2 * i] = u * a.c[i] - v * s;
      z[2 * i + 1] = v * a.c[i] + u * s;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float o = __shfl_sync(0xFFFFFFFFu, z[i], a.partner);
    if (a.rotated) z[i] = z[i] * a.c[i] + o * (BACK ? -a.s[i] : a.s[i]);
  }
}

// Unit u -> token, queries (0) or keys (1), first head.
template <int LANES>
__device__ __forceinline__ void unit_of(const P& p, int64_t u, int64_t& t, int& which, int& h0) {
  const int per = p.chunks[0] + p.chunks[1];
  t = u / per;
  int c = static_cast<int>(u - t * per);
  which = c >= p.chunks[0];
  if (which) c -= p.chunks[0];
  h0 = c * kSteps * (32 / LANES);
}

template <int D>
__global__ void __launch_bounds__(kWarps * 32) norm_rope_kernel(const P p) {
  constexpr int L = D / 8;
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, l = lane % L;
  const int64_t u = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  pdl_wait();
  if (u >= p.units) return;
  int64_t t;
  int which, h0;
  unit_of<L>(p, u, t, which, h0);
  const int heads = p.heads[which];
  const __nv_bfloat16* x = p.x[which] + t * p.ldx[which] + l * 8;
  uint4 v[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int h = h0 + i * (32 / L) + lane / L;
    v[i] = make_uint4(0u, 0u, 0u, 0u);
    if (h < heads) v[i] = load_chained(reinterpret_cast<const uint4*>(x + static_cast<int64_t>(h) * D));
  }
  Angles a;
  load_angles<L>(p, t, l, lane, a);
  float w[8];
  const bool norm = p.w[which] != nullptr;
  if (norm) load8(p.w[which] + l * 8, w);
  __nv_bfloat16* out = p.out[which] + t * p.ldo[which] + l * 8;
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int h = h0 + i * (32 / L) + lane / L;
    float z[8];
    unpack8(v[i], z);
    if (norm) {
      float ss = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(z[e], z[e], ss);
      const float r = rsqrtf(head_sum<L>(ss) * (1.0f / D) + p.eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = z[e] * r * w[e];
    }
    rotate<false>(p, a, z);
    if (h < heads) *reinterpret_cast<uint4*>(out + static_cast<int64_t>(h) * D) = pack8(z);
  }
}

// Warps take units one after the other and sum the weights' gradients of their lanes' features over them, always the same
// units in the same order; a block's sums go to its own place among the partial sums, which norm_grad_sum_kernel adds up.
template <int D>
__global__ void __launch_bounds__(kWarps * 32) norm_rope_backward_kernel(const P p) {
  constexpr int L = D / 8;
  __shared__ float s_dw[kWarps][2][D];
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, l = lane % L, warp = threadIdx.x >> 5;
  float dw[2][8] = {};
  pdl_wait();
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * kWarps + warp; u < p.units; u += static_cast<int64_t>(gridDim.x) * kWarps) {
    int64_t t;
    int which, h0;
    unit_of<L>(p, u, t, which, h0);
    const int heads = p.heads[which];
    const bool norm = p.w[which] != nullptr;
    const __nv_bfloat16* x = p.x[which] + t * p.ldx[which] + l * 8;
    const __nv_bfloat16* dy = p.dy[which] + t * p.lddy[which] + l * 8;
    uint4 v[kSteps], d[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int h = h0 + i * (32 / L) + lane / L;
      v[i] = d[i] = make_uint4(0u, 0u, 0u, 0u);
      if (h < heads) {
        d[i] = load_chained(reinterpret_cast<const uint4*>(dy + static_cast<int64_t>(h) * D));
        if (norm) v[i] = load_chained(reinterpret_cast<const uint4*>(x + static_cast<int64_t>(h) * D));
      }
    }
    Angles a;
    load_angles<L>(p, t, l, lane, a);
    float w[8];
    if (norm) load8(p.w[which] + l * 8, w);
    __nv_bfloat16* out = p.out[which] + t * p.ldo[which] + l * 8;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int h = h0 + i * (32 / L) + lane / L;
      float g[8];
      unpack8(d[i], g);
      rotate<true>(p, a, g);
      if (norm) {
        float z[8], ss = 0.0f, dot = 0.0f;
        unpack8(v[i], z);
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(z[e], z[e], ss);
        const float r = rsqrtf(head_sum<L>(ss) * (1.0f / D) + p.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          z[e] *= r;
          if (h < heads) {
            if (which == 0)
              dw[0][e] = fmaf(g[e], z[e], dw[0][e]);
            else
              dw[1][e] = fmaf(g[e], z[e], dw[1][e]);
          }
          g[e] *= w[e];
          dot = fmaf(g[e], z[e], dot);
        }
        const float mean = head_sum<L>(dot) * (1.0f / D);
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = r * (g[e] - z[e] * mean);
      }
      if (h < heads) *reinterpret_cast<uint4*>(out + static_cast<int64_t>(h) * D) = pack8(g);
    }
  }
  if (!p.partial) return;
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float s = dw[k][e];
#pragma unroll
      for (int o = L; o < 32; o <<= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
      if (lane < L) s_dw[warp][k][l * 8 + e] = s;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * D; i += kWarps * 32) {
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) s += s_dw[k][i / D][i % D];
    p.partial[static_cast<int64_t>(blockIdx.x) * 2 * D + i] = s;
  }
}

// Sums of the blocks' partial sums: a warp per weight (queries' D, then keys'), lanes over the blocks.
__global__ void __launch_bounds__(256) norm_grad_sum_kernel(const float* partial, int blocks, int D, float* dwq, float* dwk) {
  pdl_launch_dependents();
  const int i = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  pdl_wait();
  if (i >= 2 * D) return;
  float s = 0.0f;
  for (int b = lane; b < blocks; b += 32) s += load_chained(partial + static_cast<int64_t>(b) * 2 * D + i);
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  if (lane == 0) (i < D ? dwq : dwk)[i < D ? i : i - D] = s;
}

P params(const NormRopeArgs& a) {
  P p{};
  p.x[0] = static_cast<const __nv_bfloat16*>(a.q), p.x[1] = static_cast<const __nv_bfloat16*>(a.k);
  p.dy[0] = static_cast<const __nv_bfloat16*>(a.dq), p.dy[1] = static_cast<const __nv_bfloat16*>(a.dk);
  p.out[0] = static_cast<__nv_bfloat16*>(a.oq), p.out[1] = static_cast<__nv_bfloat16*>(a.ok);
  p.ldx[0] = a.ldq, p.ldx[1] = a.ldk, p.lddy[0] = a.lddq, p.lddy[1] = a.lddk, p.ldo[0] = a.ldoq, p.ldo[1] = a.ldok;
  p.heads[0] = a.Hq, p.heads[1] = a.H;
  const int per = kSteps * (32 / (a.D / 8));
  p.chunks[0] = (a.Hq + per - 1) / per, p.chunks[1] = (a.H + per - 1) / per;
  p.w[0] = a.wq, p.w[1] = a.wk;
  p.table = a.table, p.positions = a.positions, p.far = a.far;
  p.units = a.T * (p.chunks[0] + p.chunks[1]);
  p.rot = a.rot, p.neighbours = a.neighbours, p.eps = a.eps;
  return p;
}

}  // namespace

int launch_norm_rope(const NormRopeArgs& a, cudaStream_t st) {
  const P p = params(a);
  const int64_t grid = (p.units + kWarps - 1) / kWarps;
  if (grid > 0x7FFFFFFF) return ZQ_ERR_SHAPE;
  const cudaError_t e = launch_chained(a.D == 128 ? norm_rope_kernel<128> : norm_rope_kernel<64>, dim3(static_cast<unsigned>(grid)),
                                       dim3(kWarps * 32), 0, st, false, p);
  count_launch();
  return e == cudaSuccess ? ZQ_OK : ZQ_ERR_CUDA;
}

int launch_norm_rope_backward(const NormRopeArgs& a, cudaStream_t st) {
  P p = params(a);
  if (a.wq) p.partial = a.partial;
  const int64_t want = (p.units + kWarps - 1) / kWarps;
  const int grid = static_cast<int>(want < kNormGradBlocks ? want : kNormGradBlocks);
  cudaError_t e = launch_chained(a.D == 128 ? norm_rope_backward_kernel<128> : norm_rope_backward_kernel<64>, dim3(grid),
                                 dim3(kWarps * 32), 0, st, false, p);
  count_launch();
  if (e != cudaSuccess) return ZQ_ERR_CUDA;
  if (a.wq) {
    e = launch_chained(norm_grad_sum_kernel, dim3(2 * a.D / 8), dim3(256), 0, st, false, a.partial, grid, a.D, a.dwq, a.dwk);
    count_launch();
  }
  return e == cudaSuccess ? ZQ_OK : ZQ_ERR_CUDA;
}

}  // namespace kv
}  // namespace zq
