// Norms of queries and keys for each head with the position rotation in the same pass, and its backward pass.
//   n = x / sqrt(mean(x^2) + eps);  z = n w;  y = R(p) z      (R rotates pairs of features by the position's angles)
//   backward:  g = R(-p) dy;  dw = sum g n;  dx = (g w - n mean(g w n)) / sqrt(mean(x^2) + eps)
//
// Bound by memory: 4 bytes per element forward, 6 backward.  A lane holds 16 bytes (8 features) of a head, so a warp takes 2 heads
// of 128 features (4 of 64) at a time, kSteps of them per unit.  Warps walk over contiguous ranges of units, the next unit's rows
// on their way while one is worked on; a token's angles and weights become two factors per feature that all of its heads share:
//   y = (x c w + x' s' w') / sqrt(..)     (x', w': the feature it is paired with; s' carries the sign)
// The partner's x comes as bf16 pairs from one other lane (halves) or from the lane itself (neighbours).  All arithmetic in FP32, one
// rounding to bf16 at the end.  16384 tokens of 40 heads of 128: without the walk and the shared factors 84 us (32 warps per SM,
// each waiting for its position, then for its angles; half of the issue slots used).
#include "kv_cache.cuh"

namespace zq {
namespace kv {
namespace {

constexpr int kWarps = 8;
constexpr int kSteps = 4;
constexpr int kBackSteps = 2;       // in flight at a time, backward
constexpr int kForwardBlocks = 3;   // per SM: 24 warps with the registers that a unit ahead needs
constexpr int kBackwardBlocks = 3;

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

// A unit: token, chunk of it; queries (0) or keys (1), first head.  Divisions only for a warp's first one.
struct Unit {
  int64_t t;
  int c, which, h0;
};
template <int LANES>
__device__ __forceinline__ void place(const P& p, Unit& n) {
  n.which = n.c >= p.chunks[0];
  n.h0 = (n.which ? n.c - p.chunks[0] : n.c) * kSteps * (32 / LANES);
}
template <int LANES>
__device__ __forceinline__ Unit first_unit(const P& p, int64_t u) {
  const int per = p.chunks[0] + p.chunks[1];
  Unit n;
  n.t = u / per;
  n.c = static_cast<int>(u - n.t * per);
  place<LANES>(p, n);
  return n;
}
template <int LANES>
__device__ __forceinline__ Unit next_unit(const P& p, Unit n) {
  if (++n.c == p.chunks[0] + p.chunks[1]) {
    n.c = 0;
    ++n.t;
  }
  place<LANES>(p, n);
  return n;
}
// A warp's units: contiguous, as even as can be.
__device__ __forceinline__ void range_of(const P& p, int64_t& u0, int64_t& u1) {
  const int64_t warps = static_cast<int64_t>(gridDim.x) * kWarps, w = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  const int64_t each = p.units / warps, rest = p.units % warps;
  u0 = w * each + (w < rest ? w : rest);
  u1 = u0 + each + (w < rest ? 1 : 0);
}
template <int D>
__device__ __forceinline__ void load_rows(const __nv_bfloat16* x, int64_t ld, const Unit& n, int heads, int lane, uint4* v) {
  constexpr int L = D / 8;
  const __nv_bfloat16* from = x + n.t * ld + (lane % L) * 8;
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int h = n.h0 + i * (32 / L) + lane / L;
    v[i] = make_uint4(0u, 0u, 0u, 0u);
    if (h < heads) v[i] = load_chained(reinterpret_cast<const uint4*>(from + static_cast<int64_t>(h) * D));
  }
}

// Cosines and sines for a lane's 8 features at position `pos` (NaN where the table lacks it), the sine's sign as the forward pass has
// it; 1 and 0 where nothing is rotated.  `partner`: the lane of the paired features (halves).
template <int LANES>
__device__ __forceinline__ void load_angles(const P& p, int pos, int l, int lane, float* c, float* s, int& partner) {
  const bool known = pos >= 0 && pos < p.far;
  const int half = p.rot >> 1;
  const float* row = p.table + static_cast<int64_t>(known ? pos : 0) * p.rot;
  partner = lane;
  if (l * 8 >= p.rot) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = 1.0f, s[i] = 0.0f;
    return;
  }
  if (p.neighbours) {
    const float4 a = load_chained(reinterpret_cast<const float4*>(row + l * 4)), b = load_chained(reinterpret_cast<const float4*>(row + half + l * 4));
    c[0] = c[1] = a.x, c[2] = c[3] = a.y, c[4] = c[5] = a.z, c[6] = c[7] = a.w;
    s[0] = -b.x, s[1] = b.x, s[2] = -b.y, s[3] = b.y, s[4] = -b.z, s[5] = b.z, s[6] = -b.w, s[7] = b.w;
  } else {
    const int hl = half >> 3;  // lanes of one half
    const bool second = l >= hl;
    partner = second ? lane - hl : lane + hl;
    load8(row + (second ? l - hl : l) * 8, c);
    load8(row + half + (second ? l - hl : l) * 8, s);
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = second ? s[i] : -s[i];
  }
  if (!known) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = s[i] = __uint_as_float(0x7FC00000u);
  }
}
// The paired features of 8, as bf16 pairs.  All lanes of the warp take part.
__device__ __forceinline__ uint4 paired(const P& p, uint4 v, int partner, bool rotated) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    w[i] = p.neighbours ? __byte_perm(w[i], 0u, 0x1032) : __shfl_sync(0xFFFFFFFFu, w[i], partner);
    if (!rotated) w[i] = 0u;  // (times a sine of zero: an infinity must not become NaN)
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// The weights of the paired features.
__device__ __forceinline__ void paired_weights(const P& p, const float* w, int partner, float* wp) {
#pragma unroll
  for (int i = 0; i < 8; ++i) wp[i] = p.neighbours ? w[i ^ 1] : __shfl_sync(0xFFFFFFFFu, w[i], partner);
}

template <int D>
__global__ void __launch_bounds__(kWarps * 32, kForwardBlocks) norm_rope_kernel(const P p) {
  constexpr int L = D / 8;
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, l = lane % L;
  const bool rotated = l * 8 < p.rot, norm = p.w[0] != nullptr;
  int64_t u, end;
  range_of(p, u, end);
  pdl_wait();
  if (u >= end) return;
  Unit n = first_unit<L>(p, u);
  int pos = load_chained(p.positions + n.t), partner = lane;
  uint4 v[kSteps];
  load_rows<D>(p.x[n.which], p.ldx[n.which], n, p.heads[n.which], lane, v);
  bool fresh = true;   // another token or kind: other factors
  float wc[8], ws[8];  // of the feature and of the one paired with it
  for (; u < end; ++u) {
    if (fresh) {
      load_angles<L>(p, pos, l, lane, wc, ws, partner);
      if (norm) {
        float w[8], wp[8];
        load8(p.w[n.which] + l * 8, w);
        paired_weights(p, w, partner, wp);
#pragma unroll
        for (int e = 0; e < 8; ++e) wc[e] *= w[e], ws[e] *= wp[e];
      }
      if (!rotated) {
#pragma unroll
        for (int e = 0; e < 8; ++e) ws[e] = -0.0f;  // -0 is added to what passes: adding +0 would turn a -0 into +0
      }
    }
    Unit next = n;
    uint4 ahead[kSteps];
    if (u + 1 < end) {
      next = next_unit<L>(p, n);
      if (next.t != n.t) pos = load_chained(p.positions + next.t);
      load_rows<D>(p.x[next.which], p.ldx[next.which], next, p.heads[next.which], lane, ahead);
    }
    __nv_bfloat16* out = p.out[n.which] + n.t * p.ldo[n.which] + l * 8;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int h = n.h0 + i * (32 / L) + lane / L;
      float z[8], y[8];
      unpack8(paired(p, v[i], partner, rotated), y);
      unpack8(v[i], z);
      float r = 1.0f;
      if (norm) {
        float ss = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(z[e], z[e], ss);
        r = rsqrtf(head_sum<L>(ss) * (1.0f / D) + p.eps);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = r * fmaf(z[e], wc[e], y[e] * ws[e]);
      if (h < p.heads[n.which]) *reinterpret_cast<uint4*>(out + static_cast<int64_t>(h) * D) = pack8(y);
    }
    fresh = next.t != n.t || next.which != n.which;
    n = next;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) v[i] = ahead[i];
  }
}

// Warps sum the weights' gradients of their lanes' features over their units, always the same ones in the same order; a block's sums
// go to its own place among the partial sums, which norm_grad_sum_kernel adds up.
template <int D>
__global__ void __launch_bounds__(kWarps * 32, kBackwardBlocks) norm_rope_backward_kernel(const P p) {
  constexpr int L = D / 8;
  __shared__ float s_dw[kWarps][2][D];
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, l = lane % L, warp = threadIdx.x >> 5;
  const bool rotated = l * 8 < p.rot, norm = p.w[0] != nullptr;
  float dw[8] = {};  // of the kind at hand; on a change of kind it goes to shared memory
  int64_t u, end;
  range_of(p, u, end);
  if (norm)
    for (int i = lane; i < 2 * D; i += 32) s_dw[warp][i / D][i % D] = 0.0f;
  __syncwarp();
  auto settle = [&](int which) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float v = dw[e];
#pragma unroll
      for (int o = L; o < 32; o <<= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
      if (lane < L) s_dw[warp][which][l * 8 + e] += v;
      dw[e] = 0.0f;
    }
  };
  pdl_wait();
  if (u < end) {
    Unit n = first_unit<L>(p, u);
    int pos = load_chained(p.positions + n.t), partner = lane;
    uint4 d[kBackSteps], v[kBackSteps];
    bool fresh = true;
    float c[8], s[8], w[8];
    for (; u < end; ++u) {
      const int heads = p.heads[n.which];
      if (fresh) {
        load_angles<L>(p, pos, l, lane, c, s, partner);
        if (norm) load8(p.w[n.which] + l * 8, w);
      }
      Unit next = n;
      if (u + 1 < end) {
        next = next_unit<L>(p, n);
        if (next.t != n.t) pos = load_chained(p.positions + next.t);
      }
      const __nv_bfloat16* x = p.x[n.which] + n.t * p.ldx[n.which] + l * 8;
      const __nv_bfloat16* dy = p.dy[n.which] + n.t * p.lddy[n.which] + l * 8;
      __nv_bfloat16* out = p.out[n.which] + n.t * p.ldo[n.which] + l * 8;
#pragma unroll
      for (int i0 = 0; i0 < kSteps; i0 += kBackSteps) {
#pragma unroll
        for (int i = 0; i < kBackSteps; ++i) {
          const int h = n.h0 + (i0 + i) * (32 / L) + lane / L;
          v[i] = d[i] = make_uint4(0u, 0u, 0u, 0u);
          if (h < heads) {
            d[i] = load_chained(reinterpret_cast<const uint4*>(dy + static_cast<int64_t>(h) * D));
            if (norm) v[i] = load_chained(reinterpret_cast<const uint4*>(x + static_cast<int64_t>(h) * D));
          }
        }
#pragma unroll
        for (int i = 0; i < kBackSteps; ++i) {
          const int h = n.h0 + (i0 + i) * (32 / L) + lane / L;
          float g[8], y[8];
          unpack8(paired(p, d[i], partner, rotated), y);
          unpack8(d[i], g);
#pragma unroll
          for (int e = 0; e < 8; ++e) g[e] = fmaf(g[e], c[e], -y[e] * s[e]);  // by the opposite angle
          if (norm) {
            float z[8], ss = 0.0f, dot = 0.0f;
            unpack8(v[i], z);
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(z[e], z[e], ss);
            const float square = head_sum<L>(ss) * (1.0f / D) + p.eps;
            const float r = h < heads ? rsqrtf(square) : 0.0f;  // (where there is no head it need not be a number: eps may be 0)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              z[e] *= r;
              dw[e] = fmaf(g[e], z[e], dw[e]);  // (zeros where there is no head)
              g[e] *= w[e];
              dot = fmaf(g[e], z[e], dot);
            }
            const float mean = head_sum<L>(dot) * (1.0f / D);
#pragma unroll
            for (int e = 0; e < 8; ++e) g[e] = r * fmaf(-z[e], mean, g[e]);
          }
          if (h < heads) *reinterpret_cast<uint4*>(out + static_cast<int64_t>(h) * D) = pack8(g);
        }
      }
      fresh = next.t != n.t || next.which != n.which;
      if (norm && (next.which != n.which || u + 1 == end)) settle(n.which);
      n = next;
    }
  }
  if (!norm) return;
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * D; i += kWarps * 32) {
    float v = 0.0f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) v += s_dw[k][i / D][i % D];
    p.partial[static_cast<int64_t>(blockIdx.x) * 2 * D + i] = v;
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
  const int64_t want = (p.units + kWarps - 1) / kWarps, room = static_cast<int64_t>(kForwardBlocks) * sm_count();
  const cudaError_t e = launch_chained(a.D == 128 ? norm_rope_kernel<128> : norm_rope_kernel<64>,
                                       dim3(static_cast<unsigned>(want < room ? want : room)), dim3(kWarps * 32), 0, st, false, p);
  count_launch();
  return e == cudaSuccess ? ZQ_OK : ZQ_ERR_CUDA;
}

int launch_norm_rope_backward(const NormRopeArgs& a, cudaStream_t st) {
  P p = params(a);
  if (a.wq) p.partial = a.partial;
  int64_t grid = (p.units + kWarps - 1) / kWarps;
  const int64_t room = static_cast<int64_t>(kBackwardBlocks) * sm_count();
  if (grid > room) grid = room;
  if (grid > kNormGradBlocks) grid = kNormGradBlocks;
  cudaError_t e = launch_chained(a.D == 128 ? norm_rope_backward_kernel<128> : norm_rope_backward_kernel<64>, dim3(static_cast<unsigned>(grid)),
                                 dim3(kWarps * 32), 0, st, false, p);
  count_launch();
  if (e != cudaSuccess) return ZQ_ERR_CUDA;
  if (a.wq) {
    e = launch_chained(norm_grad_sum_kernel, dim3(2 * a.D / 8), dim3(256), 0, st, false, a.partial, static_cast<int>(grid), a.D, a.dwq, a.dwk);
    count_launch();
  }
  return e == cudaSuccess ? ZQ_OK : ZQ_ERR_CUDA;
}

}  // namespace kv
}  // namespace zq
