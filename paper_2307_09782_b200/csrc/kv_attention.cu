// Attention over the 8-bit cache: o = softmax(scale q k^T + mask) v.
#include "kv_attention.cuh"

namespace zq {
namespace kv {
namespace {

// One warp per row (token and query head), one pass over the keys with a running maximum and sum.
template <int D, bool F32>
__global__ void __launch_bounds__(256) attention_row_kernel(const AttnArgs a) {
  constexpr int E = D / 32;
  const Cache& c = a.c;
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const int64_t task = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
  pdl_wait();
  const int64_t t = task / a.Hq;
  const int hq = static_cast<int>(task % a.Hq);
  if (t >= c.T) return;
  const int b = c.cu ? unit_sequence(t, c.B, 1, 0, [&](int j) { return static_cast<int64_t>(load_chained(c.cu + j)); }) : static_cast<int>(t);
  int first, n;
  rows_of(c, b, first, n);
  if (t < first || t >= first + n) return;
  if (static_cast<int64_t>(n) * (a.Hq / c.H) <= kFewRows) return;
  const int L = max(load_chained(c.lens + b), 0);
  const int pos = L - n + static_cast<int>(t - first);
  const int hi = a.causal ? min(L, pos + 1) : L;
  const int lo = a.causal && a.window > 0 ? max(0, pos + 1 - a.window) : 0;
  const int h = hq / (a.Hq / c.H);
  const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.q) + t * a.ldq + static_cast<int64_t>(hq) * D;
  float qf[E], o[E] = {};
  for (int e = 0; e < E; ++e) qf[e] = __bfloat162float(q[lane * E + e]) * a.sm_scale;
  float m = -INFINITY, l = 0.0f;
  for (int p = lo; p < hi; ++p) {
    const int page = page_of(c, b, p / c.page);
    const int64_t kb = block_at(c, max(page, 0), 0, h), vb = kb + c.H;
    const int64_t in = static_cast<int64_t>(p % c.page) * D + lane * E;
    const uint8_t* kc = c.codes + kb * c.page * D + in;
    const uint8_t* vc = c.codes + vb * c.page * D + in;
    float s = 0.0f, vf[E];
    for (int e = 0; e < E; e += 2) {
      const float2 kk = fp8b::decode2(*reinterpret_cast<const uint16_t*>(kc + e)), vv = fp8b::decode2(*reinterpret_cast<const uint16_t*>(vc + e));
      s = fmaf(kk.x, qf[e], fmaf(kk.y, qf[e + 1], s));
      vf[e] = vv.x, vf[e + 1] = vv.y;
    }
    for (int x = 16; x; x >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, x);
    s *= page < 0 ? NAN : load_chained(c.scale + kb);
    const float vs = load_chained(c.scale + vb);
    const float mn = fmaxf(m, s), f = __expf(m - mn), w = __expf(s - mn);
    l = l * f + w;
    for (int e = 0; e < E; ++e) o[e] = o[e] * f + w * vs * vf[e];
    m = mn;
  }
  for (int e = 0; e < E; ++e) {
    const float r = hi > lo ? o[e] / l : 0.0f;
    const int64_t at = t * a.ldo + static_cast<int64_t>(hq) * D + lane * E + e;
    if (F32)
      static_cast<float*>(a.out)[at] = r;
    else
      static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(r);
  }
  if (a.lse && lane == 0) a.lse[t * a.Hq + hq] = hi > lo ? m + logf(l) : -INFINITY;
}

}  // namespace

int launch_attention(const AttnArgs& a, cudaStream_t st) {
  const int G = a.Hq / a.c.H;
  if (G <= kFewRows) {
    const int64_t most = a.c.cu ? (a.c.T * G < kFewRows ? a.c.T * G : kFewRows) : G;
    if (int e = launch_attention_few(a, static_cast<int>(most), st)) return e;
    if (!a.c.cu) return ZQ_OK;
  }
  const int64_t grid = (a.c.T * a.Hq + 7) / 8;
  if (grid > 0x7FFFFFFF) return ZQ_ERR_SHAPE;
  auto kernel = a.c.D == 128 ? (a.dt == ZQ_OUT_F32 ? attention_row_kernel<128, true> : attention_row_kernel<128, false>)
                             : (a.dt == ZQ_OUT_F32 ? attention_row_kernel<64, true> : attention_row_kernel<64, false>);
  const cudaError_t e = launch_chained(kernel, dim3(static_cast<unsigned>(grid)), dim3(256), 0, st, false, a);
  count_launch();
  return e == cudaSuccess ? ZQ_OK : ZQ_ERR_CUDA;
}

}  // namespace kv
}  // namespace zq
