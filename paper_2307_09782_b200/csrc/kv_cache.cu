// The 8-bit cache of keys and values: new tokens are quantized as they are written into their pages, and read back.
//
// Both are bound by memory: 3 bytes per element (2 read, 1 written; reading back 1 + 2 or 1 + 4).
#include <climits>

#include "kv_cache.cuh"

namespace zq {
namespace kv {
namespace {

// The first sequence that owns unit u, found by all threads of the block at once; -1 where none does.
template <int THREADS>
__device__ __forceinline__ int block_sequence(const Cache& c, int64_t u, int extra, int* shared) {
  if (threadIdx.x == 0) *shared = INT_MAX;
  __syncthreads();
  const int b = unit_sequence(u, c.B, c.page, extra, [&](int i) { return load_chained(c.cu + i); }, c.T, threadIdx.x, THREADS);
  if (b >= 0) atomicMin(shared, b);
  __syncthreads();
  return *shared == INT_MAX ? -1 : *shared;
}

// ---- writing ------------------------------------------------------------------------------------------------------
// A CTA takes a page that a sequence writes to, and some of its blocks (keys or values, head), one per team of N threads at a time:
// the block's new rows are in the team's registers between the maximum and the cast, 32 elements per thread, so they are
// read once.  Where the block had been begun before and its scale has to grow, the team rounds the codes there to the new scale.
// Which page it is, and whose, takes four dependent loads, once per CTA (3.5 us: with one block per CTA and the sequence found by
// bisection, 180 sequences of up to 27 tokens and 64 blocks took 331 us).
constexpr int kVec = 4;  // 16-byte pieces per thread

template <int N, int THREADS>
__global__ void __launch_bounds__(THREADS)
write_kernel(const Cache c, const __nv_bfloat16* k, int64_t ldk, const __nv_bfloat16* v, int64_t ldv, bool pow2, int per_cta) {
  __shared__ uint32_t s_max[2][THREADS / 32];
  __shared__ int s_b;
  pdl_launch_dependents();
  constexpr int kTeams = THREADS / N;
  const int team = threadIdx.x / N, i = threadIdx.x % N, warp = threadIdx.x >> 5;
  const int64_t u = blockIdx.x;
  pdl_wait();
  // the unit's sequence, page and rows r0 .. r1 - 1 of it; the blocks are begun here where r0 is 0
  const int b = c.cu ? block_sequence<THREADS>(c, u, 2, &s_b) : static_cast<int>(u);
  if (b < 0) return;
  int first, n;
  rows_of(c, b, first, n);
  const int pos0 = load_chained(c.lens + b) - n;  // of the sequence's first new token
  const int64_t at = c.cu ? u - unit_base(first, b, c.page, 2) : 0;
  if (n <= 0 || pos0 < 0 || at < 0 || at * c.page >= (pos0 % c.page) + static_cast<int64_t>(n)) return;
  const int64_t pi = pos0 / c.page + at;
  const int64_t lo = max(static_cast<int64_t>(pos0), pi * c.page), hi = min(static_cast<int64_t>(pos0) + n, (pi + 1) * c.page);
  const int r0 = static_cast<int>(lo - pi * c.page), r1 = static_cast<int>(hi - pi * c.page);
  const int64_t row = first + (lo - pos0);  // of the tensors, at r0
  const int page = page_of(c, b, static_cast<int>(pi));
  if (page < 0) return;
  const int lanes = c.D / 8, col = (i % lanes) * 8, rows = N / lanes;
  for (int it = 0; it < per_cta; ++it) {
    const int task = (blockIdx.y * per_cta + it) * kTeams + team;
    const bool mine = task < 2 * c.H;
    const int which = mine && task >= c.H, h = mine ? task - which * c.H : 0;
    const __nv_bfloat16* src = (which ? v + row * ldv : k + row * ldk) + static_cast<int64_t>(h) * c.D + col;
    const int64_t ld = which ? ldv : ldk;
    uint4 x[kVec];
    uint32_t amax = 0u;
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int r = i / lanes + j * rows;
      x[j] = make_uint4(0u, 0u, 0u, 0u);
      if (mine && r >= r0 && r < r1) x[j] = load_chained(reinterpret_cast<const uint4*>(src + (r - r0) * ld));
    }
    const int64_t block = block_at(c, page, which, h);
    const float old = mine && r0 > 0 ? load_chained(c.scale + block) : 0.0f;  // 0: begun here
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const uint32_t w[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) amax = max(amax, max((w[e] << 16) & 0x7FFF0000u, w[e] & 0x7FFF0000u));
    }
    amax = __reduce_max_sync(0xFFFFFFFFu, amax);
    if (N > 32) {
      if ((threadIdx.x & 31) == 0) s_max[it & 1][warp] = amax;
      __syncthreads();  // (behind it every thread has read the old scale as well)
#pragma unroll
      for (int j = 0; j < N / 32; ++j) amax = max(amax, s_max[it & 1][team * (N / 32) + j]);
    }
    float s = cache_scale(amax, pow2);
    const bool grown = !(s <= old);  // also where s is not a number
    if (!grown || isnan(old)) s = old;
    if (!mine) continue;
    const bool bad = isnan(s);
    const float inv = fp8b::block_inv(s);
    uint8_t* dst = c.codes + (block * c.page) * c.D + col;
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      const int r = i / lanes + j * rows;
      uint2* q = reinterpret_cast<uint2*>(dst + static_cast<int64_t>(r) * c.D);
      if (r >= r0 && r < r1) {
        *q = bad ? make_uint2(0u, 0u) : cast8(x[j], inv);
      } else if (r < r0 && grown) {
        const uint2 was = load_chained(q);
        uint32_t o[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t w = e ? was.y : was.x;
          const float2 lo2 = fp8b::decode2(static_cast<uint16_t>(w)), hi2 = fp8b::decode2(static_cast<uint16_t>(w >> 16));
          o[e] = fp8b::cast4(__fmul_rn(lo2.x, old), __fmul_rn(lo2.y, old), __fmul_rn(hi2.x, old), __fmul_rn(hi2.y, old), inv);
        }
        *q = bad ? make_uint2(0u, 0u) : make_uint2(o[0], o[1]);
      }
    }
    if (i == 0) c.scale[block] = s;
  }
}

// ---- reading back ---------------------------------------------------------------------------------------------------
// A CTA takes a page and some of its heads, for keys or values; pieces of V codes, whose results are 16 bytes, kReadVec of them in
// flight per thread.  (With 4 KB of codes per CTA, behind the loads that tell which page it is, 16 caches of up to 4095 tokens
// took 270 us in FP32.)
constexpr int kReadThreads = 256, kReadVec = 8, kReadHeads = 16;

template <int D, bool F32>
__global__ void __launch_bounds__(kReadThreads) read_kernel(const Cache c, void* k, void* v, int per_cta, int page_bits) {
  constexpr int V = F32 ? 4 : 8, kPerRow = D / V;
  __shared__ float s_scale[kReadHeads];
  __shared__ int s_b;
  pdl_launch_dependents();
  const int64_t u = blockIdx.x;
  const int which = blockIdx.z, h0 = blockIdx.y * per_cta, heads = min(per_cta, c.H - h0);
  pdl_wait();
  const int b = block_sequence<kReadThreads>(c, u, 1, &s_b);
  if (b < 0) return;
  int first, n;
  rows_of(c, b, first, n);
  const int64_t pi = u - unit_base(first, b, c.page, 1);
  if (pi < 0 || pi * c.page >= n) return;
  const int page = page_of(c, b, static_cast<int>(pi));
  const int rows = min(c.page, n - static_cast<int>(pi) * c.page);
  const int64_t block0 = block_at(c, max(page, 0), which, h0);
  if (threadIdx.x < heads) s_scale[threadIdx.x] = page < 0 ? __uint_as_float(0x7FC00000u) : load_chained(c.scale + block0 + threadIdx.x);
  __syncthreads();
  const int pieces = (heads * kPerRow) << page_bits;
  const uint8_t* src = c.codes + block0 * c.page * D;
  uint8_t* dst = static_cast<uint8_t*>(which ? v : k) + (((first + pi * c.page) * c.H + h0) * D) * (F32 ? 4 : 2);
  for (int i0 = threadIdx.x; i0 < pieces; i0 += kReadThreads * kReadVec) {
    uint2 w[kReadVec];
#pragma unroll
    for (int j = 0; j < kReadVec; ++j) {
      const int i = i0 + j * kReadThreads;
      w[j] = make_uint2(0u, 0u);
      if (i < pieces && page >= 0) {
        if (F32)
          w[j].x = load_chained(reinterpret_cast<const uint32_t*>(src + static_cast<int64_t>(i) * V));
        else
          w[j] = load_chained(reinterpret_cast<const uint2*>(src + static_cast<int64_t>(i) * V));
      }
    }
#pragma unroll
    for (int j = 0; j < kReadVec; ++j) {
      const int i = i0 + j * kReadThreads;
      const int r = (i / kPerRow) & (c.page - 1), h = (i / kPerRow) >> page_bits;
      if (i >= pieces || r >= rows) continue;
      const float s = s_scale[h];
      const float2 a = fp8b::decode2(static_cast<uint16_t>(w[j].x)), e = fp8b::decode2(static_cast<uint16_t>(w[j].x >> 16));
      uint8_t* to = dst + ((static_cast<int64_t>(r) * c.H + h) * D + i % kPerRow * V) * (F32 ? 4 : 2);
      if (F32) {
        *reinterpret_cast<float4*>(to) = make_float4(a.x * s, a.y * s, e.x * s, e.y * s);
      } else {
        const float2 f = fp8b::decode2(static_cast<uint16_t>(w[j].y)), g = fp8b::decode2(static_cast<uint16_t>(w[j].y >> 16));
        *reinterpret_cast<uint4*>(to) = make_uint4(fp8b::pack_bf16(a.x * s, a.y * s), fp8b::pack_bf16(e.x * s, e.y * s),
                                                   fp8b::pack_bf16(f.x * s, f.y * s), fp8b::pack_bf16(g.x * s, g.y * s));
      }
    }
  }
}

template <int N>
cudaError_t launch_write_team(const WriteArgs& a, int64_t units, cudaStream_t st) {
  constexpr int kThreads = N < 256 ? 256 : N, kTeams = kThreads / N;
  // blocks per CTA: as many CTAs as find room three times over, and no more
  const int rounds = (2 * a.c.H + kTeams - 1) / kTeams;
  const int64_t room = static_cast<int64_t>(3) * sm_count() * (2048 / kThreads);
  const int64_t per = units * rounds / room + 1;
  const int per_cta = static_cast<int>(per < rounds ? per : rounds);
  return launch_chained(write_kernel<N, kThreads>, dim3(static_cast<unsigned>(units), (rounds + per_cta - 1) / per_cta), dim3(kThreads), 0, st,
                        false, a.c, static_cast<const __nv_bfloat16*>(a.k), a.ldk, static_cast<const __nv_bfloat16*>(a.v), a.ldv,
                        a.mode == ZQ_SCALE_M1, per_cta);
}

}  // namespace

int launch_write(const WriteArgs& a, cudaStream_t st) {
  const int64_t units = a.c.cu ? unit_base(a.c.T, a.c.B, a.c.page, 2) : a.c.B;
  if (units > 0x7FFFFFFF) return ZQ_ERR_SHAPE;
  cudaError_t e;
  switch (a.c.page * a.c.D / 32) {
    case 32: e = launch_write_team<32>(a, units, st); break;
    case 64: e = launch_write_team<64>(a, units, st); break;
    case 128: e = launch_write_team<128>(a, units, st); break;
    case 256: e = launch_write_team<256>(a, units, st); break;
    default: e = launch_write_team<512>(a, units, st); break;
  }
  count_launch();
  return e == cudaSuccess ? ZQ_OK : ZQ_ERR_CUDA;
}

int launch_read(const ReadArgs& a, cudaStream_t st) {
  const int64_t units = unit_base(a.c.T, a.c.B, a.c.page, 1);
  if (units > 0x7FFFFFFF) return ZQ_ERR_SHAPE;
  int bits = 4;
  while ((1 << bits) < a.c.page) ++bits;
  // heads per CTA: 16 KB of codes or a little less
  const int fit = 16384 / (a.c.page * a.c.D);
  const int per = fit < 1 ? 1 : fit < kReadHeads ? fit : kReadHeads, per_cta = per < a.c.H ? per : a.c.H;
  auto kernel = a.c.D == 128 ? (a.dt == ZQ_OUT_F32 ? read_kernel<128, true> : read_kernel<128, false>)
                             : (a.dt == ZQ_OUT_F32 ? read_kernel<64, true> : read_kernel<64, false>);
  const cudaError_t e = launch_chained(kernel, dim3(static_cast<unsigned>(units), (a.c.H + per_cta - 1) / per_cta, 2), dim3(kReadThreads), 0, st,
                                       false, a.c, a.k, a.v, per_cta, bits);
  count_launch();
  return e == cudaSuccess ? ZQ_OK : ZQ_ERR_CUDA;
}

}  // namespace kv
}  // namespace zq
