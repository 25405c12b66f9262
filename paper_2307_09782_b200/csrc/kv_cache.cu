// The 8-bit cache of keys and values: new tokens are quantized as they are written into their pages, and read back.
//
// Both are bound by memory: 3 bytes per element (2 read, 1 written; reading back 1 + 2 or 1 + 4).
#include "kv_cache.cuh"

namespace zq {
namespace kv {
namespace {

// ---- writing ------------------------------------------------------------------------------------------------------
// A team of N threads takes a block (page, keys or values, head): the whole block's new rows are in its registers between the
// maximum and the cast, 32 elements per thread, so they are read once.  Where the block had been begun before and its scale has
// to grow, the team rounds the codes there to the new scale.  Teams of a CTA are neighbouring heads of the same page.
constexpr int kVec = 4;  // 16-byte pieces per thread

template <int N, int THREADS>
__global__ void __launch_bounds__(THREADS)
write_kernel(const Cache c, const __nv_bfloat16* k, int64_t ldk, const __nv_bfloat16* v, int64_t ldv, bool pow2) {
  __shared__ uint32_t s_max[THREADS / 32];
  pdl_launch_dependents();
  const int team = threadIdx.x / N, i = threadIdx.x % N, warp = threadIdx.x >> 5;
  const int64_t task = static_cast<int64_t>(blockIdx.x) * (THREADS / N) + team;
  const int blocks = 2 * c.H;
  const int64_t u = task / blocks;
  const int which = static_cast<int>(task % blocks) / c.H, h = static_cast<int>(task % blocks) % c.H;
  pdl_wait();
  // the unit's sequence, page and rows r0 .. r1 - 1 of it; the block is begun here where r0 is 0
  const int b = c.cu ? unit_sequence(u, c.B, c.page, 2, [&](int j) { return static_cast<int64_t>(load_chained(c.cu + j)); })
                     : static_cast<int>(u < c.B ? u : c.B - 1);
  int first, n;
  rows_of(c, b, first, n);
  const int pos0 = load_chained(c.lens + b) - n;  // of the sequence's first new token
  const int64_t at = c.cu ? u - unit_base(first, b, c.page, 2) : u - b;
  int r0 = 0, r1 = 0, page = -1;
  int64_t row = 0;  // of the tensors, at r0
  if (n > 0 && pos0 >= 0 && at >= 0 && at * c.page < (pos0 % c.page) + static_cast<int64_t>(n)) {
    const int pi = pos0 / c.page + static_cast<int>(at);
    const int64_t lo = max(static_cast<int64_t>(pos0), static_cast<int64_t>(pi) * c.page);
    const int64_t hi = min(static_cast<int64_t>(pos0) + n, static_cast<int64_t>(pi + 1) * c.page);
    page = page_of(c, b, pi);
    r0 = static_cast<int>(lo - static_cast<int64_t>(pi) * c.page);
    r1 = page >= 0 ? static_cast<int>(hi - static_cast<int64_t>(pi) * c.page) : r0;
    row = first + (lo - pos0);
  }
  const bool mine = page >= 0;
  const int lanes = c.D / 8, col = (i % lanes) * 8, rows = N / lanes;
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
  const int64_t block = block_at(c, mine ? page : 0, which, h);
  const float old = mine && r0 > 0 ? load_chained(c.scale + block) : 0.0f;  // 0: begun here
#pragma unroll
  for (int j = 0; j < kVec; ++j) {
    const uint32_t w[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) amax = max(amax, max((w[e] << 16) & 0x7FFF0000u, w[e] & 0x7FFF0000u));
  }
  amax = __reduce_max_sync(0xFFFFFFFFu, amax);
  if (N > 32) {
    if ((threadIdx.x & 31) == 0) s_max[warp] = amax;
    __syncthreads();  // (behind it every thread has read the old scale as well)
#pragma unroll
    for (int j = 0; j < N / 32; ++j) amax = max(amax, s_max[team * (N / 32) + j]);
  }
  float s = cache_scale(amax, pow2);
  const bool grown = !(s <= old);  // also where s is not a number
  if (!grown || isnan(old)) s = old;
  if (!mine) return;
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
        const float2 lo = fp8b::decode2(static_cast<uint16_t>(w)), hi = fp8b::decode2(static_cast<uint16_t>(w >> 16));
        o[e] = fp8b::cast4(__fmul_rn(lo.x, old), __fmul_rn(lo.y, old), __fmul_rn(hi.x, old), __fmul_rn(hi.y, old), inv);
      }
      *q = bad ? make_uint2(0u, 0u) : make_uint2(o[0], o[1]);
    }
  }
  if (i == 0) c.scale[block] = s;
}

// ---- reading back ---------------------------------------------------------------------------------------------------
// A CTA takes some of a page's rows and heads, for keys or values: pieces of V codes whose results are 16 bytes.
constexpr int kReadThreads = 256, kReadVec = 4;

template <bool F32>
__global__ void __launch_bounds__(kReadThreads) read_kernel(const Cache c, void* k, void* v) {
  constexpr int V = F32 ? 4 : 8;
  pdl_launch_dependents();
  const int64_t u = blockIdx.x;
  const int which = blockIdx.z;
  pdl_wait();
  const int b = unit_sequence(u, c.B, c.page, 1, [&](int j) { return static_cast<int64_t>(load_chained(c.cu + j)); });
  int first, n;
  rows_of(c, b, first, n);
  const int64_t pi = u - unit_base(first, b, c.page, 1);
  if (pi < 0 || pi * c.page >= n) return;
  const int page = page_of(c, b, static_cast<int>(pi));
  const int rows = min(c.page, n - static_cast<int>(pi) * c.page);
  const int per_row = c.D / V;
  const int pieces = c.H * c.page * per_row;
  const int64_t block0 = block_at(c, max(page, 0), which, 0);
  const uint8_t* src = c.codes + block0 * c.page * c.D;
  uint8_t* dst = static_cast<uint8_t*>(which ? v : k);
  uint2 w[kReadVec];
  float s[kReadVec];
#pragma unroll
  for (int j = 0; j < kReadVec; ++j) {
    const int i = (blockIdx.y * kReadVec + j) * kReadThreads + threadIdx.x;
    const int h = i / (c.page * per_row), r = i / per_row % c.page;
    w[j] = make_uint2(0u, 0u);
    s[j] = __uint_as_float(0x7FC00000u);  // a page the table lacks
    if (i < pieces && r < rows && page >= 0) {
      if (F32)
        w[j].x = load_chained(reinterpret_cast<const uint32_t*>(src + static_cast<int64_t>(i) * V));
      else
        w[j] = load_chained(reinterpret_cast<const uint2*>(src + static_cast<int64_t>(i) * V));
      s[j] = load_chained(c.scale + block0 + h);
    }
  }
#pragma unroll
  for (int j = 0; j < kReadVec; ++j) {
    const int i = (blockIdx.y * kReadVec + j) * kReadThreads + threadIdx.x;
    const int h = i / (c.page * per_row), r = i / per_row % c.page, d = i % per_row * V;
    if (i >= pieces || r >= rows) continue;
    const int64_t o = ((first + pi * c.page + r) * c.H + h) * c.D + d;
    const float2 a = fp8b::decode2(static_cast<uint16_t>(w[j].x)), e = fp8b::decode2(static_cast<uint16_t>(w[j].x >> 16));
    if (F32) {
      *reinterpret_cast<float4*>(dst + o * 4) = make_float4(a.x * s[j], a.y * s[j], e.x * s[j], e.y * s[j]);
    } else {
      const float2 f = fp8b::decode2(static_cast<uint16_t>(w[j].y)), g = fp8b::decode2(static_cast<uint16_t>(w[j].y >> 16));
      *reinterpret_cast<uint4*>(dst + o * 2) =
          make_uint4(fp8b::pack_bf16(a.x * s[j], a.y * s[j]), fp8b::pack_bf16(e.x * s[j], e.y * s[j]),
                     fp8b::pack_bf16(f.x * s[j], f.y * s[j]), fp8b::pack_bf16(g.x * s[j], g.y * s[j]));
    }
  }
}

template <int N>
cudaError_t launch_write_team(const WriteArgs& a, int64_t tasks, cudaStream_t st) {
  constexpr int kThreads = N < 256 ? 256 : N;
  const int64_t grid = (tasks + kThreads / N - 1) / (kThreads / N);
  if (grid > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
  return launch_chained(write_kernel<N, kThreads>, dim3(static_cast<unsigned>(grid)), dim3(kThreads), 0, st, false, a.c,
                        static_cast<const __nv_bfloat16*>(a.k), a.ldk, static_cast<const __nv_bfloat16*>(a.v), a.ldv,
                        a.mode == ZQ_SCALE_M1);
}

}  // namespace

int launch_write(const WriteArgs& a, cudaStream_t st) {
  const int64_t units = a.c.cu ? unit_base(a.c.T, a.c.B, a.c.page, 2) : a.c.B;
  const int64_t tasks = units * 2 * a.c.H;
  cudaError_t e;
  switch (a.c.page * a.c.D / 32) {
    case 32: e = launch_write_team<32>(a, tasks, st); break;
    case 64: e = launch_write_team<64>(a, tasks, st); break;
    case 128: e = launch_write_team<128>(a, tasks, st); break;
    case 256: e = launch_write_team<256>(a, tasks, st); break;
    default: e = launch_write_team<512>(a, tasks, st); break;
  }
  count_launch();
  return e == cudaSuccess ? ZQ_OK : ZQ_ERR_CUDA;
}

int launch_read(const ReadArgs& a, cudaStream_t st) {
  const int64_t units = unit_base(a.c.T, a.c.B, a.c.page, 1);
  const int pieces = a.c.H * a.c.page * a.c.D / (a.dt == ZQ_OUT_F32 ? 4 : 8);
  const int per = kReadThreads * kReadVec;
  if (units > 0x7FFFFFFF) return ZQ_ERR_SHAPE;
  const cudaError_t e = launch_chained(a.dt == ZQ_OUT_F32 ? read_kernel<true> : read_kernel<false>,
                                       dim3(static_cast<unsigned>(units), static_cast<unsigned>((pieces + per - 1) / per), 2),
                                       dim3(kReadThreads), 0, st, false, a.c, a.k, a.v);
  count_launch();
  return e == cudaSuccess ? ZQ_OK : ZQ_ERR_CUDA;
}

}  // namespace kv
}  // namespace zq
