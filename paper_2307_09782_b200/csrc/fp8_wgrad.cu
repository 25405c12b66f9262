// Weight gradient from an 8-bit activation checkpoint:
//   dW[p][n, k] = sum_m G[p][m, n] * bf16(code[m, k] * s[k / 128, m])
//
// The sum runs over tokens, along which the checkpoint's scales change with every row: they cannot be taken out of
// the sum, so the codes are turned back into bf16 on the way to the tensor core (exactly, with power-of-two scales)
// and multiplied by the bf16 gradient.  Only the codes cross HBM and L2; the bf16 values exist in shared memory.
//
// Tile: 128 input features (the MMA's 128-row operand, converted once per 256 outputs) x 256 outputs, tokens by 64.
// In memory both operands have the token index outermost, so both are MN-major for the tensor core: 64 elements
// (128 bytes) of a token per row, 64 token rows = 8 KB per chunk of 64 columns, 128-byte swizzle.
// Converters (a token row and 64 features per thread) read a stage's 8 KB of codes, scale, round and write
// 16 KB of bf16 into a ring of their own; the gradient's tiles go from the copy engine to the tensor core untouched.
// Per 64 tokens the MMAs take 512 cycles, the conversion about 180 issue slots of each SM quarter.
//
// With few tiles and many tokens a cluster of up to 8 CTAs shares a tile's tokens; its partial sums meet through
// distributed shared memory.
// Two accumulators of 256 columns: bf16 results take them in turn, so that the stores of one tile overlap the sums of the
// next; FP32 results use the second for running sums (see kFold).
// Warp roles: 0..7 epilogue, 8..23 converters (four groups, each with a stage of its own), 24 producer, 25 tensor memory
// and MMAs.
#include "fp8_block.cuh"
#include "fp8_index.h"

namespace zq {
namespace fp8b {
namespace {

constexpr int kTok = 64;                         // tokens per stage
constexpr int kTileK = 128, kTileN = 256;
constexpr int kGBytes = kTok * kTileN * 2;       // four chunks of 64 outputs x 64 tokens
constexpr int kXBytes = kTok * kTileK;           // codes
constexpr int kCBytes = kTok * kTileK * 2;       // converted: two chunks of 64 features x 64 tokens
constexpr int kChunk = kTok * 128;               // bytes of a chunk
constexpr int kStages = 4, kConv = 4;            // converter group c owns stage c and converted tile c
constexpr int kOffG = 0;
constexpr int kOffC = kOffG + kStages * kGBytes;
constexpr int kOffX = kOffC + kConv * kCBytes;
constexpr int kOffBars = kOffX + kStages * kXBytes;
constexpr int kNumBars = 2 * kStages + 2 * kConv + 4 + 1;
constexpr int kOffMisc = kOffBars + kNumBars * 8;
constexpr int kSmemBytes = kOffMisc + 16;
static_assert(kSmemBytes <= 227 * 1024, "shared memory");
static_assert(kTileN * kTileK * 4 <= kOffC, "a tile's partial sums must fit the gradient's stages");
constexpr int kEpiWarps = 8;
constexpr int kConvWarp0 = 8, kProducerWarp = 24, kMmaWarp = 25, kThreads = 832;
// Stages whose products go to one accumulator before it is folded into the running sums (FP32 results only).  The tensor
// core rounds every addition to its accumulator towards zero: over 16384 tokens that adds up to 8.5e-6 of the result,
// over 2048 to 6e-7 at most, the size of the rounding errors of an FP32 sum; a fold holds the MMAs up for about 800 cycles.
// (bf16 results round by 4e-3 anyway: half a million tokens in one call would add a tenth of that.)
constexpr int kFold = 32;

enum { kErrProducerW = 31, kErrMmaW = 32, kErrEpilogueW = 33, kErrAlignW = 34, kErrConvertW = 35 };

struct PW {
  int M, N, K;
  int steps;    // stages (of 64 tokens) per tile
  int cluster;  // CTAs that share a tile's tokens
  int k_tiles, n_tiles, n_group;
  int whole, tiles;  // tiles 128 x 256, and with the halves (128 x 128) of the others
  const float* s;
  void* dw;
  int* status;
};

// Position of the launch order -> part, block of features, first output, and whether the tile has 256 outputs or 128.
// (The tiles of the last, incomplete round are cut in halves where those fit one round: 512 tiles on 148 SMs are three
// rounds and 136 halves instead of four rounds.)
__device__ __forceinline__ void tile_of(const PW& p, int pos, int& part, int& kt, int& n0, bool& wide) {
  int cut = 0;
  wide = pos < p.whole;
  if (!wide) {
    cut = (pos - p.whole) & 1;
    pos = p.whole + ((pos - p.whole) >> 1);
  }
  const int per_part = p.n_tiles * p.k_tiles;
  part = pos / per_part;
  pos -= part * per_part;
  const int per_group = p.n_group * p.k_tiles;
  const int g = pos / per_group, within = pos - g * per_group;
  const int gn = min(p.n_group, p.n_tiles - g * p.n_group);
  n0 = (g * p.n_group + within % gn) * kTileN + cut * (kTileN / 2);
  kt = within / gn;
}

// MN-major operand, 128-byte swizzle: 64 elements of the M / N extent per 128-byte row, 8 rows of K per atom.
// Leading offset: the next 64 elements (a chunk further); stride offset: the next 8 rows of K.
__device__ __forceinline__ uint64_t desc_mn128(uint32_t smem_addr) {
  uint64_t d = 0;
  d |= uint64_t((smem_addr >> 4) & 0x3FFF);
  d |= uint64_t(kChunk >> 4) << 16;
  d |= uint64_t(1024 >> 4) << 32;
  d |= uint64_t(1) << 46;
  d |= uint64_t(2) << 61;
  return d;
}
// bf16 x bf16 -> FP32, both operands MN-major, D is 128 x n
__device__ __forceinline__ uint32_t idesc_bf16_mn(uint32_t n) {
  return (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((n >> 3) << 17) | ((128u >> 4) << 24);
}
__device__ __forceinline__ void umma_f16(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// Two codes -> two bf16 values of code * s.
__device__ __forceinline__ uint32_t widen2(uint16_t w, float s) {
  const float2 f = decode2(w);
  return pack_bf16(f.x * s, f.y * s);
}

template <bool F32>
__global__ void __launch_bounds__(kThreads, 1)
fp8_wgrad_kernel(const __grid_constant__ CUtensorMap tm_g, const __grid_constant__ CUtensorMap tm_x, const PW p) {
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kOffBars);
  uint64_t* full = bars;                    // [stages] gradient and codes landed                (converters, MMA wait)
  uint64_t* empty = full + kStages;         // [stages] the MMAs that read the stage are done     (producer waits)
  uint64_t* conv_full = empty + kStages;    // [conv] the converted tile is written               (MMA waits)
  uint64_t* conv_empty = conv_full + kConv; // [conv] the MMAs that read it are done              (converters wait)
  uint64_t* acc_full = conv_empty + kConv;  // [2] a tile's sums are complete                     (epilogue waits)
  uint64_t* acc_empty = acc_full + 2;       // [2] the epilogue has read them                     (MMA waits)
  uint64_t* drain_bar = acc_empty + 2;
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(smem + kOffMisc);
  volatile int* s_abort = reinterpret_cast<volatile int*>(smem + kOffMisc + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < kConv; ++i) {
      mbar_init(&conv_full[i], 4);
      mbar_init(&conv_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&acc_full[i], 1);
      mbar_init(&acc_empty[i], kEpiWarps);
    }
    mbar_init(drain_bar, 1);
    *s_abort = 0;
    fence_mbar_init();
    if ((smem_u32(smem) & 1023u) != 0) raise_error8(p.status, s_abort, kErrAlignW);
  }
  if (warp == kProducerWarp && lane == 0) {
    prefetch_tensormap(&tm_g);
    prefetch_tensormap(&tm_x);
  }
  if (warp == kMmaWarp) tmem_alloc(s_tmem, 512);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = *s_tmem;
  const bool ok_start = *s_abort == 0;
  if (threadIdx.x == 0) pdl_launch_dependents();
  // this CTA's tiles: pos0, + stride, ...; of each the stages step0 .. step0 + steps - 1
  const int rank = static_cast<int>(blockIdx.x) % p.cluster;
  const int pos0 = static_cast<int>(blockIdx.x) / p.cluster, stride = static_cast<int>(gridDim.x) / p.cluster;
  const int step0 = static_cast<int>(static_cast<int64_t>(p.steps) * rank / p.cluster);
  const int steps = static_cast<int>(static_cast<int64_t>(p.steps) * (rank + 1) / p.cluster) - step0;

  if (warp == kProducerWarp) {
    if (ok_start) {
      const bool issuer = elect_one();
      pdl_wait();
      int s = 0, issued = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int pos = pos0; ok && pos < p.tiles; pos += stride) {
        int part, kt, n0;
        bool wide;
        tile_of(p, pos, part, kt, n0, wide);
        for (int i = 0; i < steps; ++i) {
          if (issued >= kStages && !mbar_wait(&empty[s], ph ^ 1, s_abort)) {
            if (issuer) raise_error8(p.status, s_abort, kErrProducerW);
            ok = false;
            break;
          }
          if (issuer) {
            mbar_arrive_expect_tx(&full[s], (wide ? kGBytes : kGBytes / 2) + kXBytes);
            tma_load_3d(smem + kOffX + s * kXBytes, &tm_x, kt * kTileK, (step0 + i) * kTok, 0, &full[s]);
#pragma unroll
            for (int c = 0; c < 4; ++c)
              if (c < 2 || wide) tma_load_3d(smem + kOffG + s * kGBytes + c * kChunk, &tm_g, n0 + c * 64, (step0 + i) * kTok, part, &full[s]);
          }
          __syncwarp();
          ++issued;
          if (++s == kStages) {
            s = 0;
            ph ^= 1;
          }
        }
      }
      // never leave with copies still in flight
      for (int i = max(0, issued - kStages); i < issued; ++i) {
        uint32_t spin = 0;
        while (!mbar_try_wait(&full[i % kStages], (i / kStages) & 1) && ++spin < kSpinLimit) {
        }
      }
    }
  } else if (warp == kMmaWarp) {
    if (ok_start) {
      const bool issuer = elect_one();
      const uint64_t adesc0 = desc_mn128(smem_u32(smem + kOffC));
      const uint64_t bdesc0 = desc_mn128(smem_u32(smem + kOffG));
      int s = 0, c = 0, sum = 0;  // sum: accumulations begun
      uint32_t ph = 0, cph = 0;
      bool failed = false;
      for (int pos = pos0; !failed && pos < p.tiles; pos += stride) {
        const uint32_t idesc = idesc_bf16_mn(pos < p.whole ? kTileN : kTileN / 2);
        for (int i = 0; i < steps; ++i) {
          const bool begin = F32 ? i % kFold == 0 : i == 0, end = i + 1 == steps || (F32 && (i + 1) % kFold == 0);
          if (begin) {
            // FP32: always the first accumulator, the second holds the running sums; bf16: in turn
            const int uses = F32 ? sum : sum >> 1;  // of this accumulator before
            if (uses > 0 && !mbar_wait(&acc_empty[F32 ? 0 : sum & 1], (uses - 1) & 1, s_abort)) {
              failed = true;
              break;
            }
            ++sum;
          }
          const int buf = F32 ? 0 : (sum - 1) & 1;
          if (!mbar_wait(&full[s], ph, s_abort) || !mbar_wait(&conv_full[c], cph, s_abort)) {
            failed = true;
            break;
          }
          tc_fence_after_sync();
          if (issuer) {
            const uint64_t ad = adesc0 + static_cast<uint64_t>((c * kCBytes) >> 4);
            const uint64_t bd = bdesc0 + static_cast<uint64_t>((s * kGBytes) >> 4);
#pragma unroll
            for (int k = 0; k < kTok / 16; ++k)  // 16 token rows of 128 bytes further
              umma_f16(tmem_base + buf * kTileN, ad + k * (2048 >> 4), bd + k * (2048 >> 4), idesc, (!begin || k > 0) ? 1u : 0u);
            umma_commit(&empty[s]);
            umma_commit(&conv_empty[c]);
            if (end) umma_commit(&acc_full[buf]);
          }
          __syncwarp();
          if (++s == kStages) {
            s = 0;
            ph ^= 1;
          }
          if (++c == kConv) {
            c = 0;
            cph ^= 1;
          }
        }
      }
      if (failed && issuer) raise_error8(p.status, s_abort, kErrMmaW);
      // tensor memory is released only when every MMA has completed, also where another role has given up
      if (issuer) umma_commit(drain_bar);
      uint32_t spin = 0;
      while (!mbar_try_wait(drain_bar, 0) && ++spin < kSpinLimit) {
      }
      __syncwarp();
    }
  } else if (warp >= kConvWarp0) {
    // ---- converters: group g (4 warps) takes every fourth stage; thread = token row (t % 64) and chunk of 64
    // features (t / 64)
    const int g = (warp - kConvWarp0) >> 2;
    const int t = (threadIdx.x - kConvWarp0 * 32) & 127;
    const int row = t & 63, chunk = t >> 6;
    const int sw = row & 7;
    const uint4* src = reinterpret_cast<const uint4*>(smem + kOffX + g * kXBytes + row * 128);
    uint4* dst = reinterpret_cast<uint4*>(smem + kOffC + g * kCBytes + chunk * kChunk + row * 128);
    bool failed = !ok_start;
    int n0 = 0;  // stages before this tile
    pdl_wait();
    for (int pos = pos0; !failed && pos < p.tiles; pos += stride, n0 += steps) {
      int part, kt, n_unused;
      bool wide;
      tile_of(p, pos, part, kt, n_unused, wide);
      const float* sc = p.s + static_cast<int64_t>(kt) * p.M;
      int i = (g - n0) & 3;  // this group's first stage of the tile
      auto fetch = [&](int stage) {
        const int m = stage_token(step0, stage, steps, row, p.M);
        return m >= 0 ? load_chained(sc + m) : 0.0f;
      };
      float s_next = fetch(i);
      for (; i < steps; i += 4) {
        const float scale = s_next;
        s_next = fetch(i + 4);
        const int use = (n0 + i) >> 2;  // use of stage g
        if (!mbar_wait_all(&full[g], use & 1, s_abort) || (use > 0 && !mbar_wait_all(&conv_empty[g], (use - 1) & 1, s_abort))) {
          if (lane == 0) raise_error8(p.status, s_abort, kErrConvertW);
          failed = true;
          break;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint4 v = src[(chunk * 4 + j) ^ sw];
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
          uint32_t o[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            o[2 * e] = widen2(static_cast<uint16_t>(w[e]), scale);
            o[2 * e + 1] = widen2(static_cast<uint16_t>(w[e] >> 16), scale);
          }
          dst[(2 * j) ^ sw] = make_uint4(o[0], o[1], o[2], o[3]);
          dst[(2 * j + 1) ^ sw] = make_uint4(o[4], o[5], o[6], o[7]);
        }
        fence_proxy_async_smem();  // the tensor core reads what these stores wrote
        __syncwarp();
        if (lane == 0) mbar_arrive(&conv_full[g]);
      }
    }
  } else {
    // ---- epilogue: thread = input feature and column half; a column is one output channel, 32 neighbouring features
    // per warp
    bool failed = !ok_start;
    constexpr int kCols = kTileN / 2;
    const int half = warp >> 2;
    const uint32_t lane_base = (static_cast<uint32_t>((warp & 3) * 32) << 16) + half * kCols;
    int sum = 0;
    pdl_wait();
    for (int pos = pos0; !failed && pos < p.tiles; pos += stride) {
      int part, kt, n0;
      bool wide;
      tile_of(p, pos, part, kt, n0, wide);
      const bool mine = wide || half == 0;  // a tile of 128 outputs has the first half's columns only
      const int folds = F32 ? (steps + kFold - 1) / kFold : 1;
      for (int f = 0; f < folds; ++f, ++sum) {
        const int buf = F32 ? 0 : sum & 1;
        if (!mbar_wait_all(&acc_full[buf], (F32 ? sum : sum >> 1) & 1, s_abort)) {
          if (lane == 0) raise_error8(p.status, s_abort, kErrEpilogueW);
          failed = true;
          break;
        }
        tc_fence_after_sync();
        if (F32) {
          // into the running sums (of the same lanes and columns: no other warp touches them), then the MMAs may go on
          const uint32_t ta = tmem_base + lane_base, tr = ta + kTileN;
#pragma unroll 1
          for (int c = 0; mine && c < kCols; c += 16) {
            float v[16], r[16];
            tmem_ld16(ta + c, v);
            if (f > 0) tmem_ld16(tr + c, r);
            tmem_ld_wait_regs<16>(v);
            if (f > 0) {
              tmem_ld_wait_regs<16>(r);
#pragma unroll
              for (int e = 0; e < 16; ++e) v[e] += r[e];
            }
            tmem_st16(tr + c, reinterpret_cast<const uint32_t*>(v));
          }
          tmem_st_wait();
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive(&acc_empty[0]);
        }
      }
      if (failed) break;
      const int k = kt * kTileK + (warp & 3) * 32 + lane;
      n0 += half * kCols;
      const int cols = k < p.K ? p.N - n0 : 0;
      const int64_t base = (static_cast<int64_t>(part) * p.N + n0) * p.K + k;
      const int buf = F32 ? 1 : (sum - 1) & 1;
      const uint32_t ta = tmem_base + buf * kTileN + lane_base;
      if (p.cluster > 1) {
        // partial sums of the cluster's CTAs (outputs x 128 features, in the stages' memory, which is done with): they meet
        // below
        float* red = reinterpret_cast<float*>(smem) + half * kCols * kTileK + (warp & 3) * 32 + lane;
#pragma unroll 1
        for (int c = 0; mine && c < kCols; c += 8) {
          float v[8];
          tmem_ld8(ta + c, v);
          tmem_ld_wait_regs<8>(v);
#pragma unroll
          for (int e = 0; e < 8; ++e) red[(c + e) * kTileK] = v[e];
        }
        break;  // a cluster has one tile
      }
#pragma unroll 1
      for (int c = 0; mine && c < kCols; c += 8) {
        float v[8];
        tmem_ld8(ta + c, v);
        tmem_ld_wait_regs<8>(v);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (c + e < cols) {
            const int64_t o = base + static_cast<int64_t>(c + e) * p.K;
            if (F32)
              static_cast<float*>(p.dw)[o] = v[e];
            else
              static_cast<__nv_bfloat16*>(p.dw)[o] = __float2bfloat16_rn(v[e]);
          }
      }
      if (!F32) {
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&acc_empty[buf]);
      }
    }
  }

  tc_fence_before_sync();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after_sync();
    tmem_dealloc(tmem_base, 512);
  }
  if (p.cluster > 1) {
    // rank r adds up outputs r * per .. of the tile, in rank order (the same result every time), and stores them
    cluster_sync_all();
    int part, kt, n0;
    bool wide;
    tile_of(p, pos0, part, kt, n0, wide);
    const int per = (wide ? kTileN : kTileN / 2) / p.cluster;
    const int f = threadIdx.x & (kTileK - 1), k = kt * kTileK + f;
    if (*s_abort == 0 && k < p.K && threadIdx.x < 6 * kTileK) {
      for (int c = rank * per + static_cast<int>(threadIdx.x >> 7); c < (rank + 1) * per && n0 + c < p.N; c += 6) {
        const uint32_t at = smem_u32(smem) + (c * kTileK + f) * 4;
        float v[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) v[r] = r < p.cluster ? ld_cluster(map_to_rank(at, r)) : 0.0f;
#pragma unroll
        for (int r = 1; r < 8; ++r) v[0] += v[r];
        const int64_t o = (static_cast<int64_t>(part) * p.N + n0 + c) * p.K + k;
        if (F32)
          static_cast<float*>(p.dw)[o] = v[0];
        else
          static_cast<__nv_bfloat16*>(p.dw)[o] = __float2bfloat16_rn(v[0]);
      }
    }
    cluster_leave();  // nobody leaves while a peer reads its sums
  }
}

// G as a 3-D tensor [parts][M][N] of bf16, boxes of 64 elements x 64 tokens.
bool make_grad_map(CUtensorMap* m, const WgradArgs& a) {
  gemm::EncodeTiledFn fn = gemm::encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(a.N), static_cast<cuuint64_t>(a.M), static_cast<cuuint64_t>(a.parts)};
  const int64_t part = a.parts > 1 ? a.g_stride : a.M * a.ldg;
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(a.ldg) * 2, static_cast<cuuint64_t>(part) * 2};
  const cuuint32_t box[3] = {64, kTok, 1};
  const cuuint32_t estr[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(a.g), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool F32>
int launch_cfg(const CUtensorMap& tg, const CUtensorMap& tx, const PW& p, unsigned grid, cudaStream_t st) {
  static DeviceOnce once;
  if (!allow_shared_memory(once, fp8_wgrad_kernel<F32>, kSmemBytes)) return ZQ_ERR_CUDA;
  const cudaError_t e = launch_clustered(fp8_wgrad_kernel<F32>, dim3(grid), dim3(kThreads), kSmemBytes, st, p.cluster, tg, tx, p);
  count_launch();
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? ZQ_OK : ZQ_ERR_CUDA;
}

}  // namespace

int launch_wgrad(const WgradArgs& a, cudaStream_t st) {
  PW p{};
  p.M = static_cast<int>(a.M);
  p.N = static_cast<int>(a.N);
  p.K = static_cast<int>(a.K);
  p.steps = static_cast<int>((a.M + kTok - 1) / kTok);
  p.k_tiles = static_cast<int>(blocks_of(a.K));
  p.n_tiles = static_cast<int>((a.N + kTileN - 1) / kTileN);
  p.n_group = 8;
  const int64_t tiles = static_cast<int64_t>(p.k_tiles) * p.n_tiles * a.parts;
  if (tiles > 0x3FFFFFFF) return ZQ_ERR_SHAPE;
  const int sms = sm_count(), tail = static_cast<int>(tiles % sms);
  p.whole = static_cast<int>(2 * tail <= sms ? tiles - tail : tiles);
  p.tiles = static_cast<int>(p.whole + 2 * (tiles - p.whole));
  // Few tiles and many tokens: a cluster shares a tile's tokens, at least 512 of them each.  Of whole tiles and halves the
  // form that is expected to be done first (a stage of 64 tokens takes 0.47 us with 256 outputs, 0.4 with 128).
  p.cluster = 1;
  if (2 * tiles <= sms) {
    auto clusters = [&](int64_t t) {
      int c = 1;
      while (c < 8 && t * c * 2 <= sms && p.steps >= c * 16) c *= 2;
      return c;
    };
    const int cw = clusters(tiles), ch = clusters(2 * tiles);
    const bool halves = (p.steps + ch - 1) / ch * 40 <= (p.steps + cw - 1) / cw * 47;
    p.cluster = halves ? ch : cw;
    p.whole = halves ? 0 : static_cast<int>(tiles);
    p.tiles = static_cast<int>(halves ? 2 * tiles : tiles);
  }
  p.s = a.s;
  p.dw = a.dw;
  p.status = a.status;
  CUtensorMap tg, tx;
  if (!make_grad_map(&tg, a) ||
      !make_code_map(&tx, a.q, static_cast<uint64_t>(a.K), static_cast<uint64_t>(a.M), 1, kTok))
    return ZQ_ERR_CUDA;
  const unsigned grid = static_cast<unsigned>(p.tiles * p.cluster < sms ? p.tiles * p.cluster : sms);
  return a.dwdt == ZQ_OUT_F32 ? launch_cfg<true>(tg, tx, p, grid, st) : launch_cfg<false>(tg, tx, p, grid, st);
}

}  // namespace fp8b
}  // namespace zq
