// Matrix product of E4M3 operands with block scales, few tokens: the linear layer and the gated linear layer of
// decoding.
//
// What bounds it is the weights' way from HBM.  Orientation: output channels are the lanes (the MMA's 128-row
// operand), so that a weight tile is read once for all tokens of the call, and BM = 16, 32 or 64 tokens are
// its columns.  A tile of 128 channels (kGated: 128 of the gate and the same 128 of the up projection) is worked on by
// a cluster of 1, 2, 4 or 8 CTAs that share its K blocks; several CTAs are resident on an SM, so that the device has
// enough copies in flight.  The cluster's partial sums meet through distributed shared memory: rank r adds up the
// tokens that are its share, in rank order (the same result every time), and finishes them: one launch, no
// scratch in global memory.
//
// A pipeline stage is a K block: weight tile, token tile, token scales and an accumulator of its own in tensor memory, so
// that the roles meet at three barriers per block and run up to kStages blocks apart (with two accumulators for all
// stages their hand-over took 1.1 us per block whatever the copies took).
// The tensor core adds up one block of 128; the epilogue warps multiply it by the block's scale (of the weight
// tile, one number; of the tokens, one per column, read from shared memory) and add it to running sums in registers.
//
// RAW (up to 16 tokens): the kernel quantizes the activations itself, one launch per layer.  A block's scale belongs to
// 128 features of one token, so a CTA needs nothing but its own K blocks of x for it: four warps read them (from L2:
// every cluster reads the same), find the maximum, cast, and write the operand tile and its scales.  The codes are
// those of zq_quantize_fp8_block.  With more tokens the cast of a K block in every CTA takes longer than its weights'
// way from HBM (32 tokens, 7168 -> 28672: 134 us), and a separate quantizer costs less.
//
// Warp roles: epilogue (four warps per matrix, with 64 tokens eight: each takes 32 tokens), then 4 quantizer warps (without RAW they
// bring the tokens' scales; the weight tiles' scales in both forms), 1 producer, 1 tensor memory and MMAs.
#include "fp8_block.cuh"

namespace zq {
namespace fp8b {
namespace {

enum { kErrProducerF = 41, kErrMmaF = 42, kErrEpilogueF = 43, kErrAlignF = 44, kErrQuantF = 45 };

struct PF {
  int M, N, K;
  int kblocks, segs, nblocks;
  int n_tiles, cluster;
  const float* sa;
  const float* sb;
  const __nv_bfloat16* x;  // RAW
  int64_t ldx;
  void* y;
  int64_t ldy;
  int y_f32, y_vec;  // y_vec: four neighbouring outputs can be stored at once
  uint8_t* q;
  float* s;
  uint8_t* ck;
  float* cks;
  int act, pow2;
  int* status;
};

template <int BM, bool GATED>
struct FewCfg {
  static constexpr int kMats = GATED ? 2 : 1;
  static constexpr int kSplit = BM == 64 ? 2 : 1;  // warps that share a channel's tokens
  static constexpr int kCols1 = BM / kSplit;                 // tokens per epilogue thread
  static constexpr int kEpiWarps = 4 * kMats * kSplit;
  static constexpr int kQuantWarp0 = kEpiWarps, kQuantWarps = 4;
  static constexpr int kProducerWarp = kEpiWarps + 4, kMmaWarp = kEpiWarps + 5;
  static constexpr int kThreads = 32 * (kEpiWarps + 6);
  static constexpr int kWBytes = kMats * 128 * kBlk, kTokBytes = BM * kBlk;
  static constexpr int kStageBytes = kWBytes + kTokBytes;
  // CTAs per SM wanted, and with them the stages that fit
  static constexpr int kCtas = GATED && BM > 32 ? 1 : 2;
  static constexpr int kSmemEach = 226 * 1024 / kCtas - 1024;
  static constexpr int kMisc = 1024 + 4 * BM * 12;
  static constexpr int kStagesFit = (kSmemEach - kMisc) / kStageBytes;
  // a stage has its accumulator in tensor memory: 512 columns for all CTAs of an SM
  static constexpr int kStagesTmem = 512 / kCtas / (kMats * BM);
  static constexpr int kStages = gemm::cmin(8, gemm::cmin(kStagesFit, kStagesTmem));
  static constexpr int kRedBytes = kMats * BM * 128 * 4;  // partial sums, in the stages' memory once they are done
  static constexpr int kCols = kStages * kMats * BM;
  static constexpr int kTmemCols = kCols <= 32 ? 32 : (kCols <= 64 ? 64 : (kCols <= 128 ? 128 : (kCols <= 256 ? 256 : 512)));
  static constexpr int offTok = kStages * kWBytes;
  static constexpr int offSc = offTok + kStages * kTokBytes;  // [stages][BM] token scales
  static constexpr int offSw = offSc + kStages * BM * 4;      // [stages][2] scales of the weight tiles
  static constexpr int offBars = offSw + kStages * 8;
  static constexpr int kNumBars = 5 * kStages + 1;
  static constexpr int offMisc = offBars + kNumBars * 8;
  static constexpr int kSmemBytes = offMisc + 16;
  static_assert(kStages >= 3, "pipeline depth");
  static_assert(kRedBytes <= offSc, "the partial sums must fit the stages");
  static_assert(kSmemBytes <= kSmemEach, "shared memory");
  static_assert(kTmemCols * kCtas <= 512, "tensor memory");
  static_assert((BM * 4) % 16 == 0 && kTokBytes % 1024 == 0, "alignment");
};

__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void store_bf16x4(__nv_bfloat16* y, const float* v, int n_here, bool vec) {
  if (vec && n_here >= 4) {
    *reinterpret_cast<uint2*>(y) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n_here) y[e] = __float2bfloat16_rn(v[e]);
  }
}
// One warp, one block: scale and codes of 128 values, four per lane (their number is a multiple of 16).
__device__ __forceinline__ void quantize_token(const float* v, uint8_t* q, float* s, int n_here, bool pow2, int lane) {
  uint32_t a = max(max(abs_bits(v[0]), abs_bits(v[1])), max(abs_bits(v[2]), abs_bits(v[3])));
#pragma unroll
  for (int o = 16; o; o >>= 1) a = max(a, __shfl_xor_sync(0xFFFFFFFFu, a, o));
  const float sc = block_scale(a, pow2), inv = block_inv(sc);
  if (n_here >= 4) *reinterpret_cast<uint32_t*>(q) = cast4(v[0], v[1], v[2], v[3], inv);
  if (lane == 0) *s = sc;
}
__device__ __forceinline__ float act_any(int act, float v) {
  if (act == ZQ_ACT_SILU) return act_value<ZQ_ACT_SILU>(v);
  if (act == ZQ_ACT_GELU_TANH) return act_value<ZQ_ACT_GELU_TANH>(v);
  return act_value<ZQ_ACT_RELU>(v);
}

template <int BM, bool GATED, bool RAW>
__global__ void __launch_bounds__(FewCfg<BM, GATED>::kThreads, FewCfg<BM, GATED>::kCtas)
fp8_block_few_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_q, const PF p) {
  using C = FewCfg<BM, GATED>;
  constexpr int NS = C::kStages;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::offBars);
  uint64_t* full = bars;                // [NS] the copies of the stage landed                        (MMA waits)
  uint64_t* tok_full = full + NS;       // [NS] RAW: the token codes are written                      (MMA waits)
  uint64_t* acc_full = tok_full + NS;   // [NS] the stage's products are complete, its token scales written (epilogue waits)
  uint64_t* empty = acc_full + NS;      // [NS] the MMAs that read the stage are done                  (producer waits)
  uint64_t* acc_empty = empty + NS;     // [NS] the epilogue warps have read products and scales      (MMA, quantizer wait)
  uint64_t* drain_bar = acc_empty + NS;
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(smem + C::offMisc);
  volatile int* s_abort = reinterpret_cast<volatile int*>(smem + C::offMisc + 4);
  float* s_sc = reinterpret_cast<float*>(smem + C::offSc);
  float* s_sw = reinterpret_cast<float*>(smem + C::offSw);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < NS; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&tok_full[i], 1);
      mbar_init(&acc_full[i], 2);  // the MMAs' commit and the warp that wrote the scales
      mbar_init(&empty[i], 1);
      mbar_init(&acc_empty[i], C::kEpiWarps);
    }
    mbar_init(drain_bar, 1);
    *s_abort = 0;
    fence_mbar_init();
    if ((smem_u32(smem) & 1023u) != 0) raise_error8(p.status, s_abort, kErrAlignF);
  }
  if (warp == C::kProducerWarp && lane == 0) {
    prefetch_tensormap(&tm_w);
    if (!RAW) prefetch_tensormap(&tm_q);
  }
  if (warp == C::kMmaWarp) tmem_alloc(s_tmem, C::kTmemCols);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = *s_tmem;
  const bool ok_start = *s_abort == 0;
  if (threadIdx.x == 0) pdl_launch_dependents();

  // this CTA's share: K blocks [kb0, kb1) of tile nt, tokens [m0, m0 + BM)
  const int rank = static_cast<int>(blockIdx.x) % p.cluster, nt = static_cast<int>(blockIdx.x) / p.cluster;
  const int m0 = static_cast<int>(blockIdx.y) * BM;
  const int kb_all = p.segs * p.kblocks;
  const int kb0 = static_cast<int>(static_cast<int64_t>(kb_all) * rank / p.cluster);
  const int kb1 = static_cast<int>(static_cast<int64_t>(kb_all) * (rank + 1) / p.cluster);
  const int nkb = kb1 - kb0;
  const int m_here = min(BM, p.M - m0);

  uint64_t run[C::kCols1 / 2];  // epilogue warps: one channel's sums, tokens in pairs
#pragma unroll
  for (int c = 0; c < C::kCols1 / 2; ++c) run[c] = 0ull;

  if (warp == C::kProducerWarp) {
    if (ok_start) {
      const bool issuer = elect_one();
      auto issue = [&](int s, int kb) {
        if (!issuer) return;
        const int seg = kb / p.kblocks, k = (kb - seg * p.kblocks) * kBlk;
        uint8_t* d = smem + s * C::kWBytes;
        mbar_arrive_expect_tx(&full[s], C::kWBytes + (RAW ? 0 : C::kTokBytes));
        tma_load_3d(d, &tm_w, k, nt * kBlk, GATED ? 0 : seg, &full[s]);
        if (GATED) tma_load_3d(d + C::kWBytes / 2, &tm_w, k, nt * kBlk, 1, &full[s]);
        if (!RAW) tma_load_3d(smem + C::offTok + s * C::kTokBytes, &tm_q, k, m0, seg, &full[s]);
      };
      // The first weight tiles are fetched to L2 while the kernel ahead in the stream may still run.  They are copied from there
      // after the wait for it, and not before: it may be the kernel that writes the weights, or that followed it, and until then
      // nothing orders its stores before the copies.
      const int first = min(NS, nkb);
      for (int i = 0; i < first; ++i) {
        if (!issuer) continue;
        const int kb = kb0 + i, seg = kb / p.kblocks, k = (kb - seg * p.kblocks) * kBlk;
        tma_prefetch_3d(&tm_w, k, nt * kBlk, GATED ? 0 : seg);
        if (GATED) tma_prefetch_3d(&tm_w, k, nt * kBlk, 1);
      }
      __syncwarp();
      pdl_wait();
      for (int i = 0; i < first; ++i) issue(i, kb0 + i);
      __syncwarp();
      bool ok = true;
      int s = first == NS ? 0 : first, issued = first;
      uint32_t ph = 1;
      for (int i = first; i < nkb; ++i) {
        if (!mbar_wait(&empty[s], ph ^ 1, s_abort)) {
          if (issuer) raise_error8(p.status, s_abort, kErrProducerF);
          ok = false;
          break;
        }
        issue(s, kb0 + i);
        __syncwarp();
        ++issued;
        if (++s == NS) {
          s = 0;
          ph ^= 1;
        }
      }
      (void)ok;
      // never leave with copies still in flight
      for (int i = max(0, issued - NS); i < issued; ++i) {
        uint32_t spin = 0;
        while (!mbar_try_wait(&full[i % NS], (i / NS) & 1) && ++spin < kSpinLimit) {
        }
      }
    }
  } else if (warp == C::kMmaWarp) {
    if (ok_start) {
      const bool issuer = elect_one();
      const uint64_t adesc0 = umma_desc_k128(smem_u32(smem));
      const uint64_t bdesc0 = umma_desc_k128(smem_u32(smem + C::offTok));
      const uint32_t idesc = umma_idesc_e4m3(BM);
      int s = 0;
      uint32_t ph = 0;
      bool failed = false;
      for (int i = 0; i < nkb; ++i) {
        if ((i >= NS && !mbar_wait(&acc_empty[s], ph ^ 1, s_abort)) || !mbar_wait(&full[s], ph, s_abort) ||
            (RAW && !mbar_wait(&tok_full[s], ph, s_abort))) {
          failed = true;
          break;
        }
        tc_fence_after_sync();
        if (issuer) {
          const uint64_t ad = adesc0 + static_cast<uint64_t>((s * C::kWBytes) >> 4);
          const uint64_t bd = bdesc0 + static_cast<uint64_t>((s * C::kTokBytes) >> 4);
#pragma unroll
          for (int mat = 0; mat < C::kMats; ++mat)
#pragma unroll
            for (int k = 0; k < kBlk / 32; ++k)
              umma_f8(tmem_base + (s * C::kMats + mat) * BM, ad + ((mat * 128 * kBlk) >> 4) + 2 * k, bd + 2 * k, idesc,
                      k > 0 ? 1u : 0u);
          umma_commit(&acc_full[s]);
          umma_commit(&empty[s]);
        }
        __syncwarp();
        if (++s == NS) {
          s = 0;
          ph ^= 1;
        }
      }
      if (failed && issuer) raise_error8(p.status, s_abort, kErrMmaF);
      // tensor memory is released only when every MMA has completed, also where another role has given up
      if (issuer) umma_commit(drain_bar);
      uint32_t spin = 0;
      while (!mbar_try_wait(drain_bar, 0) && ++spin < kSpinLimit) {
      }
      __syncwarp();
    }
  } else if (warp >= C::kQuantWarp0) {
    const int qw = warp - C::kQuantWarp0;
    // A warp takes the K blocks of the stages that are its own (stage % 4 == qw), so that four blocks are under way at a
    // time.  A stage belongs to one warp because a parity wait tells only two neighbouring phases of a barrier apart:
    // whoever waits for a stage has to see every use of it.
    auto next_own = [&](int i) {
      do ++i;
      while ((i % NS) % C::kQuantWarps != qw);
      return i;
    };
    int i_next = ok_start && qw < NS ? qw : nkb;  // with fewer stages than warps some have nothing to do
    // the weight tiles' scales of a K block, one per lane 0 .. kMats - 1
    auto weight_scale = [&](int kb) {
      const int seg = kb / p.kblocks;
      const int64_t part = static_cast<int64_t>(p.nblocks) * p.kblocks;
      return lane < C::kMats ? load_chained(p.sb + (GATED ? lane : seg) * part + static_cast<int64_t>(nt) * p.kblocks + (kb - seg * p.kblocks))
                             : 0.0f;
    };
    pdl_wait();
    if (RAW) {
      // 16 lanes per token row, two rows at a time
      constexpr int kPairs = BM / 2;
      const int hl = lane & 15, r0 = lane >> 4;
      uint4 v[kPairs];
      auto fetch = [&](int kb) {
        const int k = kb * kBlk + hl * 8;
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
          const int r = r0 + 2 * j;
          v[j] = make_uint4(0u, 0u, 0u, 0u);
          if (r < m_here && k < p.K) v[j] = load_chained(reinterpret_cast<const uint4*>(p.x + static_cast<int64_t>(m0 + r) * p.ldx + k));
        }
      };
      while (i_next < nkb) {
        const int i = i_next;
        const int s = i % NS;
        i_next = next_own(i);
        fetch(kb0 + i);
        const float sw = weight_scale(kb0 + i);
        if (i >= NS && !mbar_wait_all(&acc_empty[s], ((i / NS) - 1) & 1, s_abort)) {
          if (lane == 0) raise_error8(p.status, s_abort, kErrQuantF);
          break;
        }
        uint8_t* tok = smem + C::offTok + s * C::kTokBytes;
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
          const int r = r0 + 2 * j;
          if (2 * j < m_here) {  // uniform: one of the two rows is a token
            const uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
            uint32_t a = 0u;
#pragma unroll
            for (int e = 0; e < 4; ++e) a = max(a, max((w[e] << 16) & 0x7FFF0000u, w[e] & 0x7FFF0000u));
#pragma unroll
            for (int o = 8; o; o >>= 1) a = max(a, __shfl_xor_sync(0xFFFFFFFFu, a, o));
            const float sc = block_scale(a, p.pow2 != 0), inv = block_inv(sc);
            // the operand's 128-byte swizzle: 16-byte piece XOR row; columns past the last token stay what they
            // were, their sums are never looked at
            if (r < m_here) {
              *reinterpret_cast<uint2*>(tok + r * kBlk + (((hl >> 1) ^ (r & 7)) << 4) + (hl & 1) * 8) = cast8(v[j], inv);
              if (hl == 0) s_sc[s * BM + r] = sc;
            }
          }
        }
        if (lane < C::kMats) s_sw[2 * s + lane] = sw;
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&tok_full[s]);
          mbar_arrive(&acc_full[s]);
        }
      }
    } else {
      while (i_next < nkb) {
        const int i = i_next;
        const int s = i % NS;
        i_next = next_own(i);
        const float* src = p.sa + static_cast<int64_t>(kb0 + i) * p.M + m0;  // [segs][kblocks][M]
        float v[BM / 32 + 1];
#pragma unroll
        for (int c = 0; c < BM; c += 32) v[c / 32] = c + lane < m_here ? load_chained(src + c + lane) : 0.0f;
        const float sw = weight_scale(kb0 + i);
        if (i >= NS && !mbar_wait_all(&acc_empty[s], ((i / NS) - 1) & 1, s_abort)) {
          if (lane == 0) raise_error8(p.status, s_abort, kErrQuantF);
          break;
        }
#pragma unroll
        for (int c = 0; c < BM; c += 32)
          if (c + lane < BM) s_sc[s * BM + c + lane] = v[c / 32];
        if (lane < C::kMats) s_sw[2 * s + lane] = sw;
        __syncwarp();
        if (lane == 0) mbar_arrive(&acc_full[s]);
      }
    }
  } else {
    // ---- epilogue warps: running sums of one channel and all tokens
    const int mat = (warp >> 2) / C::kSplit;
    const int col0 = (warp >> 2) % C::kSplit * C::kCols1;  // first of this warp's tokens
    const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
    bool failed = !ok_start;
    int s = 0;
    uint32_t ph = 0;
    pdl_wait();
    for (int i = 0; i < nkb; ++i) {
      if (!failed && !mbar_wait_all(&acc_full[s], ph, s_abort)) {
        if (lane == 0) raise_error8(p.status, s_abort, kErrEpilogueF);
        failed = true;
      }
      tc_fence_after_sync();
      if (!failed) {
        const uint32_t t = tmem_base + (s * C::kMats + mat) * BM + col0 + lane_base;
        const ulonglong2* sc = reinterpret_cast<const ulonglong2*>(s_sc + s * BM + col0);  // pairs of tokens
        const float sw = s_sw[2 * s + mat];
        const uint64_t sw2 = pack2(sw, sw);
        float nxt[16];
        tmem_ld16(t, nxt);
#pragma unroll
        for (int c = 0; c < C::kCols1; c += 16) {
          float v[16];
          tmem_ld_wait_regs<16>(nxt);
#pragma unroll
          for (int e = 0; e < 16; ++e) v[e] = nxt[e];
          if (c + 16 < C::kCols1) tmem_ld16(t + c + 16, nxt);
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            const ulonglong2 f = sc[(c + e) / 4];
            run[(c + e) / 2] = fma2(mul2(f.x, sw2), pack2(v[e], v[e + 1]), run[(c + e) / 2]);
            run[(c + e) / 2 + 1] = fma2(mul2(f.y, sw2), pack2(v[e + 2], v[e + 3]), run[(c + e) / 2 + 1]);
          }
        }
      }
      tc_fence_before_sync();
      __syncwarp();
      // a warp that has given up counts itself in nowhere: nobody may take what it has not waited for as free
      if (failed) break;
      if (lane == 0) mbar_arrive(&acc_empty[s]);
      if (++s == NS) {
        s = 0;
        ph ^= 1;
      }
    }
  }

  // Every copy has landed and every MMA has completed once all roles are here: the stages' memory is free.
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  if (warp == C::kMmaWarp) tmem_dealloc(tmem_base, C::kTmemCols);
  float* red = reinterpret_cast<float*>(smem);  // [kMats][BM][128]
  if (warp < C::kEpiWarps) {
#pragma unroll
    for (int c = 0; c < C::kCols1 / 2; ++c) {
      float lo, hi;
      unpack2(run[c], lo, hi);
      // [kMats][BM][128]: a matrix's tokens, by the warps that share them, one after the other
      float* r = red + ((warp >> 2) * C::kCols1 + 2 * c) * 128 + (warp & 3) * 32 + lane;
      r[0] = lo;
      r[128] = hi;
    }
  }
  cluster_sync_all();
  if (warp < C::kEpiWarps && *s_abort == 0) {
    // a warp finishes one token at a time (rank * per + warp, + kEpiWarps, ...), a lane four neighbouring channels
    const int n = nt * kBlk + 4 * lane;
    const int n_here = p.N - n;  // may be <= 0
    const int per = BM / p.cluster;
    const int c_end = min(m_here, (rank + 1) * per);
    const uint32_t base = smem_u32(red) + lane * 16;
    for (int c = rank * per + warp; c < c_end; c += C::kEpiWarps) {
      const int64_t m = m0 + c;
      float v[C::kMats][4];
#pragma unroll
      for (int mat = 0; mat < C::kMats; ++mat) {
        float4 part[8];  // all ranks' sums on their way before the first is added
#pragma unroll
        for (int r = 0; r < 8; ++r)
          part[r] = r < p.cluster ? ld_cluster4(map_to_rank(base + (mat * BM + c) * 512, r)) : make_float4(0.f, 0.f, 0.f, 0.f);
        v[mat][0] = part[0].x;
        v[mat][1] = part[0].y;
        v[mat][2] = part[0].z;
        v[mat][3] = part[0].w;
#pragma unroll
        for (int r = 1; r < 8; ++r) {
          v[mat][0] += part[r].x;
          v[mat][1] += part[r].y;
          v[mat][2] += part[r].z;
          v[mat][3] += part[r].w;
        }
      }
      if (!GATED) {
        if (p.y_f32) {
          float* y = static_cast<float*>(p.y) + m * p.ldy + n;
          if (p.y_vec && n_here >= 4) {
            *reinterpret_cast<float4*>(y) = make_float4(v[0][0], v[0][1], v[0][2], v[0][3]);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (e < n_here) y[e] = v[0][e];
          }
        } else {
          store_bf16x4(static_cast<__nv_bfloat16*>(p.y) + m * p.ldy + n, v[0], n_here, p.y_vec != 0);
        }
      } else {
        float* g = v[0];
        float* u = v[C::kMats - 1];
        // channels past N hold zeros (the copy engine filled their weights with zeros)
        float h[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = act_any(p.act, g[e]) * u[e];
        if (p.y) store_bf16x4(static_cast<__nv_bfloat16*>(p.y) + m * p.ldy + n, h, n_here, p.y_vec != 0);
        const int64_t MN = static_cast<int64_t>(p.M) * p.N, SM = static_cast<int64_t>(p.nblocks) * p.M;
        if (p.q) quantize_token(h, p.q + m * p.N + n, p.s + static_cast<int64_t>(nt) * p.M + m, n_here, p.pow2 != 0, lane);
        if (p.ck) {
          quantize_token(g, p.ck + m * p.N + n, p.cks + static_cast<int64_t>(nt) * p.M + m, n_here, p.pow2 != 0, lane);
          quantize_token(u, p.ck + MN + m * p.N + n, p.cks + SM + static_cast<int64_t>(nt) * p.M + m, n_here, p.pow2 != 0, lane);
        }
      }
    }
  }
  cluster_leave();  // nobody leaves while a peer reads its sums
}

template <int BM, bool GATED, bool RAW>
int launch_cfg(const CUtensorMap& tw, const CUtensorMap& tq, const PF& p, int m_tiles, cudaStream_t st) {
  using C = FewCfg<BM, GATED>;
  static DeviceOnce once;
  if (!allow_shared_memory(once, fp8_block_few_kernel<BM, GATED, RAW>, C::kSmemBytes)) return ZQ_ERR_CUDA;
  const cudaError_t e = launch_clustered(fp8_block_few_kernel<BM, GATED, RAW>,
                                         dim3(static_cast<unsigned>(p.n_tiles * p.cluster), static_cast<unsigned>(m_tiles)),
                                         dim3(C::kThreads), C::kSmemBytes, st, p.cluster, tw, tq, p);
  count_launch();
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? ZQ_OK : ZQ_ERR_CUDA;
}

template <int BM>
constexpr int ctas_per_sm(bool gated) {
  return gated ? FewCfg<BM, true>::kCtas : FewCfg<BM, false>::kCtas;
}

}  // namespace

namespace {

int few_width(int64_t M) { return M <= 16 ? 16 : (M <= 32 ? 32 : 64); }
int few_slots(int bm, bool gated) {
  return sm_count() * (bm == 16 ? ctas_per_sm<16>(gated) : (bm == 32 ? ctas_per_sm<32>(gated) : ctas_per_sm<64>(gated)));
}
// The widest cluster with which all CTAs are resident at once and none has fewer than two K blocks.
int few_cluster(int64_t tiles, int64_t kb_all, int slots) {
  int c = 1;
  while (c < 8 && tiles * c * 2 <= slots && kb_all >= c * 4) c *= 2;
  return c;
}

}  // namespace

// Which of the two kernels.  Up to 32 tokens this one: it streams the weights at 0.8 - 0.9 of the copy bandwidth.  Beyond, the
// one that is expected to be done first.  Here a CTA with 64 tokens takes 0.75 us per K block (gated: 0.85), all of it in
// `waves`, and 4 us more; the other kernel 0.6 us per K block of a tile of 128 x 256 and 2 us more.  Measured (us, this
// kernel / the other): 64 tokens 4096 -> 4096 9.7 / 19.6, 17920 -> 6656 29 / 71, 7168 -> 28672 44.5 / 39.6, gated 4096 ->
// 11008 29 / 23.5; 256 tokens 4096 -> 4096 17 / 22, 11008 -> 4096 35 / 50; 512 tokens 4096 -> 4096 28 / 22.
bool few_takes(const GemmArgs8& a) {
  if (a.kind == kGatedBwd) return false;
  if (a.M <= 32) return true;
  const bool gated = a.kind == kGated;
  const int64_t kb = blocks_of(a.K) * (gated ? 1 : a.parts), nb = blocks_of(a.N);
  const int slots = few_slots(64, gated);
  const int64_t tiles = (a.M + 63) / 64 * nb;
  const int c = few_cluster(tiles, kb, slots);
  const int64_t waves = (tiles * c + slots - 1) / slots;
  const int64_t here = 4000 + waves * ((kb + c - 1) / c) * (gated ? 850 : 750);
  const int64_t cols = gated ? nb : (a.N + 255) / 256;
  const int64_t rounds = ((a.M + 127) / 128 * cols + sm_count() - 1) / sm_count();
  return here < 2000 + rounds * kb * 600;
}
bool few_takes_raw(const GemmArgs8& a) { return a.M <= 16 && a.kind != kGatedBwd; }

int launch_block_few(const GemmArgs8& a, cudaStream_t st) {
  const bool gated = a.kind == kGated, raw = a.x != nullptr;
  PF p{};
  p.M = static_cast<int>(a.M);
  p.N = static_cast<int>(a.N);
  p.K = static_cast<int>(a.K);
  p.kblocks = static_cast<int>(blocks_of(a.K));
  p.segs = gated ? 1 : a.parts;
  p.nblocks = p.n_tiles = static_cast<int>(blocks_of(a.N));
  p.sa = a.sa;
  p.sb = a.sb;
  p.x = static_cast<const __nv_bfloat16*>(a.x);
  p.ldx = a.ldx;
  p.y = a.y;
  p.ldy = a.ldy;
  p.y_f32 = a.ydt == ZQ_OUT_F32;
  p.y_vec = (reinterpret_cast<uintptr_t>(a.y) & (p.y_f32 ? 15u : 7u)) == 0 && a.ldy % 4 == 0;
  p.q = a.q;
  p.s = a.s;
  p.ck = a.ck;
  p.cks = a.cks;
  p.act = a.act;
  p.pow2 = a.mode == ZQ_SCALE_M1;
  p.status = a.status;
  const int bm = few_width(a.M);
  const int64_t m_tiles64 = (a.M + bm - 1) / bm;
  if (m_tiles64 > 65535) return ZQ_ERR_SHAPE;
  const int m_tiles = static_cast<int>(m_tiles64);
  p.cluster = few_cluster(m_tiles64 * p.n_tiles, static_cast<int64_t>(p.segs) * p.kblocks, few_slots(bm, gated));
  if (static_cast<int64_t>(p.n_tiles) * p.cluster > 0x7FFFFFFF) return ZQ_ERR_SHAPE;
  CUtensorMap tw, tq;
  if (!make_code_map(&tw, a.b, static_cast<uint64_t>(a.K), static_cast<uint64_t>(a.N),
                     gated ? 2u : static_cast<uint64_t>(p.segs), kBlk))
    return ZQ_ERR_CUDA;
  if (raw)
    tq = tw;  // not used
  else if (!make_code_map(&tq, a.a, static_cast<uint64_t>(a.K), static_cast<uint64_t>(a.M), static_cast<uint64_t>(p.segs),
                          static_cast<uint32_t>(bm)))
    return ZQ_ERR_CUDA;
  if (gated) {
    if (raw) return launch_cfg<16, true, true>(tw, tq, p, m_tiles, st);
    if (bm == 16) return launch_cfg<16, true, false>(tw, tq, p, m_tiles, st);
    if (bm == 32) return launch_cfg<32, true, false>(tw, tq, p, m_tiles, st);
    return launch_cfg<64, true, false>(tw, tq, p, m_tiles, st);
  }
  if (raw) return launch_cfg<16, false, true>(tw, tq, p, m_tiles, st);
  if (bm == 16) return launch_cfg<16, false, false>(tw, tq, p, m_tiles, st);
  if (bm == 32) return launch_cfg<32, false, false>(tw, tq, p, m_tiles, st);
  return launch_cfg<64, false, false>(tw, tq, p, m_tiles, st);
}

}  // namespace fp8b
}  // namespace zq
