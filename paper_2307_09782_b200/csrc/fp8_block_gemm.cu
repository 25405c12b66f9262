// Matrix product of E4M3 operands with block scales, many rows:
//   y[m, n] = sum_p sum_kb sa[p, kb, m] sb[p, n / 128, kb] * sum_{k in block kb} a[p, m, k] b[p, n, k]
// and, in the epilogue, the gated feed-forward block's product (kGated) and its gradient (kGatedBwd).
//
// The FP32 scales change every 128 elements of K, so the tensor core can add up one block only: its four MMAs fill
// one of two accumulators, and while the next block's MMAs fill the other, the epilogue warps take the finished one
// out of tensor memory, multiply it by the block's scale and add it to running sums in registers (in FP32, one rounding
// to nearest per block).
// Orientation: token rows are the lanes (the MMA's 128-row operand), so that a thread's scale sa * sb is ONE number
// for its 128 columns, and a promotion is one packed FMA per two columns.
// Tile: 128 tokens x 256 columns, two accumulators of 256 columns = all of tensor memory, eight epilogue warps with 128
// running sums per thread.  The two column halves (four warps each) give their accumulators back separately.
//
// What bounds it: the time of the epilogue warps, block by block.  Per K block the MMAs take 480 cycles; the promotion takes 460
// (286 alone; tensor memory serves both), and waits, fences and hand-over around it 350, one after the other: about 870 with two
// accumulators, 55 % of the tensor core's cycles.  A free accumulator is not what is missing: CTA pairs with four
// accumulators of 128 columns took the same time (with single CTAs MMAs of 128 columns read the token operand twice, 716
// cycles).  Tried and not faster either: sixteen epilogue warps (5 % faster without the gated epilogues, which then
// spill), polling instead of parked waits (slower).
// Spills: with 227 KB of shared memory the first-level cache holds none of them; 100 bytes per thread in the gradient's
// epilogue doubled the kernel's time.  The gated layer's epilogue has 12 - 16 bytes, the others none.
//
// Powers of two (MX): where all scales are (rule M1 on both sides, the caller's promise), they are E8M0 bytes that the
// tensor core multiplies in by itself, exactly: one accumulator takes all of K, nothing is promoted, and the epilogue, with
// the sums in registers, runs behind the next tile's MMAs.  A K block's scale stands for the four blocks of 32 that the MMA
// has in it; four warps write the bytes straight into tensor memory (tcgen05.st), stage by stage: no second operand
// format.  A pair of CTAs takes 256 tokens x 256 columns, so that a CTA loads half of the columns and has six stages.
// Measured, us, promotion -> MX (2048 tokens unless said): product 4096 -> 11008 93 -> 68; 8192 tokens 7168 -> 28672 1640 -> 1220
// (2.7 PFLOP/s); gated layer 4096 -> 11008 191 -> 144; gradient 170 -> 120, its epilogue bound.  What the steps gave, on the
// product: single CTAs 86; pairs 84; scales loaded four K blocks ahead and made bytes only when used 73 (with two ahead, the
// loads' latency set the pace); sums out of tensor memory with one wait 68.
// What bounds MX: at 2.7 PFLOP/s and the clock that the power cap leaves (1.6 - 1.7 GHz) the MMAs run about 2/3 of the time.
//
// Warp roles: 0..7 epilogue (lane quarter warp % 4, column half warp / 4), 8 producer, 9 tensor memory and MMAs (MX: the
// leader's for both CTAs), 10 and 11 scales, MX: 12..15 scales.
// Persistent: one CTA per SM (MX: one pair per two) walks the tiles, blockIdx.x, + gridDim.x, ..., token tiles in groups so that
// the CTAs running at one time share operands in L2.
#include "fp8_block.cuh"
#include "fp8_index.h"

namespace zq {
namespace fp8b {
namespace {

using gemm::named_bar_sync;

constexpr int kTileM = 128, kTileN = 256;  // of one CTA
constexpr int kEpiWarps = 8, kEpiThreads = 256;
constexpr int kProducerWarp = 8, kMmaWarp = 9;
constexpr int kThreads = 384;  // three warpgroups; the two epilogue ones take registers over from the third
// 384 threads start with 168 registers each; 2 x 128 x epilogue + 128 x other is what the block was given
// With block scales in the tensor core (MX) there are 512 threads with 128 registers each, and a second other warpgroup.
template <int KIND, bool MX>
struct Regs {
  static constexpr int kEpi = MX ? (KIND == kGatedBwd ? 208 : 192) : (KIND == kGatedBwd ? 232 : (KIND == kGated ? 216 : 224));
  static constexpr int kOther = MX ? (4 * 128 - 2 * kEpi) / 2 : 3 * 168 - 2 * kEpi;
};
constexpr int threads_of(bool mx) { return mx ? 512 : kThreads; }
constexpr int kSfWarp0 = 12;    // MX: 12..15 write the block scales, one per lane quarter of tensor memory
constexpr int kSfCol0 = kTileN; // MX: one accumulator, then 16 columns of scales per stage (4 rows' blocks, 8 columns' blocks)
constexpr int kStageBuf = 32 * 128;  // staging of one epilogue warp: 32 rows of 128 bytes
// MX: the two CTAs of a pair bring half of the columns each, so that more stages fit
__host__ __device__ constexpr int stages_of(bool mx) { return mx ? 6 : 4; }
constexpr int kABytes = kTileM * kBlk;
__host__ __device__ constexpr int b_bytes_of(bool mx) { return (mx ? kTileN / 2 : kTileN) * kBlk; }
constexpr int kOffStage = 4 * (kABytes + b_bytes_of(false));
static_assert(kOffStage == 6 * (kABytes + b_bytes_of(true)), "the stages of both forms take the same room");
constexpr int kOffBars = kOffStage + kEpiWarps * kStageBuf;
constexpr int kNumBars = 3 * 6 + 8 + 1;
constexpr int kOffScale = kOffBars + ((kNumBars * 8 + 15) / 16) * 16;  // [2 halves][2 accumulators][kScaleRow] scales of a K block
constexpr int kScaleRow = kTileM + 4;  // the rows' scales, then the columns' (kGated: gate, up)
constexpr int kOffMisc = kOffScale + 4 * kScaleRow * 4;
constexpr int kSmemBytes = kOffMisc + 16;
static_assert(kSmemBytes <= 227 * 1024, "shared memory");

enum { kErrProducer8 = 21, kErrMma8 = 22, kErrEpilogue8 = 23, kErrAlign8 = 24, kErrScale8 = 25 };

struct P8 {
  int M, N, K;
  int kblocks, segs;      // K blocks per segment, segments
  int nblocks;            // blocks of 128 along N
  int m_tiles, n_tiles, m_group;
  const float* sa;
  const float* sb;
  void* y;
  int64_t ldy;
  int y_vec;              // rows of y start on 16-byte boundaries
  uint8_t* q;
  float* s;
  uint8_t* ck;
  float* cks;
  int pow2;
  int* status;
};

__device__ __forceinline__ void tile_of(const P8& p, int pos, int& mt, int& nt) {
  const int per_group = p.m_group * p.n_tiles;
  const int g = pos / per_group, within = pos - g * per_group;
  const int gm = min(p.m_group, p.m_tiles - g * p.m_group);
  mt = g * p.m_group + within % gm;
  nt = within / gm;
}

// 32 rows (one per lane) x PIECES 16-byte pieces through the warp's staging buffer.  A row's pieces are stored
// XORed with its index, so that neither the writes (a row per lane) nor the reads (rows by groups of lanes) meet
// in a bank.
__device__ __forceinline__ void stage_put(uint4* buf, int lane, int piece, uint4 v) { buf[lane * 8 + (piece ^ (lane & 7))] = v; }
__device__ __forceinline__ uint4 stage_get(const uint4* buf, int row, int piece) { return buf[row * 8 + (piece ^ (row & 7))]; }

// Staged rows -> global memory, `rows` of them and `bytes` of each; ES: element size.  Rows that do not start on 16-byte
// boundaries are written row by row, neighbouring lanes neighbouring elements.
template <int PIECES, int ES>
__device__ __forceinline__ void store_rows(const uint4* buf, uint8_t* dst, int64_t ld_bytes, int rows, int bytes, bool vec,
                                           int lane) {
  __syncwarp();
  if (vec) {
    constexpr int kRowsPer = 32 / PIECES;
#pragma unroll
    for (int it = 0; it < PIECES; ++it) {
      const int r = it * kRowsPer + lane / PIECES, c = lane % PIECES;
      if (r < rows && c * 16 < bytes) {
        const uint4 v = stage_get(buf, r, c);
        uint8_t* d = dst + r * ld_bytes + c * 16;
        if (ES == 1 || c * 16 + 16 <= bytes) {  // (rows of codes are multiples of 16 bytes)
          *reinterpret_cast<uint4*>(d) = v;
        } else {
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int e = 0; e < 16 / ES; ++e)
            if (c * 16 + e * ES < bytes) {
              if (ES == 4) reinterpret_cast<uint32_t*>(d)[e] = w[e];
              if (ES == 2) reinterpret_cast<uint16_t*>(d)[e] = static_cast<uint16_t>(w[e >> 1] >> (16 * (e & 1)));
            }
        }
      }
    }
  } else if (ES > 1) {
#pragma unroll 1
    for (int r = 0; r < rows; ++r) {
      uint8_t* d = dst + r * ld_bytes;
#pragma unroll
      for (int o = 0; o < PIECES * 16; o += 32 * ES) {
        const int at = o + lane * ES;  // byte of the row
        const uint8_t* src = reinterpret_cast<const uint8_t*>(buf + r * 8 + ((at >> 4) ^ (r & 7))) + (at & 15);
        if (at < bytes) {
          if (ES == 4) *reinterpret_cast<uint32_t*>(d + at) = *reinterpret_cast<const uint32_t*>(src);
          if (ES == 2) *reinterpret_cast<uint16_t*>(d + at) = *reinterpret_cast<const uint16_t*>(src);
        }
      }
    }
  }
  __syncwarp();
}

// Accumulator columns -> run (packed pairs) += scale * columns, in pieces of 32 and 16 columns that alternate between two
// register buffers, so that one is in flight while the other is added up.  (Each wait drains everything in flight; pieces
// of 16 alone make eight waits of it, and two buffers of 32 do not fit beside 128 sums.)
template <int N>
__device__ __forceinline__ void add_piece(const float* v, uint64_t* run, uint64_t s2) {
#pragma unroll
  for (int e = 0; e < N / 2; ++e) run[e] = fma2(s2, pack2(v[2 * e], v[2 * e + 1]), run[e]);
}
// 128 columns: the first 64 with one scale, the others with another
__device__ __forceinline__ void promote(uint32_t t, uint64_t* run, float s0, float s1) {
  const uint64_t p0 = pack2(s0, s0), p1 = pack2(s1, s1);
  float a[32], b[16];
  tmem_ld32(t, a);
  tmem_ld_wait32(a);
  tmem_ld16(t + 32, b);
  add_piece<32>(a, run, p0);
  tmem_ld_wait_regs<16>(b);
  tmem_ld32(t + 48, a);
  add_piece<16>(b, run + 16, p0);
  tmem_ld_wait32(a);
  tmem_ld16(t + 80, b);
  add_piece<16>(a, run + 24, p0);
  add_piece<16>(a + 16, run + 32, p1);
  tmem_ld_wait_regs<16>(b);
  tmem_ld32(t + 96, a);
  add_piece<16>(b, run + 40, p1);
  tmem_ld_wait32(a);
  add_piece<32>(a, run + 48, p1);
}

// run[0 .. N) moves to the end: a rolled loop over N sums at a time works on run[0 .. N) and rotates, so that its code is
// fetched once instead of once per chunk (fully unrolled, the gradient epilogue took 35 us per tile for its instructions).
template <int N>
__device__ __forceinline__ void rotate(uint64_t* run) {
  uint64_t t[N];
#pragma unroll
  for (int e = 0; e < N; ++e) t[e] = run[e];
#pragma unroll
  for (int e = 0; e + N < 64; ++e) run[e] = run[e + N];
#pragma unroll
  for (int e = 0; e < N; ++e) run[64 - N + e] = t[e];
}

template <int KIND, int ACT, bool F32, bool MX>
__global__ void __launch_bounds__(threads_of(MX), 1)
fp8_block_gemm_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b, const P8 p) {
  constexpr int kStages = stages_of(MX), kBBytes = b_bytes_of(MX);
  constexpr int kOffA = 0, kOffB = kStages * kABytes;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kOffBars);
  uint64_t* full = bars;                 // [stages] the stage's copies landed; MX: both CTAs', the leader's counts (MMA waits)
  uint64_t* empty = full + kStages;      // [stages] the MMAs that read it are done       (producer waits)
  // per column half h and accumulator a, at 2 h + a:
  uint64_t* acc_full = empty + kStages;  // [4] a K block's products are in the accumulator, its scales in shared memory (epilogue waits)
  uint64_t* acc_empty = acc_full + 4;    // [4] the half's epilogue warps have read it (MMA, scale warp wait)
  uint64_t* sf_full = acc_empty + 4;     // [stages] MX: the stage's block scales are in tensor memory (MMA waits)
  uint64_t* drain_bar = sf_full + kStages;
  float* s_scale = reinterpret_cast<float*>(smem + kOffScale);
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(smem + kOffMisc);
  volatile int* s_abort = reinterpret_cast<volatile int*>(smem + kOffMisc + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
      mbar_init(&sf_full[i], 8);  // four warps of each CTA, the leader's counts
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(&acc_full[i], MX ? 1 : 2);  // the MMAs' commit and the half's scale warp
      mbar_init(&acc_empty[i], MX ? 2 * kEpiWarps : kEpiWarps / 2);  // MX: both CTAs' warps, the leader's counts
    }
    mbar_init(drain_bar, 1);
    *s_abort = 0;
    fence_mbar_init();
    if ((smem_u32(smem) & 1023u) != 0) raise_error8(p.status, s_abort, kErrAlign8);
  }
  if (warp == kProducerWarp && lane == 0) {
    prefetch_tensormap(&tm_a);
    prefetch_tensormap(&tm_b);
  }
  if (warp == kMmaWarp) {
    if (MX)
      tmem_alloc_pair(s_tmem, 512);
    else
      tmem_alloc(s_tmem, 512);
  }
  tc_fence_before_sync();
  if (MX)
    cluster_sync_all();  // both CTAs' barriers are initialized and their tensor memory is allocated
  else
    __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = *s_tmem;
  const bool ok_start = *s_abort == 0;
  // MX: a pair of CTAs takes a tile of 256 rows, 128 each
  const int rank = MX ? static_cast<int>(cluster_ctarank()) : 0;
  const int pos0 = MX ? static_cast<int>(blockIdx.x >> 1) : static_cast<int>(blockIdx.x);
  const int stride = MX ? static_cast<int>(gridDim.x >> 1) : static_cast<int>(gridDim.x);
  const int tiles = p.m_tiles * p.n_tiles;
  const int kb_all = p.segs * p.kblocks;
  if (threadIdx.x == 0) pdl_launch_dependents();

  if (warp >= kEpiWarps) {
  regs_give<Regs<KIND, MX>::kOther>();
  if (warp == kProducerWarp) {
    if (ok_start) {
      const bool issuer = elect_one();
      pdl_wait();  // the codes may be the output of the kernel ahead in the stream
      int s = 0, issued = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int pos = pos0; ok && pos < tiles; pos += stride) {
        int mt, nt;
        tile_of(p, pos, mt, nt);
        for (int i = 0; i < kb_all; ++i) {
          if (issued >= kStages && !mbar_wait(&empty[s], ph ^ 1, s_abort)) {
            if (issuer) raise_error8(p.status, s_abort, kErrProducer8);
            ok = false;
            break;
          }
          if (issuer) {
            const int seg = KIND == kPlain && i >= p.kblocks ? 1 : 0;  // at most two segments
            const int k = (i - seg * p.kblocks) * kBlk;
            uint8_t* sa = smem + kOffA + s * kABytes;
            uint8_t* sb = smem + kOffB + s * kBBytes;
            // the columns; kGated: per column half 64 of the gate and the same 64 of the up projection
            if (MX) {
              const uint32_t bar = map_to_rank(smem_u32(&full[s]), 0);
              if (rank == 0) mbar_arrive_expect_tx(&full[s], 2 * (kABytes + kBBytes));
              tma_load_3d_pair(sa, &tm_a, k, (2 * mt + rank) * kTileM, seg, bar);
              if (KIND == kGated) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                  tma_load_3d_pair(sb + h * (kBBytes / 2), &tm_b, k, nt * kBlk + rank * 64, h, bar);
              } else {
                tma_load_3d_pair(sb, &tm_b, k, nt * kTileN + rank * kBlk, seg, bar);
              }
            } else {
              mbar_arrive_expect_tx(&full[s], kABytes + kBBytes);
              tma_load_3d(sa, &tm_a, k, mt * kTileM, seg, &full[s]);
            }
            if (MX) {
            } else if (KIND == kGated) {
#pragma unroll
              for (int h = 0; h < 4; ++h)
                tma_load_3d(sb + h * (kBBytes / 4), &tm_b, k, nt * kBlk + (h >> 1) * 64, h & 1, &full[s]);
            } else {
              tma_load_3d(sb, &tm_b, k, nt * kTileN, seg, &full[s]);
            }
          }
          __syncwarp();
          ++issued;
          if (++s == kStages) {
            s = 0;
            ph ^= 1;
          }
        }
      }
      // never leave with copies still in flight (MX: the leader's barriers count them; the other CTA sees the stages that it
      // filled last released by the MMAs that read them)
      for (int i = max(0, issued - kStages); i < issued; ++i) {
        uint64_t* bar = (rank == 0 ? full : empty) + i % kStages;
        uint32_t spin = 0;
        while (!mbar_try_wait(bar, (i / kStages) & 1) && ++spin < kSpinLimit) {
        }
      }
    }
  } else if (warp == kMmaWarp) {
    if (ok_start && rank == 0) {
      const bool issuer = elect_one();
      const uint64_t adesc0 = umma_desc_k128(smem_u32(smem + kOffA));
      const uint64_t bdesc0 = umma_desc_k128(smem_u32(smem + kOffB));
      // MX: 256 rows, 128 in each CTA
      const uint32_t idesc = MX ? umma_idesc_mx_e4m3_e4m3(kTileN, 0, 0) + ((128u >> 4) << 24) : umma_idesc_e4m3(kTileN);
      int s = 0;
      uint32_t ph = 0;
      bool failed = false;
      int count = 0;  // K blocks so far: block c goes to accumulator c % 2
      int tile = 0;
      for (int pos = pos0; !failed && pos < tiles; pos += stride, ++tile) {
        for (int i = 0; i < kb_all; ++i, ++count) {
          const int buf = MX ? 0 : count & 1;
          const uint32_t free_ph = ((count >> 1) - 1) & 1;
          if (MX) {
            if ((i == 0 && tile > 0 && !mbar_wait(&acc_empty[0], (tile - 1) & 1, s_abort)) || !mbar_wait(&full[s], ph, s_abort) ||
                !mbar_wait(&sf_full[s], ph, s_abort)) {
              failed = true;
              break;
            }
          } else if (!mbar_wait(&full[s], ph, s_abort) || (count >= 2 && !mbar_wait(&acc_empty[buf], free_ph, s_abort)) ||
              (count >= 2 && !mbar_wait(&acc_empty[2 + buf], free_ph, s_abort))) {
            failed = true;
            break;
          }
          tc_fence_after_sync();
          const uint64_t ad = adesc0 + static_cast<uint64_t>((s * kABytes) >> 4);
          const uint64_t bd = bdesc0 + static_cast<uint64_t>((s * kBBytes) >> 4);
          const uint32_t d = tmem_base + buf * kTileN;
          if (MX) {
            if (issuer) {
              const uint32_t sf = tmem_base + kSfCol0 + 16 * s;
#pragma unroll
              for (int k = 0; k < kBlk / 32; ++k)
                umma_mxf8f6f4_pair(d, ad + 2 * k, bd + 2 * k, idesc, sf, sf + 4, (i > 0 || k > 0) ? 1u : 0u);
              if (i + 1 == kb_all) umma_commit_pair(&acc_full[0]);
              umma_commit_pair(&empty[s]);
            }
          } else if (issuer) {
#pragma unroll
            for (int k = 0; k < kBlk / 32; ++k) umma_f8(d, ad + 2 * k, bd + 2 * k, idesc, k > 0 ? 1u : 0u);
            umma_commit(&acc_full[buf]);
            umma_commit(&acc_full[2 + buf]);
            umma_commit(&empty[s]);
          }
          __syncwarp();
          if (++s == kStages) {
            s = 0;
            ph ^= 1;
          }
        }
      }
      if (failed && issuer) raise_error8(p.status, s_abort, kErrMma8);
      // tensor memory is released only when every MMA has completed, also where another role has given up
      if (issuer) {
        if (MX)
          umma_commit_pair(drain_bar);
        else
          umma_commit(drain_bar);
      }
    }
    if (ok_start) {  // (MX: in both CTAs, so that neither ends before the commit has arrived at it)
      uint32_t spin = 0;
      while (!mbar_try_wait(drain_bar, 0) && ++spin < kSpinLimit) {
      }
      __syncwarp();
    }
  } else if (MX) {
    if (ok_start && warp >= kSfWarp0) {
      // ---- block scales (powers of two) as E8M0 bytes, the same for the four blocks of 32 that a K block has: rows l, l + 32,
      // l + 64, l + 96 of the tokens in lane l of four columns, the columns' likewise in eight; every lane quarter of
      // tensor memory holds a copy, which its warp writes.  Loaded four blocks ahead.
      constexpr int kAhead = 4;
      pdl_wait();
      int s = 0, issued = 0;
      uint32_t ph = 0;
      bool ok = true;
      const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
      for (int pos = pos0; ok && pos < tiles; pos += stride) {
        int mt, nt;
        tile_of(p, pos, mt, nt);
        const int m0 = (2 * mt + rank) * kTileM + lane;
        const int64_t part = static_cast<int64_t>(p.nblocks) * p.kblocks;
        // kGated: columns 0..63 and 128..191 are the gate's, the others the up projection's
        const float* sb0 = p.sb + static_cast<int64_t>(KIND == kGated ? nt : 2 * nt) * p.kblocks;
        const float* sb1 = KIND == kGated ? sb0 + part : p.sb + static_cast<int64_t>(min(2 * nt + 1, p.nblocks - 1)) * p.kblocks;
        float a[kAhead][4], b[kAhead][2];  // (made bytes when they are used: nothing waits for a load before that)
        // The exponent's byte, which is E8M0, four times.  A scale that is no power of two, against the caller's promise, shows as NaN
        // (all bits set; infinities and NaN have that exponent anyway; a zero stands for 2^-127).
        auto byte4 = [](float v) {
          const uint32_t b = __float_as_uint(v);
          return (b & 0x807FFFFFu) != 0u ? 0xFFFFFFFFu : __byte_perm(b << 1, 0u, 0x3333);
        };
        const float* sa = p.sa + m0;
        auto fetch = [&](int i, int slot) {  // called for i = 0, 1, 2, ...
          if (KIND == kPlain && i == p.kblocks) {  // the second segment
            sb0 += part - p.kblocks;
            sb1 += part - p.kblocks;
          }
          b[slot][0] = load_chained(sb0++);
          b[slot][1] = load_chained(sb1++);
#pragma unroll
          for (int j = 0; j < 4; ++j) a[slot][j] = m0 + 32 * j < p.M ? load_chained(sa + 32 * j) : 1.0f;
          sa += p.M;
        };
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
          if (i < kb_all) fetch(i, i);
        for (int i0 = 0; ok && i0 < kb_all; i0 += kAhead) {
#pragma unroll
          for (int u = 0; u < kAhead; ++u) {
            const int i = i0 + u;
            if (ok && i < kb_all) {
              // (the MMAs that read the stage's scales last are those that release its shared memory)
              if (issued >= kStages && !mbar_wait_all(&empty[s], ph ^ 1, s_abort)) {
                if (lane == 0) raise_error8(p.status, s_abort, kErrScale8);
                ok = false;
              } else {
                tc_fence_after_sync();
                const uint32_t t = tmem_base + kSfCol0 + 16 * s + lane_base, b0 = byte4(b[u][0]), b1 = byte4(b[u][1]);
                tmem_st4(t, byte4(a[u][0]), byte4(a[u][1]), byte4(a[u][2]), byte4(a[u][3]));
                if (KIND == kGated) {
                  tmem_st4(t + 4, b0, b0, b1, b1);
                  tmem_st4(t + 8, b0, b0, b1, b1);
                } else {
                  tmem_st4(t + 4, b0, b0, b0, b0);
                  tmem_st4(t + 8, b1, b1, b1, b1);
                }
                tmem_st_wait();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive_tmem(&sf_full[s]);
                if (i + kAhead < kb_all) fetch(i + kAhead, u);
                ++issued;
                if (++s == kStages) {
                  s = 0;
                  ph ^= 1;
                }
              }
            }
          }
        }
      }
    }
  } else if (ok_start) {
    // ---- scale warps, one per column half: the scales of a K block's 128 rows and of its columns, loaded two blocks
    // ahead: the epilogue warps, whose time is what the kernel waits for, find them in shared memory (their own loads, one
    // block ahead, cost 700 of 1500 cycles a block).
    constexpr int kAhead = 2;
    const int h = warp - kMmaWarp - 1;
    pdl_wait();
    int count = 0;
    bool ok = true;
    for (int pos = pos0; ok && pos < tiles; pos += stride) {
      int mt, nt;
      tile_of(p, pos, mt, nt);
      const int m0 = mt * kTileM + lane;
      // columns: block 2 nt + h (kGated: lane 0 block nt of the gate, lane 1 of the up projection)
      const int64_t part = static_cast<int64_t>(p.nblocks) * p.kblocks;
      const float* sb = p.sb + static_cast<int64_t>(KIND == kGated ? nt : min(2 * nt + h, p.nblocks - 1)) * p.kblocks +
                        (KIND == kGated ? (lane & 1) * part : 0);
      float a[kAhead][4], b[kAhead];
      auto fetch = [&](int i, int slot) {
        const int seg = KIND == kPlain && i >= p.kblocks ? 1 : 0;  // at most two segments
        b[slot] = load_chained(sb + seg * part + (i - seg * p.kblocks));
#pragma unroll
        for (int j = 0; j < 4; ++j)
          a[slot][j] = m0 + 32 * j < p.M ? load_chained(p.sa + static_cast<int64_t>(i) * p.M + m0 + 32 * j) : 0.0f;
      };
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (i < kb_all) fetch(i, i);
      for (int i0 = 0; ok && i0 < kb_all; i0 += kAhead) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          const int i = i0 + u;
          if (ok && i < kb_all) {
            const int slot = 2 * h + (count & 1);
            if (count >= 2 && !mbar_wait_all(&acc_empty[slot], ((count >> 1) - 1) & 1, s_abort)) {
              if (lane == 0) raise_error8(p.status, s_abort, kErrScale8);
              ok = false;
            } else {
              float* d = s_scale + slot * kScaleRow;
#pragma unroll
              for (int j = 0; j < 4; ++j) d[32 * j + lane] = a[u][j];
              if (lane < 2) d[kTileM + lane] = b[u];
              __syncwarp();
              if (lane == 0) mbar_arrive(&acc_full[slot]);
              if (i + kAhead < kb_all) fetch(i + kAhead, u);
              ++count;
            }
          }
        }
      }
    }
  }
  } else {
    // ---- epilogue warps
    regs_take<Regs<KIND, MX>::kEpi>();
    const int quarter = warp & 3, half = warp >> 2;
    const int row = quarter * 32 + lane;
    const uint32_t lane_base = static_cast<uint32_t>(quarter * 32) << 16;
    uint4* buf = reinterpret_cast<uint4*>(smem + kOffStage + warp * kStageBuf);
    bool failed = !ok_start;
    int count = 0;
    pdl_wait();
    for (int pos = pos0; pos < tiles; pos += stride) {
      if (KIND == kGatedBwd) {
        // the checkpoint's codes that this tile's epilogue will read: on their way to L2 while the MMAs run
        int mt, nt;
        tile_of(p, pos, mt, nt);
        const int m = (MX ? 2 * mt + rank : mt) * kTileM + row, n0 = (2 * nt + half) * kBlk;
        if (m < p.M && n0 < p.N) {
          const uint8_t* g = p.ck + static_cast<int64_t>(m) * p.N + n0;
          const uint8_t* u = g + static_cast<int64_t>(p.M) * p.N;
          const int last = min(kBlk, p.N - n0) - 1;  // a row's codes can lie in two lines
          prefetch_l2(g);
          prefetch_l2(g + last);
          prefetch_l2(u);
          prefetch_l2(u + last);
        }
      }
      uint64_t run[64];
#pragma unroll
      for (int e = 0; e < 64; ++e) run[e] = 0ull;
      if (MX) {
        // the tile's sums, complete: into registers, and the MMAs of the next tile may begin
        if (!failed && !mbar_wait_all(&acc_full[0], count & 1, s_abort)) {
          if (lane == 0) raise_error8(p.status, s_abort, kErrEpilogue8);
          failed = true;
        }
        ++count;
        tc_fence_after_sync();
        if (!failed) {
          const uint32_t t = tmem_base + half * (kTileN / 2) + lane_base;
          if (KIND == kGatedBwd) {  // (its registers hold no more than 16 columns in flight; all at once, they spill: 138 us for 128)
#pragma unroll
            for (int c = 0; c < 8; ++c) {
              float v[16];
              tmem_ld16(t + 16 * c, v);
              tmem_ld_wait_regs<16>(v);
#pragma unroll
              for (int e = 0; e < 8; ++e) run[8 * c + e] = pack2(v[2 * e], v[2 * e + 1]);
            }
          } else {
            float v[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld32(t + 32 * c, v[c]);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              tmem_ld_wait32(v[c]);
#pragma unroll
              for (int e = 0; e < 16; ++e) run[16 * c + e] = pack2(v[c][2 * e], v[c][2 * e + 1]);
            }
          }
        }
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0 && !failed) mbar_arrive_tmem(&acc_empty[0]);
      }
      for (int i = 0; !MX && i < kb_all; ++i, ++count) {
        const int b = 2 * half + (count & 1);
        if (!failed && !mbar_wait_all(&acc_full[b], (count >> 1) & 1, s_abort)) {
          if (lane == 0) raise_error8(p.status, s_abort, kErrEpilogue8);
          failed = true;
        }
        tc_fence_after_sync();
        if (!failed) {
          const float* sc = s_scale + b * kScaleRow;
          const float sr = sc[row], s0 = sr * sc[kTileM], s1 = KIND == kGated ? sr * sc[kTileM + 1] : s0;
          promote(tmem_base + (count & 1) * kTileN + half * (kTileN / 2) + lane_base, run, s0, s1);
        }
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0 && !failed) mbar_arrive(&acc_empty[b]);
      }
      int mt, nt;
      tile_of(p, pos, mt, nt);
      const int m0 = (MX ? 2 * mt + rank : mt) * kTileM, m = m0 + row;
      const bool m_ok = m < p.M;
      const int wm0 = m0 + quarter * 32;
      const int rows = failed ? 0 : min(32, p.M - wm0);  // may be <= 0

      if (KIND == kPlain) {
        const int n0 = nt * kTileN + half * 128;
        constexpr int kCols = F32 ? 32 : 64, ES = F32 ? 4 : 2;
        uint8_t* yb = static_cast<uint8_t*>(p.y) + (static_cast<int64_t>(wm0) * p.ldy + n0) * ES;
#pragma unroll
        for (int c = 0; c < 128 / kCols; ++c) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            float f[8];
            uint4 v;
            if (F32) {
              unpack2(run[c * 16 + 2 * j], f[0], f[1]);
              unpack2(run[c * 16 + 2 * j + 1], f[2], f[3]);
              v = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) unpack2(run[c * 32 + 4 * j + e], f[2 * e], f[2 * e + 1]);
              v = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
            }
            stage_put(buf, lane, j, v);
          }
          store_rows<8, ES>(buf, yb + c * 128, p.ldy * ES, rows, row_bytes(p.N - n0 - c * kCols, kCols, ES), p.y_vec != 0, lane);
        }
      } else if (KIND == kGated) {
        const int n0 = nt * kBlk + half * 64;
        const int cols = p.N - n0;  // may be <= 0
        float* g = reinterpret_cast<float*>(run);
        float* u = g + 64;
        const int64_t MN = static_cast<int64_t>(p.M) * p.N, SM = static_cast<int64_t>(p.nblocks) * p.M;
        float* mine = reinterpret_cast<float*>(buf);
        const float* other = reinterpret_cast<const float*>(smem + kOffStage + (warp ^ 4) * kStageBuf);
        // columns beyond N hold zeros (the copy engine filled the operand with zeros): they do not move a maximum
        if (p.ck) {
          uint32_t ag = 0u, au = 0u;
#pragma unroll
          for (int e = 0; e < 64; ++e) {
            ag = max(ag, abs_bits(g[e]));
            au = max(au, abs_bits(u[e]));
          }
          mine[lane] = __uint_as_float(ag);
          mine[32 + lane] = __uint_as_float(au);
          named_bar_sync(1, kEpiThreads);
          ag = max(ag, __float_as_uint(other[lane]));
          au = max(au, __float_as_uint(other[32 + lane]));
          named_bar_sync(1, kEpiThreads);
#pragma unroll
          for (int part = 0; part < 2; ++part) {
            const float* v = part ? u : g;
            const float sc = block_scale(part ? au : ag, p.pow2 != 0), inv = block_inv(sc);
            if (m_ok && half == 0 && !failed) p.cks[part * SM + static_cast<int64_t>(nt) * p.M + m] = sc;
#pragma unroll
            for (int j = 0; j < 4; ++j)
              stage_put(buf, lane, j, make_uint4(cast4(v[16 * j], v[16 * j + 1], v[16 * j + 2], v[16 * j + 3], inv),
                                                 cast4(v[16 * j + 4], v[16 * j + 5], v[16 * j + 6], v[16 * j + 7], inv),
                                                 cast4(v[16 * j + 8], v[16 * j + 9], v[16 * j + 10], v[16 * j + 11], inv),
                                                 cast4(v[16 * j + 12], v[16 * j + 13], v[16 * j + 14], v[16 * j + 15], inv)));
            store_rows<4, 1>(buf, p.ck + part * MN + static_cast<int64_t>(wm0) * p.N + n0, p.N, rows, min(64, cols), true, lane);
          }
        }
        uint32_t ah = 0u;
#pragma unroll
        for (int e = 0; e < 64; ++e) {
          g[e] = act_value<ACT>(g[e]) * u[e];
          ah = max(ah, abs_bits(g[e]));
        }
        if (p.q) {
          mine[lane] = __uint_as_float(ah);
          named_bar_sync(1, kEpiThreads);
          ah = max(ah, __float_as_uint(other[lane]));
          named_bar_sync(1, kEpiThreads);
          const float sc = block_scale(ah, p.pow2 != 0), inv = block_inv(sc);
          if (m_ok && half == 0 && !failed) p.s[static_cast<int64_t>(nt) * p.M + m] = sc;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            stage_put(buf, lane, j, make_uint4(cast4(g[16 * j], g[16 * j + 1], g[16 * j + 2], g[16 * j + 3], inv),
                                               cast4(g[16 * j + 4], g[16 * j + 5], g[16 * j + 6], g[16 * j + 7], inv),
                                               cast4(g[16 * j + 8], g[16 * j + 9], g[16 * j + 10], g[16 * j + 11], inv),
                                               cast4(g[16 * j + 12], g[16 * j + 13], g[16 * j + 14], g[16 * j + 15], inv)));
          store_rows<4, 1>(buf, p.q + static_cast<int64_t>(wm0) * p.N + n0, p.N, rows, min(64, cols), true, lane);
        }
        if (p.y) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            stage_put(buf, lane, j, make_uint4(pack_bf16(g[8 * j], g[8 * j + 1]), pack_bf16(g[8 * j + 2], g[8 * j + 3]),
                                               pack_bf16(g[8 * j + 4], g[8 * j + 5]), pack_bf16(g[8 * j + 6], g[8 * j + 7])));
          store_rows<8, 2>(buf, static_cast<uint8_t*>(p.y) + (static_cast<int64_t>(wm0) * p.ldy + n0) * 2, p.ldy * 2, rows,
                           row_bytes(cols, 64, 2), p.y_vec != 0, lane);
        }
      } else {  // kGatedBwd
        const int fb = 2 * nt + half;
        const int n0 = fb * kBlk, cols = p.N - n0;  // may be <= 0
        const int64_t MN = static_cast<int64_t>(p.M) * p.N, SM = static_cast<int64_t>(p.nblocks) * p.M;
        const bool any = cols > 0;
        float sg = 0.0f, su = 0.0f;
        if (any && m_ok) {
          sg = load_chained(p.cks + static_cast<int64_t>(fb) * p.M + m);
          su = load_chained(p.cks + SM + static_cast<int64_t>(fb) * p.M + m);
        }
        // 32 columns at a time through the staging buffer (dh in FP32), so that eight lanes share a row: they read the
        // codes of g and u and write dg and du in whole sectors.  The bf16 pairs of dg and du take the place of the sums
        // they come from; a rolled loop, since its code unrolled is more than the instruction caches hold.
        const int rr = lane >> 3, cc = lane & 7;  // rows rr, rr + 4, ...; columns 4 cc .. 4 cc + 3 of the 32
        const uint8_t* ck = p.ck + static_cast<int64_t>(wm0) * p.N + n0 + 4 * cc;
        uint8_t* yd = static_cast<uint8_t*>(p.y) + (static_cast<int64_t>(wm0) * p.N + n0 + 4 * cc) * 2;
        // the next 32 columns' codes, on their way while these are worked on (MX: the MMAs do not wait for this epilogue, and
        // its warps have no registers to spare)
        uint32_t gn[8], un[8];
        auto fetch = [&](int c) {
#pragma unroll
          for (int it = 0; it < 8; ++it) {
            const int r = it * 4 + rr;
            gn[it] = un[it] = 0u;
            if (r < rows && 32 * c + 4 * cc < cols) {  // N is a multiple of 16: the four are inside or outside together
              gn[it] = load_chained(reinterpret_cast<const uint32_t*>(ck + static_cast<int64_t>(r) * p.N + 32 * c));
              un[it] = load_chained(reinterpret_cast<const uint32_t*>(ck + MN + static_cast<int64_t>(r) * p.N + 32 * c));
            }
          }
        };
        if (!MX) fetch(0);
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          if (MX) fetch(c);
          uint32_t gc[8], uc[8];
#pragma unroll
          for (int it = 0; it < 8; ++it) {
            gc[it] = gn[it];
            uc[it] = un[it];
          }
          if (!MX && c < 3) fetch(c + 1);
          __syncwarp();
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            float f[4];
            unpack2(run[2 * j], f[0], f[1]);
            unpack2(run[2 * j + 1], f[2], f[3]);
            stage_put(buf, lane, j, make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])));
          }
          __syncwarp();
#pragma unroll
          for (int it = 0; it < 8; ++it) {
            const int r = it * 4 + rr;
            const uint4 dv = stage_get(buf, r, cc);
            const uint64_t d[2] = {pack2(__uint_as_float(dv.x), __uint_as_float(dv.y)),
                                   pack2(__uint_as_float(dv.z), __uint_as_float(dv.w))};
            const uint64_t g_s = twice(__shfl_sync(0xFFFFFFFFu, sg, r)), u_s = twice(__shfl_sync(0xFFFFFFFFu, su, r));
            uint32_t dg[2], du[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float2 gv = decode2(static_cast<uint16_t>(gc[it] >> (16 * e)));
              const float2 vv = decode2(static_cast<uint16_t>(uc[it] >> (16 * e)));
              uint64_t a, b;
              act_both2<ACT>(mul2(pack2(gv.x, gv.y), g_s), a, b);
              float x0, x1;
              unpack2(mul2(mul2(d[e], mul2(pack2(vv.x, vv.y), u_s)), b), x0, x1);
              dg[e] = pack_bf16(x0, x1);
              unpack2(mul2(d[e], a), x0, x1);
              du[e] = pack_bf16(x0, x1);
            }
            run[2 * it] = (static_cast<uint64_t>(dg[1]) << 32) | dg[0];
            run[2 * it + 1] = (static_cast<uint64_t>(du[1]) << 32) | du[0];
            if (r < rows && 32 * c + 4 * cc < cols) {
              uint8_t* yr = yd + (static_cast<int64_t>(r) * p.N + 32 * c) * 2;
              *reinterpret_cast<uint64_t*>(yr) = run[2 * it];
              *reinterpret_cast<uint64_t*>(yr + MN * 2) = run[2 * it + 1];
            }
          }
          rotate<16>(run);
        }
        // The rows' maxima, from the finished pairs (kept up to date in the loop above they would be more registers than it
        // has): of bf16 numbers, whose absolute values order like their bits, g's in the lower half of a word, u's in the upper.
        uint32_t top[8];
#pragma unroll
        for (int it = 0; it < 8; ++it) {
          uint32_t ag = 0u, au = 0u;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const uint64_t vg = run[16 * c + 2 * it], vu = run[16 * c + 2 * it + 1];
            ag = max_u16x2(ag, max_u16x2(static_cast<uint32_t>(vg) & 0x7FFF7FFFu, static_cast<uint32_t>(vg >> 32) & 0x7FFF7FFFu));
            au = max_u16x2(au, max_u16x2(static_cast<uint32_t>(vu) & 0x7FFF7FFFu, static_cast<uint32_t>(vu >> 32) & 0x7FFF7FFFu));
          }
          top[it] = max_u16x2(__byte_perm(ag, au, 0x5410), __byte_perm(ag, au, 0x7632));
        }
        // over the eight lanes of a row: each exchange halves the rows that a lane still has, until lane cc has row 4 cc + rr,
        // whose two scales it computes and hands round
#pragma unroll
        for (int o = 4; o; o >>= 1) {
          const bool upper = (cc & o) != 0;
#pragma unroll
          for (int e = 0; e < o; ++e) {
            const uint32_t give = upper ? top[e] : top[e + o], keep = upper ? top[e + o] : top[e];
            top[e] = max_u16x2(keep, __shfl_xor_sync(0xFFFFFFFFu, give, o));
          }
        }
        const float scg = block_scale(top[0] << 16, p.pow2 != 0), scu = block_scale(top[0] & 0xFFFF0000u, p.pow2 != 0);
        if (any && 4 * cc + rr < rows) {
          float* sd = p.s + static_cast<int64_t>(fb) * p.M + wm0 + 4 * cc + rr;
          sd[0] = scg;
          sd[SM] = scu;
        }
        const float invg = block_inv(scg), invu = block_inv(scu);
        float ig[8], iu[8];
#pragma unroll
        for (int it = 0; it < 8; ++it) {
          ig[it] = __shfl_sync(0xFFFFFFFFu, invg, 8 * rr + it);
          iu[it] = __shfl_sync(0xFFFFFFFFu, invu, 8 * rr + it);
        }
        uint8_t* qd = p.q + static_cast<int64_t>(wm0) * p.N + n0 + 4 * cc;
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
#pragma unroll
          for (int it = 0; it < 8; ++it) {
            const int r = it * 4 + rr;
            const uint32_t g0 = static_cast<uint32_t>(run[2 * it]), g1 = static_cast<uint32_t>(run[2 * it] >> 32);
            const uint32_t u0 = static_cast<uint32_t>(run[2 * it + 1]), u1 = static_cast<uint32_t>(run[2 * it + 1] >> 32);
            const uint32_t qg = cast4(bf16_lo(g0), bf16_hi(g0), bf16_lo(g1), bf16_hi(g1), ig[it]);
            const uint32_t qu = cast4(bf16_lo(u0), bf16_hi(u0), bf16_lo(u1), bf16_hi(u1), iu[it]);
            if (r < rows && 32 * c + 4 * cc < cols) {
              uint8_t* qr = qd + static_cast<int64_t>(r) * p.N + 32 * c;
              *reinterpret_cast<uint32_t*>(qr) = qg;
              *reinterpret_cast<uint32_t*>(qr + MN) = qu;
            }
          }
          rotate<16>(run);
        }
      }
    }
  }

  tc_fence_before_sync();
  if (MX)
    cluster_sync_all();  // both CTAs are done with both CTAs' tensor memory and barriers
  else
    __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after_sync();
    if (MX)
      tmem_dealloc_pair(tmem_base, 512);
    else
      tmem_dealloc(tmem_base, 512);
  }
}

template <int KIND, int ACT, bool F32, bool MX>
int launch_cfg(const CUtensorMap& ta, const CUtensorMap& tb, const P8& p, cudaStream_t st) {
  static DeviceOnce once;
  if (!allow_shared_memory(once, fp8_block_gemm_kernel<KIND, ACT, F32, MX>, kSmemBytes)) return ZQ_ERR_CUDA;
  const int tiles = p.m_tiles * p.n_tiles, slots = MX ? sm_count() / 2 : sm_count();
  const unsigned grid = (MX ? 2u : 1u) * static_cast<unsigned>(tiles < slots ? tiles : slots);
  const cudaError_t e = launch_clustered(fp8_block_gemm_kernel<KIND, ACT, F32, MX>, dim3(grid), dim3(threads_of(MX)), kSmemBytes, st, MX ? 2 : 1,
                                       ta, tb, p);
  count_launch();
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? ZQ_OK : ZQ_ERR_CUDA;
}

template <int KIND, int ACT>
int launch_mx(bool mx, const CUtensorMap& ta, const CUtensorMap& tb, const P8& p, cudaStream_t st) {
  return mx ? launch_cfg<KIND, ACT, false, true>(ta, tb, p, st) : launch_cfg<KIND, ACT, false, false>(ta, tb, p, st);
}
template <int KIND>
int launch_act(int act, bool mx, const CUtensorMap& ta, const CUtensorMap& tb, const P8& p, cudaStream_t st) {
  if (act == ZQ_ACT_SILU) return launch_mx<KIND, ZQ_ACT_SILU>(mx, ta, tb, p, st);
  if (act == ZQ_ACT_GELU_TANH) return launch_mx<KIND, ZQ_ACT_GELU_TANH>(mx, ta, tb, p, st);
  return launch_mx<KIND, ZQ_ACT_RELU>(mx, ta, tb, p, st);
}

}  // namespace

int launch_block_gemm(const GemmArgs8& a, cudaStream_t st) {
  P8 p{};
  p.M = static_cast<int>(a.M);
  p.N = static_cast<int>(a.N);
  p.K = static_cast<int>(a.K);
  p.kblocks = static_cast<int>(blocks_of(a.K));
  p.segs = a.kind == kPlain ? a.parts : 1;
  p.nblocks = static_cast<int>(blocks_of(a.N));
  p.n_tiles = a.kind == kGated ? p.nblocks : static_cast<int>((a.N + kTileN - 1) / kTileN);
  // FP32 results keep the promotion: the tensor core rounds its running sum towards zero, about 1e-8 of it per block.  A
  // round of tiles takes the pairs 3/4 of the single CTAs' time, but the last pair of an odd number of token tiles has an idle
  // half.  Measured, us, single CTAs / pairs: 128 tokens, 7168 -> 28672 (1 and 2 rounds) 44 / 54; 384 tokens, 4096 -> 11008 (1 and
  // 2) 21 / 27; 256 tokens (1 and 1) 20.7 / 16.6; 1024 tokens, 4096 -> 4096 (1 and 1) 20.6 / 17.3; 640 tokens (2 and 2) 38.6 / 29.4.
  const int64_t mt1 = (a.M + kTileM - 1) / kTileM, mt2 = (mt1 + 1) / 2;
  const int64_t rounds1 = (mt1 * p.n_tiles + sm_count() - 1) / sm_count();
  const int64_t rounds2 = (mt2 * p.n_tiles + sm_count() / 2 - 1) / (sm_count() / 2);
  const bool mx = a.pow2_scales && a.ydt != ZQ_OUT_F32 && 3 * rounds2 <= 4 * rounds1;
  p.m_tiles = static_cast<int>(mx ? mt2 : mt1);
  p.m_group = mx ? 8 : 16;
  const int64_t tiles = static_cast<int64_t>(p.m_tiles) * p.n_tiles;
  if (tiles > 0x3FFFFFFF) return ZQ_ERR_SHAPE;
  p.sa = a.sa;
  p.sb = a.sb;
  p.y = a.y;
  p.ldy = a.ldy;
  p.y_vec = (reinterpret_cast<uintptr_t>(a.y) & 15u) == 0 && (a.ldy * (a.ydt == ZQ_OUT_F32 ? 4 : 2)) % 16 == 0;
  p.q = a.q;
  p.s = a.s;
  p.ck = a.ck;
  p.cks = a.cks;
  p.pow2 = a.mode == ZQ_SCALE_M1;
  p.status = a.status;
  CUtensorMap ta, tb;
  if (!make_code_map(&ta, a.a, static_cast<uint64_t>(a.K), static_cast<uint64_t>(a.M), static_cast<uint64_t>(p.segs), kTileM) ||
      !make_code_map(&tb, a.b, static_cast<uint64_t>(a.K), static_cast<uint64_t>(a.N),
                     a.kind == kGated ? 2u : static_cast<uint64_t>(p.segs), a.kind == kGated ? 64 : (mx ? kBlk : kTileN)))
    return ZQ_ERR_CUDA;
  if (a.kind == kGated) return launch_act<kGated>(a.act, mx, ta, tb, p, st);
  if (a.kind == kGatedBwd) return launch_act<kGatedBwd>(a.act, mx, ta, tb, p, st);
  return a.ydt == ZQ_OUT_F32 ? launch_cfg<kPlain, ZQ_ACT_RELU, true, false>(ta, tb, p, st)
                             : launch_mx<kPlain, ZQ_ACT_RELU>(mx, ta, tb, p, st);
}

}  // namespace fp8b
}  // namespace zq
