// Matrix product of E4M3 operands with block scales, many rows:
//   y[m, n] = sum_p sum_kb sa[p, kb, m] sb[p, n / 128, kb] * sum_{k in block kb} a[p, m, k] b[p, n, k]
// and, in the epilogue, the gated feed-forward block's product (kGated) and its gradient (kGatedBwd).
//
// The FP32 scales change every 128 elements of K, so the tensor core can add up one block only: its four MMAs fill
// one of two accumulators, and while the next block's MMAs fill the other, the epilogue warps take the finished one
// out of tensor memory, multiply it by the block's scale and add it to running sums in registers (in FP32: nothing
// is rounded between the blocks).
// Orientation: token rows are the lanes (the MMA's 128-row operand), so that a thread's scale sa * sb is ONE number
// for its 128 columns, and a promotion is one packed FMA per two columns.
// Tile: 128 tokens x 256 columns, two accumulators of 256 columns = all of tensor memory, eight epilogue warps
// with 128 running sums per thread.
//
// Warp roles: 0..7 epilogue (lane quarter warp % 4, column half warp / 4), 8 producer, 9 tensor memory and MMAs,
// 10 and 11 scales.
// Persistent: one CTA per SM walks the tiles, blockIdx.x, + gridDim.x, ..., token tiles in groups so that the CTAs
// running at one time share operands in L2.
#include "fp8_block.cuh"

namespace zq {
namespace fp8b {
namespace {

using gemm::named_bar_sync;

constexpr int kStages = 4;
constexpr int kTileM = 128, kTileN = 256;
constexpr int kABytes = kTileM * kBlk, kBBytes = kTileN * kBlk;
constexpr int kEpiWarps = 8, kEpiThreads = 256;
constexpr int kProducerWarp = 8, kMmaWarp = 9;
constexpr int kThreads = 384;  // three warpgroups; the two epilogue ones take registers over from the third
// 384 threads start with 168 registers each: 2 x 128 x 224 + 128 x 56 is what the block was given
constexpr int kEpiRegs = 224, kOtherRegs = 56;
static_assert(256 * kEpiRegs + 128 * kOtherRegs <= kThreads * 168, "register split");
constexpr int kStageBuf = 32 * 128;  // staging of one epilogue warp: 32 rows of 128 bytes
constexpr int kOffA = 0;
constexpr int kOffB = kOffA + kStages * kABytes;
constexpr int kOffStage = kOffB + kStages * kBBytes;
constexpr int kOffBars = kOffStage + kEpiWarps * kStageBuf;
constexpr int kNumBars = 2 * kStages + 4 + 1;
constexpr int kOffScale = kOffBars + ((kNumBars * 8 + 15) / 16) * 16;  // [2][2][128] scales of a K block: accumulator, half, row
constexpr int kOffMisc = kOffScale + 2 * 2 * kTileM * 4;
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

// Staged rows -> global memory, `rows` of them and `bytes` of each; ES: element size for the ragged and unaligned ends.
template <int PIECES, int ES>
__device__ __forceinline__ void store_rows(const uint4* buf, uint8_t* dst, int64_t ld_bytes, int rows, int bytes, bool vec,
                                           int lane) {
  __syncwarp();
  constexpr int kRowsPer = 32 / PIECES;
#pragma unroll
  for (int it = 0; it < PIECES; ++it) {
    const int r = it * kRowsPer + lane / PIECES, c = lane % PIECES;
    if (r < rows && c * 16 < bytes) {
      const uint4 v = stage_get(buf, r, c);
      uint8_t* d = dst + r * ld_bytes + c * 16;
      if (vec && c * 16 + 16 <= bytes) {
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
  __syncwarp();
}
// Accumulator columns [taddr, taddr + 16 * NCH) -> run (packed pairs) += s * columns, the next 16 in flight meanwhile.
// (Alone this takes 286 cycles for 128 rows x 256 columns, with 32 columns at a time 271, but those registers do not fit
// beside the sums.)
template <int NCH>
__device__ __forceinline__ void promote(uint32_t taddr, uint64_t* run, float s) {
  const uint64_t s2 = pack2(s, s);
  float nxt[16];
  tmem_ld16(taddr, nxt);
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    float v[16];
    tmem_ld_wait_regs<16>(nxt);
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = nxt[e];
    if (c + 1 < NCH) tmem_ld16(taddr + 16 * (c + 1), nxt);
#pragma unroll
    for (int e = 0; e < 8; ++e) run[c * 8 + e] = fma2(s2, pack2(v[2 * e], v[2 * e + 1]), run[c * 8 + e]);
  }
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

template <int KIND, int ACT, bool F32>
__global__ void __launch_bounds__(kThreads, 1)
fp8_block_gemm_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b, const P8 p) {
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kOffBars);
  uint64_t* full = bars;                 // [stages] the stage's copies landed           (MMA waits)
  uint64_t* empty = full + kStages;      // [stages] the MMAs that read it are done       (producer waits)
  uint64_t* acc_full = empty + kStages;  // [2] a K block's products are in the accumulator, its scales in shared memory (epilogue waits)
  uint64_t* acc_empty = acc_full + 2;    // [2] the epilogue warps have read it           (MMA waits)
  uint64_t* drain_bar = acc_empty + 2;
  float* s_scale = reinterpret_cast<float*>(smem + kOffScale);
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(smem + kOffMisc);
  volatile int* s_abort = reinterpret_cast<volatile int*>(smem + kOffMisc + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&acc_full[i], 3);  // the MMAs' commit and the two scale warps
      mbar_init(&acc_empty[i], kEpiWarps);
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
  if (warp == kMmaWarp) tmem_alloc(s_tmem, 512);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_base = *s_tmem;
  const bool ok_start = *s_abort == 0;
  const int tiles = p.m_tiles * p.n_tiles;
  const int kb_all = p.segs * p.kblocks;
  if (threadIdx.x == 0) pdl_launch_dependents();

  if (warp >= kEpiWarps) {
  regs_give<kOtherRegs>();
  if (warp == kProducerWarp) {
    if (ok_start) {
      const bool issuer = elect_one();
      pdl_wait();  // the codes may be the output of the kernel ahead in the stream
      int s = 0, issued = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int pos = blockIdx.x; ok && pos < tiles; pos += gridDim.x) {
        int mt, nt;
        tile_of(p, pos, mt, nt);
        for (int i = 0; i < kb_all; ++i) {
          if (issued >= kStages && !mbar_wait(&empty[s], ph ^ 1, s_abort)) {
            if (issuer) raise_error8(p.status, s_abort, kErrProducer8);
            ok = false;
            break;
          }
          if (issuer) {
            const int seg = KIND == kPlain ? i / p.kblocks : 0, k = (i - seg * p.kblocks) * kBlk;
            uint8_t* sb = smem + kOffB + s * kBBytes;
            mbar_arrive_expect_tx(&full[s], kABytes + kBBytes);
            tma_load_3d(smem + kOffA + s * kABytes, &tm_a, k, mt * kTileM, seg, &full[s]);
            if (KIND == kGated) {  // 128 rows of the gate, the same 128 of the up projection
              tma_load_3d(sb, &tm_b, k, nt * kBlk, 0, &full[s]);
              tma_load_3d(sb + kBBytes / 2, &tm_b, k, nt * kBlk, 1, &full[s]);
            } else {
              tma_load_3d(sb, &tm_b, k, nt * kTileN, seg, &full[s]);
              tma_load_3d(sb + kBBytes / 2, &tm_b, k, nt * kTileN + kBlk, seg, &full[s]);
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
      const uint64_t adesc0 = umma_desc_k128(smem_u32(smem + kOffA));
      const uint64_t bdesc0 = umma_desc_k128(smem_u32(smem + kOffB));
      const uint32_t idesc = umma_idesc_e4m3(kTileN);
      int s = 0;
      uint32_t ph = 0;
      bool failed = false;
      int count = 0;  // K blocks so far: block c goes to accumulator c % 2
      for (int pos = blockIdx.x; !failed && pos < tiles; pos += gridDim.x) {
        for (int i = 0; i < kb_all; ++i, ++count) {
          const int buf = count & 1;
          if ((count >= 2 && !mbar_wait(&acc_empty[buf], ((count >> 1) - 1) & 1, s_abort)) ||
              !mbar_wait(&full[s], ph, s_abort)) {
            failed = true;
            break;
          }
          tc_fence_after_sync();
          if (issuer) {
            const uint64_t ad = adesc0 + static_cast<uint64_t>((s * kABytes) >> 4);
            const uint64_t bd = bdesc0 + static_cast<uint64_t>((s * kBBytes) >> 4);
#pragma unroll
            for (int k = 0; k < kBlk / 32; ++k)
              umma_f8(tmem_base + buf * kTileN, ad + 2 * k, bd + 2 * k, idesc, k > 0 ? 1u : 0u);
            umma_commit(&empty[s]);
            umma_commit(&acc_full[buf]);
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
      if (issuer) umma_commit(drain_bar);
      uint32_t spin = 0;
      while (!mbar_try_wait(drain_bar, 0) && ++spin < kSpinLimit) {
      }
      __syncwarp();
    }
  } else if (ok_start) {
    // ---- scale warps: one per column half (kGated: gate, up).  The products of the rows' and the columns' scales of a
    // K block, a row per thread and quarter, loaded two blocks ahead: the epilogue warps, whose time is what the
    // kernel waits for, find them in shared memory (their own loads, one block ahead, cost 700 of 1500 cycles a block).
    constexpr int kAhead = 2;
    const int h = warp - kMmaWarp - 1;
    pdl_wait();
    int count = 0;
    bool ok = true;
    for (int pos = blockIdx.x; ok && pos < tiles; pos += gridDim.x) {
      int mt, nt;
      tile_of(p, pos, mt, nt);
      const int m0 = mt * kTileM + lane;
      // block 2 nt + h of the columns (kGated: block nt of part h)
      const int nb = KIND == kGated ? nt : min(2 * nt + h, p.nblocks - 1);
      const int64_t part = static_cast<int64_t>(p.nblocks) * p.kblocks;
      const float* sb = p.sb + static_cast<int64_t>(nb) * p.kblocks + (KIND == kGated ? h * part : 0);
      float a[kAhead][4], b[kAhead];
      auto fetch = [&](int i, int slot) {
        const int seg = KIND == kPlain && i >= p.kblocks ? 1 : 0;  // at most two segments
        b[slot] = __ldg(sb + seg * part + (i - seg * p.kblocks));
#pragma unroll
        for (int j = 0; j < 4; ++j)
          a[slot][j] = m0 + 32 * j < p.M ? __ldg(p.sa + static_cast<int64_t>(i) * p.M + m0 + 32 * j) : 0.0f;
      };
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (i < kb_all) fetch(i, i);
      for (int i0 = 0; ok && i0 < kb_all; i0 += kAhead) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          const int i = i0 + u;
          if (ok && i < kb_all) {
            const int buf = count & 1;
            if (count >= 2 && !mbar_wait_all(&acc_empty[buf], ((count >> 1) - 1) & 1, s_abort)) {
              if (lane == 0) raise_error8(p.status, s_abort, kErrScale8);
              ok = false;
            } else {
#pragma unroll
              for (int j = 0; j < 4; ++j) s_scale[(buf * 2 + h) * kTileM + 32 * j + lane] = a[u][j] * b[u];
              __syncwarp();
              if (lane == 0) mbar_arrive(&acc_full[buf]);
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
    regs_take<kEpiRegs>();
    const int quarter = warp & 3, half = warp >> 2;
    const int row = quarter * 32 + lane;
    const uint32_t lane_base = static_cast<uint32_t>(quarter * 32) << 16;
    uint4* buf = reinterpret_cast<uint4*>(smem + kOffStage + warp * kStageBuf);
    bool failed = !ok_start;
    int count = 0;
    pdl_wait();
    for (int pos = blockIdx.x; pos < tiles; pos += gridDim.x) {
      int mt, nt;
      tile_of(p, pos, mt, nt);
      const int m0 = mt * kTileM, m = m0 + row;
      const bool m_ok = m < p.M;
      uint64_t run[64];
#pragma unroll
      for (int e = 0; e < 64; ++e) run[e] = 0ull;
      for (int i = 0; i < kb_all; ++i, ++count) {
        const int b = count & 1;
        if (!failed && !mbar_wait_all(&acc_full[b], (count >> 1) & 1, s_abort)) {
          if (lane == 0) raise_error8(p.status, s_abort, kErrEpilogue8);
          failed = true;
        }
        tc_fence_after_sync();
        if (!failed) {
          const uint32_t t = tmem_base + b * kTileN + lane_base;
          const float* sc = s_scale + b * 2 * kTileM + row;
          const float s0 = sc[(KIND == kGated ? 0 : half) * kTileM], s1 = KIND == kGated ? sc[kTileM] : 0.0f;
          if (KIND == kGated) {
            promote<4>(t + half * 64, run, s0);
            promote<4>(t + 128 + half * 64, run + 32, s1);
          } else {
            promote<8>(t + half * 128, run, s0);
          }
        }
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0 && !failed) mbar_arrive(&acc_empty[b]);
      }
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
          store_rows<8, ES>(buf, yb + c * 128, p.ldy * ES, rows, min(128, (p.N - n0 - c * kCols) * ES), p.y_vec != 0, lane);
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
                           min(128, cols * 2), p.y_vec != 0, lane);
        }
      } else {  // kGatedBwd
        const int fb = 2 * nt + half;
        const int n0 = fb * kBlk, cols = p.N - n0;  // may be <= 0
        const int64_t MN = static_cast<int64_t>(p.M) * p.N, SM = static_cast<int64_t>(p.nblocks) * p.M;
        const bool any = cols > 0;
        float sg = 0.0f, su = 0.0f;
        if (any && m_ok) {
          sg = __ldg(p.cks + static_cast<int64_t>(fb) * p.M + m);
          su = __ldg(p.cks + SM + static_cast<int64_t>(fb) * p.M + m);
        }
        // a thread reads its own row's codes, 16 of g and of u at a time (both halves of a 32-byte sector in turn), the
        // next ones in flight; each pair of running sums (dh) is replaced by the bf16 pairs of dg and du
        const uint4* gp = reinterpret_cast<const uint4*>(p.ck + static_cast<int64_t>(m_ok ? m : 0) * p.N + (any ? n0 : 0));
        const uint4* up = reinterpret_cast<const uint4*>(reinterpret_cast<const uint8_t*>(gp) + MN);
        const int pieces = m_ok && any ? min(8, cols >> 4) : 0;
        uint4 gn = make_uint4(0u, 0u, 0u, 0u), un = gn;
        if (pieces > 0) {
          gn = __ldg(gp);
          un = __ldg(up);
        }
        uint32_t ag = 0u, au = 0u;
#pragma unroll 1
        for (int j = 0; j < 8; ++j) {
          const uint32_t gw[4] = {gn.x, gn.y, gn.z, gn.w}, uw[4] = {un.x, un.y, un.z, un.w};
          gn = un = make_uint4(0u, 0u, 0u, 0u);
          if (j + 1 < pieces) {
            gn = __ldg(gp + j + 1);
            un = __ldg(up + j + 1);
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float2 gv = decode2(static_cast<uint16_t>(gw[e >> 1] >> (16 * (e & 1))));
            const float2 vv = decode2(static_cast<uint16_t>(uw[e >> 1] >> (16 * (e & 1))));
            float d0, d1, a0, a1, b0, b1;
            unpack2(run[e], d0, d1);
            act_both<ACT>(gv.x * sg, a0, b0);
            act_both<ACT>(gv.y * sg, a1, b1);
            const uint32_t dg = pack_bf16(d0 * (vv.x * su) * b0, d1 * (vv.y * su) * b1);
            const uint32_t du = pack_bf16(d0 * a0, d1 * a1);
            ag = max(ag, max((dg << 16) & 0x7FFF0000u, dg & 0x7FFF0000u));
            au = max(au, max((du << 16) & 0x7FFF0000u, du & 0x7FFF0000u));
            run[e] = (static_cast<uint64_t>(du) << 32) | dg;
          }
          rotate<8>(run);
        }
        const float scg = block_scale(ag, p.pow2 != 0), scu = block_scale(au, p.pow2 != 0);
        if (any && m_ok && !failed) {
          p.s[static_cast<int64_t>(fb) * p.M + m] = scg;
          p.s[SM + static_cast<int64_t>(fb) * p.M + m] = scu;
        }
        // (dg, du) x (first, second 64 columns)
#pragma unroll 1
        for (int it = 0; it < 4; ++it) {
          const int part = it >> 1, c = it & 1;
          const float inv = block_inv(part ? scu : scg);
          uint32_t w[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) w[e] = part ? static_cast<uint32_t>(run[e] >> 32) : static_cast<uint32_t>(run[e]);
#pragma unroll
          for (int j = 0; j < 8; ++j) stage_put(buf, lane, j, make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]));
          const int64_t o = part * MN + static_cast<int64_t>(wm0) * p.N + n0 + 64 * c;
          store_rows<8, 2>(buf, static_cast<uint8_t*>(p.y) + o * 2, static_cast<int64_t>(p.N) * 2, rows,
                           min(128, (cols - 64 * c) * 2), true, lane);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t o4[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t lo = w[8 * j + 2 * e], hi = w[8 * j + 2 * e + 1];
              o4[e] = cast4(bf16_lo(lo), bf16_hi(lo), bf16_lo(hi), bf16_hi(hi), inv);
            }
            stage_put(buf, lane, j, make_uint4(o4[0], o4[1], o4[2], o4[3]));
          }
          store_rows<4, 1>(buf, p.q + o, p.N, rows, min(64, cols - 64 * c), true, lane);
          rotate<32>(run);
        }
      }
    }
  }

  tc_fence_before_sync();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after_sync();
    tmem_dealloc(tmem_base, 512);
  }
}

template <int KIND, int ACT, bool F32>
int launch_cfg(const CUtensorMap& ta, const CUtensorMap& tb, const P8& p, unsigned grid, cudaStream_t st) {
  static std::once_flag once;
  static cudaError_t attr = cudaSuccess;
  std::call_once(once, [] {
    attr = cudaFuncSetAttribute(fp8_block_gemm_kernel<KIND, ACT, F32>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
  });
  if (attr != cudaSuccess) return ZQ_ERR_CUDA;
  const cudaError_t e = launch_chained(fp8_block_gemm_kernel<KIND, ACT, F32>, dim3(grid), dim3(kThreads), kSmemBytes, st, false,
                                       ta, tb, p);
  count_launch();
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? ZQ_OK : ZQ_ERR_CUDA;
}

template <int KIND>
int launch_act(int act, const CUtensorMap& ta, const CUtensorMap& tb, const P8& p, unsigned grid, cudaStream_t st) {
  if (act == ZQ_ACT_SILU) return launch_cfg<KIND, ZQ_ACT_SILU, false>(ta, tb, p, grid, st);
  if (act == ZQ_ACT_GELU_TANH) return launch_cfg<KIND, ZQ_ACT_GELU_TANH, false>(ta, tb, p, grid, st);
  return launch_cfg<KIND, ZQ_ACT_RELU, false>(ta, tb, p, grid, st);
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
  p.m_tiles = static_cast<int>((a.M + kTileM - 1) / kTileM);
  p.n_tiles = a.kind == kGated ? p.nblocks : static_cast<int>((a.N + kTileN - 1) / kTileN);
  p.m_group = 16;
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
                     a.kind == kGated ? 2u : static_cast<uint64_t>(p.segs), kBlk))
    return ZQ_ERR_CUDA;
  const unsigned grid = static_cast<unsigned>(tiles < sm_count() ? tiles : sm_count());
  if (a.kind == kGated) return launch_act<kGated>(a.act, ta, tb, p, grid, st);
  if (a.kind == kGatedBwd) return launch_act<kGatedBwd>(a.act, ta, tb, p, grid, st);
  return a.ydt == ZQ_OUT_F32 ? launch_cfg<kPlain, ZQ_ACT_RELU, true>(ta, tb, p, grid, st)
                             : launch_cfg<kPlain, ZQ_ACT_RELU, false>(ta, tb, p, grid, st);
}

}  // namespace fp8b
}  // namespace zq
