// Attention over the 8-bit cache where a sequence and cache head have few rows (new tokens x query heads of the head, up to 64):
// decoding, bf16 results.  Bound by the codes, which are read once.
//
// Keys' and values' codes go from memory to the tensor core as they are; what meets them is written as sums of E4M3 numbers, side
// by side in the columns:
//   S^T [128 tokens, 2 x rows] = K [tokens, D] q^T      q = q1 + q2 / 2^5, exact for bf16 features from 2^-14 of the row's largest on
//   O^T [D, 3 x rows] += V^T [D, tokens] P^T            P = P1 + P2 / 2^4 + P3 / 2^8, each the rest of the one before, with
//                                                       accumulators of its own: 12 bits, and something down to 2^-26 of the largest
// Tokens and features are the tensor core's 128 lanes, the rows its columns: more columns for more terms cost little.  (With the
// values widened to FP16 in shared memory and P in FP16 a tile of 32 KB moved 132 KB through shared memory, which takes 1050 of
// the 1370 cycles that its bytes take from memory, a 148th of the copy bandwidth: 64 sequences of up to 8192 tokens took 143 us.)
//
// Work: the (sequence, head, tile of 128 tokens) triples of the batch are dealt out evenly, as one contiguous range per CTA; the
// lengths are on the device, so each CTA finds its range itself.  A range is walked in segments (one per sequence and head), a
// segment in chunks of kTiles tiles: the scores of a whole chunk stay in tensor memory, two chunks in turn, and a chunk has
// accumulators of its own, so that a new maximum costs one multiplication per result and chunk in the epilogue's registers.
// Where several CTAs share a sequence and head, each leaves its sums, maximum and results in the workspace;
// attention_join_kernel adds them up in the order of the tiles.
//
// Warp roles: 0..7 softmax (thread = token), 8..11 queries and epilogue (thread = feature), 12 keys' copies, 13 values' copies,
// 14 MMAs, 15 the walk over the segments and the block scales.
#include "kv_attention.cuh"

namespace zq {
namespace kv {
namespace {

constexpr int kSoftmaxWarps = 8, kEpiWarp0 = 8, kKeyWarp = 12, kValueWarp = 13, kMmaWarp = 14, kWalkWarp = 15;
constexpr int kThreads = 16 * 32;
enum { kErrKeysA = 51, kErrValuesA = 52, kErrMmaA = 53, kErrWalkA = 54, kErrQueriesA = 55, kErrSoftmaxA = 56, kErrEpilogueA = 58, kErrAlignA = 59 };

struct P {
  Cache c;
  const __nv_bfloat16* q;
  int64_t ldq;
  int G;             // query heads of a cache head
  float scale_log2;  // sm_scale log2(e)
  int causal, window;
  void* out;
  int64_t ldo;
  float* lse;
  float* partial;    // [CTAs][2][RS (D + 2)]
  int4* shared;      // [CTAs] what begins in the CTA and goes on in the next: sequence, head, CTAs (0: nothing does)
  int* status;
};

// A segment, as the walk announces it to the others in shared memory (kSegs of them in turn).
struct alignas(16) Seg {
  int nt;           // tiles; 0: no more segments
  int tile0;        // the first of them, of the sequence's tiles of 128 tokens
  int L, n;         // tokens and new tokens of the sequence
  int b, h, first;  // sequence, head, the sequence's first row
  int flags;        // 1: begins with the first tile that the sequence and head have here; 2: ends with the last
};
constexpr int kSegs = 4;

// RS: rows that are worked on, at least those there are (the rest are computed from whatever lies there and not looked at: a jump
// past them costs more, in instructions fetched anew).
template <int D, int RS>
struct Cfg {
  static constexpr int kScoreCols = RS < 8 ? 16 : 2 * RS;                       // two terms of q (16 columns at the least)
  static constexpr int kProbCols = RS == 4 ? 16 : RS == 8 ? 32 : 3 * RS;        // three terms of P (multiples of 16)
  static constexpr int kProbRow = RS <= 8 ? 32 : RS == 16 ? 64 : RS == 32 ? 128 : 256;  // bytes of a token's probabilities
  static constexpr int kTiles = 128 / kScoreCols;                               // tiles of a chunk
  static constexpr int kOutBufs = RS == 64 ? 1 : 2;                             // accumulators: 512 columns, 256 of them scores
  static constexpr int kTileBytes = kTok * D;
  static constexpr int kProbBytes = kTok * kProbRow;                            // of a tile
  static constexpr int kOffProbs = 0;                                           // [2][kTiles]
  static constexpr int kOffQueries = kOffProbs + 2 * kTiles * kProbBytes;       // [3][kScoreCols rows of D]
  static constexpr int kOffScales = kOffQueries + 3 * kScoreCols * D;           // [2][kTiles][8] float4
  static constexpr int kOffRows = kOffScales + 2 * kTiles * 8 * 16;             // [3][RS] int4: factor, first and last token + 1 seen
  static constexpr int kOffMax = kOffRows + 3 * RS * 16;                        // [2][RS] maximum, [2][RS] factor of what came before
  static constexpr int kOffRed = kOffMax + 4 * RS * 4;                          // [RS][8] warps' maxima
  static constexpr int kOffSum = kOffRed + RS * 8 * 4;                          // [2] x ([RS][8] warps' sums, [RS] maxima)
  static constexpr int kOffSegs = kOffSum + 2 * RS * 9 * 4;                     // [kSegs]
  static constexpr int kOffMiss = kOffSegs + kSegs * 32;                        // [value slots] pages that were not copied
  static constexpr int kOffBars = kOffMiss + 64;
  static constexpr int kMaxBars = 72;
  static constexpr int kFixed = (kOffBars + kMaxBars * 8 + 36 * 8 + 1023) / 1024 * 1024;
  static constexpr int kSlots0 = (227 * 1024 - kFixed) / kTileBytes;
  static constexpr int kSlots = kSlots0 < 18 ? kSlots0 : 18;
  static constexpr int kKeySlots = (kSlots + 1) / 2, kValueSlots = kSlots / 2;
  static constexpr int kOffKeys = kFixed;
  static constexpr int kOffCodes = kOffKeys + kKeySlots * kTileBytes;
  static constexpr int kSmemBytes = kOffCodes + kValueSlots * kTileBytes;
  // slots; six pairs from s_full to o_empty; q, l, meet and drain; g
  static constexpr int kNumBars = 2 * kKeySlots + 2 * kValueSlots + 6 * 2 + 2 * 3 + 2 * 2 + 2 + 1 + 2 * kSegs;
  static_assert(kSmemBytes <= 227 * 1024 && kNumBars <= kMaxBars && kSlots >= 4 && kValueSlots <= 16, "shared memory");
  static_assert(256 + kOutBufs * kProbCols <= 512, "tensor memory");
};

// A sequence's part in this kernel: its rows and tiles (none where it has too many rows, or none).
struct Seq {
  int first, n, L;   // first row of the tensors, new tokens, tokens
  int tile0, tiles;  // tiles that some row sees (one at least, so that rows that see nothing are written)
};
__device__ __forceinline__ Seq seq_of(const P& p, int b) {
  Seq s;
  rows_of(p.c, b, s.first, s.n);
  s.L = max(load_chained(p.c.lens + b), 0);
  s.tile0 = s.tiles = 0;
  if (s.n > 0 && static_cast<int64_t>(s.n) * p.G <= kFewRows) {
    const int64_t lo = p.window > 0 ? static_cast<int64_t>(s.L) - s.n + 1 - p.window : 0;
    s.tile0 = lo > 0 ? static_cast<int>(lo / kTok) : 0;
    s.tiles = max(s.L / kTok + (s.L % kTok != 0) - s.tile0, 1);
  }
  return s;
}

// The walk over a CTA's units.
struct Walk {
  Seq s;
  int b, h, t;       // t: tile of the sequence's, from 0
  int64_t left;      // units left
  int nt;            // tiles of this segment
  __device__ __forceinline__ bool start(const P& p, const int64_t* range) {
    left = range[0];
    b = static_cast<int>(range[1]);
    if (left <= 0) return false;
    s = seq_of(p, b);
    h = static_cast<int>(range[2] / s.tiles);
    t = static_cast<int>(range[2] % s.tiles);
    nt = static_cast<int>(min(static_cast<int64_t>(s.tiles - t), left));
    return true;
  }
  __device__ __forceinline__ bool next(const P& p) {
    left -= nt;
    if (left <= 0) return false;
    t = 0;
    if (++h == p.c.H) {
      h = 0;
      do {
        if (++b >= p.c.B) return false;
        s = seq_of(p, b);
      } while (s.tiles == 0);
    }
    nt = static_cast<int>(min(static_cast<int64_t>(s.tiles), left));
    return true;
  }
};

template <int S>
__device__ __forceinline__ void load_scores(uint32_t taddr, float* v) {
  if (S == 4)
    tmem_ld4(taddr, v);
  else
    tmem_ld8(taddr, v);
}

// A ring position.
struct Ring {
  int i = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void step(int n) {
    if (++i == n) {
      i = 0;
      phase ^= 1;
    }
  }
};

template <int D, int RS>
__global__ void __launch_bounds__(kThreads, 1) attention_few_kernel(const __grid_constant__ CUtensorMap tm, const P p) {
  using C = Cfg<D, RS>;
  constexpr int kTiles = C::kTiles;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* bar = reinterpret_cast<uint64_t*>(smem + C::kOffBars);
  uint64_t* k_full = bar;                            // [key slots] a tile's keys have landed                  (MMA)
  uint64_t* k_empty = k_full + C::kKeySlots;         // their products are done                                (keys' copies)
  uint64_t* v_full = k_empty + C::kKeySlots;         // [value slots] a tile's values have landed              (MMA)
  uint64_t* v_empty = v_full + C::kValueSlots;       // their products are done                                (values' copies)
  uint64_t* s_full = v_empty + C::kValueSlots;                  // [2] scores of a chunk                                  (softmax)
  uint64_t* s_empty = s_full + 2;                    // [2] they have been used, with the scales               (MMA, walk)
  uint64_t* e_full = s_empty + 2;                    // [2] block scales of a chunk                            (softmax)
  uint64_t* p_full = e_full + 2;                     // [2] probabilities and row factors of a chunk           (MMA, epilogue)
  uint64_t* o_full = p_full + 2;                     // [2] results of a chunk                                 (epilogue)
  uint64_t* o_empty = o_full + 2;                    // [2] they are in registers                              (MMA, softmax)
  uint64_t* q_full = o_empty + 2;                    // [3] queries of a segment                               (MMA, softmax)
  uint64_t* q_empty = q_full + 3;                    // [3] nobody needs them any more                         (queries)
  uint64_t* l_full = q_empty + 3;                    // [2] sums of a segment                                  (epilogue)
  uint64_t* l_empty = l_full + 2;                    // [2] they have been read                                (softmax)
  uint64_t* meet = l_empty + 2;                      // [2] softmax warps that share rows
  uint64_t* g_full = meet + 2;                       // [kSegs] a segment is announced                         (all)
  uint64_t* g_empty = g_full + kSegs;                // [kSegs] everybody is through with it                   (walk)
  uint64_t* drain = g_empty + kSegs;
  const Seg* s_seg = reinterpret_cast<const Seg*>(smem + C::kOffSegs);
  int64_t* s_range = reinterpret_cast<int64_t*>(smem + C::kOffBars + C::kMaxBars * 8);  // units, first sequence, first unit in it
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(s_range + 3);
  volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);
  int64_t* s_scan = s_range + 4;  // [32]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < C::kKeySlots; ++i) {
      mbar_init(&k_full[i], 1);
      mbar_init(&k_empty[i], 1);
    }
    for (int i = 0; i < C::kValueSlots; ++i) {
      mbar_init(&v_full[i], 1);
      mbar_init(&v_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&s_empty[i], kSoftmaxWarps);
      mbar_init(&e_full[i], 1);
      mbar_init(&p_full[i], kSoftmaxWarps);
      mbar_init(&o_full[i], 1);
      mbar_init(&o_empty[i], 4);
      mbar_init(&l_full[i], kSoftmaxWarps);
      mbar_init(&l_empty[i], 4);
    }
    for (int i = 0; i < 3; ++i) {
      mbar_init(&q_full[i], 4);
      mbar_init(&q_empty[i], 1 + kSoftmaxWarps);
    }
    mbar_init(&meet[0], RS == 64 ? 4 : 8);
    mbar_init(&meet[1], 4);
    for (int i = 0; i < kSegs; ++i) {
      mbar_init(&g_full[i], 1);
      mbar_init(&g_empty[i], kThreads / 32 - 1);
    }
    mbar_init(drain, 1);
    *s_abort = 0;
    s_range[0] = 0;
    fence_mbar_init();
    if ((smem_u32(smem) & 1023u) != 0) fp8b::raise_error8(p.status, s_abort, kErrAlignA);
    prefetch_tensormap(&tm);
  }
  if (warp == kMmaWarp) tmem_alloc(s_tmem, 512);
  pdl_launch_dependents();
  pdl_wait();
  // ---- this CTA's range: units (H x tiles of a sequence) before each thread's sequences by a scan over the block
  {
    const int per = (p.c.B + kThreads - 1) / kThreads;
    const int b0 = min(static_cast<int>(threadIdx.x) * per, p.c.B), b1 = min(b0 + per, p.c.B);
    int64_t mine = 0;
    for (int b = b0; b < b1; ++b) mine += static_cast<int64_t>(seq_of(p, b).tiles) * p.c.H;
    int64_t incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t x = __shfl_up_sync(0xFFFFFFFFu, incl, o);
      if (lane >= o) incl += x;
    }
    if (lane == 31) s_scan[warp] = incl;
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    int64_t before = 0, total = 0;
    for (int w = 0; w < kThreads / 32; ++w) {
      if (w < warp) before += s_scan[w];
      total += s_scan[w];
    }
    const int64_t begin = before + incl - mine;
    const int64_t ctas = min(static_cast<int64_t>(gridDim.x), total);  // each of these has a unit at least
    const int64_t u0 = blockIdx.x < ctas ? total * blockIdx.x / ctas : 0, u1 = blockIdx.x < ctas ? total * (blockIdx.x + 1) / ctas : 0;
    if (u1 > u0 && begin <= u0 && u0 < begin + mine) {
      int64_t at = begin;
      int b = b0;
      for (;; ++b) {
        const int64_t n = static_cast<int64_t>(seq_of(p, b).tiles) * p.c.H;
        if (u0 < at + n) break;
        at += n;
      }
      s_range[1] = b;
      s_range[2] = u0 - at;
      s_range[0] = u1 - u0;
    }
    if (threadIdx.x == 0) s_scan[31] = total;
  }
  __syncthreads();
  const uint32_t tmem = *s_tmem;
  const bool any = *s_abort == 0 && s_range[0] > 0;
  // The next segment of a role: false behind the last one, and where something has failed.
  auto segment = [&](int seg, int& nt) {
    if (!fp8b::mbar_wait_all(&g_full[seg % kSegs], (seg / kSegs) & 1, s_abort)) return false;
    nt = s_seg[seg % kSegs].nt;
    return nt > 0;
  };
  auto done_with = [&](int seg) {  // a warp, converged
    if (lane == 0) mbar_arrive(&g_empty[seg % kSegs]);
  };

  if (warp == kKeyWarp || warp == kValueWarp) {
    // ---- copies: a lane per page of the tile
    const bool keys = warp == kKeyWarp;
    const int slots = keys ? C::kKeySlots : C::kValueSlots;
    uint64_t *full = keys ? k_full : v_full, *empty = keys ? k_empty : v_empty;
    uint8_t* to = smem + (keys ? C::kOffKeys : C::kOffCodes);
    const int per = kTok / p.c.page, page_bytes = p.c.page * D;
    uint32_t* miss = reinterpret_cast<uint32_t*>(smem + C::kOffMiss);
    Ring r;
    int issued = 0, nt;
    bool ok = any;
    for (int seg = 0; ok && segment(seg, nt); ++seg) {
      const Seg& g = s_seg[seg % kSegs];
      const int t0 = g.tile0, h = g.h;
      PageWalk pages;
      pages.start(p.c, g.b, g.L, t0 * per, lane);
      __syncwarp();
      done_with(seg);
      for (int j = 0; j < nt; ++j) {
        const int page = pages.get(p.c, (t0 + j) * per, lane);
        if (issued >= slots && !mbar_wait_warp(&empty[r.i], r.phase ^ 1, s_abort)) {
          if (lane == 0) fp8b::raise_error8(p.status, s_abort, keys ? kErrKeysA : kErrValuesA);
          ok = false;
          break;
        }
        const bool has = lane < per && page >= 0;
        const uint32_t n = __ballot_sync(0xFFFFFFFFu, has);
        if (lane == 0) {
          if (!keys) miss[r.i] = ~n & ((1u << per) - 1u);
          mbar_arrive_expect_tx(&full[r.i], __popc(n) * page_bytes);
        }
        __syncwarp();
        if (has) {
          uint8_t* dst = to + r.i * C::kTileBytes + lane * page_bytes;
          const int64_t block = block_at(p.c, page, keys ? 0 : 1, h);
          tma_load_3d(dst, &tm, 0, 0, static_cast<int>(block), &full[r.i]);
        }
        __syncwarp();
        ++issued;
        r.step(slots);
      }
    }
    // never leave with copies still in flight
    for (int i = max(0, issued - slots); i < issued; ++i) {
      uint32_t spin = 0;
      while (!mbar_try_wait(&full[i % slots], (i / slots) & 1) && ++spin < kSpinLimit) {
      }
    }
  } else if (warp == kMmaWarp) {
    const bool issuer = elect_one();
    const uint64_t kdesc = desc_rows<D>(smem_u32(smem + C::kOffKeys)), qdesc = desc_rows<D>(smem_u32(smem + C::kOffQueries));
    const uint64_t vdesc = desc_tokens<D>(smem_u32(smem + C::kOffCodes)), pdesc = desc_tokens<C::kProbRow>(smem_u32(smem + C::kOffProbs));
    const uint32_t sdesc_i = umma_idesc_e4m3(C::kScoreCols), odesc_i = idesc_e4m3_mn(C::kProbCols);
    const uint32_t* miss = reinterpret_cast<const uint32_t*>(smem + C::kOffMiss);
    Ring k, v;
    bool failed = false;
    int chunk = 0, seg = 0;
    // Results of tile j of a chunk: `left` tokens from the tile on.
    auto results = [&](int c, int j, bool last, int64_t left) {
      const int cb = c & 1, ob = C::kOutBufs == 2 ? cb : 0, before = c - C::kOutBufs;  // the chunk that had these columns before
      if (j == 0 && (!mbar_wait(&p_full[cb], (c >> 1) & 1, s_abort) || (before >= 0 && !mbar_wait(&o_empty[before & 1], (before >> 1) & 1, s_abort))))
        return false;
      if (!mbar_wait(&v_full[v.i], v.phase, s_abort)) return false;
      const uint32_t gone = miss[v.i];
      if (gone != 0u || left < kTok) {
        // what lies behind the last token, or in pages that were not copied, must not turn into NaN by a product with zero
        uint8_t* at = smem + C::kOffCodes + v.i * C::kTileBytes;
        const int from = static_cast<int>(max(left, static_cast<int64_t>(0)));
        for (int i = from * (D / 16) + lane; i < kTok * D / 16; i += 32) *reinterpret_cast<uint4*>(at + i * 16) = make_uint4(0u, 0u, 0u, 0u);
        for (uint32_t rest = gone; rest != 0u; rest &= rest - 1u) {
          uint8_t* page = at + (__ffs(rest) - 1) * p.c.page * D;
          for (int i = lane; i < p.c.page * D / 16; i += 32) *reinterpret_cast<uint4*>(page + i * 16) = make_uint4(0u, 0u, 0u, 0u);
        }
        fence_proxy_async_smem();
        __syncwarp();
      }
      tc_fence_after_sync();
      if (issuer) {
        const uint64_t ad = vdesc + static_cast<uint64_t>((v.i * C::kTileBytes) >> 4);
        const uint64_t bd = pdesc + static_cast<uint64_t>(((cb * kTiles + j) * C::kProbBytes) >> 4);
        constexpr int kRow = C::kProbRow < 128 ? C::kProbRow : 128;  // (256: two halves of 128 bytes)
#pragma unroll
        for (int s = 0; s < kTok / 32; ++s)  // 32 tokens further
          umma_f8(tmem + 256 + ob * C::kProbCols, ad + s * ((32 * D) >> 4), bd + s * ((32 * kRow) >> 4), odesc_i, (j > 0 || s > 0) ? 1u : 0u);
        umma_commit(&v_empty[v.i]);
        if (last) umma_commit(&o_full[cb]);
      }
      __syncwarp();
      v.step(C::kValueSlots);
      return true;
    };
    // Scores of a chunk go tile by tile in turn with the results of the chunk two before: keys and values are used up evenly, while
    // the softmax works on the chunk in between.
    int had[2] = {0, 0};          // tiles of the last chunk and the one before it
    int64_t had_left[2] = {0, 0};
    int nt_seg;
    for (; any && !failed && segment(seg, nt_seg); ++seg) {
      const int64_t left = s_seg[seg % kSegs].L - static_cast<int64_t>(s_seg[seg % kSegs].tile0) * kTok;
      __syncwarp();
      done_with(seg);
      for (int t = 0; t < nt_seg && !failed; t += kTiles, ++chunk) {
        const int nt = min(kTiles, nt_seg - t), cb = chunk & 1;
        int done = 0;  // of the results that are due
        if (t == 0 && !__all_sync(0xFFFFFFFFu, mbar_try_wait(&q_full[seg % 3], (seg / 3) & 1))) {
          // a new segment's queries are late: what is due does not wait for them
          for (; done < had[1] && !failed; ++done) failed = !results(chunk - 2, done, done + 1 == had[1], had_left[1] - static_cast<int64_t>(done) * kTok);
          if (!failed && !mbar_wait(&q_full[seg % 3], (seg / 3) & 1, s_abort)) failed = true;
        }
        if (!failed && chunk >= 2 && !mbar_wait(&s_empty[cb], ((chunk >> 1) - 1) & 1, s_abort)) failed = true;
        for (int j = 0; j < max(nt, had[1] - done) && !failed; ++j) {
          if (j < nt) {
            if (!mbar_wait(&k_full[k.i], k.phase, s_abort)) {
              failed = true;
              break;
            }
            tc_fence_after_sync();
            if (issuer) {
              const uint64_t ad = kdesc + static_cast<uint64_t>((k.i * C::kTileBytes) >> 4);
              const uint64_t bd = qdesc + static_cast<uint64_t>(((seg % 3) * C::kScoreCols * D) >> 4);
#pragma unroll
              for (int s = 0; s < D / 32; ++s) umma_f8(tmem + cb * 128 + j * C::kScoreCols, ad + s * 2, bd + s * 2, sdesc_i, s > 0 ? 1u : 0u);
              umma_commit(&k_empty[k.i]);
              if (j + 1 == nt) umma_commit(&s_full[cb]);
              if (t + j + 1 == nt_seg) umma_commit(&q_empty[seg % 3]);
            }
            __syncwarp();
            k.step(C::kKeySlots);
          }
          if (done == 0 && j < had[1] && !results(chunk - 2, j, j + 1 == had[1], had_left[1] - static_cast<int64_t>(j) * kTok)) failed = true;
        }
        had[1] = had[0];
        had_left[1] = had_left[0];
        had[0] = nt;
        had_left[0] = left - static_cast<int64_t>(t) * kTok;
      }
    }
    for (int c = 1; c >= 0; --c)  // the last two chunks
      for (int j = 0; j < had[c] && !failed; ++j) failed = !results(chunk - 1 - c, j, j + 1 == had[c], had_left[c] - static_cast<int64_t>(j) * kTok);
    if (failed && issuer) fp8b::raise_error8(p.status, s_abort, kErrMmaA);
    // tensor memory is released only when every MMA has completed, also where another role has given up
    if (issuer) umma_commit(drain);
    uint32_t spin = 0;
    while (!mbar_try_wait(drain, 0) && ++spin < kSpinLimit) {
    }
    __syncwarp();
  } else if (warp == kWalkWarp) {
    // ---- the walk: segments, and their chunks' block scales (a lane per 16 tokens), which are on their way one chunk ahead
    float4* table = reinterpret_cast<float4*>(smem + C::kOffScales);
    int seg = 0, chunk = 0;
    Walk w;  // of the segment announced last
    bool more = any && w.start(p, s_range), ok = more;
    // Announces segment `seg`, or that there are no more.  Segments are announced two ahead: the epilogue fetches queries ahead and
    // must not wait for chunks that wait for the epilogue.
    auto announce = [&] {
      if (seg >= kSegs && !mbar_wait_warp(&g_empty[seg % kSegs], (seg / kSegs - 1) & 1, s_abort)) return false;
      if (lane == 0) {
        Seg g{};
        if (more) {
          g.nt = w.nt, g.tile0 = w.s.tile0 + w.t, g.L = w.s.L, g.n = w.s.n, g.b = w.b, g.h = w.h, g.first = w.s.first;
          g.flags = (w.t == 0 ? 1 : 0) | (w.t + w.nt == w.s.tiles ? 2 : 0);
        }
        *const_cast<Seg*>(s_seg + seg % kSegs) = g;
        mbar_arrive(&g_full[seg % kSegs]);
      }
      __syncwarp();
      ++seg;
      return true;
    };
    // what the scales need of a segment: the one at hand and the two announced
    struct Place {
      int b, h, L, nt, tile0;
    };
    auto place = [&] { return more ? Place{w.b, w.h, w.s.L, w.nt, w.s.tile0 + w.t} : Place{0, 0, 0, 0, 0}; };
    auto advance = [&] {
      if (!more) return true;  // the end has been announced
      more = w.next(p);
      return announce();
    };
    constexpr int kMany = (kTiles * 8 + 31) / 32;
    RawScales next[kMany];
    auto load = [&](int b, int h, int tile, int L) {
#pragma unroll
      for (int i = 0; i < kMany; ++i)
        next[i] = load_scales(p.c, b, h, lane < kTiles * 8 ? static_cast<int64_t>(tile) * kTok + (i * 32 + lane) * 16 : L, L);
    };
    if (ok) {
      ok = announce();
      Place here = place();
      if (ok) ok = advance();
      Place after = place();
      load(here.b, here.h, here.tile0, here.L);
      while (ok && here.nt > 0) {
        ok = advance();
        const Place last = place();
        for (int t = 0; ok && t < here.nt; t += kTiles, ++chunk) {
          const int cb = chunk & 1;
          float4 e[kMany];
#pragma unroll
          for (int i = 0; i < kMany; ++i) e[i] = scale_entry(next[i]);
          if (t + kTiles < here.nt)
            load(here.b, here.h, here.tile0 + t + kTiles, here.L);
          else if (after.nt > 0)
            load(after.b, after.h, after.tile0, after.L);
          if (chunk >= 2 && !mbar_wait_warp(&s_empty[cb], ((chunk >> 1) - 1) & 1, s_abort)) ok = false;
          if (!ok) break;
#pragma unroll
          for (int i = 0; i < kMany; ++i)
            if (lane < kTiles * 8) table[cb * kTiles * 8 + i * 32 + lane] = e[i];
          __syncwarp();
          if (lane == 0) mbar_arrive(&e_full[cb]);
        }
        here = after;
        after = last;
      }
      if (!ok && lane == 0) fp8b::raise_error8(p.status, s_abort, kErrWalkA);
    }
  } else if (warp < kSoftmaxWarps) {
    // ---- softmax: thread = token of a tile.  Two groups of four warps take tiles in turn; with 64 rows (one tile per chunk)
    // they take half of its rows each.
    constexpr bool kHalves = RS == 64;
    constexpr int RR = kHalves ? 32 : RS;
    const int group = warp >> 2, r0 = kHalves ? group * 32 : 0;
    const int tok = (warp & 3) * 32 + lane;
    const int me = kHalves ? threadIdx.x & 127 : threadIdx.x;  // among those threads
    constexpr int S = RS < 8 ? RS : 8;        // rows at a time
    constexpr int kMine = kTiles > 1 ? kTiles / 2 : 1;  // tiles of a chunk
    const int j0 = kHalves ? 0 : group, dj = 2;
    const int red_i = kHalves ? warp & 3 : warp;
    const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const float4* table = reinterpret_cast<const float4*>(smem + C::kOffScales);
    float* s_max = reinterpret_cast<float*>(smem + C::kOffMax);
    float* s_red = reinterpret_cast<float*>(smem + C::kOffRed);
    float* s_sum = reinterpret_cast<float*>(smem + C::kOffSum);
    bool failed = !any;
    int chunk = 0, seg = 0;
    uint32_t met = 0;
    auto meet_others = [&] {  // the warps that share rows; a barrier whose wait is bounded
      uint64_t* at = &meet[kHalves ? group : 0];
      __syncwarp();
      if (lane == 0) mbar_arrive(at);
      return fp8b::mbar_wait_all(at, met++ & 1, s_abort);
    };
    int nt_seg;
    for (; !failed && segment(seg, nt_seg); ++seg) {
        const Seg& g = s_seg[seg % kSegs];
        const int rows = min(max(g.n * p.G - r0, 0), RR), tile0 = g.tile0;
        const float4* info = reinterpret_cast<const float4*>(smem + C::kOffRows) + (seg % 3) * RS + r0;
        if (!fp8b::mbar_wait_all(&q_full[seg % 3], (seg / 3) & 1, s_abort)) {
          failed = true;
          break;
        }
        float l[RR];
#pragma unroll
        for (int r = 0; r < RR; ++r) l[r] = 0.0f;
        float m_run = -INFINITY;  // of row r0 + me
        const int seen_to = p.causal ? g.L - g.n : g.L - 1, seen_from = p.window > 0 ? g.L - p.window : 0;
        __syncwarp();
        done_with(seg);
        for (int t = 0; t < nt_seg; t += kTiles, ++chunk) {
          const int nt = min(kTiles, nt_seg - t), cb = chunk & 1;
          const uint32_t parity = (chunk >> 1) & 1;
          float x[kMine][RR];
#pragma unroll
          for (int k = 0; k < kMine; ++k)
#pragma unroll
            for (int r = 0; r < RR; ++r) x[k][r] = -INFINITY;
          if (!fp8b::mbar_wait_all(&s_full[cb], parity, s_abort) || !fp8b::mbar_wait_all(&e_full[cb], parity, s_abort)) {
            failed = true;
            break;
          }
          tc_fence_after_sync();
          // scores of this thread's token of its tiles, x[k][r] for the k-th, plus the values' scale:
          // (a + b / 2^5) (row's factor) (keys' scale) + log2(values' scale)
          float inv[kMine];
#pragma unroll
          for (int k = 0; k < kMine; ++k) {
            const int j = j0 + k * dj;
            if (j >= nt) break;
            const float4 e = table[(cb * kTiles + j) * 8 + (tok >> 4)];
            inv[k] = e.z;
            const int tile = (tile0 + t + j) * kTok;
            const uint32_t from = tmem + lane_base + cb * 128 + j * C::kScoreCols + r0;
#pragma unroll
            for (int r = 0; r < RR; r += S) {
              float y[S];
              load_scores<S>(from + r, x[k] + r);
              load_scores<S>(from + RS + r, y);
              tmem_ld_wait_regs<S>(x[k] + r);
              tmem_ld_wait_regs<S>(y);
#pragma unroll
              for (int i = 0; i < S; i += 2) {
                float a, b;
                unpack2(fma2(pack2(y[i], y[i + 1]), fp8b::twice(1.0f / (1 << kRestBits)), pack2(x[k][r + i], x[k][r + i + 1])), a, b);
                x[k][r + i] = fmaf(a, info[r + i].x * e.x, e.y);
                x[k][r + i + 1] = fmaf(b, info[r + i + 1].x * e.x, e.y);
              }
            }
            // all of the tile is seen by all rows (the first row sees the fewest behind, the last the fewest before)
            if (!(tile + (kTok - 1) <= seen_to && tile >= seen_from)) {
#pragma unroll
              for (int r = 0; r < RR; ++r) {
                const float4 ri = info[r];
                if (tile + tok < __float_as_int(ri.y) || tile + tok >= __float_as_int(ri.z)) x[k][r] = -INFINITY;
              }
            }
          }
#pragma unroll
          for (int r = 0; r < RR; ++r) {
            float v = x[0][r];
#pragma unroll
            for (int k = 1; k < kMine; ++k) v = fmaxf(v, x[k][r]);
            v = warp_max(v);
            if (lane == 0) s_red[(r0 + r) * 8 + red_i] = v;
          }
          // the chunk two before is through the epilogue: its factors, and its probabilities, make room
          if (chunk >= 2 && !fp8b::mbar_wait_all(&o_empty[cb], ((chunk >> 1) - 1) & 1, s_abort)) failed = true;
          if (!meet_others()) failed = true;
          if (me < rows) {
            const float4* v = reinterpret_cast<const float4*>(s_red + (r0 + me) * 8);
            const float4 a = v[0];
            float m = fmaxf(fmaxf(m_run, fmaxf(a.x, a.y)), fmaxf(a.z, a.w));
            if (!kHalves) {
              const float4 b = v[1];
              m = fmaxf(m, fmaxf(fmaxf(b.x, b.y), fmaxf(b.z, b.w)));
            }
            const float safe = m == -INFINITY ? 0.0f : m;
            s_max[cb * RS + r0 + me] = kShift - safe;
            s_max[2 * RS + cb * RS + r0 + me] = exp2f(m_run - safe);
            m_run = m;
          }
          if (!meet_others()) failed = true;
          if (failed) break;
#pragma unroll
          for (int r = 0; r < RR; ++r) l[r] *= s_max[2 * RS + cb * RS + r0 + r];
#pragma unroll
          for (int k = 0; k < kMine; ++k) {
            const int j = j0 + k * dj;
            if (j >= nt) break;
            // the token's row of the operand: the first terms of all rows, the second, the third (RS bytes each)
            uint32_t term[3][RR / 4];
#pragma unroll
            for (int r = 0; r < RR; r += 4) {
              const float4 m = *reinterpret_cast<const float4*>(s_max + cb * RS + r0 + r);
              const float w0 = fp8b::sfu_ex2(x[k][r] + m.x), w1 = fp8b::sfu_ex2(x[k][r + 1] + m.y);
              const float w2 = fp8b::sfu_ex2(x[k][r + 2] + m.z), w3 = fp8b::sfu_ex2(x[k][r + 3] + m.w);
              l[r] = fmaf(w0, inv[k], l[r]);
              l[r + 1] = fmaf(w1, inv[k], l[r + 1]);
              l[r + 2] = fmaf(w2, inv[k], l[r + 2]);
              l[r + 3] = fmaf(w3, inv[k], l[r + 3]);
              uint32_t a[3], b[3];
              split3(pack_f16(w0, w1), a);
              split3(pack_f16(w2, w3), b);
#pragma unroll
              for (int i = 0; i < 3; ++i) term[i][r / 4] = a[i] | (b[i] << 16);
            }
            uint8_t* to = smem + C::kOffProbs + (cb * kTiles + j) * C::kProbBytes;
            if (RS == 4) {
              *reinterpret_cast<uint4*>(to + token_piece<C::kProbRow>(tok, 0)) = make_uint4(term[0][0], term[1][0], term[2][0], 0u);
            } else if (RS == 8) {
              *reinterpret_cast<uint4*>(to + token_piece<C::kProbRow>(tok, 0)) = make_uint4(term[0][0], term[0][RR / 4 - 1], term[1][0], term[1][RR / 4 - 1]);
              *reinterpret_cast<uint2*>(to + token_piece<C::kProbRow>(tok, 1)) = make_uint2(term[2][0], term[2][RR / 4 - 1]);
            } else {
#pragma unroll
              for (int i = 0; i < 3; ++i)
#pragma unroll
                for (int c = 0; c < RR / 16; ++c)
                  *reinterpret_cast<uint4*>(to + token_piece<C::kProbRow>(tok, (i * RS + r0) / 16 + c)) =
                      make_uint4(term[i][c * 4], term[i][c * 4 + 1], term[i][c * 4 + 2], term[i][c * 4 + 3]);
            }
          }
          fence_proxy_async_smem();
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(&s_empty[cb]);
            mbar_arrive(&p_full[cb]);
          }
        }
        if (failed) break;
        // sums of the segment
        if (seg >= 2 && !fp8b::mbar_wait_all(&l_empty[seg & 1], ((seg >> 1) - 1) & 1, s_abort)) {
          failed = true;
          break;
        }
        float* sums = s_sum + (seg & 1) * RS * 9;
#pragma unroll
        for (int r = 0; r < RR; ++r) {
          float v = l[r];
#pragma unroll
          for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
          if (lane == 0) sums[(r0 + r) * 8 + red_i] = v;
        }
        if (me < rows) sums[RS * 8 + r0 + me] = m_run;
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&l_full[seg & 1]);
          mbar_arrive(&q_empty[seg % 3]);
        }
    }
    if (failed && any && lane == 0) fp8b::raise_error8(p.status, s_abort, kErrSoftmaxA);
  } else {
    // ---- epilogue: thread = feature
    const int d = (warp & 3) * 32 + lane;
    const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const float* s_max = reinterpret_cast<const float*>(smem + C::kOffMax);
    const float* s_sum = reinterpret_cast<const float*>(smem + C::kOffSum);
    constexpr int S = RS < 8 ? RS : 8;
    const int64_t total = s_scan[31], ctas = min(static_cast<int64_t>(gridDim.x), total);
    bool failed = !any;
    int chunk = 0, seg = 0;
    int64_t unit = any ? total * blockIdx.x / ctas : 0;
    if (threadIdx.x == kEpiWarp0 * 32) p.shared[blockIdx.x] = make_int4(0, 0, 0, 0);
    // queries of segment `sg` (D / 8 lanes per row), once nobody needs those of the segment three before
    constexpr int kLanes = D / 8, kAtOnce = 128 / kLanes, kBatch = RS < 2 * kAtOnce ? 1 : 2;
    auto queries = [&](int sg) {
      const Seg& g = s_seg[sg % kSegs];
      const int rows = g.n * p.G, qb = sg % 3, i = threadIdx.x - kEpiWarp0 * 32;
      uint8_t* to = smem + C::kOffQueries + qb * C::kScoreCols * D;
      int4* info = reinterpret_cast<int4*>(smem + C::kOffRows) + qb * RS;
      for (int r0 = 0; r0 < rows; r0 += kAtOnce * kBatch) {
        uint4 x[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
          const int r = r0 + k * kAtOnce + i / kLanes;
          x[k] = make_uint4(0u, 0u, 0u, 0u);
          if (r < rows)
            x[k] = load_chained(reinterpret_cast<const uint4*>(p.q + (g.first + r / p.G) * p.ldq + (static_cast<int64_t>(g.h) * p.G + r % p.G) * D + (i % kLanes) * 8));
        }
        if (r0 == 0 && sg >= 3 && !fp8b::mbar_wait_all(&q_empty[qb], (sg / 3 - 1) & 1, s_abort)) return false;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
          const int r = r0 + k * kAtOnce + i / kLanes;
          uint32_t a = absmax_bits8(x[k]);
#pragma unroll
          for (int o = kLanes / 2; o; o >>= 1) a = max(a, __shfl_xor_sync(0xFFFFFFFFu, a, o));
          const RowScale s = row_scale(a);
          uint2 term[2];
          split8<true, 2>(x[k], s.up, term);
          if (r < rows) {
            const int piece = (i % kLanes) >> 1, half = (i & 1) * 8;
            *reinterpret_cast<uint2*>(to + row_piece<D>(r, piece) + half) = term[0];
            *reinterpret_cast<uint2*>(to + row_piece<D>(RS + r, piece) + half) = term[1];
            if (i % kLanes == 0) {
              const int64_t pos = static_cast<int64_t>(g.L) - g.n + r / p.G;
              const int64_t hi = p.causal ? min(pos + 1, static_cast<int64_t>(g.L)) : g.L;
              const int64_t lo = p.window > 0 ? pos + 1 - p.window : 0;
              info[r] = make_int4(__float_as_int(s.down * p.scale_log2), static_cast<int>(max(lo, static_cast<int64_t>(0))),
                                  static_cast<int>(max(hi, static_cast<int64_t>(0))), 0);
            }
          }
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&q_full[qb]);
      return true;
    };
    // segments `seg`, seg + 1, seg + 2 are announced, the queries of the first two on their way (or there are no more)
    int nt_seg = 0, nt_next = 0, nt_last = 0;
    if (!failed && segment(0, nt_seg)) {
      failed = !queries(0);
      if (!failed && segment(1, nt_next)) failed = !queries(1);
    }
    for (; !failed && nt_seg > 0; ++seg, nt_seg = nt_next, nt_next = nt_last) {
        const Seg& g = s_seg[seg % kSegs];
        const int rows = g.n * p.G, first = g.first, h = g.h, b = g.b, flags = g.flags;
        __syncwarp();
        done_with(seg);
        nt_last = 0;
        if (nt_next > 0 && segment(seg + 2, nt_last) && !queries(seg + 2)) {
          if (lane == 0) fp8b::raise_error8(p.status, s_abort, kErrQueriesA);
          failed = true;
          break;
        }
        float o[RS];
#pragma unroll
        for (int r = 0; r < RS; ++r) o[r] = 0.0f;
        for (int t = 0; t < nt_seg; t += kTiles, ++chunk) {
          const int cb = chunk & 1;
          const uint32_t parity = (chunk >> 1) & 1;
          if (!fp8b::mbar_wait_all(&p_full[cb], parity, s_abort) || !fp8b::mbar_wait_all(&o_full[cb], parity, s_abort)) {
            failed = true;
            break;
          }
          tc_fence_after_sync();
#pragma unroll
          for (int r = 0; r < RS; r += S) {
            float x[3][S];
#pragma unroll
            for (int i = 0; i < 3; ++i) load_scores<S>(tmem + lane_base + 256 + (C::kOutBufs == 2 ? cb : 0) * C::kProbCols + i * RS + r, x[i]);
#pragma unroll
            for (int i = 0; i < 3; ++i) tmem_ld_wait_regs<S>(x[i]);
#pragma unroll
            for (int i = 0; i < S; ++i)
              o[r + i] = fmaf(o[r + i], s_max[2 * RS + cb * RS + r + i], fmaf(x[2][i], 1.0f / 256.0f, fmaf(x[1][i], 1.0f / 16.0f, x[0][i])));
          }
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive(&o_empty[cb]);
        }
        if (failed || !fp8b::mbar_wait_all(&l_full[seg & 1], (seg >> 1) & 1, s_abort)) {
          failed = true;
          break;
        }
        // each warp sums every row up for itself, a row per lane (and the 32nd after), and hands its factor round
        const bool whole = flags == 3;
        float* part = p.partial + (static_cast<int64_t>(blockIdx.x) * 2 + (flags & 1)) * (RS * (D + 2));
        const float* sums = s_sum + (seg & 1) * RS * 9;
        float factor[(RS + 31) / 32];
#pragma unroll
        for (int k = 0; k < (RS + 31) / 32; ++k) {
          const int r = k * 32 + lane;
          factor[k] = 1.0f;
          if (r < rows) {
            const float4* v = reinterpret_cast<const float4*>(sums + r * 8);
            const float4 x = v[0];
            float sum = ((x.x + x.y) + x.z) + x.w;
            if (RS != 64) {
              const float4 y = v[1];
              sum = (((sum + y.x) + y.y) + y.z) + y.w;
            }
            const float m = sums[RS * 8 + r];
            if (whole) factor[k] = sum == 0.0f ? 0.0f : kCodeUnit / sum;
            if (warp == kEpiWarp0) {
              if (!whole) {
                part[RS * D + r] = sum;
                part[RS * D + RS + r] = m;
              } else if (p.lse) {
                p.lse[(first + r / p.G) * (static_cast<int64_t>(p.G) * p.c.H) + h * p.G + r % p.G] =
                    sum == 0.0f ? -INFINITY : (log2f(sum) + m + 8.0f - kShift) * (1.0f / kLog2e);
              }
            }
          }
        }
        // row by row without divisions, which would be most of the code: G rows of a token side by side, then the next token
        // (partial results: all rows one after the other)
        const int esize = whole ? 2 : 4, group = whole ? p.G : kFewRows;
        const int64_t jump = whole ? (p.ldo - static_cast<int64_t>(p.G - 1) * D) * esize : 0;
        uint8_t* to = whole ? static_cast<uint8_t*>(p.out) + (first * p.ldo + static_cast<int64_t>(h) * p.G * D + d) * esize
                            : reinterpret_cast<uint8_t*>(part + d);
        int left = group;
#pragma unroll
        for (int r = 0; r < RS; ++r) {
          const float v = o[r] * __shfl_sync(0xFFFFFFFFu, factor[r / 32], r & 31);
          if (r < rows && d < D) {
            if (esize == 4)
              *reinterpret_cast<float*>(to) = v;
            else
              *reinterpret_cast<__nv_bfloat16*>(to) = __float2bfloat16_rn(v);
          }
          const bool next = --left == 0;
          to += next ? jump : static_cast<int64_t>(D) * esize;
          if (next) left = group;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&l_empty[seg & 1]);
        if (flags == 1 && threadIdx.x == kEpiWarp0 * 32) {
          // goes on in the next CTAs, to the one whose range holds the last tile
          const int64_t last = unit + seq_of(p, b).tiles - 1;
          int64_t cta = last * ctas / total;
          while (total * (cta + 1) / ctas <= last) ++cta;
          p.shared[blockIdx.x] = make_int4(b, h, static_cast<int>(cta - blockIdx.x) + 1, 0);
        }
        unit += nt_seg;
    }
    if (failed && any && lane == 0) fp8b::raise_error8(p.status, s_abort, kErrEpilogueA);
  }

  tc_fence_before_sync();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, 512);
  }
}

// Results of sequences and heads that several CTAs share: blocks for each CTA that one begins in, a row at a time; a thread per
// feature and every fourth CTA.
template <int D, int RS>
__global__ void __launch_bounds__(4 * D) attention_join_kernel(const P p) {
  __shared__ float s_w[kMaxCtas];
  __shared__ float s_l;
  __shared__ float s_o[4][D];
  pdl_launch_dependents();
  pdl_wait();
  const int x = blockIdx.x;
  const uint4 shared = load_chained(reinterpret_cast<const uint4*>(p.shared + x));
  const int b = static_cast<int>(shared.x), h = static_cast<int>(shared.y), n = static_cast<int>(shared.z);
  if (n <= 1 || n > kMaxCtas) return;
  const Seq s = seq_of(p, b);
  const int rows = s.n * p.G;
  constexpr int64_t kPart = RS * (D + 2);
  // piece i: the first CTA's second place, the others' first
  auto part = [&](int i) { return p.partial + (static_cast<int64_t>(x + i) * 2 + (i == 0 ? 1 : 0)) * kPart; };
  for (int r = blockIdx.y; r < rows; r += gridDim.y) {
    __syncthreads();
    if (threadIdx.x < 32) {
      float m = -INFINITY;
      for (int i = threadIdx.x; i < n; i += 32) m = fmaxf(m, load_chained(part(i) + RS * D + RS + r));
      m = warp_max(m);
      float l = 0.0f;
      for (int i = threadIdx.x; i < n; i += 32) {
        const float mi = load_chained(part(i) + RS * D + RS + r);
        const float f = mi == -INFINITY ? 0.0f : exp2f(mi - m);
        s_w[i] = f;
        l = fmaf(f, load_chained(part(i) + RS * D + r), l);
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, o);
      if (threadIdx.x == 0) {
        s_l = l;
        const int64_t row = s.first + r / p.G;
        const int hq = h * p.G + r % p.G;
        if (p.lse) p.lse[row * (static_cast<int64_t>(p.G) * p.c.H) + hq] = l == 0.0f ? -INFINITY : (log2f(l) + m + 8.0f - kShift) * (1.0f / kLog2e);
      }
    }
    __syncthreads();
    const int d = threadIdx.x % D, k = threadIdx.x / D;
    float o = 0.0f;
#pragma unroll 4
    for (int i = k; i < n; i += 4) o = fmaf(s_w[i], load_chained(part(i) + r * D + d), o);
    s_o[k][d] = o;
    __syncthreads();
    if (k == 0) {
      o = s_o[0][d] + s_o[1][d] + s_o[2][d] + s_o[3][d];
      const float v = s_l == 0.0f ? 0.0f : o * kCodeUnit / s_l;
      const int64_t at = (s.first + r / p.G) * p.ldo + (static_cast<int64_t>(h) * p.G + r % p.G) * D + d;
      static_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(v);
    }
  }
}

template <int D, int RS>
int launch_cfg(const CUtensorMap& tm, const P& p, int grid, int max_rows, cudaStream_t st) {
  using C = Cfg<D, RS>;
  static DeviceOnce once;
  if (!allow_shared_memory(once, attention_few_kernel<D, RS>, C::kSmemBytes)) return ZQ_ERR_CUDA;
  cudaError_t e = launch_chained(attention_few_kernel<D, RS>, dim3(grid), dim3(kThreads), C::kSmemBytes, st, false, tm, p);
  count_launch();
  if (e != cudaSuccess) return ZQ_ERR_CUDA;
  e = launch_chained(attention_join_kernel<D, RS>, dim3(grid, max_rows < 16 ? max_rows : 16), dim3(4 * D), 0, st, false, p);
  count_launch();
  return e == cudaSuccess ? ZQ_OK : ZQ_ERR_CUDA;
}
template <int D>
int launch_rows(const CUtensorMap& tm, const P& p, int grid, int max_rows, cudaStream_t st) {
  if (max_rows <= 4) return launch_cfg<D, 4>(tm, p, grid, max_rows, st);
  if (max_rows <= 8) return launch_cfg<D, 8>(tm, p, grid, max_rows, st);
  if (max_rows <= 16) return launch_cfg<D, 16>(tm, p, grid, max_rows, st);
  if (max_rows <= 32) return launch_cfg<D, 32>(tm, p, grid, max_rows, st);
  return launch_cfg<D, 64>(tm, p, grid, max_rows, st);
}

}  // namespace

// Sums of two pieces per CTA, and what goes on in the next one.
size_t few_workspace_bytes(int64_t D) { return sizeof(float) * kMaxCtas * 2 * kFewRows * (D + 2) + sizeof(int4) * kMaxCtas; }

// max_rows: no sequence and head of this kernel has more rows.
int launch_attention_few(const AttnArgs& a, int max_rows, cudaStream_t st) {
  P p{};
  p.c = a.c;
  p.q = static_cast<const __nv_bfloat16*>(a.q), p.ldq = a.ldq, p.G = a.Hq / a.c.H;
  p.scale_log2 = a.sm_scale * kLog2e;
  p.causal = a.causal, p.window = a.window;
  p.out = a.out, p.ldo = a.ldo, p.lse = a.lse;
  uint8_t* ws = static_cast<uint8_t*>(a.workspace);
  p.status = reinterpret_cast<int*>(ws);
  p.shared = reinterpret_cast<int4*>(ws + kWsHeadBytes);
  p.partial = reinterpret_cast<float*>(p.shared + kMaxCtas);
  CUtensorMap tm;
  if (!make_page_map(&tm, a.c)) return ZQ_ERR_CUDA;
  const int sms = sm_count(), grid = sms < kMaxCtas ? sms : kMaxCtas;
  return a.c.D == 128 ? launch_rows<128>(tm, p, grid, max_rows, st) : launch_rows<64>(tm, p, grid, max_rows, st);
}

}  // namespace kv
}  // namespace zq
