// Attention over the 8-bit cache where a sequence and cache head have many rows (new tokens x query heads of the head, more than
// 64): prompts.  Bound by arithmetic: the tensor core's 4 D operations and one power of two per row and visible token.
//
//   S [128 rows, 128 tokens] = q K^T       q is the sum of an E4M3 and an E5M2 number (FP32 results: and of another), so two
//                                          products: the keys' codes go to the tensor core as they are, at the price of one FP16 product
//   O [128 rows, D] += P V                 FP16 x FP16 (FP32 results: P is the sum of two FP16 numbers, 11 bits are not enough for
//                                          them, and the sequences with few rows are here too); P from tensor memory, over the
//                                          scores it was made of; the values' codes are widened in shared memory, once for 256 rows
// Rows are the tensor core's lanes and a softmax thread's own: maxima and sums need no other thread.  A CTA works on two tiles of
// 128 rows in turn, each in steps of 64 tokens whose scores alternate between two places in tensor memory: the next step's are there
// when a softmax is done (with steps of 128 and one place it waited 2400 of 5800 cycles).  The running maximum only moves when a
// score exceeds it by more than kSlack (in powers of two; FP16 has the room): the accumulator is then multiplied by the row's own
// warp.
//
// The tensor core adds to an accumulator by cutting off (2^-23 of it at most for each product of 16 tokens; a tenth to a third of
// that, measured), so a long sum shrinks: with two terms of P by 1e-5 to 4e-5 over 8192 tokens.  For FP32 results the row's warp
// therefore adds it after kSumSteps steps, rounding to nearest, to a sum in the workspace (the CTA's own, which the L2 keeps), and
// the next product begins anew: 1e-6 to 3e-6 whatever the number of tokens, chunks of 777 tokens behind others 331 -> 343 us (16 steps:
// twice the error).  bf16 results, with one term, are left as they are: N tokens take N 2^-27 at most, below their rounding of 2^-9
// up to 2^18 tokens (and the loop would not be the same: prompt of 8191 tokens 696 -> 745 us).
//
// All items (sequence, 256 rows, head) stand in a row, each as long as its tokens and what it costs to begin and end one, and every CTA
// gets an equal part of the row (whole items in rounds: a prompt of 8191 tokens 732 us instead of 655).  An item that reaches over a
// boundary is worked on by the CTAs on both sides (by many, where there are few items), and attention_join_rows_kernel adds up their
// results in order.
//
// Warp roles: 0..3, 4..7 softmax and epilogue of the two tiles (thread = row), 8..11 queries and values (conversion), 12 copies, 13,
// 14 MMAs of the two tiles (one warp for both spent 1400 cycles a step on issuing, and waited for either tile in turn), 15 the
// walk over the items and the block scales.
#include "kv_attention.cuh"

namespace zq {
namespace kv {
namespace {

constexpr int kConvWarp0 = 8, kCopyWarp = 12, kMmaWarp = 13, kWalkWarp = 15;  // kMmaWarp + 1: of the second row tile
constexpr int kThreads = 512;
constexpr int kRows = 256;       // of an item
constexpr int kSegs = 4, kScaleSlots = 4;
constexpr int kStep = 64;        // tokens of a step
// What beginning and ending an item costs, in tokens: 13000 cycles, and the masked steps at its ends (a prompt of 8191 tokens took
// 824, 681, 658, 670 us with 256, 512, 768, 1024).
constexpr int kItemTokens = 768;
constexpr int kLeastTiles = 4;   // no item is split for less (chunks of 777 tokens behind others: 2 262 us, 4 255, 8 270)
constexpr float kSlack = 7.0f;   // 2^(kShift + kSlack) = 32768 fits FP16
enum { kErrCopyR = 61, kErrMmaR = 63, kErrWalkR = 64, kErrSoftmaxR = 65, kErrConvertR = 66, kErrAlignR = 67 };
// Registers per thread behind the set-up: softmax 184 (two warpgroups), converters and the others 72;
// 2 x 184 + 2 x 72 = 512, the four warpgroups' 4 x 128 at launch.

struct P {
  Cache c;
  const __nv_bfloat16* q;
  int64_t ldq;
  int G, boxes;
  float scale_log2;
  int causal, window;
  void* out;
  int64_t ldo;
  int f32;
  float* lse;
  int4* shared;    // [CTAs] the item that begins in the CTA and goes on in the next: sequence, number, 1 (0: none does); and of the
                   // item that came from the CTA before: 1 it goes on, 2 it ends here (0: none came)
  float* partial;  // [CTAs][2: what came from the CTA before, what goes on][256 (D + 2)]
  float* sums;     // [CTAs][256 D] of the item at hand (sum_at)
  int* status;
};

template <int D, bool EXACT>
struct Cfg {
  static constexpr int kSumSteps = 8;                                       // that an accumulator takes (EXACT)
  static constexpr int kTerms = EXACT ? 3 : 2;                              // of the queries
  static constexpr int kTileBytes = kTok * D;
  static constexpr int kValueBytes = kTok * D * 2;
  static constexpr int kKeySlots = EXACT && D == 128 ? 2 : 3, kValueSlots = 2;  // (what there is room for)
  static constexpr int kOffQueries = 0;                                     // [2 tiles][kTerms][128 rows of D]
  static constexpr int kOffValues = kOffQueries + 2 * kTerms * kTileBytes;  // [2] widened
  static constexpr int kOffKeys = kOffValues + 2 * kValueBytes;
  static constexpr int kOffCodes = kOffKeys + kKeySlots * kTileBytes;
  static constexpr int kOffScales = kOffCodes + kValueSlots * kTileBytes;   // [kScaleSlots][8] float4
  static constexpr int kOffRows = kOffScales + kScaleSlots * 8 * 16;        // [256] rows' factors
  static constexpr int kOffSegs = kOffRows + kRows * 4;
  static constexpr int kOffBars = kOffSegs + kSegs * 48;
  static constexpr int kMaxBars = 64;
  // slots; w; s, p and pv; q and r; e; g; drain
  static constexpr int kNumBars = 2 * kKeySlots + 2 * kValueSlots + 2 * 2 + 3 * 4 + 3 + 2 * kScaleSlots + 2 * kSegs + 2;
  static constexpr int kOffScan = kOffBars + kMaxBars * 8;                  // [16 + 4] 64-bit words, then two of 32
  static constexpr int kSmemBytes = kOffScan + 20 * 8 + 16;
  static_assert(kSmemBytes <= 227 * 1024 && kNumBars <= kMaxBars, "shared memory");
};

struct Seq {
  int first, n, L;
  int blocks;  // of 256 rows, 0 where the kernel for few rows takes the sequence
};
__device__ __forceinline__ Seq seq_of(const P& p, int b) {
  Seq s;
  rows_of(p.c, b, s.first, s.n);
  s.L = max(load_chained(p.c.lens + b), 0);
  const int64_t rows = static_cast<int64_t>(s.n) * p.G;
  s.blocks = rows > (p.f32 ? 0 : kFewRows) ? static_cast<int>((rows + kRows - 1) / kRows) : 0;
  return s;
}
// An item's tokens, in tiles: those that some of its rows see (at least one).
struct Item {
  int t0, nt;
  int half;  // 1: nobody sees the last tile's second half
};
__device__ __forceinline__ Item item_of(const P& p, const Seq& s, int64_t row0, int rows) {
  const int64_t p0 = static_cast<int64_t>(s.L) - s.n + row0 / p.G, p1 = static_cast<int64_t>(s.L) - s.n + (row0 + rows - 1) / p.G;
  const int64_t lo = p.window > 0 ? max(p0 + 1 - p.window, static_cast<int64_t>(0)) : 0;
  const int64_t hi = max(p.causal ? p1 + 1 : static_cast<int64_t>(s.L), static_cast<int64_t>(1));
  Item i;
  i.t0 = static_cast<int>(lo / kTok);
  i.nt = max(static_cast<int>((hi + kTok - 1) / kTok) - i.t0, 1);
  i.half = hi - static_cast<int64_t>(i.t0 + i.nt - 1) * kTok <= kStep ? 1 : 0;
  return i;
}
// Rows of a sequence's block k, counted from the last, which sees most.
__device__ __forceinline__ int64_t block_row0(const Seq& s, int k) { return static_cast<int64_t>(s.blocks - 1 - k) * kRows; }
__device__ __forceinline__ int block_rows(const P& p, const Seq& s, int64_t row0) {
  return static_cast<int>(min(static_cast<int64_t>(s.n) * p.G - row0, static_cast<int64_t>(kRows)));
}

// Lengths of a sequence's items in the row of all, in 1 / G tokens (a block's rows are 256 / G tokens), and sums of them in closed
// form: the blocks' tokens fall by 256 from one to the next, except where a window cuts them off.
struct Lengths {
  int64_t top, cap, item;
  __device__ __forceinline__ Lengths(const P& p, const Seq& s) {
    const int64_t all = static_cast<int64_t>(s.L) * p.G;
    item = kItemTokens * static_cast<int64_t>(p.G);
    cap = p.window > 0 ? min(static_cast<int64_t>(p.window) * p.G + kRows, all) : all;
    top = p.causal ? max(static_cast<int64_t>(s.L) - s.n, static_cast<int64_t>(0)) * p.G + static_cast<int64_t>(s.blocks) * kRows : kNone;
  }
  static constexpr int64_t kNone = int64_t{1} << 62;
  __device__ __forceinline__ int64_t of(int k) const { return (k == 0 ? cap : min(top - static_cast<int64_t>(k) * kRows, cap)) + item; }
  __device__ __forceinline__ int64_t before(int k) const {  // of the blocks 0 .. k - 1
    if (k == 0) return 0;
    // of 1 .. k - 1 the first `cut` are cut off
    int64_t cut = k - 1;
    if (top != kNone) cut = max(min((top - cap + kRows - 1) / kRows - 1, cut), static_cast<int64_t>(0));
    const int64_t rest = k - 1 - cut;
    int64_t sum = (1 + cut) * cap + k * item;
    if (rest > 0) sum += rest * top - rest * (k + cut) * (kRows / 2);
    return sum;
  }
};
__device__ __forceinline__ int64_t length_of(const P& p, const Seq& s) { return s.blocks > 0 ? Lengths(p, s).before(s.blocks) * p.c.H : 0; }
// Begin of a CTA's part of a row of that length.
__device__ __forceinline__ int64_t part_begin(int64_t total, int cta, int ctas) { return total / ctas * cta + total % ctas * cta / ctas; }

// A place in the row: a sequence, its item (block x heads + head; all of them: its end), and a tile of that.
struct Place {
  int b, k, tile;
};
__device__ __forceinline__ Place place_of(const P& p, const Seq& s, int b, int64_t at, int64_t share) {
  const Lengths w(p, s);
  int k = 0;
  for (int n = s.blocks; n > 1;) {  // the last block that begins at or before `at` is among the n from k on
    const int m = n / 2;
    if (w.before(k + m) * p.c.H <= at) {
      k += m;
      n -= m;
    } else {
      n = m;
    }
  }
  const int64_t length = w.of(k), in = at - w.before(k) * p.c.H;
  const int h = static_cast<int>(min(in / length, static_cast<int64_t>(p.c.H - 1)));
  const int64_t off = in - h * length;
  // too short a piece is left with its neighbour
  const int64_t least = min(share / 8, static_cast<int64_t>(kLeastTiles * kTok) * p.G);
  const int64_t row0 = block_row0(s, k);
  const int nt = item_of(p, s, row0, block_rows(p, s, row0)).nt;
  int tile = static_cast<int>(min(off * nt / length, static_cast<int64_t>(nt - 1)));
  int item = k * p.c.H + h;
  if (off < least) {
    tile = 0;
  } else if (length - off < least) {
    tile = 0;
    ++item;
  }
  return {b, item, tile};
}

struct alignas(16) Seg {
  int nt;            // tiles of tokens; 0: no more items
  int steps;         // steps of 64 tokens in them: 2 per tile, the last has one where nobody sees its second half
  int tile0;         // the first
  int L, n;
  int b, h, first;
  int row0, rows;    // first of the item's rows among the sequence's, and their number
  int part;          // place among the partial results, or -1
  int pad;
};
static_assert(sizeof(Seg) == 48, "Seg");

// Features d .. d + 3 of row r in a sum: rows side by side, as the threads are that have them.
__device__ __forceinline__ int64_t sum_at(int r, int d) { return (static_cast<int64_t>(d >> 2) * kRows + r) * 4; }

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

__device__ __forceinline__ void umma_f16_tmem_a(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// Results of a row: features f .. f + 15.
__device__ __forceinline__ void store16(const P& p, int64_t at, const float* v) {
  if (p.f32) {
    float4* o = reinterpret_cast<float4*>(static_cast<float*>(p.out) + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
  } else {
    uint4* o = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + at);
#pragma unroll
    for (int i = 0; i < 2; ++i)
      o[i] = make_uint4(fp8b::pack_bf16(v[8 * i], v[8 * i + 1]), fp8b::pack_bf16(v[8 * i + 2], v[8 * i + 3]),
                        fp8b::pack_bf16(v[8 * i + 4], v[8 * i + 5]), fp8b::pack_bf16(v[8 * i + 6], v[8 * i + 7]));
  }
}

// A softmax thread's step of scores x (its row, 64 tokens) -> probabilities in tensor memory.  `scales`: of its 4 groups of 16 tokens;
// `lo`, `hi`: tokens of the step that the row sees (looked at with MASK).  May move the row's reference m and multiplies l and,
// unless it begins anew (`first`), what is in the accumulator by the factor.
template <int D, bool EXACT, bool MASK, typename Wait>
__device__ __forceinline__ bool softmax_step(float* x, const float4* scales, float c, int lo, int hi, float& m, float& l, uint32_t probs,
                                             uint32_t acc, bool first, Wait accumulated) {
  float top = -INFINITY;
#pragma unroll
  for (int g = 0; g < kStep / 16; ++g) {
    const float4 e = scales[g];
    float w[4];  // (four at a time: one after the other a maximum takes 4 cycles each)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int at = g * 16 + i;
      if (MASK && (at < lo || at >= hi)) x[at] = -INFINITY;
      w[i & 3] = i < 4 ? x[at] : fmaxf(w[i & 3], x[at]);
    }
    const float v = fmaxf(fmaxf(w[0], w[1]), fmaxf(w[2], w[3]));
    top = fmaxf(top, fmaf(v, e.x * c, e.y));  // (0 x infinity where all is masked: NaN, which fmaxf drops)
  }
  // a row that has seen nothing yet takes the first maximum as it is: its sums are zero
  const bool move = top > m + kSlack || (m == -INFINITY && top > m);
  if (__any_sync(0xFFFFFFFFu, move)) {
    const float f = move && m > -INFINITY ? fp8b::sfu_ex2(m - top) : 1.0f;
    if (move) m = top;
    l *= f;
    if (!first && __any_sync(0xFFFFFFFFu, f != 1.0f)) {
      if (!accumulated()) return false;
      tc_fence_after_sync();
#pragma unroll 1
      for (int d = 0; d < D; d += 16) {
        float o[16];
        tmem_ld16(acc + d, o);
        tmem_ld_wait_regs<16>(o);
#pragma unroll
        for (int i = 0; i < 16; ++i) o[i] *= f;
        tmem_st16(acc + d, reinterpret_cast<const uint32_t*>(o));
      }
      tmem_st_wait();
    }
  }
  const float base = kShift - (m == -INFINITY ? 0.0f : m);
#pragma unroll
  for (int g = 0; g < kStep / 16; g += 2) {
    uint32_t h[16], r[EXACT ? 16 : 1];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float4 e = scales[g + k];
      const uint64_t f2 = fp8b::twice(e.x * c), a2 = fp8b::twice(e.y + base);
      uint64_t sum = 0ull;
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const int at = (g + k) * 16 + i;
        float a, b;
        unpack2(fma2(pack2(x[at], x[at + 1]), f2, a2), a, b);
        a = fp8b::sfu_ex2(a);
        b = fp8b::sfu_ex2(b);
        if (MASK) {
          if (at < lo || at >= hi) a = 0.0f;
          if (at + 1 < lo || at + 1 >= hi) b = 0.0f;
        }
        sum = add2(sum, pack2(a, b));
        h[k * 8 + i / 2] = pack_f16(a, b);
        if (EXACT) {
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[k * 8 + i / 2]));
          r[k * 8 + i / 2] = pack_f16(a - f.x, b - f.y);
        }
      }
      float s0, s1;
      unpack2(sum, s0, s1);
      l = fmaf(s0 + s1, e.z, l);
    }
    tmem_st16(probs + g * 8, h);
    if (EXACT) tmem_st16(probs + kStep / 2 + g * 8, r);
  }
  tmem_st_wait();
  return true;
}

// Results o of a row, features d .. d + 31, and the sum in the workspace times f.
__device__ __forceinline__ void add_sum32(float* o, const float* sum, int r, int d, float f) {
  float4 s[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) s[k] = *reinterpret_cast<const float4*>(sum + sum_at(r, d + 4 * k));
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    o[4 * k] = fmaf(s[k].x, f, o[4 * k]);
    o[4 * k + 1] = fmaf(s[k].y, f, o[4 * k + 1]);
    o[4 * k + 2] = fmaf(s[k].z, f, o[4 * k + 2]);
    o[4 * k + 3] = fmaf(s[k].w, f, o[4 * k + 3]);
  }
}
// What a sum with the reference m_sum is multiplied by where the reference is m.
__device__ __forceinline__ float carried(float m_sum, float m) { return m_sum == m ? 1.0f : fp8b::sfu_ex2(m_sum - m); }
// The accumulator of a row into its sum in the workspace (into nothing where there is none yet).  The features stand where the
// accumulator has them, until the item ends.
template <int D>
__device__ __forceinline__ void add_to_sum(uint32_t acc, float* sum, int r, bool has, float f) {
#pragma unroll 1
  for (int d = 0; d < D; d += 32) {
    float o[32];
    fp8b::tmem_ld32(acc + d, o);
    fp8b::tmem_ld_wait32(o);
    if (has) add_sum32(o, sum, r, d, f);
#pragma unroll
    for (int k = 0; k < 8; ++k) *reinterpret_cast<float4*>(sum + sum_at(r, d + 4 * k)) = make_float4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
  }
}

template <int D, bool EXACT>
__global__ void __launch_bounds__(kThreads, 1) attention_rows_kernel(const __grid_constant__ CUtensorMap tm, const __grid_constant__ CUtensorMap tm_q, const P p) {
  using C = Cfg<D, EXACT>;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* bar = reinterpret_cast<uint64_t*>(smem + C::kOffBars);
  uint64_t* k_full = bar;                          // [key slots] a tile's keys have landed                 (MMA)
  uint64_t* k_empty = k_full + C::kKeySlots;       // their products are done                               (copies)
  uint64_t* v_full = k_empty + C::kKeySlots;       // [value slots] a tile's values have landed             (converters)
  uint64_t* v_empty = v_full + C::kValueSlots;     // they are widened                                      (copies)
  uint64_t* w_full = v_empty + C::kValueSlots;     // [2] widened values                                    (MMA)
  uint64_t* w_empty = w_full + 2;                  // [2] their products are done                           (converters)
  uint64_t* s_full = w_empty + 2;                  // [2 row tiles][2] scores                               (softmax)
  // (a barrier for each place: a warp can be a step ahead of another, or of the products)
  uint64_t* p_full = s_full + 4;                   // [2][2] probabilities, the accumulator up to date      (MMA)
  uint64_t* pv_done = p_full + 4;                  // [2][2] they have been multiplied                      (MMA, softmax)
  uint64_t* q_full = pv_done + 4;                  // an item's queries                                     (MMA, softmax)
  uint64_t* q_empty = q_full + 1;                  // nobody needs them any more                            (converters)
  uint64_t* r_full = q_empty + 1;                  // an item's queries have landed                         (converters)
  uint64_t* e_full = r_full + 1;                   // [scale slots] a tile's block scales                   (softmax)
  uint64_t* e_empty = e_full + kScaleSlots;        // they have been used                                   (walk)
  uint64_t* g_full = e_empty + kScaleSlots;        // [kSegs] an item is announced                          (all)
  uint64_t* g_empty = g_full + kSegs;              // [kSegs] everybody is through with it                  (walk)
  uint64_t* drain = g_empty + kSegs;               // [2]
  int64_t* s_scan = reinterpret_cast<int64_t*>(smem + C::kOffScan);
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(s_scan + 20);
  volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);
  Seg* s_seg = reinterpret_cast<Seg*>(smem + C::kOffSegs);
  float* s_rows = reinterpret_cast<float*>(smem + C::kOffRows);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < C::kKeySlots; ++i) {
      mbar_init(&k_full[i], 1);
      mbar_init(&k_empty[i], 2);
    }
    for (int i = 0; i < C::kValueSlots; ++i) {
      mbar_init(&v_full[i], 1);
      mbar_init(&v_empty[i], 4);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&w_full[i], 4);
      mbar_init(&w_empty[i], 2);
      mbar_init(&s_full[2 * i], 1);
      mbar_init(&s_full[2 * i + 1], 1);
      mbar_init(&p_full[2 * i], 4);
      mbar_init(&p_full[2 * i + 1], 4);
      mbar_init(&pv_done[2 * i], 1);
      mbar_init(&pv_done[2 * i + 1], 1);
    }
    mbar_init(q_full, 4);
    mbar_init(q_empty, 2 + 8);
    mbar_init(r_full, 1);
    for (int i = 0; i < kScaleSlots; ++i) {
      mbar_init(&e_full[i], 1);
      mbar_init(&e_empty[i], 8);
    }
    for (int i = 0; i < kSegs; ++i) {
      mbar_init(&g_full[i], 1);
      mbar_init(&g_empty[i], kThreads / 32 - 1);
    }
    mbar_init(&drain[0], 1);
    mbar_init(&drain[1], 1);
    *s_abort = 0;
    fence_mbar_init();
    if ((smem_u32(smem) & 1023u) != 0) fp8b::raise_error8(p.status, s_abort, kErrAlignR);
    prefetch_tensormap(&tm);
    if (p.boxes) prefetch_tensormap(&tm_q);
  }
  if (warp == kMmaWarp) tmem_alloc(s_tmem, 512);
  pdl_launch_dependents();
  pdl_wait();
  // ---- lengths of the items before each thread's sequences, by a scan over the block; the threads that have them leave the ends of
  // this CTA's part
  {
    const int per = (p.c.B + kThreads - 1) / kThreads;
    const int b0 = min(static_cast<int>(threadIdx.x) * per, p.c.B), b1 = min(b0 + per, p.c.B);
    int64_t mine = 0;
    for (int b = b0; b < b1; ++b) mine += length_of(p, seq_of(p, b));
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
    Place* ends = reinterpret_cast<Place*>(s_scan + 17);
    if (threadIdx.x == 0) {
      s_scan[16] = total;
      ends[1] = {p.c.B, 0, 0};
    }
    __syncthreads();
    for (int e = 0; e < 2; ++e) {
      const int64_t place = part_begin(total, blockIdx.x + e, gridDim.x);
      if (place < total && begin <= place && place < begin + mine) {
        int64_t at = begin;
        int b = b0;
        Seq s;
        for (;; ++b) {
          s = seq_of(p, b);
          const int64_t n = length_of(p, s);
          if (place < at + n) break;
          at += n;
        }
        ends[e] = place_of(p, s, b, place - at, total / gridDim.x);
      }
    }
  }
  __syncthreads();
  const uint32_t tmem = *s_tmem;
  const bool any = *s_abort == 0 && s_scan[16] > 0;
  // The next item of a role: false behind the last one, and where something has failed.
  auto segment = [&](int seg, int& nt) {
    if (!fp8b::mbar_wait_all(&g_full[seg % kSegs], (seg / kSegs) & 1, s_abort)) return false;
    nt = s_seg[seg % kSegs].nt;
    return nt != 0;
  };
  auto done_with = [&](int seg) {  // a warp, converged
    if (lane == 0) mbar_arrive(&g_empty[seg % kSegs]);
  };

  if (warp == kCopyWarp) {
    // ---- copies: a lane per page of the tile, keys, then values
    fp8b::regs_give<72>();
    const int per = kTok / p.c.page, page_bytes = p.c.page * D;
    Ring rk, rv;
    int keys = 0, values = 0, nt;
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
        const bool has = lane < per && page >= 0;
        const uint32_t bytes = __popc(__ballot_sync(0xFFFFFFFFu, has)) * page_bytes;
        const int64_t block = block_at(p.c, has ? page : 0, 0, h);
        if (keys >= C::kKeySlots && !mbar_wait_warp(&k_empty[rk.i], rk.phase ^ 1, s_abort)) ok = false;
        if (!ok) break;
        if (lane == 0) mbar_arrive_expect_tx(&k_full[rk.i], bytes);
        __syncwarp();
        if (has) tma_load_3d(smem + C::kOffKeys + rk.i * C::kTileBytes + lane * page_bytes, &tm, 0, 0, static_cast<int>(block), &k_full[rk.i]);
        __syncwarp();
        ++keys;
        if (values >= C::kValueSlots && !mbar_wait_warp(&v_empty[rv.i], rv.phase ^ 1, s_abort)) ok = false;
        if (!ok) break;
        if (lane == 0) mbar_arrive_expect_tx(&v_full[rv.i], bytes);
        __syncwarp();
        if (has) bulk_load(smem + C::kOffCodes + rv.i * C::kTileBytes + lane * page_bytes, p.c.codes + (block + p.c.H) * page_bytes, page_bytes, &v_full[rv.i]);
        __syncwarp();
        ++values;
        rk.step(C::kKeySlots);
        rv.step(C::kValueSlots);
      }
    }
    if (!ok && any && lane == 0) fp8b::raise_error8(p.status, s_abort, kErrCopyR);
    // never leave with copies still in flight (only those that were asked for are waited for)
    for (int i = max(0, keys - C::kKeySlots); i < keys; ++i) {
      uint32_t spin = 0;
      while (!mbar_try_wait(&k_full[i % C::kKeySlots], (i / C::kKeySlots) & 1) && ++spin < kSpinLimit) {
      }
    }
    for (int i = max(0, values - C::kValueSlots); i < values; ++i) {
      uint32_t spin = 0;
      while (!mbar_try_wait(&v_full[i % C::kValueSlots], (i / C::kValueSlots) & 1) && ++spin < kSpinLimit) {
      }
    }
  } else if (warp == kMmaWarp || warp == kMmaWarp + 1) {
    // ---- products of row tile q
    fp8b::regs_give<72>();
    const int q = warp - kMmaWarp;
    const bool issuer = elect_one();
    const uint64_t kdesc = desc_rows<D>(smem_u32(smem + C::kOffKeys)), qdesc = desc_rows<D>(smem_u32(smem + C::kOffQueries + q * C::kTerms * C::kTileBytes));
    const uint64_t vdesc = desc_values(smem_u32(smem + C::kOffValues));
    const uint32_t sdesc_i = umma_idesc_e4m3(kStep), odesc_i = idesc_f16(D, false, true);
    const uint32_t to_s = tmem + q * kTok, to_o = tmem + 256 + q * 128;
    Ring k, v;
    int done = 0, scored = 0, items = 0;  // steps of products with values, and of scores, begun
    bool failed = false;
    int nt;
    for (int seg = 0; any && !failed && segment(seg, nt); ++seg) {
      const bool active = q == 0 || s_seg[seg % kSegs].rows > kTok;
      const int steps = s_seg[seg % kSegs].steps;
      __syncwarp();
      done_with(seg);
      if (!mbar_wait(q_full, items++ & 1, s_abort)) {
        failed = true;
        break;
      }
      if (!active) {  // no rows: the other tile's operands pass by
        if (lane == 0) mbar_arrive(q_empty);
        for (int j = 0; j < nt; ++j) {
          if (!mbar_wait_warp(&k_full[k.i], k.phase, s_abort)) failed = true;
          if (!failed && lane == 0) mbar_arrive(&k_empty[k.i]);
          if (!failed && !mbar_wait_warp(&w_full[v.i], v.phase, s_abort)) failed = true;
          if (failed) break;
          if (lane == 0) mbar_arrive(&w_empty[v.i]);
          __syncwarp();
          k.step(C::kKeySlots);
          v.step(2);
        }
        continue;
      }
      // Scores of the item's next step.  They go to the place of the probabilities two steps before, once these are used.
      int at = 0;
      auto scores = [&] {
        if (at >= steps) return true;
        const int buf = scored & 1, half = at & 1;
        const bool ends = half != 0 || at + 1 == steps;  // of the tile of keys
        if (half == 0 && !mbar_wait(&k_full[k.i], k.phase, s_abort)) return false;
        if (scored >= 2 && !mbar_wait(&pv_done[q * 2 + buf], ((scored >> 1) - 1) & 1, s_abort)) return false;
        tc_fence_after_sync();
        if (issuer) {
          const uint64_t bd = kdesc + static_cast<uint64_t>((k.i * C::kTileBytes + half * kStep * D) >> 4);
#pragma unroll
          for (int term = 0; term < C::kTerms; ++term)
#pragma unroll
            for (int s = 0; s < D / 32; ++s)
              umma_f8(to_s + buf * kStep, qdesc + static_cast<uint64_t>((term * C::kTileBytes) >> 4) + s * 2, bd + s * 2,
                      term > 0 ? sdesc_i | kFirstE5m2 : sdesc_i, (term > 0 || s > 0) ? 1u : 0u);
          umma_commit(&s_full[q * 2 + buf]);
          if (ends) umma_commit(&k_empty[k.i]);
          if (at + 1 == steps) umma_commit(q_empty);
        }
        __syncwarp();
        if (ends) k.step(C::kKeySlots);
        ++scored;
        ++at;
        return true;
      };
      failed = !scores() || !scores();
      for (int st = 0; st < steps && !failed; ++st) {
        const int buf = done & 1;
        const bool ends = (st & 1) != 0 || st + 1 == steps;
        if (((st & 1) == 0 && !mbar_wait(&w_full[v.i], v.phase, s_abort)) || !mbar_wait(&p_full[q * 2 + buf], (done >> 1) & 1, s_abort)) {
          failed = true;
          break;
        }
        tc_fence_after_sync();
        if (issuer) {
          const uint64_t bd = vdesc + static_cast<uint64_t>((v.i * C::kValueBytes + (st & 1) * kStep * 128) >> 4);
#pragma unroll
          for (int s = 0; s < kStep / 16; ++s)
            umma_f16_tmem_a(to_o, to_s + buf * kStep + s * 8, bd + s * (2048 >> 4), odesc_i, ((EXACT ? st % C::kSumSteps : st) != 0 || s > 0) ? 1u : 0u);
          if (EXACT)
#pragma unroll
            for (int s = 0; s < kStep / 16; ++s)
              umma_f16_tmem_a(to_o, to_s + buf * kStep + kStep / 2 + s * 8, bd + s * (2048 >> 4), odesc_i, 1u);
          umma_commit(&pv_done[q * 2 + buf]);
          if (ends) umma_commit(&w_empty[v.i]);
        }
        __syncwarp();
        ++done;
        if (ends) v.step(2);
        failed = !scores();
      }
    }
    if (failed && issuer) fp8b::raise_error8(p.status, s_abort, kErrMmaR);
    // tensor memory is released only when every MMA has completed, also where another role has given up
    if (issuer) umma_commit(&drain[q]);
    uint32_t spin = 0;
    while (!mbar_try_wait(&drain[q], 0) && ++spin < kSpinLimit) {
    }
    __syncwarp();
  } else if (warp == kWalkWarp) {
    // ---- the items of this CTA, and the block scales of their tiles: a lane per 16 tokens, four tiles at a time
    fp8b::regs_give<72>();
    float4* table = reinterpret_cast<float4*>(smem + C::kOffScales);
    const Place begin = reinterpret_cast<const Place*>(s_scan + 17)[0], end = reinterpret_cast<const Place*>(s_scan + 17)[1];
    int seg = 0, tiles = 0;
    bool ok = any;
    auto announce = [&](const Seg& g) {
      if (seg >= kSegs && !mbar_wait_warp(&g_empty[seg % kSegs], (seg / kSegs - 1) & 1, s_abort)) return false;
      if (lane == 0) {
        s_seg[seg % kSegs] = g;
        mbar_arrive(&g_full[seg % kSegs]);
      }
      __syncwarp();
      ++seg;
      return true;
    };
    const bool same = begin.b == end.b && begin.k == end.k;
    if (lane == 0) {
      const bool goes_on = any && end.tile > 0 && (!same || begin.tile == 0);
      const int came = any && begin.tile > 0 && !(same && end.tile == begin.tile) ? (same ? 1 : 2) : 0;
      p.shared[blockIdx.x] = make_int4(goes_on ? end.b : 0, goes_on ? end.k : 0, goes_on ? 1 : 0, came);
    }
    if (any) {
      int b = begin.b, k = begin.k, tile = begin.tile;
      Seq s = seq_of(p, b);
      for (; ok; ++k, tile = 0) {
        while (b < end.b && k >= s.blocks * p.c.H) {
          k = 0;
          if (++b < p.c.B) s = seq_of(p, b);
        }
        const bool ends = b == end.b && k == end.k;  // the part ends in this item
        if (b == p.c.B || (b == end.b && k > end.k) || (ends && tile >= end.tile)) break;
        Seg g{};
        g.L = s.L, g.n = s.n, g.b = b, g.h = k % p.c.H, g.first = s.first;
        const int64_t row0 = block_row0(s, k / p.c.H);
        g.row0 = static_cast<int>(row0);
        g.rows = block_rows(p, s, row0);
        const Item item = item_of(p, s, row0, g.rows);
        const int c1 = ends ? end.tile : item.nt;
        g.tile0 = item.t0 + tile;
        g.nt = c1 - tile;
        g.steps = 2 * g.nt - (ends ? 0 : item.half);
        g.part = tile > 0 ? 2 * blockIdx.x : ends ? 2 * blockIdx.x + 1 : -1;
        if (!announce(g)) {
          ok = false;
          break;
        }
        for (int j0 = 0; j0 < g.nt && ok; j0 += 4) {
          const int64_t token = (static_cast<int64_t>(g.tile0) + j0) * kTok + lane * 16;
          const float4 e = scale_entry(load_scales(p.c, b, g.h, token, s.L));
          for (int j = 0; j < 4 && j0 + j < g.nt; ++j, ++tiles) {
            const int slot = tiles % kScaleSlots;
            if (tiles >= kScaleSlots && !mbar_wait_warp(&e_empty[slot], (tiles / kScaleSlots - 1) & 1, s_abort)) {
              ok = false;
              break;
            }
            if (lane >> 3 == j) table[slot * 8 + (lane & 7)] = e;
            __syncwarp();
            if (lane == 0) mbar_arrive(&e_full[slot]);
          }
        }
      }
      if (ok) ok = announce(Seg{});
      if (!ok && lane == 0) fp8b::raise_error8(p.status, s_abort, kErrWalkR);
    }
  } else if (warp >= kConvWarp0) {
    fp8b::regs_give<72>();
    constexpr int kLanes = D / 8, kRowsPer = 32 / kLanes, kRowsStep = 4 * kRowsPer, kBatch = 4;
    const int i = threadIdx.x - kConvWarp0 * 32;
    Ring v, o;
    int n = 0, nt, items = 0;
    bool ok = any;
    for (int seg = 0; ok && segment(seg, nt); ++seg) {
      const Seg& g = s_seg[seg % kSegs];
      const int64_t left0 = g.L - static_cast<int64_t>(g.tile0) * kTok;  // tokens from the first tile on
      const int first = g.first, h = g.h, row0 = g.row0, rows = g.rows;
      __syncwarp();
      done_with(seg);
      // Queries, once those there are done with (two steps before the item's end): all rows are copied to where they are going to
      // be, half of a row in the place of each of its first two terms, then converted there.  (Loads to registers, of which there were
      // 16 per warp on their way, cost 28000 cycles between two items, and copies of rows 10000 just to ask for, where two boxes
      // per tile cannot have them.)
      if (items > 0 && !fp8b::mbar_wait_all(q_empty, (items - 1) & 1, s_abort)) {
        if (lane == 0) fp8b::raise_error8(p.status, s_abort, kErrConvertR);
        break;
      }
      if (p.boxes) {
        if (i == 0) {
          mbar_arrive_expect_tx(r_full, (rows > kTok ? kRows : kTok) * 2 * D);
          for (int r = 0; r < rows; r += kTok)
            for (int half = 0; half < 2; ++half)
              tma_load_4d(smem + C::kOffQueries + (r / kTok * C::kTerms + half) * C::kTileBytes, &tm_q, 0, half, h * p.G, first + (row0 + r) / p.G, r_full);
        }
      } else {
        if (i == 0) mbar_arrive_expect_tx(r_full, rows * 2 * D);
        for (int r = i; r < rows; r += kTok) {
          const __nv_bfloat16* src = p.q + (first + (row0 + r) / p.G) * p.ldq + (static_cast<int64_t>(h) * p.G + (row0 + r) % p.G) * D;
          uint8_t* to = smem + C::kOffQueries + (r / kTok) * C::kTerms * C::kTileBytes + i * D;
          bulk_load(to, src, D, r_full);
          bulk_load(to + C::kTileBytes, src + D / 2, D, r_full);
        }
      }
      __syncwarp();
      if (!fp8b::mbar_wait_all(r_full, items & 1, s_abort)) {
        uint32_t spin = 0;  // never leave with copies still in flight
        while (!mbar_try_wait(r_full, items & 1) && ++spin < kSpinLimit) {
        }
        if (lane == 0) fp8b::raise_error8(p.status, s_abort, kErrConvertR);
        break;
      }
      ++items;
      // D / 8 lanes per row, kBatch independent rows at a time: a warp per scheduler is bound by its instructions' latencies here
#pragma unroll 1
      for (int r0 = (warp - kConvWarp0) * kRowsPer + lane / kLanes; r0 < (rows > kTok ? kRows : kTok); r0 += kBatch * kRowsStep) {
        const int l = lane % kLanes;
        uint8_t* row = smem + C::kOffQueries + (r0 / kTok * C::kTerms * kTok + r0 % kTok) * D;
        const uint8_t* from = row + l / (kLanes / 2) * C::kTileBytes + l % (kLanes / 2) * 16;
        uint8_t* to = row - r0 % kTok * D + row_piece<D>(r0 % kTok, l / 2) + (l & 1) * 8;
        uint4 x[kBatch];
        uint32_t a[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) x[u] = r0 + u * kRowsStep < rows ? *reinterpret_cast<const uint4*>(from + u * (kRowsStep * D)) : make_uint4(0u, 0u, 0u, 0u);
        __syncwarp();
#pragma unroll
        for (int u = 0; u < kBatch; ++u) a[u] = absmax_bits8(x[u]);
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1)
#pragma unroll
          for (int u = 0; u < kBatch; ++u) a[u] = max(a[u], __shfl_xor_sync(0xFFFFFFFFu, a[u], o));
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const RowScale s = row_scale(a[u]);
          uint2 term[C::kTerms];
          split8<false, C::kTerms>(x[u], s.up, term);
#pragma unroll
          for (int k = 0; k < C::kTerms; ++k)  // (a step of 8 rows or 16, which the swizzle does not see)
            *reinterpret_cast<uint2*>(to + k * C::kTileBytes + u * (kRowsStep * D)) = term[k];
          if (l == 0) s_rows[r0 + u * kRowsStep] = s.down * p.scale_log2;
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(q_full);
      for (int j = 0; j < nt; ++j, ++n) {
        if (!fp8b::mbar_wait_all(&v_full[v.i], v.phase, s_abort) || (n >= 2 && !fp8b::mbar_wait_all(&w_empty[o.i], o.phase ^ 1, s_abort))) {
          if (lane == 0) fp8b::raise_error8(p.status, s_abort, kErrConvertR);
          ok = false;
          break;
        }
        widen_values<D, 128>(smem + C::kOffCodes + v.i * C::kTileBytes, smem + C::kOffValues + o.i * C::kValueBytes, i,
                             static_cast<int>(min(left0 - static_cast<int64_t>(j) * kTok, static_cast<int64_t>(kTok))));
        fence_proxy_async_smem();  // the tensor core reads what these stores wrote
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&w_full[o.i]);
          mbar_arrive(&v_empty[v.i]);
        }
        v.step(C::kValueSlots);
        o.step(2);
      }
    }
  } else {
    // ---- softmax and epilogue: thread = row
    fp8b::regs_take<184>();
    const int q = warp >> 2, i = threadIdx.x & 127;
    const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + lane_base + q * kTok, to = tmem + lane_base + 256 + q * 128;
    const float4* table = reinterpret_cast<const float4*>(smem + C::kOffScales);
    bool failed = !any;
    int nt, tiles = 0, done = 0, items = 0;  // tiles: of the block scales; done: of this row tile
    for (int seg = 0; !failed && segment(seg, nt); ++seg) {
      const Seg& g = s_seg[seg % kSegs];
      const int r = q * kTok + i, rows = g.rows, row = g.row0 + r, L = g.L, tile0 = g.tile0, h = g.h, part = g.part, steps = g.steps;
      const int64_t t = g.first + row / p.G;  // row of the tensors
      const int64_t pos = static_cast<int64_t>(L) - g.n + row / p.G;
      __syncwarp();
      done_with(seg);
      const bool mine = r < rows;
      // tokens that the row sees (a row there is none of: all, which spares the others of its warp the masked form)
      const int hi = mine && p.causal ? static_cast<int>(max(min(pos + 1, static_cast<int64_t>(L)), static_cast<int64_t>(0))) : L;
      const int lo = mine && p.window > 0 ? static_cast<int>(max(pos + 1 - p.window, static_cast<int64_t>(0))) : 0;
      const int hi_all = __reduce_min_sync(0xFFFFFFFFu, hi), lo_all = __reduce_max_sync(0xFFFFFFFFu, lo);
      float m = -INFINITY, l = 0.0f, m_sum = -INFINITY;  // m_sum: the reference of the sum in the workspace
      if (!fp8b::mbar_wait_all(q_full, items & 1, s_abort)) {
        failed = true;
        break;
      }
      ++items;
      const float c = q * kTok < rows ? s_rows[r] : 0.0f;
      __syncwarp();
      if (lane == 0) mbar_arrive(q_empty);
      auto step = [&](int st, bool first) {
        const int slot = tiles % kScaleSlots;
        if ((st & 1) == 0 && !fp8b::mbar_wait_all(&e_full[slot], (tiles / kScaleSlots) & 1, s_abort)) return false;
        if (q * kTok < rows) {
          const int buf = done & 1;
          if (!fp8b::mbar_wait_all(&s_full[q * 2 + buf], (done >> 1) & 1, s_abort)) return false;
          tc_fence_after_sync();
          float x[kStep];
#pragma unroll
          for (int k = 0; k < kStep / 32; ++k) fp8b::tmem_ld32(ts + buf * kStep + k * 32, x + k * 32);
#pragma unroll
          for (int k = 0; k < kStep / 32; ++k) fp8b::tmem_ld_wait32(x + k * 32);
          const int base = tile0 * kTok + st * kStep;
          auto accumulated = [&] { return fp8b::mbar_wait_all(&pv_done[q * 2 + (buf ^ 1)], ((done - 1) >> 1) & 1, s_abort); };
          const float4* e = table + slot * 8 + (st & 1) * (kStep / 16);
          const uint32_t probs = ts + buf * kStep;
          const bool ok = base >= lo_all && base + (kStep - 1) < hi_all
                              ? softmax_step<D, EXACT, false>(x, e, c, 0, kStep, m, l, probs, to, first, accumulated)
                              : softmax_step<D, EXACT, true>(x, e, c, lo - base, hi - base, m, l, probs, to, first, accumulated);
          if (!ok) return false;
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive(&p_full[q * 2 + buf]);
          ++done;
        }
        if ((st & 1) != 0 || st + 1 == steps) {
          __syncwarp();
          if (lane == 0) mbar_arrive(&e_empty[slot]);
          ++tiles;
        }
        return true;
      };
      if (EXACT) {
        for (int begin = 0; begin < steps && !failed; begin += C::kSumSteps) {
          if (begin > 0 && q * kTok < rows) {
            if (!fp8b::mbar_wait_all(&pv_done[q * 2 + ((done - 1) & 1)], ((done - 1) >> 1) & 1, s_abort)) {
              failed = true;
              break;
            }
            tc_fence_after_sync();
            add_to_sum<D>(to, p.sums + static_cast<int64_t>(blockIdx.x) * (kRows * D), r, begin > C::kSumSteps, carried(m_sum, m));
            m_sum = m;
          }
          for (int st = begin; st < min(steps, begin + C::kSumSteps) && !failed; ++st) failed = !step(st, st == begin);
        }
      } else {
        for (int st = 0; st < steps && !failed; ++st) failed = !step(st, st == 0);
      }
      if (failed) break;
      if (q * kTok >= rows) continue;
      // the products of the last two steps
      if ((steps > 1 && !fp8b::mbar_wait_all(&pv_done[q * 2 + (done & 1)], ((done - 2) >> 1) & 1, s_abort)) ||
          !fp8b::mbar_wait_all(&pv_done[q * 2 + ((done - 1) & 1)], ((done - 1) >> 1) & 1, s_abort)) {
        failed = true;
        break;
      }
      tc_fence_after_sync();
      float* to_part = part < 0 ? nullptr : p.partial + static_cast<int64_t>(part) * (kRows * (D + 2));
      const int hq = h * p.G + row % p.G;
      if (part >= 0) {
        to_part[kRows * D + r] = l;
        to_part[kRows * D + kRows + r] = m;
      } else if (mine && p.lse) {
        p.lse[t * (static_cast<int64_t>(p.G) * p.c.H) + hq] = l == 0.0f ? -INFINITY : (log2f(l) + m + 8.0f - kShift) * (1.0f / kLog2e);
      }
      const float f = part >= 0 ? 1.0f : (l == 0.0f ? 0.0f : 1.0f / l);
#pragma unroll 1
      for (int d = 0; d < D; d += 32) {
        float o[32];
        fp8b::tmem_ld32(to + d, o);
        fp8b::tmem_ld_wait32(o);
        if (EXACT && steps > C::kSumSteps) add_sum32(o, p.sums + static_cast<int64_t>(blockIdx.x) * (kRows * D), r, d, carried(m_sum, m));
#pragma unroll
        for (int k = 0; k < 32; k += 4) {  // features 1 and 2 of every four change places again (see widen4)
          const float x = o[k + 1] * f;
          o[k] *= f;
          o[k + 1] = o[k + 2] * f;
          o[k + 2] = x;
          o[k + 3] *= f;
        }
        if (part >= 0) {
#pragma unroll
          for (int k = 0; k < 8; ++k) *reinterpret_cast<float4*>(to_part + r * D + d + 4 * k) = make_float4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
        } else if (mine) {
          store16(p, t * p.ldo + static_cast<int64_t>(hq) * D + d, o);
          store16(p, t * p.ldo + static_cast<int64_t>(hq) * D + d + 16, o + 16);
        }
      }
      tc_fence_before_sync();
    }
    if (failed && any && lane == 0) fp8b::raise_error8(p.status, s_abort, kErrSoftmaxR);
  }

  tc_fence_before_sync();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, 512);
  }
}

// Results of items that several CTAs share: a block per CTA where one begins and 8 rows, a warp per row, D / 32 features per lane.
template <int D>
__global__ void __launch_bounds__(256) attention_join_rows_kernel(const P p, int ctas) {
  constexpr int E = D / 32;
  __shared__ int s_came[kMaxCtas];
  __shared__ float s_w[8][kMaxCtas + 1];
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, x = blockIdx.x;
  pdl_wait();
  const uint4 shared = load_chained(reinterpret_cast<const uint4*>(p.shared + x));
  if (shared.z == 0) return;
  for (int i = threadIdx.x; i < ctas; i += 256) s_came[i] = static_cast<int>(load_chained(reinterpret_cast<const uint4*>(p.shared + i)).w);
  const Seq s = seq_of(p, static_cast<int>(shared.x));
  const int k = static_cast<int>(shared.y), h = k % p.c.H;
  const int64_t row0 = block_row0(s, k / p.c.H);
  const int r = blockIdx.y * 8 + warp;
  __syncthreads();
  if (row0 + r >= static_cast<int64_t>(s.n) * p.G) return;
  // the CTAs behind x that it reaches (one between them may have nothing of it)
  int end = x + 1;
  while (end < ctas && s_came[end] != 2) ++end;
  end = min(end + 1, ctas);
  constexpr int64_t kPart = kRows * (D + 2);
  auto piece = [&](int i) { return p.partial + (2 * i + (i == x ? 1 : 0)) * kPart; };
  auto has = [&](int i) { return i == x || s_came[i] != 0; };
  float m = -INFINITY;
  for (int i = x + lane; i < end; i += 32)
    if (has(i)) m = fmaxf(m, load_chained(piece(i) + kRows * D + kRows + r));
  m = warp_max(m);
  float l = 0.0f;
  for (int i = x + lane; i < end; i += 32) {
    float f = 0.0f;
    if (has(i)) {
      const float mi = load_chained(piece(i) + kRows * D + kRows + r), li = load_chained(piece(i) + kRows * D + r);
      // (a piece that saw nothing counts for nothing; a sum that is NaN has no maximum)
      if (li != 0.0f) f = mi == -INFINITY ? 1.0f : exp2f(mi - m);
      if (li != 0.0f) l = fmaf(f, li, l);
    }
    s_w[warp][i - x] = f;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, o);
  __syncwarp();
  float o[E] = {};
#pragma unroll 4
  for (int i = x; i < end; ++i) {
    const float f = s_w[warp][i - x];
    if (f == 0.0f) continue;  // (what lies there is nothing)
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = fmaf(f, load_chained(piece(i) + r * D + e * 32 + lane), o[e]);
  }
  const int64_t t = s.first + (row0 + r) / p.G;
  const int hq = h * p.G + static_cast<int>((row0 + r) % p.G);
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float v = l == 0.0f ? 0.0f : o[e] / l;
    const int64_t at = t * p.ldo + static_cast<int64_t>(hq) * D + e * 32 + lane;
    if (p.f32)
      static_cast<float*>(p.out)[at] = v;
    else
      static_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(v);
  }
  if (p.lse && lane == 0) p.lse[t * (static_cast<int64_t>(p.G) * p.c.H) + hq] = l == 0.0f ? -INFINITY : (log2f(l) + m + 8.0f - kShift) * (1.0f / kLog2e);
}

template <int D, bool EXACT>
int launch_cfg(const CUtensorMap& tm, const CUtensorMap& tm_q, const P& p, int grid, cudaStream_t st) {
  using C = Cfg<D, EXACT>;
  static DeviceOnce once;
  if (!allow_shared_memory(once, attention_rows_kernel<D, EXACT>, C::kSmemBytes)) return ZQ_ERR_CUDA;
  cudaError_t e = launch_chained(attention_rows_kernel<D, EXACT>, dim3(grid), dim3(kThreads), C::kSmemBytes, st, false, tm, tm_q, p);
  count_launch();
  if (e != cudaSuccess) return ZQ_ERR_CUDA;
  e = launch_chained(attention_join_rows_kernel<D>, dim3(grid, kRows / 8), dim3(256), 0, st, false, p, grid);
  count_launch();
  return e == cudaSuccess ? ZQ_OK : ZQ_ERR_CUDA;
}

// Queries [T][Hq][2 halves][D / 2], boxes of one half of a tile's rows: 128 / G tokens' G heads.
bool make_query_map(CUtensorMap* m, const AttnArgs& a, int G) {
  gemm::EncodeTiledFn fn = gemm::encode_fn();
  if (!fn) return false;
  const cuuint64_t half = static_cast<cuuint64_t>(a.c.D);  // bytes
  const cuuint64_t dims[4] = {half / 2, 2, static_cast<cuuint64_t>(a.Hq), static_cast<cuuint64_t>(a.c.T)};
  const cuuint64_t strides[3] = {half, 2 * half, static_cast<cuuint64_t>(a.ldq) * 2};
  const cuuint32_t box[4] = {static_cast<cuuint32_t>(half / 2), 1, static_cast<cuuint32_t>(G), static_cast<cuuint32_t>(kTok / G)};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(a.q), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

// (the same place as the other kernel's: the kernels of a call run one after the other)
size_t rows_workspace_bytes(int64_t D) { return sizeof(float) * kMaxCtas * kRows * (2 * (D + 2) + D) + sizeof(int4) * kMaxCtas; }

int launch_attention_rows(const AttnArgs& a, cudaStream_t st) {
  P p{};
  p.c = a.c;
  p.q = static_cast<const __nv_bfloat16*>(a.q), p.ldq = a.ldq, p.G = a.Hq / a.c.H;
  p.scale_log2 = a.sm_scale * kLog2e;
  p.causal = a.causal, p.window = a.window;
  p.out = a.out, p.f32 = a.dt == ZQ_OUT_F32, p.ldo = a.ldo, p.lse = a.lse;
  uint8_t* ws = static_cast<uint8_t*>(a.workspace);
  p.status = reinterpret_cast<int*>(ws);
  p.shared = reinterpret_cast<int4*>(ws + kWsHeadBytes);
  p.partial = reinterpret_cast<float*>(p.shared + kMaxCtas);
  p.sums = p.partial + static_cast<int64_t>(kMaxCtas) * 2 * kRows * (a.c.D + 2);
  CUtensorMap tm, tm_q{};
  // a tile's queries as two boxes where whole tokens fill it and a token's stride is one of whole heads
  p.boxes = kTok % p.G == 0 && a.ldq % a.c.D == 0 ? 1 : 0;
  if (!make_page_map(&tm, a.c) || (p.boxes && !make_query_map(&tm_q, a, p.G))) return ZQ_ERR_CUDA;
  const int sms = sm_count(), grid = sms < kMaxCtas ? sms : kMaxCtas;
  if (p.f32) return a.c.D == 128 ? launch_cfg<128, true>(tm, tm_q, p, grid, st) : launch_cfg<64, true>(tm, tm_q, p, grid, st);
  return a.c.D == 128 ? launch_cfg<128, false>(tm, tm_q, p, grid, st) : launch_cfg<64, false>(tm, tm_q, p, grid, st);
}

}  // namespace kv
}  // namespace zq
