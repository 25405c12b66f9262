// Pieces shared by the two attention kernels (few rows per sequence and head, many rows): tensor-core operands, the walk over a
// sequence's tiles of 128 tokens, the splitting of queries, block scales.
#pragma once

#include "kv_cache.cuh"

namespace zq {
namespace kv {

constexpr int kTok = 128;           // tokens of a tile
constexpr int kFewRows = 64;        // rows (new tokens x query heads of a cache head) up to which the kernel for few rows takes a sequence
constexpr int kMaxCtas = 148;       // CTAs whose partial results the workspace has room for
constexpr float kLog2e = 1.4426950408889634f;
// Probabilities are kept times 2^kShift (the row's largest at most 2^kShift), where FP16 holds 11 bits down to 2^-22 of the
// largest and something down to 2^-32.  Values are code / 256.  Both factors cancel against the sum of the probabilities.
constexpr float kShift = 8.0f;
constexpr float kCodeUnit = 1.0f / 256.0f;

int launch_attention_few(const AttnArgs& a, int max_rows, cudaStream_t st);
int launch_attention_rows(const AttnArgs& a, cudaStream_t st);
size_t rows_workspace_bytes(int64_t D);
size_t few_workspace_bytes(int64_t D);

#ifdef __CUDACC__
// ---- operands ---------------------------------------------------------------------------------------------------------
// 8-bit rows of D bytes, K-major, swizzled as the copy engine does for rows of that size (128 or 64 bytes).
template <int D>
__device__ __forceinline__ uint64_t desc_rows(uint32_t smem_addr) {
  uint64_t d = 0;
  d |= uint64_t((smem_addr >> 4) & 0x3FFF);
  d |= uint64_t(1) << 16;
  d |= uint64_t((8 * D) >> 4) << 32;  // the next 8 rows
  d |= uint64_t(1) << 46;
  d |= uint64_t(D == 128 ? 2 : 4) << 61;
  return d;
}
// Byte of 16-byte piece `piece` of row `row` in such rows.
template <int D>
__device__ __forceinline__ uint32_t row_piece(int row, int piece) {
  return row * D + ((piece ^ (D == 128 ? row & 7 : (row >> 1) & 3)) << 4);
}
// 8-bit operand with the tokens in K: a token's ROW bytes (features, or columns) side by side, 32, 64 or 128 bytes swizzled as rows of
// that size are, 8 tokens per atom; more than 128 bytes in parts of 128, each of all 128 tokens.  (Where M wants more features than
// there are, 128 of 64, it gets them twice.)
template <int ROW>
__device__ __forceinline__ uint64_t desc_tokens(uint32_t smem_addr) {
  constexpr int kRow = ROW < 128 ? ROW : 128;
  uint64_t d = 0;
  d |= uint64_t((smem_addr >> 4) & 0x3FFF);
  d |= uint64_t(ROW > 128 ? (kTok * 128) >> 4 : 0) << 16;  // the next 128 bytes
  d |= uint64_t((8 * kRow) >> 4) << 32;                    // the next 8 tokens
  d |= uint64_t(1) << 46;
  d |= uint64_t(kRow == 128 ? 2 : kRow == 64 ? 4 : 6) << 61;
  return d;
}
// Byte of 16-byte piece `piece` of a token in such an operand.
template <int ROW>
__device__ __forceinline__ uint32_t token_piece(int token, int piece) {
  constexpr int kRow = ROW < 128 ? ROW : 128, kPieces = kRow / 16;
  const int sw = kRow == 128 ? token & 7 : kRow == 64 ? (token >> 1) & 3 : (token >> 2) & 1;
  return (piece / kPieces) * (kTok * 128) + token * kRow + (((piece % kPieces) ^ sw) << 4);
}
// The first operand is E5M2 instead of E4M3 (or'ed to an instruction descriptor).
constexpr uint32_t kFirstE5m2 = 1u << 7;
// E4M3 x E4M3 -> FP32 with the tokens in K on both sides, D is 128 x n
__device__ __forceinline__ uint32_t idesc_e4m3_mn(uint32_t n) {
  return (1u << 4) | (1u << 15) | (1u << 16) | ((n >> 3) << 17) | ((128u >> 4) << 24);
}
// Two FP16 numbers up to 256 -> two E4M3 numbers, three times: w = t0 + t1 / 16 + t2 / 256, each the rest of the one before.
__device__ __forceinline__ void split3(uint32_t w, uint32_t* t) {
  asm("{\n\t.reg .b16 a, b, c;\n\t.reg .b32 x, r;\n\t"
      "cvt.rn.satfinite.e4m3x2.f16x2 a, %3;\n\t"
      "cvt.rn.f16x2.e4m3x2 x, a;\n\t"
      "sub.f16x2 r, %3, x;\n\t"
      "mul.f16x2 r, r, %4;\n\t"  // exact: a rest has 8 bits at the most
      "cvt.rn.satfinite.e4m3x2.f16x2 b, r;\n\t"
      "cvt.rn.f16x2.e4m3x2 x, b;\n\t"
      "sub.f16x2 r, r, x;\n\t"
      "mul.f16x2 r, r, %4;\n\t"
      "cvt.rn.satfinite.e4m3x2.f16x2 c, r;\n\t"
      "cvt.u32.u16 %0, a;\n\tcvt.u32.u16 %1, b;\n\tcvt.u32.u16 %2, c;\n\t}"
      : "=r"(t[0]), "=r"(t[1]), "=r"(t[2])
      : "r"(w), "r"(0x4C004C00u));
}
// FP16 values [128 tokens][64 features] (128 bytes a token, 128-byte swizzle), the features of M or N, the tokens of K; the next 64
// features 16 KB further.
__device__ __forceinline__ uint64_t desc_values(uint32_t smem_addr) {
  uint64_t d = 0;
  d |= uint64_t((smem_addr >> 4) & 0x3FFF);
  d |= uint64_t((kTok * 128) >> 4) << 16;
  d |= uint64_t(1024 >> 4) << 32;
  d |= uint64_t(1) << 46;
  d |= uint64_t(2) << 61;
  return d;
}
// FP16 x FP16 -> FP32, D is 128 x n
__device__ __forceinline__ uint32_t idesc_f16(uint32_t n, bool a_mn, bool b_mn) {
  return (1u << 4) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) | ((n >> 3) << 17) | ((128u >> 4) << 24);
}
__device__ __forceinline__ void umma_f16(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// A converter thread's share of a tile of values: codes [128][D] (rows as they lie in memory) -> FP16 code / 256 in the operand's
// layout: E4M3's exponent and mantissa bits moved into FP16's fields, which have one exponent bit more, whence the factor
// (subnormal numbers come out right as well).  The hardware's conversion would do it at a quarter of the rate (a tile 1300 cycles
// instead of about 500).  Codes are taken two and two as they lie in a word, so features 1 and 2 of every four change places
// until the results are stored.  The pattern of E4M3's NaN becomes 480 / 256: what nobody sees (a page that was not copied, say) must not turn
// into NaN by a product with zero.  Tokens from `valid` on become zeros, whatever the page holds there.  All of the share's codes
// are loaded before the first store (the compiler cannot tell their addresses apart), kAtOnce pieces of 16 at a time.
__device__ __forceinline__ uint2 widen4(uint32_t w) {
  return make_uint2(((w << 8) & 0x80008000u) | ((w << 7) & 0x3F803F80u), (w & 0x80008000u) | ((w >> 1) & 0x3F803F80u));
}
__device__ __forceinline__ uint4 widen8(uint32_t a, uint32_t b) {
  const uint2 x = widen4(a), y = widen4(b);
  return make_uint4(x.x, x.y, y.x, y.y);
}
template <int D, int THREADS>
__device__ __forceinline__ void widen_values(const uint8_t* codes, uint8_t* out, int i, int valid) {
  constexpr int kPieces = kTok * D / 16 / THREADS, kPerRow = D / 16, kAtOnce = kPieces < 4 ? kPieces : 4;
  static_assert(kTok * D / 16 % THREADS == 0 && THREADS % kPerRow == 0 && kPieces % kAtOnce == 0, "pieces per thread");
  // pieces of a thread are THREADS / kPerRow rows apart, a multiple of 8: their swizzle is the same
  static_assert(THREADS / kPerRow % 8 == 0, "rows");
  const int row0 = i / kPerRow, c = i % kPerRow, sw = row0 & 7, p = (c & 3) * 2;
  uint8_t* to = out + (c >> 2) * (kTok * 128) + row0 * 128;
  const int to0 = (p ^ sw) << 4, to1 = ((p + 1) ^ sw) << 4;
#pragma unroll
  for (int x0 = 0; x0 < kPieces; x0 += kAtOnce) {
    uint4 v[kAtOnce];
#pragma unroll
    for (int x = 0; x < kAtOnce; ++x) {
      v[x] = *reinterpret_cast<const uint4*>(codes + ((x0 + x) * THREADS + i) * 16);
      if (row0 + (x0 + x) * (THREADS / kPerRow) >= valid) v[x] = make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int x = 0; x < kAtOnce; ++x) {
      uint8_t* dst = to + (x0 + x) * (THREADS / kPerRow) * 128;
      *reinterpret_cast<uint4*>(dst + to0) = widen8(v[x].x, v[x].y);
      *reinterpret_cast<uint4*>(dst + to1) = widen8(v[x].z, v[x].w);
    }
  }
}

// ---- queries ------------------------------------------------------------------------------------------------------------
// Eight bf16 features of a row as two 8-bit numbers each: q 2^e = a + b with the row's largest feature between 128 and 256.  A bf16
// number has 8 bits, a (E4M3) 4; the rest is at most half of a's step, so 3 bits hold it, where b's smallest step does.  That
// is why b is no E4M3 number as it is (their smallest step is 2^-9: features below 2^-2 lost bits, those below 2^-10 all of them):
//   few rows    b = E4M3 / 2^5, its products in columns of their own: exact from 2^-7 on (2^-14 of the row's largest and less),
//               off by 2^-15 at most below (2^-22 of the largest)
//   many rows   b = E5M2, its products added to a's by the tensor core: exact from 2^-6 on (2^-13), off by 2^-14 at most below (2^-21)
//   and for FP32 results what b leaves as E5M2 once more: exact from 2^-9 on (2^-16), off by 2^-17 at most below (2^-24)
struct RowScale {
  float up;    // 2^e, 0 where the row is not finite
  float down;  // 2^-e, NaN there
};
__device__ __forceinline__ RowScale row_scale(uint32_t amax_bits) {  // bits of the largest |q| as FP32
  const int e = max(static_cast<int>(amax_bits >> 23), 8);           // (rows below 2^-119: their scores are nothing)
  RowScale r;
  const bool finite = amax_bits < 0x7F800000u;
  r.up = finite ? __uint_as_float(static_cast<uint32_t>(261 - e) << 23) : 0.0f;
  r.down = finite ? __uint_as_float(static_cast<uint32_t>(e - 7) << 23) : __uint_as_float(0x7FC00000u);
  return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t absmax_bits8(uint4 v) {
  const uint32_t m = max_u16x2(max_u16x2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), max_u16x2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu));
  return max(m << 16, m & 0xFFFF0000u);
}
// Eight numbers times `up` as TERMS 8-bit numbers each: an E4M3 number, then an E4M3 number times 2^-kRestBits (FEW) or E5M2 ones.  In
// between they are FP16, which holds them: 8 bits, the largest below 2^8, the steps 2^-24.  A row that is not finite has up = 0,
// NaN for what is not finite in it, and a factor that makes all of its scores NaN.
constexpr int kRestBits = 5;
template <bool FEW, int TERMS>
__device__ __forceinline__ void split8(uint4 v, float up, uint2* term) {
  static_assert(TERMS == 2 || (TERMS == 3 && !FEW), "terms");
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t t[TERMS][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t x = pack_f16(bf16_lo(w[i]) * up, bf16_hi(w[i]) * up), y;
    uint16_t c;
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(c) : "r"(x));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(y) : "h"(c));
    asm("sub.f16x2 %0, %1, %2;" : "=r"(x) : "r"(x), "r"(y));
    t[0][i] = c;
    if (FEW) {
      asm("mul.f16x2 %0, %1, %2;" : "=r"(x) : "r"(x), "r"(((15u + kRestBits) << 10) * 0x10001u));  // 2^kRestBits; at most 2^8
      asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(c) : "r"(x));
    } else {
      asm("cvt.rn.satfinite.e5m2x2.f16x2 %0, %1;" : "=h"(c) : "r"(x));
    }
    t[1][i] = c;
    if (TERMS == 3) {
      asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(y) : "h"(c));
      asm("sub.f16x2 %0, %1, %2;" : "=r"(x) : "r"(x), "r"(y));
      asm("cvt.rn.satfinite.e5m2x2.f16x2 %0, %1;" : "=h"(c) : "r"(x));
      t[TERMS - 1][i] = c;
    }
  }
#pragma unroll
  for (int k = 0; k < TERMS; ++k) term[k] = make_uint2(t[k][0] | (t[k][1] << 16), t[k][2] | (t[k][3] << 16));
}

// ---- block scales -------------------------------------------------------------------------------------------------------
// What 16 tokens of a tile (part of one page) contribute: keys' scale, log2 of the values' scale, its inverse times kCodeUnit.
// The values' scale goes into the power of two of the probability, so that nothing of it is rounded apart, and comes out of the
// sum again by its inverse times kCodeUnit.
struct RawScales {
  float ks, vs;
  bool seen;
};
__device__ __forceinline__ RawScales load_scales(const Cache& c, int b, int h, int64_t token, int L) {
  RawScales r{0.0f, 1.0f, token < L};
  if (!r.seen) return r;
  const int page = page_of(c, b, static_cast<int>(token) / c.page);
  r.ks = page < 0 ? __uint_as_float(0x7FC00000u) : load_chained(c.scale + block_at(c, page, 0, h));
  r.vs = page < 0 ? 1.0f : load_chained(c.scale + block_at(c, page, 1, h));
  return r;
}
__device__ __forceinline__ float4 scale_entry(const RawScales& r) {
  if (!r.seen) return make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  const float vs = r.vs < 5.42101086242752217e-20f ? 5.42101086242752217e-20f : r.vs;  // 2^-64: what was never written has 0
  // (a block that stands for NaN: the power is NaN where it is seen)
  return make_float4(r.ks, log2f(vs), isnan(vs) ? 1.0f : kCodeUnit / vs, 0.0f);
}

// Pages of consecutive tiles, a batch of 32 table entries per warp with the next batch on its way.
struct PageWalk {
  int b, L, base, cur, next;
  __device__ __forceinline__ int load(const Cache& c, int i) const {
    return static_cast<int64_t>(i) * c.page < L ? page_of(c, b, i) : -1;
  }
  __device__ __forceinline__ void start(const Cache& c, int seq, int len, int first_page, int lane) {
    b = seq, L = len, base = first_page;
    cur = load(c, base + lane);
    next = load(c, base + 32 + lane);
  }
  // The page of table entry `first + lane` for lane < count; first ascends by at most 32 from call to call.
  __device__ __forceinline__ int get(const Cache& c, int first, int lane) {
    if (first - base >= 32) {
      cur = next;
      base += 32;
      next = load(c, base + 32 + lane);
    }
    return __shfl_sync(0xFFFFFFFFu, cur, (first - base + lane) & 31);
  }
};

// Largest of a warp's numbers (NaN only where all are).
__device__ __forceinline__ float warp_max(float v) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}

// A 3-D tensor of bytes [blocks][page][D], boxes of one block's page x D bytes.
inline bool make_page_map(CUtensorMap* m, const Cache& c) {
  gemm::EncodeTiledFn fn = gemm::encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(c.D), static_cast<cuuint64_t>(c.page), static_cast<cuuint64_t>(c.pages) * 2 * c.H};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(c.D), static_cast<cuuint64_t>(c.D) * c.page};
  const cuuint32_t box[3] = {static_cast<cuuint32_t>(c.D), static_cast<cuuint32_t>(c.page), 1};
  const cuuint32_t estr[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, c.codes, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            c.D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
#endif

}  // namespace kv
}  // namespace zq
