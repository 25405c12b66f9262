// Pieces shared by the operators around the 8-bit cache of keys and values: E4M3 codes in pages of 16 to 128 tokens, one FP32
// scale for each block (page, keys or values, head).  See include/zqfp.h for the operators' definitions.
#pragma once

#include "fp8_block.cuh"
#include "kv_index.h"

namespace zq {
namespace kv {

// A cache and the sequences of a call.
struct Cache {
  uint8_t* codes;    // [pages][2][H][page][D]
  float* scale;      // [pages][2][H]
  int64_t pages;
  int H, page, D;
  const int* table;  // [B][table_ld]: page of each sequence's tokens 0 .. page - 1, page .. 2 page - 1, ...
  int64_t table_ld;
  const int* lens;   // [B] tokens of each sequence, the new ones included
  const int* cu;     // [B + 1] first row of each sequence's new tokens, or NULL: one each
  int B;
  int64_t T;         // rows of the tensors that hold the new tokens
};

struct WriteArgs {
  Cache c;
  const void *k, *v;  // bf16 [T][ld]: heads side by side
  int64_t ldk, ldv;
  int mode;
};
struct ReadArgs {
  Cache c;            // cu: rows of the outputs; T: their number
  void *k, *v;        // [T][H][D]
  int dt;
};
struct AttnArgs {
  Cache c;
  const void* q;      // bf16 [T][ldq]: heads side by side
  int64_t ldq;
  int Hq;
  float sm_scale;
  int causal, window;
  void* out;          // [T][ldo]
  int dt;
  int64_t ldo;
  float* lse;         // [T][Hq] or NULL
  void* workspace;
};
struct NormRopeArgs {
  const void *q, *k;             // bf16 [T][ld]
  int64_t ldq, ldk;
  const void *dq, *dk;           // backward: gradients of the outputs
  int64_t lddq, lddk;
  int64_t T;
  int Hq, H, D;
  const float *wq, *wk;          // [D] or both NULL
  float eps;
  const float* table;            // [far][rot]: cosines, then sines
  int64_t far;
  int rot, neighbours;
  const int* positions;          // [T]
  void *oq, *ok;                 // bf16 [T][ld]: outputs, or gradients of the inputs
  int64_t ldoq, ldok;
  float *dwq, *dwk;              // backward: [D]
  float* partial;                // backward: [blocks][2][D]
};
constexpr int kNormGradBlocks = 592;  // at most: partial sums of the weights' gradients that the workspace has room for

int launch_write(const WriteArgs& a, cudaStream_t st);
int launch_read(const ReadArgs& a, cudaStream_t st);
int launch_norm_rope(const NormRopeArgs& a, cudaStream_t st);
int launch_norm_rope_backward(const NormRopeArgs& a, cudaStream_t st);
int launch_attention(const AttnArgs& a, cudaStream_t st);

#ifdef __CUDACC__
using fp8b::load_chained;
__device__ __forceinline__ int load_chained(const int* p) {
  int v;
  asm volatile("ld.global.cg.s32 %0, [%1];" : "=r"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ float4 load_chained(const float4* p) {
  float4 v;
  asm volatile("ld.global.cg.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 load_chained(const uint2* p) {
  uint2 v;
  asm volatile("ld.global.cg.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}

// Rows of sequence b: [first, first + n).  Nothing (n = 0) where the offsets do not describe rows of the tensors.
__device__ __forceinline__ void rows_of(const Cache& c, int b, int& first, int& n) {
  if (!c.cu) {
    first = b;
    n = 1;
    return;
  }
  first = load_chained(c.cu + b);
  const int end = load_chained(c.cu + b + 1);
  n = first >= 0 && end > first && end <= c.T ? end - first : 0;
}
// The page of a sequence's tokens i * page .., or -1 where the table has none or names none of the cache's.
__device__ __forceinline__ int page_of(const Cache& c, int b, int i) {
  if (i < 0 || i >= c.table_ld) return -1;
  const int p = load_chained(c.table + b * c.table_ld + i);
  return p >= 0 && p < c.pages ? p : -1;
}
// Position of a block among the cache's blocks.
__device__ __forceinline__ int64_t block_at(const Cache& c, int page, int which, int h) {
  return (static_cast<int64_t>(page) * 2 + which) * c.H + h;
}

// The scale a block needs whose largest absolute value has these bits (see fp8b::block_scale on bits and not finite values).
// It is at least 2^-64, also where all is zero: it has an inverse, and a block that is begun with zeros takes its scale from the
// first values that follow.  (The largest bf16 numbers need 2^119; how far apart the attention lets scales be says include/zqfp.h.)
__device__ __forceinline__ float cache_scale(uint32_t amax_bits, bool pow2) {
  if (amax_bits >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
  float s = fmaxf(__fdiv_rn(__uint_as_float(amax_bits), 448.0f), 5.42101086242752217e-20f);
  if (pow2) s = __uint_as_float((__float_as_uint(s) + 0x7FFFFFu) & 0x7F800000u);
  return s;
}
#endif

}  // namespace kv
}  // namespace zq
