// Attention over the 8-bit cache: which kernel takes what.
#include "kv_attention.cuh"

namespace zq {
namespace kv {

// Each sequence goes to the kernel for its rows (new tokens x query heads of a cache head), as the kernels themselves find from
// the offsets on the device; a kernel that no sequence can need is not launched.
int launch_attention(const AttnArgs& a, cudaStream_t st) {
  // Rows of a sequence and head, at most: with offsets all rows could be one sequence's, and the instance for few rows works on as many
  // as it is made for.  (64 sequences of up to 8192 tokens, one new token and 4 rows each: 124 us without offsets, by the instance
  // for 4 rows, and 488 with them, by the one for 64.)
  const int64_t G = a.Hq / a.c.H, most = a.c.cu ? a.c.T * G : G;
  // FP32 results: the other kernel's probabilities have 12 bits (7e-5 of the result), this one's two terms 22 (1e-6 with all else);
  // chunks of 777 tokens behind others take 343 us so, 255 with one term, two of the queries and one accumulator.
  if (a.dt == ZQ_OUT_F32) return launch_attention_rows(a, st);
  if (G <= kFewRows)
    if (int e = launch_attention_few(a, static_cast<int>(most < kFewRows ? most : kFewRows), st)) return e;
  return most > kFewRows ? launch_attention_rows(a, st) : ZQ_OK;
}

}  // namespace kv
}  // namespace zq
