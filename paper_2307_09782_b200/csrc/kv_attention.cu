// Attention over the 8-bit cache: which kernel takes what.
#include "kv_attention.cuh"

namespace zq {
namespace kv {

// Each sequence goes to the kernel for its rows (new tokens x query heads of a cache head), as the kernels themselves find from
// the offsets on the device; a kernel that no sequence can need is not launched.
int launch_attention(const AttnArgs& a, cudaStream_t st) {
  const int64_t G = a.Hq / a.c.H, most = a.c.cu ? a.c.T * G : G;  // rows of a sequence and head, at most
  // FP32 results: the other kernel's probabilities have 12 bits (7e-5 of the result), this one's two terms 22 (1e-6 with all else);
  // chunks of 777 tokens behind others take 349 us so, 255 with one term and two of the queries.
  if (a.dt == ZQ_OUT_F32) return launch_attention_rows(a, st);
  if (G <= kFewRows)
    if (int e = launch_attention_few(a, static_cast<int>(most < kFewRows ? most : kFewRows), st)) return e;
  return most > kFewRows ? launch_attention_rows(a, st) : ZQ_OK;
}

}  // namespace kv
}  // namespace zq
