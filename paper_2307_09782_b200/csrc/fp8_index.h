// Index arithmetic of the FP8 kernels that has to hold up to the largest sizes the entry points accept (row counts close
// to 2^31).  Plain C++, so that it is tested without a GPU.
#pragma once

#ifdef __CUDACC__
#define ZQ_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define ZQ_HOST_DEVICE inline
#endif

namespace zq {
namespace fp8b {

// Token of row `row` (0 .. 63) of stage `i` of a CTA whose stages are step0 .. step0 + steps - 1, or -1 where there is none.
// The stage is compared first: past the last one the token's number does not fit 32 bits any more.
ZQ_HOST_DEVICE int stage_token(int step0, int i, int steps, int row, int M) {
  if (i >= steps) return -1;
  const int m = (step0 + i) * 64 + row;
  return m < M ? m : -1;
}

// Bytes of the part of a row that starts `left` elements of `size` bytes before the row's end (none are left where it is
// negative) and has `most` elements at the most.  Elements are compared, not bytes: 2^29 of four bytes do not fit 32 bits.
ZQ_HOST_DEVICE int row_bytes(int left, int most, int size) { return (left < most ? left : most) * size; }

}  // namespace fp8b
}  // namespace zq
