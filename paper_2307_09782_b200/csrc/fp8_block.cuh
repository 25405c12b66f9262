// Pieces shared by the FP8 operators with block scales: E4M3 codes whose scale belongs to a block of 128, one
// row by 128 input features for activations, 128 x 128 for weights (FP32 scales, or rounded up to a power of two).
// See include/zqfp.h for the operators' definitions.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "act_cast.cuh"
#include "w4a8_gemm_shared.cuh"

namespace zq {
namespace fp8b {

constexpr int kBlk = 128;
inline int64_t blocks_of(int64_t n) { return (n + kBlk - 1) / kBlk; }

enum Kind {
  kPlain = 0,     // y = a b^T
  kGated = 1,     // b is (gate, up): h = act(a g^T) (a u^T), in bf16 and / or quantized; g and u kept in 8 bits on request
  kGatedBwd = 2,  // y = a b^T is the gradient of h: the gradients of g and u, from the 8-bit g and u
};

struct GemmArgs8 {
  const uint8_t* a;  // [parts][M][K] E4M3 (kGated: [M][K])
  const float* sa;   // [parts][ceil(K / 128)][M]
  const uint8_t* b;  // [parts][N][K] E4M3 (kGated: [2][N][K])
  const float* sb;   // [parts][ceil(N / 128)][ceil(K / 128)]
  int64_t M, N, K;
  int parts;         // segments of the K sum (kPlain)
  int kind, act, mode;
  int pow2_scales;   // sa and sb are powers of two: the tensor core can apply them itself
  void* y;           // kPlain: [M][ldy] FP32 or bf16; kGated: h bf16 [M][ldy] or NULL; kGatedBwd: bf16 [2][M][N]
  int ydt;
  int64_t ldy;
  uint8_t* q;        // kGated: codes of h [M][N] or NULL; kGatedBwd: codes of the gradients [2][M][N]
  float* s;          // their scales, [ceil(N / 128)][M] each
  uint8_t* ck;       // [2][M][N] codes of g and u (kGated: written when not NULL; kGatedBwd: read)
  float* cks;        // [2][ceil(N / 128)][M]
  int* status;
  // launch_block_few only: raw activations, which the kernel quantizes itself (a and sa unused)
  const void* x;     // bf16 [M][ldx]
  int64_t ldx;
};

int launch_quantize_block(const void* x, int64_t M, int64_t K, int64_t ldx, int mode, uint8_t* q, float* s,
                          cudaStream_t st);
int launch_quantize_weight_block(const float* w, int64_t N, int64_t K, int mode, uint8_t* q, float* s, cudaStream_t st);
int launch_transpose_weight_block(const uint8_t* q, const float* s, int64_t N, int64_t K, uint8_t* qt, float* st_,
                                  cudaStream_t st);
int launch_block_gemm(const GemmArgs8& a, cudaStream_t st);  // many tokens
bool few_takes(const GemmArgs8& a);      // which of the two
bool few_takes_raw(const GemmArgs8& a);  // whether launch_block_few quantizes raw activations itself
int launch_block_few(const GemmArgs8& a, cudaStream_t st);   // few tokens
struct WgradArgs {
  const void* g;     // bf16 [parts] x [M][ldg], g_stride elements apart
  int64_t ldg, g_stride;
  const uint8_t* q;  // [M][K]
  const float* s;    // [ceil(K / 128)][M]
  int parts;
  int64_t M, N, K;
  void* dw;          // [parts][N][K]
  int dwdt;
  int* status;
};
int launch_wgrad(const WgradArgs& a, cudaStream_t st);

#ifdef __CUDACC__
// A 3-D tensor of bytes [parts][rows][K] (dense), boxes of 128 bytes x `box_rows` rows, 128-byte swizzle: one
// K-major operand tile of the tensor core.  Beyond the tensor the copy engine fills in zeros.
inline bool make_code_map(CUtensorMap* m, const void* base, uint64_t K, uint64_t rows, uint64_t parts, uint32_t box_rows) {
  gemm::EncodeTiledFn fn = gemm::encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {K, rows, parts};
  const cuuint64_t strides[2] = {K, K * rows};
  const cuuint32_t box[3] = {kBlk, box_rows, 1};
  const cuuint32_t estr[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Launch with programmatic serialization, in clusters of `cluster` CTAs along x.
template <typename... KArgs, typename... Args>
inline cudaError_t launch_clustered(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, int cluster,
                                    Args&&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = static_cast<unsigned>(cluster);
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

// The scale of a block from the bits of its absolute maximum (as unsigned numbers they order like the values, and
// NaN and infinity are above all finite ones, so a maximum over bits keeps them):
//   0 -> 1 ; not finite -> NaN (the whole block then stands for NaN) ; else max(fl32(a / 448), 2^-126), which keeps
//   1 / s finite, rounded up to a power of two on request (the carry of the mantissa moves the exponent).
__device__ __forceinline__ float block_scale(uint32_t amax_bits, bool pow2) {
  if (amax_bits == 0u) return 1.0f;
  if (amax_bits >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
  float s = fmaxf(__fdiv_rn(__uint_as_float(amax_bits), 448.0f), 1.17549435e-38f);
  if (pow2) s = __uint_as_float((__float_as_uint(s) + 0x7FFFFFu) & 0x7F800000u);
  return s;
}
__device__ __forceinline__ float block_inv(float s) { return __frcp_rn(s); }
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// Four FP32 values -> four E4M3 bytes of v * inv.
__device__ __forceinline__ uint32_t cast4(float a, float b, float c, float d, float inv) {
  return cvt_e4m3x2(__fmul_rn(a, inv), __fmul_rn(b, inv)) | (cvt_e4m3x2(__fmul_rn(c, inv), __fmul_rn(d, inv)) << 16);
}
// Two E4M3 bytes -> FP32 (exact: every E4M3 value is an FP16 value).
__device__ __forceinline__ float2 decode2(uint16_t w) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(w));
  __half2 h2;
  *reinterpret_cast<uint32_t*>(&h2) = h;
  return __half22float2(h2);
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// Loads of data that the kernel ahead in the stream may have written.  With programmatic launches that kernel can still run
// when this one begins.  So the read-only path, which is for data that nobody writes while the kernel lasts, is not for them
// (the compiler may move such a load above the wait for that kernel as well), nor are lines that the first-level cache may hold
// from before the wait: they go to L2, and stay in order with the wait.
__device__ __forceinline__ float load_chained(const float* p) {
  float v;
  asm volatile("ld.global.cg.f32 %0, [%1];" : "=f"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ uint32_t load_chained(const uint32_t* p) {
  uint32_t v;
  asm volatile("ld.global.cg.u32 %0, [%1];" : "=r"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ uint4 load_chained(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.cg.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
// A tile of a 3-D tensor map on its way to L2.  It reads nothing: whatever is written to the tile afterwards is what a copy
// after that write gets.
__device__ __forceinline__ void tma_prefetch_3d(const CUtensorMap* m, int c0, int c1, int c2) {
  asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global [%0, {%1, %2, %3}];"
               ::"l"(reinterpret_cast<uint64_t>(m)), "r"(c0), "r"(c1), "r"(c2)
               : "memory");
}
__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

// The activations.  SiLU and the tanh form of GELU are both v * sigmoid(w(v)), with w = v and
// w = 2 sqrt(2 / pi) (v + 0.044715 v^3), since (1 + tanh z) / 2 = sigmoid(2 z).  1 / (1 + 2^(-w / ln 2)) with the special
// function unit's power of two and reciprocal is good to about 5e-7 relative near zero; the power's argument is rounded in
// FP32, which adds 6e-8 |w| where w is negative (5e-6 at -80, where SiLU is 1e-33).  A bf16 result rounds by 4e-3, an E4M3
// one by 6e-2.  A power that overflows gives 0, one that underflows 1, a NaN stays one.
__device__ __forceinline__ float sfu_ex2(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float sfu_rcp(float v) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
constexpr float kSiluC = -1.4426950408889634f;                        // -1 / ln 2
constexpr float kGeluC = -1.4426950408889634f * 1.5957691216057308f;  // times 2 sqrt(2 / pi)
template <int ACT>
__device__ __forceinline__ float act_sigmoid(float v) {
  const float t = ACT == ZQ_ACT_SILU ? kSiluC * v : v * fmaf(kGeluC * 0.044715f, v * v, kGeluC);
  return sfu_rcp(1.0f + sfu_ex2(t));
}
template <int ACT>
__device__ __forceinline__ float act_value(float v) {
  if (ACT == ZQ_ACT_RELU) return v < 0.0f ? 0.0f : v;  // keeps NaN
  return v * act_sigmoid<ACT>(v);
}
__device__ __forceinline__ uint64_t twice(float v) { return pack2(v, v); }
// Two values at a time: packed arithmetic (one instruction for both), the special function unit for each.
template <int ACT>
__device__ __forceinline__ uint64_t act_sigmoid2(uint64_t v, uint64_t v2) {  // v2: v^2 (GELU)
  const uint64_t t = ACT == ZQ_ACT_SILU ? mul2(v, twice(kSiluC)) : mul2(v, fma2(v2, twice(kGeluC * 0.044715f), twice(kGeluC)));
  float t0, t1;
  unpack2(t, t0, t1);
  unpack2(fma2(pack2(sfu_ex2(t0), sfu_ex2(t1)), twice(1.0f), twice(1.0f)), t0, t1);
  return pack2(sfu_rcp(t0), sfu_rcp(t1));
}
// value and derivative: v p and p + v p (1 - p) w'
template <int ACT>
__device__ __forceinline__ void act_both2(uint64_t v, uint64_t& value, uint64_t& slope) {
  if (ACT == ZQ_ACT_RELU) {
    float a, b;
    unpack2(v, a, b);
    value = pack2(act_value<ACT>(a), act_value<ACT>(b));
    slope = pack2(a > 0.0f ? 1.0f : 0.0f, b > 0.0f ? 1.0f : 0.0f);
    return;
  }
  uint64_t v2 = 0ull;
  if (ACT == ZQ_ACT_GELU_TANH) {  // from |v| = 100 on p is 0 or 1 and (1 - p) or v p zero: v^2 must not overflow beside them
    float a, b;
    unpack2(mul2(v, v), a, b);
    v2 = pack2(fminf(a, 1e4f), fminf(b, 1e4f));
  }
  const uint64_t p = act_sigmoid2<ACT>(v, v2);
  value = mul2(v, p);
  const uint64_t q = fma2(p, twice(-1.0f), twice(1.0f));
  if (ACT == ZQ_ACT_SILU)
    slope = fma2(value, q, p);
  else
    slope = fma2(mul2(value, q), fma2(v2, twice(1.5957691216057308f * 0.134145f), twice(1.5957691216057308f)), p);
}
// Larger of two pairs of 16-bit unsigned numbers.
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// Registers per thread from here on, for a whole warpgroup (each warp of it executes one of these).
template <int N>
__device__ __forceinline__ void regs_give() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void regs_take() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }

// 32 consecutive FP32 columns of this thread's tensor-memory lane, and the wait tied to their registers.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float* v) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void tmem_ld_wait32(float* v) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])
               :
               : "memory");
}
// A bounded wait that every lane of the warp makes itself (no shuffle after it); the warp leaves it converged.
__device__ __forceinline__ bool mbar_wait_all(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  const bool ok = mbar_wait(bar, parity, abort_flag);
  return __all_sync(0xFFFFFFFFu, ok);
}

// Arrive on the leader's barrier of a CTA pair for what has been done to tensor memory (the loads or stores are waited for and
// fenced): nothing in other memory is published, and a release at cluster scope would wait for the warp's other accesses,
// about 1000 cycles.
__device__ __forceinline__ void mbar_arrive_tmem(uint64_t* bar) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(map_to_rank(smem_u32(bar), 0)) : "memory");
}
// Four 32-bit columns of this thread's tensor-memory lane.
__device__ __forceinline__ void tmem_st4(uint32_t taddr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "r"(a), "r"(b), "r"(c), "r"(d));
}
__device__ __forceinline__ float ld_cluster(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}
// The cluster's last meeting, which only keeps shared memory alive for peers that read it: nothing is published.
__device__ __forceinline__ void cluster_leave() {
  asm volatile("barrier.cluster.arrive.relaxed;\n\tbarrier.cluster.wait;" ::: "memory");
}

__device__ __forceinline__ void raise_error8(int* status, volatile int* abort_flag, int detail) {
  *abort_flag = 1;
  if (atomicCAS(status, 0, ZQ_ERR_DEVICE_TIMEOUT) == 0) status[1] = detail;
}
#endif  // __CUDACC__

}  // namespace fp8b
}  // namespace zq
