// C-ABI entry points of the FP8 operators with block scales: argument validation, workspace carving, dispatch.
// The operators are defined in include/zqfp.h.
#include "fp8_block.cuh"

using namespace zq;
using namespace zq::fp8b;

namespace {

inline bool al16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }
bool scale_rule_ok(int mode) { return mode == ZQ_SCALE_NONE || mode == ZQ_SCALE_M1; }
bool act_ok(int act) { return act == ZQ_ACT_SILU || act == ZQ_ACT_GELU_TANH || act == ZQ_ACT_RELU; }
constexpr int64_t kMaxRows = 0x7FFFFF00;
bool rows_ok(int64_t n) { return n >= 0 && n <= kMaxRows; }
bool k_ok(int64_t k) { return k >= 16 && k % 16 == 0 && k <= (int64_t(1) << 30); }

// codes and scales of raw activations, behind the head that every workspace of the library starts with
struct Ws8 {
  size_t off_q, off_s, total;
};
Ws8 ws8(int64_t M, int64_t K) {
  Ws8 w{};
  w.off_q = up256(kWsHeadBytes);
  w.off_s = w.off_q + up256(static_cast<size_t>(M) * K);
  w.total = w.off_s + up256(static_cast<size_t>(blocks_of(K)) * M * 4);
  return w;
}

// Activations given as codes or raw.  Raw ones are quantized into the workspace first, or, with few tokens, by the
// kernel that multiplies them.
int quantize_raw(const uint8_t*& q, const float*& s, const void* x, int64_t ldx, int64_t M, int64_t K, int mode,
                 void* workspace, size_t workspace_bytes, cudaStream_t st) {
  if (!x) return ZQ_OK;
  const Ws8 w = ws8(M, K);
  uint8_t* base = static_cast<uint8_t*>(workspace);
  uint8_t* q_ws = base + w.off_q;
  float* s_ws = reinterpret_cast<float*>(base + w.off_s);
  if (workspace_bytes < w.total) return ZQ_ERR_WORKSPACE;
  q = q_ws;
  s = s_ws;
  return launch_quantize_block(x, M, K, ldx, mode, q_ws, s_ws, st);
}

int launch(GemmArgs8& a, const uint8_t* q, const float* s, const void* x, int64_t ldx, void* workspace,
           size_t workspace_bytes, void* stream) {
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  a.status = static_cast<int*>(workspace);
  if (x && few_takes_raw(a)) {
    a.x = x;
    a.ldx = ldx;
    return launch_block_few(a, st);
  }
  if (int e = quantize_raw(q, s, x, ldx, a.M, a.K, a.mode, workspace, workspace_bytes, st)) return e;
  a.a = q;
  a.sa = s;
  return few_takes(a) ? launch_block_few(a, st) : launch_block_gemm(a, st);
}

int check_activations(const uint8_t* q, const float* s, const void* x, int64_t ldx, int64_t M, int64_t K, void* workspace,
                      size_t workspace_bytes) {
  if (x ? (q || s) : (!q || !s)) return ZQ_ERR_NULL;
  if (x && ldx < K) return ZQ_ERR_SHAPE;
  if (x ? (!al16(x) || ldx % 8) : !al16(q)) return ZQ_ERR_ALIGN;
  if (!workspace) return ZQ_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return ZQ_ERR_ALIGN;
  if (workspace_bytes < (x ? ws8(M, K).total : kWsHeadBytes)) return ZQ_ERR_WORKSPACE;
  return ZQ_OK;
}

}  // namespace

extern "C" {

int zq_quantize_fp8_block(const void* x, int64_t M, int64_t K, int64_t ldx, zq_scale_mode mode, uint8_t* q, float* s,
                          void* stream) {
  if (!scale_rule_ok(mode)) return ZQ_ERR_MODE;
  if (!rows_ok(M) || !k_ok(K) || ldx < K) return ZQ_ERR_SHAPE;
  if (M == 0) return ZQ_OK;
  if (!x || !q || !s) return ZQ_ERR_NULL;
  if (!al16(x) || !al16(q) || ldx % 8) return ZQ_ERR_ALIGN;
  if (int e = check_device_sm100()) return e;
  return launch_quantize_block(x, M, K, ldx, mode, q, s, static_cast<cudaStream_t>(stream));
}

int zq_quantize_weight_fp8_block(const float* W, int64_t N, int64_t K, zq_scale_mode mode, uint8_t* q, float* s,
                                 void* stream) {
  if (!scale_rule_ok(mode)) return ZQ_ERR_MODE;
  if (!rows_ok(N) || !k_ok(K)) return ZQ_ERR_SHAPE;
  if (N == 0) return ZQ_OK;
  if (!W || !q || !s) return ZQ_ERR_NULL;
  if (!al16(W) || !al16(q)) return ZQ_ERR_ALIGN;
  if (int e = check_device_sm100()) return e;
  return launch_quantize_weight_block(W, N, K, mode, q, s, static_cast<cudaStream_t>(stream));
}

int zq_transpose_weight_fp8_block(const uint8_t* q, const float* s, int64_t N, int64_t K, uint8_t* qt, float* st,
                                  void* stream) {
  if (!rows_ok(N) || !k_ok(K) || N % 16) return ZQ_ERR_SHAPE;
  if (N == 0) return ZQ_OK;
  if (!q || !s || !qt || !st) return ZQ_ERR_NULL;
  if (!al16(q) || !al16(qt)) return ZQ_ERR_ALIGN;
  if (int e = check_device_sm100()) return e;
  return launch_transpose_weight_block(q, s, N, K, qt, st, static_cast<cudaStream_t>(stream));
}

size_t zq_fp8_block_workspace_bytes(int64_t M, int64_t K) {
  if (!rows_ok(M) || !k_ok(K)) return 0;
  return ws8(M, K).total;
}

int zq_fp8_block_linear(const uint8_t* q, const float* s, const void* x_bf16, int64_t ldx, zq_scale_mode mode, int parts,
                        int64_t M, int64_t N, int64_t K, const uint8_t* w, const float* ws, void* y, zq_out_dtype ydt,
                        int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
  if (!scale_rule_ok(mode) || (ydt != ZQ_OUT_F32 && ydt != ZQ_OUT_BF16)) return ZQ_ERR_MODE;
  if (!rows_ok(M) || !rows_ok(N) || !k_ok(K) || ldy < N || parts < 1 || parts > 2 || (x_bf16 && parts != 1))
    return ZQ_ERR_SHAPE;
  if (M == 0 || N == 0) return ZQ_OK;
  if (!w || !ws || !y) return ZQ_ERR_NULL;
  if (!al16(w) || (reinterpret_cast<uintptr_t>(y) & (ydt == ZQ_OUT_F32 ? 3u : 1u))) return ZQ_ERR_ALIGN;
  if (int e = check_activations(q, s, x_bf16, ldx, M, K, workspace, workspace_bytes)) return e;
  if (int e = check_device_sm100()) return e;
  GemmArgs8 a{};
  a.b = w;
  a.sb = ws;
  a.M = M;
  a.N = N;
  a.K = K;
  a.parts = parts;
  a.kind = kPlain;
  a.mode = mode;
  a.y = y;
  a.ydt = ydt;
  a.ldy = ldy;
  return launch(a, q, s, x_bf16, ldx, workspace, workspace_bytes, stream);
}

int zq_fp8_gated_linear(const uint8_t* q, const float* s, const void* x_bf16, int64_t ldx, zq_scale_mode mode, int64_t M,
                        int64_t F, int64_t K, const uint8_t* w, const float* ws, zq_activation act, void* h_bf16,
                        int64_t ldh, uint8_t* hq, float* hs, uint8_t* gu, float* gus, void* workspace,
                        size_t workspace_bytes, void* stream) {
  if (!scale_rule_ok(mode) || !act_ok(act)) return ZQ_ERR_MODE;
  if (!rows_ok(M) || !rows_ok(F) || F % 16 || !k_ok(K) || (h_bf16 && ldh < F)) return ZQ_ERR_SHAPE;
  if (M == 0 || F == 0) return ZQ_OK;
  if (!w || !ws || (!h_bf16 && !hq) || (hq && !hs) || (gu && !gus)) return ZQ_ERR_NULL;
  if (!al16(w) || !al16(hq) || !al16(gu) || (reinterpret_cast<uintptr_t>(h_bf16) & 1u)) return ZQ_ERR_ALIGN;
  if (int e = check_activations(q, s, x_bf16, ldx, M, K, workspace, workspace_bytes)) return e;
  if (int e = check_device_sm100()) return e;
  GemmArgs8 a{};
  a.b = w;
  a.sb = ws;
  a.M = M;
  a.N = F;
  a.K = K;
  a.parts = 1;
  a.kind = kGated;
  a.act = act;
  a.mode = mode;
  a.y = h_bf16;
  a.ydt = ZQ_OUT_BF16;
  a.ldy = ldh;
  a.q = hq;
  a.s = hs;
  a.ck = gu;
  a.cks = gus;
  return launch(a, q, s, x_bf16, ldx, workspace, workspace_bytes, stream);
}

int zq_fp8_gated_linear_backward(const uint8_t* q, const float* s, const void* dy_bf16, int64_t lddy, zq_scale_mode mode,
                                 int64_t M, int64_t F, int64_t K, const uint8_t* wt, const float* wts, zq_activation act,
                                 const uint8_t* gu, const float* gus, void* dgu_bf16, uint8_t* dguq, float* dgus,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  if (!scale_rule_ok(mode) || !act_ok(act)) return ZQ_ERR_MODE;
  if (!rows_ok(M) || !rows_ok(F) || F % 16 || !k_ok(K)) return ZQ_ERR_SHAPE;
  if (M == 0 || F == 0) return ZQ_OK;
  if (!wt || !wts || !gu || !gus || !dgu_bf16 || !dguq || !dgus) return ZQ_ERR_NULL;
  if (!al16(wt) || !al16(gu) || !al16(dgu_bf16) || !al16(dguq)) return ZQ_ERR_ALIGN;
  if (int e = check_activations(q, s, dy_bf16, lddy, M, K, workspace, workspace_bytes)) return e;
  if (int e = check_device_sm100()) return e;
  GemmArgs8 a{};
  a.b = wt;
  a.sb = wts;
  a.M = M;
  a.N = F;
  a.K = K;
  a.parts = 1;
  a.kind = kGatedBwd;
  a.act = act;
  a.mode = mode;
  a.y = dgu_bf16;
  a.ydt = ZQ_OUT_BF16;
  a.ldy = F;
  a.q = dguq;
  a.s = dgus;
  a.ck = const_cast<uint8_t*>(gu);
  a.cks = const_cast<float*>(gus);
  return launch(a, q, s, dy_bf16, lddy, workspace, workspace_bytes, stream);
}

int zq_fp8_weight_grad(const void* g_bf16, int64_t ldg, int64_t g_stride, int parts, const uint8_t* q, const float* s,
                       int64_t M, int64_t N, int64_t K, void* dw, zq_out_dtype dwdt, void* workspace,
                       size_t workspace_bytes, void* stream) {
  if (dwdt != ZQ_OUT_F32 && dwdt != ZQ_OUT_BF16) return ZQ_ERR_MODE;
  if (!rows_ok(M) || !rows_ok(N) || !k_ok(K) || ldg < N || parts < 1 || parts > 64 || g_stride < 0) return ZQ_ERR_SHAPE;
  if (N == 0) return ZQ_OK;
  if (!dw || (M > 0 && (!g_bf16 || !q || !s))) return ZQ_ERR_NULL;
  if (!al16(g_bf16) || !al16(q) || !al16(dw) || ldg % 8 || g_stride % 8) return ZQ_ERR_ALIGN;
  if (!workspace || workspace_bytes < kWsHeadBytes) return ZQ_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return ZQ_ERR_ALIGN;
  if (int e = check_device_sm100()) return e;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (M == 0)  // an empty sum
    return cudaMemsetAsync(dw, 0, static_cast<size_t>(parts) * N * K * (dwdt == ZQ_OUT_F32 ? 4 : 2), st) == cudaSuccess
               ? ZQ_OK
               : ZQ_ERR_CUDA;
  WgradArgs a{};
  a.g = g_bf16;
  a.ldg = ldg;
  a.g_stride = g_stride;
  a.q = q;
  a.s = s;
  a.parts = parts;
  a.M = M;
  a.N = N;
  a.K = K;
  a.dw = dw;
  a.dwdt = dwdt;
  a.status = static_cast<int*>(workspace);
  return launch_wgrad(a, st);
}

}  // extern "C"
