// C-ABI entry points of the FP8 operators with block scales: argument validation, workspace carving, dispatch.
// The operators are defined in include/zqfp.h.
#include "fp8_block.cuh"

using namespace zq;
using namespace zq::fp8b;

namespace {

inline bool al16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }
int rule_of(int mode) { return mode & ~ZQ_SCALES_POW2; }
// raw: the call quantizes an operand itself, by a rule that has to keep the promise of ZQ_SCALES_POW2
bool scale_rule_ok(int mode, bool raw = false) {
  const int rule = rule_of(mode);
  return (rule == ZQ_SCALE_NONE && !(raw && mode != rule)) || rule == ZQ_SCALE_M1;
}
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

int zq_quantize_fp8_block(const void* x, int64_t M, int64_t K, int64_t ldx, int mode, uint8_t* q, float* s,
                          void* stream) {
  if (mode != rule_of(mode) || !scale_rule_ok(mode)) return ZQ_ERR_MODE;
  if (!rows_ok(M) || !k_ok(K) || ldx < K) return ZQ_ERR_SHAPE;
  if (M == 0) return ZQ_OK;
  if (!x || !q || !s) return ZQ_ERR_NULL;
  if (!al16(x) || !al16(q) || ldx % 8) return ZQ_ERR_ALIGN;
  if (int e = check_device_sm100()) return e;
  return launch_quantize_block(x, M, K, ldx, mode, q, s, static_cast<cudaStream_t>(stream));
}

int zq_quantize_weight_fp8_block(const float* W, int64_t N, int64_t K, int mode, uint8_t* q, float* s,
                                 void* stream) {
  if (mode != rule_of(mode) || !scale_rule_ok(mode)) return ZQ_ERR_MODE;
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

int zq_fp8_block_linear(const uint8_t* q, const float* s, const void* x_bf16, int64_t ldx, int mode, int parts,
                        int64_t M, int64_t N, int64_t K, const uint8_t* w, const float* ws, void* y, zq_out_dtype ydt,
                        int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
  if (!scale_rule_ok(mode, x_bf16 != nullptr) || (ydt != ZQ_OUT_F32 && ydt != ZQ_OUT_BF16)) return ZQ_ERR_MODE;
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
  a.mode = rule_of(mode);
  a.pow2_scales = mode != a.mode;
  a.y = y;
  a.ydt = ydt;
  a.ldy = ldy;
  return launch(a, q, s, x_bf16, ldx, workspace, workspace_bytes, stream);
}

int zq_fp8_gated_linear(const uint8_t* q, const float* s, const void* x_bf16, int64_t ldx, int mode, int64_t M,
                        int64_t F, int64_t K, const uint8_t* w, const float* ws, zq_activation act, void* h_bf16,
                        int64_t ldh, uint8_t* hq, float* hs, uint8_t* gu, float* gus, void* workspace,
                        size_t workspace_bytes, void* stream) {
  if (!scale_rule_ok(mode, x_bf16 != nullptr) || !act_ok(act)) return ZQ_ERR_MODE;
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
  a.mode = rule_of(mode);
  a.pow2_scales = mode != a.mode;
  a.y = h_bf16;
  a.ydt = ZQ_OUT_BF16;
  a.ldy = ldh;
  a.q = hq;
  a.s = hs;
  a.ck = gu;
  a.cks = gus;
  return launch(a, q, s, x_bf16, ldx, workspace, workspace_bytes, stream);
}

int zq_fp8_gated_linear_backward(const uint8_t* q, const float* s, const void* dy_bf16, int64_t lddy, int mode,
                                 int64_t M, int64_t F, int64_t K, const uint8_t* wt, const float* wts, zq_activation act,
                                 const uint8_t* gu, const float* gus, void* dgu_bf16, uint8_t* dguq, float* dgus,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  if (!scale_rule_ok(mode, dy_bf16 != nullptr) || !act_ok(act)) return ZQ_ERR_MODE;
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
  a.mode = rule_of(mode);
  a.pow2_scales = mode != a.mode;
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
  if (parts == 1) g_stride = 0;  // there is no next matrix
  if (!rows_ok(M) || !rows_ok(N) || !k_ok(K) || ldg < N || parts < 1 || parts > 64 || g_stride < 0 ||
      (parts > 1 && g_stride == 0 && M > 0))
    return ZQ_ERR_SHAPE;
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

namespace {

// What the block keeps for its backward pass.
struct Saved {
  size_t xq, xs, gu, gus, hq, hs, total;
};
Saved saved_layout(int64_t M, int64_t K, int64_t F) {
  Saved v{};
  const size_t m = static_cast<size_t>(M), kb = static_cast<size_t>(blocks_of(K)), fb = static_cast<size_t>(blocks_of(F));
  v.xs = v.xq + up256(m * K);
  v.gu = v.xs + up256(kb * m * 4);
  v.gus = v.gu + up256(2 * m * F);
  v.hq = v.gus + up256(2 * fb * m * 4);
  v.hs = v.hq + up256(m * F);
  v.total = v.hs + up256(fb * m * 4);
  return v;
}
// Workspace of the whole block: the head, then the quantized input of the pass (x or dy), then either h or the
// gradients of g and u in bf16 and quantized.
struct WsFfn {
  size_t hq, hs, d, dq, ds, total;
};
WsFfn ws_ffn(int64_t M, int64_t K, int64_t F, int64_t N, bool training) {
  WsFfn v{};
  const size_t m = static_cast<size_t>(M), fb = static_cast<size_t>(blocks_of(F));
  const size_t in_x = ws8(M, K).total, in_dy = training ? ws8(M, N).total : 0;
  v.hq = v.d = in_x > in_dy ? in_x : in_dy;
  v.hs = v.hq + up256(m * F);
  v.total = v.hs + up256(fb * m * 4);
  v.dq = v.d + up256(4 * m * F);
  v.ds = v.dq + up256(2 * m * F);
  const size_t bwd = v.ds + up256(2 * fb * m * 4);
  if (training && bwd > v.total) v.total = bwd;
  return v;
}
bool ffn_sizes_ok(int64_t M, int64_t K, int64_t F, int64_t N) {
  return rows_ok(M) && k_ok(K) && k_ok(F) && rows_ok(N);
}

}  // namespace

size_t zq_fp8_gated_ffn_saved_bytes(int64_t M, int64_t K, int64_t F) {
  return ffn_sizes_ok(M, K, F, 0) ? saved_layout(M, K, F).total : 0;
}

size_t zq_fp8_gated_ffn_workspace_bytes(int64_t M, int64_t K, int64_t F, int64_t N, int training) {
  if (!ffn_sizes_ok(M, K, F, N) || (training && !k_ok(N))) return 0;
  return ws_ffn(M, K, F, N, training != 0).total;
}

int zq_fp8_gated_ffn(const void* x, int64_t ldx, int mode, int64_t M, int64_t K, int64_t F, int64_t N,
                     const uint8_t* gate_up, const float* gate_ups, const uint8_t* down, const float* downs,
                     zq_activation act, void* y, zq_out_dtype ydt, int64_t ldy, void* saved, void* workspace,
                     size_t workspace_bytes, void* stream) {
  // everything the second call would refuse is refused before the first one launches
  if (!scale_rule_ok(mode, true) || !act_ok(act) || (ydt != ZQ_OUT_F32 && ydt != ZQ_OUT_BF16)) return ZQ_ERR_MODE;
  if (!ffn_sizes_ok(M, K, F, N) || ldx < K || ldy < N) return ZQ_ERR_SHAPE;
  if (M == 0) return ZQ_OK;
  if (!x || !gate_up || !gate_ups || (N > 0 && (!down || !downs || !y))) return ZQ_ERR_NULL;
  if (!al16(x) || ldx % 8 || !al16(gate_up) || !al16(down) || (reinterpret_cast<uintptr_t>(saved) & 255u) ||
      (reinterpret_cast<uintptr_t>(y) & (ydt == ZQ_OUT_F32 ? 3u : 1u)))
    return ZQ_ERR_ALIGN;
  if (!workspace) return ZQ_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return ZQ_ERR_ALIGN;
  const WsFfn w = ws_ffn(M, K, F, N, false);
  if (workspace_bytes < w.total) return ZQ_ERR_WORKSPACE;
  uint8_t* base = static_cast<uint8_t*>(workspace);
  if (!saved) {
    uint8_t* hq = base + w.hq;
    float* hs = reinterpret_cast<float*>(base + w.hs);
    if (int e = zq_fp8_gated_linear(nullptr, nullptr, x, ldx, mode, M, F, K, gate_up, gate_ups, act, nullptr, 0, hq, hs,
                                    nullptr, nullptr, workspace, workspace_bytes, stream))
      return e;
    return zq_fp8_block_linear(hq, hs, nullptr, 0, mode, 1, M, N, F, down, downs, y, ydt, ldy, workspace, workspace_bytes,
                               stream);
  }
  const Saved v = saved_layout(M, K, F);
  uint8_t* sv = static_cast<uint8_t*>(saved);
  uint8_t* xq = sv + v.xq;
  float* xs = reinterpret_cast<float*>(sv + v.xs);
  uint8_t* hq = sv + v.hq;
  float* hs = reinterpret_cast<float*>(sv + v.hs);
  if (int e = zq_quantize_fp8_block(x, M, K, ldx, rule_of(mode), xq, xs, stream)) return e;
  if (int e = zq_fp8_gated_linear(xq, xs, nullptr, 0, mode, M, F, K, gate_up, gate_ups, act, nullptr, 0, hq, hs, sv + v.gu,
                                  reinterpret_cast<float*>(sv + v.gus), workspace, workspace_bytes, stream))
    return e;
  return zq_fp8_block_linear(hq, hs, nullptr, 0, mode, 1, M, N, F, down, downs, y, ydt, ldy, workspace, workspace_bytes,
                             stream);
}

int zq_fp8_gated_ffn_backward(const void* dy, int64_t lddy, int mode, int64_t M, int64_t K, int64_t F, int64_t N,
                              const void* saved, const uint8_t* gate_up_t, const float* gate_up_ts, const uint8_t* down_t,
                              const float* down_ts, zq_activation act, void* dx, void* dw_gate_up, void* dw_down,
                              zq_out_dtype dt, void* workspace, size_t workspace_bytes, void* stream) {
  if (!scale_rule_ok(mode, true) || !act_ok(act) || (dt != ZQ_OUT_F32 && dt != ZQ_OUT_BF16)) return ZQ_ERR_MODE;
  if (!ffn_sizes_ok(M, K, F, N) || !k_ok(N) || lddy < N) return ZQ_ERR_SHAPE;
  if (!dw_gate_up || !dw_down || (M > 0 && (!dy || !saved || !gate_up_t || !gate_up_ts || !down_t || !down_ts || !dx)))
    return ZQ_ERR_NULL;
  if (!al16(dy) || lddy % 8 || !al16(gate_up_t) || !al16(down_t) || !al16(dw_gate_up) || !al16(dw_down) ||
      (reinterpret_cast<uintptr_t>(saved) & 255u) || (reinterpret_cast<uintptr_t>(dx) & (dt == ZQ_OUT_F32 ? 3u : 1u)))
    return ZQ_ERR_ALIGN;
  if (!workspace) return ZQ_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) & 255u) return ZQ_ERR_ALIGN;
  const WsFfn w = ws_ffn(M, K, F, N, true);
  if (workspace_bytes < w.total) return ZQ_ERR_WORKSPACE;
  const Saved v = saved_layout(M, K, F);
  const uint8_t* sv = static_cast<const uint8_t*>(saved);
  uint8_t* base = static_cast<uint8_t*>(workspace);
  uint8_t* dq = base + w.dq;
  float* ds = reinterpret_cast<float*>(base + w.ds);
  if (int e = zq_fp8_gated_linear_backward(nullptr, nullptr, dy, lddy, mode, M, F, N, down_t, down_ts, act, sv + v.gu,
                                           reinterpret_cast<const float*>(sv + v.gus), base + w.d, dq, ds, workspace,
                                           workspace_bytes, stream))
    return e;
  if (int e = zq_fp8_block_linear(dq, ds, nullptr, 0, mode, 2, M, K, F, gate_up_t, gate_up_ts, dx, dt, K, workspace,
                                  workspace_bytes, stream))
    return e;
  if (int e = zq_fp8_weight_grad(base + w.d, F, M * F, 2, sv + v.xq, reinterpret_cast<const float*>(sv + v.xs), M, F, K,
                                 dw_gate_up, dt, workspace, workspace_bytes, stream))
    return e;
  return zq_fp8_weight_grad(dy, lddy, 0, 1, sv + v.hq, reinterpret_cast<const float*>(sv + v.hs), M, N, F, dw_down, dt,
                            workspace, workspace_bytes, stream);
}

}  // extern "C"
