// C-ABI entry points of the attention half of a decoder layer: norms with the position rotation, the 8-bit cache, attention
// over it.  Argument validation and dispatch; the operators are defined in include/zqfp.h.
#include <cmath>

#include "kv_attention.cuh"

using namespace zq;
using namespace zq::kv;

namespace {

bool aligned(const void* p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
constexpr int64_t kMaxRows = 0x7FFFFF00;
constexpr int64_t kMaxHeads = 65535;
bool dim_ok(int64_t D) { return D == 64 || D == 128; }
bool page_ok(int page) { return page == 16 || page == 32 || page == 64 || page == 128; }
// rows of `heads` heads side by side
bool row_ok(int64_t ld, int64_t heads, int64_t D) { return ld >= heads * D; }

// The cache and the sequences.  T: rows of the tensors that hold the new tokens; every one belongs to its own sequence
// where cu is NULL.
int check_cache(const uint8_t* codes, const float* scale, int64_t pages, int64_t H, int page, int64_t D, const int* table,
                int64_t table_ld, const int* lens, bool needs_lens, const int* cu, int64_t B, int64_t T, Cache& c) {
  if (pages < 1 || H < 1 || H > kMaxHeads || !page_ok(page) || !dim_ok(D) || pages > 0x7FFFFFFF || pages * 2 * H > 0x7FFFFFFF)
    return ZQ_ERR_SHAPE;
  if (B < 0 || T < 0 || B > kMaxRows || T > kMaxRows || table_ld < 0 || table_ld > kMaxRows || (!cu && needs_lens && B != T))
    return ZQ_ERR_SHAPE;
  if (!codes || !scale || (B > 0 && table_ld > 0 && !table) || (B > 0 && needs_lens && !lens)) return ZQ_ERR_NULL;
  if (!aligned(codes, 16) || !aligned(scale, 4) || !aligned(table, 4) || !aligned(lens, 4) || !aligned(cu, 4)) return ZQ_ERR_ALIGN;
  c.codes = const_cast<uint8_t*>(codes);
  c.scale = const_cast<float*>(scale);
  c.pages = pages;
  c.H = static_cast<int>(H);
  c.page = page;
  c.D = static_cast<int>(D);
  c.table = table;
  c.table_ld = table_ld;
  c.lens = lens;
  c.cu = cu;
  c.B = static_cast<int>(B);
  c.T = T;
  return ZQ_OK;
}

int check_norm_rope(const NormRopeArgs& a, int pairs) {
  if (a.T < 0 || a.T > kMaxRows || a.Hq < 0 || a.H < 0 || a.Hq > kMaxHeads || a.H > kMaxHeads || !dim_ok(a.D)) return ZQ_ERR_SHAPE;
  if (a.rot < 16 || a.rot % 16 || a.rot > a.D || a.far < 1) return ZQ_ERR_SHAPE;
  if (!(a.eps >= 0.0f) || std::isinf(a.eps)) return ZQ_ERR_SHAPE;
  if (pairs != ZQ_PAIRS_HALVES && pairs != ZQ_PAIRS_NEIGHBOURS) return ZQ_ERR_MODE;
  if (!row_ok(a.ldq, a.Hq, a.D) || !row_ok(a.ldk, a.H, a.D) || !row_ok(a.ldoq, a.Hq, a.D) || !row_ok(a.ldok, a.H, a.D)) return ZQ_ERR_SHAPE;
  if ((a.wq == nullptr) != (a.wk == nullptr)) return ZQ_ERR_NULL;
  return ZQ_OK;
}
bool rows_aligned(const void* p, int64_t ld) { return aligned(p, 16) && ld % 8 == 0; }

}  // namespace

extern "C" {

int zq_qk_norm_rope(const void* q, int64_t ldq, int64_t Hq, const void* k, int64_t ldk, int64_t H, int64_t T, int64_t D,
                    const float* wq, const float* wk, float eps, const float* table, int64_t far, int64_t rot, int pairs,
                    const int32_t* positions, void* q_out, int64_t ldqo, void* k_out, int64_t ldko, void* stream) {
  if (Hq < 0 || H < 0 || Hq > kMaxHeads || H > kMaxHeads || D > 128 || rot > 128) return ZQ_ERR_SHAPE;
  NormRopeArgs a{};
  a.q = q, a.k = k, a.ldq = ldq, a.ldk = ldk, a.T = T, a.Hq = static_cast<int>(Hq), a.H = static_cast<int>(H), a.D = static_cast<int>(D);
  a.wq = wq, a.wk = wk, a.eps = eps, a.table = table, a.far = far, a.rot = static_cast<int>(rot);
  a.neighbours = pairs == ZQ_PAIRS_NEIGHBOURS;
  a.positions = positions, a.oq = q_out, a.ok = k_out, a.ldoq = ldqo, a.ldok = ldko;
  if (int e = check_norm_rope(a, pairs)) return e;
  if (T == 0 || Hq + H == 0) return ZQ_OK;
  if (!table || !positions || (Hq > 0 && (!q || !q_out)) || (H > 0 && (!k || !k_out))) return ZQ_ERR_NULL;
  if (!rows_aligned(q, ldq) || !rows_aligned(k, ldk) || !rows_aligned(q_out, ldqo) || !rows_aligned(k_out, ldko) || !aligned(table, 16) ||
      !aligned(positions, 4) || !aligned(wq, 16) || !aligned(wk, 16))
    return ZQ_ERR_ALIGN;
  if (int e = check_device_sm100()) return e;
  return launch_norm_rope(a, static_cast<cudaStream_t>(stream));
}

size_t zq_qk_norm_rope_backward_workspace_bytes(int64_t D) {
  return dim_ok(D) ? kWsHeadBytes + sizeof(float) * kNormGradBlocks * 2 * D : 0;
}

int zq_qk_norm_rope_backward(const void* dq, int64_t lddq, const void* dk, int64_t lddk, const void* q, int64_t ldq, int64_t Hq,
                             const void* k, int64_t ldk, int64_t H, int64_t T, int64_t D, const float* wq, const float* wk,
                             float eps, const float* table, int64_t far, int64_t rot, int pairs, const int32_t* positions,
                             void* dxq, int64_t lddxq, void* dxk, int64_t lddxk, float* dwq, float* dwk, void* workspace,
                             size_t workspace_bytes, void* stream) {
  if (Hq < 0 || H < 0 || Hq > kMaxHeads || H > kMaxHeads || D > 128 || rot > 128) return ZQ_ERR_SHAPE;
  NormRopeArgs a{};
  a.q = q, a.k = k, a.ldq = ldq, a.ldk = ldk, a.T = T, a.Hq = static_cast<int>(Hq), a.H = static_cast<int>(H), a.D = static_cast<int>(D);
  a.dq = dq, a.dk = dk, a.lddq = lddq, a.lddk = lddk;
  a.wq = wq, a.wk = wk, a.eps = eps, a.table = table, a.far = far, a.rot = static_cast<int>(rot);
  a.neighbours = pairs == ZQ_PAIRS_NEIGHBOURS;
  a.positions = positions, a.oq = dxq, a.ok = dxk, a.ldoq = lddxq, a.ldok = lddxk, a.dwq = dwq, a.dwk = dwk;
  if (int e = check_norm_rope(a, pairs)) return e;
  if (!row_ok(lddq, Hq, D) || !row_ok(lddk, H, D)) return ZQ_ERR_SHAPE;
  if (wq && (!dwq || !dwk)) return ZQ_ERR_NULL;
  if (!aligned(dwq, 4) || !aligned(dwk, 4)) return ZQ_ERR_ALIGN;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (T == 0 || Hq + H == 0) {
    if (wq && (cudaMemsetAsync(dwq, 0, D * 4, st) != cudaSuccess || cudaMemsetAsync(dwk, 0, D * 4, st) != cudaSuccess)) return ZQ_ERR_CUDA;
    return ZQ_OK;
  }
  if (!table || !positions || (Hq > 0 && (!dq || !dxq || (wq && !q))) || (H > 0 && (!dk || !dxk || (wk && !k)))) return ZQ_ERR_NULL;
  if (!rows_aligned(q, ldq) || !rows_aligned(k, ldk) || !rows_aligned(dq, lddq) || !rows_aligned(dk, lddk) || !rows_aligned(dxq, lddxq) ||
      !rows_aligned(dxk, lddxk) || !aligned(table, 16) || !aligned(positions, 4) || !aligned(wq, 16) || !aligned(wk, 16))
    return ZQ_ERR_ALIGN;
  if (wq) {
    if (!workspace || workspace_bytes < zq_qk_norm_rope_backward_workspace_bytes(D)) return ZQ_ERR_WORKSPACE;
    if (!aligned(workspace, 256)) return ZQ_ERR_ALIGN;
    a.partial = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + kWsHeadBytes);
  }
  if (int e = check_device_sm100()) return e;
  return launch_norm_rope_backward(a, st);
}

int zq_kv_cache_write(const void* k, int64_t ldk, const void* v, int64_t ldv, int64_t T, const int32_t* cu, int64_t B,
                      const int32_t* lens, const int32_t* table, int64_t table_ld, uint8_t* codes, float* scale, int64_t pages,
                      int64_t H, int page, int64_t D, int mode, void* stream) {
  if (mode != ZQ_SCALE_NONE && mode != ZQ_SCALE_M1) return ZQ_ERR_MODE;
  WriteArgs a{};
  if (int e = check_cache(codes, scale, pages, H, page, D, table, table_ld, lens, true, cu, B, T, a.c)) return e;
  if (!row_ok(ldk, H, D) || !row_ok(ldv, H, D)) return ZQ_ERR_SHAPE;
  if (T == 0 || B == 0) return ZQ_OK;
  if (!k || !v) return ZQ_ERR_NULL;
  if (!rows_aligned(k, ldk) || !rows_aligned(v, ldv)) return ZQ_ERR_ALIGN;
  a.k = k, a.v = v, a.ldk = ldk, a.ldv = ldv, a.mode = mode;
  if (int e = check_device_sm100()) return e;
  return launch_write(a, static_cast<cudaStream_t>(stream));
}

int zq_kv_cache_read(const uint8_t* codes, const float* scale, int64_t pages, int64_t H, int page, int64_t D,
                     const int32_t* table, int64_t table_ld, const int32_t* cu, int64_t B, int64_t T, void* k, void* v,
                     zq_out_dtype dt, void* stream) {
  if (dt != ZQ_OUT_F32 && dt != ZQ_OUT_BF16) return ZQ_ERR_MODE;
  ReadArgs a{};
  if (int e = check_cache(codes, scale, pages, H, page, D, table, table_ld, nullptr, false, cu, B, T, a.c)) return e;
  if (T == 0 || B == 0) return ZQ_OK;
  if (!cu || !k || !v) return ZQ_ERR_NULL;
  if (!aligned(k, 16) || !aligned(v, 16)) return ZQ_ERR_ALIGN;
  a.k = k, a.v = v, a.dt = dt;
  if (int e = check_device_sm100()) return e;
  return launch_read(a, static_cast<cudaStream_t>(stream));
}

size_t zq_kv_attention_workspace_bytes(int64_t T, int64_t B, int64_t Hq, int64_t H, int64_t D) {
  if (T < 0 || B < 0 || T > kMaxRows || B > kMaxRows || H < 1 || H > kMaxHeads || Hq < H || Hq > kMaxHeads || Hq % H || !dim_ok(D)) return 0;
  const size_t few = few_workspace_bytes(D), rows = rows_workspace_bytes(D);
  return kWsHeadBytes + (few > rows ? few : rows);
}

int zq_kv_attention(const void* q, int64_t ldq, int64_t Hq, int64_t T, const int32_t* cu, int64_t B, const int32_t* lens,
                    const int32_t* table, int64_t table_ld, const uint8_t* codes, const float* scale, int64_t pages, int64_t H,
                    int page, int64_t D, float sm_scale, int causal, int64_t window, void* out, zq_out_dtype dt, int64_t ldo,
                    float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  if ((dt != ZQ_OUT_F32 && dt != ZQ_OUT_BF16) || (causal != 0 && causal != 1) || (window != 0 && !causal)) return ZQ_ERR_MODE;
  AttnArgs a{};
  if (int e = check_cache(codes, scale, pages, H, page, D, table, table_ld, lens, true, cu, B, T, a.c)) return e;
  if (Hq < H || Hq > kMaxHeads || Hq % H || window < 0 || !(sm_scale > 0.0f) || std::isinf(sm_scale) || T * (Hq / H) > kMaxRows)
    return ZQ_ERR_SHAPE;
  if (!row_ok(ldq, Hq, D) || !row_ok(ldo, Hq, D)) return ZQ_ERR_SHAPE;
  if (T == 0 || B == 0) return ZQ_OK;
  if (!q || !out) return ZQ_ERR_NULL;
  if (!rows_aligned(q, ldq) || !aligned(out, 16) || ldo % (dt == ZQ_OUT_F32 ? 4 : 8) || !aligned(lse, 4)) return ZQ_ERR_ALIGN;
  if (!workspace || workspace_bytes < zq_kv_attention_workspace_bytes(T, B, Hq, H, D)) return ZQ_ERR_WORKSPACE;
  if (!aligned(workspace, 256)) return ZQ_ERR_ALIGN;
  a.q = q, a.ldq = ldq, a.Hq = static_cast<int>(Hq), a.sm_scale = sm_scale, a.causal = causal;
  a.window = static_cast<int>(window < kMaxRows ? window : 0);  // wider than any sequence: none
  a.out = out, a.dt = dt, a.ldo = ldo, a.lse = lse, a.workspace = workspace;
  if (int e = check_device_sm100()) return e;
  return launch_attention(a, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
