// Entry points of the products with MXFP4 experts: arguments, scratch, and which kernels a call goes to.
#include <algorithm>

#include "fp4.cuh"

namespace cosmoe {

namespace {

bool misaligned(const void* p) { return ((uintptr_t)p & 15u) != 0; }
int check_matrix(const moe_fp4* m) {
  if (!m || m->rows < 0 || m->n <= 0) return MOE_ERR_INVALID_ARG;
  if (m->n > MOE_FP4_MAX_N || m->rows > MOE_FP4_MAX_ROWS) return MOE_ERR_UNSUPPORTED;
  if (m->rows > 0 && (!m->codes || !m->scales || misaligned(m->codes) || misaligned(m->scales))) return MOE_ERR_INVALID_ARG;
  return MOE_OK;
}

// Scratch of moe_fp4_experts.
struct Fp4Ws {
  size_t offsets, inv;
  size_t x_codes, x_scales, h_codes, h_scales, out_slots, arrived, total;
};
Fp4Ws fp4_ws(const moe_config& c, int T) {
  Fp4Ws L{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off = (off + bytes + 255) / 256 * 256;
    return o;
  };
  const long long n = (long long)T * c.top_k;
  const Fp4Shape x = fp4_shape(n, c.d_model), h = fp4_shape(n, c.d_ff);
  L.offsets = take((size_t)(c.n_experts + 1) * 4);
  L.inv = take((size_t)n * 4);
  L.x_codes = take((size_t)n * x.pitch), L.x_scales = take((size_t)x.chunks * x.rp * 4);
  L.h_codes = take((size_t)n * h.pitch), L.h_scales = take((size_t)h.chunks * h.rp * 4);
  // (few tokens: planes of the down product's parts)
  const long long few = (long long)std::min(T, MOE_STREAM_MAX_TOKENS) * c.top_k * kFewSplits;
  L.out_slots = take((size_t)std::max(n, few) * c.d_model * 4);
  L.arrived = take((size_t)((c.d_model + 63) / 64) * 4);
  L.total = off;
  return L;
}

}  // namespace
}  // namespace cosmoe

using namespace cosmoe;

extern "C" {

int moe_fp4_product(moe_ctx* ctx, const moe_fp4* a, const moe_fp4* w, const int32_t* expert_offsets, int32_t n_experts, void* out,
                    int32_t out_dtype, int64_t out_stride, void* stream) {
  if (!ctx || n_experts < 1) return MOE_ERR_INVALID_ARG;
  int rc = check_matrix(a);
  if (rc != MOE_OK || (rc = check_matrix(w)) != MOE_OK) return rc;
  if (out_dtype != MOE_F32 && out_dtype != MOE_BF16) return MOE_ERR_UNSUPPORTED;
  if (n_experts > MOE_MAX_EXPERTS) return MOE_ERR_UNSUPPORTED;
  if (a->n != w->n || w->rows == 0 || w->rows % n_experts) return MOE_ERR_INVALID_ARG;
  const int64_t N = w->rows / n_experts;
  if (N % 8) return MOE_ERR_UNSUPPORTED;
  if (out_stride < N || out_stride % 8) return MOE_ERR_INVALID_ARG;
  if (a->rows == 0) return MOE_OK;
  if (!expert_offsets || !out || misaligned(out) || ((uintptr_t)expert_offsets & 3u)) return MOE_ERR_INVALID_ARG;
  cudaStream_t s = (cudaStream_t)stream;
  if (a->rows <= MOE_FP4_FEW_ROWS && fp4_few_applies(ctx, a->n, (int)a->rows))
    return launch_fp4_few_rows(ctx, a, w, expert_offsets, n_experts, out, out_dtype == MOE_F32, out_stride, s);
  return launch_fp4_tensor(ctx, a, w, expert_offsets, n_experts, out, out_dtype == MOE_F32, out_stride, nullptr, s);
}

int moe_fp4_workspace_bytes(const moe_config* cfg, int32_t T, size_t* bytes) {
  if (!bytes) return MOE_ERR_INVALID_ARG;
  const int rc = validate_config(cfg);
  if (rc != MOE_OK) return rc;
  if (T < 0) return MOE_ERR_INVALID_ARG;
  if ((long long)T * cfg->top_k > MOE_FP4_MAX_ROWS) return MOE_ERR_UNSUPPORTED;
  *bytes = fp4_ws(*cfg, T).total;
  return MOE_OK;
}

int moe_fp4_experts(moe_ctx* ctx, const void* x, int32_t T, const moe_fp4* gu, const moe_fp4* down, const int32_t* topk_idx,
                    const float* topk_w, void* y, void* ws, size_t ws_bytes, void* stream) {
  if (!ctx || T < 0) return MOE_ERR_INVALID_ARG;
  const moe_config& c = ctx->cfg;
  if (c.wd_rank > 0) return MOE_ERR_UNSUPPORTED;
  int rc = check_matrix(gu);
  if (rc != MOE_OK || (rc = check_matrix(down)) != MOE_OK) return rc;
  if (gu->n != c.d_model || gu->rows != (int64_t)c.n_experts * ((c.d_ff + 31) / 32) * 64 || down->n != c.d_ff ||
      down->rows != (int64_t)c.n_experts * c.d_model)
    return MOE_ERR_INVALID_ARG;
  if (T == 0) return MOE_OK;
  if ((long long)T * c.top_k > MOE_FP4_MAX_ROWS) return MOE_ERR_UNSUPPORTED;
  if (!x || !y || !ws || !topk_idx || !topk_w || misaligned(x) || misaligned(y) || misaligned(ws) ||
      (((uintptr_t)topk_idx | (uintptr_t)topk_w) & 3u))
    return MOE_ERR_INVALID_ARG;
  const Fp4Ws L = fp4_ws(c, T);
  if (ws_bytes < L.total) return MOE_ERR_WORKSPACE;
  char* const b = (char*)ws;
  cudaStream_t s = (cudaStream_t)stream;
  const int n = T * c.top_k;
  const moe_fp4 xq{b + L.x_codes, b + L.x_scales, n, c.d_model}, h{b + L.h_codes, b + L.h_scales, n, c.d_ff};
  float* const o = (float*)(b + L.out_slots);
  if (T <= MOE_STREAM_MAX_TOKENS && fp4_few_applies(ctx, c.d_model, T) && fp4_few_applies(ctx, c.d_ff, T))
    return launch_fp4_few_experts(ctx, x, T, gu, down, topk_idx, topk_w, y, &h, o, (unsigned*)(b + L.arrived), s);
  int32_t *offsets = (int32_t*)(b + L.offsets), *inv = (int32_t*)(b + L.inv);
  rc = launch_fp4_place(ctx, x, topk_idx, T, offsets, inv, b + L.x_codes, b + L.x_scales, s);
  if (rc != MOE_OK) return rc;
  rc = launch_fp4_tensor(ctx, &xq, gu, offsets, c.n_experts, nullptr, 0, 0, &h, s);
  if (rc != MOE_OK) return rc;
  rc = launch_fp4_tensor(ctx, &h, down, offsets, c.n_experts, o, 1, c.d_model, nullptr, s);
  if (rc != MOE_OK) return rc;
  return launch_combine(ctx, o, topk_w, inv, T, y, 1, s);
}

}  // extern "C"
