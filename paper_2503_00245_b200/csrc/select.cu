// Expert selection from a router's logits.  Per token, with l its E logits and b a bias that only the selection sees:
//
//     s = softmax(l) or 1 / (1 + e^-l)        key = s + b   (the logits themselves where the scores would give the same order)
//     groups: the `groups_kept` of the G groups with the largest sum of their `group_top` largest keys stay
//     the k largest keys of what stays, equal keys to the lower expert;  w_j = scale s_j, or scale s_j / sum of the chosen s
//
// Scores that are compared with one another are formed in 64 bits: which of two experts is chosen is not left to the rounding of an
// exponential.  A logit of -inf (or NaN) switches an expert off: its key is -inf and its weight 0.
//
// One warp per token, the keys in shared memory.
#include <math_constants.h>

#include <algorithm>

#include "common.cuh"

namespace cosmoe {
namespace {

constexpr int kSelWarps = 8;
constexpr int kSelPer = MOE_SELECT_MAX_EXPERTS / 32;  // experts of a lane

// doubles as unsigned words of the same order (-0 counts as 0, NaN as -inf)
__device__ __forceinline__ unsigned long long f64_key(double v) {
  if (!(v == v)) v = -CUDART_INF;
  const unsigned long long b = (unsigned long long)__double_as_longlong(v + 0.0);
  return (b >> 63) ? ~b : b | 0x8000000000000000ull;
}
__device__ __forceinline__ double f64_unkey(unsigned long long k) {
  return __longlong_as_double((long long)((k >> 63) ? k ^ 0x8000000000000000ull : ~k));
}
__device__ __forceinline__ unsigned long long warp_max64(unsigned long long v) {
  const unsigned hi = __reduce_max_sync(0xffffffffu, (unsigned)(v >> 32));
  const unsigned lo = __reduce_max_sync(0xffffffffu, (unsigned)(v >> 32) == hi ? (unsigned)v : 0u);
  return (unsigned long long)hi << 32 | lo;
}
__device__ __forceinline__ double warp_sum64(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

struct SelectParams {
  moe_select_config c;
  const void* logits;
  long long stride;
  const float* bias;
  int T;
  int32_t* idx;
  float* w;
};

__device__ __forceinline__ float logit(const float* p) { return __ldcg(p); }
__device__ __forceinline__ float logit(const __nv_bfloat16* p) { return bf16_to_float(__ldcg(reinterpret_cast<const uint16_t*>(p))); }

template <typename T>
__global__ void __launch_bounds__(kSelWarps * 32) select_kernel(const SelectParams P) {
  __shared__ unsigned long long s_key[kSelWarps][MOE_SELECT_MAX_EXPERTS];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const moe_select_config& c = P.c;
  const int E = c.n_experts, k = c.top_k, G = c.n_groups, per = E / G;
  pdl_launch_dependents();
  pdl_wait();
  const int t = blockIdx.x * kSelWarps + warp;
  if (t >= P.T) return;
  const T* row = (const T*)P.logits + t * P.stride;
  unsigned long long* const key = s_key[warp];
  // ---- logits (NaN counts as -inf), the largest, scores
  float l[kSelPer];
  float m = -CUDART_INF_F;
#pragma unroll
  for (int i = 0; i < kSelPer; ++i) {
    const int e = lane + 32 * i;
    l[i] = e < E ? logit(row + e) : -CUDART_INF_F;
    if (!(l[i] == l[i])) l[i] = -CUDART_INF_F;
    m = fmaxf(m, l[i]);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  const bool softmax = c.scoring == MOE_SCORE_SOFTMAX;
  auto score = [&](float v) -> double {  // of the softmax: before the division
    if (v == -CUDART_INF_F) return 0.0;
    if (softmax) return v == m ? 1.0 : exp((double)v - (double)m);
    return 1.0 / (1.0 + exp(-(double)v));
  };
  const bool by_logits = !P.bias && (G == 1 || c.group_top == 1);
  double tot = 1.0;
  if (softmax && (!by_logits || !c.renorm)) {
    double part = 0.0;
#pragma unroll
    for (int i = 0; i < kSelPer; ++i) part += score(l[i]);
    tot = warp_sum64(part);
    if (!(tot > 0.0)) tot = 1.0;
  }
#pragma unroll
  for (int i = 0; i < kSelPer; ++i) {
    const int e = lane + 32 * i;
    if (e >= E) break;
    double v = by_logits ? (double)l[i] : score(l[i]) / tot;
    if (P.bias) v += (double)P.bias[e];
    key[e] = f64_key(l[i] == -CUDART_INF_F ? -CUDART_INF : v);
  }
  __syncwarp();
  // ---- groups that stay: lane g ranks group g
  unsigned kept = 0xffffffffu;
  if (G > 1) {
    unsigned long long a = 0ull, b = 0ull;  // the two largest keys
    if (lane < G)
      for (int i = 0; i < per; ++i) {
        const unsigned long long v = key[lane * per + i];
        if (v > a) b = a, a = v;
        else if (v > b) b = v;
      }
    unsigned long long g = 0ull;
    if (lane < G) g = c.group_top == 1 ? a : f64_key(f64_unkey(a) + f64_unkey(b));
    kept = 0u;
    for (int j = 0; j < c.groups_kept; ++j) {
      const unsigned long long best = warp_max64(g);
      const int win = __ffs(__ballot_sync(0xffffffffu, g == best)) - 1;
      kept |= 1u << win;
      if (lane == win) g = 0ull;
    }
  }
  // ---- the k largest keys of what stays (0: taken or not there, below every key)
  unsigned long long mine[kSelPer];
#pragma unroll
  for (int i = 0; i < kSelPer; ++i) {
    const int e = lane + 32 * i;
    mine[i] = e < E && (G == 1 || (kept >> (e / per)) & 1u) ? key[e] : 0ull;
  }
  double my_s = 0.0, sum = 0.0;
  int my_e = 0;
  for (int j = 0; j < k; ++j) {
    unsigned long long best = 0ull;
    int at = 0;
#pragma unroll
    for (int i = 0; i < kSelPer; ++i)
      if (mine[i] > best) best = mine[i], at = i;
    const unsigned long long top = warp_max64(best);
    const unsigned e = __reduce_min_sync(0xffffffffu, best == top ? (unsigned)(lane + 32 * at) : 0xffffffffu);
    const bool owner = (int)(e & 31u) == lane;
    float lv = 0.f;
#pragma unroll
    for (int i = 0; i < kSelPer; ++i)
      if (owner && i == (int)(e >> 5)) mine[i] = 0ull, lv = l[i];
    lv = __shfl_sync(0xffffffffu, lv, (int)(e & 31u));
    if (lane == j) my_e = (int)e, my_s = score(lv) / tot;
  }
  if (c.renorm) {
    sum = warp_sum64(lane < k ? my_s : 0.0);
    my_s = sum > 0.0 ? my_s / sum : 0.0;
  }
  if (lane < k) {
    P.idx[(long long)t * k + lane] = my_e;
    P.w[(long long)t * k + lane] = (float)(my_s * (double)c.scale);
  }
}

}  // namespace
}  // namespace cosmoe

using namespace cosmoe;

extern "C" int moe_select(const moe_select_config* cfg, const void* logits, int32_t dtype, int64_t stride, int32_t T, const float* bias,
                          int32_t* topk_idx, float* topk_w, void* stream) {
  if (!cfg || T < 0) return MOE_ERR_INVALID_ARG;
  const moe_select_config& c = *cfg;
  if (c.n_experts < 1 || c.top_k < 1 || c.n_groups < 1 || c.groups_kept < 1 || c.group_top < 1) return MOE_ERR_INVALID_ARG;
  if (c.scoring != MOE_SCORE_SOFTMAX && c.scoring != MOE_SCORE_SIGMOID) return MOE_ERR_INVALID_ARG;
  if ((c.renorm != 0 && c.renorm != 1) || !(c.scale == c.scale)) return MOE_ERR_INVALID_ARG;
  if (dtype != MOE_F32 && dtype != MOE_BF16) return MOE_ERR_UNSUPPORTED;
  if (c.n_experts > MOE_SELECT_MAX_EXPERTS || c.n_groups > 32 || c.top_k > MOE_MAX_TOPK || c.group_top > 2) return MOE_ERR_UNSUPPORTED;
  if (c.n_experts % c.n_groups || c.groups_kept > c.n_groups) return MOE_ERR_INVALID_ARG;
  const int per = c.n_experts / c.n_groups;
  if (c.group_top > per || c.top_k > c.groups_kept * per) return MOE_ERR_INVALID_ARG;
  if (stride < c.n_experts) return MOE_ERR_INVALID_ARG;
  if (T == 0) return MOE_OK;
  if (!logits || !topk_idx || !topk_w) return MOE_ERR_INVALID_ARG;
  if ((uintptr_t)logits % (dtype == MOE_F32 ? 4 : 2) || ((uintptr_t)bias | (uintptr_t)topk_idx | (uintptr_t)topk_w) & 3u) return MOE_ERR_INVALID_ARG;
  const SelectParams P{c, logits, stride, bias, T, topk_idx, topk_w};
  const dim3 grid((T + kSelWarps - 1) / kSelWarps), block(kSelWarps * 32);
  if (dtype == MOE_F32)
    MOE_CUDA_TRY(launch_pdl(select_kernel<float>, grid, block, 0, (cudaStream_t)stream, P));
  else
    MOE_CUDA_TRY(launch_pdl(select_kernel<__nv_bfloat16>, grid, block, 0, (cudaStream_t)stream, P));
  return MOE_OK;
}
