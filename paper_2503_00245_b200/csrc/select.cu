// Expert selection from a router's logits.  Per token, with l its E logits and b a bias that only the selection sees:
//
//     s = softmax(l) or 1 / (1 + e^-l)        key = s + b   (the logits themselves where the scores would give the same order)
//     groups: the `groups_kept` of the G groups with the largest sum of their `group_top` largest keys stay
//     the k largest keys of what stays, equal keys to the lower expert;  w_j = scale s_j, or scale s_j / sum of the chosen s
//
// Scores that are compared with one another are formed in 64 bits: which of two experts is chosen is not left to the rounding of an
// exponential.  A logit of -inf (or NaN) switches an expert off: its key is -inf and its weight 0.
//
// One warp per token, eight experts to a lane at most.  Most tokens are decided in 32 bits: keys with a known bound on their error,
// and only where two neighbours among the chosen (or the next one), or the last group kept and the first one left, are nearer
// than the bound the token is decided again in 64 bits.  The bound grows with the largest |bias|: 16384 tokens of 256 experts in groups
// take 29 us with biases around 0.1, 34 where some are -1, 65 where some are -100 (or any size beyond): every token is then decided twice.
// What bounds it: 1070 instructions a token, 15 us of issue slots for those 16384 (8.4 MB of bf16 logits, 1.4 us of HBM).  The slots are
// 72 % taken while an SM works (chains of a reduction, a vote and a shuffle for each choice, with 7 warps a scheduler to hide them), and the
// busiest SM executes a fifth more than the mean: 3.5 tokens a warp, and those decided twice.  With all exponentials and the
// selection in 64 bits 68 us, in 32 bits with a search of a lane's keys for every choice 48.
#include <math_constants.h>

#include <algorithm>

#include "common.cuh"

namespace cosmoe {
namespace {

constexpr int kSelWarps = 8;
static_assert(MOE_SELECT_MAX_EXPERTS == 8 * 32, "experts of a lane");

// doubles as unsigned words of the same order (-0 counts as 0, NaN as -inf)
__device__ __forceinline__ unsigned long long f64_key(double v) {
  if (!(v == v)) v = -CUDART_INF;
  const unsigned long long b = (unsigned long long)__double_as_longlong(v + 0.0);
  return (b >> 63) ? ~b : b | 0x8000000000000000ull;
}
__device__ __forceinline__ double f64_unkey(unsigned long long k) {
  return __longlong_as_double((long long)((k >> 63) ? k ^ 0x8000000000000000ull : ~k));
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
__device__ __forceinline__ float logit_or_off(const T* row, int e) {
  const float v = logit(row + e);
  return v == v ? v : -CUDART_INF_F;
}

// ---- the same two steps on keys of either width: `Key` an unsigned word of the keys' order, 0 below every key.
__device__ __forceinline__ unsigned warp_max(unsigned v) { return __reduce_max_sync(0xffffffffu, v); }
__device__ __forceinline__ unsigned long long warp_max(unsigned long long v) {
  const unsigned hi = __reduce_max_sync(0xffffffffu, (unsigned)(v >> 32));
  const unsigned lo = __reduce_max_sync(0xffffffffu, (unsigned)(v >> 32) == hi ? (unsigned)v : 0u);
  return (unsigned long long)hi << 32 | lo;
}
__device__ __forceinline__ float reciprocal(float v) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
// e^(a - b), a <= b.  The difference is rounded, which would cost the power |a - b| 2^-24 of itself; what it lost (exact: two-sum) is
// put back, so the power is as good as expf's (within 2.6 2^-24 of itself, measured over its arguments) and one product's.  0 below
// e^-104, where fp32 ends.
__device__ __forceinline__ float exp_difference(float a, float b) {
  const float d = a - b, minus_b = d - a, lost = (a - (d - minus_b)) - (b + minus_b), e = expf(d);
  return d > -104.f ? fmaf(e, lost, e) : 0.f;
}
__device__ __forceinline__ unsigned f32_word(float v) { return f32_key(v == v ? v : -CUDART_INF_F); }
__device__ __forceinline__ unsigned key_of(float v) { return f32_word(v); }
__device__ __forceinline__ unsigned long long key_of(double v) { return f64_key(v); }
__device__ __forceinline__ float value_of(unsigned k) { return f32_unkey(k); }
__device__ __forceinline__ double value_of(unsigned long long k) { return f64_unkey(k); }

// Groups that stay, as a mask.  `lanes` (a power of two) lanes share a group, lane / lanes; keys in shared memory.
template <typename Key>
__device__ __forceinline__ unsigned groups_kept(const Key* key, const moe_select_config& c, int per, int lanes, int lane) {
  const int G = c.n_groups, g = lane / lanes, sub = lane & (lanes - 1);
  Key a = 0, b = 0;  // the two largest
  if (g < G)
    for (int i = sub; i < per; i += lanes) {
      const Key v = key[g * per + i];
      if (v > a) b = a, a = v;
      else if (v > b) b = v;
    }
  for (int o = lanes >> 1; o > 0; o >>= 1) {
    const Key oa = __shfl_xor_sync(0xffffffffu, a, o), ob = __shfl_xor_sync(0xffffffffu, b, o);
    const Key lo = a < oa ? a : oa;
    a = a < oa ? oa : a;
    b = lo > b ? lo : b;
    b = ob > b ? ob : b;
  }
  Key mine = 0;
  if (sub == 0 && g < G) mine = c.group_top == 1 ? a : key_of(value_of(a) + value_of(b));
  unsigned kept = 0u;
  for (int j = 0; j < c.groups_kept; ++j) {
    const Key best = warp_max(mine);
    const int win = __ffs(__ballot_sync(0xffffffffu, mine == best)) - 1;
    kept |= 1u << (win / lanes);
    if (lane == win) mine = 0;
  }
  return kept;
}

// The k largest of the lanes' keys mine[0..N), expert lane + 32 i, equal ones in the experts' order: lane j < k gets the j-th choice.
template <typename Key, int N>
__device__ __forceinline__ int choose(Key (&mine)[N], int k, int lane) {
  int my_e = 0;
  Key best = 0;
  int at = 0;
  auto local = [&] {
    best = mine[0], at = 0;
#pragma unroll
    for (int i = 1; i < N; ++i)
      if (mine[i] > best) best = mine[i], at = i;
  };
  local();
  for (int j = 0; j < k; ++j) {
    const Key top = warp_max(best);
    // of equal keys the lowest expert: the lane's own candidate already is its lowest
    const unsigned e = __reduce_min_sync(0xffffffffu, best == top ? (unsigned)(lane + 32 * at) : 0xffffffffu);
    if (lane == j) my_e = (int)e;
    if ((int)(e & 31u) == lane) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i == (int)(e >> 5)) mine[i] = 0;
      local();
    }
  }
  return my_e;
}

// ---- keys in 32 bits, where neighbours within `margin` are decided elsewhere, so that equal ones need no order and -inf may stand
// for "not there".  A key's three lowest bits hold which of the lane's experts it is: eight units in the last place at most.
__device__ __forceinline__ float warp_max_f(float v) {
  float r;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
// A lane's keys sorted once (a bitonic network, descending), the largest taken off the front: a few moves in place of a search.
template <int N>
__device__ __forceinline__ int choose_apart(float (&a)[N], int k, int lane, float margin, bool& near) {
#pragma unroll
  for (int size = 2; size <= N; size *= 2)
#pragma unroll
    for (int step = size / 2; step > 0; step /= 2)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int o = i ^ step;
        if (o > i) {
          const float hi = fmaxf(a[i], a[o]), lo = fminf(a[i], a[o]);
          a[i] = (i & size) == 0 ? hi : lo, a[o] = (i & size) == 0 ? lo : hi;
        }
      }
  int my_e = 0;
  float last = CUDART_INF_F;
#pragma unroll 1
  for (int j = 0; j < k; ++j) {
    const float top = warp_max_f(a[0]);
    const int win = __ffs(__ballot_sync(0xffffffffu, a[0] == top)) - 1;
    near = near || !(last - top > margin);
    last = top;
    if (lane == j) my_e = (int)(__float_as_uint(top) & (unsigned)(N - 1)) * 32 + win;
    if (lane == win) {
#pragma unroll
      for (int i = 0; i + 1 < N; ++i) a[i] = a[i + 1];
      a[N - 1] = -CUDART_INF_F;
    }
  }
  near = near || !(last - warp_max_f(a[0]) > margin);
  return my_e;
}
// Groups that stay, as groups_kept().
__device__ __forceinline__ unsigned groups_apart(const float* key, const moe_select_config& c, int per, int lanes, int lane, float margin,
                                                 bool& near) {
  const int g = lane / lanes, sub = lane & (lanes - 1);
  float a = -CUDART_INF_F, b = -CUDART_INF_F;
  if (g < c.n_groups)
    for (int i = sub; i < per; i += lanes) {
      const float v = key[g * per + i], t = fminf(a, v);
      a = fmaxf(a, v), b = fmaxf(b, t);
    }
  for (int o = lanes >> 1; o > 0; o >>= 1) {
    const float oa = __shfl_xor_sync(0xffffffffu, a, o), ob = __shfl_xor_sync(0xffffffffu, b, o), t = fminf(a, oa);
    a = fmaxf(a, oa), b = fmaxf(fmaxf(b, ob), t);
  }
  float mine = sub == 0 && g < c.n_groups ? (c.group_top == 1 ? a : a + b) : -CUDART_INF_F;
  unsigned kept = 0u;
  float last = 0.f;
#pragma unroll 1
  for (int j = 0; j < c.groups_kept; ++j) {
    last = warp_max_f(mine);
    const int win = max(__ffs(__ballot_sync(0xffffffffu, mine == last)) - 1, 0);  // (none: an infinite bias, decided in 64 bits)
    near = near || !(last > -CUDART_INF_F);
    kept |= 1u << (win / lanes);
    if (lane == win) mine = -CUDART_INF_F;
  }
  if (c.groups_kept < c.n_groups) near = near || !(last - warp_max_f(mine) > margin);
  return kept;
}

// N: experts of a lane.  Warps go from token to token with the bias in registers.  (Four blocks to an SM, 64 registers: with three,
// 16384 tokens of 256 experts take 35 us in place of 30.)
template <typename T, int N>
__global__ void __launch_bounds__(kSelWarps * 32, 4) select_kernel(const SelectParams P) {
  __shared__ unsigned long long s_key[kSelWarps][N * 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const moe_select_config& c = P.c;
  const int E = c.n_experts, k = c.top_k, G = c.n_groups, per = E / G;
  int lanes = 1;  // of a group
  while (2 * lanes * G <= 32) lanes *= 2;
  const unsigned inv_per = (65536u + per - 1) / per;  // (e inv_per >> 16 is e / per: e < 256, so the excess is below 1 / per)
  const bool softmax = c.scoring == MOE_SCORE_SOFTMAX;
  const bool by_logits = !P.bias && (G == 1 || c.group_top == 1);
  const bool weight_total = softmax && !c.renorm;  // the total of a softmax divides the weights too
  pdl_launch_dependents();
  pdl_wait();
  float bias[N];
  float most = 0.f;  // |bias|
#pragma unroll
  for (int i = 0; i < N; ++i) {
    bias[i] = P.bias && lane + 32 * i < E ? __ldg(P.bias + lane + 32 * i) : 0.f;
    most = fmaxf(most, fabsf(bias[i]));
  }
  most = warp_max_f(most);
  // Keys in 32 bits.  e^d = 2^(d log2 e) on the special-function unit: d (a softmax's difference), the exponent and its factor are
  // rounded (2.25 2^-24 |d|), the power is within 2^-22 (PTX manual), so e^d is off by (2.25 |d| + 4) 2^-24 e^d, at most 5 2^-24 of 1
  // (|d| e^d <= 1 / e).  In a sum of E such terms the part that grows with |d| is 2.25 2^-24 of their mean |d|, which is at most ln E
  // (5.6): with 4 2^-24 for the powers and 13 steps of addition, 30 2^-24 of itself; the quotient, with an approximate reciprocal
  // (2^-23): 38 2^-24 of a score of at most 1.  A sigmoid: |l| e^-l / (1 + e^-l)^2 <= 1 / 2, below 16 2^-24.  Adding the bias rounds at
  // 2^-24 of the sum, the expert's number in the low bits takes 16 2^-24, adding two keys rounds again.  So a key is known to 56
  // 2^-24 (1 + |bias|), a sum of two to 114 2^-24; twice that is below the margin of 256 2^-24 (1 + |bias|).
  const float margin = by_logits ? -1.f : (1.f + most) * (256.f / 16777216.f);

#pragma unroll 1
  for (long long t = blockIdx.x * kSelWarps + warp; t < P.T; t += gridDim.x * kSelWarps) {
    const T* row = (const T*)P.logits + t * P.stride;
    // ---- logits (NaN counts as -inf), the largest
    float l[N];
    float m = -CUDART_INF_F;
#pragma unroll
    for (int i = 0; i < N; ++i) l[i] = lane + 32 * i < E ? logit(row + lane + 32 * i) : -CUDART_INF_F;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      l[i] = fmaxf(l[i], -CUDART_INF_F);  // (the number of the two, where one is NaN)
      m = fmaxf(m, l[i]);
    }
    if (softmax) m = warp_max_f(m);
    auto score = [&](float v) -> double {  // of the softmax: before the division
      if (v == -CUDART_INF_F) return 0.0;
      if (softmax) return v == m ? 1.0 : exp((double)v - (double)m);
      return 1.0 / (1.0 + exp(-(double)v));
    };
    float tot = 1.f;
    float s[N];
    if (weight_total) {  // (to the weights' accuracy: terms within 4 2^-24 of themselves, added in 64 bits)
      double part = 0.0;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        s[i] = l[i] == -CUDART_INF_F ? 0.f : l[i] == m ? 1.f : exp_difference(l[i], m);
        part += (double)s[i];
      }
      tot = (float)warp_sum64(part);
    } else if (!by_logits) {
      float part = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float d = softmax ? l[i] - m : -l[i];
        float x;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(x) : "f"(d * 1.4426950408889634f));
        s[i] = softmax ? (l[i] == m ? 1.f : x) : reciprocal(1.f + x);
        if (l[i] == -CUDART_INF_F) s[i] = 0.f;
        part += s[i];
      }
      if (softmax) tot = warp_sum(part);
    }
    if (!(tot > 0.f)) tot = 1.f;
    bool near = false;
    int my_e;
    if (by_logits) {  // (exact as they are)
      unsigned mine[N];
#pragma unroll
      for (int i = 0; i < N; ++i) mine[i] = lane + 32 * i < E ? f32_key(l[i]) : 0u;
      if (G > 1) {
        unsigned* const key = reinterpret_cast<unsigned*>(s_key[warp]);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < N; ++i) key[lane + 32 * i] = mine[i];
        __syncwarp();
        const unsigned kept = groups_kept<unsigned>(key, c, per, lanes, lane);
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (!((kept >> ((lane + 32 * i) * inv_per >> 16)) & 1u)) mine[i] = 0u;
      }
      my_e = choose<unsigned, N>(mine, k, lane);
    } else {
      float mine[N];
      const float r = softmax ? reciprocal(tot) : 1.f;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float v = s[i] * r + bias[i];
        mine[i] = l[i] == -CUDART_INF_F ? l[i] : __uint_as_float((__float_as_uint(v) & ~(unsigned)(N - 1)) | (unsigned)i);
      }
      if (G > 1) {
        float* const key = reinterpret_cast<float*>(s_key[warp]);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < N; ++i) key[lane + 32 * i] = mine[i];
        __syncwarp();
        const unsigned kept = groups_apart(key, c, per, lanes, lane, margin, near);
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (!((kept >> ((lane + 32 * i) * inv_per >> 16)) & 1u)) mine[i] = -CUDART_INF_F;
      }
      my_e = choose_apart<N>(mine, k, lane, margin, near);
    }
    // ---- in 64 bits, where that was not enough
    if (!by_logits && near) {
      double tot64 = 1.0;
      if (softmax) {
        double part = 0.0;
#pragma unroll 1
        for (int e = lane; e < E; e += 32) part += score(logit_or_off(row, e));
        tot64 = warp_sum64(part);
        if (!(tot64 > 0.0)) tot64 = 1.0;
      }
      unsigned long long* const key = s_key[warp];
      __syncwarp();
#pragma unroll 1
      for (int e = lane; e < E; e += 32) {
        const float le = logit_or_off(row, e);
        double v = score(le) / tot64;
        if (P.bias) v += (double)P.bias[e];
        key[e] = f64_key(le == -CUDART_INF_F ? -CUDART_INF : v);
      }
      __syncwarp();
      unsigned kept = 0xffffffffu;
      if (G > 1) kept = groups_kept<unsigned long long>(key, c, per, lanes, lane);
      unsigned long long wide[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const unsigned e = lane + 32 * i;
        wide[i] = (int)e < E && (G == 1 || (kept >> (e * inv_per >> 16)) & 1u) ? key[e] : 0ull;
      }
      my_e = choose<unsigned long long, N>(wide, k, lane);
    }
    // ---- weights: the chosen scores, in 32 bits where none of them is so small that 32 bits lose it.  A score is within 4
    // (softmax) or 5 (sigmoid) 2^-24 of itself; renormalised, with a sum of eight, a quotient and the factor, a weight is within 15
    // 2^-24, else, with a total within 5, within 11.
    const float my_l = lane < k ? logit_or_off(row, my_e) : 0.f;
    float s32 = 0.f;
    if (lane < k) s32 = my_l == -CUDART_INF_F ? 0.f : softmax ? (my_l == m ? 1.f : exp_difference(my_l, m)) : 1.f / (1.f + expf(-my_l));
    float w;
    if (__all_sync(0xffffffffu, lane >= k || s32 > 1e-30f)) {
      w = c.renorm ? s32 / warp_sum(s32) : s32 / tot;
      w *= c.scale;
    } else {
      double my_s = lane < k ? score(my_l) : 0.0;
      if (c.renorm) {
        const double sum = warp_sum64(my_s);
        my_s = sum > 0.0 ? my_s / sum : 0.0;
      } else if (softmax) {
        my_s /= (double)tot;
      }
      w = (float)(my_s * (double)c.scale);
    }
    if (lane < k) {
      P.idx[t * k + lane] = my_e;
      P.w[t * k + lane] = w;
    }
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
  // (a few tokens for each warp where there are many: 148 SMs hold about 600 of these blocks)
  const dim3 grid(std::min((T - 1) / kSelWarps + 1, 592)), block(kSelWarps * 32);
  cudaStream_t s = (cudaStream_t)stream;
#define SELECT(N)                                                              \
  MOE_CUDA_TRY(dtype == MOE_F32 ? launch_pdl(select_kernel<float, N>, grid, block, 0, s, P) \
                                : launch_pdl(select_kernel<__nv_bfloat16, N>, grid, block, 0, s, P))
  if (c.n_experts <= 32) SELECT(1);
  else if (c.n_experts <= 64) SELECT(2);
  else if (c.n_experts <= 128) SELECT(4);
  else SELECT(8);
#undef SELECT
  return MOE_OK;
}
