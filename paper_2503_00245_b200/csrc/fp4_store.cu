// Rows to MXFP4 and back (formats and layout: csrc/fp4.cuh).
//
//     s = 2^(floor(log2 max|v|) - 2) over a block of 32 values      code = E2M1(v / s), nearest, ties to even, saturating at 6
//
// Dividing by a power of two is exact, so a code is decided without any rounding before it.  Both kernels move bytes and little
// else: 2 or 4 bytes in and 17/32 out per value, or the other way round.
#include <algorithm>

#include "fp4.cuh"

namespace cosmoe {
namespace {

constexpr int kQWarps = 8;

// Eight values of a row, as they come from memory.
struct Eight32 {
  float4 a, b;
};
struct Eight16 {
  uint4 w;
};
template <typename T>
struct EightOf;
template <>
struct EightOf<float> {
  typedef Eight32 type;
};
template <>
struct EightOf<__nv_bfloat16> {
  typedef Eight16 type;
};
__device__ __forceinline__ Eight32 load8(const float* p) {
  return Eight32{__ldg(reinterpret_cast<const float4*>(p)), __ldg(reinterpret_cast<const float4*>(p) + 1)};
}
__device__ __forceinline__ Eight16 load8(const __nv_bfloat16* p) { return Eight16{__ldg(reinterpret_cast<const uint4*>(p))}; }
// The scale byte of the four lanes' block, and the lane's eight codes.
__device__ __forceinline__ uint32_t quantize8(const Eight32& v, uint32_t& word) {
  const float f[8] = {v.a.x, v.a.y, v.a.z, v.a.w, v.b.x, v.b.y, v.b.z, v.b.w};
  uint32_t top = 0u;  // (as bits: a NaN is larger than everything)
#pragma unroll
  for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(f[j]) & 0x7fffffffu);
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  const uint32_t s = fp4_scale_byte(top);
  word = fp4_pack8(f, fp4_up(s));
  return s;
}
// bf16 two at a time: their bits order as unsigned words do, and a product with a power of two is exact (what it may lose below
// 2^-126 is far below the smallest code's quarter)
__device__ __forceinline__ uint32_t quantize8(const Eight16& v, uint32_t& word) {
  const uint32_t m = max_u16x2(max_u16x2(v.w.x & 0x7fff7fffu, v.w.y & 0x7fff7fffu), max_u16x2(v.w.z & 0x7fff7fffu, v.w.w & 0x7fff7fffu));
  uint32_t top = max(m & 0xffffu, m >> 16);
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  const uint32_t s = fp4_scale_byte(top << 16);
  const uint32_t up = s == 255u ? 0u : ((254u - s) << 7) * 0x10001u;
  const uint32_t w[4] = {v.w.x, v.w.y, v.w.z, v.w.w};
  uint32_t q[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t p = mul_bf16x2(w[j], up);
    q[j] = fp4_pack2(__uint_as_float(p << 16), __uint_as_float(p & 0xffff0000u));
  }
  word = s == 255u ? 0u : q[0] | q[1] << 8 | q[2] << 16 | q[3] << 24;
  return s;
}
__device__ __forceinline__ float one(const float* p) { return __ldg(p); }
__device__ __forceinline__ float one(const __nv_bfloat16* p) { return bf16_to_float(__ldg(reinterpret_cast<const uint16_t*>(p))); }

__device__ __forceinline__ long long source_row(const int32_t* row_of, int row_div, long long src_rows, long long i) {
  const long long r = row_of ? (long long)row_of[i] / row_div : i;
  return r >= 0 && r < src_rows && (!row_of || row_of[i] >= 0) ? r : -1;  // (-1: a row of zeros)
}

// Rows whose values lie side by side, n a multiple of 8, 16-byte aligned: a warp goes along a row, 256 values (eight to a lane) at a
// time with four such steps' loads on their way; gridDim.y warps share a row where there are few.  (A warp per 256 values, its row
// by a 64-bit division: 46080 x 2048 bf16 and back 152 us.)
constexpr int kFly = 4;
template <typename V>
__device__ __forceinline__ void quantize_step(const V& v, int c, int lane, const Fp4Shape& sh, uint32_t& word, uint32_t& scale) {
  const uint32_t s = quantize8(v, word);
  // a word of scales: four blocks, sixteen lanes
  scale = c < 32 * sh.nb ? s << (8 * ((lane >> 2) & 3)) : 0u;
  scale |= __shfl_xor_sync(0xffffffffu, scale, 4);
  scale |= __shfl_xor_sync(0xffffffffu, scale, 8);
}
__device__ __forceinline__ void store_step(uint32_t word, uint32_t scale, int c, long long i, int n, int lane, unsigned char* codes,
                                           uint32_t* scales, const Fp4Shape& sh) {
  if (c < 32 * sh.nb) *reinterpret_cast<uint32_t*>(codes + i * sh.pitch + c / 2) = word;
  if ((lane & 15) == 0 && c < n) scales[(long long)(c >> 7) * sh.rp + i] = scale;
}
template <typename T>
__global__ void __launch_bounds__(kQWarps * 32)
    fp4_quantize_kernel(const T* __restrict__ src, long long row_stride, long long src_rows, const int32_t* __restrict__ row_of, int row_div,
                        long long rows, int n, unsigned char* __restrict__ codes, uint32_t* __restrict__ scales, Fp4Shape sh) {
  const int lane = threadIdx.x & 31;
  pdl_launch_dependents();
  pdl_wait();
  for (long long i = (long long)blockIdx.x * kQWarps + (threadIdx.x >> 5); i < rows; i += (long long)gridDim.x * kQWarps) {
    const long long r = source_row(row_of, row_div, src_rows, i);
    const T* const row = src + (r < 0 ? 0 : r) * row_stride;
#pragma unroll 1
    for (int c0 = blockIdx.y * (256 * kFly) + lane * 8; c0 - lane * 8 < n; c0 += gridDim.y * (256 * kFly)) {
      typename EightOf<T>::type f[kFly];
#pragma unroll
      for (int u = 0; u < kFly; ++u) {
        f[u] = {};
        if (r >= 0 && c0 + 256 * u < n) f[u] = load8(row + c0 + 256 * u);
      }
#pragma unroll
      for (int u = 0; u < kFly; ++u)
        if (c0 - lane * 8 + 256 * u < n) {
          uint32_t word, scale;
          quantize_step(f[u], c0 + 256 * u, lane, sh, word, scale);
          store_step(word, scale, c0 + 256 * u, i, n, lane, codes, scales, sh);
        }
    }
  }
}

// Any strides: a thread takes a block of 32 values of a row, neighbouring threads neighbouring rows (matrices stored with their
// rows along the other axis, once when a model is loaded).
template <typename T>
__global__ void __launch_bounds__(256)
    fp4_quantize_any_kernel(const T* __restrict__ src, long long row_stride, long long col_stride, long long src_rows,
                            const int32_t* __restrict__ row_of, int row_div, long long rows, int n, int split,
                            unsigned char* __restrict__ codes, unsigned char* __restrict__ scales, Fp4Shape sh) {
  pdl_launch_dependents();
  pdl_wait();
  const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= rows) return;
  const long long r = source_row(row_of, row_div, src_rows, i);
  const long long o = split < 0 ? i : (i >> 5) * 64 + split * 32 + (i & 31);
  for (int b = blockIdx.y; b < sh.chunks * 4; b += gridDim.y) {
    unsigned char* const sb = scales + ((long long)(b >> 2) * sh.rp + o) * 4 + (b & 3);
    if (b >= sh.nb) {
      *sb = 0;
      continue;
    }
    float f[32];
    uint32_t top = 0u;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      const int c = b * 32 + j;
      f[j] = r >= 0 && c < n ? one(src + r * row_stride + c * col_stride) : 0.f;
      top = max(top, __float_as_uint(f[j]) & 0x7fffffffu);
    }
    const uint32_t s = fp4_scale_byte(top);
    const float up = fp4_up(s);
    *sb = (unsigned char)s;
    *reinterpret_cast<uint4*>(codes + o * sh.pitch + 16 * b) =
        make_uint4(fp4_pack8(f, up), fp4_pack8(f + 8, up), fp4_pack8(f + 16, up), fp4_pack8(f + 24, up));
  }
}

// Eight codes times their scale: a value and a power of two, exact in either type unless it overflows.
__device__ __forceinline__ void store8(__nv_bfloat16* p, uint32_t w, uint32_t s) {
  const uint32_t scale = fp4_scale_bf16x2(s);
  uint32_t v[4];
  fp4_bf16(w, v);
  *reinterpret_cast<uint4*>(p) = make_uint4(mul_bf16x2(v[0], scale), mul_bf16x2(v[1], scale), mul_bf16x2(v[2], scale), mul_bf16x2(v[3], scale));
}
__device__ __forceinline__ void store8(float* p, uint32_t w, uint32_t s) {
  const float scale = __uint_as_float(fp4_scale_bf16x2(s) << 16);
  uint32_t v[4];
  fp4_bf16(w, v);
#pragma unroll
  for (int h = 0; h < 2; ++h)
    reinterpret_cast<float4*>(p)[h] =
        make_float4(__uint_as_float(v[2 * h] << 16) * scale, __uint_as_float(v[2 * h] & 0xffff0000u) * scale,
                    __uint_as_float(v[2 * h + 1] << 16) * scale, __uint_as_float(v[2 * h + 1] & 0xffff0000u) * scale);
}
template <typename T>
__global__ void __launch_bounds__(kQWarps * 32)
    fp4_dequantize_kernel(const unsigned char* __restrict__ codes, const uint32_t* __restrict__ scales, long long rows, int n,
                          T* __restrict__ dst, long long row_stride, Fp4Shape sh) {
  const int lane = threadIdx.x & 31;
  pdl_launch_dependents();
  pdl_wait();
  for (long long i = (long long)blockIdx.x * kQWarps + (threadIdx.x >> 5); i < rows; i += (long long)gridDim.x * kQWarps) {
#pragma unroll 1
    for (int c0 = blockIdx.y * (256 * kFly) + lane * 8; c0 < n; c0 += gridDim.y * (256 * kFly)) {
      uint32_t w[kFly], sw[kFly];
#pragma unroll
      for (int u = 0; u < kFly; ++u) {
        const int c = min(c0 + 256 * u, n - 8);
        w[u] = __ldcg(reinterpret_cast<const uint32_t*>(codes + i * sh.pitch + c / 2));
        sw[u] = __ldcg(scales + (long long)(c >> 7) * sh.rp + i);
      }
#pragma unroll
      for (int u = 0; u < kFly; ++u) {
        const int c = c0 + 256 * u;
        if (c >= n) break;
        store8(dst + i * row_stride + c, w[u], (sw[u] >> (8 * ((c >> 5) & 3))) & 0xffu);
      }
    }
  }
}
// Blocks along the rows, and warps to share a row.
dim3 row_grid(long long rows, int n) {
  const long long x = std::min<long long>((rows + kQWarps - 1) / kQWarps, 148 * 8);
  const int most = (n + 256 * kFly - 1) / (256 * kFly);
  return dim3((unsigned)x, (unsigned)std::max(1, (int)std::min<long long>(most, 148 * 8 / x)));
}

template <typename T>
int quantize_t(const Fp4Source& q, long long rows, int n, void* codes, void* scales, long long rp, int split, cudaStream_t s) {
  Fp4Shape sh = fp4_shape(rows, n);
  sh.rp = rp;
  const T* base = (const T*)q.base;
  const bool wide = split < 0 && q.col_stride == 1 && n % 8 == 0 && (q.row_stride * (long long)sizeof(T)) % 16 == 0 && ((uintptr_t)base & 15u) == 0;
  if (wide) {
    MOE_CUDA_TRY(launch_pdl(fp4_quantize_kernel<T>, row_grid(rows, n), dim3(kQWarps * 32), 0, s, base, q.row_stride, q.rows, q.row_of,
                            q.row_div, rows, n, (unsigned char*)codes, (uint32_t*)scales, sh));
    return MOE_OK;
  }
  const long long blocks = (rows + 255) / 256;
  if (blocks > 0x7fffffffll) return MOE_ERR_UNSUPPORTED;
  MOE_CUDA_TRY(launch_pdl(fp4_quantize_any_kernel<T>, dim3((unsigned)blocks, (unsigned)std::min(sh.chunks * 4, 1024)), dim3(256), 0, s, base,
                          q.row_stride, q.col_stride, q.rows, q.row_of, q.row_div, rows, n, split, (unsigned char*)codes,
                          (unsigned char*)scales, sh));
  return MOE_OK;
}

// ---- rows of many tokens on their way to their experts: grouping and quantisation in one launch
// Pairs (token, choice) are numbered in order; a pair's slot is its expert's first slot plus the number of earlier pairs of that expert.
// Every CTA counts the pairs of all tokens by expert (n words from L2), those in front of its own tokens apart, ranks its own, and
// writes each of its tokens' rows, quantised once, to the token's k slots.  So no CTA waits for another and nothing is left to clear.
// There are two CTAs to an SM at most, whatever the number of tokens, as each walks all pairs: with 1024 tokens to a CTA and the more
// CTAs, the time went with the square (d 8, f 8, 8 of 8 experts: a call of a million tokens 9 ms, of four million 88, now 6 and 26).
// (A grouping launch of one CTA and a gathering one: 18 us for 2048 tokens, two experts each.)
constexpr int kPlaceWarps = 8;
struct PlaceParams {
  const void* x;
  const int32_t* idx;
  int T, k, E, d, tokens, piece;  // tokens of a CTA, and of those whose slots it holds at a time
  int32_t *offsets, *inv;
  unsigned char* codes;
  uint32_t* scales;
  Fp4Shape sh;
  DeviceState* st;
};
template <typename T, bool kPieces>  // (kPieces: more of them than one.  A loop in all launches cost those of one piece 0.5 us)
__global__ void __launch_bounds__(kPlaceWarps * 32) fp4_place_kernel(const PlaceParams P) {
  extern __shared__ int s_slot[];  // [piece][k]
  __shared__ int s_all[kPlaceWarps][MOE_MAX_EXPERTS], s_before[kPlaceWarps][MOE_MAX_EXPERTS], s_next[MOE_MAX_EXPERTS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_launch_dependents();
  for (int i = tid; i < kPlaceWarps * MOE_MAX_EXPERTS; i += kPlaceWarps * 32) (&s_all[0][0])[i] = 0, (&s_before[0][0])[i] = 0;
  __syncthreads();
  pdl_wait();
  const int t0 = blockIdx.x * P.tokens, t1 = min(t0 + P.tokens, P.T), n = P.T * P.k, own = t0 * P.k;
  auto expert = [&](int p) {  // -1: none
    const int e = p < n ? __ldcg(P.idx + p) : -1;
    return e >= 0 && e < P.E ? e : -1;
  };
  // ---- the warp's first row is on its way while the pairs are counted
  const int parts = (P.d + 256 * kFly - 1) / (256 * kFly);
  typename EightOf<T>::type f[kFly];
  auto fetch = [&](int from, int i) {
    const int t = i / parts, c0 = (i - t * parts) * 256 * kFly + lane * 8;
    const T* row = (const T*)P.x + (long long)(from + t) * P.d;
#pragma unroll
    for (int u = 0; u < kFly; ++u) {
      f[u] = {};
      if (c0 + 256 * u < P.d) f[u] = load8(row + c0 + 256 * u);
    }
  };
  if (warp < ((kPieces ? min(t0 + P.piece, t1) : t1) - t0) * parts) fetch(t0, warp);
  // ---- counts, by the warps' own counters; eight loads on their way
  const unsigned below = (1u << lane) - 1u;
  constexpr int kPairs = 8;
  for (int p0 = tid; p0 < n; p0 += kPairs * kPlaceWarps * 32) {
    int e[kPairs];
#pragma unroll
    for (int u = 0; u < kPairs; ++u) e[u] = expert(p0 + u * kPlaceWarps * 32);
#pragma unroll
    for (int u = 0; u < kPairs; ++u)
      if (e[u] >= 0) {
        atomicAdd(&s_all[warp][e[u]], 1);
        if (p0 + u * kPlaceWarps * 32 < own) atomicAdd(&s_before[warp][e[u]], 1);
      }
  }
  __syncthreads();
  if (warp == 0) {  // first slots of the experts, and of this CTA's pairs among theirs
    int all[2] = {0, 0}, before[2] = {0, 0};
#pragma unroll
    for (int h = 0; h < 2; ++h)
      for (int w = 0; w < kPlaceWarps; ++w) all[h] += s_all[w][lane + 32 * h], before[h] += s_before[w][lane + 32 * h];
    int a0 = all[0], a1 = all[1];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v0 = __shfl_up_sync(0xffffffffu, a0, o), v1 = __shfl_up_sync(0xffffffffu, a1, o);
      if (lane >= o) a0 += v0, a1 += v1;
    }
    const int half = __shfl_sync(0xffffffffu, a0, 31), total = half + __shfl_sync(0xffffffffu, a1, 31);
    a0 -= all[0], a1 += half - all[1];
    s_next[lane] = a0 + before[0], s_next[lane + 32] = a1 + before[1];
    if (blockIdx.x == 0) {
      if (lane < P.E) P.offsets[lane] = a0;
      if (lane + 32 < P.E) P.offsets[lane + 32] = a1;
      if (lane == 0) P.offsets[P.E] = total;
    }
    __syncwarp();
  }
  for (int from = t0;;) {
    const int to = kPieces ? min(from + P.piece, t1) : t1;
    if (warp == 0) {
      // ---- slots of the CTA's own pairs, in order
      const int mine = (to - from) * P.k, first = from * P.k;
      for (int p0 = 0; p0 < mine; p0 += 32) {
        const int p = p0 + lane, e = p < mine ? expert(first + p) : -1;
        if (p < mine && e < 0) flag_error(P.st, MOE_ERR_STATE, 0x530u);
        const unsigned peers = __match_any_sync(0xffffffffu, e);
        const int slot = e >= 0 ? s_next[e] + __popc(peers & below) : -1;
        __syncwarp();
        if (e >= 0 && (peers & below) == 0u) s_next[e] += __popc(peers);
        __syncwarp();
        // (a pair without an expert: any slot, its token is undefined)
        if (p < mine) s_slot[p] = slot, P.inv[first + p] = max(slot, 0);
      }
    }
    __syncthreads();
    // ---- the rows: a warp for 1024 values of a token
    const int tasks = (to - from) * parts;
    for (int i = warp; i < tasks; i += kPlaceWarps) {
      const int t = i / parts, c0 = (i - t * parts) * 256 * kFly + lane * 8;
      if ((kPieces && from != t0) || i != warp) fetch(from, i);
#pragma unroll
      for (int u = 0; u < kFly; ++u) {
        const int c = c0 + 256 * u;
        if (c - lane * 8 >= P.d) break;
        uint32_t word, scale;
        quantize_step(f[u], c, lane, P.sh, word, scale);
        for (int j = 0; j < P.k; ++j) {
          const int slot = s_slot[t * P.k + j];
          if (slot >= 0) store_step(word, scale, c, slot, P.d, lane, P.codes, P.scales, P.sh);
        }
      }
    }
    if (!kPieces || to == t1) break;
    __syncthreads();
    from = to;
  }
}

bool misaligned(const void* p) { return ((uintptr_t)p & 15u) != 0; }

}  // namespace

int launch_fp4_quantize(const Fp4Source& src, long long rows, int n, void* codes, void* scales, long long rp, int split, cudaStream_t s) {
  if (rows <= 0) return MOE_OK;
  return src.dtype == MOE_F32 ? quantize_t<float>(src, rows, n, codes, scales, rp, split, s)
                              : quantize_t<__nv_bfloat16>(src, rows, n, codes, scales, rp, split, s);
}

int launch_fp4_place(moe_ctx* ctx, const void* x, const int32_t* idx, int T, int32_t* offsets, int32_t* inv, void* codes, void* scales,
                     cudaStream_t s) {
  const moe_config& c = ctx->cfg;
  PlaceParams P{x, idx, T, c.top_k, c.n_experts, c.d_model, 0, 0, offsets, inv, (unsigned char*)codes, (uint32_t*)scales,
                fp4_shape((long long)T * c.top_k, c.d_model), ctx->d_state};
  P.tokens = std::max(2, (T - 1) / (2 * ctx->sm_count) + 1), P.piece = std::min(P.tokens, 1024);
  const dim3 grid((unsigned)((T - 1) / P.tokens + 1)), block(kPlaceWarps * 32);
  const size_t smem = (size_t)P.piece * c.top_k * 4;
  const bool pieces = P.piece < P.tokens;
  MOE_CUDA_TRY(launch_pdl(c.x_dtype == MOE_F32 ? (pieces ? fp4_place_kernel<float, true> : fp4_place_kernel<float, false>)
                                               : (pieces ? fp4_place_kernel<__nv_bfloat16, true> : fp4_place_kernel<__nv_bfloat16, false>),
                          grid, block, smem, s, P));
  ctx->launches++;
  return MOE_OK;
}

}  // namespace cosmoe

using namespace cosmoe;

extern "C" {

int moe_fp4_bytes(int64_t rows, int32_t n, size_t* codes_bytes, size_t* scales_bytes) {
  if (!codes_bytes || !scales_bytes || rows < 0 || n <= 0) return MOE_ERR_INVALID_ARG;
  if (n > MOE_FP4_MAX_N || rows > MOE_FP4_MAX_ROWS) return MOE_ERR_UNSUPPORTED;
  const Fp4Shape sh = fp4_shape(rows, n);
  *codes_bytes = (size_t)rows * sh.pitch, *scales_bytes = (size_t)sh.chunks * sh.rp * 4;
  return MOE_OK;
}

int moe_fp4_quantize_rows(const void* src, int32_t dtype, int64_t src_rows, int64_t row_stride, int64_t col_stride, const int32_t* row_of,
                          int32_t row_div, int64_t rows, int32_t n, void* codes, void* scales, void* stream) {
  if (rows < 0 || n <= 0 || src_rows < 0 || row_div < 1 || row_stride < 0 || col_stride < 0) return MOE_ERR_INVALID_ARG;
  if (dtype != MOE_F32 && dtype != MOE_BF16) return MOE_ERR_UNSUPPORTED;
  if (n > MOE_FP4_MAX_N || rows > MOE_FP4_MAX_ROWS) return MOE_ERR_UNSUPPORTED;
  if (!row_of && rows > src_rows) return MOE_ERR_INVALID_ARG;
  if (rows == 0) return MOE_OK;
  if (!codes || !scales || misaligned(codes) || misaligned(scales) || (src_rows > 0 && !src)) return MOE_ERR_INVALID_ARG;
  if ((uintptr_t)src % (dtype == MOE_F32 ? 4 : 2) || ((uintptr_t)row_of & 3u)) return MOE_ERR_INVALID_ARG;
  return launch_fp4_quantize(Fp4Source{src, dtype, row_stride, col_stride, src_rows, row_of, row_div}, rows, n, codes, scales,
                             fp4_shape(rows, n).rp, -1, (cudaStream_t)stream);
}

int moe_fp4_dequantize_rows(const moe_fp4* m, void* dst, int32_t dtype, int64_t row_stride, void* stream) {
  if (!m || m->rows < 0 || m->n <= 0) return MOE_ERR_INVALID_ARG;
  if (dtype != MOE_F32 && dtype != MOE_BF16) return MOE_ERR_UNSUPPORTED;
  if (m->n % 8 || m->n > MOE_FP4_MAX_N || m->rows > MOE_FP4_MAX_ROWS) return MOE_ERR_UNSUPPORTED;
  if (m->rows == 0) return MOE_OK;
  const int size = dtype == MOE_F32 ? 4 : 2;
  if (!m->codes || !m->scales || !dst || misaligned(m->codes) || misaligned(m->scales) || misaligned(dst) || row_stride < m->n ||
      (row_stride * size) % 16)
    return MOE_ERR_INVALID_ARG;
  const Fp4Shape sh = fp4_shape(m->rows, m->n);
  const dim3 grid = row_grid(m->rows, m->n), block(kQWarps * 32);
  const auto* c = (const unsigned char*)m->codes;
  const auto* sc = (const uint32_t*)m->scales;
  if (dtype == MOE_F32)
    MOE_CUDA_TRY(launch_pdl(fp4_dequantize_kernel<float>, grid, block, 0, (cudaStream_t)stream, c, sc, (long long)m->rows, m->n,
                            (float*)dst, (long long)row_stride, sh));
  else
    MOE_CUDA_TRY(launch_pdl(fp4_dequantize_kernel<__nv_bfloat16>, grid, block, 0, (cudaStream_t)stream, c, sc, (long long)m->rows, m->n,
                            (__nv_bfloat16*)dst, (long long)row_stride, sh));
  return MOE_OK;
}

int moe_fp4_pack_dense(int32_t d_model, int32_t d_ff, int32_t n_experts, const void* w_gate, const void* w_up, const void* w_down,
                       const moe_fp4* gu, const moe_fp4* down, void* stream) {
  if (d_model <= 0 || d_ff <= 0 || n_experts <= 0 || !w_gate || !w_up || !w_down || !gu || !down) return MOE_ERR_INVALID_ARG;
  if (d_model % 8 || d_ff % 8 || n_experts > MOE_MAX_EXPERTS || d_model > 16384 || d_ff > 65536) return MOE_ERR_UNSUPPORTED;
  const long long fb = (d_ff + 31) / 32, d = d_model, f = d_ff;
  if (gu->n != d_model || gu->rows != n_experts * fb * 64 || down->n != d_ff || down->rows != n_experts * d) return MOE_ERR_INVALID_ARG;
  if (!gu->codes || !gu->scales || !down->codes || !down->scales || misaligned(gu->codes) || misaligned(gu->scales) ||
      misaligned(down->codes) || misaligned(down->scales) || (((uintptr_t)w_gate | (uintptr_t)w_up | (uintptr_t)w_down) & 1u))
    return MOE_ERR_INVALID_ARG;
  cudaStream_t s = (cudaStream_t)stream;
  size_t cb, sb;
  MOE_TRY(moe_fp4_bytes(gu->rows, gu->n, &cb, &sb));
  if (d_ff % 32) {  // rows behind the last hidden unit
    MOE_CUDA_TRY(cudaMemsetAsync(const_cast<void*>(gu->codes), 0, cb, s));
    MOE_CUDA_TRY(cudaMemsetAsync(const_cast<void*>(gu->scales), 0, sb, s));
  }
  const Fp4Shape a = fp4_shape(gu->rows, gu->n), b = fp4_shape(down->rows, down->n);
  for (int e = 0; e < n_experts; ++e) {
    for (int u = 0; u < 2; ++u)  // w[:, c] of [d][f]
      MOE_TRY(launch_fp4_quantize(Fp4Source{(const __nv_bfloat16*)(u ? w_up : w_gate) + e * d * f, MOE_BF16, 1, f, f, nullptr, 1}, f, d_model,
                                  (char*)gu->codes + e * fb * 64 * a.pitch, (char*)gu->scales + e * fb * 64 * 4, a.rp, u, s));
    MOE_TRY(launch_fp4_quantize(Fp4Source{(const __nv_bfloat16*)w_down + e * f * d, MOE_BF16, 1, d, d, nullptr, 1}, d, d_ff,
                                (char*)down->codes + e * d * b.pitch, (char*)down->scales + e * d * 4, b.rp, -1, s));
  }
  return MOE_OK;
}

}  // extern "C"
