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

__device__ __forceinline__ void load8(const float* p, float* f) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
  f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float* f) { unpack8(__ldg(reinterpret_cast<const uint4*>(p)), f); }
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
template <typename T>
__device__ __forceinline__ void quantize_step(const float (&f)[8], int c, long long i, int n, int lane, unsigned char* codes, uint32_t* scales,
                                              const Fp4Shape& sh) {
  uint32_t top = 0u;  // (as bits: a NaN is larger than everything)
#pragma unroll
  for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(f[j]) & 0x7fffffffu);
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  const uint32_t s = fp4_scale_byte(top);
  if (c < 32 * sh.nb) *reinterpret_cast<uint32_t*>(codes + i * sh.pitch + c / 2) = fp4_pack8(f, fp4_up(s));
  // a word of scales: four blocks, sixteen lanes
  uint32_t w = c < 32 * sh.nb ? s << (8 * ((lane >> 2) & 3)) : 0u;
  w |= __shfl_xor_sync(0xffffffffu, w, 4);
  w |= __shfl_xor_sync(0xffffffffu, w, 8);
  if ((lane & 15) == 0 && c < n) scales[(long long)(c >> 7) * sh.rp + i] = w;
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
      float f[kFly][8];
#pragma unroll
      for (int u = 0; u < kFly; ++u) {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[u][j] = 0.f;
        if (r >= 0 && c0 + 256 * u < n) load8(row + c0 + 256 * u, f[u]);
      }
#pragma unroll
      for (int u = 0; u < kFly; ++u)
        if (c0 - lane * 8 + 256 * u < n) quantize_step<T>(f[u], c0 + 256 * u, i, n, lane, codes, scales, sh);
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

__device__ __forceinline__ void store8(float* p, const float* f) {
  reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float* f) {
  *reinterpret_cast<uint4*>(p) =
      make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
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
        const float s = fp4_scales2((sw[u] >> (8 * ((c >> 5) & 3))) & 0xffu).x;
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = fp4_value((w[u] >> (4 * j)) & 15u) * s;  // (a value and a power of two: exact in either type)
        store8(dst + i * row_stride + c, f);
      }
    }
  }
}
// Blocks along the rows, and warps to share a row.
dim3 row_grid(long long rows, int n) {
  const long long x = std::min<long long>((rows + kQWarps - 1) / kQWarps, 148 * 8);
  const int most = (n + 256 * kFly - 1) / (256 * kFly);
  return dim3((unsigned)x, (unsigned)std::max(1, (int)std::min<long long>(most, 148 * 4 / x)));
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

bool misaligned(const void* p) { return ((uintptr_t)p & 15u) != 0; }

}  // namespace

int launch_fp4_quantize(const Fp4Source& src, long long rows, int n, void* codes, void* scales, long long rp, int split, cudaStream_t s) {
  if (rows <= 0) return MOE_OK;
  return src.dtype == MOE_F32 ? quantize_t<float>(src, rows, n, codes, scales, rp, split, s)
                              : quantize_t<__nv_bfloat16>(src, rows, n, codes, scales, rp, split, s);
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
  if ((uintptr_t)src % (dtype == MOE_F32 ? 4 : 2)) return MOE_ERR_INVALID_ARG;
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
      misaligned(down->codes) || misaligned(down->scales))
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
