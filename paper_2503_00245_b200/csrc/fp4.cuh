// MXFP4 matrices: blocks of 32 values of a row share a power of two, the values are 4-bit floats.
//
// Element format E2M1 (1 sign, 2 exponent bits with bias 1, 1 mantissa bit): 0, .5, 1, 1.5, 2, 3, 4, 6 and their negatives.
// Scale format E8M0: byte s stands for 2^(s - 127), 255 for NaN.
//
//   codes   [rows][pitch] bytes, pitch = 16 ceil(n / 32): value i of a row in byte i / 2, even i in the low four bits
//   scales  [ceil(n / 128)][rows rounded up to 4] words of four bytes: byte b & 3 of word [b >> 2][r] scales block b of row r
//
// A word of scales belongs to one row and 128 values: what the tensor cores take for two instructions, and neighbouring rows'
// words are neighbours, so a warp's load is one line and needs no rearrangement on its way to tensor memory.
#pragma once

#include "common.cuh"

namespace cosmoe {

struct Fp4Shape {
  int nb, chunks;        // blocks of 32 and groups of 128 values in a row, rounded up
  long long pitch, rp;   // bytes of a row's codes; rows as the scales count them
};
inline __host__ __device__ Fp4Shape fp4_shape(long long rows, int n) {
  Fp4Shape s;
  s.nb = (n + 31) / 32, s.chunks = (s.nb + 3) / 4;
  s.pitch = 16ll * s.nb, s.rp = (rows + 3) / 4 * 4;
  return s;
}

#ifdef __CUDACC__

// Scale byte of a block from the bits of its largest magnitude: the exponent of the largest power of two not above it, less that
// of 4 (the largest power of two among the codes), 255 when the block holds an infinity or a NaN.
__device__ __forceinline__ uint32_t fp4_scale_byte(uint32_t amax_bits) {
  const uint32_t e = amax_bits >> 23;
  return e >= 255u ? 255u : e > 2u ? e - 2u : 0u;
}
// What the values are multiplied with: 2^(127 - s), exact.  (0 for NaN blocks, whose codes are zeros.)
__device__ __forceinline__ float fp4_up(uint32_t s) { return s == 255u ? 0.f : __uint_as_float((254u - s) << 23); }
// Two codes in a byte, `lo` in the low bits: nearest, ties to the even code, saturating at 6.
__device__ __forceinline__ uint32_t fp4_pack2(float lo, float hi) {
  uint32_t r;
  asm("{\n\t.reg .b8 b;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %1, %2;\n\tcvt.u32.u8 %0, b;\n\t}" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t fp4_pack8(const float* v, float up) {
  // (inf * 0 of a NaN block would be NaN, whose code is unspecified: such a block's codes are zeros)
  return up == 0.f ? 0u
                   : fp4_pack2(v[0] * up, v[1] * up) | fp4_pack2(v[2] * up, v[3] * up) << 8 |
                         fp4_pack2(v[4] * up, v[5] * up) << 16 | fp4_pack2(v[6] * up, v[7] * up) << 24;
}
// 2^(s - 127) of a scale byte, twice, in bf16 (0: 2^-127; 255: NaN).
__device__ __forceinline__ uint32_t fp4_scale_bf16x2(uint32_t s) {
  uint32_t r;
  asm("{\n\t.reg .b16 h;\n\tcvt.u16.u32 h, %1;\n\tcvt.rn.bf16x2.ue8m0x2 %0, h;\n\t}" : "=r"(r) : "r"(s | s << 8));
  return r;
}
// Eight codes' values as bf16 pairs, in order: the bytes of a magnitude's bf16 are looked up by byte permutes (a selector takes three
// bits of a code), its sign is the top bit of a byte of the word or of the word shifted by four.
__device__ __forceinline__ void fp4_bf16(uint32_t w, uint32_t (&out)[4]) {
  const uint32_t up = w << 4;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t sel = (h ? w >> 16 : w) & 0x7777u;
    const uint32_t hi = __byte_perm(0x3f3f3f00u, 0x40404040u, sel), lo = __byte_perm(0xc0800000u, 0xc0804000u, sel);
    const uint32_t top = hi | (__byte_perm(up, w, h ? 0xfbeau : 0xd9c8u) & 0x80808080u);
    out[2 * h] = __byte_perm(lo, top, 0x5140), out[2 * h + 1] = __byte_perm(lo, top, 0x7362);
  }
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

#endif  // __CUDACC__

// csrc/fp4_store.cu
// Source of a quantisation: values at row_of[i] / row_div (or i) * row_stride + column * col_stride.
struct Fp4Source {
  const void* base;
  int dtype;
  long long row_stride, col_stride, rows;  // strides in values
  const int32_t* row_of;
  int row_div;
};
// Destination rows: i, or, with `split` 0 or 1, row i of a matrix whose blocks of 32 rows alternate with another's.
int launch_fp4_quantize(const Fp4Source& src, long long rows, int n, void* codes, void* scales, long long rp, int split, cudaStream_t s);
// Rows of x quantised and placed by expert (offsets, and each pair's slot in inv).
int launch_fp4_place(moe_ctx* ctx, const void* x, const int32_t* idx, int T, int32_t* offsets, int32_t* inv, void* codes, void* scales,
                     cudaStream_t s);

// csrc/fp4_few.cu: few rows (decode)
constexpr int kFewSplits = 4;  // parts of the down product's contraction, at most
bool fp4_few_applies(const moe_ctx* ctx, int K, int n);  // (n: rows of an expert, at most, without an expert named twice by a token)
int launch_fp4_few_rows(moe_ctx* ctx, const moe_fp4* a, const moe_fp4* w, const int32_t* offsets, int E, void* out, int out_f32,
                        long long out_stride, cudaStream_t s);
int launch_fp4_few_experts(moe_ctx* ctx, const void* x, int T, const moe_fp4* gu, const moe_fp4* down, const int32_t* idx, const float* wt,
                           void* y, const moe_fp4* h, float* part, unsigned* arrived, cudaStream_t s);
// csrc/fp4_tensor.cu: many rows.  out_f32: 1 fp32, 0 bf16; h (not null): hidden rows of MXFP4 instead of `out`.
int launch_fp4_tensor(moe_ctx* ctx, const moe_fp4* a, const moe_fp4* w, const int32_t* offsets, int E, void* out, int out_f32,
                      long long out_stride, const moe_fp4* h, cudaStream_t s);

}  // namespace cosmoe
