// Few rows times MXFP4 matrices (decode): the matrices are read once, from HBM, and everything else stays on chip.
//
// A warp takes 16 rows of a matrix and 128 values of them at a time ("segment"): lane (g, t) = (lane / 4, lane % 4) holds block t
// (32 values, 16 bytes) of rows g and g + 8, straight from memory.  Codes become E4M3 bytes by three shifts and masks
// (csrc/fp4.cuh) and go to mma.sync m16n8k32: 8 tokens would be its columns, but the four lanes of a row hold four BLOCKS, whose
// sums must be scaled apart.  So a column is a (token, block) pair: column 4 q + j has the values of token q in the places of lane
// j's values and zeros elsewhere.  Four such MMAs (eight values of each block at a time) leave one sum per row, token and block,
// exact (multiples of 1/4 below 2^11, times 2^-12), in one register; it is multiplied with the two blocks' scales and added in fp32.  N = two tokens
// is far below a tcgen05 tile; what counts here is the number of instructions per byte of weights.
// Per 2048 values of a matrix: 56 instructions to widen them, 4 MMAs and 16 multiply-adds per pair of tokens.
//
// The tokens' codes lie widened in shared memory, [segment][token][block][4 words][even, odd], so that a lane's share of an MMA
// is one 8-byte read.
#include <algorithm>

#include "fp4.cuh"
#include "tcgen.cuh"

namespace cosmoe {
namespace {

constexpr int kSWarps = 8;
constexpr int kSRows = 128;          // rows of a call that go this way, at most
constexpr int kSegTok = 128 + 16;    // bytes of a token's segment in shared memory: codes and four scales
constexpr int kSmemTokens = 96 * 1024;

__device__ __forceinline__ void mma_e4m3(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// read once: past L1
__device__ __forceinline__ uint4 ld_stream(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// Tokens of a group in shared memory.
struct Tokens {
  uint32_t* codes;  // [segments][m][32]
  float* scales;    // [segments][m][4]
  int m;            // tokens, even
};
__device__ __forceinline__ void put_block(const Tokens& k, int seg, int tok, int b, uint4 w, float scale) {
  uint32_t* d = k.codes + ((seg * k.m + tok) * 4 + b) * 8;
  reinterpret_cast<uint4*>(d)[0] = make_uint4(fp4_even_e4m3(w.x), fp4_odd_e4m3(w.x), fp4_even_e4m3(w.y), fp4_odd_e4m3(w.y));
  reinterpret_cast<uint4*>(d)[1] = make_uint4(fp4_even_e4m3(w.z), fp4_odd_e4m3(w.z), fp4_even_e4m3(w.w), fp4_odd_e4m3(w.w));
  k.scales[(seg * k.m + tok) * 4 + b] = scale;
}

struct Matrix {
  const unsigned char* codes;
  const uint32_t* scales;
  Fp4Shape sh;
  int N;  // rows of an expert
};

// acc[p][h] += rows g + 8 h of the tile times token 2 p + t / 2, blocks 2 (t & 1) and the next of segments seg, seg + step, ...
// (times 2^-12; the lanes t and t ^ 1 hold the halves of a sum)
template <int PAIRS>
__device__ __forceinline__ void tile_segments(const Matrix& W, long long row0, int rows, const Tokens& k, int seg, int step, int lane,
                                              float (&acc)[PAIRS][2]) {
  constexpr int U = PAIRS <= 2 ? 4 : 2;
  const int g = lane >> 2, t = lane & 3;
  const long long ra = row0 + min(g, rows - 1), rb = row0 + min(g + 8, rows - 1);
  const unsigned char* pa = W.codes + ra * W.sh.pitch + t * 16;
  const unsigned char* pb = W.codes + rb * W.sh.pitch + t * 16;
  const bool mine = (g & 3) == t;
  for (; seg < W.sh.chunks; seg += U * step) {
    uint4 wa[U], wb[U];
    uint32_t sa[U], sb[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = seg + u * step;
      const bool in = 4 * s + t < W.sh.nb;
      wa[u] = wb[u] = make_uint4(0u, 0u, 0u, 0u);
      sa[u] = sb[u] = 0u;
      if (in) wa[u] = ld_stream(pa + s * 64), wb[u] = ld_stream(pb + s * 64);
      if (s < W.sh.chunks) sa[u] = __ldg(W.scales + s * W.sh.rp + ra), sb[u] = __ldg(W.scales + s * W.sh.rp + rb);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = seg + u * step;
      if (s >= W.sh.chunks) break;
      const uint32_t* a = reinterpret_cast<const uint32_t*>(&wa[u]);
      const uint32_t* b = reinterpret_cast<const uint32_t*>(&wb[u]);
      uint32_t ae[4], ao[4], be[4], bo[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        ae[i] = fp4_even_e4m3(a[i]), ao[i] = fp4_odd_e4m3(a[i]), be[i] = fp4_even_e4m3(b[i]), bo[i] = fp4_odd_e4m3(b[i]);
      const float2 fa = fp4_scales2((sa[u] >> (16 * (t & 1))) & 0xffffu), fb = fp4_scales2((sb[u] >> (16 * (t & 1))) & 0xffffu);
#pragma unroll
      for (int p = 0; p < PAIRS; ++p) {
        uint4 x0 = make_uint4(0u, 0u, 0u, 0u), x1 = x0;
        if (mine) {
          const uint4* x = reinterpret_cast<const uint4*>(k.codes + ((s * k.m + 2 * p + (g >> 2)) * 4 + t) * 8);
          x0 = x[0], x1 = x[1];
        }
        float c[4] = {0.f, 0.f, 0.f, 0.f};
        mma_e4m3(c, ae[0], be[0], ao[0], bo[0], x0.x, x0.y);
        mma_e4m3(c, ae[1], be[1], ao[1], bo[1], x0.z, x0.w);
        mma_e4m3(c, ae[2], be[2], ao[2], bo[2], x1.x, x1.y);
        mma_e4m3(c, ae[3], be[3], ao[3], bo[3], x1.z, x1.w);
        const float2 f = *reinterpret_cast<const float2*>(k.scales + (s * k.m + 2 * p + (t >> 1)) * 4 + 2 * (t & 1));
        acc[p][0] += c[0] * fa.x * f.x + c[1] * fa.y * f.y;
        acc[p][1] += c[2] * fb.x * f.x + c[3] * fb.y * f.y;
      }
    }
  }
}

// One warp's share of a tile, into out[row][m]
template <int PAIRS>
__device__ __forceinline__ void tile_to_smem(const Matrix& W, long long row0, int rows, const Tokens& k, int seg, int step, int lane,
                                             float* out) {
  float acc[PAIRS][2];
#pragma unroll
  for (int p = 0; p < PAIRS; ++p) acc[p][0] = acc[p][1] = 0.f;
  tile_segments<PAIRS>(W, row0, rows, k, seg, step, lane, acc);
  const int g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int p = 0; p < PAIRS; ++p)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float v = acc[p][h] + __shfl_xor_sync(0xffffffffu, acc[p][h], 1);
      if ((t & 1) == 0) out[(g + 8 * h) * k.m + 2 * p + (t >> 1)] = v * 4096.f;
    }
}
__device__ __forceinline__ void tile_to_smem_any(const Matrix& W, long long row0, int rows, const Tokens& k, int seg, int step, int lane,
                                                 float* out) {
  if (k.m <= 2) tile_to_smem<1>(W, row0, rows, k, seg, step, lane, out);
  else if (k.m <= 4) tile_to_smem<2>(W, row0, rows, k, seg, step, lane, out);
  else if (k.m <= 8) tile_to_smem<4>(W, row0, rows, k, seg, step, lane, out);
  else tile_to_smem<8>(W, row0, rows, k, seg, step, lane, out);
}

// Which expert this CTA works for, and its rows.  By warp 0; `which` counts the experts that have rows.
struct Group {
  int e, n;
  int rows[kSRows];
};
__device__ __forceinline__ void find_group(Group& grp, const int32_t* idx, const int32_t* offsets, int n, int E, int which, int lane,
                                           DeviceState* st) {
  const unsigned FULL = 0xffffffffu;
  int pe[kSRows / 32];
#pragma unroll
  for (int i = 0; i < kSRows / 32; ++i) pe[i] = -1;
  unsigned m0, m1;
  if (idx) {
    unsigned a = 0u, b = 0u;
#pragma unroll
    for (int i = 0; i < kSRows / 32; ++i) {
      const int p = lane + 32 * i;
      if (p >= n) continue;
      const int e = idx[p];
      if (e < 0 || e >= E) {
        flag_error(st, MOE_ERR_STATE, 0x500u);
        continue;
      }
      pe[i] = e;
      if (e < 32) a |= 1u << e;
      else b |= 1u << (e - 32);
    }
    m0 = __reduce_or_sync(FULL, a), m1 = __reduce_or_sync(FULL, b);
  } else {
    auto some = [&](int e) { return e < E && max(offsets[e], 0) < min(offsets[e + 1], n); };
    m0 = __ballot_sync(FULL, some(lane)), m1 = __ballot_sync(FULL, some(lane + 32));
  }
  const unsigned long long mask = (unsigned long long)m1 << 32 | m0;
  int e = -1;
  if (which < __popcll(mask)) {
    unsigned long long rest = mask;
    for (int i = 0; i < which; ++i) rest &= rest - 1;
    e = __ffsll((long long)rest) - 1;
  }
  int count = 0;
  if (e >= 0) {
    if (idx) {
#pragma unroll
      for (int i = 0; i < kSRows / 32; ++i) {
        const unsigned is = __ballot_sync(FULL, pe[i] == e);
        if (pe[i] == e) grp.rows[count + __popc(is & ((1u << lane) - 1u))] = lane + 32 * i;
        count += __popc(is);
      }
    } else {
      const int lo = max(offsets[e], 0);
      count = min(min(offsets[e + 1], n) - lo, kSRows);
      for (int i = lane; i < count; i += 32) grp.rows[i] = lo + i;
    }
  }
  if (lane == 0) grp.e = e, grp.n = count;
}

// ---------------------------------------------------------------- rows already in MXFP4
struct RowsParams {
  const unsigned char* a_codes;
  const uint32_t* a_scales;
  Fp4Shape a;
  Matrix w;
  const int32_t *idx, *offsets;  // one of the two
  int n, E, tiles, m_max;
  void* out;
  long long out_stride;
  DeviceState* st;
};

// CTA = 16 rows of an expert's matrix; the warps share out the contraction and add up in shared memory, in order.
template <typename OT>
__global__ void __launch_bounds__(kSWarps * 32, 2) fp4_rows_kernel(const RowsParams P) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ Group grp;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  pdl_launch_dependents();
  const int which = blockIdx.x / P.tiles, tile = blockIdx.x - which * P.tiles;
  if (warp == 0) find_group(grp, P.idx, P.offsets, P.n, P.E, which, lane, P.st);
  __syncthreads();
  if (grp.e < 0) return;
  const int segs = P.w.sh.chunks;
  const long long row0 = (long long)grp.e * P.w.N + tile * 16;
  const int rows = min(16, P.w.N - tile * 16);
  for (int g0 = 0; g0 < grp.n; g0 += P.m_max) {
    const int have = min(P.m_max, grp.n - g0);
    Tokens k;
    k.m = have <= 2 ? 2 : have <= 4 ? 4 : have <= 8 ? 8 : 16;
    k.codes = reinterpret_cast<uint32_t*>(smem);
    k.scales = reinterpret_cast<float*>(smem + (size_t)segs * k.m * 128);
    float* const part = reinterpret_cast<float*>(smem + (size_t)segs * P.m_max * kSegTok);
    for (int i = tid; i < segs * k.m * 4; i += kSWarps * 32) {
      const int b = i & 3, st = i >> 2, tok = st % k.m, seg = st / k.m;
      uint4 w = make_uint4(0u, 0u, 0u, 0u);
      float sc = 0.f;
      if (tok < have && 4 * seg + b < P.a.nb) {
        const long long r = grp.rows[g0 + tok];
        w = __ldcg(reinterpret_cast<const uint4*>(P.a_codes + r * P.a.pitch + (4 * seg + b) * 16));
        sc = fp4_scales2((__ldcg(P.a_scales + seg * P.a.rp + r) >> (8 * b)) & 0xffu).x;
      }
      put_block(k, seg, tok, b, w, sc);
    }
    __syncthreads();
    tile_to_smem_any(P.w, row0, rows, k, warp, kSWarps, lane, part + warp * 16 * k.m);
    __syncthreads();
    for (int i = tid; i < 16 * have; i += kSWarps * 32) {
      const int r = i & 15, tok = i >> 4;
      if (r >= rows) continue;
      float v = part[r * k.m + tok];
#pragma unroll
      for (int w = 1; w < kSWarps; ++w) v += part[(w * 16 + r) * k.m + tok];
      OT* const o = (OT*)P.out + grp.rows[g0 + tok] * P.out_stride + tile * 16 + r;
      if constexpr (sizeof(OT) == 4) *o = v;
      else *o = __float2bfloat16_rn(v);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------- gate and up products of few tokens, SiLU, hidden rows in MXFP4
struct GuParams {
  const void* x;
  int x_f32, d, f, k;
  Matrix w;
  const int32_t* idx;
  int n, E, fb, m_max;
  unsigned char* h_codes;
  unsigned char* h_scales;
  Fp4Shape h;
  DeviceState* st;
};

// CTA = 32 hidden units of an expert: their 32 gate and 32 up rows are four tiles, two warps each (halves of the contraction).
// The hidden units are one block of the next product's rows.
template <typename XT>
__global__ void __launch_bounds__(kSWarps * 32, 2) fp4_gu_kernel(const GuParams P) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ Group grp;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  pdl_launch_dependents();
  const int which = blockIdx.x / P.fb, blk = blockIdx.x - which * P.fb;
  if (warp == 0) find_group(grp, P.idx, nullptr, P.n, P.E, which, lane, P.st);
  __syncthreads();
  if (grp.e < 0) return;
  const int segs = P.w.sh.chunks;
  const long long row0 = (long long)grp.e * P.w.N + blk * 64;
  for (int g0 = 0; g0 < grp.n; g0 += P.m_max) {
    const int have = min(P.m_max, grp.n - g0);
    Tokens k;
    k.m = have <= 2 ? 2 : have <= 4 ? 4 : have <= 8 ? 8 : 16;
    k.codes = reinterpret_cast<uint32_t*>(smem);
    k.scales = reinterpret_cast<float*>(smem + (size_t)segs * k.m * 128);
    float* const part = reinterpret_cast<float*>(smem + (size_t)segs * P.m_max * kSegTok);
    // rows of x to MXFP4: four lanes per block
    for (int i = tid; i < (segs * k.m * 4) * 4; i += kSWarps * 32) {
      const int q = i & 3, b = (i >> 2) & 3, st = i >> 4, tok = st % k.m, seg = st / k.m;
      const int c = seg * 128 + b * 32 + q * 8;
      float f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = 0.f;
      if (tok < have && c < P.d) {
        const XT* src = (const XT*)P.x + (long long)(grp.rows[g0 + tok] / P.k) * P.d + c;
        if constexpr (sizeof(XT) == 4) {
          const float4 u = __ldcg(reinterpret_cast<const float4*>(src)), v = __ldcg(reinterpret_cast<const float4*>(src) + 1);
          f[0] = u.x, f[1] = u.y, f[2] = u.z, f[3] = u.w, f[4] = v.x, f[5] = v.y, f[6] = v.z, f[7] = v.w;
        } else {
          unpack8(__ldcg(reinterpret_cast<const uint4*>(src)), f);
        }
      }
      uint32_t top = 0u;
#pragma unroll
      for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(f[j]) & 0x7fffffffu);
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const uint32_t s = fp4_scale_byte(top), w = fp4_pack8(f, fp4_up(s));
      uint32_t* dst = k.codes + ((seg * k.m + tok) * 4 + b) * 8 + q * 2;
      dst[0] = fp4_even_e4m3(w), dst[1] = fp4_odd_e4m3(w);
      if (q == 0) k.scales[(seg * k.m + tok) * 4 + b] = fp4_scales2(s).x;
    }
    __syncthreads();
    tile_to_smem_any(P.w, row0 + (warp & 3) * 16, 16, k, warp >> 2, 2, lane, part + warp * 16 * k.m);
    __syncthreads();
    for (int tok = warp; tok < have; tok += kSWarps) {
      const int i = lane * k.m + tok, half = 64 * k.m;
      const float g = part[i] + part[half + i], u = part[32 * k.m + i] + part[half + 32 * k.m + i];
      const float h = silu_mul(g, u);
      const uint32_t s = fp4_scale_byte(__reduce_max_sync(0xffffffffu, __float_as_uint(h) & 0x7fffffffu));
      const float up = fp4_up(s), next = __shfl_down_sync(0xffffffffu, h, 1);
      const long long r = grp.rows[g0 + tok];
      if ((lane & 1) == 0) P.h_codes[r * P.h.pitch + blk * 16 + lane / 2] = up == 0.f ? 0 : (unsigned char)fp4_pack2(h * up, next * up);
      unsigned char* const sc = P.h_scales + ((long long)(blk >> 2) * P.h.rp + r) * 4;
      if (lane == 0) sc[blk & 3] = (unsigned char)s;
      if (blk == P.fb - 1 && lane > (blk & 3) && lane < 4) sc[lane] = 0;
    }
    __syncthreads();
  }
}

// y[t] = sum_j w[t][j] o[t k + j]
template <typename YT>
__global__ void __launch_bounds__(256) fp4_sum_kernel(const float* __restrict__ o, const float* __restrict__ w, int T, int k, int d,
                                                      YT* __restrict__ y) {
  pdl_wait();
  pdl_launch_dependents();
  const int i = blockIdx.x * 256 + threadIdx.x, quads = d / 4;
  if (i >= T * quads) return;
  const int t = i / quads, q = i - t * quads;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int j = 0; j < k; ++j) {
    const float4 v = __ldcg(reinterpret_cast<const float4*>(o) + (long long)(t * k + j) * quads + q);
    const float s = __ldcg(w + t * k + j);
    a.x += s * v.x, a.y += s * v.y, a.z += s * v.z, a.w += s * v.w;
  }
  if constexpr (sizeof(YT) == 4) {
    reinterpret_cast<float4*>(y)[i] = a;
  } else {
    reinterpret_cast<uint2*>(y)[i] = make_uint2(pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w));
  }
}

// tokens of a group: as many as fit, 16 at most
int group_size(int chunks, int n) {
  int m = 16;
  while (m > 2 && ((long long)chunks * m * kSegTok > kSmemTokens || m >= 2 * n)) m /= 2;
  return m;
}

}  // namespace

int launch_fp4_rows(moe_ctx* ctx, const moe_fp4* a, const moe_fp4* w, const int32_t* idx, const int32_t* offsets, int E, void* out,
                    int out_f32, long long out_stride, cudaStream_t s) {
  RowsParams P{};
  P.a_codes = (const unsigned char*)a->codes, P.a_scales = (const uint32_t*)a->scales, P.a = fp4_shape(a->rows, a->n);
  P.w = Matrix{(const unsigned char*)w->codes, (const uint32_t*)w->scales, fp4_shape(w->rows, w->n), (int)(w->rows / E)};
  P.idx = idx, P.offsets = offsets, P.n = (int)a->rows, P.E = E, P.tiles = (P.w.N + 15) / 16;
  P.m_max = group_size(P.w.sh.chunks, P.n);
  P.out = out, P.out_stride = out_stride, P.st = ctx->d_state;
  const size_t smem = (size_t)P.w.sh.chunks * P.m_max * kSegTok + (size_t)kSWarps * 16 * P.m_max * 4;
  if ((long long)smem > ctx->max_smem_optin - (long long)sizeof(Group)) return MOE_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)(P.tiles * std::min(E, P.n))), block(kSWarps * 32);
  if (out_f32) {
    MOE_TRY(allow_full_smem<fp4_rows_kernel<float>>(ctx));
    MOE_CUDA_TRY(launch_pdl(fp4_rows_kernel<float>, grid, block, smem, s, P));
  } else {
    MOE_TRY(allow_full_smem<fp4_rows_kernel<__nv_bfloat16>>(ctx));
    MOE_CUDA_TRY(launch_pdl(fp4_rows_kernel<__nv_bfloat16>, grid, block, smem, s, P));
  }
  ctx->launches++;
  return MOE_OK;
}

int launch_fp4_few(moe_ctx* ctx, const void* x, int T, const moe_fp4* gu, const moe_fp4* down, const int32_t* idx, const float* wt, void* y,
                   const moe_fp4* h, float* out_slots, cudaStream_t s) {
  const moe_config& c = ctx->cfg;
  const int E = c.n_experts, n = T * c.top_k;
  GuParams P{};
  P.x = x, P.d = c.d_model, P.f = c.d_ff, P.k = c.top_k;
  P.w = Matrix{(const unsigned char*)gu->codes, (const uint32_t*)gu->scales, fp4_shape(gu->rows, gu->n), (int)(gu->rows / E)};
  P.idx = idx, P.n = n, P.E = E, P.fb = (c.d_ff + 31) / 32, P.m_max = group_size(P.w.sh.chunks, n);
  P.h_codes = (unsigned char*)h->codes, P.h_scales = (unsigned char*)h->scales, P.h = fp4_shape(h->rows, h->n), P.st = ctx->d_state;
  const size_t smem = (size_t)P.w.sh.chunks * P.m_max * kSegTok + (size_t)kSWarps * 16 * P.m_max * 4;
  const dim3 grid((unsigned)(P.fb * std::min(E, n))), block(kSWarps * 32);
  if (c.x_dtype == MOE_F32) {
    MOE_TRY(allow_full_smem<fp4_gu_kernel<float>>(ctx));
    MOE_CUDA_TRY(launch_pdl(fp4_gu_kernel<float>, grid, block, smem, s, P));
  } else {
    MOE_TRY(allow_full_smem<fp4_gu_kernel<__nv_bfloat16>>(ctx));
    MOE_CUDA_TRY(launch_pdl(fp4_gu_kernel<__nv_bfloat16>, grid, block, smem, s, P));
  }
  ctx->launches++;
  MOE_TRY(launch_fp4_rows(ctx, h, down, idx, nullptr, E, out_slots, 1, c.d_model, s));
  const dim3 sgrid((T * (c.d_model / 4) + 255) / 256);
  if (c.x_dtype == MOE_F32)
    MOE_CUDA_TRY(launch_pdl(fp4_sum_kernel<float>, sgrid, dim3(256), 0, s, (const float*)out_slots, wt, T, c.top_k, c.d_model, (float*)y));
  else
    MOE_CUDA_TRY(launch_pdl(fp4_sum_kernel<__nv_bfloat16>, sgrid, dim3(256), 0, s, (const float*)out_slots, wt, T, c.top_k, c.d_model,
                            (__nv_bfloat16*)y));
  ctx->launches++;
  return MOE_OK;
}

}  // namespace cosmoe
