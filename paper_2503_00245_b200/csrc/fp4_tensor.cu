// Many rows times experts' MXFP4 matrices on the 5th-generation tensor cores (tcgen05.mma kind::mxf4, block scales):
//
//     C[m, n] = sum_k A[m, k] W_e[n, k]       for the rows m of expert e
//
// and, in the first product of an FFN, silu(gate) * up of neighbouring columns, quantised to MXFP4 again: the hidden rows leave the
// chip in 17/32 byte a value.
//
// A pair of CTAs (cta_group::2) computes tiles of 256 rows x bn <= 192 columns: each CTA stages its 128 rows of A and half of the
// tile's rows of W, 256 values (128 bytes, one swizzle row) of each at a time, and the words of scales (128 values each, csrc/fp4.cuh)
// of its own rows and of ALL the tile's columns.  Warps carry the words from shared to tensor memory, where the instruction wants
// them: word c of lane l is row 32 c + l's, the same in all four quarters of the lanes.  Tensor memory: two accumulators of 192
// columns, so that a tile's epilogue runs under the next one's MMAs, and five stages of scales in the 128 columns left.  (bn = 256
// would leave room for one accumulator.)
// (4096 rows x 2048 x 5632 to bf16: 31 us.  Scales fetched by those warps straight from memory, three stages ahead: 50; by one set of
// four warps instead of two in turn: 36.)
// Roles in each CTA:
//   warp 0      TMA producer: codes of A and W, both CTAs' on the leader's (rank 0) stage barrier; scales, on the CTA's own
//   warp 1      allocates tensor memory; in the leader one lane issues the MMAs of both CTAs
//   warps 2-9   scales, shared -> tensor memory (a warp for each quarter of the lanes, two sets that take the stages in turn)
//   warps 10-17 epilogue
// Tiles are handed out statically.  A tile may read rows of the next expert, or zeros; they are never stored.  All waits are
// bounded; one that expires sets the ctx's status word.  No copy here is multicast.
#include "fp4.cuh"
#include "tcgen.cuh"

namespace cosmoe {

namespace {

constexpr int kStages4 = 6;
constexpr int kKB = 256;           // values per stage: 128 bytes of codes
constexpr int kMaxBn = 192;
constexpr int kScaleWarps = 4, kScaleSets = 2;
constexpr int kThreads4 = (2 + kScaleSets * kScaleWarps + kEpiWarps) * 32;
constexpr int kPairRows4 = 2 * kBM;
// A tile's first row is any; a copy starts on 16 bytes, four words of scales: up to three rows before the first come along.
constexpr int kScaleRowsA = kBM + 4;
constexpr uint32_t kABytes4 = kBM * 128, kWBytes4 = kMaxBn / 2 * 128;
constexpr uint32_t kSABytes4 = 2 * kScaleRowsA * 4, kSAOff4 = kABytes4 + kWBytes4, kSWOff4 = kSAOff4 + (kSABytes4 + 127) / 128 * 128;
constexpr uint32_t kStageBytes4 = (kSWOff4 + 2 * kMaxBn * 4 + 1023) / 1024 * 1024;
constexpr int kScaleCol = 2 * kMaxBn;   // first column of the scales; a stage: A 4 + 4, W 8 + 8 columns
constexpr int kScaleCols = 24;
constexpr int kScaleSlots = 5;
// (a set of scale warps meets every stage of its ring places: it must not skip a phase of their barriers)
static_assert(kStages4 % kScaleSets == 0, "stages");
static_assert(kScaleCol + kScaleSlots * kScaleCols <= kTmemCols && kScaleSlots < kStages4, "tensor memory");
constexpr int kEpiBuf4 = 4096;

enum { EPI4_F32 = 0, EPI4_BF16 = 1, EPI4_HIDDEN = 2 };

struct Fp4Params {
  int n_rows;              // of A
  const int32_t* offsets;  // [E + 1]
  int E, N, K;
  int bn, epi;
  void* out;
  long long ld_out;
  unsigned char *h_codes, *h_scales;  // EPI4_HIDDEN
  Fp4Shape h;
  DeviceState* st;
};

struct Smem4 {
  uint64_t full[kStages4];       // leader's: the codes of the stage have landed in both CTAs
  uint64_t scales_in[kStages4];  // own: its words of scales have landed
  uint64_t scales_at[kStages4];  // leader's: both CTAs' scales are in tensor memory
  uint64_t empty[kStages4];      // own: the MMAs have finished with this CTA's stage
  uint64_t accum_full[2];        // own
  uint64_t accum_empty[2];       // leader's
  uint32_t tmem_base;
};

// Experts' rows and tiles over a warp's lanes (lane l: experts l and l + 32).
struct Tiles4 {
  int lo0, lo1, hi0, hi1, p0, p1, total;
};
__device__ __forceinline__ Tiles4 read_tiles(const Fp4Params& P, int lane) {
  Tiles4 m;
  const int e0 = min(lane, P.E), e1 = min(lane + 32, P.E);
  m.lo0 = max(P.offsets[e0], 0), m.hi0 = min(P.offsets[min(e0 + 1, P.E)], P.n_rows);
  m.lo1 = max(P.offsets[e1], 0), m.hi1 = min(P.offsets[min(e1 + 1, P.E)], P.n_rows);
  m.p0 = (max(m.hi0 - m.lo0, 0) + kPairRows4 - 1) / kPairRows4;
  m.p1 = (max(m.hi1 - m.lo1, 0) + kPairRows4 - 1) / kPairRows4;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v0 = __shfl_up_sync(0xffffffffu, m.p0, o), v1 = __shfl_up_sync(0xffffffffu, m.p1, o);
    if (lane >= o) m.p0 += v0, m.p1 += v1;
  }
  m.p1 += __shfl_sync(0xffffffffu, m.p0, 31);
  m.total = __shfl_sync(0xffffffffu, m.p1, 31);
  return m;
}
struct Tile4 {
  int e, m0, m_end, n0;
};
__device__ __forceinline__ Tile4 tile_at(const Fp4Params& P, const Tiles4& m, int idx, int n_tiles) {
  Tile4 t;
  const int mt = idx / n_tiles;
  t.n0 = (idx - mt * n_tiles) * P.bn;
  const int e = __popc(__ballot_sync(0xffffffffu, m.p0 <= mt)) + __popc(__ballot_sync(0xffffffffu, m.p1 <= mt));
  const int before0 = __shfl_sync(0xffffffffu, m.p0, (e - 1) & 31), before1 = __shfl_sync(0xffffffffu, m.p1, (e - 1) & 31);
  const int lo0 = __shfl_sync(0xffffffffu, m.lo0, e & 31), lo1 = __shfl_sync(0xffffffffu, m.lo1, e & 31);
  const int hi0 = __shfl_sync(0xffffffffu, m.hi0, e & 31), hi1 = __shfl_sync(0xffffffffu, m.hi1, e & 31);
  const int before = e == 0 ? 0 : e <= 32 ? before0 : before1;
  t.e = e;
  t.m0 = (e < 32 ? lo0 : lo1) + (mt - before) * kPairRows4;
  t.m_end = e < 32 ? hi0 : hi1;
  return t;
}

// Instruction descriptor: E2M1 x E2M1 with E8M0 scales -> fp32, M = 256 over the pair, N = n, both operands K-major; `id`: which
// half of a word of scales (0 or 2) the instruction's 64 values take.
__device__ __forceinline__ uint32_t instr_desc_mxf4(int n, uint32_t id) {
  uint32_t d = 0;
  d |= id << 4;    // scales of B
  d |= 1u << 7;    // A: E2M1
  d |= 1u << 10;   // B: E2M1
  d |= (uint32_t)(n >> 3) << 17;
  d |= 1u << 23;   // scales: E8M0
  d |= (uint32_t)(kPairRows4 >> 4) << 24;
  d |= id << 29;   // scales of A
  return d;
}
__device__ __forceinline__ void tc_mma_mxf4(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sa, uint32_t sb,
                                            uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d_tmem),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sa), "r"(sb), "r"(acc)
      : "memory");
}
__device__ __forceinline__ void tc_st4(uint32_t taddr, const uint32_t* v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3])
               : "memory");
}
__device__ __forceinline__ void tc_st2(uint32_t taddr, const uint32_t* v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x2.b32 [%0], {%1, %2};" ::"r"(taddr), "r"(v[0]), "r"(v[1]) : "memory");
}
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__global__ void __launch_bounds__(kThreads4, 1)
    fp4_tensor_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_w,
                      const __grid_constant__ CUtensorMap map_sa, const __grid_constant__ CUtensorMap map_sw, const Fp4Params P) {
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* stages = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  unsigned char* const epi_bufs = stages + (size_t)kStages4 * kStageBytes4;
  Smem4& sm = *reinterpret_cast<Smem4*>(epi_bufs + kEpiWarps * kEpiBuf4);
  const int tid = threadIdx.x, lane = tid & 31, warp = lane0(tid >> 5);
  const int num_kb = (P.K + kKB - 1) / kKB;
  const int n_tiles = (P.N + P.bn - 1) / P.bn;
  const uint32_t rank = (uint32_t)lane0((int)cluster_ctarank());
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;

  if (tid == 0) {
    for (int i = 0; i < kStages4; ++i) {
      mbar_init(&sm.full[i], 1);
      mbar_init(&sm.scales_in[i], 1);
      mbar_init(&sm.scales_at[i], 2 * kScaleWarps);
      mbar_init(&sm.empty[i], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&sm.accum_full[b], 1);
      mbar_init(&sm.accum_empty[b], 2 * kEpiWarps);
    }
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_w) : "memory");
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm.tmem_base)), "n"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  __syncwarp();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem = (uint32_t)lane0((int)sm.tmem_base);
  pdl_wait();
  pdl_launch_dependents();
  const Tiles4 tm = read_tiles(P, lane);
  const int n_work = tm.total * n_tiles;

  if (warp == 0) {
    // ================================================================= TMA producer (both CTAs)
    int it = 0;
    uint32_t slot = 0, par = 1;
    bool ok = true;
    const uint32_t tx_pair = 2u * (kABytes4 + (uint32_t)P.bn / 2u * 128u);
    const uint32_t full0 = (uint32_t)lane0((int)map_to_rank(&sm.full[0], 0u));
    const uint32_t own0 = (uint32_t)lane0((int)map_to_rank(&sm.scales_in[0], rank));
    const uint32_t st0 = (uint32_t)lane0((int)smem_u32(stages));
    for (int idx = pair; ok && idx < n_work; idx += n_pairs) {
      const Tile4 t = tile_at(P, tm, idx, n_tiles);
      const int a_row = t.m0 + (int)rank * kBM, w_row = t.e * P.N + t.n0 + (int)rank * (P.bn / 2);
      for (int kb = 0; kb < num_kb; ++kb, ++it) {
        if (it >= kStages4 && !mbar_wait_warp(&sm.empty[slot], par)) {
          if (lane == 0) flag_error(P.st, MOE_ERR_TIMEOUT, 0x600u);
          ok = false;
          break;
        }
        const uint32_t st_a = st0 + slot * kStageBytes4, bar = full0 + 8u * slot, own = own0 + 8u * slot;
        if (elect_one()) {
          mbar_arrive_expect_tx(&sm.scales_in[slot], kSABytes4 + (uint32_t)P.bn * 8u);
          tma_load_2d(st_a + kSAOff4, &map_sa, a_row & ~3, 2 * kb, own);
          tma_load_2d(st_a + kSWOff4, &map_sw, t.e * P.N + t.n0, 2 * kb, own);
          if (rank == 0) mbar_arrive_expect_tx(&sm.full[slot], tx_pair);
          tma_load_2d(st_a, &map_a, kb * 128, a_row, bar);
          tma_load_2d(st_a + kABytes4, &map_w, kb * 128, w_row, bar);
        }
        __syncwarp();
        if (++slot == (uint32_t)kStages4) slot = 0, par ^= 1u;
      }
    }
    if (!ok) {  // copies in flight must land before the pair goes away
      for (int j = max(0, it - kStages4); j < it; ++j) {
        (void)mbar_wait(&sm.scales_in[j % kStages4], (j / kStages4) & 1);
        if (rank == 0) (void)mbar_wait(&sm.full[j % kStages4], (j / kStages4) & 1);
      }
    }
  } else if (warp == 1) {
    // ================================================================= MMA issuer (leader only)
    if (rank == 0) {
      const uint32_t id0 = instr_desc_mxf4(P.bn, 0u), id2 = instr_desc_mxf4(P.bn, 2u);
      const uint64_t hi_k = smem_desc(0, 16, 1024) & 0xffffffff00000000ull;
      const uint32_t stage0 = (uint32_t)lane0((int)(smem_u32(stages) >> 4));
      uint32_t slot = 0, par = 0, st_lo = stage0, sc_slot = 0;
      int tile_i = 0;
      bool ok = true;
      for (int idx = pair; ok && idx < n_work; idx += n_pairs, ++tile_i) {
        const int buf = tile_i & 1;
        if (tile_i >= 2) {
          if (!mbar_wait_warp(&sm.accum_empty[buf], ((tile_i >> 1) - 1) & 1)) {
            if (lane == 0) flag_error(P.st, MOE_ERR_TIMEOUT, 0x603u);
            break;
          }
          tc_fence_after();
        }
        const uint32_t d_tmem = tmem + (uint32_t)(buf * kMaxBn);
        for (int kb = 0; kb < num_kb; ++kb) {
          if (!mbar_wait_warp(&sm.full[slot], par) || !mbar_wait_warp(&sm.scales_at[slot], par)) {
            if (lane == 0) flag_error(P.st, MOE_ERR_TIMEOUT, 0x601u);
            ok = false;
            break;
          }
          tc_fence_after();
          const uint64_t da = hi_k | (uint64_t)(st_lo | (1u << 16));
          const uint64_t db = hi_k | (uint64_t)((st_lo + (kABytes4 >> 4)) | (1u << 16));
          const uint32_t sc = tmem + (uint32_t)kScaleCol + sc_slot * (uint32_t)kScaleCols;
          const int steps = min(4, (P.K - kb * kKB + 63) / 64);
          if (elect_one()) {
#pragma unroll
            for (uint32_t kk = 0; kk < 4; ++kk)
              if ((int)kk < steps)
                tc_mma_mxf4(d_tmem, da + 2u * kk, db + 2u * kk, (kk & 1) ? id2 : id0, sc + 4u * (kk >> 1), sc + 8u + 8u * (kk >> 1),
                            (uint32_t)kb | kk);
            tc_commit_pair(&sm.empty[slot]);
            if (kb + 1 == num_kb) tc_commit_pair(&sm.accum_full[buf]);
          }
          __syncwarp();
          st_lo += kStageBytes4 >> 4;
          if (++sc_slot == (uint32_t)kScaleSlots) sc_slot = 0;
          if (++slot == (uint32_t)kStages4) slot = 0, par ^= 1u, st_lo = stage0;
        }
      }
    }
  } else if (warp < 2 + kScaleSets * kScaleWarps) {
    // ================================================================= scales (both CTAs)
    const uint32_t quarter = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + (uint32_t)kScaleCol;
    const uint32_t at0 = (uint32_t)lane0((int)map_to_rank(&sm.scales_at[0], 0u));
    uint32_t slot = 0, par = 0, sc_slot = 0;
    const int set = (warp - 2) / kScaleWarps;
    int it = 0, e_slot = 0, e_par = 0;  // (the stage whose MMAs must be done with the tensor memory written next)
    bool ok = true;
    for (int idx = pair; ok && idx < n_work; idx += n_pairs) {
      const Tile4 t = tile_at(P, tm, idx, n_tiles);
      const int skip = (t.m0 + (int)rank * kBM) & 3;
      for (int kb = 0; kb < num_kb; ++kb, ++it) {
        const uint32_t this_slot = slot, this_par = par, this_sc = sc_slot, this_e = e_slot, this_epar = e_par;
        if (++sc_slot == (uint32_t)kScaleSlots) sc_slot = 0;
        if (++slot == (uint32_t)kStages4) slot = 0, par ^= 1u;
        if (it >= kScaleSlots && ++e_slot == kStages4) e_slot = 0, e_par ^= 1;
        if (it % kScaleSets != set) continue;
        if (!mbar_wait_warp(&sm.scales_in[this_slot], this_par)) {
          if (lane == 0) flag_error(P.st, MOE_ERR_TIMEOUT, 0x605u);
          ok = false;
          break;
        }
        const uint32_t* sa = reinterpret_cast<const uint32_t*>(stages + this_slot * kStageBytes4 + kSAOff4) + skip + lane;
        const uint32_t* sw = reinterpret_cast<const uint32_t*>(stages + this_slot * kStageBytes4 + kSWOff4) + lane;
        uint32_t v[2][10];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int c = 0; c < 4; ++c) v[h][c] = sa[h * kScaleRowsA + 32 * c];
#pragma unroll
          for (int c = 0; c < 6; ++c) v[h][4 + c] = 32 * c < P.bn ? sw[h * P.bn + 32 * c] : 0u;
        }
        if (it >= kScaleSlots) {
          if (!mbar_wait_warp(&sm.empty[this_e], this_epar)) {
            if (lane == 0) flag_error(P.st, MOE_ERR_TIMEOUT, 0x604u);
            ok = false;
            break;
          }
          tc_fence_after();
        }
        const uint32_t at = quarter + this_sc * (uint32_t)kScaleCols;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          tc_st4(at + 4u * h, v[h]);
          tc_st4(at + 8u + 8u * h, v[h] + 4);
          tc_st2(at + 12u + 8u * h, v[h] + 8);
        }
        tc_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(at0 + 8u * this_slot);
      }
    }
  } else {
    // ================================================================= epilogue (warps 10..17, both CTAs)
    const int ew = warp - (2 + kScaleSets * kScaleWarps);
    const int q = warp & 3;
    const uint32_t acce_bar[2] = {map_to_rank(&sm.accum_empty[0], 0u), map_to_rank(&sm.accum_empty[1], 0u)};
    unsigned char* const ebuf = epi_bufs + ew * kEpiBuf4;
    int tile_i = 0;
    for (int idx = pair; idx < n_work; idx += n_pairs, ++tile_i) {
      const Tile4 t = tile_at(P, tm, idx, n_tiles);
      const int buf = tile_i & 1;
      const int cpar = (ew >> 2) ^ (tile_i & 1);
      if (!mbar_wait_warp(&sm.accum_full[buf], (tile_i >> 1) & 1)) {
        if (lane == 0) flag_error(P.st, MOE_ERR_TIMEOUT, 0x602u);
        break;
      }
      tc_fence_after();
      const int ncols = min(P.bn, P.N - t.n0);
      const int row = t.m0 + (int)rank * kBM + 32 * q + lane;
      const int rows = t.m_end - (row - lane);
      const uint32_t tbase = tmem + ((uint32_t)(32 * q) << 16) + (uint32_t)(buf * kMaxBn);
      if (rows > 0) {
        if (P.epi == EPI4_HIDDEN) {
          for (int c = 64 * cpar; c < ncols; c += 128) {  // (N is a multiple of 64)
            uint32_t g[32], u[32];
            tc_ld32(tbase + c, g);
            tc_ld32(tbase + c + 32, u);
            tc_wait_ld(g, u);
            float h[32];
            uint32_t top = 0u;
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              h[j] = silu_mul(__uint_as_float(g[j]), __uint_as_float(u[j]));
              top = max(top, __float_as_uint(h[j]) & 0x7fffffffu);
            }
            const uint32_t s = fp4_scale_byte(top);
            const float up = fp4_up(s);
            const int blk = (t.n0 + c) >> 6;
            if (lane < rows) {
              *reinterpret_cast<uint4*>(P.h_codes + (long long)row * P.h.pitch + blk * 16) =
                  make_uint4(fp4_pack8(h, up), fp4_pack8(h + 8, up), fp4_pack8(h + 16, up), fp4_pack8(h + 24, up));
              unsigned char* const sc = P.h_scales + ((long long)(blk >> 2) * P.h.rp + row) * 4;
              sc[blk & 3] = (unsigned char)s;
              if (blk == P.h.nb - 1)
                for (int z = (blk & 3) + 1; z < 4; ++z) sc[z] = 0;
            }
          }
        } else {
          for (int c = 64 * cpar; c < ncols; c += 128) {
            uint32_t a[2][32];
            tc_ld32(tbase + c, a[0]);
            tc_ld32(tbase + c + 32, a[1]);
            tc_wait_ld(a[0], a[1]);
            if (P.epi == EPI4_F32) {
              float* const o = (float*)P.out + (long long)(row - lane) * P.ld_out + t.n0 + c;
              store_rows128(ebuf, lane, a[0], o, P.ld_out * 4, rows, (ncols - c) / 4);
              store_rows128(ebuf, lane, a[1], o + 32, P.ld_out * 4, rows, (ncols - c) / 4 - 8);
            } else {
              uint32_t o[32];
#pragma unroll
              for (int j = 0; j < 32; ++j)
                o[j] = pack_bf16x2(__uint_as_float(a[j >> 4][2 * (j & 15)]), __uint_as_float(a[j >> 4][2 * (j & 15) + 1]));
              store_rows128(ebuf, lane, o, (__nv_bfloat16*)P.out + (long long)(row - lane) * P.ld_out + t.n0 + c, P.ld_out * 2, rows,
                            (ncols - c) / 8);
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(acce_bar[buf]);
    }
  }
  // ---- teardown: neither CTA leaves while the other may still count on its barriers or read its operands
  tc_fence_before();
  __syncthreads();
  __syncwarp();
  cluster_sync_all();
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kTmemCols) : "memory");
}

// rows of codes: box of 128 bytes x box_rows
int make_map_codes(CUtensorMap* m, const void* base, long long rows, long long pitch, int box_rows) {
  const cuuint64_t dims[2] = {(cuuint64_t)pitch, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)pitch};
  const cuuint32_t box[2] = {128, (cuuint32_t)box_rows};
  const cuuint32_t es[2] = {1, 1};
  const CUresult r = encode_tiled(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, base, dims, strides, box, es, CU_TENSOR_MAP_SWIZZLE_128B,
                                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
  return r == CUDA_SUCCESS ? MOE_OK : MOE_ERR_CUDA;
}

// Columns of a tile, a multiple of `step`: as many as fit, or fewer where that saves an eighth of the rounds of tiles over the pairs,
// a round costing about 96 columns more than it has (operands, barriers, the epilogue's tail).  Rows make as many tiles as even
// routing gives, the last one of each expert half full.  8 experts of d 2048, f 5632, 192 against 128 columns in the down product:
// 64 tokens 49.1 against 48.0 us, 512 tokens 54.0 against 52.2, 2048 tokens 96.5 against 102.4.
int pick_bn4(long long rows, int E, int N, int pairs, int step) {
  const long long m_tiles = std::max<long long>((rows + kPairRows4 - 1) / kPairRows4 + E / 2, std::min<long long>(E, rows));
  int best = kMaxBn;
  long long least = 0;
  for (int bn = kMaxBn; bn >= 64; bn -= step) {
    const long long cost = (m_tiles * ((N + bn - 1) / bn) + pairs - 1) / pairs * (bn + 96);
    if (bn == kMaxBn || 8 * cost <= 7 * least) least = cost, best = bn;
  }
  return best;
}

// words of scales [chunks][rp]: box of box_rows words x 2
int make_map_scales(CUtensorMap* m, const void* base, const Fp4Shape& sh, int box_rows) {
  const cuuint64_t dims[2] = {(cuuint64_t)sh.rp, (cuuint64_t)sh.chunks};
  const cuuint64_t strides[1] = {(cuuint64_t)sh.rp * 4};
  const cuuint32_t box[2] = {(cuuint32_t)box_rows, 2};
  const cuuint32_t es[2] = {1, 1};
  const CUresult r = encode_tiled(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, base, dims, strides, box, es, CU_TENSOR_MAP_SWIZZLE_NONE,
                                  CU_TENSOR_MAP_L2_PROMOTION_L2_128B);
  return r == CUDA_SUCCESS ? MOE_OK : MOE_ERR_CUDA;
}

}  // namespace

// out_f32: 1 fp32, 0 bf16; h (not null): hidden rows instead of `out`.
int launch_fp4_tensor(moe_ctx* ctx, const moe_fp4* a, const moe_fp4* w, const int32_t* offsets, int E, void* out, int out_f32,
                      long long out_stride, const moe_fp4* h, cudaStream_t s) {
  Fp4Params P{};
  const Fp4Shape sa = fp4_shape(a->rows, a->n), sw = fp4_shape(w->rows, w->n);
  P.n_rows = (int)a->rows, P.offsets = offsets, P.E = E, P.N = (int)(w->rows / E), P.K = a->n;
  P.out = out, P.ld_out = out_stride, P.epi = h ? EPI4_HIDDEN : out_f32 ? EPI4_F32 : EPI4_BF16;
  if (h) P.h_codes = (unsigned char*)h->codes, P.h_scales = (unsigned char*)h->scales, P.h = fp4_shape(h->rows, h->n);
  P.st = ctx->d_state;
  P.bn = pick_bn4(a->rows, E, P.N, ctx->sm_count / 2, h ? 64 : 32);
  CUtensorMap ma, mw, msa, msw;
  MOE_TRY(make_map_codes(&ma, a->codes, a->rows, sa.pitch, kBM));
  MOE_TRY(make_map_codes(&mw, w->codes, w->rows, sw.pitch, P.bn / 2));
  MOE_TRY(make_map_scales(&msa, a->scales, sa, kScaleRowsA));
  MOE_TRY(make_map_scales(&msw, w->scales, sw, P.bn));
  const size_t smem = (size_t)kStages4 * kStageBytes4 + kEpiWarps * kEpiBuf4 + sizeof(Smem4) + 1024 + 128;
  if ((long long)smem > ctx->max_smem_optin) return MOE_ERR_UNSUPPORTED;
  MOE_TRY(allow_full_smem<fp4_tensor_kernel>(ctx));
  const long long m_tiles = (a->rows + kPairRows4 - 1) / kPairRows4 + E;  // upper bound
  const int n_tiles = (P.N + P.bn - 1) / P.bn;
  const int pairs = (int)std::min<long long>(m_tiles * n_tiles, max_pairs<fp4_tensor_kernel>(ctx, kThreads4, smem));
  cudaLaunchConfig_t lc;
  cudaLaunchAttribute attr[2];
  pair_launch_config(lc, attr, 2 * pairs, kThreads4, smem, s);
  MOE_CUDA_TRY(cudaLaunchKernelEx(&lc, fp4_tensor_kernel, ma, mw, msa, msw, P));
  ctx->launches++;
  return MOE_OK;
}

}  // namespace cosmoe
