// Few rows times experts' MXFP4 matrices (decode), on the 5th-generation tensor cores: the matrices are read once, from HBM, and no
// other instruction touches their codes.
//
// What bounds it is latency in front of and behind the stream of bytes, and HBM between.  A CTA (one per SM) belongs to one expert and
// takes blocks of 64 of its rows, 512 values at a time ("stage": two swizzled tiles of 64 x 128 bytes and their words of scales, three
// copies), through a ring of four stages or more, beside the tokens' codes.  Both fit into half of an SM's shared memory up to 8 tokens
// at K = 5632 (four stages: 10 MB under way on 148 SMs) and 16 at K = 2048 (four; five up to 8 tokens), so that the down product's
// CTAs start beside the gate and up product's and have their first stages in place when the hidden rows are: 20 us a layer (one
// token, d 2048, f 5632), 21 where each CTA takes all of an SM and none starts early.  Longer rows of more tokens take all of it
// (8 tokens 41 us, 9 tokens 51).
// The rows are the M side of tcgen05.mma kind::mxf4 (M = 128: the lower half of an instruction's rows is whatever lies behind the block
// and is not looked at; an instruction costs its operands' 4 KB of shared-memory reads either way), the tokens N = 16 or 32 columns,
// whose codes are laid out in shared memory, swizzled.  Both operands' scales go from shared to tensor memory beside the MMAs (two sets of four warps, a stage each in
// turn).  One token, d 2048, f 5632, two of eight experts: 20 us a layer; the stream itself runs at 5.5 TB/s.
//   warp 0       copies (the ring's first fill: a stage for each warp)
//   warp 1       tensor memory, MMAs
//   warps 2-9    scales                     warps 12-13  epilogue (TMEM lanes 0-31 and 32-63)
// Most of this code runs once or twice a launch, so it is short rather than unrolled: fetching instructions that were never run costs
// more than running them (an epilogue unrolled over the tokens: 2 us a block with one token).
// (The same products on mma.sync, tiles through the same ring, codes widened to E4M3 in registers: 25 us a layer for one token at d 2048,
// f 5632, two experts; without its MMAs, whose legacy form is slow here, 19; without any arithmetic 14.)
//
// Modes: HIDDEN  gate and up rows -> silu(g) u -> rows of MXFP4 for the next product
//        OUT     rows of fp32 or bf16
//        DOWN    parts of rows; who brings a 64-column block's last part sums the block over parts, experts and the routing's weights
#include <algorithm>

#include "fp4.cuh"
#include "tcgen.cuh"

namespace cosmoe {
namespace {

constexpr int kFewThreads = 14 * 32;
constexpr int kFewRows = 128;      // pairs of a call that come this way, at most
constexpr int kBlkRows = 64;
constexpr int kStageK = 512;
constexpr uint32_t kHalfBytes = kBlkRows * 128, kWordBytes = 4 * kBlkRows * 4, kFewStage = 2 * kHalfBytes + kWordBytes;
constexpr int kFewStages = 12, kFewSlots = 6;
// tensor memory: two accumulators of 32 columns, scales of six stages, matrix and tokens (four columns for 128 values each)
constexpr int kSlotCol = 64, kSlotCols = 32, kFewTmem = 256;
static_assert(kSlotCol + kFewSlots * kSlotCols <= kFewTmem, "tensor memory");
constexpr int kSets = 2;
constexpr int kFewLast = 256;  // (d_model is at most 16384)

enum { FEW_HIDDEN = 0, FEW_OUT = 1, FEW_DOWN = 2 };

struct FewParams {
  const unsigned char* a_codes;  // the rows, in MXFP4 ...
  const uint32_t* a_scales;
  Fp4Shape a;
  const void* x;  // ... or (HIDDEN) in x_dtype: row p is x[p / k]
  int x_f32, k;
  int K;
  Fp4Shape w;
  int N;                         // rows of an expert's matrix
  const int32_t *idx, *offsets;  // one of the two: whose rows are whose
  int n, E;
  int units, splits, stages, m;  // blocks of an expert; parts of the contraction; ring; columns of an MMA
  int tok_rows;                  // rows of tokens in shared memory: m, or 8 where 16 columns show the same eight twice
  int part_stages;               // of the contraction's parts (the last one may be shorter)
  void* out;
  long long out_stride;
  int out_f32;
  unsigned char *h_codes, *h_scales;
  Fp4Shape h;
  const unsigned char* next_codes;  // the next product's matrix, to be brought into L2 (null: not)
  const uint32_t* next_scales;
  Fp4Shape next;
  int next_N;
  float* part;        // DOWN: [splits][n][N]
  unsigned* arrived;  // DOWN: parts of each block that have been stored; HIDDEN leaves zeros
  const float* wt;
  void* y;
  int y_f32, T;
  DeviceState* st;
};

struct FewSmem {
  uint64_t full[kFewStages], scales_at[kFewStages], empty[kFewStages], acc_full[2], acc_empty[2];
  uint32_t tmem_base;
  int e, cnt, rank, ctas, expected, n_last;
  int rows[kFewRows];
  int last_unit[kFewLast];  // DOWN: blocks whose last part came from here
};

// (Read once: first to leave L2, so that what the next product will read stays there.)
__device__ __forceinline__ void few_load(uint32_t dst, const CUtensorMap* map, int c0, int c1, uint64_t* bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3}], [%4], %5;" ::
          "r"(dst),
      "l"(map), "r"(c0), "r"(c1), "r"(smem_u32(bar)), "l"(policy)
      : "memory");
}
__device__ __forceinline__ void few_commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void few_mma(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d_tmem),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sa), "r"(sb), "r"(acc)
      : "memory");
}
// E2M1 x E2M1 with E8M0 scales -> fp32, M = 128, N = n, K-major; `id`: half of a word of scales (0 or 2)
__device__ __forceinline__ uint32_t few_idesc(int n, uint32_t id) {
  return id << 4 | 1u << 7 | 1u << 10 | (uint32_t)(n >> 3) << 17 | 1u << 23 | (128u >> 4) << 24 | id << 29;
}
__device__ __forceinline__ void few_st4(uint32_t taddr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void few_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// the two epilogue warps; both of them go on, or neither does
__device__ __forceinline__ void epilogue_meet() { asm volatile("bar.sync 1, 64;" ::: "memory"); }
__device__ __forceinline__ bool epilogue_all(bool ok) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
      "bar.red.and.pred q, 1, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"((uint32_t)ok)
      : "memory");
  return r != 0;
}

// Whose rows this CTA takes, by warp 0: the CTAs are dealt out to the experts that have rows.
template <int MODE>
__device__ __forceinline__ void few_find(const FewParams& P, FewSmem& sm, int lane) {
  const unsigned FULL = 0xffffffffu;
  int pe[kFewRows / 32];
  unsigned m0 = 0u, m1 = 0u;
  if (MODE != FEW_OUT) {
#pragma unroll
    for (int i = 0; i < kFewRows / 32; ++i) {
      pe[i] = -1;
      if (32 * i >= P.n) break;  // (what follows is not even fetched for a few pairs)
      const int p = lane + 32 * i;
      int e = p < P.n ? P.idx[p] : -1;
      if (p < P.n && (e < 0 || e >= P.E)) {
        if (MODE == FEW_HIDDEN) flag_error(P.st, MOE_ERR_STATE, 0x500u);
        e = -1;
      }
      pe[i] = e;
      if (e >= 32) m1 |= 1u << (e - 32);
      else if (e >= 0) m0 |= 1u << e;
    }
    m0 = __reduce_or_sync(FULL, m0), m1 = __reduce_or_sync(FULL, m1);
  } else {
    auto some = [&](int e) { return e < P.E && max(P.offsets[e], 0) < min(P.offsets[e + 1], P.n); };
    m0 = __ballot_sync(FULL, some(lane)), m1 = __ballot_sync(FULL, some(lane + 32));
  }
  unsigned long long mask = (unsigned long long)m1 << 32 | m0;
  const int active = __popcll(mask), G = gridDim.x, c = blockIdx.x;
  int e = -1, rank = 0, ctas = 1, cnt = 0, expected = 0;
  if (active > 0) {
    const int a = c * active / G, first = (a * G + active - 1) / active;
    rank = c - first, ctas = ((a + 1) * G + active - 1) / active - first;
    unsigned long long rest = mask;
    for (int i = 0; i < a; ++i) rest &= rest - 1;
    e = __ffsll((long long)rest) - 1;
    if (MODE != FEW_OUT) {
      // (DOWN: every expert's, for the number of parts that a block of y has)
      for (unsigned long long r = MODE == FEW_DOWN ? mask : 1ull << e; r; r &= r - 1) {
        const int ee = __ffsll((long long)r) - 1;
        int have = 0;
#pragma unroll
        for (int i = 0; i < kFewRows / 32; ++i) {
          if (32 * i >= P.n) break;
          const unsigned is = __ballot_sync(FULL, pe[i] == ee);
          if (ee == e && pe[i] == ee) sm.rows[have + __popc(is & ((1u << lane) - 1u))] = lane + 32 * i;
          have += __popc(is);
        }
        if (ee == e) cnt = have;
        if (MODE == FEW_DOWN) expected += have <= P.tok_rows ? 1 : (have + P.tok_rows - 1) / P.tok_rows;
      }
    } else {
      const int lo = max(P.offsets[e], 0);
      cnt = min(min(P.offsets[e + 1], P.n) - lo, kFewRows);
      for (int i = lane; i < cnt; i += 32) sm.rows[i] = lo + i;
    }
  }
  if (lane == 0) sm.n_last = 0, sm.e = e, sm.cnt = cnt, sm.rank = rank, sm.ctas = ctas, sm.expected = expected * P.splits;
}

template <int MODE>
__global__ void __launch_bounds__(kFewThreads, 2)
    fp4_few_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_s, const FewParams P) {
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  __shared__ FewSmem sm;
  unsigned char* const stages = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const int tid = threadIdx.x, lane = tid & 31, warp = lane0(tid >> 5);
  const int NS = P.stages, slots = min(NS, kFewSlots);
  // tokens: codes [256 values][tok_rows][128 bytes], words of scales [chunk][tok_rows]; behind them the epilogue's accumulators,
  // [token][row], two blocks in turn
  const int chunks = P.w.chunks, steps = (chunks + 1) / 2;
  unsigned char* const toks = stages + (((size_t)NS * kFewStage + 1023) & ~(size_t)1023);
  uint32_t* const tok_scales = reinterpret_cast<uint32_t*>(toks + (size_t)steps * P.tok_rows * 128);
  float* const accs = reinterpret_cast<float*>(tok_scales + (size_t)chunks * P.tok_rows);

  if (tid == 0) {
    for (int i = 0; i < NS; ++i) mbar_init(&sm.full[i], 1), mbar_init(&sm.scales_at[i], 4), mbar_init(&sm.empty[i], 1);
    for (int b = 0; b < 2; ++b) mbar_init(&sm.acc_full[b], 1), mbar_init(&sm.acc_empty[b], 2);
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_w) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_s) : "memory");
    fence_mbar_init();
    fence_proxy_async_smem();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm.tmem_base)), "n"(kFewTmem) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // DOWN comes behind HIDDEN, which lets it start once it has itself waited for what was before: routing and matrix are there.
  if (MODE != FEW_DOWN) pdl_wait();
  if (warp == 0) few_find<MODE>(P, sm, lane);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (MODE != FEW_DOWN) pdl_launch_dependents();
  const uint32_t tmem = (uint32_t)lane0((int)sm.tmem_base);
  const int e = sm.e, cnt = sm.cnt, rank = sm.rank, ctas = sm.ctas;
  const int items = e >= 0 ? P.units * P.splits : 0;
  const int mine = rank < items ? (items - rank + ctas - 1) / ctas : 0;
  const int all_stages = (P.K + kStageK - 1) / kStageK;
  const int groups = mine > 0 ? (cnt + P.tok_rows - 1) / P.tok_rows : 0;
  auto item_of = [&](int i, int& unit, int& sp, int& s0, int& s1) {
    const int item = rank + i * ctas;
    unit = P.splits == 1 ? item : item / P.splits, sp = item - unit * P.splits;
    s0 = sp * P.part_stages, s1 = min(s0 + P.part_stages, all_stages);
  };
  const uint32_t st0 = smem_u32(stages);

  // ---- the tokens' codes and scales.  A warp takes 256 values of a token at a time; the next ones' loads are on their way meanwhile.
  // (The first of them go out in front of the matrix's copies: behind 25 MB of those they take 3 us.)
  int tok = 0, step = 0;  // (of 256 values)
  uint4 u = make_uint4(0u, 0u, 0u, 0u), v = u;
  uint32_t word = 0u, s_word = 0u;
  auto fetch = [&](int g0) {
    const int c = step * 256 + lane * 8;
    const int r = sm.rows[g0 + tok];
    if (MODE == FEW_HIDDEN) {
      const long long at = (long long)(r / P.k) * P.K + min(c, P.K - 8);
      if (P.x_f32) {
        u = __ldcg(reinterpret_cast<const uint4*>((const float*)P.x + at));
        v = __ldcg(reinterpret_cast<const uint4*>((const float*)P.x + at) + 1);
      } else {
        u = __ldcg(reinterpret_cast<const uint4*>((const __nv_bfloat16*)P.x + at));
      }
    } else {
      word = c < 32 * P.a.nb ? __ldcg(reinterpret_cast<const uint32_t*>(P.a_codes + r * P.a.pitch + (c >> 1))) : 0u;
      s_word = (lane & 15) == 0 && c < P.K ? __ldcg(P.a_scales + (c >> 7) * P.a.rp + r) : 0u;
    }
  };
  auto first_fetch = [&](int g0, int have) {
    tok = 0, step = warp;
    while (step >= steps && tok < have) step -= steps, ++tok;
    if (tok < have) fetch(g0);
  };
  if (MODE != FEW_DOWN && groups > 0) first_fetch(0, min(P.tok_rows, cnt));

  // ---- copies, in (group, item, stage) order.  The ring's first fill is a stage for each warp, all at once: what a single warp
  // does one after the other here takes a tenth of a microsecond a copy.
  const uint64_t once = l2_policy_evict_first();
  auto copy = [&](int b, int unit, int s) {  // by one lane
    const uint32_t at = st0 + (uint32_t)b * kFewStage;
    const int row = e * P.N + unit * kBlkRows;
    mbar_arrive_expect_tx(&sm.full[b], kFewStage);
    few_load(at, &map_w, s * 256, row, &sm.full[b], once);
    few_load(at + kHalfBytes, &map_w, s * 256 + 128, row, &sm.full[b], once);
    few_load(at + 2 * kHalfBytes, &map_s, row, 4 * s, &sm.full[b], once);
  };
  int c_i = 0, c_s = 0, c_it = 0;         // item and stage of the next copy, and its number
  int c_left = warp == 0 ? NS : warp;     // (stages to walk on to it)
  if (groups > 0) {
    auto walk = [&] {  // c_left stages on; stops behind the last item
      while (c_i < mine) {
        int unit, sp, s0, s1;
        item_of(c_i, unit, sp, s0, s1);
        if (c_left < s1 - s0) {
          c_s = s0 + c_left;
          return true;
        }
        c_left -= s1 - s0, ++c_i;
      }
      return false;
    };
    if (warp < NS) {
      int unit, sp, s0, s1;
      if (warp == 0) {
        item_of(0, unit, sp, s0, s1);
        if (elect_one()) copy(0, unit, s0);
        __syncwarp();
        c_it = walk() ? NS : NS - c_left;
      } else if (walk()) {
        item_of(c_i, unit, sp, s0, s1);
        if (elect_one()) copy(warp, unit, c_s);
        __syncwarp();
      }
    }
  }
  bool copies_ok = true;
  if (MODE == FEW_DOWN) {
    pdl_wait();
    pdl_launch_dependents();
  }
  if (MODE == FEW_HIDDEN && P.arrived && blockIdx.x == 0)
    for (int i = tid; i < (P.next_N + kBlkRows - 1) / kBlkRows; i += kFewThreads) P.arrived[i] = 0u;
  if (MODE == FEW_HIDDEN && P.next_codes && mine > 0 && warp == 12) {  // this CTA's share of the expert's next matrix
    const long long bytes = P.next_N * P.next.pitch, from = e * bytes;
    const long long lo = bytes * rank / ctas / 128 * 128, hi = rank + 1 == ctas ? bytes : bytes * (rank + 1) / ctas / 128 * 128;
    for (long long o = lo + lane * 4096; o < hi; o += 32 * 4096) prefetch_l2(P.next_codes + from + o, (uint32_t)min(4096ll, hi - o));
    for (int c = rank + lane * ctas; c < P.next.chunks; c += 32 * ctas)
      prefetch_l2(P.next_scales + c * P.next.rp + (long long)e * P.next_N, (uint32_t)P.next_N * 4u);
  }

  uint32_t slot = 0, par = 0, sc_slot = 0;          // MMA and scale warps: places in the rings
  int it = 0, e_slot = 0, e_par = 0, acc_i = 0;     // stages so far; the stage that frees the scale slot; accumulators so far
  bool ok = true;
  for (int g0 = 0, grp = 0; grp < groups; g0 += P.tok_rows, ++grp) {
    const int have = min(P.tok_rows, cnt - g0);
    // (four lanes to a block of 32; columns behind the last token stay as they are)
    {
      const int q = lane & 3, b = (lane >> 2) & 3;
      if (grp > 0 || MODE == FEW_DOWN) first_fetch(g0, have);
#pragma unroll 1
      while (tok < have) {
        const int my_tok = tok, my_step = step, c = step * 256 + lane * 8;
        const uint4 mu = u, mv = v;
        uint32_t w = word, sc = s_word;
        step += kFewThreads / 32;
        while (step >= steps && tok < have) step -= steps, ++tok;
        if (tok < have) fetch(g0);
        if (MODE == FEW_HIDDEN) {
          float f[8];
          if (P.x_f32) {
            const float4 a = *reinterpret_cast<const float4*>(&mu), d = *reinterpret_cast<const float4*>(&mv);
            f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = d.x, f[5] = d.y, f[6] = d.z, f[7] = d.w;
          } else {
            unpack8(mu, f);
          }
          uint32_t top = 0u;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            if (c >= P.K) f[j] = 0.f;
            top = max(top, __float_as_uint(f[j]) & 0x7fffffffu);
          }
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
          const uint32_t byte = fp4_scale_byte(top);
          w = fp4_pack8(f, fp4_up(byte));
          sc = byte << (8 * b);
          sc |= __shfl_xor_sync(0xffffffffu, sc, 4);
          sc |= __shfl_xor_sync(0xffffffffu, sc, 8);
        }
        if (q + b == 0 && (c >> 7) < chunks) tok_scales[(c >> 7) * P.tok_rows + my_tok] = sc;
        *reinterpret_cast<uint32_t*>(toks + (size_t)my_step * (P.tok_rows * 128) + my_tok * 128 + (((lane >> 2) ^ (my_tok & 7)) << 4) + q * 4) = w;
      }
    }
    fence_proxy_async_smem();
    __syncthreads();

    if (warp == 0) {
      // ------------------------------------------------------------- copies
      int b = c_it % NS, round = c_it / NS;
      if (grp > 0) c_i = 0, c_s = -1;
      while (copies_ok && c_i < mine) {
        int unit, sp, s0, s1;
        item_of(c_i, unit, sp, s0, s1);
        if (c_s < 0) c_s = s0;
        for (; c_s < s1; ++c_s, ++c_it) {
          if (round > 0 && !mbar_wait_warp(&sm.empty[b], (round - 1) & 1)) {
            if (lane == 0) flag_error(P.st, MOE_ERR_TIMEOUT, 0x510u);
            copies_ok = false;
            break;
          }
          if (elect_one()) copy(b, unit, c_s);
          __syncwarp();
          if (++b == NS) b = 0, ++round;
        }
        ++c_i, c_s = -1;
      }
    } else if (warp == 1) {
      // ------------------------------------------------------------- MMAs
      const uint32_t id0 = few_idesc(P.m, 0u), id2 = few_idesc(P.m, 2u);
      const uint64_t hi_k = smem_desc(0, 16, 1024) & 0xffffffff00000000ull;
      // (eight rows of tokens: the second group of eight columns reads them again)
      const uint64_t hi_tok = smem_desc(0, 16, P.tok_rows == 8 ? 0 : 1024) & 0xffffffff00000000ull;
      const uint32_t tok_lo = (uint32_t)lane0((int)(smem_u32(toks) >> 4)), ring_lo = st0 >> 4;
      for (int i = 0; ok && i < mine; ++i, ++acc_i) {
        int unit, sp, s0, s1;
        item_of(i, unit, sp, s0, s1);
        const int buf = acc_i & 1;
        if (acc_i >= 2) {
          if (!mbar_wait_warp(&sm.acc_empty[buf], ((acc_i >> 1) - 1) & 1)) {
            if (lane == 0) flag_error(P.st, MOE_ERR_TIMEOUT, 0x511u);
            ok = false;
            break;
          }
          tc_fence_after();
        }
        for (int s = s0; s < s1; ++s) {
          if (!mbar_wait_warp(&sm.full[slot], par) || !mbar_wait_warp(&sm.scales_at[slot], par)) {
            if (lane == 0) flag_error(P.st, MOE_ERR_TIMEOUT, 0x512u);
            ok = false;
            break;
          }
          tc_fence_after();
          const int mmas = min(8, (P.K - s * kStageK + 63) / 64);
          const uint32_t a_lo = ring_lo + slot * (kFewStage >> 4), b_lo = tok_lo + (uint32_t)(2 * s) * (uint32_t)(P.tok_rows * 8);
          const uint32_t sa = tmem + (uint32_t)kSlotCol + (uint32_t)kSlotCols * sc_slot, sb = sa + 16u;
          if (elect_one()) {
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j)
              if ((int)j < mmas) {
                const uint64_t da = hi_k | (uint64_t)((a_lo + (j >> 2) * (kHalfBytes >> 4) + 2u * (j & 3u)) | (1u << 16));
                const uint64_t db = hi_tok | (uint64_t)((b_lo + (j >> 2) * (uint32_t)(P.tok_rows * 8) + 2u * (j & 3u)) | (1u << 16));
                few_mma(tmem + 32u * buf, da, db, (j & 1u) ? id2 : id0, sa + 4u * (j >> 1), sb + 4u * (j >> 1), (uint32_t)(s - s0) | j);
              }
            few_commit(&sm.empty[slot]);
            if (s + 1 == s1) few_commit(&sm.acc_full[buf]);
          }
          __syncwarp();
          if (++sc_slot == (uint32_t)slots) sc_slot = 0;
          if (++slot == (uint32_t)NS) slot = 0, par ^= 1u;
        }
      }
    } else if (warp < 10) {
      // ------------------------------------------------------------- scales of the matrix
      const int set = (warp - 2) >> 2;
      const uint32_t quarter = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + (uint32_t)kSlotCol;
      for (int i = 0; ok && i < mine; ++i) {
        int unit, sp, s0, s1;
        item_of(i, unit, sp, s0, s1);
        for (int s = s0; s < s1; ++s, ++it) {
          const uint32_t this_slot = slot, this_par = par, this_sc = sc_slot;
          const int this_e = e_slot, this_epar = e_par;
          if (++sc_slot == (uint32_t)slots) sc_slot = 0;
          if (++slot == (uint32_t)NS) slot = 0, par ^= 1u;
          if (it >= slots && ++e_slot == NS) e_slot = 0, e_par ^= 1;
          if (it % kSets != set) continue;
          // (First the stage whose place in tensor memory this one takes: a set sees every other stage only, and with that one done
          // the phase of `full` before this one's is over, without which the wait below would not wait.)
          if (it >= slots) {
            if (!mbar_wait_warp(&sm.empty[this_e], this_epar)) {
              if (lane == 0) flag_error(P.st, MOE_ERR_TIMEOUT, 0x514u);
              ok = false;
              break;
            }
            tc_fence_after();
          }
          if (!mbar_wait_warp(&sm.full[this_slot], this_par)) {
            if (lane == 0) flag_error(P.st, MOE_ERR_TIMEOUT, 0x513u);
            ok = false;
            break;
          }
          const uint32_t* w = reinterpret_cast<const uint32_t*>(stages + this_slot * kFewStage + 2 * kHalfBytes) + lane;
          uint32_t v[4][2];
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j][0] = w[j * kBlkRows], v[j][1] = w[j * kBlkRows + 32];
          uint32_t x[4];  // (of a token: lane = its column)
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] = lane < P.tok_rows && 4 * s + j < chunks ? tok_scales[(4 * s + j) * P.tok_rows + lane] : 0u;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            few_st4(quarter + (uint32_t)kSlotCols * this_sc + 4u * j, v[j][0], v[j][1], 0u, 0u);
            few_st4(quarter + (uint32_t)kSlotCols * this_sc + 16u + 4u * j, x[j], 0u, 0u, 0u);
          }
          few_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&sm.scales_at[this_slot]);
        }
      }
    } else if (warp >= 12) {
      // ------------------------------------------------------------- epilogue: lane = row 32 q + lane of the block
      const int q = warp - 12;
      for (int i = 0; ok && i < mine; ++i, ++acc_i) {
        int unit, sp, s0, s1;
        item_of(i, unit, sp, s0, s1);
        const int buf = acc_i & 1;
        if (!mbar_wait_warp(&sm.acc_full[buf], (acc_i >> 1) & 1)) {
          if (lane == 0) flag_error(P.st, MOE_ERR_TIMEOUT, 0x515u);
          ok = false;
        }
        ok = epilogue_all(ok);
        if (!ok) break;
        tc_fence_after();
        float(*const acc)[kBlkRows] = reinterpret_cast<float(*)[kBlkRows]>(accs + buf * P.m * kBlkRows);
#pragma unroll 1
        for (int c = 0; c < have; c += 16) {
          uint32_t v[16];
          tc_ld16(tmem + ((uint32_t)(32 * q) << 16) + 32u * buf + (uint32_t)c, v);
          tc_wait_ld16(v);
#pragma unroll
          for (int t = 0; t < 16; ++t) acc[c + t][32 * q + lane] = __uint_as_float(v[t]);
        }
        tc_fence_before();
        epilogue_meet();
        if (lane == 0) mbar_arrive(&sm.acc_empty[buf]);
        const int r = unit * kBlkRows + 32 * q + lane;
        if (MODE == FEW_HIDDEN) {
          // rows 0-31 are the gates of 32 hidden units, rows 32-63 their up values: a block of the next product's rows
#pragma unroll 1
          for (int t = q; t < have; t += 2) {
            const float h = silu_mul(acc[t][lane], acc[t][32 + lane]);
            const uint32_t s = fp4_scale_byte(__reduce_max_sync(0xffffffffu, __float_as_uint(h) & 0x7fffffffu));
            const float up = fp4_up(s), next = __shfl_down_sync(0xffffffffu, h, 1);
            const long long p = sm.rows[g0 + t];
            if ((lane & 1) == 0) P.h_codes[p * P.h.pitch + unit * 16 + lane / 2] = up == 0.f ? 0 : (unsigned char)fp4_pack2(h * up, next * up);
            unsigned char* const sc = P.h_scales + ((long long)(unit >> 2) * P.h.rp + p) * 4;
            if (lane == 0) sc[unit & 3] = (unsigned char)s;
            if (unit == P.units - 1 && lane > (unit & 3) && lane < 4) sc[lane] = 0;
          }
        } else if (r < P.N) {
#pragma unroll 1
          for (int t = 0; t < have; ++t) {
            const float v = acc[t][32 * q + lane];
            if (MODE == FEW_DOWN) P.part[((long long)sp * P.n + sm.rows[g0 + t]) * P.N + r] = v;
            else if (P.out_f32) ((float*)P.out)[sm.rows[g0 + t] * P.out_stride + r] = v;
            else ((__nv_bfloat16*)P.out)[sm.rows[g0 + t] * P.out_stride + r] = __float2bfloat16_rn(v);
          }
        }
        if (MODE == FEW_DOWN) {  // (released by one thread behind the barrier)
          epilogue_meet();
          if (warp == 12 && lane == 0 && atom_add_acq_rel(P.arrived + unit, 1u) == (unsigned)sm.expected - 1u) sm.last_unit[sm.n_last++] = unit;
        }
      }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
  }
  if (warp == 0 && !copies_ok)  // copies in flight land before the CTA goes away
    for (int j = max(0, c_it - NS); j < c_it; ++j) (void)mbar_wait(&sm.full[j % NS], (j / NS) & 1);
  if (MODE == FEW_DOWN && sm.n_last > 0) {  // (all parts of these blocks are there)
    __threadfence();
    const int planes = P.k * P.splits;
    for (int i = tid; i < sm.n_last * P.T * kBlkRows; i += kFewThreads) {
      const int c = i % kBlkRows, rest = i / kBlkRows, t = rest % P.T, r = sm.last_unit[rest / P.T] * kBlkRows + c;
      if (r >= P.N) continue;
      float y = 0.f;
#pragma unroll 1
      for (int z0 = 0; z0 < planes; z0 += 4) {  // four loads on their way; a choice's parts one after the other
        float o[4], w[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int z = min(z0 + u, planes - 1), j = z / P.splits, sp = z - j * P.splits;
          o[u] = __ldcg(P.part + ((long long)sp * P.n + t * P.k + j) * P.N + r);
          w[u] = z0 + u < planes ? __ldcg(P.wt + t * P.k + j) : 0.f;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) y += z0 + u < planes ? w[u] * o[u] : 0.f;
      }
      if (P.y_f32) ((float*)P.y)[(long long)t * P.N + r] = y;
      else ((__nv_bfloat16*)P.y)[(long long)t * P.N + r] = __float2bfloat16_rn(y);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kFewTmem) : "memory");
}

// ---------------------------------------------------------------- host
struct FewPlan {
  int m, tok_rows, stages;
  size_t smem;
};
// Whether rows of K values, n at most of an expert, fit beside a ring of four stages at least.  Half of an SM's shared memory where
// that will do: the next kernel's CTAs then start beside this one's, and the down matrices are on their way while the hidden rows are
// still being made.
bool few_plan(const moe_ctx* ctx, int K, int n, FewPlan* plan) {
  const int chunks = (K + 127) / 128;
  plan->m = n <= 16 ? 16 : 32, plan->tok_rows = n <= 8 ? 8 : plan->m;
  // (the last stage's lower half reads up to 7 KB behind the ring)
  const size_t toks = (size_t)((chunks + 1) / 2) * plan->tok_rows * 128 + (size_t)chunks * plan->tok_rows * 4;
  const size_t rest = std::max<size_t>(toks + (size_t)2 * plan->m * kBlkRows * 4, 8192) + 2048;
  const size_t all = (size_t)ctx->max_smem_optin - sizeof(FewSmem);
  const size_t half = (size_t)(ctx->max_smem_optin + 1024) / 2 - 1024 - sizeof(FewSmem);  // (1 KB of each CTA is the system's)
  const size_t room = rest + 4 * kFewStage <= half ? half : all;
  if (rest + 4 * kFewStage > room) return false;
  plan->stages = (int)std::min<size_t>(kFewStages, (room - rest) / kFewStage);
  plan->smem = plan->stages * (size_t)kFewStage + rest;
  return true;
}

int few_maps(const moe_fp4* w, CUtensorMap* codes, CUtensorMap* scales) {
  const Fp4Shape sh = fp4_shape(w->rows, w->n);
  const cuuint32_t es[2] = {1, 1};
  {
    const cuuint64_t dims[2] = {(cuuint64_t)sh.pitch, (cuuint64_t)w->rows}, strides[1] = {(cuuint64_t)sh.pitch};
    const cuuint32_t box[2] = {128, kBlkRows};
    if (encode_tiled(codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, w->codes, dims, strides, box, es, CU_TENSOR_MAP_SWIZZLE_128B,
                     CU_TENSOR_MAP_L2_PROMOTION_L2_256B) != CUDA_SUCCESS)
      return MOE_ERR_CUDA;
  }
  const cuuint64_t dims[2] = {(cuuint64_t)sh.rp, (cuuint64_t)sh.chunks}, strides[1] = {(cuuint64_t)sh.rp * 4};
  const cuuint32_t box[2] = {kBlkRows, 4};
  return encode_tiled(scales, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, w->scales, dims, strides, box, es, CU_TENSOR_MAP_SWIZZLE_NONE,
                      CU_TENSOR_MAP_L2_PROMOTION_L2_256B) == CUDA_SUCCESS
             ? MOE_OK
             : MOE_ERR_CUDA;
}

template <int MODE>
int few_launch(moe_ctx* ctx, const moe_fp4* w, FewParams& P, const FewPlan& plan, cudaStream_t s) {
  CUtensorMap codes, scales;
  MOE_TRY(few_maps(w, &codes, &scales));
  P.K = w->n, P.w = fp4_shape(w->rows, w->n), P.N = (int)(w->rows / P.E);
  const int all = (P.K + kStageK - 1) / kStageK;
  P.part_stages = (all + P.splits - 1) / P.splits, P.splits = (all + P.part_stages - 1) / P.part_stages;
  P.units = (P.N + kBlkRows - 1) / kBlkRows, P.stages = plan.stages, P.m = plan.m, P.tok_rows = plan.tok_rows, P.st = ctx->d_state;
  MOE_TRY((allow_full_smem<fp4_few_kernel<MODE>>(ctx)));
  const int most = std::min(P.E, P.n);  // experts with rows
  const long long items = (long long)P.units * P.splits * most;
  const int grid = (int)std::max<long long>(most, std::min<long long>(items, ctx->sm_count));
  MOE_CUDA_TRY(launch_pdl(fp4_few_kernel<MODE>, dim3(grid), dim3(kFewThreads), plan.smem, s, codes, scales, P));
  ctx->launches++;
  return MOE_OK;
}

}  // namespace

bool fp4_few_applies(const moe_ctx* ctx, int K, int n) {
  FewPlan p;
  return n <= kFewRows && few_plan(ctx, K, n, &p);
}

int launch_fp4_few_rows(moe_ctx* ctx, const moe_fp4* a, const moe_fp4* w, const int32_t* offsets, int E, void* out, int out_f32,
                        long long out_stride, cudaStream_t s) {
  FewPlan plan;
  if (!few_plan(ctx, w->n, (int)a->rows, &plan)) return MOE_ERR_UNSUPPORTED;
  FewParams P{};
  P.a_codes = (const unsigned char*)a->codes, P.a_scales = (const uint32_t*)a->scales, P.a = fp4_shape(a->rows, a->n);
  P.offsets = offsets, P.n = (int)a->rows, P.E = E, P.splits = 1;
  P.out = out, P.out_stride = out_stride, P.out_f32 = out_f32;
  return few_launch<FEW_OUT>(ctx, w, P, plan, s);
}

// part: kFewSplits planes of [T k][d] fp32; arrived: a word for each 64 columns.
int launch_fp4_few_experts(moe_ctx* ctx, const void* x, int T, const moe_fp4* gu, const moe_fp4* down, const int32_t* idx, const float* wt,
                           void* y, const moe_fp4* h, float* part, unsigned* arrived, cudaStream_t s) {
  const moe_config& c = ctx->cfg;
  const int E = c.n_experts, n = T * c.top_k, most = std::min(E, n);
  FewPlan plan;
  if (!few_plan(ctx, c.d_model, T, &plan)) return MOE_ERR_UNSUPPORTED;
  FewParams P{};
  P.x = x, P.x_f32 = c.x_dtype == MOE_F32, P.k = c.top_k;
  P.idx = idx, P.n = n, P.E = E, P.splits = 1;
  P.h_codes = (unsigned char*)h->codes, P.h_scales = (unsigned char*)h->scales, P.h = fp4_shape(h->rows, h->n);
  P.next = fp4_shape(down->rows, down->n), P.next_N = c.d_model;
  P.arrived = arrived;
  // the selected experts' down matrices come into L2 (126 MB) behind their gate and up rows
  if ((long long)most * c.d_model * P.next.pitch <= (64ll << 20))
    P.next_codes = (const unsigned char*)down->codes, P.next_scales = (const uint32_t*)down->scales;
  MOE_TRY(few_launch<FEW_HIDDEN>(ctx, gu, P, plan, s));
  if (!few_plan(ctx, c.d_ff, T, &plan)) return MOE_ERR_UNSUPPORTED;
  FewParams D{};
  D.a_codes = (const unsigned char*)h->codes, D.a_scales = (const uint32_t*)h->scales, D.a = P.h;
  D.idx = idx, D.n = n, D.E = E, D.k = c.top_k, D.T = T, D.wt = wt, D.y = y, D.y_f32 = P.x_f32, D.part = part, D.arrived = arrived;
  // parts of the contraction where blocks alone leave SMs idle
  const int units = (c.d_model + kBlkRows - 1) / kBlkRows, all = (c.d_ff + kStageK - 1) / kStageK;
  D.splits = std::max(1, std::min({kFewSplits, all, ctx->sm_count / (units * most)}));
  return few_launch<FEW_DOWN>(ctx, down, D, plan, s);
}

}  // namespace cosmoe
