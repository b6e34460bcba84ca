// Tree attention of 9 to 64 score columns per (sequence, kv head) at head_dim 128, with the TOKENS on the MMA's M axis.
//
//   S^T[128 tok x NC]   = K_slot[128 tok x 128] . Q^T          tcgen05.mma M128, N = NC columns
//   O^T[128 dim x NC] (+)= V_slot^T[128 dim x 128 tok] . P     tcgen05.mma M128, N = NC columns
//   L  [any     x NC] (+)= ones . P                            the columns' sums of weights, the same in every lane
//
// Why this way round.  The chunk kernel with score columns on M (chunk_tc2_kernels.cuh) spends the same time on a stage
// of 128 tokens whether its 128 rows are full or not, and its row-wise softmax is a chain through shuffles; over the
// 8-bit cache it widens K and V to 16 bits first.  Here the work of a stage is proportional to the columns there are: a
// thread owns a token, reads its NC scores from tensor memory, and writes its NC weights as one row of the second MMAs'
// B operand; no transposition, no shuffle.  The sums over tokens, which would need them, come from the tensor core, which
// is idle most of the time: summed with the same rounded weights as the numerator, in fp32.  The 8-bit scores come straight
// from the stored codes (kind::f8f6f4): a bf16 query value has 8 significant bits, so it is the sum of two E4M3 terms of
// 4 each, exactly (down to 2^-17 of its row's largest), and both terms accumulate into the same scores.  Only V is widened.
//
// A column's running maximum spans tokens, i.e. threads and warps.  It is only a reference: weights are 2^(x - ref),
// and ref, a score of the unit's first tokens, follows the true maximum when that is far above it (kTokRaise).  So a stage
// needs no maximum; its threads vote once whether any score did, and only then (and on stages with nodes of the tree, where
// a column may see its first token) the maxima are formed and the accumulators rescaled.
//
// Two pipelines t = 0, 1 work on alternating stages with softmax warps, score and weight buffers and an accumulator
// each (a split of the tokens, merged by log-sum-exp when the unit of work ends): each is a serial chain scores ->
// softmax -> P.V, and they fill each other's gaps.  A unit's stage count is padded to an even number with stages without
// tokens, so that both take part in every unit.
//
//   warps 0 - 3, 4 - 7   softmax of pipeline 0, 1 (thread = token)
//   warp 8               K producer: walks the units, TMA copies of K, posts meta words and V boxes
//   warp 9               V producer
//   warps 10, 11         one lane issues the MMAs of pipeline 0, 1
//   warps 12 - 15        8-bit cache: split the query rows into the two terms, widen V
//   warp 12              16-bit cache: TMA copies of the query rows, straight into the operand tile
// Every wait is bounded; a wait that gives up sets the status bit and the CTA's abort flag, every warp falls through to
// the common exit, and the tensor memory is released after the MMAs in flight.
//
// Measured, whole call (plan 10 us, this kernel, merge 12 us; 64 sequences of 256 to 8192 tokens, 8 kv heads; in brackets
// the causal operator over the same inputs, which has no mask to apply): 16-bit cache 9 columns 109 us (116), 16: 111 (123),
// 18: 112 (116), 32: 115 (120), 48: 124 (125), 64: 132 (128); 8-bit cache 9: 95 (124), 16: 95 (129), 18: 103 (127), 32: 105
// (129), 48: 120 (133), 64: 151 (136).  The rule's other side, the kernel with columns on M compiled with the tree's mask, in
// the same run: 36 columns 120 us here, 130 there (8-bit 135, 169); 48: 122, 132 (122, 152); 64: 131 to 136, 135 to 140
// (151, 152 to 155); 32 sequences of 4096 to 32768 tokens, 40 columns: 321, 337 (276, 365).  Beyond 64, with earlier versions
// of both: 96: 228 here, 156 there (267, 193), since scores and accumulators fill tensor memory at 64.  That last batch over the
// 8-bit cache takes 255 to 296 us from run to run, 3.1 to 3.6 TB/s of codes.  At 18 columns the 16-bit call runs at 0.85 of the
// measured copy rate, plan and merge included.  Over the 8-bit cache a stage of 128 tokens takes about 1900 cycles where its 32 KiB would take 1400, and a change of
// units some thousand more: a pipeline's chain (weights, barriers between the roles, widening, P.V) is what bounds it, two
// pipelines cannot hide all of it, and four sets of softmax warps do not fit the register file.  What mattered: deep rings
// (three K and V slots instead of two, at the price of a second weight buffer: 5 us of 120), and that the compiler knows
// the warp's number to be the same in all lanes, so that addresses live in uniform registers (17 us of 278).
#pragma once
#include <type_traits>

#include "chunk_tc2_kernels.cuh"

namespace ooco {

constexpr int kTokMeta = 8, kTokDesc = 8;  // ring sizes: meta words, V descriptors
constexpr int kTokMinColumns = 9, kTokMaxColumns = 64;  // score columns that the kernel takes (both sides measured above)
// A reference is raised when a score passes it by this much (log2 units): weights stay below 2^16 for f16 (the 8-bit
// cache), where small ones lose bits below 2^-14; bf16 has the range of fp32, and a column's sum stays below 2^60 times its tokens.
template <bool KV8>
constexpr float kTokRaise = KV8 ? 14.f : 60.f;

template <int NC, bool KV8>
struct TokSmem {
  static constexpr int SB = NC <= 48 ? 2 : 1;                               // score buffers of a pipeline (tensor memory is full)
  static constexpr int kQBytes = NC * 256;                                  // [2][NC rows][128 bytes]
  static constexpr int kPBytes = 128 * 128;                                 // [128 tok][64 columns] f16
  static constexpr int kLandBytes = KV8 ? kTc2RawSlotBytes : kTc2SlotBytes; // K (or V) of one stage as TMA writes it
  static constexpr int NK = KV8 && NC <= 48 ? 3 : 2, NV = 3, NW = 2;        // K slots, V slots, widened V slots
  // 8-bit cache: four warps widen V, together (48 columns: 278 us for the long batch above, 296 in two groups), or, where the
  // softmax is short and the widening the longer chain, in a group for each pipeline, of which one works while the other
  // waits (32 columns: 107 us, 114 together).
  static constexpr int kWidenGroups = NC <= 32 ? 2 : 1, kWidenWarps = 4 / kWidenGroups;
  static constexpr int kWarps = KV8 ? 16 : 13;
  // tensor memory: scores [2 pipelines][SB], values [2], sums [2], the operand of ones
  static constexpr int kTmemCols = 512;
  static constexpr int kColO = 2 * SB * NC, kColL = kColO + 2 * NC, kColOne = kColL + 2 * NC;
  static_assert(kColOne + 8 <= kTmemCols, "tensor memory");
  // per column: factors and references of both pipelines, factors of the unit, the warps' maxima, factors of a rescaling,
  // the references at a unit's end (two sets take turns)
  static constexpr int kColumnBytes = NC * (2 * 8 + 4 + 2 * 4 * 4 + 2 * 4 + 4 * 4);
  __host__ __device__ static constexpr size_t total() {
    return 1024 + (KV8 ? 2 : 1) * (size_t)kQBytes + 2 * (size_t)kPBytes + (size_t)(NK + NV) * kLandBytes +
           (KV8 ? (size_t)NW * kTc2SlotBytes : 0) + kTokMeta * 32 + 2 * 16 + kTokDesc * sizeof(VStageDesc) + kColumnBytes + 672;
  }
  static constexpr size_t kMost = 227 * 1024;  // shared memory of a CTA
};

// 16 fp32 columns of the calling lane's row.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}

// Whether the barrier's phase of parity `parity` is complete, without waiting for it.
__device__ __forceinline__ bool mbar_test_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// warp_wait out of line: the kernel has dozens of waits, and its code has to fit the instruction cache.
__device__ __noinline__ bool tok_wait_slow(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  uint64_t t0 = 0;  // (reading the clock takes some hundred cycles: not before it is a long wait)
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (mbar_try_wait(bar, parity)) return true;
    if (*abort_flag) return false;
    const uint64_t now = globaltimer_ns();
    if (t0 == 0) t0 = now;
    if (now - t0 > kWaitLimitNs) {
      *abort_flag = 1;
      return false;
    }
  }
}
__device__ __forceinline__ bool tok_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  return __all_sync(0xffffffffu, mbar_try_wait(bar, parity) || tok_wait_slow(bar, parity, abort_flag));
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, uint32_t v) {  // the same word into 8 columns
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%1,%1,%1,%1,%1,%1,%1};" ::"r"(taddr), "r"(v));
}
// True in one lane of the converged warp, always the same.
__device__ __forceinline__ bool elect_one() {
  uint32_t yes;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
  return yes != 0;
}
__device__ __forceinline__ float warp_max(float v) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const void* tmap, uint32_t bar, int c0, int c1, int c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
      "l"(tmap), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
      : "memory");
}

template <int NC, bool KV8>
__global__ void __launch_bounds__(TokSmem<NC, KV8>::kWarps * 32, 1)
tree_tok_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                const __grid_constant__ CUtensorMap tm_q, const DecodeParams p) {
  using L = TokSmem<NC, KV8>;
  constexpr int D = 128, TOK = kTc2StageTok;
  constexpr int SB = L::SB, NK = L::NK, NV = L::NV, NW = L::NW;
  constexpr int kWarpK = 8, kWarpV = 9, kWarpM = 10, kWarpX = 12;
  static_assert(L::total() <= L::kMost, "shared memory");
  static_assert(NC % 16 == 0 && NC <= kTokMaxColumns, "columns of an MMA with M = 128, and what shared memory holds");
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const uint32_t s_q = base;                                             // the unit's query rows as two terms
  const uint32_t s_qraw = s_q + (uint32_t)L::kQBytes;                    // ... in bf16
  const uint32_t s_p = s_qraw + (KV8 ? (uint32_t)L::kQBytes : 0u);       // [2 pipelines] weights
  const uint32_t s_k = s_p + 2u * L::kPBytes;                            // [NK] K slots
  const uint32_t s_v = s_k + (uint32_t)NK * L::kLandBytes;               // [NV] V slots
  const uint32_t s_w = s_v + (uint32_t)NV * L::kLandBytes;               // [NW] widened V slots
  const uint32_t s_unit = s_w + (KV8 ? (uint32_t)NW * kTc2SlotBytes : 0u);  // [2] int4 {sequence, kv head}, 16-bit cache
  const uint32_t s_meta = s_unit + 32;            // [kTokMeta] two int4
  const uint32_t s_vdesc = s_meta + kTokMeta * 32;                       // [kTokDesc] VStageDesc
  const uint32_t s_cr = s_vdesc + kTokDesc * (uint32_t)sizeof(VStageDesc);  // [2][NC / 2] {score factors, -references} of column pairs
  const uint32_t s_mul = s_cr + 2u * NC * 8;                             // [NC] score factor of the unit's columns
  const uint32_t s_max = s_mul + NC * 4;                                 // [2][4 warps][NC] maxima
  const uint32_t s_alpha = s_max + 2u * 4 * NC * 4;                      // [2][NC] factors of a rescaling
  const uint32_t s_ref = s_alpha + 2u * NC * 4;                          // [2 sets][2][NC] references at a unit's end
  const uint32_t s_bar = (s_ref + 4u * NC * 4 + 7u) & ~7u;
  const uint32_t s_kfull = s_bar;                    // [2 NK] K has landed                            (TMA)
  const uint32_t s_kempty = s_kfull + 2 * NK * 8;    // [NK] the score MMAs that read it are complete  (commit)
  // (K or V has landed, V is widened: twice as many barriers as slots, of which stage n takes number n % (2 slots).  So a barrier
  // is one pipeline's, which sees each of its phases; one per slot could be two phases behind, and let a wait through.)
  const uint32_t s_vland = s_kempty + NK * 8;        // [2 NV] V has landed                            (TMA)
  const uint32_t s_vtaken = s_vland + 2 * NV * 8;    // [NV] it may be overwritten                     (widening threads)
  const uint32_t s_wfull = s_vtaken + NV * 8;        // [2 NW] the widened slot is written         (widening threads)
  const uint32_t s_wempty = s_wfull + 2 * NW * 8;    // [NW] the P.V MMAs that read it are complete (commit)
  const uint32_t s_vdfull = s_wempty + NW * 8;       // [kTokDesc] the stage's V descriptor is posted
  const uint32_t s_mfull = s_vdfull + kTokDesc * 8;  // [kTokMeta] the stage's meta words are posted
  const uint32_t s_qready = s_mfull + kTokMeta * 8;  // the unit's query tile is written              (widening threads)
  const uint32_t s_qfree = s_qready + 8;             // ... may be overwritten: both pipelines' last score MMAs are
                                                     //     complete, both have read the columns' factors (4)
  const uint32_t s_sready = s_qfree + 8;             // [2 pipelines][2] the scores are in tensor memory (commit)
  const uint32_t s_sfree = s_sready + 32;            // [2][2] ... have been read                      (4 warps)
  const uint32_t s_pready = s_sfree + 32;            // [2] weights written, O rescaled, V rows clean (4 warps)
  const uint32_t s_pvdone = s_pready + 16;           // [2] the stage's P.V is complete             (commit)
  const uint32_t s_wg = s_pvdone + 16;               // [2] the four warps of a pipeline meet          (4)
  const uint32_t s_both = s_wg + 16;                 // [1] the softmax warps of both pipelines meet   (8)
  const uint32_t s_qland = s_both + 8;               // the unit's bf16 query rows have landed         (TMA)
  const uint32_t s_qtaken = s_qland + 8;             // ... have been split                            (widening threads)
  const uint32_t s_ofree = s_qtaken + 8;             // the unit's accumulators have been read               (8 warps)
  const uint32_t s_ufull = s_ofree + 8;              // [2] the unit is posted                          (16-bit cache)
  const uint32_t s_drain = s_ufull + 16;             // [2]
  const uint32_t s_slot = s_drain + 16;              // tensor-memory base, abort flag, votes [2 pipelines][2][4 warps]
  int4* g_unit = reinterpret_cast<int4*>(gen + (s_unit - base));
  int4* g_meta = reinterpret_cast<int4*>(gen + (s_meta - base));
  VStageDesc* g_vdesc = reinterpret_cast<VStageDesc*>(gen + (s_vdesc - base));
  volatile uint32_t* g_slot = reinterpret_cast<volatile uint32_t*>(gen + (s_slot - base));
  volatile int* s_abort = reinterpret_cast<volatile int*>(gen + (s_slot + 4 - base));
  volatile int* g_vote = reinterpret_cast<volatile int*>(gen + (s_slot + 8 - base));
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;  // (known to be the same in all lanes)

  if (threadIdx.x == 0) {
    *s_abort = 0;
    for (int i = 0; i < 2 * NK; ++i) mbar_init(s_kfull + 8 * i, 1);
    for (int i = 0; i < NK; ++i) mbar_init(s_kempty + 8 * i, 1);
    for (int i = 0; i < 2 * NV; ++i) mbar_init(s_vland + 8 * i, 1);
    for (int i = 0; i < NV; ++i) mbar_init(s_vtaken + 8 * i, KV8 ? L::kWidenWarps : 1);
    for (int i = 0; i < 2 * NW; ++i) mbar_init(s_wfull + 8 * i, L::kWidenWarps);
    for (int i = 0; i < NW; ++i) mbar_init(s_wempty + 8 * i, 1);
    for (int i = 0; i < kTokDesc; ++i) mbar_init(s_vdfull + 8 * i, 1);
    for (int i = 0; i < kTokMeta; ++i) mbar_init(s_mfull + 8 * i, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_wg + 8 * i, 4);
      mbar_init(s_pready + 8 * i, 4);
      mbar_init(s_pvdone + 8 * i, 1);
      mbar_init(s_drain + 8 * i, 1);
      mbar_init(s_ufull + 8 * i, 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(s_sready + 8 * i, 1);
      mbar_init(s_sfree + 8 * i, 4);
    }
    mbar_init(s_qready, KV8 ? 4 : 1);
    mbar_init(s_qfree, 4);
    mbar_init(s_both, 8);
    mbar_init(s_ofree, 8);
    mbar_init(s_qland, 1);
    mbar_init(s_qtaken, 4);
    fence_mbar_init();
  }
  // query rows of columns that do not exist are never copied: zero, so that their scores are
  for (uint32_t i = threadIdx.x; i < (s_p - s_q) / 16; i += L::kWarps * 32)
    *reinterpret_cast<uint4*>(gen + 16 * (size_t)i) = make_uint4(0u, 0u, 0u, 0u);
  fence_proxy_async_smem();
  if (warp == kWarpM) tmem_alloc(s_slot, L::kTmemCols);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *g_slot;
  if (warp < 4) {  // the operand that sums the weights: ones
    tmem_st8(tmem + ((uint32_t)(32 * warp) << 16) + L::kColOne, KV8 ? 0x3c003c00u : 0x3f803f80u);
    tmem_st_wait();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  grid_dep_wait();    // the plan must have completed
  grid_dep_launch();  // the merge kernel may queue up behind this grid

  const long long cap_tokens = (long long)p.MB * p.bs;

  // The unit's query rows: score column (query token qi, head g) is row qi * G + g, per 64-dim half a box of [Sq][G][64 dims],
  // swizzled.
  auto copy_queries = [&](uint32_t dst, uint32_t bar, int b, int h) {
    mbar_arrive_expect_tx(bar, 2u * (uint32_t)p.GQ * 128u);
    tma_load_3d(dst, &tm_q, bar, 0, h * p.G, b * p.Sq);
    tma_load_3d(dst + NC * 128, &tm_q, bar, 64, h * p.G, b * p.Sq);
  };
  if (warp == kWarpK) {
    // ================================================================= K producer (and the walk over the units)
    if (lane == 0) {
      prefetch_tmap(&tm_k);
      prefetch_tmap(&tm_q);
    }
    const int n_units = p.hdr->n_items;
    const int boxes_per_stage = TOK / p.tile_rows;  // at most 8
    const uint32_t box_bytes = (uint32_t)p.tile_rows * 128;
    int it = 0, u = 0;
    bool ok = true, violated = false;
    int item = blockIdx.x;
    auto table_entry = [&](const int32_t* e) {
      const int v = *e;
      return checked(chk_table_entry(v, p.NB), &p.hdr->status, kStatusBadTableEntry) ? v : p.NB;
    };
    // Waits for stage `it`'s K slot.  A free K slot also means that the meta words and the V descriptor that this stage
    // overwrites have been used: the scores of stage it - NK are complete, a pipeline issues the P.V of a stage before the
    // scores of the stage after the next, hence everything about stages up to it - NK - 4 is done with.
    auto acquire = [&]() { return tok_wait(s_kempty + 8 * (it % NK), (((uint32_t)(it / NK)) & 1u) ^ 1u, s_abort); };
    while (item < n_units && ok) {
      int nxt = 0;
      if (lane == 0) nxt = atomicAdd(&p.hdr->next_item, 1);
      nxt = __shfl_sync(0xffffffffu, nxt, 0);
      const int4 d = p.items[item];
      if (!checked(chk_item(d.x, d.y, d.z, d.w, p.B, p.max_items, cap_tokens), &p.hdr->status, kStatusBadItem)) {
        *s_abort = 1;
        violated = true;
        ok = false;
        break;
      }
      const int b = d.x, h = d.y % p.Hkv, t0 = d.z, t1 = d.w;
      long long T = p.context_lens[b];
      T = T < 0 ? 0 : (T > cap_tokens ? cap_tokens : T);
      const int nodes = tree_nodes(p, b), first_node = (int)T - nodes;  // token index of node 0
      const int nstage = t1 > t0 ? (t1 - t0 + TOK - 1) / TOK : 0, npad = nstage < 2 ? 2 : (nstage + 1) & ~1;
      if (KV8) {  // the query rows, for the widening warps to split
        if (!tok_wait(s_qtaken, ((uint32_t)u & 1u) ^ 1u, s_abort)) {
          ok = false;
          break;
        }
        if (lane == 0) copy_queries(s_qraw, s_qland, b, h);
      } else if (lane == 0) {  // (the unit before the last has been taken: its scores are complete)
        g_unit[u & 1] = make_int4(b, h, 0, 0);
        mbar_arrive(s_ufull + 8 * (u & 1));
      }
      __syncwarp();
      const int32_t* row = p.block_table + (size_t)b * p.MB;
      int blk_cur = 0;
      {
        const int tb = t0 + lane * p.tile_rows;
        if (lane < boxes_per_stage && tb < t1) blk_cur = table_entry(row + tb / p.bs);
      }
      ++u;
      for (int s = 0; s < npad; ++s, ++it) {
        const int tok0 = t0 + s * TOK;
        const int ntok = s < nstage ? min(TOK, t1 - tok0) : 0;
        const int nbox = (ntok + p.tile_rows - 1) / p.tile_rows;
        int blk_n = 0;  // table entries of the following stage, one stage ahead of their use
        {
          const int tb = tok0 + TOK + lane * p.tile_rows;
          if (s + 1 < nstage && lane < boxes_per_stage && tb < t1) blk_n = table_entry(row + tb / p.bs);
        }
        if (!acquire()) {
          ok = false;
          break;
        }
        const int ks = it % NK, ms = it % kTokMeta, ds = it % kTokDesc;
        const uint32_t kfull = s_kfull + 8 * (it % (2 * NK));
        if (lane == 0) {
          const int flags = (s < 2 ? 1 : 0) | (s >= npad - 2 ? 2 : 0);  // a pipeline's first / last stage of the unit
          g_meta[2 * ms] = make_int4(d.y, b, h, ntok | (flags << 16));
          g_meta[2 * ms + 1] = make_int4(tok0, first_node, nodes, u - 1);
          g_vdesc[ds].nbox = nbox;
          g_vdesc[ds].h = h;
          if (nbox > 0)
            mbar_arrive_expect_tx(kfull, (KV8 ? 1u : 2u) * (uint32_t)nbox * box_bytes);
          else
            mbar_arrive(kfull);
        }
        __syncwarp();
        bool span_ok = true;
        if (lane < nbox) {
          const int tb = tok0 + lane * p.tile_rows;
          const int c_tok = tb % p.bs;
          const uint32_t k0 = s_k + (uint32_t)ks * L::kLandBytes;
          const uint32_t dk = k0 + (uint32_t)lane * box_bytes;
          span_ok = checked(chk_span(dk, box_bytes, k0, (long long)k0 + kTc2HalfBytes) && chk_span(lane, 1, 0, 8),
                            &p.hdr->status, kStatusBadSmem);
          if (span_ok) {
            tma_load_4d(dk, &tm_k, kfull, 0, c_tok, h, blk_cur);  // (KV8: the row's 128 codes; else its first 64 dims)
            if (!KV8) tma_load_4d(dk + kTc2HalfBytes, &tm_k, kfull, 64, c_tok, h, blk_cur);
            g_vdesc[ds].blk[lane & 7] = blk_cur;
            g_vdesc[ds].c_tok[lane & 7] = c_tok;
          }
        }
        if (kChecked && !__all_sync(0xffffffffu, span_ok)) {  // a skipped copy leaves the stage incomplete: stop
          *s_abort = 1;
          violated = true;
          ok = false;
          break;
        }
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(s_vdfull + 8 * ds);
          mbar_arrive(s_mfull + 8 * ms);
        }
        blk_cur = blk_n;
      }
      item = nxt;
    }
    if (!KV8 && ok && lane == 0) {
      g_unit[u & 1] = make_int4(-1, 0, 0, 0);
      mbar_arrive(s_ufull + 8 * (u & 1));
    }
    for (int k = 0; k < 2 && ok; ++k) {  // end markers, one for each pipeline
      if (!acquire()) {
        ok = false;
        break;
      }
      if (lane == 0) {
        g_meta[2 * (it % kTokMeta)] = make_int4(-1, 0, 0, 0);
        g_vdesc[it % kTokDesc].nbox = -1;
        mbar_arrive(s_kfull + 8 * (it % (2 * NK)));
        mbar_arrive(s_vdfull + 8 * (it % kTokDesc));
        mbar_arrive(s_mfull + 8 * (it % kTokMeta));
      }
      ++it;
    }
    if (!ok) {  // stop path: record it, then wait (bounded) until every K copy already issued has landed
      if (lane == 0 && !violated) atomicOr(&p.hdr->status, kStatusWaitTimeout);
      int dummy_abort = 0;
      for (int k = 0; k < (it < NK ? it : NK); ++k) {
        const int j = it - 1 - k;
        mbar_wait_bounded(s_kfull + 8 * (j % (2 * NK)), (uint32_t)(j / (2 * NK)) & 1u, &dummy_abort, kWaitLimitNs / 8);
      }
      if (KV8 && u > 0) mbar_wait_bounded(s_qland, (uint32_t)(u - 1) & 1u, &dummy_abort, kWaitLimitNs / 8);
    }
  } else if (warp == kWarpV) {
    // ================================================================= V producer
    if (lane == 0) prefetch_tmap(&tm_v);
    const uint32_t box_bytes = (uint32_t)p.tile_rows * 128;
    int it = 0;
    bool ok = true;
    for (;; ++it) {
      const int vs = it % NV, ds = it % kTokDesc;
      if (!tok_wait(s_vdfull + 8 * ds, (uint32_t)(it / kTokDesc) & 1u, s_abort)) {
        ok = false;
        break;
      }
      const VStageDesc& vd = g_vdesc[ds];
      const int nbox = vd.nbox;
      if (nbox < 0) break;
      if (!tok_wait(s_vtaken + 8 * vs, (((uint32_t)(it / NV)) & 1u) ^ 1u, s_abort)) {
        ok = false;
        break;
      }
      const uint32_t vland = s_vland + 8 * (it % (2 * NV));
      if (nbox == 0) {  // a stage without tokens
        if (lane == 0) mbar_arrive(vland);
        continue;
      }
      if (lane == 0) mbar_arrive_expect_tx(vland, (KV8 ? 1u : 2u) * (uint32_t)nbox * box_bytes);
      __syncwarp();
      if (lane < nbox && lane < 8) {
        const uint32_t dv = s_v + (uint32_t)vs * L::kLandBytes + (uint32_t)lane * box_bytes;
        tma_load_4d(dv, &tm_v, vland, 0, vd.c_tok[lane], vd.h, vd.blk[lane]);
        if (!KV8) tma_load_4d(dv + kTc2HalfBytes, &tm_v, vland, 64, vd.c_tok[lane], vd.h, vd.blk[lane]);
      }
    }
    if (!ok) {
      if (lane == 0) atomicOr(&p.hdr->status, kStatusWaitTimeout);
      int dummy_abort = 0;
      for (int k = 0; k < (it < NV ? it : NV); ++k) {
        const int j = it - 1 - k;
        mbar_wait_bounded(s_vland + 8 * (j % (2 * NV)), (uint32_t)(j / (2 * NV)) & 1u, &dummy_abort, kWaitLimitNs / 8);
      }
    }
  } else if (warp == kWarpM || warp == kWarpM + 1) {
    // ================================================================= MMA warps: warp kWarpM + t issues pipeline t's MMAs
    // Stage i of the pipeline is stage 2 i + t of the CTA.  The scores of stage i + 1 are issued before the P.V of stage i, so
    // that they run beside the softmax of stage i, unless the weights are there before the scores' operands.
    // (the pipeline is a compile-time constant, so that the operands' addresses are known to be the same in all lanes)
    auto issue = [&](auto pipeline) {
    constexpr int t = decltype(pipeline)::value;
    const uint32_t idesc_s = KV8 ? (1u << 4) | ((uint32_t)(NC >> 3) << 17) | ((uint32_t)(TOK >> 4) << 24)  // E4M3 by E4M3
                                 : umma_idesc_16bit(TOK, NC, 0, true);
    const uint32_t idesc_l = umma_idesc_16bit(D, NC, 1, !KV8), idesc_o = idesc_l | (1u << 15);  // A (V) is M-major, too
    const uint32_t to = tmem + L::kColO + (uint32_t)t * NC, tl = tmem + L::kColL + (uint32_t)t * NC;
    bool issued = false, ok = true, ended = false;
    uint32_t i = 0, j = 0;  // next stage whose scores / P.V are issued; i - j <= 2
    auto now = [](uint32_t bar, uint32_t par) { return __all_sync(0xffffffffu, mbar_test_wait(bar, par)); };
    while (!ended || j < i) {
      const uint32_t n = 2 * i + t;
      const int ks = n % NK, ms = n % kTokMeta;
      const uint32_t kfull = s_kfull + 8 * (n % (2 * NK)), kpar = (n / (2 * NK)) & 1u;
      const uint32_t sfree = s_sfree + 8 * (2 * t + i % SB), spar = ((i - SB) / SB) & 1u;
      const bool may_s = !ended && i - j < 2, may_v = j < i;
      bool scores = may_s, there = false;  // (the scores' operands)
      if (may_s && may_v) {  // whichever can go ahead first
        uint64_t t_start = 0;
        for (uint32_t spin = 1;; ++spin) {
          if (now(kfull, kpar)) {
            const int4 meta = g_meta[2 * ms];
            const int unit = g_meta[2 * ms + 1].w;
            if (meta.x < 0 || ((i < SB || now(sfree, spar)) &&
                               (!((meta.w >> 16) & 1) || now(s_qready, (uint32_t)unit & 1u)))) {
              there = true;
              break;
            }
          }
          if (now(s_pready + 8 * t, j & 1u)) {
            scores = false;
            break;
          }
          if (spin % 1024 == 0) {
            const uint64_t t_now = globaltimer_ns();
            if (t_start == 0) t_start = t_now;
            if (__any_sync(0xffffffffu, *s_abort != 0 || t_now - t_start > kWaitLimitNs)) {
              *s_abort = 1;
              break;  // (the waits below give up soon)
            }
          }
        }
      }
      if (scores) {
        if (!there && !tok_wait(kfull, kpar, s_abort)) {
          ok = false;
          break;
        }
        const int4 meta = g_meta[2 * ms], meta2 = g_meta[2 * ms + 1];
        if (meta.x < 0) {
          ended = true;
          continue;
        }
        const int ntok = meta.w & 0xffff;
        const bool first = (meta.w >> 16) & 1, last = (meta.w >> 17) & 1;
        // (a stage without tokens waits for its unit's query rows, too: the arrivals at s_qfree below count for that unit)
        if ((i >= SB && !there && !tok_wait(sfree, spar, s_abort)) ||
            (first && !there && !tok_wait(s_qready, (uint32_t)meta2.w & 1u, s_abort))) {
          ok = false;
          break;
        }
        const uint32_t sready = s_sready + 8 * (2 * t + i % SB);
        if (ntok > 0) {
          tc_fence_after_sync();
          if (elect_one()) {
            const uint32_t ts = tmem + (uint32_t)(t * SB + i % SB) * NC;
            const uint64_t dk = umma_smem_desc(s_k + (uint32_t)ks * L::kLandBytes, 0, 1024), dq = umma_smem_desc(s_q, 0, 1024);
#pragma unroll
            for (int hh = 0; hh < 2; ++hh)  // the two terms; the two halves of the dims
#pragma unroll
              for (int k = 0; k < 4; ++k)  // 32 bytes per MMA
                if (KV8)
                  umma_f8_ss(ts, dk + 2 * k, dq + (uint64_t)(hh * NC * 8 + 2 * k), idesc_s, (hh | k) ? 1u : 0u);
                else
                  umma_ss(ts, dk + (uint64_t)(hh * (kTc2HalfBytes >> 4) + 2 * k), dq + (uint64_t)(hh * NC * 8 + 2 * k), idesc_s,
                          (hh | k) ? 1u : 0u);
            umma_commit(sready);
            umma_commit(s_kempty + 8 * ks);
            if (last) umma_commit(s_qfree);
          }
          issued = true;
        } else if (elect_one()) {  // the turn of the barriers is taken all the same
          mbar_arrive(sready);
          mbar_arrive(s_kempty + 8 * ks);
          if (last) umma_commit(s_qfree);  // the pipeline's scores of the stage before may still be on their way
        }
        __syncwarp();
        ++i;
      } else {
        const uint32_t m = 2 * j + t;
        constexpr int ring = KV8 ? NW : NV;
        const int vs = m % ring;
        const int4 meta = g_meta[2 * (m % kTokMeta)];
        const int unit = g_meta[2 * (m % kTokMeta) + 1].w;
        const bool some = (meta.w & 0xffff) > 0, first = (meta.w >> 16) & 1;
        // (a unit's first P.V overwrites the accumulator that the softmax warps read at the end of the unit before)
        if (!tok_wait((KV8 ? s_wfull : s_vland) + 8 * (m % (2 * ring)), (m / (2 * ring)) & 1u, s_abort) ||
            !tok_wait(s_pready + 8 * t, j & 1u, s_abort) ||
            (some && first && unit > 0 && !tok_wait(s_ofree, (uint32_t)(unit - 1) & 1u, s_abort))) {
          ok = false;
          break;
        }
        const uint32_t freed = (KV8 ? s_wempty : s_vtaken) + 8 * vs;
        if (some) {
          tc_fence_after_sync();
          if (elect_one()) {
            const uint64_t dp = umma_smem_desc(s_p + (uint32_t)t * L::kPBytes, 0, 1024);
            const uint64_t dv = umma_smem_desc((KV8 ? s_w : s_v) + (uint32_t)vs * kTc2SlotBytes, kTc2HalfBytes, 1024);
#pragma unroll
            for (int k = 0; k < TOK / 16; ++k)  // 16 tokens: 16 rows of 128 bytes of V and of P
              umma_ss(to, dv + (uint64_t)(k * (2048 >> 4)), dp + (uint64_t)(k * (2048 >> 4)), idesc_o, (first && k == 0) ? 0u : 1u);
#pragma unroll
            for (int k = 0; k < TOK / 16; ++k)  // the columns' sums of weights, in every lane
              umma_ts(tl, tmem + L::kColOne, dp + (uint64_t)(k * (2048 >> 4)), idesc_l, (first && k == 0) ? 0u : 1u);
            umma_commit(s_pvdone + 8 * t);
            umma_commit(freed);
          }
          issued = true;
        } else if (elect_one()) {
          mbar_arrive(s_pvdone + 8 * t);
          mbar_arrive(freed);
        }
        __syncwarp();
        ++j;
      }
    }
    if (!ok && lane == 0) atomicOr(&p.hdr->status, kStatusWaitTimeout);
    if (!ok && issued) {  // the tensor memory must not be released under MMAs in flight
      if (elect_one()) umma_commit(s_drain + 8 * t);
      __syncwarp();
      int dummy = 0;
      mbar_wait_bounded(s_drain + 8 * t, 0u, &dummy, kWaitLimitNs / 8);
    }
    };
    if (warp == kWarpM)
      issue(std::integral_constant<int, 0>{});
    else
      issue(std::integral_constant<int, 1>{});
  } else if (!KV8 && warp == kWarpX) {
    // ================================================================= query rows (16-bit cache)
    bool ok = true;
    uint32_t u = 0;
    for (;; ++u) {
      if (!tok_wait(s_ufull + 8 * (u & 1), (u >> 1) & 1u, s_abort)) {
        ok = false;
        break;
      }
      const int4 unit = g_unit[u & 1];
      if (unit.x < 0) break;
      if (!tok_wait(s_qfree, (u & 1u) ^ 1u, s_abort)) {
        ok = false;
        break;
      }
      if (lane == 0) copy_queries(s_q, s_qready, unit.x, unit.y);
      __syncwarp();
    }
    if (!ok) {
      if (lane == 0) atomicOr(&p.hdr->status, kStatusWaitTimeout);
      int dummy_abort = 0;
      if (u > 0) mbar_wait_bounded(s_qready, (u - 1) & 1u, &dummy_abort, kWaitLimitNs / 8);
    }
  } else if (KV8 && warp >= kWarpX) {
    // ================================================================= widening warps (8-bit cache)
    constexpr int kGroup = 32 * L::kWidenWarps;
    const int tid_w = threadIdx.x & (kGroup - 1);
    bool ok = true;
    uint32_t u = 0;
    for (uint32_t n = L::kWidenGroups == 2 ? (uint32_t)(warp - kWarpX) / L::kWidenWarps : 0u;; n += L::kWidenGroups) {
      const int vs = n % NV, ws = n % NW, ms = n % kTokMeta;
      if (!tok_wait(s_mfull + 8 * ms, (n / kTokMeta) & 1u, s_abort)) {
        ok = false;
        break;
      }
      const int4 meta = g_meta[2 * ms];
      if (meta.x < 0) break;
      const int ntok = meta.w & 0xffff;
      if (((meta.w >> 16) & 1) && (L::kWidenGroups == 2 || !(n & 1))) {
        // ---- a unit starts: its query rows as hi + lo, scaled by a power of two that brings the row's largest magnitude
        // into [128, 256) (E4M3 goes up to 448).  A warp takes every fourth row, lane l dims 4 l .. 4 l + 3.
        if (!tok_wait(s_qland, u & 1u, s_abort) || !tok_wait(s_qfree, (u & 1u) ^ 1u, s_abort)) {
          ok = false;
          break;
        }
        const uint8_t* src = gen + (s_qraw - base);
        uint8_t* dst = gen + (s_q - base);
        float* mul = reinterpret_cast<float*>(gen + (s_mul - base));
#pragma unroll 4
        for (int c = warp - kWarpX; c < NC; c += 4) {
          const uint2 w = *reinterpret_cast<const uint2*>(src + (size_t)(lane >> 4) * NC * 128 + (size_t)c * 128 +
                                                          ((((lane & 15) >> 1) ^ (c & 7)) << 4) + (lane & 1) * 8);
          const float x[4] = {__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                              __uint_as_float(w.y & 0xffff0000u)};
          float mx = warp_max(fmaxf(fmaxf(fabsf(x[0]), fabsf(x[1])), fmaxf(fabsf(x[2]), fabsf(x[3]))));
          if (!(mx <= 3.0e38f)) mx = 0.f;  // a row holding infinity is outside the contract: keep the scale finite
          int ae = 127 + 7 + 127 - (int)((__float_as_uint(mx) >> 23) & 0xffu);
          ae = mx > 0.f ? (ae > 254 ? 254 : ae) : 127;
          const float a = __uint_as_float((uint32_t)ae << 23), inv_a = __uint_as_float((uint32_t)(254 - ae) << 23);
          const uint32_t h01 = pack_e4m3x2(x[0] * a, x[1] * a), h23 = pack_e4m3x2(x[2] * a, x[3] * a);
          const uint32_t f01 = e4m3x2_to_f16x2<kSelB0B1>(h01), f23 = e4m3x2_to_f16x2<kSelB0B1>(h23);  // values / 256
          const uint32_t l01 = pack_e4m3x2(x[0] * a - f16_lo(f01) * kE4m3WidenFactor, x[1] * a - f16_hi(f01) * kE4m3WidenFactor);
          const uint32_t l23 = pack_e4m3x2(x[2] * a - f16_lo(f23) * kE4m3WidenFactor, x[3] * a - f16_hi(f23) * kE4m3WidenFactor);
          const uint32_t off = (uint32_t)c * 128 + ((((uint32_t)lane >> 2) ^ ((uint32_t)c & 7)) << 4) + ((uint32_t)lane & 3) * 4;
          *reinterpret_cast<uint32_t*>(dst + off) = h01 | (h23 << 16);
          *reinterpret_cast<uint32_t*>(dst + NC * 128 + off) = l01 | (l23 << 16);
          if (lane == 0) mul[c] = p.scale_log2e * inv_a;
        }
        fence_proxy_async_smem();  // the terms are read by the MMAs, the rows overwritten by TMA, through the async proxy
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(s_qready);
          mbar_arrive(s_qtaken);
        }
        ++u;
      }
      // ---- V codes to f16: exact, to value / 256; 1024 units of 16 codes, eight per thread
      if (!tok_wait(s_vland + 8 * (n % (2 * NV)), (n / (2 * NV)) & 1u, s_abort) ||
          !tok_wait(s_wempty + 8 * ws, ((n / NW) & 1u) ^ 1u, s_abort)) {
        ok = false;
        break;
      }
      if (ntok > 0) {
        const uint8_t* src = gen + (s_v - base) + (size_t)vs * kTc2RawSlotBytes;
        uint8_t* dst = gen + (s_w - base) + (size_t)ws * kTc2SlotBytes;
        // A unit of 16 codes (a 16-byte chunk of a row) becomes two chunks.  Eight lanes take four chunks of an even row and the
        // other four of the odd row behind it, so that neither their loads nor their stores meet at a bank.
        const int cl = tid_w & 3, odd = (tid_w >> 2) & 1, r0 = 2 * (tid_w >> 3) + odd;
        constexpr int kStep = kGroup / 4;  // rows r0 + kStep k
        const uint8_t* s0 = src + (size_t)r0 * 128;
        const int sa = ((cl + 4 * odd) ^ (r0 & 7)) << 4, sb = sa ^ 64;
        uint8_t* da = dst + (size_t)odd * kTc2HalfBytes + (size_t)r0 * 128;
        uint8_t* db = dst + (size_t)(odd ^ 1) * kTc2HalfBytes + (size_t)r0 * 128;
        const int x0 = ((2 * cl) ^ (r0 & 7)) << 4, x1 = x0 ^ 16;
        auto widened = [&](uint8_t* d, const uint4 w) {
          *reinterpret_cast<uint4*>(d + x0) = make_uint4(e4m3x2_to_f16x2<kSelB0B1>(w.x), e4m3x2_to_f16x2<kSelB2B3>(w.x),
                                                         e4m3x2_to_f16x2<kSelB0B1>(w.y), e4m3x2_to_f16x2<kSelB2B3>(w.y));
          *reinterpret_cast<uint4*>(d + x1) = make_uint4(e4m3x2_to_f16x2<kSelB0B1>(w.z), e4m3x2_to_f16x2<kSelB2B3>(w.z),
                                                         e4m3x2_to_f16x2<kSelB0B1>(w.w), e4m3x2_to_f16x2<kSelB2B3>(w.w));
        };
#pragma unroll 1
        for (int k = 0; k < TOK; k += 2 * kStep) {
          uint4 w[4];
#pragma unroll
          for (int i = 0; i < 2; ++i) {  // (rows beyond the stage's tokens: stale, cleared by the softmax threads)
            w[2 * i] = *reinterpret_cast<const uint4*>(s0 + (k + kStep * i) * 128 + sa);
            w[2 * i + 1] = *reinterpret_cast<const uint4*>(s0 + (k + kStep * i) * 128 + sb);
          }
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            widened(da + (k + kStep * i) * 128, w[2 * i]);
            widened(db + (k + kStep * i) * 128, w[2 * i + 1]);
          }
        }
        fence_proxy_async_smem();  // the widened slot is read by the MMAs through the async proxy
      }
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(s_wfull + 8 * (n % (2 * NW)));
        mbar_arrive(s_vtaken + 8 * vs);
      }
    }
    if (!ok && lane == 0) atomicOr(&p.hdr->status, kStatusWaitTimeout);
  } else {
    // ================================================================= softmax warps
    const int t = warp >> 2, w4 = warp & 3;           // pipeline; lane quarter of tensor memory
    const int r = 32 * w4 + lane;                     // this thread's token of the stage (and dim of the accumulator)
    const uint32_t tlane = tmem + ((uint32_t)(32 * w4) << 16);
    float4* cr = reinterpret_cast<float4*>(gen + (s_cr - base)) + t * (NC / 2);    // column pairs: two factors, two -references
    float* crf = reinterpret_cast<float*>(cr);
    auto cr_mul = [&](int c) -> float& { return crf[4 * (c >> 1) + (c & 1)]; };
    auto cr_ref = [&](int c) -> float& { return crf[4 * (c >> 1) + 2 + (c & 1)]; };
    float* wmax = reinterpret_cast<float*>(gen + (s_max - base)) + t * 4 * NC;     // [4 warps][NC]
    float* alpha_s = reinterpret_cast<float*>(gen + (s_alpha - base)) + t * NC;
    float ref_own = -INFINITY;                        // warp w4, lane l: reference of column 32 w4 + l
    constexpr int NCC = NC / 16;                      // columns are worked on 16 at a time
    uint32_t ph_wg = 0, ph_both = 0, par_vote = 0;
    bool ok = true;
    auto wg_sync = [&]() {
      __syncwarp();
      if (lane == 0) mbar_arrive(s_wg + 8 * t);
      const bool got = tok_wait(s_wg + 8 * t, ph_wg, s_abort);
      ph_wg ^= 1u;
      return got;
    };
    // Each pipeline's warps read the other's accumulators behind this: what the other's warps have waited for (its MMAs) or
    // stored (a rescaling) is ordered before these reads by their fence before the barrier and this one's behind it.
    auto both_sync = [&]() {
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(s_both);
      const bool got = tok_wait(s_both, ph_both, s_abort);
      tc_fence_after_sync();
      ph_both ^= 1u;
      return got;
    };
    // true in all threads of the pipeline when any thread's `yes` is; two sets of flags take turns
    bool vote_ok = true;
    auto wg_any = [&](bool yes) {
      volatile int* v = g_vote + t * 8 + par_vote * 4;
      const bool any = __any_sync(0xffffffffu, yes);
      if (lane == 0) v[w4] = any;
      vote_ok = wg_sync();
      const bool res = v[0] | v[1] | v[2] | v[3];
      par_vote ^= 1u;
      return res;
    };
    // ---- the end of a unit: the pipelines' partial results are merged and written.  It is put off until the next stage's
    // weights have been formed (which needs neither the weight buffer nor the accumulators), so that these run beside
    // the unit's last P.V.
    bool unit_open = false;               // a unit's results are still in the accumulators
    float e_ref = -INFINITY;              // reference of column 32 w4 + lane
    int e_slot = 0, e_b = 0, e_h = 0, e_nodes = 0, e_chunks = 1, e_unit = 0;
    auto finish_unit = [&]() {  // (after the wait for the unit's last P.V)
      unit_open = false;
      tc_fence_after_sync();
      float* refs = reinterpret_cast<float*>(gen + (s_ref - base)) + (e_unit & 1) * 2 * NC;
      if (32 * w4 + lane < NC) refs[t * NC + 32 * w4 + lane] = e_ref;
      if (!both_sync()) return false;
      const bool dst_ok = checked(chk_index(e_slot, p.max_items) && chk_index(e_b, p.B) && chk_index(e_h, p.Hkv),
                                  &p.hdr->status, kStatusBadIndex);
      const bool partial = e_chunks > 1 || p.out_f32;
      const int cols = p.G * e_nodes;  // (rows of nodes that do not exist are left alone)
#pragma unroll 1
      for (int g16 = t; 16 * g16 < min(NC, cols); g16 += 2) {  // 16 columns at a time, the pipelines' warps in turns; thread = dim
        uint32_t o0[16], o1[16];
        tmem_ld16(tlane + L::kColL + 16 * g16, o0);
        tmem_ld16(tlane + L::kColL + NC + 16 * g16, o1);
        // lane j: the common reference of column j, the pipelines' distances from it (0 where a pipeline's column saw
        // nothing: its accumulators may hold anything then, and are not used), and what their values are multiplied by
        const int cj = 16 * g16 + (lane & 15);
        const float m0 = refs[cj], m1 = refs[NC + cj], M = fmaxf(m0, m1), Ms = M == -INFINITY ? 0.f : M;
        float f0 = ex2(m0 - Ms), f1 = ex2(m1 - Ms), l0 = 0.f, l1 = 0.f;
        tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          l0 = (lane & 15) == j ? __uint_as_float(o0[j]) : l0;
          l1 = (lane & 15) == j ? __uint_as_float(o1[j]) : l1;
        }
        tmem_ld16(tlane + L::kColO + 16 * g16, o0);
        tmem_ld16(tlane + L::kColO + NC + 16 * g16, o1);
        const float den = (f0 != 0.f ? l0 * f0 : 0.f) + (f1 != 0.f ? l1 * f1 : 0.f), inv = den > 0.f ? p.v_scale / den : 0.f;
        if (partial && w4 == 0 && lane < 16 && cj < cols && (!kChecked || dst_ok))
          p.part_lse[(size_t)e_slot * p.GQ + cj] = den > 0.f ? M + lg2(den) : -INFINITY;
        f0 *= inv;
        f1 *= inv;
        tmem_ld_wait();
        float v[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const float b0 = __shfl_sync(0xffffffffu, f0, j), b1 = __shfl_sync(0xffffffffu, f1, j);
          v[j] = (b0 != 0.f ? __uint_as_float(o0[j]) * b0 : 0.f) + (b1 != 0.f ? __uint_as_float(o1[j]) * b1 : 0.f);
        }
        if (partial && (!kChecked || dst_ok)) {
          float* dst = p.part_o + ((size_t)e_slot * p.GQ + 16 * g16) * D + r;
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (16 * g16 + j < cols) dst[j * D] = v[j];
        } else if (!kChecked || dst_ok) {
          // two columns at a time: even lanes write two dims of the first, odd lanes of the second
          int qi = 16 * g16 / p.G, head = 16 * g16 - qi * p.G;
          __nv_bfloat16* const row0 = p.out + ((size_t)e_b * p.Sq * p.Hq + (size_t)e_h * p.G) * D + (r & ~1);
          const bool odd = lane & 1;
#pragma unroll
          for (int j = 0; j < 16; j += 2) {
            int q2 = qi, h2 = head;
            if (++h2 == p.G) {
              h2 = 0;
              ++q2;
            }
            const float got = __shfl_xor_sync(0xffffffffu, odd ? v[j] : v[j + 1], 1);
            const uint32_t w = odd ? pack_bf16x2(got, v[j + 1]) : pack_bf16x2(v[j], got);
            if (16 * g16 + j + (odd ? 1 : 0) < cols)
              *reinterpret_cast<uint32_t*>(row0 + ((size_t)(odd ? q2 : qi) * p.Hq + (odd ? h2 : head)) * D) = w;
            qi = q2;
            head = h2;
            if (++head == p.G) {
              head = 0;
              ++qi;
            }
          }
        }
        __syncwarp();  // the tensor-memory loads are warp-wide: reconverge before the next one
      }
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(s_ofree);
      return true;
    };
    for (uint32_t i = 0; ok; ++i) {
      const uint32_t n = 2 * i + t;
      const int ms = n % kTokMeta;
      if (!tok_wait(s_mfull + 8 * ms, (n / kTokMeta) & 1u, s_abort)) {
        ok = false;
        break;
      }
      const int4 meta = g_meta[2 * ms], meta2 = g_meta[2 * ms + 1];
      const bool end = meta.x < 0;
      const int ntok = end ? 0 : meta.w & 0xffff, b = meta.y, h = meta.z, tok0 = meta2.x, first_node = meta2.y, nodes = meta2.z;
      const bool first = !end && ((meta.w >> 16) & 1), last = !end && ((meta.w >> 17) & 1);
      if (first) ref_own = -INFINITY;
      // which columns see this thread's token: of a node's, those whose query token has the node's bit in its mask (at most 64
      // tokens, one word each; a lane fetches a word, while the scores are on their way)
      const bool tree = tok0 + ntok > first_node;  // the stage holds nodes
      uint32_t seen[2];
      seen[0] = seen[1] = r < ntok ? 0xffffffffu : 0u;
      if (tree) {
        const uint64_t* rows = p.tree_mask + (size_t)b * p.Sq;
        const uint64_t r0 = lane < p.Sq ? rows[lane] : 0ull, r1 = lane + 32 < p.Sq ? rows[lane + 32] : 0ull;
        const int node = tok0 + r - first_node;
        const uint64_t mine = (1ull << p.G) - 1ull;  // (G is at most 16, and qi * G below the 64 columns)
        uint64_t m = 0ull;
#pragma unroll 1
        for (int qi = 0; qi < p.Sq; ++qi) {
          const uint64_t row = __shfl_sync(0xffffffffu, qi < 32 ? r0 : r1, qi & 31);
          if ((row >> (node & 63)) & 1ull) m |= mine << (qi * p.G);
        }
        if (r < ntok && node >= 0) {
          seen[0] = (uint32_t)m;
          seen[1] = (uint32_t)(m >> 32);
        }
      }
      const uint32_t sb = i % SB, sfree = s_sfree + 8 * (2 * t + sb);
      if (!end && !tok_wait(s_sready + 8 * (2 * t + sb), (i / SB) & 1u, s_abort)) {
        ok = false;
        break;
      }
      const uint32_t srow = tlane + (uint32_t)(t * SB + sb) * NC;
      const bool quick = !tree && ntok > 32 * (NCC - 1);
      bool refs_due = tree || (first && !quick);
      const bool masked = tree || ntok < TOK;
      auto hide = [&](int cc, uint32_t (&s)[16]) {  // scores of 16 columns: -inf where the token is hidden
        const uint32_t m = (cc >> 1 ? seen[1] : seen[0]) >> (16 * (cc & 1));
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (!((m >> j) & 1u)) s[j] = 0xff800000u;
      };
      if (ntok > 0) {
        tc_fence_after_sync();
        if (first) {
          // The columns' factors and first references.  Any value near the scores will do as a reference: those of one token,
          // warp w's first for columns 16 w ..  (Stages with nodes or few tokens form the maxima below, which replace a
          // reference of -inf.)
          if (KV8 && !tok_wait(s_qready, (uint32_t)meta2.w & 1u, s_abort)) {
            ok = false;
            break;
          }
          const float* mul = reinterpret_cast<const float*>(gen + (s_mul - base));
          if (w4 < NCC) {
            uint32_t s[16];
            tmem_ld16(srow + 16 * w4, s);
            tmem_ld_wait();
            if (lane == 0) {
#pragma unroll
              for (int j = 0; j < 16; j += 2) {
                float2 f = KV8 ? *reinterpret_cast<const float2*>(mul + 16 * w4 + j) : make_float2(p.scale_log2e, p.scale_log2e);
                // (a factor that underflows to zero, of tiny queries or a tiny scale, would make NaN of hidden scores, -inf)
                f.x = fmaxf(f.x, 1.17549435e-38f);
                f.y = fmaxf(f.y, 1.17549435e-38f);
                cr[8 * w4 + j / 2] = make_float4(f.x, f.y, quick ? -__uint_as_float(s[j]) * f.x : 0.f,
                                                 quick ? -__uint_as_float(s[j + 1]) * f.y : 0.f);
              }
            }
          }
          if (!wg_sync()) {
            ok = false;
            break;
          }
          if (quick && 32 * w4 + lane < NC) ref_own = -cr_ref(32 * w4 + lane);
          if (w4 == 0 && lane == 0) mbar_arrive(s_qfree);
        }
      }
      // The weight buffer has to be free, and the accumulators complete where they are touched: the P.V of the pipeline's
      // stage before is complete.
      if (i > 0 && !tok_wait(s_pvdone + 8 * t, (i - 1) & 1u, s_abort)) {
        ok = false;
        break;
      }
      uint8_t* prow = gen + (s_p - base) + (size_t)t * L::kPBytes + (size_t)r * 128;  // this token's weights
      for (bool formed = ntok == 0, raised = false;;) {
        if (!formed && !refs_due) {
          // ---- weights: 2^(score * factor - reference), into the second MMAs' operand
          float top = -INFINITY;  // largest exponent
          uint32_t nxt[16];
          tmem_ld16(srow, nxt);
#pragma unroll
          for (int cc = 0; cc < NCC; ++cc) {
            uint32_t s[16];
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 16; ++j) s[j] = nxt[j];
            if (cc + 1 < NCC) tmem_ld16(srow + 16 * (cc + 1), nxt);
            if (masked) hide(cc, s);
            uint32_t pw[8];
#pragma unroll
            for (int j = 0; j < 16; j += 2) {
              const float4 f = cr[8 * cc + j / 2];  // two columns' factors and -references
              const float2 x = ffma2(make_float2(__uint_as_float(s[j]), __uint_as_float(s[j + 1])), make_float2(f.x, f.y),
                                     make_float2(f.z, f.w));
              top = fmax3(top, x.x, x.y);
              pw[j / 2] = KV8 ? pack_f16x2(ex2(x.x), ex2(x.y)) : pack_bf16x2(ex2(x.x), ex2(x.y));
            }
            *reinterpret_cast<uint4*>(prow + (((2 * cc) ^ (r & 7)) << 4)) = make_uint4(pw[0], pw[1], pw[2], pw[3]);
            *reinterpret_cast<uint4*>(prow + (((2 * cc + 1) ^ (r & 7)) << 4)) = make_uint4(pw[4], pw[5], pw[6], pw[7]);
          }
          refs_due = wg_any(top > kTokRaise<KV8> && !raised);  // (once: the rounding of the two comparisons may differ)
          if (!vote_ok) {
            ok = false;
            break;
          }
          formed = !refs_due;
          if (formed) {  // the score buffer is free
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(sfree);
          }
        }
        if (unit_open && !finish_unit()) {  // a unit that ended is written now
          ok = false;
          break;
        }
        if (formed) break;
        // ---- references: the columns' maxima over the stage, of the warp's tokens, then of the warps
        tc_fence_after_sync();
#pragma unroll 1
        for (int cc = 0; cc < NCC; ++cc) {
          uint32_t s[16];
          tmem_ld16(srow + 16 * cc, s);
          tmem_ld_wait();
          if (masked) hide(cc, s);
          float m[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) m[j] = __uint_as_float(s[j]);
#pragma unroll
          for (int o = 16, n8 = 8; o > 1; o >>= 1, n8 >>= 1) {
            const bool up = lane & o;
#pragma unroll
            for (int j = 0; j < n8; ++j) {
              const float keep = up ? m[j + n8] : m[j], send = up ? m[j] : m[j + n8];
              m[j] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, send, o));
            }
          }
          m[0] = fmaxf(m[0], __shfl_xor_sync(0xffffffffu, m[0], 1));
          if (!(lane & 1)) wmax[w4 * NC + 16 * cc + (lane >> 1)] = m[0];
        }
        if (!wg_sync()) {
          ok = false;
          break;
        }
        bool changed = false;
        if (32 * w4 + lane < NC) {
          const int c = 32 * w4 + lane;
          const float* mx = wmax + c;
          const float m = fmaxf(fmaxf(mx[0], mx[NC]), fmaxf(mx[2 * NC], mx[3 * NC])) * cr_mul(c);
          float a = 1.f;
          if (ref_own == -INFINITY) {
            ref_own = m;  // nothing accumulated for this column so far
          } else if (m > ref_own + kTokRaise<KV8>) {
            a = first ? 1.f : ex2(ref_own - m);
            ref_own = m;
            changed = !first;  // (on the unit's first stage nothing has been accumulated)
          }
          cr_ref(c) = ref_own == -INFINITY ? 0.f : -ref_own;
          alpha_s[c] = a;
        }
        const bool rescale = wg_any(changed);
        if (!vote_ok) {
          ok = false;
          break;
        }
        if (rescale) {
#pragma unroll 1
          for (int g16 = 0; g16 < 2 * NCC; ++g16) {  // values, then sums
            const int c0 = 16 * (g16 < NCC ? g16 : g16 - NCC);
            const uint32_t at = tlane + (g16 < NCC ? L::kColO : L::kColL) + (uint32_t)(t * NC + c0);
            uint32_t o[16];
            tmem_ld16(at, o);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * alpha_s[c0 + j]);
            tmem_st16(at, o);
          }
          tmem_st_wait();
          if (!wg_sync()) {  // everybody has read alpha
            ok = false;
            break;
          }
        }
        refs_due = false;
        raised = true;
      }
      if (!ok || end) break;
      if (ntok > 0) {
        if (ntok < TOK) {
          // V rows beyond the stage's tokens may hold anything (NaN included): clear them once the slot is written
          constexpr int ring = KV8 ? NW : NV;
          const int vs = n % ring;
          if (!tok_wait((KV8 ? s_wfull : s_vland) + 8 * (n % (2 * ring)), (n / (2 * ring)) & 1u, s_abort)) {
            ok = false;
            break;
          }
          if (r >= ntok) {
            uint8_t* vrow = gen + ((KV8 ? s_w : s_v) - base) + (size_t)vs * kTc2SlotBytes + (size_t)r * 128;
#pragma unroll
            for (int c = 0; c < 16; ++c)
              *reinterpret_cast<uint4*>(vrow + (size_t)(c >> 3) * kTc2HalfBytes + ((c & 7) << 4)) = make_uint4(0u, 0u, 0u, 0u);
          }
        }
        fence_proxy_async_smem();  // the weights (and cleared rows) are read by the MMAs through the async proxy
        tc_fence_before_sync();
      } else {
        if (first && w4 == 0 && lane == 0) mbar_arrive(s_qfree);
        if (lane == 0) mbar_arrive(sfree);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(s_pready + 8 * t);

      if (last) {  // the rest of the unit's work is put off (finish_unit)
        unit_open = true;
        e_slot = meta.x;
        e_b = b;
        e_h = h;
        e_nodes = nodes;
        e_unit = meta2.w;
        e_chunks = chk_index(b, p.B) ? p.seq_first[b + 1] - p.seq_first[b] : 1;
        e_ref = ref_own;
      }
    }
    if (!ok && lane == 0) atomicOr(&p.hdr->status, kStatusWaitTimeout);
  }
  // ---- common exit: release the tensor memory once every warp is done with it
  tc_fence_before_sync();
  __syncthreads();
  if (warp == kWarpM) tmem_dealloc(tmem, L::kTmemCols);
}

}  // namespace ooco
