// Attention of drafted trees' columns over the 4-bit pool on the fifth-generation tensor cores (bf16 queries).
//
// The mathematics, the orientation of both products and the expansion of the codes into tensor memory are those of
// qpool_attn_tc.cuh; what differs is that a tree brings many columns (nodes times heads) to the same slots, so that
// an expanded tile is used by NC = 64 of them instead of one sequence's heads (32 where a request has no more).  Per tile
// of 128 slots and r 512 the matrix unit needs 68 x 32 = 2180 cycles; what bounds the kernel is the issue of
// instructions: 16100 a tile (expansion, softmax, the bookkeeping of both) are 4000 cycles of the four schedulers, and
// a tile takes about 5400.  Eight requests of 64 nodes and 32 heads over 4096 slots: 204 us by itself, cold (the whole
// call takes 226, its launches overlap), where products at the measured rate of large ones would take 88.
//
// Tensor memory holds the output sums (r / 128 blocks of NC columns), one or two score tiles and operand units of 32
// columns: 64 latents of the 128 slots for the scores, or 64 slots of 128 latents for the values.  Units half as wide as
// there leave three buffers for each product beside 64 columns of r 512.
//
// Groups of columns take the place of sequences; a group's result is always a part (reference, denominator, sums in 32
// bits) that the join kernels put together with the drafted rows.  Roles (28 warps): warp 0 issues the score products,
// warp 1 the value products, warp 2 fetches the pages, warp 3 the queries; warps 4-11 expand for the scores, warps 12-19
// for the values, and write the results; warps 20-27 are softmax.  Measured on the way (the same eight requests): expanding
// warps of their own for either product 246 -> 237 us of this kernel; waits and indices of a tile outside the units'
// loop 238 -> 221; probabilities handed over in halves, queries laid out ahead and results written by the value
// warps 221 -> 212; issuing warps that ask before they wait 254 -> 245 of the whole call.  Twelve value warps instead
// of eight leave 56 registers a thread and spill more (232 us for 221; as it is, 64 columns spill 84 to 168 bytes a thread); reading a unit's bytes ahead costs more instructions
// than it hides (256 for 243).  Every wait is bounded as there.
#pragma once

#include "qpool_attn_tc.cuh"
#include "tree_kernels.cuh"

namespace mtla {
namespace tree {

constexpr int kTile = 128, kThreads = 896;
constexpr int kScoreIssuer = 0, kValueIssuer = 1, kProducerWarp = 2, kQueryWarp = 3;
constexpr int kScoreWarp0 = 4, kScoreWarps = 8, kValueWarp0 = 12, kValueWarps = 8;
constexpr int kSoftmaxWarp0 = 20, kSoftmaxThreads = 256, kSoftmaxWarps = 8;
// Registers of a thread of the issuing, expanding and softmax warps, and of all warps together.
constexpr int kIssueRegs = 40, kExpandRegs = 64, kSoftmaxRegs = 104;
constexpr int kRoleRegisters = 4 * kIssueRegs + (kScoreWarps + kValueWarps) * kExpandRegs + 8 * kSoftmaxRegs;
static_assert(kRoleRegisters <= 72 * (kThreads / 32), "there are 72 registers for each of 896 threads");
constexpr int kQRing = qp::tc::kQRing, kInfo = 16, kUnitRing = 8, kMaxStages = 4;
// Barriers for the ends of segments: a phase must not complete twice before the value warps have looked at it.  When the
// softmax warps end segment s, products of the tile two before its last one have been issued; that is a tile of segment
// s - 2 or later, for which the value warps had to be done with the segment in front of it: of segments of one
// tile s - 3, and no later one.  So three at least.  (end_fac is used by segments of over 128 tiles only.)
constexpr int kEndRing = 4;
constexpr float kShift = qp::tc::kShift, kRescale = qp::tc::kRescale;
constexpr int kFoldTiles = qp::tc::kFoldTiles;
constexpr int kFirst = 1, kLast = 2, kFold = 4, kFolded = 8, kFoldedNow = 16, kEnds = 32, kSegShift = 6;

// Tensor memory for NC columns and NB blocks of 128 latents.
template <int NC, int NB>
struct Tmem {
  static constexpr int kScores = (2 + NB) * NC + 6 * 32 <= 512 ? 2 : 1;        // score tiles
  static constexpr int kLeft = (512 - (kScores + NB) * NC) / 64;
  static constexpr int kUnits = kLeft < 4 ? kLeft : 4;                         // buffers for each product
  static constexpr int kColS = 0, kColO = kScores * NC, kColAs = kColO + NB * NC, kColAv = kColAs + 32 * kUnits;
  static_assert(kUnits >= 3 && kColAv + 32 * kUnits <= 512, "tensor memory budget");
};

struct TileInfo {
  int group, flags;          // flags: the above; the segment's number times 64
  int rows0, rows1;          // slots of the tile's two pages
  int cols, owner;           // columns of the group, the CTA of its first tile
};

struct Misc {
  unsigned long long code_full[kMaxStages], code_empty[kMaxStages], scale_full[kMaxStages];
  unsigned long long key_full[2], key_empty[2];
  unsigned long long as_full[kUnitRing], as_empty[kUnitRing], av_full[kUnitRing], av_empty[kUnitRing];
  unsigned long long s_full[2], s_empty[2], p_full[4], p_empty[4];       // a probability tile: each half of the slots
  unsigned long long q_full[kQRing], q_empty[kQRing];
  unsigned long long end_full[kEndRing], o_full[2], o_empty;
  unsigned long long info_full[kInfo];
  uint32_t tmem_base;
  int abort_word;
  TileInfo info[kInfo];
  float m_used[64];
  alignas(16) float neg_ref[64];
  alignas(16) float unit[64];
  alignas(16) float next_unit[kQRing][64];
  float fac[64], down[64];
  float red[8][32];
  float m_fold[64], end_fac[2][64];
};
constexpr int kMiscBytes = 5632;
static_assert(kEndRing <= kMaxStages && kQRing <= kMaxStages, "barriers that are set up side by side");
static_assert(sizeof(Misc) <= kMiscBytes, "misc region too small");

struct Layout {
  int scales, stage, stages, key_stage, key_stages, p_bytes, p_stages, scale_room;
  int off_codes, off_keys, off_q, off_p, off_st, off_misc, total;
  __host__ __device__ Layout(const qp::Format& f, int nc) {
    scales = kTile * f.code_row();
    stage = (scales + kTile * f.scale_row() + 127) / 128 * 128;
    key_stage = kTile * f.key_row();
    scale_room = f.scale_row() * kTile * 2;
    p_bytes = kTile * nc * 2;
    const int q_room = (nc * 2 * (f.r + f.dr) + 1023) / 1024 * 1024;
    const int room = qp::tc::kSmemMax - kMiscBytes - 1024 - q_room;
    // Three stages of codes in any shape (the expansion's waits rely on them), then a second key stage and
    // probability tile, then the fourth.
    key_stages = p_stages = 1;
    stages = 3;
    auto used = [&]() { return stages * (stage + scale_room) + key_stages * key_stage + p_stages * p_bytes; };
    if (used() + key_stage <= room) key_stages = 2;
    if (used() + p_bytes <= room) p_stages = 2;
    if (used() + stage + scale_room <= room) stages = 4;
    off_keys = 0;                                           // swizzled operands: 1024-byte aligned
    off_q = off_keys + key_stages * key_stage;
    off_p = off_q + q_room;
    off_codes = off_p + p_stages * p_bytes;
    off_st = off_codes + stages * stage;
    off_misc = (off_st + stages * scale_room + 15) / 16 * 16;
    total = off_misc + kMiscBytes + 1024;
  }
};

// Codes of four latents of two neighbouring slots -> a pair (slot, next slot) of each latent: a thread's register of the
// transposing load holds codes (4g .. 4g + 3) of slot 2t in its low half and of slot 2t + 1 in its high half.
__device__ __forceinline__ void decode_pairs(uint32_t w, uint32_t (&o)[4]) {
  uint32_t e, d;                               // latents 0, 2 and 1, 3 in the two low bytes, the next slot's above
  asm("lop3.b32 %0, %1, %2, %3, 0xe4;" : "=r"(e) : "r"(w), "r"(w >> 12), "n"(0x0f0f));
  asm("lop3.b32 %0, %1, %2, %3, 0xe4;" : "=r"(d) : "r"(w >> 4), "r"(w >> 16), "n"(0x0f0f));
  asm("{\n\t.reg .b8 a, b, c, d, x, y;\n\t"
      "mov.b32 {a, b, x, y}, %4;\n\t"
      "mov.b32 {c, d, x, y}, %5;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3])
      : "r"(e), "r"(d));
}

// A segment's output sums, this thread's latent of every block (lane 8j + g of a quarter holds latent 4g + j), into
// the segment's part [NC][128 NB], shared out among STEP groups of four warps in pieces of 16 columns of a block: added to
// what has been set down there, which `fac` brings to the present references, or without `add` as they are.
template <int NC, int NB, int STEP>
__device__ __forceinline__ void set_down(float* part, uint32_t taddr, const float* fac, bool add, int cols, int r, int lat,
                                         int grp) {
#pragma unroll 1
  for (int i = grp; i < NB * (NC / 16); i += STEP) {
    const int mb = i / (NC / 16), c0 = i % (NC / 16) * 16, row = mb * 128 + lat;
    uint32_t o[16];
    ptx::tmem_ld_x16(taddr + mb * NC + c0, o);
    ptx::tmem_wait_ld();
    if (row >= r) continue;
    constexpr int kRow = 128 * NB;             // a column's place in a part: every store has a constant offset
    float* dst = part + c0 * kRow + row;
    if (add) {
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (c0 + j < cols) o[j] = __float_as_uint(fmaf(dst[j * kRow], fac[c0 + j], __uint_as_float(o[j])));
    }
    if (c0 + 16 <= cols) {
#pragma unroll
      for (int j = 0; j < 16; ++j) dst[j * kRow] = __uint_as_float(o[j]);
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (c0 + j < cols) dst[j * kRow] = __uint_as_float(o[j]);
    }
  }
}

template <int NC, int NB>
__global__ void __launch_bounds__(kThreads, 1) tree_attend_tc_kernel(qp::GroupArgs a, Layout L) {
  using namespace ptx;
  using T = Tmem<NC, NB>;
  constexpr uint32_t IDESC_S = make_idesc_f16(128, NC, 0, 0), IDESC_K = make_idesc_bf16(128, NC, 0, 0);
  constexpr uint32_t IDESC_V = make_idesc_f16(128, NC, 0, 1);
  constexpr uint32_t P_SBO = kTile * 16;        // bytes between groups of 8 columns of a probability tile
  constexpr int U = 2 * NB, SB = T::kScores, BUFS = T::kUnits;
  extern __shared__ uint8_t smem_raw[];
  const qp::Format f = a.f;
  const int r = f.r, dr = f.dr;
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* sm = smem_raw + (base - raw);
  Misc* misc = reinterpret_cast<Misc*>(sm + L.off_misc);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;   // warp: uniform
  auto bar = [&](unsigned long long& p) { return smem_u32(&p); };

  if (threadIdx.x < kInfo) {
    const int i = threadIdx.x;
    mbar_init(bar(misc->info_full[i]), 1);
    if (i < kUnitRing) {
      mbar_init(bar(misc->as_full[i]), 4);
      mbar_init(bar(misc->as_empty[i]), 1);
      mbar_init(bar(misc->av_full[i]), 4);
      mbar_init(bar(misc->av_empty[i]), 1);
    }
    if (i < kMaxStages) {
      mbar_init(bar(misc->p_full[i]), kSoftmaxWarps / 2);
      mbar_init(bar(misc->p_empty[i]), 1);
      mbar_init(bar(misc->code_full[i]), 1);
      mbar_init(bar(misc->code_empty[i]), kScoreWarps + kValueWarps);
      mbar_init(bar(misc->scale_full[i]), kScoreWarps);
      mbar_init(bar(misc->end_full[i]), kSoftmaxWarps);
      mbar_init(bar(misc->q_full[i]), 1);
      mbar_init(bar(misc->q_empty[i]), 1);
    }
    if (i < 2) {
      mbar_init(bar(misc->key_full[i]), 1);
      mbar_init(bar(misc->key_empty[i]), 1);
      mbar_init(bar(misc->s_full[i]), 1);
      mbar_init(bar(misc->s_empty[i]), kSoftmaxWarps);
      mbar_init(bar(misc->o_full[i]), 1);
    }
    if (i == 0) mbar_init(bar(misc->o_empty), kValueWarps);
    if (i == 0) misc->abort_word = 0;
    mbar_fence_init();
  }
  if (warp == kProducerWarp) tmem_alloc(smem_u32(&misc->tmem_base), 512);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  constexpr uint32_t tmem = 0;                  // all columns are this CTA's
  grid_launch_dependents();
  grid_dependency_wait();

  const int* const prefix = a.prefix;
  const int4 share = a.shares[blockIdx.x];      // first tile, tiles, the first one's group, that group's first CTA
  const int g0 = share.x, g1 = share.x + share.y;
  const int n_tiles = __shfl_sync(0xffffffffu, share.y, 0);      // uniform
  const uint32_t q_u32 = base + L.off_q, p_u32 = base + L.off_p, st_u32 = base + L.off_st;
  auto wait = [&](unsigned long long& b, int phase) { return mbar_wait_compact(bar(b), phase & 1); };
  auto wait_warp = [&](unsigned long long& b, int phase) {                 // one answer for the warp
    return mbar_wait_eager(bar(b), phase & 1);
  };
  bool ok = true;                // false once a wait of this thread has given up
  if (threadIdx.x == 0 && misc->tmem_base != 0) misc->abort_word = 1;

  if (n_tiles == 0) {
    // nothing to do; the CTA falls through to the common end
  } else if (warp < kScoreWarp0) {
    reg_dealloc<kIssueRegs>();
    if (warp == kProducerWarp) {
      // ---------------------------------------------------------------- producer
      int v = share.z, seg = -1, st = 0, round = 0, begun = 0;
      if (lane == 0) {
        int v_begin = prefix[v], v_end = prefix[v + 1];
        int4 group = a.groups[v];
        for (int n = 0; n < n_tiles; ++n) {
          const int g = g0 + n;
          while (v_end <= g) {
            ++v;
            v_begin = v_end;
            v_end = prefix[v + 1];
            group = a.groups[v];
          }
          const int tile = g - v_begin;
          const bool first = n == 0 || tile == 0, ends = g + 1 == v_end, last = n + 1 == n_tiles || ends;
          int page[2], rows[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int t = 2 * tile + i, have = group.w - t * qp::kPageRows;
            page[i] = have > 0 && t < a.width ? __ldg(a.table + (long long)group.x * a.width + t) : -1;
            rows[i] = page[i] >= 0 && page[i] < a.n_pages ? min(have, qp::kPageRows) : 0;
          }
          ok = wait(misc->code_empty[st], round + 1);
          if (!ok) break;
          TileInfo& info = misc->info[n % kInfo];
          seg += first;
          if (first) begun = n;
          const int before = n - begun;
          info.group = v;
          info.flags = (first ? kFirst : 0) | (last ? kLast : 0) | (ends ? kEnds : 0) |
                       (before && before % kFoldTiles == 0 ? kFold : 0) | (before > kFoldTiles ? kFolded : 0) |
                       (before >= kFoldTiles ? kFoldedNow : 0) | seg << kSegShift;
          info.rows0 = rows[0];
          info.rows1 = rows[1];
          info.cols = group.z;
          info.owner = v == share.z ? share.w : (int)blockIdx.x;
          mbar_arrive(bar(misc->info_full[n % kInfo]));
          const uint32_t full = bar(misc->code_full[st]), dst = base + L.off_codes + st * L.stage;
          const uint8_t* src[2];
          uint32_t bytes = 0;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            src[i] = a.pages + (rows[i] ? (long long)page[i] * f.page_bytes() : 0);
            bytes += rows[i] * f.code_row() + (rows[i] * f.scale_row() + 15) / 16 * 16;
          }
          mbar_arrive_expect_tx(full, bytes);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (rows[i] == 0) continue;
            bulk_load(dst + L.scales + i * qp::kPageRows * f.scale_row(), src[i] + f.off_scales(),
                      (rows[i] * f.scale_row() + 15) / 16 * 16, full);
            bulk_load(dst + i * qp::kPageRows * f.code_row(), src[i], rows[i] * f.code_row(), full);
          }
          const int ks = L.key_stages == 2 ? n & 1 : 0, key_round = L.key_stages == 2 ? n >> 1 : n;
          ok = wait(misc->key_empty[ks], key_round + 1);
          if (!ok) break;
          const uint32_t key_bar = bar(misc->key_full[ks]), key_dst = base + L.off_keys + ks * L.key_stage;
          mbar_arrive_expect_tx(key_bar, (rows[0] + rows[1]) * f.key_row());
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (rows[i]) bulk_load(key_dst + i * qp::kPageRows * f.key_row(), src[i] + f.off_keys(), rows[i] * f.key_row(), key_bar);
          if (++st == L.stages) { st = 0; ++round; }
        }
      }
    } else if (warp == kQueryWarp) {
      // ---------------------------------------------------------------- queries of every segment
      int v = share.z;
      if (lane == 0) {
        for (int seg = 0, g = g0; g < g1; ++seg) {
          if (seg > 0)
            while (prefix[v + 1] <= g) ++v;
          ok = seg == 0 || wait(misc->q_empty[(seg - 1) % kQRing], (seg - 1) / kQRing);
          if (!ok) break;
          const uint8_t* src = a.image + (long long)v * image_bytes(NC, f);
          const uint32_t full = bar(misc->q_full[seg % kQRing]), rows = NC * 2 * (r + dr);
          mbar_arrive_expect_tx(full, rows + NC * 4);
          bulk_load(q_u32, src, rows, full);
          bulk_load(smem_u32(misc->next_unit[seg % kQRing]), src + rows, NC * 4, full);
          g = prefix[v + 1];
        }
      }
    } else if (warp == kScoreIssuer) {
      // ---------------------------------------------------------------- score products (whole warp, uniform)
      const uint64_t mode = dr == 64 ? kSwizzle128B : kSwizzle64B;
      const uint32_t key_sbo = 8 * f.key_row();
      const uint64_t q_desc = make_smem_desc(q_u32, 16, 1024, kSwizzle128B);
      const uint64_t qk_desc = make_smem_desc(q_u32 + NC * 2 * r, 16, key_sbo, mode);
      int buf = 0;
      bool there = false;            // the next unit, asked for before the instructions in front of it are issued
      for (int n = 0; n < n_tiles && ok; ++n) {
        const int ks = L.key_stages == 2 ? n & 1 : 0, key_round = L.key_stages == 2 ? n >> 1 : n;
        ok = wait_warp(misc->key_full[ks], key_round);
        if (!ok) break;
        const int flags = misc->info[n % kInfo].flags, seg = flags >> kSegShift;
        if (flags & kFirst) {
          ok = wait_warp(misc->q_full[seg % kQRing], seg / kQRing);
          if (!ok) break;
        }
        ok = wait_warp(misc->s_empty[n % SB], n / SB + 1);
        if (!ok) break;
        tc_fence_after_sync();
        const uint32_t d = tmem + T::kColS + (n % SB) * NC;
        const uint64_t key_desc = make_smem_desc(base + L.off_keys + ks * L.key_stage, 16, key_sbo, mode);
        if (elect_one()) {                               // RoPE part: d_R / 16 is 2 or 4
          mma_bf16_ss(d, key_desc, qk_desc, IDESC_K, 0u);
          mma_bf16_ss(d, key_desc + 2, qk_desc + 2, IDESC_K, 1u);
          if (dr == 64) {
            mma_bf16_ss(d, key_desc + 4, qk_desc + 4, IDESC_K, 1u);
            mma_bf16_ss(d, key_desc + 6, qk_desc + 6, IDESC_K, 1u);
          }
          mma_commit(bar(misc->key_empty[ks]));
        }
        __syncwarp();
#pragma unroll 1
        for (int p = 0; p < U; ++p) {
          const int k = n * U + p;
          ok = __all_sync(0xffffffffu, there) || wait_warp(misc->as_full[k % kUnitRing], k / kUnitRing);
          if (!ok) break;
          there = mbar_test(bar(misc->as_full[(k + 1) % kUnitRing]), (k + 1) / kUnitRing & 1);
          tc_fence_after_sync();
          const uint32_t at = tmem + T::kColAs + buf * 32;
          const uint32_t panel = (uint32_t)q_desc + p * NC * 8, hi = (uint32_t)(q_desc >> 32);
          if (elect_one()) {
            if (p * 64 < r) {
#pragma unroll
              for (int i = 0; i < 4; ++i) mma_f16_ts(d, at + i * 8, panel + i * 2, hi, IDESC_S, 1u);
            }
            mma_commit(bar(misc->as_empty[k % kUnitRing]));
          }
          __syncwarp();
          if (++buf == BUFS) buf = 0;
        }
        if (!ok) break;
        if (elect_one()) {
          mma_commit(bar(misc->s_full[n % SB]));
          if (flags & kLast) mma_commit(bar(misc->q_empty[seg % kQRing]));
        }
        __syncwarp();
      }
    } else if (warp == kValueIssuer) {
      // ---------------------------------------------------------------- value products (whole warp, uniform)
      const uint64_t p_desc = make_smem_desc(p_u32, 128, P_SBO, kSwizzleNone);
      int buf = 0;
      bool there = false;
      for (int n = 0; n < n_tiles && ok; ++n) {
        const int ps = L.p_stages == 2 ? n & 1 : 0, p_round = L.p_stages == 2 ? n >> 1 : n;
        ok = wait_warp(misc->p_full[2 * ps], p_round);
        if (!ok) break;
        tc_fence_after_sync();
        const int flags = misc->info[n % kInfo].flags, seg = flags >> kSegShift;
        const uint32_t fresh = (flags & (kFirst | kFold)) != 0;
        if ((flags & kFirst) && seg > 0) {               // the segment before has left the accumulators
          ok = wait_warp(misc->o_empty, seg - 1);
          if (!ok) break;
          tc_fence_after_sync();
        }
        const uint32_t pd = (uint32_t)p_desc + ps * (L.p_bytes / 16), hi = (uint32_t)(p_desc >> 32);
#pragma unroll 1
        for (int p = 0; p < U; ++p) {
          const int k = n * U + p, h = p >= NB ? 1 : 0, mb = p - h * NB;
          if (p == NB) {                                 // the first half's products are issued
            if (elect_one()) mma_commit(bar(misc->p_empty[2 * ps]));
            __syncwarp();
            ok = wait_warp(misc->p_full[2 * ps + 1], p_round);
            if (!ok) break;
          }
          ok = __all_sync(0xffffffffu, there) || wait_warp(misc->av_full[k % kUnitRing], k / kUnitRing);
          if (!ok) break;
          there = mbar_test(bar(misc->av_full[(k + 1) % kUnitRing]), (k + 1) / kUnitRing & 1);
          tc_fence_after_sync();
          const uint32_t d = tmem + T::kColO + mb * NC, at = tmem + T::kColAv + buf * 32;
          if (elect_one()) {
            mma_f16_ts(d, at, pd + h * 64, hi, IDESC_V, h ? 1u : fresh ^ 1u);
#pragma unroll
            for (int i = 1; i < 4; ++i) mma_f16_ts(d, at + i * 8, pd + h * 64 + i * 16, hi, IDESC_V, 1u);
            mma_commit(bar(misc->av_empty[k % kUnitRing]));
          }
          __syncwarp();
          if (++buf == BUFS) buf = 0;
        }
        if (ok && elect_one()) {
          mma_commit(bar(misc->p_empty[2 * ps + 1]));
          if (flags & kLast) mma_commit(bar(misc->o_full[seg & 1]));
        }
        __syncwarp();
      }
    }
  } else if (warp < kSoftmaxWarp0) {
    // ------------------------------------------------------------------ expansion
    // Groups of four warps, two for either operand, so that the scores' units never wait behind a value unit whose
    // buffer waits for the probabilities.  A group takes every second unit, decoded into registers before its buffer is
    // waited for.  What a tile needs once, waits, arrivals and addresses, is outside the units' loop: inside, it was a
    // third of all instructions.
    reg_dealloc<kExpandRegs>();
    constexpr int VG = kValueWarps / 4;
    const bool scores_role = warp < kValueWarp0;
    const int q = warp & 3, grp = (warp - (scores_role ? kScoreWarp0 : kValueWarp0)) >> 2, t = lane & 3;
    const int chunks = r / qp::kGroup, code_row = f.code_row();
    const uint32_t lane_tm = tmem + ((uint32_t)(q * 32) << 16);
    const uint32_t twist = (uint32_t)(lane & f.code_mask()) * 16;     // rows lane, lane + 32, ... twist alike
    int st = 0, round = 0, buf = grp % BUFS, k = grp;
    // The unit that had unit k's buffer has been used; a whole-warp answer.
    auto buffer_free = [&](unsigned long long* empty) {
      const int u = k - BUFS;
      return u < 0 || mbar_wait_eager<1>(smem_u32(empty) + (u % kUnitRing) * 8, u / kUnitRing & 1);
    };
    auto next_unit = [&](int step) {
      k += step;
      buf += step;
      if (buf >= BUFS) buf -= BUFS;
    };
    if (scores_role) {
      const int slot = q * 32 + lane, row = slot & 63;
#pragma unroll 1
      for (int n = 0; n < n_tiles && ok; ++n) {
        ok = mbar_wait_eager<1>(bar(misc->code_full[st]), round & 1);
        if (!ok) break;
        const TileInfo& info = misc->info[n % kInfo];
        const uint32_t live = row < (slot < 64 ? info.rows0 : info.rows1) ? 0xffffffffu : 0u;
        const uint32_t stage = base + L.off_codes + st * L.stage, codes = stage + slot * code_row;
        uint32_t scale_at = stage + L.scales + slot * f.scale_row() + 2 * grp;
        uint32_t st_out = st_u32 + st * L.scale_room + slot * 2 + 2 * grp * (kTile * 2);
        uint32_t code_at = 32 * grp;
#pragma unroll 1
        for (int i = 0; i < NB; ++i, next_unit(2), scale_at += 4, st_out += 8 * kTile, code_at += 64) {
          const bool there = code_at < (uint32_t)code_row;       // the last unit of a half block is empty
          uint32_t x[32];
          if (there) {
            const uint4 w0 = qp::lds128(codes + (code_at ^ twist)), w1 = qp::lds128(codes + ((code_at + 16) ^ twist));
            uint32_t two;
            asm volatile("{\n\t.reg .u16 x;\n\tld.shared.u16 x, [%1];\n\tcvt.u32.u16 %0, x;\n\t}"
                         : "=r"(two) : "r"(scale_at));
            // The scales also go out as half precision, a group's 128 slots in a row, for the value units;
            // zero where there is no slot, so that whatever its codes are, the product is zero.
            const uint32_t s01 = __byte_perm(two, 0, 0x4140) << 7, out = s01 & live;      // both as half precision
            asm volatile("st.shared.u16 [%0], %1;" ::"r"(st_out), "h"((uint16_t)out) : "memory");
            asm volatile("st.shared.u16 [%0], %1;" ::"r"(st_out + kTile * 2), "h"((uint16_t)(out >> 16)) : "memory");
            const uint32_t sc0 = __byte_perm(s01, 0, 0x1010), sc1 = __byte_perm(s01, 0, 0x3232);
            const uint32_t word[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              uint32_t o[4];
              qp::decode8(word[e], o);
#pragma unroll
              for (int m = 0; m < 4; ++m) x[4 * e + m] = qp::mul_h2(o[m], e < 4 ? sc0 : sc1);
            }
          }
          ok = buffer_free(misc->as_empty);
          if (!ok) break;
          tc_fence_after_sync();
          if (there) tmem_st_x32(lane_tm + T::kColAs + buf * 32, x);
          tmem_wait_st();
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(misc->as_full) + k % kUnitRing * 8);
        }
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(bar(misc->scale_full[st]));
          mbar_arrive(bar(misc->code_empty[st]));
        }
        if (++st == L.stages) { st = 0; ++round; }
      }
    } else {
      // Place p of a tile: block p % NB of 128 latents, half p / NB of the slots.
      int p = grp;
#pragma unroll 1
      for (int n = 0; n < n_tiles && ok; ++n) {
        ok = mbar_wait_eager<1>(bar(misc->scale_full[st]), round & 1);
        if (!ok) break;
        const uint32_t rows_at = base + L.off_codes + st * L.stage + lane * code_row;
        const uint32_t scale_at = st_u32 + st * L.scale_room + 4 * t;
#pragma unroll 1
        for (; p < U; p += VG, next_unit(VG)) {
          const int h = p >= NB ? 1 : 0, c = (p - h * NB) * 4 + q;
          uint32_t x[2][4][4];
          if (c < chunks) {
            const uint32_t from = rows_at + h * 64 * code_row + ((uint32_t)(c * 16) ^ twist);
            const uint32_t sc_at = scale_at + c * (kTile * 2) + h * 128;
            uint32_t w[2][4];
            qp::ldsm_x4_trans(from, w[0]);
            qp::ldsm_x4_trans(from + 32 * code_row, w[1]);
#pragma unroll
            for (int i2 = 0; i2 < 2; ++i2)
#pragma unroll
              for (int m = 0; m < 4; ++m) {
                uint32_t sc;
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(sc) : "r"(sc_at + i2 * 64 + m * 16));
                decode_pairs(w[i2][m], x[i2][m]);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[i2][m][e] = qp::mul_h2(x[i2][m][e], sc);
              }
          }
          ok = buffer_free(misc->av_empty);
          if (!ok) break;
          tc_fence_after_sync();
          if (c < chunks) {
            const uint32_t col = lane_tm + T::kColAv + buf * 32;
#pragma unroll
            for (int i2 = 0; i2 < 2; ++i2) {
              const uint32_t(&y)[4][4] = x[i2];
              const uint32_t to = col + i2 * 16;
              tmem_st_16x128_x4(to, y[0][0], y[0][1], y[1][0], y[1][1], y[2][0], y[2][1], y[3][0], y[3][1]);
              tmem_st_16x128_x4(to + (16u << 16), y[0][2], y[0][3], y[1][2], y[1][3], y[2][2], y[2][3], y[3][2], y[3][3]);
            }
          }
          tmem_wait_st();
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(misc->av_full) + k % kUnitRing * 8);
        }
        if (!ok) break;
        p -= U;
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(misc->code_empty[st]));
        if (++st == L.stages) { st = 0; ++round; }
        const TileInfo& info = misc->info[n % kInfo];
        if (info.flags & kLast) {
          // A segment's sums leave tensor memory, while the softmax warps go on.
          const int seg = info.flags >> kSegShift;
          ok = __all_sync(0xffffffffu, wait(misc->end_full[seg % kEndRing], seg / kEndRing) &&
                                           wait(misc->o_full[seg & 1], seg >> 1));
          if (!ok) break;
          tc_fence_after_sync();
          set_down<NC, NB, VG>(a.o_part + ((long long)blockIdx.x + info.group) * (NC * 128 * NB), lane_tm + T::kColO,
                               misc->end_fac[seg & 1], info.flags & kFoldedNow, info.cols, r,
                               q * 32 + 4 * (lane & 7) + (lane >> 3), grp);
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(misc->o_empty));
        }
      }
    }
  } else {
    // ------------------------------------------------------------------ softmax and epilogue
    // Two groups of four warps: group gr owns columns [gr * NHH, (gr + 1) * NHH) of the tile's 128 slots, a slot per
    // thread.  They leave the loop together (they agree on it once a tile, before anything that depends on
    // the tile's description), so the hardware barrier always completes.
    reg_alloc<kSoftmaxRegs>();
    constexpr int NHH = NC / 2;
    const int sw = warp - kSoftmaxWarp0, gr = sw >> 2, q = warp & 3, HO = gr * NHH;
    const int sidx = sw * 32 + lane, slot = q * 32 + lane;
    const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16) + HO;
    auto group_sync = [&]() { named_sync<1, kSoftmaxThreads>(); };
    // One value per column over the warp's 32 slots, left in red[sw][i], 16 columns at a time: halving exchanges, in
    // each of which a lane keeps half of its columns and adds the partner's share of them.
    auto reduce_columns = [&](const float (&x)[NHH], bool is_max) {
      auto join = [&](float c, float d) { return is_max ? fmaxf(c, d) : c + d; };
#pragma unroll
      for (int c0 = 0; c0 < NHH; c0 += 16) {
        float y[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = x[c0 + i];
#pragma unroll
        for (int n = 16, o = 16; n > 1; n >>= 1, o >>= 1) {
          const bool upper = lane & o;
#pragma unroll
          for (int i = 0; i < n / 2; ++i) {
            const float keep = upper ? y[i + n / 2] : y[i], give = upper ? y[i] : y[i + n / 2];
            y[i] = join(keep, __shfl_xor_sync(0xffffffffu, give, o));
          }
        }
        const float z = join(y[0], __shfl_xor_sync(0xffffffffu, y[0], 1));
        if (!(lane & 1)) misc->red[sw][c0 + (lane >> 1)] = z;
      }
    };
    auto reduced = [&](int h, bool is_max) {
      const float* x = &misc->red[(h / NHH) * 4][h % NHH];
      return is_max ? fmaxf(fmaxf(x[0], x[32]), fmaxf(x[64], x[96])) : (x[0] + x[32]) + (x[64] + x[96]);
    };
    auto load_scores = [&](int n, float (&x)[NHH]) {
      uint32_t s[NHH / 16][16];
#pragma unroll
      for (int i = 0; i < NHH / 16; ++i) tmem_ld_x16(lane_base + T::kColS + (n % SB) * NC + i * 16, s[i]);
      tmem_wait_ld();
#pragma unroll
      for (int i = 0; i < NHH; ++i) x[i] = __uint_as_float(s[i / 16][i % 16]);
    };
    uint8_t* const p_row = sm + L.off_p + (HO / 8) * P_SBO + slot * 16;
    float l_acc[NHH];
    bool unset = true;                                   // a column has no reference: no score above minus infinity yet
    for (int n = 0; n < n_tiles; ++n) {
      if (ok && sw == 3) ok = wait(misc->info_full[n % kInfo], n / kInfo) && wait(misc->s_full[n % SB], n / SB);
      if (named_sync_or<kSoftmaxThreads>(1, !ok)) break;
      const TileInfo& info = misc->info[n % kInfo];
      const int flags = info.flags;
      const int rows = slot < 64 ? info.rows0 : info.rows1;
      const int ps = L.p_stages == 2 ? n & 1 : 0, p_round = L.p_stages == 2 ? n >> 1 : n;
      const int ps1 = L.p_stages == 2 ? (n - 1) & 1 : 0, p_round1 = L.p_stages == 2 ? (n - 1) >> 1 : n - 1;
      if (flags & kFirst) {
        if (sidx < 64) {
          const int seg = flags >> kSegShift;
          if (ok) ok = wait(misc->q_full[seg % kQRing], seg / kQRing);       // long since; for the scales
          misc->m_used[sidx] = -INFINITY;
          misc->neg_ref[sidx] = 0.f;
          misc->unit[sidx] = sidx < NC ? misc->next_unit[seg % kQRing][sidx] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < NHH; ++i) l_acc[i] = 0.f;
        unset = true;
        group_sync();
      }
      if (__builtin_expect(flags & kFold, 0)) {
        // The sums so far are set down; this tile's products then begin new ones.
        if (ok) ok = wait(misc->p_empty[2 * ps1 + 1], p_round1);
        ok = __all_sync(0xffffffffu, ok);
        if (sidx < NC) {
          const float m = misc->m_used[sidx], m_old = misc->m_fold[sidx];
          misc->fac[sidx] = m == m_old ? 1.f : exp2f(m_old - m);        // of use from the second time on
          misc->m_fold[sidx] = m;
        }
        group_sync();
        if (ok) {
          tc_fence_after_sync();
          set_down<NC, NB, 2>(a.o_part + ((long long)blockIdx.x + info.group) * (NC * 128 * NB),
                              tmem + ((uint32_t)(q * 32) << 16) + T::kColO, misc->fac, flags & kFolded, info.cols, r,
                              q * 32 + 4 * (lane & 7) + (lane >> 3), gr);
          tc_fence_before_sync();
        }
        group_sync();                                    // fac may be rewritten
      }
      // The scores leave tensor memory at once, so that the next tile's products may begin.
      float x[NHH];
      tc_fence_after_sync();
      load_scores(n, x);
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(misc->s_empty[n % SB]));
      const bool live = (slot & 63) < rows, full = __all_sync(0xffffffffu, live);
      // x = score - reference + shift in log2 units; the bare score as long as there is no reference, which the
      // segment's first slots set.
#pragma unroll
      for (int i = 0; i < NHH; i += 4) {
        const ulonglong2 u = *reinterpret_cast<const ulonglong2*>(&misc->unit[HO + i]);
        const ulonglong2 o = *reinterpret_cast<const ulonglong2*>(&misc->neg_ref[HO + i]);
        unpack2(fma2(pack2(x[i], x[i + 1]), u.x, o.x), x[i], x[i + 1]);
        unpack2(fma2(pack2(x[i + 2], x[i + 3]), u.y, o.y), x[i + 2], x[i + 3]);
      }
      if (!full) {                                       // only a sequence's last tile
#pragma unroll
        for (int i = 0; i < NHH; ++i) x[i] = live ? x[i] : -INFINITY;
      }
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < NHH; ++i) top = fmaxf(top, x[i]);
      if (named_sync_or<kSoftmaxThreads>(1, unset || top > kShift + kRescale)) {
        // Some reference has to rise: always at a segment's first slots, else rarely.
        reduce_columns(x, true);
        group_sync();
        bool none = false;                               // this thread's column has no reference after this tile either
        if (sidx < NC) {
          // What the column's largest score is above its reference by; without one (its x are bare scores): itself.
          const float m_used = misc->m_used[sidx];
          const bool first = m_used == -INFINITY;
          const float mt = reduced(sidx, true) - (first ? 0.f : kShift), m_old = first ? 0.f : m_used;
          const bool rise = mt > (first ? -INFINITY : kRescale);
          const float by = rise ? mt : 0.f;
          none = first && !rise;
          misc->m_used[sidx] = none ? -INFINITY : m_old + by;
          misc->neg_ref[sidx] = none ? 0.f : kShift - (m_old + by);
          misc->fac[sidx] = first ? 0.f : exp2f(-by);
          misc->down[sidx] = first ? kShift - by : -by;
        }
        group_sync();
#pragma unroll
        for (int i = 0; i < NHH; ++i) {
          l_acc[i] *= misc->fac[HO + i];
          x[i] += misc->down[HO + i];
        }
        if (!(flags & (kFirst | kFold))) {
          // O is scaled to the old references: wait for the previous tile's products, rescale.
          if (ok) ok = wait(misc->p_empty[2 * ps1 + 1], p_round1);
          ok = __all_sync(0xffffffffu, ok);              // TMEM accesses are whole-warp operations
          if (ok) {
            tc_fence_after_sync();
#pragma unroll 1
            for (int i = 0; i < NB * (NHH / 16); ++i) {
              const uint32_t at = lane_base + T::kColO + (i % NB) * NC + i / NB * 16;
              uint32_t o[16];
              tmem_ld_x16(at, o);
              tmem_wait_ld();
#pragma unroll
              for (int j = 0; j < 16; ++j)
                o[j] = __float_as_uint(__uint_as_float(o[j]) * misc->fac[HO + i / NB * 16 + j]);
              tmem_st_x16(at, o);
            }
            tmem_wait_st();
          }
        }
        // fac / down / red may be rewritten from here.
        unset = named_sync_or<kSoftmaxThreads>(1, none && sidx < info.cols);
      }
      // The value products of the tile that had this half's place are done.
      if (ok) ok = wait(misc->p_empty[2 * ps + (q >> 1)], p_round + 1);
      // P as the MN-major, un-swizzled B operand: eight columns of a slot are 16 bytes, eight slots
      // follow one another, groups of eight columns are P_SBO apart.
#pragma unroll
      for (int i = 0; i < NHH / 8; ++i) {
        uint32_t pb[4];
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          const float e0 = ex2_approx(x[8 * i + j]), e1 = ex2_approx(x[8 * i + j + 1]);
          l_acc[8 * i + j] += e0;
          l_acc[8 * i + j + 1] += e1;
          const __half2 y = __floats2half2_rn(e0, e1);
          pb[j / 2] = *reinterpret_cast<const uint32_t*>(&y);
        }
        if (ok) *reinterpret_cast<uint4*>(p_row + ps * L.p_bytes + i * P_SBO) = make_uint4(pb[0], pb[1], pb[2], pb[3]);
      }
      fence_proxy_async_smem();
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(misc->p_full[2 * ps + (q >> 1)]));
      if (!(flags & kLast)) continue;

      // ---- end of a segment
      const int v = info.group, part = (int)blockIdx.x + v;
      reduce_columns(l_acc, false);
      group_sync();
      if (ok && sidx < info.cols) {
        const float m = misc->m_used[sidx];
        *reinterpret_cast<float2*>(a.ml_part + ((long long)part * a.cols + sidx) * 2) =
            make_float2(m - kShift, reduced(sidx, false));
        if (flags & kFoldedNow) {
          const float m_set = misc->m_fold[sidx];
          misc->end_fac[flags >> kSegShift & 1][sidx] = m_set == m ? 1.f : exp2f(m_set - m);
        }
      }
      if (ok && sidx == 0 && (flags & kEnds)) a.seq_parts[v] = make_int2(info.owner + v, (int)blockIdx.x - info.owner + 1);
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(misc->end_full[(flags >> kSegShift) % kEndRing]));
      group_sync();                                      // red, unit and the references may be rewritten
    }
  }

  if (!ok) misc->abort_word = 1;
  __syncthreads();
  if (threadIdx.x == 0) a.error_words[blockIdx.x] = misc->abort_word;
  if (misc->abort_word) {
    // Give copies that may still be in flight time to land before the CTA's memory is reused.
    const uint64_t t0 = global_timer_ns();
    while (global_timer_ns() - t0 < 100000ull) __nanosleep(1000);
  }
  if (warp == kProducerWarp) {
    __syncwarp();
    tc_fence_after_sync();
    tmem_dealloc(misc->tmem_base, 512);
  }
}

}  // namespace tree
}  // namespace mtla
