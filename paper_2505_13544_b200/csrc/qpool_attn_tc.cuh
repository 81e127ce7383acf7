// Attention over the 4-bit pool on the fifth-generation tensor cores (bf16 queries).
//
// The bound of this operator is the pool's bytes (400 per slot at r 512), but every slot has to be
// expanded to half precision twice, once per contraction, and what the expanded elements then cost
// decides: written to shared memory and read back by the matrix instructions they would take some 25
// cycles of its bandwidth per slot, against the 16 that the slot's bytes take to arrive.  So they
// never go there.  The matrix instructions take their A operand from tensor memory, and the expanding
// warps write it with register-to-TMEM stores, each contraction's operand in its own orientation:
//   scores  S[128 slots x heads]      = C[128 x r] . Q^T        A row = slot: a thread owns a slot, reads 16
//                                                               bytes = 32 latents, stores 16 columns
//   values  O^T[128 latents x heads] += C^T[128 x 128 slots] . P A row = latent: a transposing matrix load moves
//                                                               units of four codes; thread (g, t) gets four
//                                                               latents of slots 2t, 2t + 1, pairs the two
//                                                               slots' codes and stores them to four lanes.
//                                                               Lane 8j + g of a 32-lane quarter therefore
//                                                               holds latent 4g + j; the output undoes it.
// Shared memory then carries only the raw pages (three tiles of 128 slots deep), the queries and the
// probabilities.
//
// Measured at 128 sequences of 16384 slots, 32 heads, r 512, d_R 64: 267 us at 1965 MHz (295 us once the
// power cap holds the clock at 1.78 GHz), 3.1 TB/s of pool, 49 % of the measured copy bandwidth; the bytes
// alone would take 130 us.  Per tile of 128 slots that is 4740 cycles, start and join included.  The
// expansion's conversions and scalings need 1900 of them (46.7 pairs of latents per cycle and SM for the
// scores, 27.1 for the values, whose codes have to be paired first; measured from registers, 16 warps an
// SM), the matrix instructions 1100, the bytes 2300.  What is between is the hand-over of the operand units: a unit's buffer goes from the expanding warps
// through an mbarrier to the issuing warp, through the matrix unit and back in some 2200 cycles, since
// with the memory instruction queues full of operand stores a wait takes 300 even for what is there.
// Tensor memory has room for two units of the scores and three of the values beside the two
// accumulators (three and two: 281 us beside 270).  At 32 sequences, 91 us with one score issuer, leaving out the
// softmax gave 90 us, the matrix instructions 78, the operand stores 73, loads, arithmetic and
// stores together 76, all of it 52.
//
// A head count of 16 or 32 is the matrix instructions' N, so heads are not padded further.  The RoPE
// keys go from the pool to the score product as they are (bf16, shared memory, hardware swizzle).
//
// Roles (28 warps): warps 0 and 3 issue the score products, warp 1 the value products, warp 2 is the
// producer; warps 4-19 expand, in four groups that take turns (see there), and write the queries;
// warps 20-27 are softmax and epilogue.  The hot loops are short on purpose: with several kinds of code on every scheduler,
// fetching unrolled instructions was the longest stall (107 KB of them: 517 us at 128 x 16384
// slots, 61 KB: 362 us), then the issuing threads' scalar descriptors (a uniform warp: 331), the sharing
// out of the expansion (282) and a single score issuer (270 with two; a second value issuer adds nothing).
// The online softmax raises a head's reference only when a tile exceeds it by 2^8.  Probabilities
// are kept times 2^7: with the 2^8 they stay inside half precision.  For the value product they are rounded
// to it, 2^-11 at most, an eighth of what the bf16 output is rounded by (a second term would double that
// product and its buffers); the denominators add the unrounded ones in 32 bits.
//
// The matrix unit cuts its running sums off instead of rounding them: every 16 slots the output loses part
// of its last place, always towards zero (a segment of 2^18 slots came out 1.6e-3 too small, one of
// 2^20 slots 6.6e-3, more than the rounding of the bf16 result).  So after kFoldTiles tiles the softmax warps
// take the sums out of tensor memory and add them up, rounded, in the segment's place among the partials,
// and 6e-5 is missing at any length (2^14 and 2^20 slots alike).
//
// Every wait is bounded; after a time-out the roles unwind, each when its own next wait runs out, and
// qpool_combine_kernel answers with NaN.
#pragma once

#include "qpool_attn.cuh"

namespace mtla {
namespace qp {
namespace tc {

constexpr int kTile = 128;                  // slots per tile: two pages
constexpr int kThreads = 896;
constexpr int kMaxStages = 4;               // as many as value units' barriers
// Sequences whose prefix sums and slot counts every CTA keeps in shared memory: as many as fit beside three
// stages in the largest shape (r 512, d_R 64, 32 heads).
constexpr int kMaxBatch = 1022;
constexpr int kScoreIssuer = 0, kValueIssuer = 1, kProducerWarp = 2, kScoreIssuer2 = 3;
constexpr int kExpandWarp0 = 4, kExpandGroups = 4;
constexpr int kSoftmaxWarp0 = 20, kSoftmaxThreads = 256, kSoftmaxWarps = 8;
// Queries and scales of segments: the expanding warps are at most two segments ahead of the softmax
// (its tile has to leave the accumulator that the second next one takes), so four keep them apart.
constexpr int kQRing = 4;
constexpr int kInfo = 16;                   // ring of tile descriptions, deeper than any role's lag
// TMEM columns: two score buffers, up to four output blocks of NHP columns, two operand
// buffers of 64 columns for the scores and what is left, three (32 heads) or four, for the values.
constexpr int kTmemCols = 512;
constexpr int kColS = 0, kColO = 64;
__host__ __device__ constexpr int col_as(int nhp) { return kColO + 4 * nhp; }
__host__ __device__ constexpr int col_av(int nhp) { return col_as(nhp) + 128; }
__host__ __device__ constexpr int av_buffers(int nhp) { return nhp == 32 ? 3 : 4; }
static_assert(col_av(32) + 64 * av_buffers(32) <= kTmemCols && col_av(16) + 64 * av_buffers(16) <= kTmemCols,
              "tensor memory budget");
constexpr float kShift = 7.f, kRescale = 8.f;
constexpr int kFoldTiles = 128;             // tiles whose products are summed in tensor memory
constexpr float kUnset = 3e38f;             // in the place of -reference: any score then exceeds it
constexpr int kSmemMax = 227 * 1024 - 1024;

// First and last tile of a segment; the sums of the tiles before it are set down first; sums have been set
// down before this tile, or with it.
constexpr int kFirst = 1, kLast = 2, kFold = 4, kFolded = 8, kFoldedNow = 16, kSegShift = 5;
struct TileInfo {
  int b;
  int flags;                 // the above; the segment's number times 32
  int rows0, rows1;          // slots of the tile's two pages
};

struct Misc {
  unsigned long long raw_full[kMaxStages], raw_empty[kMaxStages], scale_full[kMaxStages];
  // Operand units (a quarter of r of one tile) are numbered through; unit k's barriers are those of k
  // mod 8 (scores) or 4 (values), its buffer is shared with fewer units.  Who fills unit k waits for the
  // unit that had the buffer before, and who reads it waits for it; both see every phase of the
  // barriers they wait for.
  unsigned long long as_full[8], as_empty[8], av_full[4], av_empty[4];
  unsigned long long s_full[2], s_empty[2], p_full[2], p_empty[2];
  unsigned long long q_full[kQRing], q_empty[kQRing];        // segment s: those of s mod 4
  unsigned long long info_full[kInfo];
  uint32_t tmem_base;
  int abort_word;
  int warp_sums[32];
  TileInfo info[kInfo];
  float m_used[32];          // reference maximum (log2 units), minus infinity before the first score
  alignas(16) float neg_ref[32];   // shift - reference: what a score is offset by
  alignas(16) float unit[32];      // scale of the head's scores
  float next_unit[kQRing][32];     // the same, as the queries' writers leave it
  float fac[32];
  float red[8][16];
  float m_fold[32];          // reference of the sums that have been set down
};
constexpr int kMiscBytes = 2688;
static_assert(sizeof(Misc) <= kMiscBytes, "misc region too small");

struct Layout {
  int codes, scales, keys;                  // offsets in a stage
  int stage, stages;
  int off_q, q_bytes, off_p, off_st, off_misc, off_prefix, off_slots, total;
  __host__ __device__ Layout(const Format& f, int nhp, int batch) {
    keys = 0;                                            // swizzled operand: 1024-byte aligned
    codes = kTile * f.key_row();
    scales = codes + kTile * f.code_row();
    stage = (scales + kTile * f.scale_row() + 1023) / 1024 * 1024;
    q_bytes = nhp * 2 * (f.r + f.dr);
    const int q_room = (q_bytes + 1023) / 1024 * 1024, p_room = 2 * kTile * nhp * 2;
    const int scale_room = f.scale_row() * kTile * 2;
    const int fixed = q_room + p_room + kMiscBytes + (2 * batch + 1) * 4 + 1024;   // 1024: alignment of the base
    // At least three (r 512, 32 heads, d_R 64: exactly), which the expansion's waits rely on; with one
    // unit a tile (r <= 128) always four, as many as a tile's value operands may lag.
    stages = (kSmemMax - fixed) / (stage + scale_room);
    if (stages > kMaxStages) stages = kMaxStages;
    off_q = stages * stage;
    off_p = off_q + q_room;
    off_st = off_p + p_room;
    off_misc = off_st + stages * scale_room;
    off_prefix = off_misc + kMiscBytes;
    off_slots = off_prefix + (batch + 1) * 4;
    total = off_slots + batch * 4 + 1024;
  }
};

}  // namespace tc

// Queries of a segment -> the score product's B operand, by the QW warps that expand the units of its
// first tile (two of the three with three), each some heads: r / 64 panels [NHP][64] half precision with
// the 128-byte swizzle and one panel [NHP][d_R] bf16 (128- or 64-byte swizzle).  A head's row is scaled
// by the power of two that brings its largest element into [2^14, 2^15); heads that do not exist are
// zero.  As a kernel of its own in front, with the image loaded from memory, this took 1 to 2.5 us more of
// a small batch's 15 to 19.  Not inlined: the loop that calls it once a segment is short of registers.
template <int NHP, int QW, int QB, int QV>
__device__ __noinline__ bool put_queries(const bf16* q, uint8_t* image, tc::Misc* misc, float scale_log2, int n_heads,
                                         Format f, int seg, int first_head) {
  using namespace tc;
  const int r = f.r, dr = f.dr, lane = threadIdx.x & 31;
  const int n8 = (r + dr) / 8;
#pragma unroll 1
  for (int h0 = first_head; h0 < NHP; h0 += QB * QW) {
    uint4 w[QB][QV];
#pragma unroll
    for (int j = 0; j < QB; ++j) {
      const int h = h0 + j * QW;
      const bf16* src = q + (long long)h * (r + dr);
#pragma unroll
      for (int i = 0; i < QV; ++i) {
        const int c = lane + 32 * i;
        w[j][i] = make_uint4(0u, 0u, 0u, 0u);
        if (c < n8 && h < n_heads) w[j][i] = *reinterpret_cast<const uint4*>(src + 8 * c);
      }
    }
    // The score products of the segment before are done.
    const bool there = seg == 0 || ptx::mbar_wait_compact(ptx::smem_u32(&misc->q_empty[(seg - 1) % kQRing]),
                                                          (seg - 1) / kQRing & 1);
    if (!__all_sync(0xffffffffu, there)) return false;
#pragma unroll
    for (int j = 0; j < QB; ++j) {
      const int h = h0 + j * QW;                    // NHP is a multiple of QB * QW
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < QV; ++i) {
        const uint32_t x[4] = {w[j][i].x, w[j][i].y, w[j][i].z, w[j][i].w};
#pragma unroll
        for (int m = 0; m < 4; ++m) top = max(top, max(x[m] & 0x7fff0000u, (x[m] << 16) & 0x7fff0000u));
      }
      top = __reduce_max_sync(0xffffffffu, top);
      // Exponents -113 .. 140 (a row of subnormal numbers only reaches less); none for zeros and specials.
      const bool fine = top > 0 && top < 0x7f800000u;
      const int e = fine ? 141 - max((int)(top >> 23), 1) : 0, e1 = e / 2, e2 = e - e1;
      const float f1 = __uint_as_float((127 + e1) << 23), f2 = __uint_as_float((127 + e2) << 23);
      if (lane == 0)
        misc->next_unit[seg % kQRing][h] =
            scale_log2 * __uint_as_float((127 - e1) << 23) * __uint_as_float((127 - e2) << 23);
#pragma unroll
      for (int i = 0; i < QV; ++i) {
        const int c = lane + 32 * i;
        if (c >= n8) break;
        const uint32_t x[4] = {w[j][i].x, w[j][i].y, w[j][i].z, w[j][i].w};
        const bool latent = 8 * c < r;
        uint32_t y[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const float lo = __uint_as_float(x[m] << 16) * f1 * f2;
          const float hi = __uint_as_float(x[m] & 0xffff0000u) * f1 * f2;
          const __half2 l2 = __floats2half2_rn(lo, hi);
          const __nv_bfloat162 k2 = __floats2bfloat162_rn(lo, hi);
          y[m] = latent ? *reinterpret_cast<const uint32_t*>(&l2) : *reinterpret_cast<const uint32_t*>(&k2);
        }
        const int at = latent ? (c >> 3) * NHP * 128 + h * 128 + ((c ^ h) & 7) * 16
                              : NHP * 2 * r + h * 2 * dr + ((c - r / 8) ^ f.key_swizzle(h)) * 16;
        *reinterpret_cast<uint4*>(image + at) = make_uint4(y[0], y[1], y[2], y[3]);
      }
    }
  }
  ptx::fence_proxy_async_smem();
  __syncwarp();
  if (lane == 0) ptx::mbar_arrive(ptx::smem_u32(&misc->q_full[seg % kQRing]));
  return true;
}

// A softmax thread's output sums (of latent `lat` of every block, heads ho ..) out of tensor memory, added to
// what the segment has set down in `part` (not yet anything without `add`), which is brought to the present
// references by fac; into `part` again, or at the segment's end, divided, into `out`.  A whole-warp call.
// Rarely reached, yet inlined: a call made the loop around it spill (128 sequences of r 384, 32 heads: 254 us,
// so 251; with no folding at all 249).
template <int NHP, int NB>
__device__ __forceinline__ void fold_output(float* part, bf16* out, const tc::Misc* misc, uint32_t taddr, int ho, int n_heads,
                                         int r, int lat, bool add) {
  constexpr int NHH = NHP / 2;
#pragma unroll 1
  for (int mb = 0; mb < NB; ++mb) {
    uint32_t ov[16];
    if (NHH == 16) ptx::tmem_ld_x16(taddr + mb * NHP, ov); else ptx::tmem_ld_x8(taddr + mb * NHP, ov);
    ptx::tmem_wait_ld();
    if (mb * 128 + lat >= r) continue;
#pragma unroll
    for (int i = 0; i < NHH; ++i) {
      if (ho + i >= n_heads) break;
      const long long e = (long long)(ho + i) * r + mb * 128 + lat;
      float v = __uint_as_float(ov[i]);
      if (add) v = fmaf(part[e], misc->fac[ho + i], v);
      if (out) out[e] = __float2bfloat16_rn(v * misc->unit[ho + i]);
      else part[e] = v;
    }
  }
}

// NHP: heads padded to 16 or 32.  NB: ceil(r / 128).
template <int NHP, int NB>
__global__ void __launch_bounds__(tc::kThreads, 1) qpool_attend_tc_kernel(AttnArgs a, tc::Layout L) {
  using namespace tc;
  using namespace ptx;
  constexpr uint32_t IDESC_S = make_idesc_f16(128, NHP, 0, 0), IDESC_K = make_idesc_bf16(128, NHP, 0, 0);
  constexpr uint32_t IDESC_V = make_idesc_f16(128, NHP, 0, 1);
  constexpr uint32_t P_BYTES = kTile * NHP * 2, P_SBO = kTile * 16;   // bytes between groups of 8 heads
  constexpr int SI = NB == 3 ? 1 : 2;           // score issuers (see there)
  constexpr int QW = NB == 4 ? 16 : NB == 1 ? 4 : 8;                  // warps that write a segment's queries
  constexpr int QB = NHP / QW < 2 ? 1 : NB == 1 ? 4 : 2;              // their heads loaded together
  constexpr int QV = (NB * 16 + 8 + 31) / 32;   // runs of eight elements of a lane
  constexpr int AVB = av_buffers(NHP), COL_AS = col_as(NHP), COL_AV = col_av(NHP);
  extern __shared__ uint8_t smem_raw[];
  const Format f = a.f;
  const int r = f.r, dr = f.dr;
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* sm = smem_raw + (base - raw);
  Misc* misc = reinterpret_cast<Misc*>(sm + L.off_misc);
  int* prefix = reinterpret_cast<int*>(sm + L.off_prefix);
  int* slots_s = reinterpret_cast<int*>(sm + L.off_slots);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;   // warp: uniform
  auto bar = [&](unsigned long long& p) { return smem_u32(&p); };

  // A thread per barrier of a kind: one thread for all of them would take 1000 cycles.
  if (threadIdx.x < kInfo) {
    const int i = threadIdx.x;
    mbar_init(bar(misc->info_full[i]), 1);
    if (i < 8) {
      mbar_init(bar(misc->as_full[i]), 4);
      mbar_init(bar(misc->as_empty[i]), 1);
    }
    if (i < 4) {
      mbar_init(bar(misc->raw_full[i]), 1);
      mbar_init(bar(misc->raw_empty[i]), 2 * NB * 4 + SI);       // a warp of each unit, the score issuers
      mbar_init(bar(misc->scale_full[i]), NB * 4);
      mbar_init(bar(misc->av_full[i]), 4);
      mbar_init(bar(misc->av_empty[i]), 1);
      mbar_init(bar(misc->q_full[i]), QW);
      mbar_init(bar(misc->q_empty[i]), SI);
    }
    if (i < 2) {
      mbar_init(bar(misc->s_full[i]), 1);
      mbar_init(bar(misc->s_empty[i]), kSoftmaxWarps);
      mbar_init(bar(misc->p_full[i]), kSoftmaxWarps);
      mbar_init(bar(misc->p_empty[i]), 1);
    }
    if (i == 0) misc->abort_word = 0;
    mbar_fence_init();
  }
  if (warp == kProducerWarp) tmem_alloc(smem_u32(&misc->tmem_base), kTmemCols);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  // All 512 columns are this CTA's, so they start at column 0: a constant that the addresses of the
  // matrix instructions are formed with (anything else would be an allocator's error, told as such).
  constexpr uint32_t tmem = 0;
  grid_launch_dependents();      // this CTA owns its TMEM columns (see decode_attn_tc.cuh)
  grid_dependency_wait();

  const long long total = tile_prefix<2>(a, prefix, misc->warp_sums, kThreads, slots_s);
  const int ctas = (int)(total < gridDim.x ? total : gridDim.x);
  int g0 = 0, g1 = 0;
  if ((int)blockIdx.x < ctas) {
    g0 = share_begin(blockIdx.x, total, ctas);
    g1 = share_begin(blockIdx.x + 1, total, ctas);
  }
  const int n_tiles = __shfl_sync(0xffffffffu, g1 - g0, 0);      // uniform
  const uint32_t q_u32 = base + L.off_q, p_u32 = base + L.off_p, st_u32 = base + L.off_st;
  auto wait = [&](unsigned long long& b, int phase) { return mbar_wait_compact(bar(b), phase & 1); };
  auto wait_warp = [&](unsigned long long& b, int phase) {                 // one answer for the warp
    return __all_sync(0xffffffffu, wait(b, phase)) != 0;
  };
  // Asks without waiting.  While the expanding warps keep the memory instruction queues full an answer
  // takes some 300 cycles, so the issuing warps ask for what comes next before they issue what is there.
  auto ask = [&](unsigned long long& b, int phase) { return mbar_test(bar(b), phase & 1); };
  bool ok = true;                // false once a wait of this thread has given up
  if (threadIdx.x == 0 && misc->tmem_base != 0) misc->abort_word = 1;

  if (n_tiles == 0) {
    // nothing to do; the CTA falls through to the common end
  } else if (warp < kExpandWarp0) {
    if (warp == kProducerWarp && lane == 0) {
      // ---------------------------------------------------------------- producer
      int b = find_seq(prefix, a.batch, g0), seg = -1, st = 0, round = 0, begun = 0;
      for (int n = 0; n < n_tiles; ++n) {
        const int g = g0 + n;
        while (prefix[b + 1] <= g) ++b;
        const int tile = g - prefix[b], slots = slots_s[b];
        const bool first = n == 0 || tile == 0, last = n + 1 == n_tiles || g + 1 == prefix[b + 1];
        int page[2], rows[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int t = 2 * tile + i, have = slots - t * kPageRows;
          page[i] = have > 0 && t < a.width ? __ldg(a.table + (long long)b * a.width + t) : -1;
          rows[i] = page[i] >= 0 && page[i] < a.n_pages ? min(have, kPageRows) : 0;
        }
        ok = wait(misc->raw_empty[st], round + 1);
        if (!ok) break;
        TileInfo& info = misc->info[n % kInfo];
        info.b = b;
        seg += first;
        if (first) begun = n;
        const int before = n - begun;
        info.flags = (first ? kFirst : 0) | (last ? kLast : 0) | (before && before % kFoldTiles == 0 ? kFold : 0) |
                     (before > kFoldTiles ? kFolded : 0) | (before >= kFoldTiles ? kFoldedNow : 0) | seg << kSegShift;
        info.rows0 = rows[0];
        info.rows1 = rows[1];
        mbar_arrive(bar(misc->info_full[n % kInfo]));
        uint32_t bytes = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i)
          bytes += rows[i] * (f.code_row() + f.key_row()) + (rows[i] * f.scale_row() + 15) / 16 * 16;
        const uint32_t full = bar(misc->raw_full[st]), dst = base + st * L.stage;
        mbar_arrive_expect_tx(full, bytes);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (rows[i] == 0) continue;
          const uint8_t* src = a.pages + (long long)page[i] * f.page_bytes();
          bulk_load(dst + L.scales + i * kPageRows * f.scale_row(), src + f.off_scales(),
                    (rows[i] * f.scale_row() + 15) / 16 * 16, full);
          bulk_load(dst + L.codes + i * kPageRows * f.code_row(), src, rows[i] * f.code_row(), full);
          bulk_load(dst + L.keys + i * kPageRows * f.key_row(), src + f.off_keys(), rows[i] * f.key_row(), full);
        }
        if (++st == L.stages) { st = 0; ++round; }
      }
    } else if (warp == kScoreIssuer || (SI == 2 && warp == kScoreIssuer2)) {
      // ---------------------------------------------------------------- score products (whole warp, uniform)
      // Two warps issue them, a tile each in turn (the tiles' accumulators alternate anyway): with the
      // memory instruction queues full of the expansion's traffic a wait, even for what is there,
      // takes some 300 cycles, and one warp's waits took all of a tile's time.  Each still looks at
      // every tile, so that it sees every phase of the barriers.  (With three units a tile the units'
      // barriers would change hands between the two, so there one warp does it all.)
      const int mine = warp == kScoreIssuer ? 0 : 1;
      const uint64_t mode = dr == 64 ? kSwizzle128B : kSwizzle64B;
      const uint32_t key_sbo = 8 * f.key_row();
      const uint64_t q_desc = make_smem_desc(q_u32, 16, 1024, kSwizzle128B);
      const uint64_t qk_desc = make_smem_desc(q_u32 + NHP * 2 * r, 16, key_sbo, mode);
      int st = 0, round = 0;
      for (int n = 0; n < n_tiles && ok; ++n) {
        ok = wait_warp(misc->raw_full[st], round);
        if (!ok) break;
        const int flags = misc->info[n % kInfo].flags, seg = flags >> kSegShift;
        if (flags & kFirst) {
          ok = wait_warp(misc->q_full[seg % kQRing], seg / kQRing);
          if (!ok) break;
        }
        if (SI == 1 || (n & 1) == mine) {
          ok = wait_warp(misc->s_empty[n & 1], (n >> 1) + 1);
          if (!ok) break;
          tc_fence_after_sync();
          const uint32_t d = tmem + kColS + (n & 1) * 32;
          const uint64_t key_desc = make_smem_desc(base + st * L.stage + L.keys, 16, key_sbo, mode);
          if (elect_one()) {                             // RoPE part: d_R / 16 is 2 or 4
            mma_bf16_ss(d, key_desc, qk_desc, IDESC_K, 0u);
            mma_bf16_ss(d, key_desc + 2, qk_desc + 2, IDESC_K, 1u);
            if (dr == 64) {
              mma_bf16_ss(d, key_desc + 4, qk_desc + 4, IDESC_K, 1u);
              mma_bf16_ss(d, key_desc + 6, qk_desc + 6, IDESC_K, 1u);
            }
          }
          __syncwarp();
#pragma unroll 1
          for (int kq = 0; kq < NB; ++kq) {
            const int k = n * NB + kq;
            ok = wait_warp(misc->as_full[k & 7], k >> 3);
            if (!ok) break;
            tc_fence_after_sync();
            const uint32_t at = tmem + COL_AS + (k & 1) * 64;
            const uint32_t panel = (uint32_t)q_desc + kq * 2 * NHP * 8, hi = (uint32_t)(q_desc >> 32);
            if (elect_one()) {
#pragma unroll
              for (int ks = 0; ks < 4; ++ks) mma_f16_ts(d, at + ks * 8, panel + ks * 2, hi, IDESC_S, 1u);
              if (kq * 128 + 64 < r) {
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)
                  mma_f16_ts(d, at + 32 + ks * 8, panel + NHP * 8 + ks * 2, hi, IDESC_S, 1u);
              }
              mma_commit(bar(misc->as_empty[k & 7]));
            }
            __syncwarp();
          }
          if (!ok) break;
          if (elect_one()) {
            mma_commit(bar(misc->s_full[n & 1]));
            mma_commit(bar(misc->raw_empty[st]));
            if (flags & kLast) mma_commit(bar(misc->q_empty[seg % kQRing]));
          }
        } else if (elect_one()) {
          mbar_arrive(bar(misc->raw_empty[st]));
          if (flags & kLast) mma_commit(bar(misc->q_empty[seg % kQRing]));
        }
        __syncwarp();
        if (++st == L.stages) { st = 0; ++round; }
      }
    } else if (warp == kValueIssuer) {
      // ---------------------------------------------------------------- value products (whole warp, uniform)
      const uint64_t p_desc = make_smem_desc(p_u32, 128, P_SBO, kSwizzleNone);
      int vb = 0;
      bool unit_there = false;
      for (int n = 0; n < n_tiles && ok; ++n) {
        ok = wait_warp(misc->p_full[n & 1], n >> 1);
        if (!ok) break;
        tc_fence_after_sync();
        const uint32_t fresh = (misc->info[n % kInfo].flags & (kFirst | kFold)) != 0;
        const uint32_t pd = (uint32_t)p_desc + (n & 1) * (P_BYTES / 16), hi = (uint32_t)(p_desc >> 32);
#pragma unroll 1
        for (int mb = 0; mb < NB; ++mb) {
          const int k = n * NB + mb;
          ok = __all_sync(0xffffffffu, unit_there) || wait_warp(misc->av_full[k & 3], k >> 2);
          if (!ok) break;
          unit_there = ask(misc->av_full[(k + 1) & 3], (k + 1) >> 2);
          tc_fence_after_sync();
          const uint32_t d = tmem + kColO + mb * NHP, at = tmem + COL_AV + vb * 64;
          if (elect_one()) {
            mma_f16_ts(d, at, pd, hi, IDESC_V, fresh ^ 1u);
#pragma unroll
            for (int ks = 1; ks < kTile / 16; ++ks) mma_f16_ts(d, at + ks * 8, pd + ks * 16, hi, IDESC_V, 1u);
            mma_commit(bar(misc->av_empty[k & 3]));
          }
          __syncwarp();
          if (++vb == AVB) vb = 0;
        }
        if (ok && elect_one()) mma_commit(bar(misc->p_empty[n & 1]));
        __syncwarp();
      }
    }
  } else if (warp < kSoftmaxWarp0) {
    // ------------------------------------------------------------------ expansion
    // Four groups of four warps take the units in turn, a group expanding unit k for the scores and then
    // unit k - NB, the same quarter of the tile before, for the values: the work is even whatever
    // r is, and a tile's probabilities are usually there when its value units are wanted.
    const int q = warp & 3, grp = (warp - kExpandWarp0) >> 2, t = lane & 3;
    const int slot = q * 32 + lane, row = slot & 63;
    const int cmask = f.code_mask(), chunks = r / kGroup, code_row = f.code_row();
    const uint32_t lane_tm = tmem + ((uint32_t)(q * 32) << 16);
    const uint32_t twist = (uint32_t)(lane & cmask) * 16;       // rows lane, lane + 32, ... twist alike
    const int n_units = n_tiles * NB;
    // The segment that tile n is in, its sequence, and the tile at which the next one begins.
    int seg = -1, b = find_seq(prefix, a.batch, g0), next_start = 0;
    // Tile n, quarter kq of unit k, the stage of tile n and how often the ring has come round; the
    // value unit is the same quarter of tile n - 1.
    int n = 0, kq = grp, st = 0, round = 0;
    auto next_tile = [&]() {
      ++n;
      if (++st == L.stages) { st = 0; ++round; }
    };
#pragma unroll 1
    while (kq >= NB) { kq -= NB; next_tile(); }
#pragma unroll 1
    for (int k = grp; k < n_units + NB; k += kExpandGroups) {
      if (k < n_units) {
        if (__builtin_expect(n >= next_start, 0)) {
          int start;
          do {
            start = next_start;
            while (prefix[b + 1] <= g0 + start) ++b;
            next_start = prefix[b + 1] - g0;
            ++seg;
          } while (n >= next_start);
          if (n == start && kq < QW / 4) {
            const int h0 = kq * 4 + q;
            ok = put_queries<NHP, QW, QB, QV>(static_cast<const bf16*>(a.q) + (long long)b * a.n_heads * (r + dr),
                                              sm + L.off_q, misc, a.scale_log2, a.n_heads, f, seg, h0);
            if (!ok) break;
          }
        }
        // The buffer first: that unit k - 2 has been used also tells that the stage's phase is the one
        // before this tile's or later, which its parity alone would not.
        ok = (k < 2 || wait(misc->as_empty[(k - 2) & 7], (k - 2) >> 3)) && wait(misc->raw_full[st], round);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after_sync();
        const TileInfo& info = misc->info[n % kInfo];
        const uint32_t live = row < (slot < 64 ? info.rows0 : info.rows1) ? 0xffffffffu : 0u;
        const uint32_t stage = base + st * L.stage;
        const uint32_t codes = stage + L.codes + slot * code_row, scales = stage + L.scales + slot * f.scale_row();
        // The scales also go out as half precision, a group's 128 slots in a row, for the value units;
        // zero where there is no slot, so that whatever its codes are, the product is zero.
        const uint32_t st_out = st_u32 + st * f.scale_row() * kTile * 2 + slot * 2;
        const int c_end = min(chunks, kq * 4 + 4);
        uint32_t at = lane_tm + COL_AS + (k & 1) * 64;
#pragma unroll 1
        for (int c = kq * 4; c < c_end; c += 2, at += 32) {
          // Two chunks at a time: their loads overlap, and a row of scales is a multiple of 2 bytes.
          const uint4 w0 = lds128(codes + ((uint32_t)(c * 16) ^ twist));
          const uint4 w1 = lds128(codes + ((uint32_t)(c * 16 + 16) ^ twist));
          uint32_t two;
          asm volatile("{\n\t.reg .u16 x;\n\tld.shared.u16 x, [%1];\n\tcvt.u32.u16 %0, x;\n\t}"
                       : "=r"(two) : "r"(scales + c));
          const uint32_t s01 = __byte_perm(two, 0, 0x4140) << 7, out = s01 & live;      // both as half precision
          asm volatile("st.shared.u16 [%0], %1;" ::"r"(st_out + c * (kTile * 2)), "h"((uint16_t)out) : "memory");
          asm volatile("st.shared.u16 [%0], %1;" ::"r"(st_out + (c + 1) * (kTile * 2)), "h"((uint16_t)(out >> 16))
                       : "memory");
          const uint32_t sc0 = __byte_perm(s01, 0, 0x1010), sc1 = __byte_perm(s01, 0, 0x3232);
          const uint32_t word[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            uint32_t v[16];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t o[4];
              decode8(word[4 * p + i], o);
#pragma unroll
              for (int m = 0; m < 4; ++m) v[4 * i + m] = mul_h2(o[m], p ? sc1 : sc0);
            }
            tmem_st_x16(at + p * 16, v);
          }
        }
        tmem_wait_st();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(bar(misc->as_full[k & 7]));
          if (NB != kExpandGroups) mbar_arrive(bar(misc->scale_full[st]));
          mbar_arrive(bar(misc->raw_empty[st]));
        }
      }
      const int kv = k - NB;
      if (kv >= 0) {
        const int c = kq * 4 + q, stv = st == 0 ? L.stages - 1 : st - 1, roundv = st == 0 ? round - 1 : round;
        // With four units a tile this group has itself expanded this very quarter for the scores: it
          // has waited for the tile, and that unit k - 2 has been used tells that its four warps have all
        // written their scales of unit k - 4; behind the last tile only that unit's own barrier does.
          ok = (kv < AVB || wait(misc->av_empty[(kv - AVB) & 3], (kv - AVB) >> 2)) &&
               (NB == kExpandGroups ? k < n_units || wait(misc->as_full[kv & 7], kv >> 3)
                                    : wait(misc->raw_full[stv], roundv) && wait(misc->scale_full[stv], roundv));
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after_sync();
        if (c < chunks) {
          uint32_t from = base + stv * L.stage + L.codes + lane * code_row + ((uint32_t)(c * 16) ^ twist);
          uint32_t sc_at = st_u32 + (stv * f.scale_row() + c) * (kTile * 2) + 4 * t;
          uint32_t col = lane_tm + COL_AV + (kv % AVB) * 64;
#pragma unroll 1
          for (int h = 0; h < 2; ++h) {                        // 64 slots each
            uint32_t w[2][4];
            ldsm_x4_trans(from, w[0]);
            ldsm_x4_trans(from + 32 * code_row, w[1]);
#pragma unroll
            for (int i2 = 0; i2 < 2; ++i2) {
              uint32_t v[4][4];
#pragma unroll
              for (int m = 0; m < 4; ++m) {
                uint32_t sc;
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(sc) : "r"(sc_at + i2 * 64 + m * 16));
                decode_pairs(w[i2][m], v[m]);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[m][i] = mul_h2(v[m][i], sc);
              }
              const uint32_t to = col + i2 * 16;
              tmem_st_16x128_x4(to, v[0][0], v[0][1], v[1][0], v[1][1], v[2][0], v[2][1], v[3][0], v[3][1]);
              tmem_st_16x128_x4(to + (16u << 16), v[0][2], v[0][3], v[1][2], v[1][3], v[2][2], v[2][3], v[3][2],
                                v[3][3]);
            }
            from += 64 * code_row;
            sc_at += 128;
            col += 32;
          }
        }
        tmem_wait_st();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(bar(misc->av_full[kv & 3]));
          mbar_arrive(bar(misc->raw_empty[stv]));
        }
      }
      if (NB == 4) {
        next_tile();
      } else {
        kq += kExpandGroups;
#pragma unroll 1
        while (kq >= NB) { kq -= NB; next_tile(); }
      }
    }
  } else {
    // ------------------------------------------------------------------ softmax and epilogue
    // Two groups of four warps: group gr owns heads [gr * NHH, (gr + 1) * NHH) of the tile's 128
    // slots, a slot per thread.  They leave the loop together (they agree on it once a tile, before
    // anything that depends on the tile's description), so the hardware barrier always completes.
    constexpr int NHH = NHP / 2;
    const int sw = warp - kSoftmaxWarp0, gr = sw >> 2, q = warp & 3, HO = gr * NHH;
    const int sidx = sw * 32 + lane, slot = q * 32 + lane;
    const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16) + HO;
    auto group_sync = [&]() { named_sync<1, kSoftmaxThreads>(); };
    auto ld_cols = [&](uint32_t addr, uint32_t (&v)[16]) {
      if (NHH == 16) tmem_ld_x16(addr, v); else tmem_ld_x8(addr, v);
    };
    auto st_cols = [&](uint32_t addr, const uint32_t (&v)[16]) {
      if (NHH == 16) tmem_st_x16(addr, v); else tmem_st_x8(addr, v);
    };
    // One value per head over the warp's 32 slots, left in red[sw][i]: halving exchanges, in each of
    // which a lane keeps half of its heads and adds the partner's share of them.
    auto reduce_heads = [&](float (&v)[NHH], bool is_max) {
      auto join = [&](float x, float y) { return is_max ? fmaxf(x, y) : x + y; };
#pragma unroll
      for (int n = NHH, o = 16; n > 1; n >>= 1, o >>= 1) {
        const bool upper = lane & o;
#pragma unroll
        for (int i = 0; i < n / 2; ++i) {
          const float keep = upper ? v[i + n / 2] : v[i], give = upper ? v[i] : v[i + n / 2];
          v[i] = join(keep, __shfl_xor_sync(0xffffffffu, give, o));
        }
      }
      float x = v[0];                                    // head (lane >> log2(32 / NHH)) of the group
#pragma unroll
      for (int o = 16 / NHH; o >= 1; o >>= 1) x = join(x, __shfl_xor_sync(0xffffffffu, x, o));
      if ((lane & (32 / NHH - 1)) == 0) misc->red[sw][lane / (32 / NHH)] = x;
    };
    auto reduced = [&](int h, bool is_max) {
      const float* x = &misc->red[(h / NHH) * 4][h % NHH];
      return is_max ? fmaxf(fmaxf(x[0], x[16]), fmaxf(x[32], x[48])) : (x[0] + x[16]) + (x[32] + x[48]);
    };
    uint8_t* const p_row = sm + L.off_p + (HO / 8) * P_SBO + slot * 16;
    float l_acc[NHH];
    for (int n = 0; n < n_tiles; ++n) {
      if (ok && sw == 3) ok = wait(misc->info_full[n % kInfo], n / kInfo) && wait(misc->s_full[n & 1], n >> 1);
      if (named_sync_or<kSoftmaxThreads>(1, !ok)) break;
      const int flags = misc->info[n % kInfo].flags;
      const int rows = slot < 64 ? misc->info[n % kInfo].rows0 : misc->info[n % kInfo].rows1;
      if (flags & kFirst) {
        if (sidx < 32) {
          const int seg = flags >> kSegShift;
          if (ok) ok = wait(misc->q_full[seg % kQRing], seg / kQRing);       // long since; for the scales
          misc->m_used[sidx] = -INFINITY;
          misc->neg_ref[sidx] = kUnset;
          misc->unit[sidx] = sidx < NHP ? misc->next_unit[seg % kQRing][sidx] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < NHH; ++i) l_acc[i] = 0.f;
        group_sync();
      }
      // Output sums of the segment: this thread's latent (lane 8j + g of a quarter holds latent 4g + j).
      auto fold = [&](bool whole, bool add) {
        const int b = misc->info[n % kInfo].b, seq_out = a.n_heads * r;
        fold_output<NHP, NB>(a.o_part + ((long long)blockIdx.x + b) * seq_out,
                             whole ? static_cast<bf16*>(a.out) + (long long)b * seq_out : nullptr, misc, lane_base + kColO, HO,
                             a.n_heads, r, q * 32 + 4 * (lane & 7) + (lane >> 3), add);
      };
      if (__builtin_expect(flags & kFold, 0)) {
        // The sums so far are set down; this tile's products then begin new ones.
        if (ok) ok = wait(misc->p_empty[(n - 1) & 1], (n - 1) >> 1);
        ok = __all_sync(0xffffffffu, ok);
        if (sidx < NHP) {
          const float m = misc->m_used[sidx], m_old = misc->m_fold[sidx];
          misc->fac[sidx] = m == m_old ? 1.f : exp2f(m_old - m);        // of use from the second time on
          misc->m_fold[sidx] = m;
        }
        group_sync();
        if (ok) {
          tc_fence_after_sync();
          fold(false, flags & kFolded);
        }
        group_sync();                                    // fac may be rewritten
      }
      float s[NHH];
      {
        uint32_t sp[16];
        tc_fence_after_sync();
        ld_cols(lane_base + kColS + (n & 1) * 32, sp);
        tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < NHH; ++i) s[i] = __uint_as_float(sp[i]);
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(misc->s_empty[n & 1]));
      }
      const bool live = (slot & 63) < rows, full = __all_sync(0xffffffffu, live);
      // x = score - reference + shift in log2 units, kept in place of the raw score.
      float top = -INFINITY;
      auto offset_scores = [&](float (&x)[NHH]) {
#pragma unroll
        for (int i = 0; i < NHH; i += 4) {
          const float4 u = *reinterpret_cast<const float4*>(&misc->unit[HO + i]);
          const float4 o = *reinterpret_cast<const float4*>(&misc->neg_ref[HO + i]);
          x[i] = fmaf(s[i], u.x, o.x);
          x[i + 1] = fmaf(s[i + 1], u.y, o.y);
          x[i + 2] = fmaf(s[i + 2], u.z, o.z);
          x[i + 3] = fmaf(s[i + 3], u.w, o.w);
        }
        if (!full) {                                     // only a sequence's last tile
#pragma unroll
          for (int i = 0; i < NHH; ++i) x[i] = live ? x[i] : -INFINITY;
        }
      };
      uint32_t pb[NHH / 2];
      float add[NHH];
      offset_scores(add);
#pragma unroll
      for (int i = 0; i < NHH; ++i) top = fmaxf(top, add[i]);
      auto probabilities = [&]() {
#pragma unroll
        for (int i = 0; i < NHH; i += 2) {
          add[i] = ex2_approx(add[i]);
          add[i + 1] = ex2_approx(add[i + 1]);
          const __half2 x = __floats2half2_rn(add[i], add[i + 1]);
          pb[i / 2] = *reinterpret_cast<const uint32_t*>(&x);
        }
      };
      // P as the MN-major, un-swizzled B operand: eight heads of a slot are 16 bytes, eight slots
      // follow one another, groups of eight heads are P_SBO apart.
      auto store_probabilities = [&]() {
#pragma unroll
        for (int i = 0; i < NHH / 8; ++i)
          *reinterpret_cast<uint4*>(p_row + (n & 1) * P_BYTES + i * P_SBO) =
              make_uint4(pb[4 * i], pb[4 * i + 1], pb[4 * i + 2], pb[4 * i + 3]);
      };
      if (sw == 3 && ok) ok = wait(misc->p_empty[n & 1], (n >> 1) + 1);    // value products of tile n - 2
      if (named_sync_or<kSoftmaxThreads>(1, top > kShift + kRescale)) {
        // Rare: some reference has to rise (always at a segment's first tile).
        {
          float x[NHH];
#pragma unroll
          for (int i = 0; i < NHH; ++i) x[i] = live ? s[i] * misc->unit[HO + i] : -INFINITY;
          reduce_heads(x, true);
        }
        group_sync();
        if (sidx < NHP) {
          const float mt = reduced(sidx, true), m_old = misc->m_used[sidx];
          const float m_new = mt > m_old + kRescale ? mt : m_old;
          misc->m_used[sidx] = m_new;
          misc->neg_ref[sidx] = m_new == -INFINITY ? kUnset : kShift - m_new;
          misc->fac[sidx] = m_new == m_old ? 1.f : exp2f(m_old - m_new);       // 0 from minus infinity
        }
        group_sync();
#pragma unroll
        for (int i = 0; i < NHH; ++i) l_acc[i] *= misc->fac[HO + i];
        if (!(flags & (kFirst | kFold))) {
          // O is scaled to the old references: wait for the previous tile's products, rescale.
          if (ok) ok = wait(misc->p_empty[(n - 1) & 1], (n - 1) >> 1);
          ok = __all_sync(0xffffffffu, ok);              // TMEM accesses are whole-warp operations
          if (ok) {
            tc_fence_after_sync();
#pragma unroll 1
            for (int mb = 0; mb < NB; ++mb) {
              uint32_t ov[16];
              ld_cols(lane_base + kColO + mb * NHP, ov);
              tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < NHH; ++i) ov[i] = __float_as_uint(__uint_as_float(ov[i]) * misc->fac[HO + i]);
              st_cols(lane_base + kColO + mb * NHP, ov);
            }
            tmem_wait_st();
          }
        }
        offset_scores(add);
        group_sync();                                    // fac / red may be rewritten
      }
      probabilities();
      if (ok) store_probabilities();
#pragma unroll
      for (int i = 0; i < NHH; ++i) l_acc[i] += add[i];
      fence_proxy_async_smem();
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(misc->p_full[n & 1]));
      if (!(flags & kLast)) continue;

      // ---- end of a segment
      const int b = misc->info[n % kInfo].b, g = g0 + n;
      const bool whole = prefix[b] >= g0 && g + 1 == prefix[b + 1];
      const int c0 = share_owner(prefix[b], total, ctas), part = (int)blockIdx.x + b;
      reduce_heads(l_acc, false);
      group_sync();
      if (sidx < NHP) misc->fac[sidx] = reduced(sidx, false);     // denominators
      group_sync();
      if (ok && sidx < a.n_heads) {
        const float l = misc->fac[sidx], m = misc->m_used[sidx] - kShift;
        if (flags & kFoldedNow) {
          const float m_set = misc->m_fold[sidx], m_now = misc->m_used[sidx];
          misc->fac[sidx] = m_set == m_now ? 1.f : exp2f(m_set - m_now);
        }
        misc->unit[sidx] = 1.f / l;                      // the units have done their work in this segment
        if (whole) {
          if (a.lse) a.lse[(long long)b * a.n_heads + sidx] = (m + log2f(l)) * 0.69314718055994531f;
        } else {
          a.ml_part[((long long)part * a.n_heads + sidx) * 2] = m;
          a.ml_part[((long long)part * a.n_heads + sidx) * 2 + 1] = l;
        }
      }
      if (ok && sidx == 0 && g + 1 == prefix[b + 1])
        a.seq_parts[b] = whole ? make_int2(0, 0) : make_int2(c0 + b, (int)blockIdx.x - c0 + 1);
      group_sync();
      if (ok) ok = wait(misc->p_empty[n & 1], n >> 1);           // the last value products
      ok = __all_sync(0xffffffffu, ok);
      if (ok && __builtin_expect(flags & kFoldedNow, 0)) {
        tc_fence_after_sync();
        fold(whole, true);
        tc_fence_before_sync();
      } else if (ok) {
        tc_fence_after_sync();
        // Lane 8j + g of a quarter holds latent 4g + j.
        const int lat = q * 32 + 4 * (lane & 7) + (lane >> 3);
        const long long at = (long long)(whole ? b : part) * a.n_heads * r + lat;
        constexpr int STEP = NB > 1 ? 2 : 1;             // blocks whose loads are in flight together
#pragma unroll 1
        for (int mb = 0; mb < NB; mb += STEP) {
          uint32_t ov[STEP][16];
#pragma unroll
          for (int j = 0; j < STEP; ++j)
            if (mb + j < NB) ld_cols(lane_base + kColO + (mb + j) * NHP, ov[j]);
          tmem_wait_ld();
#pragma unroll
          for (int j = 0; j < STEP; ++j) {
            if (mb + j >= NB || (mb + j) * 128 + lat >= r) continue;
#pragma unroll
            for (int i = 0; i < NHH; ++i) {
              if (HO + i >= a.n_heads) break;
              const long long e = at + (HO + i) * r + (mb + j) * 128;
              const float v = __uint_as_float(ov[j][i]);
              if (whole) static_cast<bf16*>(a.out)[e] = __float2bfloat16_rn(v * misc->unit[HO + i]);
              else a.o_part[e] = v;
            }
          }
        }
        tc_fence_before_sync();
      }
      group_sync();                                      // fac, unit and the references may be rewritten
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
    tmem_dealloc(misc->tmem_base, kTmemCols);
  }
}

// Self-test of the bounded wait: one CTA whose only wait, on a barrier that expects an arrival which never
// comes, gives up after 2^21 cycles (about a millisecond) instead of 2^31, and what became of it in the error
// word that the combine reads.
__global__ void __launch_bounds__(64) wait_timeout_selftest_kernel(int* error_word) {
  __shared__ unsigned long long bar;
  if (threadIdx.x == 0) {
    ptx::mbar_init(ptx::smem_u32(&bar), 1);
    ptx::mbar_fence_init();
  }
  __syncthreads();
  const bool ok = ptx::mbar_wait_compact<1u << 21>(ptx::smem_u32(&bar), 0);
  const bool failed = __syncthreads_or(!ok);
  if (threadIdx.x == 0) *error_word = failed;
}

}  // namespace qp
}  // namespace mtla
