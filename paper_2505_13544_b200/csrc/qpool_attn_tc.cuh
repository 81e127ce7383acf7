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
// probabilities, and the kernel is bound by the instructions of the expansion (conversion, scale, and
// for the values the pairing): about 60 per slot and warp lane, against 8 of matrix work.
//
// A head count of 16 or 32 is the matrix instructions' N, so heads are not padded further.  The RoPE
// keys go from the pool to the score product as they are (bf16, shared memory, hardware swizzle).
//
// Queries arrive as an image of the B operand that qpool_query_kernel has written (half precision
// scaled by a power of two per head, swizzled), so that a segment's query is one bulk copy.
//
// Roles (28 warps): warps 0-3 score issuers, one per 128 latents, each with its own accumulator
// (one thread issues a matrix instruction about every hundred cycles, several times slower than
// these execute); warp 4 producer; warps 5-6 value issuers; warps 8-11 expansion for the scores;
// warps 12-19 for the values, a page of the tile each four; warps 20-27 softmax and epilogue.
// The online softmax raises a head's reference only when a tile exceeds it by 2^8, found by a flag that is
// collected while the probabilities are already being formed.  Probabilities are kept times 2^7:
// with the 2^8 they stay inside half precision.
//
// Every wait is bounded; after a time-out the roles unwind and qpool_combine_kernel answers with NaN.
#pragma once

#include "qpool_attn.cuh"

namespace mtla {
namespace qp {
namespace tc {

constexpr int kTile = 128;                  // slots per tile: two pages
constexpr int kThreads = 896;
constexpr int kStages = 3;
constexpr int kMaxBatch = 1022;             // prefix sums kept in shared memory
constexpr int kProducerWarp = 4, kFirstValueIssuer = 5, kValueIssuers = 2;
constexpr int kScoreWarp0 = 8, kScoreWarps = 4, kValueWarp0 = 12, kValueWarps = 8;
constexpr int kSoftmaxWarp0 = 20, kSoftmaxThreads = 256;
constexpr int kInfo = 8;                    // ring of tile descriptions, deeper than any role's lag
// TMEM columns: four score accumulators, four output blocks, two operand buffers each.
constexpr int kTmemCols = 512;
constexpr int kColS = 0, kColO = 128, kColAs = 256, kColAv = 384;
constexpr float kShift = 7.f, kRescale = 8.f;
constexpr int kRegsIssuer = 40, kRegsWorker = 80;
constexpr int kRegsAtLaunch = 65536 / kThreads / 8 * 8;
static_assert(256 * kRegsIssuer + (kThreads - 256) * kRegsWorker <= kThreads * kRegsAtLaunch,
              "register re-allocation exceeds the CTA's pool");

struct TileInfo {
  int b;
  int flags;                 // 1: first tile of a segment, 2: last
  int rows0, rows1;          // slots of the tile's two pages
};

struct Misc {
  unsigned long long raw_full[kStages], raw_empty[kStages], scale_full[kStages];
  // Operand buffers: "empty" per buffer; "full" per quarter of r and parity of the tile, so that its
  // one reader sees every phase and the writers, two buffers ahead at most, never lead by two.
  unsigned long long as_full[2][4], as_empty[2], av_full[2][4], av_empty[2];
  unsigned long long s_full, s_empty, p_full[2], p_empty[2], q_full, q_empty;
  unsigned long long info_full[kInfo], flag_bar[2], group_sync;
  uint32_t tmem_base;
  int abort_word;
  int exceed_flag[2];
  int warp_sums[32];
  TileInfo info[kInfo];
  float m_used[32], unit[32], fac[32];
  float red[8][16];
};
static_assert(sizeof(Misc) <= 2048, "misc region too small");

struct Layout {
  int codes, scales, keys;                  // offsets in a stage
  int stage;
  int off_q, q_bytes, off_p, off_st, off_misc, off_prefix, total;
  __host__ __device__ Layout(const Format& f, int nhp, int batch) {
    keys = 0;                                            // swizzled operand: 1024-byte aligned
    codes = kTile * f.key_row();
    scales = codes + kTile * f.code_row();
    stage = (scales + kTile * f.scale_row() + 1023) / 1024 * 1024;
    off_q = kStages * stage;
    q_bytes = nhp * 2 * (f.r + f.dr);
    off_p = off_q + (q_bytes + 1023) / 1024 * 1024;
    off_st = off_p + 2 * kTile * nhp * 2;
    off_misc = off_st + kStages * f.scale_row() * kTile * 2;
    off_prefix = off_misc + 2048;
    total = off_prefix + (batch + 1) * 4 + 1024;         // slack for the alignment of the base
  }
};

}  // namespace tc

// Queries -> the image of the score product's B operand: per sequence r / 64 panels [NHP][64] half
// precision with the 128-byte swizzle and one panel [NHP][d_R] bf16 (128- or 64-byte swizzle), a head's
// row scaled by the power of two that brings its largest element into [2^14, 2^15); heads that do not
// exist are zero.  A warp per head.
constexpr int kQueryThreads = 256;
template <int NHP>
__global__ void __launch_bounds__(kQueryThreads) qpool_query_kernel(AttnArgs a) {
  const int b = blockIdx.y, lane = threadIdx.x & 31, h = blockIdx.x * (kQueryThreads / 32) + (threadIdx.x >> 5);
  const int r = a.f.r, dr = a.f.dr, n8 = (r + dr) / 8;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  if (b == 0 && blockIdx.x == 0 && threadIdx.x == 0) *a.error_word = 0;
  const bf16* q = static_cast<const bf16*>(a.q) + ((long long)b * a.n_heads + h) * (r + dr);
  float v[3][8];                                  // up to 72 runs of eight over 32 lanes
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const int c = lane + 32 * i;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
    if (c < n8 && h < a.n_heads) load_vec(q + 8 * c, v[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[i][j]) & 0x7fffffffu);
  }
  top = __reduce_max_sync(0xffffffffu, top);
  const bool fine = top > 0 && top < 0x7f800000u;
  const int e = fine ? 14 - ilogbf(__uint_as_float(top)) : 0;
  if (lane == 0) a.q_unit[b * 32 + h] = ldexpf(a.scale_log2, -e);
  uint8_t* img = a.q_image + (long long)b * NHP * 2 * (r + dr);
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const int c = lane + 32 * i;
    if (c >= n8) break;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] = ldexpf(v[i][j], e);
    if (8 * c < r) {
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const __half2 x = __floats2half2_rn(v[i][2 * j], v[i][2 * j + 1]);
        w[j] = *reinterpret_cast<const uint32_t*>(&x);
      }
      *reinterpret_cast<uint4*>(img + (c >> 3) * NHP * 128 + h * 128 + ((c ^ h) & 7) * 16) =
          make_uint4(w[0], w[1], w[2], w[3]);
    } else {
      const int k = c - r / 8;
      uint8_t* p = img + NHP * 2 * r + h * 2 * dr + (k ^ a.f.key_swizzle(h)) * 16;
      store_vec(reinterpret_cast<bf16*>(p), v[i]);
    }
  }
}

// NHP: heads padded to 16 or 32.  NB: ceil(r / 128).
template <int NHP, int NB>
__global__ void __launch_bounds__(tc::kThreads, 1) qpool_attend_tc_kernel(AttnArgs a) {
  using namespace tc;
  using namespace ptx;
  constexpr uint32_t IDESC_S = make_idesc_f16(128, NHP, 0, 0), IDESC_K = make_idesc_bf16(128, NHP, 0, 0);
  constexpr uint32_t IDESC_V = make_idesc_f16(128, NHP, 0, 1);
  constexpr uint32_t P_BYTES = kTile * NHP * 2, P_SBO = kTile * 16;   // bytes between groups of 8 heads
  extern __shared__ uint8_t smem_raw[];
  const Format f = a.f;
  const int r = f.r, dr = f.dr;
  const Layout L(f, NHP, a.batch);
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* sm = smem_raw + (base - raw);
  Misc* misc = reinterpret_cast<Misc*>(sm + L.off_misc);
  int* prefix = reinterpret_cast<int*>(sm + L.off_prefix);
  volatile int* abort_word = &misc->abort_word;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto bar = [&](unsigned long long& p) { return smem_u32(&p); };

  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(bar(misc->raw_full[i]), 1);
      mbar_init(bar(misc->raw_empty[i]), kScoreWarps + kValueWarps + NB);
      mbar_init(bar(misc->scale_full[i]), kScoreWarps);
    }
    for (int i = 0; i < 4; ++i) {
      for (int j = 0; j < 2; ++j) {
        mbar_init(bar(misc->as_full[j][i]), kScoreWarps);
        mbar_init(bar(misc->av_full[j][i]), kValueWarps);
      }
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(misc->as_empty[i]), 1);
      mbar_init(bar(misc->av_empty[i]), 1);
      mbar_init(bar(misc->p_full[i]), kSoftmaxThreads);
      mbar_init(bar(misc->p_empty[i]), kValueIssuers);
      mbar_init(bar(misc->flag_bar[i]), kSoftmaxThreads);
      misc->exceed_flag[i] = 0;
    }
    for (int i = 0; i < kInfo; ++i) mbar_init(bar(misc->info_full[i]), 1);
    mbar_init(bar(misc->s_full), NB);
    mbar_init(bar(misc->s_empty), kSoftmaxThreads);
    mbar_init(bar(misc->q_full), 1);
    mbar_init(bar(misc->q_empty), NB);
    mbar_init(bar(misc->group_sync), kSoftmaxThreads);
    misc->abort_word = 0;
    mbar_fence_init();
  }
  if (warp == kProducerWarp) tmem_alloc(smem_u32(&misc->tmem_base), kTmemCols);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = misc->tmem_base;
  grid_launch_dependents();      // this CTA owns its TMEM columns (see decode_attn_tc.cuh)
  grid_dependency_wait();

  const long long total = tile_prefix<2>(a, prefix, misc->warp_sums, kThreads);
  const int ctas = (int)(total < gridDim.x ? total : gridDim.x);
  int g0 = 0, g1 = 0;
  if ((int)blockIdx.x < ctas) {
    g0 = share_begin(blockIdx.x, total, ctas);
    g1 = share_begin(blockIdx.x + 1, total, ctas);
  }
  const int n_tiles = g1 - g0;
  const uint32_t q_u32 = base + L.off_q, p_u32 = base + L.off_p, st_u32 = base + L.off_st;
  auto stage_of = [&](int n) { return base + (n % kStages) * L.stage; };
  auto wait = [&](unsigned long long& b, int phase, int code) {
    return mbar_wait(bar(b), phase & 1, abort_word, a.error_word, code);
  };

  if (n_tiles == 0) {
    // nothing to do; the CTA falls through to the common end
  } else if (warp < kScoreWarp0) {
    reg_dealloc<kRegsIssuer>();
    if (warp == kProducerWarp && lane == 0) {
      // ---------------------------------------------------------------- producer
      int b = find_seq(prefix, a.batch, g0), seg = 0;
      for (int n = 0; n < n_tiles; ++n) {
        const int g = g0 + n;
        while (prefix[b + 1] <= g) ++b;
        const int tile = g - prefix[b], slots = a.slots[b];
        const bool first = n == 0 || tile == 0, last = n + 1 == n_tiles || g + 1 == prefix[b + 1];
        const int st = n % kStages;
        int page[2], rows[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int t = 2 * tile + i, have = slots - t * kPageRows;
          page[i] = have > 0 && t < a.width ? __ldg(a.table + (long long)b * a.width + t) : -1;
          rows[i] = page[i] >= 0 && page[i] < a.n_pages ? min(have, kPageRows) : 0;
        }
        if (!wait(misc->raw_empty[st], (n / kStages) + 1, 1)) break;
        TileInfo& info = misc->info[n % kInfo];
        info.b = b;
        info.flags = (first ? 1 : 0) | (last ? 2 : 0);
        info.rows0 = rows[0];
        info.rows1 = rows[1];
        mbar_arrive(bar(misc->info_full[n % kInfo]));
        uint32_t bytes = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i)
          bytes += rows[i] * (f.code_row() + f.key_row()) + (rows[i] * f.scale_row() + 15) / 16 * 16;
        const uint32_t full = bar(misc->raw_full[st]), dst = stage_of(n);
        mbar_arrive_expect_tx(full, bytes);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (rows[i] == 0) continue;
          const uint8_t* src = a.pages + (long long)page[i] * f.page_bytes();
          bulk_load(dst + L.keys + i * kPageRows * f.key_row(), src + f.off_keys(), rows[i] * f.key_row(), full);
          bulk_load(dst + L.codes + i * kPageRows * f.code_row(), src, rows[i] * f.code_row(), full);
          bulk_load(dst + L.scales + i * kPageRows * f.scale_row(), src + f.off_scales(),
                    (rows[i] * f.scale_row() + 15) / 16 * 16, full);
        }
        if (first) {
          // The segment's queries, once the score products of the segment before are done.
          if (!wait(misc->q_empty, seg + 1, 2)) break;
          mbar_arrive_expect_tx(bar(misc->q_full), L.q_bytes);
          bulk_load(q_u32, a.q_image + (long long)b * L.q_bytes, L.q_bytes, bar(misc->q_full));
          ++seg;
        }
      }
    } else if (warp < NB && lane == 0) {
      // ---------------------------------------------------------------- score issuer kq
      const int kq = warp;
      const uint32_t d = tmem + kColS + kq * 32;
      const int steps = min(8, (r - kq * 128) / 16);       // k-steps of 16 latents
      int seg = 0;
      for (int n = 0; n < n_tiles; ++n) {
        const int st = n % kStages, k = n * NB + kq, sb = k & 1;
        if (!wait(misc->raw_full[st], n / kStages, 3)) break;
        const int flags = misc->info[n % kInfo].flags;
        if (flags & 1) {
          if (!wait(misc->q_full, seg, 4)) break;
          ++seg;
        }
        if (!wait(misc->s_empty, n + 1, 5)) break;
        tc_fence_after_sync();
        uint32_t acc = 0;
        // RoPE part: its k-steps are dealt out to the issuers.
        const uint32_t key = stage_of(n) + L.keys, qk = q_u32 + NHP * 2 * r;
        const uint64_t mode = dr == 64 ? kSwizzle128B : kSwizzle64B;
        const uint32_t sbo = 8 * f.key_row();
        for (int ks = kq; ks < dr / 16; ks += NB) {
          mma_bf16_ss(d, make_smem_desc(key + ks * 32, 16, sbo, mode), make_smem_desc(qk + ks * 32, 16, sbo, mode),
                      IDESC_K, acc);
          acc = 1;
        }
        if (!wait(misc->as_full[n & 1][kq], n >> 1, 6)) break;
        tc_fence_after_sync();
        for (int ks = 0; ks < steps; ++ks) {
          const uint32_t panel = q_u32 + (kq * 2 + (ks >> 2)) * NHP * 128 + (ks & 3) * 32;
          mma_f16_ts(d, tmem + kColAs + sb * 64 + ks * 8, make_smem_desc(panel, 16, 1024, kSwizzle128B), IDESC_S, acc);
          acc = 1;
        }
        mma_commit(bar(misc->as_empty[sb]));
        mma_commit(bar(misc->s_full));
        mma_commit(bar(misc->raw_empty[st]));
        if (flags & 2) mma_commit(bar(misc->q_empty));
      }
    } else if (warp >= kFirstValueIssuer && warp < kFirstValueIssuer + kValueIssuers && lane == 0) {
      // ---------------------------------------------------------------- value issuer j: blocks j, j + 2
      const int j = warp - kFirstValueIssuer;
      bool ok = true;
      for (int n = 0; n < n_tiles && ok; ++n) {
        ok = wait(misc->p_full[n & 1], n >> 1, 7);
        if (!ok) break;
        const int flags = misc->info[n % kInfo].flags;      // p_full: written long before by the producer
        for (int mb = j; mb < NB && ok; mb += kValueIssuers) {
          const int k = n * NB + mb, vb = k & 1;
          ok = wait(misc->av_full[n & 1][mb], n >> 1, 8);
          if (!ok) break;
          tc_fence_after_sync();
#pragma unroll
          for (int ks = 0; ks < kTile / 16; ++ks)
            mma_f16_ts(tmem + kColO + mb * 32, tmem + kColAv + vb * 64 + ks * 8,
                       make_smem_desc(p_u32 + (n & 1) * P_BYTES + ks * 256, 128, P_SBO, kSwizzleNone), IDESC_V,
                       (flags & 1) && ks == 0 ? 0u : 1u);
          mma_commit(bar(misc->av_empty[vb]));
        }
        if (ok) mma_commit(bar(misc->p_empty[n & 1]));
      }
    }
  } else if (warp < kValueWarp0) {
    // ------------------------------------------------------------------ expansion for the scores
    reg_alloc<kRegsWorker>();
    const int q = warp & 3, slot = q * 32 + lane, half = slot >> 6, row = slot & 63;
    const int cmask = f.code_mask(), chunks = r / kGroup;
    const uint32_t lane_as = tmem + ((uint32_t)(q * 32) << 16) + kColAs;
    bool ok = true;
    for (int n = 0; n < n_tiles; ++n) {
      const int st = n % kStages;
      ok = __all_sync(0xffffffffu, wait(misc->raw_full[st], n / kStages, 9));
      if (!ok) break;
      const TileInfo& info = misc->info[n % kInfo];
      const bool live = row < (half ? info.rows1 : info.rows0);
      const uint32_t stage = stage_of(n);
      const uint32_t codes = stage + L.codes + slot * f.code_row(), scales = stage + L.scales + slot * f.scale_row();
      const uint32_t st_out = st_u32 + st * f.scale_row() * kTile * 2 + slot * 2;
      // The scales as half precision, a group's 128 slots in a row, for the value warps; zero
      // where there is no slot, so that whatever its codes are, the product is zero.
      for (int c = 0; c < chunks; c += 2) {
        uint32_t two;
        asm volatile("{\n\t.reg .u16 x;\n\tld.shared.u16 x, [%1];\n\tcvt.u32.u16 %0, x;\n\t}" : "=r"(two) : "r"(scales + c));
        const uint32_t s0 = live ? (two & 0xffu) << 7 : 0u, s1 = live ? (two >> 8) << 7 : 0u;
        asm volatile("st.shared.u16 [%0], %1;" ::"r"(st_out + c * kTile * 2), "h"((uint16_t)s0) : "memory");
        asm volatile("st.shared.u16 [%0], %1;" ::"r"(st_out + (c + 1) * kTile * 2), "h"((uint16_t)s1) : "memory");
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(misc->scale_full[st]));
      for (int kq = 0; kq < NB; ++kq) {
        const int k = n * NB + kq, sb = k & 1;
        ok = __all_sync(0xffffffffu, wait(misc->as_empty[sb], (k >> 1) + 1, 10));
        if (!ok) break;
        tc_fence_after_sync();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int c = kq * 4 + i;
          if (c >= chunks) break;
          const uint4 w = lds128(codes + (c ^ (row & cmask)) * 16);
          const uint32_t sc = scale_pair(lds_u8(scales + c));
          const uint32_t word[4] = {w.x, w.y, w.z, w.w};
          uint32_t v[16];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t o[4];
            decode8(word[j], o);
#pragma unroll
            for (int m = 0; m < 4; ++m) v[4 * j + m] = mul_h2(o[m], sc);
          }
          tmem_st_x16(lane_as + sb * 64 + i * 16, v);
        }
        tmem_wait_st();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(misc->as_full[n & 1][kq]));
      }
      if (!ok) break;
      if (lane == 0) mbar_arrive(bar(misc->raw_empty[st]));
    }
  } else if (warp < kSoftmaxWarp0) {
    // ------------------------------------------------------------------ expansion for the values
    reg_alloc<kRegsWorker>();
    const int q = warp & 3, half = (warp - kValueWarp0) >> 2, t = lane & 3;
    const int cmask = f.code_mask(), chunks = r / kGroup;
    const uint32_t lane_av = tmem + ((uint32_t)(q * 32) << 16) + kColAv + half * 32;
    bool ok = true;
    for (int n = 0; n < n_tiles; ++n) {
      const int st = n % kStages;
      ok = __all_sync(0xffffffffu, wait(misc->raw_full[st], n / kStages, 11) &&
                                       wait(misc->scale_full[st], n / kStages, 12));
      if (!ok) break;
      const uint32_t codes = stage_of(n) + L.codes + half * kPageRows * f.code_row();
      const uint32_t sts = st_u32 + st * f.scale_row() * kTile * 2 + (half * kPageRows + 2 * t) * 2;
      for (int mb = 0; mb < NB; ++mb) {
        const int k = n * NB + mb, vb = k & 1, c = mb * 4 + q;
        ok = __all_sync(0xffffffffu, wait(misc->av_empty[vb], (k >> 1) + 1, 13));
        if (!ok) break;
        tc_fence_after_sync();
        if (c < chunks) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int lr = h * 32 + lane;
            uint32_t w[4], v[4][4];
            ldsm_x4_trans(codes + lr * f.code_row() + (c ^ (lr & cmask)) * 16, w);
#pragma unroll
            for (int m = 0; m < 4; ++m) {
              uint32_t sc;
              asm volatile("ld.shared.u32 %0, [%1];" : "=r"(sc) : "r"(sts + (c * kTile + h * 32 + m * 8) * 2));
              decode_pairs(w[m], v[m]);
#pragma unroll
              for (int j = 0; j < 4; ++j) v[m][j] = mul_h2(v[m][j], sc);
            }
            const uint32_t col = lane_av + vb * 64 + h * 16;
            tmem_st_16x128_x4(col, v[0][0], v[0][1], v[1][0], v[1][1], v[2][0], v[2][1], v[3][0], v[3][1]);
            tmem_st_16x128_x4(col + (16u << 16), v[0][2], v[0][3], v[1][2], v[1][3], v[2][2], v[2][3], v[3][2], v[3][3]);
          }
        }
        tmem_wait_st();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(misc->av_full[n & 1][mb]));
      }
      if (!ok) break;
      if (lane == 0) mbar_arrive(bar(misc->raw_empty[st]));
    }
  } else {
    // ------------------------------------------------------------------ softmax and epilogue
    // Two groups of four warps: group gr owns heads [gr * NHH, (gr + 1) * NHH) of the tile's 128
    // slots, a slot per thread.
    reg_alloc<kRegsWorker>();
    constexpr int NHH = NHP / 2;
    const int sw = warp - kSoftmaxWarp0, gr = sw >> 2, q = warp & 3, HO = gr * NHH;
    const int sidx = sw * 32 + lane, slot = q * 32 + lane;
    const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16) + HO;
    bool ok = true;
    int sync_phase = 0;
    auto group_sync = [&]() {
      mbar_arrive(bar(misc->group_sync));
      if (ok) ok = wait(misc->group_sync, sync_phase, 14);
      ++sync_phase;
    };
    auto ld_cols = [&](uint32_t addr, uint32_t (&v)[16]) {
      if (NHH == 16) tmem_ld_x16(addr, v); else tmem_ld_x8(addr, v);
    };
    auto st_cols = [&](uint32_t addr, const uint32_t (&v)[16]) {
      if (NHH == 16) tmem_st_x16(addr, v); else tmem_st_x8(addr, v);
    };
    // One value per head over the warp's 32 slots, left in red[sw][i].
    auto reduce_heads = [&](const float (&v)[NHH], bool is_max) {
#pragma unroll
      for (int i = 0; i < NHH; ++i) {
        float x = v[i];
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) {
          const float y = __shfl_xor_sync(0xffffffffu, x, o);
          x = is_max ? fmaxf(x, y) : x + y;
        }
        if (lane == 0) misc->red[sw][i] = x;
      }
    };
    auto reduced = [&](int h, bool is_max) {
      const float* x = &misc->red[(h / NHH) * 4][h % NHH];
      return is_max ? fmaxf(fmaxf(x[0], x[16]), fmaxf(x[32], x[48])) : (x[0] + x[16]) + (x[32] + x[48]);
    };
    float l_acc[NHH];
    for (int n = 0; n < n_tiles; ++n) {
      if (ok) ok = wait(misc->info_full[n % kInfo], n / kInfo, 15);
      const TileInfo info = misc->info[n % kInfo];
      const bool seg_first = info.flags & 1, seg_last = info.flags & 2;
      const bool live = (slot & 63) < (slot < 64 ? info.rows0 : info.rows1);
      if (seg_first) {
        if (sidx < 32) {
          misc->m_used[sidx] = -INFINITY;
          misc->unit[sidx] = sidx < NHP ? a.q_unit[info.b * 32 + sidx] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < NHH; ++i) l_acc[i] = 0.f;
        group_sync();
      }
      float s[NHH];
#pragma unroll
      for (int i = 0; i < NHH; ++i) s[i] = 0.f;
      if (ok) ok = wait(misc->s_full, n, 16);
      ok = __all_sync(0xffffffffu, ok);                  // TMEM accesses are whole-warp operations
      if (ok) {
        tc_fence_after_sync();
        uint32_t sp[NB > 1 ? 2 : 1][16];
#pragma unroll
        for (int k = 0; k < NB; k += 2) {
          ld_cols(lane_base + kColS + k * 32, sp[0]);
          if (k + 1 < NB) ld_cols(lane_base + kColS + (k + 1) * 32, sp[NB > 1 ? 1 : 0]);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < NHH; ++i) {
            s[i] += __uint_as_float(sp[0][i]);
            if (k + 1 < NB) s[i] += __uint_as_float(sp[NB > 1 ? 1 : 0][i]);
          }
        }
        tc_fence_before_sync();
      }
      mbar_arrive(bar(misc->s_empty));
      float m_ref[NHH];
      bool exceed = false;
#pragma unroll
      for (int i = 0; i < NHH; ++i) {
        s[i] = live ? s[i] * misc->unit[HO + i] : -INFINITY;
        m_ref[i] = misc->m_used[HO + i];
        exceed |= s[i] > m_ref[i] + kRescale;
      }
      if (exceed) misc->exceed_flag[n & 1] = 1;
      mbar_arrive(bar(misc->flag_bar[n & 1]));

      float psum[NHH];                                   // unrounded probabilities
      uint32_t pb[NHH / 2];
      auto probabilities = [&]() {
#pragma unroll
        for (int i = 0; i < NHH; i += 2) {
          // Nothing visible so far (reference still minus infinity): every term is 0, or NaN.
          const float r0 = m_ref[i] == -INFINITY ? -kShift : m_ref[i] - kShift;
          const float r1 = m_ref[i + 1] == -INFINITY ? -kShift : m_ref[i + 1] - kShift;
          psum[i] = ex2_approx(s[i] - r0);
          psum[i + 1] = ex2_approx(s[i + 1] - r1);
          const __half2 x = __floats2half2_rn(psum[i], psum[i + 1]);
          pb[i / 2] = *reinterpret_cast<const uint32_t*>(&x);
        }
      };
      // P as the MN-major, un-swizzled B operand: eight heads of a slot are 16 bytes, eight slots
      // follow one another, groups of eight heads are P_SBO apart.
      auto store_probabilities = [&]() {
        uint8_t* d = sm + L.off_p + (n & 1) * P_BYTES + (HO / 8) * P_SBO + slot * 16;
#pragma unroll
        for (int i = 0; i < NHH / 8; ++i)
          *reinterpret_cast<uint4*>(d + i * P_SBO) = make_uint4(pb[4 * i], pb[4 * i + 1], pb[4 * i + 2], pb[4 * i + 3]);
      };
      probabilities();
      if (ok) ok = wait(misc->p_empty[n & 1], (n >> 1) + 1, 17);     // value products of tile n - 2
      if (ok) store_probabilities();
      if (ok) ok = wait(misc->flag_bar[n & 1], n >> 1, 18);
      if (ok && misc->exceed_flag[n & 1]) {
        // Rare: some reference has to rise (always at a segment's first tile).  Everybody is here:
        // the flag is read after all arrivals.
        reduce_heads(s, true);
        group_sync();
        if (sidx == 0) misc->exceed_flag[n & 1] = 0;
        if (sidx < NHP) {
          const float mt = reduced(sidx, true), m_old = misc->m_used[sidx];
          const float m_new = mt > m_old + kRescale ? mt : m_old;
          misc->m_used[sidx] = m_new;
          misc->fac[sidx] = m_new == m_old ? 1.f : exp2f(m_old - m_new);       // 0 from minus infinity
        }
        group_sync();
#pragma unroll
        for (int i = 0; i < NHH; ++i) {
          m_ref[i] = misc->m_used[HO + i];
          l_acc[i] *= misc->fac[HO + i];
        }
        if (!seg_first) {
          // O is scaled to the old references: wait for the previous tile's products, rescale.
          if (ok) ok = wait(misc->p_empty[(n - 1) & 1], (n - 1) >> 1, 19);
          ok = __all_sync(0xffffffffu, ok);
          if (ok) {
            tc_fence_after_sync();
            for (int mb = 0; mb < NB; ++mb) {
              uint32_t ov[16];
              ld_cols(lane_base + kColO + mb * 32, ov);
              tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < NHH; ++i) ov[i] = __float_as_uint(__uint_as_float(ov[i]) * misc->fac[HO + i]);
              st_cols(lane_base + kColO + mb * 32, ov);
            }
            tmem_wait_st();
          }
        }
        probabilities();
        if (ok) store_probabilities();
        group_sync();                                    // fac / red may be rewritten
      }
#pragma unroll
      for (int i = 0; i < NHH; ++i) l_acc[i] += psum[i];
      if (ok) {
        fence_proxy_async_smem();
        tc_fence_before_sync();
        mbar_arrive(bar(misc->p_full[n & 1]));
      }
      if (!seg_last) continue;

      // ---- end of a segment
      const int b = info.b, g = g0 + n;
      const bool whole = prefix[b] >= g0 && g + 1 == prefix[b + 1];
      const int c0 = share_owner(prefix[b], total, ctas), part = (int)blockIdx.x + b;
      reduce_heads(l_acc, false);
      group_sync();
      if (sidx < NHP) misc->fac[sidx] = reduced(sidx, false);
      group_sync();
      if (ok && sidx < a.n_heads) {
        const float l = misc->fac[sidx], m = misc->m_used[sidx] - kShift;
        if (whole) {
          if (a.lse) a.lse[(long long)b * a.n_heads + sidx] = (m + log2f(l)) * 0.69314718055994531f;
        } else {
          a.ml_part[((long long)part * a.n_heads + sidx) * 2] = m;
          a.ml_part[((long long)part * a.n_heads + sidx) * 2 + 1] = l;
        }
      }
      if (ok && sidx == 0 && g + 1 == prefix[b + 1])
        a.seq_parts[b] = whole ? make_int2(0, 0) : make_int2(c0 + b, (int)blockIdx.x - c0 + 1);
      if (ok) ok = wait(misc->p_empty[n & 1], n >> 1, 20);           // the last value products
      ok = __all_sync(0xffffffffu, ok);
      if (ok) {
        tc_fence_after_sync();
        // Lane 8j + g of a quarter holds latent 4g + j.
        const int lat = q * 32 + 4 * (lane & 7) + (lane >> 3);
        for (int mb = 0; mb < NB; ++mb) {
          uint32_t ov[16];
          ld_cols(lane_base + kColO + mb * 32, ov);
          tmem_wait_ld();
          if (mb * 128 + lat >= r) continue;
#pragma unroll
          for (int i = 0; i < NHH; ++i) {
            if (HO + i >= a.n_heads) continue;
            const float v = __uint_as_float(ov[i]);
            if (whole)
              static_cast<bf16*>(a.out)[((long long)b * a.n_heads + HO + i) * r + mb * 128 + lat] =
                  __float2bfloat16_rn(v / misc->fac[HO + i]);
            else
              a.o_part[((long long)part * a.n_heads + HO + i) * r + mb * 128 + lat] = v;
          }
        }
        tc_fence_before_sync();
      }
      group_sync();                                      // fac, unit and the references may be rewritten
    }
  }

  __syncthreads();
  if (*abort_word) {
    // Give copies that may still be in flight time to land before the CTA's memory is reused.
    const uint64_t t0 = global_timer_ns();
    while (global_timer_ns() - t0 < 100000ull) __nanosleep(1000);
  }
  if (warp == kProducerWarp) {
    __syncwarp();
    tc_fence_after_sync();
    tmem_dealloc(tmem, kTmemCols);
  }
}

}  // namespace qp
}  // namespace mtla
