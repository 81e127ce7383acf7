// Attention of one query per sequence over the slots of the 4-bit pool (absorbed form, Eq. 12 and
// Eq. 17): o_h = sum_j softmax_j(scale (q_h . [c_j ; k_j])) c_j, plus the logarithm of the denominator.
//
// Work is a list of 64-slot tiles (pages), sequence after sequence, dealt out in equal contiguous
// shares to the CTAs, so ragged batches and a single long sequence are balanced alike.  The lengths
// live on the device: every CTA forms their prefix sums itself.  A share may begin or end inside
// a sequence; such segments leave a partial (reference maximum, denominator, unnormalised output)
// that qpool_combine_kernel joins in share order; a sequence that lies in one share is finished at once.
//
// The kernel of this file serves fp32 queries, batches over 1022 sequences and the smallest ones (the other
// one is in qpool_attn_tc.cuh; its rule is beside the launch).  Its warps expand, multiply and reduce by
// turns: 1023 x 1024 slots, 32 heads, r 512, bf16 take 605 us, where the other needs 193 for 1022; fp32
// queries 34 us for 8 x 4112 slots of 16 heads, 135 us for 32 x 4096 of 32 heads.
//
// It runs on the warp-level matrix instructions (m16n8k16), with the codes
// expanded from shared memory into registers in both fragment layouts:
//   scores  S[heads x slots]   = Q[heads x r] . C^T   B fragment: a thread owns one slot and reads 16
//                                                     bytes = 32 latents; the order of the latents in
//                                                     the product is permuted alike in Q
//   values  O[heads x latents] = P[heads x slots] . C B fragment: a transposing matrix load moves units of
//                                                     four codes, so a thread owns four latents of two
//                                                     neighbouring slots and pairs their codes itself
// A latent is exact in half precision (see qpool_format.cuh), so the only roundings are those of
// the other operand: a query row is scaled by a power of two into half precision's range and kept as
// one (bf16 queries: exact up to 2^-39 of the row's largest element) or two (fp32: 22 bits) half-precision
// terms, its RoPE part as one or three bf16 terms against the bf16 keys, and a probability,
// relative to the running maximum's, as one or two half-precision terms: 2^-11, an eighth of what the bf16
// output is rounded by, or 2^-22.  (Exact ones would take two or three matrix products for every one.)  A
// denominator is the sum of the unrounded probabilities.  Maxima, denominators and
// all sums are fp32.  The matrix instructions cut their running sums off instead of rounding them, so a
// score collects one product per 32 latents and an output one per 32 slots, and the
// products are added outside: the error against 64 bits falls by 2 to 3 for fp32 queries (r 512, 5000 slots:
// 3.4e-6 to 1.5e-6 of the output's size), at no time; for bf16 ones outputs of 2^20 slots came out 6.6e-3
// too small (1023 x 1024 slots, 32 heads, r 512: 588 us, so 606).
#pragma once

#include <math.h>

#include "qpool_format.cuh"

namespace mtla {
namespace qp {

struct AttnArgs {
  const uint8_t* pages;
  const int* table;          // [batch][width] page of tile t
  const int* slots;          // [batch]
  const void* q;             // [batch][n_heads][r + d_R]
  void* out;                 // [batch][n_heads][r]
  float* lse;                // [batch][n_heads] or nullptr
  float* o_part;             // [batch + ctas][n_heads][r]
  float* ml_part;            // [batch + ctas][n_heads][2]: reference (log2 units) of the sums, denominator
  int2* seq_parts;           // [batch] first part, number of parts (0: finished by one CTA)
  int* error_words;          // tensor-core kernel: [n_error_words] a CTA's bounded wait gave up
  float scale_log2;          // scale * log2(e)
  int n_heads, batch, width, n_pages, n_error_words;
  Format f;
};

// Column groups of drafted trees (tree_kernels.cuh) in the place of sequences: how many there are and their tiles, the
// tiles before each, and its request, first column, columns and slots.  Their results are always parts, of `cols`
// columns.  A type of its own: as fields of all kernels' arguments these cost the tensor-core kernel over sequences
// 1.4 % (128 x 16384 slots: 268 -> 272 us).
template <bool TREE>
struct KernelArgs : AttnArgs {
  static constexpr const int2* listed = nullptr;
  static constexpr const int* prefix = nullptr;
  static constexpr const int4* groups = nullptr;
  static constexpr int cols = 0;
};
template <>
struct KernelArgs<true> : AttnArgs {
  const int2* listed;
  const int* prefix;
  const int4* groups;
  const int4* shares;        // the CTAs' shares of the tiles (tensor-core kernel)
  const uint8_t* image;      // the groups' queries as the tensor-core kernel wants them
  int cols;
};
using GroupArgs = KernelArgs<true>;

constexpr int kAttnThreads = 256;
constexpr int kAttnWarps = kAttnThreads / 32;
constexpr int kMaxBatch = 4096;
// Probabilities are kept times 2^14: half precision's smallest step, 2^-24, is then 2^-38 of the
// largest one, which matters where the largest ones meet latents that are zero.  Numerators and
// denominators carry the factor alike.
constexpr float kProbShift = 14.f;

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Four 8 x 8 matrices of 16-bit units, transposed: thread (g, t) = (lane / 4, lane % 4) gets units
// (2t, g) and (2t + 1, g) of matrix m in o[m]; lane l holds the address of row l % 8 of matrix l / 8.
__device__ __forceinline__ void ldsm_x4_trans(uint32_t addr, uint32_t (&o)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldsm_x4(uint32_t addr, uint32_t (&o)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}
__device__ __forceinline__ uint32_t lds_u8(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(addr));
  return v;
}
// 16 bytes global -> shared; bytes = 0 fills with zeros without reading.
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// A thread's register of the transposing load holds codes (4g .. 4g + 3) of slot 2t in its low half
// and of slot 2t + 1 in its high half.  o[j] = half-precision pair (slot 2t, slot 2t + 1) of latent
// 4g + j.  The pairs are gathered in the upper half with left shifts, which run beside the ALU pipe that
// the conversions and the selections share.
__device__ __forceinline__ void decode_pairs(uint32_t w, uint32_t (&o)[4]) {
  const uint32_t e = ((w << 16) & 0x0f0f0000u) | ((w << 4) & 0xf0f00000u);     // latents 0 and 2
  const uint32_t d = ((w << 12) & 0x0f0f0000u) | (w & 0xf0f00000u);            // latents 1 and 3
  asm("{\n\t.reg .b8 a, b, c, d, x, y;\n\t"
      "mov.b32 {x, y, a, b}, %4;\n\t"
      "mov.b32 {x, y, c, d}, %5;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3])
      : "r"(e), "r"(d));
}

// Prefix sums of the sequences' tile counts (PAGES pages each) into prefix[0 .. batch]; returns the total.
// With `slots` the (non-negative) slot counts are left there for whoever needs them later.
template <int PAGES>
__device__ inline long long tile_prefix(const AttnArgs& a, int* prefix, int* warp_sums, int threads,
                                        int* slots = nullptr) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // A count past the table's width is cut to it; a negative one is no slot at all.
  auto tiles_of = [&](int n) {
    return (min(n / kPageRows + (n % kPageRows != 0), a.width) + PAGES - 1) / PAGES;
  };
  if (a.batch <= 32) {                 // every warp forms the sums: one wait for the others less
    const int n = lane < a.batch ? max(a.slots[lane], 0) : 0;
    int incl = lane < a.batch ? tiles_of(n) : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    if (warp == 0 && lane < a.batch) {
      prefix[lane + 1] = incl;
      if (slots) slots[lane] = n;
      if (lane == 0) prefix[0] = 0;
    }
    __syncthreads();
    return __shfl_sync(0xffffffffu, incl, 31);
  }
  const int per = ceil_div(a.batch, threads);
  const int lo = min(a.batch, tid * per), hi = min(a.batch, lo + per);
  int sum = 0;
  for (int b = lo; b < hi; ++b) {
    const int n = max(a.slots[b], 0), t = tiles_of(n);
    prefix[b + 1] = t;
    if (slots) slots[b] = n;
    sum += t;
  }
  int incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  if (lo < hi) {                       // most warps of a small batch have nothing to add up
    int run = incl - sum;
    for (int w = 0; w < warp; ++w) run += warp_sums[w];
    for (int b = lo; b < hi; ++b) {
      run += prefix[b + 1];
      prefix[b + 1] = run;
    }
  }
  if (tid == 0) prefix[0] = 0;
  __syncthreads();
  return prefix[a.batch];
}
// Largest b with list[b] <= i in ascending global memory list[0 .. n], by a whole warp.
__device__ __forceinline__ int find_wide(const int* list, int n, int i) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32, at = lo + lane * step;
    const uint32_t below = __ballot_sync(0xffffffffu, at < hi && list[at < hi ? at : lo] <= i);
    const int k = max(1, __popc(below));             // the first ones, lane 0's among them
    lo += (k - 1) * step;
    hi = min(hi, lo + step);
  }
  return lo;
}
__device__ __forceinline__ int find_seq(const int* prefix, int batch, int g) {   // largest b with prefix[b] <= g
  int lo = 0, hi = batch;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (prefix[mid] <= g) lo = mid; else hi = mid;
  }
  return lo;
}
// The shares of `total` tiles (up to 2^31 - 1): floor(c total / ctas), in 32-bit arithmetic since every
// CTA starts with it (ctas < 2^9, so the product fits).  In proportion rather than the longer ones first:
// equal sequences then more often begin where a share does (8 x 4112 slots: 19.5 us against 21.4).
__host__ __device__ inline int share_begin(uint32_t c, uint32_t total, uint32_t ctas) {
  const uint32_t each = total / ctas, more = total - each * ctas;
  return (int)(c * each + c * more / ctas);
}
__host__ __device__ inline int share_owner(long long g, long long total, long long ctas) {
  return (int)(((g + 1) * ctas - 1) / total);
}

// MH: 16-head tiles; TERMS: half-precision terms of a query / probability (1: bf16 queries, 2: fp32).
template <int MH, int TERMS>
struct AttnLayout {
  static constexpr int kKeyTerms = TERMS == 1 ? 1 : 3;
  static constexpr int kStages = 2;
  static constexpr int kHeads = 16 * MH;
  static constexpr int kSStride = kPageRows + 4;       // fp32 scores
  static constexpr int kPStride = kPageRows + 8;       // half-precision probabilities
  // Row strides that put the two rows of a quarter-warp's 64-byte runs into different banks.
  __host__ __device__ static int q_stride(int r) { return r + 32; }
  __host__ __device__ static int k_stride(int dr) { return dr == 64 ? 96 : 32; }
  __host__ __device__ static int off_q(const Format& f) { return kStages * f.page_bytes(); }
  __host__ __device__ static int off_k(const Format& f) { return off_q(f) + TERMS * kHeads * q_stride(f.r) * 2; }
  __host__ __device__ static int off_s(const Format& f) { return off_k(f) + kKeyTerms * kHeads * k_stride(f.dr) * 2; }
  __host__ __device__ static int off_p(const Format& f) { return off_s(f) + kHeads * kSStride * 4; }
  __host__ __device__ static int off_m(const Format& f) { return off_p(f) + TERMS * kHeads * kPStride * 2; }
  __host__ __device__ static int off_prefix(const Format& f) { return off_m(f) + 4 * kHeads * 4; }
  __host__ __device__ static int bytes(const Format& f, int batch) { return off_prefix(f) + (batch + 1) * 4; }
};

// Two CTAs an SM where the registers allow it (not for fp32 queries of over 16 heads); left to itself the
// compiler takes a few registers more (1023 x 1024 slots, 32 heads, bf16: 740 us for 606; 8 x 4112 slots, 16 heads,
// fp32: 41 for 34).
// TREE: over column groups instead of sequences.
template <typename T, int MH, bool TREE = false>
__global__ void __launch_bounds__(kAttnThreads, sizeof(T) == 2 || MH == 1 ? 2 : 1) qpool_attend_kernel(KernelArgs<TREE> a) {
  constexpr int TERMS = sizeof(T) == 2 ? 1 : 2;
  using L = AttnLayout<MH, TERMS>;
  constexpr int KT = L::kKeyTerms, NH = L::kHeads;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int warp_sums[kAttnWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const Format f = a.f;
  const int r = f.r, dr = f.dr, page_bytes = f.page_bytes();
  int* own_prefix = reinterpret_cast<int*>(smem + L::off_prefix(f));
  __half* qs = reinterpret_cast<__half*>(smem + L::off_q(f));
  bf16* ks = reinterpret_cast<bf16*>(smem + L::off_k(f));
  float* ss = reinterpret_cast<float*>(smem + L::off_s(f));
  __half* ps = reinterpret_cast<__half*>(smem + L::off_p(f));
  float* m_s = reinterpret_cast<float*>(smem + L::off_m(f));       // reference maximum per head
  float *l_s = m_s + NH, *alpha_s = l_s + NH, *unit_s = alpha_s + NH;   // denominator, rescale, score unit
  const uint32_t raw_u32 = ptx::smem_u32(smem), q_u32 = ptx::smem_u32(qs), k_u32 = ptx::smem_u32(ks),
                 p_u32 = ptx::smem_u32(ps);
  const int qst = L::q_stride(r), kst = L::k_stride(dr);

  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  const int* const prefix = TREE ? a.prefix : own_prefix;
  const int2 listed = TREE ? *a.listed : make_int2(a.batch, 0);
  const int n_seqs = TREE ? max(listed.x, 0) : a.batch;
  const long long total = TREE ? listed.y : tile_prefix<1>(a, own_prefix, warp_sums, kAttnThreads);
  if (total == 0) return;
  // With fewer tiles than CTAs the rest stays out, so that every share has a tile and the parts of
  // a sequence follow one another without a gap.
  const int ctas = (int)(total < gridDim.x ? total : gridDim.x);
  if ((int)blockIdx.x >= ctas) return;
  const int g0 = share_begin(blockIdx.x, total, ctas), g1 = share_begin(blockIdx.x + 1, total, ctas);

  // Tile n of the list into its buffer; rows past the sequence's end (and pages outside the pool)
  // are filled with zeros, so that nothing behind the last slot enters a product.
  auto page_of = [&](int b, int tile) { return a.table[(long long)(TREE ? a.groups[b].x : b) * a.width + tile]; };
  auto tile_rows = [&](int b, int tile) {
    const int page = page_of(b, tile);
    return page < 0 || page >= a.n_pages ? 0 : min(kPageRows, (TREE ? a.groups[b].w : a.slots[b]) - tile * kPageRows);
  };
  auto load_tile = [&](int n, int b) {
    const int tile = n - prefix[b], rows = tile_rows(b, tile);
    const uint8_t* src = a.pages + (rows ? (long long)page_of(b, tile) * page_bytes : 0);
    const uint32_t dst = raw_u32 + ((n - g0) % L::kStages) * page_bytes;
    const int c_bytes = f.off_scales(), s_bytes = f.off_keys();
    for (int o = tid * 16; o < page_bytes; o += kAttnThreads * 16) {
      // Bytes of the 16 that belong to valid rows (a row of scales may be shorter than 16 bytes).
      int keep;
      if (o < c_bytes) keep = rows * f.code_row() - o;
      else if (o < s_bytes) keep = rows * f.scale_row() - (o - c_bytes);
      else keep = rows * f.key_row() - (o - s_bytes);
      keep = max(0, min(16, keep));
      cp_async16(dst + o, src + (keep ? o : 0), keep);
    }
  };

  int b = TREE ? find_wide(prefix, n_seqs, g0) : find_seq(prefix, n_seqs, g0), b_load = b;
  load_tile(g0, b);
  cp_async_commit();

  float acc[2][4][MH][4];            // [chunk][latent column][head tile][fragment]
  const int chunks = r / kGroup, cmask = f.code_mask();

  for (int n = g0; n < g1; ++n) {
    while (prefix[b + 1] <= n) ++b;
    const int tile = n - prefix[b], seq_tiles = prefix[b + 1] - prefix[b];
    const bool seg_first = n == g0 || tile == 0, seg_last = n + 1 == g1 || tile + 1 == seq_tiles;
    if (n + 1 < g1) {
      while (prefix[b_load + 1] <= n + 1) ++b_load;
      load_tile(n + 1, b_load);
    }
    cp_async_commit();

    if (seg_first) {
      // The sequence's query: a warp per head.  The row is scaled by a power of two so that its
      // largest element lies in [2^14, 2^15).
      const long long col0 = TREE ? (long long)a.groups[b].y : (long long)b * a.n_heads;
      const int n_cols = TREE ? a.groups[b].z : a.n_heads;
      for (int h = warp; h < NH; h += kAttnWarps) {
        const T* q = static_cast<const T*>(a.q) + (col0 + h) * (r + dr);
        float top = 0.f;
        if (h < n_cols)
          for (int i = lane; i < r + dr; i += 32) top = fmaxf(top, fabsf(Elem<T>::to_float(q[i])));
        top = warp_max(top);
        const bool fine = top > 0.f && top < INFINITY;
        const int e = fine ? 14 - ilogbf(top) : 0;
        if (lane == 0) {
          m_s[h] = -INFINITY;
          l_s[h] = 0.f;
          unit_s[h] = ldexpf(a.scale_log2, -e);
        }
        for (int i = lane; i < r; i += 32) {
          float v = h < n_cols ? ldexpf(Elem<T>::to_float(q[i]), e) : 0.f;
#pragma unroll
          for (int k = 0; k < TERMS; ++k) {
            const __half x = __float2half_rn(v);
            qs[(k * NH + h) * qst + i] = x;
            v -= __half2float(x);
          }
        }
        for (int i = lane; i < dr; i += 32) {
          float v = h < n_cols ? ldexpf(Elem<T>::to_float(q[r + i]), e) : 0.f;
#pragma unroll
          for (int k = 0; k < KT; ++k) {
            const bf16 x = __float2bfloat16_rn(v);
            ks[(k * NH + h) * kst + i] = x;
            v -= __bfloat162float(x);
          }
        }
      }
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int mh = 0; mh < MH; ++mh)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[c][j][mh][i] = 0.f;
    }
    cp_async_wait<1>();
    __syncthreads();                 // the tile has landed, the query is in place
    const uint32_t buf = raw_u32 + ((n - g0) % L::kStages) * page_bytes;
    const int rows = tile_rows(b, tile);

    {  // ---- scores of slots 8 * warp + 0..7
      float s[MH][4];
#pragma unroll
      for (int mh = 0; mh < MH; ++mh)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[mh][i] = 0.f;
      const int row = warp * 8 + g;
      const uint32_t codes = buf + row * f.code_row(), scales = buf + f.off_scales() + row * f.scale_row();
      // The chunk's 16 bytes are four words, one per thread of the slot: word t = latents 8t .. 8t + 7.
      auto query = [&](uint32_t base, int stride_bytes, int term, int mh, int at, uint4& lo, uint4& hi) {
        const uint32_t p = base + ((term * NH + mh * 16 + g) * stride_bytes) + at;
        lo = lds128(p);
        hi = lds128(p + 8 * stride_bytes);
      };
      for (int c = 0; c < chunks; ++c) {
        uint32_t w;
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w) : "r"(codes + ((c ^ (row & cmask)) * 16) + 4 * t));
        const uint32_t sc = scale_pair(lds_u8(scales + c));
        uint32_t o[4];
        decode8(w, o);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = mul_h2(o[i], sc);
        float part[MH][4];                   // of this chunk: see the head of the file
#pragma unroll
        for (int mh = 0; mh < MH; ++mh)
#pragma unroll
          for (int i = 0; i < 4; ++i) part[mh][i] = 0.f;
#pragma unroll
        for (int k = 0; k < TERMS; ++k)
#pragma unroll
          for (int mh = 0; mh < MH; ++mh) {
            uint4 lo, hi;
            query(q_u32, qst * 2, k, mh, c * 64 + t * 16, lo, hi);
            const uint32_t a0[4] = {lo.x, hi.x, lo.y, hi.y}, a1[4] = {lo.z, hi.z, lo.w, hi.w};
            mma_f16(part[mh], a0, o[0], o[1]);
            mma_f16(part[mh], a1, o[2], o[3]);
          }
#pragma unroll
        for (int mh = 0; mh < MH; ++mh)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[mh][i] += part[mh][i];
      }
      const uint32_t keys = buf + f.off_keys() + row * f.key_row();
      for (int c = 0; c < dr / 32; ++c) {
        const uint4 kv = lds128(keys + ((c * 4 + t) ^ f.key_swizzle(row)) * 16);
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
          for (int mh = 0; mh < MH; ++mh) {
            uint4 lo, hi;
            query(k_u32, kst * 2, k, mh, c * 64 + t * 16, lo, hi);
            const uint32_t a0[4] = {lo.x, hi.x, lo.y, hi.y}, a1[4] = {lo.z, hi.z, lo.w, hi.w};
            mma_bf16(s[mh], a0, kv.x, kv.y);
            mma_bf16(s[mh], a1, kv.z, kv.w);
          }
      }
#pragma unroll
      for (int mh = 0; mh < MH; ++mh) {
        float* d = ss + (mh * 16 + g) * L::kSStride + warp * 8 + 2 * t;
        *reinterpret_cast<float2*>(d) = make_float2(s[mh][0], s[mh][1]);
        *reinterpret_cast<float2*>(d + 8 * L::kSStride) = make_float2(s[mh][2], s[mh][3]);
      }
    }
    __syncthreads();
    // ---- softmax: a warp per head, two slots per lane
    for (int h = warp; h < NH; h += kAttnWarps) {
      const float2 sv = *reinterpret_cast<const float2*>(ss + h * L::kSStride + 2 * lane);
      const float unit = unit_s[h], m_old = m_s[h], l_old = l_s[h];
      const float s0 = 2 * lane < rows ? sv.x * unit : -INFINITY, s1 = 2 * lane + 1 < rows ? sv.y * unit : -INFINITY;
      const float m_new = fmaxf(m_old, warp_max(fmaxf(s0, s1)));
      const float ref = m_new == -INFINITY ? 0.f : m_new;       // nothing visible yet: every term is 0
      const float p0 = exp2f(s0 - ref + kProbShift), p1 = exp2f(s1 - ref + kProbShift), al = exp2f(m_old - ref);
      float sum = p0 + p1;           // of the unrounded ones: its logarithm is an output of its own
      const __half2 hi = __floats2half2_rn(p0, p1);
      *reinterpret_cast<__half2*>(ps + h * L::kPStride + 2 * lane) = hi;
      if constexpr (TERMS == 2) {
        const __half2 lo = __floats2half2_rn(p0 - __low2float(hi), p1 - __high2float(hi));
        *reinterpret_cast<__half2*>(ps + (NH + h) * L::kPStride + 2 * lane) = lo;
      }
      sum = warp_sum(sum);
      if (lane == 0) {
        m_s[h] = m_new;
        l_s[h] = l_old * al + sum;
        alpha_s[h] = al;
      }
    }
    __syncthreads();
    // ---- values: chunks warp and warp + 8
    {
      float al[MH][2];
#pragma unroll
      for (int mh = 0; mh < MH; ++mh) {
        al[mh][0] = alpha_s[mh * 16 + g];
        al[mh][1] = alpha_s[mh * 16 + g + 8];
      }
#pragma unroll
      for (int ci = 0; ci < 2; ++ci) {
        const int c = warp + ci * kAttnWarps;
        if (c >= chunks) break;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int mh = 0; mh < MH; ++mh) {
            acc[ci][j][mh][0] *= al[mh][0];
            acc[ci][j][mh][1] *= al[mh][0];
            acc[ci][j][mh][2] *= al[mh][1];
            acc[ci][j][mh][3] *= al[mh][1];
          }
#pragma unroll
        for (int half = 0; half < 2; ++half) {             // 32 slots: two k-steps
          const int lr = half * 32 + lane;
          uint32_t w[4];
          ldsm_x4_trans(buf + lr * f.code_row() + (c ^ (lr & cmask)) * 16, w);
          float part[4][MH][4];              // of these 32 slots
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int mh = 0; mh < MH; ++mh)
#pragma unroll
              for (int i = 0; i < 4; ++i) part[j][mh][i] = 0.f;
          uint32_t v[4][4];
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            const uint32_t sp = buf + f.off_scales() + (half * 32 + m * 8 + 2 * t) * f.scale_row() + c;
            const uint32_t sc = scale_pair(lds_u8(sp), lds_u8(sp + f.scale_row()));
            decode_pairs(w[m], v[m]);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[m][j] = mul_h2(v[m][j], sc);
          }
#pragma unroll
          for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
            for (int k = 0; k < TERMS; ++k)
#pragma unroll
              for (int mh = 0; mh < MH; ++mh) {
                // P fragment: rows mh * 16 + 0..15, slots half * 32 + k2 * 16 + 0..15.
                uint32_t p[4];
                ldsm_x4(p_u32 + ((k * NH + mh * 16 + (lane & 15)) * L::kPStride + half * 32 + k2 * 16 + (lane >> 4) * 8) * 2, p);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                  mma_f16(part[j][mh], p, v[2 * k2][j], v[2 * k2 + 1][j]);
              }
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int mh = 0; mh < MH; ++mh)
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[ci][j][mh][i] += part[j][mh][i];
        }
      }
    }
    if (seg_last) {
      // ---- end of a segment: the finished output, or a partial
      const int n_cols = TREE ? a.groups[b].z : a.n_heads, stride = TREE ? a.cols : a.n_heads;
      const bool whole = !TREE && prefix[b] >= g0 && tile + 1 == seq_tiles;
      const int c0 = share_owner(prefix[b], total, ctas);
      const int part = blockIdx.x + b;                     // unique per (CTA, sequence), parts of a sequence in a row
      if (tid == 0 && tile + 1 == seq_tiles)
        a.seq_parts[b] = whole ? make_int2(0, 0) : make_int2(c0 + b, (int)blockIdx.x - c0 + 1);
#pragma unroll
      for (int ci = 0; ci < 2; ++ci) {
        const int c = warp + ci * kAttnWarps;
        if (c >= chunks) break;
#pragma unroll
        for (int mh = 0; mh < MH; ++mh)
#pragma unroll
          for (int hh = 0; hh < 2; ++hh) {
            const int h = mh * 16 + hh * 8 + g;
            if (h >= n_cols) continue;
            // Fragment column 2t is latent 8t + j, column 2t + 1 latent 8t + 4 + j: eight in a row.
            float v[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              v[j] = acc[ci][j][mh][2 * hh];
              v[4 + j] = acc[ci][j][mh][2 * hh + 1];
            }
            if (whole) {
              const float inv = 1.f / l_s[h];
#pragma unroll
              for (int j = 0; j < 8; ++j) v[j] *= inv;
              T* d = static_cast<T*>(a.out) + ((long long)b * a.n_heads + h) * r + c * kGroup + 8 * t;
              if constexpr (sizeof(T) == 2) {
                store_vec(d, v);
              } else {
                const float v0[4] = {v[0], v[1], v[2], v[3]}, v1[4] = {v[4], v[5], v[6], v[7]};
                store_vec(d, v0);
                store_vec(d + 4, v1);
              }
            } else {
              float* d = a.o_part + ((long long)part * stride + h) * r + c * kGroup + 8 * t;
              *reinterpret_cast<float4*>(d) = make_float4(v[0], v[1], v[2], v[3]);
              *reinterpret_cast<float4*>(d + 4) = make_float4(v[4], v[5], v[6], v[7]);
            }
          }
      }
      if (tid < n_cols) {
        if (whole) {
          if (a.lse) a.lse[(long long)b * a.n_heads + tid] = (m_s[tid] - kProbShift + log2f(l_s[tid])) * 0.69314718055994531f;
        } else {
          a.ml_part[((long long)part * stride + tid) * 2] = m_s[tid] - kProbShift;
          a.ml_part[((long long)part * stride + tid) * 2 + 1] = l_s[tid];
        }
      }
    }
    __syncthreads();                 // the tile's buffer, P and the statistics may be rewritten
  }
}

// Joins the partials of sequences that several CTAs worked on, and answers for sequences without a
// slot: zeros and a logarithm of minus infinity.  Every CTA lists these sequences (the others are
// finished) and takes pieces of them in turn.  With few parts (a large batch: two parts for most
// sequences) a piece is 1024 elements, four a thread, which weighs the parts itself.  With many (a
// few long sequences over every SM) a piece is 128 columns of one head, eight groups of parts
// by 32 threads of four columns, so that many loads are in flight: one way for both cost 68 us for 148
// parts of one sequence, the other 190 us for 128 sequences of two (16 and 32 heads, r 512).  Parts
// are added in a fixed order.
constexpr int kCombineThreads = 256, kCombineCols = 128, kCombineGroups = 8;
constexpr int kFewParts = 8;
constexpr int kMaxParts = 512;                       // more than CTAs of any attention launch
__device__ __forceinline__ void store4(float* p, const float (&v)[4]) { store_vec(p, v); }
__device__ __forceinline__ void store4(bf16* p, const float (&v)[4]) {
  const __nv_bfloat162 x0 = __floats2bfloat162_rn(v[0], v[1]), x1 = __floats2bfloat162_rn(v[2], v[3]);
  *reinterpret_cast<uint2*>(p) =
      make_uint2(*reinterpret_cast<const uint32_t*>(&x0), *reinterpret_cast<const uint32_t*>(&x1));
}
template <typename T>
__global__ void __launch_bounds__(kCombineThreads) qpool_combine_kernel(AttnArgs a) {
  extern __shared__ int4 listed[];                   // [batch] sequence, first part, parts (0: no slot)
  __shared__ int2 warp_count[kCombineThreads / 32];
  __shared__ float weight[kMaxParts], red[kCombineThreads / 32], total[kCombineThreads / 32];
  __shared__ float4 sums[kCombineGroups][kCombineCols / 4];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = a.f.r, heads = a.n_heads;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  // A bounded wait gave up: no result that looks like one.
  const bool failed = __syncthreads_or(tid < a.n_error_words && a.error_words[tid] != 0);
  // Sequences with few parts (or none, or no result) from the front of the list, the others from its
  // end, both in order: every CTA has the same list.
  int n_few = 0, n_many = 0;
  for (int b0 = 0; b0 < a.batch; b0 += kCombineThreads) {
    const int b = b0 + tid;
    int kind = 0;                                    // 1 few, 2 many
    int2 parts = make_int2(0, 0);
    if (b < a.batch) {
      const int n = a.slots[b];
      parts = a.seq_parts[b];                        // (not set for a sequence without slots)
      if (n <= 0) parts.y = 0;
      kind = failed || n <= 0 ? 1 : parts.y == 0 ? 0 : parts.y <= kFewParts ? 1 : 2;
    }
    const uint32_t few = __ballot_sync(0xffffffffu, kind == 1), many = __ballot_sync(0xffffffffu, kind == 2);
    if (lane == 0) warp_count[warp] = make_int2(__popc(few), __popc(many));
    __syncthreads();
    const uint32_t below = (1u << lane) - 1u;
    int at_few = n_few + __popc(few & below), at_many = n_many + __popc(many & below);
#pragma unroll
    for (int i = 0; i < kCombineThreads / 32; ++i) {
      const int2 c = warp_count[i];
      if (i < warp) { at_few += c.x; at_many += c.y; }
      n_few += c.x;
      n_many += c.y;
    }
    if (kind == 1) listed[at_few] = make_int4(b, parts.x, parts.y, 0);
    if (kind == 2) listed[a.batch - 1 - at_many] = make_int4(b, parts.x, parts.y, 0);
    __syncthreads();
  }

  const int seq_pieces = (heads * r + 4 * kCombineThreads - 1) / (4 * kCombineThreads);
  for (long long w = blockIdx.x; w < (long long)n_few * seq_pieces; w += gridDim.x) {
    const int4 seq = listed[w / seq_pieces];
    const int b = seq.x, e = ((int)(w % seq_pieces) * kCombineThreads + tid) * 4;
    if (e >= heads * r) continue;
    const int h = e / r;
    const float fill = failed ? NAN : 0.f;
    float v[4] = {fill, fill, fill, fill};
    float lse = failed ? NAN : -INFINITY;
    if (!failed && seq.z > 0) {
      const int2 parts = make_int2(seq.y, seq.z);
      const float2* ml = reinterpret_cast<const float2*>(a.ml_part) + (long long)parts.x * heads + h;
      const float* o = a.o_part + (long long)parts.x * heads * r + e;
      const long long o_step = (long long)heads * r;
      float2 s[kFewParts];
      float4 x[kFewParts];
      float m = -INFINITY, l = 0.f;
#pragma unroll
      for (int p = 0; p < kFewParts; ++p)
        if (p < parts.y) {
          s[p] = ml[p * heads];
          x[p] = *reinterpret_cast<const float4*>(o + p * o_step);
        }
#pragma unroll
      for (int p = 0; p < kFewParts; ++p)
        if (p < parts.y) m = fmaxf(m, s[p].x);
      const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int p = 0; p < kFewParts; ++p)
        if (p < parts.y) {
          const float f = exp2f(s[p].x - ref);
          l += f * s[p].y;
          v[0] += f * x[p].x; v[1] += f * x[p].y; v[2] += f * x[p].z; v[3] += f * x[p].w;
        }
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] /= l;
      lse = (m + log2f(l)) * 0.69314718055994531f;
    }
    store4(static_cast<T*>(a.out) + (long long)b * heads * r + e, v);
    if (a.lse && e % r == 0) a.lse[(long long)b * heads + h] = lse;
  }

  const int col_blocks = (r + kCombineCols - 1) / kCombineCols;
  for (long long w = blockIdx.x; w < (long long)n_many * heads * col_blocks; w += gridDim.x) {
    const int cb = (int)(w % col_blocks), bh = (int)(w / col_blocks), h = bh % heads;
    const int4 seq = listed[a.batch - 1 - bh / heads];
    const int b = seq.x, n_parts = seq.z, col = cb * kCombineCols + lane * 4;
    float lse;
    float4 sum;
    {
      const float2* ml = reinterpret_cast<const float2*>(a.ml_part) + (long long)seq.y * heads + h;
      const float* o = a.o_part + ((long long)seq.y * heads + h) * r + col;
      const long long o_step = (long long)heads * r;
      // The first loads of the sums do not wait for the weights.
      constexpr int kU = 4;
      float4 x[kU];
      auto load = [&](int p0) {
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          const int p = p0 + u * kCombineGroups;
          x[u] = col < r && p < n_parts ? *reinterpret_cast<const float4*>(o + p * o_step)
                                        : make_float4(0.f, 0.f, 0.f, 0.f);
        }
      };
      load(warp);
      // A thread's parts: at most two (kMaxParts over the threads).
      float2 mine[2];
      float m = -INFINITY;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int p = tid + i * kCombineThreads;
        mine[i] = p < n_parts ? ml[(long long)p * heads] : make_float2(-INFINITY, 0.f);
        m = fmaxf(m, mine[i].x);
      }
      m = warp_max(m);
      if (lane == 0) red[warp] = m;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kCombineThreads / 32; ++i) m = fmaxf(m, red[i]);
      const float ref = m == -INFINITY ? 0.f : m;
      float l = 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int p = tid + i * kCombineThreads;
        const float f = p < n_parts ? exp2f(mine[i].x - ref) : 0.f;
        if (p < n_parts) weight[p] = f;
        l += p < n_parts ? f * mine[i].y : 0.f;
      }
      l = warp_sum(l);
      if (lane == 0) total[warp] = l;
      __syncthreads();
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int p0 = warp; p0 < n_parts; p0 += kU * kCombineGroups) {
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          const int p = p0 + u * kCombineGroups;
          const float f = p < n_parts ? weight[p] : 0.f;
          v.x += f * x[u].x; v.y += f * x[u].y; v.z += f * x[u].z; v.w += f * x[u].w;
        }
        load(p0 + kU * kCombineGroups);
      }
      sums[warp][lane] = v;
      __syncthreads();
      sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < kCombineGroups; ++i) {
        const float4 x = sums[i][lane];
        sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
      }
      l = 0.f;
#pragma unroll
      for (int i = 0; i < kCombineThreads / 32; ++i) l += total[i];
      sum.x /= l; sum.y /= l; sum.z /= l; sum.w /= l;
      lse = (m + log2f(l)) * 0.69314718055994531f;
    }
    if (warp == 0 && col < r) {
      const float v[4] = {sum.x, sum.y, sum.z, sum.w};
      store4(static_cast<T*>(a.out) + ((long long)b * heads + h) * r + col, v);
      if (a.lse && cb == 0 && lane == 0) a.lse[(long long)b * heads + h] = lse;
    }
    __syncthreads();                                 // the shared sums may be rewritten
  }
}

}  // namespace qp
}  // namespace mtla
