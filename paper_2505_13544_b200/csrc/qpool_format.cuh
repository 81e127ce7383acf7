// The 4-bit latent pool: page layout, element format, and the kernels that write and read rows.
//
// A page holds 64 slots in three blocks:
//   codes   [64][r/2] bytes   two e2m1 codes per byte (sign, two exponent bits, one fraction bit:
//                             0, 0.5, 1, 1.5, 2, 3, 4, 6), latent 2k in the low half of byte k
//   scales  [64][r/32] bytes  one scale per group of 32 latents: bits 14..7 of a positive half-precision
//                             number (5 exponent bits, 3 fraction bits), so decoding is a shift
//   keys    [64][d_R] bf16    the RoPE key, unquantised
// A latent is code * scale: 2 significant bits times 4, so it is exact in half precision and in
// bf16, and no product that a kernel forms from it carries a rounding of the cache.  At r 512 /
// d_R 64 a slot takes 256 + 16 + 128 = 400 bytes against 1152 in bf16.
//
// The 16-byte chunk c of row i lies at chunk position c ^ swizzle(i) of its row, so that eight
// rows' equal chunks fall into different shared-memory banks after a plain copy of the page; the
// key block's permutation is the one the tensor cores' 128-byte (64-byte) swizzle mode expects.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"
#include "sm100_ptx.cuh"

namespace mtla {
namespace qp {

constexpr int kPageRows = 64;
constexpr int kGroup = 32;
constexpr float kScaleMax = 10240.f;   // six steps of it (61440) still fit half precision
constexpr int kScaleNan = 0xff;

struct Format {
  int r, dr;
  __host__ __device__ int code_row() const { return r / 2; }
  __host__ __device__ int scale_row() const { return r / kGroup; }
  __host__ __device__ int key_row() const { return 2 * dr; }
  __host__ __device__ int off_scales() const { return 32 * r; }
  __host__ __device__ int off_keys() const { return 34 * r; }
  __host__ __device__ int page_bytes() const { return 34 * r + 128 * dr; }
  // Chunk permutations (see the head of the file).
  __host__ __device__ int code_mask() const {
    const int n = r / kGroup, low = n & -n;
    return (low < 8 ? low : 8) - 1;
  }
  __host__ __device__ int key_swizzle(int row) const { return dr == 64 ? (row & 7) : ((row >> 1) & 3); }
};

// Eight codes (32 bits) -> four half-precision pairs, in order.
__device__ __forceinline__ void decode8(uint32_t w, uint32_t (&o)[4]) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3])
      : "r"(w));
}
__device__ __forceinline__ uint32_t mul_h2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// One scale byte in both halves; two scale bytes (lo, hi).
__device__ __forceinline__ uint32_t scale_pair(uint32_t byte) { return (byte | (byte << 16)) << 7; }
__device__ __forceinline__ uint32_t scale_pair(uint32_t lo, uint32_t hi) { return (lo | (hi << 16)) << 7; }

// The smallest scale whose six steps reach `top` (a finite magnitude): 6 k q >= top with q the
// grid's step at that size.  k * q and 6 * k * q are exact, so the two corrections make the
// approximate quotient's ceiling exact.
__device__ __forceinline__ float pick_scale(float top) {
  const float t = top * (1.f / 6.f);
  const uint32_t e = max(__float_as_uint(t) >> 23, 127u - 14u);         // exponent, at least 2^-14
  const float q = __uint_as_float((e - 3u) << 23);
  float k = ceilf(t * __uint_as_float((254u - (e - 3u)) << 23));        // t / q
  if (6.f * ((k - 1.f) * q) >= top) k -= 1.f;
  if (6.f * (k * q) < top) k += 1.f;
  if (k > 16.f) k = 18.f;            // 17 q is off the grid: past 16 q its step is 2 q
  return fminf(k * q, kScaleMax);
}

struct RowArgs {
  uint8_t* pages;
  const int64_t* index;      // pool row (page * 64 + slot) of every row; outside the pool: skipped
  void* rows;                // [n][r + d_R], row_stride elements apart
  long long row_stride;
  long long pool_rows;
  int n, chunk;              // rows; rows of a CTA, at most kMaxChunk
  Format f;
};

constexpr int kRowThreads = 256, kMaxChunk = 256;

// A unit is 16 elements: half a group, so the two threads of a group are neighbours (a row has an
// even number of units).  A CTA reads the indices of its rows at once, a thread then keeps its place in
// the row and walks over rows, two or four in flight; the write walks over the rows that are kept
// only.  Both kernels should be bound by the bytes of the wide rows; what the write had to lose for
// that was instructions (131071 rows of r 512, half of them kept: 87 us comparing with all borders and
// with 64-bit index arithmetic, 51 us with threads idle at every skipped row, 31 us so).
template <typename T>
__device__ __forceinline__ void load16(const T* p, float (&x)[16]) {
  constexpr int V = Elem<T>::kVec;
#pragma unroll
  for (int i = 0; i < 16 / V; ++i) {
    float v[V];
    load_vec(p + i * V, v);
#pragma unroll
    for (int j = 0; j < V; ++j) x[i * V + j] = v[j];
  }
}
// Eight values -> eight codes, nearest, the even one on a tie, saturating.
__device__ __forceinline__ uint32_t encode8(const float (&y)[8]) {
  uint32_t o;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(o)
      : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
  return o;
}
// The same from the definition, by comparing |x| with the borders 0.25 s .. 5 s, which are exact in
// fp32: no quotient, hence no rounding that could move a value across a border.
inline __device__ __noinline__ uint32_t encode8_exact(const float* x, float s) {
  uint32_t code = 0;
  for (int i = 0; i < 8; ++i) {
    const float v = fabsf(x[i]);
    uint32_t c = (v > 0.25f * s) + (v >= 0.75f * s) + (v > 1.25f * s) + (v >= 1.75f * s) + (v > 2.5f * s) +
                 (v >= 3.5f * s) + (v > 5.f * s);
    c |= (__float_as_uint(x[i]) >> 28) & 8u;
    code |= c << (4 * i);
  }
  return code;
}
// Eight elements at scale s > 0, inv = 1 / s (off by 2^-24 at most).  An element that came from bf16
// has 8 significant bits and a border 7, so unless x / s is a border it is 2^-8 of one away from
// it, 2^-10 at least: rounding the quotient to steps of 2^-13 (by adding a number whose last bit that
// is) restores every border and moves nothing else across.  An fp32 element may be next to a
// border: if the codes of the quotient made slightly smaller and slightly larger agree they are right,
// else the definition decides.
template <typename T>
__device__ __forceinline__ uint32_t encode_group8(const float* x, float s, float inv) {
  float y[8];
  if constexpr (sizeof(T) == 2) {
    constexpr float kRound = 1536.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = copysignf(fmaf(x[i], inv, kRound) - kRound, x[i]);   // -0 keeps its sign
    return encode8(y);
  } else {
    float z[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float p = x[i] * inv;
      y[i] = p * (1.f - 0x1p-20f);
      z[i] = p * (1.f + 0x1p-20f);
    }
    const uint32_t lo = encode8(y), hi = encode8(z);
    return lo == hi ? lo : encode8_exact(x, s);
  }
}

// Rows into the pool.  A group with an infinity or a NaN gets a NaN scale.
template <typename T>
__global__ void __launch_bounds__(kRowThreads) qpool_write_kernel(RowArgs a) {
  const int units = (a.f.r + a.f.dr) / 16, lat_units = a.f.r / 16, rows = kRowThreads / units;
  const int lane_row = threadIdx.x / units, u = threadIdx.x - lane_row * units;
  const bool works = lane_row < rows;
  // One row's unit: x into the pool row `at` (outside the pool: nowhere, but the neighbour's exchange is joined).
  auto put = [&](float (&x)[16], long long at) {
    const bool keep = at >= 0;
    // The largest magnitude; a sum of x * 0 tells whether an infinity or a NaN is among them.
    float top = 0.f, odd = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      top = fmaxf(top, fabsf(x[i]));
      odd = fmaf(x[i], 0.f, odd);
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    odd += __shfl_xor_sync(0xffffffffu, odd, 1);
    if (!keep) return;
    uint8_t* page = a.pages + (at >> 6) * a.f.page_bytes();
    const int row = (int)(at & 63);
    if (u < lat_units) {
      const bool finite = odd == 0.f;
      const float s = finite ? pick_scale(top) : 0.f;
      uint32_t code[2] = {0u, 0u};
      if (s > 0.f) {
        const float inv = 1.f / s;
        code[0] = encode_group8<T>(x, s, inv);
        code[1] = encode_group8<T>(x + 8, s, inv);
      }
      const int chunk = (u >> 1) ^ (row & a.f.code_mask());
      *reinterpret_cast<uint2*>(page + row * a.f.code_row() + chunk * 16 + (u & 1) * 8) = make_uint2(code[0], code[1]);
      if (!(u & 1))
        page[a.f.off_scales() + row * a.f.scale_row() + (u >> 1)] =
            finite ? (uint8_t)(__half_as_ushort(__float2half_rn(s)) >> 7) : (uint8_t)kScaleNan;
    } else {
      const int c0 = (u - lat_units) * 2, sw = a.f.key_swizzle(row);
      uint8_t* keys = page + a.f.off_keys() + row * a.f.key_row();
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = x[h * 8 + j];
        store_vec(reinterpret_cast<bf16*>(keys + ((c0 + h) ^ sw) * 16), v);
      }
    }
  };
  __shared__ long long at_s[kMaxChunk];
  __shared__ int row_s[kMaxChunk], warp_kept[kRowThreads / 32];
  const int first = blockIdx.x * a.chunk, chunk = min(a.chunk, a.n - first), lane = threadIdx.x & 31,
            warp = threadIdx.x >> 5;
  const long long mine = (int)threadIdx.x < chunk ? a.index[first + threadIdx.x] : -1;
  const bool kept = mine >= 0 && mine < a.pool_rows;
  const uint32_t votes = __ballot_sync(0xffffffffu, kept);
  if (lane == 0) warp_kept[warp] = __popc(votes);
  __syncthreads();
  int place = __popc(votes & ((1u << lane) - 1u)), n_kept = 0;
#pragma unroll
  for (int i = 0; i < kRowThreads / 32; ++i) {
    if (i < warp) place += warp_kept[i];
    n_kept += warp_kept[i];
  }
  if (kept) {
    at_s[place] = mine;
    row_s[place] = first + threadIdx.x;
  }
  __syncthreads();
  for (int i0 = 0; i0 < n_kept; i0 += 2 * rows) {    // two rows of a thread in flight
    long long at[2];
    float x[2][16];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int k = i0 + i * rows + lane_row;
      at[i] = -1;
#pragma unroll
      for (int j = 0; j < 16; ++j) x[i][j] = 0.f;
      if (works && k < n_kept) {
        at[i] = at_s[k];
        load16(static_cast<const T*>(a.rows) + row_s[k] * a.row_stride + u * 16, x[i]);
      }
    }
    put(x[0], at[0]);
    put(x[1], at[1]);
  }
}

// Rows out of the pool, widened to T (exact in both types); zeros where the index is outside the pool.
// Eight elements a thread: a bf16 row is then written in full 16-byte steps by neighbouring threads
// (131071 rows of r 512, half of them zeros: 42 us, 151 MB written; with sixteen in two steps 44).
template <typename T>
__global__ void __launch_bounds__(kRowThreads) qpool_read_kernel(RowArgs a) {
  const int units = (a.f.r + a.f.dr) / 8, lat_units = a.f.r / 8, rows = kRowThreads / units;
  const int lane_row = threadIdx.x / units, u = threadIdx.x - lane_row * units;
  constexpr int kU = 4;                              // rows of a thread in flight
  __shared__ long long at_s[kMaxChunk];
  const int first = blockIdx.x * a.chunk, chunk = min(a.chunk, a.n - first);
  if ((int)threadIdx.x < chunk) at_s[threadIdx.x] = a.index[first + threadIdx.x];
  __syncthreads();
  if (lane_row >= rows) return;
  T* out = static_cast<T*>(a.rows) + first * a.row_stride + u * 8;
  for (int i0 = lane_row; i0 < chunk; i0 += kU * rows) {
    uint4 data[kU];                                  // a word of codes and its scale, or eight keys
#pragma unroll
    for (int i = 0; i < kU; ++i) {
      data[i] = make_uint4(0, 0, 0, 0);
      const long long at = i0 + i * rows < chunk ? at_s[i0 + i * rows] : -1;
      if (at < 0 || at >= a.pool_rows) continue;
      const uint8_t* page = a.pages + (at >> 6) * a.f.page_bytes();
      const int row = (int)(at & 63);
      if (u < lat_units) {
        const int chunk_at = (u >> 2) ^ (row & a.f.code_mask());
        data[i].x = *reinterpret_cast<const uint32_t*>(page + row * a.f.code_row() + chunk_at * 16 + (u & 3) * 4);
        data[i].y = page[a.f.off_scales() + row * a.f.scale_row() + (u >> 2)];
      } else {
        const int k = (u - lat_units) ^ a.f.key_swizzle(row);
        data[i] = *reinterpret_cast<const uint4*>(page + a.f.off_keys() + row * a.f.key_row() + k * 16);
      }
    }
#pragma unroll
    for (int i = 0; i < kU; ++i) {
      if (i0 + i * rows >= chunk) break;
      float x[8];
      if (u < lat_units) {
        uint32_t o[4];
        decode8(data[i].x, o);
        const uint32_t sc = scale_pair(data[i].y);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t v = mul_h2(o[j], sc);
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&v));
          x[2 * j] = f.x;
          x[2 * j + 1] = f.y;
        }
      } else {
        load_vec(reinterpret_cast<const bf16*>(&data[i]), x);
      }
      T* d = out + (long long)(i0 + i * rows) * a.row_stride;
      if constexpr (sizeof(T) == 2) {
        store_vec(d, x);
      } else {
        const float x0[4] = {x[0], x[1], x[2], x[3]}, x1[4] = {x[4], x[5], x[6], x[7]};
        store_vec(d, x0);
        store_vec(d + 4, x1);
      }
    }
  }
}

}  // namespace qp
}  // namespace mtla
