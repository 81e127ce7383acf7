// Products of a few rows with 4-bit weights: y[n][out] = x[n][in] . W[in][out].
//
// The weights' bytes bound the product as long as there are few rows: 4.25 bits each, 1.4 us for 4096 x 4096, behind
// some 2 us of launch and first loads (one row takes 4.5 us).  This kernel keeps everything in registers: a lane's 16
// bytes of a block are 32 inputs of one output, decoded to bf16 pairs in place as the A operand of the warp-level matrix
// instruction (m16n8k16: 16 outputs by 8 rows of x).  The order of the inputs inside a block of 128 is permuted alike
// on both sides: lane (g, t) multiplies group t, so that it also reads x 16 bytes at a time.
#pragma once

#include "qpool_attn.cuh"
#include "qweight_format.cuh"

namespace mtla {
namespace qw {

struct ProductArgs {
  const uint8_t* packed;
  const void* x;             // [n][n_in], x_stride elements apart
  void* y;                   // [n][n_out], y_stride elements apart
  long long x_stride, y_stride;
  int n;
  Shape s;
};

constexpr int kWarps = 8, kThreads = 32 * kWarps;

// Eight consecutive elements of a row as B operands: bf16 as they are, fp32 as three bf16 terms that add up to it
// exactly (cut off, 8 bits each).  An infinity is the first term alone; a NaN may have its fraction in the lower half only,
// so that its first term is an infinity, but then what is left of it is a NaN.
template <typename T>
struct Operand;
template <>
struct Operand<bf16> {
  static constexpr int kTerms = 1;
  uint4 v;
  __device__ __forceinline__ void load(const bf16* src, bool there) {
    v = make_uint4(0u, 0u, 0u, 0u);
    if (there) v = *reinterpret_cast<const uint4*>(src);
  }
  __device__ __forceinline__ void split(uint32_t (&p)[1][4]) const {
    p[0][0] = v.x; p[0][1] = v.y; p[0][2] = v.z; p[0][3] = v.w;
  }
};
template <>
struct Operand<float> {
  static constexpr int kTerms = 3;
  float v[8];
  __device__ __forceinline__ void load(const float* src, bool there) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
    if (there) {
      float lo[4], hi[4];
      load_vec(src, lo);
      load_vec(src + 4, hi);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = lo[i];
        v[4 + i] = hi[i];
      }
    }
  }
  __device__ __forceinline__ void split(uint32_t (&p)[3][4]) const {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = v[i];
#pragma unroll
    for (int t = 0; t < 3; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[t][i] = __byte_perm(__float_as_uint(x[2 * i]), __float_as_uint(x[2 * i + 1]), 0x7632);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float top = __uint_as_float(__float_as_uint(x[2 * i + h]) & 0xffff0000u);
          x[2 * i + h] = fabsf(x[2 * i + h]) == INFINITY ? 0.f : x[2 * i + h] - top;
        }
      }
  }
};

// A CTA per 16 outputs and 8 NT rows; its warps share the input blocks out, sums are joined in the warps' order.  The
// loads of U blocks (weights, scales and x) are issued before the first of them is used.  That takes registers: one row
// of 4096 x 4096, where all CTAs run at once either way, takes 5.9 us with one block at a time and 4.5 with four; of
// 8192 x 8192 it takes 12.4 and 14.2 (bytes: 5.5).  fp32 rows pass over the weights once for every 16 rows, with three
// products each: 512 rows of 4096 x 6720 take 867 us (bf16 rows on the tensor cores: 28).
template <typename T, int NT, int U>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 && NT <= 2 && U == 1 ? 4 : 2) qweight_product_kernel(ProductArgs a) {
  constexpr int TERMS = Operand<T>::kTerms;
  __shared__ float red[kWarps][kRows][8 * NT + 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int ob = blockIdx.x, n0 = blockIdx.y * 8 * NT, kbs = a.s.in_blocks();
  const int kb0 = kbs * warp / kWarps, kb1 = kbs * (warp + 1) / kWarps;
  ptx::grid_launch_dependents();
  // The weights come into L2 while the work in front of this launch ends (a request, no access: what that work may
  // still write to them is seen).  One row of 4096 x 4096: 5.1 -> 4.7 us, in a row of calls.
  if (lane == 0 && kb1 > kb0 && blockIdx.y == 0)
    ptx::prefetch_l2(a.packed + ((long long)ob * kbs + kb0) * kBlockBytes, (kb1 - kb0) * kBlockBytes);
  ptx::grid_dependency_wait();
  float acc[NT][4];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
  const uint8_t* codes = a.packed + (long long)ob * kbs * kBlockBytes + g * 64 + (t ^ (g >> 1 & 3)) * 16;
  const uint8_t* scales = a.packed + (long long)ob * kbs * kBlockBytes + kCodeBytes + 2 * lane;
  for (int kb = kb0; kb < kb1; kb += U) {
    uint4 w0[U], w1[U];
    uint32_t two[U];
    Operand<T> x[U][4][NT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool there = kb + u < kb1;
      const long long at = (long long)(kb + (there ? u : 0)) * kBlockBytes;
      w0[u] = *reinterpret_cast<const uint4*>(codes + at);
      w1[u] = *reinterpret_cast<const uint4*>(codes + at + 512);
      two[u] = *reinterpret_cast<const uint16_t*>(scales + at);
      const int k = (kb + u) * kInputs + t * kGroup;
#pragma unroll
      for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const int row = n0 + 8 * j + g;
          x[u][m][j].load(static_cast<const T*>(a.x) + row * a.x_stride + k + 8 * m,
                          there && row < a.n && k + 8 * m < a.s.n_in);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (kb + u >= kb1) break;
      const uint32_t s0 = scale_b2(two[u] & 255u), s1 = scale_b2(two[u] >> 8);
      const uint32_t word0[4] = {w0[u].x, w0[u].y, w0[u].z, w0[u].w}, word1[4] = {w1[u].x, w1[u].y, w1[u].z, w1[u].w};
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        uint32_t r0[4], r1[4];
        decode8(word0[m], r0);
        decode8(word1[m], r1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          r0[i] = mul_b2(r0[i], s0);
          r1[i] = mul_b2(r1[i], s1);
        }
        const uint32_t a0[4] = {r0[0], r1[0], r0[1], r1[1]}, a1[4] = {r0[2], r1[2], r0[3], r1[3]};
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          uint32_t p[TERMS][4];
          x[u][m][j].split(p);
          float part[4];                       // fp32: products of 32 inputs are added outside the matrix unit
#pragma unroll
          for (int i = 0; i < 4; ++i) part[i] = TERMS == 1 ? acc[j][i] : 0.f;
#pragma unroll
          for (int e = TERMS - 1; e >= 0; --e) {
            qp::mma_bf16(part, a0, p[e][0], p[e][1]);
            qp::mma_bf16(part, a1, p[e][2], p[e][3]);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[j][i] = TERMS == 1 ? part[i] : acc[j][i] + part[i];
        }
      }
    }
  }
  // Fragment: outputs g and g + 8, rows 2t and 2t + 1.
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) red[warp][g + (i >> 1) * 8][8 * j + 2 * t + (i & 1)] = acc[j][i];
  __syncthreads();
  for (int e = threadIdx.x; e < kRows * 8 * NT; e += kThreads) {
    const int o = e % kRows, c = e / kRows;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) v += red[w][o][c];
    if (ob * kRows + o < a.s.n_out && n0 + c < a.n)
      static_cast<T*>(a.y)[(n0 + c) * a.y_stride + ob * kRows + o] = Elem<T>::from_float(v * kUnit);
  }
}

}  // namespace qw
}  // namespace mtla
