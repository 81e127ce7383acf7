// Products of a few rows with 4-bit weights: y[n][out] = x[n][in] . W[in][out].
//
// The weights' bytes bound the product as long as there are few rows.  This kernel keeps everything in registers: a
// lane's 16 bytes of a block are 32 inputs of one output, decoded to bf16 pairs in place as the A operand of the
// warp-level matrix instruction (m16n8k16: 16 outputs by 8 rows of x).  The order of the inputs inside a block of 128
// is permuted alike on both sides: lane (g, t) multiplies group t, so that it also reads x 16 bytes at a time.
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
// exactly (cut off, 8 bits each; an infinity is the first term alone).
template <typename T>
struct Operand;
template <>
struct Operand<bf16> {
  static constexpr int kTerms = 1;
  uint32_t p[1][4];
  __device__ __forceinline__ void load(const bf16* src, bool there) {
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (there) v = *reinterpret_cast<const uint4*>(src);
    p[0][0] = v.x; p[0][1] = v.y; p[0][2] = v.z; p[0][3] = v.w;
  }
};
template <>
struct Operand<float> {
  static constexpr int kTerms = 3;
  uint32_t p[3][4];
  __device__ __forceinline__ void load(const float* src, bool there) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0.f;
    if (there) {
      float lo[4], hi[4];
      load_vec(src, lo);
      load_vec(src + 4, hi);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = lo[i];
        x[4 + i] = hi[i];
      }
    }
#pragma unroll
    for (int t = 0; t < 3; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[t][i] = __byte_perm(__float_as_uint(x[2 * i]), __float_as_uint(x[2 * i + 1]), 0x7632);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float top = __uint_as_float(__float_as_uint(x[2 * i + h]) & 0xffff0000u);
          x[2 * i + h] = fabsf(top) == INFINITY ? 0.f : x[2 * i + h] - top;
        }
      }
  }
};

// A CTA per 16 outputs and 8 NT rows; its warps share the input blocks out, sums are joined in the warps' order.
template <typename T, int NT>
__global__ void __launch_bounds__(kThreads) qweight_product_kernel(ProductArgs a) {
  constexpr int TERMS = Operand<T>::kTerms;
  __shared__ float red[kWarps][kRows][8 * NT + 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int ob = blockIdx.x, n0 = blockIdx.y * 8 * NT, kbs = a.s.in_blocks();
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  float acc[NT][4];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
  const int kb0 = (int)((long long)kbs * warp / kWarps), kb1 = (int)((long long)kbs * (warp + 1) / kWarps);
  const uint8_t* block = a.packed + ((long long)ob * kbs + kb0) * kBlockBytes;
  for (int kb = kb0; kb < kb1; ++kb, block += kBlockBytes) {
    const uint8_t* codes = block + g * 64 + (t ^ (g >> 1 & 3)) * 16;
    const uint4 w0 = *reinterpret_cast<const uint4*>(codes), w1 = *reinterpret_cast<const uint4*>(codes + 512);
    const uint32_t two = *reinterpret_cast<const uint16_t*>(block + kCodeBytes + 2 * lane);
    const uint32_t s0 = scale_b2(two & 255u), s1 = scale_b2(two >> 8);
    const uint32_t word0[4] = {w0.x, w0.y, w0.z, w0.w}, word1[4] = {w1.x, w1.y, w1.z, w1.w};
    const int k = kb * kInputs + t * kGroup;
    float part[NT][4];                         // fp32: a block's products are added outside the matrix unit
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) part[j][i] = TERMS == 1 ? acc[j][i] : 0.f;
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
        Operand<T> x;
        const int row = n0 + 8 * j + g;
        x.load(static_cast<const T*>(a.x) + row * a.x_stride + k + 8 * m, row < a.n && k + 8 * m < a.s.n_in);
#pragma unroll
        for (int e = 0; e < TERMS; ++e) {
          qp::mma_bf16(part[j], a0, x.p[e][0], x.p[e][1]);
          qp::mma_bf16(part[j], a1, x.p[e][2], x.p[e][3]);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[j][i] = TERMS == 1 ? part[j][i] : acc[j][i] + part[j][i];
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
