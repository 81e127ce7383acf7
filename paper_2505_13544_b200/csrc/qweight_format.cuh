// Weights in 4 bits: layout, decoding, and the kernels that pack and unpack them.
//
// A weight [in][out] is a code e2m1 times a scale per 32 inputs of an output, both as in the latent pool
// (qpool_format.cuh), so it is exact in bf16.  Blocks of 16 outputs by 128 inputs (both filled up with
// zeros) follow one another, input blocks fastest; a block is
//   codes   [16 outputs][4 groups of 32 inputs][16 bytes], the group at 16-byte chunk c ^ ((output >> 1) & 3), which
//           keeps eight rows' reads of one group in different shared-memory banks
//   scales  [8][4 groups][2]: that of output i and group c at 2 (4 (i & 7) + c) + (i >> 3)
// and takes 1088 bytes: 4.25 bits a weight.  A word of eight codes has inputs 2k in its lower and 2k + 1 in its upper
// half, k = 0 .. 3, signs at bits 15, 12, 14, 13 and magnitudes at 6, 3, 0, 9 of a half: with a magnitude at bits
// 8..6 and its sign at 15 a half is a bf16 number 2^126 times too small (a subnormal one for 0.5), so decoding a
// pair takes a mask and at most two shifts, and the product with scale * 2^113 leaves weight * 2^-13, exactly.
#pragma once

#include "qpool_format.cuh"

namespace mtla {
namespace qw {

constexpr int kRows = 16, kInputs = 128, kCodeBytes = 1024, kBlockBytes = 1088;
constexpr int kGroup = qp::kGroup;
constexpr float kUnit = 8192.f;          // what a product of decoded weights is too small by

struct Shape {
  int n_in, n_out;
  __host__ __device__ int in_blocks() const { return (n_in - 1) / kInputs + 1; }
  __host__ __device__ int out_blocks() const { return (n_out - 1) / kRows + 1; }
  __host__ __device__ long long bytes() const { return (long long)in_blocks() * out_blocks() * kBlockBytes; }
};

// A word's four pairs (of neighbouring inputs), times 2^-126.
__device__ __forceinline__ void decode8(uint32_t w, uint32_t (&o)[4]) {
  o[0] = w & 0x81c081c0u;
  o[1] = (w << 3) & 0x81c081c0u;
  o[2] = ((w << 6) & 0x01c001c0u) | ((w << 1) & 0x80008000u);
  o[3] = ((w >> 3) & 0x01c001c0u) | ((w << 2) & 0x80008000u);
}
__device__ __forceinline__ uint32_t mul_b2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// A scale byte times 2^113 in both halves (10240 * 2^113 is below 2^127; the byte 255 is NaN).
__device__ __forceinline__ uint32_t scale_b2(uint32_t byte) {
  const float s = __half2float(__ushort_as_half((unsigned short)(byte << 7))) * 0x1p113f;
  const __nv_bfloat162 v = __floats2bfloat162_rn(s, s);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// Eight codes in order, four bits each <-> a stored word.
__device__ __forceinline__ uint32_t spread(uint32_t nibbles) {
  constexpr int kSign[4] = {15, 12, 14, 13}, kMag[4] = {6, 3, 0, 9};
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t c = nibbles >> (4 * i);
    w |= (c >> 3 & 1u) << (kSign[i / 2] + 16 * (i % 2)) | (c & 7u) << (kMag[i / 2] + 16 * (i % 2));
  }
  return w;
}

struct PackArgs {
  void* w;                   // [n_in][n_out], stride elements apart
  uint8_t* packed;
  long long stride;
  Shape s;
};

// A thread per output and group of 32 inputs, 64 outputs by 4 groups a CTA: neighbouring threads read (and write)
// neighbouring outputs.  Done once for a weight, so left as it is: 4096 x 6720 is packed in 30 us from fp32 and 47 from bf16
// and unpacked in 21 and 19 (their bytes take 19 and 11).
constexpr int kPackOut = 64, kPackThreads = 256;

template <typename T>
__global__ void __launch_bounds__(kPackThreads) qweight_pack_kernel(PackArgs a) {
  const int o = blockIdx.x * kPackOut + threadIdx.x % kPackOut, c = threadIdx.x / kPackOut, kb = blockIdx.y;
  const int ob = o / kRows, i = o % kRows;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  if (ob >= a.s.out_blocks()) return;
  const T* src = static_cast<const T*>(a.w) + (long long)(kb * kInputs + c * kGroup) * a.stride + o;
  float x[kGroup], top = 0.f, odd = 0.f;
#pragma unroll
  for (int k = 0; k < kGroup; ++k) {
    x[k] = o < a.s.n_out && kb * kInputs + c * kGroup + k < a.s.n_in ? Elem<T>::to_float(src[k * a.stride]) : 0.f;
    top = fmaxf(top, fabsf(x[k]));
    odd = fmaf(x[k], 0.f, odd);                          // not zero with an infinity or a NaN among them
  }
  const bool finite = odd == 0.f;
  const float s = finite ? qp::pick_scale(top) : 0.f;
  uint32_t word[4] = {0u, 0u, 0u, 0u};
  if (s > 0.f) {
    const float inv = 1.f / s;
#pragma unroll
    for (int j = 0; j < 4; ++j) word[j] = spread(qp::encode_group8<T>(x + 8 * j, s, inv));
  }
  uint8_t* block = a.packed + ((long long)ob * a.s.in_blocks() + kb) * kBlockBytes;
  *reinterpret_cast<uint4*>(block + i * 64 + (c ^ (i >> 1 & 3)) * 16) = make_uint4(word[0], word[1], word[2], word[3]);
  block[kCodeBytes + 2 * (4 * (i & 7) + c) + (i >> 3)] =
      finite ? (uint8_t)(__half_as_ushort(__float2half_rn(s)) >> 7) : (uint8_t)qp::kScaleNan;
}

template <typename T>
__global__ void __launch_bounds__(kPackThreads) qweight_unpack_kernel(PackArgs a) {
  const int o = blockIdx.x * kPackOut + threadIdx.x % kPackOut, c = threadIdx.x / kPackOut, kb = blockIdx.y;
  const int ob = o / kRows, i = o % kRows;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  if (o >= a.s.n_out) return;
  const uint8_t* block = a.packed + ((long long)ob * a.s.in_blocks() + kb) * kBlockBytes;
  const uint4 w = *reinterpret_cast<const uint4*>(block + i * 64 + (c ^ (i >> 1 & 3)) * 16);
  const uint32_t word[4] = {w.x, w.y, w.z, w.w};
  const uint32_t sc = scale_b2(block[kCodeBytes + 2 * (4 * (i & 7) + c) + (i >> 3)]);
  const int k0 = kb * kInputs + c * kGroup;
  T* dst = static_cast<T*>(a.w) + (long long)k0 * a.stride + o;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t p[4];
    decode8(word[j], p);
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const uint32_t v = mul_b2(p[m], sc);
      const int k = 8 * j + 2 * m;
      if (k0 + k < a.s.n_in) dst[k * a.stride] = Elem<T>::from_float(__uint_as_float(v << 16) * kUnit);
      if (k0 + k + 1 < a.s.n_in) dst[(k + 1) * a.stride] = Elem<T>::from_float(__uint_as_float(v & 0xffff0000u) * kUnit);
    }
  }
}

}  // namespace qw
}  // namespace mtla
