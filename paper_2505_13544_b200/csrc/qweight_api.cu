// C ABI of the products with 4-bit weights (see include/mtla.h): argument checks and launches.
#include "mtla.h"

#include "common.cuh"
#include "ops_common.cuh"
#include "qweight_format.cuh"
#include "qweight_kernels.cuh"

using namespace mtla;
using namespace mtla::ops;

namespace {

constexpr int kMostSize = 1 << 22;               // inputs or outputs (2^19 / 8 grid rows)

bool good_shape(int n_in, int n_out) {
  return n_in >= 8 && n_in % 8 == 0 && n_in <= kMostSize && n_out >= 1 && n_out <= kMostSize;
}

int pack_call(const void* w, int64_t stride, int32_t dtype, int32_t n_in, int32_t n_out, const void* packed, void* stream,
              bool pack) {
  if (!w || !packed || !good_dtype(dtype)) return MTLA_ERR_INVALID_ARG;
  if (!good_shape(n_in, n_out)) return MTLA_ERR_UNSUPPORTED_SHAPE;
  if (!aligned(packed, 16) || !aligned(w, dtype == MTLA_DTYPE_BF16 ? 2 : 4) || stride < n_out) return MTLA_ERR_INVALID_ARG;
  OnDeviceOf dev(packed);
  if (dev.status() != MTLA_OK) return dev.status();
  qw::PackArgs a;
  a.w = const_cast<void*>(w);
  a.packed = static_cast<uint8_t*>(const_cast<void*>(packed));
  a.stride = stride;
  a.s = qw::Shape{n_in, n_out};
  auto kernel = dtype == MTLA_DTYPE_BF16 ? (pack ? qw::qweight_pack_kernel<bf16> : qw::qweight_unpack_kernel<bf16>)
                                         : (pack ? qw::qweight_pack_kernel<float> : qw::qweight_unpack_kernel<float>);
  return launch_dependent(kernel, dim3(ceil_div(n_out, qw::kPackOut), a.s.in_blocks()), qw::kPackThreads, 0,
                          static_cast<cudaStream_t>(stream), a);
}

template <typename T, int NT>
int launch_product(const qw::ProductArgs& a, cudaStream_t st) {
  return launch_dependent(qw::qweight_product_kernel<T, NT>, dim3(a.s.out_blocks(), ceil_div(a.n, 8 * NT)), qw::kThreads,
                          0, st, a);
}

}  // namespace

extern "C" {

size_t mtla_qweight_bytes(int32_t n_in, int32_t n_out) {
  return good_shape(n_in, n_out) ? (size_t)qw::Shape{n_in, n_out}.bytes() : 0;
}

int mtla_qweight_pack(const void* w, int64_t w_stride, int32_t dtype, int32_t n_in, int32_t n_out, void* packed,
                      void* stream) {
  return pack_call(w, w_stride, dtype, n_in, n_out, packed, stream, true);
}

int mtla_qweight_unpack(const void* packed, int32_t n_in, int32_t n_out, void* w, int64_t w_stride, int32_t dtype,
                        void* stream) {
  return pack_call(w, w_stride, dtype, n_in, n_out, packed, stream, false);
}

int mtla_qweight_product(const void* packed, int32_t n_in, int32_t n_out, const void* x, int64_t x_stride, int32_t n,
                         void* y, int64_t y_stride, int32_t dtype, void* stream) {
  if (!packed || n < 0 || !good_dtype(dtype) || (n > 0 && (!x || !y))) return MTLA_ERR_INVALID_ARG;
  if (!good_shape(n_in, n_out) || n > kMostSize / 8) return MTLA_ERR_UNSUPPORTED_SHAPE;
  const int vec = dtype == MTLA_DTYPE_BF16 ? 8 : 4;
  if (!aligned(packed, 16) || !aligned(x, 16) || !aligned(y, 16 / vec) ||
      (n > 1 && (x_stride < n_in || x_stride % vec || y_stride < n_out)))
    return MTLA_ERR_INVALID_ARG;
  if (n == 0) return MTLA_OK;
  OnDeviceOf dev(packed);
  if (dev.status() != MTLA_OK) return dev.status();
  qw::ProductArgs a;
  a.packed = static_cast<const uint8_t*>(packed);
  a.x = x;
  a.y = y;
  a.x_stride = x_stride;
  a.y_stride = y_stride;
  a.n = n;
  a.s = qw::Shape{n_in, n_out};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dtype == MTLA_DTYPE_BF16)
    return n <= 8 ? launch_product<bf16, 1>(a, st) : n <= 16 ? launch_product<bf16, 2>(a, st)
                                                              : launch_product<bf16, 4>(a, st);
  return n <= 8 ? launch_product<float, 1>(a, st) : launch_product<float, 2>(a, st);
}

}  // extern "C"
