// C ABI of the products with 4-bit weights (see include/mtla.h): argument checks and launches.
#include "mtla.h"

#include "common.cuh"
#include "ops_common.cuh"
#include "qweight_format.cuh"
#include "qweight_kernels.cuh"
#include "qweight_tc.cuh"

using namespace mtla;
using namespace mtla::ops;

namespace {

constexpr int kMostSize = 1 << 22;               // outputs (2^19 / 8 grid rows)
// The matrix unit cuts its running sums off instead of rounding them, so a sum of one sign falls short in proportion to its
// length: by 3.6e-4 after the 4096 steps of 2^16 inputs in one CTA, a tenth of the result's rounding to bf16.
constexpr int kMostInputs = 1 << 16;

bool good_shape(int n_in, int n_out) {
  return n_in >= 8 && n_in % 8 == 0 && n_in <= kMostInputs && n_out >= 1 && n_out <= kMostSize;
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

template <typename T, int NT, int U>
int launch_product(const qw::ProductArgs& a, cudaStream_t st) {
  return launch_dependent(qw::qweight_product_kernel<T, NT, U>, dim3(a.s.out_blocks(), ceil_div(a.n, 8 * NT)), qw::kThreads,
                          0, st, a);
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_tiled_fn() {
  static std::atomic<EncodeTiledFn> known{nullptr};
  EncodeTiledFn fn = known.load(std::memory_order_acquire);
  if (fn) return fn;
  void* p = nullptr;
  cudaDriverEntryPointQueryResult found;
  if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess ||
      found != cudaDriverEntryPointSuccess)
    return nullptr;
  fn = reinterpret_cast<EncodeTiledFn>(p);
  known.store(fn, std::memory_order_release);
  return fn;
}

// Rows of x in boxes of `box` rows by 64 inputs (the swizzle's span); zeros outside.
bool make_x_map(CUtensorMap* map, const qw::ProductArgs& a, int box) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)a.s.n_in, (cuuint64_t)a.n}, strides[1] = {(cuuint64_t)a.x_stride * 2};
  const cuuint32_t boxes[2] = {64, (cuuint32_t)box}, steps[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(a.x), dims, strides, boxes, steps,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int BN, bool RUN_OUT = false>
int launch_product_tc(const qw::ProductArgs& p, const OnDeviceOf& dev, cudaStream_t st) {
  using C = qw::tc::Config<BN>;
  if (!raise_smem<qw::tc::qweight_tc_kernel<BN, RUN_OUT>>(dev.device(), C::kBytes)) return MTLA_ERR_CUDA;
  CUtensorMap map;
  if (!make_x_map(&map, p, BN)) return MTLA_ERR_CUDA;
  qw::tc::Args a;
  a.packed = p.packed;
  a.y = static_cast<bf16*>(p.y);
  a.y_stride = p.y_stride;
  a.n = p.n;
  a.s = p.s;
  a.pairs = p.s.n_out % 2 == 0 && p.y_stride % 2 == 0 && aligned(p.y, 4);
  const int tiles = ceil_div(p.s.n_out, qw::tc::kTile), row_tiles = ceil_div(p.n, BN);
  // The inputs are shared out, at least four blocks of 128 a CTA, as long as all CTAs run at once.
  const long long at_once = 2ll * dev.sm_count();
  a.splits = 1;
  while (a.splits < 8 && 2ll * a.splits * tiles * row_tiles <= at_once && p.s.in_blocks() >= 8 * a.splits) a.splits *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * a.splits), (unsigned)row_tiles);
  cfg.blockDim = dim3(qw::tc::kThreads);
  cfg.dynamicSmemBytes = C::kBytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = a.splits;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = a.splits > 1 ? 2 : 1;
  if (cudaLaunchKernelEx(&cfg, qw::tc::qweight_tc_kernel<BN, RUN_OUT>, map, a) == cudaSuccess) return MTLA_OK;
  cudaGetLastError();
  return MTLA_ERR_CUDA;
}

// What a call is refused for; fills in the kernels' arguments.
int product_args(qw::ProductArgs& a, const void* packed, int32_t n_in, int32_t n_out, const void* x, int64_t x_stride, int32_t n,
                 void* y, int64_t y_stride, int32_t dtype) {
  if (!packed || n < 0 || !good_dtype(dtype) || (n > 0 && (!x || !y))) return MTLA_ERR_INVALID_ARG;
  if (!good_shape(n_in, n_out) || n > kMostSize / 8) return MTLA_ERR_UNSUPPORTED_SHAPE;
  const int vec = dtype == MTLA_DTYPE_BF16 ? 8 : 4;
  if (!aligned(packed, 16) || !aligned(x, 16) || !aligned(y, 16 / vec) ||
      (n > 1 && (x_stride < n_in || x_stride % vec || y_stride < n_out)))
    return MTLA_ERR_INVALID_ARG;
  a.packed = static_cast<const uint8_t*>(packed);
  a.x = x;
  a.y = y;
  a.x_stride = x_stride;
  a.y_stride = y_stride;
  a.n = n;
  a.s = qw::Shape{n_in, n_out};
  return MTLA_OK;
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
  qw::ProductArgs a;
  const int status = product_args(a, packed, n_in, n_out, x, x_stride, n, y, y_stride, dtype);
  if (status != MTLA_OK || n == 0) return status;
  OnDeviceOf dev(packed);
  if (dev.status() != MTLA_OK) return dev.status();
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dtype == MTLA_DTYPE_FP32) return n <= 8 ? launch_product<float, 1, 1>(a, st) : launch_product<float, 2, 1>(a, st);
  // Several blocks' loads ahead as long as all CTAs run at once all the same, two on an SM.
  const bool ahead = a.s.out_blocks() <= 2 * dev.sm_count();
  if (n <= 8) return ahead ? launch_product<bf16, 1, 4>(a, st) : launch_product<bf16, 1, 1>(a, st);
  if (n <= 16 && (double)n_in * n_out <= 2e7)        // 16 rows of 8192 x 8192: 23.6 us, on the tensor cores 16.6
    return ahead ? launch_product<bf16, 2, 2>(a, st) : launch_product<bf16, 2, 1>(a, st);
  // More rows: the tensor cores' set-up and joining take 3 us longer, passes over the weights 2.2 us per 10^8
  // products (on the tensor cores and here, 64 rows of 1024 x 1024: 6.5 us and 4.6; 32 of 4096 x 4096: 9.2 and 12.3; 128 of
  // 2048 x 512: 7.6 and 6.9).  A pass is longer with many inputs and few outputs, which the rule does not see: 17 rows
  // of 4096 x 1024 take 7.1 us here where the tensor cores need 6.3, 24 rows 8.5 and 6.3, 32 rows of 2048 x 2048 7.0 and 6.1.
  if ((double)n * n_in * n_out <= 1.5e8) return launch_product<bf16, 4, 1>(a, st);
  if (n <= 32) return launch_product_tc<32>(a, dev, st);
  return n <= 64 ? launch_product_tc<64>(a, dev, st) : launch_product_tc<128>(a, dev, st);
}

int mtla_selftest_qweight_timeout(const void* packed, int32_t n_in, int32_t n_out, const void* x, int64_t x_stride, int32_t n,
                                  void* y, int64_t y_stride, void* stream) {
  qw::ProductArgs a;
  const int status = product_args(a, packed, n_in, n_out, x, x_stride, n, y, y_stride, MTLA_DTYPE_BF16);
  if (status != MTLA_OK || n == 0) return status;
  OnDeviceOf dev(packed);
  if (dev.status() != MTLA_OK) return dev.status();
  return launch_product_tc<32, true>(a, dev, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
