// Host side of the operator calls, shared by their translation units: the GPU that a call runs on, limits of
// shared memory, checks of the pool's configuration, launches.  No call holds state.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>

#include "common.cuh"
#include "mtla.h"
#include "qpool_format.cuh"

namespace mtla {
namespace ops {

inline bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Makes the GPU that owns `p` current for the call and puts the old one back afterwards: a caller
// may hold tensors on another GPU than the current one.  status() is MTLA_ERR_INVALID_ARG for
// memory that no GPU can reach.
class OnDeviceOf {
 public:
  explicit OnDeviceOf(const void* p) {
    cudaPointerAttributes attr;
    if (cudaPointerGetAttributes(&attr, p) != cudaSuccess || cudaGetDevice(&old_) != cudaSuccess) {
      cudaGetLastError();
      status_ = MTLA_ERR_CUDA;
      return;
    }
    if (attr.type != cudaMemoryTypeDevice && attr.type != cudaMemoryTypeManaged) {
      status_ = MTLA_ERR_INVALID_ARG;
      return;
    }
    device_ = attr.device;
    if (device_ != old_) {
      if (cudaSetDevice(device_) != cudaSuccess) { status_ = MTLA_ERR_CUDA; return; }
      switched_ = true;
    }
  }
  ~OnDeviceOf() { if (switched_) cudaSetDevice(old_); }
  int status() const { return status_; }
  int sm_count() const {
    static std::atomic<int> known[64];       // per GPU, 0 until asked
    int n = device_ < 64 ? known[device_].load(std::memory_order_relaxed) : 0;
    if (n > 0) return n;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device_) != cudaSuccess || n < 1) return 1;
    if (device_ < 64) known[device_].store(n, std::memory_order_relaxed);
    return n;
  }
  int device() const { return device_; }

 private:
  int old_ = 0, device_ = 0, status_ = MTLA_OK;
  bool switched_ = false;
};

inline int launched() { return cudaGetLastError() == cudaSuccess ? MTLA_OK : MTLA_ERR_CUDA; }

// Raises a kernel's dynamic shared-memory limit to what one CTA may have, once per device.
template <auto Kernel>
bool raise_smem(int device, int bytes = 227 * 1024 - 1024) {
  static std::atomic<uint64_t> done{0};
  const uint64_t bit = device < 64 ? 1ull << device : 0;
  if (bit && (done.load(std::memory_order_acquire) & bit)) return true;
  if (cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess)
    return false;
  done.fetch_or(bit, std::memory_order_release);
  return true;
}

inline bool good_pool(const mtla_qpool_config* c) {
  return c && c->n_heads >= 1 && c->n_heads <= 32 && c->latent_rank >= 64 && c->latent_rank <= 512 &&
         c->latent_rank % 64 == 0 && (c->rope_dim == 32 || c->rope_dim == 64) && c->n_pages >= 1;
}
inline bool good_dtype(int32_t d) { return d == MTLA_DTYPE_FP32 || d == MTLA_DTYPE_BF16; }

inline qp::Format format_of(const mtla_qpool_config* c) { return qp::Format{c->latent_rank, c->rope_dim}; }

constexpr int kPlanSms = 148;            // workspaces are sized for this many
constexpr double kLog2e = 1.4426950408889634;

// Launches `kernel` as a dependent of what runs before it on the stream.
template <typename K, typename... Args>
int launch_dependent(K* kernel, dim3 grid, int threads, size_t smem, cudaStream_t st, const Args&... args) {
  if (launch_kernel(kernel, grid, dim3(threads), smem, st, true, args...) == cudaSuccess) return MTLA_OK;
  cudaGetLastError();
  return MTLA_ERR_CUDA;
}

}  // namespace ops
}  // namespace mtla
