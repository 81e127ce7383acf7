// C ABI of the operators around the 4-bit latent pool (see include/mtla.h): argument checks and
// launches.  They hold no state: every buffer is the caller's and nothing is allocated.
#include "mtla.h"

#include <cuda.h>
#include <math.h>

#include <atomic>

#include "common.cuh"
#include "qpool_attn.cuh"
#include "qpool_attn_tc.cuh"
#include "qpool_format.cuh"
#include "rope_kernel.cuh"
#include "slot_map_kernel.cuh"

using namespace mtla;

namespace {

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

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

int launched() { return cudaGetLastError() == cudaSuccess ? MTLA_OK : MTLA_ERR_CUDA; }

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

bool good_pool(const mtla_qpool_config* c) {
  return c && c->n_heads >= 1 && c->n_heads <= 32 && c->latent_rank >= 64 && c->latent_rank <= 512 &&
         c->latent_rank % 64 == 0 && (c->rope_dim == 32 || c->rope_dim == 64) && c->n_pages >= 1;
}
bool good_dtype(int32_t d) { return d == MTLA_DTYPE_FP32 || d == MTLA_DTYPE_BF16; }

qp::Format format_of(const mtla_qpool_config* c) { return qp::Format{c->latent_rank, c->rope_dim}; }

// ---- rows in and out of the pool

int row_call(const mtla_qpool_config* cfg, const void* pages, const void* rows, int64_t row_stride, int32_t dtype,
             const int64_t* index, int32_t n, void* stream, bool write) {
  if (!pages || n < 0 || !good_dtype(dtype) || (n > 0 && (!rows || !index))) return MTLA_ERR_INVALID_ARG;
  if (!good_pool(cfg)) return MTLA_ERR_UNSUPPORTED_SHAPE;
  const int width = cfg->latent_rank + cfg->rope_dim, vec = dtype == MTLA_DTYPE_BF16 ? 8 : 4;
  if (!aligned(pages, 16) || !aligned(rows, 16) || !aligned(index, 8) ||
      (n > 1 && (row_stride < width || row_stride % vec)))
    return MTLA_ERR_INVALID_ARG;
  if (n == 0) return MTLA_OK;
  OnDeviceOf dev(pages);
  if (dev.status() != MTLA_OK) return dev.status();
  qp::RowArgs a;
  a.pages = static_cast<uint8_t*>(const_cast<void*>(pages));
  a.index = index;
  a.rows = const_cast<void*>(rows);
  a.row_stride = row_stride;
  a.pool_rows = (long long)cfg->n_pages * qp::kPageRows;
  a.n = n;
  a.f = format_of(cfg);
  // Rows of a CTA: those that its threads hold at once when there are few, more as the SMs fill up.
  const int at_once = qp::kRowThreads / (width / (write ? 16 : 8)), even = ceil_div(n, 8 * dev.sm_count());
  a.chunk = even < at_once ? at_once : even < qp::kMaxChunk ? even : qp::kMaxChunk;
  const int ctas = ceil_div(n, a.chunk);
  auto kernel = dtype == MTLA_DTYPE_BF16 ? (write ? qp::qpool_write_kernel<bf16> : qp::qpool_read_kernel<bf16>)
                                         : (write ? qp::qpool_write_kernel<float> : qp::qpool_read_kernel<float>);
  kernel<<<(unsigned)ctas, qp::kRowThreads, 0, static_cast<cudaStream_t>(stream)>>>(a);
  return launched();
}

// ---- attention

// CTAs of the attention launch: at most this many per SM fit, and the workspace is sized for it.
constexpr int kAttnCtasPerSm = 2;
constexpr int kPlanSms = 148;
constexpr int kPlanCtas = kAttnCtasPerSm * kPlanSms;

constexpr double kLog2e = 1.4426950408889634;

struct AttnPlan { size_t o_part, ml_part, seq_parts, error_words, total; };
AttnPlan plan_attend(const mtla_qpool_config* c, int B) {
  AttnPlan p;
  const size_t parts = (size_t)B + kPlanCtas;
  p.o_part = 0;
  p.ml_part = align_up(parts * c->n_heads * c->latent_rank * 4, 256);
  p.seq_parts = p.ml_part + align_up(parts * c->n_heads * 8, 256);
  p.error_words = p.seq_parts + align_up((size_t)B * 8, 256);
  p.total = p.error_words + align_up(kPlanSms * 4, 256);
  return p;
}

// Launches `kernel` as a dependent of what runs before it on the stream.
template <typename K, typename... Args>
int launch_dependent(K* kernel, dim3 grid, int threads, size_t smem, cudaStream_t st, const Args&... args) {
  if (launch_kernel(kernel, grid, dim3(threads), smem, st, true, args...) == cudaSuccess) return MTLA_OK;
  cudaGetLastError();
  return MTLA_ERR_CUDA;
}

template <typename T>
int launch_combine(const qp::AttnArgs& a, const OnDeviceOf& dev, cudaStream_t st) {
  if (!raise_smem<qp::qpool_combine_kernel<T>>(dev.device(), qp::kMaxBatch * 16)) return MTLA_ERR_CUDA;
  // As many CTAs as there can be pieces of split or empty sequences, six per SM at most.
  const long long pieces = (long long)a.batch * a.n_heads * ceil_div(a.f.r, qp::kCombineCols), most = 6 * kPlanSms;
  return launch_dependent(qp::qpool_combine_kernel<T>, dim3((unsigned)(pieces < most ? pieces : most)),
                          qp::kCombineThreads, (size_t)a.batch * 16, st, a);
}

template <typename T, int MH>
int launch_attend(qp::AttnArgs a, const OnDeviceOf& dev, cudaStream_t st) {
  using L = qp::AttnLayout<MH, sizeof(T) == 2 ? 1 : 2>;
  if (!raise_smem<qp::qpool_attend_kernel<T, MH>>(dev.device())) return MTLA_ERR_CUDA;
  a.n_error_words = 0;                       // this kernel has no wait that could run out
  const int smem = L::bytes(a.f, a.batch);
  const int sms = dev.sm_count() < kPlanSms ? dev.sm_count() : kPlanSms;
  const int per_sm = smem <= 112 * 1024 ? kAttnCtasPerSm : 1;
  const long long most = (long long)a.batch * a.width;
  const int ctas = (int)(most < (long long)per_sm * sms ? most : (long long)per_sm * sms);
  const int status = launch_dependent(qp::qpool_attend_kernel<T, MH>, dim3(ctas), qp::kAttnThreads, smem, st, a);
  return status == MTLA_OK ? launch_combine<T>(a, dev, st) : status;
}

template <int NHP, int NB>
int launch_attend_tc(qp::AttnArgs a, const OnDeviceOf& dev, cudaStream_t st) {
  if (!raise_smem<qp::qpool_attend_tc_kernel<NHP, NB>>(dev.device())) return MTLA_ERR_CUDA;
  const qp::tc::Layout l(a.f, NHP, a.batch);
  const int sms = dev.sm_count() < kPlanSms ? dev.sm_count() : kPlanSms;
  const long long most = (long long)a.batch * ceil_div(a.width, 2);
  const int ctas = (int)(most < sms ? most : sms);
  a.n_error_words = ctas;
  const int status =
      launch_dependent(qp::qpool_attend_tc_kernel<NHP, NB>, dim3(ctas), qp::tc::kThreads, l.total, st, a, l);
  return status == MTLA_OK ? launch_combine<bf16>(a, dev, st) : status;
}
template <int NHP>
int launch_attend_tc(const qp::AttnArgs& a, const OnDeviceOf& dev, cudaStream_t st) {
  switch (ceil_div(a.f.r, 128)) {
    case 1: return launch_attend_tc<NHP, 1>(a, dev, st);
    case 2: return launch_attend_tc<NHP, 2>(a, dev, st);
    case 3: return launch_attend_tc<NHP, 3>(a, dev, st);
    default: return launch_attend_tc<NHP, 4>(a, dev, st);
  }
}

}  // namespace

extern "C" {

// ---- slot maps

int mtla_slot_map(const int32_t* held, const int32_t* fresh, int32_t B, int32_t stride, int32_t* table,
                  int32_t table_width, const int32_t* free_pages, int32_t n_free, const mtla_slot_map_out* out,
                  int32_t n_tokens, void* stream) {
  if (!held || !fresh || !table || !out || B < 1 || stride < 1 || table_width < 1 || n_free < 0 || n_tokens < 0 ||
      (n_free > 0 && !free_pages))
    return MTLA_ERR_INVALID_ARG;
  if (!out->starts || !out->slots || !out->taken) return MTLA_ERR_INVALID_ARG;
  if (n_tokens > 0 && (!out->seq || !out->position || !out->slot || !out->store)) return MTLA_ERR_INVALID_ARG;
  const void* words[] = {held, fresh, table, free_pages, out->starts, out->slots, out->taken, out->seq, out->position};
  for (const void* p : words)
    if (!aligned(p, 4)) return MTLA_ERR_INVALID_ARG;
  if (!aligned(out->slot, 8) || !aligned(out->store, 8)) return MTLA_ERR_INVALID_ARG;
  if (B > sm::kMaxBatch) return MTLA_ERR_UNSUPPORTED_SHAPE;
  OnDeviceOf dev(table);
  if (dev.status() != MTLA_OK) return dev.status();
  sm::Args a;
  a.held = held;
  a.fresh = fresh;
  a.table = table;
  a.free_pages = free_pages;
  a.starts = out->starts;
  a.seq = out->seq;
  a.position = out->position;
  a.slot = reinterpret_cast<long long*>(out->slot);
  a.store = reinterpret_cast<long long*>(out->store);
  a.slots = out->slots;
  a.taken = out->taken;
  a.batch = B;
  a.stride = stride;
  a.width = table_width;
  a.n_free = n_free;
  a.n_tokens = n_tokens;
  a.vec = aligned(out->seq, 16) && aligned(out->position, 16) && aligned(out->slot, 16) && aligned(out->store, 16);
  const size_t smem = (3 * (size_t)B + 2) * 4;
  // Four tokens a thread once that still gives every SM a CTA.
  const bool four = n_tokens >= 4 * sm::kThreads * dev.sm_count();
  if (!(four ? raise_smem<sm::slot_map_kernel<4>>(dev.device()) : raise_smem<sm::slot_map_kernel<1>>(dev.device())))
    return MTLA_ERR_CUDA;
  const int work = sm::kThreads * (four ? 4 : 1);
  const int ctas = (int)(((long long)n_tokens + work - 1) / work), most = 4 * dev.sm_count();
  const cudaError_t e = launch_kernel(four ? sm::slot_map_kernel<4> : sm::slot_map_kernel<1>,
                                      dim3(ctas < 1 ? 1 : ctas < most ? ctas : most), dim3(sm::kThreads), smem,
                                      static_cast<cudaStream_t>(stream), true, a);
  if (e != cudaSuccess) cudaGetLastError();
  return e == cudaSuccess ? MTLA_OK : MTLA_ERR_CUDA;
}

// ---- rotary positions

int mtla_rope(const mtla_rope_config* cfg, const mtla_rope_tensor* tensors, int32_t n_tensors, int32_t dtype,
              const int32_t* positions, int32_t n_tokens, int32_t inverse, void* stream) {
  if (!cfg || !tensors || (n_tokens > 0 && !positions) || n_tensors < 1 || n_tokens < 0 || !good_dtype(dtype) ||
      !aligned(positions, 4))
    return MTLA_ERR_INVALID_ARG;
  if (n_tensors > rp::kMaxTensors) return MTLA_ERR_UNSUPPORTED_SHAPE;
  const int d = cfg->rope_dim;
  if (d < 2 || d % 2 || d / 2 > rp::kMaxPairs) return MTLA_ERR_UNSUPPORTED_SHAPE;
  if (cfg->layout != MTLA_ROPE_INTERLEAVED && cfg->layout != MTLA_ROPE_HALF) return MTLA_ERR_INVALID_ARG;
  const double theta = cfg->theta == 0.f ? 10000.0 : (double)cfg->theta;
  const double factor = cfg->factor == 0.f ? 1.0 : (double)cfg->factor;
  const float magnitude = cfg->magnitude == 0.f ? 1.f : cfg->magnitude;
  if (!(theta > 0.0) || !(factor > 0.0) || !isfinite(theta) || !isfinite(factor) || !isfinite(magnitude))
    return MTLA_ERR_INVALID_ARG;
  if (cfg->scaling != MTLA_ROPE_PLAIN && cfg->scaling != MTLA_ROPE_LINEAR && cfg->scaling != MTLA_ROPE_RAMP)
    return MTLA_ERR_INVALID_ARG;
  if (cfg->scaling == MTLA_ROPE_RAMP &&
      (cfg->train_tokens < 1 || !(cfg->ramp_high > cfg->ramp_low) || !isfinite(cfg->ramp_low) ||
       !isfinite(cfg->ramp_high)))
    return MTLA_ERR_INVALID_ARG;

  rp::Args a;
  const double two_pi = 6.283185307179586476925286766559;
  for (int k = 0; k < d / 2; ++k) {
    double f = pow(theta, -2.0 * k / d);
    if (cfg->scaling == MTLA_ROPE_LINEAR) {
      f /= factor;
    } else if (cfg->scaling == MTLA_ROPE_RAMP) {
      const double turns = cfg->train_tokens * f / two_pi;
      double keep = (turns - cfg->ramp_low) / ((double)cfg->ramp_high - cfg->ramp_low);
      keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
      f = f * keep + f / factor * (1.0 - keep);
    }
    a.turns[k] = f / two_pi;
  }
  const size_t elem = dtype == MTLA_DTYPE_BF16 ? 2 : 4;
  const int vec = (int)(16 / elem);
  const bool half = cfg->layout == MTLA_ROPE_HALF;
  bool use_vec = d % vec == 0 && (!half || (d / 2) % vec == 0);
  for (int n = 0; n < n_tensors; ++n) {
    const mtla_rope_tensor& t = tensors[n];
    if ((n_tokens > 0 && (!t.x || !t.y)) || t.n_heads < 1 || t.width < 1 || t.first < 0 || !aligned(t.x, elem) || !aligned(t.y, elem))
      return MTLA_ERR_INVALID_ARG;
    if (t.x_token_stride < 0 || t.x_head_stride < 0 || t.y_token_stride < 0 || t.y_head_stride < 0)
      return MTLA_ERR_INVALID_ARG;
    if (t.first > t.width - d || (long long)t.n_heads * t.width > (1 << 24)) return MTLA_ERR_UNSUPPORTED_SHAPE;
    // Rows of the result may not share elements, or their order would decide; in place means the same strides.
    const bool one = n_tokens <= 1;
    if ((t.n_heads > 1 && t.y_head_stride < t.width) ||
        (!one && t.y_token_stride < t.width) ||
        (!one && t.n_heads > 1 && t.y_token_stride < t.y_head_stride * (t.n_heads - 1) + t.width &&
         t.y_head_stride < t.y_token_stride * ((long long)n_tokens - 1) + t.width))
      return MTLA_ERR_INVALID_ARG;
    if (t.x && t.x == t.y && ((!one && t.x_token_stride != t.y_token_stride) ||
                       (t.n_heads > 1 && t.x_head_stride != t.y_head_stride)))
      return MTLA_ERR_INVALID_ARG;
    use_vec = use_vec && t.width % vec == 0 && t.first % vec == 0 && t.x_token_stride % vec == 0 &&
              t.x_head_stride % vec == 0 && t.y_token_stride % vec == 0 && t.y_head_stride % vec == 0 &&
              aligned(t.x, 16) && aligned(t.y, 16);
  }
  if (n_tokens == 0) return MTLA_OK;
  long long units = 0;
  for (int n = 0; n < n_tensors; ++n) {
    const mtla_rope_tensor& t = tensors[n];
    const int v = use_vec ? vec : 1;
    rp::Tensor& q = a.t[n];
    q.x = t.x;
    q.y = t.y;
    q.x_token = t.x_token_stride;
    q.x_head = t.x_head_stride;
    q.y_token = t.y_token_stride;
    q.y_head = t.y_head_stride;
    q.first = t.first;
    q.copy_units = t.x == t.y ? 0 : (t.width - d) / v;
    q.units = q.copy_units + (half ? d / 2 / v : (use_vec ? d / v : d / 2));
    q.all_units = t.n_heads * q.units;
    units += q.all_units;
  }
  a.per_token = (int)units;
  a.positions = positions;
  a.magnitude = magnitude;
  a.n_tensors = n_tensors;
  a.n_tokens = n_tokens;
  a.pairs = d / 2;
  a.inverse = inverse != 0;
  OnDeviceOf dev(tensors[0].y);
  if (dev.status() != MTLA_OK) return dev.status();
  // A token's units over as few rounds of the CTA's threads as they take, evenly; as many tokens side by
  // side as then fit.
  const int rounds = ceil_div(a.per_token, rp::kThreads);
  a.lanes = ceil_div(a.per_token, rounds);
  a.rows = rp::kThreads / a.lanes;
  // Tokens per CTA: four in flight for every thread, as long as every SM keeps several CTAs.
  int per = 1;
  while (per < rp::kMaxTokens && per < 4 * a.rows && ((long long)n_tokens + 2 * per - 1) / (2 * per) >= 4 * dev.sm_count())
    per *= 2;
  a.tokens_per_cta = per;
  // With few tokens the rounds run as CTAs of their own instead of one after the other.
  const dim3 grid(ceil_div(n_tokens, per), per == 1 && rounds < 65536 ? rounds : 1);
  auto pick = [&](auto bf, auto fp) { return dtype == MTLA_DTYPE_BF16 ? bf : fp; };
  auto kernel = use_vec ? (half ? pick(rp::rope_kernel<bf16, true, true>, rp::rope_kernel<float, true, true>)
                                : pick(rp::rope_kernel<bf16, true, false>, rp::rope_kernel<float, true, false>))
                        : (half ? pick(rp::rope_kernel<bf16, false, true>, rp::rope_kernel<float, false, true>)
                                : pick(rp::rope_kernel<bf16, false, false>, rp::rope_kernel<float, false, false>));
  const cudaError_t e =
      launch_kernel(kernel, grid, dim3(rp::kThreads), (size_t)per * a.pairs * 8, static_cast<cudaStream_t>(stream),
                    true, a);
  if (e != cudaSuccess) cudaGetLastError();
  return e == cudaSuccess ? MTLA_OK : MTLA_ERR_CUDA;
}

// ---- the 4-bit pool

size_t mtla_qpool_page_bytes(const mtla_qpool_config* cfg) {
  return good_pool(cfg) ? (size_t)format_of(cfg).page_bytes() : 0;
}

int mtla_qpool_write(const mtla_qpool_config* cfg, void* pages, const void* rows, int64_t row_stride, int32_t dtype,
                     const int64_t* index, int32_t n, void* stream) {
  return row_call(cfg, pages, rows, row_stride, dtype, index, n, stream, true);
}

int mtla_qpool_read(const mtla_qpool_config* cfg, const void* pages, const int64_t* index, int32_t n, void* rows,
                    int64_t row_stride, int32_t dtype, void* stream) {
  return row_call(cfg, pages, rows, row_stride, dtype, index, n, stream, false);
}

size_t mtla_qpool_workspace_bytes(const mtla_qpool_config* cfg, int32_t B) {
  return good_pool(cfg) && B >= 1 && B <= qp::kMaxBatch ? plan_attend(cfg, B).total : 0;
}

int mtla_qpool_attend(const mtla_qpool_config* cfg, const void* pages, const int32_t* table, int32_t table_width,
                      const int32_t* slots, int32_t B, const void* q, int32_t dtype, float scale, void* out,
                      float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  if (!pages || !table || !slots || !q || !out || !workspace || B < 1 || table_width < 1 || !good_dtype(dtype) ||
      !isfinite((float)((double)scale * kLog2e)))
    return MTLA_ERR_INVALID_ARG;
  if (!good_pool(cfg) || B > qp::kMaxBatch || (long long)B * table_width > 0x7fffffffll)
    return MTLA_ERR_UNSUPPORTED_SHAPE;
  if (!aligned(pages, 16) || !aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 256) || !aligned(table, 4) ||
      !aligned(slots, 4) || !aligned(lse, 4))
    return MTLA_ERR_INVALID_ARG;
  const AttnPlan p = plan_attend(cfg, B);
  if (workspace_bytes < p.total) return MTLA_ERR_ARENA_TOO_SMALL;
  OnDeviceOf dev(pages);
  if (dev.status() != MTLA_OK) return dev.status();
  char* ws = static_cast<char*>(workspace);
  qp::AttnArgs a;
  a.pages = static_cast<const uint8_t*>(pages);
  a.table = table;
  a.slots = slots;
  a.q = q;
  a.out = out;
  a.lse = lse;
  a.o_part = reinterpret_cast<float*>(ws + p.o_part);
  a.ml_part = reinterpret_cast<float*>(ws + p.ml_part);
  a.seq_parts = reinterpret_cast<int2*>(ws + p.seq_parts);
  a.scale_log2 = (float)((double)scale * kLog2e);
  a.n_heads = cfg->n_heads;
  a.batch = B;
  a.width = table_width;
  a.n_pages = cfg->n_pages;
  a.f = format_of(cfg);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  a.error_words = reinterpret_cast<int*>(ws + p.error_words);
  const bool wide = cfg->n_heads > 16;
  // The tensor-core kernel, except where its longer set-up shows: at most a page per SM of 64 latents
  // (4 heads, 20 slots: 7.5 us against 6.9; 3 x 200 slots: 8.8 against 8.6; but 8 heads of r 256, 512
  // slots: 9.8 against 10.3; 64 sequences of two pages: 10.8 against 12.4).  fp32 queries, and batches of
  // more sequences than it keeps lists of, also take the other one (1023 x 1024 slots, 32 heads, r 512: 605
  // us, where 1022 take 193).
  const bool small = (long long)B * table_width <= kPlanSms && cfg->latent_rank <= 64;
  if (dtype == MTLA_DTYPE_BF16 && B <= qp::tc::kMaxBatch && !small)
    return wide ? launch_attend_tc<32>(a, dev, st) : launch_attend_tc<16>(a, dev, st);
  if (dtype == MTLA_DTYPE_BF16)
    return wide ? launch_attend<bf16, 2>(a, dev, st) : launch_attend<bf16, 1>(a, dev, st);
  return wide ? launch_attend<float, 2>(a, dev, st) : launch_attend<float, 1>(a, dev, st);
}

int mtla_selftest_qpool_timeout(const mtla_qpool_config* cfg, const int32_t* slots, int32_t B, int32_t dtype, void* out,
                                float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  if (!slots || !out || !workspace || B < 1 || !good_dtype(dtype) || !aligned(slots, 4) || !aligned(out, 16) ||
      !aligned(lse, 4) || !aligned(workspace, 256))
    return MTLA_ERR_INVALID_ARG;
  if (!good_pool(cfg) || B > qp::kMaxBatch) return MTLA_ERR_UNSUPPORTED_SHAPE;
  const AttnPlan p = plan_attend(cfg, B);
  if (workspace_bytes < p.total) return MTLA_ERR_ARENA_TOO_SMALL;
  OnDeviceOf dev(out);
  if (dev.status() != MTLA_OK) return dev.status();
  char* ws = static_cast<char*>(workspace);
  qp::AttnArgs a = {};
  a.slots = slots;
  a.out = out;
  a.lse = lse;
  a.o_part = reinterpret_cast<float*>(ws + p.o_part);
  a.ml_part = reinterpret_cast<float*>(ws + p.ml_part);
  a.seq_parts = reinterpret_cast<int2*>(ws + p.seq_parts);
  a.error_words = reinterpret_cast<int*>(ws + p.error_words);
  a.n_error_words = 1;
  a.n_heads = cfg->n_heads;
  a.batch = B;
  a.f = format_of(cfg);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  qp::wait_timeout_selftest_kernel<<<1, 64, 0, st>>>(a.error_words);
  if (launched() != MTLA_OK) return MTLA_ERR_CUDA;
  return dtype == MTLA_DTYPE_BF16 ? launch_combine<bf16>(a, dev, st) : launch_combine<float>(a, dev, st);
}

}  // extern "C"
