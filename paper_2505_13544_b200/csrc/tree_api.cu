// C ABI of the operators for drafted trees (see include/mtla.h): argument checks and launches.
#include "mtla.h"

#include <math.h>

#include "common.cuh"
#include "ops_common.cuh"
#include "qpool_attn.cuh"
#include "tree_kernels.cuh"
#include "tree_attn_tc.cuh"

using namespace mtla;
using namespace mtla::ops;

namespace {

constexpr int kMostCtas = 2 * kPlanSms;          // of the launch over the context
constexpr int kLeastCols = 16, kMostCols = 64;   // of a group

// Sized for any group width, so that the choice between the kernels stays the call's.
struct TreePlan { size_t o_part, ml_part, parts, groups, prefix, first, listed, shares, error_words, image, total; };
long long most_groups(const mtla_qpool_config* c, int B, int n_nodes, int cols) {
  return (long long)n_nodes * c->n_heads / cols + (B < n_nodes ? B : n_nodes);
}
bool good_tree(const mtla_qpool_config* c, int B, int n_nodes) {
  return good_pool(c) && B >= 1 && B <= tree::kMaxRequests && n_nodes >= 0 &&
         (long long)n_nodes * c->n_heads <= 0x7fffffffll;
}
TreePlan plan_tree(const mtla_qpool_config* c, int B, int n_nodes) {
  TreePlan p;
  const size_t groups = (size_t)most_groups(c, B, n_nodes, kLeastCols);
  size_t cols = 0;                               // columns of all parts
  for (int w = kLeastCols; w <= kMostCols; w *= 2) {
    const size_t n = ((size_t)most_groups(c, B, n_nodes, w) + kMostCtas) * w;
    if (n > cols) cols = n;
  }
  p.o_part = 0;
  p.ml_part = align_up(cols * align_up(c->latent_rank, 128) * 4, 256);
  p.parts = p.ml_part + align_up(cols * 8, 256);
  p.groups = p.parts + align_up(groups * 8, 256);
  p.prefix = p.groups + align_up(groups * 16, 256);
  p.first = p.prefix + align_up((groups + 1) * 4, 256);
  p.listed = p.first + align_up(((size_t)B + 1) * 4, 256);
  p.shares = p.listed + 256;
  p.error_words = p.shares + align_up(kPlanSms * 16, 256);
  p.image = p.error_words + align_up(kPlanSms * 4, 256);
  size_t image = 0;
  for (int w = 32; w <= kMostCols; w *= 2) {
    const size_t n = (size_t)most_groups(c, B, n_nodes, w) * tree::image_bytes(w, format_of(c));
    if (n > image) image = n;
  }
  p.total = p.image + align_up(image, 256);
  return p;
}

template <typename T, int MH>
int launch_context(const qp::GroupArgs& a, long long tiles, const OnDeviceOf& dev, cudaStream_t st) {
  using L = qp::AttnLayout<MH, sizeof(T) == 2 ? 1 : 2>;
  if (!raise_smem<qp::qpool_attend_kernel<T, MH, true>>(dev.device())) return MTLA_ERR_CUDA;
  const int smem = L::bytes(a.f, 0);
  const int sms = dev.sm_count() < kPlanSms ? dev.sm_count() : kPlanSms, per_sm = smem <= 112 * 1024 ? 2 : 1;
  const int ctas = (int)(tiles < (long long)per_sm * sms ? tiles : (long long)per_sm * sms);
  return launch_dependent(qp::qpool_attend_kernel<T, MH, true>, dim3(ctas), qp::kAttnThreads, smem, st, a);
}

// The roles' registers come out of what the kernel is launched with; an increase that this does not cover would wait
// for ever, so nothing is launched then.  Asked once.
template <auto Kernel>
bool registers_suffice() {
  static std::atomic<int> known{0};                // 0 not asked, 1 yes, 2 no
  int state = known.load(std::memory_order_relaxed);
  if (state == 0) {
    cudaFuncAttributes attr;
    if (cudaFuncGetAttributes(&attr, Kernel) != cudaSuccess) return false;
    constexpr int kWarps = tree::kThreads / 32;
    state = (attr.numRegs + 7) / 8 * 8 * kWarps >= tree::kRoleRegisters ? 1 : 2;
    known.store(state, std::memory_order_relaxed);
  }
  return state == 1;
}

template <int NC, int NB>
int launch_context_tc(const qp::GroupArgs& a, int ctas, const OnDeviceOf& dev, cudaStream_t st) {
  if (!raise_smem<tree::tree_attend_tc_kernel<NC, NB>>(dev.device()) ||
      !registers_suffice<tree::tree_attend_tc_kernel<NC, NB>>())
    return MTLA_ERR_CUDA;
  const tree::Layout l(a.f, NC);
  return launch_dependent(tree::tree_attend_tc_kernel<NC, NB>, dim3(ctas), tree::kThreads,
                          l.total, st, a, l);
}
template <int NC>
int launch_context_tc(const qp::GroupArgs& a, int ctas, const OnDeviceOf& dev, cudaStream_t st) {
  switch (ceil_div(a.f.r, 128)) {
    case 1: return launch_context_tc<NC, 1>(a, ctas, dev, st);
    case 2: return launch_context_tc<NC, 2>(a, ctas, dev, st);
    case 3: return launch_context_tc<NC, 3>(a, ctas, dev, st);
    default: return launch_context_tc<NC, 4>(a, ctas, dev, st);
  }
}

template <typename T>
int launch_join(const tree::JoinArgs& a, long long groups, const OnDeviceOf& dev, cudaStream_t st) {
  // A CTA per column, of eight warps as long as all of them run at once (two on an SM), of four up to twice what runs at
  // once (four on an SM): 400 columns of 32773 slots 86 us with a warp per column, 69 so; 768 of 9000 57 and 50; but
  // 1536 of 1024 slots 26.5 and 29.5.
  const long long columns = (long long)a.n_nodes * a.heads, sms = dev.sm_count();
  if (columns <= 2 * sms)
    return launch_dependent(tree::tree_join_split_kernel<T, 8>, dim3((unsigned)columns), 256, 0, st, a);
  if (columns <= 8 * sms)
    return launch_dependent(tree::tree_join_split_kernel<T, 4>, dim3((unsigned)columns), 128, 0, st, a);
  if constexpr (sizeof(T) == 2) {
    if (a.cols == 64 && groups >= sms) {         // a group for every SM
      constexpr int kBytes = tree::Dense<64>::bytes(qp::Format{512, 64});
      if (!raise_smem<tree::tree_join_dense_kernel<64>>(dev.device(), kBytes)) return MTLA_ERR_CUDA;
      return launch_dependent(tree::tree_join_dense_kernel<64>, dim3((unsigned)groups), tree::Dense<64>::kThreads,
                              tree::Dense<64>::bytes(a.f), st, a);
    }
  }
  const long long ctas = (columns + tree::kJoinWarps - 1) / tree::kJoinWarps, most = 16 * sms;
  return launch_dependent(tree::tree_join_kernel<T>, dim3((unsigned)(ctas < most ? ctas : most)), tree::kJoinThreads, 0, st,
                          a);
}

// `run_out`: the self-test, in which a wait that runs out takes the place of the attention over the context.
int attend_tree(const mtla_qpool_config* cfg, const void* pages, const int32_t* table, int32_t table_width,
                const int32_t* slots, const int32_t* starts, int32_t B, const void* rows, int64_t row_stride,
                const int64_t* seen, const void* q, int32_t n_nodes, int32_t dtype, float scale, void* out, float* lse,
                void* workspace, size_t workspace_bytes, void* stream, bool run_out) {
  if (!pages || !table || !slots || !starts || !workspace || B < 1 || n_nodes < 0 || table_width < 1 ||
      !good_dtype(dtype) || !isfinite((float)((double)scale * kLog2e)) || (n_nodes > 0 && (!rows || !seen || !q || !out)))
    return MTLA_ERR_INVALID_ARG;
  if (!good_tree(cfg, B, n_nodes) || most_groups(cfg, B, n_nodes, kLeastCols) * table_width > 0x7fffffffll)
    return MTLA_ERR_UNSUPPORTED_SHAPE;
  const int width = cfg->latent_rank + cfg->rope_dim, vec = dtype == MTLA_DTYPE_BF16 ? 8 : 4;
  if (!aligned(pages, 16) || !aligned(rows, 16) || !aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 256) ||
      !aligned(table, 4) || !aligned(slots, 4) || !aligned(starts, 4) || !aligned(seen, 8) || !aligned(lse, 4) ||
      (n_nodes > 1 && (row_stride < width || row_stride % vec)))
    return MTLA_ERR_INVALID_ARG;
  const TreePlan p = plan_tree(cfg, B, n_nodes);
  if (workspace_bytes < p.total) return MTLA_ERR_ARENA_TOO_SMALL;
  if (n_nodes == 0) return MTLA_OK;
  OnDeviceOf dev(pages);
  if (dev.status() != MTLA_OK) return dev.status();
  char* ws = static_cast<char*>(workspace);
  cudaStream_t st = static_cast<cudaStream_t>(stream);

  const long long all_cols = (long long)n_nodes * cfg->n_heads;
  const bool tensor = dtype == MTLA_DTYPE_BF16;
  const int cols = tensor ? (all_cols > 32ll * B ? 64 : 32) : (all_cols > 16ll * B ? 32 : 16);
  tree::PlanArgs pa;
  pa.slots = slots;
  pa.starts = starts;
  pa.groups = reinterpret_cast<int4*>(ws + p.groups);
  pa.prefix = reinterpret_cast<int*>(ws + p.prefix);
  pa.first = reinterpret_cast<int*>(ws + p.first);
  pa.listed = reinterpret_cast<int2*>(ws + p.listed);
  pa.shares = reinterpret_cast<int4*>(ws + p.shares);
  pa.batch = B;
  pa.n_nodes = n_nodes;
  pa.heads = cfg->n_heads;
  pa.width = table_width;
  pa.cols = cols;
  pa.tile_pages = tensor ? 2 : 1;
  pa.q = static_cast<const bf16*>(q);
  pa.image = tensor ? reinterpret_cast<uint8_t*>(ws + p.image) : nullptr;
  pa.scale_log2 = (float)((double)scale * kLog2e);
  pa.f = format_of(cfg);
  const long long groups = most_groups(cfg, B, n_nodes, cols), images = tensor ? 2 * groups : 0;
  const int sms = dev.sm_count() < kPlanSms ? dev.sm_count() : kPlanSms;
  const long long tiles = groups * ceil_div(table_width, pa.tile_pages);
  pa.ctas = !tensor ? 0 : tiles < sms ? (int)tiles : sms;
  int status = launch_dependent(tree::tree_plan_kernel, dim3(1 + (unsigned)(images < 3 * sms ? images : 3 * sms)),
                                tree::kPlanThreads, 0, st, pa);
  if (status != MTLA_OK) return status;

  qp::GroupArgs a = {};
  a.pages = static_cast<const uint8_t*>(pages);
  a.table = table;
  a.q = q;
  a.o_part = reinterpret_cast<float*>(ws + p.o_part);
  a.ml_part = reinterpret_cast<float*>(ws + p.ml_part);
  a.seq_parts = reinterpret_cast<int2*>(ws + p.parts);
  a.error_words = reinterpret_cast<int*>(ws + p.error_words);
  a.scale_log2 = pa.scale_log2;
  a.n_heads = cfg->n_heads;
  a.width = table_width;
  a.n_pages = cfg->n_pages;
  a.f = pa.f;
  a.image = pa.image;
  a.shares = pa.shares;
  a.listed = pa.listed;
  a.prefix = pa.prefix;
  a.groups = pa.groups;
  a.cols = cols;
  if (run_out) {
    qp::wait_timeout_selftest_kernel<<<1, 64, 0, st>>>(a.error_words);
    status = launched();
  } else if (tensor)
    status = cols == 64 ? launch_context_tc<64>(a, pa.ctas, dev, st) : launch_context_tc<32>(a, pa.ctas, dev, st);
  else
    status = cols == 32 ? launch_context<float, 2>(a, tiles, dev, st) : launch_context<float, 1>(a, tiles, dev, st);
  if (status != MTLA_OK) return status;

  tree::JoinArgs j;
  j.q = q;
  j.rows = rows;
  j.seen = reinterpret_cast<const long long*>(seen);
  j.starts = starts;
  j.groups = pa.groups;
  j.first = pa.first;
  j.listed = pa.listed;
  j.parts = a.seq_parts;
  j.o_part = a.o_part;
  j.ml_part = a.ml_part;
  j.error_words = a.error_words;
  j.out = out;
  j.lse = lse;
  j.row_stride = row_stride;
  j.scale_log2 = a.scale_log2;
  j.batch = B;
  j.n_nodes = n_nodes;
  j.heads = cfg->n_heads;
  j.cols = cols;
  j.part_row = tensor ? (cfg->latent_rank + 127) / 128 * 128 : cfg->latent_rank;
  j.n_error_words = run_out ? 1 : pa.ctas;
  j.f = a.f;
  return dtype == MTLA_DTYPE_BF16 ? launch_join<bf16>(j, groups, dev, st) : launch_join<float>(j, groups, dev, st);
}

}  // namespace

extern "C" {

int mtla_tree_map(const int32_t* held, const int32_t* starts, const int32_t* parents, int32_t B, int32_t stride,
                  const mtla_tree_map_out* out, int32_t n_nodes, void* stream) {
  if (!held || !starts || !out || !out->slots || B < 1 || stride < 1 || n_nodes < 0) return MTLA_ERR_INVALID_ARG;
  if (n_nodes > 0 && (!parents || !out->seq || !out->position || !out->seen)) return MTLA_ERR_INVALID_ARG;
  const void* words[] = {held, starts, parents, out->seq, out->position, out->slots};
  for (const void* p : words)
    if (!aligned(p, 4)) return MTLA_ERR_INVALID_ARG;
  if (!aligned(out->seen, 8)) return MTLA_ERR_INVALID_ARG;
  if (B > tree::kMaxRequests) return MTLA_ERR_UNSUPPORTED_SHAPE;
  OnDeviceOf dev(out->slots);
  if (dev.status() != MTLA_OK) return dev.status();
  tree::MapArgs a;
  a.held = held;
  a.starts = starts;
  a.parents = parents;
  a.seq = out->seq;
  a.position = out->position;
  a.slots = out->slots;
  a.seen = reinterpret_cast<unsigned long long*>(out->seen);
  a.batch = B;
  a.n_nodes = n_nodes;
  a.stride = stride;
  return launch_dependent(tree::tree_map_kernel, dim3(ceil_div(B, tree::kMapThreads / 32)), tree::kMapThreads, 0,
                          static_cast<cudaStream_t>(stream), a);
}

size_t mtla_qpool_tree_workspace_bytes(const mtla_qpool_config* cfg, int32_t B, int32_t n_nodes) {
  return good_tree(cfg, B, n_nodes) ? plan_tree(cfg, B, n_nodes).total : 0;
}

int mtla_qpool_attend_tree(const mtla_qpool_config* cfg, const void* pages, const int32_t* table, int32_t table_width,
                           const int32_t* slots, const int32_t* starts, int32_t B, const void* rows, int64_t row_stride,
                           const int64_t* seen, const void* q, int32_t n_nodes, int32_t dtype, float scale, void* out,
                           float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  return attend_tree(cfg, pages, table, table_width, slots, starts, B, rows, row_stride, seen, q, n_nodes, dtype, scale, out,
                     lse, workspace, workspace_bytes, stream, false);
}

int mtla_selftest_tree_timeout(const mtla_qpool_config* cfg, const void* pages, const int32_t* table, int32_t table_width,
                               const int32_t* slots, const int32_t* starts, int32_t B, const void* rows,
                               int64_t row_stride, const int64_t* seen, const void* q, int32_t n_nodes, int32_t dtype,
                               float scale, void* out, float* lse, void* workspace, size_t workspace_bytes,
                               void* stream) {
  return attend_tree(cfg, pages, table, table_width, slots, starts, B, rows, row_stride, seen, q, n_nodes, dtype, scale, out,
                     lse, workspace, workspace_bytes, stream, true);
}

}  // extern "C"
