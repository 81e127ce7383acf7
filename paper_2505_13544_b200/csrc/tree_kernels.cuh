// Drafted trees over the 4-bit pool: positions and masks of the nodes, the list of column groups that the
// attention over the context works through, and the kernel that adds the drafted rows and joins everything.
//
// A request's columns are its nodes times the heads; a column is a query row [r + d_R] and an output row [r],
// both at index column of the flat tensors.  All nodes of a request see the same context slots (a path continues
// the open slot, so only closed ones are left, and those are common), which makes the context's part the attention
// of `columns` queries over one list of pages without any mask.  Groups of up to kCols columns take the place that
// sequences have in qpool_attn.cuh.
#pragma once

#include "qpool_attn.cuh"

namespace mtla {
namespace tree {

constexpr int kMaxNodes = 64;            // of a request, as far as masks reach

// ---- positions, masks

struct MapArgs {
  const int *held, *starts, *parents;
  int *seq, *position, *slots;
  unsigned long long* seen;
  int batch, n_nodes, stride;
};

constexpr int kMapThreads = 128;

// A warp per request, two nodes a lane.  The set of a node's ancestors doubles its reach with every one of six
// rounds (path |= path of the node 2^k above), its depth is the set's size, and what it sees is the set cut
// with that of the nodes that close a chunk, plus itself.  Bound by the launch and the chain of loads.
__global__ void __launch_bounds__(kMapThreads) tree_map_kernel(MapArgs a) {
  __shared__ unsigned long long path_s[kMapThreads / 32][kMaxNodes];
  __shared__ int up_s[kMapThreads / 32][kMaxNodes];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = gridDim.x * (kMapThreads / 32);
  const int w0 = blockIdx.x * (kMapThreads / 32) + warp;
  unsigned long long* path = path_s[warp];
  int* up = up_s[warp];
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  // Every CTA looks over the whole batch: `starts` has to ascend inside the nodes.
  bool wrong = false;
  for (int b = threadIdx.x; b <= a.batch; b += kMapThreads)
    wrong |= a.starts[b] < (b ? a.starts[b - 1] : 0) || a.starts[b] > a.n_nodes;
  const bool refused = __syncthreads_or(wrong);
  // Nodes of no request.
  const int begin = refused ? a.n_nodes : a.starts[0], end = refused ? a.n_nodes : a.starts[a.batch];
  for (int k = w0 * 32 + lane; k < begin + a.n_nodes - end; k += warps * 32) {
    const int i = k < begin ? k : end + k - begin;
    a.seq[i] = -1;
    a.position[i] = 0;
    a.seen[i] = 0;
  }
  for (int b = w0; b < a.batch; b += warps) {
    const int lo = a.starts[b], hi = a.starts[b + 1], held = a.held[b], count = hi - lo;
    if (lane == 0) a.slots[b] = held > 0 ? held / a.stride : 0;
    if (refused || count == 0) continue;
    bool bad = held < 0 || count > kMaxNodes;
    unsigned long long mine[2];
    int above[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int i = lane + 32 * j;
      mine[j] = 0;
      above[j] = -1;
      if (i < count) {
        const int p = a.parents[lo + i];
        bad |= p < -1 || p >= i;
        above[j] = p;
        if (p >= 0 && p < i) mine[j] = 1ull << p;
      }
      if (i >= count || above[j] < 0 || above[j] >= i) above[j] = -1;
    }
    bad = __any_sync(0xffffffffu, bad);
#pragma unroll
    for (int k = 0; k < 6; ++k) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        path[lane + 32 * j] = mine[j];
        up[lane + 32 * j] = above[j];
      }
      __syncwarp();
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (above[j] >= 0) {
          mine[j] |= path[above[j]];
          above[j] = up[above[j]];
        }
      __syncwarp();
    }
    long long pos[2];
    uint32_t closes[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      pos[j] = (long long)held + __popcll(mine[j]);
      const bool there = lane + 32 * j < count;
      bad |= there && pos[j] > 0x7fffffffll;
      closes[j] = __ballot_sync(0xffffffffu, there && (pos[j] + 1) % a.stride == 0);
    }
    bad = __any_sync(0xffffffffu, bad);
    const unsigned long long closing = closes[0] | (unsigned long long)closes[1] << 32;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int i = lane + 32 * j;
      if (i >= count) continue;
      a.seq[lo + i] = bad ? -1 : b;
      a.position[lo + i] = bad ? 0 : (int)pos[j];
      a.seen[lo + i] = bad ? 0 : (mine[j] & closing) | 1ull << i;
    }
    for (int i = kMaxNodes + lane; i < count; i += 32) {       // only of a refused request
      a.seq[lo + i] = -1;
      a.position[lo + i] = 0;
      a.seen[lo + i] = 0;
    }
  }
}

// ---- column groups

struct PlanArgs {
  const int *slots, *starts;
  int4* groups;              // request, first column, columns, slots
  int* prefix;               // [groups + 1] tiles before every group
  int* first;                // [batch + 1] first group of every request
  int* n_groups;
  const bf16* q;             // [n_nodes][heads][r + d_R]
  uint8_t* image;            // [groups] of image_bytes, or nullptr
  float scale_log2;
  int batch, n_nodes, heads, width, cols, tile_pages;
  qp::Format f;
};

constexpr int kPlanThreads = 512;
constexpr int kMaxRequests = 4096;

// A group's queries for the tensor-core kernel, as they lie in its shared memory: r / 64 panels [cols][64] half
// precision with the 128-byte swizzle, one panel [cols][d_R] bf16 (128- or 64-byte swizzle), and what a column's scores
// are to be multiplied by.
__host__ __device__ inline int image_bytes(int cols, const qp::Format& f) { return cols * (2 * (f.r + f.dr) + 4); }

// One column into its group's image, by a warp.  The row is scaled by the power of two that brings its largest
// element into [2^14, 2^15), exactly down to 2^-39 of that; a column that does not exist is zero.
__device__ __forceinline__ void put_column(const bf16* q, bool there, uint8_t* image, int col, int cols, float scale_log2,
                                           const qp::Format& f) {
  const int lane = threadIdx.x & 31, r = f.r, dr = f.dr, n8 = (r + dr) / 8;
  uint4 w[3];                                    // r + d_R is 576 at most
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const int c = lane + 32 * i;
    w[i] = make_uint4(0u, 0u, 0u, 0u);
    if (there && c < n8) w[i] = *reinterpret_cast<const uint4*>(q + 8 * c);
    const uint32_t x[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
    for (int m = 0; m < 4; ++m) top = max(top, max(x[m] & 0x7fff0000u, (x[m] << 16) & 0x7fff0000u));
  }
  top = __reduce_max_sync(0xffffffffu, top);
  // Exponents -113 .. 140 (a row of subnormal numbers only reaches less); none for zeros and specials.
  const bool fine = top > 0 && top < 0x7f800000u;
  const int e = fine ? 141 - max((int)(top >> 23), 1) : 0, e1 = e / 2, e2 = e - e1;
  const float f1 = __uint_as_float((127 + e1) << 23), f2 = __uint_as_float((127 + e2) << 23);
  if (lane == 0)
    reinterpret_cast<float*>(image + (long long)cols * 2 * (r + dr))[col] =
        scale_log2 * __uint_as_float((127 - e1) << 23) * __uint_as_float((127 - e2) << 23);
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const int c = lane + 32 * i;
    if (c >= n8) break;
    const uint32_t x[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
    const bool latent = 8 * c < r;
    uint32_t y[4];
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const float lo = __uint_as_float(x[m] << 16) * f1 * f2, hi = __uint_as_float(x[m] & 0xffff0000u) * f1 * f2;
      const __half2 l2 = __floats2half2_rn(lo, hi);
      const __nv_bfloat162 k2 = __floats2bfloat162_rn(lo, hi);
      y[m] = latent ? *reinterpret_cast<const uint32_t*>(&l2) : *reinterpret_cast<const uint32_t*>(&k2);
    }
    const int at = latent ? (c >> 3) * cols * 128 + col * 128 + ((c ^ col) & 7) * 16
                          : cols * 2 * r + col * 2 * dr + ((c - r / 8) ^ f.key_swizzle(col)) * 16;
    *reinterpret_cast<uint4*>(image + at) = make_uint4(y[0], y[1], y[2], y[3]);
  }
}

// Two prefix sums over the requests (groups, tiles) in every CTA; the first enters the list, a warp per request, the
// others (of bf16 queries) write the groups' images, half a group each in turn.  A batch whose `starts` do not ascend inside
// the nodes gets no groups and a count of -1.  As a part of the attention, each CTA writing the image of its next
// group itself when the last one's products are done, the images took 13000 cycles of every change between groups.
__global__ void __launch_bounds__(kPlanThreads, 3) tree_plan_kernel(PlanArgs a) {
  __shared__ int s_first[kMaxRequests + 1], s_tile[kMaxRequests + 1];
  __shared__ int warp_g[kPlanThreads / 32], warp_t[kPlanThreads / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  auto tiles_of = [&](int b) {
    const int n = max(a.slots[b], 0);
    const int pages = min(n / qp::kPageRows + (n % qp::kPageRows != 0), a.width);
    return (pages + a.tile_pages - 1) / a.tile_pages;
  };
  const int per = ceil_div(a.batch, kPlanThreads), lo = min(a.batch, tid * per), hi = min(a.batch, lo + per);
  bool wrong = a.starts[0] < 0;
  for (int b = lo; b < hi; ++b) wrong |= a.starts[b] > a.starts[b + 1] || a.starts[b + 1] > a.n_nodes;
  if (__syncthreads_or(wrong)) {
    if (blockIdx.x == 0 && tid == 0) {
      *a.n_groups = -1;
      a.prefix[0] = 0;
    }
    return;
  }
  // Ascending requests have at most as many groups as there is room for, and tiles that the host has found to fit
  // 32 bits.
  int sum_g = 0, sum_t = 0;
  for (int b = lo; b < hi; ++b) {
    const int g = ceil_div((a.starts[b + 1] - a.starts[b]) * a.heads, a.cols);
    s_first[b] = sum_g;
    s_tile[b] = sum_t;
    sum_g += g;
    sum_t += g * tiles_of(b);
  }
  int in_g = sum_g, in_t = sum_t;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int g = __shfl_up_sync(0xffffffffu, in_g, o), t = __shfl_up_sync(0xffffffffu, in_t, o);
    if (lane >= o) { in_g += g; in_t += t; }
  }
  if (lane == 31) { warp_g[warp] = in_g; warp_t[warp] = in_t; }
  __syncthreads();
  int base_g = in_g - sum_g, base_t = in_t - sum_t;
  for (int w = 0; w < warp; ++w) { base_g += warp_g[w]; base_t += warp_t[w]; }
  for (int b = lo; b < hi; ++b) { s_first[b] += base_g; s_tile[b] += base_t; }
  if (hi == a.batch && lo < hi) { s_first[a.batch] = base_g + sum_g; s_tile[a.batch] = base_t + sum_t; }
  __syncthreads();
  const int total = s_first[a.batch];
  if (blockIdx.x == 0) {
    for (int b = tid; b <= a.batch; b += kPlanThreads) a.first[b] = s_first[b];
    for (int b = warp; b < a.batch; b += kPlanThreads / 32) {
      const int col0 = a.starts[b] * a.heads, cols = a.starts[b + 1] * a.heads - col0, tiles = tiles_of(b);
      const int slots = min(max(a.slots[b], 0), (int)min((long long)a.width * qp::kPageRows, 0x7fffffffll));
      const int g0 = s_first[b], n = s_first[b + 1] - g0;
      for (int i = lane; i < n; i += 32) {
        a.groups[g0 + i] = make_int4(b, col0 + i * a.cols, min(a.cols, cols - i * a.cols), slots);
        a.prefix[g0 + i] = s_tile[b] + i * tiles;
      }
    }
    if (tid == 0) {
      *a.n_groups = total;
      a.prefix[total] = s_tile[a.batch];
    }
    return;
  }
  for (int u = blockIdx.x - 1; u < 2 * total; u += gridDim.x - 1) {
    const int v = u >> 1, half = a.cols / 2;
    int b = 0, end = a.batch;                          // the request: the last one that begins at v or before it
    while (end - b > 1) {
      const int mid = (b + end) >> 1;
      if (s_first[mid] <= v) b = mid; else end = mid;
    }
    const int skip = (v - s_first[b]) * a.cols, col0 = a.starts[b] * a.heads + skip;
    const int cols = a.starts[b + 1] * a.heads - col0;
    for (int c = (u & 1) * half + warp; c < ((u & 1) + 1) * half; c += kPlanThreads / 32)
      put_column(a.q + (long long)(col0 + c) * (a.f.r + a.f.dr), c < cols, a.image + (long long)v * image_bytes(a.cols, a.f),
                 c, a.cols, a.scale_log2, a.f);
  }
}

// ---- drafted rows and the join

struct JoinArgs {
  const void* q;             // [n_nodes][heads][r + d_R]
  const void* rows;          // [n_nodes][r + d_R], row_stride elements apart
  const long long* seen;     // [n_nodes]
  const int* starts;
  const int4* groups;
  const int *first, *n_groups;
  const int2* parts;         // [groups] first part, number of parts
  const float* o_part;       // [parts][cols][r]
  const float* ml_part;      // [parts][cols][2]
  const int* error_words;
  void* out;
  float* lse;
  long long row_stride;
  float scale_log2;
  int batch, n_nodes, heads, cols, n_error_words;
  qp::Format f;
};

// What has been joined of one column: reference (log2 units), denominator, sums; a lane holds E latents.
template <typename T>
struct Running {
  static constexpr int V = Elem<T>::kVec, R = 512 / (32 * V), E = R * V;       // runs of 16 bytes of a row
  float m, l, acc[E];
  __device__ __forceinline__ void clear() {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
  }
  // Sums x with the denominator and reference of their own; minus infinity: nothing.
  __device__ __forceinline__ void add(float mx, float lx, const float (&x)[E]) {
    const float top = fmaxf(m, mx), ref = top == -INFINITY ? 0.f : top, al = exp2f(m - ref), p = exp2f(mx - ref);
    m = top;
    l = l * al + p * lx;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = fmaf(p, x[e], acc[e] * al);
  }
};
// A row's latents (16 bytes a lane and run) and key (d_R / 32 elements a lane).
template <typename T>
__device__ __forceinline__ void load_row(const T* src, const qp::Format& f, float (&x)[Running<T>::E], float (&k)[2]) {
  constexpr int V = Running<T>::V, R = Running<T>::R;
  const int lane = threadIdx.x & 31, kd = f.dr / 32;
#pragma unroll
  for (int j = 0; j < R; ++j) {
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = 0.f;
    if ((j * 32 + lane) * V < f.r) load_vec(src + (j * 32 + lane) * V, v);
#pragma unroll
    for (int e = 0; e < V; ++e) x[j * V + e] = v[e];
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) k[e] = e < kd ? Elem<T>::to_float(src[f.r + lane * kd + e]) : 0.f;
}
template <typename T>
__device__ __forceinline__ void load_part(const float* src, int r, float (&x)[Running<T>::E]) {
  constexpr int V = Running<T>::V, R = Running<T>::R;
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int j = 0; j < R; ++j)
#pragma unroll
    for (int e = 0; e < V; e += 4) {
      float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
      if ((j * 32 + lane) * V < r) w = *reinterpret_cast<const float4*>(src + (j * 32 + lane) * V + e);
      x[j * V + e] = w.x;
      x[j * V + e + 1] = w.y;
      x[j * V + e + 2] = w.z;
      x[j * V + e + 3] = w.w;
    }
}
template <typename T>
__device__ __forceinline__ float dot_row(const float (&q)[Running<T>::E], const float (&qk)[2],
                                         const float (&x)[Running<T>::E], const float (&k)[2]) {
  float s = qk[0] * k[0] + qk[1] * k[1];
#pragma unroll
  for (int e = 0; e < Running<T>::E; ++e) s = fmaf(q[e], x[e], s);
  return warp_sum(s);
}

// Where a node stands: its request's first node, the drafted rows that it sees, and its columns' groups.
struct Place {
  bool fine;                 // in a request (or the batch is refused: nothing is seen)
  int lo, first_group;
  unsigned long long seen;
};
__device__ __forceinline__ Place place_of(const JoinArgs& a, int node, bool refused) {
  Place p = {true, 0, 0, 0};
  if (refused) return p;
  const unsigned long long seen = (unsigned long long)a.seen[node];
  const int b = qp::find_wide(a.starts, a.batch, node), hi = a.starts[b + 1];
  p.lo = a.starts[b];
  p.first_group = a.first[b];
  p.fine = node >= p.lo;                               // else in front of the first request
  p.seen = hi - p.lo < kMaxNodes ? seen & ((1ull << (hi - p.lo)) - 1) : seen;
  return p;
}
// The parts of a column: x first, y number; z the column inside its group.
__device__ __forceinline__ int3 parts_of(const JoinArgs& a, const Place& p, int node, int h, bool refused) {
  if (refused) return make_int3(0, 0, 0);
  const int local = (node - p.lo) * a.heads + h, v = p.first_group + local / a.cols;
  const int2 parts = a.parts[v];                       // (not set for a group without tiles)
  return make_int3(parts.x, a.groups[v].w > 0 ? parts.y : 0, local % a.cols);
}
template <typename T>
__device__ __forceinline__ void store_column(const JoinArgs& a, long long column, float m, float l, bool failed,
                                             const float (&acc)[Running<T>::E]) {
  constexpr int V = Running<T>::V, R = Running<T>::R;
  const int lane = threadIdx.x & 31;
  // A node that sees nothing: zeros and minus infinity.
  const float inv = failed ? NAN : l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int j = 0; j < R; ++j) {
    if ((j * 32 + lane) * V >= a.f.r) continue;
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = acc[j * V + e] * inv;
    store_vec(static_cast<T*>(a.out) + column * a.f.r + (j * 32 + lane) * V, v);
  }
  if (a.lse && lane == 0) a.lse[column] = failed ? NAN : l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

// The join: the online softmax over the drafted rows that a node sees, row after row, and the parts that the attention
// over the context has left for its columns.  Masked rows are never read, so what they hold cannot reach a
// result; sums, maxima and products are fp32.  Bound by the parts' bytes when there are many columns, else by the chain
// of loads.  Two forms:
//   a warp per node and two heads, which share the rows' loads, for many columns;
//   with SPLIT a CTA per column, whose warps share rows and parts out, for few: one request of 112 columns in 74 parts
//   each took 53 us with a warp per column.
constexpr int kJoinThreads = 128, kJoinWarps = kJoinThreads / 32, kSplitThreads = 256, kSplitWarps = kSplitThreads / 32;

template <typename T>
__global__ void __launch_bounds__(kJoinThreads) tree_join_kernel(JoinArgs a) {
  using Run = Running<T>;
  constexpr int E = Run::E, HB = 2;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = a.f.r, blocks = ceil_div(a.heads, HB);
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  bool failed = false;
  for (int i = threadIdx.x; i < a.n_error_words; i += kJoinThreads) failed |= a.error_words[i] != 0;
  const bool refused = *a.n_groups < 0;
  failed = __syncthreads_or(failed) || refused;
  // Nodes behind the last request are left as they were; those of a refused batch all get NaN.
  const long long units = (long long)(refused ? a.n_nodes : a.starts[a.batch]) * blocks;
  for (long long u = (long long)blockIdx.x * kJoinWarps + warp; u < units; u += (long long)gridDim.x * kJoinWarps) {
    const int node = (int)(u / blocks), h0 = (int)(u % blocks) * HB;
    const bool two = h0 + 1 < a.heads;
    float q[HB][E], qk[HB][2];
#pragma unroll
    for (int h = 0; h < HB; ++h)
      load_row<T>(static_cast<const T*>(a.q) + ((long long)node * a.heads + h0 + (two ? h : 0)) * (r + a.f.dr), a.f, q[h],
                  qk[h]);
    Place p = place_of(a, node, refused);
    if (!p.fine) continue;
    int3 parts[HB];
#pragma unroll
    for (int h = 0; h < HB; ++h) parts[h] = parts_of(a, p, node, h0 + (two ? h : 0), refused);
    Run run[HB];
#pragma unroll
    for (int h = 0; h < HB; ++h) run[h].clear();
    while (p.seen) {
      const int at = __ffsll((long long)p.seen) - 1;
      p.seen &= p.seen - 1;
      float x[E], k[2];
      load_row<T>(static_cast<const T*>(a.rows) + (p.lo + at) * a.row_stride, a.f, x, k);
#pragma unroll
      for (int h = 0; h < HB; ++h) run[h].add(dot_row<T>(q[h], qk[h], x, k) * a.scale_log2, 1.f, x);
    }
    // Both heads' parts together, as long as either has one.
    const int most = max(parts[0].y, parts[1].y);
    for (int n = 0; n < most; ++n) {
      float2 ml[HB];
      float x[HB][E];
#pragma unroll
      for (int h = 0; h < HB; ++h) {
        const long long at = (long long)(parts[h].x + min(n, max(parts[h].y, 1) - 1)) * a.cols + parts[h].z;
        ml[h] = make_float2(-INFINITY, 0.f);
        if (n < parts[h].y) {
          ml[h] = reinterpret_cast<const float2*>(a.ml_part)[at];
          load_part<T>(a.o_part + at * r, r, x[h]);
        }
      }
#pragma unroll
      for (int h = 0; h < HB; ++h)
        if (n < parts[h].y) run[h].add(ml[h].x, ml[h].y, x[h]);
    }
#pragma unroll
    for (int h = 0; h < HB; ++h)
      if (h == 0 || two)
        store_column<T>(a, (long long)node * a.heads + h0 + h, run[h].m, run[h].l, failed, run[h].acc);
  }
}

template <typename T>
__global__ void __launch_bounds__(kSplitThreads) tree_join_split_kernel(JoinArgs a) {
  using Run = Running<T>;
  constexpr int E = Run::E;
  __shared__ float s_m[kSplitWarps], s_l[kSplitWarps];
  __shared__ float4 s_acc[kSplitWarps][E / 4][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = a.f.r;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  bool failed = false;
  for (int i = threadIdx.x; i < a.n_error_words; i += kSplitThreads) failed |= a.error_words[i] != 0;
  const bool refused = *a.n_groups < 0;
  failed = __syncthreads_or(failed) || refused;
  const long long columns = (long long)(refused ? a.n_nodes : a.starts[a.batch]) * a.heads;
  for (long long column = blockIdx.x; column < columns; column += gridDim.x) {
    const int node = (int)(column / a.heads), h = (int)(column % a.heads);
    const Place p = place_of(a, node, refused);
    if (!p.fine) continue;
    const int3 parts = parts_of(a, p, node, h, refused);
    Run run;
    run.clear();
    // Rows in turn: the warp's are the set bits number warp, warp + 8, ...
    if (__popcll(p.seen) > warp) {
      float q[E], qk[2];
      load_row<T>(static_cast<const T*>(a.q) + column * (r + a.f.dr), a.f, q, qk);
      unsigned long long seen = p.seen;
      for (int n = 0; seen; ++n) {
        const int at = __ffsll((long long)seen) - 1;
        seen &= seen - 1;
        if (n % kSplitWarps != warp) continue;
        float x[E], k[2];
        load_row<T>(static_cast<const T*>(a.rows) + (p.lo + at) * a.row_stride, a.f, x, k);
        run.add(dot_row<T>(q, qk, x, k) * a.scale_log2, 1.f, x);
      }
    }
    constexpr int U = 4;                                 // parts whose loads are in flight together
    for (int n0 = warp; n0 < parts.y; n0 += U * kSplitWarps) {
      float2 ml[U];
      float x[U][E];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int n = n0 + i * kSplitWarps;
        ml[i] = make_float2(-INFINITY, 0.f);
        if (n >= parts.y) continue;
        const long long at = (long long)(parts.x + n) * a.cols + parts.z;
        ml[i] = reinterpret_cast<const float2*>(a.ml_part)[at];
        load_part<T>(a.o_part + at * r, r, x[i]);
      }
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (n0 + i * kSplitWarps < parts.y) run.add(ml[i].x, ml[i].y, x[i]);
    }
    if (lane == 0) {
      s_m[warp] = run.m;
      s_l[warp] = run.l;
    }
#pragma unroll
    for (int e = 0; e < E; e += 4)
      s_acc[warp][e / 4][lane] = make_float4(run.acc[e], run.acc[e + 1], run.acc[e + 2], run.acc[e + 3]);
    __syncthreads();
    if (warp == 0) {
#pragma unroll 1
      for (int w = 1; w < kSplitWarps; ++w) {            // in the warps' order
        float x[E];
#pragma unroll
        for (int e = 0; e < E; e += 4) {
          const float4 v = s_acc[w][e / 4][lane];
          x[e] = v.x;
          x[e + 1] = v.y;
          x[e + 2] = v.z;
          x[e + 3] = v.w;
        }
        run.add(s_m[w], s_l[w], x);
      }
      store_column<T>(a, column, run.m, run.l, failed, run.acc);
    }
    __syncthreads();
  }
}

}  // namespace tree
}  // namespace mtla
