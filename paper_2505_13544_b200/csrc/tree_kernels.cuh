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

constexpr int kPlanThreads = 1024;
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
// others (of bf16 queries) write the groups' images, a group each in turn.  A batch whose `starts` do not ascend inside
// the nodes gets no groups and a count of -1.  As a part of the attention, each CTA writing the image of its next
// group itself when the last one's products are done, the images took 13000 cycles of every change between groups.
__global__ void __launch_bounds__(kPlanThreads) tree_plan_kernel(PlanArgs a) {
  __shared__ int s_first[kMaxRequests + 1], s_tile[kMaxRequests + 1];
  __shared__ int warp_g[32], warp_t[32];
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
  for (int v = blockIdx.x - 1; v < total; v += gridDim.x - 1) {
    int b = 0, end = a.batch;                          // the request: the last one that begins at v or before it
    while (end - b > 1) {
      const int mid = (b + end) >> 1;
      if (s_first[mid] <= v) b = mid; else end = mid;
    }
    const int skip = (v - s_first[b]) * a.cols, col0 = a.starts[b] * a.heads + skip;
    const int cols = a.starts[b + 1] * a.heads - col0;
    for (int c = warp; c < a.cols; c += kPlanThreads / 32)
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

constexpr int kJoinThreads = 128, kJoinWarps = kJoinThreads / 32;

// A warp per node and HB of its heads: the online softmax over the drafted rows that the node sees, row after row
// (a lane keeps 16 of the 512 latents of every head, a row is loaded once for all of them), and then
// the parts that the attention over the context has left for its columns.  Masked rows are never read, so what
// they hold cannot reach a result; sums, maxima and products are fp32.
// A row's latents are loaded 16 bytes a lane, V elements, in R rounds; its key as d_R / 32 elements a lane.
template <typename T, int HB>
__global__ void __launch_bounds__(kJoinThreads) tree_join_kernel(JoinArgs a) {
  constexpr int V = Elem<T>::kVec, R = 512 / (32 * V), E = R * V;
  __shared__ int s_failed;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = a.f.r, dr = a.f.dr, kd = dr / 32;
  const int blocks = ceil_div(a.heads, HB);
  if (threadIdx.x == 0) s_failed = 0;
  __syncthreads();
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  for (int i = threadIdx.x; i < a.n_error_words; i += kJoinThreads)
    if (a.error_words[i]) s_failed = 1;
  __syncthreads();
  const bool refused = *a.n_groups < 0, failed = s_failed != 0 || refused;
  // Nodes behind the last request are left as they were; those of a refused batch all get NaN.
  const long long units = (long long)(refused ? a.n_nodes : a.starts[a.batch]) * blocks;
  for (long long u = (long long)blockIdx.x * kJoinWarps + warp; u < units; u += (long long)gridDim.x * kJoinWarps) {
    const int node = (int)(u / blocks), h0 = (int)(u % blocks) * HB;
    const int b = refused ? 0 : qp::find_wide(a.starts, a.batch, node);
    const int lo = refused ? 0 : a.starts[b], hi = refused ? 0 : a.starts[b + 1];
    if (node < lo) continue;                              // in front of the first request
    unsigned long long seen = refused ? 0 : (unsigned long long)a.seen[node];
    if (hi - lo < kMaxNodes) seen &= (1ull << (hi - lo)) - 1;
    float q[HB][E], qk[HB][2], acc[HB][E], m[HB], l[HB];
#pragma unroll
    for (int h = 0; h < HB; ++h) {
      const bool there = h0 + h < a.heads;
      const T* src = static_cast<const T*>(a.q) + ((long long)node * a.heads + h0 + (there ? h : 0)) * (r + dr);
#pragma unroll
      for (int j = 0; j < R; ++j) {
        float v[V];
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = 0.f;
        if ((j * 32 + lane) * V < r) load_vec(src + (j * 32 + lane) * V, v);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          q[h][j * V + e] = v[e];
          acc[h][j * V + e] = 0.f;
        }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) qk[h][e] = e < kd ? Elem<T>::to_float(src[r + lane * kd + e]) : 0.f;
      m[h] = -INFINITY;
      l[h] = 0.f;
    }
    while (seen) {
      const int at = __ffsll((long long)seen) - 1;
      seen &= seen - 1;
      const T* src = static_cast<const T*>(a.rows) + (lo + at) * a.row_stride;
      float c[E], ck[2];
#pragma unroll
      for (int j = 0; j < R; ++j) {
        float v[V];
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = 0.f;
        if ((j * 32 + lane) * V < r) load_vec(src + (j * 32 + lane) * V, v);
#pragma unroll
        for (int e = 0; e < V; ++e) c[j * V + e] = v[e];
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) ck[e] = e < kd ? Elem<T>::to_float(src[r + lane * kd + e]) : 0.f;
#pragma unroll
      for (int h = 0; h < HB; ++h) {
        float s = qk[h][0] * ck[0] + qk[h][1] * ck[1];
#pragma unroll
        for (int e = 0; e < E; ++e) s = fmaf(q[h][e], c[e], s);
        s = warp_sum(s) * a.scale_log2;
        const float top = fmaxf(m[h], s), ref = top == -INFINITY ? 0.f : top;
        const float al = exp2f(m[h] - ref), p = exp2f(s - ref);
        m[h] = top;
        l[h] = l[h] * al + p;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[h][e] = fmaf(p, c[e], acc[h][e] * al);
      }
    }
#pragma unroll
    for (int h = 0; h < HB; ++h) {
      if (h0 + h >= a.heads) break;
      int2 parts = make_int2(0, 0);
      int col = 0;
      if (!refused) {
        const int local = (node - lo) * a.heads + h0 + h;      // column of the request
        const int v = a.first[b] + local / a.cols;
        col = local % a.cols;
        if (a.groups[v].w > 0) parts = a.parts[v];
      }
      constexpr int U = 4;                              // parts whose loads are in flight together
      for (int p0 = 0; p0 < parts.y; p0 += U) {
        float2 ml[U];
        float x[U][E];
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const long long at = (long long)(parts.x + min(p0 + i, parts.y - 1)) * a.cols + col;
          ml[i] = reinterpret_cast<const float2*>(a.ml_part)[at];
#pragma unroll
          for (int j = 0; j < R; ++j)
#pragma unroll
            for (int e = 0; e < V; e += 4) {
              float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
              if ((j * 32 + lane) * V < r)
                w = *reinterpret_cast<const float4*>(a.o_part + at * r + (j * 32 + lane) * V + e);
              x[i][j * V + e] = w.x;
              x[i][j * V + e + 1] = w.y;
              x[i][j * V + e + 2] = w.z;
              x[i][j * V + e + 3] = w.w;
            }
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
          if (p0 + i >= parts.y) break;
          const float top = fmaxf(m[h], ml[i].x), ref = top == -INFINITY ? 0.f : top;
          const float al = exp2f(m[h] - ref), p = exp2f(ml[i].x - ref);
          m[h] = top;
          l[h] = l[h] * al + p * ml[i].y;
#pragma unroll
          for (int e = 0; e < E; ++e) acc[h][e] = fmaf(p, x[i][e], acc[h][e] * al);
        }
      }
      // A node that sees nothing: zeros and minus infinity.
      const float inv = failed ? NAN : l[h] == 0.f ? 0.f : 1.f / l[h];
      const long long column = (long long)node * a.heads + h0 + h;
#pragma unroll
      for (int j = 0; j < R; ++j) {
        if ((j * 32 + lane) * V >= r) continue;
        float v8[V];
#pragma unroll
        for (int e = 0; e < V; ++e) v8[e] = acc[h][j * V + e] * inv;
        store_vec(static_cast<T*>(a.out) + column * r + (j * 32 + lane) * V, v8);
      }
      if (a.lse && lane == 0)
        a.lse[column] = failed ? NAN : l[h] == 0.f ? -INFINITY : (m[h] + log2f(l[h])) * 0.69314718055994531f;
    }
  }
}

}  // namespace tree
}  // namespace mtla
