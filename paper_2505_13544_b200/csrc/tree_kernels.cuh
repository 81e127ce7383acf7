// Drafted trees over the 4-bit pool: positions and masks of the nodes, the list of column groups that the
// attention over the context works through, and the kernel that adds the drafted rows and joins everything.
//
// A request's columns are its nodes times the heads; a column is a query row [r + d_R] and an output row [r],
// both at index column of the flat tensors.  All nodes of a request see the same context slots (a path continues
// the open slot, so only closed ones are left, and those are common), which makes the context's part the attention
// of `columns` queries over one list of pages without any mask.  Groups of up to 64 columns take the place that
// sequences have in qpool_attn.cuh.
#pragma once

#include "qpool_attn.cuh"
#include "qweight_format.cuh"

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
  int2* listed;              // groups (-1: the batch is refused), their tiles
  int4* shares;              // [ctas]: first tile, tiles, the first one's group, the CTA that begins that group
  const bf16* q;             // [n_nodes][heads][r + d_R]
  uint8_t* image;            // [groups] of image_bytes, or nullptr
  float scale_log2;
  int batch, n_nodes, heads, width, cols, tile_pages, ctas;
  qp::Format f;
};

constexpr int kPlanThreads = 512;
constexpr int kMaxRequests = 4096;

// A group's queries for the tensor-core kernel, as they lie in its shared memory: r / 64 panels [cols][64] half
// precision with the 128-byte swizzle, one panel [cols][d_R] bf16 (128- or 64-byte swizzle), and what a column's scores
// are to be multiplied by.
__host__ __device__ inline int image_bytes(int cols, const qp::Format& f) { return cols * (2 * (f.r + f.dr) + 4); }

// Columns col, col + step, ... (N of them, whose loads are issued together) into their group's image, by a warp; `q`
// is the group's first column.  A row is scaled by the power of two that brings its largest element into [2^14, 2^15),
// exactly down to 2^-39 of that; a column that does not exist is zero.  Magnitudes and scaling work on pairs of bf16
// numbers (a power of two in two factors, since one may be out of range).
template <int N>
__device__ __forceinline__ void put_columns(const bf16* q, int there, uint8_t* image, int col0, int step, int cols,
                                            float scale_log2, const qp::Format& f) {
  const int lane = threadIdx.x & 31, r = f.r, dr = f.dr;
  uint4 w[N][2], key[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int col = col0 + n * step;
    const bf16* src = q + (long long)col * (r + dr);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      w[n][i] = make_uint4(0u, 0u, 0u, 0u);
      if (col < there && (lane + 32 * i) * 8 < r) w[n][i] = *reinterpret_cast<const uint4*>(src + (lane + 32 * i) * 8);
    }
    key[n] = make_uint4(0u, 0u, 0u, 0u);
    if (col < there && lane * 8 < dr) key[n] = *reinterpret_cast<const uint4*>(src + r + lane * 8);
  }
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int col = col0 + n * step;
    uint32_t top = 0;
    auto largest = [&](const uint4& v) {
      const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int m = 0; m < 4; ++m) top = __vmaxu2(top, x[m] & 0x7fff7fffu);
    };
    largest(w[n][0]);
    largest(w[n][1]);
    largest(key[n]);
    top = __reduce_max_sync(0xffffffffu, max(top & 0xffffu, top >> 16));
    // Exponents -113 .. 140 (a row of subnormal numbers only reaches less); none for zeros and specials.
    const bool fine = top > 0 && top < 0x7f80u;
    const int e = fine ? 141 - max((int)(top >> 7), 1) : 0, e1 = e / 2, e2 = e - e1;
    const uint32_t f1 = (uint32_t)(127 + e1) * 0x00800080u, f2 = (uint32_t)(127 + e2) * 0x00800080u;
    if (lane == 0)
      reinterpret_cast<float*>(image + (long long)cols * 2 * (r + dr))[col] =
          scale_log2 * __uint_as_float((127 - e1) << 23) * __uint_as_float((127 - e2) << 23);
    auto scaled = [&](uint32_t x) { return qw::mul_b2(qw::mul_b2(x, f1), f2); };
    auto half2_of = [&](uint32_t x) {
      const uint32_t y = scaled(x);
      const __half2 h = __floats2half2_rn(__uint_as_float(y << 16), __uint_as_float(y & 0xffff0000u));
      return *reinterpret_cast<const uint32_t*>(&h);
    };
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int c = lane + 32 * i;
      if (c * 8 < r)
        *reinterpret_cast<uint4*>(image + (c >> 3) * cols * 128 + col * 128 + ((c ^ col) & 7) * 16) =
            make_uint4(half2_of(w[n][i].x), half2_of(w[n][i].y), half2_of(w[n][i].z), half2_of(w[n][i].w));
    }
    if (lane * 8 < dr)
      *reinterpret_cast<uint4*>(image + cols * 2 * r + col * 2 * dr + (lane ^ f.key_swizzle(col)) * 16) =
          make_uint4(scaled(key[n].x), scaled(key[n].y), scaled(key[n].z), scaled(key[n].w));
  }
}

// Two prefix sums over the requests (groups, tiles) in every CTA; the first enters the list, a warp per request, the
// others (of bf16 queries) write the groups' images, half a group each in turn.  A batch whose `starts` do not ascend inside
// the nodes gets no groups and a count of -1.  As a part of the attention, each CTA writing the image of its next
// group itself when the last one's products are done, the images took 13000 cycles of every change between groups.
__global__ void __launch_bounds__(kPlanThreads, 2) tree_plan_kernel(PlanArgs a) {
  __shared__ int s_first[kMaxRequests + 1], s_tile[kMaxRequests + 1];
  __shared__ int warp_g[kPlanThreads / 32], warp_t[kPlanThreads / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  auto tiles_of = [&](int slots) {
    const int n = max(slots, 0);
    const int pages = min(n / qp::kPageRows + (n % qp::kPageRows != 0), a.width);
    return (pages + a.tile_pages - 1) / a.tile_pages;
  };
  const int per = ceil_div(a.batch, kPlanThreads), lo = min(a.batch, tid * per), hi = min(a.batch, lo + per);
  bool wrong = a.starts[0] < 0;
  // (Lengths that the host has found to fit 32 bits only if the batch is in order.)
  int sum_g = 0, sum_t = 0;
  for (int b = lo; b < hi; ++b) {
    const int begin = a.starts[b], end = a.starts[b + 1], tiles = tiles_of(a.slots[b]);
    wrong |= begin > end || end > a.n_nodes || begin < 0;
    const int g = wrong ? 0 : ceil_div((end - begin) * a.heads, a.cols);
    s_first[b] = sum_g;
    s_tile[b] = sum_t;
    sum_g += g;
    sum_t += g * tiles;
  }
  if (__syncthreads_or(wrong)) {
    if (blockIdx.x == 0) {
      if (tid == 0) *a.listed = make_int2(-1, 0);
      for (int c = tid; c < a.ctas; c += kPlanThreads) a.shares[c] = make_int4(0, 0, 0, 0);
    }
    return;
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
    // The shares of the tensor-core kernel's CTAs: found here once, they need not be found there by everyone before the
    // first page is asked for (2600 cycles of a CTA's start).
    const int all = s_tile[a.batch], ctas = min(a.ctas, all);
    for (int c = tid; c < a.ctas; c += kPlanThreads) {
      int4 share = make_int4(0, 0, 0, 0);
      if (c < ctas) {
        share.x = qp::share_begin(c, all, ctas);
        share.y = qp::share_begin(c + 1, all, ctas) - share.x;
        int b = 0, end = a.batch;                        // the last request that begins at this tile or before it
        while (end - b > 1) {
          const int mid = (b + end) >> 1;
          if (s_tile[mid] <= share.x) b = mid; else end = mid;
        }
        const int tiles = tiles_of(a.slots[b]), i = (share.x - s_tile[b]) / tiles;
        share.z = s_first[b] + i;
        share.w = qp::share_owner(s_tile[b] + i * tiles, all, ctas);
      }
      a.shares[c] = share;
    }
    for (int b = tid; b <= a.batch; b += kPlanThreads) a.first[b] = s_first[b];
    for (int b = warp; b < a.batch; b += kPlanThreads / 32) {
      const int col0 = a.starts[b] * a.heads, cols = a.starts[b + 1] * a.heads - col0, n_slots = a.slots[b];
      const int tiles = tiles_of(n_slots), slots = min(max(n_slots, 0), (int)min((long long)a.width * qp::kPageRows, 0x7fffffffll));
      const int g0 = s_first[b], n = s_first[b + 1] - g0;
      for (int i = lane; i < n; i += 32) {
        a.groups[g0 + i] = make_int4(b, col0 + i * a.cols, min(a.cols, cols - i * a.cols), slots);
        a.prefix[g0 + i] = s_tile[b] + i * tiles;
      }
    }
    if (tid == 0) {
      *a.listed = make_int2(total, s_tile[a.batch]);
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
    const bf16* q = a.q + (long long)col0 * (a.f.r + a.f.dr);
    uint8_t* image = a.image + (long long)v * image_bytes(a.cols, a.f);
    // Half a group: two columns a warp of 64, one of 32.
    constexpr int kWarps = kPlanThreads / 32;
    static_assert(kWarps == 16, "half a group is one or two columns of every warp");
    if (a.cols == 64)
      put_columns<2>(q, cols, image, (u & 1) * half + warp, kWarps, a.cols, a.scale_log2, a.f);
    else
      put_columns<1>(q, cols, image, (u & 1) * half + warp, kWarps, a.cols, a.scale_log2, a.f);
  }
}

// ---- drafted rows and the join

struct JoinArgs {
  const void* q;             // [n_nodes][heads][r + d_R]
  const void* rows;          // [n_nodes][r + d_R], row_stride elements apart
  const long long* seen;     // [n_nodes]
  const int* starts;
  const int4* groups;
  const int* first;
  const int2* listed;
  const int2* parts;         // [groups] first part, number of parts; not to be read once an error word is set
  const float* o_part;       // [parts][cols][part_row], r of each row used
  const float* ml_part;      // [parts][cols][2]
  const int* error_words;
  void* out;
  float* lse;
  long long row_stride;
  float scale_log2;
  int batch, n_nodes, heads, cols, part_row, n_error_words;
  qp::Format f;
};

// What has been joined of one column: reference (log2 units), denominator, sums; a lane holds E latents, in pairs.
template <typename T>
struct Running {
  static constexpr int V = Elem<T>::kVec, R = 512 / (32 * V), E = R * V;       // runs of 16 bytes of a row
  float m, l;
  uint64_t acc[E / 2];
  __device__ __forceinline__ void clear() {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int e = 0; e < E / 2; ++e) acc[e] = 0;
  }
  // Sums x with the denominator and reference of their own; minus infinity: nothing.
  __device__ __forceinline__ void add(float mx, float lx, const uint64_t (&x)[E / 2]) {
    const float top = fmaxf(m, mx), ref = top == -INFINITY ? 0.f : top, p = exp2f(mx - ref);
    if (top != m) {
      const float al = exp2f(m - ref);
      l *= al;
      const uint64_t al2 = ptx::pack2(al, al);
#pragma unroll
      for (int e = 0; e < E / 2; ++e) acc[e] = ptx::mul2(acc[e], al2);
      m = top;
    }
    l += p * lx;
    const uint64_t p2 = ptx::pack2(p, p);
#pragma unroll
    for (int e = 0; e < E / 2; ++e) acc[e] = ptx::fma2(p2, x[e], acc[e]);
  }
};
// A row's latents (16 bytes a lane and run) and key (d_R / 32 elements a lane).
template <typename T>
__device__ __forceinline__ void load_row(const T* src, const qp::Format& f, uint64_t (&x)[Running<T>::E / 2],
                                         float (&k)[2]) {
  constexpr int V = Running<T>::V, R = Running<T>::R;
  const int lane = threadIdx.x & 31, kd = f.dr / 32;
#pragma unroll
  for (int j = 0; j < R; ++j) {
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = 0.f;
    if ((j * 32 + lane) * V < f.r) load_vec(src + (j * 32 + lane) * V, v);
#pragma unroll
    for (int e = 0; e < V; e += 2) x[(j * V + e) / 2] = ptx::pack2(v[e], v[e + 1]);
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) k[e] = e < kd ? Elem<T>::to_float(src[f.r + lane * kd + e]) : 0.f;
}
template <typename T>
__device__ __forceinline__ void load_part(const float* src, int r, uint64_t (&x)[Running<T>::E / 2]) {
  constexpr int V = Running<T>::V, R = Running<T>::R;
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int j = 0; j < R; ++j)
#pragma unroll
    for (int e = 0; e < V; e += 4) {
      ulonglong2 w = make_ulonglong2(0ull, 0ull);
      if ((j * 32 + lane) * V < r) w = *reinterpret_cast<const ulonglong2*>(src + (j * 32 + lane) * V + e);
      x[(j * V + e) / 2] = w.x;
      x[(j * V + e) / 2 + 1] = w.y;
    }
}
// A lane's share of the product of a query and a drafted row.
template <typename T>
__device__ __forceinline__ float dot_share(const uint64_t (&q)[Running<T>::E / 2], const float (&qk)[2],
                                           const uint64_t (&x)[Running<T>::E / 2], const float (&k)[2]) {
  uint64_t s = ptx::pack2(qk[0] * k[0], qk[1] * k[1]);
#pragma unroll
  for (int e = 0; e < Running<T>::E / 2; ++e) s = ptx::fma2(q[e], x[e], s);
  float lo, hi;
  ptx::unpack2(s, lo, hi);
  return lo + hi;
}

// Where a node stands: its request's first node, the drafted rows that it sees, and its columns' groups.
struct Place {
  bool fine;                 // in a request (or the batch is refused: nothing is seen)
  int lo, first_group;
  unsigned long long seen;
};
// (Columns fit 31 bits, and a group has a power of two of them.)
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
// The parts of a column: x first, y number; z the column inside its group.  None after a failure: a group's entry is
// written by the CTA that ends the group, so where that one has given up it holds whatever the workspace held.
__device__ __forceinline__ int3 parts_of(const JoinArgs& a, const Place& p, int node, int h, bool refused, bool failed) {
  if (refused) return make_int3(0, 0, 0);
  const int local = (node - p.lo) * a.heads + h, v = p.first_group + (local >> (31 - __clz(a.cols)));
  const int2 parts = a.parts[v];                       // (not set for a group without tiles)
  return make_int3(parts.x, !failed && a.groups[v].w > 0 ? parts.y : 0, local & (a.cols - 1));
}
template <typename T>
__device__ __forceinline__ void store_column(const JoinArgs& a, long long column, float m, float l, bool failed,
                                             const uint64_t (&acc)[Running<T>::E / 2]) {
  constexpr int V = Running<T>::V, R = Running<T>::R;
  const int lane = threadIdx.x & 31;
  // A node that sees nothing: zeros and minus infinity.
  const float inv = failed ? NAN : l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int j = 0; j < R; ++j) {
    if ((j * 32 + lane) * V >= a.f.r) continue;
    float v[V];
#pragma unroll
    for (int e = 0; e < V; e += 2) {
      ptx::unpack2(acc[(j * V + e) / 2], v[e], v[e + 1]);
      v[e] *= inv;
      v[e + 1] *= inv;
    }
    store_vec(static_cast<T*>(a.out) + column * a.f.r + (j * 32 + lane) * V, v);
  }
  if (a.lse && lane == 0) a.lse[column] = failed ? NAN : l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

// Pair number e of this lane's.
template <typename T>
__device__ __forceinline__ void store_pair(const JoinArgs& a, long long column, int e, float m, float l, bool failed,
                                           uint64_t sum) {
  constexpr int V = Running<T>::V;
  const int lane = threadIdx.x & 31, at = (2 * e / V * 32 + lane) * V + 2 * e % V;
  const float inv = failed ? NAN : l == 0.f ? 0.f : 1.f / l;
  if (at < a.f.r) {
    float x, y;
    ptx::unpack2(sum, x, y);
    T* out = static_cast<T*>(a.out) + column * a.f.r + at;
    if constexpr (sizeof(T) == 2)
      *reinterpret_cast<__nv_bfloat162*>(out) = __floats2bfloat162_rn(x * inv, y * inv);
    else
      *reinterpret_cast<float2*>(out) = make_float2(x * inv, y * inv);
  }
  if (a.lse && lane == 0 && e == 0)
    a.lse[column] = failed ? NAN : l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

// The join: the softmax over the drafted rows that a node sees, and the parts that the attention over the context has
// left for its columns; sums, maxima and products are fp32.  Bound by the parts' bytes when there are many columns,
// else by the chain of loads.  Three forms:
//   tree_join_split_kernel   a CTA per column, whose W warps share rows and parts out, for few columns (112 columns in 74
//                            parts each: 53 us with a warp per column, 14 so);
//   tree_join_kernel         a warp per column, row after row;
//   tree_join_dense_kernel   a CTA per group of 64 columns, all its drafted rows by matrix products, for bf16 with a group
//                            for every SM (16384 columns that see 6 of 64 rows each: 45 us with a warp per column, 36 so;
//                            52 groups: 14 us and 25).
// In the first two masked rows are never read, so what they hold cannot reach a result.
constexpr int kJoinThreads = 128, kJoinWarps = kJoinThreads / 32;

template <typename T>
__global__ void __launch_bounds__(kJoinThreads, 5) tree_join_kernel(JoinArgs a) {
  using Run = Running<T>;
  constexpr int E = Run::E;
  const int warp = threadIdx.x >> 5, r = a.f.r;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  bool failed = false;
  for (int i = threadIdx.x; i < a.n_error_words; i += kJoinThreads) failed |= a.error_words[i] != 0;
  const bool refused = a.listed->x < 0;
  failed = __syncthreads_or(failed) || refused;
  // Nodes behind the last request are left as they were; those of a refused batch all get NaN.
  const uint32_t columns = (uint32_t)(refused ? a.n_nodes : a.starts[a.batch]) * a.heads;
  for (uint32_t column = blockIdx.x * kJoinWarps + warp; column < columns; column += gridDim.x * kJoinWarps) {
    const int node = (int)(column / (uint32_t)a.heads), h = (int)(column - (uint32_t)node * a.heads);
    uint64_t q[E / 2];
    float qk[2];
    load_row<T>(static_cast<const T*>(a.q) + (long long)column * (r + a.f.dr), a.f, q, qk);
    Place p = place_of(a, node, refused);
    if (!p.fine) continue;
    const int3 parts = parts_of(a, p, node, h, refused, failed);
    float2 ml;
    uint64_t y[E / 2];
    auto load_one = [&](int n) {
      if (n >= parts.y) return;
      const long long at = (long long)(parts.x + n) * a.cols + parts.z;
      ml = reinterpret_cast<const float2*>(a.ml_part)[at];
      load_part<T>(a.o_part + at * a.part_row, r, y);
    };
    load_one(0);
    Run run;
    run.clear();
    const T* rows = static_cast<const T*>(a.rows) + p.lo * a.row_stride;
    while (p.seen) {
      const int at = __ffsll((long long)p.seen) - 1;
      p.seen &= p.seen - 1;
      uint64_t x[E / 2];
      float k[2];
      load_row<T>(rows + at * a.row_stride, a.f, x, k);
      run.add(warp_sum(dot_share<T>(q, qk, x, k)) * a.scale_log2, 1.f, x);
    }
    for (int n = 0; n < parts.y; ++n) {
      run.add(ml.x, ml.y, y);
      load_one(n + 1);
    }
    store_column<T>(a, column, run.m, run.l, failed, run.acc);
  }
}

template <typename T, int W>
__global__ void __launch_bounds__(32 * W, 16 / W) tree_join_split_kernel(JoinArgs a) {
  using Run = Running<T>;
  constexpr int E = Run::E;
  __shared__ float s_m[W], s_l[W];
  __shared__ uint64_t s_acc[W][E / 2][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = a.f.r;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  bool failed = false;
  for (int i = threadIdx.x; i < a.n_error_words; i += 32 * W) failed |= a.error_words[i] != 0;
  const bool refused = a.listed->x < 0;
  failed = __syncthreads_or(failed) || refused;
  const uint32_t columns = (uint32_t)(refused ? a.n_nodes : a.starts[a.batch]) * a.heads;
  for (uint32_t column = blockIdx.x; column < columns; column += gridDim.x) {
    const int node = (int)(column / (uint32_t)a.heads), h = (int)(column - (uint32_t)node * a.heads);
    const Place p = place_of(a, node, refused);
    if (!p.fine) continue;
    const int3 parts = parts_of(a, p, node, h, refused, failed);
    Run run;
    run.clear();
    // Rows in turn: the warp's are the set bits number warp, warp + W, ...
    if (__popcll(p.seen) > warp) {
      uint64_t q[E / 2];
      float qk[2];
      load_row<T>(static_cast<const T*>(a.q) + (long long)column * (r + a.f.dr), a.f, q, qk);
      unsigned long long seen = p.seen;
      for (int n = 0; seen; ++n) {
        const int at = __ffsll((long long)seen) - 1;
        seen &= seen - 1;
        if (n % W != warp) continue;
        uint64_t x[E / 2];
        float k[2];
        load_row<T>(static_cast<const T*>(a.rows) + (p.lo + at) * a.row_stride, a.f, x, k);
        run.add(warp_sum(dot_share<T>(q, qk, x, k)) * a.scale_log2, 1.f, x);
      }
    }
    constexpr int U = 4;                                 // parts whose loads are in flight together
    for (int n0 = warp; n0 < parts.y; n0 += U * W) {
      float2 ml[U];
      uint64_t x[U][E / 2];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int n = n0 + i * W;
        if (n >= parts.y) break;
        const long long at = (long long)(parts.x + n) * a.cols + parts.z;
        ml[i] = reinterpret_cast<const float2*>(a.ml_part)[at];
        load_part<T>(a.o_part + at * a.part_row, r, x[i]);
      }
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (n0 + i * W < parts.y) run.add(ml[i].x, ml[i].y, x[i]);
    }
    if (lane == 0) {
      s_m[warp] = run.m;
      s_l[warp] = run.l;
    }
#pragma unroll
    for (int e = 0; e < E / 2; ++e) s_acc[warp][e][lane] = run.acc[e];
    __syncthreads();
    float top = s_m[0];
#pragma unroll
    for (int w = 1; w < W; ++w) top = fmaxf(top, s_m[w]);
    const float ref = top == -INFINITY ? 0.f : top;
    float l = 0.f, share[W];
#pragma unroll
    for (int w = 0; w < W; ++w) {                        // in the warps' order
      share[w] = exp2f(s_m[w] - ref);
      l = fmaf(share[w], s_l[w], l);
    }
    for (int e = warp; e < E / 2; e += W) {              // a pair of every lane's latents
      uint64_t sum = 0;
#pragma unroll
      for (int w = 0; w < W; ++w) sum = ptx::fma2(ptx::pack2(share[w], share[w]), s_acc[w][e][lane], sum);
      store_pair<T>(a, column, e, top, l, failed, sum);
    }
    __syncthreads();
  }
}

// bf16, a CTA per group of NC columns, a warp per 16 columns and half of the rows (scores) or of the runs of 32 latents
// (values); m16n8k16 instructions.  The request's rows lie in shared memory with the
// pairs of every 32 latents transposed (pair 4 i + j at place 4 j + i): read as they are, they give lane (g, t) the
// latents 8t .. 8t + 7 of row g, which it also reads of a query in one piece; read transposed, they give the output's
// fragments eight latents in a row.  A probability enters as two bf16 terms, 2^-17 of it.  A matrix product
// touches every row, so a row with an infinity or a NaN is taken as zeros, and columns that see it get NaN.
template <int NC>
struct Dense {
  static constexpr int kThreads = NC * 4, kTiles = NC / 16;
  __host__ __device__ static constexpr int row_bytes(const qp::Format& f) { return 2 * (f.r + f.dr) + 16; }
  __host__ __device__ static constexpr int bytes(const qp::Format& f) { return kMaxNodes * row_bytes(f); }
};

template <int NC>
__global__ void __launch_bounds__(NC * 4, 2) tree_join_dense_kernel(JoinArgs a) {
  using D = Dense<NC>;
  extern __shared__ __align__(128) uint8_t rows_s[];
  __shared__ uint4 p_s[D::kTiles][4][2][32];          // A fragments of 16 columns by 16 rows, two terms
  __shared__ unsigned long long seen_s[NC];
  __shared__ float max_s[2][NC], sum_s[2][NC];
  __shared__ unsigned int bad_s[2];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int mt = warp >> 1, half = warp & 1, r = a.f.r, width = r + a.f.dr, stride = D::row_bytes(a.f);
  if (tid < 2) bad_s[tid] = 0;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  bool failed = false;
  for (int i = tid; i < a.n_error_words; i += D::kThreads) failed |= a.error_words[i] != 0;
  failed = __syncthreads_or(failed);
  const int n_groups = a.listed->x, v = blockIdx.x;
  bf16* out = static_cast<bf16*>(a.out);
  if (n_groups < 0) {                                  // the batch is refused
    const long long n = (long long)a.n_nodes * a.heads, step = (long long)gridDim.x * D::kThreads;
    const long long first = (long long)v * D::kThreads + tid;
    for (long long i = first; i < n * r; i += step) out[i] = __float2bfloat16_rn(NAN);
    for (long long i = first; a.lse && i < n; i += step) a.lse[i] = NAN;
    return;
  }
  if (v >= n_groups) return;
  const int4 group = a.groups[v];
  const int lo = a.starts[group.x], count = a.starts[group.x + 1] - lo, n_rows = min(count, kMaxNodes);
  const int steps = (n_rows + 15) / 16;                // of 16 rows
  const int2 parts = !failed && group.w > 0 ? a.parts[v] : make_int2(0, 0);      // see parts_of
  if (tid < NC) {
    unsigned long long seen = 0;
    if (tid < group.z) {
      seen = (unsigned long long)a.seen[(group.y + tid) / a.heads];
      if (count < kMaxNodes) seen &= (1ull << count) - 1;
    }
    seen_s[tid] = seen;
  }
  // ---- rows into shared memory: a warp per row, two in flight, 16 bytes a lane and up to three of those
  {
    constexpr int kWarps = D::kThreads / 32;
    const int runs = width / 8;
    const bf16* src = static_cast<const bf16*>(a.rows) + (long long)lo * a.row_stride;
    for (int row0 = warp; row0 < steps * 16; row0 += 2 * kWarps) {
      uint4 w[2][3];
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < 3; ++i) {
          const int row = row0 + k * kWarps, c = lane + 32 * i;
          w[k][i] = make_uint4(0u, 0u, 0u, 0u);
          if (row < n_rows && c < runs) w[k][i] = *reinterpret_cast<const uint4*>(src + row * a.row_stride + c * 8);
        }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int row = row0 + k * kWarps;
        if (row >= steps * 16) break;
        // A magnitude plus one in its exponent reaches the sign bit for an infinity or a NaN alone.
        uint32_t odd = 0;
#pragma unroll
        for (int i = 0; i < 3; ++i) {
          const uint32_t x[4] = {w[k][i].x, w[k][i].y, w[k][i].z, w[k][i].w};
#pragma unroll
          for (int m = 0; m < 4; ++m) odd |= (x[m] & 0x7fff7fffu) + 0x00800080u;
        }
        const bool bad = __any_sync(0xffffffffu, odd & 0x80008000u);
        if (bad && lane == 0) atomicOr(&bad_s[row >> 5], 1u << (row & 31));
        uint32_t* dst = reinterpret_cast<uint32_t*>(rows_s + row * stride + (lane >> 2) * 64) + (lane & 3);
#pragma unroll
        for (int i = 0; i < 3; ++i, dst += 128) {
          if (lane + 32 * i >= runs) break;
          dst[0] = bad ? 0u : w[k][i].x;
          dst[4] = bad ? 0u : w[k][i].y;
          dst[8] = bad ? 0u : w[k][i].z;
          dst[12] = bad ? 0u : w[k][i].w;
        }
      }
    }
  }
  __syncthreads();
  const uint32_t rows_u32 = ptx::smem_u32(rows_s);
  const int c0 = mt * 16 + g, c1 = c0 + 8;             // this lane's columns
  // ---- scores of 16 columns by 32 rows
  float s[4][4];
#pragma unroll
  for (int n = 0; n < 4; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) s[n][i] = 0.f;
  {
    const bf16* q = static_cast<const bf16*>(a.q) + (long long)group.y * width + 8 * t;
    const uint32_t at = rows_u32 + (half * 32 + (lane & 7)) * stride + (lane >> 3) * 16;
    const int chunks = width / 32;
    if (half * 32 < steps * 16) {
      constexpr int F = 6;                               // runs of a query in flight; r + d_R has at most 18
      for (int f0 = 0; f0 < chunks; f0 += F) {
        uint4 q0[F], q1[F];
#pragma unroll
        for (int f = 0; f < F; ++f) {
          const int c = f0 + f;
          q0[f] = q1[f] = make_uint4(0u, 0u, 0u, 0u);
          if (c < chunks && c0 < group.z) q0[f] = *reinterpret_cast<const uint4*>(q + (long long)c0 * width + c * 32);
          if (c < chunks && c1 < group.z) q1[f] = *reinterpret_cast<const uint4*>(q + (long long)c1 * width + c * 32);
        }
#pragma unroll
        for (int f = 0; f < F; ++f) {
          if (f0 + f >= chunks) break;
          const uint32_t a0[4] = {q0[f].x, q1[f].x, q0[f].y, q1[f].y}, a1[4] = {q0[f].z, q1[f].z, q0[f].w, q1[f].w};
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            if (half * 32 + n * 8 >= steps * 16) break;
            uint32_t w[4];
            qp::ldsm_x4(at + n * 8 * stride + (f0 + f) * 64, w);
            qp::mma_bf16(s[n], a0, w[0], w[1]);
            qp::mma_bf16(s[n], a1, w[2], w[3]);
          }
        }
      }
    }
  }
  // ---- softmax over the rows that each column sees: bits of row half * 32 + 8 n + 2 t + e
  const uint32_t see0 = (uint32_t)(seen_s[c0] >> (32 * half)), see1 = (uint32_t)(seen_s[c1] >> (32 * half));
  const unsigned long long bad = bad_s[0] | (unsigned long long)bad_s[1] << 32;
  float top0 = -INFINITY, top1 = -INFINITY;
#pragma unroll
  for (int n = 0; n < 4; ++n)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t bit = 1u << (8 * n + 2 * t + e);
      s[n][e] = see0 & bit ? s[n][e] * a.scale_log2 : -INFINITY;
      s[n][2 + e] = see1 & bit ? s[n][2 + e] * a.scale_log2 : -INFINITY;
      top0 = fmaxf(top0, s[n][e]);
      top1 = fmaxf(top1, s[n][2 + e]);
    }
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    top0 = fmaxf(top0, __shfl_xor_sync(0xffffffffu, top0, o));
    top1 = fmaxf(top1, __shfl_xor_sync(0xffffffffu, top1, o));
  }
  if (t == 0) {
    max_s[half][c0] = top0;
    max_s[half][c1] = top1;
  }
  __syncthreads();
  const float m0 = fmaxf(max_s[0][c0], max_s[1][c0]), m1 = fmaxf(max_s[0][c1], max_s[1][c1]);
  const float ref0 = m0 == -INFINITY ? 0.f : m0, ref1 = m1 == -INFINITY ? 0.f : m1;
  float sum0 = 0.f, sum1 = 0.f;
  uint32_t hi[4][2], low[4][2];                        // [n-tile][column]
#pragma unroll
  for (int n = 0; n < 4; ++n)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const float p0 = exp2f(s[n][2 * c] - (c ? ref1 : ref0)), p1 = exp2f(s[n][2 * c + 1] - (c ? ref1 : ref0));
      (c ? sum1 : sum0) += p0 + p1;
      const __nv_bfloat162 x = __floats2bfloat162_rn(p0, p1);
      const __nv_bfloat162 y = __floats2bfloat162_rn(p0 - __low2float(x), p1 - __high2float(x));
      hi[n][c] = *reinterpret_cast<const uint32_t*>(&x);
      low[n][c] = *reinterpret_cast<const uint32_t*>(&y);
    }
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    sum0 += __shfl_xor_sync(0xffffffffu, sum0, o);
    sum1 += __shfl_xor_sync(0xffffffffu, sum1, o);
  }
  if (t == 0) {
    sum_s[half][c0] = sum0;
    sum_s[half][c1] = sum1;
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    p_s[mt][half * 2 + k][0][lane] = make_uint4(hi[2 * k][0], hi[2 * k][1], hi[2 * k + 1][0], hi[2 * k + 1][1]);
    p_s[mt][half * 2 + k][1][lane] = make_uint4(low[2 * k][0], low[2 * k][1], low[2 * k + 1][0], low[2 * k + 1][1]);
  }
  __syncthreads();
  // ---- references and denominators of the whole, this lane's two columns
  float whole_m[2] = {m0, m1}, whole_l[2] = {sum_s[0][c0] + sum_s[1][c0], sum_s[0][c1] + sum_s[1][c1]}, drafted[2];
  const float2* ml = reinterpret_cast<const float2*>(a.ml_part) + (long long)parts.x * NC;
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const int col = c ? c1 : c0;
    float m = whole_m[c];
    if (col < group.z)
#pragma unroll 4
      for (int n = 0; n < parts.y; ++n) m = fmaxf(m, ml[n * NC + col].x);
    const float ref = m == -INFINITY ? 0.f : m;
    drafted[c] = exp2f(whole_m[c] - ref);
    float l = whole_l[c] * drafted[c];
    if (col < group.z)
#pragma unroll 4
      for (int n = 0; n < parts.y; ++n) {
        const float2 x = ml[n * NC + col];
        l += exp2f(x.x - ref) * x.y;
      }
    if (failed || (seen_s[col] & bad)) l = NAN;
    whole_m[c] = ref;
    whole_l[c] = l;
    if (a.lse && half == 0 && t == 0 && col < group.z)
      a.lse[group.y + col] = l == 0.f ? -INFINITY : (ref + log2f(l)) * 0.69314718055994531f;
  }
  // ---- values: runs of 32 latents, every second is this warp's
  constexpr int F = 2;                                 // parts in flight
  float w_first[2][F];
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int n = 0; n < F; ++n) {
      const int col = c ? c1 : c0;
      w_first[c][n] = n < parts.y && col < group.z ? exp2f(ml[n * NC + col].x - whole_m[c]) : 0.f;
    }
  const float inv[2] = {whole_l[0] == 0.f ? 0.f : 1.f / whole_l[0], whole_l[1] == 0.f ? 0.f : 1.f / whole_l[1]};
  for (int c = half; c < r / 32; c += 2) {
    // The first parts' loads go ahead of the products.
    float4 x0[2][F], x1[2][F];
    float w_part[2][F];
    auto load_parts = [&](int n0) {
#pragma unroll
      for (int col2 = 0; col2 < 2; ++col2)
#pragma unroll
        for (int f = 0; f < F; ++f) {
          const int col = col2 ? c1 : c0, n = n0 + f;
          x0[col2][f] = x1[col2][f] = make_float4(0.f, 0.f, 0.f, 0.f);
          w_part[col2][f] = 0.f;
          if (n < parts.y && col < group.z) {
            const float* part = a.o_part + ((long long)(parts.x + n) * NC + col) * a.part_row + c * 32 + 8 * t;
            x0[col2][f] = *reinterpret_cast<const float4*>(part);
            x1[col2][f] = *reinterpret_cast<const float4*>(part + 4);
            w_part[col2][f] = n0 == 0 ? w_first[col2][f] : exp2f(ml[n * NC + col].x - whole_m[col2]);
          }
        }
    };
    load_parts(0);
    float o[4][4];
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[n][i] = 0.f;
    // Rows k * 16 + ..: matrices of rows 0 .. 7 and 8 .. 15 at places 8 n and 8 n + 8.
    const uint32_t at = rows_u32 + (lane & 15) * stride + c * 64 + (lane >> 4) * 16;
    for (int k = 0; k < steps; ++k) {
      const uint4 x = p_s[mt][k][0][lane], y = p_s[mt][k][1][lane];
      const uint32_t p0[4] = {x.x, x.y, x.z, x.w}, p1[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int n = 0; n < 4; n += 2) {
        uint32_t w[4];
        qp::ldsm_x4_trans(at + k * 16 * stride + n * 16, w);
        qp::mma_bf16(o[n], p0, w[0], w[1]);
        qp::mma_bf16(o[n + 1], p0, w[2], w[3]);
        qp::mma_bf16(o[n], p1, w[0], w[1]);
        qp::mma_bf16(o[n + 1], p1, w[2], w[3]);
      }
    }
    // Fragment column 2t + e of tile n is latent 8t + 2n + e: eight in a row.
    float y[2][8];
#pragma unroll
    for (int col2 = 0; col2 < 2; ++col2)
#pragma unroll
      for (int i = 0; i < 8; ++i) y[col2][i] = o[i / 2][2 * col2 + i % 2] * drafted[col2];
    for (int n0 = 0; n0 < parts.y; n0 += F) {
#pragma unroll
      for (int col2 = 0; col2 < 2; ++col2)
#pragma unroll
        for (int f = 0; f < F; ++f) {
          const float w = w_part[col2][f];
          const float4 u = x0[col2][f], v4 = x1[col2][f];
          const float x[8] = {u.x, u.y, u.z, u.w, v4.x, v4.y, v4.z, v4.w};
#pragma unroll
          for (int i = 0; i < 8; ++i) y[col2][i] = fmaf(w, x[i], y[col2][i]);
        }
      if (n0 + F < parts.y) load_parts(n0 + F);
    }
#pragma unroll
    for (int col2 = 0; col2 < 2; ++col2) {
      const int col = col2 ? c1 : c0;
      if (col >= group.z) continue;
#pragma unroll
      for (int i = 0; i < 8; ++i) y[col2][i] *= inv[col2];
      store_vec(out + (long long)(group.y + col) * r + c * 32 + 8 * t, y[col2]);
    }
  }
}

}  // namespace tree
}  // namespace mtla
