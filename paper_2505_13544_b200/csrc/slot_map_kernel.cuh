// Block tables and slot maps from request lengths, on the GPU in one launch.
//
// With h_b tokens held and f_b new ones, request b ends with ceil((h_b + f_b) / s) slots and needs
// ceil(slots / 64) - ceil(ceil(h_b / s) / 64) more pages, which it takes from the free list in
// request order.  Every CTA forms the two prefix sums (new tokens, new pages) over the whole batch
// by itself, which costs less than a second launch or a grid-wide wait (a batch is at most a few
// thousand pairs of integers out of L2), and then fills its share of the token arrays.  The table
// entries of new pages follow from the prefix sums, so no CTA reads what another writes.
#pragma once

#include "common.cuh"
#include "sm100_ptx.cuh"

namespace mtla {
namespace sm {

constexpr int kThreads = 256;
constexpr int kMaxBatch = 16384;       // lengths and two prefix sums in shared memory
constexpr int kPage = 64;
constexpr int kFewPages = 2;           // new pages of a request that one thread enters by itself

struct Args {
  const int* held;
  const int* fresh;
  int* table;                // [batch][width]
  const int* free_pages;
  int *starts, *seq, *position;
  long long *slot, *store;
  int *slots, *taken;
  int batch, stride, width, n_free, n_tokens;
  int vec;                   // the token arrays are 16-byte aligned
};

// Slots and pages of `tokens` tokens, 0 .. 2^31 - 1, in 32-bit arithmetic that cannot overflow.
__device__ __forceinline__ uint32_t slots_of(uint32_t tokens, uint32_t stride) {
  return tokens ? (tokens - 1) / stride + 1 : 0;
}
__device__ __forceinline__ int pages_of(uint32_t tokens, uint32_t stride) {
  return (int)((slots_of(tokens, stride) + kPage - 1) / kPage);
}

// PER: consecutive tokens of a thread.  Four give 16-byte stores where there are tokens for every SM;
// with fewer, one token a thread keeps the chain of dependent loads short (128 requests of one token: 8.3
// us with four, 3.1 us so; 400000 tokens: 7.0 us, of which the bytes are 1.5).
template <int PER>
__global__ void __launch_bounds__(kThreads) slot_map_kernel(Args a) {
  extern __shared__ int smem[];
  int* s_start = smem;                   // [batch + 1] first token of every request
  int* s_page = smem + a.batch + 1;      // [batch + 1] first new page of every request
  int* s_held = s_page + a.batch + 1;    // [batch]
  __shared__ long long warp_tok[kThreads / 32], warp_page[kThreads / 32];
  __shared__ int s_bad;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) s_bad = 0;
  __syncthreads();
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();

  const int per = ceil_div(a.batch, kThreads);
  const int lo = min(a.batch, tid * per), hi = min(a.batch, lo + per);
  long long tok = 0, page = 0;
  bool bad = false;
  for (int b = lo; b < hi; ++b) {
    const long long h = a.held[b], f = a.fresh[b];
    const bool ok = h >= 0 && f >= 0 && h + f <= 0x7fffffffll;
    const int have = ok ? pages_of((uint32_t)h, a.stride) : 0;
    const int want = ok ? pages_of((uint32_t)(h + f), a.stride) : 0;
    s_held[b] = h > 0 ? (int)h : 0;
    bad |= !ok || want > a.width;
    s_start[b] = ok ? (int)f : 0;        // for now the counts
    s_page[b] = want - have;
    tok += ok ? f : 0;
    page += want - have;
  }
  long long tok_in = tok, page_in = page;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long t = __shfl_up_sync(0xffffffffu, tok_in, o), p = __shfl_up_sync(0xffffffffu, page_in, o);
    if (lane >= o) { tok_in += t; page_in += p; }
  }
  if (lane == 31) { warp_tok[warp] = tok_in; warp_page[warp] = page_in; }
  if (bad) s_bad = 1;
  __syncthreads();
  long long tok_at = tok_in - tok, page_at = page_in - page, n_tok = 0, n_page = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) { tok_at += warp_tok[w]; page_at += warp_page[w]; }
    n_tok += warp_tok[w];
    n_page += warp_page[w];
  }
  // A batch that does not fit is refused as a whole: no page is taken, no token gets a slot.
  const bool refuse = s_bad || n_tok > a.n_tokens || n_page > a.n_free;
  for (int b = lo; b < hi; ++b) {
    const int t = s_start[b], p = s_page[b];
    s_start[b] = refuse ? 0 : (int)tok_at;
    s_page[b] = refuse ? 0 : (int)page_at;
    tok_at += t;
    page_at += p;
  }
  if (tid == 0) {
    s_start[a.batch] = refuse ? 0 : (int)n_tok;
    s_page[a.batch] = refuse ? 0 : (int)n_page;
  }
  __syncthreads();
  const int total = s_start[a.batch];

  // Per request, a thread each: offsets, slot counts, the new entries of its table row; rows with more
  // than a few new entries are written by the whole warp.
  // Consecutive requests go to different CTAs.
  for (int i0 = warp * 32; (long long)i0 * gridDim.x + blockIdx.x < a.batch; i0 += kThreads) {
    const int b = (int)min((long long)a.batch, (long long)(i0 + lane) * gridDim.x + blockIdx.x);
    int have = 0, p0 = 0, n_new = 0;
    if (b < a.batch) {
      const int h = s_held[b], first = s_start[b];
      have = pages_of(h, a.stride);
      p0 = s_page[b];
      n_new = s_page[b + 1] - p0;
      a.starts[b] = first;
      a.slots[b] = (int)slots_of((uint32_t)h + (s_start[b + 1] - first), a.stride);
      if (n_new <= kFewPages)
        for (int i = 0; i < n_new; ++i) a.table[(long long)b * a.width + have + i] = a.free_pages[p0 + i];
    }
    uint32_t big = __ballot_sync(0xffffffffu, n_new > kFewPages);
    while (big) {
      const int src = __ffs(big) - 1;
      big &= big - 1;
      const int bb = __shfl_sync(0xffffffffu, b, src), hh = __shfl_sync(0xffffffffu, have, src), pp = __shfl_sync(0xffffffffu, p0, src),
                nn = __shfl_sync(0xffffffffu, n_new, src);
      for (int i = lane; i < nn; i += 32) a.table[(long long)bb * a.width + hh + i] = a.free_pages[pp + i];
    }
  }
  if (blockIdx.x == 0 && tid == 0) {
    a.starts[a.batch] = total;
    a.taken[0] = refuse ? -1 : (int)n_page;
  }

  // Per token.
  for (long long t0 = ((long long)blockIdx.x * kThreads + tid) * PER; t0 < a.n_tokens;
       t0 += (long long)gridDim.x * kThreads * PER) {
    int seq[PER], pos[PER];
    long long slot[PER], store[PER];
    int b = 0;
    if (t0 < total) {                              // the last request that starts at or before t0
      int lo_b = 0, hi_b = a.batch;
      while (hi_b - lo_b > 1) {
        const int mid = (lo_b + hi_b) >> 1;
        if (s_start[mid] <= t0) lo_b = mid; else hi_b = mid;
      }
      b = lo_b;
    }
    int held = t0 < total ? s_held[b] : 0, page_of = -1;
    long long page = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const long long t = t0 + i;
      seq[i] = -1; pos[i] = 0; slot[i] = -1; store[i] = -1;
      if (t >= total) continue;
      while (s_start[b + 1] <= t) {                // requests without new tokens are stepped over
        ++b;
        held = s_held[b];
        page_of = -1;
      }
      const int p = held + (int)(t - s_start[b]);
      const int j = (int)((uint32_t)p / (uint32_t)a.stride);
      if (page_of != j >> 6) {
        page_of = j >> 6;
        const int have = pages_of(held, a.stride);
        page = page_of < have ? a.table[(long long)b * a.width + page_of] : a.free_pages[s_page[b] + page_of - have];
      }
      seq[i] = b;
      pos[i] = p;
      slot[i] = page * kPage + (j & 63);
      const bool last = p - j * a.stride == a.stride - 1 || t + 1 == s_start[b + 1];
      store[i] = last ? slot[i] : -1;
    }
    if (PER == 4 && a.vec && t0 + PER <= a.n_tokens) {
      *reinterpret_cast<int4*>(a.seq + t0) = make_int4(seq[0], seq[1 % PER], seq[2 % PER], seq[3 % PER]);
      *reinterpret_cast<int4*>(a.position + t0) = make_int4(pos[0], pos[1 % PER], pos[2 % PER], pos[3 % PER]);
      *reinterpret_cast<longlong2*>(a.slot + t0) = make_longlong2(slot[0], slot[1 % PER]);
      *reinterpret_cast<longlong2*>(a.slot + t0 + 2) = make_longlong2(slot[2 % PER], slot[3 % PER]);
      *reinterpret_cast<longlong2*>(a.store + t0) = make_longlong2(store[0], store[1 % PER]);
      *reinterpret_cast<longlong2*>(a.store + t0 + 2) = make_longlong2(store[2 % PER], store[3 % PER]);
    } else {
      for (int i = 0; i < PER && t0 + i < a.n_tokens; ++i) {
        a.seq[t0 + i] = seq[i];
        a.position[t0 + i] = pos[i];
        a.slot[t0 + i] = slot[i];
        a.store[t0 + i] = store[i];
      }
    }
  }
}

}  // namespace sm
}  // namespace mtla
