// Rotary positions applied to part of every head of one or more tensors, in one launch.
//
// Pair k of a token at position p turns by the angle p f_k (y0 = x0 cos - x1 sin, y1 = x1 cos +
// x0 sin, times a magnitude); the inverse turns back, which is also the gradient.  The angle is
// formed in 64 bits as a fraction of a full turn, p * (f_k / 2 pi) minus the nearest integer: in 32
// bits a position of 10^5 would leave only about 10^-2 of the angle.  Cosine and sine of the
// fraction are then 32-bit, once per token and pair, shared by all heads through shared memory.
//
// The kernel is bound by the bytes of the heads, each read and written once (16 bytes per access
// where the layout allows it, chosen by the host).  A thread keeps one place in a token (tensor, head,
// unit) and walks over the CTA's tokens, so addresses are additions; it takes a few tokens at a time,
// all loads first, and the first ones before the angles are computed.  (With an index decoded per
// unit the rotation of 65536 x 16 heads of 128, half of them rotated, took 132 us, with one load at a
// time 197 us; so it takes 107 us, 80 % of the measured copy bandwidth.  Four CTAs an SM: without
// a limit on the registers 118 us, with five CTAs 144 us.)
#pragma once

#include "common.cuh"
#include "sm100_ptx.cuh"

namespace mtla {
namespace rp {

constexpr int kThreads = 256;
constexpr int kMaxPairs = 128;
constexpr int kMaxTensors = 4;
constexpr int kMaxTokens = 16;         // tokens per CTA

struct Tensor {
  const void* x;
  void* y;
  long long x_token, x_head, y_token, y_head;   // strides, elements
  int first;                                    // start of the rotated part
  int units, copy_units;                        // units of a head; of these plain ones (0 in place)
  int all_units;                                // units of a token: heads times units
};

struct Args {
  Tensor t[kMaxTensors];
  double turns[kMaxPairs];                      // f_k / 2 pi
  const int* positions;
  float magnitude;
  int per_token;                                // units of a token over all tensors
  int lanes, rows;                              // threads of a token; tokens side by side: lanes * rows <= kThreads
  int n_tensors, n_tokens, tokens_per_cta, pairs, inverse;
};

// A unit of work is, with VEC, 16 bytes (interleaved pairs and plain elements) or two runs of 16
// bytes, one from each half (half layout); without VEC, one pair or one plain element.
template <typename T, bool VEC, bool HALF>
__global__ void __launch_bounds__(kThreads, 4) rope_kernel(const __grid_constant__ Args a) {
  constexpr int V = VEC ? Elem<T>::kVec : 1;
  constexpr int kU = 4;                         // tokens of a thread in flight
  extern __shared__ __align__(16) float2 cs[];  // [tokens_per_cta][pairs]
  const int t0 = blockIdx.x * a.tokens_per_cta, nt = min(a.tokens_per_cta, a.n_tokens - t0), half = a.pairs;
  const int row = threadIdx.x / a.lanes, lane = threadIdx.x - row * a.lanes;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();

  // The place: x, y at token t0, first pair k (k < 0: plain).
  const T* x = nullptr;
  T* y = nullptr;
  long long x_step = 0, y_step = 0;
  int k = -1;
  auto place = [&](int u) {
    int n = 0;
    while (u >= a.t[n].all_units) u -= a.t[n++].all_units;
    const Tensor& q = a.t[n];
    const int h = u / q.units, i = u - h * q.units - q.copy_units;
    int e;
    if (i < 0) {                                // plain: in front of the part, or behind it
      e = (i + q.copy_units) * V;
      if (e >= q.first) e += 2 * half;
      k = -1;
    } else {
      e = q.first + i * (VEC ? V : (HALF ? 1 : 2));
      k = HALF ? i * V : (VEC ? i * (V / 2) : i);
    }
    x = static_cast<const T*>(q.x) + t0 * q.x_token + h * q.x_head + e;
    y = static_cast<T*>(q.y) + t0 * q.y_token + h * q.y_head + e;
    x_step = q.x_token;
    y_step = q.y_token;
  };
  struct Data {
    uint4 lo, hi;        // VEC: the runs
    float a, b;          // otherwise: the members
  };
  Data d[kU];
  auto load = [&](int t, Data& v) {
    const T* p = x + t * x_step;
    if constexpr (VEC) {
      v.lo = *reinterpret_cast<const uint4*>(p);
      if (HALF && k >= 0) v.hi = *reinterpret_cast<const uint4*>(p + half);
    } else {
      v.a = Elem<T>::to_float(p[0]);
      if (k >= 0) v.b = Elem<T>::to_float(p[HALF ? half : 1]);
    }
  };
  auto finish = [&](int t, Data& v) {
    T* p = y + t * y_step;
    const float2* r = cs + t * half + k;
    if constexpr (VEC) {
      if (k < 0) {
        *reinterpret_cast<uint4*>(p) = v.lo;
        return;
      }
      float lo[V];
      load_vec(reinterpret_cast<const T*>(&v.lo), lo);
      if constexpr (HALF) {
        float hi[V];
        load_vec(reinterpret_cast<const T*>(&v.hi), hi);
#pragma unroll
        for (int i = 0; i < V; i += 2) {
          const float4 c = *reinterpret_cast<const float4*>(r + i);         // two pairs' cosine, sine
          const float p0 = lo[i] * c.x - hi[i] * c.y, p1 = lo[i + 1] * c.z - hi[i + 1] * c.w;
          hi[i] = hi[i] * c.x + lo[i] * c.y;
          hi[i + 1] = hi[i + 1] * c.z + lo[i + 1] * c.w;
          lo[i] = p0;
          lo[i + 1] = p1;
        }
        store_vec(p, lo);
        store_vec(p + half, hi);
      } else {
#pragma unroll
        for (int i = 0; i < V / 2; i += 2) {
          const float4 c = *reinterpret_cast<const float4*>(r + i);
          const float p0 = lo[2 * i] * c.x - lo[2 * i + 1] * c.y, p1 = lo[2 * i + 2] * c.z - lo[2 * i + 3] * c.w;
          lo[2 * i + 1] = lo[2 * i + 1] * c.x + lo[2 * i] * c.y;
          lo[2 * i + 3] = lo[2 * i + 3] * c.z + lo[2 * i + 2] * c.w;
          lo[2 * i] = p0;
          lo[2 * i + 2] = p1;
        }
        store_vec(p, lo);
      }
    } else {
      if (k < 0) {
        p[0] = Elem<T>::from_float(v.a);
        return;
      }
      p[0] = Elem<T>::from_float(v.a * r->x - v.b * r->y);
      p[HALF ? half : 1] = Elem<T>::from_float(v.b * r->x + v.a * r->y);
    }
  };

  const bool works = row < a.rows;
  int u = lane + blockIdx.y * a.lanes, t = row;
  bool have = works && u < a.per_token;
  if (have) place(u);
  auto load_batch = [&]() {
#pragma unroll
    for (int i = 0; i < kU; ++i)
      if (have && t + i * a.rows < nt) load(t + i * a.rows, d[i]);
  };
  load_batch();
  for (int i = threadIdx.x; i < nt * a.pairs; i += kThreads) {
    const int tt = i / a.pairs, kk = i - tt * a.pairs;
    const double turn = (double)a.positions[t0 + tt] * a.turns[kk];
    const float frac = (float)(turn - rint(turn));
    float s, c;
    sincospif(2.f * frac, &s, &c);
    cs[i] = make_float2(c * a.magnitude, (a.inverse ? -s : s) * a.magnitude);
  }
  __syncthreads();
  while (have) {
#pragma unroll
    for (int i = 0; i < kU; ++i)
      if (t + i * a.rows < nt) finish(t + i * a.rows, d[i]);
    t += kU * a.rows;
    if (t >= nt) {                              // on to the next place
      t = row;
      u += a.lanes * gridDim.y;
      have = u < a.per_token;
      if (have) place(u);
    }
    load_batch();
  }
}

}  // namespace rp
}  // namespace mtla
