// Rotary positions applied to part of every head of one or more tensors, in one launch.
//
// Pair k of a token at position p turns by the angle p f_k (y0 = x0 cos - x1 sin, y1 = x1 cos +
// x0 sin, times a magnitude); the inverse turns back, which is also the gradient.  The angle is
// formed in 64 bits as a fraction of a full turn, p * (f_k / 2 pi) minus the nearest integer: in 32
// bits a position of 10^5 would leave only about 10^-2 of the angle.  Cosine and sine of the
// fraction are then 32-bit, once per token and pair, shared by all heads through shared memory.
//
// The kernel is bound by the bytes of the heads, each read and written once (16 bytes per access
// where the layout allows it, chosen by the host).  What it needs for that is loads in flight: a
// thread takes four units of work at a time, all their loads first, and the first four before the
// angles are computed.
#pragma once

#include "common.cuh"
#include "sm100_ptx.cuh"

namespace mtla {
namespace rp {

constexpr int kThreads = 256;
constexpr int kMaxPairs = 128;
constexpr int kMaxTensors = 4;
constexpr int kMaxTokens = 8;          // tokens per CTA

// Quotient by a divisor fixed at launch: the multiplication gives it or one more.
struct Divisor {
  uint32_t d, mul;
  void set(int divisor) {
    d = (uint32_t)divisor;
    mul = (uint32_t)((0x100000000ull + d - 1) / d);          // d = 1: 0, see below
  }
  __device__ __forceinline__ uint32_t quotient(uint32_t n) const {
    uint32_t q = __umulhi(n, mul);
    if (q * d > n) --q;
    return mul ? q : n;
  }
};

struct Tensor {
  const void* x;
  void* y;
  long long x_token, x_head, y_token, y_head;   // strides, elements
  int first;                                    // start of the rotated part
  int copy_units;                               // plain elements in front of and behind the part, in units; 0 in place
  int all_units;                                // units of a token: heads times units of a head
  Divisor units;                                // units of a head
};

struct Args {
  Tensor t[kMaxTensors];
  double turns[kMaxPairs];                      // f_k / 2 pi
  const int* positions;
  Divisor per_token;                            // units of a token over all tensors
  float magnitude;
  int n_tensors, n_tokens, tokens_per_cta, pairs, inverse;
};

// A unit of work is, with VEC, 16 bytes (interleaved pairs and plain elements) or two runs of 16
// bytes, one from each half (half layout); without VEC, one pair or one plain element.
template <typename T, bool VEC, bool HALF>
__global__ void __launch_bounds__(kThreads) rope_kernel(const __grid_constant__ Args a) {
  constexpr int V = VEC ? Elem<T>::kVec : 1;
  constexpr int kU = 4;                         // units of a thread in flight
  __shared__ float2 cs[kMaxTokens][kMaxPairs];
  const int t0 = blockIdx.x * a.tokens_per_cta, nt = min(a.tokens_per_cta, a.n_tokens - t0);
  const int total = nt * (int)a.per_token.d, half = a.pairs;
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();

  struct Unit {
    T* y;                // where the unit's first run goes
    int t, k;            // token of the CTA, first pair; k < 0: plain
    uint4 lo, hi;        // VEC: the runs
    float a, b;          // otherwise: the members
  };
  Unit u[kU];
  auto load = [&](int w, Unit& v) {
    const int t = (int)a.per_token.quotient((uint32_t)w);
    int rem = w - t * (int)a.per_token.d, n = 0;
    while (rem >= a.t[n].all_units) rem -= a.t[n++].all_units;
    const Tensor& q = a.t[n];
    const int h = (int)q.units.quotient((uint32_t)rem), i = rem - h * (int)q.units.d - q.copy_units;
    const T* x = static_cast<const T*>(q.x) + (t0 + t) * q.x_token + h * q.x_head;
    T* y = static_cast<T*>(q.y) + (t0 + t) * q.y_token + h * q.y_head;
    int e;
    v.t = t;
    if (i < 0) {                                // plain: in front of the part, or behind it
      e = (i + q.copy_units) * V;
      if (e >= q.first) e += 2 * half;
      v.k = -1;
    } else {
      e = q.first + i * (VEC ? V : (HALF ? 1 : 2));
      v.k = HALF ? i * V : (VEC ? i * (V / 2) : i);
    }
    v.y = y + e;
    x += e;
    if constexpr (VEC) {
      v.lo = *reinterpret_cast<const uint4*>(x);
      if (HALF && i >= 0) v.hi = *reinterpret_cast<const uint4*>(x + half);
    } else {
      v.a = Elem<T>::to_float(x[0]);
      if (i >= 0) v.b = Elem<T>::to_float(x[HALF ? half : 1]);
    }
  };
  auto finish = [&](Unit& v) {
    if constexpr (VEC) {
      if (v.k < 0) {
        *reinterpret_cast<uint4*>(v.y) = v.lo;
        return;
      }
      float lo[V];
      load_vec(reinterpret_cast<const T*>(&v.lo), lo);
      if constexpr (HALF) {
        float hi[V];
        load_vec(reinterpret_cast<const T*>(&v.hi), hi);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float2 r = cs[v.t][v.k + i];
          const float p = lo[i] * r.x - hi[i] * r.y, s = hi[i] * r.x + lo[i] * r.y;
          lo[i] = p;
          hi[i] = s;
        }
        store_vec(v.y, lo);
        store_vec(v.y + half, hi);
      } else {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
          const float2 r = cs[v.t][v.k + i];
          const float p = lo[2 * i] * r.x - lo[2 * i + 1] * r.y, s = lo[2 * i + 1] * r.x + lo[2 * i] * r.y;
          lo[2 * i] = p;
          lo[2 * i + 1] = s;
        }
        store_vec(v.y, lo);
      }
    } else {
      if (v.k < 0) {
        v.y[0] = Elem<T>::from_float(v.a);
        return;
      }
      const float2 r = cs[v.t][v.k];
      v.y[0] = Elem<T>::from_float(v.a * r.x - v.b * r.y);
      v.y[HALF ? half : 1] = Elem<T>::from_float(v.b * r.x + v.a * r.y);
    }
  };

  const int step = kU * kThreads;
#pragma unroll
  for (int i = 0; i < kU; ++i)
    if ((int)threadIdx.x + i * kThreads < total) load(threadIdx.x + i * kThreads, u[i]);
  for (int i = threadIdx.x; i < nt * a.pairs; i += kThreads) {
    const int t = i / a.pairs, k = i - t * a.pairs;
    const double turn = (double)a.positions[t0 + t] * a.turns[k];
    const float frac = (float)(turn - rint(turn));
    float s, c;
    sincospif(2.f * frac, &s, &c);
    cs[t][k] = make_float2(c * a.magnitude, (a.inverse ? -s : s) * a.magnitude);
  }
  __syncthreads();
  for (int w = threadIdx.x; w < total; w += step) {
#pragma unroll
    for (int i = 0; i < kU; ++i)
      if (w + i * kThreads < total) finish(u[i]);
#pragma unroll
    for (int i = 0; i < kU; ++i)
      if (w + step + i * kThreads < total) load(w + step + i * kThreads, u[i]);
  }
}

}  // namespace rp
}  // namespace mtla
