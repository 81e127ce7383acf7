// Rotary positions applied to part of every head of one or more tensors, in one launch.
//
// Pair k of a token at position p turns by the angle p f_k (y0 = x0 cos - x1 sin, y1 = x1 cos +
// x0 sin, times a magnitude); the inverse turns back, which is also the gradient.  The angle is
// formed in 64 bits as a fraction of a full turn, p * (f_k / 2 pi) minus the nearest integer: in 32
// bits a position of 10^5 would leave only about 10^-2 of the angle.  Cosine and sine of the
// fraction are then 32-bit, once per token and pair, shared by all heads through shared memory.
// The kernel is bound by the bytes of the heads, each read and written once (16 bytes per access
// where the layout allows it, chosen by the host).
#pragma once

#include "common.cuh"
#include "sm100_ptx.cuh"

namespace mtla {
namespace rp {

constexpr int kThreads = 256;
constexpr int kMaxPairs = 128;
constexpr int kMaxTensors = 4;
constexpr int kMaxTokens = 8;          // tokens per CTA

struct Tensor {
  const void* x;
  void* y;
  long long x_token, x_head, y_token, y_head;   // strides, elements
  int heads, width, first;                      // heads, their elements, start of the rotated part
  int units;                                    // work units per head (see below)
  int copy_units;                               // of these: plain elements in front of and behind the part
};

struct Args {
  Tensor t[kMaxTensors];
  double turns[kMaxPairs];                      // f_k / 2 pi
  const int* positions;
  float magnitude;
  int n_tensors, n_tokens, tokens_per_cta, pairs, inverse;
};

// A unit of work is, with VEC, 16 bytes (interleaved pairs and plain elements) or two runs of 16
// bytes, one from each half (half layout); without VEC, one pair or one plain element.
template <typename T, bool VEC, bool HALF>
__global__ void __launch_bounds__(kThreads) rope_kernel(const __grid_constant__ Args a) {
  constexpr int V = VEC ? Elem<T>::kVec : 1;
  __shared__ float2 cs[kMaxTokens][kMaxPairs];
  const int t0 = blockIdx.x * a.tokens_per_cta, nt = min(a.tokens_per_cta, a.n_tokens - t0);
  ptx::grid_launch_dependents();
  ptx::grid_dependency_wait();
  for (int i = threadIdx.x; i < nt * a.pairs; i += kThreads) {
    const int t = i / a.pairs, k = i - t * a.pairs;
    const double turn = (double)a.positions[t0 + t] * a.turns[k];
    const float frac = (float)(turn - rint(turn));
    float s, c;
    sincospif(2.f * frac, &s, &c);
    cs[t][k] = make_float2(c * a.magnitude, (a.inverse ? -s : s) * a.magnitude);
  }
  __syncthreads();
  const int half = a.pairs;                     // distance of a pair's members in the half layout
  for (int n = 0; n < a.n_tensors; ++n) {
    const Tensor& q = a.t[n];
    const bool copy = q.x != q.y;
    const int units = copy ? q.units : q.units - q.copy_units;
    const int per_token = q.heads * units, total = nt * per_token;
    for (int w = threadIdx.x; w < total; w += kThreads) {
      const int t = w / per_token, hw = w - t * per_token, h = hw / units;
      int u = hw - h * units;
      const T* x = static_cast<const T*>(q.x) + (t0 + t) * q.x_token + h * q.x_head;
      T* y = static_cast<T*>(q.y) + (t0 + t) * q.y_token + h * q.y_head;
      if (copy) {
        if (u < q.copy_units) {
          int e = u * V;
          if (e >= q.first) e += 2 * half;
          if (VEC) *reinterpret_cast<uint4*>(y + e) = *reinterpret_cast<const uint4*>(x + e);
          else y[e] = x[e];
          continue;
        }
        u -= q.copy_units;
      }
      x += q.first;
      y += q.first;
      if constexpr (HALF) {
        float lo[V], hi[V];
        if constexpr (VEC) {
          load_vec(x + u * V, lo);
          load_vec(x + half + u * V, hi);
        } else {
          lo[0] = Elem<T>::to_float(x[u]);
          hi[0] = Elem<T>::to_float(x[half + u]);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float2 r = cs[t][u * V + i];
          const float p = lo[i] * r.x - hi[i] * r.y, s = hi[i] * r.x + lo[i] * r.y;
          lo[i] = p;
          hi[i] = s;
        }
        if constexpr (VEC) {
          store_vec(y + u * V, lo);
          store_vec(y + half + u * V, hi);
        } else {
          y[u] = Elem<T>::from_float(lo[0]);
          y[half + u] = Elem<T>::from_float(hi[0]);
        }
      } else {
        constexpr int P = VEC ? V / 2 : 1;      // pairs in the unit
        float v[2 * P];
        if constexpr (VEC) {
          load_vec(x + u * V, v);
        } else {
          v[0] = Elem<T>::to_float(x[2 * u]);
          v[1] = Elem<T>::to_float(x[2 * u + 1]);
        }
#pragma unroll
        for (int i = 0; i < P; ++i) {
          const float2 r = cs[t][u * P + i];
          const float p = v[2 * i] * r.x - v[2 * i + 1] * r.y, s = v[2 * i + 1] * r.x + v[2 * i] * r.y;
          v[2 * i] = p;
          v[2 * i + 1] = s;
        }
        if constexpr (VEC) {
          store_vec(y + u * V, v);
        } else {
          y[2 * u] = Elem<T>::from_float(v[0]);
          y[2 * u + 1] = Elem<T>::from_float(v[1]);
        }
      }
    }
  }
}

}  // namespace rp
}  // namespace mtla
