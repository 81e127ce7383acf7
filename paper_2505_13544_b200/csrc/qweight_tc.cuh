// Products of many bf16 rows with 4-bit weights on the fifth-generation tensor cores.
//
// A CTA has a tile of 128 outputs by BN rows of x and a share of the inputs.  The weights are the A operand: expanding
// warps decode 64 inputs of the tile from the raw blocks in shared memory into bf16 (exactly, times 2^-13) and write them
// to tensor memory, the rows of x are the B operand, which a tensor map brings into shared memory with its 128-byte
// swizzle.  So the weights' 4 bits are all that travels of them.  Bound by the matrix unit with many rows (128 x BN x 16
// in BN / 2 cycles; 2048 rows through 4096 x 6720: 92 us, 1.23 PFLOP/s), by the length of the chain with few (load,
// decode, multiply, join: 9 us for 32 rows through 4096 x 4096).  Two CTAs an SM hide each other's starts and ends: with
// 256 outputs a CTA, which halves the reads of x, 512 rows took 33 us, so 28.
//
// With few tiles the inputs are shared out among the CTAs of a cluster, which add their sums through distributed shared
// memory in rank order (read by the CTA that needs them, four at a time: sending them took twice as long).  Every
// wait is bounded; should one give up, the tile's results are NaN.
//
// Roles (12 warps): warp 0 fetches x, warp 3 the weights (one thread for both took 1900 cycles to issue 16 copies), warp 1
// issues, warp 2 owns the tensor memory; warps 4-11 expand, four for each half of a block's inputs, and write the results.
#pragma once

#include "qpool_attn.cuh"
#include "qweight_kernels.cuh"

namespace mtla {
namespace qw {
namespace tc {

constexpr int kExpandWarp0 = 4, kGroups = 2, kExpandThreads = kGroups * 128, kThreads = kExpandWarp0 * 32 + kExpandThreads;
constexpr int kTile = 128;                         // outputs of a tile: eight blocks
constexpr int kRawStages = 4;

template <int BN>
struct Config {
  static constexpr int kAlloc = 256;                                // tensor memory columns: two CTAs an SM
  static constexpr int kUnits = (kAlloc - BN) / 32 < 8 ? (kAlloc - BN) / 32 : 8;            // buffers of 64 inputs
  static constexpr int kPanel = BN * 128;                           // 64 inputs of BN rows
  static constexpr int kStages = BN == 128 ? 4 : 6;
  static constexpr int kRaw = 8 * kBlockBytes;
  static constexpr int kSums = BN * kTile * 4;                      // a cluster's sums lie where the panels were
  static constexpr int kPanels = kStages * kPanel > kSums ? kStages * kPanel : kSums;
  static constexpr int kBytes = kPanels + kRawStages * kRaw + 1024;
  static_assert(kBytes <= 113 * 1024, "shared memory of half an SM");
};

struct Args {
  const uint8_t* packed;
  bf16* y;
  long long y_stride;
  int n, splits;
  int pairs;                 // two neighbouring outputs of a row are four aligned bytes, and n_out is even
  Shape s;
};

struct Misc {
  unsigned long long raw_full[kRawStages], raw_empty[kRawStages], b_full[8], b_empty[8], a_full[8], a_empty[8], done;
  uint32_t tmem_base;
  int failed;
};

__device__ __forceinline__ uint32_t load_cluster(uint32_t addr, uint32_t rank) {
  uint32_t remote, v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(remote) : "memory");
  return v;
}
__device__ __forceinline__ float4 load_cluster4(uint32_t addr, uint32_t rank) {
  uint32_t remote;
  float4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(remote)
               : "memory");
  return v;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// RUN_OUT, the self-test: no row of x is ever fetched, and the waits give up after 2^21 cycles (about a millisecond).
template <int BN, bool RUN_OUT = false>
__global__ void __launch_bounds__(kThreads, 2) qweight_tc_kernel(const __grid_constant__ CUtensorMap x_map, Args a) {
  using namespace ptx;
  using C = Config<BN>;
  constexpr uint32_t IDESC = make_idesc_bf16(128, BN, 0, 0);
  extern __shared__ uint8_t smem_raw[];
  __shared__ Misc misc;
  const uint32_t raw_base = smem_u32(smem_raw), base = (raw_base + 1023u) & ~1023u;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  auto bar = [&](unsigned long long& p) { return smem_u32(&p); };
  if (threadIdx.x == 32) prefetch_tensormap(&x_map);
  if (threadIdx.x < 8) {
    const int i = threadIdx.x;
    if (i < kRawStages) {
      mbar_init(bar(misc.raw_full[i]), 1);
      mbar_init(bar(misc.raw_empty[i]), kExpandThreads / 32);
    }
    mbar_init(bar(misc.b_full[i]), 1);
    mbar_init(bar(misc.b_empty[i]), 1);
    mbar_init(bar(misc.a_full[i]), 4);
    mbar_init(bar(misc.a_empty[i]), 1);
    if (i == 0) {
      mbar_init(bar(misc.done), 1);
      misc.failed = 0;
    }
    mbar_fence_init();
  }
  if (warp == 2) tmem_alloc(smem_u32(&misc.tmem_base), C::kAlloc);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = misc.tmem_base;
  const int rank = a.splits > 1 ? (int)blockIdx.x % a.splits : 0, tile = (int)blockIdx.x / a.splits;
  const int kbs = a.s.in_blocks(), ob0 = tile * 8, obs = min(8, a.s.out_blocks() - ob0);
  const int kb0 = (int)((long long)kbs * rank / a.splits), n_kb = (int)((long long)kbs * (rank + 1) / a.splits) - kb0;
  grid_launch_dependents();
  // The first weights come into L2 while the work in front of this launch ends (a request, no access): 64 rows of
  // 4096 x 6720 12.8 -> 12.2 us in a row of calls.  A CTA's whole share asked for at once stands in the way of what is
  // loaded now (128 rows of 8192 x 8192: 21.5 us for 21.0).
  const uint8_t* const my_blocks = a.packed + ((long long)(ob0 + min(lane, obs - 1)) * kbs + kb0) * kBlockBytes;
  if (warp == 3 && lane < obs && blockIdx.y == 0) prefetch_l2(my_blocks, min(n_kb, 8) * kBlockBytes);
  grid_dependency_wait();

  const int n0 = blockIdx.y * BN, n_units = 2 * n_kb;              // of 64 inputs
  const uint32_t raw_u32 = base + C::kPanels;
  constexpr uint32_t CYCLES = RUN_OUT ? 1u << 21 : 0x7fffffffu;
  auto wait = [&](unsigned long long& b, int phase) { return mbar_wait_compact<CYCLES>(bar(b), phase & 1); };
  auto wait_warp = [&](unsigned long long& b, int phase) { return mbar_wait_eager<32, CYCLES>(bar(b), phase & 1); };
  bool ok = true;                    // false once a wait of this thread has given up

  if (warp == 0) {
    // ---------------------------------------------------------------- rows of x
    if (lane == 0 && !RUN_OUT) {
      for (int u = 0; u < n_units && ok; ++u) {
        const int st = u % C::kStages;
        ok = wait(misc.b_empty[st], u / C::kStages + 1);
        if (!ok) break;
        mbar_arrive_expect_tx(bar(misc.b_full[st]), C::kPanel);
        tma_load_2d(base + st * C::kPanel, &x_map, bar(misc.b_full[st]), kb0 * kInputs + u * 64, n0);
      }
    }
  } else if (warp == 3) {
    // ---------------------------------------------------------------- weights: a lane per block of outputs
    const uint8_t* src = my_blocks;
    int st = 0, round = 0;
    for (int kb = 0; kb < n_kb && ok; ++kb, src += kBlockBytes) {
      ok = wait_warp(misc.raw_empty[st], round + 1);
      if (!ok) break;
      const uint32_t full = bar(misc.raw_full[st]);
      if (lane == 0) mbar_arrive_expect_tx(full, obs * kBlockBytes);
      __syncwarp();
      if (lane < obs) bulk_load(raw_u32 + st * C::kRaw + lane * kBlockBytes, src, kBlockBytes, full);
      if (++st == kRawStages) { st = 0; ++round; }
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------------- issuer (whole warp, uniform)
    const uint64_t b_desc = make_smem_desc(base, 16, 1024, kSwizzle128B);
    int st = 0, st_round = 0, buf = 0, buf_round = 0;
    bool there = false;              // the next unit, asked for before the instructions in front of it are issued
    for (int u = 0; u < n_units && ok; ++u) {
      ok = wait_warp(misc.b_full[st], st_round);
      if (!ok) break;
      const uint32_t panel = (uint32_t)b_desc + st * (C::kPanel / 16), hi = (uint32_t)(b_desc >> 32);
      ok = __all_sync(0xffffffffu, there) || wait_warp(misc.a_full[buf], buf_round);
      if (!ok) break;
      tc_fence_after_sync();
      const uint32_t at = tmem + BN + buf * 32, empty = bar(misc.a_empty[buf]);
      if (++buf == C::kUnits) { buf = 0; ++buf_round; }
      there = mbar_test(bar(misc.a_full[buf]), buf_round & 1);
      if (elect_one()) {
        mma_f16_ts(tmem, at, panel, hi, IDESC, u > 0);
#pragma unroll
        for (int i = 1; i < 4; ++i) mma_f16_ts(tmem, at + i * 8, panel + i * 2, hi, IDESC, 1u);
        mma_commit(empty);
        mma_commit(bar(misc.b_empty[st]));
      }
      __syncwarp();
      if (++st == C::kStages) { st = 0; ++st_round; }
    }
    if (ok && elect_one()) mma_commit(bar(misc.done));
    __syncwarp();
  } else if (warp >= kExpandWarp0) {
    // ---------------------------------------------------------------- expansion
    // Group grp has half grp of every block.
    const int q = warp & 3, grp = (warp - kExpandWarp0) >> 2, o = q * 32 + lane, i = o & 15;
    const uint32_t block = raw_u32 + (o >> 4) * kBlockBytes;
    const uint32_t twist = (uint32_t)(i >> 1 & 3) * 16, row = block + i * 64;
    const uint32_t chunk0 = (uint32_t)(grp * 32) ^ twist, chunk1 = (uint32_t)(grp * 32 + 16) ^ twist;
    const uint32_t scales = block + kCodeBytes + 8 * (i & 7) + (i >> 3) + 4 * grp;
    const uint32_t lane_tm = tmem + ((uint32_t)(q * 32) << 16) + BN;
    // A unit's bytes are read while the one before is waiting for its buffer.
    int st = 0, round = 0;
    uint4 w0, w1;
    uint32_t b0, b1;
    auto read = [&]() {
      ok = wait_warp(misc.raw_full[st], round);
      if (!ok) return;
      const uint32_t at = st * C::kRaw;
      w0 = qp::lds128(row + at + chunk0);
      w1 = qp::lds128(row + at + chunk1);
      b0 = qp::lds_u8(scales + at);
      b1 = qp::lds_u8(scales + at + 2);
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(misc.raw_empty[st]));
      if (++st == kRawStages) { st = 0; ++round; }
    };
    read();
#pragma unroll 1
    for (int kb = 0; kb < n_kb && ok; ++kb) {
      const int k = 2 * kb + grp, buf = k % C::kUnits;       // the unit's number and buffer
      const uint32_t s0 = scale_b2(b0), s1 = scale_b2(b1);
      const uint32_t word[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
      uint32_t x[32];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        uint32_t r[4];
        decode8(word[e], r);
#pragma unroll
        for (int m = 0; m < 4; ++m) x[4 * e + m] = mul_b2(r[m], e < 4 ? s0 : s1);
      }
      if (kb + 1 < n_kb) {
        read();
        if (!ok) break;
      }
      if (k >= C::kUnits) {
        ok = wait_warp(misc.a_empty[buf], k / C::kUnits + 1);
        if (!ok) break;
        tc_fence_after_sync();
      }
      tmem_st_x32(lane_tm + buf * 32, x);
      tmem_wait_st();
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(misc.a_full[buf]));
    }
    if (ok) ok = wait(misc.done, 0);
    ok = __all_sync(0xffffffffu, ok);
    if (!ok) misc.failed = 1;
    named_sync<1, kExpandThreads>();
    const bool failed = *reinterpret_cast<volatile int*>(&misc.failed) != 0;
    tc_fence_after_sync();
    // ---------------------------------------------------------------- results: lane = output, columns = rows of x
    for (int c0 = 32 * grp; c0 < BN; c0 += 32 * kGroups) {
      uint32_t v[32];
      tmem_ld_x32(tmem + ((uint32_t)(q * 32) << 16) + c0, v);
      tmem_wait_ld();
      if (a.splits > 1) {
        float* sums = reinterpret_cast<float*>(smem_raw + (base - raw_base)) + (long long)c0 * kTile + o;
#pragma unroll
        for (int j = 0; j < 32; ++j) sums[j * kTile] = __uint_as_float(v[j]);
      } else {
        const int out = ob0 * kRows + o, n = n0 + c0;
        const float unit = failed ? NAN : kUnit;
        if (a.pairs) {
          // Two outputs a lane: neighbours exchange, the even one has row n + j, the odd one the next.
          const bool odd = lane & 1;
          bf16* dst = a.y + (n + odd) * a.y_stride + (out & ~1);
#pragma unroll
          for (int j = 0; j < 32; j += 2, dst += 2 * a.y_stride) {
            const float mine = __uint_as_float(odd ? v[j + 1] : v[j]);
            const float got = __shfl_xor_sync(0xffffffffu, __uint_as_float(odd ? v[j] : v[j + 1]), 1);
            const __nv_bfloat162 two = __floats2bfloat162_rn((odd ? got : mine) * unit, (odd ? mine : got) * unit);
            if ((out | 1) < a.s.n_out && n + j + odd < a.n) *reinterpret_cast<__nv_bfloat162*>(dst) = two;
          }
        } else if (out < a.s.n_out) {
          bf16* dst = a.y + n * a.y_stride + out;
#pragma unroll
          for (int j = 0; j < 32; ++j, dst += a.y_stride)
            if (n + j < a.n) *dst = __float2bfloat16_rn(__uint_as_float(v[j]) * unit);
        }
      }
    }
    tc_fence_before_sync();
  }
  if (!ok) misc.failed = 1;
  __syncwarp();
  if (a.splits > 1) {
    cluster_sync();
    // This CTA's share of the columns: all CTAs' sums in rank order.
    const int lo = BN * rank / a.splits, hi = BN * (rank + 1) / a.splits;
    bool failed = false;
    for (int s = 0; s < a.splits; ++s) failed |= load_cluster(smem_u32(&misc.failed), s) != 0;
    for (int e = (lo * kTile + 4 * threadIdx.x); e < hi * kTile; e += 4 * kThreads) {
      float4 v[8];
#pragma unroll
      for (int s = 0; s < 8; ++s)
        if (s < a.splits) v[s] = load_cluster4(base + e * 4, s);
      float4 sum = v[0];
#pragma unroll
      for (int s = 1; s < 8; ++s)
        if (s < a.splits) { sum.x += v[s].x; sum.y += v[s].y; sum.z += v[s].z; sum.w += v[s].w; }
      const int out = ob0 * kRows + e % kTile, n = n0 + e / kTile;
      if (n >= a.n) continue;
      const float unit = failed ? NAN : kUnit, y[4] = {sum.x * unit, sum.y * unit, sum.z * unit, sum.w * unit};
      bf16* dst = a.y + n * a.y_stride + out;
      if (a.pairs && out + 3 < a.s.n_out) {
        reinterpret_cast<__nv_bfloat162*>(dst)[0] = __floats2bfloat162_rn(y[0], y[1]);
        reinterpret_cast<__nv_bfloat162*>(dst)[1] = __floats2bfloat162_rn(y[2], y[3]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (out + i < a.s.n_out) dst[i] = __float2bfloat16_rn(y[i]);
      }
    }
    __syncwarp();
    cluster_sync();                                          // the sums are read by others until here
  }
  __syncthreads();
  if (*reinterpret_cast<volatile int*>(&misc.failed)) {
    // Give copies that may still be in flight time to land before the CTA's memory is reused.
    const uint64_t t0 = global_timer_ns();
    while (global_timer_ns() - t0 < 100000ull) __nanosleep(1000);
  }
  if (warp == 2) {
    __syncwarp();
    tc_fence_after_sync();
    tmem_dealloc(tmem, C::kAlloc);
  }
}

}  // namespace tc
}  // namespace qw
}  // namespace mtla
