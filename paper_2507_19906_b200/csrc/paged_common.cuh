// Device helpers of the kernels over a cache in pages: 16-bit types, TMA copies of page boxes.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"
#include "paged.h"
#include "tc_common.cuh"

namespace calidrop {

// P is rounded to the type of V for the product P V.  In fp16 the probabilities are kept 2^kBias higher than their sum's
// reference says, so that small ones keep their bits (a probability of 2^-14 of the largest would be subnormal); in bf16 there is
// nothing to gain.
template <bool kF16>
__device__ __forceinline__ uint32_t pack16(float a, float b) {
  if constexpr (kF16) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    return pack_bf16(a, b);
  }
}
template <bool kF16>
__device__ __forceinline__ float2 unpack16(uint32_t x) {
  if constexpr (kF16) return __half22float2(*reinterpret_cast<__half2*>(&x));
  else return make_float2(bf16_lo(x), bf16_hi(x));
}

// D(16x8, f32) += A(16x16, row) * B(16x8, col) in either type
template <bool kF16>
__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
  if constexpr (kF16) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  } else {
    mma_bf16_16816(c, a0, a1, a2, a3, b0, b1);
  }
}

__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2, int c3,
                                            int c4, uint64_t pol) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint "
      "[%0], [%1, {%3, %4, %5, %6, %7}], [%2], %8;"
      ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4), "l"(pol)
      : "memory");
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Whether a wait of this CTA has run out (one thread says so in the workspace): by a bit of its own, since the word may hold those of
// bad data already.
__device__ __forceinline__ bool paged_aborted(const tc::Ctl& ctl) {
  if (!ctl.abort) return false;
  if (threadIdx.x == 0) atomicOr(ctl.status, kWaitRanOut);
  return true;
}

// 16 consecutive fp32 columns of this thread's lane of tensor memory (see tc::tmem_ld32).
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
      "tcgen05.wait::ld.sync.aligned;\n"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}

// The first eight of 16 values to as many columns of this thread's lane.
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};\n" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}

// 64 fp32 columns of 16 lanes of tensor memory, a lane's columns spread over four threads: thread t has of lane t / 4 (and t / 4 + 8)
// columns 8 c + 2 (t % 4) and the next one in r[4 c], r[4 c + 1] (and r[4 c + 2], r[4 c + 3]), c = 0..7.
__device__ __forceinline__ void tmem_ld_16x64(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x8.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
      "tcgen05.wait::ld.sync.aligned;\n"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}

// Thread q of a quad gives v[c] to thread c and has the values of threads 0..3 for itself.
__device__ __forceinline__ uint4 quad_transpose(const uint32_t (&v)[4], int lane) {
  const bool odd = lane & 1, up = lane & 2;
  const uint32_t x0 = __shfl_xor_sync(0xffffffffu, odd ? v[0] : v[1], 1), x1 = __shfl_xor_sync(0xffffffffu, odd ? v[2] : v[3], 1);
  const uint32_t a0 = odd ? x0 : v[0], a1 = odd ? v[1] : x0;     // value (q & 1) of threads q & 2 and the next
  const uint32_t b0 = odd ? x1 : v[2], b1 = odd ? v[3] : x1;     // value (q & 1) + 2
  const uint32_t y0 = __shfl_xor_sync(0xffffffffu, up ? a0 : b0, 2), y1 = __shfl_xor_sync(0xffffffffu, up ? a1 : b1, 2);
  return up ? make_uint4(y0, y1, b0, b1) : make_uint4(a0, a1, y0, y1);
}

// Rows [0, kv) of a sequence that a query at its last position sees, in blocks of 2^kLg rows: near_blocks from the first on,
// then those from `first` on.
struct PagedView {
  int kv, lo;            // rows at and beyond lo are inside the window
  int near_blocks, first, n_blocks;
  __device__ __forceinline__ int block(int j) const { return j < near_blocks ? j : j - near_blocks + first; }
};
template <int kLg>
__device__ __forceinline__ PagedView paged_view(int kv, int window, int n_sink) {
  PagedView v;
  v.kv = kv;
  v.lo = window && kv > window ? kv - window : 0;
  const int blocks = (kv + (1 << kLg) - 1) >> kLg;
  v.first = v.lo >> kLg;
  // (in 64 bits: n_sink may be anything)
  const int sink_blocks = (int)min((long long)v.first, ((long long)n_sink + (1 << kLg) - 1) >> kLg);
  v.near_blocks = sink_blocks;
  v.n_blocks = max(1, sink_blocks + blocks - v.first);   // (a sequence without rows has one block, of which nothing is visible)
  return v;
}

// Four outputs of a partial softmax, its maximum (or whatever its terms are relative to) and its sum, all in the log2 domain.
struct Partial {
  float o[4], m, l;
  __device__ __forceinline__ void clear() { o[0] = o[1] = o[2] = o[3] = 0.f; m = -INFINITY; l = 0.f; }
  __device__ __forceinline__ void join(float m2, float l2, const float4& o2) {
    const float mn = fmaxf(m, m2), ref = mn == -INFINITY ? 0.f : mn;
    const float f1 = ex2_approx(m - ref), f2 = ex2_approx(m2 - ref);
    l = l * f1 + l2 * f2;
    o[0] = o[0] * f1 + o2.x * f2; o[1] = o[1] * f1 + o2.y * f2;
    o[2] = o[2] * f1 + o2.z * f2; o[3] = o[3] * f1 + o2.w * f2;
    m = mn;
  }
};

// Rows `row(i)` of n partial rows of kStride floats, this lane's four outputs of each, joined in order.
template <typename Row>
__device__ __forceinline__ void join_rows(Partial& p, int n, int lane, Row row) {
  constexpr int kBatch = 8;   // loads in flight
  for (int i0 = 0; i0 < n; i0 += kBatch) {
    float4 o[kBatch];
    float2 ml[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const float* r = row(min(i0 + i, n - 1));
      o[i] = __ldcg(reinterpret_cast<const float4*>(r) + lane);
      ml[i] = __ldcg(reinterpret_cast<const float2*>(r + kD));
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      if (i0 + i < n) p.join(ml[i].x, ml[i].y, o[i]);
  }
}

}  // namespace calidrop
