// The scaled matrix instruction on 4-bit operands, and what a product leaves.
#pragma once

#include "mx4.hpp"
#include "mx4_dev.hpp"

namespace vsk {

// D(16x16, f32) += A(16x128) * B(128x16) in 4 bits, one exponent a lane: lane l
// feeds row (column) l % 16, columns (rows) 32 (l / 16) .. + 31; byte SA of sa and
// SB of sb hold the exponents.
template <int SA, int SB>
__device__ __forceinline__ f32x4 mfma_mx4(u32x4 a, u32x4 b, f32x4 c, uint32_t sa, uint32_t sb) {
  const i32x8 av = {static_cast<int>(a[0]), static_cast<int>(a[1]), static_cast<int>(a[2]), static_cast<int>(a[3]), 0, 0, 0, 0};
  const i32x8 bv = {static_cast<int>(b[0]), static_cast<int>(b[1]), static_cast<int>(b[2]), static_cast<int>(b[3]), 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, bv, c, 4, 4, SA, static_cast<int>(sa), SB, static_cast<int>(sb));
}

// D(32x32, f32) += A(32x64) * B(64x32): lane l feeds row (column) l % 32, columns
// (rows) 32 (l / 32) .. + 31, and holds D[8 (r / 4) + 4 (l / 32) + r % 4][l % 32] in r.
template <int SA, int SB>
__device__ __forceinline__ f32x16 mfma_mx4_32(u32x4 a, u32x4 b, f32x16 c, uint32_t sa, uint32_t sb) {
  const i32x8 av = {static_cast<int>(a[0]), static_cast<int>(a[1]), static_cast<int>(a[2]), static_cast<int>(a[3]), 0, 0, 0, 0};
  const i32x8 bv = {static_cast<int>(b[0]), static_cast<int>(b[1]), static_cast<int>(b[2]), static_cast<int>(b[3]), 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(av, bv, c, 4, 4, SA, static_cast<int>(sa), SB, static_cast<int>(sb));
}

// Behind a workgroup's write-through stores of its part of K: whether it is the last
// of its tile's to have come this far (the others' stores are in memory then; nobody
// waits, see attn_unit).
__device__ __forceinline__ bool mx4_last_of(const Mx4Split& sp, int tile, int& s_last) {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  if (threadIdx.x == 0)
    s_last = __hip_atomic_fetch_add(sp.counter + tile, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == sp.splits - 1;
  __syncthreads();
  return s_last != 0;
}

// y[row][c0 .. c0 + 3] (+ add) from float32 sums, rounded once.  Vectors need no more
// than their elements' alignment: 3,001 x 30,001 x 200, whose rows have no other, 283 us
// with a store an element, 95 so.
typedef f32x4 __attribute__((aligned(4))) Fp32x4;
typedef u32x2 __attribute__((aligned(2))) Bf16x4;
typedef u32x4 __attribute__((aligned(2))) Bf16x8;
__device__ __forceinline__ void mx4_store4(const Mx4ProductArgs& a, int row, int c0, f32x4 v) {
  const int64_t at = row * a.y_stride + c0;
  if (c0 + 3 < a.n) {
    if (a.y_fp32) {
      if (a.add != nullptr) v += *reinterpret_cast<const Fp32x4*>(static_cast<const float*>(a.add) + at);
      *reinterpret_cast<Fp32x4*>(static_cast<float*>(a.y) + at) = v;
    } else {
      if (a.add != nullptr) {
        const u32x2 x = *reinterpret_cast<const Bf16x4*>(static_cast<const uint16_t*>(a.add) + at);
        v += f32x4{bf2f(x[0] & 0xffffu), __uint_as_float(x[0] & 0xffff0000u), bf2f(x[1] & 0xffffu), __uint_as_float(x[1] & 0xffff0000u)};
      }
      *reinterpret_cast<Bf16x4*>(static_cast<uint16_t*>(a.y) + at) = u32x2{pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3])};
    }
    return;
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    if (c0 + r >= a.n) continue;
    float x = v[r];
    if (a.y_fp32) {
      if (a.add != nullptr) x += static_cast<const float*>(a.add)[at + r];
      static_cast<float*>(a.y)[at + r] = x;
    } else {
      if (a.add != nullptr) x += bf2f(static_cast<const uint16_t*>(a.add)[at + r]);
      static_cast<uint16_t*>(a.y)[at + r] = static_cast<uint16_t>(f2bf(x));
    }
  }
}

// The same of eight columns.
__device__ __forceinline__ void mx4_store8(const Mx4ProductArgs& a, int row, int c0, f32x4 lo, f32x4 up) {
  if (a.add == nullptr && !a.y_fp32 && c0 + 7 < a.n) {
    *reinterpret_cast<Bf16x8*>(static_cast<uint16_t*>(a.y) + row * a.y_stride + c0) =
        u32x4{pack_bf2(lo[0], lo[1]), pack_bf2(lo[2], lo[3]), pack_bf2(up[0], up[1]), pack_bf2(up[2], up[3])};
    return;
  }
  mx4_store4(a, row, c0, lo);
  mx4_store4(a, row, c0 + 4, up);
}

}  // namespace vsk
