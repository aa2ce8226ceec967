// Microscaled 4-bit matrices: quantisation, packing, reading back, and the product
// with a weight matrix on v_mfma_scale_f32_16x16x128_f8f6f4.
#include <algorithm>

#include "mx4_mma.hpp"

namespace vsk {

// ------------------------------------------------------------------ quantisation
// A block (32 values of a row) a thread, a tile (16 rows x 4 blocks) a wave, so
// that a tile's codes are one contiguous store.  VEC: rows are 16-byte aligned
// and k a multiple of 32.  Bound by memory: 2 (4) bytes a value read, 17/32
// written.
template <bool FP32, bool VEC>
__global__ __launch_bounds__(256) void k_mx4_quantise(const void* __restrict__ src, int64_t stride, int rows, int k,
                                                      uint8_t* __restrict__ mx, int kt_n, int n_tiles, size_t scales_at) {
  const int lane = threadIdx.x & 63;
  const int tile = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (tile >= n_tiles) return;
  const int rt = tile / kt_n, kt = tile - rt * kt_n;
  const int row = 16 * rt + (lane & 15), k0 = 128 * kt + 32 * (lane >> 4);
  const int cnt = row < rows ? min(32, max(0, k - k0)) : 0;
  u32x4 codes = u32x4{0u, 0u, 0u, 0u};
  uint32_t e = 0;
  const int64_t at = row * stride + k0;
  if constexpr (FP32) {
    float v[32];
    uint32_t top = 0;
    const float* p = static_cast<const float*>(src) + at;
#pragma unroll
    for (int i = 0; i < 32; i += 4) {
      if constexpr (VEC) {
        const f32x4 x = cnt > 0 ? *reinterpret_cast<const f32x4*>(p + i) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i + j] = x[j];
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i + j] = i + j < cnt ? p[i + j] : 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < 32; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
    e = mx4_exponent(top);
    const float sc = mx4_scale(e);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t c = mx4_encode_f32<0>(0u, v[8 * j], v[8 * j + 1], sc);
      c = mx4_encode_f32<1>(c, v[8 * j + 2], v[8 * j + 3], sc);
      c = mx4_encode_f32<2>(c, v[8 * j + 4], v[8 * j + 5], sc);
      codes[j] = mx4_encode_f32<3>(c, v[8 * j + 6], v[8 * j + 7], sc);
    }
  } else {
    uint32_t v[16];
    uint32_t top = 0;
    const uint16_t* p = static_cast<const uint16_t*>(src) + at;
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      if constexpr (VEC) {
        const u32x4 x = cnt > 0 ? *reinterpret_cast<const u32x4*>(p + 2 * i) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i + j] = x[j];
      } else {
#pragma unroll
        for (int j = i; j < i + 4; ++j)
          v[j] = (2 * j < cnt ? p[2 * j] : 0u) | (2 * j + 1 < cnt ? static_cast<uint32_t>(p[2 * j + 1]) : 0u) << 16;
      }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) top = mx4_top2(top, v[i] & 0x7fff7fffu);
    e = mx4_exponent(mx4_top(top));
    const float sc = mx4_scale(e);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t c = mx4_encode_bf16<0>(0u, v[4 * j], sc);
      c = mx4_encode_bf16<1>(c, v[4 * j + 1], sc);
      c = mx4_encode_bf16<2>(c, v[4 * j + 2], sc);
      codes[j] = mx4_encode_bf16<3>(c, v[4 * j + 3], sc);
    }
  }
  if (e == 255u) codes = u32x4{0u, 0u, 0u, 0u};
  *reinterpret_cast<u32x4*>(mx + (static_cast<size_t>(tile) * 64 + lane) * 16) = codes;
  const int kq_n = (kt_n + 3) / 4;
  uint8_t* sp = mx + scales_at + ((static_cast<size_t>(rt) * kq_n + kt / 4) * 64 + lane) * 4;
  sp[kt & 3] = static_cast<uint8_t>(e);
  // (the last tile of a row of tiles fills up its four)
  if (kt == kt_n - 1)
    for (int j = (kt & 3) + 1; j < 4; ++j) sp[j] = 0;
}

// Codes [rows][ceil(k / 2)] and exponents [rows][ceil(k / 32)] as files hold them.
__global__ __launch_bounds__(256) void k_mx4_pack(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                  int rows, int k, uint8_t* __restrict__ mx, int kt_n, int n_tiles,
                                                  size_t scales_at) {
  const int lane = threadIdx.x & 63;
  const int tile = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (tile >= n_tiles) return;
  const int rt = tile / kt_n, kt = tile - rt * kt_n;
  const int row = 16 * rt + (lane & 15), k0 = 128 * kt + 32 * (lane >> 4);
  const int cnt = row < rows ? min(32, max(0, k - k0)) : 0;
  u32x4 c = u32x4{0u, 0u, 0u, 0u};
  uint32_t e = 0;
  if (cnt > 0) {
    const uint8_t* p = codes + static_cast<size_t>(row) * ((k + 1) / 2) + k0 / 2;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      uint32_t b = 2 * i < cnt ? p[i] : 0u;
      if (2 * i + 1 >= cnt) b &= 15u;  // (an odd row's last byte holds one value)
      c[i >> 2] |= b << (8 * (i & 3));
    }
    e = scales[static_cast<size_t>(row) * ((k + 31) / 32) + k0 / 32];
  }
  *reinterpret_cast<u32x4*>(mx + (static_cast<size_t>(tile) * 64 + lane) * 16) = c;
  const int kq_n = (kt_n + 3) / 4;
  uint8_t* sp = mx + scales_at + ((static_cast<size_t>(rt) * kq_n + kt / 4) * 64 + lane) * 4;
  sp[kt & 3] = static_cast<uint8_t>(e);
  if (kt == kt_n - 1)
    for (int j = (kt & 3) + 1; j < 4; ++j) sp[j] = 0;
}

// The values a matrix stands for (exact in bf16), a block a thread.
template <bool FP32, bool VEC>
__global__ __launch_bounds__(256) void k_mx4_read(const uint8_t* __restrict__ mx, int rows, int k, void* __restrict__ dst,
                                                  int64_t stride, int kt_n, int n_tiles, size_t scales_at) {
  const int lane = threadIdx.x & 63;
  const int tile = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (tile >= n_tiles) return;
  const int rt = tile / kt_n, kt = tile - rt * kt_n;
  const int row = 16 * rt + (lane & 15), k0 = 128 * kt + 32 * (lane >> 4);
  const int cnt = row < rows ? min(32, max(0, k - k0)) : 0;
  if (cnt == 0) return;
  const u32x4 codes = *reinterpret_cast<const u32x4*>(mx + (static_cast<size_t>(tile) * 64 + lane) * 16);
  const int kq_n = (kt_n + 3) / 4;
  const float sc = mx4_scale(mx[scales_at + ((static_cast<size_t>(rt) * kq_n + kt / 4) * 64 + lane) * 4 + (kt & 3)]);
  const int64_t at = row * stride + k0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const u32x4 v = mx4_decode8(codes[j], sc);
    if constexpr (FP32) {
      float* p = static_cast<float*>(dst) + at + 8 * j;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (8 * j + i < cnt) p[i] = i & 1 ? __uint_as_float(v[i >> 1] & 0xffff0000u) : __uint_as_float(v[i >> 1] << 16);
    } else {
      uint16_t* p = static_cast<uint16_t*>(dst) + at + 8 * j;
      if constexpr (VEC) {
        *reinterpret_cast<u32x4*>(p) = v;
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (8 * j + i < cnt) p[i] = static_cast<uint16_t>(v[i >> 1] >> (16 * (i & 1)));
      }
    }
  }
}

static bool rows_aligned(const void* p, int64_t stride, int k, int size) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * size % 16 == 0 && k % 32 == 0;
}

hipError_t launch_mx4_quantise(const void* src, int dtype, int64_t stride, int rows, int k, uint8_t* mx, hipStream_t s) {
  const Mx4Shape g(rows, k);
  const int n = static_cast<int>(g.rt * g.kt);
  const dim3 grid((n + 3) / 4), block(256);
  const bool fp32 = dtype == kMxFp32, vec = rows_aligned(src, stride, k, fp32 ? 4 : 2);
  auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, block, 0, s, src, stride, rows, k, mx, static_cast<int>(g.kt), n, g.scales_at()); };
  if (fp32) vec ? go(k_mx4_quantise<true, true>) : go(k_mx4_quantise<true, false>);
  else vec ? go(k_mx4_quantise<false, true>) : go(k_mx4_quantise<false, false>);
  return hipGetLastError();
}

hipError_t launch_mx4_pack(const uint8_t* codes, const uint8_t* scales, int rows, int k, uint8_t* mx, hipStream_t s) {
  const Mx4Shape g(rows, k);
  const int n = static_cast<int>(g.rt * g.kt);
  hipLaunchKernelGGL(k_mx4_pack, dim3((n + 3) / 4), dim3(256), 0, s, codes, scales, rows, k, mx, static_cast<int>(g.kt), n,
                     g.scales_at());
  return hipGetLastError();
}

hipError_t launch_mx4_read(const uint8_t* mx, int rows, int k, void* dst, int dtype, int64_t stride, hipStream_t s) {
  const Mx4Shape g(rows, k);
  const int n = static_cast<int>(g.rt * g.kt);
  const bool fp32 = dtype == kMxFp32, vec = rows_aligned(dst, stride, k, 2);
  auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3((n + 3) / 4), dim3(256), 0, s, mx, rows, k, dst, stride, static_cast<int>(g.kt), n, g.scales_at()); };
  if (fp32) go(k_mx4_read<true, false>);
  else vec ? go(k_mx4_read<false, true>) : go(k_mx4_read<false, false>);
  return hipGetLastError();
}

// ------------------------------------------------------------------ product
// Weights streamed: a workgroup takes 16 columns and up to 16 RG rows, its eight
// waves an eighth of K each; their sums are added in wave order.
constexpr int kMxWaves = 8;
template <int RG>
__global__ __launch_bounds__(64 * kMxWaves) void k_mx4_stream(Mx4ProductArgs a) {
  __shared__ f32x4 part[kMxWaves][RG][64];
  const Mx4Shape gw(a.n, a.k), gx(a.rows, a.k);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int nt = blockIdx.x, g0 = blockIdx.y * RG;
  const int kt_n = static_cast<int>(gw.kt), kq_n = static_cast<int>(gw.kq);
  const int groups = min(RG, static_cast<int>(gx.rt) - g0);
  const u32x4* wp = reinterpret_cast<const u32x4*>(a.w) + static_cast<size_t>(nt) * kt_n * 64 + lane;
  const uint32_t* ws = reinterpret_cast<const uint32_t*>(a.w + gw.scales_at()) + static_cast<size_t>(nt) * kq_n * 64 + lane;
  const u32x4* xp = reinterpret_cast<const u32x4*>(a.x) + static_cast<size_t>(g0) * kt_n * 64 + lane;
  const uint32_t* xs = reinterpret_cast<const uint32_t*>(a.x + gx.scales_at()) + static_cast<size_t>(g0) * kq_n * 64 + lane;
  f32x4 acc[RG];
#pragma unroll
  for (int g = 0; g < RG; ++g) acc[g] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int q = w; q < kq_n; q += kMxWaves) {
    const int left = min(4, kt_n - 4 * q);
    const uint32_t sw = ws[static_cast<size_t>(q) * 64];
    uint32_t sx[RG];
#pragma unroll
    for (int g = 0; g < RG; ++g) sx[g] = xs[(static_cast<size_t>(min(g, groups - 1)) * kq_n + q) * 64];
    auto one = [&](auto jc) {
      constexpr int J = decltype(jc)::value;
      if (J >= left) return;
      const size_t kt = 4 * static_cast<size_t>(q) + J;
      const u32x4 wv = wp[kt * 64];
#pragma unroll
      for (int g = 0; g < RG; ++g) {
        const u32x4 xv = xp[(static_cast<size_t>(min(g, groups - 1)) * kt_n + kt) * 64];
        acc[g] = mfma_mx4<J, J>(wv, xv, acc[g], sw, sx[g]);
      }
    };
    one(std::integral_constant<int, 0>{});
    one(std::integral_constant<int, 1>{});
    one(std::integral_constant<int, 2>{});
    one(std::integral_constant<int, 3>{});
  }
#pragma unroll
  for (int g = 0; g < RG; ++g) part[w][g][lane] = acc[g];
  __syncthreads();
  // (the lane holds columns 16 nt + 4 (lane / 16) + r of row lane % 16)
  for (int g = w; g < groups; g += kMxWaves) {
    f32x4 y = part[0][g][lane];
#pragma unroll
    for (int i = 1; i < kMxWaves; ++i) y += part[i][g][lane];
    const int row = 16 * (g0 + g) + (lane & 15), c0 = 16 * nt + 4 * (lane >> 4);
    if (row < a.rows) mx4_store4(a, row, c0, y);
  }
}

hipError_t launch_mx4_product(const Mx4ProductArgs& a, hipStream_t s) {
  const int nt = (a.n + 15) / 16, rg = (a.rows + 15) / 16;
  if (rg > 8) return launch_mx4_tile(a, s);
  if (rg <= 1) hipLaunchKernelGGL((k_mx4_stream<1>), dim3(nt, 1), dim3(64 * kMxWaves), 0, s, a);
  else hipLaunchKernelGGL((k_mx4_stream<4>), dim3(nt, (rg + 3) / 4), dim3(64 * kMxWaves), 0, s, a);
  return hipGetLastError();
}

}  // namespace vsk
