// Microscaled 4-bit matrices: quantisation, packing, reading back, and the product
// with a weight matrix on v_mfma_scale_f32_16x16x128_f8f6f4.
#include <algorithm>

#include "mx4_mma.hpp"

namespace vsk {

// ------------------------------------------------------------------ quantisation
// Eight values of a row in registers, a quarter of a block, four lanes a block: a
// load of a wave then takes whole lines (4 rows x 256 bytes in bf16; with a block a
// lane it touched 64 of them: 16 x 11008 by every workgroup of a product took 9 us).
// WIDE: p is 16-byte aligned and cnt 8 or 0; cnt values count, the others as zero.
__device__ __forceinline__ uint32_t max_of_quad(uint32_t v) {
  v = max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), 0xb1, 0xf, 0xf, true)));  // lane ^ 1
  return max(v, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), 0x4e, 0xf, 0xf, true)));  // lane ^ 2
}
template <bool FP32>
using Mx4Elem = std::conditional_t<FP32, float, uint16_t>;
template <bool FP32>
struct Mx4Eight {
  u32x4 v[FP32 ? 2 : 1];
  template <bool WIDE>
  __device__ __forceinline__ void load(const Mx4Elem<FP32>* p, int cnt) {
    if constexpr (WIDE) {
#pragma unroll
      for (int i = 0; i < (FP32 ? 2 : 1); ++i) v[i] = cnt > 0 ? reinterpret_cast<const u32x4*>(p)[i] : u32x4{0u, 0u, 0u, 0u};
    } else if (cnt == 8) {  // (in vectors of no more than the elements' alignment)
      if constexpr (FP32) {
#pragma unroll
        for (int i = 0; i < 2; ++i) v[i] = __builtin_bit_cast(u32x4, static_cast<f32x4>(reinterpret_cast<const Fp32x4*>(p)[i]));
      } else {
        v[0] = *reinterpret_cast<const Bf16x8*>(p);
      }
    } else if constexpr (FP32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i >> 2][i & 3] = i < cnt ? __float_as_uint(p[i]) : 0u;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        v[0][i] = (2 * i < cnt ? p[2 * i] : 0u) | (2 * i + 1 < cnt ? static_cast<uint32_t>(p[2 * i + 1]) : 0u) << 16;
    }
  }
  // the codes, and the block's exponent (on each of its four lanes)
  __device__ __forceinline__ uint32_t encode(uint32_t& e) const {
    uint32_t top = 0, c;
    if constexpr (FP32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, v[i >> 2][i & 3] & 0x7fffffffu);
    } else {
      top = mx4_top(mx4_top2(mx4_top2(v[0][0] & 0x7fff7fffu, v[0][1] & 0x7fff7fffu),
                             mx4_top2(v[0][2] & 0x7fff7fffu, v[0][3] & 0x7fff7fffu)));
    }
    e = mx4_exponent(max_of_quad(top));
    const float sc = mx4_scale(e);
    if constexpr (FP32) {
      auto f = [&](int i) { return __uint_as_float(v[i >> 2][i & 3]); };
      c = mx4_encode_f32<0>(0u, f(0), f(1), sc);
      c = mx4_encode_f32<1>(c, f(2), f(3), sc);
      c = mx4_encode_f32<2>(c, f(4), f(5), sc);
      c = mx4_encode_f32<3>(c, f(6), f(7), sc);
    } else {
      c = mx4_encode_bf16<0>(0u, v[0][0], sc);
      c = mx4_encode_bf16<1>(c, v[0][1], sc);
      c = mx4_encode_bf16<2>(c, v[0][2], sc);
      c = mx4_encode_bf16<3>(c, v[0][3], sc);
    }
    return e == 255u ? 0u : c;
  }
};

// A tile (16 rows x 4 blocks) a wave, four rows at a time.  Bound by memory: 2 (4)
// bytes a value read, 17/32 written.
template <bool FP32, bool WIDE>
__global__ __launch_bounds__(256) void k_mx4_quantise(const void* __restrict__ src, int64_t stride, int rows, int k,
                                                      uint8_t* __restrict__ mx, int kt_n, int n_tiles, size_t scales_at,
                                                      int* __restrict__ counters, int n_counters) {
  for (int i = blockIdx.x * 256 + threadIdx.x; i < n_counters; i += gridDim.x * 256) counters[i] = 0;
  const int lane = threadIdx.x & 63;
  const int tile = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (tile >= n_tiles) return;
  const int rt = tile / kt_n, kt = tile - rt * kt_n;
  const int r0 = lane >> 4, b = lane >> 2 & 3, k0 = 128 * kt + 8 * (lane & 15);
  Mx4Eight<FP32> x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = 16 * rt + 4 * i + r0;
    x[i].template load<WIDE>(static_cast<const Mx4Elem<FP32>*>(src) + row * stride + k0, row < rows ? min(8, max(0, k - k0)) : 0);
  }
  uint32_t* codes = reinterpret_cast<uint32_t*>(mx + static_cast<size_t>(tile) * 1024) + (lane & 3);
  uint8_t* expo = mx + scales_at + ((static_cast<size_t>(rt) * ((kt_n + 3) / 4) + kt / 4) * 64) * 4;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int at = 4 * i + r0 + 16 * b;  // the block's place in the tile
    uint32_t e;
    codes[4 * at] = x[i].encode(e);
    if ((lane & 3) == 0) {
      expo[4 * at + (kt & 3)] = static_cast<uint8_t>(e);
      // (the last tile of a row of tiles fills up its four)
      if (kt == kt_n - 1)
        for (int j = (kt & 3) + 1; j < 4; ++j) expo[4 * at + j] = 0;
    }
  }
}

// Codes [rows][ceil(k / 2)] and exponents [rows][ceil(k / 32)] as files hold them.
// 28,672 x 4,096 24 us (a byte a load 114).
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
    typedef u32x4 __attribute__((aligned(1))) Codes;  // one load, whatever its alignment
    if (cnt == 32) {
      c = *reinterpret_cast<const Codes*>(p);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        uint32_t b = 2 * i < cnt ? p[i] : 0u;
        if (2 * i + 1 >= cnt) b &= 15u;  // (an odd row's last byte holds one value)
        c[i >> 2] |= b << (8 * (i & 3));
      }
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

// The values a matrix stands for (exact in bf16), a tile a wave as in k_mx4_quantise: a
// store takes whole lines (with a block a lane 2049 x 14336 in bf16 took 22.5 us,
// so 12.4).
template <bool FP32>
__global__ __launch_bounds__(256) void k_mx4_read(const uint8_t* __restrict__ mx, int rows, int k, void* __restrict__ dst,
                                                  int64_t stride, int kt_n, int n_tiles, size_t scales_at) {
  const int lane = threadIdx.x & 63;
  const int tile = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (tile >= n_tiles) return;
  const int rt = tile / kt_n, kt = tile - rt * kt_n;
  const int r0 = lane >> 4, b = lane >> 2 & 3, k0 = 128 * kt + 8 * (lane & 15);
  const int cnt = min(8, max(0, k - k0));
  const uint32_t* codes = reinterpret_cast<const uint32_t*>(mx + static_cast<size_t>(tile) * 1024) + (lane & 3);
  const uint8_t* expo = mx + scales_at + ((static_cast<size_t>(rt) * ((kt_n + 3) / 4) + kt / 4) * 64) * 4 + (kt & 3);
  uint32_t c[4], e[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int at = 4 * i + r0 + 16 * b;
    c[i] = codes[4 * at];
    e[i] = expo[4 * at];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = 16 * rt + 4 * i + r0;
    if (row >= rows || cnt == 0) continue;
    const u32x4 v = mx4_decode8(c[i], mx4_scale(e[i]));
    Mx4Elem<FP32>* p = static_cast<Mx4Elem<FP32>*>(dst) + row * stride + k0;
    auto f = [&](int j) { return v[j >> 1] << (j & 1 ? 0 : 16) & 0xffff0000u; };
    if (cnt == 8) {  // (in vectors of no more than the elements' alignment)
      if constexpr (FP32) {
#pragma unroll
        for (int j = 0; j < 8; j += 4)
          *reinterpret_cast<Fp32x4*>(p + j) = __builtin_bit_cast(f32x4, u32x4{f(j), f(j + 1), f(j + 2), f(j + 3)});
      } else {
        *reinterpret_cast<Bf16x8*>(p) = v;
      }
      continue;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (j >= cnt) continue;
      if constexpr (FP32) p[j] = __uint_as_float(f(j));
      else p[j] = static_cast<uint16_t>(f(j) >> 16);
    }
  }
}

// Rows that wide loads and stores of eight values take.
static bool rows_aligned(const void* p, int64_t stride, int k, int size) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * size % 16 == 0 && k % 8 == 0;
}

hipError_t launch_mx4_quantise(const void* src, int dtype, int64_t stride, int rows, int k, uint8_t* mx, int* counters,
                               int n_counters, hipStream_t s) {
  if (counters == nullptr) n_counters = 0;
  const Mx4Shape g(rows, k);
  const int n = static_cast<int>(g.rt * g.kt);
  const dim3 grid((n + 3) / 4), block(256);
  const bool fp32 = dtype == kMxFp32, vec = rows_aligned(src, stride, k, fp32 ? 4 : 2);
  auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, block, 0, s, src, stride, rows, k, mx, static_cast<int>(g.kt), n, g.scales_at(), counters, n_counters); };
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
  auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3((n + 3) / 4), dim3(256), 0, s, mx, rows, k, dst, stride, static_cast<int>(g.kt), n, g.scales_at()); };
  dtype == kMxFp32 ? go(k_mx4_read<true>) : go(k_mx4_read<false>);
  return hipGetLastError();
}

// ------------------------------------------------------------------ product
// Up to four rows as they are: weights streamed.  A workgroup takes 16 columns at a
// time (tiles blockIdx.x, + gridDim.x, ..), its eight waves every eighth four of K's
// steps of 128 columns each; their sums are added in wave order.  Each wave first
// quantises its part of x into LDS, which it alone reads: a launch less.
//
// A four's weights are in flight while the four before is used: two sets of registers
// in turn, loads without a branch around them (behind a branch, or copied from
// register to register, the compiler waits for all of them).
constexpr int kMxWaves = 8;
constexpr int kMxRawRows = 4;    // (16 rows: 16 x 4096 x 4096 7.2 us, quantised by a launch of its own 7.1)
constexpr int kMxResident = 48;  // most steps of K of x in LDS (with two workgroups a compute unit)
template <bool FP32>
__global__ __launch_bounds__(64 * kMxWaves) void k_mx4_stream(Mx4ProductArgs a) {
  __shared__ f32x4 s_part[2][kMxWaves][64];
  extern __shared__ __align__(16) unsigned char s_x[];  // [kt][64] codes, [kt][64] exponents
  const Mx4Shape gw(a.n, a.k);
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kt_n = static_cast<int>(gw.kt), kq_n = static_cast<int>(gw.kq);
  const int tiles = (static_cast<int>(gw.rt) - static_cast<int>(blockIdx.x) + static_cast<int>(gridDim.x) - 1) / static_cast<int>(gridDim.x);
  const int fours = kq_n > w ? (kq_n - w + kMxWaves - 1) / kMxWaves : 0;  // this wave's, of a tile
  u32x4* lx = reinterpret_cast<u32x4*>(s_x);
  unsigned char* le = s_x + static_cast<size_t>(kt_n) * 1024;
  struct Four {
    u32x4 w[4];
    uint32_t s;
  };
  int lt = blockIdx.x, lq = w;  // the next four to load
  auto load = [&](Four& f) __attribute__((always_inline)) {
    const u32x4* wp = reinterpret_cast<const u32x4*>(a.w) + static_cast<size_t>(lt) * kt_n * 64 + lane;
    f.s = reinterpret_cast<const uint32_t*>(a.w + gw.scales_at())[(static_cast<size_t>(lt) * kq_n + lq) * 64 + lane];
#pragma unroll
    for (int j = 0; j < 4; ++j) f.w[j] = __builtin_nontemporal_load(wp + static_cast<size_t>(min(4 * lq + j, kt_n - 1)) * 64);
    lq += kMxWaves;
    if (lq >= kq_n) {
      lq = w;
      lt += gridDim.x;
    }
  };
  const int n = tiles * fours;
  Four fa, fb;
  if (n > 0) load(fa);
  {
    // (row lane / 16 of four, a quarter of a block)
    const int row = lane >> 4, at = row + 16 * (lane >> 2 & 3), c = 8 * (lane & 15);
    for (int q = w; q < kq_n; q += kMxWaves) {
      Mx4Eight<FP32> v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int kk = 128 * (4 * q + j) + c;
        v[j].template load<true>(static_cast<const Mx4Elem<FP32>*>(a.x_raw) + row * a.x_stride + kk, row < a.rows && kk < a.k ? 8 : 0);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int kt = 4 * q + j;
        if (kt >= kt_n) break;
        uint32_t e;
        const uint32_t codes = v[j].encode(e);
        uint32_t* to = reinterpret_cast<uint32_t*>(lx + static_cast<size_t>(kt) * 64 + at) + (lane & 3);
        to[0] = codes;
        to[16] = to[32] = to[48] = 0u;  // rows 4 .. 15 are none
        if ((lane & 3) == 0) {
          unsigned char* te = le + kt * 64 + at;
          te[0] = static_cast<unsigned char>(e);
          te[4] = te[8] = te[12] = 0;
        }
      }
    }
  }
  f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
  int t = 0, cq = 0;  // the tile and four in use
  auto finish = [&]() __attribute__((always_inline)) {
    // (the lane holds columns 16 nt + 4 (lane / 16) + r of row lane % 16)
    f32x4(&p)[kMxWaves][64] = s_part[t & 1];
    p[w][lane] = acc;
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
    barrier_after_lds_reads();
    if (w == t % kMxWaves) {
      f32x4 y = p[0][lane];
#pragma unroll
      for (int i = 1; i < kMxWaves; ++i) y += p[i][lane];
      if ((lane & 15) < a.rows) mx4_store4(a, lane & 15, 16 * static_cast<int>(blockIdx.x + t * gridDim.x) + 4 * (lane >> 4), y);
    }
    ++t;
    cq = 0;
  };
  auto use = [&](const Four& f) __attribute__((always_inline)) {
    const int q = w + cq * kMxWaves;
    auto one = [&](auto jc) __attribute__((always_inline)) {
      constexpr int J = decltype(jc)::value;
      const int kt = 4 * q + J;
      if (kt < kt_n) acc = mfma_mx4<J, 0>(f.w[J], lx[kt * 64 + lane], acc, f.s, le[kt * 64 + lane]);
    };
    one(std::integral_constant<int, 0>{});
    one(std::integral_constant<int, 1>{});
    one(std::integral_constant<int, 2>{});
    one(std::integral_constant<int, 3>{});
    if (++cq == fours) finish();
  };
  int i = 0;
  for (; i + 2 < n; i += 2) {
    load(fb);
    use(fa);
    load(fa);
    use(fb);
  }
  if (i + 1 < n) {
    load(fb);
    use(fa);
    use(fb);
  } else if (i < n) {
    use(fa);
  }
  while (t < tiles) finish();  // (a wave without a four of K)
}

bool mx4_takes_rows(int dtype, const void* x, int64_t stride, int rows, int k) {
  return rows <= kMxRawRows && k <= 128 * kMxResident && rows_aligned(x, stride, k, dtype == kMxFp32 ? 4 : 2);
}

hipError_t launch_mx4_stream(const Mx4ProductArgs& a, hipStream_t s) {
  const Mx4Shape g(a.n, a.k);
  // one workgroup a compute unit up to two tiles each, beyond that two
  const int nt = static_cast<int>(g.rt), most = nt <= 512 ? 256 : 512, tiles = (nt + most - 1) / most;
  const dim3 grid((nt + tiles - 1) / tiles), block(64 * kMxWaves);
  constexpr size_t kStep = 1024 + 64;  // bytes of LDS for a step's codes and exponents
  const size_t lds = static_cast<size_t>(g.kt) * kStep;
  // with the static arrays this can be more than 64 KiB of LDS: allow it once
  auto allow = [](auto kern) {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kMxResident * kStep));
  };
  if (a.x_fp32) {
    static const hipError_t attr = allow(&k_mx4_stream<true>);
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL(k_mx4_stream<true>, grid, block, lds, s, a);
  } else {
    static const hipError_t attr = allow(&k_mx4_stream<false>);
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL(k_mx4_stream<false>, grid, block, lds, s, a);
  }
  return hipGetLastError();
}

// Up to 128 rows: a workgroup takes 16 NT columns and all rows, 16 RG, its eight waves
// every eighth two of its K's steps each; x comes from the caches.  Two steps' tiles
// are in flight while the two before are used (see k_mx4_stream).  What x is read for
// each 16 columns sets the time of many rows (77 x 4096 x 14336: 143 MB), so NT is 2
// there, and K cut over workgroups where the columns are then too few (mx4_split); the
// one that arrives last adds the sums, as in k_mx4_tile.  (Eight row groups of two tiles
// do not fit the registers: of 63 spilled ones some are in the loop.)
template <int RG, int NT>
__global__ __launch_bounds__(64 * kMxWaves, 2) void k_mx4_rows(Mx4ProductArgs a, Mx4Split sp) {
  constexpr int U = RG * NT;
  __shared__ f32x4 part[kMxWaves][U][64];
  __shared__ int s_last;
  const Mx4Shape gw(a.n, a.k), gx(a.rows, a.k);
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int bm = blockIdx.x / sp.splits, split = blockIdx.x % sp.splits;
  const int kt_n = static_cast<int>(gw.kt), kq_n = static_cast<int>(gw.kq);
  const int k0 = min(kt_n, split * sp.steps), k1 = min(kt_n, k0 + sp.steps);  // (k0 a multiple of four)
  const u32x4 *wp[NT], *xp[RG];
  const uint32_t *ws[NT], *xs[RG];
  // (rows of tiles past the last one: it again, the sums are not stored)
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int64_t t = min(static_cast<int64_t>(bm) * NT + i, gw.rt - 1);
    wp[i] = reinterpret_cast<const u32x4*>(a.w) + t * kt_n * 64;
    ws[i] = reinterpret_cast<const uint32_t*>(a.w + gw.scales_at()) + t * kq_n * 64;
  }
#pragma unroll
  for (int g = 0; g < RG; ++g) {
    const int64_t t = min(static_cast<int64_t>(g), gx.rt - 1);
    xp[g] = reinterpret_cast<const u32x4*>(a.x) + t * kt_n * 64;
    xs[g] = reinterpret_cast<const uint32_t*>(a.x + gx.scales_at()) + t * kq_n * 64;
  }
  f32x4 acc[RG][NT];
#pragma unroll
  for (int g = 0; g < RG; ++g)
#pragma unroll
    for (int i = 0; i < NT; ++i) acc[g][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  struct Two {
    u32x4 w[2][NT], x[2][RG];
    uint32_t sw[NT], sx[RG];
  };
  auto load = [&](Two& s, int i) __attribute__((always_inline)) {
    const int kt = k0 + 2 * (w + i * kMxWaves);
    const size_t q = kt >> 2, ka = kt, kb = min(kt + 1, kt_n - 1);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      s.sw[j] = ws[j][q * 64 + lane];
      s.w[0][j] = __builtin_nontemporal_load(wp[j] + ka * 64 + lane);
      s.w[1][j] = __builtin_nontemporal_load(wp[j] + kb * 64 + lane);
    }
#pragma unroll
    for (int g = 0; g < RG; ++g) {
      s.sx[g] = xs[g][q * 64 + lane];
      s.x[0][g] = xp[g][ka * 64 + lane];
      s.x[1][g] = xp[g][kb * 64 + lane];
    }
  };
  auto use = [&](const Two& s, int i) __attribute__((always_inline)) {
    const int kt = k0 + 2 * (w + i * kMxWaves), sh = 8 * (kt & 3);
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int g = 0; g < RG; ++g) acc[g][j] = mfma_mx4<0, 0>(s.w[0][j], s.x[0][g], acc[g][j], s.sw[j] >> sh, s.sx[g] >> sh);
    if (kt + 1 < k1) {
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int g = 0; g < RG; ++g) acc[g][j] = mfma_mx4<1, 1>(s.w[1][j], s.x[1][g], acc[g][j], s.sw[j] >> sh, s.sx[g] >> sh);
    }
  };
  const int twos = (k1 - k0 + 1) / 2, n = twos > w ? (twos - w + kMxWaves - 1) / kMxWaves : 0;
  Two sa, sb;
  if (n > 0) load(sa, 0);
  int i = 0;
  for (; i + 2 < n; i += 2) {
    load(sb, i + 1);
    use(sa, i);
    load(sa, i + 2);
    use(sb, i + 1);
  }
  if (i + 1 < n) {
    load(sb, i + 1);
    use(sa, i);
    use(sb, i + 1);
  } else if (i < n) {
    use(sa, i);
  }
#pragma unroll
  for (int g = 0; g < RG; ++g)
#pragma unroll
    for (int j = 0; j < NT; ++j) part[w][g * NT + j][lane] = acc[g][j];
  __syncthreads();
  constexpr int kMine = (U + kMxWaves - 1) / kMxWaves;
  f32x4 y[kMine];
  auto each = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
    for (int m = 0; m < kMine; ++m)
      if (w + m * kMxWaves < U) f(m, w + m * kMxWaves);
  };
  each([&](int m, int u) __attribute__((always_inline)) {
    y[m] = part[0][u][lane];
#pragma unroll
    for (int j = 1; j < kMxWaves; ++j) y[m] += part[j][u][lane];
  });
  if (sp.splits > 1) {
    uint8_t* mem = reinterpret_cast<uint8_t*>(sp.part) + static_cast<size_t>(bm) * sp.splits * U * 1024;
    each([&](int m, int u) __attribute__((always_inline)) { store_wt(mem + (split * U + u) * 1024 + 16 * lane, __builtin_bit_cast(u32x4, y[m])); });
    if (!mx4_last_of(sp, bm, s_last)) return;
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(mem, 0, sp.splits * U * 1024, 0x00020000);
    each([&](int m, int) __attribute__((always_inline)) { y[m] = f32x4{0.f, 0.f, 0.f, 0.f}; });
    for (int s = 0; s < sp.splits; ++s)
      each([&](int m, int u) __attribute__((always_inline)) { y[m] += load_agent4(rs, (s * U + u) * 1024 + 16 * lane); });
  }
  each([&](int m, int u) __attribute__((always_inline)) {
    const int row = 16 * (u / NT) + (lane & 15);
    if (row < a.rows) mx4_store4(a, row, 16 * (bm * NT + u % NT) + 4 * (lane >> 4), y[m]);
  });
}

hipError_t launch_mx4_rows(const Mx4ProductArgs& a, const Mx4Split& sp, hipStream_t s) {
  auto go = [&](auto c) {
    constexpr int RG = decltype(c)::value;
    const dim3 grid(sp.tiles() * sp.splits), block(64 * kMxWaves);
    if constexpr (RG >= 2)  // (as mx4_split does)
      if (sp.tm == 2) {
        hipLaunchKernelGGL((k_mx4_rows<RG, 2>), grid, block, 0, s, a, sp);
        return;
      }
    hipLaunchKernelGGL((k_mx4_rows<RG, 1>), grid, block, 0, s, a, sp);
  };
  switch (sp.tn) {
    case 1: go(std::integral_constant<int, 1>{}); break;
    case 2: go(std::integral_constant<int, 2>{}); break;
    case 3: go(std::integral_constant<int, 3>{}); break;
    case 4: go(std::integral_constant<int, 4>{}); break;
    case 5: go(std::integral_constant<int, 5>{}); break;
    case 6: go(std::integral_constant<int, 6>{}); break;
    case 7: go(std::integral_constant<int, 7>{}); break;
    default: go(std::integral_constant<int, 8>{}); break;
  }
  return hipGetLastError();
}

}  // namespace vsk
