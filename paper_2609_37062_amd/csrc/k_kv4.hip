// The 4-bit KV cache: writes, reads, and the way into either cache from the rows of
// a QKV projection.
//
// A head of a token is taken by D / 8 lanes: lane i holds dims 4 i .. 4 i + 3 and D /
// 2 + 4 i .. + 3, the rotary pairs (j, j + D / 2) of four j.  Eight lanes then hold a
// block of 32 dims in each half.
#include "kv4.hpp"
#include "mx4_dev.hpp"

namespace vsk {

constexpr int kHeadThreads = 256;
// (one load or store, whatever its alignment)
typedef u32x2 __attribute__((aligned(2))) Bf16x4;
typedef u32x4 __attribute__((aligned(2))) Bf16x8;

// A value of another lane: ^ 1, ^ 2, ^ 7, ^ 15, which a reduction over 2, 4, 8 and 16
// lanes takes in turn.
template <int CTRL>
__device__ __forceinline__ uint32_t from_lane(uint32_t v) {
  return static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), CTRL, 0xf, 0xf, true));
}
constexpr int kXor1 = 0xb1, kXor2 = 0x4e, kXor7 = 0x141, kXor15 = 0x140;
// The largest over the eight lanes of a block.
__device__ __forceinline__ uint32_t max8(uint32_t v) {
  v = max(v, from_lane<kXor1>(v));
  v = max(v, from_lane<kXor2>(v));
  return max(v, from_lane<kXor7>(v));
}
// Sum over the G lanes of a head.
template <int CTRL, class T>
__device__ __forceinline__ T add_lane(T v) {
  if constexpr (sizeof(T) == 8) {
    const u32x2 u = __builtin_bit_cast(u32x2, v);
    return v + __builtin_bit_cast(T, u32x2{from_lane<CTRL>(u[0]), from_lane<CTRL>(u[1])});
  } else {
    return v + __builtin_bit_cast(T, from_lane<CTRL>(__builtin_bit_cast(uint32_t, v)));
  }
}
template <int G, class T>
__device__ __forceinline__ T sum_head(T v) {
  static_assert(G == 8 || G == 16);
  v = add_lane<kXor7>(add_lane<kXor2>(add_lane<kXor1>(v)));
  if constexpr (G == 16) v = add_lane<kXor15>(v);
  return v;
}

// Codes of this lane's four low dims (bits 0..15) and four high ones, and their
// blocks' exponents, from bf16 pairs.
struct HeadCodes {
  uint32_t codes;
  uint32_t lo, hi;  // exponents
};
__device__ __forceinline__ HeadCodes encode_head(u32x2 lo, u32x2 hi) {
  HeadCodes h;
  auto top = [](u32x2 x) { return mx4_top(mx4_top2(x[0] & 0x7fff7fffu, x[1] & 0x7fff7fffu)); };
  h.lo = mx4_exponent(max8(top(lo)));
  h.hi = mx4_exponent(max8(top(hi)));
  const float sl = mx4_scale(h.lo), sh = mx4_scale(h.hi);
  uint32_t c = mx4_encode_bf16<0>(0u, lo[0], sl), d = mx4_encode_bf16<0>(0u, hi[0], sh);
  c = mx4_encode_bf16<1>(c, lo[1], sl);
  d = mx4_encode_bf16<1>(d, hi[1], sh);
  h.codes = (h.lo == 255u ? 0u : c & 0xffffu) | (h.hi == 255u ? 0u : d << 16);
  return h;
}

// A head of a token into its record (lane i of the head's; every lane of the head's
// calls it, `on`: the token has a slot).
template <int D>
__device__ __forceinline__ void put_k(uint8_t* rec, int t, int i, const HeadCodes& h, bool on) {
  if (!on) return;
  const int p = kv4_p(t), b = i >> 3;
  *reinterpret_cast<uint16_t*>(rec + kv4_k_byte(D, p, 4 * i)) = static_cast<uint16_t>(h.codes);
  *reinterpret_cast<uint16_t*>(rec + kv4_k_byte(D, p, D / 2 + 4 * i)) = static_cast<uint16_t>(h.codes >> 16);
  if ((i & 7) == 0) {
    rec[kv4_ks_at(D) + kv4_ks_byte(p, b)] = static_cast<uint8_t>(h.lo);
    rec[kv4_ks_at(D) + kv4_ks_byte(p, D / 64 + b)] = static_cast<uint8_t>(h.hi);
  }
}
template <int D>
__device__ __forceinline__ void put_v(uint8_t* rec, int t, int i, const HeadCodes& h, bool on) {
  // lane i collects what (t, d) holds, d = i (and i + 8 at D = 64): dim 16 c + d is
  // nibble d % 4 of lane d / 4 + 4 c of the low half, c - D / 32 of the high one
  constexpr int C = D / 32;  // of each half
  const int first = (threadIdx.x & 63) - i;
#pragma unroll
  for (int u = 0; u < 128 / D; ++u) {
    const int d = i + 8 * u;
    uint32_t lo = 0, hi = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const uint32_t x = static_cast<uint32_t>(__shfl(static_cast<int>(h.codes), first + (d >> 2) + 4 * c, 64)) >> (4 * (d & 3));
      lo |= (x & 15u) << (4 * c);
      hi |= (x >> 16 & 15u) << (4 * c);
    }
    uint8_t* to = rec + kv4_v_at(D) + kv4_v_byte(D, t, d);
    if (on) {
      if constexpr (D == 128) *reinterpret_cast<uint32_t*>(to) = lo | hi << 16;
      else *reinterpret_cast<uint16_t*>(to) = static_cast<uint16_t>(lo | hi << 8);
    }
  }
  if (on && (i & 7) == 0) {
    rec[kv4_vs_at(D) + t * (D / 32) + (i >> 3)] = static_cast<uint8_t>(h.lo);
    rec[kv4_vs_at(D) + t * (D / 32) + D / 64 + (i >> 3)] = static_cast<uint8_t>(h.hi);
  }
}

template <int D>
__device__ __forceinline__ uint8_t* kv4_rec(const Kv4Pool& p, int slot, int hk) {
  return p.pool + ((static_cast<size_t>(p.layer) * p.n_blocks + (slot >> 4)) * p.Hkv + hk) * kv4_record(D);
}

// Logical k, v [n][Hkv][D] into their slots (slots outside the pool are ignored).
// A wave takes one head of consecutive tokens, which share lines of a record: 448,000
// tokens of 8 heads x 128 658 us (a wave four heads of a token 741).
template <int D>
__global__ __launch_bounds__(kHeadThreads) void k_kv4_write(Kv4Pool p, const int32_t* __restrict__ slots, int n,
                                                            const uint16_t* __restrict__ k, const uint16_t* __restrict__ v) {
  constexpr int G = D / 8;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * (kHeadThreads / 64) + (threadIdx.x >> 6));
  const int i = threadIdx.x % G, hk = static_cast<int>(wave % p.Hkv);
  const int64_t tok = static_cast<int64_t>(wave / p.Hkv) * (64 / G) + (threadIdx.x & 63) / G;
  const bool in = tok < n;
  const int sl = in ? slots[tok] : -1;
  const bool on = sl >= 0 && sl < p.n_blocks * kBlock;
  uint8_t* rec = kv4_rec<D>(p, on ? sl : 0, hk);
  const size_t at = static_cast<size_t>(tok * p.Hkv + hk) * D + 4 * i;
  auto load = [&](const uint16_t* x) { return on ? *reinterpret_cast<const Bf16x4*>(x) : u32x2{0u, 0u}; };
  put_k<D>(rec, sl & 15, i, encode_head(load(k + at), load(k + at + D / 2)), on);
  put_v<D>(rec, sl & 15, i, encode_head(load(v + at), load(v + at + D / 2)), on);
}

// The values that slots hold, eight dims of K and of V a lane.
template <int D>
__global__ __launch_bounds__(kHeadThreads) void k_kv4_read(Kv4Pool p, const int32_t* __restrict__ slots, int n,
                                                           uint16_t* __restrict__ k, uint16_t* __restrict__ v) {
  constexpr int G = D / 8;
  const int64_t unit = (static_cast<int64_t>(blockIdx.x) * kHeadThreads + threadIdx.x) / G;
  const int i = threadIdx.x % G, first = (threadIdx.x & 63) - i;
  if (unit >= static_cast<int64_t>(n) * p.Hkv) return;  // (whole heads of lanes, here and below)
  const int tok = static_cast<int>(unit / p.Hkv), hk = static_cast<int>(unit % p.Hkv);
  const int sl = slots[tok];
  if (sl < 0 || sl >= p.n_blocks * kBlock) return;
  const uint8_t* rec = kv4_rec<D>(p, sl, hk);
  const int t = sl & 15, pl = kv4_p(t), b = i >> 2;
  const uint32_t kc = *reinterpret_cast<const uint32_t*>(rec + kv4_k_byte(D, pl, 8 * i));
  const uint8_t* vp = rec + kv4_v_at(D);
  uint32_t own;  // what (t, d) holds, d = i; D = 64: and d = i + 8 above it
  if constexpr (D == 128)
    own = *reinterpret_cast<const uint32_t*>(vp + kv4_v_byte(D, t, i));
  else
    own = *reinterpret_cast<const uint16_t*>(vp + kv4_v_byte(D, t, i)) |
          static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(vp + kv4_v_byte(D, t, i + 8))) << 16;
  const float ks = mx4_scale(rec[kv4_ks_at(D) + kv4_ks_byte(pl, b)]), vs = mx4_scale(rec[kv4_vs_at(D) + t * (D / 32) + b]);
  uint32_t vc = 0;  // dims 8 i ..: nibble i / 2 of d = 8 (i % 2) ..
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int from = D == 128 ? 8 * (i & 1) + j : j, bit = 4 * (i >> 1) + (D == 128 ? 0 : 16 * (i & 1));
    vc |= (static_cast<uint32_t>(__shfl(static_cast<int>(own), first + from, 64)) >> bit & 15u) << (4 * j);
  }
  const u32x4 ko = mx4_decode8(kc, ks), vo = mx4_decode8(vc, vs);
  const size_t at = static_cast<size_t>(unit) * D + 8 * i;
  *reinterpret_cast<Bf16x8*>(k + at) = ko;
  *reinterpret_cast<Bf16x8*>(v + at) = vo;
}

// A float that rounds to 4 bits as the double does: its first 23 bits behind the
// point, the last one set where more follow.  (Every border between codes has fewer.)
__device__ __forceinline__ float odd_float(double d) {
  u32x2 u = __builtin_bit_cast(u32x2, d);
  u[0] = (u[0] & 0xe0000000u) | ((u[0] & 0x1fffffffu) != 0u ? 0x20000000u : 0u);
  return static_cast<float>(__builtin_bit_cast(double, u));
}

__device__ __forceinline__ float inv_sqrt(float v) { return rsqrtf(v); }
__device__ __forceinline__ double inv_sqrt(double v) {  // two Newton steps from the instruction's 2^-14 and better
  double y = __builtin_amdgcn_rsq(v);
  if (v < static_cast<double>(INFINITY) && v > 0.0) {
#pragma unroll
    for (int j = 0; j < 2; ++j) y = fma(y, 0.5 * fma(-v * y, y, 1.0), y);
  }
  return y;
}

// Norm and rotation of a head, D / 8 lanes.  T: what they are computed in; keys of
// the 4-bit cache take doubles, and the rotary table's, so that their codes are those
// of the exact values: an error of float32 at a border between two codes is a whole
// step there.
template <int D, class T>
__device__ __forceinline__ void norm_rope(float eps, int i, u32x2 lo, u32x2 hi, const uint16_t* gain, const T (&c)[4],
                                          const T (&s)[4], T (&x)[4], T (&y)[4]) {
  constexpr int G = D / 8;
  float fx[4], fy[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    fx[j] = bf2f(lo[j >> 1] >> (16 * (j & 1)) & 0xffffu);
    fy[j] = bf2f(hi[j >> 1] >> (16 * (j & 1)) & 0xffffu);
  }
  T u[4], v[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    u[j] = static_cast<T>(fx[j]);
    v[j] = static_cast<T>(fy[j]);
  }
  if (gain != nullptr) {
    const u32x2 gl = *reinterpret_cast<const Bf16x4*>(gain + 4 * i), gh = *reinterpret_cast<const Bf16x4*>(gain + D / 2 + 4 * i);
    auto mean = [&](auto zero) {  // of the squares, and eps
      using S = decltype(zero);
      S ss = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        ss = fma(static_cast<S>(fx[j]), static_cast<S>(fx[j]), ss);
        ss = fma(static_cast<S>(fy[j]), static_cast<S>(fy[j]), ss);
      }
      return fma(sum_head<G>(ss), static_cast<S>(1.0 / D), static_cast<S>(eps));
    };
    auto scaled = [&](auto r) {
      using S = decltype(r);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        u[j] = static_cast<T>(static_cast<S>(fx[j]) * (r * static_cast<S>(bf2f(gl[j >> 1] >> (16 * (j & 1)) & 0xffffu))));
        v[j] = static_cast<T>(static_cast<S>(fy[j]) * (r * static_cast<S>(bf2f(gh[j >> 1] >> (16 * (j & 1)) & 0xffffu))));
      }
    };
    const T m = mean(T(0));
    scaled(inv_sqrt(m));
    // squares that a float32 does not hold, or not to its last bit (the lanes of a head agree)
    if constexpr (sizeof(T) == 4)
      if (__builtin_expect(!(m >= 0x1p-90f && m <= 0x1p120f), 0)) scaled(inv_sqrt(mean(0.0)));
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[j] = u[j] * c[j] - v[j] * s[j];
    y[j] = v[j] * c[j] + u[j] * s[j];
  }
}

// A wave takes one head of consecutive rows, D / 8 lanes each: the rows of a run are
// neighbours in a block's record, where their small stores share lines.  Bound by
// memory and, for few rows, by the launch: 1,833 rows of 32/8 heads x 128 into 4 bits,
// 41 MB, 13.2 us; 16 into 16 bits 3.4.  (Lanes along the heads of a row 14.8; two or
// four heads a wave, a row's angles loaded once for them, 14.9 and 14.5; gains as
// single loads 17.3.)
template <int D, bool FOUR>
__global__ __launch_bounds__(kHeadThreads) void k_qkv_norm_rope(QkvArgs a) {
  constexpr int G = D / 8, kRows = 64 / G;
  const int heads = a.Hq + 2 * a.Hkv;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * (kHeadThreads / 64) + (threadIdx.x >> 6));
  const int i = threadIdx.x % G, row0 = static_cast<int>(wave / heads) * kRows, head = static_cast<int>(wave % heads);
  const int row = row0 + (threadIdx.x & 63) / G;
  if (row >= a.R) return;  // (whole heads of lanes)
  const uint16_t* src = a.qkv + row * a.stride + static_cast<size_t>(head) * D + 4 * i;
  const u32x2 lo = *reinterpret_cast<const u32x2*>(src), hi = *reinterpret_cast<const u32x2*>(src + D / 2);
  const size_t turn = static_cast<size_t>(a.rot[row]) * (D / 2) + 4 * i;
  float c[4] = {}, s[4] = {};
  if (head < (FOUR ? a.Hq : a.Hq + a.Hkv)) {
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
      const f32x4 cs = *reinterpret_cast<const f32x4*>(a.rope + turn + j);
      c[j] = cs[0];
      s[j] = cs[1];
      c[j + 1] = cs[2];
      s[j + 1] = cs[3];
    }
  }
  if (head < a.Hq) {
    float x[4], y[4];
    norm_rope<D>(a.eps, i, lo, hi, a.q_gain, c, s, x, y);
    uint16_t* dst = a.q + (static_cast<size_t>(row) * a.Hq + head) * D + 4 * i;
    *reinterpret_cast<u32x2*>(dst) = u32x2{pack_bf2(x[0], x[1]), pack_bf2(x[2], x[3])};
    *reinterpret_cast<u32x2*>(dst + D / 2) = u32x2{pack_bf2(y[0], y[1]), pack_bf2(y[2], y[3])};
    return;
  }
  const int sl = a.slot[row], t = sl & 15;
  const bool is_k = head < a.Hq + a.Hkv;
  const int hk = head - a.Hq - (is_k ? 0 : a.Hkv);
  if constexpr (FOUR) {
    uint8_t* rec = kv4_rec<D>(Kv4Pool{a.pool4, a.layer, a.n_blocks, a.Hkv}, sl, hk);
    if (!is_k) {
      put_v<D>(rec, t, i, encode_head(lo, hi), true);
      return;
    }
    double dc[4], ds[4], x[4], y[4];
    const double2* exact = reinterpret_cast<const double2*>(a.rope + static_cast<size_t>(a.max_pos) * (D / 2)) + turn;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      dc[j] = exact[j].x;
      ds[j] = exact[j].y;
    }
    norm_rope<D>(a.eps, i, lo, hi, a.k_gain, dc, ds, x, y);
    float fx[4], fy[4];
    uint32_t tl = 0, th = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      fx[j] = odd_float(x[j]);
      fy[j] = odd_float(y[j]);
      tl = max(tl, __float_as_uint(fx[j]) & 0x7fffffffu);
      th = max(th, __float_as_uint(fy[j]) & 0x7fffffffu);
    }
    HeadCodes hc;
    hc.lo = mx4_exponent(max8(tl));
    hc.hi = mx4_exponent(max8(th));
    const float s0 = mx4_scale(hc.lo), s1 = mx4_scale(hc.hi);
    uint32_t cl = mx4_encode_f32<0>(0u, fx[0], fx[1], s0), ch = mx4_encode_f32<0>(0u, fy[0], fy[1], s1);
    cl = mx4_encode_f32<1>(cl, fx[2], fx[3], s0);
    ch = mx4_encode_f32<1>(ch, fy[2], fy[3], s1);
    hc.codes = (hc.lo == 255u ? 0u : cl & 0xffffu) | (hc.hi == 255u ? 0u : ch << 16);
    put_k<D>(rec, t, i, hc, true);
  } else {
    const size_t head_elems = static_cast<size_t>(kBlock) * D;
    uint16_t* blk = a.pool + ((static_cast<size_t>(a.layer) * 2 + (is_k ? 0 : 1)) * a.n_blocks + (sl >> 4)) * a.Hkv * head_elems +
                    hk * head_elems;
    if (is_k) {
      float x[4], y[4];
      norm_rope<D>(a.eps, i, lo, hi, a.k_gain, c, s, x, y);
      *reinterpret_cast<u32x2*>(blk + kv_k_index(t, 4 * i)) = u32x2{pack_bf2(x[0], x[1]), pack_bf2(x[2], x[3])};
      *reinterpret_cast<u32x2*>(blk + kv_k_index(t, D / 2 + 4 * i)) = u32x2{pack_bf2(y[0], y[1]), pack_bf2(y[2], y[3])};
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        blk[kv_v_index(t, 4 * i + j)] = static_cast<uint16_t>(lo[j >> 1] >> (16 * (j & 1)));
        blk[kv_v_index(t, D / 2 + 4 * i + j)] = static_cast<uint16_t>(hi[j >> 1] >> (16 * (j & 1)));
      }
    }
  }
}

static unsigned head_blocks(int64_t units, int hd) { return static_cast<unsigned>((units * (hd / 8) + kHeadThreads - 1) / kHeadThreads); }

// Workgroups of waves that take one head of 64 / (hd / 8) rows each.
static unsigned wave_blocks(int rows, int heads, int hd) {
  const int per = 64 / (hd / 8);
  const int64_t waves = (static_cast<int64_t>(rows) + per - 1) / per * heads;
  return static_cast<unsigned>((waves + kHeadThreads / 64 - 1) / (kHeadThreads / 64));
}

hipError_t launch_kv4_write(const Kv4Pool& p, int hd, const int32_t* slots, int n, const uint16_t* k, const uint16_t* v,
                            hipStream_t s) {
  if (n == 0) return hipSuccess;
  const dim3 grid(wave_blocks(n, p.Hkv, hd)), block(kHeadThreads);
  if (hd == 128) hipLaunchKernelGGL(k_kv4_write<128>, grid, block, 0, s, p, slots, n, k, v);
  else hipLaunchKernelGGL(k_kv4_write<64>, grid, block, 0, s, p, slots, n, k, v);
  return hipGetLastError();
}

hipError_t launch_kv4_read(const Kv4Pool& p, int hd, const int32_t* slots, int n, uint16_t* k, uint16_t* v, hipStream_t s) {
  if (n == 0) return hipSuccess;
  const dim3 grid(head_blocks(static_cast<int64_t>(n) * p.Hkv, hd)), block(kHeadThreads);
  if (hd == 128) hipLaunchKernelGGL(k_kv4_read<128>, grid, block, 0, s, p, slots, n, k, v);
  else hipLaunchKernelGGL(k_kv4_read<64>, grid, block, 0, s, p, slots, n, k, v);
  return hipGetLastError();
}

// cos and sin of pos * theta^(-2j/D) in doubles, and rounded to float in front of them:
// a pair of dims and some positions a thread.  (1 Mi of them 15 ms on the
// host, 13 us here.)
__global__ __launch_bounds__(256) void k_rope_table(float2* __restrict__ table, int max_pos, int half, double theta) {
  const int j = threadIdx.x % half, step = static_cast<int>(gridDim.x) * (256 / half);
  const double inv = pow(theta, -static_cast<double>(j) / half);
  double2* exact = reinterpret_cast<double2*>(table + static_cast<size_t>(max_pos) * half);
  for (int p = static_cast<int>(blockIdx.x) * (256 / half) + threadIdx.x / half; p < max_pos; p += step) {
    const size_t at = static_cast<size_t>(p) * half + j;
    const double c = cos(p * inv), s = sin(p * inv);
    table[at] = make_float2(static_cast<float>(c), static_cast<float>(s));
    exact[at] = make_double2(c, s);
  }
}

hipError_t launch_rope_table(float2* table, int max_pos, int hd, double theta, hipStream_t s) {
  const int per = 256 / (hd / 2), blocks = (max_pos + per - 1) / per;
  hipLaunchKernelGGL(k_rope_table, dim3(blocks < 2048 ? blocks : 2048), dim3(256), 0, s, table, max_pos, hd / 2, theta);
  return hipGetLastError();
}

hipError_t launch_qkv_norm_rope(const QkvArgs& a, int hd, hipStream_t s) {
  const dim3 grid(wave_blocks(a.R, a.Hq + 2 * a.Hkv, hd)), block(kHeadThreads);
  const bool four = a.pool4 != nullptr;
  auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, block, 0, s, a); };
  if (hd == 128) four ? go(k_qkv_norm_rope<128, true>) : go(k_qkv_norm_rope<128, false>);
  else four ? go(k_qkv_norm_rope<64, true>) : go(k_qkv_norm_rope<64, false>);
  return hipGetLastError();
}

}  // namespace vsk
