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

// The largest over the eight lanes of a block.
__device__ __forceinline__ uint32_t max8(uint32_t v) {
#pragma unroll
  for (int m = 1; m < 8; m <<= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), m, 64)));
  return v;
}
// Sum over the G lanes of a head.
template <int G, class T>
__device__ __forceinline__ T sum_head(T v) {
#pragma unroll
  for (int m = 1; m < G; m <<= 1) v += __shfl_xor(v, m, 64);
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
template <int D>
__global__ __launch_bounds__(kHeadThreads) void k_kv4_write(Kv4Pool p, const int32_t* __restrict__ slots, int n,
                                                            const uint16_t* __restrict__ k, const uint16_t* __restrict__ v) {
  constexpr int G = D / 8;
  const int64_t unit = (static_cast<int64_t>(blockIdx.x) * kHeadThreads + threadIdx.x) / G;
  const int i = threadIdx.x % G;
  const bool in = unit < static_cast<int64_t>(n) * p.Hkv;
  const int tok = in ? static_cast<int>(unit / p.Hkv) : 0, hk = in ? static_cast<int>(unit % p.Hkv) : 0;
  const int sl = in ? slots[tok] : -1;
  const bool on = sl >= 0 && sl < p.n_blocks * kBlock;
  uint8_t* rec = kv4_rec<D>(p, on ? sl : 0, hk);
  const size_t at = (static_cast<size_t>(tok) * p.Hkv + hk) * D + 4 * i;
  auto load = [&](const uint16_t* x) {
    u32x2 r = u32x2{0u, 0u};
    if (!on) return r;
    r[0] = x[0] | static_cast<uint32_t>(x[1]) << 16;
    r[1] = x[2] | static_cast<uint32_t>(x[3]) << 16;
    return r;
  };
  put_k<D>(rec, sl & 15, i, encode_head(load(k + at), load(k + at + D / 2)), on);
  put_v<D>(rec, sl & 15, i, encode_head(load(v + at), load(v + at + D / 2)), on);
}

// The values that slots hold, two dims a thread.
template <int D>
__global__ __launch_bounds__(256) void k_kv4_read(Kv4Pool p, const int32_t* __restrict__ slots, int n,
                                                  uint16_t* __restrict__ k, uint16_t* __restrict__ v) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int64_t unit = i / (D / 2);
  if (unit >= static_cast<int64_t>(n) * p.Hkv) return;
  const int j = static_cast<int>(i % (D / 2));
  const int tok = static_cast<int>(unit / p.Hkv), hk = static_cast<int>(unit % p.Hkv);
  const int sl = slots[tok];
  if (sl < 0 || sl >= p.n_blocks * kBlock) return;
  const uint8_t* rec = kv4_rec<D>(p, sl, hk);
  const int t = sl & 15, pl = kv4_p(t);
  const size_t at = static_cast<size_t>(unit) * D;
  const uint32_t kc = mx4_decode<0>(rec[kv4_k_byte(D, pl, 2 * j)], mx4_scale(rec[kv4_ks_at(D) + kv4_ks_byte(pl, j >> 4)]));
  k[at + 2 * j] = static_cast<uint16_t>(kc);
  k[at + 2 * j + 1] = static_cast<uint16_t>(kc >> 16);
  const int b = j >> 4, d = j & 15;
  const uint32_t vc = mx4_decode<0>(rec[kv4_v_at(D) + kv4_v_byte(D, t, d) + b], mx4_scale(rec[kv4_vs_at(D) + t * (D / 32) + b]));
  v[at + 32 * b + d] = static_cast<uint16_t>(vc);
  v[at + 32 * b + 16 + d] = static_cast<uint16_t>(vc >> 16);
}

// A float that rounds to 4 bits (or to bf16) as the double does: where the double
// lies beside the float, the neighbour with an odd last bit, which no border is.
__device__ __forceinline__ float odd_float(double d) {
  const float f = static_cast<float>(d);
  const double r = d - static_cast<double>(f);
  uint32_t u = __float_as_uint(f);
  if (r != 0.0 && (u & 1u) == 0u && (u & 0x7f800000u) != 0x7f800000u) u += (r > 0.0) == (u >> 31 == 0u) ? 1u : -1u;
  return __uint_as_float(u);
}

// One (row, head) for D / 8 lanes.  T: what norm and rotation are computed in; keys
// of the 4-bit cache take doubles, with the rotary table's remainders, so that their
// codes are those of the exact values: an error of float32 at a border between two
// codes is a whole step there.
template <int D, class T>
__device__ __forceinline__ void norm_rope(const QkvArgs& a, int row, int i, u32x2 lo, u32x2 hi, const uint16_t* gain,
                                          T (&x)[4], T (&y)[4]) {
  constexpr int G = D / 8;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[j] = static_cast<T>(bf2f(lo[j >> 1] >> (16 * (j & 1)) & 0xffffu));
    y[j] = static_cast<T>(bf2f(hi[j >> 1] >> (16 * (j & 1)) & 0xffffu));
  }
  if (gain != nullptr) {
    T ss = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) ss += x[j] * x[j] + y[j] * y[j];
    ss = sum_head<G>(ss);
    const T r = static_cast<T>(1) / sqrt(ss / D + static_cast<T>(a.eps));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[j] *= r * static_cast<T>(bf2f(gain[4 * i + j]));
      y[j] *= r * static_cast<T>(bf2f(gain[D / 2 + 4 * i + j]));
    }
  }
  const size_t at = static_cast<size_t>(a.rot[row]) * (D / 2) + 4 * i, more = static_cast<size_t>(a.max_pos) * (D / 2);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 cs = a.rope[at + j];
    T c = static_cast<T>(cs.x), s = static_cast<T>(cs.y);
    if constexpr (sizeof(T) == 8) {
      const float2 rest = a.rope[more + at + j];
      c += static_cast<T>(rest.x);
      s += static_cast<T>(rest.y);
    }
    const T u = x[j] * c - y[j] * s, v = y[j] * c + x[j] * s;
    x[j] = u;
    y[j] = v;
  }
}

template <int D, bool FOUR>
__global__ __launch_bounds__(kHeadThreads) void k_qkv_norm_rope(QkvArgs a) {
  constexpr int G = D / 8;
  const int heads = a.Hq + 2 * a.Hkv;
  const int64_t unit = (static_cast<int64_t>(blockIdx.x) * kHeadThreads + threadIdx.x) / G;
  const int i = threadIdx.x % G;
  if (unit >= static_cast<int64_t>(a.R) * heads) return;  // (whole heads of lanes)
  const int row = static_cast<int>(unit / heads), head = static_cast<int>(unit % heads);
  const uint16_t* src = a.qkv + row * a.stride + static_cast<size_t>(head) * D + 4 * i;
  const u32x2 lo = *reinterpret_cast<const u32x2*>(src), hi = *reinterpret_cast<const u32x2*>(src + D / 2);
  if (head < a.Hq) {
    float x[4], y[4];
    norm_rope<D>(a, row, i, lo, hi, a.q_gain, x, y);
    uint16_t* dst = a.q + (static_cast<size_t>(row) * a.Hq + head) * D + 4 * i;
    *reinterpret_cast<u32x2*>(dst) = u32x2{pack_bf2(x[0], x[1]), pack_bf2(x[2], x[3])};
    *reinterpret_cast<u32x2*>(dst + D / 2) = u32x2{pack_bf2(y[0], y[1]), pack_bf2(y[2], y[3])};
    return;
  }
  const int sl = a.slot[row], t = sl & 15;
  const bool is_k = head < a.Hq + a.Hkv;
  const int hk = head - a.Hq - (is_k ? 0 : a.Hkv);
  if constexpr (FOUR) {
    const Kv4Pool p{a.pool4, a.layer, a.n_blocks, a.Hkv};
    uint8_t* rec = kv4_rec<D>(p, sl, hk);
    if (!is_k) {
      put_v<D>(rec, t, i, encode_head(lo, hi), true);
      return;
    }
    double x[4], y[4];
    norm_rope<D>(a, row, i, lo, hi, a.k_gain, x, y);
    float fx[4], fy[4];
    uint32_t tl = 0, th = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      fx[j] = odd_float(x[j]);
      fy[j] = odd_float(y[j]);
      tl = max(tl, __float_as_uint(fx[j]) & 0x7fffffffu);
      th = max(th, __float_as_uint(fy[j]) & 0x7fffffffu);
    }
    HeadCodes h;
    h.lo = mx4_exponent(max8(tl));
    h.hi = mx4_exponent(max8(th));
    const float s0 = mx4_scale(h.lo), s1 = mx4_scale(h.hi);
    uint32_t c = mx4_encode_f32<0>(0u, fx[0], fx[1], s0), d = mx4_encode_f32<0>(0u, fy[0], fy[1], s1);
    c = mx4_encode_f32<1>(c, fx[2], fx[3], s0);
    d = mx4_encode_f32<1>(d, fy[2], fy[3], s1);
    h.codes = (h.lo == 255u ? 0u : c & 0xffffu) | (h.hi == 255u ? 0u : d << 16);
    put_k<D>(rec, t, i, h, true);
  } else {
    const size_t head_elems = static_cast<size_t>(kBlock) * D;
    uint16_t* blk = a.pool + ((static_cast<size_t>(a.layer) * 2 + (is_k ? 0 : 1)) * a.n_blocks + (sl >> 4)) * a.Hkv * head_elems +
                    hk * head_elems;
    if (is_k) {
      float x[4], y[4];
      norm_rope<D>(a, row, i, lo, hi, a.k_gain, x, y);
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

hipError_t launch_kv4_write(const Kv4Pool& p, int hd, const int32_t* slots, int n, const uint16_t* k, const uint16_t* v,
                            hipStream_t s) {
  if (n == 0) return hipSuccess;
  const dim3 grid(head_blocks(static_cast<int64_t>(n) * p.Hkv, hd)), block(kHeadThreads);
  if (hd == 128) hipLaunchKernelGGL(k_kv4_write<128>, grid, block, 0, s, p, slots, n, k, v);
  else hipLaunchKernelGGL(k_kv4_write<64>, grid, block, 0, s, p, slots, n, k, v);
  return hipGetLastError();
}

hipError_t launch_kv4_read(const Kv4Pool& p, int hd, const int32_t* slots, int n, uint16_t* k, uint16_t* v, hipStream_t s) {
  if (n == 0) return hipSuccess;
  const dim3 grid(static_cast<unsigned>((static_cast<int64_t>(n) * p.Hkv * (hd / 2) + 255) / 256)), block(256);
  if (hd == 128) hipLaunchKernelGGL(k_kv4_read<128>, grid, block, 0, s, p, slots, n, k, v);
  else hipLaunchKernelGGL(k_kv4_read<64>, grid, block, 0, s, p, slots, n, k, v);
  return hipGetLastError();
}

hipError_t launch_qkv_norm_rope(const QkvArgs& a, int hd, hipStream_t s) {
  const dim3 grid(head_blocks(static_cast<int64_t>(a.R) * (a.Hq + 2 * a.Hkv), hd)), block(kHeadThreads);
  const bool four = a.pool4 != nullptr;
  auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, block, 0, s, a); };
  if (hd == 128) four ? go(k_qkv_norm_rope<128, true>) : go(k_qkv_norm_rope<128, false>);
  else four ? go(k_qkv_norm_rope<64, true>) : go(k_qkv_norm_rope<64, false>);
  return hipGetLastError();
}

}  // namespace vsk
