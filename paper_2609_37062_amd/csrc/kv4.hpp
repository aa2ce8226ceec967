// KV cache in 4 bits: layout of the pool, launchers (k_kv4.hip).
//
// Pool = [L][n_blocks][n_kv_heads] records of one block (16 tokens) of one head,
// 17 head_dim bytes: K codes (8 head_dim bytes), V codes, K exponents (head_dim /
// 2), V exponents; K and V in microscaled 4 bits, blocks of 32 along the head's
// dims (mx4.hpp).  The order inside is the one in which attention feeds the
// 16x16x32 MFMA (attn_core.hpp):
//  * K: the head's dims in quarters of D / 4, quarter q of a token what lane
//    quarter q feeds.  p is token t with bits 2 and 3 swapped, as in the 16-bit
//    pool.  D = 128: 16 bytes of (p, q) at 16 (p + 16 q); D = 64: 8 bytes at 16 (p %
//    8 + 8 q) + 8 (p / 8).  Exponent of dims 32 b .. of p at 2 (p % 8 + 8 b) + p / 8.
//  * V: byte b of (token t, d) holds dims 32 b + d (low half) and 32 b + 16 + d; a
//    byte never holds two tokens, so a token is written without reading its
//    neighbours.  D = 128: 4 bytes at 16 (d + 16 (t / 8) + 32 (t % 8 / 4)) + 4 (t %
//    4); D = 64: 2 bytes at 16 (d + 16 (t / 8)) + 2 (t % 8).  Exponent of dims 32 b
//    .. of t at t D / 32 + b.
#pragma once

#include "internal.hpp"

namespace vsk {

__host__ __device__ constexpr size_t kv4_record(int D) { return static_cast<size_t>(17) * D; }
__host__ __device__ constexpr int kv4_v_at(int D) { return 8 * D; }
__host__ __device__ constexpr int kv4_ks_at(int D) { return 16 * D; }
__host__ __device__ constexpr int kv4_vs_at(int D) { return 16 * D + D / 2; }
__host__ __device__ inline int kv4_p(int t) { return (t & 3) | ((t & 4) << 1) | ((t & 8) >> 1); }
// byte of the codes of dims e, e + 1 (e even) of place p
__host__ __device__ inline int kv4_k_byte(int D, int p, int e) {
  const int q = e / (D / 4), in = e % (D / 4) / 2;
  return D == 128 ? 16 * (p + 16 * q) + in : 16 * ((p & 7) + 8 * q) + 8 * (p >> 3) + in;
}
__host__ __device__ inline int kv4_ks_byte(int p, int b) { return 2 * ((p & 7) + 8 * b) + (p >> 3); }
// first byte of (token t, d)
__host__ __device__ inline int kv4_v_byte(int D, int t, int d) {
  return D == 128 ? 16 * (d + 16 * (t >> 3) + 32 * (t >> 2 & 1)) + 4 * (t & 3) : 16 * (d + 16 * (t >> 3)) + 2 * (t & 7);
}

// Whether a launch takes so many heads of rows (eight values a thread, less than 2^32
// of them with what fills up a wave and a workgroup).
inline bool kv4_launches(int64_t rows, int heads, int hd) { return (rows + 8) * heads * hd <= (INT64_C(1) << 35) - 4096; }

struct Kv4Pool {
  uint8_t* pool;
  int layer, n_blocks, Hkv;
};
hipError_t launch_kv4_write(const Kv4Pool& p, int hd, const int32_t* slots, int n, const uint16_t* k, const uint16_t* v,
                            hipStream_t s);
hipError_t launch_kv4_read(const Kv4Pool& p, int hd, const int32_t* slots, int n, uint16_t* k, uint16_t* v, hipStream_t s);

// Rows of a QKV projection: norms and rotation of q and k heads, q out, k and v
// into a cache (k_kv4.hip).
struct QkvArgs {
  const uint16_t* qkv;  // [R] rows of Hq + 2 Hkv heads, `stride` apart
  int64_t stride;
  int R, Hq, Hkv;
  const uint16_t *q_gain, *k_gain;  // nullable: no norm
  float eps;
  const int32_t *rot, *slot;  // [R]
  const float2* rope;         // [max_pos][hd / 2] (cos, sin), and behind it the same in doubles
  int max_pos;
  uint16_t* q;     // [R][Hq][hd]
  uint16_t* pool;  // the 16-bit cache, or
  uint8_t* pool4;  // the 4-bit one
  int layer, n_blocks;
};
// The table of QkvArgs::rope.
hipError_t launch_rope_table(float2* table, int max_pos, int hd, double theta, hipStream_t s);
hipError_t launch_qkv_norm_rope(const QkvArgs& a, int hd, hipStream_t s);

}  // namespace vsk
