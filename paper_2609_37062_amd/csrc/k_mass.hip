// Attention weight per cached key: what the rows of a pass, over all query
// heads, gave each key of their sequence.
//
//   mass[t] = sum over rows r that see key t, heads h of 2^(s_rht - m_rh) / l_rh
//
// with s the base-2 score and (m, 1 / l) what the attention of these rows left
// for each (row, head).  Scores are taken again from K and q with the
// attention's own products, so an exponent is exactly the one that the softmax
// summed.  A workgroup owns 32 keys of a sequence and sums over every head and
// row, each wave a run of (KV head, 16-column tile) units, in a fixed order:
// no atomics, so results do not change from run to run.
#include "attn_core.hpp"

namespace vsk {

constexpr int kMassWaves = 8;

template <int D>
__global__ __launch_bounds__(64 * kMassWaves) void k_attn_mass(AttnMassArgs a) {
  constexpr int KC = D / 32;
  __shared__ float s_sum[kMassWaves][32];
  const int seq = blockIdx.y;
  const int kv_len = a.kv_len[seq];
  const int t0 = 32 * blockIdx.x;
  if (t0 >= kv_len) return;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane & 15, quad = lane >> 4;
  const int r0 = a.cu_q[seq], n = a.cu_q[seq + 1] - r0;
  const int p0 = kv_len - n;  // position of the first row
  // the rows that see any of these keys: from position t0 on, and while the
  // window reaches back to key t0 + 31 (a sink key is seen by all of them)
  const int ra = max(0, t0 - p0);
  const int rb = a.window > 0 && t0 >= a.sinks ? min(n, t0 + 31 + a.window - p0) : n;
  const int G = a.G;
  const int cols = max(0, rb - ra) * G;
  const int tiles = (cols + 15) / 16;
  const int units = tiles * a.Hkv;
  const int per = (units + kMassWaves - 1) / kMassWaves;
  const int u0 = min(units, w * per), u1 = min(units, u0 + per);
  const int nb = (kv_len + kBlock - 1) / kBlock;
  const int32_t* table = a.block_table + static_cast<size_t>(seq) * a.max_blocks;
  const int bl = t0 / kBlock;
  const size_t blk = pair_k_block(lane) ? table[min(bl + 1, nb - 1)] : table[bl];
  const size_t kv_stride = static_cast<size_t>(a.Hkv) * kBlock * D;
  const uint16_t* kblk = a.pool + (static_cast<size_t>(a.layer) * 2 * a.n_blocks + blk) * kv_stride;
  const int k0 = pair_k_index(lane, 0), k1 = pair_k_index(lane, 1);
  const float sc = a.scale_log2;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  u32x4 kg[2][KC];
  int cur = -1;
  for (int u = u0; u < u1; ++u) {
    const int hk = u / tiles, ct = u - hk * tiles;
    if (hk != cur) {
      cur = hk;
      const u32x4* kp = reinterpret_cast<const u32x4*>(kblk + static_cast<size_t>(hk) * kBlock * D);
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        kg[0][c] = kp[c * 64 + k0];
        kg[1][c] = kp[c * 64 + k1];
      }
    }
    const int col = 16 * ct + h;
    const bool on = col < cols;
    const int row = ra + (on ? col / G : 0), head = hk * G + (on ? col % G : 0);
    const uint16_t* qrow = a.q + static_cast<size_t>(r0 + row) * a.Nq + static_cast<size_t>(head) * D;
    u32x4 qf[KC];
#pragma unroll
    for (int c = 0; c < KC; ++c) qf[c] = *reinterpret_cast<const u32x4*>(qrow + 32 * c + 8 * quad);
    const float2 ml = a.ml[static_cast<size_t>(r0 + row) * (a.Hkv * G) + head];
    f32x4 s0, s1;
    pair_qk<D>(qf, kg, s0, s1);
    const int end = min(kv_len, p0 + row + 1);
    const uint32_t bits =
        on ? span_bits(t0 + 8 * quad, end, a.window > 0 && end > a.window ? end - a.window : 0, a.sinks) : 0u;
    {
      // (both sides of the difference rounded alike, as in pair_softmax)
#pragma clang fp contract(off)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float x = s0[r] * sc, y = s1[r] * sc;
        const float wx = __builtin_amdgcn_exp2f(x - ml.x) * ml.y, wy = __builtin_amdgcn_exp2f(y - ml.x) * ml.y;
        acc[r] += bits >> r & 1u ? wx : 0.f;
        acc[4 + r] += bits >> (4 + r) & 1u ? wy : 0.f;
      }
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
#pragma unroll
    for (int x = 1; x < 16; x <<= 1) acc[j] += shfl_xor(acc[j], x);
  }
  if (h == 0) {
#pragma unroll
    for (int j = 0; j < 8; ++j) s_sum[w][8 * quad + j] = acc[j];
  }
  __syncthreads();
  if (tid < 32 && t0 + tid < kv_len) {
    float* dst = a.mass + seq * a.stride + t0 + tid;
    float s = a.add != 0 ? *dst : 0.f;
    float y = s_sum[0][tid];
#pragma unroll
    for (int i = 1; i < kMassWaves; ++i) y += s_sum[i][tid];
    *dst = s + y;
  }
}

hipError_t launch_attn_mass(const AttnMassArgs& a, int n_seqs, int max_kv_len, int head_dim, hipStream_t s) {
  const dim3 grid((max_kv_len + 31) / 32, n_seqs);
  if (head_dim == 128) hipLaunchKernelGGL((k_attn_mass<128>), grid, dim3(64 * kMassWaves), 0, s, a);
  else if (head_dim == 64) hipLaunchKernelGGL((k_attn_mass<64>), grid, dim3(64 * kMassWaves), 0, s, a);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace vsk
