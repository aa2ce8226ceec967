// Eviction of cached tokens by accumulated attention weight.
//
// k_evict_select: one workgroup per sequence.  Kept are the first `sinks` and
// the last `recent` tokens and, of those between, the ones of the largest
// weights (equal weights: lowest index; NaN below everything), listed in
// index order.  The smallest kept weight is found by radix select over the
// weights' order-preserving 32-bit keys, four digits of 8 bits, the keys held
// in registers; ranks come from block-wide prefix sums.  Everything is whole
// numbers, so nothing depends on an order of arrival.
//
// k_evict_move: copies K and V of the kept tokens, every layer and KV head, to
// the destination's blocks.
#include "dev.hpp"
#include "evict.hpp"

namespace vsk {

constexpr int kSelThreads = 1024;
constexpr int kSelWaves = kSelThreads / 64;
constexpr int kSelPer = kEvictMaxLen / kSelThreads;  // tokens of a thread

// Larger weight, larger key; -0 and 0 alike; NaN 0 (below -infinity).
__device__ __forceinline__ uint32_t mass_key(float v) {
  const uint32_t u = __float_as_uint(v == 0.f ? 0.f : v);
  return v != v ? 0u : u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}

// Exclusive prefix sum over the workgroup's threads.
__device__ __forceinline__ int block_before(int v, int* s_w) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(x, d, 64);
    if (lane >= d) x += y;
  }
  __syncthreads();
  if (lane == 63) s_w[w] = x;
  __syncthreads();
  int before = x - v;
  for (int i = 0; i < w; ++i) before += s_w[i];
  return before;
}

__global__ __launch_bounds__(kSelThreads) void k_evict_select(EvictArgs a) {
  __shared__ int s_hist[kSelWaves][256];
  __shared__ int s_w[kSelWaves];
  __shared__ uint32_t s_digit;
  __shared__ int s_left;
  const int seq = blockIdx.x, tid = threadIdx.x, w = tid >> 6, lane = tid & 63;
  const int32_t* info = a.info + 4 * seq;
  const int len = info[0], keep = info[1];
  const int32_t* dst_tbl = a.dst_tbl + info[3];
  const float* mass = a.mass + seq * a.mass_stride;
  const int per = (len + kSelThreads - 1) / kSelThreads;  // tokens tid * per .. of this thread
  const int i0 = tid * per;
  const int lo = a.sinks, hi = len - a.recent;  // the tokens that compete
  float v[kSelPer];
  uint32_t key[kSelPer];
#pragma unroll
  for (int j = 0; j < kSelPer; ++j) {
    const int i = i0 + j;
    v[j] = j < per && i < len ? mass[i] : 0.f;
    key[j] = mass_key(v[j]);
  }
  auto competes = [&](int j) { return j < per && i0 + j >= lo && i0 + j < hi; };
  int left = keep - a.sinks - a.recent;  // how many of them stay
  uint32_t top = 0;                      // the digits of the smallest kept key, as found so far
  const bool all = left >= hi - lo;      // (uniform)
  if (left > 0 && !all) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < kSelWaves * 256; i += kSelThreads) (&s_hist[0][0])[i] = 0;
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kSelPer; ++j) {
        const bool in = competes(j) && (shift == 24 || key[j] >> (shift + 8) == top >> (shift + 8));
        if (in) atomicAdd(&s_hist[w][key[j] >> shift & 255u], 1);
      }
      __syncthreads();
      if (w == 0) {  // digits 4 lane .. 4 lane + 3, from the largest digit down
        int c[4], sum = 0;
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          c[d] = 0;
          for (int x = 0; x < kSelWaves; ++x) c[d] += s_hist[x][4 * lane + d];
          sum += c[d];
        }
        int above = sum;  // keys of this lane's digits and those of higher lanes
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
          const int y = __shfl_down(above, d, 64);
          if (lane + d < 64) above += y;
        }
        above -= sum;
#pragma unroll
        for (int d = 3; d >= 0; --d) {
          if (above < left && above + c[d] >= left) {
            s_digit = 4 * lane + d;
            s_left = left - above;
          }
          above += c[d];
        }
      }
      __syncthreads();
      top |= s_digit << shift;
      left = s_left;
      __syncthreads();
    }
  }
  // above `top` every token stays, of those at `top` the first `left`
  int n_tie = 0;
#pragma unroll
  for (int j = 0; j < kSelPer; ++j) n_tie += competes(j) && key[j] == top;
  int tie = block_before(n_tie, s_w);
  uint32_t stays = 0;
  int n_stay = 0;
#pragma unroll
  for (int j = 0; j < kSelPer; ++j) {
    const int i = i0 + j;
    if (j >= per || i >= len) continue;
    bool s = i < lo || i >= hi || all;
    if (!s && keep > a.sinks + a.recent) {
      s = key[j] > top || (key[j] == top && tie < left);
      tie += key[j] == top;
    }
    stays |= static_cast<uint32_t>(s) << j;
    n_stay += s;
  }
  int at = block_before(n_stay, s_w);
  int32_t* kept = a.kept + seq * a.out_stride;
  // (mass_out may be mass itself: every weight has been read above, the two
  // prefix sums' barriers since)
#pragma unroll
  for (int j = 0; j < kSelPer; ++j) {
    if (!(stays >> j & 1u)) continue;
    kept[at] = i0 + j;
    if (a.slots != nullptr) a.slots[seq * a.out_stride + at] = dst_tbl[at / kBlock] * kBlock + at % kBlock;
    if (a.mass_out != nullptr) a.mass_out[seq * a.out_stride + at] = v[j];
    ++at;
  }
  if (a.mass_out != nullptr)
    for (int64_t i = keep + tid; i < a.out_stride; i += kSelThreads) a.mass_out[seq * a.out_stride + i] = 0.f;
}

// One thread per 16-byte piece of the destination: 8 dims of a token of K, 8
// tokens of a dim of V.
__global__ __launch_bounds__(256) void k_evict_move(EvictArgs a) {
  const int seq = blockIdx.z, layer = blockIdx.y / a.Hkv, hk = blockIdx.y % a.Hkv;
  const int32_t* info = a.info + 4 * seq;
  const int keep = info[1];
  const int hd = a.hd;
  const int blk = blockIdx.x;  // destination block
  if (blk * kBlock >= keep) return;
  const int32_t* src_tbl = a.src_tbl + info[2];
  const int32_t* kept = a.kept + seq * a.out_stride + blk * kBlock;
  const int n = min(kBlock, keep - blk * kBlock);
  const size_t head = static_cast<size_t>(kBlock) * hd, stride = head * a.Hkv;
  const uint16_t* kp = a.pool + static_cast<size_t>(layer) * 2 * a.n_blocks * stride + hk * head;
  const uint16_t* vp = kp + static_cast<size_t>(a.n_blocks) * stride;
  const size_t to = static_cast<size_t>(a.dst_tbl[info[3] + blk]) * stride;
  for (int i = threadIdx.x; i < n * (hd / 8); i += blockDim.x) {
    const int t = i / (hd / 8), e = i % (hd / 8) * 8;
    const int s = kept[t];
    const size_t from = static_cast<size_t>(src_tbl[s / kBlock]) * stride;
    *reinterpret_cast<u32x4*>(const_cast<uint16_t*>(kp) + to + kv_k_index(t, e)) =
        *reinterpret_cast<const u32x4*>(kp + from + kv_k_index(s % kBlock, e));
  }
  for (int i = threadIdx.x; i < n * hd; i += blockDim.x) {
    const int t = i / hd, e = i % hd;
    const int s = kept[t];
    const size_t from = static_cast<size_t>(src_tbl[s / kBlock]) * stride;
    const_cast<uint16_t*>(vp)[to + kv_v_index(t, e)] = vp[from + kv_v_index(s % kBlock, e)];
  }
}

hipError_t launch_evict(const EvictArgs& a, int n, int max_keep, hipStream_t s) {
  hipLaunchKernelGGL(k_evict_select, dim3(n), dim3(kSelThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_evict_move, dim3((max_keep + kBlock - 1) / kBlock, a.n_layers * a.Hkv, n), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace vsk
