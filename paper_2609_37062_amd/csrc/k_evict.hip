// Eviction of cached tokens by accumulated attention weight.
//
// k_evict_select: one workgroup per sequence.  Kept are the first `sinks` and
// the last `recent` tokens and, of those between, the ones of the largest
// weights (equal weights: lowest index; NaN below everything), listed in
// index order.  The smallest kept weight is found by radix select over the
// weights' order-preserving 32-bit keys, digits of 11, 11 and 10 bits, the keys
// held in registers; ranks come from block-wide prefix sums.  Everything is whole
// numbers, so nothing depends on an order of arrival.
//
// k_evict_move: copies K and V of the kept tokens, every layer and KV head, to
// the destination's blocks.
//
// k_evict_small: both, for a few short sequences.
#include <cstring>
#include <type_traits>

#include "dev.hpp"
#include "evict.hpp"

namespace vsk {

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

// Exclusive prefix sum, in place, over N <= 256 counts in LDS, by every thread's call.
template <int N>
__device__ __forceinline__ void scan_counts(int* s) {
  constexpr int E = (N + 63) / 64;
  __syncthreads();
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x;
    int c[E], sum = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      c[e] = lane * E + e < N ? s[lane * E + e] : 0;
      sum += c[e];
    }
    int x = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(x, d, 64);
      if (lane >= d) x += y;
    }
    x -= sum;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (lane * E + e < N) s[lane * E + e] = x;
      x += c[e];
    }
  }
  __syncthreads();
}

// Token i = j T + thread is the thread's j-th: loads and stores then run along
// the tokens.  (Runs of tokens a thread: 34 us at 16,000 tokens, most of it
// 4-byte stores to 64 lines an instruction; this order 26.)
// M is EvictSmall, or int where the metadata is in its buffer already.
template <int T, int PER, typename M>
__global__ __launch_bounds__(T) void k_evict_select(EvictArgs a, M meta) {
  constexpr int W = T / 64;
  constexpr bool kSmall = std::is_same_v<M, EvictSmall>;
  __shared__ int s_hist[2048];
  __shared__ int s_w[W];
  __shared__ int s_tie[PER * W], s_stay[PER * W];  // counts of 64 tokens each, in index order
  __shared__ uint32_t s_digit;
  __shared__ int s_left;
  const int seq = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int32_t* info = a.info + 4 * seq;
  const int32_t* src_tbl = a.src_tbl;
  const int32_t* dst_tbl = a.dst_tbl;
  if constexpr (kSmall) {
    // (every sequence's workgroup stores all of it: the same values)
    for (int i = tid; i < a.n_ints; i += T) a.info[i] = meta.v[i];
    info = meta.v + 4 * seq;
    src_tbl = meta.v + (a.src_tbl - a.info);
    dst_tbl = meta.v + (a.dst_tbl - a.info);
  }
  const int len = info[0], keep = info[1];
  src_tbl += info[2];
  dst_tbl += info[3];
  int32_t* from = a.from + static_cast<int64_t>(info[3]) * kBlock;
  const float* mass = a.mass + seq * a.mass_stride;
  const int lo = a.sinks, hi = len - a.recent;  // the tokens that compete
  float v[PER];
  uint32_t key[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = j * T + tid;
    v[j] = i < len ? mass[i] : 0.f;
    key[j] = mass_key(v[j]);
  }
  auto competes = [&](int j) { return j * T + tid >= lo && j * T + tid < hi; };
  const int left0 = keep - a.sinks - a.recent;  // how many of them stay
  int left = left0;                             // and of those whose key starts with `top`
  uint32_t top = 0;                             // the smallest kept key, as far as it is known
  const bool all = left0 >= hi - lo;            // (uniform)
  if (left0 > 0 && !all) {
#pragma unroll
    for (int d = 0; d < 3; ++d) {
      constexpr int kShift[3] = {21, 10, 0}, kBits[3] = {11, 11, 10};
      const int shift = kShift[d], bins = 1 << kBits[d];
      for (int b = tid; b < bins; b += T) s_hist[b] = 0;
      __syncthreads();
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        // equal keys (zeros, above all) would queue at one counter: the lanes
        // that agree with the first one are counted together
        const bool in = competes(j) && (d == 0 || key[j] >> (shift + kBits[d]) == top >> (shift + kBits[d]));
        const uint64_t ins = __ballot(in);
        if (ins == 0) continue;
        const uint32_t first = __builtin_amdgcn_readlane(key[j], __builtin_ctzll(ins));
        const uint64_t same = __ballot(in && key[j] == first);
        if (lane == 0) atomicAdd(&s_hist[first >> shift & (bins - 1)], static_cast<int>(__popcll(same)));
        if (in && key[j] != first) atomicAdd(&s_hist[key[j] >> shift & (bins - 1)], 1);
      }
      __syncthreads();
      // bins from the largest down, `own` of them a thread
      const int own = bins / T;
      int sum = 0;
      for (int b = 0; b < own; ++b) sum += s_hist[bins - 1 - (tid * own + b)];
      int above = block_before(sum, s_w);
      if (above < left && above + sum >= left) {
        int b = bins - 1 - tid * own;
        while (above + s_hist[b] < left) above += s_hist[b--];
        s_digit = b;
        s_left = left - above;
      }
      __syncthreads();
      top |= s_digit << shift;
      left = s_left;
    }
  }
  // above `top` every token stays, of those at `top` the first `left`
  const uint64_t before = (1ull << lane) - 1ull;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int n = __popcll(__ballot(competes(j) && key[j] == top));
    if (lane == 0) s_tie[j * W + w] = n;
  }
  scan_counts<PER * W>(s_tie);
  uint32_t stays = 0;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = j * T + tid;
    const uint64_t ties = __ballot(competes(j) && key[j] == top);
    bool s = i < len && (i < lo || i >= hi || all);
    if (left0 > 0 && competes(j))
      s = s || key[j] > top || (key[j] == top && s_tie[j * W + w] + __popcll(ties & before) < left);
    stays |= static_cast<uint32_t>(s) << j;
    const int n = __popcll(__ballot(s));
    if (lane == 0) s_stay[j * W + w] = n;
  }
  scan_counts<PER * W>(s_stay);
  int32_t* kept = a.kept + seq * a.out_stride;
  // (mass_out may be mass itself: every weight has been read above, the scans'
  // barriers since)
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const bool s = stays >> j & 1u;
    const int at = s_stay[j * W + w] + __popcll(__ballot(s) & before);
    if (!s) continue;
    const int i = j * T + tid;
    kept[at] = i;
    from[at] = src_tbl[i / kBlock] * kBlock + i % kBlock;
    if (a.slots != nullptr) a.slots[seq * a.out_stride + at] = dst_tbl[at / kBlock] * kBlock + at % kBlock;
    if (a.mass_out != nullptr) a.mass_out[seq * a.out_stride + at] = v[j];
  }
  if (a.mass_out != nullptr)
    for (int64_t i = keep + tid; i < a.out_stride; i += T) a.mass_out[seq * a.out_stride + i] = 0.f;
}

// The 16-byte piece at place i of a destination block's K and V (2 hd places): 8
// dims of a token of K, 8 tokens of a dim of V, from the slots `from` of the
// block's n tokens.
__device__ __forceinline__ void move_piece(uint16_t* kp, uint16_t* vp, size_t stride, size_t to, const int32_t* from,
                                           int n, int i) {
  // K: its token's bits 2 and 3 are swapped, see kv_k_index
  const int p = i % kBlock, tk = (p & 3) | ((p & 4) << 1) | ((p & 8) >> 1), e = i / kBlock * 8;
  const int sk = from[min(tk, n - 1)];
  // V: dim and half
  const int ev = i / 32 * 16 + i % 16, t0 = i % 32 / 16 * 8;
  int sv[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) sv[j] = from[min(t0 + j, n - 1)];
  const u32x4 x = *reinterpret_cast<const u32x4*>(kp + (sk >> 4) * stride + kv_k_index(sk & 15, e));
  uint32_t y[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) y[j] = vp[(sv[j] >> 4) * stride + kv_v_index(sv[j] & 15, ev)];
  // (the block is the sequence's own: its slots behind the last token may hold anything)
  *reinterpret_cast<u32x4*>(kp + to + i * 8) = x;
  *reinterpret_cast<u32x4*>(vp + to + i * 8) =
      u32x4{y[0] | y[1] << 16, y[2] | y[3] << 16, y[4] | y[5] << 16, y[6] | y[7] << 16};
}

// One workgroup per destination block of a layer and KV head, one thread per
// piece.  Lanes run along what is contiguous in the pool: the tokens of K
// pieces, the dims of V pieces.  A line of the pool holds eight tokens of K, or
// eight tokens of eight dims of V, so where few tokens stay the lines read are
// more than the bytes moved: with one in five kept, 85% of the source.
__global__ __launch_bounds__(256) void k_evict_move(EvictArgs a) {
  const int seq = blockIdx.z, layer = blockIdx.y / a.Hkv, hk = blockIdx.y % a.Hkv;
  const int32_t* info = a.info + 4 * seq;
  const int keep = info[1], hd = a.hd;
  const int blk = blockIdx.x;  // destination block
  if (blk * kBlock >= keep) return;
  const size_t head = static_cast<size_t>(kBlock) * hd, stride = head * a.Hkv;
  uint16_t* kp = a.pool + static_cast<size_t>(layer) * 2 * a.n_blocks * stride + hk * head;
  uint16_t* vp = kp + static_cast<size_t>(a.n_blocks) * stride;
  const size_t to = static_cast<size_t>(a.dst_tbl[info[3] + blk]) * stride;
  move_piece(kp, vp, stride, to, a.from + (static_cast<int64_t>(info[3]) + blk) * kBlock,
             min(kBlock, keep - blk * kBlock), threadIdx.x);
}

// Both at once for short sequences: every workgroup (a KV head's run of
// kSmallRun destination blocks of a layer and sequence) makes the selection for
// itself, a wave alone -- the smallest kept key bit by bit, counted by ballots --
// and moves its blocks.  One launch instead of two that depend on each other:
// 96 of 201 tokens, one layer of 4 heads x 64, 6.5 us instead of 6.7 and 3.3.
// With many workgroups the selections made again cost more than the launch (calls
// with the cache read back, 400 of 512 tokens of 8 heads x 128: 4 layers, 224
// workgroups, 36 us and 47-53 apart; 16 layers, 896, 127 and 125; 8 sequences,
// 2,048, 160 and 151).
constexpr int kSmallLen = 512;  // tokens
constexpr int kSmallRun = 4;
constexpr int kSmallWgs = 512;
__global__ __launch_bounds__(256) void k_evict_small(EvictArgs a, EvictSmall meta) {
  constexpr int PER = kSmallLen / 64;
  __shared__ int32_t s_from[kSmallRun * kBlock];
  const int seq = blockIdx.z, layer = blockIdx.y, hk = blockIdx.x % a.Hkv, run = blockIdx.x / a.Hkv;
  const int32_t* info = meta.v + 4 * seq;
  const int len = info[0], keep = info[1];
  const int first = run * kSmallRun * kBlock;  // of the run's kept tokens
  if (first >= keep) return;
  const int32_t* src_tbl = meta.v + (a.src_tbl - a.info) + info[2];
  const int32_t* dst_tbl = meta.v + (a.dst_tbl - a.info) + info[3];
  const int tid = threadIdx.x, lane = tid & 63;
  if (tid < 64) {
    const float* mass = a.mass + seq * a.mass_stride;
    const int lo = a.sinks, hi = len - a.recent;  // the tokens that compete
    const int left0 = keep - a.sinks - a.recent;  // how many of them stay
    // token 64 q + lane; `in` the ones that compete
    float v[PER];
    uint32_t key[PER];
    uint64_t in[PER];
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      const int i = 64 * q + lane;
      v[q] = i < len ? mass[i] : 0.f;
      key[q] = mass_key(v[q]);
      in[q] = __ballot(i >= lo && i < hi);
    }
    auto at_least = [&](uint32_t k) {
      int n = 0;
#pragma unroll
      for (int q = 0; q < PER; ++q) n += __popcll(__ballot(key[q] >= k) & in[q]);
      return n;
    };
    uint32_t top = 0;  // at least left0 keys are as large
    int n = max(0, hi - lo);
    for (uint32_t bit = 1u << 31; bit != 0 && n != left0; bit >>= 1) {
      const int m = at_least(top | bit);
      if (m >= left0) {
        top |= bit;
        n = m;
      }
    }
    // n of them: where that is more, the ones equal to `top` stay by index
    int ties = left0 - (n == left0 ? 0 : at_least(top + 1));  // (top + 1 is at most NaN's ~0)
    const bool cut = n != left0;
    int at0 = 0;
    const uint64_t before = (1ull << lane) - 1ull;
    const bool writes = layer == 0 && hk == 0 && run == 0;
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      const int i = 64 * q + lane;
      uint64_t chosen = __ballot(left0 > 0 && key[q] >= top) & in[q];
      if (cut) {
        const uint64_t equal = __ballot(key[q] == top) & in[q];
        const int mine = __popcll(equal & before);
        chosen &= ~(equal & __ballot(mine >= ties));
        ties = max(0, ties - static_cast<int>(__popcll(equal)));
      }
      const uint64_t stay = chosen | __ballot(i < len && (i < lo || i >= hi));
      const int at = at0 + __popcll(stay & before);
      at0 += __popcll(stay);
      if (!(stay >> lane & 1u)) continue;
      if (at >= first && at < first + kSmallRun * kBlock) s_from[at - first] = src_tbl[i / kBlock] * kBlock + i % kBlock;
      if (!writes) continue;
      a.kept[seq * a.out_stride + at] = i;
      if (a.slots != nullptr) a.slots[seq * a.out_stride + at] = dst_tbl[at / kBlock] * kBlock + at % kBlock;
      if (a.mass_out != nullptr) a.mass_out[seq * a.out_stride + at] = v[q];
    }
    if (writes && a.mass_out != nullptr)
      for (int64_t i = keep + lane; i < a.out_stride; i += 64) a.mass_out[seq * a.out_stride + i] = 0.f;
  }
  __syncthreads();
  const int hd = a.hd;
  const size_t head = static_cast<size_t>(kBlock) * hd, stride = head * a.Hkv;
  uint16_t* kp = a.pool + static_cast<size_t>(layer) * 2 * a.n_blocks * stride + hk * head;
  uint16_t* vp = kp + static_cast<size_t>(a.n_blocks) * stride;
  for (int x = tid; x < kSmallRun * 2 * hd; x += 256) {
    const int b = x / (2 * hd), n = min(kBlock, keep - first - b * kBlock);
    if (n > 0)
      move_piece(kp, vp, stride, static_cast<size_t>(dst_tbl[first / kBlock + b]) * stride, s_from + b * kBlock, n,
                 x % (2 * hd));
  }
}

// Few tokens take few waves (cheaper rounds), and never more registers than tokens need.
template <typename M>
static void launch_select(const EvictArgs& a, const M& meta, int n, int max_len, hipStream_t s) {
  if (max_len <= 1024) hipLaunchKernelGGL((k_evict_select<256, 4, M>), dim3(n), dim3(256), 0, s, a, meta);
  else if (max_len <= 4096) hipLaunchKernelGGL((k_evict_select<1024, 4, M>), dim3(n), dim3(1024), 0, s, a, meta);
  else hipLaunchKernelGGL((k_evict_select<1024, kEvictMaxLen / 1024, M>), dim3(n), dim3(1024), 0, s, a, meta);
}

hipError_t launch_evict(const EvictArgs& a, const int32_t* meta, size_t ints, int n, int max_len, int max_keep,
                        hipStream_t s) {
  if (meta != nullptr) {
    if (ints > static_cast<size_t>(kEvictSmall)) return hipErrorInvalidValue;
    EvictSmall m;
    std::memset(&m, 0, sizeof(m));
    std::memcpy(m.v, meta, ints * 4);
    // (in place, another workgroup would read weights that one has replaced)
    const int runs = (max_keep + kSmallRun * kBlock - 1) / (kSmallRun * kBlock);
    if (max_len <= kSmallLen && a.mass_out != a.mass &&
        static_cast<int64_t>(runs) * a.Hkv * a.n_layers * n <= kSmallWgs) {
      hipLaunchKernelGGL(k_evict_small, dim3(runs * a.Hkv, a.n_layers, n), dim3(256), 0, s, a, m);
      return hipGetLastError();
    }
    launch_select(a, m, n, max_len, s);
  } else {
    launch_select(a, 0, n, max_len, s);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_evict_move, dim3((max_keep + kBlock - 1) / kBlock, a.n_layers * a.Hkv, n), dim3(2 * a.hd), 0, s, a);
  return hipGetLastError();
}

}  // namespace vsk
