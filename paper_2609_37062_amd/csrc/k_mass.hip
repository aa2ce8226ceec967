// Attention weight per cached key: what the rows of a pass, over all query
// heads, gave each key of their sequence.
//
//   mass[t] = sum over rows r that see key t, heads h of 2^(s_rht - m_rh) / l_rh
//
// with s the base-2 score and (m, 1 / l) what the attention of these rows left
// for each (row, head).  Scores are taken again from K and q with the
// attention's own products, or are its own, and exponents as it takes them: a
// weight is the term that the softmax summed, to 2^-11 of it (kSpanRounded: an
// exponent by a fma or rounded) and exactly at the largest scores.  Every sum is
// taken in a fixed order: no atomics, so results do not change from run to run.
//
// k_attn_mass, for sequences of one row: a workgroup owns 32 keys of a sequence
// and sums over every head and row, each wave a run of (KV head, 16-column tile)
// units.  It reads K once more, and that bounds it.  So the attention of such
// rows leaves its scores where the workspace has room for them, 4 bytes a (head,
// key) beside 4 hd of K and V a (KV head, key), and k_mass_scores sums over
// those instead: 32 sequences of 1,000-4,000 tokens (32/8 heads x 128) 32 us of
// its own; with the scores the attention takes 60 instead of 54 and their sum 5.
// (Prompt rows that are attended one a work item have theirs taken so too.)
//
// k_mass_rows, for sequences of several rows: a product of K with all the
// queries that see it, 2 hd flops for each (row, head, key) where the attention
// has 4, and an exponential.  A workgroup of four waves owns 128 keys of a KV
// head, 32 a wave, which stay in registers as the operand of
// v_mfma_f32_32x32x16_bf16; the queries pass by in tiles of as many whole rows
// as have 32 (row, head) columns, copied straight into LDS three tiles ahead,
// one read for all four waves.  (Whole rows: what a lane copies then lies at a
// constant offset from the tile's first row.)  Each wave sums its keys' weights
// per lane and across lanes once at the end.  The KV heads, and parts of the rows
// where there are few keys, are added up by k_mass_sum.  777 rows over 2,300
// cached tokens (32/8 heads x 128): 196 us as k_attn_mass (every workgroup read
// every query, 16 columns at a time), 41 with loads through registers and columns
// that ran on over rows (139 vector operations a tile of 32 x 32, 48 of them the
// exponentials), 33 so, and 4.5 for the sum (30 and 4.6 among a thousand
// calls).  64 keys a wave, which halve the reads of LDS, took 36: two waves a SIMD
// hide less.  The grid is the list of the sequences' 128-key runs: as the longest
// sequence times all of them, 20 rows of 100 tokens beside 64 single rows of up to
// 16,000 launched a million workgroups for 128, 523 us a call against 445.
#include <climits>

#include "attn_core.hpp"

namespace vsk {

constexpr int kMassWaves = 8;

// ROWS: of the listed rows, a sequence each; else of the listed tiles.
template <int D, bool ROWS>
__global__ __launch_bounds__(64 * kMassWaves) void k_attn_mass(AttnMassArgs a) {
  constexpr int KC = D / 32;
  __shared__ float s_sum[kMassWaves][32];
  const int32_t* tile = a.tiles + 2 * (blockIdx.x / (kMassTile / 32));
  const int seq = ROWS ? a.row_seq[a.rows[blockIdx.y]] : tile[0];
  const int kv_len = a.kv_len[seq];
  const int t0 = ROWS ? 32 * blockIdx.x : tile[1] + 32 * (blockIdx.x % (kMassTile / 32));
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
    // (1 / l is 0 for a Project-Only row, which has no weights: 0 x NaN would be one)
    const uint32_t bits =
        on && ml.y != 0.f ? span_bits(t0 + 8 * quad, end, a.window > 0 && end > a.window ? end - a.window : 0, a.sinks) : 0u;
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

// One workgroup per 256 keys of a sequence, four keys a lane, its four waves
// sharing the heads; the waves' sums are added in order.
__global__ __launch_bounds__(256) void k_mass_scores(AttnMassArgs a) {
  __shared__ float4 s_sum[4][64];
  const int row = a.rows[blockIdx.y], seq = a.row_seq[row];
  const int kv_len = a.kv_len[seq];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t0 = 256 * blockIdx.x;
  if (t0 >= kv_len) return;
  const int t = t0 + 4 * lane, b = t / kBlock;
  const SpanWalk span = span_walk(kv_len, kv_len, a.window, a.sinks);
  const bool in = t < kv_len && (b < span.ns || b >= span.wb);
  const int v = (b < span.ns ? b : b - span.wb + span.ns) * kBlock + t % kBlock;  // its place in the list
  const int heads = a.Nq / a.hd;
  const float* sp = a.scores + static_cast<int64_t>(blockIdx.y) * heads * a.scores_len + (in ? v : 0);
  const float2* mlp = a.ml + static_cast<int64_t>(row) * heads;
  float y[4] = {0.f, 0.f, 0.f, 0.f};
  constexpr int kU = 4;  // heads in flight
  for (int h0 = w; h0 < heads; h0 += 4 * kU) {
    float4 s[kU];
    float2 ml[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int h = min(h0 + 4 * u, heads - 1);
      s[u] = *reinterpret_cast<const float4*>(sp + static_cast<int64_t>(h) * a.scores_len);
      ml[u] = mlp[h];
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      // (both sides of a difference rounded alike, see pair_softmax; a
      // Project-Only row has no scores, and nothing to sum)
#pragma clang fp contract(off)
      const bool on = h0 + 4 * u < heads && ml[u].y != 0.f;
      const float x[4] = {s[u].x, s[u].y, s[u].z, s[u].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float z = x[j] * a.scale_log2;
        const float e = __builtin_amdgcn_exp2f(z - ml[u].x) * ml[u].y;
        y[j] += on ? e : 0.f;
      }
    }
  }
  s_sum[w][lane] = make_float4(y[0], y[1], y[2], y[3]);
  __syncthreads();
  if (w != 0) return;
  float z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 x = s_sum[i][lane];
    z[0] += x.x; z[1] += x.y; z[2] += x.z; z[3] += x.w;
  }
  // (what the row does not see has no weight from it, also where the row's sum
  // is not finite and 2^-infinity times it would be NaN)
  float* dst = a.mass + seq * a.stride + t;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const bool seen = t + j >= span.lo || t + j < a.sinks;
    if (t + j < kv_len) dst[j] = (a.add != 0 ? dst[j] : 0.f) + (seen ? z[j] : 0.f);
  }
}

constexpr int kMassCols = 32;  // columns of a tile
constexpr int kMassSlots = 4;  // tiles in LDS
constexpr int kMassLead = 3;   // of them under way
static_assert(kMassLead < kMassSlots, "a slot for the tile that is read");

template <int D>
__global__ __launch_bounds__(256, 3) void k_mass_rows(AttnMassArgs a) {
  constexpr int QC = D / 16;   // operands of a tile
  constexpr int P = D / 8;     // 16-byte pieces of a query
  constexpr int LD = kMassCols * P / 256;  // of a tile's, a thread
  // a column's pieces lie in groups of four, [group][column][four]; the four in
  // an order by column, so that 16 lanes that read the same piece of as many
  // columns take 16 different 16-byte bank groups
  __shared__ u32x4 s_q[kMassSlots][P / 4][kMassCols][4];
  __shared__ float2 s_ml[kMassSlots][4][kMassCols];  // (every wave its own)
  auto order = [](int c) { return c >> 2 & 3; };
  // KV heads fastest: an XCD then keeps few heads' queries in its L2
  const int hk = blockIdx.x % a.Hkv, tile = blockIdx.x / a.Hkv, part = blockIdx.y;
  const int seq = a.tiles[2 * tile], t0 = a.tiles[2 * tile + 1];
  const int kv_len = a.kv_len[seq];
  const int r0 = a.cu_q[seq], n = a.cu_q[seq + 1] - r0;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lc = lane & 31, hi = lane >> 5, G = a.G;
  const int p0 = kv_len - n;  // position of the first row
  // the rows that see any of the 128 keys (see k_attn_mass), and of them this
  // part's tiles, of as many whole rows as fit
  const int ra = max(0, t0 - p0);
  const int rb = a.window > 0 && t0 >= a.sinks ? min(n, t0 + kMassTile - 1 + a.window - p0) : n;
  const int Rt = kMassCols / G;
  const int all = max(0, rb - ra + Rt - 1) / Rt;
  const int per = (all + a.parts - 1) / a.parts;
  const int i0 = min(all, part * per), tiles = min(all, i0 + per) - i0;
  const int r_first = ra + i0 * Rt;

  // K of the wave's 32 keys (blocks past the sequence: its last one again)
  const int nb = (kv_len + kBlock - 1) / kBlock;
  const int tw = t0 + 32 * w, bl = tw / kBlock;
  u32x4 kt[QC];
  {
    const int32_t* table = a.block_table + static_cast<size_t>(seq) * a.max_blocks;
    const size_t head = static_cast<size_t>(kBlock) * D, stride = head * a.Hkv;
    const size_t blk = table[min(bl + (lc >> 4), nb - 1)];
    const u32x4* kp = reinterpret_cast<const u32x4*>(a.pool + (static_cast<size_t>(a.layer) * 2 * a.n_blocks + blk) * stride +
                                                     hk * head) + (lane & 15) + 16 * hi;
#pragma unroll
    for (int i = 0; i < QC; ++i) kt[i] = kp[32 * i];
  }
  // a tile's queries: the wave's 64 LD pieces from 64 LD w on, LD a lane, at the
  // same places of every tile
  const int row_bytes = 2 * a.Nq, ml_bytes = 8 * a.Hkv * G;
  int qr[LD], qo[LD];  // row in the tile, byte in the row
#pragma unroll
  for (int j = 0; j < LD; ++j) {
    const int x = 64 * (LD * w + j) + lane, c = min(x / 4 % kMassCols, Rt * G - 1);
    qr[j] = c / G;
    qo[j] = 2 * (c % G * D + 8 * (x / 128 * 4 + (x % 4 ^ order(x / 4 % kMassCols))));
  }
  const int mc = min(lane / 2, Rt * G - 1);  // the column whose (m, 1 / l) the lane copies half of
  const int mr = mc / G, mo = 8 * (mc % G) + 4 * (lane % 2);
  const char* qh = reinterpret_cast<const char*>(a.q + static_cast<size_t>(r0) * a.Nq + static_cast<size_t>(hk) * G * D);
  const char* mlh = reinterpret_cast<const char*>(a.ml + static_cast<size_t>(r0) * (a.Hkv * G) + hk * G);
  const uint32_t q_lds = lds_address(&s_q[0][0][0][0]) + 1024 * LD * w, ml_lds = lds_address(&s_ml[0][w][0]);
  constexpr int kTileLoads = LD + 1;
  // tile i's copies into its slot (rows past the last one: it again, nobody
  // counts them)
  auto copy = [&](int i) __attribute__((always_inline)) {
    const int first = min(r_first + Rt * i, n - 1), last = n - 1 - first, slot = i % kMassSlots;
    const char* q0 = qh + static_cast<size_t>(first) * row_bytes;
    const char* m0 = mlh + static_cast<size_t>(first) * ml_bytes;
#pragma unroll
    for (int j = 0; j < LD; ++j)
      lds_copy16<false>(q0, __umul24(min(qr[j], last), row_bytes) + qo[j],
                        q_lds + static_cast<uint32_t>(slot * sizeof(s_q[0]) + 1024 * j));
    lds_copy4(m0, __umul24(min(mr, last), ml_bytes) + mo, ml_lds + static_cast<uint32_t>(slot * sizeof(s_ml[0])));
  };
  // tiles of whose rows all see the wave's 32 keys start at rows f_from .. f_to:
  // the first one is at key tw + 31 or behind it, and the window of the last
  // one reaches back to key tw
  const int f_from = tw + 32 <= kv_len ? tw + 31 - p0 : INT_MAX;
  const int f_to = min(rb, a.window == 0 || tw + 32 <= a.sinks ? INT_MAX : tw + a.window - p0) - Rt;
  const int cr = lc / G;  // the lane's column's row in its tile (Rt: none)
  const bool c_on = lc < Rt * G;  // (else it counts nowhere: no bits, and times zero in full tiles)
  const float sc = a.scale_log2;
  float acc[16];
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = 0.f;
  // a tile's scores: s[r] is key tw + 8 hi + r (r < 8), tw + 16 + 8 hi + r - 8
  f32x16 s;
  float2 ml;
  auto scores = [&](int i) __attribute__((always_inline)) {
    // the tile's copies have landed once at most those of the kMassLead - 1
    // tiles behind it are under way; the barrier publishes them and frees the
    // slot of the tile before
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((kMassLead - 1) * kTileLoads) : "memory");
    barrier_after_lds_reads();
    copy(i + kMassLead);
    ml = s_ml[i % kMassSlots][w][lc];
    ml.y = c_on ? ml.y : 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
    for (int c = 0; c < QC; ++c) {
      s = mfma_32x32x16(kt[c], s_q[i % kMassSlots][c / 2][lc][(2 * (c % 2) + hi) ^ order(lc)], s);
    }
  };
  if (tiles > 0) {
#pragma unroll
    for (int j = 0; j < kMassLead; ++j) copy(j);
    int i = 0;
    scores(0);
    while (i < tiles) {
      // (a loop of its own, so that the sums stay where they are)
      while (r_first + Rt * i >= f_from && r_first + Rt * i <= f_to && !__any(fabsf(ml.x) >= kSpanRounded)) {
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[r] = fmaf(__builtin_amdgcn_exp2f(fmaf(s[r], sc, -ml.x)), ml.y, acc[r]);
        if (++i == tiles) break;
        scores(i);
      }
      if (i == tiles) break;
      {
        // (both sides of a difference rounded alike, see pair_softmax)
#pragma clang fp contract(off)
        const int row = r_first + Rt * i + cr, p = p0 + row;
        // (1 / l is 0 for columns without weights.  Behind the tile's rows they are
        // copies of its last one, under the next row's index: that row's own key
        // may be far above the copy's maximum, and 0 x infinity is NaN.  A
        // Project-Only row's keys may hold anything)
        const int end = ml.y != 0.f && row < rb ? min(kv_len, p + 1) : 0;
        const int lo = a.window > 0 && p + 1 > a.window ? p + 1 - a.window : 0;
        const uint32_t bits =
            span_bits(tw + 8 * hi, end, lo, a.sinks) | span_bits(tw + kBlock + 8 * hi, end, lo, a.sinks) << 8;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float x = s[r] * sc;
          const float y = __builtin_amdgcn_exp2f(x - ml.x) * ml.y;
          acc[r] += bits >> r & 1u ? y : 0.f;
        }
      }
      if (++i == tiles) break;
      scores(i);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (the copies past the last tile)
  }
  // The sums over the 32 columns: lanes trade halves of their keys, so that 16
  // sums of 16 lanes become one each of 2
  float y[8];
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const auto z = __builtin_amdgcn_permlane16_swap(__float_as_uint(acc[r]), __float_as_uint(acc[r + 8]), false, false);
    y[r] = __uint_as_float(z[0]) + __uint_as_float(z[1]);  // lanes 16 .. 31 of 32: key r + 8's
  }
#pragma unroll
  for (int x = 8; x > 1; x >>= 1)
#pragma unroll
    for (int r = 0; r < x / 2; ++r) {
      const float mine = lane & x ? y[r + x / 2] : y[r], theirs = lane & x ? y[r] : y[r + x / 2];
      y[r] = mine + shfl_xor(theirs, x);
    }
  y[0] += shfl_xor(y[0], 1);
  if ((lane & 1) == 0)  // (keys past the sequence's end have a place too)
    a.part[(static_cast<size_t>(part * a.Hkv + hk) * a.n_tiles + tile) * kMassTile + 32 * w + 8 * hi + 16 * (lc >> 4) +
           (lane >> 1 & 7)] = y[0];
}

// mass = (or +=) the sum over KV heads and parts, a workgroup a tile.
__global__ __launch_bounds__(kMassTile) void k_mass_sum(AttnMassArgs a) {
  const int seq = a.tiles[2 * blockIdx.x], t = a.tiles[2 * blockIdx.x + 1] + threadIdx.x;
  if (t >= a.kv_len[seq]) return;
  const int n = a.Hkv * a.parts;
  const size_t next = static_cast<size_t>(a.n_tiles) * kMassTile;
  const float* p = a.part + static_cast<size_t>(blockIdx.x) * kMassTile + threadIdx.x;
  float* dst = a.mass + seq * a.stride + t;
  float y = 0.f;
  for (int i = 0; i < n; i += 8) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = p[min(i + j, n - 1) * next];
#pragma unroll
    for (int j = 0; j < 8; ++j) y += i + j < n ? v[j] : 0.f;
  }
  *dst = (a.add != 0 ? *dst : 0.f) + y;
}

template <int D>
static hipError_t launch_mass_d(const AttnMassArgs& a, int64_t* wgs, hipStream_t s) {
  hipError_t e;
  *wgs = 0;
  auto launch = [&](auto kernel, dim3 grid, int threads) {
    *wgs += static_cast<int64_t>(grid.x) * grid.y;
    hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, s, a);
    return hipGetLastError();
  };
  // sequences of one row first: the scores lie where the others' parts go
  if (a.n_rows > 0) {
    e = a.scores != nullptr ? launch(k_mass_scores, dim3((a.max_len + 255) / 256, a.n_rows), 256)
                            : launch(k_attn_mass<D, true>, dim3((a.max_len + 31) / 32, a.n_rows), 64 * kMassWaves);
    if (e != hipSuccess) return e;
  }
  if (a.n_tiles == 0) return hipSuccess;
  if (a.parts == 0) return launch(k_attn_mass<D, false>, dim3(a.n_tiles * (kMassTile / 32)), 64 * kMassWaves);
  if ((e = launch(k_mass_rows<D>, dim3(a.n_tiles * a.Hkv, a.parts), 256)) != hipSuccess) return e;
  return launch(k_mass_sum, dim3(a.n_tiles), kMassTile);
}

hipError_t launch_attn_mass(const AttnMassArgs& a, int head_dim, int64_t* wgs, hipStream_t s) {
  if (head_dim == 128) return launch_mass_d<128>(a, wgs, s);
  if (head_dim == 64) return launch_mass_d<64>(a, wgs, s);
  return hipErrorInvalidValue;
}

}  // namespace vsk
