// General attention of prompt rows: a sliding window with sinks, or every key,
// over the paged cache.
//
// One work item per (run of a sequence's consecutive new rows, KV head); its
// columns are the run's (row, query head) pairs, up to 128, 32 a wave.  Scores
// and outputs are taken transposed on v_mfma_f32_32x32x16_bf16: S^T = K q^T of
// 32 keys (two blocks) x 32 columns, O^T += V^T P^T.  A lane then holds 16
// scores of one column, and as the cache keeps K's tokens with bits 2 and 3
// swapped, these are tokens 8 h .. 8 h + 7 (h = lane / 32) of either block: what
// P^T's operand asks of that lane, with no exchange between lanes.
//
// Why 32 columns a wave: every wave reads the step's K and V from LDS, 16 KiB
// at head_dim 128.  With 16 columns (the passes' walk) eight waves read 128 KiB
// a step, at 128 bytes a cycle longer than the step's MFMAs take; with 32 a
// byte feeds twice the work.
//
// K and V are copied straight into four LDS slots, a wave one of a step's K or V
// blocks: at step i the copies of step i + 3 are issued and those of step i + 1
// waited for, with one barrier a step.  NH halves of a workgroup walk alternate
// pairs of blocks and are joined at the end: with few work items two halves keep
// two waves on each SIMD, with many one half and two workgroups do.  Fewer work
// items than compute units with long walks are cut into splits, which
// k_rows_join adds up in their order.
//
// What bounds it: at head_dim 128 a step of a wave is 24 MFMAs (8 of the scores,
// 16 of the outputs: a weight goes in as the sum of two bf16 terms) and a softmax
// of 108 vector operations and 16 exponentials.  So steps whose keys all count
// are a loop of their own, without a register that changes on a condition, in
// which the next step's scores are issued between this step's exponentials.
// 1,000 rows of 32/8 heads x 128 through a window of 4,096 took 184 us on
// 16-column tiles, 129 on these, 116 with that loop, 112 with the next step's
// scores in it, 103 with copies into LDS instead of loads and stores; 777 rows
// after 2,300 tokens 92, 84 with the loop, 79, 72; 4 x 1,037 rows of 24/8 through
// a window of 256, whose steps are mostly cut by a mask, 60, 45, 41, and 38 with
// masks as bit inserts and finite V left as it is.  (Few calls at a time; among a
// thousand 98, 63 and 37 now.)  These MFMAs with the same
// vector operations between them and nothing else, no memory, would take 82 of
// the 103: with all of them busy the chip runs 1.45 PFLOP/s.  One bf16 term a
// weight would be a fifth faster, at errors of 2^-9 a weight.
#include "attn_core.hpp"

namespace vsk {

constexpr int kRowTiles = 4;               // 32-column tiles of a work item
static_assert(kRowTiles * 32 == kPreCols, "a work item's columns");
// A running maximum may lag by this (base 2) before the sums are rescaled: the
// weights are then up to 2^8, the float32 sums as exact as before.
constexpr float kRowsLag = 8.f;
constexpr int kRowSlots = 4;
static_assert(kRowSlots == 4, "three steps of copies ahead of the one that is read");

// Some value of V (of any lane of the wave) is an infinity or a NaN.
template <int N>
__device__ __forceinline__ bool not_finite(const u32x4 (&v)[N]) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  u16x2 top = u16x2{0, 0};
#pragma unroll
  for (int c = 0; c < N; ++c)
#pragma unroll
    for (int j = 0; j < 4; ++j) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, v[c][j] & 0x7fff7fffu));
  return __any(top[0] >= 0x7f80 || top[1] >= 0x7f80);
}

// 0xffff in the halves that hold such a value.
__device__ __forceinline__ uint32_t not_finite_halves(uint32_t v) {
  return ((v & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((v & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}

// Eight bf16 values of which those with a clear bit become zero.
__device__ __forceinline__ u32x4 keep_bits(u32x4 v, uint32_t bits) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
    v[j] &= (bits >> (2 * j) & 1u ? 0x0000ffffu : 0u) | (bits >> (2 * j + 1) & 1u ? 0xffff0000u : 0u);
  return v;
}

template <int D, int NH>
struct RowsLds {
  u32x4 kv[kRowSlots][2][NH][2][2 * D];  // [slot][K, V][half][block][16-byte piece]
  int32_t tbl[kMaxSpanBlocks];
  float m[kRowTiles][64], l[kRowTiles][64];  // the second half's, when the halves join
};

template <int D, int NH>
__global__ __launch_bounds__(256 * NH, 2) void k_attn_rows(AttnPrefillArgs a) {
  constexpr int T = 256 * NH;
  constexpr int QC = D / 16;  // q and K operands of a step
  constexpr int OC = D / 32;  // tiles of 32 dims
  constexpr int kCopies = D / 32;  // 1 KiB copies of a wave's piece of a step
  __shared__ RowsLds<D, NH> sm;

  // an item's KV heads are consecutive, then its splits (items come longest walk first)
  const int hk = blockIdx.x % a.Hkv, split = static_cast<int>(blockIdx.x / a.Hkv) % a.splits;
  const int32_t* it = a.items + static_cast<size_t>(blockIdx.x / a.Hkv / a.splits) * 3;
  const int seq = it[0], row0 = it[1], n_rows = it[2];
  const int G = a.G, n_cols = n_rows * G;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ct = w % kRowTiles, hh = w / kRowTiles;
  const int lc = lane & 31, hi = lane >> 5;
  const int kv_end = a.kv_len[seq];
  const int pos0 = a.pos[row0];  // (a run's rows are consecutive positions)
  const SpanWalk span = span_walk(pos0 + 1, pos0 + n_rows, a.window, a.sinks);
  const int32_t* table = a.block_table + static_cast<size_t>(seq) * a.max_blocks;
  for (int i = tid; i < span.nv; i += T) sm.tbl[i] = table[span.block(i)];

  // this lane's column and what it sees: keys lo .. p and below sinks
  const int c = 32 * ct + lc;
  const bool on = c < n_cols;
  const int row = on ? c / G : 0, qh = on ? c % G : 0;
  const int end = on ? min(kv_end, pos0 + row + 1) : 0;
  auto first_key = [&](int n) { return a.window > 0 && n > a.window ? n - a.window : 0; };  // of a row with n keys
  const int lo = first_key(pos0 + row + 1);
  u32x4 qf[QC];
  {
    const uint16_t* qrow = a.q + static_cast<size_t>(row0 + row) * a.Nq + static_cast<size_t>(hk * G + qh) * D + 8 * hi;
#pragma unroll
    for (int s = 0; s < QC; ++s)
      qf[s] = on ? *reinterpret_cast<const u32x4*>(qrow + 16 * s) : u32x4{0u, 0u, 0u, 0u};
  }
  // the wave's part of the list (none without a column), and from where to
  // where a key counts for all its columns
  const bool has = 32 * ct < n_cols;
  const int ra = 32 * ct / G, rb = min(32 * ct + 31, n_cols - 1) / G;  // its first and last row
  const int full_end = min(kv_end, pos0 + ra + 1), full_lo = first_key(pos0 + rb + 1);

  const size_t head = static_cast<size_t>(kBlock) * D, stride = head * a.Hkv;
  const uint16_t* kbase = a.pool + static_cast<size_t>(a.layer) * 2 * a.n_blocks * stride + hk * head;
  const uint16_t* vbase = kbase + static_cast<size_t>(a.n_blocks) * stride;
  const int n_pairs = (span.nv + 1) / 2, all_steps = (n_pairs + NH - 1) / NH;
  const int per = (all_steps + a.splits - 1) / a.splits;
  const int first = min(all_steps, split * per), n_steps = min(all_steps, first + per);  // the split's: first .. n_steps - 1
  // A step's NH x two blocks x {K, V} are one each for a wave to copy into LDS.
  // Blocks past the list: its last one again (nobody counts their keys).
  const int my_blk = w >> 1;  // of the step's 2 NH
  const uint16_t* my_base = w & 1 ? vbase : kbase;
  const uint32_t my_lds = lds_address(&sm.kv[0][w & 1][w >> 2][w >> 1 & 1][0]);
  const uint32_t lane16 = 16 * lane;
  auto copy = [&](int step) __attribute__((always_inline)) {
    const uint32_t blk = __builtin_amdgcn_readfirstlane(sm.tbl[min(2 * NH * step + my_blk, span.nv - 1)]);
    const uint16_t* src = my_base + static_cast<uint64_t>(blk) * static_cast<uint32_t>(stride);
    const uint32_t dst = my_lds + static_cast<uint32_t>(step % kRowSlots * sizeof(sm.kv[0]));
#pragma unroll
    for (int j = 0; j < kCopies; ++j) lds_copy16<false>(src + 512 * j, lane16, dst + 1024 * j);
  };
  // until all but the newest `steps` steps' copies of this wave have landed
  auto landed = [&](auto steps) __attribute__((always_inline)) {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(decltype(steps)::value * kCopies) : "memory");
  };
  float m = -INFINITY, l = 0.f;
  f32x16 o[OC];
#pragma unroll
  for (int i = 0; i < OC; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
  const float sc = a.scale_log2;

  __syncthreads();  // tbl
  // Blocks of the list of which every key counts for all columns of the wave:
  // those before f_sinks, and f_from .. f_to - 1.
  const int f_sinks = min(a.sinks / kBlock, span.ns);
  const int f_from = (full_lo + kBlock - 1) / kBlock - span.wb + span.ns;
  const int f_to = full_end / kBlock - span.wb + span.ns;
  auto pair_of = [&](int step) { return 2 * (step * NH + hh); };  // a step's first block of the list
  auto is_full = [&](int step) {  // (uniform)
    const int v = pair_of(step);
    return v + 1 < f_to && (v >= f_from || v + 1 < f_sinks);
  };
  // of a lane's keys, those that its column sees, and those that the sequence has
  auto seen = [&](int step, int b) {
    const int v = pair_of(step) + b;
    return v < span.nv ? span_bits(kBlock * span.block(v) + 8 * hi, end, lo, a.sinks) : 0u;
  };
  auto held = [&](int step, int b) {
    const int v = pair_of(step) + b;
    return step >= 0 && v < span.nv ? span_bits(kBlock * span.block(v) + 8 * hi, kv_end, 0, 0) : 0u;
  };
  // V of a step of which some keys count for some columns only.  Where all of it
  // is finite, weights of zero leave the others out.  Otherwise keys of no token
  // become zero (slots past the sequence's end may hold a NaN, and 0 x NaN is
  // NaN), and so do values that are not finite ...
  bool poisoned = false;  // (uniform)
  auto clean = [&](int step, int b, u32x4 (&vt)[OC]) __attribute__((always_inline)) {
    if (__builtin_expect(not_finite(vt), 0)) {
      const uint32_t keep = held(step, b);
      poisoned = true;
#pragma unroll
      for (int i = 0; i < OC; ++i) {
        vt[i] = keep_bits(vt[i], keep);
#pragma unroll
        for (int j = 0; j < 4; ++j) vt[i][j] &= ~not_finite_halves(vt[i][j]);
      }
    }
  };
  // ... and here the columns that see one get NaN where it enters (rare)
  auto poison = [&](int step) __attribute__((always_inline)) {
    poisoned = false;
    const u32x4* vp = &sm.kv[step % kRowSlots][1][hh][0][32 * (lc >> 4) + (lane & 15) + 16 * hi];
#pragma unroll
    for (int i = 0; i < OC; ++i) {
      f32x16 y;  // how many such values of keys that the column sees
#pragma unroll
      for (int r = 0; r < 16; ++r) y[r] = 0.f;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        u32x4 x = vp[2 * D * b + 64 * i];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = not_finite_halves(x[j]) & 0x3f803f80u;  // 1.0
        y = mfma_32x32x16(x, keep_bits(u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u}, seen(step, b)), y);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) o[i][r] = y[r] != 0.f ? NAN : o[i][r];
    }
  };

  // O^T += V^T P^T of a step, block by block.  FAST: every key counts, the
  // maximum has not moved and no score is huge -- no branch and no change of a
  // register on a condition, which the compiler would pay for with copies of
  // all the sums in every step.
  auto rest = [&](int step, const f32x16& s, auto fast_c) __attribute__((always_inline)) {
    constexpr bool FAST = decltype(fast_c)::value;
    const u32x4* vp = &sm.kv[step % kRowSlots][1][hh][0][32 * (lc >> 4) + (lane & 15) + 16 * hi];
    const float mb = !FAST && m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      u32x4 vt[OC];
#pragma unroll
      for (int i = 0; i < OC; ++i) vt[i] = vp[2 * D * b + 64 * i];
      float p[8];
      if constexpr (FAST) {
#pragma unroll
        for (int r = 0; r < 8; ++r) p[r] = __builtin_amdgcn_exp2f(fmaf(s[8 * b + r], sc, -mb));
      } else {
        // both sides of a difference rounded alike (see pair_softmax)
#pragma clang fp contract(off)
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const float x = s[8 * b + r] * sc;
          p[r] = __builtin_amdgcn_exp2f(x - mb);
        }
      }
      l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      u32x4 pt[kSpanPTerms];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float r0 = p[2 * j], r1 = p[2 * j + 1];
#pragma unroll
        for (int t = 0; t < kSpanPTerms; ++t) {
          pt[t][j] = pack_bf2(r0, r1);
          r0 -= bf2f(pt[t][j]);
          r1 -= __uint_as_float(pt[t][j] & 0xffff0000u);
        }
      }
      if constexpr (!FAST) clean(step, b, vt);
#pragma unroll
      for (int t = 0; t < kSpanPTerms; ++t)
#pragma unroll
        for (int i = 0; i < OC; ++i) o[i] = mfma_32x32x16(vt[i], pt[t], o[i]);
    }
  };

#pragma unroll
  for (int j = 0; j < 3; ++j) copy(first + j);
  bool big = false;  // (uniform) scores so large that a fma's unrounded product would be off the maximum
  f32x16 s;          // s[r]: key 8 hi + r of the step's first block (r < 8), 8 hi + r - 8 of the second
  float mx;
  auto next = [&](int step) __attribute__((always_inline)) {
    landed(std::integral_constant<int, 1>{});
    barrier_after_lds_reads();  // the next step's slot is whole, the one of the last step free
    copy(step + 3);
  };
  auto qk = [&](int step, f32x16& s) __attribute__((always_inline)) {
    const u32x4* kp = &sm.kv[step % kRowSlots][0][hh][lc >> 4][(lane & 15) + 16 * hi];
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
    for (int i = 0; i < QC; ++i) s = mfma_32x32x16(kp[32 * i], qf[i], s);
  };
  auto top = [&](const f32x16& s) __attribute__((always_inline)) {
    float x = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) x = fmaxf(x, s[r]);
    return max_xor32(x) * sc;
  };
  int step = first;
  landed(std::integral_constant<int, 2>{});
  barrier_after_lds_reads();
  qk(step, s);
  mx = top(s);
  while (step < n_steps) {
    // (a loop of its own, so that the sums stay where they are)
    while (is_full(step) && !big && !__any(mx > m + kRowsLag)) {  // (-inf + 8 is -inf: first keys always are)
      next(step);
      f32x16 sn;
      qk(step + 1, sn);
      rest(step, s, std::true_type{});
      s = sn;
      mx = top(s);
      if (++step == n_steps) break;
    }
    if (step == n_steps) break;
    if (!is_full(step)) {
      const uint32_t bits = seen(step, 0) | seen(step, 1) << 8;
      mx = -INFINITY;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[r] = bit_or_neg_inf(s[r], bits, r);
        mx = fmaxf(mx, s[r]);
      }
      mx = max_xor32(mx) * sc;
    }
    if (__any(mx > m + kRowsLag)) {
      const float mn = fmaxf(m, mx);
      const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= f;
#pragma unroll
      for (int i = 0; i < OC; ++i) o[i] *= f;
      big = __any(fabsf(m) >= kSpanRounded && m != -INFINITY);
    }
    next(step);
    rest(step, s, std::false_type{});
    if (__builtin_expect(poisoned, 0)) poison(step);
    if (++step == n_steps) break;
    qk(step, s);
    mx = top(s);
  }
  l = add_xor32(l);
  landed(std::integral_constant<int, 0>{});  // (the steps past the list: before LDS is used again or ends)

  if constexpr (NH == 2) {  // the second half's sums join the first's
    static_assert(sizeof(sm.kv) >= kRowTiles * OC * 16 * 64 * 4, "space for a half's sums");
    float* so = reinterpret_cast<float*>(&sm.kv[0][0][0][0][0]) + ct * OC * 16 * 64 + lane;
    __syncthreads();
    if (hh == 1) {
#pragma unroll
      for (int i = 0; i < OC; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) so[(i * 16 + r) * 64] = o[i][r];
      sm.m[ct][lane] = m;
      sm.l[ct][lane] = l;
    }
    __syncthreads();
    if (hh == 1) return;
    const float m2 = sm.m[ct][lane], l2 = sm.l[ct][lane];
    const float M = fmaxf(m, m2);
    const float f0 = m == -INFINITY ? 0.f : exp2f(m - M), f1 = m2 == -INFINITY ? 0.f : exp2f(m2 - M);
    m = M;
    l = l * f0 + l2 * f1;
#pragma unroll
    for (int i = 0; i < OC; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[i][r] = o[i][r] * f0 + so[(i * 16 + r) * 64] * f1;
  }
  if (!has) return;
  // a Project-Only row of a routed layer emits zero
  const int grow = row0 + row;
  const bool po = a.run_mask != nullptr && on && a.run_mask[grow] == 0;
  if (a.splits > 1) {
    const size_t at = ((static_cast<size_t>(grow) * a.Hkv + hk) * a.splits + split) * G + qh;
    if (!on) return;
    if (hi == 0) a.part_ml[at] = make_float2(m, l);
#pragma unroll
    for (int i = 0; i < OC; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4*>(a.part_o + at * D + 32 * i + 8 * g + 4 * hi) =
            f32x4{o[i][4 * g], o[i][4 * g + 1], o[i][4 * g + 2], o[i][4 * g + 3]};
    return;
  }
  const float inv = po ? 0.f : 1.f / l;
  if (a.ml != nullptr && on && hi == 0)
    a.ml[static_cast<size_t>(grow) * (a.Hkv * G) + hk * G + qh] = po ? make_float2(INFINITY, 0.f) : make_float2(m, inv);
  // the lane holds dims 32 i + 8 g + 4 hi + r of o[i][4 g + r]; two groups'
  // halves change places so that it stores eight consecutive dims
#pragma unroll
  for (int i = 0; i < OC; ++i)
#pragma unroll
    for (int g = 0; g < 4; g += 2) {
      uint32_t x[2], y[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        x[r] = po ? 0u : pack_bf2(o[i][4 * g + 2 * r] * inv, o[i][4 * g + 2 * r + 1] * inv);
        y[r] = po ? 0u : pack_bf2(o[i][4 * g + 4 + 2 * r] * inv, o[i][4 * g + 5 + 2 * r] * inv);
        const auto z = __builtin_amdgcn_permlane32_swap(x[r], y[r], false, false);
        x[r] = z[0];
        y[r] = z[1];
      }
      const int col = (hk * G + qh) * D + 32 * i + 8 * (g + hi);
      const size_t at = a.out_Rg == 0 ? static_cast<size_t>(grow) * a.Nq + col : frag_index(grow, col, a.out_Rg);
      if (on) *reinterpret_cast<u32x4*>(a.out + at) = u32x4{x[0], x[1], y[0], y[1]};
    }
}

// The splits of the items' rows joined, in split order: four dims a thread.
template <int D>
__global__ __launch_bounds__(256) void k_rows_join(AttnPrefillArgs a) {
  constexpr int kT = D / 4;  // threads of a column
  const int hk = blockIdx.x % a.Hkv;
  const int32_t* it = a.items + static_cast<size_t>(blockIdx.x / a.Hkv) * 3;
  const int c = blockIdx.y * (256 / kT) + threadIdx.x / kT, e = threadIdx.x % kT * 4;
  if (c >= it[2] * a.G) return;
  const int row = it[1] + c / a.G, qh = c % a.G;
  const bool po = a.run_mask != nullptr && a.run_mask[row] == 0;  // a Project-Only row emits zero
  const size_t at = (static_cast<size_t>(row) * a.Hkv + hk) * a.splits * a.G + qh;
  float M = -INFINITY, L = 0.f;
  f32x4 y = f32x4{0.f, 0.f, 0.f, 0.f};
  constexpr int kU = 4;  // splits in flight
  for (int s0 = 0; s0 < a.splits; s0 += kU) {
    float2 ml[kU];
    f32x4 x[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const size_t i = at + static_cast<size_t>(min(s0 + u, a.splits - 1)) * a.G;
      ml[u] = a.part_ml[i];
      x[u] = *reinterpret_cast<const f32x4*>(a.part_o + i * D + e);
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      if (s0 + u >= a.splits || ml[u].x == -INFINITY) continue;  // (a split of which the row sees nothing)
      const float mn = fmaxf(M, ml[u].x);
      const float f0 = M == -INFINITY ? 0.f : exp2f(M - mn), f1 = exp2f(ml[u].x - mn);
      L = L * f0 + ml[u].y * f1;
      y = y * f0 + x[u] * f1;
      M = mn;
    }
  }
  const float inv = po ? 0.f : 1.f / L;
  if (a.ml != nullptr && e == 0)
    a.ml[static_cast<size_t>(row) * (a.Hkv * a.G) + hk * a.G + qh] = po ? make_float2(INFINITY, 0.f) : make_float2(M, inv);
  const int col = (hk * a.G + qh) * D + e;
  const size_t to = a.out_Rg == 0 ? static_cast<size_t>(row) * a.Nq + col : frag_index(row, col, a.out_Rg);
  u32x2 pk = u32x2{0u, 0u};
  if (!po) pk = u32x2{pack_bf2(y[0] * inv, y[1] * inv), pack_bf2(y[2] * inv, y[3] * inv)};
  *reinterpret_cast<u32x2*>(a.out + to) = pk;
}

// Up to one work item a compute unit, eight waves each; beyond that two of four
// waves, which wait for each other less often.  Eight and four waves, us: 777
// rows of 32/8 heads after 2,300 tokens (200 work items) 71 and 82, 1,000 through
// a window of 4,096 (256) 116 and 129; 1,040 after 2,300 (264) 109 and 98, 1,500
// (376) 128 and 122, 2,080 (520) 207 and 184, 2 x 2,000 fresh ones (1,008) 122 and
// 101; through a window of 256 1,500 rows of 24/8 (288) 27 and 20, 4 x 1,037 (800)
// 55 and 38; 34 prompts of 5 rows (272) 13 and 8.  Only fresh prompts without a
// window, whose longest work items set the time, go the other way up to some 400
// work items (3 x 1,500 of 8/8, 288: 40 and 46; 4 x 1,500, 384: 46 and 50; 480: 55
// and 53): not told apart.
template <int D>
static void launch_rows_d(const AttnPrefillArgs& a, int n_items, hipStream_t s) {
  const int wgs = n_items * a.Hkv * a.splits;
  if (n_items * a.Hkv <= 256) hipLaunchKernelGGL((k_attn_rows<D, 2>), dim3(wgs), dim3(512), 0, s, a);
  else hipLaunchKernelGGL((k_attn_rows<D, 1>), dim3(wgs), dim3(256), 0, s, a);
  if (a.splits > 1) hipLaunchKernelGGL((k_rows_join<D>), dim3(n_items * a.Hkv, kPreCols * D / 1024), dim3(256), 0, s, a);
}

hipError_t launch_attn_rows(const AttnPrefillArgs& a, int n_items, int head_dim, hipStream_t s) {
  if (n_items <= 0) return hipSuccess;
  if (head_dim == 128) launch_rows_d<128>(a, n_items, s);
  else if (head_dim == 64) launch_rows_d<64>(a, n_items, s);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace vsk
