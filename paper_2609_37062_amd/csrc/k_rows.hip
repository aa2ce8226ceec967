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
#include <climits>

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
  int32_t wide[kRowSlots][NH][2];  // (4-bit cache) the step's V blocks that are bf16, the others fp16
  float m[kRowTiles][64], l[kRowTiles][64];  // the second half's, when the halves join
};

// Q4: the 4-bit cache.  Scores are taken on v_mfma_scale_f32_32x32x64 from K's codes and
// exponents as they are, which go through LDS in a quarter of the bytes, and from q as
// two 8-bit terms (Kv4Query).  V is turned into 16 bits once for the workgroup and
// stored in the 16-bit walk's order.  Two waves move a block, half of its K and half of
// its V each (with a wave for K and one for V the V waves held up the others at the
// barrier: 1,000 rows after 7,000 tokens 180 us, 165).  A block's codes are loaded a step
// ahead of its slot's turn, its id a step before that, and a step's slot is filled
// behind the next scores' matrix instructions, not in front of them.
//
// V becomes fp16 where that holds it exactly, which any block of ordinary size is, and
// a weight then goes in with its first 11 bits: one matrix instruction instead of two.
// A block with other exponents becomes bf16 and takes weights of two terms.
//
// 2 x 1,000 rows through a window of 4,096 took 199 us with K and V turned into bf16,
// 177 with V in fp16, 169 with K as codes, 159 with slots filled behind the scores (165
// behind the whole step; priorities for the wave that has matrix instructions: none).
// What bounds it is not one unit: the matrix cores are busy 38% of the cycles, LDS 21%,
// the vector units about half, and a wave waits 28% of its time, for the barrier of a
// step and the operands behind it; two waves a SIMD overlap the rest only in part.  At
// head_dim 128 some 20 registers are in scratch, which the masked and the rescaled steps
// reload (a window of a few hundred keys is mostly those); the loop of whole steps does
// not.
template <int D, int NH, bool Q4>
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
  u32x4 qf[Q4 ? 1 : QC];
  Kv4Query q4[Q4 ? D / 64 : 1];
  {
    const uint16_t* qrow = a.q + static_cast<size_t>(row0 + row) * a.Nq + static_cast<size_t>(hk * G + qh) * D;
    auto q8 = [&](int e) __attribute__((always_inline)) { return on ? *reinterpret_cast<const u32x4*>(qrow + e) : u32x4{0u, 0u, 0u, 0u}; };
    if constexpr (Q4) {
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        const int e = 64 * i + 16 * hi;
        const u32x4 x[4] = {q8(e), q8(e + 8), q8(e + 32), q8(e + 40)};
        q4[i] = kv4_query_32(x, hi);
      }
    } else {
#pragma unroll
      for (int s = 0; s < QC; ++s) qf[s] = q8(16 * s + 8 * hi);
    }
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
  // (Q4) of block w / 2 of the step this lane moves K's codes of place kp, 16 (D = 64: 8)
  // dims of K's quarter kq of which half kh, and the exponent of (place ep, block eb);
  // turns V of tokens 8 vth + 4 vtq + 2 vt2, + 1 of its d; and looks at V's exponents of
  // one token (two at D = 64).  Lanes in the order of LDS: neighbours store neighbouring
  // words (a wave's V stores four words apart: LDS busy 37% of the time, now 21%, and a
  // hundredth of the call).  K in LDS: for each block of 32 dims the codes of 32 places,
  // then a place's exponents, four bytes each.
  struct Codes {
    uint32_t k[D / 64], v[D / 64], vs[D / 64], ks, all;
  };
  const uint8_t* rec0 = a.pool4 + (static_cast<size_t>(a.layer) * a.n_blocks * a.Hkv + hk) * kv4_record(D);
  const int half = w & 1, ep = lane & 15, eb = lane >> 4 & (D / 32 - 1);
  const int kh = lane & 1, piece = 16 * half + (lane >> 2);  // (D = 64: of 16 bytes)
  const int kp = D == 128 ? lane >> 1 & 15 : (piece & 7) + 8 * (lane >> 1 & 1), kq = D == 128 ? 2 * half + (lane >> 5) : piece >> 3;
  const int vt2 = lane & 1, vtq = lane >> 1 & 1, vd = lane >> 2, vth = half;
  // (of a record, which the loads take as a buffer: a lane's place is 32 bits then)
  const uint32_t k_at = 4 * D * half + D / 16 * lane;
  const uint32_t v_at = kv4_v_at(D) + (D == 128 ? 16 * (vd + 16 * vth + 32 * vtq) + 8 * vt2 : 256 * half + 4 * lane);
  const uint32_t vs_at = kv4_vs_at(D) + (8 * vth + 4 * vtq + 2 * vt2) * (D / 32);
  const uint32_t ks_at = kv4_ks_at(D) + kv4_ks_byte(ep, eb), all_at = kv4_vs_at(D) + 4 * (lane & (D / 8 - 1));
  auto words = [](uint32_t (&to)[D / 64], __amdgpu_buffer_rsrc_t rs, uint32_t at) __attribute__((always_inline)) {
    if constexpr (D == 128) {
      const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rs, at, 0, 0));
      to[0] = y[0];
      to[D / 64 - 1] = y[1];
    } else {
      to[0] = __builtin_amdgcn_raw_buffer_load_b32(rs, at, 0, 0);
    }
  };
  auto id_of = [&](int step) __attribute__((always_inline)) { return sm.tbl[min(2 * NH * step + my_blk, span.nv - 1)]; };
  int32_t id = 0;  // of the next step to fetch
  auto fetch = [&](int step, Codes& x) __attribute__((always_inline)) {
    const uint32_t blk = __builtin_amdgcn_readfirstlane(id);
    id = id_of(step + 1);
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t*>(rec0 + static_cast<size_t>(blk) * (a.Hkv * kv4_record(D))), 0, kv4_record(D), 0x00020000);
    words(x.k, rs, k_at);
    words(x.v, rs, v_at);
    words(x.vs, rs, vs_at);
    x.ks = __builtin_amdgcn_raw_buffer_load_b8(rs, ks_at, 0, 0);
    x.all = __builtin_amdgcn_raw_buffer_load_b32(rs, all_at, 0, 0);
  };
  // Slots behind the rows' last key (of the list's last block, and what stands in for those
  // past it) become values of zero with an exponent that fp16 holds.
  const int last_keys = min(kv_end, pos0 + n_rows) % kBlock;
  const int cut_from = last_keys > 0 ? (span.nv - 1 - my_blk + 2 * NH - 1) / (2 * NH) : INT_MAX;  // steps
  auto cut = [&](Codes& x) __attribute__((always_inline)) {
    const uint32_t kNone = 0x78787878u;
    const int t = 8 * vth + 4 * vtq + 2 * vt2, n = last_keys;
    if constexpr (D == 128) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        x.v[j * (D / 128)] = t + j < n ? x.v[j * (D / 128)] : 0u;
        x.vs[j * (D / 128)] = t + j < n ? x.vs[j * (D / 128)] : kNone;
      }
      x.all = (lane & 15) < n ? x.all : kNone;
    } else {
      auto some = [&](int first, uint32_t y, uint32_t none) {  // of two tokens, 16 bits each
        const uint32_t keep = (first < n ? 0xffffu : 0u) | (first + 1 < n ? 0xffff0000u : 0u);
        return (y & keep) | (none & ~keep);
      };
      x.v[0] = some(t, x.v[0], 0u);
      x.vs[0] = some(t, x.vs[0], kNone);
      x.all = some(2 * (lane & 7), x.all, kNone);
    }
  };
  // fp16 holds every value of a block exactly whose exponents are 104 .. 140 (the same
  // for both waves of the block)
  auto is_wide = [](uint32_t all) __attribute__((always_inline)) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    const u16x2 even = __builtin_bit_cast(u16x2, all & 0x00ff00ffu) - u16x2{104, 104};
    const u16x2 odd = __builtin_bit_cast(u16x2, all >> 8 & 0x00ff00ffu) - u16x2{104, 104};
    const u16x2 off = __builtin_elementwise_max(even, odd);
    return static_cast<bool>(__any(off[0] > 36 || off[1] > 36));
  };
  auto expand = [&](int step, const Codes& x) __attribute__((always_inline)) {
    u32x4* kt = &sm.kv[step % kRowSlots][0][w >> 2][0][0];
    const int blk = 16 * (w >> 1 & 1);
    if constexpr (D == 128) reinterpret_cast<u32x2*>(kt + 32 * kq + blk + kp)[kh] = u32x2{x.k[0], x.k[D / 64 - 1]};
    else reinterpret_cast<uint32_t*>(kt + 32 * (kq >> 1) + blk + kp)[2 * (kq & 1) + kh] = x.k[0];
    reinterpret_cast<uint8_t*>(kt + D + (blk + ep) / 4)[4 * (ep & 3) + eb] = static_cast<uint8_t>(x.ks);
    uint32_t* vt = reinterpret_cast<uint32_t*>(&sm.kv[step % kRowSlots][1][w >> 2][w >> 1 & 1][0]) + 2 * vtq + vt2;
    auto put = [&](const Codes& x, auto half_c) __attribute__((always_inline)) {
      constexpr bool HALF = decltype(half_c)::value;
#pragma unroll
      for (int b = 0; b < D / 32; ++b) {
        uint32_t y[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const uint32_t cw = x.v[t * (D / 64) / 2], sw = x.vs[t * (D / 64) / 2];
          const int n = D == 128 ? b : 2 * t + b;
          const float sc = kv4_scale(sw, n);
          if constexpr (HALF)
            y[t] = n == 0 ? mx4_decode_half<0>(cw, sc) : n == 1 ? mx4_decode_half<1>(cw, sc) : n == 2 ? mx4_decode_half<2>(cw, sc) : mx4_decode_half<3>(cw, sc);
          else
            y[t] = n == 0 ? mx4_decode<0>(cw, sc) : n == 1 ? mx4_decode<1>(cw, sc) : n == 2 ? mx4_decode<2>(cw, sc) : mx4_decode<3>(cw, sc);
        }
        vt[4 * (32 * (2 * b) + vd + 16 * vth)] = low_halves(y[0], y[1]);
        vt[4 * (32 * (2 * b + 1) + vd + 16 * vth)] = high_halves(y[0], y[1]);
      }
    };
    bool wide = is_wide(x.all);
    if (__builtin_expect(wide, 0)) {
      // (slots of no token decide nothing: where what an earlier owner left in them is all
      // that fp16 does not hold, it goes, and where it is not, weights of zero leave it out)
      Codes y = x;
      if (step >= cut_from) {
        cut(y);
        wide = is_wide(y.all);
      }
      if (wide) put(y, std::false_type{});
      else put(y, std::true_type{});
    } else {
      put(x, std::true_type{});
    }
    if (lane == 0) sm.wide[step % kRowSlots][w >> 2][w >> 1 & 1] = wide;
  };
  Codes raw;
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
  // (Q4: FAST steps' V is fp16, and so is that of the blocks whose bit in `wide` is
  // clear: a weight goes in with its first 11 bits, one instruction instead of two.)
  auto rest = [&](int step, const f32x16& s, auto fast_c, int wide = 0) __attribute__((always_inline)) {
    constexpr bool FAST = decltype(fast_c)::value;
    const u32x4* vp = &sm.kv[step % kRowSlots][1][hh][0][32 * (lc >> 4) + (lane & 15) + 16 * hi];
    // (Q4: weights times 2^7, with the lag at most 2^15: an fp16's smallest step is then
    // 2^-32 of the largest weight's and more, and many small weights keep their sum.  The 7
    // joins the maximum where that is below 2^14, so that a weight is one fma, and the
    // difference elsewhere: from 2^24 on a float32 maximum less 7 is off by 1 and more)
    constexpr float kUp = Q4 ? 7.f : 0.f;
    const float mb = FAST ? m - kUp : m == -INFINITY ? 0.f : m;
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
          p[r] = __builtin_amdgcn_exp2f(Q4 ? x - mb + kUp : x - mb);
        }
      }
      l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      if (Q4 && (FAST || !(wide >> b & 1))) {  // (uniform)
        u32x4 ph;
#pragma unroll
        for (int j = 0; j < 4; ++j) ph[j] = pack_half2(p[2 * j], p[2 * j + 1]);
#pragma unroll
        for (int i = 0; i < OC; ++i) o[i] = mfma_32x32x16_f16(vt[i], ph, o[i]);
        continue;
      }
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

  if constexpr (Q4) {
    id = id_of(first);
#pragma unroll
    for (int j = 0; j < 3; ++j) {
      fetch(first + j, raw);
      expand(first + j, raw);
    }
    fetch(first + 3, raw);
  } else {
#pragma unroll
    for (int j = 0; j < 3; ++j) copy(first + j);
  }
  bool big = false;  // (uniform) scores so large that a fma's unrounded product would be off the maximum
  f32x16 s;          // s[r]: key 8 hi + r of the step's first block (r < 8), 8 hi + r - 8 of the second
  float mx;
  auto next = [&](int step) __attribute__((always_inline)) {
    if constexpr (!Q4) landed(std::integral_constant<int, 1>{});
    barrier_after_lds_reads();  // the next step's slot is whole, the one of the last step free
    if constexpr (!Q4) copy(step + 3);
  };
  auto refill = [&](int step) __attribute__((always_inline)) {  // (Q4: the slot that the barrier freed)
    if constexpr (Q4) {
      expand(step + 3, raw);
      fetch(step + 4, raw);
    }
  };
  auto qk = [&](int step, f32x16& s) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
    if constexpr (Q4) {
      const u32x4* kp = &sm.kv[step % kRowSlots][0][hh][0][lc];
      const int ks = static_cast<int>(reinterpret_cast<const uint32_t*>(kp - lc + D)[lc] >> (8 * hi));
      u32x4 k[D / 64];
#pragma unroll
      for (int i = 0; i < D / 64; ++i) k[i] = kp[32 * (2 * i + hi)];
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        const i32x8 x = {static_cast<int>(k[i][0]), static_cast<int>(k[i][1]), static_cast<int>(k[i][2]), static_cast<int>(k[i][3]), 0, 0, 0, 0};
        const int e = static_cast<int>(q4[i].e);
        if (i == 0) {  // (the exponent's byte is part of the instruction)
          s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, q4[i].hi, s, 4, 0, 0, ks, 0, e);
          s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, q4[i].lo, s, 4, 0, 0, ks, 1, e);
        } else {
          s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, q4[i].hi, s, 4, 0, 2, ks, 0, e);
          s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, q4[i].lo, s, 4, 0, 2, ks, 1, e);
        }
        asm("" : "+v"(s) : "v"(k[i]), "v"(ks));  // (see kv4_scores; q stays to the end of the walk)
      }
    } else {
      const u32x4* kp = &sm.kv[step % kRowSlots][0][hh][lc >> 4][(lane & 15) + 16 * hi];
#pragma unroll
      for (int i = 0; i < QC; ++i) s = mfma_32x32x16(kp[32 * i], qf[i], s);
    }
  };
  auto wide_of = [&](int step) __attribute__((always_inline)) {  // (uniform)
    if constexpr (!Q4) return 0;
    const int32_t* f = sm.wide[step % kRowSlots][hh];
    return __builtin_amdgcn_readfirstlane(f[0] | f[1] << 1);
  };
  auto top = [&](const f32x16& s) __attribute__((always_inline)) {
    float x = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) x = fmaxf(x, s[r]);
    return max_xor32(x) * sc;
  };
  int step = first;
  if constexpr (!Q4) landed(std::integral_constant<int, 2>{});
  barrier_after_lds_reads();
  qk(step, s);
  mx = top(s);
  int wide = wide_of(step);
  while (step < n_steps) {
    // (a loop of its own, so that the sums stay where they are)
    while (is_full(step) && !big && !wide && !__any(mx > m + kRowsLag)) {  // (-inf + 8 is -inf: first keys always are)
      next(step);
      f32x16 sn;
      qk(step + 1, sn);
      wide = wide_of(step + 1);
      refill(step);
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
    refill(step);
    rest(step, s, std::false_type{}, wide);
    if (__builtin_expect(poisoned, 0)) poison(step);
    if (++step == n_steps) break;
    qk(step, s);
    mx = top(s);
    wide = wide_of(step);
  }
  if constexpr (Q4) {
#pragma unroll
    for (int i = 0; i < D / 64; ++i) kv4_keep(q4[i]);
  }
  l = add_xor32(l);
  if constexpr (!Q4) landed(std::integral_constant<int, 0>{});  // (the steps past the list: before LDS is used again or ends)

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
      if (s0 + u >= a.splits) continue;
      // (a maximum of -inf: a split of which the row sees nothing, whose sums are zero, or
      // only scores that are NaN, whose sums are)
      const float mn = fmaxf(M, ml[u].x);
      const float f0 = M == -INFINITY ? 0.f : exp2f(M - mn), f1 = ml[u].x == -INFINITY ? 0.f : exp2f(ml[u].x - mn);
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
template <int D, bool Q4>
static void launch_rows_d(const AttnPrefillArgs& a, int n_items, hipStream_t s) {
  const int wgs = n_items * a.Hkv * a.splits;
  if (n_items * a.Hkv <= 256) hipLaunchKernelGGL((k_attn_rows<D, 2, Q4>), dim3(wgs), dim3(512), 0, s, a);
  else hipLaunchKernelGGL((k_attn_rows<D, 1, Q4>), dim3(wgs), dim3(256), 0, s, a);
  if (a.splits > 1) hipLaunchKernelGGL((k_rows_join<D>), dim3(n_items * a.Hkv, kPreCols * D / 1024), dim3(256), 0, s, a);
}

hipError_t launch_attn_rows(const AttnPrefillArgs& a, int n_items, int head_dim, hipStream_t s) {
  if (n_items <= 0) return hipSuccess;
  if (head_dim != 128 && head_dim != 64) return hipErrorInvalidValue;
  if (a.pool4 != nullptr) head_dim == 128 ? launch_rows_d<128, true>(a, n_items, s) : launch_rows_d<64, true>(a, n_items, s);
  else head_dim == 128 ? launch_rows_d<128, false>(a, n_items, s) : launch_rows_d<64, false>(a, n_items, s);
  return hipGetLastError();
}

}  // namespace vsk
