// Products of many rows in microscaled 4 bits: tiles of both matrices through LDS.
//
// A workgroup of WM x WN waves takes 32 WM FM columns of y (rows of w) x 32 WN FN
// rows, a wave FM x FN tiles of v_mfma_scale_f32_32x32x64_f8f6f4 (with values of all
// kinds it reaches 6.7 PFLOP/s, the 16x16x128 form 5.5).  Codes are held as the
// matrix cores take them, so a 1 KiB tile of 16 x 128 is copied straight into LDS and
// read from there 16 bytes a lane, without conflicts.  Where the tiles of y are fewer
// than the compute units, K is cut over workgroups; their sums meet in the workspace
// and the one that arrives last adds them in the order of K.
#include <algorithm>

#include "mx4_mma.hpp"

namespace vsk {

// S: slots of LDS, a step of 128 columns each, S copied ahead; exponents of four
// steps each in E slots of their own.
template <int WM, int WN, int FM, int FN, int S, int E>
__global__ __launch_bounds__(64 * WM * WN, 2) void k_mx4_tile(Mx4ProductArgs a, Mx4Split sp) {
  constexpr int NW = WM * WN, TM = 2 * WM * FM, TN = 2 * WN * FN, T = TM + TN;  // waves; 16-row tiles of w and x
  constexpr int kCopies = (T + NW - 1) / NW;                                    // 1 KiB copies of a wave for a slot
  static_assert((S - 1) * kCopies + E * kCopies <= 63, "copies in flight");
  __shared__ u32x4 s_code[S][T][64];
  __shared__ uint32_t s_exp[E][T][64];
  __shared__ int s_last;

  // an XCD's workgroups (every eighth) take neighbouring columns, all rows of each
  const int total = sp.tiles() * sp.splits, per = (total + 7) / 8;
  const int id = static_cast<int>(blockIdx.x % 8) * per + static_cast<int>(blockIdx.x / 8);
  if (static_cast<int>(blockIdx.x / 8) >= per || id >= total) return;
  const int split = id % sp.splits, tile = id / sp.splits;
  const int bm = tile / sp.tiles_n, bn = tile % sp.tiles_n;

  const Mx4Shape gw(a.n, a.k), gx(a.rows, a.k);
  const int kt_n = static_cast<int>(gw.kt), kq_n = static_cast<int>(gw.kq);
  // the split's steps k0 .. k1 - 1 (k0 a multiple of four)
  const int k0 = min(kt_n, split * sp.steps), k1 = min(kt_n, k0 + sp.steps);
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = w % WM, wn = w / WM;
  // the rows of tiles that this wave copies, w's (i < TM) and x's (past the last: it
  // again), and past a matrix's end its last row of tiles
  const uint8_t* code[kCopies];
  const uint8_t* expo[kCopies];
  uint32_t to_code[kCopies], to_exp[kCopies];
#pragma unroll
  for (int c = 0; c < kCopies; ++c) {
    const int i = min(w + c * NW, T - 1);
    const bool x = i >= TM;
    const int64_t rt = x ? min(static_cast<int64_t>(bn) * TN + i - TM, gx.rt - 1) : min(static_cast<int64_t>(bm) * TM + i, gw.rt - 1);
    code[c] = (x ? a.x : a.w) + static_cast<size_t>(rt * kt_n) * 1024;
    expo[c] = (x ? a.x + gx.scales_at() : a.w + gw.scales_at()) + static_cast<size_t>(rt * kq_n) * 256;
    to_code[c] = lds_address(&s_code[0][i][0]);
    to_exp[c] = lds_address(&s_exp[0][i][0]);
  }
  const uint32_t lane16 = 16 * lane, lane4 = 4 * lane;
  auto copy = [&](int kt, int c) __attribute__((always_inline)) {  // (past the end: the last one again)
    lds_copy16<false>(code[c] + static_cast<size_t>(min(kt, kt_n - 1)) * 1024, lane16,
                      to_code[c] + (kt - k0) % S * static_cast<uint32_t>(sizeof(s_code[0])));
  };
  auto copy_exp = [&](int q, int c) __attribute__((always_inline)) {
    lds_copy4(expo[c] + static_cast<size_t>(min(q, kq_n - 1)) * 256, lane4, to_exp[c] + q % E * static_cast<uint32_t>(sizeof(s_exp[0])));
  };

  f32x16 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  // Lane l feeds row l % 32 and the block l / 32 of half a step's two: its place in a
  // pair of 16-row tiles.
  const int place = ((lane & 31) >> 4) * 64 + (lane & 15) + 16 * (lane >> 5);
  struct Half {
    u32x4 w[FM], x[FN];
  };
  auto read = [&](Half& f, int kt, int half) __attribute__((always_inline)) {
    const u32x4* s = &s_code[(kt - k0) % S][0][0] + place + 32 * half;
#pragma unroll
    for (int j = 0; j < FN; ++j) f.x[j] = s[(TM + 2 * (wn * FN + j)) * 64];
#pragma unroll
    for (int i = 0; i < FM; ++i) f.w[i] = s[2 * (wm * FM + i) * 64];
  };
  uint32_t sw[FM][2], sx[FN][2];
  // between(m) is issued behind the m-th matrix instruction
  auto mma = [&](const Half& f, auto jc, auto hc, auto between) __attribute__((always_inline)) {
    constexpr int J = decltype(jc)::value, H = decltype(hc)::value;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        acc[i][j] = mfma_mx4_32<J, J>(f.w[i], f.x[j], acc[i][j], sw[i][H], sx[j][H]);
        between(i * FN + j);
      }
  };
#pragma unroll
  for (int q = 0; q < E; ++q)
#pragma unroll
    for (int c = 0; c < kCopies; ++c) copy_exp(k0 / 4 + q, c);
#pragma unroll
  for (int i = 0; i < S; ++i)
#pragma unroll
    for (int c = 0; c < kCopies; ++c) copy(k0 + i, c);
  // The first half of a step is read behind the middle of the step before it, the
  // second while the first is used.  In the middle all waves have read their step,
  // its slot is free, and this wave's copies for the next have landed once no more
  // than those of the S - 2 after it are outstanding (exponents, in between, only
  // wait for more; before a new four they have to have landed too).
  Half fa, fb;
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S - 1) * kCopies) : "memory");
  barrier_after_lds_reads();
  read(fa, k0, 0);
  auto step = [&](int kt, auto jc) __attribute__((always_inline)) {
    constexpr int J = decltype(jc)::value;
    if constexpr (J == 0) {
      const uint32_t* e = &s_exp[kt / 4 % E][0][0] + place;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < FM; ++i) sw[i][h] = e[2 * (wm * FM + i) * 64 + 32 * h];
#pragma unroll
        for (int j = 0; j < FN; ++j) sx[j][h] = e[(TM + 2 * (wn * FN + j)) * 64 + 32 * h];
      }
    }
    read(fb, kt, 1);
    __builtin_amdgcn_sched_barrier(0);  // (else the reads sink to where they are waited for)
    mma(fa, jc, std::integral_constant<int, 0>{}, [](int) {});
    constexpr int kLater = (J == 3 ? (S - 2 < 4 * E - 2 ? S - 2 : 4 * E - 2) : S - 2) * kCopies;
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLater) : "memory");
    barrier_after_lds_reads();
    read(fa, kt + 1, 0);
    // the copies go between the matrix instructions: issued in a row, they hold up the
    // wave (and all waves at once) until the ones before them have been taken
    mma(fb, jc, std::integral_constant<int, 1>{}, [&](int m) __attribute__((always_inline)) {
      constexpr int kM = FM * FN, kEach = (kCopies + kM - 1) / kM;
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int c = m * kEach; c < (m + 1) * kEach && c < kCopies; ++c) {
        copy(kt + S, c);
        if constexpr (J == 0) copy_exp(kt / 4 + E, c);
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  for (int kt = k0; kt < k1; kt += 4) {
    step(kt, std::integral_constant<int, 0>{});
    if (kt + 1 < k1) step(kt + 1, std::integral_constant<int, 1>{});
    if (kt + 2 < k1) step(kt + 2, std::integral_constant<int, 2>{});
    if (kt + 3 < k1) step(kt + 3, std::integral_constant<int, 3>{});
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (the copies past the end land before LDS is given back)

  if (sp.splits > 1) {
    constexpr uint32_t kWave = FM * FN * 4 * 1024, kSplit = NW * kWave;  // bytes
    uint8_t* part = reinterpret_cast<uint8_t*>(sp.part) + static_cast<size_t>(tile) * sp.splits * kSplit;
    const uint32_t mine = w * kWave + lane16;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          store_wt(part + split * kSplit + mine + ((i * FN + j) * 4 + g) * 1024,
                   __builtin_bit_cast(u32x4, f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]}));
    if (!mx4_last_of(sp, tile, s_last)) return;
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(part, 0, static_cast<int>(sp.splits * kSplit), 0x00020000);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    for (int s = 0; s < sp.splits; ++s)
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const f32x4 v = load_agent4(rs, s * kSplit + mine + ((i * FN + j) * 4 + g) * 1024);
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i][j][4 * g + r] += v[r];
          }
  }
  // acc[i][j][4 g + r] is column 8 g + 4 (lane / 32) + r, row lane % 32; two groups'
  // halves change places, so that a lane stores eight columns in a row
  const int hi = lane >> 5;
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    const int row = 16 * (bn * TN + 2 * (wn * FN + j)) + (lane & 31);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int g = 0; g < 4; g += 2) {
        f32x4 lo, up;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const auto z = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[i][j][4 * g + r]), __float_as_uint(acc[i][j][4 * g + 4 + r]), false, false);
          lo[r] = __uint_as_float(z[0]);
          up[r] = __uint_as_float(z[1]);
        }
        if (row < a.rows) mx4_store8(a, row, 16 * (bm * TM + 2 * (wm * FM + i)) + 8 * (g + hi), lo, up);
      }
  }
}

template <int WM, int WN, int FM, int FN, int S, int E>
static void launch_tile(const Mx4ProductArgs& a, const Mx4Split& sp, hipStream_t s) {
  const unsigned grid = (static_cast<unsigned>(sp.tiles()) * sp.splits + 7) / 8 * 8;
  hipLaunchKernelGGL((k_mx4_tile<WM, WN, FM, FN, S, E>), dim3(grid), dim3(64 * WM * WN), 0, s, a, sp);
}

constexpr int kMxUnits = 256;  // compute units

Mx4Split mx4_split(int rows, int n, int k) {
  const Mx4Shape gw(n, k), gx(rows, k);
  Mx4Split sp{};
  auto tiles = [&](int tm, int tn) {
    sp.tm = tm;
    sp.tn = tn;
    sp.tiles_m = static_cast<int>((gw.rt + tm - 1) / tm);
    sp.tiles_n = static_cast<int>((gx.rt + tn - 1) / tn);
    return static_cast<int64_t>(sp.tiles_m) * sp.tiles_n;
  };
  int64_t t;
  if (gx.rt <= 8) {
    const int tn = static_cast<int>(gx.rt + 1) / 2 * 2;
    t = tiles(8, tn);
    // few columns: by rows (128 columns a workgroup and K cut in eight to fill the
    // units, 32 x 6144 x 4096 10.6 us and 7.5, 128 x 4096 x 4096 14.5 and 9.5; enough of
    // them, 64 x 14336 x 4096 13.8 and 18.3).  Two tiles of columns where that leaves
    // workgroups for most units (48 x 6144 x 4096 9.5 us and 8.0) or K is long (77 x
    // 4096 x 14336 17.1 and 16.3; 128 x 4096 x 4096 9.5 and 15.7).
    if (t < 100) {
      sp.rows = 1;
      const bool two = gx.rt >= 2 && ((gw.rt >= 384 && gx.rt <= 6) || gw.kq >= 16);
      t = tiles(two ? 2 : 1, static_cast<int>(gx.rt));
    }
  } else {
    t = tiles(16, 16);
    // (half of the rows a tile where the last round of whole ones would be half empty:
    // 4096 x 6144 x 4096, 384 of them, 77.8 us and 75.5; 4096 x 28672 x 4096, seven whole
    // rounds, 283 and 303)
    if (t > kMxUnits && t % kMxUnits != 0 && t % kMxUnits <= kMxUnits / 2) t = tiles(16, 8);
    if (t < 192) t = tiles(8, 8);
  }
  // Fewer tiles than compute units: K is cut, in fours of steps, two at least a split
  // (by rows, whose eight waves cut it already, eight).
  const int fours = static_cast<int>(gw.kq), least = sp.rows ? 8 : 2;
  const int splits = t >= kMxUnits ? 1 : std::max(1, std::min(static_cast<int>(kMxUnits / t), fours / least));
  const int each = (fours + splits - 1) / splits;
  sp.steps = 4 * each;
  sp.splits = (fours + each - 1) / each;
  return sp;
}

hipError_t launch_mx4_tile(const Mx4ProductArgs& a, const Mx4Split& sp, hipStream_t s) {
  if (sp.tm == 16 && sp.tn == 16) launch_tile<2, 4, 4, 2, 4, 1>(a, sp, s);
  else if (sp.tm == 16) launch_tile<2, 2, 4, 2, 3, 1>(a, sp, s);
  else if (sp.tn == 8 && sp.tiles_n > 1) launch_tile<2, 2, 2, 2, 4, 1>(a, sp, s);
  else {
    if (sp.tn == 2) launch_tile<4, 1, 1, 1, 6, 2>(a, sp, s);
    else if (sp.tn == 4) launch_tile<4, 1, 1, 2, 6, 2>(a, sp, s);
    else if (sp.tn == 6) launch_tile<4, 1, 1, 3, 5, 2>(a, sp, s);
    else launch_tile<4, 1, 1, 4, 4, 2>(a, sp, s);
  }
  return hipGetLastError();
}

}  // namespace vsk
