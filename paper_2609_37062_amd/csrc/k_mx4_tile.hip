// Products of many rows in microscaled 4 bits: tiles of both matrices through LDS.
//
// A workgroup of WM x WN waves takes 16 WM FM columns of y (rows of w) x 16 WN FN
// rows; a wave FM x FN tiles of v_mfma_scale_f32_16x16x128_f8f6f4.  Codes are held as
// the instruction takes them, so a 1 KiB tile is copied straight into LDS and read
// from there 16 bytes a lane, without conflicts.
#include "mx4_mma.hpp"

namespace vsk {

constexpr int kMxSlots = 4;  // tiles of columns in LDS: three copied ahead of the one that is read

template <int WM, int WN, int FM, int FN>
__global__ __launch_bounds__(64 * WM * WN, 2) void k_mx4_tile(Mx4ProductArgs a, int tiles_m, int tiles_n) {
  constexpr int NW = WM * WN, TM = WM * FM, TN = WN * FN;  // waves; tiles of rows of w and x
  constexpr int kCopies = (TM + TN) / NW;                  // 1 KiB copies of a wave for a slot
  static_assert((TM + TN) % NW == 0 && kCopies % 4 == 0, "copies shared evenly, exponents of a quarter of them a slot");
  constexpr int kPer = kCopies + kCopies / 4;              // with the exponents'
  __shared__ u32x4 s_code[kMxSlots][TM + TN][64];
  __shared__ uint32_t s_exp[2][TM + TN][64];

  // an XCD's workgroups (every eighth) take neighbouring columns, all rows of each
  const int total = tiles_m * tiles_n, per = (total + 7) / 8;
  const int id = static_cast<int>(blockIdx.x % 8) * per + static_cast<int>(blockIdx.x / 8);
  if (static_cast<int>(blockIdx.x / 8) >= per || id >= total) return;
  const int bm = id / tiles_n, bn = id % tiles_n;

  const Mx4Shape gw(a.n, a.k), gx(a.rows, a.k);
  const int kt_n = static_cast<int>(gw.kt), kq_n = static_cast<int>(gw.kq);
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = w % WM, wn = w / WM;
  // the rows of tiles that this wave copies: w's (i < TM) and x's
  const uint8_t* code[kCopies];
  const uint8_t* expo[kCopies];
#pragma unroll
  for (int c = 0; c < kCopies; ++c) {
    const int i = w * kCopies + c;
    const bool x = i >= TM;
    const int64_t rt = x ? min(static_cast<int64_t>(bn) * TN + i - TM, gx.rt - 1) : min(static_cast<int64_t>(bm) * TM + i, gw.rt - 1);
    code[c] = (x ? a.x : a.w) + static_cast<size_t>(rt * kt_n) * 1024;
    expo[c] = (x ? a.x + gx.scales_at() : a.w + gw.scales_at()) + static_cast<size_t>(rt * kq_n) * 256;
  }
  const uint32_t lds_code = lds_address(&s_code[0][w * kCopies][0]), lds_exp = lds_address(&s_exp[0][w * kCopies][0]);
  const uint32_t lane16 = 16 * lane, lane4 = 4 * lane;
  // tile kt of columns (past the end: the last one again) into its slot; and copy c of
  // the exponents of four tiles, which also has to be issued three steps ahead of its
  // first use: half of them two fours ahead, once the slot's own have been read
  auto copy = [&](int kt) __attribute__((always_inline)) {
    const size_t at = static_cast<size_t>(min(kt, kt_n - 1)) * 1024;
    const uint32_t dst = lds_code + (kt % kMxSlots) * static_cast<uint32_t>(sizeof(s_code[0]));
#pragma unroll
    for (int c = 0; c < kCopies; ++c) lds_copy16<false>(code[c] + at, lane16, dst + 1024 * c);
  };
  auto copy_exp = [&](int q, int c) __attribute__((always_inline)) {
    lds_copy4(expo[c] + static_cast<size_t>(min(q, kq_n - 1)) * 256, lane4,
              lds_exp + (q & 1) * static_cast<uint32_t>(sizeof(s_exp[0])) + 256 * c);
  };

  f32x4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

#pragma unroll
  for (int c = 0; c < kCopies; ++c) copy_exp(0, c);
#pragma unroll
  for (int c = 0; c < kCopies / 2; ++c) copy_exp(1, c);
#pragma unroll
  for (int i = 0; i < kMxSlots - 1; ++i) copy(i);
  uint32_t sw[FM], sx[FN];
  auto step = [&](int kt, auto jc) __attribute__((always_inline)) {
    constexpr int J = decltype(jc)::value;
    // all but the newest two slots' copies of this wave have landed (the first
    // slots come without exponents between them, which only waits for more)
    if (kt < 3) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kCopies) : "memory");
    else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kPer) : "memory");
    barrier_after_lds_reads();
    copy(kt + kMxSlots - 1);
#pragma unroll
    for (int c = 0; c < kCopies / 4; ++c) copy_exp(kt / 4 + (J < 2 ? 1 : 2), (J + 2) % 4 * (kCopies / 4) + c);
    if constexpr (J == 0) {
#pragma unroll
      for (int i = 0; i < FM; ++i) sw[i] = s_exp[kt / 4 & 1][wm * FM + i][lane];
#pragma unroll
      for (int j = 0; j < FN; ++j) sx[j] = s_exp[kt / 4 & 1][TM + wn * FN + j][lane];
    }
    const u32x4* cw = &s_code[kt % kMxSlots][wm * FM][lane];
    const u32x4* cx = &s_code[kt % kMxSlots][TM + wn * FN][lane];
    u32x4 xv[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) xv[j] = cx[64 * j];
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const u32x4 wv = cw[64 * i];
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = mfma_mx4<J, J>(wv, xv[j], acc[i][j], sw[i], sx[j]);
    }
  };
  for (int kt = 0; kt < kt_n; kt += 4) {
    step(kt, std::integral_constant<int, 0>{});
    if (kt + 1 < kt_n) step(kt + 1, std::integral_constant<int, 1>{});
    if (kt + 2 < kt_n) step(kt + 2, std::integral_constant<int, 2>{});
    if (kt + 3 < kt_n) step(kt + 3, std::integral_constant<int, 3>{});
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (the copies past the end land before LDS is given back)
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    const int row = 16 * (bn * TN + wn * FN + j) + (lane & 15);
    if (row >= a.rows) continue;
#pragma unroll
    for (int i = 0; i < FM; ++i) mx4_store4(a, row, 16 * (bm * TM + wm * FM + i) + 4 * (lane >> 4), acc[i][j]);
  }
}

template <int WM, int WN, int FM, int FN>
static void launch_tile(const Mx4ProductArgs& a, hipStream_t s) {
  const int tm = (a.n + 16 * WM * FM - 1) / (16 * WM * FM), tn = (a.rows + 16 * WN * FN - 1) / (16 * WN * FN);
  const unsigned grid = (static_cast<unsigned>(tm) * tn + 7) / 8 * 8;
  hipLaunchKernelGGL((k_mx4_tile<WM, WN, FM, FN>), dim3(grid), dim3(64 * WM * WN), 0, s, a, tm, tn);
}

hipError_t launch_mx4_tile(const Mx4ProductArgs& a, hipStream_t s) {
  const int64_t large = static_cast<int64_t>((a.n + 255) / 256) * ((a.rows + 255) / 256);
  if (large >= 192) launch_tile<4, 2, 4, 8>(a, s);
  else launch_tile<2, 2, 4, 4>(a, s);
  return hipGetLastError();
}

}  // namespace vsk
