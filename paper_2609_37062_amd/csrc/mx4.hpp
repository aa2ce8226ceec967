// Microscaled 4-bit floating point: layout of a matrix, launchers (k_mx4.hip).
//
// The format is the OCP microscaling one with 4-bit elements (e2m1: 0, 0.5, 1,
// 1.5, 2, 3, 4, 6 and a sign) and a shared power of two (a biased 8-bit
// exponent, 255: every value NaN) for 32 consecutive values of a row.  A block's
// exponent is floor(log2(largest magnitude)) - 2, at least -127; its values are
// rounded to nearest, ties to the even code, beyond 6 to 6.
//
// A matrix X[rows][k] is held as the matrix cores take it.  Codes: 1 KiB tiles of
// 16 rows x 128 columns, tile (rt, kt) at (rt * Kt + kt) KiB; lane l (0..63) owns
// 16 bytes: row l % 16, columns 128 kt + 32 (l / 16) .. + 31, one block, the first
// value in the low half of the first byte.  Exponents, behind all codes: for four
// tiles (rt, 4 kq .. 4 kq + 3) 256 bytes, lane l's four bytes the exponents of its
// block in each.  Rows and columns that fill up tiles are zero codes.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace vsk {

struct Mx4Shape {
  int64_t rt, kt, kq;  // tiles of rows, of columns, fours of them
  __host__ __device__ Mx4Shape(int64_t rows, int64_t k) : rt((rows + 15) / 16), kt((k + 127) / 128), kq((kt + 3) / 4) {}
  __host__ __device__ size_t scales_at() const { return static_cast<size_t>(rt * kt) * 1024; }
  __host__ __device__ size_t bytes() const { return scales_at() + static_cast<size_t>(rt * kq) * 256; }
};

enum Mx4Type { kMxBf16 = 0, kMxFp32 = 1, kMxMx4 = 2 };

// counters (nullable): so many ints set to zero by the launch, for the product
// that follows.
hipError_t launch_mx4_quantise(const void* src, int dtype, int64_t stride, int rows, int k, uint8_t* mx, int* counters,
                               int n_counters, hipStream_t s);
hipError_t launch_mx4_pack(const uint8_t* codes, const uint8_t* scales, int rows, int k, uint8_t* mx, hipStream_t s);
hipError_t launch_mx4_read(const uint8_t* mx, int rows, int k, void* dst, int dtype, int64_t stride, hipStream_t s);

struct Mx4ProductArgs {
  const uint8_t* x;   // MX4 [rows][k], or
  const void* x_raw;  // rows to quantise (mx4_takes_rows), bf16 or fp32, x_stride apart
  int x_fp32;
  int64_t x_stride;
  const uint8_t* w;  // MX4 [n][k]
  int rows, n, k;
  void* y;  // [rows][n], stride y_stride, bf16 or fp32
  int y_fp32;
  int64_t y_stride;
  const void* add;  // nullable, as y
};
// Whether launch_mx4_stream takes x as it is (few short rows).
bool mx4_takes_rows(int dtype, const void* x, int64_t stride, int rows, int k);
hipError_t launch_mx4_stream(const Mx4ProductArgs& a, hipStream_t s);
// The others (k_mx4_tile.hip): y in tiles of tm x tn 16ths, K in `splits` parts of
// `steps` 128 columns, whose sums meet in `part`; `counter` an int a tile, zero.
struct Mx4Split {
  int rows;  // 1: taken by launch_mx4_rows
  int tm, tn, tiles_m, tiles_n, splits, steps;
  float __attribute__((ext_vector_type(4)))* part;
  int* counter;
  __host__ __device__ int tiles() const { return tiles_m * tiles_n; }
  int counters() const { return splits > 1 ? tiles() : 0; }
  size_t part_bytes() const { return static_cast<size_t>(counters()) * splits * tm * tn * 1024; }
};
Mx4Split mx4_split(int rows, int n, int k);
hipError_t launch_mx4_rows(const Mx4ProductArgs& a, const Mx4Split& sp, hipStream_t s);
hipError_t launch_mx4_tile(const Mx4ProductArgs& a, const Mx4Split& sp, hipStream_t s);

}  // namespace vsk
