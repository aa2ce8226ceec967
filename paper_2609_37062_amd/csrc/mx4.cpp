// C ABI of microscaled 4-bit matrices (device functions of their own, no handle).
#include "mx4.hpp"

#include <climits>
#include <cstdint>

#include "../../include/vsk.h"
#include "internal.hpp"

using namespace vsk;

namespace {

// (a launch takes a wave a tile, and less than 2^32 threads)
constexpr int64_t kMxMostTiles = (1 << 26) - 4;
bool shape_ok(int32_t rows, int32_t k) {
  if (rows < 1 || k < 1 || rows > (1 << 30) || k > (1 << 30)) return false;
  const Mx4Shape g(rows, k);
  return g.rt * g.kt <= kMxMostTiles;
}
bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
int element(int32_t dtype) { return dtype == VSK_FP32 ? 4 : 2; }
// bytes from the first to behind the last element of [rows][k] with a row stride
size_t extent(int32_t rows, int32_t k, int64_t stride, int size) {
  return (static_cast<size_t>(rows - 1) * stride + k) * size;
}
// rows whose extent in bytes 63 bits hold
bool stride_ok(int64_t stride, int32_t rows, int32_t k) { return stride >= k && stride <= INT64_MAX / 8 / rows; }
bool overlap(const void* a, size_t an, const void* b, size_t bn) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + bn && y < x + an;
}
int launched(hipError_t e) { return e == hipSuccess ? VSK_OK : VSK_E_HIP; }

}  // namespace

extern "C" {

size_t vsk_mx4_bytes(int32_t rows, int32_t k) { return shape_ok(rows, k) ? align_up(Mx4Shape(rows, k).bytes()) : 0; }

int vsk_mx4_quantise(const void* src_dev, int32_t dtype, int64_t stride, int32_t rows, int32_t k, void* mx_dev,
                     void* stream) {
  if (!src_dev || !mx_dev || !shape_ok(rows, k) || (dtype != VSK_BF16 && dtype != VSK_FP32) || !stride_ok(stride, rows, k)) return VSK_E_ARG;
  if (!aligned(mx_dev, kAlign) || !aligned(src_dev, element(dtype))) return VSK_E_ARG;
  if (overlap(src_dev, extent(rows, k, stride, element(dtype)), mx_dev, vsk_mx4_bytes(rows, k))) return VSK_E_ARG;
  return launched(launch_mx4_quantise(src_dev, dtype, stride, rows, k, static_cast<uint8_t*>(mx_dev), nullptr, 0,
                                      static_cast<hipStream_t>(stream)));
}

int vsk_mx4_pack(const uint8_t* codes_dev, const uint8_t* scales_dev, int32_t rows, int32_t k, void* mx_dev, void* stream) {
  if (!codes_dev || !scales_dev || !mx_dev || !shape_ok(rows, k) || !aligned(mx_dev, kAlign)) return VSK_E_ARG;
  const size_t bytes = vsk_mx4_bytes(rows, k);
  if (overlap(codes_dev, static_cast<size_t>(rows) * ((k + 1) / 2), mx_dev, bytes) ||
      overlap(scales_dev, static_cast<size_t>(rows) * ((k + 31) / 32), mx_dev, bytes))
    return VSK_E_ARG;
  return launched(launch_mx4_pack(codes_dev, scales_dev, rows, k, static_cast<uint8_t*>(mx_dev),
                                  static_cast<hipStream_t>(stream)));
}

int vsk_mx4_read(const void* mx_dev, int32_t rows, int32_t k, void* dst_dev, int32_t dtype, int64_t stride, void* stream) {
  if (!dst_dev || !mx_dev || !shape_ok(rows, k) || (dtype != VSK_BF16 && dtype != VSK_FP32) || !stride_ok(stride, rows, k)) return VSK_E_ARG;
  if (!aligned(mx_dev, kAlign) || !aligned(dst_dev, element(dtype))) return VSK_E_ARG;
  if (overlap(dst_dev, extent(rows, k, stride, element(dtype)), mx_dev, vsk_mx4_bytes(rows, k))) return VSK_E_ARG;
  return launched(launch_mx4_read(static_cast<const uint8_t*>(mx_dev), rows, k, dst_dev, dtype, stride,
                                  static_cast<hipStream_t>(stream)));
}

// A product's workspace: x as an MX4 matrix, the arrival counters, the split sums.
namespace {
struct ProductWs {
  size_t counter, part, total;
  Mx4Split sp;
  ProductWs(int32_t rows, int32_t n, int32_t k) : sp{} {
    counter = vsk_mx4_bytes(rows, k);
    sp = mx4_split(rows, n, k);
    part = counter + align_up(static_cast<size_t>(sp.counters()) * 4);
    total = part + align_up(sp.part_bytes());
  }
};
}  // namespace

size_t vsk_mx4_product_bytes(int32_t rows, int32_t n, int32_t k) {
  return shape_ok(rows, k) && shape_ok(n, k) ? ProductWs(rows, n, k).total : 0;
}

int vsk_mx4_product(const void* x_dev, int32_t x_dtype, int64_t x_stride, const void* w_mx_dev, int32_t rows, int32_t n,
                    int32_t k, void* y_dev, int32_t y_dtype, int64_t y_stride, const void* add_dev, void* ws_dev,
                    size_t ws_bytes, void* stream) {
  if (!x_dev || !w_mx_dev || !y_dev || !ws_dev || !shape_ok(rows, k) || !shape_ok(n, k)) return VSK_E_ARG;
  if (x_dtype != VSK_BF16 && x_dtype != VSK_FP32 && x_dtype != VSK_MX4) return VSK_E_ARG;
  if ((y_dtype != VSK_BF16 && y_dtype != VSK_FP32) || !stride_ok(y_stride, rows, n)) return VSK_E_ARG;
  const bool mx = x_dtype == VSK_MX4;
  if (mx ? !aligned(x_dev, kAlign) : !stride_ok(x_stride, rows, k) || !aligned(x_dev, element(x_dtype))) return VSK_E_ARG;
  if (!aligned(w_mx_dev, kAlign) || !aligned(y_dev, element(y_dtype)) || !aligned(add_dev, element(y_dtype))) return VSK_E_ARG;
  const ProductWs ws(rows, n, k);
  if (ws_bytes < ws.total || !aligned(ws_dev, kAlign)) return VSK_E_ARG;
  const size_t xb = mx ? vsk_mx4_bytes(rows, k) : extent(rows, k, x_stride, element(x_dtype));
  const size_t wb = vsk_mx4_bytes(n, k), yb = extent(rows, n, y_stride, element(y_dtype));
  if (overlap(y_dev, yb, x_dev, xb) || overlap(y_dev, yb, w_mx_dev, wb)) return VSK_E_ARG;
  if (add_dev && add_dev != y_dev && overlap(y_dev, yb, add_dev, yb)) return VSK_E_ARG;
  if (overlap(ws_dev, ws.total, x_dev, xb) || overlap(ws_dev, ws.total, w_mx_dev, wb) ||
      overlap(ws_dev, ws.total, y_dev, yb) || (add_dev && overlap(ws_dev, ws.total, add_dev, yb)))
    return VSK_E_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  uint8_t* base = static_cast<uint8_t*>(ws_dev);
  Mx4ProductArgs a{};
  a.w = static_cast<const uint8_t*>(w_mx_dev);
  a.rows = rows;
  a.n = n;
  a.k = k;
  a.y = y_dev;
  a.y_fp32 = y_dtype == VSK_FP32;
  a.y_stride = y_stride;
  a.add = add_dev;
  Mx4Split sp = ws.sp;
  int* counter = sp.counters() > 0 ? reinterpret_cast<int*>(base + ws.counter) : nullptr;
  sp.counter = counter;
  sp.part = reinterpret_cast<decltype(sp.part)>(base + ws.part);
  hipError_t e = hipSuccess;
  if (mx) {
    a.x = static_cast<const uint8_t*>(x_dev);
    if (counter) e = launch_fill_zero(counter, static_cast<size_t>(sp.counters()) * 4, s);
  } else if (mx4_takes_rows(x_dtype, x_dev, x_stride, rows, k)) {
    a.x_raw = x_dev;
    a.x_fp32 = x_dtype == VSK_FP32;
    a.x_stride = x_stride;
  } else {
    a.x = base;
    e = launch_mx4_quantise(x_dev, x_dtype, x_stride, rows, k, base, counter, sp.counters(), s);
  }
  if (e != hipSuccess) return VSK_E_HIP;
  if (a.x_raw) return launched(launch_mx4_stream(a, s));
  return launched(sp.rows ? launch_mx4_rows(a, sp, s) : launch_mx4_tile(a, sp, s));
}

}  // extern "C"
