// Eviction by accumulated attention weight (see k_evict.hip).
#pragma once

#include "internal.hpp"

namespace vsk {

// Metadata of so few ints goes to the selection as an argument, and from there
// to the buffer: one short sequence 25.5 us with a copy before it, 19.7 so.
constexpr int kEvictSmall = 896;
struct EvictSmall {
  int32_t v[kEvictSmall];
};
constexpr int kEvictMaxLen = 16384;  // cached tokens of a sequence (max_pos is at most that)

struct EvictArgs {
  uint16_t* pool;
  int n_layers, n_blocks, Hkv, hd;
  // per sequence of the call: [n][4]: cached tokens, tokens kept, first entry in src_tbl and in dst_tbl
  // (a destination block has 16 entries in from)
  int32_t* info;
  const int32_t* src_tbl;
  const int32_t* dst_tbl;
  int n_ints;  // of the three together
  int32_t* from;  // written by the selection: the source slot of each kept token
  int sinks, recent;
  const float* mass;
  int64_t mass_stride;
  float* mass_out;     // nullable
  int32_t* kept;       // [n][out_stride]
  int32_t* slots;      // nullable
  int64_t out_stride;
};
// meta: the `ints` ints that info, src_tbl and dst_tbl point to, where they are
// few and not in the buffer yet (nullable)
hipError_t launch_evict(const EvictArgs& a, const int32_t* meta, size_t ints, int n, int max_len, int max_keep,
                        hipStream_t s);

}  // namespace vsk
