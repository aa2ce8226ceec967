// Eviction by accumulated attention weight (see k_evict.hip).
#pragma once

#include "internal.hpp"

namespace vsk {

constexpr int kEvictMaxLen = 16384;  // cached tokens of a sequence (max_pos is at most that)

struct EvictArgs {
  uint16_t* pool;
  int n_layers, n_blocks, Hkv, hd;
  // per sequence of the call: [n][4]: cached tokens, tokens kept, first entry in src_tbl and in dst_tbl
  // (a destination block has 16 entries in from)
  const int32_t* info;
  const int32_t* src_tbl;
  const int32_t* dst_tbl;
  int32_t* from;  // written by the selection: the source slot of each kept token
  int sinks, recent;
  const float* mass;
  int64_t mass_stride;
  float* mass_out;     // nullable
  int32_t* kept;       // [n][out_stride]
  int32_t* slots;      // nullable
  int64_t out_stride;
};
hipError_t launch_evict(const EvictArgs& a, int n, int max_len, int max_keep, hipStream_t s);

}  // namespace vsk
