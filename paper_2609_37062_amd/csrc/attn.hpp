// Paged-attention decode interface (see k_attn.hip).
#pragma once

#include "internal.hpp"

namespace vsk {

// The blocks that rows see through a window with sinks, as one list: the ns
// blocks that hold the first `sinks` keys, then blocks wb .. of the window (up
// to the last row's block).  With window 0, or where the two runs meet, ns
// continues into wb and the list is the sequence's own blocks from its start.
struct SpanWalk {
  int lo;  // first key of the window of the first row (0: all of them)
  int ns, wb;
  int nv;  // blocks of the list
  __host__ __device__ int block(int v) const { return v < ns ? v : v - ns + wb; }
};
// Rows with first_end .. last_end keys (position + 1).
__host__ __device__ inline SpanWalk span_walk(int first_end, int last_end, int window, int sinks) {
  SpanWalk g;
  g.lo = window > 0 && first_end > window ? first_end - window : 0;
  g.wb = g.lo / kBlock;
  const int sb = (sinks + kBlock - 1) / kBlock;
  g.ns = sb < g.wb ? sb : g.wb;
  g.nv = g.ns + (last_end + kBlock - 1) / kBlock - g.wb;
  return g;
}

// Blocks of a split where `bps` of them at most cut a walk of nb: even splits, of
// whole steps of a work item's four waves.
__host__ __device__ inline int even_split(int nb, int bps) {
  const int n = (nb + bps - 1) / bps;
  return n > 1 ? ((nb + n - 1) / n + 7) / 8 * 8 : bps;
}
constexpr int kPackedRows = 64;  // rows of a launch whose splits a wave can count

struct AttnArgs {
  const uint16_t* q;  // [R][Nq] bf16
  const uint16_t* pool;
  int layer, n_blocks, Hkv, hd, G, Nq;
  const int32_t* block_table;  // [n_seqs][max_blocks]
  int max_blocks;
  const int32_t* row_seq;
  const int32_t* pos;
  float scale_log2;  // log2(e) / sqrt(hd)
  int bps;         // 16-token blocks per split (multiple of 8)
  int max_splits;  // split work items per (row, KV head) launched
  int split_stride;  // partials per (row, KV head) in the partial buffers
  float* part_o;   // [R][Hkv][split_stride][G][hd]
  float2* part_ml; // [R][Hkv][split_stride][G]
  int* counter;    // [R][Hkv] arrivals of splits, zero between passes
  uint16_t* out;   // o frags (K = Nq)
  int out_Rg;
  // shared prefixes (nullable): a row whose group prefix has P blocks reads
  // only blocks P.. itself; its group's prefix partials sit at split indices
  // 0..pfx_splits[row]-1 and its first split starts from them
  const int32_t* pfx_blocks;  // [R]
  const int32_t* pfx_splits;  // [R]
  const int32_t* rows;        // nullable: the rows of the launch (k_attn_decode indexes it), else all rows
  // routed layer (nullable): per row 1 RUN, 0 Project-Only; a Project-Only
  // row reads no KV and its attention output is zero (Algorithm 1)
  const uint8_t* run_mask;
  int kv_once;  // 1: most KV blocks of the launch are read by one row only (non-temporal loads)
  // general walk (launch_attn_decode with `span`): the row at position p sees
  // keys p - window + 1 .. p (0: every key) and keys 0 .. sinks - 1;
  // out_Rg 0 stores the output row-major ([R][Nq]); ml (nullable) receives
  // each (row, query head)'s softmax maximum (base 2) and 1 / sum
  int window, sinks;
  // of at most kPackedRows rows: their number (else 0), and their splits, which
  // are the launch's work items with none between that has nothing to do
  int packed, packed_items;
  float2* ml;  // [R][Nq / hd]
  // nullable: the scores too, [rows of the launch][Nq / hd][scores_len], key by
  // key of the row's SpanWalk list, -inf where the row does not see it
  float* scores;
  int64_t scores_len;
};

// Causal attention of prefill rows (see k_attn_prefill).
constexpr int kMaxPrefillBlocks = 512;  // key blocks a prefill work item can stage (8192 positions)
constexpr int kMaxSpanBlocks = 1024;    // a general one (16384 positions, the most a model can have)
struct AttnPrefillArgs {
  const uint16_t* q;  // [R][Nq] bf16
  const uint16_t* pool;
  int layer, n_blocks, Hkv, G, Nq;
  const int32_t* block_table;  // [n_seqs][max_blocks]
  int max_blocks;
  const int32_t* kv_len;       // [n_seqs]
  const int32_t* pos;          // [R]
  const int32_t* items;        // [n_items][3]: sequence, first row, rows
  float scale_log2;
  uint16_t* out;  // o frags (K = Nq)
  int out_Rg;
  const uint8_t* run_mask;  // routed layer (nullable): as in AttnArgs
  int window, sinks;        // general walk (launch_attn_rows): as in AttnArgs, as are out_Rg 0 and ml
  float2* ml;
  // general walk: an item's walk cut into `splits` work items, whose sums meet
  // in part_o [R][Hkv][splits][G][hd] and part_ml [R][Hkv][splits][G]
  int splits;
  float* part_o;
  float2* part_ml;
};

// Attention weight per key (see k_attn_mass).
struct AttnMassArgs {
  const uint16_t* q;  // [R][Nq] bf16
  const uint16_t* pool;
  int layer, n_blocks, Hkv, hd, G, Nq;
  const int32_t* block_table;  // [n_seqs][max_blocks]
  int max_blocks;
  const int32_t* kv_len;  // [n_seqs]
  const int32_t* cu_q;    // [n_seqs + 1]
  float scale_log2;
  int window, sinks;
  const float2* ml;  // [R][Nq / hd], as the attention of these rows left them
  float* mass;       // [n_seqs][stride]
  int64_t stride;
  int add;  // 0: mass = the weights, 1: mass += them
  // sequences of several rows, in runs of kMassTile keys [n_tiles][2] (sequence,
  // first key): their weights per (KV head, part of the rows) go to part
  // [Hkv * parts][n_tiles][kMassTile] first, and are added up from there; 0
  // parts: taken as those of one row are
  const int32_t* tiles;
  int n_tiles;
  float* part;
  int parts;
  // sequences of one row: their scores, as the attention left them (nullable:
  // taken again), their rows, and the longest of them
  const float* scores;
  int64_t scores_len;
  const int32_t* rows;
  int n_rows, max_len;
  const int32_t* row_seq;
};

// Shared-prefix attention: each work item reads a run of a group's prefix
// blocks once for up to kPfxCols (row, query head) columns of the group.
struct AttnPrefixArgs {
  const uint16_t* q;  // [R][Nq] bf16
  const uint16_t* pool;
  int layer, n_blocks, Hkv, G, Nq;
  const int32_t* block_table;  // [n_seqs][max_blocks]
  int max_blocks;
  const int32_t* row_seq;
  const int32_t* items;     // [n_items][5]: group, first column, first block, end block, split
  const int32_t* grp_rows;  // rows of every group
  const int32_t* grp_info;  // [n_groups][4]: first entry in grp_rows, rows, prefix blocks, first entry in pfx_tbl
  const int32_t* pfx_tbl;   // every group's prefix block ids
  float scale_log2;
  int split_stride;
  float* part_o;
  float2* part_ml;
};

// grid_splits: split work items launched per (row, KV head), at least the
// most any row has after its shared prefix and at most a.max_splits.
// max_pfx_splits: the most prefix partials any row folds in.
// span: the general walk (window, sinks, row-major output, ml).
hipError_t launch_attn_decode(const AttnArgs& a, int n_rows, int grid_splits, int max_pfx_splits, hipStream_t s,
                              LaunchEvents ev = {}, bool span = false);
hipError_t launch_attn_prefix(const AttnPrefixArgs& a, int n_items, int head_dim, hipStream_t s);
hipError_t launch_attn_prefill(const AttnPrefillArgs& a, int n_items, int head_dim, hipStream_t s);
// the general one of prompt rows (k_rows.hip)
hipError_t launch_attn_rows(const AttnPrefillArgs& a, int n_items, int head_dim, hipStream_t s);
// *wgs: the workgroups that it launched
hipError_t launch_attn_mass(const AttnMassArgs& a, int head_dim, int64_t* wgs, hipStream_t s);

}  // namespace vsk
