// Arguments of the kernels around the attention call: norm and rotation (asa_norm.hip), 8-bit
// cache (asa_cache.hip).
#pragma once

#include "asa_common.hpp"

namespace asa {

// Whether one launch holds the workgroups: HIP counts the threads along an axis in 32 bits.
inline bool launch_fits(int64_t workgroups, int threads) { return workgroups * threads < (int64_t)1 << 32; }

// Queries (side 0) or keys (side 1) of asa_qk_norm_rope and its backward.
struct NormSide {
  const void *src;        // x
  const void *grad;       // backward: gradient of the output
  void *dst;              // forward: the output; backward: dx
  TensorView in, out, dx; // strides of x; of the output and its gradient; of dx
  const float *w, *b;     // [d] or null
  float *partial;         // backward: [dweight, dbias][groups][d]
  float *dw, *db;         // [d] or null
  int heads, chunks, groups;
};
struct NormArgs {
  NormSide side[2];
  const int32_t *start;
  const float *cos_table, *sin_table;
  int B, L, tokens, tiles;
  int rot, table_rows, first_row;
  float eps;
};
int plan_norm(NormArgs *a, int D, bool backward);           // fills in the work; asa_status
size_t norm_partial_bytes(const NormSide &s, int D);
hipError_t launch_norm(const NormArgs &a, int D, bool layer, int pairing, bool backward, hipStream_t st);

// One of the two tensors of a cache call.
struct CacheSide {
  void *codes;            // [B, H_kv, max_blocks, block * d]
  float *scale;           // [B, H_kv, max_blocks]
  void *rows;             // [B, H_kv, L, d] bf16, read or written
  TensorView view;
  bool transposed;        // V's order of the codes
};
struct CacheArgs {
  CacheSide side[2];
  int n_sides;
  const int32_t *start, *count;
  int B, H, L, max_blocks;
  int reached;            // blocks of a sequence that L tokens reach into, at most
};
int plan_cache(const CacheArgs &a, int D, int block);       // asa_status
hipError_t launch_cache_write(const CacheArgs &a, int D, int block, hipStream_t st);
hipError_t launch_cache_read(const CacheArgs &a, int D, int block, hipStream_t st);

struct CacheAttnArgs {
  const void *q, *k, *v;
  const float *k_scale, *v_scale;
  const int32_t *length, *row_ptr, *col_idx;
  void *o;
  float *lse;
  float *partial;         // [unit][split][row][D + 2]: sums over a split's keys, maximum and denominator
  TensorView qv, ov;
  int B, H, H_kv, group, L, block, max_blocks;
  int n_qblocks;          // blocks of queries
  int tiles, tile_rows;   // row tiles of a block of queries, rows of a tile
  int rows_kept;          // rows of a tile that exist, at most (pitch of `partial`)
  int splits, units;      // units: (sequence, key head, block of queries, row tile)
  float scale_log2;       // scale * log2(e)
};
struct CacheAttnPlan {
  int tiles, tile_rows, rows_kept, splits, n_qblocks;
  int64_t units;          // (sequence, key head, block of queries, row tile)
};
int plan_cache_attn(const Problem &pb, int H_kv, int max_blocks, bool lists, CacheAttnPlan *plan);   // asa_status
size_t cache_attn_workspace_bytes(const Problem &pb, const CacheAttnPlan &plan);
hipError_t launch_cache_attn(const CacheAttnArgs &a, int D, hipStream_t st);

}  // namespace asa
