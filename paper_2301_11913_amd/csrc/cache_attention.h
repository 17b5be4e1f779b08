// What the kernels of the attention over the cache share.
#pragma once
#include "cache.h"

namespace swarm {

constexpr int kAttnTile = 64;          // cached tokens at a time

struct AttnArgs {
  CacheArgs c;
  const void* q;
  void* out;
  const uint64_t* tree;
  size_t q_pitch, out_pitch;
  float *part_o, *part_ml;     // splits > 1: [unit][rows][d_head], [unit][rows][2]: sums relative to 2^maximum, and maximum and total
  int group;                   // query heads per key / value head; row r of a head is token r / group, query head r % group of it
  int row_groups, splits, chunk;   // a unit: one sequence, head, group of rows and split, which takes `chunk` tiles (the last one the rest)
  bool s16;
};

// bf16, many rows: 32 * row_waves rows per workgroup, row_waves 2 or 4 (cache_attention_rows.hip)
swarm_status cache_attention_rows_launch(const AttnArgs& a, int dh, int row_waves, hipStream_t st);

}  // namespace swarm
