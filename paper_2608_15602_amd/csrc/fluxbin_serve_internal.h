// Internal declarations of the operators around the paged 8-bit cache (include/fluxbin_serve.h).
#pragma once

#include "fluxbin_quant_internal.h"
#include "fluxbin_serve.h"

namespace fluxbin {

constexpr int kTreeMaxWords = 16;

// ---- norm and rotation ----
struct RotateSide {
  const uint16_t* src;
  uint16_t* dst;
  const float* weight;   // NULL: not normalized
  int64_t ts, hs, ots, ohs;
};

struct RotateArgs {
  RotateSide side[2];   // queries, keys
  const int32_t* positions;
  const float* freq;
  int64_t rows;
  int32_t Hq, H, R;     // heads of queries, of both; rotated elements
  float eps, magnitude;
};

fluxbin_status launch_qk_rotate(const RotateArgs& a, int D, int interleaved, hipStream_t stream);

// ---- trees of drafted tokens ----
struct MasksArgs {
  const int32_t* offsets;
  const int32_t* context;
  const int32_t* parents;
  uint64_t* masks;
  int32_t* positions;
  int32_t T, B, words;
};

fluxbin_status launch_tree_masks(const MasksArgs& a, hipStream_t stream);

void launch_kv8_tree_few(Kv8AttnArgs a, int D, int cus, hipStream_t stream);   // col_shift 4
uint64_t kv8_tree_workspace(int32_t D, int cus);
fluxbin_status launch_kv8_tree_attention(Kv8AttnArgs a, int D, int cus, hipStream_t stream);

struct Kv8KeepArgs {
  Kv8Args c;
  const int32_t* keep;
  const int32_t* kept;
};

fluxbin_status launch_kv8_keep(const Kv8KeepArgs& a, int D, int cus, hipStream_t stream);

// ---- pages ----
struct PoolArgs {
  int32_t* state;
  int32_t pages, pshift;
};

struct ResizeArgs {
  PoolArgs pool;
  int32_t* table;
  int64_t stride;
  const int32_t* tokens;
  int32_t B, max_blocks;
};

struct ForkArgs {
  PoolArgs pool;
  const int32_t* table;
  int64_t stride;
  const int32_t* context;
  int32_t* child;
  int64_t child_stride;
  const int32_t* source;
  int32_t* copies;
  int32_t B, max_blocks, C, child_blocks;
};

struct CopyArgs {
  const uint8_t* from[2];   // codes of keys, values
  uint8_t* to[2];
  const float* from_scales[2];
  float* to_scales[2];
  const int32_t* copies;
  int64_t n, page_bytes;    // of one side
  int32_t Hkv, from_pages, to_pages;
};

fluxbin_status launch_pages_resize(const ResizeArgs& a, hipStream_t stream);
fluxbin_status launch_pages_fork(const ForkArgs& a, hipStream_t stream);
fluxbin_status launch_kv8_copy_pages(const CopyArgs& a, hipStream_t stream);

}  // namespace fluxbin
