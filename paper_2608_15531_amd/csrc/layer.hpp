// Internal interface between the C ABI of the decoder layer's other operators
// (layer.cpp) and their launchers (kvcache.hip, attention.hip, norm.hip).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "fq.h"

namespace fqi {

// Tokens that the attention kernels take from one page at a time: two such blocks
// are a tile of keys.
constexpr int kKvBlock = 16;
constexpr int kKvTile = 2 * kKvBlock;
// Rows and keys of a workgroup's tile in the kernel for many rows.
constexpr int kTilesRows = 128;
constexpr int kTilesKeys = 64;
constexpr float kLog2e = 1.44269504088896340736f;

// Launch plan of one attention call, from the sizes alone.
struct AttnPlan {
  int kernel;        // FQ_ATTN_*
  int rows;          // rows (token, query head) of a workgroup
  int row_blocks;    // of max_q tokens, per (sequence, KV head)
  int split;         // key ranges
  int tile;          // keys of a tile
  int split_tiles;   // tiles in a range
  int part_rows;     // rows of a partial result
  int dense_blocks;  // blocks of rows are numbered without gaps for shorter sequences
  int64_t workgroups;
  size_t lds_bytes;
  size_t partial_bytes, ws_bytes;   // beyond the counters; with them
};

// The arguments have been checked; false: sizes beyond what the kernels index.
bool plan_attention(const fq_attention& a, const fq_kv_cache& c, AttnPlan* plan);

// Each enqueues its kernel (attention over many rows also that of the join) and returns a hipError_t value (0 on success).
int launch_attention(const AttnPlan& plan, const fq_attention& a, const fq_kv_cache& c,
                     const uint16_t* Q, const int32_t* cu_q, const int32_t* kv_lens,
                     const int32_t* table, uint16_t* O, float* lse, void* workspace,
                     void* stream);
int launch_kv_write(const fq_kv_cache& c, const uint16_t* K, const uint16_t* V,
                    int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride,
                    int64_t v_head_stride, const int64_t* slots, int64_t n_tokens, void* stream);
int launch_kv_read(const fq_kv_cache& c, const int64_t* slots, int64_t n_tokens, void* K, void* V,
                   bool f32, void* stream);
int launch_norm(const fq_norm& n, const void* x, const void* residual, const uint16_t* post_weight,
                const uint16_t* gate, const uint16_t* pre_weight, void* residual_out, uint16_t* h,
                void* stream);

}  // namespace fqi
