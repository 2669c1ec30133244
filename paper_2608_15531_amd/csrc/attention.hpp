// What the kernels of fq_paged_attention share: arguments, the rows and key tiles of a
// workgroup, the joining of key ranges.
#pragma once

#include <hip/hip_runtime.h>

#include <climits>

#include "blocks.hpp"
#include "device.hpp"
#include "internal.hpp"
#include "lanes.hpp"
#include "layer.hpp"

namespace fqk {

using fqi::kKvBlock;
using fqi::kKvTile;
using fqi::TileRange;

struct AttnArgs {
  const uint16_t* Q;
  const char* k;
  const char* v;
  const uint32_t* k_meta;
  const uint32_t* v_meta;
  const int32_t* cu_q;
  const int32_t* kv_lens;
  const int32_t* table;
  uint16_t* O;
  float* lse;
  float* partials;
  uint32_t* counters;
  int64_t page_stride, head_stride, meta_page_stride, meta_head_stride, table_stride;
  int64_t q_token, q_head, o_token, o_head, total_q;
  uint32_t token_stride;   // bytes
  uint32_t page_blocks;    // kKvBlock-token blocks in a page
  uint64_t page_magic;     // ceil(2^36 / page_blocks): block / page_blocks by one product
  uint32_t n_pages;
  int group;               // query heads per KV head
  int n_heads, n_kv_heads;
  int max_q, max_kv, window, sinks;
  int row_blocks, split, split_tiles, part_rows;
  int dense_blocks;        // how blocks are numbered: by the rows before, or row_blocks a sequence
  float scale_log2;        // scale * log2(e): the softmax runs in powers of two
};

typedef __bf16 bf16x2v __attribute__((__vector_size__(4)));

__device__ __forceinline__ uint32_t pk_bf16(float lo, float hi) {
  const bf16x2v r = {static_cast<__bf16>(lo), static_cast<__bf16>(hi)};
  return __builtin_bit_cast(uint32_t, r);
}

__device__ __forceinline__ f32x4_t mfma16(bf16x8_t a, bf16x8_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// The page (a number in range, whatever the table holds) and the token in it of a block of
// kKvBlock keys.  `key` < 2^28, so the product with the rounded-up reciprocal is exact.
struct BlockPlace {
  uint32_t page, token;
};
__device__ __forceinline__ BlockPlace block_place(const AttnArgs& a, const int32_t* table, int key) {
  const uint32_t blk = uint32_t(key) / kKvBlock;
  const uint32_t col = uint32_t((uint64_t(blk) * a.page_magic) >> 36);
  // (as constant memory, so that it is a scalar load: among vector loads, waiting for it
  // would wait for those before it)
  typedef __attribute__((address_space(4))) const uint32_t constant_u32;
  const uint32_t page = reinterpret_cast<constant_u32*>(reinterpret_cast<uintptr_t>(table))[col];
  return BlockPlace{min(page, a.n_pages - 1), (blk - col * a.page_blocks) * kKvBlock};
}

// What a workgroup works on: a block of ROWS rows of one (sequence, KV head), one range of
// the key tiles that the block sees.
//
// KV heads vary fastest over the workgroups, which go to the eight XCDs in turn: the
// blocks and ranges that read the same keys meet in one L2 (with 8 KV heads, or any
// multiple or divisor).  The last rows, which see the most keys, come first.  Empty
// workgroups (past a shorter sequence's rows or keys) lie together rather than in turn
// with others, which would leave whole shader engines idle.
struct Item {
  int head, seq, rb, part, n_parts;
  int64_t t0;          // first new token of the sequence
  uint32_t row0;       // first row of the block (the plan keeps rows below 2^31)
  int rows;
  int64_t number;      // among all blocks and heads
  int p0;              // position of the sequence's first new token
  int tok_hi;          // the block's last token
  int kv_seen;
  int p_lo, p_hi;      // last keys that the block's first and last row see
  TileRange tr;
  int i_lo, i_hi;      // this range of the block's tiles

  // The block's rows and tiles; false: the sequence has no such rows.
  template <int ROWS, int TILE>
  __device__ __forceinline__ bool set_rows(const AttnArgs& a, int seq_, int rb_, int head_) {
    seq = seq_;
    rb = rb_;
    head = head_;
    t0 = min(max(int64_t(a.cu_q[seq]), int64_t(0)), a.total_q);
    const int64_t t1 = min(max(int64_t(a.cu_q[seq + 1]), t0), a.total_q);
    const int q_all = int(t1 - t0);               // before the bound: positions count from the end
    const int kv_len = max(a.kv_lens[seq], 0);
    const uint32_t group = uint32_t(a.group), n_rows = uint32_t(min(q_all, a.max_q)) * group;
    row0 = uint32_t(rb) * ROWS;
    if (row0 >= n_rows) return false;
    rows = int(min(n_rows - row0, uint32_t(ROWS)));
    const int tok_lo = int(row0 / group);
    tok_hi = int((row0 + rows - 1) / group);
    number = (a.dense_blocks ? fqi::dense_number(t0, a.group, ROWS, seq, rb) : int64_t(seq) * a.row_blocks + rb) *
                 a.n_kv_heads + head;
    p0 = kv_len - q_all;
    kv_seen = min(kv_len, a.max_kv);
    p_lo = min(p0 + tok_lo, kv_seen - 1);
    p_hi = min(p0 + tok_hi, kv_seen - 1);
    tr = fqi::tile_range<TILE>(p_lo, p_hi, a.window, a.sinks);
    return true;
  }
  // how many ranges its tiles fall into
  __device__ __forceinline__ int parts(const AttnArgs& a) const {
    return fqi::range_count(tr.n, a.split_tiles, a.split);
  }
  // What this workgroup works on; false: nothing.
  template <int ROWS, int TILE>
  __device__ __forceinline__ bool set(const AttnArgs& a) {
    const int x = int(blockIdx.x) / a.n_kv_heads;
    part = x % a.split;
    if (!set_rows<ROWS, TILE>(a, int(blockIdx.y), a.row_blocks - 1 - x / a.split, int(blockIdx.x) % a.n_kv_heads))
      return false;
    n_parts = parts(a);
    if (part >= n_parts) return false;
    i_lo = part * a.split_tiles;
    i_hi = min(i_lo + a.split_tiles, tr.n);
    return true;
  }
  // the tile of keys [key0, key0 + TILE) is seen whole by every row of the block
  template <int TILE>
  __device__ __forceinline__ bool whole(const AttnArgs& a, int key0) const {
    return key0 + TILE - 1 <= p_lo && (a.window == 0 || key0 > p0 + tok_hi - a.window || key0 + TILE <= a.sinks);
  }
};

// A lane's row.
struct Row {
  bool in;
  int token, head;
  int pos;       // last key that it sees
  int win_lo;    // first key of its window
  __device__ __forceinline__ void set(const AttnArgs& a, const Item& it, int r) {
    in = r < it.rows;
    const uint32_t row = it.row0 + uint32_t(min(r, it.rows - 1)), group = uint32_t(a.group);
    token = int(row / group);
    head = it.head * a.group + int(row - uint32_t(token) * group);
    pos = in ? min(it.p0 + token, it.kv_seen - 1) : -1;
    win_lo = a.window > 0 ? it.p0 + token - a.window + 1 : INT_MIN;
  }
  __device__ __forceinline__ bool sees(const AttnArgs& a, int key) const {
    return key <= pos && (key >= win_lo || key < a.sinks);
  }
};

constexpr float kNegInf = -__builtin_inff();

// By how much a score (before the factor c2 > 0) may pass the running maximum until the sums
// move to it: 2^8 in weights.  Finite for the smallest c2 too: -infinity, the first maximum,
// plus an infinity would be no number, and no score would pass it.
__device__ __forceinline__ float grow_of(float c2) { return fminf(8.f / c2, 3.402823466e38f); }

// Infinities and NaN of a bf16 V row that some rows of a block see and others do not: in
// the matrix product their zero weights would make NaN of them.  So in tiles that are not
// seen whole, V's values that are not finite enter the product as 0, and where there were
// any, a second walk over those tiles adds them to the rows that do see them: times a
// positive weight, an infinity or a NaN is itself.  A weight too small for fp32 is 0, and makes
// a NaN of an infinity in the product of a whole tile and where sums are moved or joined by
// it, but not in this walk: the channel is not finite either way, and no more is promised.
__device__ __forceinline__ bool nonfinite_pair(uint32_t w) {
  return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u;
}
__device__ __forceinline__ uint32_t finite_pair(uint32_t w) {
  return w & (((w & 0x7F80u) == 0x7F80u ? 0u : 0xFFFFu) | ((w & 0x7F800000u) == 0x7F800000u ? 0u : 0xFFFF0000u));
}
// The value if it is not finite, else 0.
__device__ __forceinline__ float if_nonfinite(uint32_t bits) {
  return (bits & 0x7F80u) == 0x7F80u ? bf16_bits_to_f32(bits) : 0.f;
}

// Calls add(key, row) for the V rows of tiles i0, i0 + step, .. of the item that are not
// seen whole.
template <int TILE, class F>
__device__ __forceinline__ void walk_partial_tiles(const AttnArgs& a, const Item& it, const int32_t* table,
                                                   const char* vh, int i0, int step, F&& add) {
#pragma unroll 1
  for (int i = i0; i < it.i_hi; i += step) {
    const int key0 = it.tr.tile(i) * TILE;
    if (it.whole<TILE>(a, key0)) continue;
#pragma unroll 1
    for (int key = key0; key < min(key0 + TILE, it.kv_seen); ++key) {
      const BlockPlace at = block_place(a, table, key & ~(kKvBlock - 1));
      add(key, reinterpret_cast<const uint16_t*>(vh + at.page * a.page_stride +
                                                 int64_t(at.token + (key & (kKvBlock - 1))) * a.token_stride));
    }
  }
}

// Workgroups of the join of a block of kTilesRows rows, with 128 channels.
constexpr int kJoinBlocks = fqi::kTilesRows / 16;

// attention_tiles.hip: the kernel for many rows, on `grid`.
size_t attn_tiles_lds(int head_dim);
int launch_attn_tiles(const AttnArgs& g, int kind, int head_dim, dim3 grid, hipStream_t s);

}  // namespace fqk
