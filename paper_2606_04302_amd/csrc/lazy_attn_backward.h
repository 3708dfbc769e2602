// The backward pass's plan: what the host planner writes and the kernels read (no HIP).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "lazy_attn.h"

namespace lazy {

constexpr int kGradTileKeys = 64;  // stored keys of half a key-gradient tile
constexpr int kGradHalves = 2;     // halves of a tile: 64 keys each, wherever they lie
constexpr int kGradRows = 32;      // packed query rows (token * G + head in group) of one step over a tile
// Most workgroups (tiles and row items of 128 rows) for which one launch takes both kinds of items, where 256 rows a
// workgroup would do (head_dim 128 and requests that fill them; otherwise both are one launch always).  One launch
// fills the chip with one kind's workgroups while the other kind's last ones run; two let eight waves share a tile's
// loads and rotation.  us one launch / two, tiles + items of 128 rows: 120 + 512 77 / 94, 328 + 432 92 / 94, 408 + 512
// 150 / 150, 656 + 448 137 / 135, 1024 + 512 228 / 220, 760 + 512 424 / 406, 816 + 1024 1288 / 1237, 1408 + 512 404 /
// 380, 1280 + 4096 17.8 / 16.8 ms; 840 + 1336 789 / 808.  With 128 rows: 136 + 136 37 / 46, 1824 + 480 180 / 194, 2176
// + 512 430 / 446.  Head_dim 64: 136 + 136 25 / 32, 760 + 512 208 / 200, 816 + 1024 603 / 657, 1408 + 512 193 / 193,
// 2056 + 496 163 / 169, 1280 + 4096 8.4 / 8.6 ms.
constexpr int64_t kMostTogether = 1024;

// Up to 64 stored keys (key 0 of KV head 0 at k_off / v_off).
struct GradHalf {
  int64_t k_off, v_off;
  int32_t kst, vst;
  int32_t keys;  // 0: none
  int32_t reserved;
};
static_assert(sizeof(GradHalf) == 32);

// Two halves that the same requests read, or a part of their uses.
struct GradTile {
  GradHalf half[kGradHalves];
  int32_t seg_begin, seg_end;  // the uses (none: the gradient is zero)
  int32_t part;                // -1: the whole tile; otherwise where its partial sums go
  int32_t reserved;
};
static_assert(sizeof(GradTile) == 80);

// One use of a tile: query rows row_begin .. row_end - 1 (packed over the batch) of one request.  They see the keys
// key_begin .. key_end - 1 of each half, key i at position pos + i.
struct GradSeg {
  int32_t row_begin, row_end;
  int32_t pos_shift;  // a token's position less its index in the batch
  int32_t full_from;  // rows from this one on see all of the tile's keys (no mask is needed)
  struct Half {
    int32_t pos;
    int32_t record_pos;  // pos_offset of the record (the rotation of local-position keys)
    int32_t key_begin, key_end;
  } half[kGradHalves];
};
static_assert(sizeof(GradSeg) == 48);

// A tile whose uses were cut into parts: its gradient is the sum of part .. part + parts - 1.
struct GradMerge {
  GradHalf half[kGradHalves];
  int32_t part, parts;
  int32_t reserved[2];
};
static_assert(sizeof(GradMerge) == 80);

// Query gradient: rows row0 .. of a request against key split `split` of `splits`.
struct GradRowItem {
  int32_t request, row0, split, splits;
};

// Tokens t0 .. t0 + tokens - 1 of one request, whose query gradient comes in `splits` partial sums.
struct GradBlock {
  int32_t t0, tokens, pos_shift, splits;
};

// Where the arrays lie in the plan (all multiples of 8 bytes; the blocks come first so that they are 16-byte aligned).
struct GradPlanLayout {
  size_t blocks, rows, tiles, segs, merges, bytes;
  explicit GradPlanLayout(const lazy_backward_info_t& i) {
    size_t at = 0;
    const auto put = [&at](size_t bytes) {
      const size_t here = at;
      at += bytes;
      return here;
    };
    blocks = put(sizeof(GradBlock) * (size_t)i.num_blocks);
    rows = put(sizeof(GradRowItem) * (size_t)i.num_row_items);
    segs = put(sizeof(GradSeg) * (size_t)i.num_segments);
    tiles = put(sizeof(GradTile) * (size_t)i.num_tiles);
    merges = put(sizeof(GradMerge) * (size_t)i.num_merges);
    bytes = at;
  }
};

// Rotated queries are the sum of two bf16 numbers; ALiBi rotates nothing, one is exact.
inline int query_parts(const lazy_attn_params_t* p) { return p->rope_style == LAZY_ALIBI ? 1 : 2; }

// Where the backward pass keeps its intermediate results (bytes into the workspace).
struct GradWorkLayout {
  size_t q, dout, info, dq, parts, bytes;
  GradWorkLayout(int hq, int hkv, int d, int query_parts, const lazy_backward_info_t& i) {
    const size_t rows = (size_t)i.total_q * (size_t)hq;
    size_t at = 0;
    const auto put = [&at](size_t bytes) {
      const size_t here = at;
      at += (bytes + 255) & ~(size_t)255;
      return here;
    };
    q = put(query_parts * rows * d * sizeof(uint16_t));                          // rotated queries
    dout = put(rows * d * sizeof(uint16_t));                                     // packed like the queries
    info = put(rows * 2 * sizeof(float));                                        // -lse of each row, then -delta
    dq = put((size_t)(i.row_slots > 1 ? i.row_slots : 0) * rows * d * sizeof(float));  // partial query gradients
    // partial key and value gradients
    parts = put((size_t)i.num_parts * hkv * 2 * kGradHalves * kGradTileKeys * d * sizeof(float));
    bytes = at;
  }
};

}  // namespace lazy
