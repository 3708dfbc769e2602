// Host planner of the backward pass: gathers the uses of every stored key into tiles, balances their work, and cuts
// the query gradient into row tiles and key splits.  Pure C++ with no HIP dependency: it runs on host copies of the
// tables and is testable without a GPU.
#include "lazy_attn_backward.h"

#include <string.h>

#include <algorithm>
#include <functional>
#include <map>
#include <tuple>
#include <vector>

#include "lazy_attn_params.h"

namespace {

using lazy::GradBlock, lazy::GradHalf, lazy::GradMerge, lazy::GradRowItem, lazy::GradSeg, lazy::GradTile;
using lazy::kGradRows, lazy::kGradTileKeys;

// One use of a record by a request.
struct Use {
  int32_t request, record;
};
// Records whose stored keys overlap, as one run of keys: `keys` keys from k_off / v_off, the uses in table order.
struct Slab {
  int64_t k_off, v_off;
  int32_t kst, vst;
  int64_t keys;
  std::vector<Use> uses;
};

// Do the head blocks [off + g * stride * d, + keys * d) of different slabs overlap?
bool blocks_overlap(const std::vector<Slab>& slabs, int hkv, int d, bool values) {
  std::vector<std::pair<int64_t, int64_t>> at;
  at.reserve(slabs.size() * (size_t)hkv);
  for (const Slab& s : slabs)
    for (int g = 0; g < hkv; ++g) {
      const int64_t b = values ? s.v_off + (int64_t)g * s.vst * d : s.k_off + (int64_t)g * s.kst * d;
      at.emplace_back(b, b + s.keys * d);
    }
  std::sort(at.begin(), at.end());
  for (size_t i = 1; i < at.size(); ++i)
    if (at[i].first < at[i - 1].second) return true;
  return false;
}

int64_t steps_of(const GradSeg& s) { return (s.row_end - s.row_begin + kGradRows - 1) / kGradRows; }

// Key splits of every request's row tiles.  A candidate lets no work item have more than a given number of key tiles;
// the one with the least estimated time is taken: the makespan of the items, longest first, on the workgroups that the
// chip holds, where an item costs its tiles and kItemTiles more (its prologue and its result), plus the partial
// results' way to memory and back and kFinishUs for the launch that adds them up (a request in one split writes its
// gradient by itself).  A tile of 256 rows takes a workgroup 8.8 us at head_dim 128.  With 3.7 instead, which splits
// less, one document of 1024 tokens and 32 / 8 heads took 166 us instead of 151 (head_dim 64: 87 instead of 75), 16
// heads of 64 over one KV head and 800 tokens 57 instead of 52; but 512 tokens 68 instead of 70 (64: 38 instead of 42),
// 16 / 1 heads of 128 and 1024 tokens 102 instead of 115.  kItemTiles of 1.5 to 3 are within 2% of each other but for
// one document (512 tokens: 76 with 1.5, 70 with 3).  More splits are taken for a gain of 3% only.
constexpr double kItemTiles = 3, kTileUs = 8.8, kBytesPerUs = 4.5e6, kFinishUs = 15, kClose = 0.97;
std::vector<int32_t> row_splits(const std::vector<int64_t>& key_tiles, const int32_t* q_start, int batch, int G, int hkv,
                                int d, int row_blocks) {
  const int slots = lazy::kNumCUs * (row_blocks == 2 ? 1 : 2);
  const int64_t bm = 128 * row_blocks;
  const double tile_us = kTileUs * (row_blocks / 2.0) * (d / 128.0) * (slots / (double)lazy::kNumCUs);
  const int64_t longest = batch > 0 ? *std::max_element(key_tiles.begin(), key_tiles.end()) : 0;
  std::vector<int32_t> best(batch, 1), trial(batch, 1);
  double least = -1;
  int64_t last = -1;
  for (int64_t s = 1; s <= std::min<int64_t>(32, std::max<int64_t>(1, longest)); ++s) {
    const int64_t most = lazy::ceil_div(longest, s);
    if (most == last) continue;
    last = most;
    std::vector<std::pair<double, int64_t>> items;  // cost, how many
    double bytes = 0;
    int64_t count = 0;
    for (int r = 0; r < batch; ++r) {
      const int64_t rows = (int64_t)(q_start[r + 1] - q_start[r]) * G;
      trial[r] = (int32_t)std::max<int64_t>(1, lazy::ceil_div(key_tiles[r], std::max<int64_t>(1, most)));
      if (rows == 0) continue;
      const int64_t n = lazy::ceil_div(rows, bm) * hkv * trial[r];
      items.emplace_back((double)key_tiles[r] / trial[r] + kItemTiles, n);
      if (trial[r] > 1) bytes += 8.0 * rows * hkv * d * trial[r];
      count += n;
    }
    std::sort(items.begin(), items.end(), [](const auto& a, const auto& b) { return a.first > b.first; });
    double span = 0;
    if (count <= 1 << 13) {
      std::vector<double> busy(slots, 0.0);  // a heap with the first workgroup to end on top
      for (const auto& it : items)
        for (int64_t i = 0; i < it.second; ++i) {
          std::pop_heap(busy.begin(), busy.end(), std::greater<double>());
          busy.back() += it.first;
          span = std::max(span, busy.back());
          std::push_heap(busy.begin(), busy.end(), std::greater<double>());
        }
    } else {
      for (const auto& it : items) span += it.first * (double)it.second / slots;
      span += items.front().first / 2;
    }
    const double cost = span * tile_us + bytes / kBytesPerUs + (bytes > 0 ? kFinishUs : 0.0);
    if (least < 0 || cost < kClose * least) {
      least = cost;
      best = trial;
    }
  }
  return best;
}

int make_plan(const lazy_attn_params_t* p, const int32_t* q_start, const int32_t* q_pos0, const lazy_chunk_t* chunks,
              const int32_t* chunk_start, int32_t batch, void* plan, size_t capacity, lazy_backward_info_t* info) {
  const int d = p->head_dim, hkv = p->num_kv_heads, G = p->num_q_heads / p->num_kv_heads;
  if (q_start[0] != 0 || chunk_start[0] != 0) return LAZY_EDATA;
  for (int r = 0; r < batch; ++r) {
    const int64_t n = (int64_t)q_start[r + 1] - q_start[r];
    if (n < 0 || chunk_start[r + 1] < chunk_start[r]) return LAZY_EDATA;
    if (n > 0 && (q_pos0[r] < 0 || q_pos0[r] + n > LAZY_MAX_POS)) return LAZY_EDATA;
  }
  const int64_t total_q = q_start[batch];
  // A packed row is divided by G with a 32-bit multiplication in the kernels.
  if (total_q * G * G >= (int64_t)1 << 32 || total_q * G >= INT32_MAX) return LAZY_EUNSUPPORTED;

  constexpr int64_t kMostOffset = (int64_t)1 << 56;  // sums of offsets and strides do not overflow
  // Slabs: records with the same strides, in storage order, joined where their keys overlap.
  std::vector<Use> uses;
  for (int r = 0; r < batch; ++r)
    for (int i = chunk_start[r]; i < chunk_start[r + 1]; ++i) {
      const lazy_chunk_t& c = chunks[i];
      if (c.len < 0 || c.k_stride < c.len || c.v_stride < c.len || c.k_offset < 0 || c.v_offset < 0 ||
          c.k_offset > kMostOffset || c.v_offset > kMostOffset ||
          (c.k_offset & 7) || (c.v_offset & 7) || c.pos_offset < 0 || (int64_t)c.pos_offset + c.len > LAZY_MAX_POS)
        return LAZY_EDATA;
      if (c.len > 0) uses.push_back({r, i});
    }
  const auto key = [&](const Use& u) {
    const lazy_chunk_t& c = chunks[u.record];
    return std::make_tuple(c.k_stride, c.v_stride, c.k_offset, c.v_offset, u.record);
  };
  std::sort(uses.begin(), uses.end(), [&](const Use& a, const Use& b) { return key(a) < key(b); });
  std::vector<Slab> slabs;
  for (const Use& u : uses) {
    const lazy_chunk_t& c = chunks[u.record];
    if (!slabs.empty()) {
      Slab& s = slabs.back();
      const int64_t off = c.k_offset - s.k_off;
      if (s.kst == c.k_stride && s.vst == c.v_stride && off < s.keys * d && off % d == 0 && c.v_offset - s.v_off == off) {
        s.keys = std::max(s.keys, off / d + c.len);
        s.uses.push_back(u);
        continue;
      }
    }
    slabs.push_back({c.k_offset, c.v_offset, c.k_stride, c.v_stride, c.len, {u}});
  }
  if (blocks_overlap(slabs, hkv, d, false) || blocks_overlap(slabs, hkv, d, true)) return LAZY_EDATA;

  // 64-key halves and their uses.
  struct Use64 {
    int32_t request, row_begin, full_from;
    GradSeg::Half half;
  };
  struct Half {
    GradHalf h;
    std::vector<Use64> uses;
  };
  std::vector<Half> halves;
  for (Slab& s : slabs) {
    std::sort(s.uses.begin(), s.uses.end(), [](const Use& a, const Use& b) { return a.record < b.record; });
    const size_t first = halves.size();
    for (int64_t k = 0; k < s.keys; k += kGradTileKeys)
      halves.push_back({{s.k_off + k * d, s.v_off + k * d, s.kst, s.vst,
                         (int32_t)std::min<int64_t>(kGradTileKeys, s.keys - k), 0},
                        {}});
    for (const Use& u : s.uses) {
      const lazy_chunk_t& c = chunks[u.record];
      const int32_t r = u.request, qs = q_start[r], n = q_start[r + 1] - qs;
      const int64_t begin = (c.k_offset - s.k_off) / d, end = begin + c.len;
      for (int64_t k = begin / kGradTileKeys * kGradTileKeys; k < end; k += kGradTileKeys) {
        Half& t = halves[first + k / kGradTileKeys];
        Use64 g = {};
        g.request = r;
        g.half.key_begin = (int32_t)std::max<int64_t>(0, begin - k);
        g.half.key_end = (int32_t)std::min<int64_t>(t.h.keys, end - k);
        g.half.pos = (int32_t)(c.pos_offset + k - begin);
        g.half.record_pos = c.pos_offset;
        int32_t tb = 0, tf = 0;  // first token that sees a key, and all of them
        if (p->causal && n > 0) {
          tb = (int32_t)std::min<int64_t>(n, std::max<int64_t>(0, (int64_t)g.half.pos + g.half.key_begin - q_pos0[r]));
          tf = (int32_t)std::min<int64_t>(n, std::max<int64_t>(0, (int64_t)g.half.pos + g.half.key_end - 1 - q_pos0[r]));
        }
        if (tb >= n) continue;
        g.row_begin = (qs + tb) * G;
        g.full_from = g.half.key_begin == 0 && g.half.key_end == t.h.keys ? (qs + tf) * G : (qs + n) * G;
        t.uses.push_back(g);
      }
    }
  }

  // Tiles: two halves that the same requests read, in the order in which they come (the next 64 keys of a chunk, or the
  // next block of a paged one); a half that finds no partner stays alone.
  struct Tile {
    GradTile t;
    std::vector<GradSeg> segs;
    int64_t steps = 0;
  };
  std::vector<Tile> tiles;
  std::map<std::vector<int32_t>, size_t> open;  // requests of the uses -> a tile with one half
  std::vector<int32_t> who;
  for (const Half& h : halves) {
    who.clear();
    for (const Use64& u : h.uses) who.push_back(u.request);
    const auto found = open.find(who);
    const int at = found == open.end() ? 0 : 1;
    if (at == 0) {
      open.emplace(who, tiles.size());
      tiles.emplace_back();
      tiles.back().t.part = -1;
      tiles.back().segs.resize(h.uses.size());
    }
    Tile& t = at == 0 ? tiles.back() : tiles[found->second];
    if (at == 1) open.erase(found);
    t.t.half[at] = h.h;
    for (size_t i = 0; i < h.uses.size(); ++i) {
      const Use64& u = h.uses[i];
      GradSeg& s = t.segs[i];
      const int32_t r = u.request;
      s.row_begin = at == 0 ? u.row_begin : std::min(s.row_begin, u.row_begin);
      s.full_from = at == 0 ? u.full_from : std::max(s.full_from, u.full_from);
      s.row_end = q_start[r + 1] * G;
      s.pos_shift = q_pos0[r] - q_start[r];
      s.half[at] = u.half;
    }
  }
  int64_t total_steps = 0;
  for (Tile& t : tiles)
    for (const GradSeg& s : t.segs) t.steps += steps_of(s);
  for (const Tile& t : tiles) total_steps += t.steps;

  // Parts: no work item should take much longer than half of a workgroup's share of the whole (a CU holds two), nor so
  // little that its loads and its final sums dominate.
  const int64_t limit = std::max<int64_t>(8, lazy::ceil_div(total_steps * hkv, 2 * 2 * lazy::kNumCUs));
  std::vector<GradTile> out_tiles;
  std::vector<GradSeg> out_segs;
  std::vector<GradMerge> merges;
  std::vector<int64_t> cost;
  int32_t num_parts = 0;
  for (Tile& t : tiles) {
    const int64_t parts = std::max<int64_t>(1, lazy::ceil_div(t.steps, limit + limit / 2));
    if (parts > 1)
      merges.push_back({{t.t.half[0], t.t.half[1]}, num_parts, (int32_t)parts, {0, 0}});
    size_t at = 0;
    int64_t done = 0;
    for (int64_t part = 0; part < parts; ++part) {
      GradTile g = t.t;
      g.part = parts > 1 ? num_parts++ : -1;
      g.seg_begin = (int32_t)out_segs.size();
      const int64_t until = t.steps * (part + 1) / parts;
      const int64_t before = done;
      while (done < until) {
        GradSeg& s = t.segs[at];
        const int64_t take = std::min(until - done, steps_of(s));
        GradSeg piece = s;
        piece.row_end = (int32_t)std::min<int64_t>(s.row_end, (int64_t)s.row_begin + take * kGradRows);
        out_segs.push_back(piece);
        done += take;
        s.row_begin = piece.row_end;
        if (s.row_begin == s.row_end) ++at;
      }
      g.seg_end = (int32_t)out_segs.size();
      out_tiles.push_back(g);
      cost.push_back(done - before);
    }
  }
  // Longest first: the last items to start are short ones.
  std::vector<int32_t> order(out_tiles.size());
  for (size_t i = 0; i < order.size(); ++i) order[i] = (int32_t)i;
  std::stable_sort(order.begin(), order.end(), [&](int32_t a, int32_t b) { return cost[a] > cost[b]; });

  // Query gradient: 128 rows a workgroup, in one launch with the tiles, or 256 (eight waves; head_dim 128 only) in one of
  // its own where requests fill such row tiles and there is more work than kMostTogether.
  int64_t rows1 = 0, rows2 = 0;
  std::vector<int64_t> key_tiles(batch);
  for (int r = 0; r < batch; ++r) {
    const int64_t rows = (int64_t)(q_start[r + 1] - q_start[r]) * G;
    rows1 += lazy::ceil_div(rows, 128) * 128;
    rows2 += lazy::ceil_div(rows, 256) * 256;
    for (int i = chunk_start[r]; i < chunk_start[r + 1]; ++i)
      key_tiles[r] += lazy::ceil_div(chunks[i].len, kGradTileKeys);
  }
  int row_blocks = 1;
  std::vector<int32_t> splits_of = row_splits(key_tiles, q_start, batch, G, hkv, d, 1);
  if (d == 128 && rows1 > 0 && 4 * rows2 <= 5 * rows1) {
    int64_t items = 0;
    for (int r = 0; r < batch; ++r)
      items += lazy::ceil_div((int64_t)(q_start[r + 1] - q_start[r]) * G, 128) * splits_of[r];
    if (((int64_t)out_tiles.size() + items) * hkv > lazy::kMostTogether) {
      row_blocks = 2;
      splits_of = row_splits(key_tiles, q_start, batch, G, hkv, d, 2);
    }
  }
  const int bm = 128 * row_blocks;
  std::vector<GradRowItem> rows;
  std::vector<GradBlock> blocks;
  std::vector<int64_t> row_cost;
  int32_t row_slots = 0;
  const int block_tokens = std::max(1, std::min(16, 32 / p->num_q_heads));
  for (int r = 0; r < batch; ++r) {
    const int32_t qs = q_start[r], n = q_start[r + 1] - qs;
    if (n == 0) continue;
    const int32_t splits = splits_of[r];
    row_slots = std::max(row_slots, splits);
    for (int64_t row0 = 0; row0 < (int64_t)n * G; row0 += bm)
      for (int s = 0; s < splits; ++s) {
        rows.push_back({r, (int32_t)row0, s, splits});
        row_cost.push_back(key_tiles[r] / splits);
      }
    for (int32_t t = 0; t < n; t += block_tokens)
      blocks.push_back({qs + t, std::min(block_tokens, n - t), q_pos0[r] - qs, splits});
  }
  std::vector<int32_t> row_order(rows.size());
  for (size_t i = 0; i < row_order.size(); ++i) row_order[i] = (int32_t)i;
  std::stable_sort(row_order.begin(), row_order.end(), [&](int32_t a, int32_t b) { return row_cost[a] > row_cost[b]; });

  // Launches of 256 threads a tile, row item (512 with 256 rows) and block, and eight workgroups a merged tile.
  const size_t most = (size_t)lazy::kMaxGroups - 64;
  if ((out_tiles.size() + 2 * rows.size()) * (size_t)hkv > most || out_segs.size() > INT32_MAX ||
      blocks.size() + 8 * merges.size() * (size_t)hkv > most)
    return LAZY_EUNSUPPORTED;
  *info = {};
  info->batch = batch;
  info->total_q = (int32_t)total_q;
  info->num_q_heads = p->num_q_heads;
  info->num_kv_heads = hkv;
  info->head_dim = d;
  info->causal = p->causal;
  info->key_positions = p->key_positions;
  info->num_tiles = (int32_t)out_tiles.size();
  info->num_segments = (int32_t)out_segs.size();
  info->num_merges = (int32_t)merges.size();
  info->num_parts = num_parts;
  info->num_row_items = (int32_t)rows.size();
  info->num_blocks = (int32_t)blocks.size();
  info->row_slots = row_slots;
  info->row_blocks = row_blocks;
  const lazy::GradPlanLayout at(*info);
  info->plan_bytes = (int64_t)at.bytes;
  if (capacity < at.bytes || (at.bytes > 0 && !plan)) return LAZY_EINVAL;
  char* base = static_cast<char*>(plan);
  const auto put = [](char* to, const void* from, size_t bytes) {
    if (bytes) memcpy(to, from, bytes);
  };
  put(base + at.blocks, blocks.data(), sizeof(GradBlock) * blocks.size());
  put(base + at.segs, out_segs.data(), sizeof(GradSeg) * out_segs.size());
  put(base + at.merges, merges.data(), sizeof(GradMerge) * merges.size());
  for (size_t i = 0; i < order.size(); ++i)
    memcpy(base + at.tiles + sizeof(GradTile) * i, &out_tiles[order[i]], sizeof(GradTile));
  for (size_t i = 0; i < row_order.size(); ++i)
    memcpy(base + at.rows + sizeof(GradRowItem) * i, &rows[row_order[i]], sizeof(GradRowItem));
  return LAZY_OK;
}

}  // namespace

extern "C" int lazy_attn_backward_plan(const lazy_attn_params_t* params, const int32_t* q_start, const int32_t* q_pos0,
                                       const lazy_chunk_t* chunks, const int32_t* chunk_start, int32_t batch,
                                       void* plan, size_t plan_capacity, lazy_backward_info_t* info) {
  const int e = lazy::check_params(params);
  if (e != LAZY_OK) return e;
  if (batch < 0 || !q_start || !chunk_start || !info || (batch > 0 && !q_pos0)) return LAZY_EINVAL;
  if (chunk_start[batch] > 0 && !chunks) return LAZY_EINVAL;
  try {
    return make_plan(params, q_start, q_pos0, chunks, chunk_start, batch, plan, plan_capacity, info);
  } catch (...) {  // out of memory
    return LAZY_EINVAL;
  }
}

extern "C" size_t lazy_attn_backward_workspace_size(const lazy_attn_params_t* params,
                                                    const lazy_backward_info_t* info) {
  if (lazy::check_params(params) != LAZY_OK || !info) return 0;
  return lazy::GradWorkLayout(params->num_q_heads, params->num_kv_heads, params->head_dim, lazy::query_parts(params), *info).bytes;
}
