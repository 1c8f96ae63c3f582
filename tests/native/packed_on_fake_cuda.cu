// The packed cache's host code on top of fake_cuda.cpp: no kernel ever runs; and the index arithmetic that kernels and merges share.
#include "../../paper_2607_20125_b200/csrc/packed_api.cu"

#include <string>
#include <vector>

static std::string launches;
extern "C" const void* fake_saw_launch(const char* name, void** args) {
  launches += std::string(name) + " ";
  return nullptr;
}
extern "C" const char* fake_launches() { return launches.c_str(); }
extern "C" void fake_clear_launches() { launches.clear(); }

// Walks the items of every CTA as the kernels' roles do.  Counts what each step of the line gets (1: once), and returns a negative
// number where an item lies outside its head, a slot is used twice, or the merge of a cut item would not find its parts.
extern "C" int fake_walk_attention(const int32_t* lens, int n_kv, int n_rows, int n_sm, int32_t* covered, int64_t capacity) {
  PackedAttnParams p;
  std::memset(&p, 0, sizeof(p));
  p.c.n_kv = n_kv;
  p.n_rows = n_rows;
  p.n_pairs = (n_rows + 255) / 256;
  int64_t total = 0;
  for (int h = 0; h <= PACK_MAX_HEADS; ++h) {
    p.line_first[h] = total;
    if (h < n_kv) total += static_cast<int64_t>(p.len.n[h] = lens[h], (lens[h] + PACK_TILE - 1) / PACK_TILE) * p.n_pairs;
  }
  if (total == 0) return 0;
  if (total > capacity) return -1;
  p.n_cta = static_cast<int32_t>(std::min<int64_t>(n_sm, total));
  std::vector<int64_t> slot_pair(2 * p.n_cta, -1);  // the pair, counted over all heads, whose part is in the slot
  for (int b = 0; b < p.n_cta; ++b) {
    int64_t x = share_begin(b, total, p.n_cta);
    const int64_t hi = share_begin(b + 1, total, p.n_cta);
    int head = 0;
    while (x < hi) {
      const int64_t at = x;
      const PackedItem w = packed_item(p, b, x, hi, head);
      if (w.tile_begin < 0 || w.tile_end <= w.tile_begin || w.tile_end > w.tiles || w.pair >= p.n_pairs || w.tile_begin * PACK_TILE >= lens[w.head]) return -2;
      if (at != p.line_first[w.head] + static_cast<int64_t>(w.pair) * w.tiles + w.tile_begin) return -3;
      for (int64_t i = at; i < x; ++i) ++covered[i];
      if (w.slot >= 0) {
        if (w.slot >= 2 * p.n_cta || slot_pair[w.slot] != -1) return -4;
        slot_pair[w.slot] = static_cast<int64_t>(w.head) * p.n_pairs + w.pair;
      } else if (w.tile_begin != 0 || w.tile_end != w.tiles) {
        return -5;
      }
    }
  }
  for (int h = 0; h < n_kv; ++h) {
    const int tiles = (lens[h] + PACK_TILE - 1) / PACK_TILE;
    for (int pair = 0; pair < p.n_pairs && tiles; ++pair) {
      const int64_t first = p.line_first[h] + static_cast<int64_t>(pair) * tiles, id = static_cast<int64_t>(h) * p.n_pairs + pair;
      const int b0 = share_owner(first, total, p.n_cta), n = share_owner(first + tiles - 1, total, p.n_cta) - b0 + 1;
      if (share_begin(b0, total, p.n_cta) > first || share_begin(b0 + 1, total, p.n_cta) <= first) return -6;
      int found = 0;
      for (int64_t s : slot_pair) found += s == id;
      if (found != (n > 1 ? n : 0)) return -7;
      for (int i = 0; n > 1 && i < n; ++i)
        if (slot_pair[i == 0 ? 2 * b0 + 1 : 2 * (b0 + i)] != id) return -8;
    }
  }
  return p.n_cta;
}

extern "C" int fake_walk_observe(const int32_t* lens, int n_kv, int group, int q_tiles, int n_sm, int32_t* covered, int64_t capacity) {
  PackedObserveParams p;
  std::memset(&p, 0, sizeof(p));
  p.c.n_kv = n_kv;
  p.group = group;
  p.q_tiles = q_tiles;
  int64_t total = 0;
  for (int h = 0; h <= PACK_MAX_HEADS; ++h) {
    p.line_first[h] = total;
    if (h < n_kv) total += static_cast<int64_t>((p.len.n[h] = lens[h], (lens[h] + 255) / 256)) * group * q_tiles;
  }
  if (total == 0) return 0;
  if (total > capacity) return -1;
  p.n_cta = static_cast<int32_t>(std::min<int64_t>(n_sm, total));
  std::vector<int> used(2 * p.n_cta, 0);
  for (int b = 0; b < p.n_cta; ++b) {
    int64_t x = share_begin(b, total, p.n_cta);
    const int64_t hi = share_begin(b + 1, total, p.n_cta);
    int head = 0;
    while (x < hi) {
      const int64_t at = x;
      const ObserveItem w = observe_item(p, b, x, hi, head);
      if (w.begin < 0 || w.end <= w.begin || w.end > group * q_tiles || w.pair * 256 >= lens[w.head]) return -2;
      for (int64_t i = at; i < x; ++i) ++covered[i];
      const int64_t first = at - w.begin;
      const int b0 = share_owner(first, total, p.n_cta), b1 = share_owner(first + group * q_tiles - 1, total, p.n_cta);
      if ((w.slot < 0) != (b0 == b1)) return -3;
      if (w.slot >= 0 && (used[w.slot]++ || w.slot != (b == b0 ? 2 * b + 1 : 2 * b))) return -4;
    }
  }
  return p.n_cta;
}

// The few-row kernel: a part's slot is CTA + head, of which no two may agree, and the merge reads the owners of a head's first to last tile.
extern "C" int fake_walk_rows(const int32_t* lens, int n_kv, int n_sm) {
  int32_t first[PACK_MAX_HEADS + 1];
  int total = 0;
  for (int h = 0; h <= PACK_MAX_HEADS; ++h) {
    first[h] = total;
    if (h < n_kv) total += (lens[h] + PACK_TILE - 1) / PACK_TILE;
  }
  if (total == 0) return 0;
  const int n_cta = std::min(n_sm, total);
  std::vector<int> slot_head(n_sm + n_kv, -1), slot_cta(n_sm + n_kv, -1);
  for (int b = 0; b < n_cta; ++b)
    for (int h = 0; h < n_kv; ++h) {
      const int64_t lo = std::max<int64_t>(share_begin(b, total, n_cta), first[h]), hi = std::min<int64_t>(share_begin(b + 1, total, n_cta), first[h + 1]);
      if (lo >= hi) continue;
      if (slot_head[b + h] != -1) return -2;
      slot_head[b + h] = h;
      slot_cta[b + h] = b;
    }
  for (int h = 0; h < n_kv; ++h) {
    if (first[h + 1] == first[h]) continue;
    const int b0 = share_owner(first[h], total, n_cta), b1 = share_owner(first[h + 1] - 1, total, n_cta);
    int parts = 0;
    for (size_t s = 0; s < slot_head.size(); ++s) parts += slot_head[s] == h;
    if (parts != b1 - b0 + 1) return -3;
    for (int b = b0; b <= b1; ++b)
      if (slot_head[b + h] != h || slot_cta[b + h] != b) return -4;
  }
  return n_cta;
}
