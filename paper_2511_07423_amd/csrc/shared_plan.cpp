// Host side of the batches that share pages: validation, the search for shared prefixes, and the cut of the attention's
// work into items.  No HIP call, no arithmetic of the method.
#include <algorithm>
#include <cstring>
#include <new>

#include "shared.h"

static int64_t pages_for(int64_t positions) { return (positions + SYNERA_PAGE_SIZE - 1) / SYNERA_PAGE_SIZE; }

// ------------------------------------------------------------------------------------ validation
// A page may be named again only in the same column behind the same page, and only where both requests hold it whole: then
// by induction over the columns both rows begin alike, and nothing is written to it.
static int32_t validate(int32_t B, const int32_t* ctx, const int32_t* n_new, const int32_t* table, int32_t max_pages,
                        int32_t n_pages, int32_t max_batch, int64_t max_tokens) {
  if (!ctx || !n_new || !table) return SYNERA_EINVAL;
  if (B < 1 || max_pages < 1 || n_pages < 1) return SYNERA_EINVAL;
  if (n_pages >= 1 << 27) return SYNERA_EUNSUP;
  if (B > max_batch) return SYNERA_ENOSPC;
  int64_t total = 0;
  for (int i = 0; i < B; ++i) {
    if (n_new[i] < 0) return SYNERA_EINVAL;
    if (ctx[i] < 0 || (int64_t)ctx[i] + n_new[i] > INT32_MAX - SY_SH_STEP) return SYNERA_ERANGE;   // positions are int32
    total += n_new[i];
    if (pages_for((int64_t)ctx[i] + n_new[i]) > max_pages) return SYNERA_ENOSPC;
  }
  if (total > max_tokens) return SYNERA_ENOSPC;
  struct Owner { int32_t request, column; };
  std::vector<Owner> owner((size_t)n_pages, Owner{-1, 0});
  for (int i = 0; i < B; ++i) {
    const int32_t* row = table + (size_t)i * max_pages;
    const int64_t need = pages_for((int64_t)ctx[i] + n_new[i]);
    int64_t c = 0;
    if (i > 0) {                                   // what the row above begins with too has been looked at
      const int32_t* above = row - max_pages;
      const int64_t same = std::min(ctx[i], ctx[i - 1]) / SYNERA_PAGE_SIZE;
      while (c < same && row[c] == above[c]) ++c;
    }
    for (; c < need; ++c) {
      const int32_t id = row[c];
      if (id < 0 || id >= n_pages) return SYNERA_ERANGE;
      Owner& o = owner[id];
      if (o.request < 0) {
        o = Owner{i, (int32_t)c};
        continue;
      }
      const int32_t* other = table + (size_t)o.request * max_pages;
      if (o.column != c || c >= ctx[i] / SYNERA_PAGE_SIZE || c >= ctx[o.request] / SYNERA_PAGE_SIZE) return SYNERA_ERANGE;
      if (c > 0 && other[c - 1] != row[c - 1]) return SYNERA_ERANGE;
    }
  }
  return SYNERA_OK;
}

extern "C" int32_t synera_validate_shared(int32_t B, const int32_t* h_ctx_len, const int32_t* h_n_new,
                                          const int32_t* h_block_table, int32_t max_pages, int32_t n_pages_in_pool,
                                          int32_t max_batch, int64_t max_tokens) {
  try {
    return validate(B, h_ctx_len, h_n_new, h_block_table, max_pages, n_pages_in_pool, max_batch, max_tokens);
  } catch (const std::bad_alloc&) {
    return SYNERA_ENOMEM;
  }
}

// ------------------------------------------------------------------------------------ capacities
// Blocks to cut the work for: a few times what runs at once, so that no block's last item holds up the launch.
static int64_t item_target(const ShLimits& l) { return 2 * (int64_t)l.slots; }

void sh_limits(ShLimits& l) {
  const int64_t G = l.Hq / l.Hkv, rows = (int64_t)l.max_tokens * G;        // per KV head
  l.windows = 2 * (int64_t)l.max_batch + pages_for(l.max_tokens);         // n tokens touch at most n / 16 + 2 pages
  // rows that shared nodes may hold beyond each request's own: what their partials are kept for
  l.shared_rows = std::min<int64_t>(2 * rows, ((int64_t)1 << 18) / l.Hkv);
  l.list = l.shared_rows / G;
  l.entries = l.max_batch + l.list;
  l.pages = (int64_t)l.max_batch * l.max_pages;
  // A node is cut into at most keys x cost / share + 1 ranges (shares are rounded down to whole keys, by less than 1/256): so
  // many items and, twice (the first range of a node that is cut needs partials too), their rows.
  const int64_t extra = item_target(l) + item_target(l) / 64 + 64;
  l.items = (2 * (int64_t)l.max_batch + (rows + l.shared_rows) / SY_SH_TILE_ROWS + 2) * l.Hkv + extra;
  l.part_rows = (l.shared_rows + std::min<int64_t>(rows, l.shared_rows)) * l.Hkv + 2 * extra * SY_SH_TILE_ROWS;
}

// ------------------------------------------------------------------------------------ shared prefixes
namespace {

struct Node {                       // pages [first, last) of the rows of `who`
  std::vector<int32_t> who;
  int64_t first, last;
  int64_t tokens;
  bool leaf;
};

// What a key costs `rows` query rows of one KV head, in keys fetched: fetching bounds up to two tiles of rows, the matrix
// cores more (0.45 of a fetch for each tile).
double key_cost(int64_t rows) {
  const int64_t tiles = (rows + SY_SH_TILE_ROWS - 1) / SY_SH_TILE_ROWS;
  return std::max(1.0, 0.45 * (double)tiles);
}

}  // namespace

void sh_plan(const ShLimits& l, int32_t B, const int32_t* ctx, const int32_t* n_new, const int32_t* table, int32_t max_pages,
             ShPlan& p) {
  const int P = SYNERA_PAGE_SIZE;
  const int64_t G = l.Hq / l.Hkv;
  auto row_of = [&](int i) { return table + (size_t)i * max_pages; };
  p = ShPlan();
  p.head = ShHeader{};
  // ---- the new tokens: positions, slots, and the pages they fall on
  p.req_tok.resize(B);
  int32_t T = 0;
  std::vector<int32_t> all;
  for (int i = 0; i < B; ++i) {
    p.req_tok[i] = T;
    const int32_t* row = row_of(i);
    for (int j = 0; j < n_new[i]; ++j) {
      const int64_t pos = (int64_t)ctx[i] + j;
      const int slot = (int)(pos % P);
      p.tok_pos.push_back((int32_t)pos);
      p.tok_slot.push_back(row[pos / P] * P + slot);
      if (j == 0 || slot == 0) p.windows.push_back(ShWindow{row[pos / P], T + j, slot, slot});
      p.windows.back().s1 = slot + 1;
    }
    T += n_new[i];
    if (n_new[i] > 0) all.push_back(i);
  }
  p.head.n_tokens = T;
  p.head.n_windows = (int32_t)p.windows.size();

  // ---- nodes.  A set of requests is followed down its common columns; where they part, the run of pages so far becomes a
  // node of its own if that is the shorter way, else every part reads those pages by itself.
  std::vector<Node> nodes;
  int64_t shared_rows = 0;
  struct Open { std::vector<int32_t> who; int64_t first, at; };
  std::vector<Open> open;
  if (!all.empty()) open.push_back(Open{std::move(all), 0, 0});
  while (!open.empty()) {
    Open s = std::move(open.back());
    open.pop_back();
    if (s.who.size() == 1) {
      const int i = s.who[0];
      nodes.push_back(Node{std::move(s.who), s.first, pages_for((int64_t)ctx[i] + n_new[i]), n_new[i], true});
      continue;
    }
    int64_t at = INT64_MAX;              // first column in which not all rows name one page
    for (size_t n = 1; n < s.who.size(); ++n) {
      const int a = s.who[n - 1], b = s.who[n];
      const int64_t most = std::min(std::min(ctx[a], ctx[b]) / P, (int32_t)std::min<int64_t>(at, INT32_MAX));
      int64_t c = s.at;
      while (c < most && row_of(a)[c] == row_of(b)[c]) ++c;
      at = std::min(at, c);
    }
    // parts: requests that name one page in column `at`; one whose cached pages end there stands alone
    std::vector<std::pair<int64_t, int32_t>> key;
    int64_t tokens = 0;
    for (int i : s.who) {
      const bool whole = at < ctx[i] / P;
      key.emplace_back(whole ? (int64_t)row_of(i)[at] : ((int64_t)1 << 32) + i, i);
      tokens += n_new[i];
    }
    std::sort(key.begin(), key.end());
    std::vector<Open> parts;
    double apart = 0;                    // cost of a key if every part reads it by itself
    for (size_t a = 0; a < key.size();) {
      Open part{{}, s.first, at};
      int64_t t = 0;
      for (const int64_t k = key[a].first; a < key.size() && key[a].first == k; ++a) {
        part.who.push_back(key[a].second);
        t += n_new[key[a].second];
      }
      apart += key_cost(t * G);
      parts.push_back(std::move(part));
    }
    // One pass for all leaves a partial of each row (4 hd + 8 bytes: what a key and its value take), which is read again.
    const double keys = (double)(at - s.first) * P;
    const bool split = at > s.first && (apart - key_cost(tokens * G)) * keys > 2.0 * (double)(tokens * G) + 128.0 &&
                       shared_rows + tokens * G <= l.shared_rows;
    for (Open& part : parts) {
      if (split) part.first = at;
      open.push_back(std::move(part));
    }
    if (split) {
      shared_rows += tokens * G;
      nodes.push_back(Node{std::move(s.who), s.first, at, tokens, false});
    }
  }

  // ---- how the keys are cut: equal shares of the modelled cost
  double total = 0;
  for (const Node& n : nodes) {
    const int64_t tiles = (n.tokens * G + SY_SH_TILE_ROWS - 1) / SY_SH_TILE_ROWS;
    const double w = key_cost(n.tokens * G) / (double)tiles;
    total += w * (double)tiles * (double)((n.last - n.first) * P) * l.Hkv;
  }
  const double share = total / (double)item_target(l);

  // ---- items
  struct Draft { int32_t node; int64_t chunk, base; };
  std::vector<Draft> draft(nodes.size());
  std::vector<int32_t> n_parts(B, 0);            // nodes x splits that read keys for a request's rows
  std::vector<std::vector<int32_t>> of(B);       // nodes of each request
  for (size_t k = 0; k < nodes.size(); ++k) {
    const Node& n = nodes[k];
    const int i0 = n.who[0];
    const int64_t keys = n.leaf ? (int64_t)ctx[i0] + n_new[i0] - n.first * P : (n.last - n.first) * P;
    const int64_t rows = n.tokens * G, tiles = (rows + SY_SH_TILE_ROWS - 1) / SY_SH_TILE_ROWS;
    const double w = key_cost(rows) / (double)tiles;
    int64_t chunk = (int64_t)(share / w);
    chunk = std::max<int64_t>(chunk, 256);
    int64_t splits = (keys + chunk - 1) / chunk;
    chunk = (keys + splits - 1) / splits;                                   // even shares
    chunk = (chunk + SY_SH_STEP - 1) / SY_SH_STEP * SY_SH_STEP;
    splits = (keys + chunk - 1) / chunk;
    draft[k] = Draft{(int32_t)k, chunk, 0};
    for (int i : n.who) {
      n_parts[i] += (int32_t)splits;
      of[i].push_back((int32_t)k);
    }
  }
  std::vector<int64_t> page_at(nodes.size()), list_at(nodes.size());
  std::vector<std::vector<int32_t>> row_at(nodes.size());                   // first row of each request of a shared node
  int64_t part_rows = 0;
  for (size_t k = 0; k < nodes.size(); ++k) {
    const Node& n = nodes[k];
    const int i0 = n.who[0];
    page_at[k] = (int64_t)p.pages.size();
    p.pages.insert(p.pages.end(), row_of(i0) + n.first, row_of(i0) + n.last);
    list_at[k] = (int64_t)p.list.size();
    int64_t rows = 0;
    for (int i : n.who) {
      row_at[k].push_back((int32_t)rows);
      rows += n_new[i] * G;
      if (!n.leaf)
        for (int j = 0; j < n_new[i]; ++j) p.list.push_back(p.req_tok[i] + j);
    }
    const bool direct = n.leaf && n_parts[i0] == 1;
    const int64_t keys = n.leaf ? (int64_t)ctx[i0] + n_new[i0] - n.first * P : (n.last - n.first) * P;
    const int64_t splits = (keys + draft[k].chunk - 1) / draft[k].chunk;
    draft[k].base = direct ? -1 : part_rows;
    if (!direct) part_rows += rows * l.Hkv * splits;
  }
  // Items that read the same keys go to one XCD (blocks are dealt to the eight in turn), next to each other in time: eight
  // queues, the least loaded takes the next range of keys.  Long items first.
  struct Range { double cost; int32_t node, head; int64_t split; };
  std::vector<Range> ranges;
  for (size_t k = 0; k < nodes.size(); ++k) {
    const Node& n = nodes[k];
    const int i0 = n.who[0];
    const int64_t keys = n.leaf ? (int64_t)ctx[i0] + n_new[i0] - n.first * P : (n.last - n.first) * P;
    const int64_t splits = (keys + draft[k].chunk - 1) / draft[k].chunk;
    for (int h = 0; h < l.Hkv; ++h)
      for (int64_t s = 0; s < splits; ++s)
        ranges.push_back(Range{key_cost(n.tokens * G) * (double)std::min(draft[k].chunk, keys - s * draft[k].chunk), (int32_t)k, h, s});
  }
  std::stable_sort(ranges.begin(), ranges.end(), [](const Range& a, const Range& b) { return a.cost > b.cost; });
  const int X = 8;
  std::vector<ShItem> queue[X];
  double load[X] = {};
  for (const Range& r : ranges) {
    int x = 0;
    for (int y = 1; y < X; ++y)
      if (load[y] < load[x]) x = y;
    load[x] += r.cost;
    const Node& n = nodes[r.node];
    const int i0 = n.who[0];
    const int64_t rows = n.tokens * G, chunk = draft[r.node].chunk;
    const int64_t keys = n.leaf ? (int64_t)ctx[i0] + n_new[i0] - n.first * P : (n.last - n.first) * P;
    const int64_t lim0 = n.leaf ? (int64_t)ctx[i0] - n.first * P : -1;
    for (int64_t r0 = 0; r0 < rows; r0 += SY_SH_TILE_ROWS) {
      ShItem it = {};
      it.flags = n.leaf ? SY_SH_LEAF : 0;
      it.kv_head = r.head;
      it.n_rows = (int32_t)std::min<int64_t>(SY_SH_TILE_ROWS, rows - r0);
      it.row0 = (int32_t)r0;
      it.tok = n.leaf ? p.req_tok[i0] : (int32_t)list_at[r.node];
      it.page = (int32_t)page_at[r.node];
      it.n_pages = (int32_t)(n.last - n.first);
      it.key_begin = (int32_t)(r.split * chunk);
      const int64_t seen = n.leaf ? lim0 + (r0 + it.n_rows - 1) / G + 1 : keys;   // keys that the tile's last row sees
      if (it.key_begin >= seen) continue;
      it.key_end = (int32_t)std::min(seen, (r.split + 1) * chunk);
      it.lim0 = (int32_t)lim0;
      it.part = draft[r.node].base < 0 ? -1 : (int32_t)(draft[r.node].base + (r.split * l.Hkv + r.head) * rows + r0);
      queue[x].push_back(it);
    }
  }
  for (size_t n = 0, left = 1; left; ++n) {
    left = 0;
    for (int x = 0; x < X; ++x)
      if (n < queue[x].size()) {
        p.items.push_back(queue[x][n]);
        left = 1;
      }
  }
  p.head.n_items = (int32_t)p.items.size();

  // ---- what is joined
  p.first_entry.resize(B + 1);
  for (int i = 0; i < B; ++i) {
    p.first_entry[i] = (int32_t)p.entries.size();
    if (n_parts[i] <= 1) continue;
    for (int32_t k : of[i]) {
      const Node& n = nodes[k];
      const size_t at = std::find(n.who.begin(), n.who.end(), i) - n.who.begin();
      const int64_t keys = n.leaf ? (int64_t)ctx[i] + n_new[i] - n.first * P : (n.last - n.first) * P;
      p.entries.push_back(ShEntry{(int32_t)(draft[k].base + row_at[k][at]), row_at[k][at], (int32_t)(n.tokens * G), (int32_t)keys,
                                  (int32_t)draft[k].chunk, n.leaf ? (int32_t)(ctx[i] - n.first * P) : -1, {0, 0}});
    }
    for (int j = 0; j < n_new[i]; ++j) {
      p.joined.push_back(p.req_tok[i] + j);
      p.joined.push_back(i);
    }
  }
  p.first_entry[B] = (int32_t)p.entries.size();
  p.head.n_joined = (int32_t)(p.joined.size() / 2);
}
