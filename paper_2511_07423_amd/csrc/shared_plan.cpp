// Host side of the batches that share pages: validation, the search for shared prefixes, and the cut of the attention's
// work into items.  No HIP call, no arithmetic of the method.
#include <algorithm>
#include <cstring>
#include <map>
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
// Ranges that one launch may be cut into beyond one for each node, tile of rows and KV head: enough for every rule of sh_plan.
static int64_t most_cuts(const ShLimits& l) { return 4 * (int64_t)l.slots; }
#define SH_MIN_BLOCK 256         // keys that a block's range has at least: the rings are barely filled below
#define SH_MIN_WAVE 128          // a wavefront's: one request of 900 tokens 14 us, with at least 256 18 us
#define SH_WAVES_MOST 4          // ranges that a node is cut into for wavefronts alone
#define SH_KEYS_A_ROW 16         // keys a range has for each row whose partial result it leaves
#define SH_JOIN_BYTES 16e6
#define SH_UNCUT_KEYS 512        // up to here no range is worth the launch that joins the parts: 8 requests of 300 tokens 12.5 -> 10.2 us
#define SH_KEYS_AN_ITEM 100      // what it takes to begin an item of many rows, in keys
#define SH_KEYS_A_CUT 400        // that, and its partial results

void sh_limits(ShLimits& l) {
  const int64_t G = l.Hq / l.Hkv, rows = (int64_t)l.max_tokens * G;        // per KV head
  l.windows = 2 * (int64_t)l.max_batch + pages_for(l.max_tokens);         // n tokens touch at most n / 16 + 2 pages
  // rows that shared nodes may hold beyond each request's own: what their partials are kept for
  l.shared_rows = std::min<int64_t>(2 * rows, ((int64_t)1 << 18) / l.Hkv);
  l.list = l.shared_rows / G;
  l.pages = (int64_t)l.max_batch * l.max_pages;
  // Partial results: of shared nodes and of the rows behind them, and twice those of the ranges that nodes are cut into (the first range of
  // a node that is cut needs them too).
  l.items = (2 * (int64_t)l.max_batch + (rows + l.shared_rows) / SY_SH_TILE_ROWS + 2) * l.Hkv + most_cuts(l) + 5 * SY_SH_DEAL;
  l.part_rows = (l.shared_rows + std::min<int64_t>(rows, l.shared_rows)) * l.Hkv + 2 * most_cuts(l) * SY_SH_TILE_ROWS;
  l.parts = l.part_rows / l.Hkv;
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
// cores more.  0.45 of a fetch for each tile is fitted, not derived: launches of nothing but full tiles reach 1.03 PFLOP/s, where it would be 0.62
// (65536 operations against 512 bytes at 4.99 TB/s); what a tile costs beside fetches has not been measured by itself.
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
  std::vector<int32_t> req_tok(B);               // flattened index of each request's first new token
  int32_t T = 0;
  std::vector<int32_t> all;
  for (int i = 0; i < B; ++i) {
    req_tok[i] = T;
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
    // One pass for all leaves a partial of each row (4 hd + 8 bytes: what a key and its value take), which is read again, in a
    // launch of its own: 3 us at least, or SH_JOIN_BYTES of keys and values.
    const double keys = (double)(at - s.first) * P, saved = (apart - key_cost(tokens * G)) * keys - 2.0 * (double)(tokens * G);
    const bool split = at > s.first && saved * l.Hkv * l.hd * 4 > SH_JOIN_BYTES && shared_rows + tokens * G <= l.shared_rows;
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
  const size_t N = nodes.size();
  struct Cut { int64_t keys, rows, tiles, chunk, splits; double w; bool wave; int64_t page, list, base; };
  std::vector<Cut> cut(N);
  double total = 0;
  for (size_t k = 0; k < N; ++k) {
    const Node& n = nodes[k];
    Cut& c = cut[k];
    const int i0 = n.who[0];
    c.keys = n.leaf ? (int64_t)ctx[i0] + n_new[i0] - n.first * P : (n.last - n.first) * P;
    c.rows = n.tokens * G;
    c.tiles = (c.rows + SY_SH_TILE_ROWS - 1) / SY_SH_TILE_ROWS;
    c.w = key_cost(c.rows) / (double)c.tiles;
    total += key_cost(c.rows) * (double)c.keys * l.Hkv;
  }
  // An equal share for each block that runs at once.  (Two each, so that no block's last one holds up the launch: twice the partial
  // results; 256 requests behind 8192 shared tokens 97 -> 105 us, 64 chunks of 16 behind 1000 of their own 55 -> 79.)
  const double share = total / (double)l.slots;
  // Nothing is cut where nothing is shared and no request is much longer than the share: each block takes one.  (64 requests of 32 rows
  // behind 1000 tokens 56 -> 49 us.)
  bool uncut = (int64_t)N * l.Hkv <= l.slots;
  for (size_t k = 0; k < N; ++k)
    uncut = uncut && nodes[k].leaf && cut[k].rows <= SY_SH_WAVE_ROWS && (double)cut[k].keys <= std::max((double)SH_UNCUT_KEYS, 1.15 * share);
  // Where tiles of many rows fill the chip several times over, how full the last time is counts: a few lengths are tried, the costliest
  // items handed out first.  (8 prompts of 64 heads behind 16384 tokens, 848 tiles: 3 ranges 880 us, 1 950 us.)
  double wide = 0;
  int64_t wide_tiles = 0, longest = 0;
  for (const Cut& c : cut)
    if (c.rows > SY_SH_WAVE_ROWS) {
      wide += key_cost(c.rows) * (double)c.keys * l.Hkv;
      wide_tiles += c.tiles * l.Hkv;
      longest = std::max(longest, c.keys);
    }
  int64_t wide_chunk = 0;
  if (2 * wide > total && wide_tiles >= l.slots && wide_tiles <= 8 * (int64_t)l.slots) {
    double best = 1e300;
    for (int64_t s : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 24, 32, 48, 64}) {
      const int64_t chunk = (longest + s - 1) / s;
      if (s > 1 && (chunk < SH_MIN_BLOCK || (s - 1) * wide_tiles > most_cuts(l))) break;
      std::vector<std::pair<double, int64_t>> sizes;
      for (const Cut& c : cut)
        if (c.rows > SY_SH_WAVE_ROWS) {
          const int64_t n = (c.keys + chunk - 1) / chunk;
          sizes.emplace_back(c.w * ((double)c.keys / (double)n + (n > 1 ? SH_KEYS_A_CUT : SH_KEYS_AN_ITEM)), n * c.tiles * l.Hkv);
        }
      std::sort(sizes.rbegin(), sizes.rend());
      std::map<double, int64_t> places{{0.0, l.slots}};         // when they are free, how many of them
      double end = 0;
      for (auto [size, n] : sizes)
        while (n > 0) {
          const auto first = places.begin();
          const int64_t k = std::min(n, first->second);
          const double t = first->first + size;
          if ((first->second -= k) == 0) places.erase(first);
          places[t] += k;
          end = std::max(end, t);
          n -= k;
        }
      if (end < best) {
        best = end;
        wide_chunk = chunk;
      }
    }
  }
  std::vector<int64_t> n_parts(B, 0);            // ranges of keys that are read for a request's rows
  int64_t cuts = 0;
  for (size_t k = 0; k < N; ++k) {
    Cut& c = cut[k];
    c.wave = false;
    int64_t chunk;
    if (uncut) {
      chunk = c.keys;
    } else if (c.rows <= SY_SH_WAVE_ROWS) {
      // Keys are the work.  A wavefront alone, four to a block, where that makes a few ranges; else a block's four together.
      // (64 requests of 32 rows behind 1000 tokens: 67 -> 61 us; where there is little work the rings of all units count more)
      const int64_t least = std::min<int64_t>(SH_KEYS_A_ROW * c.rows, (int64_t)(share / 2));
      const int64_t wave_chunk = std::max<int64_t>({SH_MIN_WAVE, least, (int64_t)(share / 4)});
      c.wave = c.keys <= SH_WAVES_MOST * wave_chunk;
      chunk = c.wave ? wave_chunk : std::max<int64_t>({SH_MIN_BLOCK, least, (int64_t)(2 * share)});
    } else {
      chunk = wide_chunk ? wide_chunk : std::max<int64_t>(SH_MIN_BLOCK, (int64_t)(share / c.w));
    }
    int64_t splits = (c.keys + chunk - 1) / chunk;
    // (capacity: the rules above stay within it but for shares of very many tiny nodes)
    splits = std::max<int64_t>(1, std::min(splits, 1 + (most_cuts(l) - cuts) / (c.tiles * l.Hkv)));
    c.chunk = (c.keys + splits - 1) / splits;                             // even shares
    c.chunk = (c.chunk + SY_SH_STEP - 1) / SY_SH_STEP * SY_SH_STEP;
    c.splits = (c.keys + c.chunk - 1) / c.chunk;
    cuts += (c.splits - 1) * c.tiles * l.Hkv;
    for (int i : nodes[k].who) n_parts[i] += c.splits;
  }

  // ---- page and token lists, partial results
  p.part_rows = 0;
  for (size_t k = 0; k < N; ++k) {
    const Node& n = nodes[k];
    Cut& c = cut[k];
    c.page = (int64_t)p.pages.size();
    p.pages.insert(p.pages.end(), row_of(n.who[0]) + n.first, row_of(n.who[0]) + n.last);
    c.list = (int64_t)p.list.size();
    if (!n.leaf)
      for (int i : n.who)
        for (int j = 0; j < n_new[i]; ++j) p.list.push_back(req_tok[i] + j);
    const bool direct = n.leaf && n_parts[n.who[0]] == 1;
    c.base = direct ? -1 : p.part_rows;
    if (!direct) p.part_rows += c.rows * l.Hkv * c.splits;
  }
  // the last key (exclusive) that some row of tile `t` of node k sees
  auto seen_by = [&](size_t k, int64_t t) {
    const Node& n = nodes[k];
    if (!n.leaf) return cut[k].keys;
    const int64_t last = std::min((t + 1) * SY_SH_TILE_ROWS, cut[k].rows) - 1;
    return (int64_t)ctx[n.who[0]] - n.first * P + last / G + 1;
  };
  std::vector<std::vector<std::pair<int32_t, int64_t>>> where(B);          // nodes of a request, its first row there
  for (size_t k = 0; k < N; ++k) {
    int64_t row = 0;
    for (int i : nodes[k].who) {
      if (n_parts[i] > 1) where[i].emplace_back((int32_t)k, row);
      row += n_new[i] * G;
    }
  }
  for (int i = 0; i < B; ++i) {
    if (n_parts[i] <= 1) continue;
    for (int j = 0; j < n_new[i]; ++j) {
      const int32_t first = (int32_t)p.parts.size();
      for (const auto& [k, row] : where[i]) {
        const Cut& c = cut[k];
        const int64_t r = row + j * G;           // (a token's G rows may lie in two tiles: each of them has these ranges at least)
        const int64_t keys = seen_by(k, r / SY_SH_TILE_ROWS);
        for (int64_t s = 0; s * c.chunk < keys; ++s)
          p.parts.push_back(ShPart{(int32_t)(c.base + s * l.Hkv * c.rows + r), (int32_t)c.rows});
      }
      p.joined.push_back(ShJoin{req_tok[i] + j, first, (int32_t)p.parts.size() - first, 0});
    }
  }
  p.head.n_joined = (int32_t)p.joined.size();

  // Keys and values that one item alone reads, and that no cache will hold until the next call, are read as such: 256 requests of 64 .. 1024
  // tokens (373 MB) 80 -> 72 us.  Where the last-level cache held them between the calls it costs: 16 requests (80 MB) 22.2 -> 24.2 us.
  int64_t alone = 0;
  for (size_t k = 0; k < N; ++k)
    if (nodes[k].leaf && cut[k].tiles == 1) alone += cut[k].keys * l.Hkv * l.hd * 4;
  const bool once = alone > ((int64_t)96 << 20);

  // ---- items.  Ranges of keys, the costliest first, go to the least loaded of eight queues, with all the tiles of rows that read
  // them: blocks are dealt to the eight XCDs in turn, so these meet in one L2.
  struct Range { double cost; int32_t node, head; int64_t split; };
  std::vector<Range> ranges, waves;
  for (size_t k = 0; k < N; ++k) {
    const Cut& c = cut[k];
    for (int h = 0; h < l.Hkv; ++h)
      for (int64_t s = 0; s < c.splits; ++s)
        (c.wave ? waves : ranges).push_back(Range{key_cost(c.rows) * (double)std::min(c.chunk, c.keys - s * c.chunk), (int32_t)k, h, s});
  }
  auto by_cost = [](const Range& a, const Range& b) { return a.cost > b.cost; };
  std::stable_sort(ranges.begin(), ranges.end(), by_cost);
  std::stable_sort(waves.begin(), waves.end(), by_cost);
  auto put = [&](const Range& r, int64_t t, std::vector<ShItem>& to) {
    const Node& n = nodes[r.node];
    const Cut& c = cut[r.node];
    const int i0 = n.who[0];
    ShItem it = {};
    it.flags = (n.leaf ? SY_SH_LEAF : 0) | (n.leaf && c.tiles == 1 && once ? SY_SH_ONCE : 0);
    it.kv_head = r.head;
    it.row0 = (int32_t)(t * SY_SH_TILE_ROWS);
    it.n_rows = (int32_t)std::min<int64_t>(SY_SH_TILE_ROWS, c.rows - it.row0);
    it.tok = n.leaf ? req_tok[i0] : (int32_t)c.list;
    it.page = (int32_t)c.page;
    it.n_pages = (int32_t)(n.last - n.first);
    it.key_begin = (int32_t)(r.split * c.chunk);
    const int64_t seen = seen_by(r.node, t);
    if (it.key_begin >= seen) return;
    it.key_end = (int32_t)std::min(seen, (r.split + 1) * c.chunk);
    it.lim0 = n.leaf ? (int32_t)(ctx[i0] - n.first * P) : -1;
    it.part = c.base < 0 ? -1 : (int32_t)(c.base + (r.split * l.Hkv + r.head) * c.rows + it.row0);
    for (int q = 0; q < 16; ++q) it.pages[q] = p.pages[c.page + std::min<int64_t>(it.key_begin / P + q, it.n_pages - 1)];
    to.push_back(it);
  };
  const int X = SY_SH_DEAL;
  std::vector<ShItem> queue[X];
  double load[X] = {};
  for (const Range& r : ranges) {
    const int x = (int)(std::min_element(load, load + X) - load);
    load[x] += r.cost;
    for (int64_t t = 0; t < cut[r.node].tiles; ++t) put(r, t, queue[x]);
  }
  size_t next[X] = {}, left = 0;
  for (const auto& q : queue) left += q.size();
  while (left) {
    for (int x = 0; x < X; ++x) {
      int y = x;
      if (next[x] == queue[x].size())            // this queue is done: from the longest one, so that the others keep their turn
        for (int z = 0; z < X; ++z)
          if (queue[z].size() - next[z] > queue[y].size() - next[y]) y = z;
      if (next[y] < queue[y].size()) {
        p.items.push_back(queue[y][next[y]++]);
        --left;
      } else {
        p.items.push_back(ShItem{});
      }
    }
  }
  p.head.block_groups = (int32_t)(p.items.size() / X);
  const size_t begin = p.items.size();
  for (const Range& r : waves) put(r, 0, p.items);
  while ((p.items.size() - begin) % (4 * X)) p.items.push_back(ShItem{});
  p.head.wave_groups = (int32_t)((p.items.size() - begin) / (4 * X));
}
