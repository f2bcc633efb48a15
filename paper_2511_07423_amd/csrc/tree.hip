// Trees of drafted tokens over a paged cache, with all lengths on the GPU: the handle behind synera_tree, the kernel that plans a step, the
// attention of the trees, and the walk and the move of an accepted path.  Appends are shared.hip's, over the plan that is made here.
#include <algorithm>
#include <cmath>
#include <new>

#include "../../include/synera.h"
#include "../../include/synera_tree.h"
#include "shared_attend.h"
#include "shared_checks.h"

#define TR_NODES SYNERA_TREE_NODES
#define TR_AHEAD 16              // columns behind a row of the table, filled with its last page: the attention's first pages are read without clamps
// Requests that a handle may have.  Every block of a plan looks at all of them, so plans get long as the square: 72 us for 1024 requests, 0.82 ms for 4096,
// 12 ms for 16384.
#define TR_BATCH (1 << 14)
#define TR_ROWS (1 << 30)        // max_tokens is below
#define TR_STEP SY_SH_STEP       // keys of one step, the unit of work

// ------------------------------------------------------------------------------------ the plan on the device
// The attention's work: a request's keys are cut into `ranges` of whole steps of TR_STEP keys, and a block takes one range of one KV head for one tile of
// rows.  Up to TR_UNIT tiles of a range follow each other on one XCD, so that its keys are fetched once and met in L2: each XCD has a list of its own,
// and such units (range, head, tiles) are dealt to the lists in turn.  A request begins where as many requests of its size before it would have ended.
// Requests come in the order of their items' cost, the longest first, since blocks take items as places become free.
// (Where the lists had their items in common but for the head, all had as many places as the fullest: 74 requests of 1344 rows at 5 heads 243 us, 184 so;
// 27 of 288 at 3 heads 295 and 228; 187 of one small tile at one head 45 and 28.)
// How long a range may be is chosen from TR_LENGTHS candidates by an estimate of the time (tr_estimate).
// (With the heads and tiles in one line that blocks took equal parts of, tiles of one head read its keys at different times:
// 32 requests of 48 .. 160 nodes 414 us, 64 of 8 .. 64 nodes 125.)
#define TR_LENGTHS 22
#define TR_UNIT 8                // and half as many where the heads alone do not fill the lists: with 8, the 74 requests at 5 heads took 220 us; with 4, 32 of 2 .. 5 tiles at 8 heads 360 for 335
#define TR_GRID 4                // blocks of the launch for each place
#define TR_JOIN_GRID 2           // of the joining one
// Candidate c: 2, 3, 4, 6, 8, 12, .. 1536, 2048 steps, and any.
__device__ __forceinline__ int32_t tr_ranges(int32_t steps, int c) {
  const int32_t x = (steps - 1) >> (c / 2);
  return steps == 0 ? 0 : c == TR_LENGTHS - 1 ? 1 : (c & 1 ? x / 3 : x / 2) + 1;
}
// In 16ths of what a step takes a block of 64 rows at most when all places are taken and HBM is the bound (64 KB for each with heads of 128: 5.1 us).
#define TR_ONE 16                // a step of a request's only tile
#define TR_FULL 22               // if it has more than 64 rows
#define TR_MORE 15               // of one of several, which share what is fetched: the matrix cores' and the softmax's time
#define TR_ALONE 4               // the same, where a block has a compute unit of its own, for up to 64 rows
#define TR_ALONE_FULL 10         // and more
#define TR_PAIR 5                // and where two share one
#define TR_PAIR_FULL 14
#define TR_START 16              // what it takes to begin and end an item
#define TR_JOIN_LAUNCH 10        // to join anything at all
#define TR_JOIN_ROWS 1024        // partial rows written and read in one 16th
#define TR_JOIN_RANGES 4         // ranges of a row, one after the other
struct TrHead {
  ShHeader sh;                   // tokens and windows, for the append
  int32_t B;
  int32_t joins;                 // places of the joining launch
  int32_t pad[6];
  int32_t items[SY_SH_DEAL];     // in each list
};
struct TrReq {                   // 32 bytes, scalar loads
  int32_t ctx, n, tok;           // n: 0 where the request has no nodes or is refused
  int32_t rows;                  // of those that are counted, the ones that there is room for
  int32_t steps, ranges, tiles;  // as the lists count them, refused or not
  int32_t part;                  // first of its partial rows, if it has several ranges: [range][head][row]
};
static_assert(sizeof(TrReq) == 4 * SH_FIRST_PITCH, "how the append finds a request's first row");
struct TrItem {                  // 64 bytes, the k-th of list x at 8 k + x.  All that a block has to know before it can ask for keys, in one load
  TrReq q;
  int32_t req, tile;             // (a tile that the request has not: none)
  int32_t group;                 // range x heads + head
  int32_t pad[5];
};
struct TrJoin {                  // 8 bytes: TR_JOIN_AT rows of a request (of all KV heads) from row `at` on
  int32_t req, at;
};
#define TR_JOIN_AT 8

struct synera_tree {
  ShLimits lim;                  // (head counts and sizes; no room of a host plan)
  int device;
  bool planned;
  bool replays;                  // a plan was captured: the one on the device may be another than the last one that was called
  int32_t B, n_pages, columns;
  int64_t n_rows;
  int32_t pitch;                 // columns of the table's copy
  char* dev;
  int32_t items_room, part_rows;
  TrHead* head;
  TrReq* req;
  TrItem* items;
  TrJoin* joins;
  ShWindow* windows;
  int32_t *pos, *slot, *parent, *table;
  uint32_t* masks;
  float* part_o;
  float2* part_ml;
};

// Units of a range of a head, all of the same number of tiles (the last may have fewer); items of `ranges` of them in the longest list.
__host__ __device__ __forceinline__ int32_t units_of(int32_t Hkv, int32_t tiles) {
  return Hkv % SY_SH_DEAL ? (tiles + TR_UNIT / 2 - 1) / (TR_UNIT / 2) : (tiles + TR_UNIT - 1) / TR_UNIT;
}
__host__ __device__ __forceinline__ uint64_t places_of(int32_t Hkv, int32_t units, int32_t per, int32_t ranges) {
  return ((uint64_t)(uint32_t)(Hkv * units) * (uint32_t)ranges + SY_SH_DEAL - 1) / SY_SH_DEAL * (uint32_t)per;
}

static size_t up(size_t v) { return (v + 255) / 256 * 256; }

extern "C" int32_t synera_tree_destroy(synera_tree* t) {
  if (!t) return SYNERA_OK;
  const BesideCaptures beside;
  if (t->dev) (void)hipFree(t->dev);
  delete t;
  return SYNERA_OK;
}

static hipError_t prepare_attention(int hd);

extern "C" int32_t synera_tree_create(synera_tree** out, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_batch,
                                      int32_t max_tokens, int32_t max_pages) {
  if (!out) return SYNERA_EINVAL;
  *out = nullptr;
  if (n_q_heads < 1 || n_kv_heads < 1 || max_batch < 1 || max_tokens < 1 || max_pages < 1) return SYNERA_EINVAL;
  if ((head_dim != 64 && head_dim != 128) || n_q_heads % n_kv_heads || n_q_heads > 1024) return SYNERA_EUNSUP;
  if ((int64_t)max_tokens * n_q_heads >= (int64_t)1 << 30 || (int64_t)max_batch * ((int64_t)max_pages + TR_AHEAD) >= (int64_t)1 << 30) return SYNERA_EUNSUP;
  if ((int64_t)max_batch * n_q_heads >= (int64_t)1 << 26 || max_batch > TR_BATCH) return SYNERA_EUNSUP;
  int dev = 0;
  hipDeviceProp_t prop;
  if (hipGetDevice(&dev) != hipSuccess || hipGetDeviceProperties(&prop, dev) != hipSuccess || prepare_attention(head_dim) != hipSuccess) {
    (void)hipGetLastError();
    return SYNERA_EHIP;
  }
  synera_tree* t = new (std::nothrow) synera_tree();
  if (!t) return SYNERA_ENOMEM;
  t->device = dev;
  t->lim.Hq = n_q_heads;
  t->lim.Hkv = n_kv_heads;
  t->lim.hd = head_dim;
  t->lim.max_batch = max_batch;
  t->lim.max_tokens = max_tokens;
  t->lim.max_pages = max_pages;
  t->lim.slots = 2 * std::max(1, prop.multiProcessorCount);
  t->pitch = max_pages + TR_AHEAD;
  // uncut, a request has an item in each list for every tile and eighth head, also one whose rows there is no room for
  const size_t B = (size_t)max_batch, T = (size_t)max_tokens, G = (size_t)(n_q_heads / n_kv_heads);
  size_t places = 0;
  for (int32_t tiles = 1; tiles <= (int32_t)(TR_NODES * G + SY_SH_TILE_ROWS - 1) / SY_SH_TILE_ROWS; ++tiles) {
    const int32_t units = units_of(n_kv_heads, tiles);
    places = std::max<size_t>(places, places_of(n_kv_heads, units, (tiles + units - 1) / units, 1));
  }
  t->items_room = (int32_t)std::max<size_t>((size_t)t->lim.slots, B * places);
  t->part_rows = 2 * t->lim.slots * SY_SH_TILE_ROWS;
  const size_t parts = (size_t)t->part_rows;
  const size_t sizes[] = {sizeof(TrHead), B * sizeof(TrReq), (size_t)t->items_room * SY_SH_DEAL * sizeof(TrItem),
                          // (at least two partial rows for each that is joined)
                          (parts / 2 / TR_JOIN_AT + B) * sizeof(TrJoin), B * (TR_NODES / SY_PAGE + 1) * sizeof(ShWindow),
                          T * 4, T * 4, T * 4, B * t->pitch * 4, T * SY_TREE_MASK * 4, parts * head_dim * 4, parts * 8};
  size_t all = 0;
  for (size_t s : sizes) all += up(s);
  if (hipMalloc(reinterpret_cast<void**>(&t->dev), all) != hipSuccess) {
    (void)hipGetLastError();
    delete t;
    return SYNERA_ENOMEM;
  }
  size_t off = 0, k = 0;
  auto take = [&](auto*& p) {
    p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(t->dev + off);
    off += up(sizes[k++]);
  };
  take(t->head);
  take(t->req);
  take(t->items);
  take(t->joins);
  take(t->windows);
  take(t->pos);
  take(t->slot);
  take(t->parent);
  take(t->table);
  take(t->masks);
  take(t->part_o);
  take(t->part_ml);
  // (no requests, rows or items until a plan has run: one that is captured has not)
  const TrHead none = {};
  if (hipMemcpy(t->head, &none, sizeof none, hipMemcpyHostToDevice) != hipSuccess) {
    (void)hipGetLastError();
    (void)synera_tree_destroy(t);
    return SYNERA_EHIP;
  }
  *out = t;
  return SYNERA_OK;
}

// ------------------------------------------------------------------------------------ planning
struct PlanArgs {
  const int32_t *ctx, *n_nodes, *parent, *table;
  const int32_t* held;           // columns of the table that are each request's own, or null: all
  int32_t* status;
  TrHead* head;
  TrReq* req;
  TrItem* items;
  TrJoin* joins;
  ShWindow* windows;
  int32_t *pos, *slot, *parents, *pages;
  uint32_t* masks;
  int32_t B, columns, pitch, n_pages, Hkv, G, items_room, part_rows;
  float per_place;               // 1 / blocks that run at once
  int32_t scale;                 // of what is not a step: 2 with heads of 64, whose steps take half as long
  int64_t n_rows;
};

// What a request's lengths alone say of it; every block forms it for all of them.  Rows are counted as synera_pages_update counts them, also of requests
// that are refused: what lies behind has the same rows for both.
struct TrSize {
  int32_t rows;                  // TR_ROWS at most, more than any call has
  int32_t windows, steps, tiles;
  int32_t units, per;            // tiles of a unit
};
__device__ __forceinline__ TrSize size_of(const PlanArgs& a, int32_t ctx, int32_t n) {
  TrSize s = {0, 0, 0, 0, 0, 1};
  if (n < 0 || n > (int64_t)SY_PAGE * a.columns) return s;
  s.rows = min(n, TR_ROWS);
  if (n > TR_NODES) return s;
  const int64_t keys = (int64_t)ctx + n;
  if (n == 0 || ctx < 0 || (keys + SY_PAGE - 1) / SY_PAGE > a.columns || keys > 0x7FFFFFFF - TR_STEP) return s;
  s.windows = (int32_t)((keys - 1) / SY_PAGE - ctx / SY_PAGE + 1);
  s.steps = (int32_t)((keys + TR_STEP - 1) / TR_STEP);
  s.tiles = (n * a.G + SY_SH_TILE_ROWS - 1) / SY_SH_TILE_ROWS;
  s.units = units_of(a.Hkv, s.tiles);
  s.per = (s.tiles + s.units - 1) / s.units;
  return s;
}
__device__ __forceinline__ int32_t tr_rows(int32_t x, int32_t y) { return (int32_t)min((uint32_t)x + (uint32_t)y, (uint32_t)TR_ROWS); }
// (A quotient in 32 bits of floating point: the same for every block, and no more than an estimate.)
__device__ __forceinline__ int32_t item_cost(const PlanArgs& a, const TrSize& s, int32_t ranges, int32_t step) {
  return (int32_t)((float)s.steps * step * __builtin_amdgcn_rcpf((float)ranges)) + TR_START * a.scale;
}
__device__ __forceinline__ int32_t item_cost(const PlanArgs& a, const TrSize& s, int32_t ranges) {
  return item_cost(a, s, ranges, s.tiles > 1 ? TR_MORE : s.rows * a.G > 64 ? TR_FULL : TR_ONE);
}
// What each candidate comes to, over all requests; whole numbers, so that every block finds the same.
struct TrTotals {
  unsigned long long cost, parts, items, places;              // items: of all lists; places: of each
  int32_t longest, shortest, alone, pair, ranges;             // an item's cost; the longest one's alone on a compute unit, the shortest one's beside another; most of a request
};
__device__ __forceinline__ int64_t tr_estimate(const PlanArgs& a, const TrTotals& t) {
  if (t.places > (unsigned long long)a.items_room || t.parts > (unsigned long long)a.part_rows) return INT64_MAX;
  // All places busy; as many rounds of the shortest items as there are; or the longest item, at first beside others.  More is left at the
  // end where items differ and there are few.
  const float rounds = (float)t.items * a.per_place;
  const int64_t busy = (int64_t)((float)t.cost * a.per_place), least = rounds > 0.5f ? (int64_t)ceilf(rounds) * t.pair : 0,
                longest = rounds > 0.5f ? max(t.longest * 5 / 8, t.alone) : t.alone;
  const int64_t end = t.longest / 32 + (int64_t)(t.alone * 0.2f * (1.f - (float)t.shortest * __builtin_amdgcn_rcpf((float)max(t.longest, 1))) *
                                                 __builtin_amdgcn_rcpf(fmaxf(2.f * rounds, 1.f)));
  return max(max(busy, least), longest) + end + (t.parts ? (TR_JOIN_LAUNCH + t.ranges / TR_JOIN_RANGES) * a.scale + (int64_t)(t.parts / TR_JOIN_ROWS) : 0);
}

// The sum over the block's threads, for all of them.
template <int N, typename Add>
__device__ __forceinline__ void block_sums(int32_t (&v)[N], int32_t (*parts)[N], Add add) {
  for (int o = 1; o < 64; o <<= 1)
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = add(v[k], __shfl_xor(v[k], o));
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int k = 0; k < N; ++k) parts[threadIdx.x >> 6][k] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = add(add(parts[0][k], parts[1][k]), add(parts[2][k], parts[3][k]));
}
template <int N>
__device__ __forceinline__ void block_sums(int32_t (&v)[N], int32_t (*parts)[N]) {
  block_sums(v, parts, [](int32_t x, int32_t y) { return x + y; });
}

// Block i plans request i.  It looks at all requests by itself (a few thousand numbers at most, which lie in the caches), so that one launch
// does.  Paths by doubling: in each round a node takes over what its forefather has gathered, and that one's forefather.
__global__ __launch_bounds__(256) void tree_plan_kernel(PlanArgs a) {
  constexpr int LANES = 256 / TR_LENGTHS;
  const int tid = threadIdx.x, me = blockIdx.x;
  __shared__ TrTotals totals[TR_LENGTHS];
  __shared__ TrSize sizes[256];
  __shared__ unsigned long long best;                         // estimate << 8 | candidate
  __shared__ int32_t sums_a[4][4], sums_b[4][3], sums_c[4][2 * SY_SH_DEAL], begin[SY_SH_DEAL];
  __shared__ int32_t up_[TR_NODES];
  __shared__ uint32_t gather[TR_NODES][9];                    // (9: neighbours on other banks)
  if (tid < TR_LENGTHS) totals[tid] = TrTotals{0, 0, 0, 0, 0, INT32_MAX, 0, INT32_MAX, 0};
  if (tid == 0) best = ~0ull;
  const int32_t ctx = a.ctx[me], n = a.n_nodes[me];
  const TrSize s = size_of(a, ctx, n);
  const bool few = a.B <= 256;                                // all sizes are in LDS
  // ---- rows and windows before this request, and of all
  int32_t rows[4] = {0, 0, 0, 0};                             // (windows are far fewer than TR_ROWS)
  for (int i = tid; i < a.B; i += 256) {
    const TrSize z = size_of(a, a.ctx[i], a.n_nodes[i]);
    if (few) sizes[i] = z;
    if (i < me) {
      rows[0] = tr_rows(rows[0], z.rows);
      rows[1] += z.windows;
    }
    rows[2] = tr_rows(rows[2], z.rows);
    rows[3] += z.windows;
  }
  block_sums(rows, sums_a, [](int32_t x, int32_t y) { return tr_rows(x, y); });
  const int64_t first = rows[0];

  // ---- what only this block looks at: parents and pages
  int32_t status = n < 0 || n > TR_NODES ? SYNERA_EINVAL : ctx < 0 ? SYNERA_ERANGE : SYNERA_OK;
  const int64_t keys = (int64_t)ctx + (status == SYNERA_OK ? n : 0);
  if (status == SYNERA_OK && (first + s.rows > a.n_rows || (n > 0 && s.steps == 0))) status = SYNERA_ENOSPC;
  if (status == SYNERA_OK && a.held) {                        // (entries behind may be pages of others by now)
    const int32_t held = a.held[me];
    if (held < 0 || held > a.columns) status = SYNERA_EINVAL;
    else if ((keys + SY_PAGE - 1) / SY_PAGE > held) status = SYNERA_ENOSPC;
  }
  const bool fits = status == SYNERA_OK && n > 0;
  bool bad_parent = false, bad_page = false;
  int32_t up = -1;
  if (fits && tid < n) up = a.parent[first + tid];
  const int32_t need = fits ? (int32_t)((keys + SY_PAGE - 1) / SY_PAGE) : 0;
  const int32_t* row = a.table + (size_t)me * a.columns;
  int32_t* copy = a.pages + (size_t)me * a.pitch;
  for (int c = tid; c < need + TR_AHEAD; c += 256) {
    if (need == 0) break;
    const int32_t id = row[min(c, need - 1)];
    bad_page |= id < 0 || id >= a.n_pages;
    copy[c] = id;
  }
  const int32_t parent = up;
  bad_parent = up < -1 || up >= tid;
  if (bad_parent) up = -1;
  bad_parent &= fits && tid < n;

  // ---- how long a range may be
  for (int i0 = 0; i0 < a.B; i0 += 256) {
    if (!few) {
      __syncthreads();
      if (i0 + tid < a.B) sizes[tid] = size_of(a, a.ctx[i0 + tid], a.n_nodes[i0 + tid]);
      __syncthreads();
    }
    const int c = tid / LANES, m = min(256, a.B - i0);
    if (c < TR_LENGTHS) {
      TrTotals t = {0, 0, 0, 0, 0, INT32_MAX, 0, INT32_MAX, 0};
      for (int i = tid % LANES; i < m; i += LANES) {
        const TrSize z = sizes[i];
        if (z.steps == 0) continue;
        const int32_t r = tr_ranges(z.steps, c), cost = item_cost(a, z, r);
        // (more items than 32 bits count are more than there is room for)
        const uint32_t items = (uint32_t)min((uint64_t)(uint32_t)(a.Hkv * z.tiles) * (uint32_t)r, (uint64_t)0xFFFFFFFFu);
        t.items += items;
        t.places += places_of(a.Hkv, z.units, z.per, r);
        t.cost += (uint64_t)items * (uint32_t)cost;
        t.longest = max(t.longest, cost);
        t.shortest = min(t.shortest, cost);
        t.ranges = max(t.ranges, r);
        t.pair = min(t.pair, item_cost(a, z, r, z.rows * a.G > 64 ? TR_PAIR_FULL : TR_PAIR));
        t.alone = max(t.alone, item_cost(a, z, r, z.rows * a.G > 64 ? TR_ALONE_FULL : TR_ALONE));
        if (r > 1) t.parts += (uint64_t)(uint32_t)r * (uint32_t)(a.Hkv * a.G * z.rows);
      }
      if (t.items) {
        atomicAdd(&totals[c].cost, t.cost);
        atomicAdd(&totals[c].parts, t.parts);
        atomicAdd(&totals[c].items, t.items);
        atomicAdd(&totals[c].places, t.places);
        atomicMax(&totals[c].longest, t.longest);
        atomicMin(&totals[c].shortest, t.shortest);
        atomicMax(&totals[c].alone, t.alone);
        atomicMax(&totals[c].ranges, t.ranges);
        atomicMin(&totals[c].pair, t.pair);
      }
    }
  }
  const int any = __syncthreads_or(bad_parent || bad_page), parent_bad = __syncthreads_or(bad_parent);
  if (any) status = parent_bad ? SYNERA_EINVAL : SYNERA_ERANGE;
  const bool live = fits && !any;
  if (tid < TR_LENGTHS) {
    const int64_t e = tr_estimate(a, totals[tid]);
    if (e < INT64_MAX) atomicMin(&best, (unsigned long long)e << 8 | (unsigned)tid);      // (the last candidate always has room)
  }
  __syncthreads();
  const int chosen = (int)(best & 255);
  // ---- partial rows before this request by number, items by cost
  const int32_t ranges = tr_ranges(s.steps, chosen), cost = s.steps ? item_cost(a, s, ranges) : 0;
  int32_t before[3] = {0, 0, 0};                              // and places of the joining launch, before this request and in all
  int32_t lists[2 * SY_SH_DEAL] = {};                         // items of each list, before this request's and in all
  for (int i = tid; i < a.B; i += 256) {
    const TrSize z = few ? sizes[i] : size_of(a, a.ctx[i], a.n_nodes[i]);
    if (z.steps == 0) continue;
    const int32_t r = tr_ranges(z.steps, chosen), k = item_cost(a, z, r);
    if (r > 1) {
      const int32_t all = a.Hkv * z.rows * a.G, joins = (all + TR_JOIN_AT - 1) / TR_JOIN_AT;
      if (i < me) {
        before[0] += r * all;
        before[1] += joins;
      }
      before[2] += joins;
    }
    const bool first = k > cost || (k == cost && i < me);
    const uint32_t units = (uint32_t)(a.Hkv * r * z.units), per = z.per, deal = (uint32_t)i * units;
#pragma unroll
    for (int x = 0; x < SY_SH_DEAL; ++x) {
      const int32_t items = (units + SY_SH_DEAL - 1 - (x - deal) % SY_SH_DEAL) / SY_SH_DEAL * per;
      lists[x] += first ? items : 0;
      lists[SY_SH_DEAL + x] += items;
    }
  }
  block_sums(before, sums_b);
  block_sums(lists, sums_c);
#pragma unroll
  for (int x = 0; x < SY_SH_DEAL; ++x)
    if (tid == x) begin[x] = lists[x];
  __syncthreads();

  // ---- paths
  uint32_t word[8];
#pragma unroll
  for (int w = 0; w < 8; ++w) word[w] = tid < n && (tid >> 5) == w ? 1u << (tid & 31) : 0u;
  if (live) {
    for (int round = 0; round < 8; ++round) {
      up_[tid] = up;
#pragma unroll
      for (int w = 0; w < 8; ++w) gather[tid][w] = word[w];
      const int more = __syncthreads_or(up >= 0);
      if (!more) break;
      if (up >= 0) {
#pragma unroll
        for (int w = 0; w < 8; ++w) word[w] |= gather[up][w];
        up = up_[up];
      }
      __syncthreads();
    }
  }
  // ---- each node's places
  if (!live) {
    for (int64_t at = first + tid; at < min(first + s.rows, a.n_rows); at += 256) {
      a.pos[at] = 0;
      a.slot[at] = -1;
    }
  } else if (tid < n) {
    const int64_t at = first + tid;
    int depth = -1;
#pragma unroll
    for (int w = 0; w < 8; ++w) depth += __popc(word[w]);
    const int32_t p = ctx + tid;
    a.pos[at] = ctx + depth;
    a.slot[at] = row[p / SY_PAGE] * SY_PAGE + p % SY_PAGE;
    a.parents[at] = parent;
    uint32_t* m = a.masks + at * SY_TREE_MASK;
    m[0] = m[1] = 0xFFFFFFFFu;
#pragma unroll
    for (int w = 0; w < 8; ++w) m[2 + w] = word[w];
#pragma unroll
    for (int w = 10; w < SY_TREE_MASK; ++w) m[w] = 0;
  }
  for (int w = tid; w < s.windows; w += 256) {
    const int32_t page = ctx / SY_PAGE + w, from = max(ctx, page * SY_PAGE), to = min(ctx + n, (page + 1) * SY_PAGE);
    ShWindow x = {0, 0, 0, 0};
    if (live) x = ShWindow{row[page], (int32_t)first + from - ctx, from - page * SY_PAGE, to - page * SY_PAGE};
    a.windows[rows[1] + w] = x;
  }
  // ---- the lists
  const TrReq q = {ctx, live ? n : 0, (int32_t)first, (int32_t)max((int64_t)0, min((int64_t)s.rows, a.n_rows - first)), s.steps, ranges, s.tiles, before[0]};
  const uint32_t each = s.units, units = a.Hkv * ranges * each, per = s.per;
  for (uint32_t e = tid; e < units * per; e += 256) {
    const uint32_t u = e / per, x = (u + (uint32_t)me * units) % SY_SH_DEAL;
    a.items[(size_t)(begin[x] + u / SY_SH_DEAL * per + e % per) * SY_SH_DEAL + x] =
        TrItem{q, me, (int32_t)(u % each * per + e % per), (int32_t)(u / each), {}};
  }
  if (ranges > 1)
    for (int k = tid; k * TR_JOIN_AT < a.Hkv * s.rows * a.G; k += 256) a.joins[before[1] + k] = TrJoin{me, k * TR_JOIN_AT};
  if (tid == 0) {
    a.req[me] = q;
    if (a.status) a.status[me] = status;
    if (me == 0) {
      a.head->sh.n_tokens = (int32_t)min((int64_t)rows[2], a.n_rows);
      a.head->sh.n_windows = rows[3];
#pragma unroll
      for (int x = 0; x < SY_SH_DEAL; ++x) a.head->items[x] = lists[SY_SH_DEAL + x];
      a.head->B = a.B;
      a.head->joins = before[2];
    }
  }
}

static Range ints(const int32_t* p, int64_t n) { return {reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + (p ? 4 * (uintptr_t)n : 0)}; }
static bool off4(std::initializer_list<const void*> all) {
  uintptr_t bits = 0;
  for (const void* p : all) bits |= reinterpret_cast<uintptr_t>(p);
  return bits % 4 != 0;
}

extern "C" int32_t synera_tree_plan_held(synera_tree* t, int32_t B, const int32_t* d_ctx_len, const int32_t* d_n_nodes, const int32_t* d_parent,
                                         int64_t n_rows, const int32_t* d_table, int32_t columns, const int32_t* d_held, int32_t n_pages_in_pool,
                                         int32_t* d_status, void* stream) {
  if (!t || !d_ctx_len || !d_n_nodes || !d_table || B < 1 || n_rows < 0 || columns < 1 || n_pages_in_pool < 1) return SYNERA_EINVAL;
  if (n_rows > 0 && !d_parent) return SYNERA_EINVAL;
  if (off4({d_ctx_len, d_n_nodes, d_parent, d_table, d_held, d_status})) return SYNERA_EINVAL;
  for (const Range& in : {ints(d_ctx_len, B), ints(d_n_nodes, B), ints(d_parent, n_rows), ints(d_table, (int64_t)B * columns), ints(d_held, B)})
    if (meet(ints(d_status, B), in)) return SYNERA_EINVAL;
  if (n_pages_in_pool >= 1 << 27) return SYNERA_EUNSUP;
  const ShLimits& l = t->lim;
  if (B > l.max_batch || n_rows > l.max_tokens || columns > l.max_pages) return SYNERA_ENOSPC;
  if (!rope_device_ok(t->device)) return SYNERA_EINVAL;
  const PlanArgs a = {d_ctx_len, d_n_nodes, d_parent, d_table, d_held, d_status, t->head, t->req, t->items, t->joins, t->windows, t->pos, t->slot, t->parent, t->table,
                      t->masks, B, columns, t->pitch, n_pages_in_pool, l.Hkv, l.Hq / l.Hkv, t->items_room, t->part_rows, 1.0f / l.slots, l.hd == 64 ? 2 : 1, n_rows};
  tree_plan_kernel<<<B, 256, 0, static_cast<hipStream_t>(stream)>>>(a);
  if (hipGetLastError() != hipSuccess) return SYNERA_EHIP;
  t->planned = true;
  t->replays = t->replays || capturing(static_cast<hipStream_t>(stream));
  t->B = B;
  t->n_rows = n_rows;
  t->n_pages = n_pages_in_pool;
  t->columns = columns;
  return SYNERA_OK;
}

extern "C" int32_t synera_tree_plan(synera_tree* t, int32_t B, const int32_t* d_ctx_len, const int32_t* d_n_nodes, const int32_t* d_parent,
                                    int64_t n_rows, const int32_t* d_table, int32_t columns, int32_t n_pages_in_pool, int32_t* d_status,
                                    void* stream) {
  return synera_tree_plan_held(t, B, d_ctx_len, d_n_nodes, d_parent, n_rows, d_table, columns, nullptr, n_pages_in_pool, d_status, stream);
}

// ------------------------------------------------------------------------------------ append
extern "C" int32_t synera_tree_append_rope(synera_tree* t, const synera_rope* rope, int32_t dtype, const synera_heads* q,
                                           const synera_heads* k, const synera_heads* v, float eps, void* d_k_layer, void* d_v_layer,
                                           void* stream) {
  if (!t || !t->planned) return SYNERA_EINVAL;
  const ShTarget target = {&t->lim, t->device, t->n_pages, t->n_rows, 0, false, t->replays, t->pos, t->slot, &t->head->sh, t->windows, &t->req->tok, &t->head->B};
  return sh_append(target, rope, dtype, q, k, v, eps, d_k_layer, d_v_layer, stream);
}

// ------------------------------------------------------------------------------------ attention
struct TreeAttnArgs : SharedAttnArgs {
  const TrHead* th;
  const TrReq* req;
  const TrItem* places;
  const TrJoin* joins;
  const uint32_t* masks;
  int32_t pitch;
  int32_t rows;                  // that the tensors of this call have: a plan that was replayed may have more
};
typedef SH_CONST_AS sh_i32x8v tr_i32x8;
typedef SH_CONST_AS sh_i32x2v tr_i32x2;
typedef SH_CONST_AS sh_i32x4v tr_i32x4;

__device__ __forceinline__ TrReq req_of(const TreeAttnArgs& a, int r) {
  const sh_i32x8v w = *reinterpret_cast<const tr_i32x8*>((uintptr_t)(a.req + r));
  return TrReq{w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7]};
}

template <int HD>
__global__ __launch_bounds__(256, 2) void tree_attn_kernel(TreeAttnArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int items = a.th->items[blockIdx.x % SY_SH_DEAL] * SY_SH_DEAL;
  // (the first place is looked at together with the number of items: the launch has no more blocks than the lists have places)
  for (int k = blockIdx.x; k == (int)blockIdx.x || k < items; k += gridDim.x) {
    const tr_i32x8* place = reinterpret_cast<const tr_i32x8*>((uintptr_t)(a.places + k));
    const sh_i32x8v w = place[0];
    const sh_i32x4v at = *reinterpret_cast<const tr_i32x4*>((uintptr_t)(place + 1));       // request, tile, group
    if (k >= items) return;
    const TrReq q = {w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7]};
    const int tile = at[1], group = at[2], kh = group % a.Hkv, range = group / a.Hkv;
    if (q.n == 0 || tile >= q.tiles || q.tok + q.n > a.rows) continue;
    const int rows = q.n * a.G, keys = q.ctx + q.n;
    const int each = q.steps / q.ranges, more = q.steps % q.ranges;        // the first `more` ranges have a step more
    const int begin = range * each + min(range, more), end = begin + each + (range < more ? 1 : 0);
    ShItem it;
    it.flags = SY_SH_LEAF | (q.tiles == 1 ? SY_SH_ONCE : 0);
    it.kv_head = kh;
    it.row0 = tile * SY_SH_TILE_ROWS;
    it.n_rows = min(SY_SH_TILE_ROWS, rows - it.row0);
    it.tok = q.tok;
    it.page = at[0] * a.pitch;
    it.n_pages = (keys + SY_PAGE - 1) / SY_PAGE;
    it.key_begin = begin * TR_STEP;
    it.key_end = min(keys, end * TR_STEP);
    it.lim0 = q.ctx;
    it.part = q.ranges == 1 ? -1 : q.part + group * rows + it.row0;
    const int32_t* first = a.pages + it.page + it.key_begin / SY_PAGE;
    if (it.n_rows <= 32) attend<HD, 1, 4, true>(a, it, first, lds);
    else if (it.n_rows <= 64) attend<HD, 2, 2, true>(a, it, first, lds);
    else attend<HD, 4, 1, true>(a, it, first, lds);
    __syncthreads();                                          // the next item's copies come into the same LDS
  }
}

// Joins the ranges of the requests that have several: o = sum 2^(m_s - M) O_s / sum 2^(m_s - M) l_s.  A thread takes four values of a row; FLY ranges
// are asked for together.
template <int HD, int FLY>
__device__ __forceinline__ void join_row(const TreeAttnArgs& a, const TrReq& q, const int kh, const int row, const int d4) {
  const int rows = q.n * a.G, step = a.Hkv * rows;
  float M = -3e38f, l = 0.f;
  float4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < q.ranges; s0 += FLY) {
    float2 ml[FLY];
    float4 v[FLY];
#pragma unroll
    for (int s = 0; s < FLY; ++s) {
      const size_t at = (size_t)q.part + (size_t)min(s0 + s, q.ranges - 1) * step + kh * rows + row;
      ml[s] = a.part_ml[at];
      v[s] = *reinterpret_cast<const float4*>(a.part_o + at * HD + d4);
    }
    float top = M;
#pragma unroll
    for (int s = 0; s < FLY; ++s) top = fmaxf(top, ml[s].x);
    const float f = sh_ex2(M - top);
    M = top;
    l *= f;
    sum.x *= f; sum.y *= f; sum.z *= f; sum.w *= f;
#pragma unroll
    for (int s = 0; s < FLY; ++s)
      if (s0 + s < q.ranges) {
        const float w = sh_ex2(ml[s].x - M);
        l += ml[s].y * w;
        sum.x += v[s].x * w; sum.y += v[s].y * w; sum.z += v[s].z * w; sum.w += v[s].w * w;
      }
  }
  const int tok = q.tok + row / a.G, head = kh * a.G + row % a.G;
  const float inv = 1.0f / l;
  *reinterpret_cast<uint2*>(a.o + (int64_t)tok * a.o_ts + (int64_t)head * a.o_hs + d4) =
      make_uint2(pack_bf2(sum.x * inv, sum.y * inv), pack_bf2(sum.z * inv, sum.w * inv));
  if (a.lse && d4 == 0) a.lse[(size_t)tok * a.Hq + head] = (M + __log2f(l)) * 0.69314718055994531f;
}

template <int HD>
__global__ __launch_bounds__(TR_JOIN_AT * HD / 4) void tree_join_kernel(TreeAttnArgs a) {
  const int joins = a.th->joins, d4 = threadIdx.x % (HD / 4) * 4;
  for (int k = blockIdx.x; k < joins; k += gridDim.x) {
    const sh_i32x2v at = *reinterpret_cast<const tr_i32x2*>((uintptr_t)(a.joins + k));
    const TrReq q = req_of(a, at[0]);
    const int rows = q.n * a.G, row = at[1] + threadIdx.x / (HD / 4);
    if (q.n == 0 || q.tok + q.n > a.rows || row >= a.Hkv * rows) continue;
    if (q.ranges <= 2) join_row<HD, 2>(a, q, row / rows, row % rows, d4);
    else if (q.ranges <= 4) join_row<HD, 4>(a, q, row / rows, row % rows, d4);
    else join_row<HD, 8>(a, q, row / rows, row % rows, d4);
  }
}

template <int HD>
static constexpr size_t tree_lds() { return (size_t)20 * SY_PAGE * HD * 2; }
template <int HD>
static hipError_t launch_tree(const TreeAttnArgs& a, int grid, int joins, hipStream_t s) {
  tree_attn_kernel<HD><<<grid, 256, tree_lds<HD>(), s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || joins == 0) return e;
  tree_join_kernel<HD><<<joins, TR_JOIN_AT * HD / 4, 0, s>>>(a);
  return hipGetLastError();
}
static hipError_t prepare_attention(int hd) {
  const void* kernel = hd == 128 ? reinterpret_cast<const void*>(&tree_attn_kernel<128>) : reinterpret_cast<const void*>(&tree_attn_kernel<64>);
  return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)(hd == 128 ? tree_lds<128>() : tree_lds<64>()));
}

extern "C" int32_t synera_tree_attention(synera_tree* t, const synera_heads* q, const void* d_k_layer, const void* d_v_layer, float scale,
                                         float* d_lse, void* stream) {
  if (!t || !q || !d_k_layer || !d_v_layer || !t->planned) return SYNERA_EINVAL;
  const ShLimits& l = t->lim;
  hipStream_t s = static_cast<hipStream_t>(stream);
  TreeAttnArgs a = {};
  // A plan on the device that may be another than the last one that was called is served as far as the call's tensors say that they go, as in a graph.
  const bool captured = capturing(s), graph = captured || (t->replays && q->n_rows);
  const int32_t st = sh_attention_args(a, l, t->n_pages, t->n_rows, graph, q, d_k_layer, d_v_layer, scale, d_lse);
  if (st != SYNERA_OK) return st == SH_NOTHING ? SYNERA_OK : st;
  if (!rope_device_ok(t->device)) return SYNERA_EINVAL;
  a.pages = t->table;
  a.part_o = t->part_o;
  a.part_ml = t->part_ml;
  a.th = t->head;
  a.req = t->req;
  a.places = t->items;
  a.joins = t->joins;
  a.masks = t->masks;
  a.pitch = t->pitch;
  a.rows = q->n_rows ? q->n_rows : INT32_MAX;
  // As many blocks as there may be items, up to four for each place; the kernel loops.  Captured calls serve plans of any size.
  const int grid = std::min(t->items_room * SY_SH_DEAL, TR_GRID * l.slots) / SY_SH_DEAL * SY_SH_DEAL;
  const bool cuts = (captured || t->replays ? l.max_pages : t->columns) > 2 * TR_STEP / SY_PAGE;      // no range is shorter than two steps
  const int joins = cuts ? TR_JOIN_GRID * l.slots : 0;
  const hipError_t e = l.hd == 128 ? launch_tree<128>(a, grid, joins, s) : launch_tree<64>(a, grid, joins, s);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    return SYNERA_EHIP;
  }
  return SYNERA_OK;
}

// ------------------------------------------------------------------------------------ the accepted path
struct AcceptArgs {
  const TrReq* req;
  const int32_t *parent, *tokens, *target, *anchor, *n_given;
  int32_t *accept_len, *token, *path, *n_path;
  const TrHead* head;
  int32_t rows;                  // that the arrays of this call have
};
// A wavefront walks a request's tree.  Lane l holds nodes l, l + 64, ..; a step asks all of them at once which hang on the node at hand
// with the wanted token, and the first one is the next.  Bound by latency: a few loads, then some 30 cycles a step.
__global__ __launch_bounds__(64) void tree_accept_kernel(AcceptArgs a) {
  const int i = blockIdx.x, lane = threadIdx.x;
  if (i >= a.head->B) return;                                 // (a plan that was replayed may have fewer requests, or more rows, than the call)
  TrReq q = a.req[i];
  if (q.tok + q.rows > a.rows) q.n = q.rows = 0;
  int32_t parent[4], token[4], target[4];
  int mine[4];                                                // the node's place on the path
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int j = lane + 64 * w;
    const bool on = j < q.n;
    parent[w] = on ? a.parent[q.tok + j] : -2;
    token[w] = on ? a.tokens[q.tok + j] : 0;
    target[w] = on ? a.target[q.tok + j] : 0;
    mine[w] = -1;
  }
  const int given = a.n_given ? min(max(a.n_given[i], 0), q.n) : 0;
#pragma unroll
  for (int w = 0; w < 4; ++w)
    if (lane + 64 * w < given) mine[w] = lane + 64 * w;
  auto of = [&](const int32_t (&v)[4], int node) {
    const int32_t x = node < 64 ? v[0] : node < 128 ? v[1] : node < 192 ? v[2] : v[3];
    return __builtin_amdgcn_readlane(x, node & 63);
  };
  int cur = given - 1, n = given;
  bool wanted = q.n > 0 && (given > 0 || a.anchor);
  int32_t want = !wanted ? -1 : given > 0 ? of(target, cur) : a.anchor[i];
  while (wanted) {
    int next = -1;
#pragma unroll
    for (int w = 3; w >= 0; --w) {
      const int j = lane + 64 * w;
      const uint64_t hit = __builtin_amdgcn_ballot_w64(j >= given && j < q.n && parent[w] == cur && token[w] == want);
      if (hit) next = 64 * w + __builtin_ctzll(hit);
    }
    if (next < 0) break;
#pragma unroll
    for (int w = 0; w < 4; ++w)
      if (lane + 64 * w == next) mine[w] = n;
    ++n;
    cur = next;
    want = of(target, cur);
  }
  if (lane == 0) {
    a.accept_len[i] = n - given;
    a.n_path[i] = n;
    a.token[i] = want;
  }
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int j = lane + 64 * w;
    if (j >= n && j < q.rows) a.path[q.tok + j] = -1;
    if (mine[w] >= 0) a.path[q.tok + mine[w]] = j;
  }
  for (int j = lane + TR_NODES; j < q.rows; j += 64) a.path[q.tok + j] = -1;       // (refused: more rows than a tree may have)
}

extern "C" int32_t synera_tree_accept(synera_tree* t, int64_t n_rows, const int32_t* d_tokens, const int32_t* d_target, const int32_t* d_anchor,
                                      const int32_t* d_n_given, int32_t* d_accept_len, int32_t* d_token, int32_t* d_path, int32_t* d_n_path,
                                      void* stream) {
  if (!t || !t->planned || !d_accept_len || !d_token || !d_n_path || n_rows < t->n_rows || (!d_anchor && !d_n_given)) return SYNERA_EINVAL;
  if (n_rows > 0 && (!d_tokens || !d_target || !d_path)) return SYNERA_EINVAL;
  if (off4({d_tokens, d_target, d_anchor, d_n_given, d_accept_len, d_token, d_path, d_n_path})) return SYNERA_EINVAL;
  // no output on an input or on another one, over all rows that a replayed plan may have
  const int64_t B = t->B, T = std::min<int64_t>(n_rows, t->lim.max_tokens);
  const Range outs[4] = {ints(d_accept_len, B), ints(d_token, B), ints(d_path, T), ints(d_n_path, B)};
  const Range ins[4] = {ints(d_tokens, T), ints(d_target, T), ints(d_anchor, B), ints(d_n_given, B)};
  for (int i = 0; i < 4; ++i)
    for (int k = 0; k < 4; ++k)
      if (meet(outs[i], ins[k]) || (i != k && meet(outs[i], outs[k]))) return SYNERA_EINVAL;
  if (!rope_device_ok(t->device)) return SYNERA_EINVAL;
  const AcceptArgs a = {t->req, t->parent, d_tokens, d_target, d_anchor, d_n_given, d_accept_len, d_token, d_path, d_n_path, t->head,
                        (int32_t)std::min<int64_t>(n_rows, INT32_MAX)};
  tree_accept_kernel<<<t->B, 64, 0, static_cast<hipStream_t>(stream)>>>(a);
  return hipGetLastError() == hipSuccess ? SYNERA_OK : SYNERA_EHIP;
}

// ------------------------------------------------------------------------------------ its keys and values
struct CommitArgs {
  const TrReq* req;
  const int32_t *slot, *path, *n_path;
  bf16_t *k, *v;
  int64_t layer_stride;
  int32_t n, hd;                 // n = Hkv hd
  int32_t k_parts;               // of a layer's blocks, those that move keys; the others move values
  const TrHead* head;
  int32_t rows;                  // that the arrays of this call have
};
// A block moves a part of one layer's values, or keys, of one request.  A thread keeps to its own 16 bytes of a key, or its own dim of the
// values, and takes the path in order: node k's place was read, if at all, by one before it, since path[k] >= k.  A batch's loads are on their way
// together.
// A dim's 16 slots of a page lie side by side, so a node's values are two bytes in each 32 of its page, and whole pages are read and written
// for it: 64 paths with 104 moves in 32 layers of 8 x 128 are 27 MB of keys and values, and 150 MB of pages.  Rows are written whole: two bytes at a time 57 us.
__global__ __launch_bounds__(256) void tree_commit_kernel(CommitArgs a) {
  constexpr int FLY = 8;
  __shared__ int32_t from[TR_NODES], to[TR_NODES], in_wave[4];
  const int tid = threadIdx.x, wave = tid >> 6, i = blockIdx.x;
  if (i >= a.head->B) return;
  const TrReq q = a.req[i];
  const int n = q.tok + q.n > a.rows ? 0 : min(a.n_path[i], q.n);
  int p = -1;
  if (tid < n) p = a.path[q.tok + tid];
  const bool moves = p > tid && p < q.n;
  const uint64_t hits = __builtin_amdgcn_ballot_w64(moves);
  if ((tid & 63) == 0) in_wave[wave] = __popcll(hits);
  __syncthreads();
  int at = __popcll(hits & ((1ull << (tid & 63)) - 1)), all = 0;
  for (int w = 0; w < 4; ++w) {
    if (w < wave) at += in_wave[w];
    all += in_wave[w];
  }
  if (all == 0) return;
  if (moves) {
    from[at] = a.slot[q.tok + p];
    to[at] = a.slot[q.tok + tid];
  }
  __syncthreads();
  const size_t layer = (size_t)blockIdx.y * a.layer_stride, page = (size_t)a.n * SY_PAGE;
  if ((int)blockIdx.z < a.k_parts) {
    const int piece = blockIdx.z * 256 + tid, per = a.hd / 8;               // 16 bytes of head piece / per
    if (piece >= a.n / 8) return;
    bf16_t* base = a.k + layer + (size_t)(piece / per) * SY_PAGE * a.hd + piece % per * 8;
    auto place = [&](int32_t s) { return reinterpret_cast<u32x4*>(base + (size_t)(s / SY_PAGE) * page + s % SY_PAGE * a.hd); };
    for (int m = 0; m < all; m += FLY) {
      u32x4 x[FLY];
#pragma unroll
      for (int f = 0; f < FLY; ++f) x[f] = *place(from[min(m + f, all - 1)]);
#pragma unroll
      for (int f = 0; f < FLY; ++f)
        if (m + f < all) *place(to[m + f]) = x[f];
    }
  } else {
    const int dim = (blockIdx.z - a.k_parts) * 256 + tid;
    if (dim >= a.n) return;
    bf16_t* base = a.v + layer + (size_t)dim * SY_PAGE;
    for (int m = 0; m < all;) {                               // the page that move m goes to, with all others that do
      const int at = __builtin_amdgcn_readfirstlane(to[m]) / SY_PAGE;
      u32x4* row = reinterpret_cast<u32x4*>(base + (size_t)at * page);
      u32x4 r[2] = {row[0], row[1]};
      bool more = true;
      while (more) {
        uint32_t x[FLY];
        int slot[FLY];
#pragma unroll
        for (int f = 0; f < FLY; ++f) {
          const int s = __builtin_amdgcn_readfirstlane(from[min(m + f, all - 1)]), d = __builtin_amdgcn_readfirstlane(to[min(m + f, all - 1)]);
          more = more && m + f < all && d / SY_PAGE == at;
          slot[f] = more ? d % SY_PAGE : -1;
          x[f] = 0;
          if (more) x[f] = base[(size_t)(s / SY_PAGE) * page + s % SY_PAGE];
        }
        int n_moved = 0;
#pragma unroll
        for (int f = 0; f < FLY; ++f) {
          if (slot[f] < 0) continue;
          ++n_moved;
          const uint32_t shift = 16 * (slot[f] & 1), keep = 0xFFFF0000u >> shift;
#pragma unroll
          for (int w = 0; w < 8; ++w)
            if (w == slot[f] >> 1) r[w >> 2][w & 3] = (r[w >> 2][w & 3] & keep) | x[f] << shift;
        }
        m += n_moved;
      }
      row[0] = r[0];
      row[1] = r[1];
    }
  }
}

extern "C" int32_t synera_tree_commit(synera_tree* t, int64_t n_rows, const int32_t* d_path, const int32_t* d_n_path, int32_t n_layers,
                                      int64_t layer_stride, void* d_k_pool, void* d_v_pool, void* stream) {
  if (!t || !t->planned || !d_n_path || !d_k_pool || !d_v_pool || n_rows < t->n_rows || n_layers < 1 || n_layers > 65535) return SYNERA_EINVAL;
  if (n_rows > 0 && !d_path) return SYNERA_EINVAL;
  if (off4({d_path, d_n_path}) || (reinterpret_cast<uintptr_t>(d_k_pool) | reinterpret_cast<uintptr_t>(d_v_pool)) % 16) return SYNERA_EINVAL;
  const ShLimits& l = t->lim;
  const int64_t layer = (int64_t)t->n_pages * l.Hkv * SY_PAGE * l.hd;
  if (n_layers > 1 && (layer_stride < layer || layer_stride % 8)) return SYNERA_EINVAL;
  const int64_t all = (n_layers > 1 ? (n_layers - 1) * layer_stride : 0) + layer;
  const Range k = {reinterpret_cast<uintptr_t>(d_k_pool), reinterpret_cast<uintptr_t>(d_k_pool) + 2 * (uintptr_t)all};
  const Range v = {reinterpret_cast<uintptr_t>(d_v_pool), reinterpret_cast<uintptr_t>(d_v_pool) + 2 * (uintptr_t)all};
  if (meet(k, v)) return SYNERA_EINVAL;
  for (const Range& in : {ints(d_path, std::min<int64_t>(n_rows, l.max_tokens)), ints(d_n_path, t->B)})
    if (meet(k, in) || meet(v, in)) return SYNERA_EINVAL;
  if (!rope_device_ok(t->device)) return SYNERA_EINVAL;
  if (t->n_rows == 0 && !t->replays && !capturing(static_cast<hipStream_t>(stream))) return SYNERA_OK;
  const int32_t n = l.Hkv * l.hd;
  CommitArgs a = {t->req, t->slot, d_path, d_n_path, static_cast<bf16_t*>(d_k_pool), static_cast<bf16_t*>(d_v_pool), layer_stride, n, l.hd, (n / 8 + 255) / 256, t->head,
                  (int32_t)std::min<int64_t>(n_rows, INT32_MAX)};
  tree_commit_kernel<<<dim3(t->B, n_layers, a.k_parts + (n + 255) / 256), 256, 0, static_cast<hipStream_t>(stream)>>>(a);
  return hipGetLastError() == hipSuccess ? SYNERA_OK : SYNERA_EHIP;
}
