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
#define TR_STEP SY_SH_STEP       // keys of one step, the unit of work

// ------------------------------------------------------------------------------------ the plan on the device
// The attention's work is one line: for each request in turn its streams (KV head, then tile of rows), for each stream its steps of TR_STEP keys
// and TR_START more for what it takes to begin and end one.  Block b takes the share-th part b of the line.  So only the
// places where parts begin are written down, and which parts a stream lies in follows from them.
#define TR_START 2
#define TR_SHARE 6               // the least that a block takes
struct TrHead {
  ShHeader sh;                   // tokens and windows, for the append
  int32_t n_blocks, share, B, pad[13];
};
struct TrReq {                   // 32 bytes, scalar loads
  int32_t ctx, n, tok;           // n: 0 where the request has no nodes or is refused
  int32_t steps, cost, streams, tiles;   // as the line counts them, refused or not
  int32_t rows;                  // of its n_nodes, those that there is room for
};
struct TrStart {                 // where a block's part begins
  int32_t req, stream, step, pad;
};

struct synera_tree {
  ShLimits lim;                  // (head counts and sizes; no room of a host plan)
  int device;
  bool planned;
  int32_t B, n_pages;
  int64_t n_rows;
  int32_t pitch;                 // columns of the table's copy
  char* dev;
  TrHead* head;
  TrReq* req;
  TrStart* start;
  ShWindow* windows;
  int32_t *pos, *slot, *parent, *table;
  uint32_t* masks;
  float* part_o;
  float2* part_ml;
  int32_t grid;                  // blocks of the attention
};

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
  t->grid = (t->lim.slots + SY_SH_DEAL - 1) / SY_SH_DEAL * SY_SH_DEAL;
  const size_t B = (size_t)max_batch, T = (size_t)max_tokens, parts = 2 * (size_t)t->lim.slots * SY_SH_TILE_ROWS;
  const size_t sizes[] = {sizeof(TrHead), B * sizeof(TrReq), ((size_t)t->lim.slots + 1) * sizeof(TrStart), B * (TR_NODES / SY_PAGE + 1) * sizeof(ShWindow),
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
  take(t->start);
  take(t->windows);
  take(t->pos);
  take(t->slot);
  take(t->parent);
  take(t->table);
  take(t->masks);
  take(t->part_o);
  take(t->part_ml);
  *out = t;
  return SYNERA_OK;
}

// ------------------------------------------------------------------------------------ planning
struct PlanArgs {
  const int32_t *ctx, *n_nodes, *parent, *table;
  int32_t* status;
  TrHead* head;
  TrReq* req;
  TrStart* start;
  ShWindow* windows;
  int32_t *pos, *slot, *parents, *pages;
  uint32_t* masks;
  int32_t B, columns, pitch, n_pages, Hkv, G, slots;
  int64_t n_rows;
};

// What a request's lengths alone say of it; every block forms it for all of them.
struct TrSize {
  int32_t rows, windows, steps, cost, streams, tiles;
};
__device__ __forceinline__ TrSize size_of(const PlanArgs& a, int32_t ctx, int32_t n) {
  TrSize s = {0, 0, 0, 0, 0, 0};
  if (n < 0 || n > TR_NODES) return s;
  s.rows = n;
  const int64_t keys = (int64_t)ctx + n;
  if (n == 0 || ctx < 0 || (keys + SY_PAGE - 1) / SY_PAGE > a.columns) return s;
  s.windows = (int32_t)((keys - 1) / SY_PAGE - ctx / SY_PAGE + 1);
  s.steps = (int32_t)((keys + TR_STEP - 1) / TR_STEP);
  s.cost = s.steps + TR_START;
  s.tiles = (n * a.G + SY_SH_TILE_ROWS - 1) / SY_SH_TILE_ROWS;
  s.streams = s.tiles * a.Hkv;
  return s;
}

// Block i plans request i.  It sums up the requests before it by itself (a few thousand numbers at most, which lie in the caches), so that one launch
// does.  Paths by doubling: in each round a node takes over what its forefather has gathered, and that one's forefather.
__global__ __launch_bounds__(256) void tree_plan_kernel(PlanArgs a) {
  const int tid = threadIdx.x, me = blockIdx.x;
  __shared__ int64_t sums[4][5];
  int64_t v[5] = {0, 0, 0, 0, 0};                            // rows, windows and work before this request; rows and work of all
  int32_t windows_all = 0;
  for (int i = tid; i < a.B; i += 256) {
    const TrSize s = size_of(a, a.ctx[i], a.n_nodes[i]);
    const int64_t work = (int64_t)s.streams * s.cost;
    if (i < me) {
      v[0] += s.rows;
      v[1] += s.windows;
      v[2] += work;
    }
    v[3] += s.rows;
    v[4] += work;
    windows_all += s.windows;
  }
#pragma unroll
  for (int k = 0; k < 5; ++k)
    for (int o = 1; o < 64; o <<= 1) v[k] += __shfl_xor(v[k], o);
  if ((tid & 63) == 0)
    for (int k = 0; k < 5; ++k) sums[tid >> 6][k] = v[k];
  __shared__ int32_t all_windows;
  __shared__ int32_t up_[TR_NODES];
  __shared__ uint32_t gather[TR_NODES][9];                    // (9: neighbours on other banks)
  if (tid == 0) all_windows = 0;
  __syncthreads();
  if (windows_all) atomicAdd(&all_windows, windows_all);
#pragma unroll
  for (int k = 0; k < 5; ++k) v[k] = sums[0][k] + sums[1][k] + sums[2][k] + sums[3][k];
  const int64_t first = v[0];
  const int32_t ctx = a.ctx[me], n = a.n_nodes[me];
  const TrSize s = size_of(a, ctx, n);
  const int64_t share64 = max((int64_t)TR_SHARE, (v[4] + a.slots - 1) / a.slots);
  const int32_t share = (int32_t)min(share64, (int64_t)0x7FFFFFFF);

  // ---- what only this block looks at: parents and pages
  int32_t status = n < 0 || n > TR_NODES ? SYNERA_EINVAL : ctx < 0 ? SYNERA_ERANGE : SYNERA_OK;
  const int64_t keys = (int64_t)ctx + (status == SYNERA_OK ? n : 0);
  if (status == SYNERA_OK && (first + s.rows > a.n_rows || (n > 0 && s.streams == 0))) status = SYNERA_ENOSPC;
  const bool fits = status == SYNERA_OK && n > 0;
  bool bad_parent = false, bad_page = false;
  int32_t up = -1;
  if (fits && tid < n) {
    up = a.parent[first + tid];
    bad_parent = up < -1 || up >= tid;
    if (bad_parent) up = -1;
  }
  const int32_t need = fits ? (int32_t)((keys + SY_PAGE - 1) / SY_PAGE) : 0;
  const int32_t* row = a.table + (size_t)me * a.columns;
  int32_t* copy = a.pages + (size_t)me * a.pitch;
  for (int c = tid; c < need + TR_AHEAD; c += 256) {
    if (need == 0) break;
    const int32_t id = row[min(c, need - 1)];
    bad_page |= id < 0 || id >= a.n_pages;
    copy[c] = id;
  }
  const int any = __syncthreads_or((bad_parent ? 1 : 0) | (bad_page ? 2 : 0));
  const int parent_bad = __syncthreads_or(bad_parent);
  if (any) status = parent_bad ? SYNERA_EINVAL : SYNERA_ERANGE;
  const bool live = fits && !any;

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
  if (tid < s.rows && first + tid < a.n_rows) {
    const int64_t at = first + tid;
    if (live) {
      int depth = -1;
#pragma unroll
      for (int w = 0; w < 8; ++w) depth += __popc(word[w]);
      const int32_t p = ctx + tid;
      a.pos[at] = ctx + depth;
      a.slot[at] = row[p / SY_PAGE] * SY_PAGE + p % SY_PAGE;
      a.parents[at] = a.parent[at];
      uint32_t* m = a.masks + at * SY_TREE_MASK;
      m[0] = m[1] = 0xFFFFFFFFu;
#pragma unroll
      for (int w = 0; w < 8; ++w) m[2 + w] = word[w];
#pragma unroll
      for (int w = 10; w < SY_TREE_MASK; ++w) m[w] = 0;
    } else {
      a.pos[at] = 0;
      a.slot[at] = -1;
    }
  }
  for (int w = tid; w < s.windows; w += 256) {
    const int32_t page = ctx / SY_PAGE + w, from = max(ctx, page * SY_PAGE), to = min(ctx + n, (page + 1) * SY_PAGE);
    ShWindow x = {0, 0, 0, 0};
    if (live) x = ShWindow{row[page], (int32_t)first + from - ctx, from - page * SY_PAGE, to - page * SY_PAGE};
    a.windows[v[1] + w] = x;
  }
  // ---- the line
  const int64_t work = (int64_t)s.streams * s.cost;
  for (int64_t b = (v[2] + share - 1) / share + tid; b * share < v[2] + work; b += 256) {
    const int64_t at = b * share - v[2];
    a.start[b] = TrStart{me, (int32_t)(at / s.cost), (int32_t)(at % s.cost), 0};
  }
  if (tid == 0) {
    a.req[me] = TrReq{ctx, live ? n : 0, (int32_t)first, s.steps, s.cost, s.streams, s.tiles, (int32_t)max((int64_t)0, min((int64_t)s.rows, a.n_rows - first))};
    if (a.status) a.status[me] = status;
    if (me == 0) {
      a.head->sh.n_tokens = (int32_t)min(v[3], a.n_rows);
      a.head->sh.n_windows = all_windows;
      a.head->n_blocks = (int32_t)((v[4] + share - 1) / share);
      a.head->share = share;
      a.head->B = a.B;
    }
  }
}

static bool off4(std::initializer_list<const void*> all) {
  uintptr_t bits = 0;
  for (const void* p : all) bits |= reinterpret_cast<uintptr_t>(p);
  return bits % 4 != 0;
}

extern "C" int32_t synera_tree_plan(synera_tree* t, int32_t B, const int32_t* d_ctx_len, const int32_t* d_n_nodes, const int32_t* d_parent,
                                    int64_t n_rows, const int32_t* d_table, int32_t columns, int32_t n_pages_in_pool, int32_t* d_status,
                                    void* stream) {
  if (!t || !d_ctx_len || !d_n_nodes || !d_table || B < 1 || n_rows < 0 || columns < 1 || n_pages_in_pool < 1) return SYNERA_EINVAL;
  if (n_rows > 0 && !d_parent) return SYNERA_EINVAL;
  if (off4({d_ctx_len, d_n_nodes, d_parent, d_table, d_status})) return SYNERA_EINVAL;
  if (n_pages_in_pool >= 1 << 27) return SYNERA_EUNSUP;
  const ShLimits& l = t->lim;
  if (B > l.max_batch || n_rows > l.max_tokens || columns > l.max_pages) return SYNERA_ENOSPC;
  if (!rope_device_ok(t->device)) return SYNERA_EINVAL;
  const PlanArgs a = {d_ctx_len, d_n_nodes, d_parent, d_table, d_status, t->head, t->req, t->start, t->windows, t->pos, t->slot, t->parent, t->table,
                      t->masks, B, columns, t->pitch, n_pages_in_pool, l.Hkv, l.Hq / l.Hkv, l.slots, n_rows};
  tree_plan_kernel<<<B, 256, 0, static_cast<hipStream_t>(stream)>>>(a);
  if (hipGetLastError() != hipSuccess) return SYNERA_EHIP;
  t->planned = true;
  t->B = B;
  t->n_rows = n_rows;
  t->n_pages = n_pages_in_pool;
  return SYNERA_OK;
}

// ------------------------------------------------------------------------------------ append
extern "C" int32_t synera_tree_append_rope(synera_tree* t, const synera_rope* rope, int32_t dtype, const synera_heads* q,
                                           const synera_heads* k, const synera_heads* v, float eps, void* d_k_layer, void* d_v_layer,
                                           void* stream) {
  if (!t || !t->planned) return SYNERA_EINVAL;
  const ShTarget target = {&t->lim, t->device, t->n_pages, t->n_rows, 0, false, t->pos, t->slot, &t->head->sh, t->windows};
  return sh_append(target, rope, dtype, q, k, v, eps, d_k_layer, d_v_layer, stream);
}

// ------------------------------------------------------------------------------------ attention
struct TreeAttnArgs : SharedAttnArgs {
  const TrHead* th;
  const TrReq* req;
  const TrStart* start;
  const uint32_t* masks;
  int32_t pitch;
};
typedef SH_CONST_AS sh_i32x8v tr_i32x8;
typedef SH_CONST_AS sh_i32x4v tr_i32x4;

__device__ __forceinline__ TrReq req_of(const TreeAttnArgs& a, int r) {
  const sh_i32x8v w = *reinterpret_cast<const tr_i32x8*>((uintptr_t)(a.req + r));
  return TrReq{w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7]};
}
__device__ __forceinline__ TrStart start_of(const TreeAttnArgs& a, int b) {
  const sh_i32x4v w = *reinterpret_cast<const tr_i32x4*>((uintptr_t)(a.start + b));
  return TrStart{w[0], w[1], w[2], 0};
}
// Rows of tile `tile` of a request: its first one, and how many.
__device__ __forceinline__ int tile_rows(const TreeAttnArgs& a, const TrReq& q, int tile) { return min(SY_SH_TILE_ROWS, q.n * a.G - tile * SY_SH_TILE_ROWS); }

template <int HD>
__global__ __launch_bounds__(256, 2) void tree_attn_kernel(TreeAttnArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int n_blocks = a.th->n_blocks, share = a.th->share, B = a.th->B;
  // each XCD takes a run of the line, so that tiles of rows that read the same keys meet in its L2
  const int per = (n_blocks + SY_SH_DEAL - 1) / SY_SH_DEAL, b = (int)(blockIdx.x % SY_SH_DEAL) * per + (int)(blockIdx.x / SY_SH_DEAL);
  if ((int)(blockIdx.x / SY_SH_DEAL) >= per || b >= n_blocks) return;
  const TrStart st = start_of(a, b);
  int r = st.req, s = st.stream, k0 = st.step, left = share;
  while (r < B) {
    const TrReq q = req_of(a, r);
    for (; left > 0 && s < q.streams; ++s, k0 = 0) {
      const int len = min(q.cost - k0, left), end = min(k0 + len, q.steps);
      left -= len;
      if (k0 >= q.steps || q.n == 0) continue;
      const int tile = s % q.tiles, keys = q.ctx + q.n;
      const bool whole = k0 == 0 && end == q.steps;
      ShItem it;
      it.flags = SY_SH_LEAF | (q.tiles == 1 ? SY_SH_ONCE : 0);
      it.kv_head = s / q.tiles;
      it.n_rows = tile_rows(a, q, tile);
      it.row0 = tile * SY_SH_TILE_ROWS;
      it.tok = q.tok;
      it.page = r * a.pitch;
      it.n_pages = (keys + SY_PAGE - 1) / SY_PAGE;
      it.key_begin = k0 * TR_STEP;
      it.key_end = min(keys, end * TR_STEP);
      it.lim0 = q.ctx;
      it.part = whole ? -1 : (2 * b + (k0 > 0 ? 0 : 1)) * SY_SH_TILE_ROWS;
      const int32_t* first = a.pages + it.page + it.key_begin / SY_PAGE;
      if (it.n_rows <= 32) attend<HD, 1, 4, true>(a, it, first, lds);
      else if (it.n_rows <= 64) attend<HD, 2, 2, true>(a, it, first, lds);
      else attend<HD, 4, 1, true>(a, it, first, lds);
      __syncthreads();                                        // the next item's copies come into the same LDS
    }
    if (left <= 0) return;
    ++r;
    s = 0;
    k0 = 0;
  }
}

// Joins the parts of streams that are cut: o = sum 2^(m_s - M) O_s / sum 2^(m_s - M) l_s.  Row b of the launch's blocks stands for the end of block
// b's part of the line; those that cut one stream share its rows, so that a stream of many parts is joined by many blocks (one row of them for
// each stream: 60 parts of 104 rows took 42 us).  A thread takes four values of a row.
#define TR_JOIN 4
struct TrJoin {                  // a stream that is cut
  int count, first;              // its parts; the block that begins it
  int tile, kh;
};
template <int HD, int FLY>        // FLY parts are asked for together
__device__ __forceinline__ void join_row(const TreeAttnArgs& a, const TrReq& q, const TrJoin& j, const int row, const int d4) {
  float M = -3e38f, l = 0.f;
  float4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < j.count; s0 += FLY) {
    float2 ml[FLY];
    float4 v[FLY];
#pragma unroll
    for (int s = 0; s < FLY; ++s) {
      const int p = min(s0 + s, j.count - 1);
      const size_t at = (size_t)(2 * (j.first + p) + (p == 0 ? 1 : 0)) * SY_SH_TILE_ROWS + row;
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
      if (s0 + s < j.count) {
        const float w = sh_ex2(ml[s].x - M);
        l += ml[s].y * w;
        sum.x += v[s].x * w; sum.y += v[s].y * w; sum.z += v[s].z * w; sum.w += v[s].w * w;
      }
  }
  const int in_node = j.tile * SY_SH_TILE_ROWS + row, tok = q.tok + in_node / a.G, head = j.kh * a.G + in_node % a.G;
  const float inv = 1.0f / l;
  *reinterpret_cast<uint2*>(a.o + (int64_t)tok * a.o_ts + (int64_t)head * a.o_hs + d4) =
      make_uint2(pack_bf2(sum.x * inv, sum.y * inv), pack_bf2(sum.z * inv, sum.w * inv));
  if (a.lse && d4 == 0) a.lse[(size_t)tok * a.Hq + head] = (M + __log2f(l)) * 0.69314718055994531f;
}

template <int HD>
__global__ __launch_bounds__(256) void tree_join_kernel(TreeAttnArgs a) {
  const int n_blocks = a.th->n_blocks, share = a.th->share, b = blockIdx.x;
  if (b + 1 >= n_blocks) return;
  const TrStart st = start_of(a, b + 1);
  const TrReq q = req_of(a, st.req);
  if (st.step <= 0 || st.step >= q.steps || q.n == 0) return;
  const int before = (st.step + share - 1) / share, cuts = before + (q.steps - st.step + share - 1) / share - 1;
  const TrJoin j = {cuts + 1, b + 1 - before, st.stream % q.tiles, st.stream / q.tiles};
  const int n = tile_rows(a, q, j.tile) * (HD / 4);
  for (int i = ((before - 1) * TR_JOIN + blockIdx.y) * 256 + threadIdx.x; i < n; i += cuts * TR_JOIN * 256) {
    const int row = i / (HD / 4), d4 = i % (HD / 4) * 4;
    if (j.count <= 2) join_row<HD, 2>(a, q, j, row, d4);
    else if (j.count <= 4) join_row<HD, 4>(a, q, j, row, d4);
    else join_row<HD, 8>(a, q, j, row, d4);
  }
}

template <int HD>
static constexpr size_t tree_lds() { return (size_t)20 * SY_PAGE * HD * 2; }
template <int HD>
static hipError_t launch_tree(const TreeAttnArgs& a, int grid, hipStream_t s) {
  tree_attn_kernel<HD><<<grid, 256, tree_lds<HD>(), s>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  tree_join_kernel<HD><<<dim3(grid, TR_JOIN), 256, 0, s>>>(a);
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
  const int32_t st = sh_attention_args(a, l, t->n_pages, t->n_rows, capturing(s), q, d_k_layer, d_v_layer, scale, d_lse);
  if (st != SYNERA_OK) return st == SH_NOTHING ? SYNERA_OK : st;
  if (!rope_device_ok(t->device)) return SYNERA_EINVAL;
  a.pages = t->table;
  a.part_o = t->part_o;
  a.part_ml = t->part_ml;
  a.th = t->head;
  a.req = t->req;
  a.start = t->start;
  a.masks = t->masks;
  a.pitch = t->pitch;
  const hipError_t e = l.hd == 128 ? launch_tree<128>(a, t->grid, s) : launch_tree<64>(a, t->grid, s);
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
};
// A wavefront walks a request's tree.  Lane l holds nodes l, l + 64, ..; a step asks all of them at once which hang on the node at hand
// with the wanted token, and the first one is the next.  Bound by latency: a few loads, then some 30 cycles a step.
__global__ __launch_bounds__(64) void tree_accept_kernel(AcceptArgs a) {
  const int i = blockIdx.x, lane = threadIdx.x;
  const TrReq q = a.req[i];
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
}

extern "C" int32_t synera_tree_accept(synera_tree* t, int64_t n_rows, const int32_t* d_tokens, const int32_t* d_target, const int32_t* d_anchor,
                                      const int32_t* d_n_given, int32_t* d_accept_len, int32_t* d_token, int32_t* d_path, int32_t* d_n_path,
                                      void* stream) {
  if (!t || !t->planned || !d_accept_len || !d_token || !d_n_path || n_rows < t->n_rows || (!d_anchor && !d_n_given)) return SYNERA_EINVAL;
  if (t->n_rows > 0 && (!d_tokens || !d_target || !d_path)) return SYNERA_EINVAL;
  if (off4({d_tokens, d_target, d_anchor, d_n_given, d_accept_len, d_token, d_path, d_n_path})) return SYNERA_EINVAL;
  // no output on an input or on another one
  const int64_t B = t->B, T = t->n_rows;
  auto range = [](const int32_t* p, int64_t n) { return Range{reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + (p ? 4 * n : 0)}; };
  const Range outs[4] = {range(d_accept_len, B), range(d_token, B), range(d_path, T), range(d_n_path, B)};
  const Range ins[4] = {range(d_tokens, T), range(d_target, T), range(d_anchor, B), range(d_n_given, B)};
  for (int i = 0; i < 4; ++i)
    for (int k = 0; k < 4; ++k)
      if (meet(outs[i], ins[k]) || (i != k && meet(outs[i], outs[k]))) return SYNERA_EINVAL;
  if (!rope_device_ok(t->device)) return SYNERA_EINVAL;
  const AcceptArgs a = {t->req, t->parent, d_tokens, d_target, d_anchor, d_n_given, d_accept_len, d_token, d_path, d_n_path};
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
};
// A block moves a part of one layer's values, or keys, of one request.  A thread keeps to its own 16 bytes of a key, or its own dim of the
// values, and takes the path in order: node k's place was read, if at all, by one before it, since path[k] >= k.  A batch's loads are on their way
// together.
__global__ __launch_bounds__(256) void tree_commit_kernel(CommitArgs a) {
  constexpr int FLY = 8;
  __shared__ int32_t from[TR_NODES], to[TR_NODES], in_wave[4];
  const int tid = threadIdx.x, wave = tid >> 6, i = blockIdx.x;
  const TrReq q = a.req[i];
  const int n = min(a.n_path[i], q.n);
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
    auto place = [&](int32_t s) { return base + (size_t)(s / SY_PAGE) * page + s % SY_PAGE; };
    for (int m = 0; m < all; m += FLY) {
      bf16_t x[FLY];
#pragma unroll
      for (int f = 0; f < FLY; ++f) x[f] = *place(from[min(m + f, all - 1)]);
#pragma unroll
      for (int f = 0; f < FLY; ++f)
        if (m + f < all) *place(to[m + f]) = x[f];
    }
  }
}

extern "C" int32_t synera_tree_commit(synera_tree* t, int64_t n_rows, const int32_t* d_path, const int32_t* d_n_path, int32_t n_layers,
                                      int64_t layer_stride, void* d_k_pool, void* d_v_pool, void* stream) {
  if (!t || !t->planned || !d_n_path || !d_k_pool || !d_v_pool || n_rows < t->n_rows || n_layers < 1 || n_layers > 65535) return SYNERA_EINVAL;
  if (t->n_rows > 0 && !d_path) return SYNERA_EINVAL;
  if (off4({d_path, d_n_path}) || (reinterpret_cast<uintptr_t>(d_k_pool) | reinterpret_cast<uintptr_t>(d_v_pool)) % 16) return SYNERA_EINVAL;
  const ShLimits& l = t->lim;
  const int64_t layer = (int64_t)t->n_pages * l.Hkv * SY_PAGE * l.hd;
  if (n_layers > 1 && (layer_stride < layer || layer_stride % 8)) return SYNERA_EINVAL;
  const int64_t all = (n_layers > 1 ? (n_layers - 1) * layer_stride : 0) + layer;
  const Range k = {reinterpret_cast<uintptr_t>(d_k_pool), reinterpret_cast<uintptr_t>(d_k_pool) + 2 * (uintptr_t)all};
  const Range v = {reinterpret_cast<uintptr_t>(d_v_pool), reinterpret_cast<uintptr_t>(d_v_pool) + 2 * (uintptr_t)all};
  if (meet(k, v)) return SYNERA_EINVAL;
  if (!rope_device_ok(t->device)) return SYNERA_EINVAL;
  if (t->n_rows == 0 && !capturing(static_cast<hipStream_t>(stream))) return SYNERA_OK;
  const int32_t n = l.Hkv * l.hd;
  CommitArgs a = {t->req, t->slot, d_path, d_n_path, static_cast<bf16_t*>(d_k_pool), static_cast<bf16_t*>(d_v_pool), layer_stride, n, l.hd, (n / 8 + 255) / 256};
  tree_commit_kernel<<<dim3(t->B, n_layers, a.k_parts + (n + 255) / 256), 256, 0, static_cast<hipStream_t>(stream)>>>(a);
  return hipGetLastError() == hipSuccess ? SYNERA_OK : SYNERA_EHIP;
}
