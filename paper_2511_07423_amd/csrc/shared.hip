// Batches over a paged cache whose pages requests may share: the handle behind synera_batch, the append with the rotation on
// the way, and the attention that reads a shared prefix once for all its requests.  shared_plan.cpp finds the prefixes and
// cuts the work; everything a kernel needs of a plan lies on the device, at addresses that never change, its sizes
// included: a captured launch serves any later plan.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <initializer_list>
#include <new>
#include <type_traits>

#include "../../include/synera_debug.h"
#include "rope.h"
#include "shared.h"

#define SH_STAGES 4            // plans that may run ahead of their uploads
// Blocks of a captured append for each place of the attention (two a compute unit).  One kind, whose plans all fit the caches: a 64-token step 4.5 us,
// in tensors of 3000 rows 5.4 (eager 4.4).  Any plan (33 000 rows): two, 24 prompts of 31 800 tokens 148 us (eager 138), a 64-token step 5.0; four, 148 and 5.1.
#define SH_APPEND_KEPT 4
#define SH_APPEND_ANY 2
#define SH_CONST_AS __attribute__((address_space(4)))

// ------------------------------------------------------------------------------------ the handle
enum { R_HEAD, R_POS, R_SLOT, R_WIN, R_ITEM, R_LIST, R_PAGE, R_JOINED, R_PARTS, N_REGIONS };

struct synera_batch {
  ShLimits lim;
  int device;
  ShPlan plan;                 // sizes of the current plan
  bool planned;
  int32_t n_pages;
  char* dev;                   // regions of a plan, then the partial results
  size_t at[N_REGIONS], room[N_REGIONS];
  float* part_o;               // [part_rows][hd]
  float2* part_ml;             // [part_rows]: softmax reference (exponent-2 domain) and sum
  char* host[SH_STAGES];       // pinned: a plan's regions on their way
  size_t host_bytes;
  hipEvent_t done[SH_STAGES];
  bool pending[SH_STAGES];
  uint64_t plans;
  template <typename T> const T* region(int r) const { return reinterpret_cast<const T*>(dev + at[r]); }
};

static size_t up(size_t v) { return (v + 255) / 256 * 256; }

extern "C" int32_t synera_batch_destroy(synera_batch* b) {
  if (!b) return SYNERA_OK;
  const BesideCaptures beside;
  if (b->dev) (void)hipFree(b->dev);                 // waits for the device: nothing reads the pinned memory from here on
  for (int s = 0; s < SH_STAGES; ++s) {
    if (b->done[s]) (void)hipEventDestroy(b->done[s]);
    if (b->host[s]) (void)hipHostFree(b->host[s]);
  }
  delete b;
  return SYNERA_OK;
}

static hipError_t prepare_attention(int hd);   // once for each device

extern "C" int32_t synera_batch_create(synera_batch** out, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                       int32_t max_batch, int32_t max_tokens, int32_t max_pages) {
  if (!out) return SYNERA_EINVAL;
  *out = nullptr;
  if (n_q_heads < 1 || n_kv_heads < 1 || max_batch < 1 || max_tokens < 1 || max_pages < 1) return SYNERA_EINVAL;
  if ((head_dim != 64 && head_dim != 128) || n_q_heads % n_kv_heads || n_q_heads > 1024) return SYNERA_EUNSUP;
  if ((int64_t)max_tokens * n_q_heads >= (int64_t)1 << 30 || (int64_t)max_batch * max_pages >= (int64_t)1 << 30) return SYNERA_EUNSUP;
  int dev = 0;
  hipDeviceProp_t prop;
  if (hipGetDevice(&dev) != hipSuccess || hipGetDeviceProperties(&prop, dev) != hipSuccess) {
    (void)hipGetLastError();
    return SYNERA_EHIP;
  }
  if (prepare_attention(head_dim) != hipSuccess) {
    (void)hipGetLastError();
    return SYNERA_EHIP;
  }
  synera_batch* b = new (std::nothrow) synera_batch();
  if (!b) return SYNERA_ENOMEM;
  b->device = dev;
  b->planned = false;
  b->plans = 0;
  ShLimits& l = b->lim;
  l.Hq = n_q_heads;
  l.Hkv = n_kv_heads;
  l.hd = head_dim;
  l.max_batch = max_batch;
  l.max_tokens = max_tokens;
  l.max_pages = max_pages;
  l.slots = 2 * std::max(1, prop.multiProcessorCount);
  sh_limits(l);
  const size_t T = (size_t)max_tokens;
  b->room[R_HEAD] = sizeof(ShHeader);
  b->room[R_POS] = b->room[R_SLOT] = T * 4;
  b->room[R_WIN] = (size_t)l.windows * sizeof(ShWindow);
  b->room[R_ITEM] = (size_t)l.items * sizeof(ShItem);
  b->room[R_LIST] = (size_t)l.list * 4;
  b->room[R_PAGE] = (size_t)l.pages * 4;
  b->room[R_JOINED] = T * sizeof(ShJoin);
  b->room[R_PARTS] = (size_t)l.parts * sizeof(ShPart);
  size_t off = 0;
  for (int r = 0; r < N_REGIONS; ++r) {
    b->at[r] = off;
    off += up(b->room[r]);
  }
  b->host_bytes = off;
  const size_t o_po = off, o_ml = o_po + up((size_t)l.part_rows * l.hd * 4), all = o_ml + up((size_t)l.part_rows * 8);
  if (hipMalloc(reinterpret_cast<void**>(&b->dev), all) != hipSuccess) {
    (void)hipGetLastError();
    b->dev = nullptr;
    (void)synera_batch_destroy(b);
    return SYNERA_ENOMEM;
  }
  b->part_o = reinterpret_cast<float*>(b->dev + o_po);
  b->part_ml = reinterpret_cast<float2*>(b->dev + o_ml);
  for (int s = 0; s < SH_STAGES; ++s)
    if (hipHostMalloc(reinterpret_cast<void**>(&b->host[s]), b->host_bytes, hipHostMallocDefault) != hipSuccess ||
        hipEventCreateWithFlags(&b->done[s], hipEventDisableTiming) != hipSuccess) {
      (void)hipGetLastError();
      (void)synera_batch_destroy(b);
      return SYNERA_ENOMEM;
    }
  *out = b;
  return SYNERA_OK;
}

// ------------------------------------------------------------------------------------ planning
// The regions of a plan go from pinned host memory to their places in one launch (a copy command for each took longer than
// all of them together): 8 us for 64 requests' 0.2 MB, 13 for 256 requests behind 8192 shared tokens.  Sizes in 16-byte pieces; regions are
// padded to 256 bytes on both sides.
struct ShUpload {
  const u32x4* from[N_REGIONS];
  u32x4* to[N_REGIONS];
  uint32_t end[N_REGIONS];     // pieces up to here, regions end to end
};
__global__ __launch_bounds__(256) void plan_upload_kernel(ShUpload u) {
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < u.end[N_REGIONS - 1]; i += gridDim.x * 256) {
    uint32_t before = 0;
#pragma unroll
    for (int r = 0; r < N_REGIONS; ++r) {
      if (i >= before && i < u.end[r]) u.to[r][i - before] = u.from[r][i - before];
      before = u.end[r];
    }
  }
}

static bool capturing(hipStream_t s) {
  hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(s, &st) != hipSuccess) {
    (void)hipGetLastError();
    return true;               // the legacy stream while another one is captured: nothing may be launched there
  }
  return st != hipStreamCaptureStatusNone;
}

extern "C" int32_t synera_batch_plan(synera_batch* b, int32_t B, const int32_t* h_ctx_len, const int32_t* h_n_new,
                                     const int32_t* h_block_table, int32_t max_pages, int32_t n_pages_in_pool, void* stream) {
  if (!b) return SYNERA_EINVAL;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const ShLimits& l = b->lim;
  int32_t st = synera_validate_shared(B, h_ctx_len, h_n_new, h_block_table, max_pages, n_pages_in_pool, l.max_batch, l.max_tokens);
  if (st != SYNERA_OK) return st;
  if (max_pages > l.max_pages) return SYNERA_ENOSPC;
  if (!rope_device_ok(b->device) || capturing(s)) return SYNERA_EINVAL;
  ShPlan p;
  try {
    sh_plan(l, B, h_ctx_len, h_n_new, h_block_table, max_pages, p);
  } catch (const std::bad_alloc&) {
    return SYNERA_ENOMEM;
  }
  const void* from[N_REGIONS] = {&p.head, p.tok_pos.data(), p.tok_slot.data(), p.windows.data(), p.items.data(), p.list.data(),
                                 p.pages.data(), p.joined.data(), p.parts.data()};
  const size_t bytes[N_REGIONS] = {sizeof(ShHeader), p.tok_pos.size() * 4, p.tok_slot.size() * 4, p.windows.size() * sizeof(ShWindow),
                                   p.items.size() * sizeof(ShItem), p.list.size() * 4, p.pages.size() * 4, p.joined.size() * sizeof(ShJoin),
                                   p.parts.size() * sizeof(ShPart)};
  bool room = p.part_rows <= l.part_rows;
  for (int r = 0; r < N_REGIONS; ++r) room = room && bytes[r] <= b->room[r];
  if (!room) return SYNERA_ENOMEM;                  // (the capacities cover every plan: sh_limits)
  const int slot = (int)(b->plans % SH_STAGES);
  if (b->pending[slot]) {
    if (hipEventSynchronize(b->done[slot]) != hipSuccess) {
      (void)hipGetLastError();
      return SYNERA_EHIP;
    }
    b->pending[slot] = false;
  }
  ShUpload u;
  uint32_t end = 0;
  size_t off = 0;
  for (int r = 0; r < N_REGIONS; ++r) {
    if (bytes[r]) std::memcpy(b->host[slot] + off, from[r], bytes[r]);
    u.from[r] = reinterpret_cast<const u32x4*>(b->host[slot] + off);
    u.to[r] = reinterpret_cast<u32x4*>(b->dev + b->at[r]);
    off += up(bytes[r]);
    u.end[r] = end += (uint32_t)((bytes[r] + 15) / 16);
  }
  plan_upload_kernel<<<std::min<uint32_t>((end + 255) / 256, 1024), 256, 0, s>>>(u);
  bool ok = hipGetLastError() == hipSuccess;
  ok = hipEventRecord(b->done[slot], s) == hipSuccess && ok;
  b->pending[slot] = true;
  ++b->plans;
  if (!ok) {
    (void)hipGetLastError();
    b->planned = false;
    return SYNERA_EHIP;
  }
  b->plan = std::move(p);
  b->planned = true;
  b->n_pages = n_pages_in_pool;
  return SYNERA_OK;
}

// ------------------------------------------------------------------------------------ append
// Wavefronts take queries' and keys' head groups (rope.h), or the values of one page window: 128 of a token's Hkv hd values for up
// to 16 consecutive tokens, turned in LDS from token-major to the page's [dim][slot] order so that a whole page leaves in
// 16-byte pieces.  In a page that other tokens share only the appended slots are written.  (Values are read as usual where all else is marked,
// turn_setup: marked too, 31 585 tokens 139 -> 153 us.)
// Bound by HBM where there are many tokens: 31 585 of 32 + 2 x 8 heads of 128 (776 MB) 139 us, 5.6 TB/s; a decoding step of 64 tokens 4.8 us.
struct AppendArgs {
  TurnArgs turn;
  const ShHeader* head;
  const ShWindow* windows;
  const void* v;
  int64_t v_ts, v_hs;
  bf16_t* v_layer;
  int32_t n, hd;               // n = Hkv hd
  int32_t v_blocks;            // the first blocks take values, the others heads (append_rows)
  int32_t v_pairs;             // whether two values of v can be loaded together
};

template <typename TI>
__device__ __forceinline__ uint32_t value_pair(const TI* v, bool pairs) {    // two neighbouring values as bf16
  TurnChunk<TI, 2> c;
  float f[2];
  if (pairs) {
    c.load(v);
    c.widen(f);
  } else {
    TurnChunk<TI, 1> c0, c1;
    c0.load(v);
    c1.load(v + 1);
    c0.widen(f);
    c1.widen(f + 1);
  }
  return pack_bf2(f[0], f[1]);
}

template <typename TI, int ONCE>
__device__ __forceinline__ void append_values(const AppendArgs& a, const ShWindow w, const int e0, uint32_t* turn) {
  const int lane = threadIdx.x & 63, e = e0 + 2 * lane;
  const bool on = e < a.n;
  const int head = on ? e / a.hd : 0, dim = on ? e % a.hd : 0;
  const TI* v = static_cast<const TI*>(a.v) + (int64_t)head * a.v_hs + dim;
  bf16_t* dst = a.v_layer + (size_t)w.page * a.n * SY_PAGE + (size_t)e0 * SY_PAGE;
  if (w.s1 - w.s0 == 1) {                       // one token: the shortest way
    const uint32_t x = value_pair(v + (int64_t)w.row * a.v_ts, a.v_pairs);
    if (on) {
      dst[2 * lane * SY_PAGE + w.s0] = (bf16_t)(x & 0xFFFF);
      dst[(2 * lane + 1) * SY_PAGE + w.s0] = (bf16_t)(x >> 16);
    }
    return;
  }
  uint32_t vr[SY_PAGE];
  // (slots that are not covered load a covered one's row: without branches all loads are on their way together)
#pragma unroll
  for (int j = 0; j < SY_PAGE; ++j) vr[j] = value_pair(v + (int64_t)(w.row - w.s0 + min(max(j, w.s0), w.s1 - 1)) * a.v_ts, a.v_pairs);
  // lane's two rows of 16 slots = 16 words; the pieces of 4 words rotate with the lane so that the 16-byte LDS accesses of
  // neighbouring lanes fall on different banks
  uint32_t* mine = turn + lane * 16;
#pragma unroll
  for (int q = 0; q < 4; ++q) {                 // piece q: slots (q & 1) * 8 .. + 7 of dim q >> 1
    u32x4 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t l = vr[(q & 1) * 8 + 2 * i], h = vr[(q & 1) * 8 + 2 * i + 1];
      x[i] = (q >> 1) ? (l >> 16) | (h & 0xFFFF0000u) : (l & 0xFFFFu) | (h << 16);
    }
    *reinterpret_cast<u32x4*>(mine + ((q + (lane >> 1)) & 3) * 4) = x;
  }
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int piece = j * 64 + lane, from = piece >> 2;
    if (e0 + 2 * from >= a.n) continue;
    const u32x4 x = *reinterpret_cast<const u32x4*>(turn + from * 16 + (((piece & 3) + (from >> 1)) & 3) * 4);
    const int slot0 = (piece & 1) * 8;          // the piece's first slot
    bf16_t* to = dst + piece * 8;
    if (slot0 >= w.s0 && slot0 + 8 <= w.s1) {
      if constexpr (ONCE == TURN_ONCE_BOTH) __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(to));
      else *reinterpret_cast<u32x4*>(to) = x;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool l = slot0 + 2 * i >= w.s0 && slot0 + 2 * i < w.s1, h = slot0 + 2 * i + 1 >= w.s0 && slot0 + 2 * i + 1 < w.s1;
        if (l && h) *reinterpret_cast<uint32_t*>(to + 2 * i) = x[i];
        else if (l) to[2 * i] = (bf16_t)(x[i] & 0xFFFF);
        else if (h) to[2 * i + 1] = (bf16_t)(x[i] >> 16);
      }
    }
  }
  __builtin_amdgcn_wave_barrier();              // the next window's values come into the same words
}

template <typename TI, int VEC, int ONCE>
__device__ __forceinline__ void append_rows(const AppendArgs& a, const TurnCols cols, uint32_t (*turn)[64 * 16]) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((int)blockIdx.x < a.v_blocks) {
    const uint32_t slabs = (uint32_t)(a.n + 127) / 128, items = (uint32_t)a.head->n_windows * slabs;
    for (uint32_t i = blockIdx.x * 4 + wave; i < items; i += (uint32_t)a.v_blocks * 4)
      append_values<TI, ONCE>(a, a.windows[i / slabs], (int)(i % slabs) * 128, turn[wave]);
  } else {
    const uint32_t items = (uint32_t)a.head->n_tokens * (uint32_t)cols.n;
    for (uint32_t i = (blockIdx.x - a.v_blocks) * 4 + wave; i < items; i += (gridDim.x - a.v_blocks) * 4)
      turn_item<TI, bf16_t, VEC, true, ONCE>(a.turn, cols, i);
  }
}
// PLAN_KNOWN: an eager launch.  A captured one serves later plans, so how their heads are dealt out goes by the plan that it finds.  PLAN_KEPT: no
// plan that its tensors have room for is marked.  PLAN_ANY: what is marked goes by the plan too, and, since the launch cannot have an item for each
// wavefront of the largest, values and heads are taken from one list, so that both end together.
enum { PLAN_KNOWN, PLAN_KEPT, PLAN_ANY };
template <typename TI, int VEC, int ONCE>
__device__ __forceinline__ void append_listed(const AppendArgs& a, const TurnCols cols, uint32_t (*turn)[64 * 16]) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t slabs = (uint32_t)(a.n + 127) / 128, values = (uint32_t)a.head->n_windows * slabs;
  const uint32_t all = values + (uint32_t)a.head->n_tokens * (uint32_t)cols.n;
  for (uint32_t i = blockIdx.x * 4 + wave; i < all; i += gridDim.x * 4) {
    if (i < values) append_values<TI, ONCE>(a, a.windows[i / slabs], (int)(i % slabs) * 128, turn[wave]);
    else turn_item<TI, bf16_t, VEC, true, ONCE>(a.turn, cols, i - values);
  }
}
template <typename TI, int VEC, int ONCE, int PLAN>
__global__ __launch_bounds__(256) void append_rope_kernel(AppendArgs a) {
  __shared__ __attribute__((aligned(16))) uint32_t turn[4][64 * 16];
  if constexpr (PLAN == PLAN_KNOWN) {
    append_rows<TI, VEC, ONCE>(a, a.turn.cols, turn);
  } else if constexpr (PLAN == PLAN_KEPT) {
    append_rows<TI, VEC, ONCE>(a, turn_cols(a.turn.groups, a.head->n_tokens), turn);
  } else {
    const int32_t T = a.head->n_tokens;
    const TurnCols cols = turn_cols(a.turn.groups, T);
    const int32_t once = turn_once(VEC, (T * a.turn.token_bytes) >> 20, true);
    if (once == TURN_ONCE_BOTH) append_listed<TI, VEC, TURN_ONCE_BOTH>(a, cols, turn);
    else if (once == TURN_ONCE_IN) append_listed<TI, VEC, TURN_ONCE_IN>(a, cols, turn);
    else append_listed<TI, VEC, TURN_KEPT>(a, cols, turn);
  }
}

struct Range { uintptr_t from, to; };
static bool meet(const Range& a, const Range& b) { return a.from < b.to && b.from < a.to; }
static Range heads_range(const void* p, int64_t ts, int64_t hs, int64_t heads, int64_t n, int hd, int bytes) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  return {at, at + (uintptr_t)(((n - 1) * ts + (heads - 1) * hs + hd) * bytes)};
}
static Range pool_range(const synera_batch* b, const void* p) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  return {at, at + (uintptr_t)b->n_pages * b->lim.Hkv * SY_PAGE * b->lim.hd * 2};
}

// Tokens that the checks of a call go by: the plan's; of a captured call, which serves later plans too, as many as all its tensors have room
// for.  -1: a tensor lacks room for the plan at hand.  room: tokens that any plan may bring to these tensors.
static int64_t tokens_to_check(const synera_batch* b, bool graph, std::initializer_list<const synera_heads*> heads, int64_t& room) {
  const int64_t T = b->plan.head.n_tokens;
  room = 0;
  for (const synera_heads* h : heads) {
    if (!h || !h->n_rows) continue;
    if (h->n_rows < T) return -1;
    room = room ? std::min<int64_t>(room, h->n_rows) : h->n_rows;
  }
  const int64_t said = room;
  room = std::min<int64_t>(said ? said : INT64_MAX, b->lim.max_tokens);
  if (!graph) return std::max<int64_t>(T, 1);
  return std::max<int64_t>({T, 1, said ? room : std::min<int64_t>(room, 2)});
}

template <typename TI, int VEC>
static void append_vec(const AppendArgs& a, int plan, uint32_t blocks, hipStream_t s) {
  if constexpr (VEC >= 4) {
    if (plan == PLAN_ANY) return append_rope_kernel<TI, VEC, TURN_KEPT, PLAN_ANY><<<blocks, 256, 0, s>>>(a);
    if (plan == PLAN_KNOWN && a.turn.once == TURN_ONCE_BOTH) return append_rope_kernel<TI, VEC, TURN_ONCE_BOTH, PLAN_KNOWN><<<blocks, 256, 0, s>>>(a);
    if (plan == PLAN_KNOWN && a.turn.once == TURN_ONCE_IN) return append_rope_kernel<TI, VEC, TURN_ONCE_IN, PLAN_KNOWN><<<blocks, 256, 0, s>>>(a);
  }
  if (plan == PLAN_KNOWN) return append_rope_kernel<TI, VEC, TURN_KEPT, PLAN_KNOWN><<<blocks, 256, 0, s>>>(a);
  append_rope_kernel<TI, VEC, TURN_KEPT, PLAN_KEPT><<<blocks, 256, 0, s>>>(a);
}
template <typename TI>
static hipError_t launch_append(const AppendArgs& a, int plan, int vec, uint32_t blocks, hipStream_t s) {
  switch (vec) {
    case 8: append_vec<TI, 8>(a, plan, blocks, s); break;
    case 4: append_vec<TI, 4>(a, plan, blocks, s); break;
    case 2: append_vec<TI, 2>(a, plan, blocks, s); break;
    default: append_vec<TI, 1>(a, plan, blocks, s);
  }
  return hipGetLastError();
}

extern "C" int32_t synera_append_rope(synera_batch* b, const synera_rope* rope, int32_t dtype, const synera_heads* q,
                                      const synera_heads* k, const synera_heads* v, float eps, void* d_k_layer, void* d_v_layer,
                                      void* stream) {
  if (!b || !rope || !k || !v || !d_k_layer || !d_v_layer || dtype < 0 || dtype > 2) return SYNERA_EINVAL;
  if (!b->planned || !(eps >= 0.f) || !std::isfinite(eps)) return SYNERA_EINVAL;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool graph = capturing(s);
  if (b->plan.head.n_tokens == 0 && !graph) return SYNERA_OK;          // (an empty tensor has no address)
  if ((reinterpret_cast<uintptr_t>(d_k_layer) | reinterpret_cast<uintptr_t>(d_v_layer)) % 16) return SYNERA_EINVAL;
  const ShLimits& l = b->lim;
  const int bytes = dtype == 0 ? 4 : 2, hd = l.hd;
  if (rope->desc.head_dim != hd || k->n_heads != l.Hkv || v->n_heads != l.Hkv || (q && q->n_heads != l.Hq)) return SYNERA_EINVAL;
  int64_t room;
  const int64_t n1 = tokens_to_check(b, graph, {q, k, v}, room);
  if (n1 < 0) return SYNERA_EINVAL;
  int32_t st = turn_check(*k, n1, hd, bytes, 2, false);
  if (st == SYNERA_OK) st = turn_check(*v, n1, hd, bytes, 2, false);
  if (st == SYNERA_OK && q) st = turn_check(*q, n1, hd, bytes, 2, true);
  if (st != SYNERA_OK || v->d_gain) return SYNERA_EINVAL;
  // no output lies on an input or on another output; the pools are taken as whole ranges
  const Range pools[2] = {pool_range(b, d_k_layer), pool_range(b, d_v_layer)};
  if (meet(pools[0], pools[1])) return SYNERA_EINVAL;
  for (const synera_heads* i : {k, v, q}) {
    if (!i) continue;
    const Range in = heads_range(i->d_in, i->in_token, i->in_head, i->n_heads, n1, hd, bytes);
    if (meet(in, pools[0]) || meet(in, pools[1])) return SYNERA_EINVAL;
    if (i->d_gain) {
      const Range gain = heads_range(i->d_gain, 0, 0, 1, 1, hd, 2);
      if (meet(gain, pools[0]) || meet(gain, pools[1]) || (q && turn_on_output(*q, n1, hd, 2, i->d_gain, 2 * hd))) return SYNERA_EINVAL;
    }
    if (!q) continue;
    if (i == q && dtype == 1 && q->d_in == q->d_out && (n1 == 1 || q->in_token == q->out_token) && (q->n_heads == 1 || q->in_head == q->out_head)) continue;
    if (turn_overlap(q->d_out, q->out_token, q->out_head, q->n_heads, 2, i->d_in, i->in_token, i->in_head, i->n_heads, bytes, n1, hd))
      return SYNERA_EINVAL;
  }
  if (q) {
    const Range out = heads_range(q->d_out, q->out_token, q->out_head, q->n_heads, n1, hd, 2);
    if (meet(out, pools[0]) || meet(out, pools[1])) return SYNERA_EINVAL;
  }
  if (!rope_device_ok(b->device) || rope->device != b->device) return SYNERA_EINVAL;
  AppendArgs a = {};
  const int64_t T = std::max<int64_t>(b->plan.head.n_tokens, 1);
  const int vec = turn_setup(a.turn, rope, T, q, k, bytes, 2, true, eps);
  a.turn.pos = b->region<int32_t>(R_POS);
  a.turn.slot = b->region<int32_t>(R_SLOT);
  a.turn.k_layer = static_cast<bf16_t*>(d_k_layer);
  a.turn.q.tail = a.turn.k.tail = 1;
  if (dtype == 1 && q && q->d_in == q->d_out && !q->d_gain) a.turn.q.tail = 0;
  a.head = b->region<ShHeader>(R_HEAD);
  a.windows = b->region<ShWindow>(R_WIN);
  a.v = v->d_in;
  a.v_ts = v->in_token;
  a.v_hs = v->in_head;
  a.v_layer = static_cast<bf16_t*>(d_v_layer);
  a.n = l.Hkv * hd;
  a.hd = hd;
  const uint64_t va = reinterpret_cast<uintptr_t>(v->d_in) | (uint64_t)(v->in_token * bytes) | (uint64_t)(v->in_head * bytes);
  a.v_pairs = va % (2 * bytes) == 0;
  // A wavefront for each item: of the plan at hand, or, in a captured call, of the largest that the tensors have room for; but no more than
  // fill the chip a few times, since a small plan finds them all, too.
  const int64_t slabs = (a.n + 127) / 128;
  int64_t v_items = std::max<int64_t>(1, b->plan.head.n_windows * slabs), t_items = T * a.turn.cols.n, most_v = 1 << 16, most = 1 << 20;
  int plan = PLAN_KNOWN;
  if (graph) {
    plan = turn_once(vec, (room * a.turn.token_bytes) >> 20, true) == TURN_KEPT ? PLAN_KEPT : PLAN_ANY;
    v_items = std::min(room, 2 * std::min<int64_t>(l.max_batch, room) + room / SY_PAGE) * slabs;      // (sh_limits)
    t_items = std::min(room * a.turn.groups, std::max<int64_t>(room, 4096));                          // (turn_cols)
    most_v = most = SH_APPEND_KEPT * (int64_t)l.slots;
  }
  a.v_blocks = (int32_t)std::min((v_items + 3) / 4, most_v);
  const uint32_t blocks = (uint32_t)(plan == PLAN_ANY ? SH_APPEND_ANY * (int64_t)l.slots : a.v_blocks + std::min((t_items + 3) / 4, most));
  const hipError_t e = dtype == 0   ? launch_append<float>(a, plan, vec, blocks, s)
                       : dtype == 1 ? launch_append<bf16_t>(a, plan, vec, blocks, s)
                                    : launch_append<_Float16>(a, plan, vec, blocks, s);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    return SYNERA_EHIP;
  }
  return SYNERA_OK;
}

// ------------------------------------------------------------------------------------ attention
//   o = softmax(scale q K^T) V over the keys each row sees, in one pass: p = 2^(c (s - m)), l = sum p, O = sum p V with a reference m of the
//   row that follows its scores upwards, O and l rescaled where it moves; o = O / l.
// An item is up to 128 rows (tokens x G heads of one KV head) against a range of a node's keys, in tiles of 32 keys.
//   * A block takes one, or each of its four wavefronts takes one of up to 32 rows alone (attend<HD, 1, 1>).  In a block's item of up to
//     32 rows the wavefronts take every fourth tile each; up to 64, two take the rows' halves and every second tile; above, each takes
//     32 rows and all tiles.  Wavefronts that split the keys merge through LDS at the end.
//   * Scores are computed transposed, S^T = K Q^T (v_mfma_f32_32x32x16_bf16): a lane then holds 16 keys of one row, so that the
//     statistics are the lane's own but for one exchange with the other half, and, with the rows of the K operand dealt out in
//     the order 0-3, 8-11, 4-7, 12-15 of each page's slots, its probabilities are already the B operand of O^T = V^T P^T.
//   * Pages come by asynchronous copies (no registers, 1 KB an instruction) into rings of five slots, one ring for each group of
//     wavefronts that share keys; a slot holds a page for each wavefront of the group.  80 KB in all: two blocks a compute
//     unit, whose matrix and softmax work overlap.  K chunks are swizzled by slot, V halves by dim on the way in, for
//     LDS reads without bank conflicts.
//   * The probabilities are rounded to bf16 (to nearest), the sum l takes them as they were: 2^-8 of each at most, so the output is off by at most
//     2^-8 of the values' mean magnitude, as much as by its own rounding.  Measured against 64 bits, in root mean square: 0.0018 to 0.0023 of the output,
//     0.0016 to 0.0017 with 32-bit probabilities.  Kept in two terms they would take half as many matrix products again.
// Few rows: bound by HBM.  256 requests of one token behind 8192 shared ones and 64 .. 1024 of their own (405 MB): 83 us, 4.9 TB/s.
// Many rows: by the matrix cores and the softmax's vector instructions, which take turns on a SIMD (97 % of its cycles in all, 53 % the
// matrix cores), at the clock that the power limit leaves: 1620 tokens of 64 heads against 16384 keys 870 us, 1.0 PFLOP/s.
struct SharedAttnArgs {
  const bf16_t* q;
  bf16_t* o;
  int64_t q_ts, q_hs, o_ts, o_hs;
  const bf16_t* k_layer;
  const bf16_t* v_layer;
  const ShHeader* head;
  const ShItem* items;
  const int32_t* list;
  const int32_t* pages;
  const ShJoin* joined;
  const ShPart* parts;
  float* part_o;
  float2* part_ml;
  float* lse;
  float c;                     // scale x log2 e
  float m0;                    // below all scores, and m0 c is finite
  int32_t Hq, Hkv, G;
  int32_t run;                 // groups of blocks of a kind in a row (sh_block)
  int32_t block_groups, wave_groups;   // the plan's, or -1: read on the device (graphs, which serve other plans too)
};

typedef __attribute__((ext_vector_type(8))) int sh_i32x8v;
typedef __attribute__((ext_vector_type(4))) int sh_i32x4v;
typedef __attribute__((ext_vector_type(2))) int sh_i32x2v;
typedef SH_CONST_AS sh_i32x8v sh_i32x8;                      // read with scalar loads

__device__ __forceinline__ float sh_ex2(float x) { return __builtin_amdgcn_exp2f(x); }
// Of lanes l and l ^ 32: swapping the halves of two copies leaves the lower lane's value in one and the upper lane's in the other.
__device__ __forceinline__ float both_max(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float both_sum(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// Asynchronous copies of N kilobytes, global -> LDS (16 bytes a lane; lane i of kilobyte j lands at lds_addr + 1024 j + 16 i), from a
// base in scalar registers and each lane's own offsets.  An instruction's offset counts on both sides.
template <int N>
__device__ __forceinline__ void copy_page(const bf16_t* base, uint32_t o0, uint32_t o1, uint32_t o2, uint32_t o3, uint32_t lds_addr, bool once) {
#define SH_COPY_4(MARK)                                                                                                            \
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5" MARK                                               \
               "\n\tglobal_load_lds_dwordx4 %2, %5 offset:0x400" MARK "\n\tglobal_load_lds_dwordx4 %3, %5 offset:0x800" MARK          \
               "\n\tglobal_load_lds_dwordx4 %4, %5 offset:0xc00" MARK ::"s"(lds_addr), "v"(o0), "v"(o1), "v"(o2), "v"(o3), "s"(base) \
               : "memory", "m0")
#define SH_COPY_2(MARK)                                                                                                            \
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3" MARK                                               \
               "\n\tglobal_load_lds_dwordx4 %2, %3 offset:0x400" MARK ::"s"(lds_addr), "v"(o0), "v"(o1), "s"(base) : "memory", "m0")
  if constexpr (N == 4) {
    if (once) SH_COPY_4(" nt");
    else SH_COPY_4("");
  } else {
    if (once) SH_COPY_2(" nt");
    else SH_COPY_2("");
  }
#undef SH_COPY_4
#undef SH_COPY_2
}
typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;

// At most `n` positions of IPP copies may still be on their way, and this wavefront's LDS reads are done.  USUAL: what n mostly is.
template <int IPP, int USUAL>
__device__ __forceinline__ void wait_positions(int n) {
  if (n >= USUAL) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(USUAL * IPP) : "memory");
  else if (USUAL > 2 && n == 2) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * IPP) : "memory");
  else if (USUAL > 1 && n == 1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(IPP) : "memory");
  else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
}

template <int HD>
__device__ __forceinline__ int sh_swz(int slot) { return HD == 128 ? slot : slot >> 1; }

// WR wavefronts share keys and split the rows, WK groups of them split the keys; WR WK == 1: the wavefront has an item of its own.
template <int HD, int WR, int WK>
__device__ __forceinline__ void attend(const SharedAttnArgs& a, const ShItem& it, const int32_t* first_pages, unsigned char* lds) {
  constexpr int NT = 5, PPT = 4 / WR;                         // slots of a ring; positions of a tile (K a, K b, V a, V b)
  constexpr int PAGE_B = SY_PAGE * HD * 2, SLOT_B = WR * PAGE_B, RING_B = NT * SLOT_B, IPP = PAGE_B / 1024;
  constexpr int KS = HD / 16, DB = HD / 32;
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));                              // (what follows from it is formed for each item, not kept for all of them)
  const int n32 = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = wave % WR, kp = WK == 1 ? 0 : wave / WR;
  const bool leaf = (it.flags & SY_SH_LEAF) != 0;
  const bool once = WR < 4 && (it.flags & SY_SH_ONCE) != 0;   // (four wavefronts' rows are seldom a whole request's)
  const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)lds + wave / WR * RING_B;

  // ---- keys
  const int n_tiles = (it.key_end - it.key_begin + 31) / 32;
  const int my_tiles = (n_tiles - kp + WK - 1) / WK, n_iter = (n_tiles + WK - 1) / WK;
  const int n_pos = my_tiles * PPT;
  const SH_CONST_AS int32_t* pages = reinterpret_cast<const SH_CONST_AS int32_t*>((uintptr_t)(a.pages + it.page));
  const int page0 = it.key_begin / SY_PAGE;
  const size_t page_elems = (size_t)a.Hkv * SY_PAGE * HD, head_at = (size_t)it.kv_head * SY_PAGE * HD;
  // K: 16-byte chunks swizzled by slot (kilobyte j holds 16 / IPP slots on, whose number changes bits 6 and 7 of the offset); V: the
  // 16-byte halves of every second group of 8 dims swapped.  (What follows from one register is formed again in each iteration:
  // kept, it was spilled.)
  const int c_slot = lane / (HD / 8);
  uint32_t k_off = c_slot * HD * 2 + ((lane % (HD / 8)) ^ sh_swz<HD>(c_slot)) * 16;
  const uint32_t v_off = ((lane >> 1) * 2 + ((lane & 1) ^ ((lane >> 4) & 1))) * 16;
  // position p of the ring: pages p WR .. p WR + WR - 1 of the sequence K a, K b, V a, V b of tile 0, of tile 1, ...; this wavefront
  // copies one of them
  auto page_of = [&](int p) {
    const int s = min(p, n_pos - 1) * WR + wr;
    return pages[min(page0 + 2 * ((s >> 2) * WK + kp) + (s & 1), it.n_pages - 1)];
  };
  const SH_CONST_AS int32_t* near = reinterpret_cast<const SH_CONST_AS int32_t*>((uintptr_t)first_pages);
  auto first_page_of = [&](int p) {                           // of the first NT positions: at most page 15 from key_begin on
    const int s = p * WR + wr;
    return near[2 * ((s >> 2) * WK + kp) + (s & 1)];
  };
  auto wrap = [&](uint32_t at) { return at >= RING_B ? at - RING_B : at; };
  int issued = 0;                                             // positions on their way or landed
  uint32_t fill = 0;                                          // where the next one goes in the ring
  auto issue = [&](int32_t page) {
    const uint32_t to = ring + fill + wr * PAGE_B;
    const size_t at = (size_t)(uint32_t)page * page_elems + head_at;
    if (((issued * WR + wr) & 2) == 0) {
      asm volatile("" : "+v"(k_off));
      copy_page<IPP>(a.k_layer + at, k_off, k_off ^ 64, k_off ^ 128, k_off ^ 192, to, once);
    } else {
      copy_page<IPP>(a.v_layer + at, v_off, v_off, v_off, v_off, to, once);
    }
    fill = wrap(fill + SLOT_B);
    ++issued;
  };
#pragma unroll
  for (int p = 0; p < NT; ++p)
    if (p < n_pos) issue(first_page_of(p));

  // ---- rows
  const int row = wr * 32 + n32;
  const int in_node = it.row0 + min(row, it.n_rows - 1);
  const int j_tok = in_node / a.G, head = it.kv_head * a.G + in_node % a.G;
  const int tok = leaf ? it.tok + j_tok : a.list[it.tok + j_tok];
  const int lim = leaf ? it.lim0 + j_tok : 0x7FFFFFFF;        // last key that the row sees
  const int free_end = leaf ? min(it.key_end, it.lim0 + it.row0 / a.G + 1) : it.key_end;   // keys below need no mask
  bf16x8 qf[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(a.q + (int64_t)tok * a.q_ts + (int64_t)head * a.q_hs + 16 * s + 8 * h);

  // All of that has arrived before the loop begins: a load that the compiler has not seen waited for there it would wait for inside,
  // each time, and for the copies with it.
  __builtin_amdgcn_s_waitcnt(0x0F70);                         // vmcnt(0)

  const float c = a.c;
  float m = a.m0, l = 0.f;                                    // m in units of the raw scores
  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[db][r] = 0.f;

  // where this lane reads its K rows (of two pages, behind each other but in the rings of single pages) and V rows
  const int kslot = (n32 & 3) | ((n32 >> 2) & 1) << 3 | ((n32 >> 3) & 1) << 2;
  uint32_t k_at = (WR == 1 ? 0 : (n32 >> 4) * PAGE_B) + kslot * HD * 2 + ((h ^ sh_swz<HD>(kslot)) << 4);
  const uint32_t v_at = n32 * 32 + (h ^ ((n32 >> 3) & 1)) * 16;
  bf16x8 kf[KS], vf[DB][2];
  uint32_t take = 0;                                          // where the tile at hand begins in the ring
  auto page_at = [&](uint32_t tile, int part) {               // its page `part`
    if constexpr (WR == 4) return ring + tile + part * PAGE_B;
    else if constexpr (WR == 2) return ring + wrap(tile + (part >> 1) * SLOT_B) + (part & 1) * PAGE_B;
    else return ring + wrap(tile + part * SLOT_B);
  };
  auto read_k = [&](uint32_t tile) {
    asm volatile("" : "+v"(k_at));
    const uint32_t at = k_at + (WR == 1 ? ((n32 >> 4) ? page_at(tile, 1) : page_at(tile, 0)) : page_at(tile, 0));
#pragma unroll
    for (int s = 0; s < KS; ++s) kf[s] = *(lds_bf16x8*)(uintptr_t)(at ^ (s << 5));      // chunk (2 s + h) ^ swizzle
  };
  auto read_v = [&](uint32_t tile) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint32_t at = page_at(tile, 2 + b) + v_at;
#pragma unroll
      for (int db = 0; db < DB; ++db) vf[db][b] = *(lds_bf16x8*)(uintptr_t)(at + db * 1024);
    }
  };
  auto scores = [&](f32x16& sc) {
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[r] = 0.f;
#pragma unroll
    for (int s = 0; s < KS; ++s) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s], qf[s], sc, 0, 0, 0);
  };
  // A tile's scores (register r: key kb + 16 (r / 8) + 8 h + r % 8) to probabilities; statistics and accumulators brought up.
  auto softmax = [&](f32x16& sc, bf16x8* pf, int kb, auto masked) {
    if constexpr (masked) {
      const int seen = min(it.key_end - 1, lim) - kb - 8 * h;
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[r] = 16 * (r >> 3) + (r & 7) <= seen ? sc[r] : -INFINITY;
    }
    // The reference m only has to keep 2^(c (s - m)) in range.  So no maximum is sought: the probabilities are formed with the m
    // there is, and their sum, which is wanted anyway, tells whether some score is far above it (the first tile, then hardly ever).
    float p[16], t;
    auto form = [&]() {
      const float mc = m * c;
      float t0 = 0.f, t1 = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) p[r] = sh_ex2(fmaf(sc[r], c, -mc));
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        t0 += p[r];
        t1 += p[r + 1];
      }
      t = t0 + t1;
    };
    form();
    if (__builtin_amdgcn_ballot_w64(!(t < 4096.0f)) != 0) {
      float mx = sc[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mx = fmaxf(mx, sc[r]);
      mx = both_max(mx);
      const float m_new = (mx - m) * c > 8.0f ? mx : m;
      const float alpha = sh_ex2((m - m_new) * c);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[db][r] *= alpha;
      form();
    }
    l += t;
#pragma unroll
    for (int b = 0; b < 2; ++b)
      pf[b] = __builtin_bit_cast(bf16x8, make_uint4(pack_bf2(p[8 * b], p[8 * b + 1]), pack_bf2(p[8 * b + 2], p[8 * b + 3]),
                                                    pack_bf2(p[8 * b + 4], p[8 * b + 5]), pack_bf2(p[8 * b + 6], p[8 * b + 7])));
  };
  auto values = [&](const bf16x8* pf, int kb, auto masked) {
    if constexpr (masked) {
      // Keys past the end may hold junk, and 0 x NaN is NaN: they are blanked.  So may keys that only some rows see.
      bool odd = false;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int n = it.key_end - kb - 16 * b - 8 * h;
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          u32x4 w = __builtin_bit_cast(u32x4, vf[db][b]);
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            w[d] &= (2 * d < n ? 0x0000FFFFu : 0u) | (2 * d + 1 < n ? 0xFFFF0000u : 0u);
            odd |= (w[d] & 0x7F80u) == 0x7F80u || (w[d] & 0x7F800000u) == 0x7F800000u;
          }
          vf[db][b] = __builtin_bit_cast(bf16x8, w);
        }
      }
      if (__builtin_amdgcn_ballot_w64(odd) != 0) {            // infinities or NaN among them: key by key, each to the rows that see it
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll 1
          for (int k = 0; k < 16; ++k) {
            const bool seen = kb + 16 * b + k <= lim;
            const uint32_t keep = (k >> 3) == h ? ((k & 1) ? 0xFFFF0000u : 0x0000FFFFu) : 0u;
#pragma unroll
            for (int db = 0; db < DB; ++db) {
              u32x4 w = __builtin_bit_cast(u32x4, vf[db][b]);
#pragma unroll
              for (int d = 0; d < 4; ++d) w[d] &= d == ((k & 7) >> 1) ? keep : 0u;
              f32x16 t;
#pragma unroll
              for (int r = 0; r < 16; ++r) t[r] = 0.f;
              t = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), pf[b], t, 0, 0, 0);
#pragma unroll
              for (int r = 0; r < 16; ++r) acc[db][r] += seen ? t[r] : 0.f;
              __builtin_amdgcn_sched_barrier(0);              // one t at a time
            }
          }
        return;
      }
    }
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int db = 0; db < DB; ++db) acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[db][b], pf[b], acc[db], 0, 0, 0);
  };

  // The tiles that need no mask, then (masked) the last few: the code for hidden keys stays out of the first loop's registers.
  const int free_tiles = max(0, free_end - it.key_begin) / 32;              // of all groups
  const int my_free = min(my_tiles, max(0, (free_tiles - kp + WK - 1) / WK));
  int32_t next[PPT > 1 ? PPT : 2];                            // pages of the positions to be issued next
  if (n_pos > 0) {
#pragma unroll
    for (int q = 0; q < (PPT > 1 ? PPT : 2); ++q) next[q] = page_of(NT + q);
  }
  if constexpr (WR == 1) {
    // No other wavefront touches this ring: K slots are filled again as soon as the scores' operands are in registers.
    auto tile = [&](int i, auto masked) {
      const int kb = it.key_begin + 32 * (i * WK + kp);
      f32x16 sc;
      bf16x8 pf[2];
      wait_positions<IPP, 3>(issued - (4 * i + 2));
      read_k(take);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (issued < n_pos) issue(next[0]);
      if (issued < n_pos) issue(next[1]);
      scores(sc);
      softmax(sc, pf, kb, masked);
      next[0] = page_of(4 * i + 9);
      next[1] = page_of(4 * i + 10);
      wait_positions<IPP, 3>(issued - (4 * i + 4));
      read_v(take);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (issued < n_pos) issue(next[2]);
      if (issued < n_pos) issue(next[3]);
      next[2] = page_of(4 * i + 11);
      next[3] = page_of(4 * i + 12);
      values(pf, kb, masked);
      take = wrap(take + 4 * SLOT_B);
    };
    for (int i = 0; i < my_free; ++i) tile(i, std::false_type());
    for (int i = my_free; i < my_tiles; ++i) tile(i, std::true_type());
  } else {
    // Own copies of the coming N tiles have landed and own reads of the ones before are done; the barrier extends both to the block,
    // so the slots of the ones before may be filled again.
    auto begin = [&](int i, auto n) {
      wait_positions<IPP, 1>(issued - (i + n) * PPT);
      asm volatile("s_barrier" ::: "memory");
#pragma unroll
      for (int q = 0; q < 2; ++q)
        if (issued < min(n_pos, i * PPT + NT)) issue(next[q]);
#pragma unroll
      for (int q = 0; q < 2; ++q) next[q] = page_of(issued + q);
    };
    auto tile = [&](int i, auto masked) {
      begin(i, std::integral_constant<int, 1>());
      const int kb = it.key_begin + 32 * (i * WK + kp);
      f32x16 sc;
      bf16x8 pf[2];
      read_k(take);
      scores(sc);
      read_v(take);
      softmax(sc, pf, kb, masked);
      values(pf, kb, masked);
      take = wrap(take + PPT * SLOT_B);
    };
    int i = 0;
    if constexpr (WR == 4)
      // two tiles at a time: half the barriers, waits and exchanges, and two chains of products to interleave
      for (; i + 2 <= my_free; i += 2) {
        begin(i, std::integral_constant<int, 2>());
        const uint32_t second = wrap(take + SLOT_B);
        f32x16 sc[2];
        bf16x8 pf[2];
        read_k(take);
        scores(sc[0]);
        read_k(second);
        scores(sc[1]);
        read_v(take);
        softmax(sc[0], pf, 0, std::false_type());
        values(pf, 0, std::false_type());
        read_v(second);
        softmax(sc[1], pf, 0, std::false_type());
        values(pf, 0, std::false_type());
        take = wrap(second + SLOT_B);
      }
    else
      for (; i < my_free; ++i) tile(i, std::false_type());
    for (; i < my_tiles; ++i) tile(i, std::true_type());
    if (my_tiles < n_iter) {                                  // the other key group has one tile more: its barrier
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      asm volatile("s_barrier" ::: "memory");
    }
  }

  // ---- wavefronts that split the keys: the first group takes the others' results
  if constexpr (WK > 1) {
    constexpr int WORDS = (DB * 16 + 2) * 64;
    __syncthreads();                                          // every copy has been waited for and every tile read
    float* park = reinterpret_cast<float*>(lds);
    if (kp > 0) {
      float* to = park + ((kp - 1) * WR + wr) * WORDS + lane;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) to[(db * 16 + r) * 64] = acc[db][r];
      to[DB * 16 * 64] = m;
      to[(DB * 16 + 1) * 64] = l;
    }
    __syncthreads();
    if (kp > 0) return;
#pragma unroll
    for (int g = 1; g < WK; ++g) {
      const float* from = park + ((g - 1) * WR + wr) * WORDS + lane;
      const float m1 = from[DB * 16 * 64], l1 = from[(DB * 16 + 1) * 64];
      const float top = fmaxf(m, m1), f0 = sh_ex2((m - top) * c), f1 = sh_ex2((m1 - top) * c);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[db][r] = acc[db][r] * f0 + from[(db * 16 + r) * 64] * f1;
      l = l * f0 + l1 * f1;
      m = top;
    }
  }
  l = both_sum(l);
  if (row >= it.n_rows) return;
  if (it.part < 0) {
    const float inv = 1.0f / l;
    bf16_t* to = a.o + (int64_t)tok * a.o_ts + (int64_t)head * a.o_hs + 4 * h;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *reinterpret_cast<uint2*>(to + db * 32 + 2 * r) = make_uint2(pack_bf2(acc[db][r] * inv, acc[db][r + 1] * inv),
                                                                     pack_bf2(acc[db][r + 2] * inv, acc[db][r + 3] * inv));
    if (a.lse && h == 0) a.lse[(size_t)tok * a.Hq + head] = (m * c + __log2f(l)) * 0.69314718055994531f;
  } else {
    float* to = a.part_o + (size_t)(it.part + row) * HD + 4 * h;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *reinterpret_cast<float4*>(to + db * 32 + 2 * r) = make_float4(acc[db][r], acc[db][r + 1], acc[db][r + 2], acc[db][r + 3]);
    if (h == 0) a.part_ml[it.part + row] = make_float2(m * c, l);
  }
}

__device__ __forceinline__ ShItem item_of(const ShItem* p) {
  const sh_i32x8* at = reinterpret_cast<const sh_i32x8*>((uintptr_t)p);
  const sh_i32x8v w0 = at[0], w1 = at[1];
  return ShItem{w0[0], w0[1], w0[2], w0[3], w0[4], w0[5], w0[6], w0[7], w1[0], w1[1], w1[2]};   // (its pages are looked up where they are)
}

template <int HD>
__global__ __launch_bounds__(256, 2) void shared_attn_kernel(SharedAttnArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int block_groups = a.block_groups >= 0 ? a.block_groups : a.head->block_groups;
  const int wave_groups = a.wave_groups >= 0 ? a.wave_groups : a.head->wave_groups;
  const int n = (block_groups + wave_groups) * SY_SH_DEAL;
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    bool whole;
    const ShItem* at = a.items + sh_block(block_groups, wave_groups, a.run, i, whole);
    if (!whole) at += __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const ShItem it = item_of(at);
    if (it.n_rows > 0) {
      if (!whole) attend<HD, 1, 1>(a, it, at->pages, lds);
      else if (it.n_rows <= 32) attend<HD, 1, 4>(a, it, at->pages, lds);
      else if (it.n_rows <= 64) attend<HD, 2, 2>(a, it, at->pages, lds);
      else attend<HD, 4, 1>(a, it, at->pages, lds);
    }
    __syncthreads();                                          // the next item's copies come into the same LDS
  }
}

// Joins the partial results of rows that several items worked on: o = sum 2^(m_s - M) O_s / sum 2^(m_s - M) l_s.  A thread takes four
// values of one row; FLY partials (no more than the token has, but for the last round) are asked for together, behind two
// dependent scalar loads.  Bound by latency for a step's tokens (256 of 32 heads, 4 or 5 partials: 6.3 us), by the partials' bytes for prompts'
// (1620 of 64 heads, 3 partials, 162 MB: 30 us).
template <int HD, int FLY>
__device__ __forceinline__ void join_token(const SharedAttnArgs& a, const ShJoin& jn, const int head, const int d4) {
  const SH_CONST_AS sh_i32x2v* list = reinterpret_cast<const SH_CONST_AS sh_i32x2v*>((uintptr_t)(a.parts + jn.first));
  const int kh = head / a.G, g = head % a.G;
  float M = -3e38f, l = 0.f;
  float4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < jn.count; s0 += FLY) {
    float2 ml[FLY];
    float4 v[FLY];
    sh_i32x2v part[FLY];                                      // ShPart: row, step
#pragma unroll
    for (int s = 0; s < FLY; ++s) part[s] = list[min(s0 + s, jn.count - 1)];
#pragma unroll
    for (int s = 0; s < FLY; ++s) {
      const size_t at = (size_t)part[s][0] + (size_t)kh * part[s][1] + g;
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
      if (s0 + s < jn.count) {
        const float w = sh_ex2(ml[s].x - M);
        l += ml[s].y * w;
        sum.x += v[s].x * w; sum.y += v[s].y * w; sum.z += v[s].z * w; sum.w += v[s].w * w;
      }
  }
  const float inv = 1.0f / l;
  *reinterpret_cast<uint2*>(a.o + (int64_t)jn.tok * a.o_ts + (int64_t)head * a.o_hs + d4) =
      make_uint2(pack_bf2(sum.x * inv, sum.y * inv), pack_bf2(sum.z * inv, sum.w * inv));
  if (a.lse && d4 == 0) a.lse[(size_t)jn.tok * a.Hq + head] = (M + __log2f(l)) * 0.69314718055994531f;
}

template <int HD>
__global__ __launch_bounds__(256) void shared_join_kernel(SharedAttnArgs a, int n_joined) {
  const int n = n_joined >= 0 ? n_joined : a.head->n_joined;
  const int piece = blockIdx.y * 256 + threadIdx.x;
  if (piece >= a.Hq * (HD / 4)) return;
  const int head = piece / (HD / 4), d4 = piece % (HD / 4) * 4;
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const sh_i32x4v w = *reinterpret_cast<const SH_CONST_AS sh_i32x4v*>((uintptr_t)(a.joined + i));
    const ShJoin jn = {w[0], w[1], w[2], 0};
    if (jn.count <= 2) join_token<HD, 2>(a, jn, head, d4);
    else if (jn.count <= 4) join_token<HD, 4>(a, jn, head, d4);
    else join_token<HD, 8>(a, jn, head, d4);
  }
}

template <int HD>
static constexpr size_t shared_lds() { return (size_t)20 * SY_PAGE * HD * 2; }
template <int HD>
static hipError_t launch_shared(const SharedAttnArgs& a, int blocks, int joined, hipStream_t s) {
  const size_t lds = shared_lds<HD>();
  hipError_t e = hipSuccess;
  if (blocks > 0) shared_attn_kernel<HD><<<std::min(blocks, 1 << 22), 256, lds, s>>>(a);   // a launch has less than 2^32 threads
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (joined > 0) shared_join_kernel<HD><<<dim3(joined, (a.Hq * (HD / 4) + 255) / 256), 256, 0, s>>>(a, a.block_groups < 0 ? -1 : joined);
  return hipGetLastError();
}

static hipError_t prepare_attention(int hd) {
  const void* kernel = hd == 128 ? reinterpret_cast<const void*>(&shared_attn_kernel<128>) : reinterpret_cast<const void*>(&shared_attn_kernel<64>);
  return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)(hd == 128 ? shared_lds<128>() : shared_lds<64>()));
}

extern "C" int32_t synera_shared_attention(synera_batch* b, const synera_heads* q, const void* d_k_layer, const void* d_v_layer,
                                           float scale, float* d_lse, void* stream) {
  if (!b || !q || !d_k_layer || !d_v_layer || !b->planned) return SYNERA_EINVAL;
  if (!std::isfinite(scale) || scale < 0.f) return SYNERA_EINVAL;
  const float c = (scale > 0.f ? scale : 1.0f / sqrtf((float)b->lim.hd)) * 1.4426950408889634f;
  if (!std::isfinite(c)) return SYNERA_EINVAL;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool graph = capturing(s);
  if (b->plan.head.n_tokens == 0 && !graph) return SYNERA_OK;
  if ((reinterpret_cast<uintptr_t>(d_k_layer) | reinterpret_cast<uintptr_t>(d_v_layer)) % 16 || reinterpret_cast<uintptr_t>(d_lse) % 4) return SYNERA_EINVAL;
  const ShLimits& l = b->lim;
  if (q->n_heads != l.Hq) return SYNERA_EINVAL;
  int64_t room;
  const int64_t n1 = tokens_to_check(b, graph, {q}, room);
  if (n1 < 0) return SYNERA_EINVAL;
  if (turn_check(*q, n1, l.hd, 2, 2, true) != SYNERA_OK) return SYNERA_EINVAL;
  if ((reinterpret_cast<uintptr_t>(q->d_in) | (uint64_t)(2 * q->in_token) | (uint64_t)(2 * q->in_head)) % 16) return SYNERA_EINVAL;
  if ((reinterpret_cast<uintptr_t>(q->d_out) | (uint64_t)(2 * q->out_token) | (uint64_t)(2 * q->out_head)) % 8) return SYNERA_EINVAL;
  if (turn_overlap(q->d_out, q->out_token, q->out_head, l.Hq, 2, q->d_in, q->in_token, q->in_head, l.Hq, 2, n1, l.hd)) return SYNERA_EINVAL;
  const Range out = heads_range(q->d_out, q->out_token, q->out_head, l.Hq, n1, l.hd, 2), k = pool_range(b, d_k_layer), v = pool_range(b, d_v_layer);
  if (meet(out, k) || meet(out, v)) return SYNERA_EINVAL;
  if (d_lse) {
    const Range lse = heads_range(d_lse, l.Hq, 1, l.Hq, n1, 1, 4), in = heads_range(q->d_in, q->in_token, q->in_head, l.Hq, n1, l.hd, 2);
    if (meet(lse, k) || meet(lse, v) || meet(lse, out) || meet(lse, in)) return SYNERA_EINVAL;
  }
  if (!rope_device_ok(b->device)) return SYNERA_EINVAL;
  SharedAttnArgs a = {};
  a.q = static_cast<const bf16_t*>(q->d_in);
  a.o = static_cast<bf16_t*>(q->d_out);
  a.q_ts = q->in_token;
  a.q_hs = q->in_head;
  a.o_ts = q->out_token;
  a.o_hs = q->out_head;
  a.k_layer = static_cast<const bf16_t*>(d_k_layer);
  a.v_layer = static_cast<const bf16_t*>(d_v_layer);
  a.head = b->region<ShHeader>(R_HEAD);
  a.items = b->region<ShItem>(R_ITEM);
  a.list = b->region<int32_t>(R_LIST);
  a.pages = b->region<int32_t>(R_PAGE);
  a.joined = b->region<ShJoin>(R_JOINED);
  a.parts = b->region<ShPart>(R_PARTS);
  a.part_o = b->part_o;
  a.part_ml = b->part_ml;
  a.lse = d_lse;
  a.c = c;
  a.m0 = a.c > 1.f ? -3e38f / a.c : -3e38f;
  a.Hq = l.Hq;
  a.Hkv = l.Hkv;
  a.G = l.Hq / l.Hkv;
  // A captured call serves plans of any size: both launches are made, for as much as may come; the kernels loop.
  const ShHeader& head = b->plan.head;
  a.run = std::max(1, l.slots / 2 / SY_SH_DEAL);
  a.block_groups = graph ? -1 : head.block_groups;
  a.wave_groups = graph ? -1 : head.wave_groups;
  int blocks = (head.block_groups + head.wave_groups) * SY_SH_DEAL;
  if (graph) blocks = std::max(blocks, l.slots);
  const int joined = graph ? std::min(l.max_tokens, std::max(head.n_joined, l.slots)) : head.n_joined;
  const hipError_t e = l.hd == 128 ? launch_shared<128>(a, blocks, joined, s) : launch_shared<64>(a, blocks, joined, s);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    return SYNERA_EHIP;
  }
  return SYNERA_OK;
}

// ------------------------------------------------------------------------------------ test hook
extern "C" int32_t synera_debug_shared_plan(int32_t n_q_heads, int32_t n_kv_heads, int32_t slots, int32_t max_tokens, int32_t B,
                                            const int32_t* h_ctx_len, const int32_t* h_n_new, const int32_t* h_block_table, int32_t max_pages,
                                            int32_t which, int32_t* h_out, int64_t cap, int64_t* n_words, int64_t* limits) {
  if (!h_ctx_len || !h_n_new || !h_block_table || !n_words || (cap > 0 && !h_out) || B < 1 || slots < 1 || max_tokens < 1 || max_pages < 1 ||
      n_kv_heads < 1 || n_q_heads < 1 || n_q_heads % n_kv_heads || which < 0 || which >= N_REGIONS)
    return SYNERA_EINVAL;
  int64_t tokens = 0;
  for (int i = 0; i < B; ++i) {                      // what the planner reads lies inside the table; page ids are only passed on
    const int64_t end = (int64_t)h_ctx_len[i] + h_n_new[i];
    if (h_ctx_len[i] < 0 || h_n_new[i] < 0 || end > INT32_MAX - SY_SH_STEP || end > (int64_t)max_pages * SYNERA_PAGE_SIZE) return SYNERA_EINVAL;
    tokens += h_n_new[i];
  }
  if (tokens > max_tokens) return SYNERA_EINVAL;
  try {
    ShLimits l = {};
    l.Hq = n_q_heads;
    l.Hkv = n_kv_heads;
    l.hd = 128;
    l.max_batch = B;
    l.max_tokens = max_tokens;
    l.max_pages = max_pages;
    l.slots = slots;
    sh_limits(l);
    if (limits) {
      const int64_t v[7] = {l.items, l.list, l.parts, l.pages, l.windows, l.part_rows, l.shared_rows};
      std::memcpy(limits, v, sizeof v);
    }
    ShPlan p;
    sh_plan(l, B, h_ctx_len, h_n_new, h_block_table, max_pages, p);
    const void* from[N_REGIONS] = {&p.head, p.tok_pos.data(), p.tok_slot.data(), p.windows.data(), p.items.data(), p.list.data(),
                                   p.pages.data(), p.joined.data(), p.parts.data()};
    const size_t words[N_REGIONS] = {sizeof(ShHeader) / 4, p.tok_pos.size(), p.tok_slot.size(), p.windows.size() * 4, p.items.size() * 32,
                                     p.list.size(), p.pages.size(), p.joined.size() * 4, p.parts.size() * 2};
    *n_words = (int64_t)words[which];
    if ((int64_t)words[which] > cap) return SYNERA_ENOSPC;
    if (words[which]) std::memcpy(h_out, from[which], words[which] * 4);
    return SYNERA_OK;
  } catch (const std::bad_alloc&) {
    return SYNERA_ENOMEM;
  }
}

extern "C" int32_t synera_debug_shared_block(int32_t block_groups, int32_t wave_groups, int32_t run, int32_t block, int32_t* item) {
  if (!item || block_groups < 0 || wave_groups < 0 || run < 1 || block < 0 || block / SY_SH_DEAL >= block_groups + wave_groups) return SYNERA_EINVAL;
  bool whole;
  *item = sh_block(block_groups, wave_groups, run, block, whole);
  return SYNERA_OK;
}
