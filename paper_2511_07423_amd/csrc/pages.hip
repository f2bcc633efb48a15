// Block tables and slot maps from request lengths, on the GPU: the pages of each row follow its lengths, from and to a stack of free ones.
#include <algorithm>

#include "../../include/synera.h"
#include "../../include/synera_tree.h"
#include "common.h"

struct PagesArgs {
  const int32_t *ctx, *n_new, *shared;
  int32_t *table, *held, *free_, *n_free, *cu, *pos, *slot, *status;
  int64_t n_rows;
  int32_t B, columns, n_pages;
};
struct PageStep {
  int32_t ctx, rows, held, grow, back, keep, status;         // keep: pages it holds afterwards, if it is not refused
};
__device__ __forceinline__ PageStep page_step(const PagesArgs& a, int i) {
  PageStep s = {0, 0, 0, 0, 0, 0, SYNERA_OK};
  const int32_t n = a.n_new[i];
  s.ctx = a.ctx[i];
  s.held = a.held[i];
  s.rows = n >= 0 && (int64_t)n <= (int64_t)SY_PAGE * a.columns ? n : 0;
  const int64_t keys = (int64_t)s.ctx + n, need = (keys + SY_PAGE - 1) / SY_PAGE;
  if (s.ctx < 0 || n < 0 || keys > 0x7FFFFFFF) s.status = SYNERA_ERANGE;
  else if (s.held < 0 || s.held > a.columns) s.status = SYNERA_EINVAL;
  else if (need > a.columns) s.status = SYNERA_ENOSPC;
  if (s.status != SYNERA_OK) return s;
  const int32_t stay = a.shared ? min(max(a.shared[i], 0), s.held) : 0;
  s.keep = max((int32_t)need, stay);
  s.grow = max(s.keep - s.held, 0);
  s.back = max(s.held - s.keep, 0);
  return s;
}

struct Sum3 { int64_t rows, grow, back; };
// Sums over the threads before this one, and of all.
__device__ __forceinline__ Sum3 scan3(Sum3 v, Sum3* wave_sums, Sum3& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Sum3 in = v;
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t r = __shfl_up(v.rows, o), g = __shfl_up(v.grow, o), b = __shfl_up(v.back, o);
    if (lane >= o) {
      v.rows += r;
      v.grow += g;
      v.back += b;
    }
  }
  __syncthreads();                                           // (the sums of the call before have been read)
  if (lane == 63) wave_sums[wave] = v;
  __syncthreads();
  Sum3 before = {0, 0, 0};
  total = Sum3{0, 0, 0};
  for (int w = 0; w < (int)blockDim.x / 64; ++w) {
    const Sum3 s = wave_sums[w];
    if (w < wave) {
      before.rows += s.rows;
      before.grow += s.grow;
      before.back += s.back;
    }
    total.rows += s.rows;
    total.grow += s.grow;
    total.back += s.back;
  }
  return Sum3{before.rows + v.rows - in.rows, before.grow + v.grow - in.grow, before.back + v.back - in.back};
}

// The n entries of a row and of the stack, from x and y on, that a request moves: a few by its own thread, more by its whole wavefront.
#define PG_FEW 4
__device__ __forceinline__ int64_t lane_value(int64_t v, int lane) {
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane));
}
template <typename F>
__device__ __forceinline__ void each_page(int32_t n, int64_t x, int64_t y, F move) {
  if (n <= PG_FEW)
    for (int c = 0; c < n; ++c) move(x, y, c);
  uint64_t many = __builtin_amdgcn_ballot_w64(n > PG_FEW);
  while (many) {
    const int owner = __builtin_ctzll(many);
    many &= many - 1;
    const int all = __builtin_amdgcn_readlane(n, owner);
    const int64_t ox = lane_value(x, owner), oy = lane_value(y, owner);
    for (int c = threadIdx.x & 63; c < all; c += 64) move(ox, oy, c);
  }
}

// One block.  First what each row takes (from the stack as it was) and where its tokens begin, then, when all have taken theirs, what
// rows return.  Bound by latency: two loads behind each other, three barriers for the sums, the pages.
__device__ __forceinline__ void pages_step(const PagesArgs& a, Sum3* wave_sums, int32_t* taken) {
  const int tid = threadIdx.x;
  const int32_t n_free = min(max(a.n_free[0], 0), a.n_pages);
  Sum3 done = {0, 0, 0};
  if (tid == 0) *taken = 0;
  __syncthreads();
  PageStep s;
  Sum3 at, total;
  for (int i0 = 0; i0 < a.B; i0 += 1024) {
    const int i = i0 + tid;
    s = PageStep{0, 0, 0, 0, 0, 0, SYNERA_OK};
    if (i < a.B) s = page_step(a, i);
    at = scan3(Sum3{s.rows, s.grow, s.back}, wave_sums, total);
    at.rows += done.rows;
    at.grow += done.grow;
    at.back += done.back;
    if (s.grow > 0 && at.grow + s.grow > n_free) s.status = SYNERA_ENOSPC;
    const int32_t takes = s.status == SYNERA_OK ? s.grow : 0;
    each_page(takes, (int64_t)i * a.columns + s.held, n_free - 1 - at.grow, [&](int64_t to, int64_t top, int c) { a.table[to + c] = a.free_[top - c]; });
    if (takes > 0) atomicMax(taken, (int32_t)(at.grow + s.grow));
    if (i < a.B) {
      a.cu[i] = (int32_t)at.rows;
      a.status[i] = s.status;
      if (i == a.B - 1) a.cu[a.B] = (int32_t)(at.rows + s.rows);
    }
    done.rows += total.rows;
    done.grow += total.grow;
    done.back += total.back;
  }
  __syncthreads();                                           // all have taken theirs
  const int64_t left = n_free - *taken;
  const bool one = a.B <= 1024;                              // what this thread knows of its only request is still there
  int64_t back = 0;
  for (int i0 = 0; i0 < a.B; i0 += 1024) {
    const int i = i0 + tid;
    if (!one) {
      s = PageStep{0, 0, 0, 0, 0, 0, SYNERA_OK};
      if (i < a.B) {
        s = page_step(a, i);
        s.status = a.status[i];
      }
      at = scan3(Sum3{0, 0, s.back}, wave_sums, total);
      at.back += back;
      back += total.back;
    }
    each_page(s.status == SYNERA_OK ? s.back : 0, (int64_t)i * a.columns + s.keep, left + done.back - 1 - at.back, [&](int64_t from, int64_t top, int c) {
      if (top - c < a.n_pages) a.free_[top - c] = a.table[from + c];
    });
    if (i < a.B && s.status == SYNERA_OK) a.held[i] = s.keep;
  }
  if (tid == 0) a.n_free[0] = (int32_t)min(left + done.back, (int64_t)a.n_pages);
}

// The places of a request's tokens, by `lanes` threads of which this is number `lane`.
__device__ __forceinline__ void pages_places(const PagesArgs& a, int i, int lane, int lanes) {
  const int32_t first = a.cu[i], rows = a.cu[i + 1] - first, ctx = a.ctx[i];
  const bool ok = a.status[i] == SYNERA_OK;
  for (int j = lane; j < rows; j += lanes) {
    if ((int64_t)first + j >= a.n_rows) break;
    const int32_t p = ctx + j;
    a.pos[first + j] = ok ? p : -1;
    a.slot[first + j] = ok ? a.table[(size_t)i * a.columns + p / SY_PAGE] * SY_PAGE + p % SY_PAGE : -1;
  }
}

// PLACES: the same block writes the tokens' places too.  It writes some 40 GB/s: beyond PG_ROWS tokens a second launch over all requests is shorter.
#define PG_ROWS 4096
template <bool PLACES>
__global__ __launch_bounds__(1024) void pages_kernel(PagesArgs a) {
  __shared__ Sum3 wave_sums[16];
  __shared__ int32_t taken;
  pages_step(a, wave_sums, &taken);
  if constexpr (PLACES) {
    __syncthreads();
    for (int i = threadIdx.x >> 6; i < a.B; i += 16) pages_places(a, i, threadIdx.x & 63, 64);
  }
}
__global__ __launch_bounds__(256) void pages_places_kernel(PagesArgs a) { pages_places(a, blockIdx.x, blockIdx.y * 256 + threadIdx.x, gridDim.y * 256); }

extern "C" int32_t synera_pages_update(int32_t B, const int32_t* d_ctx_len, const int32_t* d_n_new, const int32_t* d_shared, int32_t* d_table,
                                       int32_t columns, int32_t* d_held, int32_t* d_free, int32_t* d_n_free, int32_t n_pages, int64_t n_rows,
                                       int32_t* d_cu, int32_t* d_pos, int32_t* d_slot, int32_t* d_status, void* stream) {
  if (!d_ctx_len || !d_n_new || !d_table || !d_held || !d_free || !d_n_free || !d_cu || !d_status) return SYNERA_EINVAL;
  if (B < 1 || columns < 1 || n_pages < 1 || n_rows < 0 || (n_rows > 0 && (!d_pos || !d_slot))) return SYNERA_EINVAL;
  uintptr_t bits = 0;
  for (const void* p : {(const void*)d_ctx_len, (const void*)d_n_new, (const void*)d_shared, (const void*)d_table, (const void*)d_held, (const void*)d_free,
                        (const void*)d_n_free, (const void*)d_cu, (const void*)d_pos, (const void*)d_slot, (const void*)d_status})
    bits |= reinterpret_cast<uintptr_t>(p);
  if (bits % 4) return SYNERA_EINVAL;
  if (n_pages >= 1 << 27 || (int64_t)B * columns >= (int64_t)1 << 27) return SYNERA_EUNSUP;
  const PagesArgs a = {d_ctx_len, d_n_new, d_shared, d_table, d_held, d_free, d_n_free, d_cu, d_pos, d_slot, d_status, n_rows, B, columns, n_pages};
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (n_rows <= PG_ROWS) {
    pages_kernel<true><<<1, 1024, 0, s>>>(a);
  } else {
    pages_kernel<false><<<1, 1024, 0, s>>>(a);
    if (hipGetLastError() != hipSuccess) return SYNERA_EHIP;
    // (requests of a prompt's length take several blocks)
    pages_places_kernel<<<dim3(B, (uint32_t)std::min<int64_t>(64, std::max<int64_t>(1, n_rows / B / 1024))), 256, 0, s>>>(a);
  }
  return hipGetLastError() == hipSuccess ? SYNERA_OK : SYNERA_EHIP;
}
