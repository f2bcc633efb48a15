// Block tables and slot maps from request lengths, on the GPU: the pages of each row follow its lengths, from and to a stack of free ones.
#include <algorithm>

#include "../../include/synera.h"
#include "../../include/synera_tree.h"
#include "common.h"

#define PG_THREADS 1024
#define PG_ROWS 4096
#define PG_BLOCKS (1 << 20)      // of the second launch for requests, which may be more than a launch's threads

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

// (B x columns stays below 2^27: tokens, pages taken and pages returned of all requests fit 32 bits)
struct Sum3 { int32_t rows, grow, back; };
// Sums over the threads before this one, and of all.
__device__ __forceinline__ Sum3 scan3(const Sum3 in, Sum3* wave_sums, Sum3& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Sum3 v = in;
  for (int o = 1; o < 64; o <<= 1) {
    const int32_t r = __shfl_up(v.rows, o), g = __shfl_up(v.grow, o), b = __shfl_up(v.back, o);
    if (lane >= o) {
      v.rows += r;
      v.grow += g;
      v.back += b;
    }
  }
  __syncthreads();                                           // (the sums of the call before have been read)
  if (lane == 63) wave_sums[wave] = v;
  __syncthreads();
  total = Sum3{0, 0, 0};
  Sum3 before = {0, 0, 0};
#pragma unroll
  for (int w = 0; w < PG_THREADS / 64; ++w) {
    const Sum3 s = wave_sums[w];
    if (w == wave) before = total;
    total.rows += s.rows;
    total.grow += s.grow;
    total.back += s.back;
  }
  return Sum3{before.rows + v.rows - in.rows, before.grow + v.grow - in.grow, before.back + v.back - in.back};
}

struct PageLds {
  Sum3 wave_sums[PG_THREADS / 64];
  int32_t begin[PG_THREADS + 1];   // where each request's pages, or tokens, begin in what all of them move
  int32_t at[PG_THREADS];          // the first column that it moves, or its context, -1 where it is refused
  int32_t taken;
};
// The request among PG_THREADS whose part holds entry k.
__device__ __forceinline__ int request_of(const int32_t* begin, int32_t k) {
  int r = 0;
#pragma unroll
  for (int o = PG_THREADS / 2; o; o /= 2)
    if (begin[r + o] <= k) r += o;
  return r;
}

// One block.  First what each row takes (from the stack as it was) and where its tokens begin, then, when all have taken theirs, what
// rows return.  Pages are dealt out to the threads one by one, whichever request they are of: entry k of all is looked up among the
// prefix sums.  (By the requests' own wavefronts, 1024 requests of up to 32 pages took 17 us.)  Bound by latency: the lengths, three barriers for the sums, a
// search of ten steps in LDS, the pages.
__device__ __forceinline__ void pages_step(const PagesArgs& a, PageLds& l, PageStep& s, Sum3& at) {
  const int tid = threadIdx.x;
  const int32_t n_free = min(max(a.n_free[0], 0), a.n_pages);
  Sum3 done = {0, 0, 0}, total;
  if (tid == 0) l.taken = 0;
  for (int i0 = 0; i0 < a.B; i0 += PG_THREADS) {
    const int i = i0 + tid;
    s = PageStep{0, 0, 0, 0, 0, 0, SYNERA_OK};
    if (i < a.B) s = page_step(a, i);
    at = scan3(Sum3{s.rows, s.grow, s.back}, l.wave_sums, total);
    at.rows += done.rows;
    at.back += done.back;
    // (requests that the stack does not cover come behind all that it does)
    if (s.grow > 0 && done.grow + at.grow + s.grow > n_free) s.status = SYNERA_ENOSPC;
    l.begin[tid] = at.grow;
    l.at[tid] = s.held;
    if (s.grow > 0 && s.status == SYNERA_OK) atomicMax(&l.taken, done.grow + at.grow + s.grow);
    if (i < a.B) {
      a.cu[i] = at.rows;
      a.status[i] = s.status;
      if (i == a.B - 1) a.cu[a.B] = at.rows + s.rows;
    }
    __syncthreads();
    for (int k = tid; k < min(total.grow, l.taken - done.grow); k += PG_THREADS) {
      const int r = request_of(l.begin, k);
      a.table[(size_t)(i0 + r) * a.columns + l.at[r] + (k - l.begin[r])] = a.free_[n_free - 1 - done.grow - k];
    }
    done.rows += total.rows;
    done.grow += total.grow;
    done.back += total.back;
  }
  __syncthreads();                                           // all have taken theirs
  const int32_t left = n_free - l.taken;
  const bool one = a.B <= PG_THREADS;                        // what this thread knows of its only request is still there
  int32_t back = 0;
  for (int i0 = 0; i0 < a.B; i0 += PG_THREADS) {
    const int i = i0 + tid;
    Sum3 mine = {0, 0, at.back};
    if (one) {
      total = done;
    } else {
      s = PageStep{0, 0, 0, 0, 0, 0, SYNERA_OK};
      if (i < a.B) {
        s = page_step(a, i);
        s.status = a.status[i];
      }
      mine = scan3(Sum3{0, 0, s.back}, l.wave_sums, total);  // (a row that returns pages is never refused for want of them)
    }
    l.begin[tid] = mine.back;
    l.at[tid] = s.keep;
    __syncthreads();
    for (int k = tid; k < total.back; k += PG_THREADS) {
      const int r = request_of(l.begin, k);
      const int64_t to = (int64_t)left + done.back - 1 - back - k;
      if (to < a.n_pages) a.free_[to] = a.table[(size_t)(i0 + r) * a.columns + l.at[r] + (k - l.begin[r])];
    }
    if (i < a.B && s.status == SYNERA_OK) a.held[i] = s.keep;
    back += total.back;
    __syncthreads();
  }
  if (tid == 0) a.n_free[0] = (int32_t)min((int64_t)left + done.back, (int64_t)a.n_pages);
}

// PLACES: the same block writes the tokens' places too (of up to PG_THREADS requests).  It writes some 40 GB/s: beyond PG_ROWS tokens a second launch over
// all requests is shorter.
template <bool PLACES>
__global__ __launch_bounds__(PG_THREADS) void pages_kernel(PagesArgs a) {
  __shared__ PageLds l;
  PageStep s;
  Sum3 at;
  pages_step(a, l, s, at);
  if constexpr (PLACES) {
    const int tid = threadIdx.x;
    l.begin[tid] = at.rows;
    l.at[tid] = s.status == SYNERA_OK ? s.ctx : -1;
    if (tid == PG_THREADS - 1) l.begin[PG_THREADS] = at.rows + s.rows;
    __syncthreads();
    const int32_t rows = (int32_t)min((int64_t)l.begin[PG_THREADS], a.n_rows);
    for (int t = tid; t < a.n_rows; t += PG_THREADS) {
      if (t >= rows) {
        a.pos[t] = a.slot[t] = -1;
        continue;
      }
      const int r = request_of(l.begin, t);
      const int32_t ctx = l.at[r], p = ctx + t - l.begin[r];
      a.pos[t] = ctx < 0 ? -1 : p;
      a.slot[t] = ctx < 0 ? -1 : a.table[(size_t)r * a.columns + p / SY_PAGE] * SY_PAGE + p % SY_PAGE;
    }
  }
}
__global__ __launch_bounds__(256) void pages_places_kernel(PagesArgs a) {
  for (int i = blockIdx.x; i < a.B; i += gridDim.x) {
    const int32_t first = a.cu[i], rows = a.cu[i + 1] - first, ctx = a.ctx[i];
    const bool ok = a.status[i] == SYNERA_OK;
    for (int j = blockIdx.y * 256 + threadIdx.x; j < rows && (int64_t)first + j < a.n_rows; j += gridDim.y * 256) {
      const int32_t p = ctx + j;
      a.pos[first + j] = ok ? p : -1;
      a.slot[first + j] = ok ? a.table[(size_t)i * a.columns + p / SY_PAGE] * SY_PAGE + p % SY_PAGE : -1;
    }
  }
  // rows behind the last token, dealt to all blocks
  const int64_t step = (int64_t)gridDim.x * gridDim.y * 256;
  for (int64_t t = a.cu[a.B] + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x; t < a.n_rows; t += step) a.pos[t] = a.slot[t] = -1;
}

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
  // what is written lies on nothing else
  const struct { const void* p; int64_t n; } all[11] = {{d_table, (int64_t)B * columns}, {d_held, B}, {d_free, n_pages}, {d_n_free, 1}, {d_cu, (int64_t)B + 1},
                                                        {d_pos, n_rows}, {d_slot, n_rows}, {d_status, B}, {d_ctx_len, B}, {d_n_new, B}, {d_shared, B}};
  for (int i = 0; i < 8; ++i)
    for (int k = i + 1; k < 11; ++k) {
      const uintptr_t x = reinterpret_cast<uintptr_t>(all[i].p), y = reinterpret_cast<uintptr_t>(all[k].p);
      if (x && y && x < y + 4 * (uintptr_t)all[k].n && y < x + 4 * (uintptr_t)all[i].n) return SYNERA_EINVAL;
    }
  const PagesArgs a = {d_ctx_len, d_n_new, d_shared, d_table, d_held, d_free, d_n_free, d_cu, d_pos, d_slot, d_status, n_rows, B, columns, n_pages};
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (n_rows > 0 && n_rows <= PG_ROWS && B <= PG_THREADS) {
    pages_kernel<true><<<1, PG_THREADS, 0, s>>>(a);
  } else {
    pages_kernel<false><<<1, PG_THREADS, 0, s>>>(a);
    if (hipGetLastError() != hipSuccess) return SYNERA_EHIP;
    if (n_rows == 0) return SYNERA_OK;
    // (requests of a prompt's length take several blocks)
    pages_places_kernel<<<dim3(std::min(B, PG_BLOCKS), (uint32_t)std::min<int64_t>(64, std::max<int64_t>(1, n_rows / B / 1024))), 256, 0, s>>>(a);
  }
  return hipGetLastError() == hipSuccess ? SYNERA_OK : SYNERA_EHIP;
}
