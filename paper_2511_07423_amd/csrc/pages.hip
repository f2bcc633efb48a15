// Block tables and slot maps from request lengths, on the GPU: the pages of each row follow its lengths, from and to a stack of free ones.
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

// One block.  First what each row takes (from the stack as it was) and where its tokens begin, then, when all have taken theirs, what
// rows return, then the tokens' places.
__global__ __launch_bounds__(1024) void pages_kernel(PagesArgs a) {
  __shared__ Sum3 wave_sums[16];
  const int tid = threadIdx.x;
  const int32_t n_free = min(max(a.n_free[0], 0), a.n_pages);
  Sum3 done = {0, 0, 0};
  __shared__ int32_t taken;
  if (tid == 0) taken = 0;
  __syncthreads();
  int64_t all_back = 0;
  for (int i0 = 0; i0 < a.B; i0 += 1024) {
    const int i = i0 + tid;
    PageStep s = {0, 0, 0, 0, 0, 0, SYNERA_OK};
    if (i < a.B) s = page_step(a, i);
    Sum3 total;
    Sum3 at = scan3(Sum3{s.rows, s.grow, s.back}, wave_sums, total);
    at.rows += done.rows;
    at.grow += done.grow;
    if (i < a.B) {
      if (s.grow > 0 && at.grow + s.grow > n_free) s.status = SYNERA_ENOSPC;
      if (s.status == SYNERA_OK && s.grow > 0) {
        for (int c = 0; c < s.grow; ++c) a.table[(size_t)i * a.columns + s.held + c] = a.free_[n_free - 1 - (int32_t)(at.grow + c)];
        atomicMax(&taken, (int32_t)(at.grow + s.grow));
      }
      a.cu[i] = (int32_t)at.rows;
      a.status[i] = s.status;
      if (i == a.B - 1) a.cu[a.B] = (int32_t)(at.rows + s.rows);
    }
    done.rows += total.rows;
    done.grow += total.grow;
    all_back += total.back;
  }
  __syncthreads();
  const int32_t left = n_free - taken;
  int64_t back = 0;
  for (int i0 = 0; i0 < a.B; i0 += 1024) {
    const int i = i0 + tid;
    PageStep s = {0, 0, 0, 0, 0, 0, SYNERA_OK};
    if (i < a.B) s = page_step(a, i);
    Sum3 total;
    const Sum3 at = scan3(Sum3{0, 0, s.back}, wave_sums, total);
    if (i < a.B && a.status[i] == SYNERA_OK) {
      for (int c = 0; c < s.back; ++c) {
        const int64_t to = left + all_back - 1 - (back + at.back + c);
        if (to < a.n_pages) a.free_[to] = a.table[(size_t)i * a.columns + s.keep + c];
      }
      a.held[i] = s.keep;
    }
    back += total.back;
  }
  if (tid == 0) a.n_free[0] = (int32_t)min(left + all_back, (int64_t)a.n_pages);
  __syncthreads();
  const int wave = tid >> 6, lane = tid & 63;
  for (int i = wave; i < a.B; i += 16) {
    const int32_t first = a.cu[i], rows = a.cu[i + 1] - first, ctx = a.ctx[i];
    const bool ok = a.status[i] == SYNERA_OK;
    for (int j = lane; j < rows; j += 64) {
      if ((int64_t)first + j >= a.n_rows) break;
      const int32_t p = ctx + j;
      a.pos[first + j] = ok ? p : -1;
      a.slot[first + j] = ok ? a.table[(size_t)i * a.columns + p / SY_PAGE] * SY_PAGE + p % SY_PAGE : -1;
    }
  }
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
  const PagesArgs a = {d_ctx_len, d_n_new, d_shared, d_table, d_held, d_free, d_n_free, d_cu, d_pos, d_slot, d_status, n_rows, B, columns, n_pages};
  pages_kernel<<<1, 1024, 0, static_cast<hipStream_t>(stream)>>>(a);
  return hipGetLastError() == hipSuccess ? SYNERA_OK : SYNERA_EHIP;
}
