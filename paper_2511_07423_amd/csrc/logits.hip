// Penalties for tokens seen before, biases and masks on rows of logits.
#include <algorithm>

#include "../../include/synera.h"
#include "../../include/synera_tree.h"
#include "rope.h"

// A block takes a slice of the vocabulary for some rows of one request.  What is known of a token lies in one word in LDS: how often it was
// generated (bits 0 .. 19), whether it was part of the prompt (20), whether it is on some row's path (21), the last bias entry that names it, from 1
// on (22 .. 31); a bit for each token says that its word is not 0.  They are made from the history once for all rows of the block.  All counts are
// integers, so the order of the atomics does not show.
// Then all values pass as they lie in 16-byte pieces, -infinity in the place of those that the mask hides; those that are allowed and have a word
// are formed on the way.  (Nearly every wavefront meets some: with a branch for each value 2048 x 128256 masked took 325 us; formed behind the
// others, from memory, 300; this way 202, where torch copies these logits in 179 to 197.)
// Paths of trees of up to LG_NODES rows: a mask of the path for each row, and a list of the nodes whose tokens are in the slice.  Rows pass those
// tokens as they are, and behind a barrier each is formed for each row, by a lane that counts it along the list.  (198 trees of 64 nodes in a
// vocabulary of 1096: 68 us; counted on the way, where one lane keeps its wavefront waiting, 323.)  Longer paths are added to the words before a
// row, and taken away where the next row is not behind it.
#define LG_SLICE 8192
#define LG_EVEN 64               // slices are as long as each other: 9 x 64 rows of 9000 to 12000 tokens 17.6 -> 14.9 us
#define LG_THREADS 512
#define LG_PROMPT (1u << 20)
#define LG_SEEN (2 * LG_PROMPT - 1)
#define LG_PATH (1u << 21)
#define LG_BIAS 22
#define LG_MOST_ROWS (1 << 19)   // of calls with paths: counts stay below 2^20
#define LG_NODES 256
#define LG_FIRST (1u << 31)
#define LG_MOST_BIASES 1022
#define LG_EARLY 4               // tokens of the history that a thread asks for together
#define LG_FLY 4                 // 16-byte pieces of a thread on their way together

struct LogitsArgs {
  synera_logits_desc d;
  const void* in;
  void* out;
  int32_t splits;                // blocks that share the rows of a request
  int32_t slice;                 // tokens of a slice, a multiple of LG_EVEN
  bool in_place, once;
};

typedef u32x4 __attribute__((aligned(2))) lg_piece;            // 16 bytes at any address that a type of logits allows

struct LgParams {
  float rho, inv, pres, freq;    // inv: 1 / rho, rounded; x inv is within two half steps of x / rho
  const float* bias;
};
// Without branches: values without a word (w = 0) come out as they are.
__device__ __forceinline__ float lg_adjust(const LgParams& p, float x, uint32_t w) {
  const uint32_t g = w & (LG_PROMPT - 1);
  x *= w & LG_SEEN ? (x > 0.f ? p.inv : p.rho) : 1.f;
  return x - (g ? __builtin_fmaf(p.freq, (float)g, p.pres) : 0.f);
}
__device__ __forceinline__ float lg_bias(const LgParams& p, float x, uint32_t w) {
  const uint32_t entry = w >> LG_BIAS;
  return entry ? x + p.bias[entry - 1] : x;
}

// Value k of a piece, and another in its place.
template <typename T> __device__ __forceinline__ float lg_get(u32x4 v, int k) {
  if constexpr (sizeof(T) == 4) {
    return __uint_as_float(k & 2 ? (k & 1 ? v[3] : v[2]) : (k & 1 ? v[1] : v[0]));
  } else {
    TurnChunk<T, 1> c;
    float f;
    c.p[0] = (uint16_t)((k & 4 ? (k & 2 ? v[3] : v[2]) : (k & 2 ? v[1] : v[0])) >> (16 * (k & 1)));
    c.widen(&f);
    return f;
  }
}
template <typename T> __device__ __forceinline__ u32x4 lg_put(u32x4 v, int k, float f) {
  TurnChunk<T, 1> c;
  c.round(&f);
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int w = 0; w < 4; ++w) v[w] = w == k ? c.p[0] : v[w];
  } else {
    const uint32_t shift = 16 * (k & 1), bits = (uint32_t)c.p[0] << shift, keep = 0xFFFF0000u >> shift;
#pragma unroll
    for (int w = 0; w < 4; ++w) v[w] = w == k / 2 ? (v[w] & keep) | bits : v[w];
  }
  return v;
}

// The bits of a piece as they are where its VEC mask bits are set, -infinity elsewhere.
template <typename T> __device__ __forceinline__ u32x4 lg_masked(u32x4 v, uint32_t bits);
template <> __device__ __forceinline__ u32x4 lg_masked<float>(u32x4 v, uint32_t bits) {
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = (bits >> k) & 1 ? v[k] : 0xFF800000u;
  return v;
}
template <uint32_t NINF>
__device__ __forceinline__ u32x4 lg_masked16(u32x4 v, uint32_t bits) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t low = (bits >> (2 * k)) & 1 ? 0xFFFFu : 0u, high = (bits >> (2 * k)) & 2 ? 0xFFFF0000u : 0u, keep = low | high;
    v[k] = (v[k] & keep) | ((NINF << 16 | NINF) & ~keep);
  }
  return v;
}
template <> __device__ __forceinline__ u32x4 lg_masked<bf16_t>(u32x4 v, uint32_t bits) { return lg_masked16<0xFF80u>(v, bits); }
template <> __device__ __forceinline__ u32x4 lg_masked<_Float16>(u32x4 v, uint32_t bits) { return lg_masked16<0xFC00u>(v, bits); }

// ONCE: the output is marked as not wanted again.
// (6 wavefronts a SIMD: three blocks a compute unit, as many as LDS holds.  Three registers more, spilled: 2048 x 128256 masked 202 -> 220 us.)
template <typename T, bool MASK, bool ONCE>
__global__ __launch_bounds__(LG_THREADS, MASK ? 6 : 4) void logits_kernel(LogitsArgs a) {
  constexpr int VEC = 16 / (int)sizeof(T), PIECES = LG_SLICE / VEC, EACH = PIECES / LG_THREADS, ROWS = LG_FLY / EACH;
  static_assert(EACH >= 1 && ROWS >= 1 && LG_THREADS >= LG_NODES && 2 * LG_THREADS >= LG_MOST_BIASES, "what a thread takes");
  constexpr uint32_t ALL = (1u << VEC) - 1;
  __shared__ __attribute__((aligned(16))) uint32_t word[LG_SLICE];
  __shared__ uint32_t has_word[LG_SLICE / 32];
  __shared__ uint32_t on_path[LG_NODES][LG_NODES / 32 + 1];   // (+ 1: neighbours on other banks)
  __shared__ int32_t parents[LG_NODES];
  __shared__ float given[2 * LG_THREADS];                     // biases
  __shared__ uint32_t listed[LG_NODES];                       // token in the slice | node << 16 | LG_FIRST: the first one of its token
  __shared__ int32_t n_listed;
  __shared__ int32_t held;
  const int tid = threadIdx.x, i = blockIdx.y;
  const int v0 = blockIdx.x * a.slice, n = min(a.slice, (int)a.d.vocab - v0);
  int64_t first = i, rows = 1;
  if (a.d.d_cu) {
    first = min(max((int64_t)a.d.d_cu[i], (int64_t)0), a.d.rows);
    rows = min(max((int64_t)a.d.d_cu[i + 1], first), a.d.rows) - first;
  }
  if (blockIdx.z >= rows) return;
  const int64_t words = (a.d.vocab + 31) / 32;
  const int whole = n / VEC;
  auto in_of = [&](int64_t j) { return static_cast<const T*>(a.in) + (first + j) * a.d.in_stride + v0; };
  auto out_of = [&](int64_t j) { return static_cast<T*>(a.out) + (first + j) * a.d.out_stride + v0; };
  auto mask_of = [&](int64_t j) { return reinterpret_cast<const uint32_t*>(a.d.d_mask) + (first + j) * words + v0 / 32; };
  struct Rows {                                               // pieces of rows j0, j0 + splits, .., `most` of them
    uint32_t bits[ROWS][EACH];
    u32x4 x[ROWS][EACH];
  };
  auto on = [&](int64_t j0, int most, int g, int p) { return g < most && j0 + (int64_t)g * a.splits < rows && tid + p * LG_THREADS < whole; };
  auto load = [&](Rows& r, int64_t j0, int most) {
    if constexpr (MASK) {
#pragma unroll
      for (int g = 0; g < ROWS; ++g)
#pragma unroll
        for (int p = 0; p < EACH; ++p) {
          const int c = tid + p * LG_THREADS;
          r.bits[g][p] = on(j0, most, g, p) ? (mask_of(j0 + (int64_t)g * a.splits)[c * VEC / 32] >> (c * VEC % 32)) & ALL : 0;
        }
    }
#pragma unroll
    for (int g = 0; g < ROWS; ++g)
#pragma unroll
      for (int p = 0; p < EACH; ++p) {
        r.x[g][p] = u32x4{0, 0, 0, 0};
        if (MASK ? r.bits[g][p] != 0 : on(j0, most, g, p))
          r.x[g][p] = reinterpret_cast<const lg_piece*>(in_of(j0 + (int64_t)g * a.splits))[tid + p * LG_THREADS];
      }
  };
  const bool masked_paths = a.d.d_tokens && rows <= LG_NODES, added_paths = a.d.d_tokens && !masked_paths;
  const int most = added_paths ? 1 : ROWS;
  // ---- the first rows, and what the words are made from, are on their way before the barrier behind which LDS is clear
  Rows now;
  load(now, blockIdx.z, most);
  const size_t biases = (size_t)i * a.d.bias_columns;
  const int len = a.d.d_history ? min(max(a.d.d_history_len[i], 0), a.d.history_columns) : 0;
  const int prompt = a.d.d_n_prompt ? a.d.d_n_prompt[i] : 0;
  const int32_t* h = a.d.d_history + (size_t)i * a.d.history_columns;
  int32_t seen[LG_EARLY], named[2], up0 = -1, token0 = -1;
#pragma unroll
  for (int u = 0; u < LG_EARLY; ++u) seen[u] = tid + u * LG_THREADS < len ? h[tid + u * LG_THREADS] : -1;
#pragma unroll
  for (int u = 0; u < 2; ++u) named[u] = a.d.d_bias_id && tid + u * LG_THREADS < a.d.bias_columns ? a.d.d_bias_id[biases + tid + u * LG_THREADS] : -1;
#pragma unroll
  for (int u = 0; u < 2; ++u)
    if (a.d.d_bias_id && tid + u * LG_THREADS < a.d.bias_columns) given[tid + u * LG_THREADS] = a.d.d_bias[biases + tid + u * LG_THREADS];
  if (masked_paths && tid < rows) {
    up0 = a.d.d_parent[first + tid];
    token0 = a.d.d_tokens[first + tid];
    if (up0 >= tid) up0 = -1;
  }
  for (int w = tid; w < (n + 3) / 4; w += LG_THREADS) reinterpret_cast<u32x4*>(word)[w] = u32x4{0, 0, 0, 0};
  if (tid < LG_SLICE / 32) has_word[tid] = 0;
  if (tid == 0) n_listed = 0;
  if (tid < LG_NODES) {
    parents[tid] = up0;
#pragma unroll
    for (int w = 0; w < LG_NODES / 32; ++w) on_path[tid][w] = 0;
  }
  __syncthreads();
  auto slot = [&](int32_t id) { return id < 0 ? 0xFFFFFFFFu : (uint32_t)(id - v0); };      // of a token in the slice: below n
  auto touch = [&](uint32_t t, uint32_t before) {             // by the first one that finds nothing
    if (before == 0) atomicOr(&has_word[t / 32], 1u << (t % 32));
  };
  auto count = [&](int e, int32_t id) {
    const uint32_t t = slot(id);
    if (t < (uint32_t)n) touch(t, e < prompt ? atomicOr(&word[t], LG_PROMPT) : atomicAdd(&word[t], 1u));
  };
#pragma unroll
  for (int u = 0; u < LG_EARLY; ++u) count(tid + u * LG_THREADS, seen[u]);
  for (int e = tid + LG_EARLY * LG_THREADS; e < len; e += LG_EARLY * LG_THREADS) {
#pragma unroll
    for (int u = 0; u < LG_EARLY; ++u) seen[u] = e + u * LG_THREADS < len ? h[e + u * LG_THREADS] : -1;
#pragma unroll
    for (int u = 0; u < LG_EARLY; ++u) count(e + u * LG_THREADS, seen[u]);
  }
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const uint32_t t = slot(named[u]), entry = tid + u * LG_THREADS + 1;
    if (t >= (uint32_t)n) continue;
    uint32_t old = word[t];                                   // counts may come in between
    while (old >> LG_BIAS < entry) {
      const uint32_t was = atomicCAS(&word[t], old, (old & ((1u << LG_BIAS) - 1)) | entry << LG_BIAS);
      if (was == old) {
        touch(t, old);
        break;
      }
      old = was;
    }
  }
  if (masked_paths && tid < rows) {
    const uint32_t t = slot(token0);
    if (t < (uint32_t)n) {
      const uint32_t old = atomicOr(&word[t], LG_PATH);
      touch(t, old);
      listed[atomicAdd(&n_listed, 1)] = t | (uint32_t)tid << 16 | (old & LG_PATH ? 0u : LG_FIRST);
    }
    // The path of each row that this block takes: towards the root node numbers fall, so that its words are written one by one.
    if (tid >= (int)blockIdx.z && (tid - (int)blockIdx.z) % a.splits == 0) {
      uint32_t bits = 1u << (tid % 32);
      int w = tid / 32;
      for (int up = up0; up >= 0; up = parents[up]) {
        if (up / 32 != w) {
          on_path[tid][w] = bits;
          bits = 0;
          w = up / 32;
        }
        bits |= 1u << (up % 32);
      }
      on_path[tid][w] = bits;
    }
  }
  __syncthreads();
  LgParams params = {a.d.d_repetition ? a.d.d_repetition[i] : 1.f, 1.f, a.d.d_presence ? a.d.d_presence[i] : 0.f,
                     a.d.d_frequency ? a.d.d_frequency[i] : 0.f, given};
  params.inv = 1.f / params.rho;
  // ---- the rows
  auto word_of = [&](int t) {                                 // of token t of the slice, 0 where some path has it
    const uint32_t w = word[t];
    return w & LG_PATH ? 0u : w;
  };
  auto finish = [&](const Rows& r, int64_t j0) {
#pragma unroll
    for (int g = 0; g < ROWS; ++g)
#pragma unroll
      for (int p = 0; p < EACH; ++p) {
        if (!on(j0, most, g, p)) continue;
        const int64_t j = j0 + (int64_t)g * a.splits;
        const int c = tid + p * LG_THREADS;
        const uint32_t allowed = MASK ? r.bits[g][p] : ALL;
        u32x4 v = r.x[g][p];
        uint32_t todo = (has_word[c * VEC / 32] >> (c * VEC % 32)) & allowed;
        if (a.in_place && !todo && allowed == ALL) continue;
        // Under a mask few values of a piece are to be formed: one at a time.  Without one, all alike and without branches.  (2048 x 128256 bf16: under a mask
        // that leaves 3 % 202 and 226 us, without a mask 234 and 200; both ways in one kernel take too many registers.)
        if constexpr (MASK) {
          while (todo) {
            const int k = __builtin_ctz(todo);
            todo &= todo - 1;
            const uint32_t w = word_of(c * VEC + k);
            v = lg_put<T>(v, k, lg_bias(params, lg_adjust(params, lg_get<T>(v, k), w), w));
          }
        } else if (todo) {
          uint32_t w[VEC], any = 0;
          float f[VEC];
          TurnChunk<T, VEC> y;
          y.p[0] = v;
          y.widen(f);
#pragma unroll
          for (int k = 0; k < VEC; ++k) any |= w[k] = word_of(c * VEC + k);
#pragma unroll
          for (int k = 0; k < VEC; ++k) f[k] = lg_adjust(params, f[k], w[k]);
          if (any >> LG_BIAS) {
#pragma unroll
            for (int k = 0; k < VEC; ++k) f[k] = lg_bias(params, f[k], w[k]);
          }
          y.round(f);
          v = y.p[0];
        }
        v = MASK ? lg_masked<T>(v, allowed) : v;
        lg_piece* to = reinterpret_cast<lg_piece*>(out_of(j)) + c;
        if constexpr (ONCE) __builtin_nontemporal_store(v, to);
        else *to = v;
      }
    if (whole * VEC < n)                                      // the rows' last values, less than a piece
      for (int g = 0; g < most; ++g) {
        const int64_t j = j0 + (int64_t)g * a.splits;
        const int e = whole * VEC + tid;
        if (j >= rows || e >= n) continue;
        TurnChunk<T, 1> y;
        float f;
        y.load(in_of(j) + e);
        const bool allowed = !MASK || (mask_of(j)[e / 32] >> (e % 32)) & 1;
        const uint32_t w = word_of(e);
        if (w || !allowed) {
          y.widen(&f);
          f = allowed ? lg_bias(params, lg_adjust(params, f, w), w) : -INFINITY;
          y.round(&f);
        }
        y.template store<false>(out_of(j) + e);
      }
  };
  // Long paths, by one thread: the words hold that of node `held`.  If it is an ancestor of the next row, only what lies between is added.
  if (tid == 0) held = -1;
  auto add = [&](int32_t at, uint32_t by) {
    const uint32_t t = slot(a.d.d_tokens[first + at]);
    if (t < (uint32_t)n) {
      word[t] += by;
      has_word[t / 32] |= 1u << (t % 32);
    }
    const int32_t up = a.d.d_parent[first + at];
    return up >= 0 && up < at ? up : -1;
  };
  auto hold = [&](int32_t j) {
    const int32_t before = held;
    int32_t at = j;
    while (at > before) at = add(at, 1u);
    if (at != before) {
      for (int32_t old = before; old >= 0;) old = add(old, ~0u);
      while (at >= 0) at = add(at, 1u);
    }
    held = j;
  };
  for (int64_t j0 = blockIdx.z, step = (int64_t)a.splits * most; j0 < rows; j0 += step) {
    // (the next rows are asked for before these are written where a row is few registers: in 32 bits that takes a block of three off each compute unit)
    Rows next;
    if (VEC == 8 && j0 + step < rows) load(next, j0 + step, most);
    if (added_paths) {
      __syncthreads();
      if (tid == 0) hold((int32_t)j0);
      __syncthreads();
    }
    finish(now, j0);
    if (VEC == 8) now = next;
    else if (j0 + step < rows) load(now, j0 + step, most);
  }
  // ---- the listed tokens, which have passed as they are
  const int n_list = n_listed;
  if (n_list == 0) return;
  __syncthreads();
  const int mine = (int)((rows - blockIdx.z + a.splits - 1) / a.splits);
  for (int e = tid; e < n_list * mine; e += LG_THREADS) {
    const int g = e / n_list;
    const int64_t j = blockIdx.z + (int64_t)g * a.splits;
    const uint32_t own = listed[e - g * n_list];
    const int t = (int)(own & 0xFFFF);
    if (!(own & LG_FIRST) || (MASK && !((mask_of(j)[t / 32] >> (t % 32)) & 1))) continue;
    TurnChunk<T, 1> y;
    float f;
    y.load(in_of(j) + t);
    uint32_t w = word[t] & ~LG_PATH;
    for (int k = 0; k < n_list; ++k) {
      const uint32_t other = listed[k], node = (other >> 16) % LG_NODES;
      if (((other ^ own) & 0xFFFF) == 0) w += (on_path[j][node / 32] >> (node % 32)) & 1;
    }
    y.widen(&f);
    f = lg_bias(params, lg_adjust(params, f, w), w);
    y.round(&f);
    if (w) y.template store<false>(out_of(j) + t);
  }
}

template <typename T>
static void launch_logits(const LogitsArgs& a, dim3 grid, hipStream_t s) {
  if (a.once && a.d.d_mask) logits_kernel<T, true, true><<<grid, LG_THREADS, 0, s>>>(a);
  else if (a.once) logits_kernel<T, false, true><<<grid, LG_THREADS, 0, s>>>(a);
  else if (a.d.d_mask) logits_kernel<T, true, false><<<grid, LG_THREADS, 0, s>>>(a);
  else logits_kernel<T, false, false><<<grid, LG_THREADS, 0, s>>>(a);
}

static bool lg_meet(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && na > 0 && nb > 0 && x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

extern "C" int32_t synera_logits_adjust(const synera_logits_desc* desc, const void* d_in, void* d_out, void* stream) {
  if (!desc) return SYNERA_EINVAL;
  const synera_logits_desc& d = *desc;
  if (d.B < 0 || d.rows < 0 || d.vocab < 1 || d.dtype < 0 || d.dtype > 2) return SYNERA_EINVAL;
  if (d.history_columns < 0 || d.bias_columns < 0) return SYNERA_EINVAL;
  if (!d.d_cu && d.rows != d.B) return SYNERA_EINVAL;
  if ((!d.d_tokens) != (!d.d_parent) || (d.d_tokens && !d.d_cu)) return SYNERA_EINVAL;
  if ((d.d_history && !d.d_history_len) || (!d.d_bias_id) != (!d.d_bias)) return SYNERA_EINVAL;
  if (d.vocab > (int64_t)1 << 30 || d.bias_columns > LG_MOST_BIASES || d.history_columns >= 1 << 19 || d.B > 65535 || d.rows >= (int64_t)1 << 31) return SYNERA_EUNSUP;
  if (d.d_tokens && d.rows > LG_MOST_ROWS) return SYNERA_EUNSUP;
  if (d.rows == 0 || d.B == 0) return SYNERA_OK;
  if (!d_in || !d_out || (d.rows > 1 && (d.in_stride < d.vocab || d.out_stride < d.vocab))) return SYNERA_EINVAL;
  const int size = d.dtype == 0 ? 4 : 2;
  uintptr_t bits = 0;
  const int64_t words = (d.vocab + 31) / 32, B = d.B;
  const struct { const void* p; int64_t n; } arrays[] = {
      {d.d_cu, B + 1}, {d.d_history, B * d.history_columns}, {d.d_history_len, B}, {d.d_n_prompt, B}, {d.d_repetition, B}, {d.d_presence, B},
      {d.d_frequency, B}, {d.d_bias_id, B * d.bias_columns}, {d.d_bias, B * d.bias_columns}, {d.d_mask, d.rows * words}, {d.d_tokens, d.rows}, {d.d_parent, d.rows}};
  const int64_t in_bytes = ((d.rows - 1) * d.in_stride + d.vocab) * size, out_bytes = ((d.rows - 1) * d.out_stride + d.vocab) * size;
  for (const auto& x : arrays) {
    bits |= reinterpret_cast<uintptr_t>(x.p);
    if (lg_meet(d_out, out_bytes, x.p, 4 * x.n)) return SYNERA_EINVAL;
  }
  if (bits % 4 || (reinterpret_cast<uintptr_t>(d_in) | reinterpret_cast<uintptr_t>(d_out)) % size) return SYNERA_EINVAL;
  const bool in_place = d_in == d_out && (d.rows == 1 || d.in_stride == d.out_stride);
  if (!in_place && lg_meet(d_out, out_bytes, d_in, in_bytes)) return SYNERA_EINVAL;
  LogitsArgs a = {d, d_in, d_out, 1, 0, in_place, !in_place && beyond_caches((size_t)(d.rows * d.vocab * size))};
  const int64_t slices = (d.vocab + LG_SLICE - 1) / LG_SLICE, each = (d.rows + B - 1) / B;
  // Blocks that share a request's rows, up to two rounds of three blocks a compute unit: with more, what each makes from the history and the paths costs more
  // than full rounds save (3 x 64 rows of 123964, 1536 and 3968 blocks: 34 and 44 us; 198 x 64 of 1096 68 and 85; 64 x 16 of 32000 41 and 42, 1024: 44).
  a.splits = (int32_t)std::min<int64_t>(std::max<int64_t>(1, std::min<int64_t>(each, 1536 / (slices * B))), 65535);
  a.slice = (int32_t)(((d.vocab + slices - 1) / slices + LG_EVEN - 1) / LG_EVEN * LG_EVEN);
  const dim3 grid((uint32_t)slices, (uint32_t)B, (uint32_t)a.splits);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (d.dtype == 0) launch_logits<float>(a, grid, s);
  else if (d.dtype == 1) launch_logits<bf16_t>(a, grid, s);
  else launch_logits<_Float16>(a, grid, s);
  return hipGetLastError() == hipSuccess ? SYNERA_OK : SYNERA_EHIP;
}
