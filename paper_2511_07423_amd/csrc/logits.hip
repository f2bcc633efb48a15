// Penalties for tokens seen before, biases and masks on rows of logits.
#include <algorithm>

#include "../../include/synera.h"
#include "../../include/synera_tree.h"
#include "rope.h"

// A block takes a slice of the vocabulary for some rows of one request.  What is known of a token lies in one word in LDS: how often it was
// generated (bits 0 .. 19), whether it was part of the prompt (20), the last bias entry that names it, from 1 on (21 .. 31).  The words are
// made from the history once for all rows of the block; a row's path is added before the row and taken away behind it.  All counts are integers,
// so the order of the atomics does not show.  A bit for each 16 bytes of logits says whether any of their words may be set: what has none and is
// allowed passes as it is, without a conversion.
#define LG_SLICE 8192
#define LG_PROMPT (1u << 20)
#define LG_SEEN (2 * LG_PROMPT - 1)
#define LG_BIAS 21
#define LG_MOST_STEPS 65536      // of a path
#define LG_NODES 512             // of a tree whose parents and tokens are read once, into LDS
#define LG_FLY 4                 // 16-byte pieces of a thread on their way together

struct LogitsArgs {
  synera_logits_desc d;
  const void* in;
  void* out;
  int32_t splits;                // blocks that share the rows of a request
  bool in_place;
};

template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) LgBits {   // 16 bytes at any address that T allows
  u32x4 v;
};

struct LgParams {
  float rho, pres, freq;
  const float* bias;
};
__device__ __forceinline__ float lg_adjust(const LgParams& p, float x, uint32_t w) {
  if (w & LG_SEEN) x = x > 0.f ? x / p.rho : x * p.rho;
  const uint32_t g = w & (LG_PROMPT - 1);
  if (g) x -= __builtin_fmaf(p.freq, (float)g, p.pres);
  const uint32_t entry = w >> LG_BIAS;
  if (entry) x += p.bias[entry - 1];
  return x;
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

template <typename T, bool MASK>
__global__ __launch_bounds__(256) void logits_kernel(LogitsArgs a) {
  constexpr int VEC = 16 / (int)sizeof(T), PIECES = LG_SLICE / VEC;
  constexpr uint32_t ALL = (1u << VEC) - 1;
  typedef LgBits<T> Bits;
  __shared__ __attribute__((aligned(16))) uint32_t word[LG_SLICE];
  __shared__ uint32_t maybe[PIECES / 32];
  __shared__ int32_t node_token[LG_NODES], node_parent[LG_NODES];
  const int tid = threadIdx.x, i = blockIdx.y;
  const int v0 = blockIdx.x * LG_SLICE, n = min(LG_SLICE, (int)a.d.vocab - v0);
  int64_t first = i, rows = 1;
  if (a.d.d_cu) {
    first = min(max((int64_t)a.d.d_cu[i], (int64_t)0), a.d.rows);
    rows = min(max((int64_t)a.d.d_cu[i + 1], first), a.d.rows) - first;
  }
  if (blockIdx.z >= rows) return;
  // ---- the words
  auto mark = [&](uint32_t t) { atomicOr(&maybe[t / VEC / 32], 1u << (t / VEC % 32)); };
  for (int w = tid; w < (n + 3) / 4; w += 256) reinterpret_cast<u32x4*>(word)[w] = u32x4{0, 0, 0, 0};
  if (tid < PIECES / 32) maybe[tid] = 0;
  const bool staged = a.d.d_tokens && rows <= LG_NODES;
  if (staged)
    for (int t = tid; t < (int)rows; t += 256) {
      node_token[t] = a.d.d_tokens[first + t];
      node_parent[t] = a.d.d_parent[first + t];
    }
  __syncthreads();
  if (a.d.d_bias_id) {
    for (int e = tid; e < a.d.bias_columns; e += 256) {
      const uint32_t t = (uint32_t)(a.d.d_bias_id[(size_t)i * a.d.bias_columns + e] - v0);
      if (t < (uint32_t)n) {
        atomicMax(&word[t], (uint32_t)(e + 1) << LG_BIAS);
        mark(t);
      }
    }
    __syncthreads();
  }
  if (a.d.d_history) {
    const int len = min(max(a.d.d_history_len[i], 0), a.d.history_columns);
    const int prompt = a.d.d_n_prompt ? a.d.d_n_prompt[i] : 0;
    const int32_t* h = a.d.d_history + (size_t)i * a.d.history_columns;
    auto count = [&](int e, int32_t id) {
      const uint32_t t = (uint32_t)(id - v0);
      if (t >= (uint32_t)n) return;
      if (e < prompt) atomicOr(&word[t], LG_PROMPT);
      else atomicAdd(&word[t], 1u);
      mark(t);
    };
    int e = tid;
    for (; e + 3 * 256 < len; e += 4 * 256) {
      const int32_t t0 = h[e], t1 = h[e + 256], t2 = h[e + 512], t3 = h[e + 768];
      count(e, t0);
      count(e + 256, t1);
      count(e + 512, t2);
      count(e + 768, t3);
    }
    for (; e < len; e += 256) count(e, h[e]);
    __syncthreads();
  }
  const LgParams params = {a.d.d_repetition ? a.d.d_repetition[i] : 1.f, a.d.d_presence ? a.d.d_presence[i] : 0.f,
                           a.d.d_frequency ? a.d.d_frequency[i] : 0.f, a.d.d_bias + (size_t)i * a.d.bias_columns};
  // ---- the rows
  for (int64_t j = blockIdx.z; j < rows; j += a.splits) {
    const int64_t r = first + j;
    auto path = [&](uint32_t by) {
      if (!a.d.d_tokens) return;
      if (tid == 0) {
        int64_t at = j;
        for (int k = 0; k < LG_MOST_STEPS; ++k) {
          const uint32_t t = (uint32_t)((staged ? node_token[at] : a.d.d_tokens[first + at]) - v0);
          if (t < (uint32_t)n) {
            word[t] += by;
            mark(t);
          }
          const int32_t up = staged ? node_parent[at] : a.d.d_parent[first + at];
          if (up < 0 || up >= at) break;
          at = up;
        }
      }
      __syncthreads();
    };
    path(1u);
    const T* in = static_cast<const T*>(a.in) + r * a.d.in_stride + v0;
    T* out = static_cast<T*>(a.out) + r * a.d.out_stride + v0;
    const uint32_t* mask = MASK ? reinterpret_cast<const uint32_t*>(a.d.d_mask) + r * ((a.d.vocab + 31) / 32) + v0 / 32 : nullptr;
    auto piece = [&](int c, u32x4 x, uint32_t bits) {
      const bool seen = (maybe[c / 32] >> (c % 32)) & 1;
      bool changed = MASK && bits != ALL;
      if (seen) {
        TurnChunk<T, VEC> y;
        float f[VEC];
        y.p[0] = x;
        y.widen(f);
        uint32_t any = 0;
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
          const uint32_t w = word[c * VEC + k];
          any |= w;
          if (w) f[k] = lg_adjust(params, f[k], w);
        }
        y.round(f);
        if (any) {
          x = y.p[0];
          changed = true;
        }
      }
      if (MASK) x = lg_masked<T>(x, bits);
      if (a.in_place && !changed) return;
      Bits z;
      z.v = x;
      reinterpret_cast<Bits*>(out)[c] = z;
    };
    const int whole = n / VEC;
    int c = tid;
    for (; c + (LG_FLY - 1) * 256 < whole; c += LG_FLY * 256) {
      uint32_t bits[LG_FLY];
      u32x4 x[LG_FLY];
#pragma unroll
      for (int f = 0; f < LG_FLY; ++f) bits[f] = MASK ? (mask[(c + f * 256) * VEC / 32] >> ((c + f * 256) * VEC % 32)) & ALL : ALL;
#pragma unroll
      for (int f = 0; f < LG_FLY; ++f) x[f] = reinterpret_cast<const Bits*>(in)[c + f * 256].v;
#pragma unroll
      for (int f = 0; f < LG_FLY; ++f) piece(c + f * 256, x[f], bits[f]);
    }
    for (; c < whole; c += 256) piece(c, reinterpret_cast<const Bits*>(in)[c].v, MASK ? (mask[c * VEC / 32] >> (c * VEC % 32)) & ALL : ALL);
    for (int e = whole * VEC + tid; e < n; e += 256) {
      TurnChunk<T, 1> x;
      float f;
      x.load(in + e);
      const uint32_t w = word[e];
      const bool allowed = !MASK || (mask[e / 32] >> (e % 32)) & 1;
      if (a.in_place && !w && allowed) continue;
      if (w || !allowed) {
        x.widen(&f);
        if (w) f = lg_adjust(params, f, w);
        if (!allowed) f = -INFINITY;
        x.round(&f);
      }
      x.template store<false>(out + e);
    }
    __syncthreads();
    path(~0u);
  }
}

template <typename T>
static void launch_logits(const LogitsArgs& a, dim3 grid, hipStream_t s) {
  if (a.d.d_mask) logits_kernel<T, true><<<grid, 256, 0, s>>>(a);
  else logits_kernel<T, false><<<grid, 256, 0, s>>>(a);
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
  if (d.vocab > (int64_t)1 << 30 || d.bias_columns > 2046 || d.history_columns >= 1 << 19 || d.B > 65535 || d.rows >= (int64_t)1 << 31) return SYNERA_EUNSUP;
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
  LogitsArgs a = {d, d_in, d_out, 1, in_place};
  const int64_t slices = (d.vocab + LG_SLICE - 1) / LG_SLICE, each = (d.rows + B - 1) / B;
  a.splits = (int32_t)std::min<int64_t>(std::max<int64_t>(1, std::min<int64_t>(each, 2048 / (slices * B))), 65535);
  const dim3 grid((uint32_t)slices, (uint32_t)B, (uint32_t)a.splits);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (d.dtype == 0) launch_logits<float>(a, grid, s);
  else if (d.dtype == 1) launch_logits<bf16_t>(a, grid, s);
  else launch_logits<_Float16>(a, grid, s);
  return hipGetLastError() == hipSuccess ? SYNERA_OK : SYNERA_EHIP;
}
