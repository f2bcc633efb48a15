// What turns query and key heads by their positions: the handle behind synera_rope, the kernel's arguments, and the device code
// that rope.hip (whole tensors) and shared.hip (appends) build on.
//
// A head's values are dealt out in units of two chunks of VEC neighbouring values, one unit to a lane: chunk u and chunk
// u + R of the rotated part (R units; in the half layout they hold the two values of each pair, interleaved pairs lie inside a
// chunk), then the rest of the head two chunks at a time.  So every lane has VEC pairs, whose cosines and sines it forms
// once for all heads of its token, and both loads of a unit are contiguous over lanes.  A wavefront takes 64 / lanes-per-head
// heads at a time.
//
// Bound by HBM: every value is read and written once.  The angle costs a lane one 64-bit product and 40 instructions a
// pair, for all its heads.  Measured, on new inputs each time: 8192 tokens of 40 x 128 bf16, half of each head turned, 38 us, 4.4 TB/s; 16000 tokens 60 us, 5.4;
// 6000 in f32, normed, 51 us, 4.8; one token 3.1 us, 64 normed ones 4.8.
#pragma once
#include "common.h"
#include "../../include/synera_shared.h"

struct synera_rope {
  synera_rope_desc desc;       // h_inv_freq is not kept
  int device;
  double* rev;                 // device [rot_dim / 2]: turns from one position to the next
};

enum { TURN_KEPT, TURN_ONCE_IN, TURN_ONCE_BOTH };   // nothing, inputs, inputs and outputs
// How a token's head groups are dealt to wavefronts: `groups` to an item, n items.  They share the token's cosines and sines, and are
// spread while there are too few items.
struct TurnCols {
  int32_t groups, n;
};
__host__ __device__ inline TurnCols turn_cols(int32_t groups, int32_t n_tokens) {
  const int32_t want = 4096 / (n_tokens > 1 ? n_tokens : 1), cols = want > groups ? groups : want > 1 ? want : 1;
  const int32_t each = (groups + cols - 1) / cols;
  return TurnCols{each, (groups + each - 1) / each};
}
// What the last-level cache (256 MB) could not hold for the next call anyway is marked as not wanted again, so that the rest stays there.
// Inputs are read for the last time: a producer, 8192 tokens of 40 x 128 bf16 turned, a reader of the queries 81 -> 74 us; below, where
// the producer left them in the caches, 2000 tokens alone 10.4 -> 12.1.  Outputs come next, so they are marked only where they are gone by
// then: 12 000 tokens and their reader 94 -> 84 us, but 8192 and theirs 55 -> 63; appends, whose keys the attention reads with all
// else: 31 585 tokens 169 -> 139 us (with their attention 656 -> 656), 11 400 with theirs 206 -> 215.  (Chunks of one or two values, which
// have too few bytes on their way for more than 2.5 TB/s, are not marked.)  moved: MB in and out.
__host__ __device__ inline int32_t turn_once(int vec, int64_t moved, bool paged) {
  return vec < 4 || moved < 128 ? TURN_KEPT : moved < (paged ? 512 : 224) ? TURN_ONCE_IN : TURN_ONCE_BOTH;
}
struct TurnSeg {
  const void* in;
  void* out;
  const bf16_t* gain;
  int64_t in_ts, in_hs, out_ts, out_hs;
  int32_t n_heads;
  int32_t tail;                // whether values behind the rotated ones are written
};
struct TurnArgs {
  TurnSeg q, k;
  const int32_t* pos;          // [T]
  const double* rev;
  float magnitude, eps;
  int32_t T, hd, rot, half;
  int32_t rest_half;           // value i of the rest of a head (from rot on) shares a unit with value i + rest_half: goes by hd and rot alone
  int32_t as_wide;             // 1, 2 (more than 64 units): single values whose squares are summed in the order of the wider chunks that other calls
                               // for such heads take
  int32_t lanes_log2, groups;  // lanes of a head; head groups of a token
  TurnCols cols;
  int64_t token_bytes;         // moved for a token, in and out
  int32_t once;                // what is marked as not wanted again: TURN_ONCE_*
  // appends: keys go to their pages
  const int32_t* slot;         // [T] page x 16 + slot
  bf16_t* k_layer;
};

template <typename T> struct TurnType;
template <> struct TurnType<float> { typedef float raw; };
template <> struct TurnType<bf16_t> { typedef uint16_t raw; };
template <> struct TurnType<_Float16> { typedef _Float16 raw; };

template <int N> struct TurnBits { typedef u32x4 v; };
template <> struct TurnBits<8> { typedef __attribute__((ext_vector_type(2))) uint32_t v; };
template <> struct TurnBits<4> { typedef uint32_t v; };
template <> struct TurnBits<2> { typedef uint16_t v; };

// VEC values as they lie in memory, on VEC x size bytes (at most 16)
template <typename T, int VEC>
struct TurnChunk {
  static constexpr int BYTES = VEC * (int)sizeof(T), PIECE = BYTES > 16 ? 16 : BYTES, N = BYTES / PIECE;
  typename TurnBits<PIECE>::v p[N];
  template <bool ONCE = false>
  __device__ __forceinline__ void load(const T* from) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const auto* at = reinterpret_cast<const typename TurnBits<PIECE>::v*>(from) + i;
      if constexpr (ONCE) p[i] = __builtin_nontemporal_load(at);
      else p[i] = *at;
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = typename TurnBits<PIECE>::v{};
  }
  template <bool ONCE>
  __device__ __forceinline__ void store(T* to) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      auto* at = reinterpret_cast<typename TurnBits<PIECE>::v*>(to) + i;
      if constexpr (ONCE) __builtin_nontemporal_store(p[i], at);
      else *at = p[i];
    }
  }
  __device__ __forceinline__ void widen(float* f) const;
  __device__ __forceinline__ void round(const float* f);
};
template <typename T, int VEC>
__device__ __forceinline__ void TurnChunk<T, VEC>::widen(float* f) const {
  T t[VEC];
  __builtin_memcpy(t, p, BYTES);
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    if constexpr (sizeof(T) == 2 && (T)0.5f == (T)0) f[i] = bf2f((uint32_t)t[i]);   // bf16_t is the raw bits
    else f[i] = (float)t[i];
  }
}
template <typename T, int VEC>
__device__ __forceinline__ void TurnChunk<T, VEC>::round(const float* f) {
  T t[VEC];
  if constexpr (sizeof(T) == 2 && (T)0.5f == (T)0) {
    if constexpr (VEC == 1) {
      t[0] = (T)f2bf(f[0]);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; i += 2) {
        const uint32_t w = pack_bf2(f[i], f[i + 1]);
        t[i] = (T)(w & 0xFFFF);
        t[i + 1] = (T)(w >> 16);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) t[i] = (T)f[i];
  }
  __builtin_memcpy(p, t, BYTES);
}

// Cosine and sine of pos x rev turns: whole turns go in 64 bits, what is left (at most half a turn) is rounded to 32.
__device__ __forceinline__ void turn_angle(double pos, double rev, float magnitude, float& c, float& s) {
  const double t = pos * rev;
  sincospif(2.0f * (float)(t - rint(t)), &s, &c);
  c *= magnitude;
  s *= magnitude;
}

// Item `item` of the call: the item % cols.n th head groups of token item / cols.n.  TI, TO: element types in and out.
template <typename TI, typename TO, int VEC, bool PAGED, int ONCE>
__device__ __forceinline__ void turn_item(const TurnArgs& a, const TurnCols cols, const uint32_t item) {
  constexpr int NU = VEC == 1 ? 2 : 1;                      // single values: up to 128 units on 64 lanes
  // Heads of a lane whose loads are on their way together: 64 bytes in all for chunks of 8 values, 32 for 4 in 16 bits.  (Twice that: fewer wavefronts
  // fit; 6000 tokens of 40 x 128 f32 normed 54.7 -> 46.8 us, 31585 tokens appended 173 -> 169.)  Chunks of 2 and 1 are on their way for one head at a time: the
  // generated code widens each masked chunk in its own branch and waits for it there.
  constexpr int IT = NU == 1 && VEC * (int)sizeof(TI) <= 16 ? 2 : 1;
  const int lane = threadIdx.x & 63;
  const uint32_t t = item / (uint32_t)cols.n;
  const int g0 = (int)(item - t * (uint32_t)cols.n) * cols.groups;
  const int g1 = min(a.groups, g0 + cols.groups);
  const int per = 64 >> a.lanes_log2, sub = lane >> a.lanes_log2, u0 = lane & ((1 << a.lanes_log2) - 1);
  const int R = a.rot / (2 * VEC), rest_units = a.rest_half / VEC;
  const bool apart = VEC == 1 && !a.half;                   // single interleaved values: a unit is one pair
  int ca[NU], cb[NU];                                       // first value of the unit's chunks, -1: none
  float cs[NU][VEC], sn[NU][VEC];
  bool turned[NU];
  const double pos = (double)a.pos[t];
  size_t page_at = 0;
  if (PAGED) {
    const int32_t at = a.slot[t];
    page_at = ((size_t)(at / SY_PAGE) * a.k.n_heads * SY_PAGE + at % SY_PAGE) * a.hd;   // of head 0; heads lie SY_PAGE x hd apart
  }
#pragma unroll
  for (int n = 0; n < NU; ++n) {
    const int u = u0 + 64 * n;
    turned[n] = u < R;
    ca[n] = cb[n] = -1;
    if (turned[n]) {
      ca[n] = (apart ? 2 * u : u) * VEC;
      cb[n] = (apart ? 2 * u + 1 : u + R) * VEC;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const int f = a.half || VEC == 1 ? u * VEC + j : (j < VEC / 2 ? u * (VEC / 2) + j : (u + R) * (VEC / 2) + j - VEC / 2);
        turn_angle(pos, a.rev[f], a.magnitude, cs[n][j], sn[n][j]);
      }
    } else if (u - R < rest_units) {
      ca[n] = (2 * R + u - R) * VEC;
      if (ca[n] + a.rest_half < a.hd) cb[n] = ca[n] + a.rest_half;
    }
  }
  for (int g = g0; g < g1; g += IT) {
    TurnChunk<TI, VEC> xa[IT][NU], xb[IT][NU];
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int h = (g + i) * per + sub;
      const bool on = g + i < g1 && h < a.q.n_heads + a.k.n_heads;
      const bool is_q = h < a.q.n_heads;
      const TI* in = static_cast<const TI*>(is_q ? a.q.in : a.k.in) + (int64_t)t * (is_q ? a.q.in_ts : a.k.in_ts) +
                     (int64_t)(is_q ? h : h - a.q.n_heads) * (is_q ? a.q.in_hs : a.k.in_hs);
      const bool tail = is_q ? a.q.tail != 0 : a.k.tail != 0;
#pragma unroll
      for (int n = 0; n < NU; ++n) {
        xa[i][n].zero();
        xb[i][n].zero();
        if (on && (turned[n] || tail)) {
          if (ca[n] >= 0) xa[i][n].template load<ONCE != TURN_KEPT>(in + ca[n]);
          if (cb[n] >= 0) xb[i][n].template load<ONCE != TURN_KEPT>(in + cb[n]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      if (g + i >= g1) break;                               // uniform
      const int h = (g + i) * per + sub;
      const bool on = h < a.q.n_heads + a.k.n_heads;
      const bool is_q = h < a.q.n_heads;
      const bf16_t* gain = is_q ? a.q.gain : a.k.gain;
      float va[NU][VEC], vb[NU][VEC];
#pragma unroll
      for (int n = 0; n < NU; ++n) {
        xa[i][n].widen(va[n]);
        xb[i][n].widen(vb[n]);
      }
      if (a.q.gain || a.k.gain) {                           // uniform; heads without gains pass by
        // (The gains come from the nearest cache each time.  Kept from the beginning, they were waited for before the heads: 47 -> 64 us.)
        // The order of the sum goes by hd, rot and layout alone, not by VEC, which goes by sizes and alignment too: squares x[p]^2 + x[p + rot / 2]^2
        // of the turned part, then x[p]^2 + x[p + rest_half]^2 of the rest, in a binary tree over p, neighbours first.  (Heads that only single values
        // divide have an order of their own: in this one 2000 x 20 of 250 take 33 in place of 30 us.  Rows of other heads that start on odd elements pay for it:
        // 3000 x 40 of 128 71 -> 76 us, interleaved 72 -> 82.)
        auto across = [&](float v) {
          for (int o = 1; o < 1 << a.lanes_log2; o *= 2) v += __shfl_xor(v, o);
          return v;
        };
        float ss = 0.f;
#pragma unroll
        for (int n = 0; n < NU; ++n) {
          float sq[VEC];
#pragma unroll
          for (int j = 0; j < VEC; ++j) sq[j] = __builtin_fmaf(va[n][j], va[n][j], vb[n][j] * vb[n][j]);
#pragma unroll
          for (int o = 1; o < VEC; o *= 2)
#pragma unroll
            for (int j = 0; j < VEC; j += 2 * o) sq[j] += sq[j + o];
          if (VEC == 1 && a.as_wide) {
            if (apart && on && turned[n]) {                 // the lane holds a pair: the two values that are summed together are read again
              const TI* in = static_cast<const TI*>(is_q ? a.q.in : a.k.in) + (int64_t)t * (is_q ? a.q.in_ts : a.k.in_ts) +
                             (int64_t)(is_q ? h : h - a.q.n_heads) * (is_q ? a.q.in_hs : a.k.in_hs) + u0 + 64 * n;
              TurnChunk<TI, 1> x, y;
              float fx, fy;
              x.load(in);
              y.load(in + R);
              x.widen(&fx);
              y.widen(&fy);
              sq[0] = __builtin_fmaf(fx, fx, fy * fy);
            }
            if (a.as_wide > n) sq[0] = across(sq[0]);
          }
          ss += sq[0];
        }
        if (!(VEC == 1 && a.as_wide)) ss = across(ss);
        const float inv = 1.0f / sqrtf(ss / (float)a.hd + a.eps);
        if (gain && on) {
#pragma unroll
          for (int n = 0; n < NU; ++n) {
            TurnChunk<bf16_t, VEC> ga, gb;
            float fa[VEC], fb[VEC];
            ga.zero();
            gb.zero();
            if (ca[n] >= 0) ga.load(gain + ca[n]);
            if (cb[n] >= 0) gb.load(gain + cb[n]);
            ga.widen(fa);
            gb.widen(fb);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
              va[n][j] *= inv * fa[j];
              vb[n][j] *= inv * fb[j];
            }
          }
        }
      }
      if (!on) continue;
      TO* out;
      if (PAGED && !is_q)
        out = reinterpret_cast<TO*>(a.k_layer) + page_at + (size_t)(h - a.q.n_heads) * SY_PAGE * a.hd;
      else
        out = static_cast<TO*>(is_q ? a.q.out : a.k.out) + (int64_t)t * (is_q ? a.q.out_ts : a.k.out_ts) +
              (int64_t)(is_q ? h : h - a.q.n_heads) * (is_q ? a.q.out_hs : a.k.out_hs);
      const bool tail = is_q ? a.q.tail != 0 : a.k.tail != 0;
#pragma unroll
      for (int n = 0; n < NU; ++n) {
        if (turned[n]) {
          if (a.half || VEC == 1) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
              float r0, r1;
              rotate_pair(va[n][j], vb[n][j], cs[n][j], sn[n][j], r0, r1);
              va[n][j] = r0;
              vb[n][j] = r1;
            }
          } else if constexpr (VEC > 1) {
#pragma unroll
            for (int j = 0; j < VEC / 2; ++j) {
              float r0, r1;
              rotate_pair(va[n][2 * j], va[n][2 * j + 1], cs[n][j], sn[n][j], r0, r1);
              va[n][2 * j] = r0;
              va[n][2 * j + 1] = r1;
              rotate_pair(vb[n][2 * j], vb[n][2 * j + 1], cs[n][VEC / 2 + j], sn[n][VEC / 2 + j], r0, r1);
              vb[n][2 * j] = r0;
              vb[n][2 * j + 1] = r1;
            }
          }
        } else if (!tail) {
          continue;
        }
        TurnChunk<TO, VEC> y;
        if (ca[n] >= 0) {
          y.round(va[n]);
          y.template store<ONCE == TURN_ONCE_BOTH>(out + ca[n]);
        }
        if (cb[n] >= 0) {
          y.round(vb[n]);
          y.template store<ONCE == TURN_ONCE_BOTH>(out + cb[n]);
        }
      }
    }
  }
}

// Host side (rope.hip).  turn_check: EINVAL where the heads of one tensor cannot be what they say; out: whether d_out counts.
int32_t turn_check(const synera_heads& s, int64_t n_tokens, int hd, int in_bytes, int out_bytes, bool out);
// Whether an output and an input of one call, or two outputs, lie on one another other than as one tensor in place.
bool turn_overlap(const void* a, int64_t a_ts, int64_t a_hs, int a_heads, int a_bytes, const void* b, int64_t b_ts, int64_t b_hs,
                  int b_heads, int b_bytes, int64_t n_tokens, int hd);
// Whether `size` bytes of an input lie on the heads that an output writes (between tokens they may).
bool turn_on_output(const synera_heads& s, int64_t n_tokens, int hd, int out_bytes, const void* at, int64_t size);
// Fills the segments, VEC and the lane geometry of `a` from the rope and the heads (q or k may be null).
int turn_setup(TurnArgs& a, const synera_rope* rope, int64_t n_tokens, const synera_heads* q, const synera_heads* k, int in_bytes,
               int out_bytes, bool paged, float eps);
bool rope_device_ok(int device);   // whether this device is the current one
