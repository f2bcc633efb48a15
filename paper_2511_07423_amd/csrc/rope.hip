// Rotary positions and norms of query and key heads over whole tensors: the entry points of include/synera_shared.h and
// their kernel (rope.h has the arithmetic and the layout of the work).
#include <algorithm>
#include <cmath>
#include <new>

#include "../../include/synera.h"
#include "rope.h"

// ------------------------------------------------------------------------------------ the handle
extern "C" int32_t synera_rope_create(synera_rope** out, const synera_rope_desc* desc) {
  if (!out) return SYNERA_EINVAL;
  *out = nullptr;
  if (!desc) return SYNERA_EINVAL;
  const synera_rope_desc& d = *desc;
  if (d.head_dim < 2 || d.head_dim % 2 || d.rot_dim < 2 || d.rot_dim % 2 || d.rot_dim > d.head_dim) return SYNERA_EINVAL;
  if (d.layout != SYNERA_ROPE_INTERLEAVED && d.layout != SYNERA_ROPE_HALF) return SYNERA_EINVAL;
  if (!std::isfinite((float)d.magnitude)) return SYNERA_EINVAL;
  const int half = d.rot_dim / 2;
  if (!d.h_inv_freq) {
    if (!std::isfinite(d.base) || !(d.base > 1.0)) return SYNERA_EINVAL;
    if (d.scaling != SYNERA_ROPE_PLAIN && d.scaling != SYNERA_ROPE_LINEAR && d.scaling != SYNERA_ROPE_BANDS) return SYNERA_EINVAL;
    if (d.scaling != SYNERA_ROPE_PLAIN && (!std::isfinite(d.factor) || !(d.factor > 0.0))) return SYNERA_EINVAL;
    if (d.scaling == SYNERA_ROPE_BANDS &&
        (!(d.low >= 0.0) || !(d.high > d.low) || !std::isfinite(d.high) || !(d.original > 0.0) || !std::isfinite(d.original)))
      return SYNERA_EINVAL;
  }
  if (d.head_dim > 256) return SYNERA_EUNSUP;
  const double two_pi = 6.283185307179586476925;
  double rev[128];
  for (int i = 0; i < half; ++i) {
    double f;
    if (d.h_inv_freq) {
      f = d.h_inv_freq[i];
      if (!std::isfinite(f)) return SYNERA_EINVAL;
    } else {
      f = std::pow(d.base, -(double)i / (double)half);
      if (d.scaling == SYNERA_ROPE_LINEAR) f /= d.factor;
      if (d.scaling == SYNERA_ROPE_BANDS) {
        const double r = d.original * f / two_pi;
        const double t = r <= d.low ? 0.0 : r >= d.high ? 1.0 : (r - d.low) / (d.high - d.low);
        f = (1.0 - t) * f / d.factor + t * f;
      }
    }
    rev[i] = f / two_pi;
    if (!std::isfinite(rev[i] * 2147483648.0)) return SYNERA_EINVAL;     // the turns of the farthest position
  }
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) {
    (void)hipGetLastError();
    return SYNERA_EHIP;
  }
  synera_rope* r = new (std::nothrow) synera_rope();
  if (!r) return SYNERA_ENOMEM;
  r->desc = d;
  r->desc.h_inv_freq = nullptr;
  r->device = dev;
  r->rev = nullptr;
  if (hipMalloc(reinterpret_cast<void**>(&r->rev), half * sizeof(double)) != hipSuccess) {
    (void)hipGetLastError();
    delete r;
    return SYNERA_ENOMEM;
  }
  if (hipMemcpy(r->rev, rev, half * sizeof(double), hipMemcpyHostToDevice) != hipSuccess) {
    (void)hipGetLastError();
    (void)hipFree(r->rev);
    delete r;
    return SYNERA_EHIP;
  }
  *out = r;
  return SYNERA_OK;
}

extern "C" int32_t synera_rope_destroy(synera_rope* r) {
  if (!r) return SYNERA_OK;
  const BesideCaptures beside;                       // (the free waits for the device)
  (void)hipFree(r->rev);
  delete r;
  return SYNERA_OK;
}

bool rope_device_ok(int device) {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) (void)hipGetLastError();
  return dev == device;
}

// ------------------------------------------------------------------------------------ checks
int32_t turn_check(const synera_heads& s, int64_t n, int hd, int in_bytes, int out_bytes, bool out) {
  if (!s.d_in || s.n_heads < 1 || s.in_token < 0 || s.in_head < 0) return SYNERA_EINVAL;
  if (reinterpret_cast<uintptr_t>(s.d_in) % in_bytes || reinterpret_cast<uintptr_t>(s.d_gain) % 2) return SYNERA_EINVAL;
  if (!out) return SYNERA_OK;
  if (!s.d_out || reinterpret_cast<uintptr_t>(s.d_out) % out_bytes) return SYNERA_EINVAL;
  // outputs must not lie on one another: heads inside tokens, or tokens inside heads
  const bool one_head = s.n_heads == 1, one_token = n == 1;
  const int64_t ts = s.out_token, hs = s.out_head;
  if (ts < 0 || hs < 0) return SYNERA_EINVAL;
  const bool heads_inside = (one_head || hs >= hd) && (one_token || ts >= (one_head ? 0 : (int64_t)(s.n_heads - 1) * hs) + hd);
  const bool tokens_inside = (one_token || ts >= hd) && (one_head || hs >= (one_token ? 0 : (n - 1) * ts) + hd);
  return heads_inside || tokens_inside ? SYNERA_OK : SYNERA_EINVAL;
}

bool turn_overlap(const void* a, int64_t a_ts, int64_t a_hs, int a_heads, int a_bytes, const void* b, int64_t b_ts, int64_t b_hs,
                  int b_heads, int b_bytes, int64_t n, int hd) {
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
  const int64_t wa = ((int64_t)(a_heads - 1) * a_hs + hd) * a_bytes, wb = ((int64_t)(b_heads - 1) * b_hs + hd) * b_bytes;  // one token's span
  const int64_t la = (n - 1) * a_ts * a_bytes + wa, lb = (n - 1) * b_ts * b_bytes + wb;
  if (pa + la <= pb || pb + lb <= pa) return false;
  // the same step from token to token (slices of one array): apart if their spans are, on the circle of one step
  const int64_t step = a_ts * a_bytes;
  if (step > 0 && step == b_ts * b_bytes && wa <= step && wb <= step) {
    const int64_t d = pa < pb ? (int64_t)((pb - pa) % step) : (step - (int64_t)((pa - pb) % step)) % step;   // from a's span to b's
    if (d >= wa && d + wb <= step) return false;
  }
  return true;
}

bool turn_on_output(const synera_heads& s, int64_t n, int hd, int out_bytes, const void* at, int64_t size) {
  const uintptr_t out = reinterpret_cast<uintptr_t>(s.d_out), in = reinterpret_cast<uintptr_t>(at);
  const int64_t step = s.out_token * out_bytes, span = ((int64_t)(s.n_heads - 1) * s.out_head + hd) * out_bytes;
  if (!at || in + size <= out || out + (n - 1) * step + span <= in) return false;
  if (in > out && span <= step) {                    // in the gap between two tokens?
    const int64_t d = (int64_t)((in - out) % step);
    if (d >= span && d + size <= step) return false;
  }
  return true;
}

// The widest chunk that divides the head as the layout needs and whose vectors everything is aligned for.  6000 tokens of 40 x 128 bf16 in
// chunks of 8, 4, 2, 1 values: 24.7, 21.7, 32.7, 43.8 us; normed on the way into their pages (16 K tokens) 8 beats 4, 95 against 106 us.
static bool fits(int vec, const synera_rope* rope, const synera_heads* s, int in_bytes, int out_bytes, bool out) {
  if (rope->desc.head_dim % vec || rope->desc.rot_dim % (2 * vec)) return false;
  if (!s) return true;
  const int64_t ib = std::min(16, vec * in_bytes), ob = std::min(16, vec * out_bytes), gb = std::min(16, vec * 2);
  uint64_t in = reinterpret_cast<uintptr_t>(s->d_in) | (uint64_t)(s->in_token * in_bytes) | (uint64_t)(s->in_head * in_bytes);
  if (in % ib || reinterpret_cast<uintptr_t>(s->d_gain) % gb) return false;
  if (!out) return true;
  uint64_t o = reinterpret_cast<uintptr_t>(s->d_out) | (uint64_t)(s->out_token * out_bytes) | (uint64_t)(s->out_head * out_bytes);
  return o % ob == 0;
}

int turn_setup(TurnArgs& a, const synera_rope* rope, int64_t n_tokens, const synera_heads* q, const synera_heads* k, int in_bytes,
               int out_bytes, bool paged, float eps) {
  const int hd = rope->desc.head_dim, rot = rope->desc.rot_dim;
  auto fill = [&](TurnSeg& s, const synera_heads* h, bool out) {
    s = TurnSeg{};
    if (!h) return;
    s.in = h->d_in;
    s.out = out ? h->d_out : nullptr;
    s.gain = static_cast<const bf16_t*>(h->d_gain);
    s.in_ts = h->in_token;
    s.in_hs = h->in_head;
    s.out_ts = h->out_token;
    s.out_hs = h->out_head;
    s.n_heads = h->n_heads;
    s.tail = s.in != s.out || s.gain || in_bytes != out_bytes;     // in place the rest of a head is what it was
  };
  fill(a.q, q, true);
  fill(a.k, k, !paged);
  a.rev = rope->rev;
  a.magnitude = (float)rope->desc.magnitude;
  a.eps = eps;
  a.T = (int32_t)n_tokens;
  a.hd = hd;
  a.rot = rot;
  a.half = rope->desc.layout == SYNERA_ROPE_HALF;
  int widest = 8;                                            // chunk that the head takes where everything is aligned
  while (hd % widest || rot % (2 * widest)) widest /= 2;
  a.rest_half = ((hd - rot) / widest + 1) / 2 * widest;
  a.token_bytes = (int64_t)(a.q.n_heads + a.k.n_heads) * hd * (in_bytes + out_bytes);
  const int64_t moved = (n_tokens * a.token_bytes) >> 20;        // MB
  // (f32: a chunk of 8 is two vectors, each of which fills half a line.  Where the lines do not wait in a cache for their other halves, 4.  Chunks of 8
  // and 4, us, on new inputs each time: 40 x 128 normed, interleaved: 96 MB in and out 22.7, 25.0; 160 37.5, 39.0; 180 44.2, 41.7; 200 44.8, 44.7; 224 56.0, 47.8;
  // 256 61.4, 57.1; 288 68.6, 71.3; 352 82.3, 79.8; 640 141, 132.  40 x 128, half of each turned: 224 53.8, 44.1; 640 141, 125.  40 x 96: 224 67.9, 63.0; 640 176,
  // 148.  20 x 64, 10 x 256: 8 to 19 % less from 224 on, and 4 to 17 % less from 128 on.  4096 tokens of 40 x 128 appended: 37, 41.)
  int vec = in_bytes == 4 && !paged && moved >= 224 ? 4 : 8;
  while (vec > 1 && !(fits(vec, rope, q, in_bytes, out_bytes, true) && fits(vec, rope, k, in_bytes, out_bytes, !paged))) vec /= 2;
  const int units = rot / (2 * vec) + a.rest_half / vec;
  a.as_wide = vec == 1 && widest > 1 ? (units > 64 ? 2 : 1) : 0;
  a.lanes_log2 = 0;
  while ((1 << a.lanes_log2) < std::min(units, 64)) ++a.lanes_log2;
  const int per = 64 >> a.lanes_log2;
  a.groups = (a.q.n_heads + a.k.n_heads + per - 1) / per;
  a.cols = turn_cols(a.groups, a.T);
  a.once = turn_once(vec, moved, paged);
  return vec;
}

// ------------------------------------------------------------------------------------ whole tensors
template <typename T, int VEC, int ONCE>
__global__ __launch_bounds__(256) void rope_kernel(TurnArgs a) {
  const uint32_t items = (uint32_t)a.T * (uint32_t)a.cols.n;
  for (uint32_t item = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); item < items; item += gridDim.x * 4)
    turn_item<T, T, VEC, false, ONCE>(a, a.cols, item);
}

template <typename T, int VEC>
static void launch_vec(const TurnArgs& a, uint32_t blocks, hipStream_t s) {
  if constexpr (VEC >= 4) {
    if (a.once == TURN_ONCE_BOTH) return rope_kernel<T, VEC, TURN_ONCE_BOTH><<<blocks, 256, 0, s>>>(a);
    if (a.once == TURN_ONCE_IN) return rope_kernel<T, VEC, TURN_ONCE_IN><<<blocks, 256, 0, s>>>(a);
  }
  rope_kernel<T, VEC, TURN_KEPT><<<blocks, 256, 0, s>>>(a);
}
template <typename T>
static hipError_t launch_rope(const TurnArgs& a, int vec, hipStream_t s) {
  const uint32_t blocks = std::min(((uint32_t)a.T * (uint32_t)a.cols.n + 3) / 4, 1u << 22);   // a launch has less than 2^32 threads
  switch (vec) {
    case 8: launch_vec<T, 8>(a, blocks, s); break;
    case 4: launch_vec<T, 4>(a, blocks, s); break;
    case 2: launch_vec<T, 2>(a, blocks, s); break;
    default: launch_vec<T, 1>(a, blocks, s);
  }
  return hipGetLastError();
}

static int32_t turn_tensors(const synera_rope* rope, int32_t dtype, int64_t n, const int32_t* d_pos, const synera_heads* q,
                            const synera_heads* k, float eps, bool norm, void* stream) {
  if (!rope || !q || n < 0 || dtype < 0 || dtype > 2) return SYNERA_EINVAL;
  if (n == 0) return SYNERA_OK;                      // (an empty tensor has no address)
  if (!d_pos) return SYNERA_EINVAL;
  if (reinterpret_cast<uintptr_t>(d_pos) % 4) return SYNERA_EINVAL;
  const int bytes = dtype == 0 ? 4 : 2, hd = rope->desc.head_dim;
  const synera_heads* both[2] = {q, k};
  for (const synera_heads* s : both) {
    if (!s) continue;
    const int32_t st = turn_check(*s, n, hd, bytes, bytes, true);
    if (st != SYNERA_OK) return st;
    if ((s->d_gain != nullptr) != norm) return SYNERA_EINVAL;
  }
  for (const synera_heads* o : both)
    for (const synera_heads* i : both) {
      if (!o || !i) continue;
      if (o == i && o->d_in == o->d_out && (n == 1 || o->in_token == o->out_token) && (o->n_heads == 1 || o->in_head == o->out_head)) continue;
      if (turn_overlap(o->d_out, o->out_token, o->out_head, o->n_heads, bytes, i->d_in, i->in_token, i->in_head, i->n_heads, bytes, n, hd))
        return SYNERA_EINVAL;
    }
  if (k && turn_overlap(q->d_out, q->out_token, q->out_head, q->n_heads, bytes, k->d_out, k->out_token, k->out_head, k->n_heads, bytes, n, hd))
    return SYNERA_EINVAL;
  if (n * ((int64_t)q->n_heads + (k ? k->n_heads : 0)) >= (int64_t)1 << 31) return SYNERA_EUNSUP;
  for (const synera_heads* o : both)
    for (const synera_heads* i : both)
      if (o && i && (turn_on_output(*o, n, hd, bytes, d_pos, 4 * n) || turn_on_output(*o, n, hd, bytes, i->d_gain, 2 * hd))) return SYNERA_EINVAL;
  if (!rope_device_ok(rope->device)) return SYNERA_EINVAL;
  TurnArgs a = {};
  const int vec = turn_setup(a, rope, n, q, k, bytes, bytes, false, eps);
  a.pos = d_pos;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const hipError_t e = dtype == 0   ? launch_rope<float>(a, vec, s)
                       : dtype == 1 ? launch_rope<bf16_t>(a, vec, s)
                                    : launch_rope<_Float16>(a, vec, s);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    return SYNERA_EHIP;
  }
  return SYNERA_OK;
}

extern "C" int32_t synera_rope_apply(const synera_rope* rope, int32_t dtype, int64_t n_tokens, const int32_t* d_pos,
                                     const synera_heads* q, const synera_heads* k, void* stream) {
  return turn_tensors(rope, dtype, n_tokens, d_pos, q, k, 0.f, false, stream);
}

extern "C" int32_t synera_qk_norm_rope(const synera_rope* rope, int32_t dtype, int64_t n_tokens, const int32_t* d_pos,
                                       const synera_heads* q, const synera_heads* k, float eps, void* stream) {
  if (!(eps >= 0.f) || !std::isfinite(eps)) return SYNERA_EINVAL;
  return turn_tensors(rope, dtype, n_tokens, d_pos, q, k, eps, true, stream);
}
