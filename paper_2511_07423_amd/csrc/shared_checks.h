// Host-side checks that the calls over a paged cache have in common.
#pragma once
#include <algorithm>
#include <initializer_list>

#include "rope.h"
#include "shared.h"

inline bool capturing(hipStream_t s) {
  hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(s, &st) != hipSuccess) {
    (void)hipGetLastError();
    return true;               // the legacy stream while another one is captured: nothing may be launched there
  }
  return st != hipStreamCaptureStatusNone;
}

struct Range { uintptr_t from, to; };
inline bool meet(const Range& a, const Range& b) { return a.from < b.to && b.from < a.to; }
inline Range heads_range(const void* p, int64_t ts, int64_t hs, int64_t heads, int64_t n, int hd, int bytes) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  return {at, at + (uintptr_t)(((n - 1) * ts + (heads - 1) * hs + hd) * bytes)};
}
inline Range pool_range(const ShLimits& l, int32_t n_pages, const void* p) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  return {at, at + (uintptr_t)n_pages * l.Hkv * SY_PAGE * l.hd * 2};
}

// Tokens that the checks of a call go by: the plan's T; of a captured call, which serves later plans too, as many as all its tensors have room
// for.  -1: a tensor lacks room for the plan at hand.  room: tokens that any plan may bring to these tensors.
inline int64_t tokens_to_check(int64_t T, int64_t max_tokens, bool graph, std::initializer_list<const synera_heads*> heads, int64_t& room) {
  room = 0;
  for (const synera_heads* h : heads) {
    if (!h || !h->n_rows) continue;
    if (h->n_rows < T) return -1;
    room = room ? std::min<int64_t>(room, h->n_rows) : h->n_rows;
  }
  const int64_t said = room;
  room = std::min<int64_t>(said ? said : INT64_MAX, max_tokens);
  if (!graph) return std::max<int64_t>(T, 1);
  return std::max<int64_t>({T, 1, said ? room : std::min<int64_t>(room, 2)});
}
