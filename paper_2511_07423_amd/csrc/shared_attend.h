// Attention of a block, or a wavefront, over one item of work on the paged cache: the device code that shared.hip (prefixes shared by requests)
// and tree.hip (trees of drafted tokens) build on.
#pragma once
#include <type_traits>

#include "common.h"
#include "shared.h"

#define SH_CONST_AS __attribute__((address_space(4)))

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
#define SY_TREE_MASK 12          // words of a token's mask: two of ones for the context, SYNERA_TREE_NODES bits, zeros
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
// TREE: a row sees the keys before lim0 (its request's context) and those behind whose bits are set in its token's mask.
template <int HD, int WR, int WK, bool TREE = false, typename Args>
__device__ __forceinline__ void attend(const Args& a, const ShItem& it, const int32_t* first_pages, unsigned char* lds) {
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
  const int free_end = TREE ? min(it.key_end, it.lim0) : leaf ? min(it.key_end, it.lim0 + it.row0 / a.G + 1) : it.key_end;   // keys below need no mask
  const uint32_t* mask = nullptr;
  uint32_t vis = 0;                                           // which keys of the tile at hand the row sees
  if constexpr (TREE) mask = a.masks + (size_t)tok * SY_TREE_MASK;
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
    if constexpr (masked && TREE) {
      const int at = kb - it.lim0 + 64;                       // from the two words in front, which stand for the context's end: a masked tile begins
                                                              // less than 64 keys before it (the loop two tiles at a time may leave one that needs no mask)
      vis = __builtin_amdgcn_alignbit(mask[(at >> 5) + 1], mask[at >> 5], at & 31);
      const uint32_t mine = vis >> (8 * h);
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[r] = (mine >> (16 * (r >> 3) + (r & 7))) & 1 ? sc[r] : -INFINITY;
    } else if constexpr (masked) {
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
            const bool seen = TREE ? (vis >> (16 * b + k)) & 1 : kb + 16 * b + k <= lim;
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

// Host side (shared.hip): checks what calls of the attention have in common and fills in what they say.  SH_NOTHING: no tokens, no launch.
#define SH_NOTHING 1
int32_t sh_attention_args(SharedAttnArgs& a, const ShLimits& l, int32_t n_pages, int64_t n_tokens, bool graph, const synera_heads* q,
                          const void* d_k_layer, const void* d_v_layer, float scale, float* d_lse);
