// Declarations shared by the sources behind include/synera_shared.h: the rotation's handle and launcher (rope.hip), the
// batch planner (shared_plan.cpp, host only) and the kernels over a planned batch (shared.hip).
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <vector>

#include "../../include/synera.h"
#include "../../include/synera_shared.h"

// ---------------------------------------------------------------- shared_plan.cpp
#define SY_SH_TILE_ROWS 128      // query rows (tokens x group) of one tile of the attention
#define SY_SH_STEP 128           // keys that all wavefronts of a block take together at most: key ranges are cut at multiples of it
enum { SY_SH_LEAF = 1 };         // the item's rows are one request's, in order: causal, rows without a list

// One block's work: a tile of rows against a range of the keys of one node (a run of pages with the requests that all read
// it).  Keys count from the node's first page on.  64 bytes, read with scalar loads.
struct ShItem {
  int32_t flags;
  int32_t kv_head;
  int32_t n_rows;      // 1 .. SY_SH_TILE_ROWS
  int32_t row0;        // the tile's first row inside the node (row = token of the node x G + head in the group)
  int32_t tok;         // LEAF: flattened index of the request's first new token; else first entry of the node's token list
  int32_t page;        // first entry of the node's page list
  int32_t n_pages;     // its entries
  int32_t key_begin;   // multiple of SY_SH_STEP
  int32_t key_end;
  int32_t lim0;        // LEAF: last key that the request's first new token sees
  int32_t part;        // partial row of the tile's first row, or -1: no other item reads keys for these rows
  int32_t pad[5];
};
// What attn_join needs of one node of one request: 32 bytes.
struct ShEntry {
  int32_t base;        // partial row of split 0, KV head 0, the request's first row
  int32_t row0;        // that row inside the node
  int32_t rows;        // rows of the node: what lies between KV heads; rows x KV heads between splits
  int32_t keys;        // of the node
  int32_t chunk;       // keys of a split
  int32_t lim0;        // LEAF: as in ShItem; else -1
  int32_t pad[2];
};
struct ShWindow {      // the slots of one page that a plan appends to
  int32_t page, row;   // row: flattened index of the token in slot s0
  int32_t s0, s1;
};
struct ShHeader {      // first words of the plan on the device
  int32_t n_tokens, n_windows, n_items, n_joined;
  int32_t pad[12];
};

struct ShLimits {      // what a batch has room for
  int32_t Hq, Hkv, hd, max_batch, max_tokens, max_pages;
  int64_t items, list, entries, pages, windows, part_rows, shared_rows;
  int32_t slots;       // blocks that run at once: what the work is cut for
};
void sh_limits(ShLimits& l);   // fills the second and third line from the first

struct ShPlan {
  ShHeader head;
  std::vector<int32_t> tok_pos, tok_slot;           // [T]: position; page x 16 + slot
  std::vector<ShWindow> windows;
  std::vector<ShItem> items;
  std::vector<int32_t> list, pages;                 // tokens of shared nodes; pages of all nodes
  std::vector<int32_t> joined;                      // tokens whose partials are to be joined, with their request: pairs
  std::vector<int32_t> first_entry;                 // [B + 1]
  std::vector<int32_t> req_tok;                     // [B]: flattened index of the first new token
  std::vector<ShEntry> entries;
};
// The batch has been validated.  Throws std::bad_alloc.
void sh_plan(const ShLimits& l, int32_t B, const int32_t* ctx_len, const int32_t* n_new, const int32_t* table, int32_t max_pages,
             ShPlan& p);
