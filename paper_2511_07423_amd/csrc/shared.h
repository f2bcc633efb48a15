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
#define SY_SH_WAVE_ROWS 32       // rows of a tile that one wavefront can take alone
#define SY_SH_DEAL 8             // XCDs that blocks are dealt to in turn
enum {
  SY_SH_LEAF = 1,                // the item's rows are one request's, in order: causal, rows without a list
  SY_SH_ONCE = 2                 // its keys and values are marked as not wanted again
};

// A tile of rows against a range of the keys of one node (a run of pages with the requests that all read it).  Keys count from the
// node's first page on.  128 bytes, read with scalar loads.
struct ShItem {
  int32_t flags;
  int32_t kv_head;
  int32_t n_rows;      // 1 .. SY_SH_TILE_ROWS; 0: nothing to do
  int32_t row0;        // the tile's first row inside the node (row = token of the node x G + head in the group)
  int32_t tok;         // LEAF: flattened index of the request's first new token; else first entry of the node's token list
  int32_t page;        // first entry of the node's page list
  int32_t n_pages;     // its entries
  int32_t key_begin;   // multiple of SY_SH_STEP
  int32_t key_end;
  int32_t lim0;        // LEAF: last key that the request's first new token sees
  int32_t part;        // partial row of the tile's first row, or -1: no other item reads keys for these rows
  int32_t pad[5];
  int32_t pages[16];   // the first pages from key_begin on (the last one again past the node's end): no need to wait for the list
};
struct ShJoin {        // a token whose rows several items worked on
  int32_t tok, first, count, pad;
};
struct ShPart {        // where one of its partial results lies: head h's at row + h / G x step + h % G
  int32_t row, step;
};
struct ShWindow {      // the slots of one page that a plan appends to
  int32_t page, row;   // row: flattened index of the token in slot s0
  int32_t s0, s1;
};
// First words of the plan on the device.  The items come in two lists, one behind the other: those that a block takes, then those that
// a wavefront takes, four to a block; groups of SY_SH_DEAL blocks of either kind take turns (sh_block).
struct ShHeader {
  int32_t n_tokens, n_windows, n_joined;
  int32_t block_groups, wave_groups;     // groups of SY_SH_DEAL blocks
  int32_t pad[11];
};
// Which items block b of the launch takes: a block's (whole) or the first of four wavefronts'.  `run` groups of each kind follow each
// other while there are that many left: that is what one slot of each compute unit takes, so that both kinds, one bound by
// the matrix cores and one by HBM, share each unit.
#ifdef __HIPCC__
__host__ __device__
#endif
inline int32_t sh_block(int32_t block_groups, int32_t wave_groups, int32_t run, int32_t b, bool& whole) {
  const int32_t g = b / SY_SH_DEAL, x = b % SY_SH_DEAL;
  const int32_t turns = (block_groups < wave_groups ? block_groups : wave_groups) / run;
  int32_t at;
  if (g < turns * 2 * run) {
    const int32_t k = g / (2 * run), r = g % (2 * run);
    whole = r < run;
    at = k * run + (whole ? r : r - run);
  } else {
    const int32_t r = g - turns * 2 * run, left = block_groups - turns * run;
    whole = r < left;
    at = turns * run + (whole ? r : r - left);
  }
  return whole ? at * SY_SH_DEAL + x : block_groups * SY_SH_DEAL + 4 * (at * SY_SH_DEAL + x);
}

struct ShLimits {      // what a batch has room for
  int32_t Hq, Hkv, hd, max_batch, max_tokens, max_pages;
  int64_t items, list, parts, pages, windows, part_rows, shared_rows;
  int32_t slots;       // blocks that run at once: what the work is cut for
};
void sh_limits(ShLimits& l);   // fills the second and third line from the first

struct ShPlan {
  ShHeader head;
  std::vector<int32_t> tok_pos, tok_slot;           // [T]: position; page x 16 + slot
  std::vector<ShWindow> windows;
  std::vector<ShItem> items;
  std::vector<int32_t> list, pages;                 // tokens of shared nodes; pages of all nodes
  std::vector<ShJoin> joined;
  std::vector<ShPart> parts;
  int64_t part_rows;
};
// The batch has been validated.  Throws std::bad_alloc.
void sh_plan(const ShLimits& l, int32_t B, const int32_t* ctx_len, const int32_t* n_new, const int32_t* table, int32_t max_pages,
             ShPlan& p);
