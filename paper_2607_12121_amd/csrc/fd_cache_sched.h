// How the attention over an 8-bit cache goes through its work: which way, and which key steps of which item each workgroup
// runs.  Plain C++, shared by the device code (row counts are only known there), the host code and a CPU build.
//
// An item is a key head and up to 32 (few rows), 128 or 256 (tiles) of a request's rows, a row being a query under one of the
// heads that share the key head; its steps are 64 keys each in tiles, a tile per wave of a workgroup with few rows.
#pragma once

#include "fd_attn_sched.h"

namespace fd {

constexpr int kFewRows = 32;
FD_RULE constexpr int cache_tile_rows(int dh) { return dh >= 64 ? 256 : 128; }      // rows of an item of tiles
FD_RULE constexpr int cache_few_keys(int dh) { return 2 * cache_tile_rows(dh); }    // keys of a step of few rows

// Few rows rather than tiles, by the items that each way has: all waves of a workgroup work on the same 32 rows, each on keys of
// its own, where tiles would leave most waves without rows.  One request, us, few rows and tiles: 12 heads of 128 over 32760 keys,
// 64 rows (2 items of few rows a head, 1 of tiles) 52 and 62, 96 rows (3) 57 and 63, 128 rows (4) 76 and 66; 24 heads of 64 over
// 20000 keys, 64 rows 45 and 48, 96 rows 53 and 48, and 16 heads over 2 requests of 10000 keys, 128 rows (5 and 2) 25 and 28; 24
// heads of 16 over 8000 keys, 96 rows 20 and 22, 128 rows 22 and 22.5.
FD_RULE constexpr int cache_few_half_items(int dh) { return dh == 64 ? 5 : 6; }   // per item of tiles, twice
FD_RULE bool cache_few_rows(int dh, int few, int tiles) { return 2LL * few <= static_cast<long long>(cache_few_half_items(dh)) * tiles; }
// Whether every call of at most `rows` rows is of few.
FD_RULE bool cache_always_few(int dh, long long rows) { return rows <= cache_few_half_items(dh) / 2 * kFewRows; }

// Key tiles that the start of an item of tiles counts for in the shares: its queries and first key tiles on their way.  Every share
// has one start; where shares have several items, those of short ones would end late (a packed batch 276 -> 254 us).
FD_RULE int cache_item_steps(long long items, int shares) { return items > shares ? 3 : 0; }

// The shares.  In tiles attn_cuts decides whether items are cut; few rows always are, into shares of a step at least.  `start`: the
// steps that an item's start counts for, in the tables as in the item.
template <int DH>
struct CacheSched : AttnSched<cache_tile_rows(DH), DH, true, true> {
  using Base = AttnSched<cache_tile_rows(DH), DH, true, true>;
  int start;
  FD_RULE CacheSched(const SchedTables* t, const int32_t* cu_q, const int32_t* tok_off, int n_req, int kv_heads, int grid, int nkv_max, bool few,
                     bool may_cut, int start_)
      : Base(t, cu_q, tok_off, n_req, kv_heads, grid, nkv_max + start_), start(start_) {
    if (!few && may_cut) return;
    this->cut = few && may_cut;
    this->G = grid;
    this->per = div_steps(this->work, grid);
    this->extra = static_cast<int>(this->work - this->per * grid);
    if (this->cut && this->work < grid) {   // shares of one step, so that the empty ones come last
      this->G = static_cast<int>((this->work + kXcds - 1) / kXcds * kXcds);
      this->per = 1;
      this->extra = 0;
    }
  }
  // A share does not end among the steps that stand for an item's start, but before it: no piece is without keys (a share is
  // longer than those steps).
  FD_RULE long long bound(long long x) const {
    const long long q = Base::bound(x);
    if (!this->cut || start == 0 || q >= this->work) return q;
    long long i_start;
    int n, head, b, first, tau;
    this->locate(q, i_start, n, head, b, first, tau);
    return q - i_start <= start ? i_start : q;
  }
  // Last share that holds a piece of the item that ends at step i_end: the largest x whose bound, x work / G rounded down or
  // x per, is below it.  (Walked to from the item's first share it takes 5 us of 21 pieces.)
  FD_RULE int last_share(long long i_end) const {
    return static_cast<int>(this->extra == 0 ? div_steps(i_end - 1, this->per) : div_steps(i_end * this->G - 1, this->work));
  }
  FD_RULE int tile(int step) const { return step > 0 ? step - start : 0; }   // key tile (step of few rows) at an item's step
};

}  // namespace fd
