// How the attention over an 8-bit cache goes through its work.  Plain C++, shared by the device code (row counts are
// only known there), the host code and a CPU build.
#pragma once

#include "fd_rules.h"

namespace fd {

constexpr int kFewRows = 32;                                                  // rows of an item of few rows
FD_RULE constexpr int cache_tile_rows(int dh) { return dh >= 64 ? 256 : 128; }   // ... of a tile

// Few rows rather than tiles, by the items that each way has: all waves of a workgroup work on 32 rows, each on its own
// keys, where tiles would leave most waves without rows.
FD_RULE bool cache_few_rows(int few, int tiles) { return few <= 3 * tiles; }
// Whether every request of a call of at most `rows` rows is of few: 3 items of 32 rows are not too many for a tile.
FD_RULE bool cache_always_few(long long rows) { return rows <= 3 * kFewRows; }

// Key tiles that the start of an item of tiles counts for in the shares: its queries and first key tiles on their way.  Every share has one
// start; where they have more, those of short items would end late.
FD_RULE int cache_item_steps(long long items, int shares) { return items > shares ? 3 : 0; }

}  // namespace fd
