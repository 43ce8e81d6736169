// The paged token cache's layout and device helpers (pcache.hip, pattn.hip).
//
// Keys by rows, values by columns of eight rows: a lane of the second product's A operand holds one
// column of eight keys, so that its 16 bytes lie together, next to the neighbouring columns', in
// memory and in LDS.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "fc_internal.h"
#include "qcache.h"

namespace fc {
namespace {

constexpr int kPTile = FC_PCACHE_TILE;

// Which page holds an item's rows.
struct PageTable {
  const int32_t *table;     // [B][width]
  int width, pages, shift;  // page_rows = 1 << shift
  __device__ __forceinline__ int entry(int b, int i) const { return table[(long)b * width + i]; }
  __device__ __forceinline__ bool there(int page) const { return (unsigned)page < (unsigned)pages; }
  // a page that can be read, whatever the entry
  __device__ __forceinline__ int safe(int page) const { return there(page) ? page : 0; }
};

inline int log2_of(int rows) {
  int s = 0;
  while ((1 << s) < rows) ++s;
  return s;
}
inline PageTable page_table(const fc_pcache &c) {
  return PageTable{c.state, c.max_pages, c.n_pages, log2_of(c.page_rows)};
}
// The holders' counts lie behind the table, whose numbers are rounded up to whole groups of four.
__host__ __device__ inline long table_numbers(long B, long width) { return (B * width + 3) / 4 * 4; }

}  // namespace
}  // namespace fc
