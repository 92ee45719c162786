// Room for the partial results of prompts and shared prefixes: host arithmetic (and what the kernels take from it), so that a test can
// compile it by itself.
#pragma once
#include <stdint.h>

namespace lfps {

constexpr int kPartFloats = 128 + 4;       // of a partial row: weighted sum of the values, largest score (powers of two), sum of the weights

// The rows that requests of a prefix call have for themselves (prefix_groups.h): workgroups wanted of the kernel over the items, rows that
// an item has at least, items at most, and 32-bit words of their plan.
constexpr int kOwnWorkgroups = 1024, kOwnLeast = 64;
constexpr int own_items_for(int batch, int kv_heads) { return (kv_heads < kOwnWorkgroups ? kOwnWorkgroups / kv_heads : 1) + batch; }
constexpr int64_t own_plan_ints_for(int batch, int kv_heads) { return 4 * (int64_t)own_items_for(batch, kv_heads) + 2 * batch + 1; }
constexpr int64_t own_plan_rows_for(int batch, int kv_heads) { return (own_plan_ints_for(batch, kv_heads) + kPartFloats - 1) / kPartFloats; }

// Partial rows of a context.  Two parts at least of every (request, head); otherwise what 256 workgroups of 256 query rows make; and what
// cuts the rows that requests have for themselves.  Beyond 1024 KV heads the last is more than 8192 rows: one part of every
// (request, head), an item and a rest of every head's own rows, and their plan.
constexpr int64_t attn_part_rows_for(int batch, int heads, int kv_heads) {
  const int64_t two = 2 * (int64_t)batch * heads, usual = (two > 65536 ? two : 65536) + 8192;
  const int64_t prefix = (int64_t)batch * heads + (int64_t)own_items_for(batch, kv_heads) * heads + own_plan_rows_for(batch, kv_heads);
  return usual > prefix ? usual : prefix;
}

}  // namespace lfps
