// The paged cache in 8 bits as the kernels see it.
//
// Block = 64 tokens.  A complete block of a kv head is 8 KiB of keys, e4m3 [64 tokens][128], and 8 KiB of
// values, e4m3 [128][64 tokens], each with one scale, a power of two.  Values lie transposed because that is
// how the second product of the attention takes them: sixteen bytes are sixteen tokens of one channel, an
// operand of two matrix instructions as they come from memory.  The block that is still open and the draft
// rows behind it are bf16 rows of a ring, position p at row p % 128, so rows stay where they are when they
// are accepted, and every value is rounded to 8 bits once, with the scale of its whole block.
#pragma once

#include "lvspec_dev.h"
#include "lvspec_kernels.h"

namespace lvspec {

constexpr int kPageShift = 6;
constexpr int kPageTokens = 1 << kPageShift;
constexpr int kPageBytes = kPageTokens * 128;      // keys or values of one head
constexpr int kTailRows = 128;
static_assert(kPageTokens == LVSPEC_PAGE_TOKENS && kTailRows == LVSPEC_TAIL_ROWS, "public constants");

// A length as the kernels take it: inside what the table can name and the ring can hold.
LVS_DEV int paged_len(int len, int cols) {
  const int most = cols * kPageTokens + kPageTokens - 1;
  return len < 0 ? 0 : len > most ? most : len;
}

}  // namespace lvspec
