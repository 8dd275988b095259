// How many pages a call takes and how many of them are copies, as one 64-bit number, so that one
// prefix sum gives both.  No HIP in here: the host's checks and a host test use it too.
//
// Bits 0 .. 37 hold the pages.  A sequence asks for no more than its row of the table has entries (a copy
// takes the place of an entry that it holds, new pages lie behind those), so all of them together for fewer than
// KV_MAX_ENTRIES, which the entry points see to.  The bits from 38 on hold the copies, one a sequence at
// most: 2^24 of them at the most sequences, 2^62 in all, so that the number stays positive.
#pragma once

#include <stdint.h>

namespace saki {

constexpr int64_t KV_MAX_SEQ = int64_t{1} << 24;
constexpr int KV_COPY_BIT = 38;
constexpr int64_t KV_MAX_ENTRIES = int64_t{1} << KV_COPY_BIT;  // (of 4 bytes each: 1 TB)

constexpr int64_t kv_count(bool copy, int32_t fresh) {
  return (static_cast<int64_t>(copy) << KV_COPY_BIT) + fresh + copy;
}
constexpr int64_t kv_count_pages(int64_t sum) { return sum & (KV_MAX_ENTRIES - 1); }
constexpr int64_t kv_count_copies(int64_t sum) { return sum >> KV_COPY_BIT; }

static_assert(KV_MAX_SEQ <= (INT64_MAX >> KV_COPY_BIT), "a copy for every sequence fits");

}  // namespace saki
