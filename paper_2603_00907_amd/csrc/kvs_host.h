// Checks that the host layers of libkvs share.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "kvs.h"

namespace kvs {

constexpr size_t kAlign = 256;           // of workspaces and of what is carved from them
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

// A buffer that a call reads or writes.
struct Range {
  const void* p;
  size_t bytes;
  bool is_output;
};

// Every buffer is there and 16-byte aligned, and no output overlaps another buffer.
inline kvs_status check_ranges(const Range* rs, size_t n) {
  for (size_t i = 0; i < n; ++i) {
    if (rs[i].p == nullptr || ((uintptr_t)rs[i].p & 15u) != 0) return KVS_ERR_INVALID_ARG;
  }
  for (size_t i = 0; i < n; ++i) {
    if (!rs[i].is_output) continue;
    for (size_t j = 0; j < n; ++j) {
      if (i == j) continue;
      const char* a0 = (const char*)rs[i].p;
      const char* b0 = (const char*)rs[j].p;
      if (a0 < b0 + rs[j].bytes && b0 < a0 + rs[i].bytes) return KVS_ERR_ALIAS;
    }
  }
  return KVS_OK;
}

}  // namespace kvs
