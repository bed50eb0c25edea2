// Host-side helpers of the C ABI's files (internal to the library).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/tactic.h"
#include "kernels.hpp"

namespace tactic_host {

// Sets the calling thread's message and returns the status.
tactic_status fail(tactic_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
tactic_status hip_fail(hipError_t e, const char* what);

inline int64_t align_up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

struct Layout {
  int64_t cur = 0;
  int64_t take(int64_t bytes) {
    const int64_t o = cur;
    cur = align_up(cur + bytes, 256);
    return o;
  }
};

// Memory that a call reads or writes; a null or empty one overlaps nothing.
struct Span {
  const void* at;
  int64_t bytes;
};
inline bool overlap(const Span& a, const Span& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
  return x && y && a.bytes > 0 && b.bytes > 0 && x < y + (uintptr_t)b.bytes && y < x + (uintptr_t)a.bytes;
}

tactic_status check_shape(const tactic_kv_shape* s);
tactic_status check_mod(const tactic_score_mod* m);
tactic_status paged_args(const tactic_paged_kv* kv, const tactic_kv_shape* s, tactic::PagedKV* pk);
size_t dense_workspace_bytes(const tactic_kv_shape* s, int64_t grid);

}  // namespace tactic_host
