// What the calls on a spd_cache share: the checks of their arguments and the bounds that the kernels keep.
// Internal; not part of the C ABI.
#pragma once
#include <string>

#include "spd_dev.h"

namespace spd {

constexpr int kPage = 16;            // keys of a page
constexpr int kMaxSeqs = 65536;      // sequences of a cache
constexpr int kMaxPages = 1 << 26;   // pages of a sequence: 16 * kMaxPages keys fit in an int

void set_call_error(const std::string& msg);  // spd_last_error(NULL) (spd_api.cpp)

inline spd_status invalid(const char* call, const char* what) {
  set_call_error(std::string(call) + ": " + what);
  return SPD_E_INVAL;
}

inline bool misaligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) != 0; }

// The description of a cache; pages: whether the call changes which pages the sequences hold.
spd_status check_cache(const char* call, const spd_cache* c, bool pages);
spd_status check_workspace(const char* call, const void* ws, size_t bytes, size_t need);
// Rows of `heads` heads of dtype, `stride` elements apart.
spd_status check_rows(const char* call, const void* p, int64_t stride, int heads, int head_dim, int dtype);
spd_status check_launch(const char* call);  // hipGetLastError

inline size_t elem_bytes(int dtype) { return dtype == SPD_BF16 ? 2 : 4; }

}  // namespace spd
