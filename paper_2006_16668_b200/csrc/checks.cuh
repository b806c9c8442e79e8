// Argument checks shared by the C entry points.
#pragma once
#include "common.cuh"

namespace gshard {

int check_device();   // api.cu: GSHARD_OK when the current device is sm_100

inline bool is_aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// required / optional tensor pointer: 16-byte aligned
#define GS_CHECK_PTR(p)                                                               \
  do {                                                                                \
    if ((p) == nullptr || !::gshard::is_aligned16(p)) return GSHARD_ERR_INVALID_ARG;  \
  } while (0)
#define GS_CHECK_OPTIONAL_PTR(p)                                   \
  do {                                                             \
    if (!::gshard::is_aligned16(p)) return GSHARD_ERR_INVALID_ARG; \
  } while (0)
#define GS_CHECK_WORKSPACE(p, have, need)                                                            \
  do {                                                                                               \
    if ((p) == nullptr || reinterpret_cast<uintptr_t>(p) % ::gshard::kAlign) return GSHARD_ERR_INVALID_ARG; \
    if ((have) < (need)) return GSHARD_ERR_WORKSPACE_TOO_SMALL;                                      \
  } while (0)
#define GS_CHECK(expr)                     \
  do {                                     \
    const int _rc = (expr);                \
    if (_rc != GSHARD_OK) return _rc;      \
  } while (0)

}  // namespace gshard
