// Host-side checks that the entry points of a paged cache share.
#pragma once

#include "ec_paged.cuh"

namespace ec {

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline size_t round256(size_t x) { return (x + 255) / 256 * 256; }

// The caller owns the struct: every call repeats these checks.
int check_paged(const ec_paged *c);
PagedView view(const ec_paged *c);
int check_ws(const void *ws, size_t have, size_t need);

}  // namespace ec
