// Host-side argument checks shared by the entry points of the C ABI (kdn_api.hip holds the
// definitions and the calling thread's error text).
#pragma once

#include <cstdint>
#include <initializer_list>
#include <utility>

#include "kdn_internal.h"

namespace kdn {

// Sets the calling thread's error text and returns the status; ok() clears it.
kdn_status_t fail(kdn_status_t st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
kdn_status_t ok();
kdn_status_t hip_status(hipError_t e, const char* what);

inline bool head_ok(int d) { return d == 16 || d == 32 || d == 64 || d == 128; }

inline size_t esize(kdn_dtype_t dt) { return dt == KDN_F32 ? 4 : 2; }

// Byte ranges [p, p + n) and [q, q + m) overlap.
bool overlaps(const void* p, size_t n, const void* q, size_t m);

// Tensors whose innermost dimension is d_k or d_v are read and written in 16-byte pieces: each
// must start at a 16-byte boundary (null pointers are skipped).
kdn_status_t check_aligned(std::initializer_list<std::pair<const void*, const char*>> ptrs);

// Sizes of a batch of sequences, packed or not.
kdn_status_t check_seq(const int32_t* cu, int32_t N, int32_t B, int32_t T, int32_t H);

}  // namespace kdn
