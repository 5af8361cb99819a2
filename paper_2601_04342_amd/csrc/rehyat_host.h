// What the host layers of the library share.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/rehyat.h"

namespace rehyat {

// keeps the error's text for rehyat_last_hip_error; returns REHYAT_E_HIP
int hip_fail(hipError_t e, const char* what);

inline bool aligned(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }
inline bool aligned16(const void* p) { return aligned(p, 16); }
inline bool aligned4(const void* p) { return aligned(p, 4); }
inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Whether two ranges of bytes are apart.
inline bool ranges_apart(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
  return (uintptr_t)a + (uintptr_t)a_bytes <= (uintptr_t)b || (uintptr_t)b + (uintptr_t)b_bytes <= (uintptr_t)a;
}

// Whether a pass over so many bytes goes past the caches (non-temporal loads and stores): what does not fit the 256 MB in
// front of the memory is gone when the next pass comes, and what fits is there.  Each user has both sides measured.
inline bool past_caches(int64_t bytes) { return bytes > ((int64_t)256 << 20); }

inline bool valid_type(int t) { return t == REHYAT_BF16 || t == REHYAT_FP16 || t == REHYAT_FP32; }
inline size_t type_bytes(int t) { return t == REHYAT_FP32 ? 4 : 2; }

}  // namespace rehyat
