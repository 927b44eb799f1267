// What the translation units of libpab.so share; nothing here is exported.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "../../include/pab.h"

#define PAB_HIDDEN __attribute__((visibility("hidden")))

namespace pab {

// Records the calling thread's error text (pab_last_error) and returns `code`.
PAB_HIDDEN int fail(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Blocks of 128 columns from which on a matrix is too large for the quantiser: 16 threads for each are 2^32, one more than a grid holds
constexpr long long Q8_BLOCKS = 1LL << 28;
// 8-bit rows of [rows, K] in one buffer, as pab_quantized_layout places them: bytes (0: too large), and the matrix at `buffer`
PAB_HIDDEN size_t q8_bytes(long long rows, long long K);
PAB_HIDDEN pab_q8 q8_at(void *buffer, long long rows, long long K);
// checked launch of the quantising pass
PAB_HIDDEN int quantize(long long rows, int K, int dtype, const void *x, long long ldx, const pab_q8 *y, hipStream_t st);

}  // namespace pab
