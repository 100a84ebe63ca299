// Argument checks shared by the C-ABI layer's sources.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "hilore.h"

namespace {

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline bool valid_block(int block) { return block == 32 || block == 64 || block == 128 || block == 256; }

inline bool valid_code(int code) {
  return code == HILORE_CODE_INT8 || code == HILORE_CODE_FP8_E4M3FN ||
         code == HILORE_CODE_FP8_E4M3FN_CAST;
}

// The blockwise codes need a supported block size; the literal cast has no
// blocks and takes block == 0.
inline hilore_status check_code_block(int code, int block) {
  if (!valid_code(code)) return HILORE_ERR_INVALID_ARG;
  if (code == HILORE_CODE_FP8_E4M3FN_CAST) return block == 0 ? HILORE_OK : HILORE_ERR_INVALID_ARG;
  return valid_block(block) ? HILORE_OK : HILORE_ERR_UNSUPPORTED;
}

inline hilore_status hip_status(hipError_t e) { return e == hipSuccess ? HILORE_OK : HILORE_ERR_HIP; }

}  // namespace
