// What the C ABI entry points of the layer and token operators check of their arguments.
#ifndef MOSAIC_ARGUMENTS_H_
#define MOSAIC_ARGUMENTS_H_

#include <stdint.h>

#include "mosaic_layer.h"

namespace mosaic {
namespace arguments {

constexpr int64_t kMaxRows = (int64_t)1 << 31;
constexpr int64_t kMaxStride = (int64_t)1 << 21;   // elements: 256 rows of a tile stay within 2^31 bytes

inline bool misaligned(const void* p, uintptr_t bytes = 16) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

// A [rows, cols] matrix argument.  INVALID_ARG: absent or misaligned; UNSUPPORTED_SHAPE: a stride the kernels do not take.
inline int check_matrix(const void* p, int64_t ld, int64_t cols) {
  if (p == nullptr || misaligned(p)) return MOSAIC_ERR_INVALID_ARG;
  if (ld < cols || ld % 8 != 0 || ld > kMaxStride) return MOSAIC_ERR_UNSUPPORTED_SHAPE;
  return MOSAIC_OK;
}
inline int check_optional(const void* p, int64_t ld, int64_t cols) { return p == nullptr ? MOSAIC_OK : check_matrix(p, ld, cols); }

inline int check_sizes(int64_t T, int64_t cols, int64_t most) {
  if (T < 0 || cols <= 0) return MOSAIC_ERR_INVALID_ARG;
  if (T >= kMaxRows || cols % 8 != 0 || cols > most) return MOSAIC_ERR_UNSUPPORTED_SHAPE;
  return MOSAIC_OK;
}

inline bool known_type(int32_t t) { return t == MOSAIC_BF16 || t == MOSAIC_F32; }

inline int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

inline int launched(int rc) { return rc == 0 ? MOSAIC_OK : MOSAIC_ERR_HIP; }

#define MOSAIC_RETURN_IF(expr)                  \
  do {                                          \
    const int status_ = (expr);                 \
    if (status_ != MOSAIC_OK) return status_;   \
  } while (0)

}  // namespace arguments
}  // namespace mosaic
#endif
