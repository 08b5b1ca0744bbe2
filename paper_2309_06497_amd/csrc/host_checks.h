// What the host code of every operator beside the Shampoo step uses: argument checks, workspaces, launches that may fail.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/shampoo.h"

namespace shampoo {

constexpr size_t ALIGN = 256;

inline size_t align_up(size_t x) { return (x + ALIGN - 1) / ALIGN * ALIGN; }
inline int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
inline bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
inline bool dtype_ok(int32_t d) { return d == SHAMPOO_GRAD_F32 || d == SHAMPOO_GRAD_BF16; }
inline int64_t size_of(int32_t d) { return d == SHAMPOO_GRAD_F32 ? 4 : 2; }

#define HIP_TRY(expr)                          \
  do {                                         \
    hipError_t e_ = (expr);                    \
    if (e_ != hipSuccess) return SHAMPOO_ERR_HIP; \
  } while (0)
#define TRY(...)                               \
  do {                                         \
    const int rc_ = (__VA_ARGS__);             \
    if (rc_ != SHAMPOO_OK) return rc_;         \
  } while (0)

// Workspaces: arrays one behind the other
struct Arena {
  unsigned char *base; size_t used = 0;
  explicit Arena(void *p) : base(static_cast<unsigned char *>(p)) {}
  template <typename T> T *take(size_t count) {
    T *p = reinterpret_cast<T *>(base + used);
    used += align_up(count * sizeof(T));
    return p;
  }
};
inline int workspace_ok(const void *p, size_t have, size_t want) {
  return want > 0 && (!p || !aligned(p, ALIGN) || have < want) ? SHAMPOO_ERR_WORKSPACE : SHAMPOO_OK;
}

}  // namespace shampoo
