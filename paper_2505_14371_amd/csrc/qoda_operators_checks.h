// Checks of arguments that the operators' calls share, and where they leave what they found wrong.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "../../include/qoda_operators.h"
#include "qoda_operators.h"

namespace qoda {

inline thread_local char operator_error[256] = "";   // qoda_operator_error()

inline int fail(int code, const char *fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(operator_error, sizeof operator_error, fmt, ap);
  va_end(ap);
  return code;
}

inline int done(const char *call, hipError_t e) {
  if (e == hipSuccess) return QODA_OK;
  return fail(e == hipErrorOutOfMemory ? QODA_ENOMEM : QODA_EHIP, "%s: %s", call, hipGetErrorString(e));
}

constexpr int64_t kMostSide = QODA_MAX_SIDE;   // rows and columns: the kernels' 32-bit indexes go a tile beyond them
constexpr int64_t kMostStride = (int64_t)1 << 40;

inline size_t entry_bytes(int type) { return type == kF32 ? 4 : 2; }

inline bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// A matrix of rows x cols entries of `bytes` each; one without entries is not looked at.
inline int check_matrix(const char *call, const char *name, const qoda_matrix &m, int64_t rows, int64_t cols, size_t bytes, bool optional) {
  if (rows == 0 || cols == 0) return QODA_OK;
  if (!m.data) return optional ? QODA_OK : fail(QODA_EINVAL, "%s: %s is null", call, name);
  if (!aligned(m.data, bytes)) return fail(QODA_EINVAL, "%s: %s is not aligned to its entries", call, name);
  if (rows > 1 && (m.stride < cols || m.stride >= kMostStride))
    return fail(QODA_EINVAL, "%s: %s has a stride of %lld entries and rows of %lld", call, name, (long long)m.stride, (long long)cols);
  return QODA_OK;
}

inline int check_common(const char *call, int32_t dtype, int32_t activation) {
  if (dtype != QODA_F32 && dtype != QODA_BF16) return fail(QODA_EINVAL, "%s: dtype %d is none", call, dtype);
  if (activation < 0 || activation >= kNumActivations) return fail(QODA_EINVAL, "%s: activation %d is none", call, activation);
  return QODA_OK;
}

inline int check_sides(const char *call, int64_t a, int64_t b, int64_t c) {
  for (const int64_t v : {a, b, c})
    if (v < 0 || v > kMostSide) return fail(QODA_EINVAL, "%s: a size of %lld is not in [0, %lld]", call, (long long)v, (long long)kMostSide);
  return QODA_OK;
}

inline int make_drop(const char *call, double p, uint64_t seed, uint64_t offset, Drop *d) {
  if (!(p >= 0.0 && p <= 1.0)) return fail(QODA_EINVAL, "%s: p = %g is not in [0, 1]", call, p);
  const unsigned int t = (unsigned int)std::floor(p * 65536.0 + 0.5);
  const uint64_t key = seed ^ QODA_DROPOUT_KEY;
  *d = {t, (t << 16) - 1u, t < 65536u ? (float)(65536.0 / (65536u - t)) : 0.0f, (unsigned int)key, (unsigned int)(key >> 32), (unsigned int)offset,
        (unsigned int)(offset >> 32)};
  return QODA_OK;
}

inline int check_workspace(const char *call, const void *p, size_t have, size_t need) {
  if (need == 0) return QODA_OK;
  if (!p || have < need) return fail(QODA_EINVAL, "%s: %zu bytes of workspace are needed, %zu are there", call, need, p ? have : (size_t)0);
  if (!aligned(p, 16)) return fail(QODA_EINVAL, "%s: the workspace is not aligned to 16 bytes", call);
  return QODA_OK;
}

// One row's stride is never used; the kernels get one that would fit, so that their checks of alignment go by it.
inline long long stride_of(const qoda_matrix &m, int64_t rows, int64_t cols) { return rows > 1 ? m.stride : cols; }

#define TRY(call)                          \
  do {                                     \
    const int rc_ = (call);                \
    if (rc_ != QODA_OK) return rc_;        \
  } while (0)

}  // namespace qoda
