// What the operators on matrices of rows share: elements and their types, checks of arguments, the device's width.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <string>

#include "tdf_internal.h"

namespace tdf {
namespace rows {

// Kernels are instantiated on the tdf_dtype value (readable names in profiles), not on the type.
template <int DT> struct TypeOf;
template <> struct TypeOf<TDF_F32> { typedef float type; };
template <> struct TypeOf<TDF_BF16> { typedef __bf16 type; };

// ---- host --------------------------------------------------------------------------------------
inline size_t element_size(int32_t dtype) { return dtype == TDF_BF16 ? 2 : 4; }
inline bool known_type(int32_t dtype) { return dtype == TDF_F32 || dtype == TDF_BF16; }
inline tdf_status refuse(const char* who, const char* what) {
  set_error(std::string(who) + ": " + what);
  return TDF_ERR_BAD_ARG;
}
inline tdf_status launched(const char* who) {
  const hipError_t err = hipGetLastError();
  if (err == hipSuccess) return TDF_OK;
  set_error(std::string(who) + ": " + hipGetErrorString(err));
  return TDF_ERR_DEVICE;
}
// A matrix argument: there, aligned to its elements, rows that do not overlap, byte offsets within 63 bits.
inline const char* bad_matrix(const void* p, int64_t ld, int64_t n_rows, int64_t n_cols, size_t size) {
  if (!p) return "a matrix is NULL";
  if ((uintptr_t)p % size) return "a matrix is not aligned to its elements";
  if (ld < n_cols) return "the distance between rows is smaller than a row";
  if (n_rows > 0 && ld > (int64_t)(1ll << 59) / n_rows) return "a matrix is too large";
  return nullptr;
}
inline bool bad_floats(const void* p) { return (uintptr_t)p % 4 != 0; }
// Two vectors of n floats each, either of which may be NULL, have elements in common.
inline bool overlap(const void* p, const void* q, int64_t n) {
  const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
  return a && b && (a < b ? b - a : a - b) / sizeof(float) < (uintptr_t)n;
}
// The threads of a launch are counted in 32 bits: f(first, count) for runs of at most `most` of n rows.
constexpr int64_t MOST_WORKGROUPS = 1 << 23;
template <class F> void in_runs(int64_t n, int64_t most, F&& f) {
  for (int64_t first = 0; first < n; first += most) f(first, n - first < most ? n - first : most);
}
// Rows begin at multiples of `bytes`.
inline bool aligned(const void* p, int64_t ld, size_t size, size_t bytes) { return ((uintptr_t)p | (uintptr_t)(ld * (int64_t)size)) % bytes == 0; }

}  // namespace rows
}  // namespace tdf
