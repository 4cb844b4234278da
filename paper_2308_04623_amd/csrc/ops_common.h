// What the operators of ssd_ops.h share: element types, loads, reductions and
// the host's error reporting.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/ssd_ops.h"

namespace ssd {

// records the message for ssd_last_error and returns the status (runtime.hip)
ssd_status op_fail(ssd_status st, const char* msg) noexcept;

#define OP_REQUIRE(cond, status, msg) \
  do {                                \
    if (!(cond)) return ssd::op_fail(status, msg); \
  } while (0)
// after a launch: its status
#define OP_LAUNCHED()                                                                   \
  do {                                                                                  \
    hipError_t e_ = hipGetLastError();                                                  \
    if (e_ != hipSuccess) return ssd::op_fail(SSD_E_DEVICE, hipGetErrorString(e_));     \
  } while (0)

inline bool op_dtype(int t) { return t == SSD_F32 || t == SSD_BF16; }
inline int op_size(int t) { return t == SSD_F32 ? 4 : 2; }
// whether [a, a + na) and [b, b + nb) share a byte
inline bool op_overlap(const void* a, size_t na, const void* b, size_t nb) {
  return (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}
// Elements in memory, those of up to four dimensions.
struct OpView {
  const void* p;
  struct Dim {
    int64_t n, step;  // in bytes, not negative
  } dims[4];          // (the last: the elements that lie side by side)
};
// Whether two views are sure to share no byte: their bytes lie apart, or, modulo a step that divides all
// larger ones, what either has of smaller steps does (parts of the rows, heads or
// tokens of one buffer).  Others count as overlapping.
inline bool op_apart(const OpView& a, const OpView& b) {
  // bytes from the first to past the last, of dimensions whose steps are below `most`
  auto extent = [](const OpView& v, int64_t most) {
    int64_t e = 0;
    for (const auto& d : v.dims) {
      if (d.n <= 0) return (int64_t)0;
      if (d.step < most) e += (d.n - 1) * d.step;
    }
    return e + v.dims[3].step;
  };
  const int64_t ea = extent(a, INT64_MAX), eb = extent(b, INT64_MAX);
  if (ea == 0 || eb == 0 || !op_overlap(a.p, (size_t)ea, b.p, (size_t)eb)) return true;
  auto proves = [&](int64_t step) {
    for (const OpView* v : {&a, &b})
      for (const auto& d : v->dims)
        if (d.n > 1 && d.step >= step && d.step % step != 0) return false;
    const int64_t from = (((int64_t)((intptr_t)b.p - (intptr_t)a.p)) % step + step) % step;
    return extent(a, step) <= from && from + extent(b, step) <= step;
  };
  for (const OpView* v : {&a, &b})
    for (const auto& d : v->dims)
      if (d.n > 1 && d.step > 0 && proves(d.step)) return true;
  return false;
}
inline OpView op_matrix(const void* p, int64_t rows, int64_t ld, int64_t cols, int size) {
  return {p, {{1, 0}, {1, 0}, {rows, ld * size}, {cols, size}}};
}

struct bf16_t {
  uint16_t bits;
};

__device__ __forceinline__ float op_ld(const float* p, size_t i) { return p[i]; }
__device__ __forceinline__ float op_ld(const bf16_t* p, size_t i) {
  return __uint_as_float((uint32_t)p[i].bits << 16);
}
// (to bfloat16: nearest, ties to even)
__device__ __forceinline__ void op_st(float* p, size_t i, float v) { p[i] = v; }
__device__ __forceinline__ void op_st(bf16_t* p, size_t i, float v) {
  p[i].bits = __builtin_bit_cast(uint16_t, (__bf16)v);
}

}  // namespace ssd
