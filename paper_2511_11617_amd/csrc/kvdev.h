// kvdev.h — what the KV cache operators' device code shares: types,
// conversions, head runs and places in the cache, and the launch checks.
#pragma once
#include <hip/hip_runtime.h>

#include <string>

#include "kvops.h"
#include "plan.h"

namespace atp {

// A failed call also stays the thread's last HIP error, which the caller's
// next launch check would report as its own: it is reported here, so it is
// cleared.
inline void kv_hip(hipError_t e, const char *what) {
  if (e == hipSuccess) return;
  (void)hipGetLastError();
  throw Error(ATP_EHIP, std::string(what) + ": " + hipGetErrorString(e));
}

// The kernels are loaded for, and run on, the current device: a stream of
// another one is refused.
inline hipStream_t kv_stream(void *stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  int cur = 0, dev = 0;
  kv_hip(hipGetDevice(&cur), "hipGetDevice");
  if (s) {
    kv_hip(hipStreamGetDevice(s, &dev), "hipStreamGetDevice");
    if (dev != cur) throw Error(ATP_EINVAL, "stream belongs to another device than the current one");
  }
  return s;
}

using bf16x2 = __bf16 __attribute__((ext_vector_type(2)));
using f16x2 = _Float16 __attribute__((ext_vector_type(2)));
using f32x2 = float __attribute__((ext_vector_type(2)));
using u32x2_t = uint32_t __attribute__((ext_vector_type(2)));
using u32x4_t = uint32_t __attribute__((ext_vector_type(4)));

struct E4M3 {
  uint8_t b;
};

template <typename T>
__device__ inline float as_f32(T x) {
  return float(x);
}
template <>
__device__ inline float as_f32<E4M3>(E4M3 x) {
  return __builtin_amdgcn_cvt_f32_fp8(x.b, 0);
}

// Rounded once, to the nearest (ties to even).  E4M3 has no infinity: what
// lies beyond 448 becomes 448; a NaN stays one.
template <typename T>
__device__ inline T rounded(float x) {
  return T(x);
}
template <>
__device__ inline E4M3 rounded<E4M3>(float x) {
  x = x > 448.0f ? 448.0f : x < -448.0f ? -448.0f : x;
  return {uint8_t(__builtin_amdgcn_cvt_pk_fp8_f32(x, 0.0f, 0, false) & 0xff)};
}

__device__ inline void flag(int32_t *status, int32_t code) {
  if (status) __hip_atomic_store(status, code, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

}  // namespace atp
