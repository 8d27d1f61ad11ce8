// What the operators on device arrays share: element types, loads and stores at any alignment, powers of a decay.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>
#include "../../include/ob.h"
#include "ob_internal.h"

typedef __bf16 bf16;
typedef _Float16 f16;
typedef float f4 __attribute__((ext_vector_type(4)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef short s8 __attribute__((ext_vector_type(8)));
typedef int64_t i64;

// Loads and stores of N elements as one access.  Global memory takes wide accesses at any alignment of the element, so that odd widths and
// strides need no path of their own.
template <typename T, int N> struct __attribute__((packed, aligned(sizeof(T)))) Pack { typedef T V __attribute__((ext_vector_type(N))); V v; };
template <typename T, int N> __device__ __forceinline__ typename Pack<T, N>::V load_n(const T *p) { return ((const Pack<T, N> *)p)->v; }
template <typename T, int N> __device__ __forceinline__ void store_n(T *p, typename Pack<T, N>::V v) { ((Pack<T, N> *)p)->v = v; }

// lambda^n for a whole n >= 0, given log lambda <= 0 (-inf allowed: 0^0 = 1).  The rounding of the product n * g is put back, so that powers
// over many tokens are as exact as the function itself.
__device__ __forceinline__ float decay_power(float g, int n)
{
    if (n <= 0) return 1.0f;
    const float x = (float)n, p = x * g;
    if (!(p > -104.0f) && p <= 0.0f) return 0.0f;   // below the smallest fp32 (a NaN goes on)
    const float r = __builtin_fmaf(x, g, -p);
    return expf(p) * (1.0f + r);
}

// the message and code of a failed call (ob_last_error(NULL))
int ops_fail(int code, const char *fmt, ...);
static inline int ops_launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? OB_OK : ops_fail(OB_E_HIP, "%s: %s", what, hipGetErrorString(e));
}
// threads of a launch along one axis are counted in 32 bits
static inline bool launch_fits(i64 blocks, int threads) { return blocks <= 0xffffffffll / threads; }
