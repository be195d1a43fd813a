// What the operators' source (kvops.hip) needs beyond the stand-in HIP runtime (mockhip) to be compiled by a host compiler.  Their kernels
// are compiled but not run: launches are recorded.  The device's own instructions are replaced by anything of the same type.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#undef __launch_bounds__
#define __launch_bounds__(...)
#define __forceinline__ inline
#ifndef __HIP_MEMORY_SCOPE_AGENT
#define __HIP_MEMORY_SCOPE_AGENT 4
#endif
#define __hip_atomic_fetch_add(p, v, order, scope) __atomic_fetch_add(p, v, order)
#define __hip_atomic_store(p, v, order, scope) __atomic_store_n(p, v, order)
#define __hip_atomic_load(p, order, scope) __atomic_load_n(p, order)
#define __builtin_amdgcn_cosf(x) cosf(x)
#define __builtin_amdgcn_sinf(x) sinf(x)
#define __builtin_amdgcn_exp2f(x) exp2f(x)
#define __builtin_amdgcn_cvt_pk_fp8_f32(a, b, old, high) ((int)((a) + (b)) + (old))
#define __builtin_amdgcn_cvt_f32_fp8(x, byte) ((float)((x) >> 8 * (byte) & 255))
#define __builtin_amdgcn_update_dpp(old, x, ctrl, rows, banks, bound) ((old) + (x))
#define __builtin_amdgcn_s_sleep(n) ((void)0)
#define __popc(x) __builtin_popcount(x)
// "asm volatile(...)" of device code
#define asm
#define volatile(...)

struct float2 {
  float x, y;
};
using std::max;
using std::min;
inline int atomicMax(int* p, int v) { const int old = *p; *p = std::max(old, v); return old; }

enum { hipEventDisableTiming = 2 };
inline hipError_t hipEventCreateWithFlags(hipEvent_t* e, unsigned) { return hipEventCreate(e); }
// Waits for every stream that the program has named here.
inline std::vector<hipStream_t> all_streams;
inline long device_waits = 0;
inline hipError_t hipDeviceSynchronize() {
  device_waits++;
  hipError_t e = hipSuccess;
  for (hipStream_t s : all_streams)
    if (hipStreamSynchronize(s) != hipSuccess) e = hipErrorUnknown;
  return e;
}
