// Device-side pieces shared by the streaming kernels: the server's update of one parameter, rounding to bf16, loads by type.
#pragma once
#include <hip/hip_runtime.h>

#include "asgd_internal.h"
#include "mfma_common.h"

namespace asgd {

typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ inline float ldf(const float *p) { return *p; }
__device__ inline float ldf(const bf16_t *p) { return (float)*p; }
__device__ inline void stf(float *p, float v) { *p = v; }
__device__ inline void stf(bf16_t *p, float v) { *p = (bf16_t)v; }

static inline unsigned blocks_for(size_t n, unsigned per_block) { return (unsigned)((n + per_block - 1) / per_block); }
static inline int launch_ok() { return hipGetLastError() == hipSuccess ? 0 : -1; }

// One element of the update, with the contractions written out so that every code path (vector body, scalar
// tail, unaligned fallback) rounds identically: t = g + wd*w;  v = mu*v - lr*t;  w = w + v.
__device__ __forceinline__ void update1(float &w, float &v, float g, float lr, float mu, float wd)
{
    const float t = __builtin_fmaf(wd, w, g);
    v = __builtin_fmaf(mu, v, -(lr * t));
    w = w + v;
}

template <bool ONCE> __device__ __forceinline__ f32x4 load4(const f32x4 *p)
{
    if constexpr (ONCE) return __builtin_nontemporal_load(p);
    else return *p;
}

__device__ inline uint32_t f32_to_bf16_bits(uint32_t u)  // round to nearest even; NaN -> quiet NaN
{
    if ((u & 0x7F800000u) == 0x7F800000u && (u & 0x007FFFFFu)) return (u >> 16) | 0x0040u;
    return (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
}
__device__ __forceinline__ uint2 bf16x4(const f32x4 &v)
{
    return make_uint2(f32_to_bf16_bits(__float_as_uint(v.x)) | (f32_to_bf16_bits(__float_as_uint(v.y)) << 16),
                      f32_to_bf16_bits(__float_as_uint(v.z)) | (f32_to_bf16_bits(__float_as_uint(v.w)) << 16));
}

}  // namespace asgd
