// Shared by the operators of quantised transformer blocks (include/miquant.h).
#pragma once

#include "../../include/miconv.h"
#include "../../include/miquant.h"
#include "internal.h"

#include <string.h>

namespace miconv {
namespace quant {

constexpr int kF32 = 0, kBF16 = 1;   // dtype codes of the ABI
inline int dtype_bytes(int dtype) { return dtype == kF32 ? 4 : dtype == kBF16 ? 2 : 0; }
inline bool misaligned(const void *p, int bytes) { return (uintptr_t)p % (uintptr_t)bytes != 0; }
// A launch's status as the entry points return it.
inline int launched()
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? MICONV_OK : set_hip_error(e);
}

// n elements (8 at most) of a row, widened to fp32.  Whole units are one or
// two 16-byte accesses at element alignment, which global memory takes at any
// address; a row's last elements go one by one.
__device__ __forceinline__ void load8(const float *p, float (&v)[8]) { memcpy(v, p, 32); }
__device__ __forceinline__ void load8(const uint16_t *p, float (&v)[8])
{
    uint32_t raw[4];
    memcpy(raw, p, 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __builtin_bit_cast(float, raw[i] << 16);
        v[2 * i + 1] = __builtin_bit_cast(float, raw[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void load4(const float *p, float (&v)[4]) { memcpy(v, p, 16); }
__device__ __forceinline__ void load4(const uint16_t *p, float (&v)[4])
{
    uint32_t raw[2];
    memcpy(raw, p, 8);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        v[2 * i] = __builtin_bit_cast(float, raw[i] << 16);
        v[2 * i + 1] = __builtin_bit_cast(float, raw[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void store4(float *p, const float (&v)[4]) { memcpy(p, v, 16); }
__device__ __forceinline__ void store4(uint16_t *p, const float (&v)[4])
{
    const uint32_t raw[2] = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    memcpy(p, raw, 8);
}
__device__ __forceinline__ float load1(const float *p) { return *p; }
__device__ __forceinline__ float load1(const uint16_t *p) { return bf16_to_f32(*p); }
__device__ __forceinline__ void store8(float *p, const float (&v)[8]) { memcpy(p, v, 32); }
__device__ __forceinline__ void store8(uint16_t *p, const float (&v)[8])
{
    uint32_t raw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) raw[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    memcpy(p, raw, 16);
}
__device__ __forceinline__ void store1(float *p, float v) { *p = v; }
__device__ __forceinline__ void store1(uint16_t *p, float v) { *p = (uint16_t)pack_bf16x2(v, v); }

// v rounded to T, as fp32.
__device__ __forceinline__ float rounded(float v, const float *) { return v; }
__device__ __forceinline__ float rounded(float v, const uint16_t *)
{
    return __builtin_bit_cast(float, pack_bf16x2(v, v) & 0xFFFF0000u);
}

// The 4-bit cache as kernels see it.
struct Kv4 {
    uint8_t *kc, *ke, *vc, *ve;
    long slots;            // pages * page_size
    int heads, page_size, dim;
    FastDiv dv_page;
};
// Validates a cache descriptor and fills `out`.
int kv4_view(const quant_kv4 *c, Kv4 *out);

constexpr int kMaxExp = 252;   // exponent bytes above stand for groups that are not finite

}  // namespace quant
}  // namespace miconv
