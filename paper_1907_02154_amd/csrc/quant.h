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

// A paged cache as kernels see it.
struct KvView {
    uint8_t *kc, *ke, *vc, *ve;
    long slots;            // pages * page_size
    int heads, page_size, dim;
    FastDiv dv_page;
    int block, blocks;     // places that share an exponent, and such blocks in a page (8-bit cache)
    FastDiv dv_block;
};
// Validates a cache descriptor and fills `out`.
int kv4_view(const quant_kv4 *c, KvView *out);
int kv8_view(const quant_kv8 *c, KvView *out);

constexpr int kMaxExp = 252;   // 4-bit cache: exponent bytes above stand for groups that are not finite

// ------------------------------------------------------------------ 8-bit floating point in blocks
//
// e4m3 values (largest 448 = 1.75 * 2^8) that share 2^e, e the smallest in
// -117 .. 119 with max|x| <= 448 * 2^e: every value is a normal fp32 and bf16
// number or 0, and finite.
constexpr int kF8Block = 128;                    // values of a row that share an exponent
constexpr int kF8Lo = 127 - 117, kF8Hi = 127 + 119;   // exponent bytes that are written

// The exponent byte of a block from its largest magnitude's bits.
__device__ __forceinline__ int f8_byte(uint32_t top)
{
    // 8 below top's exponent, 7 below it where its significand passes 1.75
    const int e = (int)(top >> 23) - 8 + ((top & 0x7FFFFFu) > 0x600000u);
    return e < kF8Lo ? kF8Lo : e > kF8Hi ? kF8Hi : e;
}
// 2^(byte - 127); the bytes written are those of normal numbers.
__device__ __forceinline__ float f8_power(int byte) { return __builtin_bit_cast(float, (uint32_t)byte << 23); }

typedef short f8x4_bits __attribute__((ext_vector_type(2)));
// Four values over 2^e as e4m3, nearest, ties to even; beyond 448 (of the largest exponent alone) 448.
// Of a NaN one of the codes that are none.
__device__ __forceinline__ uint32_t f8_encode4(const float *x, float power)
{
    const float most = 448.0f * power;
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = x[i] > most ? most : x[i] < -most ? -most : x[i];
    f8x4_bits r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, v[0], v[1], power, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, v[2], v[3], power, true);
    return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ void f8_decode4(uint32_t code, float power, float *x)
{
    const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(code, power, false);
    const auto hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(code, power, true);
    x[0] = lo[0], x[1] = lo[1], x[2] = hi[0], x[3] = hi[1];
}

}  // namespace quant
}  // namespace miconv
