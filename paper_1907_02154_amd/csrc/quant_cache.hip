// The 4-bit cache: tokens quantised as they are written, and read back
// (quant_kv4_write, quant_kv4_read).
//
// Four lanes share a group of 32 channels, 8 channels each: 16 bytes of bf16
// in, 4 bytes of codes out (or the reverse), one conversion instruction for
// two values either way.  Bound by memory, 2 + 17/32 bytes a bf16 value: 16000
// tokens of 8 heads of 128, keys and values, 83 MB: written in 21 us (3.9
// TB/s; 24 with one unit of a thread in flight at a time), read in 16 (5.2, the
// rate of a large copy).
#include "quant.h"

namespace miconv {
namespace quant {

int kv4_view(const quant_kv4 *c, Kv4 *out)
{
    if (!c) return MICONV_ERR_NULL;
    if (c->pages < 1 || c->heads < 1 || c->page_size < 1) return MICONV_ERR_SHAPE;
    const int D = c->head_dim;
    if (D != 32 && D != 64 && D != 96 && D != 128 && D != 192 && D != 256) return MICONV_ERR_UNSUPPORTED;
    if (c->pages >= 1L << 31 || c->pages * c->page_size >= 1L << 31 || c->heads > 65535) return MICONV_ERR_TOO_LARGE;
    if (!c->k_codes || !c->k_exps || !c->v_codes || !c->v_exps) return MICONV_ERR_NULL;
    if (misaligned(c->k_codes, 16) || misaligned(c->v_codes, 16)) return MICONV_ERR_ALIGN;
    out->kc = (uint8_t *)c->k_codes, out->ke = (uint8_t *)c->k_exps;
    out->vc = (uint8_t *)c->v_codes, out->ve = (uint8_t *)c->v_exps;
    out->slots = c->pages * c->page_size;
    out->heads = c->heads, out->page_size = c->page_size, out->dim = D;
    out->dv_page = make_fastdiv((unsigned)c->page_size);
    return MICONV_OK;
}

namespace {

constexpr int kWrite = 8, kRead = 4;   // tokens a work-group handles, keys or values

struct CacheArgs {
    Kv4 c;
    void *k, *v;           // the tokens' rows (read by the write, written by the read)
    long ks, vs;           // their strides in elements
    const int32_t *slots;
    int tokens;
    int per;               // units of 8 channels in a token's row
    FastDiv dv_per, dv_head;   // division by `per` and by the units of a head
};

// First token of a work-group.  A work-group runs on the die of its number
// modulo 8, and tokens that follow one another share cache lines of codes and
// exponents: each die gets a run of tokens, so that its L2 puts the lines
// together.
__device__ __forceinline__ long first_token(int tokens)
{
    const unsigned q = gridDim.x / 8, r = gridDim.x % 8, die = blockIdx.x % 8;
    return (long)(die * q + min(die, r) + blockIdx.x / 8) * tokens;
}

// Row of the cache (of head_dim / 2 bytes of codes) that holds (slot, head).
__device__ __forceinline__ long cache_row(const Kv4 &c, int slot, int head)
{
    const unsigned page = fdiv((unsigned)slot, c.dv_page), place = (unsigned)slot - page * (unsigned)c.page_size;
    return ((long)page * c.heads + head) * c.page_size + place;
}

template <typename T>
__global__ __launch_bounds__(256) void kv4_write_kernel(CacheArgs a)
{
    const Kv4 &c = a.c;
    const bool val = blockIdx.y;
    const T *src = (const T *)(val ? a.v : a.k);
    const long stride = val ? a.vs : a.ks;
    uint8_t *codes = val ? c.vc : c.kc, *exps = val ? c.ve : c.ke;
    const long first = first_token(kWrite);
    const int units = c.dim / 8, total = kWrite * a.per;   // a multiple of 4: a group's lanes stay together
    constexpr int U = 4;                                    // units of a thread whose loads are in flight together
    for (int i0 = threadIdx.x; i0 < total; i0 += 256 * U) {
        float x[U][8];
        int slot[U], in[U];
#pragma unroll
        for (int n = 0; n < U; ++n) {
            const int i = min(i0 + 256 * n, total - 1), tok = (int)fdiv((unsigned)i, a.dv_per);
            in[n] = i - tok * a.per;
            const long t = min(first + tok, (long)a.tokens - 1);
            const bool live = i0 + 256 * n < total && first + tok < a.tokens;
            slot[n] = live ? a.slots[t] : -1;
            load8(src + t * stride + (long)in[n] * 8, x[n]);
        }
#pragma unroll
        for (int n = 0; n < U; ++n) {
            const int head = (int)fdiv((unsigned)in[n], a.dv_head), u = in[n] - head * units;
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t b = __builtin_bit_cast(uint32_t, x[n][j]) & 0x7FFFFFFFu;
                top = b > top ? b : top;
            }
            uint32_t o = (uint32_t)__shfl_xor((int)top, 1);
            top = o > top ? o : top;
            o = (uint32_t)__shfl_xor((int)top, 2);
            top = o > top ? o : top;
            // smallest e with top <= 7 * 2^e: 2 below top's exponent, 1 below it when its significand passes 1.75
            int e = (int)(top >> 23) - 2 + ((top & 0x7FFFFFu) > 0x600000u);
            e = e < 1 ? 1 : e > kMaxExp ? kMaxExp : e;
            const float s = __builtin_bit_cast(float, (uint32_t)e << 23);
            uint32_t code = 0;
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[n][0], x[n][1], s, 0);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[n][2], x[n][3], s, 1);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[n][4], x[n][5], s, 2);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[n][6], x[n][7], s, 3);
            if (top >= 0x7F800000u) e = 255, code = 0;
            if (slot[n] >= 0 && slot[n] < c.slots) {
                const long row = cache_row(c, slot[n], head);
                *(uint32_t *)(codes + row * (c.dim / 2) + u * 4) = code;
                if (u % 4 == 0) exps[row * (c.dim / 32) + u / 4] = (uint8_t)e;
            }
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void kv4_read_kernel(CacheArgs a)
{
    const Kv4 &c = a.c;
    const bool val = blockIdx.y;
    T *dst = (T *)(val ? a.v : a.k);
    const long stride = val ? a.vs : a.ks;
    const uint8_t *codes = val ? c.vc : c.kc, *exps = val ? c.ve : c.ke;
    const long first = first_token(kRead);
    const int units = c.dim / 8, total = kRead * a.per;
    for (int i = threadIdx.x; i < total; i += 256) {
        const int tok = (int)fdiv((unsigned)i, a.dv_per), in = i - tok * a.per;
        const int head = (int)fdiv((unsigned)in, a.dv_head), u = in - head * units;
        const long t = first + tok;
        if (t >= a.tokens) break;
        const int slot = a.slots[t];
        uint32_t code = 0, e = 127;
        if (slot >= 0 && slot < c.slots) {
            const long row = cache_row(c, slot, head);
            code = *(const uint32_t *)(codes + row * (c.dim / 2) + u * 4);
            e = exps[row * (c.dim / 32) + u / 4];
        }
        // an exponent byte above 252 becomes an infinite scale: all values NaN
        const float s = __builtin_bit_cast(float, (e > kMaxExp ? 255u : e) << 23);
        const auto b0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 0);
        const auto b1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 1);
        const auto b2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 2);
        const auto b3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 3);
        const float x[8] = {b0[0], b0[1], b1[0], b1[1], b2[0], b2[1], b3[0], b3[1]};
        store8(dst + t * stride + (long)in * 8, x);
    }
}

int run_cache(const quant_kv4 *cache, long tokens, int dtype, const void *k, long k_stride, const void *v,
              long v_stride, const int32_t *slots, bool write, hipStream_t st)
{
    CacheArgs a;
    const int rc = kv4_view(cache, &a.c), b = dtype_bytes(dtype);
    if (rc != MICONV_OK) return rc;
    if (!b) return MICONV_ERR_UNSUPPORTED;
    const long width = (long)a.c.heads * a.c.dim;
    if (tokens < 0 || k_stride < width || v_stride < width) return MICONV_ERR_SHAPE;
    if (tokens > 1L << 25) return MICONV_ERR_TOO_LARGE;   // a grid holds fewer than 2^32 threads
    if (tokens == 0) return MICONV_OK;
    if (!k || !v || !slots) return MICONV_ERR_NULL;
    if (misaligned(k, b) || misaligned(v, b) || misaligned(slots, 4)) return MICONV_ERR_ALIGN;
    a.k = const_cast<void *>(k), a.v = const_cast<void *>(v);
    a.ks = k_stride, a.vs = v_stride;
    a.slots = slots;
    a.tokens = (int)tokens;
    a.per = (int)(width / 8);
    a.dv_per = make_fastdiv((unsigned)a.per);
    a.dv_head = make_fastdiv((unsigned)(a.c.dim / 8));
    const int each = write ? kWrite : kRead;
    const dim3 grid((unsigned)((tokens + each - 1) / each), 2);
    if (write)
        launch_kernel(dtype == kF32 ? kv4_write_kernel<float> : kv4_write_kernel<uint16_t>, grid, dim3(256), 0, st, a);
    else
        launch_kernel(dtype == kF32 ? kv4_read_kernel<float> : kv4_read_kernel<uint16_t>, grid, dim3(256), 0, st, a);
    return launched();
}

}  // namespace
}  // namespace quant
}  // namespace miconv

extern "C" int quant_kv4_write(const quant_kv4 *cache, long tokens, int dtype, const void *k, long k_stride,
                               const void *v, long v_stride, const int32_t *slots, void *stream)
{
    return miconv::quant::run_cache(cache, tokens, dtype, k, k_stride, v, v_stride, slots, true,
                                    static_cast<hipStream_t>(stream));
}

extern "C" int quant_kv4_read(const quant_kv4 *cache, long tokens, const int32_t *slots, int dtype, void *k,
                              long k_stride, void *v, long v_stride, void *stream)
{
    return miconv::quant::run_cache(cache, tokens, dtype, k, k_stride, v, v_stride, slots, false,
                                    static_cast<hipStream_t>(stream));
}
