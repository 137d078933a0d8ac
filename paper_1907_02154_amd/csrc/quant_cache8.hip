// The 8-bit cache: tokens quantised as they are written, and read back
// (quant_kv8_write, quant_kv8_read).
//
// A work-group takes a block of a head, keys and values: the largest magnitude
// of the new tokens' values, then the block's exponent, then the codes, and
// where the exponent grew those of the tokens that the block held before.
//
// Bound by memory: 16000 tokens of 8 heads of 128, keys and values, blocks of 64,
// 98 MB, written in 21 to 23 us (4.3 to 4.7 TB/s; 28 with the tokens read twice),
// read back in 16 to 18.  A step's single tokens are two latencies and a launch: 64 sequences
// 4 us.
#include "quant.h"

#include <algorithm>

namespace miconv {
namespace quant {

int kv8_view(const quant_kv8 *c, KvView *out)
{
    if (!c) return MICONV_ERR_NULL;
    if (c->pages < 1 || c->heads < 1 || c->page_size < 1 || c->block < 1 || c->page_size % c->block) return MICONV_ERR_SHAPE;
    const int D = c->head_dim;
    if ((D != 32 && D != 64 && D != 96 && D != 128 && D != 192 && D != 256) || c->block > 256) return MICONV_ERR_UNSUPPORTED;
    if (c->pages >= 1L << 31 || c->pages * c->page_size >= 1L << 31 || c->heads > 65535) return MICONV_ERR_TOO_LARGE;
    if ((long)c->heads * c->page_size >= 1L << 31) return MICONV_ERR_TOO_LARGE;   // the kernels number a page's rows in 32 bits
    if (!c->k_codes || !c->k_exps || !c->v_codes || !c->v_exps) return MICONV_ERR_NULL;
    if (misaligned(c->k_codes, 16) || misaligned(c->v_codes, 16)) return MICONV_ERR_ALIGN;
    out->kc = (uint8_t *)c->k_codes, out->ke = (uint8_t *)c->k_exps;
    out->vc = (uint8_t *)c->v_codes, out->ve = (uint8_t *)c->v_exps;
    out->slots = c->pages * c->page_size;
    out->heads = c->heads, out->page_size = c->page_size, out->dim = D;
    out->dv_page = make_fastdiv((unsigned)c->page_size);
    out->block = c->block, out->blocks = c->page_size / c->block;
    out->dv_block = make_fastdiv((unsigned)c->block);
    return MICONV_OK;
}

namespace {

struct WriteArgs {
    KvView c;
    const void *k, *v;
    long ks, vs, tokens;           // row strides in elements, rows
    const int32_t *starts, *lens, *table;
    int table_stride, max_new;
    int units;                     // of 8 channels in a head's row
    FastDiv dv_units, dv_heads;
};

__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7FFFFFFFu; }

// PER > 0: the new tokens of a block are PER units of 8 channels a thread at most, read once and kept; 0: read twice.
template <typename T, int NT, int PER>
__global__ __launch_bounds__(NT) void kv8_write_kernel(WriteArgs a)
{
    constexpr int WAVES = NT / 64;
    __shared__ uint32_t tops[2][WAVES > 1 ? WAVES : 1], bad[256];
    const KvView &c = a.c;
    // heads first: work-groups that run together read a token's row together
    const int s = blockIdx.y, at_block = (int)fdiv(blockIdx.x, a.dv_heads), head = (int)blockIdx.x - at_block * c.heads;
    const int tid = threadIdx.x;
    long r0 = a.starts ? a.starts[s] : s, r1 = a.starts ? a.starts[s + 1] : s + 1;
    r0 = r0 < 0 ? 0 : r0 > a.tokens ? a.tokens : r0;
    r1 = r1 < r0 ? r0 : r1 > a.tokens ? a.tokens : r1;
    const int news = (int)(r1 - r0), len = max(a.lens[s], 0);
    const long room = (long)a.table_stride * c.page_size;
    // the new tokens stand at begin .. end - 1, those before place 0 and past the table's end left out
    const long begin = (long)len - news;
    const long end = min(min((long)len, begin + a.max_new), room);
    const long first = begin < 0 ? 0 : begin;
    const long p0 = ((long)fdiv((unsigned)first, c.dv_block) + at_block) * c.block;   // the block's first place
    if (p0 >= end) return;
    const int lo = (int)(max(first, p0) - p0), hi = (int)(min(end, p0 + c.block) - p0);   // its new tokens
    if (lo >= hi) return;
    const unsigned in_table = fdiv((unsigned)p0, c.dv_page);
    const int page = a.table[(long)s * a.table_stride + in_table], place = (int)(p0 - (long)in_table * c.page_size);
    if (page < 0 || (long)page * c.page_size >= c.slots) return;
    const long hp = (long)page * c.heads + head;
    const long at_exp = hp * c.blocks + (int)fdiv((unsigned)place, c.dv_block);
    const long at_code = (hp * c.page_size + place) * c.dim;
    const long src0 = r0 + (p0 - begin);                            // row of the block's first place, if it were new
    const int count = (hi - lo) * a.units;                          // units of 8 channels of the new keys (or values)
    // unit i: token lo + i / units, channels of unit i % units; values follow the keys
    const auto load = [&](int i, bool val, float (&x)[8], int &tok, int &u) {
        tok = (int)fdiv((unsigned)i, a.dv_units), u = i - tok * a.units, tok += lo;
        const T *p = (const T *)(val ? a.v : a.k) + (src0 + tok) * (val ? a.vs : a.ks) + (long)head * c.dim + 8 * u;
        load8(p, x);
    };
    float kept[PER > 0 ? PER : 1][8];
    if constexpr (PER > 0) {
#pragma unroll
        for (int n = 0; n < PER; ++n) {
            int tok, u;
            const int i = min(n * NT + tid, 2 * count - 1);
            load(i >= count ? i - count : i, i >= count, kept[n], tok, u);
        }
    }
    // f(values, token, unit, whether they are values) of this thread's units
    const auto each = [&](auto f) {
        if constexpr (PER > 0) {
#pragma unroll
            for (int n = 0; n < PER; ++n) {
                const int i = n * NT + tid, in = i >= count ? i - count : i, tok = (int)fdiv((unsigned)in, a.dv_units);
                if (i < 2 * count) f(kept[n], tok + lo, in - tok * a.units, i >= count);
            }
        } else {
            for (int i = tid; i < 2 * count; i += NT) {
                float x[8];
                int tok, u;
                load(i >= count ? i - count : i, i >= count, x, tok, u);
                f(x, tok, u, i >= count);
            }
        }
    };
    const auto reduce = [&](uint32_t &tk, uint32_t &tv) {   // the work-group's largest
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            tk = max(tk, (uint32_t)__shfl_xor((int)tk, d));
            tv = max(tv, (uint32_t)__shfl_xor((int)tv, d));
        }
        if constexpr (WAVES > 1) {
            __syncthreads();
            if (tid % 64 == 0) tops[0][tid / 64] = tk, tops[1][tid / 64] = tv;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < WAVES; ++w) tk = max(tk, tops[0][w]), tv = max(tv, tops[1][w]);
        }
    };
    uint32_t top[2] = {0, 0};
    each([&](const float (&x)[8], int, int, bool val) {
        uint32_t t = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) t = max(t, magnitude(x[j]));
        if (val) top[1] = max(top[1], t);
        else top[0] = max(top[0], t);
    });
    reduce(top[0], top[1]);
    const bool any_bad = max(top[0], top[1]) >= 0x7F800000u;   // the same for all threads
    if (any_bad) {   // which tokens, and the largest of the others
        for (int i = tid; i < 256; i += NT) bad[i] = 0;
        __syncthreads();
        for (int pass = 0; pass < 2; ++pass) {
            top[0] = top[1] = 0;
            each([&](const float (&x)[8], int tok, int, bool val) {
                uint32_t t = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) t = max(t, magnitude(x[j]));
                if (pass == 0) {
                    if (t >= 0x7F800000u) bad[tok] = 1;   // whoever writes it writes 1
                } else if (!bad[tok]) {
                    if (val) top[1] = max(top[1], t);
                    else top[0] = max(top[0], t);
                }
            });
            __syncthreads();
        }
        reduce(top[0], top[1]);
    }
    int byte[2] = {f8_byte(top[0]), f8_byte(top[1])}, was[2];
    was[0] = lo > 0 ? c.ke[at_exp] : 0, was[1] = lo > 0 ? c.ve[at_exp] : 0;
#pragma unroll
    for (int n = 0; n < 2; ++n) was[n] = min(was[n], kF8Hi), byte[n] = max(byte[n], was[n]);
    const float power[2] = {f8_power(byte[0]), f8_power(byte[1])};
    each([&](const float (&x)[8], int tok, int u, bool val) {
        const float p = val ? power[1] : power[0];
        uint32_t v[2] = {f8_encode4(x, p), f8_encode4(x + 4, p)};
        if (any_bad && bad[tok]) v[0] = v[1] = val ? 0u : 0x7F7F7F7Fu;
        memcpy((val ? c.vc : c.kc) + at_code + (long)tok * c.dim + 8 * u, v, 8);
    });
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        if (lo == 0 || byte[n] == was[n]) continue;   // nothing held, or its exponent stays
        uint32_t *held = (uint32_t *)((n ? c.vc : c.kc) + at_code);
        const float old = f8_power(was[n]);
        for (int i = tid; i < lo * c.dim / 4; i += NT) {
            const uint32_t code = held[i];
            float x[4];
            f8_decode4(code, old, x);
            // codes that are no numbers stay as they are
            const uint32_t none = ((((code & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7) * 255u;
            held[i] = (f8_encode4(x, power[n]) & ~none) | (code & none);
        }
    }
    __syncthreads();   // every thread has read what the bytes were
    if (tid < 2) (tid ? c.ve : c.ke)[at_exp] = (uint8_t)byte[tid];
}

struct ReadArgs {
    KvView c;
    void *k, *v;
    long ks, vs;
    const int32_t *slots;
    int tokens;
    int per;               // units of 8 channels in a token's row
    FastDiv dv_per, dv_head;
};

constexpr int kRead = 4;   // tokens a work-group handles, keys or values

template <typename T>
__global__ __launch_bounds__(256) void kv8_read_kernel(ReadArgs a)
{
    const KvView &c = a.c;
    const bool val = blockIdx.y;
    T *dst = (T *)(val ? a.v : a.k);
    const long stride = val ? a.vs : a.ks;
    const uint8_t *codes = val ? c.vc : c.kc, *exps = val ? c.ve : c.ke;
    // each die gets a run of tokens, which share lines of exponents
    const unsigned q = gridDim.x / 8, r = gridDim.x % 8, die = blockIdx.x % 8;
    const long first = (long)(die * q + min(die, r) + blockIdx.x / 8) * kRead;
    const int units = c.dim / 8, total = kRead * a.per;
    for (int i = threadIdx.x; i < total; i += 256) {
        const int tok = (int)fdiv((unsigned)i, a.dv_per), in = i - tok * a.per;
        const int head = (int)fdiv((unsigned)in, a.dv_head), u = in - head * units;
        const long t = first + tok;
        if (t >= a.tokens) break;
        const int slot = a.slots[t];
        uint32_t code[2] = {0, 0};
        int byte = 127;
        if (slot >= 0 && slot < c.slots) {
            const unsigned page = fdiv((unsigned)slot, c.dv_page), place = (unsigned)slot - page * (unsigned)c.page_size;
            const long hp = (long)page * c.heads + head;
            memcpy(code, codes + (hp * c.page_size + place) * c.dim + 8 * u, 8);
            byte = exps[hp * c.blocks + (int)fdiv(place, c.dv_block)];
        }
        float x[8];
        f8_decode4(code[0], f8_power(byte), x);
        f8_decode4(code[1], f8_power(byte), x + 4);
        store8(dst + t * stride + (long)in * 8, x);
    }
}

}  // namespace
}  // namespace quant
}  // namespace miconv

extern "C" int quant_kv8_write(const quant_kv8 *cache, int seqs, long tokens, int dtype, const void *k, long k_stride,
                               const void *v, long v_stride, const int32_t *starts, const int32_t *lens,
                               const int32_t *table, int table_stride, int max_new, void *stream)
{
    using namespace miconv;
    using namespace miconv::quant;
    WriteArgs a = {};
    const int rc = kv8_view(cache, &a.c), b = dtype_bytes(dtype);
    if (rc != MICONV_OK) return rc;
    if (!b) return MICONV_ERR_UNSUPPORTED;
    const long width = (long)a.c.heads * a.c.dim;
    if (seqs < 0 || tokens < 0 || k_stride < width || v_stride < width || max_new < 1 || table_stride < 1)
        return MICONV_ERR_SHAPE;
    if (seqs > 65535 || tokens >= 1L << 31) return MICONV_ERR_TOO_LARGE;
    // Blocks that new tokens can reach, wherever they begin.
    const long blocks = ((long)max_new + a.c.block - 2) / a.c.block + 1;
    const long most = std::min((long)max_new, (long)a.c.block) * (a.c.dim / 8) * 2;   // units of a block's new tokens
    // One wavefront where it holds them all: a token each of 64 sequences, 8 heads of 128, 4.0 us against 4.3 with 256
    // threads, of 256 sequences, 32 heads, 7.4 against 16.1.
    const int nt = most > 64 ? 256 : 64;
    if (blocks * a.c.heads * nt >= 1L << 32 || blocks * a.c.heads >= 1L << 31) return MICONV_ERR_TOO_LARGE;   // threads of a grid
    if (seqs == 0 || tokens == 0) return MICONV_OK;
    if (!k || !v || !lens || !table) return MICONV_ERR_NULL;
    if (misaligned(k, b) || misaligned(v, b) || misaligned(starts, 4) || misaligned(lens, 4) || misaligned(table, 4))
        return MICONV_ERR_ALIGN;
    a.k = k, a.v = v, a.ks = k_stride, a.vs = v_stride, a.tokens = tokens;
    a.starts = starts, a.lens = lens, a.table = table;
    a.table_stride = table_stride, a.max_new = max_new;
    a.units = a.c.dim / 8;
    a.dv_units = make_fastdiv((unsigned)a.units);
    a.dv_heads = make_fastdiv((unsigned)a.c.heads);
    const dim3 grid((unsigned)(blocks * a.c.heads), (unsigned)seqs);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const auto go = [&](auto of) {
        typedef decltype(of) T;
        void (*kernel)(WriteArgs) = kv8_write_kernel<T, 256, 0>;
        if (nt == 64) kernel = kv8_write_kernel<T, 64, 1>;
        else if (most <= 256) kernel = kv8_write_kernel<T, 256, 1>;
        else if (most <= 512) kernel = kv8_write_kernel<T, 256, 2>;
        else if (most <= 1024) kernel = kv8_write_kernel<T, 256, 4>;
        else if (most <= 2048) kernel = kv8_write_kernel<T, 256, 8>;
        launch_kernel(kernel, grid, dim3((unsigned)nt), 0, st, a);
        return launched();
    };
    return dtype == kF32 ? go(float()) : go(uint16_t());
}

extern "C" int quant_kv8_read(const quant_kv8 *cache, long tokens, const int32_t *slots, int dtype, void *k,
                              long k_stride, void *v, long v_stride, void *stream)
{
    using namespace miconv;
    using namespace miconv::quant;
    ReadArgs a = {};
    const int rc = kv8_view(cache, &a.c), b = dtype_bytes(dtype);
    if (rc != MICONV_OK) return rc;
    if (!b) return MICONV_ERR_UNSUPPORTED;
    const long width = (long)a.c.heads * a.c.dim;
    if (tokens < 0 || k_stride < width || v_stride < width) return MICONV_ERR_SHAPE;
    if (tokens > 1L << 25) return MICONV_ERR_TOO_LARGE;   // a grid holds fewer than 2^32 threads
    if (tokens == 0) return MICONV_OK;
    if (!k || !v || !slots) return MICONV_ERR_NULL;
    if (misaligned(k, b) || misaligned(v, b) || misaligned(slots, 4)) return MICONV_ERR_ALIGN;
    a.k = k, a.v = v, a.ks = k_stride, a.vs = v_stride, a.slots = slots;
    a.tokens = (int)tokens;
    a.per = (int)(width / 8);
    a.dv_per = make_fastdiv((unsigned)a.per);
    a.dv_head = make_fastdiv((unsigned)(a.c.dim / 8));
    const dim3 grid((unsigned)((tokens + kRead - 1) / kRead), 2);
    launch_kernel(dtype == kF32 ? kv8_read_kernel<float> : kv8_read_kernel<uint16_t>, grid, dim3(256), 0,
                  static_cast<hipStream_t>(stream), a);
    return launched();
}
