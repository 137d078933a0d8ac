// Attention over the paged caches of 4 and of 8 bits (quant_attention_kv4,
// quant_attention_kv8).
//
// Scores are computed transposed, S^T = K Q^T: the cached tokens are the rows
// of the matrix instruction and the queries its columns, so each lane holds
// scores of one query, and the probabilities leave the softmax in the very
// layout in which O^T = V^T P^T reads them as its second operand (the order of
// the tokens within a product's reduction is free).  One pass over the cache
// with a running maximum m and sum l: O and l are rescaled by 2^(m - m') when
// the maximum grows by more than 2^8, which leaves the quotient O / l as it is
// and the probabilities below 2^8.
//
// Queries that share a key head are the rows of one problem: row = token *
// (heads / key heads) + head within the group.
#include "quant.h"

#include <algorithm>
#include <stdio.h>

namespace miconv {
namespace quant {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr float kNegInf = -__builtin_inff();
constexpr float kGrow = 8.0f;   // log2 of how far scores may pass the running maximum before it moves

struct AttArgs {
    KvView c;
    const uint16_t *q;
    uint16_t *out;
    const int32_t *starts, *lens, *table;
    float *part;           // split partials: [seq][head][max_new][splits] rows of (D sums, m, l), or null
    long qs, os;           // row strides in elements
    long tokens;
    int seqs, heads, group, table_stride;
    int max_new, max_len;
    int causal, window;
    int splits, per_split; // cached tokens a split handles
    int row_blocks;
    float scale;           // of the scores, times log2(e)
    FastDiv dv_group;
};

// What a work-group works on: a sequence's queries and length, clamped.
struct Seq {
    long row0;   // first row of q
    int news, len;
    int most;    // places that can be seen: what the bound, the table and the sequence hold
};

__device__ __forceinline__ Seq sequence(const AttArgs &a, int s)
{
    Seq r;
    long b = a.starts ? a.starts[s] : s, e = a.starts ? a.starts[s + 1] : s + 1;
    b = b < 0 ? 0 : b > a.tokens ? a.tokens : b;
    e = e < b ? b : e > a.tokens ? a.tokens : e;
    r.row0 = b;
    r.news = (int)(e - b);
    const long room = (long)a.table_stride * a.c.page_size;
    const int most = room < a.max_len ? (int)room : a.max_len;
    const int n = a.lens[s];
    r.len = n < 0 ? 0 : n;   // where the queries stand, also past what can be seen
    r.most = r.len > most ? most : r.len;
    return r;
}

// The places query row i of a sequence sees: lo .. hi - 1.
__device__ __forceinline__ void seen(const AttArgs &a, const Seq &q, int i, int *lo, int *hi)
{
    const int p = q.len - q.news + i;
    int h = a.causal ? p + 1 : q.most;
    h = h > q.most ? q.most : h;
    const int l = a.window > 0 && p >= a.window ? p - a.window + 1 : 0;   // a difference that no window makes pass 32 bits
    *lo = l > q.most ? q.most : l;
    *hi = h < 0 ? 0 : h;
}

// What the kernels know of a cache's format: 32-bit words that hold 8 channels,
// whether a token's 32 channels have an exponent of their own, and the way to
// bf16, which holds every value of either format.

// Four bits a value, an exponent for each 32 channels of a token.
struct Fp4 {
    static constexpr int WORDS = 1;
    static constexpr bool GROUPS = true;
    // Scale bits of an exponent byte; above 252 an infinite scale, which converts to NaN.
    static __device__ __forceinline__ float scale(uint32_t e)
    {
        return __builtin_bit_cast(float, (e > kMaxExp ? 255u : e) << 23);
    }
    // Of keys and of values, by the exponents of both.  A value that is not finite makes the token's score NaN, which
    // reaches the queries that see it; its own NaN times a probability of 0 would reach the others too.
    static __device__ __forceinline__ float keys(uint32_t ke, uint32_t ve) { return scale(ve > kMaxExp ? 255u : ke); }
    static __device__ __forceinline__ float values(uint32_t ve) { return scale(ve > kMaxExp ? 127u : ve); }
    static __device__ __forceinline__ bf16x8 widen8(const uint32_t *w, float s)
    {
        const uint32_t code = *w;
        u32x4 r = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 0)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 1)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 2)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 3))};
        return __builtin_bit_cast(bf16x8, r);
    }
    static __device__ __forceinline__ void clean(uint32_t &) {}
};

// Eight bits a value, an exponent for a block of tokens.  Keys that are not
// numbers make the token's score NaN, which reaches the queries that see it.
// Values are written as numbers alone; a place that no one sees may hold
// anything, and its values must not bring a NaN to a product with a probability
// of 0: where a tile holds such places codes that are no numbers become 448, and
// exponents stay where the format has them.
struct Fp8 {
    static constexpr int WORDS = 2;
    static constexpr bool GROUPS = false;
    static __device__ __forceinline__ float keys(uint32_t ke, uint32_t) { return __builtin_bit_cast(float, ke << 23); }
    static __device__ __forceinline__ float values(uint32_t ve)
    {
        return __builtin_bit_cast(float, (ve > (uint32_t)kF8Hi ? (uint32_t)kF8Hi : ve) << 23);
    }
    static __device__ __forceinline__ bf16x8 widen8(const uint32_t *w, float s)
    {
        u32x4 r = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], s, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], s, true)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], s, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], s, true))};
        return __builtin_bit_cast(bf16x8, r);
    }
    static __device__ __forceinline__ void clean(uint32_t &w)   // 0x7F and 0xFF become 0x7E and 0xFE
    {
        w ^= (((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7;
    }
};

// The exponent of a token's keys or values among those of its page and head.
__device__ __forceinline__ uint64_t exponent_of(const KvView &c, unsigned page, int head, int place)
{
    return ((uint64_t)page * (unsigned)c.heads + (unsigned)head) * (unsigned)c.blocks + fdiv((unsigned)place, c.dv_block);
}

// N words from p on, which is aligned to the widest access that divides them.
template <int N>
__device__ __forceinline__ void load_words(const uint8_t *p, uint32_t (&w)[N])
{
    constexpr int V = N % 4 == 0 ? 4 : N % 2 == 0 ? 2 : 1;
    typedef uint32_t words __attribute__((ext_vector_type(V)));
#pragma unroll
    for (int i = 0; i < N / V; ++i) {
        const words v = ((const words *)p)[i];
#pragma unroll
        for (int j = 0; j < V; ++j) w[i * V + j] = v[j];
    }
}

// The factor of the scores as the kernels take it: positive, its sign in the
// queries' sign bits, and not 0, so that a masked score stays -inf.
__device__ __forceinline__ float factor(const AttArgs &a) { return fmaxf(fabsf(a.scale), 0x1p-120f); }
__device__ __forceinline__ bf16x8 query8(const AttArgs &a, const uint16_t *q)
{
    uint32_t raw[4];
    memcpy(raw, q, 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(raw[i]));   // or it is loaded again by halves for the exclusive or
    const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u;
    const u32x4 v = {raw[0] ^ flip, raw[1] ^ flip, raw[2] ^ flip, raw[3] ^ flip};
    return __builtin_bit_cast(bf16x8, v);
}

// Two probabilities 2^(s c - base) as bf16, the matrix cores' operand, added to l
// as rounded: what a rounding adds above and below the line is the same, so that
// only the difference of a value from the row's result counts.  Against 64 bits
// the results of two prompts of 4096 tokens are off by 0.0021 of their size (root
// mean square), where probabilities in fp32 and the result's own rounding to bf16
// make 0.0016.  A second part, as few rows have it below, would add half as many
// products again, and these are a good part of what binds.
__device__ __forceinline__ uint32_t weights2(float s0, float s1, float c, float base, float &l)
{
    const uint32_t w = pack_bf16x2(__builtin_amdgcn_exp2f(__builtin_fmaf(s0, c, -base)),
                                   __builtin_amdgcn_exp2f(__builtin_fmaf(s1, c, -base)));
    l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), __builtin_bit_cast(bf16x2, 0x3F803F80u), l, false);
    return w;
}

// Few rows: four wavefronts share 16 * NB query rows and take turns at tiles of
// 32 cached tokens; their sums meet in LDS at the end.
//
// Bound by memory: 16 single tokens over up to 32768 places, 32 heads of 128 on 8
// key heads, 413 MB: 89 us and 5 more for the join, 4.4 TB/s; while all
// work-groups run they read at the rate of a large copy (5.2), and the first loads
// and the last tiles take the rest.  In 8 bits the same calls read 777 MB: 164 us and
// 5, 4.7 TB/s.  Short calls are latencies in a row: one
// token over 100 places 4.3 us, 17 tokens each with a window of 1000, 12 us with
// the join.
template <class F, int D, int NB>
__device__ __forceinline__ void attend_few(const AttArgs &a)
{
    constexpr int NU = D / 32;           // units of 8 channels a lane holds of a cached row
    constexpr int CB = D / 16;           // blocks of 16 channels
    constexpr int PITCH = D * 2 + 32;    // bytes of a widened row in LDS
    constexpr int VBYTES = 32 * PITCH;   // a wavefront's tile of values
    constexpr int OPITCH = D + 4;        // floats of a query's sums in LDS
    constexpr int OBYTES = 16 * NB * OPITCH * 4;
    constexpr int LDS = 4 * VBYTES > OBYTES ? 4 * VBYTES : OBYTES;
    __shared__ __align__(16) unsigned char lds[LDS];
    __shared__ float sm[4][16 * NB], sl[4][16 * NB];

    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int col = lane % 16, quad = lane / 16;
    const int split = blockIdx.x % a.splits, rb = blockIdx.x / a.splits, kvh = blockIdx.y, s = blockIdx.z;
    const Seq sq = sequence(a, s);
    const int rows = (sq.news < a.max_new ? sq.news : a.max_new) * a.group, r0 = rb * 16 * NB;
    if (r0 >= rows) return;
    const int r_last = r0 + 16 * NB < rows ? r0 + 16 * NB - 1 : rows - 1;

    // the places that any row of the block sees, lo .. hi - 1, and that every row does, from .. all - 1; within this split
    int lo, hi, from, all;
    seen(a, sq, (int)fdiv((unsigned)r0, a.dv_group), &lo, &all);
    seen(a, sq, (int)fdiv((unsigned)r_last, a.dv_group), &from, &hi);
    lo = (lo & ~31) + split * a.per_split;   // per_split is a multiple of 64
    hi = lo + min(hi - lo, a.per_split);

    int q_lo[NB], q_hi[NB];
    bf16x8 qf[NB][NU];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int r = r0 + 16 * b + col;
        const bool live = r < rows;
        const int i = (int)fdiv((unsigned)(live ? r : 0), a.dv_group), h = kvh * a.group + (live ? r : 0) - i * a.group;
        seen(a, sq, i, &q_lo[b], &q_hi[b]);
        if (!live) q_hi[b] = 0;
        const uint16_t *qr = a.q + (sq.row0 + i) * a.qs + (long)h * D + quad * (D / 4);
#pragma unroll
        for (int u = 0; u < NU; ++u) qf[b][u] = query8(a, qr + 8 * u);
    }
    const float c = factor(a);

    float m[NB], l[NB];   // m: the running maximum times c
    f32x4 o[CB][NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        m[b] = kNegInf, l[b] = 0.0f;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) o[cb][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    const int32_t *pages = a.table + (long)s * a.table_stride;
    const int last_page = (int)(a.c.slots / a.c.page_size) - 1;
    const int page_rows = a.c.heads * a.c.page_size, head_row = kvh * a.c.page_size;
    unsigned char *vt = lds + wave * VBYTES;
    // What a lane holds of a tile: of token 16 k + col the units quad * NU .. + NU - 1 and the exponents of their groups,
    // or the token's.
    constexpr int W = F::WORDS, NE = F::GROUPS && (D == 96 || D > 128) ? 2 : 1;
    const int g0 = quad * NU / 4, g1 = min(g0 + 1, D / 32 - 1);
    struct Held {
        uint32_t kc[2][NU * W], vc[2][NU * W], ke[2][NE], ve[2][NE];
    };
    int page[2], place[2];
    const auto look = [&](int t0) {   // the pages of a tile's tokens
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            int t = t0 + 16 * k + col;
            t = t < hi ? t : hi - 1;   // past the end: a row that is seen, masked below
            const unsigned p = fdiv((unsigned)t, a.c.dv_page);
            place[k] = t - (int)p * a.c.page_size;
            page[k] = pages[p];
        }
    };
    const auto fetch = [&](Held &to) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const unsigned pg = (unsigned)min(max(page[k], 0), last_page);
            const uint64_t row = (uint64_t)pg * (unsigned)page_rows + (unsigned)(head_row + place[k]);
            load_words<NU * W>(a.c.kc + row * (D / 2 * W) + quad * (D / 8 * W), to.kc[k]);
            load_words<NU * W>(a.c.vc + row * (D / 2 * W) + quad * (D / 8 * W), to.vc[k]);
            if constexpr (F::GROUPS) {   // apart: with one index for either format they take 3% longer
                to.ke[k][0] = a.c.ke[row * (D / 32) + g0];
                to.ve[k][0] = a.c.ve[row * (D / 32) + g0];
            } else {
                const uint64_t e = exponent_of(a.c, pg, kvh, place[k]);
                to.ke[k][0] = a.c.ke[e], to.ve[k][0] = a.c.ve[e];
            }
            if constexpr (NE == 2) {
                to.ke[k][1] = a.c.ke[row * (D / 32) + g1];
                to.ve[k][1] = a.c.ve[row * (D / 32) + g1];
            }
        }
    };
    const auto tile = [&](Held &cur, Held &next, int t0) {
        if (t0 + 128 < hi) {
            fetch(next);
            if (t0 + 256 < hi) look(t0 + 256);
        }
        f32x4 sc[2][NB];
        if constexpr (!F::GROUPS)
            if (t0 < from || t0 + 32 > all)   // places that not every row sees
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int u = 0; u < NU * W; ++u) F::clean(cur.vc[k][u]);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float ks[NE], vs[NE];
#pragma unroll
            for (int e = 0; e < NE; ++e) {
                if constexpr (F::GROUPS) {   // F's, with one comparison: over heads of 64 single tokens take 1% less so
                    const bool bad = cur.ve[k][e] > (uint32_t)kMaxExp;
                    ks[e] = F::scale(bad ? 255u : cur.ke[k][e]);
                    vs[e] = F::scale(bad ? 127u : cur.ve[k][e]);
                } else ks[e] = F::keys(cur.ke[k][e], cur.ve[k][e]), vs[e] = F::values(cur.ve[k][e]);
            }
#pragma unroll
            for (int b = 0; b < NB; ++b) sc[k][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                const int e = NE == 1 ? 0 : (quad * NU + u) / 4 - g0;
                const bf16x8 kf = F::widen8(cur.kc[k] + W * u, e == 0 ? ks[0] : ks[NE - 1]);
#pragma unroll
                for (int b = 0; b < NB; ++b)
                    sc[k][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[b][u], sc[k][b], 0, 0, 0);
                *(bf16x8 *)(vt + (16 * k + col) * PITCH + quad * (D / 2) + 16 * u) =
                    F::widen8(cur.vc[k] + W * u, e == 0 ? vs[0] : vs[NE - 1]);
            }
        }
        if (t0 < from || t0 + 32 > all) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int t = t0 + 16 * k + 4 * quad + i;
                        sc[k][b][i] = t >= q_lo[b] && t < q_hi[b] ? sc[k][b][i] : kNegInf;
                    }
        }
        bf16x8 pf[NB], pl[NB];   // the probabilities in two bf16 parts: the matrix cores wait for memory here anyway
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            float top = kNegInf;
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[k][b][i]);
            top *= c;
            if (__any(top > m[b] + kGrow)) {   // also where m is still -inf
                top = fmaxf(top, m[b]);
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float f = top == m[b] ? 1.0f : __builtin_amdgcn_exp2f(m[b] - top);
                m[b] = top;
                l[b] *= f;
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) o[cb][b] *= f;
            }
            const float base = m[b] == kNegInf ? 0.0f : m[b];
            u32x4 w, v;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i / 2][b][i % 2 * 2], c, -base));
                const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i / 2][b][i % 2 * 2 + 1], c, -base));
                const uint32_t two = pack_bf16x2(p0, p1);
                w[i] = two;
                v[i] = pack_bf16x2(p0 - __builtin_bit_cast(float, two << 16), p1 - __builtin_bit_cast(float, two & 0xFFFF0000u));
                l[b] += p0 + p1;
            }
            pf[b] = __builtin_bit_cast(bf16x8, w);
            pl[b] = __builtin_bit_cast(bf16x8, v);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        // a lane's 8 tokens of the reduction: 4 * quad .. + 3 of each 16, as the scores have them
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            const unsigned char *at = vt + (4 * quad + col / 4) * PITCH + cb * 32 + (col % 4) * 8;
            const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)at);
            const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + 16 * PITCH));
            const bf16x8 vf = __builtin_shufflevector(__builtin_bit_cast(bf16x4, v0), __builtin_bit_cast(bf16x4, v1), 0, 1, 2,
                                                      3, 4, 5, 6, 7);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                o[cb][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[b], o[cb][b], 0, 0, 0);
                o[cb][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pl[b], o[cb][b], 0, 0, 0);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };
    // Loads run a tile ahead of the arithmetic, the page table's two.
    int t0 = lo + 32 * wave;
    Held even, odd;
    if (t0 < hi) {
        look(t0);
        fetch(even);
        if (t0 + 128 < hi) look(t0 + 128);
    }
    for (; t0 < hi; t0 += 256) {
        tile(even, odd, t0);
        if (t0 + 128 < hi) tile(odd, even, t0 + 128);
    }

    // The four wavefronts' sums: the joint maximum first, then O, one wavefront after another.
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        l[b] += __shfl_xor(l[b], 16);
        l[b] += __shfl_xor(l[b], 32);
        if (quad == 0) sm[wave][16 * b + col] = m[b], sl[wave][16 * b + col] = l[b];
    }
    __syncthreads();
    float *sum = (float *)lds;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (wave == w)
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const int r = 16 * b + col;
                const float mm = fmaxf(fmaxf(sm[0][r], sm[1][r]), fmaxf(sm[2][r], sm[3][r]));
                const float f = m[b] == mm ? 1.0f : __builtin_amdgcn_exp2f(m[b] - mm);
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) {
                    f32x4 *at = (f32x4 *)(sum + r * OPITCH + cb * 16 + 4 * quad);
                    *at = w == 0 ? o[cb][b] * f : *at + o[cb][b] * f;
                }
            }
        __syncthreads();
    }
    // rows out, 8 channels a thread
    for (int i = threadIdx.x; i < 16 * NB * (D / 8); i += 256) {
        const int r = i / (D / 8), u = i % (D / 8);
        if (r0 + r >= rows) break;
        const float mm = fmaxf(fmaxf(sm[0][r], sm[1][r]), fmaxf(sm[2][r], sm[3][r]));
        float ll = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) ll += sl[w][r] * (sm[w][r] == mm ? 1.0f : __builtin_amdgcn_exp2f(sm[w][r] - mm));
        float v[8];
        memcpy(v, sum + r * OPITCH + 8 * u, 32);
        const int t = (int)fdiv((unsigned)(r0 + r), a.dv_group), h = kvh * a.group + (r0 + r) - t * a.group;
        if (a.splits == 1) {
            const float f = ll == 0.0f ? 0.0f : 1.0f / ll;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= f;
            store8(a.out + (sq.row0 + t) * a.os + (long)h * D + 8 * u, v);
        } else {
            float *part = a.part + ((((long)s * a.heads + h) * a.max_new + t) * a.splits + split) * (D + 4);
            memcpy(part + 8 * u, v, 32);
            if (u == 0) part[D] = mm, part[D + 1] = ll;
        }
    }
}

template <int D, int NB>
__global__ __launch_bounds__(256, 2) void attend_kv4_kernel(AttArgs a)
{
    attend_few<Fp4, D, NB>(a);
}

template <int D, int NB>
__global__ __launch_bounds__(256, 2) void attend_kv8_kernel(AttArgs a)
{
    attend_few<Fp8, D, NB>(a);
}

// What the kernels for many rows share: eight wavefronts of 32 rows, tiles of 64
// cached tokens that a work-group widens to bf16 once, into LDS.
constexpr int kWideRows = 256;
template <int D>
struct Wide {
    static constexpr int TILE = 64;
    // Bytes between rows in LDS: keys are read by rows of 16 bytes, values by blocks of 4 rows of 64 (steps of 64 bytes
    // serve the reads alone, and put the widened rows' writes on the same banks: 272 us in place of 268, below).
    static constexpr int KP = D * 2 + 16, VP = D * 2 + 32;
    static constexpr int KBYTES = TILE * KP, VBYTES = TILE * VP;
    static constexpr int PARTS = D / 32, UNITS = TILE * PARTS;   // groups of 32 channels: of a row, of a tile's keys (or values)

    // Where a lane stands: its query row, what that sees, and what any row (lo, hi) or every row (from, all) of the
    // wavefront sees.
    int qi, qh, q_lo, q_hi, lo, hi, from, all;
    bool live;
    __device__ __forceinline__ void place(const AttArgs &a, const Seq &sq, int kvh, int r, int rows)
    {
        live = r < rows;
        qi = (int)fdiv((unsigned)(live ? r : 0), a.dv_group);
        qh = kvh * a.group + (live ? r : 0) - qi * a.group;
        seen(a, sq, qi, &q_lo, &q_hi);
        lo = live ? q_lo : 0x7FFFFFFF, hi = live ? q_hi : 0, from = live ? q_lo : 0, all = live ? q_hi : 0x7FFFFFFF;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            lo = min(lo, __shfl_xor(lo, d));
            hi = max(hi, __shfl_xor(hi, d));
            from = max(from, __shfl_xor(from, d));
            all = min(all, __shfl_xor(all, d));
        }
        lo = __builtin_amdgcn_readfirstlane(lo), hi = __builtin_amdgcn_readfirstlane(hi);
        from = __builtin_amdgcn_readfirstlane(from), all = __builtin_amdgcn_readfirstlane(all);
    }

    bf16x8 qf[D / 16];
    f32x16 o[D / 32];
    float m, l, c;   // m: the running maximum times c
    __device__ __forceinline__ void start(const AttArgs &a, const Seq &sq, int half)
    {
#pragma unroll
        for (int u = 0; u < D / 16; ++u) qf[u] = query8(a, a.q + (sq.row0 + qi) * a.qs + (long)qh * D + 8 * half + 16 * u);
        c = factor(a);
        m = kNegInf, l = 0.0f;
#pragma unroll
        for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[cb][i] = 0.0f;
    }

    // A lane's operand of the scores: row 32 b + lane % 32 of the keys, 16 bytes of step u.
    static __device__ __forceinline__ bf16x8 key(const unsigned char *kt, int lane, int b, int u)
    {
        return *(const bf16x8 *)(kt + (32 * b + lane % 32) * KP + 32 * u + 16 * (lane / 32));
    }
    // Of the values: channel 32 cb + lane % 32 of the lane's 8 tokens of a step of 16, 4 * half .. + 3 and 8 later, as
    // the scores have them.
    static __device__ __forceinline__ bf16x8 value(const unsigned char *vt, int lane, int cb, int k)
    {
        const unsigned char *at =
            vt + (16 * k + 4 * (lane / 32) + lane % 16 / 4) * VP + cb * 64 + lane / 16 % 2 * 32 + lane % 4 * 8;
        const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)at);
        const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + 8 * VP));
        return __builtin_shufflevector(__builtin_bit_cast(bf16x4, v0), __builtin_bit_cast(bf16x4, v1), 0, 1, 2, 3, 4, 5, 6, 7);
    }

    // Scores of 32 places at t0 that a row does not see become -inf.
    __device__ __forceinline__ void mask(f32x16 &x, int t0, int half)
    {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int at = t0 + i % 4 + 8 * (i / 4) + 4 * half;
            x[i] = at >= q_lo && at < q_hi ? x[i] : kNegInf;
        }
    }
    // The running maximum moves if a lane's scores, times c, pass it by far; l and o follow.
    __device__ __forceinline__ void grow(float top)
    {
        if (__any(top > m + kGrow)) {   // also where m is still -inf
            top = fmaxf(top, m);
            top = fmaxf(top, __shfl_xor(top, 32));
            const float f = top == m ? 1.0f : __builtin_amdgcn_exp2f(m - top);
            m = top;
            l *= f;
#pragma unroll
            for (int cb = 0; cb < D / 32; ++cb) o[cb] *= f;
        }
    }
    __device__ __forceinline__ float base() const { return m == kNegInf ? 0.0f : m; }

    // The row's result, or its part of a split.
    __device__ __forceinline__ void finish(const AttArgs &a, const Seq &sq, int s, int split, int half)
    {
        l += __shfl_xor(l, 32);
        if (!live) return;
        if (a.splits == 1) {
            const float f = l == 0.0f ? 0.0f : 1.0f / l;
            uint16_t *out = a.out + (sq.row0 + qi) * a.os + (long)qh * D + 4 * half;
#pragma unroll
            for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float v[4] = {o[cb][4 * i] * f, o[cb][4 * i + 1] * f, o[cb][4 * i + 2] * f, o[cb][4 * i + 3] * f};
                    store4(out + 32 * cb + 8 * i, v);
                }
        } else {
            float *part = a.part + ((((long)s * a.heads + qh) * a.max_new + qi) * a.splits + split) * (D + 4);
#pragma unroll
            for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float v[4] = {o[cb][4 * i], o[cb][4 * i + 1], o[cb][4 * i + 2], o[cb][4 * i + 3]};
                    store4(part + 32 * cb + 8 * i + 4 * half, v);
                }
            if (half == 0) part[D] = m, part[D + 1] = l;
        }
    }
};

// Keys or values of a tile on their way from the cache to LDS, by NT threads:
// groups of 32 channels by tokens.  Loads run a tile ahead of the conversion,
// the page table's two.
template <class F, int D, int NT>
struct Mover {
    static constexpr int PARTS = Wide<D>::PARTS, UNITS = Wide<D>::UNITS, PER = (UNITS + NT - 1) / NT;
    static constexpr int W = F::WORDS;
    uint32_t code[PER][4 * W];
    uint32_t exp[PER], vexp[PER];
    int page[PER], place[PER];

    __device__ __forceinline__ void look(const AttArgs &a, const int32_t *pages, int tid, int t0, int lo, int hi)
    {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            // before the start and past the end: a row that is seen, masked later
            const int t = max(lo, min(t0 + (i * NT + tid) / PARTS, hi - 1));
            const unsigned p = fdiv((unsigned)t, a.c.dv_page);
            place[i] = t - (int)p * a.c.page_size;
            page[i] = pages[p];
        }
    }
    __device__ __forceinline__ void fetch(const AttArgs &a, bool keys, int tid, int kvh)
    {
        const int last_page = (int)(a.c.slots / a.c.page_size) - 1;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const unsigned pg = (unsigned)min(max(page[i], 0), last_page);
            const uint64_t row = (uint64_t)pg * (unsigned)(a.c.heads * a.c.page_size) + (unsigned)(kvh * a.c.page_size + place[i]);
            const uint64_t at = row * PARTS + (unsigned)((i * NT + tid) % PARTS);
            load_words<4 * W>((keys ? a.c.kc : a.c.vc) + at * (16 * W), code[i]);
            const uint64_t e = F::GROUPS ? at : exponent_of(a.c, pg, kvh, place[i]);
            exp[i] = (keys ? a.c.ke : a.c.ve)[e];
            if constexpr (F::GROUPS) vexp[i] = a.c.ve[e];
        }
    }
    // One expression lets the wide kernel's two movers share their code: heads of 32 and 64 take 2.5 and 1.2% longer with an
    // expression for each, of 192 1%; of 96 and 256 it is the other way, by .6 and 1.6%.
    static constexpr bool SHARED = D <= 64 || D == 192;
    __device__ __forceinline__ float scale(int i, bool keys) const
    {
        if constexpr (F::GROUPS && SHARED) return F::scale(vexp[i] <= (uint32_t)kMaxExp ? exp[i] : keys ? 255u : 127u);
        else if constexpr (F::GROUPS) return keys ? F::keys(exp[i], vexp[i]) : F::values(exp[i]);
        else return keys ? F::keys(exp[i], 0) : F::values(exp[i]);
    }
    // For a tile with places that not every row of the block sees.
    __device__ __forceinline__ void clean()
    {
#pragma unroll
        for (int i = 0; i < PER; ++i)
#pragma unroll
            for (int j = 0; j < 4 * W; ++j) F::clean(code[i][j]);
    }
    __device__ __forceinline__ void widen(unsigned char *to, int pitch, bool keys, int tid)
    {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int idx = i * NT + tid;
            if (UNITS % NT == 0 || idx < UNITS) {
                unsigned char *at = to + idx / PARTS * pitch + idx % PARTS * 64;
                const float f = scale(i, keys);
#pragma unroll
                for (int j = 0; j < 4; ++j) *(bf16x8 *)(at + 16 * j) = F::widen8(code[i] + W * j, f);
            }
        }
    }
};

// The places that any row of a block sees within a split, and those that every row does (from, all).
__device__ __forceinline__ void block_range(const AttArgs &a, const Seq &sq, int r0, int r_last, int split, int *lo, int *hi,
                                            int *from, int *all)
{
    seen(a, sq, (int)fdiv((unsigned)r0, a.dv_group), lo, all);
    seen(a, sq, (int)fdiv((unsigned)r_last, a.dv_group), from, hi);
    *lo = (*lo & ~63) + split * a.per_split;   // per_split is a multiple of the tile
    *hi = *lo + min(*hi - *lo, a.per_split);
}

// A work-group's sequence, key head, split and block of rows, if there is one.
// A sequence's last rows see most under a causal mask: they go first, of every
// sequence and head, and the short work comes last.  Heads follow one another,
// so where they are a multiple of eight a head's work-groups share a die's L2.
__device__ __forceinline__ bool wide_place(const AttArgs &a, Seq *sq, int *s, int *kvh, int *split, int *r0, int *rows)
{
    const int pairs = a.seqs * a.c.heads, pair = blockIdx.x % pairs, rest = blockIdx.x / pairs;
    *kvh = pair % a.c.heads, *s = pair / a.c.heads, *split = rest % a.splits;
    *sq = sequence(a, *s);
    *rows = min(sq->news, a.max_new) * a.group;
    *r0 = ((*rows + kWideRows - 1) / kWideRows - 1 - rest / a.splits) * kWideRows;
    return *r0 >= 0;
}

// The wavefronts' barrier; loads of later tiles stay in flight across it.
__device__ __forceinline__ void wide_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Many rows, for heads of up to 64 channels, whose registers leave a SIMD four
// wavefronts, and of 192 and more, whose sums fill those of two (at 256 channels
// 256 registers, and 19 more in scratch).  The first four wavefronts move the
// keys and the others the values: the next tile is widened first, over the tile
// before, then this one worked on, and one barrier a tile keeps the wavefronts
// together.
//
// Two prompts of 4096 tokens, causal, 32 heads on 8 key heads: of 32 channels 133
// us, of 64 173 (755 TFLOP/s); 20 heads of 192 on 5, 283 us (870), 16 of 256 on
// 4, 294 (890), all in 4 bits; in 8 bits, where these take 130, 165, 292 and 290, 137,
// 176, 295 and 318.  Bound at few channels by vector instructions and products that
// take turns, for the barrier keeps a SIMD's wavefronts in much the same phase: of
// a SIMD's cycles the ones take 56% at 64 channels and the others 34%, 68 and 21%
// at 32.  Of the vector work the exponentials are less than a third.  At 256
// channels they take 24 and 37%; LDS is busy for 46% of the cycles, half of them
// bank conflicts, and the wavefronts wait for it and for one another.  With
// four wavefronts in place of eight, and registers for all they hold, the wide
// heads took 460 and 482 us: one wavefront a SIMD has nothing to overlap.
template <class F, int D>
__device__ __forceinline__ void attend_wide(const AttArgs &a)
{
    typedef Wide<D> W;
    constexpr int TILE = W::TILE;
    __shared__ __align__(16) unsigned char lds[2 * (W::KBYTES + W::VBYTES)];
    unsigned char *const keys = lds, *const vals = lds + 2 * W::KBYTES;

    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = lane / 32;
    int s, kvh, split, r0, rows, lo, hi, from, all;
    Seq sq;
    if (!wide_place(a, &sq, &s, &kvh, &split, &r0, &rows)) return;
    block_range(a, sq, r0, min(r0 + kWideRows, rows) - 1, split, &lo, &hi, &from, &all);
    const int tiles = hi > lo ? (hi - lo + TILE - 1) / TILE : 0;

    const int tid = threadIdx.x % 256;
    const bool mk = wave < 4;   // moves keys
    const int32_t *pages = a.table + (long)s * a.table_stride;
    Mover<F, D, 256> mv;
    const auto look = [&](int t) { mv.look(a, pages, tid, lo + t * TILE, lo, hi); };
    const auto widen = [&](int t) {
        if constexpr (!F::GROUPS)
            if (!mk && (lo + t * TILE < from || lo + (t + 1) * TILE > all)) mv.clean();
        if (mk) mv.widen(keys + (t & 1) * W::KBYTES, W::KP, true, tid);
        else mv.widen(vals + (t & 1) * W::VBYTES, W::VP, false, tid);
    };
    if (tiles > 0) look(0);
    W w;
    w.place(a, sq, kvh, r0 + 32 * wave + lane % 32, rows);
    if (tiles > 0) mv.fetch(a, mk, tid, kvh);
    w.start(a, sq, half);
    if (tiles > 0) {
        if (tiles > 1) look(1);
        widen(0);
        if (tiles > 1) mv.fetch(a, mk, tid, kvh);
        if (tiles > 2) look(2);
    }
    wide_barrier();
    for (int t = 0; t < tiles; ++t) {
        const int t0 = lo + t * TILE;
        const unsigned char *kt = keys + (t & 1) * W::KBYTES, *vt = vals + (t & 1) * W::VBYTES;
        if (t + 1 < tiles) {
            widen(t + 1);   // over a tile that was last read before the previous barrier
            if (t + 2 < tiles) mv.fetch(a, mk, tid, kvh);
            if (t + 3 < tiles) look(t + 3);
        }
        if (t0 < w.hi && t0 + TILE > w.lo) {
            f32x16 sc[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[b][i] = 0.0f;
#pragma unroll
                for (int u = 0; u < D / 16; ++u)
                    sc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(W::key(kt, lane, b, u), w.qf[u], sc[b], 0, 0, 0);
            }
            if (t0 < w.from || t0 + TILE > w.all) w.mask(sc[0], t0, half), w.mask(sc[1], t0 + 32, half);
            float top = kNegInf;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[b][i]);
            w.grow(top * w.c);
            const float base = w.base();
            bf16x8 pf[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                u32x4 p;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = 8 * (k % 2) + 2 * i;
                    p[i] = weights2(sc[k / 2][at], sc[k / 2][at + 1], w.c, base, w.l);
                }
                pf[k] = __builtin_bit_cast(bf16x8, p);
            }
#pragma unroll
            for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    w.o[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(W::value(vt, lane, cb, k), pf[k], w.o[cb], 0, 0, 0);
        }
        wide_barrier();
    }
    w.finish(a, sq, s, split, half);
}

template <int D>
__global__ __launch_bounds__(512, 2) void attend_kv4_wide_kernel(AttArgs a)
{
    attend_wide<Fp4, D>(a);
}

template <int D>   // up to 64 channels four wavefronts a SIMD, which 128 registers allow (left alone it takes 134)
__global__ __launch_bounds__(512, D <= 64 ? 4 : 2) void attend_kv8_wide_kernel(AttArgs a)
{
    attend_wide<Fp8, D>(a);
}

// Many rows, heads of 96 and 128 channels: two wavefronts on a SIMD, each of which
// gives the matrix cores and the vector unit work side by side.  A step takes 32
// cached tokens in two phases: the products of the NEXT step's scores beside
// this step's exponentials, then this step's sums of values beside the next
// step's maximum and a part of the tile that is being widened; operands are read
// from LDS a phase before their products.  Since scores run a step ahead, a
// tile's keys are those 32 tokens behind its values, and the keys of the first
// step come by themselves.
//
// Two prompts of 4096 tokens, causal, 32 heads of 128 on 8 key heads: 268 us, 975
// TFLOP/s (of 96: 229 us, 857); in 8 bits 283 (241).  The matrix cores alone would take
// 110 at full clock; with what each product has beside it a SIMD's product takes about 43
// cycles in place of 32 in a loop without memory (measured with four
// multiply-adds and two exponentials), which is 150, and the rest is barriers, LDS
// reads and the start of each block of rows.  Measured beside it: a tile's
// scores, probabilities and sums one after another 288; scores a step ahead,
// but in the compiler's order, 287, and 296 where it moves exponentials to the
// phase that needs them; 64 rows a wavefront, one on a SIMD, half the LDS reads,
// 286 (a lone wavefront's product takes 51 cycles in that loop); two groups of
// wavefronts half a tile apart 313.  Heads of 64 take 191 so, 173 in the kernel above.
template <class F, int D>
__device__ __forceinline__ void attend_steps(const AttArgs &a)
{
    typedef Wide<D> W;
    constexpr int TILE = W::TILE;
    constexpr int NQ = D / 16;   // products of a phase
    __shared__ __align__(16) unsigned char lds[2 * (W::KBYTES + W::VBYTES)];
    unsigned char *const keys = lds, *const vals = lds + 2 * W::KBYTES;

    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = lane / 32;
    int s, kvh, split, r0, rows, lo, hi, from, all;
    Seq sq;
    if (!wide_place(a, &sq, &s, &kvh, &split, &r0, &rows)) return;
    block_range(a, sq, r0, min(r0 + kWideRows, rows) - 1, split, &lo, &hi, &from, &all);
    const int tiles = hi > lo ? (hi - lo + TILE - 1) / TILE : 0;

    const int tid = threadIdx.x % 256;
    const bool mk = wave < 4;   // moves keys
    const int32_t *pages = a.table + (long)s * a.table_stride;
    Mover<F, D, 256> mv, first;
    const auto clean = [&](int t) {   // of values on their way to tile t
        if constexpr (!F::GROUPS)
            if (!mk && (lo + t * TILE < from || lo + (t + 1) * TILE > all)) mv.clean();
    };
    const auto look = [&](int t) { mv.look(a, pages, tid, lo + t * TILE + (mk ? 32 : 0), lo, hi); };
    if (tiles > 0) {
        first.look(a, pages, tid, lo - 32, lo, hi);
        look(0);
    }
    W w;
    w.place(a, sq, kvh, r0 + 32 * wave + lane % 32, rows);
    // the last step looks one ahead, past the end of a split too
    w.q_hi = min(w.q_hi, hi), w.all = min(w.all, hi);
    if (tiles > 0) {
        if (mk) first.fetch(a, true, tid, kvh);
        mv.fetch(a, mk, tid, kvh);
    }
    w.start(a, sq, half);
    if (tiles > 0) {
        if (tiles > 1) look(1);
        if (mk) {
            first.widen(keys + W::KBYTES, W::KP, true, tid);
            mv.widen(keys, W::KP, true, tid);
        } else {
            clean(0);
            mv.widen(vals, W::VP, false, tid);
        }
        if (tiles > 1) mv.fetch(a, mk, tid, kvh);
        if (tiles > 2) look(2);
    }
    wide_barrier();

    bf16x8 kf[NQ], vf[D / 32][2], pf[2];
    f32x16 even, odd;   // scores of a step, and of the next
    if (tiles > 0) {
        float top = kNegInf;
#pragma unroll
        for (int i = 0; i < 16; ++i) even[i] = 0.0f;
#pragma unroll
        for (int u = 0; u < NQ; ++u)
            even = __builtin_amdgcn_mfma_f32_32x32x16_bf16(W::key(keys + W::KBYTES, lane, 1, u), w.qf[u], even, 0, 0, 0);
        if (lo < w.from || lo + 32 > w.all) w.mask(even, lo, half);
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, even[i]);
        w.grow(top * w.c);
#pragma unroll
        for (int u = 0; u < NQ; ++u) kf[u] = W::key(keys, lane, 0, u);
    }
    wide_barrier();   // the first keys' place is that of the next tile's
    // The step of the scores x, of the 32 tokens at t0 (block h of the tile vt of values): their sums, and the next
    // step's scores y.  The barriers to the scheduler keep what stands side by side there.
    const auto step = [&](f32x16 &x, f32x16 &y, const unsigned char *vt, int h, int t0, auto between, auto beside) {
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = 0.0f;
        float f[8][2];
        u32x4 p[2];
        const float base = w.base();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 10; ++i) {   // two probabilities go through three turns: product, exponential, rounding
            if (i < 8) {
#pragma unroll
                for (int n = i * NQ / 8; n < (i + 1) * NQ / 8; ++n)
                    y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[n], w.qf[n], y, 0, 0, 0);
#pragma unroll
                for (int n = i * NQ / 8; n < (i + 1) * NQ / 8; ++n) vf[n / 2][n % 2] = W::value(vt, lane, n / 2, 2 * h + n % 2);
            }
            if (i >= 2) {
                const uint32_t two = pack_bf16x2(f[i - 2][0], f[i - 2][1]);
                w.l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), __builtin_bit_cast(bf16x2, 0x3F803F80u),
                                                      w.l, false);
                p[(i - 2) / 4][(i - 2) % 4] = two;
            }
            if (i >= 1 && i < 9)
                f[i - 1][0] = __builtin_amdgcn_exp2f(f[i - 1][0]), f[i - 1][1] = __builtin_amdgcn_exp2f(f[i - 1][1]);
            if (i < 8)
                f[i][0] = __builtin_fmaf(x[2 * i], w.c, -base), f[i][1] = __builtin_fmaf(x[2 * i + 1], w.c, -base);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            pf[k] = __builtin_bit_cast(bf16x8, p[k]);
            asm volatile("" : "+v"(pf[k]));   // or the exponentials move to the next phase
        }
        __builtin_amdgcn_sched_barrier(0);
        if (t0 + 32 < w.from || t0 + 64 > w.all) w.mask(y, t0 + 32, half);
        between();
        __builtin_amdgcn_sched_barrier(0);
        float top = kNegInf;
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            w.o[i / 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i / 2][i % 2], pf[i % 2], w.o[i / 2], 0, 0, 0);
            beside(i);
#pragma unroll
            for (int n = i * 8 / NQ; n < (i + 1) * 8 / NQ; ++n) top = fmaxf(fmaxf(top, y[2 * n]), y[2 * n + 1]);
            __builtin_amdgcn_sched_barrier(0);
        }
        w.grow(top * w.c);
    };
    static_assert(W::UNITS <= 256, "a thread moves a group of 32 channels of a tile");
    unsigned char *const put = (mk ? keys : vals) + tid / W::PARTS * (mk ? W::KP : W::VP) + tid % W::PARTS * 64;
    const int put_step = mk ? W::KBYTES : W::VBYTES;
    for (int t = 0; t < tiles; ++t) {
        const int t0 = lo + t * TILE, b = t & 1;
        const unsigned char *kt = keys + b * W::KBYTES, *kn = keys + (b ^ 1) * W::KBYTES, *vt = vals + b * W::VBYTES;
        // The next tile goes where nothing is read since the barrier before; the last one's turn writes what no one reads.
        unsigned char *const to = put + (b ^ 1) * put_step;
        const float scale = mv.scale(0, mk);
        clean(t + 1);
        step(even, odd, vt, 0, t0, [] {}, [&](int i) {
            kf[i] = W::key(kt, lane, 1, i);
            if (W::UNITS == 256 || tid < W::UNITS)
#pragma unroll
                for (int j = i * 4 / NQ; j < (i + 1) * 4 / NQ; ++j) *(bf16x8 *)(to + 16 * j) = F::widen8(mv.code[0] + F::WORDS * j, scale);
        });
        if (t + 2 < tiles) mv.fetch(a, mk, tid, kvh);
        if (t + 3 < tiles) look(t + 3);
        // past the barrier the next tile's keys are there, and this tile's values in registers
        step(odd, even, vt, 1, t0 + 32, [] { wide_barrier(); }, [&](int i) { kf[i] = W::key(kn, lane, 0, i); });
    }
    w.finish(a, sq, s, split, half);
}

template <int D>
__global__ __launch_bounds__(512, 2) void attend_kv4_steps_kernel(AttArgs a)
{
    attend_steps<Fp4, D>(a);
}

template <int D>
__global__ __launch_bounds__(512, 2) void attend_kv8_steps_kernel(AttArgs a)
{
    attend_steps<Fp8, D>(a);
}

// Joins the splits of a row of a head: four wavefronts take turns at them, four
// at a time.  All latency: the parts are asked for together, with what says
// whether there is such a row, and not after a first look at their maxima (one
// sequence of 1000 places 8.5 us, both kernels, where that takes 8.8, one of
// 30000 17.9 and 18.7; eight at a time 8.8 and 17.1).
template <int D>
__global__ __launch_bounds__(256) void attend_join_kernel(AttArgs a)
{
    constexpr int PER = (D + 63) / 64, AT = 4;
    __shared__ float sum[4][D], top[4], den[4];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, h = blockIdx.y, s = blockIdx.z, t = blockIdx.x;
    const float *part = a.part + (((long)s * a.heads + h) * a.max_new + t) * a.splits * (D + 4);
    const Seq sq = sequence(a, s);
    float m = kNegInf, l = 0.0f, v[PER] = {};
    for (int i = wave; i < a.splits; i += 4 * AT) {
        float pm[AT], pl[AT], pv[AT][PER];
#pragma unroll
        for (int k = 0; k < AT; ++k) {
            const float *p = part + (long)min(i + 4 * k, a.splits - 1) * (D + 4);
            pm[k] = p[D], pl[k] = p[D + 1];
#pragma unroll
            for (int j = 0; j < PER; ++j) pv[k][j] = p[min(j * 64 + lane, D - 1)];
        }
#pragma unroll
        for (int k = 0; k < AT; ++k) {
            const bool is = i + 4 * k < a.splits;   // not a branch, or each load waits for the one before
            pm[k] = is ? pm[k] : kNegInf, pl[k] = is ? pl[k] : 0.0f;
            const float mm = fmaxf(m, pm[k]);
            const float f = m == mm ? 1.0f : __builtin_amdgcn_exp2f(m - mm);
            const float g = pm[k] == mm ? 1.0f : __builtin_amdgcn_exp2f(pm[k] - mm);
            m = mm, l = l * f + pl[k] * g;
#pragma unroll
            for (int j = 0; j < PER; ++j) v[j] = v[j] * f + (is ? pv[k][j] : 0.0f) * g;
        }
    }
    if (lane == 0) top[wave] = m, den[wave] = l;
#pragma unroll
    for (int j = 0; j < PER; ++j)
        if (j * 64 + lane < D) sum[wave][j * 64 + lane] = v[j];
    __syncthreads();
    if (t >= sq.news || threadIdx.x >= D) return;   // of a row that is not there the parts are not set
    m = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
    float x = 0.0f;
    l = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float f = top[w] == m ? 1.0f : __builtin_amdgcn_exp2f(top[w] - m);
        l += den[w] * f, x += sum[w][threadIdx.x] * f;
    }
    store1(a.out + (sq.row0 + t) * a.os + (long)h * D + threadIdx.x, l == 0.0f ? 0.0f : x / l);
}

// Many rows: the heads that take them in steps.
constexpr bool in_steps(int D) { return D == 96 || D == 128; }

struct AttPlan {
    bool wide;
    int nb, row_blocks, splits, per_split;
    size_t bytes;
};

AttPlan plan_attend(const KvView &c, int seqs, int heads, int max_new, int max_len, int causal, int window)
{
    AttPlan p;
    const long group = heads / c.heads, rows = (long)max_new * group;
    // The kernel for few rows holds up to 64 of them in registers, fewer of wide heads.
    p.wide = rows > (c.dim <= 64 ? 64 : c.dim <= 128 ? 32 : 16);
    p.nb = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    const long block = p.wide ? kWideRows : 16 * p.nb;
    p.row_blocks = (int)((rows + block - 1) / block);
    // Places that a block of rows sees: with a window behind each, its own and those of the block's tokens.
    long len = max_len;
    // (std::min: HIP's own of two longs is that of their low 32 bits on the host.)
    if (causal && window > 0) len = std::min(len, (long)window + block / group + 1 + 64);
    // The places are split, at most until work-groups fill the card once, three on
    // a compute unit (one, with many rows): 16 sequences of up to 32768 places, 8 key
    // heads of 128, take 94 us so, 109 with four and 101 with six or eight.  Three is
    // what the registers allow there (<128, 1>), and at <64, 2> and <32, 4>; <64, 4>,
    // <96, 2>, <128, 2>, <192, 1> and <256, 1> allow two, the others four and more:
    // the fill was not measured on these.
    const long groups = (long)seqs * c.heads * p.row_blocks, fill = ((p.wide ? 1L : 3L) * cu_count() + groups - 1) / groups;
    long want = 1;
    if (p.wide) {
        // In n pieces all / n + 6 + n * part microseconds: the tiles of 64 places, the join,
        // and the parts, written and read.  16 heads on 4 key heads, causal: 1000 tokens, of
        // 128, take 33 us in one piece and 42 in two; 2000, of 96, 53 and 64; 100 tokens
        // behind 900, of 128, 20 in six pieces and 26 in two.
        const float all = (float)len / 64.0f * c.dim / 64.0f, part = 4e-6f * (float)seqs * (float)heads * (float)max_new * (c.dim + 4);
        const long n = std::max(1L, std::min({fill, (len + 127) / 128, (long)(sqrtf(all / part) + 0.5f)}));
        if (all / n + 6.0f + n * part < all) want = n;
    } else if (len > 384) {
        // 128 places at least, 256 beyond 32 splits: one sequence of 1000 takes 7.5 us so,
        // 8.5 with 256 and 7.6 with 64; one of 8000 10.0, and 10.9 with 128.  In one piece
        // 256 take 5.9 us (7.5 in two), 384 6.9 (7.6) and 640 8.4 (7.6).
        want = std::min(fill, std::max(std::min((len + 127) / 128, 32L), (len + 255) / 256));
    }
    p.per_split = (int)(((len + want - 1) / want + 63) / 64 * 64);
    p.splits = (int)((len + (long)p.per_split - 1) / p.per_split);
    p.bytes = p.splits > 1 ? (size_t)seqs * heads * max_new * p.splits * (c.dim + 4) * 4 : 0;
    return p;
}

int view(const quant_kv4 *cache, KvView *c) { return kv4_view(cache, c); }
int view(const quant_kv8 *cache, KvView *c) { return kv8_view(cache, c); }

template <class C>
int check_attend(const C *cache, int seqs, int heads, int max_new, int max_len, KvView *c)
{
    const int rc = view(cache, c);
    if (rc != MICONV_OK) return rc;
    if (seqs < 0 || heads < 1 || heads % c->heads || max_new < 1 || max_len < 1) return MICONV_ERR_SHAPE;
    if ((long)max_new * (heads / c->heads) >= 1L << 24 || max_len >= 1 << 30 || seqs > 65535 || heads > 65535)
        return MICONV_ERR_TOO_LARGE;
    if ((long)c->heads * c->page_size >= 1L << 31) return MICONV_ERR_TOO_LARGE;   // the kernels number a page's rows in 32 bits
    return MICONV_OK;
}

// Whether a grid, of fewer than 2^32 threads, holds the plan's.
bool grid_holds(const AttPlan &p, const KvView &c, int seqs)
{
    return (double)p.row_blocks * p.splits * (p.wide ? 512.0 * c.heads * seqs : 256.0) < 0x1p32;
}

template <class F, int D, int NB>
constexpr auto few_kernel()
{
    if constexpr (F::GROUPS) return attend_kv4_kernel<D, NB>;
    else return attend_kv8_kernel<D, NB>;
}

template <class F, int D>
constexpr auto many_kernel()
{
    if constexpr (F::GROUPS) {
        if constexpr (in_steps(D)) return attend_kv4_steps_kernel<D>;
        else return attend_kv4_wide_kernel<D>;
    } else {
        if constexpr (in_steps(D)) return attend_kv8_steps_kernel<D>;
        else return attend_kv8_wide_kernel<D>;
    }
}

template <class F, int D>
int launch_attend(const AttArgs &a, const AttPlan &p, hipStream_t st)
{
    const dim3 grid((unsigned)((long)p.row_blocks * p.splits), (unsigned)a.c.heads, (unsigned)a.seqs);
    if (p.wide) {
        const dim3 all(grid.x * grid.y * grid.z);
        launch_kernel(many_kernel<F, D>(), all, dim3(512), 0, st, a);
    } else {
        void (*k)(AttArgs) = few_kernel<F, D, 1>();
        if constexpr (D <= 128)
            if (p.nb == 2) k = few_kernel<F, D, 2>();
        if constexpr (D <= 64)
            if (p.nb == 4) k = few_kernel<F, D, 4>();
        launch_kernel(k, grid, dim3(256), 0, st, a);
    }
    int rc = launched();
    if (rc != MICONV_OK || p.splits == 1) return rc;
    launch_kernel(attend_join_kernel<D>, dim3((unsigned)a.max_new, (unsigned)a.heads, (unsigned)a.seqs), dim3(256), 0, st, a);
    return launched();
}

template <class C>
long attend_workspace(const C *cache, int seqs, int heads, int max_new, int max_len, int causal, int window)
{
    KvView c;
    const int rc = check_attend(cache, seqs, heads, max_new, max_len, &c);
    if (rc != MICONV_OK) return rc;
    return seqs ? (long)plan_attend(c, seqs, heads, max_new, max_len, causal, window).bytes : 0;
}

template <class C>
int attend_describe(const C *cache, int bits, int seqs, int heads, int max_new, int max_len, int causal, int window, char *buf,
                    int buflen, int *launches)
{
    if (!buf || buflen <= 0 || !launches) return MICONV_ERR_NULL;
    buf[0] = 0, *launches = 0;
    KvView c;
    const int rc = check_attend(cache, seqs, heads, max_new, max_len, &c);
    if (rc != MICONV_OK) return rc;
    if (seqs == 0) return MICONV_OK;
    const AttPlan p = plan_attend(c, seqs, heads, max_new, max_len, causal, window);
    if (!grid_holds(p, c, seqs)) return MICONV_ERR_TOO_LARGE;
    char first[64], join[64] = "";
    if (p.wide) snprintf(first, sizeof first, "attend_kv%d_%s_kernel<%d>", bits, in_steps(c.dim) ? "steps" : "wide", c.dim);
    else snprintf(first, sizeof first, "attend_kv%d_kernel<%d, %d>", bits, c.dim, p.nb);
    if (p.splits > 1) snprintf(join, sizeof join, " + attend_join_kernel<%d>", c.dim);
    *launches = p.splits > 1 ? 2 : 1;
    snprintf(buf, buflen, "%s%s", first, join);
    return MICONV_OK;
}

template <class F, class C>
int attend(const C *cache, int seqs, int heads, long tokens, const void *q, long q_stride, const int32_t *starts,
           const int32_t *lens, const int32_t *table, int table_stride, int max_new, int max_len, float scale, int causal,
           int window, void *out, long out_stride, void *ws, size_t ws_bytes, void *stream)
{
    AttArgs a = {};
    const int rc = check_attend(cache, seqs, heads, max_new, max_len, &a.c);
    if (rc != MICONV_OK) return rc;
    const long width = (long)heads * a.c.dim;
    a.scale = scale * 1.44269504088896340736f;
    if (tokens < 0 || q_stride < width || out_stride < width || table_stride < 1 || !__builtin_isfinite(a.scale))
        return MICONV_ERR_SHAPE;
    if (tokens >= 1L << 31) return MICONV_ERR_TOO_LARGE;
    if (seqs == 0 || tokens == 0) return MICONV_OK;
    if (!q || !out || !lens || !table) return MICONV_ERR_NULL;
    if (misaligned(q, 2) || misaligned(out, 2) || misaligned(starts, 4) || misaligned(lens, 4) || misaligned(table, 4))
        return MICONV_ERR_ALIGN;
    const AttPlan p = plan_attend(a.c, seqs, heads, max_new, max_len, causal, window);
    if (!grid_holds(p, a.c, seqs)) return MICONV_ERR_TOO_LARGE;
    if (p.bytes && (!ws || ws_bytes < p.bytes || misaligned(ws, 256))) return MICONV_ERR_WORKSPACE;
    a.q = (const uint16_t *)q, a.out = (uint16_t *)out;
    a.starts = starts, a.lens = lens, a.table = table;
    a.part = (float *)ws;
    a.qs = q_stride, a.os = out_stride, a.tokens = tokens;
    a.seqs = seqs, a.heads = heads, a.group = heads / a.c.heads, a.table_stride = table_stride;
    a.max_new = max_new, a.max_len = max_len;
    a.causal = causal, a.window = window;
    a.splits = p.splits, a.per_split = p.per_split, a.row_blocks = p.row_blocks;
    a.dv_group = make_fastdiv((unsigned)a.group);
    hipStream_t st = static_cast<hipStream_t>(stream);
    switch (a.c.dim) {
    case 32: return launch_attend<F, 32>(a, p, st);
    case 64: return launch_attend<F, 64>(a, p, st);
    case 96: return launch_attend<F, 96>(a, p, st);
    case 128: return launch_attend<F, 128>(a, p, st);
    case 192: return launch_attend<F, 192>(a, p, st);
    default: return launch_attend<F, 256>(a, p, st);
    }
}

}  // namespace
}  // namespace quant
}  // namespace miconv

extern "C" long quant_attention_workspace_bytes(const quant_kv4 *cache, int seqs, int heads, int max_new, int max_len,
                                                int causal, int window)
{
    return miconv::quant::attend_workspace(cache, seqs, heads, max_new, max_len, causal, window);
}

extern "C" int quant_attention_describe(const quant_kv4 *cache, int seqs, int heads, int max_new, int max_len, int causal,
                                        int window, char *buf, int buflen, int *launches)
{
    return miconv::quant::attend_describe(cache, 4, seqs, heads, max_new, max_len, causal, window, buf, buflen, launches);
}

extern "C" int quant_attention_kv4(const quant_kv4 *cache, int seqs, int heads, long tokens, const void *q,
                                   long q_stride, const int32_t *starts, const int32_t *lens, const int32_t *table,
                                   int table_stride, int max_new, int max_len, float scale, int causal, int window,
                                   void *out, long out_stride, void *ws, size_t ws_bytes, void *stream)
{
    return miconv::quant::attend<miconv::quant::Fp4>(cache, seqs, heads, tokens, q, q_stride, starts, lens, table, table_stride,
                                               max_new, max_len, scale, causal, window, out, out_stride, ws, ws_bytes, stream);
}

extern "C" long quant_attention_kv8_workspace_bytes(const quant_kv8 *cache, int seqs, int heads, int max_new, int max_len,
                                                int causal, int window)
{
    return miconv::quant::attend_workspace(cache, seqs, heads, max_new, max_len, causal, window);
}

extern "C" int quant_attention_kv8_describe(const quant_kv8 *cache, int seqs, int heads, int max_new, int max_len, int causal,
                                        int window, char *buf, int buflen, int *launches)
{
    return miconv::quant::attend_describe(cache, 8, seqs, heads, max_new, max_len, causal, window, buf, buflen, launches);
}

extern "C" int quant_attention_kv8(const quant_kv8 *cache, int seqs, int heads, long tokens, const void *q,
                                   long q_stride, const int32_t *starts, const int32_t *lens, const int32_t *table,
                                   int table_stride, int max_new, int max_len, float scale, int causal, int window,
                                   void *out, long out_stride, void *ws, size_t ws_bytes, void *stream)
{
    return miconv::quant::attend<miconv::quant::Fp8>(cache, seqs, heads, tokens, q, q_stride, starts, lens, table, table_stride,
                                               max_new, max_len, scale, causal, window, out, out_stride, ws, ws_bytes, stream);
}
