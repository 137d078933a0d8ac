// Matrix product of 8-bit integers with scales for each token and channel
// (quant_matmul_i8): y[m][n] = act(sa[m] sw[n] sum_k a[m][k] w[n][k] + bias[n] + res[m][n]).
//
// v_mfma_i32_16x16x64_i8: the channels are the rows of the matrix instruction
// and the tokens its columns, so that a lane's four sums are four consecutive
// channels of one token.  The sums are exact 32-bit integers, so no tile and no
// order of the reduction changes a result.
//
// One kernel, tiles of eight sizes.  A few tokens are bound by the weights'
// bytes, many by the matrix cores; in between by what a compute unit can fetch,
// which grows with the wavefronts that wait side by side: there several groups
// of wavefronts share a tile and divide its reduction.
#include "quant.h"

#include <stdio.h>

namespace miconv {
namespace quant {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

struct MatArgs {
    const int8_t *a, *w;
    const float *sa, *sw, *bias;
    const void *res;
    void *y;
    long as, ws, rs, ys;   // row strides in elements
    int M, N, K;
    int relu;
    // tile order: tiles along m and n, tiles in all
    int mt, nt, tiles;
    FastDiv dv_group;      // by kGroup * nt
};

constexpr int kXcds = 8;    // a work-group runs on the die of its number modulo 8
constexpr int kGroup = 4;   // tiles along m that are taken together

// The tile of a work-group: each die gets a run of tiles that follow one
// another, down kGroup tiles and on to the next channels, so that what its
// work-groups read at a time meets in its L2.
__device__ __forceinline__ void tile_of(const MatArgs &a, int id, int *m, int *n)
{
    const int x = id % kXcds, q = a.tiles / kXcds, r = a.tiles % kXcds;
    const int t = x * q + (x < r ? x : r) + id / kXcds;
    const int g = (int)fdiv((unsigned)t, a.dv_group), in = t - g * kGroup * a.nt;
    const int rows = min(a.mt - g * kGroup, kGroup);
    *n = rows == kGroup ? in / kGroup : in / rows;
    *m = g * kGroup + in - *n * rows;
}

// Four sums of token m, channels n .. n + 3, into y.
template <typename T>
__device__ __forceinline__ void finish4(const MatArgs &a, int m, int n, i32x4 sum, float sa)
{
    const int live = a.N - n;
    if (live <= 0) return;
    T *y = (T *)a.y + (long)m * a.ys + n;
    const T *res = a.res ? (const T *)a.res + (long)m * a.rs + n : nullptr;
    float v[4], f[4] = {}, b[4] = {};
    if (live >= 4) {
        memcpy(f, a.sw + n, 16);
        if (a.bias) memcpy(b, a.bias + n, 16);
    } else {
        for (int i = 0; i < live; ++i) f[i] = a.sw[n + i], b[i] = a.bias ? a.bias[n + i] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)sum[i] * sa * f[i];
    if (a.bias)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += b[i];
    if (live >= 4) {
        if (res) {
            float r[4];
            load4(res, r);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += r[i];
        }
        if (a.relu)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = v[i] < 0.0f ? 0.0f : v[i];   // a NaN stays
        store4(y, v);
    } else {
        for (int i = 0; i < live; ++i) {
            float x = v[i];
            if (res) x += load1(res + i);
            if (a.relu) x = x < 0.0f ? 0.0f : x;
            store1(y + i, x);
        }
    }
}

// The first n of 16 bytes from p on, at any alignment, and zeros: the aligned
// words that hold at least one of them, shifted.
__device__ __forceinline__ i32x4 load16(const int8_t *p, int n)
{
    const int shift = (int)((uintptr_t)p & 3u);
    const uint32_t *at = (const uint32_t *)(p - shift);
    uint32_t d[5];
#pragma unroll
    for (int j = 0; j < 5; ++j) d[j] = 4 * j - shift < n ? at[j] : 0u;
    i32x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int live = n - 4 * j;
        const uint32_t keep = live >= 4 ? ~0u : live <= 0 ? 0u : (1u << (8 * live)) - 1u;
        v[j] = (int)(__builtin_amdgcn_alignbyte(d[j + 1], d[j], (unsigned)shift) & keep);
    }
    return v;
}

template <int N>
__device__ __forceinline__ void wait_vmcnt()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

typedef __attribute__((address_space(3))) void lds_void_t;

// BM tokens x BN channels a work-group of KG groups of WM x WN wavefronts; a
// stage is 128 bytes of the reduction for each group, NST of them in LDS, and
// the groups' sums meet in LDS at the end.  A row's eight 16-byte chunks lie
// rotated by an exclusive or with the row, so that the eight rows a group of
// lanes reads at once fall into different banks.
// Rows are 16-byte aligned with K % 16 == 0 and go straight into LDS.
//
// Kernel times: 8192 tokens, 4096 to 8192 channels 264 to 275 us, 2.0 to 2.1
// POP/s, which is what the matrix cores do at the clock their power leaves (four
// wavefronts of 128 x 128 in place of eight of 64 x 128: 346); 48 tokens, 4096 to
// 4096, 7.1 us and 512 tokens 15.6 (one group of wavefronts a tile: 12 and 25);
// one token, 1024 to 1024, 2.7 us, which a launch and two latencies take.  The
// reduction split over work-groups and joined by a second launch was never the
// faster way: that launch takes 4 us.
template <typename T, int BM, int BN, int WM, int WN, int KG, int NST>
__global__ __launch_bounds__(64 * WM * WN * KG) void matmul_i8_tile_kernel(MatArgs a)
{
    constexpr int NT = 64 * WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;   // NT: threads of a group
    constexpr int LOADS = (BM + BN) * 8 / NT, WL = BN * 8 / NT;   // chunks a thread stages, WL of them weights
    constexpr int STAGE = (BM + BN) * 8;                          // chunks of a group's stage
    static_assert(BN * 8 % NT == 0 && BM * 8 % NT == 0, "whole loads");
    static_assert((KG - 1) * BM * BN / 4 <= NST * KG * STAGE, "the groups' sums fit the stages");
    __shared__ i32x4 smem[NST * KG * STAGE];
    const int lane = threadIdx.x % 64, col = lane % 16, quad = lane / 16;
    const int kg = __builtin_amdgcn_readfirstlane(threadIdx.x / NT), tid = threadIdx.x % NT;
    const int wid = __builtin_amdgcn_readfirstlane(tid / 64);
    int m0, n0;
    tile_of(a, blockIdx.x, &m0, &n0);
    m0 *= BM, n0 *= BN;
    const int nm = min(a.M - m0, BM), nn = min(a.N - n0, BN);
    const int8_t *pa = a.a + (long)m0 * a.as, *pw = a.w + (long)n0 * a.ws;
    const int steps = ceil_div(a.K, 128 * KG);   // group kg has the part of 128 at (t * KG + kg) * 128

    // Thread's chunk i: row and place of the tile, from which its address follows.
    constexpr unsigned kOutside = 0x80000000u;   // past either buffer, whatever is added: zeros
    unsigned off[LOADS];
    int at_k[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int idx = i * NT + tid - (i < WL ? 0 : BN * 8), row = idx / 8, c = idx % 8 ^ (row & 7);
        const bool live = row < (i < WL ? nn : nm);
        at_k[i] = c * 16;
        off[i] = live ? (unsigned)(row * (i < WL ? a.ws : a.as)) + c * 16 : kOutside;
    }
    i32x4 acc[TN][TM] = {};
    int waddr[TN], aaddr[TM];
#pragma unroll
    for (int i = 0; i < TN; ++i) waddr[i] = (wid / WM * (BN / WN) + 16 * i + col) * 8;
#pragma unroll
    for (int j = 0; j < TM; ++j) aaddr[j] = BN * 8 + (wid % WM * (BM / WM) + 16 * j + col) * 8;
    // A small tile's operands are read at once, a large one's by halves.
    constexpr int HALVES = TN * TM <= 8 ? 2 : 1;
    const auto compute = [&](const i32x4 *st) {
#pragma unroll
        for (int h0 = 0; h0 < 2; h0 += HALVES) {
            i32x4 fw[HALVES][TN], fa[HALVES][TM];
#pragma unroll
            for (int h = 0; h < HALVES; ++h) {
                const int c = (4 * (h0 + h) + quad) ^ (col & 7);   // the rows' low bits are col's
#pragma unroll
                for (int i = 0; i < TN; ++i) fw[h][i] = st[waddr[i] + c];
#pragma unroll
                for (int j = 0; j < TM; ++j) fa[h][j] = st[aaddr[j] + c];
            }
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int h = 0; h < HALVES; ++h)
#pragma unroll
                for (int i = 0; i < TN; ++i)
#pragma unroll
                    for (int j = 0; j < TM; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[h][i], fa[h][j], acc[i][j], 0, 0, 0);
            __builtin_amdgcn_s_setprio(0);
        }
    };

    i32x4 *mine = smem + kg * STAGE;   // this group's part of the first stage
    const __amdgpu_buffer_rsrc_t wres = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<int8_t *>(pw), (short)0, (int)((nn - 1) * a.ws + a.K), 0x00020000);
    const __amdgpu_buffer_rsrc_t ares = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<int8_t *>(pa), (short)0, (int)((nm - 1) * a.as + a.K), 0x00020000);
    const auto issue = [&](int t, int stage) {
        i32x4 *st = mine + stage * (KG * STAGE) + wid * 64;
        const int k = (t * KG + kg) * 128;
        if (k + 128 <= a.K) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const unsigned o = off[i];
                __builtin_amdgcn_raw_ptr_buffer_load_lds(i < WL ? wres : ares, (lds_void_t *)(st + i * NT), 16, o, k, 0, 0);
            }
        } else {   // past K the next row begins
            // A group's part may begin past K: its loads are all outside, and their scalar offset has to stay below the
            // buffer's size, from which the hardware's range check may subtract it.
            const int base = k < a.K ? k : 0;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const unsigned o = k + at_k[i] < a.K ? off[i] : kOutside;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(i < WL ? wres : ares, (lds_void_t *)(st + i * NT), 16, o, base, 0, 0);
            }
        }
    };
#pragma unroll
    for (int t = 0; t < NST - 1; ++t)
        if (t < steps) issue(t, t);
    int stage = 0, fill = NST - 1;   // where stage t lies, and stage t + NST - 1
    for (int t = 0; t < steps; ++t) {
        // stage t has landed once only later stages' loads are outstanding
        if (steps - 1 - t >= NST - 2) wait_vmcnt<(NST - 2) * LOADS>();
        else wait_vmcnt<0>();
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");   // for every wavefront; stage t - 1 is done with
        if (t + NST - 1 < steps) issue(t + NST - 1, fill);
        compute(mine + stage * (KG * STAGE));
        stage = stage + 1 == NST ? 0 : stage + 1;
        fill = fill + 1 == NST ? 0 : fill + 1;
    }
    if constexpr (KG > 1) {
        __syncthreads();
        constexpr int BLOCKS = TN * TM * 64;   // sums of a wavefront
        if (kg > 0) {
#pragma unroll
            for (int i = 0; i < TN; ++i)
#pragma unroll
                for (int j = 0; j < TM; ++j)
                    smem[((kg - 1) * WM * WN + wid) * BLOCKS + (i * TM + j) * 64 + lane] = acc[i][j];
        }
        __syncthreads();
        if (kg > 0) return;
#pragma unroll
        for (int g = 0; g < KG - 1; ++g)
#pragma unroll
            for (int i = 0; i < TN; ++i)
#pragma unroll
                for (int j = 0; j < TM; ++j)
                    acc[i][j] += smem[(g * WM * WN + wid) * BLOCKS + (i * TM + j) * 64 + lane];
    }
#pragma unroll
    for (int j = 0; j < TM; ++j) {
        const int m = m0 + wid % WM * (BM / WM) + 16 * j + col;
        if (m >= a.M) continue;
        const float sa = a.sa[m];
#pragma unroll
        for (int i = 0; i < TN; ++i) finish4<T>(a, m, n0 + wid / WM * (BN / WN) + 16 * i + 4 * quad, acc[i][j], sa);
    }
}

// Rows of K bytes, at any alignment, into rows of `pitch` (a multiple of 16),
// zero from K on: one operand's rows, then the other's.  5 us of the 11.5 that 333
// tokens, 1999 to 1000 channels, take; the tiles' kernel took 24 with such rows
// through registers.
struct AlignArgs {
    const int8_t *src[2];
    int8_t *dst[2];
    long stride[2];
    int rows[2];
    int K, chunks;       // 16-byte chunks of a row
    unsigned total;
    FastDiv dv_chunks;
};

__global__ __launch_bounds__(256) void matmul_i8_align_kernel(AlignArgs a)
{
    const unsigned i = blockIdx.x * 256u + threadIdx.x;
    if (i >= a.total) return;
    int r = (int)fdiv(i, a.dv_chunks);
    const int c = (int)(i - (unsigned)r * (unsigned)a.chunks), o = r >= a.rows[0];
    r -= o ? a.rows[0] : 0;
    *(i32x4 *)(a.dst[o] + ((long)r * a.chunks + c) * 16) =
        load16(a.src[o] + r * a.stride[o] + 16 * c, min(a.K - 16 * c, 16));
}

// The tiles, and what a round of them takes: microseconds at K = 4096 with a
// work-group on each of 256 compute units, or, where two fit one, with one and
// with two on each (measured, random operands; the launch's own 2 us apart).
// Of two tiles that hold the same number of outputs the wider one suits few
// tokens.  (Two 16 x 32 tiles to a compute unit leave none for one of 32 x 32.)
//
// The costs' order is taken to hold at any K.  With every tile timed at K of 256,
// 1024, 4096 and 16384, for 1024, 4096 and 11000 channels and 1 to 2048 tokens, 81
// of 84 choices are the fastest tile or within 7% of it.  The others: 128 tokens,
// 1024 channels, where 16 x 16 and 16 x 32 tie and the first is taken (K = 4096 5.6
// us, and 4.8 the other; K = 16384 14.5 and 12.1), and 16 tokens, 11000 channels
// at K = 16384 (39.8, and 34.0 in tiles of 16 x 16).
struct Tile {
    int bm, bn, wm, wn, kg, nst;   // the kernel's parameters
    int per_cu;
    float one, two;
};
constexpr Tile kTiles[] = {
    {16, 16, 1, 1, 4, 4, 2, 3.4f, 3.8f},    {16, 32, 1, 2, 4, 3, 2, 3.8f, 5.0f},    {32, 64, 1, 4, 4, 3, 1, 6.6f, 0.0f},
    {64, 32, 2, 2, 4, 3, 1, 6.6f, 0.0f},    {64, 64, 2, 2, 2, 4, 1, 9.3f, 0.0f},    {128, 64, 4, 2, 2, 3, 1, 13.8f, 0.0f},
    {128, 128, 2, 4, 1, 3, 1, 22.3f, 0.0f}, {128, 128, 2, 2, 1, 2, 2, 28.0f, 38.0f}, {256, 256, 4, 2, 1, 2, 1, 66.0f, 0.0f},
};

int pick_tile(int M, int N)
{
    const long cus = cu_count();
    int best = 0;
    double least = 1e300;
    for (int i = 0; i < (int)(sizeof(kTiles) / sizeof(kTiles[0])); ++i) {
        const Tile &t = kTiles[i];
        const long tiles = (long)ceil_div(M, t.bm) * ceil_div(N, t.bn), round = cus * t.per_cu, rest = tiles % round;
        const double full = t.per_cu == 2 ? t.two : t.one;
        const double cost = (double)(tiles / round) * full + (rest == 0 ? 0.0 : rest > cus ? full : t.one);
        if (cost < least) least = cost, best = i;
    }
    return best;
}

template <typename T, int I>
int go_tile(MatArgs a, hipStream_t st)
{
    constexpr Tile t = kTiles[I];
    constexpr int threads = 64 * t.wm * t.wn * t.kg;
    a.mt = ceil_div(a.M, t.bm), a.nt = ceil_div(a.N, t.bn);
    // a grid holds fewer than 2^32 threads
    if ((long)a.mt * a.nt * threads >= 1L << 32 || (long)kGroup * a.nt >= 1L << 31) return MICONV_ERR_TOO_LARGE;
    a.tiles = a.mt * a.nt;
    a.dv_group = make_fastdiv((unsigned)(kGroup * a.nt));
    launch_kernel(matmul_i8_tile_kernel<T, t.bm, t.bn, t.wm, t.wn, t.kg, t.nst>, dim3((unsigned)a.tiles), dim3(threads), 0, st, a);
    return launched();
}

template <typename T>
int launch_matmul(const MatArgs &a, hipStream_t st)
{
    switch (pick_tile(a.M, a.N)) {
    case 0: return go_tile<T, 0>(a, st);
    case 1: return go_tile<T, 1>(a, st);
    case 2: return go_tile<T, 2>(a, st);
    case 3: return go_tile<T, 3>(a, st);
    case 4: return go_tile<T, 4>(a, st);
    case 5: return go_tile<T, 5>(a, st);
    case 6: return go_tile<T, 6>(a, st);
    case 7: return go_tile<T, 7>(a, st);
    default: return go_tile<T, 8>(a, st);
    }
}

// Whether an operand's rows can be loaded as they are: 16-byte chunks, and the
// 256 rows of the largest tile within the 31-bit offsets of a buffer.
bool rows_aligned(const int8_t *p, long stride, long K)
{
    return K % 16 == 0 && stride % 16 == 0 && !misaligned(p, 16) && 256 * stride < 1L << 31;
}

long align_up(long v, long to) { return (v + to - 1) / to * to; }

// Bytes of the aligned copy of an operand that needs one.
long copy_bytes(long rows, const int8_t *p, long stride, long K)
{
    return rows_aligned(p, stride, K) ? 0 : align_up(rows * align_up(K, 16), 256);
}

}  // namespace
}  // namespace quant
}  // namespace miconv

namespace {

int check_matmul(long M, long N, long K, long a_stride, long w_stride)
{
    if (M < 0 || N < 1 || K < 1 || a_stride < K || w_stride < K) return MICONV_ERR_SHAPE;
    // rows and channels are numbered in 32 bits, those of the last tile that are not there too
    if (M > (1L << 31) - 256 || N > (1L << 31) - 256 || K > 131071) return MICONV_ERR_TOO_LARGE;
    return MICONV_OK;
}

}  // namespace

extern "C" long quant_matmul_workspace_bytes(long M, long N, long K, const int8_t *a, long a_stride, const int8_t *w,
                                             long w_stride)
{
    using namespace miconv::quant;
    const int rc = check_matmul(M, N, K, a_stride, w_stride);
    if (rc != MICONV_OK) return rc;
    return M ? copy_bytes(M, a, a_stride, K) + copy_bytes(N, w, w_stride, K) : 0;
}

extern "C" int quant_matmul_describe(long M, long N, long K, const int8_t *a, long a_stride, const int8_t *w, long w_stride,
                                     int out_dtype, char *buf, int buflen, int *launches)
{
    using namespace miconv::quant;
    if (!buf || buflen <= 0 || !launches) return MICONV_ERR_NULL;
    buf[0] = 0, *launches = 0;
    const int rc = check_matmul(M, N, K, a_stride, w_stride);
    if (rc != MICONV_OK) return rc;
    if (!dtype_bytes(out_dtype)) return MICONV_ERR_UNSUPPORTED;
    if (M == 0) return MICONV_OK;
    const bool copy = copy_bytes(M, a, a_stride, K) + copy_bytes(N, w, w_stride, K) > 0;
    const Tile t = kTiles[pick_tile((int)M, (int)N)];
    *launches = 1 + copy;
    snprintf(buf, buflen, "%smatmul_i8_tile_kernel<%s, %d, %d, %d, %d, %d, %d>", copy ? "matmul_i8_align_kernel + " : "",
             out_dtype == kF32 ? "float" : "unsigned short", t.bm, t.bn, t.wm, t.wn, t.kg, t.nst);
    return MICONV_OK;
}

extern "C" int quant_matmul_i8(long M, long N, long K, const int8_t *a, long a_stride, const float *a_scale,
                               const int8_t *w, long w_stride, const float *w_scale, const float *bias,
                               const void *residual, long residual_stride, int out_dtype, void *y, long y_stride,
                               int relu, void *ws, size_t ws_bytes, void *stream)
{
    using namespace miconv;
    const int rc = check_matmul(M, N, K, a_stride, w_stride);
    if (rc != MICONV_OK) return rc;
    const int b = quant::dtype_bytes(out_dtype);
    if (!b) return MICONV_ERR_UNSUPPORTED;
    if (y_stride < N || (residual && residual_stride < N)) return MICONV_ERR_SHAPE;
    if (M == 0) return MICONV_OK;
    if (!a || !a_scale || !w || !w_scale || !y) return MICONV_ERR_NULL;
    if (quant::misaligned(a_scale, 4) || quant::misaligned(w_scale, 4) || quant::misaligned(bias, 4) ||
        quant::misaligned(residual, b) || quant::misaligned(y, b))
        return MICONV_ERR_ALIGN;
    const long ca = quant::copy_bytes(M, a, a_stride, K), cw = quant::copy_bytes(N, w, w_stride, K);
    if (ca + cw && (!ws || ws_bytes < (size_t)(ca + cw) || quant::misaligned(ws, 256))) return MICONV_ERR_WORKSPACE;
    quant::MatArgs args = {a, w, a_scale, w_scale, bias, residual, y, a_stride, w_stride, residual_stride,
                           y_stride, (int)M, (int)N, (int)K, relu, 0, 0, 0, {}};
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (ca + cw) {
        const long pitch = quant::align_up(K, 16);
        int8_t *to_a = (int8_t *)ws, *to_w = to_a + ca;
        quant::AlignArgs c = {{a, w}, {to_a, to_w}, {a_stride, w_stride}, {ca ? (int)M : 0, cw ? (int)N : 0},
                              (int)K, (int)(pitch / 16), 0, make_fastdiv((unsigned)(pitch / 16))};
        const long total = ((long)c.rows[0] + c.rows[1]) * c.chunks;
        if (total >= 1L << 31) return MICONV_ERR_TOO_LARGE;
        c.total = (unsigned)total;
        launch_kernel(quant::matmul_i8_align_kernel, dim3((unsigned)((total + 255) / 256)), dim3(256), 0, st, c);
        const int e = quant::launched();
        if (e != MICONV_OK) return e;
        if (ca) args.a = to_a, args.as = pitch;
        if (cw) args.w = to_w, args.ws = pitch;
        args.K = (int)pitch;   // the copies are zero from K on; an operand read in place has K % 16 == 0
    }
    return out_dtype == quant::kF32 ? quant::launch_matmul<float>(args, st) : quant::launch_matmul<uint16_t>(args, st);
}
