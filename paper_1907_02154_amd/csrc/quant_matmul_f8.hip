// Matrix product of 8-bit floats with a power of two for each 128 values of a
// row (quant_matmul_f8):
//   y[m][n] = act(sa[m] sum_b 2^(ea[m][b] + ew[n][b]) sum_(k in b) a[m][k] w[n][k] + bias[n] + res[m][n]).
//
// bf16 outputs: v_mfma_scale_f32_16x16x128_f8f6f4.  One instruction multiplies
// a block of 128 of 16 channels and 16 tokens and takes both blocks' exponent
// bytes as they are stored, so that scaling costs no vector instruction.  It adds
// the products of eight neighbours aligned to the largest, each cut to a multiple
// of 2^-13 of the largest one's power of two (measured: next to 2^16, 8 counts
// and 6 does not, in any place of the eight and with either sign), and such sums
// in fp32 (24 bits).  Of random values that is 7e-5 of a sum, against the 1.7e-3
// of the output's rounding to bf16.
//
// fp32 outputs: the values, which bf16 holds with their exponents, go to
// v_mfma_f32_16x16x32_bf16, whose sums keep 24 bits throughout, at half the rate.
//
// The channels are the rows of the matrix instruction and the tokens its
// columns, so that a lane's four sums are four consecutive channels of one token.
// The order of a sum is fixed by the tile and the number of groups.
#include "quant_tiles.h"

#include <stdio.h>

namespace miconv {
namespace quant {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(1))) void global_void_t;

struct F8Args {
    MatArgs m;
    const uint8_t *ea, *ew;   // exponent bytes [M][blocks], [N][blocks]
    long eas, ews;            // their row strides
    int blocks;
};

// 16 values of a row as bf16.
__device__ __forceinline__ void widen(i32x4 code, int byte, bf16x8 (&to)[2])
{
    const float s = f8_power(byte);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        const uint32_t lo = (uint32_t)code[2 * n], hi = (uint32_t)code[2 * n + 1];
        const u32x4 r = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true))};
        to[n] = __builtin_bit_cast(bf16x8, r);
    }
}

// BM tokens x BN channels a work-group of KG groups of WM x WN wavefronts; a
// stage is a block of 128 for each group, its values and its exponents, NST of
// them in LDS, and the groups' sums meet in LDS at the end.  A row's eight
// 16-byte chunks lie rotated by an exclusive or with the row, so that the eight
// rows a group of lanes reads at once fall into different banks.  Which of a
// block's 128 places a lane holds is free, as long as both operands agree: a
// lane's 32 bytes are the chunks `quad` and 4 + `quad`.
// Rows are 16-byte aligned with K % 16 == 0 and go straight into LDS; so do the
// exponents, a byte a row, which arrive as words.
template <typename T, int BM, int BN, int WM, int WN, int KG, int NST>
__global__ __launch_bounds__(64 * WM * WN * KG) void matmul_f8_tile_kernel(F8Args f)
{
    const MatArgs &a = f.m;
    constexpr int NT = 64 * WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;   // NT: threads of a group
    constexpr int LOADS = (BM + BN) * 8 / NT, WL = BN * 8 / NT;   // chunks a thread stages, WL of them weights
    constexpr int STAGE = (BM + BN) * 8 + NT / 4;                 // 16-byte chunks of a group's stage, words of exponents last
    constexpr int EXPS = (BM + BN) * 8;
    static_assert(BN * 8 % NT == 0 && BM * 8 % NT == 0 && BM + BN <= NT, "whole loads, an exponent a thread at most");
    static_assert((KG - 1) * BM * BN / 4 <= NST * KG * STAGE, "the groups' sums fit the stages");
    __shared__ i32x4 smem[NST * KG * STAGE];
    const int lane = threadIdx.x % 64, col = lane % 16, quad = lane / 16;
    const int kg = __builtin_amdgcn_readfirstlane(threadIdx.x / NT), tid = threadIdx.x % NT;
    const int wid = __builtin_amdgcn_readfirstlane(tid / 64);
    int m0, n0;
    tile_of(a, blockIdx.x, &m0, &n0);
    m0 = __builtin_amdgcn_readfirstlane(m0) * BM, n0 = __builtin_amdgcn_readfirstlane(n0) * BN;
    const int nm = min(a.M - m0, BM), nn = min(a.N - n0, BN);
    const int8_t *pa = a.a + (long)m0 * a.as, *pw = a.w + (long)n0 * a.ws;
    const int steps = ceil_div(f.blocks, KG);   // group kg has blocks t * KG + kg

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
    // Its row's exponents: channels first, then tokens.  Where there is no such row, or block, those of the last stand in:
    // the values are 0 there, or belong to no output.
    const bool of_w = tid < BN;
    const int last = (of_w ? nn : nm) - 1, erow = min(max(of_w ? tid : tid - BN, 0), last);
    const uint8_t *ep = (of_w ? f.ew : f.ea) + ((of_w ? n0 : m0) + erow) * (of_w ? f.ews : f.eas);
    f32x4 acc[TN][TM] = {};
    int waddr[TN], aaddr[TM];
#pragma unroll
    for (int i = 0; i < TN; ++i) waddr[i] = wid / WM * (BN / WN) + 16 * i + col;
#pragma unroll
    for (int j = 0; j < TM; ++j) aaddr[j] = BN + wid % WM * (BM / WM) + 16 * j + col;
    const int c0 = quad ^ (col & 7), c1 = c0 ^ 4;   // the rows' low bits are col's
    const auto operand = [&](const i32x4 *st, int row) {
        return __builtin_shufflevector(st[row * 8 + c0], st[row * 8 + c1], 0, 1, 2, 3, 4, 5, 6, 7);
    };
    constexpr bool kWide = sizeof(T) == 4;
    const auto compute = [&](const i32x4 *st) {
        const int *ex = (const int *)(st + EXPS);
        int ea[TM], ew[TN];
#pragma unroll
        for (int j = 0; j < TM; ++j) ea[j] = ex[aaddr[j]];
#pragma unroll
        for (int i = 0; i < TN; ++i) ew[i] = ex[waddr[i]];
        if constexpr (kWide) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {   // a lane's chunks one after the other
                const int c = h ? c1 : c0;
                bf16x8 fa[TM][2];
#pragma unroll
                for (int j = 0; j < TM; ++j) widen(st[aaddr[j] * 8 + c], ea[j], fa[j]);
                __builtin_amdgcn_s_setprio(1);
#pragma unroll
                for (int i = 0; i < TN; ++i) {
                    bf16x8 fw[2];
                    widen(st[waddr[i] * 8 + c], ew[i], fw);
#pragma unroll
                    for (int j = 0; j < TM; ++j)
#pragma unroll
                        for (int n = 0; n < 2; ++n)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[n], fa[j][n], acc[i][j], 0, 0, 0);
                }
                __builtin_amdgcn_s_setprio(0);
            }
        } else {
            i32x8 fa[TM], fw[2];   // the next channels' weights come while these are multiplied
            fw[0] = operand(st, waddr[0]);
#pragma unroll
            for (int j = 0; j < TM; ++j) fa[j] = operand(st, aaddr[j]);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int i = 0; i < TN; ++i) {
                if (i + 1 < TN) fw[(i + 1) % 2] = operand(st, waddr[i + 1]);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < TM; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw[i % 2], fa[j], acc[i][j], 0, 0, 0, ew[i], 0, ea[j]);
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_s_setprio(0);
        }
    };

    i32x4 *mine = smem + kg * STAGE;   // this group's part of the first stage
    const __amdgpu_buffer_rsrc_t wres = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<int8_t *>(pw), (short)0, __builtin_amdgcn_readfirstlane((int)((nn - 1) * a.ws + a.K)), 0x00020000);
    const __amdgpu_buffer_rsrc_t ares = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<int8_t *>(pa), (short)0, __builtin_amdgcn_readfirstlane((int)((nm - 1) * a.as + a.K)), 0x00020000);
    constexpr int PER = LOADS + 1;   // loads of a stage
    const auto issue = [&](int t, int stage) {
        i32x4 *st = mine + stage * (KG * STAGE) + wid * 64;
        const int b = t * KG + kg, k = b * 128;
        // A group's block may lie past the last: its loads are all outside, and their scalar offset has to stay below the
        // buffer's size, from which the hardware's range check may subtract it.
        const int base = b < f.blocks ? k : 0;
        if (k + 128 <= a.K) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const unsigned o = off[i];
                __builtin_amdgcn_raw_ptr_buffer_load_lds(i < WL ? wres : ares, (lds_void_t *)(st + i * NT), 16, o, base, 0, 0);
            }
        } else {   // past K the next row begins
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const unsigned o = k + at_k[i] < a.K ? off[i] : kOutside;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(i < WL ? wres : ares, (lds_void_t *)(st + i * NT), 16, o, base, 0, 0);
            }
        }
        int *to = (int *)(mine + stage * (KG * STAGE) + EXPS) + wid * 64;
        __builtin_amdgcn_global_load_lds((const global_void_t *)(ep + min(b, f.blocks - 1)), (lds_void_t *)to, 1, 0, 0);
    };
#pragma unroll
    for (int t = 0; t < NST - 1; ++t)
        if (t < steps) issue(t, t);
    int stage = 0, fill = NST - 1;   // where stage t lies, and stage t + NST - 1
    for (int t = 0; t < steps; ++t) {
        // stage t has landed once only later stages' loads are outstanding
        if (steps - 1 - t >= NST - 2) wait_vmcnt<(NST - 2) * PER>();
        else wait_vmcnt<0>();
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");   // for every wavefront; stage t - 1 is done with
        if (t + NST - 1 < steps) issue(t + NST - 1, fill);
        compute(mine + stage * (KG * STAGE));
        stage = stage + 1 == NST ? 0 : stage + 1;
        fill = fill + 1 == NST ? 0 : fill + 1;
    }
    if constexpr (KG > 1) {
        __syncthreads();
        f32x4 *sums = (f32x4 *)smem;
        constexpr int BLOCKS = TN * TM * 64;   // sums of a wavefront
        if (kg > 0) {
#pragma unroll
            for (int i = 0; i < TN; ++i)
#pragma unroll
                for (int j = 0; j < TM; ++j)
                    sums[((kg - 1) * WM * WN + wid) * BLOCKS + (i * TM + j) * 64 + lane] = acc[i][j];
        }
        __syncthreads();
        if (kg > 0) return;
#pragma unroll
        for (int g = 0; g < KG - 1; ++g)
#pragma unroll
            for (int i = 0; i < TN; ++i)
#pragma unroll
                for (int j = 0; j < TM; ++j)
                    acc[i][j] += sums[(g * WM * WN + wid) * BLOCKS + (i * TM + j) * 64 + lane];
    }
#pragma unroll
    for (int j = 0; j < TM; ++j) {
        const int m = m0 + wid % WM * (BM / WM) + 16 * j + col;
        if (m >= a.M) continue;
        const float sa = a.sa ? a.sa[m] : 1.0f;
#pragma unroll
        for (int i = 0; i < TN; ++i) finish4<T, false>(a, m, n0 + wid / WM * (BN / WN) + 16 * i + 4 * quad, acc[i][j], sa);
    }
}

constexpr Tile kTiles[] = {
    {16, 16, 1, 1, 4, 4, 2, 3.4f, 3.8f},    {16, 32, 1, 2, 4, 3, 2, 3.8f, 5.0f},    {32, 64, 1, 4, 4, 3, 1, 6.6f, 0.0f},
    {64, 32, 2, 2, 4, 3, 1, 6.6f, 0.0f},    {64, 64, 2, 2, 2, 4, 1, 9.3f, 0.0f},    {128, 64, 4, 2, 2, 3, 1, 13.8f, 0.0f},
    {128, 128, 2, 4, 1, 3, 1, 22.3f, 0.0f}, {128, 128, 2, 2, 1, 2, 2, 28.0f, 38.0f}, {256, 256, 4, 2, 1, 2, 1, 66.0f, 0.0f},
};

int pick(int M, int N) { return pick_tile(kTiles, (int)(sizeof(kTiles) / sizeof(kTiles[0])), M, N); }

template <typename T, int I>
int go_tile(F8Args f, hipStream_t st)
{
    constexpr Tile t = kTiles[I];
    constexpr int threads = 64 * t.wm * t.wn * t.kg;
    MatArgs &a = f.m;
    a.mt = ceil_div(a.M, t.bm), a.nt = ceil_div(a.N, t.bn);
    // a grid holds fewer than 2^32 threads
    if ((long)a.mt * a.nt * threads >= 1L << 32 || (long)kGroup * a.nt >= 1L << 31) return MICONV_ERR_TOO_LARGE;
    a.tiles = a.mt * a.nt;
    a.dv_group = make_fastdiv((unsigned)(kGroup * a.nt));
    launch_kernel(matmul_f8_tile_kernel<T, t.bm, t.bn, t.wm, t.wn, t.kg, t.nst>, dim3((unsigned)a.tiles), dim3(threads), 0, st, f);
    return launched();
}

template <typename T>
int launch_matmul(const F8Args &f, hipStream_t st)
{
    switch (pick(f.m.M, f.m.N)) {
    case 0: return go_tile<T, 0>(f, st);
    case 1: return go_tile<T, 1>(f, st);
    case 2: return go_tile<T, 2>(f, st);
    case 3: return go_tile<T, 3>(f, st);
    case 4: return go_tile<T, 4>(f, st);
    case 5: return go_tile<T, 5>(f, st);
    case 6: return go_tile<T, 6>(f, st);
    case 7: return go_tile<T, 7>(f, st);
    default: return go_tile<T, 8>(f, st);
    }
}

int check_matmul(long M, long N, long K, long a_stride, long w_stride)
{
    if (M < 0 || N < 1 || K < 1 || a_stride < K || w_stride < K) return MICONV_ERR_SHAPE;
    // rows and channels are numbered in 32 bits, those of the last tile that are not there too; a copied row's 256 are
    // within a buffer's 31-bit offsets
    if (M > (1L << 31) - 256 || N > (1L << 31) - 256 || K > (1L << 23) - 16) return MICONV_ERR_TOO_LARGE;
    return MICONV_OK;
}

}  // namespace
}  // namespace quant
}  // namespace miconv

extern "C" long quant_matmul_f8_workspace_bytes(long M, long N, long K, const void *a, long a_stride, const void *w,
                                                long w_stride)
{
    using namespace miconv::quant;
    const int rc = check_matmul(M, N, K, a_stride, w_stride);
    if (rc != MICONV_OK) return rc;
    return M ? copy_bytes(M, a, a_stride, K) + copy_bytes(N, w, w_stride, K) : 0;
}

extern "C" int quant_matmul_f8_describe(long M, long N, long K, const void *a, long a_stride, const void *w, long w_stride,
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
    const Tile t = kTiles[pick((int)M, (int)N)];
    *launches = 1 + copy;
    snprintf(buf, buflen, "%smatmul_f8_tile_kernel<%s, %d, %d, %d, %d, %d, %d>", copy ? "matmul_i8_align_kernel + " : "",
             out_dtype == kF32 ? "float" : "unsigned short", t.bm, t.bn, t.wm, t.wn, t.kg, t.nst);
    return MICONV_OK;
}

extern "C" int quant_matmul_f8(long M, long N, long K, const void *a, long a_stride, const uint8_t *a_exps,
                               long a_exps_stride, const float *a_scale, const void *w, long w_stride,
                               const uint8_t *w_exps, long w_exps_stride, const float *bias, const void *residual,
                               long residual_stride, int out_dtype, void *y, long y_stride, int relu, void *ws,
                               size_t ws_bytes, void *stream)
{
    using namespace miconv;
    const int rc = quant::check_matmul(M, N, K, a_stride, w_stride);
    if (rc != MICONV_OK) return rc;
    const int b = quant::dtype_bytes(out_dtype);
    if (!b) return MICONV_ERR_UNSUPPORTED;
    const long blocks = (K + quant::kF8Block - 1) / quant::kF8Block;
    if (y_stride < N || (residual && residual_stride < N) || a_exps_stride < blocks || w_exps_stride < blocks)
        return MICONV_ERR_SHAPE;
    if (M == 0) return MICONV_OK;
    if (!a || !a_exps || !w || !w_exps || !y) return MICONV_ERR_NULL;
    if (quant::misaligned(a_scale, 4) || quant::misaligned(bias, 4) || quant::misaligned(residual, b) ||
        quant::misaligned(y, b))
        return MICONV_ERR_ALIGN;
    const long ca = quant::copy_bytes(M, a, a_stride, K), cw = quant::copy_bytes(N, w, w_stride, K);
    if (ca + cw && (!ws || ws_bytes < (size_t)(ca + cw) || quant::misaligned(ws, 256))) return MICONV_ERR_WORKSPACE;
    quant::F8Args f = {{(const int8_t *)a, (const int8_t *)w, a_scale, nullptr, bias, residual, y, a_stride, w_stride,
                        residual_stride, y_stride, (int)M, (int)N, (int)K, relu, 0, 0, 0, {}},
                       a_exps, w_exps, a_exps_stride, w_exps_stride, (int)blocks};
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (ca + cw) {
        const int e = quant::align_operands(f.m, ca, cw, ws, st);
        if (e != MICONV_OK) return e;
    }
    return out_dtype == quant::kF32 ? quant::launch_matmul<float>(f, st) : quant::launch_matmul<uint16_t>(f, st);
}
