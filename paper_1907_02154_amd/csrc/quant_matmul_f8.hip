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
#include <type_traits>
#include <utility>

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

// Calls f(0) .. f(N - 1) with numbers that are constants: an instruction's choice of a byte is one.
template <typename F, int... I>
__device__ __forceinline__ void each_of(F f, std::integer_sequence<int, I...>)
{
    (f(std::integral_constant<int, I>()), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F f)
{
    each_of(f, std::make_integer_sequence<int, N>());
}
template <int N>
using Number = std::integral_constant<int, N>;

// The largest products with bf16 outputs, N % 8 == 0: 256 tokens x 256 channels
// a work-group of four wavefronts, one on each SIMD, each a square of 128 x 128,
// whose sums take half of the registers: a block's operands are read from LDS
// twice in all (128 KB of a block; by eight wavefronts, as above, 192, which is
// as long as the products take).
// A wavefront alone on its SIMD has to keep the matrix core busy by itself, so
// everything else is placed between the products, which take 64 turns a block:
// a block's tokens lie in registers before its first turn, and its channels come
// three groups of 8 turns ahead.  After 40 turns all of a block has been read;
// there the wavefronts meet, the block after it has landed, and in the last 24
// turns its tokens, first channels and exponents are read and the block after
// that one starts on its way into the place that has become free: 12 of its 18
// loads a thread, every other turn, and the rest in the next block's first 16,
// for a compute unit takes a load of 1 KB in 16 cycles, four wavefronts' 18 in
// 1152, and more at a time hold the products up (all in 18 turns: 228 us where
// this takes 215; 8 and 10: 218).  The channels
// of a lane's sums are eight that follow one another, stored as 16 bytes, four
// lanes 64; LDS chunks are rotated so that both orders of rows are free of
// conflicts.  Exponents come as four bytes a register, of which the instruction
// picks one.
// 8192 x 8192 outputs, K = 4096: 207 to 215 us, 2.55 to 2.66 PFLOP/s (the tile
// above: 255); K = 8192, half the outputs: 196 to 206 (246).  The library's products
// of these sizes without exponents took 180 and 168 on one card, 224 for the first
// on another, and at its best, 8192 x 8192 x 8192, 3.3 and 2.75 PFLOP/s.  The
// instruction alone, on such values in registers, reaches 3.7 to 4.5, as the
// clock follows the power it takes; a product has a turn of 44 to 50 cycles
// here, of which it takes 32.  Taking the next tile's first blocks while the last
// one's outputs are stored, in a grid of one work-group on each compute unit,
// took 235 where it took 227 without.
__global__ __launch_bounds__(256) void matmul_f8_large_kernel(F8Args f)
{
    const MatArgs &a = f.m;
    constexpr int B = 256, NT = 256, L = 8;          // L: chunks of either operand that a thread stages
    constexpr int EXPS = 2 * B * 8, STAGE = EXPS + 2 * B / 4;
    __shared__ i32x4 smem[2 * STAGE];
    const int tid = threadIdx.x, lane = tid % 64, col = lane % 16, quad = lane / 16;
    const int wid = __builtin_amdgcn_readfirstlane(tid / 64), wn = wid / 2, wm = wid % 2;
    int m0, n0;
    tile_of(a, blockIdx.x, &m0, &n0);
    m0 = __builtin_amdgcn_readfirstlane(m0) * B, n0 = __builtin_amdgcn_readfirstlane(n0) * B;
    const int nm = min(a.M - m0, B), nn = min(a.N - n0, B);
    const auto buffer = [&](const void *p, long first, int rows, long stride, int len) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>((const uint8_t *)p + first * stride), (short)0,
                                                 __builtin_amdgcn_readfirstlane((int)((rows - 1) * stride + len)), 0x00020000);
    };
    const __amdgpu_buffer_rsrc_t wres = buffer(a.w, n0, nn, a.ws, a.K), ares = buffer(a.a, m0, nm, a.as, a.K);
    const __amdgpu_buffer_rsrc_t ewres = buffer(f.ew, n0, nn, f.ews, f.blocks), eares = buffer(f.ea, m0, nm, f.eas, f.blocks);

    // A thread stages chunks of rows 32 n + tid / 8; rows that are not there lie past their buffer's end.
    constexpr unsigned kOutside = 0x80000000u;
    const int srow = tid / 8, at_k = (tid % 8 ^ ((srow & 3) | (srow >> 3 & 1) << 2)) * 16;
    const unsigned offw = (unsigned)(srow * a.ws) + at_k, offa = (unsigned)(srow * a.as) + at_k;
    const unsigned nextw = (unsigned)(32 * a.ws), nexta = (unsigned)(32 * a.as);
    // Its exponents: a lane's eight lie side by side; where there is no such row, the last's, of no output.
    const int half = tid / 128 * 128, ej = tid % 8, ecol = tid % 128 / 8;
    const int erw = half + 32 * (ej / 2) + 8 * (ecol / 4) + 4 * (ej % 2) + ecol % 4, erm = half + 16 * ej + ecol;
    const unsigned offew = (unsigned)(min(erw, nn - 1) * f.ews), offea = (unsigned)(min(erm, nm - 1) * f.eas);
    // Load n, of 18, of a block; past the last block zeros, with its exponents.
    struct Block {
        int base, exps;
        unsigned outside;
    };
    const auto block_at = [&](int b) {
        const bool is = b < f.blocks;
        return Block{is ? b * 128 : 0, min(b, f.blocks - 1), is && b * 128 + at_k < a.K ? 0u : kOutside};
    };
    const auto load = [&](auto nc, int stage, const Block &b) {
        constexpr int n = decltype(nc)::value;
        i32x4 *st = smem + stage * STAGE + wid * 64;
        if constexpr (n < L)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(wres, (lds_void_t *)(st + n * NT), 16, (offw | b.outside) + n * nextw, b.base, 0, 0);
        else if constexpr (n < 2 * L)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ares, (lds_void_t *)(st + n * NT), 16, (offa | b.outside) + (n - L) * nexta, b.base,
                                                     0, 0);
        else
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                n == 2 * L ? ewres : eares, (lds_void_t *)((int *)(smem + stage * STAGE + EXPS) + (n - 2 * L) * NT + wid * 64), 1,
                n == 2 * L ? offew : offea, b.exps, 0, 0);
    };

    // Channel rows 32 (i / 2) + 8 (col / 4) + 4 (i % 2) + col % 4, token rows 16 j + col, of the wavefront's 128.
    f32x4 acc[8][8] = {};
    i32x8 fa[2][8], fw[4];
    i32x4 ex[4];
    uint32_t ea[2][2], ew[2][2];
    const int w0 = (wn * 128 + 8 * (col / 4) + col % 4) * 8 + (quad ^ (col & 7));
    const int a0 = (B + wm * 128 + col) * 8 + (quad ^ ((col & 3) | (col >> 3 & 1) << 2));
    const auto read_w = [&](int stage, auto ic) {
        constexpr int i = decltype(ic)::value;
        const i32x4 *st = smem + stage * STAGE + (32 * (i / 2) + 4 * (i % 2)) * 8;
        fw[i % 4] = __builtin_shufflevector(st[w0], st[w0 ^ 4], 0, 1, 2, 3, 4, 5, 6, 7);
    };
    const auto read_a = [&](auto pc, auto jc) {
        constexpr int p = decltype(pc)::value, j = decltype(jc)::value;
        const i32x4 *st = smem + p * STAGE + 16 * j * 8;
        fa[p][j] = __builtin_shufflevector(st[a0], st[a0 ^ 4], 0, 1, 2, 3, 4, 5, 6, 7);
    };
    const auto read_e = [&](int stage) {
        const i32x4 *e = smem + stage * STAGE + EXPS;
        const int w = wn * 32 + col * 2, t = (B / 4) + wm * 32 + col * 2;
        ex[0] = e[w], ex[1] = e[w + 1], ex[2] = e[t], ex[3] = e[t + 1];
    };
    const auto pack = [&](i32x4 v) { return (uint32_t)(v[0] | v[1] << 8 | v[2] << 16 | v[3] << 24); };
    const auto pack_e = [&](auto pc) {
        constexpr int p = decltype(pc)::value;
        ew[p][0] = pack(ex[0]), ew[p][1] = pack(ex[1]), ea[p][0] = pack(ex[2]), ea[p][1] = pack(ex[3]);
    };
    // A block in stage p, the next in the other, of which the last loads are issued first; then, once p is read, the first
    // kEarly of `after` into p.
    constexpr int kEarly = 12;
    const auto step = [&](auto pc, const Block &next, const Block &after) {
        constexpr int p = decltype(pc)::value, q = 1 - p;
        each<8>([&](auto ic) {
            constexpr int i = decltype(ic)::value;
            if constexpr (i == 5) {
                // The built-in wait, not one in asm: what has been read by now need not be waited for again.
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0)
                asm volatile("s_barrier" ::: "memory");
                __builtin_amdgcn_sched_barrier(0);
            }
            each<8>([&](auto jc) {
                constexpr int j = decltype(jc)::value;
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw[i % 4], fa[p][j], acc[i][j], 0, 0, i % 4, ew[p][i / 4],
                                                                            j % 4, ea[p][j / 4]);
                if constexpr (i < 5) {
                    if constexpr (j == 0) read_w(p, Number<i + 3>());
                    if constexpr (i < 2 && j % 3 == 1) load(Number<kEarly + 3 * i + j / 3>(), q, next);
                } else {
                    constexpr int n = (i - 5) * 8 + j;
                    if constexpr (n == 0) read_w(q, Number<0>()), read_e(q);
                    else if constexpr (n <= 8) read_a(Number<q>(), Number<n - 1>());
                    else if constexpr (n == 9) read_w(q, Number<1>());
                    else if constexpr (n == 17) read_w(q, Number<2>());
                    if constexpr (n == 15) pack_e(Number<q>());
                    if constexpr (n % 2 == 1) load(Number<n / 2>(), p, after);
                }
                __builtin_amdgcn_sched_barrier(0);
            });
        });
    };
    each<18>([&](auto n) { load(n, 0, block_at(0)); });
    each<kEarly>([&](auto n) { load(n, 1, block_at(1)); });
    wait_vmcnt<kEarly>();
    asm volatile("s_barrier" ::: "memory");
    read_w(0, Number<0>()), read_e(0);
    each<8>([&](auto j) { read_a(Number<0>(), j); });
    read_w(0, Number<1>());
    read_w(0, Number<2>());
    pack_e(Number<0>());
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
    for (int b = 0; b < f.blocks; b += 2) {   // of an odd number the last is one of zeros
        step(Number<0>(), block_at(b + 1), block_at(b + 2));
        step(Number<1>(), block_at(b + 2), block_at(b + 3));
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

    const int n = n0 + wn * 128 + 8 * quad;   // + 32 c: a lane's eight channels
    float bias[4][8] = {};
    if (a.bias)
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (n + 32 * c < a.N) memcpy(bias[c], a.bias + n + 32 * c, 32);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int m = m0 + wm * 128 + 16 * j + col;
        const float sa = a.sa ? a.sa[min(m, a.M - 1)] : 1.0f;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = acc[2 * c + e / 4][j][e % 4] * sa;
            if (a.bias)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += bias[c][e];
            if (m >= a.M || n + 32 * c >= a.N) continue;
            if (a.res) {
                float r[8];
                load8((const uint16_t *)a.res + (long)m * a.rs + n + 32 * c, r);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += r[e];
            }
            if (a.relu)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = v[e] < 0.0f ? 0.0f : v[e];   // a NaN stays
            store8((uint16_t *)a.y + (long)m * a.ys + n + 32 * c, v);
        }
    }
}

// Costs as measured for 8-bit integers, whose products take as long as those with
// bf16 outputs; the last one's its own.  fp32 outputs take up to twice as long by
// any tile, which leaves the order.  With every tile timed at K = 1024 to 4096, N =
// 1000 to 11000, M from 1 to 8192 and both outputs, the cheapest by this rule is
// the fastest or a few percent off (fp32 as bf16); worst are 128 tokens, 1024
// channels and K = 4096, 6.0 us where tiles of 16 x 32 take 5.3, and 2048 tokens,
// 11000 channels, 104 where the largest tile takes 95.
constexpr Tile kTiles[] = {
    {16, 16, 1, 1, 4, 4, 2, 3.4f, 3.8f},    {16, 32, 1, 2, 4, 3, 2, 3.8f, 5.0f},    {32, 64, 1, 4, 4, 3, 1, 6.6f, 0.0f},
    {64, 32, 2, 2, 4, 3, 1, 6.6f, 0.0f},    {64, 64, 2, 2, 2, 4, 1, 9.3f, 0.0f},    {128, 64, 4, 2, 2, 3, 1, 13.8f, 0.0f},
    {128, 128, 2, 4, 1, 3, 1, 22.3f, 0.0f}, {128, 128, 2, 2, 1, 2, 2, 28.0f, 38.0f}, {256, 256, 4, 2, 1, 2, 1, 66.0f, 0.0f},
    {256, 256, 2, 2, 1, 2, 1, 57.0f, 0.0f},   // matmul_f8_large_kernel
};
constexpr int kCount = sizeof(kTiles) / sizeof(kTiles[0]), kLarge = kCount - 1;

// far: an operand's exponents lie so far apart that 256 rows of them pass a buffer's 31-bit offsets.
int pick(int M, int N, int out_dtype, bool far)
{
    return pick_tile(kTiles, out_dtype == kBF16 && N % 8 == 0 && !far ? kCount : kLarge, M, N);
}

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
    if constexpr (I == kLarge) launch_kernel(matmul_f8_large_kernel, dim3((unsigned)a.tiles), dim3(threads), 0, st, f);
    else launch_kernel(matmul_f8_tile_kernel<T, t.bm, t.bn, t.wm, t.wn, t.kg, t.nst>, dim3((unsigned)a.tiles), dim3(threads), 0, st, f);
    return launched();
}

template <typename T>
int launch_matmul(const F8Args &f, hipStream_t st)
{
    const bool far = 256 * (f.eas > f.ews ? f.eas : f.ews) >= 1L << 31;
    switch (pick(f.m.M, f.m.N, std::is_same<T, float>::value ? kF32 : kBF16, far)) {
    case 0: return go_tile<T, 0>(f, st);
    case 1: return go_tile<T, 1>(f, st);
    case 2: return go_tile<T, 2>(f, st);
    case 3: return go_tile<T, 3>(f, st);
    case 4: return go_tile<T, 4>(f, st);
    case 5: return go_tile<T, 5>(f, st);
    case 6: return go_tile<T, 6>(f, st);
    case 7: return go_tile<T, 7>(f, st);
    case 8: return go_tile<T, 8>(f, st);
    default: return go_tile<T, kLarge>(f, st);
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
    const int at = pick((int)M, (int)N, out_dtype, false);
    const Tile t = kTiles[at];
    const char *first = copy ? "matmul_i8_align_kernel + " : "";
    *launches = 1 + copy;
    if (at == kLarge) {
        snprintf(buf, buflen, "%smatmul_f8_large_kernel", first);
        return MICONV_OK;
    }
    snprintf(buf, buflen, "%smatmul_f8_tile_kernel<%s, %d, %d, %d, %d, %d, %d>", first,
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
