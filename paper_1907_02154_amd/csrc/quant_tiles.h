// What the products of 8-bit integers and of 8-bit floats share: the order of
// the tiles, their epilogue, and aligned copies of operands.
#pragma once

#include "quant.h"

namespace miconv {
namespace quant {

typedef int i32x4 __attribute__((ext_vector_type(4)));

struct MatArgs {
    const int8_t *a, *w;         // codes
    const float *sa, *sw, *bias; // sa, sw: of integers; of 8-bit floats sa or null, and no sw
    const void *res;
    void *y;
    long as, ws, rs, ys;   // row strides in elements
    int M, N, K;
    int relu;
    // tile order: tiles along m and n, tiles in all
    int mt, nt, tiles;
    FastDiv dv_group;      // by kGroup * nt
};

// The tiles of a product, and what a round of them takes: microseconds at K =
// 4096 with a work-group on each of 256 compute units, or, where two fit one,
// with one and with two on each.
struct Tile {
    int bm, bn, wm, wn, kg, nst;   // the kernel's parameters
    int per_cu;
    float one, two;
};

// The cheapest of n tiles for M x N outputs.
inline int pick_tile(const Tile *tiles, int n, int M, int N)
{
    const long cus = cu_count();
    int best = 0;
    double least = 1e300;
    for (int i = 0; i < n; ++i) {
        const Tile &t = tiles[i];
        const long all = (long)ceil_div(M, t.bm) * ceil_div(N, t.bn), round = cus * t.per_cu, rest = all % round;
        const double full = t.per_cu == 2 ? t.two : t.one;
        const double cost = (double)(all / round) * full + (rest == 0 ? 0.0 : rest > cus ? full : t.one);
        if (cost < least) least = cost, best = i;
    }
    return best;
}

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

// Four sums of token m, channels n .. n + 3, into y; with SW times the channels' scales.
template <typename T, bool SW, typename V>
__device__ __forceinline__ void finish4(const MatArgs &a, int m, int n, V sum, float sa)
{
    const int live = a.N - n;
    if (live <= 0) return;
    T *y = (T *)a.y + (long)m * a.ys + n;
    const T *res = a.res ? (const T *)a.res + (long)m * a.rs + n : nullptr;
    float v[4], f[4] = {}, b[4] = {};
    if (live >= 4) {
        if constexpr (SW) memcpy(f, a.sw + n, 16);
        if (a.bias) memcpy(b, a.bias + n, 16);
    } else {
        for (int i = 0; i < live; ++i) f[i] = SW ? a.sw[n + i] : 1.0f, b[i] = a.bias ? a.bias[n + i] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = SW ? (float)sum[i] * sa * f[i] : (float)sum[i] * sa;
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

template <int N>
__device__ __forceinline__ void wait_vmcnt()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

typedef __attribute__((address_space(3))) void lds_void_t;

// Whether an operand's rows can be loaded as they are: 16-byte chunks, and the
// 256 rows of the largest tile within the 31-bit offsets of a buffer.
inline bool rows_aligned(const void *p, long stride, long K)
{
    return K % 16 == 0 && stride % 16 == 0 && !misaligned(p, 16) && 256 * stride < 1L << 31;
}

inline long align_up(long v, long to) { return (v + to - 1) / to * to; }

// Bytes of the aligned copy of an operand that needs one.
inline long copy_bytes(long rows, const void *p, long stride, long K)
{
    return rows_aligned(p, stride, K) ? 0 : align_up(rows * align_up(K, 16), 256);
}

// Enqueues the copies of the operands of a.M, a.N rows that need one (ca, cw:
// copy_bytes) into the workspace, and points `a` to them.
int align_operands(MatArgs &a, long ca, long cw, void *ws, hipStream_t st);

}  // namespace quant
}  // namespace miconv
