// Root-mean-square norm with the residual's addition and an 8-bit output, and
// the 8-bit output alone (quant_rmsnorm_i8, quant_rows_i8).
//
// With t = h * w and r = 1 / sqrt(mean(h^2) + eps) the normed row is t * r, its
// largest magnitude A * r with A = max |t|, and its 8-bit value
// rint(t * r * 127 / (A * r)) = rint(t * (127 / A)): r cancels.  So q depends
// on a maximum alone, which no order of evaluation changes, and the sum
// reaches the scale only.
//
// Bound by memory: a row is read once, kept in registers across the one
// reduction (sum and maximum together), and written once: 16384 rows of 4096 in
// bf16 with the residual, 470 MB, take 97 us, 4.8 TB/s (a large copy: 5.2).  A
// wavefront takes a row of up to 1024, so that short rows need no barrier; a
// work-group a longer one.
#include "quant.h"

namespace miconv {
namespace quant {
namespace {

struct RowArgs {
    const void *x, *res;
    const float *w;
    void *h;
    int8_t *q;
    float *scale;
    long xs, rs, hs, qs;   // row strides in elements
    long rows;
    int cols;
    int norm;              // 0: the 8-bit output alone
    float eps;
};

struct RowStat {
    float sum;       // of h^2
    uint32_t top;    // largest |t| as its bits: ordered like the magnitudes, infinity and NaN above all
};

__device__ __forceinline__ RowStat join(RowStat a, RowStat b)
{
    return RowStat{a.sum + b.sum, a.top > b.top ? a.top : b.top};
}

__device__ __forceinline__ RowStat wave_join(RowStat s)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) s = join(s, RowStat{__shfl_xor(s.sum, d), (uint32_t)__shfl_xor((int)s.top, d)});
    return s;
}

// The statistics of a row's WAVES wavefronts (of one wavefront: its lanes).
template <int WAVES>
__device__ __forceinline__ RowStat row_join(RowStat s, RowStat *part)
{
    s = wave_join(s);
    if (WAVES > 1) {
        if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = s;
        __syncthreads();
        s = part[0];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) s = join(s, part[i]);
    }
    return s;
}

// What fp32 holds of a sum of squares ends at magnitudes of 2^64, and below 2^-63
// squares lose bits.  Where that reaches the scale (the sum is infinite, or it
// and eps are below 2^-80) the row is read once more and the sum taken of
// (h unit^2)^2, which stays inside: rows whose h goes so far are rare, and the
// test is all that others pay.
__device__ __forceinline__ float row_unit_of_sum(const RowArgs &a, RowStat s)
{
    if (!a.norm || s.top >= 0x7F800000u || s.top < __builtin_bit_cast(uint32_t, 0x1p-100f)) return 1.0f;   // no sum is used
    return s.sum < 0x1p-80f && a.eps < 0x1p-80f ? 0x1p50f : s.sum == __builtin_inff() ? 0x1p-48f : 1.0f;
}

template <typename T, int LANES>
__device__ __forceinline__ float row_sum_again(const T *h, int cols, int lane, float unit)
{
    float sum = 0.0f;
    for (long at = (long)lane * 8; at < cols; at += LANES * 8)   // the elements that this thread wrote, where h was
        for (int i = 0; i < 8 && at + i < cols; ++i) {
            const float v = load1(h + at + i) * unit * unit;
            sum += v * v;
        }
    return sum;
}

// 127 / A and the row's scale; s.sum is that of (h unit^2)^2.
__device__ __forceinline__ float row_factor(const RowArgs &a, RowStat s, float unit, float *scale)
{
    const float top = __builtin_bit_cast(float, s.top);
    if (s.top >= 0x7F800000u) {
        *scale = __builtin_nanf("");
        return 0.0f;
    }
    if (top < 0x1p-100f) {   // 127 / A would overflow
        *scale = 0.0f;
        return 0.0f;
    }
    // in this order no step leaves fp32's range unless the scale itself does
    const float eps = a.eps * unit * unit * unit * unit;
    const float r = a.norm ? 1.0f / sqrtf(s.sum / (float)a.cols + eps) * unit : 1.0f;
    *scale = top * r * unit / 127.0f;
    return 127.0f / top;
}

__device__ __forceinline__ uint32_t quant4(const float *t, float f)
{
    uint32_t v = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) v |= ((uint32_t)(int)rintf(t[i] * f) & 255u) << (8 * i);
    return v;
}

// One unit of up to 8 elements at p: h (rounded to T) and its part of the statistics.
template <typename T>
__device__ __forceinline__ void row_unit(const RowArgs &a, const T *x, const T *res, T *h, int at, int n, float (&t)[8],
                                         RowStat &s)
{
    float w[8];
    if (n == 8) {
        load8(x + at, t);
        if (res) {
            float r[8];
            load8(res + at, r);
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = rounded(t[i] + r[i], x);
            store8(h + at, t);
        }
        if (a.w) load8(a.w + at, w);
    } else {   // all loads first: the last element stands in past the end
        float r[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int k = at + min(i, n - 1);
            t[i] = load1(x + k);
            r[i] = res ? load1(res + k) : 0.0f;
            w[i] = a.w ? a.w[k] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (res) t[i] = rounded(t[i] + r[i], x);
            if (i >= n) t[i] = 0.0f;
        }
        if (res)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < n) store1(h + at + i, t[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        s.sum += t[i] * t[i];
        if (a.w) t[i] = i < n ? t[i] * w[i] : 0.0f;
        const uint32_t b = __builtin_bit_cast(uint32_t, t[i]) & 0x7FFFFFFFu;
        s.top = b > s.top ? b : s.top;
    }
}

__device__ __forceinline__ void store_q(int8_t *q, int n, const float (&t)[8], float f)
{
    // f is 0 where q is: a NaN or an infinity times 0 must not reach the conversion
    uint32_t v[2] = {0, 0};
    if (f != 0.0f) v[0] = quant4(t, f), v[1] = quant4(t + 4, f);
    if (n == 8) {
        memcpy(q, v, 8);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) q[i] = (int8_t)(v[i / 4] >> (8 * (i % 4)));
    }
}

// LANES threads (a wavefront, or the whole work-group) share a row, U units of
// 8 elements each.
template <typename T, int LANES, int U>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void rows_i8_kernel(RowArgs a)
{
    constexpr int NT = LANES < 256 ? 256 : LANES, WAVES = LANES / 64;
    __shared__ RowStat part[WAVES > 1 ? WAVES : 1];
    const int lane = threadIdx.x % LANES;
    const long row = (long)blockIdx.x * (NT / LANES) + threadIdx.x / LANES;
    if (row >= a.rows) return;   // whole wavefronts; with LANES > 64 the grid has no such row
    const T *x = (const T *)a.x + row * a.xs;
    const T *res = a.res ? (const T *)a.res + row * a.rs : nullptr;
    T *h = a.res ? (T *)a.h + row * a.hs : nullptr;
    float t[U][8];
    RowStat s = {0.0f, 0u};
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int at = (u * LANES + lane) * 8, n = a.cols - at;
        if (n > 0) row_unit(a, x, res, h, at, n < 8 ? n : 8, t[u], s);
    }
    s = row_join<WAVES>(s, part);
    const float unit = row_unit_of_sum(a, s);   // the same for a row's threads
    if (unit != 1.0f) {
        if (WAVES > 1) __syncthreads();
        s.sum = row_join<WAVES>(RowStat{row_sum_again<T, LANES>(a.res ? h : x, a.cols, lane, unit), 0u}, part).sum;
    }
    float scale;
    const float f = row_factor(a, s, unit, &scale);
    int8_t *q = a.q + row * a.qs;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int at = (u * LANES + lane) * 8, n = a.cols - at;
        if (n > 0) store_q(q + at, n < 8 ? n : 8, t[u], f);
    }
    if (lane == 0) a.scale[row] = scale;
}

// Rows longer than the registers of a work-group hold: h is read again for the
// second pass (each thread reads back what it wrote itself), mostly from cache:
// 1024 rows of 65536 in bf16 55 us, 3.6 TB/s of what a single read and write is.
template <typename T>
__global__ __launch_bounds__(1024) void rows_i8_long_kernel(RowArgs a)
{
    __shared__ RowStat part[16];
    const long row = blockIdx.x;
    const T *x = (const T *)a.x + row * a.xs;
    const T *res = a.res ? (const T *)a.res + row * a.rs : nullptr;
    T *h = a.res ? (T *)a.h + row * a.hs : nullptr;
    RowStat s = {0.0f, 0u};
    float t[8];
    for (long at = threadIdx.x * 8; at < a.cols; at += 1024 * 8)
        row_unit(a, x, res, h, (int)at, a.cols - at < 8 ? (int)(a.cols - at) : 8, t, s);
    s = row_join<16>(s, part);
    const T *kept = a.res ? h : x;
    const float unit = row_unit_of_sum(a, s);
    if (unit != 1.0f) {
        __syncthreads();
        s.sum = row_join<16>(RowStat{row_sum_again<T, 1024>(kept, a.cols, threadIdx.x, unit), 0u}, part).sum;
    }
    float scale;
    const float f = row_factor(a, s, unit, &scale);
    int8_t *q = a.q + row * a.qs;
    for (long at = threadIdx.x * 8; at < a.cols; at += 1024 * 8) {
        const int n = a.cols - at < 8 ? (int)(a.cols - at) : 8;
        row_unit(a, kept, (const T *)nullptr, (T *)nullptr, (int)at, n, t, s);
        store_q(q + at, n, t, f);
    }
    if (threadIdx.x == 0) a.scale[row] = scale;
}

// Rows from r0 on.
RowArgs rows_from(RowArgs a, long r0, int bytes)
{
    a.x = (const char *)a.x + r0 * a.xs * bytes;
    if (a.res) a.res = (const char *)a.res + r0 * a.rs * bytes, a.h = (char *)a.h + r0 * a.hs * bytes;
    a.q += r0 * a.qs, a.scale += r0;
    a.rows -= r0;
    return a;
}

constexpr long kBlocks = 1L << 20;   // work-groups of a launch: a grid holds fewer than 2^32 threads

template <typename T, int LANES, int U>
void go(const RowArgs &a, hipStream_t st)
{
    constexpr int NT = LANES < 256 ? 256 : LANES;
    constexpr long PER = NT / LANES;
    for (long r0 = 0; r0 < a.rows; r0 += kBlocks * PER) {
        RowArgs part = rows_from(a, r0, sizeof(T));
        part.rows = part.rows < kBlocks * PER ? part.rows : kBlocks * PER;
        launch_kernel(rows_i8_kernel<T, LANES, U>, dim3((unsigned)((part.rows + PER - 1) / PER)), dim3(NT), 0, st, part);
    }
}

// Up to 1024 elements a wavefront has a row, so that there is no barrier; beyond,
// the threads and units that read fastest (without a residual, bf16 and fp32):
// 6000 rows of 12000 in 68 and 79 us (1024 threads of 4 units: 92 and 97; 512 of
// 4: 74 and 76), 3000 of 22000 in 57 and 78 (1024 of 4: 68 and 76; twice read: 60
// and 83), 1024 of 65536, twice read, 55 and 92.
template <typename T>
int launch_rows(const RowArgs &a, hipStream_t st)
{
    const int units = (int)((a.cols + 7L) / 8);
    if (units <= 64) go<T, 64, 1>(a, st);
    else if (units <= 128) go<T, 64, 2>(a, st);
    else if (units <= 256) go<T, 256, 1>(a, st);
    else if (units <= 512) go<T, 256, 2>(a, st);
    else if (units <= 1024) go<T, 256, 4>(a, st);
    else if (units <= 2048) go<T, 1024, 2>(a, st);
    else if (units <= 4096) go<T, 512, 8>(a, st);
    else
        for (long r0 = 0; r0 < a.rows; r0 += kBlocks) {
            const RowArgs part = rows_from(a, r0, sizeof(T));
            launch_kernel(rows_i8_long_kernel<T>, dim3((unsigned)(part.rows < kBlocks ? part.rows : kBlocks)), dim3(1024), 0, st, part);
        }
    return launched();
}

int run_rows(RowArgs a, long cols, int dtype, hipStream_t st)
{
    const int b = dtype_bytes(dtype);
    if (!b) return MICONV_ERR_UNSUPPORTED;
    if (a.rows < 0 || cols < 1 || a.xs < cols || a.qs < cols || !(a.eps >= 0.0f)) return MICONV_ERR_SHAPE;
    if (a.rows >= 1L << 31 || cols >= 1L << 31) return MICONV_ERR_TOO_LARGE;
    if (!a.res != !a.h) return MICONV_ERR_NULL;
    if (a.res && (a.rs < cols || a.hs < cols)) return MICONV_ERR_SHAPE;
    if (a.rows == 0) return MICONV_OK;
    if (!a.x || !a.q || !a.scale) return MICONV_ERR_NULL;
    if (misaligned(a.x, b) || misaligned(a.res, b) || misaligned(a.h, b) || misaligned(a.w, 4) || misaligned(a.scale, 4))
        return MICONV_ERR_ALIGN;
    a.cols = (int)cols;
    return dtype == kF32 ? launch_rows<float>(a, st) : launch_rows<uint16_t>(a, st);
}

}  // namespace
}  // namespace quant
}  // namespace miconv

extern "C" int quant_rmsnorm_i8(long rows, long cols, int dtype, const void *x, long x_stride, const void *residual,
                                long residual_stride, const float *weight, float eps, void *h, long h_stride,
                                int8_t *q, long q_stride, float *scale, void *stream)
{
    miconv::quant::RowArgs a = {x, residual, weight, h, q, scale, x_stride, residual_stride, h_stride, q_stride,
                                rows, 0, 1, eps};
    return miconv::quant::run_rows(a, cols, dtype, static_cast<hipStream_t>(stream));
}

extern "C" int quant_rows_i8(long rows, long cols, int dtype, const void *x, long x_stride, int8_t *q,
                             long q_stride, float *scale, void *stream)
{
    miconv::quant::RowArgs a = {x, nullptr, nullptr, nullptr, q, scale, x_stride, 0, 0, q_stride, rows, 0, 0, 0.0f};
    return miconv::quant::run_rows(a, cols, dtype, static_cast<hipStream_t>(stream));
}
