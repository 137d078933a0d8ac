// Root-mean-square norm with the residual's addition and an output in 8-bit
// floats with a power of two for each 128, and that output alone
// (quant_rmsnorm_f8, quant_rows_f8).
//
// With t = h * w the normed row is t * r, r = 1 / sqrt(mean(h^2) + eps).  The
// blocks hold t, and r is an output of its own, which the product multiplies
// its sums by: a block's exponent and values depend on a maximum of 128
// numbers alone, which no order of evaluation changes, and nothing waits for
// the sum of the row.
//
// Bound by memory: 16384 rows of 4096 in bf16 with the residual, 470 MB, 98 us,
// 4.8 TB/s (a copy of 2 GiB: 4.9).  16 lanes share a block, whose largest value
// takes four steps between lanes; sums of squares and the norm's factor are fp32.
#include "quant.h"

namespace miconv {
namespace quant {
namespace {

struct RowArgs {
    const void *x, *res;
    const float *w;
    void *h;
    uint8_t *q, *e;
    float *scale;                  // null: the 8-bit output alone
    long xs, rs, hs, qs, es;       // row strides in elements
    long rows;
    int cols;
    float eps;
};

__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7FFFFFFFu; }

// The units that LANES threads hold of a row: 8 elements each, 16 neighbours a block of 128.
template <typename T, int LANES, int U>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void rows_f8_kernel(RowArgs a)
{
    constexpr int NT = LANES < 256 ? 256 : LANES, WAVES = LANES / 64;
    __shared__ float part[WAVES > 1 ? WAVES : 1];
    const int lane = threadIdx.x % LANES;
    const long row = (long)blockIdx.x * (NT / LANES) + threadIdx.x / LANES;
    if (row >= a.rows) return;   // whole wavefronts; with LANES > 64 the grid has no such row
    const T *x = (const T *)a.x + row * a.xs;
    const T *res = a.res ? (const T *)a.res + row * a.rs : nullptr;
    T *h = a.res ? (T *)a.h + row * a.hs : nullptr;
    uint8_t *q = a.q + row * a.qs, *eo = a.e + row * a.es;
    float sum = 0.0f;
    for (long at0 = 0; at0 < a.cols; at0 += (long)U * LANES * 8) {
        float t[U][8], r[U][8];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long at = at0 + (u * LANES + lane) * 8;
            if (at + 8 <= a.cols) {
                load8(x + at, t[u]);
                if (res) load8(res + at, r[u]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {   // a row's last elements one by one, and zeros
                    t[u][i] = at + i < a.cols ? load1(x + at + i) : 0.0f;
                    r[u][i] = res && at + i < a.cols ? load1(res + at + i) : 0.0f;
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long at = at0 + (u * LANES + lane) * 8;
            const int n = at >= a.cols ? 0 : a.cols - at < 8 ? (int)(a.cols - at) : 8;
            if (res) {
#pragma unroll
                for (int i = 0; i < 8; ++i) t[u][i] = rounded(t[u][i] + r[u][i], x);
                if (n == 8) store8(h + at, t[u]);
                else
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (i < n) store1(h + at + i, t[u][i]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += t[u][i] * t[u][i];
            if (a.w) {
                float w[8];
                if (n == 8) load8(a.w + at, w);
                else
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] = i < n ? a.w[at + i] : 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) t[u][i] *= w[i];
            }
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, magnitude(t[u][i]));
#pragma unroll
            for (int d = 1; d < 16; d *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
            int byte = f8_byte(top);
            const float power = f8_power(byte);
            uint32_t v[2] = {f8_encode4(t[u], power), f8_encode4(t[u] + 4, power)};
            if (top >= 0x7F800000u) byte = 255, v[0] = v[1] = 0;   // the product makes NaN of it
            if (n == 8) memcpy(q + at, v, 8);
            else
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < n) q[at + i] = (uint8_t)(v[i / 4] >> (8 * (i % 4)));
            if (lane % 16 == 0 && n > 0) eo[at / kF8Block] = (uint8_t)byte;
        }
    }
    if (!a.scale) return;
    const auto join = [&](float s) {
#pragma unroll
        for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d);
        if (WAVES > 1) {
            __syncthreads();
            if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = s;
            __syncthreads();
            s = part[0];
#pragma unroll
            for (int i = 1; i < WAVES; ++i) s += part[i];
        }
        return s;
    };
    sum = join(sum);
    // What fp32 holds of a sum of squares ends at magnitudes of 2^64, and below 2^-63 squares lose bits: rows that go so
    // far, which are rare, are read once more and the sum taken of (h unit^2)^2.
    const float unit = sum < 0x1p-80f && a.eps < 0x1p-80f ? 0x1p50f : sum == __builtin_inff() ? 0x1p-48f : 1.0f;
    if (unit != 1.0f) {   // the same for a row's threads
        sum = 0.0f;
        const T *kept = res ? h : x;   // the elements that this thread wrote, where h was
        for (long at = (long)lane * 8; at < a.cols; at += LANES * 8)
            for (int i = 0; i < 8 && at + i < a.cols; ++i) {
                const float v = load1(kept + at + i) * unit * unit;
                sum += v * v;
            }
        sum = join(sum);
    }
    const float eps = a.eps * unit * unit * unit * unit;
    // A finite row's factor is at most fp32's largest number: what would pass that belongs to a row whose values are all 0.
    if (lane == 0)
        a.scale[row] = sum < __builtin_inff() ? fminf(1.0f / sqrtf(sum / (float)a.cols + eps) * unit * unit, 0x1.fffffep127f)
                                              : __builtin_nanf("");
}

constexpr long kBlocks = 1L << 20;   // work-groups of a launch: a grid holds fewer than 2^32 threads

template <typename T, int LANES, int U>
void go(const RowArgs &a, hipStream_t st)
{
    constexpr int NT = LANES < 256 ? 256 : LANES;
    constexpr long PER = NT / LANES;
    for (long r0 = 0; r0 < a.rows; r0 += kBlocks * PER) {
        RowArgs p = a;
        p.x = (const T *)a.x + r0 * a.xs;
        if (a.res) p.res = (const T *)a.res + r0 * a.rs, p.h = (T *)a.h + r0 * a.hs;
        p.q += r0 * a.qs, p.e += r0 * a.es;
        if (a.scale) p.scale += r0;
        p.rows = a.rows - r0 < kBlocks * PER ? a.rows - r0 : kBlocks * PER;
        launch_kernel(rows_f8_kernel<T, LANES, U>, dim3((unsigned)((p.rows + PER - 1) / PER)), dim3(NT), 0, st, p);
    }
}

template <typename T>
int launch_rows(const RowArgs &a, hipStream_t st)
{
    // A wavefront a row as far as two units a lane hold it, else a work-group.  Rows of 1024, one and 16384 of them: 2.5 and
    // 12.8 us so, 2.5 and 21.4 with a work-group each; of 2048 3.5 and 20.9 against 2.2 and 20.7; of 512, one unit a lane
    // in place of two, 2.0 and 7.9 against 2.8 and 12.7.
    const int units = (int)((a.cols + 7L) / 8);
    if (units <= 64) go<T, 64, 1>(a, st);
    else if (units <= 128) go<T, 64, 2>(a, st);
    else if (units <= 256) go<T, 256, 1>(a, st);
    else go<T, 256, 2>(a, st);
    return launched();
}

int run_rows(RowArgs a, long cols, int dtype, hipStream_t st)
{
    const int b = dtype_bytes(dtype);
    if (!b) return MICONV_ERR_UNSUPPORTED;
    const long blocks = (cols + kF8Block - 1) / kF8Block;
    if (a.rows < 0 || cols < 1 || a.xs < cols || a.qs < cols || a.es < blocks || !(a.eps >= 0.0f)) return MICONV_ERR_SHAPE;
    if (a.rows >= 1L << 31 || cols >= 1L << 31) return MICONV_ERR_TOO_LARGE;
    if (!a.res != !a.h) return MICONV_ERR_NULL;
    if (a.res && (a.rs < cols || a.hs < cols)) return MICONV_ERR_SHAPE;
    if (a.rows == 0) return MICONV_OK;
    if (!a.x || !a.q || !a.e) return MICONV_ERR_NULL;
    if (misaligned(a.x, b) || misaligned(a.res, b) || misaligned(a.h, b) || misaligned(a.w, 4) || misaligned(a.scale, 4))
        return MICONV_ERR_ALIGN;
    a.cols = (int)cols;
    return dtype == kF32 ? launch_rows<float>(a, st) : launch_rows<uint16_t>(a, st);
}

}  // namespace
}  // namespace quant
}  // namespace miconv

extern "C" int quant_rmsnorm_f8(long rows, long cols, int dtype, const void *x, long x_stride, const void *residual,
                                long residual_stride, const float *weight, float eps, void *h, long h_stride, void *q,
                                long q_stride, uint8_t *exps, long exps_stride, float *scale, void *stream)
{
    if (rows > 0 && !scale) return MICONV_ERR_NULL;
    miconv::quant::RowArgs a = {x, residual, weight, h, (uint8_t *)q, exps, scale, x_stride, residual_stride, h_stride,
                                q_stride, exps_stride, rows, 0, eps};
    return miconv::quant::run_rows(a, cols, dtype, static_cast<hipStream_t>(stream));
}

extern "C" int quant_rows_f8(long rows, long cols, int dtype, const void *x, long x_stride, void *q, long q_stride,
                             uint8_t *exps, long exps_stride, void *stream)
{
    miconv::quant::RowArgs a = {x, nullptr, nullptr, nullptr, (uint8_t *)q, exps, nullptr, x_stride, 0, 0, q_stride,
                                exps_stride, rows, 0, 0.0f};
    return miconv::quant::run_rows(a, cols, dtype, static_cast<hipStream_t>(stream));
}
