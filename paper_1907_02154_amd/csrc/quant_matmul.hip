// Matrix product of 8-bit integers with scales for each token and channel
// (quant_matmul_i8): y[m][n] = act(sa[m] sw[n] sum_k a[m][k] w[n][k] + bias[n] + res[m][n]).
//
// v_mfma_i32_16x16x64_i8: the channels are the rows of the matrix
// instruction and the tokens its columns, so that a lane's four sums are four
// consecutive channels of one token.
#include "quant.h"

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
};

// Four sums of token m, channels n .. n + 3, into y.
template <typename T>
__device__ __forceinline__ void finish4(const MatArgs &a, int m, int n, i32x4 sum, float sa)
{
    const int live = a.N - n;
    if (live <= 0) return;
    T *y = (T *)a.y + (long)m * a.ys + n;
    const T *res = a.res ? (const T *)a.res + (long)m * a.rs + n : nullptr;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < live) {
            float v = (float)sum[i] * sa * a.sw[n + i];
            if (a.bias) v += a.bias[n + i];
            if (res) v += load1(res + i);
            if (a.relu) v = v < 0.0f ? 0.0f : v;   // a NaN stays
            store1(y + i, v);
        }
}

// 16 bytes of a row from k on, zero past K.
__device__ __forceinline__ i32x4 chunk16(const int8_t *row, int k, int K)
{
    i32x4 v = {0, 0, 0, 0};
    if (k + 16 <= K) {
        memcpy(&v, row + k, 16);
    } else if (k < K) {
        uint32_t d[4] = {0, 0, 0, 0};
        for (int i = 0; i < K - k; ++i) d[i / 4] |= (uint32_t)(uint8_t)row[k + i] << (8 * (i % 4));
        v = i32x4{(int)d[0], (int)d[1], (int)d[2], (int)d[3]};
    }
    return v;
}

// 64 x 64 tile, 4 wavefronts of 32 x 32, 64 of the reduction at a time through
// registers and LDS: rows of any alignment.
template <typename T>
__global__ __launch_bounds__(256) void matmul_i8_any_kernel(MatArgs a)
{
    __shared__ i32x4 sa_[64][4], sw_[64][4];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int n0 = blockIdx.x * 64, m0 = blockIdx.y * 64;
    const int row = threadIdx.x / 4, c = threadIdx.x % 4;   // the chunk this thread stages of each operand
    const bool am = m0 + row < a.M, wn = n0 + row < a.N;
    const int8_t *ar = a.a + (long)(am ? m0 + row : 0) * a.as, *wr = a.w + (long)(wn ? n0 + row : 0) * a.ws;
    i32x4 acc[2][2] = {};
    for (int k0 = 0; k0 < a.K; k0 += 64) {
        const i32x4 va = chunk16(ar, k0 + c * 16, am ? a.K : 0), vw = chunk16(wr, k0 + c * 16, wn ? a.K : 0);
        __syncthreads();
        sa_[row][c ^ (row / 2 & 3)] = va;
        sw_[row][c ^ (row / 2 & 3)] = vw;
        __syncthreads();
        i32x4 fw[2], fa[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int rn = wave / 2 * 32 + i * 16 + lane % 16, rm = wave % 2 * 32 + i * 16 + lane % 16;
            fw[i] = sw_[rn][lane / 16 ^ (rn / 2 & 3)];
            fa[i] = sa_[rm][lane / 16 ^ (rm / 2 & 3)];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[i], fa[j], acc[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int m = m0 + wave % 2 * 32 + j * 16 + lane % 16;
        if (m >= a.M) continue;
        const float sa = a.sa[m];
#pragma unroll
        for (int i = 0; i < 2; ++i) finish4<T>(a, m, n0 + wave / 2 * 32 + i * 16 + lane / 16 * 4, acc[i][j], sa);
    }
}

template <typename T>
int launch_matmul(const MatArgs &a, hipStream_t st)
{
    launch_kernel(matmul_i8_any_kernel<T>, dim3((unsigned)ceil_div(a.N, 64), (unsigned)ceil_div(a.M, 64)), dim3(256), 0, st, a);
    return launched();
}

}  // namespace
}  // namespace quant
}  // namespace miconv

extern "C" long quant_matmul_workspace_bytes(long M, long N, long K)
{
    if (M < 0 || N < 1 || K < 1) return MICONV_ERR_SHAPE;
    if (M >= 1L << 31 || N >= 1L << 31 || K > 131071) return MICONV_ERR_TOO_LARGE;
    return 0;
}

extern "C" int quant_matmul_i8(long M, long N, long K, const int8_t *a, long a_stride, const float *a_scale,
                               const int8_t *w, long w_stride, const float *w_scale, const float *bias,
                               const void *residual, long residual_stride, int out_dtype, void *y, long y_stride,
                               int relu, void *ws, size_t ws_bytes, void *stream)
{
    using namespace miconv;
    const long need = quant_matmul_workspace_bytes(M, N, K);
    if (need < 0) return (int)need;
    const int b = quant::dtype_bytes(out_dtype);
    if (!b) return MICONV_ERR_UNSUPPORTED;
    if (a_stride < K || w_stride < K || y_stride < N || (residual && residual_stride < N)) return MICONV_ERR_SHAPE;
    if (M == 0) return MICONV_OK;
    if (!a || !a_scale || !w || !w_scale || !y) return MICONV_ERR_NULL;
    if (quant::misaligned(a_scale, 4) || quant::misaligned(w_scale, 4) || quant::misaligned(bias, 4) ||
        quant::misaligned(residual, b) || quant::misaligned(y, b))
        return MICONV_ERR_ALIGN;
    if (need && (!ws || ws_bytes < (size_t)need || quant::misaligned(ws, 256))) return MICONV_ERR_WORKSPACE;
    const quant::MatArgs args = {a, w, a_scale, w_scale, bias, residual, y, a_stride, w_stride, residual_stride,
                                 y_stride, (int)M, (int)N, (int)K, relu};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return out_dtype == quant::kF32 ? quant::launch_matmul<float>(args, st) : quant::launch_matmul<uint16_t>(args, st);
}
