// The pick of a token from each row of logits (sample_tokens).
//
// Nothing is sorted but a few candidates.  The row is read for its largest and
// smallest logit; then a histogram in LDS over evenly spaced logits finds the
// neighbourhood of a filter's end, whose few tokens are gathered, sorted by
// (logit, index) and cut off exactly; then the weights that are left are added in
// the vocabulary's order, unit by unit, and the draw looks into the one unit
// that it falls into.  Weights are whole numbers of 64 bits, so that neither the
// order of the additions nor the atomics of the histogram changes a result.
#include "../../include/misample.h"
#include "quant.h"

namespace miconv {
namespace {

using quant::kBF16;
using quant::kF32;
using quant::load1;
using quant::load8;
using quant::misaligned;

typedef unsigned long long u64;

constexpr float kNegInf = -__builtin_inff();
constexpr int kBins = 2048, kList = 4096;   // bins of a histogram; candidates that LDS holds
constexpr int kUnit = 512;                  // tokens that a wavefront takes together, 8 a lane

struct SampleArgs {
    const void *x;
    long stride;
    int vocab;
    const float *u, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    int32_t *token;
    float *logprob;
    int shift;        // weights are multiples of 2^-shift
    int units, runs;  // units of a row, and how many of them make one of the partial sums
};

// A logit's place in the order, larger for larger logits; -0 counts as 0.
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);
    return b ^ ((uint32_t)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t k)
{
    return __builtin_bit_cast(float, k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
// A token's place in the order of logit, then index: all are distinct.
__device__ __forceinline__ u64 place_of(float x, int i) { return (u64)key_of(x) << 32 | (uint32_t)~i; }

// 2^t for t <= 0, by the series of exp: |f ln 2| <= .35, the first term left out 6e-15.
__device__ __forceinline__ double power_of(double t, int shift)
{
    t = fmax(t, -1100.0);
    const double n = rint(t), f = t - n;
    double p = 4.44553827187081149760e-10;
    p = fma(p, f, 7.05491162080112332987e-9);
    p = fma(p, f, 1.01780860092396997275e-7);
    p = fma(p, f, 1.32154867901443094885e-6);
    p = fma(p, f, 1.52527338040598402800e-5);
    p = fma(p, f, 1.54035303933816099544e-4);
    p = fma(p, f, 1.33335581464284434234e-3);
    p = fma(p, f, 9.61812910762847716198e-3);
    p = fma(p, f, 5.55041086648215799532e-2);
    p = fma(p, f, 2.40226506959100712334e-1);
    p = fma(p, f, 6.93147180559945309417e-1);
    p = fma(p, f, 1.0);
    return ldexp(p, (int)n + shift);
}

struct Row {
    double top, factor;   // the largest logit; log2(e) / temperature
    int shift;
    // The weight over the largest, and as a whole number.
    __device__ __forceinline__ double share(float x) const { return power_of(((double)x - top) * factor, 0); }
    __device__ __forceinline__ u64 weight(float x) const
    {
        const double w = power_of(((double)x - top) * factor, shift) + 0x1p52;   // at most 2^51: the sum's low bits
        return __builtin_bit_cast(u64, w) & ((1ull << 52) - 1);
    }
};

// A lane's 8 logits of a unit; minus infinity past the row's end.
template <typename T>
__device__ __forceinline__ void unit_of(const T *x, int vocab, int unit, int lane, float (&v)[8])
{
    const int at = unit * kUnit + lane * 8;
    if (at + 8 <= vocab) {
        load8(x + at, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = at + i < vocab ? load1(x + at + i) : kNegInf;
    }
}

template <typename V, typename F>
__device__ __forceinline__ V wave_reduce(V v, F f)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v = f(v, (V)__shfl_xor(v, d));
    return v;
}

template <typename T, int NT>
struct Picker {
    static constexpr int WAVES = NT / 64;
    struct Shared {
        u64 list[kList];
        u64 bins[kBins];
        u64 part[WAVES], found;
        int count;
    };
    const SampleArgs &a;
    Shared &s;
    const T *x;
    int tid, lane, wave;
    Row row;
    float top, inv;   // bins: (top - x) * inv
    int last;

    __device__ Picker(const SampleArgs &args, Shared &sh, long r)
        : a(args), s(sh), x((const T *)args.x + r * args.stride), tid(threadIdx.x), lane(threadIdx.x % 64),
          wave(__builtin_amdgcn_readfirstlane(threadIdx.x / 64))
    {
    }

    // f(logit, index) of every token, and of some past the row's end as minus infinity.
    template <typename F>
    __device__ __forceinline__ void scan(F f)
    {
        constexpr int U = 2;
        for (int u0 = wave; u0 < a.units; u0 += U * WAVES) {
            float v[U][8];
#pragma unroll
            for (int n = 0; n < U; ++n) unit_of(x, a.vocab, u0 + n * WAVES, lane, v[n]);
#pragma unroll
            for (int n = 0; n < U; ++n)
                if (u0 + n * WAVES < a.units)
#pragma unroll
                    for (int i = 0; i < 8; ++i) f(v[n][i], (u0 + n * WAVES) * kUnit + lane * 8 + i);
        }
    }
    template <typename F>
    __device__ __forceinline__ u64 reduce(u64 v, F f)   // over the work-group, for every thread
    {
        v = wave_reduce(v, f);
        __syncthreads();
        if (lane == 0) s.part[wave] = v;
        __syncthreads();
        v = s.part[0];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) v = f(v, s.part[i]);
        return v;
    }
    __device__ __forceinline__ u64 sum(u64 v)
    {
        return reduce(v, [](u64 p, u64 q) { return p + q; });
    }
    // The sum of v over the threads before this one; *all: over every thread.
    __device__ __forceinline__ u64 before(u64 v, u64 *all)
    {
        u64 in = v;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const u64 o = __shfl_up(in, d);
            if (lane >= d) in += o;
        }
        __syncthreads();
        if (lane == 63) s.part[wave] = in;
        __syncthreads();
        u64 base = 0, total = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            if (i < wave) base += s.part[i];
            total += s.part[i];
        }
        *all = total;
        return base + in - v;
    }
    __device__ __forceinline__ int bin_of(float v) const { return (int)fminf((top - v) * inv, (float)(kBins - 1)); }

    __device__ __forceinline__ void clear_bins()
    {
        __syncthreads();
        for (int i = tid; i < kBins; i += NT) s.bins[i] = 0;
        __syncthreads();
    }
    // The bin in whose sums, added up from the first, `end(sum before, sum with it)` holds; *ahead: the sum before it.
    template <typename F>
    __device__ __forceinline__ int crossing(F end, u64 *ahead, u64 *with)
    {
        constexpr int PER = kBins / NT;
        __syncthreads();
        u64 own[PER], total = 0, all;
#pragma unroll
        for (int i = 0; i < PER; ++i) own[i] = s.bins[tid * PER + i], total += own[i];
        u64 b = before(total, &all);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (end(b, b + own[i])) s.found = (u64)(tid * PER + i), s.part[0] = b, s.part[WAVES - 1] = b + own[i];
            b += own[i];
        }
        __syncthreads();
        *ahead = s.part[0], *with = s.part[WAVES - 1];
        return (int)s.found;
    }
    // The places of the tokens for which f holds into the list; how many there are, also where that is more than it holds.
    template <typename F>
    __device__ __forceinline__ int gather(F f)
    {
        __syncthreads();
        if (tid == 0) s.count = 0;
        __syncthreads();
        scan([&](float v, int i) {
            if (f(v, i)) {
                const int at = atomicAdd(&s.count, 1);
                if (at < kList) s.list[at] = place_of(v, i);
            }
        });
        __syncthreads();
        return s.count;
    }
    // The first n of the list in order, the largest first.
    __device__ __forceinline__ void sort(int n)
    {
        int size = 2;
        while (size < n) size *= 2;
        for (int i = n + tid; i < size; i += NT) s.list[i] = 0;
        __syncthreads();
        for (int k = 2; k <= size; k *= 2)
            for (int j = k / 2; j > 0; j /= 2) {
                for (int t = tid; t < size / 2; t += NT) {
                    const int i = 2 * t - (t & (j - 1)), o = i + j;   // the t-th pair j apart
                    const u64 p = s.list[i], q = s.list[o];
                    if ((p < q) == ((i & k) == 0)) s.list[i] = q, s.list[o] = p;
                }
                __syncthreads();
            }
    }
    // Of the first n of the sorted list, how many have less than `most` before them, whose weights follow `ahead`; one at least.
    __device__ __forceinline__ int fit(int n, u64 ahead, double most)
    {
        int kept = 0;
        for (int i0 = 0; i0 < n; i0 += NT) {
            const int i = i0 + tid;
            u64 all;
            const u64 b = ahead + before(i < n ? row.weight(logit_of((uint32_t)(s.list[i] >> 32))) : 0, &all);
            kept += i < n && (double)b < most;
            ahead += all;
        }
        const int c = (int)sum((u64)kept);
        return c < 1 ? 1 : c;
    }
    // The place at which the order's tokens from `floor` up end that `end(before, with)` is given for: digits of 11 bits of
    // the places, the highest first, until what is left fits the list.  By(logit): what is added up.
    template <typename By, typename F>
    __device__ __forceinline__ u64 radix(u64 floor, By by, F end, bool count, u64 k, double most)
    {
        u64 prefix = 0, ahead = 0;
        for (int low = 53;; low -= 11) {   // places with the prefix's bits above low + 11
            const int at = low < 0 ? 0 : low;
            const u64 mask = low + 11 >= 64 ? 0 : ~0ull << (low + 11);
            clear_bins();
            scan([&](float v, int i) {
                const u64 p = place_of(v, i);
                if (p >= floor && (p & mask) == prefix)
                    atomicAdd(&s.bins[kBins - 1 - ((p >> at) & ((1ull << (low + 11 - at)) - 1))], by(v));
            });
            u64 b, w;
            const int bin = crossing([&](u64 p, u64 q) { return end(ahead + p, ahead + q); }, &b, &w);
            prefix |= (u64)(kBins - 1 - bin) << at, ahead += b;
            const u64 m2 = ~0ull << at;
            const int n = gather([&](float v, int i) {
                const u64 p = place_of(v, i);
                return p >= floor && (p & m2) == prefix;
            });
            if (n <= kList) {   // at the latest when every bit is fixed
                sort(n);
                const int c = count ? (int)(k - ahead) : fit(n, ahead, most);
                return s.list[max(min(c, n), 1) - 1];
            }
        }
    }

    __device__ void run(long r);
    __device__ void done(long r, int token, float logprob)
    {
        if (tid == 0) {
            a.token[r] = token;
            if (a.logprob) a.logprob[r] = logprob;
        }
    }
    __device__ __forceinline__ float logprob(float v, u64 total) const
    {
        return (float)(((double)v - row.top) * row.factor * 0.693147180559945309417 - log(ldexp((double)total, -row.shift)));
    }
};

template <typename T, int NT>
__device__ void Picker<T, NT>::run(long r)
{
    // the first token of the order, the smallest finite logit, and whether a logit is none
    u64 best = 0;
    float low = __builtin_inff();
    bool bad = false;
    scan([&](float v, int i) {
        const u64 p = place_of(v, i);
        best = p > best ? p : best;
        low = v > kNegInf && v < low ? v : low;
        bad |= !(v < __builtin_inff());
    });
    const auto larger = [](u64 p, u64 q) { return p > q ? p : q; };
    best = reduce(best, larger);
    // (largest bad, largest -low) together
    const u64 both = reduce((u64)bad << 32 | key_of(-low), larger);
    low = -logit_of((uint32_t)both);
    top = logit_of((uint32_t)(best >> 32));
    const int first = (int)~(uint32_t)best;
    if (both >> 32 || top == kNegInf) return done(r, -1, __builtin_nanf(""));
    const float t = a.temperature ? a.temperature[r] : 1.0f;
    if (!(t > 0.0f)) return done(r, first, 0.0f);
    row.top = top;
    row.factor = fmax(1.44269504088896340736 / (double)t, 1e-300);   // above 0, so that minus infinity stays below everything
    row.shift = a.shift;
    // Bins over what the row spans, or over what counts of it.
    const float span = fminf(top - low, 64.0f * fmaxf(t, 1.0f));
    inv = span > 0.0f ? fminf((float)kBins / span, 0x1p100f) : 0.0f;

    const int k = a.top_k ? a.top_k[r] : 0;
    const float p = a.top_p ? a.top_p[r] : 1.0f, m = a.min_p ? a.min_p[r] : 0.0f;
    const bool by_k = k > 0 && k < a.vocab, by_p = p < 1.0f, by_m = m > 0.0f;
    u64 cut = 0;        // places from here on are kept
    int n = 0;          // of the list, if it holds all that are kept
    if (by_k) {
        clear_bins();
        scan([&](float v, int) { atomicAdd((unsigned int *)&s.bins[bin_of(v)], 1u); });
        const auto end = [&](u64 b, u64 w) { return b < (u64)k && (u64)k <= w; };
        u64 ahead, with;
        const int bin = crossing(end, &ahead, &with);
        if (with <= (u64)kList) {
            n = gather([&](float v, int) { return bin_of(v) <= bin; });
            sort(n);
            n = k;
        } else {
            cut = radix(0, [](float) { return 1ull; }, end, true, (u64)k, 0.0);
        }
    }
    if (by_p && p > 0.0f && !n) {
        clear_bins();
        scan([&](float v, int i) {
            if (v > kNegInf && place_of(v, i) >= cut) atomicAdd(&s.bins[bin_of(v)], row.weight(v));
        });
        u64 total = 0;
        __syncthreads();
        for (int i = tid; i < kBins; i += NT) total += s.bins[i];
        total = sum(total);
        const double most = (double)p * (double)total;
        const auto end = [&](u64 b, u64 w) { return (double)b < most && most <= (double)w; };
        u64 ahead, with;
        const int bin = crossing(end, &ahead, &with);
        const int c = gather([&](float v, int i) { return bin_of(v) == bin && place_of(v, i) >= cut; });
        if (c <= kList) {
            sort(c);
            cut = s.list[fit(c, ahead, most) - 1];
        } else {
            cut = radix(cut, [&](float v) { return row.weight(v); }, end, false, 0, most);
        }
    } else if (by_p && n) {
        u64 total = 0;
        for (int i = tid; i < n; i += NT) total += row.weight(logit_of((uint32_t)(s.list[i] >> 32)));
        total = sum(total);
        n = p > 0.0f ? fit(n, 0, (double)p * (double)total) : 1;
    } else if (by_p) {
        cut = best;
    }
    const auto kept = [&](float v, int i) {
        const u64 q = place_of(v, i);
        return v > kNegInf && q >= cut && (!by_m || q == best || row.share(v) >= (double)m);
    };
    float u = a.u[r];
    u = u > 0.0f ? fminf(u, 0x1.fffffep-1f) : 0.0f;
    if (n) {   // everything is in the list: by index
        __syncthreads();
        const int held = n;
        int live = 0;
        for (int i = tid; i < held; i += NT) {
            const u64 q = s.list[i];
            const uint32_t key = (uint32_t)(q >> 32);
            const bool is = kept(logit_of(key), (int)~(uint32_t)q);
            live += is;
            s.list[i] = is ? (q & 0xFFFFFFFFull) << 32 | key : 0;   // the lowest index sorts first: places hold its complement
        }
        n = (int)sum((u64)live);
        sort(held);
        u64 total = 0;
        for (int i = tid; i < n; i += NT) total += row.weight(logit_of((uint32_t)s.list[i]));
        total = sum(total);
        const double target = (double)u * (double)total;
        u64 ahead = 0;
        for (int i0 = 0; i0 < n; i0 += NT) {
            const int i = i0 + tid;
            u64 all;
            const u64 w = i < n ? row.weight(logit_of((uint32_t)s.list[i])) : 0;
            const u64 b = ahead + before(w, &all);
            if (w && (double)b <= target && target < (double)(b + w)) {
                const u64 q = s.list[i];
                a.token[r] = (int)~(uint32_t)(q >> 32);
                if (a.logprob) a.logprob[r] = logprob(logit_of((uint32_t)q), total);
            }
            ahead += all;
        }
        return;
    }
    // Sums of runs of units, in the vocabulary's order.
    __syncthreads();
    const int parts = (a.units + a.runs - 1) / a.runs;
    for (int g = wave; g < parts; g += WAVES) {
        u64 w = 0;
        for (int un = g * a.runs; un < min((g + 1) * a.runs, a.units); ++un) {
            float v[8];
            unit_of(x, a.vocab, un, lane, v);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (kept(v[i], un * kUnit + lane * 8 + i)) w += row.weight(v[i]);
        }
        w = wave_reduce(w, [](u64 p, u64 q) { return p + q; });
        if (lane == 0) s.list[g] = w;
    }
    __syncthreads();
    u64 total = 0;
    for (int i = tid; i < parts; i += NT) total += s.list[i];
    total = sum(total);
    const double target = (double)u * (double)total;
    u64 ahead = 0;
    for (int i0 = 0; i0 < parts; i0 += NT) {
        const int i = i0 + tid;
        u64 all;
        const u64 w = i < parts ? s.list[i] : 0, b = ahead + before(w, &all);
        if (w && (double)b <= target && target < (double)(b + w)) s.found = (u64)i, s.bins[0] = b;
        ahead += all;
    }
    __syncthreads();
    if (wave != 0) return;
    const int g = (int)s.found;
    u64 b0 = s.bins[0];
    for (int un = g * a.runs; un < min((g + 1) * a.runs, a.units); ++un) {
        float v[8];
        u64 w[8], own = 0;
        unit_of(x, a.vocab, un, lane, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w[i] = kept(v[i], un * kUnit + lane * 8 + i) ? row.weight(v[i]) : 0;
            own += w[i];
        }
        u64 in = own;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const u64 o = __shfl_up(in, d);
            if (lane >= d) in += o;
        }
        u64 b = b0 + in - own;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (w[i] && (double)b <= target && target < (double)(b + w[i])) {
                a.token[r] = un * kUnit + lane * 8 + i;
                if (a.logprob) a.logprob[r] = logprob(v[i], total);
            }
            b += w[i];
        }
        b0 += __shfl(in, 63);
    }
}

template <typename T, int NT>
__global__ __launch_bounds__(NT) void sample_rows_kernel(SampleArgs a)
{
    __shared__ typename Picker<T, NT>::Shared s;
    Picker<T, NT>(a, s, blockIdx.x).run(blockIdx.x);
}

int check_sample(long rows, long vocab, int dtype)
{
    if (dtype != kF32 && dtype != kBF16) return MICONV_ERR_UNSUPPORTED;
    if (rows < 0 || vocab < 1) return MICONV_ERR_SHAPE;
    if (vocab > 1L << 25 || rows >= 1L << 22) return MICONV_ERR_TOO_LARGE;   // a grid holds fewer than 2^32 threads
    return MICONV_OK;
}

}  // namespace
}  // namespace miconv

extern "C" long sample_tokens_workspace_bytes(long rows, long vocab, int dtype)
{
    return miconv::check_sample(rows, vocab, dtype);
}

extern "C" int sample_tokens(long rows, long vocab, int dtype, const void *x, long stride, const float *u,
                             const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p,
                             int32_t *token, float *logprob, void *ws, size_t ws_bytes, void *stream)
{
    using namespace miconv;
    const int rc = check_sample(rows, vocab, dtype);
    if (rc != MICONV_OK) return rc;
    if (stride < vocab) return MICONV_ERR_SHAPE;
    if (rows == 0) return MICONV_OK;
    if (!x || !u || !token) return MICONV_ERR_NULL;
    if (misaligned(x, dtype == kF32 ? 4 : 2) || misaligned(u, 4) || misaligned(temperature, 4) || misaligned(top_k, 4) ||
        misaligned(top_p, 4) || misaligned(min_p, 4) || misaligned(token, 4) || misaligned(logprob, 4))
        return MICONV_ERR_ALIGN;
    (void)ws, (void)ws_bytes;
    int bits = 0;
    while (1L << bits < vocab) ++bits;
    SampleArgs a = {x, stride, (int)vocab, u, temperature, top_p, min_p, top_k, token, logprob,
                    62 - bits < 51 ? 62 - bits : 51, (int)((vocab + kUnit - 1) / kUnit), 0};
    a.runs = (a.units + kList - 1) / kList;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)rows);
    if (vocab <= 4096)
        launch_kernel(dtype == kF32 ? sample_rows_kernel<float, 256> : sample_rows_kernel<uint16_t, 256>, grid, dim3(256), 0, st, a);
    else
        launch_kernel(dtype == kF32 ? sample_rows_kernel<float, 1024> : sample_rows_kernel<uint16_t, 1024>, grid, dim3(1024), 0, st, a);
    return quant::launched();
}
