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

#include <type_traits>

namespace miconv {
namespace {

using quant::kBF16;
using quant::kF32;
using quant::load1;
using quant::misaligned;

typedef unsigned long long u64;

constexpr float kNegInf = -__builtin_inff();
constexpr int kList = 4096;                 // candidates that LDS holds, and partial sums of a row
constexpr int kDigit = 2048;                // values of a digit of the radix search
constexpr int kValueThreads = 1024;          // of a work-group, for bf16 rows of more than 4096
constexpr int kThreads = 512;                // for other rows of more than 4096
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
    int units, runs;  // units of a row, and how many of them, a power of two, make one of the partial sums
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

// Of a row: how a logit's weight follows from it.
//
// 2^t with t = (x - top) log2(e) / T is the power of two of t's whole part, the
// entry of a table (in LDS) for the next six bits, and the series of exp for the
// rest f: |f ln 2| <= .0055, the first term left out 4e-17.  Weights are this times
// 2^shift, and smaller than half a grain where t passes -(shift + 3).
constexpr int kTable = 64;
struct Row {
    double top, factor, least;   // the largest logit; log2(e) / temperature; the x - top from which on weights are 0
    const double *table;
    int shift;
    __device__ __forceinline__ double share(float x) const
    {
        constexpr double kRound = 0x1.8p52 / kTable;   // added, leaves multiples of 1 / kTable
        const double d = fmax((double)x - top, least);
        const double up = fma(d, factor, kRound);
        const double f = fma(d, factor, kRound - up);
        const int n = (int)(uint32_t)__builtin_bit_cast(u64, up);   // 64 t, rounded
        double p = 1.33335581464284434234e-3;
        p = fma(p, f, 9.61812910762847716198e-3);
        p = fma(p, f, 5.55041086648215799532e-2);
        p = fma(p, f, 2.40226506959100712334e-1);
        p = fma(p, f, 6.93147180559945309417e-1);
        p = fma(p, f, 1.0);
        const u64 w = __builtin_bit_cast(u64, p * table[n & (kTable - 1)]);
        return __builtin_bit_cast(double, w + ((u64)(uint32_t)((n >> 6) + shift) << 52));
    }
    static __device__ __forceinline__ u64 whole(double w)
    {
        return __builtin_bit_cast(u64, w + 0x1p52) & ((1ull << 52) - 1);   // at most 2^51: the sum's low bits
    }
    __device__ __forceinline__ u64 weight(float x) const { return whole(share(x)); }
};

// Sums over a wavefront's lanes up to each, by the data paths between lanes.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t from_lane(uint32_t v, uint32_t none = 0)
{
    return (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, CTRL, ROWS, 0xF, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 plus_lane(u64 v)
{
    return v + ((u64)from_lane<CTRL, ROWS>((uint32_t)(v >> 32)) << 32 | from_lane<CTRL, ROWS>((uint32_t)v));
}
__device__ __forceinline__ u64 wave_scan(u64 v)
{
    v = plus_lane<0x111, 0xF>(v);   // from 1, 2, 4 and 8 lanes before, within 16
    v = plus_lane<0x112, 0xF>(v);
    v = plus_lane<0x114, 0xF>(v);
    v = plus_lane<0x118, 0xF>(v);
    v = plus_lane<0x142, 0xA>(v);   // the last of 16 to the next 16, of 32 to the next 32
    return plus_lane<0x143, 0xC>(v);
}
__device__ __forceinline__ u64 last_lane(u64 v)
{
    return (u64)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), 63) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ __forceinline__ u64 wave_sum(u64 v) { return last_lane(wave_scan(v)); }
__device__ __forceinline__ uint32_t wave_sum(uint32_t v)
{
    v += from_lane<0x111, 0xF>(v);
    v += from_lane<0x112, 0xF>(v);
    v += from_lane<0x114, 0xF>(v);
    v += from_lane<0x118, 0xF>(v);
    v += from_lane<0x142, 0xA>(v);
    v += from_lane<0x143, 0xC>(v);
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    v = max(v, from_lane<0x111, 0xF>(v));
    v = max(v, from_lane<0x112, 0xF>(v));
    v = max(v, from_lane<0x114, 0xF>(v));
    v = max(v, from_lane<0x118, 0xF>(v));
    v = max(v, from_lane<0x142, 0xA>(v));
    v = max(v, from_lane<0x143, 0xC>(v));
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// A lane's 8 logits of a unit as they are held.  At a row's end a lane reads the
// last 8, of which those before its own count as minus infinity: no load depends
// on a branch, or each would be waited for.  (Rows of fewer than 8 are read one
// by one.)
typedef uint32_t words_at_2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t words_at_4 __attribute__((ext_vector_type(4), aligned(4)));
template <typename T, bool SHORT>
struct Held {
    typedef typename std::conditional<sizeof(T) == 2, words_at_2, words_at_4>::type words;
    words w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T *x, int vocab, int unit, int lane)
    {
        const int at = unit * kUnit + lane * 8;
        if constexpr (SHORT) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t b = __builtin_bit_cast(uint32_t, at + i < vocab ? load1(x + at + i) : kNegInf);
                if constexpr (sizeof(T) == 4) w[i / 4][i % 4] = b;
                else w[0][i / 2] = i % 2 ? (w[0][i / 2] & 0xFFFFu) | (b & 0xFFFF0000u) : b >> 16;
            }
        } else {
            const words *p = (const words *)(x + min(at, vocab - 8));
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = p[i];
        }
    }
    // The logits, and the index of the first.
    __device__ __forceinline__ int widen(float (&v)[8], int vocab, int unit, int units, int lane) const
    {
        const int at = unit * kUnit + lane * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t b = sizeof(T) == 4 ? w[i / 4 % (sizeof(T) / 2)][i % 4] : i % 2 ? w[0][i / 2] & 0xFFFF0000u : w[0][i / 2] << 16;
            v[i] = __builtin_bit_cast(float, b);
        }
        if (SHORT || unit < units - 1) return at;
        const int from = min(at, vocab - 8);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = from + i < at ? kNegInf : v[i];
        return from;
    }
};

// The first n of the list in order, the largest first.  (Up to a few wavefronts each thread counts what comes before its
// own: one round of reads against a barrier for each of log^2 steps.  Steps within 64 of longer lists in registers took
// 3 us off the 60 of fp32 rows of 64000 with top_p and added 0.4 to the 11 to 15 of rows with top_k: not kept.)
template <int NT>
__device__ __forceinline__ void sort_list(u64 *list, int n, int tid)
{
    if (n <= 256) {
        const u64 mine = tid < n ? list[tid] : 0;
        int rank = 0;
        if (tid / 64 * 64 < n)
#pragma unroll 4
            for (int i = 0; i < n; ++i) rank += list[i] > mine;
        __syncthreads();
        if (tid < n) list[rank] = mine;
        __syncthreads();
        return;
    }
    int size = 512;
    while (size < n) size *= 2;
    for (int i = n + tid; i < size; i += NT) list[i] = 0;
    __syncthreads();
    for (int k = 2; k <= size; k *= 2)
        for (int j = k / 2; j > 0; j /= 2) {
            for (int t = tid; t < size / 2; t += NT) {
                const int i = 2 * t - (t & (j - 1)), o = i + j;   // the t-th pair j apart
                const u64 p = list[i], q = list[o];
                if ((p < q) == ((i & k) == 0)) list[i] = q, list[o] = p;
            }
            __syncthreads();
        }
}

// A row's units: a wavefront takes runs of them, every NT / 64-th, three units in flight, the first of which may be
// on their way before they are worked on.
template <typename T, bool SHORT, int NT>
struct Units {
    static constexpr int U = 3, WAVES = NT / 64;
    Held<T, SHORT> h[U];
    int u, ahead;

    __device__ __forceinline__ int next(const SampleArgs &a, int unit) const
    {
        return (unit + 1) & (a.runs - 1) ? unit + 1 : unit + 1 + (WAVES - 1) * a.runs;
    }
    __device__ __forceinline__ void start(const SampleArgs &a, const T *x, int lane, int wave)
    {
        u = ahead = wave * a.runs;
#pragma unroll
        for (int n = 0; n < U; ++n) h[n].load(x, a.vocab, min(ahead, a.units - 1), lane), ahead = next(a, ahead);
    }
    // f(held, unit, last of a run)
    template <typename F>
    __device__ __forceinline__ void each(const SampleArgs &a, const T *x, int lane, F f)
    {
#pragma unroll 1
        while (u < a.units) {
            const Held<T, SHORT> now = h[0];
#pragma unroll
            for (int n = 0; n < U - 1; ++n) h[n] = h[n + 1];
            h[U - 1].load(x, a.vocab, min(ahead, a.units - 1), lane);
            ahead = next(a, ahead);
            f(now, u, ((u + 1) & (a.runs - 1)) == 0 || u == a.units - 1);
            u = next(a, u);
        }
    }
};

// For one wavefront: of up to 128 sums, two neighbours a lane, the one that a share u of all falls into, what comes
// before it, and the total.  (For more of them the work-group looks.)
constexpr int kPairs = 128;
struct Fall {
    int part;
    u64 before, total;
    double target;
};
__device__ __forceinline__ Fall fall_into(u64 w0, u64 w1, float u, int lane)
{
    const u64 in = wave_scan(w0 + w1), b0 = in - w0 - w1, b1 = in - w1;
    Fall f;
    f.total = last_lane(in);
    f.target = (double)u * (double)f.total;
    const bool hit0 = w0 && (double)b0 <= f.target && f.target < (double)b1;
    const bool hit1 = w1 && (double)b1 <= f.target && f.target < (double)in;
    const u64 hits = __ballot(hit0 || hit1);
    const int at = hits ? __builtin_ctzll(hits) : 0;
    f.part = 2 * at + __builtin_amdgcn_readlane((int)hit1, at);
    const u64 b = hit1 ? b1 : b0;
    f.before = (u64)(uint32_t)__builtin_amdgcn_readlane((int)(b >> 32), at) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)b, at);
    return f;
}
// The units of run g, for one wavefront, until f(held, unit) is true; the loads of up to 8 of them are in flight together.
template <typename T, bool SHORT, typename F>
__device__ __forceinline__ void each_of_run(const SampleArgs &a, const T *x, int lane, int g, F f)
{
    constexpr int U = 8;
    const int end = min((g + 1) * a.runs, a.units);
#pragma unroll 1
    for (int u0 = g * a.runs; u0 < end; u0 += U) {
        Held<T, SHORT> h[U];
#pragma unroll
        for (int n = 0; n < U; ++n)
            if (u0 + n < end) h[n].load(x, a.vocab, u0 + n, lane);
#pragma unroll 1
        for (int u = u0; u < min(u0 + U, end); ++u) {
            if (f(h[0], u)) return;
#pragma unroll
            for (int n = 0; n < U - 1; ++n) h[n] = h[n + 1];
        }
    }
}
__device__ __forceinline__ u64 from_any(u64 v, int lane)   // of one lane, the same for all
{
    return (u64)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}
// Whether top_p or min_p leave nothing but the first token.
__device__ __forceinline__ bool first_alone(float p, float m) { return (p < 1.0f && !(p > 0.0f)) || m > 1.0f; }
__device__ __forceinline__ float drawn(const SampleArgs &a, long r)   // u as it counts
{
    const float u = a.u[r];
    return u > 0.0f ? fminf(u, 0x1.fffffep-1f) : 0.0f;
}

template <typename T, int NT, bool SHORT>
struct Picker {
    static constexpr int WAVES = NT / 64, BINS = NT > 256 ? 8192 : kDigit;   // BINS: of logits, 32 bits each
    struct Shared {
        u64 list[kList], sums[NT > 256 ? kList : 8];
        union {
            uint32_t counts[BINS];
            u64 digits[kDigit];
        };
        double table[kTable];
        u64 part[2][WAVES], ahead, with;
        float guess[WAVES];
        int found, until, count;
    };
    const SampleArgs &a;
    Shared &s;
    const T *x;
    const int tid, lane, wave;
    Row row;
    float anchor, inv;   // bins: (anchor - x) * inv
    int turn = 0;        // the half of s.part that is free

    __device__ __forceinline__ Picker(const SampleArgs &args, Shared &sh, long r)
        : a(args), s(sh), x((const T *)args.x + r * args.stride), tid(threadIdx.x), lane(threadIdx.x % 64),
          wave(__builtin_amdgcn_readfirstlane(threadIdx.x / 64))
    {
    }

    // f(logits, first index, unit, last of a run) of every lane's 8 tokens of a unit, those past the row's end as minus
    // infinity.
    template <typename F>
    __device__ __forceinline__ void units(F f)
    {
        Units<T, SHORT, NT> all;
        all.start(a, x, lane, wave);
        all.each(a, x, lane, [&](const Held<T, SHORT> &h, int unit, bool last) {
            float v[8];
            const int at = h.widen(v, a.vocab, unit, a.units, lane);
            f(v, at, unit, last);
        });
    }
    // f(logit, index) of every token.
    template <typename F>
    __device__ __forceinline__ void scan(F f)
    {
        units([&](const float (&v)[8], int at, int, bool) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f(v[i], at + i);
        });
    }
    // The work-group's values of a wavefront each, for every thread; one barrier, since the halves take turns.
    __device__ __forceinline__ const u64 *share_out(u64 v)
    {
        u64 *p = s.part[turn];
        turn ^= 1;
        if (lane == 0) p[wave] = v;
        __syncthreads();
        return p;
    }
    __device__ __forceinline__ u64 sum(u64 v)
    {
        const u64 *p = share_out(wave_sum(v));
        u64 all = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) all += p[i];
        return all;
    }
    __device__ __forceinline__ uint32_t largest(uint32_t v)
    {
        const u64 *p = share_out(wave_max(v));
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) m = max(m, (uint32_t)p[i]);
        return m;
    }
    // The sum of v over the threads before this one; *all: over every thread.
    __device__ __forceinline__ u64 before(u64 v, u64 *all)
    {
        const u64 in = wave_scan(v);
        const u64 *p = share_out(last_lane(in));
        u64 base = 0, total = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            if (i < wave) base += p[i];
            total += p[i];
        }
        *all = total;
        return base + in - v;
    }
    template <int N = BINS>
    __device__ __forceinline__ int bin_of(float v) const { return (int)fminf(fmaxf((anchor - v) * inv, 0.0f), (float)(N - 1)); }

    template <typename V, int N>
    __device__ __forceinline__ void clear(V (&bins)[N])
    {
        for (int i = tid; i < N; i += NT) bins[i] = 0;
        __syncthreads();
    }
    // The bin in whose sums, added up from the first, `end(sum before, sum with it)` holds; these sums.
    template <int N, typename V, typename F>
    __device__ __forceinline__ int crossing(const V *bins, F end, u64 *ahead, u64 *with)
    {
        constexpr int PER = N / NT;
        u64 total = 0, all;
#pragma unroll
        for (int i = 0; i < PER; ++i) total += bins[tid * PER + i];
        u64 b = before(total, &all);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const u64 w = b + bins[tid * PER + i];
            if (end(b, w)) s.found = tid * PER + i, s.ahead = b, s.with = w;
            b = w;
        }
        __syncthreads();
        *ahead = s.ahead, *with = s.with;
        return s.found;
    }
    // Bins between which the weights of the counted tokens, each taken to lie in the middle of its bin, pass a share p of
    // theirs and `over` more, which come first: where they reach a 512th less, -1 if `over` does, and a 512th more.  (That
    // covers what the middles are off by, also where few logits are possible and lie many bins apart.)
    __device__ __forceinline__ void guess(float p, float over, int *from, int *to)
    {
        constexpr int PER = BINS / NT;
        const float step = -(float)row.factor / inv, first = (anchor - (float)row.top) * (float)row.factor;
        float in = 0.0f;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            in += (float)s.counts[tid * PER + i] * __builtin_amdgcn_exp2f(first + step * ((float)(tid * PER + i) + 0.5f));
        const float mine = in;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const float o = __shfl_up(in, d);
            if (lane >= d) in += o;
        }
        if (lane == 63) s.guess[wave] = in;
        if (tid == 0) s.found = -1, s.until = BINS - 1;
        __syncthreads();
        float b = in - mine + over, total = over;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            if (i < wave) b += s.guess[i];
            total += s.guess[i];
        }
        const float less = p * total * (511.0f / 512.0f), more = fminf(p * total * (513.0f / 512.0f), total * 0.99999f);
        if ((b < less && less <= b + mine) || (b < more && more <= b + mine))   // a thread's bins again
#pragma unroll 1
            for (int i = 0; i < PER; ++i) {
                const int n = tid * PER + i;
                const float w = (float)s.counts[n] * __builtin_amdgcn_exp2f(first + step * ((float)n + 0.5f));
                if (b < less && less <= b + w) s.found = n;
                if (b < more && more <= b + w) s.until = n;
                b += w;
            }
        __syncthreads();
        *from = s.found, *to = more <= over ? -1 : s.until;
    }
    // The places of the tokens for which f holds into the list; how many there are, also where that is more than it holds.
    template <typename F>
    __device__ __forceinline__ int gather(F f)
    {
        if (tid == 0) s.count = 0;
        __syncthreads();
        scan([&](float v, int i) {
            if (f(v, i)) put(v, i);
        });
        __syncthreads();
        return s.count;
    }
    __device__ __forceinline__ void put(float v, int i)
    {
        const int at = atomicAdd(&s.count, 1);
        if (at < kList) s.list[at] = place_of(v, i);
    }
    __device__ __forceinline__ void sort(int n) { sort_list<NT>(s.list, n, tid); }
    __device__ __forceinline__ float listed(int i) const { return logit_of((uint32_t)(s.list[i] >> 32)); }
    // Of the first n of the sorted list, how many have less than `most` before them, whose weights follow `ahead`; one at least.
    __device__ __forceinline__ int fit(int n, u64 ahead, double most)
    {
        u64 kept = 0;
        for (int i0 = 0; i0 < n; i0 += NT) {
            const int i = i0 + tid;
            u64 all;
            const u64 b = ahead + before(i < n ? row.weight(listed(i)) : 0, &all);
            kept += i < n && (double)b < most;
            ahead += all;
        }
        const int c = (int)sum(kept);
        return c < 1 ? 1 : c;
    }
    __device__ __forceinline__ u64 listed_sum(int n)
    {
        u64 w = 0;
        for (int i = tid; i < n; i += NT) w += row.weight(listed(i));
        return sum(w);
    }
    // The place at which the order's tokens from `floor` up end: digits of 11 bits of the places, the highest first, until
    // what is left fits the list.  By number (k of them) or by weight (less than `most` before the last).
    __device__ __forceinline__ u64 radix(u64 floor, bool count, u64 k, double most)
    {
        u64 prefix = 0, ahead = 0;
        for (int low = 53;; low -= 11) {   // places with the prefix's bits above low + 11
            const int at = low < 0 ? 0 : low;
            const u64 mask = low + 11 >= 64 ? 0 : ~0ull << (low + 11);
            __syncthreads();
            clear(s.digits);
            scan([&](float v, int i) {
                const u64 p = place_of(v, i);
                if (p >= floor && (p & mask) == prefix)
                    atomicAdd(&s.digits[kDigit - 1 - ((p >> at) & ((1ull << (low + 11 - at)) - 1))], count ? 1ull : row.weight(v));
            });
            __syncthreads();
            u64 b, w;
            const int bin = crossing<kDigit>(s.digits, [&](u64 p, u64 q) {
                return count ? ahead + p < k && k <= ahead + q : (double)(ahead + p) < most && most <= (double)(ahead + q);
            }, &b, &w);
            prefix |= (u64)(kDigit - 1 - bin) << at, ahead += b;
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

    __device__ __forceinline__ u64 search(long r, u64 floor, bool count, u64 k, double most);
    __device__ __forceinline__ void run(long r);
    // The row's units in registers, where they are few.
    static constexpr int HELD = SHORT || NT == 256 ? 1 : 8;
    Held<T, SHORT> kept_units[HELD];
    __device__ __forceinline__ bool fits() const { return a.units <= HELD * WAVES && a.runs == 1; }
    __device__ __forceinline__ void hold()
    {
#pragma unroll
        for (int n = 0; n < HELD; ++n) kept_units[n].load(x, a.vocab, min(wave + n * WAVES, a.units - 1), lane);
    }
    template <typename F>
    __device__ __forceinline__ void each_held(F f)
    {
#pragma unroll
        for (int n = 0; n < HELD; ++n) {
            const int unit = wave + n * WAVES;
            float v[8];
            const int at = kept_units[n].widen(v, a.vocab, min(unit, a.units - 1), a.units, lane);
            if (unit < a.units)
#pragma unroll
                for (int i = 0; i < 8; ++i) f(v[i], at + i);
        }
    }
    // What the first of each thread's tokens say: the order's first place, and how weights follow.  0 where the row is done
    // with: no token can be drawn, or the first is asked for.
    __device__ __forceinline__ u64 top_of(long r, float t, float most_v, int most_i, bool bad)
    {
        const uint32_t mine = key_of(most_v), top_key = largest(mine);
        const float top = logit_of(top_key);
        const int first = (int)~largest(mine == top_key ? ~(uint32_t)most_i : 0u);
        const bool none = __syncthreads_or(bad) || top == kNegInf;
        if (none || !(t > 0.0f)) {
            done(r, none ? -1 : first, none ? __builtin_nanf("") : 0.0f);
            return 0;
        }
        row.top = top;
        row.factor = fmax(1.44269504088896340736 / (double)t, 1e-300);
        row.least = -(a.shift + 3) / row.factor;
        row.table = s.table;
        row.shift = a.shift;
        return (u64)top_key << 32 | (uint32_t)~first;
    }
    // min_p as a logit: the smallest whose weight passes it.  As a rule it is one of the 64 around where the logarithm has it.
    // Near 0 logits lie closer than weights tell them apart, so that all of these may pass, or none: then it is looked for
    // among the others, 64 of them at a time.
    __device__ __forceinline__ float floor_of(float m, uint32_t top_key) const
    {
        if (!(m > 0.0f)) return kNegInf;
        const double want = ldexp((double)fminf(m, 1.0f), row.shift);
        const auto passing = [&](uint32_t key, uint32_t surely) {   // lanes whose key passes; one from `surely` on does
            return __ballot(key >= surely || row.share(logit_of(key)) >= want);
        };
        const uint32_t near = key_of((float)fmax(row.top + log2((double)fminf(m, 1.0f)) / row.factor, -3.4e38)), from = near - 32u;
        const u64 pass = passing(from + (uint32_t)lane, top_key);
        uint32_t lo = from - 1u, hi = from + (uint32_t)__builtin_ctzll(pass | 1ull << 63);   // does not pass, passes
        if (!pass) lo = from + 63u, hi = top_key;
        else if (pass & 1) lo = key_of(kNegInf);
        while (hi - lo > 1u && (!pass || pass & 1)) {
            const uint32_t step = (hi - lo + 63u) / 64u;
            const int at = __builtin_ctzll(passing(lo + ((uint32_t)lane + 1u) * step, hi));   // the last lane's passes
            hi = min(lo + ((uint32_t)at + 1u) * step, hi), lo += (uint32_t)at * step;
        }
        return fminf(logit_of(hi), logit_of(top_key));
    }
    // For few: k threads' largest logits are k tokens, so that nothing below the last of these counts.  The others into the
    // list; how many there are.
    __device__ __forceinline__ int candidates(int k, float most_v, bool held)
    {
        u64 ahead, with;
        anchor = (float)row.top;
        const float low = -logit_of(largest(most_v > kNegInf ? key_of(-most_v) : 0u));
        inv = anchor > low ? fminf((float)NT / (anchor - low), 0x1p100f) : 0.0f;
        s.counts[tid] = 0;
        __syncthreads();
        atomicAdd(&s.counts[bin_of<NT>(most_v)], 1u);
        __syncthreads();
        const int bin = crossing<NT>(s.counts, [&](u64 b, u64 w) { return b < (u64)k && (u64)k <= w; }, &ahead, &with);
        if (tid == 0) s.count = 0;
        __syncthreads();
        const auto take = [&](float v, int i) {
            if (bin_of<NT>(v) <= bin) put(v, i);
        };
        if (!held) scan(take);
        else if (bin_of<NT>(most_v) <= bin) each_held(take);
        __syncthreads();
        return s.count;
    }
    // The pick of row r among its first k tokens, if the candidates for them are 64 at most; else nothing is done.
    __device__ __forceinline__ bool few(long r, int k)
    {
        const float t = a.temperature ? a.temperature[r] : 1.0f, p = a.top_p ? a.top_p[r] : 1.0f, m = a.min_p ? a.min_p[r] : 0.0f;
        if (tid < kTable) s.table[tid] = exp2((double)tid / kTable);
        float most_v = kNegInf;
        int most_i = 0;
        bool bad = false;
        const auto look = [&](float v, int i) {
            if (v > most_v) most_v = v, most_i = i;
            bad |= !(v < __builtin_inff());
        };
        const bool held = fits();
        if (held) hold(), each_held(look);
        else scan(look);
        const u64 best = top_of(r, t, most_v, most_i, bad);
        if (!best) return true;
        const float floor_v = floor_of(m, (uint32_t)(best >> 32));
        const int n = candidates(k, most_v, held);
        if (n > 64) return false;
        if (wave == 0) finish_few(r, n, k, p, first_alone(p, m), floor_v);
        return true;
    }
    // The n <= 64 first tokens of the list, by one wavefront: ordered, cut off after k, at p (`one`: after the first) and
    // below floor_v, and drawn from.
    __device__ __forceinline__ void finish_few(long r, int n, int k, float p, bool one, float floor_v)
    {
        u64 q = lane < n ? s.list[lane] : 0;
        int rank = 0;
        for (int i = 0; i < n; ++i) rank += from_any(q, i) > q;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (lane < n) s.list[rank] = q;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        q = lane < n ? s.list[lane] : 0;
        const float v = logit_of((uint32_t)(q >> 32));
        n = min(n, k);
        u64 w = lane < n ? row.weight(v) : 0, in = wave_scan(w);
        if (one || p < 1.0f) {
            const double most = (double)p * (double)last_lane(in);
            if (lane > 0 && (one || (double)(in - w) >= most)) w = 0;
        }
        if (v < floor_v) w = 0;
        // the sum of what is kept with a lower index
        const uint32_t index = ~(uint32_t)q;
        u64 b = 0, total = 0;
        for (int i = 0; i < n; ++i) {
            const u64 o = from_any(w, i);
            b += (uint32_t)__builtin_amdgcn_readlane((int)index, i) < index ? o : 0;
            total += o;
        }
        const double target = (double)drawn(a, r) * (double)total;
        if (w && (double)b <= target && target < (double)(b + w)) {
            a.token[r] = (int)index;
            if (a.logprob) a.logprob[r] = logprob(v, total);
        }
    }
    __device__ __forceinline__ void done(long r, int token, float logprob)
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

// Apart, so that the rare search takes no registers from the rest.
template <typename T, int NT, bool SHORT>
__device__ __noinline__ u64 radix_search(SampleArgs a, typename Picker<T, NT, SHORT>::Shared *s, Row row, long r, u64 floor, bool count,
                                         u64 k, double most)
{
    Picker<T, NT, SHORT> p(a, *s, r);
    p.row = row;
    return p.radix(floor, count, k, most);
}

template <typename T, int NT, bool SHORT>
__device__ __forceinline__ u64 Picker<T, NT, SHORT>::search(long r, u64 floor, bool count, u64 k, double most)
{
    __syncthreads();
    const u64 cut = radix_search<T, NT, SHORT>(a, &s, row, r, floor, count, k, most);
    __syncthreads();
    return cut;
}

template <typename T, int NT, bool SHORT>
__device__ __forceinline__ void Picker<T, NT, SHORT>::run(long r)
{
    const float t = a.temperature ? a.temperature[r] : 1.0f;
    const int k = a.top_k ? a.top_k[r] : 0;
    const float p = a.top_p ? a.top_p[r] : 1.0f, m = a.min_p ? a.min_p[r] : 0.0f;
    const bool one = first_alone(p, m), by_k = k > 0 && k < a.vocab, by_p = p < 1.0f && !one;
    if (tid < kTable) s.table[tid] = exp2((double)tid / kTable);
    if (tid == 0) s.count = 0;

    // The first token of the order, and whether a logit is none.  For top_p alone the tokens are counted at once, in bins
    // below the largest logit of a first look; what lies above that, a few, goes to the list.
    const bool at_once = by_p && !by_k && t > 0.0f;
    inv = fminf((float)BINS / (32.0f * t), 0x1p100f);
    if (at_once) {
        Held<T, SHORT> h;
        float v[8], top = kNegInf;
        h.load(x, a.vocab, min(wave, a.units - 1), lane);
        h.widen(v, a.vocab, 0, 1 << 30, lane);   // of the row's last unit some twice
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, v[i]);
        clear(s.counts);
        anchor = logit_of(largest(key_of(top)));
    }
    float most_v = kNegInf;
    int most_i = 0;
    bool bad = false;
    // Rows of few units stay in registers for the search of the first few.
    const bool held = by_k && k <= NT / 4 && fits();
    if (held) {
        hold();
        each_held([&](float v, int i) {
            if (v > most_v) most_v = v, most_i = i;
            bad |= !(v < __builtin_inff());
        });
    } else units([&](const float (&v)[8], int at, int, bool) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (v[i] > most_v) most_v = v[i], most_i = at + i;
            bad |= !(v[i] < __builtin_inff());
        }
        if (at_once) {
            int bin[8];
            bool any = false;
#pragma unroll
            for (int i = 0; i < 8; ++i) bin[i] = bin_of(v[i]), any |= v[i] > anchor;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (v[i] > kNegInf && v[i] <= anchor) atomicAdd(&s.counts[bin[i]], 1u);
            if (any)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (v[i] > anchor) put(v[i], at + i);
        }
    });
    const u64 best = top_of(r, t, most_v, most_i, bad);
    if (!best) return;
    const float top = (float)row.top, floor_v = floor_of(m, (uint32_t)(best >> 32));
    u64 cut = one ? best : 0;   // places from here on are kept
    int n = 0;                  // of the list, if it holds all that are kept
    bool summed = false;        // whether the sums of the kept are there
    if (by_k) {
        if (k <= NT / 4) {
            n = candidates(k, most_v, held);
        } else {
            u64 ahead, with;
            anchor = top;
            inv = fminf((float)BINS / (64.0f * fmaxf(t, 1.0f)), 0x1p100f);
            clear(s.counts);
            scan([&](float v, int) { atomicAdd(&s.counts[bin_of(v)], 1u); });
            __syncthreads();
            const int bin = crossing<BINS>(s.counts, [&](u64 b, u64 w) { return b < (u64)k && (u64)k <= w; }, &ahead, &with);
            n = gather([&](float v, int) { return bin_of(v) <= bin; });
        }
        if (n <= 64) {
            if (wave == 0) finish_few(r, n, k, p, one, floor_v);
            return;
        }
        if (n <= kList) {
            sort(n);
            n = k;
        } else {
            n = 0;
            cut = max(cut, search(r, 0, true, (u64)k, 0.0));
        }
    }
    if (by_p && n) {
        n = fit(n, 0, (double)p * (double)listed_sum(n));
    } else if (n && one) {
        n = 1;
    } else if (by_p) {
        // The neighbourhood of the end, from the number of tokens in each bin alone; then the weights, once: the sums of
        // what lies above it, by units, and its tokens into the list.  Where the end turns out to lie elsewhere, or the
        // list does not hold them, it is searched for digit by digit.
        bool sure = true;
        if (!at_once) {
            anchor = top;
            inv = fminf((float)BINS / (32.0f * t), 0x1p100f);
            __syncthreads();
            clear(s.counts);
            scan([&](float v, int i) {
                if (v > kNegInf && place_of(v, i) >= cut) atomicAdd(&s.counts[bin_of(v)], 1u);
            });
            if (tid == 0) s.count = 0;
            __syncthreads();
        }
        const int above = s.count;
        sure = above <= kList;
        float over = 0.0f;   // of every thread the same: the list is short
        if (sure)
            for (int i0 = 0; i0 < above; i0 += 64)
                over += i0 + lane < above ? __builtin_amdgcn_exp2f((listed(i0 + lane) - top) * (float)row.factor) : 0.0f;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) over += __shfl_xor(over, d);
        int from, to;
        guess(p, over, &from, &to);
        // above hi: certainly kept; down to lo: the neighbourhood
        float hi = from < 2 ? __builtin_inff() : anchor - (float)(from - 1) / inv;
        float lo = anchor - (float)(to + 2) / inv;
        if (floor_v > lo) {   // min_p ends what is kept before: everything from there on
            if (floor_v > kNegInf && floor_v <= hi) lo = floor_v;
            else lo = hi = floor_v;
        }
        // what counts in full lies above `over_v`
        const bool no_list = lo == hi;
        const uint32_t below = key_of(hi) - 1u;   // -0 and 0 have one key
        const float over_v = no_list ? logit_of(below == 0x7FFFFFFFu ? below - 1u : below) : hi;
        __syncthreads();
        if (tid == 0) s.count = 0;
        clear(s.sums);
        u64 total = 0;
        const auto add_up = [&](auto partly) {   // partly: of the tokens from `cut` on
            u64 kept = 0;
            units([&](const float (&v)[8], int at, int unit, bool last) {
                bool any = false;
#pragma unroll
                for (int i = 0; i < 8; ++i) {   // no branch: the chains of eight weights run side by side
                    u64 w = row.weight(v[i]);
                    if (partly) w = place_of(v[i], at + i) < cut ? 0 : w;
                    total += w;
                    kept += v[i] > over_v ? w : 0;
                    any |= v[i] <= over_v && v[i] >= lo;
                }
                if (any)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (v[i] <= over_v && v[i] >= lo && (!partly || place_of(v[i], at + i) >= cut)) put(v[i], at + i);
                if (!last) return;
                kept = wave_sum(kept);
                if (lane == 0) s.sums[unit / a.runs] = kept;
                kept = 0;
            });
        };
        if (cut) add_up(std::true_type());
        else add_up(std::false_type());
        total = sum(total);
        u64 ahead = 0;
        const int parts = (a.units + a.runs - 1) / a.runs;
        for (int i = tid; i < parts; i += NT) ahead += s.sums[i];
        ahead = sum(ahead);
        const double most = (double)p * (double)total;
        const int c = s.count;
        const u64 near = listed_sum(min(c, kList));
        // behind a floor that the neighbourhood ends at, the end may also lie below
        const bool ends = most <= (double)(ahead + near) || (floor_v > kNegInf && lo == floor_v);
        if (sure && c <= kList && (double)ahead < most && ends) {
            sort(c);
            const int fits = c ? fit(c, ahead, most) : 0;
            const u64 last = fits ? s.list[fits - 1] : 0;
            for (int i = tid; i < fits; i += NT) atomicAdd(&s.sums[(int)(~(uint32_t)s.list[i]) / kUnit / a.runs], row.weight(listed(i)));
            if (fits) cut = last;
            else cut = max(cut, (u64)key_of(hi) << 32);
            summed = true;
        } else {
            cut = search(r, cut, false, 0, most);
        }
    }
    // The weight of a kept token, 0 of another.
    const auto kept = [&](float v, int i) {
        const u64 q = place_of(v, i);
        return v > kNegInf && q >= cut && v >= floor_v ? row.weight(v) : 0;
    };
    const float u = drawn(a, r);
    __syncthreads();
    if (n) {   // everything is in the list: by index
        const int held = n;
        u64 live = 0;
        for (int i = tid; i < held; i += NT) {
            const u64 q = s.list[i];
            const float v = logit_of((uint32_t)(q >> 32));
            const bool is = v > kNegInf && v >= floor_v;
            live += is;
            s.list[i] = is ? (q & 0xFFFFFFFFull) << 32 | (q >> 32) : 0;   // the lowest index sorts first: places hold its complement
        }
        n = (int)sum(live);
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
    const int parts = (a.units + a.runs - 1) / a.runs;
    if (!summed) {
        clear(s.sums);
        u64 w = 0;
        units([&](const float (&v)[8], int at, int unit, bool last) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w += kept(v[i], at + i);
            if (!last) return;
            w = wave_sum(w);
            if (lane == 0) s.sums[unit / a.runs] = w;
            w = 0;
        });
        __syncthreads();
    }
    int g;
    u64 b0, total = 0;
    double target;
    if (parts <= kPairs) {
        if (wave != 0) return;
        const Fall f = fall_into(2 * lane < parts ? s.sums[2 * lane] : 0, 2 * lane + 1 < parts ? s.sums[2 * lane + 1] : 0, u, lane);
        g = f.part, b0 = f.before, total = f.total, target = f.target;
    } else {
        for (int i = tid; i < parts; i += NT) total += s.sums[i];
        total = sum(total);
        target = (double)u * (double)total;
        u64 ahead = 0;
        for (int i0 = 0; i0 < parts; i0 += NT) {
            const int i = i0 + tid;
            u64 all;
            const u64 w = i < parts ? s.sums[i] : 0, b = ahead + before(w, &all);
            if (w && (double)b <= target && target < (double)(b + w)) s.found = i, s.ahead = b;
            ahead += all;
        }
        __syncthreads();
        if (wave != 0) return;
        g = s.found, b0 = s.ahead;
    }
    each_of_run<T, SHORT>(a, x, lane, g, [&](const Held<T, SHORT> &h, int un) {
        float v[8];
        u64 own = 0;
        const int at = h.widen(v, a.vocab, un, a.units, lane);
#pragma unroll
        for (int i = 0; i < 8; ++i) own += kept(v[i], at + i);
        const u64 in = wave_scan(own), with = b0 + last_lane(in);
        u64 b = b0 + in - own;
        b0 = with;
        if (!(target < (double)with)) return false;
        if ((double)b <= target && target < (double)(b + own)) {   // one lane: its tokens again
            int in_lane = 0;
            float hit = 0.0f;
#pragma unroll
            for (int i = 7; i >= 0; --i) {
                const u64 w = kept(v[i], at + i);
                own -= w;
                if (w && (double)(b + own) <= target && target < (double)(b + own + w)) in_lane = i, hit = v[i];
            }
            a.token[r] = at + in_lane;
            if (a.logprob) a.logprob[r] = logprob(hit, total);
        }
        return true;
    });
}

// A work-group a row: latencies and barriers in a row bind, not the row's bytes.
// One row of 32000 in fp32, top_k 50, top_p and min_p: 13 to 15 us on the device (its
// 128 KB by one compute unit are 3 of them); greedy 5.  Such a row stays in
// registers, 8 units of 8 tokens a lane, and a wavefront finishes up to 64
// candidates by itself: 18 us without both.  Up to 4096 tokens take 256
// threads, whose barriers are shorter, more of them 512: 256 rows in fp32 with
// top_p .9, 2000 tokens 14 against 17 us, 4096 17 either way, 16000 32 against 27,
// 32000 56 against 39.  However few rows there are each has one work-group: one of
// 128000 with top_p .9 takes 73 us, in bf16 (below) 47.
template <typename T, int NT, bool SHORT>
__global__ __launch_bounds__(NT) void sample_rows_kernel(SampleArgs a)
{
    __shared__ typename Picker<T, NT, SHORT>::Shared s;
    Picker<T, NT, SHORT>(a, s, blockIdx.x).run(blockIdx.x);
}

// bf16 rows hold few different values, so tokens are counted by value, with a
// counter for each of 2^-8 <= |x| < 2^7, and everything about the filters
// follows from counters and the values' weights: the value that they end at, and
// how many tokens of it, the lowest indexes, stay.  Each value's weight is
// computed once and looked up.  What lies outside that range, a few tokens as a
// rule, goes to a list; a row of which the list does not hold that is taken as
// rows of fp32 are.
//
// Bound by LDS: an addition to a counter for each token in the first pass and a
// look-up of 8 bytes in the second, at addresses that the logits choose.  256
// rows of 128000, top_p .9, a third of the tokens masked: 48 us, of which the
// first pass takes 17, the second 15, the steps between them 9, the draw 4 (65 MB
// from memory once: 13).  With 512 threads 67 where 1024 took 59.  Taken as rows
// of fp32 are, a weight evaluated for each token, such rows take 103; of 16000
// tokens 27 against 22, of 6000 the same 19.  Rows of which the first few tokens
// are asked for, or the first, are not counted: they go through the search that
// rows of fp32 use (top_k 50, 256 rows of 32000 18 against 28, of 128000 34
// against 51; that search with 512 threads 17 and 36).
// Tokens that are masked by the type's lowest value, not by minus infinity, lie
// outside the counters' range: of more than 2048 of them the first pass is lost, and
// the 256 rows take 163 us (without filters 121 where minus infinity takes 43; of
// 32000 72 against 27; with top_k 50 as long, 34).
// Measured beside it: the draw's run by one wavefront, unit by unit, 58 (11 of
// them that run); six units in flight in place of three no change; twice as many
// runs 1 us less in the draw and 2.5 more in the second pass.
//
// Slots, in the order of the logits: the list's x >= 2^7; the positive values;
// the list's |x| < 2^-8; the negative values; the list's x <= -2^7.
constexpr int kValues = 15 * 128, kMiddle = kValues + 1, kSlots = 2 * kValues + 3;
constexpr int kFirst = (127 - 8) << 7;   // bits of 2^-8
constexpr uint32_t kForbidden = 0xFF80;  // bits of minus infinity

// In LDS: positive values by magnitude with a place for what lies below and one for what lies above, the negative ones
// the same, the list's three slots.  The places of what has no counter stay 0.
constexpr int kSide = kValues + 2, kPlaces = 2 * kSide + 3;
constexpr int kTieBit = 56;
constexpr int kFew = 56;   // seven eighths of the candidates that one wavefront finishes

struct Values {
    uint32_t counts[kPlaces + 64];   // the last: of what has no counter, a lane's own
    u64 weights[kPlaces];      // of a token; of the list's slots the sum
    u64 list[kList / 2], sums[kList];
    uint32_t ties[kList];
    double table[kTable];
    u64 part[2][16], ahead[2];
    int found[2], count;
};

template <int NT>
struct ByValue {
    typedef uint16_t T;
    static constexpr int WAVES = NT / 64, PER = (kSlots + NT - 1) / NT;
    const SampleArgs &a;
    Values &s;
    const T *x;
    const int tid, lane, wave;
    Row row;
    double want = 0.0;   // the weight that min_p asks for
    int turn = 0, found_turn = 0;

    __device__ __forceinline__ ByValue(const SampleArgs &args, Values &sh, long r)
        : a(args), s(sh), x((const T *)args.x + r * args.stride), tid(threadIdx.x), lane(threadIdx.x % 64),
          wave(__builtin_amdgcn_readfirstlane(threadIdx.x / 64))
    {
    }
    // The slot of a value's 16 bits; kSlots for those without a counter.
    static __device__ __forceinline__ int slot_of(uint32_t b)
    {
        const int i = (int)(b & 0x7FFFu) - kFirst, j = b & 0x8000u ? i + 1 : -1 - i;
        return (unsigned)i < (unsigned)kValues ? kMiddle + j : kSlots;
    }
    // A slot's place in LDS.
    static __device__ __forceinline__ int place_in(int slot)
    {
        const int j = slot - kMiddle;
        return of_list(slot) ? 2 * kSide + (j > 0) - (j < 0) + 1 : j < 0 ? -j : kSide + j;
    }
    // Of two values' bits their places.
    typedef uint16_t two __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ two clamped(two v)
    {
        return __builtin_elementwise_min(__builtin_elementwise_max((two)(v & (two)0x7FFF), (two)(kFirst - 1)), (two)(kFirst + kValues));
    }
    static __device__ __forceinline__ two places_of(uint32_t b)
    {
        const two v = __builtin_bit_cast(two, b);
        return (v >> (two)15) * (two)kSide + (clamped(v) - (two)(kFirst - 1));
    }
    // The same for counting, `other` for values without a counter; *odd: whether there are such besides minus infinity.
    static __device__ __forceinline__ two counters_of(uint32_t b, int other, uint32_t *odd)
    {
        const two v = __builtin_bit_cast(two, b), m = clamped(v);
        const two in = m - (two)(kFirst - 1), place = (v >> (two)15) * (two)kSide + in;
        // 1 where the magnitude is below the first counter or above the last: in - 1 is kValues or 2^16 - 1 there
        const two out = __builtin_elementwise_min(__builtin_elementwise_max((two)(in - (two)1), (two)(kValues - 1)) - (two)(kValues - 1), (two)1);
        const two some = __builtin_elementwise_min((two)(v ^ (two)kForbidden), (two)1);
        *odd |= __builtin_bit_cast(uint32_t, (two)(out & some));
        return place + out * ((two)other - place);
    }
    static __device__ __forceinline__ float value_of(int slot)
    {
        return bf16_to_f32((uint16_t)(slot < kMiddle ? kMiddle - 1 - slot + kFirst : slot - kMiddle - 1 + kFirst + 0x8000));
    }
    static __device__ __forceinline__ bool of_list(int slot) { return slot == 0 || slot == kMiddle || slot == kSlots - 1; }
    static __device__ __forceinline__ int slot_of_listed(float v) { return v >= 1.0f ? 0 : v <= -1.0f ? kSlots - 1 : kMiddle; }
    __device__ __forceinline__ float listed(int i) const { return logit_of((uint32_t)(s.list[i] >> 32)); }

    // f(bits of 8 logits by twos, first index, unit, last of a run); `all` has been started.
    template <typename F>
    __device__ __forceinline__ void units(Units<T, false, NT> &all, F f)
    {
        all.each(a, x, lane, [&](const Held<T, false> &h, int unit, bool last) {
            uint32_t b[4] = {h.w[0][0], h.w[0][1], h.w[0][2], h.w[0][3]};
            int at = unit * kUnit + lane * 8;
            if (unit == a.units - 1) {   // those that the lane before has
                const int from = min(at, a.vocab - 8);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (from + 2 * i < at) b[i] = (b[i] & 0xFFFF0000u) | kForbidden;
                    if (from + 2 * i + 1 < at) b[i] = (b[i] & 0xFFFFu) | kForbidden << 16;
                }
                at = from;
            }
            f(b, at, unit, last);
        });
    }
    __device__ __forceinline__ const u64 *share_out(u64 v)
    {
        u64 *p = s.part[turn];
        turn ^= 1;
        if (lane == 0) p[wave] = v;
        __syncthreads();
        return p;
    }
    __device__ __forceinline__ u64 before(u64 v, u64 *all)   // as Picker's
    {
        const u64 in = wave_scan(v);
        const u64 *p = share_out(last_lane(in));
        u64 base = 0, total = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            if (i < wave) base += p[i];
            total += p[i];
        }
        *all = total;
        return base + in - v;
    }
    __device__ __forceinline__ u64 sum(u64 v)
    {
        const u64 *p = share_out(wave_sum(v));
        u64 all = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) all += p[i];
        return all;
    }
    // Where the order's tokens end: those of the slots before `slot` stay, and the first `tokens` of its own.
    struct End {
        int slot, tokens;
    };
    // The sum of a slot's weights as far as `end` goes; its list's tokens are sorted.
    __device__ __forceinline__ u64 sum_of(int slot, const End &end) const
    {
        if (slot > end.slot) return 0;
        if (!of_list(slot)) return (slot == end.slot ? (u64)end.tokens : (u64)s.counts[place_in(slot)]) * s.weights[place_in(slot)];
        if (slot < end.slot) return s.weights[place_in(slot)];
        u64 w = 0;
        for (int i = 0, at = first_of(slot); i < end.tokens; ++i) w += row.weight(listed(at + i));
        return w;
    }
    // The first of a slot's tokens in the sorted list.
    __device__ __forceinline__ int first_of(int slot) const
    {
        return (slot > 0 ? (int)s.counts[2 * kSide] : 0) + (slot > kMiddle ? (int)s.counts[2 * kSide + 1] : 0);
    }
    // The slot in whose sums of by(slot), added up from the first, end(before, with) holds, or kSlots; *ahead: the sum before.
    // known(sum of all) is called first.
    template <typename By, typename F, typename G>
    __device__ __forceinline__ int crossing(By by, F end, u64 *ahead, G known)
    {
        // Calls take turns at two results: of the one before, some thread may still be reading.
        const int at = found_turn;
        found_turn ^= 1;
        u64 own[PER], total = 0, all;
#pragma unroll
        for (int i = 0; i < PER; ++i) own[i] = tid * PER + i < kSlots ? by(tid * PER + i) : 0, total += own[i];
        if (tid == 0) s.found[at] = kSlots;
        u64 b = before(total, &all);
        known(all);
        if (total && end(b, b + total))   // one thread, if any
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                if (own[i] && end(b, b + own[i])) s.found[at] = tid * PER + i, s.ahead[at] = b;
                b += own[i];
            }
        __syncthreads();
        *ahead = s.ahead[at];
        return s.found[at];
    }
    // Whether the row could be taken so.
    __device__ __forceinline__ bool run(long r);
};

template <int NT>
__device__ __forceinline__ bool ByValue<NT>::run(long r)
{
    float t = a.temperature ? a.temperature[r] : 1.0f;
    int k = a.top_k ? a.top_k[r] : 0;
    float p = a.top_p ? a.top_p[r] : 1.0f, m = a.min_p ? a.min_p[r] : 0.0f;
    if (!(t > 0.0f) || m > 1.0f) k = 1, p = 1.0f, m = 0.0f;   // the first token
    if (!(t > 0.0f)) t = 1.0f;
    if (k < 1 || k > a.vocab) k = a.vocab;
    const int parts = (a.units + a.runs - 1) / a.runs;
    Units<T, false, NT> all;
    all.start(a, x, lane, wave);
    if (tid < kTable) s.table[tid] = exp2((double)tid / kTable);
    if (tid == 0) s.count = 0;
    for (int i = tid; i < kPlaces; i += NT) s.counts[i] = 0;
    // the values' weights are all written later
    if (tid < 7) s.weights[tid < 3 ? 2 * kSide + tid : tid == 3 ? 0 : tid == 4 ? kSide - 1 : tid == 5 ? kSide : 2 * kSide - 1] = 0;
    for (int i = tid; i < parts; i += NT) s.sums[i] = 0;
    __syncthreads();
    bool bad = false;
    units(all, [&](const uint32_t (&b)[4], int at, int, bool) {
        uint32_t place[4], odd = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) place[i] = __builtin_bit_cast(uint32_t, counters_of(b[i], kPlaces + lane, &odd));
#pragma unroll
        for (int i = 0; i < 8; ++i) atomicAdd(&s.counts[i % 2 ? place[i / 2] >> 16 : place[i / 2] & 0xFFFFu], 1u);
        if (odd)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t v = i % 2 ? b[i / 2] >> 16 : b[i / 2] & 0xFFFFu;
                if ((v & 0x7FFFu) - kFirst >= (unsigned)kValues && v != kForbidden) {
                    const int c = atomicAdd(&s.count, 1);
                    if (c < kList / 2) s.list[c] = place_of(bf16_to_f32((uint16_t)v), at + i);
                    bad |= (v & 0x7FFFu) >= 0x7F80u;
                }
            }
    });
    all.start(a, x, lane, wave);   // the second pass
    bad = __syncthreads_or(bad);
    const int outside = s.count;
    if (!bad && outside > kList / 2) return false;
    for (int i = tid; i < outside && !bad; i += NT) atomicAdd(&s.counts[place_in(slot_of_listed(listed(i)))], 1u);
    __syncthreads();
    const auto number = [&](int slot) { return (u64)s.counts[place_in(slot)]; };
    u64 ahead;
    uint32_t left = 0;   // slots from the first one that is taken on
#pragma unroll
    for (int i = PER - 1; i >= 0; --i)
        if (tid * PER + i < kSlots && !bad && number(tid * PER + i)) left = kSlots - (tid * PER + i);
    const u64 *lefts = share_out(wave_max(left));
#pragma unroll
    for (int i = 0; i < WAVES; ++i) left = max(left, (uint32_t)lefts[i]);
    const int best = kSlots - (int)left;
    if (best == kSlots) {
        if (tid == 0) {
            a.token[r] = -1;
            if (a.logprob) a.logprob[r] = __builtin_nanf("");
        }
        return true;
    }
    bool sorted = false;   // the list, where a slot of its own matters
    const auto of_sorted_list = [&](int slot) {
        if (of_list(slot) && !sorted) {
            __syncthreads();
            sort_list<NT>(s.list, outside, tid);
            sorted = true;
        }
        return of_list(slot);
    };
    const float top = of_sorted_list(best) ? listed(first_of(best)) : value_of(best);
    row.top = top;
    row.factor = fmax(1.44269504088896340736 / (double)t, 1e-300);
    row.least = -(a.shift + 3) / row.factor;
    row.table = s.table;
    row.shift = a.shift;
    want = m > 0.0f ? ldexp((double)m, a.shift) : 0.0;
    for (int i = tid; i < kSlots; i += NT)
        if (!of_list(i) && s.counts[place_in(i)]) s.weights[place_in(i)] = row.weight(value_of(i));   // of others none is read
    for (int i = tid; i < outside; i += NT) atomicAdd(&s.weights[place_in(slot_of_listed(listed(i)))], row.weight(listed(i)));
    __syncthreads();

    End end = {kSlots, 0};
    if (k < a.vocab) {
        const int slot = crossing(number, [&](u64 b, u64 w) { return b < (u64)k && (u64)k <= w; }, &ahead, [](u64) {});
        if (slot < kSlots) end = {slot, k - (int)ahead};   // else there are fewer
        of_sorted_list(slot);
    }
    if (p < 1.0f) {
        double most = 0.0;   // known once the sums are
        const auto within = [&](u64 b) { return (double)b < most; };
        const int slot = crossing([&](int slot) { return sum_of(slot, end); },
                                  [&](u64 b, u64 w) { return within(b) && most <= (double)w; }, &ahead,
                                  [&](u64 total) { most = (double)p * (double)total; });
        if (slot == kSlots) {   // p is not above 0
            end = {best, 1};
        } else {
            // how many have less than `most` before them
            int tokens = slot == end.slot ? end.tokens : (int)s.counts[place_in(slot)];
            if (of_sorted_list(slot)) {
                u64 b = ahead;
                int c = 0;
                for (int at = first_of(slot); c < tokens && within(b); ++c) b += row.weight(listed(at + c));
                tokens = c;
            } else {
                // the last has less than `most` before it, or is the first: about so many, and then exactly
                const u64 each = s.weights[place_in(slot)];
                int c = (int)fmin(fmax((most - (double)ahead) / (double)each, 1.0), (double)tokens);
                while (c < tokens && within(ahead + (u64)c * each)) ++c;
                while (c > 1 && !within(ahead + (u64)(c - 1) * each)) --c;
                tokens = c;
            }
            end = {slot, tokens};
        }
    }
    // What is kept: of the list's tokens and of the values' slots.  Of the last slot's tokens the first may be.
    const u64 cut = end.slot < kSlots && of_list(end.slot) ? s.list[first_of(end.slot) + end.tokens - 1] : 0;
    const auto kept = [&](float v, u64 place) {   // of the list's
        const int slot = slot_of_listed(v);
        return (slot < end.slot || (slot == end.slot && place >= cut)) && row.share(v) >= want;   // the first token's is a power of two
    };
    const bool some = end.slot < kSlots && !of_list(end.slot) && end.tokens < (int)s.counts[place_in(end.slot)];
    u64 tie = 0;   // the weight of a token of the last slot, where not all of them stay
    if (some && row.share(value_of(end.slot)) >= want) tie = s.weights[place_in(end.slot)];
    __syncthreads();
    if (m > 0.0f)
        for (int i = tid; i < kSlots; i += NT)
            if (i <= end.slot && !of_list(i) && row.share(value_of(i)) < want) s.weights[place_in(i)] = 0;
    if (some && tid == end.slot % NT) s.weights[place_in(end.slot)] = tie ? 1ull << kTieBit : 0;
    for (int i = tid; i < outside; i += NT) {
        const u64 q = s.list[i];
        if (kept(listed(i), q)) atomicAdd(&s.sums[(int)(~(uint32_t)q) / kUnit / a.runs], row.weight(listed(i)));
    }
    __syncthreads();

    // Sums of runs of units, in the vocabulary's order, and how many tokens of the last slot each holds: a lane's weights of a
    // run, at most 128, stay below 2^56, above which it counts these.  Values past the last slot are looked up in one place,
    // where lanes do not wait for one another, and which holds 0.
    const float from = end.slot == kSlots ? kNegInf : !of_list(end.slot) ? value_of(end.slot)
                       : end.slot == 0 ? __builtin_inff() : end.slot == kMiddle ? 0.0f : kNegInf;
    const auto looked_up = [&](const uint32_t (&b)[4], int i) {
        const uint32_t place = __builtin_bit_cast(uint32_t, places_of(b[i / 2]));
        const bool is = __builtin_bit_cast(float, i % 2 ? b[i / 2] & 0xFFFF0000u : b[i / 2] << 16) >= from;
        return s.weights[is ? i % 2 ? place >> 16 : place & 0xFFFFu : 0];
    };
    u64 w = 0;
    units(all, [&](const uint32_t (&b)[4], int, int unit, bool last) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w += looked_up(b, i);
        if (!last) return;
        const uint32_t ties = tie ? wave_sum((uint32_t)(w >> kTieBit)) : 0;
        w = wave_sum(w & ((1ull << kTieBit) - 1));
        if (lane == 0) {
            if (w) atomicAdd(&s.sums[unit / a.runs], w);   // beside the list's tokens
            s.ties[unit / a.runs] = ties;
        }
        w = 0;
    });
    __syncthreads();
    const float u = drawn(a, r);
    // of a part's tokens of the last slot, b of which come before them, those that stay
    const auto of_ties = [&](u64 c, u64 b) { return (b >= (u64)end.tokens ? 0 : min(c, (u64)end.tokens - b)) * tie; };
    // The run that the draw falls into, what comes before it, and the total.
    int g;
    u64 b0, t0, total = 0;
    if (parts <= kPairs) {
        if (wave == 0) {
            const int i = 2 * lane;
            u64 w0 = i < parts ? s.sums[i] : 0, w1 = i + 1 < parts ? s.sums[i + 1] : 0, c0 = 0, c1 = 0, before_c = 0;
            if (tie) {
                c0 = i < parts ? s.ties[i] : 0, c1 = i + 1 < parts ? s.ties[i + 1] : 0;
                before_c = wave_scan(c0 + c1) - c0 - c1;
                w0 += of_ties(c0, before_c), w1 += of_ties(c1, before_c + c0);
            }
            const Fall f = fall_into(w0, w1, u, lane);
            const u64 ties = from_any(f.part % 2 ? before_c + c0 : before_c, f.part / 2);
            if (lane == 0) s.found[0] = f.part, s.ahead[0] = f.before, s.ahead[1] = f.total, s.found[1] = (int)ties;
        }
        __syncthreads();
        g = s.found[0], b0 = s.ahead[0], total = s.ahead[1], t0 = (u64)s.found[1];
    } else {
        u64 all, seen = 0;
        if (tie)
            for (int i0 = 0; i0 < parts; i0 += NT) {
                const int i = i0 + tid;
                const u64 c = i < parts ? s.ties[i] : 0, b = seen + before(c, &all);
                if (i < parts) s.sums[i] += of_ties(c, b), s.ties[i] = (uint32_t)b;   // those before
                seen += all;
            }
        __syncthreads();
        for (int i = tid; i < parts; i += NT) total += s.sums[i];
        total = sum(total);
        const double target = (double)u * (double)total;
        ahead = 0;
        for (int i0 = 0; i0 < parts; i0 += NT) {
            const int i = i0 + tid;
            const u64 w = i < parts ? s.sums[i] : 0, b = ahead + before(w, &all);
            if (w && (double)b <= target && target < (double)(b + w)) s.found[0] = i, s.ahead[0] = b;
            ahead += all;
        }
        __syncthreads();
        g = s.found[0], b0 = s.ahead[0], t0 = s.ties[g];
    }
    const double target = (double)u * (double)total;
    // A unit of the run for each wavefront, its weights in registers.
    static_assert(WAVES >= 16, "a run has 16 units at most");
    const int un = g * a.runs + wave;
    const bool mine = wave < a.runs && un < a.units;
    Held<T, false> h;
    h.load(x, a.vocab, min(un, a.units - 1), lane);
    const uint32_t bits[4] = {h.w[0][0], h.w[0][1], h.w[0][2], h.w[0][3]};
    float v[8];
    u64 each[8], own = 0, tied = 0;
    const int at = h.widen(v, a.vocab, min(un, a.units - 1), a.units, lane);
    bool listed_one = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        each[i] = looked_up(bits, i);
        listed_one |= slot_of(__builtin_bit_cast(uint32_t, v[i]) >> 16) == kSlots && v[i] > kNegInf;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) each[i] = mine && v[i] > kNegInf ? each[i] : 0;   // not what the lane before has
    if (mine && listed_one)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (slot_of(__builtin_bit_cast(uint32_t, v[i]) >> 16) == kSlots && v[i] > kNegInf && kept(v[i], place_of(v[i], at + i)))
                each[i] = row.weight(v[i]);
    if (tie) {
#pragma unroll
        for (int i = 0; i < 8; ++i) tied += each[i] >> kTieBit;
        u64 all;
        u64 rank = t0 + before(tied, &all);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (each[i] >> kTieBit) each[i] = rank++ < (u64)end.tokens ? tie : 0;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) own += each[i];
    u64 all_of_run;
    b0 += before(own, &all_of_run);
    if (!((double)b0 <= target && target < (double)(b0 + own))) return true;
    int in_lane = 0;   // one lane
    float hit = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (each[i] && (double)b0 <= target && target < (double)(b0 + each[i])) in_lane = i, hit = v[i];
        b0 += each[i];
    }
    a.token[r] = at + in_lane;
    if (a.logprob)
        a.logprob[r] = (float)(((double)hit - row.top) * row.factor * 0.693147180559945309417 -
                               log(ldexp((double)total, -row.shift)));
    return true;
}

// Apart, as the rare search is.
template <int NT>
__device__ __noinline__ void row_by_bins(SampleArgs a, typename Picker<uint16_t, NT, false>::Shared *s, long r)
{
    Picker<uint16_t, NT, false>(a, *s, r).run(r);
}

template <int NT>
__global__ __launch_bounds__(NT) void sample_values_kernel(SampleArgs a)
{
    __shared__ union {
        Values values;
        typename Picker<uint16_t, NT, false>::Shared bins;
    } s;
    const int k = a.top_k ? a.top_k[blockIdx.x] : 0;
    const bool first = a.temperature && !(a.temperature[blockIdx.x] > 0.0f);   // the first token alone, which one pass finds
    if (first || (k > 0 && k <= kFew)) {
        if (Picker<uint16_t, NT, false>(a, s.bins, blockIdx.x).few(blockIdx.x, k)) return;
        __syncthreads();
    }
    if (!ByValue<NT>(a, s.values, blockIdx.x).run(blockIdx.x)) {
        __syncthreads();
        row_by_bins<NT>(a, &s.bins, blockIdx.x);
    }
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
    // Runs of up to 8 units, so that their sums are few, and 48 or more runs for the wavefronts.
    a.runs = 1;
    while ((a.units / (2 * a.runs) >= 48 && a.runs < 8) || (a.units + a.runs - 1) / a.runs > kList) a.runs *= 2;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)rows);
    const auto go = [&](auto of) {
        typedef decltype(of) T;
        if (vocab < 8) launch_kernel(sample_rows_kernel<T, 256, true>, grid, dim3(256), 0, st, a);
        else if (vocab <= 4096) launch_kernel(sample_rows_kernel<T, 256, false>, grid, dim3(256), 0, st, a);
        else if (sizeof(T) == 2) launch_kernel(sample_values_kernel<kValueThreads>, grid, dim3(kValueThreads), 0, st, a);
        else launch_kernel(sample_rows_kernel<float, kThreads, false>, grid, dim3(kThreads), 0, st, a);
    };
    if (dtype == kF32) go(float());
    else go(uint16_t());
    return quant::launched();
}
