// The next token of every row of logits: temperature, top-k, top-p, min-p and one given uniform number.
//
// With x_i = (z_i - max z) / T and w_i = e^x_i, tokens in the order (z descending, index ascending):
//   top-k keeps the first k; top-p of those each one whose predecessors' w add up to less than p times
//   the sum over top-k's; min-p those with w >= q; and the token is the first kept one, by index,
//   whose running sum of w exceeds u times the sum over the kept.
// The outcome is a whole number, so what decides it is held far finer than the logits: weights and
// sums in fp64 (an exponential of 16 operations, off by 4e-14), histograms in 64-bit fixed point, in
// orders that depend on the sizes alone.
//
// k_sample_stats reads the rows once: the maximum of every 64 vectors (a block), and where it may be asked
// for the sum of the weights of every 256 (a span), relative to their own maximum.  The other kernels
// find from these which blocks can hold a kept token and read only them:
//   no filter     the span that holds the token, then its block
//   min-p         the blocks that reach m + T ln q: their sums, then one block
//   top-k         the k-th largest span's or block's maximum bounds the last kept logit from below: the
//                 tokens above, hardly more than k, are sorted in LDS
//   top-p         a weight of (1 - p) / vocab of the whole bounds it: tokens of up to 128 blocks, if they are
//                 no more than 1024, are sorted; others are located first, by fp32 weights summed in
//                 1024 bins of equal width whose error is bounded, so that the tokens of a bin or two are
//                 sorted and all above them are summed (bound by the issue of instructions on one CU: for
//                 151936 bf16 tokens 20 us to locate, 40 to sum, 25 for the rest)
//   else          (large top-k, many ties) the border is found by 10-bit digits of the keys
// k_sample_plain does the rows of a call without filters, a wave each with no barrier to wait at; k_sample_pick
// all rows of other calls, a workgroup each of 8 waves.  Its steps are short and wait for one another: 512
// threads, whose registers hold them, took 20 us for one row of 151936 with top-20, 1024 took 26 (their
// 128 registers spill), and a wave for the rows with few tokens before a workgroup for the others 25.
#include "common.h"
#include "sample.h"
#include "wave.h"

#include <cfloat>
#include <type_traits>

namespace sparrow {
namespace {

constexpr int kStatThreads = 256;
constexpr int kStatWaves = kStatThreads / 64;
constexpr int kStatBlocks = 2048;  // workgroups that keep the device full
constexpr int kBlockVecs = 64;  // a wave's load
constexpr int kSpanBlocks = 4;
constexpr int kSpanVecs = kBlockVecs * kSpanBlocks;
constexpr int kPickThreads = 512;
constexpr int kPickWaves = kPickThreads / 64;
constexpr int kSampleSort = 1024;  // tokens that a workgroup sorts
// Blocks of which the number of tokens is seen by collecting them.  (151936 fp32 logits, top-p of 0.9, one row, with
// none, 128 and 512: of a deviation of 7 36.5, 36.5 and 52.3 us, of 14 17.8, 15.3 and 15.3, of 40 15.3, 12.3 and 12.2.)
constexpr int kFewBlocks = 128;
// Spans whose maxima take 5 registers, not 9.  (One row with top-20, 149 spans: with 9 registers 15.1 us, with 5 14.2,
// with the 3 that these would need 13.7; 256 spans: with 9 14.6, with 5 13.9.)
constexpr int kFewSpans = 320;
constexpr int kDigitBits = 10;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kMaxSpans = (kSampleMaxVocab / 4 + 1 + kSpanVecs - 1) / kSpanVecs;
constexpr int kMaxBlocks = kMaxSpans * kSpanBlocks;
constexpr int kSampleGrid = 1 << 20;  // workgroups at most
static_assert(kSampleSort == 2 * kPickThreads && kDigits == 2 * kPickThreads, "two per thread");
constexpr double kLog2e = 1.44269504088896340736;

template <bool kBf16> constexpr int kElems = kBf16 ? 8 : 4;  // of a 16-byte vector

// A row as 16-byte vectors from the boundary at or before its start; elements outside are masked.
template <bool kBf16>
struct Row {
    const char *base;  // of vector 0
    int off;           // its elements before the row
    int vocab;

    __device__ __forceinline__ Row(const SampleArgs &a, int64_t row)
    {
        constexpr int kSize = kBf16 ? 2 : 4;
        const char *p = static_cast<const char *>(a.logits) + row * a.row_stride * kSize;
        const int mis = (int)(reinterpret_cast<uintptr_t>(p) & 15u);
        base = p - mis;
        off = mis / kSize;
        vocab = a.vocab;
    }
    __device__ __forceinline__ int vecs() const
    {
        return (vocab + off + kElems<kBf16> - 1) / kElems<kBf16>;
    }
    __device__ __forceinline__ int index(int v, int e) const { return v * kElems<kBf16> + e - off; }
    // vector v, nothing past the row's ends being read (-inf there)
    __device__ __forceinline__ u32x4_t load(int v) const
    {
        const int i = index(v, 0);
        if (i >= 0 && i + kElems<kBf16> <= vocab)
            return ld16(base + (int64_t)v * 16);
        constexpr uint32_t kNone = kBf16 ? 0xff80ff80u : 0xff800000u;
        u32x4_t x = {kNone, kNone, kNone, kNone};
#pragma unroll
        for (int e = 0; e < kElems<kBf16>; ++e)
            if (i + e >= 0 && i + e < vocab) {
                if (kBf16) {
                    const uint32_t b = *reinterpret_cast<const uint16_t *>(base + (int64_t)v * 16 + 2 * e);
                    x[e >> 1] = e & 1 ? (x[e >> 1] & 0xffffu) | b << 16 : (x[e >> 1] & 0xffff0000u) | b;
                } else {
                    x[e & 3] = *reinterpret_cast<const uint32_t *>(base + (int64_t)v * 16 + 4 * e);
                }
            }
        return x;
    }
    // whether vectors [v, v + n) lie inside the row
    __device__ __forceinline__ bool inside(int v, int n) const
    {
        return index(v, 0) >= 0 && index(v + n, 0) <= vocab;
    }
    __device__ __forceinline__ u32x4_t load_inside(int v) const { return ld16(base + (int64_t)v * 16); }
    // Block b's vectors by the wave's lanes, in two steps so that several blocks' loads are under way at once:
    // one load without a branch, of the nearest vector that is inside the row, and what the two blocks
    // at the row's ends take beside it.  (A row of no whole vector: all in the second step.)
    __device__ __forceinline__ u32x4_t block_begin(int b) const
    {
        constexpr int kE = kElems<kBf16>;
        const int lo = off ? 1 : 0, hi = (vocab + off) / kE - 1;  // whole vectors
        if (hi < lo)
            return (u32x4_t){0u, 0u, 0u, 0u};
        return load_inside(min(max(b * kBlockVecs + (int)(threadIdx.x & 63), lo), hi));
    }
    __device__ __forceinline__ u32x4_t block_end(int b, u32x4_t x) const
    {
        if (!inside(b * kBlockVecs, kBlockVecs)) {
            x = load(min(b * kBlockVecs + (int)(threadIdx.x & 63), vecs()));  // (vecs(): nothing)
            asm volatile("" : "+v"(x));  // (the wait stays here)
        }
        return x;
    }
    // its logits: NaN counts as masked
    __device__ static __forceinline__ void unpack(u32x4_t v, float (&z)[kElems<kBf16>])
    {
#pragma unroll
        for (int e = 0; e < kElems<kBf16>; ++e) {
            const float f = kBf16 ? (e & 1 ? bf16_hi(v[(e >> 1) & 3]) : bf16_lo(v[(e >> 1) & 3]))
                            : __uint_as_float(v[e & 3]);
            // (the median with a NaN is the least of the others, with a signalling one the last: least last; the
            // builtin becomes two instructions)
            asm("v_med3_f32 %0, %1, %2, %3" : "=v"(z[e]) : "v"(f), "v"(INFINITY), "v"(-INFINITY));
        }
    }
    // its logits clamped to [low, high], NaN counting as low
    __device__ static __forceinline__ void unpack_clamped(u32x4_t v, float low, float high,
                                                          float (&z)[kElems<kBf16>])
    {
#pragma unroll
        for (int e = 0; e < kElems<kBf16>; ++e) {
            const float f = kBf16 ? (e & 1 ? bf16_hi(v[(e >> 1) & 3]) : bf16_lo(v[(e >> 1) & 3]))
                            : __uint_as_float(v[e & 3]);
            asm("v_med3_f32 %0, %1, %2, %3" : "=v"(z[e]) : "v"(f), "v"(high), "v"(low));
        }
    }
    // and +inf as the largest number, -0 as 0
    __device__ static __forceinline__ void unpack_whole(u32x4_t v, float (&z)[kElems<kBf16>])
    {
        unpack(v, z);
#pragma unroll
        for (int e = 0; e < kElems<kBf16>; ++e)
            z[e] = fminf(z[e], FLT_MAX) + 0.f;
    }
};

// 2^(d c), for d c in [-1020, 0]: the nearest whole power, which an addition of 1.5 2^52 leaves in the sum's
// low bits, and for the rest f, at most 1/2 either way, 1 + f q(f) with the q of degree 8 that agrees with
// (2^f - 1) / f in the 9 Chebyshev points of [-1/2, 1/2]: off by 4e-14, and exact at 0.
__device__ __forceinline__ double exp2_fast(double d, double c)
{
    constexpr double kMagic = 6755399441055744.;
    const double s = fma(d, c, kMagic), f = fma(d, c, kMagic - s);
    double p = fma(1.0203121063391729e-07, f, 1.3255224878668817e-06);
    p = fma(p, f, 1.525268684626772e-05);
    p = fma(p, f, 0.00015403455852453838);
    p = fma(p, f, 0.0013333558179043112);
    p = fma(p, f, 0.009618129159402558);
    p = fma(p, f, 0.055504108664760424);
    p = fma(p, f, 0.2402265069581299);
    p = fma(p, f, 0.6931471805599453);
    p = fma(p, f, 1.);
    // (in one instruction of 32 bits; the compiler makes five of 64 of it)
    u32x2_t b = __builtin_bit_cast(u32x2_t, p);
    asm("v_lshl_add_u32 %0, %1, 20, %2"
        : "=v"(b[1])
        : "v"(__builtin_bit_cast(u32x2_t, s)[0]), "v"(b[1]));
    return __builtin_bit_cast(double, b);
}

// 2^(d c) for any d <= 0, c >= 0: 0 below 2^-1000, and for a product that is no number.
__device__ __forceinline__ double exp2_64(double d, double c)
{
    const double t = d * c;
    const bool some = t >= -1000.;
    const double w = exp2_fast(some ? d : 0., some ? c : 0.);
    return some ? w : 0.;
}

// w of a logit relative to the maximum m, with c = log2(e) / T.
__device__ __forceinline__ double weight_of(float z, double m, double c)
{
    return exp2_64((double)z - m, c);
}

__device__ __forceinline__ uint32_t key_of(float z)
{
    const uint32_t b = __float_as_uint(z);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}

__device__ __forceinline__ float logit_of(uint32_t key)
{
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

// One DPP move of a double; lanes without a source (or in a masked row) get 0.
template <int kCtrl, int kRowMask>
__device__ __forceinline__ double dpp_move_64(double x)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = dpp_move<kCtrl, kRowMask>((uint32_t)b, 0u);
    const uint32_t hi = dpp_move<kCtrl, kRowMask>((uint32_t)(b >> 32), 0u);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// Inclusive sums over the wave's lanes in their order.
__device__ __forceinline__ double wave_scan_64(double x)
{
    x += dpp_move_64<kDppRowShr1, 0xf>(x);
    x += dpp_move_64<kDppRowShr2, 0xf>(x);
    x += dpp_move_64<kDppRowShr4, 0xf>(x);
    x += dpp_move_64<kDppRowShr8, 0xf>(x);
    x += dpp_move_64<kDppRowBcast15, 0xa>(x);
    x += dpp_move_64<kDppRowBcast31, 0xc>(x);
    return x;
}

__device__ __forceinline__ double lane_64(double x, int lane)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)b, lane);
    const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

__device__ __forceinline__ double wave_sum_64(double x) { return lane_64(wave_scan_64(x), 63); }

// The sum over the wave, in lane 63: within rows of 16 by exchanges that every lane takes part in, which need no
// zero for the others.
__device__ __forceinline__ double wave_total_64(double x)
{
    constexpr int kSwap1 = 0xb1, kSwap2 = 0x4e, kHalfMirror = 0x141, kMirror = 0x140;
    auto add = [](double v, auto ctrl) __attribute__((always_inline)) {
        const u32x2_t b = __builtin_bit_cast(u32x2_t, v);
        const u32x2_t o = {
            (uint32_t)__builtin_amdgcn_mov_dpp((int)b[0], decltype(ctrl)::value, 0xf, 0xf, true),
            (uint32_t)__builtin_amdgcn_mov_dpp((int)b[1], decltype(ctrl)::value, 0xf, 0xf, true)};
        return v + __builtin_bit_cast(double, o);
    };
    x = add(x, std::integral_constant<int, kSwap1>());
    x = add(x, std::integral_constant<int, kSwap2>());
    x = add(x, std::integral_constant<int, kHalfMirror>());
    x = add(x, std::integral_constant<int, kMirror>());
    x += dpp_move_64<kDppRowBcast15, 0xa>(x);
    x += dpp_move_64<kDppRowBcast31, 0xc>(x);
    return x;
}

// A row's settings; off is k = 0, p = 1, q = 0.
struct Filters {
    double c;  // log2(e) / T
    double t;
    int k;
    float p, q;
    bool greedy;

    __device__ __forceinline__ Filters(const SampleArgs &a, int64_t row)
    {
        const float temp = a.temperature ? a.temperature[row] : 1.f;
        t = temp;
        c = kLog2e / t;
        k = a.top_k ? a.top_k[row] : 0;
        k = k > 0 && k < a.vocab ? k : 0;
        p = a.top_p ? a.top_p[row] : 1.f;
        p = p < 1.f ? p : 1.f;  // (NaN: off)
        q = a.min_p ? a.min_p[row] : 0.f;
        q = q > 0.f ? fminf(q, 1.f) : 0.f;
        greedy = !(temp > 0.f) || k == 1 || !(p > 0.f);
    }
    __device__ __forceinline__ bool sums() const { return !greedy && k == 0; }
    __device__ __forceinline__ bool filtered() const { return !greedy && (k || p < 1.f || q > 0.f); }
};

struct Stats {
    double *sums;  // [rows][spans] weights of a span relative to its maximum
    float *maxima; // [rows][spans][kSpanBlocks]
    int spans;     // of a row, at most
};

// max without the canonical forms that the compiler makes of numbers which might be signalling NaNs (med3
// has left none).
__device__ __forceinline__ float max3(float x, float y, float z)
{
    float d;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(x), "v"(y), "v"(z));
    return d;
}

// max of two numbers, as max3 above.
__device__ __forceinline__ float max2(float x, float y)
{
    float d;
    asm("v_max_f32 %0, %1, %2" : "=v"(d) : "v"(x), "v"(y));
    return d;
}

// The maxima of four values over the wave, in rows of 16 lanes: of x[0], x[2], x[1] and x[3].  Swaps of halves, then
// of rows, bring two values into one register, whose parts are reduced together.  (A swap reads what an instruction
// wrote two states ago at the latest; the compiler does not see those inside asm.)
__device__ __forceinline__ float wave_max4(const float (&x)[4])
{
    auto halves = [](float a, float b) __attribute__((always_inline)) {
        asm("s_nop 1" : "+v"(a), "+v"(b));
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
        return max2(__uint_as_float(r[0]), __uint_as_float(r[1]));
    };
    float a = halves(x[0], x[1]), b = halves(x[2], x[3]);
    asm("s_nop 1" : "+v"(a), "+v"(b));
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    float top = max2(__uint_as_float(r[0]), __uint_as_float(r[1]));
    asm("s_nop 1\n v_max_f32_dpp %0, %0, %0 row_ror:8 row_mask:0xf bank_mask:0xf\n "
        "s_nop 1\n v_max_f32_dpp %0, %0, %0 row_ror:4 row_mask:0xf bank_mask:0xf\n "
        "s_nop 1\n v_max_f32_dpp %0, %0, %0 row_ror:2 row_mask:0xf bank_mask:0xf\n "
        "s_nop 1\n v_max_f32_dpp %0, %0, %0 row_ror:1 row_mask:0xf bank_mask:0xf"
        : "+v"(top));
    return top;
}

// The waves of a row's workgroups (blockIdx.y) take its spans in turn, the next one's loads under way.
// Bound by arithmetic where sums are wanted (24 vector instructions a logit, 17 of them for its weight: 256 fp32
// rows of 151936 in 38 us, 4.1 TB/s), else by memory.
template <bool kBf16>
__global__ __launch_bounds__(kStatThreads) void k_sample_stats(SampleArgs a, Stats st)
{
    constexpr int kE = kElems<kBf16>;
    const int lane = threadIdx.x & 63;
    const int first = blockIdx.x * kStatWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int step = gridDim.x * kStatWaves;
    if (first >= st.spans)
        return;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const Row<kBf16> r(a, row);
        const Filters f(a, row);
        const bool sums = f.sums();
        const int vecs = r.vecs();
        u32x4_t v[kSpanBlocks];
        auto load = [&](int span) __attribute__((always_inline)) {
            if (r.inside(span * kSpanVecs, kSpanVecs)) {
#pragma unroll
                for (int b = 0; b < kSpanBlocks; ++b)
                    v[b] = r.load_inside(span * kSpanVecs + b * kBlockVecs + lane);
            } else {
#pragma unroll 1
                for (int b = 0; b < kSpanBlocks; ++b) {
                    const u32x4_t x = r.load(min(span * kSpanVecs + b * kBlockVecs + lane, vecs));
#pragma unroll
                    for (int k = 0; k < kSpanBlocks; ++k)
                        v[k] = b == k ? x : v[k];
                }
            }
        };
        load(first);
        for (int span = first; span < st.spans; span += step) {
            float z[kSpanBlocks][kE], top[kSpanBlocks];
#pragma unroll
            for (int b = 0; b < kSpanBlocks; ++b) {
                // (here, not behind the loads: the wait for them would come along)
                asm volatile("" : "+v"(v[b]));
                Row<kBf16>::unpack(v[b], z[b]);
            }
            if (span + step < st.spans)
                load(span + step);
#pragma unroll
            for (int b = 0; b < kSpanBlocks; ++b) {
                top[b] = z[b][0];
#pragma unroll
                for (int e = 1; e + 1 < kE; e += 2)
                    top[b] = max3(top[b], z[b][e], z[b][e + 1]);
                top[b] = max3(top[b], z[b][kE - 1], top[b]);
            }
            // (its row's block's, as unpack_whole has the logits: -0 is 0, whose key it would not have)
            const float row_top = fminf(wave_max4(top), FLT_MAX) + 0.f;
            auto of_row = [&](int row) __attribute__((always_inline)) {
                return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(row_top), 16 * row));
            };
            const float m = fmaxf(fmaxf(of_row(0), of_row(1)), fmaxf(of_row(2), of_row(3)));
            const int64_t at = row * st.spans + span;
            if ((lane & 15) == 0)
                st.maxima[at * kSpanBlocks + ((lane >> 4 & 1) * 2 + (lane >> 5))] = row_top;
            if (!sums)
                continue;
            double sum = 0.;
            if (m > -INFINITY) {
                const double md = m;
                // logits raised to `low` have a weight of 2^-1000, which no sum here feels, and need no
                // other care; where fp32 has no such number, the temperature is far out
                const float low = (float)(md - 1000. / f.c);
                const double t = ((double)low - md) * f.c;
                if (low > -INFINITY && t >= -1019. && t <= -900.) {
#pragma unroll
                    for (int b = 0; b < kSpanBlocks; ++b)
#pragma unroll
                        for (int e = 0; e < kE; ++e)
                            sum += exp2_fast((double)__builtin_amdgcn_fmed3f(z[b][e], low, m) - md, f.c);
                } else {
#pragma unroll 1
                    for (int b = 0; b < kSpanBlocks; ++b)
#pragma unroll
                        for (int e = 0; e < kE; ++e) {
                            float x = z[0][e];
#pragma unroll
                            for (int k = 1; k < kSpanBlocks; ++k)
                                x = b == k ? z[k][e] : x;
                            sum += weight_of(fminf(x, m), md, f.c);
                        }
                }
            }
            sum = wave_total_64(sum);
            if (lane == 63)
                st.sums[at] = sum;
        }
    }
}

struct PickLds {
    alignas(16) float max[kMaxBlocks];  // the blocks' maxima
    float top[kMaxSpans];        // the spans'
    uint16_t list[kMaxBlocks];   // blocks that may hold a kept token
    double sum[kMaxBlocks];      // weights kept in a block, or in a listed one
    double red[kPickWaves];
    uint32_t cnt[kPickWaves];
    uint32_t n;                  // a counter, a result
    uint32_t found, found2;
    double total, before;
    uint64_t d0;
    union {
        struct {
            uint64_t key[kSampleSort];  // ~key of the logit and index, ascending: the filters' order
            double w[kSampleSort];
        } sort;
        struct {
            unsigned long long w[kDigits];
            uint32_t n[kDigits];
        } hist;
        uint32_t ties[kMaxBlocks];
    };
};
static_assert(sizeof(PickLds) <= 64 << 10, "LDS of a workgroup");

// Sums over the workgroup's threads in their order: inclusive scan and the total.  The LDS is free
// again after the caller's next barrier.
__device__ __forceinline__ double block_scan_64(double x, double *red, double &total)
{
    const int wave = threadIdx.x >> 6;
    x = wave_scan_64(x);
    if ((threadIdx.x & 63) == 63)
        red[wave] = x;
    __syncthreads();
    double base = 0., t = 0.;
#pragma unroll
    for (int w = 0; w < kPickWaves; ++w) {
        base = w == wave ? t : base;
        t += red[w];
    }
    total = t;
    return base + x;
}

__device__ __forceinline__ uint32_t block_scan_32(uint32_t x, uint32_t *cnt, uint32_t &total)
{
    const int wave = threadIdx.x >> 6;
    x = wave_scan_add(x);
    if ((threadIdx.x & 63) == 63)
        cnt[wave] = x;
    __syncthreads();
    uint32_t base = 0, t = 0;
#pragma unroll
    for (int w = 0; w < kPickWaves; ++w) {
        base = w == wave ? t : base;
        t += cnt[w];
    }
    total = t;
    return base + x;
}

// n different keys into ascending order, with all ones behind them up to a power of two.  Up to 256 by counting
// the smaller ones, 64 in an instruction, each wave for every 8th key; more, at most two per thread, by
// a bitonic network, whose steps are an LDS trip each (32 keys 15 of them: 1.7 us of one row's 17).
__device__ __forceinline__ void sort_keys(uint64_t *key, int n, int size)
{
    constexpr int kRanked = 256;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    if (n <= kRanked) {
        static_assert(kRanked <= 64 * kPickWaves, "a lane's own key");
        const int own = wave + kPickWaves * lane;
        uint64_t all[kRanked / 64], mine = own < n ? key[own] : 0;
#pragma unroll
        for (int r = 0; r < kRanked / 64; ++r)
            all[r] = lane + 64 * r < n ? key[lane + 64 * r] : ~0ull;
        int rank = 0;
        for (int q = 0; wave + kPickWaves * q < n; ++q) {
            const uint64_t k = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), q) << 32 |
                               (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)mine, q);
            int less = 0;
#pragma unroll
            for (int r = 0; r < kRanked / 64; ++r)
                if (64 * r < n)
                    less += __popcll(__ballot(all[r] < k));
            rank = lane == q ? less : rank;
        }
        __syncthreads();
        if (own < n)
            key[rank] = mine;
        __syncthreads();
        return;
    }
    for (int k = 2; k <= size; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
            if (t < size >> 1) {
                const int i = 2 * t - (t & (j - 1));
                const uint64_t a = key[i], b = key[i + j];
                if ((a > b) == ((i & k) == 0)) {
                    key[i] = b;
                    key[i + j] = a;
                }
            }
            __syncthreads();
        }
}

// The first of the threads' pairs that `even` or `odd` holds for, into *found unless less is there; one
// atomic of a wave.
__device__ __forceinline__ void first_of(uint32_t *found, bool even, bool odd)
{
    const uint64_t hits = __ballot(even || odd);
    if (hits && (int)(threadIdx.x & 63) == __builtin_ctzll(hits))
        atomicMin(found, 2 * threadIdx.x + (even ? 0u : 1u));
}

__device__ __forceinline__ int pow2_from(int n)
{
    return n <= 2 ? 2 : 1 << (32 - __builtin_clz(n - 1));
}

// Which tokens are kept: those above `key`, the first `ties` of those at it, and of both w >= q.
struct Rule {
    uint32_t key, ties;
    double q;
};

// A row and the tokens of its blocks, for a wave.
template <bool kBf16>
struct RowPicker {
    static constexpr int kE = kElems<kBf16>;
    const SampleArgs &a;
    const Row<kBf16> r;
    const Filters f;
    const int64_t row;
    double u;
    int vecs, blocks;
    float m;
    double md;

    __device__ __forceinline__ RowPicker(const SampleArgs &args, int64_t row_)
        : a(args), r(args, row_), f(args, row_), row(row_)
    {
        const float x = a.uniform[row];
        u = x > 0.f ? fminf(x, 1.f - FLT_EPSILON / 2) : 0.;
        vecs = r.vecs();
        blocks = (vecs + kBlockVecs - 1) / kBlockVecs;
    }

    __device__ __forceinline__ void answer(int token, double logprob)
    {
        if (threadIdx.x == 0) {
            a.tokens[row] = token;
            if (a.logprobs)
                a.logprobs[row] = (float)logprob;
        }
    }

    __device__ __forceinline__ void load_block(int b, float (&z)[kE]) const
    {
        Row<kBf16>::unpack_whole(r.block_end(b, r.block_begin(b)), z);
    }
    __device__ __forceinline__ int index_in(int b, int e) const
    {
        return r.index(b * kBlockVecs + (int)(threadIdx.x & 63), e);
    }

    // The token of block b (by its first wave) at which the running sum of w exceeds `at`; total: the sum over
    // all kept tokens.
    __device__ __forceinline__ void pick_in_block(int b, const float (&z)[kE], const double (&w)[kE],
                                                  double at, double total)
    {
        double sum = 0.;
        uint32_t at_e = 0xffffffffu, last_e = 0;
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            sum += w[e];
            last_e = w[e] > 0. ? (uint32_t)e : last_e;
        }
        double here = wave_scan_64(sum) - sum;
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            here += w[e];
            if (at_e == 0xffffffffu && w[e] > 0. && here > at)
                at_e = (uint32_t)e;
        }
        const uint64_t hits = __ballot(at_e != 0xffffffffu);
        const uint64_t some = __ballot(sum > 0.);  // (the block holds a kept token)
        // (none, by rounding: the last one)
        const int lane = hits ? __builtin_ctzll(hits) : (some ? 63 - __builtin_clzll(some) : 0);
        const uint32_t el = hits ? at_e : last_e;
        float zt = z[0];
#pragma unroll
        for (int e = 1; e < kE; ++e)
            zt = el == (uint32_t)e ? z[e] : zt;
        zt = __shfl(zt, lane, 64);
        answer(__shfl(index_in(b, (int)el), lane, 64), ((double)zt - md) / f.t - log(total));
    }

    static constexpr int kPer = (kMaxSpans + 63) / 64;  // spans of a lane at most, neighbouring ones

    // A wave's lanes take the row's spans: maxima of their blocks and of each, sums where there are any; m.
    __device__ __forceinline__ void load_stats(const Stats &st, u32x4_t (&max4)[kPer], float (&top)[kPer],
                                               double (&w)[kPer])
    {
        const int per = (st.spans + 63) / 64, first = (threadIdx.x & 63) * per;
        const float *maxima = st.maxima + row * st.spans * kSpanBlocks;
        constexpr uint32_t kNone = 0xff800000u;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            max4[i] = (u32x4_t){kNone, kNone, kNone, kNone};
            w[i] = 0.;
            if (i < per && first + i < st.spans) {
                max4[i] = ld16(maxima + (first + i) * kSpanBlocks);
                if (f.sums())
                    w[i] = st.sums[row * st.spans + first + i];
            }
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            top[i] = fmaxf(fmaxf(__uint_as_float(max4[i][0]), __uint_as_float(max4[i][1])),
                           fmaxf(__uint_as_float(max4[i][2]), __uint_as_float(max4[i][3])));
        float t = top[0];
#pragma unroll
        for (int i = 1; i < kPer; ++i)
            t = fmaxf(t, top[i]);
        m = wave_max_f(t);
        md = m;
    }

    // The largest logit's token, the draw without a filter.
    __device__ __forceinline__ void greedy(const Stats &st, const float (&top)[kPer])
    {
        const int per = (st.spans + 63) / 64, first = (threadIdx.x & 63) * per;
        const float *maxima = st.maxima + row * st.spans * kSpanBlocks;
        int span = -1;
#pragma unroll
        for (int i = kPer - 1; i >= 0; --i)
            span = top[i] == m ? first + i : span;
        span = __builtin_amdgcn_readlane(span, __builtin_ctzll(__ballot(span >= 0)));
        int b = kSpanBlocks - 1;
#pragma unroll
        for (int i = kSpanBlocks - 2; i >= 0; --i)
            b = maxima[span * kSpanBlocks + i] == m ? i : b;
        b += span * kSpanBlocks;
        float z[kE];
        load_block(b, z);
        uint32_t at = 0xffffffffu;
#pragma unroll
        for (int e = kE - 1; e >= 0; --e)
            at = z[e] == m ? (uint32_t)index_in(b, e) : at;
        answer((int)wave_min(at), 0.);
    }

    // The spans' sums brought to the row's maximum; the lanes' parts; their sum.
    __device__ __forceinline__ double whole_sum(const float (&top)[kPer], double (&w)[kPer], double &incl,
                                                double &part) const
    {
        part = 0.;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            w[i] = w[i] > 0. ? w[i] * weight_of(top[i], md, f.c) : 0.;
            part += w[i];
        }
        incl = wave_scan_64(part);
        return lane_64(incl, 63);
    }

    __device__ __forceinline__ void plain(const Stats &st, const double (&w)[kPer], double incl, double part,
                                          double total)
    {
        const int per = (st.spans + 63) / 64, first = (threadIdx.x & 63) * per;
        const double at = u * total;
        // ---- the span: the first at which the running sum exceeds it (by rounding none: the last)
        double run = incl - part, before = 0.;
        int span = -1;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (span < 0 && w[i] > 0. && run + w[i] > at) {
                span = first + i;
                before = run;
            }
            run += w[i];
        }
        const uint64_t hits = __ballot(span >= 0);
        if (hits) {
            const int from = __builtin_ctzll(hits);
            span = __builtin_amdgcn_readlane(span, from);
            before = lane_64(before, from);
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                span = w[i] > 0. ? first + i : span;
            span = __builtin_amdgcn_readlane(span, 63 - __builtin_clzll(__ballot(part > 0.)));
            before = -INFINITY;
        }
        // ---- the block, the token
        double wb[kSpanBlocks][kE], sum[kSpanBlocks];
        float z[kSpanBlocks][kE];
#pragma unroll
        for (int b = 0; b < kSpanBlocks; ++b)
            load_block(span * kSpanBlocks + b, z[b]);
#pragma unroll
        for (int b = 0; b < kSpanBlocks; ++b) {
            sum[b] = 0.;
#pragma unroll
            for (int e = 0; e < kE; ++e) {
                wb[b][e] = weight_of(z[b][e], md, f.c);
                sum[b] += wb[b][e];
            }
        }
#pragma unroll
        for (int b = 0; b < kSpanBlocks; ++b)
            sum[b] = wave_sum_64(sum[b]);
        double left = hits ? at - before : INFINITY;
        int b = -1;
        double in_block = 0.;
#pragma unroll
        for (int k = 0; k < kSpanBlocks; ++k) {
            // (`left` may be below 0 by a rounding, which a block without a kept token does not take)
            if (b < 0 && sum[k] > 0. && sum[k] > left) {
                b = k;
                in_block = left;
            }
            left -= b < 0 ? sum[k] : 0.;
        }
        if (b < 0) {
#pragma unroll
            for (int k = 0; k < kSpanBlocks; ++k)
                b = sum[k] > 0. ? k : b;
            in_block = INFINITY;
        }
        float zb[kE];
        double ws[kE];
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            zb[e] = z[0][e];
            ws[e] = wb[0][e];
#pragma unroll
            for (int k = 1; k < kSpanBlocks; ++k) {
                zb[e] = b == k ? z[k][e] : zb[e];
                ws[e] = b == k ? wb[k][e] : ws[e];
            }
        }
        pick_in_block(span * kSpanBlocks + b, zb, ws, in_block, total);
    }

    // The row, which has no filter, by a wave.
    __device__ __forceinline__ void simple(const Stats &st)
    {
        u32x4_t max4[kPer];
        float top[kPer];
        double w[kPer], incl, part;
        load_stats(st, max4, top, w);
        if (!(m > -INFINITY)) {  // every token is masked
            answer(-1, -INFINITY);
        } else if (f.greedy) {
            greedy(st, top);
        } else {
            const double total = whole_sum(top, w, incl, part);
            plain(st, w, incl, part, total);
        }
    }
};

// One row, by a workgroup with its LDS.
template <bool kBf16>
struct Picker : RowPicker<kBf16> {
    using Base = RowPicker<kBf16>;
    using Base::a;
    using Base::answer;
    using Base::blocks;
    using Base::f;
    using Base::index_in;
    using Base::load_block;
    using Base::m;
    using Base::md;
    using Base::pick_in_block;
    using Base::r;
    using Base::row;
    using Base::u;
    using Base::vecs;
    static constexpr int kE = Base::kE, kPer = Base::kPer;
    PickLds &s;

    __device__ __forceinline__ Picker(const SampleArgs &args, PickLds &lds, int64_t row_)
        : Base(args, row_), s(lds)
    {
    }

    // Calls use(j, z) with the 64 vectors of every listed block j, in the waves' turns, kAhead blocks' loads
    // under way.  kStop: until s.n tells of more tokens than are sorted.  (use's code is there kAhead times, and a
    // row runs it a few dozen times: with 8 the instructions' own loads took longer.)
    template <bool kStop = false, typename Use>
    __device__ __forceinline__ void each_block(int n, Use use)
    {
        each_vector<kStop>(n, [&](int j, u32x4_t x) __attribute__((always_inline)) {
            float z[kE];
            Row<kBf16>::unpack_whole(x, z);
            use(j, z);
        });
    }

    // The same with the vectors as they lie in memory.
    template <bool kStop = false, typename Use>
    __device__ __forceinline__ void each_vector(int n, Use use)
    {
        constexpr int kAhead = 4;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), last = max(n - 1, 0);
        u32x4_t v[kAhead];
        int id[kAhead];
        auto begin = [&](int i, int j) __attribute__((always_inline)) {
            id[i] = __builtin_amdgcn_readfirstlane(s.list[min(j, last)]);
            v[i] = r.block_begin(id[i]);
        };
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            begin(i, wave + i * kPickWaves);
#pragma unroll 1
        for (int j0 = wave; j0 < n; j0 += kAhead * kPickWaves) {
            if (kStop && *(volatile uint32_t *)&s.n > (uint32_t)kSampleSort)
                break;
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int j = j0 + i * kPickWaves;
                u32x4_t x = v[i];
                asm volatile("" : "+v"(x));
                const int b = id[i];
                begin(i, j + kAhead * kPickWaves);
                if (j < n)
                    use(j, r.block_end(b, x));
            }
        }
    }

    // The blocks whose maximum reaches tau (and holds a token at all), in order; their number.
    __device__ __forceinline__ int list_blocks(float tau)
    {
        uint32_t n = 0;
        for (int b0 = 0; b0 < blocks; b0 += kPickThreads) {
            const int b = b0 + threadIdx.x;
            const bool in = b < blocks && s.max[b] >= tau && s.max[b] > -INFINITY;
            uint32_t total;
            const uint32_t at = block_scan_32(in ? 1u : 0u, s.cnt, total);
            if (in)
                s.list[n + at - 1] = (uint16_t)b;
            n += total;
            __syncthreads();
        }
        return (int)n;
    }

    // A lower bound of the k-th largest of count maxima, of the spans where there are k, else of the blocks, exact
    // to its upper 16 key bits: bit by bit, every wave for itself, with the keys in registers and no
    // barrier.
    template <int kMost>
    __device__ __forceinline__ float kth_maximum(const float *maxima, int count, int k) const
    {
        constexpr int kRegs = (kMost + 63) / 64;
        const int lane = threadIdx.x & 63;
        uint32_t x[kRegs];
#pragma unroll
        for (int r = 0; r < kRegs; ++r)
            x[r] = lane + 64 * r < count ? key_of(maxima[lane + 64 * r]) : 0u;
        uint32_t bound = 0;
#pragma unroll 1
        for (int bit = 31; bit >= 16; --bit) {
            const uint32_t t = bound | 1u << bit;
            int n = 0;
#pragma unroll
            for (int r = 0; r < kRegs; ++r)
                n += __popcll(__ballot(x[r] >= t));
            bound = n >= k ? t : bound;
        }
        return bound_of(bound);
    }

    // The logit of a bound's key (one below that of -inf belongs to no number).
    __device__ __forceinline__ static float bound_of(uint32_t key)
    {
        return key <= key_of(-INFINITY) ? -INFINITY : logit_of(key);
    }

    // A bound that every token kept reaches (and what top-p's sum is over); kth: that of top-k's blocks.
    __device__ __forceinline__ float bound(double whole, float kth) const
    {
        float tau = -INFINITY;
        if (f.k)
            tau = kth;
        else if (f.p < 1.f)
            tau = below(md + log((1. - (double)f.p) * whole / a.vocab) * f.t);
        if (f.q > 0.f && !(f.k && f.p < 1.f))
            tau = fmaxf(tau, below(md + log((double)f.q) * f.t));
        return tau;
    }

    // Tokens of at least tau into the sorting LDS, any order; their number (more than fit: not all).
    __device__ __forceinline__ int collect(int n_list, float tau)
    {
        if (threadIdx.x == 0)
            s.n = 0;
        __syncthreads();
        each_block<true>(n_list, [&](int j, const float(&z)[kE]) __attribute__((always_inline)) {
            const int b = s.list[j];
            uint32_t mine = 0;
#pragma unroll
            for (int e = 0; e < kE; ++e)
                mine += z[e] >= tau && z[e] > -INFINITY ? 1u : 0u;
            if (__ballot(mine != 0) == 0)
                return;
            const uint32_t incl = wave_scan_add(mine);
            uint32_t at = 0;
            if ((threadIdx.x & 63) == 63)
                at = atomicAdd(&s.n, incl);
            at = (uint32_t)__builtin_amdgcn_readlane((int)at, 63) + incl - mine;
#pragma unroll
            for (int e = 0; e < kE; ++e)
                if (z[e] >= tau && z[e] > -INFINITY) {
                    if (at < (uint32_t)kSampleSort)
                        s.sort.key[at] = (uint64_t)~key_of(z[e]) << 32 | (uint32_t)index_in(b, e);
                    ++at;
                }
        });
        __syncthreads();
        return (int)s.n;
    }

    // The whole rest on n collected tokens; whole: the sum over all tokens (without top-k).
    __device__ __forceinline__ void finish_sorted(int n, double whole)
    {
        const int t = threadIdx.x;
        int size = pow2_from(n);
        for (int i = n + t; i < size; i += kPickThreads)
            s.sort.key[i] = ~0ull;
        __syncthreads();
        sort_keys(s.sort.key, n, size);
        double w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int j = 2 * t + i;
            w[i] = j < n ? weight_of(logit_of(~(uint32_t)(s.sort.key[j] >> 32)), md, f.c) : 0.;
        }
        double total;
        const double incl = block_scan_64(w[0] + w[1], s.red, total);
        const double before[2] = {incl - w[1] - w[0], incl - w[1]};
        int keep = f.k && f.k < n ? f.k : n;
        __syncthreads();
        if (f.k) {  // the sum over top-k's
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (2 * t + i == keep - 1)
                    s.total = before[i] + w[i];
            __syncthreads();
            whole = s.total;
        }
        const double most = (double)f.p * whole;
        uint32_t mine = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int j = 2 * t + i;
            if (j < keep && (j == 0 || f.p >= 1.f || before[i] < most) && w[i] >= (double)f.q)
                ++mine;
            if (j < n)
                s.sort.w[j] = w[i];
        }
        uint32_t kept;
        block_scan_32(mine, s.cnt, kept);
        keep = (int)kept;  // (the conditions hold for a first part of the order)
        // ---- the kept by index
        uint64_t key[2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
            key[i] = s.sort.key[2 * t + i < size ? 2 * t + i : 0];
        __syncthreads();
        size = pow2_from(keep);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int j = 2 * t + i;
            if (j < size)
                s.sort.key[j] = j < keep ? key[i] << 32 | (uint32_t)j : ~0ull;
        }
        if (t == 0)
            s.found = (uint32_t)keep - 1;
        __syncthreads();
        sort_keys(s.sort.key, keep, size);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int j = 2 * t + i;
            w[i] = j < keep ? s.sort.w[(uint32_t)s.sort.key[j]] : 0.;
        }
        const double run = block_scan_64(w[0] + w[1], s.red, total);
        const double at = u * total;
        // (a kept token of no weight: the sum at it may exceed by a rounding what the one before did not)
        first_of(&s.found, w[0] > 0. && run - w[1] > at, w[1] > 0. && run > at);
        __syncthreads();
        if (t == 0) {
            const uint64_t k = s.sort.key[s.found];
            answer((int)(k >> 32), log(s.sort.w[(uint32_t)k] / total));
        }
    }

    // Top-p alone, of more tokens above tau than are sorted.  whole: the sum over all tokens.  False: too many
    // lie about the border.
    __device__ __forceinline__ bool finish_located(int n_list, float tau, double whole)
    {
        constexpr uint32_t kBins = kDigits;
        const int t = threadIdx.x;
        const float width = (m - tau) * (1.f / ((float)kBins - 0.5f)), per = 1.f / width;
        const float cf = (float)f.c;
        // (a logit of `low` has a weight that no sum feels, but one that exp2_fast takes, and no bin)
        const float low = (float)(md - 1000. / f.c);
        const double low_t = ((double)low - md) * f.c;
        if (!(width > 0.f && per < 1e30f && per > 0.f && cf < 1e30f && low > -INFINITY &&
              (m - low) * per > (float)kBins && low_t >= -1019. && low_t <= -900.))
            return false;
        auto bin_of = [&](float z) -> uint32_t {  // grows as z falls
            const float x = (m - z) * per;
            return x < (float)kBins ? (uint32_t)x : kBins;
        };
        // ---- fp32 weights in units of 2^-31 of the sum.  A bin's total is off by a unit for each token, and by
        // the weights' relative error: 2^-23 from the exponential, and three roundings of the exponent, which
        // is 43 at most above tau (weights of 2^-24 / 2^19 of the sum): 43 ln 2 * 3 * 2^-24 < 2^-17.
        const float unit = (float)(2147483648. / whole);
        uint32_t *hist = s.hist.n;
        hist[t] = hist[t + kPickThreads] = 0;
        if (t == 0) {
            s.n = 0;
            s.found = s.found2 = kBins;
        }
        for (int b = t; b < blocks; b += kPickThreads)
            s.sum[b] = 0.;
        __syncthreads();
        each_vector(n_list, [&](int, u32x4_t v) __attribute__((always_inline)) {
            float z[kE];
            Row<kBf16>::unpack_clamped(v, low, m, z);
#pragma unroll
            for (int e = 0; e < kE; ++e) {
                const float d = m - z[e], x = d * per;
                if (x < (float)kBins)
                    atomicAdd(&hist[(uint32_t)x],
                              (uint32_t)(__builtin_amdgcn_exp2f(-d * cf) * unit));
            }
        });
        __syncthreads();
        const uint32_t h0 = hist[2 * t], h1 = hist[2 * t + 1];
        uint32_t total;
        const uint32_t incl = block_scan_32(h0 + h1, s.cnt, total);
        const int64_t error = (int64_t)a.vocab + (1 << 14) + 64;
        const int64_t most_u = (int64_t)((double)f.p * 2147483648.);
        const int64_t after[2] = {(int64_t)incl - h1, (int64_t)incl};
        const int64_t in_front[2] = {(int64_t)incl - h1 - h0, (int64_t)incl - h1};
        // the first bin that may not be kept whole, the first that is surely left out
        first_of(&s.found, after[0] + error >= most_u, after[1] + error >= most_u);
        first_of(&s.found2, in_front[0] - error >= most_u, in_front[1] - error >= most_u);
        __syncthreads();
        const uint32_t b0 = s.found, b1 = s.found2;
        __syncthreads();
        // ---- the sums of the kept bins, block by block; the tokens between are sorted
        const float x0 = (float)b0, x1 = (float)b1;  // (bin < b: x < b)
        auto kept_sums = [&](auto min_p) __attribute__((always_inline)) {
            each_vector(n_list, [&](int j, u32x4_t v) __attribute__((always_inline)) {
                const int b = s.list[j];
                float z[kE], x[kE];
                Row<kBf16>::unpack_clamped(v, low, m, z);
                bool some = false, between = false;
#pragma unroll
                for (int e = 0; e < kE; ++e) {
                    x[e] = (m - z[e]) * per;
                    some |= x[e] < x0;
                    between |= x[e] >= x0 && x[e] < x1;
                }
                if (__ballot(some)) {
                    double sum = 0.;
#pragma unroll
                    for (int e = 0; e < kE; ++e) {
                        const double w = exp2_fast((double)(x[e] < x0 ? z[e] : low) - md, f.c);
                        sum += !min_p() || w >= (double)f.q ? w : 0.;
                    }
                    sum = wave_sum_64(sum);
                    if ((threadIdx.x & 63) == 0)
                        s.sum[b] = sum;
                }
                if (__ballot(between) == 0)
                    return;
                uint32_t mine = 0;
#pragma unroll
                for (int e = 0; e < kE; ++e)
                    mine += x[e] >= x0 && x[e] < x1 ? 1u : 0u;
                const uint32_t run = wave_scan_add(mine);
                uint32_t at = 0;
                if ((threadIdx.x & 63) == 63)
                    at = atomicAdd(&s.n, run);
                at = (uint32_t)__builtin_amdgcn_readlane((int)at, 63) + run - mine;
#pragma unroll
                for (int e = 0; e < kE; ++e)
                    if (x[e] >= x0 && x[e] < x1) {
                        if (at < (uint32_t)kSampleSort)
                            s.sort.key[at] = (uint64_t)~key_of(z[e] + 0.f) << 32 | (uint32_t)index_in(b, e);
                        ++at;
                    }
            });
        };
        if (f.q > 0.f)
            kept_sums(std::true_type{});
        else
            kept_sums(std::false_type{});
        __syncthreads();
        const int n = (int)s.n;
        if (n > kSampleSort)
            return false;
        // ---- the sums in fixed point (their order no longer matters), and what lies above the border
        const double unit60 = fixed_unit(whole);
        const int per_thread = (blocks + kPickThreads - 1) / kPickThreads;
        const int block0 = min(blocks, t * per_thread), block1 = min(blocks, block0 + per_thread);
        uint64_t *fixed = reinterpret_cast<uint64_t *>(s.sum);
        double part = 0., above;
        for (int b = block0; b < block1; ++b) {
            part += s.sum[b];
            fixed[b] = (uint64_t)__builtin_rint(s.sum[b] * unit60);
        }
        block_scan_64(part, s.red, above);
        // ---- the border: its tokens in order, kept while the sum before is below p of the whole
        const int size = pow2_from(n);
        for (int i = n + t; i < size; i += kPickThreads)
            s.sort.key[i] = ~0ull;
        __syncthreads();
        sort_keys(s.sort.key, n, size);
        double w[2], all;
        uint64_t key[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int j = 2 * t + i;
            key[i] = j < n ? s.sort.key[j] : ~0ull;
            w[i] = j < n ? weight_of(logit_of(~(uint32_t)(key[i] >> 32)), md, f.c) : 0.;
        }
        const double run = block_scan_64(w[0] + w[1], s.red, all);
        const double before[2] = {above + (run - w[1] - w[0]), above + (run - w[1])};
        const double most = (double)f.p * whole;
        uint32_t mine = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (2 * t + i < n && before[i] < most && w[i] >= (double)f.q) {
                ++mine;
                const int v = ((int)(uint32_t)key[i] + r.off) / kE;
                atomicAdd(reinterpret_cast<unsigned long long *>(fixed + v / kBlockVecs),
                          (unsigned long long)__builtin_rint(w[i] * unit60));
            }
        uint32_t kept;
        block_scan_32(mine, s.cnt, kept);
        __syncthreads();
        // a border token is kept up to this one: of its key by index (none: no key reaches it)
        const uint64_t last = kept ? s.sort.key[kept - 1] : 0;
        const uint32_t last_key = kept ? ~(uint32_t)(last >> 32) : 0xffffffffu, last_id = (uint32_t)last;
        // ---- the draw: the block, then the token
        uint64_t mine64 = 0;
        for (int b = block0; b < block1; ++b)
            mine64 += fixed[b];
        uint64_t run64 = scan_u64(mine64) - mine64;
        if (t == 0)
            s.found = kMaxBlocks;
        __syncthreads();
        const uint64_t all64 = s.d0, at = (uint64_t)(u * (double)all64);
        uint64_t here = 0;
        uint32_t hit = kMaxBlocks;
        for (int b = block0; b < block1; ++b) {
            if (hit == kMaxBlocks && run64 + fixed[b] > at && fixed[b]) {
                hit = (uint32_t)b;
                here = run64;
            }
            run64 += fixed[b];
        }
        if (hit < kMaxBlocks)
            atomicMin(&s.found, hit);
        __syncthreads();
        if (hit < kMaxBlocks && s.found == hit)
            s.before = (double)(at - here) / unit60;  // what is left of the draw in this block
        __syncthreads();
        if (t >= 64)
            return true;
        const int b = (int)s.found;
        float z[kE];
        load_block(b, z);
        double we[kE];
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            const uint32_t k = key_of(z[e]), bin = bin_of(z[e]);
            const bool in = bin < b0 || (bin < kBins && (k > last_key ||
                                         (k == last_key && (uint32_t)index_in(b, e) <= last_id)));
            const double x = in ? weight_of(z[e], md, f.c) : 0.;
            we[e] = x >= (double)f.q ? x : 0.;
        }
        pick_in_block(b, z, we, s.before, (double)all64 / unit60);
        return true;
    }

    // A power of two that brings a sum to 2^60 .. 2^61.
    __device__ __forceinline__ static double fixed_unit(double sum)
    {
        const int exponent = (int)(__builtin_bit_cast(uint64_t, sum) >> 52) - 1023;
        return __builtin_ldexp(1., 60 - exponent);
    }

    // The draw among the listed blocks' kept tokens.
    __device__ __forceinline__ void draw(int n, const Rule &rule)
    {
        const double tie_w = weight_of(logit_of(rule.key), md, f.c);
        each_block(n, [&](int j, const float(&z)[kE]) __attribute__((always_inline)) {
            double sum = 0.;
            uint32_t ties = 0, above = 0;
#pragma unroll
            for (int e = 0; e < kE; ++e) {
                const uint32_t key = key_of(z[e]);
                above |= key > rule.key ? 1u << e : 0u;
                ties += key == rule.key ? 1u : 0u;
            }
            if (__ballot(above != 0)) {
#pragma unroll
                for (int e = 0; e < kE; ++e)
                    if (above >> e & 1) {
                        const double w = weight_of(z[e], md, f.c);
                        sum += w >= rule.q ? w : 0.;
                    }
                sum = wave_sum_64(sum);
            }
            ties = wave_scan_add(ties);
            if ((threadIdx.x & 63) == 63) {
                s.sum[j] = sum;
                s.ties[j] = ties;
            }
        });
        __syncthreads();
        const int per = (n + kPickThreads - 1) / kPickThreads;
        const int j0 = min(n, (int)threadIdx.x * per), j1 = min(n, j0 + per);
        if (threadIdx.x == 0)
            s.found = 0xffffffffu;
        uint32_t mine = 0, ties;
        for (int j = j0; j < j1; ++j)
            mine += s.ties[j];
        uint32_t first = block_scan_32(mine, s.cnt, ties) - mine;
        double part = 0.;
        const bool tie_in = tie_w >= rule.q;
        for (int j = j0; j < j1; ++j) {
            const uint32_t c = s.ties[j];
            const uint32_t in = tie_in && first < rule.ties ? min(c, rule.ties - first) : 0u;
            s.sum[j] += in * tie_w;
            s.ties[j] = in;  // (from here on: the ties of the block that are kept)
            first += c;
            part += s.sum[j];
        }
        double total;
        double run = block_scan_64(part, s.red, total) - part;
        const double at = u * total;
        uint32_t hit = 0xffffffffu;
        double hit_run = 0.;
        for (int j = j0; j < j1; ++j) {
            if (hit == 0xffffffffu && run + s.sum[j] > at && s.sum[j] > 0.) {
                hit = (uint32_t)j;
                hit_run = run;
            }
            run += s.sum[j];
        }
        if (hit != 0xffffffffu)
            atomicMin(&s.found, hit);
        __syncthreads();
        if (s.found == hit && hit != 0xffffffffu)
            s.before = hit_run;
        __syncthreads();
        bool last = false;
        if (s.found == 0xffffffffu) {  // rounding: the last kept token
            last = true;
            __syncthreads();
            if (threadIdx.x == 0)
                s.found = 0;
            __syncthreads();
            for (int j = j0; j < j1; ++j)
                if (s.sum[j] > 0.)
                    atomicMax(&s.found, (uint32_t)j);
            __syncthreads();
        }
        if (threadIdx.x >= 64)
            return;
        const int j = (int)s.found, b = s.list[j];
        float z[kE];
        double w[kE];
        load_block(b, z);
        uint32_t c = 0;
#pragma unroll
        for (int e = 0; e < kE; ++e)
            c += key_of(z[e]) == rule.key ? 1u : 0u;
        uint32_t rank = wave_scan_add(c) - c;
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            const uint32_t key = key_of(z[e]);
            const double x = weight_of(z[e], md, f.c);
            const bool keep = key == rule.key ? rank < s.ties[j] : key > rule.key && x >= rule.q;
            rank += key == rule.key ? 1u : 0u;
            w[e] = keep ? x : 0.;
        }
        pick_in_block(b, z, w, last ? INFINITY : at - s.before, total);
    }

    // ---- thresholds by digits of the keys, for more candidates than are sorted
    struct Cut {
        uint32_t key, ties;
        uint64_t w;   // fixed-point weight of the kept
        bool all;     // fewer than asked for: every candidate is kept
    };

    // The cut behind which `want` tokens (by_count), or the fixed-point weight `want`, are reached.
    __device__ __forceinline__ Cut cut(int n, uint32_t low, bool by_count, uint64_t want, double unit)
    {
        const uint32_t top = key_of(m);
        const uint32_t range = top - low;
        int bits = range ? 32 - __builtin_clz(range) : 0;
        uint32_t d0 = 0;
        uint64_t width = 1ull << bits, seen_n = 0, seen_w = 0;
        for (;;) {
            const int shift = bits > kDigitBits ? bits - kDigitBits : 0;
            for (int i = threadIdx.x; i < kDigits; i += kPickThreads) {
                s.hist.w[i] = 0;
                s.hist.n[i] = 0;
            }
            if (threadIdx.x == 0)
                s.found = 0xffffffffu;
            __syncthreads();
            each_block(n, [&](int, const float(&z)[kE]) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < kE; ++e) {
                    const uint32_t key = key_of(z[e]);
                    const uint64_t d = (uint64_t)(top - key) - d0;  // (below d0: wraps, out of width)
                    if (key >= low && key <= top && d < width) {
                        const int bin = (int)(d >> shift);
                        atomicAdd(&s.hist.w[bin], (unsigned long long)__builtin_rint(
                                                      weight_of(z[e], md, f.c) * unit));
                        atomicAdd(&s.hist.n[bin], 1u);
                    }
                }
            });
            __syncthreads();
            // two digits a thread, in order
            const int i = 2 * threadIdx.x;
            const uint64_t w0 = s.hist.w[i], w1 = s.hist.w[i + 1];
            const uint32_t n0 = s.hist.n[i], n1 = s.hist.n[i + 1];
            uint32_t total_n;
            const uint32_t incl_n = block_scan_32(n0 + n1, s.cnt, total_n);
            const uint64_t incl_w = scan_u64(w0 + w1);
            const uint64_t bn = seen_n + incl_n - n1 - n0, bw = seen_w + incl_w - w1 - w0;
            first_of(&s.found, n0 && (by_count ? bn + n0 >= want : bw + w0 >= want),
                     n1 && (by_count ? bn + n0 + n1 >= want : bw + w0 + w1 >= want));
            __syncthreads();
            const uint32_t bin = s.found;
            if (bin == 0xffffffffu) {
                const uint64_t w = seen_w + s.d0;  // (the scan's total)
                __syncthreads();
                return Cut{low, 0xffffffffu, w, true};
            }
            __syncthreads();
            if (bin >> 1 == threadIdx.x) {
                s.hist.w[0] = bin & 1 ? bw + w0 : bw;
                s.hist.n[0] = (uint32_t)(bin & 1 ? bn + n0 : bn);
                s.hist.n[1] = bin & 1 ? n1 : n0;
            }
            __syncthreads();
            seen_w = s.hist.w[0];
            seen_n = s.hist.n[0];
            const uint32_t here = s.hist.n[1];
            __syncthreads();
            d0 += bin << shift;
            if (shift == 0) {
                const uint32_t key = top - d0;
                const uint64_t w = (uint64_t)__builtin_rint(weight_of(logit_of(key), md, f.c) * unit);
                uint64_t ties = by_count ? want - seen_n
                                         : (w ? (want - seen_w + w - 1) / w : here);
                ties = ties < 1 ? 1 : (ties < here ? ties : here);
                return Cut{key, (uint32_t)ties, seen_w + ties * w, false};
            }
            bits = shift;
            width = 1ull << bits;
        }
    }

    // Inclusive scan of 64-bit whole numbers over the threads; the total stays in s.d0.
    __device__ __forceinline__ uint64_t scan_u64(uint64_t x)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t lo = __shfl_up((uint32_t)x, d, 64), hi = __shfl_up((uint32_t)(x >> 32), d, 64);
            if (lane >= d)
                x += (uint64_t)hi << 32 | lo;
        }
        __syncthreads();
        uint64_t *red = reinterpret_cast<uint64_t *>(s.red);
        if (lane == 63)
            red[wave] = x;
        __syncthreads();
        uint64_t base = 0, t = 0;
#pragma unroll
        for (int w = 0; w < kPickWaves; ++w) {
            base = w == wave ? t : base;
            t += red[w];
        }
        if (threadIdx.x == 0)
            s.d0 = t;
        return base + x;
    }

    __device__ __forceinline__ Rule cut_by_digits(int n, float tau, double whole)
    {
        const uint32_t low = key_of(fmaxf(tau, -FLT_MAX));
        if (f.k) {  // the candidates' sum, for the fixed point's unit
            double sum = 0.;
            each_block(n, [&](int, const float(&z)[kE]) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < kE; ++e)
                    sum += key_of(z[e]) >= low ? weight_of(z[e], md, f.c) : 0.;
            });
            block_scan_64(sum, s.red, whole);
            __syncthreads();
        }
        // a power of two that brings the sum to 2^60 .. 2^61: weights lose 2^-61 of it each
        const double unit = fixed_unit(whole);
        Rule rule{low, 0xffffffffu, (double)f.q};
        double most = whole * unit;
        for (int by_count = f.k ? 1 : 0; by_count >= (f.p < 1.f ? 0 : 1); --by_count) {
            const uint64_t want = by_count ? (uint64_t)f.k : (uint64_t)__builtin_ceil((double)f.p * most);
            const Cut c = cut(n, low, by_count != 0, want, unit);
            most = (double)c.w;
            if (!c.all && (c.key > rule.key || (c.key == rule.key && c.ties < rule.ties)))
                rule = Rule{c.key, c.ties, (double)f.q};
        }
        return rule;
    }

    __device__ __forceinline__ void pick(const Stats &st)
    {
        // ---- the row's statistics; m, and the sum over all tokens
        constexpr int kOwn = (kMaxSpans + kPickThreads - 1) / kPickThreads;  // spans of a thread
        const int64_t first = row * st.spans;
        const int t = threadIdx.x;
        float own[kOwn], top = -INFINITY;
        double sum[kOwn];
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int sp = t + i * kPickThreads;
            own[i] = -INFINITY;
            sum[i] = 0.;
            if (sp < st.spans) {
                const u32x4_t x = ld16(st.maxima + (first + sp) * kSpanBlocks);
                if (f.k == 0)
                    sum[i] = st.sums[first + sp];
                *reinterpret_cast<u32x4_t *>(s.max + kSpanBlocks * sp) = x;
                own[i] = fmaxf(fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1])),
                               fmaxf(__uint_as_float(x[2]), __uint_as_float(x[3])));
                s.top[sp] = own[i];
                top = fmaxf(top, own[i]);
            }
        }
        top = wave_max_f(top);
        if ((t & 63) == 0)
            s.cnt[t >> 6] = __float_as_uint(top);
        __syncthreads();
        m = -INFINITY;
#pragma unroll
        for (int w = 0; w < kPickWaves; ++w)
            m = fmaxf(m, __uint_as_float(s.cnt[w]));
        md = m;
        __syncthreads();
        if (!(m > -INFINITY)) {  // every token is masked
            answer(-1, -INFINITY);
            return;
        }
        double whole = 0.;
        if (f.k == 0) {  // the spans' sums, brought to the row's maximum
            double x = 0.;
#pragma unroll
            for (int i = 0; i < kOwn; ++i)
                x += sum[i] > 0. ? sum[i] * weight_of(own[i], md, f.c) : 0.;
            block_scan_64(x, s.red, whole);
            __syncthreads();
        }
        float kth = -INFINITY;
        if (f.k && f.k <= st.spans)
            kth = st.spans <= kFewSpans ? kth_maximum<kFewSpans>(s.top, st.spans, f.k)
                                        : kth_maximum<kMaxSpans>(s.top, st.spans, f.k);
        if (f.k && f.k <= blocks && kth == -INFINITY)  // (of most spans every token may be masked)
            kth = kth_maximum<kMaxBlocks>(s.max, blocks, f.k);
        const float tau = bound(whole, kth);
        const int n_list = list_blocks(tau);
        if (f.k == 0 && f.p >= 1.f) {
            draw(n_list, Rule{0u, 0xffffffffu, (double)f.q});
            return;
        }
        if (f.k || n_list <= kFewBlocks) {
            const int n = collect(n_list, tau);
            if (n <= kSampleSort) {
                finish_sorted(n, whole);
                return;
            }
            __syncthreads();
        }
        if (f.k == 0 && finish_located(n_list, tau, whole))
            return;
        __syncthreads();
        draw(n_list, cut_by_digits(n_list, tau, whole));
    }

    // A float below a bound by more than the bound's own error (NaN: none).
    __device__ __forceinline__ float below(double x) const
    {
        x -= 1e-6 * (fabs(x) + fabs(md));
        return x == x ? fminf((float)x, m) : -INFINITY;
    }
};

// Rows without top-k, top-p and min-p: a wave each, with no barrier to wait at.
template <bool kBf16>
__global__ __launch_bounds__(64) void k_sample_plain(SampleArgs a, Stats st)
{
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        RowPicker<kBf16> p(a, row);
        p.simple(st);
    }
}

template <bool kBf16>
__global__ __launch_bounds__(kPickThreads) void k_sample_pick(SampleArgs a, Stats st)
{
    __shared__ PickLds s;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        Picker<kBf16> p(a, s, row);
        if (!p.f.filtered()) {
            if (threadIdx.x < 64)
                p.simple(st);
            continue;
        }
        p.pick(st);
        __syncthreads();  // the LDS is written again
    }
}

int sample_spans(int vocab, bool bf16)
{
    const int e = bf16 ? 8 : 4;
    return ((vocab + 2 * (e - 1)) / e + kSpanVecs - 1) / kSpanVecs;
}

}  // namespace

size_t sample_workspace(int64_t rows, int vocab, bool bf16)
{
    return (size_t)rows * sample_spans(vocab, bf16) * (sizeof(double) + kSpanBlocks * sizeof(float));
}

hipError_t launch_sample(const SampleArgs &a, void *workspace, hipStream_t stream)
{
    const int spans = sample_spans(a.vocab, a.bf16);
    const int64_t all = a.rows * spans;
    float *maxima = static_cast<float *>(workspace);  // (16-byte aligned, a span's four in one load)
    double *sums = reinterpret_cast<double *>(maxima + all * kSpanBlocks);
    const Stats st{sums, maxima, spans};
    // a wave for each span where they are few, else as many as keep the device full
    const int groups = (spans + kStatWaves - 1) / kStatWaves;
    const int64_t want = (kStatBlocks + a.rows - 1) / a.rows;
    const int per_row = (int)(want < groups ? want : groups);
    hipLaunchKernelGGL(a.bf16 ? k_sample_stats<true> : k_sample_stats<false>,
                       dim3(per_row, (unsigned)(a.rows < 65535 ? a.rows : 65535)), dim3(kStatThreads), 0,
                       stream, a, st);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    const int64_t blocks = a.rows < kSampleGrid ? a.rows : kSampleGrid;
    if (a.top_k || a.top_p || a.min_p)
        hipLaunchKernelGGL(a.bf16 ? k_sample_pick<true> : k_sample_pick<false>, dim3((unsigned)blocks),
                           dim3(kPickThreads), 0, stream, a, st);
    else
        hipLaunchKernelGGL(a.bf16 ? k_sample_plain<true> : k_sample_plain<false>, dim3((unsigned)blocks),
                           dim3(64), 0, stream, a, st);
    return hipGetLastError();
}

}  // namespace sparrow
