// RMS norm of every query and key head with its weight, and the position rotation, in one pass
// over the rows; and the gradient of both.
//
//   r = 1 / sqrt(mean(x^2) + eps),  n = x r w                       (128 channels of a head)
//   a_i = position * inv_freq_i,  y_i = n_i cos a_i - n_{i+64} sin a_i,
//                                 y_{i+64} = n_{i+64} cos a_i + n_i sin a_i
// and with g = the rotation of dy by -a, u = g w:
//   dx = r (u - x r mean(u x r)),  dw = sum over the rows of g x r.
//
// 8 lanes own a row: lane l holds channels 8l .. 8l+7 and 64+8l .. 64+8l+7, both halves of its 8
// rotated pairs, in two 16-byte vectors, so a wave takes 8 rows (heads of one token) per pass and
// the row sums are three DPP steps.  A token's 64 angles are computed once per wave, one per
// lane: p * inv_freq / 2pi is reduced in fp64, which keeps full fp32 precision of the angle at any int32
// position, and its sine and cosine are as exact (the weights' gradients are fp32 outputs).
// Bound by HBM: 512 B per row for ~10 flops an element, 768 B for ~30 in the gradient.  64K tokens of
// 32 + 8 heads (1.39 GB) take 229 us, 6.1 TB/s; the gradient of 32K tokens (1.01 GB) 171 us, 5.9
// (a plain copy reaches 4.8 TB/s, a sum of two arrays 6.0).
#include "qk_norm_rope.h"

#include "common.h"

namespace sparrow {
namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeWaves = kRopeThreads / 64;
constexpr int kRopeBlocks = 1 << 20;  // workgroups at most
constexpr int kRows = 8;          // rows per wave and pass
constexpr int kHalf = kHeadDim / 2;
constexpr double kInvTwoPi = 0.15915494309189533577;

// DPP controls: lane ^ 1, lane ^ 2 inside a quad; the mirror image inside 8 lanes.
constexpr int kDppXor1 = 0xb1;
constexpr int kDppXor2 = 0x4e;
constexpr int kDppHalfMirror = 0x141;

template <int kCtrl>
__device__ __forceinline__ float dpp_f(float x)
{
    return __int_as_float(
        __builtin_amdgcn_update_dpp(0, __float_as_int(x), kCtrl, 0xf, 0xf, true));
}

// Sum over each 8 lanes (every lane gets it, the same bits).
__device__ __forceinline__ float sum8(float x)
{
    x += dpp_f<kDppXor1>(x);
    x += dpp_f<kDppXor2>(x);
    x += dpp_f<kDppHalfMirror>(x);
    return x;
}

// Sum over the lanes l, l + 8, ... l + 56 (every lane gets it): a rotation by 8 inside each 16, then
// swaps of 16-lane rows and of halves with a copy, which leave a lane its own and its partner's.
__device__ __forceinline__ float sum_rows(float x)
{
    constexpr int kRor8 = 0x128;
    x += dpp_f<kRor8>(x);
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

__device__ __forceinline__ void unpack8(u32x4_t v, float (&f)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = bf16_lo(v[i]);
        f[2 * i + 1] = bf16_hi(v[i]);
    }
}

__device__ __forceinline__ u32x4_t pack8(const float (&f)[8])
{
    return (u32x4_t){pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]),
                     pack_bf16(f[6], f[7])};
}

// Both halves of a row, as one lane holds them.
struct Row {
    u32x4_t lo, hi;
    __device__ __forceinline__ void load(const uint16_t *p, int l)
    {
        lo = ld16_nt(p + 8 * l);
        hi = ld16_nt(p + kHalf + 8 * l);
    }
    template <bool kStream>
    __device__ __forceinline__ void store(uint16_t *p, int l) const
    {
        if (kStream) {
            __builtin_nontemporal_store(lo, reinterpret_cast<u32x4_t *>(p + 8 * l));
            __builtin_nontemporal_store(hi, reinterpret_cast<u32x4_t *>(p + kHalf + 8 * l));
        } else {
            st16(p + 8 * l, lo);
            st16(p + kHalf + 8 * l, hi);
        }
    }
};

// Sine and cosine of a turn: its whole quarters turn the result, and what is left, at most pi / 4
// either way, goes to fp32 in one rounding and through the Taylor series (their next terms are below
// 2^-29).  Off by at most 2^-23.4 (2^-23.8 measured; an instruction each on the fp32 turn over 2^-23.1).
__device__ __forceinline__ void sincos_turn(double turns, float &sine, float &cosine)
{
    constexpr double kHalfPi = 1.57079632679489661923;
    const double quarters = 4. * (turns - __builtin_rint(turns)), n = __builtin_rint(quarters);
    const float x = (float)((quarters - n) * kHalfPi), x2 = x * x;
    const float s = x + x * x2 * (-1.f / 6 + x2 * (1.f / 120 + x2 * (-1.f / 5040 + x2 * (1.f / 362880))));
    const float c = 1.f + x2 * (-1.f / 2 + x2 * (1.f / 24 + x2 * (-1.f / 720 + x2 * (1.f / 40320 + x2 *
                                                                                  (-1.f / 3628800)))));
    const int k = (int)n;  // -2 .. 2
    sine = k & 1 ? c : s;
    cosine = k & 1 ? s : c;
    sine = k & 2 ? -sine : sine;
    cosine = (k + 1) & 2 ? -cosine : cosine;
}

// Cosines and sines of a token's angles 8l .. 8l+7: lane 8j + l computes number 8l + j.
__device__ __forceinline__ void angles(double inv_freq, int pos, int lane, float (&c)[8],
                                       float (&s)[8])
{
    float cv, sv;
    sincos_turn((double)pos * (inv_freq * kInvTwoPi), sv, cv);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        c[j] = __shfl(cv, 8 * j + (lane & 7), 64);
        s[j] = __shfl(sv, 8 * j + (lane & 7), 64);
    }
}

// 1 / sqrt(mean(x^2) + eps) of a row.
__device__ __forceinline__ float inv_rms(const float (&x0)[8], const float (&x1)[8], float eps)
{
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        ss += x0[i] * x0[i] + x1[i] * x1[i];
    return rsqrtf(sum8(ss) * (1.f / kHeadDim) + eps);
}

// The workgroup's place among `n`, counted so that each of the 8 XCDs, which take workgroups in turn,
// works on 128 neighbours out of every 1024.  (In the order of launch -> this, us in a graph, both in turn
// on two boxes: 64K tokens of 32 + 8 heads 234.4 -> 229.2, 128K of 16 + 8 279 -> 270, 32K of 40 + 8 135.6
// -> 134.0, 4K of 32 + 8 17.7 -> 17.5; two builds of the same code differ by 0.3 % at most.  With 512
// neighbours, or an eighth of all, the first three were 237, 279 and 140.)
constexpr int kXcds = 8, kXcdRun = 128;

__device__ __forceinline__ int place_by_xcd(int block, int n)
{
    constexpr int kWindow = kXcds * kXcdRun;
    const int first = block / kWindow * kWindow, r = block - first;
    return first + kWindow > n ? block : first + r % kXcds * kXcdRun + r / kXcds;
}

// A wave takes one pass (8 query rows, or 8 key rows) of one token at a time.
template <bool kStream>
__global__ __launch_bounds__(kRopeThreads) void k_qk_norm_rope(RopeArgs a, uint16_t *q_out,
                                                               uint16_t *k_out)
{
    const int lane = threadIdx.x & 63;
    const int l = lane & 7;
    const int q_passes = (a.num_q_heads + kRows - 1) / kRows;
    const int passes = q_passes + (a.num_k_heads + kRows - 1) / kRows;
    const double inv_freq = a.inv_freq[8 * l + (lane >> 3)];
    const int64_t all = a.tokens * passes;
    for (int64_t w = (int64_t)place_by_xcd(blockIdx.x, gridDim.x) * kRopeWaves +
                     __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
         w < all; w += (int64_t)gridDim.x * kRopeWaves) {
        const int64_t t = w / passes;
        const int pass = (int)(w - t * passes);
        const bool is_q = pass < q_passes;
        const int heads = is_q ? a.num_q_heads : a.num_k_heads;
        const int h = (is_q ? pass : pass - q_passes) * kRows + (lane >> 3);
        const bool live = h < heads;
        const int pos = a.positions[t];
        if (pos < 0)
            continue;
        Row x = {}, w2;
        if (live)
            x.load((is_q ? a.q + t * a.q_stride : a.k + t * a.k_stride) + h * kHeadDim, l);
        const uint16_t *wt = is_q ? a.q_weight : a.k_weight;
        w2.lo = ld16(wt + 8 * l);
        w2.hi = ld16(wt + kHalf + 8 * l);
        float c[8], s[8];
        angles(inv_freq, pos, lane, c, s);

        float x0[8], x1[8], w0[8], w1[8];
        unpack8(x.lo, x0);
        unpack8(x.hi, x1);
        unpack8(w2.lo, w0);
        unpack8(w2.hi, w1);
        const float r = inv_rms(x0, x1, a.eps);
        float y0[8], y1[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float n0 = x0[i] * r * w0[i], n1 = x1[i] * r * w1[i];
            y0[i] = n0 * c[i] - n1 * s[i];
            y1[i] = n1 * c[i] + n0 * s[i];
        }
        if (live) {
            const Row y = {pack8(y0), pack8(y1)};
            y.store<kStream>((is_q ? q_out : k_out) + (t * heads + h) * kHeadDim, l);
        }
    }
}

// One pass of the gradient: dx of 8 rows into d, and the rows' parts of dw added to dw0, dw1.
__device__ __forceinline__ void grad_rows(const Row &xr, Row &d, float eps, const Row &w,
                                          const float (&c)[8], const float (&s)[8],
                                          float (&dw0)[8], float (&dw1)[8])
{
    float x0[8], x1[8], d0[8], d1[8], w0[8], w1[8];
    unpack8(xr.lo, x0);
    unpack8(xr.hi, x1);
    unpack8(d.lo, d0);
    unpack8(d.hi, d1);
    unpack8(w.lo, w0);
    unpack8(w.hi, w1);
    const float r = inv_rms(x0, x1, eps);
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float g0 = d0[i] * c[i] + d1[i] * s[i], g1 = d1[i] * c[i] - d0[i] * s[i];
        x0[i] *= r;
        x1[i] *= r;
        dw0[i] += g0 * x0[i];
        dw1[i] += g1 * x1[i];
        d0[i] = g0 * w0[i];
        d1[i] = g1 * w1[i];
        dot += d0[i] * x0[i] + d1[i] * x1[i];
    }
    dot = sum8(dot) * (1.f / kHeadDim);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        d0[i] = r * (d0[i] - x0[i] * dot);
        d1[i] = r * (d1[i] - x1[i] * dot);
    }
    d.lo = pack8(d0);
    d.hi = pack8(d1);
}

// What a wave works through: the passes of a token one after another, then those of the token `waves`
// further on, so that neighbouring waves read neighbouring rows.  Where there are more waves than
// tokens a token's passes are shared out: run u is token u / runs, passes [r passes / runs, (r + 1)
// passes / runs) with r = u % runs, and a wave takes the runs w, w + waves, ...  `runs` is a whole
// number, so that up to twice as many waves as tokens leave some without work: 1014 tokens of 40 + 8
// heads are five passes in a row for 1014 of the query side's 1704 waves, where an even split is three.
struct Walk {
    int64_t u, t;
    int pass, stop, runs;
    bool more, fresh;  // there is a pass; it is the first of its token here

    __device__ __forceinline__ void place(int64_t tokens, int passes)
    {
        t = u / runs;
        const int r = (int)(u - t * runs);
        pass = r * passes / runs;
        stop = (r + 1) * passes / runs;
        more = t < tokens;
        fresh = true;
    }
    __device__ __forceinline__ void start(int64_t w, int64_t waves, int64_t tokens, int passes)
    {
        const int64_t share = waves / (tokens > 0 ? tokens : 1);
        runs = share < 1 ? 1 : (share < passes ? (int)share : passes);
        u = w;
        place(tokens, passes);
    }
    __device__ __forceinline__ void step(int64_t waves, int64_t tokens, int passes)
    {
        fresh = false;
        if (++pass == stop) {
            u += waves;
            place(tokens, passes);
        }
    }
};

// Workgroups [0, q_blocks) take the query heads, the others the key heads, so that a wave keeps one
// weight's gradient.  The workgroups' sums go to `partials` and are added in a fixed order by
// k_rope_dw, so that results do not depend on which workgroup ends first.
template <bool kStream>
__global__ __launch_bounds__(kRopeThreads) void k_qk_norm_rope_bwd(RopeArgs a, RopeGradArgs g,
                                                                   int q_blocks)
{
    __shared__ float s_dw[kRopeWaves * kHeadDim];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l = lane & 7;
    const bool is_q = (int)blockIdx.x < q_blocks;
    const int heads = is_q ? a.num_q_heads : a.num_k_heads;
    const uint16_t *x = is_q ? a.q : a.k;
    const uint16_t *dy = is_q ? g.dq_out : g.dk_out;
    uint16_t *dx = is_q ? g.dq : g.dk;
    const int64_t x_stride = is_q ? a.q_stride : a.k_stride;
    const int64_t dx_stride = is_q ? g.dq_stride : g.dk_stride;
    const uint16_t *weight = is_q ? a.q_weight : a.k_weight;
    const int passes = (heads + kRows - 1) / kRows;
    const int64_t waves = (int64_t)(is_q ? q_blocks : gridDim.x - q_blocks) * kRopeWaves;
    const int64_t w = (int64_t)(blockIdx.x - (is_q ? 0 : q_blocks)) * kRopeWaves + wave;
    Walk k;
    k.start(w, waves, a.tokens, passes);

    const double inv_freq = a.inv_freq[8 * l + (lane >> 3)];
    Row wt;
    wt.lo = ld16(weight + 8 * l);
    wt.hi = ld16(weight + kHalf + 8 * l);
    float dw0[8] = {}, dw1[8] = {}, c[8], s[8];
    Row xr = {}, d = {};
    int pos = 0;
    auto load = [&]() __attribute__((always_inline)) {
        const int h = k.pass * kRows + (lane >> 3);
        if (k.fresh)
            pos = a.positions[k.t];
        if (h < heads) {
            xr.load(x + k.t * x_stride + h * kHeadDim, l);
            d.load(dy + (k.t * heads + h) * kHeadDim, l);
        }
    };
    if (k.more)
        load();
    while (k.more) {
        const int64_t t = k.t;
        const bool fresh = k.fresh;
        const int h = k.pass * kRows + (lane >> 3), pos_now = pos;
        const Row x_now = xr;
        Row d_now = d;
        k.step(waves, a.tokens, passes);
        if (k.more)
            load();
        if (fresh)
            angles(inv_freq, pos_now, lane, c, s);
        if (h < heads) {  // (all 8 lanes of a row)
            if (pos_now < 0)
                d_now.lo = d_now.hi = (u32x4_t){0u, 0u, 0u, 0u};
            else
                grad_rows(x_now, d_now, a.eps, wt, c, s, dw0, dw1);
            d_now.store<kStream>(dx + t * dx_stride + h * kHeadDim, l);
        }
    }

    // ---- the wave's sums over its 8 rows, the workgroup's over its waves
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        dw0[i] = sum_rows(dw0[i]);
        dw1[i] = sum_rows(dw1[i]);
    }
    if (lane < 8)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s_dw[wave * kHeadDim + 8 * lane + i] = dw0[i];
            s_dw[wave * kHeadDim + kHalf + 8 * lane + i] = dw1[i];
        }
    __syncthreads();
    if (threadIdx.x < kHeadDim) {
        float v = 0.f;
        for (int k = 0; k < kRopeWaves; ++k)
            v += s_dw[k * kHeadDim + threadIdx.x];
        g.partials[(int64_t)blockIdx.x * kHeadDim + threadIdx.x] = v;
    }
}

// dw from the workgroups' sums: 8 channels a workgroup, 128 threads a channel with their loads all
// under way at once.
constexpr int kDwThreads = 1024;
constexpr int kDwChannels = 8;
constexpr int kDwParts = kDwThreads / kDwChannels;
constexpr int kDwLoads = kRopeGradBlocks / kDwParts;

__global__ __launch_bounds__(kDwThreads) void k_rope_dw(const float *partials, int q_blocks,
                                                        int blocks, float *dq_weight,
                                                        float *dk_weight)
{
    __shared__ float s_sum[kDwParts][kDwChannels];
    constexpr int kGroups = kHeadDim / kDwChannels;  // workgroups per weight
    const bool is_q = blockIdx.x < kGroups;
    const int ch = threadIdx.x % kDwChannels, part = threadIdx.x / kDwChannels;
    const int i = (is_q ? blockIdx.x : blockIdx.x - kGroups) * kDwChannels + ch;
    const int b0 = is_q ? 0 : q_blocks, b1 = is_q ? q_blocks : blocks;
    float v[kDwLoads];
#pragma unroll
    for (int k = 0; k < kDwLoads; ++k) {
        const int b = b0 + part + k * kDwParts;
        v[k] = b < b1 ? partials[(int64_t)b * kHeadDim + i] : 0.f;
    }
#pragma unroll
    for (int k = 1; k < kDwLoads; ++k)
        v[0] += v[k];
    s_sum[part][ch] = v[0];
    __syncthreads();
    if (threadIdx.x < 64) {
        float sum = 0.f;
        for (int p = part; p < kDwParts; p += 8)
            sum += s_sum[p][ch];
#pragma unroll
        for (int m = 8; m < 64; m <<= 1)
            sum += __shfl_xor(sum, m, 64);
        if (part == 0)
            (is_q ? dq_weight : dk_weight)[i] = sum;
    }
}

// Whether a call's rows are written past the caches.  That is faster where they would not stay in the
// 256 MB memory-side cache anyway, and takes them from the kernel that reads them where they
// would: 32 + 8 heads, this kernel / with a copy of q_out behind it, us, plain -> streamed stores:
// 168 MB of rows 54 / 92 -> 56 / 103, 252 MB 79 / 167 -> 84 / 161, 671 MB 234 / 440 -> 223 / 433.
bool stream_rows(const RopeArgs &a)
{
    return a.tokens * (a.num_q_heads + a.num_k_heads) * (int64_t)(kHeadDim * 2) >= 224 << 20;
}

}  // namespace

hipError_t launch_qk_norm_rope(const RopeArgs &a, uint16_t *q_out, uint16_t *k_out,
                               hipStream_t stream)
{
    const int64_t passes = (a.num_q_heads + kRows - 1) / kRows + (a.num_k_heads + kRows - 1) / kRows;
    int64_t blocks = (a.tokens * passes + kRopeWaves - 1) / kRopeWaves;
    blocks = blocks < kRopeBlocks ? blocks : kRopeBlocks;
    auto kernel = stream_rows(a) ? k_qk_norm_rope<true> : k_qk_norm_rope<false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kRopeThreads), 0, stream, a, q_out,
                       k_out);
    return hipGetLastError();
}

hipError_t launch_qk_norm_rope_bwd(const RopeArgs &a, const RopeGradArgs &g, hipStream_t stream)
{
    // workgroups in proportion to the two sides' items, at least one each
    const int64_t qp = (a.num_q_heads + kRows - 1) / kRows, kp = (a.num_k_heads + kRows - 1) / kRows;
    const int64_t want = (a.tokens * (qp + kp) + kRopeWaves - 1) / kRopeWaves;
    const int blocks = (int)(want < 2 ? 2 : (want < kRopeGradBlocks ? want : kRopeGradBlocks));
    int q_blocks = (int)(blocks * qp / (qp + kp));
    q_blocks = q_blocks < 1 ? 1 : (q_blocks > blocks - 1 ? blocks - 1 : q_blocks);
    auto kernel = stream_rows(a) ? k_qk_norm_rope_bwd<true> : k_qk_norm_rope_bwd<false>;
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kRopeThreads), 0, stream, a, g, q_blocks);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(k_rope_dw, dim3(2 * kHeadDim / kDwChannels), dim3(kDwThreads), 0, stream,
                       g.partials, q_blocks, blocks, g.dq_weight, g.dk_weight);
    return hipGetLastError();
}

}  // namespace sparrow
