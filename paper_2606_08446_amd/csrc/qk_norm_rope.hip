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
// lane, in fp64: p * inv_freq / 2pi less its nearest integer keeps full fp32 precision of the
// turn at any int32 position.
// Bound by HBM: 512 B per row for ~10 flops an element.
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
    __device__ __forceinline__ void store(uint16_t *p, int l) const
    {
        st16(p + 8 * l, lo);
        st16(p + kHalf + 8 * l, hi);
    }
};

// Cosines and sines of a token's angles 8l .. 8l+7: lane 8j + l computes number 8l + j.
__device__ __forceinline__ void angles(double inv_freq, int pos, int lane, float (&c)[8],
                                       float (&s)[8])
{
    const double turns = (double)pos * (inv_freq * kInvTwoPi);
    const float t = (float)(turns - __builtin_rint(turns));
    float sv, cv;
    sincospif(2.f * t, &sv, &cv);
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

// A wave takes one pass (8 query rows, or 8 key rows) of one token at a time.
__global__ __launch_bounds__(kRopeThreads) void k_qk_norm_rope(RopeArgs a, uint16_t *q_out,
                                                               uint16_t *k_out)
{
    const int lane = threadIdx.x & 63;
    const int l = lane & 7;
    const int q_passes = (a.num_q_heads + kRows - 1) / kRows;
    const int passes = q_passes + (a.num_k_heads + kRows - 1) / kRows;
    const double inv_freq = a.inv_freq[8 * l + (lane >> 3)];
    const int64_t all = a.tokens * passes;
    for (int64_t w = (int64_t)blockIdx.x * kRopeWaves +
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
            y.store((is_q ? q_out : k_out) + (t * heads + h) * kHeadDim, l);
        }
    }
}

// One pass of the gradient: dx of 8 rows, and the rows' parts of dw added to dw0, dw1.
__device__ __forceinline__ void grad_rows(const uint16_t *dy, const uint16_t *x, uint16_t *dx,
                                          int h, int heads, bool skip, int l, float eps,
                                          const Row &w, const float (&c)[8], const float (&s)[8],
                                          float (&dw0)[8], float (&dw1)[8])
{
    if (h >= heads)
        return;  // (all 8 lanes of the row)
    Row d;
    if (skip) {
        d.lo = d.hi = (u32x4_t){0u, 0u, 0u, 0u};
        d.store(dx + h * kHeadDim, l);
        return;
    }
    Row xr;
    xr.load(x + h * kHeadDim, l);
    d.load(dy + h * kHeadDim, l);
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
    d.store(dx + h * kHeadDim, l);
}

// The wave's sums over its 8 rows and the workgroup's over its waves: 128 floats at `out`.
__device__ void block_dw(float (&dw0)[8], float (&dw1)[8], float *s_dw, int lane, int wave,
                         float *out)
{
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int m = 8; m < 64; m <<= 1) {
            dw0[i] += __shfl_xor(dw0[i], m, 64);
            dw1[i] += __shfl_xor(dw1[i], m, 64);
        }
    __syncthreads();  // s_dw is free
    if (lane < 8)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s_dw[wave * kHeadDim + 8 * lane + i] = dw0[i];
            s_dw[wave * kHeadDim + kHalf + 8 * lane + i] = dw1[i];
        }
    __syncthreads();
    if (threadIdx.x < kHeadDim) {
        float v = 0.f;
        for (int w = 0; w < kRopeWaves; ++w)
            v += s_dw[w * kHeadDim + threadIdx.x];
        out[threadIdx.x] = v;
    }
}

// A wave walks over tokens with all their heads and keeps the weights' gradients in registers;
// the workgroups' sums go to `partials` and are added in a fixed order by k_rope_dw, so that
// results do not depend on which workgroup ends first.
__global__ __launch_bounds__(kRopeThreads) void k_qk_norm_rope_bwd(RopeArgs a, RopeGradArgs g)
{
    __shared__ float s_dw[kRopeWaves * kHeadDim];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l = lane & 7;
    const double inv_freq = a.inv_freq[8 * l + (lane >> 3)];
    Row wq, wk;
    wq.lo = ld16(a.q_weight + 8 * l);
    wq.hi = ld16(a.q_weight + kHalf + 8 * l);
    wk.lo = ld16(a.k_weight + 8 * l);
    wk.hi = ld16(a.k_weight + kHalf + 8 * l);
    float q0[8] = {}, q1[8] = {}, k0[8] = {}, k1[8] = {};
    for (int64_t t = (int64_t)blockIdx.x * kRopeWaves + wave; t < a.tokens;
         t += (int64_t)gridDim.x * kRopeWaves) {
        const int pos = a.positions[t];
        const bool skip = pos < 0;
        float c[8], s[8];
        angles(inv_freq, pos, lane, c, s);
        for (int h = lane >> 3; h - (lane >> 3) < a.num_q_heads; h += kRows)
            grad_rows(g.dq_out + t * a.num_q_heads * kHeadDim, a.q + t * a.q_stride,
                      g.dq + t * g.dq_stride, h, a.num_q_heads, skip, l, a.eps, wq, c, s, q0, q1);
        for (int h = lane >> 3; h - (lane >> 3) < a.num_k_heads; h += kRows)
            grad_rows(g.dk_out + t * a.num_k_heads * kHeadDim, a.k + t * a.k_stride,
                      g.dk + t * g.dk_stride, h, a.num_k_heads, skip, l, a.eps, wk, c, s, k0, k1);
    }
    float *out = g.partials + (int64_t)blockIdx.x * 2 * kHeadDim;
    block_dw(q0, q1, s_dw, lane, wave, out);
    block_dw(k0, k1, s_dw, lane, wave, out + kHeadDim);
}

// dw from the workgroups' sums: 8 channels a workgroup, 32 threads a channel.
constexpr int kDwChannels = 8;
constexpr int kDwParts = kRopeThreads / kDwChannels;

__global__ __launch_bounds__(kRopeThreads) void k_rope_dw(const float *partials, int blocks,
                                                          float *dq_weight, float *dk_weight)
{
    __shared__ float s_sum[kDwParts][kDwChannels];
    const int ch = threadIdx.x % kDwChannels, part = threadIdx.x / kDwChannels;
    const int i = blockIdx.x * kDwChannels + ch;  // of the two weights' 256
    float v = 0.f;
    for (int b = part; b < blocks; b += kDwParts)
        v += partials[(int64_t)b * 2 * kHeadDim + i];
    s_sum[part][ch] = v;
    __syncthreads();
    if (part == 0) {
        for (int p = 1; p < kDwParts; ++p)
            v += s_sum[p][ch];
        (i < kHeadDim ? dq_weight : dk_weight)[i & (kHeadDim - 1)] = v;
    }
}

}  // namespace

hipError_t launch_qk_norm_rope(const RopeArgs &a, uint16_t *q_out, uint16_t *k_out,
                               hipStream_t stream)
{
    const int64_t passes = (a.num_q_heads + kRows - 1) / kRows + (a.num_k_heads + kRows - 1) / kRows;
    int64_t blocks = (a.tokens * passes + kRopeWaves - 1) / kRopeWaves;
    blocks = blocks < kRopeBlocks ? blocks : kRopeBlocks;
    hipLaunchKernelGGL(k_qk_norm_rope, dim3((unsigned)blocks), dim3(kRopeThreads), 0, stream, a,
                       q_out, k_out);
    return hipGetLastError();
}

hipError_t launch_qk_norm_rope_bwd(const RopeArgs &a, const RopeGradArgs &g, hipStream_t stream)
{
    const int64_t want = (a.tokens + kRopeWaves - 1) / kRopeWaves;
    const int blocks = (int)(want < kRopeGradBlocks ? want : kRopeGradBlocks);
    if (blocks > 0) {
        hipLaunchKernelGGL(k_qk_norm_rope_bwd, dim3(blocks), dim3(kRopeThreads), 0, stream, a, g);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    hipLaunchKernelGGL(k_rope_dw, dim3(2 * kHeadDim / kDwChannels), dim3(kRopeThreads), 0, stream,
                       g.partials, blocks, g.dq_weight, g.dk_weight);
    return hipGetLastError();
}

}  // namespace sparrow
