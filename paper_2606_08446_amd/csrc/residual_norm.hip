// What stands between two blocks of a layer, in one pass over the rows, and its gradient:
//
//   n = x r_x post_weight (x itself without a norm behind the block),  r_x = 1 / sqrt(mean(x^2) + eps)
//   h' = h + scale sigmoid(gate) n,  y = h' r weight,  r = 1 / sqrt(mean(h'^2) + eps)
//
// and with u = dy weight, k = h' r:
//   dh = dh_out + r (u - k mean(u k)),  dweight = sum dy k
//   d = scale dh,  dgate = d n s (1 - s),  e = d s  (s = sigmoid(gate))
//   dx = r_x (v - k_x mean(v k_x)),  v = e post_weight, k_x = x r_x,  dpost_weight = sum e k_x
//
// A workgroup owns a row and holds it in registers, up to kVecs 16-byte vectors of each array a
// thread; a row's sums are a wave's DPP scan and one exchange through LDS.
#include "residual_norm.h"

#include "common.h"
#include "wave.h"

namespace sparrow {
namespace {

constexpr int kNormMaxWaves = 16;
constexpr int kNormBlocks = 1 << 20;  // workgroups at most (a grid has fewer than 2^32 threads)

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

// 8 channels of the stream as they lie in memory.
template <bool kF32> struct Stream8;
template <> struct Stream8<false> {
    u32x4_t v;
    __device__ __forceinline__ void load(const void *p, int64_t i)
    {
        v = ld16_nt(static_cast<const uint16_t *>(p) + i);
    }
    __device__ __forceinline__ void get(float (&f)[8]) const { unpack8(v, f); }
    __device__ static __forceinline__ void store(void *p, int64_t i, const float (&f)[8])
    {
        st16(static_cast<uint16_t *>(p) + i, pack8(f));
    }
};
template <> struct Stream8<true> {
    u32x4_t v[2];
    __device__ __forceinline__ void load(const void *p, int64_t i)
    {
        v[0] = ld16_nt(static_cast<const float *>(p) + i);
        v[1] = ld16_nt(static_cast<const float *>(p) + i + 4);
    }
    __device__ __forceinline__ void get(float (&f)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            f[i] = __uint_as_float(v[i >> 2][i & 3]);
    }
    __device__ static __forceinline__ void store(void *p, int64_t i, const float (&f)[8])
    {
        float *q = static_cast<float *>(p) + i;
        st16(q, __builtin_bit_cast(u32x4_t, (f32x4_t){f[0], f[1], f[2], f[3]}));
        st16(q + 4, __builtin_bit_cast(u32x4_t, (f32x4_t){f[4], f[5], f[6], f[7]}));
    }
};

// Sums of kN values over the workgroup (every thread gets them); s has room for all waves.  A
// second call needs another s, or a barrier in between.
template <int kN>
__device__ __forceinline__ void block_sums(float (&x)[kN], float (*s)[kNormMaxWaves])
{
    const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < kN; ++i)
        x[i] = wave_sum_f(x[i]);
    if (waves == 1)
        return;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < kN; ++i)
            s[i][wave] = x[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        float t = 0.f;
        for (int w = 0; w < waves; ++w)
            t += s[i][w];
        x[i] = t;
    }
}

// 1 / (1 + e^-a): expf overflows to infinity far below zero, where the result is 0.
__device__ __forceinline__ float sigmoid(float a) { return 1.f / (1.f + expf(-a)); }

// y comes from h' before its rounding to the stream's type: the row is at hand, and a second
// rounding in front of the norm would only add its error.
template <int kVecs, bool kF32>
__global__ __launch_bounds__(1024) void k_residual_norm(NormArgs a, void *h_out, uint16_t *y)
{
    __shared__ float s_x[1][kNormMaxWaves], s_h[1][kNormMaxWaves];
    const int vecs = a.channels >> 3;
    const float inv_c = 1.f / (float)a.channels;
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        Stream8<kF32> hr[kVecs];
        u32x4_t xr[kVecs], gr[kVecs];
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            const int i = threadIdx.x + j * blockDim.x;
            if (i < vecs) {
                hr[j].load(a.h, t * a.channels + 8 * i);
                if (a.x)
                    xr[j] = ld16_nt(a.x + t * a.x_stride + 8 * i);
                if (a.gate)
                    gr[j] = ld16_nt(a.gate + t * a.gate_stride + 8 * i);
            }
        }
        float rx = 1.f;
        if (a.post) {
            float sum[1] = {0.f};
#pragma unroll
            for (int j = 0; j < kVecs; ++j)
                if (threadIdx.x + j * blockDim.x < (unsigned)vecs) {
                    float x[8];
                    unpack8(xr[j], x);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        sum[0] += x[e] * x[e];
                }
            block_sums(sum, s_x);
            rx = rsqrtf(sum[0] * inv_c + a.eps);
        }
        float h[kVecs][8], sum[1] = {0.f};
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            const int i = threadIdx.x + j * blockDim.x;
            if (i < vecs) {
                hr[j].get(h[j]);
                if (a.x) {
                    float x[8];
                    unpack8(xr[j], x);
                    if (a.post) {
                        float w[8];
                        unpack8(ld16(a.post + 8 * i), w);
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            x[e] *= rx * w[e];
                    }
                    if (a.gate) {
                        float g[8];
                        unpack8(gr[j], g);
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            x[e] *= sigmoid(g[e]);
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        h[j][e] += a.scale * x[e];
                    Stream8<kF32>::store(h_out, t * a.channels + 8 * i, h[j]);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    sum[0] += h[j][e] * h[j][e];
            }
        }
        block_sums(sum, s_h);
        const float r = rsqrtf(sum[0] * inv_c + a.eps);
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            const int i = threadIdx.x + j * blockDim.x;
            if (i < vecs) {
                float w[8];
                unpack8(ld16(a.weight + 8 * i), w);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    w[e] *= h[j][e] * r;
                st16(y + t * a.channels + 8 * i, pack8(w));
            }
        }
        if (t + gridDim.x < a.tokens)
            __syncthreads();  // the sums' LDS is written again
    }
}

// One row's arrays as they lie in memory.
template <int kVecs, bool kF32>
struct GradRow {
    Stream8<kF32> h[kVecs], dh[kVecs];
    u32x4_t dy[kVecs], x[kVecs], gate[kVecs];
    __device__ __forceinline__ void load(const NormArgs &a, const NormGradArgs &g, int64_t t)
    {
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            const int i = threadIdx.x + j * blockDim.x;
            if (i < a.channels >> 3) {
                h[j].load(a.h, t * a.channels + 8 * i);
                dy[j] = ld16_nt(g.dy + t * a.channels + 8 * i);
                if (g.dh_out)
                    dh[j].load(g.dh_out, t * a.channels + 8 * i);
                if (a.x)
                    x[j] = ld16_nt(a.x + t * a.x_stride + 8 * i);
                if (a.gate)
                    gate[j] = ld16_nt(a.gate + t * a.gate_stride + 8 * i);
            }
        }
    }
};

// A workgroup takes every gridDim.x-th row, the next row's loads under way, and keeps its channels'
// sums for the weights in registers; k_norm_dw adds the workgroups' up in a fixed order.
template <int kVecs, bool kF32>
__global__ __launch_bounds__(1024) void k_residual_norm_bwd(NormArgs a, NormGradArgs g)
{
    __shared__ float s_1[3][kNormMaxWaves], s_2[1][kNormMaxWaves];
    const int vecs = a.channels >> 3;
    const float inv_c = 1.f / (float)a.channels;
    float dw[kVecs][8] = {}, dp[kVecs][8] = {};
    GradRow<kVecs, kF32> next;
    next.load(a, g, blockIdx.x);
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        const GradRow<kVecs, kF32> row = next;
        if (t + gridDim.x < a.tokens)
            next.load(a, g, t + gridDim.x);
        // ---- sums of h'^2, u h' and x^2
        float sum[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            const int i = threadIdx.x + j * blockDim.x;
            if (i < vecs) {
                float h[8], d[8], w[8];
                row.h[j].get(h);
                unpack8(row.dy[j], d);
                unpack8(ld16(a.weight + 8 * i), w);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    sum[0] += h[e] * h[e];
                    sum[1] += d[e] * w[e] * h[e];
                }
                if (a.post) {
                    unpack8(row.x[j], h);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        sum[2] += h[e] * h[e];
                }
            }
        }
        block_sums(sum, s_1);
        const float r = rsqrtf(sum[0] * inv_c + a.eps);
        const float c = sum[1] * inv_c * r;  // mean(u k)
        const float rx = a.post ? rsqrtf(sum[2] * inv_c + a.eps) : 1.f;
        // ---- dh, dgate; what goes on to x stays in e
        float e_[kVecs][8], dot[1] = {0.f};
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            const int i = threadIdx.x + j * blockDim.x;
            if (i < vecs) {
                float h[8], d[8], w[8];
                row.h[j].get(h);
                unpack8(row.dy[j], d);
                unpack8(ld16(a.weight + 8 * i), w);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float k = h[e] * r;
                    dw[j][e] += d[e] * k;
                    d[e] = r * (d[e] * w[e] - k * c);
                }
                if (g.dh_out) {
                    row.dh[j].get(h);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        d[e] += h[e];
                }
                Stream8<kF32>::store(g.dh, t * a.channels + 8 * i, d);
                if (g.dx) {
                    float x[8], p[8];
                    if (a.x)
                        unpack8(row.x[j], x);
                    if (a.post)
                        unpack8(ld16(a.post + 8 * i), p);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        d[e] *= a.scale;
                        if (a.post)
                            x[e] *= rx;
                    }
                    if (a.gate) {
                        float q[8];
                        unpack8(row.gate[j], q);
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float s = sigmoid(q[e]);
                            const float n = a.post ? x[e] * p[e] : x[e];
                            // 1 - s as the other side's sigmoid: no cancellation near s = 1
                            q[e] = d[e] * n * s * sigmoid(-q[e]);
                            d[e] *= s;
                        }
                        st16(g.dgate + t * g.dgate_stride + 8 * i, pack8(q));
                    }
                    if (a.post) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            dp[j][e] += d[e] * x[e];
                            d[e] *= p[e];
                            dot[0] += d[e] * x[e];
                            e_[j][e] = d[e];
                        }
                    } else {
                        st16(g.dx + t * g.dx_stride + 8 * i, pack8(d));
                    }
                }
            }
        }
        if (a.post) {  // (the launcher gives post only with dx)
            block_sums(dot, s_2);
            const float m = dot[0] * inv_c;
#pragma unroll
            for (int j = 0; j < kVecs; ++j) {
                const int i = threadIdx.x + j * blockDim.x;
                if (i < vecs) {
                    float x[8];
                    unpack8(row.x[j], x);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[e] = rx * (e_[j][e] - x[e] * rx * m);
                    st16(g.dx + t * g.dx_stride + 8 * i, pack8(x));
                }
            }
        } else {
            __syncthreads();  // s_1 is written again
        }
    }
    const int parts = a.post ? 2 : 1;
    float *out = g.partials + (int64_t)blockIdx.x * parts * a.channels;
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
        const int i = threadIdx.x + j * blockDim.x;
        if (i < vecs) {
            Stream8<true>::store(out, 8 * i, dw[j]);
            if (a.post)
                Stream8<true>::store(out, a.channels + 8 * i, dp[j]);
        }
    }
}

// The weights' gradients from the workgroups' sums: 32 channels a workgroup, 32 threads a channel.
constexpr int kNormDwChannels = 32;
constexpr int kNormDwParts = 32;

__global__ __launch_bounds__(kNormDwChannels *kNormDwParts) void k_norm_dw(
    const float *partials, int blocks, int channels, int parts, float *dweight, float *dpost)
{
    __shared__ float s[kNormDwParts][kNormDwChannels];
    const int ch = threadIdx.x % kNormDwChannels, part = threadIdx.x / kNormDwChannels;
    const int i = blockIdx.x * kNormDwChannels + ch;  // over [parts][channels]
    const int all = parts * channels;
    float sum = 0.f;
    if (i < all)
        for (int b = part; b < blocks; b += kNormDwParts)
            sum += partials[(int64_t)b * all + i];
    s[part][ch] = sum;
    __syncthreads();
    if (part == 0 && i < all) {
        for (int p = 1; p < kNormDwParts; ++p)
            sum += s[p][ch];
        if (i < channels)
            dweight[i] = sum;
        else
            dpost[i - channels] = sum;
    }
}

// Threads of a row: one 16-byte vector of every array each, two beyond 1024 vectors.
int norm_vecs(int channels) { return channels / 8 > 1024 ? 2 : 1; }

int norm_threads(int channels)
{
    const int v = norm_vecs(channels);
    return (channels / 8 + 64 * v - 1) / (64 * v) * 64;
}

}  // namespace

int norm_grad_blocks(int64_t tokens, int channels)
{
    int64_t b = (1 << 18) / norm_threads(channels);
    b = b < 2048 ? b : 2048;
    return (int)(b < tokens ? b : tokens);
}

size_t norm_grad_workspace(int64_t tokens, int channels)
{
    return (size_t)norm_grad_blocks(tokens, channels) * 2 * channels * sizeof(float);
}

hipError_t launch_residual_norm(const NormArgs &a, void *h_out, uint16_t *y, hipStream_t stream)
{
    auto kernel = norm_vecs(a.channels) == 1
                      ? (a.f32 ? k_residual_norm<1, true> : k_residual_norm<1, false>)
                      : (a.f32 ? k_residual_norm<2, true> : k_residual_norm<2, false>);
    const int64_t blocks = a.tokens < kNormBlocks ? a.tokens : kNormBlocks;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(norm_threads(a.channels)), 0, stream, a,
                       h_out, y);
    return hipGetLastError();
}

hipError_t launch_residual_norm_bwd(const NormArgs &a, const NormGradArgs &g, hipStream_t stream)
{
    const int blocks = norm_grad_blocks(a.tokens, a.channels);
    auto kernel = norm_vecs(a.channels) == 1
                      ? (a.f32 ? k_residual_norm_bwd<1, true> : k_residual_norm_bwd<1, false>)
                      : (a.f32 ? k_residual_norm_bwd<2, true> : k_residual_norm_bwd<2, false>);
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(norm_threads(a.channels)), 0, stream, a, g);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    const int parts = a.post ? 2 : 1;
    hipLaunchKernelGGL(k_norm_dw, dim3((parts * a.channels + kNormDwChannels - 1) / kNormDwChannels),
                       dim3(kNormDwChannels * kNormDwParts), 0, stream, g.partials, blocks,
                       a.channels, parts, g.dweight, g.dpost);
    return hipGetLastError();
}

}  // namespace sparrow
