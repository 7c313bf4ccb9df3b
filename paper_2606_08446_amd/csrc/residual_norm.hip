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
// thread; a row's sums are a wave's DPP scan and one exchange through LDS.  Both directions are bound by
// memory, every operand being read and every result written once (bf16, gate and both norms, 32768 rows of
// 4096: 10 bytes a channel forward in 217 us, 6.2 TB/s, 16 bytes backward in 397 us, 5.4 TB/s; a kernel that only
// moves as much takes 213 and 343 us, and the latter 380 where each of 512 workgroups moves 64 rows, as here).
#include "residual_norm.h"

#include "common.h"
#include "wave.h"

#include <type_traits>

namespace sparrow {
namespace {

constexpr int64_t kPastCaches = 224 << 20;  // bytes of results that the caches do not keep for a reader
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

// The place of a row's i-th 16 bytes of bf16: one 32-bit offset for every array, whose rows' starts the whole
// workgroup shares in scalar registers.  (Opaque to the compiler, which would keep a pointer for each.)
__device__ __forceinline__ uint32_t place_of(int i)
{
    uint32_t bytes = 16u * (uint32_t)i;
    asm("" : "+v"(bytes));
    return bytes;
}

template <typename T>
__device__ __forceinline__ T *in_row(T *base, int64_t row, uint32_t bytes)
{
    using Bytes = std::conditional_t<std::is_const_v<T>, const char, char>;
    return reinterpret_cast<T *>(reinterpret_cast<Bytes *>(base + row) + bytes);
}

// 16 bytes of a result, past the caches or not.
template <bool kNt>
__device__ __forceinline__ void put16(void *p, u32x4_t v)
{
    if (kNt)
        __builtin_nontemporal_store(v, reinterpret_cast<u32x4_t *>(p));
    else
        st16(p, v);
}

// 8 channels of the stream as they lie in memory, those at a place of a row that starts at `row`.
template <bool kF32> struct Stream8;
template <> struct Stream8<false> {
    u32x4_t v;
    __device__ __forceinline__ void load(const void *p, int64_t row, uint32_t place)
    {
        v = ld16_nt(in_row(static_cast<const uint16_t *>(p), row, place));
    }
    __device__ __forceinline__ void get(float (&f)[8]) const { unpack8(v, f); }
    __device__ __forceinline__ void arrive() const { asm volatile("" ::"v"(v)); }  // (waits for the load)
    template <bool kNt>
    __device__ static __forceinline__ void store(void *p, int64_t row, uint32_t place, const float (&f)[8])
    {
        put16<kNt>(in_row(static_cast<uint16_t *>(p), row, place), pack8(f));
    }
};
template <> struct Stream8<true> {
    u32x4_t v[2];
    __device__ __forceinline__ void load(const void *p, int64_t row, uint32_t place)
    {
        const float *q = in_row(static_cast<const float *>(p), row, 2 * place);
        v[0] = ld16_nt(q);
        v[1] = ld16_nt(q + 4);
    }
    __device__ __forceinline__ void get(float (&f)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            f[i] = __uint_as_float(v[i >> 2][i & 3]);
    }
    __device__ __forceinline__ void arrive() const { asm volatile("" ::"v"(v[0]), "v"(v[1])); }
    template <bool kNt>
    __device__ static __forceinline__ void store(void *p, int64_t row, uint32_t place, const float (&f)[8])
    {
        float *q = in_row(static_cast<float *>(p), row, 2 * place);
        put16<kNt>(q, __builtin_bit_cast(u32x4_t, (f32x4_t){f[0], f[1], f[2], f[3]}));
        put16<kNt>(q + 4, __builtin_bit_cast(u32x4_t, (f32x4_t){f[4], f[5], f[6], f[7]}));
    }
};

// Sums of kN values over the workgroup (every thread gets them), in the order of its waves; s has room for
// kWaves and is zero where there are fewer.  A second call needs another s, or a barrier in between.
template <int kWaves, int kN>
__device__ __forceinline__ void block_sums(float (&x)[kN], float (*s)[kN])
{
#pragma unroll
    for (int i = 0; i < kN; ++i)
        x[i] = wave_sum_f(x[i]);
    if (blockDim.x == 64)
        return;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < kN; ++i)
            s[threadIdx.x >> 6][i] = x[i];
    __syncthreads();
    float t[kWaves][kN];
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
#pragma unroll
        for (int i = 0; i < kN; ++i)
            t[w][i] = s[w][i];
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        x[i] = t[0][i];
#pragma unroll
        for (int w = 1; w < kWaves; ++w)
            x[i] += t[w][i];
    }
}

template <int kWaves, int kN>
__device__ __forceinline__ void clear_sums(float (*s)[kN])
{
    if (threadIdx.x < kWaves)
#pragma unroll
        for (int i = 0; i < kN; ++i)
            s[threadIdx.x][i] = 0.f;
}

// sigmoid(a) and its slope s (1 - s) without cancellation or overflow: with e = e^-|a|, r = 1 / (1 + e) they
// are r or e r, and e r^2.  log2(e) is taken in two parts, since the rounding of a log2(e) alone would cost
// 2^-18 of e at |a| = 88: the first, of 16 bits, gives an exact product with a bf16 number, and 2^x of
// the second's, at most 7e-4, is 1 + x ln 2 to 2^-23 (no less than 1/2 for an infinite a, where e is 0).
struct Sigmoid {
    float s, slope;
    __device__ __forceinline__ explicit Sigmoid(float a)
    {
        constexpr float kHi = 47274.f / 32768.f, kLo = 7.0526077e-06f * 0.69314718f;
        const float m = -fabsf(a);
        const float e = __builtin_amdgcn_exp2f(m * kHi) * fmaxf(fmaf(m, kLo, 1.f), 0.5f);
        const float r = __builtin_amdgcn_rcpf(1.f + e), q = e * r;
        s = a < 0.f ? q : r;
        slope = q * r;
    }
};

// The kernels' variants: vectors of every array a thread, threads at most, the stream's type, and which
// of the operands there are.  (Without a norm behind the block and a gate, x itself may be absent.)  kNt: the
// results go past the caches.
template <int kVecs_, int kThreads_, bool kF32_, bool kPost_, bool kGate_, bool kNt_>
struct NormKind {
    static constexpr int kVecs = kVecs_, kThreads = kThreads_, kWaves = kThreads_ / 64;
    static constexpr bool kF32 = kF32_, kPost = kPost_, kGate = kGate_, kX = kPost_ || kGate_, kNt = kNt_;
    // 1024 threads, of 128 registers each, keep the gradient's weight sums in LDS and no second row: 8192 x 16384
    // in 691 us with norm and gate, 502 without the gate, 404 without the norm, 244 without both; with sums and a
    // second row in registers, of which many more are spilled, 1357, 1083, 632 and 346.  As it is, 42 to 55
    // registers are spilled with a norm behind the block, up to 12 without.  (Of the smaller forms one spills, 8:
    // one vector, fp32 stream, norm and gate.)
    static constexpr bool kSumsInLds = kThreads > 512;
};

// A workgroup for each row: 8 waves a SIMD hide one row's waits behind the others' (one vector a thread up to
// 4096 channels; two took 341 us instead of 331 for the fp32 stream at 32768 x 4096, and as long for bf16).
// y comes from h' before its rounding to the stream's type: the row is at hand, and a second
// rounding in front of the norm would only add its error.
template <typename Kind>
__global__ __launch_bounds__(Kind::kThreads) void k_residual_norm(NormArgs a, void *h_out, uint16_t *y)
{
    constexpr int kVecs = Kind::kVecs, kWaves = Kind::kWaves;
    using Stream = Stream8<Kind::kF32>;
    __shared__ float s_x[kWaves][1], s_h[kWaves][1];
    const int vecs = a.channels >> 3;
    const float inv_c = 1.f / (float)a.channels;
    const bool has_x = Kind::kX || a.x;
    clear_sums<kWaves>(s_x);
    clear_sums<kWaves>(s_h);
    __syncthreads();
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        Stream hr[kVecs];
        u32x4_t xr[kVecs], gr[kVecs], wr[kVecs], pr[kVecs];
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {  // (threads past the row read its last vector)
            const int i = min((int)(threadIdx.x + j * blockDim.x), vecs - 1);
            const uint32_t place = place_of(i);
            hr[j].load(a.h, t * a.channels, place);
            if (has_x)
                xr[j] = ld16_nt(in_row(a.x, t * a.x_stride, place));
            if (Kind::kGate)
                gr[j] = ld16_nt(in_row(a.gate, t * a.gate_stride, place));
            wr[j] = ld16(a.weight + 8 * i);
            if (Kind::kPost)
                pr[j] = ld16(a.post + 8 * i);
        }
        float rx = 1.f;
        if (Kind::kPost) {
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
            block_sums<kWaves>(sum, s_x);
            rx = rsqrtf(sum[0] * inv_c + a.eps);
        }
        float h[kVecs][8], sum[1] = {0.f};
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            const int i = threadIdx.x + j * blockDim.x;
            const uint32_t place = place_of(i);
            hr[j].get(h[j]);
            if (has_x) {
                float x[8];
                unpack8(xr[j], x);
                if (Kind::kPost) {
                    float w[8];
                    unpack8(pr[j], w);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[e] *= rx * w[e];
                }
                if (Kind::kGate) {
                    float g[8];
                    unpack8(gr[j], g);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[e] *= Sigmoid(g[e]).s;
                }
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    h[j][e] += a.scale * x[e];
                if (i < vecs)
                    Stream::template store<Kind::kNt>(h_out, t * a.channels, place, h[j]);
            }
            if (i < vecs)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    sum[0] += h[j][e] * h[j][e];
        }
        block_sums<kWaves>(sum, s_h);
        const float r = rsqrtf(sum[0] * inv_c + a.eps);
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            const int i = threadIdx.x + j * blockDim.x;
            const uint32_t place = place_of(i);
            float w[8];
            unpack8(wr[j], w);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                w[e] *= h[j][e] * r;
            if (i < vecs)
                put16<Kind::kNt>(in_row(y, t * a.channels, place), pack8(w));
        }
        if (t + gridDim.x < a.tokens)
            __syncthreads();  // the sums' LDS is written again
    }
}

// One row's arrays as they lie in memory; threads past the row hold its last vector.  dh_out, which may be
// absent, comes first: a wait for what comes behind it need not know.
template <typename Kind>
struct GradRow {
    Stream8<Kind::kF32> h[Kind::kVecs], dh[Kind::kVecs];
    u32x4_t dy[Kind::kVecs], x[Kind::kVecs], gate[Kind::kVecs];
    // at: the thread's vectors in the row
    __device__ __forceinline__ void load(const NormArgs &a, const NormGradArgs &g, int64_t t,
                                         const int (&at)[Kind::kVecs])
    {
        if (g.dh_out)
#pragma unroll
            for (int j = 0; j < Kind::kVecs; ++j)
                dh[j].load(g.dh_out, t * a.channels, place_of(at[j]));
#pragma unroll
        for (int j = 0; j < Kind::kVecs; ++j) {
            const uint32_t place = place_of(at[j]);
            h[j].load(a.h, t * a.channels, place);
            dy[j] = ld16_nt(in_row(g.dy, t * a.channels, place));
            if (Kind::kX)
                x[j] = ld16_nt(in_row(a.x, t * a.x_stride, place));
            if (Kind::kGate)
                gate[j] = ld16_nt(in_row(a.gate, t * a.gate_stride, place));
        }
    }
};

// The gradient's sums and one row's work, for a workgroup.
template <typename Kind>
struct NormGrad {
    static constexpr int kVecs = Kind::kVecs, kWaves = Kind::kWaves;
    const NormArgs &a;
    const NormGradArgs &g;
    float (*s_1)[3], (*s_2)[1], *s_dw;
    float inv_c;
    int at[kVecs];
    bool live[kVecs];  // whether that is a vector of its own
    u32x4_t wr[kVecs], pr[kVecs];
    float dw[kVecs][8], dp[kVecs][8];  // (kSumsInLds: there)

    // v to the sums of the thread's j-th channels.
    __device__ __forceinline__ void add8(float (&sum)[8], float *lds, int i, bool live, const float (&v)[8])
    {
        if (!Kind::kSumsInLds) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                sum[e] += v[e];
        } else if (live) {
            f32x4_t *p = reinterpret_cast<f32x4_t *>(lds + 8 * i);
            p[0] += (f32x4_t){v[0], v[1], v[2], v[3]};
            p[1] += (f32x4_t){v[4], v[5], v[6], v[7]};
        }
    }

    __device__ __forceinline__ void row_done(const GradRow<Kind> &row, int64_t t)
    {
        // ---- sums of h'^2, u h' and x^2
        float sum[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            float h[8], d[8], w[8];
            row.h[j].get(h);
            unpack8(row.dy[j], d);
            unpack8(wr[j], w);
            float hh = 0.f, uh = 0.f, xx = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                hh += h[e] * h[e];
                uh += d[e] * w[e] * h[e];
            }
            if (Kind::kPost) {
                unpack8(row.x[j], h);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    xx += h[e] * h[e];
            }
            sum[0] += live[j] ? hh : 0.f;
            sum[1] += live[j] ? uh : 0.f;
            sum[2] += live[j] ? xx : 0.f;
        }
        // (dh may be dh_out, which another thread too holds of the row's last vector: nobody stores before
        // everybody has it)
        if (g.dh_out)
#pragma unroll
            for (int j = 0; j < kVecs; ++j)
                row.dh[j].arrive();
        block_sums<kWaves>(sum, s_1);
        const float r = rsqrtf(sum[0] * inv_c + a.eps);
        const float rc = r * (sum[1] * inv_c * r);  // r mean(u k)
        const float rx = Kind::kPost ? rsqrtf(sum[2] * inv_c + a.eps) : 1.f;
        // ---- dh, dgate; what goes on to x stays in e
        float e_[kVecs][8], dot[1] = {0.f};
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            const int i = at[j];  // (threads past the row store the last vector's results again)
            const uint32_t place = place_of(i);
            float h[8], d[8], w[8];
            row.h[j].get(h);
            unpack8(row.dy[j], d);
            unpack8(wr[j], w);
            float dk[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float k = h[e] * r;
                dk[e] = d[e] * k;
                d[e] = r * (d[e] * w[e]) - k * rc;
            }
            add8(dw[j], s_dw, i, live[j], dk);
            if (g.dh_out) {
                row.dh[j].get(h);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    d[e] += h[e];
            }
            Stream8<Kind::kF32>::template store<Kind::kNt>(g.dh, t * a.channels, place, d);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                d[e] *= a.scale;
            float x[8], p[8];
            if (Kind::kX) {
                unpack8(row.x[j], x);
                if (Kind::kPost) {
                    unpack8(pr[j], p);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[e] *= rx;
                }
            }
            if (Kind::kGate) {
                float q[8];
                unpack8(row.gate[j], q);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const Sigmoid s(q[e]);
                    const float n = Kind::kPost ? x[e] * p[e] : x[e];
                    q[e] = d[e] * s.slope * n;
                    d[e] *= s.s;
                }
                put16<Kind::kNt>(in_row(g.dgate, t * g.dgate_stride, place), pack8(q));
            }
            if (Kind::kPost) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    dk[e] = d[e] * x[e];
                add8(dp[j], s_dw + a.channels, i, live[j], dk);
                float here = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    d[e] *= p[e];
                    here += d[e] * x[e];
                    e_[j][e] = d[e];
                }
                dot[0] += live[j] ? here : 0.f;
            } else if (Kind::kGate || g.dx) {
                put16<Kind::kNt>(in_row(g.dx, t * g.dx_stride, place), pack8(d));
            }
        }
        if (Kind::kPost) {
            block_sums<kWaves>(dot, s_2);
            const float rxm = rx * rx * (dot[0] * inv_c);
#pragma unroll
            for (int j = 0; j < kVecs; ++j) {
                const uint32_t place = place_of(at[j]);
                float x[8];
                unpack8(row.x[j], x);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x[e] = rx * e_[j][e] - x[e] * rxm;
                put16<Kind::kNt>(in_row(g.dx, t * g.dx_stride, place), pack8(x));
            }
        } else {
            __syncthreads();  // s_1 is written again
        }
    }
};

// The workgroup's place among `n`: each of the 8 XCDs, which take workgroups in turn, has neighbours.
__device__ __forceinline__ int place_by_xcd(int block, int n)
{
    return n % 8 ? block : block % 8 * (n / 8) + block / 8;
}

// A workgroup takes every gridDim.x-th row, the next row's loads under way, and keeps its channels'
// sums for the weights in registers; k_norm_dw adds the workgroups' up in a fixed order.  Two vectors a thread
// where a row has 128 (one -> two, us: 65536 rows of 2048 508 -> 461, fp32 stream 32768 x 4096 597 -> 557, 16384 x
// 5120 534 -> 352): fewer waves wait at a row's barriers, each with more to do.  XCDs on neighbouring rows: 461 ->
// 434 at 2048 channels; results past the caches: 420 -> 404 at 32768 x 4096.
template <typename Kind>
__global__ __launch_bounds__(Kind::kThreads, Kind::kThreads == 512 && Kind::kVecs == 2 ? 2 : 4) void
k_residual_norm_bwd(NormArgs a, NormGradArgs g)
{
    constexpr int kVecs = Kind::kVecs, kWaves = Kind::kWaves;
    __shared__ float s_1[kWaves][3], s_2[kWaves][1];
    clear_sums<kWaves>(s_1);
    clear_sums<kWaves>(s_2);
    extern __shared__ f32x4_t s_dw4[];
    float *s_dw = reinterpret_cast<float *>(s_dw4);
    const int parts = Kind::kPost ? 2 : 1;
    if (Kind::kSumsInLds)
        for (int i = threadIdx.x; i < parts * (a.channels >> 2); i += blockDim.x)
            s_dw4[i] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    __syncthreads();
    NormGrad<Kind> n{a, g, s_1, s_2, s_dw, 1.f / (float)a.channels, {}, {}};
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
        const int own = threadIdx.x + j * blockDim.x, i = min(own, (a.channels >> 3) - 1);
        n.at[j] = i;
        n.live[j] = own == i;
        n.wr[j] = ld16(a.weight + 8 * i);
        if (Kind::kPost)
            n.pr[j] = ld16(a.post + 8 * i);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            n.dw[j][e] = n.dp[j][e] = 0.f;
    }
    int64_t t = place_by_xcd(blockIdx.x, gridDim.x);
    if (Kind::kSumsInLds) {
        for (; t < a.tokens; t += gridDim.x) {
            GradRow<Kind> row;
            row.load(a, g, t, n.at);
            n.row_done(row, t);
        }
    } else {
        // Every row's loads (of the last row again behind it) and stores are under way without a condition, and
        // the first row is done ahead of the loop: so a wait for a row's loads is for nothing that
        // came after them.
        GradRow<Kind> even, odd;
        auto ahead = [&](GradRow<Kind> &next) __attribute__((always_inline)) {
            const int64_t after = t + gridDim.x;
            next.load(a, g, after < a.tokens ? after : a.tokens - 1, n.at);
            __builtin_amdgcn_sched_barrier(0);
        };
        even.load(a, g, t, n.at);
        ahead(odd);
        n.row_done(even, t);
        for (t += gridDim.x; t < a.tokens; t += gridDim.x) {
            ahead(even);
            n.row_done(odd, t);
            t += gridDim.x;
            if (t >= a.tokens)
                break;
            ahead(odd);
            n.row_done(even, t);
        }
    }
    float *out = g.partials + (int64_t)blockIdx.x * parts * a.channels;
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
        const int i = n.at[j];
        if (n.live[j]) {
            if (Kind::kSumsInLds) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    n.dw[j][e] = s_dw[8 * i + e];
                    n.dp[j][e] = Kind::kPost ? s_dw[a.channels + 8 * i + e] : 0.f;
                }
            }
            Stream8<true>::store<false>(out, 0, place_of(i), n.dw[j]);
            if (Kind::kPost)
                Stream8<true>::store<false>(out, a.channels, place_of(i), n.dp[j]);
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

// 16-byte vectors of every array a thread, and threads of a row.
int norm_vecs(int channels, bool grad) { return channels / 8 >= (grad ? 128 : 513) ? 2 : 1; }

int norm_threads(int channels, bool grad)
{
    const int v = norm_vecs(channels, grad);
    return (channels / 8 + 64 * v - 1) / (64 * v) * 64;
}

// launch(NormKind) with the variant that the operands take.
template <typename Launch>
void with_kind(const NormArgs &a, bool grad, bool past_caches, Launch launch)
{
    auto operands = [&](auto vecs, auto threads, auto f32, auto nt) {
        constexpr int v = decltype(vecs)::value, n = decltype(threads)::value;
        constexpr bool f = decltype(f32)::value, past = decltype(nt)::value;
        if (a.post && a.gate)
            launch(NormKind<v, n, f, true, true, past>());
        else if (a.post)
            launch(NormKind<v, n, f, true, false, past>());
        else if (a.gate)
            launch(NormKind<v, n, f, false, true, past>());
        else
            launch(NormKind<v, n, f, false, false, past>());
    };
    const std::true_type yes;
    const std::false_type no;
    auto stream = [&](auto vecs, auto threads) {
        if (a.f32)
            past_caches ? operands(vecs, threads, yes, yes) : operands(vecs, threads, yes, no);
        else
            past_caches ? operands(vecs, threads, no, yes) : operands(vecs, threads, no, no);
    };
    const int threads = norm_threads(a.channels, grad);
    if (norm_vecs(a.channels, grad) == 1)
        stream(std::integral_constant<int, 1>(), std::integral_constant<int, 512>());
    else if (threads <= 512)
        stream(std::integral_constant<int, 2>(), std::integral_constant<int, 512>());
    else
        stream(std::integral_constant<int, 2>(), std::integral_constant<int, 1024>());
}

}  // namespace

int norm_grad_blocks(int64_t tokens, int channels)
{
    // As many as the device holds at once: 4 waves a SIMD, 2 for the two vectors of up to 512 threads, whose forms
    // have 140 to 255 registers.  (3 for those too took longer also where they would fit, without a norm behind
    // the block: 32768 x 4096, gated, 414 us instead of 391, 1021 x 5120 27 instead of 20.)
    const int threads = norm_threads(channels, true);
    const int waves = norm_vecs(channels, true) == 2 && threads <= 512 ? 8 : 16;
    const int64_t b = 256 * (waves * 64 / threads < 8 ? waves * 64 / threads : 8);
    return (int)(b < tokens ? b : tokens);
}

size_t norm_grad_workspace(int64_t tokens, int channels)
{
    return (size_t)norm_grad_blocks(tokens, channels) * 2 * channels * sizeof(float);
}

hipError_t launch_residual_norm(const NormArgs &a, void *h_out, uint16_t *y, hipStream_t stream)
{
    const int64_t blocks = a.tokens < kNormBlocks ? a.tokens : kNormBlocks;
    const bool nt = a.tokens * a.channels * (a.x ? a.f32 ? 6 : 4 : 2) >= kPastCaches;
    with_kind(a, false, nt, [&](auto kind) {
        hipLaunchKernelGGL(k_residual_norm<decltype(kind)>, dim3((unsigned)blocks),
                           dim3(norm_threads(a.channels, false)), 0, stream, a, h_out, y);
    });
    return hipGetLastError();
}

hipError_t launch_residual_norm_bwd(const NormArgs &a, const NormGradArgs &g, hipStream_t stream)
{
    const int blocks = norm_grad_blocks(a.tokens, a.channels);
    const int parts = a.post ? 2 : 1;
    const bool nt = a.tokens * a.channels * ((a.f32 ? 4 : 2) + (g.dx ? 2 : 0) + (g.dgate ? 2 : 0)) >=
                    kPastCaches;
    with_kind(a, true, nt, [&](auto kind) {
        hipLaunchKernelGGL(k_residual_norm_bwd<decltype(kind)>, dim3(blocks),
                           dim3(norm_threads(a.channels, true)),
                           decltype(kind)::kSumsInLds ? parts * a.channels * sizeof(float) : 0, stream, a,
                           g);
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(k_norm_dw, dim3((parts * a.channels + kNormDwChannels - 1) / kNormDwChannels),
                       dim3(kNormDwChannels * kNormDwParts), 0, stream, g.partials, blocks,
                       a.channels, parts, g.dweight, g.dpost);
    return hipGetLastError();
}

}  // namespace sparrow
