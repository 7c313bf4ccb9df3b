// GQA decode attention over a paged e4m3 cache (format in cache_e4m3.h), sparse or dense: the
// work split of attention.hip's k_attn_stream (attention_split.h) over tiles of 32 tokens.
//
//   z_t = scale 2^{ek_t} (q . k_t),  w = softmax(z),  o = sum_t w_t 2^{ev_t} v_t
// with k_t, v_t the rows' codes.  Half the bytes of a bf16 cache per token, so the same bytes in
// flight are twice the tokens: a tile is two parts of 16 tokens (of one page, or of two 16-token
// pages next to each other in the list).  Per part and wave:
//   QK  codes to bf16 (exact), 4 x mfma_f32_16x16x32_bf16, the result times scale 2^{ek}
//       lane (row = token lr, group lg) holds channels 16lg..16lg+15 and 64+16lg..: two 16-byte
//       loads; q's fragments are loaded in the same channel order
//   PV  lane (lr, lg) loads the 8 codes V[token][8lr ..] of the tokens 4lg..4lg+3 of both parts and
//       converts them with their row's scale, which gives the exact bf16 values; 8 output tiles
//       on mfma_f32_16x16x32_bf16 over the tile's 32 tokens
// The softmax numerators enter PV as the sum of two bf16 numbers (the value rounded, and what that
// rounding left), 17 bits in all: the matrix cores have the time, and the result is as exact as one
// rounded from fp32 at the end.  Sums and maxima are fp32.
#include <atomic>

#include "attention_e4m3.h"

#include "attention_split.h"
#include "cache_e4m3.h"
#include "wave.h"

namespace sparrow {
namespace {

// Streaming waves per (sequence, KV head) unit on average, at most.
constexpr int kUnitSegments = 256;
constexpr int kParts = 2;  // 16-token parts of a tile

struct Args8 {
    AttnArgs a;
    const uint8_t *k, *v, *exps;
};

struct Tile {
    u32x4_t k[kParts][2];
    u32x2_t v[kParts][4];
    u32x2_t e[kParts];  // exponents of tokens 4lg .. 4lg+3: K's bytes, V's bytes
};

__device__ __forceinline__ u32x2_t ld8_nt(const void *p)
{
    return __builtin_nontemporal_load(reinterpret_cast<const u32x2_t *>(p));
}

// Part p from the cache row `row` on.
__device__ __forceinline__ void load_part(Tile &t, int p, const Args8 &x, int64_t row, int lr,
                                          int lg)
{
    t.e[p] = *reinterpret_cast<const u32x2_t *>(x.exps + row * 2 + 8 * lg);
    const uint8_t *kp = x.k + row * kHeadDim + lr * kHeadDim + 16 * lg;
    t.k[p][0] = ld16_nt(kp);
    t.k[p][1] = ld16_nt(kp + 64);
    const uint8_t *vp = x.v + row * kHeadDim + 4 * lg * kHeadDim + 8 * lr;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        t.v[p][j] = ld8_nt(vp + j * kHeadDim);
}

__device__ __forceinline__ float byte_pow2(uint32_t w, int j)
{
    return __uint_as_float(((w >> (8 * j)) & 0xffu) << 23);
}

// The bf16 values of 8 codes times a power of two.
__device__ __forceinline__ u32x4_t values(u32x2_t c, float scale)
{
    return (u32x4_t){unpack_e4m3<false>(c[0], scale), unpack_e4m3<true>(c[0], scale),
                     unpack_e4m3<false>(c[1], scale), unpack_e4m3<true>(c[1], scale)};
}

// A tile into the wave's online-softmax state.  valid[p] tokens of part p lie inside the sequence
// (at least one in all); the others get weight 0 and zero V rows.
__device__ __forceinline__ void attend_tile(Tile &t, const int (&valid)[kParts],
                                            const bf16x8_t (&qf)[4], float scale_log2, int lg,
                                            float &m_run, float &l_run, f32x4_t (&O)[8])
{
    float z[kParts][4];
    float cm = -INFINITY;
#pragma unroll
    for (int p = 0; p < kParts; ++p) {
        f32x4_t s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const u32x4_t w = t.k[p][i >> 1];
            const u32x4_t kf = values((i & 1) ? (u32x2_t){w[2], w[3]} : (u32x2_t){w[0], w[1]}, 1.f);
            s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf), qf[i], s,
                                                        0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            z[p][j] = 4 * lg + j < valid[p] ? s[j] * (scale_log2 * byte_pow2(t.e[p][0], j))
                                            : -INFINITY;
            cm = fmaxf(cm, z[p][j]);
        }
    }
    cm = fmaxf(cm, __shfl_xor(cm, 16, 64));
    cm = fmaxf(cm, __shfl_xor(cm, 32, 64));
    const float m_new = fmaxf(m_run, cm);
    const float alpha = exp2f(m_run - m_new);
    m_run = m_new;
    float sum = 0.f;
    u32x4_t hi, lo;
#pragma unroll
    for (int p = 0; p < kParts; ++p)
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            const float a = exp2f(z[p][j] - m_new), b = exp2f(z[p][j + 1] - m_new);
            sum += a + b;
            const uint32_t h = pack_bf16(a, b);
            hi[2 * p + (j >> 1)] = h;
            lo[2 * p + (j >> 1)] = pack_bf16(a - bf16_lo(h), b - bf16_hi(h));
        }
    l_run = l_run * alpha + sum;
    if (__ballot(alpha != 1.f)) {
#pragma unroll
        for (int c = 0; c < 8; ++c)
            O[c] *= alpha;
    }
    u32x4_t v[kParts][4];
#pragma unroll
    for (int p = 0; p < kParts; ++p) {
        if (valid[p] < 16) {  // cache slots past the length may hold anything
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (4 * lg + j >= valid[p]) {
                    t.v[p][j] = (u32x2_t){0u, 0u};
                    t.e[p][1] &= ~(0xffu << (8 * j));
                }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[p][j] = values(t.v[p][j], byte_pow2(t.e[p][1], j));
    }
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const u32x4_t av = {pair_of(v[0][0], v[0][1], c), pair_of(v[0][2], v[0][3], c),
                            pair_of(v[1][0], v[1][1], c), pair_of(v[1][2], v[1][3], c)};
        O[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, av),
                                                       __builtin_bit_cast(bf16x8_t, hi), O[c], 0,
                                                       0, 0);
        O[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, av),
                                                       __builtin_bit_cast(bf16x8_t, lo), O[c], 0,
                                                       0, 0);
    }
}

// q's fragments in the channel order of the K loads.
__device__ __forceinline__ void load_q(const AttnArgs &a, int b, int h, int lr, int lg,
                                       bf16x8_t (&qf)[4])
{
    const int G = a.num_q_heads / a.num_kv_heads;
    const uint16_t *qrow = a.q + ((int64_t)b * a.num_q_heads + (int64_t)h * G + lr) * kHeadDim;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        u32x4_t v = {0u, 0u, 0u, 0u};
        if (lr < G)
            v = ld16(qrow + 64 * (i >> 1) + 16 * lg + 8 * (i & 1));
        qf[i] = __builtin_bit_cast(bf16x8_t, v);
    }
}

// The walk's state at position pos: the last sequence whose offset is <= pos holds it (empty
// sequences before it share its offset).  A wave narrows [lo, lo + span) 64-fold per round.
__device__ __forceinline__ Cursor locate(const int32_t *s_off, int B, int Hkv, int64_t pos,
                                         int lane)
{
    int lo = 0, span = B;
    while (span > 1) {
        const int step = (span + 63) >> 6;
        const bool ok = lane * step < span && (int64_t)s_off[lo + lane * step] * Hkv <= pos;
        const int t = __popcll(__ballot(ok)) - 1;
        lo += t * step;
        span = min(step, span - t * step);
    }
    Cursor c;
    c.b = lo;
    c.cnt = s_off[lo + 1] - s_off[lo];
    const int64_t rel = pos - (int64_t)s_off[lo] * Hkv;
    c.h = (int)(rel / c.cnt);
    c.j = (int)(rel - (int64_t)c.h * c.cnt);
    c.pos = pos;
    return c;
}

template <bool kSparse>
__global__ __launch_bounds__(kAttnThreads) void k_attn_stream_e4m3(Args8 x)
{
    extern __shared__ int32_t s_off[];  // [batch + 1]
    __shared__ int32_t s_tmp[kAttnWaves];
    const AttnArgs &a = x.a;

    seq_prefix<kSparse>(a, s_off, s_tmp);
    const int B = a.batch;
    const int Hkv = a.num_kv_heads;
    const int G = a.num_q_heads / Hkv;
    if (blockIdx.x == 0)
        for (int b = threadIdx.x; b <= B; b += kAttnThreads)
            a.plan_off[b] = s_off[b];

    const int64_t P = (int64_t)s_off[B] * Hkv;
    // (the rule of k_attn_stream, with tiles of twice its chunks)
    int64_t W = P * (a.ps >> 4) / (2 * kParts);
    W = W > a.fine_waves ? W : a.fine_waves;
    W = W < a.max_waves ? W : a.max_waves;
    W = W < P ? W : P;
    const int w = blockIdx.x * kAttnWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (w >= W)
        return;
    const int64_t pos_end = (int64_t)(w + 1) * P / W;
    const int lane = threadIdx.x & 63;
    const int lr = lane & 15;
    const int lg = lane >> 4;
    const int ps = a.ps;
    const int cpp = ps >> 4;  // 16-token parts per page
    Cursor cur = locate(s_off, B, Hkv, (int64_t)w * P / W, lane);

    Batch bc, bn;
    fetch_batch_begin<kSparse>(a, s_off, cur, pos_end, bc, lane);
    fetch_batch_end(a, bc);
    bool have_next = cur.pos < pos_end;
    bool bn_pending = have_next;  // bn's block-table loads not issued yet
    if (have_next)
        fetch_batch_begin<kSparse>(a, s_off, cur, pos_end, bn, lane);

    bf16x8_t qf[4], qn[4];
    load_q(a, bc.b, bc.h, lr, lg, qf);
    bool from_start = bc.j0 == 0;

    float m_run = -INFINITY;
    float l_run = 0.f;
    f32x4_t O[8];
#pragma unroll
    for (int c = 0; c < 8; ++c)
        O[c] = (f32x4_t){0.f, 0.f, 0.f, 0.f};

    // tile `ti` of batch t: parts 2 ti and 2 ti + 1; part ci is page ci / cpp, sub-part ci % cpp
    auto issue = [&](const Batch &t, int ti, Tile &tile, int (&valid)[kParts]) {
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
            valid[p] = 0;
            const int ci = kParts * ti + p;
            if (ci >= t.n * cpp)
                break;  // (an odd number of parts)
            const int pi = ci / cpp;
            const int sub = ci - pi * cpp;
            const int ph = __builtin_amdgcn_readlane(t.phys, pi);
            const int tok = __builtin_amdgcn_readlane(t.tok0, pi) + 16 * sub;
            // a block-table entry outside the cache is an absent page
            if (ph >= 0 && ph < a.num_phys && tok < t.L) {
                valid[p] = t.L - tok;
                load_part(tile, p, x, ((int64_t)ph * Hkv + t.h) * ps + 16 * sub, lr, lg);
            }
        }
    };

    // A unit's finished state: the output when the unit lies in this wave alone, else a partial
    // (segment `wave + unit`) for the merge.
    auto write_unit = [&](int b, int h, float l, bool first, bool last) {
        const int unit = b * Hkv + h;
        if (lane == 0) {
            if (first)
                a.unit_waves[2 * unit] = w;
            if (last)
                a.unit_waves[2 * unit + 1] = w;
        }
        if (lr >= G)
            return;
        if (first && last) {
            const float inv = l > 0.f ? 1.f / l : 0.f;
            const int64_t orow = ((int64_t)b * a.num_q_heads + (int64_t)h * G + lr) * kHeadDim;
#pragma unroll
            for (int c = 0; c < 8; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    store_out(a.out, a.out_bf16, orow + 32 * lg + 8 * i + c, O[c][i] * inv);
        } else {
            const int64_t seg = (int64_t)w + unit;
            float *op = a.o_part + (seg * G + lr) * kHeadDim + 32 * lg;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                st16(op + 8 * i, __builtin_bit_cast(
                                     u32x4_t, (f32x4_t){O[0][i], O[1][i], O[2][i], O[3][i]}));
                st16(op + 8 * i + 4, __builtin_bit_cast(
                                         u32x4_t, (f32x4_t){O[4][i], O[5][i], O[6][i], O[7][i]}));
            }
            if (lg == 0) {
                a.ml_part[(seg * G + lr) * 2 + 0] = m_run;
                a.ml_part[(seg * G + lr) * 2 + 1] = l;
            }
        }
    };

    Tile nxt;
    int valid_next[kParts];
    issue(bc, 0, nxt, valid_next);
    int ti = 0;
    for (;;) {
        Tile tile = nxt;
        const int valid[kParts] = {valid_next[0], valid_next[1]};
        const bool last_in_batch = kParts * (ti + 1) >= bc.n * cpp;
        if (!last_in_batch) {
            issue(bc, ti + 1, nxt, valid_next);
            if (bn_pending) {
                fetch_batch_end(a, bn);
                bn_pending = false;
            }
        } else if (have_next) {
            if (bn_pending) {  // a one-tile batch: bn is needed now
                fetch_batch_end(a, bn);
                bn_pending = false;
            }
            issue(bn, 0, nxt, valid_next);
            if (bc.ends_unit)
                load_q(a, bn.b, bn.h, lr, lg, qn);
        }

        if (valid[0] > 0 || valid[1] > 0)
            attend_tile(tile, valid, qf, a.scale_log2, lg, m_run, l_run, O);

        if (!last_in_batch) {
            ++ti;
            continue;
        }
        if (bc.ends_unit || !have_next) {
            float l_tot = l_run + __shfl_xor(l_run, 16, 64);
            l_tot += __shfl_xor(l_tot, 32, 64);
            write_unit(bc.b, bc.h, l_tot, from_start, bc.ends_unit);
            if (!have_next)
                break;
            m_run = -INFINITY;
            l_run = 0.f;
#pragma unroll
            for (int c = 0; c < 8; ++c)
                O[c] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                qf[i] = qn[i];
            from_start = bn.j0 == 0;
        }
        bc = bn;
        ti = 0;
        have_next = cur.pos < pos_end;
        bn_pending = have_next;
        if (have_next)
            fetch_batch_begin<kSparse>(a, s_off, cur, pos_end, bn, lane);
    }
}

// Streaming waves on the current device: compute units x resident workgroups x 4, capped.  (A
// cache of device attributes: concurrent first calls all store the same value.)
int device_waves()
{
    static std::atomic<int> cached[64];
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64)
        return kMaxWaves;
    int w = cached[dev].load(std::memory_order_relaxed);
    if (w == 0) {
        int per_cu = 0;
        if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, k_attn_stream_e4m3<true>,
                                                         kAttnThreads, 4096) != hipSuccess ||
            per_cu < 1)
            per_cu = 1;
        w = device_cus() * per_cu * kAttnWaves;
        w = w < kMaxWaves ? w : kMaxWaves;
        cached[dev].store(w, std::memory_order_relaxed);
    }
    return w;
}

}  // namespace

hipError_t launch_attention_e4m3(const sparrow_shape_t &s, const AttnPlan &plan, const void *q,
                                 const CacheE4m3 &c, const int32_t *block_table,
                                 const int32_t *seq_lens, const int32_t *k, const int32_t *idx,
                                 int32_t k_max, float scale, void *out, int out_dtype,
                                 void *workspace, hipStream_t stream)
{
    const int64_t units = (int64_t)s.batch * s.num_kv_heads;
    const int G = s.num_q_heads / s.num_kv_heads;
    const int64_t waves = device_waves();
    Args8 x{};
    x.k = c.k;
    x.v = c.v;
    x.exps = c.exps;
    AttnArgs &a = x.a;
    a.q = static_cast<const uint16_t *>(q);
    a.block_table = block_table;
    a.seq_lens = seq_lens;
    a.ksel = k;
    a.idx = idx;
    a.plan_off = static_cast<int32_t *>(workspace);
    a.unit_waves = a.plan_off + ((size_t)(s.batch + 1) + 63) / 64 * 64;
    a.o_part = reinterpret_cast<float *>(static_cast<char *>(workspace) + plan.plan_bytes);
    a.ml_part = a.o_part + plan.segments * G * kHeadDim;
    a.out = out;
    a.k_max = k_max;
    a.batch = s.batch;
    a.num_q_heads = s.num_q_heads;
    a.num_kv_heads = s.num_kv_heads;
    a.ps = s.page_size;
    a.max_pages = s.max_pages_per_seq;
    a.num_phys = s.num_phys_pages;
    a.out_bf16 = out_dtype == SPARROW_OUT_BF16 ? 1 : 0;
    a.max_waves = (int)(units * kUnitSegments < waves ? units * kUnitSegments : waves);
    a.fine_waves = (int)(units * 64 < waves ? units * 64 : waves);
    a.scale_log2 = scale * 1.4426950408889634f;
    auto kernel = idx != nullptr ? k_attn_stream_e4m3<true> : k_attn_stream_e4m3<false>;
    hipLaunchKernelGGL(kernel, dim3(waves / kAttnWaves), dim3(kAttnThreads), plan.lds_bytes,
                       stream, x);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : launch_attn_merge(a, stream);
}

}  // namespace sparrow
