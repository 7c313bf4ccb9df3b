// GQA decode attention over a paged e4m3 cache (format in cache_e4m3.h), sparse or dense: the
// work split of attention.hip's k_attn_stream (attention_split.h) over tiles of 32 tokens.
//
//   z_t = scale 2^{ek_t} (q . k_t),  w = softmax(z),  o = sum_t w_t 2^{ev_t} v_t
// with k_t, v_t the rows' codes.  Half the bytes of a bf16 cache per token, so the same bytes in
// flight are twice the tokens: a tile is two parts of 16 tokens (of one page, or of two 16-token
// pages next to each other in the list).  Per part and wave:
//   QK  codes to bf16 (exact), 4 x mfma_f32_16x16x32_bf16, the result times scale 2^{ek}
//       lane (row = token lr, group lg) holds channels 32lg .. 32lg+31 (see trade_rows); q's
//       fragments are loaded in the same channel order
//   PV  lane (lr, lg) loads the 8 codes V[token][8lr ..] of the tokens 4lg..4lg+3 of both parts and
//       converts them with their row's scale, which gives the exact bf16 values; 8 output tiles
//       on mfma_f32_16x16x32_bf16 over the tile's 32 tokens
// The softmax numerators enter PV as the sum of three bf16 numbers, 8 bits each from the top down,
// which is all of their 24 bits: the products are those of fp32 numerators, for an fp32 output too.
// Sums and maxima are fp32.  An fp32 output of 8 units of 4097 tokens, 64 sequences of 8K-32K and 256 at
// 10 % is 1.9e-7, 9.1e-7 and 4.8e-7 off (2-norm), elementary operations in fp32 5.8e-7, 1.2e-6 and 4.9e-7.
// (Two numbers, 17 bits: 1.6e-6, 2.4e-6 and 2.3e-6; us in a graph, two -> three: 12.0 -> 12.2, 431 -> 434,
// 257 -> 259, and 8 units of 256 tokens 5.1 -> 5.2.)
//
// Bound by HBM: 64 sequences of 8K-32K tokens (2.8 GB) take 432 us, 6.5 TB/s where a read-only stream
// reaches 7.1; the third number's matrix instructions, a third more, cost it 1 %.
#include "attention_e4m3.h"

#include "attention_split.h"
#include "cache_e4m3.h"
#include "wave.h"

namespace sparrow {
namespace {

// Streaming waves per (sequence, KV head) unit on average, at most.
constexpr int kUnitSegments = 256;
constexpr int kParts = 2;   // 16-token parts of a tile
constexpr int kPieces = 3;  // bf16 numbers of a softmax numerator

struct Args8 {
    AttnArgs a;
    const uint8_t *k, *v, *exps;
};

struct Tile {
    u32x4_t k[kParts][2];
    u32x2_t v[kParts][4];
    u32x2_t e[kParts];  // exponents of tokens 4lg .. 4lg+3: K's bytes, V's bytes
};

// An address in the cache that all lanes share, kept in scalar registers: a load then takes it
// with the lane's 32-bit offset, and no vector instruction adds them up.
typedef const __attribute__((address_space(1))) uint8_t *global_bytes;

__device__ __forceinline__ global_bytes scalar_base(const uint8_t *p)
{
    uintptr_t u = (uintptr_t)p;
    asm volatile("" : "+s"(u));
    return (global_bytes)u;
}

template <typename T>
__device__ __forceinline__ T load_nt(global_bytes p)
{
    return __builtin_nontemporal_load((const __attribute__((address_space(1))) T *)p);
}

// A lane's offsets into a part's exponents, K and V.
struct LaneOffsets {
    uint32_t e, k, v;
    __device__ __forceinline__ LaneOffsets(int lr, int lg)
        : e(8 * lg), k((lr & 7) * kHeadDim + 16 * (2 * lg + (lr >> 3))),
          v(4 * lg * kHeadDim + 8 * lr) {}
};

// K, V and the exponents of part p from the 16 cache rows `part` (their number in the cache / 16).
__device__ __forceinline__ void load_exps(Tile &t, int p, const Args8 &x, int part, uint32_t e_lane)
{
    const global_bytes ep = scalar_base(x.exps + (int64_t)part * 32);
    t.e[p] = *(const __attribute__((address_space(1))) u32x2_t *)(ep + e_lane);
}

__device__ __forceinline__ void load_keys(Tile &t, int p, const Args8 &x, int part, uint32_t k_lane)
{
    const global_bytes kp = scalar_base(x.k + (int64_t)part * (16 * kHeadDim));
    t.k[p][0] = load_nt<u32x4_t>(kp + k_lane);
    t.k[p][1] = load_nt<u32x4_t>(kp + k_lane + 8 * kHeadDim);
}

__device__ __forceinline__ void load_values(Tile &t, int p, const Args8 &x, int part,
                                            uint32_t v_lane)
{
    const global_bytes vp = scalar_base(x.v + (int64_t)part * (16 * kHeadDim));
#pragma unroll
    for (int j = 0; j < 4; ++j)
        t.v[p][j] = load_nt<u32x2_t>(vp + v_lane + j * kHeadDim);
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

// Maximum / sum over the four lanes of a head (lr, lr + 16, lr + 32, lr + 48), which every one of
// them gets.  A swap of odd with even 16-lane rows of two copies leaves each lane its own row's
// value and its neighbour's; a swap of the upper with the lower half does it for 32 lanes.
template <typename Op>
__device__ __forceinline__ float over_groups(float x, Op op)
{
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    x = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// A softmax numerator's leading 8 bits, which are a bf16 number; and two numerators' as a pair.
__device__ __forceinline__ float top_of(float x)
{
    return __uint_as_float(__float_as_uint(x) & 0xffff0000u);
}

__device__ __forceinline__ uint32_t tops_of(float a, float b)
{
    return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}

// K of a part in operand order.  A load that gave lane (lr, lg) 16 bytes of its own row lr would touch
// 16 rows, half a line of each, and the memory reads lines; so each load takes 8 whole rows, and lane
// (lr, lg) holds chunk 2lg + lr / 8 of row lr % 8 and of row 8 + lr % 8.  Lanes lr and lr ^ 8 then
// trade the one that is not their row's, which leaves each with chunks 2lg and 2lg + 1 of its own.
// (Loads alone, 64 sequences of 8K-32K tokens: 457 us by half lines, 434 by rows.)
__device__ __forceinline__ void trade_rows(u32x4_t (&k)[2])
{
    constexpr int kRor8 = 0x128;  // lane ^ 8 inside each 16
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        const int a = (int)k[0][d], b = (int)k[1][d];
        k[0][d] = (uint32_t)__builtin_amdgcn_update_dpp(a, b, kRor8, 0xf, 0xc, false);
        k[1][d] = (uint32_t)__builtin_amdgcn_update_dpp(b, a, kRor8, 0xf, 0x3, false);
    }
}

// A tile into the wave's online-softmax state.  v0 and v1 tokens of its parts lie inside the
// sequence (16 or more: all; 0 or less: none); the others get weight 0 and zero V rows.  k_done() is
// called when the tile's K is read, v_done() when its V and exponents are: they may load the next.
template <typename KDone, typename VDone>
__device__ __forceinline__ void attend_tile(Tile &t, int v0, int v1, const bf16x8_t (&qf)[4],
                                            float scale_log2, int lg, float &m_run, float &l_run,
                                            f32x4_t (&O)[8], KDone k_done, VDone v_done)
{
    float z[kParts][4];
#pragma unroll
    for (int p = 0; p < kParts; ++p) {
        f32x4_t s = {0.f, 0.f, 0.f, 0.f};
        trade_rows(t.k[p]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const u32x4_t w = t.k[p][i >> 1];
            const u32x4_t kf = values((i & 1) ? (u32x2_t){w[2], w[3]} : (u32x2_t){w[0], w[1]}, 1.f);
            s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf), qf[i], s,
                                                        0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            z[p][j] = s[j] * (scale_log2 * byte_pow2(t.e[p][0], j));
    }
    k_done();
    if (min(v0, v1) < 16) {  // cache slots past the length, and parts that are not there, may
                             // hold anything
#pragma unroll
        for (int p = 0; p < kParts; ++p)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (4 * lg + j >= (p == 0 ? v0 : v1)) {
                    z[p][j] = -INFINITY;
                    t.v[p][j] = (u32x2_t){0u, 0u};
                    t.e[p][1] &= ~(0xffu << (8 * j));
                }
    }
    float cm = fmaxf(fmaxf(fmaxf(z[0][0], z[0][1]), fmaxf(z[0][2], z[0][3])),
                     fmaxf(fmaxf(z[1][0], z[1][1]), fmaxf(z[1][2], z[1][3])));
    cm = over_groups(cm, [](float a, float b) { return fmaxf(a, b); });
    const float m_old = m_run;
    m_run = fmaxf(m_run, cm);
    const float m = m_run == -INFINITY ? 0.f : m_run;  // (no token so far)
    const float alpha = __builtin_amdgcn_exp2f(m_old - m);
    float sum = 0.f;
    u32x4_t w[kPieces];
#pragma unroll
    for (int p = 0; p < kParts; ++p)
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            float a = __builtin_amdgcn_exp2f(z[p][j] - m);
            float b = __builtin_amdgcn_exp2f(z[p][j + 1] - m);
            sum += a + b;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                w[i][2 * p + (j >> 1)] = tops_of(a, b);
                a -= top_of(a);
                b -= top_of(b);
            }
        }
    l_run = l_run * alpha + sum;
    if (__ballot(alpha != 1.f)) {
#pragma unroll
        for (int c = 0; c < 8; ++c)
            O[c] *= alpha;
    }
    u32x4_t v[kParts][4];
#pragma unroll
    for (int p = 0; p < kParts; ++p)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[p][j] = values(t.v[p][j], byte_pow2(t.e[p][1], j));
    v_done();
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const u32x4_t av = {pair_of(v[0][0], v[0][1], c), pair_of(v[0][2], v[0][3], c),
                            pair_of(v[1][0], v[1][1], c), pair_of(v[1][2], v[1][3], c)};
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
            O[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, av),
                                                           __builtin_bit_cast(bf16x8_t, w[i]),
                                                           O[c], 0, 0, 0);
    }
}

// q's fragments of a unit (sequence, KV head) in the channel order of the K loads.
__device__ __forceinline__ void load_q(const AttnArgs &a, int unit, int lr, int lg,
                                       bf16x8_t (&qf)[4])
{
    const int G = a.num_q_heads / a.num_kv_heads;
    const uint16_t *qrow = a.q + ((int64_t)unit * G + lr) * kHeadDim;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        u32x4_t v = {0u, 0u, 0u, 0u};
        if (lr < G)
            v = ld16(qrow + 32 * lg + 8 * i);
        qf[i] = __builtin_bit_cast(bf16x8_t, v);
    }
}

// An LDS word that every lane reads, as a scalar.
__device__ __forceinline__ int32_t uniform(int32_t v) { return __builtin_amdgcn_readfirstlane(v); }

// A word at an address that every lane shares, by the scalar unit (the kernel does not write it).
__device__ __forceinline__ int32_t scalar_load(const int32_t *p)
{
    typedef const __attribute__((address_space(4))) int32_t *constant_ptr;
    return *(constant_ptr)(uintptr_t)p;
}

// The walk over a wave's range of (sequence, KV head, list position), in batches of at most
// kBatch pages of one unit.  Everything in it is the same for all lanes, but for what a lane knows
// of its page of the batch.
struct Walk {
    int unit, b, h, j, cnt, len;
    int64_t left;  // pages of the range not yet taken

    // The place of range position pos: the last sequence whose offset is <= pos holds it (empty
    // sequences before it share its offset).  A wave narrows [lo, lo + span) 64-fold per round.
    __device__ __forceinline__ void start(const AttnArgs &a, const int32_t *s_off, int64_t pos,
                                          int64_t end, int lane)
    {
        const int Hkv = a.num_kv_heads;
        int lo = 0, span = a.batch;
        while (span > 1) {
            const int step = (span + 63) >> 6;
            const bool ok = lane * step < span && (int64_t)s_off[lo + lane * step] * Hkv <= pos;
            const int t = __popcll(__ballot(ok)) - 1;
            lo += t * step;
            span = min(step, span - t * step);
        }
        b = lo;
        const int off = uniform(s_off[lo]);
        cnt = uniform(s_off[lo + 1]) - off;
        const int64_t rel = pos - (int64_t)off * Hkv;
        h = (int)(rel / cnt);
        j = (int)(rel - (int64_t)h * cnt);
        unit = b * Hkv + h;
        len = scalar_load(a.seq_lens + b);
        left = end - pos;
    }
};

constexpr int kCloses = 1, kLast = 2;  // a batch, or a tile, ends its unit; the range

// A batch of pages: what all lanes know of it.
struct PageBatch {
    int unit, b, len, n, ends;
};

// The next batch of the walk (n = 0 behind the last one).  Returns the lane's entry of its list; lanes
// past the batch read the first entry, so that the load is the same for all.
template <bool kSparse>
__device__ __forceinline__ int take(const AttnArgs &a, const int32_t *s_off, Walk &w, PageBatch &t,
                                    int lane)
{
    t.unit = w.unit;
    t.b = w.b;
    t.len = w.len;
    int n = min(w.cnt - w.j, kBatch);
    n = n < w.left ? n : (int)w.left;
    t.n = n;
    int lp = w.j + lane;
    if (kSparse)
        lp = a.idx[(int64_t)w.unit * a.k_max + (lane < n ? lp : 0)];
    w.left -= n;
    w.j += n;
    const bool closes = w.j == w.cnt;
    t.ends = (closes ? kCloses : 0) | (w.left == 0 ? kLast : 0);
    if (closes && w.left > 0) {  // the next unit with pages
        w.j = 0;
        ++w.unit;
        if (++w.h == a.num_kv_heads) {
            w.h = 0;
            do {
                ++w.b;
                w.cnt = uniform(s_off[w.b + 1]) - uniform(s_off[w.b]);
            } while (w.cnt == 0);
            w.unit = w.b * a.num_kv_heads;
            w.len = scalar_load(a.seq_lens + w.b);
        }
    }
    return lp;
}

// Whether a lane's list entry is a page of the batch's sequence.
__device__ __forceinline__ bool in_sequence(const AttnArgs &a, const PageBatch &t, int lp, int lane)
{
    const int L = clamp_len(t.len, a.ps, a.max_pages);
    return lane < t.n && lp >= 0 && lp < (L + a.ps - 1) >> (__ffs(a.ps) - 1);
}

// The physical page of a lane's list entry (entries outside the sequence read the row's first).
__device__ __forceinline__ int look_up(const AttnArgs &a, const PageBatch &t, int lp, int lane)
{
    return a.block_table[(int64_t)t.b * a.max_pages + (in_sequence(a, t, lp, lane) ? lp : 0)];
}

// What a lane's page of the batch at work is loaded by.
struct Pages {
    int part;    // number of its first 16 cache rows, / 16
    int tokens;  // inside the sequence; 0, with rows that exist, where there is no page

    // (a block-table entry outside the cache is an absent page)
    __device__ __forceinline__ void settle(const AttnArgs &a, const PageBatch &t, int lp, int phys,
                                           int lane)
    {
        const int L = clamp_len(t.len, a.ps, a.max_pages);
        const bool live = in_sequence(a, t, lp, lane) && phys >= 0 && phys < a.num_phys;
        part = live ? (phys * a.num_kv_heads + (t.unit - t.b * a.num_kv_heads)) * (a.ps >> 4) : 0;
        tokens = live ? min(L - lp * a.ps, a.ps) : 0;
    }
};

// A tile whose loads are issued.
struct Step {
    int v0, v1;  // tokens of its parts inside the sequence
    int unit, ends;
};

// A wave's range, tile by tile, with two tiles' loads in flight while a third is computed.  The
// buffers take turns, so that no tile is copied, and every tile is loaded (a part that is not there
// reads rows that exist and gets no weight), so that the loads in flight can be counted and the wait
// is for the tile at hand only.  The page lists and the block table are read two and one batches
// ahead, at the end of a batch, and nothing is done with their loads until the next one ends: loads
// return in order, so that a use of the youngest would make the wave wait for the tiles as well.
template <bool kSparse>
__global__ __launch_bounds__(kAttnThreads, 2) void k_attn_stream_e4m3(Args8 x)
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

    const int64_t P = (int64_t)uniform(s_off[B]) * Hkv;
    // A wave has at least one tile, with more than 8 query heads per KV head four (the merge reads a
    // row per head and wave), and at least one page.  A whole dense call, us, tiles 1 / 2 / 4: 8 units
    // of 4097 tokens x 2 heads 12.3 / 13.4 / 15.1, of 2048 10.8 / 11.6 / 13.4, 16 of 4096 x 16 heads
    // 18.9 / 18.8 / 16.9; no difference from 32 units of 8192 tokens on.  Shares are whole pages: with
    // pages of 128 tokens and little more than one a wave, some waves have twice the others' tiles.
    int64_t W = P * (a.ps >> 4) / (kParts * (G > 8 ? 4 : 1));
    W = W > 1 ? W : 1;
    W = W < a.max_waves ? W : a.max_waves;
    W = W < P ? W : P;
    const int w = blockIdx.x * kAttnWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (w >= W)
        return;
    const int lane = threadIdx.x & 63;
    const int lr = lane & 15;
    const int lg = lane >> 4;
    const LaneOffsets at(lr, lg);
    const int log_cpp = __ffs(a.ps) - 5;  // 16-token parts per page: ps / 16
    Walk walk;
    walk.start(a, s_off, (int64_t)w * P / W, (int64_t)(w + 1) * P / W, lane);
    bool from_start = walk.j == 0;  // the unit at work begins in this wave

    // the batch at work, the one with its block-table loads under way, the one with its list's
    PageBatch now, b1, b2;
    Pages pages;
    const int lp0 = take<kSparse>(a, s_off, walk, now, lane);
    int lp1 = take<kSparse>(a, s_off, walk, b1, lane);
    int lp2 = take<kSparse>(a, s_off, walk, b2, lane);
    const int phys0 = look_up(a, now, lp0, lane);
    int phys1 = look_up(a, b1, lp1, lane);
    bf16x8_t qf[4];
    load_q(a, now.unit, lr, lg, qf);
    pages.settle(a, now, lp0, phys0, lane);
    int ti = 0;
    int tiles = ((now.n << log_cpp) + kParts - 1) / kParts;

    // ---- the next tile of the range into a buffer (behind the last one: rows that exist)
    auto issue = [&](Tile &tile, Step &s) __attribute__((always_inline)) {
        const int c0 = kParts * ti, c1 = c0 + 1;  // parts of the batch
        const int p0 = (c0 >> log_cpp) & 63, p1 = (c1 >> log_cpp) & 63;  // their pages
        const int u0 = c0 & ((1 << log_cpp) - 1), u1 = c1 & ((1 << log_cpp) - 1);
        const int part[kParts] = {__builtin_amdgcn_readlane(pages.part, p0) + u0,
                                  __builtin_amdgcn_readlane(pages.part, p1) + u1};
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
            load_exps(tile, p, x, part[p], at.e);
            load_keys(tile, p, x, part[p], at.k);
            load_values(tile, p, x, part[p], at.v);
        }
        s.v0 = __builtin_amdgcn_readlane(pages.tokens, p0) - 16 * u0;
        s.v1 = __builtin_amdgcn_readlane(pages.tokens, p1) - 16 * u1;
        s.unit = now.unit;
        s.ends = 0;
        if (++ti < tiles)
            return;
        s.ends = now.ends;
        now = b1;
        pages.settle(a, now, lp1, phys1, lane);
        ti = 0;
        tiles = ((now.n << log_cpp) + kParts - 1) / kParts;
        b1 = b2;
        lp1 = lp2;
        phys1 = look_up(a, b1, lp1, lane);
        lp2 = take<kSparse>(a, s_off, walk, b2, lane);
    };

    float m_run = -INFINITY;
    float l_run = 0.f;
    f32x4_t O[8];
#pragma unroll
    for (int c = 0; c < 8; ++c)
        O[c] = (f32x4_t){0.f, 0.f, 0.f, 0.f};

    // ---- a unit's finished state: the output when the unit lies in this wave alone, else a
    // partial (segment `wave + unit`) for the merge
    auto write_unit = [&](int unit, bool first, bool last) __attribute__((always_inline)) {
        const float l = over_groups(l_run, [](float u, float v) { return u + v; });
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
            const int64_t orow = ((int64_t)unit * G + lr) * kHeadDim;
            // (channels 32lg + 8i + c are 8 in a row)
            if (a.out_bf16) {
                uint16_t *o = static_cast<uint16_t *>(a.out) + orow + 32 * lg;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    st16(o + 8 * i, (u32x4_t){pack_bf16(O[0][i] * inv, O[1][i] * inv),
                                              pack_bf16(O[2][i] * inv, O[3][i] * inv),
                                              pack_bf16(O[4][i] * inv, O[5][i] * inv),
                                              pack_bf16(O[6][i] * inv, O[7][i] * inv)});
            } else {
                float *o = static_cast<float *>(a.out) + orow + 32 * lg;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int c = 0; c < 8; c += 4)
                        st16(o + 8 * i + c,
                             __builtin_bit_cast(u32x4_t, (f32x4_t){O[c][i], O[c + 1][i], O[c + 2][i],
                                                                   O[c + 3][i]} * inv));
            }
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

    // ---- a tile's turn; true when the range is done
    auto turn = [&](Tile &tile, const Step &s, const Step &after) __attribute__((always_inline)) {
        attend_tile(tile, s.v0, s.v1, qf, a.scale_log2, lg, m_run, l_run, O, [] {}, [] {});
        if (s.ends != 0) {
            write_unit(s.unit, from_start, s.ends & kCloses);
            if (s.ends & kLast)
                return true;
            from_start = true;
            m_run = -INFINITY;
            l_run = 0.f;
#pragma unroll
            for (int c = 0; c < 8; ++c)
                O[c] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
            load_q(a, after.unit, lr, lg, qf);
            // waited for here, not at every use: an operand that might be this load's would make
            // each tile wait for all loads before it
#pragma unroll
            for (int i = 0; i < 4; ++i)
                asm volatile("" : "+v"(qf[i]));
        }
        return false;
    };

    Tile t0, t1, t2;
    Step s0, s1, s2;
    issue(t0, s0);
    issue(t1, s1);
    for (;;) {
        issue(t2, s2);
        if (turn(t0, s0, s1))
            break;
        issue(t0, s0);
        if (turn(t1, s1, s2))
            break;
        issue(t1, s1);
        if (turn(t2, s2, s0))
            break;
    }
}

// Short lists: one workgroup per (sequence, KV head), its waves' states joined in LDS in wave order, so
// that there are no partials in memory and no second launch.  Every wave knows the whole list, a page
// per lane, and takes an equal share of its tiles.  A call of a few microseconds waits for its code as
// well as for its data, so the loop body is there once: it has one tile's registers, and the next
// tile's K is loaded where this one's is read, its V and exponents where they are (1024 tokens, 4 query
// heads, us in a graph, with numerators of two numbers: three tiles' registers in turn 11.9 for 8 units
// and 14.9 for 128; this 9.8 and 12.2; with 4 waves 11.0 and 14.0).  What is left is latency: a wave has
// one tile in flight, and 1024 tokens are four tiles a wave, one after another.
//
// Against the streaming waves and their merge, us in a graph, streaming -> this, 4 query heads:
//   units x tokens  8 x 256 10.4 -> 5.3, 8 x 1024 10.5 -> 9.7, 128 x 1024 16.6 -> 13.0, 256 x 1024
//   21.8 -> 14.8, 512 x 1024 33.1 -> 28.9, 768 x 256 21.3 -> 17.8, 768 x 1024 47.3 -> 43.5; lists of
//   50 to 1024 tokens, 256 units 20.0 -> 12.7, 768 34.9 -> 31.9
// and past 3 units a CU the other way (1024 x 256 20.2 -> 23.1, x 1024 54.1 -> 57.6).  Longer lists,
// bound by what one CU can fetch, pay where most CUs have one:
//   192 x 2048 28.1 -> 21.5, 256 x 2048 33.2 -> 25.6 (lists of 400 to 2048 tokens 27.0 -> 21.6); but
//   8 x 1536 10.9 -> 13.8, 128 x 2048 22.1 -> 21.4 (18.8 -> 18.2), 384 x 2048 45.7 -> 46.2.
// A dense call goes by the block table's width, the only bound on the lengths that the host knows.
constexpr int kUnitsPerCu = 3;
constexpr int kUnitMaxTokens = 1024;    // list bound x page size; twice that, see unit_path
constexpr int kUnitThreads = 512;
constexpr int kUnitWaves = kUnitThreads / 64;
constexpr int kUnitMaxGroup = 8;        // query heads per KV head (sizes the LDS)
constexpr int kUnitRow = kHeadDim + 4;  // LDS row stride of a wave's o (floats)

template <bool kSparse>
__global__ __launch_bounds__(kUnitThreads, 2) void k_attn_unit_e4m3(Args8 x)
{
    __shared__ __align__(16) float s_o[kUnitWaves * kUnitMaxGroup * kUnitRow];
    __shared__ float s_m[kUnitWaves * kUnitMaxGroup], s_l[kUnitWaves * kUnitMaxGroup];
    const AttnArgs &a = x.a;
    const int Hkv = a.num_kv_heads;
    const int G = a.num_q_heads / Hkv;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int lr = lane & 15;
    const int lg = lane >> 4;
    const int log_cpp = __ffs(a.ps) - 5;

    PageBatch t;
    t.unit = blockIdx.x;
    t.b = t.unit / Hkv;
    t.len = scalar_load(a.seq_lens + t.b);
    int lp = lane;
    if (kSparse) {  // (lanes past the row read its first entry)
        const int c = scalar_load(a.ksel + t.b);
        lp = a.idx[(int64_t)t.unit * a.k_max + (lane < a.k_max ? lane : 0)];
        t.n = c < 0 ? 0 : min(c, a.k_max);
    } else {
        t.n = (clamp_len(t.len, a.ps, a.max_pages) + a.ps - 1) >> (log_cpp + 4);
    }
    bf16x8_t qf[4];
    load_q(a, t.unit, lr, lg, qf);
    Pages pages;
    pages.settle(a, t, lp, look_up(a, t, lp, lane), lane);

    const int tiles = ((t.n << log_cpp) + kParts - 1) / kParts;
    const int end = (wv + 1) * tiles / kUnitWaves;
    int ti = wv * tiles / kUnitWaves;
    // the next tile's place; behind the share all lanes take one word of the last one
    const LaneOffsets in_part(lr, lg);
    LaneOffsets at = in_part;
    int part[kParts], v0, v1;
    auto place = [&]() __attribute__((always_inline)) {
        const int c0 = kParts * min(ti, end - 1), c1 = c0 + 1;
        const int p0 = c0 >> log_cpp, p1 = (c1 >> log_cpp) & 63;
        const int u0 = c0 & ((1 << log_cpp) - 1), u1 = c1 & ((1 << log_cpp) - 1);
        part[0] = __builtin_amdgcn_readlane(pages.part, p0) + u0;
        part[1] = __builtin_amdgcn_readlane(pages.part, p1) + u1;
        v0 = __builtin_amdgcn_readlane(pages.tokens, p0) - 16 * u0;
        v1 = __builtin_amdgcn_readlane(pages.tokens, p1) - 16 * u1;
        at.e = ti < end ? in_part.e : 0;
        at.k = ti < end ? in_part.k : 0;
        at.v = ti < end ? in_part.v : 0;
        ++ti;
    };
    float m_run = -INFINITY;
    float l_run = 0.f;
    f32x4_t O[8];
#pragma unroll
    for (int c = 0; c < 8; ++c)
        O[c] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    if (ti < end) {
        Tile t;
        auto load_k = [&]() __attribute__((always_inline)) {
            load_keys(t, 0, x, part[0], at.k);
            load_keys(t, 1, x, part[1], at.k);
        };
        auto load_v = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int p = 0; p < kParts; ++p) {
                load_exps(t, p, x, part[p], at.e);
                load_values(t, p, x, part[p], at.v);
            }
        };
        place();
        load_k();
        load_v();
#pragma unroll 1
        do {
            attend_tile(t, v0, v1, qf, a.scale_log2, lg, m_run, l_run, O,
                        [&]() __attribute__((always_inline)) {
                            place();
                            load_k();
                        },
                        load_v);
        } while (ti <= end);
    }

    // ---- the waves' states into LDS (lane (g, r) holds head g, channels 32r .. 32r+31)
    const float l_tot = over_groups(l_run, [](float u, float w) { return u + w; });
    if (lr < G) {
        float *op = s_o + (wv * kUnitMaxGroup + lr) * kUnitRow + 32 * lg;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            *reinterpret_cast<f32x4_t *>(op + 8 * i) = (f32x4_t){O[0][i], O[1][i], O[2][i], O[3][i]};
            *reinterpret_cast<f32x4_t *>(op + 8 * i + 4) =
                (f32x4_t){O[4][i], O[5][i], O[6][i], O[7][i]};
        }
        if (lg == 0) {
            s_m[wv * kUnitMaxGroup + lr] = m_run;
            s_l[wv * kUnitMaxGroup + lr] = l_tot;
        }
    }
    __syncthreads();

    // ---- o = sum_w 2^(m_w - M) o_w / sum_w 2^(m_w - M) l_w
    for (int i = threadIdx.x; i < G * kHeadDim; i += kUnitThreads) {
        const int g = i / kHeadDim;
        const int d = i - g * kHeadDim;
        float M = -INFINITY;
#pragma unroll
        for (int w = 0; w < kUnitWaves; ++w)
            M = fmaxf(M, s_m[w * kUnitMaxGroup + g]);
        M = M == -INFINITY ? 0.f : M;  // (no tokens: every weight below is 0)
        float lsum = 0.f, acc = 0.f;
#pragma unroll
        for (int w = 0; w < kUnitWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(s_m[w * kUnitMaxGroup + g] - M);
            lsum += f * s_l[w * kUnitMaxGroup + g];
            acc += f * s_o[(w * kUnitMaxGroup + g) * kUnitRow + d];
        }
        const float inv = lsum > 0.f ? 1.f / lsum : 0.f;
        store_out(a.out, a.out_bf16, ((int64_t)t.unit * G + g) * kHeadDim + d, acc * inv);
    }
}

// Whether a call takes one workgroup per unit; list_bound: k_max, or the block table's width.
bool unit_path(const sparrow_shape_t &s, int64_t list_bound)
{
    const int64_t units = (int64_t)s.batch * s.num_kv_heads, cus = device_cus();
    const int64_t tokens = list_bound * s.page_size;
    return s.num_q_heads / s.num_kv_heads <= kUnitMaxGroup && list_bound <= kBatch &&
           ((tokens <= kUnitMaxTokens && units <= kUnitsPerCu * cus) ||
            (tokens <= 2 * kUnitMaxTokens && units > cus / 2 && units <= cus));
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
    // One workgroup per CU, four waves with two tiles in flight each: 64 KiB, which keeps the memory
    // busy; more waves only add partials and uneven ends (1 / 2 workgroups: 64 sequences of 8K-32K
    // tokens 448 / 450 us, 256 sequences at 10 % 259 / 265, 128 units of 1024 tokens 16.7 / 19.6, on one
    // box in turn).
    int64_t waves = (int64_t)device_cus() * kAttnWaves;
    waves = waves < kMaxWaves ? waves : kMaxWaves;
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
    a.scale_log2 = scale * 1.4426950408889634f;
    if (unit_path(s, idx != nullptr ? k_max : s.max_pages_per_seq)) {
        auto unit = idx != nullptr ? k_attn_unit_e4m3<true> : k_attn_unit_e4m3<false>;
        hipLaunchKernelGGL(unit, dim3((unsigned)units), dim3(kUnitThreads), 0, stream, x);
        return hipGetLastError();
    }
    auto kernel = idx != nullptr ? k_attn_stream_e4m3<true> : k_attn_stream_e4m3<false>;
    hipLaunchKernelGGL(kernel, dim3(waves / kAttnWaves), dim3(kAttnThreads), plan.lds_bytes,
                       stream, x);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : launch_attn_merge(a, stream);
}

}  // namespace sparrow
