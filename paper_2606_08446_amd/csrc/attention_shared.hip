// Decode attention of groups of sequences whose first tokens are the same: the samples of one prompt.
// The shared pages are read once per group for all of its query rows, the others per sequence, and the
// parts are joined by their softmax maxima and sums:
//
//   z_t = scale q . K[t],  m = max z,  l = sum e^(z - m),  o = sum e^(z - m) V[t]   of each part,
//   out = sum o e^(m - M) / sum l e^(m - M),  M the largest m.
//
// Work split.  A unit is (group, KV head, block of kTiles * 16 query rows) over the group's shared
// tokens, or (sequence, KV head) over the sequence's own.  All units' 32-token tiles are laid end
// to end and every wave takes one equal, contiguous range of them.  Each part of a unit that a
// wave finds in its range leaves (m, l, o) in the workspace, in slot wave + unit, which grows along
// the order; k_shared_merge joins what belongs to a query head.
//
// Per 32-token tile a wave reads K and V once, straight into MFMA operands, for all of its row tiles:
//   logits  D[t][row] = sum_d K[t][d] q[row][d]  - 2 x 4 x mfma_f32_16x16x32_bf16: lane (row lr, lg)
//           then holds tokens 4 lg .. 4 lg + 3 of both halves;
//   O^T[d][row] += sum_t V[t][d] p[t][row]       - 8 x mfma_f32_16x16x32_bf16, whose 32 terms are
//           taken in the order the logits left them in: lane group lg has tokens 4 lg + j of the first
//           half, then of the second.  V rows are loaded 8 channels a lane, tile c takes element c.
// The softmax numerators enter the second product as bf16 for bf16 outputs (half a step of the output's
// own type each) and as three bf16 terms, all of their 24 bits, for fp32 ones.
#include "attention_shared.h"

#include <cfloat>

#include "attention_split.h"
#include "common.h"
#include "wave.h"

namespace sparrow {
namespace {

constexpr int kSharedThreads = 256;
constexpr int kSharedWaves = kSharedThreads / 64;
constexpr int kTileTokens = 32;
constexpr float kNoLogit = -FLT_MAX;  // a part's maximum before its first token

struct SharedArgs {
    const uint16_t *q, *k_cache, *v_cache;
    const int32_t *block_table, *seq_lens, *cu_groups, *prefix_lens;
    int32_t *plan_off;   // [groups + batch + 1] tiles of a KV head before each entry
    int32_t *seq_group;  // [batch] its group, -1: none
    int32_t *plan_cu;    // [groups + 1] the groups' first sequences as the plan took them
    float *o_group, *ml_group;  // [waves + group units][kTiles * 16] rows
    float *o_seq, *ml_seq;      // [waves + sequence units][G] rows
    void *out;
    int64_t num_phys;
    int groups, batch, num_q_heads, num_kv_heads, ps, ps_log2, max_pages, out_bf16;
    int max_waves, min_tiles;
    float scale_log2;
};

// Waves that share P tiles out, and which of them has one.
__device__ __forceinline__ int64_t wave_count(const SharedArgs &a, int64_t P)
{
    const int64_t W = (P + a.min_tiles - 1) / a.min_tiles;
    return W < a.max_waves ? W : a.max_waves;
}

__device__ __forceinline__ int wave_of(int64_t pos, int64_t P, int64_t W)
{
    return (int)(((pos + 1) * W - 1) / P);  // the last w with w P / W <= pos
}

// A number for the units of groups before g, in steps that leave room for each group's row blocks.
__device__ __forceinline__ int unit_base(const SharedArgs &a, int g, int begin, int rows_per_unit)
{
    return a.num_kv_heads * (begin * (a.num_q_heads / a.num_kv_heads) / rows_per_unit + g);
}

// LDS of a workgroup's plan: the tiles before each entry (groups, then sequences), the sequences' first
// own page with their tiles, the groups' shared tokens, the groups' first sequences.
struct Plan {
    int32_t *off, *seq, *lim, *cu;
    __device__ __forceinline__ Plan(int32_t *lds, const SharedArgs &a)
        : off(lds), seq(off + a.groups + a.batch + 1), lim(seq + a.batch), cu(lim + a.groups)
    {
    }
};

// seq entries: own tiles (16 bits) under the first own page.
constexpr int kSeqTileBits = 16;
static_assert(SPARROW_MAX_PAGES_PER_SEQ * 128 / kTileTokens < 1 << kSeqTileBits, "tiles of a sequence");
static_assert(SPARROW_MAX_PAGES_PER_SEQ < 1 << (31 - kSeqTileBits), "pages of a sequence");

template <int kTiles>
__device__ void make_plan(const SharedArgs &a, const Plan &p, int32_t *s_tmp)
{
    const int tid = threadIdx.x;
    const int G = a.num_q_heads / a.num_kv_heads;
    // ---- the groups' first sequences, inside the batch and never decreasing
    {
        const int n = a.groups ? a.groups + 1 : 0, per = (n + kSharedThreads - 1) / kSharedThreads;
        const int g0 = min(n, tid * per), g1 = min(n, g0 + per);
        uint32_t top = 0;
        for (int g = g0; g < g1; ++g)
            top = max(top, (uint32_t)min(max(a.cu_groups[g], 0), a.batch));
        const uint32_t incl =
            wave_scan(top, 0u, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
        if ((tid & 63) == 63)
            s_tmp[tid >> 6] = (int32_t)incl;
        __syncthreads();
        top = __shfl_up(incl, 1, 64);
        top = (tid & 63) ? top : 0u;
        for (int w = 0; w < tid >> 6; ++w)
            top = max(top, (uint32_t)s_tmp[w]);
        for (int g = g0; g < g1; ++g) {
            top = max(top, (uint32_t)min(max(a.cu_groups[g], 0), a.batch));
            p.cu[g] = (int32_t)top;
            if (g < a.groups)
                p.lim[g] = 0;
            if (blockIdx.x == 0)
                a.plan_cu[g] = (int32_t)top;
        }
        __syncthreads();
    }
    for (int b = tid; b < a.batch; b += kSharedThreads) {
        const int L = clamp_len(a.seq_lens[b], a.ps, a.max_pages);
        int lo = 0, hi = a.groups;  // the last group that begins at or before b
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (p.cu[mid] <= b)
                lo = mid;
            else
                hi = mid;
        }
        int first = 0, group = -1;
        if (a.groups && p.cu[lo] <= b && b < p.cu[lo + 1] && p.cu[lo + 1] - p.cu[lo] > 1) {
            group = lo;
            first = min(max(a.prefix_lens[lo], 0) >> a.ps_log2, a.max_pages);
            atomicMax(&p.lim[lo], min(L, first << a.ps_log2));
        }
        const int own = max(0, L - (first << a.ps_log2));
        p.seq[b] = first << kSeqTileBits | (own + kTileTokens - 1) / kTileTokens;
        if (blockIdx.x == 0)
            a.seq_group[b] = group;
    }
    __syncthreads();
    // ---- exclusive prefix of the entries' tiles
    const int n = a.groups + a.batch;
    auto tiles = [&](int e) -> int {
        if (e >= a.groups)
            return p.seq[e - a.groups] & ((1 << kSeqTileBits) - 1);
        const int rows = (p.cu[e + 1] - p.cu[e]) * G;
        return (p.lim[e] + kTileTokens - 1) / kTileTokens * ((rows + 16 * kTiles - 1) / (16 * kTiles));
    };
    const int per = (n + kSharedThreads - 1) / kSharedThreads;
    const int e0 = min(n, tid * per), e1 = min(n, e0 + per);
    int local = 0;
    for (int e = e0; e < e1; ++e)
        local += tiles(e);
    const int incl = (int)wave_scan_add((uint32_t)local);
    if ((tid & 63) == 63)
        s_tmp[tid >> 6] = incl;
    __syncthreads();
    int run = incl - local;
    for (int w = 0; w < tid >> 6; ++w)
        run += s_tmp[w];
    for (int e = e0; e < e1; ++e) {
        p.off[e] = run;
        run += tiles(e);
    }
    if (tid == kSharedThreads - 1)
        p.off[n] = run;
    __syncthreads();
    if (blockIdx.x == 0)
        for (int e = tid; e <= n; e += kSharedThreads)
            a.plan_off[e] = p.off[e];
}

// K and V of a tile's half: A operands of the logits, rows 4 lg + j of V.
struct Half {
    u32x4_t k[4], v[4];
};

__device__ __forceinline__ void load_half(Half &c, const uint16_t *kbase, const uint16_t *vbase, int lr,
                                          int lg)
{
    const uint16_t *kp = kbase + lr * kHeadDim + 8 * lg;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        c.k[i] = ld16_nt(kp + 32 * i);
    const uint16_t *vp = vbase + 4 * lg * kHeadDim + 8 * lr;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        c.v[j] = ld16_nt(vp + j * kHeadDim);
}

struct Tile {
    Half h[2];
    int tok;        // its first token
    bool live[2];   // a half inside the unit's tokens, on a page that is there
};

// A wave's part of a unit.
struct Part {
    const int32_t *table;  // the block-table row that its pages are read from
    int h, lim;            // KV head; its tokens end here
    int rows, row0;        // query rows of this block, and the first one's number in its entry
    int b0;                // the entry's first sequence
};

template <int kTiles, int kTerms>
struct Streamer {
    const SharedArgs &a;
    const int lane, lr, lg, G;
    bf16x8_t q[kTiles][4];
    int len[kTiles];  // tokens of the row's sequence
    int full;         // tokens that every row has
    float m[kTiles], l[kTiles];
    f32x4_t O[kTiles][8];
    // the block table's entries [page0, page0 + 64) and the 64 behind them, one a lane
    int page0, phys, phys_next;

    __device__ __forceinline__ Streamer(const SharedArgs &args)
        : a(args), lane(threadIdx.x & 63), lr(lane & 15), lg(lane >> 4),
          G(args.num_q_heads / args.num_kv_heads)
    {
    }

    __device__ __forceinline__ int entry(const Part &u, int page) const
    {
        return page << a.ps_log2 < u.lim ? u.table[page] : -1;
    }

    __device__ __forceinline__ void begin(const Part &u, int tok)
    {
        page0 = tok >> a.ps_log2;
        phys = entry(u, page0 + lane);
        phys_next = entry(u, page0 + 64 + lane);
        int least = 0x7fffffff;
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const int r = 16 * t + lr;
            const bool in = r < u.rows;
            const int b = u.b0 + (u.row0 + r) / G, j = (u.row0 + r) % G;
            len[t] = in ? clamp_len(a.seq_lens[in ? b : u.b0], a.ps, a.max_pages) : 0x7fffffff;
            least = min(least, len[t]);
            const uint16_t *row = a.q + ((int64_t)b * a.num_q_heads + u.h * G + j) * kHeadDim + 8 * lg;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                u32x4_t v = {0u, 0u, 0u, 0u};
                if (in)
                    v = ld16(row + 32 * i);
                q[t][i] = __builtin_bit_cast(bf16x8_t, v);
            }
            m[t] = kNoLogit;
            l[t] = 0.f;
#pragma unroll
            for (int c = 0; c < 8; ++c)
                O[t][c] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
        }
        full = min((int)wave_min((uint32_t)least), u.lim);
    }

    __device__ __forceinline__ void issue(const Part &u, int tok, Tile &t)
    {
        t.tok = tok;
        if ((tok >> a.ps_log2) >= page0 + 64) {
            page0 += 64;
            phys = phys_next;
            phys_next = entry(u, page0 + 64 + lane);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = tok + 16 * i;
            const int ph = __builtin_amdgcn_readlane(phys, (at >> a.ps_log2) - page0);
            t.live[i] = ph >= 0 && ph < a.num_phys && at < u.lim;
            if (t.live[i]) {
                const int64_t off = (((int64_t)ph * a.num_kv_heads + u.h) * a.ps + (at & (a.ps - 1))) *
                                    kHeadDim;
                load_half(t.h[i], a.k_cache + off, a.v_cache + off, lr, lg);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    t.h[i].k[j] = t.h[i].v[j] = (u32x4_t){0u, 0u, 0u, 0u};
            }
        }
    }

    __device__ __forceinline__ void attend(const Part &u, Tile &t)
    {
        bf16x8_t p[kTerms][kTiles];
        const bool whole = t.live[0] && t.live[1] && t.tok + kTileTokens <= full;
        if (!whole) {  // tokens past the unit's: zero V (cache slots may hold anything)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (t.tok + 16 * i + 4 * lg + j >= u.lim)
                        t.h[i].v[j] = (u32x4_t){0u, 0u, 0u, 0u};
        }
#pragma unroll
        for (int r = 0; r < kTiles; ++r) {
            f32x4_t s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        __builtin_bit_cast(bf16x8_t, t.h[i].k[j]), q[r][j], s[i], 0, 0, 0);
            float z[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                z[e] = s[e >> 2][e & 3] * a.scale_log2;
            if (!whole) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int at = t.tok + 16 * (e >> 2) + 4 * lg + (e & 3);
                    z[e] = t.live[e >> 2] && at < u.lim && at < len[r] ? z[e] : -INFINITY;
                }
            }
            float top = fmaxf(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])),
                              fmaxf(fmaxf(z[4], z[5]), fmaxf(z[6], z[7])));
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float m_new = fmaxf(m[r], top);
            const float alpha = exp2f(m[r] - m_new);
            m[r] = m_new;
            float sum = 0.f;
            u32x4_t pk[kTerms];
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                float x0 = exp2f(z[e] - m_new), x1 = exp2f(z[e + 1] - m_new);
                if (kTerms > 1)
                    sum += x0 + x1;
#pragma unroll
                for (int k = 0; k < kTerms; ++k) {
                    const uint32_t b = pack_bf16(x0, x1);
                    pk[k][e >> 1] = b;
                    if (kTerms == 1) {
                        sum += bf16_lo(b) + bf16_hi(b);  // (the weights as they are used)
                    } else {
                        x0 -= bf16_lo(b);
                        x1 -= bf16_hi(b);
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < kTerms; ++k)
                p[k][r] = __builtin_bit_cast(bf16x8_t, pk[k]);
            l[r] = l[r] * alpha + sum;
            if (__ballot(alpha != 1.f)) {
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    O[r][c] *= alpha;
            }
        }
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const u32x4_t av = {
                pair_of(t.h[0].v[0], t.h[0].v[1], c), pair_of(t.h[0].v[2], t.h[0].v[3], c),
                pair_of(t.h[1].v[0], t.h[1].v[1], c), pair_of(t.h[1].v[2], t.h[1].v[3], c)};
#pragma unroll
            for (int r = 0; r < kTiles; ++r)
#pragma unroll
                for (int k = 0; k < kTerms; ++k)
                    O[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        __builtin_bit_cast(bf16x8_t, av), p[k][r], O[r][c], 0, 0, 0);
        }
    }

    // (m, l, o) of the part's rows to slot `slot` of slots of `stride` rows.
    __device__ __forceinline__ void write(const Part &u, float *o, float *ml, int64_t slot, int stride)
    {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            float sum = l[t] + __shfl_xor(l[t], 16, 64);
            sum += __shfl_xor(sum, 32, 64);
            const int r = 16 * t + lr;
            if (r >= u.rows)
                continue;
            const int64_t row = slot * stride + r;
            float *op = o + row * kHeadDim + 32 * lg;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                st16(op + 8 * i, __builtin_bit_cast(u32x4_t, (f32x4_t){O[t][0][i], O[t][1][i],
                                                                      O[t][2][i], O[t][3][i]}));
                st16(op + 8 * i + 4, __builtin_bit_cast(u32x4_t, (f32x4_t){O[t][4][i], O[t][5][i],
                                                                          O[t][6][i], O[t][7][i]}));
            }
            if (lg == 0) {
                ml[2 * row] = m[t];
                ml[2 * row + 1] = sum;
            }
        }
    }

    // Tiles [t0, t0 + n) of a unit whose first token is `first`.
    __device__ __forceinline__ void run(const Part &u, int first, int t0, int n)
    {
        const int tok = first + kTileTokens * t0;
        begin(u, tok);
        Tile x, y;
        issue(u, tok, x);
        for (int i = 0; i < n; i += 2) {
            if (i + 1 < n)
                issue(u, tok + kTileTokens * (i + 1), y);
            attend(u, x);
            if (i + 1 >= n)
                break;
            if (i + 2 < n)
                issue(u, tok + kTileTokens * (i + 2), x);
            attend(u, y);
        }
    }
};

template <int kTiles, int kTerms>
__global__ __launch_bounds__(kSharedThreads, kTiles == 4 ? 1 : 2) void k_shared_stream(SharedArgs a)
{
    extern __shared__ int32_t s_plan[];
    __shared__ int32_t s_tmp[kSharedWaves];
    const Plan plan(s_plan, a);
    make_plan<kTiles>(a, plan, s_tmp);

    constexpr int kRows = 16 * kTiles;
    const int Hkv = a.num_kv_heads, G = a.num_q_heads / Hkv, n = a.groups + a.batch;
    const int64_t P = (int64_t)plan.off[n] * Hkv;
    const int64_t W = wave_count(a, P);
    const int w = blockIdx.x * kSharedWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (w >= W)
        return;
    int64_t pos = (int64_t)w * P / W;
    const int64_t end = (int64_t)(w + 1) * P / W;
    // the entry that holds pos: the last whose offset is at or before it (empty ones share it)
    int e = 0;
    {
        int span = n;
        const int lane = threadIdx.x & 63;
        while (span > 1) {
            const int step = (span + 63) >> 6;
            const bool ok = lane * step < span && (int64_t)plan.off[e + lane * step] * Hkv <= pos;
            const int t = __popcll(__ballot(ok)) - 1;
            e += t * step;
            span = min(step, span - t * step);
        }
        e = __builtin_amdgcn_readfirstlane(e);
    }
    Streamer<kTiles, kTerms> st(a);
    while (pos < end) {
        while (plan.off[e + 1] == plan.off[e])
            ++e;
        const int64_t first = (int64_t)__builtin_amdgcn_readfirstlane(plan.off[e]) * Hkv;
        const int cnt = __builtin_amdgcn_readfirstlane(plan.off[e + 1] - plan.off[e]);
        const int rel = (int)(pos - first);  // (below the tiles of one entry: 2^31 at most)
        const int h = rel / cnt;
        int at = rel - h * cnt;
        Part u;
        u.h = h;
        int tok0, tiles;
        int64_t slot;
        if (e < a.groups) {
            const int b0 = __builtin_amdgcn_readfirstlane(plan.cu[e]);
            const int rows = (__builtin_amdgcn_readfirstlane(plan.cu[e + 1]) - b0) * G;
            const int blocks = (rows + kRows - 1) / kRows;
            tiles = cnt / blocks;
            const int rb = at / tiles;
            at -= rb * tiles;
            u.b0 = b0;
            u.row0 = rb * kRows;
            u.rows = min(kRows, rows - u.row0);
            u.lim = __builtin_amdgcn_readfirstlane(plan.lim[e]);
            tok0 = 0;
            slot = (int64_t)w + unit_base(a, e, b0, kRows) + h * blocks + rb;
        } else {
            const int b = e - a.groups;
            const int packed = __builtin_amdgcn_readfirstlane(plan.seq[b]);
            tiles = cnt;
            u.b0 = b;
            u.row0 = 0;
            u.rows = G;
            u.lim = clamp_len(a.seq_lens[b], a.ps, a.max_pages);
            tok0 = (packed >> kSeqTileBits) << a.ps_log2;
            slot = (int64_t)w + b * Hkv + h;
        }
        u.table = a.block_table + (int64_t)u.b0 * a.max_pages;
        const int64_t left = end - pos;
        const int take = tiles - at < left ? tiles - at : (int)left;
        st.run(u, tok0, at, take);
        if (e < a.groups)
            st.write(u, a.o_group, a.ml_group, slot, kRows);
        else
            st.write(u, a.o_seq, a.ml_seq, slot, G);
        pos += take;
        if (h == Hkv - 1 && pos == first + (int64_t)cnt * Hkv)
            ++e;
    }
}

// One workgroup per query head and sequence: its parts from the group's waves and from its own, eight
// at a time.
__global__ __launch_bounds__(kSharedThreads) void k_shared_merge(SharedArgs a, int rows_per_unit)
{
    constexpr int kSides = kSharedThreads / 32;
    __shared__ float s_o[kSides][kHeadDim], s_l[kSides], s_m[kSharedWaves];
    const int row = blockIdx.x;  // [batch][num_q_heads]
    const int b = row / a.num_q_heads, hq = row - b * a.num_q_heads;
    const int Hkv = a.num_kv_heads, G = a.num_q_heads / Hkv, h = hq / G, j = hq - h * G;
    const int n = a.groups + a.batch;
    const int64_t P = (int64_t)a.plan_off[n] * Hkv;
    const int64_t W = P ? wave_count(a, P) : 1;
    // ---- the parts: n_g slots of the group from g0, n_s of the sequence from s0
    int64_t g0 = 0, s0 = 0;
    int n_g = 0, n_s = 0, g_row = 0;
    const int g = a.seq_group[b];
    if (g >= 0) {
        const int first = a.plan_off[g], cnt = a.plan_off[g + 1] - first;
        if (cnt > 0) {
            const int b0 = a.plan_cu[g];
            const int rows = (a.plan_cu[g + 1] - b0) * G;
            const int blocks = (rows + rows_per_unit - 1) / rows_per_unit, tiles = cnt / blocks;
            const int r = (b - b0) * G + j, rb = r / rows_per_unit;
            g_row = r - rb * rows_per_unit;
            const int64_t p0 = (int64_t)first * Hkv + (int64_t)h * cnt + (int64_t)rb * tiles;
            const int w0 = wave_of(p0, P, W);
            n_g = wave_of(p0 + tiles - 1, P, W) - w0 + 1;
            g0 = (int64_t)w0 + unit_base(a, g, b0, rows_per_unit) + h * blocks + rb;
        }
    }
    {
        const int first = a.plan_off[a.groups + b], cnt = a.plan_off[a.groups + b + 1] - first;
        if (cnt > 0) {
            const int64_t p0 = (int64_t)first * Hkv + (int64_t)h * cnt;
            const int w0 = wave_of(p0, P, W);
            n_s = wave_of(p0 + cnt - 1, P, W) - w0 + 1;
            s0 = (int64_t)w0 + b * Hkv + h;
        }
    }
    auto part_row = [&](int i) -> int64_t {
        return i < n_g ? (g0 + i) * rows_per_unit + g_row : (s0 + (i - n_g)) * G + j;
    };
    const int parts = n_g + n_s;
    float top = kNoLogit;
    for (int i = threadIdx.x; i < parts; i += kSharedThreads)
        top = fmaxf(top, (i < n_g ? a.ml_group : a.ml_seq)[2 * part_row(i)]);
    top = wave_max_f(top);
    if ((threadIdx.x & 63) == 0)
        s_m[threadIdx.x >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
    const int side = threadIdx.x >> 5, c = 4 * (threadIdx.x & 31);
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
    for (int i = side; i < parts; i += kSides) {
        const int64_t r = part_row(i);
        const float *ml = (i < n_g ? a.ml_group : a.ml_seq) + 2 * r;
        const float x = exp2f(ml[0] - top);
        l += ml[1] * x;
        o += __builtin_bit_cast(f32x4_t, ld16((i < n_g ? a.o_group : a.o_seq) + r * kHeadDim + c)) * x;
    }
    *reinterpret_cast<f32x4_t *>(&s_o[side][c]) = o;
    if (c == 0)
        s_l[side] = l;
    __syncthreads();
    if (threadIdx.x < kHeadDim) {
        float sum = 0.f, den = 0.f;
#pragma unroll
        for (int k = 0; k < kSides; ++k) {
            sum += s_o[k][threadIdx.x];
            den += s_l[k];
        }
        store_out(a.out, a.out_bf16, (int64_t)row * kHeadDim + threadIdx.x, den > 0.f ? sum / den : 0.f);
    }
}

// Row tiles of 16 that a wave takes against the shared tokens: what a group has on average.
int shared_tiles(const sparrow_shape_t &s, int groups)
{
    if (groups < 1)
        return 1;
    const int64_t rows = (int64_t)((s.batch + groups - 1) / groups) * (s.num_q_heads / s.num_kv_heads);
    return rows <= 16 ? 1 : (rows <= 32 ? 2 : 4);
}

// Resident waves of a device of `cus` compute units; the workspace is sized for kMaxCus of them.
constexpr int kMaxCus = 256;

int shared_max_waves(int tiles, int cus)
{
    return (cus < kMaxCus ? cus : kMaxCus) * kSharedWaves * (tiles == 4 ? 1 : 2);
}

struct SharedPlan {
    int tiles, waves;
    size_t plan_bytes, group_slots, seq_slots, bytes;
};

size_t round_up(size_t n) { return (n + 255) / 256 * 256; }

SharedPlan plan_shared(const sparrow_shape_t &s, int groups)
{
    SharedPlan p;
    const int G = s.num_q_heads / s.num_kv_heads;
    p.tiles = shared_tiles(s, groups);
    p.waves = shared_max_waves(p.tiles, kMaxCus);
    p.plan_bytes = round_up(sizeof(int32_t) * (2 * ((size_t)groups + s.batch) + 2));
    p.group_slots = groups ? p.waves + (size_t)s.num_kv_heads *
                                           ((size_t)s.batch * G / (16 * p.tiles) + groups)
                           : 0;
    p.seq_slots = p.waves + (size_t)s.batch * s.num_kv_heads;
    const size_t rows = p.group_slots * 16 * p.tiles + p.seq_slots * G;
    p.bytes = p.plan_bytes + rows * (kHeadDim + 2) * sizeof(float);
    return p;
}

template <int kTiles>
void launch_stream(const SharedArgs &a, size_t lds, hipStream_t stream)
{
    auto kernel = a.out_bf16 ? k_shared_stream<kTiles, 1> : k_shared_stream<kTiles, 3>;
    hipLaunchKernelGGL(kernel, dim3(a.max_waves / kSharedWaves), dim3(kSharedThreads), lds, stream, a);
}

}  // namespace

size_t shared_attention_workspace(const sparrow_shape_t &s, int groups)
{
    return plan_shared(s, groups).bytes;
}

hipError_t launch_shared_attention(const sparrow_shape_t &s, const Groups &g, const void *q,
                                   const void *k_cache, const void *v_cache,
                                   const int32_t *block_table, const int32_t *seq_lens, float scale,
                                   void *out, int out_dtype, void *workspace, hipStream_t stream)
{
    const SharedPlan p = plan_shared(s, g.n);
    SharedArgs a;
    a.q = static_cast<const uint16_t *>(q);
    a.k_cache = static_cast<const uint16_t *>(k_cache);
    a.v_cache = static_cast<const uint16_t *>(v_cache);
    a.block_table = block_table;
    a.seq_lens = seq_lens;
    a.cu_groups = g.cu;
    a.prefix_lens = g.prefix;
    a.groups = g.n;
    a.batch = s.batch;
    a.num_q_heads = s.num_q_heads;
    a.num_kv_heads = s.num_kv_heads;
    a.ps = s.page_size;
    a.ps_log2 = __builtin_ctz(s.page_size);
    a.max_pages = s.max_pages_per_seq;
    a.num_phys = s.num_phys_pages;
    a.out = out;
    a.out_bf16 = out_dtype == SPARROW_OUT_BF16;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.max_waves = shared_max_waves(p.tiles, device_cus());
    a.min_tiles = 2;
    char *ws = static_cast<char *>(workspace);
    a.plan_off = reinterpret_cast<int32_t *>(ws);
    a.seq_group = a.plan_off + g.n + s.batch + 1;
    a.plan_cu = a.seq_group + s.batch;
    const size_t group_rows = p.group_slots * 16 * p.tiles;
    const size_t seq_rows = p.seq_slots * (s.num_q_heads / s.num_kv_heads);
    a.o_group = reinterpret_cast<float *>(ws + p.plan_bytes);
    a.o_seq = a.o_group + group_rows * kHeadDim;
    a.ml_group = a.o_seq + seq_rows * kHeadDim;
    a.ml_seq = a.ml_group + group_rows * 2;
    const size_t lds = sizeof(int32_t) * (3 * (size_t)g.n + 2 * (size_t)s.batch + 2);
    if (p.tiles == 1)
        launch_stream<1>(a, lds, stream);
    else if (p.tiles == 2)
        launch_stream<2>(a, lds, stream);
    else
        launch_stream<4>(a, lds, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(k_shared_merge, dim3((unsigned)(s.batch * s.num_q_heads)), dim3(kSharedThreads), 0,
                       stream, a, 16 * p.tiles);
    return hipGetLastError();
}

}  // namespace sparrow
