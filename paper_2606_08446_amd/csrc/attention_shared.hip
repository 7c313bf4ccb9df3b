// Decode attention of groups of sequences whose first tokens are the same: the samples of one prompt.
// The shared pages are read once per group for all of its query rows, the others per sequence, and the
// parts are joined by their softmax maxima and sums:
//
//   z_t = scale q . K[t],  m = max z,  l = sum e^(z - m),  o = sum e^(z - m) V[t]   of each part,
//   out = sum o e^(m - M) / sum l e^(m - M),  M the largest m.
//
// Work split.  A group has (group, KV head, block of 64 query rows) units over its shared tokens, a sequence
// one unit per KV head over its own.  The groups' units are laid end to end in 32-token tiles and a part of
// the workgroups takes an equal, contiguous range of them each; so are the sequences' for the waves of the
// other workgroups.  Each part of a unit that falls into a range leaves (m, l, o) in the workspace, in a
// slot that grows along the order; k_shared_merge joins what belongs to a query head.
//
// A workgroup on a group's tiles (Team) brings each tile into LDS once, a fourth of it per wave, three
// tiles ahead in registers, and every wave attends with 16 of the rows.  A wave on a sequence's (Stream)
// reads its tiles straight into MFMA operands, the next one always under way.  Per tile and 16 rows:
//   logits  D[t][row] = sum_d K[t][d] q[row][d]  - 2 x 4 x mfma_f32_16x16x32_bf16: lane (row lr, lg)
//           then holds tokens 4 lg .. 4 lg + 3 of both halves;
//   O^T[d][row] += sum_t V[t][d] p[t][row]       - 8 x mfma_f32_16x16x32_bf16, whose 32 terms are
//           taken in the order the logits left them in: lane group lg has tokens 4 lg + j of the first
//           half, then of the second.  V rows are loaded 8 channels a lane, tile c takes element c.
// The softmax numerators enter the second product as three bf16 terms, which is all of their 24 bits, for
// either type of output: a bf16 one is the fp32 one rounded once.  The matrix cores have the time: with one term
// 16 groups of 16 took 866 instead of 872 us, 7 uneven ones 54 instead of 55, 8 short samples 15.0 instead of 15.1.
//
// Bound by memory: 16 groups of 16 sequences with 8K-16K shared and up to 8K own tokens read 5.46 GB in 858 us,
// 6.4 TB/s (8 x 8 of up to 4K + 4K: 627 MB in 104 us, 6.0 TB/s); the merge takes 5-9 us more.  What a group costs
// is decided by how often its tiles reach a compute unit: the same call took 1228 us with waves that each read
// them for 16 rows, and 1833 with waves that held all of a unit's rows.
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
constexpr int kRows = 16;       // query rows of a wave
constexpr int kTeamRows = kRows * kSharedWaves;
constexpr int kTerms = 3;       // bf16 terms of a softmax numerator
constexpr float kNoLogit = -FLT_MAX;  // a part's maximum before its first token

struct SharedArgs {
    const uint16_t *q, *k_cache, *v_cache;
    const int32_t *block_table, *seq_lens, *cu_groups, *prefix_lens;
    int32_t *plan_off;   // [groups + batch + 1] positions before each entry, groups' first
    int32_t *seq_group;  // [batch] its group, -1: none
    int32_t *plan_takers; // [2] workgroups of the groups, waves of the sequences
    int32_t *plan_cu;    // [groups + 1] the groups' first sequences as the plan took them
    float *o_group, *ml_group;  // [slots][kRows] rows: a slot for each 16 rows of a part
    float *o_seq, *ml_seq;      // [slots][G] rows
    void *out;
    uint32_t num_phys, page_elems;  // pages (what an int32 entry can name), elements of one
    int groups, batch, num_q_heads, num_kv_heads, ps, ps_log2, max_pages, out_bf16;
    int min_tiles;
    int step_log2;  // a position is 2^step_log2 tiles (more than one only where 2^31 would not do)
    float scale_log2;
};

// How many workgroups take the groups' positions (P1 of them) and how many waves the sequences' (P2): all of
// the launch's, in proportion, or where that would be less than min_tiles each, fewer.
struct Sides {
    uint32_t w1, w2;
    __device__ __forceinline__ Sides(const SharedArgs &a, uint32_t P1, uint32_t P2, uint32_t blocks)
    {
        w1 = (P1 + a.min_tiles - 1) / a.min_tiles;
        w2 = (P2 + a.min_tiles - 1) / a.min_tiles;
        if (w1 + (w2 + kSharedWaves - 1) / kSharedWaves > blocks) {
            const float c1 = (float)P1;
            uint32_t n = (uint32_t)(c1 / (c1 + (float)P2) * blocks + 0.5f);
            n = P1 ? max(n, 1u) : 0u;
            n = P2 ? min(n, blocks - 1) : blocks;
            w1 = min(w1, n);
            w2 = min(w2, (blocks - n) * kSharedWaves);
        }
    }
};

// One side's positions shared out over W takers: the first r take q + 1 of them, the others q.
struct Share {
    uint32_t W, q, r;
    __device__ __forceinline__ Share(uint32_t P, uint32_t takers) : W(takers)
    {
        q = W ? P / W : 1;
        r = P - W * q;
    }
    __device__ __forceinline__ uint32_t begin(uint32_t w) const { return w * q + min(w, r); }
    __device__ __forceinline__ uint32_t taker_of(uint32_t pos) const
    {
        const uint32_t big = r * (q + 1);
        return pos < big ? pos / (q + 1) : r + (pos - big) / q;
    }
};

// Row blocks of 16 of the units before one of a group that begins with sequence `begin`, in steps that leave
// room for each group's (at most begin * G / kRows + g of them for a KV head).
__device__ __forceinline__ uint32_t blocks_before(const SharedArgs &a, int g, int begin, int rows, int h,
                                                  int row0)
{
    const int G = a.num_q_heads / a.num_kv_heads;
    return a.num_kv_heads * (begin * G / kRows + g) + h * ((rows + kRows - 1) / kRows) + row0 / kRows;
}

// LDS of a workgroup's plan: the positions before each entry (groups, then sequences), each sequence's first
// own page with its own positions, each group's shared tokens and first sequence.
struct Plan {
    int32_t *off, *seq, *lim, *cu;
    __device__ __forceinline__ Plan(int32_t *lds, const SharedArgs &a)
        : off(lds), seq(off + a.groups + a.batch + 1), lim(seq + a.batch), cu(lim + a.groups)
    {
    }
};

constexpr size_t plan_lds(size_t batch, size_t groups)
{
    return sizeof(int32_t) * (3 * groups + 2 * batch + 2);
}

// A unit takes kPartCost positions more than it has: what a part costs beside its tiles.
constexpr int kPartCost = 2;

// seq entries: own positions (16 bits) under the first own page.
constexpr int kSeqTileBits = 16;
static_assert(SPARROW_MAX_PAGES_PER_SEQ * 128 / kTileTokens < 1 << kSeqTileBits, "tiles of a sequence");
static_assert(SPARROW_MAX_PAGES_PER_SEQ < 1 << (31 - kSeqTileBits), "pages of a sequence");

__device__ __forceinline__ int positions_of(const SharedArgs &a, int tokens)
{
    const int log2 = 5 + a.step_log2;
    return (tokens + (1 << log2) - 1) >> log2;
}
static_assert(kTileTokens == 1 << 5, "positions_of");

__device__ __forceinline__ int with_cost(int positions)
{
    return positions ? positions + kPartCost : 0;
}

// pages: LDS of the groups' size, scratch.
__device__ void make_plan(const SharedArgs &a, const Plan &p, int32_t *pages, int32_t *s_tmp)
{
    const int tid = threadIdx.x;
    const int Hkv = a.num_kv_heads, G = a.num_q_heads / Hkv;
    for (int g = tid; g <= a.groups; g += kSharedThreads) {
        p.cu[g] = a.groups ? min(max(a.cu_groups[g], 0), a.batch) : 0;
        if (g < a.groups) {
            pages[g] = min(max(a.prefix_lens[g], 0) >> a.ps_log2, a.max_pages);
            p.lim[g] = 0;
        }
    }
    for (int b = tid; b < a.batch; b += kSharedThreads)
        p.seq[b] = clamp_len(a.seq_lens[b], a.ps, a.max_pages);
    __syncthreads();
    bool falls = false;
    for (int g = tid; g < a.groups; g += kSharedThreads)
        falls = falls || p.cu[g + 1] < p.cu[g];
    if (__syncthreads_or(falls)) {  // (no order that a caller should give)
        if (tid == 0)
            for (int g = 0; g < a.groups; ++g)
                p.cu[g + 1] = max(p.cu[g + 1], p.cu[g]);
        __syncthreads();
    }
    for (int b = tid; b < a.batch; b += kSharedThreads) {
        const int L = p.seq[b];
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
            first = pages[lo];
            atomicMax(&p.lim[lo], min(L, first << a.ps_log2));
        }
        p.seq[b] = first << kSeqTileBits | positions_of(a, max(0, L - (first << a.ps_log2)));
        if (blockIdx.x == 0)
            a.seq_group[b] = group;
    }
    __syncthreads();
    // ---- exclusive prefix of the entries' positions, over all KV heads
    const int n = a.groups + a.batch;
    auto positions = [&](int e) -> int {
        if (e >= a.groups)
            return Hkv * with_cost(p.seq[e - a.groups] & ((1 << kSeqTileBits) - 1));
        return Hkv * with_cost(positions_of(a, p.lim[e])) *
               (((p.cu[e + 1] - p.cu[e]) * G + kTeamRows - 1) / kTeamRows);
    };
    const int per = (n + kSharedThreads - 1) / kSharedThreads;
    const int e0 = min(n, tid * per), e1 = min(n, e0 + per);
    int local = 0;
    for (int e = e0; e < e1; ++e)
        local += positions(e);
    const int incl = (int)wave_scan_add((uint32_t)local);
    if ((tid & 63) == 63)
        s_tmp[tid >> 6] = incl;
    __syncthreads();
    int run = incl - local;
    for (int w = 0; w < tid >> 6; ++w)
        run += s_tmp[w];
    for (int e = e0; e < e1; ++e) {
        p.off[e] = run;
        run += positions(e);
    }
    if (tid == kSharedThreads - 1)
        p.off[n] = run;
    __syncthreads();
    if (blockIdx.x == 0) {
        for (int e = tid; e <= n; e += kSharedThreads)
            a.plan_off[e] = p.off[e];
        for (int g = tid; g <= a.groups; g += kSharedThreads)
            a.plan_cu[g] = p.cu[g];
    }
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

// The last of n entries whose positions begin at or before pos (empty ones share their place).
__device__ __forceinline__ int entry_at(const int32_t *off, int n, uint32_t pos)
{
    const int lane = threadIdx.x & 63;
    int e = 0, span = n;
    while (span > 1) {
        const int step = (span + 63) >> 6;
        const bool ok = lane * step < span && (uint32_t)off[e + lane * step] <= pos;
        const int t = __popcll(__ballot(ok)) - 1;
        e += t * step;
        span = min(step, span - t * step);
    }
    return __builtin_amdgcn_readfirstlane(e);
}

// A taker's part of a unit.
struct Part {
    const int32_t *table;  // the block-table row that its pages are read from
    int h, lim;            // KV head; its tokens end here
    int rows, row0;        // query rows of this unit, and the first one's number in its entry
    int b0;                // the entry's first sequence
    uint32_t slot;
    int tok, tiles;        // its first token, its tiles
};

// The parts of a range, one after another.
template <bool kTeam>
struct Walk {
    const SharedArgs &a;
    const Plan &plan;
    const int w, Hkv, G;
    const int32_t *off;
    uint32_t pos, end;
    int e;

    __device__ __forceinline__ Walk(const SharedArgs &args, const Plan &p, int w_, const Share &s)
        : a(args), plan(p), w(w_), Hkv(args.num_kv_heads), G(args.num_q_heads / args.num_kv_heads),
          off(p.off + (kTeam ? 0 : args.groups))
    {
        const uint32_t before = __builtin_amdgcn_readfirstlane(off[0]);
        pos = before + s.begin(w);
        end = before + s.begin(w + 1);
        e = entry_at(off, kTeam ? a.groups : a.batch, pos);
    }

    __device__ __forceinline__ bool next(Part &u)
    {
        while (pos < end) {
            while (off[e + 1] == off[e])
                ++e;
            const uint32_t first = __builtin_amdgcn_readfirstlane(off[e]);
            const int step = kTileTokens << a.step_log2;
            uint32_t at, unit;
            if (kTeam) {
                u.b0 = __builtin_amdgcn_readfirstlane(plan.cu[e]);
                u.lim = __builtin_amdgcn_readfirstlane(plan.lim[e]);
                const int rows = (__builtin_amdgcn_readfirstlane(plan.cu[e + 1]) - u.b0) * G;
                const uint32_t blocks = (rows + kTeamRows - 1) / kTeamRows;
                unit = with_cost(positions_of(a, u.lim));
                const uint32_t n = (pos - first) / unit;
                at = pos - first - n * unit;
                u.h = n / blocks;
                u.row0 = (n - u.h * blocks) * kTeamRows;
                u.rows = min(kTeamRows, rows - u.row0);
                u.slot = w * kSharedWaves + blocks_before(a, e, u.b0, rows, u.h, u.row0);
                u.tok = 0;
            } else {
                const int packed = __builtin_amdgcn_readfirstlane(plan.seq[e]);
                unit = with_cost(packed & ((1 << kSeqTileBits) - 1));
                u.b0 = e;
                u.lim = clamp_len(a.seq_lens[e], a.ps, a.max_pages);
                u.h = (pos - first) / unit;
                at = pos - first - u.h * unit;
                u.slot = w + e * Hkv + u.h;
                u.row0 = 0;
                u.rows = G;
                u.tok = packed >> kSeqTileBits << a.ps_log2;
            }
            u.table = a.block_table + (int64_t)u.b0 * a.max_pages;
            const uint32_t take = min(unit - at, end - pos);
            pos += take;
            if (pos == (uint32_t)__builtin_amdgcn_readfirstlane(off[e + 1]))
                ++e;
            const int from = max((int)at - kPartCost, 0), to = (int)(at + take) - kPartCost;
            if (to > from) {
                u.tok += from * step;
                // (tiles of the last position may lie behind the unit's tokens)
                u.tiles = min((to - from) << a.step_log2, (u.lim - u.tok + kTileTokens - 1) / kTileTokens);
                return true;
            }
        }
        return false;
    }
};

// 64 entries of a block-table row from `page0` on and the 64 behind them, one a lane.
struct Window {
    int page0, phys, phys_next;

    __device__ __forceinline__ static int entry(const SharedArgs &a, const Part &u, int page)
    {
        return page << a.ps_log2 < u.lim ? u.table[page] : -1;
    }
    __device__ __forceinline__ void begin(const SharedArgs &a, const Part &u, int lane)
    {
        page0 = u.tok >> a.ps_log2;
        phys = entry(a, u, page0 + lane);
        phys_next = entry(a, u, page0 + 64 + lane);
    }
    // Moves on to token `tok`, at most a window further than the one before.
    __device__ __forceinline__ void reach(const SharedArgs &a, const Part &u, int tok, int lane)
    {
        if ((tok >> a.ps_log2) >= page0 + 64) {
            page0 += 64;
            phys = phys_next;
            phys_next = entry(a, u, page0 + 64 + lane);
        }
    }
    // Where the 16 tokens from `at` on lie in the caches, in elements; 0 and false: nowhere.
    __device__ __forceinline__ int64_t place(const SharedArgs &a, const Part &u, int at, bool &live) const
    {
        const int ph = __builtin_amdgcn_readlane(phys, ((at >> a.ps_log2) - page0) & 63);
        live = (uint32_t)ph < a.num_phys && at < u.lim;  // (a negative entry is above any count)
        return live ? (int64_t)((uint64_t)(uint32_t)ph * a.page_elems) +
                          ((u.h << a.ps_log2) + (at & (a.ps - 1))) * kHeadDim
                    : 0;
    }
};

// A row's value over its four lanes (a row is in lanes lr, 16 + lr, 32 + lr, 48 + lr): swaps of 16-lane rows
// and of halves with a copy, which leave a lane its own and its partner's.
template <typename Op>
__device__ __forceinline__ float over_groups(float x, Op op)
{
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// 16 query rows of a part at work, by one wave.
struct Rows {
    const SharedArgs &a;
    const int lane, lr, lg, G;
    bf16x8_t q[4];
    int len;   // tokens of the row's sequence
    int full;  // tokens that every row has
    int ends;  // where the first row with tokens ends, if that is inside the unit
    int lim, rows;
    float m, l;
    f32x4_t O[8];

    __device__ __forceinline__ Rows(const SharedArgs &args)
        : a(args), lane(threadIdx.x & 63), lr(lane & 15), lg(lane >> 4),
          G(args.num_q_heads / args.num_kv_heads)
    {
    }

    // The query rows from row0 of the part on and the lengths of their sequences (lanes beyond its rows take
    // the first one again: nothing is made of them).
    __device__ __forceinline__ void load(const Part &u, int row0, bf16x8_t (&x)[4], int &tokens) const
    {
        const int at = row0 + lr < u.rows ? row0 + lr : 0;
        const int r = u.row0 + at, b = u.b0 + r / G, j = r % G;
        const uint16_t *row = a.q + ((int64_t)b * a.num_q_heads + u.h * G + j) * kHeadDim + 8 * lg;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            x[i] = __builtin_bit_cast(bf16x8_t, ld16(row + 32 * i));
        tokens = a.seq_lens[b];
    }

    __device__ __forceinline__ void begin(const Part &u, int row0, const bf16x8_t (&x)[4], int tokens)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            q[i] = x[i];
        lim = u.lim;
        rows = min(max(u.rows - row0, 0), kRows);
        len = lr < rows ? clamp_len(tokens, a.ps, a.max_pages) : 0x7fffffff;
        full = min((int)wave_min((uint32_t)len), lim);
        ends = (int)wave_min(len > 0 ? (uint32_t)len : 0x7fffffffu);
        ends = ends < lim ? ends : 0x7fffffff - kTileTokens;
        m = kNoLogit;
        l = 0.f;
#pragma unroll
        for (int c = 0; c < 8; ++c)
            O[c] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    }

    // kGroup: the rows are of several sequences.
    template <bool kGroup>
    __device__ __forceinline__ void attend(Tile &t)
    {
        const bool whole = t.live[0] && t.live[1] && t.tok + kTileTokens <= full;
        f32x4_t s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    __builtin_bit_cast(bf16x8_t, t.h[i].k[j]), q[j], s[i], 0, 0, 0);
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            z[e] = s[e >> 2][e & 3] * a.scale_log2;
        if (!whole) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int at = t.tok + 16 * (e >> 2) + 4 * lg + (e & 3);
                const bool there = t.live[e >> 2] && at < lim;
                z[e] = there && at < len ? z[e] : -INFINITY;
                if (!there)  // zero V: cache slots may hold anything
                    t.h[e >> 2].v[e & 3] = (u32x4_t){0u, 0u, 0u, 0u};
            }
            if (kGroup && t.tok + kTileTokens > ends && !finite(t))
                take_out(t);
        }
        float top = fmaxf(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])),
                          fmaxf(fmaxf(z[4], z[5]), fmaxf(z[6], z[7])));
        top = over_groups(top, [](float x, float y) { return fmaxf(x, y); });
        const float m_new = fmaxf(m, top);
        const float alpha = __builtin_amdgcn_exp2f(m - m_new);
        m = m_new;
        float sum = 0.f;
        u32x4_t p[kTerms];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            float x0 = __builtin_amdgcn_exp2f(z[e] - m_new), x1 = __builtin_amdgcn_exp2f(z[e + 1] - m_new);
            sum += x0 + x1;
#pragma unroll
            for (int k = 0; k < kTerms; ++k) {
                const uint32_t b = pack_bf16(x0, x1);
                p[k][e >> 1] = b;
                x0 -= bf16_lo(b);
                x1 -= bf16_hi(b);
            }
        }
        l = l * alpha + sum;
        if (__ballot(alpha != 1.f)) {
#pragma unroll
            for (int c = 0; c < 8; ++c)
                O[c] *= alpha;
        }
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const u32x4_t v = v_of(t, c);
#pragma unroll
            for (int k = 0; k < kTerms; ++k)
                O[c] = product(v, p[k], O[c]);
        }
    }

    // Whether all of the tile's V rows are, for the wave.
    __device__ __forceinline__ static bool finite(const Tile &t)
    {
        typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
        u16x2_t most = {0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                most = __builtin_elementwise_max(
                    most, __builtin_bit_cast(u16x2_t, t.h[e >> 2].v[e & 3][i] & 0x7fff7fffu));
        return __ballot(most[0] >= 0x7f80 || most[1] >= 0x7f80) == 0;
    }

    // Takes what is not finite out of the tile's V rows and adds it to the rows that reach it, with a weight of 1
    // for its own, whatever that is: the sum is no number, or infinite, then.  In the others its weight is 0,
    // whose product with it would be no number either.  (A row at a time, of which its lanes keep theirs.)
    // Looking for it, where a sequence ends inside the prefix, takes 605 us instead of 561 for 16 groups of 16 of
    // which every other sequence does, and nothing where none does (870).
    __device__ __forceinline__ void take_out(Tile &t)
    {
        constexpr uint32_t kOnes = 0x3f803f80u;
#pragma unroll 1
        for (int r = 0; r < kRows; ++r) {
            const int left = __builtin_amdgcn_readlane(len, r) - t.tok - 4 * lg;
            u32x4_t in;  // of two tokens each, as a product has them
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = 16 * (i >> 1) + 2 * (i & 1);
                in[i] = left > at + 1 ? 0xffffffffu : (left > at ? 0x0000ffffu : 0u);
            }
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                u32x4_t v = v_of(t, c);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    v[i] &= odd_halves(v[i]) & in[i];
                const f32x4_t x = product(v, (u32x4_t){kOnes, kOnes, kOnes, kOnes}, O[c]);
                O[c] = lr == r ? x : O[c];
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                t.h[e >> 2].v[e & 3][i] &= ~odd_halves(t.h[e >> 2].v[e & 3][i]);
    }

    // All ones where one of two bf16 numbers is not finite.
    __device__ __forceinline__ static uint32_t odd_halves(uint32_t x)
    {
        return ((x & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((x & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
    }

    // Element c of the tile's V rows, in the order of the numerators.
    __device__ __forceinline__ static u32x4_t v_of(const Tile &t, int c)
    {
        return (u32x4_t){
            pair_of(t.h[0].v[0], t.h[0].v[1], c), pair_of(t.h[0].v[2], t.h[0].v[3], c),
            pair_of(t.h[1].v[0], t.h[1].v[1], c), pair_of(t.h[1].v[2], t.h[1].v[3], c)};
    }

    __device__ __forceinline__ static f32x4_t product(u32x4_t v, u32x4_t p, f32x4_t o)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, v),
                                                       __builtin_bit_cast(bf16x8_t, p), o, 0, 0, 0);
    }

    // (m, l, o) of the rows to slot `slot` of slots of `stride` rows.
    __device__ __forceinline__ void write(float *o, float *ml, uint32_t slot, int stride) const
    {
        const float sum = over_groups(l, [](float x, float y) { return x + y; });
        if (lr >= rows)
            return;
        const int64_t row = (int64_t)slot * stride + lr;
        float *op = o + row * kHeadDim + 32 * lg;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            st16(op + 8 * i, __builtin_bit_cast(u32x4_t, (f32x4_t){O[0][i], O[1][i], O[2][i], O[3][i]}));
            st16(op + 8 * i + 4,
                 __builtin_bit_cast(u32x4_t, (f32x4_t){O[4][i], O[5][i], O[6][i], O[7][i]}));
        }
        if (lg == 0) {
            ml[2 * row] = m;
            ml[2 * row + 1] = sum;
        }
    }
};

// A wave's way through its sequences: the loads of the next tile, the next part's first one too, are always
// under way, and the next part's block-table entries with them.
struct Stream {
    const SharedArgs &a;
    Walk<false> walk;
    Rows work;
    Part load, next;  // the part whose tiles are being loaded, the one behind it
    bool have_next;
    Window win, win_next;
    bf16x8_t q_load[4];  // the loaded part's
    int len_load;
    uint32_t slot;  // of the part at work

    struct Item {
        Tile t;
        bool first, last;  // of its part
    };

    __device__ __forceinline__ Stream(const SharedArgs &args, const Walk<false> &wk)
        : a(args), walk(wk), work(args)
    {
        load.tiles = 0;
        have_next = walk.next(next);
        if (have_next)
            win_next.begin(a, next, work.lane);
    }

    // The loads of the next tile; false: there is none.  They are issued whatever the tile holds (from the
    // cache's first page where there is none), so that the wait for an earlier tile can count the
    // loads behind it.
    __device__ __forceinline__ bool issue(Item &x)
    {
        bool there = true;
        x.first = load.tiles == 0;
        if (x.first && have_next) {
            load = next;
            win = win_next;
            work.load(load, 0, q_load, len_load);
            have_next = walk.next(next);
            if (have_next)
                win_next.begin(a, next, work.lane);
        } else if (x.first) {
            there = false;
            load.lim = 0;
        }
        x.t.tok = load.tok;
        win.reach(a, load, load.tok, work.lane);
        int64_t off[2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
            off[i] = win.place(a, load, load.tok + 16 * i, x.t.live[i]);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            load_half(x.t.h[i], a.k_cache + off[i], a.v_cache + off[i], work.lr, work.lg);
        load.tok += kTileTokens;
        --load.tiles;
        x.last = load.tiles == 0;
        return there;
    }

    // One tile of the part at work, with the next one's loads issued in front; false: it was the last.
    __device__ __forceinline__ bool step(Item &x, Item &behind)
    {
        if (x.first) {  // (the part whose first tile was issued last)
            work.begin(load, 0, q_load, len_load);
            slot = load.slot;
        }
        const bool more = issue(behind);
        __builtin_amdgcn_sched_barrier(0);  // (all of them in front of the wait for this tile)
        work.attend<false>(x.t);
        if (x.last)
            work.write(a.o_seq, a.ml_seq, slot, work.G);
        return more;
    }

    __device__ __forceinline__ void run()
    {
        if (!have_next)
            return;
        Item x, y;
        issue(x);
        while (step(x, y) && step(y, x)) {
        }
    }
};

// A workgroup's way through its groups.  Wave w brings K (even w) or V (odd) of the tiles' half w / 2, 4 rows
// of 256 bytes an instruction, and keeps kStages - 1 tiles under way in registers; in LDS a row's
// 16-byte chunk c lies at place c ^ (row % 16), so that the 16 rows of an operand are in different banks.
constexpr int kStages = 4;  // (even: the LDS has two tiles in turn)
constexpr int kChunks = kHeadDim * 2 / 16;
constexpr int kTileChunks = 2 * kTileTokens * kChunks;  // K and V
static_assert(2 * kTileChunks * 16 >= kMaxGroups * sizeof(int32_t), "the plan's scratch");
static_assert(2 * kTileChunks * 16 + plan_lds(kMaxBatch, kMaxGroups) + 1024 <= 160 << 10,
              "LDS of a workgroup");

struct Team {
    const SharedArgs &a;
    u32x4_t *s_tile;
    const int wave;
    Walk<true> ahead, walk;
    Rows work;
    Part load, next, u;  // being loaded, behind that one, at work
    bool have_next;
    Window win, win_next;

    struct Stage {
        u32x4_t v[4];
        int tok;
        bool live[2];
    };

    __device__ __forceinline__ Team(const SharedArgs &args, const Walk<true> &wk, u32x4_t *lds)
        : a(args), s_tile(lds), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), ahead(wk),
          walk(wk), work(args)
    {
        load.tiles = 0;
        have_next = ahead.next(next);
        if (have_next)
            win_next.begin(a, next, work.lane);
    }

    __device__ __forceinline__ void issue(Stage &x)
    {
        if (load.tiles == 0) {
            if (have_next) {
                load = next;
                win = win_next;
                have_next = ahead.next(next);
                if (have_next)
                    win_next.begin(a, next, work.lane);
            } else {  // nothing left: the cache's first page, for the count of loads
                load.lim = 0;
                load.tiles = 0x7fffffff;
            }
        }
        x.tok = load.tok;
        win.reach(a, load, load.tok, work.lane);
        int64_t off[2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
            off[i] = win.place(a, load, load.tok + 16 * i, x.live[i]);
        const uint16_t *p = (wave & 1 ? a.v_cache : a.k_cache) + (wave >> 1 ? off[1] : off[0]) +
                            work.lg * kHeadDim + 8 * work.lr;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            x.v[j] = ld16_nt(p + 4 * j * kHeadDim);
        load.tok += load.lim ? kTileTokens : 0;
        --load.tiles;
    }

    __device__ __forceinline__ void put(const Stage &x, int turn)
    {
        u32x4_t *s = s_tile + turn * kTileChunks + (wave & 1) * (kTileTokens * kChunks);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int row = 4 * j + work.lg;  // (its number in 16)
            s[(16 * (wave >> 1) + row) * kChunks + (work.lr ^ row)] = x.v[j];
        }
    }

    __device__ __forceinline__ void get(Tile &t, int turn) const
    {
        const u32x4_t *k = s_tile + turn * kTileChunks, *v = k + kTileTokens * kChunks;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                t.h[i].k[j] = k[(16 * i + work.lr) * kChunks + ((4 * j + work.lg) ^ work.lr)];
                const int row = 4 * work.lg + j;
                t.h[i].v[j] = v[(16 * i + row) * kChunks + (work.lr ^ row)];
            }
    }

    __device__ __forceinline__ bool next_part()
    {
        if (!walk.next(u))
            return false;
        bf16x8_t x[4];
        int tokens;
        work.load(u, kRows * wave, x, tokens);
        work.begin(u, kRows * wave, x, tokens);
        return true;
    }

    // Brings a tile on its way and attends with the one that was kStages - 1 steps ago; false: it was the last.
    // The LDS tile that put() writes was read two steps ago, before the last barrier.
    __device__ __forceinline__ bool step(Stage &behind, const Stage &x, int turn)
    {
        issue(behind);
        __builtin_amdgcn_sched_barrier(0);  // (in front of the wait for this tile)
        put(x, turn);
        __syncthreads();
        if (work.rows > 0) {
            Tile t;
            t.tok = x.tok;
            t.live[0] = x.live[0];
            t.live[1] = x.live[1];
            get(t, turn);
            work.attend<true>(t);
        }
        if (--u.tiles == 0) {
            if (work.rows > 0)
                work.write(a.o_group, a.ml_group, u.slot + wave, kRows);
            return next_part();
        }
        return true;
    }

    __device__ __forceinline__ void run()
    {
        Stage s0, s1, s2, s3;
        static_assert(kStages == 4, "stages by name");
        if (!next_part())
            return;
        issue(s0);
        issue(s1);
        issue(s2);
        while (step(s3, s0, 0) && step(s0, s1, 1) && step(s1, s2, 0) && step(s2, s3, 1)) {
        }
    }
};

// The workgroup's place among `n`: each of the 8 XCDs, which take workgroups in turn, works on
// neighbours, so that its cache serves tiles that more than a workgroup's waves read.
__device__ __forceinline__ int place_by_xcd(int block, int n)
{
    constexpr int kXcds = 8;
    return n % kXcds ? block : block % kXcds * (n / kXcds) + block / kXcds;
}

__global__ __launch_bounds__(kSharedThreads, 2) void k_shared_stream(SharedArgs a)
{
    extern __shared__ int32_t s_plan[];
    __shared__ int32_t s_tmp[kSharedWaves];
    __shared__ u32x4_t s_tile[2 * kTileChunks];
    const Plan plan(s_plan, a);
    make_plan(a, plan, reinterpret_cast<int32_t *>(s_tile), s_tmp);

    const uint32_t all = __builtin_amdgcn_readfirstlane(plan.off[a.groups + a.batch]);
    const uint32_t P1 = __builtin_amdgcn_readfirstlane(plan.off[a.groups]), P2 = all - P1;
    const Sides sides(a, P1, P2, gridDim.x);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        a.plan_takers[0] = sides.w1;
        a.plan_takers[1] = sides.w2;
    }
    // Those on the groups are spread evenly over the XCDs and their compute units, and launched first: of two
    // workgroups on a unit the older one goes ahead, and the sequences' have no order to keep among them.
    const uint32_t half = gridDim.x / 2, late = blockIdx.x >= half ? 1 : 0;
    const uint32_t mine = late ? gridDim.x - half : half, w1 = sides.w1;
    const uint32_t n = late ? w1 - min(w1, half) : min(w1, half);  // of this half's workgroups
    const uint32_t place = place_by_xcd(blockIdx.x - (late ? half : 0), mine), before = place * n / mine;
    if ((place + 1) * n / mine > before) {
        const uint32_t w = (late ? half : 0) + before;
        Team team(a, Walk<true>(a, plan, w, Share(P1, w1)), s_tile);
        team.run();
    } else {
        const uint32_t w = ((late ? half - min(w1, half) : 0) + place - before) * kSharedWaves +
                           __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (w < sides.w2) {
            Stream stream(a, Walk<false>(a, plan, w, Share(P2, sides.w2)));
            stream.run();
        }
    }
}

// The parts of one query head of a sequence: those of its group's unit and those of its own.
struct Parts {
    int64_t g0, s0;  // the first ones' rows
    int n_g, n_s, G;

    // (What the plan says of the sequence and of both sides is loaded at once, in front of what the group needs.)
    __device__ __forceinline__ Parts(const SharedArgs &a, int b, int hq)
    {
        const int Hkv = a.num_kv_heads;
        G = a.num_q_heads / Hkv;
        const int h = hq / G, j = hq - h * G;
        const int32_t *seq = a.plan_off + a.groups;
        const int g = a.seq_group[b];
        const uint32_t begin_s = seq[0], end_s = seq[a.batch], off = seq[b], off_next = seq[b + 1];
        const uint32_t takers_g = a.plan_takers[0], takers_s = a.plan_takers[1];
        n_g = n_s = 0;
        g0 = s0 = 0;
        if (g >= 0) {
            const uint32_t first = a.plan_off[g], all = a.plan_off[g + 1] - first;
            const int begin = a.plan_cu[g], rows = (a.plan_cu[g + 1] - begin) * G;
            if (all > 0) {
                const Share share(begin_s, takers_g);
                const uint32_t blocks = (rows + kTeamRows - 1) / kTeamRows, unit = all / (blocks * Hkv);
                const int r = (b - begin) * G + j;
                const uint32_t p0 = first + (h * blocks + r / kTeamRows) * unit;
                const uint32_t w0 = share.taker_of(p0 + kPartCost);
                n_g = share.taker_of(p0 + unit - 1) - w0 + 1;
                // (the 16 rows' slot of taker w is that of the part, kSharedWaves further for each taker)
                g0 = (int64_t)(w0 * kSharedWaves + blocks_before(a, g, begin, rows, h, r)) * kRows + r % kRows;
            }
        }
        const uint32_t own = (off_next - off) / Hkv;
        if (own > 0) {
            const Share share(end_s - begin_s, takers_s);
            const uint32_t p0 = off - begin_s + h * own, w0 = share.taker_of(p0 + kPartCost);
            n_s = share.taker_of(p0 + own - 1) - w0 + 1;
            s0 = (int64_t)(w0 + b * Hkv + h) * G + j;
        }
    }

    __device__ __forceinline__ int count() const { return n_g + n_s; }

    // Part i: its row of o (128 numbers) and its (m, l).
    __device__ __forceinline__ void at(const SharedArgs &a, int i, const float *&o, const float *&ml) const
    {
        const bool shared = i < n_g;
        const int64_t r = shared ? g0 + (int64_t)i * kTeamRows : s0 + (int64_t)(i - n_g) * G;
        o = (shared ? a.o_group : a.o_seq) + r * kHeadDim;
        ml = (shared ? a.ml_group : a.ml_seq) + 2 * r;
    }
};

// kWaves waves per query head and sequence (four, or one where there are many), half a wave per part.
template <int kWaves>
__global__ __launch_bounds__(kSharedThreads) void k_shared_merge(SharedArgs a)
{
    constexpr int kHere = kSharedWaves / kWaves;  // rows of a workgroup
    constexpr int kSides = 2 * kWaves;
    __shared__ float s_o[kHere][kSides][kHeadDim], s_l[kHere][kSides], s_m[kHere][kWaves];
    const int here = threadIdx.x / (64 * kWaves), t = threadIdx.x % (64 * kWaves);
    const int row = min(blockIdx.x * kHere + here, a.batch * a.num_q_heads - 1);  // (the last one again)
    const int b = row / a.num_q_heads;
    const Parts parts(a, b, row - b * a.num_q_heads);
    const int n = parts.count();
    const int side = t >> 5, c = 4 * (t & 31);
    const float *op, *ml;
    // the side's first part, while the parts' maxima are gathered
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    float m0 = kNoLogit, l = 0.f;
    if (side < n) {
        parts.at(a, side, op, ml);
        o = __builtin_bit_cast(f32x4_t, ld16(op + c));
        m0 = ml[0];
        l = ml[1];
    }
    float top = kNoLogit;
    for (int i = t; i < n; i += 64 * kWaves) {
        parts.at(a, i, op, ml);
        top = fmaxf(top, ml[0]);
    }
    top = wave_max_f(top);
    if (kWaves > 1) {
        if ((t & 63) == 0)
            s_m[here][t >> 6] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            top = fmaxf(top, s_m[here][w]);
    }
    const float x0 = __builtin_amdgcn_exp2f(m0 - top);
    l *= x0;
    o *= x0;
    for (int i = side + kSides; i < n; i += kSides) {
        parts.at(a, i, op, ml);
        const float x = __builtin_amdgcn_exp2f(ml[0] - top);
        l += ml[1] * x;
        o += __builtin_bit_cast(f32x4_t, ld16(op + c)) * x;
    }
    *reinterpret_cast<f32x4_t *>(&s_o[here][side][c]) = o;
    if (c == 0)
        s_l[here][side] = l;
    __syncthreads();
    for (int i = t; i < kHeadDim; i += 64 * kWaves) {
        float sum = 0.f, den = 0.f;
#pragma unroll
        for (int k = 0; k < kSides; ++k) {
            sum += s_o[here][k][i];
            den += s_l[here][k];
        }
        // (0: no token; NaN, from a logit that is no number, is a row's result)
        store_out(a.out, a.out_bf16, (int64_t)row * kHeadDim + i, den == 0.f ? 0.f : sum / den);
    }
}

// Workgroups of a launch on `cus` compute units; the workspace is sized for kMaxCus of them.
constexpr int kMaxCus = 256;

int shared_blocks(int cus) { return (cus < kMaxCus ? cus : kMaxCus) * 2; }

// Query heads and sequences from which a wave merges each.  (Four waves and one, whole calls: 128 of them 15.1 and
// 19.3 us, 512 20.0 and 21.4, 1024 23.2 and 23.3, 2048 35.6 and 34.2, 5120 60.0 and 54.2.)
constexpr int kNarrowRows = 1024;

struct SharedPlan {
    size_t plan_bytes, group_slots, seq_slots, bytes;
};

size_t round_up(size_t n) { return (n + 255) / 256 * 256; }

SharedPlan plan_shared(const sparrow_shape_t &s, int groups)
{
    SharedPlan p;
    const int G = s.num_q_heads / s.num_kv_heads;
    const size_t waves = (size_t)shared_blocks(kMaxCus) * kSharedWaves;
    p.plan_bytes = round_up(sizeof(int32_t) * (2 * ((size_t)groups + s.batch) + 4));
    p.group_slots =
        groups ? waves + (size_t)s.num_kv_heads * ((size_t)s.batch * G / kRows + groups) : 0;
    p.seq_slots = waves + (size_t)s.batch * s.num_kv_heads;
    const size_t rows = p.group_slots * kRows + p.seq_slots * G;
    p.bytes = p.plan_bytes + rows * (kHeadDim + 2) * sizeof(float);
    return p;
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
    a.num_phys = (uint32_t)(s.num_phys_pages < 0x7fffffff ? s.num_phys_pages : 0x80000000ll);
    a.page_elems = (uint32_t)(s.num_kv_heads * s.page_size * kHeadDim);
    a.out = out;
    a.out_bf16 = out_dtype == SPARROW_OUT_BF16;
    a.scale_log2 = scale * 1.4426950408889634f;
    // (with 1, 2, 4 and 8: 8 samples of 2001 shared tokens 16.2, 15.1, 14.9 and 18.2 us, of 500 12.1, 12.7, 14.3 and
    // 18.5, one sequence of 4096 20.6, 16.3, 18.6 and 24.4; calls that fill the device do not feel it)
    a.min_tiles = 2;
    char *ws = static_cast<char *>(workspace);
    a.plan_off = reinterpret_cast<int32_t *>(ws);
    a.seq_group = a.plan_off + g.n + s.batch + 1;
    a.plan_cu = a.seq_group + s.batch;
    a.plan_takers = a.plan_cu + g.n + 1;
    const size_t group_rows = p.group_slots * kRows;
    const size_t seq_rows = p.seq_slots * (s.num_q_heads / s.num_kv_heads);
    a.o_group = reinterpret_cast<float *>(ws + p.plan_bytes);
    a.o_seq = a.o_group + group_rows * kHeadDim;
    a.ml_group = a.o_seq + seq_rows * kHeadDim;
    a.ml_seq = a.ml_group + group_rows * 2;
    // positions of all units at most, with the longest sequences everywhere, stay below 2^31
    const int64_t units = (int64_t)s.num_kv_heads *
                          (s.batch + (int64_t)s.batch * (s.num_q_heads / s.num_kv_heads) / kTeamRows + g.n);
    const int64_t tiles = ((int64_t)s.max_pages_per_seq * s.page_size + kTileTokens - 1) / kTileTokens;
    for (a.step_log2 = 0; ((tiles >> a.step_log2) + 1 + kPartCost) * units > 0x7fffffff;)
        ++a.step_log2;
    const size_t lds = plan_lds(s.batch, g.n);
    hipLaunchKernelGGL(k_shared_stream, dim3(shared_blocks(device_cus())), dim3(kSharedThreads), lds, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    const int rows = s.batch * s.num_q_heads;
    if (rows >= kNarrowRows)
        hipLaunchKernelGGL(k_shared_merge<1>, dim3((rows + kSharedWaves - 1) / kSharedWaves),
                           dim3(kSharedThreads), 0, stream, a);
    else
        hipLaunchKernelGGL(k_shared_merge<kSharedWaves>, dim3(rows), dim3(kSharedThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace sparrow
