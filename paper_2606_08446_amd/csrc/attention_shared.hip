// Decode attention of groups of sequences whose first tokens are the same: the samples of one prompt.
// The shared pages are read once per group for all of its query rows, the others per sequence, and the
// parts are joined by their softmax maxima and sums:
//
//   z_t = scale q . K[t],  m = max z,  l = sum e^(z - m),  o = sum e^(z - m) V[t]   of each part,
//   out = sum o e^(m - M) / sum l e^(m - M),  M the largest m.
//
// Work split.  Query rows are taken 16 at a time: a group has (group, KV head, row block) units over its
// shared tokens, a sequence one unit per KV head over its own.  All units' 32-token tiles are laid
// end to end and every wave takes one equal, contiguous range of them.  A group's units are cut into
// segments of as many tiles as a wave takes and laid out segment by segment, row block by row block
// inside: neighbouring waves, which run side by side on one compute unit, then go through the same
// tiles for different rows at the same time, and the tiles come from memory once.  Each part of a
// segment or unit that a wave finds in its range leaves (m, l, o) in the workspace, in slot wave + a
// number that grows along the order; k_shared_merge joins what belongs to a query head.
//
// Per 32-token tile a wave reads K and V straight into MFMA operands:
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
constexpr int kRows = 16;  // query rows of a unit at most
constexpr float kNoLogit = -FLT_MAX;  // a part's maximum before its first token

struct SharedArgs {
    const uint16_t *q, *k_cache, *v_cache;
    const int32_t *block_table, *seq_lens, *cu_groups, *prefix_lens;
    int32_t *plan_off;   // [groups + batch + 1] positions before each entry, groups' first
    int32_t *seq_group;  // [batch] its group, -1: none
    int32_t *plan_waves; // [2] waves of the groups, of the sequences
    int32_t *plan_cu;    // [groups + 1] the groups' first sequences as the plan took them
    float *o_group, *ml_group;  // [slots][kRows] rows
    float *o_seq, *ml_seq;      // [slots][G] rows
    void *out;
    int64_t num_phys;
    int groups, batch, num_q_heads, num_kv_heads, ps, ps_log2, max_pages, out_bf16;
    int max_waves, min_tiles;
    int step_log2;  // a position is 2^step_log2 tiles (more than one only where 2^31 would not do)
    float scale_log2;
};

// Which of the launch's waves take the groups' positions (P1 of them) and which the sequences' (P2): all of
// them in proportion, in whole workgroups, or where that would be less than min_tiles each, fewer.
struct Sides {
    uint32_t w1, w2;
    __device__ __forceinline__ Sides(const SharedArgs &a, uint32_t P1, uint32_t P2, uint32_t waves)
    {
        w1 = (P1 + a.min_tiles - 1) / a.min_tiles;
        w2 = (P2 + a.min_tiles - 1) / a.min_tiles;
        const uint32_t blocks = waves / kSharedWaves;
        if ((w1 + kSharedWaves - 1) / kSharedWaves + (w2 + kSharedWaves - 1) / kSharedWaves > blocks) {
            const float part = (float)P1 / ((float)P1 + (float)P2);
            uint32_t n = (uint32_t)(part * blocks + 0.5f);
            n = P1 ? max(n, 1u) : 0u;
            n = P2 ? min(n, blocks - 1) : blocks;
            w1 = min(w1, n * kSharedWaves);
            w2 = min(w2, (blocks - n) * kSharedWaves);
        }
    }
};

// One side's positions shared out over W waves: the first r take q + 1 of them, the others q.
struct Share {
    uint32_t W, q, r;
    __device__ __forceinline__ Share(uint32_t P, uint32_t waves) : W(waves)
    {
        q = W ? P / W : 1;
        r = P - W * q;
    }
    __device__ __forceinline__ uint32_t begin(uint32_t w) const { return w * q + min(w, r); }
    __device__ __forceinline__ uint32_t wave_of(uint32_t pos) const
    {
        const uint32_t big = r * (q + 1);
        return pos < big ? pos / (q + 1) : r + (pos - big) / q;
    }
    // positions of a segment: what a wave takes at most
    __device__ __forceinline__ uint32_t segment() const { return q + (r ? 1 : 0); }
};

// One segment's row block: where it lies, and a number for its slots that grows along the order (whole
// segments count by their positions, a unit's last one by its row block).
struct Segment {
    uint32_t pos, len, number;
};

// Segment `seg` (of `size` positions) of row block rb, of a group's KV head; begin: the group's first
// sequence, first: its first position, unit: positions of one of its units.
__device__ __forceinline__ Segment segment_at(const SharedArgs &a, int g, int begin, uint32_t first,
                                              uint32_t unit, uint32_t blocks, uint32_t size, int h,
                                              uint32_t seg, uint32_t rb)
{
    const int G = a.num_q_heads / a.num_kv_heads;
    const uint32_t at = seg * size;
    const bool last = unit - at <= size;
    Segment s;
    s.len = last ? unit - at : size;
    s.pos = first + (h * unit + at) * blocks + rb * s.len;
    // (row blocks of the groups before: at most begin * G / kRows + g)
    s.number = s.pos / size + a.num_kv_heads * (begin * G / kRows + g) + h * blocks + (last ? rb : 0);
    return s;
}

// LDS of a workgroup's plan: the positions before each entry (groups, then sequences), each sequence's first
// own page with its own positions, each group's shared tokens, first sequence and shared pages.
struct Plan {
    int32_t *off, *seq, *lim, *cu, *pages;
    __device__ __forceinline__ Plan(int32_t *lds, const SharedArgs &a)
        : off(lds), seq(off + a.groups + a.batch + 1), lim(seq + a.batch), cu(lim + a.groups),
          pages(cu + a.groups + 1)
    {
    }
};

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

__device__ void make_plan(const SharedArgs &a, const Plan &p, int32_t *s_tmp)
{
    const int tid = threadIdx.x;
    const int Hkv = a.num_kv_heads, G = a.num_q_heads / Hkv;
    for (int g = tid; g <= a.groups; g += kSharedThreads) {
        p.cu[g] = a.groups ? min(max(a.cu_groups[g], 0), a.batch) : 0;
        if (g < a.groups) {
            p.pages[g] = min(max(a.prefix_lens[g], 0) >> a.ps_log2, a.max_pages);
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
            first = p.pages[lo];
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
            return Hkv * (p.seq[e - a.groups] & ((1 << kSeqTileBits) - 1));
        return Hkv * positions_of(a, p.lim[e]) * (((p.cu[e + 1] - p.cu[e]) * G + kRows - 1) / kRows);
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

// kOnce: streamed past the caches.
template <bool kOnce>
__device__ __forceinline__ void load_half(Half &c, const uint16_t *kbase, const uint16_t *vbase, int lr,
                                          int lg)
{
    const uint16_t *kp = kbase + lr * kHeadDim + 8 * lg;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        c.k[i] = kOnce ? ld16_nt(kp + 32 * i) : ld16(kp + 32 * i);
    const uint16_t *vp = vbase + 4 * lg * kHeadDim + 8 * lr;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        c.v[j] = kOnce ? ld16_nt(vp + j * kHeadDim) : ld16(vp + j * kHeadDim);
}

struct Tile {
    Half h[2];
    int tok;        // its first token
    bool live[2];   // a half inside the unit's tokens, on a page that is there
    bool first, last;  // of its part
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

// A wave's part of a unit.
struct Part {
    const int32_t *table;  // the block-table row that its pages are read from
    int h, lim;            // KV head; its tokens end here
    int rows, row0;        // query rows of this block, and the first one's number in its entry
    int b0;                // the entry's first sequence
    uint32_t slot;
    int tok, tiles;        // its first token, its tiles that are left to load
};

// The parts of a wave's range, one after another.
struct Walk {
    const SharedArgs &a;
    const Plan &plan;
    const bool shared;
    const int w, Hkv, G;
    const int32_t *off;
    uint32_t size, pos, end;
    int e;

    __device__ __forceinline__ Walk(const SharedArgs &args, const Plan &p, bool shared_, int w_,
                                    const Share &s)
        : a(args), plan(p), shared(shared_), w(w_), Hkv(args.num_kv_heads),
          G(args.num_q_heads / args.num_kv_heads), off(p.off + (shared_ ? 0 : args.groups))
    {
        const uint32_t before = __builtin_amdgcn_readfirstlane(off[0]);
        size = s.segment();
        pos = before + s.begin(w);
        end = before + s.begin(w + 1);
        e = entry_at(off, shared ? a.groups : a.batch, pos);
    }

    __device__ __forceinline__ bool next(Part &u)
    {
        if (pos >= end)
            return false;
        while (off[e + 1] == off[e])
            ++e;
        const uint32_t first = __builtin_amdgcn_readfirstlane(off[e]);
        const int step = kTileTokens << a.step_log2;
        uint32_t at, left;
        if (shared) {
            u.b0 = __builtin_amdgcn_readfirstlane(plan.cu[e]);
            u.lim = __builtin_amdgcn_readfirstlane(plan.lim[e]);
            const int rows = (__builtin_amdgcn_readfirstlane(plan.cu[e + 1]) - u.b0) * G;
            const uint32_t blocks = (rows + kRows - 1) / kRows, unit = positions_of(a, u.lim);
            u.h = (pos - first) / (unit * blocks);
            at = pos - first - u.h * unit * blocks;
            const uint32_t seg = at / (min(size, unit) * blocks);
            at -= seg * size * blocks;
            left = min(size, unit - seg * size);
            const uint32_t rb = at / left;
            at -= rb * left;
            u.slot = w + segment_at(a, e, u.b0, first, unit, blocks, size, u.h, seg, rb).number;
            u.row0 = rb * kRows;
            u.rows = min(kRows, rows - u.row0);
            u.tok = (int)(seg * size + at) * step;
        } else {
            const int packed = __builtin_amdgcn_readfirstlane(plan.seq[e]);
            left = packed & ((1 << kSeqTileBits) - 1);
            u.b0 = e;
            u.lim = clamp_len(a.seq_lens[e], a.ps, a.max_pages);
            u.h = (pos - first) / left;
            at = pos - first - u.h * left;
            u.slot = w + e * Hkv + u.h;
            u.row0 = 0;
            u.rows = G;
            u.tok = (packed >> kSeqTileBits << a.ps_log2) + (int)at * step;
        }
        u.table = a.block_table + (int64_t)u.b0 * a.max_pages;
        const uint32_t take = min(left - at, end - pos);
        // (tiles of the last position may lie behind the unit's tokens)
        u.tiles = min((int)take << a.step_log2, (u.lim - u.tok + kTileTokens - 1) / kTileTokens);
        pos += take;
        if (pos == (uint32_t)__builtin_amdgcn_readfirstlane(off[e + 1]))
            ++e;
        return true;
    }
};

// 64 entries of a block-table row from `page0` on and the 64 behind them, one a lane.
struct Window {
    int page0, phys, phys_next;
};

// A wave's way through its parts: the loads of the next tile, the next part's first one too, are always
// under way, and the next part's block-table entries with them.
template <int kTerms>
struct Streamer {
    const SharedArgs &a;
    const int lane, lr, lg, G;
    Walk &walk;
    Part load, next;  // the part whose tiles are being loaded, the one behind it
    bool have_next;
    Window win, win_next;
    bf16x8_t q_load[4];  // the loaded part's query rows, tokens of their sequences
    int len_load;
    // ---- the part at work
    bf16x8_t q[4];
    int len;   // tokens of the row's sequence
    int full;  // tokens that every row has
    int lim, rows;
    uint32_t slot;
    float m, l;
    f32x4_t O[8];

    __device__ __forceinline__ Streamer(const SharedArgs &args, Walk &wk)
        : a(args), lane(threadIdx.x & 63), lr(lane & 15), lg(lane >> 4),
          G(args.num_q_heads / args.num_kv_heads), walk(wk)
    {
        load.tiles = 0;
        have_next = walk.next(next);  // (a wave has a position at least)
        window(next, win_next);
    }

    __device__ __forceinline__ int entry(const Part &u, int page) const
    {
        return page << a.ps_log2 < u.lim ? u.table[page] : -1;
    }
    __device__ __forceinline__ void window(const Part &u, Window &x) const
    {
        x.page0 = u.tok >> a.ps_log2;
        x.phys = entry(u, x.page0 + lane);
        x.phys_next = entry(u, x.page0 + 64 + lane);
    }

    // The loads of the next tile; false: there is none.  They are issued whatever the tile holds (from the
    // cache's first page where there is none), so that the wait for an earlier tile can count the
    // loads behind it.
    __device__ __forceinline__ bool issue(Tile &t)
    {
        bool there = true;
        t.first = load.tiles == 0;
        if (t.first && have_next) {
            load = next;
            win = win_next;
            // (lanes beyond the block's rows hold its first one again: nothing is made of them)
            const bool in = lr < load.rows;
            const int r = load.row0 + (in ? lr : 0), b = load.b0 + r / G, j = r % G;
            const uint16_t *row = a.q + ((int64_t)b * a.num_q_heads + load.h * G + j) * kHeadDim + 8 * lg;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                q_load[i] = __builtin_bit_cast(bf16x8_t, ld16(row + 32 * i));
            len_load = a.seq_lens[b];
            have_next = walk.next(next);
            if (have_next)
                window(next, win_next);
        } else if (t.first) {
            there = false;
            load.lim = 0;
        }
        const int tok = load.tok;
        t.tok = tok;
        if ((tok >> a.ps_log2) >= win.page0 + 64) {
            win.page0 += 64;
            win.phys = win.phys_next;
            win.phys_next = entry(load, win.page0 + 64 + lane);
        }
        int64_t off[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = tok + 16 * i;
            const int ph = __builtin_amdgcn_readlane(win.phys, ((at >> a.ps_log2) - win.page0) & 63);
            t.live[i] = ph >= 0 && ph < a.num_phys && at < load.lim;
            off[i] = t.live[i] ? (((int64_t)ph * a.num_kv_heads + load.h) * a.ps + (at & (a.ps - 1))) *
                                     kHeadDim
                               : 0;
        }
        if (walk.shared) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                load_half<false>(t.h[i], a.k_cache + off[i], a.v_cache + off[i], lr, lg);
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                load_half<true>(t.h[i], a.k_cache + off[i], a.v_cache + off[i], lr, lg);
        }
        load.tok += kTileTokens;
        --load.tiles;
        t.last = load.tiles == 0;
        return there;
    }

    // The part whose first tile was issued last becomes the one at work.
    __device__ __forceinline__ void begin()
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            q[i] = q_load[i];
        lim = load.lim;
        rows = load.rows;
        slot = load.slot;
        len = lr < rows ? clamp_len(len_load, a.ps, a.max_pages) : 0x7fffffff;
        full = min((int)wave_min((uint32_t)len), lim);
        m = kNoLogit;
        l = 0.f;
#pragma unroll
        for (int c = 0; c < 8; ++c)
            O[c] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    }

    // One tile of the part at work, with the next one's loads issued in front; false: it was the last.
    __device__ __forceinline__ bool step(Tile &t, Tile &behind)
    {
        if (t.first)
            begin();
        const bool more = issue(behind);
        attend(t);
        if (t.last)
            write();
        return more;
    }

    __device__ __forceinline__ void run()
    {
        Tile x, y;
        issue(x);
        while (step(x, y) && step(y, x)) {
        }
    }

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
        }
        float top = fmaxf(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])),
                          fmaxf(fmaxf(z[4], z[5]), fmaxf(z[6], z[7])));
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float m_new = fmaxf(m, top);
        const float alpha = exp2f(m - m_new);
        m = m_new;
        float sum = 0.f;
        u32x4_t p[kTerms];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            float x0 = exp2f(z[e] - m_new), x1 = exp2f(z[e + 1] - m_new);
            if (kTerms > 1)
                sum += x0 + x1;
#pragma unroll
            for (int k = 0; k < kTerms; ++k) {
                const uint32_t b = pack_bf16(x0, x1);
                p[k][e >> 1] = b;
                if (kTerms == 1) {
                    sum += bf16_lo(b) + bf16_hi(b);  // (the weights as they are used)
                } else {
                    x0 -= bf16_lo(b);
                    x1 -= bf16_hi(b);
                }
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
            const u32x4_t av = {
                pair_of(t.h[0].v[0], t.h[0].v[1], c), pair_of(t.h[0].v[2], t.h[0].v[3], c),
                pair_of(t.h[1].v[0], t.h[1].v[1], c), pair_of(t.h[1].v[2], t.h[1].v[3], c)};
#pragma unroll
            for (int k = 0; k < kTerms; ++k)
                O[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, av),
                                                               __builtin_bit_cast(bf16x8_t, p[k]),
                                                               O[c], 0, 0, 0);
        }
    }

    // (m, l, o) of the part's rows to its slot.
    __device__ __forceinline__ void write()
    {
        float sum = l + __shfl_xor(l, 16, 64);
        sum += __shfl_xor(sum, 32, 64);
        if (lr >= rows)
            return;
        const int64_t row = (int64_t)slot * (walk.shared ? kRows : G) + lr;
        float *op = (walk.shared ? a.o_group : a.o_seq) + row * kHeadDim + 32 * lg;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            st16(op + 8 * i, __builtin_bit_cast(u32x4_t, (f32x4_t){O[0][i], O[1][i], O[2][i], O[3][i]}));
            st16(op + 8 * i + 4,
                 __builtin_bit_cast(u32x4_t, (f32x4_t){O[4][i], O[5][i], O[6][i], O[7][i]}));
        }
        if (lg == 0) {
            float *ml = (walk.shared ? a.ml_group : a.ml_seq) + 2 * row;
            ml[0] = m;
            ml[1] = sum;
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

template <int kTerms>
__global__ __launch_bounds__(kSharedThreads, 2) void k_shared_stream(SharedArgs a)
{
    extern __shared__ int32_t s_plan[];
    __shared__ int32_t s_tmp[kSharedWaves];
    const Plan plan(s_plan, a);
    make_plan(a, plan, s_tmp);

    const uint32_t all = __builtin_amdgcn_readfirstlane(plan.off[a.groups + a.batch]);
    const uint32_t P1 = __builtin_amdgcn_readfirstlane(plan.off[a.groups]), P2 = all - P1;
    const Sides sides(a, P1, P2, gridDim.x * kSharedWaves);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        a.plan_waves[0] = sides.w1;
        a.plan_waves[1] = sides.w2;
    }
    // n of the workgroups take the groups, evenly spread among the others over the XCDs and the order of
    // launch: they share their tiles, so that the memory's time belongs to the others
    const uint32_t place = place_by_xcd(blockIdx.x, gridDim.x), n = (sides.w1 + kSharedWaves - 1) / kSharedWaves;
    const uint32_t before = place * n / gridDim.x;
    const bool shared = (place + 1) * n / gridDim.x > before;
    const uint32_t w = (shared ? before : place - before) * kSharedWaves +
                       __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (w >= (shared ? sides.w1 : sides.w2))
        return;
    const Share share(shared ? P1 : P2, shared ? sides.w1 : sides.w2);
    Walk walk(a, plan, shared, w, share);
    Streamer<kTerms> st(a, walk);
    st.run();
}

// The parts of one query head of a sequence: those of its group's segments, at most two waves each (a
// segment is a position longer than the shortest wave at most), and those of its own unit.
struct Parts {
    const SharedArgs &a;
    Share gs;
    uint32_t first, unit, blocks, rb, size, segs, s0;
    int g, h, j, begin, row, n_s;

    __device__ __forceinline__ Parts(const SharedArgs &args, int b, int hq)
        : a(args), gs(args.plan_off[args.groups], args.plan_waves[0])
    {
        const int Hkv = a.num_kv_heads, G = a.num_q_heads / Hkv;
        h = hq / G;
        j = hq - h * G;
        g = a.seq_group[b];
        size = gs.segment();
        segs = 0;
        if (g >= 0) {
            first = a.plan_off[g];
            begin = a.plan_cu[g];
            blocks = ((a.plan_cu[g + 1] - begin) * G + kRows - 1) / kRows;
            unit = (a.plan_off[g + 1] - first) / (blocks * Hkv);
            const int r = (b - begin) * G + j;
            rb = r / kRows;
            row = r - rb * kRows;
            segs = (unit + size - 1) / size;
        }
        n_s = 0;
        const int32_t *seq = a.plan_off + a.groups;
        const uint32_t own = (seq[b + 1] - seq[b]) / Hkv;
        if (own > 0) {
            const Share ss(seq[a.batch] - seq[0], a.plan_waves[1]);
            const uint32_t p0 = seq[b] - seq[0] + h * own, w0 = ss.wave_of(p0);
            n_s = ss.wave_of(p0 + own - 1) - w0 + 1;
            s0 = w0 + b * Hkv + h;
        }
    }

    __device__ __forceinline__ int count() const { return 2 * segs + n_s; }

    // Part i: its row of o (128 numbers) and its (m, l); false: there is none.
    __device__ __forceinline__ bool at(int i, const float *&o, const float *&ml) const
    {
        int64_t r;
        if (i < 2 * (int)segs) {
            const Segment s = segment_at(a, g, begin, first, unit, blocks, size, h, i >> 1, rb);
            const uint32_t w = gs.wave_of(s.pos) + (i & 1);
            if (w > gs.wave_of(s.pos + s.len - 1))
                return false;
            r = (int64_t)(w + s.number) * kRows + row;
            o = a.o_group + r * kHeadDim;
            ml = a.ml_group + 2 * r;
        } else {
            r = (int64_t)(s0 + i - 2 * segs) * (a.num_q_heads / a.num_kv_heads) + j;
            o = a.o_seq + r * kHeadDim;
            ml = a.ml_seq + 2 * r;
        }
        return true;
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
    const float *op, *ml;
    float top = kNoLogit;
    for (int i = t; i < n; i += 64 * kWaves)
        if (parts.at(i, op, ml))
            top = fmaxf(top, ml[0]);
    top = wave_max_f(top);
    if (kWaves > 1) {
        if ((t & 63) == 0)
            s_m[here][t >> 6] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            top = fmaxf(top, s_m[here][w]);
    }
    const int side = t >> 5, c = 4 * (t & 31);
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
    for (int i = side; i < n; i += kSides)
        if (parts.at(i, op, ml)) {
            const float x = exp2f(ml[0] - top);
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
        store_out(a.out, a.out_bf16, (int64_t)row * kHeadDim + i, den > 0.f ? sum / den : 0.f);
    }
}

// Resident waves of a device of `cus` compute units; the workspace is sized for kMaxCus of them.
constexpr int kMaxCus = 256;

int shared_max_waves(int cus) { return (cus < kMaxCus ? cus : kMaxCus) * kSharedWaves * 2; }

constexpr int kNarrowRows = 1024;  // query heads and sequences from which a wave merges each

struct SharedPlan {
    size_t plan_bytes, group_slots, seq_slots, bytes;
};

size_t round_up(size_t n) { return (n + 255) / 256 * 256; }

SharedPlan plan_shared(const sparrow_shape_t &s, int groups)
{
    SharedPlan p;
    const int G = s.num_q_heads / s.num_kv_heads;
    const size_t waves = shared_max_waves(kMaxCus);
    p.plan_bytes = round_up(sizeof(int32_t) * (2 * ((size_t)groups + s.batch) + 4));
    // slots of a wave and a segment: whole segments are no more than waves, and every row block has
    // one that is not
    p.group_slots =
        groups ? 2 * waves + (size_t)s.num_kv_heads * ((size_t)s.batch * G / kRows + groups) : 0;
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
    a.num_phys = s.num_phys_pages;
    a.out = out;
    a.out_bf16 = out_dtype == SPARROW_OUT_BF16;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.max_waves = shared_max_waves(device_cus());
    a.min_tiles = 2;
    char *ws = static_cast<char *>(workspace);
    a.plan_off = reinterpret_cast<int32_t *>(ws);
    a.seq_group = a.plan_off + g.n + s.batch + 1;
    a.plan_cu = a.seq_group + s.batch;
    a.plan_waves = a.plan_cu + g.n + 1;
    const size_t group_rows = p.group_slots * kRows;
    const size_t seq_rows = p.seq_slots * (s.num_q_heads / s.num_kv_heads);
    a.o_group = reinterpret_cast<float *>(ws + p.plan_bytes);
    a.o_seq = a.o_group + group_rows * kHeadDim;
    a.ml_group = a.o_seq + seq_rows * kHeadDim;
    a.ml_seq = a.ml_group + group_rows * 2;
    // positions of all units at most, with the longest sequences everywhere, stay below 2^31
    const int64_t units = (int64_t)s.num_kv_heads *
                          (s.batch + (int64_t)s.batch * (s.num_q_heads / s.num_kv_heads) / kRows + g.n);
    const int64_t tiles = ((int64_t)s.max_pages_per_seq * s.page_size + kTileTokens - 1) / kTileTokens;
    for (a.step_log2 = 0; ((tiles >> a.step_log2) + 1) * units > 0x7fffffff;)
        ++a.step_log2;
    const size_t lds = sizeof(int32_t) * (4 * (size_t)g.n + 2 * (size_t)s.batch + 2);
    auto kernel = a.out_bf16 ? k_shared_stream<1> : k_shared_stream<3>;
    hipLaunchKernelGGL(kernel, dim3(a.max_waves / kSharedWaves), dim3(kSharedThreads), lds, stream, a);
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
