// Writing new tokens into an e4m3 cache, with the landmarks of their pages, and reading tokens
// back as bf16 rows (the format is in cache_e4m3.h).
//
// 16 lanes own a row: lane l holds channels 8l .. 8l+7 (16 bytes of bf16, 8 of codes), so the
// row's largest magnitude is four DPP steps over one 16-lane DPP row, and a wave takes 4 rows.
// Both directions are bound by HBM: 512 B of bf16 and 258 B of cache per (token, KV head).  64K tokens
// of 8 heads (ragged prompts): append 102 us, 4.8 TB/s, read 76 us, 5.1 TB/s, what a plain copy reaches
// (4.8).
//
// The new tokens of a sequence lie in consecutive rows and end at its length.  A decode step
// (one row each) has a kernel of its own, 16 lanes per (sequence, KV head).  Otherwise the work is laid
// out by page, so that a page's landmark is made by one workgroup with no atomics: sequence b with
// rows c_b .. c_{b+1} overlaps at most (c_{b+1} - c_b) / ps + 2 pages, so the slots
//     s_b = c_b / ps + 2 b  ..  s_{b+1} - 1
// are enough for it, and a workgroup finds the sequence of its slot by searching the row offsets.
#include "cache_e4m3.h"

#include "wave.h"

namespace sparrow {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// DPP control: rotation by n lanes inside each row of 16.
constexpr int ror(int n) { return 0x120 + n; }

template <int kCtrl>
__device__ __forceinline__ uint32_t dpp_u(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kCtrl, 0xf, 0xf, true);
}

// Maximum over each 16 lanes (every lane gets it).
__device__ __forceinline__ uint32_t max16(uint32_t x)
{
    x = max(x, dpp_u<ror(8)>(x));
    x = max(x, dpp_u<ror(4)>(x));
    x = max(x, dpp_u<ror(2)>(x));
    return max(x, dpp_u<ror(1)>(x));
}

// Largest magnitude of 8 bf16 (their bits without the sign order like the values).
__device__ __forceinline__ uint32_t amax8(u32x4_t v)
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        m = max(m, max(v[i] & 0x7fffu, (v[i] >> 16) & 0x7fffu));
    return m;
}

// Codes of 8 bf16 under a row's exponent.
__device__ __forceinline__ u32x2_t quantise8(u32x4_t v, int byte)
{
    const float inv = pow2_of_byte(254 - byte);
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = bf16_lo(v[i]) * inv;
        f[2 * i + 1] = bf16_hi(v[i]) * inv;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)  // (reached only past 448 * 2^119)
        f[i] = fminf(fmaxf(f[i], -448.f), 448.f);
    return (u32x2_t){pack_e4m3(f[0], f[1], f[2], f[3]), pack_e4m3(f[4], f[5], f[6], f[7])};
}

// The bf16 values of 8 codes.
__device__ __forceinline__ u32x4_t values8(u32x2_t c, int byte)
{
    const float scale = pow2_of_byte(byte);
    return (u32x4_t){unpack_e4m3<false>(c[0], scale), unpack_e4m3<true>(c[0], scale),
                     unpack_e4m3<false>(c[1], scale), unpack_e4m3<true>(c[1], scale)};
}

// Exponent byte of a slot in a (page, head)'s group of them.
__device__ __forceinline__ int exp_at(int slot, bool is_v)
{
    return (slot >> 2) * 8 + (is_v ? 4 : 0) + (slot & 3);
}

// One token per sequence.
template <bool kMean>
__global__ __launch_bounds__(kThreads) void k_append_e4m3(
    NewRows rows, CacheE4m3 c, const int32_t *__restrict__ block_table,
    const int32_t *__restrict__ seq_lens, void *__restrict__ meta, int batch, int num_kv_heads,
    int ps, int max_pages, int64_t num_phys)
{
    const int l = threadIdx.x & 15;
    const int64_t unit = (int64_t)blockIdx.x * (kThreads / 16) + (threadIdx.x >> 4);
    if (unit >= (int64_t)batch * num_kv_heads)
        return;
    const int b = (int)(unit / num_kv_heads);
    const int h = (int)(unit - (int64_t)b * num_kv_heads);
    const u32x4_t kn = ld16(rows.k + b * rows.k_stride + h * kHeadDim + 8 * l);
    const u32x4_t vn = ld16(rows.v + b * rows.v_stride + h * kHeadDim + 8 * l);
    const int L = seq_lens[b];
    if (L < 1 || L > ps * max_pages)
        return;  // nothing to append, or a position the block table cannot address
    const int lp = (L - 1) / ps;
    const int slot = L - 1 - lp * ps;
    const int64_t phys = block_table[(int64_t)b * max_pages + lp];
    if (phys < 0 || phys >= num_phys)
        return;  // the page is outside the cache: nothing is written
    const int64_t ph = phys * num_kv_heads + h;
    const int kb = row_byte(max16(amax8(kn))), vb = row_byte(max16(amax8(vn)));
    const u32x2_t kc = quantise8(kn, kb), vc = quantise8(vn, vb);
    const int64_t row = (ph * ps + slot) * kHeadDim + 8 * l;
    *reinterpret_cast<u32x2_t *>(c.k + row) = kc;
    *reinterpret_cast<u32x2_t *>(c.v + row) = vc;
    if (l < 2)
        c.exps[ph * ps * 2 + exp_at(slot, l == 1)] = (uint8_t)(l == 1 ? vb : kb);
    const u32x4_t key = values8(kc, kb);
    if (kMean) {
        float *m = static_cast<float *>(meta) + ph * kHeadDim + 8 * l;
        st16(m, sums_with_key(slot == 0, ld16(m), (u32x2_t){key[0], key[1]}));
        st16(m + 4, sums_with_key(slot == 0, ld16(m + 4), (u32x2_t){key[2], key[3]}));
    } else {
        uint16_t *m = static_cast<uint16_t *>(meta) + ph * 2 * kHeadDim + 8 * l;
        st16(m, meta_with_key(ld16(m), key, false, slot == 0));
        st16(m + kHeadDim, meta_with_key(ld16(m + kHeadDim), key, true, slot == 0));
    }
}

// The tokens of one page slot.
struct PageRows {
    int b;
    int64_t lp;      // logical page (any value: the caller checks it)
    int t0, t1;      // its slots with new tokens
    int64_t row0;    // row of slot 0 (negative where the new tokens begin inside the page)
    int64_t L;
};

// First row of sequence b, kept inside the rows that there are.
__device__ __forceinline__ int64_t first_row(const int32_t *cu, int b, int64_t num_rows)
{
    const int64_t c = cu == nullptr ? b : cu[b];
    return c < 0 ? 0 : (c > num_rows ? num_rows : c);
}

// Page slot `s` of the layout above (every lane of the wave takes part in the search): the last
// sequence whose first slot is <= s.  64 candidates a round; in the last round a lane loads all that is
// wanted of its candidate, so that up to 64 sequences cost one trip to memory.
__device__ __forceinline__ PageRows find_page(const int32_t *cu, const int32_t *seq_lens,
                                              int64_t num_rows, int batch, int ps, int64_t s)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, span = batch;
    while (span > 64) {
        const int step = (span + 63) >> 6;
        const int b = lo + lane * step;
        const bool ok = lane * step < span && first_row(cu, b, num_rows) / ps + 2 * (int64_t)b <= s;
        const int t = max(__popcll(__ballot(ok)) - 1, 0);
        lo += t * step;
        span = min(step, span - t * step);
    }
    int c = 0, next = 0, len = 0;
    bool ok = false;
    if (lane < span) {
        c = (int)first_row(cu, lo + lane, num_rows);
        next = (int)first_row(cu, lo + lane + 1, num_rows);
        len = seq_lens[lo + lane];
        ok = c / ps + 2 * (int64_t)(lo + lane) <= s;
    }
    const int t = max(__popcll(__ballot(ok)) - 1, 0);
    PageRows p;
    p.b = lo + t;
    const int64_t c0 = __builtin_amdgcn_readlane(c, t);
    int64_t n = __builtin_amdgcn_readlane(next, t) - c0;
    n = n < 0 ? 0 : n;
    p.L = __builtin_amdgcn_readlane(len, t);
    const int64_t p0 = p.L - n;  // position of row c0
    const int64_t first = p0 >= 0 ? p0 / ps : -((-p0 + ps - 1) / ps);
    p.lp = first + (s - (c0 / ps + 2 * (int64_t)p.b));
    const int64_t at = p.lp * ps;
    p.t0 = (int)(p0 > at ? p0 - at : 0);
    const int64_t end = p.L - at;  // (<= 0 past the sequence's end)
    p.t1 = end <= 0 ? 0 : (int)(end < ps ? end : ps);
    p.row0 = c0 + (at - p0);
    return p;
}

int64_t page_slots(int64_t num_rows, int batch, int ps) { return num_rows / ps + 2 * (int64_t)batch; }

// Packed pairs of 16-bit integers.
typedef short s16x2_t __attribute__((ext_vector_type(2)));

// order16 of both halves of a word, and its inverse.
__device__ __forceinline__ uint32_t order16x2(uint32_t w)
{
    const s16x2_t s = __builtin_bit_cast(s16x2_t, w);
    return w ^ (__builtin_bit_cast(uint32_t, s >> 15) & 0x7fff7fffu);
}

__device__ __forceinline__ uint32_t min16x2(uint32_t a, uint32_t b)
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(s16x2_t, a),
                                                                  __builtin_bit_cast(s16x2_t, b)));
}

__device__ __forceinline__ uint32_t max16x2(uint32_t a, uint32_t b)
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(s16x2_t, a),
                                                                  __builtin_bit_cast(s16x2_t, b)));
}

// Many tokens per sequence: kPer waves per (page slot, KV head), each with every kPer-th group of
// 4 slots.  The mean landmark's sums are added in token order, from LDS.
template <int kPs, bool kMean>
__global__ __launch_bounds__(kThreads) void k_append_pages_e4m3(
    NewRows rows, CacheE4m3 c, const int32_t *__restrict__ block_table,
    const int32_t *__restrict__ seq_lens, void *__restrict__ meta, int batch, int num_kv_heads,
    int max_pages, int64_t num_phys)
{
    constexpr int kPer = kPs / 16 < kWaves ? kPs / 16 : kWaves;  // waves per (page, head)
    constexpr int kHeads = kWaves / kPer;                        // heads per workgroup
    constexpr int kGroups = kPs / 4 / kPer;                      // groups of 4 slots per wave
    __shared__ u32x4_t s_key[kMean ? kHeads * kPs * 16 : kWaves * 32];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int l = lane & 15, r = lane >> 4;
    const int part = wave % kPer;
    const int h = blockIdx.y * kHeads + wave / kPer;
    const PageRows p = find_page(rows.cu_tokens, seq_lens, rows.num_rows, batch, kPs, blockIdx.x);
    // (the same for the whole workgroup)
    if (p.t1 <= p.t0 || p.lp < 0 || p.lp >= max_pages || p.L > (int64_t)max_pages * kPs)
        return;
    const int64_t phys = block_table[(int64_t)p.b * max_pages + p.lp];
    if (phys < 0 || phys >= num_phys)
        return;  // the page is outside the cache: nothing is written
    const bool head = h < num_kv_heads;
    const int64_t ph = phys * num_kv_heads + h;

    u32x4_t mn, mx;  // landmarks of this lane's channels over its rows, as ordered integers
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        mn[i] = 0x7fff7fffu;
        mx[i] = 0x80008000u;
    }
    constexpr int kAhead = kGroups < 4 ? kGroups : 4;
    for (int g0 = 0; g0 < kGroups; g0 += kAhead) {
        u32x4_t kn[kAhead], vn[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int slot = 4 * ((g0 + i) * kPer + part) + r;
            kn[i] = vn[i] = (u32x4_t){0u, 0u, 0u, 0u};
            if (head && slot >= p.t0 && slot < p.t1) {
                const int64_t row = p.row0 + slot;
                kn[i] = ld16_nt(rows.k + row * rows.k_stride + h * kHeadDim + 8 * l);
                vn[i] = ld16_nt(rows.v + row * rows.v_stride + h * kHeadDim + 8 * l);
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int slot = 4 * ((g0 + i) * kPer + part) + r;
            const int kb = row_byte(max16(amax8(kn[i]))), vb = row_byte(max16(amax8(vn[i])));
            const u32x2_t kc = quantise8(kn[i], kb), vc = quantise8(vn[i], vb);
            const u32x4_t key = values8(kc, kb);
            if (head && slot >= p.t0 && slot < p.t1) {
                const int64_t at = (ph * kPs + slot) * kHeadDim + 8 * l;
                *reinterpret_cast<u32x2_t *>(c.k + at) = kc;
                *reinterpret_cast<u32x2_t *>(c.v + at) = vc;
                if (l < 2)
                    c.exps[ph * kPs * 2 + exp_at(slot, l == 1)] = (uint8_t)(l == 1 ? vb : kb);
                if (kMean) {
                    s_key[((wave / kPer) * kPs + slot) * 16 + l] = key;
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t o = order16x2(key[j]);
                        mn[j] = min16x2(mn[j], o);
                        mx[j] = max16x2(mx[j], o);
                    }
                }
            }
        }
    }

    const bool fresh = p.t0 == 0;  // the page begins with these tokens
    if (kMean) {
        __syncthreads();
        if (part != 0 || !head)
            return;
        float *m = static_cast<float *>(meta) + ph * kHeadDim + 2 * lane;
        float a = 0.f, b = 0.f;
        if (!fresh) {
            a = m[0];
            b = m[1];
        }
        const uint32_t *k = reinterpret_cast<const uint32_t *>(s_key + (wave / kPer) * kPs * 16);
        for (int t = p.t0; t < p.t1; ++t) {
            const uint32_t w = k[t * 64 + lane];
            a += bf16_lo(w);
            b += bf16_hi(w);
        }
        m[0] = a;
        m[1] = b;
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int d = 16; d < 64; d <<= 1) {
            mn[j] = min16x2(mn[j], (uint32_t)__shfl_xor((int)mn[j], d, 64));
            mx[j] = max16x2(mx[j], (uint32_t)__shfl_xor((int)mx[j], d, 64));
        }
    u32x4_t v = r == 0 ? mn : mx;  // lanes 0-15 finish the minimum, 16-31 the maximum
    if (kPer > 1) {
        if (r < 2)
            s_key[wave * 32 + lane] = v;
        __syncthreads();
        if (part != 0)
            return;
        if (r < 2)
            for (int w = 1; w < kPer; ++w) {
                const u32x4_t o = s_key[(wave + w) * 32 + lane];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    v[j] = r == 0 ? min16x2(v[j], o[j]) : max16x2(v[j], o[j]);
            }
    }
    if (!head || r >= 2)
        return;
    uint16_t *m = static_cast<uint16_t *>(meta) + (ph * 2 + r) * kHeadDim + 8 * l;
    if (!fresh) {
        const u32x4_t old = ld16(m);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            v[j] = r == 0 ? min16x2(v[j], order16x2(old[j])) : max16x2(v[j], order16x2(old[j]));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        v[j] = order16x2(v[j]);
    st16(m, v);
}

// A wave per (page slot, KV head) and 16 slots.
template <bool kStream>
__global__ __launch_bounds__(kThreads) void k_read_e4m3(
    CacheE4m3 c, const int32_t *__restrict__ block_table, const int32_t *__restrict__ seq_lens,
    const int32_t *__restrict__ cu_tokens, int64_t num_rows, uint16_t *__restrict__ k_out,
    uint16_t *__restrict__ v_out, int batch, int num_kv_heads, int ps, int max_pages,
    int64_t num_phys)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int l = lane & 15, r = lane >> 4;
    const PageRows p = find_page(cu_tokens, seq_lens, num_rows, batch, ps, blockIdx.x);
    if (p.t1 <= p.t0)
        return;
    int64_t phys = -1;
    if (p.lp >= 0 && p.lp < max_pages)
        phys = block_table[(int64_t)p.b * max_pages + p.lp];
    const bool live = phys >= 0 && phys < num_phys;
    const int parts = ps / 16;
    for (int w = blockIdx.y * kWaves + wave; w < num_kv_heads * parts; w += gridDim.y * kWaves) {
        const int h = w / parts;
        const int s0 = (w - h * parts) * 16;
        const int64_t ph = phys * num_kv_heads + h;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int slot = s0 + 4 * i + r;
            if (slot < p.t0 || slot >= p.t1)
                continue;
            u32x4_t k = {0u, 0u, 0u, 0u}, v = k;
            if (live) {
                const int64_t at = (ph * ps + slot) * kHeadDim + 8 * l;
                const uint8_t *e = c.exps + ph * ps * 2;
                k = values8(*reinterpret_cast<const u32x2_t *>(c.k + at), e[exp_at(slot, false)]);
                v = values8(*reinterpret_cast<const u32x2_t *>(c.v + at), e[exp_at(slot, true)]);
            }
            const int64_t to = ((p.row0 + slot) * num_kv_heads + h) * kHeadDim + 8 * l;
            if (kStream) {
                __builtin_nontemporal_store(k, reinterpret_cast<u32x4_t *>(k_out + to));
                __builtin_nontemporal_store(v, reinterpret_cast<u32x4_t *>(v_out + to));
            } else {
                st16(k_out + to, k);
                st16(v_out + to, v);
            }
        }
    }
}

template <int kPs>
void append_pages(const sparrow_shape_t &s, const NewRows &rows, const CacheE4m3 &c,
                  const int32_t *block_table, const int32_t *seq_lens, void *meta,
                  hipStream_t stream)
{
    constexpr int kHeads = kWaves / (kPs / 16 < kWaves ? kPs / 16 : kWaves);
    const dim3 grid((unsigned)page_slots(rows.num_rows, s.batch, kPs),
                    (s.num_kv_heads + kHeads - 1) / kHeads);
    auto kernel = s.landmark == SPARROW_LANDMARK_MEAN ? k_append_pages_e4m3<kPs, true>
                                                      : k_append_pages_e4m3<kPs, false>;
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, rows, c, block_table, seq_lens,
                       meta, s.batch, s.num_kv_heads, s.max_pages_per_seq, s.num_phys_pages);
}

}  // namespace

hipError_t launch_append_e4m3(const sparrow_shape_t &s, const NewRows &rows, const CacheE4m3 &c,
                              const int32_t *block_table, const int32_t *seq_lens, void *meta,
                              hipStream_t stream)
{
    if (rows.cu_tokens == nullptr) {
        const int64_t units = (int64_t)s.batch * s.num_kv_heads;
        auto kernel = s.landmark == SPARROW_LANDMARK_MEAN ? k_append_e4m3<true>
                                                          : k_append_e4m3<false>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)((units + 15) / 16)), dim3(kThreads), 0, stream,
                           rows, c, block_table, seq_lens, meta, s.batch, s.num_kv_heads,
                           s.page_size, s.max_pages_per_seq, s.num_phys_pages);
        return hipGetLastError();
    }
    switch (s.page_size) {
    case 16: append_pages<16>(s, rows, c, block_table, seq_lens, meta, stream); break;
    case 32: append_pages<32>(s, rows, c, block_table, seq_lens, meta, stream); break;
    case 64: append_pages<64>(s, rows, c, block_table, seq_lens, meta, stream); break;
    default: append_pages<128>(s, rows, c, block_table, seq_lens, meta, stream); break;
    }
    return hipGetLastError();
}

hipError_t launch_read_e4m3(const sparrow_shape_t &s, const CacheE4m3 &c,
                            const int32_t *block_table, const int32_t *seq_lens,
                            const int32_t *cu_tokens, int64_t num_rows, void *k_out, void *v_out,
                            hipStream_t stream)
{
    const int waves = s.num_kv_heads * (s.page_size / 16);
    const int per_slot = (waves + kWaves - 1) / kWaves;  // (the kernel strides over the rest)
    const dim3 grid((unsigned)page_slots(num_rows, s.batch, s.page_size),
                    per_slot < 65535 ? per_slot : 65535);
    // Rows that would not stay in the 256 MB memory-side cache are written past it (268 MB of rows
    // 80 -> 76 us where each call reads another cache, 83 -> 60 where it reads the same one again, and
    // no difference to a copy of the rows behind it; 134 MB 32 either way, but a copy behind it
    // 79 -> 91).
    const bool stream_rows = num_rows * s.num_kv_heads * (int64_t)(4 * kHeadDim) >= 224 << 20;
    auto kernel = stream_rows ? k_read_e4m3<true> : k_read_e4m3<false>;
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, c, block_table, seq_lens,
                       cu_tokens, num_rows, static_cast<uint16_t *>(k_out),
                       static_cast<uint16_t *>(v_out), s.batch, s.num_kv_heads, s.page_size,
                       s.max_pages_per_seq, s.num_phys_pages);
    return hipGetLastError();
}

}  // namespace sparrow
