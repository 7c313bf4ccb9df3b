// The e4m3 cache: what a row holds, and the launchers of the kernels around it.
//
// K and V of a (token, KV head) are 128 float8_e4m3fn codes and one biased exponent byte each; a
// channel's value is code * 2^(byte - 127).  The scale is a power of two: it costs a floating
// format no precision, the quotient before the rounding is exact, and every value is a bf16
// number, so the landmarks of the cache are exact as well.
//   codes  [num_phys_pages][num_kv_heads][page_size][128]
//   exps   [num_phys_pages][num_kv_heads][page_size / 4][2][4]: K's four bytes, V's four, so that
//          a lane of the attention finds both scales of its four tokens in one 8-byte load
#pragma once

#include "common.h"

namespace sparrow {

constexpr int kByteMin = 10, kByteMax = 246;  // of the exponents: 2^-117 .. 2^119

// Biased exponent of a row from the bf16 bits of its largest magnitude (sign cleared): the least
// power of two that brings it within 448 = 1.75 * 2^8.  Adding 31 carries into the exponent
// exactly where the 7 mantissa bits exceed 96, that is 1.75.  Between the limits every value, and
// the smallest code of a row, are normal bf16 numbers; what lies above 448 * 2^119 saturates.
__device__ __forceinline__ int row_byte(uint32_t amax)
{
    const int b = (int)((amax + 31u) >> 7) - 8;
    return b < kByteMin ? kByteMin : (b > kByteMax ? kByteMax : b);
}

__device__ __forceinline__ float pow2_of_byte(int byte)
{
    return __uint_as_float((uint32_t)byte << 23);
}

// Four values, already divided by the row's scale, as e4m3 codes (round to nearest even).
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d)
{
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}

// Codes 0 and 1 (kHigh: 2 and 3) of a word times a power of two, as two bf16.
template <bool kHigh>
__device__ __forceinline__ uint32_t unpack_e4m3(uint32_t codes, float scale)
{
    return __builtin_bit_cast(uint32_t,
                              __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, kHigh));
}

struct CacheE4m3 {
    uint8_t *k, *v, *exps;
};

// Rows of new tokens: row r of head h starts at r * stride + h * 128 elements.
struct NewRows {
    const uint16_t *k, *v;
    int64_t k_stride, v_stride;
    const int32_t *cu_tokens;  // [batch + 1] first row of each sequence, or nullptr: one row each
    int64_t num_rows;
};

hipError_t launch_append_e4m3(const sparrow_shape_t &s, const NewRows &rows, const CacheE4m3 &c,
                              const int32_t *block_table, const int32_t *seq_lens, void *meta,
                              hipStream_t stream);
hipError_t launch_read_e4m3(const sparrow_shape_t &s, const CacheE4m3 &c,
                            const int32_t *block_table, const int32_t *seq_lens,
                            const int32_t *cu_tokens, int64_t num_rows, void *k_out, void *v_out,
                            hipStream_t stream);

}  // namespace sparrow
