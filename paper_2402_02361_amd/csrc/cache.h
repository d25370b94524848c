// Keys and values in 8 bits, in pages (see include/pruner.h): where they lie, and how codes become operands.
//
// A key's columns and a value's tokens are the depth of the products that read them, and of an operand a lane holds neighbouring depths of one row.  So keys
// lie in units of 16 columns of all tokens of a page, values in units of 16 tokens of all columns: 32 lanes' 16 bytes are 512 in a row, straight into registers.
#pragma once
#include "common.h"

namespace pruner {
namespace cache {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr int64_t kCached = 256 << 20;   // bytes: the last cache
constexpr int kUnit = 16;            // columns of a key, tokens of values, that lie side by side
constexpr uint32_t kNotANumber = 0x7Fu;   // e4m3's
constexpr uint32_t kLargestFraction = 0x600000u;   // of 448 = 1.75 x 2^8

struct Cache {
    uint8_t *k, *v, *k_exps, *v_exps;
    const int32_t* table;
    int32_t pages, shift, kv_heads, head_dim, seq_pages;   // shift: a page has 1 << shift tokens
    __host__ __device__ __forceinline__ int page_tokens() const { return 1 << shift; }
    __host__ __device__ __forceinline__ int page_bytes() const { return head_dim << shift; }   // of a head
    // The number that stands for token at (0 .. seq_pages * page_tokens - 1) of sequence b, as it is in the table, and whether it is a page: apart, so that who asks ahead does not wait for it there.
    __device__ __forceinline__ int number_of(int b, int at) const
    {
        const int64_t i = (int64_t)b * seq_pages + (at >> shift);
        typedef const __attribute__((address_space(4))) int32_t* read_only;   // (read by the scalar unit where all lanes ask for the same)
        return table ? *((read_only)(uintptr_t)table + i) : (int)i;
    }
    __device__ __forceinline__ bool is_page(int number) const { return (uint32_t)number < (uint32_t)pages; }
    // The page that holds it, or -1: there is none.
    __device__ __forceinline__ int page_of(int b, int at) const
    {
        const int p = number_of(b, at);
        return is_page(p) ? p : -1;
    }
    __device__ __forceinline__ int64_t head_of(int page, int h) const { return (int64_t)page * kv_heads + h; }
    // From the begin of a page's head: column d of the key at a place, column d of the value at a place.
    __device__ __forceinline__ int key_at(int place, int d) const { return ((((d >> 4) << shift) + place) << 4) + (d & 15); }
    __device__ __forceinline__ int value_at(int place, int d) const { return (((place >> 4) * head_dim + d) << 4) + (place & 15); }
};

__device__ __forceinline__ float two_to(int byte) { return __uint_as_float((uint32_t)byte << 23); }   // 2^(byte - 127), byte 1..254
// Of a page's values of which `there` are a sequence's tokens.  Of none: the page may be reserved and not yet written, or not there, and the byte anything; 255 is NaN to the scaled conversions whatever the
// code is, and a weight of 0 does not take that away.
__device__ __forceinline__ float two_to(int byte, int there) { return two_to(there > 0 ? byte : 127); }

// Two codes (the low or the high half of a word) times a power of two, in the operands' type: exact but for binary16's range.
template <bool HIGH> __device__ __forceinline__ uint32_t pair_from(uint32_t codes, float scale, __bf16)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HIGH));
}
template <bool HIGH> __device__ __forceinline__ uint32_t pair_from(uint32_t codes, float scale, _Float16)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, HIGH));
}
template <typename T> __device__ __forceinline__ u32x4 eight_from(uint32_t lo, uint32_t hi, float scale)
{
    return u32x4{pair_from<false>(lo, scale, T{}), pair_from<true>(lo, scale, T{}), pair_from<false>(hi, scale, T{}), pair_from<true>(hi, scale, T{})};
}

bool cache_ok(const pruner_cache* c);   // sizes and pointers
Cache cache_of(const pruner_cache* c);

}  // namespace cache
}  // namespace pruner
