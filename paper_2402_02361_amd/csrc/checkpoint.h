// Activations in 8 bits: 32 neighbouring values of a row share a power of two (see include/pruner.h).  What the kernels that write
// and read them have in common, and eight neighbouring values of a row in any of the three types.
#pragma once
#include "common.h"

namespace pruner {
namespace ckpt {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr int kGroup = PRUNER_CHECKPOINT_GROUP;
constexpr int kEach = 8;                        // values of a row that a thread holds; four threads hold a group
static_assert(kGroup == 4 * kEach, "a group is four threads' values");

__device__ __forceinline__ uint32_t pair_of(float a, float b, __bf16) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2)); }
__device__ __forceinline__ uint32_t pair_of(float a, float b, _Float16) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), f16x2)); }
__device__ __forceinline__ f32x2 pair_to(uint32_t w, __bf16) { return f32x2{__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)}; }
__device__ __forceinline__ f32x2 pair_to(uint32_t w, _Float16) { return __builtin_convertvector(__builtin_bit_cast(f16x2, w), f32x2); }

// How many of eight values from a place in a row, where `left` of the row's values remain, `after` rows follow and `before` values precede it, lie within the
// matrix; -1 where these are fewer but the eight that end with the last of them do.
__device__ __forceinline__ int room_of(int64_t after, int64_t pitch, int left, int64_t before)
{
    if (after >= 8) return 8;
    const int64_t n = after * pitch + left;
    return n >= 8 ? 8 : before >= 8 - left ? -1 : (int)n;
}

// Eight neighbouring values as they lie in memory (T).  V = 8: rows begin at multiples of 16 bytes and hold whole eights.  V = 1: they begin anywhere; an
// eight moves by accesses that need no alignment.  Of a row's last values the read takes the next row's along, where the matrix has that much room
// (one by one a row's tail is what such rows then cost: the weight gradient 1601 x 903 over 30000 rows took 522 us), or those before them (one by one the gradients of
// three rows of 102 took 13 us, and take 11).  Values at or beyond `left` are 0
// after a read and are not written.
template <typename T, int V> struct Eight {
    static constexpr int kWords = 2 * (int)sizeof(T);
    typedef u32x4 Loose __attribute__((aligned(2)));
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const T* __restrict__ p, int left, int room)
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0u;
        if (V == 8 ? left >= kEach : left > 0 && room >= kEach) {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
                u32x4 q;
                if constexpr (V == 8)
                    q = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint32_t*>(p) + i);
                else
                    q = *reinterpret_cast<const Loose*>(p + i * 4 / (int)sizeof(T));
#pragma unroll
                for (int j = 0; j < 4; ++j) w[i + j] = q[j];
            }
            if constexpr (V == 1) {
#pragma unroll
                for (int i = 0; i < kWords; ++i) {
                    if constexpr (sizeof(T) == 4)
                        w[i] = i < left ? w[i] : 0u;
                    else
                        w[i] = 2 * i + 1 < left ? w[i] : 2 * i < left ? w[i] & 0xFFFFu : 0u;
                }
            }
        } else if constexpr (V == 1) {
            if (left > 0 && room < 0) {   // (the matrix's last values)
                const int by = kEach - left;
#pragma unroll
                for (int i = 0; i < kWords; i += 4) {
                    const u32x4 q = *reinterpret_cast<const Loose*>(p - by + i * 4 / (int)sizeof(T));
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[i + j] = q[j];
                }
                down<4>(by & 4);
                down<2>(by & 2);
                down<1>(by & 1);
            } else if (left > 0) {   // (and there are not eight)
#pragma unroll 1
                for (int j = 0; j < left; ++j) {
                    uint32_t v;
                    if constexpr (sizeof(T) == 4)
                        v = __builtin_bit_cast(uint32_t, p[j]);
                    else
                        v = (uint32_t)__builtin_bit_cast(uint16_t, p[j]) << (16 * (j % 2));
#pragma unroll
                    for (int i = 0; i < kWords; ++i) w[i] |= i == j * (int)sizeof(T) / 4 ? v : 0u;
                }
            }
        }
    }
    template <int VALUES> __device__ __forceinline__ void down(bool move)   // by so many values, zeros behind
    {
        constexpr int kFar = VALUES * (int)sizeof(T) / 4;   // words (0: half a word)
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            uint32_t moved = 0u;
            if constexpr (kFar == 0) {
                moved = w[i] >> 16;
                if (i + 1 < kWords) moved |= w[i + 1 < kWords ? i + 1 : 0] << 16;
            } else {
                if (i + kFar < kWords) moved = w[i + kFar < kWords ? i + kFar : 0];
            }
            w[i] = move ? moved : w[i];
        }
    }
    __device__ __forceinline__ void store(T* __restrict__ p, int left) const
    {
        if (left >= kEach) {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
                const u32x4 q = {w[i], w[i + 1], w[i + 2], w[i + 3]};
                if constexpr (V == 8)
                    *reinterpret_cast<u32x4*>(reinterpret_cast<uint32_t*>(p) + i) = q;
                else
                    *reinterpret_cast<Loose*>(p + i * 4 / (int)sizeof(T)) = q;
            }
        } else if constexpr (V == 1) {
            if (left > 0) {   // a row's tail: four, two and one of its values
                typedef uint32_t Word __attribute__((aligned(2)));
                typedef u32x2 Pair __attribute__((aligned(2)));
                const bool four = left & 4;
                if constexpr (sizeof(T) == 4) {
                    if (four) {
                        *reinterpret_cast<Loose*>(p) = u32x4{w[0], w[1], w[2], w[3]};
                        if (left > 4) p[4] = __builtin_bit_cast(T, w[4]);
                        if (left > 5) p[5] = __builtin_bit_cast(T, w[5]);
                        if (left > 6) p[6] = __builtin_bit_cast(T, w[6]);
                    } else {
                        p[0] = __builtin_bit_cast(T, w[0]);
                        if (left > 1) p[1] = __builtin_bit_cast(T, w[1]);
                        if (left > 2) p[2] = __builtin_bit_cast(T, w[2]);
                    }
                } else {
                    if (four) *reinterpret_cast<Pair*>(p) = u32x2{w[0], w[1]};
                    const uint32_t two = four ? +w[2] : +w[0], one = left & 2 ? (four ? +w[3] : +w[1]) : two;
                    if (left & 2) *reinterpret_cast<Word*>(p + (left & 4)) = two;
                    if (left & 1) p[left & 6] = __builtin_bit_cast(T, (uint16_t)one);
                }
            }
        }
    }
    __device__ __forceinline__ void to_floats(float (&v)[kEach]) const
    {
#pragma unroll
        for (int j = 0; j < kEach; j += 2) {
            if constexpr (sizeof(T) == 4) {
                v[j] = __uint_as_float(w[j]);
                v[j + 1] = __uint_as_float(w[j + 1]);
            } else {
                const f32x2 q = pair_to(w[j / 2], T{});
                v[j] = q[0];
                v[j + 1] = q[1];
            }
        }
    }
    __device__ __forceinline__ void from_floats(const float (&v)[kEach])   // nearest, ties to even
    {
#pragma unroll
        for (int j = 0; j < kEach; j += 2) {
            if constexpr (sizeof(T) == 4) {
                w[j] = __float_as_uint(v[j]);
                w[j + 1] = __float_as_uint(v[j + 1]);
            } else {
                w[j / 2] = pair_of(v[j], v[j + 1], T{});
            }
        }
    }
};

// Eight codes, as above.
template <int V> struct EightCodes {
    typedef u32x2 Loose __attribute__((aligned(1)));
    uint32_t w[2];
    __device__ __forceinline__ void load(const int8_t* __restrict__ p, int left, int room)   // (what is beyond `left` may be anything)
    {
        w[0] = w[1] = 0u;
        if (V == 8 ? left >= kEach : left > 0 && room >= kEach) {
            u32x2 q;
            if constexpr (V == 8)
                q = *reinterpret_cast<const u32x2*>(p);
            else
                q = *reinterpret_cast<const Loose*>(p);
            w[0] = q[0];
            w[1] = q[1];
        } else if constexpr (V == 1) {
            if (left > 0 && room < 0) {
                const Loose q = *reinterpret_cast<const Loose*>(p - (kEach - left));
                const uint64_t all = (((uint64_t)q[1] << 32) | q[0]) >> (8 * (kEach - left));
                w[0] = (uint32_t)all;
                w[1] = (uint32_t)(all >> 32);
            } else if (left > 0)
#pragma unroll
                for (int j = 0; j < kEach; ++j)
                    if (j < left) w[j / 4] |= (uint32_t)(uint8_t)p[j] << (8 * (j % 4));
        }
    }
    __device__ __forceinline__ void store(int8_t* __restrict__ p, int left) const
    {
        if (left >= kEach) {
            if constexpr (V == 8)
                *reinterpret_cast<u32x2*>(p) = u32x2{w[0], w[1]};
            else
                *reinterpret_cast<Loose*>(p) = u32x2{w[0], w[1]};
        } else if constexpr (V == 1) {
            if (left > 0)
#pragma unroll
                for (int j = 0; j < kEach; ++j)
                    if (j < left) p[j] = (int8_t)(uint8_t)(w[j / 4] >> (8 * (j % 4)));
        }
    }
};

// The exponent byte of a group from the largest |x| of it (its bits: a NaN's are above an infinity's, an infinity's above all others).
__device__ __forceinline__ uint32_t exponent_byte(uint32_t top)
{
    const uint32_t field = top >> 23, byte = field - 6u + ((top & 0x7FFFFFu) > 0x7E0000u ? 1u : 0u);   // 127 = 1.984375 x 2^6
    return field == 255u ? 255u : field < 7u ? 1u : byte;
}

// What four neighbouring threads hold becomes one group's codes; every one of the four gets the exponent byte.  Values beyond a row's
// end are 0.  The four threads must be lanes 4 i .. 4 i + 3, all active.
__device__ __forceinline__ uint32_t pack_group(const float (&v)[kEach], uint32_t (&codes)[2])
{
    uint32_t top = 0u;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const uint32_t b = __float_as_uint(v[j]) & 0x7FFFFFFFu;
        top = b > top ? b : top;
    }
    uint32_t other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xf, 0xf, false);   // quad_perm 1,0,3,2
    top = other > top ? other : top;
    other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xf, 0xf, false);            // quad_perm 2,3,0,1
    top = other > top ? other : top;
    const uint32_t byte = exponent_byte(top);
    const float inverse = __uint_as_float(byte == 255u ? 0u : (254u - byte) << 23);   // 2^-e: the product is exact
    codes[0] = codes[1] = 0u;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int c = byte == 255u ? 0 : (int)__builtin_rintf(v[j] * inverse);
        codes[j / 4] |= ((uint32_t)c & 0xFFu) << (8 * (j % 4));
    }
    return byte;
}

__device__ __forceinline__ void restore_eight(const uint32_t (&codes)[2], uint32_t byte, float (&v)[kEach], int left = kEach)   // (0 from `left` on)
{
    const float unit = __uint_as_float(byte == 255u ? 0x7FC00000u : byte << 23);   // NaN x any code, 0 included, is NaN
#pragma unroll
    for (int j = 0; j < kEach; ++j) v[j] = j < left ? (float)(int8_t)(codes[j / 4] >> (8 * (j % 4))) * unit : 0.f;
}

// Whether all of a call's matrices lie so that accesses of eight values are aligned and rows hold whole eights (8), or not (1).
struct Access {
    int v = 8;
    void fits(const void* p, size_t elem_bytes, int64_t pitch)
    {
        const size_t bytes = 8 * elem_bytes < 16 ? 8 * elem_bytes : 16;
        if (p && !(aligned(p, bytes) && pitch % 8 == 0)) v = 1;
    }
};

inline bool type_known(int32_t dtype) { return dtype == PRUNER_BF16 || dtype == PRUNER_F16 || dtype == PRUNER_F32; }
inline size_t type_bytes(int32_t dtype) { return dtype == PRUNER_F32 ? 4 : 2; }

#define BY_TYPE_AND_ACCESS(dtype, v, fn, ...)                                                   \
    ((dtype) == PRUNER_F32    ? ((v) == 8 ? fn<float, 8>(__VA_ARGS__) : fn<float, 1>(__VA_ARGS__))   \
     : (dtype) == PRUNER_BF16 ? ((v) == 8 ? fn<__bf16, 8>(__VA_ARGS__) : fn<__bf16, 1>(__VA_ARGS__)) \
                              : ((v) == 8 ? fn<_Float16, 8>(__VA_ARGS__) : fn<_Float16, 1>(__VA_ARGS__)))

}  // namespace ckpt
}  // namespace pruner
