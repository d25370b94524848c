// New keys and values into a cache of pages in 8 bits, and the cache read back.
//
// A page of a head holds e4m3 codes times one power of two: the smallest 2^e with max |x| <= 448 2^e over the tokens that came in one call, and not below what the page's
// older tokens have.  Codes of four significant bits only lose what falls below e4m3's smallest steps when they are divided by a power of two, so a page whose
// exponent grows is rounded again without hurting what it can still hold.
// A workgroup takes one page of one head, its keys and its values: nothing is shared with another, and one launch does a whole call.  Values lie with 16 tokens side by side and arrive
// row by row, so they are turned over in LDS, four columns of four tokens at a time.  Bound: memory; 2 x 8191 tokens in binary16, 8 heads of 128, stored and read back 44 us a pair of calls, kernels of 19 and 23 us (5.2 and 4.4 TB/s), stored alone 24; one token of each
// of 64 sequences stored and up to 190 read back 17.8 us, kernels of 5 and 14, stored alone 9.
#include "cache.h"

namespace pruner {
namespace cache {
namespace {

struct Rows {
    char* p;
    int64_t batch, token, head;   // elements
};
// i / n for i < 4096 and n <= 128: by a multiplication with the quotient of 2^19, which is off by less than i / 2^19.
struct Over {
    uint32_t by, n;
    __host__ __device__ explicit Over(int n) : by((1u << 19) / (uint32_t)n + 1u), n((uint32_t)n) {}
    __device__ __forceinline__ int quotient(int i) const { return (int)((uint32_t)i * by >> 19); }
};

struct Call {
    Cache c;
    Rows k, v;
    const int32_t *q_len, *k_len;
    int32_t batch, tokens, slots;   // slots: pages of a sequence that a call can touch
    Over units, columns, fours;     // of a head: units of sixteen columns, columns, fours of them
};

typedef u32x4 Loose __attribute__((aligned(2)));
typedef u32x4 LooseF __attribute__((aligned(4)));
__device__ __forceinline__ f32x2 pair_to(uint32_t w, __bf16) { return f32x2{__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)}; }
__device__ __forceinline__ f32x2 pair_to(uint32_t w, _Float16) { return __builtin_convertvector(__builtin_bit_cast(f16x2, w), f32x2); }
__device__ __forceinline__ uint32_t pair_of(float a, float b, __bf16) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2)); }
__device__ __forceinline__ uint32_t pair_of(float a, float b, _Float16) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), f16x2)); }

// Sixteen neighbouring values of a row, anywhere in memory, as they lie there.
template <typename T> struct Sixteen {
    static constexpr int kWords = sizeof(T);
    u32x4 w[kWords];
    __device__ __forceinline__ void load(const T* p)
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            if constexpr (sizeof(T) == 4)
                w[i] = *reinterpret_cast<const LooseF*>(p + 4 * i);
            else
                w[i] = *reinterpret_cast<const Loose*>(p + 8 * i);
        }
    }
    __device__ __forceinline__ float at(int i) const
    {
        if constexpr (sizeof(T) == 4)
            return __uint_as_float(w[i / 4][i % 4]);
        else
            return pair_to(w[i / 8][i / 2 % 4], T{})[i % 2];
    }
};
template <typename T, bool ONCE> __device__ __forceinline__ void store16(T* p, const Sixteen<T>& x)
{
#pragma unroll
    for (int i = 0; i < Sixteen<T>::kWords; ++i) {
        Loose* const to = reinterpret_cast<Loose*>(p + i * 16 / (int)sizeof(T));
        if constexpr (ONCE)
            __builtin_nontemporal_store(x.w[i], to);
        else
            *to = x.w[i];
    }
}
// Codes of sixteen values divided by a power of two: the nearest ones, ties to even; an infinity or a NaN becomes e4m3's NaN.  (What is finite is at most 448.)
template <typename T> __device__ __forceinline__ u32x4 codes_of(const Sixteen<T>& x, float scale)
{
    typedef short i16x2 __attribute__((ext_vector_type(2)));
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        i16x2 two = {0, 0};
        if constexpr (sizeof(T) == 4) {
            two = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(two, __uint_as_float(x.w[i][0]), __uint_as_float(x.w[i][1]), scale, false);
            two = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(two, __uint_as_float(x.w[i][2]), __uint_as_float(x.w[i][3]), scale, true);
        } else if constexpr (__is_same(T, __bf16)) {
            two = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(two, __builtin_bit_cast(bf16x2, +x.w[i / 2][2 * (i % 2)]), scale, false);
            two = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(two, __builtin_bit_cast(bf16x2, +x.w[i / 2][2 * (i % 2) + 1]), scale, true);
        } else {
            two = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(two, __builtin_bit_cast(f16x2, +x.w[i / 2][2 * (i % 2)]), scale, false);
            two = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(two, __builtin_bit_cast(f16x2, +x.w[i / 2][2 * (i % 2) + 1]), scale, true);
        }
        r[i] = __builtin_bit_cast(uint32_t, two);
    }
    return r;
}
// Sixteen codes times a power of two, rounded to the type.
template <typename T> __device__ __forceinline__ Sixteen<T> values_of(u32x4 codes, float scale)
{
    Sixteen<T> x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[i], true);
            x.w[i] = u32x4{__float_as_uint(lo[0] * scale), __float_as_uint(lo[1] * scale), __float_as_uint(hi[0] * scale), __float_as_uint(hi[1] * scale)};
        } else {
            x.w[i / 2][2 * (i % 2)] = pair_from<false>(codes[i], scale, T{});
            x.w[i / 2][2 * (i % 2) + 1] = pair_from<true>(codes[i], scale, T{});
        }
    }
    return x;
}
__device__ __forceinline__ u32x4 rounded_again(u32x4 codes, float scale) { return codes_of<float>(values_of<float>(codes, scale), 1.f); }

// The largest |x|: of values as they lie, two side by side where they have 16 bits (bits of sizes are in the sizes' order).
template <typename T> __device__ __forceinline__ uint32_t larger(uint32_t top, const Sixteen<T>& x)
{
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < Sixteen<T>::kWords; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (sizeof(T) == 4) {
                const uint32_t size = x.w[i][j] & 0x7FFFFFFFu;
                top = top > size ? top : size;
            } else {
                top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top), __builtin_bit_cast(u16x2, x.w[i][j] & 0x7FFF7FFFu)));
            }
        }
    return top;
}
template <typename T> __device__ __forceinline__ uint32_t as_binary32(uint32_t top)   // its bits
{
    if constexpr (sizeof(T) == 4) {
        return top;
    } else {
        const uint32_t one = (top & 0xFFFFu) > top >> 16 ? top & 0xFFFFu : top >> 16;
        return __float_as_uint(pair_to(one, T{})[0]);
    }
}
constexpr uint32_t kInfinity = 0x7F800000u;
template <typename T> __device__ __forceinline__ uint32_t larger_finite(uint32_t top, const Sixteen<T>& x)   // binary32's bits
{
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const uint32_t size = __float_as_uint(x.at(j)) & 0x7FFFFFFFu;
        top = size < kInfinity && size > top ? size : top;
    }
    return top;
}

// Four words of four bytes each, turned over.
__device__ __forceinline__ u32x4 turned_over(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    const uint32_t ab01 = __builtin_amdgcn_perm(b, a, 0x05010400u), ab23 = __builtin_amdgcn_perm(b, a, 0x07030602u), cd01 = __builtin_amdgcn_perm(d, c, 0x05010400u), cd23 = __builtin_amdgcn_perm(d, c, 0x07030602u);
    return u32x4{__builtin_amdgcn_perm(cd01, ab01, 0x05040100u), __builtin_amdgcn_perm(cd01, ab01, 0x07060302u), __builtin_amdgcn_perm(cd23, ab23, 0x05040100u), __builtin_amdgcn_perm(cd23, ab23, 0x07060302u)};
}

__device__ __forceinline__ uint32_t byte_for(uint32_t top)   // of the smallest power of two 2^e, e >= -126, with top <= 448 2^e; top as bits
{
    const int byte = (int)(top >> 23) - 8 + ((top & 0x7FFFFFu) > kLargestFraction ? 1 : 0);
    return (uint32_t)(byte < 1 ? 1 : byte);
}
__device__ __forceinline__ int clamped(const int32_t* p, int b, int most)
{
    if (!p) return most;
    const int n = p[b];
    return n < 0 ? 0 : n > most ? most : n;
}

constexpr int kPad = 4;   // bytes that a row of codes in LDS is longer, so that tokens 16 apart lie in other banks

template <typename T> __global__ void __launch_bounds__(256) append_kernel(Call a)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];   // values' codes [token][head_dim + kPad]
    __shared__ uint32_t tops[2][4];
    const Cache& c = a.c;
    const int h = (int)(blockIdx.x % (uint32_t)c.kv_heads), slot = (int)(blockIdx.x / (uint32_t)c.kv_heads % (uint32_t)a.slots), b = (int)(blockIdx.x / (uint32_t)c.kv_heads / (uint32_t)a.slots);
    // tokens begin .. begin + n - 1 come; those that lie before the first place or behind the last page are left out
    const int n = clamped(a.q_len, b, a.tokens), begin = (a.k_len ? clamped(a.k_len, b, INT32_MAX) : n) - n, pt = c.page_tokens();
    const int64_t stop = (int64_t)begin + n;
    const int page0 = begin > 0 ? begin >> c.shift : 0;
    if ((int64_t)page0 + slot >= c.seq_pages) return;
    const int first = (page0 + slot) << c.shift;   // of the page
    const int lo = begin > first ? begin - first : 0;
    const int hi = (int)(stop - first < pt ? stop - first : pt);
    if (hi <= lo) return;
    const int page = c.page_of(b, first);
    if (page < 0) return;

    const int64_t head = c.head_of(page, h);
    uint8_t* const codes[2] = {c.k + head * c.page_bytes(), c.v + head * c.page_bytes()};
    uint8_t* const exps[2] = {c.k_exps + head, c.v_exps + head};
    const int units = c.head_dim / kUnit, rows = hi - lo, chunks = rows * units, stride = c.head_dim + kPad;
    const T* x[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const Rows& from = s ? a.v : a.k;
        x[s] = reinterpret_cast<const T*>(from.p) + b * from.batch + h * from.head + (int64_t)(first + lo - begin) * from.token;
    }
    auto load = [&](Sixteen<T>& t, int s, int i) {
        const int row = a.units.quotient(i);
        t.load(x[s] + row * (s ? a.v.token : a.k.token) + (i - row * units) * kUnit);
    };
    // the first kHeld chunks of a thread stay in its registers until the exponents are known, others are read again
    constexpr int kHeld = sizeof(T) == 4 ? 1 : 2;
    Sixteen<T> held[2][kHeld];
#pragma unroll
    for (int m = 0; m < kHeld; ++m)
#pragma unroll
        for (int s = 0; s < 2; ++s)
            if ((int)threadIdx.x + 256 * m < chunks) load(held[s][m], s, threadIdx.x + 256 * m);
    const uint32_t was[2] = {*exps[0] < 254u ? *exps[0] : 254u, *exps[1] < 254u ? *exps[1] : 254u};
    auto each = [&](int s, auto&& use) {
#pragma unroll
        for (int m = 0; m < kHeld; ++m)
            if ((int)threadIdx.x + 256 * m < chunks) use(held[s][m], (int)threadIdx.x + 256 * m);
        for (int i = threadIdx.x + 256 * kHeld; i < chunks; i += 256) {
            Sixteen<T> t;
            load(t, s, i);
            use(t, i);
        }
    };
    uint32_t top[2];
    auto meet = [&] {   // a thread's largest are the workgroup's after
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint32_t of_wave = wave_inclusive_max(top[s]);
            if ((threadIdx.x & 63) == 63) tops[s][threadIdx.x >> 6] = of_wave;
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            top[s] = tops[s][0];
#pragma unroll
            for (int w = 1; w < 4; ++w) top[s] = top[s] > tops[s][w] ? top[s] : tops[s][w];
        }
    };
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        uint32_t most = 0u;
        each(s, [&](const Sixteen<T>& t, int) { most = larger(most, t); });
        top[s] = as_binary32<T>(most);
    }
    meet();
    if (top[0] >= kInfinity || top[1] >= kInfinity) {   // something is not finite: once more without it
        __syncthreads();
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            uint32_t most = 0u;
            each(s, [&](const Sixteen<T>& t, int) { most = larger_finite(most, t); });
            top[s] = most;
        }
        meet();
    }
    uint32_t byte[2];
    bool again[2];   // the page's older tokens get a larger power of two
    float scale[2], older[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        byte[s] = byte_for(top[s]);
        again[s] = lo > 0 && byte[s] > was[s];
        if (lo > 0 && byte[s] < was[s]) byte[s] = was[s];
        scale[s] = two_to((int)byte[s]);
        older[s] = two_to(was[s] + 127u > byte[s] ? (int)(was[s] + 127u - byte[s]) : 1);
    }
    if (threadIdx.x == 0) {
        *exps[0] = (uint8_t)byte[0];
        *exps[1] = (uint8_t)byte[1];
    }
    each(1, [&](const Sixteen<T>& t, int i) {
        const int row = a.units.quotient(i);
        const u32x4 w = codes_of(t, scale[1]);
        uint8_t* const to = lds + row * stride + (i - row * units) * kUnit;
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<uint32_t*>(to + 4 * j) = w[j];
    });
    each(0, [&](const Sixteen<T>& t, int i) {
        const int row = a.units.quotient(i);
        *reinterpret_cast<u32x4*>(codes[0] + c.key_at(lo + row, (i - row * units) * kUnit)) = codes_of(t, scale[0]);
    });
    if (again[0])
        for (int i = threadIdx.x; i < lo * units; i += 256) {
            const int row = a.units.quotient(i);
            u32x4* const p = reinterpret_cast<u32x4*>(codes[0] + c.key_at(row, (i - row * units) * kUnit));
            *p = rounded_again(*p, older[0]);
        }
    __syncthreads();
    // sixteen tokens that are all new, four columns at a time
    const int fours = c.head_dim / 4, unit0 = again[1] ? 0 : lo / 16, unit1 = (hi + 15) / 16;
    int full0 = (lo + 15) / 16, full1 = hi / 16;
    if (full1 <= full0) full0 = full1 = unit1;
    for (int i = threadIdx.x; i < (full1 - full0) * fours; i += 256) {
        const int over = a.fours.quotient(i), d = 4 * (i - over * fours), place0 = (full0 + over) * 16;
        const uint8_t* const from = lds + (place0 - lo) * stride + d;
        u32x4 t[4];
#pragma unroll
        for (int q = 0; q < 4; ++q)
            t[q] = turned_over(*reinterpret_cast<const uint32_t*>(from + (4 * q) * stride), *reinterpret_cast<const uint32_t*>(from + (4 * q + 1) * stride),
                               *reinterpret_cast<const uint32_t*>(from + (4 * q + 2) * stride), *reinterpret_cast<const uint32_t*>(from + (4 * q + 3) * stride));
#pragma unroll
        for (int k = 0; k < 4; ++k) *reinterpret_cast<u32x4*>(codes[1] + c.value_at(place0, d + k)) = u32x4{t[0][k], t[1][k], t[2][k], t[3][k]};
    }
    // the others, a column at a time: new tokens, older ones (rounded again, or as they are), and what lies behind, as it is
    for (int i = threadIdx.x; i < (full0 - unit0 + unit1 - full1) * c.head_dim; i += 256) {
        const int over = a.columns.quotient(i), d = i - over * c.head_dim, place0 = (over < full0 - unit0 ? unit0 + over : full1 + over - (full0 - unit0)) * 16;
        u32x4* const p = reinterpret_cast<u32x4*>(codes[1] + c.value_at(place0, d));
        u32x4 w = *p;
        if (again[1] && place0 < lo) {
            const u32x4 r = rounded_again(w, older[1]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int bytes = lo - place0 - 4 * j;
                const uint32_t old = bytes >= 4 ? ~0u : bytes <= 0 ? 0u : (1u << (8 * bytes)) - 1u;
                w[j] = (r[j] & old) | (w[j] & ~old);
            }
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const int place = place0 + j;
            if (place >= lo && place < hi) {
                const uint32_t one = lds[(place - lo) * stride + d];
                w[j / 4] = (w[j / 4] & ~(0xFFu << (8 * (j % 4)))) | one << (8 * (j % 4));
            }
        }
        *p = w;
    }
}

// Rows at or beyond a sequence's length, and those of a page that is not there, are zeros.  ONCE: results are more than the caches are good for.
template <typename T, bool ONCE> __global__ void __launch_bounds__(256) restore_kernel(Call a)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const Cache& c = a.c;
    const int h = (int)(blockIdx.x % (uint32_t)c.kv_heads), slot = (int)(blockIdx.x / (uint32_t)c.kv_heads % (uint32_t)a.slots), b = (int)(blockIdx.x / (uint32_t)c.kv_heads / (uint32_t)a.slots);
    const int first = slot << c.shift, pt = c.page_tokens();
    const int found = c.page_of(b, first), kl = clamped(a.k_len, b, a.tokens), page = first < kl ? found : -1;
    const int rows = a.tokens - first < pt ? a.tokens - first : pt, there = page < 0 ? 0 : kl - first < rows ? kl - first : rows;
    const int64_t head = c.head_of(page < 0 ? 0 : page, h);
    const uint8_t *const k = c.k + head * c.page_bytes(), *const v = c.v + head * c.page_bytes();
    const float k_scale = there > 0 ? two_to(c.k_exps[head]) : 0.f, v_scale = there > 0 ? two_to(c.v_exps[head]) : 0.f;
    const int units = c.head_dim / kUnit, stride = c.head_dim + kPad, fours = c.head_dim / 4;
    for (int i = threadIdx.x; i < (there + 15) / 16 * fours; i += 256) {
        const int over = a.fours.quotient(i), d = 4 * (i - over * fours), place0 = over * 16;
        u32x4 w[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) w[n] = *reinterpret_cast<const u32x4*>(v + c.value_at(place0, d + n));
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const u32x4 t = turned_over(w[0][q], w[1][q], w[2][q], w[3][q]);
#pragma unroll
            for (int j = 0; j < 4; ++j) *reinterpret_cast<uint32_t*>(lds + (place0 + 4 * q + j) * stride + d) = t[j];
        }
    }
    T* const k_out = reinterpret_cast<T*>(a.k.p) + b * a.k.batch + h * a.k.head + (int64_t)first * a.k.token;
    T* const v_out = reinterpret_cast<T*>(a.v.p) + b * a.v.batch + h * a.v.head + (int64_t)first * a.v.token;
    for (int i = threadIdx.x; i < rows * units; i += 256) {
        const int row = a.units.quotient(i), unit = i - row * units;
        u32x4 w = {0u, 0u, 0u, 0u};
        if (row < there) w = *reinterpret_cast<const u32x4*>(k + c.key_at(row, unit * kUnit));
        store16<T, ONCE>(k_out + row * a.k.token + unit * kUnit, values_of<T>(w, k_scale));
    }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * units; i += 256) {
        const int row = a.units.quotient(i), unit = i - row * units;
        u32x4 w = {0u, 0u, 0u, 0u};
        if (row < there)
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = *reinterpret_cast<const uint32_t*>(lds + row * stride + unit * kUnit + 4 * j);
        store16<T, ONCE>(v_out + row * a.v.token + unit * kUnit, values_of<T>(w, v_scale));
    }
}

// Bytes of results from which on they go past the caches: a quarter of the last one.  (us past them and not: an append and a restore of 50 MB that finds the last call's memory 22 and 18, of 67 MB 44 and 47; a restore to
// new memory of 33 MB 13.8 and 15.5, 57 MB 23.7 and 25.7, 67 MB 25.4 and 28.4, 98 MB 37.6 and 39.6, 131 MB 49.3 and 49.4, 197 MB 67.1 and 69.5.)
constexpr int64_t kResults = 64 << 20;
// And only where an access leaves no parts of lines to others, which are not put together there: in 16 bits (in binary32 a thread's sixteen columns are a line, which four accesses write), of heads, or of a page's rows
// where there is one head, that are lines.  (100 MB, us past the caches and not: bfloat16, 8 heads of 128 37 and 41, 112 63 and 50, 96 39 and 46, 80 73 and 53, 48 99 and 61, 32 28 and 56, one head of 80 35 and 40;
// binary32, 8 heads of 128 114 and 44, of 64 98 and 43.)
bool leaves_no_parts(const Rows& y, int64_t heads, int64_t head_dim)   // y: of 16 bits
{
    if (heads == 1 && y.token == head_dim) return aligned(y.p, 16);
    return head_dim % 32 == 0 && aligned(y.p, 64) && y.batch % 32 == 0 && y.token % 32 == 0 && y.head % 32 == 0;
}
size_t size_of(int32_t dtype) { return dtype == PRUNER_F32 ? 4 : 2; }
bool rows_ok(const pruner_heads* h, int32_t dtype) { return h && h->p && aligned(h->p, size_of(dtype)) && h->batch >= 0 && h->token >= 0 && h->head >= 0; }
Rows rows_of(const pruner_heads* h) { return Rows{static_cast<char*>(h->p), h->batch, h->token, h->head}; }

// What both calls refuse; slots: pages of a sequence, a workgroup for each of a head's.
int check(const pruner_cache* c, int32_t dtype, int32_t batch, int32_t tokens, const int32_t* q_len, const int32_t* k_len, const pruner_heads* k, const pruner_heads* v, int64_t slots)
{
    if (!cache_ok(c) || dtype < PRUNER_BF16 || dtype > PRUNER_F32 || batch < 0 || tokens < 0 || tokens >= (1 << 30)) return PRUNER_EINVAL;
    if (!c->table && (int64_t)batch * c->seq_pages > c->pages) return PRUNER_EINVAL;
    if ((q_len && !aligned(q_len, 4)) || (k_len && !aligned(k_len, 4))) return PRUNER_EINVAL;
    if (batch == 0 || tokens == 0) return PRUNER_OK;
    if (!rows_ok(k, dtype) || !rows_ok(v, dtype)) return PRUNER_EINVAL;
    return (double)slots * batch * c->kv_heads < (double)(1 << 24) ? PRUNER_OK : PRUNER_EINVAL;   // (a launch is below 2^24 workgroups of 256 threads)
}

}  // namespace

bool cache_ok(const pruner_cache* c)
{
    if (!c || c->pages < 0 || c->kv_heads < 1 || c->kv_heads > 65535 || c->seq_pages < 0) return false;
    if (c->page_tokens < 16 || c->page_tokens > PRUNER_MAX_PAGE_TOKENS || (c->page_tokens & (c->page_tokens - 1))) return false;
    if (c->head_dim < kUnit || c->head_dim > 128 || c->head_dim % kUnit) return false;
    if ((int64_t)c->seq_pages * c->page_tokens >= (1ll << 30)) return false;
    if (c->table && !aligned(c->table, 4)) return false;
    if (c->pages > 0 && (!c->k_codes || !c->v_codes || !c->k_exps || !c->v_exps || !aligned(c->k_codes, 16) || !aligned(c->v_codes, 16))) return false;
    return true;
}
Cache cache_of(const pruner_cache* c)
{
    int shift = 4;
    while ((1 << shift) < c->page_tokens) ++shift;
    return Cache{c->k_codes, c->v_codes, c->k_exps, c->v_exps, c->table, c->pages, shift, c->kv_heads, c->head_dim, c->seq_pages};
}

}  // namespace cache
}  // namespace pruner

using namespace pruner;

extern "C" int pruner_cache_append(const pruner_cache* c, int32_t dtype, int32_t batch, int32_t tokens, const pruner_heads* k, const pruner_heads* v, const int32_t* q_len, const int32_t* k_len,
                                   void* stream)
{
    const int64_t slots = cache::cache_ok(c) ? ((int64_t)tokens + 2 * c->page_tokens - 2) / c->page_tokens : 0;   // (tokens that begin with a page's last one)
    const int rc = cache::check(c, dtype, batch, tokens, q_len, k_len, k, v, slots);
    if (rc) return rc;
    if (batch == 0 || tokens == 0 || c->pages == 0 || c->seq_pages == 0) return PRUNER_OK;
    const cache::Call call{cache::cache_of(c), cache::rows_of(k), cache::rows_of(v), q_len, k_len, batch, tokens, (int32_t)slots, cache::Over(c->head_dim / cache::kUnit), cache::Over(c->head_dim), cache::Over(c->head_dim / 4)};
    const dim3 grid((unsigned)(slots * batch * c->kv_heads));
    const size_t lds = (size_t)(tokens < c->page_tokens ? tokens : c->page_tokens) * (c->head_dim + cache::kPad);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == PRUNER_BF16)
        hipLaunchKernelGGL((cache::append_kernel<__bf16>), grid, dim3(256), lds, st, call);
    else if (dtype == PRUNER_F16)
        hipLaunchKernelGGL((cache::append_kernel<_Float16>), grid, dim3(256), lds, st, call);
    else
        hipLaunchKernelGGL((cache::append_kernel<float>), grid, dim3(256), lds, st, call);
    PRUNER_LAUNCH_CHECK();
    return PRUNER_OK;
}

extern "C" int pruner_cache_restore(const pruner_cache* c, int32_t dtype, int32_t batch, int32_t tokens, const int32_t* k_len, const pruner_heads* k, const pruner_heads* v, void* stream)
{
    const int64_t slots = cache::cache_ok(c) ? ((int64_t)tokens + c->page_tokens - 1) / c->page_tokens : 0;
    const int rc = cache::check(c, dtype, batch, tokens, nullptr, k_len, k, v, slots);
    if (rc) return rc;
    if (tokens > (int64_t)c->seq_pages * c->page_tokens) return PRUNER_EINVAL;
    if (batch == 0 || tokens == 0) return PRUNER_OK;
    const cache::Call call{cache::cache_of(c), cache::rows_of(k), cache::rows_of(v), nullptr, k_len, batch, tokens, (int32_t)slots, cache::Over(c->head_dim / cache::kUnit), cache::Over(c->head_dim), cache::Over(c->head_dim / 4)};
    const dim3 grid((unsigned)(slots * batch * c->kv_heads));
    const size_t lds = (size_t)c->page_tokens * (c->head_dim + cache::kPad);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool once = dtype != PRUNER_F32 && 2 * (int64_t)batch * tokens * c->kv_heads * c->head_dim * 2 > cache::kResults && cache::leaves_no_parts(call.k, c->kv_heads, c->head_dim) &&
                      cache::leaves_no_parts(call.v, c->kv_heads, c->head_dim);
    void (*const kernel)(cache::Call) = dtype == PRUNER_BF16  ? (once ? cache::restore_kernel<__bf16, true> : cache::restore_kernel<__bf16, false>)
                                        : dtype == PRUNER_F16 ? (once ? cache::restore_kernel<_Float16, true> : cache::restore_kernel<_Float16, false>)
                                                              : cache::restore_kernel<float, false>;
    hipLaunchKernelGGL(kernel, grid, dim3(256), lds, st, call);
    PRUNER_LAUNCH_CHECK();
    return PRUNER_OK;
}
