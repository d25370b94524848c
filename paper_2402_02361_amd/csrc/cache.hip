// New keys and values into a cache of pages in 8 bits, and the cache read back.
//
// A page of a head holds e4m3 codes times one power of two: the smallest 2^e with max |x| <= 448 2^e over the tokens that came in one call, and not below what the page's
// older tokens have.  Codes of four significant bits only lose what falls below e4m3's smallest steps when they are divided by a power of two, so a page whose
// exponent grows is rounded again without hurting what it can still hold.
// A workgroup takes one page of one head, keys or values: nothing is shared with another, and one launch does a whole call.  Values lie with 16 tokens side by side and arrive
// row by row, so they are turned over in LDS.
#include "cache.h"

namespace pruner {
namespace cache {
namespace {

struct Rows {
    char* p;
    int64_t batch, token, head;   // elements
};
// i / n for i < 4096 and n = 16 k <= 128, or i < 4096 and n <= 8: by a multiplication with the quotient of 2^19, which is off by less than i / 2^19.
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
    Over units, columns;            // of a head
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
template <typename T> __device__ __forceinline__ void store16(T* p, const float (&x)[16])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<LooseF*>(p + 4 * i) = u32x4{__float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]), __float_as_uint(x[4 * i + 2]), __float_as_uint(x[4 * i + 3])};
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            *reinterpret_cast<Loose*>(p + 8 * i) = u32x4{pair_of(x[8 * i], x[8 * i + 1], T{}), pair_of(x[8 * i + 2], x[8 * i + 3], T{}), pair_of(x[8 * i + 4], x[8 * i + 5], T{}),
                                                         pair_of(x[8 * i + 6], x[8 * i + 7], T{})};
    }
}
// To the nearest codes, ties to even; an infinity or a NaN becomes e4m3's NaN.  (|x| is at most 448.)
__device__ __forceinline__ u32x4 codes_of(const float (&x)[16])
{
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i], x[4 * i + 1], 0, false);
        w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2], x[4 * i + 3], lo, true);
    }
    return w;
}
__device__ __forceinline__ void values_of(float (&x)[16], u32x4 w, float scale)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
        x[4 * i] = lo[0] * scale;
        x[4 * i + 1] = lo[1] * scale;
        x[4 * i + 2] = hi[0] * scale;
        x[4 * i + 3] = hi[1] * scale;
    }
}
__device__ __forceinline__ uint32_t finite_bits(float x)   // of |x|; of what is not finite 0
{
    const uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
    return b < 0x7F800000u ? b : 0u;
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
    extern __shared__ __attribute__((aligned(16))) uint8_t turned[];   // [place][head_dim + kPad]
    __shared__ uint32_t tops[4];
    const Cache& c = a.c;
    const bool values = blockIdx.x & 1;
    const uint32_t id = blockIdx.x >> 1;
    const int h = (int)(id % (uint32_t)c.kv_heads), slot = (int)(id / (uint32_t)c.kv_heads % (uint32_t)a.slots), b = (int)(id / (uint32_t)c.kv_heads / (uint32_t)a.slots);
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
    uint8_t* const codes = (values ? c.v : c.k) + head * c.page_bytes();
    uint8_t* const exps = (values ? c.v_exps : c.k_exps) + head;
    const Rows& from = values ? a.v : a.k;
    const int units = c.head_dim / kUnit, rows = hi - lo, chunks = rows * units;
    const T* const x = reinterpret_cast<const T*>(from.p) + b * from.batch + h * from.head + (int64_t)(first + lo - begin) * from.token;

    // the first kHeld chunks of a thread stay in its registers until the exponent is known, others are read again
    constexpr int kHeld = 4;
    Sixteen<T> held[kHeld];
    auto place_of = [&](int i, int& row, int& unit) {
        row = a.units.quotient(i);
        unit = i - row * units;
        return x + (int64_t)row * from.token + unit * kUnit;
    };
    uint32_t top = 0u;
    auto count = [&](const Sixteen<T>& t) {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const uint32_t bits = finite_bits(t.at(j));
            top = top > bits ? top : bits;
        }
    };
#pragma unroll
    for (int n = 0; n < kHeld; ++n) {
        const int i = threadIdx.x + 256 * n;
        int row, unit;
        if (i < chunks) held[n].load(place_of(i, row, unit));
    }
#pragma unroll
    for (int n = 0; n < kHeld; ++n)
        if ((int)threadIdx.x + 256 * n < chunks) count(held[n]);
    for (int i = threadIdx.x + 256 * kHeld; i < chunks; i += 256) {
        Sixteen<T> t;
        int row, unit;
        t.load(place_of(i, row, unit));
        count(t);
    }
    const uint32_t was = *exps < 254u ? *exps : 254u;
    top = wave_inclusive_max(top);
    if ((threadIdx.x & 63) == 63) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    top = tops[0];
#pragma unroll
    for (int w = 1; w < 4; ++w) top = top > tops[w] ? top : tops[w];
    uint32_t byte = byte_for(top);
    const bool again = lo > 0 && byte > was;   // the page's older tokens get a larger power of two
    if (lo > 0 && byte < was) byte = was;
    if (threadIdx.x == 0) *exps = (uint8_t)byte;
    const float down = __uint_as_float((254u - byte) << 23), older = two_to(was + 127u > byte ? (int)(was + 127u - byte) : 1);

    const int stride = c.head_dim + kPad;
    auto put = [&](const Sixteen<T>& from16, int row, int unit) {
        float t[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) t[j] = from16.at(j) * down;
        const u32x4 w = codes_of(t);
        if (values) {
#pragma unroll
            for (int j = 0; j < 4; ++j) *reinterpret_cast<uint32_t*>(turned + row * stride + unit * kUnit + 4 * j) = w[j];
        } else {
            *reinterpret_cast<u32x4*>(codes + c.key_at(lo + row, unit * kUnit)) = w;
        }
    };
#pragma unroll
    for (int n = 0; n < kHeld; ++n) {
        const int i = threadIdx.x + 256 * n;
        int row, unit;
        place_of(i, row, unit);
        if (i < chunks) put(held[n], row, unit);
    }
    for (int i = threadIdx.x + 256 * kHeld; i < chunks; i += 256) {
        Sixteen<T> t;
        int row, unit;
        t.load(place_of(i, row, unit));
        put(t, row, unit);
    }
    if (!values) {
        if (again)
            for (int i = threadIdx.x; i < lo * units; i += 256) {
                const int row = a.units.quotient(i);
                u32x4* const p = reinterpret_cast<u32x4*>(codes + c.key_at(row, (i - row * units) * kUnit));
                float t[16];
                values_of(t, *p, older);
                *p = codes_of(t);
            }
        return;
    }
    __syncthreads();
    // sixteen tokens of a column: new ones, older ones (rounded again, or as they are), and what lies behind, as it is
    const int unit0 = again ? 0 : lo / 16, unit1 = (hi + 15) / 16;
    for (int i = threadIdx.x; i < (unit1 - unit0) * c.head_dim; i += 256) {
        const int over = a.columns.quotient(i), d = i - over * c.head_dim, place0 = (unit0 + over) * 16;
        u32x4* const p = reinterpret_cast<u32x4*>(codes + c.value_at(place0, d));
        u32x4 w = {0u, 0u, 0u, 0u};
        if (place0 < lo || place0 + 16 > hi) {
            w = *p;
            if (again && place0 < lo) {
                float t[16];
                values_of(t, w, older);
                const u32x4 r = codes_of(t);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int bytes = lo - place0 - 4 * j;
                    const uint32_t old = bytes >= 4 ? ~0u : bytes <= 0 ? 0u : (1u << (8 * bytes)) - 1u;
                    w[j] = (r[j] & old) | (w[j] & ~old);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const int place = place0 + j;
            if (place >= lo && place < hi) {
                const uint32_t one = turned[(place - lo) * stride + d];
                w[j / 4] = (w[j / 4] & ~(0xFFu << (8 * (j % 4)))) | one << (8 * (j % 4));
            }
        }
        *p = w;
    }
}

// Rows at or beyond a sequence's length, and those of a page that is not there, are zeros.
template <typename T> __global__ void __launch_bounds__(256) restore_kernel(Call a)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t turned[];
    const Cache& c = a.c;
    const bool values = blockIdx.x & 1;
    const uint32_t id = blockIdx.x >> 1;
    const int h = (int)(id % (uint32_t)c.kv_heads), slot = (int)(id / (uint32_t)c.kv_heads % (uint32_t)a.slots), b = (int)(id / (uint32_t)c.kv_heads / (uint32_t)a.slots);
    const int first = slot << c.shift, pt = c.page_tokens(), kl = clamped(a.k_len, b, a.tokens);
    const int rows = a.tokens - first < pt ? a.tokens - first : pt, page = first < kl ? c.page_of(b, first) : -1;
    const int there = page < 0 ? 0 : kl - first < rows ? kl - first : rows;
    const int64_t head = c.head_of(page < 0 ? 0 : page, h);
    const uint8_t* const codes = (values ? c.v : c.k) + head * c.page_bytes();
    const float scale = there > 0 ? two_to((values ? c.v_exps : c.k_exps)[head]) : 0.f;
    const int units = c.head_dim / kUnit, stride = c.head_dim + kPad;
    if (values) {
        for (int i = threadIdx.x; i < (there + 15) / 16 * c.head_dim; i += 256) {
            const int over = a.columns.quotient(i), d = i - over * c.head_dim, place0 = over * 16;
            const u32x4 w = *reinterpret_cast<const u32x4*>(codes + c.value_at(place0, d));
#pragma unroll
            for (int j = 0; j < 16; ++j) turned[(place0 + j) * stride + d] = (uint8_t)(w[j / 4] >> (8 * (j % 4)));
        }
        __syncthreads();
    }
    const Rows& to = values ? a.v : a.k;
    T* const out = reinterpret_cast<T*>(to.p) + b * to.batch + h * to.head + (int64_t)first * to.token;
    for (int i = threadIdx.x; i < rows * units; i += 256) {
        const int row = a.units.quotient(i), unit = i - row * units;
        float t[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) t[j] = 0.f;
        if (row < there) {
            u32x4 w;
            if (values) {
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = *reinterpret_cast<const uint32_t*>(turned + row * stride + unit * kUnit + 4 * j);
            } else {
                w = *reinterpret_cast<const u32x4*>(codes + c.key_at(row, unit * kUnit));
            }
            values_of(t, w, scale);
        }
        store16(out + (int64_t)row * to.token + unit * kUnit, t);
    }
}

size_t size_of(int32_t dtype) { return dtype == PRUNER_F32 ? 4 : 2; }
bool rows_ok(const pruner_heads* h, int32_t dtype) { return h && h->p && aligned(h->p, size_of(dtype)) && h->batch >= 0 && h->token >= 0 && h->head >= 0; }
Rows rows_of(const pruner_heads* h) { return Rows{static_cast<char*>(h->p), h->batch, h->token, h->head}; }

// What both calls refuse; slots: pages of a sequence, workgroups for each of a head's keys and values.
int check(const pruner_cache* c, int32_t dtype, int32_t batch, int32_t tokens, const int32_t* q_len, const int32_t* k_len, const pruner_heads* k, const pruner_heads* v, int64_t slots)
{
    if (!cache_ok(c) || dtype < PRUNER_BF16 || dtype > PRUNER_F32 || batch < 0 || tokens < 0 || tokens >= (1 << 30)) return PRUNER_EINVAL;
    if (!c->table && (int64_t)batch * c->seq_pages > c->pages) return PRUNER_EINVAL;
    if ((q_len && !aligned(q_len, 4)) || (k_len && !aligned(k_len, 4))) return PRUNER_EINVAL;
    if (batch == 0 || tokens == 0) return PRUNER_OK;
    if (!rows_ok(k, dtype) || !rows_ok(v, dtype)) return PRUNER_EINVAL;
    return 2 * (double)slots * batch * c->kv_heads < (double)(1 << 24) ? PRUNER_OK : PRUNER_EINVAL;   // (a launch is below 2^24 workgroups of 256 threads)
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
    const cache::Call call{cache::cache_of(c), cache::rows_of(k), cache::rows_of(v), q_len, k_len, batch, tokens, (int32_t)slots, cache::Over(c->head_dim / cache::kUnit), cache::Over(c->head_dim)};
    const dim3 grid((unsigned)(2 * slots * batch * c->kv_heads));
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
    const cache::Call call{cache::cache_of(c), cache::rows_of(k), cache::rows_of(v), nullptr, k_len, batch, tokens, (int32_t)slots, cache::Over(c->head_dim / cache::kUnit), cache::Over(c->head_dim)};
    const dim3 grid((unsigned)(2 * slots * batch * c->kv_heads));
    const size_t lds = (size_t)c->page_tokens * (c->head_dim + cache::kPad);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == PRUNER_BF16)
        hipLaunchKernelGGL((cache::restore_kernel<__bf16>), grid, dim3(256), lds, st, call);
    else if (dtype == PRUNER_F16)
        hipLaunchKernelGGL((cache::restore_kernel<_Float16>), grid, dim3(256), lds, st, call);
    else
        hipLaunchKernelGGL((cache::restore_kernel<float>), grid, dim3(256), lds, st, call);
    PRUNER_LAUNCH_CHECK();
    return PRUNER_OK;
}
