// Positions by rotation: pairs of a head's columns turn by an angle that grows with the position,
//     (a, b) -> amplitude (a cos t - b sin t, b cos t + a sin t),   t = p f_i;    its gradient is the same by -t.
// Angles are exact at any position: a frequency is held as turns per position in 64 bits of fraction, so that the product with the position wraps at whole
// turns as the angle does; the quadrant is its two highest bits, and what is left, at most an eighth of a turn, goes to binary32 and the series of sine and cosine
// (x^9 / 9!, x^10 / 10!; the next terms are below 2e-9).
// A thread takes pairs of one token for several heads in turn, and forms their sines and cosines once.  Bound: memory.
#include "common.h"

#include <math.h>

namespace pruner {
namespace rotary {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Rows {
    char* p;
    int64_t batch, token, head;   // elements
};
struct Call {
    Rows x[2], y[2];   // queries, keys
    int32_t heads[2];
    const int32_t *positions, *q_len, *k_len;
    int32_t batch, tokens, head_dim, pairs, rest;   // rest: columns behind the pairs that are copied
    int32_t units, rest_units, each;                // of a head; heads that a thread takes
    float amplitude;
    int32_t back;
    uint64_t turn[PRUNER_MAX_ROTARY_DIM / 2];       // 2^-64 turns per position
};

// sin and cos of p times a pair's frequency.
__device__ __forceinline__ void angle_of(uint64_t turn, int p, float& s, float& c)
{
    const uint64_t at = turn * (uint64_t)(int64_t)p;
    const uint32_t quarter = (uint32_t)((at + (1ull << 61)) >> 62);
    const int64_t left = (int64_t)(at - ((uint64_t)quarter << 62));
    const float x = __builtin_fmaf((float)(int32_t)(left >> 32), 0x1p32f, (float)(uint32_t)left) * 0x1.921fb6p-62f;   // 2 pi 2^-64
    const float q = x * x;
    float a = __builtin_fmaf(q, 0x1.71de3ap-19f, -0x1.a01a02p-13f);   // 1 / 9!, -1 / 7!, 1 / 5!, -1 / 3!
    a = __builtin_fmaf(q, a, 0x1.111112p-7f);
    a = __builtin_fmaf(q, a, -0x1.555556p-3f);
    a = __builtin_fmaf(x * q, a, x);
    float b = __builtin_fmaf(q, -0x1.27e4fcp-22f, 0x1.a01a02p-16f);   // -1 / 10!, 1 / 8!, -1 / 6!, 1 / 4!, -1 / 2!
    b = __builtin_fmaf(q, b, -0x1.6c16c2p-10f);
    b = __builtin_fmaf(q, b, 0x1.555556p-5f);
    b = __builtin_fmaf(q, b, -0.5f);
    b = __builtin_fmaf(q, b, 1.f);
    s = quarter & 1 ? b : a;
    c = quarter & 1 ? a : b;
    s = quarter & 2 ? -s : s;
    c = (quarter + 1) & 2 ? -c : c;
}

// Sixteen bytes of neighbouring values, anywhere in memory.
template <typename T> struct Vec {
    static constexpr int kN = 16 / (int)sizeof(T);
    typedef T Values __attribute__((ext_vector_type(kN)));
    typedef Values Loose __attribute__((aligned(sizeof(T))));
    Values w;
    template <bool ONCE> __device__ __forceinline__ void load(const T* p)
    {
        if constexpr (ONCE)
            w = __builtin_nontemporal_load(reinterpret_cast<const Loose*>(p));
        else
            w = *reinterpret_cast<const Loose*>(p);
    }
    __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<Loose*>(p) = w; }
};

// ONCE: inputs are more than the caches keep, and are not to take the outputs' place there (us a call with and without: 168 MB of bfloat16 in, 59 and 71, 126 MB 46 and 46, 42 MB 19 and 17;
// writes that are not kept either: 70).
template <typename T, bool SIDE_BY_SIDE, bool ONCE> __global__ void __launch_bounds__(256) turn_kernel(Call a, int rows_each)
{
    constexpr int kN = Vec<T>::kN, kPairs = SIDE_BY_SIDE ? kN / 2 : kN;   // pairs of a unit: of one sixteen bytes, or of two
    const int all = a.units + a.rest_units, unit = (int)threadIdx.x % all, mine = (int)threadIdx.x / all;
    const int64_t row = (int64_t)blockIdx.x * rows_each + mine;
    if (mine >= rows_each || row >= (int64_t)a.batch * a.tokens) return;
    const int b = (int)(row / a.tokens), t = (int)(row % a.tokens);
    const int groups = (a.heads[0] + a.each - 1) / a.each, which = (int)blockIdx.y >= groups ? 1 : 0;
    const int first = ((int)blockIdx.y - (which ? groups : 0)) * a.each, last = first + a.each < a.heads[which] ? first + a.each : a.heads[which];
    const Rows& from = a.x[which];
    const Rows& to = a.y[which];
    const T* x = reinterpret_cast<const T*>(from.p) + b * from.batch + t * from.token + first * from.head;
    T* y = reinterpret_cast<T*>(to.p) + b * to.batch + t * to.token + first * to.head;
    if (unit >= a.units) {   // columns that do not turn
        const int d = 2 * a.pairs + (unit - a.units) * kN, n = a.head_dim - d < kN ? a.head_dim - d : kN;
        if (n == kN) {
#pragma unroll 4
            for (int h = first; h < last; ++h, x += from.head, y += to.head) {
                Vec<T> v;
                v.template load<ONCE>(x + d);
                v.store(y + d);
            }
        } else {
            for (int h = first; h < last; ++h, x += from.head, y += to.head)
                for (int i = 0; i < n; ++i) y[d + i] = x[d + i];
        }
        return;
    }
    int p;
    if (a.positions)
        p = a.positions[row];
    else
        p = t + (a.k_len ? a.k_len[b] - (a.q_len ? a.q_len[b] : a.tokens) : 0);
    const int pair0 = unit * kPairs, n = a.pairs - pair0 < kPairs ? a.pairs - pair0 : kPairs;
    float s[kPairs], c[kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
        angle_of(a.turn[pair0 + i < a.pairs ? pair0 + i : a.pairs - 1], p, s[i], c[i]);
        s[i] *= a.back ? -a.amplitude : a.amplitude;
        c[i] *= a.amplitude;
    }
    if (n == kPairs) {
#pragma unroll 4
        for (int h = first; h < last; ++h, x += from.head, y += to.head) {
            if constexpr (SIDE_BY_SIDE) {
                Vec<T> u;
                u.template load<ONCE>(x + 2 * pair0);
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    const float p0 = (float)u.w[2 * i], q0 = (float)u.w[2 * i + 1];
                    u.w[2 * i] = (T)__builtin_fmaf(p0, c[i], -(q0 * s[i]));
                    u.w[2 * i + 1] = (T)__builtin_fmaf(q0, c[i], p0 * s[i]);
                }
                u.store(y + 2 * pair0);
            } else {
                Vec<T> u, v;
                u.template load<ONCE>(x + pair0);
                v.template load<ONCE>(x + a.pairs + pair0);
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    const float p0 = (float)u.w[i], q0 = (float)v.w[i];
                    u.w[i] = (T)__builtin_fmaf(p0, c[i], -(q0 * s[i]));
                    v.w[i] = (T)__builtin_fmaf(q0, c[i], p0 * s[i]);
                }
                u.store(y + pair0);
                v.store(y + a.pairs + pair0);
            }
        }
    } else {
        for (int h = first; h < last; ++h, x += from.head, y += to.head)
#pragma unroll
            for (int i = 0; i < kPairs; ++i)
                if (i < n) {
                    const int at0 = SIDE_BY_SIDE ? 2 * (pair0 + i) : pair0 + i, at1 = SIDE_BY_SIDE ? at0 + 1 : a.pairs + at0;
                    const float p0 = (float)x[at0], q0 = (float)x[at1];
                    y[at0] = (T)__builtin_fmaf(p0, c[i], -(q0 * s[i]));
                    y[at1] = (T)__builtin_fmaf(q0, c[i], p0 * s[i]);
                }
    }
}

size_t size_of(int32_t dtype) { return dtype == PRUNER_F32 ? 4 : 2; }
bool rows_ok(const pruner_heads* h, int32_t dtype) { return h && h->p && aligned(h->p, size_of(dtype)) && h->batch >= 0 && h->token >= 0 && h->head >= 0; }
Rows rows_of(const pruner_heads* h) { return Rows{static_cast<char*>(h->p), h->batch, h->token, h->head}; }

constexpr int64_t kThreads = 1 << 18;   // that fill the device
constexpr int64_t kCached = 128 << 20;   // bytes of input: half of the last cache

template <typename T> int launch(Call& a, bool side_by_side, bool in_place, hipStream_t st)
{
    constexpr int kN = Vec<T>::kN;
    const int pairs = side_by_side ? kN / 2 : kN;
    a.units = (a.pairs + pairs - 1) / pairs;
    a.rest_units = in_place ? 0 : (a.rest + kN - 1) / kN;
    const int all = a.units + a.rest_units, rows_each = 256 / all;
    const int64_t rows = (int64_t)a.batch * a.tokens, threads = rows * all, blocks = (rows + rows_each - 1) / rows_each;
    if (blocks >= (1 << 24)) return PRUNER_EINVAL;   // (a launch is below 2^24 workgroups of 256 threads)
    const int heads = a.heads[0] > a.heads[1] ? a.heads[0] : a.heads[1];
    int64_t each = threads * (a.heads[0] + a.heads[1]) / kThreads;
    each = each < 1 ? 1 : each > 8 ? 8 : each;
    while ((a.heads[0] + a.heads[1]) / each > 60000) each *= 2;   // (a launch has at most 65535 workgroups in its second axis)
    a.each = (int)(each < heads ? each : heads);
    const int groups = (a.heads[0] + a.each - 1) / a.each + (a.heads[1] + a.each - 1) / a.each;
    const dim3 grid((unsigned)blocks, (unsigned)groups);
    const bool once = rows * (a.heads[0] + a.heads[1]) * a.head_dim * (int64_t)sizeof(T) > kCached;
    void (*const kernel)(Call, int) = side_by_side ? (once ? turn_kernel<T, true, true> : turn_kernel<T, true, false>) : once ? turn_kernel<T, false, true> : turn_kernel<T, false, false>;
    hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a, rows_each);
    PRUNER_LAUNCH_CHECK();
    return PRUNER_OK;
}

int turn(const pruner_rotation* r, const pruner_heads* q, const pruner_heads* k, const pruner_heads* q_out, const pruner_heads* k_out, bool back, void* stream)
{
    if (!r || r->dtype < PRUNER_BF16 || r->dtype > PRUNER_F32 || r->batch < 0 || r->tokens < 0 || r->tokens >= (1 << 30)) return PRUNER_EINVAL;
    if (r->q_heads < 0 || r->kv_heads < 0 || r->q_heads > 65535 || r->kv_heads > 65535 || r->head_dim < 2 || r->head_dim > PRUNER_MAX_ROTARY_HEAD) return PRUNER_EINVAL;
    if (r->rotary_dim < 2 || r->rotary_dim % 2 || r->rotary_dim > r->head_dim || r->rotary_dim > PRUNER_MAX_ROTARY_DIM || (r->flags & ~PRUNER_ROTARY_INTERLEAVED)) return PRUNER_EINVAL;
    if ((int64_t)r->batch * r->tokens >= (1 << 30) || !(fabsf(r->amplitude) < 3.0e38f) || !r->freqs) return PRUNER_EINVAL;
    if ((r->positions && !aligned(r->positions, 4)) || (r->q_len && !aligned(r->q_len, 4)) || (r->k_len && !aligned(r->k_len, 4))) return PRUNER_EINVAL;
    Call a{};
    a.pairs = r->rotary_dim / 2;
    for (int i = 0; i < a.pairs; ++i) {
        if (!(fabs(r->freqs[i]) <= PRUNER_MAX_ROTARY_FREQUENCY)) return PRUNER_EINVAL;
        a.turn[i] = (uint64_t)(__int128)((long double)r->freqs[i] * 2935890503282001226.496L);   // 2^64 / (2 pi), to the 64 bits of a long double; whole turns are the bits above
    }
    if (r->batch == 0 || r->tokens == 0 || r->q_heads + r->kv_heads == 0) return PRUNER_OK;
    if (r->q_heads > 0 && (!rows_ok(q, r->dtype) || !rows_ok(q_out, r->dtype))) return PRUNER_EINVAL;
    if (r->kv_heads > 0 && (!rows_ok(k, r->dtype) || !rows_ok(k_out, r->dtype))) return PRUNER_EINVAL;
    bool in_place = true;
    const pruner_heads* const from[2] = {q, k};
    const pruner_heads* const to[2] = {q_out, k_out};
    for (int w = 0; w < 2; ++w) {
        a.heads[w] = w ? r->kv_heads : r->q_heads;
        if (a.heads[w] == 0) continue;
        a.x[w] = rows_of(from[w]);
        a.y[w] = rows_of(to[w]);
        const bool same = from[w]->p == to[w]->p;
        if (same && (from[w]->batch != to[w]->batch || from[w]->token != to[w]->token || from[w]->head != to[w]->head)) return PRUNER_EINVAL;
        in_place = in_place && same;
    }
    a.positions = r->positions;
    a.q_len = r->q_len;
    a.k_len = r->k_len;
    a.batch = r->batch;
    a.tokens = r->tokens;
    a.head_dim = r->head_dim;
    a.rest = r->head_dim - r->rotary_dim;
    a.amplitude = r->amplitude;
    a.back = back;
    const bool side_by_side = r->flags & PRUNER_ROTARY_INTERLEAVED;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return r->dtype == PRUNER_BF16  ? launch<__bf16>(a, side_by_side, in_place, st)
           : r->dtype == PRUNER_F16 ? launch<_Float16>(a, side_by_side, in_place, st)
                                    : launch<float>(a, side_by_side, in_place, st);
}

}  // namespace
}  // namespace rotary
}  // namespace pruner

extern "C" int pruner_rotary(const pruner_rotation* r, const pruner_heads* q, const pruner_heads* k, const pruner_heads* q_out, const pruner_heads* k_out, void* stream)
{
    return pruner::rotary::turn(r, q, k, q_out, k_out, false, stream);
}

extern "C" int pruner_rotary_grad(const pruner_rotation* r, const pruner_heads* dq_out, const pruner_heads* dk_out, const pruner_heads* dq, const pruner_heads* dk, void* stream)
{
    return pruner::rotary::turn(r, dq_out, dk_out, dq, dk, true, stream);
}
