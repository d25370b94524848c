// Positions by rotation: pairs of a head's columns turn by an angle that grows with the position,
//     (a, b) -> amplitude (a cos t - b sin t, b cos t + a sin t),   t = p f_i;    its gradient is the same by -t.
// Angles are exact at any position: a frequency is held as turns per position in 64 bits of fraction, so that the product with the position wraps at whole
// turns as the angle does; the quadrant is its two highest bits, and what is left, at most an eighth of a turn, goes to binary32 and the series of sine and cosine
// (x^9 / 9!, x^10 / 10!; the next terms are below 2e-9).
// A workgroup takes a few tokens: it forms their sines and cosines once, in LDS, and goes through the columns of all their heads as they lie in memory, sixteen bytes (with pairs half
// of the columns apart, twice sixteen) to a thread.  Bound: memory; in bfloat16 16384 tokens, 40 heads of 128, 62 us, 5.4 TB/s (a large copy: 5.2); gradients of 9009 tokens in binary32, 15 heads of 100, whose rows begin and end
// inside lines, 26 us, 4.2 TB/s; one token 10 us a call, of which the kernel is 4.
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
    int32_t units, all_units;   // of a head: those that turn, and with those that are copied
    int32_t rows_each;          // tokens of a workgroup
    int32_t first;              // workgroup, of those of a call, that a launch begins with
    float amplitude;
    int32_t back;
    uint64_t turn[PRUNER_MAX_ROTARY_DIM / 2];       // 2^-64 turns per position
    __device__ __forceinline__ int queries(int b) const   // (as the cache and its attention take them)
    {
        if (!q_len) return tokens;
        const int n = q_len[b];
        return n < 0 ? 0 : n > tokens ? tokens : n;
    }
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
    template <bool ONCE> __device__ __forceinline__ void store(T* p) const
    {
        if constexpr (ONCE)
            __builtin_nontemporal_store(w, reinterpret_cast<Loose*>(p));
        else
            *reinterpret_cast<Loose*>(p) = w;
    }
};

struct RowAt {
    int64_t x[2], y[2];   // elements: where a token's queries and keys begin
};

// ONCE: inputs and outputs are more than the caches are good for.
template <typename T, bool SIDE_BY_SIDE, bool ONCE> __global__ void __launch_bounds__(256) turn_kernel(Call a)
{
    constexpr int kN = Vec<T>::kN, kPairs = SIDE_BY_SIDE ? kN / 2 : kN, kAtOnce = 4;   // pairs of a unit; units that a thread asks for before it works on them
    extern __shared__ __attribute__((aligned(16))) char lds[];
    RowAt* const rows_at = reinterpret_cast<RowAt*>(lds);
    f32x2* const angles = reinterpret_cast<f32x2*>(lds + a.rows_each * sizeof(RowAt));   // [token][pair] sine and cosine
    const int64_t all_rows = (int64_t)a.batch * a.tokens, row0 = ((int64_t)a.first + blockIdx.x) * a.rows_each;
    const int rows = all_rows - row0 < a.rows_each ? (int)(all_rows - row0) : a.rows_each;
    for (int i = threadIdx.x; i < rows * a.pairs; i += 256) {
        const int row = i / a.pairs, pair = i - row * a.pairs, b = (int)((row0 + row) / a.tokens), t = (int)((row0 + row) - (int64_t)b * a.tokens);
        const int p = a.positions ? a.positions[row0 + row] : (int)((uint32_t)t + (a.k_len ? (uint32_t)a.k_len[b] - (uint32_t)a.queries(b) : 0u));
        float s, c;
        angle_of(a.turn[pair], p, s, c);
        angles[i] = f32x2{(a.back ? -s : s) * a.amplitude, c * a.amplitude};
        if (pair == 0)
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                rows_at[row].x[w] = b * a.x[w].batch + t * a.x[w].token;
                rows_at[row].y[w] = b * a.y[w].batch + t * a.y[w].token;
            }
    }
    __syncthreads();
    // (unit, head, token) of this thread's first item, and how far the next one is
    const int heads = a.heads[0] + a.heads[1];
    int unit = (int)threadIdx.x % a.all_units, head = (int)threadIdx.x / a.all_units % heads, row = (int)threadIdx.x / a.all_units / heads;
    const int unit_step = 256 % a.all_units, head_step = 256 / a.all_units % heads, row_step = 256 / a.all_units / heads;
    while (row < rows) {
        Vec<T> u[kAtOnce], v[kAtOnce];
        T* to[kAtOnce];
        const f32x2* by[kAtOnce];
        int pairs[kAtOnce];   // pairs of the unit; 0: none, below 0: columns that are copied
#pragma unroll
        for (int n = 0; n < kAtOnce; ++n) {
            const int which = head >= a.heads[0] ? 1 : 0, h = head - (which ? a.heads[0] : 0), first = unit * kPairs;
            const bool turns = unit < a.units;
            const int d = !turns ? 2 * a.pairs + (unit - a.units) * kN : SIDE_BY_SIDE ? 2 * first : first;
            pairs[n] = 0;
            if (row < rows) {
                const T* const x = reinterpret_cast<const T*>(which ? a.x[1].p : a.x[0].p) + rows_at[row].x[which] + h * (which ? a.x[1].head : a.x[0].head) + d;
                to[n] = reinterpret_cast<T*>(which ? a.y[1].p : a.y[0].p) + rows_at[row].y[which] + h * (which ? a.y[1].head : a.y[0].head) + d;
                by[n] = angles + row * a.pairs + first;
                if (turns) {
                    pairs[n] = a.pairs - first < kPairs ? a.pairs - first : kPairs;
                    if (pairs[n] == kPairs) {
                        u[n].template load<ONCE>(x);
                        if constexpr (!SIDE_BY_SIDE) v[n].template load<ONCE>(x + a.pairs);
                    } else {
#pragma unroll
                        for (int i = 0; i < kPairs; ++i)
                            if (i < pairs[n]) {
                                if constexpr (SIDE_BY_SIDE) {
                                    u[n].w[2 * i] = x[2 * i];
                                    u[n].w[2 * i + 1] = x[2 * i + 1];
                                } else {
                                    u[n].w[i] = x[i];
                                    v[n].w[i] = x[a.pairs + i];
                                }
                            }
                    }
                } else {
                    pairs[n] = a.head_dim - d < kN ? d - a.head_dim : -kN;
                    if (pairs[n] == -kN) {
                        u[n].template load<ONCE>(x);
                    } else {
#pragma unroll
                        for (int i = 0; i < kN; ++i)
                            if (i < -pairs[n]) u[n].w[i] = x[i];
                    }
                }
            }
            unit += unit_step;
            const int carry = unit >= a.all_units ? 1 : 0;
            unit -= carry ? a.all_units : 0;
            head += head_step + carry;
            const int over = head >= heads ? 1 : 0;
            head -= over ? heads : 0;
            row += row_step + over;
        }
#pragma unroll
        for (int n = 0; n < kAtOnce; ++n) {
            if (pairs[n] > 0)
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    const f32x2 sc = by[n][i < pairs[n] ? i : 0];
                    if constexpr (SIDE_BY_SIDE) {
                        const float p = (float)u[n].w[2 * i], q = (float)u[n].w[2 * i + 1];
                        u[n].w[2 * i] = (T)__builtin_fmaf(p, sc[1], -(q * sc[0]));
                        u[n].w[2 * i + 1] = (T)__builtin_fmaf(q, sc[1], p * sc[0]);
                    } else {
                        const float p = (float)u[n].w[i], q = (float)v[n].w[i];
                        u[n].w[i] = (T)__builtin_fmaf(p, sc[1], -(q * sc[0]));
                        v[n].w[i] = (T)__builtin_fmaf(q, sc[1], p * sc[0]);
                    }
                }
            if (pairs[n] == kPairs) {
                u[n].template store<ONCE>(to[n]);
                if constexpr (!SIDE_BY_SIDE) v[n].template store<ONCE>(to[n] + a.pairs);
            } else if (pairs[n] == -kN) {
                u[n].template store<ONCE>(to[n]);
            } else if (pairs[n] > 0) {
#pragma unroll
                for (int i = 0; i < kPairs; ++i)
                    if (i < pairs[n]) {
                        if constexpr (SIDE_BY_SIDE) {
                            to[n][2 * i] = u[n].w[2 * i];
                            to[n][2 * i + 1] = u[n].w[2 * i + 1];
                        } else {
                            to[n][i] = u[n].w[i];
                            to[n][a.pairs + i] = v[n].w[i];
                        }
                    }
            } else if (pairs[n] < 0) {
#pragma unroll
                for (int i = 0; i < kN; ++i)
                    if (i < -pairs[n]) to[n][i] = u[n].w[i];
            }
        }
    }
}

size_t size_of(int32_t dtype) { return dtype == PRUNER_F32 ? 4 : 2; }
bool rows_ok(const pruner_heads* h, int32_t dtype) { return h && h->p && aligned(h->p, size_of(dtype)) && h->batch >= 0 && h->token >= 0 && h->head >= 0; }
Rows rows_of(const pruner_heads* h) { return Rows{static_cast<char*>(h->p), h->batch, h->token, h->head}; }

// Bytes of input from which on accesses go past the caches: half of the last one.  (us a call past them and not: heads of 128 in bfloat16, 42 MB 21 and 24 where results lie in new memory each time, 20 and 17
// where they find the last call's; new memory, 63 MB 26 and 28, 105 MB 40 and 46, 127 MB 48 and 53, 168 MB 61 and 68, 246 MB 88 and 96; with loads alone past them 168 MB 67.)
constexpr int64_t kCached = 128 << 20;
// And only where an access leaves no parts of lines to others: past the caches those are not put together.  What is written lies in pieces: with pairs side by side and nothing copied a token's heads, else half
// heads, or what turns of a head, and what is copied.  (168 MB, us a call past the caches and not.  Pairs half of the columns apart: bfloat16, heads of 128 61 and 68, 96 74 and 69, 80 75 and 69, 100 170 and 100;
// binary32, heads of 96 64 and 68, 80 69 and 68, 100 122 and 77; bfloat16 in place in rows that begin 2 bytes behind a line 94 and 71.  Side by side: bfloat16, heads of 80 61 and 67, 100 104 and 79, 80 in place in
// such rows 104 and 73, 128 of which 64 turn 64 and 74; binary32, heads of 100 60 and 67, of which 36 turn 101 and 81.)
constexpr int64_t kLine = 64;
bool whole(int64_t piece) { return piece % kLine == 0 && piece >= 2 * kLine; }   // bytes; (pieces of 64: 67.9 and 67.5, 67.1 and 69.0, 73.6 and 70.7)
bool leaves_no_parts(const Call& a, bool side_by_side, bool in_place, int64_t size)
{
    const bool copied = a.rest > 0 && !in_place;
    for (int w = 0; w < 2; ++w) {
        if (a.heads[w] == 0) continue;
        const Rows& y = a.y[w];
        const int64_t row = (int64_t)a.heads[w] * a.head_dim;
        const bool side_by_side_rows = side_by_side && a.rest == 0 && a.pairs * 2 * size % 16 == 0 && (a.heads[w] == 1 || y.head == a.head_dim) && (y.token == row || row * size >= 1024) && aligned(y.p, 16);
        if (side_by_side_rows) continue;
        if (!whole((side_by_side ? 2 : 1) * a.pairs * size) || (copied && !whole(a.rest * size))) return false;
        if (!aligned(y.p, kLine) || y.batch * size % kLine || y.token * size % kLine || y.head * size % kLine) return false;
    }
    return true;
}
// Units of a workgroup, about.  (1024, 2048 and 4096, us a call: 168 MB in 64, 69, 75; 54 MB in heads of 100 30, 30, 32.)
constexpr int kItems = 1024;

template <typename T> int launch(Call& a, bool side_by_side, bool in_place, hipStream_t st)
{
    constexpr int kN = Vec<T>::kN;
    const int pairs = side_by_side ? kN / 2 : kN, heads = a.heads[0] + a.heads[1];
    a.units = (a.pairs + pairs - 1) / pairs;
    a.all_units = a.units + (in_place ? 0 : (a.rest + kN - 1) / kN);
    const int64_t rows = (int64_t)a.batch * a.tokens, items = (int64_t)a.all_units * heads;
    a.rows_each = items >= kItems ? 1 : (int)(kItems / items < 16 ? kItems / items : 16);
    const int64_t blocks = (rows + a.rows_each - 1) / a.rows_each;
    const bool once = rows * heads * a.head_dim * (int64_t)sizeof(T) > kCached && leaves_no_parts(a, side_by_side, in_place, sizeof(T));
    void (*const kernel)(Call) = side_by_side ? (once ? turn_kernel<T, true, true> : turn_kernel<T, true, false>) : once ? turn_kernel<T, false, true> : turn_kernel<T, false, false>;
    constexpr int64_t kLaunch = 1 << 23;   // (a launch is below 2^24 workgroups of 256 threads)
    for (int64_t first = 0; first < blocks; first += kLaunch) {
        a.first = (int32_t)first;
        hipLaunchKernelGGL(kernel, dim3((unsigned)(blocks - first < kLaunch ? blocks - first : kLaunch)), dim3(256), (size_t)a.rows_each * (sizeof(RowAt) + (size_t)a.pairs * 8), st, a);
        PRUNER_LAUNCH_CHECK();
    }
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
