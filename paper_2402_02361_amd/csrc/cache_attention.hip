// Attention over keys and values held in 8 bits in pages: pruner_rel_attention's formulas with k^ = code 2^e, v^ = code 2^e.
//
// A column is a pair of a query and a head, of those that share a key head: query t of the group's head g is column t * group + g.  S^T = K Q^T leaves a column's scores in a few lanes, whose softmax runs
// with a maximum and a sum, and the weights are the next product's operand as they stand (O^T += V^T P^T).  Which key a row of the first product's operand is, is ours to choose: a lane's sixteen
// scores are made to be of sixteen neighbouring keys, the depth that sixteen bytes of values have.  A page's powers of two go in with the conversion, which is exact (binary16: within its range).  The
// second product is of 16-bit operands, the rate of the matrix cores; the weights' sum is of the unrounded ones.  Few columns have weights in two terms (bfloat16, off by 2^-16), for which there is room beside the
// reading.  Of many columns they are rounded to the operands' type: two terms take 685 us where one takes 515 to 520, a second term in 8 bits, by products of 64 keys that take the codes as they are, 637 (2048 tokens
// against 16384, 32 heads of 128 sharing 8, one card; the result is off by 2.4e-3 of itself, of which its own rounding makes 1.65e-3, in binary16 2.9e-4 and 2.1e-4; with either second term by its rounding alone).
//
//   tokens_kernel       at most 32 columns, on v_mfma_f32_16x16x32: the four wavefronts of a workgroup take 64 keys each in turn and meet in LDS at the end.  Codes go from memory straight to the lanes whose
//                       operands they become, 64 bytes a lane ahead of the products for keys and values each.  Products of 32 x 32 x 16 held half as many wavefronts and took 315 us where this takes 200.
//                       Bound by memory: one token against 32 caches of up to 32768, 32 heads of 128 sharing 8, 195 to 200 us, 5.3 to 5.5 TB/s (a large copy: 5.2 read and written together);
//                       short ones by a workgroup's chain of lengths, pages, codes: one token against a cache of 300, 8 heads of 64, 11.6 us a call, with 5 queries each of 16 sequences of up to 5003
//                       in pages of 16, 16 heads of 80 sharing 4, 21.5 (heads of 64 20.6, of 128 26.4).
//   codes_kernel        more columns, 32 to a wavefront, on v_mfma_f32_32x32x16, over pages of 64 tokens and more.  The four wavefronts share tiles of 64 keys and values in LDS, which are requested straight
//                       to it as codes and converted by who reads them.  Bound by the matrix cores, the exponentials and conversions beside their products, and the clock under both: 2048 tokens against
//                       16384, 32 heads of 128 sharing 8, in hundreds of calls in a row 505 to 530 us, 970 to 1020 TFLOP/s (the first dozen after a pause 535 to 600); heads of 112, 96 and 80 511, 498 and 492, since the products
//                       are those of 128 columns; 2000 against 8000, 16 heads of 64 sharing 4, 127 us; 64 against 30000 58.
//                       Converted tiles in LDS as below: 543, 138 and 61.  Codes in LDS without the next tile's scores among this one's weights 542 (three wavefronts to a SIMD, by scores of 32 keys, 557);
//                       with them, but a memory access for each tile's page, its requests all between the steps, and scores copied there from register to register, 545.
//   chunk_kernel        the same over smaller pages: tiles in LDS hold operands, so that a code is converted once for 128 columns, and the next tile's are parked among this one's scores and softmax.
//                       8 sequences of 100 tokens against up to 800 in pages of 16, 16 heads of 64 sharing 4, 27 us, by a workgroup's start and chain of tiles; 2048 tokens against 16384 in pages of 16 or 32, 32 heads of 128
//                       sharing 8, 610 (516 over pages of 128), by LDS and the threads that convert and park.
//                       (Wavefronts' priorities raised for products or for the softmax: 1 to 4 % longer; eight wavefronts that share a tile 4 % longer; 64 columns to a wavefront a quarter longer.)
//   join_groups_kernel  the parts of a key axis that was split over workgroups.
#include "attention_softmax.h"
#include "cache.h"

namespace pruner {
namespace att {
namespace {

constexpr int kTile = 64;   // keys of a step

constexpr int kBiasHeads = 128;   // heads whose biases a workgroup holds: its columns', at most

// A wavefront's 32 columns (those past the last are the last once more, and not its own).
struct Columns {
    int t, h, bias, p, limit, all_see, q_first, q_last;   // of this lane: query, head, where its head's biases lie, position, keys that it sees; of the wavefront: keys that all see, its queries
    bool mine;
    __device__ __forceinline__ void set(const Args& a, int hk, int from, int first, int columns, int ql, int kl, int lane)   // from: the workgroup's first column, first: the wavefront's
    {
        const int last = first + 31 < columns ? first + 31 : columns - 1, c = first + (lane & 31) < last ? first + (lane & 31) : last;
        t = c / a.group;
        h = hk * a.group + c % a.group;
        bias = a.group <= kBiasHeads ? c % a.group : c - from;
        mine = first + (lane & 31) <= last && t < ql;
        p = kl - ql + t;
        limit = a.causal ? (p + 1 < kl ? p + 1 : kl) : kl;
        q_first = first / a.group;
        q_last = last / a.group < ql ? last / a.group : ql - 1;
        const int sees = kl - ql + q_first + 1;
        all_see = a.causal && sees < kl ? sees : kl;
    }
};

// In LDS: the biases of the heads of a workgroup's columns (all of a group, or those of 128 columns from `from` on), and the bucket of every r that a step which
// is not wholly at one end can ask for.
struct BiasLds {
    int n_buckets, heads, biases, buckets;   // bytes
    __host__ __device__ explicit BiasLds(const Args& a)
        : n_buckets(a.table ? (a.n_edges + 1) * (a.two_sided ? 2 : 1) : 0), heads(a.group < kBiasHeads ? a.group : kBiasHeads), biases((n_buckets * heads * 4 + 15) & ~15),
          buckets(a.table ? (Window(a.left, a.right).size + 15) & ~15 : 0)
    {
    }
    __host__ __device__ int bytes() const { return biases + buckets; }
    template <typename T> __device__ __forceinline__ void fill(const Args& a, const Window& window, char* lds, int hk, int from) const
    {
        float* const bias = reinterpret_cast<float*>(lds);
        uint8_t* const bucket = reinterpret_cast<uint8_t*>(lds + biases);
        for (int i = threadIdx.x; i < n_buckets * heads; i += 256) bias[i] = a.bias<T>(i / heads, hk * a.group + (a.group <= kBiasHeads ? i % heads : (from + i % heads) % a.group));
        for (int i = threadIdx.x; i < window.size; i += 256) bucket[i] = (uint8_t)a.bucket(window.first + i);
    }
};

// ---- few columns: products of 16 x 16 x 32

__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c, __bf16)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c, _Float16)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// Eight weights as sums of two bfloat16: the nearest one, and the nearest to what that leaves, so off by 2^-16 of the weight at most (2^-8 of 2^-8), however small it is.  One term would be off by 2^-8, one of
// binary16 by 2^-11, and its smallest ones by all they are.
struct TwoTerms {
    u32x4 first, rest;
    __device__ __forceinline__ void set(f32x4 a, f32x4 b)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = (i < 2 ? a : b)[2 * (i % 2)], y = (i < 2 ? a : b)[2 * (i % 2) + 1];
            first[i] = pair_of(x, y, __bf16{});
            rest[i] = pair_of(x - __uint_as_float(first[i] << 16), y - __uint_as_float(first[i] & 0xFFFF0000u), __bf16{});
        }
    }
};
// Of a lane and the three of the same column in the other rows of sixteen.
__device__ __forceinline__ float max_of_rows(float v)
{
    const TwoFloats t = across_rows(v);
    return max_of_halves(__builtin_fmaxf(t.a, t.b));
}
__device__ __forceinline__ float sum_of_rows(float v)
{
    const TwoFloats t = across_rows(v);
    return sum_of_halves(t.a + t.b);
}

// 64 keys' codes: keys in four operands of 16 rows, row 4 u + j of operand t being key 16 u + 4 t + j, so that lane (n = lane & 15, g = lane >> 4) of the results has column n's scores of the sixteen
// keys 16 g + 4 t + j; of values it has the sixteen of those keys.  WHOLE: the 64 keys lie in one page, whose place all lanes share.
template <typename T, int DP, bool WHOLE, bool ONCE> struct Few {
    static constexpr int kChunks = (DP + 63) / 64, kBlocks = DP / 16, kSure = DP == 32 ? 1 : DP / 32 + 1;   // kSure: blocks of 16 columns that every head of this instance has; others may be past the last
    u32x4 k[4][kChunks], v[kBlocks];
    int k_byte, v_byte, k_page, v_page, there;   // (exponents and pages as memory has them: what is asked for ahead is looked at when it is used.  16 sequences of up to 5003 in pages of 16, us a call, without and with: 24.9 and 23.7)
    __device__ __forceinline__ void find(const cache::Cache& c, int b, int key0, int most, int lane)   // most: the sequences' room (their lengths may still be on the way)
    {
        if constexpr (WHOLE) {
            k_page = v_page = key0 < most ? c.number_of(b, key0) : -1;
        } else {
            const int k_at = key0 + 16 * (lane >> 2 & 3), v_at = key0 + 16 * (lane >> 4);
            k_page = k_at < most ? c.number_of(b, k_at) : -1;
            v_page = v_at < most ? c.number_of(b, v_at) : -1;
        }
    }
    __device__ __forceinline__ void load_keys(const cache::Cache& c, int h, int key0, int lane)
    {
        const int64_t head = c.head_of(c.is_page(k_page) ? k_page : 0, h);
        const int g = lane >> 4, in = c.page_tokens() - 1, place = WHOLE ? key0 & in : (key0 + 16 * (lane >> 2 & 3)) & in, units = c.head_dim / cache::kUnit;
        const uint8_t* const p = c.k + head * c.page_bytes() + 16 * place;
        k_byte = c.k_exps[head];
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            const int unit = 4 * i + g < units ? 4 * i + g : units - 1;   // (past the last one: the query's columns are 0 there)
            const uint32_t at = ((uint32_t)unit << (c.shift + 4)) + 16 * ((WHOLE ? 16 * (lane >> 2 & 3) : 0) + (lane & 3));
            if constexpr (ONCE) {
#pragma unroll
                for (int t = 0; t < 4; ++t) k[t][i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + at + 64 * t));
            } else {
#pragma unroll
                for (int t = 0; t < 4; ++t) k[t][i] = *reinterpret_cast<const u32x4*>(p + at + 64 * t);
            }
        }
    }
    __device__ __forceinline__ void load_values(const cache::Cache& c, int h, int key0, int kl, int lane)
    {
        const int64_t head = c.head_of(c.is_page(v_page) ? v_page : 0, h);
        const int g = lane >> 4, in = c.page_tokens() - 1, place = WHOLE ? key0 & in : (key0 + 16 * g) & in, units = c.head_dim / cache::kUnit, left = kl - (key0 + 16 * g);
        there = !c.is_page(v_page) || left < 0 ? 0 : left < 16 ? left : 16;
        const uint8_t* const p = c.v + head * c.page_bytes() + place * c.head_dim;
        v_byte = c.v_exps[head];
        const uint32_t at = 16 * ((WHOLE ? g * c.head_dim : 0) + (lane & 15));
#pragma unroll
        for (int i = 0; i < kBlocks; ++i)
            if (i < kSure || i < units) {
                if constexpr (ONCE)
                    v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + at + 256 * i));
                else
                    v[i] = *reinterpret_cast<const u32x4*>(p + at + 256 * i);
            }
    }
    __device__ __forceinline__ void clear_values()   // those that are not there (their page's byte may be anything as well: see two_to)
    {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int bytes = there - 4 * w;
            const uint32_t keep = bytes >= 4 ? ~0u : bytes <= 0 ? 0u : (1u << (8 * bytes)) - 1u;
#pragma unroll
            for (int i = 0; i < kBlocks; ++i) v[i][w] &= keep;
        }
    }
};

// ONCE: the caches hold more than stays cached from one call to the next, and are read past it (us a call with and without: 32 caches of 32768, 8 heads of 128, 348 and 379, of up to 32768 201 and 208;
// 8 of up to 20000 51 and 52; 16 of up to 5003, 4 heads of 80, 26 and 24; with other caches in each call 4 of 8000 20.2 and 21.3, 8 of 8000 31 and 34, of 12000 42 and 46, of 16000 52 and 58, of 20000 63 and 71;
// heads of 32 to 112 as those of 128).
template <typename T, int DP, int CT, bool WHOLE, bool ONCE>
__global__ void __launch_bounds__(256, (CT == 1 && (WHOLE || DP < 128) ? 3 : 2)) tokens_kernel(Args a, cache::Cache c, Heads out, float* __restrict__ lse, Parts parts)
{
    using Step = Few<T, DP, WHOLE, ONCE>;
    constexpr int kChunks = Step::kChunks, kBlocks = Step::kBlocks, kStep = 4 * kTile;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
    const int columns = a.q_tokens * a.group;
    const int hk = blockIdx.x % a.kv_heads, part = blockIdx.x / a.kv_heads % parts.count, b = blockIdx.x / a.kv_heads / parts.count;
    const int begin = part * parts.keys;
    int key0 = begin + kTile * wave;
    Step codes;
    codes.find(c, b, key0, a.k_tokens, lane);
    const int ql = a.queries(b), kl = a.keys(b);
    int end = ql == 0 ? 0 : kl;   // (the last query sees all keys under the causal mask too)
    if (parts.count > 1) end = end < begin + parts.keys ? end : begin + parts.keys;

    // this lane's columns (those past the last are the last once more, and not its own)
    int t[CT], p[CT], limit[CT], head[CT];
    bool mine[CT];
#pragma unroll
    for (int x = 0; x < CT; ++x) {
        const int at = 16 * x + n < columns ? 16 * x + n : columns - 1;
        t[x] = at / a.group;
        head[x] = at % a.group;
        mine[x] = 16 * x + n < columns && t[x] < ql;
        p[x] = kl - ql + t[x];
        limit[x] = a.causal ? (p[x] + 1 < kl ? p[x] + 1 : kl) : kl;
    }
    const int all_see = a.causal ? (kl - ql + 1 < kl ? kl - ql + 1 : kl) : kl;
    float m[CT], l[CT];
    f32x4 o[CT][kBlocks];
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < CT; ++x) {
        m[x] = -ATT_INF;
        l[x] = 0.f;
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) o[x][i] = zero;
    }
    if (begin < end) {
        if (key0 < end) {
            codes.load_keys(c, hk, key0, lane);
            codes.load_values(c, hk, key0, kl, lane);
            codes.find(c, b, key0 + kStep, a.k_tokens, lane);
        }
        u32x4 qf[CT][2 * kChunks];
#pragma unroll
        for (int x = 0; x < CT; ++x) {
            const T* const from = a.q.at<T>(b, hk * a.group + head[x]) + (int64_t)t[x] * a.q.token;
#pragma unroll
            for (int i = 0; i < 2 * kChunks; ++i) {
                const int d = 64 * (i / 2) + 16 * g + 8 * (i % 2);
                qf[x][i] = u32x4{0u, 0u, 0u, 0u};
                if (mine[x] && d < a.head_dim) qf[x][i] = *reinterpret_cast<const u32x4*>(from + d);
            }
        }
        const Window window(a.left, a.right);
        const BiasLds places(a);
        float bias_left[CT], bias_right[CT];
        if (a.table) {
#pragma unroll
            for (int x = 0; x < CT; ++x) {
                bias_left[x] = a.bias<T>(a.n_edges, hk * a.group + head[x]);
                bias_right[x] = a.bias<T>(a.two_sided ? 2 * a.n_edges + 1 : 0, hk * a.group + head[x]);
            }
            if (kl - ql - (end + kTile) < a.left) {   // (else all of this part's keys lie beyond the last edge)
                places.fill<T>(a, window, lds, hk, 0);
            }
            __syncthreads();
        }
        for (; key0 < end; key0 += kStep) {
            f32x4 s[CT][4];
            const float k_scale = cache::two_to(codes.k_byte);
#pragma unroll
            for (int x = 0; x < CT; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[x][i] = zero;
#pragma unroll
            for (int i = 0; i < 2 * kChunks; ++i)
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const u32x4 row = cache::eight_from<T>(codes.k[u][i / 2][2 * (i % 2)], codes.k[u][i / 2][2 * (i % 2) + 1], k_scale);
#pragma unroll
                    for (int x = 0; x < CT; ++x) s[x][u] = mfma16(row, qf[x][i], s[x][u], T{});
                }
            const int there = codes.there, next = key0 + kStep;
            const bool short_of = __any(there < 16);
            if (short_of) codes.clear_values();
            if (next < end) codes.load_keys(c, hk, next, lane);
            const int r_lo = key0 - (kl - ql + a.q_tokens - 1), r_hi = key0 + kTile - 1 - (kl - ql);
            const int place = a.table ? place_of(a, r_lo, r_hi) : kLeft;
#pragma unroll
            for (int x = 0; x < CT; ++x) {
                float shift = 0.f;
                bool fused = true;
                if (a.table) {
                    shift = place == kRight ? bias_right[x] : bias_left[x];
                    if (place == kNear) {
                        const uint8_t* const of = reinterpret_cast<const uint8_t*>(lds + places.biases) + (key0 - p[x] - window.first + 16 * g);
                        const float* const bias = reinterpret_cast<const float*>(lds) + head[x];
                        fused = false;
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[x][i / 4][i % 4] = __builtin_fmaf(s[x][i / 4][i % 4], a.scale, bias[of[i] * places.heads]);
                    } else if (__any(!(__builtin_fabsf(shift) < kLarge))) {   // (lanes have biases of different heads)
                        fused = false;
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[x][i / 4][i % 4] = __builtin_fmaf(s[x][i / 4][i % 4], a.scale, shift);
                    }
                }
                if (short_of || key0 + kTile > all_see) {
                    const int seen = limit[x] - (key0 + 16 * g), left = seen < there ? seen : there;
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[x][i / 4][i % 4] = i < left ? s[x][i / 4][i % 4] : -ATT_INF;
                }
                float top = s[x][0][0];
#pragma unroll
                for (int i = 1; i < 16; ++i) top = __builtin_fmaxf(top, s[x][i / 4][i % 4]);
                top = max_of_rows(top);
                if (fused) top = __builtin_fmaf(top, a.scale, shift);
                if (__any(top > m[x] + kSlack)) {   // (from minus infinity: any score)
                    const float now = __builtin_fmaxf(m[x], top), factor = now == -ATT_INF ? 1.f : exp2_of((m[x] - now) * kLog2e);
                    m[x] = now;
                    l[x] *= factor;
#pragma unroll
                    for (int i = 0; i < kBlocks; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[x][i][e] *= factor;
                }
                const float from = m[x] == -ATT_INF ? 0.f : m[x];   // (no key yet: every weight is exp(-infinity))
                float sum = 0.f;
                if (fused) {
                    const float scale = a.scale * kLog2e, off = (shift - from) * kLog2e;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        s[x][i / 4][i % 4] = exp2_of(__builtin_fmaf(s[x][i / 4][i % 4], scale, off));
                        sum += s[x][i / 4][i % 4];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        s[x][i / 4][i % 4] = exp2_of((s[x][i / 4][i % 4] - from) * kLog2e);
                        sum += s[x][i / 4][i % 4];
                    }
                }
                l[x] += sum;
            }
            const float v_scale = cache::two_to(codes.v_byte, there);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                TwoTerms w[CT];
#pragma unroll
                for (int x = 0; x < CT; ++x) w[x].set(s[x][2 * u], s[x][2 * u + 1]);
#pragma unroll
                for (int i = 0; i < kBlocks; ++i)
                    if (i < Step::kSure || 16 * i < a.head_dim) {
                        const u32x4 row = cache::eight_from<__bf16>(codes.v[i][2 * u], codes.v[i][2 * u + 1], v_scale);
#pragma unroll
                        for (int x = 0; x < CT; ++x) o[x][i] = mfma16(row, w[x].rest, mfma16(row, w[x].first, o[x][i], __bf16{}), __bf16{});
                    }
            }
            if (next < end) {
                codes.load_values(c, hk, next, kl, lane);
                codes.find(c, b, next + kStep, a.k_tokens, lane);
            }
        }
    }
    const Meeting<DP> at(lds);
    __syncthreads();
#pragma unroll
    for (int x = 0; x < CT; ++x) {
        const float sum = sum_of_rows(l[x]);
        if (g == 0) at.stats[wave * 32 + 16 * x + n] = make_float2(m[x], mine[x] ? sum : 0.f);
        if (16 * x + n < columns)
#pragma unroll
            for (int i = 0; i < kBlocks; ++i) *reinterpret_cast<f32x4*>(at.sums + (wave * columns + 16 * x + n) * Meeting<DP>::kStride + 16 * i + 4 * g) = o[x][i];
    }
    __syncthreads();
    at.template join<T>(a, out, lse, parts, b, hk, part, columns);
}

// ---- many columns, pages that hold whole tiles: codes in LDS

// Where a tile's codes lie: the head's place in the pool, and the exponents' bytes (keys', 256 times values'), or 0: the page is not there.
struct Held {
    uint32_t lo, hi, exps;
    __device__ __forceinline__ int bytes(const cache::Cache& c) const { return exps ? c.page_bytes() : 0; }
    __device__ __forceinline__ const uint8_t* in(const uint8_t* pool) const { return pool + ((uint64_t)hi << 32 | lo); }
    __device__ __forceinline__ float k_scale() const { return cache::two_to(exps & 255); }
    __device__ __forceinline__ float v_scale() const { return cache::two_to(exps >> 8 & 255); }
};

// 64 keys' codes of one page on their way to a tile that four wavefronts share, without registers on the way and as they lie in memory: keys in units of 16 columns of 64 keys, values in units of 16 tokens of
// DP columns.  A lane's sixteen bytes are two operands' eight, which it converts when it has read them.
template <int DP> struct Codes {
    static constexpr int kKeyBytes = kTile * DP, kBytes = 2 * kKeyBytes, kRequests = DP >= 64 ? DP / 64 : 1;   // requests of a wavefront for keys, and for values (32 columns: two wavefronts')
    uint32_t k_at[kRequests], v_at[kRequests];
    __device__ __forceinline__ void set(const cache::Cache& c, int wave, int lane)
    {
#pragma unroll
        for (int i = 0; i < kRequests; ++i) {
            const int unit = wave + 4 * i, group = (64 * unit + lane) / DP, d = (64 * unit + lane) % DP;
            k_at[i] = unit < c.head_dim / cache::kUnit ? 16u * (uint32_t)lane : 0x80000000u;   // (columns past the last are zeros: a query's are, but anything may be a NaN)
            v_at[i] = 16u * (uint32_t)(group * c.head_dim + (d < c.head_dim ? d : c.head_dim - 1));   // (columns past the last are not stored)
        }
    }
    // Request i of this wavefront's for the tile from key0 on.  A page that is not there: zeros.
    __device__ __forceinline__ void request_keys(const cache::Cache& c, const Held& of, int key0, uint32_t tile, int wave, int i) const
    {
        const u32x4 from = buffer_of(of.in(c.k), of.bytes(c));
        const uint32_t place = 16u * (uint32_t)(key0 & (c.page_tokens() - 1)), unit = (uint32_t)(wave + 4 * i);
        if (DP >= 64 || wave < 2) request_16(tile + 1024u * unit, k_at[i], from, (unit << (c.shift + 4)) + place);
    }
    __device__ __forceinline__ void request_values(const cache::Cache& c, const Held& of, int key0, uint32_t tile, int wave, int i) const
    {
        const u32x4 from = buffer_of(of.in(c.v), of.bytes(c));
        const uint32_t place = (uint32_t)((key0 & (c.page_tokens() - 1)) * c.head_dim);
        if (DP >= 64 || wave < 2) request_16(tile + kKeyBytes + 1024u * (uint32_t)(wave + 4 * i), v_at[i], from, place);
    }
    // Values of the tile's tokens from `there` on become zeros.  (Their weight is 0, but anything may be a NaN.)
    __device__ __forceinline__ static void clear(char* tile, int there)
    {
        for (int i = threadIdx.x; i < 4 * DP; i += 256) {
            u32x4* const p = reinterpret_cast<u32x4*>(tile + kKeyBytes + 16 * i);
            u32x4 w = *p;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int bytes = there - 16 * (i / DP) - 4 * j;
                w[j] &= bytes >= 4 ? ~0u : bytes <= 0 ? 0u : (1u << (8 * bytes)) - 1u;
            }
            *p = w;
        }
    }
};

// While a tile's weights are formed and its values added up, the next one's scores are made: a step's products and its exponentials do not wait for each other, which two wavefronts to a SIMD (as many as the
// queries' and sums' registers leave) do not hide.  So a step has the next tile's keys and this one's values, and asks for the keys after and the next values.  Queries' operands lie in LDS, for want of registers.
template <typename T, int DP> __global__ void __launch_bounds__(256, 2) codes_kernel(Args a, cache::Cache c, Heads out, float* __restrict__ lse, Parts parts, int tiles)
{
    using Turn = Codes<DP>;
    constexpr int kSteps = DP / 16, kBlocks = DP / 32;
    static_assert(2 * Turn::kBytes <= kRequestRoom, "tiles lie where requests reach");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), half = lane >> 5, l32 = lane & 31;
    u32x4* const queries = reinterpret_cast<u32x4*>(lds + 2 * Turn::kBytes) + kSteps * 64 * wave + lane;   // this lane's operands, 64 apart
    char* const bias_lds = lds + 2 * Turn::kBytes + 4096 * kSteps;
    const int columns = a.q_tokens * a.group;
    const Item it = item_of(blockIdx.x, (uint32_t)a.batch * a.kv_heads, 1, (uint32_t)tiles * parts.count);
    const int b = it.head / a.kv_heads, hk = it.head % a.kv_heads, part = it.tile % parts.count, from = it.tile / parts.count * 128, first = from + 32 * wave;
    const int begin = part * parts.keys;
    // pages and exponents of 64 tiles, one to a lane: accesses for each tile would be waited for at each
    Held lanes;
    auto hold = [&](int tile) {
        const int at = begin + kTile * (tile + lane), number = at < a.k_tokens ? c.number_of(b, at) : -1;
        const bool is = c.is_page(number);
        const int64_t head = c.head_of(is ? number : 0, hk), place = head * c.page_bytes();
        lanes.lo = (uint32_t)place;
        lanes.hi = (uint32_t)(place >> 32);
        lanes.exps = is ? (uint32_t)c.k_exps[head] | (uint32_t)c.v_exps[head] << 8 | 0x10000u : 0u;
    };
    auto held = [&](int tile) {
        auto of = [&](uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, tile & 63); };
        return Held{of(lanes.lo), of(lanes.hi), of(lanes.exps)};
    };
    const int ql = a.queries(b), kl = a.keys(b);
    Columns at;
    at.set(a, hk, from, first < columns ? first : columns - 1, columns, ql, kl, lane);
    if (first >= columns) at.mine = false;
    const Window window(a.left, a.right);
    const BiasLds places(a);
    // the keys that this workgroup's queries see, and of them this part's
    const int last_column = from + 127 < columns ? from + 127 : columns - 1, last = last_column / a.group < ql ? last_column / a.group : ql - 1;
    int end = a.causal && kl - ql + last + 1 < kl ? kl - ql + last + 1 : kl;
    if (from / a.group >= ql) end = 0;
    if (parts.count > 1) end = end < begin + parts.keys ? end : begin + parts.keys;

    float bias_left = 0.f, bias_right = 0.f;
    if (a.table) {
        bias_left = a.bias<T>(a.n_edges, at.h);
        bias_right = a.bias<T>(a.two_sided ? 2 * a.n_edges + 1 : 0, at.h);
    }
    float m = -ATT_INF, l = 0.f;
    floatx16 o[kBlocks];
#pragma unroll
    for (int d = 0; d < kBlocks; ++d) o[d] = zero16();
    if (begin < end) {
        Turn codes;
        codes.set(c, wave, lane);
        hold(0);
        Held h0 = held(0), h1 = held(1), h2 = held(2);   // of this tile and the next ones
        int after = 3;                                   // the one behind them
        // (a query's fragments: operand 2 j + n has columns 16 (2 j + half) + 8 n ..)
        {
            const T* const p = a.q.at<T>(b, at.h) + (int64_t)at.t * a.q.token;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const int d = 32 * (i / 2) + 16 * half + 8 * (i % 2);
                u32x4 one = {0u, 0u, 0u, 0u};
                if (at.mine && d < a.head_dim) one = *reinterpret_cast<const u32x4*>(p + d);
                queries[64 * i] = one;
            }
        }
        if (a.table) places.fill<T>(a, window, bias_lds, hk, from);
        settle();
#pragma unroll
        for (int i = 0; i < Turn::kRequests; ++i) {
            codes.request_keys(c, h0, begin, 0, wave, i);
            codes.request_values(c, h0, begin, 0, wave, i);
            codes.request_keys(c, h1, begin + kTile, Turn::kBytes, wave, i);
        }
        const float k_scale0 = h0.k_scale();
        // (row 8 q + 4 h + j of an operand of keys is key 16 h + 4 q + j of 32)
        const int key_at = 1024 * half + 16 * ((l32 >> 2 & 1) * 16 + (l32 >> 3) * 4 + (l32 & 3)), value_at = Turn::kKeyBytes + 16 * (DP * half + l32);
        auto key = [&](const char* tile, int x) { return *reinterpret_cast<const u32x4*>(tile + key_at + 2048 * (x / 2) + 512 * (x % 2)); };
        auto value = [&](const char* tile, int x) { return *reinterpret_cast<const u32x4*>(tile + value_at + 32 * DP * (x / kBlocks) + 512 * (x % kBlocks)); };   // block x % kBlocks of 32 columns, keys 32 (x / kBlocks) + 16 half ..
        // a weight is exp2(score factor + off), or, where scores are not scaled on the way (scaled is false), of the score less `base`
        float factor = 0.f, off = 0.f, base = 0.f;
        bool scaled = true;
        // tiles up to here have all their tokens, seen by all columns and with the last bucket's bias
        int plain = at.all_see < kl ? at.all_see : kl;
        if (a.table) {
            const int near = kl - ql + at.q_first - a.left + 1;
            plain = near < plain ? near : plain;
            if (__any(!(__builtin_fabsf(bias_left) < kLarge))) plain = 0;
        }
        plain = __builtin_amdgcn_readfirstlane(plain);
        // A tile's scores as the softmax takes them; the running maximum, and what it asks of the weights.
        auto finish = [&](floatx16 (&s)[2], float top, int key0, int there) {
            float bias = bias_left;
            scaled = true;
            if (key0 + kTile > plain || there < kTile) {
                const int r_lo = key0 - (kl - ql + at.q_last), r_hi = key0 + kTile - 1 - (kl - ql + at.q_first);
                const int place = a.table ? place_of(a, r_lo, r_hi) : kLeft;
                bias = place == kRight ? bias_right : bias_left;
                if (place == kNear) {
                    const uint8_t* const n = reinterpret_cast<const uint8_t*>(bias_lds + places.biases) + (key0 - at.p - window.first + 16 * half);
                    const float* const of = reinterpret_cast<const float*>(bias_lds) + at.bias;
                    scaled = false;
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[x][i] = __builtin_fmaf(s[x][i], a.scale, of[n[32 * x + i] * places.heads]);
                } else if (__any(!(__builtin_fabsf(bias) < kLarge))) {   // (lanes have biases of different heads)
                    scaled = false;
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[x][i] = __builtin_fmaf(s[x][i], a.scale, bias);
                }
                if (!scaled || there < kTile || key0 + kTile > at.all_see) {
                    top = -ATT_INF;
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int are = there - 32 * x - 16 * half, to = at.limit - (key0 + 32 * x + 16 * half), left = to < are ? to : are;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            s[x][i] = i < left ? s[x][i] : -ATT_INF;
                            top = __builtin_fmaxf(top, s[x][i]);
                        }
                    }
                }
            }
            top = max_of_halves(top);
            if (scaled) top = __builtin_fmaf(top, a.scale, bias);
            if (__any(top > m + kSlack)) {   // (from minus infinity: any score)
                const float now = __builtin_fmaxf(m, top), f = now == -ATT_INF ? 1.f : exp2_of((m - now) * kLog2e);
                m = now;
                l *= f;
#pragma unroll
                for (int d = 0; d < kBlocks; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] *= f;
            }
            base = m == -ATT_INF ? 0.f : m;   // (no key yet: every weight is exp(-infinity))
            factor = scaled ? a.scale * kLog2e : kLog2e;
            off = scaled ? (bias - base) * kLog2e : 0.f;
        };
        auto there_of = [&](uint32_t exps, int key0) { return exps ? kl - key0 : 0; };
        floatx16 s0[2], s1[2];
        wait_for<0>();
        __syncthreads();
        if (there_of(h0.exps, begin) < kTile) Turn::clear(lds, there_of(h0.exps, begin));   // (the barrier before they are read is the first step's)
        s0[0] = s0[1] = zero16();
#pragma unroll
        for (int x = 0; x < kSteps; ++x) {
            const u32x4 w = key(lds, x);
#pragma unroll
            for (int n = 0; n < 2; ++n) s0[x % 2] = mfma(cache::eight_from<T>(w[2 * n], w[2 * n + 1], k_scale0), queries[64 * (x / 2 * 2 + n)], s0[x % 2], T{});
        }
        {
            float top = s0[0][0];
#pragma unroll
            for (int i = 1; i < 32; ++i) top = __builtin_fmaxf(top, s0[i / 16][i % 16]);
            finish(s0, top, begin, there_of(h0.exps, begin));
        }
        // The next tile's scores among this one's (s) weights, and this one's sums among the search for the next one's largest.
        auto step = [&](floatx16 (&s)[2], floatx16 (&next)[2], int key0, int here) {
            constexpr int kQk = 2 * kSteps, kPv = 4 * kBlocks, kReads = kSteps + 2 * kBlocks, kAhead = 4, kFirst = 8;   // kFirst: pairs of weights among the scores (those of the first 32 keys, at least)
            const int other = here ^ Turn::kBytes;
            const float k_scale = h1.k_scale(), v_scale = h0.v_scale();
            wait_for<0>();
            __syncthreads();   // (the next tile's keys and this one's values are there)
            const int there = there_of(h1.exps, key0 + kTile);
            const bool more = key0 + kTile < end;
            if (there_of(h0.exps, key0) < kTile && key0 > begin) {
                Turn::clear(lds + here, there_of(h0.exps, key0));
                __syncthreads();
            }
            const Held of_values = h1, of_keys = h2;
            if ((after & 63) == 0) hold(after);
            h0 = h1;
            h1 = h2;
            h2 = held(after++);
            const char *const keys = lds + other, *const values = lds + here;
            auto read = [&](int x) { return x < kSteps ? key(keys, x) : value(values, x - kSteps); };
            u32x4 w[4], op[kAhead], q[4];
            float top = -ATT_INF;
            auto weigh = [&](int p) {
                const int i = 2 * p;
                const float e = exp2_of(__builtin_fmaf(s[i / 16][i % 16], factor, off)), f = exp2_of(__builtin_fmaf(s[i / 16][i % 16 + 1], factor, off));
                l += e;
                l += f;
                w[i / 8][i / 2 % 4] = pair_of(e, f, T{});
            };
            if (!scaled)
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[x][i] -= base;
            next[0] = next[1] = zero16();
#pragma unroll
            for (int x = 0; x < kAhead; ++x) op[x] = read(x);
            q[0] = queries[0];
            q[1] = queries[64];
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int x = 0; x < kReads; x += 2) {   // two reads and four products at a time
                const u32x4 v[2] = {op[x % kAhead], op[(x + 1) % kAhead]};
                const int asks = x / 2 - (DP >= 64 ? 1 : 0);
                if (asks >= 0 && asks < Turn::kRequests) codes.request_keys(c, of_keys, key0 + 2 * kTile, here, wave, asks);
                if (asks >= Turn::kRequests && asks < 2 * Turn::kRequests) codes.request_values(c, of_values, key0 + kTile, other, wave, asks - Turn::kRequests);
                if (x + 2 < kSteps) {
                    q[(x + 2) % 4] = queries[64 * (x + 2)];
                    q[(x + 3) % 4] = queries[64 * (x + 3)];
                }
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        if (x < kSteps) {
                            next[y] = mfma(cache::eight_from<T>(v[y][2 * n], v[y][2 * n + 1], k_scale), q[(x + n) % 4], next[y], T{});
                            const int slot = 2 * x + 2 * n + y;
#pragma unroll
                            for (int p = kFirst * slot / kQk; p < kFirst * (slot + 1) / kQk; ++p) weigh(p);
                        } else {
                            const int z = x - kSteps + y, d = z % kBlocks, slot = 2 * (x - kSteps) + 2 * n + y;
                            o[d] = mfma(cache::eight_from<T>(v[y][2 * n], v[y][2 * n + 1], v_scale), w[2 * (z / kBlocks) + n], o[d], T{});
                            if (slot < kPv / 2) {
#pragma unroll
                                for (int p = kFirst + (16 - kFirst) * slot / (kPv / 2); p < kFirst + (16 - kFirst) * (slot + 1) / (kPv / 2); ++p) weigh(p);
                            } else {
                                const int t = slot - kPv / 2;
#pragma unroll
                                for (int i = 32 * t / (kPv / 2); i < 32 * (t + 1) / (kPv / 2); i += 2) top = __builtin_fmaxf(__builtin_fmaxf(top, next[i / 16][i % 16]), next[i / 16][i % 16 + 1]);
                            }
                        }
                        if (n == 1 && x + kAhead < kReads) op[(x + y) % kAhead] = read(x + y + kAhead);
                        __builtin_amdgcn_sched_barrier(0);
                    }
            }
            if (more) finish(next, top, key0 + kTile, there);
        };
        for (int key0 = begin;; key0 += 2 * kTile) {
            step(s0, s1, key0, 0);
            if (key0 + kTile >= end) break;
            step(s1, s0, key0 + kTile, Turn::kBytes);
            if (key0 + 2 * kTile >= end) break;
        }
        wait_for<0>();   // (nothing may arrive in LDS that is no longer this workgroup's)
    }
    if (first + (lane & 31) >= columns) return;
    l = sum_of_halves(l);
    const int64_t row = ((int64_t)b * a.q_heads + at.h) * a.q_tokens + at.t;
    if (parts.count > 1) {
        const int64_t slot = (int64_t)part * a.batch * a.q_heads * a.q_tokens + row;
        store_row32<DP>(parts.sums + slot * DP, o, half);
        if (half == 0) parts.stats[slot] = make_float2(m, at.mine ? l : 0.f);
        return;
    }
    const bool any = at.mine && l != 0.f;   // (a NaN counts as something)
    if (!any)
#pragma unroll
        for (int d = 0; d < Tile<DP>::kBlocks; ++d) o[d] = zero16();
    store_row<T, DP>(out.at<T>(b, at.h) + (int64_t)at.t * out.token, o, any ? 1.f / l : 0.f, a.head_dim, half);
    if (lse && half == 0) lse[row] = at.mine ? lse_of(m, l) : -ATT_INF;
}

// ---- many columns, pages of fewer tokens than a tile: operands in LDS

// 64 keys' codes on their way to a tile that four wavefronts share: a thread takes sixteen columns of a key, or tokens of a column, at a time, and parks them as operands' type: keys in rows of DP
// columns, row 8 q + 4 h + j of a block of 32 being key 16 h + 4 q + j, so that a lane's sixteen scores are of sixteen neighbouring keys; values in rows of 64 tokens.  Rows past the sequence's end, or
// whose page is not there, hold anything; of values they are cleared, and their page's byte is left out (their weight is 0, but anything may be a NaN).
template <typename T, int DP> struct Shared {
    static constexpr int kEach = kTile * DP / 16 / 256, kKeyBytes = kTile * Tile<DP>::kRowBytes, kValueBytes = DP * Tile<kTile>::kRowBytes, kBytes = kKeyBytes + kValueBytes;
    static_assert(kTile == 64 && DP <= 128, "a wavefront's lanes are the keys of a tile; a thread's second chunk is four units of keys, two of values further");
    static constexpr int kLoads = kEach > 0 ? kEach : 1;   // (32 columns: half of the threads have a chunk)
    u32x4 k[kLoads], v[kLoads];
    int k_byte, v_byte[kLoads], k_page, v_page[kLoads];   // (as in Few)
    int there[kLoads];               // tokens of a chunk of values
    int unit, group, d, k_at, v_at;  // this thread's first chunks: unit of columns of a key, of tokens of column d; where they are parked
    uint32_t v_from;                 // where column d lies behind a unit's first
    __device__ __forceinline__ void set(const cache::Cache& c)
    {
        const int key = (int)threadIdx.x & 63, row = (key & 32) | (key & 12) << 1 | (key >> 4 & 1) << 2 | (key & 3);
        unit = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        group = (int)threadIdx.x / DP;
        d = (int)threadIdx.x % DP;
        k_at = Tile<DP>::at(row, 2 * unit & (Tile<DP>::kChunks - 1));
        v_at = kKeyBytes + Tile<kTile>::at(d, 2 * group & 7);
        v_from = 16u * (uint32_t)(d < c.head_dim ? d : c.head_dim - 1);   // (columns past the last are not stored)
    }
    __device__ __forceinline__ bool has_keys(int i) const { return kEach > 0 || unit + 4 * i < DP / 16; }
    __device__ __forceinline__ bool has_values() const { return kEach > 0 || group < 4; }
    __device__ __forceinline__ void find(const cache::Cache& c, int b, int key0, int most)   // most: the sequences' room
    {
        const int at = key0 + ((int)threadIdx.x & 63);
        k_page = at < most ? c.number_of(b, at) : -1;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int first = key0 + 16 * (group + 2 * i);
            v_page[i] = has_values() && first < most ? c.number_of(b, first) : -1;
        }
    }
    __device__ __forceinline__ void load(const cache::Cache& c, int h, int key0, int kl)
    {
        const int in = c.page_tokens() - 1, units = c.head_dim / cache::kUnit;
        const int64_t head = c.head_of(c.is_page(k_page) ? k_page : 0, h);
        const uint8_t* const p = c.k + head * c.page_bytes() + 16 * ((key0 + ((int)threadIdx.x & 63)) & in);
        k_byte = c.k_exps[head];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            k[i] = u32x4{0u, 0u, 0u, 0u};   // (columns past the last: a query's are 0 there)
            if (unit + 4 * i < units) k[i] = *reinterpret_cast<const u32x4*>(p + ((uint32_t)(unit + 4 * i) << (c.shift + 4)));
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int first = key0 + 16 * (group + 2 * i);
            there[i] = c.is_page(v_page[i]) ? kl - first : 0;
            const int64_t of = c.head_of(c.is_page(v_page[i]) ? v_page[i] : 0, h);
            v_byte[i] = c.v_exps[of];
            v[i] = *reinterpret_cast<const u32x4*>(c.v + of * c.page_bytes() + (first & in) * c.head_dim + v_from);
        }
    }
    __device__ __forceinline__ void park(char* tile, int* there_of)
    {
        const float k_scale = cache::two_to(k_byte);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const float v_scale = cache::two_to(v_byte[i], there[i]);
            if (has_keys(i))
#pragma unroll
                for (int u = 0; u < 2; ++u) *reinterpret_cast<u32x4*>(tile + (k_at ^ (128 * i + 16 * u))) = cache::eight_from<T>(k[i][2 * u], k[i][2 * u + 1], k_scale);
            if (has_values()) {
                if (there[i] < 16) {
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const int bytes = there[i] - 4 * w;
                        v[i][w] &= bytes >= 4 ? ~0u : bytes <= 0 ? 0u : (1u << (8 * bytes)) - 1u;
                    }
                }
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    *reinterpret_cast<u32x4*>(tile + (v_at ^ (64 * i + 16 * u))) = cache::eight_from<T>(v[i][2 * u], v[i][2 * u + 1], v_scale);
                if (d == 0) there_of[group + 2 * i] = there[i];
            }
        }
    }
};

template <typename T, int DP> __global__ void __launch_bounds__(256, 2) chunk_kernel(Args a, cache::Cache c, Heads out, float* __restrict__ lse, Parts parts, int tiles)
{
    using Turn = Shared<T, DP>;
    constexpr int kSteps = DP / 16, kBlocks = DP / 32;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int(*const there_of)[4] = reinterpret_cast<int(*)[4]>(lds + 2 * Turn::kBytes);   // by turn, of sixteen tokens
    char* const bias_lds = lds + 2 * Turn::kBytes + 32;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), half = lane >> 5;
    const int columns = a.q_tokens * a.group;
    const Item it = item_of(blockIdx.x, (uint32_t)a.batch * a.kv_heads, 1, (uint32_t)tiles * parts.count);
    const int b = it.head / a.kv_heads, hk = it.head % a.kv_heads, part = it.tile % parts.count, from = it.tile / parts.count * 128, first = from + 32 * wave;
    const int begin = part * parts.keys;
    Turn codes;
    codes.set(c);
    codes.find(c, b, begin, a.k_tokens);
    const int ql = a.queries(b), kl = a.keys(b);
    Columns at;
    at.set(a, hk, from, first < columns ? first : columns - 1, columns, ql, kl, lane);
    if (first >= columns) at.mine = false;
    const Window window(a.left, a.right);
    const BiasLds places(a);
    // the keys that this wavefront's and this workgroup's queries see, and of them this part's
    auto seen_by = [&](int last_column) {
        int q = last_column / a.group;
        q = q < ql ? q : ql - 1;
        const int n = a.causal ? kl - ql + q + 1 : kl;
        return n < kl ? n : kl;
    };
    const int last = from + 127 < columns ? from + 127 : columns - 1;
    int end = from / a.group >= ql ? 0 : seen_by(last), seen = first >= columns || at.q_first >= ql ? 0 : seen_by(first + 31 < columns ? first + 31 : columns - 1);
    if (parts.count > 1) end = end < begin + parts.keys ? end : begin + parts.keys;

    float bias_left = 0.f, bias_right = 0.f;
    if (a.table) {
        bias_left = a.bias<T>(a.n_edges, at.h);
        bias_right = a.bias<T>(a.two_sided ? 2 * a.n_edges + 1 : 0, at.h);
    }
    Running<T, DP> run;
    run.clear();
    if (begin < end) {
        codes.load(c, hk, begin, kl);
        codes.find(c, b, begin + kTile, a.k_tokens);
        u32x4 qf[kSteps];
        load_row<T, DP>(qf, a.q.at<T>(b, at.h) + (int64_t)at.t * a.q.token, at.mine, a.head_dim, half);
        if (a.table) places.fill<T>(a, window, bias_lds, hk, from);
        const int l32 = lane & 31, row_at = Tile<DP>::at(l32, half), value_at = Tile<kTile>::at(l32, 2 * half);
        int turn = 0;
        codes.park(lds, there_of[0]);
        if (begin + kTile < end) {
            codes.load(c, hk, begin + kTile, kl);
            codes.find(c, b, begin + 2 * kTile, a.k_tokens);
        }
        for (int key0 = begin; key0 < end; key0 += kTile) {
            __syncthreads();   // (what was parked is there, and the tile before is done with)
            char* const tile = lds + turn * Turn::kBytes;
            auto next = [&] {
                if (key0 + kTile < end) {
                    codes.park(lds + (turn ^ 1) * Turn::kBytes, there_of[turn ^ 1]);
                    if (key0 + 2 * kTile < end) {
                        codes.load(c, hk, key0 + 2 * kTile, kl);
                        codes.find(c, b, key0 + 3 * kTile, a.k_tokens);
                    }
                }
            };
            if (key0 >= seen) next();
            if (key0 < seen) {
                floatx16 s[2] = {zero16(), zero16()};
                auto key = [&](int x) { return *reinterpret_cast<const u32x4*>(tile + (row_at ^ ((x / 2) << 5)) + (x % 2) * 32 * Tile<DP>::kRowBytes); };
                Operands<2 * kSteps, 4> keys;
                keys.start(key);
                keys.products(key, [&](int x, u32x4 w) { s[x % 2] = mfma(w, qf[x / 2], s[x % 2], T{}); });
                // (product x: depth step x / kBlocks of 16 keys in the scores' order, block x % kBlocks of 32 columns)
                auto value = [&](int x) {
                    const int step = x / kBlocks, d = x % kBlocks;
                    return *reinterpret_cast<const u32x4*>(tile + Turn::kKeyBytes + (value_at ^ ((4 * (step / 2) + step % 2) << 4)) + d * 32 * Tile<kTile>::kRowBytes);
                };
                Operands<4 * kBlocks, 4> values;
                next();
                values.start(value);
                const int there[2] = {there_of[turn][half], there_of[turn][2 + half]};
                const bool short_of = __any(there[0] < 16 || there[1] < 16);
                const int r_lo = key0 - (kl - ql + at.q_last), r_hi = key0 + kTile - 1 - (kl - ql + at.q_first);
                const int place = a.table ? place_of(a, r_lo, r_hi) : kLeft;
                const float bias = place == kRight ? bias_right : bias_left;
                bool fused = true;
                if (place == kNear) {
                    const uint8_t* const n = reinterpret_cast<const uint8_t*>(bias_lds + places.biases) + (key0 - at.p - window.first + 16 * half);
                    const float* const of = reinterpret_cast<const float*>(bias_lds) + at.bias;
                    fused = false;
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[x][i] = __builtin_fmaf(s[x][i], a.scale, of[n[32 * x + i] * places.heads]);
                } else if (__any(!(__builtin_fabsf(bias) < kLarge))) {   // (lanes have biases of different heads)
                    fused = false;
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[x][i] = __builtin_fmaf(s[x][i], a.scale, bias);
                }
                if (short_of || key0 + kTile > at.all_see)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int to = at.limit - (key0 + 32 * x + 16 * half), left = to < there[x] ? to : there[x];
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[x][i] = i < left ? s[x][i] : -ATT_INF;
                    }
                run.weigh(s, fused, a.scale, bias);
                u32x4 weights{};
                values.products(value, [&](int x, u32x4 w) {
                    const int step = x / kBlocks, d = x % kBlocks;
                    if (d == 0) weights = weights_of<T>(s[step / 2], step % 2);
                    run.o[d] = mfma(w, weights, run.o[d], T{});
                });
            }
            turn ^= 1;
        }
    }
    if (first + (lane & 31) >= columns) return;
    const float l = sum_of_halves(run.l);
    const int64_t row = ((int64_t)b * a.q_heads + at.h) * a.q_tokens + at.t;
    if (parts.count > 1) {
        const int64_t slot = (int64_t)part * a.batch * a.q_heads * a.q_tokens + row;
        store_row32<DP>(parts.sums + slot * DP, run.o, half);
        if (half == 0) parts.stats[slot] = make_float2(run.m, at.mine ? l : 0.f);
        return;
    }
    const bool any = at.mine && l != 0.f;   // (a NaN counts as something)
    if (!any)
#pragma unroll
        for (int d = 0; d < Tile<DP>::kBlocks; ++d) run.o[d] = zero16();
    store_row<T, DP>(out.at<T>(b, at.h) + (int64_t)at.t * out.token, run.o, any ? 1.f / l : 0.f, a.head_dim, half);
    if (lse && half == 0) lse[row] = at.mine ? lse_of(run.m, l) : -ATT_INF;
}

// ---- the parts of a key axis that was cut

// A row's DP columns, four to a thread, by `groups` threads that take every so many parts and meet in LDS: few rows of many parts would leave one thread to go through all of them in turn (8 rows of
// 118 parts: 54 us a call where this takes 18).
template <typename T, int DP> __global__ void __launch_bounds__(256) join_groups_kernel(Args a, Heads out, float* __restrict__ lse, Parts parts, int groups)
{
    constexpr int kFours = DP / 4;
    __shared__ __attribute__((aligned(16))) f32x4 sums[256];
    __shared__ float2 stats[256];
    const int64_t rows = (int64_t)a.batch * a.q_heads * a.q_tokens;
    const int four = threadIdx.x % kFours, group = threadIdx.x / kFours % groups, each = 256 / kFours / groups;
    const int64_t row = (int64_t)blockIdx.x * each + threadIdx.x / kFours / groups;
    float m = -ATT_INF, total = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    if (row < rows && 4 * four < a.head_dim)
#pragma unroll 4
        for (int n = group; n < parts.count; n += groups) {
            const float2 st = parts.stats[n * rows + row];
            const f32x4 x = *reinterpret_cast<const f32x4*>(parts.sums + (n * rows + row) * DP + 4 * four);
            const bool any = st.y != 0.f;   // (a part that no key reached counts for nothing, whatever it left)
            const float now = any ? __builtin_fmaxf(m, st.x) : m, keep = m == -ATT_INF ? 0.f : exp2_of((m - now) * kLog2e), f = any ? exp2_of((st.x - now) * kLog2e) : 0.f;
            m = now;
            total = __builtin_fmaf(f, any ? st.y : 0.f, total * keep);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(f, any ? x[e] : 0.f, o[e] * keep);
        }
    sums[threadIdx.x] = o;
    stats[threadIdx.x] = make_float2(m, total);
    __syncthreads();
    if (group != 0 || row >= rows) return;
    for (int n = 1; n < groups; ++n) {
        const float2 st = stats[threadIdx.x + n * kFours];
        const f32x4 x = sums[threadIdx.x + n * kFours];
        if (st.y == 0.f) continue;
        const float now = __builtin_fmaxf(m, st.x), keep = m == -ATT_INF ? 0.f : exp2_of((m - now) * kLog2e), f = exp2_of((st.x - now) * kLog2e);
        m = now;
        total = __builtin_fmaf(f, st.y, total * keep);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(f, x[e], o[e] * keep);
    }
    const float f = total != 0.f ? 1.f / total : 0.f;
    const int i = (int)(row % a.q_tokens), bh = (int)(row / a.q_tokens), b = bh / a.q_heads, h = bh % a.q_heads, d = 4 * four;
    if (d < a.head_dim) *reinterpret_cast<u32x2*>(out.at<T>(b, h) + (int64_t)i * out.token + d) = u32x2{pair_of(o[0] * f, o[1] * f, T{}), pair_of(o[2] * f, o[3] * f, T{})};
    if (lse && d == 0) lse[row] = lse_of(m, total);
}

// Which kernel, and into how many parts the keys are cut.
struct Plan {
    bool tokens;
    int tiles, parts, part_keys;
    int64_t rows;
    size_t workspace;
};
constexpr int64_t kEnough = 4096;   // workgroups that fill the device where all they do is read, and their sequences' lengths differ (1024, 2048, 4096 and 8192, us a call: 32 caches of up to 32768,
                                    // 8 heads of 128, 247, 212, 200, 236; of 32768 each 325, 328, 341, -)
Plan plan_of(const pruner_attention* a)
{
    Plan p{};
    const int group = a->q_heads / a->kv_heads;
    const int64_t columns = (int64_t)a->q_tokens * group;
    p.rows = (int64_t)a->batch * a->q_heads * a->q_tokens;
    p.tokens = columns <= 32;
    p.tiles = (int)((columns + 127) / 128);
    const int64_t groups = (int64_t)a->batch * a->kv_heads * (p.tokens ? 1 : p.tiles);
    int64_t parts = 1;
    if (groups > 0) {
        if (p.tokens) {
            // keys of a part at least, where there are more than twice as many (256, 512, 1024 and 2048, us of the kernel: 64 caches of up to 4000, 4 heads of 128, -, 37, 37, 35, 8 of up to 20000,
            // 8 heads, -, 44, 40, 49, 16 of up to 5003, 4 heads of 80, 22, 21, 24, 29; 16 of 1000, 8 heads, in one part 15.5, in two 13.3 and 3.9 to join)
            const int fewest = 512;
            parts = (kEnough + groups - 1) / groups;
            const int64_t most = a->k_tokens <= 2 * fewest ? 1 : ((int64_t)a->k_tokens + fewest - 1) / fewest;
            parts = parts < most ? parts : most;
        } else {
            parts = parts_of((double)groups, (a->k_tokens + kTile - 1) / kTile, false, 512, 1.5, 2.2, (double)p.rows * padded_dim(a->head_dim) * 4);
        }
    }
    if (parts < 1) parts = 1;
    const int64_t keys = ((a->k_tokens + parts - 1) / parts + kTile - 1) / kTile * kTile;
    p.part_keys = (int)(keys > 0 ? keys : kTile);
    p.parts = (int)((a->k_tokens + (int64_t)p.part_keys - 1) / p.part_keys);
    if (p.parts < 1) p.parts = 1;
    p.workspace = p.parts > 1 ? round_up((size_t)p.parts * p.rows * 8, 256) + round_up((size_t)p.parts * p.rows * padded_dim(a->head_dim) * 4, 256) : 0;
    return p;
}

template <typename T, int DP, int CT> int run_tokens(const Args& args, const cache::Cache& c, const Plan& plan, const Parts& parts, const Heads& out, float* lse, hipStream_t st)
{
    static PerDeviceFlag ready;
    const int dev = current_device(nullptr);
    if (dev < 0) return PRUNER_EHIP;
    if (!ready.get(dev)) {
        for (const void* fn : {reinterpret_cast<const void*>(&tokens_kernel<T, DP, CT, false, false>), reinterpret_cast<const void*>(&tokens_kernel<T, DP, CT, true, false>),
                               reinterpret_cast<const void*>(&tokens_kernel<T, DP, CT, true, true>)})
            if (hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) != hipSuccess) return PRUNER_EHIP;
        ready.mark(dev);
    }
    const size_t biases = (size_t)BiasLds(args).bytes(), last = Meeting<DP>::bytes(args.q_tokens * args.group);
    const bool once = 2 * (int64_t)args.batch * args.kv_heads * args.k_tokens * args.head_dim > cache::kCached;
    void (*const kernel)(Args, cache::Cache, Heads, float*, Parts) = c.page_tokens() < kTile ? tokens_kernel<T, DP, CT, false, false> : once ? tokens_kernel<T, DP, CT, true, true> : tokens_kernel<T, DP, CT, true, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((int64_t)args.batch * args.kv_heads * plan.parts)), dim3(256), last > biases ? last : biases, st, args, c, out, lse, parts);
    PRUNER_LAUNCH_CHECK();
    return PRUNER_OK;
}
template <typename T, int DP> int run_chunk(const Args& args, const cache::Cache& c, const Plan& plan, const Parts& parts, const Heads& out, float* lse, hipStream_t st)
{
    static PerDeviceFlag ready;
    const int dev = current_device(nullptr);
    if (dev < 0) return PRUNER_EHIP;
    if (!ready.get(dev)) {
        for (const void* fn : {reinterpret_cast<const void*>(&codes_kernel<T, DP>), reinterpret_cast<const void*>(&chunk_kernel<T, DP>)})
            if (hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) != hipSuccess) return PRUNER_EHIP;
        ready.mark(dev);
    }
    const bool whole = c.page_tokens() >= kTile;
    void (*const kernel)(Args, cache::Cache, Heads, float*, Parts, int) = whole ? codes_kernel<T, DP> : chunk_kernel<T, DP>;
    const size_t lds = (whole ? 2 * (size_t)Codes<DP>::kBytes + 256 * DP : 2 * (size_t)Shared<T, DP>::kBytes + 32) + BiasLds(args).bytes();
    hipLaunchKernelGGL(kernel, dim3((unsigned)((int64_t)args.batch * args.kv_heads * plan.tiles * plan.parts)), dim3(256), lds, st, args, c, out, lse, parts, plan.tiles);
    PRUNER_LAUNCH_CHECK();
    return PRUNER_OK;
}
template <typename T, int DP> int run(const Args& args, const cache::Cache& c, const Plan& plan, const Heads& out, float* lse, void* workspace, hipStream_t st)
{
    Parts parts{nullptr, nullptr, plan.parts, plan.part_keys};
    if (plan.parts > 1) {
        parts.stats = static_cast<float2*>(workspace);
        parts.sums = reinterpret_cast<float*>(static_cast<char*>(workspace) + round_up((size_t)plan.parts * plan.rows * 8, 256));
    }
    if (plan.tokens) {
        const int rc = args.q_tokens * args.group <= 16 ? run_tokens<T, DP, 1>(args, c, plan, parts, out, lse, st) : run_tokens<T, DP, 2>(args, c, plan, parts, out, lse, st);
        if (rc) return rc;
    } else {
        const int rc = run_chunk<T, DP>(args, c, plan, parts, out, lse, st);
        if (rc) return rc;
    }
    if (plan.parts > 1) {
        int groups = 1;
        while (groups < plan.parts && groups < 256 / (DP / 4)) groups *= 2;
        const int64_t each = 256 / (DP / 4) / groups;
        hipLaunchKernelGGL((join_groups_kernel<T, DP>), dim3((unsigned)((plan.rows + each - 1) / each)), dim3(256), 0, st, args, out, lse, parts, groups);
        PRUNER_LAUNCH_CHECK();
    }
    return PRUNER_OK;
}

// What this call refuses about sizes beyond what attention over 16-bit keys does.
bool sizes_ok(const pruner_attention* a) { return attention_sizes_ok(a) && a->head_dim % cache::kUnit == 0; }

}  // namespace
}  // namespace att
}  // namespace pruner

using namespace pruner;

extern "C" size_t pruner_cache_attention_workspace_bytes(const pruner_attention* a) { return att::sizes_ok(a) ? att::plan_of(a).workspace : 0; }

extern "C" int pruner_cache_attention(const pruner_attention* a, const pruner_cache* kept, const pruner_heads* q, const pruner_heads* o, float* lse, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!att::sizes_ok(a) || !cache::cache_ok(kept)) return PRUNER_EINVAL;
    if (kept->kv_heads != a->kv_heads || kept->head_dim != a->head_dim || a->k_tokens > (int64_t)kept->seq_pages * kept->page_tokens) return PRUNER_EINVAL;
    if (!kept->table && a->k_tokens > 0 && (int64_t)a->batch * kept->seq_pages > kept->pages) return PRUNER_EINVAL;
    if (a->batch == 0 || a->q_tokens == 0) return PRUNER_OK;
    pruner_attention sizes = *a;
    if (kept->pages == 0) sizes.k_tokens = 0;   // (no page is there)
    att::Args args;
    const pruner_heads nothing{kept->k_codes ? kept->k_codes : reinterpret_cast<uint8_t*>(16), 0, 0, 0};
    const int rc = att::attention_args(&sizes, q, &nothing, &nothing, &args);
    if (rc) return rc;
    if (!att::heads_ok(o) || (lse && !aligned(lse, 4))) return PRUNER_EINVAL;
    const att::Plan plan = att::plan_of(a);
    if (plan.parts > 1 && (!workspace || !aligned(workspace, 256) || workspace_bytes < plan.workspace)) return PRUNER_EWORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const cache::Cache c = cache::cache_of(kept);
    const att::Heads out = att::heads_of(o);
    const int dp = att::padded_dim(a->head_dim);
    if (a->dtype == PRUNER_BF16)
        return dp == 32   ? att::run<__bf16, 32>(args, c, plan, out, lse, workspace, st)
               : dp == 64 ? att::run<__bf16, 64>(args, c, plan, out, lse, workspace, st)
                          : att::run<__bf16, 128>(args, c, plan, out, lse, workspace, st);
    return dp == 32   ? att::run<_Float16, 32>(args, c, plan, out, lse, workspace, st)
           : dp == 64 ? att::run<_Float16, 64>(args, c, plan, out, lse, workspace, st)
                      : att::run<_Float16, 128>(args, c, plan, out, lse, workspace, st);
}
