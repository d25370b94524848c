// Attention with a learned relative position bias by buckets, forward: o = softmax(scale q k^T + bias) v and lse, one pass over the keys
// with the running maximum and sum of the softmax.
//
//   tile_kernel   a wavefront owns 32 queries, one per lane of a half: S^T = K Q^T leaves a query's scores in its two lanes, so the softmax is a
//                 lane's own work but for one exchange, and the weights are the next product's operand as they stand (O^T += V^T P^T).  Four
//                 wavefronts share the key and value tiles (64 keys, two turns in LDS), or, for sequences of at most 32 queries and 64 keys, each has
//                 a sequence and head of its own.  The bias is a function of j - p: tiles beyond the largest edge add one number, the others read a
//                 window of it in LDS.
//   rows_kernel   few queries: the queries of all heads that share a key head, at most 32 together, are the 32 columns; the four wavefronts take
//                 32 keys each in turn, through LDS of their own (keys straight from memory into operand registers, 32 bytes of a row at a time:
//                 476 us where this takes 400), and meet at the end.  Neighbouring workgroups take the heads of one sequence, whose
//                 rows lie side by side (parts of one head instead: 584 us).
//   join_kernel   the parts of a key axis that was split over workgroups.
//
// tile_kernel is bound by the matrix cores and the exponentials between their products, under a clock that falls with the load: 8192 causal tokens, 16 heads
// of 128 sharing 4, 262 to 283 us, 970 to 1050 TFLOP/s at 1.6 GHz, products alone 194 us, without exponentials 257, without reads of LDS 258 (a large matrix product:
// 1445 TFLOP/s).  A tile's exponentials go before the other wavefront's products (310 us without that).  (The next tile's scores among this tile's exponentials, in one wavefront: 273 us where this takes 269, and
// 16 sequences of up to 777 tokens, 12 heads of 64, 41 us where this takes 34.)  Short sequences are bound by a workgroup's start (4 us of its 18) and chain of tiles.
// The weights are rounded to the operands' type for the second product, which is the rate of the matrix cores' 16-bit forms; their sum is of the unrounded ones.  8192 causal tokens in
// bfloat16: o is off by 2.0e-3 of itself, where its own rounding makes 1.5e-3; 16 sequences of up to 777 in binary16 2.8e-4 and 2.1e-4.
// rows_kernel is bound by memory: one token against 32 caches of up to 32768, 8 heads of 128, 400 us and 12 to join, 5.2 TB/s.
#include "attention_softmax.h"

namespace pruner {
namespace att {
namespace {

constexpr int kKeys = 64;          // keys of a shared tile
constexpr int kOwnKeys = 32;       // keys of a wavefront's own tile

// Keys at or beyond `limit` leave the softmax.
template <int N> __device__ __forceinline__ void mask_scores(floatx16 (&s)[N], int key0, int limit, int half)
{
    const int left = limit - key0 - 4 * half;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[n][i] = 32 * n + row_of(i, 0) < left ? s[n][i] : -ATT_INF;
}

// Scores with their bias and mask for one query (position p) against keys key0 + 32 n + row.  bias_end: the bias of tiles at either end.
// Returns whether scaling is left to the softmax, and the shift that goes with it.
template <int N>
__device__ __forceinline__ bool finish_scores(floatx16 (&s)[N], const Args& a, const float* window, int first, int place, float bias, int key0, int p, int limit, bool masked, int half)
{
    bool fused = true;
    if (place == kNear) {
        const float* const w = window + (key0 - p - first + 4 * half);
        fused = false;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[n][i] = __builtin_fmaf(s[n][i], a.scale, w[32 * n + 8 * (i >> 2) + (i & 3)]);
    } else if (!(__builtin_fabsf(bias) < kLarge)) {
        fused = false;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[n][i] = __builtin_fmaf(s[n][i], a.scale, bias);
    }
    if (masked) mask_scores(s, key0, limit, half);
    return fused;
}

template <typename T, int DP, bool SHARED>
__global__ void __launch_bounds__(256, (DP == 128 ? 2 : 3)) tile_kernel(Args a, Heads out, float* __restrict__ lse, Parts parts, int q_tiles)
{
    constexpr int kN = SHARED ? kKeys : kOwnKeys, kThreads = SHARED ? 256 : 64, kTileBytes = kN * Tile<DP>::kRowBytes, kTurns = turns_of(DP, SHARED, kN);
    static_assert((SHARED ? kTurns : 4) * 2 * kTileBytes <= kRequestRoom, "tiles lie where requests reach");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), half = lane >> 5, l32 = lane & 31, thread = SHARED ? (int)threadIdx.x : lane;
    const uint32_t heads = (uint32_t)a.batch * a.q_heads;
    int part = 0, bh, q0;
    if constexpr (SHARED) {
        const Item it = item_of(blockIdx.x, (uint32_t)a.batch * a.kv_heads, a.group, (uint32_t)q_tiles * parts.count);
        bh = it.head;
        part = it.tile % parts.count;
        q0 = it.tile / parts.count * 128 + 32 * wave;
    } else {
        bh = (int)(blockIdx.x * 4 + wave);
        q0 = 0;
        if (bh >= (int)heads) return;   // (wavefronts have nothing in common)
    }
    const int b = bh / a.q_heads, h = bh % a.q_heads, hk = h / a.group;
    const Window window(a.left, a.right);
    WindowFill<T, kThreads> fill;
    float bias_left = 0.f, bias_right = 0.f;
    if (a.table) {
        fill.load(a, window, h, thread);
        bias_left = a.bias<T>(a.n_edges, h);
        bias_right = a.bias<T>(a.two_sided ? 2 * a.n_edges + 1 : 0, h);
    }
    const int ql = a.queries(b), kl = a.keys(b);
    const int window_bytes = a.table ? (window.size * 4 + 15) & ~15 : 0;
    char* const tiles = lds + (SHARED ? 0 : wave * 2 * kTileBytes);
    float* const biases = reinterpret_cast<float*>(lds + (SHARED ? kTurns : 4) * 2 * kTileBytes + (SHARED ? 0 : wave * window_bytes));

    // the keys that this workgroup's queries see, and of them this part's
    const int first_q = SHARED ? q0 - 32 * wave : 0, rows_here = SHARED ? 128 : 32;
    const int last_q = first_q + rows_here < ql ? first_q + rows_here - 1 : ql - 1;
    int end = first_q >= ql ? 0 : a.causal ? kl - ql + last_q + 1 : kl;
    end = end < kl ? end : kl;
    const int begin = part * parts.keys;
    if (parts.count > 1) end = end < begin + parts.keys ? end : begin + parts.keys;

    const T* const kp = a.k.at<T>(b, hk);
    const T* const vp = a.v.at<T>(b, hk);
    Flow<T, DP, kN, kThreads> kf, vf;
    kf.set(a.k.token, a.head_dim, thread, SHARED ? wave : 0);
    vf.set(a.v.token, a.head_dim, thread, SHARED ? wave : 0);
    auto request = [&](int key0, int turn) {
        const uint32_t to = (uint32_t)((SHARED ? turn : wave) * 2 * kTileBytes);
        const int left = key0 < end ? kl - key0 : 0;
        kf.request(kp + (int64_t)key0 * a.k.token, left, to);
        vf.request(vp + (int64_t)key0 * a.v.token, left, to + kTileBytes);
    };
    constexpr int kAheadK = 4, kAheadV = 4;
    constexpr int kAhead = SHARED ? kTurns - 1 : 1;   // tiles on their way before the first is worked on
    if (begin < end)
#pragma unroll
        for (int t = 0; t < kAhead; ++t) request(begin + t * kN, t);
    Lane<DP> at;
    at.set(lane);
    const int i = q0 + l32, p = kl - ql + i;
    u32x4 qf[Tile<DP>::kSteps];
    load_row<T, DP>(qf, a.q.at<T>(b, h) + (int64_t)i * a.q.token, i < ql, a.head_dim, half);
    Running<T, DP> run;
    run.clear();
    if (begin < end) {
        if (a.table) fill.store(a, window, biases, h, thread);
        // of this wavefront's queries
        const int wave_last = q0 + 31 < ql ? q0 + 31 : ql - 1;
        const int seen = q0 >= ql ? 0 : a.causal ? (kl - ql + wave_last + 1 < kl ? kl - ql + wave_last + 1 : kl) : kl;
        const int limit = a.causal ? (p + 1 < kl ? p + 1 : kl) : kl, all_see = a.causal ? (kl - ql + q0 + 1 < kl ? kl - ql + q0 + 1 : kl) : kl;
        settle();
        int turn = 0;
        for (int key0 = begin; key0 < end; key0 += kN) {
            if constexpr (SHARED) {
                wait_for<(kTurns - 2) * 2 * Flow<T, DP, kN, kThreads>::kEach>();
                __syncthreads();   // (and the tile before is done with)
                request(key0 + (kTurns - 1) * kN, turn == 0 ? kTurns - 1 : turn - 1);
            } else {
                wait_for<0>();
                wave_fence();
            }
            const char* const kt = tiles + (SHARED ? turn * 2 * kTileBytes : 0);
            if (key0 < seen) {
                floatx16 s[kN / 32];
#pragma unroll
                for (int n = 0; n < kN / 32; ++n) s[n] = zero16();
                auto key = [&](int x) { return at.rows(kt, x % (kN / 32), x / (kN / 32)); };
                Operands<kN / 32 * Tile<DP>::kSteps, kAheadK> keys;
                __builtin_amdgcn_s_setprio(0);
                keys.start(key);
                keys.products(key, [&](int x, u32x4 w) { s[x % (kN / 32)] = mfma(w, qf[x / (kN / 32)], s[x % (kN / 32)], T{}); });
                auto value = [&](int x) { return at.columns(kt + kTileBytes, x % Tile<DP>::kBlocks, x / Tile<DP>::kBlocks); };
                Operands<kN / 16 * Tile<DP>::kBlocks, kAheadV> values;
                values.start(value);
                __builtin_amdgcn_s_setprio(1);
                const int r_lo = key0 - (kl - ql + q0 + 31), r_hi = key0 + kN - 1 - (kl - ql + q0);
                const int place = a.table ? place_of(a, r_lo, r_hi) : kLeft;
                const float bias = place == kRight ? bias_right : bias_left;
                const bool fused = finish_scores(s, a, biases, window.first, place, bias, key0, p, limit, key0 + kN > all_see, half);
                run.weigh(s, fused, a.scale, bias);
                __builtin_amdgcn_s_setprio(0);
                u32x4 weights{};
                values.products(value, [&](int x, u32x4 w) {
                    const int step = x / Tile<DP>::kBlocks, d = x % Tile<DP>::kBlocks;
                    if (d == 0) weights = weights_of<T>(s[step / 2], step % 2);
                    run.o[d] = mfma(w, weights, run.o[d], T{});
                });
            }
            if constexpr (SHARED) {
                turn = turn == kTurns - 1 ? 0 : turn + 1;
            } else {
                wait_for_reads();
                wave_fence();
                if (key0 + kN < end) request(key0 + kN, 0);
            }
        }
        wait_for<0>();   // (nothing may arrive in LDS that is no longer this workgroup's)
    }
    if (i >= a.q_tokens) return;
    const float l = sum_of_halves(run.l);
    const int64_t row = (int64_t)bh * a.q_tokens + i;
    if (parts.count > 1) {
        const int64_t slot = (int64_t)part * heads * a.q_tokens + row;
        store_row32<DP>(parts.sums + slot * DP, run.o, half);
        if (half == 0) parts.stats[slot] = make_float2(run.m, i < ql ? l : 0.f);
        return;
    }
    const bool any = i < ql && l != 0.f;   // (a NaN counts as something)
    if (!any)   // (a row that no key reaches may hold anything)
#pragma unroll
        for (int d = 0; d < Tile<DP>::kBlocks; ++d) run.o[d] = zero16();
    store_row<T, DP>(out.at<T>(b, h) + (int64_t)i * out.token, run.o, any ? 1.f / l : 0.f, a.head_dim, half);
    if (lse && half == 0) lse[row] = i < ql ? lse_of(run.m, l) : -ATT_INF;
}

// LDS of rows_kernel before the tiles: the biases of the group's heads, and the bucket of every r that a tile which is not wholly at one end can ask for.
struct RowsLds {
    int n_buckets, biases, buckets;   // bytes
    __host__ __device__ explicit RowsLds(const Args& a)
        : n_buckets(a.table ? (a.n_edges + 1) * (a.two_sided ? 2 : 1) : 0), biases((n_buckets * a.group * 4 + 15) & ~15),
          buckets(a.table ? (Window(a.left, a.right).size + 15) & ~15 : 0)
    {
    }
};

// Query t of head hk * group + g is column t * group + g.
template <typename T, int DP> __global__ void __launch_bounds__(256, 2) rows_kernel(Args a, Heads out, float* __restrict__ lse, Parts parts)
{
    constexpr int kTileBytes = kOwnKeys * Tile<DP>::kRowBytes;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), half = lane >> 5, l32 = lane & 31;
    const int columns = a.q_tokens * a.group;
    const int hk = blockIdx.x % a.kv_heads, part = blockIdx.x / a.kv_heads % parts.count, b = blockIdx.x / a.kv_heads / parts.count;
    const int ql = a.queries(b), kl = a.keys(b);
    const int t = l32 / a.group, g = l32 % a.group, h = hk * a.group + (l32 < columns ? g : 0);
    const bool mine = l32 < columns && t < ql;
    const int p = kl - ql + (l32 < columns ? t : 0);
    const Window window(a.left, a.right);
    float* const biases = reinterpret_cast<float*>(lds);   // [bucket][group]
    const RowsLds places(a);
    uint8_t* const buckets = reinterpret_cast<uint8_t*>(lds + places.biases);   // by r
    char* const tile = lds + places.biases + places.buckets + wave * 2 * kTileBytes;

    int end = ql == 0 ? 0 : kl;   // (the last query sees all keys under the causal mask too)
    const int begin = part * parts.keys;
    if (parts.count > 1) end = end < begin + parts.keys ? end : begin + parts.keys;
    const int limit = a.causal ? (p + 1 < kl ? p + 1 : kl) : kl, all_see = a.causal ? (kl - ql + 1 < kl ? kl - ql + 1 : kl) : kl;

    Lane<DP> at;
    at.set(lane);
    u32x4 qf[Tile<DP>::kSteps];
    load_row<T, DP>(qf, a.q.at<T>(b, h) + (int64_t)t * a.q.token, mine, a.head_dim, half);
    Running<T, DP> run;
    run.clear();
    if (begin < end) {
        const T* const kp = a.k.at<T>(b, hk);
        const T* const vp = a.v.at<T>(b, hk);
        Stage<T, DP, kOwnKeys, 64> ks, vs;
        ks.set(a.k.token, a.head_dim, lane);
        vs.set(a.v.token, a.head_dim, lane);
        int key0 = begin + kOwnKeys * wave;
        if (key0 < end) {
            ks.fetch(kp + (int64_t)key0 * a.k.token, kl - key0);
            vs.fetch(vp + (int64_t)key0 * a.v.token, kl - key0);
        }
        float bias_left = 0.f, bias_right = 0.f;
        if (a.table) {
            bias_left = a.bias<T>(a.n_edges, h);
            bias_right = a.bias<T>(a.two_sided ? 2 * a.n_edges + 1 : 0, h);
            if (kl - ql - (end + kOwnKeys) < a.left) {   // (else all of this part's keys lie beyond the last edge)
                const int n = places.n_buckets * a.group;
                for (int i = threadIdx.x; i < n; i += 256) biases[i] = a.bias<T>(i / a.group, hk * a.group + i % a.group);
                for (int i = threadIdx.x; i < window.size; i += 256) buckets[i] = (uint8_t)a.bucket(window.first + i);
            }
        }
        __syncthreads();
        for (; key0 < end; key0 += 4 * kOwnKeys) {
            ks.park(tile + kTileBytes, lane);
            wave_fence();
            floatx16 s[1] = {zero16()};
#pragma unroll
            for (int st = 0; st < Tile<DP>::kSteps; ++st) s[0] = mfma(at.rows(tile + kTileBytes, 0, st), qf[st], s[0], T{});
            const int next = key0 + 4 * kOwnKeys;
            if (next < end) ks.fetch(kp + (int64_t)next * a.k.token, kl - next);
            vs.park(tile, lane);
            if (next < end) vs.fetch(vp + (int64_t)next * a.v.token, kl - next);
            const int r_lo = key0 - (kl - ql + a.q_tokens - 1), r_hi = key0 + kOwnKeys - 1 - (kl - ql);
            const int place = a.table ? place_of(a, r_lo, r_hi) : kLeft;
            const float bias = place == kRight ? bias_right : bias_left;
            bool fused = true;
            if (place == kNear) {
                const uint8_t* const n = buckets + (key0 - p - window.first + 4 * half);
                const float* const mine_of = biases + (l32 < columns ? g : 0);
                fused = false;
#pragma unroll
                for (int i = 0; i < 16; ++i) s[0][i] = __builtin_fmaf(s[0][i], a.scale, mine_of[n[8 * (i >> 2) + (i & 3)] * a.group]);
            } else if (__any(!(__builtin_fabsf(bias) < kLarge))) {   // (lanes have biases of different heads)
                fused = false;
#pragma unroll
                for (int i = 0; i < 16; ++i) s[0][i] = __builtin_fmaf(s[0][i], a.scale, bias);
            }
            if (key0 + kOwnKeys > all_see) mask_scores(s, key0, limit, half);
            run.weigh(s, fused, a.scale, bias);
            wave_fence();
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                const u32x4 w = weights_of<T>(s[0], st);
#pragma unroll
                for (int d = 0; d < Tile<DP>::kBlocks; ++d) run.o[d] = mfma(at.columns(tile, d, st), w, run.o[d], T{});
            }
            wave_fence();
        }
    }
    meet<T, DP>(run, lds, a, out, lse, parts, b, hk, part, columns, mine);
}

// Four neighbouring values of a row per thread.
template <typename T, int DP> __global__ void __launch_bounds__(256) join_kernel(Args a, Heads out, float* __restrict__ lse, Parts parts)
{
    const int64_t rows = (int64_t)a.batch * a.q_heads * a.q_tokens, item = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = item / (DP / 4);
    const int d = 4 * (int)(item % (DP / 4));
    if (row >= rows) return;
    float m = -ATT_INF, total = 0.f;
#pragma unroll 8
    for (int n = 0; n < parts.count; ++n) {
        const float2 st = parts.stats[n * rows + row];
        m = __builtin_fmaxf(m, st.y != 0.f ? st.x : -ATT_INF);
    }
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int n = 0; n < parts.count; ++n) {
        const float2 st = parts.stats[n * rows + row];
        const f32x4 x = *reinterpret_cast<const f32x4*>(parts.sums + (n * rows + row) * DP + d);
        const bool any = st.y != 0.f;   // (a part that no key reached counts for nothing, whatever it left)
        const float f = any ? exp2_of((st.x - m) * kLog2e) : 0.f;
        total = __builtin_fmaf(f, st.y, total);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(f, any ? x[e] : 0.f, o[e]);
    }
    const float f = total != 0.f ? 1.f / total : 0.f;
    const int i = (int)(row % a.q_tokens), bh = (int)(row / a.q_tokens), b = bh / a.q_heads, h = bh % a.q_heads;
    if (d < a.head_dim)
        *reinterpret_cast<u32x2*>(out.at<T>(b, h) + (int64_t)i * out.token + d) = u32x2{pair_of(o[0] * f, o[1] * f, T{}), pair_of(o[2] * f, o[3] * f, T{})};
    if (lse && d == 0) lse[row] = lse_of(m, total);
}

// Which kernel, and into how many parts the keys are cut.
enum class Route { kOwn, kRows, kTiles };
struct Plan {
    Route route;
    int q_tiles, parts, part_keys;
    int64_t rows;
    size_t workspace;
};
constexpr int64_t kEnoughRows = 4096;   // workgroups that fill the device where all they do is read, and their sequences' lengths differ (32 caches of up to 32768 tokens, 8 heads of 128:
                                        // 536 us with 2048, 476 with 4096, 468 and more to join with 8192)
Plan plan_of(const pruner_attention* a)
{
    Plan p{};
    const int group = a->q_heads / a->kv_heads;
    p.rows = (int64_t)a->batch * a->q_heads * a->q_tokens;
    p.q_tiles = (a->q_tokens + 127) / 128;
    p.parts = 1;
    // (us, by wavefronts of their own, by the queries of a key head side by side, by shared tiles: 2048 sequences of up to 8 tokens, 64 wide, 7, 16, 17; 300 of 30 queries and
    // 60 keys, 8 heads of 64, 14, 27, 22; one token against 32 caches of up to 32768, 8 heads of 128 for 32, -, 405, 903; against 300, 8 heads of 64, -, 8, 10)
    p.route = a->q_tokens <= 32 && a->k_tokens <= 2 * kOwnKeys ? Route::kOwn : (int64_t)a->q_tokens * group <= 32 ? Route::kRows : Route::kTiles;
    const int64_t groups = p.route == Route::kRows ? (int64_t)a->batch * a->kv_heads : (int64_t)a->batch * a->q_heads * p.q_tiles;
    if (p.route != Route::kOwn && groups > 0) {
        const int dp = padded_dim(a->head_dim);
        int64_t parts;
        if (p.route == Route::kRows) {
            // keys of a part at least (256, 512 and 1024, us a call: one token against 5000 keys, 8 heads of 64, 18, 17, 18; 2 tokens of 4 sequences against 3000, 16 heads of 128 sharing 4,
            // 18, 18, 20; one against 60000, 8 heads of 128 sharing one, 100, 58, 39)
            const int fewest = 512;
            parts = (kEnoughRows + groups - 1) / groups;
            const int64_t most = ((int64_t)a->k_tokens + fewest - 1) / fewest;
            parts = parts < most ? parts : most;
        } else {   // (steps as measured: 8192 causal tokens, 16 heads of 128; 5417, 4 of 64; those of 32 wide heads: 200 queries and
                   // 9000 keys, 4 heads, 34 us by 64 wide heads' steps, 28 by these, 1500 causal tokens, 2 heads, 17 either way)
            parts = parts_of((double)groups, (a->k_tokens + kKeys - 1) / kKeys, a->flags & PRUNER_ATTENTION_CAUSAL, dp == 128 ? 512 : 768, dp == 128 ? 1.5 : dp == 64 ? 1.1 : 0.8,
                             dp == 32 ? 1.6 : 2.2, (double)p.rows * dp * 4);
        }
        if (parts < 1) parts = 1;
        const int64_t keys = ((a->k_tokens + parts - 1) / parts + kKeys - 1) / kKeys * kKeys;
        p.part_keys = (int)(keys > 0 ? keys : kKeys);
        p.parts = (int)((a->k_tokens + (int64_t)p.part_keys - 1) / p.part_keys);
        if (p.parts < 1) p.parts = 1;
    }
    p.workspace = p.parts > 1 ? round_up((size_t)p.parts * p.rows * 8, 256) + round_up((size_t)p.parts * p.rows * padded_dim(a->head_dim) * 4, 256) : 0;
    return p;
}

template <typename T, int DP> int run(const Args& args, const Plan& plan, const Heads& out, float* lse, void* workspace, hipStream_t st)
{
    static PerDeviceFlag ready;
    int dev = current_device(nullptr);
    if (dev < 0) return PRUNER_EHIP;
    if (!ready.get(dev)) {
        for (const void* fn : {reinterpret_cast<const void*>(&tile_kernel<T, DP, true>), reinterpret_cast<const void*>(&tile_kernel<T, DP, false>),
                               reinterpret_cast<const void*>(&rows_kernel<T, DP>)})
            if (hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) != hipSuccess) return PRUNER_EHIP;
        ready.mark(dev);
    }
    Parts parts{nullptr, nullptr, plan.parts, plan.part_keys};
    if (plan.parts > 1) {
        parts.stats = static_cast<float2*>(workspace);
        parts.sums = reinterpret_cast<float*>(static_cast<char*>(workspace) + round_up((size_t)plan.parts * plan.rows * 8, 256));
    }
    const Window w(args.left, args.right);
    const size_t window = args.table ? round_up((size_t)w.size * 4, 16) : 0;
    const int64_t heads = (int64_t)args.batch * args.q_heads;
    if (plan.route == Route::kOwn) {
        hipLaunchKernelGGL((tile_kernel<T, DP, false>), dim3((unsigned)((heads + 3) / 4)), dim3(256), 4 * (window + 2 * kOwnKeys * DP * 2), st, args, out, lse, parts, 1);
    } else if (plan.route == Route::kRows) {
        const size_t columns = (size_t)args.q_tokens * args.group, last = 4 * 32 * 8 + 4 * columns * (DP + 4) * 4;
        const RowsLds places(args);
        const size_t tiles = (size_t)places.biases + places.buckets + 8 * kOwnKeys * DP * 2;
        hipLaunchKernelGGL((rows_kernel<T, DP>), dim3((unsigned)((int64_t)args.batch * args.kv_heads * plan.parts)), dim3(256), last > tiles ? last : tiles, st, args, out, lse, parts);
    } else {
        hipLaunchKernelGGL((tile_kernel<T, DP, true>), dim3((unsigned)(heads * plan.q_tiles * plan.parts)), dim3(256), window + turns_of(DP, true, kKeys) * 2 * kKeys * DP * 2, st, args, out, lse, parts,
                           plan.q_tiles);
    }
    PRUNER_LAUNCH_CHECK();
    if (plan.parts > 1) {
        hipLaunchKernelGGL((join_kernel<T, DP>), dim3((unsigned)((plan.rows * (DP / 4) + 255) / 256)), dim3(256), 0, st, args, out, lse, parts);
        PRUNER_LAUNCH_CHECK();
    }
    return PRUNER_OK;
}

}  // namespace

bool heads_ok(const pruner_heads* h)
{
    return h && h->p && aligned(h->p, 16) && h->batch % 8 == 0 && h->token % 8 == 0 && h->head % 8 == 0 && h->token >= 0 && h->token <= (1 << 22) && h->batch >= 0 && h->head >= 0;
}
Heads heads_of(const pruner_heads* h) { return Heads{static_cast<char*>(h->p), h->batch, h->head, (int32_t)h->token}; }

bool attention_sizes_ok(const pruner_attention* a)
{
    if (!a || (a->dtype != PRUNER_BF16 && a->dtype != PRUNER_F16)) return false;
    if (a->batch < 0 || a->q_tokens < 0 || a->k_tokens < 0 || a->q_tokens >= (1 << 30) || a->k_tokens >= (1 << 30)) return false;
    if (a->q_heads < 1 || a->kv_heads < 1 || a->q_heads % a->kv_heads || a->q_heads > (1 << 20)) return false;
    if (a->head_dim < 8 || a->head_dim > 128 || a->head_dim % 8) return false;
    // (a launch is below 2^24 workgroups of 256 threads)
    const int64_t heads = (int64_t)a->batch * a->q_heads;
    if (heads >= (1 << 24) || heads * (a->q_tokens / 64 + 1) >= (1 << 24) || heads * a->q_tokens >= (1ll << 31)) return false;
    if (a->flags & ~(PRUNER_ATTENTION_CAUSAL | PRUNER_ATTENTION_TWO_SIDED)) return false;
    if (!(a->scale > 0.f) || !(a->scale < 3.0e38f)) return false;
    if (a->n_edges < 0 || a->n_edges > PRUNER_MAX_BIAS_EDGES) return false;
    return true;
}

int attention_args(const pruner_attention* a, const pruner_heads* q, const pruner_heads* k, const pruner_heads* v, Args* out)
{
    const pruner_heads none{nullptr, 0, 0, 0};
    const bool queries = a->batch > 0 && a->q_tokens > 0, keys = a->batch > 0 && a->k_tokens > 0;
    if (!queries) q = &none;
    if (!keys) k = v = &none;
    if ((queries && !heads_ok(q)) || (keys && (!heads_ok(k) || !heads_ok(v)))) return PRUNER_EINVAL;
    if ((a->q_len && !aligned(a->q_len, 4)) || (a->k_len && !aligned(a->k_len, 4)) || (a->table && !aligned(a->table, 2)) || (a->table && a->n_edges > 0 && !a->edges)) return PRUNER_EINVAL;
    Args r{};
    r.q = heads_of(q);
    r.k = heads_of(k);
    r.v = heads_of(v);
    r.q_len = a->q_len;
    r.k_len = a->k_len;
    r.table = a->table;
    r.batch = a->batch;
    r.q_tokens = a->q_tokens;
    r.k_tokens = a->k_tokens;
    r.q_heads = a->q_heads;
    r.kv_heads = a->kv_heads;
    r.group = a->q_heads / a->kv_heads;
    r.head_dim = a->head_dim;
    r.causal = (a->flags & PRUNER_ATTENTION_CAUSAL) != 0;
    r.two_sided = (a->flags & PRUNER_ATTENTION_TWO_SIDED) != 0;
    r.scale = a->scale;
    for (int e = 0; e < PRUNER_MAX_BIAS_EDGES; ++e) r.edges[e] = INT32_MAX;
    if (a->table) {
        int last = 0;
        for (int e = 0; e < a->n_edges; ++e) {
            if (a->edges[e] <= last || a->edges[e] > PRUNER_MAX_BIAS_DISTANCE) return PRUNER_EINVAL;
            last = r.edges[e] = a->edges[e];
        }
        r.n_edges = a->n_edges;
        // r > right - 1 and r < -left + 1 are of one bucket each; neither needs to lie beyond what the lengths can reach
        const int64_t reach = (int64_t)a->q_tokens + a->k_tokens;
        r.left = (int)(last < reach ? last : reach);
        r.right = !r.two_sided ? 0 : last > 1 ? r.left : 1;
        if (r.two_sided && r.right < 1) r.right = 1;
    }
    *out = r;
    return PRUNER_OK;
}

}  // namespace att
}  // namespace pruner

using namespace pruner;

extern "C" size_t pruner_rel_attention_workspace_bytes(const pruner_attention* a) { return att::attention_sizes_ok(a) ? att::plan_of(a).workspace : 0; }

extern "C" int pruner_rel_attention(const pruner_attention* a, const pruner_heads* q, const pruner_heads* k, const pruner_heads* v, const pruner_heads* o, float* lse,
                                    void* workspace, size_t workspace_bytes, void* stream)
{
    if (!att::attention_sizes_ok(a)) return PRUNER_EINVAL;
    if (a->batch == 0 || a->q_tokens == 0) return PRUNER_OK;
    att::Args args;
    const int rc = att::attention_args(a, q, k, v, &args);
    if (rc) return rc;
    if (!att::heads_ok(o) || (lse && !aligned(lse, 4))) return PRUNER_EINVAL;
    const att::Plan plan = att::plan_of(a);
    if (plan.parts > 1 && (!workspace || !aligned(workspace, 256) || workspace_bytes < plan.workspace)) return PRUNER_EWORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const att::Heads out = att::heads_of(o);
    const int dp = att::padded_dim(a->head_dim);
    if (a->dtype == PRUNER_BF16)
        return dp == 32   ? att::run<__bf16, 32>(args, plan, out, lse, workspace, st)
               : dp == 64 ? att::run<__bf16, 64>(args, plan, out, lse, workspace, st)
                          : att::run<__bf16, 128>(args, plan, out, lse, workspace, st);
    return dp == 32   ? att::run<_Float16, 32>(args, plan, out, lse, workspace, st)
           : dp == 64 ? att::run<_Float16, 64>(args, plan, out, lse, workspace, st)
                      : att::run<_Float16, 128>(args, plan, out, lse, workspace, st);
}
