// Attention with a learned relative position bias by buckets, backward.  With P = exp(s - lse), dP = dO V^T, delta_i = sum_d dO o:
//     dS = P (dP - delta);   dQ = scale dS K;   dK = scale dS^T Q;   dV = P^T dO;   dtable[n][h] = sum of dS over the pairs of bucket n
//
//   queries   a wavefront owns 32 queries, as in the forward pass: S^T and dP^T leave a query's values in its two lanes; dQ^T += K^T dS^T.
//             It also leaves the sums of dS along the diagonals j - p: a tile beyond the largest edge adds into one register, the others add
//             into LDS, where every wavefront has diagonals of its own.
//   keys      a wavefront owns 32 keys: S and dP leave a key's values in its two lanes; dV^T += dO^T P, dK^T += Q^T dS.  It goes
//             through the query tiles of all heads that share the key head.
//   Where either has too few tiles for the device, their long axis is cut into parts, whose sums go to the workspace (join_kernel adds them in order).
//   stats_kernel, both_kernel    lse and delta of every query (and what its weights sum to, where lse does not tell), then queries and keys in one launch.
//   queries_kernel, keys_kernel  the same for sequences of few queries and keys, each by a wavefront; delta is the sum of P dP there.
//   diagonals_kernel, buckets_kernel   the workgroups' diagonals added in order, and the diagonals of a bucket (where the workgroups are few, by the
//             latter alone).
// S and dP are formed twice (14 products of a pair's depth where 10 would do), so that nothing is added across workgroups but in a fixed order.
//
// P and dS are rounded to the operands' type for the products that sum them, at the rate of the matrix cores' 16-bit forms, and delta is taken from o as it is given, rounded (a pass over the
// keys would have it from P dP, as own tiles have): dq is off by 2.4e-3 of itself with 5001 causal tokens in bfloat16, where its own rounding makes 1.66e-3, dS's 2.34e-3 with that and delta's
// 1.71e-3; with 150 causal tokens 2.53e-3, 2.35e-3 and 1.92e-3.
// Bound: the matrix cores with the exponentials and LDS reads between their products.  5001 causal tokens, 16 heads of 128 sharing 4: 414 us in all, queries alone on the device
// 190 (820 TFLOP/s), keys 240 (860), where a large matrix product reaches 1445.  16 sequences of up to 500, 12 heads of 64: 75 us in all, bound by a
// workgroup's chain of tiles and its start (5 us).
#include "rel_attention.h"

namespace pruner {
namespace att {
namespace {

constexpr int kOwn = 32;   // rows of a wavefront's own tile

// Weights before the second product are at most 1: in binary16, which has fewer bits below 2^-14, they are held times 2^15.
template <typename T> struct Held;
template <> struct Held<__bf16> {
    static constexpr float kShift = 0.f, kUnit = 1.f;
};
template <> struct Held<_Float16> {
    static constexpr float kShift = 15.f, kUnit = 1.f / 32768.f;
};

// A row's gradients of its scores, rounded to the type for the product that sums them: in binary16 they are held times a power of two, the same for the row's
// sums, because they are about a row's length smaller than the output's gradient and what lies below 2^-24 is lost (5000 keys, an output's gradient of 1e-3, 64 wide: dq and dk off by
// 6.4e-3 of themselves as they are, by 7.6e-4 where held, of which 7.3e-4 is the result's own rounding; 16 sequences of up to 500, 12 heads of 64, take 74 us where they took 71, 5001
// causal tokens, 16 heads of 128, 452 and 439).  The largest so far lies between 2^10 and 2^15 times the unit: the power changes, and the sums with it, only where it would pass that.
// (bfloat16 has binary32's range.)
template <typename T, int BLOCKS> struct Holder {
    static constexpr bool kAny = __is_same(T, _Float16);
    float up = kAny ? 0x1p100f : 1.f;
    __device__ __forceinline__ void hold(floatx16& x, floatx16 (&sums)[BLOCKS])   // x: this lane's values of its row, the other half's lane has the others
    {
        if constexpr (kAny) {
            float top = __builtin_fabsf(x[0]);
#pragma unroll
            for (int e = 1; e < 16; ++e) top = __builtin_fmaxf(top, __builtin_fabsf(x[e]));
            top = max_of_halves(top);
            if (__any(top * up > 0x1p15f)) {
                const float now = top * up > 0x1p15f ? __uint_as_float((264u - (__float_as_uint(top) >> 23)) << 23) : up, factor = now * down();   // now: top x now in 2^10 .. 2^11
                up = now;
#pragma unroll
                for (int d = 0; d < BLOCKS; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) sums[d][i] *= factor;
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] *= up;
        }
    }
    __device__ __forceinline__ float down() const { return __uint_as_float((254u << 23) - __float_as_uint(up)); }   // 1 / up
    __device__ __forceinline__ void release(floatx16 (&sums)[BLOCKS]) const
    {
        if constexpr (kAny)
#pragma unroll
            for (int d = 0; d < BLOCKS; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) sums[d][i] *= down();
    }
};

struct Grad {
    Heads dout, o, out0, out1;   // out0, out1: dq, or dk and dv
    const float* lse;
    float* stats;                // [kStats][batch][q_heads][stat_rows]: see leave_stats
    int stat_rows;               // q_tokens rounded up to 32
    float* diagonals;            // [part][q_heads][window + 2]
    float* sums;                 // of the parts: [part][batch][q_heads][q_tokens][DP], or [part][batch][kv_heads][k_tokens][2][DP]
    int parts, part_keys;        // part_keys: of the queries' kernel, a multiple of 64
};

// What the keys' kernel needs of a query: lse (plus infinity without a key, or where there is no query: every weight is then exp(-infinity)), what is added to the exponent of 2, -delta,
// as they go with the form in which the weights are held, and what the weights exp(s - lse) are multiplied by.  more: log2 of what these sum to.
constexpr int kStats = 4;
template <typename T> __device__ __forceinline__ void leave_stats(const Grad& gr, int64_t heads, int bh, int i, float lse, float delta, float more)
{
    if (i >= gr.stat_rows) return;
    const int64_t all = heads * gr.stat_rows, row = (int64_t)bh * gr.stat_rows + i;
    gr.stats[row] = lse;
    gr.stats[all + row] = Held<T>::kShift - lse * kLog2e - more;
    gr.stats[2 * all + row] = -delta * Held<T>::kUnit;
    gr.stats[3 * all + row] = exp2_of(-more);
}
// Whether a row's weights have to be summed again because of lse binary32 keeps too few digits (at 1024 they sum to 1 within 6e-5; a row that sees nothing but a mask's -1e9 has
// lse = -1e9, whatever the number of its keys, and weights of 1 each).
__device__ __forceinline__ bool sums_unknown(float lse) { return __builtin_fabsf(lse) > kLarge && __builtin_fabsf(lse) < ATT_INF; }

// Sums of a 32 x 32 result along its diagonals, sixteen rows at a time: element (row, column) goes to place row of line row - column + 31, so a
// line is a diagonal; lane d adds line d's sixteen places (those that no element reaches stay zero) and adds that to its diagonal's sum.  Lines are 18
// floats apart: 32 columns' writes meet two to a bank, the lanes' 8-byte reads none.  (Adding element by element into the sums, by LDS additions,
// took the queries' kernel 157 us where this took 53: 16 sequences of up to 500 tokens, 12 heads of 64, edges up to 128.)
constexpr int kLine = 18, kLines = 47, kSkewFloats = kLines * kLine + 2;
constexpr bool skew_in_values(int dp, bool shared) { return !shared && dp >= 64; }
__device__ __forceinline__ void add_diagonals(float* skew, float* sums, const floatx16& x, int lane, int half, int l32)
{
    float* const to = skew + (4 * half - l32 + 31) * kLine + 4 * half;
    const float* const from = skew + (lane < kLines ? lane : 0) * kLine;
#pragma unroll
    for (int hb = 0; hb < 2; ++hb) {
#pragma unroll
        for (int e = 0; e < 8; ++e) to[(8 * (e >> 2) + (e & 3)) * (kLine + 1)] = x[8 * hb + e];
        wave_fence();
        float s = 0.f;
#pragma unroll
        for (int t = 0; t < 16; t += 2) {
            const f32x2 v = *reinterpret_cast<const f32x2*>(from + t);
            s += v[0] + v[1];
        }
        if (lane < kLines) sums[16 * hb + lane] += s;
        wave_fence();
    }
}

template <typename T, int DP, bool SHARED> __device__ __forceinline__ void queries_of(const Args& a, const Grad& gr, int q_tiles, uint32_t block)
{
    constexpr int kN = SHARED && DP < 128 ? 64 : kOwn, kThreads = SHARED ? 256 : 64, kTileBytes = kN * Tile<DP>::kRowBytes, kTurns = turns_of(DP, SHARED, kN);   // (64 keys of 128 would leave no room for a second workgroup)
    static_assert((SHARED ? kTurns : 4) * 2 * kTileBytes <= kRequestRoom, "tiles lie where requests reach");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), half = lane >> 5, l32 = lane & 31, thread = SHARED ? (int)threadIdx.x : lane;
    const uint32_t heads = (uint32_t)a.batch * a.q_heads;
    int bh, q0, tile_id = 0, part = 0;   // (tile_id: of the tiles and their parts)
    if constexpr (SHARED) {
        const Item it = item_of(block, (uint32_t)a.batch * a.kv_heads, a.group, (uint32_t)q_tiles * gr.parts);
        bh = it.head;
        tile_id = it.tile;
        part = it.tile % gr.parts;
        q0 = it.tile / gr.parts * 128 + 32 * wave;
    } else {
        bh = (int)(block * 4 + wave);
        q0 = 0;
        if (bh >= (int)heads) return;
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
    const int window_floats = a.table ? (window.size + 3) & ~3 : 0;
    // LDS: tiles, biases, every wavefront's diagonals and its skewed square
    char* const tiles = lds + (SHARED ? 0 : wave * 2 * kTileBytes);
    float* const floats = reinterpret_cast<float*>(lds + (SHARED ? 2 * kTurns : 8) * kTileBytes);
    float* const biases = floats + (SHARED ? 0 : wave * window_floats);
    float* const all_diagonals = floats + (SHARED ? 1 : 4) * window_floats;
    float* const diagonals = all_diagonals + wave * window_floats;
    // (a wavefront's own, where it fits: where its values lie, once they have been used)
    constexpr bool kInValues = skew_in_values(DP, SHARED);
    static_assert(!kInValues || kSkewFloats * 4 <= kTileBytes, "the square fits the values' tile");
    float* const skew = kInValues ? reinterpret_cast<float*>(tiles + kTileBytes) : all_diagonals + 4 * window_floats + wave * kSkewFloats;

    const int first_q = SHARED ? q0 - 32 * wave : 0, rows_here = SHARED ? 128 : 32;
    const int last_q = first_q + rows_here < ql ? first_q + rows_here - 1 : ql - 1;
    int end = first_q >= ql ? 0 : a.causal ? kl - ql + last_q + 1 : kl;
    end = end < kl ? end : kl;
    const int begin = SHARED ? part * gr.part_keys : 0;
    if (SHARED && gr.parts > 1) end = end < begin + gr.part_keys ? end : begin + gr.part_keys;

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
    constexpr int kAhead = SHARED ? kTurns - 1 : 1;   // tiles on their way before the first is worked on
    if (begin < end)
#pragma unroll
        for (int t = 0; t < kAhead; ++t) request(begin + t * kN, t);
    Lane<DP> at;
    at.set(lane);
    const int i = q0 + l32, p = kl - ql + i;
    const bool mine = i < ql;
    u32x4 qf[Tile<DP>::kSteps], df[Tile<DP>::kSteps];
    load_row<T, DP>(qf, a.q.at<T>(b, h) + (int64_t)i * a.q.token, mine, a.head_dim, half);
    load_row<T, DP>(df, gr.dout.at<T>(b, h) + (int64_t)i * gr.dout.token, mine, a.head_dim, half);
    float delta = 0.f, lse = ATT_INF, more = 0.f;
    const int64_t row = (int64_t)bh * a.q_tokens + i;
    if (mine) {
        if constexpr (SHARED) {
            const int64_t stat = (int64_t)bh * gr.stat_rows + i;
            lse = gr.stats[stat];
            delta = gr.stats[2 * (int64_t)heads * gr.stat_rows + stat] * (-1.f / Held<T>::kUnit);
            more = -__builtin_amdgcn_logf(gr.stats[3 * (int64_t)heads * gr.stat_rows + stat]);   // (base 2; 0 of 1)
        } else {
            lse = gr.lse[row];
            lse = lse == -ATT_INF ? ATT_INF : lse;   // (no key: every weight is exp(-infinity))
        }
    }
    floatx16 dq[Tile<DP>::kBlocks];
#pragma unroll
    for (int d = 0; d < Tile<DP>::kBlocks; ++d) dq[d] = zero16();
    Holder<T, Tile<DP>::kBlocks> holder;
    float sum_left = 0.f, sum_right = 0.f;
    if (a.table) {
        for (int n = lane; n < window_floats; n += kWave) diagonals[n] = 0.f;
        if constexpr (!kInValues)
            for (int n = lane; n < kSkewFloats; n += kWave) skew[n] = 0.f;
    }
    if (begin < end) {
        if (a.table) fill.store(a, window, biases, h, thread);
        const int wave_last = q0 + 31 < ql ? q0 + 31 : ql - 1;
        const int seen = q0 >= ql ? 0 : a.causal ? (kl - ql + wave_last + 1 < kl ? kl - ql + wave_last + 1 : kl) : kl;
        const int limit = a.causal ? (p + 1 < kl ? p + 1 : kl) : kl, all_see = a.causal ? (kl - ql + q0 + 1 < kl ? kl - ql + q0 + 1 : kl) : kl;
        // P (in s) and dP (in ds) of 32 keys from k0; returns where they lie
        auto weigh = [&](const char* kt, int n, int k0, floatx16& s, floatx16& ds) {
            s = ds = zero16();
            auto key_or_value = [&](int x) { return at.rows(kt + x % 2 * kTileBytes, n, x / 2); };
            Operands<2 * Tile<DP>::kSteps, 6> rows;
            rows.start(key_or_value);
            rows.products(key_or_value, [&](int x, u32x4 w) {
                if (x % 2 == 0)
                    s = mfma(w, qf[x / 2], s, T{});
                else
                    ds = mfma(w, df[x / 2], ds, T{});
            });
            const int r_lo = k0 - (kl - ql + q0 + 31), r_hi = k0 + 31 - (kl - ql + q0);
            const int place = a.table ? place_of(a, r_lo, r_hi) : kLeft;
            const float bias = place == kRight ? bias_right : bias_left;
            if (place == kNear || !(__builtin_fabsf(bias) < kLarge)) {
                const float* const w = biases + (k0 - p - window.first + 4 * half);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float t = __builtin_fmaf(s[e], a.scale, place == kNear ? w[8 * (e >> 2) + (e & 3)] : bias);
                    s[e] = exp2_of(__builtin_fmaf(t - lse, kLog2e, -more));
                }
            } else {
                const float c = a.scale * kLog2e, d = __builtin_fmaf(bias - lse, kLog2e, -more);
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = exp2_of(__builtin_fmaf(s[e], c, d));
            }
            if (k0 + 32 > all_see) {
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = k0 + row_of(e, half) < limit ? s[e] : 0.f;
            }
            return place;
        };
        settle();
        if constexpr (!SHARED) {
            // delta as the sum of P dP: o is rounded, and with a few keys what it lost is as large as the gradient's own rounding
            float total = 0.f;
            for (int key0 = 0; key0 < end; key0 += kN) {
                wait_for<0>();
                wave_fence();
                if (key0 < seen) {
                    floatx16 s, dp;
                    weigh(tiles, 0, key0, s, dp);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        delta = __builtin_fmaf(s[e], dp[e], delta);
                        total += s[e];
                    }
                }
                wait_for_reads();
                wave_fence();
                if (end > kN) request(key0 + kN < end ? key0 + kN : 0, 0);
            }
            delta = sum_of_halves(delta);
            total = sum_of_halves(total);
            if (sums_unknown(lse)) {
                more = __builtin_amdgcn_logf(total);   // (base 2)
                delta /= total;
            }
        }
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
#pragma unroll
            for (int n = 0; n < kN / 32; ++n) {
                const int k0 = key0 + 32 * n;
                if (k0 >= seen) continue;
                floatx16 s, ds;
                const int place = weigh(kt, n, k0, s, ds);
                auto key = [&](int x) { return at.columns(kt, x % Tile<DP>::kBlocks, 2 * n + x / Tile<DP>::kBlocks); };
                Operands<2 * Tile<DP>::kBlocks, 4> columns;
                columns.start(key);
#pragma unroll
                for (int e = 0; e < 16; ++e) ds[e] = s[e] * (ds[e] - delta);
                if (a.table) {
                    if (place == kNear) {
                        if constexpr (kInValues) {
                            wait_for_reads();
                            wave_fence();
                            for (int n = lane; n < kSkewFloats; n += kWave) skew[n] = 0.f;
                            wave_fence();
                        }
                        add_diagonals(skew, diagonals + (k0 - (kl - ql + q0) - 31 - window.first), ds, lane, half, l32);
                    } else {
                        float sum = 0.f;
#pragma unroll
                        for (int e = 0; e < 16; ++e) sum += ds[e];
                        if (place == kRight)
                            sum_right += sum;
                        else
                            sum_left += sum;
                    }
                }
                holder.hold(ds, dq);
                u32x4 weights{};
                columns.products(key, [&](int x, u32x4 w) {
                    if (x % Tile<DP>::kBlocks == 0) weights = weights_of<T>(ds, x / Tile<DP>::kBlocks);
                    dq[x % Tile<DP>::kBlocks] = mfma(w, weights, dq[x % Tile<DP>::kBlocks], T{});
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
        wait_for<0>();   // (nothing may arrive in LDS that is used for other things, or no longer this workgroup's)
    }
    if (!SHARED && half == 0) leave_stats<T>(gr, heads, bh, i, lse, delta, more);
    holder.release(dq);
    if (i < a.q_tokens) {
        if (SHARED && gr.parts > 1)
            store_row32<DP>(gr.sums + ((int64_t)part * heads * a.q_tokens + row) * DP, dq, half);
        else
            store_row<T, DP>(gr.out0.at<T>(b, h) + (int64_t)i * gr.out0.token, dq, a.scale, a.head_dim, half);
    }
    if (!a.table) return;
    // what this workgroup (wavefront) saw of every diagonal
    const int width = window.size + 2;
    float* const to = gr.diagonals + ((int64_t)(SHARED ? b * q_tiles * gr.parts + tile_id : b) * a.q_heads + h) * width;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        sum_left += __shfl_xor(sum_left, o, kWave);
        sum_right += __shfl_xor(sum_right, o, kWave);
    }
    if constexpr (SHARED) {
        __syncthreads();   // (the tiles are no longer needed)
        float* const ends = reinterpret_cast<float*>(tiles);
        if (lane == 0) {
            ends[2 * wave] = sum_left;
            ends[2 * wave + 1] = sum_right;
        }
        __syncthreads();
        for (int n = threadIdx.x; n < width; n += 256) {
            float s = 0.f;
            if (n < window.size)
                for (int w = 0; w < 4; ++w) s += all_diagonals[w * window_floats + n];
            else
                for (int w = 0; w < 4; ++w) s += ends[2 * w + (n - window.size)];
            to[n] = s;
        }
    } else {
        wave_fence();
        for (int n = lane; n < width; n += kWave) to[n] = n < window.size ? diagonals[n] : n == window.size ? sum_left : sum_right;
    }
}

template <typename T, int DP> __global__ void __launch_bounds__(256, 2) queries_kernel(Args a, Grad gr) { queries_of<T, DP, false>(a, gr, 1, blockIdx.x); }

// A wavefront's keys and values are operands in registers; of 128 wide heads the values' lie in LDS, each lane's own sixteen bytes of every step side by side (in
// registers they left the sums no room: 821 us where this took 295 at 5001 causal tokens).
template <typename T, int DP, bool SHARED> struct KeysShape {
    static constexpr bool kWide = SHARED && DP == 128;
    static constexpr int kWaves = 4;                          // of a workgroup (wide: eight would share a tile's requests, but wait for each other: 252 us where this took 228)
    static constexpr int kQ = SHARED && !kWide ? 64 : 32;     // queries of a tile
    static constexpr int kTurns = SHARED ? (kWide ? 2 : 3) : 1;
    // Shared tiles have their stats behind them; own tiles, which 128 wide fill what requests reach, lie side by side and their stats, which arrive through registers, behind
    // them all (three wavefronts instead: 783 sequences of 6 queries and 55 keys, 16 heads of 128 sharing two, 250 us where this takes 225).
    static constexpr int kStat = SHARED ? 64 : 32;            // floats of one of a tile's stats
    static constexpr int kStatBytes = kStats * kStat * 4, kTileBytes = kQ * Tile<DP>::kRowBytes, kTurnBytes = 2 * kTileBytes + (SHARED ? kStatBytes : 0);
    static constexpr int kHeldBytes = kWide ? Tile<DP>::kSteps * 1024 : 0;   // of a wavefront
    static constexpr int kKeys = SHARED ? 32 * kWaves : 32;
    static_assert((SHARED ? kTurns : kWaves) * kTurnBytes <= kRequestRoom, "tiles lie where requests reach");
    static constexpr int kBytes = SHARED ? kTurns * kTurnBytes + kWaves * kHeldBytes : kWaves * (kTurnBytes + kStatBytes);   // of LDS before the biases
};
template <typename T, int DP, bool SHARED> __device__ __forceinline__ void keys_of(const Args& a, const Grad& gr, int k_tiles, uint32_t block)
{
    typedef KeysShape<T, DP, SHARED> Shape;
    constexpr int kQ = Shape::kQ, kThreads = SHARED ? 64 * Shape::kWaves : 64, kTileBytes = Shape::kTileBytes, kTurnBytes = Shape::kTurnBytes;
    constexpr bool kWide = Shape::kWide;
    constexpr int kTurns = Shape::kTurns, kStat = Shape::kStat;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), half = lane >> 5, l32 = lane & 31, thread = SHARED ? (int)threadIdx.x : lane;
    const uint32_t heads = (uint32_t)a.batch * a.kv_heads;
    int part = 0, bh, k0;
    if constexpr (SHARED) {
        const Item it = item_of(block, heads, 1, (uint32_t)k_tiles * gr.parts);
        bh = it.head;
        part = it.tile % gr.parts;
        k0 = (k_tiles - 1 - it.tile / gr.parts) * Shape::kKeys + 32 * wave;   // (under a causal mask the first keys are seen by the most queries)
    } else {
        const int64_t unit = (int64_t)block * Shape::kWaves + wave;
        if (unit >= (int64_t)heads * k_tiles) return;
        bh = (int)(unit / k_tiles);
        k0 = (int)(unit % k_tiles) * 32;
    }
    const int b = bh / a.kv_heads, hk = bh % a.kv_heads;
    const int ql = a.queries(b), kl = a.keys(b);
    const Window window(a.left, a.right);
    const int window_floats = a.table ? (window.size + 3) & ~3 : 0;
    char* const turns = lds + (SHARED ? 0 : wave * kTurnBytes);
    char* const held = lds + Shape::kTurns * kTurnBytes + wave * Shape::kHeldBytes + 16 * lane;
    float* const own_stats = reinterpret_cast<float*>(lds + Shape::kWaves * kTurnBytes + wave * Shape::kStatBytes);
    float* const biases = reinterpret_cast<float*>(lds + Shape::kBytes) + (SHARED ? 0 : wave * window_floats);

    // query tiles that see any of this workgroup's keys
    const int first_key = SHARED ? k0 - 32 * wave : k0, shift = kl - ql;
    int first_tile = 0;
    if (a.causal && first_key > shift) first_tile = (first_key - shift) / kQ;
    int each = (ql + kQ - 1) / kQ - first_tile;
    if (each < 0 || first_key >= kl) each = 0;
    const int64_t total = (int64_t)each * a.group;
    const int from = (int)(total * part / gr.parts), to = (int)(total * (part + 1) / gr.parts);

    Flow<T, DP, kQ, kThreads> qf, of;
    qf.set(a.q.token, a.head_dim, thread, SHARED ? wave : 0);
    of.set(gr.dout.token, a.head_dim, thread, SHARED ? wave : 0);
    const int64_t all = (int64_t)a.batch * a.q_heads * gr.stat_rows;
    float stat_in[2] = {0.f, 0.f};   // own tiles: this lane's values of the next tile's stats
    static_assert(!SHARED || Shape::kWaves == kStats, "of those that share a tile each asks for one of its stats");
    auto request = [&](int n, int turn) {
        const bool some = n < to;
        const int h = some ? hk * a.group + n / each : 0, i0 = some ? (first_tile + n % each) * kQ : 0, left = some ? ql - i0 : 0;
        const uint32_t place = (uint32_t)((SHARED ? turn : wave) * kTurnBytes);
        qf.request(a.q.at<T>(b, h) + (int64_t)i0 * a.q.token, left, place);
        of.request(gr.dout.at<T>(b, h) + (int64_t)i0 * gr.dout.token, left, place + kTileBytes);
        const float* const stats = gr.stats + ((int64_t)b * a.q_heads + h) * gr.stat_rows + i0;
        if constexpr (SHARED) {
            request_4(place + 2 * kTileBytes + 4 * kStat * wave, lane < kQ ? 4u * (uint32_t)lane : 0x80000000u, buffer_of(stats + wave * all, some ? 4 * (gr.stat_rows - i0) : 0));
        } else if (some) {   // (32 rows of a tile, as many of stats: stat_rows is a multiple of 32)
#pragma unroll
            for (int w = 0; w < 2; ++w) stat_in[w] = stats[(2 * w + half) * all + l32];
        }
    };
    constexpr int kAhead = SHARED ? kTurns - 1 : 1;   // tiles on their way before the first is worked on
    if (from < to)
#pragma unroll
        for (int t = 0; t < kAhead; ++t) request(from + t, t);
    WindowFill<T, kThreads> fill;
    float bias_left = 0.f, bias_right = 0.f;
    int head_loaded = 0;
    auto load = [&](int g) {
        const int h = hk * a.group + g;
        fill.load(a, window, h, thread);
        bias_left = a.bias<T>(a.n_edges, h);
        bias_right = a.bias<T>(a.two_sided ? 2 * a.n_edges + 1 : 0, h);
        head_loaded = g;
    };
    if (from < to && a.table) load(from / each);
    Lane<DP> at;
    at.set(lane);
    const int j = k0 + l32;
    u32x4 kf[Tile<DP>::kSteps], vf[Tile<DP>::kSteps];
    load_row<T, DP>(kf, a.k.at<T>(b, hk) + (int64_t)j * a.k.token, j < kl, a.head_dim, half);
    load_row<T, DP>(vf, a.v.at<T>(b, hk) + (int64_t)j * a.v.token, j < kl, a.head_dim, half);
    if constexpr (kWide) {
#pragma unroll
        for (int st = 0; st < Tile<DP>::kSteps; ++st) *reinterpret_cast<u32x4*>(held + 1024 * st) = vf[st];
    }
    auto value = [&](int st) -> u32x4 {
        if constexpr (kWide)
            return *reinterpret_cast<const u32x4*>(held + 1024 * st);
        else
            return vf[st];
    };
    constexpr int kAheadR = kWide ? 4 : 6, kAheadC = 4;
    floatx16 dk[Tile<DP>::kBlocks], dv[Tile<DP>::kBlocks];
#pragma unroll
    for (int d = 0; d < Tile<DP>::kBlocks; ++d) dk[d] = dv[d] = zero16();
    Holder<T, Tile<DP>::kBlocks> holder;

    if (from < to) {
        settle();
        int turn = 0, head_filled = -1;
        for (int n = from; n < to; ++n) {
            const int g = n / each, h = hk * a.group + g, i0 = (first_tile + n % each) * kQ;
            if (a.table && g != head_filled) {
                if constexpr (SHARED) __syncthreads(); else wave_fence();   // (the head before is done with its biases)
                if (g != head_loaded) load(g);
                fill.store(a, window, biases, h, thread);
                settle();
                head_filled = g;
            }
            if constexpr (SHARED) {
                wait_for<(kTurns - 2) * (2 * Flow<T, DP, kQ, kThreads>::kEach + 1)>();
                __syncthreads();   // (and the tile before is done with)
                request(n + kTurns - 1, turn == 0 ? kTurns - 1 : turn - 1);
            } else {
                wait_for<0>();
#pragma unroll
                for (int w = 0; w < 2; ++w) own_stats[(2 * w + half) * kStat + l32] = stat_in[w];
                wave_fence();
            }
            if constexpr (kWide) at.forget();
            const char* const qt = turns + (SHARED ? turn * kTurnBytes : 0);
            const float* const st = SHARED ? reinterpret_cast<const float*>(qt + 2 * kTileBytes) : own_stats;
#pragma unroll
            for (int m = 0; m < kQ / 32; ++m) {
                const int p0 = shift + i0 + 32 * m;   // position of the block's first query
                const int r_lo = k0 - (p0 + 31), r_hi = k0 + 31 - p0;
                if (k0 >= kl || i0 + 32 * m >= ql || (a.causal && r_lo > 0)) continue;   // (no pair here that counts)
                floatx16 s = zero16(), dp = zero16();
                auto query_or_gradient = [&](int x) { return at.rows(qt + x % 2 * kTileBytes, m, x / 2); };
                Operands<2 * Tile<DP>::kSteps, kAheadR> rows;
                u32x4 of_value[2];   // (wide: values two steps ahead as well)
                if constexpr (kWide) {
                    of_value[0] = value(0);
                    of_value[1] = value(1);
                }
                rows.start(query_or_gradient);
                rows.products(query_or_gradient, [&](int x, u32x4 w) {
                    const int step = x / 2;
                    if (x % 2 == 0) {
                        s = mfma(w, kf[step], s, T{});
                    } else if constexpr (kWide) {
                        dp = mfma(w, of_value[step % 2], dp, T{});
                        if (step + 2 < Tile<DP>::kSteps) of_value[step % 2] = value(step + 2);
                    } else {
                        dp = mfma(w, vf[step], dp, T{});
                    }
                });
                auto turned = [&](int x) { return at.columns(qt + (x % 2 == 0 ? kTileBytes : 0), x / 2 % Tile<DP>::kBlocks, 2 * m + x / (2 * Tile<DP>::kBlocks)); };
                Operands<4 * Tile<DP>::kBlocks, kAheadC> columns;
                if constexpr (!kWide) columns.start(turned);
                const int place = a.table ? place_of(a, r_lo, r_hi) : kLeft;
                const float bias = place == kRight ? bias_right : bias_left;
                if (place == kNear || !(__builtin_fabsf(bias) < kLarge)) {
                    const float* const w = biases + (j - p0 - window.first - 4 * half);
#pragma unroll
                    for (int g4 = 0; g4 < 4; ++g4) {
                        const f32x4 lse = *reinterpret_cast<const f32x4*>(st + 32 * m + 8 * g4 + 4 * half);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float t = __builtin_fmaf(s[4 * g4 + e], a.scale, place == kNear ? w[-(8 * g4 + e)] : bias);
                            s[4 * g4 + e] = exp2_of(__builtin_fmaf(t - lse[e], kLog2e, Held<T>::kShift));
                        }
                    }
                    if (__any(st[3 * kStat + 32 * m + l32] != 1.f)) {   // (rare; kept with the others, these take sixteen registers)
#pragma unroll
                        for (int g4 = 0; g4 < 4; ++g4) {
                            const f32x4 x = *reinterpret_cast<const f32x4*>(st + 3 * kStat + 32 * m + 8 * g4 + 4 * half);
#pragma unroll
                            for (int e = 0; e < 4; ++e) s[4 * g4 + e] *= x[e];
                        }
                    }
                } else {
                    const float c = a.scale * kLog2e, d = bias * kLog2e;
#pragma unroll
                    for (int g4 = 0; g4 < 4; ++g4) {
                        const f32x4 x = *reinterpret_cast<const f32x4*>(st + kStat + 32 * m + 8 * g4 + 4 * half);
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[4 * g4 + e] = exp2_of(__builtin_fmaf(s[4 * g4 + e], c, x[e] + d));
                    }
                }
                if (a.causal && r_hi > 0) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[e] = j <= p0 + row_of(e, half) ? s[e] : 0.f;
                }
#pragma unroll
                for (int g4 = 0; g4 < 4; ++g4) {
                    const f32x4 x = *reinterpret_cast<const f32x4*>(st + 2 * kStat + 32 * m + 8 * g4 + 4 * half);
#pragma unroll
                    for (int e = 0; e < 4; ++e) dp[4 * g4 + e] = s[4 * g4 + e] * __builtin_fmaf(dp[4 * g4 + e], Held<T>::kUnit, x[e]);
                }
                holder.hold(dp, dk);
                if constexpr (kWide) columns.start(turned);
                u32x4 wp{}, wd{};
                columns.products(turned, [&](int x, u32x4 w) {
                    const int step = x / (2 * Tile<DP>::kBlocks), d = x / 2 % Tile<DP>::kBlocks;
                    if (x % (2 * Tile<DP>::kBlocks) == 0) {
                        wp = weights_of<T>(s, step);
                        wd = weights_of<T>(dp, step);
                    }
                    if (x % 2 == 0)
                        dv[d] = mfma(w, wp, dv[d], T{});
                    else
                        dk[d] = mfma(w, wd, dk[d], T{});
                });
            }
            if constexpr (SHARED) {
                turn = turn == kTurns - 1 ? 0 : turn + 1;
            } else {
                wait_for_reads();
                wave_fence();
                if (n + 1 < to) request(n + 1, 0);
            }
        }
        wait_for<0>();   // (nothing may arrive in LDS that is no longer this workgroup's)
    }
    if (j >= a.k_tokens) return;
    holder.release(dk);
    if (j >= kl)   // (what was formed for a key that is not there)
#pragma unroll
        for (int d = 0; d < Tile<DP>::kBlocks; ++d) dk[d] = dv[d] = zero16();
    if (gr.parts > 1) {
        float* const sum = gr.sums + (((int64_t)part * heads + bh) * a.k_tokens + j) * 2 * DP;
        store_row32<DP>(sum, dk, half);
        store_row32<DP>(sum + DP, dv, half);
    } else {
        store_row<T, DP>(gr.out0.at<T>(b, hk) + (int64_t)j * gr.out0.token, dk, a.scale, a.head_dim, half);
        store_row<T, DP>(gr.out1.at<T>(b, hk) + (int64_t)j * gr.out1.token, dv, Held<T>::kUnit, a.head_dim, half);
    }
}

template <typename T, int DP> __global__ void __launch_bounds__(256, (DP == 32 ? 3 : DP == 64 ? 2 : 1)) keys_kernel(Args a, Grad gr, int k_tiles) { keys_of<T, DP, false>(a, gr, k_tiles, blockIdx.x); }

// Some workgroups take queries, the others keys, those with the longer way to go first (9 sequences of up to 1001, 32 heads of 80 sharing 8: keys first 250 us, queries first
// 350; 5001 causal tokens, 16 heads of 128 sharing 4, 444 and 412).  With either alone on the device, 2 x 810 causal tokens, 4 heads of 128, took 73 us where this takes
// 50, 16 sequences of up to 500, 12 heads of 64, 87 and 76, 5001 causal tokens 439 and 412.  The stats that both need come from a launch before.
template <typename T, int DP> __global__ void __launch_bounds__(256, 2) both_kernel(Args a, Grad queries, Grad keys, int q_tiles, int k_tiles, uint32_t first, int keys_first)
{
    const bool in_first = blockIdx.x < first;
    const uint32_t block = in_first ? blockIdx.x : blockIdx.x - first;
    if (in_first == (keys_first != 0))
        keys_of<T, DP, true>(a, keys, k_tiles, block);
    else
        queries_of<T, DP, true>(a, queries, q_tiles, block);
}
// Log2 of what the weights exp(s - lse) of a wavefront's eight queries from i0 on sum to (lane: query i0 + lane / 8), for rows of which lse does not tell.  Queries are columns
// eight at a time, four times over, keys rows of 32 straight from memory, and scores are formed step by step as queries_of forms them, so that both round alike.  Not fast, as such
// rows are few: where all are, 5001 causal tokens, 16 heads of 128 sharing 4, take 3.3 ms and not 0.47, 16 sequences of 500, 12 heads of 64, 0.53 and not 0.09.
template <typename T> __device__ __forceinline__ float row_sums(const Args& a, int b, int h, int i0, float lse_of_lane, int lane)
{
    const int half = lane >> 5, l32 = lane & 31, hk = h / a.group, ql = a.queries(b), kl = a.keys(b), i = i0 + (l32 & 7), p = kl - ql + i;
    const float lse = __shfl(lse_of_lane, 8 * (l32 & 7), kWave);
    const bool mine = i < ql;
    const T* const q = a.q.at<T>(b, h) + (int64_t)i * a.q.token;
    const int limit = a.causal ? (p + 1 < kl ? p + 1 : kl) : kl, last = i0 + 7 < ql ? i0 + 7 : ql - 1, end = a.causal ? (kl - ql + last + 1 < kl ? kl - ql + last + 1 : kl) : kl;
    float total = 0.f;
    for (int k0 = 0; k0 < end; k0 += 32) {
        const int j = k0 + l32;
        const T* const k = a.k.at<T>(b, hk) + (int64_t)j * a.k.token;
        floatx16 s = zero16();
        for (int d = 0; d < a.head_dim; d += 16) {
            const int at = d + 8 * half;
            u32x4 kf{0u, 0u, 0u, 0u}, qf{0u, 0u, 0u, 0u};
            if (at < a.head_dim && j < kl) kf = *reinterpret_cast<const u32x4*>(k + at);
            if (at < a.head_dim && mine) qf = *reinterpret_cast<const u32x4*>(q + at);
            s = mfma(kf, qf, s, T{});
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int key = k0 + row_of(e, half);
            if (key < limit) total += exp2_of((__builtin_fmaf(s[e], a.scale, a.table ? a.bias<T>(a.bucket(key - p), h) : 0.f) - lse) * kLog2e);
        }
    }
    total = sum_of_halves(total);
    return __builtin_amdgcn_logf(__shfl(total, lane >> 3, kWave));
}

// Eight threads per query, sixteen values of its row each.  Bound: memory, and of short sequences its launch (3 us).
template <typename T> __global__ void __launch_bounds__(256) stats_kernel(Args a, Grad gr)
{
    const int64_t heads = (int64_t)a.batch * a.q_heads;
    const int t = threadIdx.x & 7;
    for (int64_t item = (int64_t)blockIdx.x * 32 + (threadIdx.x >> 3); item < heads * gr.stat_rows; item += (int64_t)gridDim.x * 32) {   // (eight threads together)
        const int bh = (int)(item / gr.stat_rows), i = (int)(item % gr.stat_rows), b = bh / a.q_heads, h = bh % a.q_heads;
        float delta = 0.f, lse = ATT_INF, more = 0.f;
        if (i < a.queries(b)) {
            const T* const o = gr.o.at<T>(b, h) + (int64_t)i * gr.o.token;
            const T* const d = gr.dout.at<T>(b, h) + (int64_t)i * gr.dout.token;
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const int at = 64 * n + 8 * t;
                if (at >= a.head_dim) continue;
                const u32x4 x = *reinterpret_cast<const u32x4*>(o + at), y = *reinterpret_cast<const u32x4*>(d + at);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const f32x2 u = pair_to(x[w], T{}), v = pair_to(y[w], T{});
                    delta = __builtin_fmaf(u[0], v[0], delta);
                    delta = __builtin_fmaf(u[1], v[1], delta);
                }
            }
            lse = gr.lse[(int64_t)bh * a.q_tokens + i];
            lse = lse == -ATT_INF ? ATT_INF : lse;
        }
#pragma unroll
        for (int n = 1; n < 8; n <<= 1) delta += __shfl_xor(delta, n, kWave);
        const bool unknown = sums_unknown(lse);
        if (__any(unknown)) {   // (a wavefront's eight queries are of one head: stat_rows is a multiple of 32)
            const float sum = row_sums<T>(a, b, h, __builtin_amdgcn_readfirstlane(i), lse, threadIdx.x & 63);
            more = unknown ? sum : 0.f;
        }
        if (t == 0) leave_stats<T>(gr, heads, bh, i, lse, delta, more);
    }
}

// The parts of a key's (a query's) sums, four neighbouring values a thread.  Bound: memory (seven parts of 5001 x 4 x 256 floats: 23 us, 6.7 TB/s with what the caches hold).
template <typename T, int DP> __device__ __forceinline__ void keys_join(const Args& a, const Grad& gr, uint32_t block)
{
    const int64_t rows = (int64_t)a.batch * a.kv_heads * a.k_tokens, item = (int64_t)block * 256 + threadIdx.x;
    const int64_t row = item / (DP / 2);
    const int at = 4 * (int)(item % (DP / 2)), d = at % DP;
    if (row >= rows || d >= a.head_dim) return;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int n = 0; n < gr.parts; ++n) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(gr.sums + (n * rows + row) * 2 * DP + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += x[e];
    }
    const int j = (int)(row % a.k_tokens), bh = (int)(row / a.k_tokens), b = bh / a.kv_heads, hk = bh % a.kv_heads;
    const bool is_k = at < DP;
    const Heads& out = is_k ? gr.out0 : gr.out1;
    const float f = is_k ? a.scale : Held<T>::kUnit;
    *reinterpret_cast<u32x2*>(out.at<T>(b, hk) + (int64_t)j * out.token + d) = u32x2{pair_of(s[0] * f, s[1] * f, T{}), pair_of(s[2] * f, s[3] * f, T{})};
}

template <typename T, int DP> __device__ __forceinline__ void queries_join(const Args& a, const Grad& gr, uint32_t block)
{
    const int64_t rows = (int64_t)a.batch * a.q_heads * a.q_tokens, item = (int64_t)block * 256 + threadIdx.x;
    const int64_t row = item / (DP / 4);
    const int d = 4 * (int)(item % (DP / 4));
    if (row >= rows || d >= a.head_dim) return;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int n = 0; n < gr.parts; ++n) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(gr.sums + (n * rows + row) * DP + d);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += x[e];
    }
    const int i = (int)(row % a.q_tokens), bh = (int)(row / a.q_tokens), b = bh / a.q_heads, h = bh % a.q_heads;
    *reinterpret_cast<u32x2*>(gr.out0.at<T>(b, h) + (int64_t)i * gr.out0.token + d) =
        u32x2{pair_of(s[0] * a.scale, s[1] * a.scale, T{}), pair_of(s[2] * a.scale, s[3] * a.scale, T{})};
}

template <typename T, int DP> __global__ void __launch_bounds__(256) join_kernel(Args a, Grad queries, Grad keys, uint32_t q_blocks)
{
    if (blockIdx.x < q_blocks)
        queries_join<T, DP>(a, queries, blockIdx.x);
    else
        keys_join<T, DP>(a, keys, blockIdx.x - q_blocks);
}

// Diagonals of a head: 64 of them and 16 runs of workgroups.  (2048 workgroups, 1 head: 9 us.)
__global__ void __launch_bounds__(1024) diagonals_kernel(const float* __restrict__ diagonals, int parts, int heads, int width, float* __restrict__ sums)
{
    __shared__ float runs[16][64];
    const int n = blockIdx.x * 64 + (threadIdx.x & 63), run = threadIdx.x >> 6, h = blockIdx.y;
    const int each = (parts + 15) / 16, lo = run * each, hi = lo + each < parts ? lo + each : parts;
    float s = 0.f;
    if (n < width) {
#pragma unroll 8
        for (int p = lo; p < hi; ++p) s += diagonals[((int64_t)p * heads + h) * width + n];
    }
    runs[run][threadIdx.x & 63] = s;
    __syncthreads();
    if (run == 0 && n < width) {
#pragma unroll
        for (int r = 1; r < 16; ++r) s += runs[r][threadIdx.x & 63];
        sums[(int64_t)h * width + n] = s;
    }
}

// A workgroup per bucket and head: its distances' diagonals on either side and what lay beyond the window, over `parts` workgroups' sums (each wavefront
// a run of them).
template <typename T> __global__ void __launch_bounds__(256) buckets_kernel(Args a, const float* __restrict__ diagonals, int parts, T* __restrict__ dtable)
{
    __shared__ float runs[4];
    const Window window(a.left, a.right);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = blockIdx.y, n = blockIdx.x, width = window.size + 2;
    const bool right = a.two_sided && n > a.n_edges;
    const int e = right ? n - a.n_edges - 1 : n;
    const int near = e == 0 ? 0 : a.edges[e - 1];                         // distances near .. far - 1
    const int far = e == a.n_edges ? (1 << 30) : a.edges[e];
    // r = lo .. hi - 1; the first bucket of a one-sided table also has every r > 0, that of the right side begins at 1
    int lo = right ? (near > 1 ? near : 1) : 1 - far, hi = right ? far : e == 0 && !a.two_sided ? (1 << 30) : 1 - near;
    const int last = window.first + window.size;
    lo = (lo > window.first ? lo : window.first) - window.first;
    hi = (hi < last ? hi : last) - window.first;
    // tiles wholly at one end: one place each behind the window
    const bool left_end = !right && e == a.n_edges, right_end = a.two_sided ? right && e == a.n_edges : e == 0;
    const int each = (parts + 3) / 4, first = wave * each, end = first + each < parts ? first + each : parts;
    float s = 0.f;
    for (int at = lo + lane; at < hi; at += kWave) {
#pragma unroll 8
        for (int p = first; p < end; ++p) s += diagonals[((int64_t)p * a.q_heads + h) * width + at];
    }
    if ((lane == 0 && left_end) || (lane == 1 && right_end)) {
#pragma unroll 8
        for (int p = first; p < end; ++p) s += diagonals[((int64_t)p * a.q_heads + h) * width + window.size + lane];
    }
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) s += __shfl_xor(s, o, kWave);
    if (lane == 0) runs[wave] = s;
    __syncthreads();
    if (threadIdx.x == 0) dtable[(int64_t)n * a.q_heads + h] = (T)(((runs[0] + runs[1]) + runs[2]) + runs[3]);
}

constexpr int kOwnMost = 64;    // keys of a sequence that is one wavefront's own
constexpr int kFewParts = 64;   // workgroups whose diagonals the buckets' kernel adds itself (64 of them 5.7 us, by a launch of their own 4.9 and 4.8)
struct Plan {
    bool own, keys_first;
    int q_tiles, q_parts, q_part_keys, k_tiles, parts, diagonal_parts;
    size_t stats, diagonals, q_sums, sums, tables, total;   // bytes (sums: of the queries' parts and, q_sums further, of the keys')
};
Plan plan_of(const pruner_attention* a)
{
    Plan p{};
    const int dp = padded_dim(a->head_dim), group = a->q_heads / a->kv_heads;
    const bool causal = a->flags & PRUNER_ATTENTION_CAUSAL;
    // A workgroup's four wavefronts share tiles, or, where queries and keys are few, each has a sequence and head of its own (us in all, shared and own: 2048 sequences of 8 queries
    // and keys, 64 wide, 67 and 32; 783 of 6 and 55, 16 heads sharing two, 264 and 125, of 128 311 and 225; 200 of 20 and 60, 4 heads, 41 and 34, of 128 51 and 49;
    // 200 of 20 and 120 46 and 50).
    p.own = a->q_tokens <= 32 && a->k_tokens <= kOwnMost;
    p.q_tiles = (a->q_tokens + 127) / 128;
    const int tile_keys = p.own ? 32 : dp == 128 ? KeysShape<__bf16, 128, true>::kKeys : KeysShape<__bf16, 64, true>::kKeys;
    p.k_tiles = (a->k_tokens + tile_keys - 1) / tile_keys;
    p.q_parts = p.parts = 1;
    p.q_part_keys = a->k_tokens;
    const double rows = (double)a->batch * a->q_heads * a->q_tokens, keys = (double)a->batch * a->kv_heads * a->k_tokens;
    const double q_blocks = (double)a->batch * a->q_heads * p.q_tiles, k_blocks = (double)a->batch * a->kv_heads * p.k_tiles;
    const int held = 512;   // workgroups that the device has room for
    // (steps as measured: 5001 causal tokens, 16 heads of 128 sharing 4; 16 sequences of up to 500, 12 of 64)
    if (!p.own && rows > 0 && keys > 0) {
        const int step = dp < 128 ? 64 : 32;
        const int64_t q_chain = (a->k_tokens + step - 1) / step, k_chain = (int64_t)group * ((a->q_tokens + step - 1) / step);
        const double q_alone = dp == 128 ? 1.2 : dp == 64 ? 1.4 : 1.0, k_alone = dp == 128 ? 1.5 : dp == 64 ? 1.5 : 1.0;
        const double q_full = dp == 128 ? 1.9 : dp == 64 ? 2.4 : 1.8, k_full = dp == 128 ? 2.4 : dp == 64 ? 2.5 : 1.8, part = (causal ? 0.5 : 1.0) / held;
        const int parts = parts_of(q_blocks, q_chain, causal, held, q_alone, q_full, rows * dp * 4, k_blocks * (double)k_chain * part * k_full);
        p.q_part_keys = ((a->k_tokens + parts - 1) / parts + 63) / 64 * 64;
        p.q_parts = (a->k_tokens + p.q_part_keys - 1) / p.q_part_keys;
        p.parts = parts_of(k_blocks, k_chain, causal, held, k_alone, k_full, keys * 2 * dp * 4, q_blocks * (double)q_chain * part * q_full);
        p.keys_first = k_alone * (double)k_chain / p.parts > q_alone * (double)q_chain / p.q_parts;
    }
    // (the window for the largest edge that there can be: sizes alone decide)
    const int64_t reach = (int64_t)a->q_tokens + a->k_tokens;
    const int most = (int)(reach < PRUNER_MAX_BIAS_DISTANCE ? reach : PRUNER_MAX_BIAS_DISTANCE);
    const int widest = Window(most, a->flags & PRUNER_ATTENTION_TWO_SIDED ? (most > 1 ? most : 1) : 0).size + 2;
    p.diagonal_parts = p.own ? a->batch : a->batch * p.q_tiles * p.q_parts;
    p.stats = round_up((size_t)a->batch * a->q_heads * round_up((size_t)a->q_tokens, 32) * kStats * 4, 256);
    p.diagonals = a->table ? round_up((size_t)p.diagonal_parts * a->q_heads * widest * 4, 256) : 0;
    p.tables = a->table ? round_up((size_t)a->q_heads * widest * 4, 256) : 0;
    const size_t of_queries = p.q_parts > 1 ? (size_t)p.q_parts * (size_t)rows * dp * 4 : 0, of_keys = p.parts > 1 ? (size_t)p.parts * (size_t)keys * 2 * dp * 4 : 0;
    p.q_sums = round_up(of_queries, 256);
    p.sums = p.q_sums + round_up(of_keys, 256);
    p.total = p.stats + p.diagonals + p.tables + p.sums;
    return p;
}

struct Call {
    Args args;
    Grad queries, keys;
    Plan plan;
    float* table_sums;
    void* dtable;
    hipStream_t st;
};
template <typename T, int DP> int run(const Call& c)
{
    static PerDeviceFlag ready;
    const int dev = current_device(nullptr);
    if (dev < 0) return PRUNER_EHIP;
    if (!ready.get(dev)) {
        for (const void* fn : {reinterpret_cast<const void*>(&queries_kernel<T, DP>), reinterpret_cast<const void*>(&keys_kernel<T, DP>), reinterpret_cast<const void*>(&both_kernel<T, DP>)})
            if (hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) != hipSuccess) return PRUNER_EHIP;
        ready.mark(dev);
    }
    const Args& a = c.args;
    const Window w(a.left, a.right);
    const size_t window = a.table ? round_up((size_t)w.size, 4) * 4 : 0, skew = a.table ? kSkewFloats * 4 : 0;
    const int64_t q_heads = (int64_t)a.batch * a.q_heads, k_heads = (int64_t)a.batch * a.kv_heads;
    if (c.plan.own) {
        if (a.q_tokens > 0) {
            hipLaunchKernelGGL((queries_kernel<T, DP>), dim3((unsigned)((q_heads + 3) / 4)), dim3(256), 8 * window + (skew_in_values(DP, false) ? 0 : 4 * skew) + 4 * 2 * kOwn * DP * 2, c.st, a, c.queries);
            PRUNER_LAUNCH_CHECK();
        }
        if (a.k_tokens > 0) {
            typedef KeysShape<T, DP, false> Shape;
            hipLaunchKernelGGL((keys_kernel<T, DP>), dim3((unsigned)((k_heads * c.plan.k_tiles + Shape::kWaves - 1) / Shape::kWaves)), dim3(64 * Shape::kWaves),
                               Shape::kBytes + Shape::kWaves * window, c.st, a, c.keys, c.plan.k_tiles);
            PRUNER_LAUNCH_CHECK();
        }
    } else if (q_heads > 0) {
        typedef KeysShape<T, DP, true> Shape;
        static_assert(Shape::kWaves == 4, "workgroups of 256 threads");
        constexpr int kStep = DP < 128 ? 64 : 32;
        const size_t q_lds = 5 * window + 4 * skew + turns_of(DP, true, kStep) * 2 * kStep * DP * 2, k_lds = window + Shape::kBytes;
        const unsigned q_blocks = (unsigned)(q_heads * c.plan.q_tiles * c.plan.q_parts), k_blocks = (unsigned)(k_heads * c.plan.k_tiles * c.plan.parts);
        if (a.q_tokens > 0) {
            const int64_t need = (q_heads * c.queries.stat_rows + 31) / 32;
            hipLaunchKernelGGL(stats_kernel<T>, dim3((unsigned)(need < 65536 ? need : 65536)), dim3(256), 0, c.st, a, c.queries);
            PRUNER_LAUNCH_CHECK();
        }
        hipLaunchKernelGGL((both_kernel<T, DP>), dim3(q_blocks + k_blocks), dim3(256), q_lds > k_lds ? q_lds : k_lds, c.st, a, c.queries, c.keys, c.plan.q_tiles, c.plan.k_tiles,
                           c.plan.keys_first ? k_blocks : q_blocks, (int)c.plan.keys_first);
        PRUNER_LAUNCH_CHECK();
        const unsigned q_join = c.plan.q_parts > 1 ? (unsigned)((q_heads * a.q_tokens * (DP / 4) + 255) / 256) : 0, k_join = c.plan.parts > 1 ? (unsigned)((k_heads * a.k_tokens * (DP / 2) + 255) / 256) : 0;
        if (q_join + k_join > 0) {
            hipLaunchKernelGGL((join_kernel<T, DP>), dim3(q_join + k_join), dim3(256), 0, c.st, a, c.queries, c.keys, q_join);
            PRUNER_LAUNCH_CHECK();
        }
    }
    if (a.table) {
        const int width = w.size + 2, buckets = (a.n_edges + 1) * (a.two_sided ? 2 : 1);
        const float* from = c.queries.diagonals;
        int parts = a.q_tokens > 0 ? c.plan.diagonal_parts : 0;
        if (parts > kFewParts) {
            hipLaunchKernelGGL(diagonals_kernel, dim3((width + 63) / 64, a.q_heads), dim3(1024), 0, c.st, from, parts, a.q_heads, width, c.table_sums);
            PRUNER_LAUNCH_CHECK();
            from = c.table_sums;
            parts = 1;
        }
        hipLaunchKernelGGL(buckets_kernel<T>, dim3(buckets, a.q_heads), dim3(256), 0, c.st, a, from, parts, static_cast<T*>(c.dtable));
        PRUNER_LAUNCH_CHECK();
    }
    return PRUNER_OK;
}

bool grad_sizes_ok(const pruner_attention* a)
{
    if (!attention_sizes_ok(a)) return false;
    // (a launch takes queries and keys)
    return (int64_t)a->batch * a->q_heads * (a->q_tokens / 64 + 1) + (int64_t)a->batch * a->kv_heads * (a->k_tokens / 64 + 1) < (1 << 24) && a->q_heads <= 65535;
}

}  // namespace
}  // namespace att
}  // namespace pruner

using namespace pruner;

extern "C" size_t pruner_rel_attention_grad_workspace_bytes(const pruner_attention* a) { return att::grad_sizes_ok(a) ? att::plan_of(a).total : 0; }

extern "C" int pruner_rel_attention_grad(const pruner_attention* a, const pruner_heads* dout, const pruner_heads* q, const pruner_heads* k, const pruner_heads* v,
                                         const pruner_heads* o, const float* lse, const pruner_heads* dq, const pruner_heads* dk, const pruner_heads* dv, void* dtable,
                                         void* workspace, size_t workspace_bytes, void* stream)
{
    if (!att::grad_sizes_ok(a)) return PRUNER_EINVAL;
    if ((a->table != nullptr) != (dtable != nullptr) || (dtable && !aligned(dtable, 2))) return PRUNER_EINVAL;
    const pruner_heads none{nullptr, 0, 0, 0};
    const bool queries = a->batch > 0 && a->q_tokens > 0, keys = a->batch > 0 && a->k_tokens > 0;
    if (!queries) q = dout = o = dq = &none;
    if (!keys) k = v = dk = dv = &none;
    att::Call c{};
    const int rc = att::attention_args(a, q, k, v, &c.args);
    if (rc) return rc;
    if (queries && (!att::heads_ok(dout) || !att::heads_ok(o) || !att::heads_ok(dq) || !lse || !aligned(lse, 4))) return PRUNER_EINVAL;
    if (keys && (!att::heads_ok(dk) || !att::heads_ok(dv))) return PRUNER_EINVAL;
    c.plan = att::plan_of(a);
    if (c.plan.total > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < c.plan.total)) return PRUNER_EWORKSPACE;
    char* const ws = static_cast<char*>(workspace);
    att::Grad g{};
    g.dout = att::heads_of(dout);
    g.o = att::heads_of(o);
    g.lse = lse;
    g.stats = reinterpret_cast<float*>(ws);
    g.diagonals = reinterpret_cast<float*>(ws + c.plan.stats);
    c.table_sums = reinterpret_cast<float*>(ws + c.plan.stats + c.plan.diagonals);
    g.sums = reinterpret_cast<float*>(ws + c.plan.stats + c.plan.diagonals + c.plan.tables);
    g.part_keys = c.plan.q_part_keys;
    g.stat_rows = (int)round_up((size_t)a->q_tokens, 32);
    c.queries = c.keys = g;
    c.queries.parts = c.plan.q_parts;
    c.keys.parts = c.plan.parts;
    c.keys.sums = reinterpret_cast<float*>(reinterpret_cast<char*>(g.sums) + c.plan.q_sums);
    c.queries.out0 = att::heads_of(dq);
    c.keys.out0 = att::heads_of(dk);
    c.keys.out1 = att::heads_of(dv);
    c.dtable = dtable;
    c.st = static_cast<hipStream_t>(stream);
    if (a->batch == 0) {   // (no pair: a table's gradient is zero)
        c.args.batch = 0;
        c.args.q_tokens = c.args.k_tokens = 0;
    }
    const int dp = att::padded_dim(a->head_dim);
    if (a->dtype == PRUNER_BF16) return dp == 32 ? att::run<__bf16, 32>(c) : dp == 64 ? att::run<__bf16, 64>(c) : att::run<__bf16, 128>(c);
    return dp == 32 ? att::run<_Float16, 32>(c) : dp == 64 ? att::run<_Float16, 64>(c) : att::run<_Float16, 128>(c);
}
