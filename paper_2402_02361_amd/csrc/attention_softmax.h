// What kernels of attention that go over the keys once have in common: the running softmax of a query, and what its parts leave where the key axis is cut, by wavefronts that meet in LDS or by
// workgroups whose parts a later launch joins.
#pragma once
#include "rel_attention.h"

namespace pruner {
namespace att {
namespace {

constexpr float kSlack = 8.f;   // a running maximum may lag this far behind: weights stay below e^8, within binary16

// What a part of the key axis leaves per row: its weighted sum (binary32, unnormalised) and (maximum, sum).
struct Parts {
    float* sums;    // [part][row][DP]
    float2* stats;  // [part][row]
    int count, keys;   // parts, keys of a part (a multiple of 64)
};

// The running softmax of one query over 32-key blocks of scores.
template <typename T, int DP> struct Running {
    float m, l;
    floatx16 o[Tile<DP>::kBlocks];
    __device__ __forceinline__ void clear()
    {
        m = -ATT_INF;
        l = 0.f;
#pragma unroll
        for (int b = 0; b < Tile<DP>::kBlocks; ++b) o[b] = zero16();
    }
    // s: scores; where fused, scaled by `scale` and shifted by `bias` on the way, else they are what the softmax takes.  On return s holds the weights.
    template <int N> __device__ __forceinline__ void weigh(floatx16 (&s)[N], bool fused, float scale, float bias)
    {
        float top = s[0][0];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = __builtin_fmaxf(top, s[n][i]);
        top = max_of_halves(top);
        if (fused) top = __builtin_fmaf(top, scale, bias);
        if (__any(top > m + kSlack)) {   // (from minus infinity: any score)
            const float now = __builtin_fmaxf(m, top), factor = now == -ATT_INF ? 1.f : exp2_of((m - now) * kLog2e);
            m = now;
            l *= factor;
#pragma unroll
            for (int b = 0; b < Tile<DP>::kBlocks; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[b][i] *= factor;
        }
        const float from = m == -ATT_INF ? 0.f : m;   // (no key yet: every weight is exp(-infinity))
        float sum = 0.f;
        if (fused) {
            const float c = scale * kLog2e, d = (bias - from) * kLog2e;
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[n][i] = exp2_of(__builtin_fmaf(s[n][i], c, d));
                    sum += s[n][i];
                }
        } else {
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[n][i] = exp2_of((s[n][i] - from) * kLog2e);
                    sum += s[n][i];
                }
        }
        l += sum;
    }
};

__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.f ? -ATT_INF : __builtin_fmaf(__builtin_amdgcn_logf(l), kLn2, m); }   // (logf: base 2)

// Where a workgroup's four wavefronts, each of which has seen keys of its own for the same columns (query t of head hk * group + g is column t * group + g), leave what they have: a column's
// (maximum, sum), and its weighted sums in rows of DP + 4 floats, so that neighbouring rows lie in other banks.
template <int DP> struct Meeting {
    static constexpr int kStride = DP + 4;
    float2* stats;   // [4][32]
    float* sums;     // [4][columns][kStride]
    __device__ __forceinline__ explicit Meeting(char* lds) : stats(reinterpret_cast<float2*>(lds)), sums(reinterpret_cast<float*>(lds + 4 * 32 * 8)) {}
    static constexpr size_t bytes(int columns) { return 4 * 32 * 8 + (size_t)4 * columns * kStride * 4; }
    // The rows' results, or what this part leaves of them.
    template <typename T> __device__ __forceinline__ void join(const Args& a, const Heads& out, float* __restrict__ lse, const Parts& parts, int b, int hk, int part, int columns) const
    {
        for (int item = threadIdx.x; item < columns * (DP / 4); item += 256) {
            const int c = item / (DP / 4), d = 4 * (item % (DP / 4));
            if (d >= a.head_dim) continue;   // (whoever joins parts does not store these columns)
            float m = -ATT_INF;
#pragma unroll
            for (int w = 0; w < 4; ++w) m = __builtin_fmaxf(m, stats[w * 32 + c].y != 0.f ? stats[w * 32 + c].x : -ATT_INF);
            float total = 0.f;
            f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float2 st = stats[w * 32 + c];
                if (st.y == 0.f) continue;
                const float f = exp2_of((st.x - m) * kLog2e);
                total = __builtin_fmaf(f, st.y, total);
                const f32x4 x = *reinterpret_cast<const f32x4*>(sums + (w * columns + c) * kStride + d);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(f, x[e], o[e]);
            }
            const int tt = c / a.group, hh = hk * a.group + c % a.group;
            const int64_t row = ((int64_t)b * a.q_heads + hh) * a.q_tokens + tt;
            if (parts.count > 1) {
                const int64_t slot = (int64_t)part * a.batch * a.q_heads * a.q_tokens + row;
                *reinterpret_cast<f32x4*>(parts.sums + slot * DP + d) = o;
                if (d == 0) parts.stats[slot] = make_float2(m, total);
            } else {
                const float f = total != 0.f ? 1.f / total : 0.f;
                if (d < a.head_dim)
                    *reinterpret_cast<u32x2*>(out.at<T>(b, hh) + (int64_t)tt * out.token + d) = u32x2{pair_of(o[0] * f, o[1] * f, T{}), pair_of(o[2] * f, o[3] * f, T{})};
                if (lse && d == 0) lse[row] = lse_of(m, total);
            }
        }
    }
};

// What a wavefront of 32 columns leaves, and the joint result.  mine: this lane's column has a query.
template <typename T, int DP>
__device__ __forceinline__ void meet(const Running<T, DP>& run, char* lds, const Args& a, const Heads& out, float* __restrict__ lse, const Parts& parts, int b, int hk, int part, int columns, bool mine)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), half = lane >> 5, l32 = lane & 31;
    const Meeting<DP> at(lds);
    __syncthreads();
    const float l = sum_of_halves(run.l);
    if (half == 0) at.stats[wave * 32 + l32] = make_float2(run.m, mine ? l : 0.f);
    if (l32 < columns) store_row32<DP>(at.sums + (wave * columns + l32) * Meeting<DP>::kStride, run.o, half);
    __syncthreads();
    at.template join<T>(a, out, lse, parts, b, hk, part, columns);
}

}  // namespace
}  // namespace att
}  // namespace pruner
