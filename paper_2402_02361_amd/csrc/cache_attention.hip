// Attention over keys and values held in 8 bits in pages: pruner_rel_attention's formulas with k^ = code 2^e, v^ = code 2^e.
//
// S^T = K Q^T and O^T += V^T P^T on v_mfma_f32_32x32x16, as where keys are of 16 bits.  Codes go from memory straight to the lanes whose operands they become: which
// key a row of the first product's operand is, is ours to choose, and with row 8 q + 4 half + j being key 16 half + 4 q + j of 32, a lane's sixteen scores are of
// sixteen neighbouring keys, the depth that its sixteen bytes of values have.  The page's powers of two go in with the conversion.
// The columns of a wavefront are 32 pairs of a query and a head that share a key head: query t of the group's head g is column t * group + g.
//   tokens_kernel   at most 32 columns: the four wavefronts of a workgroup take 64 keys each in turn, and meet at the end
//   chunk_kernel    more: 32 columns each
#include "attention_softmax.h"
#include "cache.h"

namespace pruner {
namespace att {
namespace {

constexpr int kTile = 64;   // keys of a step

// 64 keys' codes on their way to a wavefront: two blocks of 32.  Rows past the sequence's end, or whose page is not there, hold anything; of values they are cleared
// before use (their weight is 0, but anything may be a NaN).
template <typename T, int DP> struct Codes {
    static constexpr int kChunks = DP / 32;
    u32x4 k[2][kChunks], v[2][kChunks];
    float k_scale[2], v_scale[2];
    int k_page[2], v_page[2], there[2];   // there: tokens of this lane's sixteen
    __device__ __forceinline__ static int key_of(int lane) { return ((lane >> 2 & 1) << 4) | ((lane >> 3 & 3) << 2) | (lane & 3); }   // this lane's row of the keys' operand
    __device__ __forceinline__ void find(const cache::Cache& c, int b, int key0, int kl, int lane)
    {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int at = key0 + 32 * n + key_of(lane), first = key0 + 32 * n + 16 * (lane >> 5);
            k_page[n] = at < kl ? c.page_of(b, at) : -1;
            v_page[n] = first < kl ? c.page_of(b, first) : -1;
        }
    }
    __device__ __forceinline__ void load_keys(const cache::Cache& c, int h, int key0, int lane)
    {
        const int half = lane >> 5, units = c.head_dim / cache::kUnit;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int64_t head = c.head_of(k_page[n] < 0 ? 0 : k_page[n], h);
            const uint8_t* const p = c.k + head * c.page_bytes() + (((key0 + 32 * n + key_of(lane)) & (c.page_tokens() - 1)) << 4);
            k_scale[n] = cache::two_to(c.k_exps[head]);
#pragma unroll
            for (int i = 0; i < kChunks; ++i) {
                const int unit = 2 * i + half < units ? 2 * i + half : units - 1;   // (past the last one: the query's columns are 0 there)
                k[n][i] = *reinterpret_cast<const u32x4*>(p + ((int64_t)unit << (c.shift + 4)));
            }
        }
    }
    __device__ __forceinline__ void load_values(const cache::Cache& c, int h, int key0, int kl, int lane)
    {
        const int half = lane >> 5, l32 = lane & 31;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int first = key0 + 32 * n + 16 * half, left = kl - first;
            there[n] = v_page[n] < 0 ? 0 : left < 16 ? left : 16;
            const int64_t head = c.head_of(v_page[n] < 0 ? 0 : v_page[n], h);
            const uint8_t* const p = c.v + head * c.page_bytes() + ((int64_t)((first & (c.page_tokens() - 1)) >> 4) * c.head_dim << 4);
            v_scale[n] = cache::two_to(c.v_exps[head]);
#pragma unroll
            for (int i = 0; i < kChunks; ++i) {
                const int d = 32 * i + l32 < c.head_dim ? 32 * i + l32 : c.head_dim - 1;   // (columns past the last are not stored)
                v[n][i] = *reinterpret_cast<const u32x4*>(p + (d << 4));
            }
        }
    }
    __device__ __forceinline__ void clear_values()   // those that are not there
    {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int bytes = there[n] - 4 * w;
                const uint32_t keep = bytes >= 4 ? ~0u : bytes <= 0 ? 0u : (1u << (8 * bytes)) - 1u;
#pragma unroll
                for (int i = 0; i < kChunks; ++i) v[n][i][w] &= keep;
            }
    }
    __device__ __forceinline__ void scores(floatx16 (&s)[2], const u32x4 (&q)[2 * kChunks]) const
    {
#pragma unroll
        for (int n = 0; n < 2; ++n) s[n] = zero16();
#pragma unroll
        for (int i = 0; i < kChunks; ++i)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int n = 0; n < 2; ++n) s[n] = mfma(cache::eight_from<T>(k[n][i][2 * u], k[n][i][2 * u + 1], k_scale[n]), q[2 * i + u], s[n], T{});
    }
    __device__ __forceinline__ void add(floatx16 (&o)[kChunks], const floatx16 (&s)[2]) const
    {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const u32x4 w = weights_of<T>(s[n], u);
#pragma unroll
                for (int i = 0; i < kChunks; ++i) o[i] = mfma(cache::eight_from<T>(v[n][i][2 * u], v[n][i][2 * u + 1], v_scale[n]), w, o[i], T{});
            }
    }
};

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

// One step: scores with bias and mask, weights, their sums of values; the next step's codes are asked for as soon as these are used.
template <typename T, int DP>
__device__ __forceinline__ void step(Running<T, DP>& run, Codes<T, DP>& codes, const u32x4 (&qf)[DP / 16], const Args& a, const cache::Cache& c, const Columns& at, const char* lds,
                                     const BiasLds& places, const Window& window, float bias_left, float bias_right, int b, int hk, int ql, int kl, int key0, int next, int after, int end, int lane)
{
    const int half = lane >> 5;
    floatx16 s[2];
    codes.scores(s, qf);
    int there[2] = {codes.there[0], codes.there[1]};
    const bool short_of = __any(there[0] < 16 || there[1] < 16);
    if (short_of) codes.clear_values();
    if (next < end) codes.load_keys(c, hk, next, lane);
    const int r_lo = key0 - (kl - ql + at.q_last), r_hi = key0 + kTile - 1 - (kl - ql + at.q_first);
    const int place = a.table ? place_of(a, r_lo, r_hi) : kLeft;
    const float bias = place == kRight ? bias_right : bias_left;
    bool fused = true;
    if (place == kNear) {
        const uint8_t* const n = reinterpret_cast<const uint8_t*>(lds + places.biases) + (key0 - at.p - window.first + 16 * half);
        const float* const of = reinterpret_cast<const float*>(lds) + at.bias;
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
            const int seen = at.limit - (key0 + 32 * x + 16 * half), left = seen < there[x] ? seen : there[x];
#pragma unroll
            for (int i = 0; i < 16; ++i) s[x][i] = i < left ? s[x][i] : -ATT_INF;
        }
    run.weigh(s, fused, a.scale, bias);
    codes.add(run.o, s);
    if (next < end) {
        codes.load_values(c, hk, next, kl, lane);
        codes.find(c, b, after, after < end ? kl : 0, lane);
    }
}

template <typename T, int DP> __device__ __forceinline__ void load_query(u32x4 (&f)[DP / 16], const Args& a, int b, const Columns& at, int half)
{
    const T* const p = a.q.at<T>(b, at.h) + (int64_t)at.t * a.q.token;
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) {
        const int d = 32 * (i / 2) + 16 * half + 8 * (i % 2);
        f[i] = u32x4{0u, 0u, 0u, 0u};
        if (at.mine && d < a.head_dim) f[i] = *reinterpret_cast<const u32x4*>(p + d);
    }
}

template <typename T, int DP> __global__ void __launch_bounds__(256, 2) tokens_kernel(Args a, cache::Cache c, Heads out, float* __restrict__ lse, Parts parts)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), half = lane >> 5;
    const int columns = a.q_tokens * a.group;
    const int hk = blockIdx.x % a.kv_heads, part = blockIdx.x / a.kv_heads % parts.count, b = blockIdx.x / a.kv_heads / parts.count;
    const int ql = a.queries(b), kl = a.keys(b);
    Columns at;
    at.set(a, hk, 0, 0, columns, ql, kl, lane);
    const Window window(a.left, a.right);
    const BiasLds places(a);
    int end = ql == 0 ? 0 : kl;   // (the last query sees all keys under the causal mask too)
    const int begin = part * parts.keys;
    if (parts.count > 1) end = end < begin + parts.keys ? end : begin + parts.keys;

    Running<T, DP> run;
    run.clear();
    if (begin < end) {
        constexpr int kStep = 4 * kTile;
        int key0 = begin + kTile * wave;
        Codes<T, DP> codes;
        codes.find(c, b, key0, key0 < end ? kl : 0, lane);
        u32x4 qf[DP / 16];
        load_query<T, DP>(qf, a, b, at, half);
        if (key0 < end) {
            codes.load_keys(c, hk, key0, lane);
            codes.load_values(c, hk, key0, kl, lane);
            codes.find(c, b, key0 + kStep, key0 + kStep < end ? kl : 0, lane);
        }
        float bias_left = 0.f, bias_right = 0.f;
        if (a.table) {
            bias_left = a.bias<T>(a.n_edges, at.h);
            bias_right = a.bias<T>(a.two_sided ? 2 * a.n_edges + 1 : 0, at.h);
            if (kl - ql - (end + kTile) < a.left) places.fill<T>(a, window, lds, hk, 0);   // (else all of this part's keys lie beyond the last edge)
        }
        __syncthreads();
        for (; key0 < end; key0 += kStep)
            step<T, DP>(run, codes, qf, a, c, at, lds, places, window, bias_left, bias_right, b, hk, ql, kl, key0, key0 + kStep, key0 + 2 * kStep, end, lane);
    }
    meet<T, DP>(run, lds, a, out, lse, parts, b, hk, part, columns, at.mine);
}

template <typename T, int DP> __global__ void __launch_bounds__(256, 2) chunk_kernel(Args a, cache::Cache c, Heads out, float* __restrict__ lse, Parts parts, int tiles)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), half = lane >> 5;
    const int columns = a.q_tokens * a.group;
    const Item it = item_of(blockIdx.x, (uint32_t)a.batch * a.kv_heads, 1, (uint32_t)tiles * parts.count);
    const int b = it.head / a.kv_heads, hk = it.head % a.kv_heads, part = it.tile % parts.count, first = it.tile / parts.count * 128 + 32 * wave;
    const int ql = a.queries(b), kl = a.keys(b);
    Columns at;
    at.set(a, hk, first - 32 * wave, first < columns ? first : columns - 1, columns, ql, kl, lane);
    if (first >= columns) at.mine = false;
    const Window window(a.left, a.right);
    const BiasLds places(a);
    // the keys that this wavefront's queries see, and of them this part's
    int end = first >= columns || at.q_first >= ql ? 0 : a.causal ? kl - ql + at.q_last + 1 : kl;
    end = end < kl ? end : kl;
    const int begin = part * parts.keys;
    if (parts.count > 1) end = end < begin + parts.keys ? end : begin + parts.keys;

    float bias_left = 0.f, bias_right = 0.f;
    if (a.table) {
        bias_left = a.bias<T>(a.n_edges, at.h);
        bias_right = a.bias<T>(a.two_sided ? 2 * a.n_edges + 1 : 0, at.h);
        places.fill<T>(a, window, lds, hk, first - 32 * wave);
        __syncthreads();
    }
    Running<T, DP> run;
    run.clear();
    if (begin < end) {
        Codes<T, DP> codes;
        codes.find(c, b, begin, kl, lane);
        u32x4 qf[DP / 16];
        load_query<T, DP>(qf, a, b, at, half);
        codes.load_keys(c, hk, begin, lane);
        codes.load_values(c, hk, begin, kl, lane);
        codes.find(c, b, begin + kTile, begin + kTile < end ? kl : 0, lane);
        for (int key0 = begin; key0 < end; key0 += kTile)
            step<T, DP>(run, codes, qf, a, c, at, lds, places, window, bias_left, bias_right, b, hk, ql, kl, key0, key0 + kTile, key0 + 2 * kTile, end, lane);
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

// Which kernel, and into how many parts the keys are cut.
struct Plan {
    bool tokens;
    int tiles, parts, part_keys;
    int64_t rows;
    size_t workspace;
};
constexpr int64_t kEnough = 4096;   // workgroups that fill the device where all they do is read, and their sequences' lengths differ
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
            const int fewest = 512;
            parts = (kEnough + groups - 1) / groups;
            const int64_t most = ((int64_t)a->k_tokens + fewest - 1) / fewest;
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

template <typename T, int DP> int run(const Args& args, const cache::Cache& c, const Plan& plan, const Heads& out, float* lse, void* workspace, hipStream_t st)
{
    static PerDeviceFlag ready;
    int dev = current_device(nullptr);
    if (dev < 0) return PRUNER_EHIP;
    if (!ready.get(dev)) {
        for (const void* fn : {reinterpret_cast<const void*>(&tokens_kernel<T, DP>), reinterpret_cast<const void*>(&chunk_kernel<T, DP>)})
            if (hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) != hipSuccess) return PRUNER_EHIP;
        ready.mark(dev);
    }
    Parts parts{nullptr, nullptr, plan.parts, plan.part_keys};
    if (plan.parts > 1) {
        parts.stats = static_cast<float2*>(workspace);
        parts.sums = reinterpret_cast<float*>(static_cast<char*>(workspace) + round_up((size_t)plan.parts * plan.rows * 8, 256));
    }
    const size_t biases = (size_t)BiasLds(args).bytes();
    const int64_t key_heads = (int64_t)args.batch * args.kv_heads;
    if (plan.tokens) {
        const size_t columns = (size_t)args.q_tokens * args.group, last = 4 * 32 * 8 + 4 * columns * (DP + 4) * 4;
        hipLaunchKernelGGL((tokens_kernel<T, DP>), dim3((unsigned)(key_heads * plan.parts)), dim3(256), last > biases ? last : biases, st, args, c, out, lse, parts);
    } else {
        hipLaunchKernelGGL((chunk_kernel<T, DP>), dim3((unsigned)(key_heads * plan.tiles * plan.parts)), dim3(256), biases, st, args, c, out, lse, parts, plan.tiles);
    }
    PRUNER_LAUNCH_CHECK();
    if (plan.parts > 1) {
        hipLaunchKernelGGL((join_kernel<T, DP>), dim3((unsigned)((plan.rows * (DP / 4) + 255) / 256)), dim3(256), 0, st, args, out, lse, parts);
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
