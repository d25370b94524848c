// The norm behind one block and the norm before the next with the gate and the residual scale between them, and its gradients:
//     z1 = norm(f), u = z1 w_post;   h = alpha x + s u, s = sigmoid(gate);   z2 = norm(h), y = z2 w_pre
//     norm(v) = (v - m) r, r = 1 / sqrt(mean((v - m)^2) + eps), m = mean(v) or 0
// Backward, with <.> the mean over a row and N(d, z, r) = r (d - [<d>] - z <d z>) (the middle term with the mean only):
//     dH = dh + N(dy w_pre, z2, r2);   dx = alpha dH;   dgate = dH u s (1 - s);   df = N(dH s w_post, z1, r1)
//     dw_pre = sum over rows of dy z2;   dw_post = sum over rows of dH s z1;   without a norm after (no y): dH = dh
// A row lives in the registers of T threads, eight neighbouring values each, T the power of two that covers it, or beyond 64 the whole wavefronts that do: every matrix is
// read once and written once, and the statistics are formed again in the backward pass, where they cost no bytes.
// All in binary32.  Bound: memory: 65536 x 2048 bfloat16 rows' gradients 411 us, 4.9 TB/s, 65536 x 256 49 us, 5.2 TB/s; forward, 16384 x 1100 binary32 rows 64 us, 4.5 TB/s.  A
// large copy reaches 5.2.  Rows of more than 64 threads wait for each other's sums: gradients over 16384 x 4096 rows 248 us (4.1 TB/s), over 8192 x 8192, where a thread
// has 128 registers, 400 (2.5); rows that begin anywhere cost selections: over 16384 x 1111 rows 129 us, where 1112 take 86.
#include "checkpoint.h"

namespace pruner {
namespace {

using namespace ckpt;

constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ float sigmoid(float g) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-g * kLog2e)); }

// Sums over the T threads of a row, N of them at once, the same bits in all of them.  T a power of two in 4..64, or whole wavefronts; the wavefronts of a
// row of more than 64 threads meet in LDS (two places in turn, so one barrier is enough).
template <int CTRL> __device__ __forceinline__ float moved(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
struct RowSum {
    float (*meet)[16][2];   // [2][16 wavefronts][N <= 2]
    int threads, slot, turn;   // slot: which of the workgroup's rows
    template <int N> __device__ __forceinline__ void of(float (&v)[N])
    {
        // by moves inside the vector unit: pairs, fours, eights and sixteens of a row of 16 lanes, rows, halves
#pragma unroll
        for (int n = 0; n < N; ++n) {
            v[n] += moved<0xB1>(v[n]);                        // quad_perm 1,0,3,2
            v[n] += moved<0x4E>(v[n]);                        // quad_perm 2,3,0,1
            if (threads >= 8) v[n] += moved<0x141>(v[n]);     // row_half_mirror: the other four of eight
            if (threads >= 16) v[n] += moved<0x140>(v[n]);    // row_mirror: the other eight of sixteen
            if (threads >= 32) {
                const TwoFloats t = across_rows(v[n]);
                v[n] = t.a + t.b;
            }
            if (threads >= 64) {
                const TwoFloats t = across_halves(v[n]);
                v[n] = t.a + t.b;
            }
        }
        if (threads <= kWave) return;
        const int wave = threadIdx.x >> 6, waves = threads >> 6, first = slot * waves;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int n = 0; n < N; ++n) meet[turn][wave][n] = v[n];
        __syncthreads();
        // (a lane per wavefront, at most 16, then as above: read one after the other: gradients over 16384 x 4096 rows 341 us where this takes 248, 5000 x 5000
        // 184 and 124)
        const int at = threadIdx.x & 15;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            v[n] = at < waves ? meet[turn][first + at][n] : 0.f;
            v[n] += moved<0xB1>(v[n]);
            v[n] += moved<0x4E>(v[n]);
            v[n] += moved<0x141>(v[n]);
            v[n] += moved<0x140>(v[n]);
        }
        turn ^= 1;
    }
};

// 1 / sqrt(x), also where x is below the smallest normal number, which the instruction takes for 0 (rows of values below 1e-19 and eps of 0).
__device__ __forceinline__ float inverse_root(float x)
{
    const bool tiny = x < 0x1p-126f;
    float r = __builtin_amdgcn_rsqf(x);
    if (__any(tiny)) r = tiny ? __builtin_amdgcn_rsqf(x * 0x1p64f) * 0x1p32f : r;   // (a selection for all rows: gradients over 8192 x 8192 rows 466 us where this takes 401)
    return r;
}

// z <- norm(v) over a row, of which `left` values begin here (those past its end are 0 and stay 0); returns r.  Where accesses take all eight values (V = 8)
// a thread has all of them or none.
template <int V>
__device__ __forceinline__ float normalise(RowSum& sum, const float (&v)[kEach], float (&z)[kEach], int left, float per_dim, bool center, float eps)
{
    float m = 0.f;
    if (center) {
        float s[1] = {((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]))};
        sum.of(s);
        m = left > 0 ? s[0] * per_dim : 0.f;
    }
    float q[1] = {0.f};
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        z[j] = V == 8 || j < left ? v[j] - m : 0.f;
        q[0] = __builtin_fmaf(z[j], z[j], q[0]);
    }
    sum.of(q);
    const float of_row = inverse_root(__builtin_fmaf(q[0], per_dim, eps)), r = left > 0 ? of_row : 0.f;   // (it may be infinite where eps is 0)
#pragma unroll
    for (int j = 0; j < kEach; ++j) z[j] = V == 8 || j < left ? z[j] * r : 0.f;
    return r;
}

// d <- r (d - [<d>] - z <d z>)
template <int V>
__device__ __forceinline__ void back(RowSum& sum, float (&d)[kEach], const float (&z)[kEach], float r, int left, float per_dim, bool center)
{
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        s[0] = __builtin_fmaf(d[j], z[j], s[0]);
        s[1] += d[j];
    }
    sum.of(s);
    const float a = s[0] * per_dim, b = center ? s[1] * per_dim : 0.f;
#pragma unroll
    for (int j = 0; j < kEach; ++j) d[j] = V == 8 || j < left ? r * __builtin_fmaf(-z[j], a, d[j] - b) : 0.f;   // (r is 0 where nothing is left)
}

__device__ __forceinline__ void load_vector(const float* __restrict__ p, int col, int left, float (&v)[kEach])
{
#pragma unroll
    for (int j = 0; j < kEach; ++j) v[j] = p && j < left ? p[col + j] : 0.f;
}

struct Norm {
    int64_t rows;
    int dim, threads, center;
    float alpha, eps, per_dim;
    const float *w_post, *w_pre;
    const void* gate;
    int64_t gate_pitch;
};

// GATE_ROWS: the gate is a matrix; else one for all rows, or none (known here because a gate's rows take 16 registers in binary32 and with them a workgroup per
// unit: a call on 16384 x 1100 rows with one gate takes 74 us where this takes 70, 65536 x 256 without a gate 33 and 31; 5000 x 5000 in binary16 45 and 55).
template <typename T, int V, int BLOCK, bool GATE_ROWS>
__global__ void __launch_bounds__(BLOCK) norm_kernel(Norm p, const T* __restrict__ x, int64_t x_pitch, const T* __restrict__ f, int64_t f_pitch, T* __restrict__ h,
                                                    T* __restrict__ y, int8_t* __restrict__ codes, uint8_t* __restrict__ exps)
{
    __shared__ float meet[2][16][2];
    const int in_block = (int)blockDim.x / p.threads, slot = (int)threadIdx.x / p.threads, t = (int)threadIdx.x - slot * p.threads;
    RowSum sum{meet, p.threads, slot, 0};
    const int col = 8 * t, left = p.dim - col;
    float w_post[kEach], w_pre[kEach];   // (w_post: with the gate that all rows share)
    load_vector(p.w_post, col, left, w_post);
    load_vector(p.w_pre, col, left, w_pre);
    if (!GATE_ROWS && p.gate) {
        float g[kEach];
        load_vector(static_cast<const float*>(p.gate), col, left, g);
#pragma unroll
        for (int j = 0; j < kEach; ++j) w_post[j] *= sigmoid(g[j]);
    }
    const int64_t stride = (int64_t)gridDim.x * in_block;
    Eight<T, V> xin, fin, gin, x_next, f_next, g_next;   // the next row's values are on their way while a row is worked on
    auto fetch = [&](int64_t row) {
        const int some = row < p.rows ? left : 0;
        const int64_t after = p.rows - 1 - row;
        x_next.load(x + row * x_pitch + col, some, room_of(after, x_pitch, left, row * x_pitch + col));
        if (f) f_next.load(f + row * f_pitch + col, some, room_of(after, f_pitch, left, row * f_pitch + col));
        if constexpr (GATE_ROWS) g_next.load(static_cast<const T*>(p.gate) + row * p.gate_pitch + col, some, room_of(after, p.gate_pitch, left, row * p.gate_pitch + col));
    };
    fetch((int64_t)blockIdx.x * in_block + slot);
    for (int64_t first = (int64_t)blockIdx.x * in_block; first < p.rows; first += stride) {
        // (threads past the last row go through the same steps on zeros: the wavefront's exchanges and the barriers need them)
        const int64_t row = first + slot;
        const int mine = row < p.rows ? left : 0;
        xin = x_next;
        fin = f_next;
        gin = g_next;
        fetch(row + stride);
        float v[kEach], z[kEach];
        xin.to_floats(v);
#pragma unroll
        for (int j = 0; j < kEach; ++j) v[j] *= p.alpha;
        if (f) {
            float u[kEach], g[kEach];
            fin.to_floats(u);
            normalise<V>(sum, u, z, mine, p.per_dim, p.center, p.eps);
            if constexpr (GATE_ROWS) gin.to_floats(g);
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                if constexpr (GATE_ROWS)
                    v[j] = __builtin_fmaf(sigmoid(g[j]), z[j] * w_post[j], v[j]);
                else
                    v[j] = __builtin_fmaf(z[j], w_post[j], v[j]);
            }
        }
        Eight<T, V> out;
        if (h) {
            out.from_floats(v);
            out.store(h + row * p.dim + col, mine);
        }
        if (!y && !codes) continue;
        normalise<V>(sum, v, z, mine, p.per_dim, p.center, p.eps);
#pragma unroll
        for (int j = 0; j < kEach; ++j) z[j] *= w_pre[j];
        out.from_floats(z);
        if (y) out.store(y + row * p.dim + col, mine);
        if (codes) {
            out.to_floats(z);   // the checkpoint is that of y as it is stored
            EightCodes<V> packed;
            const uint32_t byte = pack_group(z, packed.w);
            packed.store(codes + row * p.dim + col, mine);
            if ((t & 3) == 0 && mine > 0) exps[row * ((p.dim + kGroup - 1) / kGroup) + t / 4] = (uint8_t)byte;
        }
    }
}

// sums: [3][dim] of every workgroup (dw_post, dw_pre, dgate of one gate for all rows)
// VECTOR: the gate is one for all rows.  Y: there is a norm after (asked for in the kernel this took 65536 x 2048 rows 421 us where it takes 400, and 8192 x 8192 319 and 400).
template <typename T, int V, int BLOCK, bool VECTOR, bool Y>
__global__ void __launch_bounds__(BLOCK) norm_grad_kernel(Norm p, const T* __restrict__ dh, int64_t dh_pitch, const T* __restrict__ dy, int64_t dy_pitch,
                                                         const T* __restrict__ x, int64_t x_pitch, const T* __restrict__ f, int64_t f_pitch,
                                                         const int8_t* __restrict__ codes, const uint8_t* __restrict__ exps, T* __restrict__ dx, T* __restrict__ df,
                                                         T* __restrict__ dgate, float* __restrict__ sums)
{
    __shared__ float meet[2][16][2];
    __shared__ float fold[256 * kEach];
    const int in_block = (int)blockDim.x / p.threads, slot = (int)threadIdx.x / p.threads, t = (int)threadIdx.x - slot * p.threads;
    RowSum sum{meet, p.threads, slot, 0};
    const int col = 8 * t, left = p.dim - col;
    const bool gate_rows = !VECTOR && p.gate;
    const bool has_f = f || codes;
    const int groups = (p.dim + kGroup - 1) / kGroup;
    float w_post[kEach], w_pre[kEach], s_all[kEach], sum_post[kEach], sum_pre[kEach], sum_gate[kEach];
    load_vector(p.w_post, col, left, w_post);
    load_vector(p.w_pre, col, left, w_pre);
    if constexpr (VECTOR) load_vector(static_cast<const float*>(p.gate), col, left, s_all);
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        s_all[j] = VECTOR ? sigmoid(s_all[j]) : 1.f;
        sum_post[j] = sum_pre[j] = sum_gate[j] = 0.f;
    }
    const int64_t stride = (int64_t)gridDim.x * in_block;
    struct Row {
        Eight<T, V> x, f, g, dh, dy;
        EightCodes<V> c;
        uint32_t byte;
    } now, next;
    auto fetch = [&](int64_t row) {
        const int some = row < p.rows ? left : 0;
        const int64_t after = p.rows - 1 - row;
        if constexpr (Y) {   // (x stands only in what the norm after sees)
            next.x.load(x + row * x_pitch + col, some, room_of(after, x_pitch, left, row * x_pitch + col));
            next.dy.load(dy + row * dy_pitch + col, some, room_of(after, dy_pitch, left, row * dy_pitch + col));
        }
        if (f) next.f.load(f + row * f_pitch + col, some, room_of(after, f_pitch, left, row * f_pitch + col));
        if (codes) {
            next.c.load(codes + row * p.dim + col, some, room_of(after, p.dim, left, row * p.dim + col));
            next.byte = some > 0 ? exps[row * groups + t / 4] : 1u;
        }
        if (gate_rows) next.g.load(static_cast<const T*>(p.gate) + row * p.gate_pitch + col, some, room_of(after, p.gate_pitch, left, row * p.gate_pitch + col));
        if (dh) next.dh.load(dh + row * dh_pitch + col, some, room_of(after, dh_pitch, left, row * dh_pitch + col));
    };
    fetch((int64_t)blockIdx.x * in_block + slot);
    for (int64_t first = (int64_t)blockIdx.x * in_block; first < p.rows; first += stride) {
        const int64_t row = first + slot;
        const int mine = row < p.rows ? left : 0;
        now = next;
        fetch(row + stride);
        float v[kEach], z1[kEach], z2[kEach], s[kEach], d[kEach], w[kEach];
        float r1 = 0.f;
        now.x.to_floats(v);
#pragma unroll
        for (int j = 0; j < kEach; ++j) v[j] *= p.alpha;
        if (has_f) {
            if (codes)
                restore_eight(now.c.w, now.byte, w, mine);
            else
                now.f.to_floats(w);
            r1 = normalise<V>(sum, w, z1, mine, p.per_dim, p.center, p.eps);
            if (gate_rows) {
                now.g.to_floats(s);
#pragma unroll
                for (int j = 0; j < kEach; ++j) s[j] = sigmoid(s[j]);
            } else {
#pragma unroll
                for (int j = 0; j < kEach; ++j) s[j] = s_all[j];
            }
#pragma unroll
            for (int j = 0; j < kEach; ++j) v[j] = __builtin_fmaf(s[j], z1[j] * w_post[j], v[j]);
        }
        if constexpr (Y) {
            const float r2 = normalise<V>(sum, v, z2, mine, p.per_dim, p.center, p.eps);
            now.dy.to_floats(d);
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                sum_pre[j] = __builtin_fmaf(d[j], z2[j], sum_pre[j]);
                d[j] *= w_pre[j];
            }
            back<V>(sum, d, z2, r2, mine, p.per_dim, p.center);
            if (dh) {
                now.dh.to_floats(w);
#pragma unroll
                for (int j = 0; j < kEach; ++j) d[j] += w[j];
            }
        } else {
            now.dh.to_floats(d);
        }
        Eight<T, V> out;
#pragma unroll
        for (int j = 0; j < kEach; ++j) w[j] = p.alpha * d[j];
        out.from_floats(w);
        out.store(dx + row * p.dim + col, mine);
        if (!has_f) continue;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            d[j] *= s[j];
            w[j] = d[j] * z1[j];
            sum_post[j] += w[j];
            d[j] *= w_post[j];
        }
        if (VECTOR || gate_rows) {   // dgate = dH u s (1 - s)
#pragma unroll
            for (int j = 0; j < kEach; ++j) w[j] *= w_post[j] * (1.f - s[j]);
            if constexpr (VECTOR) {
#pragma unroll
                for (int j = 0; j < kEach; ++j) sum_gate[j] += w[j];
            } else {
                out.from_floats(w);
                out.store(dgate + row * p.dim + col, mine);
            }
        }
        back<V>(sum, d, z1, r1, mine, p.per_dim, p.center);
        out.from_floats(d);
        out.store(df + row * p.dim + col, mine);
    }
    // the workgroup's rows side by side, one after the other
    auto leave = [&](float (&mine)[kEach], float* to) {
        if (in_block > 1) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kEach; ++j) fold[threadIdx.x * kEach + j] = mine[j];
            __syncthreads();
            if (slot == 0)
                for (int o = 1; o < in_block; ++o)
#pragma unroll
                    for (int j = 0; j < kEach; ++j) mine[j] += fold[(o * p.threads + t) * kEach + j];
        }
        if (slot == 0)
#pragma unroll
            for (int j = 0; j < kEach; ++j)
                if (j < left) to[col + j] = mine[j];
    };
    float* const to = sums + (int64_t)blockIdx.x * 3 * p.dim;
    if constexpr (Y) leave(sum_pre, to + p.dim);
    if (has_f) {
        leave(sum_post, to);
        if constexpr (VECTOR) leave(sum_gate, to + 2 * p.dim);
    }
}

// The workgroups' sums, added in their order: 32 columns and 32 runs of workgroups per workgroup.
__global__ void __launch_bounds__(1024) norm_sums_kernel(const float* __restrict__ sums, int parts, int dim, float* __restrict__ dw_post, float* __restrict__ dw_pre,
                                                         float* __restrict__ dgate)
{
    __shared__ float runs[32][33];
    const int which = blockIdx.y, col = blockIdx.x * 32 + (threadIdx.x & 31), run = threadIdx.x >> 5;
    float* const out = which == 0 ? dw_post : which == 1 ? dw_pre : dgate;
    if (!out) return;
    const int each = (parts + 31) / 32, lo = run * each, hi = lo + each < parts ? lo + each : parts;
    float s = 0.f;
    if (col < dim) {
#pragma unroll 8
        for (int i = lo; i < hi; ++i) s += sums[((int64_t)i * 3 + which) * dim + col];
    }
    runs[run][threadIdx.x & 31] = s;
    __syncthreads();
    if (run == 0 && col < dim) {
#pragma unroll
        for (int r = 1; r < 32; ++r) s += runs[r][threadIdx.x & 31];
        out[col] = s;
    }
}

int row_threads(int32_t dim)   // threads per row
{
    int t = 4;
    while (8 * t < dim && t < kWave) t *= 2;
    return 8 * t < dim ? (dim + 8 * kWave - 1) / (8 * kWave) * kWave : t;
}
struct Shape {
    int threads, block, blocks;
};
constexpr int64_t kMaxParts = 2048;   // of the backward pass, for its workspace: more than a device of 256 units holds (768 of 256 threads)
Shape shape_of(int64_t rows, int32_t dim, int64_t most_blocks)
{
    // (workgroups of 128, 256 and 512 threads, us a call: gradients over 20000 x 1024 rows 78, 75, 90, over 40000 x 256 40, 38, 38; forward 46, 44, 44 and 23, 22, 23)
    const int t = row_threads(dim), block = t <= 128 ? 256 : t;
    const int64_t need = (rows + block / t - 1) / (block / t);
    return Shape{t, block, (int)(need < most_blocks ? need : most_blocks)};
}

bool norm_ok(const pruner_norm* p)
{
    const float big = 3.0e38f;
    return p && type_known(p->dtype) && p->rows >= 0 && p->dim >= 1 && p->dim <= PRUNER_MAX_NORM_DIM && p->rows < (1ll << 40) / p->dim && p->alpha >= -big && p->alpha <= big &&
           p->eps >= 0.f && p->eps <= big && p->gate_pitch >= 0 && (p->gate_pitch == 0 || !p->gate || p->gate_pitch >= p->dim);
}
bool matrix_ok(const void* m, int64_t pitch, const pruner_norm* p)
{
    return m && pitch >= p->dim && pitch < (1ll << 40) && aligned(m, type_bytes(p->dtype));
}
bool vector_ok(const float* v) { return v && aligned(v, 4); }
bool gate_ok(const pruner_norm* p) { return !p->gate || (p->gate_pitch ? matrix_ok(p->gate, p->gate_pitch, p) : aligned(p->gate, 4)); }
bool kept_ok(const pruner_checkpoint* c) { return c->codes && c->exps && aligned(c->codes, 8); }

Norm norm_of(const pruner_norm* p, int threads)
{
    return Norm{p->rows, p->dim, threads, p->center != 0, p->alpha, p->eps, 1.f / (float)p->dim, p->w_post, p->w_pre, p->gate, p->gate_pitch};
}

// Workgroups of a kernel that the current device holds at once: as many are started, each takes its rows in turn (1024 where 768 fit: the last quarter ran alone,
// 531 us over 65536 x 2048 rows where this takes 427).
struct Held {
    int of[kMaxDevices] = {};
    int64_t get(const void* kernel, int block, int64_t most)
    {
        int cus = 0, each = 0;
        const int dev = current_device(&cus);
        if (dev < 0) return -1;
        if (dev < kMaxDevices && of[dev]) return of[dev] < most ? of[dev] : most;
        if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&each, kernel, block, 0) != hipSuccess || each < 1) return -1;
        if (dev < kMaxDevices) of[dev] = each * cus;
        return (int64_t)each * cus < most ? (int64_t)each * cus : most;
    }
};

template <typename T, int V>
int run_norm(const pruner_norm* p, const Shape& s, const void* x, int64_t x_pitch, const void* f, int64_t f_pitch, void* h, void* y, const pruner_checkpoint* kept, hipStream_t st)
{
    const bool rows = p->gate && p->gate_pitch;
    static Held held[2][17];   // by wavefronts of a workgroup
    auto* const kernel = s.block > 256 ? (rows ? &norm_kernel<T, V, 1024, true> : &norm_kernel<T, V, 1024, false>) : (rows ? &norm_kernel<T, V, 256, true> : &norm_kernel<T, V, 256, false>);
    const int64_t blocks = held[rows][s.block / kWave].get(reinterpret_cast<const void*>(kernel), s.block, s.blocks);
    if (blocks < 0) return PRUNER_EHIP;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(s.block), 0, st, norm_of(p, s.threads), static_cast<const T*>(x), x_pitch, static_cast<const T*>(f), f_pitch,
                       static_cast<T*>(h), static_cast<T*>(y), kept ? kept->codes : nullptr, kept ? kept->exps : nullptr);
    PRUNER_LAUNCH_CHECK();
    return PRUNER_OK;
}

template <typename T, int V>
int run_norm_grad(const pruner_norm* p, const Shape& s, const void* dh, int64_t dh_pitch, const void* dy, int64_t dy_pitch, const void* x, int64_t x_pitch, const void* f,
                  int64_t f_pitch, const pruner_checkpoint* kept, void* dx, void* df, void* dgate, float* sums, int* parts, hipStream_t st)
{
    const bool vector = p->gate && !p->gate_pitch, has_y = p->w_pre;
    auto* const kernel = !has_y          ? (vector ? &norm_grad_kernel<T, V, 1024, true, false> : &norm_grad_kernel<T, V, 1024, false, false>)   // (128 registers are enough)
                         : s.block > 512 ? (vector ? &norm_grad_kernel<T, V, 1024, true, true> : &norm_grad_kernel<T, V, 1024, false, true>)
                         : s.block > 256 ? (vector ? &norm_grad_kernel<T, V, 512, true, true> : &norm_grad_kernel<T, V, 512, false, true>)
                                         : (vector ? &norm_grad_kernel<T, V, 256, true, true> : &norm_grad_kernel<T, V, 256, false, true>);
    static Held held[2][2][17];
    const int64_t blocks = held[has_y][vector][s.block / kWave].get(reinterpret_cast<const void*>(kernel), s.block, s.blocks);
    if (blocks < 0) return PRUNER_EHIP;
    *parts = (int)blocks;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(s.block), 0, st, norm_of(p, s.threads), static_cast<const T*>(dh), dh_pitch, static_cast<const T*>(dy),
                       dy_pitch, static_cast<const T*>(x), x_pitch, static_cast<const T*>(f), f_pitch, kept ? kept->codes : nullptr, kept ? kept->exps : nullptr,
                       static_cast<T*>(dx), static_cast<T*>(df), static_cast<T*>(dgate), sums);
    PRUNER_LAUNCH_CHECK();
    return PRUNER_OK;
}

}  // namespace
}  // namespace pruner

using namespace pruner;

extern "C" int pruner_gated_norm(const pruner_norm* p, const void* x, int64_t x_pitch, const void* f, int64_t f_pitch, void* h, void* y, const pruner_checkpoint* kept_y,
                                 void* stream)
{
    if (!norm_ok(p)) return PRUNER_EINVAL;
    if (p->rows == 0) return PRUNER_OK;
    const size_t bytes = type_bytes(p->dtype);
    if (!matrix_ok(x, x_pitch, p) || (f && !matrix_ok(f, f_pitch, p)) || (f && !vector_ok(p->w_post)) || !gate_ok(p)) return PRUNER_EINVAL;
    if ((h && !aligned(h, bytes)) || (y && !aligned(y, bytes)) || (kept_y && !kept_ok(kept_y)) || ((y || kept_y) && !vector_ok(p->w_pre))) return PRUNER_EINVAL;
    if (!h && !y && !kept_y) return PRUNER_EINVAL;
    Access a;
    a.fits(x, bytes, x_pitch);
    a.fits(f, bytes, f_pitch);
    if (p->gate_pitch) a.fits(p->gate, bytes, p->gate_pitch);
    a.fits(h, bytes, p->dim);
    a.fits(y, bytes, p->dim);
    if (kept_y) a.fits(kept_y->codes, 1, p->dim);
    const Shape s = shape_of(p->rows, p->dim, 1 << 22);
    return BY_TYPE_AND_ACCESS(p->dtype, a.v, run_norm, p, s, x, x_pitch, f, f_pitch, h, y, kept_y, static_cast<hipStream_t>(stream));
}

extern "C" size_t pruner_gated_norm_grad_workspace_bytes(int64_t rows, int32_t dim)
{
    if (rows <= 0 || dim < 1 || dim > PRUNER_MAX_NORM_DIM) return 0;
    return round_up((size_t)shape_of(rows, dim, kMaxParts).blocks * 3 * (size_t)dim * 4, 256);
}

extern "C" int pruner_gated_norm_grad(const pruner_norm* p, const void* dh, int64_t dh_pitch, const void* dy, int64_t dy_pitch, const void* x, int64_t x_pitch, const void* f,
                                      int64_t f_pitch, const pruner_checkpoint* kept_f, void* dx, void* df, void* dgate, float* dw_post, float* dw_pre, void* workspace,
                                      size_t workspace_bytes, void* stream)
{
    if (!norm_ok(p) || (f && kept_f)) return PRUNER_EINVAL;
    const bool has_f = f || kept_f || (p->rows == 0 && dw_post);   // (a matrix without rows may have no address: its sums are zero)
    const bool has_y = p->w_pre != nullptr;
    if (has_y ? !vector_ok(dw_pre) || !vector_ok(p->w_pre) : dw_pre || dy || (p->rows > 0 && !dh)) return PRUNER_EINVAL;
    if (has_f && (!vector_ok(dw_post) || !vector_ok(p->w_post))) return PRUNER_EINVAL;
    const size_t bytes = type_bytes(p->dtype);
    const bool gate_rows = has_f && p->gate && p->gate_pitch, gate_vector = has_f && p->gate && !p->gate_pitch;
    if (has_f && p->gate && (!dgate || !aligned(dgate, gate_vector ? 4 : bytes))) return PRUNER_EINVAL;
    if (p->rows > 0) {
        if (!matrix_ok(x, x_pitch, p) || (has_y && !matrix_ok(dy, dy_pitch, p)) || (dh && !matrix_ok(dh, dh_pitch, p)) || (f && !matrix_ok(f, f_pitch, p)) || (kept_f && !kept_ok(kept_f)) ||
            !gate_ok(p))
            return PRUNER_EINVAL;
        if (!dx || !aligned(dx, bytes) || (has_f && (!df || !aligned(df, bytes)))) return PRUNER_EINVAL;
        if (!workspace || !aligned(workspace, 256) || workspace_bytes < pruner_gated_norm_grad_workspace_bytes(p->rows, p->dim)) return PRUNER_EWORKSPACE;
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    float* const sums = static_cast<float*>(workspace);
    int parts = 0;
    if (p->rows > 0) {
        Access a;
        a.fits(x, bytes, x_pitch);
        a.fits(dy, bytes, dy_pitch);
        a.fits(dh, bytes, dh_pitch);
        a.fits(f, bytes, f_pitch);
        if (gate_rows) a.fits(p->gate, bytes, p->gate_pitch);
        if (gate_rows) a.fits(dgate, bytes, p->dim);
        if (kept_f) a.fits(kept_f->codes, 1, p->dim);
        a.fits(dx, bytes, p->dim);
        a.fits(df, bytes, p->dim);
        Norm n = norm_of(p, 0);
        if (!has_f) n.gate = nullptr;
        const Shape s = shape_of(p->rows, p->dim, kMaxParts);
        const pruner_norm q{p->rows, p->dim, p->dtype, p->center, p->alpha, p->eps, p->w_post, p->w_pre, n.gate, p->gate_pitch};
        const int rc = BY_TYPE_AND_ACCESS(p->dtype, a.v, run_norm_grad, &q, s, dh, dh_pitch, dy, dy_pitch, x, x_pitch, f, f_pitch, kept_f, dx, df, gate_rows ? dgate : nullptr, sums, &parts, st);
        if (rc) return rc;
    }
    hipLaunchKernelGGL(norm_sums_kernel, dim3((p->dim + 31) / 32, 3), dim3(1024), 0, st, sums, parts, p->dim, has_f ? dw_post : nullptr, dw_pre,
                       gate_vector ? static_cast<float*>(dgate) : nullptr);
    PRUNER_LAUNCH_CHECK();
    return PRUNER_OK;
}
