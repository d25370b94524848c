// Checkpoints of activations in 8 bits (pack, restore) and a linear layer's weight gradient from its input's checkpoint.
#include "checkpoint.h"
#include "mfma_tile.h"

namespace pruner {
namespace {

using namespace ckpt;

// n / d for n below 2^31 and 1 <= d < 2^31, by a multiplication (Granlund and Montgomery, Division by invariant integers using multiplication, 1994): q = (hi(n m) + n) >> s with m = floor(2^32 (2^s - d) / d) + 1, s = ceil(log2 d).
struct Divisor {
    uint32_t d, m, s;
    explicit Divisor(uint32_t by) : d(by), m(0), s(0)
    {
        while ((1ull << s) < d) ++s;
        m = (uint32_t)(((1ull << 32) * ((1ull << s) - d)) / d + 1);
    }
    __device__ __forceinline__ uint32_t of(uint32_t n) const { return (__umulhi(n, m) + n) >> s; }
};

// A thread takes eight neighbouring values; four threads make a group.  Bound: memory (each value read once, a little over a byte written; restored the other
// way round): 8191 x 1100 binary32 rows packed and restored in 18.6 us, 4.9 TB/s.
template <typename T, int V>
__global__ void __launch_bounds__(256) pack_kernel(const T* __restrict__ x, int64_t pitch, int64_t rows, int dim, uint32_t items, Divisor per_row, int8_t* __restrict__ codes,
                                                   uint8_t* __restrict__ exps)
{
    const uint32_t item = blockIdx.x * 256 + threadIdx.x;   // (items is a multiple of 4: the lanes of a group are active together)
    if (item >= items) return;
    const uint32_t row = per_row.of(item), at = item - row * per_row.d;
    const int col = 8 * (int)at, left = dim - col;
    Eight<T, V> in;
    in.load(x + (int64_t)row * pitch + col, left, room_of(rows - 1 - row, pitch, left, (int64_t)row * pitch + col));
    float v[kEach];
    in.to_floats(v);
    EightCodes<V> out;
    const uint32_t byte = pack_group(v, out.w);
    out.store(codes + (int64_t)row * dim + col, left);
    if ((at & 3u) == 0) exps[(int64_t)row * (per_row.d / 4) + at / 4] = (uint8_t)byte;
}

template <typename T, int V>
__global__ void __launch_bounds__(256) restore_kernel(const int8_t* __restrict__ codes, const uint8_t* __restrict__ exps, int64_t rows, int dim, uint32_t items, Divisor per_row,
                                                      T* __restrict__ x, int64_t pitch)
{
    const uint32_t item = blockIdx.x * 256 + threadIdx.x;
    if (item >= items) return;
    const uint32_t row = per_row.of(item), at = item - row * per_row.d;
    const int col = 8 * (int)at, left = dim - col;
    EightCodes<V> in;
    in.load(codes + (int64_t)row * dim + col, left, room_of(rows - 1 - row, dim, left, (int64_t)row * dim + col));
    float v[kEach];
    restore_eight(in.w, exps[(int64_t)row * (per_row.d / 4) + at / 4], v);
    Eight<T, V> out;
    out.from_floats(v);
    out.store(x + (int64_t)row * pitch + col, left);
}

// ---- the weight gradient: dW[n][k] = sum_r dy[r][n] x^[r][k] -------------------------------------------------------------
// A matrix product whose depth is the rows, which is the outer index of both operands: tiles of 64 rows lie in LDS as they lie in memory
// (x^ restored to dy's type on the way, exactly), and ds_read_b64_tr_b16 hands them to v_mfma_f32_32x32x16 turned over.  That read takes, per 16
// lanes, four rows of 16 columns (lane t the 8 bytes at row t / 4, column 4 (t % 4)) and gives lane t column t of them.
// A workgroup of four wavefronts owns 128 x 128 of dW, a wavefront 64 x 64; or, where there are enough of these for the device, one of eight owns 256 x 256, a
// wavefront 64 x 128.  What bounds it is LDS: a wavefront's 16 rows take 4 KB of reads for four products of 32 x 32 (128 cycles, in which
// LDS hands out 16 KB to four wavefronts), or 6 KB for eight: 2048 x 1024 over 65536 rows in 262 us, 1.05 PFLOP/s (a large matrix product: 1.445).  Where the tiles of dW are too few for the device, the rows are cut into
// parts whose sums go to the workspace and are added in their order.

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
using tile::bf16x8;
using tile::floatx16;

__device__ __forceinline__ floatx16 mfma(u32x4 a, u32x4 b, floatx16 c, __bf16)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ floatx16 mfma(u32x4 a, u32x4 b, floatx16 c, _Float16)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

constexpr int kTileR = 64;
template <bool BIG> struct WgradShape {
    static constexpr int kSide = BIG ? 256 : 128, kThreads = 2 * kSide;
    static constexpr int kChunks = kSide / 8, kRowBytes = 2 * kSide, kTileBytes = kTileR * kRowBytes;   // a tile of either operand: rows of kSide values of 16 bits
    static constexpr int kRowStep = kThreads / kChunks, kEach = kTileR / kRowStep;                      // 16-byte chunks of a tile per thread
    static constexpr int kN = 2, kK = BIG ? 4 : 2;                                                      // blocks of 32 of a wavefront
    // Where a row's 16-byte chunk lies: chunks are permuted row by row so that neither the writes (16 lanes, one row) nor the turning reads (four
    // rows of 64 bytes at once) meet in a bank.
    __device__ __forceinline__ static int chunk_at(int row, int chunk) { return row * kRowBytes + ((chunk ^ (((row & 3) << 2) | ((row >> 2) & 3))) << 4); }
};

struct WgradPlan {
    bool big;
    int tiles_n, tiles_k, parts;
    int64_t rows_each;   // rows of a part, a multiple of kTileR
};
// Small or large tiles and how many parts, by what they cost (microseconds): a start, the steps of 64 rows that the busiest unit goes through in turn, and the parts'
// sums read again (at 4 TB/s, by one more launch).  A step as measured where workgroups are alone on their units and, of the small ones, two share one;
// rows that begin anywhere take longer.  (Kernel and join, large and small: 2048 x 1024 over 65536 rows 273 and 386; 512 x 512 55 and 64; 4096 x 4096 over 2048 rows
// 73 and 99; 1024 x 1024 over 8192 rows 42 and 39.  Parts: 1600 x 904 over 30000 rows nine, 252 workgroups, 116, ten, 280 workgroups, 170; 44 x 16 over 1885 rows
// four 26, fifteen 17.)
WgradPlan wgrad_plan(int64_t rows, int32_t n_out, int32_t dim)
{
    const bool loose = n_out % 8 || dim % 8;
    const int64_t chain = (rows + kTileR - 1) / kTileR;
    const double part_us = (double)n_out * dim * 4 / 4e6;
    WgradPlan best{};
    double least = 0;
    for (int big = 0; big < 2; ++big) {
        WgradPlan p;
        const int side = big ? 256 : 128;
        p.big = big;
        p.tiles_n = (n_out + side - 1) / side;
        p.tiles_k = (dim + side - 1) / side;
        const int64_t tiles = (int64_t)p.tiles_n * p.tiles_k;
        const double alone = big ? (loose ? 4.2 : 2.1) : loose ? 2.5 : 1.05, full = loose ? 3.3 : 1.5;
        for (int64_t parts = 1; parts == 1 || (parts <= chain && parts <= 512); parts += parts < 16 ? 1 : parts / 8) {
            const int64_t steps = (chain + parts - 1) / parts, blocks = tiles * parts, units = big || blocks <= 256 ? 256 : 512;
            const double us = 7.0 + (double)((blocks + units - 1) / units * steps) * (units == 256 ? alone : full) + (parts > 1 ? 8.0 + (double)parts * (part_us + 0.06) : 0.0);
            if ((big || parts > 1) && us >= least) continue;
            least = us;
            best = p;
            best.rows_each = (steps > 0 ? steps : 1) * kTileR;
        }
    }
    best.parts = (int)((rows + best.rows_each - 1) / best.rows_each);
    if (best.parts < 1) best.parts = 1;
    return best;
}

template <typename T, int V, bool BIG>
__global__ void __launch_bounds__(WgradShape<BIG>::kThreads, 2) wgrad_kernel(const T* __restrict__ dy, int64_t dy_pitch, const int8_t* __restrict__ codes, const uint8_t* __restrict__ exps,
                                                       int64_t rows, int n_out, int dim, WgradPlan plan, float* __restrict__ out, int accumulate)
{
    typedef WgradShape<BIG> S;
    constexpr int kSide = S::kSide, kEach_ = S::kEach;
    extern __shared__ __attribute__((aligned(16))) char lds[];   // [turn][dy, x^] tiles
    // workgroups go to the eight dies in turn: each takes a run of the tiles, part by part, so that a part's rows stay in its cache
    const uint32_t total = gridDim.x, die = blockIdx.x & 7, in_die = blockIdx.x >> 3, whole = total >> 3, extra = total & 7;
    const uint32_t id = die * whole + (die < extra ? die : extra) + in_die;
    const uint32_t tiles = (uint32_t)plan.tiles_n * plan.tiles_k, part = id / tiles, tile_id = id % tiles;
    const int n0 = (int)(tile_id / plan.tiles_k) * kSide, k0 = (int)(tile_id % plan.tiles_k) * kSide;
    const int64_t r_begin = (int64_t)part * plan.rows_each, r_end = r_begin + plan.rows_each < rows ? r_begin + plan.rows_each : rows;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, l32 = lane & 31;
    const int groups = (dim + kGroup - 1) / kGroup;

    const int s_row = threadIdx.x / S::kChunks, s_chunk = threadIdx.x % S::kChunks;   // this thread's chunks: rows s_row + kRowStep u
    const int n_left = n_out - (n0 + 8 * s_chunk), k_left = dim - (k0 + 8 * s_chunk);
    Eight<T, V> dy_in[kEach_];
    EightCodes<V> x_in[kEach_];
    uint32_t x_exp[kEach_];
    // One of a thread's chunks of the tile from r0.  Accesses of all eight values are bounds-checked buffer loads: what is beyond the part's rows or the
    // matrix's columns arrives as zeros (an exponent byte of 0 restores as 0), and so does a tile beyond the part.
    auto fetch = [&](int u, int64_t r0) {
        if constexpr (V == 8) {
            const int64_t rows_left = r_end - r0;
            const int n_rows = rows_left < 0 ? 0 : rows_left < kTileR ? (int)rows_left : kTileR;
            auto from = [&](const void* base, int64_t row_bytes, int width) {
                return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(base) + r0 * row_bytes), 0, n_rows > 0 ? (n_rows - 1) * (int)row_bytes + width : 0,
                                                         0x00027000);
            };
            const uint32_t row = (uint32_t)(s_row + S::kRowStep * u), none = 0x80000000u;
            const u32x4 d = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(from(dy, dy_pitch * 2, n_out * 2),
                                                                                           (int)(n_left > 0 ? row * (uint32_t)(dy_pitch * 2) + 2u * (uint32_t)(n0 + 8 * s_chunk) : none), 0, 0));
            const u32x2 c = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(from(codes, dim, dim), (int)(k_left > 0 ? row * (uint32_t)dim + (uint32_t)(k0 + 8 * s_chunk) : none), 0, 0));
            x_exp[u] = __builtin_amdgcn_raw_buffer_load_b8(from(exps, groups, groups), (int)(k_left > 0 ? row * (uint32_t)groups + (uint32_t)((k0 >> 5) + (s_chunk >> 2)) : none), 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) dy_in[u].w[i] = d[i];
            x_in[u].w[0] = c[0];
            x_in[u].w[1] = c[1];
        } else {
            const int64_t r = r0 + s_row + S::kRowStep * u;
            const bool in = r < r_end;
            // (columns past the matrix's may hold anything: their results are not kept)
            const int n_room = room_of(rows - 1 - r, dy_pitch, n_left, r * dy_pitch + n0 + 8 * s_chunk), k_room = room_of(rows - 1 - r, dim, k_left, r * dim + k0 + 8 * s_chunk);
            dy_in[u].load(dy + r * dy_pitch + n0 + 8 * s_chunk, in && n_left > 0 ? (n_room >= 8 ? 8 : n_left) : 0, n_room);
            x_in[u].load(codes + r * dim + k0 + 8 * s_chunk, in && k_left > 0 ? (k_room >= 8 ? 8 : k_left) : 0, k_room);
            x_exp[u] = in && k_left > 0 ? exps[r * groups + (k0 >> 5) + (s_chunk >> 2)] : 0u;
        }
    };
    auto park = [&](int u, int turn) {
        const int at = S::chunk_at(s_row + S::kRowStep * u, s_chunk);
        *reinterpret_cast<u32x4*>(lds + 2 * turn * S::kTileBytes + at) = u32x4{dy_in[u].w[0], dy_in[u].w[1], dy_in[u].w[2], dy_in[u].w[3]};
        float v[kEach];
        restore_eight(x_in[u].w, x_exp[u], v);
        Eight<T, 8> x;
        x.from_floats(v);
        *reinterpret_cast<u32x4*>(lds + (2 * turn + 1) * S::kTileBytes + at) = u32x4{x.w[0], x.w[1], x.w[2], x.w[3]};
    };
    // this lane's places in a tile: block of 32 columns, four rows q of the eight of its half
    const int wn = S::kN * (wave >> 1), wk = S::kK * (wave & 1), t = lane & 15, g = (lane >> 4) & 1;
    int at_n[S::kN][2], at_k[S::kK][2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int row = 8 * half + 4 * q + (t >> 2), within = 2 * g + ((t >> 1) & 1);
#pragma unroll
        for (int b = 0; b < S::kN; ++b) at_n[b][q] = S::chunk_at(row, 4 * (wn + b) + within) + 8 * (t & 1);
#pragma unroll
        for (int b = 0; b < S::kK; ++b) at_k[b][q] = S::chunk_at(row, 4 * (wk + b) + within) + 8 * (t & 1);
    }
    auto turned = [&](const char* p, const int (&at)[2], int step) {
        typedef __attribute__((address_space(3))) i16x4* lds_ptr;
        const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + at[0] + step * 16 * S::kRowBytes));
        const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + at[1] + step * 16 * S::kRowBytes));
        const u32x2 lo = __builtin_bit_cast(u32x2, a), hi = __builtin_bit_cast(u32x2, b);
        return u32x4{lo[0], lo[1], hi[0], hi[1]};
    };

    floatx16 acc[S::kN][S::kK];
#pragma unroll
    for (int a = 0; a < S::kN; ++a)
#pragma unroll
        for (int b = 0; b < S::kK; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.f;
    if (r_begin < r_end) {
        // In iteration i the products of tile i run between the parking of tile i + 1, whose values have arrived since the iteration before, and the requests for tile
        // i + 2: a chunk of each per step of 16 rows, so that the matrix cores work while codes are restored (all of it after the products: 330 us
        // for 2048 x 1024 over 65536 rows, where this takes 258).
        static_assert(kEach_ == kTileR / 16, "a chunk per step");
#pragma unroll
        for (int u = 0; u < kEach_; ++u) fetch(u, r_begin);
#pragma unroll
        for (int u = 0; u < kEach_; ++u) {
            park(u, 0);
            fetch(u, r_begin + kTileR);
        }
        int turn = 0;
        for (int64_t r0 = r_begin; r0 < r_end; r0 += kTileR, turn ^= 1) {
            __syncthreads();
#pragma unroll
            for (int step = 0; step < kTileR / 16; ++step) {
                u32x4 fn[S::kN], fk[S::kK];
#pragma unroll
                for (int b = 0; b < S::kN; ++b) fn[b] = turned(lds + 2 * turn * S::kTileBytes, at_n[b], step);
#pragma unroll
                for (int b = 0; b < S::kK; ++b) fk[b] = turned(lds + (2 * turn + 1) * S::kTileBytes, at_k[b], step);
#pragma unroll
                for (int a = 0; a < S::kN; ++a)
#pragma unroll
                    for (int b = 0; b < S::kK; ++b) acc[a][b] = mfma(fn[a], fk[b], acc[a][b], T{});
                park(step, turn ^ 1);
                fetch(step, r0 + 2 * kTileR);
            }
        }
    }
    float* const to = out + (plan.parts > 1 ? (int64_t)part * n_out * dim : 0);
#pragma unroll
    for (int a = 0; a < S::kN; ++a)
#pragma unroll
        for (int b = 0; b < S::kK; ++b) {
            const int k = k0 + 32 * (wk + b) + l32;
            if (k >= dim) continue;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int n = n0 + 32 * (wn + a) + 8 * (i / 4) + 4 * half + i % 4;
                if (n >= n_out) continue;
                float* const p = to + (int64_t)n * dim + k;
                *p = accumulate && plan.parts == 1 ? *p + acc[a][b][i] : acc[a][b][i];
            }
        }
}

// dW (+)= the parts, one after the other; four neighbouring values a thread where all is aligned for it.
template <int V>
__global__ void __launch_bounds__(256) wgrad_join_kernel(const float* __restrict__ parts, int n_parts, int64_t n, float* __restrict__ dw, int accumulate)
{
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * V;
    if (i >= n) return;
    float s[V];
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = accumulate ? dw[i + j] : 0.f;
#pragma unroll 8
    for (int p = 0; p < n_parts; ++p) {
        const float* const q = parts + p * n + i;
        if constexpr (V == 4) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(q);
#pragma unroll
            for (int j = 0; j < 4; ++j) s[j] += v[j];
        } else {
            s[0] += q[0];
        }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) dw[i + j] = s[j];
}

template <typename T, int V>
int run_wgrad(const void* dy, int64_t dy_pitch, const pruner_checkpoint* kept, int64_t rows, int32_t n_out, int32_t dim, const WgradPlan& plan, float* dw, int32_t accumulate,
              float* parts, hipStream_t st)
{
    const int64_t blocks = (int64_t)plan.tiles_n * plan.tiles_k * plan.parts;
    static PerDeviceFlag ready;
    const int dev = current_device(nullptr);
    if (dev < 0) return PRUNER_EHIP;
    if (!ready.get(dev)) {
        for (const void* fn : {reinterpret_cast<const void*>(&wgrad_kernel<T, V, false>), reinterpret_cast<const void*>(&wgrad_kernel<T, V, true>)})
            if (hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, 4 * WgradShape<true>::kTileBytes) != hipSuccess) return PRUNER_EHIP;
        ready.mark(dev);
    }
    auto* const kernel = plan.big ? &wgrad_kernel<T, V, true> : &wgrad_kernel<T, V, false>;
    const int threads = plan.big ? WgradShape<true>::kThreads : WgradShape<false>::kThreads, bytes = 4 * (plan.big ? WgradShape<true>::kTileBytes : WgradShape<false>::kTileBytes);
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(threads), bytes, st, static_cast<const T*>(dy), dy_pitch, kept->codes, kept->exps, rows, n_out, dim, plan,
                       plan.parts > 1 ? parts : dw, accumulate);
    PRUNER_LAUNCH_CHECK();
    if (plan.parts > 1) {
        const int64_t n = (int64_t)n_out * dim;
        if (n % 4 == 0 && aligned(dw, 16))
            hipLaunchKernelGGL(wgrad_join_kernel<4>, dim3((unsigned)((n / 4 + 255) / 256)), dim3(256), 0, st, parts, plan.parts, n, dw, accumulate);
        else
            hipLaunchKernelGGL(wgrad_join_kernel<1>, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, parts, plan.parts, n, dw, accumulate);
        PRUNER_LAUNCH_CHECK();
    }
    return PRUNER_OK;
}

bool wgrad_sizes_ok(int64_t rows, int32_t n_out, int32_t dim)
{
    return rows >= 0 && rows < (1ll << 40) && n_out >= 1 && n_out <= (1 << 20) && dim >= 1 && dim <= (1 << 20) && (int64_t)n_out * dim <= (1ll << 31);
}

bool sizes_ok(int32_t dtype, int64_t rows, int32_t dim, int64_t pitch)
{
    return type_known(dtype) && rows >= 0 && dim >= 1 && dim <= (1 << 28) && pitch >= dim && (rows == 0 || pitch < (1ll << 40) / rows);
}
bool kept_ok(const pruner_checkpoint* c) { return c && c->codes && c->exps && aligned(c->codes, 8); }

// Rows in launches of below 2^31 threads.
template <typename Launch> int in_row_chunks(int64_t rows, int32_t dim, Launch&& launch)
{
    const Divisor per_row(4u * ((uint32_t)(dim + kGroup - 1) / kGroup));
    int64_t most = ((1ll << 31) - 512) / per_row.d;
    for (int64_t r = 0; r < rows; r += most) {
        const int64_t n = rows - r < most ? rows - r : most;
        const uint32_t items = (uint32_t)(n * per_row.d);
        launch(r, items, dim3((items + 255) / 256), per_row);
        PRUNER_LAUNCH_CHECK();
    }
    return PRUNER_OK;
}

template <typename T, int V>
int pack_rows(const void* x, int64_t rows, int32_t dim, int64_t pitch, const pruner_checkpoint* kept, hipStream_t st)
{
    return in_row_chunks(rows, dim, [&](int64_t r, uint32_t items, dim3 grid, const Divisor& per_row) {
        hipLaunchKernelGGL((pack_kernel<T, V>), grid, dim3(256), 0, st, static_cast<const T*>(x) + r * pitch, pitch, rows - r, dim, items, per_row, kept->codes + r * dim,
                           kept->exps + r * (per_row.d / 4));
    });
}
template <typename T, int V>
int restore_rows(const pruner_checkpoint* kept, int64_t rows, int32_t dim, void* x, int64_t pitch, hipStream_t st)
{
    return in_row_chunks(rows, dim, [&](int64_t r, uint32_t items, dim3 grid, const Divisor& per_row) {
        hipLaunchKernelGGL((restore_kernel<T, V>), grid, dim3(256), 0, st, kept->codes + r * dim, kept->exps + r * (per_row.d / 4), rows - r, dim, items, per_row,
                           static_cast<T*>(x) + r * pitch, pitch);
    });
}

}  // namespace
}  // namespace pruner

using namespace pruner;

extern "C" int pruner_checkpoint_pack(const void* x, int32_t dtype, int64_t rows, int32_t dim, int64_t pitch, const pruner_checkpoint* kept, void* stream)
{
    if (!sizes_ok(dtype, rows, dim, pitch)) return PRUNER_EINVAL;
    if (rows == 0) return PRUNER_OK;
    if (!x || !aligned(x, type_bytes(dtype)) || !kept_ok(kept)) return PRUNER_EINVAL;
    Access a;
    a.fits(x, type_bytes(dtype), pitch);
    a.fits(kept->codes, 1, dim);
    return BY_TYPE_AND_ACCESS(dtype, a.v, pack_rows, x, rows, dim, pitch, kept, static_cast<hipStream_t>(stream));
}

extern "C" int pruner_checkpoint_restore(const pruner_checkpoint* kept, int32_t dtype, int64_t rows, int32_t dim, void* x, int64_t pitch, void* stream)
{
    if (!sizes_ok(dtype, rows, dim, pitch)) return PRUNER_EINVAL;
    if (rows == 0) return PRUNER_OK;
    if (!x || !aligned(x, type_bytes(dtype)) || !kept_ok(kept)) return PRUNER_EINVAL;
    Access a;
    a.fits(x, type_bytes(dtype), pitch);
    a.fits(kept->codes, 1, dim);
    return BY_TYPE_AND_ACCESS(dtype, a.v, restore_rows, kept, rows, dim, x, pitch, static_cast<hipStream_t>(stream));
}

extern "C" size_t pruner_checkpoint_wgrad_workspace_bytes(int64_t rows, int32_t n_out, int32_t dim)
{
    if (!wgrad_sizes_ok(rows, n_out, dim)) return 0;
    const WgradPlan p = wgrad_plan(rows, n_out, dim);
    return p.parts > 1 ? round_up((size_t)p.parts * (size_t)n_out * (size_t)dim * 4, 256) : 0;
}

extern "C" int pruner_checkpoint_wgrad(const void* dy, int32_t dtype, int64_t dy_pitch, const pruner_checkpoint* kept, int64_t rows, int32_t n_out, int32_t dim, float* dw,
                                       int32_t accumulate, void* workspace, size_t workspace_bytes, void* stream)
{
    if ((dtype != PRUNER_BF16 && dtype != PRUNER_F16) || !wgrad_sizes_ok(rows, n_out, dim) || !dw || !aligned(dw, 4) || (accumulate != 0 && accumulate != 1)) return PRUNER_EINVAL;
    if (rows > 0 && (!dy || !aligned(dy, 2) || !kept_ok(kept) || dy_pitch < n_out || dy_pitch >= (1 << 24))) return PRUNER_EINVAL;
    if (rows == 0 && accumulate) return PRUNER_OK;
    const WgradPlan plan = wgrad_plan(rows, n_out, dim);
    if (plan.parts > 1 && (!workspace || !aligned(workspace, 256) || workspace_bytes < pruner_checkpoint_wgrad_workspace_bytes(rows, n_out, dim))) return PRUNER_EWORKSPACE;
    Access a;
    const pruner_checkpoint none{nullptr, nullptr};
    if (rows > 0) {
        a.fits(dy, 2, dy_pitch);
        a.fits(kept->codes, 1, dim);
        if (n_out % 8) a.v = 1;   // (a row's last access must not pass its end)
    }
    const pruner_checkpoint* const c = rows > 0 ? kept : &none;
    float* const parts = static_cast<float*>(workspace);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == PRUNER_BF16)
        return a.v == 8 ? run_wgrad<__bf16, 8>(dy, dy_pitch, c, rows, n_out, dim, plan, dw, accumulate, parts, st)
                        : run_wgrad<__bf16, 1>(dy, dy_pitch, c, rows, n_out, dim, plan, dw, accumulate, parts, st);
    return a.v == 8 ? run_wgrad<_Float16, 8>(dy, dy_pitch, c, rows, n_out, dim, plan, dw, accumulate, parts, st)
                    : run_wgrad<_Float16, 1>(dy, dy_pitch, c, rows, n_out, dim, plan, dw, accumulate, parts, st);
}
