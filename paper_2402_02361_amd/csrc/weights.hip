// Linear layers whose weights are held in 4 bits, for few rows: y = x W^T + bias with W = (code - 8) scale, a scale for each 32, 64 or 128 neighbouring inputs of an output.
//
// On v_mfma_f32_16x16x32 with 16 outputs as the rows and 16 rows of x as the columns: of a result, lane (n = lane & 15, g = lane >> 4) holds column n and rows 4 g .. 4 g + 3; of
// operands it holds row (column) n and depths 8 g .. 8 g + 7.  Weights lie as a wavefront takes them: 16 outputs x 128 inputs are 1 KB in a row, a lane's sixteen
// bytes its eight depths of four products.  A group's depths are those of whole products, so a group's sum is a result of its own and is scaled in binary32 when it is added.
// Codes become operands without a conversion: a code under the bits of 128 is the bfloat16 128 + code, and the products start from -136 times the sum of x (one more product,
// shared by all outputs); in binary16 1024 + code, less 1032, which is exact.
// (bfloat16 by conversions to code - 8, which costs no digits of binary32: 32768 x 8192 for one row 39.5 us where this takes 30.3; as 16 + code, from -24 times the sum, 30.9.)
// The wavefronts of a workgroup take every so many blocks of 128 inputs and meet in LDS.  Bound: reading the weights, 32768 x 8192 for one row 29 us, 4.75 TB/s with the launch; where they are few, start and end, 1603 x 1100 8.4 us, 16384 x 4096 for 12 rows 11.6;
// from 17 rows on x, which every 32 or 64 outputs read again: 32 rows over 8192 x 8192 21 us.  One row over 34 MB of codes takes 11 to 13 us (8192 x 8192, 4096 x 16384, 16384 x 4096; the bytes ask for 6.7): a workgroup's start
// and end, 5 us, are not covered by the two blocks that a wavefront has on the way.
#include "common.h"

namespace pruner {
namespace weights {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef u32x4 Loose __attribute__((aligned(2)));

constexpr int kOutputs = 16, kBlock = 128, kBlockWords = kOutputs * kBlock / 8;
constexpr int kZero = 8;   // the code of 0
constexpr int64_t kCached = 96 << 20;   // bytes of codes (us a call read past the caches and not: 32768 x 8192 30.1 and 31.8, 16384 x 4096 13.2 and 12.7, 8192 x 8192 11.5 and 10.7; with other weights in each call 67 MB 17.3 and 18.1, 98 MB 23.6 and 24.6, 115 MB 29.4 and 30.7)

__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c, __bf16)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c, _Float16)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t pair_of(float a, float b, __bf16) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2)); }
__device__ __forceinline__ uint32_t pair_of(float a, float b, _Float16) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), f16x2)); }
__device__ __forceinline__ f32x2 pair_to(uint32_t w) { return f32x2{__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)}; }   // of bfloat16
__device__ __forceinline__ u32x4 operand(uint32_t w, __bf16)
{
    return u32x4{(w & 0x000F000Fu) | 0x43004300u, ((w >> 4) & 0x000F000Fu) | 0x43004300u, ((w >> 8) & 0x000F000Fu) | 0x43004300u, ((w >> 12) & 0x000F000Fu) | 0x43004300u};
}
__device__ __forceinline__ u32x4 operand(uint32_t w, _Float16)
{
    u32x4 r;
    const f16x2 off = {(_Float16)-1032.f, (_Float16)-1032.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, ((w >> (4 * i)) & 0x000F000Fu) | 0x64006400u) + off);
    return r;
}

// Eight weights without their scale, code - 8, in bfloat16.
__device__ __forceinline__ u32x4 weights_of(uint32_t w)
{
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = pair_of((float)((int)(w >> (4 * i) & 15u) - kZero), (float)((int)(w >> (4 * i + 16) & 15u) - kZero), __bf16{});
    return r;
}

__device__ __forceinline__ bool is_finite(float x) { return __builtin_fabsf(x) < __builtin_inff(); }

struct Call {
    const uint32_t* codes;
    const uint16_t* scales;
    const float* bias;
    const char* x;
    char* y;
    int64_t x_pitch, y_pitch;   // elements
    int32_t rows, n_out, dim, blocks;
};

// A wavefront's operands of one block of inputs.
template <typename T, int GROUP, int RT, int CT, bool ONCE> struct Block {
    static constexpr int kGroups = kBlock / GROUP;
    u32x4 w[RT], x[CT][4];
    u32x2 s[RT][kGroups];   // four bfloat16 each
    __device__ __forceinline__ void load(const Call& a, const T* const (&x_row)[CT], int tile0, int tiles, int block, int lane)
    {
        const int g = lane >> 4;
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const int64_t at = (int64_t)(tile0 + t < tiles ? tile0 + t : tiles - 1) * a.blocks + block;
            const u32x4* const p = reinterpret_cast<const u32x4*>(a.codes + at * kBlockWords + 4 * lane);
            if constexpr (ONCE)
                w[t] = __builtin_nontemporal_load(p);
            else
                w[t] = *p;
#pragma unroll
            for (int u = 0; u < kGroups; ++u) s[t][u] = *reinterpret_cast<const u32x2*>(a.scales + ((at * 4 + g) * kGroups + u) * 4);
        }
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            if (!x_row[c]) continue;   // (columns past the last: what they give is not stored)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int at = kBlock * block + 32 * j + 8 * g;
                if (at + 8 <= a.dim) {
                    x[c][j] = *reinterpret_cast<const Loose*>(x_row[c] + at);
                } else {
                    x[c][j] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (at + i < a.dim) x[c][j][i / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, x_row[c][at + i]) << (16 * (i % 2));
                }
            }
        }
    }
    __device__ __forceinline__ void add(f32x4 (&acc)[RT][CT]) const
    {
        constexpr int kEach = GROUP / 32;
        const uint32_t off = __builtin_bit_cast(uint32_t, (bf16x2{(__bf16)-136.f, (__bf16)-136.f}));
#pragma unroll
        for (int u = 0; u < kGroups; ++u) {
            f32x4 from[CT];
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                from[c] = f32x4{0.f, 0.f, 0.f, 0.f};
                if constexpr (sizeof(T) == 2 && __is_same(T, __bf16))
#pragma unroll
                    for (int e = 0; e < kEach; ++e) from[c] = mfma(u32x4{off, off, off, off}, x[c][u * kEach + e], from[c], T{});
            }
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                f32x4 sum[CT];
#pragma unroll
                for (int e = 0; e < kEach; ++e) {
                    const u32x4 o = operand(w[t][u * kEach + e], T{});
#pragma unroll
                    for (int c = 0; c < CT; ++c) sum[c] = mfma(o, x[c][u * kEach + e], e == 0 ? from[c] : sum[c], T{});
                }
                scaled(t, u, sum, acc[t]);
            }
        }
    }
    __device__ __forceinline__ void scaled(int t, int u, const f32x4 (&sum)[CT], f32x4 (&acc)[CT]) const   // a group's sums, added up
    {
        const f32x2 lo = pair_to(s[t][u][0]), hi = pair_to(s[t][u][1]);
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            acc[c][0] = __builtin_fmaf(lo[0], sum[c][0], acc[c][0]);
            acc[c][1] = __builtin_fmaf(lo[1], sum[c][1], acc[c][1]);
            acc[c][2] = __builtin_fmaf(hi[0], sum[c][2], acc[c][2]);
            acc[c][3] = __builtin_fmaf(hi[1], sum[c][3], acc[c][3]);
        }
    }
};

// In bfloat16 the products above reach infinities of their own where x has one, or is so large that 143 of it are one: sums that came out not finite are made again, of x times 2^-16 and the weights without
// their scale, which no finite x takes out of binary32's range before a group's sum is scaled.  (Others stay as they are, whatever other rows hold.)
constexpr float kSmaller = 0x1p-16f;
template <int GROUP, int RT, int CT, bool ONCE>
__device__ __forceinline__ void again(const Call& a, const __bf16* const (&x_row)[CT], int tile0, int tiles, int wave, int waves, int lane, f32x4 (&acc)[RT][CT])
{
    using Turn = Block<__bf16, GROUP, RT, CT, ONCE>;
    constexpr int kEach = GROUP / 32;
    f32x4 made[RT][CT];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int c = 0; c < CT; ++c) made[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int block = wave; block < a.blocks; block += waves) {
        Turn now;
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) now.x[c][j] = u32x4{0u, 0u, 0u, 0u};
        now.load(a, x_row, tile0, tiles, block, lane);
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x2 x = pair_to(now.x[c][j][i]);
                    now.x[c][j][i] = pair_of(x[0] * kSmaller, x[1] * kSmaller, __bf16{});
                }
#pragma unroll
        for (int u = 0; u < Turn::kGroups; ++u)
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                f32x4 sum[CT];
#pragma unroll
                for (int c = 0; c < CT; ++c) sum[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int e = 0; e < kEach; ++e) {
                    const u32x4 o = weights_of(now.w[t][u * kEach + e]);
#pragma unroll
                    for (int c = 0; c < CT; ++c) sum[c] = mfma(o, now.x[c][u * kEach + e], sum[c], __bf16{});
                }
                now.scaled(t, u, sum, made[t]);
            }
    }
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[t][c][e] = is_finite(acc[t][c][e]) ? acc[t][c][e] : made[t][c][e] * (1.f / kSmaller);
}

// ONCE: the weights are more than stays cached from one call to the next, and are read past it.
template <typename T, int GROUP, int RT, int CT, bool ONCE> __global__ void __launch_bounds__(RT == 1 && CT == 1 ? 1024 : 512) linear_kernel(Call a)
{
    extern __shared__ __attribute__((aligned(16))) float sums[];   // [wavefront][RT * CT][64][4]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), waves = (int)blockDim.x >> 6;
    const int tiles = (a.n_out + kOutputs - 1) / kOutputs, tile0 = (int)blockIdx.x * RT, row0 = (int)blockIdx.y * 16 * CT;
    const T* x_row[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const int row = row0 + 16 * c + (lane & 15);
        x_row[c] = row < a.rows ? reinterpret_cast<const T*>(a.x) + (int64_t)row * a.x_pitch : nullptr;
    }
    f32x4 acc[RT][CT];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int c = 0; c < CT; ++c) acc[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    Block<T, GROUP, RT, CT, ONCE> on_way[2];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) on_way[n].x[c][j] = u32x4{0u, 0u, 0u, 0u};
    if (wave < a.blocks) on_way[0].load(a, x_row, tile0, tiles, wave, lane);
    for (int block = wave; block < a.blocks;) {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            if (block + waves < a.blocks) on_way[n ^ 1].load(a, x_row, tile0, tiles, block + waves, lane);
            if (block < a.blocks) on_way[n].add(acc);
            block += waves;
        }
    }
    if constexpr (__is_same(T, __bf16)) {
        bool all = true;
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) all = all && is_finite(acc[t][c][e]);
        if (!__all(all)) again<GROUP, RT, CT, ONCE>(a, x_row, tile0, tiles, wave, waves, lane, acc);
    }
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int c = 0; c < CT; ++c) *reinterpret_cast<f32x4*>(sums + ((wave * RT * CT + t * CT + c) * 64 + lane) * 4) = acc[t][c];
    __syncthreads();
    for (int i = threadIdx.x; i < RT * CT * 64; i += blockDim.x) {
        const int l = i & 63, t = i / 64 / CT, c = i / 64 % CT, n = row0 + 16 * c + (l & 15), o = (tile0 + t) * kOutputs + 4 * (l >> 4);
        if (n >= a.rows || o >= a.n_out) continue;
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < waves; ++w) {
            const f32x4 one = *reinterpret_cast<const f32x4*>(sums + ((int64_t)w * RT * CT * 64 + i) * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] += one[e];
        }
        T* const out = reinterpret_cast<T*>(a.y) + (int64_t)n * a.y_pitch + o;
        const int left = a.n_out - o < 4 ? a.n_out - o : 4;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) out[e] = (T)(a.bias ? y[e] + a.bias[o + e] : y[e]);
    }
}

// ---- there and back: a thread takes 32 neighbouring inputs of an output; neighbouring threads those of the same block
// (Once per set of weights, so written for clearness: 32768 x 8192 in bfloat16 packed in 630 us and restored in 2.1 ms, where the bytes ask for 134; single values, 32 apart between lanes, are the cause.)

template <typename T> __device__ __forceinline__ float value_of(const T* p) { return (float)*p; }

template <typename T, int GROUP> __global__ void __launch_bounds__(256) pack_kernel(const T* __restrict__ w, int64_t pitch, uint32_t* __restrict__ codes, uint16_t* __restrict__ scales, int n_out, int dim, int blocks)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, all = (int64_t)((n_out + kOutputs - 1) / kOutputs) * kOutputs * blocks * 4;
    const int64_t at = i < all ? i : all - 1;   // (every lane takes part in the exchange)
    const int j = (int)(at & 3), block = (int)(at / 4 % blocks);
    const int64_t row = at / 4 / blocks;
    const int first = kBlock * block + 32 * j, n = row >= n_out || first >= dim ? 0 : dim - first < 32 ? dim - first : 32;
    float x[32];
    float top = 0.f;
#pragma unroll
    for (int k = 0; k < 32; ++k) {
        x[k] = k < n ? (float)w[row * pitch + first + k] : 0.f;
        const float size = __builtin_fabsf(x[k]);
        top = size > top || size != size ? size : top;   // (a NaN stays)
    }
    if constexpr (GROUP >= 64) {
        const float other = __shfl_xor(top, 1, kWave);
        top = other > top || other != other ? other : top;
    }
    if constexpr (GROUP >= 128) {
        const float other = __shfl_xor(top, 2, kWave);
        top = other > top || other != other ? other : top;
    }
    if (i >= all) return;
    const float step = top < __builtin_inff() ? (float)(__bf16)(top / 7.f) : __builtin_nanf("");
    const int64_t tile = row / kOutputs;
    const int r = (int)(row % kOutputs);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        uint32_t word = 0u;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float q = step > 0.f ? __builtin_rintf(x[8 * g + k] / step) : 0.f;
            const int code = (int)(q < -8.f ? -8.f : q > 7.f ? 7.f : q) + kZero;
            word |= (uint32_t)code << (4 * (k / 2) + 16 * (k % 2));
        }
        codes[(tile * blocks + block) * kBlockWords + (g * kOutputs + r) * 4 + j] = word;
    }
    constexpr int kGroups = kBlock / GROUP;
    if (j % (GROUP / 32) == 0) scales[(((tile * blocks + block) * 4 + r / 4) * kGroups + j / (GROUP / 32)) * 4 + r % 4] = __builtin_bit_cast(uint16_t, (__bf16)step);
}

template <typename T> __global__ void __launch_bounds__(256) unpack_kernel(const uint32_t* __restrict__ codes, const uint16_t* __restrict__ scales, T* __restrict__ w, int64_t pitch, int n_out, int dim, int blocks, int group)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int j = (int)(i & 3), block = (int)(i / 4 % blocks);
    const int64_t row = i / 4 / blocks;
    const int first = kBlock * block + 32 * j;
    if (row >= n_out || first >= dim) return;
    const int64_t tile = row / kOutputs;
    const int r = (int)(row % kOutputs), groups = kBlock / group;
    const float step = __uint_as_float((uint32_t)scales[(((tile * blocks + block) * 4 + r / 4) * groups + 32 * j / group) * 4 + r % 4] << 16);
    for (int g = 0; g < 4; ++g) {
        const uint32_t word = codes[(tile * blocks + block) * kBlockWords + (g * kOutputs + r) * 4 + j];
        for (int k = 0; k < 8; ++k)
            if (first + 8 * g + k < dim) w[row * pitch + first + 8 * g + k] = (T)((float)((int)(word >> (4 * (k / 2) + 16 * (k % 2)) & 15u) - kZero) * step);
    }
}

bool weights_ok(const pruner_weights* w)
{
    if (!w || w->n_out < 1 || w->dim < 1 || w->n_out > (1 << 24) || w->dim > (1 << 24) || (w->group != 32 && w->group != 64 && w->group != 128)) return false;
    return w->codes && w->scales && aligned(w->codes, 16) && aligned(w->scales, 8);
}
int blocks_of(const pruner_weights* w) { return (w->dim + kBlock - 1) / kBlock; }
size_t size_of(int32_t dtype) { return dtype == PRUNER_F32 ? 4 : 2; }

template <typename T, int GROUP, int RT, int CT, bool ONCE = false> int launch(const Call& a, int waves, hipStream_t st)
{
    static PerDeviceFlag ready;
    const int dev = current_device(nullptr);
    if (dev < 0) return PRUNER_EHIP;
    if (!ready.get(dev)) {
        if (hipFuncSetAttribute(reinterpret_cast<const void*>(&linear_kernel<T, GROUP, RT, CT, ONCE>), hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) != hipSuccess) return PRUNER_EHIP;
        ready.mark(dev);
    }
    const dim3 grid((unsigned)((a.n_out + kOutputs * RT - 1) / (kOutputs * RT)), (unsigned)((a.rows + 16 * CT - 1) / (16 * CT)));
    hipLaunchKernelGGL((linear_kernel<T, GROUP, RT, CT, ONCE>), grid, dim3(64 * waves), (size_t)waves * RT * CT * 1024, st, a);
    PRUNER_LAUNCH_CHECK();
    return PRUNER_OK;
}
template <typename T, int GROUP> int route(const Call& a, hipStream_t st)
{
    // Output tiles of a wavefront: the more, the less often x is read, and the fewer workgroups there are.  (us a call of up to 16 rows, one tile and two, by 8 and 16 wavefronts: 32768 x 8192 41
    // and 49, 32 and 38; 8192 x 8192 12.2 and 13.3, 10.8 and 10.6; 4096 x 16384 14 and 11, 17 and 15.  More rows, two tiles and four: 32 over 8192 x 8192 21 and 24, 100 over 4096 x 4096 22 and
    // 16, 64 over 16384 x 4096 42 and 29, 17 over 2000 x 3000 10.6 and 12.7.)
    const int tiles = (a.n_out + kOutputs - 1) / kOutputs, eight = a.blocks < 8 ? a.blocks : 8;
    if (a.rows > 16) {
        if constexpr (GROUP > 32)   // (the scales of four tiles in groups of 32 do not fit the registers)
            if ((int64_t)((tiles + 3) / 4) * ((a.rows + 31) / 32) >= 256) return launch<T, GROUP, 4, 2>(a, eight, st);
        return launch<T, GROUP, 2, 2>(a, eight, st);
    }
    if (tiles >= 512) return (int64_t)a.n_out * a.dim / 2 > kCached ? launch<T, GROUP, 2, 1, true>(a, eight, st) : launch<T, GROUP, 2, 1>(a, eight, st);
    return launch<T, GROUP, 1, 1>(a, a.blocks < 16 ? a.blocks : 16, st);
}
template <typename T> int by_group(const Call& a, int group, hipStream_t st) { return group == 32 ? route<T, 32>(a, st) : group == 64 ? route<T, 64>(a, st) : route<T, 128>(a, st); }

template <typename T> int pack(const pruner_weights* p, const void* w, int64_t pitch, hipStream_t st)
{
    const int blocks = blocks_of(p);
    const int64_t all = (int64_t)((p->n_out + kOutputs - 1) / kOutputs) * kOutputs * blocks * 4;
    const dim3 grid((unsigned)((all + 255) / 256));
    const T* const from = static_cast<const T*>(w);
    uint32_t* const codes = reinterpret_cast<uint32_t*>(p->codes);
    if (p->group == 32)
        hipLaunchKernelGGL((pack_kernel<T, 32>), grid, dim3(256), 0, st, from, pitch, codes, p->scales, p->n_out, p->dim, blocks);
    else if (p->group == 64)
        hipLaunchKernelGGL((pack_kernel<T, 64>), grid, dim3(256), 0, st, from, pitch, codes, p->scales, p->n_out, p->dim, blocks);
    else
        hipLaunchKernelGGL((pack_kernel<T, 128>), grid, dim3(256), 0, st, from, pitch, codes, p->scales, p->n_out, p->dim, blocks);
    PRUNER_LAUNCH_CHECK();
    return PRUNER_OK;
}
template <typename T> int unpack(const pruner_weights* p, void* w, int64_t pitch, hipStream_t st)
{
    const int blocks = blocks_of(p);
    const dim3 grid((unsigned)(((int64_t)p->n_out * blocks * 4 + 255) / 256));
    hipLaunchKernelGGL((unpack_kernel<T>), grid, dim3(256), 0, st, reinterpret_cast<const uint32_t*>(p->codes), p->scales, static_cast<T*>(w), pitch, p->n_out, p->dim, blocks, p->group);
    PRUNER_LAUNCH_CHECK();
    return PRUNER_OK;
}
bool dense_ok(const pruner_weights* p, const void* w, int32_t dtype, int64_t pitch)
{
    // (a launch is below 2^24 workgroups of 256 threads)
    return weights_ok(p) && dtype >= PRUNER_BF16 && dtype <= PRUNER_F32 && w && aligned(w, size_of(dtype)) && pitch >= p->dim && ((int64_t)p->n_out + 15) * blocks_of(p) * 4 / 256 < (1 << 24) - 1;
}

}  // namespace
}  // namespace weights
}  // namespace pruner

using namespace pruner;

extern "C" int pruner_weights_pack(const void* w, int32_t dtype, int64_t pitch, const pruner_weights* packed, void* stream)
{
    if (!weights::dense_ok(packed, w, dtype, pitch)) return PRUNER_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == PRUNER_BF16  ? weights::pack<__bf16>(packed, w, pitch, st)
           : dtype == PRUNER_F16 ? weights::pack<_Float16>(packed, w, pitch, st)
                                 : weights::pack<float>(packed, w, pitch, st);
}

extern "C" int pruner_weights_restore(const pruner_weights* packed, int32_t dtype, void* w, int64_t pitch, void* stream)
{
    if (!weights::dense_ok(packed, w, dtype, pitch)) return PRUNER_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == PRUNER_BF16  ? weights::unpack<__bf16>(packed, w, pitch, st)
           : dtype == PRUNER_F16 ? weights::unpack<_Float16>(packed, w, pitch, st)
                                 : weights::unpack<float>(packed, w, pitch, st);
}

extern "C" int pruner_weights_linear(const pruner_weights* packed, const void* x, int32_t dtype, int64_t rows, int64_t x_pitch, const float* bias, void* y, int64_t y_pitch, void* stream)
{
    if (!weights::weights_ok(packed) || (dtype != PRUNER_BF16 && dtype != PRUNER_F16) || rows < 0 || rows > PRUNER_MAX_LINEAR_ROWS) return PRUNER_EINVAL;
    if ((bias && !aligned(bias, 4)) || x_pitch < packed->dim || y_pitch < packed->n_out) return PRUNER_EINVAL;
    if (rows == 0) return PRUNER_OK;
    if (!x || !y || !aligned(x, 2) || !aligned(y, 2)) return PRUNER_EINVAL;
    const weights::Call a{reinterpret_cast<const uint32_t*>(packed->codes), packed->scales, bias, static_cast<const char*>(x), static_cast<char*>(y), x_pitch, y_pitch, (int32_t)rows,
                          packed->n_out, packed->dim, weights::blocks_of(packed)};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == PRUNER_BF16 ? weights::by_group<__bf16>(a, packed->group, st) : weights::by_group<_Float16>(a, packed->group, st);
}
