// What the kernels of attention with a learned relative position bias have in common (see include/pruner.h for the formulas).
//
// Products run on v_mfma_f32_32x32x16 with both operands' outer index in the lanes: of a 32 x 32 result, lane (l32 = lane & 31, half = lane >> 5)
// holds column l32 and the sixteen rows 8 (i / 4) + 4 half + i % 4.  An operand of depth 16 holds, per lane, the eight depths of its half.  Any
// numbering of the depth will do as long as both operands use the same one, and with depth (half, j) meaning row 8 (j / 4) + 4 half + j % 4 of a
// 16-row step, a result's registers 8 s .. 8 s + 7, rounded to 16 bits, are the operand of the next product as they stand: softmax weights and
// their gradients never leave the registers.  The other operand of that product is a tile turned over, read by ds_read_b64_tr_b16 (16 lanes take
// four rows of 16 columns; lane t gives the address of row t / 4, columns 4 (t % 4) .., and gets column t of the four rows).
#pragma once
#include "common.h"

namespace pruner {
namespace att {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.693147180559945309417f;
constexpr float kLarge = 1024.f;   // a bias beyond this is added to a score before anything else is done with either, as where biases lie in a window; see also row_sums
#define ATT_INF __builtin_inff()

__device__ __forceinline__ floatx16 mfma(u32x4 a, u32x4 b, floatx16 c, __bf16)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ floatx16 mfma(u32x4 a, u32x4 b, floatx16 c, _Float16)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t pair_of(float a, float b, __bf16) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2)); }
__device__ __forceinline__ uint32_t pair_of(float a, float b, _Float16) { return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), f16x2)); }
__device__ __forceinline__ f32x2 pair_to(uint32_t w, __bf16) { return f32x2{__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)}; }
__device__ __forceinline__ f32x2 pair_to(uint32_t w, _Float16) { return __builtin_convertvector(__builtin_bit_cast(f16x2, w), f32x2); }

__device__ __forceinline__ floatx16 zero16()
{
    floatx16 z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.f;
    return z;
}
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
// Of a lane and the one of the same column in the other half.
__device__ __forceinline__ float sum_of_halves(float v)
{
    const TwoFloats t = across_halves(v);
    return t.a + t.b;
}
__device__ __forceinline__ float max_of_halves(float v)
{
    const TwoFloats t = across_halves(v);
    return __builtin_fmaxf(t.a, t.b);
}
__device__ __forceinline__ int row_of(int i, int half) { return 8 * (i >> 2) + 4 * half + (i & 3); }

// What this wavefront's lanes wrote to LDS is there for its other lanes after.
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

struct Heads {
    char* p;
    int64_t batch, head;
    int32_t token;   // elements
    template <typename T> __device__ __forceinline__ T* at(int b, int h) const { return reinterpret_cast<T*>(p) + b * batch + h * head; }
};

struct Args {
    Heads q, k, v;
    const int32_t *q_len, *k_len;
    const void* table;
    int32_t batch, q_tokens, k_tokens, q_heads, kv_heads, group, head_dim, causal, two_sided, n_edges;
    float scale;
    int32_t left, right;   // pairs at r <= -left share one bucket, those at r >= right share one (both cut to what the lengths can reach)
    int32_t edges[PRUNER_MAX_BIAS_EDGES];   // INT32_MAX from n_edges on
    __device__ __forceinline__ int queries(int b) const { return clamped(q_len, b, q_tokens); }
    __device__ __forceinline__ int keys(int b) const { return clamped(k_len, b, k_tokens); }
    __device__ __forceinline__ static int clamped(const int32_t* p, int b, int most)
    {
        if (!p) return most;
        const int n = p[b];
        return n < 0 ? 0 : n > most ? most : n;
    }
    __device__ __forceinline__ int bucket(int r) const
    {
        const int d = two_sided ? (r < 0 ? -r : r) : (r < 0 ? -r : 0);
        int n = 0;
        for (int e = 0; e < n_edges; e += 16)   // (sixteen by one scalar load; those past the last are beyond every distance)
#pragma unroll
            for (int k = 0; k < 16; ++k) n += edges[e + k] <= d ? 1 : 0;
        return n + (two_sided && r > 0 ? n_edges + 1 : 0);
    }
    template <typename T> __device__ __forceinline__ float bias(int n, int h) const { return (float)static_cast<const T*>(table)[(int64_t)n * q_heads + h]; }
};

// Biases by r in LDS: those that a tile which is not wholly at one end can ask for, r = first .. first + size - 1.
constexpr int kWindowPad = 96;   // a tile spans 32 places on one side and at most 64 on the other
struct Window {
    int first, size;
    __host__ __device__ Window(int left, int right) : first(-left - kWindowPad), size(left + right + 2 * kWindowPad) {}
};
// Filled by THREADS threads in two calls, so that the table's first values come while other things are asked for: a thread's first kAtOnce places are loaded
// by load(), the rest by store().
template <typename T, int THREADS> struct WindowFill {
    static constexpr int kAtOnce = THREADS >= 256 ? 2 : 4;
    T x[kAtOnce];
    __device__ __forceinline__ void load_from(const Args& a, const Window& w, int h, int first)
    {
        int d[kAtOnce], n[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int r = w.first + first + THREADS * u;
            d[u] = r < 0 ? -r : a.two_sided ? r : 0;
            n[u] = a.two_sided && r > 0 ? a.n_edges + 1 : 0;
        }
        for (int e = 0; e < a.n_edges; e += 16)   // (sixteen edges by one scalar load; those past the last are beyond every distance)
#pragma unroll
            for (int k = 0; k < 16; ++k)
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) n[u] += a.edges[e + k] <= d[u] ? 1 : 0;
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) x[u] = static_cast<const T*>(a.table)[(int64_t)n[u] * a.q_heads + h];   // (a bucket for every r)
    }
    __device__ __forceinline__ void store_to(float* lds, const Window& w, int first) const
    {
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
            if (first + THREADS * u < w.size) lds[first + THREADS * u] = (float)x[u];
    }
    __device__ __forceinline__ void load(const Args& a, const Window& w, int h, int thread) { load_from(a, w, h, thread); }
    __device__ __forceinline__ void store(const Args& a, const Window& w, float* lds, int h, int thread)
    {
        store_to(lds, w, thread);
        for (int i = thread + THREADS * kAtOnce; i < w.size; i += THREADS * kAtOnce) {
            load_from(a, w, h, i);
            store_to(lds, w, i);
        }
    }
};
// Where a tile with r = r_lo .. r_hi lies.
enum { kNear, kLeft, kRight };
__device__ __forceinline__ int place_of(const Args& a, int r_lo, int r_hi) { return r_hi <= -a.left ? kLeft : r_lo >= a.right ? kRight : kNear; }

// Tiles of DP columns (the head dimension rounded up; columns past it are zero) in LDS: rows of DP values, their 16-byte chunks permuted row by
// row so that neither 16 rows' reads of one chunk nor a turning read's four rows of 64 bytes meet in a bank.
template <int DP> struct Tile {
    static constexpr int kChunks = DP / 8, kRowBytes = DP * 2, kSteps = DP / 16, kBlocks = DP / 32;
    __device__ __forceinline__ static int turn_of(int row)
    {
        if constexpr (DP == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
        if constexpr (DP == 64) return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
        return (row >> 2) & 3;
    }
    __device__ __forceinline__ static int at(int row, int chunk) { return row * kRowBytes + ((chunk ^ turn_of(row)) << 4); }
};

// The places of a lane's fragments in a tile.  A step or a block further is one bit pattern further in the chunk's number, so all of them come from three
// places by an exclusive or.
template <int DP> struct Lane {
    int row;         // rows as the outer index: row l32, depths 16 s + 8 half .. at row ^ (s << 5)
    int turned[2];   // columns as the outer index: columns 32 b + l32, rows 8 q + 4 half .. + 3 of a 16-row step at turned[q] ^ (b << 6)
    __device__ __forceinline__ void set(int lane)
    {
        const int l32 = lane & 31, half = lane >> 5, t = lane & 15, g = (lane >> 4) & 1;
        row = Tile<DP>::at(l32, half);
#pragma unroll
        for (int q = 0; q < 2; ++q) turned[q] = Tile<DP>::at(8 * q + 4 * half + (t >> 2), 2 * g + ((t >> 1) & 1)) + 8 * (t & 1);
    }
    // Inside a loop whose registers are all taken: the places are formed again from the three, not kept.
    __device__ __forceinline__ void forget() { asm volatile("" : "+v"(row), "+v"(turned[0]), "+v"(turned[1])); }
    __device__ __forceinline__ u32x4 rows(const char* tile, int block, int s) const
    {
        return *reinterpret_cast<const u32x4*>(tile + (row ^ (s << 5)) + block * 32 * Tile<DP>::kRowBytes);
    }
    __device__ __forceinline__ u32x4 columns(const char* tile, int b, int step) const
    {
        typedef __attribute__((address_space(3))) i16x4* lds_ptr;
        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(tile + (turned[0] ^ (b << 6)) + step * 16 * Tile<DP>::kRowBytes));
        const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(tile + (turned[1] ^ (b << 6)) + step * 16 * Tile<DP>::kRowBytes));
        const u32x2 a = __builtin_bit_cast(u32x2, lo), c = __builtin_bit_cast(u32x2, hi);
        return u32x4{a[0], a[1], c[0], c[1]};
    }
};

// N products, each with an operand from LDS that is read AHEAD products before it is needed: left to itself the compiler reads each right before its
// product and waits for it (gradients of 5001 causal tokens, 16 heads of 128: keys' kernel 280 us where this took 252, queries' 196 and 188).
template <int N, int AHEAD> struct Operands {
    u32x4 w[AHEAD];
    template <typename Read> __device__ __forceinline__ void start(const Read& read)
    {
#pragma unroll
        for (int i = 0; i < AHEAD && i < N; ++i) w[i] = read(i);
        __builtin_amdgcn_sched_barrier(6);
    }
    template <typename Read, typename Use> __device__ __forceinline__ void products(const Read& read, const Use& use)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            use(i, w[i % AHEAD]);
            if (i + AHEAD < N) w[i % AHEAD] = read(i + AHEAD);
            __builtin_amdgcn_sched_barrier(6);   // (vector and scalar arithmetic may cross, reads and products stay as written)
        }
    }
};

// ROWS rows on their way from memory to a tile, by THREADS threads.  Reads are bounds-checked buffer loads: rows at or beyond `rows` and columns at or beyond
// the head dimension arrive as zeros.  (Where tokens lie closer than a head is wide, rows overlap and a row that is not there may arrive as one that
// is; nothing depends on it, its pairs are masked.)
template <typename T, int DP, int ROWS, int THREADS> struct Stage {
    static constexpr int kEach = ROWS * Tile<DP>::kChunks / THREADS, kRowStep = THREADS / Tile<DP>::kChunks;
    static_assert(kEach >= 1 && ROWS * Tile<DP>::kChunks % THREADS == 0 && THREADS % Tile<DP>::kChunks == 0, "whole chunks per thread, of one column");
    u32x4 w[kEach];
    uint32_t at;
    int32_t row_bytes, width;
    __device__ __forceinline__ void set(int32_t token, int head_dim, int thread)
    {
        row_bytes = token * 2;
        width = head_dim * 2;
        const int chunk = thread % Tile<DP>::kChunks;
        at = 16 * chunk < width ? (uint32_t)(thread / Tile<DP>::kChunks) * (uint32_t)row_bytes + 16u * (uint32_t)chunk : 0x80000000u;
    }
    __device__ __forceinline__ void fetch(const T* base, int rows)   // base and rows: the same in all lanes
    {
        rows = rows < ROWS ? rows : ROWS;
        const int bytes = rows > 0 ? (rows - 1) * row_bytes + width : 0;
        const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(base), 0, bytes, 0x00027000);
#pragma unroll
        for (int u = 0; u < kEach; ++u) w[u] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(from, (int)at, u * kRowStep * row_bytes, 0));
    }
    __device__ __forceinline__ void park(char* tile, int thread) const
    {
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
            const int id = thread + THREADS * u;
            *reinterpret_cast<u32x4*>(tile + Tile<DP>::at(id / Tile<DP>::kChunks, id % Tile<DP>::kChunks)) = w[u];
        }
    }
};

// The same without registers on the way: bounds-checked buffer loads whose data go to LDS (64 lanes' 16 bytes side by side from M0 on), for a tile that all
// wavefronts of a workgroup share, or one's own.  What was requested has arrived after wait_for<n>(), n the number of this wavefront's later requests, and is
// there for the others after a barrier.  What these fill lies in the first kRequestRoom bytes of LDS (a place of 16 bits).  (A row's chunks are permuted on the way: a
// lane asks for the chunk whose place it fills.)  The requests are written out because the compiler, seeing them, would wait for all
// of them before any read of LDS; they return nothing in registers.
constexpr int kRequestRoom = 65536;
__device__ __forceinline__ void request_16(uint32_t lds, uint32_t at, u32x4 from, uint32_t offset)
{
    asm volatile("s_nop 4\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(at), "s"(from), "s"(offset) : "memory", "m0");
}
__device__ __forceinline__ void request_4(uint32_t lds, uint32_t at, u32x4 from)   // 4 bytes a lane
{
    asm volatile("s_nop 4\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds), "v"(at), "s"(from) : "memory", "m0");
}
template <int N> __device__ __forceinline__ void wait_for() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// Before a loop: all that was loaded into registers has come.  (Where the compiler finds a first use inside the loop, it waits there each time, and with
// that for the requests, of which it does not know.)
__device__ __forceinline__ void settle() { __builtin_amdgcn_s_waitcnt(0x0F70); }   // vmcnt(0)
// Before a wavefront asks for a tile of its own again: what it read of the last one has come.
__device__ __forceinline__ void wait_for_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ u32x4 buffer_of(const void* base, int bytes)   // base and bytes: the same in all lanes
{
    const uint64_t p = reinterpret_cast<uint64_t>(base);
    return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)p), (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(p >> 32)),
                 (uint32_t)__builtin_amdgcn_readfirstlane(bytes), 0x00027000u};
}
template <typename T, int DP, int ROWS, int THREADS> struct Flow {
    static constexpr int kEach = ROWS * Tile<DP>::kChunks / THREADS, kRowStep = THREADS / Tile<DP>::kChunks;
    static constexpr int kWays = kRowStep >= 16 ? 1 : 16 / kRowStep;   // permutations that a thread's rows go through in turn
    static_assert(kEach >= 1 && ROWS * Tile<DP>::kChunks % THREADS == 0 && THREADS % Tile<DP>::kChunks == 0, "a thread's chunks are of whole rows");
    uint32_t at[kWays], place;
    int32_t row_bytes, width;
    __device__ __forceinline__ void set(int32_t token, int head_dim, int thread, int wave)   // wave: of those that share the tile
    {
        row_bytes = token * 2;
        width = head_dim * 2;
        place = 1024u * (uint32_t)wave;
        const int row = thread / Tile<DP>::kChunks;
#pragma unroll
        for (int w = 0; w < kWays; ++w) {
            const int chunk = (thread % Tile<DP>::kChunks) ^ Tile<DP>::turn_of(row + w * kRowStep);
            at[w] = 16 * chunk < width ? (uint32_t)row * (uint32_t)row_bytes + 16u * (uint32_t)chunk : 0x80000000u;
        }
    }
    __device__ __forceinline__ void request(const T* base, int rows, uint32_t tile) const   // tile: its place in LDS
    {
        rows = rows < ROWS ? rows : ROWS;
        const u32x4 from = buffer_of(base, rows > 0 ? (rows - 1) * row_bytes + width : 0);
#pragma unroll
        for (int u = 0; u < kEach; ++u) request_16(tile + place + u * THREADS * 16u, at[u % kWays], from, (uint32_t)(u * kRowStep * row_bytes));
    }
};

// A row's fragments straight from memory (its owner is lane l32, depths 16 s + 8 half ..); zero where there is no such row or column.
template <typename T, int DP> __device__ __forceinline__ void load_row(u32x4 (&f)[Tile<DP>::kSteps], const T* p, bool in, int head_dim, int half)
{
#pragma unroll
    for (int s = 0; s < Tile<DP>::kSteps; ++s) {
        f[s] = u32x4{0u, 0u, 0u, 0u};
        if (in && 16 * s + 8 * half < head_dim) f[s] = *reinterpret_cast<const u32x4*>(p + 16 * s + 8 * half);
    }
}
// A column of a result to memory: this lane's rows of the 32-row blocks are a row's values 32 b + 8 g + 4 half ..
template <typename T, int DP> __device__ __forceinline__ void store_row(T* p, const floatx16 (&acc)[Tile<DP>::kBlocks], float factor, int head_dim, int half)
{
#pragma unroll
    for (int b = 0; b < Tile<DP>::kBlocks; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * b + 8 * g + 4 * half;
            if (d < head_dim)
                *reinterpret_cast<u32x2*>(p + d) = u32x2{pair_of(acc[b][4 * g] * factor, acc[b][4 * g + 1] * factor, T{}), pair_of(acc[b][4 * g + 2] * factor, acc[b][4 * g + 3] * factor, T{})};
        }
}
template <int DP> __device__ __forceinline__ void store_row32(float* p, const floatx16 (&acc)[Tile<DP>::kBlocks], int half)
{
#pragma unroll
    for (int b = 0; b < Tile<DP>::kBlocks; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g) *reinterpret_cast<f32x4*>(p + 32 * b + 8 * g + 4 * half) = f32x4{acc[b][4 * g], acc[b][4 * g + 1], acc[b][4 * g + 2], acc[b][4 * g + 3]};
}
template <typename T> __device__ __forceinline__ u32x4 weights_of(const floatx16& p, int step)   // a result's registers as the next product's operand
{
    return u32x4{pair_of(p[8 * step], p[8 * step + 1], T{}), pair_of(p[8 * step + 2], p[8 * step + 3], T{}), pair_of(p[8 * step + 4], p[8 * step + 5], T{}),
                 pair_of(p[8 * step + 6], p[8 * step + 7], T{})};
}

// Workgroups go to the eight dies in turn.  Item i of (sequences x key heads) x (query heads that share one) x tiles, for a kernel whose workgroups read what
// the others of their key head read: a die takes every eighth key head, so that sequences of different lengths spread over the dies (a run of heads per
// die instead: 16 sequences of up to 777 tokens, 12 heads of 64, 43 us where this took 37), of all of them the last tiles first: under a causal
// mask these are the longest, and without one the tiles that short sequences do not have spread what follows over the units (first tiles first: 40 us where this takes 34).
struct Item {
    int head, tile;
};
__device__ __forceinline__ Item item_of(uint32_t id, uint32_t key_heads, uint32_t group, uint32_t tiles)
{
    if (key_heads % 8 == 0) {
        const uint32_t own = key_heads / 8 * group, die = id % 8, j = id / 8, at = j % own;
        return Item{(int)((at / group * 8 + die) * group + at % group), (int)(tiles - 1 - j / own)};
    }
    const uint32_t heads = key_heads * group;
    return Item{(int)(id % heads), (int)(tiles - 1 - id / heads)};
}

// Turns of a shared tile in LDS: the one that is worked on and those on their way.
constexpr int turns_of(int dp, bool shared, int rows) { return !shared ? 1 : dp * rows >= 8192 ? 2 : 3; }

// ---- host

// Into how many parts the long axis of `blocks` workgroups is cut, each of up to `chain` steps, `held` of them on the device at once.  A step takes alone_us
// microseconds where a workgroup goes through its steps by itself, and full_us where all are at work (and a quarter of a workgroup's steps is left when the others are done); a part has fewer steps to go through in turn, but
// leaves sums (of sum_bytes) that one more launch reads again, at 4 TB/s (they are written while others compute).  other_us: what else the device does in the same launch.
// (Without that quarter, us a call: 2 x 3000 causal tokens, 3 heads of 128, 50 where this takes 44, their gradients 101 and 114; 200 queries and 9000 keys, 4 heads of 32, 34 and 28,
// gradients 32 and 36; 5417 causal tokens, 4 heads of 64, 46 and 51.  Parts from no gain at all on, not from a tenth: the same in all of these.)
inline int parts_of(double blocks, int64_t chain, bool causal, double held, double alone_us, double full_us, double sum_bytes, double other_us = 0.0)
{
    int best = 1;
    double least = 0;
    const double share = blocks * (double)chain * (causal ? 0.5 : 1.0) / held * full_us + other_us;
    for (int p = 1; p == 1 || (p <= 64 && 2 * p <= chain); p += p < 8 ? 1 : p / 4) {
        const double steps = (double)((chain + p - 1) / p) * alone_us, both = share + 0.25 * steps, us = (steps > both ? steps : both) + (p > 1 ? 5.0 + p * sum_bytes / 4e6 : 0.0);
        if (p == 1 || us < (best == 1 ? 0.9 : 1.0) * least) {
            best = p;
            least = us;
        }
    }
    return best;
}

bool heads_ok(const pruner_heads* h);
// Everything that is refused about sizes and pointers but outputs; fills the kernels' arguments.
int attention_args(const pruner_attention* a, const pruner_heads* q, const pruner_heads* k, const pruner_heads* v, Args* out);
bool attention_sizes_ok(const pruner_attention* a);
Heads heads_of(const pruner_heads* h);
inline int padded_dim(int head_dim) { return head_dim <= 32 ? 32 : head_dim <= 64 ? 64 : 128; }

}  // namespace att
}  // namespace pruner
