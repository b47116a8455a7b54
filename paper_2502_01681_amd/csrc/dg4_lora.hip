// The Q|K|V projection with low-rank adapters: [Q|K|V][r] = S[r] W + gain_a (S[r] D_a) U_a with a = adapter[r], for rows of
// many circuits at once, each with its own adapter or none.
//
//  lora_pack_kernel      lays W, D_a and U_a out once in matrix-core operand order.
//  lora_stream_kernel    a tile of 32 rows goes to LDS, the output columns take S W, streaming from the L2, then T U_a on
//                        top in the same accumulators, with T = gain (S D_a) for every row by its own adapter: fp32, and
//                        calls with few rows.
//  lora_resident_kernel  the same with W in registers and a workgroup walking over tiles of 64 rows, half of its waves
//                        fetching rows and forming T ahead of the others: bfloat16, many rows.
//
// A row takes 2 D 3D + 2 R 4D products and 4 D elements of memory: in bfloat16 the memory is the bound, in fp32 the products.
//
// A row's arithmetic is the same in either kernel, whatever else its tile holds and however many rows a call covers: the
// products of a row on the matrix cores do not see the other rows, T always comes from the same chain of 16x16 products, and
// where rows of a tile differ in their adapter each adapter's product is formed apart and kept for its own rows only (so
// nothing of another circuit's adapter, not even a NaN, reaches a row).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "dg4_device.h"
#include "dg4_internal.h"
#include "dg4_rowops.h"

namespace {

// Weights are the A operand of the 32x32 products and the rows the B operand, so that a lane's 16 accumulators belong to one
// row; with column 16 hi + 4 a + b at operand row 8 a + 4 hi + b they are 16 neighbouring columns.
__device__ __forceinline__ int column_of(int m) { return 16 * ((m >> 2) & 1) + 4 * (m >> 3) + (m & 3); }

// Calls with up to so many elements of S split the columns over workgroups. Measured, split | not split, in us, rank 16:
// bfloat16 at hidden 256, 4000 rows 8.8 | 9.9, 8000 rows 12.7 | 13.5, 10,000 rows 15.8 | 14.0; at 128, 4000 rows 5.5 | 9.7,
// 14,000 rows 8.9 | 9.8; fp32 at 256, 4000 rows 28.9 | 43.9, 8000 rows 44.6 | 41.3, 16,000 rows 78.6 | 64.9; at 128, 4000 rows
// 11.7 | 15.0, 12,000 rows 21.5 | 22.4, 16,000 rows 24.7 | 22.9, 24,000 rows 34.3 | 30.7. Other ranks cross within a few per cent of the
// same places: bfloat16 at 256, 8000 rows, rank 1 11.9 | 11.1, rank 64 17.4 | 18.2; fp32 at 128, 14,000 rows 22.3 | 21.0 and 34.2 | 35.8.
// Rows with 16 adapters in any order: 8000 rows 34.8 | 44.9, 10,000 47.2 | 45.1; fp32 at 128, 14,000 rows 77.7 | 68.3.
template <typename T> constexpr int64_t SPREAD_ELEMENTS = sizeof(T) == 2 ? 1 << 21 : 7 << 18;
template <typename T> constexpr int PIECE = 16 / (int)sizeof(T);      // elements of 16 bytes
inline int rank8(int rank) { return (rank + 7) / 8 * 8; }

// W: unit (tile * KC + c) * 64 + lane holds rows k = (2c + lane/32) E .. + E-1 of column 32 tile + column_of(lane % 32).
// Down: per adapter, unit (k/E) * rank + n holds rows k .. k+E-1 of column n. Up: per adapter, unit (q/E) * 3D + column holds rows
// q .. q+E-1, zero from `rank` on (up to the next multiple of eight).
template <typename T, int D>
__global__ void lora_pack_kernel(dg4_lora_pack_args p)
{
    constexpr int E = PIECE<T>, KC = D / (2 * E);
    const int64_t w_units = (int64_t)3 * D * D / E, down_units = (int64_t)D / E * p.rank, up_units = (int64_t)3 * D * p.rank8 / E;
    const int64_t all = w_units + p.n_adapters * (down_units + up_units);
    for (int64_t u = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; u < all; u += (int64_t)gridDim.x * blockDim.x) {
        T piece[E];
        T* dst;
        if (u < w_units) {
            const int lane = (int)(u & 63);
            const int c = (int)((u >> 6) % KC), tile = (int)((u >> 6) / KC);
            const int col = tile * 32 + column_of(lane & 31), k0 = (2 * c + (lane >> 5)) * E;
#pragma unroll
            for (int i = 0; i < E; ++i) piece[i] = ((const T*)p.w)[(int64_t)(k0 + i) * (3 * D) + col];
            dst = (T*)p.w_packed + u * E;
        } else if (u < w_units + p.n_adapters * down_units) {
            const int64_t v = u - w_units, a = v / down_units, x = v % down_units;
            const int n = (int)(x % p.rank), k0 = (int)(x / p.rank) * E;
#pragma unroll
            for (int i = 0; i < E; ++i) piece[i] = ((const T*)p.down)[(a * D + k0 + i) * p.rank + n];
            dst = (T*)p.down_packed + v * E;
        } else {
            const int64_t v = u - w_units - p.n_adapters * down_units, a = v / up_units, x = v % up_units;
            const int col = (int)(x % (3 * D)), q0 = (int)(x / (3 * D)) * E;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                if (q0 + i < p.rank) piece[i] = ((const T*)p.up)[(a * p.rank + q0 + i) * (3 * D) + col];
                else piece[i] = T{};
            }
            dst = (T*)p.up_packed + v * E;
        }
        *(uint4*)dst = *(const uint4*)piece;
    }
    if (blockIdx.x == 0)
        for (int64_t a = threadIdx.x; a < p.n_adapters; a += blockDim.x) p.gain_packed[a] = p.gain ? p.gain[a] : 1.f;
}

constexpr int ROWS = 32;                          // rows of a product, and of a tile of the streaming kernel
constexpr int RANKS = 8;                          // ranks per chunk of T U_a, either type

// Rows of T in LDS, elements: bfloat16 keeps T as a sum of two (high parts, then low parts), so that the product with U_a
// loses nothing that the output's own rounding would not
template <typename T> __host__ __device__ constexpr int low_stride(int r8) { return sizeof(T) == 2 ? 2 * r8 + 8 : r8 + 4; }

// One step of a 16x16 product: sixteen bytes of either operand, of row lane % 16 of each, part lane / 16 of the step's 4 E
// elements; accumulator i of a lane is row 4 (lane / 16) + i of the first operand, row lane % 16 of the second.
__device__ __forceinline__ void mma16(const uint4& a, const uint4& b, f32x4& c, bf16_t)
{
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ void mma16(const uint4& a, const uint4& b, f32x4& c, float)
{
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
}

// The sixteen columns of D_a from q0 on, as operand of all its steps
template <typename T, int D> constexpr int DOWN_STEPS = D / (4 * PIECE<T>);
template <typename T, int D>
__device__ __forceinline__ void fetch_down(const dg4_lora_args& p, int a, int q0, int lane, uint4 (&d)[DOWN_STEPS<T, D>])
{
    // (columns behind the last rank are not used)
    const uint4* src = (const uint4*)p.down_packed + ((int64_t)a * (D / PIECE<T>) + lane / 16) * p.rank + min(q0 + lane % 16, p.rank - 1);
#pragma unroll
    for (int k = 0; k < DOWN_STEPS<T, D>; ++k) d[k] = src[4 * k * p.rank];
}
// Sixteen rows of S (in LDS, `stride` elements apart) times sixteen columns of D_a: a lane has four columns of row lane % 16
template <typename T, int D>
__device__ __forceinline__ f32x4 down_product(const uint4 (&d)[DOWN_STEPS<T, D>], const T* rows, int stride, int lane)
{
    f32x4 sum = { 0.f, 0.f, 0.f, 0.f };
    const T* row = rows + (lane % 16) * stride + lane / 16 * PIECE<T>;
#pragma unroll
    for (int k = 0; k < DOWN_STEPS<T, D>; ++k) mma16(d[k], *(const uint4*)(row + 4 * k * PIECE<T>), sum, T{});
    return sum;
}
// A lane's four ranks q .. q + 3 of a row of T, into that row in LDS
template <typename T> __device__ __forceinline__ void put_low(T* row, int q, int rank, int r8, const f32x4& sum, float gain)
{
    if (q >= r8) return;
    float v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = q + k < rank ? sum[k] * gain : 0.f;
    if constexpr (sizeof(T) == 2) {
        // The high part is cut off towards zero, strictly below v, so that the low part is not zero and has v's sign: where a
        // number of U_a is infinite, both products are the infinity that v times it is. What is left out is at most 2^-16 of v.
        // (Rounded to nearest, the parts gave a NaN there wherever the low one was zero or had the other sign, and a high part of
        // infinity from 3.396e38 on.) An infinity is the largest number and an infinity; a NaN stays one.
        uint32_t h[4];
        float rest[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            h[k] = v[k] == 0.f ? 0u : (__float_as_uint(v[k]) - 1u) >> 16;
            rest[k] = v[k] - __uint_as_float(h[k] << 16);
        }
        *(uint2*)(row + q) = make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
        *(uint2*)(row + r8 + q) = make_uint2(pack_bf16x2(rest[0], rest[1]), pack_bf16x2(rest[2], rest[3]));
    } else {
        *(float4*)(row + q) = make_float4(v[0], v[1], v[2], v[3]);
    }
}
// T of sixteen rows whose adapters differ, ranks q0 .. q0 + 15: adapter after adapter, kept for its own rows
template <typename T, int D>
__device__ __forceinline__ f32x4 down_product_mixed(const dg4_lora_args& p, int mine, int q0, const T* rows, int stride, int lane)
{
    f32x4 kept = { 0.f, 0.f, 0.f, 0.f };
    uint64_t todo = __ballot(mine >= 0);
    while (todo) {
        const int a = __builtin_amdgcn_readlane(mine, (int)__builtin_ctzll(todo));
        todo &= ~__ballot(mine == a);
        uint4 d[DOWN_STEPS<T, D>];
        fetch_down<T, D>(p, a, q0, lane, d);
        const f32x4 sum = down_product<T, D>(d, rows, stride, lane);
#pragma unroll
        for (int i = 0; i < 4; ++i) kept[i] = mine == a ? sum[i] : kept[i];
    }
    return kept;
}

// The adapters of a wave's rows; a row has one or more lanes (-1: none).
struct Adapters {
    int mine, first;                              // this lane's row's; row 0's
    bool any, one;                                // some row has one; all rows have the same
    __device__ __forceinline__ void set(int id, int64_t n_adapters)
    {
        mine = id >= 0 && id < n_adapters ? id : -1;
        first = __builtin_amdgcn_readfirstlane(mine);
        any = __ballot(mine >= 0) != 0;
        one = __ballot(mine != first) == 0;
    }
};

// Chunk c of T as operand: bfloat16 has the high parts of eight ranks in one half of the wave and their low parts in the other,
// against the same eight rows of U_a
template <typename T> __device__ __forceinline__ uint4 low_operand(const dg4_lora_args& p, const T* low, int c, int n, int hi)
{
    const T* row = low + n * low_stride<T>(p.rank8);
    return *(const uint4*)(sizeof(T) == 2 ? row + hi * p.rank8 + c * 8 : row + (2 * c + hi) * 4);
}

// T U_a for a column tile, on top of S W in the accumulators, two chunks of ranks at a time. A tile of rows with one adapter has its
// first two chunks requested ahead, by first(). Otherwise adapter after adapter, the next two chunks (of the same adapter or the
// next) requested before these are multiplied; the sums are kept for its own rows.
template <typename T, int D> struct UpProduct {
    uint4 up[2];
    __device__ __forceinline__ static void fetch(const dg4_lora_args& p, int a, int c0, int tile, int n, int hi, uint4 (&to)[2])
    {
        constexpr int E = PIECE<T>;
        const int chunks = p.rank8 / RANKS;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int at = min(c0 + c, chunks - 1), unit = sizeof(T) == 2 ? at : 2 * at + hi;
            to[c] = ((const uint4*)p.up_packed)[((int64_t)a * (p.rank8 / E) + unit) * (3 * D) + tile * 32 + column_of(n)];
        }
    }
    __device__ __forceinline__ void first(const dg4_lora_args& p, const Adapters& ad, int tile, int n, int hi)
    {
        if (ad.any && ad.one) fetch(p, ad.first, 0, tile, n, hi, up);
    }
    __device__ __forceinline__ void run_one(const dg4_lora_args& p, const Adapters& ad, const T* low, int tile, int n, int hi, f32x16& acc)
    {
        const int chunks = p.rank8 / RANKS;
        for (int c0 = 0; c0 < chunks; c0 += 2) {
#pragma unroll
            for (int c = 0; c < 2; ++c)
                if (c0 + c < chunks) Mma<T>::run(up[c], low_operand(p, low, c0 + c, n, hi), acc);
            if (c0 + 2 < chunks) fetch(p, ad.first, c0 + 2, tile, n, hi, up);
        }
    }
    __device__ __forceinline__ static void run_mixed(const dg4_lora_args& p, const Adapters& ad, const T* low, int tile, int n, int hi, f32x16& acc)
    {
        const int chunks = p.rank8 / RANKS;
        uint64_t todo = __ballot(ad.mine >= 0);
        int a = __builtin_amdgcn_readlane(ad.mine, (int)__builtin_ctzll(todo));
        todo &= ~__ballot(ad.mine == a);
        uint4 now[2], next[2];
        fetch(p, a, 0, tile, n, hi, now);
        f32x16 part = acc;                        // (S W for the rows whose turn has not come; the others are not kept again)
        for (int c0 = 0;;) {
            const bool ends = c0 + 2 >= chunks, more = !ends || todo != 0;
            const int a_next = ends && todo ? __builtin_amdgcn_readlane(ad.mine, (int)__builtin_ctzll(todo)) : a;
            if (more) fetch(p, a_next, ends ? 0 : c0 + 2, tile, n, hi, next);
#pragma unroll
            for (int c = 0; c < 2; ++c)
                if (c0 + c < chunks) Mma<T>::run(now[c], low_operand(p, low, c0 + c, n, hi), part);
            if (ends) {
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[i] = ad.mine == a ? part[i] : acc[i];
                part = acc;
            }
            if (!more) break;
            now[0] = next[0]; now[1] = next[1];
            c0 = ends ? 0 : c0 + 2;
            todo &= ~__ballot(ad.mine == a_next);
            a = a_next;
        }
    }
};

// Where Q, K and V go: K's distance from Q and V's from K, to be added by mask. (Chosen with ?: per lane, the address is loaded
// from the kernel's arguments, or from the stack, for every store, and every store waits for those before it.)
struct Outputs {
    uint64_t q, k_q, v_k;
    __device__ __forceinline__ explicit Outputs(const dg4_lora_args& p)
        : q((uint64_t)p.out[0]), k_q((uint64_t)p.out[1] - (uint64_t)p.out[0]), v_k((uint64_t)p.out[2] - (uint64_t)p.out[1]) {}
    template <typename T, int D> __device__ __forceinline__ T* at(int64_t row, int col) const
    {
        const uint64_t base = q + (k_q & (uint64_t)((int64_t)(D - 1 - col) >> 63)) + (v_k & (uint64_t)((int64_t)(2 * D - 1 - col) >> 63));
        return (T*)base + row * D + col % D;
    }
};

// JT finished column tiles of the wave's rows, through its own corner of LDS (a wave's LDS operations complete in order), as
// 16-byte pieces of rows to Q, K or V, past the caches, which are the weights' (a million rows of bfloat16 at hidden 256: 641 us, through
// them 652)
template <typename T, int D, int JT, int STRIDE>
__device__ __forceinline__ void put_tiles(const Outputs& to, const f32x16* acc, T* out_rows, int64_t r0, int64_t r_end, int tile, int lane)
{
    constexpr int E = PIECE<T>, PPR = JT * 32 / E;             // pieces per row
    const int n = lane & 31, hi = lane >> 5;
#pragma unroll
    for (int j = 0; j < JT; ++j) {
        uint4* dst = (uint4*)(out_rows + n * STRIDE + j * 32 + 16 * hi);
        const f32x16& x = acc[j];
        if constexpr (sizeof(T) == 2) {
            dst[0] = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
            dst[1] = make_uint4(pack_bf16x2(x[8], x[9]), pack_bf16x2(x[10], x[11]), pack_bf16x2(x[12], x[13]), pack_bf16x2(x[14], x[15]));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                dst[i] = make_uint4(__float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]), __float_as_uint(x[4 * i + 2]), __float_as_uint(x[4 * i + 3]));
        }
    }
    constexpr int PIECES = ROWS * PPR / 64;
    uint4 v[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) v[i] = *((const uint4*)(out_rows + (lane + 64 * i) / PPR * STRIDE) + (lane + 64 * i) % PPR);
    const int rows = (int)min((int64_t)ROWS, r_end - r0);
    T* at = to.at<T, D>(r0 + lane / PPR, tile * 32 + lane % PPR * E);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int piece = lane + 64 * i, row = piece / PPR;
        if (64 % PPR != 0 && i > 0) at = to.at<T, D>(r0 + row, tile * 32 + piece % PPR * E);
        if (row < rows) store_stream(at, v[i]);
        at += 64 / PPR * D;
    }
}

// LDS of the streaming kernel, in bytes: the rows, T, rows on their way out
template <typename T, int D> struct StreamLds {
    static constexpr int S_STRIDE = D + PIECE<T>;                                  // elements
    static constexpr int S_BYTES = ROWS * S_STRIDE * (int)sizeof(T);
    static constexpr int O_STRIDE = 32 + PIECE<T>;
    __host__ __device__ static constexpr int out_at(int r8) { return S_BYTES + ROWS * low_stride<T>(r8) * (int)sizeof(T); }
    __host__ __device__ static constexpr int bytes(int r8) { return out_at(r8) + 4 * ROWS * O_STRIDE * (int)sizeof(T); }
};

// A workgroup of four waves takes a tile of rows, a wave one column tile after the other: weights arrive from the L2 a few chunks before
// they are multiplied, the next pass's among them, and two or three workgroups to a compute unit fill each other's waits. SPREAD, for
// calls with few rows, where latency counts: a wave takes one column tile, the others go to 3D/32/4 workgroups along y, and a
// tile holds p.tile_rows <= 32 rows (the rest of its operand repeats the last).
// Measured, rank 16: 64 rows of bfloat16 at hidden 256, each with its own adapter, 5.2 us, waits of memory after one another
// (adapters, D_a, U_a) and two products that hang on each other; 20,257 rows of fp32 at 128 in 28 us, 77 TFLOP/s, bound by the
// matrix cores of the compute units that get three tiles (634 tiles on 256; a tile is some 7 us of products); 150,000 rows of fp32
// at 256 in 548 us, 120 TFLOP/s. Two or three column tiles to a wave at once are no faster (552; at 128, 24,000 rows 34 for 31),
// nor are three workgroups to a compute unit with D_a fetched where it is used (555).
template <typename T, int D, bool SPREAD>
__global__ __launch_bounds__(256, 2) void lora_stream_kernel(dg4_lora_args p)
{
    constexpr int E = PIECE<T>, KC = D / (2 * E), TILES = 3 * D / 32, PASSES = SPREAD ? 1 : TILES / 4;
    using L = StreamLds<T, D>;
    constexpr int RING = sizeof(T) == 2 ? 8 : 4;  // chunks of weights requested ahead
    static_assert(KC % RING == 0, "the ring's place of a chunk is the same in every pass");
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, hi = lane >> 5;
    const int tile_rows = SPREAD ? p.tile_rows : ROWS;
    const int64_t r0 = p.row_begin + (int64_t)blockIdx.x * tile_rows;
    const int64_t r_end = min(p.row_end, r0 + tile_rows);
    auto row_at = [&](int i) { const int64_t r = r0 + i; return r < r_end ? r : r_end - 1; };

    T* const rows = (T*)smem;
    T* const low = (T*)(smem + L::S_BYTES);
    T* const out_rows = (T*)(smem + L::out_at(p.rank8)) + wave * ROWS * L::O_STRIDE;

    // Requests, in the order in which they are waited for: the rows' adapters, the rows, the first chunks of weights
    const int id = p.adapter ? p.adapter[row_at(n)] : -1;
    constexpr int CPR = D / E, PIECES = ROWS * CPR / 256;
    uint4 row_piece[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int piece = (int)threadIdx.x + 256 * i;
        row_piece[i] = *((const uint4*)((const T*)p.s + row_at(piece / CPR) * D) + piece % CPR);
    }
    const int tile0 = SPREAD ? (int)blockIdx.y * 4 + wave : wave * PASSES;
    const uint4* wp = (const uint4*)p.w_packed + (int64_t)tile0 * KC * 64 + lane;
    uint4 ring[RING];
#pragma unroll
    for (int c = 0; c < RING; ++c) ring[c] = wp[c * 64];

    Adapters ad;
    ad.set(id, p.n_adapters);
    // T: waves 0 and 2 take rows 0 .. 15, waves 1 and 3 rows 16 .. 31, each every second sixteen ranks
    const int half = wave & 1;
    Adapters ad16;
    ad16.set(__shfl(ad.mine, half * 16 + lane % 16), p.n_adapters);
    const bool down_ahead = ad16.any && ad16.one && wave / 2 * 16 < p.rank;
    uint4 d[DOWN_STEPS<T, D>];
    if (down_ahead) fetch_down<T, D>(p, ad16.first, wave / 2 * 16, lane, d);
    UpProduct<T, D> up;
    up.first(p, ad, tile0, n, hi);
    const float gain = ad16.mine >= 0 ? p.gain_packed[ad16.mine] : 0.f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int piece = (int)threadIdx.x + 256 * i;
        *((uint4*)(rows + (piece / CPR) * L::S_STRIDE) + piece % CPR) = row_piece[i];
    }
    __syncthreads();
    const Outputs outputs(p);
    auto row_operand = [&](int c) __attribute__((always_inline)) { return *(const uint4*)(rows + n * L::S_STRIDE + (2 * c + hi) * E); };
    // (unrolled, so that the weights on their way are waited for one by one and not behind the stores of a pass)
#pragma unroll
    for (int pass = 0; pass < PASSES; ++pass) {
        f32x16 acc;
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] = 0.f;
        const int tile = tile0 + pass;
        uint4 b[2];                               // rows as operand: this chunk's and the next's
        b[0] = row_operand(0);
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            if (c + 1 < KC) b[(c + 1) & 1] = row_operand(c + 1);
            Mma<T>::run(ring[c % RING], b[c & 1], acc);
            const int ahead = pass * KC + c + RING;            // chunk, on through the passes
            if (ahead < PASSES * KC) ring[c % RING] = wp[ahead * 64];
            __builtin_amdgcn_sched_barrier(0);
        }
        if (ad.any) {
            if (pass == 0) {                      // (T is needed from here on; its D_a has travelled under the first pass)
                for (int q0 = wave / 2 * 16; ad16.any && q0 < p.rank; q0 += 32) {
                    const T* mine = rows + half * 16 * L::S_STRIDE;
                    f32x4 sum;
                    if (ad16.one) {
                        if (q0 >= 32) fetch_down<T, D>(p, ad16.first, q0, lane, d);
                        sum = down_product<T, D>(d, mine, L::S_STRIDE, lane);
                    } else {
                        sum = down_product_mixed<T, D>(p, ad16.mine, q0, mine, L::S_STRIDE, lane);
                    }
                    // (rows without an adapter get, or have, what is kept for no row)
                    put_low<T>(low + (half * 16 + lane % 16) * low_stride<T>(p.rank8), q0 + lane / 16 * 4, p.rank, p.rank8, sum, gain);
                }
                __syncthreads();
            }
            if (ad.one) up.run_one(p, ad, low, tile, n, hi, acc);
            else up.run_mixed(p, ad, low, tile, n, hi, acc);
        }
        if (pass + 1 < PASSES) up.first(p, ad, tile + 1, n, hi);
        put_tiles<T, D, 1, L::O_STRIDE>(outputs, &acc, out_rows, r0, r_end, tile, lane);
    }
}

// LDS of the resident kernel, in bytes: two buffers each of the rows of a tile, of their T and of their adapters; U_a of
// this workgroup's columns; rows on their way out
template <int D, int JT> struct WalkLds {
    static constexpr int TILE = 64;
    static constexpr int S_STRIDE = D + 8;                                         // elements
    static constexpr int S_BYTES = TILE * S_STRIDE * 2;
    static constexpr int O_STRIDE = JT * 32 + 8;
    __host__ __device__ static constexpr int low_bytes(int r8) { return TILE * low_stride<bf16_t>(r8) * 2; }
    __host__ __device__ static constexpr int ids_at(int r8) { return 2 * (S_BYTES + low_bytes(r8)); }
    __host__ __device__ static constexpr int up_at(int r8) { return ids_at(r8) + 2 * TILE * 4; }
    // (operand units of 16 bytes: [wave][chunk][column tile][32])
    __host__ __device__ static constexpr int out_at(int r8) { return up_at(r8) + 4 * (r8 / RANKS) * JT * 32 * 16; }
    __host__ __device__ static constexpr int bytes(int r8) { return out_at(r8) + 4 * ROWS * O_STRIDE * 2; }
};

// bfloat16, many rows. A workgroup of eight waves per compute unit keeps its share of W in the registers of four of them, JT
// column tiles each: all columns at hidden 128 (96 registers), one of Q, K and V at 256 (128 registers; PARTS = 3; the
// workgroups of one walk sit on one XCD, so that the rows come from memory once: 0.59 GB fetched where S has 0.51). These four
// multiply and store and wait for no load; U_a sits in LDS until the adapter changes. The other four, sixteen rows each, request
// the rows two tiles ahead, put the next tile's into LDS and form their T, with D_a in registers until the adapter changes. One
// barrier per tile. A tile whose rows differ in their adapter goes half by half, U_a of one adapter after the other.
// Measured, rank 16, a million rows of 40 circuits with 16 adapters at hidden 256: 631 us (of 200 circuits 662: most tiles at a change
// of adapter are mixed), 0.68 PFLOP/s and 3.3 TB/s; the multiplying waves bind it, one to each SIMD, 2900 cycles of S W (the matrix
// cores: 2050), 850 of T U and 2600 to hand a tile to the memory, one after the other. Without the stores 500 us; two workgroups of four
// waves to a compute unit instead 680 us; rows in registers and W from the L2 654 us. 500,000 rows at 128: 121 us, 4.2 TB/s.
// Adapters in any order, 200,000 rows: a tile forms T U of each of its adapters for all its rows. Of 4, 16 and 64 adapters at 256
// 259, 647 and 1070 us (in runs 130 to 137), at 128 104, 271 and 461 (45 to 48); the streaming kernel, not split, 268, 633 and 1030,
// at 128 99, 226 and 366, but 177 and 57 in runs.
template <int D, int PARTS>
__global__ __launch_bounds__(512, 2) void lora_resident_kernel(dg4_lora_args p)
{
    typedef bf16_t T;
    constexpr int E = PIECE<T>, KC = D / (2 * E), JT = 3 * D / 32 / PARTS / 4;
    using L = WalkLds<D, JT>;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, hi = lane >> 5;
    // workgroups go to the eight XCDs in turn
    const int walks = (int)gridDim.x / PARTS, whole = walks / 8 * (8 * PARTS);     // (those of the walks left over by eight go apart)
    const int xcd = (int)blockIdx.x & 7, slot = (int)blockIdx.x >> 3, over = (int)blockIdx.x - whole;
    const int share = (over < 0 ? slot : over) % PARTS, walk = over < 0 ? slot / PARTS * 8 + xcd : (whole + over) / PARTS;
    const int64_t tiles = (p.row_end - p.row_begin + L::TILE - 1) / L::TILE;
    const int64_t steps = walk < tiles ? (tiles - walk + walks - 1) / walks : 0;   // tiles walk, walk + walks, ...
    if (steps == 0) return;
    auto rows_of = [&](int64_t step) { return (T*)(smem + (step & 1) * L::S_BYTES); };
    auto low_of = [&](int64_t step) { return (T*)(smem + 2 * L::S_BYTES + (step & 1) * L::low_bytes(p.rank8)); };
    auto ids_of = [&](int64_t step) { return (int*)(smem + L::ids_at(p.rank8)) + (step & 1) * L::TILE; };

    if (wave >= 4) {
        // rows 16 h .. 16 h + 15 of every tile
        const int h = wave - 4;
        constexpr int CPR = D / E, RPL = 64 / CPR, LOADS = 16 / RPL;               // rows per load instruction; a wave's loads of a tile
        typedef uint32_t Pieces __attribute__((ext_vector_type(4 * LOADS)));       // (an array was kept in scratch memory)
        struct Ahead { Pieces piece; int id; };
        auto request = [&](int64_t step, Ahead& to) __attribute__((always_inline)) {
            const int64_t r0 = p.row_begin + (walk + step * walks) * L::TILE + 16 * h;
            auto row_at = [&](int i) { return min(r0 + i, p.row_end - 1); };
            to.id = p.adapter ? p.adapter[row_at(lane % 16)] : -1;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const uint4 v = *((const uint4*)((const T*)p.s + row_at(i * RPL + lane / CPR) * D) + lane % CPR);
                to.piece[4 * i] = v.x; to.piece[4 * i + 1] = v.y; to.piece[4 * i + 2] = v.z; to.piece[4 * i + 3] = v.w;
            }
        };
        uint4 d[DOWN_STEPS<T, D>];
        int held = -1;                            // the adapter whose first sixteen ranks d holds
        auto put = [&](int64_t step, const Ahead& from) __attribute__((always_inline)) {
            Adapters ad;
            ad.set(from.id, p.n_adapters);
            const float gain = ad.mine >= 0 ? p.gain_packed[ad.mine] : 0.f;
            if (ad.any && ad.one && ad.first != held) { fetch_down<T, D>(p, ad.first, 0, lane, d); held = ad.first; }
            T* const rows = rows_of(step) + 16 * h * L::S_STRIDE;
#pragma unroll
            for (int i = 0; i < LOADS; ++i)
                *((uint4*)(rows + (i * RPL + lane / CPR) * L::S_STRIDE) + lane % CPR) =
                    make_uint4(from.piece[4 * i], from.piece[4 * i + 1], from.piece[4 * i + 2], from.piece[4 * i + 3]);
            if (lane < 16) ids_of(step)[16 * h + lane] = ad.mine;
            if (!ad.any) return;
            // (the rows are this wave's own: its LDS operations complete in order)
            T* const low = low_of(step) + (16 * h + lane % 16) * low_stride<T>(p.rank8);
            for (int q0 = 0; q0 < p.rank; q0 += 16) {
                f32x4 sum;
                if (!ad.one) {
                    sum = down_product_mixed<T, D>(p, ad.mine, q0, rows, L::S_STRIDE, lane);
                } else if (q0 == 0) {
                    sum = down_product<T, D>(d, rows, L::S_STRIDE, lane);
                } else {
                    uint4 more[DOWN_STEPS<T, D>];
                    fetch_down<T, D>(p, ad.first, q0, lane, more);
                    sum = down_product<T, D>(more, rows, L::S_STRIDE, lane);
                }
                put_low<T>(low, q0 + lane / 16 * 4, p.rank, p.rank8, sum, gain);
            }
        };
        Ahead even, odd;
        request(0, even);
        if (steps > 1) request(1, odd);
        put(0, even);
        if (steps > 2) request(2, even);
        __syncthreads();
        for (int64_t step = 0; step < steps; step += 2) {
            // while tile `step` is multiplied
            if (step + 1 < steps) put(step + 1, odd);
            if (step + 3 < steps) request(step + 3, odd);
            __syncthreads();
            if (step + 1 >= steps) return;
            if (step + 2 < steps) put(step + 2, even);
            if (step + 4 < steps) request(step + 4, even);
            __syncthreads();
        }
        return;
    }

    const Outputs outputs(p);
    const int tile0 = (share * 4 + wave) * JT;
    uint4 w[JT][KC];
    {
        const uint4* wp = (const uint4*)p.w_packed + (int64_t)tile0 * KC * 64 + lane;
#pragma unroll
        for (int j = 0; j < JT; ++j)
#pragma unroll
            for (int c = 0; c < KC; ++c) w[j][c] = wp[(j * KC + c) * 64];
        // (used here, so that they are waited for here and not, behind the stores of the step before, in every step)
        typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int j = 0; j < JT; ++j)
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                u32x4 pin = __builtin_bit_cast(u32x4, w[j][c]);
                __asm__ volatile("" : "+v"(pin));
                w[j][c] = __builtin_bit_cast(uint4, pin);
            }
    }
    const int chunks = p.rank8 / RANKS;
    uint4* const up_held = (uint4*)(smem + L::up_at(p.rank8)) + wave * chunks * JT * 32;     // this wave's columns
    int held = -1;                                // the adapter it holds
    T* const out_rows = (T*)(smem + L::out_at(p.rank8)) + wave * ROWS * L::O_STRIDE;
    __syncthreads();
    for (int64_t step = 0; step < steps; ++step) {
        // (a lane number of its own in every step: what is worked out from it is not kept over the loop, where W has the registers)
        int lane = (int)threadIdx.x & 63;
        __asm__ volatile("" : "+v"(lane));
        const int n = lane & 31, hi = lane >> 5;
        const T* rows = rows_of(step) + n * L::S_STRIDE + hi * E;
        const T* low = low_of(step);
        constexpr int H = L::TILE / ROWS;         // halves of the tile, multiplied together if all rows have one adapter
        constexpr int WINDOW = 2;                 // rows as operand: this chunk's and the next's
        // COUNT halves from `t0` on times W
        auto multiply = [&](auto count, int t0, f32x16 (*acc)[JT]) __attribute__((always_inline)) {
            constexpr int COUNT = count;
            uint4 b[WINDOW][COUNT];
            auto fetch_rows = [&](int c) __attribute__((always_inline)) {
#pragma unroll
                for (int t = 0; t < COUNT; ++t) b[c % WINDOW][t] = *(const uint4*)(rows + (t0 + t) * ROWS * L::S_STRIDE + 2 * c * E);
            };
            fetch_rows(0);
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                if (c + WINDOW - 1 < KC) fetch_rows(c + WINDOW - 1);
#pragma unroll
                for (int j = 0; j < JT; ++j)
#pragma unroll
                    for (int t = 0; t < COUNT; ++t) {
                        if (c == 0) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) acc[t][j][i] = 0.f;
                        }
                        Mma<T>::run(w[j][c], b[c % WINDOW][t], acc[t][j]);
                    }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        // T U_a on top for the same halves
        auto multiply_up = [&](auto count, int t0, int a, f32x16 (*acc)[JT]) __attribute__((always_inline)) {
            constexpr int COUNT = count;
            if (a != held) {                      // (32 lanes a column tile: either half of the wave multiplies the same rows of U_a)
                held = a;
                for (int c = hi; c < chunks; c += 2)
#pragma unroll
                    for (int j = 0; j < JT; ++j)
                        up_held[(c * JT + j) * 32 + n] = ((const uint4*)p.up_packed)[((int64_t)held * chunks + c) * (3 * D) + (tile0 + j) * 32 + column_of(n)];
            }
            for (int c0 = 0; c0 < chunks; c0 += 2) {
                uint4 x[2][COUNT], y[2][JT];
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int at = min(c0 + c, chunks - 1);
#pragma unroll
                    for (int t = 0; t < COUNT; ++t) x[c][t] = low_operand(p, low + (t0 + t) * ROWS * low_stride<T>(p.rank8), at, n, hi);
#pragma unroll
                    for (int j = 0; j < JT; ++j) y[c][j] = up_held[(at * JT + j) * 32 + n];
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    if (c0 + c < chunks) {
#pragma unroll
                        for (int j = 0; j < JT; ++j)
#pragma unroll
                            for (int t = 0; t < COUNT; ++t) Mma<T>::run(y[c][j], x[c][t], acc[t][j]);
                    }
                }
            }
        };
        const int64_t r0 = p.row_begin + (walk + step * walks) * L::TILE;
        int id[H];
#pragma unroll
        for (int t = 0; t < H; ++t) id[t] = ids_of(step)[t * ROWS + n];
        const int first = __builtin_amdgcn_readfirstlane(id[0]);
        if (__ballot(id[0] != first || id[H - 1] != first) == 0) {
            f32x16 acc[H][JT];
            multiply(std::integral_constant<int, H>{}, 0, acc);
            if (first >= 0) multiply_up(std::integral_constant<int, H>{}, 0, first, acc);
            __asm__ volatile("" : "+v"(lane));
#pragma unroll
            for (int t = 0; t < H; ++t) put_tiles<T, D, JT, L::O_STRIDE>(outputs, acc[t], out_rows, r0 + t * ROWS, p.row_end, tile0, lane);
        } else {
            // Adapter after adapter, on top of S W, kept for its own rows
#pragma unroll 1
            for (int t = 0; t < H; ++t) {
                const int mine = t == 0 ? id[0] : id[H - 1];
                f32x16 acc[1][JT];
                multiply(std::integral_constant<int, 1>{}, t, acc);
                uint64_t todo = __ballot(mine >= 0);
#pragma unroll 1
                while (todo) {
                    const int a = __builtin_amdgcn_readlane(mine, (int)__builtin_ctzll(todo));
                    todo &= ~__ballot(mine == a);
                    f32x16 part[1][JT];
#pragma unroll
                    for (int j = 0; j < JT; ++j) part[0][j] = acc[0][j];
                    multiply_up(std::integral_constant<int, 1>{}, t, a, part);
#pragma unroll
                    for (int j = 0; j < JT; ++j)
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[0][j][i] = mine == a ? part[0][j][i] : acc[0][j][i];
                }
                put_tiles<T, D, JT, L::O_STRIDE>(outputs, acc[0], out_rows, r0 + t * ROWS, p.row_end, tile0, lane);
            }
        }
        __syncthreads();
    }
}

template <typename T, int D>
int launch_pack(const dg4_lora_pack_args& a, hipStream_t s)
{
    constexpr int E = PIECE<T>;
    const int64_t units = (int64_t)3 * D * D / E + a.n_adapters * ((int64_t)D / E * a.rank + (int64_t)3 * D * a.rank8 / E);
    const unsigned grid = (unsigned)std::min<int64_t>((units + 255) / 256, 1 << 16);
    hipLaunchKernelGGL((lora_pack_kernel<T, D>), dim3(grid), dim3(256), 0, s, a);
    return hipGetLastError();
}

// (64 KB need no leave. It is given for the largest rank, so that a call of a smaller one in another thread takes none of it away
// between this and the launch.)
template <typename K> int allow_lds(K kernel, int bytes, int most)
{
    return bytes <= 65536 ? hipSuccess : hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, most);
}

template <typename T, int D>
int launch_proj(dg4_lora_args a, hipStream_t s)
{
    const int64_t rows = a.row_end - a.row_begin;
    if (rows * D <= SPREAD_ELEMENTS<T>) {
        const auto kernel = lora_stream_kernel<T, D, true>;
        // Rows per tile: few enough for two workgroups per compute unit. bfloat16 at 256, in us with 256, 512 and 1024 workgroups instead:
        // 64 rows with an adapter each 5.6, 5.1 and 5.1 (tiles of 2 rows and of 1), 170 rows 7.8, 6.5, 7.5, 340 rows 11.3, 8.4, 10.1; rows of
        // eight circuits in runs 4.5, 5.2, 5.1; 5.6, 6.3, 7.6; 5.6, 6.3, 8.6. fp32 at 128, 340 rows 11.1, 11.0, 15.3 and 8.1, 10.7, 15.3.
        a.tile_rows = 1;
        while (a.tile_rows < ROWS && rows * (3 * D / 128) > (int64_t)512 * a.tile_rows) a.tile_rows *= 2;
        const int smem = StreamLds<T, D>::bytes(a.rank8);
        if (const int e = allow_lds(kernel, smem, StreamLds<T, D>::bytes(DG4_MAX_RANK)); e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, dim3((unsigned)((rows + a.tile_rows - 1) / a.tile_rows), 3 * D / 128), dim3(256), smem, s, a);
    } else if constexpr (sizeof(T) == 2) {
        constexpr int PARTS = D == 256 ? 3 : 1;
        using L = WalkLds<D, 3 * D / 128 / PARTS>;
        const auto kernel = lora_resident_kernel<D, PARTS>;
        const int smem = L::bytes(a.rank8);
        if (const int e = allow_lds(kernel, smem, L::bytes(DG4_MAX_RANK)); e != hipSuccess) return e;
        int dev = 0, cus = 0;
        if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) return hipErrorInvalidDevice;
        // one workgroup per compute unit
        const int64_t walks = std::min<int64_t>(std::max(1, cus / PARTS), (rows + L::TILE - 1) / L::TILE);
        hipLaunchKernelGGL(kernel, dim3((unsigned)(PARTS * walks)), dim3(512), smem, s, a);
    } else {
        const auto kernel = lora_stream_kernel<T, D, false>;
        const int smem = StreamLds<T, D>::bytes(a.rank8);
        if (const int e = allow_lds(kernel, smem, StreamLds<T, D>::bytes(DG4_MAX_RANK)); e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, dim3((unsigned)((rows + ROWS - 1) / ROWS)), dim3(256), smem, s, a);
    }
    return hipGetLastError();
}

}  // namespace

int64_t dg4_lora_bytes(int dtype, int hidden, int64_t n_adapters, int rank, int64_t* down, int64_t* up, int64_t* gain)
{
    const int64_t es = dtype == DG4_F32 ? 4 : 2, d = hidden;
    *down = 3 * d * d * es;
    *up = *down + n_adapters * d * rank * es;
    *gain = *up + n_adapters * rank8(rank) * 3 * d * es;
    return *gain + (n_adapters * 4 + 255) / 256 * 256;
}
int dg4_launch_lora_pack(int dtype, int hidden, dg4_lora_pack_args a, hipStream_t s)
{
    a.rank8 = rank8(a.rank);
    if (dtype == DG4_F32) return hidden == 128 ? launch_pack<float, 128>(a, s) : launch_pack<float, 256>(a, s);
    return hidden == 128 ? launch_pack<bf16_t, 128>(a, s) : launch_pack<bf16_t, 256>(a, s);
}
int dg4_launch_lora_proj(int dtype, int hidden, dg4_lora_args a, hipStream_t s)
{
    a.rank8 = rank8(a.rank);
    if (dtype == DG4_F32) return hidden == 128 ? launch_proj<float, 128>(a, s) : launch_proj<float, 256>(a, s);
    return hidden == 128 ? launch_proj<bf16_t, 128>(a, s) : launch_proj<bf16_t, 256>(a, s);
}
