// Products of rows and weights in 4 bits, both by blocks of 32 along the summed axis (dg4_fp4.h), on the scaled matrix cores:
//
//  mx4_pack_kernel  a weight matrix once into blocks, in matrix-core operand order.
//  mx4_proj_kernel  [Q | K | V] = q(S) q(Wqkv): to rows, or Q to rows and K and V straight from the accumulators into the store
//                   in 4 bits, whose blocks are the heads of a row.
//  mx4_ffn_kernel   Out = LayerNorm(S + q(max(q(S) q(W1), 0)) q(W2)).
//
// Weights are the A operand of 32x32x64 products and rows the B operand, so that a lane's sixteen accumulators belong to one
// row; operand row 8 a + 4 hi + b is column 16 hi + 4 a + b of a tile, so they are sixteen neighbouring columns, half a block.
// A product of two codes is a whole number of quarters, up to 144 of them, under the powers of two of its blocks. Sums of k of them in fp32
// are exact where (largest by smallest power of two of the row) * (the same of the column) * 144 k is at most 2^24: with the two
// ratios together up to 2^9 at k = 128, 2^8 at 256, 2^7 at 512 and 2^6 at 1024.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "dg4_device.h"
#include "dg4_fp4.h"
#include "dg4_internal.h"

namespace {

__device__ __forceinline__ int column_of(int m) { return 16 * ((m >> 2) & 1) + 4 * (m >> 3) + (m & 3); }

constexpr int ROWS = 32;                          // rows of a tile

// A packed matrix [k, n]: unit (tile * k/64 + c) * 64 + lane, 16 bytes, is the block of rows 64 c + 32 (lane / 32) .. + 31 of column
// 32 tile + column_of(lane % 32). Behind the units, word (tile * C4 + c/4) * 64 + lane holds the block's scale in byte c % 4.
__host__ __device__ constexpr int scale_words(int k) { return (k / 64 + 3) / 4; }

// One thread per block: 32 rows of a column, whose neighbours other lanes take
template <typename T>
__global__ __launch_bounds__(256) void mx4_pack_kernel(dg4_mx4_pack_args p)
{
    const int kc = p.k / 64, c4 = scale_words(p.k);
    const int at = (int)(blockIdx.x * blockDim.x + threadIdx.x);
    if (at >= p.k / 32 * p.n) return;
    const int col = at % p.n, block = at / p.n;
    float x[32];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        x[i] = Elem<T>::load1(p.w, (int64_t)(32 * block + i) * p.n + col);
        top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    }
    const uint32_t byte = fp4_scale_byte(top);
    uint4 w = make_uint4(0, 0, 0, 0);
    const uint32_t scale = byte << 23;
    if (byte != FP4_BAD) w = make_uint4(fp4_put8(x, scale), fp4_put8(x + 8, scale), fp4_put8(x + 16, scale), fp4_put8(x + 24, scale));
    // column 16 hi + 4 a + b is operand row 8 a + 4 hi + b
    const int in_tile = col % 32, tile = col / 32, m = 8 * ((in_tile >> 2) & 3) + 4 * (in_tile >> 4) + (in_tile & 3);
    const int c = block / 2, lane = block % 2 * 32 + m;
    ((uint4*)p.packed)[(tile * kc + c) * 64 + lane] = w;
    uint8_t* scales = (uint8_t*)p.packed + (int64_t)p.k * p.n / 2 + ((tile * c4 + c / 4) * 64 + lane) * 4;
    scales[c % 4] = (uint8_t)byte;
    if (kc < 4) scales[c + kc] = 0;               // (bytes that are not used)
}

// Chunk C of a product, its scales byte C % 4 of either word
template <int C> __device__ __forceinline__ void mma_mx(const uint4& a, uint32_t sa, const uint4& b, uint32_t sb, f32x16& acc)
{
    const i32x8 x = { (int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0 }, y = { (int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0 };
    acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, acc, 4, 4, C % 4, (int)sa, C % 4, (int)sb);
}
// f(C) for C = 0 .. N-1, each a constant
template <int N, int C = 0, typename F> __device__ __forceinline__ void each(F&& f)
{
    if constexpr (C < N) {
        f(std::integral_constant<int, C>{});
        each<N, C + 1>(f);
    }
}

// What stands in LDS goes in and out in pieces of 16 bytes, so every row of it is whole pieces at a whole piece's address.
// Rows in 4 bits, as B operand: 16 bytes of codes per block, a word of scale bytes for every four chunks and parity of the block
template <int D> struct alignas(16) MxRows {
    static constexpr int STRIDE = D / 2 + 16;     // bytes
    static constexpr int WORDS = (D / 32 + 7) / 8 * 2;         // scale words of a row
    uint8_t codes[ROWS][STRIDE];
    uint32_t scales[WORDS][ROWS];
    __device__ __forceinline__ uint8_t* scale_at(int row, int block)
    {
        return (uint8_t*)&scales[block / 8 * 2 + block % 2][row] + block / 2 % 4;
    }
    __device__ __forceinline__ uint4 operand(int n, int hi, int c) const { return *(const uint4*)(codes[n] + (2 * c + hi) * 16); }
    __device__ __forceinline__ uint32_t scale(int n, int hi, int c) const { return scales[c / 4 * 2 + hi][n]; }
};

// Rows as they are
template <typename T, int D> struct alignas(16) FullRows { T x[ROWS][D + 16 / (int)sizeof(T)]; };

// Rows of the store, K | V codes and scale bytes
template <int D> struct alignas(16) StoreRows {
    uint8_t codes[ROWS][D + 16];
    uint8_t scales[ROWS][2 * D / 32];             // (in pieces of 8)
};

// Rows of a tile as a buffer: what lies behind the call's last row reads as zeros and is not written, without a branch (behind
// which a wait for loads would be one for every store before it, too). No rows at all (r0 past the end, or not yet there): nothing.
typedef int i32x4 __attribute__((ext_vector_type(4)));
constexpr int PAST_CACHES = 2;                    // a buffer store's cache policy: non-temporal
__device__ i32x4 dg4_raw_buffer_load16(i32x4 rsrc, int voffset, int soffset, int aux) __asm("llvm.amdgcn.raw.buffer.load.v4i32");
__device__ void dg4_raw_buffer_store16(i32x4 v, i32x4 rsrc, int voffset, int soffset, int aux) __asm("llvm.amdgcn.raw.buffer.store.v4i32");
template <typename T, int D> __device__ __forceinline__ i32x4 tile_buffer(const void* rows, int64_t r0, int64_t r_end)
{
    const uint64_t a = (uint64_t)rows + (uint64_t)r0 * (D * sizeof(T));
    const int n = (int)max((int64_t)0, min((int64_t)ROWS, r_end - r0));
    return i32x4{ (int)(uint32_t)a, (int)((uint32_t)(a >> 32) & 0xFFFFu), n * (D * (int)sizeof(T)), 0x00020000 };
}

// A tile's rows of S, in pieces of half a block to each of THREADS threads
template <typename T, int D, int THREADS> struct TileRows {
    static constexpr int PPR = D / 16, PIECES = ROWS * PPR / THREADS;
    static_assert(PIECES * THREADS == ROWS * PPR, "whole pieces");
    Values<T, 16> x[PIECES];
    __device__ __forceinline__ void load(const void* s, int64_t r0, int64_t r_end)
    {
        const i32x4 tile = tile_buffer<T, D>(s, r0, r_end);
#pragma unroll
        for (int k = 0; k < PIECES; ++k)
#pragma unroll
            for (int i = 0; i < Values<T, 16>::PIECES; ++i)
                x[k].w[i] = __builtin_bit_cast(uint4, dg4_raw_buffer_load16(tile, ((int)threadIdx.x + k * THREADS) * (16 * (int)sizeof(T)) + 16 * i, 0, 0));
    }
    __device__ __forceinline__ void put(MxRows<D>& to) const
    {
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            const int piece = (int)threadIdx.x + k * THREADS, row = piece / PPR, sub = piece % PPR;
            const uint32_t top = max_of_lanes<2>(x[k].top()), scale = fp4_scale_bits(top);
            const uint32_t byte = top >= 0x7F800000u ? FP4_BAD : scale >> 23;
            uint32_t c[2];
            x[k].codes(scale, c);                 // (any, where the byte says that they are none)
            *(uint2*)(to.codes[row] + sub * 8) = make_uint2(c[0], c[1]);
            *to.scale_at(row, sub / 2) = (uint8_t)byte;        // (the block's other lane the same)
        }
    }
    __device__ __forceinline__ void keep(FullRows<T, D>& to) const
    {
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            const int piece = (int)threadIdx.x + k * THREADS;
            x[k].store(to.x[piece / PPR] + piece % PPR * 16);
        }
    }
};

// A lane's value and that of lane ^ 32
struct Pair { float a, b; };
__device__ __forceinline__ Pair both_halves(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return { __uint_as_float(r[0]), __uint_as_float(r[1]) };
}
// The largest magnitude, as bits, of a block of which a lane has sixteen values and lane ^ 32 the others. LOWER: what is below zero counts
// as zero. (The maximum keeps a NaN, whose bits are above infinity's whatever its sign.)
template <bool LOWER> __device__ __forceinline__ uint32_t block_top(const f32x16& x)
{
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = __builtin_elementwise_maximum(top, LOWER ? x[i] : fabsf(x[i]));
    const Pair p = both_halves(top);
    return __float_as_uint(__builtin_elementwise_maximum(p.a, p.b));
}
__device__ __forceinline__ uint2 half_codes(const f32x16& x, uint32_t scale_bits)
{
    float v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = x[i];
    return make_uint2(fp4_put8(v, scale_bits), fp4_put8(v + 8, scale_bits));
}
// Codes below zero to (minus) zero
__device__ __forceinline__ uint32_t no_less_than_zero(uint32_t w)
{
    const uint32_t t = w & 0x88888888u;
    return w & ~(t - (t >> 3));
}

// Sixteen neighbouring values of a row
template <typename T> __device__ __forceinline__ void put16(T* to, const f32x16& v)
{
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = v[i];
    if constexpr (sizeof(T) == 2) {
        uint4 a, b;
        Elem<bf16_t>::pack(x, a, b);
        ((uint4*)to)[0] = a;
        ((uint4*)to)[1] = b;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            ((uint4*)to)[i] = make_uint4(__float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]), __float_as_uint(x[4 * i + 2]), __float_as_uint(x[4 * i + 3]));
    }
}
template <typename T> __device__ __forceinline__ void get16(const T* from, float* x)
{
    const uint4* p = (const uint4*)from;
    if constexpr (sizeof(T) == 2) {
        Elem<bf16_t>::unpack(p[0], p[1], x);
    } else {
        Elem<float>::unpack(p[0], p[1], x);
        Elem<float>::unpack(p[2], p[3], x + 8);
    }
}

// A workgroup has a wave for every head, whose columns of Wq, Wk and Wv stay in its registers, and takes tiles of rows in turn: the
// rows of the next tile travel while this one is multiplied. Results leave by way of LDS, so that a store is whole rows.
// Bound by HBM: a million rows of bfloat16 at hidden 256 to Q, K and V 377 us (2.06 GB, 5.5 TB/s), to Q and into the store 236 (1.30 GB);
// 400,000 of fp32 at 256 313 and 500,000 of bfloat16 at 128 91, where lanes that store their own pieces take 395 and 108 (372 and 294 for the
// first two). Workgroups: 256 at hidden 256 (512: 406 and 250), 512 at 128 (256: 95).
template <typename T, int D, bool STORE>
__global__ __launch_bounds__(2 * D) void mx4_proj_kernel(dg4_mx4_proj_args p)
{
    constexpr int HEADS = D / 32, KC = D / 64, OUTS = STORE ? 1 : 3;
    __shared__ MxRows<D> rows[2];
    __shared__ FullRows<T, D> outs[OUTS];
    struct Nothing {};
    __shared__ std::conditional_t<STORE, StoreRows<D>, Nothing> kv;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, hi = lane >> 5;
    const int64_t step = (int64_t)gridDim.x * ROWS;
    TileRows<T, D, 2 * D> x;
    int64_t r0 = p.row_begin + (int64_t)blockIdx.x * ROWS;
    x.load(p.s, r0, p.row_end);                   // (ahead of the weights: loads return in order)
    uint4 w[3][KC];
    uint32_t sw[3];
#pragma unroll
    for (int j = 0; j < 3; ++j) {
        const int tile = j * HEADS + wave;
#pragma unroll
        for (int c = 0; c < KC; ++c) w[j][c] = ((const uint4*)p.w_packed)[(tile * KC + c) * 64 + lane];
        sw[j] = ((const uint32_t*)((const uint4*)p.w_packed + 3 * D / 32 * KC * 64))[tile * 64 + lane];
    }
    for (int t = 0; r0 < p.row_end; r0 += step, t ^= 1) {
        x.put(rows[t]);
        __syncthreads();
        x.load(p.s, r0 + step, p.row_end);
        const uint32_t sb = rows[t].scale(n, hi, 0);
        uint4 b[KC];
#pragma unroll
        for (int c = 0; c < KC; ++c) b[c] = rows[t].operand(n, hi, c);
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            f32x16 acc;
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[i] = 0.f;
            each<KC>([&](auto c) __attribute__((always_inline)) { mma_mx<c>(w[j][c], sw[j], b[c], sb, acc); });
            if constexpr (STORE) {
                if (j > 0) {
                    const uint32_t byte = fp4_scale_byte(block_top<false>(acc));
                    *(uint2*)(kv.codes[n] + (j - 1) * (D / 2) + wave * 16 + hi * 8) = byte == FP4_BAD ? make_uint2(0, 0) : half_codes(acc, byte << 23);
                    kv.scales[n][wave * 2 + j - 1] = (uint8_t)byte;               // (lane ^ 32 the same)
                    continue;
                }
            }
            put16<T>(outs[STORE ? 0 : j].x[n] + wave * 32 + hi * 16, acc);
        }
        __syncthreads();
        constexpr int PPR = D * (int)sizeof(T) / 16, PIECES = ROWS * PPR / (2 * D);
#pragma unroll
        for (int j = 0; j < OUTS; ++j) {
            const i32x4 tile = tile_buffer<T, D>(p.out[j], r0, p.row_end);
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const int piece = (int)threadIdx.x + 2 * D * i;
                dg4_raw_buffer_store16(__builtin_bit_cast(i32x4, *((const uint4*)outs[j].x[piece / PPR] + piece % PPR)), tile, piece * 16, 0, PAST_CACHES);
            }
        }
        if constexpr (STORE) {
            const int row = (int)threadIdx.x / (D / 16), piece = (int)threadIdx.x % (D / 16);
            const int64_t r = r0 + row;
            int64_t at = -1;
            if (r < p.row_end) at = p.ids ? (int64_t)p.ids[r] : r;
            if (at >= 0 && at < p.n_store) {
                *(uint4*)(p.codes + at * D + piece * 16) = *(const uint4*)(kv.codes[row] + piece * 16);
                if (piece < HEADS / 4) *(uint2*)(p.scales + at * (2 * HEADS) + piece * 8) = *(const uint2*)(kv.scales[row] + piece * 8);
            }
        }
    }
}

// A workgroup of eight waves takes tiles of rows in turn; both matrices stay in its registers. Four waves, one to a SIMD, put rows into LDS and
// form the activations, a quarter of W1's columns each; the other four multiply the activations, which go through LDS in 4 bits, by a quarter of
// W2's columns each, and normalise. Between two barriers the former are a tile ahead of the latter: vector instructions of the one
// (rounding to 4 bits, LayerNorm) run beside products of the other.
// A million rows of bfloat16 at hidden 256: 325 to 330 us here, 354 on another card, 3.2 and 3.0 PFLOP/s, where the bytes take 199 at the rate of a
// copy and the products 149 at that of a loop of them; at 128 124 (bytes: 99). A turn of a tile is 4900 cycles (256; counted, with the start shared
// out) at 1.85 GHz in calls one after the other. Vector instructions and the issue of products take 3310 of them, 64 products keep the
// matrix core for 2040; for some 1600 a SIMD issues nothing: it has one wave of each role, of 254 and 355 vector instructions to a
// tile, which meet at a barrier for every tile, and a fifth of the waves' cycles is waiting.
// Eight waves that all do everything, an eighth of either matrix each, in step: 365 us (their products and vector instructions come at the same
// time), with rows and residual from memory instead of LDS, so that waits for loads were waits for stores: 412, with three barriers to a
// tile: 520. Half the waves in the opposite order need more registers than there are. The residual of bfloat16 added by products with a unit
// matrix and sums of squares for the variance: 324 for 332 on one card, but rows far off zero lose the variance's digits.
constexpr int FFN_THREADS = 512;
template <typename T, int D>
__global__ __launch_bounds__(FFN_THREADS) void mx4_ffn_kernel(dg4_mx4_ffn_args p)
{
    constexpr int KC = D / 64, KC2 = 4 * D / 64;
    constexpr int TILES1 = D / 32, WORDS = TILES1 / 4, TILES2 = D / 128;       // of a wave: tiles of columns, and scale words of a row that the former make up
    __shared__ MxRows<D> rows[2];
    __shared__ MxRows<4 * D> hidden[2];
    __shared__ FullRows<T, D> full[3];
    __shared__ float2 part[2][4][ROWS];
    constexpr int OUT_ROWS = sizeof(T) == 2 ? ROWS : 8;       // (what LDS has room for)
    __shared__ __align__(16) T outs[4][OUT_ROWS][32 * TILES2 + 16 / (int)sizeof(T)];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, hi = lane >> 5;
    const int64_t step = (int64_t)gridDim.x * ROWS;
    int64_t r0 = p.row_begin + (int64_t)blockIdx.x * ROWS;
    if (wave < 4) {
        TileRows<T, D, FFN_THREADS / 2> x;
        x.load(p.s, r0, p.row_end);               // (ahead of the weights: loads return in order)
        uint4 w1[TILES1][KC];
        uint32_t sw1[TILES1];
        const uint4* u1 = (const uint4*)p.w1_packed;
        const uint32_t* s1 = (const uint32_t*)(u1 + 4 * D / 32 * KC * 64);
        // Scale word w of a row holds the blocks 8 (w / 2) + w % 2 + 0, 2, 4, 6
        auto block_of = [&](int i) __attribute__((always_inline)) { const int w = wave * WORDS + i / 4; return w / 2 * 8 + w % 2 + i % 4 * 2; };
#pragma unroll
        for (int i = 0; i < TILES1; ++i) {
#pragma unroll
            for (int c = 0; c < KC; ++c) w1[i][c] = u1[(block_of(i) * KC + c) * 64 + lane];
            sw1[i] = s1[block_of(i) * 64 + lane];
        }
        auto first = [&](const MxRows<D>& from, MxRows<4 * D>& to) __attribute__((always_inline)) {
            const uint32_t sb = from.scale(n, hi, 0);
            uint4 b[KC];
#pragma unroll
            for (int c = 0; c < KC; ++c) b[c] = from.operand(n, hi, c);
#pragma unroll
            for (int w = 0; w < WORDS; ++w) {
                uint32_t bytes = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int i = 4 * w + j;
                    f32x16 acc;
#pragma unroll
                    for (int k = 0; k < 16; ++k) acc[k] = 0.f;
                    each<KC>([&](auto c) __attribute__((always_inline)) { mma_mx<c>(w1[i][c], sw1[i], b[c], sb, acc); });
                    const uint32_t top = block_top<true>(acc), scale = fp4_scale_bits(top);
                    const uint2 codes = half_codes(acc, scale);
                    *(uint2*)(to.codes[n] + block_of(i) * 16 + hi * 8) = make_uint2(no_less_than_zero(codes.x), no_less_than_zero(codes.y));
                    bytes |= (top >= 0x7F800000u ? FP4_BAD : scale >> 23) << (8 * j);
                }
                to.scales[wave * WORDS + w][n] = bytes;        // (lane ^ 32 the same)
            }
        };
        x.put(rows[0]);
        x.keep(full[0]);
        x.load(p.s, r0 + step, p.row_end);
        __syncthreads();
        first(rows[0], hidden[0]);
        if (r0 + step < p.row_end) {
            x.put(rows[1]);
            x.keep(full[1]);
        }
        x.load(p.s, r0 + 2 * step, p.row_end);
        int t = 0, t3 = 0;
        for (; r0 < p.row_end; r0 += step, t ^= 1, t3 = t3 == 2 ? 0 : t3 + 1) {
            __syncthreads();
            if (r0 + step < p.row_end) {
                first(rows[t ^ 1], hidden[t ^ 1]);
                x.put(rows[t]);
                x.keep(full[t3 == 0 ? 2 : t3 - 1]);
                x.load(p.s, r0 + 3 * step, p.row_end);
            }
        }
        __syncthreads();
    } else {
        const int quarter = wave - 4;
        __syncthreads();                          // (W1, which is needed first, is on its way)
        uint4 w2[TILES2][KC2];
        uint32_t sw2[TILES2][KC2 / 4];
        const uint4* u2 = (const uint4*)p.w2_packed;
        const uint32_t* s2 = (const uint32_t*)(u2 + D / 32 * KC2 * 64);
#pragma unroll
        for (int i = 0; i < TILES2; ++i) {
            const int tile = quarter * TILES2 + i;
#pragma unroll
            for (int c = 0; c < KC2; ++c) w2[i][c] = u2[(tile * KC2 + c) * 64 + lane];
#pragma unroll
            for (int c = 0; c < KC2 / 4; ++c) sw2[i][c] = s2[(tile * (KC2 / 4) + c) * 64 + lane];
        }
        const int col = quarter * (32 * TILES2) + hi * 16;     // of the first tile's sixteen; the next tile's are 32 further
        // The activations' first chunks, requested before there is time to wait for them, and their scales
        constexpr int RING = 4;
        uint4 ring[RING];
        uint32_t sb[KC2 / 4];
        auto request = [&](const MxRows<4 * D>& from) __attribute__((always_inline)) {
#pragma unroll
            for (int c = 0; c < KC2 / 4; ++c) sb[c] = from.scale(n, hi, 4 * c);
#pragma unroll
            for (int c = 0; c < RING; ++c) ring[c] = from.operand(n, hi, c);
        };
        // The row's mean and variance: of the lane's and lane ^ 32's columns; of the row (Chan's update: no difference of large sums).
        // v: the sums less the wave's mean
        f32x16 v[TILES2];
        float mean = 0.f;
        auto second = [&](const MxRows<4 * D>& from, const FullRows<T, D>& rest, float2 (&to)[4][ROWS]) __attribute__((always_inline)) {
            f32x16 acc[TILES2];
#pragma unroll
            for (int i = 0; i < TILES2; ++i)
#pragma unroll
                for (int k = 0; k < 16; ++k) acc[i][k] = 0.f;
            each<KC2>([&](auto c) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < TILES2; ++i) mma_mx<c>(w2[i][c], sw2[i][c / 4], ring[c % RING], sb[c / 4], acc[i]);
                if constexpr (c + RING < KC2) ring[c % RING] = from.operand(n, hi, c + RING);
                __builtin_amdgcn_sched_barrier(0);
            });
            mean = 0.f;
#pragma unroll
            for (int i = 0; i < TILES2; ++i) {
                float s[16];
                get16<T>(rest.x[n] + col + 32 * i, s);
#pragma unroll
                for (int k = 0; k < 16; ++k) { v[i][k] = s[k] + acc[i][k]; mean += v[i][k]; }
            }
            const Pair sums = both_halves(mean);
            mean = (sums.a + sums.b) * (1.f / (32 * TILES2));
            float m2 = 0.f;
#pragma unroll
            for (int i = 0; i < TILES2; ++i)
#pragma unroll
                for (int k = 0; k < 16; ++k) { v[i][k] -= mean; m2 = fmaf(v[i][k], v[i][k], m2); }
            const Pair squares = both_halves(m2);
            to[quarter][n] = make_float2(mean, squares.a + squares.b);         // (lane ^ 32 the same)
        };
        auto finish = [&](int64_t r0, const float2 (&q)[4]) __attribute__((always_inline)) {
            const float all = (q[0].x + q[1].x + q[2].x + q[3].x) * 0.25f;
            float var = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float d = q[i].x - all;
                var += fmaf((float)(D / 4) * d, d, q[i].y);
            }
            const float rstd = rsqrtf(fmaf(var, 1.f / D, p.ln_eps));
            const float rest = (mean - all) * rstd;
            const i32x4 tile = tile_buffer<T, D>(p.out, r0, p.row_end);
#pragma unroll
            for (int i = 0; i < TILES2; ++i)
#pragma unroll
                for (int k = 0; k < 16; ++k) v[i][k] = fmaf(v[i][k], rstd, rest);
            // OUT_ROWS rows at a time through the wave's own LDS (a wave's LDS operations complete in order), so that lanes side by side store
            // pieces side by side
            constexpr int PPR = 2 * TILES2 * (int)sizeof(T), PIECES = OUT_ROWS * PPR / 64;             // pieces of 16 bytes: of the wave's part of a row, of a lane
#pragma unroll
            for (int r = 0; r < ROWS; r += OUT_ROWS) {
                if (OUT_ROWS == ROWS || n / OUT_ROWS * OUT_ROWS == r) {
#pragma unroll
                    for (int i = 0; i < TILES2; ++i) put16<T>(outs[quarter][n % OUT_ROWS] + 32 * i + hi * 16, v[i]);
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
                for (int i = 0; i < PIECES; ++i) {
                    const int piece = lane + 64 * i, row = piece / PPR;
                    const uint4 x = *((const uint4*)outs[quarter][row] + piece % PPR);
                    dg4_raw_buffer_store16(__builtin_bit_cast(i32x4, x), tile, (r + row) * (D * (int)sizeof(T)) + (quarter * PPR + piece % PPR) * 16, 0, PAST_CACHES);
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            }
        };
        auto parts = [&](const float2 (&from)[4][ROWS], float2 (&q)[4]) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = from[i][n];
        };
        float2 q[4];
        int t = 0, t3 = 0;
        for (; r0 < p.row_end; r0 += step, t ^= 1, t3 = t3 == 2 ? 0 : t3 + 1) {
            __syncthreads();
            parts(part[t ^ 1], q);
            request(hidden[t]);
            __builtin_amdgcn_sched_barrier(0);
            if (r0 - step >= p.row_begin) finish(r0 - step, q);
            second(hidden[t], full[t3], part[t]);
        }
        __syncthreads();
        parts(part[t ^ 1], q);
        finish(r0 - step, q);
    }
}

// Workgroups that walk over the tiles of a call
inline dim3 walks(int64_t rows, int most) { return dim3((unsigned)std::min<int64_t>((rows + ROWS - 1) / ROWS, most)); }

template <typename F> int by_shape(int dtype, int hidden, F&& f)
{
    auto with_type = [&](auto t) { return hidden == 128 ? f(t, std::integral_constant<int, 128>{}) : f(t, std::integral_constant<int, 256>{}); };
    return dtype == DG4_F32 ? with_type(float{}) : with_type(bf16_t{});
}

}  // namespace

int64_t dg4_mx4_bytes(int k, int n)
{
    return ((int64_t)k * n / 2 + (int64_t)(n / 32) * scale_words(k) * 64 * 4 + 255) / 256 * 256;
}
int dg4_launch_mx4_pack(int dtype, const dg4_mx4_pack_args& a, hipStream_t s)
{
    const dim3 grid((unsigned)((a.k / 32 * a.n + 255) / 256));
    return launch(dtype == DG4_F32 ? mx4_pack_kernel<float> : mx4_pack_kernel<bf16_t>, grid, 256, s, a);
}
int dg4_launch_mx4_proj(int dtype, int hidden, const dg4_mx4_proj_args& a, hipStream_t s)
{
    return by_shape(dtype, hidden, [&](auto t, auto d) {
        using T = decltype(t);
        constexpr int D = d.value;
        const dim3 grid = walks(a.row_end - a.row_begin, D == 256 ? 256 : 512);
        return launch(a.codes ? mx4_proj_kernel<T, D, true> : mx4_proj_kernel<T, D, false>, grid, 2 * D, s, a);
    });
}
int dg4_launch_mx4_ffn(int dtype, int hidden, const dg4_mx4_ffn_args& a, hipStream_t s)
{
    return by_shape(dtype, hidden, [&](auto t, auto d) {
        using T = decltype(t);
        constexpr int D = d.value;
        return launch(mx4_ffn_kernel<T, D>, walks(a.row_end - a.row_begin, D == 256 ? 256 : 512), FFN_THREADS, s, a);
    });
}
