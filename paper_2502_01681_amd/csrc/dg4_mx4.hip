// Products of rows and weights in 4 bits, both by blocks of 32 along the summed axis (dg4_fp4.h), on the scaled matrix cores:
//
//  mx4_pack_kernel  a weight matrix once into blocks, in matrix-core operand order.
//  mx4_proj_kernel  [Q | K | V] = q(S) q(Wqkv): to rows, or Q to rows and K and V straight from the accumulators into the store
//                   in 4 bits, whose blocks are the heads of a row.
//  mx4_ffn_kernel   Out = LayerNorm(S + q(max(q(S) q(W1), 0)) q(W2)).
//
// Weights are the A operand of 32x32x64 products and rows the B operand, so that a lane's sixteen accumulators belong to one
// row; operand row 8 a + 4 hi + b is column 16 hi + 4 a + b of a tile, so they are sixteen neighbouring columns, half a block.
// A product of two codes has at most 6 bits and a power of two takes none: sums in fp32 are exact as long as the powers of two of a
// row's and a column's blocks lie within some 2^8 of each other.
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
    if (byte != FP4_BAD) w = make_uint4(fp4_put8(x, byte), fp4_put8(x + 8, byte), fp4_put8(x + 16, byte), fp4_put8(x + 24, byte));
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

// Rows in 4 bits in LDS, as B operand: 16 bytes of codes per block, a word of scale bytes for every eight blocks of one parity
template <int D> struct MxRows {
    static constexpr int STRIDE = D / 2 + 16;     // bytes
    static constexpr int WORDS = (D / 32 + 7) / 8 * 2;         // scale words of a row
    uint8_t codes[ROWS][STRIDE];
    uint32_t scales[ROWS][WORDS];
    __device__ __forceinline__ uint8_t* scale_at(int row, int block)
    {
        return (uint8_t*)&scales[row][block / 8 * 2 + block % 2] + block / 2 % 4;
    }
};

// A tile's rows of S: a thread takes pieces of eight features, PIECES of them, 2 D threads to a workgroup
template <typename T, int D> struct TileRows {
    static constexpr int PPR = D / 8, PIECES = ROWS * PPR / (2 * D);
    Eighth<T> x[PIECES];
    __device__ __forceinline__ void load(const T* s, int64_t r0, int64_t r_end)
    {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int piece = (int)threadIdx.x + 2 * D * i;
            x[i].load(s + min(r0 + piece / PPR, r_end - 1) * D + piece % PPR * 8);
        }
    }
    __device__ __forceinline__ void put(MxRows<D>& to) const
    {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int piece = (int)threadIdx.x + 2 * D * i, row = piece / PPR, sub = piece % PPR;
            const uint32_t byte = fp4_scale_byte(max_of_4_lanes(x[i].top()));
            *(uint32_t*)(to.codes[row] + sub * 4) = byte == FP4_BAD ? 0u : x[i].codes(byte);
            if (sub % 4 == 0) *to.scale_at(row, sub / 4) = (uint8_t)byte;
        }
    }
};

// Half a block, a lane's sixteen accumulators, in 4 bits; the other half is lane ^ 32's. (A NaN, which an ordinary maximum passes
// over, makes the block one that is not finite.)
__device__ __forceinline__ uint2 half_block(const float* x, uint32_t& byte)
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    byte = fp4_scale_byte(top);
    return byte == FP4_BAD ? make_uint2(0, 0) : make_uint2(fp4_put8(x, byte), fp4_put8(x + 8, byte));
}

// Sixteen neighbouring values of a row
template <typename T> __device__ __forceinline__ void put16(T* to, const float* x)
{
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
// rows of the next tile travel while this one is multiplied.
template <typename T, int D, bool STORE>
__global__ __launch_bounds__(2 * D) void mx4_proj_kernel(dg4_mx4_proj_args p)
{
    constexpr int HEADS = D / 32, KC = D / 64;
    __shared__ MxRows<D> rows[2];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, hi = lane >> 5;
    uint4 w[3][KC];
    uint32_t sw[3];
#pragma unroll
    for (int j = 0; j < 3; ++j) {
        const int tile = j * HEADS + wave;
#pragma unroll
        for (int c = 0; c < KC; ++c) w[j][c] = ((const uint4*)p.w_packed)[(tile * KC + c) * 64 + lane];
        sw[j] = ((const uint32_t*)((const uint4*)p.w_packed + 3 * D / 32 * KC * 64))[tile * 64 + lane];
    }
    const int64_t step = (int64_t)gridDim.x * ROWS;
    TileRows<T, D> x;
    int64_t r0 = p.row_begin + (int64_t)blockIdx.x * ROWS;
    x.load((const T*)p.s, r0, p.row_end);
    for (int t = 0; r0 < p.row_end; r0 += step, t ^= 1) {
        x.put(rows[t]);
        __syncthreads();
        if (r0 + step < p.row_end) x.load((const T*)p.s, r0 + step, p.row_end);
        f32x16 acc[3];
#pragma unroll
        for (int j = 0; j < 3; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[j][i] = 0.f;
        const uint32_t sb = rows[t].scales[n][hi];
        each<KC>([&](auto c) __attribute__((always_inline)) {
            const uint4 b = *(const uint4*)(rows[t].codes[n] + (2 * c + hi) * 16);
#pragma unroll
            for (int j = 0; j < 3; ++j) mma_mx<c>(w[j][c], sw[j], b, sb, acc[j]);
        });
        const int64_t r = r0 + n;
        int64_t at = -1;
        if (r < p.row_end) at = STORE && p.ids ? (int64_t)p.ids[r] : r;
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            float v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = acc[j][i];
            if (STORE && j > 0) {
                uint32_t byte;
                const uint2 codes = half_block(v, byte);
                if (at >= 0 && at < p.n_store) {
                    *(uint2*)(p.codes + at * D + (j - 1) * (D / 2) + wave * 16 + hi * 8) = codes;
                    if (hi == 0) p.scales[(at * HEADS + wave) * 2 + j - 1] = (uint8_t)byte;
                }
            } else if (r < p.row_end) {
                put16<T>((T*)p.out[j] + r * D + wave * 32 + hi * 16, v);
            }
        }
    }
}

// A workgroup has a wave for every 32 columns of the output and takes tiles of rows in turn. Each wave holds its share of both
// matrices in registers: four tiles of W1's columns, and its own columns of W2. The activations of a tile go through LDS in 4 bits.
template <typename T, int D>
__global__ __launch_bounds__(2 * D) void mx4_ffn_kernel(dg4_mx4_ffn_args p)
{
    constexpr int WAVES = D / 32, KC = D / 64, KC2 = 4 * D / 64;
    __shared__ MxRows<D> rows;
    __shared__ MxRows<4 * D> hidden;
    __shared__ float2 part[ROWS][WAVES];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, hi = lane >> 5;
    uint4 w1[4][KC], w2[KC2];
    uint32_t sw1[4], sw2[KC2 / 4];
    const uint4* u1 = (const uint4*)p.w1_packed;
    const uint4* u2 = (const uint4*)p.w2_packed;
    const uint32_t* s1 = (const uint32_t*)(u1 + 4 * D / 32 * KC * 64);
    const uint32_t* s2 = (const uint32_t*)(u2 + D / 32 * KC2 * 64);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int c = 0; c < KC; ++c) w1[j][c] = u1[((4 * wave + j) * KC + c) * 64 + lane];
        sw1[j] = s1[(4 * wave + j) * 64 + lane];
    }
#pragma unroll
    for (int c = 0; c < KC2; ++c) w2[c] = u2[(wave * KC2 + c) * 64 + lane];
#pragma unroll
    for (int c = 0; c < KC2 / 4; ++c) sw2[c] = s2[(wave * (KC2 / 4) + c) * 64 + lane];

    const int64_t step = (int64_t)gridDim.x * ROWS;
    TileRows<T, D> x;
    int64_t r0 = p.row_begin + (int64_t)blockIdx.x * ROWS;
    x.load((const T*)p.s, r0, p.row_end);
    for (; r0 < p.row_end; r0 += step) {
        x.put(rows);
        __syncthreads();
        if (r0 + step < p.row_end) x.load((const T*)p.s, r0 + step, p.row_end);
        const uint32_t sb = rows.scales[n][hi];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            f32x16 acc;
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[i] = 0.f;
            each<KC>([&](auto c) __attribute__((always_inline)) {
                mma_mx<c>(w1[j][c], sw1[j], *(const uint4*)(rows.codes[n] + (2 * c + hi) * 16), sb, acc);
            });
            float v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = acc[i] < 0.f ? 0.f : acc[i];       // (a NaN stays one)
            uint32_t byte;
            const int block = 4 * wave + j;
            *(uint2*)(hidden.codes[n] + block * 16 + hi * 8) = half_block(v, byte);
            if (hi == 0) *hidden.scale_at(n, block) = (uint8_t)byte;
        }
        __syncthreads();
        f32x16 acc;
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] = 0.f;
        each<KC2>([&](auto c) __attribute__((always_inline)) {
            mma_mx<c>(w2[c], sw2[c / 4], *(const uint4*)(hidden.codes[n] + (2 * c + hi) * 16), hidden.scales[n][c / 4 * 2 + hi], acc);
        });
        // The row's mean and variance: of a lane's sixteen columns, of the wave's 32, of the row (Chan's update: no difference of large sums)
        const int64_t r = min(r0 + n, p.row_end - 1);
        const int col = wave * 32 + hi * 16;
        float v[16];
        get16<T>((const T*)p.s + r * D + col, v);
        float mean = 0.f, m2 = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) { v[i] += acc[i]; mean += v[i]; }
        mean += __shfl_xor(mean, 32);
        mean *= 1.f / 32;
#pragma unroll
        for (int i = 0; i < 16; ++i) m2 = fmaf(v[i] - mean, v[i] - mean, m2);
        m2 += __shfl_xor(m2, 32);
        if (hi == 0) part[n][wave] = make_float2(mean, m2);
        __syncthreads();
        float all = 0.f, var = 0.f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) all += part[n][i].x;
        all *= 1.f / WAVES;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            const float2 q = part[n][i];
            var += fmaf(32.f * (q.x - all), q.x - all, q.y);
        }
        const float rstd = 1.f / sqrtf(fmaf(var, 1.f / D, p.ln_eps));
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = (v[i] - all) * rstd;
        if (r0 + n < p.row_end) put16<T>((T*)p.out + r * D + col, v);
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
    if (dtype == DG4_F32) hipLaunchKernelGGL(mx4_pack_kernel<float>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(mx4_pack_kernel<bf16_t>, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}
int dg4_launch_mx4_proj(int dtype, int hidden, const dg4_mx4_proj_args& a, hipStream_t s)
{
    return by_shape(dtype, hidden, [&](auto t, auto d) {
        using T = decltype(t);
        constexpr int D = d.value;
        const dim3 grid = walks(a.row_end - a.row_begin, 512);
        if (a.codes) hipLaunchKernelGGL((mx4_proj_kernel<T, D, true>), grid, dim3(2 * D), 0, s, a);
        else hipLaunchKernelGGL((mx4_proj_kernel<T, D, false>), grid, dim3(2 * D), 0, s, a);
        return (int)hipGetLastError();
    });
}
int dg4_launch_mx4_ffn(int dtype, int hidden, const dg4_mx4_ffn_args& a, hipStream_t s)
{
    return by_shape(dtype, hidden, [&](auto t, auto d) {
        using T = decltype(t);
        constexpr int D = d.value;
        hipLaunchKernelGGL((mx4_ffn_kernel<T, D>), walks(a.row_end - a.row_begin, 256), dim3(2 * D), 0, s, a);
        return (int)hipGetLastError();
    });
}
