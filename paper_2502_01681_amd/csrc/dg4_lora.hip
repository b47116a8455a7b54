// The Q|K|V projection with low-rank adapters: [Q|K|V][r] = S[r] W + gain_a (S[r] D_a) U_a with a = adapter[r], for rows of
// many circuits at once, each with its own adapter or none.
//
//  lora_pack_kernel  lays W, D_a and U_a out once in matrix-core operand order.
//  lora_proj_kernel  one launch: a tile of rows goes to LDS, T = gain (S D_a) for every row by its own adapter, then the
//                    output columns, first T U_a, then S W on top in the same accumulators.
//
// A row's arithmetic is the same whatever else its tile holds and however many rows a call covers: the products of a row on
// the matrix cores do not see the other rows, T is always summed as two halves of the features, and where rows of a tile
// differ in their adapter each adapter's product is formed apart and kept for its own rows only (so nothing of another
// circuit's adapter, not even a NaN, reaches a row).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "dg4_device.h"
#include "dg4_internal.h"
#include "dg4_rowops.h"

namespace {

// Weights are the A operand of the 32x32 products and the rows the B operand, so that a lane's 16 accumulators belong to one
// row; with column 16 hi + 4 a + b at operand row 8 a + 4 hi + b they are 16 neighbouring columns.
__device__ __forceinline__ int column_of(int m) { return 16 * ((m >> 2) & 1) + 4 * (m >> 3) + (m & 3); }

constexpr int GROUP = 3;                          // column tiles of 32 that a wave takes at a time
template <typename T> constexpr int PIECE = 16 / (int)sizeof(T);      // elements of 16 bytes
inline int rank8(int rank) { return (rank + 7) / 8 * 8; }

// W: unit ((group * KC + c) * GROUP + j) * 64 + lane holds rows k = (2c + lane/32) E .. + E-1 of column 32 (GROUP group + j) +
// column_of(lane % 32). Down: per adapter, unit (k/E) * rank + n holds rows k .. k+E-1 of column n. Up: per adapter, unit
// (q/E) * 3D + column holds rows q .. q+E-1, zero from `rank` on (up to the next multiple of eight).
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
            const int64_t t = u >> 6;
            const int j = (int)(t % GROUP), c = (int)(t / GROUP % KC), group = (int)(t / GROUP / KC);
            const int col = (group * GROUP + j) * 32 + column_of(lane & 31), k0 = (2 * c + (lane >> 5)) * E;
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

// LDS of a workgroup, in bytes: the rows; T of every row; what is needed before T is finished (its two halves) and after it
// (rows on their way out), one place.
template <typename T, int D, int RT, int JT> struct Lds {
    static constexpr int ROWS = RT * 32;
    static constexpr int S_STRIDE = D + PIECE<T>;                                  // elements
    static constexpr int O_STRIDE = JT * 32 + PIECE<T>;
    static constexpr int S_BYTES = ROWS * S_STRIDE * (int)sizeof(T);
    // T: bfloat16 keeps it as a sum of two (high and low part), so that the product with U_a loses nothing that the
    // output's own rounding would not
    __host__ __device__ static constexpr int t_stride(int r8) { return sizeof(T) == 2 ? 2 * r8 + 8 : r8 + 4; }
    __host__ __device__ static constexpr int t_bytes(int r8) { return ROWS * t_stride(r8) * (int)sizeof(T); }
    __host__ __device__ static constexpr int half_stride(int r8) { return (r8 + 31) / 32 * 32 + 4; }     // floats
    static int bytes(int r8)
    {
        return S_BYTES + t_bytes(r8) + std::max(2 * ROWS * half_stride(r8) * 4, 4 * 32 * O_STRIDE * (int)sizeof(T));
    }
};

// A workgroup of four waves takes RT * 32 rows; a wave takes column tiles in passes of JT. SPREAD: one pass per wave, the
// columns go to 3D/32/4 workgroups along y, and a tile holds p.tile_rows <= 32 rows (the rest of its operand repeats the
// last): calls with few rows, where latency counts. Else the workgroup takes all columns.
template <typename T, int D, int RT, int JT, bool SPREAD>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void lora_proj_kernel(dg4_lora_args p)
{
    using L = Lds<T, D, RT, JT>;
    constexpr int E = PIECE<T>, KC = D / (2 * E), TILES = 3 * D / 32;
    constexpr int PASSES = SPREAD ? 1 : TILES / 4 / JT;
    static_assert(SPREAD ? JT == 1 && RT == 1 : JT == GROUP && TILES % (4 * JT) == 0, "column tiles");
    constexpr int RING = 4;                       // chunks of weights requested ahead
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, hi = lane >> 5;
    const int tile_rows = SPREAD ? p.tile_rows : L::ROWS;
    const int64_t r0 = p.row_begin + (int64_t)blockIdx.x * tile_rows;
    const int64_t r_end = min(p.row_end, r0 + tile_rows);
    auto row_at = [&](int i) { const int64_t r = r0 + i; return r < r_end ? r : r_end - 1; };

    T* const rows = (T*)smem;
    T* const low = (T*)(smem + L::S_BYTES);
    float* const half_sum = (float*)(smem + L::S_BYTES + L::t_bytes(p.rank8));
    T* const out_rows = (T*)half_sum + wave * 32 * L::O_STRIDE;

    // this wave's weights: a linear stream over its passes
    const int tile0 = SPREAD ? (int)blockIdx.y * 4 + wave : wave * PASSES * JT;
    const uint4* wp = (const uint4*)p.w_packed + ((int64_t)(tile0 / GROUP) * KC * GROUP + tile0 % GROUP) * 64 + lane;
    auto weight = [&](int f) { return wp[(int64_t)(SPREAD ? f * GROUP : f) * 64]; };      // f = chunk * JT + j, on through the passes
    {
        constexpr int CPR = D / E;
        uint4 v[L::ROWS * CPR / 256];
#pragma unroll
        for (int i = 0; i < L::ROWS * CPR / 256; ++i) {
            const int piece = (int)threadIdx.x + 256 * i;
            v[i] = *((const uint4*)((const T*)p.s + row_at(piece / CPR) * D) + piece % CPR);
        }
#pragma unroll
        for (int i = 0; i < L::ROWS * CPR / 256; ++i) {
            const int piece = (int)threadIdx.x + 256 * i;
            *((uint4*)(rows + (piece / CPR) * L::S_STRIDE) + piece % CPR) = v[i];
        }
    }
    // adapter of this lane's row of each row tile (-1: none)
    int ad[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        ad[t] = p.adapter ? p.adapter[row_at(t * 32 + n)] : -1;
        if (ad[t] < 0 || ad[t] >= p.n_adapters) ad[t] = -1;
    }
    uint64_t any = 0;
    bool one = true;                              // one adapter for the whole tile
    const int first_ad = __builtin_amdgcn_readfirstlane(ad[0]);
#pragma unroll
    for (int t = 0; t < RT; ++t) { any |= __ballot(ad[t] >= 0); one = one && __ballot(ad[t] != first_ad) == 0; }
    __syncthreads();

    if (any) {
        // T, by (row tile, half of the features): waves 0 .. 2 RT - 1
        if (wave < 2 * RT) {
            const int t = wave >> 1, half = wave & 1;
            int mine = ad[0];
#pragma unroll
            for (int q = 1; q < RT; ++q) mine = t == q ? ad[q] : mine;
            uint64_t todo = __ballot(mine >= 0);
            while (todo) {
                const int a = __builtin_amdgcn_readlane(mine, (int)__builtin_ctzll(todo));
                todo &= ~__ballot(mine == a);
                const uint4* dp = (const uint4*)p.down_packed + (int64_t)a * (D / E) * p.rank;
                for (int nt = 0; nt * 32 < p.rank; ++nt) {
                    const int col = nt * 32 + column_of(n);
                    uint4 d[KC / 2];
#pragma unroll
                    for (int c = 0; c < KC / 2; ++c)
                        d[c] = col < p.rank ? dp[(int64_t)(2 * (half * (KC / 2) + c) + hi) * p.rank + col] : make_uint4(0, 0, 0, 0);
                    f32x16 acc;
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
#pragma unroll
                    for (int c = 0; c < KC / 2; ++c)
                        Mma<T>::run(d[c], *(const uint4*)(rows + (t * 32 + n) * L::S_STRIDE + (2 * (half * (KC / 2) + c) + hi) * E), acc);
                    if (mine == a) {
                        float4* dst = (float4*)(half_sum + (half * L::ROWS + t * 32 + n) * L::half_stride(p.rank8) + nt * 32 + 16 * hi);
#pragma unroll
                        for (int i = 0; i < 4; ++i) dst[i] = make_float4(acc[4 * i], acc[4 * i + 1], acc[4 * i + 2], acc[4 * i + 3]);
                    }
                }
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < L::ROWS * (p.rank8 / 4); i += 256) {
            const int row = i % L::ROWS, q0 = i / L::ROWS * 4;
            const float* h0 = half_sum + row * L::half_stride(p.rank8) + q0;
            const float* h1 = h0 + L::ROWS * L::half_stride(p.rank8);
            const int a = p.adapter[row_at(row)];
            const bool has = a >= 0 && a < p.n_adapters;
            const float gain = has ? p.gain_packed[a] : 0.f;
            float v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = has && q0 + k < p.rank ? (h0[k] + h1[k]) * gain : 0.f;
            T* dst = low + row * L::t_stride(p.rank8) + q0;
            if constexpr (sizeof(T) == 2) {
                uint32_t h[4];
                float rest[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    h[k] = f32_to_bf16_bits(v[k]);
                    const float back = __uint_as_float(h[k] << 16);
                    rest[k] = fabsf(back) < INFINITY ? v[k] - back : 0.f;
                }
                *(uint2*)dst = make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
                *(uint2*)(dst + p.rank8) = make_uint2(pack_bf16x2(rest[0], rest[1]), pack_bf16x2(rest[2], rest[3]));
            } else {
                *(float4*)dst = make_float4(v[0], v[1], v[2], v[3]);
            }
        }
        __syncthreads();
    }
    // chunk c of T as operand: bfloat16 has the high parts of eight ranks in one half of the wave and their low parts in
    // the other, against the same eight rows of U_a
    constexpr int RANKS = 8;                      // ranks per chunk, either type
    const int chunks = p.rank8 / RANKS;
    auto low_at = [&](int t, int c) {
        const T* row = low + (t * 32 + n) * L::t_stride(p.rank8);
        return *(const uint4*)(sizeof(T) == 2 ? row + hi * p.rank8 + c * 8 : row + (2 * c + hi) * 4);
    };
    auto up_at = [&](int a, int c, int tile) {
        const int64_t unit = sizeof(T) == 2 ? c : 2 * c + hi;
        return ((const uint4*)p.up_packed)[((int64_t)a * (p.rank8 / E) + unit) * (3 * D) + tile * 32 + column_of(n)];
    };

    uint4 ring[RING][JT];
#pragma unroll
    for (int c = 0; c < RING; ++c)
#pragma unroll
        for (int j = 0; j < JT; ++j) ring[c][j] = weight(c * JT + j);
#pragma unroll 1
    for (int pass = 0; pass < PASSES; ++pass) {
        f32x16 acc[RT][JT];
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int j = 0; j < JT; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[t][j][i] = 0.f;
        const int tile = tile0 + pass * JT;
        if (any && one) {
            for (int c = 0; c < chunks; ++c) {
                uint4 u[JT];
#pragma unroll
                for (int j = 0; j < JT; ++j) u[j] = up_at(first_ad, c, tile + j);
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    const uint4 b = low_at(t, c);
#pragma unroll
                    for (int j = 0; j < JT; ++j) Mma<T>::run(u[j], b, acc[t][j]);
                }
            }
        } else if (any) {
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                uint64_t todo = __ballot(ad[t] >= 0);
                while (todo) {
                    const int a = __builtin_amdgcn_readlane(ad[t], (int)__builtin_ctzll(todo));
                    todo &= ~__ballot(ad[t] == a);
#pragma unroll
                    for (int j = 0; j < JT; ++j) {
                        f32x16 part;
#pragma unroll
                        for (int i = 0; i < 16; ++i) part[i] = 0.f;
                        for (int c = 0; c < chunks; ++c) Mma<T>::run(up_at(a, c, tile + j), low_at(t, c), part);
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[t][j][i] = ad[t] == a ? part[i] : acc[t][j][i];
                    }
                }
            }
        }
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            uint4 b[RT];
#pragma unroll
            for (int t = 0; t < RT; ++t) b[t] = *(const uint4*)(rows + (t * 32 + n) * L::S_STRIDE + (2 * c + hi) * E);
#pragma unroll
            for (int j = 0; j < JT; ++j)
#pragma unroll
                for (int t = 0; t < RT; ++t) Mma<T>::run(ring[c % RING][j], b[t], acc[t][j]);
            if (c + RING < KC || pass + 1 < PASSES) {
#pragma unroll
                for (int j = 0; j < JT; ++j) ring[c % RING][j] = weight((pass * KC + c + RING) * JT + j);
            }
        }
        // out through this wave's own corner of LDS (its operations complete in order), as 16-byte pieces of rows
        constexpr int PPR = JT * 32 / E;          // pieces per row
#pragma unroll
        for (int t = 0; t < RT; ++t) {
#pragma unroll
            for (int j = 0; j < JT; ++j) {
                uint4* dst = (uint4*)(out_rows + n * L::O_STRIDE + j * 32 + 16 * hi);
                const f32x16& x = acc[t][j];
                if constexpr (sizeof(T) == 2) {
                    dst[0] = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
                    dst[1] = make_uint4(pack_bf16x2(x[8], x[9]), pack_bf16x2(x[10], x[11]), pack_bf16x2(x[12], x[13]), pack_bf16x2(x[14], x[15]));
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        dst[i] = make_uint4(__float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]), __float_as_uint(x[4 * i + 2]), __float_as_uint(x[4 * i + 3]));
                }
            }
#pragma unroll
            for (int i = 0; i < 32 * PPR / 64; ++i) {
                const int piece = lane + 64 * i, row = piece / PPR, cc = piece % PPR;
                const uint4 v = *((const uint4*)(out_rows + row * L::O_STRIDE) + cc);
                const int col = tile * 32 + cc * E;
                const int64_t r = r0 + t * 32 + row;
                T* dst = (T*)(col < D ? p.out[0] : col < 2 * D ? p.out[1] : p.out[2]);
                if (r < r_end) *(uint4*)(dst + r * D + col % D) = v;
            }
        }
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

// (64 KB need no leave)
template <typename K> int allow_lds(K kernel, int bytes)
{
    return bytes <= 65536 ? hipSuccess : hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

template <typename T, int D>
int launch_proj(dg4_lora_args a, hipStream_t s)
{
    const int64_t rows = a.row_end - a.row_begin;
    if (rows <= 4096) {
        using L = Lds<T, D, 1, 1>;
        const auto kernel = lora_proj_kernel<T, D, 1, 1, true>;
        // rows per tile: few enough for two workgroups per compute unit
        a.tile_rows = 1;
        while (a.tile_rows < 32 && rows * (3 * D / 128) > (int64_t)512 * a.tile_rows) a.tile_rows *= 2;
        const int smem = L::bytes(a.rank8);
        if (const int e = allow_lds(kernel, smem); e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, dim3((unsigned)((rows + a.tile_rows - 1) / a.tile_rows), 3 * D / 128), dim3(256), smem, s, a);
    } else {
        using L = Lds<T, D, 2, GROUP>;
        const auto kernel = lora_proj_kernel<T, D, 2, GROUP, false>;
        const int smem = L::bytes(a.rank8);
        if (const int e = allow_lds(kernel, smem); e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, dim3((unsigned)((rows + L::ROWS - 1) / L::ROWS)), dim3(256), smem, s, a);
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
