// The K|V store in 8 bits: rows written into it, read back, and attended over.
//
//  kv8_write_kernel  quantises K and V rows by blocks of one head (32 features): the largest magnitude of the block
//                    picks a power of two, every value divided by it is rounded once. HBM-bound.
//  kv8_read_kernel   the reverse.
//  kv8_attn_kernel   scores, softmax and aggregation over cone rows (Section 3.5) straight from the codes: the power of
//                    two of a head's K comes out of its dot product, that of its V into the entry's weight, so a code
//                    costs its conversion and one multiply-add. HBM- and L2-bound gather of half (a quarter of) the bytes.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "dg4_device.h"
#include "dg4_internal.h"
#include "dg4_rowops.h"

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));

// Bytes of codes up to which buffer addressing is used: offsets are 32 bits, and there is room for one that is past the end
constexpr uint32_t KV8_NEAR_BYTES = 0xC0000000u;

// Which run of rows a workgroup takes. Workgroups go to the eight XCDs in turn, and neighbouring rows read the same sources:
// runs of 128 workgroups (1024 to 4096 rows) go to one XCD, so that its L2 serves them (a million gates of bf16 / 256, two
// hops: lines missed in the L2s 30 M -> 18 M, 491 -> 452 us). What is left behind the last eight whole runs goes in turn.
__device__ __forceinline__ uint32_t kv8_block(uint32_t block, uint32_t blocks)
{
    constexpr uint32_t RUN = 128;
    const uint32_t base = block / (8 * RUN) * (8 * RUN);
    return base + 8 * RUN <= blocks ? base + block % 8 * RUN + (block - base) / 8 : block;
}

// What a block is scaled by, from the bits of its largest magnitude: the biased exponent of the smallest power of two with
// which that magnitude stays within the format's largest code, 448 = 1.75 * 2^8 or 127 = 1.984375 * 2^6. Adding what the
// mantissa may miss to the next power carries into the exponent exactly where it is above the code's. A block with an
// infinity or a NaN gets 255.
template <int FMT> __device__ __forceinline__ uint32_t scale_byte(uint32_t top)
{
    constexpr uint32_t MANT = FMT == DG4_KV_E4M3 ? 0x600000u : 0x7E0000u;
    constexpr int EXP = FMT == DG4_KV_E4M3 ? 8 : 6;
    const int e = (int)((top + (0x7FFFFFu - MANT)) >> 23) - EXP;
    return top >= 0x7F800000u ? 255u : (uint32_t)(e > 0 ? e : 0);
}
// 2^(byte - 127); 255 stands for NaN, 0 for the subnormal 2^-127
__device__ __forceinline__ float scale_value(uint32_t byte)
{
    const uint32_t bits = byte == 0 ? 0x00400000u : byte << 23;
    return __uint_as_float(byte == 255u ? 0x7FC00000u : bits);
}

// Four values, already divided by their block's scale, as codes: to nearest, ties to even.
template <int FMT> __device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d)
{
    if constexpr (FMT == DG4_KV_E4M3) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    } else {
        // 1.5 * 2^23 + v: the sum is rounded to a whole number, whose low byte is v's two's complement
        const float magic = 12582912.f;
        const uint32_t ab = __builtin_amdgcn_perm(__float_as_uint(b + magic), __float_as_uint(a + magic), 0x0C0C0400u);
        const uint32_t cd = __builtin_amdgcn_perm(__float_as_uint(d + magic), __float_as_uint(c + magic), 0x04000C0Cu);
        return ab | cd;
    }
}
// The four codes of a word as numbers
template <int FMT> __device__ __forceinline__ void decode4(uint32_t w, float* f)
{
    if constexpr (FMT == DG4_KV_E4M3) {
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        f[0] = lo.x; f[1] = lo.y; f[2] = hi.x; f[3] = hi.y;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = (float)(int8_t)(w >> (8 * i));
    }
}
// Eight values of a row in one lane, as loaded
template <typename T> struct Eight;
template <> struct Eight<float> {
    uint4 a, b;
    __device__ void load(const float* p) { a = ((const uint4*)p)[0]; b = ((const uint4*)p)[1]; }
    __device__ void get(float* f) const { Elem<float>::unpack(a, b, f); }
};
template <> struct Eight<bf16_t> {
    uint4 a;
    __device__ void load(const bf16_t* p) { a = *(const uint4*)p; }
    __device__ void get(float* f) const
    {
        const uint32_t w[4] = { a.x, a.y, a.z, a.w };
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = bf16_lo(w[i]); f[2 * i + 1] = bf16_hi(w[i]); }
    }
};

// A lane takes eight features, so a head is four lanes and a gate's K | V row a whole wave at hidden 256 (two gates at
// 128): one 512-byte (256-byte) row of codes per store instruction. U gates per lane, all requested before the first is used;
// with two there are enough loads on their way for the whole card and enough workgroups for a level: 1, 2 and 4 gates per lane
// take 259, 256 and 269 us for a million rows of bfloat16 at hidden 256 (1.56 GB moved, 6.1 TB/s) and 3.1, 3.3 and 3.9 us for
// 264. Codes leave through the caches, where the next level's attention finds them (past them: 249 us).
template <typename T, int FMT, int D, int U>
__global__ __launch_bounds__(256) void kv8_write_kernel(dg4_kv8_args p)
{
    constexpr int LPG = 2 * D / 8;                // lanes per gate
    constexpr int GPB = 256 / LPG;                // gates per workgroup and pass
    const int sub = (int)threadIdx.x % LPG;
    const int64_t r0 = p.row_begin + (int64_t)blockIdx.x * (GPB * U) + (int)threadIdx.x / LPG;
    const bool is_v = sub >= LPG / 2;
    const int col = (sub % (LPG / 2)) * 8;
    const T* src = (const T*)(is_v ? p.v : p.k) + col;
    Eight<T> x[U];
    int64_t at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t r = r0 + (int64_t)u * GPB;
        const bool in = r < p.row_end;
        const int64_t row = in ? r : p.row_end - 1;           // loads stay in bounds, stores are masked
        x[u].load(src + row * D);
        at[u] = p.ids ? (int64_t)p.ids[row] : row;
        if (!in || at[u] >= p.n_store) at[u] = -1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float f[8];
        x[u].get(f);
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(f[i]) & 0x7FFFFFFFu);
        top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, true));    // the other lanes
        top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xF, 0xF, true));    // of the head
        const uint32_t byte = scale_byte<FMT>(top);
        const bool bad = byte == 255u;
        const float inv = __uint_as_float(bad ? 0u : (254u - byte) << 23);                            // 2^(127 - byte)
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = f[i] * inv;        // exact, or far below the smallest code
        uint2 w = make_uint2(encode4<FMT>(f[0], f[1], f[2], f[3]), encode4<FMT>(f[4], f[5], f[6], f[7]));
        if (bad) w = make_uint2(0, 0);
        if (at[u] >= 0) {
            *(uint2*)(p.codes + at[u] * (2 * D) + sub * 8) = w;
            if ((sub & 3) == 0) p.scales[at[u] * (2 * D / 32) + (sub % (LPG / 2)) / 4 * 2 + (is_v ? 1 : 0)] = (uint8_t)byte;
        }
    }
}

// A lane takes what it stores as 16 bytes, so that a wave's store is whole lines: four features of fp32, eight of bfloat16
// (402,193 rows of fp32 at hidden 256, 1.04 GB moved: 250 us with two 16-byte stores a lane, of every other piece each, 155 us, 6.7
// TB/s, so; 181 us where rows leave through the caches). U rows per lane: 185, 155 and 175 us with 1, 2 and 4.
template <typename T, int FMT, int D, int U>
__global__ __launch_bounds__(256) void kv8_read_kernel(dg4_kv8_args p)
{
    constexpr int PER = 16 / (int)sizeof(T);
    constexpr int LPG = 2 * D / PER;
    constexpr int GPB = 256 / LPG;
    const int sub = (int)threadIdx.x % LPG;
    const int64_t r0 = p.row_begin + (int64_t)blockIdx.x * (GPB * U) + (int)threadIdx.x / LPG;
    const bool is_v = sub >= LPG / 2;
    const int col = (sub % (LPG / 2)) * PER;
    T* dst = (T*)(is_v ? p.v_out : p.k_out) + col;
    uint32_t w[U][PER / 4];
    uint32_t byte[U];
    bool in[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t r = r0 + (int64_t)u * GPB;
        in[u] = r < p.row_end;
        int64_t at = 0;
        if (in[u]) at = p.ids ? (int64_t)p.ids[r] : r;
        in[u] = in[u] && at >= 0 && at < p.n_store;
        if (!in[u]) at = 0;                                   // (the store has a row: the launcher checks)
        const uint8_t* from = p.codes + at * (2 * D) + sub * PER;
        if constexpr (PER == 8) {
            const uint2 two = *(const uint2*)from;
            w[u][0] = two.x; w[u][1] = two.y;
        } else {
            w[u][0] = *(const uint32_t*)from;
        }
        byte[u] = p.scales[at * (2 * D / 32) + col / 32 * 2 + (is_v ? 1 : 0)];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float f[PER];
#pragma unroll
        for (int i = 0; i < PER / 4; ++i) decode4<FMT>(w[u][i], f + 4 * i);
        const float scale = scale_value(byte[u]);
#pragma unroll
        for (int i = 0; i < PER; ++i) f[i] *= scale;
        uint4 out;
        if constexpr (PER == 8) out = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
        else out = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
        if (in[u]) store_stream(dst + (r0 + (int64_t)u * GPB) * D, out);
    }
}

// ------------------------------------------------------------------------------------------------- attention

// What an entry that is none reads where buffer addressing does not reach (FAR, below)
__device__ __align__(256) const uint8_t nothing[512] = {};

__device__ dg4_i32x4 dg4_raw_buffer_load16(dg4_i32x4 rsrc, int voffset, int soffset, int aux) __asm("llvm.amdgcn.raw.buffer.load.v4i32");
__device__ uint16_t dg4_raw_buffer_load2(dg4_i32x4 rsrc, int voffset, int soffset, int aux) __asm("llvm.amdgcn.raw.buffer.load.i16");

// The four codes of a word. e4m3: times the power of two of `byte`, which the conversion takes along (0: 2^-127, 255: NaN);
// int8: as they are.
template <int FMT> __device__ __forceinline__ void decode4_scaled(uint32_t w, uint32_t byte, float* f)
{
    if constexpr (FMT == DG4_KV_E4M3) {
        const float scale = __uint_as_float(byte << 23);
        const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, true);
        f[0] = lo.x; f[1] = lo.y; f[2] = hi.x; f[3] = hi.y;
    } else {
        decode4<FMT>(w, f);
    }
}

// A lane's sixteen values of q, and their product with as many codes. dot: in fp32 / e4m3 with the codes' power of two; in int8
// without it, for the whole sum to be multiplied by; bfloat16 against e4m3 as pairs of bfloat16 numbers, a code times its power of
// two, two products and a sum in fp32 per instruction. The two short forms have their ends: sums of q times codes overflow from
// |q| = 2^116 on, and such an instruction takes what is below 2^-126, as a code times 2^-117 and less may be, as zero. Up to LARGE_Q
// the one does not happen and the other costs a score at most 32 * 2^-126 * LARGE_Q = 2^-41; rows of Q that go further take
// dot_large, every value of K in fp32 (which holds it exactly).
constexpr uint32_t LARGE_Q = (127u + 80u) << 23;              // 2^80, as a float's bits
template <typename T, int FMT> struct LaneQ {
    static constexpr bool SHORT = FMT != DG4_KV_E4M3;
    float q[16];
    __device__ __forceinline__ void load(const T* p)
    {
        const uint4* v = (const uint4*)p;
        if constexpr (sizeof(T) == 2) {
            Elem<bf16_t>::unpack(v[0], v[1], q);
        } else {
            Elem<float>::unpack(v[0], v[1], q);
            Elem<float>::unpack(v[2], v[3], q + 8);
        }
    }
    __device__ __forceinline__ bool large() const
    {
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(q[i]));            // (a NaN is one either way)
        return top > __uint_as_float(LARGE_Q);
    }
    __device__ __forceinline__ float dot(const uint4& w, uint32_t byte) const
    {
        const uint32_t words[4] = { w.x, w.y, w.z, w.w };
        float d = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float k[4];
            decode4_scaled<FMT>(words[i], byte, k);
#pragma unroll
            for (int x = 0; x < 4; ++x) d = i + x == 0 ? q[0] * k[0] : fmaf(q[4 * i + x], k[x], d);
        }
        return d;
    }
    __device__ __forceinline__ float dot_large(const uint4& w, uint32_t byte) const
    {
        const uint32_t words[4] = { w.x, w.y, w.z, w.w };
        const float scale = scale_value(byte);
        float d = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float k[4];
            decode4<FMT>(words[i], k);
#pragma unroll
            for (int x = 0; x < 4; ++x) d = fmaf(q[4 * i + x], k[x] * scale, d);
        }
        return d;
    }
};
template <> struct LaneQ<bf16_t, DG4_KV_E4M3> {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    static constexpr bool SHORT = true;
    uint4 a, b;
    __device__ __forceinline__ void load(const bf16_t* p) { a = ((const uint4*)p)[0]; b = ((const uint4*)p)[1]; }
    __device__ __forceinline__ bool large() const
    {
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        const uint32_t words[8] = { a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w };
        u16x2 top = { 0, 0 };
#pragma unroll
        for (int i = 0; i < 8; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, words[i] & 0x7FFF7FFFu));
        return max(top.x, top.y) > (LARGE_Q >> 16);
    }
    __device__ __forceinline__ float dot(const uint4& w, uint32_t byte) const
    {
        const float scale = __uint_as_float(byte << 23);
        float d = 0.f;
        auto four = [&](uint32_t codes, uint32_t q0, uint32_t q1) __attribute__((always_inline)) {
            d = __builtin_amdgcn_fdot2_f32_bf16(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false), __builtin_bit_cast(bf16x2, q0), d, false);
            d = __builtin_amdgcn_fdot2_f32_bf16(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true), __builtin_bit_cast(bf16x2, q1), d, false);
        };
        four(w.x, a.x, a.y); four(w.y, a.z, a.w); four(w.z, b.x, b.y); four(w.w, b.z, b.w);
        return d;
    }
    __device__ __forceinline__ float dot_large(const uint4& w, uint32_t byte) const
    {
        const uint32_t codes[4] = { w.x, w.y, w.z, w.w }, words[8] = { a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w };
        float d = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float k[4];
            decode4_scaled<DG4_KV_E4M3>(codes[i], byte, k);
            uint32_t q0 = words[2 * i], q1 = words[2 * i + 1];
            __asm__ volatile("" : "+v"(q0), "+v"(q1));         // (unpacked here and not, for every row, ahead of the loop)
            d = fmaf(bf16_hi(q1), k[3], fmaf(bf16_lo(q1), k[2], fmaf(bf16_hi(q0), k[1], fmaf(bf16_lo(q0), k[0], d))));
        }
        return d;
    }
};

// A lane owns sixteen features (half a head) and a destination row is S groups of D / 16 lanes: a source's K codes are one
// load instruction over whole 128-byte lines, its V codes another. The row's entries go to the groups in turn, CH at a time;
// each group keeps a running maximum, denominator and weighted sum (32 bits), joined at the end by lane exchange. ONCE: the
// groups take the whole row at one go. Entries that are none (padding, a relation whose bias is -inf) ask the buffers for an
// offset past the end: zeros, no request, no branch, and what the store holds there cannot matter. The offsets of buffer
// addressing are 32 bits: FAR, for larger stores, has addresses of 64 bits and reads zeros from memory for them.
// Up to eight entries a row are two groups of four (2,4: one group of eight 504 us for a million two-hop rows of bfloat16 at 256,
// two of four 491 us, before the rows were grouped by XCD), up to sixteen two of eight; longer rows have a whole wave, whose groups
// keep their loads in flight (15,135 rows of eight-hop cones of bfloat16 at 128: 59.8 us, 3 more where each step moves on to its maximum).
// Measured: 446 us for that million rows, 2.34 GB fetched and 0.51 written (6.4 TB/s) where the store, Q, the table and A are 1.6 GB:
// bound by sources that several XCDs fetch. Long rows are bound by vector instructions, 70 for an entry in bfloat16 / e4m3: 16
// conversions, 8 and 16 products, and what finds, scales and weighs it. Counted for those 15,135 rows: 29.9 M instructions, 119,000
// cycles of each SIMD, 49 of the 60 us at 2.4 GHz. fp32 / int8 at 128: 84 us, bfloat16 / int8 at 256: 155, fp32 / e4m3 at 256: 116.
// 20,256 short rows of fp32 at 128, int8: 8.9 us. One row: 2.7 us, three waits of memory after one another.
template <typename T, int FMT, int D, int S, int CH, bool ONCE, bool FAR>
__global__ __launch_bounds__(256, !ONCE && sizeof(T) == 2 && FMT == DG4_KV_E4M3 ? 5 : 1) void kv8_attn_kernel(dg4_kv8_attn_args p)
{
    constexpr int LPR = D / 16, HEADS = D / 32, GPW = 64 / LPR;
    constexpr int RPW = GPW / S;                  // rows per wave
    constexpr uint32_t NONE = KV8_NEAR_BYTES / (2 * D);        // past the end of a store that buffer addressing reaches
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int sub = lane % LPR, group = lane / LPR, part = group % S;
    const int head = sub >> 1;
    // biases of a head by relation code
    __shared__ float bias[HEADS][4];
    if (threadIdx.x < HEADS * 4) bias[threadIdx.x / 4][threadIdx.x % 4] = p.rel_bias[threadIdx.x];
    __syncthreads();
    const int64_t r = p.row_begin + ((int64_t)(ONCE ? kv8_block(blockIdx.x, gridDim.x) : blockIdx.x) * 4 + wave) * RPW + group / S;
    // (what leaves here leaves as whole rows)
    if (r >= p.row_end) return;
    const int64_t v = p.ids ? (int64_t)p.ids[r] : r;
    if (v < 0 || v >= p.n) return;

    const dg4_i32x4 code_bytes = row_buffer(p.codes, 0, FAR ? 0 : (uint32_t)(p.n * 2 * D));
    const dg4_i32x4 scale_bytes = row_buffer(p.scales, 0, FAR ? 0 : (uint32_t)(p.n * 2 * HEADS));
    const uint32_t* erow = p.ell + v * (int64_t)p.ell_w;
    uint4 ent[CH / 4];
    auto entries = [&](int c0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < CH / 4; ++i)
            ent[i] = c0 + 4 * i < p.ell_w ? *(const uint4*)(erow + c0 + 4 * i) : make_uint4(DG4_ELL_PAD, DG4_ELL_PAD, DG4_ELL_PAD, DG4_ELL_PAD);
    };
    entries(part * CH);
    LaneQ<T, FMT> q;
    q.load((const T*)p.q + r * D + sub * 16);
    bool large = false;                           // the same for all lanes of the row, so that a row does not see its neighbours
    if constexpr (LaneQ<T, FMT>::SHORT) {
        constexpr int LANES = LPR * S;
        large = (__ballot(q.large()) >> (lane / LANES * LANES) & (~0ull >> (64 - LANES))) != 0;
    }
    const float c = 0.17677669529663687f;         // 1/sqrt(32)
    const float log2e = 1.4426950408889634f;      // (not taken into the scores: the lowest bias times this is no number)
    float m = -INFINITY, z = 0.f;
    float acc[16];
    if constexpr (!ONCE) {
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] = 0.f;
    }
    // (A long row has the wave to itself and goes one way throughout: the choice inside the loop costs 15,135 rows of bfloat16 at 128
    // 62.4 us instead of 59.8. The registers of five waves to a SIMD hold the ordinary way; the other spills a few.)
    constexpr int SHORT_FORM = 0, LARGE = 1, BY_ROW = 2;
    auto walk = [&](auto way_) __attribute__((always_inline)) {
        constexpr int way = way_;
        for (int c0 = part * CH; ONCE || c0 < p.ell_w; c0 += S * CH) {
            if (!ONCE && ent[0].x == DG4_ELL_PAD) break;           // padding stands at the end only; the same for all lanes of the group
            uint4 kw[CH], vw[CH];
            uint32_t sw[CH];                          // scales: of K, and of V from bit 8
            float b[CH];
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const uint32_t e = j % 4 == 0 ? ent[j / 4].x : j % 4 == 1 ? ent[j / 4].y : j % 4 == 2 ? ent[j / 4].z : ent[j / 4].w;
                const float bj = bias[head][e >> 30];
                b[j] = e == DG4_ELL_PAD ? -INFINITY : bj;
                const bool none = b[j] == -INFINITY;
                if constexpr (FAR) {
                    const int64_t row = e & 0x3FFFFFFFu;
                    const uint8_t* at = none ? nothing : p.codes + row * (2 * D);
                    sw[j] = *(const uint16_t*)((none ? nothing : p.scales + row * (2 * HEADS)) + head * 2);
                    kw[j] = *(const uint4*)(at + sub * 16);
                    vw[j] = *(const uint4*)(at + D + sub * 16);
                } else {
                    const uint32_t row = none ? NONE : e & 0x3FFFFFFFu;
                    const int at = (int)(row * (2 * D) + sub * 16);
                    sw[j] = dg4_raw_buffer_load2(scale_bytes, (int)(row * (2 * HEADS) + head * 2), 0, 0);
                    kw[j] = __builtin_bit_cast(uint4, dg4_raw_buffer_load16(code_bytes, at, 0, 0));
                    vw[j] = __builtin_bit_cast(uint4, dg4_raw_buffer_load16(code_bytes, at + D, 0, 0));
                }
            }
            if constexpr (!ONCE) entries(c0 + S * CH);             // the next step's entries travel with this step's rows
            float s[CH];
            float cm = m;
            auto score = [&](int j, float dot, float factor) __attribute__((always_inline)) {
                dot += xor1(dot);
                // (zeros times a q that is not finite are NaN: an entry that is none has no product)
                dot = b[j] == -INFINITY ? 0.f : dot;
                s[j] = fmaf(dot, factor, b[j]);
                cm = fmaxf(cm, s[j]);
            };
            if (way == SHORT_FORM || (way == BY_ROW && !large)) {
#pragma unroll
                for (int j = 0; j < CH; ++j) score(j, q.dot(kw[j], sw[j] & 255u), FMT == DG4_KV_E4M3 ? c : scale_value(sw[j] & 255u) * c);
            } else if constexpr (LaneQ<T, FMT>::SHORT) {
#pragma unroll
                for (int j = 0; j < CH; ++j) {
                    // (taken as others than the words above, or what both ways share is kept in registers from before the branch)
                    uint4 w = kw[j];
                    __asm__ volatile("" : "+v"(w.x), "+v"(w.y), "+v"(w.z), "+v"(w.w));
                    score(j, q.dot_large(w, sw[j] & 255u), c);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            // What weights are relative to: the maximum; in a wave with steps to come (one row) what it was when some lane's last was more
            // than 4 past it, so that few steps have sums to scale down. e^4 < 2^6, which every weight there is divided by: no sum of V is
            // larger than it would be, and a source alone in its row still leaves as it is.
            // (Nothing so far, -inf: any finite base will do, every weight is 0.)
            if constexpr (ONCE) {
                m = cm;
            } else if (__any(cm > m + 4.f)) {
                const float corr = __builtin_amdgcn_exp2f((m - (cm == -INFINITY ? 0.f : cm)) * log2e);
                m = cm;
                z *= corr;
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[i] *= corr;
            }
            const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const float pj = __builtin_amdgcn_exp2f(ONCE ? (s[j] - base) * log2e : fmaf(s[j] - base, log2e, -6.f));
                z += pj;
                const float pv = FMT == DG4_KV_E4M3 ? pj : pj * scale_value(sw[j] >> 8);
                const uint32_t words[4] = { vw[j].x, vw[j].y, vw[j].z, vw[j].w };
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float x[4];
                    decode4_scaled<FMT>(words[i], sw[j] >> 8, x);
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[4 * i + k] = ONCE && j == 0 ? pv * x[k] : fmaf(pv, x[k], acc[4 * i + k]);
                }
            }
            if constexpr (ONCE) break;
        }
    };
    if constexpr (ONCE || !LaneQ<T, FMT>::SHORT) walk(std::integral_constant<int, BY_ROW>{});
    else if (large) walk(std::integral_constant<int, LARGE>{});
    else walk(std::integral_constant<int, SHORT_FORM>{});
    // join the groups of the row: one maximum, then sums, each exchange leaving a lane half the features it had
    constexpr int KEPT = 16 / S;
    int first = 0;
    if constexpr (S > 1) {
        float mm = m;
#pragma unroll
        for (int x = 1; x < S; x *= 2) mm = fmaxf(mm, __shfl_xor(mm, x * LPR));
        const float f = __builtin_amdgcn_exp2f((m - (mm == -INFINITY ? 0.f : mm)) * log2e);
        z *= f;
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] *= f;
        auto halve = [&](auto distance) __attribute__((always_inline)) {
            constexpr int x = distance, half = 16 * x / S;                 // features a lane keeps
            const bool upper = (group & x) != 0;
            z += __shfl_xor(z, x * LPR);
#pragma unroll
            for (int i = 0; i < half; ++i) {
                const float keep = upper ? acc[i + half] : acc[i], give = upper ? acc[i] : acc[i + half];
                acc[i] = keep + __shfl_xor(give, x * LPR);
            }
            first += upper ? half : 0;
        };
        static_assert(S <= 8 && KEPT % 2 == 0, "exchanges");
        if constexpr (S >= 8) halve(std::integral_constant<int, 4>{});
        if constexpr (S >= 4) halve(std::integral_constant<int, 2>{});
        halve(std::integral_constant<int, 1>{});
    }
    const float rz = z == 0.f ? 0.f : 1.0f / z;
    T* out = (T*)p.a + r * D + sub * 16 + first;
    constexpr int WORDS = KEPT * (int)sizeof(T) / 4;
    uint32_t w[WORDS];
#pragma unroll
    for (int i = 0; i < KEPT; i += 2) {
        if constexpr (sizeof(T) == 2) w[i / 2] = pack_bf16x2(acc[i] * rz, acc[i + 1] * rz);
        else { w[i] = __float_as_uint(acc[i] * rz); w[i + 1] = __float_as_uint(acc[i + 1] * rz); }
    }
    if constexpr (WORDS >= 4) {
#pragma unroll
        for (int i = 0; i < WORDS; i += 4) store_stream(out + i * (4 / (int)sizeof(T)), make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]));
    } else if constexpr (WORDS == 2) {
        *(uint2*)out = make_uint2(w[0], w[1]);
    } else {
        *(uint32_t*)out = w[0];
    }
}

// launch(args, workgroups) for the rows of a call. A launch holds fewer than 2^32 threads, 2^24 workgroups: longer calls take several.
template <typename A, typename F> int launch_rows(A a, int rows_per_block, F&& launch)
{
    const int64_t end = a.row_end, most = ((int64_t)1 << 23) * rows_per_block;
    for (; a.row_begin < end; a.row_begin = a.row_end) {
        a.row_end = std::min(end, a.row_begin + most);
        launch(a, dim3((unsigned)((a.row_end - a.row_begin + rows_per_block - 1) / rows_per_block)));
        if (const int e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <typename T, int FMT, int D>
int launch_write(const dg4_kv8_args& args, hipStream_t s)
{
    constexpr int U = 2;
    return launch_rows(args, 256 / (2 * D / 8) * U, [&](const dg4_kv8_args& a, dim3 grid) {
        hipLaunchKernelGGL((kv8_write_kernel<T, FMT, D, U>), grid, dim3(256), 0, s, a);
    });
}
template <typename T, int FMT, int D>
int launch_read(const dg4_kv8_args& args, hipStream_t s)
{
    constexpr int U = 2;
    return launch_rows(args, 256 / (2 * D / (16 / (int)sizeof(T))) * U, [&](const dg4_kv8_args& a, dim3 grid) {
        hipLaunchKernelGGL((kv8_read_kernel<T, FMT, D, U>), grid, dim3(256), 0, s, a);
    });
}
// The split goes by the table's width alone, so a row's result does not depend on which rows a call covers.
template <typename T, int FMT, int D, bool FAR>
int launch_attn_from(const dg4_kv8_attn_args& args, hipStream_t s)
{
    constexpr int GPW = 64 / (D / 16);
    const bool once = args.ell_w <= 16;
    return launch_rows(args, once ? 4 * GPW / 2 : 4, [&](const dg4_kv8_attn_args& a, dim3 grid) {
        if (a.ell_w <= 8) hipLaunchKernelGGL((kv8_attn_kernel<T, FMT, D, 2, 4, true, FAR>), grid, dim3(256), 0, s, a);
        else if (once) hipLaunchKernelGGL((kv8_attn_kernel<T, FMT, D, 2, 8, true, FAR>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((kv8_attn_kernel<T, FMT, D, GPW, 4, false, FAR>), grid, dim3(256), 0, s, a);
    });
}
template <typename T, int FMT, int D>
int launch_attn(const dg4_kv8_attn_args& a, hipStream_t s)
{
    return a.n * (2 * D) <= (int64_t)KV8_NEAR_BYTES ? launch_attn_from<T, FMT, D, false>(a, s) : launch_attn_from<T, FMT, D, true>(a, s);
}

// f<T, format, hidden>() of the call's configuration
template <typename F> int by_shape(int dtype, int format, int hidden, F&& f)
{
    auto with_type = [&](auto t) {
        using T = decltype(t);
        if (format == DG4_KV_E4M3) return hidden == 128 ? f(t, std::integral_constant<int, DG4_KV_E4M3>{}, std::integral_constant<int, 128>{})
                                                         : f(t, std::integral_constant<int, DG4_KV_E4M3>{}, std::integral_constant<int, 256>{});
        return hidden == 128 ? f(t, std::integral_constant<int, DG4_KV_INT8>{}, std::integral_constant<int, 128>{})
                             : f(t, std::integral_constant<int, DG4_KV_INT8>{}, std::integral_constant<int, 256>{});
    };
    return dtype == DG4_F32 ? with_type(float{}) : with_type(bf16_t{});
}

}  // namespace

int dg4_launch_kv8_write(int dtype, int format, int hidden, const dg4_kv8_args& a, hipStream_t s)
{
    return by_shape(dtype, format, hidden, [&](auto t, auto fmt, auto d) { return launch_write<decltype(t), fmt.value, d.value>(a, s); });
}
int dg4_launch_kv8_read(int dtype, int format, int hidden, const dg4_kv8_args& a, hipStream_t s)
{
    return by_shape(dtype, format, hidden, [&](auto t, auto fmt, auto d) { return launch_read<decltype(t), fmt.value, d.value>(a, s); });
}
int dg4_launch_kv8_attn(int dtype, int format, int hidden, const dg4_kv8_attn_args& a, hipStream_t s)
{
    return by_shape(dtype, format, hidden, [&](auto t, auto fmt, auto d) { return launch_attn<decltype(t), fmt.value, d.value>(a, s); });
}
