// The K|V store in 4 bits: rows written into it, read back, and attended over. A block is a head (32 features) of K or V.
//
//  kv4_write_kernel  a block's largest magnitude picks its power of two, every value divided by it is rounded once. HBM-bound.
//  kv4_read_kernel   the reverse.
//  kv4_attn_kernel   scores, softmax and aggregation over cone rows (Section 3.5) straight from the codes: the power of two of a
//                    head's K comes out of its dot product, that of its V into the entry's weight.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cstring>
#include <type_traits>

#include "dg4_device.h"
#include "dg4_fp4.h"
#include "dg4_internal.h"
#include "dg4_rowops.h"

namespace {

// Bytes of codes up to which buffer addressing is used: offsets are 32 bits, and there is room for one that is past the end
constexpr uint32_t KV4_NEAR_BYTES = 0xC0000000u;

// Which run of rows a workgroup takes. Workgroups go to the eight XCDs in turn, and neighbouring rows read the same sources: runs of 64
// workgroups (2048 rows of two hops at hidden 256) go to one XCD, so that its L2 serves them. (A million rows, runs of 16, 32, 64 and 128:
// 311, 300, 299 and 302 us.) What is left behind the last eight whole runs goes in turn.
__device__ __forceinline__ uint32_t kv4_block(uint32_t block, uint32_t blocks)
{
    constexpr uint32_t RUN = 64;
    const uint32_t base = block / (8 * RUN) * (8 * RUN);
    return base + 8 * RUN <= blocks ? base + block % 8 * RUN + (block - base) / 8 : block;
}

// A lane takes eight features, so a block is four lanes and a gate's K | V row a whole wave at hidden 256 (two gates at 128).
// U gates per lane, all requested before the first is used. Bound by HBM: 1, 2, 4 and 8 gates per lane take 216, 215, 227 and 232 us for a
// million rows of bfloat16 at hidden 256 (1.30 GB moved, 6.0 TB/s), 160, 169, 175 and 176 for 402,193 of fp32 and 2.1, 2.2, 2.5 and 3.1 for 264 of
// bfloat16: two of bfloat16, one of fp32. Codes leave through the caches, where the next level's attention finds them (past them: 209).
template <typename T, int D, int U>
__global__ __launch_bounds__(256) void kv4_write_kernel(dg4_kv8_args p)
{
    constexpr int LPG = 2 * D / 8;                // lanes per gate
    constexpr int GPB = 256 / LPG;                // gates per workgroup and pass
    const int sub = (int)threadIdx.x % LPG;
    const int64_t r0 = p.row_begin + (int64_t)blockIdx.x * (GPB * U) + (int)threadIdx.x / LPG;
    const bool is_v = sub >= LPG / 2;
    const int col = (sub % (LPG / 2)) * 8;
    const T* src = (const T*)(is_v ? p.v : p.k) + col;
    Values<T, 8> x[U];
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
        const uint32_t byte = fp4_scale_byte(max_of_lanes<4>(x[u].top()));
        uint32_t w[1];
        x[u].codes(byte << 23, w);
        if (byte == FP4_BAD) w[0] = 0;
        if (at[u] >= 0) {
            *(uint32_t*)(p.codes + at[u] * D + sub * 4) = w[0];
            if ((sub & 3) == 0) p.scales[at[u] * (2 * D / 32) + col / 32 * 2 + (is_v ? 1 : 0)] = (uint8_t)byte;
        }
    }
}

// A lane takes what it stores as 16 bytes, so that a wave's store is whole lines: four features of fp32, eight of bfloat16. U rows per lane:
// 232, 204 and 222 us with 1, 2 and 4 for a million rows of bfloat16 at hidden 256 (1.30 GB moved, 6.4 TB/s; 215 where rows leave through the
// caches), 128, 128 and 145 for 402,193 of fp32 (149).
template <typename T, int D, int U>
__global__ __launch_bounds__(256) void kv4_read_kernel(dg4_kv8_args p)
{
    constexpr int PER = 16 / (int)sizeof(T);
    constexpr int LPG = 2 * D / PER;
    constexpr int GPB = 256 / LPG;
    const int sub = (int)threadIdx.x % LPG;
    const int64_t r0 = p.row_begin + (int64_t)blockIdx.x * (GPB * U) + (int)threadIdx.x / LPG;
    const bool is_v = sub >= LPG / 2;
    const int col = (sub % (LPG / 2)) * PER;
    T* dst = (T*)(is_v ? p.v_out : p.k_out) + col;
    uint32_t w[U], byte[U];
    bool in[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t r = r0 + (int64_t)u * GPB;
        in[u] = r < p.row_end;
        int64_t at = 0;
        if (in[u]) at = p.ids ? (int64_t)p.ids[r] : r;
        in[u] = in[u] && at >= 0 && at < p.n_store;
        if (!in[u]) at = 0;                                   // (the store has a row: the launcher checks)
        const uint8_t* from = p.codes + at * D + sub * (PER / 2);
        if constexpr (PER == 8) w[u] = *(const uint32_t*)from;
        else w[u] = *(const uint16_t*)from;
        byte[u] = p.scales[at * (2 * D / 32) + col / 32 * 2 + (is_v ? 1 : 0)];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const float scale = __uint_as_float(byte[u] << 23);   // (the conversions take 0 and 255 for what they stand for)
        uint4 out;
        if constexpr (PER == 8) {
            out.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[u], scale, 0));
            out.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[u], scale, 1));
            out.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[u], scale, 2));
            out.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[u], scale, 3));
        } else {
            const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], scale, 1);
            out = make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
        }
        if (in[u]) store_stream(dst + (r0 + (int64_t)u * GPB) * D, out);
    }
}

// ------------------------------------------------------------------------------------------------- attention

// What an entry that is none reads where buffer addressing does not reach (FAR, below)
__device__ __align__(256) const uint8_t nothing4[256] = {};

__device__ dg4_i32x4 dg4_raw_buffer_load16(dg4_i32x4 rsrc, int voffset, int soffset, int aux) __asm("llvm.amdgcn.raw.buffer.load.v4i32");
__device__ uint16_t dg4_raw_buffer_load2(dg4_i32x4 rsrc, int voffset, int soffset, int aux) __asm("llvm.amdgcn.raw.buffer.load.i16");

// A head's 32 values of q in a lane, and their product with the 32 codes of a source's K, which the conversions multiply by their
// power of two (0: 2^-127, 255: NaN). fp32: value by value. bfloat16: as pairs, two products and a sum in fp32 per instruction, which
// takes what is below 2^-126 as zero. Values of K there cost a score nothing as long as |q| is at most 2^80 (32 * 2^-126 * 2^80), and values of
// q there do not occur in rows that have none: rows with a |q| above 2^80 or below 2^-126 take dot_exact, every product in fp32.
// A zero counts as below. Rows of a product in bfloat16 hold next to none, but of the rows of dg4_qkv_proj_mx4 and dg4_qkv_proj_kv4, sums of coarse
// steps, one in four to six has one, and a wave that holds such a row goes both ways. Time with Q of the one and of the other (us): a million
// rows of two hops at hidden 256 311 and 337 (at 128 170 and 176), 200,000 of three 97 and 135, 90,000 of four 83 and 118, 15,135 of eight
// at 128 56 and 62. (In a zero's place either way has the same product.)
constexpr uint32_t LARGE_Q = (127u + 80u) << 23;  // 2^80, as a float's bits
constexpr uint32_t SMALL_Q = 1u << 23;            // 2^-126
template <typename T> struct HeadQ;
template <> struct HeadQ<float> {
    static constexpr bool ONE_WAY = true;
    float q[32];
    __device__ __forceinline__ void load(const float* p)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) Elem<float>::unpack(((const uint4*)p)[2 * i], ((const uint4*)p)[2 * i + 1], q + 8 * i);
    }
    __device__ __forceinline__ bool odd() const { return false; }
    __device__ __forceinline__ float dot(const uint4& w, uint32_t byte) const
    {
        const uint32_t words[4] = { w.x, w.y, w.z, w.w };
        float d = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float k[8];
            fp4_get8(words[i], byte, k);
#pragma unroll
            for (int x = 0; x < 8; ++x) d = i + x == 0 ? q[0] * k[0] : fmaf(q[8 * i + x], k[x], d);
        }
        return d;
    }
    __device__ __forceinline__ float dot_exact(const uint4& w, uint32_t byte) const { return dot(w, byte); }
};
template <> struct HeadQ<bf16_t> {
    static constexpr bool ONE_WAY = false;
    uint4 q[4];
    __device__ __forceinline__ void load(const bf16_t* p)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = ((const uint4*)p)[i];
    }
    __device__ __forceinline__ bool odd() const
    {
        // Twice the bits, which leaves the sign out, less twice 2^-126's: what is below that is far above everything else
        constexpr uint16_t low = SMALL_Q >> 15;
        u16x2 top = { 0, 0 };
        const u16x2 twos = { 2, 2 }, lows = { low, low };
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w[4] = { q[i].x, q[i].y, q[i].z, q[i].w };
#pragma unroll
            for (int x = 0; x < 4; ++x) top = __builtin_elementwise_max(top, (u16x2)(__builtin_bit_cast(u16x2, w[x]) * twos - lows));
        }
        return max(top.x, top.y) > (LARGE_Q >> 15) - low;
    }
    __device__ __forceinline__ float dot(const uint4& w, uint32_t byte) const
    {
        const float scale = __uint_as_float(byte << 23);
        float d = 0.f;
        auto eight = [&](uint32_t codes, const uint4& x) __attribute__((always_inline)) {
            d = __builtin_amdgcn_fdot2_f32_bf16(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0), __builtin_bit_cast(bf16x2, x.x), d, false);
            d = __builtin_amdgcn_fdot2_f32_bf16(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1), __builtin_bit_cast(bf16x2, x.y), d, false);
            d = __builtin_amdgcn_fdot2_f32_bf16(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2), __builtin_bit_cast(bf16x2, x.z), d, false);
            d = __builtin_amdgcn_fdot2_f32_bf16(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3), __builtin_bit_cast(bf16x2, x.w), d, false);
        };
        eight(w.x, q[0]); eight(w.y, q[1]); eight(w.z, q[2]); eight(w.w, q[3]);
        return d;
    }
    __device__ __forceinline__ float dot_exact(const uint4& w, uint32_t byte) const
    {
        const uint32_t words[4] = { w.x, w.y, w.z, w.w };
        float d = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float k[8];
            fp4_get8(words[i], byte, k);
            uint32_t x[4] = { q[i].x, q[i].y, q[i].z, q[i].w };
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                __asm__ volatile("" : "+v"(x[j]));             // (unpacked here and not, for every row, ahead of the loop)
                d = fmaf(bf16_hi(x[j]), k[2 * j + 1], fmaf(bf16_lo(x[j]), k[2 * j], d));
            }
        }
        return d;
    }
};

// A lane owns a head of a destination row, a row is S groups of D / 32 lanes: a source's K codes are one load instruction over
// a whole line, its V codes another, and a score needs no other lane. The row's entries go to the groups in turn, CH at a time; each
// group keeps a running maximum, denominator and weighted sum (32 bits), joined at the end by lane exchange. ONCE: the groups take the
// whole row at one go. Entries that are none (padding, a relation whose bias is -inf) ask the buffers for an offset past the end: zeros, no
// request, no branch, and what the store holds there cannot matter. The offsets of buffer addressing are 32 bits: FAR, for larger stores,
// has addresses of 64 bits and reads zeros from memory for them.
// Measured. A million two-hop rows of bfloat16 at hidden 256, one source in five anywhere in the store: 300 to 313 us on several cards,
// 1.36 GB fetched past the L2s and 0.51 written, 6.0 TB/s; vector instructions keep the SIMDs for two thirds of it (912 for a
// wave's eight rows: 104 for an entry and lane, of which 80 convert and multiply codes). Six waves a SIMD instead of four (without the
// branch for rows of Q that are odd) change nothing. Two groups of four entries, which have to be joined: 327, in fp32 (300,000 rows) 197
// for 144. Lanes that store their own 64 bytes past the caches: 471; Q read past them: 366. Long rows are bound by vector instructions:
// 15,135 of eight hops at 128 take 56 us two entries a step, 64 with four, of which the row's last step leaves more unused; at hidden 256
// 99, with sums scaled down in every step 108.
template <typename T, int D, int S, int CH, bool ONCE, bool FAR>
__global__ __launch_bounds__(256) void kv4_attn_kernel(dg4_kv8_attn_args p)
{
    constexpr int LPR = D / 32, HEADS = D / 32, GPW = 64 / LPR, QUADS = (CH + 3) / 4;
    constexpr int RPW = GPW / S;                  // rows per wave
    constexpr uint32_t NONE = KV4_NEAR_BYTES / D; // past the end of a store that buffer addressing reaches
    static_assert((S == 1 && ONCE) || CH == 2 || CH % 4 == 0, "a group's entries are whole pieces");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int head = lane % LPR, group = lane / LPR, part = group % S;
    // biases of a head by relation code
    __shared__ float bias[HEADS][4];
    if (threadIdx.x < HEADS * 4) bias[threadIdx.x / 4][threadIdx.x % 4] = p.rel_bias[threadIdx.x];
    __syncthreads();
    const int64_t r = p.row_begin + ((int64_t)(ONCE ? kv4_block(blockIdx.x, gridDim.x) : blockIdx.x) * 4 + wave) * RPW + group / S;
    // (a row that is none goes along with the first gate's, if its wave holds another, and is not written)
    int64_t v = -1;
    if (r < p.row_end) v = p.ids ? (int64_t)p.ids[r] : r;
    const bool in = v >= 0 && v < p.n;
    const uint64_t rows_in = __ballot(in);
    if (rows_in == 0) return;
    if (!in) v = 0;

    const dg4_i32x4 code_bytes = row_buffer(p.codes, 0, FAR ? 0 : (uint32_t)(p.n * D));
    const dg4_i32x4 scale_bytes = row_buffer(p.scales, 0, FAR ? 0 : (uint32_t)(p.n * 2 * HEADS));
    const uint32_t* erow = p.ell + v * (int64_t)p.ell_w;
    uint32_t ent[4 * QUADS];
    auto entries = [&](int c0) __attribute__((always_inline)) {
        using Piece = std::conditional_t<CH == 2, uint2, uint4>;
        constexpr int E = sizeof(Piece) / 4;
#pragma unroll
        for (int i = 0; i < (CH + E - 1) / E; ++i) {
            Piece e;
            if (c0 + E * i < p.ell_w) e = *(const Piece*)(erow + c0 + E * i);
            else memset(&e, 0xFF, sizeof(e));
            memcpy(ent + E * i, &e, sizeof(e));
        }
    };
    entries(part * CH);
    HeadQ<T> q;
    q.load((const T*)p.q + (in ? r : p.row_begin) * D + head * 32);
    // whether it is so for some lane of the row: a row does not see its neighbours
    constexpr int LANES = LPR * S;
    auto some = [&](bool x) __attribute__((always_inline)) { return (__ballot(x) >> (lane / LANES * LANES) & (~0ull >> (64 - LANES))) != 0; };
    const bool odd = some(q.odd());
    const float c = 0.17677669529663687f;         // 1/sqrt(32)
    const float log2e = 1.4426950408889634f;      // (not taken into the scores: the lowest bias times this is no number)
    float m = -INFINITY, z = 0.f;
    float acc[32];
    if constexpr (!ONCE) {
#pragma unroll
        for (int i = 0; i < 32; ++i) acc[i] = 0.f;
    }
    for (int c0 = part * CH; ONCE || c0 < p.ell_w; c0 += S * CH) {
        if (!ONCE && ent[0] == DG4_ELL_PAD) break;           // padding stands at the end only; the same for all lanes of the group
        uint4 kw[CH], vw[CH];
        uint32_t sw[CH];                          // scales: of K, and of V from bit 8
        float b[CH];
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const uint32_t e = ent[j];
            const float bj = bias[head][e >> 30];
            b[j] = e == DG4_ELL_PAD ? -INFINITY : bj;
            const bool none = b[j] == -INFINITY;
            if constexpr (FAR) {
                const int64_t row = e & 0x3FFFFFFFu;
                const uint8_t* at = none ? nothing4 : p.codes + row * D;
                sw[j] = *(const uint16_t*)((none ? nothing4 : p.scales + row * (2 * HEADS)) + head * 2);
                kw[j] = *(const uint4*)(at + head * 16);
                vw[j] = *(const uint4*)(at + D / 2 + head * 16);
            } else {
                const uint32_t row = none ? NONE : e & 0x3FFFFFFFu;
                const int at = (int)(row * D + head * 16);
                sw[j] = dg4_raw_buffer_load2(scale_bytes, (int)(row * (2 * HEADS) + head * 2), 0, 0);
                kw[j] = __builtin_bit_cast(uint4, dg4_raw_buffer_load16(code_bytes, at, 0, 0));
                vw[j] = __builtin_bit_cast(uint4, dg4_raw_buffer_load16(code_bytes, at + D / 2, 0, 0));
            }
        }
        if constexpr (!ONCE) entries(c0 + S * CH);             // the next step's entries travel with this step's rows
        float s[CH];
        float cm = m;
        auto score = [&](int j, float dot) __attribute__((always_inline)) {
            // (zeros times a q that is not finite are NaN: an entry that is none has no product)
            dot = b[j] == -INFINITY ? 0.f : dot;
            s[j] = fmaf(dot, c, b[j]);
            cm = fmaxf(cm, s[j]);
        };
        if (HeadQ<T>::ONE_WAY || !odd) {
#pragma unroll
            for (int j = 0; j < CH; ++j) score(j, q.dot(kw[j], sw[j] & 255u));
        } else {
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                // (taken as others than the words above, or what both ways share is kept in registers from before the branch)
                uint4 w = kw[j];
                __asm__ volatile("" : "+v"(w.x), "+v"(w.y), "+v"(w.z), "+v"(w.w));
                score(j, q.dot_exact(w, sw[j] & 255u));
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        // What weights are relative to: the maximum; where there are steps to come, what it was when some lane of the row's last was more than 4
        // past it, so that few steps have sums to scale down. e^4 < 2^6, which every weight there is divided by: no sum of V is larger than it
        // would be, and a source alone in its row still leaves as it is. (Nothing so far, -inf: any finite base will do, every weight is 0.)
        if constexpr (ONCE) {
            m = cm;
        } else if (some(cm > m + 4.f)) {
            const float corr = __builtin_amdgcn_exp2f((m - (cm == -INFINITY ? 0.f : cm)) * log2e);
            m = cm;
            z *= corr;
#pragma unroll
            for (int i = 0; i < 32; ++i) acc[i] *= corr;
        }
        const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const float pj = __builtin_amdgcn_exp2f(ONCE ? (s[j] - base) * log2e : fmaf(s[j] - base, log2e, -6.f));
            z += pj;
            const uint32_t words[4] = { vw[j].x, vw[j].y, vw[j].z, vw[j].w };
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float x[8];
                fp4_get8(words[i], sw[j] >> 8, x);
#pragma unroll
                for (int k = 0; k < 8; ++k) acc[8 * i + k] = ONCE && j == 0 ? pj * x[k] : fmaf(pj, x[k], acc[8 * i + k]);
            }
        }
        if constexpr (ONCE) break;
    }
    // join the groups of the row: one maximum, then sums, each exchange leaving a lane half the features it had
    constexpr int KEPT = 32 / S;
    int first = 0;
    if constexpr (S > 1) {
        float mm = m;
#pragma unroll
        for (int x = 1; x < S; x *= 2) mm = fmaxf(mm, __shfl_xor(mm, x * LPR));
        const float f = __builtin_amdgcn_exp2f((m - (mm == -INFINITY ? 0.f : mm)) * log2e);
        z *= f;
#pragma unroll
        for (int i = 0; i < 32; ++i) acc[i] *= f;
        auto halve = [&](auto distance) __attribute__((always_inline)) {
            constexpr int x = distance, half = 32 * x / S;                 // features a lane keeps
            const bool upper = (group & x) != 0;
            z += __shfl_xor(z, x * LPR);
#pragma unroll
            for (int i = 0; i < half; ++i) {
                const float keep = upper ? acc[i + half] : acc[i], give = upper ? acc[i] : acc[i + half];
                acc[i] = keep + __shfl_xor(give, x * LPR);
            }
            first += upper ? half : 0;
        };
        static_assert(S <= 16, "exchanges");
        if constexpr (S >= 16) halve(std::integral_constant<int, 8>{});
        if constexpr (S >= 8) halve(std::integral_constant<int, 4>{});
        if constexpr (S >= 4) halve(std::integral_constant<int, 2>{});
        halve(std::integral_constant<int, 1>{});
    }
    const float rz = z == 0.f ? 0.f : 1.0f / z;
    constexpr int WORDS = KEPT * (int)sizeof(T) / 4;
    uint32_t w[WORDS];
#pragma unroll
    for (int i = 0; i < KEPT; i += 2) {
        if constexpr (sizeof(T) == 2) w[i / 2] = pack_bf16x2(acc[i] * rz, acc[i + 1] * rz);
        else { w[i] = __float_as_uint(acc[i] * rz); w[i + 1] = __float_as_uint(acc[i + 1] * rz); }
    }
    if constexpr (WORDS > 4) {
        // A lane's pieces of 16 bytes go through LDS (the wave's own part of it), so that a store is whole rows: 64 pieces side by side
        constexpr int PIECES = WORDS / 4, PPR = D * (int)sizeof(T) / 16;
        __shared__ uint4 stage[4][64 * (PIECES + 1)];
        const int place = ((group / S) * LPR + head) * S + first / KEPT;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) stage[wave][place * (PIECES + 1) + i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const int64_t r0 = r - group / S;         // the wave's first row
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int piece = lane + 64 * i;
            const uint4 x = stage[wave][piece / PIECES * (PIECES + 1) + piece % PIECES];
            if (rows_in >> (piece / PPR * LANES) & 1) store_stream((T*)p.a + r0 * D + piece * (16 / (int)sizeof(T)), x);
        }
    } else if (in) {
        T* out = (T*)p.a + r * D + head * 32 + first;
        if constexpr (WORDS == 4) store_stream(out, make_uint4(w[0], w[1], w[2], w[3]));
        else if constexpr (WORDS == 2) *(uint2*)out = make_uint2(w[0], w[1]);
        else *(uint32_t*)out = w[0];
    }
}

// f(args, workgroups), a launch, for the rows of a call. A launch holds fewer than 2^32 threads, 2^24 workgroups: longer calls take several.
template <typename A, typename F> int launch_rows(A a, int rows_per_block, F&& f)
{
    const int64_t end = a.row_end, most = ((int64_t)1 << 23) * rows_per_block;
    for (; a.row_begin < end; a.row_begin = a.row_end) {
        a.row_end = std::min(end, a.row_begin + most);
        if (const int e = f(a, dim3((unsigned)((a.row_end - a.row_begin + rows_per_block - 1) / rows_per_block))); e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <typename T, int D>
int launch_write(const dg4_kv8_args& args, hipStream_t s)
{
    constexpr int U = sizeof(T) == 2 ? 2 : 1;
    return launch_rows(args, 256 / (2 * D / 8) * U, [&](const dg4_kv8_args& a, dim3 grid) {
        return launch(kv4_write_kernel<T, D, U>, grid, 256, s, a);
    });
}
template <typename T, int D>
int launch_read(const dg4_kv8_args& args, hipStream_t s)
{
    constexpr int U = 2;
    return launch_rows(args, 256 / (2 * D / (16 / (int)sizeof(T))) * U, [&](const dg4_kv8_args& a, dim3 grid) {
        return launch(kv4_read_kernel<T, D, U>, grid, 256, s, a);
    });
}
// The split of a row goes by the cones' depth alone, so its result does not depend on which rows a call covers. A cone of one hop
// holds three gates, of two hops seven, fifteen, ...; MOST: what a call's cones hold at most. Measured with 1, 2, 4, 8 groups a row in bfloat16 (us;
// two entries a step): 90,000 rows of four hops at 256 80, 83, 92, 119, but 1000 at 128 12.5, 7.9, 5.4, 4.8; 60,000 of five hops at 128 60, 56, 55,
// 61; 30,000 of six hops at 256 107, 89, 82, 84; 20,000 of seven hops at 128 106, 72, 56, 51 (sixteen: 52); 15,135 of eight hops at 128 153, 101,
// 72, 61 (sixteen: 56). Three hops go in one go by two groups, for calls of few rows: 1000 of fp32 at 256 take 5.6 where one group with four
// entries a step takes 8.6. Calls of many pay 5 to 8 % for it, or nothing: 200,000 rows of bfloat16 at 256 101 (one group 102), at 128 58.0 (53.7),
// 60,000 of fp32 at 256 42.9 (40.7), 100,000 at 128 41.0 (37.6).
template <typename T, int D, bool FAR, int MOST>
int launch_attn_of(const dg4_kv8_attn_args& args, hipStream_t s)
{
    constexpr int GPW = 64 / (D / 32);
    constexpr bool ONCE = MOST <= 15;
    constexpr int S = MOST <= 7 ? 1 : MOST <= 31 ? 2 : MOST <= 127 ? 4 : MOST <= 255 ? 8 : GPW;
    constexpr int CH = MOST <= 7 ? MOST : ONCE ? 8 : 2;
    return launch_rows(args, 4 * GPW / S, [&](const dg4_kv8_attn_args& a, dim3 grid) {
        return launch(kv4_attn_kernel<T, D, S, CH, ONCE, FAR>, grid, 256, s, a);
    });
}
template <typename T, int D, bool FAR>
int launch_attn_from(const dg4_kv8_attn_args& a, hipStream_t s)
{
    return a.most <= 3 ? launch_attn_of<T, D, FAR, 3>(a, s) : a.most <= 7 ? launch_attn_of<T, D, FAR, 7>(a, s)
         : a.most <= 15 ? launch_attn_of<T, D, FAR, 15>(a, s) : a.most <= 31 ? launch_attn_of<T, D, FAR, 31>(a, s)
         : a.most <= 127 ? launch_attn_of<T, D, FAR, 127>(a, s) : a.most <= 255 ? launch_attn_of<T, D, FAR, 255>(a, s)
         : launch_attn_of<T, D, FAR, 511>(a, s);
}
template <typename T, int D>
int launch_attn(const dg4_kv8_attn_args& a, hipStream_t s)
{
    return a.n * D <= (int64_t)KV4_NEAR_BYTES ? launch_attn_from<T, D, false>(a, s) : launch_attn_from<T, D, true>(a, s);
}

// f<T, hidden>() of the call's configuration
template <typename F> int by_shape(int dtype, int hidden, F&& f)
{
    auto with_type = [&](auto t) { return hidden == 128 ? f(t, std::integral_constant<int, 128>{}) : f(t, std::integral_constant<int, 256>{}); };
    return dtype == DG4_F32 ? with_type(float{}) : with_type(bf16_t{});
}

}  // namespace

int dg4_launch_kv4_write(int dtype, int hidden, const dg4_kv8_args& a, hipStream_t s)
{
    return by_shape(dtype, hidden, [&](auto t, auto d) { return launch_write<decltype(t), d.value>(a, s); });
}
int dg4_launch_kv4_read(int dtype, int hidden, const dg4_kv8_args& a, hipStream_t s)
{
    return by_shape(dtype, hidden, [&](auto t, auto d) { return launch_read<decltype(t), d.value>(a, s); });
}
int dg4_launch_kv4_attn(int dtype, int hidden, const dg4_kv8_attn_args& a, hipStream_t s)
{
    return by_shape(dtype, hidden, [&](auto t, auto d) { return launch_attn<decltype(t), d.value>(a, s); });
}
