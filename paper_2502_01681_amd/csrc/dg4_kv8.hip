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

#include "dg4_device.h"
#include "dg4_internal.h"

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));

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
template <int FMT> __device__ __forceinline__ void decode16(const uint4& w, float* f)
{
    decode4<FMT>(w.x, f); decode4<FMT>(w.y, f + 4); decode4<FMT>(w.z, f + 8); decode4<FMT>(w.w, f + 12);
}

// Eight values of a row in one lane, as loaded
template <typename T> struct Eight;
template <> struct Eight<float> {
    uint4 a, b;
    __device__ void load(const float* p) { a = ((const uint4*)p)[0]; b = ((const uint4*)p)[1]; }
    __device__ void get(float* f) const { Elem<float>::unpack(a, b, f); }
    __device__ static void put(const float* f, float* p) { uint4 a, b; Elem<float>::pack(f, a, b); ((uint4*)p)[0] = a; ((uint4*)p)[1] = b; }
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
    __device__ static void put(const float* f, bf16_t* p)
    {
        *(uint4*)p = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
    }
};

// A lane takes eight features, so a head is four lanes and a gate's K | V row a whole wave at hidden 256 (two gates at
// 128): one 512-byte (256-byte) row of codes per store instruction. U gates per lane, all requested before the first is used.
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

template <typename T, int FMT, int D, int U>
__global__ __launch_bounds__(256) void kv8_read_kernel(dg4_kv8_args p)
{
    constexpr int LPG = 2 * D / 8;
    constexpr int GPB = 256 / LPG;
    const int sub = (int)threadIdx.x % LPG;
    const int64_t r0 = p.row_begin + (int64_t)blockIdx.x * (GPB * U) + (int)threadIdx.x / LPG;
    const bool is_v = sub >= LPG / 2;
    const int col = (sub % (LPG / 2)) * 8;
    T* dst = (T*)(is_v ? p.v_out : p.k_out) + col;
    uint2 w[U];
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
        w[u] = *(const uint2*)(p.codes + at * (2 * D) + sub * 8);
        byte[u] = p.scales[at * (2 * D / 32) + (sub % (LPG / 2)) / 4 * 2 + (is_v ? 1 : 0)];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float f[8];
        decode4<FMT>(w[u].x, f); decode4<FMT>(w[u].y, f + 4);
        const float scale = scale_value(byte[u]);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] *= scale;
        if (in[u]) Eight<T>::put(f, dst + (r0 + (int64_t)u * GPB) * D);
    }
}

// ------------------------------------------------------------------------------------------------- attention

// One destination row per S groups of D / 16 lanes; a lane owns 16 features (half a head). Chunks of CH entries go to the
// groups in turn, each keeps a running maximum, denominator and weighted sum (32 bits), and the groups' results are joined
// at the end: by lane exchange inside a wave, through LDS where WPR waves share the row. Entries that are none (padding, a
// relation whose bias is -inf) are not read, so what the store holds there cannot matter.
template <typename T, int FMT, int D, int S, int WPR, int CH>
__global__ __launch_bounds__(256) void kv8_attn_kernel(dg4_kv8_attn_args p)
{
    constexpr int LPR = D / 16, GPW = 64 / LPR;
    constexpr int RPW = GPW / S;                  // rows per wave
    static_assert(WPR == 1 || (S == GPW && WPR == 4), "a row is a part of a wave, a wave or the workgroup");
    constexpr int PARTS = S * WPR;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int sub = lane % LPR, group = lane / LPR;
    const int part = WPR == 1 ? group % S : wave * S + group;
    const int64_t r = WPR == 1 ? p.row_begin + ((int64_t)blockIdx.x * 4 + wave) * RPW + group / S : p.row_begin + blockIdx.x;
    // (what leaves here leaves as whole rows)
    if (r >= p.row_end) return;
    const int64_t v = p.ids ? (int64_t)p.ids[r] : r;
    if (v < 0 || v >= p.n) return;
    const int head = sub >> 1;

    const uint8_t* codes = p.codes + sub * 16;
    const uint8_t* scales = p.scales + head * 2;
    const uint32_t* erow = p.ell + v * (int64_t)p.ell_w;
    auto entries = [&](int c0, uint32_t (&e)[CH]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < CH; i += 4) {
            const uint4 e4 = c0 + i < p.ell_w ? *(const uint4*)(erow + c0 + i) : make_uint4(DG4_ELL_PAD, DG4_ELL_PAD, DG4_ELL_PAD, DG4_ELL_PAD);
            e[i] = e4.x; e[i + 1] = e4.y; e[i + 2] = e4.z; e[i + 3] = e4.w;
        }
    };
    uint32_t ent[CH];
    entries(part * CH, ent);
    const float* bp = p.rel_bias + head * 4;
    const float4 bias = make_float4(bp[0], bp[1], bp[2], bp[3]);
    float q[16];
    {
        const uint4* qp = (const uint4*)((const T*)p.q + r * D + sub * 16);
        if constexpr (sizeof(T) == 2) {
            Elem<bf16_t>::unpack(qp[0], qp[1], q);
        } else {
            Elem<float>::unpack(qp[0], qp[1], q);
            Elem<float>::unpack(qp[2], qp[3], q + 8);
        }
    }
    const float c = 0.17677669529663687f;         // 1/sqrt(32)
    const float log2e = 1.4426950408889634f;
    float m = -INFINITY, z = 0.f;
    float acc[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;

    for (int c0 = part * CH; c0 < p.ell_w; c0 += PARTS * CH) {
        if (ent[0] == DG4_ELL_PAD) break;         // padding stands at the end only; the same for all lanes of the group
        uint4 kw[CH], vw[CH];
        uint32_t sw[CH];
        float b[CH];
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const uint32_t rel = ent[j] >> 30;
            b[j] = ent[j] == DG4_ELL_PAD ? -INFINITY : rel == 0 ? bias.x : rel == 1 ? bias.y : rel == 2 ? bias.z : bias.w;
            if (b[j] != -INFINITY) {
                const int64_t row = ent[j] & 0x3FFFFFFFu;
                sw[j] = *(const uint16_t*)(scales + row * (2 * D / 32));
                kw[j] = *(const uint4*)(codes + row * (2 * D));
                vw[j] = *(const uint4*)(codes + row * (2 * D) + D);
            } else {
                sw[j] = 0;
                kw[j] = make_uint4(0, 0, 0, 0); vw[j] = kw[j];
            }
        }
        entries(c0 + PARTS * CH, ent);            // the next step's entries travel with this step's rows
        float s[CH];
        float cm = m;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            float k[16];
            decode16<FMT>(kw[j], k);
            float dot = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) dot = fmaf(q[i], k[i], dot);
            dot += xor1(dot);
            s[j] = b[j] == -INFINITY ? -INFINITY : fmaf(dot, scale_value(sw[j] & 255u) * c, b[j]);
            cm = fmaxf(cm, s[j]);
        }
        // (nothing so far: any finite base will do, every weight is 0)
        const float base = cm == -INFINITY ? 0.f : cm;
        const float corr = __builtin_amdgcn_exp2f((m - base) * log2e);
        z *= corr;
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] *= corr;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const float pj = __builtin_amdgcn_exp2f((s[j] - base) * log2e);
            z += pj;
            const float pv = pj * scale_value(sw[j] >> 8);
            float x[16];
            decode16<FMT>(vw[j], x);
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[i] = fmaf(pv, x[i], acc[i]);
        }
        m = cm;
    }
    // join the groups of the row
    auto join = [&](float m2, float z2, auto&& other) __attribute__((always_inline)) {
        const float mm = fmaxf(m, m2), base = mm == -INFINITY ? 0.f : mm;
        const float a = __builtin_amdgcn_exp2f((m - base) * log2e), b = __builtin_amdgcn_exp2f((m2 - base) * log2e);
        z = z * a + z2 * b;
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] = acc[i] * a + other(i) * b;
        m = mm;
    };
#pragma unroll
    for (int x = 1; x < S; x *= 2) join(__shfl_xor(m, x * LPR), __shfl_xor(z, x * LPR), [&](int i) { return __shfl_xor(acc[i], x * LPR); });
    if constexpr (WPR > 1) {
        __shared__ float sm[WPR][LPR], sz[WPR][LPR], sacc[WPR][16][LPR];
        if (group == 0) {
            sm[wave][sub] = m; sz[wave][sub] = z;
#pragma unroll
            for (int i = 0; i < 16; ++i) sacc[wave][i][sub] = acc[i];
        }
        __syncthreads();
        if (wave != 0) return;
#pragma unroll
        for (int w = 1; w < WPR; ++w) join(sm[w][sub], sz[w][sub], [&](int i) { return sacc[w][i][sub]; });
    }
    if (group % S != 0) return;
    const float rz = z == 0.f ? 0.f : 1.0f / z;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] *= rz;
    uint4* op = (uint4*)((T*)p.a + r * D + sub * 16);
    if constexpr (sizeof(T) == 2) {
        uint4 oa, ob;
        Elem<bf16_t>::pack(acc, oa, ob);
        op[0] = oa; op[1] = ob;
    } else {
        uint4 oa, ob;
        Elem<float>::pack(acc, oa, ob);
        op[0] = oa; op[1] = ob;
        Elem<float>::pack(acc + 8, oa, ob);
        op[2] = oa; op[3] = ob;
    }
}

template <typename T, int FMT, int D>
int launch_write(const dg4_kv8_args& a, hipStream_t s)
{
    constexpr int GPB = 256 / (2 * D / 8);
    const int64_t rows = a.row_end - a.row_begin;
    const unsigned grid = (unsigned)((rows + GPB * 4 - 1) / (GPB * 4));
    hipLaunchKernelGGL((kv8_write_kernel<T, FMT, D, 4>), dim3(grid), dim3(256), 0, s, a);
    return hipGetLastError();
}
template <typename T, int FMT, int D>
int launch_read(const dg4_kv8_args& a, hipStream_t s)
{
    constexpr int GPB = 256 / (2 * D / 8);
    const int64_t rows = a.row_end - a.row_begin;
    const unsigned grid = (unsigned)((rows + GPB * 4 - 1) / (GPB * 4));
    hipLaunchKernelGGL((kv8_read_kernel<T, FMT, D, 4>), dim3(grid), dim3(256), 0, s, a);
    return hipGetLastError();
}
// The split goes by the table's width alone, so a row's result does not depend on which rows a call covers.
template <typename T, int FMT, int D>
int launch_attn(const dg4_kv8_attn_args& a, hipStream_t s)
{
    constexpr int GPW = 64 / (D / 16);
    const int64_t rows = a.row_end - a.row_begin;
    auto grid = [&](int rows_per_block) { return dim3((unsigned)((rows + rows_per_block - 1) / rows_per_block)); };
    if (a.ell_w <= 8)
        hipLaunchKernelGGL((kv8_attn_kernel<T, FMT, D, 1, 1, 8>), grid(4 * GPW), dim3(256), 0, s, a);
    else if (a.ell_w <= 16)
        hipLaunchKernelGGL((kv8_attn_kernel<T, FMT, D, 2, 1, 8>), grid(4 * GPW / 2), dim3(256), 0, s, a);
    else if (a.ell_w <= 64)
        hipLaunchKernelGGL((kv8_attn_kernel<T, FMT, D, GPW, 1, 8>), grid(4), dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((kv8_attn_kernel<T, FMT, D, GPW, 4, 8>), grid(1), dim3(256), 0, s, a);
    return hipGetLastError();
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
