// What the kernels of 8-bit products have in common (k_q8_few.hip, k_q8_many.hip).
//
// A product of 16 rows of weights by 16 rows of a over a block of 128 columns is one v_mfma_scale_f32_16x16x128_f8f6f4: a lane
// brings 32 codes of a row and that row's scale byte for the block, the powers of two are applied inside, and the sum is fp32.
// Which 32 of the 128 columns a lane holds need only be the same on both sides.  The weights are the first operand, so that a
// lane ends up with neighbouring columns of a result row.
//
// That instruction adds eight neighbouring products at a time and cuts off what lies 13 binary places below the largest one's
// exponent (found by trying it: 1 + 2^-13 comes out whole, 1 + 2^-14 as 1, while between groups of eight and with the sum all
// of fp32 counts): 1.5 - 2.3 10^-5 of a result in 2-norm, where bf16's rounding is 70 to 110 times that.  So it serves results in bf16 and in
// 8 bits.  With dtype fp32 the codes are brought into bf16, in which they are exact with their power of two, and multiplied there
// (1.2 10^-7): half the rate, and an instruction for every two codes.
#pragma once
#include "k_q8.h"

namespace aif {

// Rows of fp32 or bf16: N neighbouring values (4 or 8) of them.
template <bool F32, int N> __device__ __forceinline__ void load_values(const void *p, int64_t i, float (&v)[N])
{
    if constexpr (F32) {
#pragma unroll
        for (int e = 0; e < N; e += 4) {
            const q8_f4 u = *(const q8_f4 *)((const float *)p + i + e);
            v[e] = u[0], v[e + 1] = u[1], v[e + 2] = u[2], v[e + 3] = u[3];
        }
    } else {
        typedef uint32_t words __attribute__((ext_vector_type(N / 2)));
        const words u = *(const words *)((const uint16_t *)p + i);
#pragma unroll
        for (int e = 0; e < N; e += 2) v[e] = q8_bf16(u[e / 2] & 0xffffu), v[e + 1] = __uint_as_float(u[e / 2] & 0xffff0000u);
    }
}
template <bool F32, int N> __device__ __forceinline__ void store_values(void *p, int64_t i, const float (&v)[N])
{
    if constexpr (F32) {
#pragma unroll
        for (int e = 0; e < N; e += 4) *(q8_f4 *)((float *)p + i + e) = q8_f4{v[e], v[e + 1], v[e + 2], v[e + 3]};
    } else {
        typedef uint32_t words __attribute__((ext_vector_type(N / 2)));
        words u;
#pragma unroll
        for (int e = 0; e < N; e += 2) u[e / 2] = q8_two_bf16(v[e], v[e + 1]);
        *(words *)((uint16_t *)p + i) = u;
    }
}

// Value e of 16 bytes of such a row.
template <bool F32> __device__ __forceinline__ float value_of(q8_u4 u, int e)
{
    if constexpr (F32) return __uint_as_float(u[e]);
    return __uint_as_float(e % 2 ? u[e / 2] & 0xffff0000u : u[e / 2] << 16);
}

// 16 codes of a row from column `at` on, zeros from k on (a multiple of 8).
__device__ __forceinline__ q8_u4 load16(const uint8_t *row, int at, int k)
{
    if (at + 16 <= k) return *(const q8_u4 *)(row + at);
    if (at >= k) return q8_u4{};
    const q8_u2 v = *(const q8_u2 *)(row + at);
    return q8_u4{v[0], v[1], 0, 0};
}

// 32 codes in bf16, times their power of two.
struct Wide {
    q8_b8 v[4];
};
__device__ __forceinline__ Wide widen(q8_i8 c, int scale)
{
    Wide w;
    const float unit = __uint_as_float((uint32_t)scale << 23);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const q8_b2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)c[i], unit, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)c[i], unit, true);
        w.v[i / 2][i % 2 * 4] = lo[0], w.v[i / 2][i % 2 * 4 + 1] = lo[1], w.v[i / 2][i % 2 * 4 + 2] = hi[0], w.v[i / 2][i % 2 * 4 + 3] = hi[1];
    }
    return w;
}

// One operand of a product as the instructions take it.
// WHOLE: for results in fp32.
template <bool WHOLE> struct Side {
    q8_i8 codes;
    int scale;
    __device__ __forceinline__ Side(q8_i8 c, int s) : codes(c), scale(s) {}
};
template <> struct Side<true> {
    Wide w;
    __device__ __forceinline__ Side(q8_i8 c, int s) : w(widen(c, s)) {}
};

__device__ __forceinline__ q8_f4 mma(const Side<false> &w, const Side<false> &a, q8_f4 acc)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w.codes, a.codes, acc, 0, 0, 0, w.scale, 0, a.scale);
}
__device__ __forceinline__ q8_f4 mma(const Side<true> &w, const Side<true> &a, q8_f4 acc)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.w.v[i], a.w.v[i], acc, 0, 0, 0);
    return acc;
}

// z / (1 + exp(-z)) for every z whose result is a normal number, down to -92: exp(-z) itself passes 2^128 at -88.7, and the reciprocal instruction gives
// nothing for what is above 2^126, so that both are held 2^-8 smaller.  Off by (|z| / 2 + 6.8) 2^-23 of the result: the exponent's rounding grows with |z|, as does
// what the last bit of z itself is worth (through the root of exp(-|z|), with the exponent's rounding made good, 7 2^-23 throughout: fp32 gated 32000 x 512 x 2048 in
// 8 bits 181 us, with expf 192, without either 155).  The reciprocal times 2^-8 has steps of 2^-149 behind z = -87, which bf16 and codes do not see; for fp32 half of the 2^-8 goes to z, and
// it has them behind -90.
template <bool WHOLE> __device__ __forceinline__ float silu(float z)
{
    const float r = __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(__builtin_fmaf(z, -1.44269504f, -8.0f)) + 0x1p-8f);
    return WHOLE ? (z * 0x1p-4f) * (r * 0x1p-4f) : z * (r * 0x1p-8f);
}

}  // namespace aif
