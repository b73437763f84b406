// The user cache's pages: rows in and out, table entries, whole pages moved (include/aif_cache.h).
// All of it is data movement.  A thread takes eight features of a row, which is four bytes of codes; the four threads of a
// block of 32 features find its largest magnitude among themselves.
#include "aif_cache_dev.h"

namespace aif {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// features [at, at + 8) of a row of d features, zeros past its end
template <int DT> __device__ __forceinline__ void load8(const char *row, int at, int d, float *x)
{
    if constexpr (DT == 0) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (at + 4 * h < d) v = *(const float4 *)(row + 4 * (at + 4 * h));
            x[4 * h] = v.x, x[4 * h + 1] = v.y, x[4 * h + 2] = v.z, x[4 * h + 3] = v.w;
        }
    } else {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (at < d) v = *(const uint4 *)(row + 2 * at);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

template <int DT> __device__ __forceinline__ void store8(char *row, int at, int d, uint32_t codes, float scale)
{
    if constexpr (DT == 0) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            bf16x2 v;
            if (i == 0) v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
            if (i == 1) v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
            if (i == 2) v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
            if (i == 3) v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
            const uint32_t w = __builtin_bit_cast(uint32_t, v);
            x[2 * i] = __uint_as_float(w << 16), x[2 * i + 1] = __uint_as_float(w & 0xffff0000u);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (at + 4 * h < d) *(float4 *)(row + 4 * (at + 4 * h)) = make_float4(x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]);
    } else if (at < d) {
        uint4 v;
        v.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
        v.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
        v.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
        v.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
        *(uint4 *)(row + 2 * at) = v;
    }
}

// Eight features as codes, and the byte of the block that this thread and its three neighbours hold (all four lanes active).
__device__ __forceinline__ uint32_t encode8(const float *x, uint32_t &byte)
{
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t m = __float_as_uint(x[i]) & 0x7fffffffu;
        most = m > most ? m : most;
    }
#pragma unroll
    for (int o = 1; o < 4; o *= 2) {
        const uint32_t m = __shfl_xor(most, o);
        most = m > most ? m : most;
    }
    // most = f 2^E with f in [1, 2): e = E - 2 where f <= 3/2, else E - 1; the sum's exponent is E + 1 just where f > 3/2
    int e = (int)((most + 0x3fffffu) >> 23) - 127 - 2;
    e = e < CACHE_E_MIN ? CACHE_E_MIN : e > CACHE_E_MAX ? CACHE_E_MAX : e;
    const bool finite = most < 0x7f800000u;
    byte = finite ? (uint32_t)(e + 127) : CACHE_NAN;
    const float scale = __uint_as_float((uint32_t)(e + 127) << 23);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], scale, 3);
    return finite ? c : 0;
}

// where a row's codes and scales lie in its head's part of a page
struct RowAt {
    char *codes, *scales;       // the keys'; the values' are 16 dp and 32 dp / 32 bytes behind
};
__device__ __forceinline__ RowAt row_at(char *head, int dp, int row)
{
    char *tile = head + (size_t)(row / CACHE_TILE) * cache_tile_bytes(dp);
    const int r = row % CACHE_TILE;
    return RowAt{tile + r * (dp / 2), tile + 32 * dp + r * (dp / 32)};
}

// One block: one unit, one head.  It names the page in the table, brings the rows that a shared page held, and writes its own.
template <int DT, class ARGS> __global__ __launch_bounds__(256) void k_cache_append(ARGS list, CacheShape c)
{
    const CacheUnit u = cache_desc<CacheUnit>(list, (size_t)blockIdx.x * sizeof(CacheUnit));
    const int head = blockIdx.y, dp = c.dp, per_row = dp / 8, esz = DT == 0 ? 4 : 2;
    char *page = c.pool + (size_t)u.page * c.page_bytes + (size_t)head * cache_head_bytes(c);
    if (threadIdx.x == 0 && head == 0) c.table[u.entry] = u.page;
    if (u.cow >= 0) {
        const char *from = c.pool + (size_t)u.cow * c.page_bytes + (size_t)head * cache_head_bytes(c);
        // codes in pieces of 16 bytes, scales byte by byte: the rest of either belongs to rows that this launch writes
        const int pieces = dp / 32, nb = dp / 32;
        for (int i = threadIdx.x; i < u.row0 * pieces; i += 256) {
            const int row = i / pieces, at = i % pieces * 16;
            const RowAt a = row_at((char *)from, dp, row), b = row_at(page, dp, row);
            *(uint4 *)(b.codes + at) = *(const uint4 *)(a.codes + at);
            *(uint4 *)(b.codes + 16 * dp + at) = *(const uint4 *)(a.codes + 16 * dp + at);
        }
        for (int i = threadIdx.x; i < u.row0 * nb; i += 256) {
            const int row = i / nb, at = i % nb;
            const RowAt a = row_at((char *)from, dp, row), b = row_at(page, dp, row);
            b.scales[at] = a.scales[at];
            b.scales[dp + at] = a.scales[dp + at];
        }
    }
    for (int i = threadIdx.x; i < 2 * u.n * per_row; i += 256) {
        const int half = i >= u.n * per_row, j = half ? i - u.n * per_row : i;
        const int row = j / per_row, at = j % per_row * 8;
        const char *src = (half ? u.vals + (size_t)row * u.val_stride * esz : u.keys + (size_t)row * u.key_stride * esz) + (size_t)head * c.d_head * esz;
        float x[8];
        load8<DT>(src, at, c.d_head, x);
        uint32_t byte;
        const uint32_t codes = encode8(x, byte);
        const RowAt to = row_at(page, dp, u.row0 + row);
        *(uint32_t *)(to.codes + (half ? 16 * dp : 0) + at / 2) = codes;
        if (at % CACHE_BLOCK == 0) to.scales[(half ? dp : 0) + at / CACHE_BLOCK] = (char)byte;
    }
}

// The way back: rows of a page to keys and vals (null: not wanted), which are written.
template <int DT, class ARGS> __global__ __launch_bounds__(256) void k_cache_read(ARGS list, CacheShape c)
{
    const CacheUnit u = cache_desc<CacheUnit>(list, (size_t)blockIdx.x * sizeof(CacheUnit));
    const int head = blockIdx.y, dp = c.dp, per_row = dp / 8, esz = DT == 0 ? 4 : 2;
    char *page = c.pool + (size_t)u.page * c.page_bytes + (size_t)head * cache_head_bytes(c);
    for (int i = threadIdx.x; i < 2 * u.n * per_row; i += 256) {
        const int half = i >= u.n * per_row, j = half ? i - u.n * per_row : i;
        const int row = j / per_row, at = j % per_row * 8;
        char *dst = const_cast<char *>(half ? u.vals : u.keys);
        if (!dst) continue;
        dst += (size_t)row * (half ? u.val_stride : u.key_stride) * esz + (size_t)head * c.d_head * esz;
        const RowAt from = row_at(page, dp, u.row0 + row);
        const uint32_t codes = *(const uint32_t *)(from.codes + (half ? 16 * dp : 0) + at / 2);
        const uint32_t byte = (uint8_t)from.scales[(half ? dp : 0) + at / CACHE_BLOCK];
        store8<DT>(dst, at, c.d_head, codes, __uint_as_float(byte << 23));
    }
}

template <class ARGS> __global__ __launch_bounds__(256) void k_cache_fill(ARGS list, int32_t *table)
{
    const CacheFill f = cache_desc<CacheFill>(list, (size_t)blockIdx.x * sizeof(CacheFill));
    const int i = blockIdx.y * 256 + threadIdx.x;
    if (i < f.n) table[f.dst + i] = f.src < 0 ? f.value : table[f.src + i];
}

constexpr int MOVE_BYTES = 4 * 16 * 256;        // of one block: four pieces a thread in flight

template <class ARGS> __global__ __launch_bounds__(256) void k_cache_move(ARGS list, CacheShape c)
{
    const CacheMove m = cache_desc<CacheMove>(list, (size_t)blockIdx.x * sizeof(CacheMove));
    if (m.entry >= 0 && blockIdx.y == 0 && threadIdx.x == 0) c.table[m.entry] = m.dst;
    if (m.src < 0) return;
    const uint4 *src = (const uint4 *)(c.pool + (size_t)m.src * c.page_bytes);
    uint4 *dst = (uint4 *)(c.pool + (size_t)m.dst * c.page_bytes);
    const int n = (int)(c.page_bytes / 16), at = blockIdx.y * (MOVE_BYTES / 16) + threadIdx.x;
    uint4 v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (at + 256 * j < n) v[j] = src[at + 256 * j];
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (at + 256 * j < n) dst[at + 256 * j] = v[j];
}

}  // namespace

hipError_t launch_cache_append(const CacheShape &c, const CacheList &units, hipStream_t s)
{
    if (units.n == 0) return hipSuccess;
    return cache_launch(units, [&](auto args) {
        using A = decltype(args);
        const dim3 grid(units.n, c.n_kv);
        if (c.dtype == 0) hipLaunchKernelGGL((k_cache_append<0, A>), grid, dim3(256), 0, s, args, c);
        else hipLaunchKernelGGL((k_cache_append<1, A>), grid, dim3(256), 0, s, args, c);
    });
}

hipError_t launch_cache_read(const CacheShape &c, const CacheList &units, hipStream_t s)
{
    if (units.n == 0) return hipSuccess;
    return cache_launch(units, [&](auto args) {
        using A = decltype(args);
        const dim3 grid(units.n, c.n_kv);
        if (c.dtype == 0) hipLaunchKernelGGL((k_cache_read<0, A>), grid, dim3(256), 0, s, args, c);
        else hipLaunchKernelGGL((k_cache_read<1, A>), grid, dim3(256), 0, s, args, c);
    });
}

hipError_t launch_cache_fill(const CacheShape &c, const CacheList &fills, int longest, hipStream_t s)
{
    if (fills.n == 0 || longest == 0) return hipSuccess;
    return cache_launch(fills, [&](auto args) {
        hipLaunchKernelGGL((k_cache_fill<decltype(args)>), dim3(fills.n, (longest + 255) / 256), dim3(256), 0, s, args, c.table);
    });
}

hipError_t launch_cache_move(const CacheShape &c, const CacheList &moves, hipStream_t s)
{
    if (moves.n == 0) return hipSuccess;
    return cache_launch(moves, [&](auto args) {
        hipLaunchKernelGGL((k_cache_move<decltype(args)>), dim3(moves.n, (unsigned)((c.page_bytes + MOVE_BYTES - 1) / MOVE_BYTES)), dim3(256), 0, s, args, c);
    });
}

}  // namespace aif
