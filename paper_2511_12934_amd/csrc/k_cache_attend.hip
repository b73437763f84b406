// Attention over sequences held in 4 bits (include/aif_cache.h: aif_cache_attend).
//
// One wave to a query row and head: 64 keys at a time, a lane to a key for the scores (the row's features from LDS), a lane
// to four features for the values.  One pass over the sequence with a running maximum m and sum l:
//   m' = max(m, s),  l' = l 2^(m - m') + sum 2^(s - m'),  o' = o 2^(m - m') + sum 2^(s - m') v,   s = score log2 e
#include "aif_cache_dev.h"

namespace aif {

namespace {

__device__ __forceinline__ float code_value(uint32_t c, float scale)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0);
    return __uint_as_float(__builtin_bit_cast(uint32_t, v) << 16);
}

template <int DT, class ARGS> __global__ __launch_bounds__(64) void k_cache_attend_row(ARGS list, CacheShape c, int n)
{
    __shared__ float qs[CACHE_MAX_DP];
    const size_t firsts = (size_t)n * sizeof(CacheAsk);
    const int lane = threadIdx.x, row = blockIdx.x, head = blockIdx.y;
    int r = 0;
    while (cache_desc<int32_t>(list, firsts + 4 * (size_t)(r + 1)) <= row) ++r;
    const CacheAsk a = cache_desc<CacheAsk>(list, (size_t)r * sizeof(CacheAsk));
    const int i = row - cache_desc<int32_t>(list, firsts + 4 * (size_t)r), esz = DT == 0 ? 4 : 2;
    const char *q = a.q + (size_t)i * a.q_stride + (size_t)head * c.d_head * esz;
    for (int f = lane; f < c.dp; f += 64) {
        float x = 0.f;
        if (f < c.d_head) x = DT == 0 ? ((const float *)q)[f] : bf2f(((const uint16_t *)q)[f]);
        qs[f] = x;
    }
    __syncthreads();
    int p = a.pos ? a.pos[i] : a.len - 1;
    p = p < -1 ? -1 : p;
    const float k2 = c.scale * 1.44269504088896340736f;
    const size_t head_at = (size_t)(head / c.group) * cache_head_bytes(c);
    float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    const int end = p < a.len - 1 ? p + 1 : a.len;
    for (int base = 0; base < end; base += 64) {
        const int j = base + lane;
        bool see = j < end && (a.window == 0 || j > p - a.window || j < a.sinks);
        int page = -1;
        if (see) page = c.table[a.entry + j / c.page_len];
        see = page >= 0;
        const char *tile = c.pool + (size_t)(see ? page : 0) * c.page_bytes + head_at + (size_t)(j % c.page_len / CACHE_TILE) * cache_tile_bytes(c.dp);
        const int jr = j % CACHE_TILE, nb = c.dp / 32;
        float s = -INFINITY;
        if (see) {
            float sum = 0.f;
            for (int b = 0; b < nb; ++b) {
                const float scale = __uint_as_float((uint32_t)(uint8_t)tile[32 * c.dp + jr * nb + b] << 23);
                for (int w = 0; w < 4; ++w) {
                    const uint32_t codes = *(const uint32_t *)(tile + jr * (c.dp / 2) + 16 * b + 4 * w);
                    for (int e = 0; e < 8; ++e) sum += qs[32 * b + 8 * w + e] * code_value(codes >> (4 * e), scale);
                }
            }
            s = sum * k2;
        }
        float most = s;
        for (int d = 1; d < 64; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
        const float m2 = fmaxf(m, most), ref = m2 == -INFINITY ? 0.f : m2;
        const float w = see ? __builtin_amdgcn_exp2f(s - ref) : 0.f, back = __builtin_amdgcn_exp2f(m - ref);
        m = m2;
        float sum = w;
        for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
        l = l * back + sum;
        for (int f = 0; f < 4; ++f) o[f] *= back;
        unsigned long long seen = __ballot(see);
        while (seen) {
            const int t = __ffsll(seen) - 1;
            seen &= seen - 1;
            const float wt = __shfl(w, t);
            const char *vt = (const char *)(((unsigned long long)(uint32_t)__shfl((int)((uintptr_t)tile >> 32), t) << 32) | (uint32_t)__shfl((int)(uintptr_t)tile, t));
            const int vr = (base + t) % CACHE_TILE;
            if (4 * lane < c.dp) {
                const uint32_t codes = *(const uint16_t *)(vt + 16 * c.dp + vr * (c.dp / 2) + 2 * lane);
                const float scale = __uint_as_float((uint32_t)(uint8_t)vt[33 * c.dp + vr * nb + lane / 8] << 23);
                for (int f = 0; f < 4; ++f) o[f] += wt * code_value(codes >> (4 * f), scale);
            }
        }
    }
    char *out = a.out + (size_t)i * a.out_stride + (size_t)head * c.d_head * esz;
    for (int f = 0; f < 4; ++f)
        if (4 * lane + f < c.d_head) {
            const float v = l == 0.f ? 0.f : o[f] / l;
            if (DT == 0) ((float *)out)[4 * lane + f] = v;
            else ((uint16_t *)out)[4 * lane + f] = f2bf(v);
        }
    if (a.lse && lane == 0) a.lse[(size_t)i * c.n_heads + head] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
}

}  // namespace

hipError_t launch_cache_attend(const CacheShape &c, const CacheList &asks, int64_t rows, hipStream_t s)
{
    if (rows == 0) return hipSuccess;
    return cache_launch(asks, [&](auto args) {
        using A = decltype(args);
        const dim3 grid((unsigned)rows, c.n_heads);
        if (c.dtype == 0) hipLaunchKernelGGL((k_cache_attend_row<0, A>), grid, dim3(64), 0, s, args, c, asks.n);
        else hipLaunchKernelGGL((k_cache_attend_row<1, A>), grid, dim3(64), 0, s, args, c, asks.n);
    });
}

}  // namespace aif
