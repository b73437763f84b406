// The user cache's attention for many rows of narrow heads (up to 64 features): a wave takes 32 CT rows and brings keys and values
// to bf16 for itself.
//
// Up to 64 features a tile of 32 keys is 32 conversions of two codes, a fifth of what its 64 rows' softmax takes (see
// k_cache_many.hip): less than a share in staging, and no wave waits for another.  Keys go from memory to registers to the 32x32x16 products; of a
// tile's 32 keys a lane holds one, half of its features, whichever stand in which slot (heads of up to 16 features: eight, one product).  Values are turned through the wave's own
// LDS, as in k_cache_few.  Tile n + 1's codes travel while tile n is worked on.
#include "k_cache_attend.h"

namespace aif {

namespace {

template <int DT, int NW, int CT, int KS> __global__ __launch_bounds__(256, 2) void k_cache_own(CacheFew few /* first: kernel_arg */, const char *dev, CacheGrid g, CacheShape c, float *part)
{
    constexpr int DP = 32 * NW, NP = DT == 0 ? 3 : 1, ROWS = 128 * CT, VST = v_stride(DP);
    __shared__ __align__(16) char lds[4][CACHE_TILE * VST];
    (void)few;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5, kvh = blockIdx.y;
    const int r = ask_of(dev, g, blockIdx.x, lane);
    const CacheAsk a = ask_at(dev, r);
    int row_tile = (int)blockIdx.x - first_at(dev, g, r), split = 0;
    const int unit = row_tile;
    if (a.splits > 1) row_tile = unit / a.splits, split = unit % a.splits;
    const int n_rows = a.n_q * c.group, in_block = 32 * CT * wave, row0 = row_tile * ROWS + in_block;
    if (row0 >= n_rows) return;                 // no wave waits for another

    Sight see[CT];
    bf16x8 q[CT][NP][KS];
    Reach reach;
#pragma unroll
    for (int t = 0; t < CT; ++t) {
        const int row = row0 + 32 * t + col;
        const bool is_row = row < n_rows;
        const RowOf o = row_of(c, kvh, is_row ? row : row0);
        see[t] = sight_of(a, o.i, is_row);
        reach.add(see[t], is_row);
        const char *qr = a.q + (size_t)o.i * a.q_stride + (size_t)o.head * c.d_head * (DT == 0 ? 4 : 2);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            bf16x8 p[NP];
            query8<DT, NP>(qr, half * (8 * KS) + 8 * k, c.d_head, is_row, p);
#pragma unroll
            for (int i = 0; i < NP; ++i) q[t][i][k] = p[i];
        }
    }
    const Walk walk = reach.walk<32>(a);
    int t = 0, t_end = walk.count();
    if (a.splits > 1) {
        const int64_t n = t_end;
        t = (int)(n * split / a.splits);
        t_end = (int)(n * (split + 1) / a.splits);
    }

    f32x16 acc[CT][NW];
    float m[CT], l[CT];
#pragma unroll
    for (int i = 0; i < CT; ++i) {
        m[i] = -INFINITY, l[i] = 0.f;
#pragma unroll
        for (int f = 0; f < NW; ++f)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][f][e] = 0.f;
    }
    const float k2 = c.scale * LOG2E;
    typedef s16x4 __attribute__((address_space(3))) *lds4_t;
    char *mine = lds[wave];
    // four keys of 16 features a group of 16 lanes
    const char *turned = mine + (4 * half + (lane & 15) / 4) * VST + 32 * (lane >> 4 & 1) + (lane & 3) * 8;

    const char *pool = as_global(c.pool) + (size_t)kvh * cache_head_bytes(c);
    TileList<DP> list;
    list.fill(c, a, walk, t, 1, t_end, lane);
    struct Raw {
        uint32_t k[KS], v[KS], ks, vs;             // words of eight codes: features half 8 KS on, of a key
        bool here;
    };
    const uint32_t word_at = col * (DP / 2) + half * (4 * KS), byte_at = col * NW + (NW == 2 ? half : 0);
    auto ask = [&](int t, Raw &raw) {           // a tile that is dropped or behind the end reads page 0
        if (t - list.from == 64) list.fill(c, a, walk, t, 1, t_end, lane);
        const int64_t off = list.offset(t - list.from);
        const char *tile = pool + (off < 0 ? 0 : off);
        __builtin_memcpy(raw.k, __builtin_assume_aligned(tile + word_at, 4 * KS), 4 * KS);
        __builtin_memcpy(raw.v, __builtin_assume_aligned(tile + 16 * DP + word_at, 4 * KS), 4 * KS);
        raw.ks = *(const uint8_t *)(tile + 32 * DP + byte_at);
        raw.vs = *(const uint8_t *)(tile + 33 * DP + byte_at);
        raw.here = off >= 0;
    };
    auto work = [&](int t, Raw &now) {
        if (!now.here) return;
        asm volatile("" : "+v"(now.ks), "+v"(now.vs));      // (made use of here, not where they are asked for)
        const int tile = walk.tile(t), j0 = tile * CACHE_TILE + 4 * half;

        f32x16 s[CT];
#pragma unroll
        for (int i = 0; i < CT; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[i][e] = 0.f;
        const float ks = scale_of(now.ks);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const bf16x8 kf = decode8(now.k[k], ks);
#pragma unroll
            for (int i = 0; i < CT; ++i)
#pragma unroll
                for (int p = NP - 1; p >= 0; --p) s[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[i][p][k], s[i], 0, 0, 0);
        }
        // a block of values that is not finite becomes zeros: who sees it gets NaN below
        float vs = scale_of(now.vs);
        const bool fine = vs < 0x1p126f;
        vs = fine ? vs : 1.f;
#pragma unroll
        for (int w = 0; w < KS; ++w) *(bf16x8 *)(mine + col * VST + (half * KS + w) * 16) = decode8(fine ? now.v[w] : 0u, vs);

        const bool whole = walk.whole(tile);
        bf16x8 weights[CT][2][NP];
#pragma unroll
        for (int i = 0; i < CT; ++i) {
            if (!whole) see[i].hide(s[i], j0, tile, walk.sinks);
            float top = -INFINITY;
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, s[i][e]);
            top *= k2;
            if (__ballot(top > m[i] + LAZY)) {
                top = fmaxf(top, __shfl_xor(top, 32));
                const float m2 = fmaxf(m[i], top);
                if (__ballot(m[i] != -INFINITY)) {
                    const float back = m2 == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[i] - m2);
                    l[i] *= back;
#pragma unroll
                    for (int f = 0; f < NW; ++f) acc[i][f] *= back;
                }
                m[i] = m2;
            }
            const float ref = m[i] == -INFINITY ? 0.f : m[i];
            float x[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][e], k2, -ref));
                l[i] += x[e];
            }
            pieces8<NP>(x, weights[i][0]);
            pieces8<NP>(x + 8, weights[i][1]);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int f = 0; f < NW; ++f) {
                union {
                    s16x4 h[2];
                    bf16x8 all;
                } v;
                v.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_t)(turned + 16 * k * VST + 64 * f));
                v.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_t)(turned + (16 * k + 8) * VST + 64 * f));
#pragma unroll
                for (int i = 0; i < CT; ++i)
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p) acc[i][f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v.all, weights[i][k][p], acc[i][f], 0, 0, 0);
            }
        if (__ballot(!fine && tile * CACHE_TILE + col <= reach.hi_last)) {
            // a row that sees a block of values that is not finite: its features are NaN
#pragma unroll 1
            for (int key = 0; key < CACHE_TILE; ++key)
#pragma unroll
                for (int f = 0; f < NW; ++f) {
                    if (__shfl(fine ? 1 : 0, key + 32 * f)) continue;       // (lane half f holds block f; one block: either)
#pragma unroll
                    for (int i = 0; i < CT; ++i)
                        if (see[i].sees(tile * CACHE_TILE + key)) acc[i][f] += __builtin_nanf("");
                }
        }
    };
    // two sets of registers by turns: what one is loaded with is not waited for while the other is worked on
    Raw raw0, raw1;
    ask(t, raw0);
    for (; t < t_end; t += 2) {
        ask(t + 1, raw1);
        work(t, raw0);
        ask(t + 2, raw0);
        if (t + 1 < t_end) work(t + 1, raw1);
    }
    finish_rows<DT, NW, CT, ROWS>(a, c, part, kvh, unit, n_rows, row_tile * ROWS, in_block, col, half, acc, m, l);
}

template <int DT, int NW, int CT> void own(const CacheFew &args, const char *dev, const CacheGrid &g, const CacheShape &c, const CachePart &p, hipStream_t s)
{
    const dim3 grid(p.units, c.n_kv), block(256);
    if constexpr (NW == 1)
        if (c.d_head <= 16) {
            hipLaunchKernelGGL((k_cache_own<DT, NW, CT, 1>), grid, block, 0, s, args, dev, g, c, p.part);
            return;
        }
    hipLaunchKernelGGL((k_cache_own<DT, NW, CT, 2 * NW>), grid, block, 0, s, args, dev, g, c, p.part);
}

}  // namespace

void launch_cache_own(const CacheFew &args, const char *dev, const CacheGrid &g, const CacheShape &c, const CachePart &p, hipStream_t s)
{
    if (c.dp == 32) {
        if (c.dtype == 0) own<0, 1, 1>(args, dev, g, c, p, s);
        else if (p.rows_of_tile == 128) own<1, 1, 1>(args, dev, g, c, p, s);
        else own<1, 1, 2>(args, dev, g, c, p, s);
    } else {
        if (c.dtype == 0) own<0, 2, 1>(args, dev, g, c, p, s);
        else if (p.rows_of_tile == 128) own<1, 2, 1>(args, dev, g, c, p, s);
        else own<1, 2, 2>(args, dev, g, c, p, s);
    }
}

}  // namespace aif
