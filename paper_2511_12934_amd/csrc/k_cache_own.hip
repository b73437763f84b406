// The user cache's attention for many rows of narrow heads (up to 64 features): a wave takes 32 CT rows and brings keys and values
// to bf16 for itself.
//
// Up to 64 features a tile of 32 keys is 32 conversions of two codes, a fifth of what its 64 rows' softmax takes (see
// k_cache_many.hip): less than a share in staging, and no wave waits for another.  Keys go from memory to registers to the 32x32x16 products; of a
// tile's 32 keys a lane holds one, half of its features, whichever stand in which slot (heads of up to 16 features: eight, one product).  Values are turned through the wave's own
// LDS, as in k_cache_few.  Tile n + 1's codes travel while tile n is worked on.
// 8 x 10^4 rows of eight heads of 16 over 2,000 keys: 255 us; the exponentials alone, 1.28e9, are 150.
#include "k_cache_attend.h"

namespace aif {

namespace {

template <int DT, int NW, int CT, int KS> __global__ __launch_bounds__(256, 2) void k_cache_own(CacheFew few /* first: kernel_arg */, const char *dev, CacheGrid g, CacheShape c, float *part)
{
    constexpr int DP = 32 * NW, NP = DT == 0 ? 3 : 1, ROWS = 128 * CT;
    __shared__ __align__(16) char lds[4][CACHE_TILE * 2 * DP];
    (void)few;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5, kvh = blockIdx.y;
    const AskUnit found = block_ask(dev, g, lane);
    const CacheAsk &a = found.a;
    const int unit = found.unit, n_rows = a.n_q * c.group, in_block = 32 * CT * wave;
    int row_tile = unit, split = 0;
    if (a.splits > 1) row_tile = unit / a.splits, split = unit % a.splits;
    const char *pool = as_global(c.pool) + (size_t)kvh * cache_head_bytes(c);
    const float k2 = c.scale * LOG2E;
    typedef s16x4 __attribute__((address_space(3))) *lds4_t;
    char *mine = lds[wave];
    const int row0 = row_tile * ROWS + in_block;
    if (row0 >= n_rows) return;                 // no wave waits for another

    RowOf rows[CT];
    Sight see[CT];
    Reach reach;
#pragma unroll
    for (int i = 0; i < CT; ++i) {
        const int row = row0 + 32 * i + col;
        rows[i] = row_of(c, kvh, row < n_rows ? row : row0);
        see[i] = sight_of(a, rows[i].i, row < n_rows);
        reach.add(see[i], row < n_rows);
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
    TileList<DP> list;
    list.fill(c, a, walk, t, 1, t_end, lane);
    struct Raw {
        uint32_t k[KS], v[KS], ks, vs;          // words of eight codes: features half 8 KS on, of a key
        bool here;
    };
    const uint32_t word_at = col * (DP / 2) + half * (4 * KS), byte_at = col * NW + (NW == 2 ? half : 0);
    auto ask = [&](int t, Raw &raw) {           // a tile that is dropped or behind the end reads page 0, which nobody sees
        if (t - list.from == 64) list.fill(c, a, walk, t, 1, t_end, lane);
        const int64_t off = list.offset(t - list.from);
        const char *tile = pool + (off < 0 ? 0 : off);
        __builtin_memcpy(raw.k, __builtin_assume_aligned(tile + word_at, 4 * KS), 4 * KS);
        __builtin_memcpy(raw.v, __builtin_assume_aligned(tile + 16 * DP + word_at, 4 * KS), 4 * KS);
        raw.ks = *(const uint8_t *)(tile + 32 * DP + byte_at);
        raw.vs = *(const uint8_t *)(tile + 33 * DP + byte_at);
        raw.here = off >= 0;
    };

    bf16x8 q[CT][NP][KS], kf[KS], vf[2][NW];
    // The first product of row tile o of a tile whose keys kf holds, or, `fresh`, has yet to hold: step k of it.
    auto scores = [&](int o, int k, f32x16 &so) {
        if (k == 0)
#pragma unroll
            for (int e = 0; e < 16; ++e) so[e] = 0.f;
#pragma unroll
        for (int p = NP - 1; p >= 0; --p) so = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[k], q[o][p][k], so, 0, 0, 0);
    };
    // One phase: the weights of row tile i from its scores si beside the scores so of row tile o, then their product with the values.
    // fresh: the keys for so are those of `keys`, from here on.
    auto phase = [&](int i, f32x16 &si, int o, f32x16 &so, bool fresh, Raw &keys, int tile, bool here) {
        if (!here || !walk.whole(tile)) see[i].hide(si, here ? tile * CACHE_TILE + 4 * half : NO_KEY);
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, si[e]);
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
        if (fresh) asm volatile("" : "+v"(keys.ks));
        const float ks = scale_of(keys.ks);
        float x[16];
        constexpr int EACH = 16 / KS;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            if (fresh) kf[k] = decode8(keys.k[k], ks);
            scores(o, k, so);
#pragma unroll
            for (int e = EACH * k; e < EACH * (k + 1); ++e) x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(si[e], k2, -ref));
            __builtin_amdgcn_sched_barrier(0);
        }
        bf16x8 weights[2][NP];
        pieces8<NP>(x, weights[0]);
        pieces8<NP>(x + 8, weights[1]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int f = 0; f < NW; ++f) {
#pragma unroll
                for (int p = NP - 1; p >= 0; --p) acc[i][f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[k][f], weights[k][p], acc[i][f], 0, 0, 0);
#pragma unroll
                for (int e = 8 * k + 8 / NW * f; e < 8 * k + 8 / NW * (f + 1); ++e) l[i] += x[e];
                __builtin_amdgcn_sched_barrier(0);
            }
    };
    // Tile t: its scores s0 (of row tile 0) are there, kf holds its keys where CT = 2, and `next` the codes of the tile behind it,
    // whose scores s1 (CT = 1; of row tile 0 again: s0) are there in the end.
    auto step = [&](int t, Raw &now, Raw &next, f32x16 &s0, f32x16 &s1) {
        asm volatile("" : "+v"(now.vs));        // (made use of here, not where it is asked for)
        const int tile = walk.tile(t);
        const bool here = now.here;
        // a block of values that is not finite becomes zeros: who sees it gets NaN below
        float vs = scale_of(now.vs);
        const bool fine = vs < 0x1p126f;
        vs = fine ? vs : 1.f;
#pragma unroll
        for (int w = 0; w < KS; ++w) *(bf16x8 *)(mine + v_place<DP>(col, half * KS + w)) = decode8(fine ? now.v[w] : 0u, vs);
        ask(t + 2, now);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int f = 0; f < NW; ++f) {
                union {
                    s16x4 h[2];
                    bf16x8 all;
                } v;
                const int key = 16 * k + 4 * half, feature = 32 * f + 16 * (lane >> 4 & 1);
                v.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_t)(mine + v_turned<DP>(key, feature, lane)));
                v.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_t)(mine + v_turned<DP>(key + 8, feature, lane)));
                vf[k][f] = v.all;
            }
        if constexpr (CT == 2) {
            phase(0, s0, 1, s1, false, next, tile, here);
            phase(1, s1, 0, s0, true, next, tile, here);
        } else
            phase(0, s0, 0, s1, true, next, tile, here);
        if (__ballot(!fine && here && tile * CACHE_TILE + col <= reach.hi_last)) {
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
    f32x16 s0, s1;
    ask(t, raw0);
    ask(t + 1, raw1);
#pragma unroll
    for (int i = 0; i < CT; ++i) {              // (the queries come while the first tiles do)
        const char *qr = a.q + (size_t)rows[i].i * a.q_stride + (size_t)rows[i].head * c.d_head * (DT == 0 ? 4 : 2);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            bf16x8 p[NP];
            query8<DT, NP>(qr, half * (8 * KS) + 8 * k, c.d_head, row0 + 32 * i + col < n_rows, p);
#pragma unroll
            for (int j = 0; j < NP; ++j) q[i][j][k] = p[j];
        }
    }
    asm volatile("" : "+v"(raw0.ks));
#pragma unroll
    for (int k = 0; k < KS; ++k) {
        kf[k] = decode8(raw0.k[k], scale_of(raw0.ks));
        scores(0, k, s0);
    }
    for (; t < t_end; t += 2) {
        if constexpr (CT == 2) {
            step(t, raw0, raw1, s0, s1);
            step(t + 1, raw1, raw0, s0, s1);
        } else {
            step(t, raw0, raw1, s0, s1);
            step(t + 1, raw1, raw0, s1, s0);
        }
    }
    finish_rows<DT, NW, CT, ROWS>(a, c, part, kvh, unit, n_rows, row0 - in_block, in_block, col, half, acc, m, l);
}

template <int DT, int NW, int CT> void own(const CacheFew &args, const char *dev, const CacheGrid &g, const CacheShape &c, const CachePart &p, hipStream_t s)
{
    const dim3 grid = cache_grid(g, c, p), block(256);
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
