// Attention over sequences held in 4 bits (include/aif_cache.h: aif_cache_attend).
//
// One pass over a sequence with a running maximum m and sum l of a row's weights, in powers of two:
//   s = scale log2 e <q, k>,  m' = max(m, s),  l' = l 2^(m - m') + sum 2^(s - m'),  o' = o 2^(m - m') + sum 2^(s - m') v
// and o / l at the end.  Any reference in the place of m gives the same quotient, so m only follows a maximum that has grown by
// more than 2^8 beyond it: the weights stay below 2^8, and nearly every tile goes without a reduction across lanes.
//
// k_cache_few.  What bounds it is the cache itself, 34 dp bytes per kv head and 32 keys, read once.  A wave takes 32 keys at a
// time.  Codes go from memory to registers to bf16 (exact: v_cvt_scalef32_pk_bf16_fp4, two codes an instruction) and on to
// the 16x16x32 products: S^T = K Q^T (a lane's codes of a key are the k-slots; which features stand in which slot is free, so a
// lane takes dp / 4 neighbouring ones), whose result leaves a lane with eight keys of ONE row: the weights are the second
// product's operand where they are, O^T = V^T P^T.  V has to be turned, features to rows: bf16 rows of 32 keys in the wave's own LDS,
// read back by ds_read_b64_tr_b16 (four keys of one feature a lane; which lanes meet in a bank: v_place).  No barrier in the loop; the four or eight waves of a block take the tiles in turn, each
// with the next tile's codes already asked for, and join through LDS.  16 users' histories of 131,072 behaviours, 4 kv heads of 128, one query of 16 heads:
// 207 us, 5.5 TB/s.  With 32 rows to a tile conversions, products and softmax take as long as the bytes do: 0.25 us a tile and block at heads of 128, the bytes
// at that rate 0.20.  Short calls take the launch, 4 us of loads one behind the other (arguments, table, codes), and the
// join's launch where keys are split.
#include "k_cache_attend.h"

namespace aif {

namespace {

// What a lane holds of a tile: of key lane % 16 (+ 16) the features [lane / 16 * dp / 4, + dp / 4), NW words of eight.
// (blocks that a lane's NW words can lie in)
template <int NW> constexpr int blocks_of() { return NW == 7 ? 3 : NW == 3 || NW > 4 ? 2 : 1; }
template <int NW> struct RawTile {
    uint32_t k[2][NW], v[2][NW], ks[2][blocks_of<NW>()], vs[2][blocks_of<NW>()];    // ks, vs: scale bytes, from the first block of the lane's features on
    bool here;
    // what is made of the bytes is made behind this, not where they are asked for: that would wait for them
    __device__ __forceinline__ void pin()
    {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int b = 0; b < blocks_of<NW>(); ++b) asm volatile("" : "+v"(ks[h][b]), "+v"(vs[h][b]));
    }
};

template <int NW> __device__ __forceinline__ void load_words(const char *p, uint32_t *w)
{
    if constexpr (NW % 4 == 0) {
#pragma unroll
        for (int i = 0; i < NW / 4; ++i) {
            const uint4 x = ((const uint4 *)p)[i];
            w[4 * i] = x.x, w[4 * i + 1] = x.y, w[4 * i + 2] = x.z, w[4 * i + 3] = x.w;
        }
    } else if constexpr (NW % 2 == 0) {
#pragma unroll
        for (int i = 0; i < NW / 2; ++i) {
            const uint2 x = ((const uint2 *)p)[i];
            w[2 * i] = x.x, w[2 * i + 1] = x.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < NW; ++i) w[i] = ((const uint32_t *)p)[i];
    }
}

template <int NW> __device__ __forceinline__ void load_tile(const char *tile, int lane, RawTile<NW> &r)
{
    constexpr int DP = 32 * NW;
    const int key = lane & 15, grp = lane >> 4, lo = grp * NW / 4;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int row = 16 * h + key;
        load_words<NW>(tile + row * (DP / 2) + grp * (DP / 8), r.k[h]);
        load_words<NW>(tile + 16 * DP + row * (DP / 2) + grp * (DP / 8), r.v[h]);
        const uint8_t *ks = (const uint8_t *)tile + 32 * DP + row * NW, *vs = ks + DP;
#pragma unroll
        for (int b = 0; b < blocks_of<NW>(); ++b) {         // (the last group may hold fewer blocks)
            const int at = lo + b < NW ? lo + b : NW - 1;
            r.ks[h][b] = ks[at];
            r.vs[h][b] = vs[at];
        }
    }
}

// the scale of word w of a lane's NW
template <int NW> __device__ __forceinline__ float word_scale(const uint32_t (&bytes)[blocks_of<NW>()], int grp, int w)
{
    uint32_t b = bytes[0];
    if constexpr (NW == 8) b = bytes[w / 4];
    else if constexpr (blocks_of<NW>() > 1) {
        const int i = (grp * NW + w) / 4 - grp * NW / 4;
        if (i == 1) b = bytes[1];
        if constexpr (blocks_of<NW>() > 2)
            if (i == 2) b = bytes[2];
    }
    return scale_of(b);
}

// Four features of a row from their sums o, the row's reference m and its sum of weights; the row's logarithm with the first of them.
template <int DT> __device__ __forceinline__ void store_row(const CacheAsk &a, const CacheShape &c, int kvh, int row, int f, const f32x4 &o, float m, float sum)
{
    const RowOf at = row_of(c, kvh, row);
    if (f == 0 && a.lse) as_global(a.lse)[(size_t)at.i * c.n_heads + at.head] = sum == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * LN2;
    if (f >= c.d_head) return;
    const f32x4 v = sum == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o * (1.f / sum);
    char *out = as_global(a.out) + (size_t)at.i * a.out_stride + ((size_t)at.head * c.d_head + f) * (DT == 0 ? 4 : 2);
    if constexpr (DT == 0) *(f32x4 *)out = v;
    else *(bf16x4 *)out = __builtin_convertvector(v, bf16x4);
}

template <int DT, int NW, int NT, int WAVES> __global__ __launch_bounds__(64 * WAVES) void k_cache_few(CacheFew few /* first: kernel_arg */, const char *dev, CacheGrid g, CacheShape c, float *part)
{
    constexpr int DP = 32 * NW, NP = DT == 0 ? 3 : 1, ROWS = 16 * NT, FT = DP / 16;
    constexpr int WAVE_BYTES = 64 * DP + 256;       // 32 rows of values; in the end 16 rows of sums, four apart
    static_assert(WAVE_BYTES == 16 * (DP + 4) * 4);
    __shared__ __align__(16) char lds[WAVES * WAVE_BYTES];
    __shared__ float ml[2][WAVES][ROWS], total[2][ROWS];
    (void)few;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4, kvh = blockIdx.y;
    const AskUnit found = block_ask(dev, g, lane);
    const CacheAsk &a = found.a;
    const int unit = found.unit, n_rows = a.n_q * c.group;
    int tile_of_rows = unit, split = 0;
    if (a.splits > 1) tile_of_rows = unit / a.splits, split = unit % a.splits;
    const int row0 = tile_of_rows * ROWS;

    RowOf rows[NT];
    Sight see[NT];
    Reach reach;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int row = row0 + 16 * i + col;
        rows[i] = row_of(c, kvh, row < n_rows ? row : 0);
        see[i] = sight_of(a, rows[i].i, row < n_rows);
        reach.add(see[i], row < n_rows);
    }
    const Walk walk = reach.walk<16>(a);
    int t = wave, t_end = walk.count();
    if (a.splits > 1) {
        const int64_t n = t_end;
        t += (int)(n * split / a.splits);
        t_end = (int)(n * (split + 1) / a.splits);
    }

    const char *pool = as_global(c.pool) + (size_t)kvh * cache_head_bytes(c);
    f32x4 acc[NT][FT];
    float m[NT], l[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        m[t] = -INFINITY, l[t] = 0.f;
#pragma unroll
        for (int f = 0; f < FT; ++f) acc[t][f] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const float k2 = c.scale * LOG2E;
    char *mine = lds + wave * WAVE_BYTES;
    typedef s16x4 __attribute__((address_space(3))) *lds4_t;

    TileList<DP> list;
    list.fill(c, a, walk, t, WAVES, t_end, lane);
    auto ask = [&](int t, RawTile<NW> &to) {            // a tile that is dropped or behind the end reads page 0
        if (t - list.from >= 64 * WAVES) list.fill(c, a, walk, t, WAVES, t_end, lane);
        const int64_t off = list.offset((t - list.from) / WAVES);
        to.here = off >= 0;
        load_tile<NW>(pool + (off < 0 ? 0 : off), lane, to);
    };
    bf16x8 q[NT][NP][NW];
    auto work = [&](int t, RawTile<NW> &now) {
        now.pin();
        const bool here = now.here;
        const int tile = walk.tile(t), j0 = here ? tile * CACHE_TILE + 4 * grp : NO_KEY;        // (dropped or behind the end: nobody sees it)

        // values: as bf16 rows of the wave's LDS.  A block that is not finite -- NaN, or bytes that nobody wrote -- becomes zeros:
        // who sees it gets NaN below.
        uint32_t odd = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float sc = word_scale<NW>(now.vs[h], grp, w);
                const bool fine = sc < 0x1p126f;
                odd |= fine || !here || tile * CACHE_TILE + 16 * h + col > reach.hi_last ? 0u : 1u;
                *(bf16x8 *)(mine + v_place<DP>(16 * h + col, grp * NW + w)) = decode8(fine ? now.v[h][w] : 0u, fine ? sc : 1.f);
            }
        }

        // scores
        f32x4 s[NT][2];
#pragma unroll
        for (int i = 0; i < NT; ++i) s[i][0] = s[i][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const bf16x8 k = decode8(now.k[h][w], word_scale<NW>(now.ks[h], grp, w));
#pragma unroll
                for (int i = 0; i < NT; ++i)
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p) s[i][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[i][p][w], s[i][h], 0, 0, 0);
            }

        const bool whole = here && walk.whole(tile);
        bf16x8 weights[NT][NP];
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            float x[8], top = -INFINITY;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = s[i][e / 4][e % 4] * k2;
            if (!whole) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = see[i].sees(j0 + 16 * (e / 4) + e % 4) ? x[e] : -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, x[e]);
            if (__ballot(top > m[i] + LAZY)) {
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float m2 = fmaxf(m[i], top), back = m2 == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[i] - m2);
                m[i] = m2;
                l[i] *= back;
#pragma unroll
                for (int f = 0; f < FT; ++f) acc[i][f] *= back;
            }
            const float ref = m[i] == -INFINITY ? 0.f : m[i];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = __builtin_amdgcn_exp2f(x[e] - ref);
                l[i] += x[e];
            }
            pieces8<NP>(x, weights[i]);
        }

#pragma unroll
        for (int f = 0; f < FT; ++f) {
            union {
                s16x4 h[2];
                bf16x8 all;
            } v;
            v.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_t)(mine + v_turned<DP>(4 * grp, 16 * f, lane)));
            v.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_t)(mine + v_turned<DP>(16 + 4 * grp, 16 * f, lane)));
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int p = NP - 1; p >= 0; --p) acc[i][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.all, weights[i][p], acc[i][f], 0, 0, 0);
        }

        if (__ballot(odd)) {
            // a row that sees a block of values that is not finite: its 32 features are NaN
#pragma unroll 1
            for (int key = 0; key < CACHE_TILE; ++key) {
                const int from = key & 15;
#pragma unroll
                for (int f = 0; f < FT; ++f) {              // 16 features of block f / 2, whose first word group f / 2 * 4 / NW holds
                    const int gr = f / 2 * 4 / NW, b = f / 2 - gr * NW / 4;
                    const uint32_t byte = __shfl(key < 16 ? now.vs[0][b] : now.vs[1][b], from + 16 * gr);
                    if (scale_of(byte) < 0x1p126f) continue;
#pragma unroll
                    for (int i = 0; i < NT; ++i)
                        if (see[i].sees(tile * CACHE_TILE + key)) acc[i][f] += __builtin_nanf("");
                }
            }
        }
    };
    // Two sets of registers by turns: what one is loaded with is not waited for while the other is worked on.  (Four of them: no faster where there
    // are many tiles, and slower where each wave has few.)
    constexpr int DEPTH = 2;
    RawTile<NW> raw[DEPTH];
#pragma unroll
    for (int i = 0; i < DEPTH - 1; ++i) {
        ask(t + WAVES * i, raw[i]);
        __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {              // (the queries come while the first tiles do)
        const char *qr = a.q + (size_t)rows[i].i * a.q_stride + (size_t)rows[i].head * c.d_head * (DT == 0 ? 4 : 2);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            bf16x8 p[NP];
            query8<DT, NP>(qr, grp * (DP / 4) + 8 * w, c.d_head, row0 + 16 * i + col < n_rows, p);
#pragma unroll
            for (int j = 0; j < NP; ++j) q[i][j][w] = p[j];
        }
    }
    for (; t < t_end; t += WAVES * DEPTH)
#pragma unroll
        for (int i = 0; i < DEPTH; ++i) {
            ask(t + WAVES * (i + DEPTH - 1), raw[(i + DEPTH - 1) % DEPTH]);
            __builtin_amdgcn_sched_barrier(0);
            work(t + WAVES * i, raw[i]);
        }

    // the waves' parts become one: a common reference, then sums through LDS
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        l[i] += __shfl_xor(l[i], 16);
        l[i] += __shfl_xor(l[i], 32);
        if (grp == 0) ml[0][wave][16 * i + col] = m[i], ml[1][wave][16 * i + col] = l[i];
    }
    __syncthreads();
    const int rows_here = min(ROWS, n_rows - row0);
    const size_t each = cache_part_floats(ROWS, DP);
    const size_t first_part = (size_t)a.part + (size_t)(kvh * ((n_rows + ROWS - 1) / ROWS) + tile_of_rows) * a.splits;     // (splits > 1)
    float *pt = as_global(part) + (first_part + split) * each;
    if (threadIdx.x < ROWS) {
        float mt = -INFINITY, sum = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) mt = fmaxf(mt, ml[0][w][threadIdx.x]);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float mw = ml[0][w][threadIdx.x];
            sum += mw == -INFINITY ? ml[1][w][threadIdx.x] : ml[1][w][threadIdx.x] * __builtin_amdgcn_exp2f(mw - mt);    // (no maximum: 0, or NaN)
        }
        total[0][threadIdx.x] = mt, total[1][threadIdx.x] = sum;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        if (16 * i >= rows_here) break;
        const float top = total[0][16 * i + col];
        const float back = m[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[i] - top);
        f32x4 *sums = (f32x4 *)mine;            // [16 rows][DP + 4]
        if (i) __syncthreads();
        if (16 * i + col < rows_here) {
#pragma unroll
            for (int f = 0; f < FT; ++f) sums[(col * (DP + 4) + 16 * f + 4 * grp) / 4] = acc[i][f] * back;
        }
        __syncthreads();
        for (int x = threadIdx.x; x < min(16, rows_here - 16 * i) * (DP / 4); x += 64 * WAVES) {
            const int cl = x / (DP / 4), f = x % (DP / 4) * 4, row = row0 + 16 * i + cl;
            f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) o += ((const f32x4 *)(lds + w * WAVE_BYTES))[(cl * (DP + 4) + f) / 4];
            if (a.splits > 1) {
                *(f32x4 *)(pt + (16 * i + cl) * DP + f) = o;
                if (f == 0) pt[ROWS * DP + 16 * i + cl] = total[0][16 * i + cl], pt[ROWS * DP + ROWS + 16 * i + cl] = total[1][16 * i + cl];
            } else
                store_row<DT>(a, c, kvh, row, f, o, total[0][16 * i + cl], total[1][16 * i + cl]);
        }
    }
}

// Rows whose keys several blocks shared: their parts, in the order of the keys.  A block to a row and kv head.
template <int DT> __global__ __launch_bounds__(128) void k_cache_join(CacheFew few /* first: kernel_arg */, const char *dev, CacheGrid g, CacheShape c, const float *part, int rows_of_tile)
{
    (void)few;
    const int lane = threadIdx.x & 63, kvh = blockIdx.y;
    const int r = entry_of(dev, g.n, g.firsts, blockIdx.x, lane);
    const CacheAsk a = ask_at(dev, g, r);
    const int row = (int)blockIdx.x - first_at(dev, g.firsts, r), n_rows = a.n_q * c.group, tiles = (n_rows + rows_of_tile - 1) / rows_of_tile;
    const size_t each = cache_part_floats(rows_of_tile, c.dp);
    const float *p = as_global(part) + ((size_t)a.part + ((size_t)kvh * tiles + row / rows_of_tile) * a.splits) * each;
    const int cl = row % rows_of_tile;
    const float *ms = p + (size_t)rows_of_tile * c.dp + cl, *ls = ms + rows_of_tile;
    // a lane to a split for what its part counts; MAX_SPLITS is 128
    __shared__ float back[128];
    float mw[2], lw[2], mt = -INFINITY;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int s = lane + 64 * h;
        mw[h] = s < a.splits ? ms[s * each] : -INFINITY;
        lw[h] = s < a.splits ? ls[s * each] : 0.f;
        mt = fmaxf(mt, mw[h]);
    }
    for (int x = 1; x < 64; x *= 2) mt = fmaxf(mt, __shfl_xor(mt, x));
    float sum = 0.f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float w = mw[h] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mw[h] - mt);      // without a maximum: zeros, or NaN
        if (threadIdx.x < 64) back[lane + 64 * h] = w;
        sum += lw[h] * w;
    }
    for (int x = 1; x < 64; x *= 2) sum += __shfl_xor(sum, x);
    __syncthreads();
    const RowOf at = row_of(c, kvh, row);
    float o[2] = {0.f, 0.f};
    for (int s = 0; s < a.splits; s += 8)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int f = threadIdx.x + 128 * h;
            if (f >= c.dp) break;
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = p[(size_t)min(s + i, a.splits - 1) * each + (size_t)cl * c.dp + f];
#pragma unroll
            for (int i = 0; i < 8; ++i) o[h] += s + i < a.splits ? x[i] * back[s + i] : 0.f;
        }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int f = threadIdx.x + 128 * h;
        if (f >= c.d_head) continue;
        const float v = sum == 0.f ? 0.f : o[h] / sum;
        char *out = a.out + (size_t)at.i * a.out_stride + ((size_t)at.head * c.d_head + f) * (DT == 0 ? 4 : 2);
        if (DT == 0) *(float *)out = v;
        else *(uint16_t *)out = f2bf(v);
    }
    if (threadIdx.x == 0 && a.lse) a.lse[(size_t)at.i * c.n_heads + at.head] = sum == 0.f ? -INFINITY : (mt + __builtin_amdgcn_logf(sum)) * LN2;
}

}  // namespace

namespace {
template <int DT, int NW, int NT> void few(const CacheFew &args, const char *dev, const CacheGrid &g, const CacheShape &c, const CachePart &p, hipStream_t s)
{
    if constexpr (NW <= 4) {
        if (p.eight) {
            hipLaunchKernelGGL((k_cache_few<DT, NW, NT, 8>), cache_grid(g, c, p), dim3(512), 0, s, args, dev, g, c, p.part);
            return;
        }
    }
    hipLaunchKernelGGL((k_cache_few<DT, NW, NT, 4>), cache_grid(g, c, p), dim3(256), 0, s, args, dev, g, c, p.part);
}
template <int NW> void few_of(const CacheFew &args, const char *dev, const CacheGrid &g, const CacheShape &c, const CachePart &p, hipStream_t s)
{
    if (c.dtype == 0) few<0, NW, 1>(args, dev, g, c, p, s);
    else if (p.rows_of_tile == 16) few<1, NW, 1>(args, dev, g, c, p, s);
    else few<1, NW, 2>(args, dev, g, c, p, s);
}
}  // namespace

static void launch_cache_few(const CacheFew &args, const char *dev, const CacheGrid &g, const CacheShape &c, const CachePart &p, hipStream_t s)
{
    switch (c.dp / 32) {
    case 1: few_of<1>(args, dev, g, c, p, s); break;
    case 2: few_of<2>(args, dev, g, c, p, s); break;
    case 3: few_of<3>(args, dev, g, c, p, s); break;
    case 4: few_of<4>(args, dev, g, c, p, s); break;
    case 5: few_of<5>(args, dev, g, c, p, s); break;
    case 6: few_of<6>(args, dev, g, c, p, s); break;
    case 7: few_of<7>(args, dev, g, c, p, s); break;
    default: few_of<8>(args, dev, g, c, p, s); break;
    }
}

hipError_t launch_cache_attend(const CacheShape &c, const CacheList &asks, const CachePlan &p, hipStream_t s)
{
    CacheFew args;
    if (!asks.dev) __builtin_memcpy(args.w, asks.host, asks.bytes);
    CacheGrid g{asks.n, (int32_t)cache_asks_bytes(asks.n, asks.lean), 0, asks.lean};
    for (int kind = 0; kind < 2; ++kind) {
        const CachePart &of = kind ? p.many : p.few;
        if (of.units == 0) continue;
        g.each = of.each;
        hipError_t e = hipSuccess;
        if (kind && of.own) launch_cache_own(args, asks.dev, g, c, of, s);
        else if (kind) e = launch_cache_many(args, asks.dev, g, c, of, s);
        else launch_cache_few(args, asks.dev, g, c, of, s);
        if (e == hipSuccess) e = hipGetLastError();
        if (e != hipSuccess) return e;
        g.firsts += 4 * (asks.n + 1);
        if (of.joins) {
            if (c.dtype == 0) hipLaunchKernelGGL(k_cache_join<0>, dim3(of.joins, c.n_kv), dim3(128), 0, s, args, asks.dev, g, c, of.part, of.rows_of_tile);
            else hipLaunchKernelGGL(k_cache_join<1>, dim3(of.joins, c.n_kv), dim3(128), 0, s, args, asks.dev, g, c, of.part, of.rows_of_tile);
            if (hipError_t j = hipGetLastError(); j != hipSuccess) return j;
        }
        g.firsts += 4 * (asks.n + 1);
    }
    return hipSuccess;
}

}  // namespace aif
