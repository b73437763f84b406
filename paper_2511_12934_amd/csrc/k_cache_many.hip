// The user cache's attention for many rows (candidates): a block takes 32 CT rows a wave, 4 or 8 waves, and 64 keys a stage.
//
// With hundreds of rows to a key the codes are the smaller part: a stage's keys and values are brought to bf16 once for the block, 32 features
// and their scale a thread, and lie in LDS as rows; the next stage's codes travel meanwhile, and one barrier a stage parts the two
// buffers.  Products are 32x32x16: S^T = K Q^T with a wave's queries in registers throughout, so that a lane holds 16 keys
// of one row, and these, as weights, are the operand of O^T = V^T P^T as they stand; V comes turned (ds_read_b64_tr_b16).  What bounds it is
// the vector ALU: per score one fused multiply-add, half a maximum, one exponential (2.3 times a plain instruction), half a conversion and one
// addition.  Heads of 64: eight waves of 32 rows, four waves a SIMD (64 x 10^4 rows over 500 keys 121 us, 0.68
// PFLOP/s; four waves of 64 rows that each bring the keys over for themselves, k_cache_own.hip, 130).
// Rows of K are 16 bytes longer than their features, so that the lanes of a read meet in no bank; those of V do where heads are a multiple of 64 (v_place).
#include "k_cache_attend.h"

namespace aif {

namespace {


constexpr int k_stride(int dp) { return 2 * dp + 16; }
constexpr int stage_bytes(int dp) { return 2 * CACHE_TILE * (k_stride(dp) + 2 * dp); }

template <int DT, int NW, int CT, int WAVES, int KS> __global__ __launch_bounds__(64 * WAVES, WAVES == 8 ? 4 : 1) void k_cache_many(CacheFew few /* first: kernel_arg */, const char *dev, CacheGrid g, CacheShape c, float *part)
{
    constexpr int DP = 32 * NW, NP = DT == 0 ? 3 : 1, ROWS = 32 * WAVES * CT, THREADS = 64 * WAVES, KST = k_stride(DP);
    constexpr int ITEMS = (128 * NW + THREADS - 1) / THREADS;       // pieces of 32 features a thread brings to LDS per stage
    __shared__ __align__(16) char lds[2][stage_bytes(DP)];
    __shared__ int odd_now[3];                          // whether a stage has blocks of values that are not finite
    (void)few;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5, kvh = blockIdx.y;
    const AskUnit found = block_ask(dev, g, lane);
    const CacheAsk &a = found.a;
    const int unit = found.unit, n_rows = a.n_q * c.group;
    int row_tile = unit, split = 0;
    if (a.splits > 1) row_tile = unit / a.splits, split = unit % a.splits;
    const char *pool = as_global(c.pool) + (size_t)kvh * cache_head_bytes(c);
    const float k2 = c.scale * LOG2E;
    typedef s16x4 __attribute__((address_space(3))) *lds4_t;
    const int row0 = row_tile * ROWS;

    Reach reach;
    if (a.pos) {
        for (int i = lane; i < ROWS; i += 64)
            if (row0 + i < n_rows) reach.add(sight_of(a, row_of(c, 0, row0 + i).i, true), true);
    } else
        reach.add(sight_of(a, 0, true), true);
    const Walk walk = reach.walk<64>(a);
    const int hi_last = reach.hi_last;
    int t_begin = 0, t_end = walk.count();
    if (a.splits > 1) {
        const int64_t n = t_end;
        t_begin = (int)(n * split / a.splits);
        t_end = (int)(n * (split + 1) / a.splits);
    }
    TileList<DP> list;
    list.fill(c, a, walk, t_begin, 1, t_end, lane);
    // tile t of the walk (t - list.from in 0..63); dead: behind the end, or in a page that was dropped.  A dead tile reads
    // page 0, which nobody sees.
    auto locate = [&](int t, bool &dead) {
        const int64_t off = list.offset(t - list.from);
        dead = off < 0;
        return pool + (dead ? 0 : off);
    };

    // A thread's pieces of a stage of two tiles: piece id of (tile, keys or values, 32 rows, NW blocks), 16 bytes of codes and a byte.
    // Which tile is the same for a wave's lanes, and so is, NW even, which of keys and values.
    uint4 raw[ITEMS];
    uint32_t byte[ITEMS];
    auto fetch = [&](const char *t0, const char *t1) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int id64 = (wave + WAVES * i) * 64, id = id64 + lane, b = id % (32 * NW), kv = id / (32 * NW) % 2;
            if (id64 >= 128 * NW) break;
            const char *tile = as_global(id64 < 64 * NW ? t0 : t1);
            raw[i] = *(const uint4 *)(tile + (uint32_t)(kv * 16 * DP + b * 16));
            byte[i] = *(const uint8_t *)(tile + (uint32_t)((32 + kv) * DP + b));
        }
    };
    auto place = [&](int buf, int flag, int j0, int j1) {       // j0, j1: the tiles' first keys, beyond every row's where one is dead
        bool odd = false;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int id64 = (wave + WAVES * i) * 64, id = id64 + lane, b = id % (32 * NW), tile = id64 / (64 * NW);
            if (id64 >= 128 * NW) break;
            const bool vals = NW % 2 == 0 ? id64 / (32 * NW) % 2 : id / (32 * NW) % 2;
            const int row = b / NW, blk = b % NW;
            asm volatile("" : "+v"(byte[i]));              // (what is made of a byte is made here, not where it is asked for: that would wait for it)
            float sc = scale_of(byte[i]);
            if (vals) {                                     // a block of values that is not finite becomes zeros, and is noted
                const bool fine = sc < 0x1p126f;
                odd |= !fine && (tile ? j1 : j0) + row <= hi_last;
                sc = fine ? sc : 1.f;
                raw[i].x = fine ? raw[i].x : 0u, raw[i].y = fine ? raw[i].y : 0u, raw[i].z = fine ? raw[i].z : 0u, raw[i].w = fine ? raw[i].w : 0u;
            }
            char *keys = lds[buf] + (tile * CACHE_TILE + row) * KST + blk * 64, *turn = lds[buf] + 2 * CACHE_TILE * (KST + tile * DP);
            const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
            for (int x = 0; x < 4; ++x) *(bf16x8 *)(vals ? turn + v_place<DP>(row, 4 * blk + x) : keys + 16 * x) = decode8(w[x], sc);
        }
        if (odd) odd_now[flag] = 1;
    };

    // this wave's rows
    const int w_row0 = row0 + 32 * CT * wave;
    const bool busy = w_row0 < n_rows;
    Sight see[CT];
    bf16x8 q[CT][NP][KS];
#pragma unroll
    for (int t = 0; t < CT; ++t) {
        const int row = w_row0 + 32 * t + col;
        const bool is_row = row < n_rows;
        const RowOf o = row_of(c, kvh, is_row ? row : 0);
        see[t] = sight_of(a, o.i, is_row);
        const char *qr = a.q + (size_t)o.i * a.q_stride + (size_t)o.head * c.d_head * (DT == 0 ? 4 : 2);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            bf16x8 p[NP];
            query8<DT, NP>(qr, 16 * k + 8 * half, c.d_head, is_row, p);
#pragma unroll
            for (int i = 0; i < NP; ++i) q[t][i][k] = p[i];
        }
    }
    f32x16 acc[CT][NW];
    float m[CT], l[CT];
#pragma unroll
    for (int t = 0; t < CT; ++t) {
        m[t] = -INFINITY, l[t] = 0.f;
#pragma unroll
        for (int f = 0; f < NW; ++f)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[t][f][e] = 0.f;
    }
    if (threadIdx.x < 3) odd_now[threadIdx.x] = 0;
    if (t_begin < t_end) {
    bool dead0, dead1;
    const char *t0 = locate(t_begin, dead0), *t1 = locate(t_begin + 1, dead1);
    auto first_key = [&](int t, bool dead) { return dead ? INT32_MAX - CACHE_TILE : walk.tile(t) * CACHE_TILE; };
    fetch(t0, t1);
    __syncthreads();                                    // (odd_now)
    place(0, 0, first_key(t_begin, dead0), first_key(t_begin + 1, dead1));
    __syncthreads();
    int stage = 0, flag = 0;
    for (int t = t_begin; t < t_end; t += 2) {
        if (t + 2 - list.from >= 64) list.fill(c, a, walk, t + 2, 1, t_end, lane);
        bool next_dead0, next_dead1;
        const char *n0 = locate(t + 2, next_dead0), *n1 = locate(t + 3, next_dead1);
        fetch(n0, n1);
        const char *kb = lds[stage], *vb = kb + 2 * CACHE_TILE * KST;
        const int odd = odd_now[flag];
        if (busy) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (h ? dead1 : dead0) continue;
                const int tile = walk.tile(t + h), j0 = tile * CACHE_TILE + 4 * half;
                f32x16 s[CT];
#pragma unroll
                for (int i = 0; i < CT; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[i][e] = 0.f;
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    const bf16x8 kf = *(const bf16x8 *)(kb + (h * CACHE_TILE + col) * KST + 32 * k + 16 * half);
#pragma unroll
                    for (int i = 0; i < CT; ++i)
#pragma unroll
                        for (int p = NP - 1; p >= 0; --p) s[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[i][p][k], s[i], 0, 0, 0);
                }
                const bool whole = walk.whole(tile);
                bf16x8 weights[CT][2][NP];
#pragma unroll
                for (int i = 0; i < CT; ++i) {
                    if (!whole) see[i].hide(s[i], j0);
                    float top = -INFINITY;
#pragma unroll
                    for (int e = 0; e < 16; ++e) top = fmaxf(top, s[i][e]);
                    top *= k2;
                    if (__ballot(top > m[i] + LAZY)) {
                        top = fmaxf(top, __shfl_xor(top, 32));
                        const float m2 = fmaxf(m[i], top), back = m2 == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[i] - m2);
                        m[i] = m2;
                        l[i] *= back;
#pragma unroll
                        for (int f = 0; f < NW; ++f) acc[i][f] *= back;
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
                        // four keys of 16 features a group of 16 lanes: keys 16 k + 4 half (+ 8), features 32 f + 16 (lane / 16 % 2)
                        const char *turn = vb + h * CACHE_TILE * 2 * DP;
                        const int key = 16 * k + 4 * half, feature = 32 * f + 16 * (lane >> 4 & 1);
                        union {
                            s16x4 h[2];
                            bf16x8 all;
                        } v;
                        v.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_t)(turn + v_turned<DP>(key, feature, lane)));
                        v.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4_t)(turn + v_turned<DP>(key + 8, feature, lane)));
#pragma unroll
                        for (int i = 0; i < CT; ++i)
#pragma unroll
                            for (int p = NP - 1; p >= 0; --p) acc[i][f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v.all, weights[i][k][p], acc[i][f], 0, 0, 0);
                    }
                if (odd) {
                    // a row that sees a block of values that is not finite: its features are NaN
#pragma unroll 1
                    for (int key = 0; key < CACHE_TILE; ++key)
#pragma unroll
                        for (int f = 0; f < NW; ++f) {
                            if (scale_of(*(const uint8_t *)((h ? t1 : t0) + 33 * DP + key * NW + f)) < 0x1p126f) continue;
#pragma unroll
                            for (int i = 0; i < CT; ++i)
                                if (see[i].sees(tile * CACHE_TILE + key)) acc[i][f] += __builtin_nanf("");
                        }
                }
            }
        }
        const int next = flag == 2 ? 0 : flag + 1;
        place(stage ^ 1, next, first_key(t + 2, next_dead0), first_key(t + 3, next_dead1));
        if (threadIdx.x == 0) odd_now[next == 2 ? 0 : next + 1] = 0;
        t0 = n0, t1 = n1;
        dead0 = next_dead0, dead1 = next_dead1;
        stage ^= 1, flag = next;
        __syncthreads();
    }
    }
    if (busy) finish_rows<DT, NW, CT, ROWS>(a, c, part, kvh, unit, n_rows, row0, 32 * CT * wave, col, half, acc, m, l);
}

template <int DT, int NW, int CT, int WAVES> void many(const CacheFew &args, const char *dev, const CacheGrid &g, const CacheShape &c, const CachePart &p, hipStream_t s)
{
    const dim3 grid = cache_grid(g, c, p), block(64 * WAVES);
    hipLaunchKernelGGL((k_cache_many<DT, NW, CT, WAVES, 2 * NW>), grid, block, 0, s, args, dev, g, c, p.part);
}
template <int NW> void many_of(const CacheFew &args, const char *dev, const CacheGrid &g, const CacheShape &c, const CachePart &p, hipStream_t s)
{
    if constexpr (NW == 2) many<1, NW, 1, 8>(args, dev, g, c, p, s);
    else if (c.dtype == 0) many<0, NW, 1, 4>(args, dev, g, c, p, s);
    else if (NW <= 4 && p.rows_of_tile == 256) many<1, NW, NW <= 4 ? 2 : 1, 4>(args, dev, g, c, p, s);
    else many<1, NW, 1, 4>(args, dev, g, c, p, s);
}

}  // namespace

hipError_t launch_cache_many(const CacheFew &args, const char *dev, const CacheGrid &g, const CacheShape &c, const CachePart &p, hipStream_t s)
{
    switch (c.dp / 32) {
    case 2: many_of<2>(args, dev, g, c, p, s); break;
    case 3: many_of<3>(args, dev, g, c, p, s); break;
    case 4: many_of<4>(args, dev, g, c, p, s); break;
    case 5: many_of<5>(args, dev, g, c, p, s); break;
    case 6: many_of<6>(args, dev, g, c, p, s); break;
    case 7: many_of<7>(args, dev, g, c, p, s); break;
    case 8: many_of<8>(args, dev, g, c, p, s); break;
    default: return hipErrorInvalidValue;       // (heads of up to 32 are k_cache_own's)
    }
    return hipGetLastError();
}

}  // namespace aif
