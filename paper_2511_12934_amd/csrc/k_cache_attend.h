// What the user cache's attention kernels share: entries and blocks, who sees what, the tiles of 32 keys that a block walks, and
// four-bit codes on their way to the matrix cores.
#pragma once
#include "aif_cache_dev.h"

namespace aif {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr float LAZY = 8.f;             // how far, in powers of two, a score may pass the reference of its row's weights
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

// The blocks of a launch: running numbers of units behind the asks.  A unit is (row tile, split), tiles first.
struct CacheGrid {
    int32_t n, firsts;          // asks; byte offset of int32 first[n + 1]
    int32_t each;               // CachePart::each
    int32_t lean;               // CacheList::lean
};

inline dim3 cache_grid(const CacheGrid &g, const CacheShape &c, const CachePart &p) { return p.each ? dim3(g.n, c.n_kv, p.each) : dim3(p.units, c.n_kv, 1); }

void launch_cache_own(const CacheFew &args, const char *dev, const CacheGrid &g, const CacheShape &c, const CachePart &p, hipStream_t s);
hipError_t launch_cache_many(const CacheFew &args, const char *dev, const CacheGrid &g, const CacheShape &c, const CachePart &p, hipStream_t s);

__device__ __forceinline__ CacheAsk ask_at(const char *dev, const CacheGrid &g, int r)
{
    if (g.lean) {               // (in the arguments)
        const CacheLean l = arg_copy(kernel_arg<CacheLean>(0));
        const CacheOwn o = arg_copy(kernel_arg<CacheOwn>(sizeof(CacheLean) + (size_t)r * sizeof(CacheOwn)));
        CacheAsk a = l.a;
        a.q += r * l.q_step;
        a.out += r * l.out_step;
        a.lse = (float *)((char *)a.lse + r * l.lse_step);
        a.pos = (const int32_t *)((const char *)a.pos + r * l.pos_step);
        a.len = o.len, a.entry = o.entry, a.splits = o.splits, a.part = o.part;
        return a;
    }
    return desc_at<CacheAsk>(dev, r);
}
// The block's ask and its unit of it.
struct AskUnit {
    CacheAsk a;
    int unit;
};
__device__ __forceinline__ AskUnit block_ask(const char *dev, const CacheGrid &g, int lane)
{
    AskUnit u;
    if (g.each) {
        u.a = ask_at(dev, g, blockIdx.x);
        u.unit = blockIdx.z;
        return u;
    }
    const int r = entry_of(dev, g.n, g.firsts, blockIdx.x, lane);
    u.a = ask_at(dev, g, r);
    u.unit = (int)blockIdx.x - first_at(dev, g.firsts, r);
    return u;
}

// What a row (query i and a head) sees: keys j <= last, and of those beyond `from` or before `sinks` only.
struct Sight {
    int last, from, sinks;
    __device__ __forceinline__ bool sees(int j) const { return (j <= last) & ((j >= from) | (j < sinks)); }
    // scores of the keys j0 + 8 (e / 4) + e % 4: minus infinity where not seen (j0 = NO_KEY: everywhere)
    __device__ __forceinline__ void hide(f32x16 &s, int j0) const
    {
        const uint32_t at = (uint32_t)j0 - (uint32_t)from, span = last >= from ? last - from + 1 : 0;      // last - from < window
        const int head = min(sinks, last + 1);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int o = 8 * (e / 4) + e % 4;
            s[e] = ((at + o < span) | (j0 + o < head)) ? s[e] : -INFINITY;
        }
    }
};
constexpr int NO_KEY = INT32_MAX - 2 * CACHE_TILE;
__device__ __forceinline__ Sight sight_of(const CacheAsk &a, int i, bool is_row)
{
    int p = a.len - 1;
    if (a.pos && is_row) p = as_global(a.pos)[i];
    p = is_row && p > -1 ? p : -1;
    Sight s;
    s.last = p < a.len - 1 ? p : a.len - 1;
    s.from = a.window ? p - a.window + 1 : 0;       // p >= -1, window > 0: no overflow
    s.sinks = a.window ? a.sinks : 0;
    return s;
}

// The tiles of 32 keys that some row of a block sees: [0, head) and [body, end).  all_from, all_to: keys that every row of it sees.
struct Walk {
    int head, body, end;
    int all_last, all_from, sinks;
    __device__ __forceinline__ int count() const { return head + (end > body ? end - body : 0); }
    __device__ __forceinline__ int tile(int t) const { return t < head ? t : t - head + body; }
    __device__ __forceinline__ bool whole(int tile) const
    {
        const int j = tile * CACHE_TILE;
        return j + CACHE_TILE - 1 <= all_last && (j >= all_from || j + CACHE_TILE <= sinks);
    }
};
// What the rows of a wave or block see together.
struct Reach {
    int lo_last = INT32_MAX, hi_last = -1, lo_from = INT32_MAX, hi_from = INT32_MIN;
    __device__ __forceinline__ void add(const Sight &s, bool is_row)
    {
        if (!is_row) return;
        lo_last = min(lo_last, s.last);
        hi_last = max(hi_last, s.last);
        hi_from = max(hi_from, s.from);
        if (s.last >= 0) lo_from = min(lo_from, s.from);    // (one that sees nothing widens nothing)
    }
    // the tiles, of the rows that LANES neighbouring lanes have added (the same in every such group); all lanes alike
    template <int LANES> __device__ __forceinline__ Walk walk(const CacheAsk &a)
    {
        if (a.pos) {                                        // else every row sees the same
#pragma unroll
            for (int x = 1; x < LANES; x *= 2) {
                lo_last = min(lo_last, __shfl_xor(lo_last, x));
                hi_last = max(hi_last, __shfl_xor(hi_last, x));
                lo_from = min(lo_from, __shfl_xor(lo_from, x));
                hi_from = max(hi_from, __shfl_xor(hi_from, x));
            }
        }
        // (lane 0 has a row wherever a lane has one)
        lo_last = __builtin_amdgcn_readfirstlane(lo_last);
        hi_last = __builtin_amdgcn_readfirstlane(hi_last);
        lo_from = __builtin_amdgcn_readfirstlane(lo_from);
        hi_from = __builtin_amdgcn_readfirstlane(hi_from);
        Walk w;
        w.sinks = a.window ? a.sinks : 0;
        w.all_last = lo_last;
        w.all_from = hi_from;
        w.end = (hi_last + CACHE_TILE) / CACHE_TILE;        // hi_last = -1: none
        w.body = min((lo_from > 0 ? lo_from : 0) / CACHE_TILE, w.end);
        w.head = min((min(w.sinks, hi_last + 1) + CACHE_TILE - 1) / CACHE_TILE, w.body);
        return w;
    }
};

// Where the tiles of a walk lie: a wave keeps 64 of them, a lane each -- tile from + step * lane of the walk --, so that the page table
// is asked once for 64 tiles and a tile's address is two v_readlane.
template <int DP> struct TileList {
    uint32_t lo;
    int32_t hi;                 // offset into the pool; below 0: none, or its page was dropped
    int from;
    __device__ __forceinline__ void fill(const CacheShape &c, const CacheAsk &a, const Walk &w, int first, int step, int end, int lane)
    {
        from = first;
        const int t = first + step * lane;
        int64_t off = -1;
        if (t < end) {
            const uint32_t tile = w.tile(t), i = c.tpp_magic ? __umulhi(tile, c.tpp_magic) : tile;
            const int page = as_global(c.table)[a.entry + (int)i];
            if (page >= 0) off = (int64_t)page * c.page_bytes + (tile - i * (uint32_t)(c.page_len / CACHE_TILE)) * (uint32_t)cache_tile_bytes(DP);
        }
        lo = (uint32_t)off;
        hi = (int32_t)(off >> 32);
    }
    __device__ __forceinline__ int64_t offset(int i) const       // i in 0..63
    {
        return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane(hi, i) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)lo, i));
    }
};

// Eight codes as bf16, times 2^(byte - 127) (a byte of 255 gives NaN).
__device__ __forceinline__ bf16x8 decode8(uint32_t codes, float scale)
{
    union {
        bf16x2 h[4];
        bf16x8 all;
    } u;
    u.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
    u.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
    u.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
    u.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    return u.all;
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight fp32 numbers as NP bf16 pieces: rounded once (NP = 1), or cut after 8, 16 and 24 bits, whose sum is the number (NP = 3).
// With NP = 1 go the weights of bf16 calls, whose sum is of the unrounded ones: outputs, themselves rounded to bf16, are off by 2.2 to 2.35e-3 (2-norm, relative, against 64
// bits).  A second piece would make that 1.66e-3, which is the outputs' own rounding, and cost 3 to 10 % of the time in row tiles of 16, 8 to 20 % in those of
// 32 and 15 to 51 % in the larger ones (64 x 10^4 rows over 500 keys 117 us, 154; eight heads of 16 over 2,000 255 and 385).
template <int NP> __device__ __forceinline__ void pieces8(const float *x, bf16x8 *out)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if constexpr (NP == 1) {
            out[0][e] = (__bf16)x[e];
        } else {
            float r = x[e];
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                const uint32_t h = __float_as_uint(r) & 0xffff0000u;
                out[p][e] = __builtin_bit_cast(__bf16, (uint16_t)(h >> 16));
                r -= __uint_as_float(h);
            }
        }
    }
}

// Features [at, at + 8) of a query as NP pieces, zeros past its end; an infinity is its first piece alone.
template <int DT, int NP> __device__ __forceinline__ void query8(const char *q, int at, int d, bool live, bf16x8 *out)
{
    if constexpr (DT == 1) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (live && at < d) v = *(const uint4 *)(as_global(q) + 2 * at);
        out[0] = __builtin_bit_cast(bf16x8, v);
    } else {
        float x[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (live && at + 4 * h < d) v = *(const float4 *)(as_global(q) + 4 * (at + 4 * h));
            x[4 * h] = v.x, x[4 * h + 1] = v.y, x[4 * h + 2] = v.z, x[4 * h + 3] = v.w;
        }
        pieces8<NP>(x, out);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (__builtin_isinf(x[e])) out[1][e] = out[2][e] = (__bf16)0.f;
    }
}

// Which query and query head row `row` of a kv head is, and where its features lie.
struct RowOf {
    int i, head;
};
__device__ __forceinline__ RowOf row_of(const CacheShape &c, int kvh, int row)
{
    const int i = c.group_magic ? (int)__umulhi((uint32_t)row, c.group_magic) >> c.group_shift : row;
    return RowOf{i, kvh * c.group + row - i * c.group};
}

// Values in LDS: rows of 2 dp bytes in pieces of 16, piece `at` of row `key` in the place of piece at ^ f(key).  Pieces that are written together do not
// meet in a bank.  The turned reads, which could take 2 cycles a wave, take by the addresses 2 for odd dp / 32; in the row tiles of 16 and 32 2 for dp 64 and 192 and
// 4 for 128 and 256, whose piece 2 f of row r lies where piece 2 f + 1 of row r ^ 1 would; in the larger ones, which ask for four pieces of four rows, 4 and 8.
// The counters say the same: 2 cycles more for each read at dp 128 in the small tiles and at dp 64 in the large ones, a quarter of the LDS' active cycles.
template <int DP> __device__ __forceinline__ int v_place(int key, int at) { return key * (2 * DP) + (at ^ (DP % 64 ? key / 2 % 4 : key % 8)) * 16; }
// Where a lane's eight bytes of the turned read lie (four keys of one feature come back): keys key0 + lane % 16 / 4, 16 features from feature0 on
// (both multiples of 4 and 16).
template <int DP> __device__ __forceinline__ int v_turned(int key0, int feature0, int lane)
{
    return v_place<DP>(key0 + (lane & 15) / 4, feature0 / 8 + (lane & 3) / 2) + (lane & 1) * 8;
}

// The end of a wave's rows in_block + 32 i + col of a block's ROWS from `row0` on: quotients and logarithms, or a part for the join.  A lane holds
// the features 32 f + 8 (e / 4) + 4 half + e % 4 of its row, and its own share of the sum l.
template <int DT, int NW, int CT, int ROWS>
__device__ __forceinline__ void finish_rows(const CacheAsk &a, const CacheShape &c, float *part, int kvh, int unit, int n_rows, int row0, int in_block, int col, int half,
                                            f32x16 (&acc)[CT][NW], const float (&m)[CT], float (&l)[CT])
{
    constexpr int DP = 32 * NW;
#pragma unroll
    for (int i = 0; i < CT; ++i) {
        l[i] += __shfl_xor(l[i], 32);
        const int at = in_block + 32 * i + col, row = row0 + at;
        if (a.splits > 1) {
            float *pt = part + ((size_t)a.part + (size_t)kvh * ((n_rows + ROWS - 1) / ROWS) * a.splits + unit) * cache_part_floats(ROWS, DP);
#pragma unroll
            for (int f = 0; f < NW; ++f)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    *(float4 *)(pt + (size_t)at * DP + 32 * f + 8 * e + 4 * half) = make_float4(acc[i][f][4 * e], acc[i][f][4 * e + 1], acc[i][f][4 * e + 2], acc[i][f][4 * e + 3]);
            if (half == 0) pt[ROWS * DP + at] = m[i], pt[ROWS * DP + ROWS + at] = l[i];
            continue;
        }
        if (row >= n_rows) continue;
        if (l[i] == 0.f) {                      // no key, or scores of minus infinity alone
#pragma unroll
            for (int f = 0; f < NW; ++f)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][f][e] = 0.f;
        }
        const RowOf o = row_of(c, kvh, row);
        const float over = l[i] == 0.f ? 0.f : 1.f / l[i];
        char *out = as_global(a.out) + (size_t)o.i * a.out_stride + ((size_t)o.head * c.d_head + 4 * half) * (DT == 0 ? 4 : 2);
#pragma unroll
        for (int f = 0; f < NW; ++f)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int first = 32 * f + 8 * e;
                if (first >= c.d_head || (DT == 0 && first + 4 * half >= c.d_head)) continue;
                f32x4 x = f32x4{acc[i][f][4 * e], acc[i][f][4 * e + 1], acc[i][f][4 * e + 2], acc[i][f][4 * e + 3]} * over;
                if constexpr (DT == 0) *(f32x4 *)(out + 4 * first) = x;
                else *(bf16x4 *)(out + 2 * first) = __builtin_convertvector(x, bf16x4);
            }
        if (a.lse && half == 0) as_global(a.lse)[(size_t)o.i * c.n_heads + o.head] = l[i] == 0.f ? -INFINITY : (m[i] + __builtin_amdgcn_logf(l[i])) * LN2;
    }
}

}  // namespace aif
