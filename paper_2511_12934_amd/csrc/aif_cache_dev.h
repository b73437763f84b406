// Internal device-side types and launcher prototypes of the user cache of libaif (gfx950 only).
#pragma once
#include "aif_dev.h"

namespace aif {

// A page holds page_len rows of one sequence, head after head, a head's rows in tiles of 32:
//   keys' codes [32][dp / 2] | values' codes [32][dp / 2] | keys' scale bytes [32][dp / 32] | values' scale bytes [32][dp / 32]
// with dp = d_head rounded up to blocks of 32 features (zeros past d_head), two codes a byte, the even feature low.
// A tile is one address and 34 dp contiguous bytes: what a wave reads for 32 keys and values.
constexpr int CACHE_TILE = 32;
constexpr int CACHE_BLOCK = 32;
constexpr int CACHE_MAX_DP = 256;
constexpr int CACHE_E_MIN = -125, CACHE_E_MAX = 125;    // every value is a normal bf16: no flush, no overflow
constexpr int CACHE_NAN = 255;

struct CacheShape {
    char *pool;
    int32_t *table;             // [max_seqs, pages_per_seq]: pages of each sequence, -1 = dropped
    size_t page_bytes;
    int32_t n_heads, n_kv, group, d_head, dp, page_len, pages_per_seq, dtype;
    uint32_t group_magic;       // row / group for rows below 2^31: the high word of row * magic, shifted; 0: group is 1
    int32_t group_shift;
    uint32_t tpp_magic;         // ceil(2^32 / tiles of a page): the high word of its product with a tile (< 2^27) is the tile's page; 0: one tile a page
    float scale;
};
__host__ __device__ inline size_t cache_tile_bytes(int dp) { return (size_t)34 * dp; }
__host__ __device__ inline size_t cache_head_bytes(const CacheShape &c) { return (size_t)(c.page_len / CACHE_TILE) * 34 * c.dp; }

// n rows for the end of a sequence of `have` rows whose table entries start at `entry`, to the pages from `page` on, which follow each other; the first
// row goes into the first of them.  cow >= 0: that page is a new one in the place of page cow, whose rows before `have` it gets first.
struct CacheIn {
    const char *keys, *vals;
    uint32_t key_stride, val_stride;    // in 16 bytes
    int32_t entry, have, n;
    int32_t page, cow, pad_;
};
// Rows [first, first + n) of a sequence whose table entries start at `entry`, to keys and vals (or null; strides in elements).
struct CacheOut {
    char *keys, *vals;
    int64_t key_stride, val_stride;
    int32_t entry, first, n, pad_;
};
// Pages of a sequence copied to new ones that follow each other: those that table entries [src, src + n) name become the pages from `page` on, and
// entries [dst, dst + n) name them.  page < 0: the entries become -1.
struct CacheRun {
    int32_t src, dst, page, n;
};
// Table entries [dst, dst + n): those at src, or `value` where src < 0.
struct CacheFill {
    int32_t dst, n, src, value;
};
// Page src becomes page dst (src < 0: no page is copied); entry >= 0: that table entry becomes dst.
struct CacheMove {
    int32_t src, dst, entry;
};
// One entry of aif_cache_attend.
struct CacheAsk {
    const char *q;
    char *out;
    float *lse;
    const int32_t *pos;
    int64_t q_stride, out_stride;   // bytes
    int32_t n_q, len, sinks, window, entry;
    int32_t splits;             // blocks that share a row tile's keys
    int32_t part;               // splits > 1: the first of its partial results
    int32_t pad_;
};

// Entries that differ in their sequence and in what a step from one to the next makes of their pointers (a batch's queries and outputs lie in one
// tensor): entry 0's ask, the steps in bytes, and for each entry what it has of its own.
struct CacheLean {
    CacheAsk a;
    int64_t q_step, out_step, lse_step, pos_step;
};
struct CacheOwn {
    int32_t len, entry, splits, part;
};

// Descriptors of a launch.  Few of them travel in the kernel's arguments (which hold 4 KB), more are uploaded.
constexpr int CACHE_FEW_BYTES = 3456;
struct CacheFew {
    uint32_t w[CACHE_FEW_BYTES / 4];
};
struct CacheFar {
    const char *dev;
};
struct CacheList {
    const void *host;           // as they are on the host
    const char *dev;            // where they are on the device, or null: in the arguments
    int32_t n;
    size_t bytes;
    bool lean = false;          // asks: CacheLean, CacheOwn[n] in the place of CacheAsk[n]
};
inline size_t cache_asks_bytes(int n, bool lean) { return lean ? sizeof(CacheLean) + n * sizeof(CacheOwn) : n * sizeof(CacheAsk); }

// ins: n CacheIn, then int32 first[n + 1], running numbers of their units (see unit_of_row); outs likewise; runs: n CacheRun, then those of their pages.
hipError_t launch_cache_append(const CacheShape &c, const CacheList &ins, int units, hipStream_t s);
hipError_t launch_cache_read(const CacheShape &c, const CacheList &outs, int units, hipStream_t s);
hipError_t launch_cache_copy(const CacheShape &c, const CacheList &runs, int pages, hipStream_t s);
hipError_t launch_cache_fill(const CacheShape &c, const CacheList &fills, int longest, hipStream_t s);
hipError_t launch_cache_move(const CacheShape &c, const CacheList &moves, hipStream_t s);

constexpr int UNIT_ROWS = 64;               // rows of a page that one block of the append and read kernels takes
// the unit that a row of a sequence lies in: a page's rows in pieces of UNIT_ROWS, the last one shorter
__host__ __device__ inline int unit_of_row(int row, int page_len) { return row / page_len * ((page_len + UNIT_ROWS - 1) / UNIT_ROWS) + row % page_len / UNIT_ROWS; }

// Attention.  A row is a query and one of the `group` heads that share a kv head; a unit is a tile of rows and one of the splits of
// its keys.  An entry of few rows goes to one kernel, one of many to another.  asks: cache_asks_bytes() of entries, then for each of the two kernels that
// has any (few first) int32 first[n + 1], running numbers of units, and int32 joins[n + 1], running numbers of the rows whose keys are split.
struct CachePart {
    int32_t units, joins;       // of all asks
    int32_t each;               // > 0: every entry has that many units
    int32_t rows_of_tile;
    bool eight;                 // few rows: blocks of eight waves, not four
    bool own;                   // many rows: the kernel whose waves bring keys and values to bf16 for themselves
    float *part;                // partial results of split keys, a unit and kv head each: [rows][dp] sums, [rows] maxima, [rows] sums of weights
};
struct CachePlan {
    CachePart few, many;
};
__host__ __device__ inline size_t cache_part_floats(int rows, int dp) { return (size_t)rows * (dp + 2); }
hipError_t launch_cache_attend(const CacheShape &c, const CacheList &asks, const CachePlan &plan, hipStream_t s);

// A descriptor in a kernel whose first argument holds or names them.
template <class T> __device__ __forceinline__ T cache_desc(const CacheFew &, size_t off) { return arg_copy(kernel_arg<T>(off)); }
template <class T> __device__ __forceinline__ T cache_desc(const CacheFar &far, size_t off) { return *(const T *)(as_global(far.dev) + off); }

template <class T> __device__ __forceinline__ T desc_at(const char *dev, int i)
{
    return dev ? *(const T *)(as_global(dev) + (size_t)i * sizeof(T)) : arg_copy(kernel_arg<T>((size_t)i * sizeof(T)));
}
__device__ __forceinline__ int first_at(const char *dev, int firsts, int i)
{
    const size_t off = (size_t)firsts + 4 * (size_t)i;
    return dev ? *(const int32_t *)(as_global(dev) + off) : *kernel_arg<int32_t>(off);
}
// The entry that a unit belongs to, by running numbers int32 first[n + 1] at byte `firsts` of the descriptors: 64 of them are looked at at a time.
__device__ __forceinline__ int entry_of(const char *dev, int n, int firsts, int unit, int lane)
{
    int r = 0, end = n;                 // first[r] <= unit < first[end + 1]
    while (r < end) {
        const int step = (end - r + 63) / 64, i = r + (lane + 1) * step;
        const int f = first_at(dev, firsts, i <= end ? i : end);
        r += step * __builtin_amdgcn_readfirstlane(__popcll(__ballot(i <= end && f <= unit)));
        end = min(end, r + step - 1);
    }
    return r;
}

template <class F> hipError_t cache_launch(const CacheList &list, F &&go)
{
    if (list.dev) {
        go(CacheFar{list.dev});
    } else {
        CacheFew few;
        __builtin_memcpy(few.w, list.host, list.bytes);
        go(few);
    }
    return hipGetLastError();
}

}  // namespace aif
