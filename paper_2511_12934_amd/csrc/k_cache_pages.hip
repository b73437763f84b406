// The user cache's pages: rows in and out, table entries, whole pages moved (include/aif_cache.h).
// All of it is data movement, and memory bounds it (16 histories of 20,011 rows, two heads of 128 in fp32: appended in 151 us, 4.9 TB/s; calls of few
// rows, the launch).  A thread takes eight features of a row, which is four bytes of codes; the four threads of a
// block of 32 features find its largest magnitude among themselves.
#include "aif_cache_dev.h"

namespace aif {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

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

// Of n rows of a sequence from `first` on, those in the unit-th unit that they touch: rows [lo, lo + n) on page in_seq, which begins with row page_row.
struct UnitRows {
    int in_seq, page_row, lo, n;
};
__device__ __forceinline__ UnitRows unit_rows(int first, int n, int unit, int page_len)
{
    const int pieces = (page_len + UNIT_ROWS - 1) / UNIT_ROWS;
    unit += unit_of_row(first, page_len);
    UnitRows u;
    u.in_seq = unit / pieces;
    u.page_row = u.in_seq * page_len;
    const int from = unit % pieces * UNIT_ROWS;
    u.lo = max(u.page_row + from, first);
    u.n = min(u.page_row + min(from + UNIT_ROWS, page_len), first + n) - u.lo;
    return u;
}

// One block: rows of one page, one head.  It names the page in the table, brings the rows that a shared page held, and writes its own.
template <int DT> __global__ __launch_bounds__(256) void k_cache_append(CacheFew few /* first: kernel_arg */, const char *dev, int n_ins, CacheShape c)
{
    (void)few;
    const int firsts = n_ins * (int)sizeof(CacheIn), in = entry_of(dev, n_ins, firsts, blockIdx.x, threadIdx.x & 63);
    const CacheIn u = desc_at<CacheIn>(dev, in);
    const UnitRows at_rows = unit_rows(u.have, u.n, (int)blockIdx.x - first_at(dev, firsts, in), c.page_len);
    const int row0 = at_rows.lo - at_rows.page_row, page_no = u.page + at_rows.in_seq - u.have / c.page_len;
    const int head = blockIdx.y, dp = c.dp, per_row = dp / 8, esz = DT == 0 ? 4 : 2;
    char *page = as_global(c.pool) + (size_t)page_no * c.page_bytes + (size_t)head * cache_head_bytes(c);
    if (threadIdx.x == 0 && head == 0) c.table[u.entry + at_rows.in_seq] = page_no;
    if (u.cow >= 0 && at_rows.lo == u.have) {
        const char *from = c.pool + (size_t)u.cow * c.page_bytes + (size_t)head * cache_head_bytes(c);
        // codes in pieces of 16 bytes, scales byte by byte: the rest of either belongs to rows that this launch writes
        const int pieces = dp / 32, nb = dp / 32;
        for (int i = threadIdx.x; i < row0 * pieces; i += 256) {
            const int row = i / pieces, at = i % pieces * 16;
            const RowAt a = row_at((char *)from, dp, row), b = row_at(page, dp, row);
            *(uint4 *)(b.codes + at) = *(const uint4 *)(a.codes + at);
            *(uint4 *)(b.codes + 16 * dp + at) = *(const uint4 *)(a.codes + 16 * dp + at);
        }
        for (int i = threadIdx.x; i < row0 * nb; i += 256) {
            const int row = i / nb, at = i % nb;
            const RowAt a = row_at((char *)from, dp, row), b = row_at(page, dp, row);
            b.scales[at] = a.scales[at];
            b.scales[dp + at] = a.scales[dp + at];
        }
    }
    // a thread keeps its features; two rows' keys and values are asked for before the first is worked on
    const int step = 256 / per_row, at = threadIdx.x % per_row * 8;
    const size_t ks = (size_t)u.key_stride * 16, vs = (size_t)u.val_stride * 16, done = at_rows.lo - u.have;
    const char *keys = as_global(u.keys) + done * ks + (size_t)head * c.d_head * esz, *vals = as_global(u.vals) + done * vs + (size_t)head * c.d_head * esz;
    for (int row = threadIdx.x / per_row; row < at_rows.n && threadIdx.x < step * per_row; row += 2 * step) {
        float x[4][8];
        const bool two = row + step < at_rows.n;
        load8<DT>(keys + row * ks, at, c.d_head, x[0]);
        load8<DT>(vals + row * vs, at, c.d_head, x[1]);
        load8<DT>(keys + (two ? row + step : row) * ks, at, c.d_head, x[2]);
        load8<DT>(vals + (two ? row + step : row) * vs, at, c.d_head, x[3]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i >= 2 && !two) break;
            uint32_t byte;
            const uint32_t codes = encode8(x[i], byte);
            const RowAt to = row_at(page, dp, row0 + row + (i >= 2 ? step : 0));
            *(uint32_t *)(to.codes + (i & 1 ? 16 * dp : 0) + at / 2) = codes;
            if (at % CACHE_BLOCK == 0) to.scales[(i & 1 ? dp : 0) + at / CACHE_BLOCK] = (char)byte;
        }
    }
}

// The way back: rows of a page to keys and vals (null: not wanted), which are written.  A thread takes 16 bytes of them, so that neighbours'
// pieces make whole lines (16 histories of 20,011 rows, two heads of 128 in fp32: 142 us, in pieces
// of 32 bytes 378).
template <int DT> __global__ __launch_bounds__(256) void k_cache_read(CacheFew few /* first: kernel_arg */, const char *dev, int n_outs, CacheShape c)
{
    constexpr int WIDE = DT == 0 ? 4 : 8, ESZ = DT == 0 ? 4 : 2;
    (void)few;
    const int firsts = n_outs * (int)sizeof(CacheOut), out = entry_of(dev, n_outs, firsts, blockIdx.x, threadIdx.x & 63);
    const CacheOut u = desc_at<CacheOut>(dev, out);
    const UnitRows at_rows = unit_rows(u.first, u.n, (int)blockIdx.x - first_at(dev, firsts, out), c.page_len);
    const int lo = at_rows.lo, n = at_rows.n, page_row = at_rows.page_row;
    const int head = blockIdx.y, dp = c.dp, per_row = dp / WIDE;
    char *page = as_global(c.pool) + (size_t)as_global(c.table)[u.entry + at_rows.in_seq] * c.page_bytes + (size_t)head * cache_head_bytes(c);
    const int step = 256 / per_row, at = threadIdx.x % per_row * WIDE;
    const size_t to = (size_t)head * c.d_head + at;
    char *keys = u.keys ? as_global(u.keys) + ((size_t)(lo - u.first) * u.key_stride + to) * ESZ : nullptr;
    char *vals = u.vals ? as_global(u.vals) + ((size_t)(lo - u.first) * u.val_stride + to) * ESZ : nullptr;
    if (at >= c.d_head) return;
    for (int row = threadIdx.x / per_row; row < n && threadIdx.x < step * per_row; row += 4 * step) {
        uint32_t codes[8], byte[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = row + i / 2 * step;
            const RowAt from = row_at(page, dp, lo - page_row + (r < n ? r : row));
            const char *p = from.codes + (i & 1 ? 16 * dp : 0) + at / 2;
            codes[i] = DT == 0 ? *(const uint16_t *)p : *(const uint32_t *)p;
            byte[i] = (uint8_t)from.scales[(i & 1 ? dp : 0) + at / CACHE_BLOCK];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = row + i / 2 * step;
            char *dst = i & 1 ? vals : keys;
            if (r >= n || !dst) continue;
            const float scale = __uint_as_float(byte[i] << 23);
            u32x4 v;
            v.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], scale, 0));
            v.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], scale, 1));
            if constexpr (DT == 0) {
                v = u32x4{v.x << 16, v.x & 0xffff0000u, v.y << 16, v.y & 0xffff0000u};
            } else {
                v.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], scale, 2));
                v.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], scale, 3));
            }
            __builtin_nontemporal_store(v, (u32x4 *)(dst + (size_t)r * (i & 1 ? u.val_stride : u.key_stride) * ESZ));
        }
    }
}

template <class ARGS> __global__ __launch_bounds__(256) void k_cache_fill(ARGS list, int32_t *table)
{
    const CacheFill f = cache_desc<CacheFill>(list, (size_t)blockIdx.x * sizeof(CacheFill));
    const int i = blockIdx.y * 256 + threadIdx.x;
    if (i < f.n) table[f.dst + i] = f.src < 0 ? f.value : table[f.src + i];
}

constexpr int MOVE_PIECES = 4 * 256;            // at most, of one block: four pieces of 16 bytes a thread in flight

// a page's blocks share it evenly
__device__ __forceinline__ void move_page(const CacheShape &c, int from, int to)
{
    const u32x4 *src = (const u32x4 *)(as_global(c.pool) + (size_t)from * c.page_bytes);
    u32x4 *dst = (u32x4 *)(as_global(c.pool) + (size_t)to * c.page_bytes);
    const int all = (int)(c.page_bytes / 16), each = (all + gridDim.y - 1) / gridDim.y;
    const int at = blockIdx.y * each + threadIdx.x, end = min(all, (int)(blockIdx.y + 1) * each);
    u32x4 v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (at + 256 * j < end) v[j] = __builtin_nontemporal_load(src + at + 256 * j);
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (at + 256 * j < end) __builtin_nontemporal_store(v[j], dst + at + 256 * j);
}
template <class ARGS> __global__ __launch_bounds__(256) void k_cache_move(ARGS list, CacheShape c)
{
    const CacheMove m = cache_desc<CacheMove>(list, (size_t)blockIdx.x * sizeof(CacheMove));
    if (m.entry >= 0 && blockIdx.y == 0 && threadIdx.x == 0) c.table[m.entry] = m.dst;
    if (m.src >= 0) move_page(c, m.src, m.dst);
}
// Whole sequences: the pages that are copied are the table's to know, and the new ones mostly follow each other.  (A descriptor a page,
// read from the host's memory: 14.8 us for 1,277 pages of 17 KB, 10 with runs of them in the arguments.)
__global__ __launch_bounds__(256) void k_cache_copy(CacheFew few /* first: kernel_arg */, const char *dev, int n_runs, CacheShape c)
{
    (void)few;
    const int firsts = n_runs * (int)sizeof(CacheRun), run = entry_of(dev, n_runs, firsts, blockIdx.x, threadIdx.x & 63);
    const CacheRun m = desc_at<CacheRun>(dev, run);
    const int i = (int)blockIdx.x - first_at(dev, firsts, run);
    if (blockIdx.y == 0 && threadIdx.x == 0) c.table[m.dst + i] = m.page < 0 ? -1 : m.page + i;
    if (m.page >= 0) move_page(c, as_global(c.table)[m.src + i], m.page + i);
}

}  // namespace

hipError_t launch_cache_append(const CacheShape &c, const CacheList &ins, int units, hipStream_t s)
{
    if (units == 0) return hipSuccess;
    CacheFew args;
    if (!ins.dev) __builtin_memcpy(args.w, ins.host, ins.bytes);
    const dim3 grid(units, c.n_kv);
    if (c.dtype == 0) hipLaunchKernelGGL(k_cache_append<0>, grid, dim3(256), 0, s, args, ins.dev, ins.n, c);
    else hipLaunchKernelGGL(k_cache_append<1>, grid, dim3(256), 0, s, args, ins.dev, ins.n, c);
    return hipGetLastError();
}

hipError_t launch_cache_read(const CacheShape &c, const CacheList &outs, int units, hipStream_t s)
{
    if (units == 0) return hipSuccess;
    CacheFew args;
    if (!outs.dev) __builtin_memcpy(args.w, outs.host, outs.bytes);
    const dim3 grid(units, c.n_kv);
    if (c.dtype == 0) hipLaunchKernelGGL(k_cache_read<0>, grid, dim3(256), 0, s, args, outs.dev, outs.n, c);
    else hipLaunchKernelGGL(k_cache_read<1>, grid, dim3(256), 0, s, args, outs.dev, outs.n, c);
    return hipGetLastError();
}

static unsigned blocks_of_page(const CacheShape &c) { return (unsigned)((c.page_bytes / 16 + MOVE_PIECES - 1) / MOVE_PIECES); }

hipError_t launch_cache_copy(const CacheShape &c, const CacheList &runs, int pages, hipStream_t s)
{
    if (pages == 0) return hipSuccess;
    CacheFew args;
    if (!runs.dev) __builtin_memcpy(args.w, runs.host, runs.bytes);
    hipLaunchKernelGGL(k_cache_copy, dim3(pages, blocks_of_page(c)), dim3(256), 0, s, args, runs.dev, runs.n, c);
    return hipGetLastError();
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
        hipLaunchKernelGGL((k_cache_move<decltype(args)>), dim3(moves.n, blocks_of_page(c)), dim3(256), 0, s, args, c);
    });
}

}  // namespace aif
