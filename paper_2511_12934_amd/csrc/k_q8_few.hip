// Products of 8-bit matrices with few rows (include/aif_q8.h: aif_q8_linear).
//
// Few rows are bound by the weights' bytes and by latency, so that all of the device has to ask for them at once: a block takes few columns
// (16, or the 128 of a scale where 8 bits come out) and shares the contraction among its waves, who meet in LDS.  A wave
// loads up to four blocks of 128 columns before it waits: whole rows' pieces of 128 bytes, eight lanes each, and passes them through LDS to the lanes that
// multiply them.  (Loaded by those lanes themselves, each of 16 neighbouring ones from another row, a unit gets 16 bytes a cycle from its cache: 1 x 4096 x 4096
// 5.8 us instead of 4.9, 64 x 4096 x 4096 15.1 and 12.1, gated 1 x 1024 x 4096 in 8 bits, where 32 blocks do it all, 10.4 and 6.2.)
//
// One row: 4096 x 4096 4.9 us (3.4 TB/s), 8192 x 8192 12.9 us (5.2 TB/s), 1024 x 1024 3.8 us, of which 2.5 are the launch; 64 x 2048 x 1024 4.0 us.
#include "k_q8_product.h"

#include <type_traits>

namespace aif {

namespace {

// A tile of 16 MT rows by 16 NT WN columns (with a gate of both sides): WK waves share the blocks of columns of a and w, WN the tile's columns.
template <int MT, int NT, int WK, int WN, bool GATE, bool WHOLE, bool CODES> __global__ __launch_bounds__(64 * WK * WN) void k_q8_few(const Q8LinearCall c, int tiles_n)
{
    constexpr int SIDES = GATE ? 2 : 1, ROWS = 16 * MT, COLS = 16 * NT * WN, PITCH = COLS + 4;
    constexpr int ITEMS = ROWS * COLS / 4, THREADS = 64 * WK * WN;               // pieces of four columns that threads end with
    static_assert(!CODES || COLS == Q8_BLOCK, "a scale's columns are the block's");
    static_assert(Q8_BLOCK % COLS == 0, "one scale of w");
    __shared__ float part[WK][SIDES][ROWS][PITCH];
    __shared__ q8_u4 turned[WK * WN][16 * 8];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wk = wave / WN, wn = wave % WN, r = lane % 16, g = lane / 16;
    const int ahead = lane % 8 * 16;                                             // a lane loads 16 codes from here on of rows lane / 8 and lane / 8 + 8 of a tile's 16
    const int n0 = (int)(blockIdx.x % tiles_n) * COLS;
    const int64_t m0 = (int64_t)(blockIdx.x / tiles_n) * ROWS;
    const int whole = c.k / Q8_BLOCK, left = c.k % Q8_BLOCK;

    const uint8_t *a_row[MT][2], *as_row[MT], *w_row[SIDES][NT][2], *ws[SIDES];
#pragma unroll
    for (int ta = 0; ta < MT; ++ta) {
        as_row[ta] = c.a.scales + min(m0 + ta * 16 + r, (int64_t)c.m - 1) * c.a.scale_stride;
#pragma unroll
        for (int h = 0; h < 2; ++h) a_row[ta][h] = c.a.codes + min(m0 + ta * 16 + h * 8 + lane / 8, (int64_t)c.m - 1) * c.a.stride + ahead;
    }
#pragma unroll
    for (int side = 0; side < SIDES; ++side) {
        const Q8Mat &w = side ? c.up : c.w;
        ws[side] = w.scales + (int64_t)(n0 / Q8_BLOCK) * w.scale_stride;
#pragma unroll
        for (int tw = 0; tw < NT; ++tw)
#pragma unroll
            for (int h = 0; h < 2; ++h) w_row[side][tw][h] = w.codes + (int64_t)min(n0 + (wn * NT + tw) * 16 + h * 8 + lane / 8, c.n - 1) * w.stride + ahead;
    }
    q8_f4 acc[SIDES][NT][MT] = {};
    // From the lanes that loaded them to those that multiply them: row r, columns 16 g and 64 + 16 g on.  A wave's accesses of LDS come in order.
    q8_u4 *const slot = turned[wave];
    auto turn = [&](const q8_u4 (&x)[2]) __attribute__((always_inline)) -> q8_i8 {
        slot[lane ^ lane / 8] = x[0], slot[64 + (lane ^ lane / 8)] = x[1];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const q8_u4 lo = slot[r * 8 + (g ^ r % 8)], hi = slot[r * 8 + ((g + 4) ^ r % 8)];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        return q8_i8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
    };
    // U blocks from `first` on, every WK-th; the last one's codes, where it is short, up to column `end` of it
    auto blocks = [&](int first, auto many, int end) __attribute__((always_inline)) {
        constexpr int U = decltype(many)::value;
        q8_u4 a[U][MT][2], w[U][SIDES][NT][2];
        int as[U][MT], wsc[U][SIDES];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = (int64_t)(first + u * WK) * Q8_BLOCK;
#pragma unroll
            for (int side = 0; side < SIDES; ++side) {
                wsc[u][side] = ws[side][first + u * WK];
#pragma unroll
                for (int tw = 0; tw < NT; ++tw)
#pragma unroll
                    for (int h = 0; h < 2; ++h) w[u][side][tw][h] = load16(w_row[side][tw][h] + at, 0, end - ahead);
            }
#pragma unroll
            for (int ta = 0; ta < MT; ++ta) {
                as[u][ta] = as_row[ta][first + u * WK];
#pragma unroll
                for (int h = 0; h < 2; ++h) a[u][ta][h] = load16(a_row[ta][h] + at, 0, end - ahead);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            q8_i8 turned_w[SIDES][NT];
#pragma unroll
            for (int side = 0; side < SIDES; ++side)
#pragma unroll
                for (int tw = 0; tw < NT; ++tw) turned_w[side][tw] = turn(w[u][side][tw]);
#pragma unroll
            for (int ta = 0; ta < MT; ++ta) {
                const Side<WHOLE> sa(turn(a[u][ta]), as[u][ta]);
#pragma unroll
                for (int side = 0; side < SIDES; ++side)
#pragma unroll
                    for (int tw = 0; tw < NT; ++tw) acc[side][tw][ta] = mma(Side<WHOLE>(turned_w[side][tw], wsc[u][side]), sa, acc[side][tw][ta]);
            }
        }
    };
    constexpr int ROOM = WK * WN > 8 ? 64 : 128, EACH = (MT + SIDES * NT) * 8, MOST = 4 * EACH <= ROOM ? 4 : 2 * EACH <= ROOM ? 2 : 1;   // registers for codes, blocks they hold
    int b = wk;
    for (; b + (MOST - 1) * WK < whole; b += MOST * WK) blocks(b, std::integral_constant<int, MOST>{}, Q8_BLOCK);
    if (MOST > 2 && b + WK < whole) blocks(b, std::integral_constant<int, 2>{}, Q8_BLOCK), b += 2 * WK;
    for (; b < whole; b += WK) blocks(b, std::integral_constant<int, 1>{}, Q8_BLOCK);
    if (left && b == whole) blocks(b, std::integral_constant<int, 1>{}, left);

#pragma unroll
    for (int side = 0; side < SIDES; ++side)
#pragma unroll
        for (int tw = 0; tw < NT; ++tw)
#pragma unroll
            for (int ta = 0; ta < MT; ++ta) *(q8_f4 *)&part[wk][side][ta * 16 + r][(wn * NT + tw) * 16 + g * 4] = acc[side][tw][ta];
    __syncthreads();
#pragma unroll
    for (int first = 0; first < ITEMS; first += THREADS) {
        const int item = first + threadIdx.x;
        if (ITEMS % THREADS && item >= ITEMS) break;
        const int row = item / (COLS / 4), col = item % (COLS / 4) * 4;
        q8_f4 z[SIDES] = {};
#pragma unroll
        for (int side = 0; side < SIDES; ++side)
#pragma unroll
            for (int w = 0; w < WK; ++w) z[side] += *(const q8_f4 *)&part[w][side][row][col];
        const bool live = m0 + row < c.m && n0 + col < c.n;
        uint32_t top = 0;
        float v[4] = {z[0][0], z[0][1], z[0][2], z[0][3]};
        if (live) {
            if (c.bias) {
                float x[4];
                load_values<WHOLE>(c.bias, n0 + col, x);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] += x[i];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (c.act == Q8_ACT_RELU) v[i] = v[i] < 0.f ? 0.f : v[i];
                if constexpr (GATE) v[i] = silu<WHOLE>(v[i]) * z[1][i];
            }
            if (c.residual) {
                float x[4];
                load_values<WHOLE>(c.residual, (m0 + row) * c.residual_stride + n0 + col, x);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] += x[i];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) top = max(top, q8_magnitude(v[i]));
        }
        if constexpr (!CODES) {
            if (live) store_values<WHOLE>(c.out, (m0 + row) * c.out_stride + n0 + col, v);
        } else {
#pragma unroll
            for (int o = 1; o < 32; o *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
            const uint32_t byte = q8_scale_byte(top);
            if (!live) continue;
            *(uint32_t *)(c.q.codes + (m0 + row) * c.q.stride + n0 + col) = q8_codes4(v, q8_unit(top, byte));
            if (col == 0) c.q.scales[(m0 + row) * c.q.scale_stride + n0 / Q8_BLOCK] = (uint8_t)byte;
        }
    }
}

template <int MT, int NT, int WK, int WN, bool GATE, bool WHOLE, bool CODES> hipError_t go(const Q8LinearCall &c, hipStream_t s)
{
    constexpr int COLS = 16 * NT * WN;
    const int tiles_n = (c.n + COLS - 1) / COLS, tiles_m = (c.m + 16 * MT - 1) / (16 * MT);
    k_q8_few<MT, NT, WK, WN, GATE, WHOLE, CODES><<<dim3((unsigned)(tiles_m * tiles_n)), dim3(64 * WK * WN), 0, s>>>(c, tiles_n);
    return hipGetLastError();
}

// mt: tiles of 16 rows a block, 1, 2 or 4
template <bool GATE, bool WHOLE> hipError_t few(const Q8LinearCall &c, int mt, hipStream_t s)
{
    if (!c.out) return go<1, 2, 4, 4, GATE, WHOLE, true>(c, s);
    if (mt == 1) return go<1, 1, 8, 1, GATE, WHOLE, false>(c, s);
    if (mt == 2) return go<2, 1, 8, 1, GATE, WHOLE, false>(c, s);
    return go<4, 1, 8, 1, GATE, WHOLE, false>(c, s);
}

}  // namespace

hipError_t launch_q8_few(const Q8LinearCall &c, int mt, hipStream_t s)
{
    if (c.act == Q8_ACT_GATE) return c.f32 ? few<true, true>(c, mt, s) : few<true, false>(c, mt, s);
    return c.f32 ? few<false, true>(c, mt, s) : few<false, false>(c, mt, s);
}

}  // namespace aif
