// Products of 8-bit matrices with many rows (include/aif_q8.h: aif_q8_linear).
//
// A block of 2 WM waves makes a tile of 16 WM MT rows by 128 NG columns of the result (with a gate: of 128 columns of each side), a wave 16 MT
// rows by 64 NG columns, in registers.  128 columns of a and w at a time go straight from memory to LDS, two steps of them there.  A row of LDS is
// 128 bytes, its eight pieces of 16 shuffled by the row, so that eight lanes that read the same piece of eight rows meet no bank twice.
//
// A step: the weights' codes for a wave's columns lie in registers, read while the step before ended; those of 16 rows of a are read a
// turn ahead of their products.  Once all waves have their weights, the next but one step's are asked for into their place, a few loads a
// turn (a wave that asks for many at once waits for their addresses with its products); before the last turn all waves have read their rows of
// a as well, and the next step has come, asked for a step ago.
//
// Blocks stay and take tile after tile: the loads run two steps ahead across a tile's end, so that the next one's codes come while this one's sums
// are written.  (Its stores are in the same counter as these loads and are not counted in the next tile's first two waits, which therefore see them done.)  With one wave to a matrix core nothing hides what else a wave issues: everything (reads of LDS, loads, the next
// addresses) stands between two products, and the steps that need no branch run in a loop without one.
//
// The matrix cores bound large calls: 8192 x 8192 x 8192 takes 389 us, 2.8 PFLOP/s, where the instruction by itself reaches 4.1 - 4.5 on random codes
// and a library's product with one scale for all 337 us; a step of LDS reads costs little less than its products, and the clock falls to 2.1 GHz.
// 65536 x 4096 x 4096 takes 828 us, with residual 941: 1.4 us a step, and 6.3 or 13.4 for a tile's end, which its products do not hide (the residual: at its reading below).  Gated
// 16000 x 1024 x 4096 122 - 128 us (1.39 us a step, 4.7 a tile's end, most of it exponentials and reciprocals), 32000 x 512 x 2048 in 8 bits 80 - 82 us.  Tried and slower: eight waves a
// tile of 256 by 256 (411 us for 8192^3), two blocks a unit with tiles of 128 by 256, blocks started apart in time.  fp32 (bf16 products of whole codes) 4096 x 4096 x 4096 117 us, 1.17 PFLOP/s, gated
// 206 us, gated 16000 x 1024 x 4096 243 us, 32000 x 512 x 2048 in 8 bits 161 us.
#include "k_q8_form.h"
#include "k_q8_product.h"
#include "mfma_util.h"

#include <algorithm>
#include <type_traits>

namespace aif {

namespace {

// Which 16 rows of the weights a product takes: a lane of the result has four neighbouring rows of each of four products of a group of 64, and
// these are to be RUN neighbouring columns, four lanes' runs side by side: 64 bytes of a row of the result, whatever its type.
template <int RUN> __device__ __forceinline__ constexpr int w_row(int t, int r) { return t * 4 / RUN * 4 * RUN + (r >> 2) * RUN + t * 4 % RUN + (r & 3); }
// The shuffle of a row's pieces: another one for each of eight neighbouring lanes' rows.
__device__ __forceinline__ int a_key(int row) { return row & 7; }
template <int RUN> __device__ __forceinline__ int w_key(int row) { return (row & 3) | ((row / RUN) & 1) << 2; }

// Lane's 4 bytes to lds_dst + 4 lane, as dma16 of mfma_util.h.
__device__ __forceinline__ void dma4(const char *gsrc, uint32_t lds_dst)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds_dst), "v"(gsrc) : "memory");
}

// A sum out of its accumulation register, here and now (four waves a unit have sums for these registers alone; eight hold them among the others): left to itself the compiler moves them to and fro around every branch.  The products that
// made them must be over (32 wait states: 16 x 16 x 128 takes 8 passes of 4 cycles, 16 x 16 x 32 fewer).
__device__ __forceinline__ float from_sum(float a)
{
    float x;
    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(a));
    return x;
}

// The lane's number, found where it is wanted: what is derived from one kept from the kernel's start would be too, in registers that the main loop lacks.
__device__ __forceinline__ int lane_now()
{
    int x;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(x));
    return x;
}

// The same address, in scalar registers.
__device__ __forceinline__ const char *uniform(const char *p)
{
    const uint64_t u = (uint64_t)p;
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)u), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(u >> 32));
    return (const char *)((uint64_t)hi << 32 | lo);
}

// A tile of the result: which it is.  The XCDs take blocks in turn: each has a run of tiles, 8 columns of tiles wide, so that its units, who are
// at neighbouring ones, share rows and weights in its L2.
struct Tiles {
    int m, n, per, of_xcd, at, step;        // tiles down and across, of an XCD; this block's first, and what it goes on by
    __device__ __forceinline__ Tiles(int tiles_m, int tiles_n) : m(tiles_m), n(tiles_n)
    {
        per = (m * n + 7) / 8;
        const int first = (int)(blockIdx.x % 8) * per;
        of_xcd = min(first + per, m * n);
        at = first + (int)(blockIdx.x / 8);
        step = (int)(gridDim.x / 8);
    }
    __device__ __forceinline__ void place(int id, int &row, int &col) const
    {
        const int band = id / (8 * m), in_band = id - band * 8 * m, width = min(8, n - band * 8);
        row = in_band / width, col = band * 8 + in_band % width;
    }
};

// RES: with a residual.
template <int WM, int MT, int NG, bool GATE, bool WHOLE, bool CODES, bool RES> __global__ __launch_bounds__(128 * WM) void k_q8_many(const Q8LinearCall c, int tiles_m, int tiles_n)
{
    constexpr int WAVES = 2 * WM, TM = 16 * WM * MT, TN = 128 * NG, NW = 4 * NG; // rows of a and of w of a step, products across of a wave
    constexpr int A_SLOTS = TM / 8 / WAVES, W_SLOTS = TN / 8 / WAVES;            // loads of 8 rows each wave makes for a step
    constexpr bool TWICE = WM == 2;                                              // a wave has registers for the weights of two steps
    constexpr int COLS = GATE ? TN / 2 : TN, OWN = COLS / 2;                     // of the result: the tile's, a wave's
    constexpr int A_BYTES = TM * Q8_BLOCK, W_BYTES = TN * Q8_BLOCK, A_AT = 2 * W_BYTES, S_AT = A_AT + 2 * A_BYTES;
    constexpr int SCALES = TM * 4 + 256;                                         // a step's scale bytes, with its neighbours': a dword for each row of a, and for the blocks of w
    constexpr int RUN = CODES ? 16 : WHOLE ? 4 : 8;
    static_assert((A_BYTES & (A_BYTES - 1)) == 0 && (W_BYTES & (W_BYTES - 1)) == 0 && A_AT % (2 * A_BYTES) == 0, "the two steps' places differ in one bit");
    static_assert(TWICE || NW == 8, "the last turn's sums");
    static_assert(W_SLOTS % 4 == 0 && A_SLOTS % 2 == 0 && TM / 64 <= WAVES && TM >= 64 && MT % 4 == 0 && (!GATE || NG == 2), "turns, w_key, scales, both sides in a wave");
    __shared__ __align__(65536) char lds[S_AT + 2 * SCALES];
    __shared__ uint32_t s_top[CODES ? 2 : 1][CODES ? TM : 1];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wm = wave / 2, wn = wave % 2, r = lane % 16, g = lane / 16;
    const int steps = (c.k + Q8_BLOCK - 1) / Q8_BLOCK, left = c.k % Q8_BLOCK;    // columns of the last step, 0: all
    const uint32_t lds0 = lds_address(lds);
    const Tiles tiles(tiles_m, tiles_n);
    if (tiles.at >= tiles.of_xcd) return;

    // ---- what is asked for: step by step, tile after tile, two steps ahead of the products; behind the last step that one again, which nobody reads
    int ld_tile = tiles.at, ld_t = 0;                                            // its tile, its step in that one
    uint32_t ld_at = 0;                                                          // bit 0: which of the two places in LDS
    const int lrow = lane / 8, slot = lane % 8;
    const int a_col = (slot ^ a_key(lrow)) << 4, w_even = (slot ^ w_key<RUN>(lrow)) << 4, w_odd = (slot ^ w_key<RUN>(lrow + RUN)) << 4;
    constexpr auto of_w = [](int i, int even, int odd) { return RUN != 4 && (RUN == 8 ? i : i / 2) % 2 ? odd : even; };      // (a row's shuffle, of load i)
    uint32_t a_off[A_SLOTS], w_off[W_SLOTS];                                     // this lane's places: eight rows a load, rows behind the last one that one again
    const Q8Mat &w_side = GATE && wave >= WM ? c.up : c.w;                       // with a gate one side's 128 rows come first, then the other's
    int last_row, last_col;
    uint32_t as_off, ws_off;
    const char *a_ptr, *w_ptr, *as_base, *ws_base, *us_base;
    // Pieces behind the last column are those of the step's first, and zeroed when they have come.
    auto clip = [&]() __attribute__((always_inline)) {
        if (left == 0 || ld_t != steps - 1) return;
#pragma unroll
        for (int i = 0; i < A_SLOTS; ++i) a_off[i] -= a_col >= left ? a_col : 0;
#pragma unroll
        for (int i = 0; i < W_SLOTS; ++i) w_off[i] -= of_w(i, w_even, w_odd) >= left ? of_w(i, w_even, w_odd) : 0;
    };
    auto aim = [&]() __attribute__((always_inline)) {
        int tm, tn;
        tiles.place(ld_tile, tm, tn);
        const int64_t m0 = (int64_t)tm * TM;
        const int n0 = tn * COLS;
        last_row = __builtin_amdgcn_readfirstlane((int)min((int64_t)TM, c.m - m0) - 1);
        last_col = __builtin_amdgcn_readfirstlane(min(COLS, c.n - n0) - 1);
        a_ptr = uniform((const char *)c.a.codes + m0 * c.a.stride), w_ptr = uniform((const char *)w_side.codes + (int64_t)n0 * w_side.stride);
        as_base = uniform((const char *)c.a.scales + m0 * c.a.scale_stride);
        ws_base = uniform((const char *)c.w.scales + (int64_t)(n0 / Q8_BLOCK) * c.w.scale_stride);
        if constexpr (GATE) us_base = uniform((const char *)c.up.scales + (int64_t)(n0 / Q8_BLOCK) * c.up.scale_stride);
        as_off = __umul24(min((wave & (TM / 64 - 1)) * 64 + lane, last_row), (int)c.a.scale_stride);
        ws_off = __umul24(min(lane, last_col / Q8_BLOCK), (int)c.w.scale_stride);
#pragma unroll
        for (int i = 0; i < A_SLOTS; ++i) a_off[i] = __umul24(min((wave * A_SLOTS + i) * 8 + lrow, last_row), (int)c.a.stride) + a_col;
#pragma unroll
        for (int i = 0; i < W_SLOTS; ++i)
            w_off[i] = __umul24(min(((GATE ? wave % WM : wave) * W_SLOTS + i) * 8 + lrow, last_col), (int)w_side.stride) + of_w(i, w_even, w_odd);
        clip();
    };
    // the scale bytes of four steps, this one among them: each wave those of 64 rows (where TM is less, doubled), and all of them the same ones of w
    auto load_scales = [&]() __attribute__((always_inline)) {
        const uint32_t at = lds0 + S_AT + (ld_at & 1) * SCALES;
        const int t = ld_t & ~3;
        dma_s<4>(as_base + t, as_off, at + (wave & (TM / 64 - 1)) * 256, 0);
        if constexpr (GATE) dma4((lane_now() == 0 ? ws_base : us_base) + t, at + TM * 4);
        else dma_s<4>(ws_base + t, ws_off, at + TM * 4, 0);
    };
    auto load_a = [&](int from, int to) __attribute__((always_inline)) {
        const uint32_t at = lds0 + A_AT + (ld_at & 1) * A_BYTES + wave * A_SLOTS * 1024;
#pragma unroll
        for (int i = 0; i < A_SLOTS; ++i)
            if (i >= from && i < to) dma_s<16>(a_ptr, a_off[i], at, i * 1024);
    };
    auto load_w = [&](int from, int to) __attribute__((always_inline)) {
        const uint32_t at = lds0 + (ld_at & 1) * W_BYTES + wave * W_SLOTS * 1024;
#pragma unroll
        for (int i = 0; i < W_SLOTS; ++i)
            if (i >= from && i < to) dma_s<16>(w_ptr, w_off[i], at, i * 1024);
    };
    // on to the next step; FAST: it is the same tile's, and not its last one where that is short
    auto load_next = [&](auto fast) __attribute__((always_inline)) {
        ++ld_at;
        if (decltype(fast)::value || ld_t + 1 < steps) {
            ++ld_t;
            a_ptr += Q8_BLOCK, w_ptr += Q8_BLOCK;
            if constexpr (!decltype(fast)::value) clip();
        } else if (ld_tile + tiles.step < tiles.of_xcd) {
            ld_t = 0;
            ld_tile += tiles.step;
            aim();
        }
    };

    // ---- what has come
    auto meet = [&]() __attribute__((always_inline)) {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // The pieces that this wave has loaded of a tile's last columns: zeros behind the last.
    auto zero_a = [&](uint32_t buf) __attribute__((always_inline)) {
        const int lane = lane_now(), col = ((lane % 8) ^ a_key(lane / 8)) << 4;
        char *const at = lds + A_AT + buf * A_BYTES + wave * A_SLOTS * 1024 + lane * 16;
#pragma unroll 1
        for (int i = 0; i < A_SLOTS; ++i) {
            if (col >= left) *(q8_u4 *)(at + i * 1024) = q8_u4{};
            else if (col + 8 == left) *(q8_u2 *)(at + i * 1024 + 8) = q8_u2{};
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
    auto zero_w = [&](uint32_t buf) __attribute__((always_inline)) {
        const int lane = lane_now(), even = ((lane % 8) ^ w_key<RUN>(lane / 8)) << 4, odd = ((lane % 8) ^ w_key<RUN>(lane / 8 + RUN)) << 4;
        char *const at = lds + buf * W_BYTES + wave * W_SLOTS * 1024 + lane * 16;
#pragma unroll 1
        for (int i = 0; i < W_SLOTS; ++i) {
            const int col = of_w(i, even, odd);
            if (col >= left) *(q8_u4 *)(at + i * 1024) = q8_u4{};
            else if (col + 8 == left) *(q8_u2 *)(at + i * 1024 + 8) = q8_u2{};
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
    // 32 codes of a row in LDS: pieces g and g + 4, which are 64 bytes apart either way.  The addresses are those of this step; the next one's differ in a bit.
    uint32_t a_lo = (uint32_t)(A_AT + (wm * MT * 16 + r) * Q8_BLOCK + ((g ^ a_key(r)) << 4));
    uint32_t w_lo = (uint32_t)((wn * (GATE ? 64 : 64 * NG) + w_row<RUN>(0, r)) * Q8_BLOCK + ((g ^ w_key<RUN>(w_row<RUN>(0, r))) << 4));
    auto codes = [&](uint32_t lo_at, int row) {
        const q8_u4 lo = *(const q8_u4 *)(lds + lo_at + row * Q8_BLOCK), hi = *(const q8_u4 *)(lds + (lo_at ^ 64) + row * Q8_BLOCK);
        return q8_i8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
    };
    auto read_w = [&](uint32_t at, int tw) { return codes(at, (GATE ? tw / 4 * 128 : tw / 4 * 64) + w_row<RUN>(tw % 4, 0)); };
    const uint32_t as_lane = (uint32_t)(S_AT + (wm * MT * 16 + r) * 4);
    auto scale_a = [&](uint32_t at, int ta) { return (int)*(const uint8_t *)(lds + as_lane + at + ta * 64); };
    auto scale_w = [&](uint32_t at, int side) { return (int)*(const uint8_t *)(lds + S_AT + TM * 4 + at + (GATE ? side : NG == 2 ? wn : 0) * 4); };

    uint32_t buf = 0;                                                            // which of the two places this step has
    aim();
    load_w(0, W_SLOTS);
    load_scales();
    load_a(0, A_SLOTS);
    load_next(std::false_type{});
    load_w(0, W_SLOTS);
    load_scales();
    load_a(0, A_SLOTS / 2);
    wait_vmcnt<A_SLOTS / 2 + W_SLOTS + 2>();
    if (left != 0 && steps == 1) zero_a(0), zero_w(0);
    meet();

    constexpr int SIDES = GATE ? 2 : 1, HALF = MT / 2;      // the turn from which the next step's weights are read
    constexpr int W_EACH = W_SLOTS / HALF;                  // loads of w in each of the turns from the second on, HALF of them
    constexpr int W_SETS = TWICE ? 2 : 1;
    static_assert(W_SLOTS % HALF == 0, "as many loads in each turn");
    for (int tile = tiles.at; tile < tiles.of_xcd; tile += tiles.step) {
        q8_f4 acc[NW][MT] = {};
        q8_i8 wf[W_SETS][NW], af[2];
        int sw[2][SIDES], sa[2];
        uint32_t sat = buf * SCALES;
#pragma unroll
        for (int tw = 0; tw < NW; ++tw) wf[0][tw] = read_w(w_lo, tw);
#pragma unroll
        for (int q = 0; q < SIDES; ++q) sw[0][q] = scale_w(sat, q);
        af[0] = codes(a_lo, 0), sa[0] = scale_a(sat, 0);
        if constexpr (TWICE) {                              // all waves have read them here: the first step asks for others into their place
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            meet();
        }

        // Step t; FAST: those that it asks for are this tile's, and none of them its short last one.  (Branches and scalar sums between the products
        // take as long as the products do.)
        auto step = [&](int t, auto fast) __attribute__((always_inline)) {
            constexpr bool FAST = decltype(fast)::value;
            const bool turns = !FAST && t + 1 == steps;     // the next step is the next tile's first
            const uint32_t next_sat = (buf ^ 1) * SCALES + (turns ? 0 : (t + 1) & 3);
            const bool next_last = !FAST && left != 0 && (turns ? steps == 1 : t + 2 == steps);
            const uint32_t a_next = a_lo ^ A_BYTES, w_next = w_lo ^ W_BYTES;
#pragma unroll
            for (int ta = 0; ta < MT; ++ta) {
                __builtin_amdgcn_sched_barrier(0);
                if (!TWICE && ta == 1) meet();  // all waves have this step's weights in registers
                if (TWICE && ta == HALF) {      // the next step's weights have come: older than its rows of a and what was asked for of the one after
                    wait_vmcnt<A_SLOTS + 2 + W_EACH * (HALF - 1)>();
                    if (next_last) zero_w(buf ^ 1);
                    meet();
                }
                if (ta == MT - 1) {             // its rows of a (and else its weights) have come, and all waves have read this step's
                    wait_vmcnt<W_SLOTS>();
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    if (next_last) zero_a(buf ^ 1);
                    if (!TWICE && next_last) zero_w(buf ^ 1);
                    meet();
                }
                const Side<WHOLE> a(af[ta % 2], sa[ta % 2]);
#pragma unroll
                for (int tw = 0; tw < NW; ++tw) {
                    acc[tw][ta] = mma(Side<WHOLE>(wf[0][tw], sw[0][GATE ? tw / 4 : 0]), a, acc[tw][ta]);
                    // (no instruction: without it the compiler puts the step's products behind its barriers)
                    if constexpr (TWICE) asm volatile("" : "+a"(acc[tw][ta]));
                    else asm volatile("" : "+v"(acc[tw][ta]));
                    // what else there is to do goes between the products: a wave that comes to several such instructions in a row leaves the matrix core idle
                    if (tw == 0) af[(ta + 1) % 2] = ta + 1 < MT ? codes(a_lo, (ta + 1) * 16) : codes(a_next, 0);
                    if (tw == 1) {
                        sa[(ta + 1) % 2] = ta + 1 < MT ? scale_a(sat, ta + 1) : scale_a(next_sat, 0);
                        if (ta == MT - 1) {
#pragma unroll
                            for (int q = 0; q < SIDES; ++q) sw[1][q] = scale_w(next_sat, q);
                        }
                    }
                    if (tw >= 2) {
                        // loads of this place among the turn's
                        constexpr int SPOTS = NW - 2;
                        const int h = A_SLOTS / 2, spot = tw - 2;
                        if (ta == 0) load_a(h + spot * h / SPOTS, h + (spot + 1) * h / SPOTS);
                        if (ta >= 1 && ta <= HALF) load_w((ta - 1) * W_EACH + spot * W_EACH / SPOTS, (ta - 1) * W_EACH + (spot + 1) * W_EACH / SPOTS);
                        if (ta == MT - 1) {
                            if (spot == 0) load_scales();
                            load_a(spot * h / SPOTS, (spot + 1) * h / SPOTS);
                        }
                        // weights of the next step: NW in the turns from HALF to the last but one, at a turn's last places
                        constexpr int TURNS = MT - 1 - HALF, EACH = (NW + TURNS - 1) / TURNS, PLACES = EACH < SPOTS ? EACH : SPOTS;
#pragma unroll
                        for (int i = 0; i < EACH; ++i) {
                            const int f = (ta - HALF) * EACH + i;
                            if (TWICE && ta >= HALF && ta < MT - 1 && f < NW && tw == NW - PLACES + i * PLACES / EACH) wf[W_SETS - 1][f] = read_w(w_next, f);
                        }
                    }
                    if (ta == MT - 1) wf[0][tw] = TWICE ? wf[W_SETS - 1][tw] : read_w(w_next, tw);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (ta == 0) load_next(fast);
            }
#pragma unroll
            for (int q = 0; q < SIDES; ++q) sw[0][q] = sw[1][q];
            sat = next_sat, buf ^= 1, a_lo = a_next, w_lo = w_next;
        };
        int t = 0;
#pragma unroll 1
        for (const int fast = steps - 2 - (left != 0); t < fast; ++t) step(t, std::true_type{});
#pragma unroll 1
        for (; t < steps; ++t) step(t, std::false_type{});

        // the end: a lane has runs of neighbouring columns of the wave's, of a row for each ta
        constexpr int P = WHOLE ? 4 : 8, PIECES = OWN / 4 / P;                   // columns of a piece, of which there are all or none
        int tm, tn;
        tiles.place(tile, tm, tn);
        const int64_t m0 = (int64_t)tm * TM;
        const int n0 = tn * COLS, lane_end = lane_now(), r = lane_end % 16, g = lane_end / 16;
        // the last products' sums are there for from_sum, and for what reads them where they are
        if constexpr (TWICE) asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
        else
            asm volatile("s_nop 15\n\ts_nop 15"
                         : "+v"(acc[0][MT - 1]), "+v"(acc[1][MT - 1]), "+v"(acc[2][MT - 1]), "+v"(acc[3][MT - 1]), "+v"(acc[4][MT - 1]), "+v"(acc[5][MT - 1]), "+v"(acc[6][MT - 1]),
                           "+v"(acc[7][MT - 1]));
        // the first column of piece i
        auto column = [&](int i) { return n0 + wn * OWN + i * P / 16 * 64 + w_row<RUN>(i * P % 16 / 4, g * 4); };
        const int64_t row0 = m0 + wm * MT * 16 + r;
        constexpr int ESZ = WHOLE ? 4 : 2;
        // A row's residual is asked for a turn before it is added.  As built that gains little: the reads stand in branches of their own, the additions in those of the
        // stores, and the compiler has each store of a turn wait for all that is under way, the stores before it and the next tile's codes among it.
        q8_u4 res[RES ? 2 : 1][PIECES] = {};
        const char *res_at = RES ? (const char *)c.residual + (row0 * c.residual_stride + column(0)) * ESZ : nullptr;
        auto read_residual = [&](int ta) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
                if (row0 + ta * 16 < c.m && column(i) < c.n) res[RES ? ta % 2 : 0][i] = *(const q8_u4 *)(res_at + (column(i) - column(0)) * ESZ);
            res_at += 16 * c.residual_stride * ESZ;
        };
        if constexpr (RES) read_residual(0);
        char *out = CODES ? (char *)c.q.codes + row0 * c.q.stride + column(0) : (char *)c.out + (row0 * c.out_stride + column(0)) * ESZ;
        const int64_t out_step = 16 * (CODES ? c.q.stride : c.out_stride * ESZ);
        // The tile's last columns are none.  (Without bias and residual what stands there is the last one's value once more.)
        const bool cut = n0 + COLS > c.n && (!GATE || RES);
#pragma unroll
        for (int ta = 0; ta < MT; ++ta) {
            const bool live = row0 + ta * 16 < c.m;
            if (RES && ta + 1 < MT) read_residual(ta + 1);
            float z[PIECES][P];
#pragma unroll
            for (int tw = 0; tw < PIECES * P / 4; ++tw) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float &v = z[(tw * 4 + e) / P][(tw * 4 + e) % P];
                    v = TWICE ? from_sum(acc[tw][ta][e]) : acc[tw][ta][e];
                    if constexpr (GATE) v = silu<WHOLE>(v) * (TWICE ? from_sum(acc[4 + tw][ta][e]) : acc[4 + tw][ta][e]);
                }
            }
            // (read again for every 16 rows, and waited for together with all that is under way; kept for a tile it would take PIECES * P registers more)
            if (!GATE && c.bias) {
#pragma unroll
                for (int i = 0; i < PIECES; ++i) {
                    q8_u4 b = {};
                    if (column(i) < c.n) b = *(const q8_u4 *)((const char *)c.bias + (int64_t)column(i) * ESZ);
#pragma unroll
                    for (int e = 0; e < P; ++e) z[i][e] += value_of<WHOLE>(b, e);
                }
            }
            if (!GATE && c.act == Q8_ACT_RELU) {
#pragma unroll
                for (int i = 0; i < PIECES; ++i)
#pragma unroll
                    for (int e = 0; e < P; ++e) z[i][e] = z[i][e] < 0.f ? 0.f : z[i][e];
            }
            if constexpr (RES) {
#pragma unroll
                for (int i = 0; i < PIECES; ++i)
#pragma unroll
                    for (int e = 0; e < P; ++e) z[i][e] += value_of<WHOLE>(res[ta % 2][i], e);
            }
            if constexpr (!CODES) {
#pragma unroll
                for (int i = 0; i < PIECES; ++i)
                    if (live && column(i) < c.n) store_values<WHOLE>(out, column(i) - column(0), z[i]);
            } else {
                if (cut) {
#pragma unroll
                    for (int i = 0; i < PIECES; ++i)
#pragma unroll
                        for (int e = 0; e < P; ++e) z[i][e] = column(i) < c.n ? z[i][e] : 0.f;
                }
                uint32_t top = 0;
#pragma unroll
                for (int i = 0; i < PIECES; ++i)
#pragma unroll
                    for (int e = 0; e < P; e += 2) top = max(max(top, q8_magnitude(z[i][e])), q8_magnitude(z[i][e + 1]));
                top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
                top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
                constexpr int SHARE = Q8_BLOCK / OWN;
                if constexpr (SHARE == 2) {     // the other half of a scale's 128 columns is the neighbouring wave's
                    const int at = (wm * MT + ta) * 16 + r;
                    if (g == 0) s_top[wn][at] = top;
                    __syncthreads();
                    top = max(s_top[0][at], s_top[1][at]);
                }
                const uint32_t byte = q8_scale_byte(top);
                const float unit = q8_unit(top, byte);
#pragma unroll
                for (int q = 0; q < PIECES * P / 16; ++q) {
                    const int col = column(q * 16 / P);
                    q8_u4 u;
#pragma unroll
                    for (int i = 0; i < 4; ++i) u[i] = q8_codes4(&z[(q * 16 + i * 4) / P][i * 4 % P], unit);
                    if (live && col + 16 <= c.n) *(q8_u4 *)(out + (col - column(0))) = u;
                    else if (live && col < c.n) *(q8_u2 *)(out + (col - column(0))) = q8_u2{u[0], u[1]};
                }
                if (wn % SHARE == 0 && g == 0 && live && column(0) < c.n) c.q.scales[(row0 + ta * 16) * c.q.scale_stride + column(0) / Q8_BLOCK] = (uint8_t)byte;
            }
            out += out_step;
        }
    }
    wait_vmcnt<0>();        // what was asked for behind the end has come before this block's LDS is another's
}

template <int WM, int MT, int NG, bool GATE, bool WHOLE> hipError_t go(const Q8LinearCall &c, int units, hipStream_t s)
{
    constexpr int TM = 16 * WM * MT, COLS = (GATE ? 64 : 128) * NG;
    const int tiles_m = (c.m + TM - 1) / TM, tiles_n = (c.n + COLS - 1) / COLS;
    const int64_t total = (int64_t)tiles_m * tiles_n;
    const dim3 grid((unsigned)(std::min<int64_t>((total + 7) / 8, std::max(units / 8, 1)) * 8)), block(128 * WM);
    if (c.out && c.residual) k_q8_many<WM, MT, NG, GATE, WHOLE, false, true><<<grid, block, 0, s>>>(c, tiles_m, tiles_n);
    else if (c.out) k_q8_many<WM, MT, NG, GATE, WHOLE, false, false><<<grid, block, 0, s>>>(c, tiles_m, tiles_n);
    else if (c.residual) k_q8_many<WM, MT, NG, GATE, WHOLE, true, true><<<grid, block, 0, s>>>(c, tiles_m, tiles_n);
    else k_q8_many<WM, MT, NG, GATE, WHOLE, true, false><<<grid, block, 0, s>>>(c, tiles_m, tiles_n);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_q8_linear(const Q8LinearCall &c, int n_cu, hipStream_t s)
{
    const bool gate = c.act == Q8_ACT_GATE;
    const Q8Form f = q8_form(c, n_cu);
    if (f.few) return launch_q8_few(c, f.rows / 16, s);
    if (c.f32) return gate ? go<2, 4, 2, true, true>(c, n_cu, s) : go<2, 4, 1, false, true>(c, 2 * n_cu, s);
    if (gate) return f.rows == 256 ? go<4, 4, 2, true, false>(c, n_cu, s) : go<2, 4, 2, true, false>(c, n_cu, s);
    return f.rows == 256 ? go<2, 8, 2, false, false>(c, n_cu, s) : go<2, 4, 1, false, false>(c, 2 * n_cu, s);
}

}  // namespace aif
