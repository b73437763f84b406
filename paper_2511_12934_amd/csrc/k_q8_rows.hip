// Rows summed, normalised and left in 8 bits (include/aif_q8.h: aif_q8_rows).
//
// A row lies in the registers of LPR lanes, V pieces of 8 values each, so that it is read once whatever comes of it; a scale's
// 128 columns are 16 neighbouring lanes.  h and y are formed in 64 bits -- the vector unit's rate is that of 32 -- and left in
// 32 with the last bit set where more followed (q8_odd), from which each output is rounded as from y itself: the codes are
// those of the formula but for its last bits in 64.
//
// Memory bounds it where rows are many: 200000 rows of 1024 in bf16 with residual, sum and codes take 289 us, 4.96 TB/s, where a copy of 1 GB reaches 5.2;
// 25000 x 8192 315 us, fp32 100000 x 1024 243 us (5.46 TB/s).  The vector instructions, 41 a value there, take three quarters of that time beside it, at 256 and
// 512 columns 57 a value: 32000 x 256 17.4 us, half of them instructions, 32000 x 512 30, seven tenths (two divisions and a root a lane, the weight once more for every
// row).  A block has asked for its next rows before it works on these (as many blocks as rows: 200000 x 1024 314 us, 25000 x 8192 384) where a grid of 2^21
// threads goes round (2^19: 300 us): not below, where each takes one turn.  One row of 1024 takes 2.8 us.
#include "k_q8.h"

#include <algorithm>

namespace aif {

namespace {

// The value in 32 bits, of which 21 are the first ones of d and the last says whether d has more: rounding that to 20 bits or
// fewer is rounding d.  (Below 2^-126 and above 2^128 as the conversion has it.)
__device__ __forceinline__ float q8_odd(double d)
{
    const uint32_t lo = (uint32_t)__double2loint(d), hi = (uint32_t)__double2hiint(d);
    return (float)__hiloint2double((int)(hi | (lo ? 1u : 0u)), 0);
}

template <int LPR> __device__ __forceinline__ double row_sum(double s, double *lds)
{
#pragma unroll
    for (int o = 1; o < (LPR < 64 ? LPR : 64); o *= 2) s += __shfl_xor(s, o, 64);
    if constexpr (LPR > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
        __syncthreads();
        s = 0;
        const int first = threadIdx.x / LPR * (LPR / 64);
#pragma unroll
        for (int i = 0; i < LPR / 64; ++i) s += lds[first + i];
        __syncthreads();
    }
    return s;
}

// Eight neighbouring values of a row as they lie in memory, zeros from the row's end on.
template <class T> struct Eight {
    q8_u4 u[sizeof(T) / 2];
};

template <class T> __device__ __forceinline__ Eight<T> load8(const T *p, int valid)
{
    Eight<T> x = {};
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i)
        if (valid > 4 * i) x.u[i] = *(const q8_u4 *)(p + 4 * i);
    return x;
}

template <class T> __device__ __forceinline__ double value8(const Eight<T> &x, int i)
{
    if constexpr (sizeof(T) == 2) return (double)q8_bf16(i % 2 ? x.u[0][i / 2] >> 16 : x.u[0][i / 2] & 0xffffu);
    else return (double)__uint_as_float(x.u[i / 4][i % 4]);
}

template <class T> __device__ __forceinline__ void read8(const T *p, int valid, double (&v)[8])
{
    const Eight<T> x = load8(p, valid);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = value8(x, i);
}

template <class T> __device__ __forceinline__ void write8(T *p, int valid, const double (&v)[8])
{
    if constexpr (sizeof(T) == 2) {
        if (valid <= 0) return;
        q8_u4 u;
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = q8_two_bf16(q8_odd(v[2 * i]), q8_odd(v[2 * i + 1]));
        *(q8_u4 *)p = u;
    } else {
        if (valid > 0) *(q8_f4 *)p = q8_f4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
        if (valid > 4) *(q8_f4 *)(p + 4) = q8_f4{(float)v[4], (float)v[5], (float)v[6], (float)v[7]};
    }
}

template <class T, int LPR, int V, int THREADS> __global__ __launch_bounds__(THREADS, sizeof(T) == 2 && THREADS >= 512 ? 4 : 1) void k_q8_rows(const Q8RowsCall c)
{
    __shared__ double lds[THREADS / 64];
    constexpr int RPB = THREADS / LPR;
    const int lane = threadIdx.x % LPR;
    const int64_t rounds = ((int64_t)c.n_rows + RPB - 1) / RPB;
    Eight<T> x[V], res[V];
    auto ask = [&](int64_t b) __attribute__((always_inline)) {
        const int64_t row = b * RPB + threadIdx.x / LPR;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = (v * LPR + lane) * 8, valid = row < c.n_rows ? c.width - col : 0;
            x[v] = load8((const T *)c.x + row * c.x_stride + col, valid);
            if (c.residual) res[v] = load8((const T *)c.residual + row * c.residual_stride + col, valid);
        }
    };
    ask(blockIdx.x);
    for (int64_t b = blockIdx.x; b < rounds; b += gridDim.x) {
        const int64_t row = b * RPB + threadIdx.x / LPR;
        const bool live = row < c.n_rows;
        double h[V][8], sum = 0;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) h[v][i] = c.residual ? value8(x[v], i) + value8(res[v], i) : value8(x[v], i);
        ask(b + gridDim.x);
#pragma unroll
        for (int v = 0; v < V; ++v) {
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = __builtin_fma(h[v][i], h[v][i], sum);
        }
        double r = 1.0;
        if (c.norm) {
            sum = row_sum<LPR>(sum, lds);
            r = 1.0 / __builtin_sqrt(sum / c.width + (double)c.eps);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = (v * LPR + lane) * 8, valid = live ? c.width - col : 0;
            if (c.sum_out) write8((T *)c.sum_out + row * c.sum_stride + col, valid, h[v]);
            if (c.norm) {
                double w[8];
                if (c.weight) read8((const T *)c.weight + col, valid, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[v][i] = c.weight ? h[v][i] * r * w[i] : h[v][i] * r;
            }
            if (c.out) write8((T *)c.out + row * c.out_stride + col, valid, h[v]);
            if (c.q.codes) {
                float y[8];
                uint32_t top = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = q8_odd(h[v][i]), top = max(top, q8_magnitude(y[i]));
#pragma unroll
                for (int o = 1; o < 16; o *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
                const uint32_t byte = q8_scale_byte(top);
                const float unit = q8_unit(top, byte);
                if (valid > 0) {
                    *(q8_u2 *)(c.q.codes + row * c.q.stride + col) = q8_u2{q8_codes4(y, unit), q8_codes4(y + 4, unit)};
                    if (col % Q8_BLOCK == 0) c.q.scales[row * c.q.scale_stride + col / Q8_BLOCK] = (uint8_t)byte;
                }
            }
        }
    }
}

constexpr int ROWS_THREADS = 1 << 21;       // of all blocks of k_q8_rows
constexpr int MAX_GRID = 1 << 21;           // blocks go round where there is more

template <class T, int LPR, int V> hipError_t go(const Q8RowsCall &c, hipStream_t s)
{
    constexpr int THREADS = LPR > 256 ? LPR : 256, RPB = THREADS / LPR;
    const int64_t blocks = std::min<int64_t>(((int64_t)c.n_rows + RPB - 1) / RPB, ROWS_THREADS / THREADS);
    k_q8_rows<T, LPR, V, THREADS><<<dim3((unsigned)blocks), dim3(THREADS), 0, s>>>(c);
    return hipGetLastError();
}

// Lanes of a row: 64 hold 1024 columns without a barrier; where rows are too few for the device, more of them take one in less time (one row of 1024: 128
// lanes 2.8 us, 64 3.7; 32000 rows: 65 and 58; of 4096: 512 lanes 3.7 us, 256 4.2; 50000 rows 381 and 367).  Two waves more a unit are worth the few registers they cost with 8192
// columns of bf16 (315 us, without 406), not with fp32 (603, without 531).  Above 8192 columns 1024 threads leave 128 registers, of which fp32 wants two more (10000 x 16384
// 409 us, 5.2 TB/s).  A width just above 1024, 2048, 4096 or 8192 leaves nearly half of the lanes without columns: 100000 x 1040 301 us (x 1024 147), 100000 x 2064 511
// (x 2048 322), 50000 x 4112 477 (x 4096 294), 25000 x 8208 573 (x 8192 314).
template <class T> hipError_t rows(const Q8RowsCall &c, hipStream_t s)
{
    const int w = c.width;
    if (w <= 128) return go<T, 16, 1>(c, s);
    if (w <= 256) return go<T, 32, 1>(c, s);
    if (w <= 512) return go<T, 64, 1>(c, s);
    if (w <= 1024) return c.n_rows <= 1024 ? go<T, 128, 1>(c, s) : go<T, 64, 2>(c, s);
    if (w <= 2048) return go<T, 256, 1>(c, s);
    if (w <= 4096) return c.n_rows <= 256 ? go<T, 512, 1>(c, s) : go<T, 256, 2>(c, s);
    if (w <= 8192) return go<T, 512, 2>(c, s);
    return go<T, 1024, 2>(c, s);
}

// A block of a matrix, BLOCK_ROWS by 128, brought into 8 bits by 256 threads: 16 of them take 128 columns of a row.  A layer's 16384 x 16384 in bf16 173 us (4.65 TB/s, the
// rows read once from memory and once more from the caches), 4096 x 4096 11.2 us, in fp32 23; by rows 200000 x 1024 in bf16 122 us (5.0 TB/s), in fp32 189 (5.4).
template <class T, int BLOCK_ROWS> __global__ __launch_bounds__(256) void k_q8_weights(const Q8ConvertCall c)
{
    __shared__ uint32_t tops[4];
    const int across = (c.width + Q8_BLOCK - 1) / Q8_BLOCK;
    constexpr int ROWS = BLOCK_ROWS == 1 ? 16 : 128;        // of a unit: 16 blocks of a row, or one of 128
    const int64_t units = ((int64_t)c.n_rows + ROWS - 1) / ROWS * across;
    for (int64_t b = blockIdx.x; b < units; b += gridDim.x) {
        const int64_t row0 = b / across * ROWS;
        const int col = (int)(b % across) * Q8_BLOCK + threadIdx.x % 16 * 8;
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < ROWS; i += 16) {
            const int64_t row = row0 + i + threadIdx.x / 16;
            double x[8];
            read8((const T *)c.rows + row * c.stride + col, row < c.n_rows ? c.width - col : 0, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, q8_magnitude((float)x[e]));
        }
#pragma unroll
        for (int o = 1; o < (BLOCK_ROWS == 1 ? 16 : 64); o *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
        if constexpr (BLOCK_ROWS > 1) {
            if (threadIdx.x % 64 == 0) tops[threadIdx.x / 64] = top;
            __syncthreads();
            top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
            __syncthreads();
        }
        const uint32_t byte = q8_scale_byte(top);
        const float unit = q8_unit(top, byte);
#pragma unroll
        for (int i = 0; i < ROWS; i += 16) {
            const int64_t row = row0 + i + threadIdx.x / 16;
            if (row >= c.n_rows || col >= c.width) continue;
            double x[8];
            float y[8];
            read8((const T *)c.rows + row * c.stride + col, c.width - col, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = (float)x[e];
            *(q8_u2 *)(c.q.codes + row * c.q.stride + col) = q8_u2{q8_codes4(y, unit), q8_codes4(y + 4, unit)};
            if (BLOCK_ROWS == 1 && col % Q8_BLOCK == 0) c.q.scales[row * c.q.scale_stride + col / Q8_BLOCK] = (uint8_t)byte;
        }
        if (BLOCK_ROWS > 1 && threadIdx.x == 0) c.q.scales[row0 / BLOCK_ROWS * c.q.scale_stride + col / Q8_BLOCK] = (uint8_t)byte;
    }
}

// Values of codes and scales: a thread takes eight columns of a row.  200000 x 1024 to bf16 106 us (5.8 TB/s), to fp32 175.
template <class T> __global__ __launch_bounds__(256) void k_q8_values(const Q8ConvertCall c)
{
    const int pieces = c.width / 8;
    const int64_t all = (int64_t)c.n_rows * pieces, step = (int64_t)gridDim.x * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += step) {
        const int64_t row = i / pieces;
        const int col = (int)(i % pieces) * 8;
        const q8_u2 codes = *(const q8_u2 *)(c.q.codes + row * c.q.stride + col);
        const float unit = __uint_as_float((uint32_t)c.q.scales[row / c.block_rows * c.q.scale_stride + col / Q8_BLOCK] << 23);
        T *to = (T *)c.rows + row * c.stride + col;
        float v[8];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int u = (int)codes[e];
            v[4 * e] = __builtin_amdgcn_cvt_f32_fp8(u, 0) * unit, v[4 * e + 1] = __builtin_amdgcn_cvt_f32_fp8(u, 1) * unit;
            v[4 * e + 2] = __builtin_amdgcn_cvt_f32_fp8(u, 2) * unit, v[4 * e + 3] = __builtin_amdgcn_cvt_f32_fp8(u, 3) * unit;
        }
        if constexpr (sizeof(T) == 2) {
            q8_u4 u;
#pragma unroll
            for (int f = 0; f < 4; ++f) u[f] = q8_two_bf16(v[2 * f], v[2 * f + 1]);
            *(q8_u4 *)to = u;
        } else {
            *(q8_f4 *)to = q8_f4{v[0], v[1], v[2], v[3]};
            *(q8_f4 *)(to + 4) = q8_f4{v[4], v[5], v[6], v[7]};
        }
    }
}

}  // namespace

hipError_t launch_q8_rows(const Q8RowsCall &c, hipStream_t s) { return c.f32 ? rows<float>(c, s) : rows<uint16_t>(c, s); }

hipError_t launch_q8_weights(const Q8ConvertCall &c, hipStream_t s)
{
    const int64_t per = c.block_rows == 1 ? 16 : 128;
    const int64_t units = (c.n_rows + per - 1) / per * ((c.width + Q8_BLOCK - 1) / Q8_BLOCK);
    const dim3 grid((unsigned)std::min<int64_t>(units, MAX_GRID)), block(256);
    if (c.block_rows == 1) {
        if (c.f32) k_q8_weights<float, 1><<<grid, block, 0, s>>>(c);
        else k_q8_weights<uint16_t, 1><<<grid, block, 0, s>>>(c);
    } else {
        if (c.f32) k_q8_weights<float, 128><<<grid, block, 0, s>>>(c);
        else k_q8_weights<uint16_t, 128><<<grid, block, 0, s>>>(c);
    }
    return hipGetLastError();
}

hipError_t launch_q8_values(const Q8ConvertCall &c, hipStream_t s)
{
    const int64_t all = (int64_t)c.n_rows * (c.width / 8);
    const dim3 grid((unsigned)std::min<int64_t>((all + 255) / 256, MAX_GRID)), block(256);
    if (c.f32) k_q8_values<float><<<grid, block, 0, s>>>(c);
    else k_q8_values<uint16_t><<<grid, block, 0, s>>>(c);
    return hipGetLastError();
}

}  // namespace aif
