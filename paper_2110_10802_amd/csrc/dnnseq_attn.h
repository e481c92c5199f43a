// What the attention kernels share (device code).
//
// Tiles of 64 rows (keys, or queries in the pass over dk and dv) x RS elements (the head's dimension
// filled up to 64 or 128 with zeros) go from memory straight into LDS; rows past the request's length
// and units past the dimension arrive as zeros, whatever memory holds there.  The 32x32x16 matrix
// instructions take a tile in two ways:
//   along   its rows are matrix rows, the dimension is contracted: 16 consecutive bytes per lane
//   across  its rows are contracted, the dimension gives the matrix rows: two transposing reads
// A product whose result has (tile row, own row) as (matrix row, column) leaves lane l = 32 h + c with
// the rows 8 (r/4) + 4 h + r % 4 of column c in register r.  Registers 8 m .. 8 m + 7, packed, are the
// column operand of a product that contracts rows 16 m .. 16 m + 15, with the rows in the order
// 4 h + {0..3}, 8 + 4 h + {0..3}: the across reads use the same order, so probabilities and score
// gradients go from one product into the next without leaving their lane.
#pragma once
#include "dnnseq_dev.h"

namespace dsq {

constexpr int kTileRows = 64;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// The 16-byte unit of row `row` at which unit u is kept: both kinds of reads meet 64 banks evenly.
template <int RS>
__device__ __forceinline__ int unit_swizzle(int row)
{
    return RS == 128 ? (row & 3) << 2 | (row >> 2 & 1) : (row >> 1 & 1) << 2 | (row >> 2 & 1);
}

// Loads of tiles of one tensor (one head of one request).
template <int RS, int THREADS>
struct TileLoader {
    static constexpr int kUnits = RS / 8, kLoads = kTileRows * kUnits / THREADS;
    static constexpr int kBytes = kTileRows * RS * 2;
    const char *base;
    uint32_t pitch, width; // bytes
    uint32_t off[kLoads];
    __device__ __forceinline__ void init(const void *p, int64_t token, int dim)
    {
        base = (const char *)p;
        pitch = (uint32_t)token * 2;
        width = dim * 2;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int id = i * THREADS + (int)threadIdx.x, row = id / kUnits;
            const int unit = id % kUnits ^ unit_swizzle<RS>(row);
            off[i] = unit * 8 < dim ? row * pitch + unit * 16 : kNowhere;
        }
    }
    // rows first .. of `rows` rows in all
    __device__ __forceinline__ void load(char *lds, int first, int rows) const
    {
        const int n = min(rows - first, kTileRows);
        const auto r = buffer(base + (int64_t)first * pitch, n > 0 ? (n - 1) * pitch + width : 0);
        const uint32_t w0 = wave_id() * (kWave * 16);
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            load_lds(r, lds + i * (THREADS * 16) + w0, off[i]);
    }
};

// Rows 32 b .. 32 b + 31, elements 16 s .. 16 s + 15.
template <int RS>
struct AlongReader {
    uint32_t off;
    uint32_t flip;
    __device__ __forceinline__ void init()
    {
        const int lane = threadIdx.x % kWave, row = lane % 32;
        off = row * (RS * 2);
        flip = (lane / 32 ^ unit_swizzle<RS>(row)) * 16;
    }
    __device__ __forceinline__ u32x4 get(const char *lds, int b, int s) const
    {
        return *(const u32x4 *)(lds + off + (flip ^ (s * 32)) + b * (32 * RS * 2));
    }
};

// Contracted rows 16 m .. 16 m + 15 in the order above, elements 32 e .. 32 e + 31.
template <int RS>
struct AcrossReader {
    uint32_t off, flip;
    __device__ __forceinline__ void init()
    {
        const int lane = threadIdx.x % kWave, i = lane % 16, row = lane / 32 * 4 + i / 4;
        off = row * (RS * 2) + i % 2 * 8;
        flip = ((lane / 16 % 2 * 2 + i % 4 / 2) ^ unit_swizzle<RS>(row)) * 16;
    }
    __device__ __forceinline__ u32x4 get(const char *lds, int m, int e) const
    {
        const char *p = lds + off + (flip ^ (e * 64)) + m * (16 * RS * 2);
        return join(read_tr((const uint16_t *)p), read_tr((const uint16_t *)(p + 8 * RS * 2)));
    }
};

// A lane's own row as a column operand: elements 16 s + 8 (lane / 32) .. + 7; zeros outside.
__device__ __forceinline__ u32x4 own_fragment(const uint16_t *row, bool inside, int dim, int s)
{
    const int c = 16 * s + (threadIdx.x % kWave) / 32 * 8;
    return inside && c < dim ? *(const u32x4 *)(row + c) : u32x4{0, 0, 0, 0};
}

// Maximum and sum of a lane's value and that of lane ^ 32, the same bits in both (a swap of a value
// with itself leaves the lower half's in one register and the upper half's in the other).
__device__ __forceinline__ float halves_max(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float halves_sum(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// The same over the four lanes that share lane % 16.
__device__ __forceinline__ float quarters_max(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return halves_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float quarters_sum(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return halves_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

__device__ __forceinline__ int clamp_len(const int32_t *lens, int b, int top)
{
    return lens ? min(max(lens[b], 0), top) : top;
}

// Workgroup -> work item: each of the eight XCDs (workgroup b runs on XCD b % 8) gets a run of
// consecutive items, so the items that read the same keys share an L2.
__device__ __forceinline__ uint32_t xcd_order(uint32_t b, uint32_t n)
{
    const uint32_t x = b % 8, each = n / 8, more = n % 8;
    return x * each + min(x, more) + b / 8;
}

} // namespace dsq
