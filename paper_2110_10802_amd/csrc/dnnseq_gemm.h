// Tiled matrix product on 16-bit operands for the linear layers (device code).
//
// out[q][p] = sum_c P(p,c) Q(q,c): p runs along the contiguous dimension of the output, q along its
// rows, c is contracted.  Each operand lies in memory in one of two ways:
//   along  the contraction is its contiguous dimension (rows p or q, ld elements apart): x and w in
//          the forward product, dy in the data gradient
//   across the contraction runs over its rows (ld elements apart): w in the data gradient, both
//          operands of the weight gradient
// A step takes 64 elements of the contraction, in two halves of 32.  Both tiles go from memory straight into LDS, 16
// bytes per lane; what lies past the operand's end arrives as zeros (a bounded buffer, lanes past a
// row's end sent out of bounds).  LDS holds rows of 128 bytes (along: whole lines of the caches) or TILE * 2 bytes (across) as
// memory has them, 16-byte units permuted within a row so that the reads meet the 64 banks evenly:
//   along   unit u of row r at u ^ (r & 7); a lane reads 8 consecutive c of its row (ds_read_b128)
//   across  unit pair v of row c at v ^ ((c & 3) | (c >> 3 & 1) << 2); two transposing reads give a
//           lane 8 consecutive c of its column
// The products are v_mfma_f32_16x16x32 with P as the matrix rows, so a lane ends with four
// consecutive p of one q: packed stores.
#pragma once
#include "dnnseq_dev.h"

namespace dsq {

constexpr int kStep = 64; // elements of the contraction per step

template <bool ACROSS, int TILE>
struct Tile {
    static_assert(!ACROSS || TILE >= 128, "the permutation takes eight unit pairs to a row");
    static constexpr int kRows = ACROSS ? kStep : TILE;
    static constexpr int kUnits = ACROSS ? TILE / 8 : kStep / 8; // 16-byte units per row
    static constexpr int kBytes = TILE * kStep * 2;
    static __device__ __forceinline__ int swizzle(int row)
    {
        return ACROSS ? ((row & 3) | (row >> 1 & 4)) << 1 : row & 7;
    }
};

// Loads of one operand: the parts that do not change from step to step.
template <bool ACROSS, int TILE, int THREADS>
struct Loader {
    typedef Tile<ACROSS, TILE> L;
    static constexpr int kLoads = L::kBytes / 16 / THREADS;
    const char *base; // of the step's tile
    int64_t step;     // bytes from one step to the next
    uint32_t off[kLoads];
    uint32_t ld;      // bytes from row to row
    int limit;        // rows of the operand from the tile's start (along)
    int width;        // contiguous elements from the tile's start (across)
    __device__ __forceinline__ void init(const void *p, int64_t ld_elems, int first, int extent, int c0)
    {
        ld = (uint32_t)ld_elems * 2;
        limit = min(extent - first, TILE);
        width = limit;
        if (ACROSS) {
            base = (const char *)p + ((int64_t)c0 * ld_elems + first) * 2;
            step = (int64_t)ld_elems * (kStep * 2);
        } else {
            base = (const char *)p + ((int64_t)first * ld_elems + c0) * 2;
            step = kStep * 2;
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int id = i * THREADS + (int)threadIdx.x, row = id / L::kUnits;
            const int unit = id % L::kUnits ^ L::swizzle(row);
            off[i] = row * ld + unit * 16;
            if (ACROSS && unit * 8 >= width)
                off[i] = kNowhere;
        }
    }
    // left: elements of the contraction from this step's start; none: no memory is read.  ONCE: no other
    // workgroup reads the operand, it passes by the caches
    template <bool ONCE>
    __device__ __forceinline__ void load(char *lds, int left)
    {
        const int rows = ACROSS ? min(left, kStep) : limit;
        const int last = (ACROSS ? width : min(left, kStep)) * 2;
        const auto r = buffer(base, ((uint32_t)(rows - 1) * ld + last) & (0u - (uint32_t)(left > 0)));
        const uint32_t w0 = wave_id() * (kWave * 16);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            uint32_t o = off[i];
            if (!ACROSS) { // a row's end inside the step
                const int id = i * THREADS + (int)threadIdx.x;
                const int unit = id % L::kUnits ^ L::swizzle(id / L::kUnits);
                o = unit * 8 < left ? o : kNowhere;
            }
            if (ONCE)
                load_lds_once(r, lds + i * (THREADS * 16) + w0, o);
            else
                load_lds(r, lds + i * (THREADS * 16) + w0, o);
        }
        base += step;
    }
};

// Fragments of 16 rows (p or q) x 32 c from a tile in LDS.
template <bool ACROSS, int TILE>
struct Reader {
    uint32_t off[ACROSS ? 8 : 1];
    __device__ __forceinline__ void init(int first)
    {
        const int lane = threadIdx.x % kWave, i = lane % 16, g = lane / 16;
        if (ACROSS) {
#pragma unroll
            for (int f = 0; f < 8; ++f) {
                const int pair = first / 16 + f, s = i / 4 | (g & 1) << 2;
                off[f] = (g * 8 + i / 4) * (TILE * 2) + ((pair & ~7) | ((pair & 7) ^ s)) * 32 + i % 4 * 8;
            }
        } else {
            off[0] = (first + i) * 128 + (g ^ (i & 7)) * 16;
        }
    }
    // fragment f (rows first + 16 f ..) of half kk
    __device__ __forceinline__ u32x4 get(const char *lds, int f, int kk) const
    {
        if (ACROSS) {
            const char *p = lds + off[f & 7] + (f >> 3) * 256 + kk * (32 * TILE * 2);
            return join(read_tr((const uint16_t *)p), read_tr((const uint16_t *)(p + 4 * TILE * 2)));
        }
        return *(const u32x4 *)(lds + (off[0] ^ (kk * 64)) + f * (16 * 128));
    }
};

} // namespace dsq
