// Attention backward on 16-bit tensors: the probabilities are computed again from q, k and lse.
//   p = exp(s - lse), dp = dout v^T, ds = p (dp - delta), delta = rowsum(dout o)
//   dq = scale ds k,  dk = scale ds^T q,  dv = p^T dout
// Two passes, each with one owner for every output element, so nothing is added atomically: seven
// products instead of the five of a single pass.
//
//   attn_delta  delta of every row (and, for fp16, the factor that keeps ds in range)
//   attn_dkv    128 keys per workgroup, 32 per wavefront (columns of s = q k^T): walks the query rows
//               of the key head's group in tiles of 64; p and ds come out as the column operands of
//               dv^T += dout^T p and dk^T += q^T ds
//   attn_dq     128 rows per workgroup, 32 per wavefront (columns of s^T = k q^T): walks the keys;
//               ds^T is the column operand of dq^T += k^T ds^T
//
// fp16: ds has entries of the size of dp / keys, which fp16 may not hold.  All of them are multiplied
// by one power of two c, taken from max |dout_i| max |v_j| >= max |dp|, and dq and dk divided by it.
#include "dnnseq_attn.h"
#include "dnnseq_launch.h"

#include <algorithm>

namespace dsq {
namespace {

struct Backward {
    const uint16_t *q, *k, *v, *o, *dout;
    const float *lse;
    const int32_t *q_lens, *kv_lens;
    uint16_t *dq, *dk, *dv;
    dnnseq_stride sq, sk, sv, so, sdo, sdq, sdk, sdv;
    int batch, q_heads, kv_heads, group, q_len, kv_len, dim, causal;
    float scale, scale2;
    float *delta;    // [batch][q_heads][q_len]
    float *bound;    // fp16: [bounds] squares of row norms, their maxima per workgroup (dout, then v)
    int bounds_q, bounds_v;
    int head_splits; // workgroups that share the heads of a group in attn_dkv
    float *part;     // [head_splits][dk, dv][batch][kv_heads][kv_len][dim]
};

__device__ __forceinline__ int64_t row_offset(const dnnseq_stride &s, int b, int head, int token)
{
    return b * s.batch + head * s.head + token * s.token;
}

// 16 lanes to a row; rows of dout first (delta and norm), then, for fp16, rows of v (norm).
template <class T>
__global__ __launch_bounds__(256) void attn_delta_kernel(Backward a)
{
    const int lane = threadIdx.x % 16, c = lane * 8;
    const bool of_v = (int)blockIdx.x >= a.bounds_q;
    const size_t row = (size_t)(blockIdx.x - (of_v ? a.bounds_q : 0)) * 16 + threadIdx.x / 16;
    const int len = of_v ? a.kv_len : a.q_len, heads = of_v ? a.kv_heads : a.q_heads;
    float dot = 0.f, norm = 0.f;
    const bool in = row < (size_t)a.batch * heads * len;
    if (in) {
        const int t = row % len, h = row / len % heads, b = row / len / heads;
        const int top = of_v ? clamp_len(a.kv_lens, b, len) : clamp_len(a.q_lens, b, len);
        if (t < top && c < a.dim) {
            const u32x4 x = *(const u32x4 *)((of_v ? a.v + row_offset(a.sv, b, h, t) : a.dout + row_offset(a.sdo, b, h, t)) + c);
            const u32x4 y = of_v ? x : *(const u32x4 *)(a.o + row_offset(a.so, b, h, t) + c);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                dot += T::lo(x[i]) * T::lo(y[i]) + T::hi(x[i]) * T::hi(y[i]);
                norm += T::lo(x[i]) * T::lo(x[i]) + T::hi(x[i]) * T::hi(x[i]);
            }
        }
    }
    dot = mbk::row16_sum(dot);
    if (in && !of_v && lane == 0)
        a.delta[row] = dot;
    if (T::kHalf) {
        norm = mbk::row16_sum(norm);
        __shared__ float red[16];
        if (lane == 0)
            red[threadIdx.x / 16] = norm;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int i = 1; i < 16; ++i)
                norm = fmaxf(norm, red[i]);
            a.bound[blockIdx.x] = norm;
        }
    }
}

// The maxima over the workgroups of attn_delta, one number each.
__global__ __launch_bounds__(1024) void attn_bound_kernel(Backward a)
{
    const int n = blockIdx.x ? a.bounds_v : a.bounds_q;
    float *in = a.bound + (blockIdx.x ? a.bounds_q : 0), top = 0.f;
    for (int i = threadIdx.x; i < n; i += 1024)
        top = fmaxf(top, in[i]);
    __shared__ float red[16];
    for (int o = 32; o; o >>= 1)
        top = fmaxf(top, __shfl_xor(top, o, kWave));
    if (threadIdx.x % kWave == 0)
        red[threadIdx.x / kWave] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 16; ++i)
            top = fmaxf(top, red[i]);
        a.bound[a.bounds_q + a.bounds_v + blockIdx.x] = top;
    }
}

// c: |ds| <= p |dp - delta| <= 2 max|dp|; 2 max|dp| c stays below 2^15.
template <class T>
__device__ __forceinline__ float range_factor(const Backward &a)
{
    if (!T::kHalf)
        return 1.0f;
    const float *n = a.bound + a.bounds_q + a.bounds_v;
    const float top = sqrtf(n[0]) * sqrtf(n[1]);
    if (!(top > 0.f) || !(top < INFINITY))
        return 1.0f;
    const int e = 13 - (int)ceilf(__builtin_amdgcn_logf(top));
    return ldexpf(1.0f, min(max(e, -100), 100));
}

template <class T>
__device__ __forceinline__ u32x4 pack8(const f32x16 &s, int h)
{
    u32x4 p;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        p[i] = T::pack(s[8 * h + 2 * i], s[8 * h + 2 * i + 1]);
    return p;
}

// Four consecutive elements of a transposed result (register 4 i .. 4 i + 3 of block e).
template <class T, int NS>
__device__ __forceinline__ void store_row(uint16_t *row, const f32x16 (&acc)[NS], int dim, float f)
{
    const int lane = threadIdx.x % kWave;
#pragma unroll
    for (int e = 0; e < NS; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = 32 * e + 8 * i + lane / 32 * 4;
            if (d < dim)
                *(u32x2 *)(row + d) = u32x2{T::pack(acc[e][4 * i] * f, acc[e][4 * i + 1] * f),
                                            T::pack(acc[e][4 * i + 2] * f, acc[e][4 * i + 3] * f)};
        }
}
template <int NS>
__device__ __forceinline__ void store_part(float *row, const f32x16 (&acc)[NS], int dim, float f)
{
    const int lane = threadIdx.x % kWave;
#pragma unroll
    for (int e = 0; e < NS; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = 32 * e + 8 * i + lane / 32 * 4;
            if (d < dim)
                *(f32x4 *)(row + d) =
                    f32x4{acc[e][4 * i] * f, acc[e][4 * i + 1] * f, acc[e][4 * i + 2] * f, acc[e][4 * i + 3] * f};
        }
}

// ---- dk, dv --------------------------------------------------------------------------------------
// A tile of 64 query rows for 32 keys.  Row t sees keys up to t + shift.
template <class T, int NS, int RS, bool MASK>
__device__ __forceinline__ void dkv_tile(const char *__restrict__ qt, const char *__restrict__ dt,
                                         const float *__restrict__ lse2, const float *__restrict__ delta,
                                         const AlongReader<RS> &along, const AcrossReader<RS> &across,
                                         const u32x4 (&k)[2 * NS], const u32x4 (&v)[2 * NS], f32x16 (&dk)[NS],
                                         f32x16 (&dv)[NS], int t0, int key, int shift, float scale2, float c)
{
    const int half = threadIdx.x % kWave / 32;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        f32x16 s = {}, dp = {};
#pragma unroll
        for (int i = 0; i < 2 * NS; ++i)
            s = T::mma32(along.get(qt, b, i), k[i], s);
#pragma unroll
        for (int i = 0; i < 2 * NS; ++i)
            dp = T::mma32(along.get(dt, b, i), v[i], dp);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r0 = 32 * b + 8 * i + 4 * half;
            const f32x4 ls = *(const f32x4 *)(lse2 + r0), de = *(const f32x4 *)(delta + r0);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float p = __builtin_amdgcn_exp2f(fmaf(s[4 * i + j], scale2, -ls[j]));
                if (MASK)
                    p = key <= t0 + r0 + j + shift ? p : 0.f;
                s[4 * i + j] = p;
                dp[4 * i + j] = p * (dp[4 * i + j] - de[j]) * c;
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) { // p and ds are rounded to the operands' type
            const u32x4 p = pack8<T>(s, h);
#pragma unroll
            for (int e = 0; e < NS; ++e)
                dv[e] = T::mma32(across.get(dt, 2 * b + h, e), p, dv[e]);
            const u32x4 ds = pack8<T>(dp, h);
#pragma unroll
            for (int e = 0; e < NS; ++e)
                dk[e] = T::mma32(across.get(qt, 2 * b + h, e), ds, dk[e]);
        }
    }
}

template <class T, int NS>
__global__ __launch_bounds__(256, NS > 2 ? 1 : 2) void attn_dkv_kernel(Backward a)
{
    constexpr int RS = NS > 2 ? 128 : 64, KEYS = 128;
    typedef TileLoader<RS, 256> Load;
    constexpr int BUF = 2 * Load::kBytes + 2 * kTileRows * 4;
    __shared__ __attribute__((aligned(256))) char lds[2 * BUF]; // [2][q, dout, lse, delta]
    const int tiles = (a.kv_len + KEYS - 1) / KEYS;
    const uint32_t item = xcd_order(blockIdx.x, gridDim.x);
    const int hs = item % a.head_splits, tile = item / a.head_splits % tiles, unit = item / a.head_splits / tiles;
    const int b = unit / a.kv_heads, g = unit % a.kv_heads;
    const int key0 = tile * KEYS; // (the first keys are seen by most rows: they come first)
    const int ql = clamp_len(a.q_lens, b, a.q_len), kl = clamp_len(a.kv_lens, b, a.kv_len);
    const int lane = threadIdx.x % kWave, w = wave_id();
    const int key = key0 + w * 32 + lane % 32, shift = kl - ql;
    const float c = range_factor<T>(a);

    u32x4 k[2 * NS], v[2 * NS];
    const uint16_t *krow = a.k + row_offset(a.sk, b, g, key), *vrow = a.v + row_offset(a.sv, b, g, key);
#pragma unroll
    for (int i = 0; i < 2 * NS; ++i) {
        k[i] = own_fragment(krow, key < kl, a.dim, i);
        v[i] = own_fragment(vrow, key < kl, a.dim, i);
    }
    AlongReader<RS> along;
    AcrossReader<RS> across;
    along.init();
    across.init();
    f32x16 dk[NS], dv[NS];
#pragma unroll
    for (int e = 0; e < NS; ++e)
        dk[e] = dv[e] = f32x16{};

    // rows that see any key of the workgroup: t >= key0 - shift, in whole tiles
    const int t_first = a.causal ? max(0, key0 - shift) / kTileRows * kTileRows : 0;
    const int per_head = key0 < kl && ql > t_first ? (ql - t_first + kTileRows - 1) / kTileRows : 0;
    const int h0 = a.group * hs / a.head_splits, h1 = a.group * (hs + 1) / a.head_splits;
    Load lq, ld;
    const auto issue = [&](int step, char *buf) __attribute__((always_inline)) {
        const int h = g * a.group + h0 + step / per_head, t0 = t_first + step % per_head * kTileRows;
        lq.base = (const char *)(a.q + row_offset(a.sq, b, h, 0));
        ld.base = (const char *)(a.dout + row_offset(a.sdo, b, h, 0));
        lq.load(buf, t0, ql);
        ld.load(buf + Load::kBytes, t0, ql);
        // lse (base 2; +infinity where a row sees nothing: p = 0) and delta of 64 rows
        if (w == 0) {
            const size_t at = ((size_t)b * a.q_heads + h) * a.q_len;
            const int t = t0 + lane;
            const float l = t < ql ? a.lse[at + t] : -INFINITY;
            float *f = (float *)(buf + 2 * Load::kBytes);
            f[lane] = l == -INFINITY ? INFINITY : l * kLog2e;
            f[kTileRows + lane] = t < ql ? a.delta[at + t] : 0.f;
        }
    };
    lq.init(a.q, a.sq.token, a.dim);
    ld.init(a.dout, a.sdo.token, a.dim);
    const int steps = per_head * (h1 - h0);
    if (steps)
        issue(0, lds);
    for (int n = 0; n < steps; ++n) {
        __builtin_amdgcn_s_waitcnt(0x0f70); // vmcnt(0): this wavefront's part of the tile has landed
        __syncthreads();                    // and everyone's; the other buffer is no longer read
        const auto step = [&](const char *__restrict__ cur, char *__restrict__ nxt) __attribute__((always_inline)) {
            if (n + 1 < steps)
                issue(n + 1, nxt);
            const float *f = (const float *)(cur + 2 * Load::kBytes);
            const int t0 = t_first + n % per_head * kTileRows, w0 = key0 + w * 32;
            if (!a.causal || w0 + 31 <= t0 + shift)
                dkv_tile<T, NS, RS, false>(cur, cur + Load::kBytes, f, f + kTileRows, along, across, k, v, dk, dv, t0,
                                           key, shift, a.scale2, c);
            else if (w0 <= t0 + kTileRows - 1 + shift)
                dkv_tile<T, NS, RS, true>(cur, cur + Load::kBytes, f, f + kTileRows, along, across, k, v, dk, dv, t0,
                                          key, shift, a.scale2, c);
        };
        step(lds + (n & 1) * BUF, lds + (~n & 1) * BUF);
    }
    if (key >= a.kv_len)
        return;
    if (key >= kl) // (what stands there came from zeros in place of the key)
#pragma unroll
        for (int e = 0; e < NS; ++e)
            dk[e] = dv[e] = f32x16{};
    if (a.part) {
        const size_t plane = (size_t)a.batch * a.kv_heads * a.kv_len * a.dim;
        float *out = a.part + hs * 2 * plane + (((size_t)b * a.kv_heads + g) * a.kv_len + key) * a.dim;
        store_part<NS>(out, dk, a.dim, a.scale / c);
        store_part<NS>(out + plane, dv, a.dim, 1.0f);
        return;
    }
    store_row<T, NS>(a.dk + row_offset(a.sdk, b, g, key), dk, a.dim, a.scale / c);
    store_row<T, NS>(a.dv + row_offset(a.sdv, b, g, key), dv, a.dim, 1.0f);
}

// The parts of dk and dv added, eight elements per thread.
template <class T>
__global__ __launch_bounds__(256) void attn_dkv_sum_kernel(Backward a)
{
    const size_t plane = (size_t)a.batch * a.kv_heads * a.kv_len * a.dim;
    const int units = a.dim / 8;
    const size_t i = blockIdx.x * (size_t)256 + threadIdx.x;
    if (i >= plane / 8)
        return;
    f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
    for (int s = 0; s < a.head_splits; ++s) {
        const float *p = a.part + (s * 2 + blockIdx.y) * plane + i * 8;
        x += *(const f32x4 *)p;
        y += *(const f32x4 *)(p + 4);
    }
    const size_t row = i / units;
    const int key = row % a.kv_len, g = row / a.kv_len % a.kv_heads, b = row / a.kv_len / a.kv_heads;
    uint16_t *out = blockIdx.y ? a.dv + row_offset(a.sdv, b, g, key) : a.dk + row_offset(a.sdk, b, g, key);
    *(u32x4 *)(out + i % units * 8) = u32x4{T::pack(x[0], x[1]), T::pack(x[2], x[3]), T::pack(y[0], y[1]), T::pack(y[2], y[3])};
}

// ---- dq ------------------------------------------------------------------------------------------
template <class T, int NS, int RS, bool MASK>
__device__ __forceinline__ void dq_tile(const char *__restrict__ kt, const char *__restrict__ vt,
                                        const AlongReader<RS> &along, const AcrossReader<RS> &across,
                                        const u32x4 (&q)[2 * NS], const u32x4 (&d)[2 * NS], f32x16 (&dq)[NS], int key0,
                                        int limit, float lse2, float delta, float scale2, float c)
{
    const int half = threadIdx.x % kWave / 32;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        f32x16 s = {}, dp = {};
#pragma unroll
        for (int i = 0; i < 2 * NS; ++i)
            s = T::mma32(along.get(kt, b, i), q[i], s);
#pragma unroll
        for (int i = 0; i < 2 * NS; ++i)
            dp = T::mma32(along.get(vt, b, i), d[i], dp);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            float p = __builtin_amdgcn_exp2f(fmaf(s[r], scale2, -lse2));
            if (MASK)
                p = key0 + 32 * b + 8 * (r / 4) + 4 * half + r % 4 < limit ? p : 0.f;
            dp[r] = p * (dp[r] - delta) * c;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const u32x4 ds = pack8<T>(dp, h);
#pragma unroll
            for (int e = 0; e < NS; ++e)
                dq[e] = T::mma32(across.get(kt, 2 * b + h, e), ds, dq[e]);
        }
    }
}

template <class T, int NS>
__global__ __launch_bounds__(256, 2) void attn_dq_kernel(Backward a)
{
    constexpr int RS = NS > 2 ? 128 : 64, ROWS = 128;
    typedef TileLoader<RS, 256> Load;
    __shared__ __attribute__((aligned(256))) char lds[4 * Load::kBytes]; // [2][keys, values]
    const int rows = a.q_len * a.group, tiles = (rows + ROWS - 1) / ROWS;
    const uint32_t item = xcd_order(blockIdx.x, gridDim.x);
    const int unit = item / tiles, b = unit / a.kv_heads, g = unit % a.kv_heads;
    const int r0 = (tiles - 1 - item % tiles) * ROWS;
    const int ql = clamp_len(a.q_lens, b, a.q_len), kl = clamp_len(a.kv_lens, b, a.kv_len);
    const int lane = threadIdx.x % kWave, w = wave_id();
    const auto limit_of = [&](int r) {
        const int t = r / a.group;
        return r >= rows || t >= ql ? 0 : a.causal ? min(kl, t + kl - ql + 1) : kl;
    };
    const int r = r0 + w * 32 + lane % 32, limit = limit_of(r);
    const int end = limit_of(min(r0 + ROWS, ql * a.group) - 1 >= r0 ? min(r0 + ROWS, ql * a.group) - 1 : rows);
    const int wr = min(r0 + w * 32 + 32, ql * a.group) - 1;
    const int wave_end = wr >= r0 + w * 32 ? limit_of(wr) : 0;
    const int wave_free = min(limit_of(r0 + w * 32), limit_of(r0 + w * 32 + 31));
    const float c = range_factor<T>(a);

    u32x4 q[2 * NS], d[2 * NS];
    const int head = g * a.group + r % a.group, token = r / a.group;
    const bool in = r < rows && token < ql;
    const uint16_t *qrow = a.q + row_offset(a.sq, b, head, token), *drow = a.dout + row_offset(a.sdo, b, head, token);
#pragma unroll
    for (int i = 0; i < 2 * NS; ++i) {
        q[i] = own_fragment(qrow, in, a.dim, i);
        d[i] = own_fragment(drow, in, a.dim, i);
    }
    const size_t ri = ((size_t)b * a.q_heads + head) * a.q_len + token;
    const float lse = in ? a.lse[ri] : -INFINITY, delta = in ? a.delta[ri] : 0.f;
    const float lse2 = lse == -INFINITY ? INFINITY : lse * kLog2e;
    Load lk, lv;
    lk.init(a.k + row_offset(a.sk, b, g, 0), a.sk.token, a.dim);
    lv.init(a.v + row_offset(a.sv, b, g, 0), a.sv.token, a.dim);
    AlongReader<RS> along;
    AcrossReader<RS> across;
    along.init();
    across.init();
    f32x16 dq[NS];
#pragma unroll
    for (int e = 0; e < NS; ++e)
        dq[e] = f32x16{};
    if (0 < end) {
        lk.load(lds, 0, kl);
        lv.load(lds + Load::kBytes, 0, kl);
    }
    for (int k0 = 0, turn = 0; k0 < end; k0 += kTileRows, turn ^= 1) {
        __builtin_amdgcn_s_waitcnt(0x0f70); // vmcnt(0): this wavefront's part of the tile has landed
        __syncthreads();                    // and everyone's; the other buffer is no longer read
        const auto step = [&](const char *__restrict__ cur, char *__restrict__ nxt) __attribute__((always_inline)) {
            if (k0 + kTileRows < end) {
                lk.load(nxt, k0 + kTileRows, kl);
                lv.load(nxt + Load::kBytes, k0 + kTileRows, kl);
            }
            if (k0 + kTileRows <= wave_free)
                dq_tile<T, NS, RS, false>(cur, cur + Load::kBytes, along, across, q, d, dq, k0, limit, lse2, delta,
                                          a.scale2, c);
            else if (k0 < wave_end)
                dq_tile<T, NS, RS, true>(cur, cur + Load::kBytes, along, across, q, d, dq, k0, limit, lse2, delta,
                                         a.scale2, c);
        };
        step(lds + turn * (2 * Load::kBytes), lds + (turn ^ 1) * (2 * Load::kBytes));
    }
    if (r < rows)
        store_row<T, NS>(a.dq + row_offset(a.sdq, b, head, token), dq, a.dim, a.scale / c);
}

struct Layout {
    size_t delta, bound, part, total;
    int bounds_q, bounds_v, head_splits;
};
size_t align(size_t v) { return (v + 255) / 256 * 256; }

Layout layout(const dnnseq_attention_desc &d)
{
    Layout l = {};
    const size_t rows_q = (size_t)d.batch * d.q_heads * d.q_len, rows_v = (size_t)d.batch * d.kv_heads * d.kv_len;
    const bool half = d.dtype == DNNSEQ_FP16;
    l.bounds_q = (int)((rows_q + 15) / 16);
    l.bounds_v = half ? (int)((rows_v + 15) / 16) : 0;
    l.bound = align(rows_q * 4);
    l.part = l.bound + (half ? align(((size_t)l.bounds_q + l.bounds_v + 2) * 4) : 0);
    // a group's heads over several workgroups until there are two for every CU
    const int group = d.q_heads / d.kv_heads;
    const int64_t items = (int64_t)d.batch * d.kv_heads * ((d.kv_len + 127) / 128);
    l.head_splits = (int)std::max<int64_t>(1, std::min<int64_t>(group, 1024 / std::max<int64_t>(items, 1)));
    l.total = l.part + (l.head_splits > 1 ? (size_t)l.head_splits * 2 * rows_v * d.head_dim * 4 : 0);
    return l;
}

template <class T, int NS>
hipError_t backward(const Backward &a, hipStream_t st)
{
    if (a.bounds_q + a.bounds_v) {
        attn_delta_kernel<T><<<a.bounds_q + a.bounds_v, 256, 0, st>>>(a);
        if (T::kHalf)
            attn_bound_kernel<<<2, 1024, 0, st>>>(a);
    }
    if (a.kv_len) {
        const int items = a.batch * a.kv_heads * ((a.kv_len + 127) / 128) * a.head_splits;
        attn_dkv_kernel<T, NS><<<items, 256, 0, st>>>(a);
        if (a.head_splits > 1) {
            const size_t units = (size_t)a.batch * a.kv_heads * a.kv_len * a.dim / 8;
            attn_dkv_sum_kernel<T><<<dim3((unsigned)((units + 255) / 256), 2), 256, 0, st>>>(a);
        }
    }
    if (a.q_len) {
        const int items = a.batch * a.kv_heads * (int)(((int64_t)a.q_len * a.group + 127) / 128);
        attn_dq_kernel<T, NS><<<items, 256, 0, st>>>(a);
    }
    return hipGetLastError();
}

template <class T>
hipError_t backward_dim(const Backward &a, hipStream_t st)
{
    switch ((a.dim + 31) / 32) {
    case 1:
        return backward<T, 1>(a, st);
    case 2:
        return backward<T, 2>(a, st);
    case 3:
        return backward<T, 3>(a, st);
    default:
        return backward<T, 4>(a, st);
    }
}

} // namespace

size_t attention_backward_scratch(const dnnseq_attention_desc &d)
{
    return d.batch && (d.q_len || d.kv_len) ? layout(d).total : 0;
}

hipError_t launch_attention_backward(const dnnseq_attention_desc &d, const void *q, const void *k, const void *v,
                                     const void *o, const void *dout, const float *lse, const int32_t *q_lens,
                                     const int32_t *kv_lens, void *dq, void *dk, void *dv, void *scratch,
                                     hipStream_t st)
{
    const Layout l = layout(d);
    char *ws = (char *)scratch;
    Backward a = {};
    a.q = (const uint16_t *)q, a.k = (const uint16_t *)k, a.v = (const uint16_t *)v, a.o = (const uint16_t *)o;
    a.dout = (const uint16_t *)dout, a.lse = lse, a.q_lens = q_lens, a.kv_lens = kv_lens;
    a.dq = (uint16_t *)dq, a.dk = (uint16_t *)dk, a.dv = (uint16_t *)dv;
    a.sq = d.q, a.sk = d.k, a.sv = d.v, a.so = d.o, a.sdo = d.dout, a.sdq = d.dq, a.sdk = d.dk, a.sdv = d.dv;
    a.batch = d.batch, a.q_heads = d.q_heads, a.kv_heads = d.kv_heads, a.group = d.q_heads / d.kv_heads;
    a.q_len = d.q_len, a.kv_len = d.kv_len, a.dim = d.head_dim, a.causal = d.causal;
    a.scale = d.scale, a.scale2 = d.scale * kLog2e;
    a.delta = (float *)(ws + l.delta), a.bound = (float *)(ws + l.bound);
    a.bounds_q = l.bounds_q, a.bounds_v = l.bounds_v, a.head_splits = l.head_splits;
    a.part = l.head_splits > 1 ? (float *)(ws + l.part) : nullptr;
    return d.dtype == DNNSEQ_FP16 ? backward_dim<FP16>(a, st) : backward_dim<BF16>(a, st);
}

} // namespace dsq
