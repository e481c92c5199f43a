// Linear layers on 16-bit tensors: y = act(x w^T + bias) + residual and its gradients.
//
//   forward        y[m][n]: P = w (along k), Q = x (along k)
//   data gradient  dx[m][k]: P = w (across n), Q = g (along n),  g = dy act'(z)
//   weight gradient dw[n][k]: P = x (across m), Q = g (across m)
// One kernel (dnnseq_gemm.h) serves the three: only the loaders and fragment readers differ.  g is
// written once by an elementwise pass that also sums db, in the type of the tensors: the matrix
// cores take 16-bit operands, so it is rounded where any of its uses would round it.
#include "dnnseq_gemm.h"
#include "dnnseq_launch.h"

#include <algorithm>

namespace dsq {
namespace {

struct Product {
    const void *p, *q;
    int64_t ldp, ldq;
    int np, nq, nc; // extents of p, q and the contraction
    int steps;      // steps of the contraction per split
    int act, out32;
    const float *bias;  // [np]
    const void *add;    // [nq][np]
    void *out, *z;
    int64_t ldadd, ldo, ldz;
    float *partial;     // [splits][nq][np], instead of the epilogue
};

__device__ __forceinline__ float activation(int act, float z)
{
    switch (act) {
    case DNNSEQ_ACT_RELU:
        return z < 0.f ? 0.f : z; // (NaN stays NaN)
    case DNNSEQ_ACT_GELU:
        return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
    case DNNSEQ_ACT_SILU:
        // -z beyond 126 log 2: the exponential's reciprocal is denormal; the product is below 1e-36
        return z * mbk::sigmoidf_fast(z);
    case DNNSEQ_ACT_MISH: {
        // tanh(log(1 + e)) = n/(n + 2), n = e (e + 2); 1 to fp32's precision from z = 20 on
        const float e = __expf(fminf(z, 20.0f)), n = e * (e + 2.0f);
        return z * n * __builtin_amdgcn_rcpf(n + 2.0f);
    }
    }
    return z;
}

__device__ __forceinline__ float activation_grad(int act, float z)
{
    switch (act) {
    case DNNSEQ_ACT_RELU:
        return z > 0.f ? 1.f : (z != z ? z : 0.f);
    case DNNSEQ_ACT_GELU:
        return 0.5f * (1.0f + erff(z * 0.70710678118654752f)) + z * 0.39894228040143268f * __expf(-0.5f * z * z);
    case DNNSEQ_ACT_SILU: {
        const float s = mbk::sigmoidf_fast(z);
        return s * (1.0f + z * (1.0f - s));
    }
    case DNNSEQ_ACT_MISH: {
        // tanh' = 1 - t^2 = w (2 - w) with w = 1 - t = 2/(n + 2)
        const float e = __expf(fminf(z, 20.0f)), n = e * (e + 2.0f), w = 2.0f * __builtin_amdgcn_rcpf(n + 2.0f);
        return n * w * 0.5f + z * w * (2.0f - w) * mbk::sigmoidf_fast(z);
    }
    }
    return 1.f;
}

// Four consecutive p of row q: bias, z, activation, what is added, and the store.
template <class T>
__device__ __forceinline__ void finish(const Product &a, int q, int p, f32x4 v)
{
    if (a.bias)
        v += *(const f32x4 *)(a.bias + p);
    if (a.z)
        *(u32x2 *)((uint16_t *)a.z + q * a.ldz + p) = u32x2{T::pack(v[0], v[1]), T::pack(v[2], v[3])};
    if (a.act)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            v[r] = activation(a.act, v[r]);
    if (a.add) {
        const u32x2 w = *(const u32x2 *)((const uint16_t *)a.add + q * a.ldadd + p);
        v += f32x4{T::lo(w[0]), T::hi(w[0]), T::lo(w[1]), T::hi(w[1])};
    }
    if (a.out32)
        *(f32x4 *)((float *)a.out + q * a.ldo + p) = v;
    else
        *(u32x2 *)((uint16_t *)a.out + q * a.ldo + p) = u32x2{T::pack(v[0], v[1]), T::pack(v[2], v[3])};
}

// Tiles in the order of workgroups: the eight XCDs (workgroup b runs on XCD b % 8) take runs of
// consecutive tiles each, and within a run bands of 4 rows of tiles are walked column by column, so
// that what an XCD's cache holds of both operands is used again.
__device__ __forceinline__ void tile_of(uint32_t b, uint32_t n, uint32_t np, uint32_t nq, uint32_t &tp, uint32_t &tq)
{
    const uint32_t x = b % 8, each = n / 8, more = n % 8;
    const uint32_t t = x * each + min(x, more) + b / 8;
    const uint32_t band = t / (4 * np), rows = min(nq - band * 4, 4u), r = t - band * 4 * np;
    tq = band * 4 + r % rows;
    tp = r / rows;
}

// One step: the next step's tiles are requested, this one's multiplied.  (The two buffers are
// restrict arguments: without that every read of LDS waits for the loads into the other buffer.)
template <class T, class LP, class LQ, class RP, class RQ, int FP, int FQ, int QOFF>
__device__ __forceinline__ void product_step(const char *__restrict__ cur, char *__restrict__ nxt, LP &lp, LQ &lq,
                                             const RP &rp, const RQ &rq, f32x4 (&acc)[FP][FQ], int left)
{
    if (left > 0) {
        lp.load(nxt, left);
        lq.load(nxt + QOFF, left);
    }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
        u32x4 fp[FP], fq[FQ];
#pragma unroll
        for (int i = 0; i < FP; ++i)
            fp[i] = rp.get(cur, i, kk);
#pragma unroll
        for (int j = 0; j < FQ; ++j)
            fq[j] = rq.get(cur + QOFF, j, kk);
#pragma unroll
        for (int j = 0; j < FQ; ++j)
#pragma unroll
            for (int i = 0; i < FP; ++i)
                acc[i][j] = T::mma16(fp[i], fq[j], acc[i][j]);
    }
}

template <class T, bool PX, bool QX, int TP, int TQ, int WP, int WQ>
__global__ __launch_bounds__(WP *WQ *kWave) void product_kernel(Product a)
{
    constexpr int THREADS = WP * WQ * kWave, FP = TP / WP / 16, FQ = TQ / WQ / 16;
    typedef Tile<PX, TP> LP;
    typedef Tile<QX, TQ> LQ;
    constexpr int BUF = LP::kBytes + LQ::kBytes;
    __shared__ __attribute__((aligned(256))) char lds[2 * BUF]; // [2][P tile, Q tile]
    const uint32_t np = (a.np + TP - 1) / TP, nq = (a.nq + TQ - 1) / TQ;
    uint32_t tp, tq;
    tile_of(blockIdx.x, np * nq, np, nq, tp, tq);
    const int p0 = tp * TP, q0 = tq * TQ;
    const int c0 = blockIdx.y * a.steps * kStep, left = a.nc - c0;
    const int steps = min(a.steps, (left + kStep - 1) / kStep);
    Loader<PX, TP, THREADS> lp;
    Loader<QX, TQ, THREADS> lq;
    lp.init(a.p, a.ldp, p0, a.np, c0);
    lq.init(a.q, a.ldq, q0, a.nq, c0);
    const int w = wave_id();
    const int wp = w % WP * (TP / WP), wq = w / WP * (TQ / WQ);
    Reader<PX, TP> rp;
    Reader<QX, TQ> rq;
    rp.init(wp);
    rq.init(wq);
    f32x4 acc[FP][FQ];
#pragma unroll
    for (int i = 0; i < FP; ++i)
#pragma unroll
        for (int j = 0; j < FQ; ++j)
            acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (steps > 0) {
        lp.load(lds, left);
        lq.load(lds + LP::kBytes, left);
    }
    for (int s = 0; s < steps; ++s) {
        __builtin_amdgcn_s_waitcnt(0x0f70); // vmcnt(0): this wavefront's part of the tile has landed
        __syncthreads();                    // and everyone's; the other buffer is no longer read
        product_step<T, Loader<PX, TP, THREADS>, Loader<QX, TQ, THREADS>, Reader<PX, TP>, Reader<QX, TQ>, FP, FQ,
                     LP::kBytes>(lds + (s & 1) * BUF, lds + (~s & 1) * BUF, lp, lq, rp, rq, acc,
                                 s + 1 < steps ? left - (s + 1) * kStep : 0);
    }
    const int lane = threadIdx.x % kWave;
#pragma unroll
    for (int j = 0; j < FQ; ++j) {
        const int q = q0 + wq + j * 16 + lane % 16;
        if (q >= a.nq)
            continue;
#pragma unroll
        for (int i = 0; i < FP; ++i) {
            const int p = p0 + wp + i * 16 + lane / 16 * 4;
            if (p >= a.np)
                continue;
            if (a.partial)
                *(f32x4 *)(a.partial + ((size_t)blockIdx.y * a.nq + q) * a.np + p) = acc[i][j];
            else
                finish<T>(a, q, p, acc[i][j]);
        }
    }
}

// The sum over the splits of a contraction, and the epilogue.
template <class T>
__global__ __launch_bounds__(256) void product_finish_kernel(Product a, int splits)
{
    const size_t quads = (size_t)a.nq * (a.np / 4), plane = (size_t)a.nq * a.np;
    for (size_t i = blockIdx.x * (size_t)256 + threadIdx.x; i < quads; i += (size_t)gridDim.x * 256) {
        f32x4 v = *(const f32x4 *)(a.partial + i * 4);
        for (int s = 1; s < splits; ++s)
            v += *(const f32x4 *)(a.partial + s * plane + i * 4);
        const int q = (int)(i / (a.np / 4));
        finish<T>(a, q, (int)(i * 4 - (size_t)q * a.np), v);
    }
}

// g = dy act'(z) and the sums of its columns: a workgroup takes 64 rows x 256 columns (lane: four
// columns, wavefront: every fourth row), column sums in fp32 before g is rounded, one partial row
// per 64 rows.
constexpr int kGradRows = 64;
template <class T>
__global__ __launch_bounds__(256) void act_grad_kernel(const void *dy, int64_t lddy, const void *z, int64_t ldz,
                                                       int act, int m, int n, void *g, float *psum)
{
    const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
    const int c = (blockIdx.x * kWave + lane) * 4, r0 = blockIdx.y * kGradRows;
    __shared__ f32x4 red[4][kWave];
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    if (c < n)
        for (int r = r0 + w; r < min(r0 + kGradRows, m); r += 4) {
            const u32x2 d = *(const u32x2 *)((const uint16_t *)dy + r * lddy + c);
            f32x4 v = {T::lo(d[0]), T::hi(d[0]), T::lo(d[1]), T::hi(d[1])};
            if (act) {
                const u32x2 e = *(const u32x2 *)((const uint16_t *)z + r * ldz + c);
                const f32x4 t = {T::lo(e[0]), T::hi(e[0]), T::lo(e[1]), T::hi(e[1])};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    v[i] *= activation_grad(act, t[i]);
                *(u32x2 *)((uint16_t *)g + (size_t)r * n + c) = u32x2{T::pack(v[0], v[1]), T::pack(v[2], v[3])};
            }
            s += v;
        }
    if (!psum)
        return;
    red[w][lane] = s;
    __syncthreads();
    if (w == 0 && c < n)
        *(f32x4 *)(psum + (size_t)blockIdx.y * n + c) = (red[0][lane] + red[1][lane]) + (red[2][lane] + red[3][lane]);
}

// out[c] = sum over rows of in[rows][n]: a workgroup per 64 columns, its wavefronts take every
// fourth row.
__global__ __launch_bounds__(256) void column_sum_kernel(const float *in, int rows, int n, float *out)
{
    const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave, c = blockIdx.x * kWave + lane;
    __shared__ float red[4][kWave];
    float s = 0.f;
    if (c < n)
        for (int r = w; r < rows; r += 4)
            s += in[(size_t)r * n + c];
    red[w][lane] = s;
    __syncthreads();
    if (w == 0 && c < n)
        out[c] = (red[0][lane] + red[1][lane]) + (red[2][lane] + red[3][lane]);
}

constexpr int kCUs = 256;

int splits_for(int np, int nq, int nc, int tile)
{
    const int64_t tiles = std::max<int64_t>(1, (int64_t)((np + tile - 1) / tile) * ((nq + tile - 1) / tile));
    const int steps = (nc + kStep - 1) / kStep;
    return (int)std::max<int64_t>(1, std::min<int64_t>(kCUs / tiles, steps / 8));
}

template <class T, bool PX, bool QX>
hipError_t launch_product(Product a, float *scratch, hipStream_t st)
{
    constexpr int TILE = 128;
    const int splits = splits_for(a.np, a.nq, a.nc, TILE);
    const int steps = (a.nc + kStep - 1) / kStep;
    a.steps = (steps + splits - 1) / splits;
    const int used = std::max(1, (steps + a.steps - 1) / std::max(a.steps, 1));
    a.partial = used > 1 ? scratch : nullptr;
    const dim3 grid(((a.np + TILE - 1) / TILE) * ((a.nq + TILE - 1) / TILE), used);
    product_kernel<T, PX, QX, TILE, TILE, 2, 2><<<grid, 256, 0, st>>>(a);
    if (used > 1) {
        const size_t quads = (size_t)a.nq * (a.np / 4);
        product_finish_kernel<T><<<(unsigned)std::min<size_t>((quads + 255) / 256, 4096), 256, 0, st>>>(a, used);
    }
    return hipGetLastError();
}

size_t product_scratch(int np, int nq, int nc)
{
    const int s = splits_for(np, nq, nc, 128);
    return s > 1 ? (size_t)s * np * nq * 4 : 0;
}

size_t align(size_t v) { return (v + 255) / 256 * 256; }

template <class T>
hipError_t forward(const dnnseq_linear_desc &d, const void *x, const void *w, const float *bias, const void *residual,
                   void *y, void *z, void *scratch, hipStream_t st)
{
    Product a = {};
    a.p = w, a.ldp = d.ldw, a.np = d.n;
    a.q = x, a.ldq = d.ldx, a.nq = d.m;
    a.nc = d.k;
    a.act = d.activation, a.bias = bias, a.add = residual, a.ldadd = d.ldresidual;
    a.out = y, a.ldo = d.ldy, a.z = z, a.ldz = d.ldz;
    return launch_product<T, false, false>(a, (float *)scratch, st);
}

struct BackwardScratch {
    size_t g, psum, product, total;
};
BackwardScratch backward_layout(const dnnseq_linear_desc &d)
{
    BackwardScratch s;
    s.g = 0;
    s.psum = d.activation ? align((size_t)d.m * d.n * 2) : 0;
    s.product = s.psum + align((size_t)((d.m + kGradRows - 1) / kGradRows) * d.n * 4);
    s.total = s.product + std::max(product_scratch(d.k, d.m, d.n), product_scratch(d.k, d.n, d.m));
    return s;
}

template <class T>
hipError_t backward(const dnnseq_linear_desc &d, const void *x, const void *w, const void *z, const void *dy,
                    const void *dx_add, void *dx, void *dw, float *db, void *scratch, hipStream_t st)
{
    const BackwardScratch l = backward_layout(d);
    char *ws = (char *)scratch;
    const void *g = dy;
    int64_t ldg = d.lddy;
    const int parts = (d.m + kGradRows - 1) / kGradRows;
    if ((d.activation || db) && d.m) {
        act_grad_kernel<T><<<dim3((d.n + 255) / 256, parts), 256, 0, st>>>(
            dy, d.lddy, z, d.ldz, d.activation, d.m, d.n, ws + l.g, db ? (float *)(ws + l.psum) : nullptr);
        if (d.activation) {
            g = ws + l.g;
            ldg = d.n;
        }
    }
    if (db)
        column_sum_kernel<<<(d.n + kWave - 1) / kWave, 256, 0, st>>>((const float *)(ws + l.psum), parts, d.n, db);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && dx && d.m) {
        Product a = {};
        a.p = w, a.ldp = d.ldw, a.np = d.k;
        a.q = g, a.ldq = ldg, a.nq = d.m;
        a.nc = d.n;
        a.add = dx_add, a.ldadd = d.lddx_add, a.out = dx, a.ldo = d.lddx;
        e = launch_product<T, true, false>(a, (float *)(ws + l.product), st);
    }
    if (e == hipSuccess && dw) {
        Product a = {};
        a.p = x, a.ldp = d.ldx, a.np = d.k;
        a.q = g, a.ldq = ldg, a.nq = d.n;
        a.nc = d.m;
        a.out = dw, a.ldo = d.lddw, a.out32 = d.dw_fp32;
        e = launch_product<T, true, true>(a, (float *)(ws + l.product), st);
    }
    return e;
}

} // namespace

size_t linear_forward_scratch(const dnnseq_linear_desc &d) { return product_scratch(d.n, d.m, d.k); }
size_t linear_backward_scratch(const dnnseq_linear_desc &d) { return backward_layout(d).total; }

hipError_t launch_linear_forward(const dnnseq_linear_desc &d, const void *x, const void *w, const float *bias,
                                 const void *residual, void *y, void *z, void *scratch, hipStream_t st)
{
    return d.dtype == DNNSEQ_FP16 ? forward<FP16>(d, x, w, bias, residual, y, z, scratch, st)
                                  : forward<BF16>(d, x, w, bias, residual, y, z, scratch, st);
}
hipError_t launch_linear_backward(const dnnseq_linear_desc &d, const void *x, const void *w, const void *z,
                                  const void *dy, const void *dx_add, void *dx, void *dw, float *db, void *scratch,
                                  hipStream_t st)
{
    return d.dtype == DNNSEQ_FP16 ? backward<FP16>(d, x, w, z, dy, dx_add, dx, dw, db, scratch, st)
                                  : backward<BF16>(d, x, w, z, dy, dx_add, dx, dw, db, scratch, st);
}

} // namespace dsq
