// Layer normalisation of 16-bit rows, forward and backward: bound by memory, every tensor read or
// written once (16384 x 4096, bf16: forward 49 us, 5.5 TB/s; backward with the residual's gradient 98 us, 5.5
// TB/s); a few rows by the launches (77 x 1001: 5 us each way).
//
// A row stays in the registers of TPR threads (NU units of eight elements each, unit u of thread t at
// element 8 (u TPR + t)), so the statistics and what follows them need one read.  Mean and variance
// over several wavefronts take one exchange: each wavefront has its own mean and sum of squares about
// it, and sum (x - mu)^2 = sum over wavefronts of (M2_w + n_w (mean_w - mu)^2).  The column sums of the
// weight gradients are kept per thread over the rows a workgroup walks, combined over its thread
// groups in LDS, and added over the workgroups by a second launch in a fixed order; few rows take them
// beside the rows' own pass.
// Rows need not be aligned: gfx950 takes 16-byte accesses at any even address, and only a row's last
// cols % 8 elements are read one by one.
#include "dnnseq_dev.h"
#include "dnnseq_launch.h"

#include <algorithm>

namespace dsq {
namespace {

typedef u32x4 __attribute__((aligned(2))) u32x4_any; // 16 bytes at any element

template <int NU>
struct Units {
    u32x4 v[NU];
    template <int TPR>
    __device__ __forceinline__ void load(const uint16_t *row, int cols, int t)
    {
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            const int c = (u * TPR + t) * 8;
            if (c + 8 <= cols)
                v[u] = *(const u32x4_any *)(row + c);
            else {
                v[u] = u32x4{0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < 7; ++i)
                    if (c + i < cols)
                        v[u][i / 2] |= (uint32_t)row[c + i] << (i % 2 * 16);
            }
        }
    }
};

template <class T>
__device__ __forceinline__ float element(const u32x4 &v, int i)
{
    return i % 2 ? T::hi(v[i / 2]) : T::lo(v[i / 2]);
}

template <class T, bool STREAM>
__device__ __forceinline__ void store_unit(uint16_t *row, int cols, int c, const float (&f)[8])
{
    const u32x4 v = {T::pack(f[0], f[1]), T::pack(f[2], f[3]), T::pack(f[4], f[5]), T::pack(f[6], f[7])};
    if (c + 8 <= cols) {
        if (STREAM)
            __builtin_nontemporal_store(v, (u32x4_any *)(row + c));
        else
            *(u32x4_any *)(row + c) = v;
        return;
    }
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (c + i < cols)
            row[c + i] = (uint16_t)(v[i / 2] >> (i % 2 * 16));
}

__device__ __forceinline__ void load_vector(float (&f)[8], const float *p, int cols, int c)
{
    if (c + 8 <= cols) {
        const f32x4 a = *(const f32x4 *)(p + c), b = *(const f32x4 *)(p + c + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            f[i] = a[i], f[i + 4] = b[i];
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        f[i] = c + i < cols ? p[c + i] : 0.f;
}

// Sum over the threads of a row within a wavefront, in all of its lanes.
template <int TPR>
__device__ __forceinline__ float lane_sum(float v)
{
    return TPR == 16 ? mbk::row16_sum(v) : mbk::wave_sum(v);
}

template <class T, int TPR, int NU, bool STREAM>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_fwd_kernel(const uint16_t *x, int64_t ldx,
                                                                         const float *gamma, const float *beta,
                                                                         float eps, int rows, int cols, uint16_t *y,
                                                                         int64_t ldy, float *mean, float *rstd)
{
    constexpr int THREADS = TPR > 256 ? TPR : 256, G = THREADS / TPR, W = TPR / kWave;
    __shared__ float red[2][W > 1 ? 2 * W : 1];
    const int t = threadIdx.x % TPR;
    float g[NU][8], b[NU][8];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        load_vector(g[u], gamma, cols, (u * TPR + t) * 8);
        load_vector(b[u], beta, cols, (u * TPR + t) * 8);
    }
    const float inv = 1.0f / (float)cols;
    int turn = 0;
    for (int r = blockIdx.x * G + threadIdx.x / TPR; r < rows; r += gridDim.x * G, turn ^= 1) {
        Units<NU> a;
        a.template load<TPR>(x + r * ldx, cols, t);
        float s = 0.f;
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) // (past the row's end there are zeros)
                s += element<T>(a.v[u], i);
        s = lane_sum<TPR>(s);
        // elements of the row in this wavefront (TPR <= 64: all of them)
        int n = cols;
        if (W > 1) {
            n = 0;
            const int w0 = t / kWave * kWave;
#pragma unroll
            for (int u = 0; u < NU; ++u)
                n += max(0, min(cols - (u * TPR + w0) * 8, kWave * 8));
        }
        float mu = W > 1 ? (n ? s / (float)n : 0.f) : s * inv;
        float q = 0.f;
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = element<T>(a.v[u], i) - mu;
                q = (u * TPR + t) * 8 + i < cols ? fmaf(d, d, q) : q;
            }
        q = lane_sum<TPR>(q);
        if (W > 1) {
            float *e = red[turn];
            if (threadIdx.x % kWave == 0) {
                e[t / kWave * 2] = s;
                e[t / kWave * 2 + 1] = q;
            }
            __syncthreads();
            float total = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w)
                total += e[w * 2];
            mu = total * inv;
            q = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                int nw = 0;
#pragma unroll
                for (int u = 0; u < NU; ++u)
                    nw += max(0, min(cols - (u * TPR + w * kWave) * 8, kWave * 8));
                const float d = nw ? e[w * 2] / (float)nw - mu : 0.f;
                q += e[w * 2 + 1] + (float)nw * d * d;
            }
        }
        const float rs = 1.0f / sqrtf(q * inv + eps);
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                f[i] = fmaf(g[u][i], (element<T>(a.v[u], i) - mu) * rs, b[u][i]);
            store_unit<T, STREAM>(y + r * ldy, cols, (u * TPR + t) * 8, f);
        }
        if (t == 0) {
            mean[r] = mu;
            rstd[r] = rs;
        }
    }
}

// dgamma and dbeta of kCols columns in full: groups of as many lanes take every row of their number, eight
// rows on the way at a time; their sums are added in order.
constexpr int kCols = 32;
struct Columns {
    const uint16_t *x, *dy;
    int64_t ldx, lddy;
    const float *mean, *rstd;
    int rows, cols;
    float *dgamma, *dbeta; // NULL: the rows' workgroups leave partial sums
};
template <class T, int THREADS>
__device__ __forceinline__ void norm_columns(const Columns &a, int block)
{
    constexpr int GROUPS = THREADS / kCols;
    __shared__ float red[2][GROUPS][kCols];
    const int g = threadIdx.x / kCols, i = threadIdx.x % kCols, c = block * kCols + i, at = min(c, a.cols - 1);
    float sg = 0.f, sb = 0.f;
    for (int r0 = g; r0 < a.rows; r0 += 8 * GROUPS) {
        uint16_t x[8], d[8];
        float mu[8], rs[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int64_t r = min(r0 + u * GROUPS, a.rows - 1);
            x[u] = a.x[r * a.ldx + at];
            d[u] = a.dy[r * a.lddy + at];
            mu[u] = a.mean[r];
            rs[u] = a.rstd[r];
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (r0 + u * GROUPS >= a.rows)
                break;
            const float v = T::lo(d[u]);
            sg = fmaf(v, (T::lo(x[u]) - mu[u]) * rs[u], sg);
            sb += v;
        }
    }
    red[0][g][i] = sg;
    red[1][g][i] = sb;
    __syncthreads();
    if (g < 2 && c < a.cols) {
        float s = red[g][0][i];
#pragma unroll
        for (int j = 1; j < GROUPS; ++j)
            s += red[g][j][i];
        (g ? a.dbeta : a.dgamma)[c] = s;
    }
}

template <class T, int TPR, int NU, bool ADD, bool STREAM>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_bwd_kernel(
    const uint16_t *x, int64_t ldx, const uint16_t *dy, int64_t lddy, const float *gamma, const float *mean,
    const float *rstd, const uint16_t *add, int64_t ldadd, int rows, int cols, uint16_t *dx, int64_t lddx,
    float *pgamma, float *pbeta, int groups, float *dgamma, float *dbeta)
{
    constexpr int THREADS = TPR > 256 ? TPR : 256, G = THREADS / TPR, W = TPR / kWave;
    if ((int)blockIdx.x >= groups) {
        norm_columns<T, THREADS>({x, dy, ldx, lddy, mean, rstd, rows, cols, dgamma, dbeta}, blockIdx.x - groups);
        return;
    }
    __shared__ float red[2][W > 1 ? 2 * W : 1];
    const int t = threadIdx.x % TPR;
    float g[NU][8], ag[NU][8], ab[NU][8];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        load_vector(g[u], gamma, cols, (u * TPR + t) * 8);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            ag[u][i] = ab[u][i] = 0.f;
    }
    const float inv = 1.0f / (float)cols;
    const int first = blockIdx.x * G + threadIdx.x / TPR, step = groups * G;
    Units<NU> nx, nd, na;
    const auto fetch = [&](int r) __attribute__((always_inline)) {
        nx.template load<TPR>(x + r * ldx, cols, t);
        nd.template load<TPR>(dy + r * lddy, cols, t);
        if (ADD)
            na.template load<TPR>(add + r * ldadd, cols, t);
    };
    constexpr bool AHEAD = TPR * NU <= 1024; // longer rows have no registers for it
    if (AHEAD && first < rows)
        fetch(first);
    int turn = 0;
    for (int r = first; r < rows; r += step, turn ^= 1) {
        if (!AHEAD)
            fetch(r);
        const Units<NU> a = nx, d = nd, o = na;
        const float mu = mean[r], rs = rstd[r];
        if (AHEAD && r + step < rows)
            fetch(r + step);
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) { // (past the row's end dy and gamma are zeros)
                const float v = element<T>(d.v[u], i), gg = v * g[u][i];
                const float xh = (element<T>(a.v[u], i) - mu) * rs;
                ag[u][i] = fmaf(v, xh, ag[u][i]);
                ab[u][i] += v;
                s1 += gg;
                // (xh of an element past the end may be infinite: 0 * that is no zero)
                s2 = (u * TPR + t) * 8 + i < cols ? fmaf(gg, xh, s2) : s2;
            }
        s1 = lane_sum<TPR>(s1);
        s2 = lane_sum<TPR>(s2);
        if (W > 1) {
            float *e = red[turn];
            if (threadIdx.x % kWave == 0) {
                e[t / kWave * 2] = s1;
                e[t / kWave * 2 + 1] = s2;
            }
            __syncthreads();
            s1 = s2 = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                s1 += e[w * 2];
                s2 += e[w * 2 + 1];
            }
        }
        const float m1 = s1 * inv, m2 = s2 * inv;
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float xh = (element<T>(a.v[u], i) - mu) * rs;
                f[i] = rs * (element<T>(d.v[u], i) * g[u][i] - m1 - xh * m2);
                if (ADD)
                    f[i] += element<T>(o.v[u], i);
            }
            store_unit<T, STREAM>(dx + r * lddx, cols, (u * TPR + t) * 8, f);
        }
    }
    if (dgamma)
        return;
    // one partial row per workgroup, its thread groups added in a fixed order
    __shared__ float part[G > 1 ? G : 1][G > 1 ? TPR * NU * 8 : 1];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        float *out = (k ? pbeta : pgamma) + (size_t)blockIdx.x * cols;
        if (G == 1) {
#pragma unroll
            for (int u = 0; u < NU; ++u)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int c = (u * TPR + t) * 8 + i;
                    if (c < cols)
                        out[c] = k ? ab[u][i] : ag[u][i];
                }
            continue;
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                part[threadIdx.x / TPR][(G > 1 ? (u * TPR + t) * 8 + i : 0)] = k ? ab[u][i] : ag[u][i];
        __syncthreads();
        for (int c = threadIdx.x; c < cols; c += THREADS) {
            float s = part[0][c];
            for (int j = 1; j < G; ++j)
                s += part[j][c];
            out[c] = s;
        }
    }
}

// out[c] = sum over parts of in[parts][cols]; y: gamma or beta.  A workgroup per 64 columns, each of its
// sixteen wavefronts takes every sixteenth part.
__global__ __launch_bounds__(1024) void norm_sum_kernel(const float *pgamma, const float *pbeta, int parts, int cols,
                                                        float *dgamma, float *dbeta)
{
    const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave, c = blockIdx.x * kWave + lane;
    const float *in = blockIdx.y ? pbeta : pgamma;
    __shared__ float red[16][kWave];
    float s = 0.f;
    if (c < cols) {
#pragma unroll 8
        for (int p = w; p < parts; p += 16)
            s += in[(size_t)p * cols + c];
    }
    red[w][lane] = s;
    __syncthreads();
    if (w == 0 && c < cols) {
#pragma unroll
        for (int v = 1; v < 16; ++v)
            s += red[v][lane];
        (blockIdx.y ? dbeta : dgamma)[c] = s;
    }
}

// Threads per row and units per thread for a row length.
#define NORM_FORMS(F)                                                                                                  \
    if (d.cols <= 128)                                                                                                 \
        F(16, 1);                                                                                                      \
    else if (d.cols <= 512)                                                                                            \
        F(64, 1);                                                                                                      \
    else if (d.cols <= 1024)                                                                                           \
        F(64, 2);                                                                                                      \
    else if (d.cols <= 2048)                                                                                           \
        F(256, 1);                                                                                                     \
    else if (d.cols <= 4096)                                                                                           \
        F(256, 2);                                                                                                     \
    else if (d.cols <= 8192)                                                                                           \
        F(1024, 1);                                                                                                    \
    else                                                                                                               \
        F(1024, 2)

int rows_per_group(int cols) { return cols <= 128 ? 16 : cols <= 1024 ? 4 : 1; }

// Workgroups, and so partial rows: more of them hide the latency of few rows each, and cost 16 bytes per
// column on their way to memory and back (rows x columns, us with 128 / 256 / 512: 512 x 4096 14.5 / 16.1 / 24.3,
// 2048 x 4096 32.4 / 24.3 / 26.4, 8192 x 2048 74 / 42 / 31; rows past 4096 columns have one workgroup a CU).
int backward_groups(const dnnseq_layernorm_desc &d)
{
    const int per = rows_per_group(d.cols), fill = std::max({128, std::min(d.rows / 4, 256), d.rows / 8});
    return std::min({(d.rows + per - 1) / per, fill, d.cols <= 4096 ? 512 : 256});
}

// Few rows: workgroups beside the rows' read x and dy a second time for the columns' sums, a launch less
// (rows x columns, direct / in parts: 77 x 1001 5.1 / 8.1 us, 192 x 2048 8.3 / 9.2, 256 x 2048 12.9 / 8.5, 512 x 8192
// 13.8 / 21.1, 1024 x 8192 25.5 / 27.0).
bool direct_columns(const dnnseq_layernorm_desc &d) { return d.rows > 0 && d.rows <= (d.cols <= 4096 ? 192 : 512); }

// Results past the caches: from 16 MiB on what is read next is not in an L2 anyway, and what the other tensors
// leave there stays (backward of 16384 x 4096 with dx_add in a trace 112 -> 95 us, forward of 8192 x 2048 17.5 -> 14.6, a forward pass that
// reads the result included 33.2 -> 32.4; 4096 x 1024, 8 MiB: no difference).
bool streamed(const dnnseq_layernorm_desc &d) { return (int64_t)d.rows * d.cols >= 8 << 20; }

template <class T, bool STREAM>
void forward(const dnnseq_layernorm_desc &d, const void *x, const float *gamma, const float *beta, void *y,
             float *mean, float *rstd, hipStream_t st)
{
    const int per = rows_per_group(d.cols), grid = std::min((d.rows + per - 1) / per, 2048);
#define NORM_FWD(TPR, NU)                                                                                              \
    norm_fwd_kernel<T, TPR, NU, STREAM><<<grid, TPR > 256 ? TPR : 256, 0, st>>>((const uint16_t *)x, d.ldx, gamma, beta,        \
                                                                        d.eps, d.rows, d.cols, (uint16_t *)y, d.ldy,   \
                                                                        mean, rstd)
    NORM_FORMS(NORM_FWD);
#undef NORM_FWD
}

template <class T, bool ADD, bool STREAM>
void backward(const dnnseq_layernorm_desc &d, const void *x, const void *dy, const float *gamma, const float *mean,
              const float *rstd, const void *add, void *dx, float *pgamma, float *pbeta, int groups, float *dgamma,
              float *dbeta, hipStream_t st)
{
    const int grid = groups + (dgamma ? (d.cols + kCols - 1) / kCols : 0);
#define NORM_BWD(TPR, NU)                                                                                              \
    norm_bwd_kernel<T, TPR, NU, ADD, STREAM><<<grid, TPR > 256 ? TPR : 256, 0, st>>>(                                          \
        (const uint16_t *)x, d.ldx, (const uint16_t *)dy, d.lddy, gamma, mean, rstd, (const uint16_t *)add,            \
        d.lddx_add, d.rows, d.cols, (uint16_t *)dx, d.lddx, pgamma, pbeta, groups, dgamma,    \
        dbeta)
    NORM_FORMS(NORM_BWD);
#undef NORM_BWD
}

} // namespace

size_t norm_backward_scratch(const dnnseq_layernorm_desc &d)
{
    return 2 * (size_t)backward_groups(d) * d.cols * 4;
}

hipError_t launch_norm_forward(const dnnseq_layernorm_desc &d, const void *x, const float *gamma, const float *beta,
                               void *y, float *mean, float *rstd, hipStream_t st)
{
    const auto f = streamed(d) ? (d.dtype == DNNSEQ_FP16 ? forward<FP16, true> : forward<BF16, true>)
                               : (d.dtype == DNNSEQ_FP16 ? forward<FP16, false> : forward<BF16, false>);
    f(d, x, gamma, beta, y, mean, rstd, st);
    return hipGetLastError();
}

hipError_t launch_norm_backward(const dnnseq_layernorm_desc &d, const void *x, const void *dy, const float *gamma,
                                const float *mean, const float *rstd, const void *dx_add, void *dx, float *dgamma,
                                float *dbeta, void *scratch, hipStream_t st)
{
    const int grid = backward_groups(d);
    const bool direct = direct_columns(d);
    float *pgamma = (float *)scratch, *pbeta = pgamma + (size_t)grid * d.cols;
    const bool half = d.dtype == DNNSEQ_FP16;
    const auto f = streamed(d) ? (half ? (dx_add ? backward<FP16, true, true> : backward<FP16, false, true>)
                                       : (dx_add ? backward<BF16, true, true> : backward<BF16, false, true>))
                               : (half ? (dx_add ? backward<FP16, true, false> : backward<FP16, false, false>)
                                       : (dx_add ? backward<BF16, true, false> : backward<BF16, false, false>));
    if (d.rows)
        f(d, x, dy, gamma, mean, rstd, dx_add, dx, pgamma, pbeta, grid, direct ? dgamma : nullptr,
          direct ? dbeta : nullptr, st);
    if (!direct)
        norm_sum_kernel<<<dim3((d.cols + kWave - 1) / kWave, 2), 1024, 0, st>>>(pgamma, pbeta, grid, d.cols, dgamma, dbeta);
    return hipGetLastError();
}

} // namespace dsq
