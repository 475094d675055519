// Layer norm over the neurons of each sample, forward and backward, on blocks [n][B].
//
// Two launches each: sums over the rows of a range per workgroup, then every workgroup adds up the ranges' sums for its columns and
// writes its part of the result.  Sums are fp64 and in a fixed order.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "sdnn_internal.h"
#include "sdnn_pack8.h"

#define NORM_THREADS 256

// The block that is normalized, as it is ...
struct PlainBlock {
    const float *x;
    template <int V> __device__ __forceinline__ void load(size_t e, float (&v)[V]) const
    {
        if constexpr (V == 4) {
            const float4 t = *reinterpret_cast<const float4 *>(x + e);
            v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
        } else {
            v[0] = x[e];
        }
    }
};
// ... or in 8 bits
struct PackedBlock {
    const uint8_t *codes;
    const uint16_t *scales;
    float cap, below;
    template <int V> __device__ __forceinline__ void load(size_t e, float (&v)[V]) const
    {
        const float t = __uint_as_float((unsigned)scales[e / PACK_GROUP] << 16);
        if constexpr (V == 4) {
            const unsigned c = *reinterpret_cast<const unsigned *>(codes + e);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = pack8_value(c >> (8 * k) & 255u, t, cap, below);
        } else {
            v[0] = pack8_value(codes[e], t, cap, below);
        }
    }
};

// A workgroup's threads: 1 << cl_log2 of them lie across the columns, V columns each, the others across the rows.
struct Shape {
    int32_t n, B, cl_log2, rows; // rows: of a range
};

// Adds up V pairs of sums over the threads that share columns; afterwards the threads of the first row have them.
template <int V> __device__ __forceinline__ void add_up(double (&a)[V], double (&b)[V], int cl_log2, double2 (*lds)[V])
{
    const int tid = threadIdx.x, cl = 1 << cl_log2;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) lds[tid][v] = make_double2(a[v], b[v]);
    __syncthreads();
    if (tid < cl)
        for (int t = tid + cl; t < NORM_THREADS; t += cl)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                a[v] += lds[t][v].x;
                b[v] += lds[t][v].y;
            }
}

// part [range][B]: sums of x - x0 and of its square, x0 the sample's first value: no cancellation where the mean is large
// (and firsts [B]: x0, which the second launch may write its results over)
template <int V>
__global__ void __launch_bounds__(NORM_THREADS) k_norm_sums(const float *__restrict__ x, Shape sh, double2 *__restrict__ part, float *__restrict__ firsts)
{
    __shared__ double2 lds[NORM_THREADS][V];
    const int col = ((int)(blockIdx.x << sh.cl_log2) + (int)(threadIdx.x & ((1 << sh.cl_log2) - 1))) * V;
    const int r0 = (int)blockIdx.y * sh.rows, r1 = min(sh.n, r0 + sh.rows);
    double s1[V] = {}, s2[V] = {};
    if (col < sh.B) {
        float first[V];
        PlainBlock{x}.load<V>((size_t)col, first);
        for (int r = r0 + (int)(threadIdx.x >> sh.cl_log2); r < r1; r += NORM_THREADS >> sh.cl_log2) {
            float t[V];
            PlainBlock{x}.load<V>((size_t)r * sh.B + col, t);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const double d = (double)t[v] - (double)first[v];
                s1[v] += d;
                s2[v] = fma(d, d, s2[v]);
            }
        }
    }
    add_up<V>(s1, s2, sh.cl_log2, lds);
    if ((int)threadIdx.x < 1 << sh.cl_log2 && col < sh.B)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            part[(size_t)blockIdx.y * sh.B + col + v] = make_double2(s1[v], s2[v]);
            if (blockIdx.y == 0) firsts[col + v] = x[col + v];
        }
}

// The sums of all ranges for a workgroup's columns, in all of its threads.
template <int V>
__device__ __forceinline__ void total(const double2 *__restrict__ part, int ranges, int col, const Shape &sh, double (&a)[V], double (&b)[V], double2 (*lds)[V])
{
#pragma unroll
    for (int v = 0; v < V; ++v) a[v] = b[v] = 0.0;
    if (col < sh.B)
        for (int k = (int)(threadIdx.x >> sh.cl_log2); k < ranges; k += NORM_THREADS >> sh.cl_log2)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const double2 p = part[(size_t)k * sh.B + col + v];
                a[v] += p.x;
                b[v] += p.y;
            }
    add_up<V>(a, b, sh.cl_log2, lds);
    const int c = threadIdx.x & ((1 << sh.cl_log2) - 1);
    __syncthreads();
    if ((int)threadIdx.x == c)
#pragma unroll
        for (int v = 0; v < V; ++v) lds[c][v] = make_double2(a[v], b[v]);
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) {
        a[v] = lds[c][v].x;
        b[v] = lds[c][v].y;
    }
}

template <int V> __device__ __forceinline__ void store(float *p, const float (&v)[V])
{
    if constexpr (V == 4) *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else *p = v[0];
}

template <int V>
__global__ void __launch_bounds__(NORM_THREADS) k_norm_apply(const float *x, const float *__restrict__ gamma, const float *__restrict__ beta, Shape sh,
                                                             double eps, const double2 *__restrict__ part, float *y, double *__restrict__ stats, int ranges,
                                                             const float *__restrict__ firsts)
{
    __shared__ double2 lds[NORM_THREADS][V];
    const int col = ((int)(blockIdx.x << sh.cl_log2) + (int)(threadIdx.x & ((1 << sh.cl_log2) - 1))) * V;
    double mean[V], rstd[V];
    total<V>(part, ranges, col, sh, mean, rstd, lds);
    if (col >= sh.B) return;
    const double inv = 1.0 / (double)sh.n;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const double m = mean[v] * inv, var = rstd[v] * inv - m * m;
        mean[v] = (double)firsts[col + v] + m;
        rstd[v] = 1.0 / sqrt((var < 0.0 ? 0.0 : var) + eps); // an infinity or NaN in a sample: NaN, and so is all of its result
    }
    if (blockIdx.y == 0 && stats && (int)threadIdx.x < 1 << sh.cl_log2)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            stats[col + v] = mean[v];
            stats[sh.B + col + v] = rstd[v];
        }
    const int r0 = (int)blockIdx.y * sh.rows, r1 = min(sh.n, r0 + sh.rows);
    for (int r = r0 + (int)(threadIdx.x >> sh.cl_log2); r < r1; r += NORM_THREADS >> sh.cl_log2) {
        const double g = gamma ? (double)gamma[r] : 1.0, b = beta ? (double)beta[r] : 0.0;
        float t[V];
        PlainBlock{x}.load<V>((size_t)r * sh.B + col, t);
#pragma unroll
        for (int v = 0; v < V; ++v) t[v] = (float)fma(((double)t[v] - mean[v]) * rstd[v], g, b);
        store<V>(y + (size_t)r * sh.B + col, t);
    }
}

// The backward pass's sums: over a range of rows p = sum g dY and q = sum g dY h for every sample, h = (x - mean) rstd, and over the
// samples dg = sum dY h and db = sum dY for every row of the range.
#define GRAD_ROWS 512 // rows of a range at most
template <int V, class Block>
__global__ void __launch_bounds__(NORM_THREADS) k_norm_grad_sums(const float *__restrict__ dy, const Block x, const double *__restrict__ stats,
                                                                 const float *__restrict__ gamma, Shape sh, double2 *__restrict__ part,
                                                                 float *__restrict__ dgamma, float *__restrict__ dbeta)
{
    __shared__ double2 lds[NORM_THREADS][V], row_sum[GRAD_ROWS];
    const int cl = 1 << sh.cl_log2, c = threadIdx.x & (cl - 1);
    const int r0 = (int)blockIdx.x * sh.rows, r1 = min(sh.n, r0 + sh.rows);
    for (int r = threadIdx.x; r < GRAD_ROWS; r += NORM_THREADS) row_sum[r] = make_double2(0.0, 0.0);
    __syncthreads();
    for (int col0 = 0; col0 < sh.B; col0 += cl * V) {
        const int col = col0 + c * V;
        const bool live = col < sh.B;
        double p[V] = {}, q[V] = {}, mean[V] = {}, rstd[V] = {};
        if (live)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                mean[v] = stats[col + v];
                rstd[v] = stats[sh.B + col + v];
            }
        for (int r = r0 + (int)(threadIdx.x >> sh.cl_log2); r < r1; r += NORM_THREADS >> sh.cl_log2) {
            const double g = gamma ? (double)gamma[r] : 1.0;
            double dg = 0.0, db = 0.0;
            if (live) {
                float t[V], d[V];
                const size_t e = (size_t)r * sh.B + col;
                x.template load<V>(e, t);
                PlainBlock{dy}.load<V>(e, d);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const double h = ((double)t[v] - mean[v]) * rstd[v], gd = g * (double)d[v];
                    p[v] += gd;
                    q[v] = fma(gd, h, q[v]);
                    dg = fma((double)d[v], h, dg);
                    db += (double)d[v];
                }
            }
            for (int m = 1; m < cl; m *= 2) {
                dg += __shfl_xor(dg, m);
                db += __shfl_xor(db, m);
            }
            if (c == 0) { // always the same thread for a row
                row_sum[r - r0].x += dg;
                row_sum[r - r0].y += db;
            }
        }
        add_up<V>(p, q, sh.cl_log2, lds);
        if ((int)threadIdx.x < cl && live)
#pragma unroll
            for (int v = 0; v < V; ++v) part[(size_t)blockIdx.x * sh.B + col + v] = make_double2(p[v], q[v]);
    }
    __syncthreads();
    for (int r = r0 + (int)threadIdx.x; r < r1; r += NORM_THREADS) {
        if (dgamma) dgamma[r] = (float)row_sum[r - r0].x;
        if (dbeta) dbeta[r] = (float)row_sum[r - r0].y;
    }
}

template <int V, class Block>
__global__ void __launch_bounds__(NORM_THREADS) k_norm_grad_apply(const float *dy, const Block x, const double *__restrict__ stats, const float *__restrict__ gamma,
                                                                  Shape sh, const double2 *__restrict__ part, int ranges, float *dx)
{
    __shared__ double2 lds[NORM_THREADS][V];
    const int col = ((int)(blockIdx.x << sh.cl_log2) + (int)(threadIdx.x & ((1 << sh.cl_log2) - 1))) * V;
    double p[V], q[V], mean[V], rstd[V];
    total<V>(part, ranges, col, sh, p, q, lds);
    if (col >= sh.B) return;
    const double inv = 1.0 / (double)sh.n;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        p[v] *= inv;
        q[v] *= inv;
        mean[v] = stats[col + v];
        rstd[v] = stats[sh.B + col + v];
    }
    const int r0 = (int)blockIdx.y * sh.rows, r1 = min(sh.n, r0 + sh.rows);
    for (int r = r0 + (int)(threadIdx.x >> sh.cl_log2); r < r1; r += NORM_THREADS >> sh.cl_log2) {
        const double g = gamma ? (double)gamma[r] : 1.0;
        float t[V], d[V];
        const size_t e = (size_t)r * sh.B + col;
        x.template load<V>(e, t);
        PlainBlock{dy}.load<V>(e, d);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const double h = ((double)t[v] - mean[v]) * rstd[v];
            t[v] = (float)(rstd[v] * (fma(g, (double)d[v], -p[v]) - h * q[v]));
        }
        store<V>(dx + e, t);
    }
}

// ---- host side ------------------------------------------------------------------------------------------------------------
// Ranges of rows: enough workgroups to fill the chip, and not so many that their sums are a load to add up.
static int forward_ranges(int n, int B) { return std::max(1, std::min(1024 / ((B - 1) / 256 + 1), (n - 1) / 32 + 1)); }
static int backward_ranges(int n) { return std::max(std::min(1024, (n - 1) / 16 + 1), (n - 1) / GRAD_ROWS + 1); }
static int range_rows(int n, int ranges) { return (n - 1) / ranges + 1; }

static Shape shape_for(int n, int B, int V, int ranges)
{
    Shape sh;
    sh.n = n; sh.B = B; sh.cl_log2 = 0; sh.rows = range_rows(n, ranges);
    while (sh.cl_log2 < 6 && (V << sh.cl_log2) < B) ++sh.cl_log2;
    return sh;
}
static unsigned tiles(const Shape &sh, int V) { return (unsigned)((sh.B - 1) / (V << sh.cl_log2) + 1); }

static int check_norm(int32_t n, int32_t B)
{
    if (n < 1 || B < 1 || n > 1 << 30 || B > 1 << 30 || (int64_t)n * B >= (int64_t)1 << 40)
        return sdnn_fail(SDNN_EINVAL, "a block of %d x %d values: n and B from 1 to 2^30 and less than 2^40 values are wanted", n, B);
    return SDNN_OK;
}
static size_t workspace(int n, int B)
{
    return (16 * (size_t)std::max(forward_ranges(n, B), backward_ranges(n)) * (size_t)B + 4 * (size_t)B + 255) & ~(size_t)255;
}
static int check_work(const void *d_work, size_t work_bytes, int32_t n, int32_t B)
{
    const int rc = check_norm(n, B);
    if (rc) return rc;
    if (!d_work) return sdnn_fail(SDNN_EINVAL, "d_work is NULL");
    if ((uintptr_t)d_work & 15) return sdnn_fail(SDNN_EINVAL, "d_work must be 16-byte aligned");
    if (work_bytes < workspace(n, B)) return sdnn_fail(SDNN_ENOMEM, "workspace of %zu bytes, %zu needed", work_bytes, workspace(n, B));
    return SDNN_OK;
}
static bool wide(int B, const void *a, const void *b) { return B % 4 == 0 && (((uintptr_t)a | (uintptr_t)b) & 15) == 0; }

extern "C" int sdnn_layernorm_workspace_bytes(int32_t n, int32_t B, size_t *bytes)
{
    if (!bytes) return sdnn_fail(SDNN_EINVAL, "bytes is NULL");
    const int rc = check_norm(n, B);
    if (rc) return rc;
    *bytes = workspace(n, B);
    return SDNN_OK;
}

template <int V>
static int forward(const float *x, const float *gamma, const float *beta, int n, int B, double eps, float *y, double *stats, void *work, hipStream_t stream)
{
    const int ranges = forward_ranges(n, B);
    const Shape sh = shape_for(n, B, V, ranges);
    double2 *part = (double2 *)work;
    float *firsts = (float *)(part + (size_t)ranges * B);
    const dim3 grid(tiles(sh, V), (unsigned)ranges);
    hipLaunchKernelGGL(k_norm_sums<V>, grid, dim3(NORM_THREADS), 0, stream, x, sh, part, firsts);
    hipLaunchKernelGGL(k_norm_apply<V>, grid, dim3(NORM_THREADS), 0, stream, x, gamma, beta, sh, eps, part, y, stats, ranges, firsts);
    return sdnn_launched();
}

extern "C" int sdnn_layernorm(const float *d_X, const float *d_gamma, const float *d_beta, int32_t n, int32_t B, double eps, float *d_Y,
                              double *d_stats, void *d_work, size_t work_bytes, void *stream)
{
    const int rc = check_work(d_work, work_bytes, n, B);
    if (rc) return rc;
    if (!d_X || !d_Y) return sdnn_fail(SDNN_EINVAL, "d_X or d_Y is NULL");
    if (!(eps > 0.0) || !(eps <= 1e30)) return sdnn_fail(SDNN_EINVAL, "eps must be > 0");
    return wide(B, d_X, d_Y) ? forward<4>(d_X, d_gamma, d_beta, n, B, eps, d_Y, d_stats, d_work, (hipStream_t)stream)
                             : forward<1>(d_X, d_gamma, d_beta, n, B, eps, d_Y, d_stats, d_work, (hipStream_t)stream);
}

template <int V, class Block>
static int backward(const float *dy, const Block &x, const double *stats, const float *gamma, int n, int B, float *dx, float *dgamma, float *dbeta, void *work,
                    hipStream_t stream)
{
    const int ranges = backward_ranges(n);
    Shape sh = shape_for(n, B, V, ranges);
    double2 *part = (double2 *)work;
    hipLaunchKernelGGL((k_norm_grad_sums<V, Block>), dim3((unsigned)range_rows(n, sh.rows)), dim3(NORM_THREADS), 0, stream, dy, x, stats, gamma, sh, part, dgamma, dbeta);
    const int used = range_rows(n, sh.rows); // ranges that have rows
    if (dx) {
        const int f = forward_ranges(n, B);
        sh.rows = range_rows(n, f);
        hipLaunchKernelGGL((k_norm_grad_apply<V, Block>), dim3(tiles(sh, V), (unsigned)f), dim3(NORM_THREADS), 0, stream, dy, x, stats, gamma, sh, part, used, dx);
    }
    return sdnn_launched();
}

static int check_backward(const float *d_dY, const double *d_stats, const float *d_dX, const float *d_dgamma, const float *d_dbeta)
{
    if (!d_dY || !d_stats) return sdnn_fail(SDNN_EINVAL, "d_dY or d_stats is NULL");
    if (!d_dX && !d_dgamma && !d_dbeta) return sdnn_fail(SDNN_EINVAL, "no result is asked for");
    return SDNN_OK;
}

extern "C" int sdnn_layernorm_backward(const float *d_dY, const float *d_X, const double *d_stats, const float *d_gamma, int32_t n, int32_t B, float *d_dX,
                                       float *d_dgamma, float *d_dbeta, void *d_work, size_t work_bytes, void *stream)
{
    int rc = check_work(d_work, work_bytes, n, B);
    if (!rc) rc = check_backward(d_dY, d_stats, d_dX, d_dgamma, d_dbeta);
    if (rc) return rc;
    if (!d_X) return sdnn_fail(SDNN_EINVAL, "d_X is NULL");
    const PlainBlock x{d_X};
    return wide(B, d_X, d_dY) && wide(B, d_dX, nullptr)
               ? backward<4>(d_dY, x, d_stats, d_gamma, n, B, d_dX, d_dgamma, d_dbeta, d_work, (hipStream_t)stream)
               : backward<1>(d_dY, x, d_stats, d_gamma, n, B, d_dX, d_dgamma, d_dbeta, d_work, (hipStream_t)stream);
}

extern "C" int sdnn_layernorm_backward_packed(const float *d_dY, const void *d_packed, size_t packed_bytes, float cap, const double *d_stats,
                                              const float *d_gamma, int32_t n, int32_t B, float *d_dX, float *d_dgamma, float *d_dbeta, void *d_work,
                                              size_t work_bytes, void *stream)
{
    int rc = check_work(d_work, work_bytes, n, B);
    if (!rc) rc = check_backward(d_dY, d_stats, d_dX, d_dgamma, d_dbeta);
    if (!rc) rc = sdnn_check_pack8(d_packed, packed_bytes, n, B, cap);
    if (rc) return rc;
    PackedBlock x;
    x.codes = (const uint8_t *)d_packed;
    x.scales = (const uint16_t *)(x.codes + PACK_GROUP * pack8_groups((int64_t)n * B));
    x.cap = cap; x.below = nextafterf(cap, 0.0f);
    return wide(B, d_dX, d_dY) ? backward<4>(d_dY, x, d_stats, d_gamma, n, B, d_dX, d_dgamma, d_dbeta, d_work, (hipStream_t)stream)
                               : backward<1>(d_dY, x, d_stats, d_gamma, n, B, d_dX, d_dgamma, d_dbeta, d_work, (hipStream_t)stream);
}
