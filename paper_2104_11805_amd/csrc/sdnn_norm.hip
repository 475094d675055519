// Layer norm over the neurons of each sample, forward and backward, on blocks [n][B].
//
// The sums of a sample run down a column of the block, those of gamma's and beta's gradients along a row.  Two launches each, over
// tiles of CL * 4 columns and a range of rows: the first leaves every tile's sums over its rows (back: and over its columns), the
// second adds up the sums of the tiles above and below (back: to the left and right) and writes the result.  A lane holds four
// neighbouring columns, CL lanes lie across a tile, the others of a wavefront over the rows; NORM_ROWS rows per thread are requested
// at a time.  Sums are fp64 and in a fixed order, a result is rounded once.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "sdnn_internal.h"
#include "sdnn_lanes.h"
#include "sdnn_pack8.h"

#define NORM_THREADS 512
#define NORM_ROWS 4

typedef float F4 __attribute__((ext_vector_type(4), aligned(4))); // 16 bytes at any multiple of 4
struct __attribute__((packed, aligned(1))) U1 { unsigned v; }; // 4 bytes anywhere

// A lane's four columns.  They end with the block's last column at the latest: the last lane's first ones may be its neighbour's, and
// are left out of everything.  SMALL: B < 4, one lane across.
template <int CL, bool SMALL> struct Columns {
    static constexpr bool small = SMALL;
    int tile0, base, first, B; // columns base .. base + 3, of which those from `first` on are the lane's own; none if first >= B
    __device__ __forceinline__ Columns(int tile, int B_)
    {
        B = B_;
        tile0 = tile * 4 * CL;
        first = tile0 + 4 * (int)(threadIdx.x & (CL - 1));
        base = SMALL ? 0 : min(first, B - 4);
    }
    __device__ __forceinline__ bool any() const { return first < B; }
    __device__ __forceinline__ bool whole() const { return !SMALL && base == first; }
    __device__ __forceinline__ bool own(int v) const { return SMALL ? v < B : base + v >= first; }
    __device__ __forceinline__ bool ragged() const { return SMALL || tile0 + 4 * CL > B; } // some lane of the tile is not whole (uniform)
};

// The block that is normalized, as it is ... (PAST: read past the caches, a block that they do not hold)
template <bool PAST> struct PlainBlock {
    const float *x;
    struct Raw { float v[4]; };
    template <class C> __device__ __forceinline__ void request(const C &c, size_t row, Raw &t) const
    {
        const float *p = x + row * (size_t)c.B + c.base;
        if constexpr (C::small) {
#pragma unroll
            for (int v = 0; v < 4; ++v) t.v[v] = v < c.B ? p[v] : 0.0f;
        } else {
            const F4 f = PAST ? __builtin_nontemporal_load(reinterpret_cast<const F4 *>(p)) : *reinterpret_cast<const F4 *>(p);
#pragma unroll
            for (int v = 0; v < 4; ++v) t.v[v] = f[v];
        }
    }
    __device__ __forceinline__ void values(const Raw &t, float (&x4)[4]) const
    {
#pragma unroll
        for (int v = 0; v < 4; ++v) x4[v] = t.v[v];
    }
};
// ... or in 8 bits: four codes, and the scales of the first and the last of them
struct PackedBlock {
    const uint8_t *codes;
    const uint16_t *scales;
    float cap, below;
    struct Raw { unsigned code; float scale[2]; int place; };
    template <class C> __device__ __forceinline__ void request(const C &c, size_t row, Raw &t) const
    {
        const size_t e = row * (size_t)c.B + c.base;
        const int last = C::small ? c.B - 1 : 3;
        if constexpr (C::small) {
            t.code = codes[e];
            for (int v = 1; v <= last; ++v) t.code |= (unsigned)codes[e + v] << (8 * v);
        } else {
            t.code = reinterpret_cast<const U1 *>(codes + e)->v;
        }
        t.place = (int)(e % PACK_GROUP);
        t.scale[0] = __uint_as_float((unsigned)scales[e / PACK_GROUP] << 16);
        t.scale[1] = __uint_as_float((unsigned)scales[(e + last) / PACK_GROUP] << 16);
    }
    __device__ __forceinline__ void values(const Raw &t, float (&x4)[4]) const
    {
#pragma unroll
        for (int v = 0; v < 4; ++v) x4[v] = pack8_value(t.code >> (8 * v) & 255u, t.place + v < PACK_GROUP ? t.scale[0] : t.scale[1], cap, below);
    }
};

// The sum of a value over the lanes that hold the same columns, in all of them.
template <int CL> __device__ __forceinline__ double add_rows(double v)
{
    if constexpr (CL <= 1) v += lane_xor<0>(v);
    if constexpr (CL <= 2) v += lane_xor<1>(v);
    if constexpr (CL <= 4) v += lane_xor<2>(v);
    if constexpr (CL <= 8) v += lane_xor<3>(v);
    if constexpr (CL <= 16) v = add_lane_xor<4>(v);
    if constexpr (CL <= 32) v = add_lane_xor<5>(v);
    return v;
}

// Stores the sums that the workgroup's threads have of their columns: part [B].
template <int CL, class C>
__device__ __forceinline__ void store_column_sums(const C &c, const double (&a)[4], const double (&b)[4], double2 *__restrict__ part)
{
    __shared__ double2 lds[NORM_THREADS / 64][4 * CL];
    const int tid = threadIdx.x;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const double2 s = make_double2(add_rows<CL>(a[v]), add_rows<CL>(b[v]));
        if ((tid & 63) < CL) lds[tid >> 6][4 * (tid & 63) + v] = s;
    }
    __syncthreads();
    const int col = c.tile0 + tid;
    if (tid < 4 * CL && col < c.B) {
        const int slot = 4 * (tid >> 2) + (col - max(0, min(c.tile0 + 4 * (tid >> 2), c.B - 4)));
        double2 s = lds[0][slot];
        for (int w = 1; w < NORM_THREADS / 64; ++w) {
            s.x += lds[w][slot].x;
            s.y += lds[w][slot].y;
        }
        part[col] = s;
    }
}

// The sums of all ranges for the tile's columns, put through `finish`; the results for the lane's columns.
template <int CL, class C, class F>
__device__ __forceinline__ void load_column_sums(const C &c, const double2 *__restrict__ part, int ranges, double (&a)[4], double (&b)[4], F finish)
{
    constexpr int CT = 4 * CL, K = NORM_THREADS / CT;
    __shared__ double2 lds[NORM_THREADS];
    const int tid = threadIdx.x, col = c.tile0 + (tid & (CT - 1));
    double2 s = make_double2(0.0, 0.0);
    if (col < c.B)
#pragma unroll 8
        for (int k = tid / CT; k < ranges; k += K) {
            const double2 t = part[(size_t)k * c.B + col];
            s.x += t.x;
            s.y += t.y;
        }
    lds[tid] = s;
    __syncthreads();
    if (tid < CT) {
        for (int k = 1; k < K; ++k) {
            s.x += lds[k * CT + tid].x;
            s.y += lds[k * CT + tid].y;
        }
        if (col < c.B) s = finish(col, s);
        lds[tid] = s;
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const double2 t = lds[max(0, min(c.base + v - c.tile0, CT - 1))];
        a[v] = t.x;
        b[v] = t.y;
    }
}

// The rows that a thread walks: its first one, and NORM_ROWS of them at a time, row_of<CL>(r, u), of those below r1.
template <int CL> __device__ __forceinline__ int first_row(int r0) { return r0 + (int)threadIdx.x / CL; }
template <int CL> __device__ __forceinline__ int row_of(int r, int u) { return r + u * (NORM_THREADS / CL); }
template <int CL> __device__ __forceinline__ int next_rows(int r) { return row_of<CL>(r, NORM_ROWS); }

struct NormArgs {
    int32_t n, B, rows;            // rows of a range
    int32_t tiles, ranges, splits; // tiles across; ranges; second launches: parts of a range
};
// Which part a workgroup takes.  Workgroup ids go round the XCDs: an XCD takes whole rows of the block (a tile's columns of all rows lie
// in the same few of an L2's channels), and in the second launch those that it had in the first.  Few ranges: any.
__device__ __forceinline__ bool find_tile(const NormArgs &a, int splits, int &tile, int &range, int &r0, int &r1)
{
    const unsigned across = (unsigned)a.tiles * (unsigned)splits, id = a.ranges < 8 ? blockIdx.x : blockIdx.x >> 3;
    range = (int)(id / across);
    if (a.ranges >= 8) range = 8 * range + (int)(blockIdx.x & 7);
    if (range >= a.ranges) return false;
    const unsigned at = id % across, split = at / (unsigned)a.tiles;
    tile = (int)(at % (unsigned)a.tiles);
    const int rows = (a.rows + splits - 1) / splits;
    r0 = min(a.n, range * a.rows + (int)split * rows);
    r1 = min(min(a.n, (range + 1) * a.rows), r0 + rows);
    return true;
}

// part [range][B]: sums of x - x0 and of its square, x0 the sample's first value: nothing cancels where the mean is large.
// firsts [B]: x0, which the second launch may write its results over.
template <int CL, bool SMALL, bool PAST>
__global__ void __launch_bounds__(NORM_THREADS) k_norm_sums(const float *__restrict__ x, const NormArgs a, double2 *__restrict__ part, float *__restrict__ firsts)
{
    int tile, range, r0, r1;
    if (!find_tile(a, 1, tile, range, r0, r1)) return;
    const Columns<CL, SMALL> c(tile, a.B);
    const PlainBlock<PAST> in{x};
    double s1[4] = {}, s2[4] = {};
    if (c.any()) {
        typename PlainBlock<PAST>::Raw first, t[NORM_ROWS];
        in.request(c, 0, first);
        if (range == 0 && (int)threadIdx.x < CL)
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (c.own(v)) firsts[c.base + v] = first.v[v];
        for (int r = first_row<CL>(r0); r < r1; r = next_rows<CL>(r)) {
#pragma unroll
            for (int u = 0; u < NORM_ROWS; ++u)
                if (row_of<CL>(r, u) < r1) in.request(c, row_of<CL>(r, u), t[u]);
#pragma unroll
            for (int u = 0; u < NORM_ROWS; ++u)
                if (row_of<CL>(r, u) < r1)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const double d = (double)t[u].v[v] - (double)first.v[v];
                        s1[v] += d;
                        s2[v] = fma(d, d, s2[v]);
                    }
        }
    }
    store_column_sums<CL>(c, s1, s2, part + (size_t)range * a.B);
}

template <class C> __device__ __forceinline__ void store_row(const C &c, float *p, const float (&o)[4])
{
    if (c.whole()) {
        __builtin_nontemporal_store(F4{o[0], o[1], o[2], o[3]}, reinterpret_cast<F4 *>(p));
    } else {
#pragma unroll
        for (int v = 0; v < 4; ++v)
            if (c.own(v)) p[v] = o[v];
    }
}

template <int CL, bool SMALL, bool PAST>
__global__ void __launch_bounds__(NORM_THREADS) k_norm_apply(const float *x, const float *__restrict__ gamma, const float *__restrict__ beta, const NormArgs a,
                                                             double eps, const double2 *__restrict__ part, const float *__restrict__ firsts, float *y,
                                                             double *__restrict__ stats)
{
    int tile, range, r0, r1;
    if (!find_tile(a, a.splits, tile, range, r0, r1)) return;
    const Columns<CL, SMALL> c(tile, a.B);
    const PlainBlock<PAST> in{x};
    struct Rows {
        typename PlainBlock<PAST>::Raw t[NORM_ROWS];
        float g[NORM_ROWS], b[NORM_ROWS];
    } now, next;
    auto request = [&](int r, Rows &w) {
#pragma unroll
        for (int u = 0; u < NORM_ROWS; ++u)
            if (row_of<CL>(r, u) < r1 && c.any()) {
                in.request(c, row_of<CL>(r, u), w.t[u]);
                w.g[u] = gamma ? gamma[row_of<CL>(r, u)] : 1.0f;
                w.b[u] = beta ? beta[row_of<CL>(r, u)] : 0.0f;
            }
    };
    int r = first_row<CL>(r0);
    request(r, now); // on their way while the sums are added up
    double mean[4], rstd[4];
    const double inv = 1.0 / (double)a.n;
    load_column_sums<CL>(c, part, a.ranges, mean, rstd, [&](int col, double2 s) {
        const double m = s.x * inv, var = s.y * inv - m * m;
        const double2 out = make_double2((double)firsts[col] + m, 1.0 / sqrt((var < 0.0 ? 0.0 : var) + eps)); // an infinity or NaN in a sample: NaN, and
        if (r0 == 0 && stats) {                                                                              // so is all of its result
            stats[col] = out.x;
            stats[a.B + col] = out.y;
        }
        return out;
    });
    if (!c.any()) return;
    for (; r < r1; r = next_rows<CL>(r), now = next) {
        request(next_rows<CL>(r), next);
#pragma unroll
        for (int u = 0; u < NORM_ROWS; ++u)
            if (row_of<CL>(r, u) < r1) {
                float o[4];
#pragma unroll
                for (int v = 0; v < 4; ++v) o[v] = (float)fma(((double)now.t[u].v[v] - mean[v]) * rstd[v], (double)now.g[u], (double)now.b[u]);
                store_row(c, y + (size_t)row_of<CL>(r, u) * a.B + c.base, o);
            }
    }
}

// Eight sums over the CL lanes of a row: afterwards p[0 ..] of a lane are those from `first` on, as many as the return value, and `keep`
// says whether it is the lane that has them to store.
template <int CL> __device__ __forceinline__ int add_columns(double (&p)[8], int lane, int &first, bool &keep)
{
    keep = true;
    if constexpr (CL == 1) {
        first = 0;
        return 8;
    } else if constexpr (CL == 4) {
        halve<8, 1>(p, lane);
        halve<4, 0>(p, lane);
        first = 2 * (2 * (lane >> 1 & 1) + (lane & 1));
        return 2;
    } else {
        constexpr int BIT = CL == 64 ? 5 : CL == 32 ? 4 : CL == 16 ? 3 : 2;
        halve<8, BIT>(p, lane);
        halve<4, BIT - 1>(p, lane);
        halve<2, BIT - 2>(p, lane);
        if constexpr (CL >= 64) p[0] += lane_exchange<2>(p[0]);
        if constexpr (CL >= 32) p[0] += lane_exchange<1>(p[0]);
        if constexpr (CL >= 16) p[0] += lane_exchange<0>(p[0]);
        first = 4 * (lane >> BIT & 1) + 2 * (lane >> (BIT - 1) & 1) + (lane >> (BIT - 2) & 1);
        keep = (lane & (CL / 8 - 1)) == 0;
        return 1;
    }
}

// Where the sums along the rows go: dgamma and dbeta, or (more than one tile across) row_part [tile][n][2].
struct RowSums {
    double *part;
    float *dgamma, *dbeta;
};

// part [range][B]: sums of g dY and of g dY h over the rows of a range, h = (x - mean) rstd; and the sums of dY h and dY over the
// tile's columns.
template <int CL, bool SMALL, bool PAST, class Block>
__global__ void __launch_bounds__(NORM_THREADS) k_norm_grad_sums(const float *__restrict__ dy, const Block x, const double *__restrict__ stats,
                                                                 const float *__restrict__ gamma, const NormArgs a, double2 *__restrict__ part, const RowSums rs)
{
    static_assert(NORM_ROWS == 4, "eight sums at a time");
    const int lane = threadIdx.x & 63;
    int tile, range, r0, r1;
    if (!find_tile(a, 1, tile, range, r0, r1)) return;
    const Columns<CL, SMALL> c(tile, a.B);
    const PlainBlock<PAST> up{dy};
    double p[4] = {}, q[4] = {}, mean[4] = {}, rstd[4] = {};
#pragma unroll
    for (int v = 0; v < 4; ++v)
        if (c.any() && c.own(v)) {
            mean[v] = stats[c.base + v];
            rstd[v] = stats[a.B + c.base + v];
        }
    for (int r = first_row<CL>(r0); r < r1; r = next_rows<CL>(r)) {
        typename PlainBlock<PAST>::Raw d[NORM_ROWS];
        typename Block::Raw t[NORM_ROWS];
        float g[NORM_ROWS];
#pragma unroll
        for (int u = 0; u < NORM_ROWS; ++u)
            if (row_of<CL>(r, u) < r1 && c.any()) {
                const size_t row = (size_t)row_of<CL>(r, u);
                up.request(c, row, d[u]);
                x.request(c, row, t[u]);
                g[u] = gamma ? gamma[row] : 1.0f;
            }
        double sum[8] = {};
#pragma unroll
        for (int u = 0; u < NORM_ROWS; ++u)
            if (row_of<CL>(r, u) < r1 && c.any()) {
                float xv[4];
                x.values(t[u], xv);
                if (c.ragged())
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        if (!c.own(v)) d[u].v[v] = xv[v] = 0.0f;
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const double h = ((double)xv[v] - mean[v]) * rstd[v], dv = (double)d[u].v[v], gd = (double)g[u] * dv;
                    p[v] += gd;
                    q[v] = fma(gd, h, q[v]);
                    sum[2 * u] = fma(dv, h, sum[2 * u]);
                    sum[2 * u + 1] += dv;
                }
            }
        int first;
        bool keep;
        const int n_sums = add_columns<CL>(sum, lane, first, keep);
        if (keep)
#pragma unroll
            for (int j = 0; j < n_sums; ++j) {
                const int u = (first + j) >> 1, w = (first + j) & 1;
                const size_t row = (size_t)row_of<CL>(r, u);
                if (row < (size_t)r1) {
                    if (rs.part) rs.part[2 * ((size_t)tile * a.n + row) + w] = sum[j];
                    else if (w == 0 && rs.dgamma) rs.dgamma[row] = (float)sum[j];
                    else if (w == 1 && rs.dbeta) rs.dbeta[row] = (float)sum[j];
                }
            }
    }
    store_column_sums<CL>(c, p, q, part + (size_t)range * a.B);
}

// rs.part: not NULL in the last launch over the tiles of a block with more than one across.
template <int CL, bool SMALL, bool PAST, class Block>
__global__ void __launch_bounds__(NORM_THREADS) k_norm_grad_apply(const float *dy, const Block x, const double *__restrict__ stats, const float *__restrict__ gamma,
                                                                  const NormArgs a, const double2 *__restrict__ part, float *dx, const RowSums rs)
{
    int tile, range, r0, r1;
    if (!find_tile(a, a.splits, tile, range, r0, r1)) return;
    if (rs.part) { // the rows' sums: every tile across adds up a share of the range's
        const int share = (r1 - r0 + a.tiles - 1) / a.tiles, e1 = 2 * min(r1, r0 + (tile + 1) * share);
        for (int e = 2 * (r0 + tile * share) + (int)threadIdx.x; e < e1; e += NORM_THREADS) {
            double s = 0.0;
#pragma unroll 4
            for (int k = 0; k < a.tiles; ++k) s += rs.part[2 * (size_t)k * a.n + e];
            float *out = e & 1 ? rs.dbeta : rs.dgamma;
            if (out) out[e >> 1] = (float)s;
        }
    }
    if (!dx) return;
    const Columns<CL, SMALL> c(tile, a.B);
    const PlainBlock<PAST> up{dy};
    struct Rows {
        typename PlainBlock<PAST>::Raw d[NORM_ROWS];
        typename Block::Raw t[NORM_ROWS];
        float g[NORM_ROWS];
    } now, next;
    auto request = [&](int r, Rows &w) {
#pragma unroll
        for (int u = 0; u < NORM_ROWS; ++u)
            if (row_of<CL>(r, u) < r1 && c.any()) {
                up.request(c, row_of<CL>(r, u), w.d[u]);
                x.request(c, row_of<CL>(r, u), w.t[u]);
                w.g[u] = gamma ? gamma[row_of<CL>(r, u)] : 1.0f;
            }
    };
    int r = first_row<CL>(r0);
    request(r, now); // on their way while the sums are added up
    double p[4], q[4], mean[4] = {}, rstd[4] = {};
    const double inv = 1.0 / (double)a.n;
    load_column_sums<CL>(c, part, a.ranges, p, q, [&](int, double2 s) { return make_double2(s.x * inv, s.y * inv); });
    if (!c.any()) return;
#pragma unroll
    for (int v = 0; v < 4; ++v)
        if (c.own(v)) {
            mean[v] = stats[c.base + v];
            rstd[v] = stats[a.B + c.base + v];
        }
    for (; r < r1; r = next_rows<CL>(r), now = next) {
        request(next_rows<CL>(r), next);
#pragma unroll
        for (int u = 0; u < NORM_ROWS; ++u)
            if (row_of<CL>(r, u) < r1) {
                float xv[4], o[4];
                x.values(now.t[u], xv);
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const double h = ((double)xv[v] - mean[v]) * rstd[v];
                    o[v] = (float)(rstd[v] * fma(-h, q[v], fma((double)now.g[u], (double)now.d[u].v[v], -p[v])));
                }
                store_row(c, dx + (size_t)row_of<CL>(r, u) * a.B + c.base, o);
            }
    }
}

// ---- host side ------------------------------------------------------------------------------------------------------------
static int across(int B) { return B < 4 ? 1 : B <= 16 ? 4 : B <= 32 ? 8 : B <= 64 ? 16 : B <= 128 ? 32 : 64; } // lanes, CL
static int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// Tiles: enough workgroups to fill the chip, but not so many ranges that their sums are a load to add up.
struct NormPlan {
    NormArgs a;
    int cl;
    bool past;
    size_t row_part, firsts, total; // bytes into the workspace
};
static NormPlan plan_norm(int n, int B)
{
    NormPlan p;
    NormArgs &a = p.a;
    a.n = n; a.B = B;
    p.past = (int64_t)n * B >= (int64_t)48 << 20;
    const int most = std::max(1, (int)std::sqrt(n / 4.0)); // the second launch reads 16 bytes per range and column, and 4 per row
    int unit;
    for (p.cl = across(B);; p.cl /= 2) { // narrower tiles where there would be few
        unit = NORM_ROWS * NORM_THREADS / p.cl;
        a.tiles = ceil_div(B, 4 * p.cl);
        a.rows = std::max(unit, ceil_div(ceil_div(n, std::max(1, std::min(most, 1024 / a.tiles))), unit) * unit);
        a.ranges = ceil_div(n, a.rows);
        if (p.cl <= 16 || (int64_t)a.tiles * a.ranges >= 256) break;
    }
    a.splits = 1;
    while (a.splits < 8 && (int64_t)a.ranges * a.tiles * a.splits < 512 && a.rows / (2 * a.splits) >= unit) a.splits *= 2;
    p.row_part = 16 * (size_t)a.ranges * (size_t)B;
    p.firsts = p.row_part + (a.tiles > 1 ? 16 * (size_t)a.tiles * (size_t)n : 0);
    p.total = (p.firsts + 4 * (size_t)B + 255) & ~(size_t)255;
    return p;
}
static dim3 norm_grid(const NormArgs &a, int splits) { return dim3((unsigned)(a.tiles * splits * (a.ranges < 8 ? a.ranges : (a.ranges + 7) & ~7))); }

static int check_norm(int32_t n, int32_t B)
{
    if (n < 1 || B < 1 || n > 1 << 30 || B > 1 << 30 || (int64_t)n * B >= (int64_t)1 << 40)
        return sdnn_fail(SDNN_EINVAL, "a block of %d x %d values: n and B from 1 to 2^30 and less than 2^40 values are wanted", n, B);
    return SDNN_OK;
}
static int check_work(const void *d_work, size_t work_bytes, int32_t n, int32_t B)
{
    const int rc = check_norm(n, B);
    if (rc) return rc;
    if (!d_work) return sdnn_fail(SDNN_EINVAL, "d_work is NULL");
    if ((uintptr_t)d_work & 15) return sdnn_fail(SDNN_EINVAL, "d_work must be 16-byte aligned");
    const size_t need = plan_norm(n, B).total;
    if (work_bytes < need) return sdnn_fail(SDNN_ENOMEM, "workspace of %zu bytes, %zu needed", work_bytes, need);
    return SDNN_OK;
}

extern "C" int sdnn_layernorm_workspace_bytes(int32_t n, int32_t B, size_t *bytes)
{
    if (!bytes) return sdnn_fail(SDNN_EINVAL, "bytes is NULL");
    const int rc = check_norm(n, B);
    if (rc) return rc;
    *bytes = plan_norm(n, B).total;
    return SDNN_OK;
}

template <int CL, bool SMALL, bool PAST>
static int forward(const float *x, const float *gamma, const float *beta, double eps, float *y, double *stats, void *work, const NormPlan &pl, hipStream_t stream)
{
    double2 *part = (double2 *)work;
    float *firsts = (float *)((char *)work + pl.firsts);
    const NormArgs &a = pl.a;
    hipLaunchKernelGGL((k_norm_sums<CL, SMALL, PAST>), norm_grid(a, 1), dim3(NORM_THREADS), 0, stream, x, a, part, firsts);
    hipLaunchKernelGGL((k_norm_apply<CL, SMALL, PAST>), norm_grid(a, a.splits), dim3(NORM_THREADS), 0, stream, x, gamma, beta, a, eps, part, firsts, y, stats);
    return sdnn_launched();
}

extern "C" int sdnn_layernorm(const float *d_X, const float *d_gamma, const float *d_beta, int32_t n, int32_t B, double eps, float *d_Y,
                              double *d_stats, void *d_work, size_t work_bytes, void *stream_)
{
    const int rc = check_work(d_work, work_bytes, n, B);
    if (rc) return rc;
    if (!d_X || !d_Y) return sdnn_fail(SDNN_EINVAL, "d_X or d_Y is NULL");
    if (!(eps > 0.0) || !(eps <= 1e30)) return sdnn_fail(SDNN_EINVAL, "eps must be > 0");
    const NormPlan pl = plan_norm(n, B);
    hipStream_t stream = (hipStream_t)stream_;
    switch (pl.cl) {
    case 1: return forward<1, true, false>(d_X, d_gamma, d_beta, eps, d_Y, d_stats, d_work, pl, stream);
    case 4: return forward<4, false, false>(d_X, d_gamma, d_beta, eps, d_Y, d_stats, d_work, pl, stream);
    case 8: return forward<8, false, false>(d_X, d_gamma, d_beta, eps, d_Y, d_stats, d_work, pl, stream);
    case 16: return forward<16, false, false>(d_X, d_gamma, d_beta, eps, d_Y, d_stats, d_work, pl, stream);
    case 32: return forward<32, false, false>(d_X, d_gamma, d_beta, eps, d_Y, d_stats, d_work, pl, stream);
    default:
        if (pl.past) return forward<64, false, true>(d_X, d_gamma, d_beta, eps, d_Y, d_stats, d_work, pl, stream);
        return forward<64, false, false>(d_X, d_gamma, d_beta, eps, d_Y, d_stats, d_work, pl, stream);
    }
}

template <int CL, bool SMALL, bool PAST, class Block>
static int backward(const float *dy, const Block &x, const double *stats, const float *gamma, float *dx, RowSums rs, void *work, const NormPlan &pl, hipStream_t stream)
{
    double2 *part = (double2 *)work;
    const NormArgs &a = pl.a;
    rs.part = a.tiles > 1 ? (double *)((char *)work + pl.row_part) : nullptr;
    hipLaunchKernelGGL((k_norm_grad_sums<CL, SMALL, PAST, Block>), norm_grid(a, 1), dim3(NORM_THREADS), 0, stream, dy, x, stats, gamma, a, part, rs);
    if (dx || rs.part)
        hipLaunchKernelGGL((k_norm_grad_apply<CL, SMALL, PAST, Block>), norm_grid(a, a.splits), dim3(NORM_THREADS), 0, stream, dy, x, stats, gamma, a, part, dx, rs);
    return sdnn_launched();
}
template <bool PACKED>
static int backward_any(const float *dy, const float *x, const PackedBlock &x8, const double *stats, const float *gamma, int n, int B, float *dx, float *dgamma,
                        float *dbeta, void *work, void *stream_)
{
    const NormPlan pl = plan_norm(n, B);
    const RowSums rs{nullptr, dgamma, dbeta};
    hipStream_t stream = (hipStream_t)stream_;
    auto go = [&](auto cl, auto small, auto past) {
        if constexpr (PACKED) return backward<cl.value, small.value, past.value>(dy, x8, stats, gamma, dx, rs, work, pl, stream);
        else return backward<cl.value, small.value, past.value>(dy, PlainBlock<past.value>{x}, stats, gamma, dx, rs, work, pl, stream);
    };
    const std::integral_constant<bool, true> yes;
    const std::integral_constant<bool, false> no;
    switch (pl.cl) {
    case 1: return go(std::integral_constant<int, 1>(), yes, no);
    case 4: return go(std::integral_constant<int, 4>(), no, no);
    case 8: return go(std::integral_constant<int, 8>(), no, no);
    case 16: return go(std::integral_constant<int, 16>(), no, no);
    case 32: return go(std::integral_constant<int, 32>(), no, no);
    default: return pl.past ? go(std::integral_constant<int, 64>(), no, yes) : go(std::integral_constant<int, 64>(), no, no);
    }
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
    return backward_any<false>(d_dY, d_X, PackedBlock(), d_stats, d_gamma, n, B, d_dX, d_dgamma, d_dbeta, d_work, stream);
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
    return backward_any<true>(d_dY, nullptr, x, d_stats, d_gamma, n, B, d_dX, d_dgamma, d_dbeta, d_work, stream);
}
