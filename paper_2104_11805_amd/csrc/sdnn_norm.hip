// Layer norm over the neurons of each sample, forward and backward, on blocks [n][B].
//
// The sums of a sample run down a column of the block, those of gamma's and beta's gradients along a row.  Two launches each, over
// tiles of CL * 4 columns and a range of rows: the first leaves every tile's sums over its rows (back: and over its columns), the
// second adds up the sums of the tiles above and below (back: to the left and right) and writes the result.  A lane holds four
// neighbouring columns, CL lanes lie across a tile, the others of a wavefront over the rows; NORM_ROWS rows per thread are requested
// at a time.  Sums are fp64 and in a fixed order, a result is rounded once.
//
// What bounds it: the block is read twice (one that the chip's registers do not hold has to be, and the caches give the second reading no more than
// memory does), 12 bytes a value forward, 20 back, 14.03 back from 8 bits.  16384 x 4096 forward 128 us, 6.3 TB/s of them; 8192 x 2048 back from 8 bits 44 us,
// 5.4 TB/s.  Blocks of up to a few hundred thousand values: two launches (an empty one 3.5 us) and two chains of loads.
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
    int tile0, B, lane_row;    // lane_row: of the rows that the wavefront has at a time
    int base, first;           // columns base .. base + 3, of which those from `first` on are the lane's own; none if first >= B
    __device__ __forceinline__ Columns(int tile, int B_)
    {
        B = B_;
        tile0 = tile * 4 * CL;
        first = tile0 + 4 * (int)(threadIdx.x & (CL - 1));
        base = SMALL ? 0 : min(first, B - 4);
        lane_row = (int)(threadIdx.x & 63) / CL;
    }
    __device__ __forceinline__ unsigned at() const { return (unsigned)(lane_row * B + base); } // from the start of the wavefront's first row

    __device__ __forceinline__ const float *in(const float *p) const { return (const float *)((const char *)p + 4u * at()); } // 32 bits beside a uniform address
    __device__ __forceinline__ float *in(float *p) const { return (float *)((char *)p + 4u * at()); }
    __device__ __forceinline__ bool any() const { return first < B; }
    __device__ __forceinline__ bool whole() const { return !SMALL && base == first; }
    __device__ __forceinline__ bool own(int v) const { return SMALL ? v < B : base + v >= first; }
    __device__ __forceinline__ bool ragged() const { return SMALL || tile0 + 4 * CL > B; } // some lane of the tile is not whole (uniform)
};

// The block that is normalized, as it is ... (PAST: read past the caches)
template <bool PAST> struct PlainBlock {
    const float *x;
    struct Raw { float v[4]; };
    // start: of the wavefront's first row
    template <class C> __device__ __forceinline__ void request(const C &c, size_t start, Raw &t) const
    {
        const float *p = c.in(x + start);
        if constexpr (C::small) {
#pragma unroll
            for (int v = 0; v < 4; ++v) t.v[v] = v < c.B ? p[v] : 0.0f;
        } else {
            const F4 f = PAST ? __builtin_nontemporal_load(reinterpret_cast<const F4 *>(p)) : *reinterpret_cast<const F4 *>(p);
#pragma unroll
            for (int v = 0; v < 4; ++v) t.v[v] = f[v];
        }
    }
    template <class C> __device__ __forceinline__ void values(const C &, const Raw &t, float (&x4)[4]) const
    {
#pragma unroll
        for (int v = 0; v < 4; ++v) x4[v] = t.v[v];
    }
};
// ... or in 8 bits: four codes, and the scales of the first and the last of them (the same where rows are whole fours)
struct PackedArgs {
    const uint8_t *codes;
    const uint16_t *scales;
    float cap, below;
};
template <bool SIGNED> struct PackedBlock : PackedArgs {
    struct Raw { unsigned code; float scale[2]; int place; };
    template <class C> __device__ __forceinline__ void request(const C &c, size_t start, Raw &t) const
    {
        const int last = C::small ? c.B - 1 : 3;
        const uint8_t *code = codes + start + c.at();
        const unsigned at = (unsigned)(start % PACK_GROUP) + c.at(); // from the first row's first group on
        const uint16_t *scale = scales + start / PACK_GROUP;
        if constexpr (C::small) {
            t.code = code[0];
            for (int v = 1; v <= last; ++v) t.code |= (unsigned)code[v] << (8 * v);
        } else {
            t.code = reinterpret_cast<const U1 *>(code)->v;
        }
        t.place = (int)(at % PACK_GROUP);
        t.scale[0] = __uint_as_float((unsigned)scale[at / PACK_GROUP] << 16);
        if (c.B & 3) t.scale[1] = __uint_as_float((unsigned)scale[(at + last) / PACK_GROUP] << 16);
    }
    template <class C> __device__ __forceinline__ void values(const C &c, const Raw &t, float (&x4)[4]) const
    {
        float scale[4] = {t.scale[0], t.scale[0], t.scale[0], t.scale[0]};
        if (c.B & 3)
#pragma unroll
            for (int v = 1; v < 4; ++v) scale[v] = t.place + v < PACK_GROUP ? t.scale[0] : t.scale[1];
#pragma unroll
        for (int v = 0; v < 4; ++v) x4[v] = pack8_value_of<SIGNED>(t.code >> (8 * v) & 255u, scale[v], cap, below);
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

// The sums of every step-th range from k on, eight of them requested at a time; part: of a column.
__device__ __forceinline__ double2 add_ranges(const double2 *__restrict__ part, int B, int k, int step, int ranges)
{
    double2 s = make_double2(0.0, 0.0);
    for (; k < ranges; k += 8 * step) {
        double2 t[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) t[u] = k + u * step < ranges ? part[(size_t)(k + u * step) * B] : make_double2(0.0, 0.0);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            s.x += t[u].x;
            s.y += t[u].y;
        }
    }
    return s;
}

// The sums of all ranges for the tile's columns, put through `finish`; the results for the lane's columns.  ready: there they are.
template <int CL, bool READY, class C, class F>
__device__ __forceinline__ void load_column_sums(const C &c, const double2 *__restrict__ part, int ranges, const double2 *__restrict__ ready, double (&a)[4],
                                                 double (&b)[4], F finish)
{
    constexpr int CT = 4 * CL, K = NORM_THREADS / CT;
    __shared__ double2 lds[NORM_THREADS];
    const int tid = threadIdx.x, col = c.tile0 + (tid & (CT - 1));
    if constexpr (READY) {
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const double2 t = ready[min(c.base + v, c.B - 1)];
            a[v] = t.x;
            b[v] = t.y;
        }
    } else {
        double2 s = make_double2(0.0, 0.0);
        if (col < c.B) s = add_ranges(part + col, c.B, tid / CT, K, ranges);
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
}

// The rows that a wavefront walks: from its first one on 64 / CL at a time, the lane's is lane_row further, and NORM_ROWS times that, row_of<CL>(r,
// u), are requested together.  r and where that row starts, e, are the same for the wavefront.
template <int CL> __device__ __forceinline__ int first_row(int r0) { return r0 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) * (64 / CL); }
template <int CL> __device__ __forceinline__ int row_of(int r, int u) { return r + u * (NORM_THREADS / CL); }
template <int CL> __device__ __forceinline__ int next_rows(int r) { return row_of<CL>(r, NORM_ROWS); }
// Whether all of them are there.  Then nothing is asked row by row: a condition around a row's loads has the compiler move what is done with
// them to where they are, and a row waits for the one before it.  Lanes without columns of their own read their neighbours'.
template <int CL> __device__ __forceinline__ bool full_rows(int r, int r1) { return row_of<CL>(r, NORM_ROWS - 1) + 64 / CL <= r1; }
typedef std::integral_constant<bool, true> Full;
typedef std::integral_constant<bool, false> Rest;
// gamma or beta of a row: `other`, which has n values and more, is read where there is none, and dropped where the value is used
__device__ __forceinline__ float of_row(const float *p, const float *other, int row) { return (p ? p : other)[row]; }
template <class C> __device__ __forceinline__ size_t first_start(const C &c, int r) { return (size_t)r * (size_t)c.B; }
template <int CL, class C> __device__ __forceinline__ size_t start_of(const C &c, size_t e, int u) { return e + (size_t)u * (NORM_THREADS / CL) * (size_t)c.B; }
template <int CL, class C> __device__ __forceinline__ size_t next_start(const C &c, size_t e) { return start_of<CL>(c, e, NORM_ROWS); }

struct NormArgs {
    int32_t n, B, rows;            // rows of a range
    int32_t tiles, ranges, splits; // tiles across; ranges; second launches: parts of a range
    double2 *ready;                // NULL, or [B]: the ranges' sums are added up by a launch between the two (k_norm_finish)
};

// A sample's mean and 1/sqrt(variance + eps) from its sums; an infinity or NaN in a sample: NaN, and so is all of its result.
__device__ __forceinline__ double2 statistics(double2 s, float first, double inv, double eps)
{
    const double m = s.x * inv, var = s.y * inv - m * m;
    return make_double2((double)first + m, 1.0 / sqrt((var < 0.0 ? 0.0 : var) + eps));
}

// The ranges' sums (back), added up and divided by n, where the second launch does not do it: 32 threads a column.  8192 x 2048 4.7 us, a launch's time.
#define FINISH_COLUMNS 16
__global__ void __launch_bounds__(512) k_norm_finish(const NormArgs a, const double2 *__restrict__ part)
{
    __shared__ double2 lds[512];
    const int tid = threadIdx.x, col = (int)blockIdx.x * FINISH_COLUMNS + (tid & (FINISH_COLUMNS - 1));
    double2 s = make_double2(0.0, 0.0);
    if (col < a.B) s = add_ranges(part + col, a.B, tid / FINISH_COLUMNS, 512 / FINISH_COLUMNS, a.ranges);
    lds[tid] = s;
    __syncthreads();
    if (tid >= FINISH_COLUMNS || col >= a.B) return;
#pragma unroll 8
    for (int k = FINISH_COLUMNS + tid; k < 512; k += FINISH_COLUMNS) {
        s.x += lds[k].x;
        s.y += lds[k].y;
    }
    const double inv = 1.0 / (double)a.n;
    a.ready[col] = make_double2(s.x * inv, s.y * inv);
}
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

// part [range][B]: sums of x - x0 and of its square, x0 the sample's first value: nothing cancels where the mean is large (an outlier of a
// sample of n values is sqrt(n) standard deviations off at most: the variance loses n 2^-53).  16384 x 4096 39 us: 6.9 TB/s.
// firsts [B]: x0, which the second launch may write its results over.
template <int CL, bool SMALL>
__global__ void __launch_bounds__(NORM_THREADS) k_norm_sums(const float *__restrict__ x, const NormArgs a, double2 *__restrict__ part, float *__restrict__ firsts)
{
    int tile, range, r0, r1;
    if (!find_tile(a, 1, tile, range, r0, r1)) return;
    const Columns<CL, SMALL> c(tile, a.B);
    const PlainBlock<false> in{x};
    double s1[4] = {}, s2[4] = {};
    float first[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) first[v] = x[min(c.base + v, a.B - 1)];
    if (range == 0 && (int)threadIdx.x < CL && c.any())
#pragma unroll
        for (int v = 0; v < 4; ++v)
            if (c.own(v)) firsts[c.base + v] = first[v];
    int r = first_row<CL>(r0);
    size_t e = first_start(c, r);
    auto rows = [&](auto full) {
        typename PlainBlock<false>::Raw t[NORM_ROWS];
#pragma unroll
        for (int u = 0; u < NORM_ROWS; ++u)
            if (full.value || row_of<CL>(r, u) + c.lane_row < r1) in.request(c, start_of<CL>(c, e, u), t[u]);
#pragma unroll
        for (int u = 0; u < NORM_ROWS; ++u)
            if (full.value || row_of<CL>(r, u) + c.lane_row < r1)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const double d = (double)t[u].v[v] - (double)first[v];
                    s1[v] += d;
                    s2[v] = fma(d, d, s2[v]);
                }
        r = next_rows<CL>(r);
        e = next_start<CL>(c, e);
    };
    while (full_rows<CL>(r, r1)) rows(Full());
    while (r < r1) rows(Rest());
    store_column_sums<CL>(c, s1, s2, part + (size_t)range * a.B);
}

template <bool PAST = true, class C> __device__ __forceinline__ void store_row(const C &c, float *p, const float (&o)[4])
{
    if (c.whole()) { // (not so for lanes without columns)
        if constexpr (PAST) __builtin_nontemporal_store(F4{o[0], o[1], o[2], o[3]}, reinterpret_cast<F4 *>(p));
        else *reinterpret_cast<F4 *>(p) = F4{o[0], o[1], o[2], o[3]};
    } else {
#pragma unroll
        for (int v = 0; v < 4; ++v)
            if (c.own(v)) p[v] = o[v];
    }
}

// 16384 x 4096 79 us: 6.8 TB/s, 4 bytes read and 4 written a value.
template <int CL, bool SMALL>
__global__ void __launch_bounds__(NORM_THREADS) k_norm_apply(const float *x, const float *__restrict__ gamma, const float *__restrict__ beta, const NormArgs a,
                                                             double eps, const double2 *__restrict__ part, const float *__restrict__ firsts, float *y,
                                                             double *__restrict__ stats)
{
    int tile, range, r0, r1;
    if (!find_tile(a, a.splits, tile, range, r0, r1)) return;
    const Columns<CL, SMALL> c(tile, a.B);
    const PlainBlock<false> in{x};
    int r = first_row<CL>(r0);
    size_t e = first_start(c, r);
    typename PlainBlock<false>::Raw t[NORM_ROWS];
    float g[NORM_ROWS], b[NORM_ROWS];
    auto request = [&](auto full) {
#pragma unroll
        for (int u = 0; u < NORM_ROWS; ++u)
            if (full.value || row_of<CL>(r, u) + c.lane_row < r1) {
                in.request(c, start_of<CL>(c, e, u), t[u]);
                g[u] = of_row(gamma, x, row_of<CL>(r, u) + c.lane_row);
                b[u] = of_row(beta, x, row_of<CL>(r, u) + c.lane_row);
            }
    };
    if (full_rows<CL>(r, r1)) request(Full()); // on their way while the sums are added up
    double mean[4], rstd[4];
    const double inv = 1.0 / (double)a.n;
    load_column_sums<CL, false>(c, part, a.ranges, nullptr, mean, rstd, [&](int col, double2 s) {
        const double2 out = statistics(s, firsts[col], inv, eps);
        if (r0 == 0 && stats) {
            stats[col] = out.x;
            stats[a.B + col] = out.y;
        }
        return out;
    });
    auto rows = [&](auto full) {
#pragma unroll
        for (int u = 0; u < NORM_ROWS; ++u)
            if (full.value || row_of<CL>(r, u) + c.lane_row < r1) {
                const double gd = gamma ? (double)g[u] : 1.0, bd = beta ? (double)b[u] : 0.0;
                float o[4];
#pragma unroll
                for (int v = 0; v < 4; ++v) o[v] = (float)fma(((double)t[u].v[v] - mean[v]) * rstd[v], gd, bd);
                store_row(c, c.in(y + start_of<CL>(c, e, u)), o);
            }
        r = next_rows<CL>(r);
        e = next_start<CL>(c, e);
    };
    while (full_rows<CL>(r, r1)) {
        rows(Full());
        if (full_rows<CL>(r, r1)) request(Full());
    }
    while (r < r1) {
        request(Rest());
        rows(Rest());
    }
}

// Blocks of so few rows that a workgroup holds all of them of CL * 4 columns in registers, ROWS per thread: one launch, and every value is read
// once.  LINES: results are stored past the caches, where rows start at multiples of 64 bytes (1024 x 4096 7.8 us, 9.8 through them); elsewhere the parts of a
// line that two workgroups write have to meet in a cache (1000 x 20001 45.5 us, 64.5 past it).
#define WHOLE_THREADS 1024
template <int CL, int ROWS, bool LINES>
__global__ void __launch_bounds__(WHOLE_THREADS) k_norm_whole(const float *x, const float *__restrict__ gamma, const float *__restrict__ beta, int n, int B, double eps,
                                                              double inv, float *y, double *__restrict__ stats)
{
    constexpr int CT = 4 * CL, WAVES = WHOLE_THREADS / 64, STEP = WHOLE_THREADS / CL;
    __shared__ double2 lds[WAVES][CT];
    // an XCD takes neighbouring columns: they share cache lines
    const int per = (int)gridDim.x >> 3, id = (int)blockIdx.x, tid = threadIdx.x;
    const Columns<CL, false> c(id < 8 * per ? (id & 7) * per + (id >> 3) : id, B);
    const int r = __builtin_amdgcn_readfirstlane(tid >> 6) * (64 / CL);
    // all that is read is requested before anything waits for it
    const int lane_first = c.tile0 + (tid & ~3), col = min(lane_first, B - 4) + (tid & 3); // of the statistics that this thread makes
    typename PlainBlock<false>::Raw t[ROWS];
    float first[4], g[ROWS], b[ROWS], own_first = 0.0f;
    if (tid < CT && lane_first < B) own_first = x[col];
#pragma unroll
    for (int v = 0; v < 4; ++v) first[v] = x[c.base + v];
#pragma unroll
    for (int u = 0; u < ROWS; ++u) { // (rows that are not there: the last one again)
        const int row = min(r + u * STEP + c.lane_row, n - 1);
        const F4 f = *reinterpret_cast<const F4 *>(x + (size_t)row * (size_t)B + (size_t)c.base);
#pragma unroll
        for (int v = 0; v < 4; ++v) t[u].v[v] = f[v];
        g[u] = of_row(gamma, x, row);
        b[u] = of_row(beta, x, row);
    }
    double s1[4] = {}, s2[4] = {};
#pragma unroll
    for (int u = 0; u < ROWS; ++u)
            if (r + u * STEP + c.lane_row < n) {
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const double d = (double)t[u].v[v] - (double)first[v];
                    s1[v] += d;
                    s2[v] = fma(d, d, s2[v]);
                }
                // added here: else the rows' values are converted ahead, which takes twice their registers
                asm volatile("" : "+v"(s1[0]), "+v"(s1[1]), "+v"(s1[2]), "+v"(s1[3]), "+v"(s2[0]), "+v"(s2[1]), "+v"(s2[2]), "+v"(s2[3]));
            }
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const double2 s = make_double2(add_rows<CL>(s1[v]), add_rows<CL>(s2[v]));
        if ((tid & 63) < CL) lds[tid >> 6][4 * (tid & 63) + v] = s;
    }
    __syncthreads();
    if (tid < CT) {
        double2 s = lds[0][tid];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) {
            s.x += lds[w][tid].x;
            s.y += lds[w][tid].y;
        }
        if (lane_first < B) {
            s = statistics(s, own_first, inv, eps);
            if (stats && col >= lane_first) {
                stats[col] = s.x;
                stats[B + col] = s.y;
            }
            lds[0][tid] = s;
        }
    }
    __syncthreads(); // (and y may be x: everyone has read all that it needs of it)
    if (!c.any()) return;
    double mean[4], rstd[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const double2 s = lds[0][4 * (tid & (CL - 1)) + v];
        mean[v] = s.x;
        rstd[v] = s.y;
    }
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
        const int row = r + u * STEP + c.lane_row;
        if (row < n) {
            const double gd = gamma ? (double)g[u] : 1.0, bd = beta ? (double)b[u] : 0.0;
            float o[4];
#pragma unroll
            for (int v = 0; v < 4; ++v) o[v] = (float)fma(((double)t[u].v[v] - mean[v]) * rstd[v], gd, bd);
            store_row<LINES>(c, y + (size_t)row * (size_t)B + (size_t)c.base, o);
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
// tile's columns.  From 8 bits 8192 x 2048 17.5 us: 4.8 TB/s, three fifths of the clocks instructions (eight fp64 ones and three to get a value out of its byte,
// and eight sums along the rows at a time, halved at every step: seven exchanges for all eight instead of six for each).
template <int CL, bool SMALL, bool PAST, class Block>
__global__ void __launch_bounds__(NORM_THREADS, 4) k_norm_grad_sums(const float *__restrict__ dy, const Block x, const double *__restrict__ stats,
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
    for (int v = 0; v < 4; ++v) {
        const int col = min(c.base + v, a.B - 1);
        const double m = stats[col], k = stats[a.B + col];
        mean[v] = c.own(v) ? m : 0.0; // (columns that are not the lane's own must add nothing to the rows' sums)
        rstd[v] = c.own(v) ? k : 0.0;
    }
    int r = first_row<CL>(r0);
    size_t e = first_start(c, r);
    auto rows = [&](auto full) {
        typename PlainBlock<PAST>::Raw d[NORM_ROWS];
        typename Block::Raw t[NORM_ROWS];
        float g[NORM_ROWS];
#pragma unroll
        for (int u = 0; u < NORM_ROWS; ++u)
            if (full.value || row_of<CL>(r, u) + c.lane_row < r1) {
                up.request(c, start_of<CL>(c, e, u), d[u]);
                x.request(c, start_of<CL>(c, e, u), t[u]);
                g[u] = of_row(gamma, dy, row_of<CL>(r, u) + c.lane_row);
            }
        double sum[8] = {};
#pragma unroll
        for (int u = 0; u < NORM_ROWS; ++u)
            if (full.value || row_of<CL>(r, u) + c.lane_row < r1) {
                const double gr = gamma ? (double)g[u] : 1.0;
                float xv[4];
                x.values(c, t[u], xv);
                if (c.ragged())
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        if (!c.own(v)) d[u].v[v] = xv[v] = 0.0f;
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const double h = ((double)xv[v] - mean[v]) * rstd[v], dv = (double)d[u].v[v], gd = gr * dv;
                    p[v] += gd;
                    q[v] = fma(gd, h, q[v]);
                    sum[2 * u] = fma(dv, h, sum[2 * u]);
                    sum[2 * u + 1] += dv;
                }
                // a row's values are made doubles when it is its turn, not all rows' ahead (registers)
                asm volatile("" : "+v"(p[0]), "+v"(p[1]), "+v"(p[2]), "+v"(p[3]), "+v"(q[0]), "+v"(q[1]), "+v"(q[2]), "+v"(q[3]));
            }
        int first;
        bool keep;
        const int n_sums = add_columns<CL>(sum, lane, first, keep);
        if (keep)
#pragma unroll
            for (int j = 0; j < n_sums; ++j) {
                const int u = (first + j) >> 1, w = (first + j) & 1;
                const int row = row_of<CL>(r, u) + c.lane_row;
                if (full.value || row < r1) {
                    if (rs.part) rs.part[2 * ((size_t)tile * a.n + row) + w] = sum[j];
                    else if (w == 0 && rs.dgamma) rs.dgamma[row] = (float)sum[j];
                    else if (w == 1 && rs.dbeta) rs.dbeta[row] = (float)sum[j];
                }
            }
        r = next_rows<CL>(r);
        e = next_start<CL>(c, e);
    };
    while (full_rows<CL>(r, r1)) rows(Full());
    while (r < r1) rows(Rest());
    store_column_sums<CL>(c, p, q, part + (size_t)range * a.B);
}

// rs.part: not NULL in the last launch over the tiles of a block with more than one across.  From 8 bits 8192 x 2048 24 us: 6.3 TB/s.
template <int CL, bool SMALL, bool PAST, bool READY, class Block>
__global__ void __launch_bounds__(NORM_THREADS, 4) k_norm_grad_apply(const float *dy, const Block x, const double *__restrict__ stats, const float *__restrict__ gamma,
                                                                  const NormArgs a, const double2 *__restrict__ part, float *dx, const RowSums rs)
{
    int tile, range, r0, r1;
    if (!find_tile(a, a.splits, tile, range, r0, r1)) return;
    if (rs.part) { // the rows' sums: every tile across adds up a share of the range's
        const int share = (r1 - r0 + a.tiles - 1) / a.tiles, end = 2 * min(r1, r0 + (tile + 1) * share);
        for (int i = 2 * (r0 + tile * share) + (int)threadIdx.x; i < end; i += NORM_THREADS) {
            double s = 0.0;
            for (int k = 0; k < a.tiles; k += 4) {
                double t[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) t[u] = k + u < a.tiles ? rs.part[2 * (size_t)(k + u) * a.n + i] : 0.0;
                s += (t[0] + t[1]) + (t[2] + t[3]);
            }
            float *out = i & 1 ? rs.dbeta : rs.dgamma;
            if (out) out[i >> 1] = (float)s;
        }
    }
    if (!dx) return;
    const Columns<CL, SMALL> c(tile, a.B);
    const PlainBlock<PAST> up{dy};
    int r = first_row<CL>(r0);
    size_t e = first_start(c, r);
    typename PlainBlock<PAST>::Raw d[NORM_ROWS];
    typename Block::Raw t[NORM_ROWS];
    float g[NORM_ROWS];
    auto request = [&](auto full) {
#pragma unroll
        for (int u = 0; u < NORM_ROWS; ++u)
            if (full.value || row_of<CL>(r, u) + c.lane_row < r1) {
                up.request(c, start_of<CL>(c, e, u), d[u]);
                x.request(c, start_of<CL>(c, e, u), t[u]);
                g[u] = of_row(gamma, dy, row_of<CL>(r, u) + c.lane_row);
            }
    };
    double mean[4] = {}, rstd[4] = {};
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const int col = min(c.base + v, a.B - 1);
        mean[v] = stats[col];
        rstd[v] = stats[a.B + col];
    }
    if (full_rows<CL>(r, r1)) request(Full()); // on their way while the sums are added up
    double p[4], q[4]; // dX = rstd (g dY - p - (x - mean) q): q becomes that constant of a column
    const double inv = 1.0 / (double)a.n;
    load_column_sums<CL, READY>(c, part, a.ranges, a.ready, p, q, [&](int, double2 s) { return make_double2(s.x * inv, s.y * inv); });
#pragma unroll
    for (int v = 0; v < 4; ++v) q[v] *= rstd[v];
    auto rows = [&](auto full) {
#pragma unroll
        for (int u = 0; u < NORM_ROWS; ++u)
            if (full.value || row_of<CL>(r, u) + c.lane_row < r1) {
                const double gr = gamma ? (double)g[u] : 1.0;
                float xv[4], o[4];
                x.values(c, t[u], xv);
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    o[v] = (float)(fma(mean[v] - (double)xv[v], q[v], fma(gr, (double)d[u].v[v], -p[v])) * rstd[v]);
                store_row(c, c.in(dx + start_of<CL>(c, e, u)), o);
            }
        r = next_rows<CL>(r);
        e = next_start<CL>(c, e);
    };
    while (full_rows<CL>(r, r1)) {
        rows(Full());
        if (full_rows<CL>(r, r1)) request(Full());
    }
    while (r < r1) {
        request(Rest());
        rows(Rest());
    }
}

// ---- host side ------------------------------------------------------------------------------------------------------------
static int across(int B) { return B < 4 ? 1 : B <= 16 ? 4 : B <= 32 ? 8 : B <= 64 ? 16 : B <= 128 ? 32 : 64; } // lanes, CL
static int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

#define MOST_COLUMNS (1 << 26) // of the launches with 32 threads a column: a launch holds less than 2^32
#define ROW_PAIRS (1 << 29) // columns up to which a wavefront may have two rows: a lane's offset, Columns::in, is 32 bits of bytes from the first of them (and 128 columns a tile of 512 threads make less than 2^32)
#define PAST_COUNT ((int64_t)48 << 20) // blocks of 200 MB and more that have tiles of 256 columns are read past the caches by the backward pass (16384 x 4096 244 us, 268 through them; forward 143, 128)
struct NormPlan {
    NormArgs a;
    int cl;
    bool past;
    size_t row_part, firsts, ready, total; // bytes into the workspace; ready 0: there is none
};
// Forward, and back over blocks of less than 7 << 20 values: 256 workgroups in the first launch, one a CU (264 take as long as 512), so the fewest ranges
// that fill the chip; every workgroup of the second adds up the ranges' sums for its columns, 16 bytes per range and column, which with 256 workgroups
// grow with the square of the tile's width, so few or narrow blocks have narrow tiles.  us at CL = 8 / 16 / 32 / 64: forward 65536 x 64 11.7 / 15.4 / 17.5 / 24.2,
// 16384 x 256 11.2 / 12.1 / 15.5 / 28.8, 3001 x 777 15.5 / 10.3 / 10.5 / 12.7, 37984 x 400 36 / 35 / 38 / 47, 16384 x 1024 38.4 / 36.1 / 36.4 / 39.5,
// 65536 x 1024 140 / 135 / 132 / 136; back (where a row's sums of many tiles have to be joined) 4001 x 160 9.7 / 9.4 / 10.0 / 13.1, 16384 x 256 17.8 / 16.9 /
// 20.1 / 33.8, 2100 x 3000 55 / 39 / 33 / 30.  As many parts of them as there are with up to 1024 workgroups in the second launch (at 256 / 512 / 1024 / 2048:
// 262144 x 64 37.8 / 36.9 / 35.8 / 39.9, 16384 x 1024 36.9 / 36.1 / 35.0 / 39.8).
// Back over larger blocks, two workgroups a CU in both launches, and the ranges' sums by a launch of their own (4 us).  That / the other way: 10007 x 777 from
// 8 bits 34.4 / 39.8, 5000 x 1500 25.1 / 27.9, 200000 x 40 36.2 / 39.5, 65536 x 1024 157 / 182; 20000 x 400 31.5 / 31.1, 16384 x 256 16.9 / 14.7.
static NormPlan plan_norm(int n, int B, bool back)
{
    NormPlan p;
    NormArgs &a = p.a;
    a.n = n; a.B = B; a.ready = nullptr;
    const int64_t count = (int64_t)n * B;
    const bool finish = back && B <= MOST_COLUMNS && count >= 7 << 20;
    p.cl = across(B);
    if (finish) {
        if (p.cl == 64 && 4 * ceil_div(B, 128) <= 6 * ceil_div(B, 256)) p.cl = 32; // a quarter of the lanes and more would have no columns
    } else {
        const bool large = (double)count * B >= 8.6e9;
        const int widest = (back && B >= 2048) || B > ROW_PAIRS ? 64 : large ? 32 : B > (back ? 160 : 256) ? 16 : n < 2048 ? 16 : 8; // (8: ranges of 256 rows and more, one an XCD)
        p.cl = std::min(p.cl, widest);
    }
    p.past = back && p.cl == 64 && count >= PAST_COUNT;
    const int unit = NORM_ROWS * NORM_THREADS / p.cl;
    a.tiles = ceil_div(B, 4 * p.cl);
    int ranges = std::max(1, (finish ? 512 : 256) / a.tiles);
    if (ranges > 8) ranges &= ~7; // as many for each XCD
    a.rows = ceil_div(ceil_div(n, unit), ranges) * unit;
    a.ranges = ceil_div(n, a.rows);
    a.splits = 1;
    for (int k = 2; k <= 16; ++k) // parts of whole units
        if (a.rows % (k * unit) == 0 && (int64_t)a.ranges * a.tiles * k <= (finish ? 512 : 1024)) a.splits = k;
    p.row_part = 16 * (size_t)a.ranges * (size_t)B;
    p.firsts = p.row_part + (back && a.tiles > 1 ? 16 * (size_t)a.tiles * (size_t)n : 0);
    p.total = p.firsts + (back ? 0 : 4 * (size_t)B);
    p.ready = 0;
    if (finish) {
        p.ready = (p.total + 15) & ~(size_t)15;
        p.total = p.ready + 16 * (size_t)B;
    }
    p.total = (p.total + 255) & ~(size_t)255;
    return p;
}
static size_t workspace(int n, int B) { return std::max(plan_norm(n, B, false).total, plan_norm(n, B, true).total); }
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
    const size_t need = workspace(n, B);
    if (work_bytes < need) return sdnn_fail(SDNN_ENOMEM, "workspace of %zu bytes, %zu needed", work_bytes, need);
    return SDNN_OK;
}

extern "C" int sdnn_layernorm_workspace_bytes(int32_t n, int32_t B, size_t *bytes)
{
    if (!bytes) return sdnn_fail(SDNN_EINVAL, "bytes is NULL");
    const int rc = check_norm(n, B);
    if (rc) return rc;
    *bytes = workspace(n, B);
    return SDNN_OK;
}

// Whether a block takes k_norm_whole: lanes across, or 0.  That / two launches, us: 1024 x 64 4.9 / 6.7, 1024 x 4096 7.8 / 11.6, 1000 x 70000 134 / 176,
// 2000 x 2000 8.9 / 11.3, 2048 x 6000 27.1 / 31.5, 2048 x 8192 45.7 / 35.1; with few rows most of a workgroup is idle: 64 x 2048 3.9 / 6.2, 100 x 10000
// 7.9 / 8.0, 100 x 100000 49.8 / 26.8.  Up to 1024 rows over 4096 columns and more 32 columns a workgroup, whole lines, and 8 rows a thread.
static int whole_lanes(int n, int B)
{
    if (B < 4 || B > MOST_COLUMNS || n > 2048 || (n > 1024 && (int64_t)n * B >= 16 << 20) || (n < 128 && B > 8192)) return 0;
    return n <= 1024 && B >= 4096 ? 8 : 4;
}
template <int CL, int ROWS>
static int forward_whole(const float *x, const float *gamma, const float *beta, int n, int B, double eps, float *y, double *stats, hipStream_t stream)
{
    const dim3 grid((unsigned)ceil_div(B, 4 * CL)), block(WHOLE_THREADS);
    if (B % 16 == 0) hipLaunchKernelGGL((k_norm_whole<CL, ROWS, true>), grid, block, 0, stream, x, gamma, beta, n, B, eps, 1.0 / (double)n, y, stats);
    else hipLaunchKernelGGL((k_norm_whole<CL, ROWS, false>), grid, block, 0, stream, x, gamma, beta, n, B, eps, 1.0 / (double)n, y, stats);
    return sdnn_launched();
}
template <int CL, bool SMALL>
static int forward(const float *x, const float *gamma, const float *beta, double eps, float *y, double *stats, void *work, const NormPlan &pl, hipStream_t stream)
{
    double2 *part = (double2 *)work;
    float *firsts = (float *)((char *)work + pl.firsts);
    const NormArgs &a = pl.a;
    hipLaunchKernelGGL((k_norm_sums<CL, SMALL>), norm_grid(a, 1), dim3(NORM_THREADS), 0, stream, x, a, part, firsts);
    hipLaunchKernelGGL((k_norm_apply<CL, SMALL>), norm_grid(a, a.splits), dim3(NORM_THREADS), 0, stream, x, gamma, beta, a, eps, part, firsts, y, stats);
    return sdnn_launched();
}

extern "C" int sdnn_layernorm(const float *d_X, const float *d_gamma, const float *d_beta, int32_t n, int32_t B, double eps, float *d_Y,
                              double *d_stats, void *d_work, size_t work_bytes, void *stream_)
{
    const int rc = check_work(d_work, work_bytes, n, B);
    if (rc) return rc;
    if (!d_X || !d_Y) return sdnn_fail(SDNN_EINVAL, "d_X or d_Y is NULL");
    if (!(eps > 0.0) || !(eps <= 1e30)) return sdnn_fail(SDNN_EINVAL, "eps must be > 0 and at most 1e30");
    const NormPlan pl = plan_norm(n, B, false);
    hipStream_t stream = (hipStream_t)stream_;
    switch (whole_lanes(n, B)) {
    case 4:
        return n <= 1024 ? forward_whole<4, 4>(d_X, d_gamma, d_beta, n, B, eps, d_Y, d_stats, stream)
                         : forward_whole<4, 8>(d_X, d_gamma, d_beta, n, B, eps, d_Y, d_stats, stream);
    case 8: return forward_whole<8, 8>(d_X, d_gamma, d_beta, n, B, eps, d_Y, d_stats, stream);
    }
    switch (pl.cl) {
    case 1: return forward<1, true>(d_X, d_gamma, d_beta, eps, d_Y, d_stats, d_work, pl, stream);
    case 4: return forward<4, false>(d_X, d_gamma, d_beta, eps, d_Y, d_stats, d_work, pl, stream);
    case 8: return forward<8, false>(d_X, d_gamma, d_beta, eps, d_Y, d_stats, d_work, pl, stream);
    case 16: return forward<16, false>(d_X, d_gamma, d_beta, eps, d_Y, d_stats, d_work, pl, stream);
    case 32: return forward<32, false>(d_X, d_gamma, d_beta, eps, d_Y, d_stats, d_work, pl, stream);
    default: return forward<64, false>(d_X, d_gamma, d_beta, eps, d_Y, d_stats, d_work, pl, stream);
    }
}

template <int CL, bool SMALL, bool PAST, class Block>
static int backward(const float *dy, const Block &x, const double *stats, const float *gamma, float *dx, RowSums rs, void *work, const NormPlan &pl, hipStream_t stream)
{
    double2 *part = (double2 *)work;
    NormArgs a = pl.a;
    a.ready = pl.ready ? (double2 *)((char *)work + pl.ready) : nullptr;
    rs.part = a.tiles > 1 ? (double *)((char *)work + pl.row_part) : nullptr;
    hipLaunchKernelGGL((k_norm_grad_sums<CL, SMALL, PAST, Block>), norm_grid(a, 1), dim3(NORM_THREADS), 0, stream, dy, x, stats, gamma, a, part, rs);
    if (dx && a.ready) {
        hipLaunchKernelGGL(k_norm_finish, dim3((unsigned)ceil_div(a.B, FINISH_COLUMNS)), dim3(512), 0, stream, a, part);
        hipLaunchKernelGGL((k_norm_grad_apply<CL, SMALL, PAST, true, Block>), norm_grid(a, a.splits), dim3(NORM_THREADS), 0, stream, dy, x, stats, gamma, a, part, dx, rs);
    } else if (dx || rs.part) {
        hipLaunchKernelGGL((k_norm_grad_apply<CL, SMALL, PAST, false, Block>), norm_grid(a, a.splits), dim3(NORM_THREADS), 0, stream, dy, x, stats, gamma, a, part, dx, rs);
    }
    return sdnn_launched();
}
// KIND 0: x; 1 and 2: x8, of values of both signs and of activations
template <int KIND>
static int backward_any(const float *dy, const float *x, const PackedArgs &x8, const double *stats, const float *gamma, int n, int B, float *dx, float *dgamma,
                        float *dbeta, void *work, void *stream_)
{
    const NormPlan pl = plan_norm(n, B, true);
    const RowSums rs{nullptr, dgamma, dbeta};
    hipStream_t stream = (hipStream_t)stream_;
    auto go = [&](auto cl, auto small, auto past) {
        if constexpr (KIND > 0) return backward<cl.value, small.value, past.value>(dy, PackedBlock<KIND == 1>{x8}, stats, gamma, dx, rs, work, pl, stream);
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
    return backward_any<0>(d_dY, d_X, PackedArgs(), d_stats, d_gamma, n, B, d_dX, d_dgamma, d_dbeta, d_work, stream);
}

extern "C" int sdnn_layernorm_backward_packed(const float *d_dY, const void *d_packed, size_t packed_bytes, float cap, const double *d_stats,
                                              const float *d_gamma, int32_t n, int32_t B, float *d_dX, float *d_dgamma, float *d_dbeta, void *d_work,
                                              size_t work_bytes, void *stream)
{
    int rc = check_work(d_work, work_bytes, n, B);
    if (!rc) rc = check_backward(d_dY, d_stats, d_dX, d_dgamma, d_dbeta);
    if (!rc) rc = sdnn_check_pack8(d_packed, packed_bytes, n, B, cap);
    if (rc) return rc;
    PackedArgs x;
    x.codes = (const uint8_t *)d_packed;
    x.scales = (const uint16_t *)(x.codes + PACK_GROUP * pack8_groups((int64_t)n * B));
    x.cap = cap; x.below = nextafterf(cap, 0.0f);
    return cap > 0.0f ? backward_any<2>(d_dY, nullptr, x, d_stats, d_gamma, n, B, d_dX, d_dgamma, d_dbeta, d_work, stream)
                      : backward_any<1>(d_dY, nullptr, x, d_stats, d_gamma, n, B, d_dX, d_dgamma, d_dbeta, d_work, stream);
}
