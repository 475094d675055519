// Activations in 8 bits (sdnn_pack8.h): single blocks, and X_0 .. X_L of a training net in one launch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "sdnn_internal.h"
#include "sdnn_pack8.h"

typedef float F4 __attribute__((ext_vector_type(4), aligned(4))); // 16 bytes at any multiple of 4
struct __attribute__((packed, aligned(1))) U1 { unsigned v; };     // 4 bytes anywhere

// The largest of a value >= 0, as bits, over a half of the wavefront, in all of its lanes.  (Whole numbers: the exchange is part of the comparison.)
__device__ __forceinline__ unsigned largest_of_half(unsigned v)
{
    v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, true)); // row_ror:8
    v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, true)); // row_half_mirror
    v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, true));  // quad_perm
    v = max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, true));
    const auto t = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return max(t[0], t[1]);
}
// A wavefront's half packs one group: lane g of 32 holds its values 4 g .. 4 g + 3.
template <bool SIGNED> __device__ __forceinline__ void pack_group(const float (&x)[4], float cap, int lane, uint8_t *codes, uint16_t *scale)
{
    int largest = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) largest = max(largest, __float_as_int(pack8_size<SIGNED>(x[k], cap))); // (below zero: less than zero as bits too)
    const unsigned t = pack8_scale<SIGNED>(__uint_as_float(largest_of_half((unsigned)largest)));
    const double inverse = pack8_inverse(t);
    unsigned c = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) c |= pack8_code<SIGNED>(x[k], cap, inverse) << (8 * k);
    reinterpret_cast<unsigned *>(codes)[lane] = c;
    if (lane == 0) *scale = (uint16_t)t;
}

// What bounds it: 4 bytes read and one written a value.  A wavefront's half has two groups of the workgroup's stretch of 8 KB requested at a time, and reads past
// the caches, so that they are left to the codes.  65536 x 1024 66 us by itself (5.1 TB/s), 65536 x 4096 252.  With k_unpack8 after it, which reads part of the codes from
// the caches, 104 to 110 us (6.1 to 6.5 TB/s) and 436; through the caches 111 and 489, one group at a time strided by the grid 115 and 560.  Codes stored past the caches as
// well: 3 us less here, but 20 more in k_unpack8.
template <bool SIGNED>
__global__ void __launch_bounds__(256) k_pack8(const float *__restrict__ x, int64_t count, int64_t groups, float cap, uint8_t *__restrict__ packed)
{
    const int lane = threadIdx.x & 31;
    uint16_t *scales = reinterpret_cast<uint16_t *>(packed + PACK_GROUP * groups);
    constexpr int U = 2, NEXT = 8;
    const int64_t whole = count / PACK_GROUP;
    int64_t g = (int64_t)blockIdx.x * (U * NEXT) + (threadIdx.x >> 5);
    for (; g < whole; g += (int64_t)gridDim.x * (U * NEXT)) {
        F4 f[U];
#pragma unroll
        for (int u = 0; u < U; ++u) f[u] = __builtin_nontemporal_load(reinterpret_cast<const F4 *>(x + (PACK_GROUP * min(g + u * NEXT, whole - 1) + 4 * lane)));
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (g + u * NEXT < whole) {
                const float v[4] = {f[u][0], f[u][1], f[u][2], f[u][3]};
                pack_group<SIGNED>(v, cap, lane, packed + PACK_GROUP * (g + u * NEXT), scales + g + u * NEXT);
            }
    }
    if (whole < groups && blockIdx.x == 0 && threadIdx.x < 32) { // the block's end: zeros after it
        const int64_t e = PACK_GROUP * whole + 4 * lane;
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = e + k < count ? x[e + k] : 0.0f;
        pack_group<SIGNED>(v, cap, lane, packed + PACK_GROUP * whole, scales + whole);
    }
}

// One piece of four values a thread, stored past the caches.  What bounds it: one byte read and 4 written a value; 65536 x 1024 47 us (7.2 TB/s).
template <bool SIGNED>
__global__ void __launch_bounds__(256) k_unpack8(const uint8_t *__restrict__ packed, int64_t count, int64_t groups, float cap, float below, float *__restrict__ x, int64_t first)
{
    const int64_t q = first + (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (4 * q >= count) return;
    const unsigned c = reinterpret_cast<const unsigned *>(packed)[q];
    const float t = __uint_as_float((unsigned)reinterpret_cast<const uint16_t *>(packed + PACK_GROUP * groups)[q / (PACK_GROUP / 4)] << 16);
    float v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = pack8_value_of<SIGNED>(c >> (8 * k) & 255u, t, cap, below);
    if (4 * q + 4 <= count) {
        __builtin_nontemporal_store(F4{v[0], v[1], v[2], v[3]}, reinterpret_cast<F4 *>(x + 4 * q));
    } else {
#pragma unroll
        for (int k = 0; k < 3; ++k)
            if (4 * q + k < count) x[4 * q + k] = v[k];
    }
}

// X_0 .. X_L of a training net, rows of ld floats, to and from one packed block after the other.  grid = (parts, blocks): blockIdx.y + l0 is l.
// What bounds it: 4 bytes a value on one side, one on the other, after the chain from the layer's record to the block.  4 layers of 65536 neurons, 64 samples 24.4 us
// into it and 17.7 out of it (4.3 and 5.9 TB/s), 16384 neurons and 255 samples (rows that are not whole fours) 31 and 26; 8 layers of 4096, 128 samples 8.1 and 6.1.
struct NetBlocks {
    const LayerDev *layers;
    float *x0;
    int32_t B, Bp, ld;
    float cap, below;
    uint8_t *packed;
    int32_t per_row;     // out of a checkpoint: pieces of four samples in a row
    double per_row_inv;  // 1 / that; into one: 1 / B
};
// i / d for i + 1 < 2^51: the quotient of i + 1/2, which is half of 1/d and more away from whole numbers
__device__ __forceinline__ int64_t quotient(int64_t i, double inv) { return (int64_t)fma((double)i, inv, 0.5 * inv); }
// Where X_l's packed block starts: the sizes of those before it, added up by the lanes.
__device__ __forceinline__ int64_t block_start(const NetBlocks &a, int l, int lane)
{
    int64_t bytes = 0;
    for (int k = lane; k < l; k += 64) {
        const int64_t count = (int64_t)(k == 0 ? a.layers[0].n_in : a.layers[k - 1].n_out) * a.B;
        bytes += ((PACK_GROUP + 2) * ((count + PACK_GROUP - 1) / PACK_GROUP) + 255) & ~(int64_t)255;
    }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) bytes += __shfl_xor(bytes, m);
    return bytes;
}
// (Loads of several groups or pieces together, at places that are there, without conditions between them.)
template <bool SIGNED> __device__ __forceinline__ void pack_block(const NetBlocks &a, const float *__restrict__ x, int64_t count, uint8_t *__restrict__ packed)
{
    const int lane = threadIdx.x & 31;
    const int64_t groups = (count + PACK_GROUP - 1) / PACK_GROUP, stride = (int64_t)gridDim.x * 8;
    uint16_t *scales = reinterpret_cast<uint16_t *>(packed + PACK_GROUP * groups);
    const bool dense = a.ld == a.B;
    const int64_t wide = dense || (a.B & 3) == 0 ? count / PACK_GROUP : 0; // groups whose fours lie in one piece
    constexpr int U = 2, NEXT = 8;
    int64_t g = (int64_t)blockIdx.x * (U * NEXT) + (threadIdx.x >> 5);
    for (; g < wide; g += U * stride) {
        F4 f[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t e = PACK_GROUP * min(g + u * NEXT, wide - 1) + 4 * lane, row = dense ? 0 : quotient(e, a.per_row_inv);
            f[u] = *reinterpret_cast<const F4 *>(x + (e + row * (a.ld - a.B)));
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (g + u * NEXT < wide) {
                const float v[4] = {f[u][0], f[u][1], f[u][2], f[u][3]};
                pack_group<SIGNED>(v, a.cap, lane, packed + PACK_GROUP * (g + u * NEXT), scales + g + u * NEXT);
            }
    }
    // the others; each is the next of somebody's
    for (g = wide + ((int64_t)blockIdx.x * 8 + (threadIdx.x >> 5)); g < groups; g += stride) {
        const int64_t e = PACK_GROUP * g + 4 * lane;
        int64_t row = quotient(e, a.per_row_inv), s = e - row * a.B;
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[k] = e + k < count ? x[row * a.ld + s] : 0.0f;
            if (++s == a.B) { s = 0; ++row; }
        }
        pack_group<SIGNED>(v, a.cap, lane, packed + PACK_GROUP * g, scales + g);
    }
}
__global__ void __launch_bounds__(256) k_pack_net(const NetBlocks a, int l0)
{
    const int l = l0 + (int)blockIdx.y;
    uint8_t *packed = a.packed + block_start(a, l, threadIdx.x & 63);
    if (l == 0) pack_block<true>(a, a.x0, (int64_t)a.layers[0].n_in * a.B, packed);
    else pack_block<false>(a, a.layers[l - 1].X, (int64_t)a.layers[l - 1].n_out * a.B, packed);
}
// Columns B .. Bp - 1 become zeros, as the passes leave them.  A piece of four samples of a row holds one of the batch at least; the four bytes
// from its first one on lie in the block, also where they run into its scales.
template <bool SIGNED> __device__ __forceinline__ void unpack_block(const NetBlocks &a, float *__restrict__ x, int64_t n, const uint8_t *__restrict__ packed)
{
    const int64_t groups = (n * a.B + PACK_GROUP - 1) / PACK_GROUP, pieces = n * a.per_row, stride = (int64_t)gridDim.x * 256;
    const uint16_t *scales = reinterpret_cast<const uint16_t *>(packed + PACK_GROUP * groups);
    constexpr int U = 4;
    if (a.ld == a.B && (a.B & 3) == 0) { // rows without gaps, of whole fours: as a block
        for (int64_t q = (int64_t)blockIdx.x * (U * 256) + threadIdx.x; q < pieces; q += U * stride) {
            unsigned c[U];
            uint16_t t[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t p = min(q + u * 256, pieces - 1);
                c[u] = reinterpret_cast<const unsigned *>(packed)[p];
                t[u] = scales[p / (PACK_GROUP / 4)];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (q + u * 256 >= pieces) break;
                const float scale = __uint_as_float((unsigned)t[u] << 16);
                F4 v;
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = pack8_value_of<SIGNED>(c[u] >> (8 * k) & 255u, scale, a.cap, a.below);
                *reinterpret_cast<F4 *>(x + 4 * (q + u * 256)) = v;
            }
        }
        return;
    }
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < pieces; q += U * stride) {
        unsigned c[U];
        uint16_t t[U][2];
        int64_t at[U];
        int have[U], place[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t p = min(q + u * stride, pieces - 1), row = quotient(p, a.per_row_inv), s = 4 * (p - row * a.per_row), e = row * a.B + s;
            have[u] = (int)min((int64_t)4, a.B - s);
            at[u] = row * a.ld + s;
            place[u] = (int)(e % PACK_GROUP);
            c[u] = reinterpret_cast<const U1 *>(packed + e)->v;
            t[u][0] = scales[e / PACK_GROUP];
            t[u][1] = scales[(e + have[u] - 1) / PACK_GROUP];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (q + u * stride >= pieces) break;
            float v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float scale = __uint_as_float((unsigned)(place[u] + k < PACK_GROUP ? t[u][0] : t[u][1]) << 16);
                v[k] = k < have[u] ? pack8_value_of<SIGNED>(c[u] >> (8 * k) & 255u, scale, a.cap, a.below) : 0.0f;
            }
            if (a.Bp >= 4 * a.per_row) { // room for whole pieces
                *reinterpret_cast<F4 *>(x + at[u]) = F4{v[0], v[1], v[2], v[3]};
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (k < have[u]) x[at[u] + k] = v[k];
            }
        }
    }
}
__global__ void __launch_bounds__(256) k_unpack_net(const NetBlocks a, int l0)
{
    const int l = l0 + (int)blockIdx.y;
    const uint8_t *packed = a.packed + block_start(a, l, threadIdx.x & 63);
    if (l == 0) unpack_block<true>(a, a.x0, a.layers[0].n_in, packed);
    else unpack_block<false>(a, a.layers[l - 1].X, a.layers[l - 1].n_out, packed);
}

// The launches that sdnn_checkpoint_save (restore = 0) and _load make; the return value is a hipError_t.
int sdnn_launch_checkpoint(const LayerDev *d_layers, float *d_x0, int32_t n_layers, int64_t max_n, int32_t B, int32_t Bp, int32_t ld, float cap,
                           void *d_ckpt, int restore, void *stream)
{
    NetBlocks a;
    a.layers = d_layers; a.x0 = d_x0; a.B = B; a.Bp = Bp; a.ld = ld; a.cap = cap; a.below = nextafterf(cap, 0.0f);
    a.packed = (uint8_t *)d_ckpt;
    a.per_row = (Bp + 3) / 4;
    a.per_row_inv = 1.0 / (restore ? a.per_row : B);
    // workgroups that stay: each has to find its block's start first
    const int64_t work = restore ? (max_n * a.per_row + 1023) / 1024 : (max_n * B + 2047) / 2048;
    const unsigned gx = (unsigned)std::min<int64_t>(std::max<int64_t>(work, 1), std::max(32, 4096 / (n_layers + 1)));
    for (int l0 = 0; l0 <= n_layers; l0 += 65535) {
        const dim3 grid(gx, (unsigned)std::min(65535, n_layers + 1 - l0));
        if (restore) hipLaunchKernelGGL(k_unpack_net, grid, dim3(256), 0, (hipStream_t)stream, a, l0);
        else hipLaunchKernelGGL(k_pack_net, grid, dim3(256), 0, (hipStream_t)stream, a, l0);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return (int)e;
    }
    return 0;
}

static int check_block(int32_t n, int32_t B)
{
    if (n < 0 || B < 1 || (int64_t)n * B >= (int64_t)1 << 40)
        return sdnn_fail(SDNN_EINVAL, "a block of %d x %d values: n >= 0, B >= 1 and less than 2^40 values are wanted", n, B);
    return SDNN_OK;
}

extern "C" int sdnn_pack8_bytes(int32_t n, int32_t B, size_t *bytes)
{
    if (!bytes) return sdnn_fail(SDNN_EINVAL, "bytes is NULL");
    const int rc = check_block(n, B);
    if (rc) return rc;
    *bytes = (size_t)pack8_bytes((int64_t)n * B);
    return SDNN_OK;
}

int sdnn_check_pack8(const void *d_packed, size_t packed_bytes, int32_t n, int32_t B, float cap)
{
    const int rc = check_block(n, B);
    if (rc) return rc;
    if (!(cap >= 0.0f)) return sdnn_fail(SDNN_EINVAL, "cap must be 0 (values of both signs) or > 0");
    if (n == 0) return SDNN_OK;
    if (!d_packed) return sdnn_fail(SDNN_EINVAL, "d_packed is NULL");
    if ((uintptr_t)d_packed & 15) return sdnn_fail(SDNN_EINVAL, "d_packed must be 16-byte aligned");
    if (packed_bytes < (size_t)pack8_bytes((int64_t)n * B))
        return sdnn_fail(SDNN_ENOMEM, "packed block of %zu bytes, %zu needed", packed_bytes, (size_t)pack8_bytes((int64_t)n * B));
    return SDNN_OK;
}

extern "C" int sdnn_pack8(const float *d_X, int32_t n, int32_t B, float cap, void *d_packed, size_t packed_bytes, void *stream)
{
    const int rc = sdnn_check_pack8(d_packed, packed_bytes, n, B, cap);
    if (rc || n == 0) return rc;
    if (!d_X) return sdnn_fail(SDNN_EINVAL, "d_X is NULL");
    const int64_t count = (int64_t)n * B;
    const dim3 grid((unsigned)std::min<int64_t>((pack8_groups(count) + 15) / 16, 16384)); // (65536 x 1024: 8192 2 us more, no bound 5 more)
    if (cap > 0.0f) hipLaunchKernelGGL(k_pack8<false>, grid, dim3(256), 0, (hipStream_t)stream, d_X, count, pack8_groups(count), cap, (uint8_t *)d_packed);
    else hipLaunchKernelGGL(k_pack8<true>, grid, dim3(256), 0, (hipStream_t)stream, d_X, count, pack8_groups(count), cap, (uint8_t *)d_packed);
    return sdnn_launched();
}

extern "C" int sdnn_unpack8(const void *d_packed, size_t packed_bytes, int32_t n, int32_t B, float cap, float *d_X, void *stream)
{
    const int rc = sdnn_check_pack8(d_packed, packed_bytes, n, B, cap);
    if (rc || n == 0) return rc;
    if (!d_X) return sdnn_fail(SDNN_EINVAL, "d_X is NULL");
    const int64_t count = (int64_t)n * B;
    const uint8_t *packed = (const uint8_t *)d_packed;
    const float below = nextafterf(cap, 0.0f);
    const int64_t blocks = (count + 1023) / 1024, most = 1 << 23; // (a launch holds less than 2^32 threads)
    for (int64_t b = 0; b < blocks; b += most) {
        const dim3 grid((unsigned)std::min(most, blocks - b));
        if (cap > 0.0f) hipLaunchKernelGGL(k_unpack8<false>, grid, dim3(256), 0, (hipStream_t)stream, packed, count, pack8_groups(count), cap, below, d_X, 256 * b);
        else hipLaunchKernelGGL(k_unpack8<true>, grid, dim3(256), 0, (hipStream_t)stream, packed, count, pack8_groups(count), cap, below, d_X, 256 * b);
    }
    return sdnn_launched();
}
