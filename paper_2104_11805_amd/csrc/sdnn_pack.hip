// Activations in 8 bits (sdnn_pack8.h): single blocks, and X_0 .. X_L of a training net in one launch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "sdnn_internal.h"
#include "sdnn_pack8.h"

// What a wavefront's half has to do with one group: lane g of 32 holds its values 4 g .. 4 g + 3.
__device__ __forceinline__ void pack_group(const float (&x)[4], float cap, int lane, uint8_t *codes, uint16_t *scale)
{
    float largest = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (pack8_live(x[k], cap)) largest = fmaxf(largest, fabsf(x[k]));
#pragma unroll
    for (int m = 1; m < 32; m *= 2) largest = fmaxf(largest, __shfl_xor(largest, m));
    const unsigned t = pack8_scale(largest, cap > 0.0f ? 253.0f : 127.0f);
    const double inverse = pack8_inverse(t);
    unsigned c = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) c |= pack8_code(x[k], cap, inverse) << (8 * k);
    reinterpret_cast<unsigned *>(codes)[lane] = c;
    if (lane == 0) *scale = (uint16_t)t;
}

__global__ void __launch_bounds__(256) k_pack8(const float *__restrict__ x, int64_t count, int64_t groups, float cap, uint8_t *__restrict__ packed)
{
    const int lane = threadIdx.x & 31;
    uint16_t *scales = reinterpret_cast<uint16_t *>(packed + PACK_GROUP * groups);
    for (int64_t g = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); g < groups; g += (int64_t)gridDim.x * 8) {
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t e = PACK_GROUP * g + 4 * lane + k;
            v[k] = e < count ? x[e] : 0.0f;
        }
        pack_group(v, cap, lane, packed + PACK_GROUP * g, scales + g);
    }
}

__global__ void __launch_bounds__(256) k_unpack8(const uint8_t *__restrict__ packed, int64_t count, int64_t groups, float cap, float below, float *__restrict__ x)
{
    const uint16_t *scales = reinterpret_cast<const uint16_t *>(packed + PACK_GROUP * groups);
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; 4 * q < count; q += (int64_t)gridDim.x * 256) {
        const unsigned c = reinterpret_cast<const unsigned *>(packed)[q];
        const float t = __uint_as_float((unsigned)scales[q / (PACK_GROUP / 4)] << 16);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (4 * q + k < count) x[4 * q + k] = pack8_value(c >> (8 * k) & 255u, t, cap, below);
    }
}

// X_0 .. X_L of a training net, rows of ld floats, to and from one packed block after the other.  grid = (parts, blocks of
// 64 threads' worth of layers): blockIdx.y + l0 is l.
struct NetBlocks {
    const LayerDev *layers;
    float *x0;
    int32_t n_layers, B, Bp, ld;
    float cap, below;
    uint8_t *packed;
};
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
__global__ void __launch_bounds__(256) k_pack_net(const NetBlocks a, int l0)
{
    const int l = l0 + (int)blockIdx.y, lane = threadIdx.x & 31;
    uint8_t *packed = a.packed + block_start(a, l, threadIdx.x & 63);
    const float *x = l == 0 ? a.x0 : a.layers[l - 1].X, cap = l == 0 ? 0.0f : a.cap;
    const int64_t count = (int64_t)(l == 0 ? a.layers[0].n_in : a.layers[l - 1].n_out) * a.B;
    const int64_t groups = (count + PACK_GROUP - 1) / PACK_GROUP;
    uint16_t *scales = reinterpret_cast<uint16_t *>(packed + PACK_GROUP * groups);
    for (int64_t g = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); g < groups; g += (int64_t)gridDim.x * 8) {
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t e = PACK_GROUP * g + 4 * lane + k, row = e / a.B;
            v[k] = e < count ? x[row * a.ld + (e - row * a.B)] : 0.0f;
        }
        pack_group(v, cap, lane, packed + PACK_GROUP * g, scales + g);
    }
}
// Columns B .. Bp - 1 become zeros, as the passes leave them.
__global__ void __launch_bounds__(256) k_unpack_net(const NetBlocks a, int l0)
{
    const int l = l0 + (int)blockIdx.y;
    const uint8_t *packed = a.packed + block_start(a, l, threadIdx.x & 63);
    float *x = l == 0 ? a.x0 : a.layers[l - 1].X;
    const float cap = l == 0 ? 0.0f : a.cap;
    const int64_t n = l == 0 ? a.layers[0].n_in : a.layers[l - 1].n_out, groups = (n * a.B + PACK_GROUP - 1) / PACK_GROUP;
    const uint16_t *scales = reinterpret_cast<const uint16_t *>(packed + PACK_GROUP * groups);
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < n * a.Bp; q += (int64_t)gridDim.x * 256) {
        const int64_t row = q / a.Bp, s = q - row * a.Bp, e = row * a.B + s;
        float v = 0.0f;
        if (s < a.B) v = pack8_value(packed[e], __uint_as_float((unsigned)scales[e / PACK_GROUP] << 16), cap, a.below);
        x[row * a.ld + s] = v;
    }
}

static unsigned parts_for(int64_t items) // workgroups of 256 threads, each walking the items
{
    return (unsigned)std::min<int64_t>(std::max<int64_t>((items + 255) / 256, 1), 8192);
}

// The launches that sdnn_checkpoint_save (restore = 0) and _load make; the return value is a hipError_t.
int sdnn_launch_checkpoint(const LayerDev *d_layers, float *d_x0, int32_t n_layers, int64_t max_n, int32_t B, int32_t Bp, int32_t ld, float cap,
                           void *d_ckpt, int restore, void *stream)
{
    NetBlocks a;
    a.layers = d_layers; a.x0 = d_x0; a.n_layers = n_layers; a.B = B; a.Bp = Bp; a.ld = ld; a.cap = cap; a.below = nextafterf(cap, 0.0f);
    a.packed = (uint8_t *)d_ckpt;
    const unsigned gx = std::min(parts_for(restore ? max_n * Bp : (max_n * B + 3) / 4), 2048u);
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
    hipLaunchKernelGGL(k_pack8, dim3(parts_for(count / 4)), dim3(256), 0, (hipStream_t)stream, d_X, count, pack8_groups(count), cap, (uint8_t *)d_packed);
    return sdnn_launched();
}

extern "C" int sdnn_unpack8(const void *d_packed, size_t packed_bytes, int32_t n, int32_t B, float cap, float *d_X, void *stream)
{
    const int rc = sdnn_check_pack8(d_packed, packed_bytes, n, B, cap);
    if (rc || n == 0) return rc;
    if (!d_X) return sdnn_fail(SDNN_EINVAL, "d_X is NULL");
    const int64_t count = (int64_t)n * B;
    hipLaunchKernelGGL(k_unpack8, dim3(parts_for((count + 3) / 4)), dim3(256), 0, (hipStream_t)stream, (const uint8_t *)d_packed, count,
                       pack8_groups(count), cap, nextafterf(cap, 0.0f), d_X);
    return sdnn_launched();
}
