// Exchanges and sums over the lanes of a wavefront, without LDS.
#pragma once
#include <hip/hip_runtime.h>

// Exchange with the lane that differs in one bit of its number (bits 1 and 0: exactly that lane; bit 3: lane ^ 8; bit 2:
// lane ^ 7, which is as good where all lanes that agree in the higher bits hold the same set of values).
template <int BIT> __device__ __forceinline__ double lane_exchange(double v)
{
    constexpr int CTRL = BIT == 3 ? 0x128 : BIT == 2 ? 0x141 : BIT == 1 ? 0x4e : 0xb1; // row_ror:8, row_half_mirror, quad_perm
    const int lo = __builtin_amdgcn_mov_dpp(__double2loint(v), CTRL, 0xf, 0xf, true);
    const int hi = __builtin_amdgcn_mov_dpp(__double2hiint(v), CTRL, 0xf, 0xf, true);
    return __hiloint2double(hi, lo);
}
// The value of the lane whose number differs in exactly that bit (bits 0 to 3), and the sum with it (bits 4 and 5).
template <int BIT> __device__ __forceinline__ double lane_xor(double v)
{
    if constexpr (BIT != 2) {
        return lane_exchange<BIT>(v);
    } else { // lane ^ 7, then ^ 3
        const int lo = __builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp(__double2loint(v), 0x141, 0xf, 0xf, true), 0x1b, 0xf, 0xf, true);
        const int hi = __builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp(__double2hiint(v), 0x141, 0xf, 0xf, true), 0x1b, 0xf, 0xf, true);
        return __hiloint2double(hi, lo);
    }
}
template <int BIT> __device__ __forceinline__ double add_lane_xor(double v)
{
    const unsigned l = (unsigned)__double2loint(v), h = (unsigned)__double2hiint(v);
    const auto lo = BIT == 5 ? __builtin_amdgcn_permlane32_swap(l, l, false, false) : __builtin_amdgcn_permlane16_swap(l, l, false, false);
    const auto hi = BIT == 5 ? __builtin_amdgcn_permlane32_swap(h, h, false, false) : __builtin_amdgcn_permlane16_swap(h, h, false, false);
    return __hiloint2double((int)hi[0], (int)lo[0]) + __hiloint2double((int)hi[1], (int)lo[1]);
}
// One halving step of a sum over lanes of N values: the lane keeps the half of the values whose number has the bit that
// its own number has in place BIT, and adds its partner's share of them.
template <int N, int BIT, int SIZE> __device__ __forceinline__ void halve(double (&p)[SIZE], int lane)
{
#pragma unroll
    for (int j = 0; j < N / 2; ++j) {
        if constexpr (BIT >= 4) {
            const unsigned al = (unsigned)__double2loint(p[j]), ah = (unsigned)__double2hiint(p[j]);
            const unsigned bl = (unsigned)__double2loint(p[j + N / 2]), bh = (unsigned)__double2hiint(p[j + N / 2]);
            const auto lo = BIT == 5 ? __builtin_amdgcn_permlane32_swap(al, bl, false, false) : __builtin_amdgcn_permlane16_swap(al, bl, false, false);
            const auto hi = BIT == 5 ? __builtin_amdgcn_permlane32_swap(ah, bh, false, false) : __builtin_amdgcn_permlane16_swap(ah, bh, false, false);
            p[j] = __hiloint2double((int)hi[0], (int)lo[0]) + __hiloint2double((int)hi[1], (int)lo[1]);
        } else {
            const bool up = (lane >> BIT) & 1;
            const double keep = up ? p[j + N / 2] : p[j], send = up ? p[j] : p[j + N / 2];
            p[j] = keep + lane_exchange<BIT>(send);
        }
    }
}
