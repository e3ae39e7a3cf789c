// The decode cache in 4 bits: where things stand in it, and the rule by which a row is rounded (see lte_cache4_bytes in lte.h).
//
// A row is cut into groups of 32 channels, each with two bf16 parameters, zero = bf16(min) and step = bf16((max - min) / 15); a channel is a
// 4-bit code c and stands for zero + c step.  Why this form: 32 channels keep the largest of them from setting the step of the
// whole row, at 4 bytes of parameters to 16 of codes; both parameters in bf16 have the range of the rows themselves (fp16 would overflow or
// lose small rows), and c step has at most 12 bits, so that the value is exact up to one rounding of the sum.  zero differs from the minimum
// by half a bf16 step at most (2^-9 of it), which for a group around 0 is a hundredth of `step`.
//
// The order of the codes is that of the tensor-core decode kernel's operands, which take them from memory without a shuffle:
//   keys    4-byte word j of a row: group j mod (d/32), channels 8t .. 8t+7 of it with t = j / (d/32), lowest nibble first
//   values  2-byte unit u of a row: group u mod (d/32), channels 4g .. 4g+3 of it with g = u / (d/32), lowest nibble first
#pragma once
#include "common.cuh"

namespace lte {

constexpr int kGroup4 = 32;                                    // channels that share a step and a zero

struct Cache4Layout {
    size_t off_k, off_v;                                       // codes, [W+R][d/2] bytes each
    size_t off_kp, off_vp;                                     // parameters, [W+R][d/32] words: step in the low half, zero in the high one
    size_t off_z, off_pidx, off_meta;                          // as in an ordinary cache (common.cuh)
    size_t stride, header;
};
__host__ __device__ inline Cache4Layout cache4_layout(int d, int W, int R)
{
    const size_t rows = (size_t)W + R;
    auto up = [](size_t x) { return (x + 15) / 16 * 16; };     // every part starts on a 16-byte boundary
    Cache4Layout L;
    L.off_k = 0;
    L.off_v = up(rows * d / 2);
    L.off_kp = L.off_v + up(rows * d / 2);
    L.off_vp = L.off_kp + up(rows * d / 8);
    L.off_z = L.off_vp + up(rows * d / 8);
    L.off_pidx = L.off_z + up(rows * 4);
    L.off_meta = L.off_pidx + up((size_t)R * 4);
    L.stride = (L.off_meta + 16 + 255) / 256 * 256;
    L.header = 256;
    return L;
}

// channel of element e (0..7) of 4-byte word j of a row's key codes, of its value codes
__device__ __forceinline__ int key4_channel(int j, int e, int groups) { return (j % groups) * kGroup4 + (j / groups) * 8 + e; }
__device__ __forceinline__ int value4_channel(int j, int e, int groups)
{
    const int u = 2 * j + (e >> 2);
    return (u % groups) * kGroup4 + (u / groups) * 4 + (e & 3);
}

__device__ __forceinline__ float par4_step(uint32_t par) { return __uint_as_float(par << 16); }
__device__ __forceinline__ float par4_zero(uint32_t par) { return __uint_as_float(par & 0xffff0000u); }
// The value of a code: the product is exact (4 by 8 bits), so that the fused form rounds once, like the separate one.
__device__ __forceinline__ float value4(uint32_t code, uint32_t par) { return fmaf((float)code, par4_step(par), par4_zero(par)); }

// Parameters of a group from its extremes; `bad`: a channel is not finite.  A group that two finite bf16 numbers cannot describe reads
// back as NaN.
__device__ __forceinline__ uint32_t group4(float lo, float hi, bool bad)
{
    const uint32_t step = __bfloat16_as_ushort(__float2bfloat16_rn(__fdiv_rn(hi - lo, 15.f)));
    const uint32_t zero = __bfloat16_as_ushort(__float2bfloat16_rn(lo));
    if (bad || (step & 0x7f80u) == 0x7f80u || (zero & 0x7f80u) == 0x7f80u) return 0x7fc07fc0u;
    return step | (zero << 16);
}
// clamp(rint((x - zero) / step), 0, 15) in fp32 arithmetic; 0 where step is 0 or the group NaN.  The quotient is taken by the reciprocal, which is
// off by a few units in the last place: only within 2^-10 of the middle between two codes can that decide, and there it is divided.
__device__ __forceinline__ uint32_t code4(float x, uint32_t par)
{
    const float step = par4_step(par), r = x - par4_zero(par);
    if (!(step > 0.f)) return 0u;
    float q = r * __frcp_rn(step), c = rintf(q);
    if (!(fabsf(q - c) < 0.5f - 0x1p-10f)) c = rintf(__fdiv_rn(r, step));    // (so do a quotient and a reciprocal out of range)
    return (uint32_t)fminf(fmaxf(c, 0.f), 15.f);
}

// A group of the row in `x` (one channel per lane) into the 4-bit cache, by a whole warp.
__device__ __forceinline__ void store_group4(float x, int lane, bool values, int group, int groups, unsigned char* codes, uint32_t* par)
{
    float lo = x, hi = x;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    const bool bad = __any_sync(0xffffffffu, !(fabsf(x) < INFINITY));
    const uint32_t p = group4(lo, hi, bad);
    uint32_t w = code4(x, p) << (4 * (lane & (values ? 3 : 7)));
    w |= __shfl_xor_sync(0xffffffffu, w, 1);
    w |= __shfl_xor_sync(0xffffffffu, w, 2);
    if (!values) w |= __shfl_xor_sync(0xffffffffu, w, 4);
    if (lane == 0) par[group] = p;
    if (values) { if ((lane & 3) == 0) reinterpret_cast<uint16_t*>(codes)[(lane >> 2) * groups + group] = (uint16_t)w; }
    else if ((lane & 7) == 0) reinterpret_cast<uint32_t*>(codes)[(lane >> 3) * groups + group] = w;
}

}  // namespace lte
