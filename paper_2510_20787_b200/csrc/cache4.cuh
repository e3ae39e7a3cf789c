// The decode cache in 4 bits: where things stand in it, and the rule by which a row is rounded (see lte_cache4_bytes in lte.h).
//
// A row is cut into groups of 32 channels, each with two bf16 parameters, zero = bf16(min) and step = bf16((max - min) (1/15)), 1/15 and the product
// rounded to fp32; a channel is a 4-bit code c and stands for zero + c step.  Why this form: 32 channels keep the largest of them from setting the
// step of the whole row, at 4 bytes of parameters to 16 of codes; both parameters in bf16 have the range of the rows themselves (fp16 would overflow
// or lose small rows), and c step has at most 12 bits, so that the value is exact up to one rounding of the sum.  zero is the minimum itself for
// bf16 rows, and within 2^-9 of it for fp32 ones, which for a group around 0 is a hundredth of `step`.
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
    const uint32_t step = __bfloat16_as_ushort(__float2bfloat16_rn((hi - lo) * (1.f / 15.f)));
    const uint32_t zero = __bfloat16_as_ushort(__float2bfloat16_rn(lo));
    if (bad || (step & 0x7f80u) == 0x7f80u || (zero & 0x7f80u) == 0x7f80u) return 0x7fc07fc0u;
    return step | (zero << 16);
}
// clamp(rint((x - zero) / step), 0, 15) in fp32 arithmetic; 0 where step is 0 or the group NaN
__device__ __forceinline__ uint32_t code4(float x, uint32_t par)
{
    const float step = par4_step(par);
    if (!(step > 0.f)) return 0u;
    return (uint32_t)fminf(fmaxf(rintf(__fdiv_rn(x - par4_zero(par), step)), 0.f), 15.f);
}
// The codes of eight channels, the first in the lowest nibble.  The quotient d / step, d = x - zero, comes from the reciprocal y of step (the
// instruction's, within 2^-23) by one correction, q + (d - q step) y (Markstein, Computation of elementary functions on the IBM RISC System/6000
// processor, 1990): a rounding of the exact quotient moved by less than 4 units of its last place times 2^-23.  That rounds to the same code as the correctly rounded quotient: an
// exact half k + 1/2 stays one (bf16 rows have them all the time), and the two could part only where the quotient is that close to the border
// between k + 1/2 and its neighbour, a number of 25 bits, which times step is no fp32 number d (step has 8 bits, so that what is not on
// the border is further off).  Rounding is by adding 1.5 2^23, which leaves the code in the lowest bits.  Steps outside 2^-100 .. 2^100, where
// the terms might leave the range of fp32, are divided by.
// EXACT: the channels are bf16 numbers.  zero is then the minimum itself, and quotients lie between 0 and 15 (1 + 2^-8): nothing to clamp.
template <bool EXACT> __device__ __forceinline__ uint32_t codes4(const float (&f)[8], uint32_t par)
{
    constexpr float MAGIC = 12582912.f;
    constexpr uint32_t REST = 0x4b400000u * 0x11111111u;       // (modulo 2^32: what the bits above the codes add up to)
    const float step = par4_step(par), zero = par4_zero(par);
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(step));
    uint32_t w = 0u;
    if (step > 0x1p-100f && step < 0x1p100f) {
        w = 0u - REST;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = f[i] - zero, q0 = d * y, q = fmaf(fmaf(-q0, step, d), y, q0);
            w += __float_as_uint((EXACT ? q : fminf(fmaxf(q, 0.f), 15.f)) + MAGIC) << (4 * i);
        }
    } else if (step > 0.f) {
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {
            float x = f[0];
#pragma unroll
            for (int e = 1; e < 8; ++e) x = e == i ? f[e] : x;
            w |= code4(x, par) << (4 * i);
        }
    }
    return w;
}
// Extremes of a group from four lanes' eight channels each; NaN and infinities go through.
__device__ __forceinline__ uint32_t group4_of(const uint4& u)     // bf16
{
    auto bf = [](uint32_t x) { return *reinterpret_cast<const __nv_bfloat162*>(&x); };
    __nv_bfloat162 lo = __hmin2_nan(__hmin2_nan(bf(u.x), bf(u.y)), __hmin2_nan(bf(u.z), bf(u.w)));
    __nv_bfloat162 hi = __hmax2_nan(__hmax2_nan(bf(u.x), bf(u.y)), __hmax2_nan(bf(u.z), bf(u.w)));
    __nv_bfloat162 x = __halves2bfloat162(__hmin_nan(lo.x, lo.y), __hneg(__hmax_nan(hi.x, hi.y)));   // (min, -max)
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
        const uint32_t other = __shfl_xor_sync(0xffffffffu, *reinterpret_cast<const uint32_t*>(&x), o);
        x = __hmin2_nan(x, bf(other));
    }
    // (as group4, with the minimum's bits as they are)
    const float step = (-__bfloat162float(x.y) - __bfloat162float(x.x)) * (1.f / 15.f);
    const __nv_bfloat162 par = __floats2bfloat162_rn(step, __bfloat162float(x.x));
    const uint32_t p = *reinterpret_cast<const uint32_t*>(&par);
    return (p & 0x7f80u) == 0x7f80u || (p & 0x7f800000u) == 0x7f800000u ? 0x7fc07fc0u : p;
}
__device__ __forceinline__ uint32_t group4_of(const float (&f)[8])
{
    float lo = f[0], hi = f[0];
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) { lo = fminf(lo, f[i]); hi = fmaxf(hi, f[i]); bad |= !(fabsf(f[i]) < INFINITY); }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        bad |= __shfl_xor_sync(0xffffffffu, (int)bad, o) != 0;
    }
    return group4(lo, hi, bad);
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
