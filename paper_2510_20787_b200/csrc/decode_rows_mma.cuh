// Decode step (lte_attn_decode_accum, lte_attn_decode4, lte_attn_decode4_accum) for bf16 calls: rows go from memory straight into tensor-core
// operands, as in decode_mma.cu, every query head of a group at once, heads split over warps and clusters where there are few.
//
// Bound by memory where rows are bf16; rows in 4 bits are 3.2 times smaller, and there the instructions that unpack and weigh them count for more
// (about 190 per 16 rows at d = 64, of which the two products' operands are 60, and 1,900 a warp beside them, at 0.51 to 0.55 per cycle: 14 warps an SM do
// not hide their latencies, and registers for more are not there).  Every warp walks units of 16 or 32 rows (interleaved over the warps of all blocks that share the head) that pass
// through stages of its own in shared memory, keeps its own reference, sum and output, and meets the others once at the end.  The incoming token
// is no row: its logit is a dot product on the fp32 ALUs, and it joins where the warps meet.
//
// Scores (accumulated attention): a row's weight needs the sum over all rows, so the raw logits of a warp's rows stay in shared memory until the
// blocks have met (or, where they do not fit, come from the keys once more); then every warp adds its rows' weights, summed over the query heads, to
// their scores.  One read and one write of 4 bytes a row.
//
// Products are mma.sync m16n8k16: logits S^T[16 rows][8 queries] = K q^T, output O^T[16 channels][8 queries] += V^T P^T, N = 8 queries.
// Rows in 4 bits.  A code is an fp16 number as it stands: the low ten bits of a half are its fraction, so that c in bits 0-3 is the subnormal number
// c 2^-24, in bits 4-7 16 c 2^-24; a mask on two codes at a time is all the conversion there is.  With value = zero + c step:
//   logits   per group of 32 channels, step c.q + zero sum(q): the group's product starts from zero, and its two scalars, which belong to a
//            row, are applied to the products in fp32 (a lane holds rows of both).  q is scaled by a power of two per query head to at most 2^15 (and
//            by 1/16 where it meets 16 c), in which fp16 holds bf16 numbers exactly down to 2^-24; logits are kept in that scale;
//   output   P step takes the place of P, per group, and P zero, the same for all channels of a group, is summed beside it in fp32.  P step is
//            rounded to fp16, 2^-12 of it: an error of o of at most 2^-12 sum(w c step) (o against 64 bits, in the mean square: 1.67e-3 to 1.73e-3,
//            1.66e-3 with the rounding of o alone).  It is scaled by a power of two, per group and query, that follows the largest product
//            (not the largest step: a row whose weight is nothing may have any).  That stands at 2^11 or above, so that one too
//            small for fp16's normal numbers is off by 2^-36 of it.
// The contraction index may be permuted freely: the nibbles i and i + 4 of a key word are neighbours in it, and so are the two rows whose value
// units a byte permute joins.  The order of the codes in the cache (cache4.cuh) makes these the words that a lane loads.
//
// Measured (B200, us a step in a CUDA graph of steps over three caches in turn, full pools; bytes that cannot be avoided at 6.56 TB/s):
//                                                    accumulated, bf16    4 bits, accumulated    4 bits, learned
//   2,048 heads x 256 rows, d = 64                       27.8 (21.5)          19.5 (7.2)            19.1 (6.7)
//   256 x 1,280, four query heads each, d = 64           20.5 (13.3)          14.8 (4.5)            12.9 (4.2)
//   2,048 x 1,024, d = 64                                 109 (85.3)          58.3 (28.8)           50.7 (26.9)
//   512 x 1,024, d = 128                                 47.4 (41.9)          28.7 (13.6)           26.7 (13.1)
//   4,096 x 400, d = 32                                  49.9 (34.7)          37.5 (12.5)           34.7 (11.0)
//   8 x 17,408, four query heads each, d = 128           27.4 (11.1)          19.5 (3.7)            16.8 (3.6)
//   16 x 1,024, d = 128 (one user)                        8.8 (1.3)            8.8 (0.4)             7.9 (0.4)
// Of a step 5 to 8 us are the chain of launch, counters, first rows, meeting and write-back (what 32 rows a head take).  What did not help: 4-bit
// rows in 80 registers and 24 warps an SM (2,048 x 256: 27.8), bulk copies with a barrier per stage in the place of 16-byte ones (the same for bf16,
// and 35 instructions per 16 rows more), codes as bf16 numbers 16 + c with P in two terms (1.05 us per 16 rows of 2,048 heads, now 0.67).
#pragma once
#include <cfloat>
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "decode_rows.cuh"
#include "row_mma.cuh"
#include "tc_common.cuh"

namespace lte {
namespace cg = cooperative_groups;
namespace {

constexpr int MQ = 8;                                          // query heads per pass
// resident warps the registers (and the stages in shared memory) are budgeted for
__host__ __device__ constexpr int warps_per_sm(int d, bool four) { return d == 128 && four ? 8 : 16; }
constexpr int MAX_WARPS = 8;                                   // per block
// blocks of so many warps come in clusters (at d = 128 with four already: eight 4-bit ones take an SM's registers, and the next step's blocks then
// find no room beside them)
__host__ __device__ constexpr bool clusters(int d, int nw) { return nw == MAX_WARPS || (d == 128 && nw == 4); }
constexpr int MAX_SPLIT = 16;                                  // blocks per head

// A head's rows in use are rows 0 .. total - 1 of its block (while the ring fills up the pool is empty).  A warp takes units of UR of them, 16 to
// a product, which pass through STAGES of its own in shared memory by 16-byte asynchronous copies.  (With the units in registers, enough of them
// in flight and the products' operands did not fit 128 registers: 256 heads x 1,280 rows in 4 bits 23.7 us, through shared memory 18.5.)
struct Rows {
    const unsigned char *K, *V, *KP, *VP;
    int total;
};
template <int D, bool FOUR> struct Stage {
    static constexpr int UR = FOUR || D < 128 ? 32 : 16;
    static constexpr int ROW = FOUR ? D / 2 : 2 * D, PAR = FOUR ? D / 8 : 0;   // bytes of a row's keys, of its key parameters
    static constexpr int K = 0, V = UR * ROW, KP = 2 * V, VP = KP + UR * PAR, BYTES = VP + UR * PAR;
    static constexpr int ACC = MQ * (D + 8) * 4;               // a warp's outputs stand where its stages were
    static_assert(ACC <= BYTES, "the outputs' place");
};

// N 4-byte words of shared memory (one load; from reinterpreted pointers the compiler makes single words)
template <int N> __device__ __forceinline__ void lds(uint32_t (&x)[N], uint32_t at)
{
    if constexpr (N == 1) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x[0]) : "r"(at) : "memory");
    else if constexpr (N == 2) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(x[0]), "=r"(x[1]) : "r"(at) : "memory");
    else asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(at) : "memory");
}

// The two products with a span of 16 rows that stands in shared memory, lane (g, t) = (lane / 4, lane % 4).  Rows past the last one and those that the
// step leaves out have weight zero, and what they hold is cleared (zero times an infinite value is NaN).
template <int D, bool SWZ, bool FOUR> struct Group;

template <int D, bool SWZ> struct Group<D, SWZ, false> {
    static constexpr int KP = D / 32, VB = D / 16, PITCH = D * 2, MT = D / 16;
    static constexpr float LIFT = 1.f;
    struct Raw { uint4 u[KP]; };                               // pieces t, t + 4, .. of query g
    struct Query { uint4 f[KP]; float unit[2]; };
    struct Acc { float a[MT][4]; };
    struct Pars {};
    struct Weights {};
    static __device__ __forceinline__ void load_pars(Pars&, uint32_t, int, int) {}
    static __device__ __forceinline__ int rho(int g) { return g; }
    static __device__ __forceinline__ void load_q(Raw& r, const __nv_bfloat16* q, bool some, int g, int t)
    {
#pragma unroll
        for (int j = 0; j < KP; ++j) r.u[j] = some ? reinterpret_cast<const uint4*>(q + (size_t)g * D)[t + 4 * j] : make_uint4(0, 0, 0, 0);
    }
    static __device__ __forceinline__ void set_q(Query& Q, const Raw& r, int)
    {
#pragma unroll
        for (int j = 0; j < KP; ++j) Q.f[j] = r.u[j];
        Q.unit[0] = Q.unit[1] = 1.f;
    }
    // c: rows g (0, 1) and g + 8 (2, 3), queries 2t and 2t + 1.  A product rounds its running sum towards zero, so every one starts from zero
    // and the parts are added to the nearest (see decode_mma.cu).  Lane (g, t) takes pieces t, t + 4, .. of rows g and g + 8.
    static __device__ __forceinline__ void logits(float (&c)[4], const Query& Q, uint32_t st, int span, int g, int t)
    {
        uint32_t k[2][KP][4];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < KP; ++j)
                lds(k[u][j], st + g * PITCH + ((t ^ (SWZ ? g & 3 : 0)) << 4) + Stage<D, false>::K + (16 * span + 8 * u) * PITCH + ((4 * j) ^ (SWZ ? g & 4 : 0)) * 16);
        constexpr int NS = D == 128 ? 2 : 1;
        float cs[NS][4];
#pragma unroll
        for (int i = 0; i < 2 * KP; ++i) {
            const int j = i >> 1, s = 2 * (i & 1);
            float part[4] = {0.f, 0.f, 0.f, 0.f};
            mma16816(part, k[0][j][s], k[1][j][s], k[0][j][s + 1], k[1][j][s + 1], word(Q.f[j], s), word(Q.f[j], s + 1));
#pragma unroll
            for (int e = 0; e < 4; ++e) cs[i % NS][e] = i < NS ? part[e] : cs[i % NS][e] + part[e];
        }
#pragma unroll
        for (int w = NS / 2; w > 0; w >>= 1)
#pragma unroll
            for (int j = 0; j < w; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) cs[j][e] += cs[j + w][e];
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = cs[0][e];
    }
    static __device__ __forceinline__ void start(Acc& A)
    {
#pragma unroll
        for (int m = 0; m < MT; ++m) A.a[m][0] = A.a[m][1] = A.a[m][2] = A.a[m][3] = 0.f;
    }
    static __device__ __forceinline__ void rescale(Acc& A, float f0, float f1)
    {
#pragma unroll
        for (int m = 0; m < MT; ++m) { A.a[m][0] *= f0; A.a[m][1] *= f1; A.a[m][2] *= f0; A.a[m][3] *= f1; }
    }
    // what the rows of a unit that `gone` names hold as values
    static __device__ __forceinline__ void clear(unsigned char* st, unsigned gone, int lane)
    {
        for (; gone; gone &= gone - 1u)
            if (lane < D / 8) *reinterpret_cast<uint4*>(st + Stage<D, false>::V + (__ffs(gone) - 1) * PITCH + 16 * lane) = make_uint4(0, 0, 0, 0);
    }
    // Lane (g, t) takes pieces g, g + 8 of rows 2t, 2t + 1, 2t + 8, 2t + 9.
    static __device__ __forceinline__ void output(Acc& A, const float (&p)[4], const Weights&, const Pars&, uint32_t st, int span, int g, int t)
    {
        uint32_t v[4][VB];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int r = 2 * t + (u & 1) + 8 * (u >> 1);
            const uint32_t base = st + Stage<D, false>::V + (16 * span + r) * PITCH;
            if constexpr (D == 32) {
                lds(v[u], base + (g << 3));
            } else {
#pragma unroll
                for (int j = 0; j < D / 64; ++j) {
                    uint32_t x[4];
                    lds(x, base + (((g + 8 * j) ^ (SWZ ? r & 7 : 0)) << 4));
#pragma unroll
                    for (int w = 0; w < 4; ++w) v[u][4 * j + w] = x[w];
                }
            }
        }
        const uint32_t hi0 = pack_bf16(p[0], p[1]), hi1 = pack_bf16(p[2], p[3]);
        const uint32_t lo0 = pack_bf16(p[0] - __uint_as_float(hi0 << 16), p[1] - __uint_as_float(hi0 & 0xffff0000u));
        const uint32_t lo1 = pack_bf16(p[2] - __uint_as_float(hi1 << 16), p[3] - __uint_as_float(hi1 & 0xffff0000u));
        const uint32_t h0 = movmatrix_trans(hi0), h1 = movmatrix_trans(hi1), e0 = movmatrix_trans(lo0), e1 = movmatrix_trans(lo1);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const uint32_t a0 = __byte_perm(v[0][m], v[1][m], 0x5410), a1 = __byte_perm(v[0][m], v[1][m], 0x7632);
            const uint32_t a2 = __byte_perm(v[2][m], v[3][m], 0x5410), a3 = __byte_perm(v[2][m], v[3][m], 0x7632);
            mma16816(A.a[m], a0, a1, a2, a3, h0, h1);
            mma16816(A.a[m], a0, a1, a2, a3, e0, e1);
        }
    }
    static __device__ __forceinline__ void finish(Acc&) {}
    static __device__ __forceinline__ int channel(int m, int g) { return D == 32 ? g * 4 + 2 * m : (m >> 2) * 64 + g * 8 + 2 * (m & 3); }
};

// Rows in 4 bits: a span stands in shared memory, where the products take their operands from.  M-row r of a product is row rho(r) of the span,
// rho(2t + b + 8c) = t + 4b + 8c: the value units that the lanes load at once then lie in different banks.
template <int D, bool SWZ> struct Group<D, SWZ, true> {
    static constexpr int GR = D / kGroup4, MT = D / 16;
    static constexpr uint32_t MOST_INV = 246u;                 // exponent of the largest scale, 2^119 (times a weight, below 2^8: finite)
    static constexpr float CODE = 16777216.f;                  // 2^24: products are sums of c 2^-24 q
    // A logit is the product, times LIFT, times the query's unit, which has the rest of CODE: split so that neither the products of keys as large as
    // 2^120 nor the units of the largest queries leave the range of fp32.
    static constexpr float LIFT = 1024.f, UNIT = CODE / LIFT;
    struct Raw { uint4 u[GR]; };                               // channels 8t .. 8t + 7 of every group of query g
    struct Query { uint32_t f[GR][4]; float sum[GR][2], unit[2]; };   // of query g, scaled; sums over a group's channels and units of queries 2t, 2t + 1
    struct Acc { float a[MT][4], z[GR][2], inv[GR][2]; };      // inv: the scale of P step, per group and query
    struct Weights { uint32_t h[GR][2]; };                     // P step inv of two queries, of rows rho(g), rho(g) + 8
    struct Pars { uint32_t p[2][GR]; };                        // of rows rho(g), rho(g) + 8
    static __device__ __forceinline__ int rho(int g) { return (g >> 1) + 4 * (g & 1); }     // (g < 8)
    static __device__ __forceinline__ void load_q(Raw& r, const __nv_bfloat16* q, bool some, int g, int t)
    {
#pragma unroll
        for (int j = 0; j < GR; ++j) r.u[j] = some ? reinterpret_cast<const uint4*>(q + (size_t)g * D + j * kGroup4)[t] : make_uint4(0, 0, 0, 0);
    }
    static __device__ __forceinline__ void set_q(Query& Q, const Raw& r, int t)
    {
        const uint4 (&u)[GR] = r.u;
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < GR; ++j) {
#pragma unroll
            for (int w = 0; w < 4; ++w) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(word(u[j], w) << 16)), fabsf(__uint_as_float(word(u[j], w) & 0xffff0000u))));
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // the power of two that takes the largest channel to 2^14 .. 2^15 (1 for a query that is zero or not finite)
        const uint32_t ex = __float_as_uint(top) >> 23, field = top > 0.f && top < INFINITY ? min(268u - ex, 253u) : 127u;
        const float scale = __uint_as_float(field << 23), unit = __uint_as_float((254u - field) << 23) * UNIT;
#pragma unroll
        for (int j = 0; j < GR; ++j) {
            float x[8], s = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                x[2 * w] = __uint_as_float(word(u[j], w) << 16) * scale;
                x[2 * w + 1] = __uint_as_float(word(u[j], w) & 0xffff0000u) * scale;
                s += x[2 * w] + x[2 * w + 1];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {                      // channels i and i + 4
                const __half2 h = i & 1 ? __floats2half2_rn(x[i] * 0.0625f, x[i + 4] * 0.0625f) : __floats2half2_rn(x[i], x[i + 4]);
                Q.f[j][i] = *reinterpret_cast<const uint32_t*>(&h);
            }
            s += __shfl_xor_sync(0xffffffffu, s, 1);
            s += __shfl_xor_sync(0xffffffffu, s, 2);
            s *= 1.f / CODE;
            Q.sum[j][0] = __shfl_sync(0xffffffffu, s, 8 * t);
            Q.sum[j][1] = __shfl_sync(0xffffffffu, s, 8 * t + 4);
        }
        Q.unit[0] = __shfl_sync(0xffffffffu, unit, 8 * t);
        Q.unit[1] = __shfl_sync(0xffffffffu, unit, 8 * t + 4);
    }
    static __device__ __forceinline__ void logits(float (&c)[4], const Query& Q, uint32_t st, int span, int g, int t)
    {
        const uint32_t keys = st + rho(g) * (D / 2) + t * (4 * GR), pars = st + rho(g) * (4 * GR);
        uint32_t k[2][GR], kp[2][GR];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            lds(k[u], keys + Stage<D, true>::K + (2 * span + u) * (4 * D));
            lds(kp[u], pars + Stage<D, true>::KP + (2 * span + u) * (32 * GR));
        }
#pragma unroll
        for (int j = 0; j < GR; ++j) {
            float p[4] = {0.f, 0.f, 0.f, 0.f};
            const uint32_t x = k[0][j], y = k[1][j], x8 = x >> 8, y8 = y >> 8;
            mma16816_f16(p, x & 0x000f000fu, y & 0x000f000fu, x & 0x00f000f0u, y & 0x00f000f0u, Q.f[j][0], Q.f[j][1]);
            mma16816_f16(p, x8 & 0x000f000fu, y8 & 0x000f000fu, x8 & 0x00f000f0u, y8 & 0x00f000f0u, Q.f[j][2], Q.f[j][3]);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float s = par4_step(kp[i][j]), z = par4_zero(kp[i][j]);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float v = j == 0 ? z * Q.sum[j][e] : fmaf(z, Q.sum[j][e], c[2 * i + e]);
                    c[2 * i + e] = fmaf(s, p[2 * i + e], v);
                }
            }
        }
    }
    static __device__ __forceinline__ void start(Acc& A)
    {
#pragma unroll
        for (int m = 0; m < MT; ++m) A.a[m][0] = A.a[m][1] = A.a[m][2] = A.a[m][3] = 0.f;
#pragma unroll
        for (int j = 0; j < GR; ++j) A.z[j][0] = A.z[j][1] = 0.f;
#pragma unroll
        for (int j = 0; j < GR; ++j) A.inv[j][0] = A.inv[j][1] = __uint_as_float(MOST_INV << 23);
    }
    // A new reference, under which weights are f0, f1 times as large (at most 1) and this unit's are p.  A scale takes f up, rounded up to a power of
    // two, as far as it can, so that the largest product so far does not get smaller in fp16; where the unit has a product above 2^15, its scale goes
    // to where the largest is 2^11 .. 2^12, which leaves four binary places for later ones.
    template <int UNIT> static __device__ __forceinline__ void rescale(Acc& A, float f0, float f1, const float (&p)[UNIT][4], const Pars (&P)[UNIT])
    {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float f = e ? f1 : f0;
            const uint32_t up = 127u - min(__float_as_uint(f) >> 23, 127u);
#pragma unroll
            for (int j = 0; j < GR; ++j) {
                float top = 0.f;                               // 2^-10 of the largest (which need not be finite)
#pragma unroll
                for (int x = 0; x < UNIT; ++x)
#pragma unroll
                    for (int u = 0; u < 2; ++u) top = fmaxf(top, p[x][2 * u + e] * 0x1p-10f * par4_step(P[x].p[u][j]));
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                const uint32_t old = __float_as_uint(A.inv[j][e]) >> 23, raised = min(old + up, MOST_INV);
                const uint32_t now = top * __uint_as_float(raised << 23) > 32.f ? min(255u - (__float_as_uint(top) >> 23), MOST_INV) : raised;
                const float part = f * __uint_as_float((127u + raised - old) << 23) * __uint_as_float((uint32_t)max(127 + (int)now - (int)raised, 0) << 23);
                A.inv[j][e] = __uint_as_float(now << 23);
                A.z[j][e] *= f;
#pragma unroll
                for (int m = 2 * j; m < 2 * j + 2; ++m) { A.a[m][e] *= part; A.a[m][2 + e] *= part; }
            }
        }
    }
    // what the rows of a unit that `gone` names hold as values: with step and zero 0 it is 0
    static __device__ __forceinline__ void clear(unsigned char* st, unsigned gone, int lane)
    {
        if ((gone >> lane) & 1u)
#pragma unroll
            for (int j = 0; j < GR; ++j) reinterpret_cast<uint32_t*>(st + Stage<D, true>::VP)[lane * GR + j] = 0u;
    }
    // parameters of a span's values
    static __device__ __forceinline__ void load_pars(Pars& P, uint32_t st, int span, int g)
    {
#pragma unroll
        for (int u = 0; u < 2; ++u) lds(P.p[u], st + rho(g) * (4 * GR) + Stage<D, true>::VP + (2 * span + u) * (32 * GR));
    }
    // A span's weights times the steps of its rows, as the second product's operand.  True where one of this lane's is above 2^15.
    // (The scale meets the weight first: a row that weighs next to nothing may have any step.)
    static __device__ __forceinline__ bool weigh(Weights& w, const Acc& A, const float (&p)[4], const Pars& P)
    {
        __half2 top = __floats2half2_rn(0.f, 0.f);
#pragma unroll
        for (int j = 0; j < GR; ++j) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const float s = par4_step(P.p[u][j]);
                const __half2 x = __floats2half2_rn(p[2 * u] * A.inv[j][0] * s, p[2 * u + 1] * A.inv[j][1] * s);
                top = __hmax2(top, x);
                w.h[j][u] = *reinterpret_cast<const uint32_t*>(&x);
            }
        }
        return __hgt2_mask(top, __floats2half2_rn(32768.f, 32768.f)) != 0u;
    }
    static __device__ __forceinline__ void output(Acc& A, const float (&p)[4], const Weights& W, const Pars& P, uint32_t st, int span, int g, int t)
    {
        const uint32_t values = st + t * (D / 2) + g * (2 * GR) + Stage<D, true>::V + span * (8 * D);
        uint32_t v[4][(GR + 1) / 2];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if constexpr (GR == 1) {                           // M-rows 2t + (u & 1) + 8 (u / 2)
                uint16_t x;
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(values + u * (2 * D)) : "memory");
                v[u][0] = x;
            } else {
                lds(v[u], values + u * (2 * D));
            }
        }
#pragma unroll
        for (int j = 0; j < GR; ++j) {
            const float z0 = par4_zero(P.p[0][j]), z1 = par4_zero(P.p[1][j]);
            A.z[j][0] = fmaf(p[2], z1, fmaf(p[0], z0, A.z[j][0]));
            A.z[j][1] = fmaf(p[3], z1, fmaf(p[1], z0, A.z[j][1]));
            const uint32_t h0 = movmatrix_trans(W.h[j][0]), h1 = movmatrix_trans(W.h[j][1]);
            const uint32_t u = __byte_perm(v[0][j / 2], v[1][j / 2], j & 1 ? 0x7632 : 0x5410), u8 = u >> 8;   // four codes of M-row 2t, of M-row 2t + 1
            const uint32_t w = __byte_perm(v[2][j / 2], v[3][j / 2], j & 1 ? 0x7632 : 0x5410), w8 = w >> 8;
            mma16816_f16(A.a[2 * j], u & 0x000f000fu, u & 0x00f000f0u, w & 0x000f000fu, w & 0x00f000f0u, h0, h1);
            mma16816_f16(A.a[2 * j + 1], u8 & 0x000f000fu, u8 & 0x00f000f0u, w8 & 0x000f000fu, w8 & 0x00f000f0u, h0, h1);
        }
    }
    // the groups' constant parts, summed over the lanes of a query, into the outputs
    static __device__ __forceinline__ void finish(Acc& A)
    {
#pragma unroll
        for (int j = 0; j < GR; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float z = A.z[j][e];
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
                const float back = __uint_as_float((254u << 23) - __float_as_uint(A.inv[j][e]));   // (the second channel of a pair: sums of 16 c)
#pragma unroll
                for (int m = 2 * j; m < 2 * j + 2; ++m) {
                    A.a[m][e] = fmaf(A.a[m][e] * CODE, back, z);
                    A.a[m][2 + e] = fmaf(A.a[m][2 + e] * (CODE / 16), back, z);
                }
            }
    }
    static __device__ __forceinline__ int channel(int m, int g) { return (m >> 1) * kGroup4 + 4 * g + 2 * (m & 1); }
};

// Where the weights of accumulated attention come from: logits kept in shared memory, or the keys once more (see launch_rows_mma).
enum { LEARNED = 0, KEPT = 1, AGAIN = 2 };

// LONG: 4 bits, and a warp may have more than kLongRows rows.  Sums of codes are positive and cancel against those of zero; the tensor cores round their
// running sums towards zero, and after some thousand rows of equal weight that shows (32,768 rows to a warp: 2 % of o).  Every 512 rows what they have
// then goes to a second sum, which is rounded to the nearest.  It stands in local memory: there are no registers for it, and even so the loop takes
// up to a fifth longer (256 heads x 1,280 rows, d = 64, accumulated 14.6 -> 17.6 us), which is why it is a variant of its own.
constexpr int kLongRows = 2048;

template <int D, int NW, int STAGES, bool SWZ, bool FOUR, int RULE, bool LONG>
__global__ void __launch_bounds__(NW * 32, warps_per_sm(D, FOUR) / NW) decode_rows_mma_kernel(
    unsigned char* __restrict__ cache, RowsLayout L, const __nv_bfloat16* __restrict__ q1, const __nv_bfloat16* __restrict__ k1,
    const __nv_bfloat16* __restrict__ v1, __nv_bfloat16* __restrict__ o1, float* __restrict__ lse1, RowsRule rule, int H, int W, int R, int sink,
    float scale, int G, int most, int* __restrict__ status)    // most: rows whose logits a warp may have to keep (whole units)
{
    using Gr = Group<D, SWZ, FOUR>;
    constexpr bool ACCUM = RULE != LEARNED;
    constexpr int NT = NW * 32, MT = D / 16, PITCH = D + 8, CPL = D / 32, GR = D / kGroup4;
    using St = Stage<D, FOUR>;
    constexpr int UR = St::UR, UNIT = UR / 16;
    constexpr int SPLIT = clusters(D, NW) ? MAX_SPLIT : 1;
    extern __shared__ __align__(128) unsigned char s_dyn[];    // the warps' stages; [NW][nq][most + 4] logits, behind them [NW][most + 4] sums over passes
    float* const s_log = reinterpret_cast<float*>(s_dyn + NW * STAGES * St::BYTES);
    auto s_acc = [&](int w, int u) { return reinterpret_cast<float*>(s_dyn + w * (STAGES * St::BYTES)) + u * PITCH; };
    __shared__ float s_unit[MQ];
    __shared__ float s_m[NW][MQ], s_l[NW][MQ], s_new[MQ];
    __shared__ float s_in[2][SPLIT > 1 ? MQ * D + SPLIT : 1];
    __shared__ __align__(16) float s_ml[2][SPLIT][MQ][2];      // the cluster's shares of this block's output elements (by pass parity)
    __shared__ __align__(16) __nv_bfloat16 s_kv[2][D];         // the incoming token
    __shared__ float s_tap[NW];
    __shared__ uint32_t s_wkey[NW];
    __shared__ int s_wpos[NW], s_wslot[NW];
    __shared__ __align__(16) int4 s_worst[SPLIT];
    __shared__ __align__(16) uint32_t s_holds[4];              // the cache's header
    cg::cluster_group cluster = cg::this_cluster();
    const int nsplit = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int bh = blockIdx.x / nsplit, h = bh % H;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, g = lane >> 2, t = lane & 3;
    unsigned char* blk = cache + L.header + (size_t)bh * L.stride;
    float* zc = reinterpret_cast<float*>(blk + L.off_z);
    int32_t* pidx = reinterpret_cast<int32_t*>(blk + L.off_pidx);
    int32_t* meta = reinterpret_cast<int32_t*>(blk + L.off_meta);
    const bool shared_head = SPLIT > 1 && nsplit > 1;          // (uniform in the cluster)
    if (shared_head) cluster.barrier_arrive();                 // (awaited before the first store into another block's shared memory)
    pdl_launch_dependents();
    pdl_wait();

    // What is small and waited for first is asked for first; then the rows that a warp begins with, whether or not they turn out to be in use (behind
    // them the counters took two thousand cycles); then what needs the counters, and the rest of the stages.
    const int n_held = meta[0], cnt_held = meta[1];
    typename Gr::Raw q_raw;
    Gr::load_q(q_raw, q1 + (size_t)bh * G * D, g < G, g, t);
    constexpr int PRE = NT < 256 ? 4 : 2;                      // scores and positions of the pool, before it is known whether the decision needs them
    // A pool that the cluster's blocks would each take several rounds to look through they look through together, which costs a meeting.
    const bool share_scan = shared_head && R > 4 * PRE * NT;
    const int part = share_scan ? (R + nsplit - 1) / nsplit : R, pre0 = share_scan ? rank * part : 0, pre1 = min(R, pre0 + part);
    float pz[PRE];
    int pp[PRE];
#pragma unroll
    for (int u = 0; u < PRE; ++u) {
        const int m = pre0 + tid + u * NT;
        pz[u] = m < pre1 ? zc[W + m] : INFINITY;
        pp[u] = m < pre1 ? pidx[m] : -1;
    }
    Rows rows;
    rows.K = blk + L.off_k; rows.V = blk + L.off_v; rows.KP = blk + L.off_kp; rows.VP = blk + L.off_vp;
    rows.total = W + R;
    const int step = NW * nsplit, first = wid * nsplit + rank;
    unsigned char* const stage = s_dyn + wid * (STAGES * St::BYTES);
    const uint32_t stage_at = tc::smem_u32(stage);
    // What is copied next of the keys (values): unit `unit` of the head, its rows and parameters from `row` and `par` on (this lane's 16 bytes).
    struct Source { const unsigned char *row, *par; int unit; };
    int units = (W + R + UR - 1) / UR, full = (W + R) / UR;    // of the head; whole ones
    constexpr int P = UR * St::PAR;                            // bytes of a unit's key parameters
    const bool par_lane = 16 * lane < P;
    auto ask = [&](Source& S, uint32_t to, int par_to) {       // its next unit to `to`, the parameters `par_to` bytes behind
        to += 16 * lane;
        if (S.unit < full) {
#pragma unroll
            for (int u = 0; u < UR * St::ROW / 512; ++u) tc::cp_async16(to + 512 * u, S.row + 512 * u, 16);
            if (FOUR && par_lane) tc::cp_async16(to + par_to, S.par, 16);
        } else if (S.unit < units) {
            const int n_rows = rows.total - UR * S.unit;
#pragma unroll
            for (int u = 0; u < UR * St::ROW / 512; ++u)
                if (16 * lane + 512 * u < n_rows * St::ROW) tc::cp_async16(to + 512 * u, S.row + 512 * u, 16);
            if (FOUR && par_lane && 16 * lane < n_rows * St::PAR) tc::cp_async16(to + par_to, S.par, 16);   // (the last 16 bytes of a part of the cache are its own)
        }
        S.unit += step;
        S.row += (size_t)step * (UR * St::ROW);
        S.par += (size_t)step * P;
    };
    Source sk, sv;
    auto ask_keys = [&](uint32_t to) { ask(sk, to + St::K, St::KP - St::K); };
    auto ask_values = [&](uint32_t to) { ask(sv, to + St::V, St::VP - St::V); };
    // bf16: keys and values are refilled as soon as each has been read, in copy groups of their own; 4 bits: together, which takes fewer instructions
    constexpr int PENDING = FOUR ? STAGES - 1 : 2 * STAGES - 1;    // copy groups that may be on their way when the next one is waited for
    auto fill = [&](int s) {                                   // the next unit into stage s
        ask_keys(stage_at + s * St::BYTES);
        if (!FOUR) tc::cp_async_commit();
        ask_values(stage_at + s * St::BYTES);
        tc::cp_async_commit();
    };
    auto begin = [&]() {                                       // the first unit of a pass
        sk = {rows.K + (size_t)first * (UR * St::ROW) + 16 * lane, rows.KP + (size_t)first * P + 16 * lane, first};
        sv = {rows.V + (size_t)first * (UR * St::ROW) + 16 * lane, rows.VP + (size_t)first * P + 16 * lane, first};
        fill(0);
    };
    if (tid == 0) tc::cp_async16(tc::smem_u32(s_holds), cache, 16);
    begin();
    const int n = max(n_held, 0), cnt_old = min(max(cnt_held, 0), R);
    typename Gr::Query qf;
    Gr::set_q(qf, q_raw, t);
    if (tid < D / 4) reinterpret_cast<uint4*>(s_kv)[tid] = reinterpret_cast<const uint4*>((tid < D / 8 ? k1 : v1) + (size_t)bh * D)[tid % (D / 8)];
    const int slot = n % W, p = n - W, half = rule.K / 2;
    rows.total = n < W ? n : W + cnt_old;
    units = (rows.total + UR - 1) / UR; full = rows.total / UR;
    const float zp = p >= 0 ? zc[slot] : 0.f;
    // Learned rule, the first block: logit of the newest token whose receptive field is complete.  A lane takes eight channels under a tap: a
    // word of the row's key or value codes, two runs of four weights.
    const int jsc = ACCUM ? -1 : n - half;
    constexpr int LT = D / 4, TAPS = 32 / LT;                  // lanes per tap, taps of a warp at a time
    struct Tap { uint32_t x, par[2]; float w[8]; };
    const int tap_values = lane % LT / (D / 8), tap_word = lane % (D / 8);
    const int tap_ch0 = tap_values ? value4_channel(tap_word, 0, GR) : key4_channel(tap_word, 0, GR);
    const int tap_ch4 = tap_values ? value4_channel(tap_word, 4, GR) : key4_channel(tap_word, 4, GR);
    auto tap_ask = [&](Tap& T, int tap) {                      // tap < K - 1: the token n - (K - 1) + tap, in the ring (which holds at least K)
        const int back = slot + tap - (rule.K - 1), r = back < 0 ? back + W : back;
        T.x = T.par[0] = T.par[1] = 0u;
#pragma unroll
        for (int e = 0; e < 8; ++e) T.w[e] = 0.f;
        if (tap >= rule.K - 1 || n - (rule.K - 1) + tap < 0) return;
        const float* w = rule.w + ((size_t)h * rule.K + tap) * 2 * D + tap_values * D;
        if ((reinterpret_cast<uintptr_t>(rule.w) & 15u) == 0) {
            const float4 a = *reinterpret_cast<const float4*>(w + tap_ch0), b = *reinterpret_cast<const float4*>(w + tap_ch4);
            T.w[0] = a.x; T.w[1] = a.y; T.w[2] = a.z; T.w[3] = a.w; T.w[4] = b.x; T.w[5] = b.y; T.w[6] = b.z; T.w[7] = b.w;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) { T.w[e] = w[tap_ch0 + e]; T.w[4 + e] = w[tap_ch4 + e]; }
        }
        T.x = reinterpret_cast<const uint32_t*>((tap_values ? rows.V : rows.K) + (size_t)r * (D / 2))[tap_word];
        const uint32_t* par = reinterpret_cast<const uint32_t*>(tap_values ? rows.VP : rows.KP) + (size_t)r * GR;
        T.par[0] = par[tap_ch0 / kGroup4]; T.par[1] = par[tap_ch4 / kGroup4];
    };
    auto tap_sum = [&](const Tap& T) {
        float a = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) a = fmaf(T.w[e], value4((T.x >> (4 * e)) & 15u, T.par[e >> 2]), a);
        return a;
    };
    Tap tap0;
    const bool scores = !ACCUM && rank == 0 && jsc >= 0;
    float tap_new = 0.f;                                       // the last tap: the incoming token, as given
    if (scores) {
        tap_ask(tap0, wid * TAPS + lane / LT);
        if (wid == NW - 1) {
            const float* w = rule.w + ((size_t)h * rule.K + rule.K - 1) * 2 * D;
#pragma unroll
            for (int c = 0; c < CPL; ++c)
                tap_new += w[lane + 32 * c] * __bfloat162float(k1[(size_t)bh * D + lane + 32 * c]) + w[D + lane + 32 * c] * __bfloat162float(v1[(size_t)bh * D + lane + 32 * c]);
        }
    }

#pragma unroll
    for (int s = 1; s < STAGES; ++s) fill(s);

    // ---- what happens to the token leaving the window ------------------------------------------------------------
    int dst = -1, cnt_new = cnt_old;
    bool met = false;                                          // the cluster's blocks have met already
    if (p >= 0 && R > 0 && (ACCUM || p < sink || zp > rule.zthr)) {
        if (cnt_old < R) { dst = cnt_old; cnt_new = cnt_old + 1; }
        else if (p >= sink) {
            Worst w;
#pragma unroll
            for (int u = 0; u < PRE; ++u) if (pre0 + tid + u * NT < min(cnt_old, pre1)) w.offer(pz[u], pp[u], pre0 + tid + u * NT, sink);
            constexpr int MORE = 4;                            // loads in flight
            for (int m0 = pre0 + tid + PRE * NT; m0 < min(cnt_old, pre1); m0 += MORE * NT) {
                float z[MORE];
                int at[MORE];
#pragma unroll
                for (int u = 0; u < MORE; ++u) {
                    const int m = min(m0 + u * NT, cnt_old - 1);   // (an entry offered twice is one)
                    z[u] = zc[W + m]; at[u] = pidx[m];
                }
#pragma unroll
                for (int u = 0; u < MORE; ++u) w.offer(z[u], at[u], min(m0 + u * NT, cnt_old - 1), sink);
            }
            w.over_warp();
            if (NW > 1) {
                if (lane == 0) { s_wkey[wid] = w.key; s_wpos[wid] = w.pos; s_wslot[wid] = w.slot; }
                __syncthreads();
                w.key = lane < NW ? s_wkey[lane] : 0xffffffffu; w.pos = lane < NW ? s_wpos[lane] : -1; w.slot = lane < NW ? s_wslot[lane] : -1;
                w.over_warp();
            }
            if (share_scan) {                                  // each block has looked at its part
                cluster.barrier_wait();                        // (every block of the cluster has started)
                met = true;
                if (wid == 0 && lane < nsplit) *reinterpret_cast<int4*>(cluster.map_shared_rank(&s_worst[rank], lane)) = make_int4((int)w.key, w.pos, w.slot, 0);
                cluster.sync();
                const int4 x = s_worst[min(lane, nsplit - 1)];
                w.key = (uint32_t)x.x; w.pos = x.y; w.slot = x.z;
                w.over_warp();
            }
            if (w.slot >= 0 && Worst::rank(zp) > w.key) dst = w.slot;
        }
    }
    const int masked_ring = p >= 0 && dst < 0 ? slot : -32;    // the popped row counts iff the pool takes it ...
    const int masked_pool = dst >= 0 && dst < cnt_old ? W + dst : -32;   // ... and then the entry it replaces does not

    if (scores) {
        float a = tap_new + tap_sum(tap0);
        for (int tap = (wid + NW) * TAPS; tap < rule.K - 1; tap += NW * TAPS) {
            tap_ask(tap0, tap + lane / LT);
            a += tap_sum(tap0);
        }
        a = warp_sum(a);
        if (lane == 0) s_tap[wid] = a;
    }

    // 4 bits: the incoming row's codes, in the last warp of the first block, while the first rows are on their way: eight channels a lane, four
    // lanes a group
    const int new_piece = min(lane, D / 4 - 1) % (D / 8);
    const bool new_values = min(lane, D / 4 - 1) >= D / 8;
    uint32_t new_codes = 0u, new_par = 0u;
    if constexpr (FOUR) {
        if (rank == 0 && wid == NW - 1) {
            const uint4 u = reinterpret_cast<const uint4*>((new_values ? v1 : k1) + (size_t)bh * D)[new_piece];
            float f[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(word(u, i) << 16); f[2 * i + 1] = __uint_as_float(word(u, i) & 0xffff0000u); }
            new_par = group4_of(u);
            new_codes = codes4<true>(f, new_par);
        }
    }

    // the popped row's words, read before the slot is written: thread e of the last ones moves word e
    constexpr int WORDS = FOUR ? 2 * (D / 8 + GR) : 2 * (D / 8), MOVES = (WORDS + NT - 1) / NT;   // (bf16: 16-byte pieces)
    using Move = std::conditional_t<FOUR, uint32_t, uint4>;
    auto place = [&](int e, int row) -> Move* {                // word e of a row's keys, key parameters, values, value parameters
        if constexpr (FOUR) {
            constexpr int P = D / 8 + GR;
            const bool values = e >= P;
            const int w = e - (values ? P : 0);
            return reinterpret_cast<uint32_t*>(blk + (w < D / 8 ? (values ? L.off_v : L.off_k) : (values ? L.off_vp : L.off_kp)))
                   + (w < D / 8 ? (size_t)row * (D / 8) + w : (size_t)row * GR + (w - D / 8));
        } else {
            const int c = e % (D / 8);
            return reinterpret_cast<uint4*>(blk + (e < D / 8 ? L.off_k : L.off_v)) + (size_t)row * (D / 8) + (SWZ ? c ^ (row & 7) : c);
        }
    };
    Move mv[MOVES];

    const float scale2 = scale * 1.44269504088896340736f;
    const int nqs = min(G, MQ);                                // logits kept per row
    const int lpitch = most + 4;                               // (so that the queries of a store lie in different banks)
    float* wlog = s_log + wid * lpitch * nqs;                  // this warp's
    float* wsum = s_log + NW * lpitch * nqs + wid * lpitch;
    float fresh = 0.f;                                         // the incoming token's weights (thread 0 of the first block)
    for (int g0 = 0; g0 < G; g0 += MQ) {
        const int nq = min(MQ, G - g0);
        if (g0 > 0) {                                          // further query heads read the rows again
            Gr::load_q(q_raw, q1 + ((size_t)bh * G + g0) * D, g < nq, g, t);
            __syncthreads();                                   // the previous pass's outputs, which stand in the stages, have been combined
            begin();
#pragma unroll
            for (int s = 1; s < STAGES; ++s) fill(s);
            Gr::set_q(qf, q_raw, t);
        }
        if (rank == 0)                                         // the incoming token's logits
            for (int u = wid; u < nq; u += NW) {
                float a = 0.f;
#pragma unroll
                for (int c = 0; c < CPL; ++c)
                    a = fmaf(__bfloat162float(q1[((size_t)bh * G + g0 + u) * D + lane + 32 * c]), __bfloat162float(k1[(size_t)bh * D + lane + 32 * c]), a);
                a = warp_sum(a);
                const float unit = __shfl_sync(0xffffffffu, u & 1 ? qf.unit[1] : qf.unit[0], u >> 1);
                if (lane == 0) s_new[u] = a * __uint_as_float((254u << 23) - __float_as_uint(unit));   // (the inverse of a power of two)
            }
        typename Gr::Acc acc;
        Gr::start(acc);
        // logits, references in units of `unit` per query; jump: a factor of 2^8 between weights
        const float sq0 = scale2 * qf.unit[0], sq1 = scale2 * qf.unit[1], jump0 = 8.f / sq0, jump1 = 8.f / sq1;
        float m0 = -FLT_MAX, m1 = -FLT_MAX, l0 = 0.f, l1 = 0.f;
        int kept = 0;                                          // rows whose logits this warp has kept
        volatile float second[MT][4];                          // LONG: the second sums,
        bool have = false;                                     // whether there is anything in them,
        int left = 512 / UR;                                   // units until the next
        auto gather = [&]() {                                  // ... back into the running sums
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc.a[m][e] += second[m][e];
            have = false;
        };

        const int ring_unit = masked_ring / UR, pool_unit = masked_pool / UR;
        int at_stage = 0;                                      // in bytes
#pragma unroll 1
        for (int i = first; i < units; i += step) {
            float c[UNIT][4], p[UNIT][4];
            const uint32_t st = stage_at + at_stage;
            at_stage = at_stage == (STAGES - 1) * St::BYTES ? 0 : at_stage + St::BYTES;
            tc::cp_async_wait<PENDING>();
            __syncwarp();                                      // every lane's copies of this unit (bf16: of its keys) are there
#pragma unroll
            for (int x = 0; x < UNIT; ++x) Gr::logits(c[x], qf, st, x, g, t);
            if (!FOUR) {
                __syncwarp();                                  // every lane has read the keys
                ask_keys(st);
                tc::cp_async_commit();
                tc::cp_async_wait<PENDING>();
                __syncwarp();                                  // ... every lane's copies of its values
            }
            if (i >= full || i == ring_unit || i == pool_unit) {
                unsigned gone = i >= full ? ~0u << (rows.total - UR * i) : 0u;   // rows of the unit that do not count
                if (i == ring_unit) gone |= 1u << (masked_ring % UR);
                if (i == pool_unit) gone |= 1u << (masked_pool % UR);
#pragma unroll
                for (int x = 0; x < UNIT; ++x) {
                    if ((gone >> (16 * x + Gr::rho(g))) & 1u) c[x][0] = c[x][1] = -INFINITY;
                    if ((gone >> (16 * x + Gr::rho(g) + 8)) & 1u) c[x][2] = c[x][3] = -INFINITY;
                }
                Gr::clear(stage + (st - stage_at), UR < 32 ? gone & ((1u << UR) - 1u) : gone, lane);
                __syncwarp();
            }
            if constexpr (RULE == KEPT) {                      // raw logits [query][row]
                float* at = wlog + 2 * t * lpitch + kept + Gr::rho(g);
#pragma unroll
                for (int x = 0; x < UNIT; ++x) {
                    if (2 * t < nq) { at[16 * x] = c[x][0]; at[16 * x + 8] = c[x][2]; }
                    if (2 * t + 1 < nq) { at[lpitch + 16 * x] = c[x][1]; at[lpitch + 16 * x + 8] = c[x][3]; }
                }
                kept += UR;
            }
            typename Gr::Pars vpar[UNIT];
            typename Gr::Weights weights[UNIT];
#pragma unroll
            for (int x = 0; x < UNIT; ++x) Gr::load_pars(vpar[x], st, x, g);
            // The reference m follows the maximum only when that has grown by 2^8 (weights stay below 2^8, in fp32): a vote per
            // unit instead of a reduction over its rows.  4 bits: the same vote says whether a product with a step has grown too large.
            auto exponentials = [&]() {                        // p from c
#pragma unroll
                for (int x = 0; x < UNIT; ++x)
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[x][e] = exp2_fast(fmaf(c[x][e], Gr::LIFT, e & 1 ? -m1 : -m0) * (e & 1 ? sq1 : sq0));
            };
            auto times_steps = [&]() {                         // 4 bits: true where a product is too large
                bool over = false;
                if constexpr (FOUR)
#pragma unroll
                    for (int x = 0; x < UNIT; ++x) over |= Gr::weigh(weights[x], acc, p[x], vpar[x]);
                return over;
            };
            auto largest = [&](const float (&y)[UNIT][4], int e) {
                float x = fmaxf(y[0][e], y[0][2 + e]);
#pragma unroll
                for (int u = 1; u < UNIT; ++u) x = fmaxf(x, fmaxf(y[u][e], y[u][2 + e]));
                return x;
            };
            bool far;
            if constexpr (FOUR) {
                exponentials();
                far = fmaxf(largest(p, 0), largest(p, 1)) > 256.f;
                far |= times_steps();
            } else {
                far = fmaf(largest(c, 0), Gr::LIFT, -m0) > jump0 || fmaf(largest(c, 1), Gr::LIFT, -m1) > jump1;
            }
            if (__any_sync(0xffffffffu, far)) {
                float y0 = largest(c, 0) * Gr::LIFT, y1 = largest(c, 1) * Gr::LIFT;
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) {
                    y0 = fmaxf(y0, __shfl_xor_sync(0xffffffffu, y0, o));
                    y1 = fmaxf(y1, __shfl_xor_sync(0xffffffffu, y1, o));
                }
                y0 = fmaxf(y0, m0); y1 = fmaxf(y1, m1);
                const float f0 = exp2_fast((m0 - y0) * sq0), f1 = exp2_fast((m1 - y1) * sq1);
                m0 = y0; m1 = y1;
                l0 *= f0; l1 *= f1;
                if constexpr (FOUR) {
                    if constexpr (LONG) { if (have) gather(); }
                    exponentials();
                    Gr::rescale(acc, f0, f1, p, vpar);
                    (void)times_steps();
                } else {
                    Gr::rescale(acc, f0, f1);
                }
            }
            if (!FOUR) exponentials();
#pragma unroll
            for (int x = 0; x < UNIT; ++x) { l0 += p[x][0] + p[x][2]; l1 += p[x][1] + p[x][3]; }
#pragma unroll
            for (int x = 0; x < UNIT; ++x) Gr::output(acc, p[x], weights[x], vpar[x], st, x, g, t);
            if constexpr (LONG) {
                if (--left == 0) {
                    left = 512 / UR;
                    if (have) gather();
                    have = true;
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int e = 0; e < 4; ++e) { second[m][e] = acc.a[m][e]; acc.a[m][e] = 0.f; }
                }
            }
            __syncwarp();                                      // every lane has read the stage
            if (FOUR) ask_keys(st);
            ask_values(st);
            tc::cp_async_commit();
        }
        tc::cp_async_wait<0>();                                // (units asked for before it was known how many rows are in use)
        __syncwarp();
        const bool last = g0 + MQ >= G;
        if (rank == 0 && last && dst >= 0)                     // (back by the time the write-back needs them)
#pragma unroll
            for (int u = 0; u < MOVES; ++u)
                if (NT - 1 - tid + u * NT < WORDS) mv[u] = *place(NT - 1 - tid + u * NT, slot);
        // Scores of this warp's rows: asked for before the warps meet, a batch at a time.  Row e of a warp is row e % UR of its unit e / UR.
        auto row_of = [&](int e) { return UR * (first + e / UR * step) + e % UR; };
        auto counts = [&](int row) { return row < rows.total && row != masked_ring && row != masked_pool; };
        constexpr int BATCH = 8;
        float old[BATCH];
        auto load_old = [&](int e0) {
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                const int e = e0 + 32 * b, row = row_of(e);
                old[b] = e < kept && counts(row) ? row == slot && p >= 0 ? zp : zc[row] : 0.f;   // (the popped row's place may already have been written)
            }
        };
        if (RULE == KEPT && last) load_old(lane);
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) { l0 += __shfl_xor_sync(0xffffffffu, l0, o); l1 += __shfl_xor_sync(0xffffffffu, l1, o); }
        if constexpr (LONG) { if (have) gather(); }
        Gr::finish(acc);
        __syncthreads();                                       // the incoming token is there; the previous pass has been combined
        if (g0 == 0 && wrong_cache<FOUR, ACCUM>(cache_holds(s_holds))) {   // (every block of the launch; nothing has been written yet)
            if (shared_head && !met) cluster.barrier_wait();
            if (blockIdx.x == 0 && tid == 0) atomicExch(status, kWrongCache);
            return;
        }
        if (wid == 0 && g == 0) { s_unit[2 * t] = qf.unit[0]; s_unit[2 * t + 1] = qf.unit[1]; }
        if (g == 0) { s_m[wid][2 * t] = m0; s_m[wid][2 * t + 1] = m1; s_l[wid][2 * t] = l0; s_l[wid][2 * t + 1] = l1; }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int ch = Gr::channel(i, g);
            if (2 * t < nq) *reinterpret_cast<float2*>(&s_acc(wid, 2 * t)[ch]) = make_float2(acc.a[i][0], acc.a[i][2]);
            if (2 * t + 1 < nq) *reinterpret_cast<float2*>(&s_acc(wid, 2 * t + 1)[ch]) = make_float2(acc.a[i][1], acc.a[i][3]);
        }
        __syncthreads();
        if (shared_head && g0 == 0 && !met) cluster.barrier_wait();    // every block of the cluster has started: its shared memory is there
        const int per = (nq * D + nsplit - 1) / nsplit, par = (g0 / MQ) & 1;  // output elements each block of the cluster finishes
        // Lane u of every warp: reference and sum of query u over this block's rows (and the incoming token, in the first block)
        float qm = -FLT_MAX, qt = 0.f, qs = 0.f;
        if (lane < nq) {
            qs = scale2 * s_unit[lane];
            if (rank == 0) qm = fmaxf(s_new[lane], -FLT_MAX);
#pragma unroll
            for (int w2 = 0; w2 < NW; ++w2) qm = fmaxf(qm, s_m[w2][lane]);
            if (rank == 0) qt = exp2_fast((s_new[lane] - qm) * qs);
#pragma unroll
            for (int w2 = 0; w2 < NW; ++w2) qt = fmaf(exp2_fast((s_m[w2][lane] - qm) * qs), s_l[w2][lane], qt);   // (a warp without rows: 0)
        }
        float qi = 1.f / qt;
        if (!shared_head && wid == 0 && lane < nq) lse1[(size_t)bh * G + g0 + lane] = qm * (scale * s_unit[lane]) + logf(qt);
        for (int e = tid; e < nq * D; e += NT) {               // (a warp's elements are of one query)
            const int u = e / D, ch = e - u * D;
            const float m = __shfl_sync(0xffffffffu, qm, u), sum = __shfl_sync(0xffffffffu, qt, u), sq = __shfl_sync(0xffffffffu, qs, u);
            float o = rank == 0 ? exp2_fast((s_new[u] - m) * sq) * __bfloat162float(s_kv[1][ch]) : 0.f;
#pragma unroll
            for (int w2 = 0; w2 < NW; ++w2) o = fmaf(exp2_fast((s_m[w2][u] - m) * sq), s_acc(w2, u)[ch], o);
            if (!shared_head) {
                o1[((size_t)bh * G + g0 + u) * D + ch] = __float2bfloat16_rn(o * __shfl_sync(0xffffffffu, qi, u));
            } else {                                           // into the shared memory of the block that finishes this element
                const int own = e / per;
                *cluster.map_shared_rank(&s_in[par][rank * per + (e - own * per)], own) = o;
                if (ch < nsplit) *reinterpret_cast<float2*>(cluster.map_shared_rank(&s_ml[par][rank][u][0], ch)) = make_float2(m, sum);
            }
        }
        if (shared_head) {
            cluster.sync();                                    // all shares have arrived, and every row has been read
            if (lane < nq) {                                   // the same over the whole head
                qm = -FLT_MAX; qt = 0.f;
                for (int r2 = 0; r2 < nsplit; ++r2) qm = fmaxf(qm, s_ml[par][r2][lane][0]);
                for (int r2 = 0; r2 < nsplit; ++r2) qt = fmaf(exp2_fast((s_ml[par][r2][lane][0] - qm) * qs), s_ml[par][r2][lane][1], qt);
            }
            qi = 1.f / qt;
            if (rank == 0 && wid == 0 && lane < nq) lse1[(size_t)bh * G + g0 + lane] = qm * (scale * s_unit[lane]) + logf(qt);
            for (int e0 = wid * 32; e0 < per; e0 += NT) {
                const int e = min(e0 + lane, per - 1), el = min(rank * per + e, nq * D - 1), u = el / D, ch = el - u * D;
                const float m = __shfl_sync(0xffffffffu, qm, u), inv = __shfl_sync(0xffffffffu, qi, u), sq = __shfl_sync(0xffffffffu, qs, u);
                float o = 0.f;
                for (int r2 = 0; r2 < nsplit; ++r2) o = fmaf(exp2_fast((s_ml[par][r2][u][0] - m) * sq), s_in[par][r2 * per + e], o);
                if (e0 + lane < per && rank * per + e < nq * D) o1[((size_t)bh * G + g0 + u) * D + ch] = __float2bfloat16_rn(o * inv);
            }
        }
        if constexpr (RULE == KEPT) {
            // ---- weights of this warp's rows into their scores.  Every block has read the old ones that its decision needs.
            for (int base = 0; base < kept; base += 32 * BATCH) {   // (the same in the whole warp)
                const int e0 = base + lane;
                if (last && base > 0) load_old(e0);
                float a[BATCH] = {};
#pragma unroll 1
                for (int u = 0; u < nq; ++u) {
                    const float m = __shfl_sync(0xffffffffu, qm, u), inv = __shfl_sync(0xffffffffu, qi, u), sq = __shfl_sync(0xffffffffu, qs, u);
#pragma unroll
                    for (int b = 0; b < BATCH; ++b)
                        if (32 * b < kept - base)
                            a[b] = fmaf(exp2_fast(fmaf(wlog[u * lpitch + min(e0 + 32 * b, kept - 1)], Gr::LIFT, -m) * sq), inv, a[b]);
                }
#pragma unroll
                for (int b = 0; b < BATCH; ++b) {
                    const int e = e0 + 32 * b, row = row_of(e);
                    if (e >= kept) continue;
                    if (G > MQ) { if (g0 > 0) a[b] += wsum[e]; wsum[e] = a[b]; }
                    if (last && counts(row)) zc[row == slot && p >= 0 ? W + dst : row] = rule.decay > 0.f ? fmaf(rule.decay, old[b], a[b]) : a[b];
                }
            }
            __syncwarp();                                      // (the next pass writes logits where these were)
        }
        if constexpr (RULE == AGAIN) {
            // ---- the same from the keys, which are read once more.  Lane (g, t) has the logits of rows rho(g), + 8 (+ 16, + 24) for two queries; the four
            // lanes of a g add them up, and lane t is left with row rho(g) + 8 t.  The passes add to the scores in the order of the query heads.
            __syncthreads();                                   // the outputs, which stand in the stages, have been combined
            const float ma = __shfl_sync(0xffffffffu, qm, 2 * t), mb = __shfl_sync(0xffffffffu, qm, 2 * t + 1);
            const float wa = __shfl_sync(0xffffffffu, qi, 2 * t), wb = __shfl_sync(0xffffffffu, qi, 2 * t + 1);
            sk = {rows.K + (size_t)first * (UR * St::ROW) + 16 * lane, rows.KP + (size_t)first * P + 16 * lane, first};
#pragma unroll
            for (int s = 0; s < STAGES; ++s) { ask_keys(stage_at + s * St::BYTES); tc::cp_async_commit(); }
            int at_stage = 0;
#pragma unroll 1
            for (int i = first; i < units; i += step) {
                const uint32_t st = stage_at + at_stage;
                at_stage = at_stage == (STAGES - 1) * St::BYTES ? 0 : at_stage + St::BYTES;
                const int row = UR * i + Gr::rho(g) + 8 * t;
                const bool mine = t < 2 * UNIT && counts(row), leaves = row == slot && p >= 0;
                float* const to = zc + (leaves ? W + dst : row);
                // (the popped row's place may already have the incoming token's score)
                const float before = !mine ? 0.f : g0 > 0 ? *to : rule.decay > 0.f ? rule.decay * (leaves ? zp : *to) : 0.f;
                tc::cp_async_wait<STAGES - 1>();
                __syncwarp();
                float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int u = 0; u < UNIT; ++u) {
                    float c[4];
                    Gr::logits(c, qf, st, u, g, t);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float a = 2 * t < nq ? exp2_fast(fmaf(c[2 * e], Gr::LIFT, -ma) * sq0) * wa : 0.f;
                        x[2 * u + e] = 2 * t + 1 < nq ? fmaf(exp2_fast(fmaf(c[2 * e + 1], Gr::LIFT, -mb) * sq1), wb, a) : a;
                    }
                }
                __syncwarp();                                  // every lane has read the stage
                ask_keys(st);
                tc::cp_async_commit();
                const bool odd = t & 1, high = t & 2;
                const float y0 = (odd ? x[1] : x[0]) + __shfl_xor_sync(0xffffffffu, odd ? x[0] : x[1], 1);
                const float y1 = (odd ? x[3] : x[2]) + __shfl_xor_sync(0xffffffffu, odd ? x[2] : x[3], 1);
                const float z = (high ? y1 : y0) + __shfl_xor_sync(0xffffffffu, high ? y0 : y1, 2);
                if (mine) *to = before + z;
            }
            tc::cp_async_wait<0>();
            __syncwarp();
        }
        if constexpr (ACCUM) {
            if (rank == 0 && wid == 0) {
                float a = lane < nq ? exp2_fast((s_new[lane] - qm) * qs) * qi : 0.f;
                a = warp_sum(a);
                fresh += a;
            }
        }
    }

    // ---- write-back: only what changed; every read of the old block lies before the barriers above and here ------------------
    if (RULE == AGAIN) {                                       // (the keys of the rows that are written now have been read a second time)
        if (shared_head) cluster.sync();
        else __syncthreads();
    }
    if (rank != 0) return;
    if (dst >= 0)
#pragma unroll
        for (int u = 0; u < MOVES; ++u)
            if (NT - 1 - tid + u * NT < WORDS) *place(NT - 1 - tid + u * NT, W + dst) = mv[u];
    if constexpr (FOUR) {
        if (wid == NW - 1 && lane < D / 4) {
            unsigned char* codes = blk + (new_values ? L.off_v : L.off_k) + (size_t)slot * (D / 2);
            const int grp = new_piece / 4, tt = new_piece % 4;
            if (new_values) {
                reinterpret_cast<uint16_t*>(codes)[2 * tt * GR + grp] = (uint16_t)new_codes;
                reinterpret_cast<uint16_t*>(codes)[(2 * tt + 1) * GR + grp] = (uint16_t)(new_codes >> 16);
            } else {
                reinterpret_cast<uint32_t*>(codes)[tt * GR + grp] = new_codes;
            }
            if (tt == 0) reinterpret_cast<uint32_t*>(blk + (new_values ? L.off_vp : L.off_kp))[(size_t)slot * GR + grp] = new_par;
        }
    } else {
        for (int e = tid; e < WORDS; e += NT) *reinterpret_cast<uint4*>(place(e, slot)) = reinterpret_cast<const uint4*>(s_kv)[e];
    }
    if (tid == 0) {
        if (dst >= 0) pidx[dst] = p;
        if (ACCUM) {
            zc[slot] = fresh;
        } else {
            if (dst >= 0) zc[W + dst] = zp;
            float znew = rule.bias ? rule.bias[h] : 0.f;
            if (jsc >= 0)
                for (int w = 0; w < NW; ++w) znew += s_tap[w];
            zc[slot] = -INFINITY;                              // the incoming token is not scored yet ...
            if (jsc >= 0) zc[slot - half < 0 ? slot - half + W : slot - half] = znew;   // ... unless K == 1 (then jsc == n)
        }
        meta[0] = n + 1;
        meta[1] = cnt_new;
    }
}

constexpr size_t kMostSmem = 200 * 1024;                       // dynamic, of a block

// The most blocks that a cluster of a head may have so that `heads` of them run at once with one block to an SM; 0 where not even single blocks do.
// (Clusters lie within a group of SMs, and the groups differ in size: of 148 SMs, 7 clusters of 16 find room, 11 of 10, 15 of 8 or 9, 22 of 6, 33 of 4.
// Clusters of an odd size, which share pairs of SMs, do not reach their number: of the 26 of 5 and 45 of 3 that the runtime counts, 24 and 44 took up to
// 23 % longer than the launch without this path (all of them 37 %), three fewer up to 13 % less.)
template <bool FOUR, bool ACCUM>
int one_block_an_sm(int heads, int* blocks)
{
    struct Counts { int of[MAX_SPLIT + 1]; };                  // clusters at a time, by their blocks
    static PerDevice<Counts> table;
    Counts n;
    if (int e = table.get(&n, [&](Counts* out) {
            auto kern = decode_rows_mma_kernel<128, MAX_WARPS, FOUR ? 3 : 2, false, FOUR, ACCUM ? KEPT : LEARNED, false>;
            if (cudaError_t x = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem)) return cuda_status(x);
            if (cudaError_t x = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1)) return cuda_status(x);
            for (int c = 1; c <= MAX_SPLIT; ++c) {
                cudaLaunchConfig_t cfg = {};
                cudaLaunchAttribute attr;
                attr.id = cudaLaunchAttributeClusterDimension;
                attr.val.clusterDim.x = c; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
                cfg.gridDim = dim3(c); cfg.blockDim = dim3(MAX_WARPS * 32); cfg.dynamicSmemBytes = kMostSmem;
                cfg.attrs = &attr; cfg.numAttrs = 1;
                if (cudaOccupancyMaxActiveClusters(&out->of[c], kern, &cfg) != cudaSuccess) { (void)cudaGetLastError(); out->of[c] = 0; }
            }
            return (int)LTE_OK; })) return e;
    *blocks = n.of[MAX_SPLIT] > 0 ? MAX_SPLIT : 8;             // (a launch takes more than 8 only where 16 are possible)
    while (*blocks > 0 && n.of[*blocks] < heads + (*blocks > 1 && *blocks % 2 ? 3 : 0)) --*blocks;
    return LTE_OK;
}

// How many warps share a head: all warps of the launch are resident at once where that is possible, as in decode_mma.cu.
template <bool FOUR, bool ACCUM>
int launch_rows_mma(const Params& p, const RowsLayout& L, bool swz, const RowsRule& rule, void* cache, const void* q1, const void* k1, const void* v1,
                    void* o1, float* lse1, cudaStream_t st)
{
    int n_sm = 0, *status = nullptr;
    if (int e = device_sm_count(&n_sm)) return e;
    if (int e = cache_status_word(&status)) return e;
    const int BH = p.B * p.H, rows = p.W + p.R, wps = warps_per_sm(p.d, FOUR), warps = wps * n_sm;
    const int UR = FOUR || p.d < 128 ? 32 : 16;                // rows that a warp takes at a time (Stage::UR)
    // Long rows of few heads take more warps and blocks: 8 heads x 17,408 rows at d = 128, four query heads each, take 39.5 us with four warps,
    // 30.9 with eight (bf16; a 4-bit block of eight takes an SM's registers, and clusters of those are for `wide` below).  Clusters of 16 only where
    // each block may have an SM to itself: 16 heads took as long as 32.
    const bool is_long = rows > 4096;
    const int most_w = p.d == 128 && (FOUR || !is_long) ? 4 : MAX_WARPS, most_split = is_long ? MAX_SPLIT : 8;
    int nw = 1, nsplit = 1;
    for (int c : {2, 4, 8})
        if (c <= most_w && BH <= n_sm * (wps / c) && rows / c >= 16) nw = c;
    if (nw == most_w)
        while (nsplit < most_split && BH * nw * nsplit * 2 <= (nsplit < 8 ? warps : warps / 2) && rows / (nw * nsplit * 2) >= 8) nsplit *= 2;
    // Accumulated attention: the logits stay in shared memory while those of the blocks that share an SM fit beside their stages.  Where they do not,
    // the keys are read once more: their half of the bytes (of which L2 has some) and of the instructions.  For bf16 rows, whose bytes count, more
    // blocks a head with fewer logits each come first, if no SM then has fewer warps and it takes at most two rounds.  Kept in more blocks | again:
    //   bf16    256 heads x 4,024 rows, 4 query heads, d = 64     59.9 | 66.7 us     64 x 17,408, 4, d = 128   113 | 139      64 x 8,192, 8, d = 128   65 | 71
    //           256 x 2,816, 8, d = 64 (half the warps)           73.3 | 48.6        512 x 2,048, 8, d = 64 (3.5 rounds)      81 | 70
    //   4 bits  256 x 2,816, 8, d = 64     39.8 | 32.8     the same at d = 128     113 | 51     256 x 4,024, 4     44 | 43     64 x 17,408, 4, d = 128    77 | 85
    const int kept = (p.G < MQ ? p.G : MQ) + (p.G > MQ ? 1 : 0);               // floats per row
    auto smem = [&](int w, int split) { return (size_t)w * (((rows + UR - 1) / UR + w * split - 1) / (w * split) * UR + 4) * kept * 4; };
    bool keep = smem(nw, nsplit) * (size_t)fmax(1., fmin(wps / nw, ((double)BH * nsplit + n_sm - 1) / n_sm)) <= 96 * 1024;
    if (!FOUR && ACCUM && !keep) {
        int more = nsplit;
        while (more < MAX_SPLIT && smem(most_w, more) > 64 * 1024) more *= 2;
        const size_t block = smem(most_w, more) + (size_t)most_w * 8 * 1024 + 12 * 1024;   // with its stages (8 KB a warp)
        if (block * (wps / most_w) <= 224 * 1024 && (long long)BH * more <= 2ll * n_sm * (wps / most_w)) { keep = true; nw = most_w; nsplit = more; }
    }
    // Heads that leave an SM one block take blocks of eight warps with a stage more, in clusters of which every block finds an SM of its own: two
    // on one SM take as long as one with the rows of both, and a block of eight 4-bit warps that finds none waits for the whole step of another.
    // us a step without | with (four query heads; bf16 accumulated, 4 bits learned):
    //   d = 128    8 heads x 17,408 rows   29.3 | 27.4, 18.5 | 16.6       12 x 17,408   46.6 | 29.9, 28.1 | 18.9       16 x 17,408   47.9 | 39.9, 28.4 | 23.8
    //              8 x 4,024   16.5 | 13.3, 11.4 | 10.0       32 x 2,560   22.0 | 16.2, 14.2 | 10.8       32 x 384   12.7 | 8.9, 12.0 | 8.4
    //              148 x 1,248   36.0 | 22.2, 14.8 | 12.6       128 x 1,536   25.5 | 23.5, 16.1 | 14.3       64 x 1,536   20.0 | 17.6, 11.8 | 11.5
    //   d = 64     16 x 17,408   31.1 | 26.8, 19.4 | 23.3       32 x 384   8.2 | 7.9       32 x 1,024   11.3 | 8.4       128 x 1,536   17.0 | 16.1
    // so not 4 bits at d = 64 (32 codes a lane leave 16 warps room).  Not few rows either (8 x 1,024, bf16: 9.9 | 9.1 at d = 128, 7.9 | 8.1 at d = 64;
    // 4 bits accumulated 9.6 | 9.8; 128 x 96, d = 64: 5.8 | 6.1).  Long bf16 rows need many SMs: 64 x 6,024 take 32.8 | 34.4 at d = 128, 20.9 | 22.5
    // at d = 64, 28 x 17,408 (112 SMs) 50.6 | 54.9, but 40 x 6,024 (120) 29.5 | 25.3.  One block a head gains up to some 4,000 rows (119 heads x 3,000, d = 128
    // 37.5 | 36.6, 148 x 3,000 61.3 | 42.6) and loses behind (119 x 8,192, one query head each: 85.6 | 86.9, d = 64 51.1 | 53.6; 148 x 17,408 223 | 233).
    bool wide = false;
    if ((FOUR ? p.d == 128 : p.d >= 64) && rows >= 128 && BH <= n_sm && (long long)BH * rows >= 12288) {
        int c = 0;
        if (int e = one_block_an_sm<FOUR, ACCUM>(BH, &c)) return e;
        const bool fits = !ACCUM || (c > 0 && smem(MAX_WARPS, c) + MAX_WARPS * (FOUR ? 3 * 5 : 2 * 8) * 1024 <= kMostSmem);
        const bool enough = rows <= 2048 || c >= 6 || ((c == 1 ? rows <= 4096 : c != 2) && BH * c * 5 >= n_sm * 4);
        if (c > 0 && (FOUR || (fits && enough))) { wide = true; keep = fits; nw = MAX_WARPS; nsplit = c; }
    }
    auto go = [&](auto d, auto w, auto s) {
        constexpr int D = decltype(d)::value, NW = decltype(w)::value;
        auto with_length = [&](auto stages, auto kind, auto is_long) {
            constexpr int STAGES = decltype(stages)::value, RULE = decltype(kind)::value;
            auto kern = decode_rows_mma_kernel<D, NW, STAGES, decltype(s)::value, FOUR, RULE, decltype(is_long)::value>;
            cudaLaunchConfig_t cfg = {};
            cudaLaunchAttribute attr[2];
            attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
            attr[0].val.programmaticStreamSerializationAllowed = 1;
            attr[1].id = cudaLaunchAttributeClusterDimension;
            attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
            static PerDevice<int> table;                       // blocks that a cluster may have, and the kernel's limits raised
            int split_most = 1;
            if (int e = table.get(&split_most, [&](int* out) {
                    if (cudaError_t x = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem)) return cuda_status(x);
                    *out = 8;
                    if (!clusters(D, NW)) return (int)LTE_OK;
                    // clusters of 16 are not portable: taken where the device can place one with the most shared memory
                    if (cudaError_t x = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1)) return cuda_status(x);
                    cfg.gridDim = dim3(MAX_SPLIT); cfg.blockDim = dim3(NW * 32); cfg.dynamicSmemBytes = kMostSmem;
                    attr[1].val.clusterDim.x = MAX_SPLIT;
                    cfg.attrs = attr + 1; cfg.numAttrs = 1;
                    int n = 0;
                    if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) == cudaSuccess && n > 0) *out = MAX_SPLIT;
                    else (void)cudaGetLastError();
                    return (int)LTE_OK; })) return e;
            const int split = nsplit < split_most ? nsplit : split_most;
            cfg.gridDim = dim3(BH * split); cfg.blockDim = dim3(NW * 32); cfg.stream = st;
            cfg.dynamicSmemBytes = (RULE == KEPT ? smem(nw, split) : 0) + NW * STAGES * Stage<D, FOUR>::BYTES;
            if (cfg.dynamicSmemBytes > kMostSmem) return (int)LTE_ERR_UNSUPPORTED;
            attr[1].val.clusterDim.x = split;
            cfg.attrs = attr; cfg.numAttrs = split > 1 ? 2 : 1;
            return cuda_status(cudaLaunchKernelEx(&cfg, kern, (unsigned char*)cache, L, (const __nv_bfloat16*)q1, (const __nv_bfloat16*)k1,
                                                  (const __nv_bfloat16*)v1, (__nv_bfloat16*)o1, lse1, rule, p.H, p.W, p.R, p.sink, p.scale, p.G,
                                                  ((rows + UR - 1) / UR + nw * split - 1) / (nw * split) * UR, status));
        };
        auto with_kind = [&](auto stages, auto kind) {
            if constexpr (FOUR) { if ((rows + nw * nsplit - 1) / (nw * nsplit) > kLongRows) return with_length(stages, kind, std::true_type()); }
            return with_length(stages, kind, std::false_type());
        };
        auto with = [&](auto stages) {
            if constexpr (!ACCUM) return with_kind(stages, std::integral_constant<int, LEARNED>());
            else return keep ? with_kind(stages, std::integral_constant<int, KEPT>()) : with_kind(stages, std::integral_constant<int, AGAIN>());
        };
        // two stages a warp; three where eight warps of an SM have the room, one where 16 have not (bf16 at d = 128: 8 KB a stage), unless few
        // heads leave it (16 x 1,024 rows: 9.7 us with one, 9.3 with two)
        if constexpr (!FOUR && D >= 64 && NW == MAX_WARPS && !decltype(s)::value) { if (wide) return with(std::integral_constant<int, 2>()); }
        if constexpr (D < 128) return with(std::integral_constant<int, FOUR || D == 32 ? 2 : 1>());
        else if constexpr (FOUR) return with(std::integral_constant<int, 3>());
        else if constexpr (NW == 4) return BH * nsplit * NW <= 8 * n_sm ? with(std::integral_constant<int, 2>()) : with(std::integral_constant<int, 1>());
        else return with(std::integral_constant<int, 1>());
    };
    auto widths = [&](auto d, auto s) {
        switch (nw) {
            case 1: return go(d, std::integral_constant<int, 1>(), s);
            case 2: return go(d, std::integral_constant<int, 2>(), s);
            case 4: return go(d, std::integral_constant<int, 4>(), s);
            default: return go(d, std::integral_constant<int, 8>(), s);
        }
    };
    switch (p.d) {
        case 32: return widths(std::integral_constant<int, 32>(), std::false_type());
        case 64:
            if constexpr (!FOUR) { if (swz) return widths(std::integral_constant<int, 64>(), std::true_type()); }
            return widths(std::integral_constant<int, 64>(), std::false_type());
        case 128: return widths(std::integral_constant<int, 128>(), std::false_type());
    }
    return LTE_ERR_UNSUPPORTED;
}

}  // namespace
}  // namespace lte
