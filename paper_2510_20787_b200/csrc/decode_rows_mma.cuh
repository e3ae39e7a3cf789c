// Decode step (lte_attn_decode_accum, lte_attn_decode4, lte_attn_decode4_accum) for bf16 calls: rows go from memory straight into tensor-core
// operands, as in decode_mma.cu, every query head of a group at once, heads split over warps and clusters where there are few.
//
// Bound by memory where rows are bf16; rows in 4 bits are 3.2 times smaller, and there unpacking and memory are about even.  Every warp
// walks spans of 16 rows (interleaved over the warps of all blocks that share the head) with NBUF spans in flight, keeps its own
// reference, sum and output, and meets the others once at the end.  The incoming token is no row: its logit is a dot product on the fp32 ALUs, and it
// joins where the warps meet.
//
// Scores (accumulated attention): a row's weight needs the sum over all rows, so the raw logits of a warp's rows stay in shared memory until the
// blocks have met; then every warp adds its rows' weights, summed over the query heads, to their scores.  One read and one write of 4 bytes a row.
//
// Products are mma.sync m16n8k16: logits S^T[16 rows][8 queries] = K q^T, output O^T[16 channels][8 queries] += V^T P^T, N = 8 queries.
// Rows in 4 bits.  A code c becomes the bf16 number 16 + c by a shift and one three-input logic operation on two codes at a time (the code is
// the top of the mantissa): exact, no conversion.  With value = zero + c step = (zero - 16 step) + step (16 + c):
//   logits   per group of 32 channels, step (16 + c).q + (zero - 16 step) sum(q): the group's product starts from zero, and its two scalars,
//            which belong to a row, are applied to the products in fp32 (a lane holds rows g and g + 8 of both);
//   output   P step takes the place of P, per group, and P (zero - 16 step), which is the same for all channels of a group, is summed beside it.
// The contraction index may be permuted freely: the nibbles i and i + 4 of a key word are neighbours in it, and so are the two rows whose value
// units a byte permute joins.  The order of the codes in the cache (cache4.cuh) makes these the words that a lane loads.
// P (times step) is split into two bf16 terms: 16 bits of mantissa.  With one term o would be off by more than its own rounding: the 16 + c
// are all positive, so that o is the small difference of sums as large as the rows.
#pragma once
#include <cfloat>
#include <cooperative_groups.h>

#include <type_traits>

#include "decode_rows.cuh"
#include "row_mma.cuh"
#include "tc_common.cuh"

namespace lte {
namespace cg = cooperative_groups;
namespace {

constexpr int MQ = 8;                                          // query heads per pass
// resident warps the registers (and the stages in shared memory) are budgeted for
__host__ __device__ constexpr int warps_per_sm(int d, bool four) { return d == 128 ? 8 : 16; }
__host__ __device__ constexpr int max_warps(int d) { return d == 128 ? 4 : 8; }       // per block
constexpr int MAX_SPLIT = 8;                                   // blocks per head

// A head's rows in use are rows 0 .. total - 1 of its block (while the ring fills up the pool is empty).  A warp takes units of UR of them, 16 to
// a product, which pass through STAGES of its own in shared memory: bulk copies that its lane 0 starts, a barrier per stage.  (With the units in
// registers, enough of them in flight and the products' operands did not fit 128 registers, and every load cost its address arithmetic in
// every lane: 256 heads x 1,280 rows in 4 bits 23.7 us, through shared memory 18.5.)
struct Rows {
    const unsigned char *K, *V, *KP, *VP;
    int total;
};
template <int D, bool FOUR> struct Stage {
    static constexpr int UR = FOUR ? 32 : 16, STAGES = FOUR ? 3 : 2;
    static constexpr int ROW = FOUR ? D / 2 : 2 * D, PAR = FOUR ? D / 8 : 0;   // bytes of a row's keys, of its key parameters
    static constexpr int K = 0, V = UR * ROW, KP = 2 * V, VP = KP + UR * PAR, BYTES = VP + UR * PAR;
    static constexpr int ACC = MQ * (D + 8) * 4;               // a warp's outputs stand where its stages were
    static_assert(ACC <= STAGES * BYTES, "");
};

// The two products with a span of 16 rows that stands in shared memory, lane (g, t) = (lane / 4, lane % 4).  Rows past the last one and those that the
// step leaves out have weight zero, and what they hold is cleared (zero times an infinite value is NaN).
template <int D, bool SWZ, bool FOUR> struct Group;

template <int D, bool SWZ> struct Group<D, SWZ, false> {
    static constexpr int KP = D / 32, VB = D / 16, PITCH = D * 2, MT = D / 16;
    struct Query { uint4 f[KP]; };                             // pieces t, t + 4, .. of query g
    struct Acc { float a[MT][4]; };
    static __device__ __forceinline__ int rho(int g) { return g; }
    static __device__ __forceinline__ void load_q(Query& Q, const __nv_bfloat16* q, bool some, int g, int t)
    {
#pragma unroll
        for (int j = 0; j < KP; ++j) Q.f[j] = some ? reinterpret_cast<const uint4*>(q + (size_t)g * D)[t + 4 * j] : make_uint4(0, 0, 0, 0);
    }
    // c: rows g (0, 1) and g + 8 (2, 3), queries 2t and 2t + 1.  A product rounds its running sum towards zero, so every one starts from zero
    // and the parts are added to the nearest (see decode_mma.cu).  Lane (g, t) takes pieces t, t + 4, .. of rows g and g + 8.
    static __device__ __forceinline__ void logits(float (&c)[4], const Query& Q, const unsigned char* st, int span, int g, int t)
    {
        uint4 k[2][KP];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < KP; ++j)
                k[u][j] = *reinterpret_cast<const uint4*>(st + Stage<D, false>::K + (16 * span + g + 8 * u) * PITCH + (((t + 4 * j) ^ (SWZ ? g & 7 : 0)) << 4));
        constexpr int NS = D == 128 ? 2 * KP : 1;
        float cs[NS][4];
#pragma unroll
        for (int i = 0; i < 2 * KP; ++i) {
            const int j = i >> 1, s = 2 * (i & 1);
            float part[4] = {0.f, 0.f, 0.f, 0.f};
            mma16816(part, word(k[0][j], s), word(k[1][j], s), word(k[0][j], s + 1), word(k[1][j], s + 1), word(Q.f[j], s), word(Q.f[j], s + 1));
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
    // gone: bit r: row r of the span does not count.  Lane (g, t) takes pieces g, g + 8 of rows 2t, 2t + 1, 2t + 8, 2t + 9.
    static __device__ __forceinline__ void output(Acc& A, const float (&p)[4], const unsigned char* st, int span, unsigned gone, int g, int t)
    {
        uint32_t v[4][VB];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int r = 2 * t + (u & 1) + 8 * (u >> 1);
            const unsigned char* base = st + Stage<D, false>::V + (16 * span + r) * PITCH;
            if constexpr (D == 32) {
                const uint2 x = *reinterpret_cast<const uint2*>(base + (g << 3));
                v[u][0] = x.x; v[u][1] = x.y;
            } else {
#pragma unroll
                for (int j = 0; j < D / 64; ++j) {
                    const uint4 x = *reinterpret_cast<const uint4*>(base + (((g + 8 * j) ^ (SWZ ? r & 7 : 0)) << 4));
#pragma unroll
                    for (int w = 0; w < 4; ++w) v[u][4 * j + w] = word(x, w);
                }
            }
        }
        if (gone)
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if ((gone >> (2 * t + (u & 1) + 8 * (u >> 1))) & 1u)
#pragma unroll
                    for (int j = 0; j < VB; ++j) v[u][j] = 0u;
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

// two codes of a word, at bits 4i and 4i + 16, as the bf16 numbers 16 + c
// (one LOP3: with both constants as immediates the compiler takes two)
__device__ __forceinline__ uint32_t reg(uint32_t x) { asm("" : "+r"(x)); return x; }
template <int I> __device__ __forceinline__ uint32_t codes2(uint32_t x, uint32_t mask, uint32_t sixteen)
{
    const uint32_t y = I == 0 ? x << 3 : x >> (4 * I - 3);
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(y), "r"(mask), "r"(sixteen));     // (y & mask) | sixteen
    return r;
}

// Rows in 4 bits: a span stands in shared memory, where the products take their operands from.  M-row r of a product is row rho(r) of the span,
// rho(2t + b + 8c) = t + 4b + 8c: the value units that the lanes load at once then lie in different banks.
template <int D, bool SWZ> struct Group<D, SWZ, true> {
    static constexpr int GR = D / kGroup4, MT = D / 16;
    struct Query { uint32_t f[GR][4]; float sum[GR][2]; };     // of query g; sums of queries 2t, 2t + 1 over a group's channels
    struct Acc { float a[MT][4], z[GR][2]; };
    template <typename U> static __device__ __forceinline__ void get(uint32_t (&x)[GR], const unsigned char* p)
    {
        const U u = *reinterpret_cast<const U*>(p);
        memcpy(x, &u, sizeof(U));
    }
    using Words = std::conditional_t<GR == 1, uint32_t, std::conditional_t<GR == 2, uint2, uint4>>;
    using Units = std::conditional_t<GR == 1, uint16_t, std::conditional_t<GR == 2, uint32_t, uint2>>;
    static __device__ __forceinline__ int rho(int g) { return (g >> 1) + 4 * (g & 1); }     // (g < 8)
    static __device__ __forceinline__ void load_q(Query& Q, const __nv_bfloat16* q, bool some, int g, int t)
    {
        const int lane = 4 * g + t;
#pragma unroll
        for (int j = 0; j < GR; ++j) {
            const uint4 u = some ? reinterpret_cast<const uint4*>(q + (size_t)g * D + j * kGroup4)[t] : make_uint4(0, 0, 0, 0);
            Q.f[j][0] = __byte_perm(u.x, u.z, 0x5410); Q.f[j][1] = __byte_perm(u.x, u.z, 0x7632);   // channels 0, 4 | 1, 5
            Q.f[j][2] = __byte_perm(u.y, u.w, 0x5410); Q.f[j][3] = __byte_perm(u.y, u.w, 0x7632);   // 2, 6 | 3, 7
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) s += __uint_as_float(word(u, w) << 16) + __uint_as_float(word(u, w) & 0xffff0000u);
            s += __shfl_xor_sync(0xffffffffu, s, 1);
            s += __shfl_xor_sync(0xffffffffu, s, 2);
            Q.sum[j][0] = __shfl_sync(0xffffffffu, s, 8 * (lane & 3));
            Q.sum[j][1] = __shfl_sync(0xffffffffu, s, 8 * (lane & 3) + 4);
        }
    }
    static __device__ __forceinline__ void logits(float (&c)[4], const Query& Q, const unsigned char* st, int span, int g, int t)
    {
        const unsigned char *keys = st + Stage<D, true>::K + span * (8 * D), *pars = st + Stage<D, true>::KP + span * (64 * GR);
        const uint32_t M = reg(0x00780078u), S = reg(0x41804180u);
        uint32_t k[2][GR], kp[2][GR];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            get<Words>(k[u], keys + (rho(g) + 8 * u) * (D / 2) + t * (4 * GR));
            get<Words>(kp[u], pars + (rho(g) + 8 * u) * (4 * GR));
        }
#pragma unroll
        for (int j = 0; j < GR; ++j) {
            float p[4] = {0.f, 0.f, 0.f, 0.f};
            mma16816(p, codes2<0>(k[0][j], M, S), codes2<0>(k[1][j], M, S), codes2<1>(k[0][j], M, S), codes2<1>(k[1][j], M, S), Q.f[j][0], Q.f[j][1]);
            mma16816(p, codes2<2>(k[0][j], M, S), codes2<2>(k[1][j], M, S), codes2<3>(k[0][j], M, S), codes2<3>(k[1][j], M, S), Q.f[j][2], Q.f[j][3]);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float s = par4_step(kp[i][j]), z = fmaf(-16.f, s, par4_zero(kp[i][j]));
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float x = fmaf(s, p[2 * i + e], z * Q.sum[j][e]);
                    c[2 * i + e] = j == 0 ? x : c[2 * i + e] + x;
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
    }
    static __device__ __forceinline__ void rescale(Acc& A, float f0, float f1)
    {
#pragma unroll
        for (int m = 0; m < MT; ++m) { A.a[m][0] *= f0; A.a[m][1] *= f1; A.a[m][2] *= f0; A.a[m][3] *= f1; }
#pragma unroll
        for (int j = 0; j < GR; ++j) { A.z[j][0] *= f0; A.z[j][1] *= f1; }
    }
    static __device__ __forceinline__ void output(Acc& A, const float (&p)[4], const unsigned char* st, int span, unsigned gone, int g, int t)
    {
        const unsigned char *values = st + Stage<D, true>::V + span * (8 * D), *pars = st + Stage<D, true>::VP + span * (64 * GR);
        const uint32_t M = reg(0x00780078u), S = reg(0x41804180u);
        uint32_t v[4][(GR + 1) / 2], vp[2][GR];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const Units x = *reinterpret_cast<const Units*>(values + (t + 4 * u) * (D / 2) + g * (2 * GR));   // M-rows 2t + (u & 1) + 8 (u / 2)
            if constexpr (GR == 1) v[u][0] = x;
            else memcpy(v[u], &x, sizeof(x));
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) get<Words>(vp[u], pars + (rho(g) + 8 * u) * (4 * GR));
        if (gone)
#pragma unroll
            for (int u = 0; u < 2; ++u)
                if ((gone >> (rho(g) + 8 * u)) & 1u)
#pragma unroll
                    for (int j = 0; j < GR; ++j) vp[u][j] = 0u;
#pragma unroll
        for (int j = 0; j < GR; ++j) {
            const float s0 = par4_step(vp[0][j]), s1 = par4_step(vp[1][j]);
            const float z0 = fmaf(-16.f, s0, par4_zero(vp[0][j])), z1 = fmaf(-16.f, s1, par4_zero(vp[1][j]));
            A.z[j][0] = fmaf(p[2], z1, fmaf(p[0], z0, A.z[j][0]));
            A.z[j][1] = fmaf(p[3], z1, fmaf(p[1], z0, A.z[j][1]));
            const float x0 = p[0] * s0, x1 = p[1] * s0, x2 = p[2] * s1, x3 = p[3] * s1;
            const uint32_t hi0 = pack_bf16(x0, x1), hi1 = pack_bf16(x2, x3);
            const uint32_t lo0 = pack_bf16(x0 - __uint_as_float(hi0 << 16), x1 - __uint_as_float(hi0 & 0xffff0000u));
            const uint32_t lo1 = pack_bf16(x2 - __uint_as_float(hi1 << 16), x3 - __uint_as_float(hi1 & 0xffff0000u));
            const uint32_t h0 = movmatrix_trans(hi0), h1 = movmatrix_trans(hi1), e0 = movmatrix_trans(lo0), e1 = movmatrix_trans(lo1);
            const uint32_t u = __byte_perm(v[0][j / 2], v[1][j / 2], j & 1 ? 0x7632 : 0x5410);   // four codes of M-row 2t, of M-row 2t + 1
            const uint32_t w = __byte_perm(v[2][j / 2], v[3][j / 2], j & 1 ? 0x7632 : 0x5410);
            const uint32_t u0 = codes2<0>(u, M, S), u1 = codes2<1>(u, M, S), u2 = codes2<2>(u, M, S), u3 = codes2<3>(u, M, S);
            const uint32_t w0 = codes2<0>(w, M, S), w1 = codes2<1>(w, M, S), w2 = codes2<2>(w, M, S), w3 = codes2<3>(w, M, S);
            mma16816(A.a[2 * j], u0, u1, w0, w1, h0, h1);
            mma16816(A.a[2 * j + 1], u2, u3, w2, w3, h0, h1);
            mma16816(A.a[2 * j], u0, u1, w0, w1, e0, e1);
            mma16816(A.a[2 * j + 1], u2, u3, w2, w3, e0, e1);
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
                A.a[2 * j][e] += z; A.a[2 * j][2 + e] += z; A.a[2 * j + 1][e] += z; A.a[2 * j + 1][2 + e] += z;
            }
    }
    static __device__ __forceinline__ int channel(int m, int g) { return (m >> 1) * kGroup4 + 4 * g + 2 * (m & 1); }
};

__device__ StatusWord g_rows_status = LTE_STATUS_INIT;

__device__ __forceinline__ void bulk_copy(uint32_t to, const unsigned char* from, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(bytes), "r"(bar) : "memory");
}

template <int D, int NW, bool SWZ, bool FOUR, bool ACCUM>
__global__ void __launch_bounds__(NW * 32, warps_per_sm(D, FOUR) / NW) decode_rows_mma_kernel(
    unsigned char* __restrict__ cache, RowsLayout L, const __nv_bfloat16* __restrict__ q1, const __nv_bfloat16* __restrict__ k1,
    const __nv_bfloat16* __restrict__ v1, __nv_bfloat16* __restrict__ o1, float* __restrict__ lse1, RowsRule rule, int H, int W, int R, int sink,
    float scale, int G, int most)                              // most: rows whose logits a warp keeps (whole spans)
{
    using Gr = Group<D, SWZ, FOUR>;
    constexpr int NT = NW * 32, MT = D / 16, PITCH = D + 8, CPL = D / 32, GR = D / kGroup4;
    using St = Stage<D, FOUR>;
    constexpr int UR = St::UR, UNIT = UR / 16;
    constexpr int SPLIT = NW == max_warps(D) ? MAX_SPLIT : 1;  // (only the largest blocks come in clusters)
    extern __shared__ __align__(128) unsigned char s_dyn[];    // the warps' stages; [NW][most][nq] logits, behind them [NW][most] sums over passes
    float* const s_log = reinterpret_cast<float*>(s_dyn + NW * St::STAGES * St::BYTES);
    auto s_acc = [&](int w, int u) { return reinterpret_cast<float*>(s_dyn + w * (St::STAGES * St::BYTES)) + u * PITCH; };
    __shared__ __align__(8) uint64_t s_bar[NW * St::STAGES];
    __shared__ float s_m[NW][MQ], s_l[NW][MQ], s_new[MQ];
    __shared__ float s_in[2][SPLIT > 1 ? MQ * D : 1];
    __shared__ __align__(16) float s_ml[2][SPLIT][MQ][2];      // the cluster's shares of this block's output elements (by pass parity)
    __shared__ __align__(16) __nv_bfloat16 s_kv[2][D];         // the incoming token
    __shared__ float s_tap[NW];
    __shared__ uint32_t s_wkey[NW];
    __shared__ int s_wpos[NW], s_wslot[NW];
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
    if (lane == 0) {
        for (int i = 0; i < St::STAGES; ++i) tc::mbar_init(tc::smem_u32(&s_bar[wid * St::STAGES + i]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    pdl_wait();

    // Everything whose address is known is asked for at once: the rows that a warp begins with too, whether or not they turn out to be in use.
    Rows rows;
    rows.K = blk + L.off_k; rows.V = blk + L.off_v; rows.KP = blk + L.off_kp; rows.VP = blk + L.off_vp;
    rows.total = W + R;
    const int step = NW * nsplit, first = wid * nsplit + rank;
    unsigned char* const stage = s_dyn + wid * (St::STAGES * St::BYTES);
    const uint32_t bar = tc::smem_u32(&s_bar[wid * St::STAGES]);
    int asked = 0, taken = 0;                                  // units of this warp, over all passes: number j goes through stage j % STAGES
    auto ask = [&](int i) {
        if (lane == 0) {
            const uint32_t nr = min(UR, rows.total - UR * i), row = nr * St::ROW, par = (nr * St::PAR + 15) & ~15u;   // (a part's size in the cache is a multiple of 16)
            const uint32_t b = bar + 8 * (asked % St::STAGES), to = tc::smem_u32(stage + (asked % St::STAGES) * St::BYTES);
            tc::mbar_expect_tx(b, 2 * (row + par));
            bulk_copy(to + St::K, rows.K + (size_t)i * (UR * St::ROW), row, b);
            if (FOUR) bulk_copy(to + St::KP, rows.KP + (size_t)i * (UR * St::PAR), par, b);
            bulk_copy(to + St::V, rows.V + (size_t)i * (UR * St::ROW), row, b);
            if (FOUR) bulk_copy(to + St::VP, rows.VP + (size_t)i * (UR * St::PAR), par, b);
        }
        ++asked;
    };
    auto wait = [&](int code) { tc::mbar_wait_uni(bar + 8 * (taken % St::STAGES), (taken / St::STAGES) & 1, code, &g_rows_status); };
    auto begin = [&](int units_there) {                        // the first units of a pass
#pragma unroll
        for (int b = 0; b < St::STAGES; ++b)
            if (first + b * step < units_there) ask(first + b * step);
    };
    begin((rows.total + UR - 1) / UR);
    const int n = max(meta[0], 0), cnt_old = min(max(meta[1], 0), R);
    typename Gr::Query qf;
    Gr::load_q(qf, q1 + (size_t)bh * G * D, g < G, g, t);
    constexpr int PRE = NT < 256 ? 4 : 2;                      // scores and positions of the pool, before it is known whether the decision needs them
    float pz[PRE];
    int pp[PRE];
#pragma unroll
    for (int u = 0; u < PRE; ++u) {
        const int m = tid + u * NT;
        pz[u] = m < R ? zc[W + m] : INFINITY;
        pp[u] = m < R ? pidx[m] : -1;
    }
    if (tid < D / 4) reinterpret_cast<uint4*>(s_kv)[tid] = reinterpret_cast<const uint4*>((tid < D / 8 ? k1 : v1) + (size_t)bh * D)[tid % (D / 8)];
    const int slot = n % W, p = n - W, half = rule.K / 2;
    rows.total = n < W ? n : W + cnt_old;
    const int units = (rows.total + UR - 1) / UR, full = rows.total / UR;
    const float zp = p >= 0 ? zc[slot] : 0.f;
    // Learned rule, the first block: logit of the newest token whose receptive field is complete.  A lane takes eight channels under a tap: a
    // word of the row's key or value codes, two runs of four weights.
    const int jsc = ACCUM ? -1 : n - half;
    constexpr int LT = D / 4, TAPS = 32 / LT;                  // lanes per tap, taps of a warp at a time
    struct Tap { uint4 x; float w[8]; uint32_t par[2]; bool held; };
    const int tap_word = lane % LT % (D / 8), tap_values = lane % LT / (D / 8);
    auto tap_ask = [&](Tap& T, int tap) {
        const int pos = n - (rule.K - 1) + tap;                // (the ring holds at least K tokens)
        T.held = pos != n;
        T.x = make_uint4(0, 0, 0, 0);
        T.par[0] = T.par[1] = 0u;
#pragma unroll
        for (int e = 0; e < 8; ++e) T.w[e] = 0.f;
        if (tap >= rule.K || pos < 0) return;
        const int ch0 = tap_values ? value4_channel(tap_word, 0, GR) : key4_channel(tap_word, 0, GR);
        const int ch4 = tap_values ? value4_channel(tap_word, 4, GR) : key4_channel(tap_word, 4, GR);
        const float* w = rule.w + ((size_t)h * rule.K + tap) * 2 * D + tap_values * D;
        if ((reinterpret_cast<uintptr_t>(rule.w) & 15u) == 0) {
            const float4 a = *reinterpret_cast<const float4*>(w + ch0), b = *reinterpret_cast<const float4*>(w + ch4);
            T.w[0] = a.x; T.w[1] = a.y; T.w[2] = a.z; T.w[3] = a.w; T.w[4] = b.x; T.w[5] = b.y; T.w[6] = b.z; T.w[7] = b.w;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) { T.w[e] = w[ch0 + e]; T.w[4 + e] = w[ch4 + e]; }
        }
        if (T.held) {
            const int back = slot + tap - (rule.K - 1), r = back < 0 ? back + W : back;
            T.x.x = reinterpret_cast<const uint32_t*>((tap_values ? rows.V : rows.K) + (size_t)r * (D / 2))[tap_word];
            const uint32_t* par = reinterpret_cast<const uint32_t*>(tap_values ? rows.VP : rows.KP) + (size_t)r * GR;
            T.par[0] = par[ch0 / kGroup4]; T.par[1] = par[ch4 / kGroup4];
        } else {                                               // the incoming token, as given
            const __nv_bfloat16* x = (tap_values ? v1 : k1) + (size_t)bh * D;
            const uint2 a = *reinterpret_cast<const uint2*>(x + ch0), b = *reinterpret_cast<const uint2*>(x + ch4);
            T.x = make_uint4(a.x, a.y, b.x, b.y);
        }
    };
    auto tap_sum = [&](const Tap& T) {
        float a = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t u = word(T.x, e >> 1);
            const float x = T.held ? value4((T.x.x >> (4 * e)) & 15u, T.par[e >> 2]) : __uint_as_float(e & 1 ? u & 0xffff0000u : u << 16);
            a = fmaf(T.w[e], x, a);
        }
        return a;
    };
    Tap tap0;
    const bool scores = !ACCUM && rank == 0 && jsc >= 0;
    if (scores) tap_ask(tap0, wid * TAPS + lane / LT);

    // ---- what happens to the token leaving the window ------------------------------------------------------------
    int dst = -1, cnt_new = cnt_old;
    if (p >= 0 && R > 0 && (ACCUM || p < sink || zp > rule.zthr)) {
        if (cnt_old < R) { dst = cnt_old; cnt_new = cnt_old + 1; }
        else if (p >= sink) {
            Worst w;
#pragma unroll
            for (int u = 0; u < PRE; ++u) if (tid + u * NT < cnt_old) w.offer(pz[u], pp[u], tid + u * NT, sink);
            for (int m = tid + PRE * NT; m < cnt_old; m += NT) w.offer(zc[W + m], pidx[m], m, sink);
            w.over_warp();
            if (NW > 1) {
                if (lane == 0) { s_wkey[wid] = w.key; s_wpos[wid] = w.pos; s_wslot[wid] = w.slot; }
                __syncthreads();
                w.key = lane < NW ? s_wkey[lane] : 0xffffffffu; w.pos = lane < NW ? s_wpos[lane] : -1; w.slot = lane < NW ? s_wslot[lane] : -1;
                w.over_warp();
            }
            if (w.slot >= 0 && order_key(zp + 0.f) > w.key) dst = w.slot;
        }
    }
    const int masked_ring = p >= 0 && dst < 0 ? slot : -32;    // the popped row counts iff the pool takes it ...
    const int masked_pool = dst >= 0 && dst < cnt_old ? W + dst : -32;   // ... and then the entry it replaces does not

    if (scores) {
        float a = tap_sum(tap0);
        for (int tap = (wid + NW) * TAPS; tap < rule.K; tap += NW * TAPS) {
            tap_ask(tap0, tap + lane / LT);
            a += tap_sum(tap0);
        }
        a = warp_sum(a);
        if (lane == 0) s_tap[wid] = a;
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

    const float scale2 = scale * 1.44269504088896340736f, jump = 8.f / scale2;   // jump: a factor of 2^8 between weights, unscaled
    const int nqs = min(G, MQ);                                // logits kept per row
    float* wlog = s_log + (size_t)wid * most * nqs;            // this warp's
    float* wsum = s_log + (size_t)NW * most * nqs + (size_t)wid * most;
    float fresh = 0.f;                                         // the incoming token's weights (thread 0 of the first block)
    for (int g0 = 0; g0 < G; g0 += MQ) {
        const int nq = min(MQ, G - g0);
        if (g0 > 0) {                                          // further query heads read the rows again
            Gr::load_q(qf, q1 + ((size_t)bh * G + g0) * D, g < nq, g, t);
            __syncthreads();                                   // the previous pass's outputs, which stand in the stages, have been combined
            tc::fence_proxy_async();
            begin(units);
        }
        typename Gr::Acc acc;
        Gr::start(acc);
        float m0 = -FLT_MAX, m1 = -FLT_MAX, l0 = 0.f, l1 = 0.f;
        int kept = 0;                                          // rows whose logits this warp has kept

#pragma unroll 1
        for (int i = first; i < units; i += step) {
            float c[UNIT][4], p[UNIT][4];
            const unsigned char* st = stage + (taken % St::STAGES) * St::BYTES;
            wait(1);
#pragma unroll
            for (int x = 0; x < UNIT; ++x) Gr::logits(c[x], qf, st, x, g, t);
            unsigned gone = 0;                                 // rows of the unit that do not count
            if (i >= full || i == masked_ring / UR || i == masked_pool / UR) {
                if (i >= full) gone = ~0u << (rows.total - UR * i);
                if (i == masked_ring / UR) gone |= 1u << (masked_ring % UR);
                if (i == masked_pool / UR) gone |= 1u << (masked_pool % UR);
#pragma unroll
                for (int x = 0; x < UNIT; ++x) {
                    if ((gone >> (16 * x + Gr::rho(g))) & 1u) c[x][0] = c[x][1] = -INFINITY;
                    if ((gone >> (16 * x + Gr::rho(g) + 8)) & 1u) c[x][2] = c[x][3] = -INFINITY;
                }
            }
            if constexpr (ACCUM) {                             // raw logits [row][query]
                float* at = wlog + (size_t)(kept + Gr::rho(g)) * nq + 2 * t;
#pragma unroll
                for (int x = 0; x < UNIT; ++x) {
                    if (2 * t < nq) { at[16 * x * nq] = c[x][0]; at[(16 * x + 8) * nq] = c[x][2]; }
                    if (2 * t + 1 < nq) { at[16 * x * nq + 1] = c[x][1]; at[(16 * x + 8) * nq + 1] = c[x][3]; }
                }
                kept += UR;
            }
            // The reference m follows the maximum only when that has grown by 2^8 (weights stay below 2^8, in fp32): a vote per
            // unit instead of a reduction over its rows.
            float x0 = fmaxf(c[0][0], c[0][2]), x1 = fmaxf(c[0][1], c[0][3]);
#pragma unroll
            for (int x = 1; x < UNIT; ++x) { x0 = fmaxf(x0, fmaxf(c[x][0], c[x][2])); x1 = fmaxf(x1, fmaxf(c[x][1], c[x][3])); }
            if (__any_sync(0xffffffffu, x0 > m0 + jump || x1 > m1 + jump)) {
                float y0 = x0, y1 = x1;
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) {
                    y0 = fmaxf(y0, __shfl_xor_sync(0xffffffffu, y0, o));
                    y1 = fmaxf(y1, __shfl_xor_sync(0xffffffffu, y1, o));
                }
                y0 = fmaxf(y0, m0); y1 = fmaxf(y1, m1);
                const float f0 = exp2_fast((m0 - y0) * scale2), f1 = exp2_fast((m1 - y1) * scale2);
                m0 = y0; m1 = y1;
                l0 *= f0; l1 *= f1;
                Gr::rescale(acc, f0, f1);
            }
#pragma unroll
            for (int x = 0; x < UNIT; ++x) {
#pragma unroll
                for (int e = 0; e < 4; ++e) p[x][e] = exp2_fast((c[x][e] - (e & 1 ? m1 : m0)) * scale2);
                l0 += p[x][0] + p[x][2]; l1 += p[x][1] + p[x][3];
            }
#pragma unroll
            for (int x = 0; x < UNIT; ++x) Gr::output(acc, p[x], st, x, (gone >> (16 * x)) & 0xffffu, g, t);
            ++taken;
            __syncwarp();                                      // every lane has read the stage
            if (i + St::STAGES * step < units) ask(i + St::STAGES * step);
        }
        for (; taken < asked; ++taken) wait(2);                // units asked for before it was known how many rows are in use
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
        if (ACCUM && last) load_old(lane);
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) { l0 += __shfl_xor_sync(0xffffffffu, l0, o); l1 += __shfl_xor_sync(0xffffffffu, l1, o); }
        Gr::finish(acc);
        __syncthreads();                                       // the incoming token is there; the previous pass has been combined
        if (g == 0) { s_m[wid][2 * t] = m0; s_m[wid][2 * t + 1] = m1; s_l[wid][2 * t] = l0; s_l[wid][2 * t + 1] = l1; }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int ch = Gr::channel(i, g);
            if (2 * t < nq) *reinterpret_cast<float2*>(&s_acc(wid, 2 * t)[ch]) = make_float2(acc.a[i][0], acc.a[i][2]);
            if (2 * t + 1 < nq) *reinterpret_cast<float2*>(&s_acc(wid, 2 * t + 1)[ch]) = make_float2(acc.a[i][1], acc.a[i][3]);
        }
        if (rank == 0)                                         // the incoming token's logits
            for (int u = wid; u < nq; u += NW) {
                float a = 0.f;
#pragma unroll
                for (int c = 0; c < CPL; ++c)
                    a = fmaf(__bfloat162float(q1[((size_t)bh * G + g0 + u) * D + lane + 32 * c]), __bfloat162float(s_kv[0][lane + 32 * c]), a);
                a = warp_sum(a);
                if (lane == 0) s_new[u] = a;
            }
        __syncthreads();
        if (shared_head && g0 == 0) cluster.barrier_wait();    // every block of the cluster has started: its shared memory is there
        const int per = nq * D / nsplit, par = (g0 / MQ) & 1;  // output elements each block of the cluster finishes
        // reference and sum of a query over this block's rows (and the incoming token, in the first block)
        auto block_sum = [&](int u, float& m, float& tot) {
            m = rank == 0 ? fmaxf(s_new[u], -FLT_MAX) : -FLT_MAX;
#pragma unroll
            for (int w2 = 0; w2 < NW; ++w2) m = fmaxf(m, s_m[w2][u]);
            tot = rank == 0 ? exp2_fast((s_new[u] - m) * scale2) : 0.f;
#pragma unroll
            for (int w2 = 0; w2 < NW; ++w2) tot = fmaf(exp2_fast((s_m[w2][u] - m) * scale2), s_l[w2][u], tot);   // (a warp without rows: 0)
        };
        for (int e = tid; e < nq * D; e += NT) {
            const int u = e / D, ch = e - u * D;
            float m, tot;
            block_sum(u, m, tot);
            float o = rank == 0 ? exp2_fast((s_new[u] - m) * scale2) * __bfloat162float(s_kv[1][ch]) : 0.f;
#pragma unroll
            for (int w2 = 0; w2 < NW; ++w2) o = fmaf(exp2_fast((s_m[w2][u] - m) * scale2), s_acc(w2, u)[ch], o);
            if (!shared_head) {
                o1[((size_t)bh * G + g0 + u) * D + ch] = __float2bfloat16_rn(o / tot);
                if (ch == 0) lse1[(size_t)bh * G + g0 + u] = m * scale + logf(tot);
            } else {                                           // into the shared memory of the block that finishes this element
                const int own = e / per;
                *cluster.map_shared_rank(&s_in[par][rank * per + (e - own * per)], own) = o;
                if (ch < nsplit) *reinterpret_cast<float2*>(cluster.map_shared_rank(&s_ml[par][rank][u][0], ch)) = make_float2(m, tot);
            }
        }
        auto head_sum = [&](int u, float& m, float& tot) {     // over the whole head, once the blocks have met
            if (!shared_head) { block_sum(u, m, tot); return; }
            m = -FLT_MAX; tot = 0.f;
#pragma unroll
            for (int r2 = 0; r2 < SPLIT; ++r2) if (r2 < nsplit) m = fmaxf(m, s_ml[par][r2][u][0]);
#pragma unroll
            for (int r2 = 0; r2 < SPLIT; ++r2) if (r2 < nsplit) tot = fmaf(exp2_fast((s_ml[par][r2][u][0] - m) * scale2), s_ml[par][r2][u][1], tot);
        };
        if (shared_head) {
            cluster.sync();                                    // all shares have arrived, and every row has been read
            for (int e = tid; e < per; e += NT) {
                const int el = rank * per + e, u = el / D, ch = el - u * D;
                float m, tot, o = 0.f;
                head_sum(u, m, tot);
                for (int r2 = 0; r2 < nsplit; ++r2) o = fmaf(exp2_fast((s_ml[par][r2][u][0] - m) * scale2), s_in[par][r2 * per + e], o);
                o1[((size_t)bh * G + g0 + u) * D + ch] = __float2bfloat16_rn(o / tot);
                if (ch == 0) lse1[(size_t)bh * G + g0 + u] = m * scale + logf(tot);
            }
        }
        if constexpr (ACCUM) {
            // ---- weights of this warp's rows into their scores.  Every block has read the old ones that its decision needs.
            float fm = 0.f, fi = 0.f, ms[MQ], is[MQ];
            if (lane < nq) { head_sum(lane, fm, fi); fi = 1.f / fi; }
#pragma unroll
            for (int u = 0; u < MQ; ++u) { ms[u] = __shfl_sync(0xffffffffu, fm, u); is[u] = __shfl_sync(0xffffffffu, fi, u); }
            for (int e0 = lane; e0 < kept; e0 += 32 * BATCH) {
                if (last && e0 >= 32 * BATCH) load_old(e0);
#pragma unroll
                for (int b = 0; b < BATCH; ++b) {
                    const int e = e0 + 32 * b, row = row_of(e);
                    if (e >= kept) break;
                    float a = 0.f;
#pragma unroll
                    for (int u = 0; u < MQ; ++u)
                        if (u < nq) a = fmaf(exp2_fast((wlog[(size_t)e * nq + u] - ms[u]) * scale2), is[u], a);
                    if (G > MQ) { if (g0 > 0) a += wsum[e]; wsum[e] = a; }
                    if (last && counts(row)) zc[row == slot && p >= 0 ? W + dst : row] = rule.decay > 0.f ? fmaf(rule.decay, old[b], a) : a;
                }
            }
            __syncwarp();                                      // (the next pass writes logits where these were)
            if (rank == 0 && wid == 0)
#pragma unroll
                for (int u = 0; u < MQ; ++u)
                    if (u < nq) fresh = fmaf(exp2_fast((s_new[u] - ms[u]) * scale2), is[u], fresh);
        }
    }

    // ---- write-back: only what changed; every read of the old block lies before the barriers above ------------------
    if (rank != 0) return;
    if (dst >= 0)
#pragma unroll
        for (int u = 0; u < MOVES; ++u)
            if (NT - 1 - tid + u * NT < WORDS) *place(NT - 1 - tid + u * NT, W + dst) = mv[u];
    if constexpr (FOUR) {
        // the incoming row's codes: eight channels a lane, four lanes a group
        if (wid == NW - 1) {
            const int e = min(lane, D / 4 - 1), piece = e % (D / 8), grp = piece / 4, tt = piece % 4;
            const bool values = e >= D / 8;
            const uint4 u = reinterpret_cast<const uint4*>(s_kv[values])[piece];
            float f[8], lo, hi;
            bool bad = false;
#pragma unroll
            for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(word(u, i) << 16); f[2 * i + 1] = __uint_as_float(word(u, i) & 0xffff0000u); }
            lo = hi = f[0];
#pragma unroll
            for (int i = 0; i < 8; ++i) { lo = fminf(lo, f[i]); hi = fmaxf(hi, f[i]); bad |= !(fabsf(f[i]) < INFINITY); }
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) {
                lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
                hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
                bad |= __shfl_xor_sync(0xffffffffu, (int)bad, o) != 0;
            }
            const uint32_t par = group4(lo, hi, bad);
            uint32_t w = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) w |= code4(f[i], par) << (4 * i);
            if (lane < D / 4) {
                unsigned char* codes = blk + (values ? L.off_v : L.off_k) + (size_t)slot * (D / 2);
                if (values) {
                    reinterpret_cast<uint16_t*>(codes)[2 * tt * GR + grp] = (uint16_t)w;
                    reinterpret_cast<uint16_t*>(codes)[(2 * tt + 1) * GR + grp] = (uint16_t)(w >> 16);
                } else {
                    reinterpret_cast<uint32_t*>(codes)[tt * GR + grp] = w;
                }
                if (tt == 0) reinterpret_cast<uint32_t*>(blk + (values ? L.off_vp : L.off_kp))[(size_t)slot * GR + grp] = par;
            }
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

// How many warps share a head: all warps of the launch are resident at once where that is possible, as in decode_mma.cu.  Under accumulated
// attention a block's logits have to fit beside those of the SM's other blocks.
template <bool FOUR, bool ACCUM>
int launch_rows_mma(const Params& p, const RowsLayout& L, bool swz, const RowsRule& rule, void* cache, const void* q1, const void* k1, const void* v1,
                    void* o1, float* lse1, cudaStream_t st)
{
    int n_sm = 0;
    if (int e = device_sm_count(&n_sm)) return e;
    const int BH = p.B * p.H, rows = p.W + p.R, wps = warps_per_sm(p.d, FOUR), warps = wps * n_sm, most_w = max_warps(p.d);
    constexpr int UR = Stage<64, FOUR>::UR;                    // rows that a warp takes at a time
    const int kept = ACCUM ? (p.G < MQ ? p.G : MQ) + (p.G > MQ ? 1 : 0) : 0;   // floats per row in shared memory
    auto most = [&](int all) { return ((rows + UR - 1) / UR + all - 1) / all * UR; };   // rows of a warp at most, `all` of which share the head
    auto smem = [&](int nw, int split) { return (size_t)nw * most(nw * split) * kept * 4; };   // of logits
    int nw = 1, nsplit = 1;
    for (int c : {2, 4, 8})
        if (c <= most_w && ((BH <= n_sm * (wps / c) && rows / c >= 16) || smem(c / 2, 1) * (wps / (c / 2)) > 96 * 1024)) nw = c;
    if (nw == most_w)
        while (nsplit < MAX_SPLIT && ((BH * nw * nsplit * 2 <= warps && rows / (nw * nsplit * 2) >= 8) || smem(nw, nsplit) > 64 * 1024)) nsplit *= 2;
    auto go = [&](auto d, auto w, auto s) {
        constexpr int D = decltype(d)::value, NW = decltype(w)::value;
        if constexpr (NW <= max_warps(D)) {
            auto kern = decode_rows_mma_kernel<D, NW, decltype(s)::value, FOUR, ACCUM>;
            static PerDeviceOnce once;
            if (int e = once.run([&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024); })) return e;
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(BH * nsplit); cfg.blockDim = dim3(NW * 32); cfg.stream = st; cfg.dynamicSmemBytes = smem(nw, nsplit) + NW * Stage<D, FOUR>::STAGES * Stage<D, FOUR>::BYTES;
            cudaLaunchAttribute attr[2];
            attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
            attr[0].val.programmaticStreamSerializationAllowed = 1;
            attr[1].id = cudaLaunchAttributeClusterDimension;
            attr[1].val.clusterDim.x = nsplit; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
            cfg.attrs = attr; cfg.numAttrs = nsplit > 1 ? 2 : 1;
            return cuda_status(cudaLaunchKernelEx(&cfg, kern, (unsigned char*)cache, L, (const __nv_bfloat16*)q1, (const __nv_bfloat16*)k1,
                                                  (const __nv_bfloat16*)v1, (__nv_bfloat16*)o1, lse1, rule, p.H, p.W, p.R, p.sink, p.scale, p.G,
                                                  most(nw * nsplit)));
        }
        return (int)LTE_ERR_UNSUPPORTED;
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
