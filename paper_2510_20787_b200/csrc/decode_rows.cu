// Decode step (lte_attn_decode_accum, lte_attn_decode4, lte_attn_decode4_accum) on the fp32 ALUs.
//
// A block of 256 threads a head, or a cluster of up to eight that share its rows where heads are few.  Pool decision, logits of the block's
// rows into shared memory, softmax over them, weighted values; the blocks then meet through distributed shared memory, and each adds
// the weights of its rows to their scores: the weights need the sum over all rows, so the logits stay until then.
#include <cfloat>
#include <cooperative_groups.h>

#include <type_traits>

#include "decode_rows.cuh"

namespace lte {
namespace cg = cooperative_groups;
namespace {

constexpr int DT = 256;
constexpr int QP = 4;                                          // query heads per pass
constexpr int MAX_SPLIT = 8;

// How a lane sees a row: LPR lanes of E channels each.
template <typename T, int D, bool FOUR> struct Held {
    static constexpr int E = FOUR ? 8 : 16 / (int)sizeof(T), LPR = D / E, GROUPS = D / kGroup4;
    static __device__ __forceinline__ int channel(bool values, int seg, int e)
    {
        return !FOUR ? seg * E + e : values ? value4_channel(seg, e, GROUPS) : key4_channel(seg, e, GROUPS);
    }
    static __device__ __forceinline__ void load(const unsigned char* rows, const unsigned char* par, const CacheLayout& C, bool values, int row, int seg,
                                                float (&f)[E])
    {
        if constexpr (FOUR) {
            const uint32_t w = reinterpret_cast<const uint32_t*>(rows)[(size_t)row * LPR + seg];
            const uint32_t* p = reinterpret_cast<const uint32_t*>(par) + (size_t)row * GROUPS;
#pragma unroll
            for (int e = 0; e < E; ++e) f[e] = value4((w >> (4 * e)) & 15u, p[channel(values, seg, e) / kGroup4]);
        } else {
            const int at = sizeof(T) == 2 ? cache_chunk_pos(C, row, seg) : seg;
            const uint4 u = reinterpret_cast<const uint4*>(rows)[(size_t)row * LPR + at];
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(T) == 2) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
                else f[i] = __uint_as_float(w[i]);
            }
        }
    }
};

template <typename T, int D, bool FOUR, bool ACCUM>
__global__ void __launch_bounds__(DT) decode_rows_kernel(unsigned char* __restrict__ cache, RowsLayout L, CacheLayout C, const T* __restrict__ q1,
                                                         const T* __restrict__ k1, const T* __restrict__ v1, T* __restrict__ o1,
                                                         float* __restrict__ lse1, RowsRule rule, int H, int W, int R, int sink, float scale, int G,
                                                         int most)                       // most: rows a block may have
{
    using Row = Held<T, D, FOUR>;
    constexpr int E = Row::E, LPR = Row::LPR, RPP = DT / LPR, NW = DT / 32;
    extern __shared__ __align__(16) float s_log[];             // [most][nq] logits, then weights; behind them [most] sums over passes
    __shared__ float s_q[QP][D], s_kn[D], s_vn[D];
    __shared__ float s_red[NW][QP][D], s_o[QP][D], s_m[QP], s_l[QP], s_new[QP], s_part[NW][QP];
    __shared__ float s_tap[kMaxTaps];
    __shared__ uint32_t s_wkey[NW];
    __shared__ int s_wpos[NW], s_wslot[NW];
    cg::cluster_group cluster = cg::this_cluster();
    const int nsplit = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int bh = blockIdx.x / nsplit, h = bh % H;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, seg = tid % LPR, rsub = tid / LPR;
    unsigned char* blk = cache + L.header + (size_t)bh * L.stride;
    float* zc = reinterpret_cast<float*>(blk + L.off_z);
    int32_t* pidx = reinterpret_cast<int32_t*>(blk + L.off_pidx);
    int32_t* meta = reinterpret_cast<int32_t*>(blk + L.off_meta);
    pdl_launch_dependents();
    pdl_wait();

    const int n = max(meta[0], 0), cnt_old = min(max(meta[1], 0), R), slot = n % W, p = n - W;
    for (int c = tid; c < D; c += DT) { s_kn[c] = to_f<T>(k1[(size_t)bh * D + c]); s_vn[c] = to_f<T>(v1[(size_t)bh * D + c]); }

    // ---- what happens to the token leaving the window (every block of the cluster finds the same) ------------------
    const float zp = p >= 0 ? zc[slot] : 0.f;
    int dst = -1, cnt_new = cnt_old;
    if (p >= 0 && R > 0 && (ACCUM || p < sink || zp > rule.zthr)) {
        if (cnt_old < R) { dst = cnt_old; cnt_new = cnt_old + 1; }
        else if (p >= sink) {
            Worst w;
            for (int m = tid; m < cnt_old; m += DT) w.offer(zc[W + m], pidx[m], m, sink);
            w.over_warp();
            if (lane == 0) { s_wkey[wid] = w.key; s_wpos[wid] = w.pos; s_wslot[wid] = w.slot; }
            __syncthreads();
            w.key = lane < NW ? s_wkey[lane] : 0xffffffffu; w.pos = lane < NW ? s_wpos[lane] : -1; w.slot = lane < NW ? s_wslot[lane] : -1;
            w.over_warp();
            if (w.slot >= 0 && order_key(zp + 0.f) > w.key) dst = w.slot;
        }
    }
    const int masked_ring = p >= 0 && dst < 0 ? slot : -1;     // the popped row counts iff the pool takes it ...
    const int masked_pool = dst >= 0 && dst < cnt_old ? W + dst : -1;   // ... and then the entry it replaces does not

    // the block's rows: [first, first + mine) of the ring's and the pool's rows in use
    const int n_ring = min(n, W), total = n_ring + cnt_old, per = (total + nsplit - 1) / nsplit;
    const int first = min(rank * per, total), mine = min(per, total - first);
    auto row_of = [&](int u) { const int i = first + u; return i < n_ring ? i : W + i - n_ring; };
    auto seen = [&](int row) { return row != masked_ring && row != masked_pool; };
    float* s_sum = s_log + (size_t)most * min(G, QP);

    for (int g0 = 0; g0 < G; g0 += QP) {
        const int nq = min(QP, G - g0);
        __syncthreads();
        for (int c = tid; c < QP * D; c += DT) s_q[c / D][c % D] = c / D < nq ? to_f<T>(q1[((size_t)bh * G + g0) * D + c]) : 0.f;
        __syncthreads();
        // ---- logits -----------------------------------------------------------------------------------------------
        {
            float qf[QP][E];
#pragma unroll
            for (int u = 0; u < QP; ++u)
#pragma unroll
                for (int e = 0; e < E; ++e) qf[u][e] = s_q[u][Row::channel(false, seg, e)];
            for (int r0 = 0; r0 < mine; r0 += RPP) {
                const int u = r0 + rsub, row = row_of(min(u, mine - 1));
                float kf[E], x[QP];
                Row::load(blk + L.off_k, blk + L.off_kp, C, false, row, seg, kf);
#pragma unroll
                for (int g = 0; g < QP; ++g) {
                    x[g] = 0.f;
#pragma unroll
                    for (int e = 0; e < E; ++e) x[g] = fmaf(qf[g][e], kf[e], x[g]);
#pragma unroll
                    for (int o = LPR / 2; o > 0; o >>= 1) x[g] += __shfl_xor_sync(0xffffffffu, x[g], o);
                }
                if (seg == 0 && u < mine)
                    for (int g = 0; g < nq; ++g) s_log[u * nq + g] = seen(row) ? x[g] * scale : -INFINITY;
            }
        }
        if (wid < nq) {                                        // the incoming token's
            float a = 0.f;
            for (int c = lane; c < D; c += 32) a = fmaf(s_q[wid][c], s_kn[c], a);
            a = warp_sum(a) * scale;
            if (lane == 0) s_new[wid] = a;
        }
        __syncthreads();
        // ---- softmax over the block's rows (the first block has the incoming token besides) ---------------------------
        float mx[QP], sum[QP];
#pragma unroll
        for (int g = 0; g < QP; ++g) {
            mx[g] = g < nq && rank == 0 ? s_new[g] : -INFINITY;
            if (g < nq) for (int u = tid; u < mine; u += DT) mx[g] = fmaxf(mx[g], s_log[u * nq + g]);
            mx[g] = warp_max(mx[g]);
            if (lane == 0) s_part[wid][g] = mx[g];
        }
        __syncthreads();
#pragma unroll
        for (int g = 0; g < QP; ++g) {
            for (int w = 0; w < NW; ++w) mx[g] = fmaxf(mx[g], s_part[w][g]);
            mx[g] = fmaxf(mx[g], -FLT_MAX);                    // no row, or none with a weight: finite (no inf - inf)
        }
        __syncthreads();
#pragma unroll
        for (int g = 0; g < QP; ++g) {
            sum[g] = 0.f;
            if (g < nq)
                for (int u = tid; u < mine; u += DT) {
                    const float w = __expf(s_log[u * nq + g] - mx[g]);
                    s_log[u * nq + g] = w;
                    sum[g] += w;
                }
            sum[g] = warp_sum(sum[g]);
            if (lane == 0) s_part[wid][g] = sum[g];
        }
        __syncthreads();
        // ---- weighted values ----------------------------------------------------------------------------------------
        {
            float acc[QP][E];
#pragma unroll
            for (int g = 0; g < QP; ++g)
#pragma unroll
                for (int e = 0; e < E; ++e) acc[g][e] = 0.f;
            for (int u = rsub; u < mine; u += RPP) {
                const int row = row_of(u);
                if (!seen(row)) continue;
                float vf[E];
                Row::load(blk + L.off_v, blk + L.off_vp, C, true, row, seg, vf);
#pragma unroll
                for (int g = 0; g < QP; ++g) {
                    const float w = g < nq ? s_log[u * nq + g] : 0.f;
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[g][e] = g < nq ? fmaf(w, vf[e], acc[g][e]) : 0.f;
                }
            }
#pragma unroll
            for (int o = 16; o >= LPR; o >>= 1)
#pragma unroll
                for (int g = 0; g < QP; ++g)
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[g][e] += __shfl_xor_sync(0xffffffffu, acc[g][e], o);
            if (lane < LPR)
#pragma unroll
                for (int g = 0; g < QP; ++g)
#pragma unroll
                    for (int e = 0; e < E; ++e) s_red[wid][g][Row::channel(true, seg, e)] = acc[g][e];
        }
        __syncthreads();
        for (int e = tid; e < nq * D; e += DT) {
            const int g = e / D, c = e % D;
            const float w = rank == 0 ? __expf(s_new[g] - mx[g]) : 0.f;
            float l = w, o = rank == 0 ? w * s_vn[c] : 0.f;
#pragma unroll
            for (int w2 = 0; w2 < NW; ++w2) { l += s_part[w2][g]; o += s_red[w2][g][c]; }
            s_o[g][c] = o;
            if (c == 0) { s_m[g] = mx[g]; s_l[g] = l; }
        }
        // ---- the cluster's blocks meet -----------------------------------------------------------------------------
        cluster.sync();
        float top[QP], tot[QP];
#pragma unroll
        for (int g = 0; g < QP; ++g) {
            top[g] = -FLT_MAX; tot[g] = 0.f;
            if (g < nq) {
                for (int r = 0; r < nsplit; ++r) top[g] = fmaxf(top[g], *cluster.map_shared_rank(&s_m[g], r));
                for (int r = 0; r < nsplit; ++r) tot[g] += __expf(*cluster.map_shared_rank(&s_m[g], r) - top[g]) * *cluster.map_shared_rank(&s_l[g], r);
            }
        }
        for (int e = rank * DT + tid; e < nq * D; e += nsplit * DT) {
            const int g = e / D, c = e % D;
            float m = 0.f, l = 1.f;
#pragma unroll
            for (int g2 = 0; g2 < QP; ++g2) if (g2 == g) { m = top[g2]; l = tot[g2]; }
            float o = 0.f;
            for (int r = 0; r < nsplit; ++r) o += __expf(*cluster.map_shared_rank(&s_m[g], r) - m) * *cluster.map_shared_rank(&s_o[g][c], r);
            o1[((size_t)bh * G + g0) * D + e] = from_f<T>(o / l);
            if (c == 0) lse1[(size_t)bh * G + g0 + g] = m + logf(l);
        }
        if constexpr (ACCUM) {
            // ---- weights of the block's rows into their scores.  Every block has read the old ones it needs for the decision.
            float f[QP];
            const bool last = g0 + QP >= G;
#pragma unroll
            for (int g = 0; g < QP; ++g) f[g] = g < nq ? __expf(mx[g] - top[g]) / tot[g] : 0.f;
            for (int u = tid; u < mine; u += DT) {
                float a = 0.f;
                for (int g = 0; g < nq; ++g) a += f[g] * s_log[u * nq + g];
                if (G > QP) { a += g0 > 0 ? s_sum[u] : 0.f; s_sum[u] = a; }
                const int row = row_of(u);
                if (last && seen(row)) zc[row == slot && p >= 0 ? W + dst : row] = rule.decay > 0.f ? fmaf(rule.decay, zc[row], a) : a;
            }
            if (rank == 0 && tid == 0) {
                float a = g0 > 0 ? s_tap[0] : 0.f;
                for (int g = 0; g < nq; ++g) a += __expf(s_new[g] - top[g]) / tot[g];
                s_tap[0] = a;                                  // (of the incoming token, over the passes)
            }
        }
        cluster.sync();                                        // shared memory has been read, and every row
    }
    if (rank != 0) return;

    // ---- learned rule: logit of the newest token whose receptive field is complete ------------------------------------
    const int jsc = ACCUM ? -1 : n - rule.K / 2;
    if (jsc >= 0) {
        for (int t = wid; t < rule.K; t += NW) {
            const int pos = jsc + t - rule.K / 2;
            const float* wt = rule.w + ((size_t)h * rule.K + t) * 2 * D;
            float a = 0.f;
            if (pos == n) {
                for (int c = lane; c < D; c += 32) a += wt[c] * s_kn[c] + wt[D + c] * s_vn[c];
            } else if (pos >= 0) {
                for (int s = lane; s < LPR; s += 32) {
                    float kf[E], vf[E];
                    Row::load(blk + L.off_k, blk + L.off_kp, C, false, pos % W, s, kf);
                    Row::load(blk + L.off_v, blk + L.off_vp, C, true, pos % W, s, vf);
#pragma unroll
                    for (int e = 0; e < E; ++e) a += wt[Row::channel(false, s, e)] * kf[e] + wt[D + Row::channel(true, s, e)] * vf[e];
                }
            }
            a = warp_sum(a);
            if (lane == 0) s_tap[t] = a;
        }
    }

    // ---- write-back ---------------------------------------------------------------------------------------------------
    __syncthreads();
    constexpr int WORDS = FOUR ? D / 8 : D * (int)sizeof(T) / 4, GROUPS = FOUR ? D / kGroup4 : 0;   // 4-byte words of a row, of its parameters
    if (dst >= 0)
        for (int e = tid; e < 2 * (WORDS + GROUPS); e += DT) {
            const bool values = e >= WORDS + GROUPS, par = e % (WORDS + GROUPS) >= WORDS;
            const int w = e % (WORDS + GROUPS) - (par ? WORDS : 0), len = par ? GROUPS : WORDS;
            uint32_t* a = reinterpret_cast<uint32_t*>(blk + (par ? (values ? L.off_vp : L.off_kp) : (values ? L.off_v : L.off_k)));
            auto at = [&](int row) { return (size_t)row * len + (!FOUR && sizeof(T) == 2 ? (cache_chunk_pos(C, row, w >> 2) << 2) | (w & 3) : w); };
            a[at(W + dst)] = a[at(slot)];
        }
    __syncthreads();
    if constexpr (FOUR) {
        for (int e = wid; e < 2 * GROUPS; e += NW) {
            const bool values = e >= GROUPS;
            const int g = e % GROUPS;
            store_group4((values ? s_vn : s_kn)[g * kGroup4 + lane], lane, values, g, GROUPS, blk + (values ? L.off_v : L.off_k) + (size_t)slot * (D / 2),
                         reinterpret_cast<uint32_t*>(blk + (values ? L.off_vp : L.off_kp)) + (size_t)slot * GROUPS);
        }
    } else {
        for (int e = tid; e < 2 * D; e += DT) {
            const bool values = e >= D;
            const int c = e % D, at = sizeof(T) == 2 ? (cache_chunk_pos(C, slot, c >> 3) << 3) | (c & 7) : c;
            reinterpret_cast<T*>(blk + (values ? L.off_v : L.off_k))[(size_t)slot * D + at] = (values ? v1 : k1)[(size_t)bh * D + c];
        }
    }
    if (tid == 0) {
        if (dst >= 0) pidx[dst] = p;
        if (ACCUM) {
            zc[slot] = s_tap[0];
        } else {
            if (dst >= 0) zc[W + dst] = zp;
            float znew = rule.bias ? rule.bias[h] : 0.f;
            if (jsc >= 0) for (int t = 0; t < rule.K; ++t) znew += s_tap[t];
            zc[slot] = -INFINITY;                              // the incoming token is not scored yet ...
            if (jsc >= 0) zc[jsc % W] = znew;                  // ... unless K == 1 (then jsc == n)
        }
        meta[0] = n + 1;
        meta[1] = cnt_new;
    }
}

}  // namespace

int launch_decode_rows(const Params& p, bool four, bool accum, float decay, void* cache, const void* q1, const void* k1, const void* v1, void* o1,
                       float* lse1, cudaStream_t st)
{
    const RowsRule rule = {decay, p.zthr, p.K, p.w, p.bias};
    if (p.dtype == LTE_BF16)
        return four ? launch_decode_rows4_bf16(p, accum, rule, cache, q1, k1, v1, o1, lse1, st) : launch_decode_rows_bf16(p, rule, cache, q1, k1, v1, o1, lse1, st);
    const CacheLayout C = cache_layout(p.d, p.W, p.R, p.dtype);
    const RowsLayout L = four ? rows_layout(cache4_layout(p.d, p.W, p.R)) : rows_layout(C);
    int n_sm = 0;
    if (int e = device_sm_count(&n_sm)) return e;
    const int BH = p.B * p.H, rows = p.W + p.R, nq = p.G < QP ? p.G : QP;
    auto smem = [&](int split) { return (size_t)((rows + split - 1) / split) * (nq + (p.G > QP ? 1 : 0)) * 4; };
    int nsplit = 1;
    while (nsplit < MAX_SPLIT && (smem(nsplit) > 48 * 1024 || (BH * nsplit * 2 <= 2 * n_sm && rows / (nsplit * 2) >= 32))) nsplit *= 2;
    auto go = [&](auto t, auto d, auto f4, auto acc) {
        using T = decltype(t);
        constexpr int D = decltype(d)::value;
        auto kern = decode_rows_kernel<T, D, decltype(f4)::value, decltype(acc)::value>;
        static PerDeviceOnce once;
        if (int e = once.run([&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 128 * 1024); })) return e;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(BH * nsplit); cfg.blockDim = dim3(DT); cfg.stream = st; cfg.dynamicSmemBytes = smem(nsplit);
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = nsplit; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
        cfg.attrs = attr; cfg.numAttrs = nsplit > 1 ? 2 : 1;
        return cuda_status(cudaLaunchKernelEx(&cfg, kern, (unsigned char*)cache, L, C, (const T*)q1, (const T*)k1, (const T*)v1, (T*)o1, lse1, rule, p.H,
                                              p.W, p.R, p.sink, p.scale, p.G, (rows + nsplit - 1) / nsplit));
    };
    auto kinds = [&](auto t, auto d) {
        if (!four) return go(t, d, std::false_type(), std::true_type());   // (the learned rule over ordinary caches is lte_attn_decode)
        return accum ? go(t, d, std::true_type(), std::true_type()) : go(t, d, std::true_type(), std::false_type());
    };
    auto dims = [&](auto t) {
        switch (p.d) {
            case 32: return kinds(t, std::integral_constant<int, 32>());
            case 64: return kinds(t, std::integral_constant<int, 64>());
            case 128: return kinds(t, std::integral_constant<int, 128>());
        }
        return (int)LTE_ERR_UNSUPPORTED;
    };
    return dims(0.f);
}

}  // namespace lte
