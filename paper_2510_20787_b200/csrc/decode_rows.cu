// Decode step (lte_attn_decode_accum, lte_attn_decode4, lte_attn_decode4_accum) for fp32 calls, on the fp32 ALUs.
//
// A block of 256 threads a head, or a cluster of up to eight that share its rows where heads are few.  Pool decision, logits of the block's
// rows into shared memory, softmax over them, weighted values; the blocks then meet through distributed shared memory, and each adds
// the weights of its rows to their scores: the weights need the sum over all rows, so the logits stay until then.
// A row is shared by the LPR lanes that hold its 16-byte pieces (4 bits: its 4-byte words).  What bounds it is the latency of its loads and the sums over
// those lanes: a thread has BATCH rows in flight, and their partial sums for all query heads are added up together, half of them handed to
// the other half of the lanes in every round (15 shuffles in the place of 64 for four rows, four query heads and 16 lanes).
// Measured (B200, a step in a CUDA graph; before: a row at a time): 64 heads x 1,280 rows, four query heads each, d = 64 23.0 us (43 MB: 6.6 at 6.56 TB/s),
// before 39.5; 256 x 256 13.5 us (5.3), before 27.8; 2 heads x 24 rows, d = 32 5.7 us, before 6.3.  In 4 bits, accumulated | learned: 64 x 1,280 21.0 | 20.5 us
// (1.1: the same latencies, and eight conversions and multiply-adds a code word), 256 x 256 9.9 | 10.4 (0.9).
#include <cfloat>
#include <cooperative_groups.h>

#include <type_traits>

#include "decode_rows.cuh"

namespace lte {
namespace cg = cooperative_groups;
namespace {

constexpr int DT = 256;
constexpr int BATCH = 4;                                       // rows a thread has in flight
constexpr int MAX_SPLIT = 8;

// How a lane sees a row: LPR lanes of E channels each.
template <int D, bool FOUR> struct Held {
    static constexpr int E = FOUR ? 8 : 4, LPR = D / E, GROUPS = D / kGroup4;
    struct Raw { uint4 u; };                                   // four channels, or a word of codes and its two parameters
    static __device__ __forceinline__ int channel(bool values, int seg, int e)
    {
        return !FOUR ? seg * E + e : values ? value4_channel(seg, e, GROUPS) : key4_channel(seg, e, GROUPS);
    }
    static __device__ __forceinline__ Raw load(const unsigned char* rows, const unsigned char* par, bool values, int row, int seg)
    {
        Raw r;
        if constexpr (FOUR) {
            r.u.x = reinterpret_cast<const uint32_t*>(rows)[(size_t)row * LPR + seg];
            const uint32_t* p = reinterpret_cast<const uint32_t*>(par) + (size_t)row * GROUPS;
            r.u.y = p[channel(values, seg, 0) / kGroup4]; r.u.z = p[channel(values, seg, 4) / kGroup4];
        } else {
            r.u = reinterpret_cast<const uint4*>(rows)[(size_t)row * LPR + seg];
        }
        return r;
    }
    static __device__ __forceinline__ void unpack(const Raw& r, float (&f)[E])
    {
        if constexpr (FOUR) {
#pragma unroll
            for (int e = 0; e < E; ++e) f[e] = value4((r.u.x >> (4 * e)) & 15u, e < 4 ? r.u.y : r.u.z);
        } else {
            f[0] = __uint_as_float(r.u.x); f[1] = __uint_as_float(r.u.y); f[2] = __uint_as_float(r.u.z); f[3] = __uint_as_float(r.u.w);
        }
    }
};

// V values per lane, summed over the L lanes that share `seg` (0 .. L - 1): afterwards lane seg has, in x[0 .. max(V / L, 1) - 1], the sums of the values
// from index (seg's bits, the lowest first, as halves of V) on; `first` is that index.
template <int V, int L> __device__ __forceinline__ int sum_lanes(float (&x)[V], int seg)
{
    int first = 0, n = V;
#pragma unroll
    for (int o = 1; o < L; o <<= 1) {
        if (n > 1) {
            n >>= 1;
            const bool up = seg & o;
#pragma unroll
            for (int i = 0; i < V / 2; ++i)
                if (i < n) {
                    const float give = up ? x[i] : x[i + n], keep = up ? x[i + n] : x[i];
                    x[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
                }
            first += up ? n : 0;
        } else {
            x[0] += __shfl_xor_sync(0xffffffffu, x[0], o);
        }
    }
    return first;
}

template <int D, int QP, bool FOUR, bool ACCUM>                // QP: query heads per pass
__global__ void __launch_bounds__(DT) decode_rows_kernel(unsigned char* __restrict__ cache, RowsLayout L, const float* __restrict__ q1,
                                                         const float* __restrict__ k1, const float* __restrict__ v1, float* __restrict__ o1,
                                                         float* __restrict__ lse1, RowsRule rule, int H, int W, int R, int sink, float scale, int G,
                                                         int most, int* __restrict__ status)   // most: rows a block may have
{
    using Row = Held<D, FOUR>;
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

    const bool wrong = wrong_cache<FOUR, ACCUM>(cache_holds(cache));
    const int n = max(meta[0], 0), cnt_old = min(max(meta[1], 0), R), slot = n % W, p = n - W;
    for (int c = tid; c < D; c += DT) { s_kn[c] = k1[(size_t)bh * D + c]; s_vn[c] = v1[(size_t)bh * D + c]; }

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
            if (w.slot >= 0 && Worst::rank(zp) > w.key) dst = w.slot;
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
        for (int c = tid; c < QP * D; c += DT) s_q[c / D][c % D] = c / D < nq ? q1[((size_t)bh * G + g0) * D + c] : 0.f;
        __syncthreads();
        // ---- logits -----------------------------------------------------------------------------------------------
        {
            float qf[QP][E];
#pragma unroll
            for (int u = 0; u < QP; ++u)
#pragma unroll
                for (int e = 0; e < E; ++e) qf[u][e] = s_q[u][Row::channel(false, seg, e)];
            // value r * QP + g of a lane: row r of the batch, query head g
            typename Row::Raw raw[BATCH];
            auto ask = [&](int r0) {
#pragma unroll
                for (int r = 0; r < BATCH; ++r) raw[r] = Row::load(blk + L.off_k, blk + L.off_kp, false, row_of(min(r0 + r * RPP + rsub, mine - 1)), seg);
            };
            if (mine > 0) ask(0);
            for (int r0 = 0; r0 < mine; r0 += BATCH * RPP) {
                float x[BATCH * QP];
#pragma unroll
                for (int r = 0; r < BATCH; ++r) {
                    float kf[E];
                    Row::unpack(raw[r], kf);
#pragma unroll
                    for (int g = 0; g < QP; ++g) {
                        x[r * QP + g] = 0.f;
#pragma unroll
                        for (int e = 0; e < E; ++e) x[r * QP + g] = fmaf(qf[g][e], kf[e], x[r * QP + g]);
                    }
                }
                if (r0 + BATCH * RPP < mine) ask(r0 + BATCH * RPP);
                const int at = sum_lanes<BATCH * QP, LPR>(x, seg);
                constexpr int LEFT = BATCH * QP > LPR ? BATCH * QP / LPR : 1;   // sums a lane is left with (some lanes have the same one)
                if (BATCH * QP >= LPR || seg < BATCH * QP)
#pragma unroll
                    for (int i = 0; i < LEFT; ++i) {
                        const int u = r0 + (at + i) / QP * RPP + rsub, g = (at + i) % QP;
                        if (u < mine && g < nq) s_log[u * nq + g] = seen(row_of(u)) ? x[i] * scale : -INFINITY;
                    }
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
            typename Row::Raw raw[BATCH];
            auto ask = [&](int r0) {
#pragma unroll
                for (int r = 0; r < BATCH; ++r) raw[r] = Row::load(blk + L.off_v, blk + L.off_vp, true, row_of(min(r0 + r * RPP + rsub, mine - 1)), seg);
            };
            if (mine > 0) ask(0);
            for (int r0 = 0; r0 < mine; r0 += BATCH * RPP) {
                float vf[BATCH][E];
#pragma unroll
                for (int r = 0; r < BATCH; ++r) Row::unpack(raw[r], vf[r]);
                if (r0 + BATCH * RPP < mine) ask(r0 + BATCH * RPP);
#pragma unroll
                for (int r = 0; r < BATCH; ++r) {
                    const int u = r0 + r * RPP + rsub;
                    if (u >= mine || !seen(row_of(u))) continue;   // (zero times an infinite value is NaN)
#pragma unroll
                    for (int g = 0; g < QP; ++g)
                        if (g < nq) {
                            const float w = s_log[u * nq + g];
#pragma unroll
                            for (int e = 0; e < E; ++e) acc[g][e] = fmaf(w, vf[r][e], acc[g][e]);
                        }
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
        if (wrong) {                                           // (every block of the launch; nothing has been written yet)
            if (blockIdx.x == 0 && tid == 0) atomicExch(status, kWrongCache);
            return;
        }
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
            o1[((size_t)bh * G + g0) * D + e] = o / l;
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
                    Row::unpack(Row::load(blk + L.off_k, blk + L.off_kp, false, pos % W, s), kf);
                    Row::unpack(Row::load(blk + L.off_v, blk + L.off_vp, true, pos % W, s), vf);
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
    constexpr int WORDS = FOUR ? D / 8 : D, GROUPS = FOUR ? D / kGroup4 : 0;   // 4-byte words of a row, of its parameters
    if (dst >= 0)
        for (int e = tid; e < 2 * (WORDS + GROUPS); e += DT) {
            const bool values = e >= WORDS + GROUPS, par = e % (WORDS + GROUPS) >= WORDS;
            const int w = e % (WORDS + GROUPS) - (par ? WORDS : 0), len = par ? GROUPS : WORDS;
            uint32_t* a = reinterpret_cast<uint32_t*>(blk + (par ? (values ? L.off_vp : L.off_kp) : (values ? L.off_v : L.off_k)));
            a[(size_t)(W + dst) * len + w] = a[(size_t)slot * len + w];
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
            reinterpret_cast<float*>(blk + (values ? L.off_v : L.off_k))[(size_t)slot * D + e % D] = (values ? s_vn : s_kn)[e % D];
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
        return (!four ? launch_decode_rows_bf16 : accum ? launch_decode_rows4_accum_bf16 : launch_decode_rows4_bf16)(p, rule, cache, q1, k1, v1, o1, lse1, st);
    const RowsLayout L = four ? rows_layout(cache4_layout(p.d, p.W, p.R)) : rows_layout(cache_layout(p.d, p.W, p.R, p.dtype));
    int n_sm = 0, *status = nullptr;
    if (int e = device_sm_count(&n_sm)) return e;
    if (int e = cache_status_word(&status)) return e;
    const int BH = p.B * p.H, rows = p.W + p.R;
    auto go = [&](auto d, auto qp, auto f4, auto acc) {
        constexpr int D = decltype(d)::value, QP = decltype(qp)::value;
        const int nq = p.G < QP ? p.G : QP;
        auto smem = [&](int split) { return (size_t)((rows + split - 1) / split) * (nq + (p.G > QP ? 1 : 0)) * 4; };
        // two blocks an SM, each with 32 rows at least; more where a block's logits would take too much shared memory
        int nsplit = 1;
        while (nsplit < MAX_SPLIT && (smem(nsplit) > 48 * 1024 || (BH * nsplit * 2 <= 2 * n_sm && rows / (nsplit * 2) >= 32))) nsplit *= 2;
        auto kern = decode_rows_kernel<D, QP, decltype(f4)::value, decltype(acc)::value>;
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
        return cuda_status(cudaLaunchKernelEx(&cfg, kern, (unsigned char*)cache, L, (const float*)q1, (const float*)k1, (const float*)v1, (float*)o1, lse1,
                                              rule, p.H, p.W, p.R, p.sink, p.scale, p.G, (rows + nsplit - 1) / nsplit, status));
    };
    auto kinds = [&](auto d, auto qp) {
        if (!four) return go(d, qp, std::false_type(), std::true_type());   // (the learned rule over ordinary caches is lte_attn_decode)
        return accum ? go(d, qp, std::true_type(), std::true_type()) : go(d, qp, std::true_type(), std::false_type());
    };
    auto heads = [&](auto d) { return p.G == 1 ? kinds(d, std::integral_constant<int, 1>()) : kinds(d, std::integral_constant<int, 4>()); };
    switch (p.d) {
        case 32: return heads(std::integral_constant<int, 32>());
        case 64: return heads(std::integral_constant<int, 64>());
        case 128: return heads(std::integral_constant<int, 128>());
    }
    return LTE_ERR_UNSUPPORTED;
}

}  // namespace lte
