// What the decode steps of decode_rows.cu (fp32) and decode_rows_mma.cuh (bf16) share: eviction by accumulated attention over ordinary
// caches, and both eviction rules over caches in 4 bits.
#pragma once
#include "cache4.cuh"

namespace lte {

constexpr int kRowsMost = 32768;                               // W + R that the steps take (fp32: a head's logits stay in the shared memory of eight blocks)

// Where a head's parts stand, whichever way its rows are held.
struct RowsLayout {
    size_t off_k, off_v, off_kp, off_vp, off_z, off_pidx, off_meta, stride, header;
};
inline RowsLayout rows_layout(const CacheLayout& L) { return {L.off_k, L.off_v, 0, 0, L.off_z, L.off_pidx, L.off_meta, L.stride, L.header}; }
inline RowsLayout rows_layout(const Cache4Layout& L) { return {L.off_k, L.off_v, L.off_kp, L.off_vp, L.off_z, L.off_pidx, L.off_meta, L.stride, L.header}; }

// The rule's parameters.  accum: decay and no threshold; learned: the scorer of K taps, w [H, K, 2d], bias [H] or NULL.
struct RowsRule {
    float decay, zthr;
    int K;
    const float *w, *bias;
};

// A cache that a step cannot read: of the other width, or attention sums where it reads logits.  (A cache without a mark is what the caller says.)
template <bool FOUR, bool ACCUM> __device__ __forceinline__ bool wrong_cache(uint32_t holds)
{
    return !FOUR ? (holds & kCacheFour) != 0u : ACCUM ? holds == kCacheAccum : (holds & kCacheAccum) != 0u;
}

// The pool's worst entry: lowest score, the youngest among equals.  As a key whose minimum is wanted and the position to break ties.
struct Worst {
    uint32_t key = 0xffffffffu;
    int pos = -1, slot = -1;
    // -0 counts as 0, NaN of either sign as more than any number (what an addition makes of a NaN's sign is not defined)
    static __device__ __forceinline__ uint32_t rank(float z)
    {
        return (__float_as_uint(z) & 0x7fffffffu) > 0x7f800000u ? 0xffffffffu : order_key(z + 0.f);
    }
    __device__ __forceinline__ void offer(float z, int at, int m, int sink)
    {
        const uint32_t k = rank(z);
        if (at >= sink && (k < key || (k == key && at > pos))) { key = k; pos = at; slot = m; }
    }
    __device__ __forceinline__ void over_warp()                // every lane then has it
    {
        const uint32_t kmin = __reduce_min_sync(0xffffffffu, key);
        const int pmax = __reduce_max_sync(0xffffffffu, key == kmin ? pos : -1);
        const unsigned who = __ballot_sync(0xffffffffu, key == kmin && pos == pmax);
        slot = __shfl_sync(0xffffffffu, slot, __ffs(who) - 1);
        key = kmin; pos = pmax;
    }
};

int launch_decode_rows_bf16(const Params& p, const RowsRule& rule, void* cache, const void* q1, const void* k1, const void* v1, void* o1, float* lse1,
                            cudaStream_t st);
int launch_decode_rows4_bf16(const Params& p, const RowsRule& rule, void* cache, const void* q1, const void* k1, const void* v1, void* o1, float* lse1,
                             cudaStream_t st);
int launch_decode_rows4_accum_bf16(const Params& p, const RowsRule& rule, void* cache, const void* q1, const void* k1, const void* v1, void* o1,
                                   float* lse1, cudaStream_t st);
int launch_decode_rows(const Params& p, bool four, bool accum, float decay, void* cache, const void* q1, const void* k1, const void* v1, void* o1,
                       float* lse1, cudaStream_t st);

}  // namespace lte
