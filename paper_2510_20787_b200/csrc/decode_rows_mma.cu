// Decode step under eviction by accumulated attention over bf16 caches (decode_rows_mma.cuh).
#include "decode_rows_mma.cuh"

namespace lte {

int launch_decode_rows_bf16(const Params& p, const RowsRule& rule, void* cache, const void* q1, const void* k1, const void* v1, void* o1, float* lse1,
                            cudaStream_t st)
{
    const CacheLayout C = cache_layout(p.d, p.W, p.R, p.dtype);
    return launch_rows_mma<false, true>(p, rows_layout(C), C.swz != 0, rule, cache, q1, k1, v1, o1, lse1, st);
}

}  // namespace lte
