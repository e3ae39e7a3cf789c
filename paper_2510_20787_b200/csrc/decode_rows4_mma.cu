// Decode step under the learned rule over caches in 4 bits, bf16 calls (decode_rows_mma.cuh).
#include "decode_rows_mma.cuh"

namespace lte {

int launch_decode_rows4_bf16(const Params& p, const RowsRule& rule, void* cache, const void* q1, const void* k1, const void* v1, void* o1, float* lse1,
                             cudaStream_t st)
{
    return launch_rows_mma<true, false>(p, rows_layout(cache4_layout(p.d, p.W, p.R)), false, rule, cache, q1, k1, v1, o1, lse1, st);
}

}  // namespace lte
