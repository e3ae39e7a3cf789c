// An ordinary decode cache into 4 bits, and back (see cache4.cuh for the rule and the order of the codes).
//
// Bound by memory and, for the rounding, nearly as much by instructions: a thread takes eight channels of the key and of the value of ROWS rows (16
// or 32 bytes each), four threads a group; they meet in two shuffles for its extremes.  Scores, positions and counters are copied by the same
// blocks.
// Measured (B200, 256 heads x 1,280 rows, d = 64, bf16; 84 MB and 27 MB, 17.4 us at 6.56 TB/s): pack 30.7 us, of which instructions take about 25 (150
// per eight channels; with a division per channel it took 70), unpack 22.7 us.  fp32 (30.1 us of bytes): pack 37.4, unpack 45.9 us.
#include <type_traits>

#include "cache4.cuh"

namespace lte {
namespace {

constexpr int PT = 256;
constexpr int PROWS = 64;                                      // rows per block

template <typename T> struct Piece8 { uint4 u[sizeof(T) / 2]; };                          // eight channels
template <typename T> __device__ __forceinline__ void unpack8(const Piece8<T>& p, float (&f)[8]);
template <> __device__ __forceinline__ void unpack8<__nv_bfloat16>(const Piece8<__nv_bfloat16>& p, float (&f)[8])
{
    const uint32_t w[4] = {p.u[0].x, p.u[0].y, p.u[0].z, p.u[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
template <> __device__ __forceinline__ void unpack8<float>(const Piece8<float>& p, float (&f)[8])
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        f[4 * i] = __uint_as_float(p.u[i].x); f[4 * i + 1] = __uint_as_float(p.u[i].y);
        f[4 * i + 2] = __uint_as_float(p.u[i].z); f[4 * i + 3] = __uint_as_float(p.u[i].w);
    }
}
__device__ __forceinline__ Piece8<__nv_bfloat16> pack8(const float (&f)[8], __nv_bfloat16)
{
    Piece8<__nv_bfloat16> p;
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    p.u[0] = make_uint4(w[0], w[1], w[2], w[3]);
    return p;
}
__device__ __forceinline__ Piece8<float> pack8(const float (&f)[8], float)
{
    Piece8<float> p;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        p.u[i] = make_uint4(__float_as_uint(f[4 * i]), __float_as_uint(f[4 * i + 1]), __float_as_uint(f[4 * i + 2]), __float_as_uint(f[4 * i + 3]));
    return p;
}

// where eight channels of a row of an ordinary cache stand (in pieces); only bf16 rows are ever swizzled
__device__ __forceinline__ size_t piece_at(const CacheLayout& L, int row, int piece, int pieces)
{
    return (size_t)row * pieces + (L.esz == 2 ? cache_chunk_pos(L, row, piece) : piece);
}

// scores, positions, counters and padding of a head
__device__ __forceinline__ void copy_tail(const unsigned char* from, size_t fz, size_t fp, size_t fm, unsigned char* to, size_t tz, size_t tp, size_t tm,
                                          size_t to_end, int rows, int R, int part, int parts)
{
    for (int e = part * PT + threadIdx.x; e < rows; e += parts * PT)
        reinterpret_cast<uint32_t*>(to + tz)[e] = reinterpret_cast<const uint32_t*>(from + fz)[e];
    for (int e = part * PT + threadIdx.x; e < R; e += parts * PT)
        reinterpret_cast<uint32_t*>(to + tp)[e] = reinterpret_cast<const uint32_t*>(from + fp)[e];
    if (part == 0)
        for (int e = threadIdx.x; e < (int)((to_end - tm) / 4); e += PT)
            reinterpret_cast<uint32_t*>(to + tm)[e] = e < 4 ? reinterpret_cast<const uint32_t*>(from + fm)[e] : 0u;
}

template <typename T, int D>
__global__ void __launch_bounds__(PT) cache4_pack_kernel(const unsigned char* __restrict__ cache, CacheLayout L, unsigned char* __restrict__ cache4,
                                                         Cache4Layout Q, int W, int R, int parts)
{
    constexpr int PIECES = D / 8, GROUPS = D / kGroup4;
    pdl_launch_dependents();
    pdl_wait();
    const int bh = blockIdx.x / parts, part = blockIdx.x - bh * parts, rows = W + R;
    const unsigned char* src = cache + L.header + (size_t)bh * L.stride;
    unsigned char* dst = cache4 + Q.header + (size_t)bh * Q.stride;
    // thread: piece tid % PIECES of rows r0 + tid / PIECES + u (PT / PIECES); rows past the last one repeat it and are not stored
    constexpr int STEP = PT / PIECES, ROWS = PROWS / STEP;
    const int r0 = part * PROWS + threadIdx.x / PIECES, piece = threadIdx.x % PIECES, group = piece / 4, t = piece % 4;
    Piece8<T> p[ROWS][2];
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
        const size_t at = piece_at(L, min(r0 + u * STEP, rows - 1), piece, PIECES);
        p[u][0] = reinterpret_cast<const Piece8<T>*>(src + L.off_k)[at];
        p[u][1] = reinterpret_cast<const Piece8<T>*>(src + L.off_v)[at];
    }
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
        const int row = r0 + u * STEP;
#pragma unroll
        for (int values = 0; values < 2; ++values) {
            float f[8];
            unpack8<T>(p[u][values], f);
            uint32_t par;
            if constexpr (sizeof(T) == 2) par = group4_of(p[u][values].u[0]);
            else par = group4_of(f);
            const uint32_t w = codes4<sizeof(T) == 2>(f, par);
            if (row < rows) {
                unsigned char* codes = dst + (values ? Q.off_v : Q.off_k) + (size_t)row * (D / 2);
                if (values) {
                    reinterpret_cast<uint16_t*>(codes)[2 * t * GROUPS + group] = (uint16_t)w;
                    reinterpret_cast<uint16_t*>(codes)[(2 * t + 1) * GROUPS + group] = (uint16_t)(w >> 16);
                } else {
                    reinterpret_cast<uint32_t*>(codes)[t * GROUPS + group] = w;
                }
                if (t == 0) reinterpret_cast<uint32_t*>(dst + (values ? Q.off_vp : Q.off_kp))[(size_t)row * GROUPS + group] = par;
            }
        }
    }
    copy_tail(src, L.off_z, L.off_pidx, L.off_meta, dst, Q.off_z, Q.off_pidx, Q.off_meta, Q.stride, rows, R, part, parts);
    if (part == 0 && threadIdx.x < 6) {                        // what lies between the parts: a cache's bytes are those of its contents
        const size_t len = threadIdx.x < 2 ? (size_t)rows * D / 2 : threadIdx.x < 4 ? (size_t)rows * D / 8 : 4 * (size_t)(threadIdx.x == 4 ? rows : R);
        const size_t off[7] = {Q.off_k, Q.off_v, Q.off_kp, Q.off_vp, Q.off_z, Q.off_pidx, Q.off_meta};
#pragma unroll
        for (int i = 0; i < 6; ++i)
            if (threadIdx.x == i)
                for (size_t e = off[i] + len; e < off[i + 1]; e += 4) *reinterpret_cast<uint32_t*>(dst + e) = 0u;
    }
    if (blockIdx.x == 0 && threadIdx.x < Q.header / 4)
        reinterpret_cast<uint32_t*>(cache4)[threadIdx.x] = threadIdx.x == 0 ? kCacheMark | kCacheFour | cache_holds(cache) : 0u;
}

template <typename T, int D>
__global__ void __launch_bounds__(PT) cache4_unpack_kernel(const unsigned char* __restrict__ cache4, Cache4Layout Q, unsigned char* __restrict__ cache,
                                                           CacheLayout L, int W, int R, int parts, int* status)
{
    constexpr int PIECES = D / 8, GROUPS = D / kGroup4;
    pdl_launch_dependents();
    pdl_wait();
    const int bh = blockIdx.x / parts, part = blockIdx.x - bh * parts, rows = W + R;
    const unsigned char* src = cache4 + Q.header + (size_t)bh * Q.stride;
    unsigned char* dst = cache + L.header + (size_t)bh * L.stride;
    constexpr int STEP = PT / PIECES, ROWS = PROWS / STEP;
    const int r0 = part * PROWS + threadIdx.x / PIECES, piece = threadIdx.x % PIECES, group = piece / 4, t = piece % 4;
    uint32_t w[ROWS][2], par[ROWS][2];
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
        const int row = min(r0 + u * STEP, rows - 1);
        w[u][0] = reinterpret_cast<const uint32_t*>(src + Q.off_k + (size_t)row * (D / 2))[t * GROUPS + group];
        const uint16_t* v = reinterpret_cast<const uint16_t*>(src + Q.off_v + (size_t)row * (D / 2)) + 2 * t * GROUPS + group;
        w[u][1] = v[0] | (uint32_t)v[GROUPS] << 16;
        par[u][0] = reinterpret_cast<const uint32_t*>(src + Q.off_kp)[(size_t)row * GROUPS + group];
        par[u][1] = reinterpret_cast<const uint32_t*>(src + Q.off_vp)[(size_t)row * GROUPS + group];
    }
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
        const int row = r0 + u * STEP;
#pragma unroll
        for (int values = 0; values < 2; ++values) {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = row < rows ? value4((w[u][values] >> (4 * i)) & 15u, par[u][values]) : 0.f;   // (behind the last row: zero)
            if (row < L.rows_alloc)
                reinterpret_cast<Piece8<T>*>(dst + (values ? L.off_v : L.off_k))[piece_at(L, row, piece, PIECES)] = pack8(f, T());
        }
    }
    copy_tail(src, Q.off_z, Q.off_pidx, Q.off_meta, dst, L.off_z, L.off_pidx, L.off_meta, L.stride, rows, R, part, parts);
    const uint32_t holds = blockIdx.x == 0 ? cache_holds(cache4) : 0u;
    if (blockIdx.x == 0 && threadIdx.x == 0 && holds == kCacheAccum) atomicExch(status, kWrongCache);   // an ordinary cache
    if (blockIdx.x == 0 && threadIdx.x < L.header / 4)
        reinterpret_cast<uint32_t*>(cache)[threadIdx.x] = threadIdx.x == 0 && (holds & kCacheAccum) ? kCacheMark | kCacheAccum : 0u;
}

template <typename F> int by_type(const Params& p, F&& f)      // f(element, head dimension)
{
    auto dims = [&](auto t) {
        switch (p.d) {
            case 32: return f(t, std::integral_constant<int, 32>());
            case 64: return f(t, std::integral_constant<int, 64>());
            case 128: return f(t, std::integral_constant<int, 128>());
        }
        return (int)LTE_ERR_UNSUPPORTED;
    };
    return p.dtype == LTE_BF16 ? dims(__nv_bfloat16()) : dims(0.f);
}

}  // namespace

int launch_cache4_pack(const Params& p, const void* cache, void* cache4, cudaStream_t st)
{
    const CacheLayout L = cache_layout(p.d, p.W, p.R, p.dtype);
    const Cache4Layout Q = cache4_layout(p.d, p.W, p.R);
    const int parts = (p.W + p.R + PROWS - 1) / PROWS;
    return by_type(p, [&](auto t, auto d) {
        return cuda_status(launch_pdl(cache4_pack_kernel<decltype(t), decltype(d)::value>, dim3(parts * p.B * p.H), dim3(PT), 0, st,
                                      (const unsigned char*)cache, L, (unsigned char*)cache4, Q, p.W, p.R, parts)); });
}

int launch_cache4_unpack(const Params& p, const void* cache4, void* cache, cudaStream_t st)
{
    const CacheLayout L = cache_layout(p.d, p.W, p.R, p.dtype);
    const Cache4Layout Q = cache4_layout(p.d, p.W, p.R);
    const int parts = (L.rows_alloc + PROWS - 1) / PROWS;
    int* status = nullptr;
    if (int e = cache_status_word(&status)) return e;
    return by_type(p, [&](auto t, auto d) {
        return cuda_status(launch_pdl(cache4_unpack_kernel<decltype(t), decltype(d)::value>, dim3(parts * p.B * p.H), dim3(PT), 0, st,
                                      (const unsigned char*)cache4, Q, (unsigned char*)cache, L, p.W, p.R, parts, status)); });
}

}  // namespace lte
