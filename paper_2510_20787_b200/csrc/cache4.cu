// An ordinary decode cache into 4 bits, and back (see cache4.cuh for the rule and the order of the codes).
//
// Bound by memory: a thread takes eight channels of a row (16 or 32 bytes), four threads a group; they meet in two shuffles for its
// extremes.  Scores, positions and counters are copied by the same blocks.
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
    const int r0 = part * PROWS, n = min(PROWS, rows - r0) * PIECES;   // (a multiple of 4: the threads of a group stay together)
    for (int e = threadIdx.x; e < (n + 31) / 32 * 32; e += PT) {       // whole warps
        const int at = min(e, n - 1), row = r0 + at / PIECES, piece = at % PIECES, group = piece / 4, t = piece % 4;
#pragma unroll
        for (int values = 0; values < 2; ++values) {
            const Piece8<T> p = reinterpret_cast<const Piece8<T>*>(src + (values ? L.off_v : L.off_k))[piece_at(L, row, piece, PIECES)];
            float f[8];
            unpack8<T>(p, f);
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
            const uint32_t par = group4(lo, hi, bad);
            uint32_t w = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) w |= code4(f[i], par) << (4 * i);
            if (e < n) {
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
    if (blockIdx.x == 0 && threadIdx.x < Q.header / 4) reinterpret_cast<uint32_t*>(cache4)[threadIdx.x] = 0u;
}

template <typename T, int D>
__global__ void __launch_bounds__(PT) cache4_unpack_kernel(const unsigned char* __restrict__ cache4, Cache4Layout Q, unsigned char* __restrict__ cache,
                                                           CacheLayout L, int W, int R, int parts)
{
    constexpr int PIECES = D / 8, GROUPS = D / kGroup4;
    pdl_launch_dependents();
    pdl_wait();
    const int bh = blockIdx.x / parts, part = blockIdx.x - bh * parts, rows = W + R;
    const unsigned char* src = cache4 + Q.header + (size_t)bh * Q.stride;
    unsigned char* dst = cache + L.header + (size_t)bh * L.stride;
    const int r0 = part * PROWS, n = min(PROWS, L.rows_alloc - r0) * PIECES;
    for (int e = threadIdx.x; e < n; e += PT) {
        const int row = r0 + e / PIECES, piece = e % PIECES, group = piece / 4, t = piece % 4;
#pragma unroll
        for (int values = 0; values < 2; ++values) {
            float f[8];
            if (row < rows) {
                const unsigned char* codes = src + (values ? Q.off_v : Q.off_k) + (size_t)row * (D / 2);
                const uint32_t par = reinterpret_cast<const uint32_t*>(src + (values ? Q.off_vp : Q.off_kp))[(size_t)row * GROUPS + group];
                const uint32_t w = values ? reinterpret_cast<const uint16_t*>(codes)[2 * t * GROUPS + group] |
                                                (uint32_t)reinterpret_cast<const uint16_t*>(codes)[(2 * t + 1) * GROUPS + group] << 16
                                          : reinterpret_cast<const uint32_t*>(codes)[t * GROUPS + group];
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = value4((w >> (4 * i)) & 15u, par);
            } else {                                           // the swizzled layout's rows behind the last one
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = 0.f;
            }
            reinterpret_cast<Piece8<T>*>(dst + (values ? L.off_v : L.off_k))[piece_at(L, row, piece, PIECES)] = pack8(f, T());
        }
    }
    copy_tail(src, Q.off_z, Q.off_pidx, Q.off_meta, dst, L.off_z, L.off_pidx, L.off_meta, L.stride, rows, R, part, parts);
    if (blockIdx.x == 0 && threadIdx.x < L.header / 4) reinterpret_cast<uint32_t*>(cache)[threadIdx.x] = 0u;
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
    return by_type(p, [&](auto t, auto d) {
        return cuda_status(launch_pdl(cache4_unpack_kernel<decltype(t), decltype(d)::value>, dim3(parts * p.B * p.H), dim3(PT), 0, st,
                                      (const unsigned char*)cache4, Q, (unsigned char*)cache, L, p.W, p.R, parts)); });
}

}  // namespace lte
