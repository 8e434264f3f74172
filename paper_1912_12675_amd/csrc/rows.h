// A row of logits held in the registers of a workgroup: 16-byte chunks, chunk c
// of the row with thread c mod T, as they lie in memory (float32 or bfloat16).
// A row that does not start on a 16-byte boundary is cut at the boundaries; the
// elements of its first and last chunk are then one more for a few threads each
// (loaded into their chunk's place, element by element, they held up the row by
// several us, or took its registers twice).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "grid.h"

namespace psw {

typedef uint32_t Chunk __attribute__((ext_vector_type(4)));  // a value of its own, where a uint4 is four

template <typename E>
struct Row {
    static constexpr int kPer = 16 / (int)sizeof(E);  // elements of a chunk
    const E* p;
    int count;  // elements
    int shift;  // elements of chunk 0 that lie before the row
    int chunks;

    __device__ Row(const E* row, int n) : p(row), count(n), shift((int)((uintptr_t)row % 16 / sizeof(E)))
    {
        chunks = (int)(((int64_t)n + shift + kPer - 1) / kPer);
    }
    // first element of chunk c, negative where it begins before the row
    __device__ int first(int c) const { return c * kPer - shift; }
    __device__ bool inside(int c) const { return first(c) >= 0 && first(c) + kPer <= count; }

    static __device__ Chunk none() { return Chunk(sizeof(E) == 4 ? 0xff800000u : 0xff80ff80u); }
    // The whole chunks of c0 <= c < c1 are lo <= c < hi; the rest's elements go to single threads.
    __device__ int lo(int c0) const { return c0 == 0 && !inside(0) ? 1 : c0; }
    __device__ int hi(int c1) const { return c1 == chunks && !inside(chunks - 1) ? chunks - 1 : c1; }
    // Chunks c0 + i T + thread, -inf where they are not between lo and hi.
    template <int T, int NV>
    __device__ void load(Chunk (&v)[NV], int c0, int lo, int hi) const
    {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = c0 + i * T + threadIdx.x;
            v[i] = none();
            if (c >= lo && c < hi) v[i] = *reinterpret_cast<const Chunk*>(p + first(c));
        }
    }
    // the element of a cut chunk that is this thread's, or -1
    __device__ int single(int c0, int c1) const
    {
        const int tid = threadIdx.x, last = chunks - 1;
        int e = -1;
        if (tid < kPer && c0 == 0 && c1 > 0 && !inside(0)) e = first(0) + tid;
        if (tid >= kPer && tid < 2 * kPer && last > 0 && c1 == chunks && c0 <= last && !inside(last))
            e = first(last) + tid - kPer;
        return e >= 0 && e < count ? e : -1;
    }
};

// The logarithm of a sum or probability, within 1e-7: the exponent's part exact, the rest's in fp32 (many short rows are
// bound by 64-bit arithmetic; the library's logarithm takes ten times the instructions).
__device__ __forceinline__ double log_of(double x)
{
    const float m = (float)__builtin_amdgcn_frexp_mant(x);
    return ((double)__builtin_amdgcn_frexp_exp(x) + (double)__builtin_amdgcn_logf(m)) * 0.69314718055994530942;
}

// Past this product of a row's largest logit m and a factor k, exponents x k - m k are formed as (x - m) k.  Up to it the
// rounding of m k is at most 4, and taken back from the sums.  x - m is exact in float where x is at least half of m, and
// in bfloat16 where it is less than 256 of the smaller's steps; otherwise it is at least |m| / 2 and its exponential 0, also
// with a factor 2^16 times smaller.
constexpr float kFar = 0x1p26f;

// Bytes of chunks that a row can take, where it is not known how rows lie: a chunk more where one begins inside another.
inline int64_t row_bytes(int classes, int size) { return (int64_t)classes * size + 16; }
inline int64_t row_bytes(int classes, int size, const void* z, int64_t ld, int n)
{
    const bool even = (uintptr_t)z % 16 == 0 && (n == 1 || ld * size % 16 == 0);
    return (int64_t)classes * size + (even ? 0 : 16);
}

// element j of a chunk
template <typename E>
__device__ __forceinline__ float element(Chunk w, int j)
{
    if constexpr (sizeof(E) == 4) return __uint_as_float(w[j]);
    return __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
}

// Reductions over a workgroup of T threads, in a fixed order, every thread with
// the result.  `sh` [T / 64] is used by one reduction between two barriers of
// the caller's (a workgroup of one wave needs neither).
template <typename V, typename F>
__device__ __forceinline__ V wave_reduce(V v, F f)
{
#pragma unroll
    for (int d = 32; d >= 1; d /= 2) v = f(v, __shfl_xor(v, d));
    return v;
}
template <int T, typename V, typename F>
__device__ __forceinline__ V block_reduce(V v, V* sh, F f)
{
    v = wave_reduce(v, f);
    if constexpr (T == 64) return v;
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sh[0];
#pragma unroll
    for (int w = 1; w < T / 64; ++w) v = f(v, sh[w]);
    return v;
}

}  // namespace psw
