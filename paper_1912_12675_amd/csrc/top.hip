// A row's k largest logits in order, with their classes, and the logarithm of
// its sum of exponentials (psw_top_logits in include/psw.h).
//
// A number and its class make one 64-bit key, larger for the larger number and,
// among equal ones, for the lower class, so no two keys are equal and the result
// is one set in one order.  A workgroup holds its row in registers (rows.h).
// The k-th largest of the maxima of 64 or more groups of threads is at most the
// row's k-th largest.  The few chunks whose largest element is from there up go
// to a list in LDS, their elements from there up to a list of keys, and a key's
// place is the number of larger ones there.
// Where equal numbers make a list too long (a row that a mask has left nearly
// empty), binary searches find the k-th largest number and the last class that
// belongs to the result of those that are equal to it.
//
// Rows too long are cut into pieces, whose first k a second kernel merges.
//
// A row is read once.  Bound by instructions nearly as much as by memory: 2048
// rows of 50257 bfloat16, 64 wanted, take 62 us for 206 MB (3.3 TB/s), in which
// a logit has 10 instructions, four of them its exponential's; the two rows of a
// CU load and reckon in step.  The largest of three with NaN kept is one
// instruction (with NaN looked for apart, and all chunks' elements compared where
// the chunk lies, 87 us).  Few rows are launches and latency: 16 rows of 1000 6 us.
#include <math.h>

#include <algorithm>

#include "distill.h"
#include "internal.h"
#include "rows.h"

namespace psw {
namespace {

// Keys and chunks of a list, by the workgroup's threads: those of one wave leave LDS for 32 workgroups a CU.
__host__ __device__ constexpr int keys_of(int t) { return t == 64 ? 256 : 1024; }
__host__ __device__ constexpr int chunks_of(int t) { return t == 64 ? 128 : 512; }
constexpr int kFirst = 640;                // of a row's pieces, 2 k and one for each piece at most: 577
constexpr float kLog2e = 1.4426950408889634f;
typedef unsigned long long u64;

struct TopArgs {
    const void* z;
    int64_t ld;
    int n, classes, k;
    double inv_tau;  // 1 / tau
    float kt;        // log2(e) / tau
    float *val, *lse;
    int32_t* idx;
    int splits, per;  // pieces of a row, chunks of a piece
    u64* keys;        // [n][splits][k]
    float2* part;     // [n][splits]: largest, sum of exponentials
};

// numbers in order as unsigned integers above 0: NaN above all, -0 as 0
__device__ __forceinline__ uint32_t order(float v)
{
    if (v != v) return 0xffffffffu;
    const uint32_t u = __float_as_uint(v + 0.f);
    return u >> 31 ? ~u : u | 0x80000000u;
}

// A number that at least k of the workgroup's elements reach, 1 where all are
// wanted, from the orders of its threads' largest, most[T], by one wave.  Of the
// number the first BITS bits are found, the others are 0.
template <int T, int BITS>
__device__ __forceinline__ uint32_t reached(int k, const uint32_t* most)
{
    // groups of threads, twice as many as are wanted where there are as many
    uint32_t t = 0;
    auto kth = [&](auto groups) {
        constexpr int G = decltype(groups)::value;
        uint32_t m[G];
#pragma unroll
        for (int i = 0; i < G; ++i) {
            m[i] = 0;
#pragma unroll
            for (int j = 0; j < T / 64; j += G) m[i] = max(m[i], most[(threadIdx.x & 63) + 64 * (i + j)]);
        }
        if (k > 64 * G) return;  // every key
#pragma unroll 1
        for (uint32_t bit = 0x80000000u; bit >> (32 - BITS); bit >>= 1) {
            int c = 0;
#pragma unroll
            for (int i = 0; i < G; ++i) c += __popcll(__ballot(m[i] >= (t | bit)));
            if (c >= k) t |= bit;
        }
    };
    if (T == 64 || k <= 32)
        kth(std::integral_constant<int, 1>{});
    else if (T == 128 || k <= 64)
        kth(std::integral_constant<int, (T >= 128 ? 2 : 1)>{});
    else if (T == 256 || k <= 128)
        kth(std::integral_constant<int, (T >= 256 ? 4 : 1)>{});
    else
        kth(std::integral_constant<int, (T >= 512 ? 8 : 1)>{});
    return max(t, 1u);
}

// Of the list's keys each of the k largest goes to put(place, key).
template <int T, typename Put>
__device__ __forceinline__ void place_all(const u64* list, int count, int k, Put put)
{
    for (int i = threadIdx.x; i < count; i += T) {
        const u64 key = list[i];
        int place = 0, j = 0;
        for (; j + 8 <= count; j += 8) {
            u64 other[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) other[e] = list[j + e];
#pragma unroll
            for (int e = 0; e < 8; ++e) place += other[e] > key;
        }
        for (; j < count; ++j) place += list[j] > key;
        if (place < k) put(place, key);
    }
}

__device__ __forceinline__ int class_of(u64 key) { return (int)~(uint32_t)key; }
__device__ __forceinline__ float number_of(uint32_t o) { return __uint_as_float(o >> 31 ? o & 0x7fffffffu : ~o); }

// the larger of two, NaN where one is
__device__ __forceinline__ float largest(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// what a sum of exponentials is relative to: the largest logit, or 0 where that is no number to take away
__device__ __forceinline__ float base(float m) { return m == INFINITY || m == -INFINITY ? 0.f : m; }

template <typename E, int T, int NV, bool PIECE>
__global__ __launch_bounds__(T) void top_k(TopArgs a)
{
    constexpr int P = Row<E>::kPer, kList = keys_of(T), kCuts = chunks_of(T);
    __shared__ float shf[2][T / 64];
    __shared__ uint32_t most[T], bound;
    __shared__ int sum[T / 64], count, cuts, place[kCuts];
    __shared__ u64 list[kList];
    __shared__ __attribute__((aligned(16))) E cut[kCuts * P];
    const int tid = threadIdx.x, row = PIECE ? blockIdx.x / a.splits : blockIdx.x, piece = PIECE ? blockIdx.x % a.splits : 0;
    const Row<E> z((const E*)a.z + (int64_t)row * a.ld, a.classes);
    const int c0 = PIECE ? piece * a.per : 0, c1 = PIECE ? min(z.chunks, c0 + a.per) : z.chunks;
    Chunk v[NV];
    const int lo = z.lo(c0), hi = z.hi(c1), es = z.single(c0, c1);
    const float xs = es >= 0 ? (float)z.p[es] : -INFINITY;
    z.template load<T>(v, c0, lo, hi);
    // calls f(chunk of the row, its elements) for this thread's chunks
    auto rows = [&](auto f) {
        // Floats (and comparisons of them) are formed anew for every pass: kept, they would take twice the row's registers.
        int t = tid, half = 16, same = 0;
        asm volatile("" : "+v"(t), "+s"(half), "+s"(same));
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (c0 + i * T < hi)
                f(c0 + i * T + t, [&](int j) {
                    if constexpr (sizeof(E) == 4) return __uint_as_float(v[i][j] ^ (uint32_t)same);
                    const uint32_t low = v[i][j / 2] << half, high = v[i][j / 2] >> half << half;
                    return __uint_as_float(j & 1 ? high : low);
                });
    };
    // B1: every thread's largest.  One wave finds the bound while the others begin with the sum.  B2: bound and sum.
    float m = xs;
    rows([&](int, auto x) {
#pragma unroll
        for (int j = 0; j < P; ++j) m = largest(m, x(j));
    });
    const int lane = tid & 63, wave = tid >> 6;
    const int have = max(min(z.first(c1), a.classes) - max(z.first(c0), 0), 0);  // elements of the row or piece
    const int k = min(a.k, have);
    most[tid] = order(m);
    m = wave_reduce(m, [](float x, float y) { return fmaxf(x, y); });
    if (lane == 0) shf[0][wave] = m;
    if (tid == 0) count = cuts = 0;
    __syncthreads();
    if (wave == 0) {
        const uint32_t t = reached<T, sizeof(E) == 4 ? 24 : 16>(k, most);
        if (lane == 0) bound = t;
    }
    if (a.lse) {
        m = shf[0][0];
#pragma unroll
        for (int w = 1; w < T / 64; ++w) m = fmaxf(m, shf[0][w]);
        const float m0 = base(m), kt = a.kt;
        // 2^(x kt - b) with b the rounded m0 kt, whose rounding is taken back below
        const float b = m0 * kt;
        const bool far = fabsf(b) > kFar;
        float s = __builtin_amdgcn_exp2f(far ? (xs - m0) * kt : fmaf(xs, kt, -b));
        if (far)
            rows([&](int, auto x) {
#pragma unroll
                for (int j = 0; j < P; ++j) s += __builtin_amdgcn_exp2f((x(j) - m0) * kt);
            });
        else
            rows([&](int, auto x) {
#pragma unroll
                for (int j = 0; j < P; ++j) s += __builtin_amdgcn_exp2f(fmaf(x(j), kt, -b));
            });
        s = wave_reduce(s, [](float x, float y) { return x + y; });
        if (lane == 0) shf[1][wave] = s;
        __syncthreads();
        if (tid == 0) {
#pragma unroll
            for (int w = 1; w < T / 64; ++w) s += shf[1][w];
            if (!far) s *= __builtin_amdgcn_exp2f(-fmaf(m0, kt, -b));
            if constexpr (PIECE)
                a.part[(int64_t)row * a.splits + piece] = make_float2(m, s);
            else
                a.lse[row] = (float)((double)m0 * a.inv_tau + log_of((double)s));
        }
    } else {
        __syncthreads();
    }

    // What is taken: numbers of order `u` and up, by a comparison of floats (past infinity's order there is only NaN,
    // below -inf's everything); of those equal to it only classes up to `last` where ties > 0.
    uint32_t u = bound;
    int last = a.classes;
    bool ties = false;
    auto value_of = [](uint32_t o) { return o > 0xff800000u ? INFINITY : o <= 0x007fffffu ? -INFINITY : number_of(o); };
    for (int round = 0;; ++round) {
        const float x0 = value_of(u);
        const u64 least = (u64)u << 32 | (ties ? (uint32_t)~last : 0u);
        auto key = [&](float x, int e) { return (u64)order(x) << 32 | (uint32_t)~e; };
        auto take = [&](u64 x) {
            if (x < least) return;
            const int at = atomicAdd(&count, 1);
            if (at < kList) list[at] = x;
        };
        rows([&](int c, auto x) {
            float top = x(0);
#pragma unroll
            for (int j = 1; j < P; ++j) top = largest(top, x(j));
            if (top < x0 || c < lo || c >= hi) return;
            if (ties) {
                bool any = false;
#pragma unroll
                for (int j = 0; j < P; ++j) any |= key(x(j), z.first(c) + j) >= least;
                if (!any) return;
            }
            const int at = atomicAdd(&cuts, 1);
            if (at >= kCuts) return;
            place[at] = z.first(c);
#pragma unroll
            for (int j = 0; j < P; ++j) cut[at * P + j] = (E)x(j);
        });
        if (es >= 0) take(key(xs, es));
        __syncthreads();
        for (int i = tid; i < min(cuts, kCuts) * P; i += T) take(key((float)cut[i], place[i / P] + i % P));
        __syncthreads();
        if ((cuts <= kCuts && count <= kList) || round > 0) break;
        // Too many: the k-th largest number, bit by bit, ...
        uint32_t t = 0;
#pragma unroll 1
        for (uint32_t bit = 0x80000000u; bit; bit >>= 1) {
            const uint32_t want = t | bit;
            int c = 0;
            if (want > 0x007fffffu) {
                const float x1 = value_of(want);
                const bool nan1 = want > 0xff800000u;
                c = nan1 ? xs != xs : !(xs < x1);
                rows([&](int, auto x) {
#pragma unroll
                    for (int j = 0; j < P; ++j) {
                        const float y = x(j);
                        c += nan1 ? y != y : !(y < x1);
                    }
                });
                c = block_reduce<T>(c, sum, [](int x, int y) { return x + y; });
                __syncthreads();
            } else {
                c = have;
            }
            if (c >= k) t = want;
        }
        // ... and the place of the last that counts among those equal to it: `before` elements are larger
        const float xk = value_of(t);
        const bool nank = t > 0xff800000u;
        int before = !nank && !(xs <= xk);
        rows([&](int, auto x) {
#pragma unroll
            for (int j = 0; j < P; ++j) {
                before += nank ? 0 : !(x(j) <= xk);
            }
        });
        before = block_reduce<T>(before, sum, [](int x, int y) { return x + y; });
        __syncthreads();
        int at = 0;
#pragma unroll 1
        for (int bit = 1 << (31 - __clz(a.classes)); bit; bit >>= 1) {
            const int want = at | bit;
            int c = (nank ? xs != xs : xs == xk) && es >= 0 && es < want;
            rows([&](int chunk, auto x) {
                const int e0 = z.first(chunk);
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    const float y = x(j);
                    c += (nank ? y != y : y == xk) && chunk >= lo && chunk < hi && e0 + j < want;
                }
            });
            c = block_reduce<T>(c, sum, [](int x, int y) { return x + y; });
            __syncthreads();
            if (before + c < k) at = want;
        }
        u = t;
        last = at;
        ties = true;
        if (tid == 0) count = cuts = 0;
        __syncthreads();
    }
    if constexpr (PIECE) {
        u64* out = a.keys + ((int64_t)row * a.splits + piece) * a.k;
        for (int i = k + tid; i < a.k; i += T) out[i] = 0;
        place_all<T>(list, min(count, kList), k, [&](int place, u64 x) { out[place] = x; });
    } else {
        place_all<T>(list, min(count, kList), k, [&](int place, u64 x) {
            a.val[(int64_t)row * a.k + place] = number_of((uint32_t)(x >> 32));
            a.idx[(int64_t)row * a.k + place] = class_of(x);
        });
    }
}

// The pieces' first k together, N a thread: 11 us for 33 pieces of 128, half of it
// the bound and the places' comparisons of one workgroup (a search of all keys' bits 14).
template <int T, int N>
__global__ __launch_bounds__(T) void top_merge_k(TopArgs a)
{
    constexpr int W = T / 64, kList = 1024;
    __shared__ float sh[2][W];
    __shared__ u64 list[kList];
    __shared__ int count, sum[W];
    __shared__ uint32_t first[kFirst], bound;
    const int tid = threadIdx.x, row = blockIdx.x;
    const u64* in = a.keys + (int64_t)row * a.splits * a.k;
    const int total = a.splits * a.k;
    u64 v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = i * T + tid < total ? in[i * T + tid] : 0;
    // The pieces' first `each`, at least 2 k of all: the k-th largest number of them is at most the result's last.
    const int each = min(a.k, (2 * a.k + a.splits - 1) / a.splits), firsts = each * a.splits;
    if (tid == 0) count = 0;
    for (int i = tid; i < kFirst; i += T)
        first[i] = i < firsts ? (uint32_t)(in[i / each * a.k + i % each] >> 32) : 0;
    __syncthreads();
    if (tid < 64) {
        uint32_t m[kFirst / 64], t = 0;
#pragma unroll
        for (int i = 0; i < kFirst / 64; ++i) m[i] = first[i * 64 + tid];
#pragma unroll 1
        for (uint32_t bit = 0x80000000u; bit; bit >>= 1) {
            int c = 0;
#pragma unroll
            for (int i = 0; i < kFirst / 64; ++i)
                if (i * 64 < firsts) c += __popcll(__ballot(m[i] >= (t | bit)));
            if (c >= a.k) t |= bit;
        }
        if (tid == 0) bound = t;
    }
    if (a.lse) {
        const float2* part = a.part + (int64_t)row * a.splits;
        const float kt = a.kt;
        float m = -INFINITY, s = 0.f;
        for (int i = tid; i < a.splits; i += T) m = fmaxf(m, part[i].x);
        m = block_reduce<T>(m, sh[0], [](float x, float y) { return fmaxf(x, y); });
        for (int i = tid; i < a.splits; i += T) {
            const float2 f = part[i];
            // a piece without a logit above -inf adds nothing (or a NaN): relative to a row far below 0 its base, 0, is infinite
            const bool as_is = f.x == m || f.x == -INFINITY;
            s += as_is ? f.y : f.y * __builtin_amdgcn_exp2f((base(f.x) - base(m)) * kt);
        }
        s = block_reduce<T>(s, sh[1], [](float x, float y) { return x + y; });
        if (tid == 0) a.lse[row] = (float)((double)base(m) * a.inv_tau + log_of((double)s));
    }
    __syncthreads();
    u64 least = (u64)max(bound, 1u) << 32;
    auto take = [&] {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (v[i] >= least) {
                const int at = atomicAdd(&count, 1);
                if (at < kList) list[at] = v[i];
            }
        __syncthreads();
    };
    take();
    if (count > kList) {
        // Equal numbers, or a piece with most of the result: the bits of a key that k reach, from the highest down, until
        // those that do are few (placing them takes their square).
        __syncthreads();
        int reach = total;
        least = 0;
#pragma unroll 1
        for (int bit = 63; bit >= 0 && reach > max(2 * a.k, 128); --bit) {
            const u64 want = least | (u64)1 << bit;
            int c = 0;
#pragma unroll
            for (int i = 0; i < N; ++i) c += v[i] >= want;
            c = block_reduce<T>(c, sum, [](int x, int y) { return x + y; });
            __syncthreads();
            if (c >= a.k) {
                least = want;
                reach = c;
            }
        }
        least = least ? least : 1;
        if (tid == 0) count = 0;
        __syncthreads();
        take();
    }
    place_all<T>(list, min(count, kList), a.k, [&](int place, u64 x) {
        a.val[(int64_t)row * a.k + place] = number_of((uint32_t)(x >> 32));
        a.idx[(int64_t)row * a.k + place] = class_of(x);
    });
}

// Chunks of a piece; 0: rows whole, wherever a workgroup's registers hold one (8 rows of 30000 float32: 9.4 us, in pieces 6.8
// and 9.2; 120 rows of 50000: 12.5, in pieces 11.8 and 8.4; 1024 of 60000: 72, in pieces 67 and 11).  Small pieces for few
// rows and entries, so that the chip is full; with large ones there are fewer keys to merge.
struct Cut {
    int per, splits;
    Cut(int n, int64_t bytes, int k)
    {
        per = 0;
        splits = 1;
        if (bytes <= 16 * 1024 * 16) return;
        per = 256 * 4;
        splits = (int)((bytes + 16 * per - 1) / (16 * per));
        if (n >= 128 || k > 128 || (int64_t)splits * k > 8 * 1024) {
            per = 512 * 8;
            splits = (int)((bytes + 16 * per - 1) / (16 * per));
        }
    }
    // of the workspace: the pieces' first k and sums
    size_t ws_bytes(int n, int k) const { return splits > 1 ? (size_t)n * splits * (k * sizeof(u64) + sizeof(float2)) : 0; }
};

// Calls f(bytes of a row) with and without a chunk more for rows that begin inside one: the launch's are one of the two.  More
// bytes can mean fewer pieces (33 small ones of 128 entries turn to 17 large ones).
template <typename F>
void each_bytes(int classes, int size, F f)
{
    f((int64_t)classes * size);
    f(row_bytes(classes, size));
}

// Threads of a workgroup with a whole row.  Enough for groups to choose the bound from: with k of 2 k groups the list holds
// about 1.4 k keys, with k of k groups k times the logarithm of k, which is too many from 256 on.
int threads_of(int64_t bytes, int k)
{
    if (bytes <= 16 * 64 * 4 && k <= 32) return 64;
    if (bytes <= 16 * 256 * 8 && k <= 128) return 256;
    return bytes <= 16 * 512 * 16 ? 512 : 1024;
}
int merge_threads(int splits, int k) { return splits * k <= 8 * 256 ? 256 : 1024; }

template <typename E>
void launch(const TopArgs& a, int64_t bytes, const Work& w, hipStream_t st)
{
    const dim3 rows((unsigned)a.n);
#define PSW_TOP(T, NV, PIECE, GRID) \
    PSW_LAUNCH(kname("top_k", (int)sizeof(E), T, NV, PIECE), w, (top_k<E, T, NV, PIECE>), GRID, dim3(T), 0, st, a)
    if (a.splits > 1) {
        const dim3 pieces((unsigned)a.n * (unsigned)a.splits);
        if (a.per == 256 * 4)
            PSW_TOP(256, 4, true, pieces);
        else
            PSW_TOP(512, 8, true, pieces);
#define PSW_MERGE(T, N) PSW_LAUNCH(kname("top_merge_k", T, N), w, (top_merge_k<T, N>), rows, dim3(T), 0, st, a)
        if (merge_threads(a.splits, a.k) == 256)
            PSW_MERGE(256, 8);
        else if (a.splits * a.k <= 8 * 1024)
            PSW_MERGE(1024, 8);
        else
            PSW_MERGE(1024, 20);
#undef PSW_MERGE
        return;
    }
    const int t = threads_of(bytes, a.k);
    if (t == 64)
        PSW_TOP(64, 4, false, rows);
    else if (t == 256 && bytes <= 16 * 256 * 4)
        PSW_TOP(256, 4, false, rows);
    else if (t == 256)
        PSW_TOP(256, 8, false, rows);
    else if (t == 512 && bytes <= 16 * 512 * 8)
        PSW_TOP(512, 8, false, rows);
    else if (t == 512)
        PSW_TOP(512, 16, false, rows);
    else
        PSW_TOP(1024, 16, false, rows);
#undef PSW_TOP
}

}  // namespace

size_t top_logits_ws_bytes(int n, int classes, int k)
{
    size_t need = 0;
    for (int size : {2, 4})
        each_bytes(classes, size, [&](int64_t bytes) { need = std::max(need, Cut(n, bytes, k).ws_bytes(n, k)); });
    return need;
}

bool top_logits_fits(int n, int classes, int k, int bf16)
{
    int64_t most = 0;
    each_bytes(classes, bf16 ? 2 : 4, [&](int64_t bytes) {
        const Cut c(n, bytes, k);
        const int64_t pieces = (int64_t)c.splits * (c.per == 256 * 4 ? 256 : 512);
        most = std::max(most, c.splits > 1 ? std::max<int64_t>(pieces, merge_threads(c.splits, k)) : threads_of(bytes, k));
    });
    return n * most <= kGridThreads;
}

hipError_t top_logits(int n, int classes, int bf16, const void* z, int64_t ld, int k, float tau, float* val, int32_t* idx,
                      float* lse, void* ws, hipStream_t st)
{
    TopArgs a{};
    a.z = z; a.ld = ld; a.n = n; a.classes = classes; a.k = k; a.inv_tau = 1.0 / (double)tau; a.kt = kLog2e / tau;
    a.val = val; a.idx = idx; a.lse = lse;
    const int64_t bytes = row_bytes(classes, bf16 ? 2 : 4, z, ld, n);
    const Cut c(n, bytes, k);
    a.splits = c.splits;
    a.per = c.per;
    a.keys = (u64*)ws;
    a.part = (float2*)((u64*)ws + (size_t)n * c.splits * k);
    const Work w{4.0 * n * classes, (bf16 ? 2.0 : 4.0) * n * classes + 8.0 * n * k};
    if (bf16)
        launch<__bf16>(a, bytes, w, st);
    else
        launch<float>(a, bytes, w, st);
    return hipGetLastError();
}

}  // namespace psw
