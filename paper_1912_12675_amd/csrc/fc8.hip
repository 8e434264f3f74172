// Fully connected products of 8-bit operands (q8.hip): C[m][n] (+)= sum_k
// A[m][k] B[n][k], both operands' rows contiguous along k in whole blocks of
// 128, a power-of-two scale for each row (or 128 rows) and block.
//
// Two ways through the matrix cores:
//  - bfloat16 results: v_mfma_scale_f32_32x32x64_f8f6f4, which takes e4m3 values
//    and the scales' exponents as they are, 4.7 PFLOP/s on this card.  It aligns
//    the products of a few neighbouring k to the largest of them and drops what
//    falls below: measured on normal, half-normal and long-tailed operands an
//    error of 1.5e-5 to 7e-5 of the root of the summed squares (any depth, any of
//    the 8-bit instructions), a fiftieth of bfloat16's own rounding, 2^-9 to 2^-8 of
//    a result that is as large.
//  - float32 results, and few rows of either type: the values times their scales
//    as bfloat16 (e4m3 has four significant bits, so that is exact from 2^-133,
//    bfloat16's smallest, up to below 2^128) by v_cvt_scalef32_pk_bf16_fp8, and
//    v_mfma_f32_32x32x16_bf16, whose products are exact, of subnormal numbers too,
//    and whose sums are fp32: 1e-8 to 4e-7 on the same operands, at 2.45 PFLOP/s.
#include <algorithm>
#include <type_traits>

#include "internal.h"
#include "q8.h"

namespace psw {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v2b __attribute__((ext_vector_type(2)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));

struct MmArgs {
    const uint8_t *A, *B;    // [M][kp], [N][kp]
    const uint8_t *sa, *sb;  // scale bytes [M >> ashift][sp], [N >> bshift][sp]
    void* C;                 // [M][N] float or bfloat16; of a part: float [parts][M][N]
    const float* bias;       // per column n, or null
    int M, N, K;             // K in blocks of 128
    int64_t kp;
    int sp, ashift, bshift;
    int mblocks, nblocks;
    int chunk;               // blocks of K in a part (blockIdx.y), a multiple of four
    int relu, accumulate, bf16;
};

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float((byte & 255u) << 23); }

// 16 values at their scale, two operands of eight
__device__ __forceinline__ void widen(v4i w, float s, v8b& lo, v8b& hi)
{
    v2b p[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        p[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)w[i], s, false);
        p[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)w[i], s, true);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        lo[2 * i] = p[i][0]; lo[2 * i + 1] = p[i][1];
        hi[2 * i] = p[4 + i][0]; hi[2 * i + 1] = p[4 + i][1];
    }
}

typedef float Four __attribute__((ext_vector_type(4), aligned(4)));  // in memory: gfx950 takes it at any float's address

// bias, ReLU and the result's type for four neighbours of a row; without
// `whole` (a part's sums) the plain floats
__device__ __forceinline__ void store4(const MmArgs& a, void* C, int m, int n, v4f v, bool whole)
{
    const int64_t at = (int64_t)m * a.N + n;
    const bool all = n + 3 < a.N;
    if (whole) {
        if (a.bias)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < a.N) v[e] += a.bias[n + e];
        if (a.relu)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = v[e] < 0.f ? 0.f : v[e];  // NaN stays
    }
    if (whole && a.bf16) {
        __bf16* p = (__bf16*)C + at;
        if (all && !a.accumulate) {
            typedef __bf16 v4b __attribute__((ext_vector_type(4), aligned(2)));
            *reinterpret_cast<v4b*>(p) = v4b{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
            return;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < a.N) p[e] = (__bf16)(a.accumulate ? (float)p[e] + v[e] : v[e]);
        return;
    }
    float* p = (float*)C + at;
    const bool add = whole && a.accumulate;
    if (all) {
        Four* q = reinterpret_cast<Four*>(p);
        *q = add ? *q + v : v;
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (n + e < a.N) p[e] = add ? p[e] + v[e] : v[e];
}

typedef __amdgpu_buffer_rsrc_t Buffer;
// `bytes` from p on; what lies behind them reads as zero, without a memory access
__device__ __forceinline__ Buffer buffer_of(const uint8_t* p, uint32_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, (int)bytes, 0x00020000);
}
// 16 bytes a lane from memory to LDS: lane i to `to` + 16 i
__device__ __forceinline__ void to_lds(Buffer b, uint32_t lane_bytes, int uniform_bytes, uint8_t* to)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(b, (__attribute__((address_space(3))) void*)to, 16, (int)lane_bytes,
                                             uniform_bytes, 0, 0);
}

// The waves of a workgroup meet; what this wave waited for before is done.
__device__ __forceinline__ void meet()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// The order of what lies between two barriers of the scheduler, left to itself
// it puts the reads last, where they save registers and are waited for: COUNT
// instructions of the kind `mask`, spread over MFMA matrix instructions.
constexpr int kReadLds = 0x100, kLoad = 0x010;
template <int MASK, int COUNT, int MFMA, int I = 0>
__device__ __forceinline__ void weave()
{
    if constexpr (I < MFMA) {
        constexpr int n = (I + 1) * COUNT / MFMA - I * COUNT / MFMA;
        if constexpr (n > 0) __builtin_amdgcn_sched_group_barrier(MASK, n, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        weave<MASK, COUNT, MFMA, I + 1>();
    }
}

// A tile of BM x BN by WM x WN waves.  A block (128) of the depth of an operand's
// rows is a stage of LDS, 128 bytes a row, loaded there directly in whole lines
// (a half block's 64 bytes a row pass at half the rate: 61 bytes a ns and CU
// from L2, whole lines 130); D + 1 stages of A and D of B.  D is 2 where tiles
// are many: 80 KB for 128 x 128, two workgroups a CU, and 160 KB for 256 x 256; 4
// where a CU has one small tile and memory's latency shows (128 x 16384 x 4096 by
// 128 x 64: 30.5 us with 2, 24.6 with 4, 27.2 with 5).  While one half of a block
// is on the matrix cores the next half's operands are read into registers.  In
// the middle of block k the waves meet: k is then read to its end, so B's loads
// of k + D can go where k was, and k + 1's loads have landed.  A's loads of k + D
// went out in the first half.  A load so has the time of D - 1 to D - 1/2 blocks,
// and matrix instructions lie between the loads and reads (all loads of a block in
// one go wait for each other, and the matrix cores behind them).
// The 16-byte unit u of row r lies in place u ^ (r / 2 & 7): a wave's loads fill
// eight rows in lane order (each lane fetches the unit that belongs in its
// place), and the 16 lanes that LDS serves in a cycle meet no bank twice.
// Bound by the matrix cores and the power they draw where tiles are many, at 1.7
// GHz: 4096 x 16384 -> 8192 float32 724 to 783 us by card and clock (1.4 to 1.52
// PFLOP/s; the matrix cores are busy in 82% of a CU's cycles), 8192 x 4096 -> 16384
// bfloat16 450 to 550 us (2.0 to 2.4 PFLOP/s; 60%: a tile's first loads and last
// stores, 12 us of each of the eight rounds, are not hidden).  With few tiles by the
// operand that is read once: 128 x 16384 -> 4096 25 us for 69 MB, of which 14
// are the bytes, the rest the conversions of 96 operands for 16 matrix
// instructions and the rows' 128 bytes at a time from HBM; the same number of
// tiles and blocks with rows 4 KB apart (dx of that layer) 37 us.
// The matrix instruction's rows are C's columns, so that a lane ends with four
// neighbours of a row of C; a wave's rows turn in LDS and are stored whole.
template <int BM, int BN, int WM, int WN, int D, bool F8>
__global__ __launch_bounds__(64 * WM * WN) void mm8_tiles(MmArgs a)
{
    constexpr int W = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32, LA = BM / 8 / W, LB = BN / 8 / W;
    static_assert(W % 2 == 0, "a wave's rows begin at the same place of the units' turn");
    constexpr int kA = D + 1, kB = D, kAt = kA * BM * kQ8Block, kBytes = kAt + kB * BN * kQ8Block;
    constexpr int kStrip = 32 * TN * 32 * 4;  // bytes of 32 rows of a wave's sums
    static_assert(W * kStrip <= kBytes, "the strips lie where the operands did");
    __shared__ __align__(1024) uint8_t lds[kBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // workgroups with the same id modulo 8 share an L2: each takes a run of tiles, in bands of four tiles of rows
    const int64_t tiles = (int64_t)a.mblocks * a.nblocks, per = (tiles + 7) / 8;
    const int64_t t = (int64_t)(blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int64_t)(blockIdx.x >> 3) >= per || t >= tiles) return;
    const int64_t band = 4 * (int64_t)a.nblocks;
    const int first = (int)(t / band) * 4, deep = min(4, a.mblocks - first), in = (int)(t % band);
    const int m0 = (first + in % deep) * BM, n0 = in / deep * BN;
    const int k0 = (int)blockIdx.y * a.chunk, steps = min(a.K, k0 + a.chunk) - k0;

    // offsets in a tile's rows: at most 256 rows of 2^23 bytes
    const int mrows = min(BM, a.M - m0), nrows = min(BN, a.N - n0);
    const uint8_t *pa = a.A + (int64_t)m0 * a.kp, *pb = a.B + (int64_t)n0 * a.kp;
    uint32_t oa[LA], ob[LB];
    const uint32_t unit = ((lane & 7) ^ (4 * (wave & 1) + (lane >> 4))) * 16, kp = (uint32_t)a.kp;
#pragma unroll
    for (int i = 0; i < LA; ++i) oa[i] = (uint32_t)min((wave + i * W) * 8 + (lane >> 3), mrows - 1) * kp + unit;
#pragma unroll
    for (int i = 0; i < LB; ++i) ob[i] = (uint32_t)min((wave + i * W) * 8 + (lane >> 3), nrows - 1) * kp + unit;
    // loads of a block behind the last are loads of nothing
    auto load_a = [&](int k, int slot) {
        const Buffer from = buffer_of(pa, k < steps ? (uint32_t)mrows * kp : 0);
#pragma unroll
        for (int i = 0; i < LA; ++i)
            to_lds(from, oa[i], (k0 + k) * kQ8Block, lds + slot * BM * kQ8Block + (wave + i * W) * 1024);
    };
    auto load_b = [&](int k, int slot) {
        const Buffer from = buffer_of(pb, k < steps ? (uint32_t)nrows * kp : 0);
#pragma unroll
        for (int i = 0; i < LB; ++i)
            to_lds(from, ob[i], (k0 + k) * kQ8Block, lds + kAt + slot * BN * kQ8Block + (wave + i * W) * 1024);
    };

    const int wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN), r = lane & 31, h = lane >> 5;
    // this lane's rows' scales, four blocks a word
    const uint8_t *qa = a.sa + (int64_t)(m0 >> a.ashift) * a.sp, *qb = a.sb + (int64_t)(n0 >> a.bshift) * a.sp;
    const uint32_t qa_bytes = (uint32_t)(((mrows - 1) >> a.ashift) + 1) * (uint32_t)a.sp;
    const uint32_t qb_bytes = (uint32_t)(((nrows - 1) >> a.bshift) + 1) * (uint32_t)a.sp;
    uint32_t ua[TM], ub[TN], sa[TM], sb[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) ua[i] = (uint32_t)(min(wm + 32 * i + r, mrows - 1) >> a.ashift) * (uint32_t)a.sp;
#pragma unroll
    for (int j = 0; j < TN; ++j) ub[j] = (uint32_t)(min(wn + 32 * j + r, nrows - 1) >> a.bshift) * (uint32_t)a.sp;
    auto scales = [&](int k, uint32_t(&x)[TM], uint32_t(&y)[TN]) {
        const int at = (k0 + k) & ~3;
        const Buffer fa = buffer_of(qa, k < steps ? qa_bytes : 0), fb = buffer_of(qb, k < steps ? qb_bytes : 0);
#pragma unroll
        for (int i = 0; i < TM; ++i) x[i] = __builtin_amdgcn_raw_buffer_load_b32(fa, (int)ua[i], at, 0);
#pragma unroll
        for (int j = 0; j < TN; ++j) y[j] = __builtin_amdgcn_raw_buffer_load_b32(fb, (int)ub[j], at, 0);
    };

    v16f acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

    struct Half {
        v4i a[TM][2], b[TN][2];
    };
    auto read = [&](int in_a, int in_b, int s, Half& f) {
        const uint8_t* la = lds + in_a * BM * kQ8Block + (wm + r) * kQ8Block;
        const uint8_t* lb = lds + kAt + in_b * BN * kQ8Block + (wn + r) * kQ8Block;
        const int u0 = ((4 * s + 2 * h) ^ (r >> 1 & 7)) * 16, u1 = ((4 * s + 2 * h + 1) ^ (r >> 1 & 7)) * 16;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            f.b[j][0] = *reinterpret_cast<const v4i*>(lb + j * 32 * kQ8Block + u0);
            f.b[j][1] = *reinterpret_cast<const v4i*>(lb + j * 32 * kQ8Block + u1);
        }
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            f.a[i][0] = *reinterpret_cast<const v4i*>(la + i * 32 * kQ8Block + u0);
            f.a[i][1] = *reinterpret_cast<const v4i*>(la + i * 32 * kQ8Block + u1);
        }
    };
    // with byte `at` of the scale words
    auto multiply = [&](const Half& f, auto at) {
        constexpr int kByte = decltype(at)::value;
        if constexpr (F8) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    const v8i x = __builtin_shufflevector(f.a[i][0], f.a[i][1], 0, 1, 2, 3, 4, 5, 6, 7);
                    const v8i y = __builtin_shufflevector(f.b[j][0], f.b[j][1], 0, 1, 2, 3, 4, 5, 6, 7);
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(y, x, acc[i][j], 0, 0, kByte, (int)sb[j], kByte,
                                                                                (int)sa[i]);
                }
        } else {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                v8b y[TN][2];
#pragma unroll
                for (int j = 0; j < TN; ++j) widen(f.b[j][u], scale_of(sb[j] >> (8 * kByte)), y[j][0], y[j][1]);
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    v8b x[2];
                    widen(f.a[i][u], scale_of(sa[i] >> (8 * kByte)), x[0], x[1]);
#pragma unroll
                    for (int q = 0; q < 2; ++q)
#pragma unroll
                        for (int j = 0; j < TN; ++j)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(y[j][q], x[q], acc[i][j], 0, 0, 0);
                }
            }
        }
    };

    Half x, y;
    constexpr int kMfma = TM * TN * (F8 ? 1 : 4), kReads = 2 * (TM + TN), kScales = TM + TN;
    int in_a = 0, in_b = 0;  // stages of block k
    // Block k, its two halves, with byte `at` of the scale words; `ahead` > 0: the words of block k + ahead are loaded (a
    // row's each from a line of its own, so not more often than needed: with every block they took a quarter of the time).
    // Without branches, so that the order given here can be kept.
    uint32_t na[TM], nb[TN];
    auto step = [&](int k, auto at, auto ahead) {
        constexpr int kAt = decltype(at)::value, kAhead = decltype(ahead)::value;
        // what may be under way when block k + 1 has to be in LDS: the loads of D - 1 blocks of A and D - 2 of B, and the
        // scales' where one of those steps began with them
        constexpr bool kTold = kAhead > 0 || kAt <= D - 2;
        constexpr int kBehind = (D - 1) * LA + (D - 2) * LB + (kTold ? kScales : 0);
        static_assert(kBehind < 64, "six bits");
        const int next_a = in_a == D ? 0 : in_a + 1, next_b = in_b == D - 1 ? 0 : in_b + 1;
        if constexpr (kAhead > 0) scales(k + kAhead, na, nb);  // first: who waits for them waits for what went out before
        __builtin_amdgcn_sched_barrier(0);
        read(in_a, in_b, 1, y);
        load_a(k + D, in_a == 0 ? D : in_a - 1);  // where block k - 1 was
        multiply(x, at);
        weave<kReadLds, kReads, kMfma / 2>();
        weave<kLoad, LA, kMfma / 2>();
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kBehind) : "memory");
        meet();  // block k + 1 is in LDS, block k is read
        __builtin_amdgcn_sched_barrier(0);
        load_b(k + D, in_b);
        read(next_a, next_b, 0, x);  // of a block behind the last: zeros, not used
        multiply(y, at);
        weave<kLoad, LB, kMfma / 2>();
        weave<kReadLds, kReads, kMfma / 2>();
        __builtin_amdgcn_sched_barrier(0);
        in_a = next_a;
        in_b = next_b;
    };
    constexpr std::integral_constant<int, 0> c0{};
    constexpr std::integral_constant<int, 1> c1{};
    constexpr std::integral_constant<int, 2> c2{};
    constexpr std::integral_constant<int, 3> c3{};
    constexpr std::integral_constant<int, 4> c4{};
    scales(0, sa, sb);  // k0 is a multiple of four
#pragma unroll
    for (int d = 0; d < D; ++d) {
        load_a(d, d);
        load_b(d, d);
    }
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((D - 1) * (LA + LB)) : "memory");  // block 0's loads
    meet();
#pragma unroll
    for (int i = 0; i < TM; ++i) asm volatile("" : "+v"(sa[i]));  // waited for here, not in the loop
#pragma unroll
    for (int j = 0; j < TN; ++j) asm volatile("" : "+v"(sb[j]));
    read(0, 0, 0, x);
    int k = 0;
    for (; k + 4 <= steps; k += 4) {
        step(k, c0, c4);
        step(k + 1, c1, c0);
        step(k + 2, c2, c0);
        step(k + 3, c3, c0);
#pragma unroll
        for (int i = 0; i < TM; ++i) sa[i] = na[i];
#pragma unroll
        for (int j = 0; j < TN; ++j) sb[j] = nb[j];
    }
    for (; k < steps; ++k) {
        step(k, c0, c1);
        const int down = 8 * ((k + 1) & 3);
#pragma unroll
        for (int i = 0; i < TM; ++i) sa[i] = na[i] >> down;
#pragma unroll
        for (int j = 0; j < TN; ++j) sb[j] = nb[j] >> down;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // nothing writes to LDS any more
    meet();

    const bool whole = gridDim.y == 1;
    void* const C = whole ? a.C : (void*)((float*)a.C + (int64_t)blockIdx.y * a.M * a.N);
    v4f* const strip = reinterpret_cast<v4f*>(lds + wave * kStrip);
    constexpr int Q = TN * 8;  // quads of a row
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                strip[r * Q + ((8 * j + 2 * g + h) ^ (r & (Q - 1)))] =
                    v4f{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this wave's own strip
        const int n = n0 + wn + lane % Q * 4;
#pragma unroll 4
        for (int p = 0; p < Q / 2; ++p) {  // 64 / Q rows at a time
            const int d = p * (64 / Q) + lane / Q, m = m0 + wm + 32 * i + d;
            const v4f v = strip[d * Q + (lane % Q ^ (d & (Q - 1)))];
            if (m < a.M && n < a.N) store4(a, C, m, n, v, whole);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

// Few rows: 16 columns of C a workgroup, its WK waves sharing the depth, the
// operands from memory to registers (a row's block of 128 is one line, read by
// four lanes), 16 MT rows of A.  Bound by the bytes of B: one row 4096 -> 4096 6
// us, of which 3.5 are the bytes and 2 the launch; 16384 -> 4096 20 us (3.4 TB/s).
// A wave takes four blocks in a row, whose scales are one word (byte by byte, for
// every fourth block, 32 rows took 35 us, so 28).  The waves' sums meet in LDS in
// wave order.
template <int MT, int WK>
__global__ __launch_bounds__(64 * WK) void mm8_rows(MmArgs a)
{
    __shared__ v4f red[WK > 1 ? WK - 1 : 1][MT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int n0 = (int)(blockIdx.x % a.nblocks) * 16, m0 = (int)(blockIdx.x / a.nblocks) * 16 * MT;
    const int k0 = (int)blockIdx.y * a.chunk, k1 = min(a.K, k0 + a.chunk);
    const int nr = min(n0 + r, a.N - 1);
    const uint8_t* pb = a.B + (int64_t)nr * a.kp + g * 32;
    const uint8_t* qb = a.sb + (int64_t)(nr >> a.bshift) * a.sp;
    const uint8_t *pa[MT], *qa[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int mr = min(m0 + 16 * i + r, a.M - 1);
        pa[i] = a.A + (int64_t)mr * a.kp + g * 32;
        qa[i] = a.sa + (int64_t)(mr >> a.ashift) * a.sp;
    }
    v4f acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = v4f{0.f, 0.f, 0.f, 0.f};
    // four blocks at a time, whose scales are one word of a row
    for (int kk = k0 + 4 * wave; kk < k1; kk += 4 * WK) {
        v4i b[4][2], x[4][MT][2];
        uint32_t fa[MT];
        const uint32_t fb = *reinterpret_cast<const uint32_t*>(qb + kk);
#pragma unroll
        for (int i = 0; i < MT; ++i) fa[i] = *reinterpret_cast<const uint32_t*>(qa[i] + kk);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t off = (int64_t)min(kk + u, k1 - 1) * kQ8Block;  // past the end: read again, not used
            b[u][0] = *reinterpret_cast<const v4i*>(pb + off);
            b[u][1] = *reinterpret_cast<const v4i*>(pb + off + 16);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                x[u][i][0] = *reinterpret_cast<const v4i*>(pa[i] + off);
                x[u][i][1] = *reinterpret_cast<const v4i*>(pa[i] + off + 16);
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (kk + u >= k1) break;
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                v8b y[2];
                widen(b[u][p], scale_of(fb >> (8 * u)), y[0], y[1]);
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    v8b z[2];
                    widen(x[u][i][p], scale_of(fa[i] >> (8 * u)), z[0], z[1]);
                    acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y[0], z[0], acc[i], 0, 0, 0);
                    acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y[1], z[1], acc[i], 0, 0, 0);
                }
            }
        }
    }
    if constexpr (WK > 1) {
        if (wave > 0)
#pragma unroll
            for (int i = 0; i < MT; ++i) red[wave - 1][i][lane] = acc[i];
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int w = 0; w < WK - 1; ++w)
#pragma unroll
            for (int i = 0; i < MT; ++i) acc[i] += red[w][i][lane];
    }
    const bool whole = gridDim.y == 1;
    void* C = whole ? a.C : (void*)((float*)a.C + (int64_t)blockIdx.y * a.M * a.N);
    const int n = n0 + 4 * g;
#pragma unroll
    for (int i = 0; i < MT; ++i)
        if (m0 + 16 * i + r < a.M && n < a.N) store4(a, C, m0 + 16 * i + r, n, acc[i], whole);
}

// The parts' sums, in order, and what the whole's epilogue does.  Bound by the
// parts' bytes and a launch: four parts of 128 x 4096 4.9 us.
__global__ __launch_bounds__(256) void mm8_join(MmArgs a, int parts, const float* part)
{
    const int quads = (a.N + 3) / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)a.M * quads) return;
    const int m = (int)(i / quads), n = (int)(i % quads) * 4;
    const float* p = part + (int64_t)m * a.N + n;
    const int64_t step = (int64_t)a.M * a.N;
    v4f v{0.f, 0.f, 0.f, 0.f};
    if (n + 3 < a.N) {
        // eight loads at a time: one after the other 256 parts of 100 x 10 results took 200 us
        for (int z = 0; z < parts; z += 8) {
            v4f x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[e] = z + e < parts ? (v4f)*reinterpret_cast<const Four*>(p + (z + e) * step) : v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int e = 0; e < 8; ++e) v += x[e];
        }
    } else {
        for (int z = 0; z < parts; z += 8) {
            v4f x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[i][e] = z + i < parts && n + e < a.N ? p[(z + i) * step + e] : 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) v += x[i];
        }
    }
    store4(a, a.C, m, n, v, true);
}

enum Kind { ROWS16, ROWS32, ROWS64, TILE64, TILE128, TILE256, WIDE };
// Which kernel, and in how many parts of the depth (which a second kernel adds
// up).  Figures: us on this card, float32 results unless they say otherwise.
struct Plan {
    Kind kind;
    int parts = 1, chunk;
    Plan(int64_t M, int64_t N, int K, bool bf16)
    {
        auto ceil = [](int64_t x, int64_t y) { return (x + y - 1) / y; };
        int64_t z = 1;
        if (M <= 64) {
            const int mt = M <= 16 ? 1 : M <= 32 ? 2 : 4;
            kind = mt == 1 ? ROWS16 : mt == 2 ? ROWS32 : ROWS64;
            const int64_t blocks = ceil(N, 16);
            z = std::min<int64_t>(256 / blocks, K / 64);
            // The rows' kernel reads A again for every 16 columns, 28 bytes a ns and CU; above 16 rows that soon takes
            // longer than tiles do (N 4096: 32 rows of 4096 8.7 here, 11.4 in tiles, of 16384 28.2 and 24.4; 64 rows of
            // 4096 13.5 and 12.3, of 16384 47.5 and 26.2).
            double us = 0.073 * (mt + 1) * K * (double)ceil(N, 4096);
            int64_t parts = 1;
            if (mt > 1 && tiles_us(M, N, K, bf16, ceil(N, 64), parts) < us) {
                kind = TILE64;
                z = parts;
            }
        } else {
            const int64_t wide = ceil(M, 128) * ceil(N, 64), n128 = ceil(M, 128) * ceil(N, 128), n256 = ceil(M, 256) * ceil(N, 256);
            // Rounds over the CUs in tenths of a 128 x 128 tile's time: a round of 256 x 256 holds four times the work of
            // half a round of 128 x 128 and passes one in ten faster (3840 x 3840 x 4096: 98 and 112); its first loads and
            // last stores overlap with nothing, so a depth below 2048 takes the smaller (4096 x 16384 x 128: 75 and 69;
            // 8192 x 8192 x 1024: 148 and 142; x 2048: 230 and 232).
            const int64_t rest = n128 % 512, t128 = n128 / 512 * 22 + (rest > 256 ? 22 : rest ? 13 : 0), t256 = ceil(n256, 256) * 40;
            if (wide <= 256) {
                // half the columns: twice the workgroups, for half the parts (128 x 16384 x 4096: 24.6, 35.8 as four parts
                // of 128 x 128; 128 x 4096 x 16384: 30.1 as four, 34.2 as sixteen)
                kind = WIDE;
                tiles_us(M, N, K, bf16, wide, z);
            } else if (K >= 16 && t256 <= t128) {
                kind = TILE256;
            } else {
                kind = TILE128;
            }
        }
        chunk = (int)(ceil(ceil(K, std::max<int64_t>(z, 1)), 4) * 4);
        parts = (int)ceil(K, chunk);
    }
    // `blocks` <= 256 tiles of 64 columns: the best number of parts and its time but for what is common to all.  A part's
    // block takes 0.45 us (0.3 by the 8-bit instructions, for bfloat16 results), the second kernel 4 and its
    // bytes.
    static double tiles_us(int64_t M, int64_t N, int K, bool bf16, int64_t blocks, int64_t& parts)
    {
        const double step = bf16 ? 0.3 : 0.45;
        double best = K * step * (double)((blocks + 255) / 256);
        parts = 1;
        for (int64_t z = 2; z <= 256 / blocks; ++z) {
            const double us = (double)((K + 4 * z - 1) / (4 * z) * 4) * step + 4 + (double)(z * M * N) * 8 / 4.7e6;
            if (us < best) {
                best = us;
                parts = z;
            }
        }
        return best;
    }
};

template <int BM, int BN, int WM, int WN, int D>
void tiles(MmArgs& a, const Plan& p, bool f8, const Work& w, hipStream_t st)
{
    a.mblocks = (a.M + BM - 1) / BM;
    a.nblocks = (a.N + BN - 1) / BN;
    const dim3 grid((unsigned)(((int64_t)a.mblocks * a.nblocks + 7) / 8 * 8), (unsigned)p.parts);
    if (f8)
        PSW_LAUNCH(kname("mm8_tiles", BM, BN, WM, WN, D, true), w, (mm8_tiles<BM, BN, WM, WN, D, true>), grid, dim3(64 * WM * WN), 0,
                   st, a);
    else
        PSW_LAUNCH(kname("mm8_tiles", BM, BN, WM, WN, D, false), w, (mm8_tiles<BM, BN, WM, WN, D, false>), grid,
                   dim3(64 * WM * WN), 0, st, a);
}

template <int MT, int WK>
void rows(MmArgs& a, const Plan& p, const Work& w, hipStream_t st)
{
    a.nblocks = (a.N + 15) / 16;
    const dim3 grid((unsigned)((int64_t)a.nblocks * ((a.M + 16 * MT - 1) / (16 * MT))), (unsigned)p.parts);
    PSW_LAUNCH(kname("mm8_rows", MT, WK), w, (mm8_rows<MT, WK>), grid, dim3(64 * WK), 0, st, a);
}

}  // namespace

size_t mm8_ws_bytes(int M, int N, int depth)
{
    int parts = 1;
    for (bool bf16 : {false, true}) parts = std::max(parts, Plan(M, N, (int)(q8_depth(depth) / kQ8Block), bf16).parts);
    return parts > 1 ? (size_t)parts * M * N * sizeof(float) : 0;
}

bool mm8_fits(int M, int N, int depth, int bf16)
{
    auto ceil = [](int64_t x, int64_t y) { return (x + y - 1) / y; };
    const Plan p(M, N, (int)(q8_depth(depth) / kQ8Block), bf16);
    int64_t threads = 0;
    switch (p.kind) {
    case ROWS16: threads = ceil(N, 16) * ceil(M, 16) * 512; break;
    case ROWS32: threads = ceil(N, 16) * ceil(M, 32) * 512; break;
    case ROWS64: threads = ceil(N, 16) * ceil(M, 64) * 512; break;
    case TILE64: threads = ceil(ceil(M, 64) * ceil(N, 64), 8) * 8 * 256; break;
    case WIDE: threads = ceil(ceil(M, 128) * ceil(N, 64), 8) * 8 * 256; break;
    case TILE128: threads = ceil(ceil(M, 128) * ceil(N, 128), 8) * 8 * 256; break;
    case TILE256: threads = ceil(ceil(M, 256) * ceil(N, 256), 8) * 8 * 256; break;
    }
    if (p.parts > 1) threads = std::max(threads, ceil(M * ceil(N, 4), 256) * 256);
    return threads <= kGridThreads;
}

hipError_t mm8(int M, int N, int depth, const uint8_t* A, const uint8_t* sa, bool atiles, const uint8_t* B,
               const uint8_t* sb, bool btiles, const float* bias, int relu, void* C, int bf16, int accumulate, void* ws,
               hipStream_t st)
{
    MmArgs a{};
    a.A = A; a.B = B; a.sa = sa; a.sb = sb; a.bias = bias;
    a.M = M; a.N = N; a.kp = q8_depth(depth); a.K = (int)(a.kp / kQ8Block);
    a.sp = q8_scales(depth); a.ashift = atiles ? 7 : 0; a.bshift = btiles ? 7 : 0;
    a.relu = relu; a.accumulate = accumulate; a.bf16 = bf16;
    const Plan p(M, N, a.K, bf16);
    a.chunk = p.chunk;
    const bool one = p.parts == 1;
    a.C = one ? C : ws;
    const Work w{2.0 * M * N * depth, ((double)M + N) * a.kp + (one && bf16 ? 2.0 : 4.0) * M * N * p.parts};
    switch (p.kind) {
    case ROWS16: rows<1, 8>(a, p, w, st); break;
    case ROWS32: rows<2, 8>(a, p, w, st); break;
    case ROWS64: rows<4, 8>(a, p, w, st); break;
    case TILE64: tiles<64, 64, 2, 2, 4>(a, p, bf16 != 0, w, st); break;
    case WIDE: tiles<128, 64, 2, 2, 4>(a, p, bf16 != 0, w, st); break;
    case TILE128: tiles<128, 128, 2, 2, 2>(a, p, bf16 != 0, w, st); break;
    case TILE256: tiles<256, 256, 2, 2, 2>(a, p, bf16 != 0, w, st); break;
    }
    if (!one) {
        a.C = C;
        const int64_t n = (int64_t)M * ((N + 3) / 4);
        PSW_LAUNCH(kname("mm8_join"), (Work{(double)p.parts * M * N, kF * (p.parts + 1.0) * M * N}), mm8_join,
                   dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, a, p.parts, (const float*)ws);
    }
    return hipGetLastError();
}

}  // namespace psw
