// 8-bit operands: float32 or bfloat16 matrices as e4m3 values with a
// power-of-two scale for each block of 128 along the depth of a product.
//
// For a block with the largest finite magnitude a, the scale is 2^E with E the
// smallest integer (at least -126) that has a <= 448 * 2^E, 448 being the
// largest e4m3; x * 2^-E is then exact and rounds once, to nearest even, by the
// conversion instruction (but for numbers nearest to 2^128: below_2_128).  A
// scale that is a power of two costs no accuracy against a / 448 (a floating-point
// format's steps are relative) and is what the matrix instruction takes as an
// operand's scale.  1.75 * 2^8 = 448, so E comes from a's bits: its exponent - 8,
// and one more where its fraction is past 1.75.
//
// A product's depth runs along the rows of one operand and, in the next product,
// along the columns of the same matrix (dy in dx = dy w and dw = dy^T x), so a
// workgroup reads a 128 x 128 tile once and writes it in both orders, each with
// the scales of its own blocks; the transposed bytes turn in LDS.
#include <type_traits>

#include "internal.h"
#include "q8.h"

namespace psw {
namespace {

constexpr int kTile = 128, kThreads = 512;
constexpr int kPieces = kTile * kTile / 16 / kThreads;  // of 4 x 4, a thread
constexpr int kTurn = kTile / 4 + 1;  // words of a turned row: odd, so that neighbours start in other banks

struct QuantArgs {
    const void* x;
    int64_t ld;
    int rows, cols;
    uint8_t *q, *s, *qt, *st;
    double* colsum;    // [row tiles][cols], or null
    float* total;      // the column sums, of one row tile
    int64_t kp, rp;    // bytes of a row of q, of qt
    int sp, spt;       // bytes of a row of s, of st
    int cblocks, rblocks;
};

__device__ __forceinline__ uint32_t finite_bits(float v)
{
    const uint32_t u = __float_as_uint(v) & 0x7fffffffu;
    return u < 0x7f800000u ? u : 0u;
}

// the scale byte of a block from its largest finite magnitude's bits
__device__ __forceinline__ uint32_t scale_byte(uint32_t bits)
{
    const int e = (int)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u);
    return (uint32_t)(e < 1 ? 1 : e);
}

// four values at 2^-E, rounded to e4m3; infinities and NaN become NaN
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d, float by)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * by, b * by, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * by, d * by, w, true);
}

// Numbers from 248 * 2^120 on (the lowest of either type, as masks have it) have the largest scale, 2^120, and are nearest to
// 256 * 2^120 = 2^128, which neither float32 nor bfloat16 has: an infinity in a product, and NaN times a weight of 0.  They
// become 240 * 2^120, the number below: four rounded values of a block with that scale.
constexpr uint32_t kLargest = 247;  // its byte
__device__ __forceinline__ uint32_t below_2_128(uint32_t w)
{
    const uint32_t off = (w & 0x7f7f7f7fu) ^ 0x78787878u;    // 0 in bytes of 256
    return w - ((~(off + 0x7f7f7f7fu) & 0x80808080u) >> 7);  // one less there: no byte borrows
}

__device__ __forceinline__ float inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// Four neighbours in one load, which gfx950 takes at any element's address
// (4000 x 5003 bfloat16 one by one: 48 us, so 29).
template <typename T>
__device__ __forceinline__ float4 load4(const T* p)
{
    typedef uint32_t Words __attribute__((ext_vector_type(sizeof(T)), aligned(sizeof(T))));
    const Words u = *reinterpret_cast<const Words*>(p);
    if constexpr (sizeof(T) == 4)
        return make_float4(__uint_as_float(u[0]), __uint_as_float(u[1]), __uint_as_float(u[2]), __uint_as_float(u[3]));
    else
        return make_float4(__uint_as_float(u[0] << 16), __uint_as_float(u[0] & 0xffff0000u), __uint_as_float(u[1] << 16),
                           __uint_as_float(u[1] & 0xffff0000u));
}

// Both orders, column sums, or square blocks: a 128 x 128 tile.  A thread holds
// two pieces of 4 rows x 4 columns (32 threads side by side read 128 columns of
// a row): 512 threads a tile leave two to four tiles a CU, of which one loads
// while others turn (bfloat16 three rather than two: 8192 x 4096 35.5 us, so 34,
// and 36 with the largest scale's question; float32, whose tiles are twice the
// bytes, 41 us, with three 47).  Bound by memory: 16384 x 4096 float32, square
// blocks, 80 us (5.0 TB/s), 8192 x 4096 by rows and columns with sums 41 us (4.9
// TB/s); 2047 x 4104 so 17 us (2.9 TB/s; its 528 tiles are one round of the chip
// and 16 more).
template <typename T, bool TILES>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 6 : 4) void q8_quant_k(QuantArgs a)
{
    constexpr int W = kThreads / 64, R = 4 * kPieces, S = kTile / kPieces;  // waves, rows a thread, rows from piece to piece
    __shared__ uint32_t rowmax[kTile], colpart[W][kTile], turn[kTile * kTurn];
    __shared__ double sums[W][kTile];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l = tid & 31, rg = tid >> 5;
    const int cb = blockIdx.x % a.cblocks, rb = blockIdx.x / a.cblocks;
    const int c0 = cb * kTile + 4 * l, r0 = rb * kTile + 4 * rg;
    const T* x = (const T*)a.x + (int64_t)r0 * a.ld + c0;
    float v[R][4];
    if ((rb + 1) * kTile <= a.rows && (cb + 1) * kTile <= a.cols) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const float4 f = load4(x + (int64_t)(i / 4 * S + i % 4) * a.ld);
            v[i][0] = f.x; v[i][1] = f.y; v[i][2] = f.z; v[i][3] = f.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int r = r0 + i / 4 * S + i % 4;
            const T* p = x + (int64_t)(i / 4 * S + i % 4) * a.ld;
            if (r < a.rows && c0 + 3 < a.cols) {
                const float4 f = load4(p);
                v[i][0] = f.x; v[i][1] = f.y; v[i][2] = f.z; v[i][3] = f.w;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[i][e] = r < a.rows && c0 + e < a.cols ? (float)p[e] : 0.f;
            }
        }
    }

    if (a.colsum || a.total) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            double s = 0.0;
#pragma unroll
            for (int i = 0; i < R; ++i) s += (double)v[i][e];
            s += __shfl_xor(s, 32);
            if (lane < 32) sums[wave][4 * l + e] = s;
        }
    }

    // the largest magnitudes: of a row over 32 threads, of a column over 16
    uint32_t cm[4] = {0, 0, 0, 0}, rm[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        uint32_t u = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t f = finite_bits(v[i][e]);
            u = max(u, f);
            cm[e] = max(cm[e], f);
        }
        rm[i] = u;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) cm[e] = max(cm[e], (uint32_t)__shfl_xor((int)cm[e], 32));
    if (lane < 32) *reinterpret_cast<uint4*>(&colpart[wave][4 * l]) = make_uint4(cm[0], cm[1], cm[2], cm[3]);
    if constexpr (!TILES) {
        // half of the rows change places at every step, so that four lanes end with a row
        static_assert(R == 8, "lane bits 4, 3 and 2 choose the row");
#pragma unroll
        for (int half = R / 2; half >= 1; half /= 2) {
            const bool up = lane & (4 * half);
#pragma unroll
            for (int i = 0; i < half; ++i) {
                const uint32_t mine = up ? rm[i + half] : rm[i], theirs = up ? rm[i] : rm[i + half];
                rm[i] = max(mine, (uint32_t)__shfl_xor((int)theirs, 4 * half));
            }
        }
        rm[0] = max(rm[0], (uint32_t)__shfl_xor((int)rm[0], 2));
        rm[0] = max(rm[0], (uint32_t)__shfl_xor((int)rm[0], 1));
        const int i = l >> 2;
        if (!(l & 3)) rowmax[4 * rg + i / 4 * S + i % 4] = rm[0];
    }
    __syncthreads();

    uint32_t ce[4];  // scale bytes of the thread's columns
    {
        uint4 t = *reinterpret_cast<const uint4*>(&colpart[0][4 * l]);
#pragma unroll
        for (int w = 1; w < W; ++w) {
            const uint4 o = *reinterpret_cast<const uint4*>(&colpart[w][4 * l]);
            t = make_uint4(max(t.x, o.x), max(t.y, o.y), max(t.z, o.z), max(t.w, o.w));
        }
        if constexpr (TILES) {
            uint32_t u = max(max(t.x, t.y), max(t.z, t.w));
#pragma unroll
            for (int d = 1; d < 32; d *= 2) u = max(u, (uint32_t)__shfl_xor((int)u, d));
            t = make_uint4(u, u, u, u);
        }
        ce[0] = scale_byte(t.x); ce[1] = scale_byte(t.y); ce[2] = scale_byte(t.z); ce[3] = scale_byte(t.w);
    }

    // some block of the tile, whose columns are all in every wave, has the largest scale
    const bool far = __any(max(max(ce[0], ce[1]), max(ce[2], ce[3])) == kLargest);
    if (a.q) {
        uint8_t* q = a.q + (int64_t)r0 * a.kp + c0;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int down = i / 4 * S + i % 4;
            const float by = inverse(TILES ? ce[0] : scale_byte(rowmax[4 * rg + down]));
            if (r0 + down < a.rows)
                *reinterpret_cast<uint32_t*>(q + (int64_t)down * a.kp) = pack4(v[i][0], v[i][1], v[i][2], v[i][3], by);
        }
        if (TILES ? tid == 0 : tid < kTile && rb * kTile + tid < a.rows) {
            uint8_t* p = a.s + (int64_t)(TILES ? rb : rb * kTile + tid) * a.sp;
            p[cb] = (uint8_t)(TILES ? ce[0] : scale_byte(rowmax[tid]));
            if (cb == a.cblocks - 1)
                for (int i = a.cblocks; i < a.sp; ++i) p[i] = 127;
        }
    }
    if (a.qt) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float by = inverse(ce[e]);
#pragma unroll
            for (int i = 0; i < R; i += 4)
                turn[(4 * l + e) * kTurn + i / 4 * (S / 4) + rg] = pack4(v[i][e], v[i + 1][e], v[i + 2][e], v[i + 3][e], by);
        }
        if (TILES ? tid == 0 : rg == 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (TILES ? e > 0 : c0 + e >= a.cols) break;
                uint8_t* p = a.st + (int64_t)(TILES ? cb : c0 + e) * a.spt;
                p[rb] = (uint8_t)ce[e];
                if (rb == a.rblocks - 1)
                    for (int i = a.rblocks; i < a.spt; ++i) p[i] = 127;
            }
        }
        __syncthreads();
#pragma unroll 4
        for (int c = rg; c < kTile; c += kThreads / 32)
            if (cb * kTile + c < a.cols)
                *reinterpret_cast<uint32_t*>(a.qt + (int64_t)(cb * kTile + c) * a.rp + rb * kTile + 4 * l) =
                    turn[c * kTurn + l];
    }
    if ((a.colsum || a.total) && tid < kTile && cb * kTile + tid < a.cols) {
        double s = sums[0][tid];
#pragma unroll
        for (int w = 1; w < W; ++w) s += sums[w][tid];
        if (a.colsum)
            a.colsum[(int64_t)rb * a.cols + cb * kTile + tid] = s;
        else
            a.total[cb * kTile + tid] = (float)s;
    }
    // Every thread's own words again, from memory: a look at each word's scale as it is made took 5% to 10% of the time, the
    // numbers changed before registers that bfloat16 has not (8192 x 4096 35 us, so 58).
    if (far) {
#pragma unroll 1
        for (int i = 0; a.q && i < R; ++i) {
            const int r = 4 * rg + i / 4 * S + i % 4;
            uint32_t* p = reinterpret_cast<uint32_t*>(a.q + (int64_t)(rb * kTile + r) * a.kp + c0);
            if (rb * kTile + r < a.rows && (TILES || scale_byte(rowmax[r]) == kLargest)) *p = below_2_128(*p);
        }
#pragma unroll 1
        for (int c = rg; a.qt && c < kTile; c += kThreads / 32) {
            uint32_t top = 0;
            for (int w = 0; w < W; ++w) top = max(top, colpart[w][c]);
            uint32_t* p = reinterpret_cast<uint32_t*>(a.qt + (int64_t)(cb * kTile + c) * a.rp + rb * kTile + 4 * l);
            if (cb * kTile + c < a.cols && (TILES || scale_byte(top) == kLargest)) *p = below_2_128(*p);
        }
    }
}

// Rows alone (a forward pass): sixteen lanes a block of 128, eight values each,
// so that small batches too give every CU work.  8192 x 4096 bfloat16 25 us (4.0
// TB/s), 128 x 16384 float32 4.2-5 us.
template <typename T>
__global__ __launch_bounds__(256) void q8_rows_k(QuantArgs a)
{
    constexpr int U = 2;  // blocks a thread
    const int l = threadIdx.x & 15;
    // units: blocks of a row, the empty ones of its last scale word included; the workgroup's first one's place
    const int64_t first = (int64_t)blockIdx.x * (16 * U);
    const int r0 = first < INT32_MAX ? (int)((uint32_t)first / (uint32_t)a.sp) : (int)(first / a.sp);
    const int b0 = (int)(first - (int64_t)r0 * a.sp);
    float v[U][8];
    int64_t row[U];
    int cb[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
        row[k] = r0;
        cb[k] = b0 + 16 * k + (threadIdx.x >> 4);
        while (cb[k] >= a.sp) {  // at most eight times: a row has four units or more
            cb[k] -= a.sp;
            ++row[k];
        }
        const int c = cb[k] * kTile + 8 * l;
        const T* p = (const T*)a.x + row[k] * a.ld + c;
        if (row[k] < a.rows && c + 7 < a.cols) {
            const float4 f = load4(p), g = load4(p + 4);
            v[k][0] = f.x; v[k][1] = f.y; v[k][2] = f.z; v[k][3] = f.w;
            v[k][4] = g.x; v[k][5] = g.y; v[k][6] = g.z; v[k][7] = g.w;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[k][e] = row[k] < a.rows && c + e < a.cols ? (float)p[e] : 0.f;
        }
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, finite_bits(v[k][e]));
#pragma unroll
        for (int d = 1; d < 16; d *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, d));
        if (row[k] >= a.rows) continue;
        const uint32_t e = scale_byte(m);
        const float by = inverse(e);
        if (cb[k] < a.cblocks) {
            uint2 w = make_uint2(pack4(v[k][0], v[k][1], v[k][2], v[k][3], by), pack4(v[k][4], v[k][5], v[k][6], v[k][7], by));
            if (e == kLargest) w = make_uint2(below_2_128(w.x), below_2_128(w.y));
            *reinterpret_cast<uint2*>(a.q + row[k] * a.kp + cb[k] * kTile + 8 * l) = w;
        }
        if (l == 0) a.s[row[k] * a.sp + cb[k]] = (uint8_t)(cb[k] < a.cblocks ? e : 127u);
    }
}

// the column sums of the row tiles, in order, in 64 bits (as all of a column's are): a launch of 4 us, a few
// loads of latency
__global__ __launch_bounds__(256) void q8_colsum_k(int parts, int cols, const double* part, float* out)
{
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= cols) return;
    double s = 0.0;
    int p = 0;
    for (; p + 8 <= parts; p += 8) {
        double v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = part[(int64_t)(p + i) * cols + c];
#pragma unroll
        for (int i = 0; i < 8; ++i) s += v[i];
    }
    for (; p < parts; ++p) s += part[(int64_t)p * cols + c];
    out[c] = (float)s;
}

template <typename T>
void launch(const QuantArgs& a, bool tiles, const Work& w, hipStream_t st)
{
    const dim3 grid((unsigned)((int64_t)a.cblocks * a.rblocks));
    if (tiles)
        PSW_LAUNCH(kname("q8_quant_k", (int)sizeof(T), true), w, (q8_quant_k<T, true>), grid, dim3(kThreads), 0, st, a);
    else
        PSW_LAUNCH(kname("q8_quant_k", (int)sizeof(T), false), w, (q8_quant_k<T, false>), grid, dim3(kThreads), 0, st, a);
}

}  // namespace

size_t q8_quant_ws_bytes(int rows, int cols)
{
    const int64_t parts = ((int64_t)rows + kTile - 1) / kTile;
    return parts > 1 ? (size_t)parts * cols * sizeof(double) : 0;
}

bool q8_quant_fits(int rows, int cols, bool rows_alone)
{
    if (rows_alone) return ((int64_t)rows * q8_scales(cols) + 31) / 32 * 256 <= kGridThreads;
    return q8_depth(cols) / kTile * (q8_depth(rows) / kTile) <= kGridThreads / kThreads;
}

hipError_t q8_quant(int rows, int cols, int bf16, const void* x, int64_t ld, bool tiles, uint8_t* q, uint8_t* s,
                    uint8_t* qt, uint8_t* stp, float* colsum, void* ws, hipStream_t st)
{
    QuantArgs a{};
    a.x = x; a.ld = ld; a.rows = rows; a.cols = cols;
    a.q = q; a.s = s; a.qt = qt; a.st = stp;
    a.kp = q8_depth(cols); a.rp = q8_depth(rows);
    a.sp = q8_scales(cols); a.spt = q8_scales(rows);
    a.cblocks = (int)(a.kp / kTile); a.rblocks = (int)(a.rp / kTile);
    const int size = bf16 ? 2 : 4;
    a.colsum = colsum && a.rblocks > 1 ? (double*)ws : nullptr;
    a.total = colsum && a.rblocks == 1 ? colsum : nullptr;
    const double n = (double)rows * cols;
    const Work w{2 * n, size * n + (q ? n : 0.0) + (qt ? n : 0.0)};
    if (!tiles && !qt && !colsum) {
        const dim3 grid((unsigned)(((int64_t)rows * a.sp + 31) / 32));
        if (bf16)
            PSW_LAUNCH(kname("q8_rows_k", size), w, (q8_rows_k<__bf16>), grid, dim3(256), 0, st, a);
        else
            PSW_LAUNCH(kname("q8_rows_k", size), w, (q8_rows_k<float>), grid, dim3(256), 0, st, a);
    } else if (bf16) {
        launch<__bf16>(a, tiles, w, st);
    } else {
        launch<float>(a, tiles, w, st);
    }
    if (colsum && a.rblocks > 1)
        PSW_LAUNCH(kname("q8_colsum_k"), (Work{(double)a.rblocks * cols, (8.0 * a.rblocks + kF) * cols}), q8_colsum_k,
                   dim3((unsigned)((cols + 255) / 256)), dim3(256), 0, st, a.rblocks, cols, (const double*)ws, colsum);
    return hipGetLastError();
}

}  // namespace psw
