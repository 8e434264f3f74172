// The loss of a student over a teacher's top logits, and its gradient
// (psw_distill in include/psw.h has the formulas).
//
// A workgroup holds its row of logits in registers, so that memory sees each
// logit once and each gradient once: the largest logit, the sums of
// exponentials, then the gradient, all from there.  Rows past 128 KB are cut into
// pieces of 8 or 32 KB, whose maxima and sums (`distill_k` in its second form) the
// gradient's workgroups (third form), which read the logits again, put together
// in order: 1024 rows of 100000 bfloat16 63 + 84 us.
//
// What the teacher says about the rest of the classes is a probability, r, for
// all of them together; the student's probability of the rest, R, is summed
// from the rest's own exponentials, relative to the rest's own largest logit
// (one minus the members' probabilities would leave nothing of a small R).  A
// bit for each element in LDS marks the members, which turn to -inf in the
// registers before the first pass, so that every pass is one over the rest; a
// member's and the label's parts are formed by a thread each, in 64 bits where
// they are summed, and their gradients written over the rest's after a barrier.
//
// In bfloat16 the exponentials bound it: a logit takes one in the sums and one in
// the gradient, and two each where a label's softmax has another temperature.
// That one is a power of the first where the temperature is 2 or 4, and an
// exponential's argument one fused multiply-add, x k - b with b the rounded
// product of the largest logit and k; what the rounding of b makes of all terms
// alike is taken back from the sums (`corr`).  A row whose b is past kFar has the
// largest logit taken from all others first: what that rounds is so far below
// that its exponential is 0.
//
// 4096 rows of 32000 bfloat16, 64 entries and a label, take 110 us for 524 MB (4.76
// TB/s, what a large copy reaches), rows of 50257 246 us for 823 MB (3.3 TB/s: 16
// chunks a thread leave one workgroup a CU, since room for two spills and takes
// 332 us), 2048 rows of 30000 float32 127 us (3.9 TB/s).  128 rows of 1000 are a
// chain of latencies, 5.4 us.  64-bit arithmetic is kept to sums, differences and
// the exponentials that leave r: its library logarithms and quotients took 122 us
// of the first and 6.9 of the last.
#include <math.h>

#include "distill.h"
#include "internal.h"
#include "rows.h"

namespace psw {
namespace {

constexpr int kMost = 256;        // entries of a teacher's row
constexpr int kTable = 2 * kMost; // slots of the table that finds an index given twice
constexpr float kLog2e = 1.4426950408889634f;

struct DistillArgs {
    const void* z;
    void* d;  // null: the loss only
    int64_t ld, ldd;
    int n, classes, k;
    const int32_t* idx;
    const float *val, *lse, *weight;
    const int32_t* labels;
    float tau, alpha, each;  // each: a row's weight where none are given
    double inv_tau;
    float kt;                // log2(e) / tau
    float* row_loss;
    int splits, per;         // pieces of a row, chunks of a piece
    float* part;             // [n][splits][4]: the rest's largest, its sums of exponentials at both temperatures
    float* zk;               // [n][k + 1]: the members' logits, the label's
};

enum Form { WHOLE, PIECE, GRADIENT };
// The label's softmax beside the teacher's: none or the same one, an exponential of its own, the square or the fourth
// power of the teacher's.
enum Beside { SAME, OWN, SQUARE, FOURTH };

// waves a SIMD that the registers are to leave room for: rows of 16 chunks a thread do not fit twice
constexpr int waves_of(int t, int nv) { return nv == 16 ? 2 : 4; }

__device__ __forceinline__ double over(double x) { return (double)__builtin_amdgcn_rcpf((float)x); }

// KI: entries a thread.
template <typename E, int T, int NV, bool TAIL, int FORM, int KI>
__global__ __launch_bounds__(T, waves_of(T, NV)) void distill_k(DistillArgs a)
{
    constexpr int P = Row<E>::kPer, W = T / 64;
    __shared__ float shf[3][W], sht[2][W];
    __shared__ double shd[3][W], shl[W];
    __shared__ int tidx[kMost], table[kTable], twice, among;
    __shared__ double tp[kMost];
    __shared__ uint32_t bits[TAIL ? T * NV / 4 : 1];  // a byte for each chunk
    const int tid = threadIdx.x;
    if (FORM == GRADIENT && !a.d && blockIdx.x % a.splits) return;  // the loss is the first piece's
    const int row = FORM == WHOLE ? blockIdx.x : blockIdx.x / a.splits, piece = FORM == WHOLE ? 0 : blockIdx.x % a.splits;
    const float weight = a.weight ? a.weight[row] : a.each;
    const Row<E> z((const E*)a.z + (int64_t)row * a.ld, a.classes);
    const int c0 = FORM == WHOLE ? 0 : piece * a.per, c1 = FORM == WHOLE ? z.chunks : min(z.chunks, c0 + a.per);
    E* const d = (E*)a.d + (int64_t)row * a.ldd;
    const bool even = (int)((uintptr_t)d % 16 / sizeof(E)) == z.shift;  // chunks of d are chunks of z

    const int lo = z.lo(c0), hi = z.hi(c1), es = z.single(c0, c1);
    auto store = [&](int c, const float (&g)[P]) {
        const int e0 = z.first(c);
        if (even) {
            Chunk w;
            if constexpr (sizeof(E) == 4) {
#pragma unroll
                for (int j = 0; j < P; ++j) w[j] = __float_as_uint(g[j]);
            } else {
                typedef __bf16 v2b __attribute__((ext_vector_type(2)));
#pragma unroll
                for (int j = 0; j < P / 2; ++j)
                    w[j] = __builtin_bit_cast(uint32_t, v2b{(__bf16)g[2 * j], (__bf16)g[2 * j + 1]});
            }
            *reinterpret_cast<Chunk*>(d + e0) = w;
            return;
        }
#pragma unroll
        for (int j = 0; j < P; ++j) d[e0 + j] = (E)g[j];
    };

    if (weight == 0.f) {  // nothing of the row is looked at
        if (FORM != PIECE) {
            if (piece == 0 && tid == 0) a.row_loss[row] = 0.f;
            if (a.d) {
                const float g[P] = {};
                for (int c = lo + tid; c < hi; c += T) store(c, g);
                if (es >= 0) d[es] = (E)0.f;
            }
        }
        return;
    }

    Chunk v[NV];
    z.template load<T>(v, c0, lo, FORM == GRADIENT && !a.d ? lo : hi);
    float xs = es >= 0 ? (float)z.p[es] : -INFINITY;

    // the teacher's entries, up to KI a thread; none where the loss is the label's (0 times an infinite loss is NaN)
    const int label = a.labels ? a.labels[row] : -1;
    const bool has = a.alpha != 0.f && label >= 0 && label < a.classes;
    int idx[KI];
    float val[KI], zk[KI], zlabel = 0.f;
    float* const kept = a.zk + (int64_t)row * (a.k + 1);
#pragma unroll
    for (int i = 0; i < KI; ++i) {
        const int k = tid + i * T;
        idx[i] = -1;
        val[i] = -INFINITY;
        zk[i] = -INFINITY;
        if (k < a.k) {
            const int e = a.idx[(int64_t)row * a.k + k];
            val[i] = a.val[(int64_t)row * a.k + k];
            if (e >= 0 && e < a.classes && !(val[i] == -INFINITY) && a.alpha != 1.f) {
                idx[i] = e;
                zk[i] = FORM == GRADIENT ? kept[k] : (float)z.p[e];
                if (FORM == PIECE && piece == 0) kept[k] = zk[i];
            } else {
                val[i] = -INFINITY;
            }
        }
    }
    if (has) zlabel = FORM == GRADIENT ? kept[a.k] : (float)z.p[label];
    if (FORM == PIECE && piece == 0 && tid == 0) kept[a.k] = zlabel;

    if constexpr (TAIL) {
        for (int i = tid; i < T * NV / 4; i += T) bits[i] = 0;
    }
    if constexpr (FORM != PIECE) {
        for (int i = tid; i < kTable; i += T) table[i] = -1;
        if (tid == 0) twice = among = 0;
    }
    __syncthreads();
    if constexpr (TAIL) {
#pragma unroll
        for (int i = 0; i < KI; ++i) {
            const int e = idx[i] + z.shift - c0 * P;  // from the piece's first chunk
            if (idx[i] >= 0 && e >= 0 && e < (c1 - c0) * P) atomicOr(&bits[e / P / 4], 1u << (e / P % 4 * 8 + e % P));
        }
    }
    if constexpr (FORM != PIECE) {
#pragma unroll
        for (int i = 0; i < KI; ++i)
            if (idx[i] >= 0) {
                int slot = idx[i] & (kTable - 1), old;
                while ((old = atomicCAS(&table[slot], -1, idx[i])) != -1 && old != idx[i]) slot = (slot + 1) & (kTable - 1);
                if (old == idx[i]) twice = 1;
                if (idx[i] == label) among = 1;
            }
    }
    // Element j of chunk i.  Before each pass `half` turns opaque, so that the floats of bfloat16 pairs are formed anew:
    // kept, they would take twice the row's registers.
    int half = 16;
    auto at = [&](int i, int j) {
        if constexpr (sizeof(E) == 4) return __uint_as_float(v[i][j]);
        return __uint_as_float(j & 1 ? v[i][j / 2] >> half << half : v[i][j / 2] << half);
    };
    const auto larger = [](float x, float y) { return fmaxf(x, y); };
    const auto add = [](auto x, auto y) { return x + y; };
    const int lane = tid & 63, wave = tid >> 6;
    const bool holds = wave * 64 < a.k;  // this wave has entries

    // the rest's largest logit (without TAIL, all classes are the rest) and sums of exponentials, relative to it
    if constexpr (TAIL) {
        __syncthreads();
        const uint8_t* const members = reinterpret_cast<const uint8_t*>(bits);
        if (es >= 0 && members[(es + z.shift) / P - c0] >> (es + z.shift) % P & 1) xs = -INFINITY;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t m = members[i * T + tid];
            if (m) {
                const Chunk gone = Row<E>::none();
                if constexpr (sizeof(E) == 4) {
#pragma unroll
                    for (int j = 0; j < P; ++j) v[i][j] = m >> j & 1 ? gone[j] : v[i][j];
                } else {
#pragma unroll
                    for (int j = 0; j < P / 2; ++j) {
                        const uint32_t two = m >> (2 * j), mask = (two & 1 ? 0xffffu : 0u) | (two & 2 ? 0xffff0000u : 0u);
                        v[i][j] = (v[i][j] & ~mask) | (gone[j] & mask);
                    }
                }
            }
        }
    }
    const float kt = a.kt;
    const int beside = !has || a.tau == 1.f ? SAME : a.tau == 2.f ? SQUARE : a.tau == 4.f ? FOURTH : OWN;
    // the largest logit of the rest, of all classes, and the teacher's largest, in one exchange
    float mt = -INFINITY, mall = -INFINITY, most = -INFINITY;
    if constexpr (FORM != GRADIENT) {
        mt = xs;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (c0 + i * T < hi)
#pragma unroll
                for (int j = 0; j < P; ++j) mt = fmaxf(mt, at(i, j));
    } else {
        const float4* q = reinterpret_cast<const float4*>(a.part) + (int64_t)row * a.splits;
        for (int s = tid; s < a.splits; s += T) mt = fmaxf(mt, q[s].x);
    }
    if (holds) {
#pragma unroll
        for (int i = 0; i < KI; ++i) {
            if constexpr (TAIL)
                mall = fmaxf(mall, zk[i]);
            else
                most = fmaxf(most, val[i]);
        }
    }
    mt = wave_reduce(mt, larger);
    if (holds) {
        mall = wave_reduce(mall, larger);
        most = wave_reduce(most, larger);
    }
    if constexpr (T > 64) {
        if (lane == 0) {
            shf[0][wave] = mt;
            shf[1][wave] = mall;
            shf[2][wave] = most;
        }
        __syncthreads();  // the table, `twice` and `among` are whole too
        mt = shf[0][0];
        mall = shf[1][0];
        most = shf[2][0];
#pragma unroll
        for (int w = 1; w < W; ++w) {
            mt = fmaxf(mt, shf[0][w]);
            mall = fmaxf(mall, shf[1][w]);
            most = fmaxf(most, shf[2][w]);
        }
    } else {
        __syncthreads();
    }
    mall = fmaxf(mall, mt);
    float ref = mt == -INFINITY ? 0.f : mt;
    if (fabsf(mt) * fmaxf(kt, kLog2e) > kFar && fabsf(mt) < INFINITY) {
        xs -= mt;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < P; ++j) {
                const E y = (E)(element<E>(v[i], j) - mt);
                if constexpr (sizeof(E) == 4)
                    v[i][j] = __float_as_uint(y);
                else
                    v[i][j / 2] = j & 1 ? (v[i][j / 2] & 0xffffu) | (uint32_t)__builtin_bit_cast(uint16_t, y) << 16
                                        : (v[i][j / 2] & 0xffff0000u) | __builtin_bit_cast(uint16_t, y);
            }
        ref = 0.f;
    }
    const float b = ref * kt, b1 = ref * kLog2e;
    // what the terms 2^(x kt - b) of the rest are to be multiplied by, and the label's: 2^(b - ref kt), which is 1 but for
    // the rounding of b
    const float corr = __builtin_amdgcn_exp2f(-fmaf(ref, kt, -b));
    const float corr1 = beside == OWN ? __builtin_amdgcn_exp2f(-fmaf(ref, kLog2e, -b1))
                                      : beside == SAME ? 1.f : beside == SQUARE ? corr * corr : (corr * corr) * (corr * corr);
    // the exponential at the teacher's temperature, and the label's
    auto both = [&](float x, auto kind, float& e, float& e1) {
        constexpr int K = decltype(kind)::value;
        e = __builtin_amdgcn_exp2f(fmaf(x, kt, -b));
        if constexpr (K == SAME) e1 = 0.f;
        if constexpr (K == OWN) e1 = __builtin_amdgcn_exp2f(fmaf(x, kLog2e, -b1));
        if constexpr (K == SQUARE) e1 = e * e;
        if constexpr (K == FOURTH) e1 = (e * e) * (e * e);
    };
    auto by_kind = [&](auto f) {
        if (beside == SAME)
            f(std::integral_constant<int, SAME>{});
        else if (beside == OWN)
            f(std::integral_constant<int, OWN>{});
        else if (beside == SQUARE)
            f(std::integral_constant<int, SQUARE>{});
        else
            f(std::integral_constant<int, FOURTH>{});
    };
    // The sums, in one exchange: of the rest's exponentials, and in 64 bits of the teacher's probabilities (what they
    // leave is a small difference) and the members' exponentials.
    float st = 0.f, s1 = 0.f;
    if constexpr (FORM != GRADIENT) {
        by_kind([&](auto kind) {
            asm volatile("" : "+s"(half));
            both(xs, kind, st, s1);
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (c0 + i * T < hi) {
#pragma unroll
                    for (int j = 0; j < P; ++j) {
                        float e, e1 = 0.f;
                        both(at(i, j), kind, e, e1);
                        st += e;
                        if constexpr (decltype(kind)::value != SAME) s1 += e1;
                    }
                    __builtin_amdgcn_sched_barrier(0);  // chunk after chunk: no registers for many at once
                }
        });
        st *= corr;
        s1 *= corr1;
    } else {
        // of the pieces; one without a logit above -inf adds nothing (or a NaN)
        const float4* q = reinterpret_cast<const float4*>(a.part) + (int64_t)row * a.splits;
        for (int s = tid; s < a.splits; s += T) {
            const float4 f = q[s];
            const float down = f.x == mt ? 0.f : f.x - mt;
            st += f.x == -INFINITY ? f.y : f.y * __builtin_amdgcn_exp2f(down * kt);
            s1 += f.x == -INFINITY ? f.z : f.z * __builtin_amdgcn_exp2f(down * kLog2e);
        }
    }
    st = wave_reduce(st, add);
    if (beside != SAME) s1 = wave_reduce(s1, add);

    const double inv_tau = a.inv_tau;
    auto soft_exp = [&](float x) { return __builtin_amdgcn_exp2f((x - mall) * kt); };
    auto hard_exp = [&](float x) { return __builtin_amdgcn_exp2f((x - mall) * kLog2e); };
    double p[KI], logp[KI], sum = 0.0, members = 0.0, members1 = 0.0;
    bool lead[KI];          // the first of equal indices
    float eq[KI], eq1[KI];  // exponentials of this thread's members
#pragma unroll
    for (int i = 0; i < KI; ++i) {
        lead[i] = idx[i] >= 0;
        p[i] = logp[i] = 0.0;
        eq[i] = eq1[i] = 0.f;
    }
    if (FORM != PIECE && holds) {
        const double l = TAIL ? (double)a.lse[row] : 0.0;
#pragma unroll
        for (int i = 0; i < KI; ++i)
            if (lead[i]) {
                // in 64 bits where r is what they leave of 1
                logp[i] = TAIL ? (double)val[i] * inv_tau - l : ((double)val[i] - (double)most) * inv_tau;
                p[i] = TAIL ? exp(logp[i]) : (double)__builtin_amdgcn_exp2f((float)logp[i] * kLog2e);
                sum += p[i];
            }
    }
    if constexpr (FORM != PIECE)
        if (twice) {
#pragma unroll
            for (int i = 0; i < KI; ++i)
                if (tid + i * T < kMost) {
                    tidx[tid + i * T] = idx[i];
                    tp[tid + i * T] = p[i];
                }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < KI; ++i)
                if (lead[i]) {
                    double same = 0.0;
                    for (int k = 0; k < a.k; ++k)
                        if (tidx[k] == idx[i]) {
                            same += tp[k];
                            if (k < tid + i * T) lead[i] = false;
                        }
                    p[i] = same;
                    logp[i] = log_of(same);
                }
        }
    if (FORM != PIECE && holds) {
#pragma unroll
        for (int i = 0; i < KI; ++i)
            if (lead[i]) {
                eq[i] = soft_exp(zk[i]);
                if (has) eq1[i] = beside == SAME ? eq[i] : hard_exp(zk[i]);
                members += (double)eq[i];
                members1 += (double)eq1[i];
            }
        sum = wave_reduce(sum, add);
        if constexpr (TAIL) {
            members = wave_reduce(members, add);
            members1 = wave_reduce(members1, add);
        }
    }
    if constexpr (T > 64) {
        if (lane == 0) {
            sht[0][wave] = st;
            sht[1][wave] = s1;
            shd[0][wave] = sum;
            shd[1][wave] = members;
            shd[2][wave] = members1;
        }
        __syncthreads();
        st = sht[0][0];
        s1 = sht[1][0];
        sum = shd[0][0];
        members = shd[1][0];
        members1 = shd[2][0];
#pragma unroll
        for (int w = 1; w < W; ++w) {
            st += sht[0][w];
            s1 += sht[1][w];
            if (w * 64 < a.k) {
                sum += shd[0][w];
                members += shd[1][w];
                members1 += shd[2][w];
            }
        }
    }
    if constexpr (FORM == PIECE) {
        if (tid == 0)
            *reinterpret_cast<float4*>(a.part + 4 * ((int64_t)row * a.splits + piece)) = make_float4(mt, st, s1, 0.f);
        return;
    }
    if constexpr (!TAIL) {
        const double by = over(sum), logs = log_of(sum);
#pragma unroll
        for (int i = 0; i < KI; ++i) {
            p[i] = idx[i] >= 0 ? p[i] * by : 0.0;
            logp[i] -= logs;
        }
    }
    // r; sums of all exponentials, at both temperatures, relative to mall
    double rest = 0.0, total = (double)st, total1 = (double)(beside == SAME ? st : s1);
    float down = 1.f, down1 = 1.f;  // from the rest's largest logit to mall
    bool some = false;              // the rest has classes that are not masked, and the teacher gives them something
    if constexpr (TAIL) {
        rest = sum != sum ? sum : fmax(0.0, 1.0 - sum);
        some = mt != -INFINITY && !(rest == 0.0);
        down = mt == -INFINITY ? 0.f : soft_exp(mt);
        total = (double)st * (double)down + members;
        total1 = total;
        if (beside != SAME) {
            down1 = mt == -INFINITY ? 0.f : hard_exp(mt);
            total1 = (double)s1 * (double)down1 + members1;
        }
    }
    const double full = TAIL ? sum + (some ? rest : 0.0) : sum > 0.0 || sum != sum ? 1.0 : 0.0;

    if (a.d) {
        // The gradient of the rest: coefficients of its exponentials as the passes form them; st can be 0 only where
        // nothing is taken of it
        const double soft = (1.0 - (double)a.alpha) * (double)a.tau, q0 = full * over(total);
        const double hard = has ? (double)a.alpha * over(total1) : 0.0, rq = TAIL && some ? rest * over((double)st) : 0.0;
        double cr = soft * (q0 * (double)down - rq);
        if (beside == SAME) cr += hard * (double)down;
        const float ce = (float)((double)weight * cr * (double)corr);
        const float ch = (float)((double)weight * hard * (double)down1 * (double)corr1);
        by_kind([&](auto kind) {
            asm volatile("" : "+s"(half));
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = c0 + i * T + tid;
                if (c >= lo && c < hi) {
                    float g[P];
#pragma unroll
                    for (int j = 0; j < P; ++j) {
                        float e, e1;
                        both(at(i, j), kind, e, e1);
                        g[j] = ce * e;
                        if constexpr (decltype(kind)::value != SAME) g[j] = fmaf(ch, e1, g[j]);
                    }
                    store(c, g);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (es >= 0) {
                float e, e1;
                both(xs, kind, e, e1);
                d[es] = (E)fmaf(ch, e1, ce * e);
            }
        });
        __syncthreads();
        auto here = [&](int e) { return FORM == WHOLE || ((e + z.shift) / P >= c0 && (e + z.shift) / P < c1); };
#pragma unroll
        for (int i = 0; i < KI; ++i)
            if (lead[i] && here(idx[i])) {
                double g = soft * (q0 * (double)eq[i] - p[i]) + hard * (double)eq1[i];
                if (has && idx[i] == label) g -= (double)a.alpha;
                d[idx[i]] = (E)(float)((double)weight * g);
            }
        if (tid == T - 1 && has && !among && here(label)) {
            const float e = soft_exp(zlabel), e1 = beside == SAME ? e : hard_exp(zlabel);
            double g = soft * q0 * (double)e + hard * (double)e1 - (double)a.alpha;
            if (TAIL && some) g -= soft * rq * (double)__builtin_amdgcn_exp2f((zlabel - mt) * kt);
            d[label] = (E)(float)((double)weight * g);
        }
    }

    if (piece == 0) {
        const double logt = log_of(total);
        double l = 0.0;
#pragma unroll
        for (int i = 0; i < KI; ++i)
            if (holds && lead[i] && !(p[i] == 0.0)) l += p[i] * (logp[i] - (((double)zk[i] - (double)mall) * inv_tau - logt));
        if (holds) l = wave_reduce(l, add);
        if constexpr (T > 64) {
            if (lane == 0) shl[wave] = l;
            __syncthreads();
            l = shl[0];
            for (int w = 1; w * 64 < a.k && w < W; ++w) l += shl[w];
        }
        if (tid == 0) {
            if (TAIL && some) l += rest * (log_of(rest) - (((double)mt - (double)mall) * inv_tau + log_of((double)st) - logt));
            l *= (1.0 - (double)a.alpha) * (double)a.tau * (double)a.tau;
            if (has) l += (double)a.alpha * (log_of(total1) + (double)mall - (double)zlabel);
            a.row_loss[row] = (float)l;
        }
    }
}

// loss = sum of weight * row_loss in a fixed order, in 64 bits: a launch of 2 us, 5 for 4096 rows
__global__ __launch_bounds__(1024) void distill_sum_k(int n, const float* row_loss, const float* weight, float each,
                                                       float* loss)
{
    __shared__ double sh[16];
    double s = 0.0;
    for (int i0 = threadIdx.x; i0 < n; i0 += 4096) {  // four loads on their way at a time
        float w[4], l[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = i0 + 1024 * k;
            w[k] = i >= n ? 0.f : weight ? weight[i] : each;
            l[k] = i < n ? row_loss[i] : 0.f;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (w[k] != 0.f) s += (double)w[k] * (double)l[k];
    }
    s = block_reduce<1024>(s, sh, [](double x, double y) { return x + y; });
    if (threadIdx.x == 0) loss[0] = (float)s;
}

// Pieces of a row, 1: rows whole, and chunks of one.  Whole wherever a workgroup's registers hold a row (8 rows of 30000
// float32: 10.8 us, in pieces 4.6 and 7.7; 120 rows 13.7, in pieces 7.6 and 14.0).  Small pieces fill the chip with few rows
// (8 rows of 50000: 4.5 and 7.7, in large ones 5.4 and 10.8), large ones leave less to put together (120 rows: 9.4 and 14.3,
// in small ones 10.5 and 17.4).
struct Cut {
    int splits = 1, per = 0;
    Cut(int n, int64_t bytes)
    {
        if (bytes <= 16 * 512 * 16) return;
        per = n >= 64 ? 256 * 8 : 256 * 2;
        splits = (int)((bytes + 16 * per - 1) / (16 * per));
    }
};

template <typename E, bool TAIL>
void launch(const DistillArgs& a, int64_t bytes, const Work& w, hipStream_t st)
{
    const dim3 rows((unsigned)a.n);
#define PSW_WHOLE(T, NV, KI)                                                                                      \
    PSW_LAUNCH(kname("distill_k", (int)sizeof(E), T, NV, TAIL, (int)WHOLE, KI), w, (distill_k<E, T, NV, TAIL, WHOLE, KI>), \
               rows, dim3(T), 0, st, a)
    if (a.splits == 1) {
        // one wave a row where it holds it, with an entry a thread where that is enough (8192 rows of 100 bfloat16, 26
        // entries: 12.7 us, with room for four 14.8; 100 entries of 6000 rows of 1000 by four waves a row 34.7, so 18.6)
        if (bytes <= 16 * 64 * 4 && a.k <= 64)
            PSW_WHOLE(64, 4, 1);
        else if (bytes <= 16 * 64 * 4)
            PSW_WHOLE(64, 4, 4);
        else if (bytes <= 16 * 256 * 4)
            PSW_WHOLE(256, 4, 1);
        else if (bytes <= 16 * 256 * 8)
            PSW_WHOLE(256, 8, 1);
        else if (bytes <= 16 * 512 * 8)
            PSW_WHOLE(512, 8, 1);
        else
            PSW_WHOLE(512, 16, 1);
        return;
    }
#undef PSW_WHOLE
    const dim3 pieces((unsigned)a.n * (unsigned)a.splits);
#define PSW_PIECES(NV, FORM)                                                                                      \
    PSW_LAUNCH(kname("distill_k", (int)sizeof(E), 256, NV, TAIL, (int)FORM, 1), w, (distill_k<E, 256, NV, TAIL, FORM, 1>), pieces, \
               dim3(256), 0, st, a)
    if (a.per == 256 * 2) {
        PSW_PIECES(2, PIECE);
        PSW_PIECES(2, GRADIENT);
    } else {
        PSW_PIECES(8, PIECE);
        PSW_PIECES(8, GRADIENT);
    }
#undef PSW_PIECES
}

}  // namespace

// row losses, then the pieces' sums and the members' logits
size_t distill_ws_bytes(int n, int classes)
{
    const int splits = Cut(n, row_bytes(classes, 4)).splits;  // bfloat16 takes as many or fewer
    const size_t rows = ((size_t)n * sizeof(float) + 15) / 16 * 16;
    return rows + (splits > 1 ? (size_t)n * (4 * (size_t)splits + kMost + 1) * sizeof(float) : 0);
}

bool distill_fits(int n, int classes, int bf16)
{
    const int64_t bytes = row_bytes(classes, bf16 ? 2 : 4);  // the more, the more threads
    const int splits = Cut(n, bytes).splits, whole = bytes <= 16 * 64 * 4 ? 64 : bytes <= 16 * 256 * 8 ? 256 : 512;
    return (int64_t)n * (splits > 1 ? splits * 256 : whole) <= kGridThreads;
}

hipError_t distill(int n, int classes, int bf16, const void* z, int64_t ld, int k, const int32_t* idx, const float* val,
                   const float* lse, const int32_t* labels, const float* weight, float tau, float alpha, float* loss,
                   float* row_loss, void* dz, int64_t ldd, void* ws, hipStream_t st)
{
    DistillArgs a{};
    a.z = z; a.d = dz; a.ld = ld; a.ldd = ldd;
    a.n = n; a.classes = classes; a.k = k;
    a.idx = idx; a.val = val; a.lse = lse; a.weight = weight; a.labels = labels;
    a.tau = tau; a.alpha = alpha; a.each = 1.f / (float)n; a.inv_tau = 1.0 / (double)tau; a.kt = kLog2e / tau;
    float* const scratch = (float*)((char*)ws + ((size_t)n * sizeof(float) + 15) / 16 * 16);
    a.row_loss = row_loss ? row_loss : (float*)ws;
    const int size = bf16 ? 2 : 4;
    const int64_t bytes = row_bytes(classes, size, z, ld, n);
    const Cut cut(n, bytes);
    a.splits = cut.splits;
    a.per = cut.per;
    a.part = scratch;
    a.zk = scratch + 4 * (size_t)n * a.splits;
    const double nv = (double)n * classes;
    const Work w{8 * nv, size * nv * (dz ? 2 : 1) + 8.0 * n * k};
    if (bf16)
        lse ? launch<__bf16, true>(a, bytes, w, st) : launch<__bf16, false>(a, bytes, w, st);
    else
        lse ? launch<float, true>(a, bytes, w, st) : launch<float, false>(a, bytes, w, st);
    if (loss)
        PSW_LAUNCH(kname("distill_sum_k"), (Work{2.0 * n, 2 * kF * n}), distill_sum_k, dim3(1), dim3(1024), 0, st, n,
                   a.row_loss, weight, a.each, loss);
    return hipGetLastError();
}

}  // namespace psw
