// Drafted tokens: which of a tree's tokens stand (psa_verify_drafts), and what the cache keeps of them (psa_cache_keep).
//
// Verification walks a sequence's tree from its root.  At a token with target probabilities p = softmax(logits / T) and children x_1, x_2, .. (drawn from draft
// probabilities q = softmax(drafts / T)), child x_m stands if u_m q_m(x_m) < w(x_m) / Z, where w = p, Z = 1 at first, and behind every child that does not stand
//     w <- max(w / Z - q_m, 0),   Z <- sum_v w(v).
// As q_m is q times a number (1, or 1 / (1 - what was drawn before) where siblings are drawn without replacement; tokens drawn before have w = 0 already), a child that is refused costs two
// numbers, by which w follows from p and q wherever it is needed, and one sum over the row.  (In one step w is max(a p - b q, 0), but a grows with 1 / Z, and behind a few refused children of drafts
// near p nothing is left of the difference.)  Where nobody stands the next token is the first one at
// which the sum of w along the vocabulary passes u_root times the whole.
//
// A number next to a border decides about a token.  A draw has as many borders as the vocabulary has tokens, and with sums in 32 bits one draw in a hundred would fall on the other side of one:
// it is made from exponentials and sums in 64 bits (11 operations of that pipe a number, a sixth of a clock on an SM).  Whether a child stands is one comparison: it is made with sums of
// 32-bit exponentials first, and only where both sides are nearer to each other than those may be off, or where a child with drafts is refused, with the others.
// Sums are formed in an order that depends on the sizes alone.
//
// Measured (one B200; by chance more or fewer tokens stand): 64 chains of 6 rows of 128,000 numbers in bf16 with drafts 125 to 133 us (the bytes alone 13, the exponentials in 64 bits 20); 16 trees of 33 in fp32,
// 50,001 numbers, 59 to 68 us; one greedy chain of 5, 32,000 numbers, 4.9 us where none stands, 8.4 to 13 where all do.  46 % of the issue slots at the first: a level costs a warp 800 instructions beside 9 for every 32 numbers of a row, an exponential in 64 bits 60, and the sequence with the longest path
// decides.  (Neither rows in shared memory by bulk copies nor exponentials with half the 64-bit operations make it faster.)
//
// To read: the rows of the tokens on the path, and no others; which ones these are is known one after the other, so that what counts is how fast one row is read.  A
// cluster of CTAs shares the rows of a sequence; a row costs one pass with a running maximum and one exchange of partial maxima and sums between the CTAs, a child with drafts that is refused two
// more passes over what is then in the L2 cache.
#include <string.h>
#include <algorithm>
#include <type_traits>

#include "psa_cache.cuh"
#include "psa_internal.h"
#include "psa_sched.h"
#include "sm100.cuh"

namespace psa {

namespace {

constexpr int MOST_CLUSTER = 8;
constexpr int V_CTAS = 4;                       // an SM: with 64 registers a thread.  (With three, 80 registers and two rounds 156 us where this takes 128)
// Relative error of a sum of 32-bit exponentials, in 2^-24.  The number that weights are relative to is raised when it is passed by 2^8 only, so that a weight 2^-a of the greatest one has gone through
// arguments of a + 16 and (a + 16) / 8 raises; over the sum's weights a is 30 on average at most (their entropy, 2^30 of them).  An argument goes through three roundings (1 / T ln 2, difference, product):
// 3 ln 2 46 = 96; a weight's own ex2 4 (2^-22), a raise 5 with its product: 29; the factors of thread, warp, CTA and cluster 5 each: 20; 36 additions before the sums go on in 64 bits and 14 in those of the
// threads, warps and CTAs: 50.  199 altogether, below 2^-16.
constexpr float COARSE = 1.f / 65536;
// A comparison is certain where its sides are further apart than this, relative to the greater one (absolute without drafts, where both are 1 at most): a sum on each, and a weight, which is
// 3 ln 2 100 + 5 off where it is 1e-30 of the sum or more.  825 of 2^-24 together.
constexpr float SURE = 4 * COARSE, LEAST_SURE = 1e-30f;

// What is left of two distributions of sum one that are the same but for roundings: tokens that could not have been drawn get there (a child with q = 0 behind all others), a drawn one with less than this
// probability.
constexpr double NOTHING = 1e-13;

struct VerifyArgs {
    const void *logits, *drafts;
    long long logit_stride, draft_stride;
    const int *tokens, *parents, *starts;
    const float *temperatures, *uniform;
    int *path, *accepted, *next;
    int vocab, sequences, rows, distinct;
    int slice;                                  // of a CTA: numbers of the vocabulary
};

template <class T> __device__ __forceinline__ float number(T x) { return static_cast<float>(x); }
template <> __device__ __forceinline__ float number<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float number<__half>(__half x) { return __half2float(x); }

// What the CTAs of a cluster tell each other: about a row, greatest numbers and sums in 32 bits; about a pass in 64 bits, sums.
struct __align__(16) Record {
    float p_max, q_max, p_sum, q_sum;
    int likeliest, bad, unused[2];
};
struct __align__(16) Sums {
    double p, q, a, b;
};

__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
    for (int s = 16; s > 0; s /= 2) x += __shfl_xor_sync(0xffffffffu, x, s);
    return x;
}
// x to the same place in CTA `rank`'s shared memory; X: words of 16 bytes.
template <class X>
__device__ __forceinline__ void tell(X* to, const X& x, uint32_t rank) {
    static_assert(sizeof(X) % 16 == 0 && alignof(X) == 16, "");
    const uint32_t a = cluster_map(to, rank);
    uint4 words[sizeof(X) / 16];
    memcpy(words, &x, sizeof(X));
#pragma unroll
    for (int i = 0; i < (int)(sizeof(X) / 16); ++i) {
        const uint4 v = words[i];
        asm volatile("st.shared::cluster.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(a + 16 * i), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
    }
}

// exp((x - top) / T) for x <= top, called by all lanes of a warp together, to 2^-48 beside 2^-53 of the exponent: with z = 32 (x - top) / (T ln 2), 2^(k / 32) (1 + e), k being the nearest whole number, the power from a table of
// 32 (one a lane), e by its Taylor series up to the fifth power, which leaves 2^-48.7 (table-driven exponentials: Tang, 1989).  Zero below 2^-1018 and for -inf.
struct Exp {
    double power, top, C;                        // 2^(lane / 32); C: 32 / (T ln 2)
    float top32, c;                              // the same in 32 bits; c: 1 / (T ln 2)
    __device__ __forceinline__ Exp(double power_, float top_, double C_) : power(power_), top(top_), C(C_), top32(top_), c((float)(C_ / 32)) {}
    __device__ __forceinline__ double operator()(float x) const {
        constexpr double L = 0.69314718055994530942 / 32;
        const double z = ((double)x - top) * C, t = z + 6755399441055744.0, s = z - (t - 6755399441055744.0);
        const int k = __double2loint(t);
        const double e = s * fma(s, fma(s, fma(s, fma(s, L * L * L * L * L / 120, L * L * L * L / 24), L * L * L / 6), L * L / 2), L);
        const double p = __hiloint2double(__shfl_sync(0xffffffffu, __double2hiint(power), k & 31), __shfl_sync(0xffffffffu, __double2loint(power), k & 31));
        const double w = fma(p, e, p);
        return c * (x - top32) > -1018.f ? __hiloint2double(__double2hiint(w) + (k >> 5) * 1048576, __double2loint(w)) : 0.0;
    }
};

// f(number of the first row, number of the second, v) for v = low .. high - 1, by a warp, every call by all lanes: those that have no v call it with -inf.  Numbers are read two at a time,
// one by one up to a boundary of two and where the rows lie differently.
template <class T, bool TWO, class F>
__device__ __forceinline__ void over(const T* p, const T* q, int low, int high, int lane, F f) {
    if (low >= high) return;
    const uintptr_t at = reinterpret_cast<uintptr_t>(p + low) / sizeof(T), too = TWO ? reinterpret_cast<uintptr_t>(q + low) / sizeof(T) : at;
    const bool alike = ((at ^ too) & 1u) == 0;
    struct __align__(2 * sizeof(T)) Two { T x, y; };
    const int lead = alike ? (int)(at & 1u) : high - low, pairs = (high - low - lead) / 2;
    const Two* const p2 = reinterpret_cast<const Two*>(p + low + lead);
    const Two* const q2 = TWO ? reinterpret_cast<const Two*>(q + low + lead) : p2;
    constexpr int AHEAD = 2;                     // rounds
    Two x[AHEAD], y[AHEAD];
    auto load = [&](int i, int k) {
        if (i >= pairs) return;
        x[k] = p2[i];
        if (TWO) y[k] = q2[i];
    };
    load(lane, 0);
    load(lane + 32, 1);
#pragma unroll 1
    for (int i0 = 0; i0 < pairs; i0 += 32) {
        const Two x0 = x[0], y0 = y[0];
        const int i = i0 + lane, v = low + lead + 2 * i;
        x[0] = x[1];
        if (TWO) y[0] = y[1];
        load(i + 32 * AHEAD, 1);
        const bool is = i < pairs;
        f(is ? number(x0.x) : -INFINITY, TWO && is ? number(y0.x) : -INFINITY, v);
        f(is ? number(x0.y) : -INFINITY, TWO && is ? number(y0.y) : -INFINITY, v + 1);
    }
#pragma unroll 1
    for (int v0 = low; v0 < high;) {             // one by one: those ahead of the pairs, then those behind
        const int end = v0 < low + lead ? low + lead : high, v = v0 + lane;
        if (end == high && v0 < low + lead + 2 * pairs && v0 >= low + lead) { v0 = low + lead + 2 * pairs; continue; }
        f(v < end ? number(p[v]) : -INFINITY, TWO && v < end ? number(q[v]) : -INFINITY, v);
        v0 = min(v0 + 32, end);
    }
}
// Sum of exp over a part of a row, without the tokens of a list.
template <class T>
__device__ __noinline__ double sum_one(const T* row, int low, int high, const Exp& exp_of, const int* without, int n, int lane) {
    const Exp e = exp_of;
    double sum = 0;
    over<T, false>(row, nullptr, low, high, lane, [&](float x, float, int v) {
        double w = e(x);
        for (int k = 0; k < n; ++k)
            if (without[k] == v) w = 0;
        sum += w;
    });
    return sum;
}
// Over a part of two rows: sums of exp_p and of exp_q, and of both where exp_p > k exp_q.
template <class T>
__device__ __noinline__ Sums sum_both(const T* p, const T* q, int low, int high, const Exp& exp_p, const Exp& exp_q, double k, int lane) {
    const Exp ep = exp_p, eq = exp_q;
    Sums s = {0, 0, 0, 0};
    over<T, true>(p, q, low, high, lane, [&](float x, float y, int) {
        const double pw = ep(x), qw = eq(y);     // (by all lanes)
        s.p += pw;
        s.q += qw;
        if (pw > k * qw) { s.a += pw; s.b += qw; }
    });
    return s;
}
// What `n` refused children leave of a weight, by the numbers of each.
struct Refused {
    double up, less;                             // 1 / Z ahead of it; what exp_q is multiplied with
};
__device__ __forceinline__ double left_of(double pw, double qw, const Refused* refused, int n) {
    for (int j = 0; j < n; ++j) pw = fma(-refused[j].less, qw, pw * refused[j].up);      // (what is below zero stays there)
    return fmax(pw, 0.0);
}
// Its sum.
template <class T>
__device__ __noinline__ double sum_rest(const T* p, const T* q, int low, int high, const Exp& exp_p, const Exp& exp_q, const Refused* refused, int n, int lane) {
    const Exp ep = exp_p, eq = exp_q;
    double sum = 0, a = 1, b = 0;                // in one step: max(a p - b q, 0)
    for (int j = 0; j < n; ++j) {
        a *= refused[j].up;
        b = fma(b, refused[j].up, refused[j].less);
    }
    if (a <= 1e4) {                              // (nearly always: what cancels is 1e-12 of the sum at most.  16 trees of 33: 61 us, child by child 65)
        const double k = b / a;
        over<T, true>(p, q, low, high, lane, [&](float x, float y, int) {
            const double pw = ep(x), qw = eq(y);
            sum += fmax(fma(-k, qw, pw), 0.0);
        });
        sum *= a;
    } else {
        over<T, true>(p, q, low, high, lane, [&](float x, float y, int) {
            const double pw = ep(x), qw = eq(y);
            sum += left_of(pw, qw, refused, n);
        });
    }
    return sum;
}

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Two numbers at a time.
__device__ __forceinline__ uint64_t pair_of(float x, float y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ float2 pair_as(uint64_t x) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t x, uint64_t y) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t x, uint64_t y) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
    return r;
}

// Of a thread's share of a part of a row (vectors of 16 bytes in turn): the greatest number, the first place that has it (GREEDY), whether a number is NaN or +inf, and the sum of
// 2^(c (x - greatest)) in 32 bits (not GREEDY; on the way relative to a number that the greatest one passes by no more than 2^8, see COARSE).  Bound by ex2, 16 a clock on an SM: everything else is
// done two numbers at a time, and a NaN is found in the sum.
struct Part {
    float top, sum;
    int arg;
    bool bad;
};
template <class T, int THREADS, bool GREEDY>
__device__ __forceinline__ Part part_of_row(const T* row, int low, int high, float c, int tid) {
    constexpr int VEC = 16 / sizeof(T), LONGEST = 8;     // vectors whose sum is formed in 32 bits
    Part r = {-INFINITY, 0.f, 0x7fffffff, false};
    uint64_t sum2 = 0;
    double whole = 0;
    int chain = 0;
    float most = -INFINITY, limit = -INFINITY;   // the greatest number; where the one that weights are relative to (r.top) is raised
    const float slack = fminf(8.f / c, 1e38f);
    const uintptr_t at = reinterpret_cast<uintptr_t>(row + low);
    const int n = high - low, lead = min((int)((16 - (at & 15u)) % 16 / sizeof(T)), n), vecs = (n - lead) / VEC, done = lead + vecs * VEC;
    auto raise = [&](float m) {
        const float f = r.top > -INFINITY ? exp2_fast(c * (r.top - m)) : 0.f;
        sum2 = mul2(sum2, pair_of(f, f));
        whole *= (double)f;
        r.top = m;
        limit = m + slack;
    };
    auto one = [&](int v) {
        const float x = number(row[v]);
        if (GREEDY) {
            r.bad |= !(x <= 3.402823466e38f);
            if (x > r.top || (x == r.top && v < r.arg)) { r.top = x; r.arg = v; }
        } else {
            most = fmaxf(most, x);
            if (x > limit) raise(x);
            sum2 = add2(sum2, pair_of(exp2_fast(c * (x - (r.top > -INFINITY ? r.top : 0.f))), 0.f));
        }
    };
    if (tid < lead) one(low + tid);
    const uint4* const row4 = reinterpret_cast<const uint4*>(row + low + lead);
    constexpr int AHEAD = 4;
    for (int i0 = 0; i0 < vecs; i0 += AHEAD * THREADS) {
        uint4 x[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (i0 + k * THREADS + tid < vecs) x[k] = __ldg(row4 + i0 + k * THREADS + tid);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int i = i0 + k * THREADS + tid;
            if (i < vecs) {
                float y[VEC], m = -INFINITY;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    y[e] = number(reinterpret_cast<const T*>(&x[k])[e]);
                    if (GREEDY) r.bad |= !(y[e] <= 3.402823466e38f);
                    m = fmaxf(m, y[e]);
                }
                if (GREEDY) {
                    if (m > r.top) {
                        r.top = m;
#pragma unroll
                        for (int e = VEC - 1; e >= 0; --e)
                            if (y[e] == m) r.arg = low + lead + i * VEC + e;
                    }
                } else {
                    most = fmaxf(most, m);
                    if (m > limit) raise(m);
                    const float from = r.top > -INFINITY ? -r.top : 0.f;
                    const uint64_t from2 = pair_of(from, from), c2 = pair_of(c, c);
#pragma unroll
                    for (int e = 0; e < VEC; e += 2) {
                        const float2 z = pair_as(mul2(add2(pair_of(y[e], y[e + 1]), from2), c2));
                        sum2 = add2(sum2, pair_of(exp2_fast(z.x), exp2_fast(z.y)));
                    }
                    if (++chain == LONGEST) {
                        whole += (double)pair_as(sum2).x + (double)pair_as(sum2).y;
                        sum2 = 0;
                        chain = 0;
                    }
                }
            }
        }
    }
    if (tid < n - done) one(low + done + tid);
    if (!GREEDY) {
        whole += (double)(pair_as(sum2).x + pair_as(sum2).y);
        if (most > r.top) whole *= (double)exp2_fast(c * (r.top - most));
        r.top = most;
        r.sum = (float)whole;
        r.bad = !(r.sum < INFINITY) || r.top == INFINITY;
    }
    return r;
}

template <class T, int V_WARPS>
__global__ void __launch_bounds__(32 * V_WARPS, V_WARPS == 8 ? V_CTAS : 1) verify_kernel(const VerifyArgs a, DeviceCounters* dc, DeviceCounters* dc_next) {
    constexpr int V_THREADS = 32 * V_WARPS;
    __shared__ int parent_s[PSA_TREE_MOST], token_s[PSA_TREE_MOST], tried_s[PSA_TREE_MOST];
    __shared__ Record warps_s[V_WARPS];
    __shared__ Sums parts_s[V_WARPS];
    __shared__ double sums_s[V_WARPS], fine_s[V_WARPS];
    __shared__ Refused refused_s[PSA_TREE_MOST];
    __shared__ int drawn_s;
    // What the CTAs tell each other, in two places by turns: written ahead of a barrier, read behind it.  (Each writes to all others.  Read from there by every warp it was 3 us a token with 32 warps.)
    __shared__ Record records[2][MOST_CLUSTER];
    __shared__ Sums sums[2][MOST_CLUSTER];

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int ranks = (int)gridDim.x, rank = (int)blockIdx.x, b = (int)blockIdx.y;       // (a cluster is a row of the grid)
    grid_dependency_wait();
    if (tid == 0 && rank == 0 && b == 0 && dc_next) *dc_next = DeviceCounters{0, 0, 0, 0, 0, 0, 0};
    const int first = min(max(a.starts[b], 0), a.rows), count = max(min(max(a.starts[b + 1], 0), a.rows) - first, 0);
    const float temperature = a.temperatures ? a.temperatures[b] : 1.f;
    const bool greedy = temperature < 1.17549435e-38f;     // (zero, and what 1 / T could not be formed of)
    const bool refused = count > PSA_TREE_MOST || !(temperature >= 0.f && temperature <= 3.0e38f);
    if (refused || count == 0) {
        if (rank == 0) {
            for (int i = tid; i < count; i += V_THREADS) a.path[first + i] = -1;
            if (tid == 0) {
                a.accepted[b] = 0;
                a.next[b] = -1;
                if (refused) atomicExch(&dc->status, (int)PSA_ERR_SHAPE);
            }
        }
        return;                                  // (the whole cluster)
    }
    bool strange = false;                        // a parent that is no earlier token, or a token that the vocabulary does not have
    for (int i = tid; i < count; i += V_THREADS) {
        const int p = a.parents[first + i], x = a.tokens[first + i];
        const bool good_p = i == 0 ? p == -1 : p >= -1 && p < i;
        strange |= !good_p || (i > 0 && (x < 0 || x >= a.vocab));
        parent_s[i] = i > 0 && good_p ? p : -1;
        token_s[i] = x >= 0 && x < a.vocab ? x : -1;
        if (rank == 0) a.path[first + i] = i == 0 ? 0 : -1;
    }
    if (__syncthreads_or(strange) && tid == 0) atomicExch(&dc->status, (int)PSA_ERR_SHAPE);

    // (shared memory of another CTA is there once that one has begun: arrived here, waited for ahead of the first word to it)
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    bool met = false;
    const double C = greedy ? 1.0 : 46.166241308446828384 / (double)temperature;         // 32 / (T ln 2): units of Exp
    const float c = (float)(C / 32);
    const T* const all_logits = static_cast<const T*>(a.logits);
    const T* const all_drafts = static_cast<const T*>(a.drafts);
    const int low = min(rank * a.slice, a.vocab), high = min(low + a.slice, a.vocab);    // this CTA's part of the vocabulary
    const int each = (high - low + V_WARPS - 1) / V_WARPS;                               // of its warps, one after another
    const int w_low = min(low + warp * each, high), w_high = min(w_low + each, high);

    int turn = 0;                                // of records and sums: one exchange, one turn
    int node = 0, stood = 0, next = -1;
    for (;;) {
        const T* const lrow = all_logits + (size_t)(first + node) * a.logit_stride;
        // the token's first child, and what it is tried with (asked for here, used behind the exchange)
        int child = count;
        for (int i0 = node + 1; i0 < count && child == count; i0 += 32) {
            const uint32_t m = __ballot_sync(0xffffffffu, i0 + lane < count && parent_s[min(i0 + lane, count - 1)] == node);
            if (m) child = i0 + __ffs(m) - 1;
        }
        const bool use_q = all_drafts && !greedy && child < count;
        const T* const qrow = all_drafts + (use_q ? (size_t)(first + node) * a.draft_stride : 0);
        float child_u = 0.f, child_l = 0.f, child_q = 0.f;
        if (!greedy && child < count && token_s[child] >= 0) {
            child_u = a.uniform[first + child];
            child_l = number(lrow[token_s[child]]);
            child_q = number((use_q ? qrow : lrow)[token_s[child]]);
        }
        // ---- the rows' greatest numbers and sums: of the threads, the warp, the CTA, the cluster
        Part p = greedy ? part_of_row<T, V_THREADS, true>(lrow, low, high, 0.f, tid) : part_of_row<T, V_THREADS, false>(lrow, low, high, c, tid);
        Part q = {-INFINITY, 0.f, 0, false};
        if (use_q) q = part_of_row<T, V_THREADS, false>(qrow, low, high, c, tid);
        auto joined = [&](Record r, int most) {  // of a lane each, as one (those of lanes from `most` on hold nothing)
            float t = r.p_max, qt = r.q_max;
#pragma unroll
            for (int s = 16; s > 0; s /= 2) {
                if (s >= most) continue;
                const float y = __shfl_xor_sync(0xffffffffu, t, s);
                if (greedy) {
                    const int k = __shfl_xor_sync(0xffffffffu, r.likeliest, s);
                    if (y > t || (y == t && k < r.likeliest)) r.likeliest = k;
                }
                t = fmaxf(t, y);
                if (use_q) qt = fmaxf(qt, __shfl_xor_sync(0xffffffffu, qt, s));
            }
            r.bad = __any_sync(0xffffffffu, r.bad != 0);
            if (!greedy) {
                r.p_sum = r.p_max > -INFINITY ? r.p_sum * exp2_fast(c * (r.p_max - t)) : 0.f;
                r.q_sum = r.q_max > -INFINITY ? r.q_sum * exp2_fast(c * (r.q_max - qt)) : 0.f;
#pragma unroll
                for (int s = 16; s > 0; s /= 2) {
                    if (s >= most) continue;
                    r.p_sum += __shfl_xor_sync(0xffffffffu, r.p_sum, s);
                    if (use_q) r.q_sum += __shfl_xor_sync(0xffffffffu, r.q_sum, s);
                }
            }
            r.p_max = t;
            r.q_max = qt;
            return r;
        };
        const Record none = {-INFINITY, -INFINITY, 0.f, 0.f, 0x7fffffff, 0, {0, 0}};
        {
            const Record r = joined(Record{p.top, q.top, p.sum, q.sum, p.arg, p.bad || q.bad, {0, 0}}, 32);
            if (lane == 0) warps_s[warp] = r;
        }
        if (!met) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        met = true;
        __syncthreads();
        if (warp == 0) {
            const Record r = joined(lane < V_WARPS ? warps_s[lane] : none, 32);
            if (lane < ranks) tell(&records[turn][rank], r, lane);
        }
        __syncwarp();
        cluster_sync();
        static_assert((MOST_CLUSTER & (MOST_CLUSTER - 1)) == 0, "");
        const Record row = joined(lane % MOST_CLUSTER < ranks ? records[turn][lane % MOST_CLUSTER] : none, MOST_CLUSTER);        // (the same in every group of lanes)
        turn ^= 1;
        if (row.bad || row.p_max == -INFINITY || (use_q && row.q_max == -INFINITY)) {      // numbers that are no distribution
            if (rank == 0 && tid == 0) atomicExch(&dc->status, (int)PSA_ERR_NUMERIC);
            break;
        }
        const float top = row.p_max, q_top = use_q ? row.q_max : 0.f;
        int taken = -1;
        if (greedy) {
            for (int i0 = child; i0 < count && taken < 0; i0 += 32) {
                const int i = min(i0 + lane, count - 1);
                const uint32_t m = __ballot_sync(0xffffffffu, i0 + lane < count && parent_s[i] == node && token_s[i] == row.likeliest);
                if (m) taken = i0 + __ffs(m) - 1;
            }
            if (taken < 0) {
                next = row.likeliest;
                break;
            }
            node = taken;
            ++stood;
            if (rank == 0 && tid == 0) a.path[first + stood] = taken;
            continue;
        }
        // ---- the first child by the sums in 32 bits: taken where that is certain
        if (child < count && token_s[child] >= 0) {
            const float px = exp2_fast(c * (child_l - top)) / row.p_sum;
            const float left = use_q ? child_u * (exp2_fast(c * (child_q - q_top)) / row.q_sum) : child_u, right = px;
            if (right - left > SURE * (use_q ? right : 1.f) && right > LEAST_SURE) {
                node = child;
                ++stood;
                if (rank == 0 && tid == 0) a.path[first + stood] = child;
                continue;
            }
        }
        // ---- in 64 bits from here on, w in units of p's sum: left_of, or p without the children that were refused
        const double power = exp2(lane / 32.0);
        const Exp exp_p(power, top, C), exp_q(power, q_top, C);
        Sums told = {0, 0, 0, 0};                // of all CTAs, by `exchange`, which leaves the warps' in parts_s
        auto exchange = [&](Sums s) {
            s.p = warp_sum(s.p);
            s.q = warp_sum(s.q);
            if (use_q) {
                s.a = warp_sum(s.a);
                s.b = warp_sum(s.b);
            }
            __syncthreads();
            if (lane == 0) parts_s[warp] = s;
            __syncthreads();
            if (warp == 0) {
                Sums x = lane < V_WARPS ? parts_s[lane] : Sums{0, 0, 0, 0};
                x = Sums{warp_sum(x.p), warp_sum(x.q), warp_sum(x.a), warp_sum(x.b)};
                if (lane < ranks) tell(&sums[turn][rank], x, lane);
            }
            __syncwarp();
            cluster_sync();
            told = Sums{0, 0, 0, 0};
            for (int k = 0; k < ranks; ++k) {
                const Sums x = sums[turn][k];
                told.p += x.p;
                told.q += x.q;
                told.a += x.a;
                told.b += x.b;
            }
            turn ^= 1;
        };
        double p_sum = 0, q_sum = 0;
        bool sharp = false;                      // these are known
        double Z = 1, rest = 1, k = 0;
        int tried = 0;
        bool only_p = true;                      // nothing was refused yet, or nothing is left
        // How the sums of w follow from parts_s and sums: a part's is p, or a - k b where both were summed over the numbers that are left.
        bool by_ab = false, summed = false, nothing = false;
        auto part_sum = [&](const Sums& s) { return by_ab ? fmax(fma(-k, s.b, s.a), 0.0) : s.p; };
        auto sum_weights = [&] {
            by_ab = false;
            const double s = !only_p && use_q ? sum_rest(lrow, qrow, w_low, w_high, exp_p, exp_q, refused_s, tried, lane) : sum_one(lrow, w_low, w_high, exp_p, tried_s, only_p ? 0 : tried, lane);
            exchange(Sums{s, 0, 0, 0});
            summed = true;
        };
        for (int i = child; i < count && taken < 0 && !nothing; ++i) {
            if (parent_s[i] != node || token_s[i] < 0) continue;
            const int x = token_s[i];
            bool again = false;                  // a sibling with the same token was refused: nothing is left of it
            if (!use_q || a.distinct)
                for (int n = 0; n < tried; ++n) again |= tried_s[n] == x;
            if (again) continue;
            const double u = a.uniform[first + i], px = exp_p(number(lrow[x])), qx = use_q ? exp_q(number(qrow[x])) : 0.0;
            // Refused for certain by the sums in 32 bits?  (Without drafts the comparison is sharpened only where it is near; with drafts w needs the sums anyway.)
            const bool clear = !sharp && only_p && use_q && u * (qx / (double)row.q_sum) - px / (double)row.p_sum > (double)SURE * u * (qx / (double)row.q_sum);
            double part = 1.0;                   // q_m over q, for tokens that are left
            if (clear) {
                // both rows' sums and those over the numbers that are left, by k in 32 bits, in one pass.  The numbers that k's last bits move from one side to the other are second order in its error,
                // relative to what is left squared; where that is more than 1e-12 the pass is made again.
                const double k0 = (double)row.p_sum / (double)row.q_sum;
                exchange(sum_both(lrow, qrow, w_low, w_high, exp_p, exp_q, k0, lane));
                p_sum = told.p;
                q_sum = told.q;
                sharp = true;
                k = p_sum / q_sum;
                const double off = k0 / k - 1, left = fmax(fma(-k, told.b, told.a), 0.0) / p_sum;
                by_ab = summed = off * off <= 1e-12 * left * left;
            } else {
                if (!sharp && (use_q || fabs(u * Z - px / (double)row.p_sum) <= (double)SURE)) {
                    exchange(Sums{sum_one(lrow, w_low, w_high, exp_p, tried_s, 0, lane), use_q ? sum_one(qrow, w_low, w_high, exp_q, tried_s, 0, lane) : 0.0, 0, 0});
                    p_sum = told.p;
                    q_sum = told.q;
                    sharp = true;
                    if (!use_q) {                // (what was refused before, again)
                        Z = 1;
                        for (int n = 0; n < tried; ++n) Z -= exp_p(number(lrow[tried_s[n]])) / p_sum;
                    }
                }
                // What siblings leave of q is one minus a sum; where that is nearly nothing (a distribution with one likely token) it is summed itself, over the others.
                if (use_q && a.distinct && rest < 1e-6 && tried > 0) {
                    exchange(Sums{sum_one(qrow, w_low, w_high, exp_q, tried_s, tried, lane), 0, 0, 0});
                    rest = told.p / q_sum;
                }
                if (use_q && a.distinct) part = rest > 1e-290 ? 1.0 / rest : 0.0;                // (nothing is left of q: zero everywhere)
                const double pp = px / (sharp ? p_sum : (double)row.p_sum), qq = use_q ? qx / q_sum : 0.0;
                if (use_q ? u * (qq * part) * Z < left_of(px, qx, refused_s, tried) / p_sum : u * Z < pp) {
                    taken = i;
                    continue;
                }
                by_ab = summed = false;
                if (!use_q) Z -= pp;
            }
            const Refused by = {1.0 / Z, use_q ? fmin(part * (p_sum / q_sum), 1e300) : 0.0};
            if (use_q) rest -= qx / q_sum;
            __syncthreads();
            if (tid == 0) {
                tried_s[tried] = x;
                refused_s[tried] = by;
            }
            ++tried;
            __syncthreads();
            only_p = false;
            if (use_q) {
                if (!summed) sum_weights();
                Z = (by_ab ? fmax(fma(-k, told.b, told.a), 0.0) : told.p) / p_sum;
                nothing = !(Z > NOTHING);
            } else if (Z < 1e-6) {               // one minus a sum again (the sums are sharp: in 32 bits nothing is refused that leaves so little)
                sum_weights();
                Z = told.p / p_sum;
                nothing = !(Z > NOTHING);
            }
        }
        if (taken >= 0) {
            node = taken;
            ++stood;
            if (rank == 0 && tid == 0) a.path[first + stood] = taken;
            continue;
        }
        // ---- the draw: the first token at which the running sum of w passes u times the whole
        if (nothing) { only_p = true; summed = false; }
        if (!summed) sum_weights();
        auto whole = [&] {
            double s = 0;
            for (int n = 0; n < ranks; ++n) s += part_sum(sums[turn ^ 1][n]);
            return s;
        };
        const double all = whole();
        // which CTA, then which warp's part; where roundings leave none behind the target, the last one with any weight
        double target = (double)a.uniform[first] * all, before = 0;
        int owner = -1, last = 0;
        for (int n = 0; n < ranks && owner < 0; ++n) {
            const double s = part_sum(sums[turn ^ 1][n]);
            if (s > 0) last = n;
            if (s > 0 && before + s > target) owner = n; else before += s;
        }
        bool end = owner < 0;                    // the last one with any weight is meant
        if (end) owner = last;
        if (owner == rank) {
            auto pick = [&](const double* of_warps) {    // of the warps' parts; target: from there on
                int part = -1;
                before = 0;
                last = 0;
                for (int w = 0; w < V_WARPS && part < 0; ++w) {
                    const double s = of_warps[w];
                    if (s > 0) last = w;
                    if (!end && s > 0 && before + s > target) part = w; else before += s;
                }
                if (part < 0) { part = last; end = true; }
                target -= before;
                return part;
            };
            if (tid < V_WARPS) sums_s[tid] = part_sum(parts_s[tid]);
            __syncthreads();
            target -= before;
            const int part = pick(sums_s);
            // that part once more, each warp a part of it
            const bool two = !only_p && use_q;
            const int p_low = min(low + part * each, high), p_high = min(p_low + each, high), fine = (p_high - p_low + V_WARPS - 1) / V_WARPS;
            const int f_low = min(p_low + warp * fine, p_high), f_high = min(f_low + fine, p_high);
            auto at = [&](int v) -> double {
                const double pw = exp_p(v < f_high ? number(lrow[v]) : -INFINITY);
                if (two) {
                    const double qw = exp_q(v < f_high ? number(qrow[v]) : -INFINITY);
                    return left_of(pw, qw, refused_s, tried);
                }
                bool gone = false;
                for (int n = 0; n < tried && !only_p; ++n) gone |= tried_s[n] == v;
                return gone ? 0.0 : pw;
            };
            const double s = warp_sum(two ? sum_rest(lrow, qrow, f_low, f_high, exp_p, exp_q, refused_s, tried, lane) : sum_one(lrow, f_low, f_high, exp_p, tried_s, only_p ? 0 : tried, lane));
            if (lane == 0) fine_s[warp] = s;
            __syncthreads();
            if (warp == pick(fine_s)) {
                before = 0;
                int found = -1, some = -1;
                for (int v0 = f_low; v0 < f_high && found < 0; v0 += 32) {
                    const double x = at(v0 + lane);
                    double sum = x;
#pragma unroll
                    for (int n = 1; n < 32; n *= 2) {
                        const double y = __shfl_up_sync(0xffffffffu, sum, n);
                        if (lane >= n) sum += y;
                    }
                    const uint32_t past = __ballot_sync(0xffffffffu, !end && x > 0 && before + sum > target), any = __ballot_sync(0xffffffffu, x > 0);
                    if (past) found = v0 + __ffs(past) - 1;
                    if (any) some = v0 + 31 - __clz(any);
                    before += __shfl_sync(0xffffffffu, sum, 31);
                }
                if (lane == 0) drawn_s = found >= 0 ? found : some;
            }
            __syncthreads();
            if (tid == 0) a.next[b] = drawn_s;
        }
        if (rank == 0 && tid == 0) a.accepted[b] = stood;
        return;
    }
    if (rank == 0 && tid == 0) {
        a.accepted[b] = stood;
        a.next[b] = next;
    }
}

// ---------------------------------------------------------------- what the cache keeps
constexpr int KEEP_WARPS = 4;
constexpr int KEEP_TOKENS = 4;                  // in flight

struct KeepArgs {
    uint8_t* pool;
    const int *tables, *lens, *seqs, *starts, *path, *accepted;
    int* new_lens;
    long long layer_bytes;
    int pages, slots, width, page_size, kv_heads, layers, sequences, rows;
    uint32_t units;                             // (sequence, layer, head), a warp each
    FastDiv by_heads, by_sequence, by_page;     // by_sequence: by layers * heads
};

struct Kept {
    int slot, first, count, base, keep;         // keep: tokens that stay, 0: none of this sequence's arguments hold
};
__device__ __forceinline__ Kept claimed(const KeepArgs& a, int b) {
    Kept k;
    k.slot = a.seqs[b];
    k.first = min(max(a.starts[b], 0), a.rows);
    k.count = max(min(max(a.starts[b + 1], 0), a.rows) - k.first, 0);
    const bool known = k.slot >= 0 && k.slot < a.slots;
    const int len = known ? a.lens[k.slot] : 0, stand = a.accepted[b];
    k.base = len - k.count;
    k.keep = known && k.base >= 0 && (long long)len <= (long long)a.width * a.page_size && stand >= 0 && stand < k.count ? stand + 1 : 0;
    return k;
}
// Whether a path goes on at its place i: it ascends from 0 and ends inside the tree.
__device__ __forceinline__ bool ascends(const KeepArgs& a, const Kept& k, int i) {
    const int p = a.path[k.first + i];
    return i == 0 ? p == 0 : p > a.path[k.first + i - 1] && p < k.count;
}
// One sequence, by a warp, and by a thread.
__device__ __forceinline__ Kept kept_of(const KeepArgs& a, int b, int lane) {
    Kept k = claimed(a, b);
    bool good = true;
    for (int i = lane; i < k.keep; i += 32) good &= ascends(a, k, i);
    if (!__all_sync(0xffffffffu, good)) k.keep = 0;
    return k;
}
__device__ __forceinline__ Kept kept_of(const KeepArgs& a, int b) {
    Kept k = claimed(a, b);
    bool good = true;
#pragma unroll 4
    for (int i = 0; i < k.keep; ++i) good &= ascends(a, k, i);
    if (!good) k.keep = 0;
    return k;
}

// Bound by the latency of its look-ups for a few sequences, else by memory: 5 d / 4 bytes a token and head are read and written.  A token's bytes are pieces of 4 and
// of 2 (V shares words with its neighbour), an element a lane.  Tokens move towards the front, in order, KEEP_TOKENS at a time: what is written lies ahead of all that is still to be read.
template <int D>
__global__ void __launch_bounds__(32 * KEEP_WARPS) cache_keep_kernel(const KeepArgs a, DeviceCounters* dc, DeviceCounters* dc_next) {
    using B = CacheBlock<D>;
    constexpr int G = D / 32, WORDS = 5 * G, HALVES = 10 * G, ROUNDS = (WORDS + HALVES + 31) / 32;
    __shared__ int last_s;
    grid_dependency_wait();
    if (threadIdx.x == 0 && blockIdx.x == 0 && dc_next) *dc_next = DeviceCounters{0, 0, 0, 0, 0, 0, 0};
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t unit = blockIdx.x * KEEP_WARPS + warp;
    if (unit < a.units) {
        const int b = (int)fastdiv(unit, a.by_sequence);
        const uint32_t rest = unit - (uint32_t)b * a.by_sequence.d;
        const int layer = (int)fastdiv(rest, a.by_heads), h = (int)(rest - (uint32_t)layer * a.by_heads.d);
        const Kept k = kept_of(a, b, lane);
        if (k.count > 0 && k.keep == 0 && rest == 0 && lane == 0) atomicExch(&dc->status, (int)PSA_ERR_SHAPE);
        uint8_t* const pool = a.pool + (size_t)layer * a.layer_bytes;
        // where the lane's element of each round lies behind its block's beginning: base, and what a pair of tokens and the odd one of a pair add
        int base[ROUNDS], of_pair[ROUNDS], of_odd[ROUNDS];
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int e = r * 32 + lane;
            if (e < 4 * G) { base[r] = B::K_CODES + 4 * e; of_pair[r] = D; of_odd[r] = D / 2; }
            else if (e < WORDS) { base[r] = B::K_SCALES + 4 * (e - 4 * G); of_pair[r] = 8 * G; of_odd[r] = 4 * G; }
            else if (e < WORDS + 8 * G) { base[r] = B::V_CODES + 4 * (e - WORDS); of_pair[r] = D; of_odd[r] = 2; }
            else { base[r] = B::V_SCALES + 4 * (e - WORDS - 8 * G); of_pair[r] = 8 * G; of_odd[r] = 2; }
        }
        auto place = [&](int r, int tok) { return base[r] + (tok >> 1) * of_pair[r] + (tok & 1) * of_odd[r]; };
        for (int i0 = 1; i0 < k.keep; i0 += KEEP_TOKENS) {       // (the root stays where it is)
            // lane l looks up: source of token i0 + l, destination of token i0 + l - KEEP_TOKENS
            const int i = i0 + lane % KEEP_TOKENS;
            uint8_t* at = nullptr;
            int tok = 0;
            if (lane < 2 * KEEP_TOKENS && i < k.keep) {
                const int from = a.path[k.first + i], pos = k.base + (lane < KEEP_TOKENS ? from : i);
                if (from != i) {
                    const int col = (int)fastdiv((uint32_t)pos, a.by_page), in = pos - col * a.page_size;
                    const int page = a.tables[(size_t)k.slot * a.width + col];
                    tok = in % CACHE_BLOCK;
                    if (page >= 0 && page < a.pages) at = pool + (((size_t)page * a.kv_heads + h) * (a.page_size / CACHE_BLOCK) + in / CACHE_BLOCK) * B::BYTES;
                    else atomicExch(&dc->status, (int)PSA_ERR_SHAPE);
                }
            }
            uint32_t x[KEEP_TOKENS][ROUNDS];
            uint8_t* to[KEEP_TOKENS];
            int to_tok[KEEP_TOKENS];
#pragma unroll
            for (int t = 0; t < KEEP_TOKENS; ++t) {
                const uint8_t* from = reinterpret_cast<const uint8_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(at), t));
                to[t] = reinterpret_cast<uint8_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(at), t + KEEP_TOKENS));
                const int from_tok = __shfl_sync(0xffffffffu, tok, t);
                to_tok[t] = __shfl_sync(0xffffffffu, tok, t + KEEP_TOKENS);
                if (!from) to[t] = nullptr;
                if (!to[t]) continue;
#pragma unroll
                for (int r = 0; r < ROUNDS; ++r) {
                    const int e = r * 32 + lane;
                    if (e < WORDS) x[t][r] = *reinterpret_cast<const uint32_t*>(from + place(r, from_tok));
                    else if (e < WORDS + HALVES) x[t][r] = *reinterpret_cast<const uint16_t*>(from + place(r, from_tok));
                }
            }
            __syncwarp();
#pragma unroll
            for (int t = 0; t < KEEP_TOKENS; ++t) {
                if (!to[t]) continue;
#pragma unroll
                for (int r = 0; r < ROUNDS; ++r) {
                    const int e = r * 32 + lane;
                    if (e < WORDS) *reinterpret_cast<uint32_t*>(to[t] + place(r, to_tok[t])) = x[t][r];
                    else if (e < WORDS + HALVES) *reinterpret_cast<uint16_t*>(to[t] + place(r, to_tok[t])) = (uint16_t)x[t][r];
                }
            }
            __syncwarp();
        }
    }
    // ---- the lengths, which may be the ones read above: by the CTA that is done last
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        last_s = atomicAdd(&dc->next_item, 1u) == gridDim.x - 1;
        __threadfence();
    }
    __syncthreads();
    if (last_s)                                  // (a thread a sequence: with a warp a sequence this took 14 of 20 us for 64 of them)
        for (int b = threadIdx.x; b < a.sequences; b += 32 * KEEP_WARPS) {
            const Kept k = kept_of(a, b);
            if (k.keep > 0) a.new_lens[k.slot] = k.base + k.keep;
            else if (a.new_lens != a.lens && k.slot >= 0 && k.slot < a.slots) a.new_lens[k.slot] = a.lens[k.slot];       // (left as it is)
        }
}

cudaLaunchConfig_t config(dim3 grid, int threads, size_t smem, cudaStream_t stream, cudaLaunchAttribute (&attr)[2], int cluster) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster ? 2 : 1;
    return cfg;
}

template <class T>
int launch_verify(VerifyArgs a, DeviceCounters* dc, DeviceCounters* dc_next, cudaStream_t stream) {
    // As many CTAs a sequence as the GPU holds at a time, eight at most and of 2048 numbers at least; with no more than one an SM, of 16 warps, else of 8.  (us of chains in bf16 with drafts, with at most
    // one / two rounds of CTAs: 100 of 128,000 numbers 193, 219, 200 of 64,000 176, 190, 400 of 32,000 156, 166; with 8 / 16 warps: 4 of 128,000 90, 59, 64 of 128,000 152, 219, 16 trees of
    // 50,000 numbers in fp32 82, 68; with one CTA a sequence 64 of 128,000 498.  Sixteen CTAs a sequence take longer than eight: a level costs a warp 800 instructions beside 9 a 32 numbers.)
    int ranks = 1;
    while (ranks < MOST_CLUSTER && 2LL * ranks * a.sequences <= V_CTAS * 148 && a.vocab > 2048 * ranks) ranks *= 2;
    const bool few = (long long)ranks * a.sequences <= 148;
    a.slice = ((a.vocab + ranks - 1) / ranks + 7) / 8 * 8;
    cudaLaunchAttribute attr[2];
    for (int b0 = 0; b0 < a.sequences; b0 += 65535) {
        VerifyArgs x = a;
        x.sequences = std::min(a.sequences - b0, 65535);
        x.starts += b0;
        x.accepted += b0;
        x.next += b0;
        if (x.temperatures) x.temperatures += b0;
        const cudaLaunchConfig_t cfg = config(dim3(ranks, x.sequences), few ? 512 : 256, 0, stream, attr, ranks);
        DeviceCounters* const next = b0 == 0 ? dc_next : nullptr;
        const cudaError_t e = few ? cudaLaunchKernelEx(&cfg, verify_kernel<T, 16>, x, dc, next) : cudaLaunchKernelEx(&cfg, verify_kernel<T, 8>, x, dc, next);
        if (e != cudaSuccess) { set_cuda_error(e, "verify_kernel launch"); return PSA_ERR_CUDA; }
    }
    return PSA_OK;
}

template <int D>
cudaError_t launch_keep(const KeepArgs& a, DeviceCounters* dc, DeviceCounters* dc_next, cudaStream_t stream) {
    cudaLaunchAttribute attr[2];
    const cudaLaunchConfig_t cfg = config(dim3((a.units + KEEP_WARPS - 1) / KEEP_WARPS), 32 * KEEP_WARPS, 0, stream, attr, 0);
    return cudaLaunchKernelEx(&cfg, cache_keep_kernel<D>, a, dc, dc_next);
}

}  // namespace

int verify_drafts(const void* logits, long long logit_stride, const void* drafts, long long draft_stride, int vocab, int dtype, const int* tokens, const int* parents, const int* starts,
                  int sequences, int rows, const float* temperatures, const float* uniform, int distinct, int* path, int* accepted, int* next, DeviceCounters* dc,
                  DeviceCounters* dc_next, cudaStream_t stream) {
    const VerifyArgs a = {logits, drafts, logit_stride, draft_stride, tokens, parents, starts, temperatures, uniform, path, accepted, next, vocab, sequences, rows, distinct, 0};
    switch (dtype) {
        case PSA_F32: return launch_verify<float>(a, dc, dc_next, stream);
        case PSA_BF16: return launch_verify<__nv_bfloat16>(a, dc, dc_next, stream);
        case PSA_F16: return launch_verify<__half>(a, dc, dc_next, stream);
        default: return PSA_ERR_UNSUPPORTED;
    }
}

int cache_keep(const psa_cache& c, int layers, const int* seqs, const int* starts, const int* path, const int* accepted, int sequences, int rows, int* new_lens, DeviceCounters* dc,
               DeviceCounters* dc_next, cudaStream_t stream) {
    const long long units = (long long)sequences * layers * c.kv_heads;
    const KeepArgs a = {static_cast<uint8_t*>(c.pool), c.tables, c.lens, seqs, starts, path, accepted, new_lens, (long long)c.pages * (long long)psa_cache_page_bytes(c.kv_heads, c.page_size, c.d_k),
                        c.pages, c.slots, c.width, c.page_size, c.kv_heads, layers, sequences, rows, (uint32_t)units, fastdiv_make((uint32_t)c.kv_heads),
                        fastdiv_make((uint32_t)layers * (uint32_t)c.kv_heads), fastdiv_make((uint32_t)c.page_size)};
    cudaError_t e = cudaErrorInvalidValue;
    switch (c.d_k) {
        case 32: e = launch_keep<32>(a, dc, dc_next, stream); break;
        case 64: e = launch_keep<64>(a, dc, dc_next, stream); break;
        case 96: e = launch_keep<96>(a, dc, dc_next, stream); break;
        case 128: e = launch_keep<128>(a, dc, dc_next, stream); break;
        case 256: e = launch_keep<256>(a, dc, dc_next, stream); break;
        default: return PSA_ERR_UNSUPPORTED;
    }
    if (e != cudaSuccess) { set_cuda_error(e, "cache_keep_kernel launch"); return PSA_ERR_CUDA; }
    return PSA_OK;
}

}  // namespace psa
