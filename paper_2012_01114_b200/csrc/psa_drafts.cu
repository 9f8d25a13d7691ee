// Drafted tokens: which of a tree's tokens stand (psa_verify_drafts), and what the cache keeps of them (psa_cache_keep).
//
// Verification walks a sequence's tree from its root.  At a token with target probabilities p = softmax(logits / T) and children x_1, x_2, .. (drawn from draft
// probabilities q = softmax(drafts / T)), child x_m stands if u_m q_m(x_m) < w(x_m) / Z, where w = p, Z = 1 at first, and behind every child that does not stand
//     w <- max(w / Z - q_m, 0),   Z <- sum_v w(v).
// As q_m is q times a number (1, or 1 / (1 - what was drawn before) where siblings are drawn without replacement; tokens drawn before have w = 0 already), w is
// max(a p - b q, 0) throughout, and a child that is refused costs two numbers and one sum over the row.  Where nobody stands the next token is the first one at
// which the sum of w along the vocabulary passes u_root times the whole.
//
// A number next to a border decides about a token.  A draw has as many borders as the vocabulary has tokens, and with sums in 32 bits one draw in a hundred would fall on the other side of one:
// it is made from exponentials and sums in 64 bits (11 operations of that pipe a number, a sixth of a clock on an SM).  Whether a child stands is one comparison: it is made with sums of
// 32-bit exponentials first, and only where both sides are nearer to each other than those may be off, or where a child with drafts is refused, with the others.
// Sums are formed in an order that depends on the sizes alone.
//
// To read: the rows of the tokens on the path, and no others; which ones these are is known one after the other, so that what counts is how fast one row is read.  A
// cluster of CTAs shares the rows of a sequence; a row costs one pass with a running maximum and one exchange of partial maxima and sums between the CTAs, a child with drafts that is refused two
// more passes over what is then in the L2 cache.
#include <algorithm>
#include <type_traits>

#include "psa_cache.cuh"
#include "psa_internal.h"
#include "psa_sched.h"
#include "sm100.cuh"

namespace psa {

namespace {

constexpr int V_WARPS = 8, V_THREADS = 32 * V_WARPS;
constexpr int MOST_CLUSTER = 8;
// Relative error of a sum of 32-bit exponentials: their argument goes through two roundings of 2^-24 of itself, 30 at most where a weight counts (2^-18.6 of the weight), ex2 gives 2^-22, and a number
// takes part in no more than 8 + 64 additions before the sums go on in 64 bits (2^-17.8): below 2^-17 altogether.
constexpr double COARSE = 1.0 / 65536;

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

// What the CTAs of a cluster tell each other about a row.
struct Record {
    double p_sum, q_sum;
    float p_max, q_max;
    int likeliest, bad;
};

__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
    for (int s = 16; s > 0; s /= 2) x += __shfl_xor_sync(0xffffffffu, x, s);
    return x;
}
template <class X>
__device__ __forceinline__ X read_cluster(const X* p, uint32_t rank) {      // of CTA `rank`; X: words of 32 bits
    X x;
    const uint32_t a = cluster_map(p, rank);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(X) / 4); ++i) asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(reinterpret_cast<uint32_t*>(&x)[i]) : "r"(a + 4 * i) : "memory");
    return x;
}

// exp2(z / 32) for z <= 0, called by all lanes of a warp together, to 2^-50: 2^(k / 32) (1 + e) with k the nearest whole number, the power from a table of 32 (one a lane), e by its Taylor series
// (table-driven exponentials: Tang, 1989).
struct Exp {
    double power;                                // 2^(lane / 32)
    __device__ __forceinline__ Exp(int lane) : power(exp2(lane / 32.0)) {}
    __device__ __forceinline__ double operator()(double z) const {
        constexpr double L = 0.69314718055994530942 / 32;
        z = fmax(z, -32704.0);                   // 2^-1022
        const double t = z + 6755399441055744.0, s = z - (t - 6755399441055744.0);
        const int k = __double2loint(t);
        const double e = s * fma(s, fma(s, fma(s, fma(s, L * L * L * L * L / 120, L * L * L * L / 24), L * L * L / 6), L * L / 2), L);
        const double p = __hiloint2double(__shfl_sync(0xffffffffu, __double2hiint(power), k & 31), __shfl_sync(0xffffffffu, __double2loint(power), k & 31));
        const double w = fma(p, e, p);
        return k <= -32672 ? 0.0 : __hiloint2double(__double2hiint(w) + (k >> 5) * 1048576, __double2loint(w));
    }
};

// f(number of the first row, number of the second, v, whether there is such a v) for v = low .. high - 1, by a warp, every call by all lanes.  The rows may begin anywhere: up to a
// boundary of 16 bytes, and behind the last, numbers are read one by one, and all are where the rows lie differently.
template <class T, bool TWO, class F>
__device__ __forceinline__ void over(const T* p, const T* q, int low, int high, int lane, F f) {
    constexpr int VEC = 16 / sizeof(T);
    if (low >= high) return;
    const uintptr_t at = reinterpret_cast<uintptr_t>(p + low), too = TWO ? reinterpret_cast<uintptr_t>(q + low) : at;
    const bool alike = ((at ^ too) & 15u) == 0;
    const int lead = alike ? min((int)((16 - (at & 15u)) % 16 / sizeof(T)), high - low) : high - low, vecs = (high - low - lead) / VEC;
    auto singly = [&](int from, int to) {
        for (int v0 = from; v0 < to; v0 += 32) {
            const int v = v0 + lane;
            const bool is = v < to;
            f(is ? number(p[v]) : -INFINITY, TWO && is ? number(q[v]) : -INFINITY, v, is);
        }
    };
    singly(low, low + lead);
    const uint4* const p4 = reinterpret_cast<const uint4*>(p + low + lead);
    const uint4* const q4 = TWO ? reinterpret_cast<const uint4*>(q + low + lead) : p4;
    constexpr int AHEAD = 4;
    for (int i0 = 0; i0 < vecs; i0 += 32 * AHEAD) {
        uint4 x[AHEAD], y[TWO ? AHEAD : 1];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int i = min(i0 + 32 * k + lane, vecs - 1);
            x[k] = __ldg(p4 + i);
            if (TWO) y[TWO ? k : 0] = __ldg(q4 + i);
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (i0 + 32 * k >= vecs) break;
            const int i = i0 + 32 * k + lane;
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                f(i < vecs ? number(reinterpret_cast<const T*>(&x[k])[e]) : -INFINITY, TWO && i < vecs ? number(reinterpret_cast<const T*>(&y[TWO ? k : 0])[e]) : -INFINITY, low + lead + i * VEC + e,
                  i < vecs);
        }
    }
    singly(low + lead + vecs * VEC, high);
}

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Greatest number of a part of a row, the first place that has it (ARG), whether a number is NaN or infinite, and the sum of 2^(c (x - greatest)) in 32 bits (SUM).  Threads take vectors of 16 bytes in turn.
struct Part {
    float top;
    int arg;
    bool bad;
    double sum;
};
template <class T, bool GREEDY>
__device__ __forceinline__ Part part_of_row(const T* row, int low, int high, float c, int tid) {
    constexpr int VEC = 16 / sizeof(T);
    Part r = {-INFINITY, 0x7fffffff, false, 0.0};
    float sum = 0.f;
    int chains = 0;
    const uintptr_t at = reinterpret_cast<uintptr_t>(row + low);
    const int n = high - low, lead = min((int)((16 - (at & 15u)) % 16 / sizeof(T)), n), vecs = (n - lead) / VEC, done = lead + vecs * VEC;
    auto raise = [&](float m) {                  // a new greatest number
        const float f = r.top > -INFINITY ? exp2_fast(c * (r.top - m)) : 0.f;
        sum *= f;
        r.sum *= (double)f;
        r.top = m;
    };
    auto one = [&](int v) {
        const float x = number(row[v]);
        r.bad |= !(x <= 3.402823466e38f);
        if (GREEDY) {
            if (x > r.top || (x == r.top && v < r.arg)) { r.top = x; r.arg = v; }
        } else if (x > -INFINITY) {
            if (x > r.top) raise(x);
            sum += exp2_fast(c * (x - r.top));
        }
    };
    if (tid < lead) one(low + tid);
    const uint4* const row4 = reinterpret_cast<const uint4*>(row + low + lead);
    constexpr int AHEAD = 4;
    for (int i0 = 0; i0 < vecs; i0 += AHEAD * V_THREADS) {
        uint4 x[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (i0 + k * V_THREADS + tid < vecs) x[k] = __ldg(row4 + i0 + k * V_THREADS + tid);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int i = i0 + k * V_THREADS + tid;
            if (i >= vecs) break;
            float y[VEC], m = -INFINITY;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                y[e] = number(reinterpret_cast<const T*>(&x[k])[e]);
                r.bad |= !(y[e] <= 3.402823466e38f);
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
                if (m > r.top) raise(m);
                const float from = r.top > -INFINITY ? r.top : 0.f;
                float s = 0.f;
#pragma unroll
                for (int e = 0; e < VEC; ++e) s += exp2_fast(c * (y[e] - from));
                sum += s;
                if (++chains == 64) { r.sum += (double)sum; sum = 0.f; chains = 0; }
            }
        }
    }
    if (tid < n - done) one(low + done + tid);
    r.sum += (double)sum;
    return r;
}

template <class T>
__global__ void __launch_bounds__(V_THREADS) verify_kernel(const VerifyArgs a, DeviceCounters* dc, DeviceCounters* dc_next) {
    __shared__ int parent_s[PSA_TREE_MOST], token_s[PSA_TREE_MOST], tried_s[PSA_TREE_MOST];
    __shared__ double sums_s[V_WARPS], sums2_s[V_WARPS];
    __shared__ float max_s[V_WARPS], max2_s[V_WARPS];
    __shared__ int arg_s[V_WARPS], bad_s[V_WARPS], drawn_s;
    __shared__ Record records[2];               // told in turn

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

    const double C = greedy ? 1.0 : 46.166241308446828384 / (double)temperature;         // 32 / (T ln 2): units of Exp
    const float c = (float)(C / 32);
    const Exp exp_of(lane);
    const T* const all_logits = static_cast<const T*>(a.logits);
    const T* const all_drafts = static_cast<const T*>(a.drafts);
    const int low = min(rank * a.slice, a.vocab), high = min(low + a.slice, a.vocab);    // this CTA's part of the vocabulary
    const int each = (high - low + V_WARPS - 1) / V_WARPS;                               // of its warps, one after another
    const int w_low = min(low + warp * each, high), w_high = min(w_low + each, high);

    int turn = 0;                                // of records
    int node = 0, stood = 0, next = -1;
    for (;;) {
        const T* const lrow = all_logits + (size_t)(first + node) * a.logit_stride;
        bool leaf = true;
        for (int i = node + 1 + tid; i < count; i += V_THREADS) leaf &= parent_s[i] != node;
        leaf = !__syncthreads_or(!leaf);         // (also: what the token before left in shared memory is done with)
        const bool use_q = all_drafts && !greedy && !leaf;
        const T* const qrow = all_drafts + (use_q ? (size_t)(first + node) * a.draft_stride : 0);
        // ---- the rows' greatest numbers and sums: of the threads, the CTA, the cluster
        Part p = greedy ? part_of_row<T, true>(lrow, low, high, 0.f, tid) : part_of_row<T, false>(lrow, low, high, c, tid);
        Part q = {-INFINITY, 0, false, 0.0};
        if (use_q) q = part_of_row<T, false>(qrow, low, high, c, tid);
        auto warp_joined = [&](Part& x) {
            float top = x.top;
            int arg = x.arg;
#pragma unroll
            for (int s = 16; s > 0; s /= 2) {
                const float y = __shfl_xor_sync(0xffffffffu, top, s);
                const int k = __shfl_xor_sync(0xffffffffu, arg, s);
                if (y > top || (y == top && k < arg)) { top = y; arg = k; }
            }
            x.sum = warp_sum(x.top > -INFINITY ? x.sum * (double)exp2_fast(c * (x.top - top)) : 0.0);
            x.top = top;
            x.arg = arg;
            x.bad = __any_sync(0xffffffffu, x.bad);
        };
        warp_joined(p);
        if (use_q) warp_joined(q);
        if (lane == 0) { max_s[warp] = p.top; max2_s[warp] = q.top; arg_s[warp] = p.arg; bad_s[warp] = p.bad || q.bad; sums_s[warp] = p.sum; sums2_s[warp] = q.sum; }
        __syncthreads();
        if (tid == 0) {
            Record r = {0.0, 0.0, -INFINITY, -INFINITY, 0x7fffffff, 0};
            for (int w = 0; w < V_WARPS; ++w) {
                if (max_s[w] > r.p_max || (max_s[w] == r.p_max && arg_s[w] < r.likeliest)) { r.p_max = max_s[w]; r.likeliest = arg_s[w]; }
                r.q_max = fmaxf(r.q_max, max2_s[w]);
                r.bad |= bad_s[w];
            }
            for (int w = 0; w < V_WARPS; ++w) {
                if (max_s[w] > -INFINITY) r.p_sum += sums_s[w] * (double)exp2_fast(c * (max_s[w] - r.p_max));
                if (max2_s[w] > -INFINITY) r.q_sum += sums2_s[w] * (double)exp2_fast(c * (max2_s[w] - r.q_max));
            }
            records[turn] = r;
        }
        cluster_sync();
        float top = -INFINITY, q_top = -INFINITY;
        int arg = 0x7fffffff;
        bool bad = false;
        double p_sum = 0, q_sum = 0;
        {
            const Record r = lane < ranks ? read_cluster(&records[turn], lane) : Record{0.0, 0.0, -INFINITY, -INFINITY, 0x7fffffff, 0};
            top = r.p_max;
            arg = r.likeliest;
            q_top = r.q_max;
#pragma unroll
            for (int s = MOST_CLUSTER / 2; s > 0; s /= 2) {
                const float y = __shfl_xor_sync(0xffffffffu, top, s);
                const int k = __shfl_xor_sync(0xffffffffu, arg, s);
                if (y > top || (y == top && k < arg)) { top = y; arg = k; }
                q_top = fmaxf(q_top, __shfl_xor_sync(0xffffffffu, q_top, s));
            }
            bad = __any_sync(0xffffffffu, r.bad != 0);
            p_sum = r.p_max > -INFINITY ? r.p_sum * (double)exp2_fast(c * (r.p_max - top)) : 0.0;
            q_sum = r.q_max > -INFINITY ? r.q_sum * (double)exp2_fast(c * (r.q_max - q_top)) : 0.0;
#pragma unroll
            for (int s = MOST_CLUSTER / 2; s > 0; s /= 2) {
                p_sum += __shfl_xor_sync(0xffffffffu, p_sum, s);
                q_sum += __shfl_xor_sync(0xffffffffu, q_sum, s);
            }
            // (lanes from MOST_CLUSTER on hold nothing: the first one's are the cluster's)
            top = __shfl_sync(0xffffffffu, top, 0);
            arg = __shfl_sync(0xffffffffu, arg, 0);
            q_top = __shfl_sync(0xffffffffu, q_top, 0);
            p_sum = __shfl_sync(0xffffffffu, p_sum, 0);
            q_sum = __shfl_sync(0xffffffffu, q_sum, 0);
        }
        turn ^= 1;
        if (bad || top == -INFINITY || (use_q && q_top == -INFINITY)) {      // numbers that are no distribution
            if (rank == 0 && tid == 0) atomicExch(&dc->status, (int)PSA_ERR_NUMERIC);
            break;
        }
        // ---- in 64 bits: sums over the warps' parts into sums_s (and sums2_s), of all CTAs into the two results; every CTA tells its own
        const double p_top = top, q_high = use_q ? q_top : 0.f;
        double told[2];
        auto exchange = [&](double x, double y) {
            x = warp_sum(x);
            y = warp_sum(y);
            __syncthreads();
            if (lane == 0) { sums_s[warp] = x; sums2_s[warp] = y; }
            __syncthreads();
            if (tid == 0) {
                Record& r = records[turn];
                r.p_sum = r.q_sum = 0;
                for (int w = 0; w < V_WARPS; ++w) { r.p_sum += sums_s[w]; r.q_sum += sums2_s[w]; }
            }
            cluster_sync();
            const double mine = lane < ranks ? read_cluster(&records[turn].p_sum, lane) : 0.0, mine2 = lane < ranks ? read_cluster(&records[turn].q_sum, lane) : 0.0;
            told[0] = told[1] = 0;
            for (int k = 0; k < ranks; ++k) {
                told[0] += __shfl_sync(0xffffffffu, mine, k);
                told[1] += __shfl_sync(0xffffffffu, mine2, k);
            }
            turn ^= 1;
        };
        bool sharp = false;                      // p_sum and q_sum are in 64 bits
        auto sharpen = [&] {
            if (sharp) return;
            sharp = true;
            double x = 0, y = 0;
            over<T, false>(lrow, nullptr, w_low, w_high, lane, [&](float l, float, int, bool is) { const double w = exp_of(((double)l - p_top) * C); x += is ? w : 0.0; });
            if (use_q) over<T, false>(qrow, nullptr, w_low, w_high, lane, [&](float l, float, int, bool is) { const double w = exp_of(((double)l - q_high) * C); y += is ? w : 0.0; });
            exchange(x, y);
            p_sum = told[0];
            q_sum = told[1];
        };
        // ---- w = max(ka p - kb q, 0), or p without the children that were refused; not divided by p's sum
        double ka = 1, kb = 0, Z = 1, rest = 1;
        int tried = 0;
        bool only_p = true;                      // nothing was refused yet, or nothing is left
        double over_q = 0;                       // p_sum / q_sum
        auto weight = [&](float l, float g, int v, bool is) -> double {
            const double pw = exp_of(((double)l - p_top) * C);
            if (!only_p && use_q) {
                const double qw = exp_of(((double)g - q_high) * C);          // (by all lanes, also those that have no v)
                return is ? fmax(ka * pw - kb * over_q * qw, 0.0) : 0.0;
            }
            bool gone = !is;
            if (!only_p)
                for (int k = 0; k < tried; ++k) gone |= tried_s[k] == v;
            return gone ? 0.0 : pw;
        };
        auto sum_weights = [&]() -> double {
            double s = 0;
            if (!only_p && use_q) over<T, true>(lrow, qrow, w_low, w_high, lane, [&](float l, float g, int v, bool is) { s += weight(l, g, v, is); });
            else over<T, false>(lrow, nullptr, w_low, w_high, lane, [&](float l, float g, int v, bool is) { s += weight(l, g, v, is); });
            exchange(s, 0.0);
            return told[0];
        };
        int taken = -1;
        bool summed = false, nothing = false;
        for (int i = node + 1; i < count && taken < 0 && !nothing; ++i) {
            if (parent_s[i] != node || token_s[i] < 0) continue;
            const int x = token_s[i];
            if (greedy) {
                if (x == arg) taken = i;
                continue;
            }
            bool again = false;                  // a sibling with the same token was refused: nothing is left of it
            if (!use_q || a.distinct)
                for (int k = 0; k < tried; ++k) again |= tried_s[k] == x;
            if (again) continue;
            const double u = a.uniform[first + i], px = exp_of(((double)number(lrow[x]) - p_top) * C);
            const double qx = use_q ? exp_of(((double)number(qrow[x]) - q_high) * C) : 0.0, part = use_q && a.distinct ? 1.0 / fmax(rest, 1e-300) : 1.0;
            double left, right;
            auto sides = [&] {
                left = use_q ? u * (qx / q_sum * part) * Z : u * Z;
                right = only_p || !use_q ? px / p_sum : fmax(ka * (px / p_sum) - kb * (qx / q_sum), 0.0);
            };
            sides();
            if (!sharp && fabs(left - right) <= 3 * COARSE * (use_q ? fmax(left, right) : 1.0)) {
                sharpen();
                sides();
            }
            if (left < right) { taken = i; continue; }
            if (use_q) {
                sharpen();
                kb = kb / Z + part;
                ka = ka / Z;
                rest -= qx / q_sum;
            } else {
                Z -= px / p_sum;
            }
            __syncthreads();
            if (tid == 0) tried_s[tried] = x;
            ++tried;
            __syncthreads();
            only_p = false;
            if (use_q) {
                over_q = p_sum / q_sum;
                Z = sum_weights() / p_sum;
                summed = true;
                nothing = !(Z > 0);
            }
        }
        if (taken >= 0) {
            node = taken;
            ++stood;
            if (rank == 0 && tid == 0) a.path[first + stood] = taken;
            continue;
        }
        if (greedy) {
            next = arg;
            break;
        }
        // ---- the draw: the first token at which the running sum of w passes u times the whole
        if (nothing) { only_p = true; summed = false; }
        double all = summed ? told[0] : sum_weights();
        if (!(all > 0)) { only_p = true; all = sum_weights(); }              // (all of p refused)
        // which CTA, then which warp's part; where roundings leave none behind the target, the last one with any weight
        double target = (double)a.uniform[first] * all, before = 0;
        int owner = -1, last = 0;
        for (int k = 0; k < ranks && owner < 0; ++k) {
            const double s = read_cluster(&records[turn ^ 1].p_sum, k);
            if (s > 0) last = k;
            if (s > 0 && before + s > target) owner = k; else before += s;
        }
        bool end = owner < 0;                    // the last one with any weight is meant
        if (end) owner = last;
        if (owner == rank) {
            auto pick = [&](const double* sums) {        // of the warps' parts; target: from there on
                int part = -1;
                before = 0;
                last = 0;
                for (int w = 0; w < V_WARPS && part < 0; ++w) {
                    if (sums[w] > 0) last = w;
                    if (!end && sums[w] > 0 && before + sums[w] > target) part = w; else before += sums[w];
                }
                if (part < 0) { part = last; end = true; }
                target -= before;
                return part;
            };
            target -= before;
            const int part = pick(sums_s);
            // that part once more, an eighth a warp
            const bool two = !only_p && use_q;
            const int p_low = min(low + part * each, high), p_high = min(p_low + each, high), fine = (p_high - p_low + V_WARPS - 1) / V_WARPS;
            const int f_low = min(p_low + warp * fine, p_high), f_high = min(f_low + fine, p_high);
            auto at = [&](int v) { const bool is = v < f_high; return weight(is ? number(lrow[v]) : -INFINITY, is && two ? number(qrow[v]) : -INFINITY, v, is); };
            double s = 0;
            for (int v0 = f_low; v0 < f_high; v0 += 32) s += at(v0 + lane);
            s = warp_sum(s);
            __syncthreads();
            if (lane == 0) sums2_s[warp] = s;
            __syncthreads();
            if (warp == pick(sums2_s)) {
                before = 0;
                int found = -1, some = -1;
                for (int v0 = f_low; v0 < f_high && found < 0; v0 += 32) {
                    const double x = at(v0 + lane);
                    double sum = x;
#pragma unroll
                    for (int k = 1; k < 32; k *= 2) {
                        const double y = __shfl_up_sync(0xffffffffu, sum, k);
                        if (lane >= k) sum += y;
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
        cluster_sync();                          // (nobody leaves while its shared memory is read)
        return;
    }
    if (rank == 0 && tid == 0) {
        a.accepted[b] = stood;
        a.next[b] = next;
    }
    cluster_sync();
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
// One sequence, by a warp: its path ascends from 0 and ends inside the tree.
__device__ __forceinline__ Kept kept_of(const KeepArgs& a, int b, int lane) {
    Kept k;
    k.slot = a.seqs[b];
    k.first = min(max(a.starts[b], 0), a.rows);
    k.count = max(min(max(a.starts[b + 1], 0), a.rows) - k.first, 0);
    const bool known = k.slot >= 0 && k.slot < a.slots;
    const int len = known ? a.lens[k.slot] : 0;
    k.base = len - k.count;
    k.keep = 0;
    const int stand = a.accepted[b];
    if (!known || k.base < 0 || (long long)len > (long long)a.width * a.page_size || stand < 0 || stand >= k.count) return k;
    bool good = true;
    for (int i = lane; i <= stand; i += 32) {
        const int p = a.path[k.first + i];
        good &= i == 0 ? p == 0 : p > a.path[k.first + i - 1] && p < k.count;
    }
    if (__all_sync(0xffffffffu, good)) k.keep = stand + 1;
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
        // where the lane's elements of a token lie: behind its block's beginning, for an even token and an odd one
        auto place = [&](int round, int tok) {
            const int e = round * 32 + lane;
            if (e < 4 * G) return B::K_CODES + tok * (D / 2) + 4 * e;
            if (e < WORDS) return B::K_SCALES + tok * 4 * G + 4 * (e - 4 * G);
            if (e < WORDS + 8 * G) return B::V_CODES + (tok >> 1) * D + 4 * (e - WORDS) + 2 * (tok & 1);
            return B::V_SCALES + (tok >> 1) * 8 * G + 4 * (e - WORDS - 8 * G) + 2 * (tok & 1);
        };
        for (int i0 = 0; i0 < k.keep; i0 += KEEP_TOKENS) {
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
#pragma unroll
                for (int r = 0; r < ROUNDS; ++r) {
                    const int e = r * 32 + lane;
                    x[t][r] = 0;
                    if (to[t] && e < WORDS) x[t][r] = *reinterpret_cast<const uint32_t*>(from + place(r, from_tok));
                    else if (to[t] && e < WORDS + HALVES) x[t][r] = *reinterpret_cast<const uint16_t*>(from + place(r, from_tok));
                }
            }
            __syncwarp();
#pragma unroll
            for (int t = 0; t < KEEP_TOKENS; ++t)
#pragma unroll
                for (int r = 0; r < ROUNDS; ++r) {
                    const int e = r * 32 + lane;
                    if (to[t] && e < WORDS) *reinterpret_cast<uint32_t*>(to[t] + place(r, to_tok[t])) = x[t][r];
                    else if (to[t] && e < WORDS + HALVES) *reinterpret_cast<uint16_t*>(to[t] + place(r, to_tok[t])) = (uint16_t)x[t][r];
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
    if (last_s)
        for (int b = warp; b < a.sequences; b += KEEP_WARPS) {
            const Kept k = kept_of(a, b, lane);
            __syncwarp();
            if (lane == 0 && k.keep > 0) a.new_lens[k.slot] = k.base + k.keep;
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
    // as many CTAs a sequence as the GPU holds at a time, two an SM, of 2048 numbers at least
    int ranks = 1;
    while (ranks < MOST_CLUSTER && 2LL * ranks * a.sequences <= 2 * 148 && a.vocab > 2048 * ranks) ranks *= 2;
    a.slice = ((a.vocab + ranks - 1) / ranks + 7) / 8 * 8;
    cudaLaunchAttribute attr[2];
    for (int b0 = 0; b0 < a.sequences; b0 += 65535) {
        VerifyArgs x = a;
        x.sequences = std::min(a.sequences - b0, 65535);
        x.starts += b0;
        x.accepted += b0;
        x.next += b0;
        if (x.temperatures) x.temperatures += b0;
        const cudaLaunchConfig_t cfg = config(dim3(ranks, x.sequences), V_THREADS, 0, stream, attr, ranks);
        const cudaError_t e = cudaLaunchKernelEx(&cfg, verify_kernel<T>, x, dc, b0 == 0 ? dc_next : nullptr);
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
