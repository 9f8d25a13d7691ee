// Drafted tokens: which of a tree's tokens stand (psa_verify_drafts), and what the cache keeps of them (psa_cache_keep).
//
// Verification walks a sequence's tree from its root.  At a token with target probabilities p = softmax(logits / T) and children x_1, x_2, .. (drawn from draft
// probabilities q = softmax(drafts / T)), child x_m stands if u_m q_m(x_m) < w(x_m) / Z, where w = p, Z = 1 at first, and behind every child that does not stand
//     w <- max(w / Z - q_m, 0),   Z <- sum_v w(v).
// As q_m is q times a number (1, or 1 / (1 - what was drawn before) where siblings are drawn without replacement; tokens drawn before have w = 0 already), w is
// max(a p - b q, 0) throughout, and a child that is refused costs two numbers and one sum over the row.  Where nobody stands the next token is the first one at
// which the sum of w along the vocabulary passes u_root times the whole.
//
// A number next to a border decides about a token, so exponentials and sums are in 64 bits: the sums along the row have up to 10^5 borders, and with an error of
// 2^-24 of a likely token's weight one draw in a hundred would fall on the other side of one.  Sums are formed in an order that depends on the sizes alone.
//
// To read: the rows of the tokens on the path, and no others; which ones these are is known one after the other, so that what counts is how fast one row is read.  A
// cluster of CTAs shares the rows of a sequence, each a part that it keeps in shared memory while the token is looked at; a row costs one exchange of partial maxima and sums
// between the CTAs, a child that is refused another.
#include <algorithm>
#include <type_traits>

#include "psa_cache.cuh"
#include "psa_internal.h"
#include "psa_sched.h"
#include "sm100.cuh"

namespace psa {

namespace {

constexpr int V_WARPS = 16, V_THREADS = 32 * V_WARPS;
constexpr int MOST_CLUSTER = 8;
constexpr int MOST_SLICE_BYTES = 100 * 1024;    // of a row's part that is kept in shared memory, target and drafts each

struct VerifyArgs {
    const void *logits, *drafts;
    long long logit_stride, draft_stride;
    const int *tokens, *parents, *starts;
    const float *temperatures, *uniform;
    int *path, *accepted, *next;
    int vocab, sequences, rows, distinct;
    int slice;                                  // of a CTA: numbers of the vocabulary
    int staged;                                 // the parts of a row are kept in shared memory
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

template <class T>
__global__ void __launch_bounds__(V_THREADS) verify_kernel(const VerifyArgs a, DeviceCounters* dc, DeviceCounters* dc_next) {
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ int parent_s[PSA_TREE_MOST], token_s[PSA_TREE_MOST], tried_s[PSA_TREE_MOST];
    __shared__ double sums_s[V_WARPS], sums2_s[V_WARPS];
    __shared__ float max_s[V_WARPS], max2_s[V_WARPS];
    __shared__ int arg_s[V_WARPS], bad_s[V_WARPS], drawn_s;
    __shared__ Record records[2];               // told in turn
    __shared__ double totals[2];

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int ranks = (int)gridDim.x, rank = (int)blockIdx.x, b = (int)blockIdx.y;       // (a cluster is a row of the grid)
    grid_dependency_wait();
    if (tid == 0 && rank == 0 && b == 0 && dc_next) *dc_next = DeviceCounters{0, 0, 0, 0, 0, 0, 0};
    const int first = min(max(a.starts[b], 0), a.rows), count = max(min(max(a.starts[b + 1], 0), a.rows) - first, 0);
    const float temperature = a.temperatures ? a.temperatures[b] : 1.f;
    const bool greedy = temperature == 0.f;
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
    const double c = greedy ? 1.0 : 1.0 / (double)temperature;
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

    const T* const all_logits = static_cast<const T*>(a.logits);
    const T* const all_drafts = static_cast<const T*>(a.drafts);
    const int low = min(rank * a.slice, a.vocab), high = min(low + a.slice, a.vocab);    // this CTA's part of the vocabulary
    const int each = (high - low + V_WARPS - 1) / V_WARPS;                               // of its warps, one after another
    const int w_low = min(low + warp * each, high), w_high = min(w_low + each, high);
    constexpr int VEC = 16 / sizeof(T);

    int turn = 0;                                // of records and totals
    int node = 0, stood = 0, next = -1;
    for (;;) {
        const T* const lrow = all_logits + (size_t)(first + node) * a.logit_stride;
        bool leaf = true;
        for (int i = node + 1 + tid; i < count; i += V_THREADS) leaf &= parent_s[i] != node;
        leaf = !__syncthreads_or(!leaf);
        const bool use_q = all_drafts && !greedy && !leaf;
        const T* const qrow = all_drafts + (use_q ? (size_t)(first + node) * a.draft_stride : 0);
        // ---- the row's part into shared memory (at the place in 16 bytes that it has in memory), its greatest number
        const T *lp = lrow, *qp = qrow;          // the part's number v is lp[v]
        float top = -INFINITY, q_top = -INFINITY;
        int arg = 0x7fffffff;
        bool bad = false;
        auto fetch = [&](const T* row, uint8_t* to, float& m, bool with_arg) -> const T* {
            const T* const from = row + low;
            const int n = high - low, shift = (int)((reinterpret_cast<uintptr_t>(from) & 15u) / sizeof(T)), lead = min((VEC - shift) % VEC, n), vecs = (n - lead) / VEC;
            T* const dst = reinterpret_cast<T*>(to) + shift;
            auto look = [&](T x, int v) {
                const float f = number(x);
                bad |= !(f <= 3.402823466e38f);
                if (f > m) { m = f; if (with_arg) arg = v; }
            };
            if (tid < lead) { if (a.staged) dst[tid] = from[tid]; look(from[tid], low + tid); }
            const uint4* const src4 = reinterpret_cast<const uint4*>(from + lead);
            uint4* const dst4 = reinterpret_cast<uint4*>(dst + lead);
            constexpr int AHEAD = 4;
            for (int i = tid; i < vecs; i += AHEAD * V_THREADS) {
                uint4 x[AHEAD];
#pragma unroll
                for (int k = 0; k < AHEAD; ++k)
                    if (i + k * V_THREADS < vecs) x[k] = __ldg(src4 + i + k * V_THREADS);
#pragma unroll
                for (int k = 0; k < AHEAD; ++k)
                    if (i + k * V_THREADS < vecs) {
                        if (a.staged) dst4[i + k * V_THREADS] = x[k];
#pragma unroll
                        for (int e = 0; e < VEC; ++e) look(reinterpret_cast<const T*>(&x[k])[e], low + lead + (i + k * V_THREADS) * VEC + e);
                    }
            }
            const int done = lead + vecs * VEC;
            if (tid < n - done) { if (a.staged) dst[done + tid] = from[done + tid]; look(from[done + tid], low + done + tid); }
            return a.staged ? dst - low : row;
        };
        __syncthreads();                         // (the part before is done with)
        const int part_bytes = (a.slice * (int)sizeof(T) + 31) / 16 * 16;
        lp = fetch(lrow, smem, top, greedy);
        if (use_q) qp = fetch(qrow, smem + part_bytes, q_top, false);
        // greatest numbers of the CTA; of equal ones the first
#pragma unroll
        for (int s = 16; s > 0; s /= 2) {
            const float y = __shfl_xor_sync(0xffffffffu, top, s), z = __shfl_xor_sync(0xffffffffu, q_top, s);
            const int k = __shfl_xor_sync(0xffffffffu, arg, s);
            if (y > top || (y == top && k < arg)) { top = y; arg = k; }
            q_top = fmaxf(q_top, z);
        }
        bad = __any_sync(0xffffffffu, bad);
        if (lane == 0) { max_s[warp] = top; max2_s[warp] = q_top; arg_s[warp] = arg; bad_s[warp] = bad; }
        __syncthreads();
        top = q_top = -INFINITY;
        arg = 0x7fffffff;
        bad = false;
        for (int w = 0; w < V_WARPS; ++w) {
            if (max_s[w] > top || (max_s[w] == top && arg_s[w] < arg)) { top = max_s[w]; arg = arg_s[w]; }
            q_top = fmaxf(q_top, max2_s[w]);
            bad |= bad_s[w] != 0;
        }
        // ---- its sums
        double p_sum = 0, q_sum = 0;
        if (!greedy && !bad) {
            if (top > -INFINITY)
                for (int v = w_low + lane; v < w_high; v += 32) p_sum += exp(((double)number(lp[v]) - (double)top) * c);
            if (use_q && q_top > -INFINITY)
                for (int v = w_low + lane; v < w_high; v += 32) q_sum += exp(((double)number(qp[v]) - (double)q_top) * c);
            p_sum = warp_sum(p_sum);
            q_sum = warp_sum(q_sum);
        }
        if (lane == 0) { sums_s[warp] = p_sum; sums2_s[warp] = q_sum; }
        __syncthreads();
        p_sum = q_sum = 0;
        for (int w = 0; w < V_WARPS; ++w) { p_sum += sums_s[w]; q_sum += sums2_s[w]; }
        // ---- of all CTAs
        if (tid == 0) records[turn] = Record{p_sum, q_sum, top, q_top, arg, bad};
        cluster_sync();
        {
            float t = -INFINITY, qt = -INFINITY;
            arg = 0x7fffffff;
            for (int k = 0; k < ranks; ++k) {
                const Record r = read_cluster(&records[turn], k);
                if (r.p_max > t || (r.p_max == t && r.likeliest < arg)) { t = r.p_max; arg = r.likeliest; }
                qt = fmaxf(qt, r.q_max);
                bad |= r.bad != 0;
            }
            p_sum = q_sum = 0;
            for (int k = 0; k < ranks; ++k) {
                const Record r = read_cluster(&records[turn], k);
                if (r.p_max > -INFINITY) p_sum += r.p_sum * exp(((double)r.p_max - (double)t) * c);
                if (r.q_max > -INFINITY) q_sum += r.q_sum * exp(((double)r.q_max - (double)qt) * c);
            }
            top = t;
            q_top = qt;
        }
        turn ^= 1;
        if (bad || top == -INFINITY || (use_q && q_top == -INFINITY)) {      // numbers that are no distribution
            if (rank == 0 && tid == 0) atomicExch(&dc->status, (int)PSA_ERR_NUMERIC);
            break;
        }
        const double p_scale = 1.0 / p_sum, q_scale = use_q ? 1.0 / q_sum : 0.0;
        auto p_of = [&](float l) { return exp(((double)l - (double)top) * c) * p_scale; };
        auto q_of = [&](float g) { return exp(((double)g - (double)q_top) * c) * q_scale; };
        // ---- w = max(ka p - kb q, 0), or p without the children that were refused
        double ka = 1, kb = 0, Z = 1, rest = 1;
        int tried = 0;
        bool only_p = true;                      // nothing was refused yet, or nothing is left
        auto weight = [&](int v) -> double {
            const double p = p_of(number(lp[v]));
            if (only_p) return p;
            if (use_q) return fmax(ka * p - kb * q_of(number(qp[v])), 0.0);
            for (int k = 0; k < tried; ++k)
                if (tried_s[k] == v) return 0.0;
            return p;
        };
        // Sums of w over the warps' parts into sums_s; the CTA's own; of all CTAs (every CTA tells its own).
        double own_sum = 0;
        auto sum_weights = [&]() -> double {
            double s = 0;
            for (int v = w_low + lane; v < w_high; v += 32) s += weight(v);
            s = warp_sum(s);
            __syncthreads();
            if (lane == 0) sums_s[warp] = s;
            __syncthreads();
            own_sum = 0;
            for (int w = 0; w < V_WARPS; ++w) own_sum += sums_s[w];
            if (tid == 0) totals[turn] = own_sum;
            cluster_sync();
            double all = 0;
            for (int k = 0; k < ranks; ++k) all += read_cluster(&totals[turn], k);
            turn ^= 1;
            return all;
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
            const double u = a.uniform[first + i], px = p_of(number(lrow[x]));
            if (!use_q) {
                if (u * Z < px) { taken = i; continue; }
                Z -= px;
            } else {
                const double qx = q_of(number(qrow[x])), part = a.distinct ? 1.0 / fmax(rest, 1e-300) : 1.0;
                if (u * (qx * part) * Z < (only_p ? px : fmax(ka * px - kb * qx, 0.0))) { taken = i; continue; }
                kb = kb / Z + part;
                ka = ka / Z;
                rest -= qx;
            }
            __syncthreads();
            if (tid == 0) tried_s[tried] = x;
            ++tried;
            __syncthreads();
            only_p = false;
            summed = false;
            if (use_q) {
                Z = sum_weights();
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
        double all = summed ? Z : sum_weights();
        if (!(all > 0)) { only_p = true; all = sum_weights(); }              // (all of p refused)
        // which CTA, then which warp's part; where roundings leave none behind the target, the last one with any weight
        double target = (double)a.uniform[first] * all, before = 0;
        int owner = -1, last = 0;
        for (int k = 0; k < ranks && owner < 0; ++k) {
            const double s = read_cluster(&totals[turn ^ 1], k);
            if (s > 0) last = k;
            if (s > 0 && before + s > target) owner = k; else before += s;
        }
        bool end = owner < 0;                    // the last one with any weight is meant
        if (end) owner = last;
        if (owner == rank) {
            target -= before;
            before = 0;
            int part = -1;
            last = 0;
            for (int w = 0; w < V_WARPS && part < 0; ++w) {
                if (sums_s[w] > 0) last = w;
                if (!end && sums_s[w] > 0 && before + sums_s[w] > target) part = w; else before += sums_s[w];
            }
            if (part < 0) { part = last; end = true; }
            target -= before;
            // that part once more, a sixteenth a warp
            const int p_low = min(low + part * each, high), p_high = min(p_low + each, high), fine = (p_high - p_low + V_WARPS - 1) / V_WARPS;
            const int f_low = min(p_low + warp * fine, p_high), f_high = min(f_low + fine, p_high);
            double s = 0;
            for (int v = f_low + lane; v < f_high; v += 32) s += weight(v);
            s = warp_sum(s);
            if (lane == 0) sums2_s[warp] = s;
            __syncthreads();
            before = 0;
            part = -1;
            last = 0;
            for (int w = 0; w < V_WARPS && part < 0; ++w) {
                if (sums2_s[w] > 0) last = w;
                if (!end && sums2_s[w] > 0 && before + sums2_s[w] > target) part = w; else before += sums2_s[w];
            }
            if (part < 0) { part = last; end = true; }
            target -= before;
            if (warp == part) {
                before = 0;
                int found = -1, some = -1;
                for (int v0 = f_low; v0 < f_high && found < 0; v0 += 32) {
                    const double x = v0 + lane < f_high ? weight(v0 + lane) : 0.0;
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
            next = drawn_s;
            if (tid == 0) a.next[b] = next;
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
    static DeviceSetup setup;
    const int sms = device_setup(&setup, [] {
        return cudaFuncSetAttribute(verify_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * (MOST_SLICE_BYTES + 32));
    }, "verification set-up");
    if (sms <= 0) return PSA_ERR_CUDA;
    // as many CTAs a sequence as fit the GPU, of 2048 numbers at least
    int ranks = 1;
    while (ranks < MOST_CLUSTER && 2LL * ranks * a.sequences <= sms && a.vocab > 2048 * ranks) ranks *= 2;
    a.slice = ((a.vocab + ranks - 1) / ranks + 7) / 8 * 8;
    const size_t part = ((size_t)a.slice * sizeof(T) + 31) / 16 * 16;
    a.staged = part <= MOST_SLICE_BYTES;
    const size_t smem = a.staged ? part * (a.drafts ? 2 : 1) : 0;
    cudaLaunchAttribute attr[2];
    for (int b0 = 0; b0 < a.sequences; b0 += 65535) {
        VerifyArgs x = a;
        x.sequences = std::min(a.sequences - b0, 65535);
        x.starts += b0;
        x.accepted += b0;
        x.next += b0;
        if (x.temperatures) x.temperatures += b0;
        const cudaLaunchConfig_t cfg = config(dim3(ranks, x.sequences), V_THREADS, smem, stream, attr, ranks);
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
    const VerifyArgs a = {logits, drafts, logit_stride, draft_stride, tokens, parents, starts, temperatures, uniform, path, accepted, next, vocab, sequences, rows, distinct, 0, 0};
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
