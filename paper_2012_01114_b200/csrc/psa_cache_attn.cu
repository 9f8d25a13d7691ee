// Attention of a few query tokens of each sequence over its cache held in 4 bits (layout: psa_cache.cuh).
//
//     S_ij = scale q_i k_j,  w_ij = exp(S_ij),  out_i = sum_j w_ij v_j / sum_j w_ij,  j <= len - queries + i,  k_j and v_j being M + S (1 + c / 16)
//
// Bound by memory, if the instructions between the loads and the products stay few: at the measured 6.45 TB/s an SM gets 23 bytes of cache a clock, 37
// codes.  The heads of a group are the columns of one product, so that a code is looked at once for all of them:
//   phase 1  S^T = K Q^T     mma.m16n8k16, 16 tokens x 8 columns (heads of the group x query tokens).  The operand holds the codes themselves: four bits at the low
//                            end of a half are the subnormal fp16 number c 2^-24, one place further up c 2^-20, so that a mask is all that it takes; the
//                            queries carry the powers of two that belong to that.  S and M enter in fp32 behind the products of a group of 32 channels,
//                            S_w sum c q / 16, and by one more product, sum_w (M_w + S_w) (sum_w q) with the sums in two fp16 numbers each.  No rounding but
//                            that of Q to fp16, which a power of two per row keeps in range.
//   phase 2  running maximum and sum per column, 32 tokens at a time; the maximum is raised (and sums and output rescaled) only when a score passes it by 2^8
//   phase 3  O^T += V^T P^T  one fp16 fma per pair of codes gives v (rounded to fp16), the weights change sides by a transposing move.  (V's codes
//                            as the operand too, the weights times S, M by a product of its own, is 207 -> 170 instructions per block of 16 tokens and slower
//                            all the same, 49.0 -> 52.2 us and 33.1 -> 35.8 for the calls below: more that has to wait for another; and its error is
//                            2^-12 of a group's range instead of 2^-12 of the number.)
// Work is split over the long axis: a row (sequence, head, tile of columns) of more 32-token steps than a piece is cut into parts of equal length, the piece being chosen on the
// device from all lengths so that the parts fill the GPU (nothing has to be known on the host).  A CTA takes a part: its warps take the steps in turn, each with a
// ring of blocks of its own filled by bulk copies, and are joined through shared memory; a row of several parts is joined by the CTA that finishes last, in
// the parts' order, so that results do not depend on who that is.  Where there are more rows than CTAs, short ones go to single warps, eight a CTA (looking up, converting the
// queries and joining cost a CTA 8000 cycles a row, the 16 steps of a row of 512 tokens 7000).
// Measured, 32 heads on 8 of d = 128, one query each: two sequences of up to 131,072 tokens 49.1 us a call (204 MB: 4.2 TB/s; over a million tokens 5.3 TB/s, the
// loads without the products 6.4), 64 of up to 8000 32.0 us (68 MB: 2.2 TB/s).  59 % of the issue slots and 48 % of the memory's rate at the first size: warps wait for each
// other's slots, for results of a fixed latency and for the integer pipe in turn.
// What comes once a call: finding the parts 2.5 us, look-ups and queries 1.6, the CTA's join 3, the join of the parts 4 to 5.
#include <type_traits>

#include "psa_cache.cuh"
#include "psa_internal.h"
#include "psa_sched.h"
#include "sm100.cuh"

namespace psa {

namespace {

constexpr int WARPS = 8;                        // of a CTA.  (Four, twice as many CTAs: one sequence of 131,072 tokens, 8 heads of 128 47.8 -> 53.2 us, 64 of 1 to 8000 37.5 -> 43.0)
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float RAISE = 8.f;                    // log2 units, see phase 2
// Weights are held 2^HEADROOM times as large, and so are their sums: see HEADROOM in psa_prompt.cu.  2^(RAISE + HEADROOM) is half of what fp16 takes.
constexpr float HEADROOM = 7.f;
constexpr int STEP_BLOCKS = 2, STEP = STEP_BLOCKS * CACHE_BLOCK;              // blocks and tokens of a step
constexpr int MAX_CTAS = 148 * 4 + 64;          // partial results and arrival counts: two per CTA
constexpr int SEQ_BITS = 9, SEQS = 1 << SEQ_BITS;                            // sequences of one launch
constexpr int BRIEFS = 4;                       // see `brief`
constexpr int LONG_PIECE = 48;                  // see `crowded`
// Steps: a row up to LEAST_CUT is not cut, longer ones not into less than LEAST_PIECE.  (One sequence, 32 heads on 8 of d = 128 / 8 on 2 of 64, whole and in parts of 16: 600 tokens
// 9.4 10.6 / 7.4 9.1 us, 1000 11.2 11.1 / 8.7 9.4, 1300 13.5 11.0 / 10.1 9.4, 4000 26.7 11.1 / 19.9 9.4; in parts of 32: 13.8 / 11.5.)
constexpr int LEAST_CUT = 32, LEAST_PIECE = 16;
constexpr int MOST_ROWS = 1 << 30;              // of a call; parts are two per CTA more at most
constexpr int MOST_STEPS = 1 << 27;             // no row has as many

template <int D, int NT>
struct ACfg {
    static constexpr int COLS = 8 * NT, THREADS = 32 * WARPS;
    static constexpr int CTAS = (D * NT <= 128 ? 16 : 8) / WARPS;            // per SM: 128 registers a thread, or 255
    static constexpr int STAGES = D >= 256 || (D == 128 && NT == 1) ? 2 : D == 96 ? 3 : 4;       // steps that a warp has in flight or in hand
    static constexpr int STAGE_BYTES = STEP_BLOCKS * CacheBlock<D>::BYTES;
    static constexpr int RING = WARPS * STAGES * STAGE_BYTES;
    static constexpr int OPITCH = D + 4;        // floats between columns of the joining buffer (keeps its 16-byte stores off each other's banks)
    static constexpr int JOIN = WARPS * COLS * OPITCH * 4;
    static constexpr int SMEM = RING > JOIN ? RING : JOIN;
    static constexpr int MOST_PARTS = (SMEM - THREADS * 16) / (8 * COLS);    // of a row: two numbers a column each, and a result a thread
};

struct AttnArgs {
    const uint8_t* pool;
    const int *tables, *lens, *seqs, *q_starts;
    const uint16_t* q;
    uint16_t* out;
    float *lse, *part;                          // part: per part of a row [COLS][D] outputs, then [COLS] maxima and [COLS] sums
    long long q_stride;
    int pages, slots, width, page_size, kv_heads, group, sequences, rows, f16;
    int wide;                                   // the steps of all rows may be more than 32 bits count, by the tables' width (many rows and room for 2^20 tokens and more)
    float scale;
    FastDiv by_group, by_blocks;                // by query heads of a group, by blocks of a page
};

// Arrivals on a row of several parts, at the number of its first part.  Every arrival that completes a row wraps its count to zero again, and a CTA
// that gave up a wait arrives all the same: the counts are zero between calls.
__device__ unsigned g_arrived[2 * MAX_CTAS];

// Counts an arrival behind everything that the CTA's threads stored before the barrier ahead of it; true for the one that completes the row.
__device__ __forceinline__ bool arrive(unsigned* count, unsigned last) {
    unsigned old;
    asm volatile("fence.acq_rel.gpu;\n\tatom.acq_rel.gpu.global.inc.u32 %0, [%1], %2;" : "=r"(old) : "l"(count), "r"(last) : "memory");
    return old == last;
}

template <int N>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t (&r)[N]) {
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const uint4 v = *reinterpret_cast<const uint4*>(p + 4 * i);
            r[i] = v.x; r[i + 1] = v.y; r[i + 2] = v.z; r[i + 3] = v.w;
        }
    } else if constexpr (N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const uint2 v = *reinterpret_cast<const uint2*>(p + 4 * i);
            r[i] = v.x; r[i + 1] = v.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) r[i] = *reinterpret_cast<const uint32_t*>(p + 4 * i);
    }
}
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16816_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_weights(float lo, float hi) {      // (to fp16; never to infinity)
    uint32_t y;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(y) : "f"(hi), "f"(lo));
    return y;
}
__device__ __forceinline__ uint32_t h2_bits(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }
__device__ __forceinline__ __half2 bits_h2(uint32_t u) { return *reinterpret_cast<__half2*>(&u); }
__device__ __forceinline__ float finite_or_zero(float m) { return m == -INFINITY ? 0.f : m; }

// One sequence of the call: tokens held, query rows, tiles of columns, steps.
struct Seq {
    int slot, len, q0, nq, qtiles, steps, bad;   // bad: no such slot, or longer than its table
};
template <int COLS>
__device__ __forceinline__ Seq sequence(const AttnArgs& a, int b) {
    Seq s;
    s.slot = a.seqs[b];
    const bool there = s.slot >= 0 && s.slot < a.slots;
    s.q0 = min(max(a.q_starts[b], 0), a.rows);
    s.nq = max(min(max(a.q_starts[b + 1], 0), a.rows) - s.q0, 0);
    const int held = there ? max(a.lens[s.slot], 0) : 0;
    s.len = min(held, a.width * a.page_size);
    s.bad = !there || held != s.len;
    s.qtiles = (int)(((long long)s.nq * a.group + COLS - 1) / COLS);
    s.steps = max((int)(((uint32_t)s.len + STEP - 1) / STEP), 1);         // (a length may come within STEP of 2^31)
    return s;
}

// A part of a row: steps [step0, step1) of it, part `part` of `parts`, whose results have numbers `first`, `first` + 1, .. (if there are several).
struct Piece {
    Seq s;
    int h, qt, step0, step1, part, parts, first;
};
struct Totals {
    uint32_t steps, rows;
    float about;                                // AttnArgs::wide: the steps, which may be more than 32 bits count
};
__device__ __forceinline__ int parts_of(int steps, int piece) { return steps <= LEAST_CUT ? 1 : (int)((uint32_t)(steps + piece - 1) / (uint32_t)piece); }
// Item `r` of a sequence whose rows are cut into pieces of at most `piece` steps.
__device__ __forceinline__ Piece piece_of(const Seq& s, int r, int piece, int first) {
    const int parts = parts_of(s.steps, piece), row = parts == 1 ? r : r / parts, each = parts == 1 ? s.steps : (s.steps + parts - 1) / parts;
    Piece p;
    p.s = s;
    p.h = s.qtiles == 1 ? row : row / s.qtiles;
    p.qt = row - p.h * s.qtiles;
    p.part = r - row * parts;
    p.parts = parts;
    p.step0 = p.part * each;
    p.step1 = min(p.step0 + each, s.steps);
    p.first = first + row * parts;
    return p;
}

// MANY: there may be more items than CTAs, that is, rows by more than a half (parts are no more than CTAs by a half).  (Without it the loop has less to keep: two sequences of up to 131,072 tokens 50.2 -> 49.1 us, eight of up to 8000 14.0 -> 13.6.)
template <int D, int NT, bool MANY>
__global__ void __launch_bounds__(ACfg<D, NT>::THREADS, ACfg<D, NT>::CTAS)
cache_attn_kernel(const AttnArgs a, DeviceCounters* dc, DeviceCounters* dc_next) {
    using Cfg = ACfg<D, NT>;
    using B = CacheBlock<D>;
    constexpr int G = B::G, GQ = (G + 3) / 4, COLS = Cfg::COLS, ST = Cfg::STAGES, THREADS = Cfg::THREADS;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ uint64_t full[WARPS][ST];
    __shared__ float m_s[WARPS][COLS], l_s[WARPS][COLS], top_s[COLS], sum_s[COLS];
    __shared__ unsigned long long scan_s[WARPS];
    __shared__ Totals total_s[WARPS];
    __shared__ uint32_t briefs_s[2 * BRIEFS];
    __shared__ uint2 seq_s[MANY ? SEQS : 1];     // of the sequences: steps and tiles of columns of a row; then steps of an item, and items of a head * 2 + whether rows are cut
    __shared__ __align__(16) uint32_t unsorted_s[SEQS];                      // steps of a sequence's items << SEQ_BITS | SEQS - 1 - sequence
    __shared__ uint16_t order_s[SEQS];                                       // where items are handed out: the sequences, longest items first
    __shared__ int abort_flag, last_s;
    __shared__ int base_s[SEQS + 1], split_s[SEQS];                          // items ahead of a sequence, and parts that are joined with others
    __shared__ Piece pieces[2], own_s[WARPS];                                // of the CTA, this one and the next; of the warps, where each has a row of its own
    __shared__ int item_s[2];                                                // this item and the next, -1: none

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    if (tid < 2 * BRIEFS) briefs_s[tid] = 0;
    if (tid == 0) {
        abort_flag = 0;
        for (int w = 0; w < WARPS; ++w)
            for (int s = 0; s < ST; ++s) mbar_init(&full[w][s], STEP_BLOCKS);
        fence_mbar_init();
    }
    volatile int* abortp = &abort_flag;
    grid_dependency_wait();
    if (tid == 0 && blockIdx.x == 0 && dc_next) *dc_next = DeviceCounters{0, 0, 0, 0, 0, 0, 0};

    // ---- the list: how long a piece is, and the items ahead of every sequence
    auto block_scan = [&](unsigned long long v, unsigned long long* total) {                 // exclusive; two 32-bit sums at a time
        unsigned long long x = v;
#pragma unroll
        for (int s = 1; s < 32; s *= 2) {
            const unsigned long long y = __shfl_up_sync(0xffffffffu, x, s);
            if (lane >= s) x += y;
        }
        __syncthreads();
        if (lane == 31) scan_s[warp] = x;
        __syncthreads();
        unsigned long long before = 0, all = 0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) { if (w < warp) before += scan_s[w]; all += scan_s[w]; }
        *total = all;
        return before + x - v;
    };
    Seq s0 = {};                                 // sequence tid
    uint32_t steps = 0, rows = 0;
    float about = 0.f;
    bool descends = false;
    for (int b = tid; b < a.sequences; b += THREADS) {
        const Seq x = sequence<COLS>(a, b);
        descends |= a.q_starts[b + 1] < a.q_starts[b];
        if (b == tid) s0 = x;
        if (MANY) seq_s[b] = make_uint2((uint32_t)x.steps, (uint32_t)x.qtiles);
        const uint32_t r = (uint32_t)x.qtiles * a.kv_heads;
        steps += r * x.steps;
        rows += r;
        about = fmaf((float)r, (float)x.steps, about);
    }
    if (a.wide)
#pragma unroll
        for (int s = 1; s < 32; s *= 2) about += __shfl_xor_sync(0xffffffffu, about, s);
    steps = __reduce_add_sync(0xffffffffu, steps);
    rows = __reduce_add_sync(0xffffffffu, rows);
    if (lane == 0) total_s[warp] = Totals{steps, rows, about};
    if (__syncthreads_or(descends)) {            // rows counted more than once: the numbers below would not hold; nothing is computed, and the call reports it
        if (tid == 0) atomicExch(&dc->status, (int)PSA_ERR_SHAPE);
        return;
    }
    steps = rows = 0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) { steps += total_s[w].steps; rows += total_s[w].rows; }
    bool beyond = false;                         // more steps than 32 bits count
    if (a.wide) {
        about = 0.f;
        for (int w = 0; w < WARPS; ++w) about += total_s[w].about;
        beyond = about > 2.0e9f;
    }
    // (steps + up) / n, there somewhat more
    auto share_of_steps = [&](uint32_t n, uint32_t up) -> int { return beyond ? (int)fminf(__fdividef(about * 1.0001f, (float)n) + 1.f, (float)MOST_STEPS) : (int)((steps + up) / n); };
    // Rows cut into pieces of steps / (CTAs - rows) make no more parts than there are CTAs.  Where rows alone are that many, or leave so few CTAs that pieces get long, they are
    // cut into more parts than that, and items are handed out one by one, the longest first.  (us a call, one query, 32 heads on 8 of d = 128, by the first rule alone and so:
    // 30 sequences of up to 8000 tokens 39.3 and 28.1, 32 of up to 2000 20.3 and 15.9; what looking costs where pieces are short: 20 of up to 4000 13.0 and 13.7.)
    const uint32_t ctas = min(gridDim.x, (uint32_t)Cfg::MOST_PARTS), half = (ctas + 1) / 2;
    auto piece_of_budget = [&](uint32_t budget) { return max(share_of_steps(budget, budget - 1), LEAST_PIECE); };
    int piece = piece_of_budget(rows < ctas ? ctas - rows : half);
    const bool crowded = MANY && (rows >= ctas || (rows > half && piece > LONG_PIECE));
    if (crowded) piece = piece_of_budget(half);
    bool sorted = MANY && rows > gridDim.x;
    // Rows up to `brief` steps are a warp's, eight to an item: a warp's share of all steps, or the first of 1, 2, 4 and 8 with which the CTAs need one item each, else 8.
    // (A CTA takes as long for a row of a step as a warp takes for 16 steps; but a row that has a CTA of its own is done sooner.  us a call, by share alone, with at least 1, 4
    // and 8, and so, one query, 32 heads on 8 of d = 128: 64 sequences of up to 300 tokens 16.0 10.8 14.2 18.8 11.1, 40 of up to 600 17.8 13.1 16.0 19.7 13.6, 256 of up to 100
    // 22.6 22.7 16.4 16.4 16.6, 64 of up to 8000 33.2 33.1 32.8 32.7 32.6.)
    int brief = 0;
    if (crowded) {
        brief = share_of_steps(gridDim.x * WARPS, 0);
        uint32_t count[2 * BRIEFS] = {};         // rows up to 2^k steps, and parts of longer ones
        for (int b = tid; b < a.sequences; b += THREADS) {
            const uint2 x = seq_s[b];
            const uint32_t parts = (uint32_t)parts_of((int)x.x, piece), each = parts == 1 ? x.x : (x.x + parts - 1) / parts, n = x.y * parts;
            seq_s[b] = make_uint2(each, n << 1 | (parts > 1));              // (parts are longer than half a piece, and so than `brief`)
#pragma unroll
            for (int k = 0; k < BRIEFS; ++k) { count[k] += each <= 1u << k ? n : 0u; count[BRIEFS + k] += each <= 1u << k ? 0u : n; }
        }
        if (!sorted || brief < 1 << (BRIEFS - 1)) {
#pragma unroll
            for (int k = 0; k < 2 * BRIEFS; ++k) {
                const uint32_t all = __reduce_add_sync(0xffffffffu, count[k]);
                if (lane == k) count[0] = all;
            }
            if (lane < 2 * BRIEFS) atomicAdd(&briefs_s[lane], count[0]);
            __syncthreads();
            sorted = (briefs_s[0] + briefs_s[BRIEFS]) * a.kv_heads > gridDim.x;
            int first = 1 << (BRIEFS - 1);
#pragma unroll
            for (int k = BRIEFS - 2; k >= 0; --k)
                if ((briefs_s[k] * a.kv_heads + WARPS - 1) / WARPS + briefs_s[BRIEFS + k] * a.kv_heads <= gridDim.x) first = 1 << k;
            brief = max(brief, first);
        }
    }
    if (sorted) {
        for (int b = tid; b < (a.sequences + 3) / 4 * 4; b += THREADS) {
            const uint32_t each = b < a.sequences ? min(seq_s[b].x, (1u << (32 - SEQ_BITS)) - 1) : 0u;
            unsorted_s[b] = each << SEQ_BITS | (uint32_t)(SEQS - 1 - b);     // (no two alike)
        }
        __syncthreads();
        for (int b = tid; b < a.sequences; b += THREADS) {                   // as many places down as there are larger ones
            const uint32_t x = unsorted_s[b];
            int rank = 0;
            for (int k = 0; k < a.sequences; k += 4) {
                const uint4 y = *reinterpret_cast<const uint4*>(unsorted_s + k);
                rank += (y.x > x) + (y.y > x) + (y.z > x) + (y.w > x);
            }
            order_s[rank] = (uint16_t)b;
        }
        __syncthreads();
    }
    auto nth = [&](int k) { return sorted ? (int)order_s[k] : k; };        // the k-th sequence of the list
    uint32_t items = 0, splits = 0;              // of sequences with brief rows: rows
    int longs = 0;                               // sequences with longer ones: the first of the list
    for (int k0 = 0; k0 < a.sequences; k0 += THREADS) {
        unsigned long long all;
        const int k = k0 + tid;
        Seq x = s0;
        uint32_t n = 0, cut = 0, each = 0;       // items, those of several parts a row, steps of one
        if (sorted) {
            if (k < a.sequences) {
                const uint2 y = seq_s[order_s[k]];
                each = y.x;
                n = (y.y >> 1) * a.kv_heads;
                cut = y.y & 1 ? n : 0u;
            }
        } else if (k < a.sequences) {
            if (k0 > 0) x = sequence<COLS>(a, k);
            const uint32_t parts = (uint32_t)parts_of(x.steps, piece);
            n = (uint32_t)x.qtiles * a.kv_heads * parts;
            cut = parts > 1 ? n : 0u;
        }
        const unsigned long long before = block_scan((unsigned long long)n << 32 | cut, &all);
        if (k < a.sequences) { base_s[k] = (int)(items + (uint32_t)(before >> 32)); split_s[k] = (int)(splits + (uint32_t)before); }
        const int r = (int)blockIdx.x - (int)(items + (uint32_t)(before >> 32));
        if (!sorted && r >= 0 && r < (int)n) pieces[0] = piece_of(x, r, piece, (int)(splits + (uint32_t)before));          // this CTA's first item
        items += (uint32_t)(all >> 32);
        splits += (uint32_t)all;
        if (sorted) longs += __syncthreads_count((int)each > brief);
    }
    if (tid == 0) base_s[a.sequences] = (int)items;
    int whole_items = (int)items, singles = 0;   // items of a CTA, and rows behind them that are a warp's, eight to an item
    if (sorted) {
        __syncthreads();
        whole_items = base_s[longs];
        singles = (int)items - whole_items;
    }
    const int bundles = (singles + WARPS - 1) / WARPS, all_items = bundles + whole_items;    // (those of single rows first: they last longest)
    if ((int)blockIdx.x >= all_items) return;
    const bool more = all_items > (int)gridDim.x;
    if (tid == 0) item_s[0] = (int)blockIdx.x;
    // Decodes item `i` (by one warp).
    auto decode = [&](int i, Piece* to) {
        for (int k = lane; k < a.sequences; k += 32)
            if (base_s[k] <= i && i < base_s[k + 1]) *to = piece_of(sequence<COLS>(a, nth(k)), i - base_s[k], piece, split_s[k]);
    };

    if (sorted && warp == 0 && (int)blockIdx.x >= bundles) decode((int)blockIdx.x - bundles, &pieces[0]);

    uint8_t* const ring = smem + warp * ST * Cfg::STAGE_BYTES;
    float* const join = reinterpret_cast<float*>(smem);
    int load_slot = 0, use_slot = 0;            // places of the ring: next to be filled, next to be worked off
    uint32_t use_phase = 0, in_flight = 0;
    bool ok = true;

    for (int turn = 0;; turn ^= 1) {
        __syncthreads();                         // (the piece is there; the one before it is done with)
        const int item = item_s[turn];
        if (item < 0) break;
        const bool single = MANY && item < bundles;
        if (single) {                            // eight rows, one each for the warps
            const int row = whole_items + item * WARPS + warp;
            if (row >= whole_items + singles) continue;                      // (never warp 0)
            decode(row, &own_s[warp]);
            __syncwarp();
        }
        const Piece& pc = single ? own_s[warp] : pieces[turn];
        auto step_of = [&](int i) { return single ? i : pc.step0 + warp + WARPS * i; };          // of the row, the warp's i-th
        const int qt = pc.qt, h = pc.h, len = pc.s.len, nq = pc.s.nq, q0 = pc.s.q0;
        const bool whole = pc.parts == 1;

        // ---- the row's queries, column n = g of tile nt, channels 32 w + 8 t .. + 7: asked for ahead of all that has to be looked up first
        uint4 raw[NT][G];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int rho = qt * COLS + nt * 8 + g, token = (int)fastdiv((uint32_t)rho, a.by_group);
#pragma unroll
            for (int w = 0; w < G; ++w) {
                raw[nt][w] = make_uint4(0, 0, 0, 0);
                if (token < nq)
                    raw[nt][w] = *reinterpret_cast<const uint4*>(a.q + (size_t)(q0 + token) * a.q_stride + ((size_t)h * a.group + (rho - token * a.group)) * D + 32 * w + 8 * t);
            }
        }
        // ---- blocks: lane l looks up, and asks for, block l % 2 of steps l / 2, l / 2 + 16, .. of the warp's : step_of(i)
        const int nsteps = single ? pc.step1 : (pc.step1 - pc.step0 - warp + WARPS - 1) / WARPS;
        const uint8_t* addr = nullptr;
        uint32_t there[2] = {0, 0};             // blocks that exist (not those behind the end, nor in a page that does not exist), of these and the 16 steps before
        auto look_up = [&](int i0) {
            const int i = i0 + (lane >> 1), block = step_of(i) * STEP_BLOCKS + (lane & 1);
            addr = nullptr;
            if (i < nsteps && block * CACHE_BLOCK < len) {
                const int blocks = (int)a.by_blocks.d, col = (int)fastdiv((uint32_t)block, a.by_blocks);
                const int page = a.tables[(size_t)pc.s.slot * a.width + col];
                if (page >= 0 && page < a.pages) addr = a.pool + (((size_t)page * a.kv_heads + h) * blocks + (block - col * blocks)) * B::BYTES;
                else atomicExch(&dc->status, (int)PSA_ERR_SHAPE);            // (no such page: its tokens are left out, and the call reports it)
            }
            there[1] = there[0];
            there[0] = __ballot_sync(0xffffffffu, addr != nullptr);
        };
        // Step i into the ring.
        auto load = [&](int i) {
            if (i >= nsteps) return;
            if ((i & 15) == 0) look_up(i);
            if ((lane >> 1) == (i & 15)) {
                uint64_t* bar = &full[warp][load_slot];
                if (addr) {
                    mbar_arrive_expect_tx(bar, B::BYTES);
                    bulk_load_1d(ring + load_slot * Cfg::STAGE_BYTES + (lane & 1) * B::BYTES, addr, B::BYTES, bar);
                } else {
                    mbar_arrive(bar);
                }
            }
            load_slot = load_slot + 1 == ST ? 0 : load_slot + 1;
            ++in_flight;
        };
        if (ok)
            for (int i = 0; i < ST - 1; ++i) load(i);
        if (warp == 0) {                         // while the first blocks are on their way: the next item
            int i = -1;
            if (more) {
                if (lane == 0) i = (int)gridDim.x + (int)atomicAdd(&dc->next_item, 1u);
                i = __shfl_sync(0xffffffffu, i, 0);
                if (i >= all_items) i = -1;
                else if (i >= bundles) decode(i - bundles, &pieces[turn ^ 1]);
            }
            if (lane == 0) item_s[turn ^ 1] = i;
        }
        if ((warp == 0 || single) && lane == 0 && pc.s.bad) atomicExch(&dc->status, (int)PSA_ERR_SHAPE);

        // ---- the queries as the second operand
        uint32_t qb[NT][G][4];
        uint32_t qaff[NT][GQ][2];               // sums of the queries over groups t, t + 4, ..: leading and trailing part, each twice
        float cs[NT][2];                        // of columns 2t, 2t + 1: score factor (log2 units)
        int limit[NT][2];                       // the last token that the column sees
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float top = 0.f;
            float f[G][8];
#pragma unroll
            for (int w = 0; w < G; ++w) {
                const uint32_t x[4] = {raw[nt][w].x, raw[nt][w].y, raw[nt][w].z, raw[nt][w].w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (a.f16) {
                        const float2 v = __half22float2(bits_h2(x[k]));
                        f[w][2 * k] = v.x; f[w][2 * k + 1] = v.y;
                    } else {
                        f[w][2 * k] = __uint_as_float(x[k] << 16); f[w][2 * k + 1] = __uint_as_float(x[k] & 0xffff0000u);
                    }
                    top = fmaxf(top, fmaxf(fabsf(f[w][2 * k]), fabsf(f[w][2 * k + 1])));
                }
            }
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            // 2^e <= top < 2^(e+1): the row goes in as q 2^(13 - e) beside codes at a half's low end and as q 2^(9 - e) beside those one place up, exact but for
            // what lies 2^23 below its largest number.  A product of a code c is then c q 2^(-11 - e): 2^(7 + e) short of (c / 16) q, which the factor has.
            const uint32_t e = min(max(__float_as_uint(top) >> 23, 1u), 253u);
            const float down = __uint_as_float((254u - e) << 23), up = __uint_as_float(e << 23);
            float part[G];
#pragma unroll
            for (int w = 0; w < G; ++w) {
                part[w] = 0.f;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float place = k & 1 ? 512.f : 8192.f;
                    const __half2 v = __floats2half2_rn(f[w][2 * k] * down * place, f[w][2 * k + 1] * down * place);
                    qb[nt][w][k] = h2_bits(v);
                    const float2 r = __half22float2(v);
                    part[w] = fmaf(r.x + r.y, 1.f / (128.f * place), part[w]);
                }
                part[w] += __shfl_xor_sync(0xffffffffu, part[w], 1);
                part[w] += __shfl_xor_sync(0xffffffffu, part[w], 2);
            }
#pragma unroll
            for (int x = 0; x < GQ; ++x) {
                float mine = 0.f;
#pragma unroll
                for (int w = 4 * x; w < 4 * x + 4 && w < G; ++w)
                    if (t == w - 4 * x) mine = part[w];
                const __half hi = __float2half_rn(mine), lo = __float2half_rn(mine - __half2float(hi));
                qaff[nt][x][0] = h2_bits(__half2half2(hi));
                qaff[nt][x][1] = h2_bits(__half2half2(lo));
            }
            // from the lanes that hold column g to those that own it behind the product
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int owner = (2 * t + c) * 4;
                cs[nt][c] = fmaxf(__shfl_sync(0xffffffffu, up, owner) * (a.scale * LOG2E * 128.f), 1.2e-38f);
                limit[nt][c] = len - nq + min((int)fastdiv(qt * COLS + nt * 8 + 2 * t + c, a.by_group), nq - 1);
            }
        }
        const int seen_by_all = len - nq + (int)fastdiv(qt * COLS, a.by_group);          // the last token that every column sees

        const CacheOnes cache_ones;
        // m: running maximum of the scores before their factor; limit_up: where it is raised; shift: HEADROOM - m in log2 units
        float o[NT][2 * G][4], m[NT][2], limit_up[NT][2], shift[NT][2], l[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int i = 0; i < 2 * G; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) o[nt][i][c] = 0.f;
            m[nt][0] = m[nt][1] = limit_up[nt][0] = limit_up[nt][1] = -INFINITY;
            shift[nt][0] = shift[nt][1] = 0.f;
            l[nt][0] = l[nt][1] = 0.f;
        }

        for (int i = 0; i < nsteps && ok; ++i) {
            load(i + ST - 1);                    // (into the place that step i - 1 has left)
            ok = __all_sync(0xffffffffu, mbar_wait(&full[warp][use_slot], use_phase, abortp));
            if (!ok) break;
            const uint8_t* const stage = ring + use_slot * Cfg::STAGE_BYTES;
            --in_flight;
            if (++use_slot == ST) { use_slot = 0; use_phase ^= 1; }
            const int tok0 = step_of(i) * STEP;
            // (step i is one of the 16 looked up last, or of those before)
            const uint32_t have = ((i >> 4) == (min(i + ST - 1, nsteps - 1) >> 4) ? there[0] : there[1]) >> (2 * (i & 15)) & 3u;
            const bool masked = tok0 + STEP - 1 > seen_by_all || have != 3u;
            // ---- phase 1
            float sc[STEP_BLOCKS][NT][4];
#pragma unroll
            for (int s = 0; s < STEP_BLOCKS; ++s) {
                const uint8_t* const blk = stage + s * B::BYTES;
                uint32_t ka[G], kb[G], sa[G], sb[G];
                load_words<G>(blk + B::K_CODES + g * (D / 2) + t * G * 4, ka);
                load_words<G>(blk + B::K_CODES + (g + 8) * (D / 2) + t * G * 4, kb);
                load_words<G>(blk + B::K_SCALES + g * G * 4, sa);
                load_words<G>(blk + B::K_SCALES + (g + 8) * G * 4, sb);
#pragma unroll
                for (int x = 0; x < GQ; ++x) {   // (lanes beyond the last group repeat one, against sums of zero)
                    const int w = 4 * x + t < G ? 4 * x + t : 0;
                    const uint32_t fa = *reinterpret_cast<const uint32_t*>(blk + B::K_SCALES + (g * G + w) * 4), fb = *reinterpret_cast<const uint32_t*>(blk + B::K_SCALES + ((g + 8) * G + w) * 4);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
                        if (x == 0) mma16816_first(sc[s][nt], fa, fb, fa, fb, qaff[nt][0][0], qaff[nt][0][1]);
                        else mma16816(sc[s][nt], fa, fb, fa, fb, qaff[nt][x][0], qaff[nt][x][1]);
                }
#pragma unroll
                for (int w = 0; w < G; ++w) {
                    const float fa = __low2float(bits_h2(sa[w])), fb = __low2float(bits_h2(sb[w]));
                    const uint32_t ha = ka[w] >> 8, hb = kb[w] >> 8;
                    float d[NT][4];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        mma16816_first(d[nt], ka[w] & 0x000F000Fu, kb[w] & 0x000F000Fu, ka[w] & 0x00F000F0u, kb[w] & 0x00F000F0u, qb[nt][w][0], qb[nt][w][1]);
                        mma16816(d[nt], ha & 0x000F000Fu, hb & 0x000F000Fu, ha & 0x00F000F0u, hb & 0x00F000F0u, qb[nt][w][2], qb[nt][w][3]);
                        sc[s][nt][0] = fmaf(fa, d[nt][0], sc[s][nt][0]);
                        sc[s][nt][1] = fmaf(fa, d[nt][1], sc[s][nt][1]);
                        sc[s][nt][2] = fmaf(fb, d[nt][2], sc[s][nt][2]);
                        sc[s][nt][3] = fmaf(fb, d[nt][3], sc[s][nt][3]);
                    }
                }
            }
            // ---- phase 2
            if (masked) {
#pragma unroll
                for (int s = 0; s < STEP_BLOCKS; ++s)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            if (tok0 + s * CACHE_BLOCK + g + 8 * (c >> 1) > limit[nt][c & 1] || !(have >> s & 1u)) sc[s][nt][c] = -INFINITY;
            }
            bool raise = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float x = fmaxf(sc[0][nt][c], sc[0][nt][c + 2]);
#pragma unroll
                    for (int s = 1; s < STEP_BLOCKS; ++s) x = fmaxf(x, fmaxf(sc[s][nt][c], sc[s][nt][c + 2]));
                    raise |= x > limit_up[nt][c];
                }
            if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float x = fmaxf(sc[0][nt][c], sc[0][nt][c + 2]);
#pragma unroll
                        for (int s = 1; s < STEP_BLOCKS; ++s) x = fmaxf(x, fmaxf(sc[s][nt][c], sc[s][nt][c + 2]));
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
                        const float top = fmaxf(m[nt][c], x), f = ex2((m[nt][c] - finite_or_zero(top)) * cs[nt][c]);
                        m[nt][c] = top;
                        limit_up[nt][c] = top + RAISE / cs[nt][c];
                        shift[nt][c] = fmaf(-finite_or_zero(top), cs[nt][c], HEADROOM);
                        l[nt][c] *= f;
#pragma unroll
                        for (int k = 0; k < 2 * G; ++k) { o[nt][k][c] *= f; o[nt][k][c + 2] *= f; }
                    }
            }
            uint32_t pb[STEP_BLOCKS][NT][2];
#pragma unroll
            for (int s = 0; s < STEP_BLOCKS; ++s)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const float p0 = ex2(fmaf(sc[s][nt][0], cs[nt][0], shift[nt][0])), p1 = ex2(fmaf(sc[s][nt][1], cs[nt][1], shift[nt][1]));
                    const float p2 = ex2(fmaf(sc[s][nt][2], cs[nt][0], shift[nt][0])), p3 = ex2(fmaf(sc[s][nt][3], cs[nt][1], shift[nt][1]));
                    l[nt][0] += p0 + p2;
                    l[nt][1] += p1 + p3;
                    pb[s][nt][0] = transpose8x8(pack_weights(p0, p1));
                    pb[s][nt][1] = transpose8x8(pack_weights(p2, p3));
                }
            // ---- phase 3
#pragma unroll
            for (int s = 0; s < STEP_BLOCKS; ++s) {
                const uint8_t* const blk = stage + s * B::BYTES;
                uint32_t va[G], vb[G], ma[2 * G], mb[2 * G];
                load_words<G>(blk + B::V_CODES + t * D + g * G * 4, va);
                load_words<G>(blk + B::V_CODES + (t + 4) * D + g * G * 4, vb);
                load_words<2 * G>(blk + B::V_SCALES + t * G * 8, ma);
                load_words<2 * G>(blk + B::V_SCALES + (t + 4) * G * 8, mb);
                uint32_t nans[G];                // tokens of the block whose group reads back as NaN, if the block has any that a column must not see
                bool any_nan = false;
                if (masked) {
                    // Behind the sequence's end lies whatever the page held before; and a weight of zero does not keep a NaN out of the sum.  Such groups
                    // go in as zeros here, and come back below for the columns that do see their token.
                    const int ta = tok0 + s * CACHE_BLOCK + 2 * t, tb = ta + 8, end_tok = (have >> s & 1u) ? len : 0;
                    const uint32_t keep_a = (ta < end_tok ? 0xffffu : 0u) | (ta + 1 < end_tok ? 0xffff0000u : 0u), keep_b = (tb < end_tok ? 0xffffu : 0u) | (tb + 1 < end_tok ? 0xffff0000u : 0u);
#pragma unroll
                    for (int w = 0; w < G; ++w) {
                        uint32_t bits = 0;
                        auto one = [&](uint32_t& S, uint32_t& M, uint32_t keep, int at) {
                            S &= keep; M &= keep;
                            // (an exponent of all ones, in either half of either word)
                            const uint32_t x = (((S & 0x7c007c00u) + 0x04000400u) | ((M & 0x7c007c00u) + 0x04000400u)) & 0x80008000u;
                            const uint32_t drop = (x >> 15) * 0xffffu;
                            S &= ~drop; M &= ~drop;
                            bits |= ((x >> 15 & 1u) | (x >> 30 & 2u)) << at;
                        };
                        one(ma[2 * w], ma[2 * w + 1], keep_a, 2 * t);
                        one(mb[2 * w], mb[2 * w + 1], keep_b, 2 * t + 8);
                        nans[w] = __reduce_or_sync(0xffffffffu, bits);
                        any_nan |= nans[w] != 0;
                    }
                }
#pragma unroll
                for (int w = 0; w < G; ++w) {
                    const __half2 Sa = bits_h2(ma[2 * w]), Ma = bits_h2(ma[2 * w + 1]), Sb = bits_h2(mb[2 * w]), Mb = bits_h2(mb[2 * w + 1]);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const uint32_t a0 = h2_bits(__hfma2(bits_h2(cache_ones(va[w], 2 * k)), Sa, Ma)), a1 = h2_bits(__hfma2(bits_h2(cache_ones(va[w], 2 * k + 1)), Sa, Ma));
                        const uint32_t a2 = h2_bits(__hfma2(bits_h2(cache_ones(vb[w], 2 * k)), Sb, Mb)), a3 = h2_bits(__hfma2(bits_h2(cache_ones(vb[w], 2 * k + 1)), Sb, Mb));
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma16816(o[nt][2 * w + k], a0, a1, a2, a3, pb[s][nt][0], pb[s][nt][1]);
                    }
                }
                if (any_nan) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const int n = limit[nt][c] - (tok0 + s * CACHE_BLOCK) + 1;       // tokens of the block that the column sees
                            const uint32_t sees = n >= 16 ? 0xffffu : n <= 0 ? 0u : (1u << n) - 1u;
#pragma unroll
                            for (int w = 0; w < G; ++w)
                                if (nans[w] & sees) {
#pragma unroll
                                    for (int k = 0; k < 2; ++k) { o[nt][2 * w + k][c] = NAN; o[nt][2 * w + k][c + 2] = NAN; }
                                }
                        }
                }
            }
            __syncwarp();                        // all lanes are done with the block before it is overwritten
        }

        // ---- the columns' sums
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                if (m[nt][c] > -INFINITY) m[nt][c] *= cs[nt][c];             // log2 units from here on
                l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], 4);
                l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], 8);
                l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], 16);
            }
        const int cols = min(COLS, nq * a.group - qt * COLS);              // columns that are rows of the call
        auto store = [&](int col, int ch, float4 v, float inv) {             // four channels of a column, final
            const int rho = qt * COLS + col, token = (int)fastdiv((uint32_t)rho, a.by_group);
            const size_t at = ((size_t)(q0 + token) * a.kv_heads * a.group + (size_t)h * a.group + (rho - token * a.group)) * D + ch;
            uint2 y;
            if (a.f16) y = make_uint2(h2_bits(__floats2half2_rn(v.x * inv, v.y * inv)), h2_bits(__floats2half2_rn(v.z * inv, v.w * inv)));
            else y = make_uint2(pack_bf16x2(v.x * inv, v.y * inv), pack_bf16x2(v.z * inv, v.w * inv));
            *reinterpret_cast<uint2*>(a.out + at) = y;
        };
        auto store_lse = [&](int col, float top, float sum) {
            const int rho = qt * COLS + col, token = (int)fastdiv((uint32_t)rho, a.by_group);
            a.lse[(size_t)(q0 + token) * a.kv_heads * a.group + (size_t)h * a.group + (rho - token * a.group)] = sum == 0.f ? -INFINITY : (finite_or_zero(top) - HEADROOM + log2f(sum)) * LN2;
        };
        if (single) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int col = nt * 8 + 2 * t + c;
                    if (col >= cols) continue;
                    const float inv = l[nt][c] == 0.f ? 0.f : 1.f / l[nt][c];
#pragma unroll
                    for (int w = 0; w < G; ++w) store(col, 32 * w + 4 * g, make_float4(o[nt][2 * w][c], o[nt][2 * w][c + 2], o[nt][2 * w + 1][c], o[nt][2 * w + 1][c + 2]), inv);
                    if (a.lse && g == 0) store_lse(col, m[nt][c], l[nt][c]);
                }
            continue;
        }
        // ---- the warps' results into one
        if (g == 0) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 2; ++c) { m_s[warp][nt * 8 + 2 * t + c] = m[nt][c]; l_s[warp][nt * 8 + 2 * t + c] = l[nt][c]; }
        }
        __syncthreads();                         // (also: every warp is done with its ring, which the joining buffer overlays)
        if (tid < COLS) {
            float top = m_s[0][tid], sum = 0.f;
#pragma unroll
            for (int w = 1; w < WARPS; ++w) top = fmaxf(top, m_s[w][tid]);
#pragma unroll
            for (int w = 0; w < WARPS; ++w) sum += l_s[w][tid] * ex2(m_s[w][tid] - finite_or_zero(top));
            top_s[tid] = top;
            sum_s[tid] = sum;
        }
        __syncthreads();
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int col = nt * 8 + 2 * t + c;
                const float f = ex2(m[nt][c] - finite_or_zero(top_s[col]));
                float* to = join + (warp * COLS + col) * Cfg::OPITCH + 4 * g;
#pragma unroll
                for (int w = 0; w < G; ++w)
                    *reinterpret_cast<float4*>(to + 32 * w) = make_float4(o[nt][2 * w][c] * f, o[nt][2 * w][c + 2] * f, o[nt][2 * w + 1][c] * f, o[nt][2 * w + 1][c + 2] * f);
            }
        __syncthreads();
        float* const slot = a.part + (size_t)(pc.first + pc.part) * COLS * (D + 2);
        for (int e = tid; e < cols * (D / 4); e += THREADS) {
            const int col = e / (D / 4), ch = 4 * (e - col * (D / 4));
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                const float4 x = *reinterpret_cast<const float4*>(join + (w * COLS + col) * Cfg::OPITCH + ch);
                v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
            }
            if (whole) store(col, ch, v, sum_s[col] == 0.f ? 0.f : 1.f / sum_s[col]);
            else __stcg(reinterpret_cast<float4*>(slot + col * D + ch), v);
        }
        if (tid < cols) {
            if (!whole) { __stcg(slot + COLS * D + tid, top_s[tid]); __stcg(slot + COLS * (D + 1) + tid, sum_s[tid]); }
            else if (a.lse) store_lse(tid, top_s[tid], sum_s[tid]);
        }
        if (!whole) {
            const int parts = pc.parts;
            __syncthreads();
            if (tid == 0) last_s = arrive(&g_arrived[pc.first], (unsigned)(parts - 1));
            __syncthreads();
            if (last_s) {                        // all other parts are there: join them in their order
                auto part_of = [&](int p) { return a.part + (size_t)(pc.first + p) * COLS * (D + 2); };
                // With fewer groups of four channels than threads, several threads share one and take its parts in turn; what a thread needs first is asked
                // for ahead of the factors.
                constexpr int AHEAD = 8;
                const int n = cols * (D / 4), sharers = max(THREADS / n, 1), mine = sharers > 1 ? tid / n : 0, step = sharers;
                const int e1 = sharers > 1 ? tid - mine * n : tid;
                auto part_at = [&](int p, int e) { return __ldcg(reinterpret_cast<const float4*>(part_of(p) + 4 * e)); };      // (column e / (D / 4): they lie one after another)
                float4 x[AHEAD];
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) {
                    const int p = mine + k * step;
                    x[k] = e1 < n && mine < sharers && p < parts ? part_at(p, e1) : make_float4(0.f, 0.f, 0.f, 0.f);
                }
                // the parts' maxima and sums; maxima become factors.  (parts <= MOST_PARTS: they fit the ring)
                float* const mp = join;
                float* const lp = join + parts * COLS;
#pragma unroll 4
                for (int e = tid; e < parts * COLS; e += THREADS) {
                    const int p = e / COLS, col = e - p * COLS;
                    const float* from = part_of(p) + COLS * D + col;
                    mp[e] = col < cols ? __ldcg(from) : -INFINITY;
                    lp[e] = col < cols ? __ldcg(from + COLS) : 0.f;
                }
                __syncthreads();
                {
                    constexpr int PER = THREADS / COLS < 32 ? THREADS / COLS : 32;       // neighbouring lanes on a column
                    const int col = tid / PER, part = tid % PER;
                    if (tid < COLS * PER) {
                        float top = -INFINITY, sum = 0.f;
                        for (int p = part; p < parts; p += PER) top = fmaxf(top, mp[p * COLS + col]);
#pragma unroll
                        for (int s = 1; s < PER; s *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
                        for (int p = part; p < parts; p += PER) {
                            const float f = ex2(mp[p * COLS + col] - finite_or_zero(top));
                            mp[p * COLS + col] = f;
                            sum += f * lp[p * COLS + col];
                        }
#pragma unroll
                        for (int s = 1; s < PER; s *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, s);
                        if (part == 0) {
                            sum_s[col] = sum;
                            if (a.lse && col < cols) store_lse(col, top, sum);
                        }
                    }
                }
                __syncthreads();
                float4* const some = reinterpret_cast<float4*>(join + (2 * parts * COLS + 3) / 4 * 4);
                for (int e = e1; e - e1 < n; e += THREADS) {                 // (one round where threads share)
                    const int col = e / (D / 4);
                    const bool takes = e < n && mine < sharers;
                    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                    for (int p0 = mine; p0 < parts; p0 += AHEAD * step) {
                        if (e != e1 || p0 != mine) {
#pragma unroll
                            for (int k = 0; k < AHEAD; ++k) {
                                const int p = p0 + k * step;
                                x[k] = takes && p < parts ? part_at(p, e) : make_float4(0.f, 0.f, 0.f, 0.f);
                            }
                        }
#pragma unroll
                        for (int k = 0; k < AHEAD; ++k) {
                            const int p = p0 + k * step;
                            const float f = takes && p < parts ? mp[p * COLS + col] : 0.f;
                            v.x = fmaf(f, x[k].x, v.x); v.y = fmaf(f, x[k].y, v.y); v.z = fmaf(f, x[k].z, v.z); v.w = fmaf(f, x[k].w, v.w);
                        }
                    }
                    if (sharers > 1) {
                        some[tid] = v;
                        __syncthreads();
                        for (int k = 1; k < sharers && mine == 0; ++k) {
                            const float4 y = some[k * n + e];
                            v.x += y.x; v.y += y.y; v.z += y.z; v.w += y.w;
                        }
                    }
                    if (takes && mine == 0) store(col, 4 * (e - col * (D / 4)), v, sum_s[col] == 0.f ? 0.f : 1.f / sum_s[col]);
                }
            }
        }
        fence_async_smem();                      // the ring is written by copies again
    }
    if (!ok)                                     // copies already asked for land before shared memory is released
        for (; in_flight > 0; --in_flight) {
            mbar_wait_drain(&full[warp][use_slot], use_phase);
            if (++use_slot == ST) { use_slot = 0; use_phase ^= 1; }
        }
    if (lane == 0 && abort_flag) atomicExch(&dc->status, (int)PSA_ERR_TIMEOUT);
}

template <int D, int NT, bool MANY>
int launch_attn(const AttnArgs& all, DeviceCounters* dc, DeviceCounters* dc_next, cudaStream_t stream) {
    using Cfg = ACfg<D, NT>;
    static DeviceSetup setup;
    const int sms = device_setup(&setup, [] {
        return cudaFuncSetAttribute(cache_attn_kernel<D, NT, MANY>, cudaFuncAttributeMaxDynamicSharedMemorySize, ACfg<D, NT>::SMEM);
    }, "cache attention set-up");
    if (sms <= 0) return PSA_ERR_CUDA;
    for (int b0 = 0; b0 < all.sequences; b0 += SEQS) {
        AttnArgs a = all;
        a.sequences = all.sequences - b0 < SEQS ? all.sequences - b0 : SEQS;
        a.seqs += b0;
        a.q_starts += b0;
        // (upper bounds: the lengths are known on the device only)
        const long long tiles = ((long long)a.rows * a.group + Cfg::COLS - 1) / Cfg::COLS + a.sequences;
        if (tiles > MOST_ROWS / a.kv_heads) return PSA_ERR_UNSUPPORTED;
        const long long most = tiles * a.kv_heads * (((long long)a.width * a.page_size + STEP - 1) / STEP);
        a.wide = most > 0x7fffffffLL;
        long long grid = (long long)sms * Cfg::CTAS;
        if (grid > MAX_CTAS) grid = MAX_CTAS;
        if (grid > most) grid = most;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)grid);
        cfg.blockDim = dim3(Cfg::THREADS);
        cfg.dynamicSmemBytes = Cfg::SMEM;
        cfg.stream = stream;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        // (the counter that items are handed out by serves one launch)
        cudaError_t e = b0 == 0 ? cudaSuccess : cudaMemsetAsync(&dc->next_item, 0, sizeof(dc->next_item), stream);
        if (e == cudaSuccess) e = cudaLaunchKernelEx(&cfg, cache_attn_kernel<D, NT, MANY>, a, dc, b0 == 0 ? dc_next : nullptr);
        if (e != cudaSuccess) { set_cuda_error(e, "cache_attn_kernel launch"); return PSA_ERR_CUDA; }
    }
    return PSA_OK;
}

}  // namespace

size_t cache_attention_scratch_bytes(int d) { return (size_t)2 * MAX_CTAS * 16 * (d + 2) * sizeof(float); }

int cache_attention(const psa_cache& c, const void* Q, long long q_stride, const int* seqs, const int* q_starts, int sequences, int rows, int heads, int max_q,
                    float scale, int dtype, void* out, float* lse, void* scratch, DeviceCounters* dc, DeviceCounters* dc_next, cudaStream_t stream) {
    const AttnArgs a = {static_cast<const uint8_t*>(c.pool), c.tables, c.lens, seqs, q_starts, static_cast<const uint16_t*>(Q), static_cast<uint16_t*>(out), lse,
                        static_cast<float*>(scratch), q_stride, c.pages, c.slots, c.width, c.page_size, c.kv_heads, heads / c.kv_heads, sequences, rows,
                        dtype == PSA_F16, 0, scale, fastdiv_make((uint32_t)(heads / c.kv_heads)), fastdiv_make((uint32_t)(c.page_size / CACHE_BLOCK))};
    const bool wide = (long long)max_q * a.group > 8;        // more than eight columns: two tiles of them share a block's codes
    auto launch = [&](auto width, auto tiles_of_columns) {
        constexpr int D = decltype(width)::value, NT = decltype(tiles_of_columns)::value;
        const long long tiles = (long long)max_q * a.group <= 8 * NT ? sequences : ((long long)rows * a.group + 8 * NT - 1) / (8 * NT) + sequences;
        return 2 * tiles * c.kv_heads > 148 * ACfg<D, NT>::CTAS ? launch_attn<D, NT, true>(a, dc, dc_next, stream) : launch_attn<D, NT, false>(a, dc, dc_next, stream);
    };
    using std::integral_constant;
    const integral_constant<int, 1> one;
    const integral_constant<int, 2> two;
    switch (c.d_k) {
        case 32: return wide ? launch(integral_constant<int, 32>{}, two) : launch(integral_constant<int, 32>{}, one);
        case 64: return wide ? launch(integral_constant<int, 64>{}, two) : launch(integral_constant<int, 64>{}, one);
        case 96: return wide ? launch(integral_constant<int, 96>{}, two) : launch(integral_constant<int, 96>{}, one);
        case 128: return wide ? launch(integral_constant<int, 128>{}, two) : launch(integral_constant<int, 128>{}, one);
        case 256: return launch(integral_constant<int, 256>{}, one);         // (two tiles' output and queries would not fit the registers)
        default: return PSA_ERR_UNSUPPORTED;
    }
}

}  // namespace psa
