// Attention of a few query tokens of each sequence over its cache held in 4 bits (layout: psa_cache.cuh).
//
//     S_ij = scale q_i k_j,  w_ij = exp(S_ij),  out_i = sum_j w_ij v_j / sum_j w_ij,  j <= len - queries + i,  k_j and v_j being M + S (1 + c / 16)
//
// Bound by memory, if the instructions between the loads and the products stay few: at the measured 6.45 TB/s an SM gets 23 bytes of cache a clock, 37
// codes.  The heads of a group are the columns of one product, so that a code is looked at once for all of them:
//   phase 1  S^T = K Q^T     mma.m16n8k16, 16 tokens x 8 columns (heads of the group x query tokens).  The operand holds 1 + c / 16 exactly; S and M of a
//                            token enter behind the product, in fp32 (S_w (K Q)_w + M_w sum_w q, w a group of 32 channels): the scores have no rounding
//                            but that of Q to fp16, which a power of two per row keeps in range.
//   phase 2  running maximum and sum per column, 16 tokens at a time; the maximum is raised (and sums and output rescaled) only when a score passes it by 2^8
//   phase 3  O^T += V^T P^T  one fp16 fma per pair of codes gives v (rounded to fp16), the weights change sides by a transposing move
// Work is split over the long axis: all (sequence, head, tile of columns) rows of all their 16-token steps form one list, of which every CTA takes an
// equal piece whatever the lengths are (the kernel finds its piece from the lengths; nothing has to be known on the host).  The warps of a CTA take the
// steps of a row in turn, each with a ring of blocks of its own filled by bulk copies, and are joined through shared memory; a row that several CTAs share is
// joined by the one that finishes last, in the order of the list, so that results do not depend on who that is.
#include "psa_cache.cuh"
#include "psa_internal.h"
#include "sm100.cuh"

namespace psa {

namespace {

constexpr int WARPS = 4;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float RAISE = 8.f;                    // log2 units, see phase 2
constexpr int MAX_CTAS = 148 * 4 + 64;          // partial results and arrival counts are kept per CTA
constexpr int LEAST_STEPS = 2 * WARPS;          // a CTA's piece is not shorter than this

template <int D, int NT>
struct ACfg {
    static constexpr int COLS = 8 * NT;
    static constexpr int CTAS = D * NT <= 128 ? 4 : 2;
    static constexpr int STAGES = D >= 256 ? 4 : D == 128 ? 5 : D == 96 ? 6 : 8;
    static constexpr int RING = WARPS * STAGES * CacheBlock<D>::BYTES;
    static constexpr int OPITCH = D + 4;        // floats between columns of the joining buffer (keeps its 16-byte stores off each other's banks)
    static constexpr int JOIN = WARPS * COLS * OPITCH * 4;
    static constexpr int SMEM = RING > JOIN ? RING : JOIN;
};

struct AttnArgs {
    const uint8_t* pool;
    const int *tables, *lens, *seqs, *q_starts;
    const uint16_t* q;
    uint16_t* out;
    float *lse, *part;                          // part: 2 per CTA, [COLS][D] outputs, then [COLS] maxima and [COLS] sums
    long long q_stride;
    int pages, slots, width, page_size, kv_heads, group, sequences, rows, f16;
    float scale;
};

// Arrivals on a row that several CTAs share, at the index of the first of them.  Every arrival that completes a row wraps its count to zero again, and a CTA
// that gave up a wait arrives all the same: the counts are zero between calls.
__device__ unsigned g_arrived[MAX_CTAS];

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
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t h2_bits(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }
__device__ __forceinline__ __half2 bits_h2(uint32_t u) { return *reinterpret_cast<__half2*>(&u); }
__device__ __forceinline__ float finite_or_zero(float m) { return m == -INFINITY ? 0.f : m; }

// One sequence of the call: tokens held, query rows, and the steps of the work list that it has.
struct Seq {
    int slot, len, q0, nq, qtiles, steps;
    long long units;
};
template <int COLS>
__device__ __forceinline__ Seq sequence(const AttnArgs& a, int b) {
    Seq s;
    s.slot = a.seqs[b];
    const bool there = s.slot >= 0 && s.slot < a.slots;
    s.q0 = min(max(a.q_starts[b], 0), a.rows);
    s.nq = max(min(max(a.q_starts[b + 1], 0), a.rows) - s.q0, 0);
    s.len = there ? (int)min((long long)max(a.lens[s.slot], 0), (long long)a.width * a.page_size) : 0;
    s.qtiles = (int)(((long long)s.nq * a.group + COLS - 1) / COLS);
    s.steps = max((s.len + CACHE_BLOCK - 1) / CACHE_BLOCK, 1);
    s.units = (long long)s.steps * s.qtiles * a.kv_heads;
    return s;
}

template <int D, int NT>
__global__ void __launch_bounds__(32 * WARPS, ACfg<D, NT>::CTAS)
cache_attn_kernel(const AttnArgs a, DeviceCounters* dc, DeviceCounters* dc_next) {
    using Cfg = ACfg<D, NT>;
    using B = CacheBlock<D>;
    constexpr int G = B::G, COLS = Cfg::COLS, ST = Cfg::STAGES;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ uint64_t full[WARPS][ST];
    __shared__ float m_s[WARPS][COLS], l_s[WARPS][COLS], top_s[COLS], sum_s[COLS];
    __shared__ long long scan_s[WARPS];
    __shared__ int abort_flag, last_s, found_b;
    __shared__ long long found_first;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    if (tid == 0) {
        abort_flag = 0;
        for (int w = 0; w < WARPS; ++w)
            for (int s = 0; s < ST; ++s) mbar_init(&full[w][s], 1);
        fence_mbar_init();
    }
    volatile int* abortp = &abort_flag;
    grid_dependency_wait();
    if (tid == 0 && blockIdx.x == 0 && dc_next) *dc_next = DeviceCounters{0, 0, 0, 0, 0, 0, 0};

    // ---- this CTA's piece of the list: units [begin, end) of all, and the sequence that `begin` lies in
    long long mine0 = 0;                        // (units of sequence tid: the only chunk, up to 128 sequences)
    auto block_scan = [&](long long v, long long* total) -> long long {      // exclusive
        long long x = v;
#pragma unroll
        for (int s = 1; s < 32; s *= 2) {
            const long long y = __shfl_up_sync(0xffffffffu, x, s);
            if (lane >= s) x += y;
        }
        __syncthreads();
        if (lane == 31) scan_s[warp] = x;
        __syncthreads();
        long long before = 0, all = 0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) { if (w < warp) before += scan_s[w]; all += scan_s[w]; }
        *total = all;
        return before + x - v;
    };
    long long W = 0;
    for (int b0 = 0; b0 < a.sequences; b0 += 32 * WARPS) {
        long long all;
        const long long v = b0 + tid < a.sequences ? sequence<COLS>(a, b0 + tid).units : 0;
        block_scan(v, &all);
        if (b0 == 0) mine0 = v;
        W += all;
    }
    const long long ctas = min((long long)gridDim.x, max(W / LEAST_STEPS, 1LL));
    if (W == 0 || blockIdx.x >= ctas) return;
    const long long begin = W * blockIdx.x / ctas, end = W * (blockIdx.x + 1) / ctas;
    {
        long long done = 0;
        for (int b0 = 0; b0 < a.sequences && done <= begin; b0 += 32 * WARPS) {
            long long all;
            const long long v = b0 == 0 ? mine0 : b0 + tid < a.sequences ? sequence<COLS>(a, b0 + tid).units : 0;
            const long long first = done + block_scan(v, &all);
            if (v > 0 && first <= begin && begin < first + v) { found_b = b0 + tid; found_first = first; }
            done += all;
        }
        __syncthreads();
    }
    int b = found_b;
    long long seq_first = found_first;          // unit index of the sequence's first step
    Seq s = sequence<COLS>(a, b);
    auto cta_of = [&](long long u) { return (int)(((u + 1) * ctas - 1) / W); };

    uint8_t* const ring = smem + warp * ST * B::BYTES;
    float* const join = reinterpret_cast<float*>(smem);
    uint32_t loaded = 0;                        // blocks this warp has asked for so far (position in the ring)
    uint32_t used = 0;                          // blocks it has worked off
    bool ok = true;
    const int blocks = a.page_size / CACHE_BLOCK;

    for (long long u = begin; u < end;) {
        while (u >= seq_first + s.units) { seq_first += s.units; s = sequence<COLS>(a, ++b); }
        const int row = (int)((u - seq_first) / s.steps), step0 = (int)((u - seq_first) - (long long)row * s.steps);
        const int h = row / s.qtiles, qt = row - h * s.qtiles;
        const int step1 = (int)min((long long)s.steps, step0 + (end - u));
        const long long row_first = u - step0;
        const bool whole = step0 == 0 && step1 == s.steps;
        if (tid == 0 && (s.slot < 0 || s.slot >= a.slots || a.lens[s.slot] != s.len)) atomicExch(&dc->status, (int)PSA_ERR_SHAPE);

        // ---- blocks: lane l looks up the block of the warp's step first + l, 32 at a time
        const int nsteps = (step1 - step0 - warp + WARPS - 1) / WARPS;       // steps of this warp: step0 + warp + WARPS i
        const uint8_t* addr = nullptr;
        int looked = 0;
        auto look_up = [&](int i0) {
            const int step = step0 + warp + WARPS * (i0 + lane);
            addr = nullptr;
            if (i0 + lane < nsteps && step * CACHE_BLOCK < s.len) {
                const int col = step / blocks;
                const int page = a.tables[(size_t)s.slot * a.width + col];
                if (page >= 0 && page < a.pages) addr = a.pool + (((size_t)page * a.kv_heads + h) * blocks + (step - col * blocks)) * B::BYTES;
                else atomicExch(&dc->status, (int)PSA_ERR_SHAPE);            // (no such page: its tokens are left out, and the call reports it)
            }
        };
        // Step i of the warp into the ring; a step without a block (an empty sequence, a page that does not exist) takes no place in it.
        uint32_t missing = 0;                   // bit i % 32: step i has no block
        auto load = [&](int i) {
            if (i >= nsteps) return;
            if ((i & 31) == 0) look_up(i);
            const unsigned long long p = __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(addr), i & 31);
            const uint32_t bit = 1u << (i & 31);
            missing = p ? missing & ~bit : missing | bit;
            if (!p) return;
            if (lane == 0) {
                uint64_t* bar = &full[warp][loaded % ST];
                mbar_arrive_expect_tx(bar, B::BYTES);
                bulk_load_1d(ring + (loaded % ST) * B::BYTES, reinterpret_cast<const void*>(p), B::BYTES, bar);
            }
            ++loaded;
        };
        if (ok)
            for (; looked < ST - 1; ++looked) load(looked);

        // ---- the row's queries as the second operand: column n = g of tile nt, channels 32 w + 8 t .. + 7
        uint32_t qb[NT][G][4];
        float cs[NT][2], qsum[NT][G][2];        // of columns 2t, 2t + 1: score factor (log2 units) and sums over the groups
        int limit[NT][2];                       // the last token that the column sees
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int rho = qt * COLS + nt * 8 + g, token = rho / a.group;
            uint4 raw[G];
            float top = 0.f;
#pragma unroll
            for (int w = 0; w < G; ++w) {
                raw[w] = make_uint4(0, 0, 0, 0);
                if (token < s.nq)
                    raw[w] = *reinterpret_cast<const uint4*>(a.q + (size_t)(s.q0 + token) * a.q_stride + ((size_t)h * a.group + (rho - token * a.group)) * D + 32 * w + 8 * t);
            }
            float f[G][8];
#pragma unroll
            for (int w = 0; w < G; ++w) {
                const uint32_t x[4] = {raw[w].x, raw[w].y, raw[w].z, raw[w].w};
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
            // 2^e <= top < 2^(e+1): the row goes in as q 2^-e, exact but for what lies 2^14 below its largest number
            const uint32_t e = min(max(__float_as_uint(top) >> 23, 1u), 253u);
            const float down = __uint_as_float((254u - e) << 23), up = __uint_as_float(e << 23);
            float part[G];
#pragma unroll
            for (int w = 0; w < G; ++w) {
                part[w] = 0.f;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const __half2 v = __floats2half2_rn(f[w][2 * k] * down, f[w][2 * k + 1] * down);
                    qb[nt][w][k] = h2_bits(v);
                    const float2 r = __half22float2(v);
                    part[w] += r.x + r.y;
                }
                part[w] += __shfl_xor_sync(0xffffffffu, part[w], 1);
                part[w] += __shfl_xor_sync(0xffffffffu, part[w], 2);
            }
            // from the lanes that hold column g to those that own it behind the product
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int from = (2 * t + c) * 4;
                cs[nt][c] = __shfl_sync(0xffffffffu, up, from) * (a.scale * LOG2E);
#pragma unroll
                for (int w = 0; w < G; ++w) qsum[nt][w][c] = __shfl_sync(0xffffffffu, part[w], from);
                limit[nt][c] = s.len - s.nq + min((qt * COLS + nt * 8 + 2 * t + c) / a.group, s.nq - 1);
            }
        }
        const int seen_by_all = s.len - s.nq + qt * COLS / a.group;          // the last token that every column sees

        float o[NT][2 * G][4], m[NT][2], l[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int i = 0; i < 2 * G; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) o[nt][i][c] = 0.f;
            m[nt][0] = m[nt][1] = -INFINITY;
            l[nt][0] = l[nt][1] = 0.f;
        }

        for (int i = 0; i < nsteps && ok; ++i) {
            const bool skip = (missing >> (i & 31)) & 1u;
            load(looked++);                      // (into the place that step i - 1 has left)
            if (skip) continue;
            ok = __all_sync(0xffffffffu, mbar_wait(&full[warp][used % ST], (used / ST) & 1, abortp));
            if (!ok) break;
            const uint8_t* blk = ring + (used % ST) * B::BYTES;
            ++used;
            const int tok0 = (step0 + warp + WARPS * i) * CACHE_BLOCK;
            const bool masked = tok0 + CACHE_BLOCK - 1 > seen_by_all;
            // ---- phase 1
            float sc[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) sc[nt][0] = sc[nt][1] = sc[nt][2] = sc[nt][3] = 0.f;
            {
                uint32_t ka[G], kb[G], sa[G], sb[G];
                load_words<G>(blk + B::K_CODES + g * (D / 2) + t * G * 4, ka);
                load_words<G>(blk + B::K_CODES + (g + 8) * (D / 2) + t * G * 4, kb);
                load_words<G>(blk + B::K_SCALES + g * G * 4, sa);
                load_words<G>(blk + B::K_SCALES + (g + 8) * G * 4, sb);
#pragma unroll
                for (int w = 0; w < G; ++w) {
                    const float2 fa = __half22float2(bits_h2(sa[w])), fb = __half22float2(bits_h2(sb[w]));
                    float d[NT][4];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) d[nt][0] = d[nt][1] = d[nt][2] = d[nt][3] = 0.f;
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const uint32_t a0 = cache_ones(ka[w], 2 * k), a1 = cache_ones(kb[w], 2 * k), a2 = cache_ones(ka[w], 2 * k + 1), a3 = cache_ones(kb[w], 2 * k + 1);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma16816(d[nt], a0, a1, a2, a3, qb[nt][w][2 * k], qb[nt][w][2 * k + 1]);
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        sc[nt][0] = fmaf(fa.x, d[nt][0], fmaf(fa.y, qsum[nt][w][0], sc[nt][0]));
                        sc[nt][1] = fmaf(fa.x, d[nt][1], fmaf(fa.y, qsum[nt][w][1], sc[nt][1]));
                        sc[nt][2] = fmaf(fb.x, d[nt][2], fmaf(fb.y, qsum[nt][w][0], sc[nt][2]));
                        sc[nt][3] = fmaf(fb.x, d[nt][3], fmaf(fb.y, qsum[nt][w][1], sc[nt][3]));
                    }
                }
            }
            // ---- phase 2
            uint32_t pb[NT][2];
            bool raise = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int c = 0; c < 4; ++c) sc[nt][c] *= cs[nt][c & 1];
                if (masked) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (tok0 + g + 8 * (c >> 1) > limit[nt][c & 1]) sc[nt][c] = -INFINITY;
                }
                raise |= fmaxf(sc[nt][0], sc[nt][2]) > m[nt][0] + RAISE || fmaxf(sc[nt][1], sc[nt][3]) > m[nt][1] + RAISE;
            }
            if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float x = fmaxf(sc[nt][c], sc[nt][c + 2]);
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
                        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
                        const float top = fmaxf(m[nt][c], x), f = ex2(m[nt][c] - finite_or_zero(top));
                        m[nt][c] = top;
                        l[nt][c] *= f;
#pragma unroll
                        for (int k = 0; k < 2 * G; ++k) { o[nt][k][c] *= f; o[nt][k][c + 2] *= f; }
                    }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float m0 = finite_or_zero(m[nt][0]), m1 = finite_or_zero(m[nt][1]);
                const float p0 = ex2(sc[nt][0] - m0), p1 = ex2(sc[nt][1] - m1), p2 = ex2(sc[nt][2] - m0), p3 = ex2(sc[nt][3] - m1);
                l[nt][0] += p0 + p2;
                l[nt][1] += p1 + p3;
                pb[nt][0] = transpose8x8(h2_bits(__floats2half2_rn(p0, p1)));
                pb[nt][1] = transpose8x8(h2_bits(__floats2half2_rn(p2, p3)));
            }
            // ---- phase 3
            uint32_t va[G], vb[G], ma[2 * G], mb[2 * G];
            load_words<G>(blk + B::V_CODES + t * D + g * G * 4, va);
            load_words<G>(blk + B::V_CODES + (t + 4) * D + g * G * 4, vb);
            load_words<2 * G>(blk + B::V_SCALES + t * G * 8, ma);
            load_words<2 * G>(blk + B::V_SCALES + (t + 4) * G * 8, mb);
            uint32_t nans[G];                    // tokens of the block whose group reads back as NaN, if the block has any that a column must not see
            bool any_nan = false;
            if (masked) {
                // Behind the sequence's end lies whatever the page held before; and a weight of zero does not keep a NaN out of the sum.  Such groups
                // go in as zeros here, and come back below for the columns that do see their token.
                const int ta = tok0 + 2 * t, tb = ta + 8;
                const uint32_t keep_a = (ta < s.len ? 0xffffu : 0u) | (ta + 1 < s.len ? 0xffff0000u : 0u), keep_b = (tb < s.len ? 0xffffu : 0u) | (tb + 1 < s.len ? 0xffff0000u : 0u);
#pragma unroll
                for (int w = 0; w < G; ++w) {
                    uint32_t bits = 0;
                    auto one = [&](uint32_t& S, uint32_t& M, uint32_t keep, int at) {
                        S &= keep; M &= keep;
                        const __half2 hs = bits_h2(S), hm = bits_h2(M);
                        const bool lo = __hisnan(__low2half(hs)) || __hisinf(__low2half(hs)) || __hisnan(__low2half(hm)) || __hisinf(__low2half(hm));
                        const bool hi = __hisnan(__high2half(hs)) || __hisinf(__high2half(hs)) || __hisnan(__high2half(hm)) || __hisinf(__high2half(hm));
                        const uint32_t drop = (lo ? 0xffffu : 0u) | (hi ? 0xffff0000u : 0u);
                        S &= ~drop; M &= ~drop;
                        bits |= (lo ? 1u << at : 0u) | (hi ? 2u << at : 0u);
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
                    for (int nt = 0; nt < NT; ++nt) mma16816(o[nt][2 * w + k], a0, a1, a2, a3, pb[nt][0], pb[nt][1]);
                }
            }
            if (any_nan) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int n = limit[nt][c] - tok0 + 1;               // tokens of the block that the column sees
                        const uint32_t sees = n >= 16 ? 0xffffu : n <= 0 ? 0u : (1u << n) - 1u;
#pragma unroll
                        for (int w = 0; w < G; ++w)
                            if (nans[w] & sees) {
#pragma unroll
                                for (int k = 0; k < 2; ++k) { o[nt][2 * w + k][c] = NAN; o[nt][2 * w + k][c + 2] = NAN; }
                            }
                    }
            }
            __syncwarp();                        // all lanes are done with the block before it is overwritten
        }

        // ---- the warps' results into one
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], 4);
                l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], 8);
                l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], 16);
                if (g == 0) { m_s[warp][nt * 8 + 2 * t + c] = m[nt][c]; l_s[warp][nt * 8 + 2 * t + c] = l[nt][c]; }
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
        const int cols = min(COLS, s.nq * a.group - qt * COLS);              // columns that are rows of the call
        float* const slot = a.part + (size_t)(2 * blockIdx.x + (u == begin ? 0 : 1)) * COLS * (D + 2);
        auto store = [&](int col, int ch, float4 v, float inv) {             // four channels of a column, final
            const int rho = qt * COLS + col, token = rho / a.group;
            const size_t at = ((size_t)(s.q0 + token) * a.kv_heads * a.group + (size_t)h * a.group + (rho - token * a.group)) * D + ch;
            uint2 y;
            if (a.f16) y = make_uint2(h2_bits(__floats2half2_rn(v.x * inv, v.y * inv)), h2_bits(__floats2half2_rn(v.z * inv, v.w * inv)));
            else y = make_uint2(pack_bf16x2(v.x * inv, v.y * inv), pack_bf16x2(v.z * inv, v.w * inv));
            *reinterpret_cast<uint2*>(a.out + at) = y;
        };
        auto store_lse = [&](int col, float top, float sum) {
            const int rho = qt * COLS + col, token = rho / a.group;
            a.lse[(size_t)(s.q0 + token) * a.kv_heads * a.group + (size_t)h * a.group + (rho - token * a.group)] = sum == 0.f ? -INFINITY : (finite_or_zero(top) + log2f(sum)) * LN2;
        };
        for (int e = tid; e < cols * (D / 4); e += 32 * WARPS) {
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
            const int c0 = cta_of(row_first), c1 = cta_of(row_first + s.steps - 1), parts = c1 - c0 + 1;
            __threadfence();
            __syncthreads();
            if (tid == 0) last_s = atomicInc(&g_arrived[c0], (unsigned)(parts - 1)) == (unsigned)(parts - 1);
            __syncthreads();
            if (last_s) {                        // all other parts are there: join them in the order of the list
                __threadfence();
                const bool c0_first = W * c0 / ctas == row_first;            // the row's first part is its CTA's first piece, or its last
                auto part_of = [&](int p) { return a.part + (size_t)(2 * (c0 + p) + (p > 0 || c0_first ? 0 : 1)) * COLS * (D + 2); };
                if (tid < COLS) {
                    float top = -INFINITY, sum = 0.f;
                    if (tid < cols) {
                        for (int p = 0; p < parts; ++p) top = fmaxf(top, __ldcg(part_of(p) + COLS * D + tid));
                        for (int p = 0; p < parts; ++p) sum += __ldcg(part_of(p) + COLS * (D + 1) + tid) * ex2(__ldcg(part_of(p) + COLS * D + tid) - finite_or_zero(top));
                        if (a.lse) store_lse(tid, top, sum);
                    }
                    top_s[tid] = top;
                    sum_s[tid] = sum;
                }
                __syncthreads();
                for (int e = tid; e < cols * (D / 4); e += 32 * WARPS) {
                    const int col = e / (D / 4), ch = 4 * (e - col * (D / 4));
                    const float top = finite_or_zero(top_s[col]);
                    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
                    for (int p = 0; p < parts; ++p) {
                        const float* from = part_of(p);
                        const float f = ex2(__ldcg(from + COLS * D + col) - top);
                        const float4 x = __ldcg(reinterpret_cast<const float4*>(from + col * D + ch));
                        v.x = fmaf(f, x.x, v.x); v.y = fmaf(f, x.y, v.y); v.z = fmaf(f, x.z, v.z); v.w = fmaf(f, x.w, v.w);
                    }
                    store(col, ch, v, sum_s[col] == 0.f ? 0.f : 1.f / sum_s[col]);
                }
            }
        }
        fence_async_smem();                      // the ring is written by copies again
        __syncthreads();
        u += step1 - step0;
    }
    if (!ok)                                     // copies already asked for land before shared memory is released
        for (uint32_t c = used; c < loaded; ++c) mbar_wait_drain(&full[warp][c % ST], (c / ST) & 1);
    if (lane == 0 && abort_flag) atomicExch(&dc->status, (int)PSA_ERR_TIMEOUT);
}

template <int D, int NT>
int launch_attn(const AttnArgs& a, DeviceCounters* dc, DeviceCounters* dc_next, cudaStream_t stream) {
    using Cfg = ACfg<D, NT>;
    static DeviceSetup setup;
    const int sms = device_setup(&setup, [] {
        return cudaFuncSetAttribute(cache_attn_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, ACfg<D, NT>::SMEM);
    }, "cache attention set-up");
    if (sms <= 0) return PSA_ERR_CUDA;
    // every CTA works on at least one step: no more of them than the tables have room for
    const long long tiles = ((long long)a.rows * a.group + Cfg::COLS - 1) / Cfg::COLS + a.sequences;
    const long long most = tiles * a.kv_heads * (((long long)a.width * a.page_size + CACHE_BLOCK - 1) / CACHE_BLOCK);
    long long grid = (long long)sms * Cfg::CTAS;
    if (grid > MAX_CTAS) grid = MAX_CTAS;
    if (grid > (most + LEAST_STEPS - 1) / LEAST_STEPS) grid = (most + LEAST_STEPS - 1) / LEAST_STEPS;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(32 * WARPS);
    cfg.dynamicSmemBytes = Cfg::SMEM;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, cache_attn_kernel<D, NT>, a, dc, dc_next);
    if (e != cudaSuccess) { set_cuda_error(e, "cache_attn_kernel launch"); return PSA_ERR_CUDA; }
    return PSA_OK;
}

}  // namespace

size_t cache_attention_scratch_bytes(int d) { return (size_t)2 * MAX_CTAS * 16 * (d + 2) * sizeof(float); }

int cache_attention(const psa_cache& c, const void* Q, long long q_stride, const int* seqs, const int* q_starts, int sequences, int rows, int heads, int max_q,
                    float scale, int dtype, void* out, float* lse, void* scratch, DeviceCounters* dc, DeviceCounters* dc_next, cudaStream_t stream) {
    const AttnArgs a = {static_cast<const uint8_t*>(c.pool), c.tables, c.lens, seqs, q_starts, static_cast<const uint16_t*>(Q), static_cast<uint16_t*>(out), lse,
                        static_cast<float*>(scratch), q_stride, c.pages, c.slots, c.width, c.page_size, c.kv_heads, heads / c.kv_heads, sequences, rows,
                        dtype == PSA_F16, scale};
    const bool wide = (long long)max_q * a.group > 8;        // more than eight columns: two tiles of them share a block's codes
    switch (c.d_k) {
        case 32: return wide ? launch_attn<32, 2>(a, dc, dc_next, stream) : launch_attn<32, 1>(a, dc, dc_next, stream);
        case 64: return wide ? launch_attn<64, 2>(a, dc, dc_next, stream) : launch_attn<64, 1>(a, dc, dc_next, stream);
        case 96: return wide ? launch_attn<96, 2>(a, dc, dc_next, stream) : launch_attn<96, 1>(a, dc, dc_next, stream);
        case 128: return wide ? launch_attn<128, 2>(a, dc, dc_next, stream) : launch_attn<128, 1>(a, dc, dc_next, stream);
        case 256: return launch_attn<256, 1>(a, dc, dc_next, stream);       // (two tiles' output and queries would not fit the registers)
        default: return PSA_ERR_UNSUPPORTED;
    }
}

}  // namespace psa
