// Attention of trees of drafted tokens over the cache held in 4 bits (layout: psa_cache.cuh), where a key/value head has many query rows (a row: a token of the tree and a query head of the
// group; psa_cache_attn.cu takes the others, and d = 256).
//
//     S_ij = scale q_i k_j,  w_ij = exp(S_ij),  out_i = sum_j w_ij v_j / sum_j w_ij,   j ahead of the tree, or i itself, or an ancestor of i
//
// 128 rows are a tile of the tensor core, so that a code is made a number once for all of them: at d = 128 a tile of 128 tokens is 20 KB of cache, 890 cycles at an SM's share of the memory's rate,
// and 1536 cycles of MMAs.  A persistent CTA an SM; every role walks the CTA's share of the work by itself and meets the others at barriers of two or three stages:
//   one warp each  fetch blocks of K and of V by bulk copies into rings of three tiles, looking page numbers up four tiles ahead
//   8 warps, K     fp16 operands of M + S (1 + c / 16), two stages, a block of 16 tokens of a tile each.  A key goes in in two parts (the number rounded, and what that leaves: 2^-22 of it, or 2^-25
//                  where that is more, is lost), each a pass over the codes and an operand.  One part would lose 2^-12 of a key, and a log-sum-exp as much of scale sum_c |q_c k_c|, however long
//                  the context is where a row attends to a few tokens or channels are large (with it 32 sequences of up to 8000 tokens took 66 us, two of up to 131,072 122).
//   4 warps, V     fp16 operands, two stages, rounded as in psa_cache_attn.cu
//   one thread     issues the MMAs: scores of tile j + 1 ahead of the product of tile j's weights with V, with queries, scores (twice) and output in tensor memory
//   8 warps        softmax, 16 rows each: scores are read twice, for the maximum (raised only when it is passed by 2^8) and for the weights, which go over the scores as fp16, held 2^7 times as
//                  large (HEADROOM in psa_prompt.cu)
//   one warp       the sets of tokens that a row sees, as bits
// Work is the list of all tiles of all rows' tiles, weighed and cut into as many equal pieces as there are CTAs, whatever the lengths: a CTA ends one row tile, has some whole, and begins another.
// Parts of a row tile are stored in fp32 and joined in their order by a second small kernel, since no CTA waits for another; rows with one part are finished where they are.
//
// Measured (one B200, clocks 1.9 GHz): a tile takes 5900 cycles, at 104 rows of 128 as at 48.  With keys in one part it took 3500, in which a softmax warp was busy 2950, one that
// turns codes of K 2730, of V 2800, and the thread that issues MMAs waited for weights: 20 warps that all wait for results of a fixed latency, and for instructions, whose caches five roles share (loops that are unrolled further are slower;
// half the work of one role took 2 to 7 % off a call, of all three 19).  What comes once a row tile costs about two tiles and a half: 2000 cycles to read the queries, 2000 to the first scores, 4000 for the masked
// ones, 5000 for the results.  32 sequences of up to 8000 tokens, trees of 12, 32 heads on 8 of d = 128 90 us; two of up to 131,072, trees of 26 164 us (340 TFLOP/s of the rows that exist); eight of up to
// 6000, trees of 64, 32 on 4, fp16 51 us.
#include <type_traits>

#include "psa_cache.cuh"
#include "psa_internal.h"
#include "psa_sched.h"
#include "psa_softmax.cuh"
#include "sm100.cuh"

namespace psa {

namespace {

constexpr int ROWS = 128, KEYS = 128, BLOCKS = KEYS / CACHE_BLOCK;
constexpr int MMA_WARP = 0, K_WARP = 1, V_WARP = 2, SET_WARP = 3, SOFT0 = 4, SOFTS = 8, TURN_K = SOFT0 + SOFTS, TURN_V = TURN_K + BLOCKS, V_WARPS = BLOCKS / 2, T_WARPS = TURN_V + V_WARPS, T_THREADS = 32 * T_WARPS;
constexpr int T_SEQS = 512;                     // sequences of one launch
constexpr int T_CTAS = 160;                     // at most
// What work takes, in thirds of a tile of keys: a tile, and what a row tile takes beside its tiles; the least that a CTA is given.
constexpr int COST = 3, COST_ROW = 8, LEAST = 8;
constexpr int TREE_WORDS = PSA_TREE_MOST / 32 + 1;
constexpr float UP = 7.f;                       // log2 of what weights are held larger by
constexpr float T_LN2 = 0.6931471805599453f;

template <int D>
struct TCfg {
    static constexpr int DT = D <= 64 ? 64 : 128, SUB = DT / 64, KS = D / 16, G = D / 32;
    static constexpr int SUBTILE = KEYS * 128, TILE = SUB * SUBTILE;         // an operand tile: sub-tiles of 64 columns, 128-byte rows swizzled
    static constexpr int HALF = 10 * D;         // bytes of K, and of V, in a block
    static constexpr int RING = 3;              // tiles of codes
    // two of each operand, the rings, the sets
    static constexpr int K = 0, V = K + 2 * TILE, RAW_K = V + 2 * TILE, RAW_V = RAW_K + RING * BLOCKS * HALF, TREE = RAW_V + RING * BLOCKS * HALF;
    static constexpr int SMEM = TREE + ROWS * TREE_WORDS * 4 + 1024;
};
constexpr int TM_S = 0, TM_O = 256, TM_Q = 384;  // columns of tensor memory: S twice (P over its first half), O, the queries

struct TreeArgs {
    const uint8_t* pool;
    const int *tables, *lens, *seqs, *q_starts, *parents;
    const uint16_t* q;
    uint16_t* out;
    float *lse, *part;
    struct TreeRow* rows_cut;
    long long q_stride;
    int pages, slots, width, page_size, kv_heads, group, sequences, rows, f16;
    float scale;
    FastDiv by_group, by_blocks;
};
// A row tile that is cut: by the CTA that has its first part.  parts 0: none.
struct TreeRow {
    int parts, q0, nq, h, qt;
};
// Part `p` of the row tile that CTA c begins: [ROWS][d] sums, then as many maxima (log2) and sums of weights.
__device__ __forceinline__ float* part_at(float* part, int c, int p, int d) { return part + (size_t)(p == 0 ? 2 * c + 1 : 2 * (c + p)) * ROWS * (d + 2); }

struct TBars {
    uint64_t k_raw[3], k_raw_free[3], v_raw[3], v_raw_free[3];
    uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], p_ready[2], q_full, sets_full, sets_free;
};
// Tiles t0 .. t0 + nt - 1 of row tile qt of head h of a sequence.
struct TItem {
    int len, nq, q0, slot, t0, nt, h, qt, ctx, tok0;       // ctx: the tree's first token; tok0: the row tile's first
    int first_cta, part, parts;                             // of the row tile; a CTA has one part of it
    int row, rows;                                          // the row tile's place among those of its sequence (heads times row tiles), and their number
    bool meets_tree;
};

__device__ __forceinline__ uint32_t t_bits(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }
__device__ __forceinline__ __half2 t_h2(uint32_t u) { return *reinterpret_cast<__half2*>(&u); }
__device__ __forceinline__ uint32_t t_weights(float lo, float hi) {
    uint32_t v;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(v) : "f"(hi), "f"(lo));
    return v;
}
// Two numbers at a time.
__device__ __forceinline__ uint64_t t_pair(float x, float y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ float2 t_pair(uint64_t x) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
    return r;
}
// Sixteen rows, 32 columns of fp32 in the quad layout.
__device__ __forceinline__ void t_ld_quad32(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
                   "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ uint64_t t_add2(uint64_t x, uint64_t y) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
    return r;
}
__device__ __forceinline__ uint64_t t_fma2(uint64_t x, uint64_t y, uint64_t z) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(x), "l"(y), "l"(z));
    return r;
}
__host__ __device__ constexpr uint32_t t_idesc(uint32_t n, uint32_t b_major) { return umma_idesc_bf16(128, n, UMMA_K_MAJOR, b_major) & ~((1u << 7) | (1u << 10)); }      // fp16 operands

template <int D>
__global__ void __launch_bounds__(T_THREADS, 1) tree_kernel(const TreeArgs a, DeviceCounters* dc, DeviceCounters* dc_next) {
    using Cfg = TCfg<D>;
    using B = CacheBlock<D>;
    constexpr int G = Cfg::G;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint32_t* const tree = reinterpret_cast<uint32_t*>(smem + Cfg::TREE);       // [ROWS][TREE_WORDS]: by token of the row tile, the tree's tokens that it sees
    __shared__ TBars bars;
    __shared__ uint32_t tmem_s;
    __shared__ int abort_flag;
    __shared__ long long base_s[T_SEQS + 1], scan_s[T_WARPS];
    __shared__ int len_s[T_SEQS], q0_s[T_SEQS], nq_s[T_SEQS], slot_s[T_SEQS];
    __shared__ __align__(8) uint8_t have_s[2][16][BLOCKS];       // blocks of a tile that are there, by tile modulo 16; as the warp found them that fetches V, or K
    __shared__ int any_nan_s[2];                // by items in turn: whether there are marks in
    __shared__ uint32_t nan_s[2][G][PSA_TREE_MOST / 32];         // by items in turn: tokens of the tree whose group of V reads back as NaN or infinite

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        abort_flag = 0;
        for (int s = 0; s < 3; ++s) {
            mbar_init(&bars.k_raw[s], BLOCKS); mbar_init(&bars.k_raw_free[s], BLOCKS);
            mbar_init(&bars.v_raw[s], BLOCKS); mbar_init(&bars.v_raw_free[s], V_WARPS);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(&bars.k_full[s], BLOCKS); mbar_init(&bars.k_empty[s], 1);
            mbar_init(&bars.v_full[s], V_WARPS); mbar_init(&bars.v_empty[s], 1);
            mbar_init(&bars.s_full[s], 1); mbar_init(&bars.p_ready[s], SOFTS);
        }
        mbar_init(&bars.q_full, SOFTS);
        mbar_init(&bars.sets_full, 1); mbar_init(&bars.sets_free, SOFTS + V_WARPS);
        fence_mbar_init();
    }
    if (warp == 1) { tmem_alloc(&tmem_s, 512); tmem_relinquish(); }
    volatile int* const abortp = &abort_flag;
    grid_dependency_wait();
    if (tid == 0 && blockIdx.x == 0 && dc_next) *dc_next = DeviceCounters{0, 0, 0, 0, 0, 0, 0};
    if (tid == 0) a.rows_cut[blockIdx.x].parts = 0;
    // ---- the list: tiles ahead of every sequence
    bool descends = false, strange = false;
    long long ahead = 0;
    for (int b0 = 0; b0 < a.sequences; b0 += T_THREADS) {
        const int b = b0 + tid;
        long long n = 0;
        if (b < a.sequences) {
            const int slot = a.seqs[b], s0 = a.q_starts[b], s1 = a.q_starts[b + 1];
            const bool there = slot >= 0 && slot < a.slots;
            descends |= s1 < s0;
            const int q0 = min(max(s0, 0), a.rows), all = max(min(max(s1, 0), a.rows) - q0, 0), nq = all > PSA_TREE_MOST ? 0 : all;
            const int held = there ? max(a.lens[slot], 0) : 0, len = (int)min((long long)held, (long long)a.width * a.page_size);
            strange |= (nq > 0 && (!there || held != len)) || nq != s1 - s0;
            const int tiles = max((int)(((uint32_t)len + KEYS - 1) / KEYS), 1), row_tiles = (nq * a.group + ROWS - 1) / ROWS;
            n = (long long)row_tiles * a.kv_heads * ((long long)tiles * COST + COST_ROW);
            len_s[b] = len;
            q0_s[b] = q0;
            nq_s[b] = nq;
            slot_s[b] = there ? slot : 0;
        }
        long long x = n;
#pragma unroll
        for (int s = 1; s < 32; s *= 2) {
            const long long y = __shfl_up_sync(0xffffffffu, x, s);
            if (lane >= s) x += y;
        }
        __syncthreads();
        if (lane == 31) scan_s[warp] = x;
        __syncthreads();
        long long before = ahead;
        for (int w = 0; w < T_WARPS; ++w) { if (w < warp) before += scan_s[w]; ahead += scan_s[w]; }
        if (b < a.sequences) base_s[b] = before + x - n;
    }
    if (tid == 0) base_s[a.sequences] = ahead;
    if (strange && blockIdx.x == 0) atomicExch(&dc->status, (int)PSA_ERR_SHAPE);
    const bool refused = __syncthreads_or(descends) != 0;        // rows named more than once: nothing is computed, and the call reports it
    if (refused && tid == 0 && blockIdx.x == 0) atomicExch(&dc->status, (int)PSA_ERR_SHAPE);
    const long long per = max((ahead + gridDim.x - 1) / (long long)gridDim.x, (long long)LEAST);
    const long long mine0 = min(per * (long long)blockIdx.x, ahead), mine1 = refused ? mine0 : min(mine0 + per, ahead);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_s;

    // ---- Every role walks the CTA's items by itself: its share of the list.  A row tile is COST_ROW units and COST for each tile of keys, which belongs to the CTA that has its first unit.
    // Behind an item comes the next row tile from its beginning: only the first one takes divisions, and those that are cut.
    auto next_item = [&](long long& at, TItem& x) -> bool {
        while (at < mine1) {
            int u0 = 0;
            const bool first = x.rows < 0;
            if (x.row + 1 < x.rows) {
                ++x.row;
                if (++x.qt * ROWS >= x.nq * a.group) { x.qt = 0; ++x.h; }
            } else {
                int lo = 0, hi = a.sequences - 1;    // the last sequence that begins at or before it (and has tiles: those without begin where the next one does)
                while (lo < hi) {
                    const int mid = (lo + hi + 1) / 2;
                    if (base_s[mid] <= at) lo = mid; else hi = mid - 1;
                }
                x.len = len_s[lo];
                x.nq = nq_s[lo];
                x.q0 = q0_s[lo];
                x.slot = slot_s[lo];
                x.ctx = x.len - x.nq;
                x.row = x.h = x.qt = 0;
                const int row_tiles = (x.nq * a.group + ROWS - 1) / ROWS;
                x.rows = row_tiles * a.kv_heads;
                if (first) {
                    const int units = max((int)(((uint32_t)x.len + KEYS - 1) / KEYS), 1) * COST + COST_ROW;
                    const long long inside = at - base_s[lo];
                    x.row = (int)(inside / units);
                    u0 = (int)(inside - (long long)x.row * units);
                    x.h = x.row / row_tiles;
                    x.qt = x.row - x.h * row_tiles;
                }
            }
            const int units = max((int)(((uint32_t)x.len + KEYS - 1) / KEYS), 1) * COST + COST_ROW, u1 = (int)min((long long)units, u0 + (mine1 - at));
            const long long row0 = at - u0;
            at += u1 - u0;
            auto tile_of = [](int u) { return (max(u - COST_ROW, 0) + COST - 1) / COST; };
            x.t0 = tile_of(u0);
            const int t1 = tile_of(u1);
            if (t1 <= x.t0) continue;
            x.nt = x.len > 0 ? t1 - x.t0 : 0;
            x.tok0 = (int)fastdiv((uint32_t)(x.qt * ROWS), a.by_group);
            x.first_cta = (int)blockIdx.x;
            x.parts = 1;
            if (u1 - u0 < units) {
                x.first_cta = (int)((row0 + COST_ROW) / per);
                x.parts = (int)((row0 + units - COST) / per) - x.first_cta + 1;
            }
            x.part = (int)blockIdx.x - x.first_cta;
            x.meets_tree = x.nt > 0 && t1 * (long long)KEYS > x.ctx;
            return true;
        }
        return false;
    };
    long long at = mine0;
    TItem x;
    x.row = 0;
    x.rows = -1;
    uint32_t n = 0;                             // tiles of the CTA so far: the phases of all barriers follow from it, but those that go by items
    bool ok = true;

    if (warp == MMA_WARP) {
        if (elect_one()) {
            constexpr uint32_t idescS = t_idesc(KEYS, UMMA_K_MAJOR), idescO = t_idesc(D, UMMA_MN_MAJOR);
            const uint32_t k_lo = umma_desc_lo_kmajor(smem_u32(smem + Cfg::K)), v_lo = umma_desc_lo_mnmajor(smem_u32(smem + Cfg::V), Cfg::SUBTILE);
            uint32_t items = 0, fills = 0;       // items that have tiles; operands of K
            while (ok && next_item(at, x)) {
                if (x.nt == 0) continue;
                ok = mbar_wait(&bars.q_full, items++ & 1, abortp);
                for (int j = 0; j <= x.nt && ok; ++j) {
                    const uint32_t m = n + j;
                    if (j < x.nt) {
                        // (where P of tile j - 2 was: its product has been issued)
                        const uint32_t dS = tmem + TM_S + (m & 1) * KEYS;
                        for (int part = 0; part < 2; ++part, ++fills) {
                            const uint32_t s = fills & 1, k = k_lo + s * (Cfg::TILE >> 4);
                            ok = mbar_wait(&bars.k_full[s], (fills >> 1) & 1, abortp);
                            if (!ok) break;
                            tc_fence_after();
#pragma unroll
                            for (int kk = 0; kk < Cfg::KS; ++kk)
                                umma_ts(dS, tmem + TM_Q + kk * 8, umma_desc_join(k + (((kk >> 2) * Cfg::SUBTILE + (kk & 3) * 32) >> 4), UMMA_DESC_HI_SW128), idescS, part > 0 || kk > 0);
                            if (part == 1) umma_commit(&bars.s_full[m & 1]);
                            umma_commit(&bars.k_empty[s]);
                        }
                        if (!ok) break;
                    }
                    if (j > 0) {
                        const uint32_t s = (m - 1) & 1;
                        ok = mbar_wait(&bars.v_full[s], ((m - 1) >> 1) & 1, abortp) && mbar_wait(&bars.p_ready[s], ((m - 1) >> 1) & 1, abortp);
                        if (!ok) break;
                        tc_fence_after();
#pragma unroll
                        for (int kk = 0; kk < KEYS / 16; ++kk)
                            umma_ts(tmem + TM_O, tmem + TM_S + s * KEYS + kk * 8, umma_desc_join(v_lo + s * (Cfg::TILE >> 4) + kk * (2048 >> 4), UMMA_DESC_HI_SW128), idescO, j > 1 || kk > 0);
                        umma_commit(&bars.v_empty[s]);
                    }
                }
                n += x.nt;
            }
        }
    } else if (warp == K_WARP || warp == V_WARP) {
        // ------------------------------------------------------------ codes of K, and of V, into their rings: a block of 16 tokens a lane, four tiles looked up at a time, four ahead of their use
        const bool is_k = warp == K_WARP;
        constexpr int stages = Cfg::RING;
        uint64_t *const full = is_k ? bars.k_raw : bars.v_raw, *const empty = is_k ? bars.k_raw_free : bars.v_raw_free;
        uint8_t* const ring = smem + (is_k ? Cfg::RAW_K : Cfg::RAW_V);
        const int blocks = (int)a.by_blocks.d;
        while (ok && next_item(at, x)) {
            auto look_up = [&](int i0) -> const uint8_t* {
                const int i = i0 + lane / BLOCKS;
                const long long block = (long long)(x.t0 + i) * BLOCKS + lane % BLOCKS;
                if (i >= x.nt || block * CACHE_BLOCK >= x.len) return nullptr;
                const int col = (int)fastdiv((uint32_t)block, a.by_blocks), page = a.tables[(size_t)x.slot * a.width + col];
                if (page >= 0 && page < a.pages) return a.pool + (((size_t)page * a.kv_heads + x.h) * blocks + ((int)block - col * blocks)) * B::BYTES + (is_k ? 0 : Cfg::HALF);
                atomicExch(&dc->status, (int)PSA_ERR_SHAPE);             // (no such page: its tokens are left out, and the call reports it)
                return nullptr;
            };
            const uint8_t *from = look_up(0), *ahead = nullptr;
            for (int i = 0; i < x.nt; ++i, ++n) {
                if (i % (32 / BLOCKS) == 0) {
                    if (i > 0) from = ahead;
                    ahead = look_up(i + 32 / BLOCKS);
                }
                const int s = n % stages;
                if (n >= (uint32_t)stages) ok = __all_sync(0xffffffffu, mbar_wait(&empty[s], (n / stages - 1) & 1, abortp));
                if (!ok) break;
                if (lane / BLOCKS == i % (32 / BLOCKS)) {
                    have_s[is_k][n & 15][lane % BLOCKS] = from != nullptr;
                    if (from) {
                        mbar_arrive_expect_tx(&full[s], Cfg::HALF);
                        bulk_load_1d(ring + (s * BLOCKS + lane % BLOCKS) * Cfg::HALF, from, Cfg::HALF, &full[s]);
                    } else {
                        mbar_arrive(&full[s]);
                    }
                }
                __syncwarp();
            }
        }
        if (!ok)                                 // copies already asked for land before shared memory is released
            for (uint32_t m = n > (uint32_t)stages ? n - stages : 0; m < n; ++m) mbar_wait_drain(&full[m % stages], (m / stages) & 1);
    } else if (warp == SET_WARP) {
        // ------------------------------------------------------------ the tokens' sets of the tree: each its own and its ancestors.  A barrier's parity tells one phase from the next and no further: all
        // who read the sets or write marks wait for sets_full of every item, those without keys or tree tokens too, and let go of every item, so that nobody is more than one phase away from this warp.
        for (uint32_t it = 0; ok && next_item(at, x); ++it) {
            if (it > 0) ok = __all_sync(0xffffffffu, mbar_wait(&bars.sets_free, (it - 1) & 1, abortp));
            if (!ok) break;
            for (int i = lane; i < G * (PSA_TREE_MOST / 32); i += 32) (&nan_s[it & 1][0][0])[i] = 0u;
            if (lane == 0) any_nan_s[it & 1] = 0;
            if (x.meets_tree) {
                const int words = (x.nq + 31) / 32, last = min((int)fastdiv((uint32_t)(x.qt * ROWS + ROWS - 1), a.by_group), x.nq - 1);
                for (int tok = x.tok0 + lane; tok <= last; tok += 32) {
                    uint32_t* const mine = tree + (tok - x.tok0) * TREE_WORDS;
                    for (int i = 0; i < words; ++i) mine[i] = 0u;
                    int k = tok;
                    while (k >= 0) {
                        mine[k >> 5] |= 1u << (k & 31);
                        const int up = __ldg(a.parents + x.q0 + k);
                        if (up < -1 || up >= k) atomicExch(&dc->status, (int)PSA_ERR_SHAPE);         // (no earlier token: taken for the root of a tree of its own)
                        k = up < k ? up : -1;
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars.sets_full);
        }
    } else if (warp >= TURN_K && warp < TURN_V) {
        // ------------------------------------------------------------ codes of K into operands: a block of 16 tokens of every tile a warp
        const int me = warp - TURN_K;
        const CacheOnes ones;
        uint32_t fills = 0;
        // Eight tokens are G rounds of 32 chunks of 16 bytes (chunk: eight channels of a token); where a lane's are in the codes, the scales and the operand.  The other eight lie behind them.
        int from_codes[G], from_scales[G], to_chunk[G];
#pragma unroll
        for (int z = 0; z < G; ++z) {
            const int e = z * 32 + lane, tok = e / (4 * G), chunk = e - tok * (4 * G), w = chunk >> 2;
            from_codes[z] = tok * (D / 2) + ((chunk & 3) * G + w) * 4;
            from_scales[z] = B::K_SCALES + (tok * G + w) * 4;
            to_chunk[z] = (chunk >> 3) * Cfg::SUBTILE + (int)swz128_offset(me * CACHE_BLOCK + tok, chunk & 7);
        }
        for (; ok && next_item(at, x);)
            for (int i = 0; i < x.nt && ok; ++i, ++n) {
                const int s = n % Cfg::RING;
                ok = __all_sync(0xffffffffu, mbar_wait(&bars.k_raw[s], (n / Cfg::RING) & 1, abortp));
                if (!ok) break;
                const bool have = have_s[1][n & 15][me] != 0;
                const uint8_t* const from = smem + Cfg::RAW_K + (s * BLOCKS + me) * Cfg::HALF;
                auto fill = [&](auto rest) {     // rest: what fp16 leaves of the numbers
                    if (fills >= 2) ok = __all_sync(0xffffffffu, mbar_wait(&bars.k_empty[fills & 1], ((fills >> 1) - 1) & 1, abortp));
                    if (!ok) return;
                    uint8_t* const to = smem + Cfg::K + (fills & 1) * Cfg::TILE;
                    if (have) {
                        // (All of eight tokens is read ahead of the first store: the compiler cannot know that what is read and written lies apart.)
#pragma unroll 1
                        for (int eight = 0; eight < 2; ++eight) {
                            uint32_t codes[G], sm[G];
#pragma unroll
                            for (int z = 0; z < G; ++z) {
                                codes[z] = *reinterpret_cast<const uint32_t*>(from + from_codes[z] + eight * (8 * D / 2));
                                sm[z] = *reinterpret_cast<const uint32_t*>(from + from_scales[z] + eight * (8 * G * 4));
                            }
#pragma unroll
                            for (int z = 0; z < G; ++z) {
                                const __half2 S = t_h2(__byte_perm(sm[z], sm[z], 0x1010)), M = t_h2(__byte_perm(sm[z], sm[z], 0x3232));
                                uint32_t y[4];
#pragma unroll
                                for (int c = 0; c < 4; ++c) {
                                    const __half2 one = t_h2(ones(codes[z], c)), v = __hfma2(one, S, M);
                                    if constexpr (decltype(rest)::value) {
                                        const float2 o = __half22float2(one), h = __half22float2(v);
                                        const float Sf = __low2float(S), Mf = __low2float(M);
                                        y[c] = t_bits(__floats2half2_rn(fmaf(o.x, Sf, Mf) - h.x, fmaf(o.y, Sf, Mf) - h.y));
                                    } else {
                                        y[c] = t_bits(v);
                                    }
                                }
                                *reinterpret_cast<uint4*>(to + to_chunk[z] + eight * 1024) = make_uint4(y[0], y[1], y[2], y[3]);
                            }
                        }
                    }
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars.k_full[fills & 1]);
                    ++fills;
                };
                fill(std::false_type{});
                if (ok) fill(std::true_type{});
                if (ok && lane == 0) mbar_arrive(&bars.k_raw_free[s]);
            }
    } else if (warp >= TURN_V) {
        // ------------------------------------------------------------ codes of V into its operand: two blocks of every tile a warp
        const CacheOnes ones;
        // A block is G rounds of 32 chunks (chunk: eight channels of a pair of tokens); where a lane's are in the codes, the scales and the operand.
        int from_codes[G], from_scales[G], to_chunk[G];
#pragma unroll
        for (int z = 0; z < G; ++z) {
            const int e = z * 32 + lane, pair = e / (4 * G), chunk = e - pair * (4 * G), w = chunk >> 2;
            from_codes[z] = pair * D + (2 * (chunk & 3) * G + w) * 4;
            from_scales[z] = (B::V_SCALES - B::V_CODES) + (pair * G + w) * 8;
            to_chunk[z] = (chunk >> 3) * Cfg::SUBTILE + (int)swz128_offset(2 * pair, chunk & 7);
        }
        // block `me` of tile m; first: its first token
        auto turn_v = [&](uint32_t m, int me, long long first, int ctx, int len, int nq, uint32_t (*nan)[PSA_TREE_MOST / 32], int& any_nan) {
            const int s = m % Cfg::RING;
            const uint8_t* const from = smem + Cfg::RAW_V + (s * BLOCKS + me) * Cfg::HALF;
            uint8_t* const to = smem + Cfg::V + (m & 1) * Cfg::TILE + me * (CACHE_BLOCK * 128);
            uint32_t c0[G], c1[G];
            uint2 sm[G];
#pragma unroll
            for (int z = 0; z < G; ++z) {
                c0[z] = *reinterpret_cast<const uint32_t*>(from + from_codes[z]);
                c1[z] = *reinterpret_cast<const uint32_t*>(from + from_codes[z] + 4 * G);
                sm[z] = *reinterpret_cast<const uint2*>(from + from_scales[z]);
            }
            const bool have = have_s[0][m & 15][me] != 0;
            if (first + CACHE_BLOCK > ctx || !have) {
                // The block has tokens that not all rows see, or that are none of the sequence's.  Behind the sequence's end lies whatever the page held before, and a weight of zero does not keep a NaN out
                // of the sum: such tokens, and groups of the tree's that are not finite, go in as zeros; rows that see these get a NaN at the end.
#pragma unroll
                for (int z = 0; z < G; ++z) {
                    const int e = z * 32 + lane, pair = e / (4 * G), w = (e - pair * (4 * G)) >> 2;
                    const long long tok = first + 2 * pair;
                    const uint32_t keep = have ? (tok < len ? 0xffffu : 0u) | (tok + 1 < len ? 0xffff0000u : 0u) : 0u;
                    sm[z].x &= keep;
                    sm[z].y &= keep;
                    uint32_t bad = (((sm[z].x & 0x7c007c00u) + 0x04000400u) | ((sm[z].y & 0x7c007c00u) + 0x04000400u)) & 0x80008000u;      // an exponent of all ones
                    if (tok < ctx) bad &= 0x80000000u;
                    if (tok + 1 < ctx) bad = 0;
                    if (bad) {
                        const uint32_t drop = (bad >> 15) * 0xffffu;
                        sm[z].x &= ~drop;
                        sm[z].y &= ~drop;
                        const int at0 = (int)(tok - ctx);
                        any_nan = 1;
                        if ((bad & 0x8000u) && at0 < nq) atomicOr(&nan[w][at0 >> 5], 1u << (at0 & 31));
                        if ((bad & 0x80000000u) && at0 + 1 < nq) atomicOr(&nan[w][(at0 + 1) >> 5], 1u << ((at0 + 1) & 31));
                    }
                }
            }
#pragma unroll
            for (int z = 0; z < G; ++z) {
                const __half2 S = t_h2(sm[z].x), M = t_h2(sm[z].y);
                uint32_t v[8];                   // channels 8 (chunk) + k: of the even token in the lower half, of the odd one in the upper
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    v[k] = t_bits(__hfma2(t_h2(ones(c0[z], k)), S, M));
                    v[4 + k] = t_bits(__hfma2(t_h2(ones(c1[z], k)), S, M));
                }
                *reinterpret_cast<uint4*>(to + to_chunk[z]) =
                    make_uint4(__byte_perm(v[0], v[1], 0x5410), __byte_perm(v[2], v[3], 0x5410), __byte_perm(v[4], v[5], 0x5410), __byte_perm(v[6], v[7], 0x5410));
                *reinterpret_cast<uint4*>(to + ((to_chunk[z] ^ 16) + 128)) =
                    make_uint4(__byte_perm(v[0], v[1], 0x7632), __byte_perm(v[2], v[3], 0x7632), __byte_perm(v[4], v[5], 0x7632), __byte_perm(v[6], v[7], 0x7632));
            }
        };
        for (uint32_t it = 0; ok && next_item(at, x); ++it) {
            bool sets = false;                   // the item's marks of NaN are known to be clear
            for (int i = 0; i < x.nt && ok; ++i, ++n) {
                const long long first = (long long)(x.t0 + i) * KEYS;
                if (!sets && first + KEYS > x.ctx) {
                    ok = __all_sync(0xffffffffu, mbar_wait(&bars.sets_full, it & 1, abortp));
                    sets = true;
                }
                const int s = n % Cfg::RING;
                ok = ok && __all_sync(0xffffffffu, mbar_wait(&bars.v_raw[s], (n / Cfg::RING) & 1, abortp));
                if (ok && n >= 2) ok = __all_sync(0xffffffffu, mbar_wait(&bars.v_empty[n & 1], ((n >> 1) - 1) & 1, abortp));
                if (!ok) break;
#pragma unroll 1
                for (int me = warp - TURN_V; me < BLOCKS; me += V_WARPS) turn_v(n, me, first + me * CACHE_BLOCK, x.ctx, x.len, x.nq, nan_s[it & 1], any_nan_s[it & 1]);
                fence_async_smem();
                __syncwarp();
                if (lane == 0) { mbar_arrive(&bars.v_full[n & 1]); mbar_arrive(&bars.v_raw_free[s]); }
            }
            if (ok && !sets) ok = __all_sync(0xffffffffu, mbar_wait(&bars.sets_full, it & 1, abortp));
            if (ok && lane == 0) mbar_arrive(&bars.sets_free);       // (its marks are written: __syncwarp above)
        }
    } else {
        // ------------------------------------------------------------ softmax: 16 rows a warp, in the quad layout
        const int sw = warp - SOFT0, r0 = (warp & 3) * 32 + (sw >> 2) * 16, rA = r0 + (lane >> 2), rB = rA + 8, cq = 2 * (lane & 3);
        const uint32_t lanes = (uint32_t)r0 << 16, tO = tmem + TM_O + lanes;
        for (uint32_t it = 0; ok && next_item(at, x); ++it) {
            const int rhoA = x.qt * ROWS + rA, rhoB = x.qt * ROWS + rB, tokA = (int)fastdiv((uint32_t)rhoA, a.by_group), tokB = (int)fastdiv((uint32_t)rhoB, a.by_group);
            float fA = 1.f, fB = 1.f;            // factors of the rows' scores, to log2 units
            if (x.nt > 0) {
                // ---- the queries into tensor memory: 64 columns of K, 32 words, at a time
                uint32_t raw[Cfg::SUB][16];          // [2 g]: channels 64 u + 8 g + cq .. of row A, [2 g + 1] of row B
                float topA = 0.f, topB = 0.f;
                auto number = [&](uint32_t w) { return a.f16 ? __half22float2(t_h2(w)) : make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); };
                auto from = [&](int token, int rho) { return a.q + (size_t)(x.q0 + token) * a.q_stride + ((size_t)x.h * a.group + (rho - token * a.group)) * D + cq; };
                const uint16_t *const qA = from(tokA, rhoA), *const qB = from(tokB, rhoB);
#pragma unroll
                for (int u = 0; u < Cfg::SUB; ++u)
#pragma unroll
                    for (int g = 0; g < 8; ++g) {
                        const bool is = 64 * u + 8 * g < D;
                        raw[u][2 * g] = is && tokA < x.nq ? *reinterpret_cast<const uint32_t*>(qA + 64 * u + 8 * g) : 0u;
                        raw[u][2 * g + 1] = is && tokB < x.nq ? *reinterpret_cast<const uint32_t*>(qB + 64 * u + 8 * g) : 0u;
                    }
#pragma unroll
                for (int u = 0; u < Cfg::SUB; ++u)
#pragma unroll
                    for (int g = 0; g < 8; ++g) {
                        const float2 v0 = number(raw[u][2 * g]), v1 = number(raw[u][2 * g + 1]);
                        topA = max3(topA, fabsf(v0.x), fabsf(v0.y));
                        topB = max3(topB, fabsf(v1.x), fabsf(v1.y));
                    }
                // 2^e <= top < 2^(e + 1): a row goes in as q 2^(8 - e), exact but for what lies 2^32 below its largest number
                const uint32_t eA = min(max(__float_as_uint(quad_max(topA)) >> 23, 1u), 253u), eB = min(max(__float_as_uint(quad_max(topB)) >> 23, 1u), 253u);
                const float downA = __uint_as_float((254u - eA) << 23), downB = __uint_as_float((254u - eB) << 23);
                fA = fmaxf(__uint_as_float(eA << 23) * (a.scale * LOG2E * 0.00390625f), 1.2e-38f);
                fB = fmaxf(__uint_as_float(eB << 23) * (a.scale * LOG2E * 0.00390625f), 1.2e-38f);
#pragma unroll
                for (int u = 0; u < Cfg::SUB; ++u) {
#pragma unroll
                    for (int g = 0; g < 8; ++g) {
                        const float2 v0 = number(raw[u][2 * g]), v1 = number(raw[u][2 * g + 1]);
                        raw[u][2 * g] = t_bits(__floats2half2_rn(v0.x * downA * 256.f, v0.y * downA * 256.f));
                        raw[u][2 * g + 1] = t_bits(__floats2half2_rn(v1.x * downB * 256.f, v1.y * downB * 256.f));
                    }
                    tmem_st_quad32(tmem + TM_Q + 32 * u + lanes, raw[u]);
                }
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars.q_full);
            }
            const uint32_t* const setA = tree + (min(tokA, x.nq - 1) - x.tok0) * TREE_WORDS;
            const uint32_t* const setB = tree + (min(tokB, x.nq - 1) - x.tok0) * TREE_WORDS;
            const int words = (x.nq + 31) / 32;
            bool sets = false;                   // they are known to be there
            float mA = -INFINITY, mB = -INFINITY, lA = 0.f, lB = 0.f;
            const bool some = x.qt * ROWS + r0 < x.nq * a.group;             // the warp has rows
            for (int j = 0; j < x.nt && ok; ++j) {
                const uint32_t m = n + j, buf = m & 1;
                ok = __all_sync(0xffffffffu, mbar_wait(&bars.s_full[buf], (m >> 1) & 1, abortp));
                if (!ok) break;
                if (!some) {                     // (what is there instead of weights stays in these rows)
                    if (lane == 0) mbar_arrive(&bars.p_ready[buf]);
                    continue;
                }
                tc_fence_after();
                const uint32_t tS = tmem + TM_S + buf * KEYS + lanes;
                const unsigned long long have = *reinterpret_cast<const unsigned long long*>(have_s[1][m & 15]);
                const long long key0 = (long long)(x.t0 + j) * KEYS;
                const bool masked = key0 + KEYS > x.ctx || have != 0x0101010101010101ull;
                if (masked && x.meets_tree && !sets) {
                    ok = __all_sync(0xffffffffu, mbar_wait(&bars.sets_full, it & 1, abortp));
                    if (!ok) break;
                    sets = true;
                }
                // Twice over the scores, 64 columns at a time, in loops that are not unrolled: instructions of five kinds of warps share the caches next to the pipes.
                uint32_t s[32];
                float bA = -INFINITY, bB = -INFINITY;
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    tmem_ld_quad64(tS + 64 * half, s);
                    tc_wait_ld();
                    const bool mask = masked && (have != 0x0101010101010101ull || key0 + 64 * half + 64 > x.ctx);
                    if (mask) {
                        // the tile's tokens that a row sees, 32 a word: all ahead of the tree, and the row's set in it; none of blocks that are not there
#pragma unroll
                        for (int z = 0; z < 2; ++z) {
                            const int at32 = (int)(key0 + 64 * half + 32 * z - x.ctx), word = at32 >> 5;
                            const uint32_t both = ((have >> (16 * (2 * half + z)) & 1) ? 0xffffu : 0u) | ((have >> (16 * (2 * half + z) + 8) & 1) ? 0xffff0000u : 0u);
                            auto seen = [&](const uint32_t* set) {
                                const uint32_t l = word < 0 ? 0xffffffffu : word < words ? set[word] : 0u, u = word + 1 < 0 ? 0xffffffffu : word + 1 < words ? set[word + 1] : 0u;
                                return (__funnelshift_r(l, u, at32) & both) >> cq;
                            };
                            const uint32_t A = seen(setA), Bm = seen(setB);
#pragma unroll
                            for (int g = 0; g < 4; ++g) {
                                uint32_t* const v = s + 16 * z + 4 * g;
                                if (!(A >> (8 * g) & 1u)) v[0] = 0xff800000u;
                                if (!(A >> (8 * g + 1) & 1u)) v[1] = 0xff800000u;
                                if (!(Bm >> (8 * g) & 1u)) v[2] = 0xff800000u;
                                if (!(Bm >> (8 * g + 1) & 1u)) v[3] = 0xff800000u;
                            }
                        }
                        tmem_st_quad64(tS + 64 * half, s);
                    }
                    max_quad64(s, bA, bB);
                }
                if (masked) tc_wait_st();
                bA = quad_max(bA) * fA;
                bB = quad_max(bB) * fB;
                float alphaA = 1.f, alphaB = 1.f;
                if (bA > mA + RESCALE_THRESHOLD) { alphaA = ex2_mufu(mA - bA); mA = bA; }        // (also the first tile that the row sees anything of)
                if (bB > mB + RESCALE_THRESHOLD) { alphaB = ex2_mufu(mB - bB); mB = bB; }
                const float nA = mA == -INFINITY ? 0.f : UP - mA, nB = mB == -INFINITY ? 0.f : UP - mB;
                uint64_t sumA = 0, sumB = 0;
                const uint64_t fA2 = t_pair(fA, fA), fB2 = t_pair(fB, fB), nA2 = t_pair(nA, nA), nB2 = t_pair(nB, nB);
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    tmem_ld_quad64(tS + 64 * half, s);
                    tc_wait_ld();
                    uint32_t p[16];
#pragma unroll
                    for (int g = 0; g < 8; ++g) {
                        const float2 v0 = t_pair(t_fma2(t_pair(__uint_as_float(s[4 * g]), __uint_as_float(s[4 * g + 1])), fA2, nA2)), v1 = t_pair(t_fma2(t_pair(__uint_as_float(s[4 * g + 2]), __uint_as_float(s[4 * g + 3])), fB2, nB2));
                        const float x0 = ex2_mufu(v0.x), x1 = ex2_mufu(v0.y), y0 = ex2_mufu(v1.x), y1 = ex2_mufu(v1.y);
                        sumA = t_add2(sumA, t_pair(x0, x1));
                        sumB = t_add2(sumB, t_pair(y0, y1));
                        p[2 * g] = t_weights(x0, x1);
                        p[2 * g + 1] = t_weights(y0, y1);
                    }
                    tmem_st_quad32(tS + 32 * half, p);       // (over scores that this warp alone reads, and has read)
                }
                lA = fmaf(lA, alphaA, t_pair(sumA).x + t_pair(sumA).y);
                lB = fmaf(lB, alphaB, t_pair(sumB).x + t_pair(sumB).y);
                if (j > 0 && __any_sync(0xffffffffu, alphaA != 1.f || alphaB != 1.f)) {
                    // O is in use by the product before this one.  (That of tile m - 2 is done: scores of this tile have come behind it.)
                    ok = __all_sync(0xffffffffu, mbar_wait(&bars.v_empty[buf ^ 1], ((m - 1) >> 1) & 1, abortp));
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int c = 0; c < Cfg::SUB; ++c) {
                        uint32_t v[32];
                        tmem_ld_quad64(tO + 64 * c, v);
                        tc_wait_ld();
#pragma unroll
                        for (int g = 0; g < 8; ++g) {
                            v[4 * g] = __float_as_uint(__uint_as_float(v[4 * g]) * alphaA);
                            v[4 * g + 1] = __float_as_uint(__uint_as_float(v[4 * g + 1]) * alphaA);
                            v[4 * g + 2] = __float_as_uint(__uint_as_float(v[4 * g + 2]) * alphaB);
                            v[4 * g + 3] = __float_as_uint(__uint_as_float(v[4 * g + 3]) * alphaB);
                        }
                        tmem_st_quad64(tO + 64 * c, v);
                    }
                }
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars.p_ready[buf]);
            }
            if (ok && x.nt > 0) ok = __all_sync(0xffffffffu, mbar_wait(&bars.v_empty[(n + x.nt - 1) & 1], ((n + x.nt - 1) >> 1) & 1, abortp));
            if (ok && !sets) ok = __all_sync(0xffffffffu, mbar_wait(&bars.sets_full, it & 1, abortp));
            if (!ok) break;
            // ---- the rows' results
            tc_fence_after();
            lA = quad_sum(lA);
            lB = quad_sum(lB);
            const bool whole = x.parts == 1, isA = tokA < x.nq, isB = tokB < x.nq;
            float* const to = whole ? nullptr : part_at(a.part, x.first_cta, x.part, D);
            const size_t outA = ((size_t)(x.q0 + tokA) * a.kv_heads * a.group + (size_t)x.h * a.group + (rhoA - tokA * a.group)), outB = ((size_t)(x.q0 + tokB) * a.kv_heads * a.group + (size_t)x.h * a.group + (rhoB - tokB * a.group));
            const float iA = lA == 0.f ? 0.f : 1.f / lA, iB = lB == 0.f ? 0.f : 1.f / lB;
            uint32_t nanA = 0, nanB = 0;     // groups of V in which the row sees a NaN
            if (x.meets_tree && any_nan_s[it & 1]) {
                for (int i = lane & 3; i < words; i += 4)
#pragma unroll
                    for (int w = 0; w < G; ++w) {
                        if (nan_s[it & 1][w][i] & setA[i]) nanA |= 1u << w;
                        if (nan_s[it & 1][w][i] & setB[i]) nanB |= 1u << w;
                    }
                nanA |= __shfl_xor_sync(0xffffffffu, nanA, 1); nanA |= __shfl_xor_sync(0xffffffffu, nanA, 2);
                nanB |= __shfl_xor_sync(0xffffffffu, nanB, 1); nanB |= __shfl_xor_sync(0xffffffffu, nanB, 2);
            }
            // (32 columns at a time, in a loop that is not unrolled: this code is fetched anew for every item, and its length is its time)
            const size_t rowA = whole ? outA * D : (size_t)rA * D, rowB = whole ? outB * D : (size_t)rB * D;
#pragma unroll 1
            for (int w = 0; w < G; ++w) {
                uint32_t v[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = 0u;
                if (x.nt > 0) {
                    t_ld_quad32(tO + 32 * w, v);
                    tc_wait_ld();
                }
                const float gA = nanA >> w & 1u ? NAN : whole ? iA : 1.f, gB = nanB >> w & 1u ? NAN : whole ? iB : 1.f;
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int col = 32 * w + 8 * g + cq;
                    const float x0 = __uint_as_float(v[4 * g]) * gA, x1 = __uint_as_float(v[4 * g + 1]) * gA, y0 = __uint_as_float(v[4 * g + 2]) * gB, y1 = __uint_as_float(v[4 * g + 3]) * gB;
                    if (whole) {
                        auto both = [&](float u, float w) { return a.f16 ? t_bits(__floats2half2_rn(u, w)) : pack_bf16x2(u, w); };
                        if (isA) *reinterpret_cast<uint32_t*>(a.out + rowA + col) = both(x0, x1);
                        if (isB) *reinterpret_cast<uint32_t*>(a.out + rowB + col) = both(y0, y1);
                    } else {
                        if (isA) __stcg(reinterpret_cast<float2*>(to + rowA + col), make_float2(x0, x1));
                        if (isB) __stcg(reinterpret_cast<float2*>(to + rowB + col), make_float2(y0, y1));
                    }
                }
            }
            // the rows' maxima and sums: the first lane of a quad those of row A, the second of row B
            if ((lane & 3) < 2) {
                const bool second = lane & 1;
                const float m = second ? mB : mA, l = second ? lB : lA;
                const int r = second ? rB : rA;
                if (second ? isB : isA) {
                    if (!whole) { __stcg(to + ROWS * D + r, m); __stcg(to + ROWS * (D + 1) + r, l); }
                    else if (a.lse) a.lse[second ? outB : outA] = l == 0.f ? -INFINITY : ((m == -INFINITY ? 0.f : m) - UP + log2f(l)) * T_LN2;
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars.sets_free);
            if (warp == SOFT0 && lane == 0 && x.part == 0 && x.parts > 1) a.rows_cut[blockIdx.x] = TreeRow{x.parts, x.q0, x.nq, x.h, x.qt};
            n += x.nt;
        }
    }
    // ---- the end, for all: also of a CTA whose waits ran out
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem, 512);
    if (tid == 0 && abort_flag) atomicExch(&dc->status, (int)PSA_ERR_TIMEOUT);
}

// Joins the parts of the row tiles that were cut: sixteen rows a CTA, a thread four channels, parts in their order.
constexpr int JOIN_ROWS = 16;
template <int D>
__global__ void __launch_bounds__(JOIN_ROWS * D / 4) tree_join_kernel(const TreeArgs a) {
    grid_dependency_wait();
    const TreeRow x = a.rows_cut[blockIdx.x];
    const int r = blockIdx.y * JOIN_ROWS + threadIdx.x / (D / 4), ch = threadIdx.x % (D / 4) * 4, rho = x.qt * ROWS + r;
    if (x.parts == 0 || rho >= x.nq * a.group) return;
    const int c = (int)blockIdx.x, token = (int)fastdiv((uint32_t)rho, a.by_group);
    float top = -INFINITY, sum = 0.f;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    constexpr int AHEAD = 8;
    for (int p0 = 0; p0 < x.parts; p0 += AHEAD) {
        float4 o[AHEAD];
        float m[AHEAD], l[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const float* from = part_at(a.part, c, min(p0 + k, x.parts - 1), D);
            o[k] = __ldcg(reinterpret_cast<const float4*>(from + r * D + ch));
            m[k] = p0 + k < x.parts ? __ldcg(from + ROWS * D + r) : -INFINITY;
            l[k] = p0 + k < x.parts ? __ldcg(from + ROWS * (D + 1) + r) : 0.f;
        }
        float most = top;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) most = fmaxf(most, m[k]);
        const float from = most == -INFINITY ? 0.f : most, old = ex2_mufu(top - from);
        top = most;
        sum *= old;
        v.x *= old; v.y *= old; v.z *= old; v.w *= old;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (p0 + k >= x.parts) break;
            const float f = ex2_mufu(m[k] - from);
            sum = fmaf(f, l[k], sum);
            // (a part in which the row sees nothing: its sums are zeros and its factor is too, and a NaN among them is the row's)
            v.x = fmaf(f, o[k].x, v.x); v.y = fmaf(f, o[k].y, v.y); v.z = fmaf(f, o[k].z, v.z); v.w = fmaf(f, o[k].w, v.w);
        }
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const size_t row = (size_t)(x.q0 + token) * a.kv_heads * a.group + (size_t)x.h * a.group + (rho - token * a.group);
    uint2 y;
    if (a.f16) y = make_uint2(t_bits(__floats2half2_rn(v.x * inv, v.y * inv)), t_bits(__floats2half2_rn(v.z * inv, v.w * inv)));
    else y = make_uint2(pack_bf16x2(v.x * inv, v.y * inv), pack_bf16x2(v.z * inv, v.w * inv));
    *reinterpret_cast<uint2*>(a.out + row * D + ch) = y;
    if (a.lse && ch == 0) a.lse[row] = sum == 0.f ? -INFINITY : ((top == -INFINITY ? 0.f : top) - UP + log2f(sum)) * T_LN2;
}

template <int D>
int launch_tree(const TreeArgs& all, DeviceCounters* dc, DeviceCounters* dc_next, cudaStream_t stream) {
    static DeviceSetup setup;
    const int sms = device_setup(&setup, [] { return cudaFuncSetAttribute(tree_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, TCfg<D>::SMEM); }, "tree attention set-up");
    if (sms <= 0) return PSA_ERR_CUDA;
    const int grid = sms < T_CTAS ? sms : T_CTAS;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    for (int b0 = 0; b0 < all.sequences; b0 += T_SEQS) {
        TreeArgs a = all;
        a.sequences = all.sequences - b0 < T_SEQS ? all.sequences - b0 : T_SEQS;
        a.seqs += b0;
        a.q_starts += b0;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(grid);
        cfg.blockDim = dim3(T_THREADS);
        cfg.dynamicSmemBytes = TCfg<D>::SMEM;
        cfg.stream = stream;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        cudaError_t e = cudaLaunchKernelEx(&cfg, tree_kernel<D>, a, dc, b0 == 0 ? dc_next : nullptr);
        cfg.gridDim = dim3(grid, ROWS / JOIN_ROWS);
        cfg.blockDim = dim3(JOIN_ROWS * D / 4);
        cfg.dynamicSmemBytes = 0;
        if (e == cudaSuccess) e = cudaLaunchKernelEx(&cfg, tree_join_kernel<D>, a);
        if (e != cudaSuccess) { set_cuda_error(e, "tree_kernel launch"); return PSA_ERR_CUDA; }
    }
    return PSA_OK;
}

}  // namespace

// (the rows that are cut, then the parts)
size_t tree_attention_scratch_bytes(int d) { return d > 128 ? 0 : (size_t)T_CTAS * 32 + (size_t)(2 * T_CTAS + 1) * ROWS * (d + 2) * sizeof(float); }

int tree_attention(const psa_cache& c, const void* Q, long long q_stride, const int* parents, const int* seqs, const int* q_starts, int sequences, int rows, int heads, float scale, int dtype,
                   void* out, float* lse, void* scratch, DeviceCounters* dc, DeviceCounters* dc_next, cudaStream_t stream) {
    static_assert(sizeof(TreeRow) <= 32, "");
    const int group = heads / c.kv_heads;
    const TreeArgs a = {static_cast<const uint8_t*>(c.pool), c.tables, c.lens, seqs, q_starts, parents, static_cast<const uint16_t*>(Q), static_cast<uint16_t*>(out), lse,
                        reinterpret_cast<float*>(static_cast<char*>(scratch) + (size_t)T_CTAS * 32), static_cast<TreeRow*>(scratch), q_stride, c.pages, c.slots, c.width, c.page_size, c.kv_heads,
                        group, sequences, rows, dtype == PSA_F16, scale, fastdiv_make((uint32_t)group), fastdiv_make((uint32_t)(c.page_size / CACHE_BLOCK))};
    switch (c.d_k) {
        case 32: return launch_tree<32>(a, dc, dc_next, stream);
        case 64: return launch_tree<64>(a, dc, dc_next, stream);
        case 96: return launch_tree<96>(a, dc, dc_next, stream);
        case 128: return launch_tree<128>(a, dc, dc_next, stream);
        default: return PSA_ERR_UNSUPPORTED;
    }
}

}  // namespace psa
