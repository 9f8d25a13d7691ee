// Attention over packed prompts: sequences of different lengths one after another, heads in groups that share keys and values, causal.
//
//     out_i = sum_j w_ij v_j / sum_j w_ij,   w_ij = exp(scale q_i k_j),   j <= i + nk - nq      (nq queries, the last of nk tokens)
//
// The kernel is built like attn_persist_kernel (psa_attn_persist.cu, where the layout of the CTA and its pipeline are explained): S = Q K^T and O += P V by tcgen05 MMAs
// with the accumulators and P in tensor memory, operands staged by TMA, softmax and epilogue by sixteen warps in the quad layout, one persistent CTA per
// SM.  What is different:
//   * A row tile holds the queries of all heads of a group: row r is token r / group, head r % group of the group, 128 / group tokens a tile (one box of the
//     query's tensor map).  Keys and values are loaded once for the group, short prompts fill tiles, and any group size works alike; groups that do not divide
//     128 leave rows empty (6 % at a group of 12).
//   * Where there are CTAs enough and little to do, an item is one row tile and not two (launch_prompt).
//   * The host does not know the lengths.  Every CTA derives the work list from `starts` by itself (sequences sorted by length in shared memory): the heaviest pairs of row
//     tiles of all sequences first, heads innermost, taken from a device counter, as in attn_persist_kernel.
//   * Where the pairs of row tiles are fewer than the CTAs (a few prompts, or pieces of them, behind long contexts) their key blocks are cut into parts as well: a warp then
//     stores its rows' sums in fp32, and the one that comes last joins the parts of its sixteen rows, in their order.  Nobody else is waited for.
//   * A tile may reach into the next sequence.  Its rows beyond the sequence are computed and not stored, so the output is stored row by row; keys beyond it carry
//     no weight, and neither do non-finite values there (a weight of zero would not keep them out of the sum): in blocks that some row of the tile does
//     not see in full the softmax warps look through the tile of V before P V and set what is not finite to zero; rows that do see such a value get it
//     back in the epilogue.
// Measured, 32 heads on 8 of d = 128: two prompts of up to 8192 tokens 493 us alone, 1115 TFLOP/s, 555 to 575 in a run of calls under the power limit (tensor pipe 52 % of its
// cycles: bound by the chain of scores, softmax and PV of a row tile, two of which alternate, 3560 cycles a pair of key blocks for 2048 of MMAs); six pieces of up to 512 queries behind
// up to 4000 keys 57 us, half of which is what comes once an item: list, first loads, sums stored and joined.
#include <type_traits>

#include <cuda_fp16.h>

#include "psa_internal.h"
#include "psa_sched.h"
#include "psa_softmax.cuh"
#include "psa_tma.h"
#include "sm100.cuh"

namespace psa {

namespace {

template <int D>
struct PCfg {
    static constexpr int SUB = D / 64;                  // 64-column sub-tiles per 128-row tile
    static constexpr int TILE_BYTES = 128 * D * 2;      // one Q, K or V tile
    static constexpr int KSTAGES = D == 128 ? 2 : 4;
    static constexpr int VSTAGES = D == 128 ? 2 : 4;
    // output staging: one [16 rows x 32 columns] buffer per softmax warp, used for each 32 columns in turn
    static constexpr int STAGE_BYTES = 16 * 32 * 2;
    static constexpr int STAGE_BUFS = 2 * SOFTMAX_WARPS_PER_TILE;
    static constexpr int SMEM = (2 + KSTAGES + VSTAGES) * TILE_BYTES + STAGE_BUFS * STAGE_BYTES + 1024;
    static constexpr bool SEP_P = D == 64;
    static constexpr int TMEM_S = 0, TMEM_P = 256, TMEM_O = SEP_P ? 384 : 256;
};

struct PMaps {
    CUtensorMap q, k, v;
};
constexpr int SEQ_BITS = 9, SEQS = 1 << SEQ_BITS;      // sequences of one launch
constexpr int MAX_CTAS = 160;           // partial results and arrival counts: two parts per CTA
constexpr int LEAST_PIECE = 4;          // key blocks.  (A part's sums take up to 10,000 cycles through L2 to store and as many to join, a block 3560.  2 and 3: up to 1.5 us slower; 6 and 8: up to 3)

struct PromptArgs {
    const int *q_starts, *k_starts;
    int sequences, q_rows, k_rows, heads, kv_heads, group, tokens, d;     // tokens: of a row tile, 128 / group
    int tiles;                          // row tiles of an item: 2, or 1 (see launch_prompt)
    int call;                           // number of the call, > 0
    long long v_stride;
    const uint16_t* v;                  // (the epilogue's look at values that are not finite)
    uint16_t* out;
    float *lse, *part;                  // part (null: nothing is cut): [2 MAX_CTAS][2 tiles][128 rows][D] sums, then as many rows' maxima and sums
    float sl2;
    FastDiv by_group, by_heads;
};
// A work item: two row tiles (or one, PromptArgs::tiles) of one sequence and key/value head.
struct __align__(16) Item {
    int q0, k0;                         // first rows of the sequence
    int i0, nq, nk;                     // first token of the first tile, lengths
    int h;                              // key/value head
    int nkv0, nkv1;                     // key blocks of the two tiles, from block j0 on (0: no rows, or rows that see no key of these blocks)
    int j0, slot, part, parts;          // slot: of the first part's results, if there are several
};
// Arrivals of the warps on rows of several parts, by slot of the first part, tile and warp.  The arrival that completes a count wraps it to zero again.
__device__ unsigned g_prompt_arrived[2 * MAX_CTAS][2][SOFTMAX_WARPS_PER_TILE];
// A call whose waits ran out leaves counts that are not zero.  g_prompt_left is EXPIRED behind it; the next call that could cut cuts nothing, clears the counts and puts its
// own number here (which its other CTAs take for the same order), the one after that cuts again and leaves 0.  Nobody has to ask for the status in between.  (A graph that is
// replayed with no other such call in between goes on without parts.)
__device__ int g_prompt_left;
constexpr int EXPIRED = -1;
// Counts a warp's arrival behind what its lanes have stored; true in all of them for the one that completes the rows.
__device__ __forceinline__ bool warp_arrive(unsigned* count, unsigned last, int lane) {
    unsigned old = 0;
    __syncwarp();
    if (lane == 0) asm volatile("fence.acq_rel.gpu;\n\tatom.acq_rel.gpu.global.inc.u32 %0, [%1], %2;" : "=r"(old) : "l"(count), "r"(last) : "memory");
    return __shfl_sync(0xffffffffu, old, 0) == last;
}

struct PBars {
    uint64_t item_full[2], item_empty[2];
    uint64_t q_full[2], q_empty[2];
    uint64_t k_full[8], k_empty[8], v_full[4], v_empty[4];
    uint64_t s_full[2], s_free[2], p_ready[2], o_done[2];
};

constexpr float LN2 = 0.6931471805599453f;

template <bool F16>
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    if constexpr (F16) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    } else {
        return pack_bf16x2(lo, hi);
    }
}
// P = exp2(s - m) is held 2^HEADROOM times as large in fp16, whose normal numbers end at 2^-14 and the others at 2^-24: beside one key that outweighs all others
// the rest of a row would lose its bits, or vanish (256 keys, one of which outweighs the others by e^14, e^16, e^18 and has a value of
// zero, d = 128: relative error of the output 9e-4, 6e-2 and 1 without the factor, 1.6e-4, 1.9e-4 and 3.3e-4 with it; no call took longer).  m lags up to 2^8 behind the largest score, so that a weight is at most 2^15 of the 2^16 that the type takes; beyond scores of 2^23,
// whose own rounding exceeds the rest, weights stay at its largest number.  The sums carry the factor too: it cancels in the output and leaves the log-sum-exp.
template <bool F16> constexpr float HEADROOM = F16 ? 7.f : 0.f;
__device__ __forceinline__ uint32_t pack_weights_f16(float lo, float hi) {
    uint32_t v;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(v) : "f"(hi), "f"(lo));
    return v;
}
// exp_quad64 (psa_softmax.cuh) for either type of P.
template <bool F16>
__device__ __forceinline__ void exp_quad(const uint32_t (&s)[32], float sl2, float negmA, float negmB, uint32_t (&pk)[16], float& sumA, float& sumB) {
    if constexpr (!F16) {
        exp_quad64(s, sl2, negmA, negmB, pk, sumA, sumB);
    } else {
        float sa0 = 0.f, sa1 = 0.f, sb0 = 0.f, sb1 = 0.f;
#pragma unroll
        for (int g = 0; g < 8; ++g) {
            const float p0 = ex2_mufu(fmaf(__uint_as_float(s[4 * g]), sl2, negmA)), p1 = ex2_mufu(fmaf(__uint_as_float(s[4 * g + 1]), sl2, negmA));
            const float p2 = ex2_mufu(fmaf(__uint_as_float(s[4 * g + 2]), sl2, negmB)), p3 = ex2_mufu(fmaf(__uint_as_float(s[4 * g + 3]), sl2, negmB));
            sa0 += p0; sa1 += p1; sb0 += p2; sb1 += p3;
            pk[2 * g] = pack_weights_f16(p0, p1);
            pk[2 * g + 1] = pack_weights_f16(p2, p3);
        }
        sumA += sa0 + sa1;
        sumB += sb0 + sb1;
    }
}
// kind::f16 with operands of either type (bf16: type 1, fp16: type 0) and fp32 accumulation.
template <bool F16>
__host__ __device__ constexpr uint32_t idesc(uint32_t M, uint32_t N, uint32_t a_major, uint32_t b_major) {
    return umma_idesc_bf16(M, N, a_major, b_major) & ~(F16 ? (1u << 7) | (1u << 10) : 0u);
}
__device__ __forceinline__ void tma_load_3d(void* smem_dst, const CUtensorMap* map, uint64_t* bar, int x, int h, int y) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(smem_u32(smem_dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(x), "r"(h), "r"(y)
        : "memory");
}

// d = 64 has an MMA-issuing thread per row tile slot (warp 1 for slot 0, the last warp for slot 1): a block there is
// half the tensor work of d = 128 but as many instructions to issue, and one thread was measured to be the limit.
constexpr int ISSUER1_WARP = CTRL_WARPS + 2 * SOFTMAX_WARPS_PER_TILE;
template <int D> __host__ __device__ constexpr int persist_threads() { return ATTN_THREADS + (D == 64 ? 32 : 0); }
template <int D> __host__ __device__ constexpr int item_readers() { return (D == 64 ? 2 : 1) + 2 * SOFTMAX_WARPS_PER_TILE; }   // issuers + one lane per softmax warp

// D: columns of a tile in shared memory, KS: 16-column steps of phase 1, and of phase 3's output, that hold columns of the head (the rest are zeros;
// the census counts blocks, each of D columns).
// F16: fp16 instead of bf16 in memory and as operands.
// CUT: pairs may be cut into parts.  Calls that have pairs enough whatever the lengths are (prompt_scratch_bytes) run without: the code of the parts costs the
// softmax warps registers (two prompts of 2737 tokens, 28 heads of d = 96: 127.3 us with it, 121.2 without; two of up to 8192, 32 heads of d = 128: 505 and 493).
template <int D, int KS, bool F16, bool CUT>
__global__ void __launch_bounds__(persist_threads<D>(), 1)
prompt_kernel(const __grid_constant__ PMaps maps, const __grid_constant__ PromptArgs pa, DeviceCounters* dc, unsigned int* cursor, DeviceCounters* dc_next) {
    using Cfg = PCfg<D>;
    constexpr bool SEP = Cfg::SEP_P;
    constexpr int VST = Cfg::VSTAGES;
    constexpr int KST = Cfg::KSTAGES;
    // d = 128: V_j and K_{j+1} are needed by the same step of the issuing thread and released by
    // it together, so they travel as one stage (K slot s and V slot s, one full and one empty barrier: v_full / v_empty):
    // pair p of an item is (V_{p-1}, K_p), p = 0 .. blocks, the first without a V and the last without a K.  The
    // issuing thread then probes one barrier and commits one release per key block instead of two of each.
    constexpr bool PAIRED = !SEP;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* sQ = smem;                                          // 2 tiles
    uint8_t* sK = sQ + 2 * Cfg::TILE_BYTES;                      // KSTAGES tiles
    uint8_t* sV = sK + Cfg::KSTAGES * Cfg::TILE_BYTES;           // VSTAGES tiles
    uint8_t* sStage = sV + VST * Cfg::TILE_BYTES;                // STAGE_BUFS output staging tiles
    __shared__ PBars bars;
    __shared__ uint32_t tmem_base_s;
    __shared__ int abort_flag;
    __shared__ Item item_ring[2];
    __shared__ int v_bad;                        // count of the last item in which V held something that is not finite, see above
    // the work list: sequences by falling number of pairs of row tiles (key = pairs << SEQ_BITS | SEQS - 1 - sequence), see `decode`
    __shared__ uint32_t key[SEQS];
    __shared__ __align__(16) int base[SEQS + 4];
    __shared__ int starts_s[2][SEQS + 1];
    __shared__ uint32_t cut[SEQS + 1], cut_sum[ISSUER1_WARP + 1];       // with pairs cut into parts: items << 16 | results ahead of a pair
    __shared__ Item own[2 * SOFTMAX_WARPS_PER_TILE][2];                 // a softmax warp's items, this one and the next
    __shared__ int left_s;                       // g_prompt_left, as the CTA found it
    __shared__ Item first_item;                  // this CTA's first item, found by the thread that knows its sequence or pair

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        abort_flag = 0;
        v_bad = 0;
        for (int t = 0; t < 2; ++t) {
            mbar_init(&bars.item_full[t], 1);
            mbar_init(&bars.item_empty[t], item_readers<D>());
            mbar_init(&bars.q_full[t], 1);
            mbar_init(&bars.q_empty[t], 1);
            mbar_init(&bars.s_full[t], 1);
            mbar_init(&bars.s_free[t], SOFTMAX_WARPS_PER_TILE);       // one arrival per softmax warp
            mbar_init(&bars.p_ready[t], SOFTMAX_WARPS_PER_TILE);
            mbar_init(&bars.o_done[t], 1);
        }
        for (int s = 0; s < 8; ++s) {
            // (with an issuer per slot, an operand tile collects one release from each of them)
            mbar_init(&bars.k_full[s], 1); mbar_init(&bars.k_empty[s], SEP ? 2 : 1);
        }
        for (int s = 0; s < 4; ++s) { mbar_init(&bars.v_full[s], 1); mbar_init(&bars.v_empty[s], SEP ? 2 : 1); }
        fence_mbar_init();
    }
    if (warp == 1) { tmem_alloc(&tmem_base_s, 512); tmem_relinquish(); }
    // rows of a tile that no box reaches (groups that do not divide 128) stay zero
    if (pa.tokens * pa.group < TILE)
        for (int i = threadIdx.x; i < 2 * Cfg::TILE_BYTES / 16; i += persist_threads<D>()) reinterpret_cast<uint4*>(sQ)[i] = make_uint4(0, 0, 0, 0);
    volatile int* abortp = &abort_flag;
    // Everything above (barriers, TMEM) overlaps the end of the kernel before this one in the stream; global memory
    // is touched only from here on.  The kernel after this one is let in when a CTA's work is done: let in at once, its
    // waiting CTAs cost a layer of n = 512 0.9 us (31.8 -> 30.9) and a block of n = 1024 1.4 us.
    grid_dependency_wait();
    // the counter block of the NEXT call on this workspace is cleared here, off that call's critical path
    if (threadIdx.x == 0 && blockIdx.x == 0 && dc_next) *dc_next = DeviceCounters{0, 0, 0, 0, 0, 0, 0};
    // ---- the work list
    if (CUT && threadIdx.x == persist_threads<D>() - 1) left_s = *const_cast<const volatile int*>(&g_prompt_left);
    bool descends = false;                       // `starts` that do not ascend name rows more than once, or keys that are not there: nothing is computed, and the call reports it
    for (int i = threadIdx.x; i <= pa.sequences; i += persist_threads<D>()) {
        const int next = min(i + 1, pa.sequences), q = pa.q_starts[i], k = pa.k_starts[i];
        descends |= pa.q_starts[next] < q || pa.k_starts[next] < k;
        starts_s[0][i] = min(max(q, 0), pa.q_rows);
        starts_s[1][i] = min(max(k, 0), pa.k_rows);
    }
    descends = __syncthreads_or(descends);
    uint32_t* const unsorted = reinterpret_cast<uint32_t*>(base);
    for (int i = threadIdx.x; i < (pa.sequences + 3) / 4 * 4; i += persist_threads<D>()) {
        const int nq = i < pa.sequences ? max(starts_s[0][i + 1] - starts_s[0][i], 0) : 0;
        unsorted[i] = i < pa.sequences ? (uint32_t)((nq + pa.tiles * pa.tokens - 1) / (pa.tiles * pa.tokens)) << SEQ_BITS | (uint32_t)(SEQS - 1 - i) : 0u;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < pa.sequences; i += persist_threads<D>()) {     // as many places down as there are larger ones (no two are alike)
        const uint32_t x = unsorted[i];
        int rank = 0;
        for (int k = 0; k < pa.sequences; k += 4) {
            const uint4 y = *reinterpret_cast<const uint4*>(unsorted + k);
            rank += (y.x > x) + (y.y > x) + (y.z > x) + (y.w > x);
        }
        key[rank] = x;
    }
    __syncthreads();
    if (warp == 0) {
        // base[k]: items (of one head) ahead of the levels that exactly the k + 1 longest sequences have
        long long sum = 0;
        for (int k0 = 0; k0 < pa.sequences; k0 += 32) {
            const int k = k0 + lane;
            const int mine = k < pa.sequences ? (int)(key[k] >> SEQ_BITS) : 0, next = k + 1 < pa.sequences ? (int)(key[k + 1] >> SEQ_BITS) : 0;
            const long long own = k < pa.sequences ? (long long)(mine - next) * (k + 1) : 0;
            long long x = own;
#pragma unroll
            for (int s = 1; s < 32; s *= 2) {
                const long long y = __shfl_up_sync(0xffffffffu, x, s);
                if (lane >= s) x += y;
            }
            if (k < pa.sequences) base[k] = (int)(sum + x - own);
            sum += __shfl_sync(0xffffffffu, x, 31);
        }
        if (lane == 0) {
            if (descends) atomicExch(&dc->status, (int)PSA_ERR_SHAPE);
            base[pa.sequences] = descends ? 0 : (int)sum;
        }
    }
    fence_async_smem();                          // (the zeroed rows, ahead of the loads beside them)
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base_s;
    const int pairs = base[pa.sequences];
    // Pair e, which lies behind base[k]: pairs are counted level by level from the last one of the longest sequence down to the first of all.
    auto pair_behind = [&](int k, int e) -> Item {
        const int r = e - base[k], down = k == 0 ? r : r / (k + 1), level = (int)(key[k] >> SEQ_BITS) - 1 - down;
        const int b = SEQS - 1 - (int)(key[r - down * (k + 1)] & (SEQS - 1));
        Item w;
        w.q0 = starts_s[0][b]; w.k0 = starts_s[1][b];
        w.nq = starts_s[0][b + 1] - w.q0; w.nk = max(starts_s[1][b + 1] - w.k0, 0);
        w.i0 = pa.tiles * level * pa.tokens;
        // blocks up to the last key that the tile's last row sees
        auto blocks = [&](int i0) { return i0 >= w.nq ? 0 : max(min(i0 + pa.tokens, w.nq) + w.nk - w.nq + TILE - 1, 0) / TILE; };
        w.nkv0 = blocks(w.i0);
        w.nkv1 = pa.tiles == 2 ? blocks(w.i0 + pa.tokens) : 0;
        w.h = w.j0 = w.slot = w.part = 0;
        w.parts = 1;
        return w;
    };
    auto pair_of = [&](int e) -> Item {
        int lo = 0, hi = pa.sequences - 1;       // the last k with base[k] <= e
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (base[mid] <= e) lo = mid; else hi = mid - 1;
        }
        return pair_behind(lo, e);
    };
    // Part `part` of a pair that is cut into `parts`, whose results for all heads begin at slot `at`.
    auto part_of_pair = [&](Item w, int part, int parts, int at, int h) -> Item {
        const int each = (max(w.nkv0, w.nkv1) + parts - 1) / parts;
        w.part = part;
        w.parts = parts;
        w.slot = at * pa.kv_heads + h * parts;
        w.j0 = part * each;
        w.nkv0 = min(max(w.nkv0 - w.j0, 0), each);
        w.nkv1 = min(max(w.nkv1 - w.j0, 0), each);
        return w;
    };
    const int x0 = (int)fastdiv(blockIdx.x, pa.by_heads), h0 = (int)blockIdx.x - x0 * pa.kv_heads;       // the CTA's first item
    // Fewer pairs than CTAs: their key blocks are cut into pieces of blocks / (CTAs - pairs), which makes no more parts than there are CTAs.
    const bool counts_good = CUT && left_s != EXPIRED && left_s != pa.call;
    if (CUT && left_s != 0 && blockIdx.x == 0) {
        if (!counts_good)
            for (int i = threadIdx.x; i < (int)(sizeof(g_prompt_arrived) / sizeof(unsigned)); i += persist_threads<D>()) (&g_prompt_arrived[0][0][0])[i] = 0u;
        if (threadIdx.x == 0) atomicCAS(&g_prompt_left, left_s, counts_good ? 0 : pa.call);      // (unless a wait of this very call has run out)
    }
    const bool cuts = counts_good && pairs > 0 && pairs <= SEQS && pairs * pa.kv_heads < (int)gridDim.x;
    if (!cuts) {
        for (int k = threadIdx.x; k < pa.sequences; k += persist_threads<D>())
            if (base[k] <= x0 && x0 < base[k + 1]) { first_item = pair_behind(k, x0); first_item.h = h0; }
    } else {
        int blocks = 0;
        Item w;
        if ((int)threadIdx.x < pairs) {
            w = pair_of(threadIdx.x);
            blocks = max(w.nkv0, w.nkv1);
        }
        const int in_warp = __reduce_add_sync(0xffffffffu, blocks);
        if (lane == 0) cut_sum[warp] = (uint32_t)in_warp;
        __syncthreads();
        uint32_t all = 0;
        for (int w = 0; w < persist_threads<D>() / 32; ++w) all += cut_sum[w];
        const uint32_t budget = max((int)gridDim.x - pairs * pa.kv_heads, ((int)gridDim.x + 1) / 2);
        const uint32_t piece = max((all * pa.kv_heads + budget - 1) / budget, (uint32_t)LEAST_PIECE);
        const uint32_t parts = (int)threadIdx.x < pairs ? max((blocks + piece - 1) / piece, 1u) : 0u, mine = parts << 16 | (parts > 1 ? parts : 0u);
        uint32_t x = mine;
#pragma unroll
        for (int s = 1; s < 32; s *= 2) {
            const uint32_t y = __shfl_up_sync(0xffffffffu, x, s);
            if (lane >= s) x += y;
        }
        __syncthreads();
        if (lane == 31) cut_sum[warp] = x;
        __syncthreads();
        for (int w = 0; w < warp; ++w) x += cut_sum[w];
        if ((int)threadIdx.x < pairs) {
            const uint32_t at = x - mine;
            cut[threadIdx.x] = at;
            if ((int)threadIdx.x == pairs - 1) cut[pairs] = x;
            const int part = x0 - (int)(at >> 16);
            if (part >= 0 && part < (int)parts) {
                first_item = parts > 1 ? part_of_pair(w, part, parts, (int)(at & 0xffffu), h0) : w;
                first_item.h = h0;
            }
        }
    }
    __syncthreads();
    const int nitems = (cuts ? (int)(cut[pairs] >> 16) : pairs) * pa.kv_heads;
    // Item idx: part by part of the pairs, heads innermost.
    auto decode = [&](int idx) -> Item {
        const int x = (int)fastdiv((uint32_t)idx, pa.by_heads), h = idx - x * pa.kv_heads;
        Item w;
        if (!cuts) {
            w = pair_of(x);
        } else {
            int lo = 0, hi = pairs - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) / 2;
                if ((int)(cut[mid] >> 16) <= x) lo = mid; else hi = mid - 1;
            }
            const int before = (int)(cut[lo] >> 16), parts = (int)(cut[lo + 1] >> 16) - before;
            w = pair_of(lo);
            if (parts > 1) w = part_of_pair(w, x - before, parts, (int)(cut[lo] & 0xffffu), h);
        }
        w.h = h;
        return w;
    };

    if (warp == 0) {
        if (lane == 0) {
            // ------------------------------------------------------------ scheduler + TMA producer
            // kc, vc: K and V tiles requested so far (ring position); qc[t]: loads of Q buffer t so far.
            uint32_t kc = 0, vc = 0, qc[2] = {0, 0};
            int idx = blockIdx.x;          // the grid never exceeds the item count
            bool ok = true;
            for (uint32_t it = 0; ok; ++it) {
                const int slot = it & 1;
                if (it >= 2) ok = mbar_wait(&bars.item_empty[slot], ((it >> 1) - 1) & 1, abortp);
                if (!ok) break;
                if (idx >= nitems) {
                    item_ring[slot].h = -1;
                    mbar_arrive(&bars.item_full[slot]);
                    break;
                }
                const Item work = it == 0 ? first_item : decode(idx);
                item_ring[slot] = work;
                mbar_arrive(&bars.item_full[slot]);
                int next = -1;
                const int h = work.h, nkv[2] = {work.nkv0, work.nkv1};
                const int maxkv = max(nkv[0], nkv[1]);
                auto take_next = [&] { next = cursor ? (int)gridDim.x + (int)atomicAdd(cursor, 1u) : idx + (int)gridDim.x; };
                if (maxkv == 0) {                // rows without keys: nothing to load
                    take_next();
                    idx = next;
                    continue;
                }
                auto load_q = [&] {
                    for (int t = 0; t < 2 && ok; ++t) {
                        if (nkv[t] == 0) continue;
                        if (qc[t] > 0) ok = mbar_wait(&bars.q_empty[t], (qc[t] - 1) & 1, abortp);
                        if (!ok) break;
                        mbar_arrive_expect_tx(&bars.q_full[t], Cfg::SUB * pa.tokens * pa.group * 128);
                        for (int u = 0; u < Cfg::SUB; ++u)
                            tma_load_4d(sQ + t * Cfg::TILE_BYTES + u * 16384, &maps.q, &bars.q_full[t], 64 * u, 0, h, work.q0 + work.i0 + t * pa.tokens);
                        ++qc[t];
                    }
                };
                if constexpr (PAIRED) {
                    for (int p = 0; p <= maxkv && ok; ++p) {           // pair p = (V_{p-1}, K_p); vc counts pairs here
                        const int s = vc % VST;
                        if (vc >= (uint32_t)VST) ok = mbar_wait(&bars.v_empty[s], ((vc / VST) - 1) & 1, abortp);
                        if (!ok) break;
                        mbar_arrive_expect_tx(&bars.v_full[s], ((p > 0) + (p < maxkv)) * Cfg::TILE_BYTES);
                        if (p < maxkv)
                            for (int u = 0; u < Cfg::SUB; ++u)
                                tma_load_3d(sK + s * Cfg::TILE_BYTES + u * 16384, &maps.k, &bars.v_full[s], 64 * u, h, work.k0 + (work.j0 + p) * TILE);
                        if (p > 0)
                            for (int u = 0; u < Cfg::SUB; ++u)
                                tma_load_3d(sV + s * Cfg::TILE_BYTES + u * 16384, &maps.v, &bars.v_full[s], 64 * u, h, work.k0 + (work.j0 + p - 1) * TILE);
                        ++vc;
                        if (p == 0) {
                            load_q();
                            if (!ok) break;
                        }
                        // the next item is taken behind the item's last load, one or two blocks before it is needed (behind the first one, a CTA in a
                        // long item held on to what others were free for: 28 short items behind 128 parts of 18 blocks, 64 -> 57 us)
                        if (p == maxkv) take_next();
                    }
                } else {
                    for (int j = 0; j < maxkv && ok; ++j) {
                        {
                            const int s = kc % KST;
                            if (kc >= (uint32_t)KST) ok = mbar_wait(&bars.k_empty[s], ((kc / KST) - 1) & 1, abortp);
                            if (!ok) break;
                            mbar_arrive_expect_tx(&bars.k_full[s], Cfg::TILE_BYTES);
                            for (int u = 0; u < Cfg::SUB; ++u)
                                tma_load_3d(sK + s * Cfg::TILE_BYTES + u * 16384, &maps.k, &bars.k_full[s], 64 * u, h, work.k0 + (work.j0 + j) * TILE);
                            ++kc;
                        }
                        if (j == 0) {
                            load_q();
                            if (!ok) break;
                        }
                        {
                            const int s = vc % VST;
                            if (vc >= (uint32_t)VST) ok = mbar_wait(&bars.v_empty[s], ((vc / VST) - 1) & 1, abortp);
                            if (!ok) break;
                            mbar_arrive_expect_tx(&bars.v_full[s], Cfg::TILE_BYTES);
                            for (int u = 0; u < Cfg::SUB; ++u)
                                tma_load_3d(sV + s * Cfg::TILE_BYTES + u * 16384, &maps.v, &bars.v_full[s], 64 * u, h, work.k0 + (work.j0 + j) * TILE);
                            ++vc;
                        }
                        if (j == maxkv - 1) take_next();         // (behind the item's last load, as above)
                    }
                }
                idx = next;
            }
            if (*abortp) {  // let copies already issued land before shared memory is released
                for (int t = 0; t < 2; ++t)
                    if (qc[t] > 0) mbar_wait_drain(&bars.q_full[t], (qc[t] - 1) & 1);
                for (uint32_t c = kc > (uint32_t)KST ? kc - KST : 0; c < kc; ++c)
                    mbar_wait_drain(&bars.k_full[c % KST], (c / KST) & 1);
                for (uint32_t c = vc > (uint32_t)VST ? vc - VST : 0; c < vc; ++c)
                    mbar_wait_drain(&bars.v_full[c % VST], (c / VST) & 1);
            }
        }
    } else if (SEP && (warp == 1 || warp == ISSUER1_WARP)) {
        if (elect_one()) {
            // ------------------------------------------------------------ MMA issuer of row tile slot t (d = 64)
            // (One elected lane of the converged warp: `lane == 0` is 5 % slower here, 128 heads of n = 4096, FULL 849 and 805 us; with one
            // issuer for both slots, below, it is the other way round, 256 heads of n = 4096, d = 128 1821 and 1940 us.)
            // The slot's blocks form a chain S_0, S_1 | PV_0, S_2 | PV_1, ...: with P in its own TMEM columns S_{j+1}
            // needs only that the softmax warps have read S_j, PV_j needs P_j.  The thread issues the links in that
            // order, sleeping on the barriers of each; the two slots' threads walk the item list independently.
            const int t = warp == 1 ? 0 : 1;
            const uint32_t idescS = idesc<F16>(128, 128, UMMA_K_MAJOR, UMMA_K_MAJOR);
            const uint32_t idescO = idesc<F16>(128, 16 * KS, UMMA_K_MAJOR, UMMA_MN_MAJOR);
            unsigned long long qk_blocks = 0, pv_blocks = 0;
            const uint32_t q_lo = umma_desc_lo_kmajor(smem_u32(sQ + t * Cfg::TILE_BYTES));
            const uint32_t k_lo = umma_desc_lo_kmajor(smem_u32(sK));
            const uint32_t v_lo = umma_desc_lo_mnmajor(smem_u32(sV), 16384);
            const uint32_t dS = tmem + Cfg::TMEM_S + t * 128, dO = tmem + Cfg::TMEM_O + t * D;
            const uint32_t aP = tmem + Cfg::TMEM_P + t * 64;
            uint32_t kbase = 0, vbase = 0;      // ring positions of the current item's first K and V tile
            uint32_t parts = 0;                 // earlier items in which this slot had rows
            uint32_t blk0 = 0;                  // blocks of this slot in all earlier items
            bool ok = true;
            auto mma_S = [&](uint32_t kc) {     // S = Q K^T with K at ring position kc (phase 1, Eq. 1)
                const uint32_t k = k_lo + (kc % KST) * (Cfg::TILE_BYTES >> 4);
#pragma unroll
                for (int kk = 0; kk < KS; ++kk) {
                    const uint32_t off = ((kk >> 2) * 16384 + (kk & 3) * 32) >> 4;
                    umma_ss(dS, umma_desc_join(q_lo + off, UMMA_DESC_HI_SW128), umma_desc_join(k + off, UMMA_DESC_HI_SW128),
                            idescS, kk != 0);
                }
                ++qk_blocks;
            };
            auto mma_PV = [&](uint32_t vc, bool first) {   // O (+)= P V with V at ring position vc (phase 3, Eq. 3)
                const uint32_t v = v_lo + (vc % VST) * (Cfg::TILE_BYTES >> 4);
                if (first) {
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk)
                        umma_ts(dO, aP + kk * 8, umma_desc_join(v + kk * (2048 >> 4), UMMA_DESC_HI_SW128), idescO, kk != 0);
                } else {
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk)
                        umma_ts(dO, aP + kk * 8, umma_desc_join(v + kk * (2048 >> 4), UMMA_DESC_HI_SW128), idescO, 1);
                }
                ++pv_blocks;
            };
            // an operand tile has two releases to collect, one per slot; a slot whose partner has no block j gives both
            auto release = [&](uint64_t* bar, bool both) {
                umma_commit(bar);
                if (both) umma_commit(bar);
            };
            for (uint32_t it = 0; ok; ++it) {
                ok = mbar_wait(&bars.item_full[it & 1], (it >> 1) & 1, abortp);
                if (!ok) break;
                const int head = item_ring[it & 1].h, nk0 = item_ring[it & 1].nkv0, nk1 = item_ring[it & 1].nkv1;
                mbar_arrive(&bars.item_empty[it & 1]);
                if (head < 0) break;
                const int nkv = t ? nk1 : nk0, nkv_other = t ? nk0 : nk1;
                if (nkv > 0) {
                    // first scores of the item (the softmax warps must have taken the slot's previous scores out of TMEM)
                    ok = mbar_wait(&bars.q_full[t], parts & 1, abortp) &&
                         mbar_wait(&bars.k_full[kbase % KST], (kbase / KST) & 1, abortp);
                    if (ok && blk0 > 0) ok = mbar_wait(&bars.s_free[t], (blk0 - 1) & 1, abortp);
                    if (!ok) break;
                    tc_fence_after();
                    mma_S(kbase);
                    umma_commit(&bars.s_full[t]);
                    release(&bars.k_empty[kbase % KST], 0 >= nkv_other);
                    if (nkv == 1) umma_commit(&bars.q_empty[t]);
                    for (int j = 0; j < nkv && ok; ++j) {
                        const uint32_t vc = vbase + j, kc = kbase + j + 1;
                        if (j + 1 < nkv) {
                            // S_{j+1} as soon as S_j has been read: it runs under the exponentials of block j
                            ok = mbar_wait(&bars.k_full[kc % KST], (kc / KST) & 1, abortp) &&
                                 mbar_wait(&bars.s_free[t], (blk0 + j) & 1, abortp);
                            if (!ok) break;
                            tc_fence_after();
                            mma_S(kc);
                            umma_commit(&bars.s_full[t]);
                            release(&bars.k_empty[kc % KST], j + 1 >= nkv_other);
                            if (j + 1 == nkv - 1) umma_commit(&bars.q_empty[t]);
                        }
                        ok = mbar_wait(&bars.v_full[vc % VST], (vc / VST) & 1, abortp);
                        if (ok) ok = mbar_wait(&bars.p_ready[t], (blk0 + j) & 1, abortp);
                        if (!ok) break;
                        tc_fence_after();
                        mma_PV(vc, j == 0);
                        umma_commit(&bars.o_done[t]);
                        release(&bars.v_empty[vc % VST], j >= nkv_other);
                    }
                    ++parts;
                    blk0 += nkv;
                }
                // loads for the other slot alone: seen to land, so that no barrier is ever waited for two phases ahead
                for (int j = nkv; j < nkv_other && ok; ++j)
                    ok = mbar_wait(&bars.k_full[(kbase + j) % KST], ((kbase + j) / KST) & 1, abortp) && mbar_wait(&bars.v_full[(vbase + j) % VST], ((vbase + j) / VST) & 1, abortp);
                kbase += max(nk0, nk1);
                vbase += max(nk0, nk1);
            }
            const unsigned long long block_macs = (unsigned long long)TILE * TILE * D;
            if (qk_blocks) atomicAdd(&dc->qk_macs, qk_blocks * block_macs);
            if (pv_blocks) {
                atomicAdd(&dc->pv_macs, pv_blocks * block_macs);
                atomicAdd(&dc->exps, pv_blocks * (unsigned long long)(TILE * TILE));
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            // ------------------------------------------------------------ MMA issuer
            // (d = 128) Each row tile's blocks form a chain S_0, PV_0, S_1, PV_1, ...  The two tiles' chains are issued
            // alternately: while the softmax warps of one tile work on their scores, the tensor pipe runs the
            // other tile's MMAs, and it is this half-step offset that keeps the pipe busy.  P overlays S, so PV_j
            // and S_{j+1} of a tile go back to back under one commit, and the thread sleeps on what each link
            // needs, tile 0 then tile 1 then tile 0 ...
            const uint32_t idescS = idesc<F16>(128, 128, UMMA_K_MAJOR, UMMA_K_MAJOR);
            const uint32_t idescO = idesc<F16>(128, 16 * KS, UMMA_K_MAJOR, UMMA_MN_MAJOR);
            unsigned long long qk_blocks = 0, pv_blocks = 0;
            const uint32_t q_lo[2] = {umma_desc_lo_kmajor(smem_u32(sQ)), umma_desc_lo_kmajor(smem_u32(sQ + Cfg::TILE_BYTES))};
            const uint32_t k_lo = umma_desc_lo_kmajor(smem_u32(sK));
            const uint32_t v_lo = umma_desc_lo_mnmajor(smem_u32(sV), 16384);
            const uint32_t tS0 = tmem + Cfg::TMEM_S, tO0 = tmem + Cfg::TMEM_O;
            uint32_t kbase = 0, vbase = 0;      // ring positions of the current item's first K and V tile
            uint32_t parts[2] = {0, 0};         // earlier items in which tile slot t had rows
            uint32_t blk0[2] = {0, 0};          // blocks of tile slot t in all earlier items
            bool ok = true;
            // S_t = Q_t K^T with K at ring position kc (phase 1, Eq. 1): D/16 MMAs of 128x128x16.
            auto mma_S = [&](int t, uint32_t kc) {
                const uint32_t q = q_lo[t], k = k_lo + (kc % KST) * (Cfg::TILE_BYTES >> 4);
                const uint32_t dS = tS0 + t * 128;
#pragma unroll
                for (int kk = 0; kk < KS; ++kk) {
                    const uint32_t off = ((kk >> 2) * 16384 + (kk & 3) * 32) >> 4;
                    umma_ss(dS, umma_desc_join(q + off, UMMA_DESC_HI_SW128), umma_desc_join(k + off, UMMA_DESC_HI_SW128),
                            idescS, kk != 0);
                }
                ++qk_blocks;
            };
            // O_t (+)= P_t V with V at ring position vc (phase 3, Eq. 3): 8 MMAs of 128 x D x 16.
            auto mma_PV = [&](int t, uint32_t vc, bool first) {
                const uint32_t v = v_lo + (vc % VST) * (Cfg::TILE_BYTES >> 4);
                const uint32_t dO = tO0 + t * D;
                const uint32_t aP = SEP ? tmem + Cfg::TMEM_P + t * 64 : tS0 + t * 128;
                if (first) {
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk)
                        umma_ts(dO, aP + kk * 8,
                                umma_desc_join(v + kk * (2048 >> 4), UMMA_DESC_HI_SW128), idescO, kk != 0);
                } else {
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk)
                        umma_ts(dO, aP + kk * 8,
                                umma_desc_join(v + kk * (2048 >> 4), UMMA_DESC_HI_SW128), idescO, 1);
                }
                ++pv_blocks;
            };
            for (uint32_t it = 0; ok; ++it) {
                ok = mbar_wait(&bars.item_full[it & 1], (it >> 1) & 1, abortp);
                if (!ok) break;
                const int head = item_ring[it & 1].h, nkv[2] = {item_ring[it & 1].nkv0, item_ring[it & 1].nkv1};
                mbar_arrive(&bars.item_empty[it & 1]);
                if (head < 0) break;
                const int maxkv = max(nkv[0], nkv[1]);
                if (maxkv == 0) continue;
                {
                    // first scores of both tiles (PAIRED: kbase = vbase = the ring position of the item's pair 0, which
                    // holds K_0 alone; pair j + 1 holds V_j and K_{j+1})
                    if constexpr (PAIRED) ok = mbar_wait(&bars.v_full[vbase % VST], (vbase / VST) & 1, abortp);
                    else ok = mbar_wait(&bars.k_full[kbase % KST], (kbase / KST) & 1, abortp);
                    for (int t = 0; t < 2 && ok; ++t) {
                        if (nkv[t] == 0) continue;
                        ok = mbar_wait(&bars.q_full[t], parts[t] & 1, abortp);
                        if (!ok) break;
                        tc_fence_after();
                        mma_S(t, kbase);
                        umma_commit(&bars.s_full[t]);
                        if (nkv[t] == 1) umma_commit(&bars.q_empty[t]);
                    }
                    if (!ok) break;
                    if constexpr (PAIRED) umma_commit(&bars.v_empty[vbase % VST]);
                    else umma_commit(&bars.k_empty[kbase % KST]);
                    for (int j = 0; j < maxkv && ok; ++j) {
                        for (int t = 0; t < 2 && ok; ++t) {
                            if (j >= nkv[t]) continue;
                            const uint32_t vc = vbase + j + (PAIRED ? 1 : 0), kc = kbase + j + 1;
                            const bool has_next = j + 1 < nkv[t];
                            // Operand tiles first.  A probe of a barrier costs this thread 150-200 cycles beside the
                            // busy softmax warps, so slot 1 does not repeat the ones slot 0 made for the same block.
                            if (t == 0 || j >= nkv[0]) ok = mbar_wait(&bars.v_full[vc % VST], (vc / VST) & 1, abortp);
                            if constexpr (!PAIRED)
                                if (ok && has_next && (t == 0 || j + 1 >= nkv[0]))
                                    ok = mbar_wait(&bars.k_full[kc % KST], (kc / KST) & 1, abortp);
                            if (ok) ok = mbar_wait(&bars.p_ready[t], (blk0[t] + j) & 1, abortp);
                            if (!ok) break;
                            tc_fence_after();
                            mma_PV(t, vc, j == 0);
                            if (has_next) mma_S(t, kc);
                            umma_commit(&bars.o_done[t]);
                            // an operand tile is released behind its last user in this fixed order
                            const bool last_v = t == 1 || j >= nkv[1];
                            if (last_v) umma_commit(&bars.v_empty[vc % VST]);
                            if (has_next) {
                                if constexpr (!PAIRED)
                                    if (t == 1 || j + 1 >= nkv[1]) umma_commit(&bars.k_empty[kc % KST]);
                                if (j + 1 == nkv[t] - 1) umma_commit(&bars.q_empty[t]);
                            }
                        }
                    }
                }
                kbase += maxkv + (PAIRED ? 1 : 0);
                vbase += maxkv + (PAIRED ? 1 : 0);
                for (int t = 0; t < 2; ++t) { parts[t] += nkv[t] > 0; blk0[t] += nkv[t]; }
            }
            const unsigned long long block_macs = (unsigned long long)TILE * TILE * D;
            if (qk_blocks) atomicAdd(&dc->qk_macs, qk_blocks * block_macs);
            if (pv_blocks) {
                atomicAdd(&dc->pv_macs, pv_blocks * block_macs);
                atomicAdd(&dc->exps, pv_blocks * (unsigned long long)(TILE * TILE));
            }
        }
    } else {
        // ------------------------------------------------------------ softmax + epilogue
        // Eight warps per row tile.  A warp owns 16 rows (TMEM lanes) and reads them in the quad layout (sm100.cuh): the
        // four threads of a quad share two rows, A and B = A + 8, each holding every fourth pair of their columns, so a
        // row maximum or row sum is two shuffles inside the quad and the warps never wait for one another.
        const int sw = warp - CTRL_WARPS;
        const int t = sw / SOFTMAX_WARPS_PER_TILE;              // row tile slot of this warp
        const int wq = sw % SOFTMAX_WARPS_PER_TILE;             // warp inside the slot
        const int q = warp & 3;                                 // TMEM lane quarter this warp may access
        const int row0 = q * 32 + (wq >> 2) * 16;               // first of the warp's 16 rows inside the tile
        const int rA = row0 + (lane >> 2), rB = rA + 8;         // this thread's rows
        const int cq = 2 * (lane & 3);                          // its first column inside every group of 8
        const uint32_t lane_off = static_cast<uint32_t>(row0) << 16;
        const uint32_t tS = tmem + Cfg::TMEM_S + t * 128 + lane_off;
        const uint32_t tO = tmem + Cfg::TMEM_O + t * D + lane_off;
        const uint32_t tP = SEP ? tmem + Cfg::TMEM_P + t * 64 + lane_off : tS;     // P: 64 columns, over S at d = 128
        uint8_t* stage = sStage + (t * SOFTMAX_WARPS_PER_TILE + wq) * Cfg::STAGE_BYTES;   // this warp's output staging buffer
        uint32_t my_items = 0;                                  // items this tile slot took part in
        uint32_t blk = 0;                                       // blocks this tile slot has processed, all items
        uint32_t vbase = 0;                                     // ring position of the item's first V tile (PAIRED: of its pair 0)
        bool ok = true;
        // Takes entry `it` of the item ring to the warp's own copy (what is needed of it is read from there again and again rather than kept in
        // registers); its head, -1 at the end of the list, -2 when the wait ran out.
        auto take_item = [&](uint32_t it) -> int {
            if (!__all_sync(0xffffffffu, mbar_wait(&bars.item_full[it & 1], (it >> 1) & 1, abortp))) return -2;
            const int h = item_ring[it & 1].h;
            if (lane < (int)(sizeof(Item) / 4)) reinterpret_cast<int*>(&own[sw][it & 1])[lane] = reinterpret_cast<const int*>(&item_ring[it & 1])[lane];
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars.item_empty[it & 1]);
            return h;
        };
        // Output rows of this thread's two rows (rows as tokens of a tile and heads of a group), -1 for a row of the tile that is none of the sequence's.
        auto out_row = [&](const Item& w, int r) -> long long {
            const int tok = (int)fastdiv((uint32_t)r, pa.by_group), i = w.i0 + t * pa.tokens + tok;
            return tok < pa.tokens && t < pa.tiles && i < w.nq ? (long long)(w.q0 + i) * pa.heads + w.h * pa.group + (r - tok * pa.group) : -1;
        };
        uint32_t it = 0;
        int head = take_item(it++);
        while (head >= 0) {
            const Item& work = own[sw][(it - 1) & 1];
            const int nkv = t ? work.nkv1 : work.nkv0, j0 = work.j0;
            const int vfirst = vbase + (PAIRED ? 1 : 0);
            if (max(work.nkv0, work.nkv1) > 0) vbase += max(work.nkv0, work.nkv1) + (PAIRED ? 1 : 0);
            const int parts = CUT ? work.parts : 1;
            if (nkv == 0 && (parts == 1 || t >= pa.tiles || work.i0 + t * pa.tokens >= work.nq)) {         // rows without keys, or no rows
                const long long outA = out_row(work, rA), outB = out_row(work, rB);
                for (int c = 8 * (lane & 3); c < pa.d; c += 32) {
                    if (outA >= 0) *reinterpret_cast<uint4*>(pa.out + outA * pa.d + c) = make_uint4(0, 0, 0, 0);
                    if (outB >= 0) *reinterpret_cast<uint4*>(pa.out + outB * pa.d + c) = make_uint4(0, 0, 0, 0);
                }
                if (pa.lse && (lane & 3) == 0) {
                    if (outA >= 0) pa.lse[outA] = -INFINITY;
                    if (outB >= 0) pa.lse[outB] = -INFINITY;
                }
                head = take_item(it++);
                continue;
            }
            // the last keys that the rows see, and the first block that not all rows of the tile see in full
            const int i0 = work.i0 + t * pa.tokens, off = work.nk - work.nq;
            const int limA = min(i0 + (int)fastdiv((uint32_t)rA, pa.by_group) + off, work.nk - 1), limB = min(i0 + (int)fastdiv((uint32_t)rB, pa.by_group) + off, work.nk - 1);
            const int part0 = max(i0 + off + 1, 0) / TILE;
            float mA = -INFINITY, mB = -INFINITY, lA = 0.f, lB = 0.f;       // running maxima (log2 units) and row sums
            for (int j = 0; j < nkv; ++j, ++blk) {
                if (SEP) {
                    ok = mbar_wait(&bars.s_full[t], blk & 1, abortp);                 // every S has its own commit
                } else {
                    // block 0 waits for the item's first S; later blocks for the commit behind PV_{j-1} and S_j
                    if (j == 0) ok = mbar_wait(&bars.s_full[t], my_items & 1, abortp);
                    else ok = mbar_wait(&bars.o_done[t], (blk - 1) & 1, abortp);
                }
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                const bool diag = j0 + j >= part0;
                const int cbA = limA - (j0 + j) * TILE, cbB = limB - (j0 + j) * TILE;       // last kept columns
                // ---- the rows' 2 x 64 scores of this block
                uint32_t s0[32], s1[32];
                tc_fence_after();
                tmem_ld_quad64(tS, s0);
                tmem_ld_quad64(tS + 64, s1);
                tc_wait_ld();
                if (SEP) {
                    // S is in registers: the issuer may overwrite it with the next scores while the exponentials run
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars.s_free[t]);
                }
                // ---- pass 1: row maxima of the block, completed inside the quad
                float bA = -INFINITY, bB = -INFINITY;
                if (diag) {
                    mask_quad64(s0, cq, cbA, cbB);
                    mask_quad64(s1, 64 + cq, cbA, cbB);
                }
                max_quad64(s0, bA, bB);
                max_quad64(s1, bA, bB);
                bA = quad_max(bA) * pa.sl2;
                bB = quad_max(bB) * pa.sl2;
                float alphaA = 1.f, alphaB = 1.f;
                if (bA > mA + RESCALE_THRESHOLD) {   // also taken on the first block (m = -inf)
                    alphaA = ex2_mufu(mA - bA);
                    mA = bA;
                }
                if (bB > mB + RESCALE_THRESHOLD) {
                    alphaB = ex2_mufu(mB - bB);
                    mB = bB;
                }
                // ---- pass 2: P = exp2(S*sl2 - m) as bf16, keys 0-63 then keys 64-127
                float sumA = 0.f, sumB = 0.f;
                uint32_t pk[16];
                const float nmA = mA == -INFINITY ? 0.f : HEADROOM<F16> - mA, nmB = mB == -INFINITY ? 0.f : HEADROOM<F16> - mB;     // (rows that have seen no key)
                exp_quad<F16>(s0, pa.sl2, nmA, nmB, pk, sumA, sumB);
                if (SEP && blk > 0) {
                    // P and O are still in use by the PV before this one until its commit
                    ok = mbar_wait(&bars.o_done[t], (blk - 1) & 1, abortp);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    tc_fence_after();
                }
                tmem_st_quad32(tP, pk);
                exp_quad<F16>(s1, pa.sl2, nmA, nmB, pk, sumA, sumB);
                tmem_st_quad32(tP + 32, pk);
                lA = fmaf(lA, alphaA, sumA);
                lB = fmaf(lB, alphaB, sumB);
                if (j > 0 && __any_sync(0xffffffffu, alphaA != 1.f || alphaB != 1.f)) {   // rare: a row maximum grew by > 2^8
                    const int nA = __popc(__ballot_sync(0xffffffffu, (lane & 3) == 0 && alphaA != 1.f));
                    const int nB = __popc(__ballot_sync(0xffffffffu, (lane & 3) == 0 && alphaB != 1.f));
                    if (lane == 0) atomicAdd(&dc->rescales, (unsigned long long)(nA + nB));
#pragma unroll 1
                    for (int c = 0; c < D / 64; ++c) {
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
                if (diag) {
                    // the warp's share of the tile of V: what is not finite becomes zero
                    const uint32_t vc = vfirst + j;
                    ok = __all_sync(0xffffffffu, mbar_wait(&bars.v_full[vc % VST], (vc / VST) & 1, abortp));
                    if (!ok) break;
                    uint4* v = reinterpret_cast<uint4*>(sV + (vc % VST) * Cfg::TILE_BYTES) + wq * (Cfg::TILE_BYTES / 16 / SOFTMAX_WARPS_PER_TILE) + lane;
                    constexpr uint32_t EXP = F16 ? 0x7c007c00u : 0x7f807f80u, ONE = F16 ? 0x04000400u : 0x00800080u;
                    uint32_t bad = 0;
#pragma unroll
                    for (int i = 0; i < Cfg::TILE_BYTES / 16 / SOFTMAX_WARPS_PER_TILE / 32; ++i) {
                        const uint4 x = v[32 * i];
                        bad |= ((x.x & EXP) + ONE) | ((x.y & EXP) + ONE) | ((x.z & EXP) + ONE) | ((x.w & EXP) + ONE);
                    }
                    if (__any_sync(0xffffffffu, bad & 0x80008000u)) {
                        if (lane == 0) atomicMax(&v_bad, (int)it);      // (it: items taken so far, this one included)
                        __threadfence_block();
                        __syncwarp();
                        for (int i = 0; i < Cfg::TILE_BYTES / 16 / SOFTMAX_WARPS_PER_TILE / 32; ++i) {
                            uint32_t* x = reinterpret_cast<uint32_t*>(v + 32 * i);
                            for (int k = 0; k < 4; ++k) {
                                const uint32_t m = ((x[k] & EXP) + ONE) & 0x80008000u;
                                if (m) x[k] &= ~((m >> 15) * 0xffffu);
                            }
                        }
                        fence_async_smem();
                    }
                }
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars.p_ready[t]);      // (one arrival per warp: 32 on one barrier serialise)
            }
            if (!ok) break;
            // The next item is taken now, while the last PV runs, rather than after the epilogue.
            const int items_now = (int)it;
            const int head_next = take_item(it++);
            if (head_next == -2) break;
            if (nkv > 0) {
                ok = mbar_wait(&bars.o_done[t], (blk - 1) & 1, abortp);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
            }
            // ---- epilogue: O / l, 32 columns at a time through the warp's staging buffer (chunks of 16 bytes swizzled) to whole sectors of the rows
            tc_fence_after();
            lA = quad_sum(lA);
            lB = quad_sum(lB);
            const bool bad = nkv > 0 && *reinterpret_cast<volatile int*>(&v_bad) >= items_now;
            // 64 columns of O, with values that are not finite put back: they were left out of the blocks from the item's first partial one on
            auto load_o = [&](int u, uint32_t (&v)[32]) {
                tmem_ld_quad64(tO + 64 * u, v);
                tc_wait_ld();
                if (bad) {
                    const int first = max(max(work.i0 + off + 1, 0) / TILE, j0) * TILE, last = min(max(limA, limB), (j0 + nkv) * TILE - 1);
                    for (int k = first; k <= last; ++k) {
                        const uint16_t* row = pa.v + (size_t)(work.k0 + k) * pa.v_stride + work.h * pa.d;
#pragma unroll
                        for (int g = 0; g < 8; ++g) {
                            const int c = 64 * u + 8 * g + cq;
                            if (c >= pa.d) continue;
                            const float2 x = F16 ? __half22float2(*reinterpret_cast<const __half2*>(row + c)) : __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(row + c));
                            const float ax = isfinite(x.x) ? 0.f : x.x, ay = isfinite(x.y) ? 0.f : x.y;
                            if (k <= limA) { v[4 * g] = __float_as_uint(__uint_as_float(v[4 * g]) + ax); v[4 * g + 1] = __float_as_uint(__uint_as_float(v[4 * g + 1]) + ay); }
                            if (k <= limB) { v[4 * g + 2] = __float_as_uint(__uint_as_float(v[4 * g + 2]) + ax); v[4 * g + 3] = __float_as_uint(__uint_as_float(v[4 * g + 3]) + ay); }
                        }
                    }
                }
            };
            bool mine = true;                                   // whether this warp stores the rows' outputs
            // A part's sums as the warp holds them: [SUB][8][32 lanes] of four, lane by lane next to each other.
            auto part_sums = [&](int p, int u) { return reinterpret_cast<float4*>(pa.part) + ((((size_t)(work.slot + p) * 2 + t) * SOFTMAX_WARPS_PER_TILE + wq) * Cfg::SUB + u) * 256 + lane; };
            float2* const ml = reinterpret_cast<float2*>(pa.part + (size_t)2 * MAX_CTAS * 2 * TILE * D);
            auto part_row = [&](int p, int r) { return (size_t)((work.slot + p) * 2 + t) * TILE + r; };
            if (parts > 1) {
                if (nkv > 0) {
#pragma unroll
                    for (int u = 0; u < Cfg::SUB; ++u) {
                        uint32_t v[32];
                        load_o(u, v);
                        float4* to = part_sums(work.part, u);
#pragma unroll
                        for (int g = 0; g < 8; ++g)
                            __stcg(to + 32 * g, make_float4(__uint_as_float(v[4 * g]), __uint_as_float(v[4 * g + 1]), __uint_as_float(v[4 * g + 2]), __uint_as_float(v[4 * g + 3])));
                    }
                }
                if ((lane & 3) == 0) {
                    __stcg(ml + part_row(work.part, rA), make_float2(mA, lA));
                    __stcg(ml + part_row(work.part, rB), make_float2(mB, lB));
                }
                mine = warp_arrive(&g_prompt_arrived[work.slot][t][wq], (unsigned)(parts - 1), lane);
                if (mine) {                                     // the rows' maxima and sums over all parts
                    float topA = -INFINITY, topB = -INFINITY, sumA = 0.f, sumB = 0.f;
#pragma unroll 4
                    for (int p = 0; p < parts; ++p) {
                        topA = fmaxf(topA, __ldcg(ml + part_row(p, rA)).x);
                        topB = fmaxf(topB, __ldcg(ml + part_row(p, rB)).x);
                    }
#pragma unroll 4
                    for (int p = 0; p < parts; ++p) {
                        const float2 a = __ldcg(ml + part_row(p, rA)), bb = __ldcg(ml + part_row(p, rB));
                        if (a.y != 0.f) sumA += a.y * ex2_mufu(a.x - (topA == -INFINITY ? 0.f : topA));
                        if (bb.y != 0.f) sumB += bb.y * ex2_mufu(bb.x - (topB == -INFINITY ? 0.f : topB));
                    }
                    mA = topA; mB = topB; lA = sumA; lB = sumB;
                }
            }
            if (mine) {
                const long long outA = out_row(work, rA), outB = out_row(work, rB);
                const float invA = lA == 0.f ? 0.f : 1.f / lA, invB = lB == 0.f ? 0.f : 1.f / lB;
                if (pa.lse && (lane & 3) == 0) {
                    if (outA >= 0) pa.lse[outA] = lA == 0.f ? -INFINITY : (mA - HEADROOM<F16> + log2f(lA)) * LN2;
                    if (outB >= 0) pa.lse[outB] = lB == 0.f ? -INFINITY : (mB - HEADROOM<F16> + log2f(lB)) * LN2;
                }
#pragma unroll
                for (int u = 0; u < Cfg::SUB; ++u) {
                    uint32_t v[32];
                    if (parts == 1) {
                        load_o(u, v);
                    } else {
#pragma unroll
                        for (int g = 0; g < 32; ++g) v[g] = 0u;
                        for (int p = 0; p < parts; ++p) {
                            const float2 ma = __ldcg(ml + part_row(p, rA)), mb = __ldcg(ml + part_row(p, rB));
                            // (a part without keys for the row has no sums; its place holds anything)
                            const float fA = ma.y == 0.f ? 0.f : ex2_mufu(ma.x - (mA == -INFINITY ? 0.f : mA)), fB = mb.y == 0.f ? 0.f : ex2_mufu(mb.x - (mB == -INFINITY ? 0.f : mB));
                            const float4* from = part_sums(p, u);
#pragma unroll
                            for (int g = 0; g < 8; ++g) {
                                const float4 x = __ldcg(from + 32 * g);
                                if (fA != 0.f) { v[4 * g] = __float_as_uint(fmaf(fA, x.x, __uint_as_float(v[4 * g]))); v[4 * g + 1] = __float_as_uint(fmaf(fA, x.y, __uint_as_float(v[4 * g + 1]))); }
                                if (fB != 0.f) { v[4 * g + 2] = __float_as_uint(fmaf(fB, x.z, __uint_as_float(v[4 * g + 2]))); v[4 * g + 3] = __float_as_uint(fmaf(fB, x.w, __uint_as_float(v[4 * g + 3]))); }
                            }
                        }
                    }
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int r = lane >> 2;
#pragma unroll
                        for (int c = 0; c < 4; ++c) {           // chunk c of the rows' 64 bytes: columns 8 (4 half + c) + cq, + 1
                            const int e = 4 * (4 * half + c);
                            const uint32_t a = pack<F16>(__uint_as_float(v[e]) * invA, __uint_as_float(v[e + 1]) * invA);
                            const uint32_t bb = pack<F16>(__uint_as_float(v[e + 2]) * invB, __uint_as_float(v[e + 3]) * invB);
                            const int at = r * 64 + ((c ^ (r >> 1)) & 3) * 16 + 2 * cq;
                            *reinterpret_cast<uint32_t*>(stage + at) = a;
                            *reinterpret_cast<uint32_t*>(stage + at + 512) = bb;
                        }
                        __syncwarp();
                        const int at = r * 64 + (((lane & 3) ^ (r >> 1)) & 3) * 16, col = 64 * u + 32 * half + 8 * (lane & 3);
                        if (col < pa.d) {
                            if (outA >= 0) *reinterpret_cast<uint4*>(pa.out + outA * pa.d + col) = *reinterpret_cast<const uint4*>(stage + at);
                            if (outB >= 0) *reinterpret_cast<uint4*>(pa.out + outB * pa.d + col) = *reinterpret_cast<const uint4*>(stage + at + 512);
                        }
                        __syncwarp();
                    }
                }
            }
            // (the next write to O_t, PV_0 of the tile's next item, waits for P of that item, which every
            // thread of the tile signals only after these reads)
            tc_fence_before();
            if (nkv > 0) ++my_items;
            head = head_next;
        }
        if (sw == 0 && lane == 0) grid_launch_dependents();
    }
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && abort_flag) {
        atomicExch(&dc->status, (int)PSA_ERR_TIMEOUT);
        if (cuts) atomicExch(&g_prompt_left, EXPIRED);
    }
    if (warp == 1) tmem_dealloc(tmem, 512);
}

// Row tiles of queries: boxes of `tokens` rows x all heads of a group x 64 columns.
bool query_map(CUtensorMap* m, const void* Q, int rows, int kv_heads, int group, int d, long long stride, int tokens) {
    const uint64_t dims[4] = {(uint64_t)d, (uint64_t)group, (uint64_t)kv_heads, (uint64_t)rows}, strides[3] = {(uint64_t)d * 2, (uint64_t)group * d * 2, (uint64_t)stride * 2};
    const uint32_t box[4] = {64, (uint32_t)group, 1, (uint32_t)tokens};
    return make_tensor_map_16bit(m, Q, 4, dims, strides, box);
}
bool key_map(CUtensorMap* m, const void* K, int rows, int kv_heads, int d, long long stride) {
    const uint64_t dims[3] = {(uint64_t)d, (uint64_t)kv_heads, (uint64_t)rows}, strides[2] = {(uint64_t)d * 2, (uint64_t)stride * 2};
    const uint32_t box[3] = {64, 1, TILE};
    return make_tensor_map_16bit(m, K, 3, dims, strides, box);
}

template <int D, int KS, bool F16, bool CUT>
int launch_prompt(const PMaps& maps, const PromptArgs& all, DeviceCounters* dc, unsigned int* cursor, DeviceCounters* dc_next, cudaStream_t stream) {
    using Cfg = PCfg<D>;
    static DeviceSetup setup;
    const int sm_count = device_setup(&setup, [] {
        return cudaFuncSetAttribute(prompt_kernel<D, KS, F16, CUT>, cudaFuncAttributeMaxDynamicSharedMemorySize, PCfg<D>::SMEM);
    }, "prompt kernel set-up");
    if (sm_count <= 0) return PSA_ERR_CUDA;
    for (int s0 = 0; s0 < all.sequences; s0 += SEQS) {
        PromptArgs pa = all;
        pa.sequences = all.sequences - s0 < SEQS ? all.sequences - s0 : SEQS;
        pa.q_starts += s0;
        pa.k_starts += s0;
        // (an upper bound: the lengths are known on the device only)
        // Two tiles a CTA keep the tensor pipe busier (3560 cycles a pair of key blocks of d = 128), one alone is done sooner: each has a CTA of its own where there are CTAs
        // enough and little to do for each, by what the host knows (that is, sequences of one length).  (us, two and one, 32 heads on 8 of d = 128: 256 tokens 14.2 12.1,
        // 512 18.2 15.9, 512 behind 500 26.8 23.9, 128 behind 4000 39.6 34.5, 64 behind 8000 50.9 41.4, with 7 blocks a CTA; 512 behind 1000 33.4 32.6, behind 2000
        // 40.9 46.8, 256 behind 4000 41.5 46.9, with 10, 17 and 14.)
        const int ctas = sm_count < MAX_CTAS ? sm_count : MAX_CTAS;
        const long long blocks = (long long)pa.q_rows * pa.kv_heads / pa.tokens * ((pa.k_rows / pa.sequences + TILE - 1) / TILE);
        pa.tiles = ((long long)pa.q_rows / pa.tokens + pa.sequences) * pa.kv_heads <= ctas && blocks <= 8 * ctas ? 1 : 2;
        long long items = ((long long)pa.q_rows / (pa.tiles * pa.tokens) + pa.sequences) * pa.kv_heads;
        if (CUT) items *= ((long long)pa.k_rows + TILE * LEAST_PIECE - 1) / (TILE * LEAST_PIECE);
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(items < ctas ? items : ctas));
        cfg.blockDim = dim3(persist_threads<D>());
        cfg.dynamicSmemBytes = Cfg::SMEM;
        cfg.stream = stream;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;     // the kernel waits for its predecessor itself
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        // (the counter serves the first launch; the items of further ones go round in turn)
        const cudaError_t e = cudaLaunchKernelEx(&cfg, prompt_kernel<D, KS, F16, CUT>, maps, pa, dc, s0 == 0 ? cursor : nullptr, s0 == 0 ? dc_next : nullptr);
        if (e != cudaSuccess) { set_cuda_error(e, "prompt_kernel launch"); return PSA_ERR_CUDA; }
    }
    return PSA_OK;
}

}  // namespace

// Whether a call may have fewer pairs of row tiles than CTAs, with enough key blocks to be cut; and what that needs: a result in fp32 per part.
size_t prompt_scratch_bytes(int sequences, int q_rows, int k_rows, int heads, int kv_heads, int d) {
    const int group = heads / kv_heads, tokens = TILE / group;
    if ((long long)q_rows / (2 * tokens) * kv_heads >= MAX_CTAS || k_rows <= 2 * LEAST_PIECE * TILE || sequences > SEQS) return 0;
    return (size_t)2 * MAX_CTAS * 2 * TILE * ((d <= 64 ? 64 : 128) + 2) * sizeof(float);
}
// For the self-test of the failure path: what a call that had cut its pairs when its waits ran out leaves behind.
static __global__ void prompt_expired_kernel() {
    for (int i = threadIdx.x; i < (int)(sizeof(g_prompt_arrived) / sizeof(unsigned)); i += blockDim.x) (&g_prompt_arrived[0][0][0])[i] = 1u;
    if (threadIdx.x == 0) atomicExch(&g_prompt_left, EXPIRED);
}
cudaError_t launch_prompt_expired(cudaStream_t stream) {
    prompt_expired_kernel<<<1, 256, 0, stream>>>();
    return cudaGetLastError();
}

int prompt_attention(const void* Q, const void* K, const void* V, long long q_stride, long long k_stride, long long v_stride, const int* q_starts, const int* k_starts,
                     int sequences, int q_rows, int k_rows, int heads, int kv_heads, int d, float scale, int dtype, void* out, float* lse, void* scratch, int call, DeviceCounters* dc,
                     unsigned int* cursor, DeviceCounters* dc_next, cudaStream_t stream) {
    const int group = heads / kv_heads, tokens = TILE / group;
    if ((long long)q_rows / (2 * tokens) >= 1LL << (32 - SEQ_BITS) || ((long long)q_rows / (2 * tokens) + SEQS) * kv_heads > 0x7fff0000LL) return PSA_ERR_SHAPE;
    PMaps maps;
    if (!query_map(&maps.q, Q, q_rows, kv_heads, group, d, q_stride, tokens)) return PSA_ERR_CUDA;
    maps.k = maps.v = maps.q;                    // (without keys no block of them is ever loaded)
    if (k_rows > 0 && (!key_map(&maps.k, K, k_rows, kv_heads, d, k_stride) || !key_map(&maps.v, V, k_rows, kv_heads, d, v_stride))) return PSA_ERR_CUDA;
    const PromptArgs pa = {q_starts, k_starts, sequences, q_rows, k_rows, heads, kv_heads, group, tokens, d, 2, call, v_stride, static_cast<const uint16_t*>(V),
                           static_cast<uint16_t*>(out), lse, static_cast<float*>(scratch), scale * LOG2E, fastdiv_make((uint32_t)group), fastdiv_make((uint32_t)kv_heads)};
    auto launch = [&](auto width, auto steps) {
        constexpr int D = decltype(width)::value, KS = decltype(steps)::value;
        if (scratch) return dtype == PSA_F16 ? launch_prompt<D, KS, true, true>(maps, pa, dc, cursor, dc_next, stream) : launch_prompt<D, KS, false, true>(maps, pa, dc, cursor, dc_next, stream);
        return dtype == PSA_F16 ? launch_prompt<D, KS, true, false>(maps, pa, dc, cursor, dc_next, stream) : launch_prompt<D, KS, false, false>(maps, pa, dc, cursor, dc_next, stream);
    };
    using std::integral_constant;
    const integral_constant<int, 64> narrow;
    const integral_constant<int, 128> wide;
    // (column steps as in bf16_attention_persist, which gives the measurements)
    switch ((d + 15) / 16) {
        case 1: case 2: return launch(narrow, integral_constant<int, 2>{});
        case 3: case 4: return launch(narrow, integral_constant<int, 4>{});
        case 5: return launch(wide, integral_constant<int, 5>{});
        case 6: return launch(wide, integral_constant<int, 6>{});
        default: return launch(wide, integral_constant<int, 8>{});
    }
}

}  // namespace psa
