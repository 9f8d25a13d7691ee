// Appending keys and values to the cache held in 4 bits (layout: psa_cache.cuh).
//
// Per token, head and group of 32 channels, lo and hi being the group's least and greatest number:
//     S = fp16(16 (hi - lo) / 15),   M = fp16(lo - S),   c = rint((x - M - S) 16 / S) in 0 .. 15,
// so that c = 0 stands for lo and c = 15 for hi up to the roundings of S and M; the codes are taken against the rounded numbers, and the error of
// a number is half a step, (hi - lo) / 30.  All in fp32, every operation rounded by itself (no contraction), so that the result is one of definition.
//
// To read and write: 2 bytes and 5 bits per number, 2 bytes more when the held values are asked for.  A warp takes the two tokens of a pair (they share
// the words of V's codes and scales), K and V, eight lanes a group (four channels each, one load of 8 bytes), for one head after another, the loads of the next
// head ahead of the work on this one.  Where there are few tokens a warp has one head.  What it spends its time on is instructions (the first form had 50 a number, this
// one 29, and 68 % of the issue slots; the rest are waits for their results): least and greatest numbers are found in the inputs' own 16 bits, two at a time, the greatest as the least of the negated ones in the other half of the
// same register; the numbers of a group are worked out once, a group per lane, and handed round; and a code is the low end of y + 1.5 2^23.
// Measured: 16 prompts of up to 2500 tokens, 8 heads of 128 (14 million numbers) with held values 18.1 us, 3.7 TB/s; the first form 30.7.
//
// With rotation (ROT): a pair of channels (a, b) of a key becomes A (a cos - b sin, b cos + a sin), the angle being the token's position times the pair's frequency, and
// is rounded to the inputs' type, so that the cache holds the same bytes as if a turned tensor had been appended.  Angles are kept as fractions of a turn in 64 bits: a
// frequency becomes one once, and the product with the position wraps by itself where whole turns drop out, so that position 2^31 costs no accuracy and no division; sine and
// cosine of what is left are good to 2^-23.  They are worked out once a token and channel for all heads that a warp takes.  The queries are turned by further blocks of the
// same launch: a thread has four pairs of channels of one token, for one head after another.
// Measured: 16 packed prompts of up to 2500 tokens, 32 heads on 8 of 128, half of each turning, with held values (123 MB) 29.9 us, 4.1 TB/s; 64 trees of up to 16 tokens 6.3 us;
// one token 4.5.
#include <algorithm>
#include <type_traits>

#include "psa_cache.cuh"
#include "psa_internal.h"
#include "psa_sched.h"
#include "sm100.cuh"

namespace psa {

namespace {

constexpr int APPEND_WARPS = 8;
constexpr int ROT_CTAS = 3;                     // an SM, with rotation: 80 registers a thread.  (With two, three, four: 16 packed prompts of up to 2500 tokens, 32 heads on 8 of 128, 35.4, 29.6, 32.3 us with a frequency's fraction in one double)

struct AppendArgs {
    uint8_t* pool;
    const int *tables, *lens, *seqs, *starts;
    const uint16_t *k, *v;
    uint16_t *k_held, *v_held;
    long long k_stride, v_stride;
    int pages, slots, width, page_size, kv_heads, sequences, rows;
    int heads_per_warp, units;                  // units: pairs of tokens, see unit_of
    FastDiv by_chunks, by_page;                 // by warps per unit, by tokens of a page
};
// What turns, and the queries (q null: none).
struct RotaryArgs {
    const double* freqs;
    const int* depths;
    float amplitude;
    int rot, interleaved;
    const uint16_t* q;
    uint16_t* q_out;
    long long q_stride;
    int heads, key_blocks;                      // blocks below key_blocks append, those from there on turn queries
    FastDiv by_slots, by_groups;                // by threads of a head (eight channels each), by groups of heads of a row
};

// Position times frequency, as sine and cosine.  freq / 2 pi is formed in two doubles (in one a frequency of 50 was off by 2^-17 of an angle at position 2^31) and rounded to 2^-63 of a turn, what is left of
// the product to 2^-25 of half a turn.
__device__ __forceinline__ long long turns_of(double freq) {
    constexpr double HIGH = 0.15915494309189535, LOW = -9.839338337591243e-18, ONE = 18446744073709551616.0;      // 1 / 2 pi in two parts; a turn
    const double t = freq * HIGH, rest = fma(freq, LOW, fma(freq, HIGH, -t));
    return (long long)((unsigned long long)__double2ll_rn((t - rint(t)) * ONE) + (unsigned long long)__double2ll_rn((rest - rint(rest)) * ONE));
}
__device__ __forceinline__ void sin_cos(long long turns, long long position, float& s, float& c) {
    const unsigned long long at = (unsigned long long)turns * (unsigned long long)position;
    sincospif((float)(int)(at >> 32) * 4.656612873077392578125e-10f, &s, &c);
}

// Units are pairs of neighbouring tokens, the first at an even position.  Sequence b has those from starts[b] / 2 + b on (one more than it can need
// where its tokens begin at an even position, so that the numbers follow from `starts` alone).  The sequence of unit u: the last b with starts[b] / 2 + b <= u,
// 32 numbers at a time, so that a batch of up to 1024 takes two loads.
__device__ __forceinline__ int unit_of(const AppendArgs& a, int u, int lane) {
    int lo = 0, n = a.sequences;               // the answer lies in lo .. lo + n - 1
    while (n > 1) {
        const int step = (n + 31) / 32, at = lo + lane * step;
        const bool le = lane * step < n && max(a.starts[at], 0) / 2 + at <= u;
        const uint32_t m = __ballot_sync(0xffffffffu, le);
        const int k = m ? 31 - __clz(m) : 0;
        lo += k * step;
        n = min(step, n - k * step);
    }
    return lo;
}

// The smaller of two pairs of numbers of the input's type; a NaN stays one.
template <bool F16>
__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {
    uint32_t r;
    if constexpr (F16) asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
template <bool F16>
__device__ __forceinline__ float low_of(uint32_t x) {
    if constexpr (F16) return __half2float(__ushort_as_half((uint16_t)x));
    else return __uint_as_float(x << 16);
}
template <bool F16>
__device__ __forceinline__ float high_of(uint32_t x) {
    if constexpr (F16) return __half2float(__ushort_as_half((uint16_t)(x >> 16)));
    else return __uint_as_float(x & 0xffff0000u);
}

template <bool F16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    if constexpr (F16) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    } else {
        return pack_bf16x2(lo, hi);
    }
}

// The queries' part: thread = (row, group of heads, slot of eight channels).  A slot that turns has channels 4 s .. and their partners half a part further on, or
// eight neighbours (interleaved); one that does not copies eight neighbours.
template <int D, bool F16>
__device__ __forceinline__ void turn_queries(const AppendArgs& a, const RotaryArgs& ro) {
    const uint32_t id = (blockIdx.x - ro.key_blocks) * (32 * APPEND_WARPS) + threadIdx.x;
    const uint32_t rest = fastdiv(id, ro.by_slots), row_of = fastdiv(rest, ro.by_groups);
    const int slot = (int)(id - rest * ro.by_slots.d), h0 = (int)(rest - row_of * ro.by_groups.d);
    // the last sequence that begins at or before the row: for the warp's first row together, from there on by each thread
    const int r = (int)min(row_of, (uint32_t)a.rows - 1), r0 = __shfl_sync(0xffffffffu, r, 0);
    int lo = 0;
    for (int n = a.sequences; n > 1;) {
        const int step = (n + 31) / 32, lane = threadIdx.x & 31;
        const uint32_t m = __ballot_sync(0xffffffffu, lane * step < n && a.starts[lo + min(lane * step, n - 1)] <= r0);
        const int k = m ? 31 - __clz(m) : 0;
        lo += k * step;
        n = min(step, n - k * step);
    }
    if (row_of >= (uint32_t)a.rows) return;
    while (lo + 1 < a.sequences && a.starts[lo + 1] <= r) ++lo;
    const bool turns = 8 * slot < ro.rot;
    long long f[4] = {0, 0, 0, 0};
    if (turns)
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = turns_of(ro.freqs[4 * slot + e]);
    const int first = max(a.starts[lo], 0), end = min(max(a.starts[lo + 1], 0), a.rows), seq = a.seqs[lo];
    if (r < first || r >= end || seq < 0 || seq >= a.slots) return;
    const long long position = (long long)a.lens[seq] - (end - first) + (ro.depths ? ro.depths[r] : r - first);
    float s[4], c[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        s[e] = 0.f;
        c[e] = 1.f;
        if (turns) {
            sin_cos(f[e], position, s[e], c[e]);
            s[e] *= ro.amplitude;
            c[e] *= ro.amplitude;
        }
    }
    const bool halves = turns && !ro.interleaved;
    const int ca = halves ? 4 * slot : 8 * slot, cb = halves ? ca + ro.rot / 2 : ca + 4;
    const uint16_t* from = ro.q + (size_t)r * ro.q_stride;
    uint16_t* to = ro.q_out + (size_t)r * ro.heads * D;
    const int step = (int)ro.by_groups.d;
    constexpr int AHEAD = 4;
    for (int h = h0; h < ro.heads; h += AHEAD * step) {
        uint2 xa[AHEAD], xb[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (h + k * step < ro.heads) {
                xa[k] = *reinterpret_cast<const uint2*>(from + (size_t)(h + k * step) * D + ca);
                xb[k] = *reinterpret_cast<const uint2*>(from + (size_t)(h + k * step) * D + cb);
            }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (h + k * step < ro.heads) {
                if (turns) {
                    const float x[8] = {low_of<F16>(xa[k].x), high_of<F16>(xa[k].x), low_of<F16>(xa[k].y), high_of<F16>(xa[k].y),
                                        low_of<F16>(xb[k].x), high_of<F16>(xb[k].x), low_of<F16>(xb[k].y), high_of<F16>(xb[k].y)};
                    float y[8];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float u = ro.interleaved ? x[2 * e] : x[e], v = ro.interleaved ? x[2 * e + 1] : x[e + 4];
                        const float p = fmaf(u, c[e], -v * s[e]), w = fmaf(v, c[e], u * s[e]);
                        if (ro.interleaved) { y[2 * e] = p; y[2 * e + 1] = w; }
                        else { y[e] = p; y[e + 4] = w; }
                    }
                    xa[k] = make_uint2(pack2<F16>(y[0], y[1]), pack2<F16>(y[2], y[3]));
                    xb[k] = make_uint2(pack2<F16>(y[4], y[5]), pack2<F16>(y[6], y[7]));
                }
                *reinterpret_cast<uint2*>(to + (size_t)(h + k * step) * D + ca) = xa[k];
                *reinterpret_cast<uint2*>(to + (size_t)(h + k * step) * D + cb) = xb[k];
            }
    }
}

template <int D, bool F16, bool ROT>
__global__ void __launch_bounds__(32 * APPEND_WARPS, ROT ? (D <= 128 ? ROT_CTAS : 1) : 0) cache_append_kernel(const AppendArgs a, const RotaryArgs ro, DeviceCounters* dc, DeviceCounters* dc_next) {
    constexpr int G = D / 32;
    constexpr bool SAME_LANE = G % 4 == 0;      // both tokens' codes come to the same lane, G / 4 rounds apart: whole words of V
    using B = CacheBlock<D>;
    grid_dependency_wait();
    if (threadIdx.x == 0 && blockIdx.x == 0 && dc_next) *dc_next = DeviceCounters{0, 0, 0, 0, 0, 0, 0};
    if constexpr (ROT)
        if ((int)blockIdx.x >= ro.key_blocks) return turn_queries<D, F16>(a, ro);
    const int lane = threadIdx.x & 31;
    const uint32_t id = blockIdx.x * APPEND_WARPS + (threadIdx.x >> 5);
    const int unit = (int)fastdiv(id, a.by_chunks);
    if (unit >= a.units) return;
    const int h0 = (int)(id - (uint32_t)unit * a.by_chunks.d) * a.heads_per_warp, h1 = min(h0 + a.heads_per_warp, a.kv_heads);
    // ---- where the pair goes: rows r, r + 1 of the call are tokens pos, pos + 1 of the sequence, as far as they are new
    const int b = unit_of(a, unit, lane);
    const int first = max(a.starts[b], 0), end = min(max(a.starts[b + 1], 0), a.rows), seq = a.seqs[b];
    if (first >= end) return;
    const bool known = seq >= 0 && seq < a.slots;
    const int pos0 = (known ? a.lens[seq] : 0) - (end - first), pos = (pos0 & ~1) + 2 * (unit - (first / 2 + b)), r = first + (pos - pos0);
    const bool has0 = r >= first && r < end, has1 = r + 1 >= first && r + 1 < end;
    if (!has0 && !has1) return;
    uint8_t* dst = nullptr;
    const int col = (int)fastdiv((uint32_t)max(pos, 0), a.by_page), in = pos - col * a.page_size;
    if (known && pos0 >= 0 && col < a.width) {
        const int page = a.tables[(size_t)seq * a.width + col];
        if (page >= 0 && page < a.pages) dst = a.pool + ((size_t)page * a.kv_heads * (a.page_size / CACHE_BLOCK) + in / CACHE_BLOCK) * B::BYTES;
    }
    if (!dst && lane == 0) atomicExch(&dc->status, (int)PSA_ERR_SHAPE);       // (device-side arguments that name no place: reported, nothing written)
    const size_t head_bytes = (size_t)(a.page_size / CACHE_BLOCK) * B::BYTES;
    const int t16 = in % CACHE_BLOCK;           // of the first token: even
    // ---- subgroup of eight lanes = one (K or V, token of the pair, group); q = lane inside it, channels 4q .. 4q+3 of the group.  Where each round of a
    // lane reads and writes, from head to head by a constant step.
    const int q = lane & 7;
    auto kv_of = [&](int it) { return SAME_LANE ? it / max(G / 2, 1) : (it * 4 + (lane >> 3)) / (2 * G); };
    auto parity_of = [&](int it) { return SAME_LANE ? it / max(G / 4, 1) % 2 : (it * 4 + (lane >> 3)) / G % 2; };
    const uint16_t* src[G];
    uint16_t* back[G];
    int codes_at[G], scales_at[G];
    const bool holds = a.k_held || a.v_held;
#pragma unroll
    for (int it = 0; it < G; ++it) {
        const int w = (it * 4 + (lane >> 3)) % G, tok = t16 + parity_of(it), channel = h0 * D + 32 * w + 4 * q;
        const long long row = r + parity_of(it);
        src[it] = (kv_of(it) ? a.v + row * a.v_stride : a.k + row * a.k_stride) + channel;
        uint16_t* const held = kv_of(it) ? a.v_held : a.k_held;
        back[it] = held ? held + row * a.kv_heads * D + channel : nullptr;
        codes_at[it] = kv_of(it) ? B::V_CODES + (t16 >> 1) * D + (q * G + w) * 4 : B::K_CODES + tok * (D / 2) + ((q >> 1) * G + w) * 4;
        scales_at[it] = kv_of(it) ? B::V_SCALES + ((t16 >> 1) * G + w) * 8 + q * 4 : B::K_SCALES + (tok * G + w) * 4;
    }
    // ---- rotation: of the lane's four channels in each round of keys, cosines and signed sines; `other`: from the channels to their partners
    constexpr int KR = ROT ? (G + 1) / 2 : 0;    // rounds that have keys
    [[maybe_unused]] float cs[KR + 1][4], sn[KR + 1][4];
    [[maybe_unused]] int other[KR + 1];          // (0: the partners are among the four, or nothing turns)
    [[maybe_unused]] uint2 partner[KR + 1], partner_ahead[KR + 1];
    if constexpr (ROT) {
#pragma unroll
        for (int it = 0; it < KR; ++it) {
            const int c0 = 32 * ((it * 4 + (lane >> 3)) % G) + 4 * q, half = ro.rot / 2, row = r + parity_of(it);
            const bool turns = kv_of(it) == 0 && c0 < ro.rot && (parity_of(it) ? has1 : has0), upper = c0 >= half;
            other[it] = turns && !ro.interleaved ? (upper ? -half : half) : 0;
#pragma unroll
            for (int c = 0; c < 4; ++c) { cs[it][c] = 1.f; sn[it][c] = 0.f; }
            if (turns) {
                const long long position = ro.depths ? (long long)pos0 + ro.depths[row] : (long long)pos + parity_of(it);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    if (ro.interleaved && (c & 1)) {
                        cs[it][c] = cs[it][c - 1];
                        sn[it][c] = -sn[it][c - 1];
                        continue;
                    }
                    float s, co;
                    sin_cos(turns_of(ro.freqs[ro.interleaved ? (c0 + c) / 2 : c0 + c - (upper ? half : 0)]), position, s, co);
                    cs[it][c] = co * ro.amplitude;
                    sn[it][c] = (ro.interleaved || !upper ? -s : s) * ro.amplitude;
                }
            }
        }
    }
    uint2 x[G], ahead[G];
    auto load = [&] {                            // (of the next head)
        if constexpr (ROT) {
#pragma unroll
            for (int it = 0; it < KR; ++it) {
                partner_ahead[it] = make_uint2(0, 0);
                if (other[it]) partner_ahead[it] = *reinterpret_cast<const uint2*>(src[it] + other[it]);
            }
        }
#pragma unroll
        for (int it = 0; it < G; ++it) {
            ahead[it] = make_uint2(0, 0);
            if (parity_of(it) ? has1 : has0) ahead[it] = *reinterpret_cast<const uint2*>(src[it]);
            src[it] += D;
        }
    };
    load();
    uint8_t* to = dst ? dst + (size_t)h0 * head_bytes : nullptr;
    for (int h = h0; h < h1; ++h) {
#pragma unroll
        for (int it = 0; it < G; ++it) x[it] = ahead[it];
        if constexpr (ROT) {
#pragma unroll
            for (int it = 0; it < KR; ++it) partner[it] = partner_ahead[it];
        }
        if (h + 1 < h1) load();
        if constexpr (ROT) {
#pragma unroll
            for (int it = 0; it < KR; ++it) {
                const int c0 = 32 * ((it * 4 + (lane >> 3)) % G) + 4 * q;
                if (kv_of(it) != 0 || c0 >= ro.rot) continue;
                const float u[4] = {low_of<F16>(x[it].x), high_of<F16>(x[it].x), low_of<F16>(x[it].y), high_of<F16>(x[it].y)};
                const float v[4] = {low_of<F16>(partner[it].x), high_of<F16>(partner[it].x), low_of<F16>(partner[it].y), high_of<F16>(partner[it].y)};
                float y[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) y[c] = fmaf(u[c], cs[it][c], (ro.interleaved ? u[c ^ 1] : v[c]) * sn[it][c]);
                x[it] = make_uint2(pack2<F16>(y[0], y[1]), pack2<F16>(y[2], y[3]));
            }
        }
        // ---- least and (negated) greatest number of every group; lane l then has those of group l of the 4 G that the warp works on
        uint32_t mine = 0;
#pragma unroll
        for (int it = 0; it < G; ++it) {
            const uint32_t low = min2<F16>(x[it].x, x[it].y), high = min2<F16>(x[it].x ^ 0x80008000u, x[it].y ^ 0x80008000u);
            uint32_t m = min2<F16>(__byte_perm(low, high, 0x5410), __byte_perm(low, high, 0x7632));
#pragma unroll
            for (int s = 1; s < 8; s *= 2) m = min2<F16>(m, __shfl_xor_sync(0xffffffffu, m, s));
            const uint32_t of = __shfl_sync(0xffffffffu, m, (lane & 3) * 8);
            if ((lane >> 2) == it) mine = of;
        }
        float lo = low_of<F16>(mine), hi = -high_of<F16>(mine);
        const bool wide = __any_sync(0xffffffffu, lo < -CACHE_MAX || hi > CACHE_MAX);
        lo = lo < -CACHE_MAX ? -CACHE_MAX : lo > CACHE_MAX ? CACHE_MAX : lo;             // (a NaN stays one, and makes S and M such)
        hi = hi < -CACHE_MAX ? -CACHE_MAX : hi > CACHE_MAX ? CACHE_MAX : hi;
        const __half S = __float2half_rn(__fmul_rn(__fsub_rn(hi, lo), 16.f / 15.f));
        const __half M = __float2half_rn(__fsub_rn(lo, __half2float(S)));
        const uint32_t scales_of_mine = (uint32_t)__half_as_ushort(S) | (uint32_t)__half_as_ushort(M) << 16;
        const float step_of_mine = __half2float(S) > 0.f ? 16.f * __frcp_rn(__half2float(S)) : 0.f, base_of_mine = __fadd_rn(__half2float(M), __half2float(S));
        // ---- codes; `all`: both tokens are new, have a place, and no number lies beyond the grid, which is checked once instead of at every store
        auto write = [&](auto all) {
            constexpr bool WHOLE = decltype(all)::value;
            [[maybe_unused]] uint32_t v_low[G];  // codes of V of the pair's first token, and its scales, where the second one's follow in the same lane
            [[maybe_unused]] uint16_t s_low[G];
#pragma unroll
            for (int it = 0; it < G; ++it) {
                const int kv = kv_of(it), parity = parity_of(it);
                const int owner = it * 4 + (lane >> 3);
                const uint32_t sm = __shfl_sync(0xffffffffu, scales_of_mine, owner);
                const float step = __shfl_sync(0xffffffffu, step_of_mine, owner), base = __shfl_sync(0xffffffffu, base_of_mine, owner);
                float f[4] = {low_of<F16>(x[it].x), high_of<F16>(x[it].x), low_of<F16>(x[it].y), high_of<F16>(x[it].y)};
                if (!WHOLE && wide) {                // (rare: numbers beyond the grid)
#pragma unroll
                    for (int c = 0; c < 4; ++c) f[c] = fminf(fmaxf(f[c], -CACHE_MAX), CACHE_MAX);
                }
                uint32_t code[4];                    // + 0x4b400000
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float y = fminf(fmaxf(__fmul_rn(__fsub_rn(f[c], base), step), 0.f), 15.f);      // (a NaN: 0)
                    f[c] = __fadd_rn(y, 12582912.f);
                    code[c] = __float_as_uint(f[c]);
                }
                // K: the word of a pair of lanes (q even, q odd); V: the lane's own 16 bits
                const uint32_t part = (code[0] + code[2] * 16u + code[1] * 65536u + code[3] * 1048576u - 0x4b400000u * (1u + 16u + 65536u + 1048576u)) << (8 * (q & 1));
                const uint32_t word = part | __shfl_xor_sync(0xffffffffu, part, 1);
                const uint16_t v_codes = (uint16_t)(code[0] + code[1] * 16u + code[2] * 256u + code[3] * 4096u), v_scale = (uint16_t)(q ? sm >> 16 : sm);
                uint8_t* const codes = to + codes_at[it];
                uint8_t* const scales = to + scales_at[it];
                if (kv == 0) {
                    if (WHOLE || (to && (parity ? has1 : has0))) {
                        if (!(q & 1)) *reinterpret_cast<uint32_t*>(codes) = word;
                        if (q == 0) *reinterpret_cast<uint32_t*>(scales) = sm;
                    }
                } else if (WHOLE && SAME_LANE) {
                    if (parity == 0) {
                        v_low[it] = v_codes;
                        s_low[it] = v_scale;
                    } else {
                        *reinterpret_cast<uint32_t*>(codes) = v_low[max(it - G / 4, 0)] | (uint32_t)v_codes << 16;
                        if (q < 2) *reinterpret_cast<uint32_t*>(scales) = s_low[max(it - G / 4, 0)] | (uint32_t)v_scale << 16;
                    }
                } else if (WHOLE || (to && (parity ? has1 : has0))) {
                    *reinterpret_cast<uint16_t*>(codes + parity * 2) = v_codes;
                    if (q < 2) *reinterpret_cast<uint16_t*>(scales + parity * 2) = v_scale;
                }
                if (holds && back[it] && (WHOLE || (dst && (parity ? has1 : has0)))) {
                    const float Sf = low_of<true>(sm), Mf = high_of<true>(sm);
                    float held[4];                   // M + S (1 + c / 16): the product is exact, so that one rounding is all there is
#pragma unroll
                    for (int c = 0; c < 4; ++c) held[c] = fmaf(Sf, fmaf(f[c] - 12582912.f, 0.0625f, 1.f), Mf);
                    uint2 y;
                    if constexpr (F16) {
                        const __half2 u = __floats2half2_rn(held[0], held[1]), v = __floats2half2_rn(held[2], held[3]);
                        y = make_uint2(*reinterpret_cast<const uint32_t*>(&u), *reinterpret_cast<const uint32_t*>(&v));
                    } else {
                        y = make_uint2(pack_bf16x2(held[0], held[1]), pack_bf16x2(held[2], held[3]));
                    }
                    *reinterpret_cast<uint2*>(back[it] + (h - h0) * D) = y;
                }
            }
        };
        if (has0 && has1 && dst && !wide) write(std::true_type{});
        else write(std::false_type{});
        if (to) to += head_bytes;
    }
}

template <int D, bool F16, bool ROT>
cudaError_t launch_append(const AppendArgs& a, RotaryArgs ro, DeviceCounters* dc, DeviceCounters* dc_next, cudaStream_t stream) {
    const long long warps = (long long)a.units * a.by_chunks.d;
    cudaLaunchConfig_t cfg = {};
    ro.key_blocks = (int)((warps + APPEND_WARPS - 1) / APPEND_WARPS);
    long long blocks = ro.key_blocks;
    if (ro.q) {
        // A thread takes one head while an SM has room for more blocks, then up to eight (the angles are worked out once), or so many that all threads can be counted.  (64 trees of up to 16 tokens, 32
        // heads: 6.3 us; one head a thread up to 2048 threads an SM, in rounds, 1.6 more.)
        const long long slots = D / 8, full = 148LL * 32 * APPEND_WARPS * ROT_CTAS, most = 0x7fffff00LL - 64 * APPEND_WARPS;
        long long groups = ro.heads;
        if (groups * slots * a.rows > full) groups = std::max(std::max((long long)(ro.heads + 7) / 8, std::min(groups, full / (slots * a.rows))), 1LL);
        if (groups * slots * a.rows > most) groups = std::max(most / (slots * a.rows), 1LL);
        const long long each = (ro.heads + groups - 1) / groups;                       // (as many heads for all, up to the last group)
        groups = (ro.heads + each - 1) / each;
        if (groups * slots * a.rows > most) return cudaErrorInvalidConfiguration;      // (refused ahead of this)
        ro.by_slots = fastdiv_make((uint32_t)slots);
        ro.by_groups = fastdiv_make((uint32_t)groups);
        blocks += (groups * slots * a.rows + 32 * APPEND_WARPS - 1) / (32 * APPEND_WARPS);
    }
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(32 * APPEND_WARPS);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, cache_append_kernel<D, F16, ROT>, a, ro, dc, dc_next);
}

}  // namespace

int cache_append(const psa_cache& c, const psa_rotary* rotary, const void* Q, const void* K, const void* V, long long q_stride, long long k_stride, long long v_stride,
                 const int* depths, const int* seqs, const int* starts, int sequences, int rows, int heads, int dtype, void* q_out, void* k_held, void* v_held, DeviceCounters* dc,
                 DeviceCounters* dc_next, cudaStream_t stream) {
    if ((long long)rows / 2 + sequences > 0x7fffffffLL) return PSA_ERR_SHAPE;
    const int units = rows / 2 + sequences;
    // one head a warp until the GPU is full of warps, then up to eight (their look-ups are made once)
    const long long full = 148 * 16;
    const int per_warp = (int)std::min(std::max((long long)units * c.kv_heads / full, 1LL), 8LL), chunks = (c.kv_heads + per_warp - 1) / per_warp;
    if ((long long)units * chunks > 0x7fffff00LL) return PSA_ERR_SHAPE;
    const AppendArgs a = {static_cast<uint8_t*>(c.pool), c.tables, c.lens, seqs, starts, static_cast<const uint16_t*>(K), static_cast<const uint16_t*>(V),
                          static_cast<uint16_t*>(k_held), static_cast<uint16_t*>(v_held), k_stride, v_stride,
                          c.pages, c.slots, c.width, c.page_size, c.kv_heads, sequences, rows, per_warp, units, fastdiv_make((uint32_t)chunks),
                          fastdiv_make((uint32_t)c.page_size)};
    RotaryArgs ro = {};
    if (rotary)
        ro = RotaryArgs{rotary->freqs, depths, rotary->amplitude, rotary->rot, rotary->interleaved != 0, static_cast<const uint16_t*>(Q), static_cast<uint16_t*>(q_out), q_stride, heads,
                        0, FastDiv{}, FastDiv{}};
    cudaError_t e = cudaErrorInvalidValue;
    const bool f16 = dtype == PSA_F16;
    auto launch = [&](auto width) {
        constexpr int D = decltype(width)::value;
        if (rotary) return f16 ? launch_append<D, true, true>(a, ro, dc, dc_next, stream) : launch_append<D, false, true>(a, ro, dc, dc_next, stream);
        return f16 ? launch_append<D, true, false>(a, ro, dc, dc_next, stream) : launch_append<D, false, false>(a, ro, dc, dc_next, stream);
    };
    using std::integral_constant;
    switch (c.d_k) {
        case 32: e = launch(integral_constant<int, 32>{}); break;
        case 64: e = launch(integral_constant<int, 64>{}); break;
        case 96: e = launch(integral_constant<int, 96>{}); break;
        case 128: e = launch(integral_constant<int, 128>{}); break;
        case 256: e = launch(integral_constant<int, 256>{}); break;
        default: return PSA_ERR_UNSUPPORTED;
    }
    if (e != cudaSuccess) { set_cuda_error(e, "cache_append_kernel launch"); return PSA_ERR_CUDA; }
    return PSA_OK;
}

}  // namespace psa
