// Appending keys and values to the cache held in 4 bits (layout: psa_cache.cuh).
//
// Per token, head and group of 32 channels, lo and hi being the group's least and greatest number:
//     S = fp16(16 (hi - lo) / 15),   M = fp16(lo - S),   c = rint((x - M - S) 16 / S) in 0 .. 15,
// so that c = 0 stands for lo and c = 15 for hi up to the roundings of S and M; the codes are taken against the rounded numbers, and the error of
// a number is half a step, (hi - lo) / 30.  All in fp32, every operation rounded by itself (no contraction), so that the result is one of definition.
//
// Bound by memory: 2 bytes read and 5 bits written per number, 2 more written when the held values are asked for.  A warp takes two tokens of a head,
// K and V, eight lanes a group (four channels each, one load of 8 bytes), so that all its loads are in flight together.
#include "psa_cache.cuh"
#include "psa_internal.h"
#include "sm100.cuh"

namespace psa {

namespace {

constexpr int APPEND_WARPS = 8;

struct AppendArgs {
    uint8_t* pool;
    const int *tables, *lens, *seqs, *starts;
    const uint16_t *k, *v;
    uint16_t *k_held, *v_held;
    long long k_stride, v_stride;
    int pages, slots, width, page_size, kv_heads, sequences, rows;
};

// The sequence that row r belongs to: the last b with starts[b] <= r.  32 numbers at a time, so that a batch of up to 1024 takes two loads.
__device__ __forceinline__ int sequence_of(const int* starts, int sequences, int r, int lane) {
    int lo = 0, n = sequences;                 // the answer lies in lo .. lo + n - 1
    while (n > 1) {
        const int step = (n + 31) / 32, at = lo + lane * step;
        const bool le = lane * step < n && starts[at] <= r;
        const uint32_t m = __ballot_sync(0xffffffffu, le);
        const int k = m ? 31 - __clz(m) : 0;
        lo += k * step;
        n = min(step, n - k * step);
    }
    return lo;
}

template <int D, bool F16>
__global__ void __launch_bounds__(32 * APPEND_WARPS) cache_append_kernel(const AppendArgs a, DeviceCounters* dc, DeviceCounters* dc_next) {
    constexpr int G = D / 32;
    using B = CacheBlock<D>;
    grid_dependency_wait();
    if (threadIdx.x == 0 && blockIdx.x == 0 && dc_next) *dc_next = DeviceCounters{0, 0, 0, 0, 0, 0, 0};
    const int lane = threadIdx.x & 31;
    const long long unit = (long long)blockIdx.x * APPEND_WARPS + (threadIdx.x >> 5);
    const int pair = (int)(unit / a.kv_heads), h = (int)(unit - (long long)pair * a.kv_heads);
    if (2LL * pair >= a.rows) return;
    const int r = 2 * pair + (lane & 1);       // lanes take the two rows in turn to find out where they go
    // (rows outside starts[0] .. starts[sequences] belong to no sequence)
    uint8_t* dst = nullptr;
    int tok = 0;
    {
        const int b0 = sequence_of(a.starts, a.sequences, 2 * pair, lane);
        int b = b0;
        if (2 * pair + 1 < a.rows) {
            const int b1 = sequence_of(a.starts, a.sequences, 2 * pair + 1, lane);
            if (lane & 1) b = b1;
        }
        if (r < a.rows) {
            const int first = a.starts[b], end = a.starts[b + 1], seq = a.seqs[b];
            if (r >= first && r < end && seq >= 0 && seq < a.slots) {
                const int pos = a.lens[seq] - (end - r);
                const int col = pos / a.page_size;
                if (pos >= 0 && col < a.width) {
                    const int page = a.tables[(size_t)seq * a.width + col];
                    if (page >= 0 && page < a.pages) {
                        const int in = pos - col * a.page_size, blocks = a.page_size / CACHE_BLOCK;
                        tok = in % CACHE_BLOCK;
                        dst = a.pool + (((size_t)page * a.kv_heads + h) * blocks + in / CACHE_BLOCK) * B::BYTES;
                    }
                }
            }
            if (!dst) atomicExch(&dc->status, (int)PSA_ERR_SHAPE);      // (device-side arguments that name no place: reported, nothing written)
        }
    }
    const unsigned long long dst_bits = reinterpret_cast<unsigned long long>(dst);
    // ---- loads: subgroup of eight lanes = one (K or V, row, group); q = lane inside it, channels 4q .. 4q+3 of the group
    const int q = lane & 7;
    uint2 x[G];
#pragma unroll
    for (int it = 0; it < G; ++it) {
        const int sg = it * 4 + (lane >> 3), kv = sg / (2 * G), row = 2 * pair + (sg / G) % 2, w = sg % G;
        x[it] = make_uint2(0, 0);
        if (row < a.rows) {
            const uint16_t* src = kv ? a.v + (size_t)row * a.v_stride : a.k + (size_t)row * a.k_stride;
            x[it] = *reinterpret_cast<const uint2*>(src + h * D + 32 * w + 4 * q);
        }
    }
#pragma unroll
    for (int it = 0; it < G; ++it) {
        const int sg = it * 4 + (lane >> 3), kv = sg / (2 * G), parity = (sg / G) % 2, row = 2 * pair + parity, w = sg % G;
        uint8_t* const to = reinterpret_cast<uint8_t*>(__shfl_sync(0xffffffffu, dst_bits, parity));
        const int t16 = __shfl_sync(0xffffffffu, tok, parity);
        float f[4];
        if constexpr (F16) {
            const float2 u = __half22float2(*reinterpret_cast<const __half2*>(&x[it].x)), v = __half22float2(*reinterpret_cast<const __half2*>(&x[it].y));
            f[0] = u.x; f[1] = u.y; f[2] = v.x; f[3] = v.y;
        } else {
            f[0] = __uint_as_float(x[it].x << 16); f[1] = __uint_as_float(x[it].x & 0xffff0000u);
            f[2] = __uint_as_float(x[it].y << 16); f[3] = __uint_as_float(x[it].y & 0xffff0000u);
        }
        bool nan = false;
        float lo = INFINITY, hi = -INFINITY;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            nan |= f[c] != f[c];
            f[c] = fminf(fmaxf(f[c], -CACHE_MAX), CACHE_MAX);
            lo = fminf(lo, f[c]);
            hi = fmaxf(hi, f[c]);
        }
#pragma unroll
        for (int s = 1; s < 8; s *= 2) {
            lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, s));
            hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, s));
        }
        const uint32_t nans = __ballot_sync(0xffffffffu, nan);
        const bool bad = (nans >> (lane & 24)) & 0xffu;          // a NaN anywhere in the group: the group reads back as NaN
        __half S = __float2half_rn(__fmul_rn(__fsub_rn(hi, lo), 16.f / 15.f));
        __half M = __float2half_rn(__fsub_rn(lo, __half2float(S)));
        if (bad) S = M = __ushort_as_half(0x7fff);
        const float Sf = __half2float(S), Mf = __half2float(M);
        const float step = Sf > 0.f ? __fdiv_rn(16.f, Sf) : 0.f, base = __fadd_rn(Mf, Sf);
        uint32_t code[4];
        float held[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const float y = rintf(__fmul_rn(__fsub_rn(f[c], base), step));
            code[c] = bad ? 0u : (uint32_t)fminf(fmaxf(y, 0.f), 15.f);
            held[c] = __fadd_rn(Mf, __fmul_rn(Sf, 1.f + (float)code[c] * 0.0625f));
        }
        // K: the word of a pair of lanes (q even, q odd); V: the lane's own 16 bits
        const uint32_t part = (code[0] | code[2] << 4 | (code[1] | code[3] << 4) << 16) << (8 * (q & 1));
        const uint32_t word = part | __shfl_xor_sync(0xffffffffu, part, 1);
        if (!to || row >= a.rows) continue;
        if (kv == 0) {
            if (!(q & 1)) *reinterpret_cast<uint32_t*>(to + B::K_CODES + t16 * (D / 2) + ((q >> 1) * G + w) * 4) = word;
            if (q == 0) *reinterpret_cast<__half2*>(to + B::K_SCALES + (t16 * G + w) * 4) = __halves2half2(S, M);
        } else {
            *reinterpret_cast<uint16_t*>(to + B::V_CODES + (t16 >> 1) * D + (q * G + w) * 4 + (t16 & 1) * 2) = (uint16_t)(code[0] | code[1] << 4 | code[2] << 8 | code[3] << 12);
            if (q < 2) *reinterpret_cast<__half*>(to + B::V_SCALES + ((t16 >> 1) * G + w) * 8 + q * 4 + (t16 & 1) * 2) = q ? M : S;
        }
        uint16_t* const back = kv ? a.v_held : a.k_held;
        if (back) {
            uint2 y;
            if constexpr (F16) {
                const __half2 u = __floats2half2_rn(held[0], held[1]), v = __floats2half2_rn(held[2], held[3]);
                y = make_uint2(*reinterpret_cast<const uint32_t*>(&u), *reinterpret_cast<const uint32_t*>(&v));
            } else {
                y = make_uint2(pack_bf16x2(held[0], held[1]), pack_bf16x2(held[2], held[3]));
            }
            *reinterpret_cast<uint2*>(back + ((size_t)row * a.kv_heads + h) * D + 32 * w + 4 * q) = y;
        }
    }
}

template <int D, bool F16>
cudaError_t launch_append(const AppendArgs& a, DeviceCounters* dc, DeviceCounters* dc_next, cudaStream_t stream) {
    const long long warps = ((long long)a.rows + 1) / 2 * a.kv_heads;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((warps + APPEND_WARPS - 1) / APPEND_WARPS));
    cfg.blockDim = dim3(32 * APPEND_WARPS);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, cache_append_kernel<D, F16>, a, dc, dc_next);
}

}  // namespace

int cache_append(const psa_cache& c, const void* K, const void* V, long long k_stride, long long v_stride, const int* seqs, const int* starts,
                 int sequences, int rows, int dtype, void* k_held, void* v_held, DeviceCounters* dc, DeviceCounters* dc_next, cudaStream_t stream) {
    const AppendArgs a = {static_cast<uint8_t*>(c.pool), c.tables, c.lens, seqs, starts, static_cast<const uint16_t*>(K), static_cast<const uint16_t*>(V),
                          static_cast<uint16_t*>(k_held), static_cast<uint16_t*>(v_held), k_stride, v_stride,
                          c.pages, c.slots, c.width, c.page_size, c.kv_heads, sequences, rows};
    cudaError_t e = cudaErrorInvalidValue;
    const bool f16 = dtype == PSA_F16;
    switch (c.d_k) {
        case 32: e = f16 ? launch_append<32, true>(a, dc, dc_next, stream) : launch_append<32, false>(a, dc, dc_next, stream); break;
        case 64: e = f16 ? launch_append<64, true>(a, dc, dc_next, stream) : launch_append<64, false>(a, dc, dc_next, stream); break;
        case 96: e = f16 ? launch_append<96, true>(a, dc, dc_next, stream) : launch_append<96, false>(a, dc, dc_next, stream); break;
        case 128: e = f16 ? launch_append<128, true>(a, dc, dc_next, stream) : launch_append<128, false>(a, dc, dc_next, stream); break;
        case 256: e = f16 ? launch_append<256, true>(a, dc, dc_next, stream) : launch_append<256, false>(a, dc, dc_next, stream); break;
        default: return PSA_ERR_UNSUPPORTED;
    }
    if (e != cudaSuccess) { set_cuda_error(e, "cache_append_kernel launch"); return PSA_ERR_CUDA; }
    return PSA_OK;
}

}  // namespace psa
