// The pages of a cache: who holds which.  Tables of pages per sequence (a row of `width` entries each, -1 where there is none), tokens per
// sequence and references per page lie on the device and are changed there, in stream order, so that no step of a server has to come back to the host.
//
//   free     the pages of a sequence lose a reference each, its row and length are cleared
//   fork     a sequence without pages gets those of another, one reference more each
//   reserve  room for so many more tokens of each sequence; a page that is partly filled and shared is copied before it is written to, pages behind a length that was
//            taken back are given back first (left in the table they would be overwritten there, and stay counted for ever)
//   compact  live pages beyond the first `live` ones move into the holes before them
//   copy     pages by list
// Free pages are those without references, and are handed out in ascending order in the order of the list: what a call does depends on its arguments alone,
// not on the order in which CTAs run.  Tables and counts are a few hundred KB at most and are worked on by one CTA (latency bounds it); pages are
// moved by the whole GPU (the copy rate of the memory bounds it).  Measured: compaction of a pool of one layer, 330 MB read and written
// in 57 us (5.8 TB/s), 7 of them the map.  All new pages of a sequence are written by one thread: room for a prompt of 131,072 tokens in pages of 16 takes 450 us, for 64 of
// 2048 25.
#include "psa_internal.h"
#include "sm100.cuh"

namespace psa {

namespace {

constexpr int META_THREADS = 1024;
constexpr int FREE_NEAR = 2048;                 // free pages of a call that are kept in shared memory
constexpr int PAIRWISE = 256;                   // see pages_reserve_kernel
constexpr int RESERVE_MOST = 4096;              // sequences of one call (their last pages are compared in shared memory)
// A list in which a sequence grows by more pages is summed up in 64 bits (which costs a call of 64 sequences 0.3 us of 18): RESERVE_MOST times this is no more than 31 bits take.
constexpr int MANY_PAGES = 1 << 18;

struct PageArgs {
    int *tables, *lens, *refs;
    int slots, width, pages, page_size;
};

__device__ __forceinline__ void bad_argument(DeviceCounters* dc) { atomicExch(&dc->status, (int)PSA_ERR_SHAPE); }
__device__ __forceinline__ void next_block(DeviceCounters* dc_next) {
    if (threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0 && dc_next) *dc_next = DeviceCounters{0, 0, 0, 0, 0, 0, 0};
}

__global__ void __launch_bounds__(128) pages_free_kernel(const PageArgs p, const int* seqs, DeviceCounters* dc, DeviceCounters* dc_next) {
    grid_dependency_wait();
    next_block(dc_next);
    const int s = seqs[blockIdx.x];
    if (s < 0 || s >= p.slots) { if (threadIdx.x == 0) bad_argument(dc); return; }
    int* row = p.tables + (size_t)s * p.width;
    for (int i = threadIdx.x; i < p.width; i += 128) {
        const int page = atomicExch(row + i, -1);       // (a sequence listed twice gives its pages back once)
        if (page < 0) continue;
        if (page < p.pages) atomicSub(p.refs + page, 1);
        else bad_argument(dc);
    }
    if (threadIdx.x == 0) p.lens[s] = 0;
}

__global__ void __launch_bounds__(128) pages_fork_kernel(const PageArgs p, const int* parents, const int* children, DeviceCounters* dc, DeviceCounters* dc_next) {
    grid_dependency_wait();
    next_block(dc_next);
    const int from = parents[blockIdx.x], to = children[blockIdx.x];
    if (from < 0 || from >= p.slots || to < 0 || to >= p.slots || from == to) { if (threadIdx.x == 0) bad_argument(dc); return; }
    const int* src = p.tables + (size_t)from * p.width;
    int* dst = p.tables + (size_t)to * p.width;
    bool held = false;
    for (int i = threadIdx.x; i < p.width; i += 128) held |= dst[i] >= 0;
    if (__syncthreads_or(held)) { if (threadIdx.x == 0) bad_argument(dc); return; }      // a child that still holds pages would lose them
    for (int i = threadIdx.x; i < p.width; i += 128) {
        const int page = src[i];
        dst[i] = page;
        if (page < 0) continue;
        if (page < p.pages) atomicAdd(p.refs + page, 1);
        else bad_argument(dc);
    }
    if (threadIdx.x == 0) p.lens[to] = p.lens[from];
}

// Exclusive sum over the CTA; *total: of all.  `tmp`: 32 numbers of shared memory.
template <class T>
__device__ __forceinline__ T cta_scan(T v, T* tmp, T* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    T x = v;
#pragma unroll
    for (int s = 1; s < 32; s *= 2) {
        const T y = __shfl_up_sync(0xffffffffu, x, s);
        if (lane >= s) x += y;
    }
    __syncthreads();
    if (lane == 31) tmp[warp] = x;
    __syncthreads();
    T w = tmp[lane];                            // META_THREADS / 32 = 32 warps
#pragma unroll
    for (int s = 1; s < 32; s *= 2) {
        const T y = __shfl_up_sync(0xffffffffu, w, s);
        if (lane >= s) w += y;
    }
    *total = __shfl_sync(0xffffffffu, w, 31);
    return __shfl_sync(0xffffffffu, w, warp) - tmp[warp] + x - v;
}

// Pages are looked through 16 at a time and thread, one round of the CTA per 16,384: bit c of the result says whether `what` holds of the count of page first + c.
constexpr int PER_THREAD = 16, ROUND = META_THREADS * PER_THREAD;
struct Counts16 {
    int4 c[PER_THREAD / 4];
};
__device__ __forceinline__ Counts16 load_counts(const int* refs, int pages, long long first) {
    Counts16 r;
    const bool aligned = (reinterpret_cast<uintptr_t>(refs) & 15u) == 0;
#pragma unroll
    for (int i = 0; i < PER_THREAD / 4; ++i) {
        const long long at = first + 4 * i;
        r.c[i] = make_int4(-1, -1, -1, -1);      // (no such page: neither free nor live)
        if (at + 3 < pages && aligned) {
            r.c[i] = *reinterpret_cast<const int4*>(refs + at);
        } else {
            if (at < pages) r.c[i].x = refs[at];
            if (at + 1 < pages) r.c[i].y = refs[at + 1];
            if (at + 2 < pages) r.c[i].z = refs[at + 2];
            if (at + 3 < pages) r.c[i].w = refs[at + 3];
        }
    }
    return r;
}
template <class What>
__device__ __forceinline__ uint32_t bits_of(const Counts16& r, What what) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < PER_THREAD / 4; ++i)
        m |= ((what(r.c[i].x) ? 1u : 0u) | (what(r.c[i].y) ? 2u : 0u) | (what(r.c[i].z) ? 4u : 0u) | (what(r.c[i].w) ? 8u : 0u)) << (4 * i);
    return m;
}

// What reserve does to sequence i of the list.
struct Need {
    int seq, held, add, have, want, last;       // last: its last page, if that is partly filled and about to be written to (else -1)
    bool over;                                  // it holds pages behind its length (which was taken back): they are given back
};
__device__ __forceinline__ Need need_of(const PageArgs& p, const int* seqs, const int* add, int i) {
    Need n = {seqs[i], 0, 0, 0, 0, -1, false};
    if (n.seq < 0 || n.seq >= p.slots) { n.seq = -1; return n; }
    n.held = max(p.lens[n.seq], 0);
    n.add = max(add[i], 0);
    n.have = (int)(((long long)n.held + p.page_size - 1) / p.page_size);
    const long long want = ((long long)n.held + n.add + p.page_size - 1) / p.page_size;
    if (want > p.width || n.have > p.width) { n.seq = -1; return n; }
    n.want = (int)want;
    const int* row = p.tables + (size_t)n.seq * p.width;
    const bool part = n.add > 0 && n.held % p.page_size;
    const int last = part ? row[n.have - 1] : -1, behind = n.have < p.width ? row[n.have] : -1;      // (asked for together)
    n.over = behind >= 0;
    if (part) {
        n.last = last;
        if (last < 0 || last >= p.pages) n.seq = -1;
    }
    return n;
}

// free_list: room for p.pages numbers, marks: for twice as many (long lists only); pairs: (from, to) per sequence of the list, -1 where nothing is to be copied.
__global__ void __launch_bounds__(META_THREADS) pages_reserve_kernel(const PageArgs p, const int* seqs, const int* add, int count, int* short_by, int* free_list, int* marks,
                                                                     int2* pairs, DeviceCounters* dc, DeviceCounters* dc_next) {
    __shared__ __align__(16) int last_s[RESERVE_MOST];
    __shared__ int free_near[FREE_NEAR];
    __shared__ int tmp[32];
    __shared__ long long tmp_long[32];
    __shared__ int bad_s;
    const int tid = threadIdx.x;
    if (tid == 0) bad_s = 0;
    grid_dependency_wait();
    next_block(dc_next);
    grid_launch_dependents();
    Counts16 counts = load_counts(p.refs, p.pages, (long long)tid * PER_THREAD);         // (asked for ahead: nothing below depends on it for long)
    constexpr int PER = RESERVE_MOST / META_THREADS;
    Need n[PER];
    bool bad = false, many = false, over = false;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int i = k * META_THREADS + tid;
        n[k] = Need{-1, 0, 0, 0, 0, -1, false};
        if (i < count) {
            n[k] = need_of(p, seqs, add, i);
            bad |= n[k].seq < 0;
            last_s[i] = n[k].seq < 0 ? -1 : n[k].last;
            many |= n[k].want - n[k].have > MANY_PAGES;
            over |= n[k].over;
        }
    }
    if (__syncthreads_or(bad || many || over)) {         // (rare)
        many = __syncthreads_or(many);
        if (__syncthreads_or(over)) {
            auto behind = [&](auto what) {               // the columns behind the lengths, up to the first without a page
                for (int k = 0; k < PER; ++k)
                    if (n[k].seq >= 0 && n[k].over)
                        for (int c = n[k].have; c < p.width && p.tables[(size_t)n[k].seq * p.width + c] >= 0; ++c) what(p.tables + (size_t)n[k].seq * p.width + c);
            };
            behind([&](int* at) { bad |= *at >= p.pages; });
            if (!__syncthreads_or(bad)) {
                behind([&](int* at) {
                    const int page = atomicExch(at, -1);
                    if (page >= 0) atomicSub(p.refs + page, 1);
                });
                __syncthreads();
                counts = load_counts(p.refs, p.pages, (long long)tid * PER_THREAD);
            }
        }
    }
    // pages that each sequence needs: those that it grows by, and one for a shared last page.  Of several in the list that share one, all but the
    // last reference copy it, in the order of the list: the one that is left alone with the page keeps it.
    // Longer lists count the references to a page that are in the list, and find the last one, beside the page (1024 sequences that all share their last page, freed,
    // forked and reserved for, 19 us so and 27 by looking at all entries before, 2048 22.5 and 68.6, 256 19 either way, which is the host's side of the three calls).
    auto listed = [&](int page) { return marks + 2 * (size_t)page; };
    auto latest = [&](int page) { return marks + 2 * (size_t)page + 1; };
    if (count > PAIRWISE) {
        for (int i = tid; i < count; i += META_THREADS)
            if (last_s[i] >= 0) *reinterpret_cast<int2*>(listed(last_s[i])) = make_int2(0, 0);
        __syncthreads();
        for (int i = tid; i < count; i += META_THREADS)
            if (last_s[i] >= 0) { atomicAdd(listed(last_s[i]), 1); atomicMax(latest(last_s[i]), i + 1); }
        __syncthreads();
    }
    long long total = 0;
    int first[PER];                              // (read only if the pages are there, so that it fits)
    bool copy[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int i = k * META_THREADS + tid;
        copy[k] = false;
        first[k] = 0;
        if (k * META_THREADS >= count) continue;        // (uniform)
        const int refs = i < count && n[k].seq >= 0 && n[k].last >= 0 ? p.refs[n[k].last] : 0;
        if (count <= PAIRWISE) {
            if (refs > 1) {
                int before = 0;
                for (int j = 0; j < i; ++j) before += last_s[j] == n[k].last;
                copy[k] = refs - before > 1;
            }
        } else {
            copy[k] = refs > 1 && (__ldcg(listed(n[k].last)) < refs || __ldcg(latest(n[k].last)) != i + 1);
        }
        const int need = n[k].seq >= 0 ? n[k].want - n[k].have + copy[k] : 0;
        if (many) {
            long long all;
            first[k] = (int)(total + cta_scan((long long)need, tmp_long, &all));
            total += all;
        } else {
            int all;
            first[k] = (int)total + cta_scan(need, tmp, &all);
            total += all;
        }
    }
    if (bad) bad_s = 1;
    // ---- the first `total` pages without references, ascending: in shared memory, those that it has no room for behind
    int found = 0;
    for (long long at = 0; at < p.pages && found < total; at += ROUND) {
        const long long mine = at + (long long)tid * PER_THREAD;
        if (at > 0) counts = load_counts(p.refs, p.pages, mine);
        const uint32_t is_free = bits_of(counts, [](int c) { return c == 0; });
        int all, k = found + cta_scan(__popc(is_free), tmp, &all);
        for (uint32_t m = is_free; m && k < total; m &= m - 1, ++k) {
            const int page = (int)(mine + __ffs(m) - 1);
            if (k < FREE_NEAR) free_near[k] = page;
            else free_list[k] = page;
        }
        found += all;
    }
    __syncthreads();                            // (the list is read by other threads of this CTA; bad_s is complete)
    auto free_page = [&](int k) { return k < FREE_NEAR ? free_near[k] : free_list[k]; };
    const bool go = !bad_s && found >= total;
    if (tid == 0) {
        *short_by = (int)min(max(total - found, 0LL), 0x7fffffffLL);
        if (bad_s) bad_argument(dc);
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int i = k * META_THREADS + tid;
        if (i >= count) break;
        int2 pair = make_int2(-1, -1);
        if (go) {
            int* row = p.tables + (size_t)n[k].seq * p.width;
            int at = first[k];
            if (copy[k]) {
                const int page = free_page(at++);
                pair = make_int2(n[k].last, page);
                row[n[k].have - 1] = page;
                p.refs[page] = 1;
                atomicSub(p.refs + n[k].last, 1);
            }
            for (int c = n[k].have; c < n[k].want; ++c) {
                const int page = free_page(at++);
                row[c] = page;
                p.refs[page] = 1;
            }
            p.lens[n[k].seq] = n[k].held + n[k].add;
        }
        pairs[i] = pair;
    }
}

// Bytes of whole pages from place to place, 16 at a time.  grid.x: parts of a page, grid.y: pages of the list, in turns.
constexpr int COPY_THREADS = 256, COPY_PER = 8;
struct PoolCopy {
    const uint8_t* from;
    uint8_t* to;
    long long page_bytes, from_layer, to_layer;         // bytes between layers
    int from_pages, to_pages, layers, count;
};
// next(i): the pages of entry i.
template <class Next>
__device__ __forceinline__ void copy_pages(const PoolCopy& c, Next next) {
    const long long words = c.page_bytes / 16;
    for (int i = blockIdx.y; i < c.count; i += gridDim.y) {
        const int2 p = next(i);
        if (p.x < 0 || p.y < 0 || p.x >= c.from_pages || p.y >= c.to_pages) continue;
        for (int layer = 0; layer < c.layers; ++layer) {
            const uint4* src = reinterpret_cast<const uint4*>(c.from + layer * c.from_layer + p.x * c.page_bytes);
            uint4* dst = reinterpret_cast<uint4*>(c.to + layer * c.to_layer + p.y * c.page_bytes);
            if (src == dst) continue;
            for (long long w = (long long)blockIdx.x * COPY_THREADS * COPY_PER + threadIdx.x; w < words; w += (long long)gridDim.x * COPY_THREADS * COPY_PER) {
                uint4 v[COPY_PER];
#pragma unroll
                for (int k = 0; k < COPY_PER; ++k)
                    if (w + k * COPY_THREADS < words) v[k] = __ldcs(src + w + k * COPY_THREADS);
#pragma unroll
                for (int k = 0; k < COPY_PER; ++k)
                    if (w + k * COPY_THREADS < words) __stcs(dst + w + k * COPY_THREADS, v[k]);
            }
        }
    }
}
__global__ void __launch_bounds__(COPY_THREADS) copy_pairs_kernel(const PoolCopy c, const int2* pairs) {
    grid_dependency_wait();
    copy_pages(c, [&](int i) { return pairs[i]; });
}
__global__ void __launch_bounds__(COPY_THREADS) copy_lists_kernel(const PoolCopy c, const int* src, const int* dst, DeviceCounters* dc, DeviceCounters* dc_next) {
    grid_dependency_wait();
    next_block(dc_next);
    copy_pages(c, [&](int i) {
        const int2 p = make_int2(src[i], dst[i]);
        if (threadIdx.x == 0 && (p.x < 0 || p.y < 0 || p.x >= c.from_pages || p.y >= c.to_pages)) bad_argument(dc);
        return p;
    });
}

// Where every page goes: map[page] (-1: nowhere), the counts in their new places and the number of live pages.  One CTA; the counts may be changed in place.
// holes, movers: room for `pages` numbers each.
__global__ void __launch_bounds__(META_THREADS) compact_map_kernel(const int* refs, int pages, int* new_refs, int* live, int* map, int* holes, int* movers,
                                                                   DeviceCounters* dc_next) {
    __shared__ int tmp[32];
    const int tid = threadIdx.x;
    grid_dependency_wait();
    next_block(dc_next);
    grid_launch_dependents();
    auto is_live = [](int c) { return c > 0; };
    Counts16 counts = load_counts(refs, pages, (long long)tid * PER_THREAD);
    int n = __popc(bits_of(counts, is_live));
    for (long long at = ROUND; at < pages; at += ROUND) n += __popc(bits_of(load_counts(refs, pages, at + (long long)tid * PER_THREAD), is_live));
    int L;
    cta_scan(n, tmp, &L);
    int nholes = 0, nmovers = 0;
    for (long long at = 0; at < pages; at += ROUND) {
        const long long mine = at + (long long)tid * PER_THREAD;
        if (at > 0) counts = load_counts(refs, pages, mine);
        const uint32_t live_bits = bits_of(counts, is_live);
        // pages of the thread before L: bits below `front`
        const int front = (int)min(max((long long)L - mine, 0LL), (long long)PER_THREAD), there = (int)min(max((long long)pages - mine, 0LL), (long long)PER_THREAD);
        const uint32_t before = (1u << front) - 1u, hole = ~live_bits & before, mover = live_bits & ~before;
        // a round may hold both kinds: counted together, holes in the low half
        int all;
        const int k = cta_scan(__popc(hole) | __popc(mover) << 16, tmp, &all);
        int h = nholes + (k & 0xffff), v = nmovers + (k >> 16);
        for (int c = 0; c < there; ++c) {
            const int i = (int)mine + c;
            if (hole >> c & 1u) holes[h++] = i;
            if (mover >> c & 1u) movers[v++] = i;
            else map[i] = live_bits >> c & 1u ? i : -1;
        }
        nholes += all & 0xffff;
        nmovers += all >> 16;
    }
    __syncthreads();
    for (int k = tid; k < nmovers; k += META_THREADS) map[movers[k]] = holes[k];         // (as many holes as movers)
    if (new_refs != refs)
        for (int i = tid; i < pages; i += META_THREADS) new_refs[i] = i < L ? refs[i] : 0;
    __syncthreads();
    for (int k = tid; k < nmovers; k += META_THREADS) new_refs[holes[k]] = refs[movers[k]];
    __syncthreads();
    if (new_refs == refs)
        for (int k = tid; k < nmovers; k += META_THREADS) new_refs[movers[k]] = 0;
    if (tid == 0) *live = L;
}
// grid.y turns over the pages; the last rows of the grid rewrite the tables.
__global__ void __launch_bounds__(COPY_THREADS) compact_move_kernel(const PoolCopy c, const int* map, const int* tables, int* new_tables, long long entries, DeviceCounters* dc) {
    grid_dependency_wait();
    const long long stride = (long long)gridDim.x * gridDim.y * COPY_THREADS;
    for (long long i = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * COPY_THREADS + threadIdx.x; i < entries; i += stride) {
        const int page = tables[i];
        int to = page;
        if (page >= 0) {
            to = page < c.from_pages ? map[page] : -1;
            if (to < 0) bad_argument(dc);       // a table names a page that nobody counts
        }
        new_tables[i] = to;
    }
    copy_pages(c, [&](int i) { return make_int2(i, map[i]); });
}

template <class... P, class... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, int threads, cudaStream_t stream, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}
PageArgs args_of(const psa_pages& p) { return PageArgs{p.tables, p.lens, p.refs, p.slots, p.width, p.pages, p.page_size}; }
int status_of(cudaError_t e, const char* what) {
    if (e == cudaSuccess) return PSA_OK;
    set_cuda_error(e, what);
    return PSA_ERR_CUDA;
}
// Parts that a page is copied in, and pages copied at a time: a few rounds of the whole GPU.
dim3 copy_grid(const PoolCopy& c) {
    const long long parts = (c.page_bytes / 16 + COPY_THREADS * COPY_PER - 1) / (COPY_THREADS * COPY_PER);
    return dim3((unsigned)(parts < 64 ? parts : 64), (unsigned)(c.count < 32768 ? c.count : 32768));
}

}  // namespace

int pages_free(const psa_pages& p, const int* seqs, int count, DeviceCounters* dc, DeviceCounters* dc_next, cudaStream_t stream) {
    return status_of(launch(pages_free_kernel, dim3(count), 128, stream, args_of(p), seqs, dc, dc_next), "pages_free_kernel launch");
}
int pages_fork(const psa_pages& p, const int* parents, const int* children, int count, DeviceCounters* dc, DeviceCounters* dc_next, cudaStream_t stream) {
    return status_of(launch(pages_fork_kernel, dim3(count), 128, stream, args_of(p), parents, children, dc, dc_next), "pages_fork_kernel launch");
}
size_t pages_reserve_scratch_bytes(int pages, int count) { return ((size_t)pages * 4 + 255) / 256 * 256 + ((size_t)count * 8 + 255) / 256 * 256 + (count > PAIRWISE ? (size_t)pages * 8 : 0); }
int pages_reserve(const psa_pages& p, void* pool, long long page_bytes, int layers, const int* seqs, const int* add, int count, int* short_by, void* scratch,
                  DeviceCounters* dc, DeviceCounters* dc_next, cudaStream_t stream) {
    if (count > RESERVE_MOST) return PSA_ERR_UNSUPPORTED;
    int* free_list = static_cast<int*>(scratch);
    int2* pairs = reinterpret_cast<int2*>(static_cast<char*>(scratch) + ((size_t)p.pages * 4 + 255) / 256 * 256);
    int* marks = reinterpret_cast<int*>(reinterpret_cast<char*>(pairs) + ((size_t)count * 8 + 255) / 256 * 256);
    const int rc = status_of(launch(pages_reserve_kernel, dim3(1), META_THREADS, stream, args_of(p), seqs, add, count, short_by, free_list, marks, pairs, dc, dc_next), "pages_reserve_kernel launch");
    if (rc != PSA_OK) return rc;
    const long long layer = page_bytes * p.pages;
    const PoolCopy c = {static_cast<const uint8_t*>(pool), static_cast<uint8_t*>(pool), page_bytes, layer, layer, p.pages, p.pages, layers, count};
    return status_of(launch(copy_pairs_kernel, copy_grid(c), COPY_THREADS, stream, c, const_cast<const int2*>(pairs)), "copy_pairs_kernel launch");
}
size_t pages_compact_scratch_bytes(int pages) { return 3 * (((size_t)pages * 4 + 255) / 256 * 256); }
int pages_compact(const psa_pages& p, const void* pool, long long page_bytes, int layers, int* new_tables, int* new_refs, void* new_pool, int* live, void* scratch,
                  DeviceCounters* dc, DeviceCounters* dc_next, cudaStream_t stream) {
    const size_t part = ((size_t)p.pages * 4 + 255) / 256 * 256;
    int* map = static_cast<int*>(scratch);
    int* holes = reinterpret_cast<int*>(static_cast<char*>(scratch) + part);
    int* movers = reinterpret_cast<int*>(static_cast<char*>(scratch) + 2 * part);
    int rc = status_of(launch(compact_map_kernel, dim3(1), META_THREADS, stream, const_cast<const int*>(p.refs), p.pages, new_refs, live, map, holes, movers, dc_next), "compact_map_kernel launch");
    if (rc != PSA_OK) return rc;
    const long long layer = page_bytes * p.pages;
    const PoolCopy c = {static_cast<const uint8_t*>(pool), static_cast<uint8_t*>(new_pool), page_bytes, layer, layer, p.pages, p.pages, layers, p.pages};
    return status_of(launch(compact_move_kernel, copy_grid(c), COPY_THREADS, stream, c, const_cast<const int*>(map), const_cast<const int*>(p.tables), new_tables, (long long)p.slots * p.width, dc),
                     "compact_move_kernel launch");
}
int pages_copy(const void* pool, int pages, void* new_pool, int new_pages, long long page_bytes, int layers, const int* src, const int* dst, int count,
               DeviceCounters* dc, DeviceCounters* dc_next, cudaStream_t stream) {
    const PoolCopy c = {static_cast<const uint8_t*>(pool), static_cast<uint8_t*>(new_pool), page_bytes, page_bytes * pages, page_bytes * new_pages, pages, new_pages, layers, count};
    return status_of(launch(copy_lists_kernel, copy_grid(c), COPY_THREADS, stream, c, src, dst, dc, dc_next), "copy_lists_kernel launch");
}

}  // namespace psa
