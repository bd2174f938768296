// Upkeep of the pages of the KV cache: copying pages, forking branches, making room for new tokens, giving
// pages back, closing the holes of the pool.  A page id names the same slot of every layer's K and V pool,
// so one call moves a page in all of them.  Which pages are taken is a pure function of the arguments: free
// pages are handed out lowest id first, to branches in their order.
//
// What bounds these calls: the page copies are HBM traffic (one page of the 32B shape is 4 MiB over 64
// layers' K and V); the integer work on tables and reference counts is latency (one CTA that scans the
// counts, then one kernel over table rows and copies).  Copies are cut into 4 KiB page-head tiles, one warp
// each, eight 16-byte loads per lane in flight before the first store, so that one page of a few layers
// already spreads over many SMs.
#include "launch.cuh"
#include "tts_internal.cuh"

#include <algorithm>

namespace tts {

namespace {

constexpr int kMaxScanThreads = 1024;
constexpr int kPerThread = 16;                         // reference counts a thread looks at per step of a scan
constexpr int kTileBytes = kPage * kHeadDim * 2;       // one page of one KV head: 4 KiB
constexpr int kTileChunks = kTileBytes / 16 / 32;      // 16-byte chunks of a tile per lane
constexpr int kCopyThreads = 256;

template <typename T>
__device__ __forceinline__ T warp_scan(T v, int lane) {                                // inclusive
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T n = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += n;
    }
    return v;
}
// Exclusive scan over the block; *total gets the sum.  `warp_sums`: 32 values, which every warp adds up for itself.
template <typename T>
__device__ T block_scan(T v, T* warp_sums, T* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const T s = warp_scan(v, lane);
    __syncthreads();                                    // the previous scan's sums have been read
    if (lane == 31) warp_sums[warp] = s;
    __syncthreads();
    const T w = lane < (int)(blockDim.x >> 5) ? warp_sums[lane] : 0, t = warp_scan(w, lane);
    *total = __shfl_sync(0xffffffffu, t, 31);
    return __shfl_sync(0xffffffffu, t - w, warp) + s - v;
}

// The counts refs[first .. first + kPerThread) of a thread; pages past the pool count as `pad`.
__device__ __forceinline__ void load_refs(const int32_t* refs, int num_pages, long first, int pad, int (&r)[kPerThread]) {
    if (first + kPerThread <= num_pages) {
#pragma unroll
        for (int i = 0; i < kPerThread / 4; ++i) {
            const int4 x = reinterpret_cast<const int4*>(refs + first)[i];
            r[4 * i] = x.x; r[4 * i + 1] = x.y; r[4 * i + 2] = x.z; r[4 * i + 3] = x.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) r[i] = first + i < num_pages ? refs[first + i] : pad;
    }
}

// The `need` lowest pages without a reference, ascending, into `list` (global).  Returns whether there are as
// many.  `r`: the counts of this thread's first kPerThread pages, which the caller has asked for ahead of its
// own chain of loads.  All threads of the block; ends with the list visible to the block.
__device__ bool lowest_free(const int32_t* refs, int num_pages, int need, int32_t* list, int* warp_sums, int (&r)[kPerThread]) {
    int found = 0;
    for (long base = 0; base < num_pages && found < need; base += (int)blockDim.x * kPerThread) {
        const long first = base + (long)threadIdx.x * kPerThread;
        if (base > 0) load_refs(refs, num_pages, first, 1, r);
        int n = 0;
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) n += r[i] == 0;
        int total;
        int at = found + block_scan(n, warp_sums, &total);
#pragma unroll
        for (int i = 0; i < kPerThread; ++i)
            if (r[i] == 0) { if (at < need) list[at] = (int)first + i; ++at; }
        found += total;
    }
    __syncthreads();
    return found >= need;
}

// In the word behind the others' errors, which take the lowest code: too few pages must not hide a wait that ran out.
__device__ __forceinline__ void raise_pages(int32_t* status) { status[1] = TTS_ERR_DEVICE_PAGES; }

__device__ __forceinline__ bool page_ok(int page, int num_pages) { return page >= 0 && page < num_pages; }

// One reference less; false, and the counts as they were, for a page outside the pool or one that nothing refers to.
__device__ __forceinline__ bool give_back(int32_t* refs, int page, int num_pages) {
    if (page >= num_pages) return false;
    if (atomicSub(refs + page, 1) > 0) return true;
    atomicAdd(refs + page, 1);
    return false;
}

// One 4 KiB tile by one warp.
__device__ __forceinline__ void copy_tile(const uint4* src, uint4* dst, int lane) {
    uint4 x[kTileChunks];
#pragma unroll
    for (int i = 0; i < kTileChunks; ++i) x[i] = __ldcs(src + i * 32 + lane);
#pragma unroll
    for (int i = 0; i < kTileChunks; ++i) __stcs(dst + i * 32 + lane, x[i]);
}

// Copies list entry k (src[k] -> dst[k]) in all pools, for k < n; a negative page on either side is skipped.
__device__ void copy_pages(const PagePools& pools, const int32_t* src, const int32_t* dst, int n, int Hkv, int num_pages,
                           int32_t* status, int worker, int n_workers) {
    const int lane = threadIdx.x & 31;
    const int per_page = 2 * pools.n_layers * Hkv;      // tiles of one page: (K or V, layer, head)
    const long total = (long)n * per_page;
    for (long w = worker; w < total; w += n_workers) {
        const int k = (int)(w / per_page), rest = (int)(w - (long)k * per_page);
        const int pool = rest / Hkv, h = rest - pool * Hkv;
        const int s = src[k], d = dst[k];
        if (s < 0 || d < 0 || s == d) continue;
        if (s >= num_pages || d >= num_pages) { if (lane == 0) atomicMin(status, (int)TTS_ERR_DEVICE_BOUNDS); continue; }
        char* base = static_cast<char*>(pools.p[pool]);
        copy_tile(reinterpret_cast<const uint4*>(base + ((size_t)s * Hkv + h) * kTileBytes),
                  reinterpret_cast<uint4*>(base + ((size_t)d * Hkv + h) * kTileBytes), lane);
    }
}

__global__ void __launch_bounds__(kCopyThreads)
copy_pages_kernel(const __grid_constant__ PagePools pools, const int32_t* src, const int32_t* dst, int n, int Hkv, int num_pages, int32_t* status) {
    grid_dependency_wait();
    grid_launch_dependents();
    copy_pages(pools, src, dst, n, Hkv, num_pages, status, (blockIdx.x * kCopyThreads + threadIdx.x) >> 5, gridDim.x * (kCopyThreads / 32));
}

// ------------------------------------------------------------------------------------------------ fork
// Block 0 decides, the other blocks carry the counts over into new_refs.  Per child: its parent (or -1),
// how many leading entries it shares, and the page that takes the copy of the parent's part-filled one.
__global__ void __launch_bounds__(kMaxScanThreads)
fork_plan_kernel(const int32_t* table, int max_blocks, int prefix_len, const int32_t* lens, int n_branches,
                 const int32_t* parents, int n_children, const int32_t* refs, int32_t* new_refs, int num_pages, PageWork wk, int32_t* status) {
    grid_dependency_wait();
    grid_launch_dependents();
    if (blockIdx.x > 0) {
        if (new_refs != refs)
            for (long i = (blockIdx.x - 1) * (long)blockDim.x + threadIdx.x; i < num_pages; i += (gridDim.x - 1) * (long)blockDim.x) new_refs[i] = refs[i];
        return;
    }
    __shared__ int first[kMaxBranches];                 // lowest child of each parent
    __shared__ int sums[32];
    const int c = threadIdx.x;
    int free_refs[kPerThread];
    load_refs(refs, num_pages, (long)c * kPerThread, 1, free_refs);
    for (int i = c; i < n_branches; i += (int)blockDim.x) first[i] = 0x7fffffff;
    __syncthreads();
    int p = -1, len = 0;
    if (c < n_children) {
        p = parents[c];
        if (p < -1 || p >= n_branches) { atomicMin(status, (int)TTS_ERR_DEVICE_BOUNDS); p = -1; }
        if (p >= 0) {
            len = lens[p];
            if (len < 0 || (long)prefix_len + len > (long)max_blocks * kPage) {
                atomicMin(status, (int)TTS_ERR_DEVICE_BOUNDS);
                atomicMin(&first[p], c);                // an empty row for the child, but the parent's pages are not given back
                p = -1; len = 0;
            }
        }
        if (p >= 0) atomicMin(&first[p], c);
    }
    __syncthreads();
    const int tokens = prefix_len + len, full = tokens / kPage;
    const bool is_first = p >= 0 && first[p] == c;
    int src = -1;
    if (p >= 0 && !is_first && tokens % kPage != 0) {
        src = table[(size_t)p * max_blocks + full];
        if (!page_ok(src, num_pages)) { atomicMin(status, (int)TTS_ERR_DEVICE_BOUNDS); src = -1; }
    }
    int need;
    const int rank = block_scan((int)(src >= 0), sums, &need);
    const bool ok = lowest_free(refs, num_pages, need, wk.list_dst, sums, free_refs);
    if (c == 0) {
        wk.head[0] = ok ? need : 0;
        wk.head[1] = ok;
        if (!ok) raise_pages(status);
    }
    if (!ok) return;
    if (c < n_children) {
        wk.child[c] = make_int4(p, p < 0 ? 0 : is_first ? max_blocks : full, src >= 0 ? wk.list_dst[rank] : -1, len);
        if (src >= 0) wk.list_src[rank] = src;
    }
    for (int i = c; i < n_branches; i += (int)blockDim.x) wk.childless[i] = first[i] == 0x7fffffff;
}

// Blocks [0, n_children): the children's table rows; the next n_branches: references of branches without a
// child are dropped; the rest copy pages.
__global__ void __launch_bounds__(kCopyThreads)
fork_kernel(const __grid_constant__ PagePools pools, const int32_t* table, int max_blocks, int n_branches, int n_children,
            int32_t* new_table, int32_t* new_lens, int32_t* new_refs, int Hkv, int num_pages, PageWork wk, int32_t* status) {
    grid_dependency_wait();
    grid_launch_dependents();
    if (!wk.head[1]) return;
    const int blk = blockIdx.x;
    if (blk < n_children) {
        const int4 ch = wk.child[blk];
        const bool shares = ch.y < max_blocks;          // not the first child: what it keeps has one more reference
        for (int i = threadIdx.x; i < max_blocks; i += kCopyThreads) {
            int e = -1;
            if (i < ch.y) {
                e = table[(size_t)ch.x * max_blocks + i];
                // (a page whose entries are counted has one reference at all times, the first child's)
                if (e >= num_pages || (e >= 0 && __ldcg(new_refs + e) <= 0)) { atomicMin(status, (int)TTS_ERR_DEVICE_BOUNDS); e = -1; }
                e = e < 0 ? -1 : e;
                if (shares && e >= 0) atomicAdd(new_refs + e, 1);
            } else if (i == ch.y && ch.z >= 0) {
                e = ch.z;
                new_refs[e] = 1;
            }
            new_table[(size_t)blk * max_blocks + i] = e;
        }
        if (threadIdx.x == 0) new_lens[blk] = ch.w;
    } else if (blk < n_children + n_branches) {
        const int b = blk - n_children;
        if (!wk.childless[b]) return;
        for (int i = threadIdx.x; i < max_blocks; i += kCopyThreads) {
            const int e = table[(size_t)b * max_blocks + i];
            if (e >= 0 && !give_back(new_refs, e, num_pages)) atomicMin(status, (int)TTS_ERR_DEVICE_BOUNDS);
        }
    } else {
        const int blk0 = n_children + n_branches;
        copy_pages(pools, wk.list_src, wk.list_dst, wk.head[0], Hkv, num_pages, status,
                   ((blk - blk0) * kCopyThreads + threadIdx.x) >> 5, (gridDim.x - blk0) * (kCopyThreads / 32));
    }
}

// ------------------------------------------------------------------------------------------------ grow
// One CTA, one thread per branch: which entries of its row lack a page, then pages in that order.  A row that lacks
// one in front of its new tokens (the prefix's, after tts_kv_free or a fork from -1) is refused: the tokens
// would stand behind a hole.  That look is the warps', a row each, 256 entries in flight,
// the first of them before the row's length is known (16 rows of 240 entries: 2.0 us without, 2.7 with it; 64 rows 2.7 and 5.7;
// units of 32 entries that any warp takes, 3.9 and 7.6).
__global__ void __launch_bounds__(kMaxScanThreads)
grow_kernel(int32_t* table, int max_blocks, int prefix_len, int32_t* lens, const int32_t* n_new, int n_branches, int32_t* refs,
            int num_pages, PageWork wk, int32_t* status) {
    grid_dependency_wait();
    grid_launch_dependents();
    __shared__ int sums[32];
    __shared__ long long wants[32];
    __shared__ int held[kMaxBranches];                  // entries of each growing row that have to hold a page
    const int b = threadIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int free_refs[kPerThread], e[8];
    load_refs(refs, num_pages, (long)b * kPerThread, 1, free_refs);
    auto entries = [&](int r, int i0, int n, int (&to)[8]) {
#pragma unroll
        for (int k = 0; k < 8; ++k) to[k] = i0 + 32 * k < n ? table[(size_t)r * max_blocks + i0 + 32 * k] : 0;
    };
    entries(warp, lane, warp < n_branches ? max_blocks : 0, e);
    bool bad = false;
    int lo = 0, hi = 0, more = 0, len = 0;
    if (b < n_branches) {
        more = n_new[b]; len = lens[b];
        const long after = (long)prefix_len + len + more;
        bad = more < 0 || len < 0 || after > (long)max_blocks * kPage;
        if (!bad && more > 0) { lo = ceil_div(prefix_len + len, kPage); hi = ceil_div((int)after, kPage); }
        held[b] = lo;
    }
    __syncthreads();
    int32_t* row = table + (size_t)b * max_blocks;
    const int next = lo < hi ? row[lo] : 0;             // (asked for ahead of the look)
    for (int r = warp; r < n_branches; r += (int)blockDim.x >> 5) {
        const int n = held[r];
        for (int i0 = lane; i0 < n; i0 += 8 * 32) {
            if (r != warp || i0 != lane) entries(r, i0, n, e);
#pragma unroll
            for (int k = 0; k < 8; ++k) bad |= i0 + 32 * k < n && !page_ok(e[k], num_pages);
        }
    }
    // A branch that lacks more pages than there are is refused whatever the others ask for, so the count may stop there;
    // 1024 such counts and rows of 2^26 entries add up to more than 32 bits hold.
    constexpr long long kBad = 1ll << 50;               // above any sum of counts
    long long want = 0, need;
    for (int i = lo; i < hi && want <= num_pages; ++i) {
        const int page = i == lo ? next : row[i];
        if (page < 0) ++want;
        else bad |= page >= num_pages || refs[page] <= 0;
    }
    long long at = block_scan(bad ? kBad : want, wants, &need);
    if (need >= kBad) { if (b == 0) atomicMin(status, (int)TTS_ERR_DEVICE_BOUNDS); return; }
    if (need > num_pages || !lowest_free(refs, num_pages, (int)need, wk.list_dst, sums, free_refs)) { if (b == 0) raise_pages(status); return; }
    for (int i = lo; i < hi; ++i)
        if (row[i] < 0) {
            const int page = wk.list_dst[at++];
            row[i] = page;
            refs[page] = 1;
        }
    if (b < n_branches && more > 0) lens[b] = len + more;
}

// One block per branch.
__global__ void __launch_bounds__(kCopyThreads)
free_kernel(int32_t* table, int max_blocks, int32_t* lens, const int32_t* freed, int32_t* refs, int num_pages, int32_t* status) {
    grid_dependency_wait();
    grid_launch_dependents();
    const int b = blockIdx.x;
    if (!freed[b]) return;
    for (int i = threadIdx.x; i < max_blocks; i += kCopyThreads) {
        const int e = table[(size_t)b * max_blocks + i];
        table[(size_t)b * max_blocks + i] = -1;
        if (e < 0) continue;
        if (!give_back(refs, e, num_pages)) atomicMin(status, (int)TTS_ERR_DEVICE_BOUNDS);
    }
    if (threadIdx.x == 0) lens[b] = 0;
}

// --------------------------------------------------------------------------------------------- compact
// One CTA.  U = pages in use; holes = free pages below U, movers = used pages from U on: as many of either,
// and the k-th mover goes to the k-th hole.
__global__ void __launch_bounds__(kMaxScanThreads)
compact_plan_kernel(const int32_t* refs, int32_t* new_refs, int num_pages, int32_t* page_map, int32_t* n_used, PageWork wk) {
    grid_dependency_wait();
    grid_launch_dependents();
    __shared__ int sums[32];
    int mine = 0, used, r[kPerThread];
    for (long base = (long)threadIdx.x * kPerThread; base < num_pages; base += (int)blockDim.x * kPerThread) {
        load_refs(refs, num_pages, base, 0, r);
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) mine += r[i] > 0;
    }
    block_scan(mine, sums, &used);
    int holes = 0, movers = 0;
    for (long base = 0; base < num_pages; base += (int)blockDim.x * kPerThread) {
        const long first = base + (long)threadIdx.x * kPerThread;
        if (num_pages > (int)blockDim.x * kPerThread) load_refs(refs, num_pages, first, 0, r);
        else if (first >= num_pages) { for (int i = 0; i < kPerThread; ++i) r[i] = 0; }      // (else they are still at hand)
        int hole = 0, mover = 0;
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
            const long p = first + i;
            hole += p < used && r[i] <= 0;
            mover += p >= used && r[i] > 0;
        }
        int total_h, total_m;
        int at_h = holes + block_scan(hole, sums, &total_h);
        int at_m = movers + block_scan(mover, sums, &total_m);
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
            const long p = first + i;
            if (p < used && r[i] <= 0) wk.list_dst[at_h++] = (int)p;
            if (p >= used && r[i] > 0) wk.list_src[at_m++] = (int)p;
        }
        holes += total_h; movers += total_m;
    }
    // the map and the counts of the pages that stay, in coalesced steps of four pages per thread; movers follow
    for (long p = (long)threadIdx.x * 4; p < num_pages; p += (int)blockDim.x * 4) {
        if (p + 4 <= num_pages) {
            const int4 c = *reinterpret_cast<const int4*>(refs + p);
            const int v[4] = {c.x, c.y, c.z, c.w};
            int m[4], k[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) { const bool stays = v[i] > 0 && p + i < used; m[i] = stays ? (int)p + i : -1; k[i] = stays ? v[i] : 0; }
            *reinterpret_cast<int4*>(page_map + p) = make_int4(m[0], m[1], m[2], m[3]);
            if (new_refs != refs) *reinterpret_cast<int4*>(new_refs + p) = make_int4(k[0], k[1], k[2], k[3]);
        } else {
            for (long i = p; i < num_pages; ++i) {
                const int v = refs[i];
                const bool stays = v > 0 && i < used;
                page_map[i] = stays ? (int)i : -1;
                if (new_refs != refs) new_refs[i] = stays ? v : 0;
            }
        }
    }
    __syncthreads();
    for (int k = threadIdx.x; k < movers; k += (int)blockDim.x) {
        const int s = wk.list_src[k], d = wk.list_dst[k];
        page_map[s] = d;
        new_refs[d] = refs[s];
        if (new_refs == refs) new_refs[s] = 0;
    }
    if (threadIdx.x == 0) { wk.head[0] = movers; *n_used = used; }
}

// Blocks [0, n_branches): table rows through the map; the rest copy pages.
__global__ void __launch_bounds__(kCopyThreads)
compact_kernel(const __grid_constant__ PagePools pools, const int32_t* table, int max_blocks, int n_branches, int32_t* new_table,
               const int32_t* page_map, int Hkv, int num_pages, PageWork wk, int32_t* status) {
    grid_dependency_wait();
    grid_launch_dependents();
    if ((int)blockIdx.x < n_branches) {
        for (int i = threadIdx.x; i < max_blocks; i += kCopyThreads) {
            const size_t at = (size_t)blockIdx.x * max_blocks + i;
            const int e = table[at];
            int to = -1;
            if (e >= 0) {
                to = e < num_pages ? page_map[e] : -1;
                if (to < 0) atomicMin(status, (int)TTS_ERR_DEVICE_BOUNDS);    // an entry that the counts do not know
            }
            new_table[at] = to;
        }
    } else {
        copy_pages(pools, wk.list_src, wk.list_dst, wk.head[0], Hkv, num_pages, status,
                   ((blockIdx.x - n_branches) * kCopyThreads + threadIdx.x) >> 5, (gridDim.x - n_branches) * (kCopyThreads / 32));
    }
}

// Blocks for n copies: one warp per tile, at most 8 blocks of 8 warps per SM (the register file's worth).
int copy_blocks(long n, const PagePools& pools, int Hkv, int n_sms) {
    const long tiles = n * 2 * pools.n_layers * Hkv, blocks = (tiles + kCopyThreads / 32 - 1) / (kCopyThreads / 32);
    return (int)(blocks < 8l * n_sms ? blocks : 8l * n_sms);
}

}  // namespace

// Threads of a plan: one for each branch and for every kPerThread pages, and no more, since every warp is issue time for
// the others (a fork of 16 branches and room for four rows, 64 layers: 14.7 us, 16.3 with 1024 threads each).
static int scan_threads(int n_branches, int num_pages) {
    return std::min(kMaxScanThreads, std::max(ceil_div(n_branches, 32), ceil_div(num_pages, 32 * kPerThread)) * 32);
}

cudaError_t launch_copy_pages(const PagePools& pools, const int32_t* src, const int32_t* dst, int n, int Hkv, int num_pages, int n_sms,
                              int32_t* status, cudaStream_t st) {
    return launch_dependent(copy_pages_kernel, copy_blocks(n, pools, Hkv, n_sms), kCopyThreads, 0, st, pools, src, dst, n, Hkv, num_pages, status);
}

cudaError_t launch_fork(const PagePools& pools, const int32_t* table, int max_blocks, int prefix_len, const int32_t* lens, int n_branches,
                        const int32_t* parents, int n_children, const int32_t* refs, int32_t* new_table, int32_t* new_lens, int32_t* new_refs,
                        int Hkv, int num_pages, int n_sms, const PageWork& wk, int32_t* status, cudaStream_t st) {
    const int threads = scan_threads(n_children, num_pages), carriers = new_refs == refs ? 0 : ceil_div(num_pages, 8 * threads);
    cudaError_t e = launch_dependent(fork_plan_kernel, 1 + carriers, threads, 0, st, table, max_blocks, prefix_len, lens, n_branches, parents,
                                     n_children, refs, new_refs, num_pages, wk, status);
    if (e != cudaSuccess) return e;
    return launch_dependent(fork_kernel, n_children + n_branches + copy_blocks(n_children, pools, Hkv, n_sms), kCopyThreads, 0, st, pools, table,
                            max_blocks, n_branches, n_children, new_table, new_lens, new_refs, Hkv, num_pages, wk, status);
}

cudaError_t launch_grow(int32_t* table, int max_blocks, int prefix_len, int32_t* lens, const int32_t* n_new, int n_branches, int32_t* refs,
                        int num_pages, const PageWork& wk, int32_t* status, cudaStream_t st) {
    const int threads = std::max(scan_threads(n_branches, num_pages), 32 * std::min(32, n_branches));       // and a warp for each row
    return launch_dependent(grow_kernel, 1, threads, 0, st, table, max_blocks, prefix_len, lens, n_new, n_branches, refs, num_pages, wk, status);
}

cudaError_t launch_free(int32_t* table, int max_blocks, int32_t* lens, const int32_t* freed, int n_branches, int32_t* refs, int num_pages,
                        int32_t* status, cudaStream_t st) {
    return launch_dependent(free_kernel, n_branches, kCopyThreads, 0, st, table, max_blocks, lens, freed, refs, num_pages, status);
}

cudaError_t launch_compact(const PagePools& pools, const int32_t* table, int max_blocks, int n_branches, const int32_t* refs, int32_t* new_table,
                           int32_t* new_refs, int32_t* page_map, int32_t* n_used, int Hkv, int num_pages, int n_sms, const PageWork& wk,
                           int32_t* status, cudaStream_t st) {
    cudaError_t e = launch_dependent(compact_plan_kernel, 1, scan_threads(0, num_pages), 0, st, refs, new_refs, num_pages, page_map, n_used, wk);
    if (e != cudaSuccess) return e;
    return launch_dependent(compact_kernel, n_branches + copy_blocks(num_pages / 2 + 1, pools, Hkv, n_sms), kCopyThreads, 0, st, pools, table, max_blocks,
                            n_branches, new_table, page_map, Hkv, num_pages, wk, status);
}

}  // namespace tts
