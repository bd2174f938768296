// The schedule of one chunk-attention call, worked out on the device by one CTA: entries, how their KV
// tiles are cut into pieces, and the order in which the pieces are handed out.
//
// The unit of cost is one KV tile of a narrow entry; a wide entry's tile costs two (256 query rows instead of
// 128).  Entries are handed out in four classes of cost, the costliest first, and within a class branch by
// branch, all KV heads of a piece one after the other, so that CTAs that run at the same time read neighbouring
// keys.  The first entries, with which every CTA starts, stay whole; later ones are cut so that a piece costs
// what is left for each CTA when its turn comes (chunk_cuts), down to the call's bound (chunk_bound), and all
// CTAs end within about one small piece of each other.  With whole entries alone the last CTA ended 8 % behind
// the mean at 8192 new tokens over 24576 (1280 entries for 148 CTAs), 30 % behind it with 64 single tokens over
// 1 k to 8 k keys.  Everything here is a function of the lengths alone: the cuts, and with them the results, do
// not depend on timing.
//
// The kernel is latency: its code runs once, cold, and every warp more is issue time for the others, so that it has no
// more threads than the call may need (the attention of 24 prompts, some 360 entries: 56.1 us with 1024 threads, 55.0 with 192).  Sorting the entries and trying 32 bounds took 15 us where
// this takes 7, for no better balance.
#include "chunk_attn.cuh"
#include "launch.cuh"

#include <algorithm>

namespace tts {

namespace {

constexpr int kMaxThreads = 1024;
constexpr int kPer = 2;                               // entries per thread
constexpr int kMaxCut = kMaxThreads * kPer;             // calls with more entries do not cut them: 14 and more per CTA even
                                                      // themselves out, if they are alike (a long branch behind short ones ends alone)

struct Scan { unsigned long long warp[32]; };

__device__ unsigned long long warp_scan(unsigned long long v, int lane) {              // inclusive
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const unsigned long long n = __shfl_up_sync(0xffffffffu, v, o); if (lane >= o) v += n; }
    return v;
}
// Exclusive, over the block.  Every warp adds up the warps' sums for itself: one barrier.  A scan has an `sc` of its own.
__device__ unsigned long long block_scan(unsigned long long v, Scan& sc, unsigned long long* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const unsigned long long s = warp_scan(v, lane);
    if (lane == 31) sc.warp[warp] = s;
    __syncthreads();
    const unsigned long long w = lane < (int)(blockDim.x >> 5) ? sc.warp[lane] : 0, t = warp_scan(w, lane);
    *total = __shfl_sync(0xffffffffu, t, 31);
    return __shfl_sync(0xffffffffu, t - w, warp) + s - v;
}

struct Branches {
    int first[kMaxBranches + 1];                       // first entry of each branch
    int start[kMaxBranches + 1], keys[kMaxBranches];
};

__device__ ChunkEntry entry_of(const ChunkParams& p, const Branches& br, int e) {
    int lo = 0, hi = p.n_branches - 1;                 // the last branch whose first entry is at or before this one
    while (lo < hi) { const int mid = (lo + hi + 1) >> 1; if (br.first[mid] <= e) lo = mid; else hi = mid - 1; }
    return chunk_entry(p.T, lo, br.first[lo + 1] - 1 - e, br.start[lo], br.start[lo + 1] - br.start[lo], br.keys[lo]);
}

__device__ void write_pieces(const ChunkParams& p, const ChunkEntry& r, int e, int k, int at, int part_row) {
#pragma unroll 1
    for (int i = 0; i < k; ++i) {
        const ChunkPiece x = chunk_piece(r, e, i, k, part_row);
        const int4* src = reinterpret_cast<const int4*>(&x);
        int4* dst = reinterpret_cast<int4*>(p.pieces + at + i);
        dst[0] = src[0]; dst[1] = src[1]; dst[2] = src[2];
    }
}

__global__ void __launch_bounds__(kMaxThreads)
chunk_plan_kernel(const ChunkParams p) {
    grid_dependency_wait();
    grid_launch_dependents();
    __shared__ Branches br;
    __shared__ Scan sc[4];
    __shared__ unsigned short order[kMaxCut];
    __shared__ int largest;
    const int tid = threadIdx.x;
    if (tid == 0) largest = 0;

    // entries of each branch
    int n_mine = 0;
    bool bad = false;
    if (tid < p.n_branches) {
        const int lo = p.row_start[tid], hi = p.row_start[tid + 1], L = p.branch_lens[tid];
        br.start[tid] = lo; br.keys[tid] = p.prefix_len + L;
        if (tid == p.n_branches - 1) br.start[p.n_branches] = hi;
        bad = !chunk_branch_ok(p, lo, hi, L);
        n_mine = ceil_div(hi - lo, 2 * p.T);
    }
    bad = __syncthreads_or(bad);                       // then nothing is computed
    unsigned long long sum;
    const int at_branch = (int)block_scan(bad ? 0 : n_mine, sc[0], &sum);
    const int n = (int)sum;
    if (tid < p.n_branches) br.first[tid] = at_branch;
    if (tid == 0) {
        br.first[p.n_branches] = n;
        if (bad) atomicMin(p.status, (int)TTS_ERR_DEVICE_BOUNDS);
    }
    __syncthreads();
    if (n > kMaxCut) {
#pragma unroll 1
        for (int e = tid; e < n; e += blockDim.x) write_pieces(p, entry_of(p, br, e), e, 1, e, 0);
        if (tid == 0) { p.head->pieces = n; p.head->part_rows = 0; }
        return;
    }

    // classes of cost: above three quarters of the largest, above a half, above a quarter, the rest
    int mine[kPer], most = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        mine[i] = kPer * tid + i < n ? chunk_cost(entry_of(p, br, kPer * tid + i), p.T) : -1;
        most = max(most, mine[i]);
    }
    most = __reduce_max_sync(0xffffffffu, most);
    if ((tid & 31) == 0) atomicMax(&largest, most);
    __syncthreads();
    unsigned long long in_class = 0;                   // 16 bits for each class
    int cls[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        cls[i] = 3 - min(3, (int)(4.f * mine[i] / (largest + 1)));
        if (mine[i] >= 0) in_class += 1ull << (16 * cls[i]);
    }
    unsigned long long at_class = block_scan(in_class, sc[1], &sum);
    at_class += (sum << 16) + (sum << 32) + (sum << 48);         // each class begins where those before it end
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (mine[i] >= 0) {
            order[at_class >> (16 * cls[i]) & 0xffffu] = (unsigned short)(kPer * tid + i);
            at_class += 1ull << (16 * cls[i]);
        }
    __syncthreads();

    ChunkEntry r[kPer];
    int e[kPer], cost[kPer] = {0, 0};
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (kPer * tid + i < n) {
            e[i] = order[kPer * tid + i];
            r[i] = entry_of(p, br, e[i]);
            cost[i] = chunk_cost(r[i], p.T);
        }
    const unsigned long long ahead = block_scan((unsigned)cost[0] + (unsigned)cost[1], sc[2], &sum);
    const float total = (float)sum, left[kPer] = {(float)(sum - ahead), (float)(sum - ahead - cost[0])};
    ChunkBound bound = chunk_bound(p, total, n, (float)largest);
    for (;;) {
        int k[kPer] = {0, 0};
        unsigned long long mine = 0;                   // pieces, and from bit 20 on partial-result rows
        int rows0 = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (kPer * tid + i < n) {
                k[i] = chunk_cuts(p, r[i], kPer * tid + i, left[i], total, bound);
                const int rows = k[i] > 1 ? k[i] * r[i].n_tok * p.G : 0;
                if (i == 0) rows0 = rows;
                mine += (unsigned)k[i] + ((unsigned long long)rows << 20);
            }
        const unsigned long long at = block_scan(mine, sc[3], &sum);
        const int pieces = (int)(sum & 0xfffffu);
        const long rows = (long)(sum >> 20);
        if (bound.narrow != kChunkNoBound && (pieces > p.max_pieces || rows * p.Hkv > p.part_rows)) {
            bound = chunk_coarser(bound);
            __syncthreads();                           // everyone has read the sums
            continue;
        }
        const int at0 = (int)(at & 0xfffffu), row0 = (int)(at >> 20);
        if (k[0] > 0) write_pieces(p, r[0], e[0], k[0], at0, row0);
        if (k[1] > 0) write_pieces(p, r[1], e[1], k[1], at0 + k[0], row0 + rows0);
        if (tid == 0) { p.head->pieces = pieces; p.head->part_rows = (int)rows; }
        break;
    }
}

}  // namespace

cudaError_t launch_chunk_plan(const ChunkParams& p, cudaStream_t st) {
    // a thread for each branch and one for every two entries that there may be
    const long entries = (long)p.total_rows / (2 * p.T) + p.n_branches;
    const long threads = entries > kMaxCut ? kMaxThreads : std::max((long)p.n_branches, (entries + kPer - 1) / kPer);
    return launch_dependent(chunk_plan_kernel, 1, (int)((threads + 31) / 32 * 32), 0, st, p);
}

}  // namespace tts
