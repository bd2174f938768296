// The schedule of one chunk-attention call, worked out on the device by one CTA: entries, how their KV
// tiles are cut into pieces, and the order in which the pieces are handed out.
//
// How long a piece may be is chosen so that the estimated time of the call is smallest: with C KV tiles per
// piece at most, P pieces in all and an overhead of kOverhead tiles per piece, that is C + overhead where
// every piece has a CTA of its own, and (all tiles + P x overhead) / CTAs + half a piece where they queue.
// 32 values of C are tried, a warp each.  Pieces go out longest first within a KV head, and one KV head after
// the other, so that CTAs that run at the same time read the same keys.
#include "chunk_attn.cuh"
#include "launch.cuh"

namespace tts {

namespace {

constexpr int kThreads = 1024;
constexpr int kBuckets = 1024;                        // pieces are ordered by their entry's KV tiles
constexpr float kOverhead = 1.5f, kSplitOverhead = 2.5f;   // in KV tiles; the second: of a piece that leaves a partial result
// into how many pieces the longest entry is cut
__constant__ int kCuts[32] = {1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 12, 14, 16, 18, 20, 24, 28, 32, 37, 42, 49, 56, 64, 74, 86, 99, 114, 132, 148, 170, 222, 296};

__device__ int block_scan(int v, int* sums, int* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int n = __shfl_up_sync(0xffffffffu, s, o); if (lane >= o) s += n; }
    __syncthreads();
    if (lane == 31) sums[warp] = s;
    __syncthreads();
    if (warp == 0) {
        const int w = sums[lane];
        int t = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const int n = __shfl_up_sync(0xffffffffu, t, o); if (lane >= o) t += n; }
        sums[lane] = t - w;
        if (lane == 31) sums[32] = t;
    }
    __syncthreads();
    *total = sums[32];
    return sums[warp] + s - v;
}

__global__ void __launch_bounds__(kThreads)
chunk_plan_kernel(const ChunkParams p) {
    grid_dependency_wait();
    grid_launch_dependents();
    __shared__ int first[kMaxBranches + 1];            // first entry of each branch
    __shared__ int bucket[kBuckets];
    __shared__ int sums[33];
    __shared__ float est[32];
    __shared__ int bad, longest, shortest, rows_used;
    __shared__ unsigned long long tiles_sum;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) { bad = 0; longest = 0; shortest = 0x7fffffff; rows_used = 0; tiles_sum = 0; }
    for (int i = tid; i < kBuckets; i += kThreads) bucket[i] = 0;
    __syncthreads();

    // entries of each branch; a call whose row starts or lengths make no sense computes nothing
    int n_mine = 0;
    if (tid < p.n_branches) {
        const int lo = p.row_start[tid], hi = p.row_start[tid + 1], L = p.branch_lens[tid];
        if (lo < 0 || hi < lo || hi > p.total_rows || L < 0 || (long)p.prefix_len + L > (long)p.max_blocks * kPage) bad = 1;
        else n_mine = ceil_div(hi - lo, 2 * p.T);
    }
    __syncthreads();
    if (bad) n_mine = 0;
    int n_entries;
    const int at = block_scan(n_mine, sums, &n_entries);
    if (tid < p.n_branches) first[tid] = at;
    if (tid == 0) {
        first[p.n_branches] = n_entries;
        if (bad) atomicMin(p.status, (int)TTS_ERR_DEVICE_BOUNDS);
    }
    __syncthreads();

    struct Entry { int b, row0, n_tok, limit0, keys, tiles, once; };
    auto entry = [&](int e) {
        int lo = 0, hi = p.n_branches - 1;             // the last branch whose first entry is <= e
        while (lo < hi) { const int mid = (lo + hi + 1) >> 1; if (first[mid] <= e) lo = mid; else hi = mid - 1; }
        const int start = p.row_start[lo], c = p.row_start[lo + 1] - start, tok0 = (e - first[lo]) * 2 * p.T;
        Entry r;
        r.b = lo; r.row0 = start + tok0; r.n_tok = min(2 * p.T, c - tok0);
        r.keys = p.prefix_len + p.branch_lens[lo];
        r.limit0 = r.keys - c + tok0 + 1;
        r.tiles = ceil_div(min(r.keys, max(0, r.limit0 + r.n_tok - 1)), kChunkTile);
        r.once = c <= 2 * p.T;
        return r;
    };
    {
        int mx = 0, mn = 0x7fffffff;
        long sum = 0;
        for (int e = tid; e < n_entries; e += kThreads) {
            const Entry r = entry(e);
            const int n = r.tiles;
            p.entry_tiles[e] = make_int2(n, r.n_tok);
            mx = max(mx, n); mn = min(mn, n); sum += n;
        }
        if (tid < n_entries) { atomicMax(&longest, mx); atomicMin(&shortest, mn); atomicAdd(&tiles_sum, (unsigned long long)sum); }
        for (long i = tid; i < 2l * n_entries * p.Hkv; i += kThreads) p.arrived[i] = 0;
    }
    __syncthreads();

    // the length of a piece
    {
        const int C = max(1, ceil_div(longest, kCuts[warp]));
        long pieces = 0, rows = 0;
        for (int e = lane; e < n_entries; e += 32) {
            const int2 t = p.entry_tiles[e];
            const int k = max(1, ceil_div(t.x, C));
            pieces += k;
            if (k > 1) rows += (long)k * t.y * p.G;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) { pieces += __shfl_xor_sync(0xffffffffu, pieces, o); rows += __shfl_xor_sync(0xffffffffu, rows, o); }
        if (lane == 0) {
            const float over = kOverhead + (C < longest ? kSplitOverhead : 0.f);
            const float P = (float)pieces * p.Hkv, avg = ((float)tiles_sum * p.Hkv + P * over) / p.grid;
            float t;
            if (P <= p.grid) t = C + over;
            else if (longest == shortest) t = ceilf(P / p.grid) * (C + over);
            else t = avg + 0.5f * (C + over);
            const bool fits = warp == 0 || (pieces <= p.max_pieces && rows * p.Hkv <= p.part_rows);
            est[warp] = fits ? t : 3.0e38f;
        }
    }
    __syncthreads();
    int best = 0;
    for (int i = 1; i < 32; ++i) if (est[i] < est[best]) best = i;
    const int C = max(1, ceil_div(longest, kCuts[best]));

    // places: longest entries first
    for (int e = tid; e < n_entries; e += kThreads)
        atomicAdd(&bucket[kBuckets - 1 - min(p.entry_tiles[e].x, kBuckets - 1)], max(1, ceil_div(p.entry_tiles[e].x, C)));
    __syncthreads();
    int total;
    const int place = block_scan(bucket[tid], sums, &total);
    bucket[tid] = place;
    __syncthreads();
    for (int e = tid; e < n_entries; e += kThreads) {
        const Entry r = entry(e);
        const int k = max(1, ceil_div(r.tiles, C));
        const int at_piece = atomicAdd(&bucket[kBuckets - 1 - min(r.tiles, kBuckets - 1)], k);
        const int part_row = k > 1 ? atomicAdd(&rows_used, k * r.n_tok * p.G) : 0;
        for (int i = 0; i < k; ++i) {
            ChunkPiece x;
            x.branch = r.b; x.row0 = r.row0; x.n_tok = r.n_tok; x.limit0 = r.limit0; x.keys = r.keys;
            x.tile_begin = (int)((long)r.tiles * i / k); x.tile_end = (int)((long)r.tiles * (i + 1) / k);
            x.parts = k; x.part = i; x.part_row = part_row; x.entry = e; x.once = r.once;
            p.pieces[at_piece + i] = x;
        }
    }
    __syncthreads();
    if (tid == 0) { p.head->pieces_per_head = total; p.head->next = p.grid; p.head->rows_per_head = rows_used; p.head->entries = n_entries; }
}
static_assert(kBuckets == kThreads, "one bucket per thread in the scan");

}  // namespace

cudaError_t launch_chunk_plan(const ChunkParams& p, cudaStream_t st) {
    return launch_dependent(chunk_plan_kernel, 1, kThreads, 0, st, p);
}

}  // namespace tts
