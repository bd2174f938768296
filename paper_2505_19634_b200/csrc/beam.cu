// Beam search: the best continuations of all beams of a question, and their states in the new order.
//
//   score(r, x) = beam_score[r] + logit[r][x] - log sum_y exp(logit[r][y]),   ties to the lowest (beam, token)
//
// Within a row the score rises with the logit, so a question's n best are among the n largest logits of each row: a first
// kernel reads every logit once and leaves, per row, the logarithm of the sum and the n largest; a second one, a block per
// question, puts the rows together.
//
// Rows: bound by HBM (or, for few rows, by latency).  A row is one cluster of 1 to 8 CTAs, each with a contiguous part of it in
// chunks of 8192 logits that stay in registers: 32 for each thread, whose largest serves both the running sum of exponentials
// and the search.  A thread looks at its 32 one by one only if its largest passes the threshold, a lower bound of the n-th best
// logit so far; those that pass go to a list in shared memory.  The threshold is a logit and a token number in one 64-bit
// word, so that no two entries are equal and the lists stay short whatever the logits are (all equal, rising, ..).
// Exponentials are fp32; 32 of them are summed in fp32, everything beyond in 64 bits, as are the scores: which of two
// candidates is better does not hang on a rounding to 32 bits.
#include <cooperative_groups.h>
#include <math.h>

#include <type_traits>

#include "beam.cuh"
#include "launch.cuh"

namespace tts {

namespace {

typedef unsigned long long u64;

constexpr int kThreads = 256;
constexpr int kPer = 32;                                            // logits of a thread per chunk
constexpr int kChunk = kThreads * kPer;
constexpr int kSlackThreads = 16;                                   // threads that may pass the threshold beyond n_select before it is raised
constexpr int kDirect = 512;                                        // entries that are ranked by comparing each with each

__host__ __device__ constexpr int per_chunk(int n) { return kPer * (n + kSlackThreads); }       // entries that a chunk adds at most
__host__ __device__ constexpr int capacity(int n) { return n + 2 * per_chunk(n); }

// Order-preserving map of fp32 to unsigned words; -infinity is the least number.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ u64 key_of(double x) {
    const u64 b = (u64)__double_as_longlong(x);
    return b >> 63 ? ~b : b | 1ull << 63;
}
__device__ __forceinline__ double value_of(u64 k) { return __longlong_as_double((long long)(k >> 63 ? k & ~(1ull << 63) : ~k)); }

__device__ __forceinline__ u64 entry(float x, int token) { return (u64)key_of(x) << 32 | (0xffffffffu - (uint32_t)token); }
constexpr u64 kLeast = (u64)(0x007fffffu + 1u) << 32;               // above every entry of -infinity

__device__ __forceinline__ float exp2_approx(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

struct RowShared {
    u64 maxima[kThreads];
    double sums[kThreads / 32];
    float tops[kThreads / 32];
    u64 threshold;
    int n;                                                          // entries of the list
    int count;                                                      // scratch of the pruning
    // what the cluster's first CTA reads
    double sum;
    float top;
    int n_best;
};

__device__ __forceinline__ u64 max64(u64 a, u64 b) { return a > b ? a : b; }

// Sorts the list into best[0 .. min(n, k)) (descending) and returns that number.  All threads; `list` has sh.n entries.
__device__ int prune(RowShared& sh, u64* list, u64* best, int k) {
    const int tid = threadIdx.x;
    int n = sh.n;
    if (n > kDirect) {
        // the k-th largest, bit by bit from the top (entries differ, so exactly k are at or above it)
        u64 t = 0;
        for (int bit = 63; bit >= 0; --bit) {
            const u64 trial = t | 1ull << bit;
            int c = 0;
            for (int i = tid; i < n; i += kThreads) c += list[i] >= trial;
            c = __reduce_add_sync(0xffffffffu, c);
            if (tid == 0) sh.count = 0;
            __syncthreads();
            if ((tid & 31) == 0 && c) atomicAdd(&sh.count, c);
            __syncthreads();
            if (sh.count >= k) t = trial;
            __syncthreads();
        }
        if (tid == 0) sh.count = 0;
        __syncthreads();
        for (int i = tid; i < n; i += kThreads)
            if (list[i] >= t) sh.maxima[atomicAdd(&sh.count, 1)] = list[i];       // (n_select <= kThreads of them)
        __syncthreads();
        n = sh.count;
        for (int i = tid; i < n; i += kThreads) list[i] = sh.maxima[i];
        __syncthreads();
    }
    for (int i = tid; i < n; i += kThreads) {
        const u64 mine = list[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += list[j] > mine;
        if (rank < k) best[rank] = mine;
    }
    __syncthreads();
    return min(n, k);
}

template <typename T, bool kAligned>
__global__ void __launch_bounds__(kThreads)
beam_rows_kernel(const __grid_constant__ BeamParams p) {
    extern __shared__ __align__(16) unsigned char smem[];
    RowShared& sh = *reinterpret_cast<RowShared*>(smem);
    u64* list = reinterpret_cast<u64*>(smem + (sizeof(RowShared) + 15) / 16 * 16);
    u64* best = list + capacity(p.n_select);
    namespace cg = cooperative_groups;
    const cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, row = blockIdx.y, k = p.n_select;
    const int rank = (int)cluster.block_rank(), ranks = (int)cluster.num_blocks();
    grid_dependency_wait();
    grid_launch_dependents();
    if (!isfinite(p.beam_scores[row]) || (p.finished && p.finished[row])) return;      // (the whole cluster)

    const T* x = static_cast<const T*>(p.logits) + (size_t)row * p.row_stride;
    const int begin = min(p.vocab, rank * p.per_cta), end = min(p.vocab, begin + p.per_cta);
    if (tid == 0) { sh.threshold = kLeast; sh.n = 0; }
    __syncthreads();

    constexpr int kVec = 16 / sizeof(T);                            // logits of a 16-byte load
    auto index = [&](int base, int i) { return kAligned ? base + (i / kVec) * (kThreads * kVec) + tid * kVec + i % kVec : base + i * kThreads + tid; };
    float top = -INFINITY;                                          // of this thread's logits so far
    double sum = 0.0;                                               // of exp(logit - top)
    for (int base = begin; base < end; base += kChunk) {
        float v[kPer];
        if constexpr (kAligned) {
#pragma unroll
            for (int c = 0; c < kPer / kVec; ++c) {
                const int at = index(base, c * kVec);
                if (at + kVec <= end) {
                    const uint4 w = *reinterpret_cast<const uint4*>(x + at);
                    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if constexpr (sizeof(T) == 2) { v[c * kVec + 2 * j] = __uint_as_float(u[j] << 16); v[c * kVec + 2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u); }
                        else v[c * kVec + j] = __uint_as_float(u[j]);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < kVec; ++j) v[c * kVec + j] = at + j < end ? (float)x[at + j] : -INFINITY;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i) v[i] = index(base, i) < end ? (float)x[index(base, i)] : -INFINITY;
        }
        float high = v[0];
#pragma unroll
        for (int i = 1; i < kPer; ++i) high = fmaxf(high, v[i]);
        if (high > top) {
            sum *= exp2_approx((top - high) * 1.4426950408889634f);
            top = high;
        }
        float part = 0.f;
        const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int i = 0; i < kPer; ++i) part += exp2_approx((v[i] - ref) * 1.4426950408889634f);
        sum += part;

        // ---- candidates
        u64 t = sh.threshold;
        bool pass = key_of(high) >= (uint32_t)(t >> 32);
        int passing = __syncthreads_count(pass);
        if (passing == 0) continue;
        auto largest = [&]() {                                      // this thread's largest entry, the lowest token of equal ones
            u64 e = 0;
#pragma unroll
            for (int i = kPer - 1; i >= 0; --i) if (v[i] == high) e = entry(v[i], index(base, i));
            return e;
        };
        if (passing > k + kSlackThreads) {
            // raise the threshold: the k-th largest of the maxima of 2^a groups of threads is not above the k-th largest logit
            int width = 1;
            while (kThreads / (2 * width) >= 2 * k && width < 32) width *= 2;
            u64 m = pass ? largest() : 0;
            for (int o = 1; o < width; o <<= 1) m = max64(m, __shfl_xor_sync(0xffffffffu, m, o));
            for (;;) {
                const int groups = kThreads / width;
                if (tid % width == 0) sh.maxima[tid / width] = m;
                __syncthreads();
                if (tid < groups) {
                    const u64 mine = sh.maxima[tid];
                    int r = 0;
                    for (int j = 0; j < groups; ++j) r += sh.maxima[j] > mine;
                    if (r == k - 1 && mine > sh.threshold) sh.threshold = mine;      // (one thread: nonzero entries differ)
                }
                __syncthreads();
                t = sh.threshold;
                pass = pass && key_of(high) >= (uint32_t)(t >> 32) && largest() >= t;
                passing = __syncthreads_count(pass);
                if (passing <= k + kSlackThreads || width == 1) break;
                width = 1;                                          // the logits lie together: once more, thread by thread
                m = pass ? largest() : 0;
            }
        }
        if (pass) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const u64 e = entry(v[i], index(base, i));
                if (e >= t) list[atomicAdd(&sh.n, 1)] = e;
            }
        }
        __syncthreads();
        if (sh.n > capacity(k) - per_chunk(k)) {
            const int n = prune(sh, list, best, k);
            for (int i = tid; i < n; i += kThreads) list[i] = best[i];
            if (tid == 0) { sh.n = n; if (n == k) sh.threshold = max64(sh.threshold, best[k - 1]); }
            __syncthreads();
        }
    }

    // ---- this CTA's sum and best
    float all = top;
#pragma unroll
    for (int o = 16; o; o >>= 1) all = fmaxf(all, __shfl_xor_sync(0xffffffffu, all, o));
    if (lane == 0) sh.tops[warp] = all;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) all = fmaxf(all, sh.tops[w]);
    double s = top == -INFINITY && sum == 0.0 ? 0.0 : sum * exp((double)top - (double)all);
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) sh.sums[warp] = s;
    const int mine = prune(sh, list, best, k);                      // (its barriers stand between the sums and their reader)
    __syncthreads();
    if (tid == 0) {
        s = 0.0;
        for (int w = 0; w < kThreads / 32; ++w) s += sh.sums[w];
        sh.sum = s; sh.top = all; sh.n_best = mine;
    }
    cluster.sync();
    if (rank == 0) {
        // ---- the row's: the others' lists behind this one's
        if (tid == 0) {
            float m = -INFINITY;
            for (int c = 0; c < ranks; ++c) m = fmaxf(m, cluster.map_shared_rank(&sh, c)->top);
            double z = 0.0;
            for (int c = 0; c < ranks; ++c) {
                const RowShared* other = cluster.map_shared_rank(&sh, c);
                if (!(other->top == -INFINITY && other->sum == 0.0)) z += other->sum * exp((double)other->top - (double)m);
            }
            p.lse[row] = (double)m + log(z);                        // NaN where a logit was, or all were -infinity
        }
        int n = 0;
        for (int c = 0; c < ranks; ++c) {
            const int from = cluster.map_shared_rank(&sh, c)->n_best;
            const u64* theirs = cluster.map_shared_rank(best, c);
            for (int i = tid; i < from; i += kThreads) list[n + i] = theirs[i];        // (at most 8 k, which the list holds)
            n += from;
        }
        if (tid == 0) sh.n = n;
        __syncthreads();
        if (ranks > 1) n = prune(sh, list, best, k);
        for (int i = tid; i < n; i += kThreads) p.best[(size_t)row * k + i] = best[i];
        if (tid == 0) p.count[row] = n;
    }
    cluster.sync();                                                 // nobody leaves while its lists are read
}

// One block per question: candidates of all rows with their scores in 64 bits, ranked.
constexpr int kJoinThreads = 1024;

__global__ void __launch_bounds__(kJoinThreads)
beam_join_kernel(const __grid_constant__ BeamParams p) {
    extern __shared__ __align__(16) unsigned char smem[];
    const int cap = p.n_beams * p.n_select;
    u64* keys = reinterpret_cast<u64*>(smem);                       // [cap] of the scores
    uint32_t* places = reinterpret_cast<uint32_t*>(keys + cap);     // [cap] beam * vocab + token
    u64* few_keys = reinterpret_cast<u64*>(smem + (size_t)(cap * 12 + 15) / 16 * 16);      // [n_select]
    uint32_t* few_places = reinterpret_cast<uint32_t*>(few_keys + p.n_select);
    __shared__ int n_all, n_few, counted;
    const int tid = threadIdx.x, k = p.n_select, row0 = blockIdx.x * p.n_beams;
    grid_dependency_wait();
    grid_launch_dependents();
    if (tid == 0) n_all = n_few = 0;
    __syncthreads();
    auto put = [&](double score, uint32_t place) {
        if (!(score > -INFINITY) || !isfinite(score)) return;
        const int at = atomicAdd(&n_all, 1);
        keys[at] = key_of(score); places[at] = place;
    };
    for (int i = tid; i < cap; i += kJoinThreads) {
        const int b = i / k, j = i - b * k, row = row0 + b;
        const float before = p.beam_scores[row];
        if (!isfinite(before)) continue;
        if (p.finished && p.finished[row]) {
            if (j == 0) put((double)before, (uint32_t)b * (uint32_t)p.vocab + (uint32_t)p.pad_token);
        } else if (j < p.count[row]) {
            const u64 e = p.best[(size_t)row * k + j];
            put((double)before + ((double)value_of((uint32_t)(e >> 32)) - p.lse[row]), (uint32_t)b * (uint32_t)p.vocab + (0xffffffffu - (uint32_t)e));
        }
    }
    __syncthreads();
    int n = n_all;
    const u64* from_keys = keys;
    const uint32_t* from_places = places;
    // how many entries satisfy a condition; all threads
    auto count = [&](auto holds) {
        int c = 0;
        for (int i = tid; i < n; i += kJoinThreads) c += holds(i);
        c = __reduce_add_sync(0xffffffffu, c);
        __syncthreads();
        if (tid == 0) counted = 0;
        __syncthreads();
        if ((tid & 31) == 0 && c) atomicAdd(&counted, c);
        __syncthreads();
        return counted;
    };
    if (n > kJoinThreads) {
        // the k-th largest score, bit by bit; of the entries equal to it, those of the lowest places
        u64 t = 0;
        for (int bit = 63; bit >= 0; --bit) {
            const u64 trial = t | 1ull << bit;
            if (count([&](int i) { return keys[i] >= trial; }) >= k) t = trial;
        }
        const int above = count([&](int i) { return keys[i] > t; });
        uint32_t last = 0;                                          // the (k - above)-th lowest place of those
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t trial = last | ((1u << bit) - 1u);       // all places of this prefix with a 0 here
            if (count([&](int i) { return keys[i] == t && places[i] <= trial; }) < k - above) last |= 1u << bit;
        }
        for (int i = tid; i < n; i += kJoinThreads)
            if (keys[i] > t || (keys[i] == t && places[i] <= last)) {
                const int at = atomicAdd(&n_few, 1);
                few_keys[at] = keys[i]; few_places[at] = places[i];
            }
        __syncthreads();
        n = n_few; from_keys = few_keys; from_places = few_places;
    }
    // ranks by comparing each with each, `share` threads to an entry
    int share = 1;
    while (share < 32 && n * share * 2 <= kJoinThreads) share *= 2;
    const int i = tid / share;
    int rank = 0;
    u64 key = 0;
    uint32_t place = 0;
    if (i < n) {
        key = from_keys[i]; place = from_places[i];
        for (int j = tid % share; j < n; j += share) {
            const u64 other = from_keys[j];
            rank += other > key || (other == key && from_places[j] < place);
        }
    }
    for (int o = 1; o < share; o <<= 1) rank += __shfl_xor_sync(0xffffffffu, rank, o);
    const size_t out = (size_t)blockIdx.x * k;
    if (i < n && tid % share == 0 && rank < k) {
        const uint32_t b = place / (uint32_t)p.vocab;
        p.parents[out + rank] = row0 + (int)b;
        p.tokens[out + rank] = (int)(place - b * (uint32_t)p.vocab);
        p.scores[out + rank] = (float)value_of(key);
    }
    if (tid >= n && tid < k) { p.parents[out + tid] = -1; p.tokens[out + tid] = -1; p.scores[out + tid] = -INFINITY; }
}

// Rows of many arrays: dst[i] = src[parents[i]].  Bound by HBM; a block moves 32 KiB of a row (8 loads of 16 bytes a thread before
// the first store), or less where rows are not whole 16-byte units.
template <typename U>
__device__ __forceinline__ void move_units(const unsigned char* src, unsigned char* dst, long units, long first) {
    const U* from = reinterpret_cast<const U*>(src);
    U* to = reinterpret_cast<U*>(dst);
    U x[kReorderUnits / kReorderThreads];
#pragma unroll
    for (int i = 0; i < kReorderUnits / kReorderThreads; ++i) {
        const long at = first + i * kReorderThreads + threadIdx.x;
        if (at < units) x[i] = __ldcs(from + at);
    }
#pragma unroll
    for (int i = 0; i < kReorderUnits / kReorderThreads; ++i) {
        const long at = first + i * kReorderThreads + threadIdx.x;
        if (at < units) __stcs(to + at, x[i]);
    }
}

__global__ void __launch_bounds__(kReorderThreads)
beam_reorder_kernel(const __grid_constant__ ReorderParams p) {
    grid_dependency_wait();
    grid_launch_dependents();
    int lo = 0, hi = p.n_states - 1;                                // the array of this block
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.first[mid] <= (int)blockIdx.x) lo = mid; else hi = mid - 1;
    }
    const int within = (int)blockIdx.x - p.first[lo];
    const int per_row = (p.first[lo + 1] - p.first[lo]) / p.n_out, row = within / per_row, part = within - row * per_row;
    const int from = p.parents[row];
    if (from < 0 || from >= p.n_in) {
        if (from != -1 && threadIdx.x == 0) atomicMin(p.status, (int)TTS_ERR_DEVICE_BOUNDS);
        return;
    }
    const long bytes = p.row_bytes[lo];
    const unsigned char* src = p.src[lo] + (size_t)from * bytes;
    unsigned char* dst = p.dst[lo] + (size_t)row * bytes;
    const uintptr_t x = reinterpret_cast<uintptr_t>(p.src[lo]) | reinterpret_cast<uintptr_t>(p.dst[lo]) | (uintptr_t)bytes;
    const long first = (long)part * kReorderUnits;
    if ((x & 15) == 0) move_units<uint4>(src, dst, bytes / 16, first);
    else if ((x & 3) == 0) move_units<uint32_t>(src, dst, bytes / 4, first);
    else move_units<unsigned char>(src, dst, bytes, first);
}

}  // namespace

cudaError_t launch_beam_select(BeamParams p, int logits_dtype, int n_sms, cudaStream_t st) {
    const int rows = p.n_groups * p.n_beams;
    const size_t elt = logits_dtype == TTS_LOGITS_BF16 ? 2 : 4;
    const bool vectors = ((reinterpret_cast<uintptr_t>(p.logits) | (uintptr_t)(p.row_stride * elt)) & 15) == 0;
    // CTAs to a row: until there are four to an SM, and as long as each has half a chunk
    int ctas = 1;
    while (ctas < 8 && rows * ctas < 4 * n_sms && p.vocab / (2 * ctas) >= kChunk / 2) ctas *= 2;
    p.per_cta = ceil_div(ceil_div(p.vocab, ctas), 8) * 8;
    const size_t smem = (sizeof(RowShared) + 15) / 16 * 16 + (size_t)(capacity(p.n_select) + p.n_select) * 8;
    auto rows_kernel = [&](auto kernel) {
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(ctas, rows); cfg.blockDim = kThreads; cfg.dynamicSmemBytes = smem; cfg.stream = st;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = ctas; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
        cfg.attrs = attr; cfg.numAttrs = 2;
        return cudaLaunchKernelEx(&cfg, kernel, p);
    };
    cudaError_t e;
    if (logits_dtype == TTS_LOGITS_BF16) e = vectors ? rows_kernel(beam_rows_kernel<__nv_bfloat16, true>) : rows_kernel(beam_rows_kernel<__nv_bfloat16, false>);
    else e = vectors ? rows_kernel(beam_rows_kernel<float, true>) : rows_kernel(beam_rows_kernel<float, false>);
    if (e != cudaSuccess) return e;
    const int cap = p.n_beams * p.n_select;
    const size_t join = (size_t)(cap * 12 + 15) / 16 * 16 + (size_t)p.n_select * 12;
    e = cudaFuncSetAttribute(beam_join_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)join);
    if (e != cudaSuccess) return e;
    return launch_dependent(beam_join_kernel, p.n_groups, kJoinThreads, join, st, p);
}

cudaError_t launch_beam_reorder(const ReorderParams& p, cudaStream_t st) {
    return launch_dependent(beam_reorder_kernel, p.first[p.n_states], kReorderThreads, 0, st, p);
}

}  // namespace tts
