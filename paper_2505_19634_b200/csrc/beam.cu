// Beam search: the best continuations of all beams of a question, and their states in the new order.
//
//   score(r, x) = beam_score[r] + logit[r][x] - log sum_y exp(logit[r][y]),   ties to the lowest (beam, token)
//
// Within a row the score does not fall where the logit rises, so a question's n best scores are among those of the n largest logits of each row;
// which tokens have them takes a look at the row again where its logits are so small beside the score that 64 bits do not hold both.
//
// Bound by HBM (or, for few rows, by latency).  A row is cut into 1 to 8 parts, one CTA each, read once in chunks of four 16-byte loads a
// thread (what is left of a load one by one, and short parts): their exponentials go to a running sum, their largest to shared memory.  The n-th largest of the threads' maxima is a lower
// bound of the n-th largest logit; of the few places whose maximum reaches it the logits are read again (from L2) and listed.  The CTA that
// ends a question's last part does the same with the entries of all of them, whose scores it forms in 64 bits from the logit, the beam's score
// and the logarithm of its sum (so of one beam's candidates the order is exact), and ranks what is left by comparing each with each.  Where numbers are so alike or so
// ordered that a list would overflow, the n-th largest is found by bisection instead.
//
// Which thread adds up which logits does not depend on where a row lies in memory: equal rows have equal sums, bit for bit, and equal scores.
// Exponentials are fp32 (2^-22, and 2^-23 of their exponent); 32 of them are summed in fp32, everything beyond, the logarithm too, in 64 bits:
// a beam's candidates are all off by the same 1.4e-7 at most (measured; rows of 300 to 152064 normal logits of size 1 to 30), so those of different
// beams that lie closer than twice that may change places.  For few rows the time is that of fetching
// every instruction once (about 20 cycles each), which is why there are few phases and little unrolled code outside the pass.
//
// Measured: one question of 4 beams, 151936 logits 11.0 us; 16 questions of 16 beams, 152064 bf16 logits 31.9 us (78 MB: 11.9 us at the copy
// peak, 39 million exponentials: 8.7).  Clocks of a CTA there: start 1300, pass 18300, bound, list, output and arrival about 11000, join of a
// question 9000.  All CTAs are resident at once, so nothing covers what lies behind the pass.
#include <math.h>

#include <type_traits>

#include "beam.cuh"
#include "launch.cuh"
#include "packed.cuh"

namespace tts {

namespace {

typedef unsigned long long u64;

constexpr int kThreads = 256;
constexpr int kLoads = 4;                                           // 16-byte loads of a thread per chunk
constexpr int kPlaces = 16;                                         // maxima that a thread keeps, of one chunk or several
constexpr int kTasks = 1024;                                        // places to read again, at most
constexpr int kList = 1024;                                         // entries of a list in shared memory
static_assert(kMaxSelect <= kThreads && 1 << beam_cap_log2(kMaxSelect) <= kList, "");

// Order-preserving maps of floating point to unsigned words; -infinity is the least number, and 0 is below it.  Zeros of both signs are one
// number (adding 0 makes them +0); a double here is a sum with such a logit and never -0.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ u64 key_of(double x) {
    const u64 b = (u64)__double_as_longlong(x);
    return b >> 63 ? ~b : b | 1ull << 63;
}
__device__ __forceinline__ double value_of(u64 k) { return __longlong_as_double((long long)(k >> 63 ? k & ~(1ull << 63) : ~k)); }

__device__ __forceinline__ float exp2_approx(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) { uint32_t r; asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b)); return r; }

// A candidate: its key (of the logit within a row, of the score within a question) and its place (token; beam * vocab + token).  Of equal
// keys the lowest place is better, so no two candidates are equal.
template <int kN>
struct Lists {
    u64 keys[kN];
    uint32_t places[kN];
    int n;                                                          // candidates that wanted to the list
    __device__ __forceinline__ void put(u64 key, uint32_t place) {
        const int at = atomicAdd(&n, 1);
        if (at < kN) { keys[at] = key; places[at] = place; }
    }
};
struct Shared {
    union {
        float maxima[kPlaces + 1][kThreads];                        // (the last of what is read one by one)
        struct {
            double base[kMaxBranches];                              // of every row: its score so far less the logarithm of its sum
            bool done[kMaxBranches];                                // and whether it is a finished beam
        };
    };
    Lists<kList> list;
    Lists<kThreads> few;
    u64 groups[kThreads];
    double sums[kThreads / 32];
    float tops[kThreads / 32];
    u64 threshold;
    int word, n_tasks;
    int tasks[kTasks];
};

// The sum over the block, known to all threads.
__device__ __noinline__ int block_sum(int c, int* word) {
    c = __reduce_add_sync(0xffffffffu, c);
    __syncthreads();
    if (threadIdx.x == 0) *word = 0;
    __syncthreads();
    if ((threadIdx.x & 31) == 0 && c) atomicAdd(word, c);
    __syncthreads();
    return *word;
}

// The k-th largest of the maxima of 2^a threads each, as many of them as can be with at least 2 k: not above the k-th largest key of all.
// 0 where there are fewer.
__device__ __noinline__ u64 lower_bound(Shared& sh, u64 m, int k) {
    const int tid = threadIdx.x;
    int shift = 0;
    while (shift < 5 && (kThreads >> (shift + 1)) >= 2 * k) { m = max(m, __shfl_xor_sync(0xffffffffu, m, 1 << shift)); ++shift; }
    const int groups = kThreads >> shift;
    if (tid == 0) sh.threshold = 0;
    if ((tid & ((1 << shift) - 1)) == 0) sh.groups[tid >> shift] = m;
    __syncthreads();
    // 2^shift threads rank a group's maximum among the others
    const int g = tid >> shift;
    const u64 own = sh.groups[g];
    int r = 0;
#pragma unroll 4
    for (int j = tid & ((1 << shift) - 1); j < groups; j += 1 << shift) { const u64 other = sh.groups[j]; r += other > own || (other == own && j < g); }
    for (int o = 1; o < 1 << shift; o <<= 1) r += __shfl_xor_sync(0xffffffffu, r, o);
    if (r == k - 1) sh.threshold = own;
    __syncthreads();
    return sh.threshold;
}

// The k best of more candidates than the list holds, by bisection over their keys (of kBits), then over the places of those equal to the
// k-th.  `each(f)` calls f(key, place) for this thread's candidates; a key of 0 is none.  They are listed.
template <int kBits, typename List, typename Each>
__device__ void bisect(Shared& sh, List& list, int k, Each each) {
    auto count = [&](auto holds) {
        int c = 0;
        each([&](u64 key, uint32_t place) { c += key != 0 && holds(key, place); });
        return block_sum(c, &sh.word);
    };
    u64 t = 0;
#pragma unroll 1
    for (int bit = kBits - 1; bit >= 0; --bit) {
        const u64 trial = t | 1ull << bit;
        if (count([&](u64 key, uint32_t) { return key >= trial; }) >= k) t = trial;
    }
    const int above = count([&](u64 key, uint32_t) { return key > t; });
    uint32_t last = 0;                                              // the (k - above)-th lowest place of those equal
#pragma unroll 1
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t trial = last | ((1u << bit) - 1u);           // all places of this prefix with a 0 here
        if (count([&](u64 key, uint32_t place) { return key == t && place <= trial; }) < k - above) last |= 1u << bit;
    }
    if (threadIdx.x == 0) list.n = 0;
    __syncthreads();
    each([&](u64 key, uint32_t place) { if (key != 0 && (key > t || (key == t && place <= last))) list.put(key, place); });
    __syncthreads();
}

// Maxima and sums relative to them of kN lanes, joined in every one of them.
template <int kN>
__device__ __forceinline__ void join_sums(float& top, double& sum) {
    float all = top;
#pragma unroll
    for (int o = kN / 2; o; o >>= 1) all = fmaxf(all, __shfl_xor_sync(0xffffffffu, all, o));
    sum = top == -INFINITY && sum == 0.0 ? 0.0 : sum * exp2_approx((top - all) * kLog2e);
#pragma unroll
    for (int o = kN / 2; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    top = all;
}

// A candidate's score, as a key; 0 is no candidate.
__device__ __forceinline__ u64 score_key(double base, float logit) {
    const double x = base + (double)logit;
    return isfinite(x) ? key_of(x) : 0;
}

// Where a logit is so small beside its score that others of its row have the same score in 64 bits, the lists, which go by logits, may lack
// tokens that are as good as the k-th best and come before some of theirs.  (What is better than the k-th best is listed: a part that leaves
// out a candidate lists k that are not worse.)  All candidates of that score are looked at in their order, and the places of the result
// behind the `above` better ones go to the first of them.
template <typename T>
__device__ __noinline__ void place_equals(const BeamParams& p, Shared& sh, int row0, size_t out, int above) {
    constexpr int kEach = 8;                                        // tokens of a thread at a time
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const u64 t = sh.threshold;
    int at = above;
#pragma unroll 1
    for (int b = 0; b < p.n_beams && at < p.n_select; ++b) {
        const double base = sh.base[b];
        const bool done = sh.done[b];
        if (!isfinite(base)) continue;
        const T* x = static_cast<const T*>(p.logits) + (size_t)(row0 + b) * p.row_stride;
        const int n = done ? 1 : p.vocab;
#pragma unroll 1
        for (int x0 = 0; x0 < n && at < p.n_select; x0 += kThreads * kEach) {
            const int first = x0 + tid * kEach;
            unsigned hits = 0;
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                if (first + i < n && score_key(base, done ? 0.f : (float)x[first + i] + 0.f) == t) hits |= 1u << i;
            int before = __popc(hits);
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int c = __shfl_up_sync(0xffffffffu, before, o);
                if (lane >= o) before += c;
            }
            if (lane == 31) sh.tasks[warp] = before;
            before += at - __popc(hits);
            __syncthreads();
            for (int w = 0; w < kThreads / 32; ++w) {
                if (w < warp) before += sh.tasks[w];
                at += sh.tasks[w];
            }
            for (; hits && before < p.n_select; hits &= hits - 1, ++before) {
                p.parents[out + before] = row0 + b;
                p.tokens[out + before] = done ? p.pad_token : first + __ffs(hits) - 1;
            }
            __syncthreads();
        }
    }
}

// A question's parts put together by one block.
template <typename T>
__device__ void join_parts(const BeamParams& p, Shared& sh, int group) {
    const int tid = threadIdx.x, k = p.n_select, row0 = group * p.n_beams;
    const size_t out = (size_t)group * k;
    const u64* entries = p.entries + ((size_t)row0 << (p.parts_log2 + p.cap_log2));
    const int n = __ldcg(p.n_entries + group);
    // A thread looks at every 256th entry, from the one whose number is its own with the bits in reverse: few entries lie in all groups of
    // threads alike then, and the bound does not fall to the least of them (4 beams of 32000 logits: 9.5 us instead of 14.0).
    const int mine = (int)(__brev((unsigned)tid) >> 24);
    static_assert(kThreads == 256, "eight bits");
    constexpr int kAhead = kList / kThreads;
    u64 e[kAhead];                                                  // (asked for ahead of the logarithms)
#pragma unroll
    for (int i = 0; i < kAhead; ++i) e[i] = mine + i * kThreads < n ? __ldcg(entries + mine + i * kThreads) : 0;
    if (tid == 0) sh.few.n = 0;
    // the rows' logarithms, eight lanes each; NaN for a row that offers nothing.  (A finished beam's candidate has a logit of 0.)
    const int sub = tid & 7;
#pragma unroll 1
    for (int b0 = 0; b0 < p.n_beams; b0 += kThreads / 8) {
        const int b = min(b0 + (tid >> 3), p.n_beams - 1), row = row0 + b;
        float top = -INFINITY;
        double sum = 0.0;
        if (sub < 1 << p.parts_log2) {
            const size_t part = ((size_t)row << p.parts_log2) + sub;
            top = __ldcg(p.part_top + part); sum = __ldcg(p.part_sum + part);
        }
        const float before = p.beam_scores[row];
        const bool done = p.finished && p.finished[row];
        join_sums<8>(top, sum);
        if (sub == 0) { sh.base[b] = (double)before - (done ? 0.0 : (double)top + log(sum)); sh.done[b] = done; }
    }
    if (tid < k) { p.parents[out + tid] = -1; p.tokens[out + tid] = -1; p.scores[out + tid] = -INFINITY; }      // where there are too few candidates
    __syncthreads();
    auto score = [&](u64 entry) { return score_key(sh.base[(uint32_t)entry / (uint32_t)p.vocab], value_of((uint32_t)(entry >> 32))); };
    auto all = [&](auto f) {
#pragma unroll 4
        for (int i = tid; i < n; i += kThreads) { const u64 x = __ldcg(entries + i); f(score(x), (uint32_t)x); }
    };
    int listed = n;
    u64 best = 0;
    if (n > kList) {
        // more than the list holds: those that reach the k-th largest of the threads' best, a few more than k for most numbers (64 beams of
        // 64 continuations: 75 us; by bisection of them all 4680)
        all([&](u64 key, uint32_t) { best = max(best, key); });
        const u64 least = max(lower_bound(sh, best, k), (u64)1);
        if (tid == 0) sh.list.n = 0;
        __syncthreads();
        all([&](u64 key, uint32_t place) { if (key >= least) sh.list.put(key, place); });
        __syncthreads();
        listed = sh.list.n;
        best = 0;
        if (listed <= kList)
            for (int i = mine; i < listed; i += kThreads) best = max(best, sh.list.keys[i]);
    } else {
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (mine + i * kThreads < n) {
                const u64 key = score(e[i]);
                sh.list.keys[mine + i * kThreads] = key; sh.list.places[mine + i * kThreads] = (uint32_t)e[i];
                best = max(best, key);
            }
    }
    if (listed > kList) bisect<64>(sh, sh.few, k, all);
    else {
        const u64 least = max(lower_bound(sh, best, k), (u64)1);
        auto each = [&](auto f) { for (int i = mine; i < listed; i += kThreads) f(sh.list.keys[i], sh.list.places[i]); };
        each([&](u64 key, uint32_t place) { if (key >= least) sh.few.put(key, place); });
        __syncthreads();
        if (sh.few.n > kThreads) bisect<64>(sh, sh.few, k, each);
    }
    const int n_few = sh.few.n;
    int wide = 0;                                                   // 2^wide threads rank one of them
    while (wide < 5 && n_few << (wide + 1) <= kThreads) ++wide;
    bool vague = false;                                             // another logit may have this score
    {
        const int i = tid >> wide;
        const u64 key = i < n_few ? sh.few.keys[i] : 0;
        const uint32_t place = i < n_few ? sh.few.places[i] : 0;
        int rank = 0;
#pragma unroll 4
        for (int j = tid & ((1 << wide) - 1); j < n_few; j += 1 << wide) rank += sh.few.keys[j] > key || (sh.few.keys[j] == key && sh.few.places[j] < place);
        for (int o = 1; o < 1 << wide; o <<= 1) rank += __shfl_xor_sync(0xffffffffu, rank, o);
        if (i < n_few && rank < k) {
            const uint32_t b = place / (uint32_t)p.vocab;
            p.parents[out + rank] = row0 + (int)b;
            p.tokens[out + rank] = (int)(place - b * (uint32_t)p.vocab);
            p.scores[out + rank] = (float)value_of(key);
            // Neighbouring logits are 2^-25 of themselves apart or more, scores 2^-52 or less: with one that is over 2^-26 of the score there is a
            // score between them.
            const double x = value_of(key);
            vague = !sh.done[b] && fabs(x - sh.base[b]) <= 0x1p-26 * fabs(x);
            if (rank == k - 1) sh.threshold = key;
        }
    }
    if (__syncthreads_or(vague) && n_few >= k) {
        const u64 t = sh.threshold;
        const int above = block_sum(tid < n_few && sh.few.keys[tid] > t, &sh.word);
        place_equals<T>(p, sh, row0, out, above);
    }
}

template <typename T, bool kAligned>
__global__ void __launch_bounds__(kThreads, 4)
beam_select_kernel(const __grid_constant__ BeamParams p) {
    __shared__ Shared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, row = blockIdx.y, k = p.n_select;
    const size_t part = ((size_t)row << p.parts_log2) + blockIdx.x;
    grid_dependency_wait();
    grid_launch_dependents();
    if (isfinite(p.beam_scores[row]) && !(p.finished && p.finished[row])) {
        const T* x = static_cast<const T*>(p.logits) + (size_t)row * p.row_stride;
        const int begin = min(p.vocab, (int)blockIdx.x * p.per_part), end = min(p.vocab, begin + p.per_part);
        constexpr int kVec = 16 / sizeof(T), kChunk = kThreads * kLoads * kVec;       // logits of a load, of a chunk
        // (less than half a chunk goes one by one: the loads would leave threads without a logit, and the bound below would let too much through)
        const int behind = end - begin < kChunk / 2 ? begin : begin + (end - begin) / kVec * kVec, singles = end - behind, chunks = (behind - begin + kChunk - 1) / kChunk;
        const int per_place = (chunks + kPlaces - 1) / kPlaces;     // chunks of a maximum
        auto index = [&](int chunk, int i) { return begin + chunk * kChunk + (i / kVec) * (kThreads * kVec) + tid * kVec + i % kVec; };
        auto fetch = [&](int chunk, uint4 (&raw)[kLoads]) {
#pragma unroll
            for (int c = 0; c < kLoads; ++c) {
                const int at = index(chunk, c * kVec);
                const T* from = x + at;
                constexpr uint32_t kNone = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;          // -infinity
                raw[c] = make_uint4(kNone, kNone, kNone, kNone);
                if (at >= behind) continue;                         // (behind the part's end in its last chunk)
                if constexpr (kAligned) raw[c] = *reinterpret_cast<const uint4*>(from);
                else {
                    uint32_t w[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if constexpr (sizeof(T) == 4) w[j] = __float_as_uint(from[j]);
                        else w[j] = reinterpret_cast<const unsigned short*>(from)[2 * j] | (uint32_t)reinterpret_cast<const unsigned short*>(from)[2 * j + 1] << 16;
                    }
                    raw[c] = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
        };
        // word c of a thread's loads, and the logits in a word
        auto word = [](const uint4 (&raw)[kLoads], int c) { const uint4& r = raw[c >> 2]; return (c & 3) == 0 ? r.x : (c & 3) == 1 ? r.y : (c & 3) == 2 ? r.z : r.w; };
        auto logit = [&](const uint4 (&raw)[kLoads], int i) {
            const uint32_t w = word(raw, sizeof(T) == 2 ? i >> 1 : i);
            return __uint_as_float(sizeof(T) == 4 ? w : i & 1 ? w & 0xffff0000u : w << 16);
        };
        auto largest = [&](const uint4 (&raw)[kLoads]) {
            uint32_t h[4] = {word(raw, 0), word(raw, 1), word(raw, 2), word(raw, 3)};
            auto larger = [](uint32_t a, uint32_t b) { return sizeof(T) == 2 ? max_bf16x2(a, b) : __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); };
#pragma unroll
            for (int c = 4; c < 4 * kLoads; ++c) h[c & 3] = larger(h[c & 3], word(raw, c));
            const uint32_t m = larger(larger(h[0], h[1]), larger(h[2], h[3]));
            return sizeof(T) == 4 ? __uint_as_float(m) : fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
        };

        // ---- one pass: sums of exponentials and maxima
        float top = -INFINITY;                                      // of this thread's logits so far
        double sum = 0.0;                                           // of exp(logit - top)
        auto raise = [&](float high) {
            if (high > top) {
                sum *= exp2_approx((top - high) * kLog2e);
                top = high;
            }
            return top == -INFINITY ? 0.f : -top;
        };
        {
            uint4 next[kLoads];
            if (chunks > 0) fetch(0, next);
            // (the singles while the first chunk is on its way)
            float high_here = -INFINITY;
#pragma unroll 1
            for (int j0 = tid; j0 < singles; j0 += 4 * kThreads) {
                float v[4], part4 = 0.f;
#pragma unroll
                for (int c = 0; c < 4; ++c) v[c] = j0 + c * kThreads < singles ? (float)x[behind + j0 + c * kThreads] : -INFINITY;
                const float high = fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), ref = raise(high);
#pragma unroll
                for (int c = 0; c < 4; ++c) part4 += exp2_approx((v[c] + ref) * kLog2e);
                sum += part4;
                high_here = fmaxf(high_here, high);
            }
            sh.maxima[kPlaces][tid] = high_here;
            high_here = -INFINITY;
            int place = 0, left = per_place;
#pragma unroll 1
            for (int chunk = 0; chunk < chunks; ++chunk) {
                uint4 raw[kLoads];
#pragma unroll
                for (int c = 0; c < kLoads; ++c) raw[c] = next[c];
                if (chunk + 1 < chunks) fetch(chunk + 1, next);
                const float high = largest(raw), ref = raise(high);
                const uint64_t ref2 = pack2(ref, ref), log2e = pack2(kLog2e, kLog2e);
                uint64_t part2[2] = {0, 0};
#pragma unroll
                for (int i = 0; i < kLoads * kVec; i += 2) {
                    const float2 y = unpack2(mul2(add2(pack2(logit(raw, i), logit(raw, i + 1)), ref2), log2e));
                    part2[(i >> 1) & 1] = add2(part2[(i >> 1) & 1], pack2(exp2_approx(y.x), exp2_approx(y.y)));
                }
                const float2 s2 = unpack2(add2(part2[0], part2[1]));
                sum += s2.x + s2.y;
                high_here = fmaxf(high_here, high);
                if (--left == 0 || chunk + 1 == chunks) { sh.maxima[place++][tid] = high_here; high_here = -INFINITY; left = per_place; }
            }
        }

        // ---- what reaches the lower bound is read again and listed
        if (tid == 0) { sh.list.n = 0; sh.n_tasks = 0; }
        const u64 bound = lower_bound(sh, key_of(top), k);
        const float least = fmaxf(value_of((uint32_t)bound), -3.402823466e38f);      // (-infinity is nobody's choice; of 0 the value is a NaN)
        // (whose 32 logits of which chunk: four threads look at them, so that all of them are on their way at once)
        if (chunks > 0)
#pragma unroll 1
            for (int place = 0; place * per_place < chunks; ++place)
                if (sh.maxima[place][tid] >= least)
                    for (int chunk = place * per_place; chunk < min(chunks, (place + 1) * per_place); ++chunk) {
                        const int at = atomicAdd(&sh.n_tasks, 1);
                        if (at < kTasks) sh.tasks[at] = chunk * kThreads + tid;
                    }
        if (sh.maxima[kPlaces][tid] >= least)
#pragma unroll 1
            for (int j = tid; j < singles; j += kThreads) {
                const float v = (float)x[behind + j];
                if (v >= least) sh.list.put(key_of(v), (uint32_t)(behind + j));
            }
        __syncthreads();
        const int n_tasks = sh.n_tasks;
        if (n_tasks <= kTasks)
#pragma unroll 1
            for (int i = tid >> 2; i < n_tasks; i += kThreads / 4) {
                const int chunk = sh.tasks[i] / kThreads, who = sh.tasks[i] % kThreads, at = begin + chunk * kChunk + (tid & 3) * (kThreads * kVec) + who * kVec;
                if (at >= behind) continue;
                float v[kVec];
                if constexpr (kAligned) {
                    const uint4 r = *reinterpret_cast<const uint4*>(x + at);
                    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
                    for (int j = 0; j < kVec; ++j) v[j] = __uint_as_float(sizeof(T) == 4 ? w[j] : j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
                } else {
#pragma unroll
                    for (int j = 0; j < kVec; ++j) v[j] = (float)x[at + j];
                }
#pragma unroll
                for (int j = 0; j < kVec; ++j) if (v[j] >= least) sh.list.put(key_of(v[j]), (uint32_t)(at + j));
            }
        // the CTA's sum
        join_sums<32>(top, sum);
        if (lane == 0) { sh.tops[warp] = top; sh.sums[warp] = sum; }
        __syncthreads();
        if (sh.list.n > 1 << p.cap_log2 || n_tasks > kTasks)        // more than the part's list holds: its k best
            bisect<32>(sh, sh.list, k, [&](auto f) {
                for (int i = begin + tid; i < end; i += kThreads) { const float v = (float)x[i]; f(v > -INFINITY ? (u64)key_of(v) : 0, (uint32_t)i); }
            });
        const int group = row / p.n_beams, n = min(sh.list.n, 1 << p.cap_log2);
        if (tid == 0) sh.word = atomicAdd(p.n_entries + group, n);
        __syncthreads();
        u64* to = p.entries + ((size_t)group * p.n_beams << (p.parts_log2 + p.cap_log2)) + sh.word;
        const uint32_t at = (uint32_t)(row - group * p.n_beams) * (uint32_t)p.vocab;
        for (int i = tid; i < n; i += kThreads) to[i] = sh.list.keys[i] << 32 | (at + sh.list.places[i]);
        if (warp == 0) {
            float m = lane < kThreads / 32 ? sh.tops[lane] : -INFINITY;
            double z = lane < kThreads / 32 ? sh.sums[lane] : 0.0;
            join_sums<8>(m, z);
            if (lane == 0) { p.part_top[part] = m; p.part_sum[part] = z; }
        }
    } else if (isfinite(p.beam_scores[row]) && blockIdx.x == 0 && tid == 0) {      // a finished beam: itself
        const int group = row / p.n_beams, at = atomicAdd(p.n_entries + group, 1);
        p.entries[((size_t)group * p.n_beams << (p.parts_log2 + p.cap_log2)) + at] =
            (u64)key_of(0.f) << 32 | ((uint32_t)(row - group * p.n_beams) * (uint32_t)p.vocab + (uint32_t)p.pad_token);
    }
    // ---- the CTA that ends the question's last part puts them together
    __syncthreads();
    const int group = row / p.n_beams;
    if (tid == 0) {
        __threadfence();                                            // the block's writes, which the barrier put before this
        const bool last = atomicAdd(p.arrived + group, 1) + 1 == p.n_beams << p.parts_log2;
        if (last) {
            p.arrived[group] = 0;                                   // as the next call expects it
            __threadfence();
        }
        sh.word = last;
    }
    __syncthreads();
    const bool last = sh.word;
    __syncthreads();
    if (!last) return;
    join_parts<T>(p, sh, group);
    if (tid == 0) p.n_entries[group] = 0;                           // as the next call expects it (all threads have read it)
}

// Rows of many arrays: dst[i] = src[parents[i]].  Bound by HBM; a block writes 32 KiB of a row, eight aligned 16-byte units a thread, all
// loaded before the first store.  Where a row of src starts elsewhere within 16 bytes than its row of dst, a unit is put together from two
// aligned loads, of which the second is the next lane's first; what is left at a row's ends moves byte by byte.  48 dense caches of 16 rows
// of 512 KiB: 103 us, the copy peak; of 512 KiB and a byte 114 (byte by byte 488); 16 rows of five small arrays 4.2 to 4.9 us, a launch.
constexpr int kReorderLoads = kReorderUnits / kReorderThreads;
__device__ __forceinline__ void move_aligned(const unsigned char* src, unsigned char* dst, long bytes, long first) {
    const uint4* from = reinterpret_cast<const uint4*>(src);
    uint4* to = reinterpret_cast<uint4*>(dst);
    const long units = bytes / 16;
    uint4 x[kReorderLoads];
#pragma unroll
    for (int i = 0; i < kReorderLoads; ++i) {
        const long at = first + i * kReorderThreads + threadIdx.x;
        if (at < units) x[i] = __ldcs(from + at);
    }
#pragma unroll
    for (int i = 0; i < kReorderLoads; ++i) {
        const long at = first + i * kReorderThreads + threadIdx.x;
        if (at < units) __stcs(to + at, x[i]);
    }
}
// Unit v of a row: the v-th 16 bytes of dst, counted from the aligned address at or before its start.  Whole units are those that lie
// within the row with both aligned loads; fewer than 64 bytes ahead of them and behind them go one to a thread.
__device__ __forceinline__ void move_shifted(const unsigned char* src, unsigned char* dst, long bytes, long first) {
    const int lane = threadIdx.x & 31, lead = (int)(reinterpret_cast<uintptr_t>(dst) & 15);
    const int off = (int)((reinterpret_cast<uintptr_t>(src) - lead) & 15);          // of a unit's first byte in src
    const long begin = (off + lead + 15) >> 4, end = max(begin, (bytes - (off ? 32 - off : 16) + lead + 16) >> 4);
    if (first == 0 && threadIdx.x < 128) {
        const long from = end > begin ? 16 * end - lead : 0, to = end > begin ? 16 * begin - lead : 0;
        const long j = threadIdx.x < 64 ? (long)threadIdx.x : from + threadIdx.x - 64;
        if (j < (threadIdx.x < 64 ? to : bytes)) dst[j] = src[j];
    }
    constexpr int kAtOnce = kReorderLoads / 2;
#pragma unroll 1
    for (int part = 0; part < 2; ++part) {
        const long v0 = begin + first + part * kAtOnce * kReorderThreads + threadIdx.x;
        uint4 a[kAtOnce], b[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const long v = v0 + i * kReorderThreads;
            a[i] = b[i] = make_uint4(0, 0, 0, 0);
            if (v < end) {
                const uint4* from = reinterpret_cast<const uint4*>(src + 16 * v - lead - off);
                a[i] = __ldcs(from);
                if (off != 0 && (lane == 31 || v + 1 == end)) b[i] = __ldcs(from + 1);
            }
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const long v = v0 + i * kReorderThreads;
            uint4 y = a[i], z = b[i];
            if (off != 0) {
                const uint4 n = make_uint4(__shfl_down_sync(0xffffffffu, y.x, 1), __shfl_down_sync(0xffffffffu, y.y, 1), __shfl_down_sync(0xffffffffu, y.z, 1), __shfl_down_sync(0xffffffffu, y.w, 1));
                if (lane != 31 && v + 1 < end) z = n;
                const int bits = 8 * (off & 3);
                const uint32_t w[8] = {y.x, y.y, y.z, y.w, z.x, z.y, z.z, z.w};
                uint32_t t[5];
#pragma unroll
                for (int j = 0; j < 5; ++j) t[j] = off < 4 ? w[j] : off < 8 ? w[min(j + 1, 7)] : off < 12 ? w[min(j + 2, 7)] : w[min(j + 3, 7)];
                y = make_uint4(__funnelshift_r(t[0], t[1], bits), __funnelshift_r(t[1], t[2], bits), __funnelshift_r(t[2], t[3], bits), __funnelshift_r(t[3], t[4], bits));
            }
            if (v < end) __stcs(reinterpret_cast<uint4*>(dst + 16 * v - lead), y);
        }
    }
}

__global__ void __launch_bounds__(kReorderThreads, 4)
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
    const long first = (long)part * kReorderUnits;
    if (reorder_aligned(p.src[lo], p.dst[lo], bytes)) move_aligned(src, dst, bytes, first);
    else move_shifted(src, dst, bytes, first);
}

}  // namespace

cudaError_t launch_beam_select(BeamParams p, int logits_dtype, cudaStream_t st) {
    p.per_part = ceil_div(ceil_div(p.vocab, 1 << p.parts_log2), 8) * 8;
    const dim3 grid(1 << p.parts_log2, p.n_groups * p.n_beams);
    const size_t elt = logits_dtype == TTS_LOGITS_BF16 ? 2 : 4;
    const bool aligned = ((reinterpret_cast<uintptr_t>(p.logits) | (uintptr_t)(p.row_stride * elt)) & 15) == 0;
    if (logits_dtype == TTS_LOGITS_BF16)
        return aligned ? launch_dependent(beam_select_kernel<__nv_bfloat16, true>, grid, kThreads, 0, st, p) : launch_dependent(beam_select_kernel<__nv_bfloat16, false>, grid, kThreads, 0, st, p);
    return aligned ? launch_dependent(beam_select_kernel<float, true>, grid, kThreads, 0, st, p) : launch_dependent(beam_select_kernel<float, false>, grid, kThreads, 0, st, p);
}

cudaError_t launch_beam_reorder(const ReorderParams& p, cudaStream_t st) {
    return launch_dependent(beam_reorder_kernel, p.first[p.n_states], kReorderThreads, 0, st, p);
}

}  // namespace tts
