// How attention over the 8-bit cache is cut into work.
//
// An item is a (branch, KV head, block of stacked rows), from the prefix's first token on: what branches share is worked through for each.
// It has a unit for every kUnitTokens tokens (an empty branch's: one), behind
// kStart units for what a piece of an item costs besides (queries, the join of its parts): so a CTA with many short items gets
// fewer tokens.  All items follow one another, a CTA owns a contiguous run of units and walks over its pieces of items; what it has of
// an item that others work on too it leaves as a part, and the last one to do so joins them.  Where there are CTAs enough to give each
// a small share of one item only, items are cut evenly instead.
#pragma once
#include "kv8.cuh"

namespace tts {

namespace {

// Tokens of a branch; a bad length raises the status and counts as an empty branch.
__device__ __forceinline__ int kv8_tokens(const Kv8AttnParams& p, int b, bool raise) {
    const int L = p.branch_lens[b];
    const long n = (long)p.prefix_len + L;
    if (L < 0 || n > (long)p.max_blocks * kPage) {
        if (raise) atomicMin(p.status, (int)TTS_ERR_DEVICE_BOUNDS);
        return 0;
    }
    return (int)n;
}
template <int kUnitTokens, int kStart>
__device__ __forceinline__ int kv8_units(int tokens) { return kStart + max(1, (tokens + kUnitTokens - 1) / kUnitTokens); }

// Units before each branch (per KV head and row block together), in 64 bits; all threads of the block.
template <int kThreads, int kUnitTokens, int kStart>
__device__ void kv8_scan_units(const Kv8AttnParams& p, long long* cum, long long* warp_sums) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = p.Hkv * p.n_rb;
    long long carry = 0;
    for (int base = 0; base < p.n_branches; base += kThreads) {
        const int b = base + threadIdx.x;
        long long v = b < p.n_branches ? (long long)kv8_units<kUnitTokens, kStart>(kv8_tokens(p, b, blockIdx.x == 0)) * per : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long n = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += n;
        }
        if (lane == 31) warp_sums[warp] = v;
        __syncthreads();
        long long before = carry, all = 0;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w < warp) before += warp_sums[w];
            all += warp_sums[w];
        }
        if (b < p.n_branches) cum[b + 1] = before + v;
        carry += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) cum[0] = 0;
    __syncthreads();
}

// The CTA's run: n units from `begin` on; all threads of the block.  Joining an item's parts takes time in proportion to their number, so
// an even cut makes shares of 1.5 times the root of the longest item's units, at least `least`, more where CTAs are few; it is for
// shares of up to `most`, or of no more than a CTA's run would be (16 branches of 2000 keys, 8 KV heads: 19.4 us, in runs 23.8).
// Otherwise a CTA has at least `least` units of tokens.
struct Kv8Run {
    long long begin, per_cta;
    int n;
    int cut, each;          // an even cut: CTAs to an item, units of tokens to a CTA; or 0
};
template <int kThreads, int kStart>
__device__ __forceinline__ Kv8Run kv8_run(const Kv8AttnParams& p, const long long* cum, int* word, int least, int most) {
    const int per_branch = p.Hkv * p.n_rb;
    const long long total = cum[p.n_branches];
    Kv8Run r;
    r.cut = r.each = 0;
    r.per_cta = max((long long)kStart + least, (total + gridDim.x - 1) / gridDim.x);
    if (p.n_branches * per_branch <= (int)gridDim.x) {
        if (threadIdx.x == 0) *word = 0;
        __syncthreads();
        for (int b = threadIdx.x; b < p.n_branches; b += kThreads) atomicMax(word, (int)((cum[b + 1] - cum[b]) / per_branch) - kStart);
        __syncthreads();
        const int longest = *word, share = max(least, (int)(1.5f * sqrtf((float)longest)));
        const int cut = min((longest + share - 1) / share, (int)gridDim.x / (p.n_branches * per_branch)), each = (longest + cut - 1) / cut;
        if (each <= max((long long)max(most, share), r.per_cta)) {
            r.cut = cut; r.each = each;
            const int item = blockIdx.x / cut, b = item / per_branch;
            r.n = 0; r.begin = 0;
            if (b < p.n_branches) {
                const int units = (int)((cum[b + 1] - cum[b]) / per_branch), first = (int)(blockIdx.x - item * cut) * r.each;
                r.n = min(units - kStart - first, r.each);          // (not positive where the branch has no tokens left for this CTA)
                r.begin = cum[b] + (long long)(item - b * per_branch) * units + kStart + first;
            }
            return r;
        }
    }
    r.begin = (long long)blockIdx.x * r.per_cta;
    r.n = (int)min(max(total - r.begin, 0ll), r.per_cta);           // (fits: the host refuses more than 2^31 units to a CTA)
    return r;
}

// The pieces of a CTA's run, one after another, each its part of an item (KV head * n_rb + row block) of a branch.
template <int kUnitTokens, int kStart>
struct Kv8Walk {
    int b, item;
    int units, tokens;      // of the branch
    int from;               // first unit of the piece within its item
    int first, n;           // its units of tokens
    int left;               // units of the run from the piece on
    int nth;                // number of the piece
    __device__ __forceinline__ void cut() {
        first = max(0, from - kStart);
        n = max(0, min(units, from + left) - kStart) - first;
    }
    // false where the run has no tokens (its units are an item's start)
    __device__ bool init(const Kv8AttnParams& p, const long long* cum, long long begin, int run) {
        int lo = 0, hi = p.n_branches - 1;                          // the last branch that starts at or before the unit
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (cum[mid] <= begin) lo = mid; else hi = mid - 1;
        }
        b = lo; left = run; nth = 0;
        tokens = kv8_tokens(p, b, false); units = kv8_units<kUnitTokens, kStart>(tokens);
        const unsigned long long within = begin - cum[lo];
        item = (int)(within / (unsigned)units);
        from = (int)(within - (unsigned long long)item * (unsigned)units);
        cut();
        return n > 0;
    }
    __device__ __forceinline__ bool next(const Kv8AttnParams& p) {
        left -= units - from;
        if (left <= kStart) return false;                           // none of the next item's tokens
        ++nth; from = 0;
        if (++item == p.Hkv * p.n_rb) { item = 0; ++b; tokens = kv8_tokens(p, b, false); units = kv8_units<kUnitTokens, kStart>(tokens); }
        cut();
        return true;
    }
    __device__ __forceinline__ bool whole() const { return first == 0 && n == units - kStart; }
    static constexpr int kItemStart = kStart;
};

// The parts of a piece's item, where others have some of it.  A CTA leaves parts of its first and of its last item only, in two
// places of its own; only the first part of an item may be the last of its CTA's run.
struct Kv8Parts {
    int cta0, n;
    bool behind;            // the item begins behind its first CTA's first unit
    __device__ __forceinline__ int slot(int k) const { return 2 * (cta0 + k) + (k == 0 && behind ? 1 : 0); }
};
template <class Walk>
__device__ __forceinline__ Kv8Parts kv8_parts(const Walk& w, const Kv8Run& run) {
    Kv8Parts c;
    if (run.cut) {
        c.cta0 = (int)blockIdx.x - (int)blockIdx.x % run.cut; c.n = (w.units - Walk::kItemStart + run.each - 1) / run.each; c.behind = false;
        return c;
    }
    const long long item = run.begin + (run.n - w.left) - w.from, tokens = item + Walk::kItemStart;
    c.cta0 = (int)(tokens / run.per_cta); c.n = (int)((item + w.units - 1) / run.per_cta) - c.cta0 + 1;
    c.behind = item > c.cta0 * run.per_cta;
    return c;
}

}  // namespace

}  // namespace tts
