// Attention of a few rows per branch (drafted chains and trees, single tokens) over the 8-bit cache.
//
//   out[r] = sum_t softmax_t(scale <q_r, ck_t> sk_t) cv_t sv_t,   codes c and scales s of kv8.cuh
//
// Bound by HBM where a branch has few rows per KV head: a record of 4224 bytes (16 tokens) is read once for all rows
// of the branch.  Work is cut into items (branch, KV head, block of up to 32 stacked rows) of as many units as the branch
// has pages; a CTA of 8 warps owns a contiguous run of all units, warp w takes its pages w, w + 8, .. and works on them
// without meeting the other warps: they come by asynchronous copies into a ring of the warp's own.  At the end of an item
// (or of the run) the warps join their results through shared memory; items cut between CTAs are joined by the last CTA
// to finish one of their parts, which the others leave in global memory.
//
// Per page, with tokens on the M side and rows on the N side of the warp-level matrix instruction m16n8k16 (fp16 operands,
// fp32 sums):
//     S^T[16 tokens][rows] = K Q^T      O^T[128 dims][rows] += V^T P^T
// Codes are exact in fp16, so K and V need no rounding; a row of Q is scaled by a power of two so that bf16 fits fp16 too.
// The scale of K goes into the score; p sv goes into the second product, rounded to fp16 (11 bits) in units of the largest
// power of two in sv so far.  The order in which K's 128 dims are summed and V's tokens are numbered is free, and chosen so
// that a lane's operands are 16-byte runs of the record: lane (g, t) = (lane / 4, lane mod 4) holds, of K, the dims 32 t ..
// 32 t + 31 of the tokens 4 (g / 2) + (g mod 2) and two more, and of V the dims 16 g .. 16 g + 15 of the tokens 4 t .. 4 t + 3.
//
// The running maximum moves only when a score exceeds it by more than 2^8: p <= 2^8 then, and p sv fits fp16 with 2^6 to
// spare.  Sums and accumulators are fp32.
#include <cuda_fp16.h>

#include <type_traits>

#include "kv8.cuh"
#include "launch.cuh"

namespace tts {

namespace {

constexpr float kFar = -1e30f;                                      // "no key yet": finite, so that differences are never NaN
constexpr float kSlack = 8.f;                                       // log2 of how far a score may exceed the running maximum
constexpr int kRoom = 6;                                            // p sv is held times 2^kRoom

// Warps of a CTA and pages that each has in its ring, for up to 8 kNB rows, and the shared memory (bytes).  The sums of O take
// 32 kNB registers a thread: with one group of rows 12 warps fit the register file, else 8.
template <int kNB>
struct Lay {
    static constexpr int kWarps = kNB == 1 ? 12 : 8, kThreads = kWarps * 32;
    static constexpr int kStages = kNB == 1 ? 3 : kNB == 2 ? 5 : 4;
    static constexpr int kOffQ = kWarps * kStages * kKv8Record;     // (behind the ring) [rows][256]: fp16 rows, 16-byte chunks exchanged (q_place)
    static constexpr int kRows = kNB * 8;
    static constexpr int kOffMask = kOffQ + kRows * 256;            // [rows] which of the branch's last rows each row sees
    static constexpr int kOffFactor = kOffMask + kRows * 8;         // [rows] what a row's scores are multiplied by
    static constexpr int kOffRowAt = kOffFactor + kRows * 4;        // [rows] (branch, row, head) of the results, as one number
    static constexpr int kOffMl = kOffRowAt + kRows * 4;            // [warps][rows] (maximum, sum)
    static constexpr int kOffTotal = kOffMl + kWarps * kRows * 8;   // [rows] of all warps
    static constexpr int kOffBack = kOffTotal + kRows * 8;          // [warps][rows] what a warp's sums are multiplied by
    static constexpr int kOffExp = kOffBack + kWarps * kRows * 4;   // [warps] exponent of the sums' unit; then a flag
    static constexpr int kOffCum = kOffExp + 64;                    // [branches + 1] units before each branch
    static constexpr int kOffJoin = kOffCum + (kMaxBranches + 8) * 8;   // [warps][rows][64] floats
    static constexpr int kBytes = kOffJoin + kWarps * kRows * 64 * 4;
    static_assert(kBytes <= 232448 && kOffJoin % 16 == 0 && kWarps * 4 + 4 <= 64, "shared memory of a CTA");
};

// Where chunk (u, t) of a row of Q lies (8 halves: dims 32 t + 8 u ..), so that the lanes of a quarter warp, two rows and
// four t of one u, read eight different bank groups.
__device__ __forceinline__ int q_place(int u, int t, int row) { return (u * 4 + t) ^ ((row & 1) << 2); }

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// 16 bytes to shared memory, asynchronously; zeros where `there` is false
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ float exp2_approx(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float log2_approx(float x) { float y; asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ uint64_t pack2(float a, float b) { uint64_t r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float2 unpack2(uint64_t v) { float2 r; asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v)); return r; }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) { uint64_t r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) { uint64_t r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) { uint64_t r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }      // -126 <= e <= 127
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// A place in the list of units: unit `page` of item `item` (KV head * n_rb + row block) of branch b.
struct Place { int b, item, page, units, tokens; };

// Tokens of a branch; a bad length raises the status and counts as an empty branch.
__device__ __forceinline__ int branch_tokens(const Kv8AttnParams& p, int b, bool raise) {
    const int L = p.branch_lens[b];
    const long n = (long)p.prefix_len + L;
    if (L < 0 || n > (long)p.max_blocks * kPage) {
        if (raise) atomicMin(p.status, (int)TTS_ERR_DEVICE_BOUNDS);
        return 0;
    }
    return (int)n;
}
__device__ __forceinline__ int units_of(int tokens) { return max(1, (tokens + kPage - 1) / kPage); }

// Units before each branch (per KV head and row block together), in 64 bits; all threads of the block.
template <int kThreads>
__device__ void scan_units(const Kv8AttnParams& p, long long* cum, long long* warp_sums) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = p.Hkv * p.n_rb;
    long long carry = 0;
    for (int base = 0; base < p.n_branches; base += kThreads) {
        const int b = base + threadIdx.x;
        long long v = b < p.n_branches ? (long long)units_of(branch_tokens(p, b, blockIdx.x == 0)) * per : 0;
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

__device__ __forceinline__ void load_branch(const Kv8AttnParams& p, Place& at) {
    at.tokens = branch_tokens(p, at.b, false);
    at.units = units_of(at.tokens);
}
__device__ Place place_of(const Kv8AttnParams& p, const long long* cum, long long unit) {
    int lo = 0, hi = p.n_branches - 1;                              // the last branch that starts at or before the unit
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (cum[mid] <= unit) lo = mid; else hi = mid - 1;
    }
    Place at;
    at.b = lo;
    load_branch(p, at);
    const unsigned within = (unsigned)(unit - cum[lo]);            // (of one branch: below 2^31)
    at.item = (int)(within / (unsigned)at.units);
    at.page = (int)(within - (unsigned)at.item * (unsigned)at.units);
    return at;
}
// `n` units further (the caller knows that they are there)
__device__ __forceinline__ void advance(const Kv8AttnParams& p, Place& at, int n) {
    at.page += n;
    while (at.page >= at.units) {
        at.page -= at.units;
        if (++at.item == p.Hkv * p.n_rb) { at.item = 0; ++at.b; load_branch(p, at); }
    }
}

// S^T = K Q^T of one page: s[n][j], j: (token a or b) * 2 + (row 2 t or 2 t + 1)
template <int kFormat, int kNB>
__device__ __forceinline__ void scores(const unsigned char* rec, const unsigned char* q_rows, int g, int t, float (&s)[kNB][4]) {
    const int tok_a = 4 * (g >> 1) + (g & 1), tok_b = tok_a + 2;    // both have chunk_place g
    uint4 xa[2], xb[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const int place = ((2 * t + c) ^ g) * 16;
        xa[c] = *reinterpret_cast<const uint4*>(rec + tok_a * kHeadDim + place);
        xb[c] = *reinterpret_cast<const uint4*>(rec + tok_b * kHeadDim + place);
    }
#pragma unroll
    for (int n = 0; n < kNB; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[n][j] = 0.f;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const uint32_t wa[4] = {xa[c].x, xa[c].y, xa[c].z, xa[c].w}, wb[4] = {xb[c].x, xb[c].y, xb[c].z, xb[c].w};
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint32_t a[2][4];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t x = kv8_biased<kFormat>(wa[2 * half + k]), y = kv8_biased<kFormat>(wb[2 * half + k]);
                a[k][0] = kv8_decode2<kFormat>(x, 0); a[k][2] = kv8_decode2<kFormat>(x, 1);
                a[k][1] = kv8_decode2<kFormat>(y, 0); a[k][3] = kv8_decode2<kFormat>(y, 1);
            }
#pragma unroll
            for (int n = 0; n < kNB; ++n) {
                const uint4 q = *reinterpret_cast<const uint4*>(q_rows + (n * 8 + g) * 256 + q_place(2 * c + half, t, g) * 16);
                mma(s[n], a[0][0], a[0][1], a[0][2], a[0][3], q.x, q.y);
                mma(s[n], a[1][0], a[1][1], a[1][2], a[1][3], q.z, q.w);
            }
        }
    }
}

template <int kFormat, int kNB>
__global__ void __launch_bounds__(Lay<kNB>::kThreads, 1)
kv8_attn_kernel(const __grid_constant__ Kv8AttnParams p) {
    using L = Lay<kNB>;
    constexpr int kWarps = L::kWarps, kThreads = L::kThreads, kStages = L::kStages, kRows = L::kRows;
    extern __shared__ __align__(128) unsigned char smem[];
    long long* cum = reinterpret_cast<long long*>(smem + L::kOffCum);
    unsigned char* q_rows = smem + L::kOffQ;
    unsigned long long* masks = reinterpret_cast<unsigned long long*>(smem + L::kOffMask);
    float* factors = reinterpret_cast<float*>(smem + L::kOffFactor);
    int* row_at = reinterpret_cast<int*>(smem + L::kOffRowAt);
    float2* ml = reinterpret_cast<float2*>(smem + L::kOffMl);
    float2* totals = reinterpret_cast<float2*>(smem + L::kOffTotal);
    float* backs = reinterpret_cast<float*>(smem + L::kOffBack);
    int* exps = reinterpret_cast<int*>(smem + L::kOffExp);
    float* join = reinterpret_cast<float*>(smem + L::kOffJoin);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;

    grid_dependency_wait();
    grid_launch_dependents();
    scan_units<kThreads>(p, cum, reinterpret_cast<long long*>(join));
    const long long total = cum[p.n_branches];
    const long long per_cta = max((long long)kWarps, (total + gridDim.x - 1) / gridDim.x);       // at least a page for each warp
    const long long begin = (long long)blockIdx.x * per_cta;
    if (begin >= total) return;
    const int n_units = (int)min(total - begin, per_cta);           // (at most 2^26 pages of 1024 branches x 128 heads x 2 row blocks over 148 CTAs)

    // ---- the warp's own pages: begin + warp, + 8, ..; `next` runs kStages ahead of the work
    unsigned char* ring = smem + warp * kStages * kKv8Record;
    Place next = place_of(p, cum, begin + min(warp, n_units - 1));
    int next_unit = warp;                                           // (counted from `begin`, as all units below)
    int next_page = -1;                                             // of the pool, asked for one copy ahead
    auto look_up = [&]() {
        next_page = -1;
        if (next_unit < n_units && next.page * kPage < next.tokens) next_page = p.block_table[(size_t)next.b * p.max_blocks + next.page];
    };
    auto copy = [&](int stage) {                                    // the page that was looked up, and on to the one after it
        if (next_unit < n_units) {
            const bool there = next_page >= 0 && next_page < p.num_pages;
            if (!there && next.page * kPage < next.tokens && lane == 0) atomicMin(p.status, (int)TTS_ERR_DEVICE_BOUNDS);
            const unsigned char* src = p.pool + ((size_t)(there ? next_page : 0) * p.Hkv + next.item / p.n_rb) * kKv8Record + lane * 16;
            const uint32_t dst = smem_u32(ring + stage * kKv8Record) + lane * 16;
#pragma unroll
            for (int i = 0; i < kKv8Record / 512; ++i) copy16(dst + i * 512, src + i * 512, there);
            if (lane < (kKv8Record % 512) / 16) copy16(dst + kKv8Record / 512 * 512, src + kKv8Record / 512 * 512, there);
            next_unit += kWarps;
            if (next_unit < n_units) advance(p, next, kWarps);
            look_up();
        }
        copy_commit();
    };
    look_up();
#pragma unroll
    for (int i = 0; i < kStages; ++i) copy(i);
    int stage = 0;

    Place item = place_of(p, cum, begin);                           // the item that is worked on, at its first unit here
    // rows warp, warp + kWarps, .. of the item's queries (4 dims a lane), asked for ahead
    constexpr int kQPer = (kRows + kWarps - 1) / kWarps;
    uint2 q_raw[kQPer];
    auto ask_q = [&]() {
        const int h = item.item / p.n_rb, row0 = (item.item - h * p.n_rb) * p.rb_rows, rows = min(p.rb_rows, p.nr - row0);
#pragma unroll
        for (int k = 0; k < kQPer; ++k) {
            const int r = warp + k * kWarps, stacked = row0 + r, i = stacked / p.G, head = h * p.G + stacked - i * p.G;
            q_raw[k] = make_uint2(0, 0);
            if (r < rows) q_raw[k] = *reinterpret_cast<const uint2*>(p.q + ((size_t)item.b * p.R + i) * p.q_stride + (size_t)head * kHeadDim + lane * 4);
        }
    };
    ask_q();
    int unit = 0;
    for (int nth = 0; unit < n_units; ++nth) {
        const int h = item.item / p.n_rb, rb = item.item - h * p.n_rb, b = item.b;
        const int row0 = rb * p.rb_rows, rows = min(p.rb_rows, p.nr - row0), tokens = item.tokens, units = item.units;
        const int item_begin = unit - item.page, stop = min(n_units, item_begin + units);
        const int tail = tokens - p.R;                              // the first of the branch's last R tokens (may be negative)

        // ---- Q, scaled to fp16 by the power of two that puts a row's largest at 2^14
#pragma unroll
        for (int k = 0; k < kQPer; ++k) {
            const int r = warp + k * kWarps;
            if (r >= kRows) break;
            const uint2 x = q_raw[k];
            const float f[4] = {__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xffff0000u), __uint_as_float(x.y << 16), __uint_as_float(x.y & 0xffff0000u)};
            int top = 0;                                            // the largest finite magnitude, as bits
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int bits = __float_as_int(f[j]) & 0x7fffffff;
                top = max(top, bits < 0x7f800000 ? bits : 0);
            }
            const int e = max(-100, min(126, (__reduce_max_sync(0xffffffffu, top) >> 23) - 127)) - 14;
            const float down = power_of_two(-e);
            // dims 4 lane ..: chunk (u, t) = ((lane / 2) mod 4, lane / 8), half lane mod 2
            *reinterpret_cast<uint2*>(q_rows + r * 256 + q_place((lane >> 1) & 3, lane >> 3, r) * 16 + (lane & 1) * 8) =
                make_uint2(pack_half2(f[0] * down, f[1] * down), pack_half2(f[2] * down, f[3] * down));
            if (lane == 0) {
                const int stacked = row0 + r, i = stacked / p.G;
                factors[r] = r < rows ? power_of_two(e) * p.scale_log2 : 0.f;
                row_at[r] = (b * p.R + i) * p.Hq + h * p.G + stacked - i * p.G;
                unsigned long long m = 0;
                if (r < rows) {
                    if (p.tree_parents == nullptr) m = i >= 63 ? ~0ull : (2ull << i) - 1ull;
                    else
                        for (int a = i, guard = 0; a >= 0 && guard < kMaxTreeRows; ++guard) {
                            m |= 1ull << a;
                            const int parent = p.tree_parents[(size_t)b * p.R + a];
                            a = parent < a ? parent : -1;           // malformed parents end the walk
                        }
                }
                masks[r] = m;
            }
        }
        __syncthreads();

        float o[8][kNB][4];
        uint64_t neg_m[kNB], l[kNB], factor[kNB];                   // of rows 2 t and 2 t + 1
        int unit_exp = 7;                                           // exponent field of the power of two that p sv is held in units of,
        float unit_end = 0.f, up = 0.f;                             // a scale from which on it is too small, and its reciprocal times 2^kRoom
#pragma unroll
        for (int n = 0; n < kNB; ++n) {
            neg_m[n] = pack2(-kFar, -kFar); l[n] = 0; factor[n] = pack2(factors[n * 8 + 2 * t], factors[n * 8 + 2 * t + 1]);
#pragma unroll
            for (int d = 0; d < 8; ++d)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[d][n][j] = 0.f;
        }

        // ---- this warp's pages of the item; the next page's scores are under way while a page's probabilities are formed
        const int first_unit = unit + (warp - unit % kWarps + kWarps) % kWarps;
        float s[kNB][4];
        // the page in the ring's stage `at`: it has come, and what it holds beyond the branch's end is made harmless (the codes of V;
        // K's are never looked at, for their scores are replaced)
        auto arrive = [&](auto behind, int at, int left) {           // (copies behind it that may be in flight)
            copy_wait<decltype(behind)::value>();
            __syncwarp();
            if (left < kPage) {
                unsigned char* rec = ring + at * kKv8Record;
                for (int r = max(0, left); r < kPage; ++r) {
                    if (lane < 8) *reinterpret_cast<uint4*>(rec + kKv8Codes + r * kHeadDim + lane * 16) = make_uint4(0, 0, 0, 0);
                    if (lane < 2) reinterpret_cast<float*>(rec + 2 * kKv8Codes)[lane * kPage + r] = 0.f;
                }
                __syncwarp();
            }
        };
        if (first_unit < stop) {
            arrive(std::integral_constant<int, kStages - 1>{}, stage, tokens - (first_unit - item_begin) * kPage);
            scores<kFormat, kNB>(ring + stage * kKv8Record, q_rows, g, t, s);
        }
        for (int u = first_unit; u < stop; u += kWarps) {
            const int first = (u - item_begin) * kPage, left = tokens - first;       // the page's first token; tokens from it on
            const unsigned char* rec = ring + stage * kKv8Record;
            const int after = stage + 1 == kStages ? 0 : stage + 1;
            const int tok_a = 4 * (g >> 1) + (g & 1), tok_b = tok_a + 2;
            const float* scales = reinterpret_cast<const float*>(rec + 2 * kKv8Codes);
            const float ka = scales[tok_a], kb = scales[tok_b], va = scales[kPage + tok_a], vb = scales[kPage + tok_b];
            // d: scores less the running maximum, in log2 units, [row group][token a, b] of rows 2 t and 2 t + 1
            float2 d[kNB][2];
            uint64_t x[kNB][2];
            const uint64_t ka2 = pack2(ka, ka), kb2 = pack2(kb, kb);
#pragma unroll
            for (int n = 0; n < kNB; ++n) {
                x[n][0] = mul2(pack2(s[n][0], s[n][1]), ka2); x[n][1] = mul2(pack2(s[n][2], s[n][3]), kb2);
                d[n][0] = unpack2(fma2(x[n][0], factor[n], neg_m[n])); d[n][1] = unpack2(fma2(x[n][1], factor[n], neg_m[n]));
            }
            unsigned seen = ~0u;                                    // bit 4 n + 2 (token b) + (row 2 t + 1)
            const bool masked = first + kPage > tail;
            if (masked) {
                seen = 0;
#pragma unroll
                for (int n = 0; n < kNB; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int tok = j < 2 ? tok_a : tok_b, a = first + tok - tail;
                        if (tok < left && (a < 0 || (a < 64 && (masks[n * 8 + 2 * t + (j & 1)] >> a & 1)))) seen |= 1u << (4 * n + j);
                        else if (j & 1) d[n][j >> 1].y = -INFINITY;
                        else d[n][j >> 1].x = -INFINITY;
                    }
            }
            float over = -INFINITY;
#pragma unroll
            for (int n = 0; n < kNB; ++n) over = fmaxf(over, fmaxf(fmaxf(d[n][0].x, d[n][0].y), fmaxf(d[n][1].x, d[n][1].y)));
            if (__any_sync(0xffffffffu, over > kSlack || fmaxf(va, vb) >= unit_end)) {
                // ---- seldom: the maximum moves, or the unit (the largest exponent in sv so far; a NaN or an infinity is not a unit)
                const int ea = __float_as_int(va) >> 23 & 255, eb = __float_as_int(vb) >> 23 & 255;
                const int e = max(unit_exp, __reduce_max_sync(0xffffffffu, max(ea == 255 ? 0 : ea, eb == 255 ? 0 : eb)));
                const float unit_back = unit_exp - e < -126 ? 0.f : power_of_two(unit_exp - e);
                unit_exp = e; unit_end = __int_as_float((e + 1) << 23); up = power_of_two(kRoom + 127 - e);
#pragma unroll
                for (int n = 0; n < kNB; ++n) {
                    const float2 xa = unpack2(mul2(x[n][0], factor[n])), xb = unpack2(mul2(x[n][1], factor[n])), old = unpack2(neg_m[n]);
                    const float v[4] = {seen >> (4 * n) & 1 ? xa.x : -INFINITY, seen >> (4 * n + 1) & 1 ? xa.y : -INFINITY,
                                        seen >> (4 * n + 2) & 1 ? xb.x : -INFINITY, seen >> (4 * n + 3) & 1 ? xb.y : -INFINITY};
                    float neg[2], back[2];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float top = fmaxf(v[j], v[2 + j]);
#pragma unroll
                        for (int i = 4; i < 32; i <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, i));
                        const float was = j ? old.y : old.x;
                        neg[j] = fminf(was, -top);
                        back[j] = exp2_approx(neg[j] - was);
                    }
                    d[n][0] = make_float2(v[0] + neg[0], v[1] + neg[1]); d[n][1] = make_float2(v[2] + neg[0], v[3] + neg[1]);
                    neg_m[n] = pack2(neg[0], neg[1]);
                    l[n] = mul2(l[n], pack2(back[0], back[1]));
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) o[i][n][j] *= back[j & 1] * unit_back;
                }
            }
            if (u + kWarps < stop) {
                arrive(std::integral_constant<int, kStages - 2>{}, after, left - kWarps * kPage);
                scores<kFormat, kNB>(ring + after * kKv8Record, q_rows, g, t, s);
            }
            const float fa = va * up, fb = vb * up;
            const uint64_t fa2 = pack2(fa, fa), fb2 = pack2(fb, fb);
            uint32_t pb[kNB][2];                                    // P^T as the B operand: tokens 4 t, 4 t + 1 and 4 t + 2, 4 t + 3 of row g
#pragma unroll
            for (int n = 0; n < kNB; ++n)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint64_t e = pack2(exp2_approx(d[n][j].x), exp2_approx(d[n][j].y));
                    l[n] = add2(l[n], e);
                    float2 w = unpack2(mul2(e, j ? fb2 : fa2));
                    if (masked) {                                   // a hidden token's scale may be a NaN
                        if (!(seen >> (4 * n + 2 * j) & 1)) w.x = 0.f;
                        if (!(seen >> (4 * n + 2 * j + 1) & 1)) w.y = 0.f;
                    }
                    pb[n][j] = transpose8x8(pack_half2(w.x, w.y));
                }
            // O^T += V^T P^T: four bytes (tokens 4 t ..) of dims 2 e, 2 e + 1 of the lane's 16 make the A operand of tile e
            uint4 v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                v[j] = *reinterpret_cast<const uint4*>(rec + kKv8Codes + (4 * t + j) * kHeadDim + (g ^ ((j & 1) | 2 * t)) * 16);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint32_t y[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = kv8_biased<kFormat>(q == 0 ? v[j].x : q == 1 ? v[j].y : q == 2 ? v[j].z : v[j].w);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint32_t lo = __byte_perm(y[0], y[1], half ? 0x7362 : 0x5140), hi = __byte_perm(y[2], y[3], half ? 0x7362 : 0x5140);
                    const uint32_t a0 = kv8_decode2<kFormat>(lo, 0), a1 = kv8_decode2<kFormat>(lo, 1), a2 = kv8_decode2<kFormat>(hi, 0), a3 = kv8_decode2<kFormat>(hi, 1);
#pragma unroll
                    for (int n = 0; n < kNB; ++n) mma(o[2 * q + half][n], a0, a1, a2, a3, pb[n][0], pb[n][1]);
                }
            }
            __syncwarp();                                           // all lanes have read the page
            copy(stage);
            stage = after;
        }

        // ---- join the warps: of every row the maximum and the sum, and from them what each warp's O is multiplied by
        const bool whole = item.page == 0 && stop == item_begin + units;
        const long long item0 = begin + item_begin;
        if (stop < n_units) { advance(p, item, stop - unit); ask_q(); }
        unit = stop;
#pragma unroll
        for (int n = 0; n < kNB; ++n) {
            const float2 sums = unpack2(l[n]), neg = unpack2(neg_m[n]);
            float a = sums.x, z = sums.y;
#pragma unroll
            for (int i = 4; i < 32; i <<= 1) { a += __shfl_xor_sync(0xffffffffu, a, i); z += __shfl_xor_sync(0xffffffffu, z, i); }
            if (g == 0) *reinterpret_cast<float4*>(ml + warp * kRows + n * 8 + 2 * t) = make_float4(-neg.x, a, -neg.y, z);
        }
        if (lane == 0) exps[warp] = unit_exp;
        __syncthreads();
        if (threadIdx.x < kRows) {
            const int r = threadIdx.x;
            float top = kFar, sum = 0.f;
#pragma unroll 4
            for (int w = 0; w < kWarps; ++w) top = fmaxf(top, ml[w * kRows + r].x);
#pragma unroll 4
            for (int w = 0; w < kWarps; ++w) { const float2 x = ml[w * kRows + r]; sum += x.y * exp2_approx(x.x - top); }
            totals[r] = make_float2(top, sum);
            const float inv = sum == 0.f ? 0.f : 1.f / sum;         // (a row that saw nothing: m = kFar and l = 0 everywhere; zeros)
#pragma unroll 4
            for (int w = 0; w < kWarps; ++w) backs[w * kRows + r] = exp2_approx(ml[w * kRows + r].x - top) * inv * power_of_two(exps[w] - 127 - kRoom);
        }
        __syncthreads();
        const int slot = 2 * blockIdx.x + (nth == 0 ? 0 : 1);       // a CTA leaves parts of its first and of its last item only
        auto write_out = [&](int r, int dim, const float4& x) {
            const size_t at = (size_t)row_at[r] * kHeadDim + dim;
            if (p.out_dtype == TTS_OUT_FP32) *reinterpret_cast<float4*>(static_cast<float*>(p.out) + at) = x;
            else {
                const __nv_bfloat162 lo = __floats2bfloat162_rn(x.x, x.y), hi = __floats2bfloat162_rn(x.z, x.w);
                *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + at) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
            }
        };
        auto write_lse = [&](int r, float top, float sum) {         // natural logarithm
            p.lse[row_at[r]] = sum == 0.f ? -INFINITY : (top + log2_approx(sum)) * 0.6931471805599453f;
        };
        float2 back[kNB];
#pragma unroll
        for (int n = 0; n < kNB; ++n) back[n] = *reinterpret_cast<const float2*>(backs + warp * kRows + n * 8 + 2 * t);
#pragma unroll 1
        for (int round = 0; round < 2; ++round) {                   // dims 16 g + 8 round .. + 7 of every g
            auto put = [&](auto half) {
                constexpr int kHalf = decltype(half)::value;
#pragma unroll
                for (int n = 0; n < kNB; ++n)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float4* to = reinterpret_cast<float4*>(join + ((warp * kNB + n) * 8 + 2 * t + j) * 64 + g * 8);
                        const float f = j ? back[n].y : back[n].x;
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const float(&a)[4] = o[4 * kHalf + 2 * k][n], (&z)[4] = o[4 * kHalf + 2 * k + 1][n];
                            to[k] = make_float4(a[j] * f, a[2 + j] * f, z[j] * f, z[2 + j] * f);
                        }
                    }
            };
            if (round == 0) put(std::integral_constant<int, 0>{}); else put(std::integral_constant<int, 1>{});
            __syncthreads();
#pragma unroll 1
            for (int i = threadIdx.x; i < rows * 16; i += kThreads) {
                const int r = i >> 4, c = i & 15, dim = (c >> 1) * 16 + round * 8 + (c & 1) * 4;
                float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    const float4 x = *reinterpret_cast<const float4*>(join + (w * kRows + r) * 64 + c * 4);
                    sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
                }
                if (whole) write_out(r, dim, sum);
                else *reinterpret_cast<float4*>(p.part_o + ((size_t)slot * kKv8MaxRows + r) * kHeadDim + dim) = sum;
            }
            if (round == 0) __syncthreads();
        }
        if (threadIdx.x < rows) {
            const int r = threadIdx.x;
            if (!whole) p.part_ml[slot * kKv8MaxRows + r] = totals[r];
            else if (p.lse) write_lse(r, totals[r].x, totals[r].y);
        }
        __syncthreads();
        if (!whole) {
            // ---- the last CTA to leave a part of the item joins them all
            const int cta0 = (int)(item0 / per_cta), parts = (int)((item0 + units - 1) / per_cta) - cta0 + 1;
            const size_t id = ((size_t)b * p.Hkv + h) * p.n_rb + rb;
            if (threadIdx.x == 0) {
                __threadfence();                                    // the block's writes, which the barrier put before this
                const bool last = atomicAdd(p.arrived + id, 1u) + 1 == (unsigned)parts;
                if (last) p.arrived[id] = 0;                        // as the next call expects it
                __threadfence();
                exps[kWarps] = last;
            }
            __syncthreads();
            if (exps[kWarps]) {
                // a part is the first item of its CTA unless it starts the item behind the CTA's first unit
                auto slot_of = [&](int k) { return 2 * (cta0 + k) + (k == 0 && item0 != cta0 * per_cta ? 1 : 0); };
#pragma unroll 1
                for (int i = threadIdx.x; i < rows * 32; i += kThreads) {
                    const int r = i >> 5, dim = (i & 31) * 4;       // a warp takes a row
                    float top = kFar;
                    for (int k = lane; k < parts; k += 32) top = fmaxf(top, __ldcg(p.part_ml + slot_of(k) * kKv8MaxRows + r).x);
#pragma unroll
                    for (int x = 16; x; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
                    float sum = 0.f;
                    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
                    for (int k = 0; k < parts; ++k) {
                        const size_t at = (size_t)slot_of(k) * kKv8MaxRows + r;
                        const float2 x = __ldcg(p.part_ml + at);
                        const float4 y = __ldcg(reinterpret_cast<const float4*>(p.part_o + at * kHeadDim + dim));
                        const float w = x.y * exp2_approx(x.x - top);
                        sum += w;
                        acc.x += w * y.x; acc.y += w * y.y; acc.z += w * y.z; acc.w += w * y.w;
                    }
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;
                    write_out(r, dim, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
                    if (p.lse && lane == 0) write_lse(r, top, sum);
                }
            }
            __syncthreads();                                        // Q, the masks and the sums are free again
        }
    }
}

}  // namespace

cudaError_t launch_kv8_attn(const Kv8AttnParams& p, int format, cudaStream_t st) {
    auto launch = [&](auto fmt, auto nb) {
        constexpr int kFormat = decltype(fmt)::value, kNB = decltype(nb)::value;
        auto kernel = kv8_attn_kernel<kFormat, kNB>;
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Lay<kNB>::kBytes);
        if (e != cudaSuccess) return e;
        return launch_dependent(kernel, p.grid, Lay<kNB>::kThreads, Lay<kNB>::kBytes, st, p);
    };
    auto by_rows = [&](auto fmt) {
        switch ((p.rb_rows + 7) / 8) {
            case 1: return launch(fmt, std::integral_constant<int, 1>{});
            case 2: return launch(fmt, std::integral_constant<int, 2>{});
            case 3: return launch(fmt, std::integral_constant<int, 3>{});
            default: return launch(fmt, std::integral_constant<int, 4>{});
        }
    };
    return format == TTS_KV8_E4M3 ? by_rows(std::integral_constant<int, TTS_KV8_E4M3>{}) : by_rows(std::integral_constant<int, TTS_KV8_INT8>{});
}

}  // namespace tts
