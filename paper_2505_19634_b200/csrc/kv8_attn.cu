// Attention of a few rows per branch (drafted chains and trees, single tokens) over the 8-bit cache.
//
//   out[r] = sum_t softmax_t(scale <q_r, ck_t> sk_t) cv_t sv_t,   codes c and scales s of kv8.cuh
//
// For up to 48 rows to a KV head (kv8_attn_wide.cu: more).  Bound by HBM: a record of 4224 bytes (16 tokens) is read once for all rows
// of the branch.  Work is cut into items (branch, KV head, block of up to 24 stacked rows; kv8_run.cuh); a CTA of 8 warps (or
// 12) owns a contiguous run of pages, warp w takes its pairs of pages w, w + 8, .. and works on them without meeting the other warps: they
// come by bulk copies into a ring of the warp's own.  At the end of an item (or of the run) the warps join their results through
// shared memory; items cut between CTAs are joined by the last CTA to finish one of their parts, which the others leave in
// global memory.
//
// Measured (B200, copy peak 6538 GB/s): 64 single tokens over 1 k to 8 k keys, 40 / 8 heads, 110 to 118 us by the card = 4.6 to 4.9 TB/s (twelve warps); a drafted step
// of 16 branches with 20 rows to a KV head over 4 k to 5 k keys 55.6 us = 2.5 TB/s; 4 single tokens over 500 keys 9.1 us.  Of eight, a warp takes about 1850 clocks for a
// page of up to 8 rows (1460 without the copies, 950 with nothing but them) and 2240 for 24: conversion, products and exponentials of two
// warps to a scheduler.  A piece of an item costs 16000 clocks besides (queries 3000, the warps' join 9000, that of its parts 3700), a
// third of the drafted step.  Tiles converted for the tensor cores' own products took 88 and 246 us for the first two.
//
// Per page (and two at a time, for what one leaves idle), with tokens on the M side and rows on the N side of the warp-level
// matrix instruction m16n8k16 (fp16 operands, fp32 sums):
//     S^T[16 tokens][rows] = K Q^T      O^T[128 dims][rows] += V^T P^T
// Codes are exact in fp16, so K and V need no rounding; a row of Q is scaled by a power of two so that bf16 fits fp16 too.
// The scale of K goes into the score; p sv goes into the second product, rounded to fp16 (11 bits) in units of the largest
// power of two in sv that the row has seen so far (a token that it does not see is none of its business).  The order in which K's 128 dims are summed and V's tokens are numbered is free, and chosen so
// that a lane's operands are 16-byte runs of the record: lane (g, t) = (lane / 4, lane mod 4) holds, of K, the dims 32 t ..
// 32 t + 31 of the tokens 4 (g / 2) + (g mod 2) and two more, and of V the dims 16 g .. 16 g + 15 of the tokens 4 t .. 4 t + 3.
//
// The running maximum moves only when a score exceeds it by more than 2^8: p <= 2^8 then, and p sv fits fp16 with 2^6 to
// spare.  Sums and accumulators are fp32.
#include <cuda_fp16.h>

#include <type_traits>

#include "kv8_run.cuh"
#include "launch.cuh"
#include "packed.cuh"
#include "umma_ptx.cuh"

namespace tts {

namespace {

using namespace ptx;

constexpr int kPair = 2 * kKv8Record;                               // a warp works on two pages at a time
constexpr float kFar = -1e30f;                                      // "no key yet": finite, so that differences are never NaN
constexpr float kSlack = 8.f;                                       // log2 of how far a score may exceed the running maximum
constexpr int kRoom = 6;                                            // p sv is held times 2^kRoom
constexpr int kLargestUp = 126;                                     // so a unit is 2^(kRoom - 126) or more

// The warps of a CTA for up to 8 kNB rows, the pairs of pages that each has in its ring, and the shared memory (bytes).
template <int kNB, int kCtaWarps>
struct Lay {
    static constexpr int kWarps = kCtaWarps, kThreads = 32 * kWarps;
    static constexpr int kStages = kNB == 1 && kWarps == 8 ? 3 : 2;
    // the join: 16-byte chunks of a row and round, threads to a row
    static constexpr int kRounds = kNB == 2 ? 1 : 2;                // the warps' sums are joined all dims at once, or half of them twice
    static constexpr int kOffQ = kWarps * kStages * kPair;              // (behind the ring) [rows][256]: fp16 rows, 16-byte chunks exchanged (q_place)
    static constexpr int kChunks = 32 / kRounds, kPerRow = kNB <= 2 ? 16 : 8;
    static constexpr int kRows = kNB * 8;
    static constexpr int kOffMask = kOffQ + kRows * 256;            // [rows] which of the branch's last rows each row sees
    static constexpr int kOffFactor = kOffMask + kRows * 8;         // [rows] what a row's scores are multiplied by
    static constexpr int kOffRowAt = kOffFactor + kRows * 4;        // [rows] (branch, row, head) of the results, as one number
    static constexpr int kOffMl = kOffRowAt + kRows * 4;            // [warps][rows] (maximum, sum)
    static constexpr int kOffUnit = kOffMl + kWarps * kRows * 8;    // [warps][rows] the sums' unit, over 2^kRoom
    static constexpr int kOffLast = kOffUnit + kWarps * kRows * 4;  // a flag
    static constexpr int kOffJoin = kOffLast + 64;                  // [warps][rows][128 / rounds] floats
    static constexpr int kOffCum = kOffJoin + 256;                  // [branches + 1] units before each branch, until the first piece is found
    static constexpr int kOffBar = kOffJoin + kWarps * kRows * kHeadDim / kRounds * 4;   // [warps][stages]
    static constexpr int kOffAbort = kOffBar + kWarps * kStages * 8;   // [0] flag; [1 ..] scratch of each warp
    static constexpr int kBytes = kOffAbort + (1 + kWarps) * 4 + 12;
    static_assert(kBytes <= 232448 && kOffJoin % 16 == 0, "shared memory of a CTA");
    static_assert(256 + (kMaxBranches + 1) * 8 <= kWarps * kRows * kHeadDim / kRounds * 4 && kWarps * 8 <= 256, "the branches' units, where the sums will be");
};

// Where chunk c of row r of a warp's sums lies: rows 2 t of the four t of a lane's group, and two groups, hit eight different bank groups.
template <int kRounds>
__device__ __forceinline__ int join_place(int c, int r) { const int t = (r & 7) >> 1; return c ^ (kRounds == 1 ? t : (t & 1) << 2 | t >> 1); }
// Where chunk (u, t) of a row of Q lies (8 halves: dims 32 t + 8 u ..), so that the lanes of a quarter warp, two rows and
// four t of one u, read eight different bank groups.
__device__ __forceinline__ int q_place(int u, int t, int row) { return (u * 4 + t) ^ ((row & 1) << 2); }


__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ float inverse(float power) { return __int_as_float(0x7f000000 - __float_as_int(power)); }      // of 2^-126 .. 2^126

// An item's start and end (queries, join of the warps) take about as long as so many pages (kv8_run.cuh).  64 single tokens of 1024 to
// 8192 keys: 120 us, 125 with 16, 137 with none; a drafted step of 20 rows 55.5, 56.3, 57.3.
constexpr int kItemUnits = 48;
// Of a CTA's share of an item, where items are cut evenly: two to eight for a warp.  One branch of 1000 keys, 40 / 8 heads: 10.1 us with 16 pages to
// a CTA, 12.3 with 64; 16 branches of 500 keys: 10.4 us uncut, 15.5 with 16.
constexpr int kLeastPages = 16, kMostPages = 64;
using Walk = Kv8Walk<kPage, kItemUnits>;

// S^T = K Q^T of two pages: s[page][n][j], j: (token a or b) * 2 + (row 2 t or 2 t + 1)
template <int kFormat, int kNB>
__device__ __forceinline__ void scores(const unsigned char* pair, const unsigned char* q_rows, int g, int t, float (&s)[2][kNB][4]) {
    const int tok_a = 4 * (g >> 1) + (g & 1), tok_b = tok_a + 2;    // both have chunk_place g
#pragma unroll
    for (int pg = 0; pg < 2; ++pg)
#pragma unroll
        for (int n = 0; n < kNB; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[pg][n][j] = 0.f;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const int place = ((2 * t + c) ^ g) * 16;
        uint4 xa[2], xb[2];
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) {
            xa[pg] = *reinterpret_cast<const uint4*>(pair + pg * kKv8Record + tok_a * kHeadDim + place);
            xb[pg] = *reinterpret_cast<const uint4*>(pair + pg * kKv8Record + tok_b * kHeadDim + place);
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint32_t a[2][2][4];
#pragma unroll
            for (int pg = 0; pg < 2; ++pg)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t x = kv8_biased<kFormat>(half == 0 ? (k == 0 ? xa[pg].x : xa[pg].y) : (k == 0 ? xa[pg].z : xa[pg].w));
                    const uint32_t y = kv8_biased<kFormat>(half == 0 ? (k == 0 ? xb[pg].x : xb[pg].y) : (k == 0 ? xb[pg].z : xb[pg].w));
                    a[pg][k][0] = kv8_decode2<kFormat>(x, 0); a[pg][k][2] = kv8_decode2<kFormat>(x, 1);
                    a[pg][k][1] = kv8_decode2<kFormat>(y, 0); a[pg][k][3] = kv8_decode2<kFormat>(y, 1);
                }
            uint4 q[kNB];
#pragma unroll
            for (int n = 0; n < kNB; ++n) q[n] = *reinterpret_cast<const uint4*>(q_rows + (n * 8 + g) * 256 + q_place(2 * c + half, t, g) * 16);
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int n = 0; n < kNB; ++n)
#pragma unroll
                    for (int pg = 0; pg < 2; ++pg)
                        mma(s[pg][n], a[pg][k][0], a[pg][k][1], a[pg][k][2], a[pg][k][3], k == 0 ? q[n].x : q[n].z, k == 0 ? q[n].y : q[n].w);
        }
    }
}

template <int kFormat, int kNB, int kCtaWarps>
__global__ void __launch_bounds__(32 * kCtaWarps, 1)
kv8_attn_kernel(const __grid_constant__ Kv8AttnParams p) {
    using L = Lay<kNB, kCtaWarps>;
    constexpr int kWarps = L::kWarps, kThreads = L::kThreads, kStages = L::kStages, kRows = L::kRows;
    extern __shared__ __align__(128) unsigned char smem[];
    long long* cum = reinterpret_cast<long long*>(smem + L::kOffCum);
    unsigned char* q_rows = smem + L::kOffQ;
    unsigned long long* masks = reinterpret_cast<unsigned long long*>(smem + L::kOffMask);
    float* factors = reinterpret_cast<float*>(smem + L::kOffFactor);
    int* row_at = reinterpret_cast<int*>(smem + L::kOffRowAt);
    float2* ml = reinterpret_cast<float2*>(smem + L::kOffMl);
    float* units = reinterpret_cast<float*>(smem + L::kOffUnit);
    int* is_last = reinterpret_cast<int*>(smem + L::kOffLast);
    float* join = reinterpret_cast<float*>(smem + L::kOffJoin);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;

    if (threadIdx.x < kWarps * kStages) mbar_init(smem_u32(smem + L::kOffBar) + threadIdx.x * 8, 1);
    if (threadIdx.x == 0) *reinterpret_cast<int*>(smem + L::kOffAbort) = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async();
    grid_dependency_wait();
    grid_launch_dependents();
    kv8_scan_units<kThreads, kPage, kItemUnits>(p, cum, reinterpret_cast<long long*>(join));
    const Kv8Run run = kv8_run<kThreads, kItemUnits>(p, cum, reinterpret_cast<int*>(join), kLeastPages, kMostPages);
    const long long begin = run.begin;
    const int n_units = run.n;
    if (n_units <= 0) return;

    // ---- the warp's own pairs: of all pairs of the run's pieces, laid end to end, warp, warp + 8, ..; `ahead` runs kStages ahead
    unsigned char* ring = smem + warp * kStages * kPair;
    const uint32_t bars = smem_u32(smem + L::kOffBar) + warp * kStages * 8;
    volatile int* flags = reinterpret_cast<volatile int*>(smem + L::kOffAbort);
    const Abort ab{flags, p.status};
    bool alive = true;                                              // no wait has run out; else the work goes on with whatever is there
    Walk item, ahead;
    if (!item.init(p, cum, begin, n_units)) return;
    ahead = item;
    int ahead_pair = warp;
    bool more = true;
    int next_page = -1;                                             // lanes 0 and 1: the pool's page, asked for one copy ahead
    unsigned flying = 0, phases = 0;                                // bit of a stage: a copy into it has not been waited for; its barrier's phase
    auto pairs_of = [](const Walk& w) { return (w.n + 1) >> 1; };
    auto look_up = [&]() {                                          // where the next pair is
        while (ahead_pair >= pairs_of(ahead)) {
            ahead_pair -= pairs_of(ahead);
            more = ahead.next(p);
            if (!more) return;
        }
        const int page = 2 * ahead_pair + lane;                     // (of the piece)
        next_page = -1;
        if (lane < 2 && page < ahead.n && (ahead.first + page) * kPage < ahead.tokens)
            next_page = p.block_table[(size_t)ahead.b * p.max_blocks + ahead.first + page];
    };
    auto copy = [&](int stage) {                                    // the pair that was looked up, and on to the one after it
        if (more && alive) {
            unsigned char* dst = ring + stage * kPair;
            const uint32_t bar = bars + stage * 8;
            const bool wanted = lane < 2 && 2 * ahead_pair + lane < ahead.n && (ahead.first + 2 * ahead_pair + lane) * kPage < ahead.tokens;
            const bool there = next_page >= 0 && next_page < p.num_pages && wanted;
            const unsigned good = __ballot_sync(0xffffffffu, there), bad = __ballot_sync(0xffffffffu, wanted && !there);
            if (bad) {                                              // a page outside the pool counts as zeros
                if (lane == 0) atomicMin(p.status, (int)TTS_ERR_DEVICE_BOUNDS);
                for (int i = lane; i < kPair / 16; i += 32)
                    if (bad >> (i >= kKv8Record / 16) & 1) *reinterpret_cast<uint4*>(dst + i * 16) = make_uint4(0, 0, 0, 0);
                fence_proxy_async();                                // (before a later copy into the stage)
                __syncwarp();
            }
            if (lane == 0) { if (good) mbar_arrive_expect_tx(bar, __popc(good) * kKv8Record); else mbar_arrive(bar); }
            __syncwarp();
            if (there) bulk_load(smem_u32(dst) + lane * kKv8Record, p.pool + ((size_t)next_page * p.Hkv + ahead.item / p.n_rb) * kKv8Record, kKv8Record, bar);
            flying |= 1u << stage;
            ahead_pair += kWarps;
            look_up();
        }
    };
    look_up();
#pragma unroll 1
    for (int i = 0; i < kStages; ++i) copy(i);
    int stage = 0, pairs_before = 0;                                // pairs of the run before the piece

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
    for (bool more_items = true; more_items;) {
        const int h = item.item / p.n_rb, rb = item.item - h * p.n_rb, b = item.b;
        const int row0 = rb * p.rb_rows, rows = min(p.rb_rows, p.nr - row0), tokens = item.tokens;
        const int page0 = item.first, pages = item.n, pairs = pairs_of(item), nth = item.nth;
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
        uint64_t up[kNB];                                           // 2^kRoom over the power of two that p sv is held in units of
        float unit_end = 0.f;                                       // a scale from which on the smallest of all rows' units is too small
#pragma unroll
        for (int n = 0; n < kNB; ++n) {
            neg_m[n] = pack2(-kFar, -kFar); l[n] = 0; up[n] = pack2(power_of_two(kLargestUp), power_of_two(kLargestUp)); factor[n] = pack2(factors[n * 8 + 2 * t], factors[n * 8 + 2 * t + 1]);
#pragma unroll
            for (int d = 0; d < 8; ++d)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[d][n][j] = 0.f;
        }

        // ---- this warp's pairs of the piece
        for (int u = (warp - pairs_before % kWarps + kWarps) % kWarps; u < pairs; u += kWarps) {
            const int first = (page0 + 2 * u) * kPage;              // the first token
            const int left = min(tokens - first, min(2, pages - 2 * u) * kPage);       // tokens here, at most 32 (may be 0)
            unsigned char* pair = ring + stage * kPair;
            if (flying >> stage & 1) {
                alive = alive && mbar_wait(bars + stage * 8, phases >> stage & 1, ab);
                alive = __all_sync(0xffffffffu, alive);
                if (alive) { flying &= ~(1u << stage); phases ^= 1u << stage; }
            }
            const bool masked = first + 2 * kPage > tail || left < 2 * kPage;
            if (left < 2 * kPage) {                                 // what is not there is made harmless: V's codes and all scales (K's scores are replaced)
                for (int r = max(0, left); r < 2 * kPage; ++r) {
                    unsigned char* rec = pair + (r >> 4) * kKv8Record;
                    if (lane < 8) *reinterpret_cast<uint4*>(rec + kKv8Codes + (r & 15) * kHeadDim + lane * 16) = make_uint4(0, 0, 0, 0);
                    if (lane < 2) reinterpret_cast<float*>(rec + 2 * kKv8Codes)[lane * kPage + (r & 15)] = 0.f;
                }
                fence_proxy_async();                                // (before the next copy into the stage)
                __syncwarp();
            }
            float s[2][kNB][4];
            scores<kFormat, kNB>(pair, q_rows, g, t, s);
            const int tok_a = 4 * (g >> 1) + (g & 1), tok_b = tok_a + 2;
            float sk[2][2], sv[2][2];                               // [page][token a, b]
#pragma unroll
            for (int pg = 0; pg < 2; ++pg) {
                const float* scales = reinterpret_cast<const float*>(pair + pg * kKv8Record + 2 * kKv8Codes);
                sk[pg][0] = scales[tok_a]; sk[pg][1] = scales[tok_b]; sv[pg][0] = scales[kPage + tok_a]; sv[pg][1] = scales[kPage + tok_b];
            }
            // d: scores less the running maximum, in log2 units, [page][row group][token a, b] of rows 2 t and 2 t + 1
            float2 d[2][kNB][2];
            uint64_t x[2][kNB][2];
            float over = -INFINITY;
#pragma unroll
            for (int pg = 0; pg < 2; ++pg)
#pragma unroll
                for (int n = 0; n < kNB; ++n)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        x[pg][n][j] = mul2(pack2(s[pg][n][2 * j], s[pg][n][2 * j + 1]), pack2(sk[pg][j], sk[pg][j]));
                        d[pg][n][j] = unpack2(fma2(x[pg][n][j], factor[n], neg_m[n]));
                    }
            unsigned seen = ~0u;                                    // bit 16 page + 4 n + 2 (token b) + (row 2 t + 1)
            if (masked) {
                seen = 0;
#pragma unroll
                for (int pg = 0; pg < 2; ++pg)
#pragma unroll
                    for (int n = 0; n < kNB; ++n)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int tok = pg * kPage + (j < 2 ? tok_a : tok_b), a = first + tok - tail;
                            if (tok < left && (a < 0 || (a < 64 && (masks[n * 8 + 2 * t + (j & 1)] >> a & 1)))) seen |= 1u << (16 * pg + 4 * n + j);
                            else if (j & 1) d[pg][n][j >> 1].y = -INFINITY;
                            else d[pg][n][j >> 1].x = -INFINITY;
                        }
            }
#pragma unroll
            for (int pg = 0; pg < 2; ++pg)
#pragma unroll
                for (int n = 0; n < kNB; ++n) over = fmaxf(over, fmaxf(fmaxf(d[pg][n][0].x, d[pg][n][0].y), fmaxf(d[pg][n][1].x, d[pg][n][1].y)));
            const float sv_top = fmaxf(fmaxf(sv[0][0], sv[0][1]), fmaxf(sv[1][0], sv[1][1]));
            if (__any_sync(0xffffffffu, over > kSlack || sv_top >= unit_end)) {
                // ---- seldom: the maximum moves, or a row's unit (the largest power of two in the sv that it sees so far; a NaN or an infinity is none)
                float pow2[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) { const int e = __float_as_int(sv[k >> 1][k & 1]) & 0x7f800000; pow2[k] = e == 0x7f800000 ? 0.f : __int_as_float(e); }
                float most_up = 0.f;                                // the largest of all rows
#pragma unroll
                for (int n = 0; n < kNB; ++n) {
                    const float2 old = unpack2(neg_m[n]), up_old = unpack2(up[n]);
                    float v[2][4], neg[2], back[2], up_new[2], unit_back[2];
#pragma unroll
                    for (int pg = 0; pg < 2; ++pg) {
                        const float2 xa = unpack2(mul2(x[pg][n][0], factor[n])), xb = unpack2(mul2(x[pg][n][1], factor[n]));
                        const float y[4] = {xa.x, xa.y, xb.x, xb.y};
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[pg][j] = seen >> (16 * pg + 4 * n + j) & 1 ? y[j] : -INFINITY;
                    }
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float top = fmaxf(fmaxf(v[0][j], v[0][2 + j]), fmaxf(v[1][j], v[1][2 + j])), unit = 0.f;
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (seen >> (16 * (k >> 1) + 4 * n + 2 * (k & 1) + j) & 1) unit = fmaxf(unit, pow2[k]);
#pragma unroll
                        for (int i = 4; i < 32; i <<= 1) { top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, i)); unit = fmaxf(unit, __shfl_xor_sync(0xffffffffu, unit, i)); }
                        // (powers of two: their exponent fields are added and taken apart)
                        const int was_up = __float_as_int(j ? up_old.y : up_old.x) >> 23, now_up = min(was_up, kRoom + 254 - (__float_as_int(unit) >> 23));
                        up_new[j] = __int_as_float(now_up << 23);
                        unit_back[j] = now_up - was_up < -126 ? 0.f : power_of_two(now_up - was_up);
                        most_up = fmaxf(most_up, up_new[j]);
                        const float was = j ? old.y : old.x;
                        neg[j] = fminf(was, -top);
                        back[j] = ex2(neg[j] - was);
                    }
#pragma unroll
                    for (int pg = 0; pg < 2; ++pg) {
                        d[pg][n][0] = make_float2(v[pg][0] + neg[0], v[pg][1] + neg[1]);
                        d[pg][n][1] = make_float2(v[pg][2] + neg[0], v[pg][3] + neg[1]);
                    }
                    neg_m[n] = pack2(neg[0], neg[1]); up[n] = pack2(up_new[0], up_new[1]);
                    l[n] = mul2(l[n], pack2(back[0], back[1]));
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) o[i][n][j] *= back[j & 1] * unit_back[j & 1];
                }
                // (all lanes of a t agree on their rows already)
                most_up = fmaxf(most_up, __shfl_xor_sync(0xffffffffu, most_up, 1));
                most_up = fmaxf(most_up, __shfl_xor_sync(0xffffffffu, most_up, 2));
                unit_end = __int_as_float((kRoom + 255 - (__float_as_int(most_up) >> 23)) << 23);
            }
            uint32_t pb[2][kNB][2];                                 // P^T as the B operand: tokens 4 t, 4 t + 1 and 4 t + 2, 4 t + 3 of row g
#pragma unroll
            for (int pg = 0; pg < 2; ++pg)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint64_t f = pack2(sv[pg][j], sv[pg][j]);
#pragma unroll
                    for (int n = 0; n < kNB; ++n) {
                        const uint64_t e = pack2(ex2(d[pg][n][j].x), ex2(d[pg][n][j].y));
                        l[n] = add2(l[n], e);
                        float2 w = unpack2(mul2(e, mul2(f, up[n])));
                        if (masked) {                               // a hidden token's scale may be a NaN
                            if (!(seen >> (16 * pg + 4 * n + 2 * j) & 1)) w.x = 0.f;
                            if (!(seen >> (16 * pg + 4 * n + 2 * j + 1) & 1)) w.y = 0.f;
                        }
                        pb[pg][n][j] = transpose8x8(pack_half2(w.x, w.y));
                    }
                }
            // O^T += V^T P^T: four bytes (tokens 4 t ..) of dims 2 e, 2 e + 1 of the lane's 16 make the A operand of tile e
#pragma unroll
            for (int pg = 0; pg < 2; ++pg) {
                uint4 v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    v[j] = *reinterpret_cast<const uint4*>(pair + pg * kKv8Record + kKv8Codes + (4 * t + j) * kHeadDim + (g ^ ((j & 1) | 2 * t)) * 16);
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
                        for (int n = 0; n < kNB; ++n) mma(o[2 * q + half][n], a0, a1, a2, a3, pb[pg][n][0], pb[pg][n][1]);
                    }
                }
            }
            __syncwarp();                                           // all lanes have read the pair
            copy(stage);
            stage = stage + 1 == kStages ? 0 : stage + 1;
        }

        // ---- join the warps: maxima, sums and O of every row
        const bool whole = item.whole();
        const Kv8Parts cut = kv8_parts(item, run);
        pairs_before += pairs;
        more_items = item.next(p);
        if (more_items) ask_q();
#pragma unroll
        for (int n = 0; n < kNB; ++n) {
            const float2 sums = unpack2(l[n]), neg = unpack2(neg_m[n]);
            float a = sums.x, z = sums.y;
#pragma unroll
            for (int i = 4; i < 32; i <<= 1) { a += __shfl_xor_sync(0xffffffffu, a, i); z += __shfl_xor_sync(0xffffffffu, z, i); }
            if (g == 0) {
                const float2 u = unpack2(up[n]);
                *reinterpret_cast<float4*>(ml + warp * kRows + n * 8 + 2 * t) = make_float4(-neg.x, a, -neg.y, z);
                *reinterpret_cast<float2*>(units + warp * kRows + n * 8 + 2 * t) = make_float2(inverse(u.x), inverse(u.y));
            }
        }
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
        // kPerRow threads to a row: what each warp's sums are multiplied by
        const int r = threadIdx.x / L::kPerRow, c0 = threadIdx.x % L::kPerRow;
        float back[kWarps];
#pragma unroll 1
        for (int round = 0; round < L::kRounds; ++round) {          // all dims, or 16 g + 8 round .. + 7 of every g
            auto put = [&](auto half) {
                constexpr int kHalf = decltype(half)::value;
#pragma unroll
                for (int n = 0; n < kNB; ++n)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int row = n * 8 + 2 * t + j;
                        float4* to = reinterpret_cast<float4*>(join + (warp * kRows + row) * (L::kChunks * 4));
#pragma unroll
                        for (int k = 0; k < 4 / L::kRounds; ++k) {
                            const float(&a)[4] = o[4 * kHalf + 2 * k][n], (&z)[4] = o[4 * kHalf + 2 * k + 1][n];
                            to[join_place<L::kRounds>(g * (4 / L::kRounds) + k, row)] = make_float4(a[j], a[2 + j], z[j], z[2 + j]);
                        }
                    }
            };
            if (round == 0) put(std::integral_constant<int, 0>{});
            if constexpr (L::kRounds == 2) { if (round == 1) put(std::integral_constant<int, 1>{}); }
            __syncthreads();
            if (r < rows) {
                if (round == 0) {
                    float top = kFar, sum = 0.f;
                    float2 x[kWarps];
#pragma unroll
                    for (int w = 0; w < kWarps; ++w) { x[w] = ml[w * kRows + r]; top = fmaxf(top, x[w].x); }
#pragma unroll
                    for (int w = 0; w < kWarps; ++w) { back[w] = ex2(x[w].x - top); sum += x[w].y * back[w]; }
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;      // (a row that saw nothing: m = kFar and l = 0 everywhere; zeros)
#pragma unroll
                    for (int w = 0; w < kWarps; ++w) back[w] *= inv * units[w * kRows + r];
                    if (c0 == 0) {
                        if (!whole) p.part_ml[slot * p.rb_rows + r] = make_float2(top, sum);
                        else if (p.lse) write_lse(r, top, sum);
                    }
                }
#pragma unroll 1
                for (int c = c0; c < L::kChunks; c += L::kPerRow) {
                    const int dim = L::kRounds == 1 ? c * 4 : (c >> 1) * 16 + round * 8 + (c & 1) * 4;
                    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                    for (int w = 0; w < kWarps; ++w) {
                        const float4 x = *reinterpret_cast<const float4*>(join + ((w * kRows + r) * L::kChunks + join_place<L::kRounds>(c, r)) * 4);
                        sum.x = fmaf(x.x, back[w], sum.x); sum.y = fmaf(x.y, back[w], sum.y); sum.z = fmaf(x.z, back[w], sum.z); sum.w = fmaf(x.w, back[w], sum.w);
                    }
                    if (whole) write_out(r, dim, sum);
                    else *reinterpret_cast<float4*>(p.part_o + ((size_t)slot * p.rb_rows + r) * kHeadDim + dim) = sum;
                }
            }
            __syncthreads();
        }
        if (!whole) {
            // ---- the last CTA to leave a part of the item joins them all
            const size_t id = ((size_t)b * p.Hkv + h) * p.n_rb + rb;
            if (threadIdx.x == 0) {
                // (releases the block's writes, which the barrier put before it, and acquires the others')
                unsigned before;
                asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(before) : "l"(p.arrived + id) : "memory");
                const bool last = before + 1 == (unsigned)cut.n;
                if (last) p.arrived[id] = 0;                        // as the next call expects it
                *is_last = last;
            }
            __syncthreads();
            if (*is_last) {
                if (r < rows) {
                    float top = kFar, sum = 0.f;
                    float4 acc[32 / L::kPerRow];
#pragma unroll
                    for (int x = 0; x < 32 / L::kPerRow; ++x) acc[x] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
                    for (int k = 0; k < cut.n; ++k) {               // (a running maximum: parts are few)
                        const size_t from = (size_t)cut.slot(k) * p.rb_rows + r;
                        const float2 x = __ldcg(p.part_ml + from);
                        float4 y[32 / L::kPerRow];
#pragma unroll
                        for (int i = 0; i < 32 / L::kPerRow; ++i) y[i] = __ldcg(reinterpret_cast<const float4*>(p.part_o + from * kHeadDim) + c0 + i * L::kPerRow);
                        const float now = fmaxf(top, x.x), keep = ex2(top - now), w = x.y * ex2(x.x - now);
                        top = now; sum = sum * keep + w;
#pragma unroll
                        for (int i = 0; i < 32 / L::kPerRow; ++i) {
                            acc[i].x = acc[i].x * keep + w * y[i].x; acc[i].y = acc[i].y * keep + w * y[i].y;
                            acc[i].z = acc[i].z * keep + w * y[i].z; acc[i].w = acc[i].w * keep + w * y[i].w;
                        }
                    }
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
                    for (int i = 0; i < 32 / L::kPerRow; ++i)
                        write_out(r, (c0 + i * L::kPerRow) * 4, make_float4(acc[i].x * inv, acc[i].y * inv, acc[i].z * inv, acc[i].w * inv));
                    if (p.lse && c0 == 0) write_lse(r, top, sum);
                }
            }
            __syncthreads();                                        // Q, the masks and the sums are free again
        }
    }
    // after a wait that ran out: copies in flight land before the CTA ends
    if (!alive) {
        flags[1 + warp] = 0;
        const Abort quiet{flags + 1 + warp, p.status};
        for (int i = 0; i < kStages; ++i)
            if (flying >> i & 1) mbar_wait(bars + i * 8, phases >> i & 1, quiet);
    }
}

}  // namespace

cudaError_t launch_kv8_attn(const Kv8AttnParams& p, int format, cudaStream_t st) {
    auto launch = [&](auto fmt, auto nb, auto warps) {
        constexpr int kFormat = decltype(fmt)::value, kNB = decltype(nb)::value, kWarps = decltype(warps)::value;
        using L = Lay<kNB, kWarps>;
        auto kernel = kv8_attn_kernel<kFormat, kNB, kWarps>;
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kBytes);
        if (e != cudaSuccess) return e;
        return launch_dependent(kernel, p.grid, L::kThreads, L::kBytes, st, p);
    };
    const std::integral_constant<int, 8> eight;
    auto by_rows = [&](auto fmt) {
        // Twelve warps where there are more than three items to a CTA: 64 single tokens of 1 k to 8 k keys, 8 KV heads 111 us, with eight 120; 64 of
        // 300 26.8 and 28.2; 32 of 500 21.9 and 20.3.  (More rows take more registers than twelve warps have.)
        if (p.rb_rows <= 8 && (long)p.n_branches * p.Hkv * p.n_rb > 3l * p.grid) return launch(fmt, std::integral_constant<int, 1>{}, std::integral_constant<int, 12>{});
        return p.rb_rows <= 8 ? launch(fmt, std::integral_constant<int, 1>{}, eight)
             : p.rb_rows <= 16 ? launch(fmt, std::integral_constant<int, 2>{}, eight) : launch(fmt, std::integral_constant<int, 3>{}, eight);
    };
    return format == TTS_KV8_E4M3 ? by_rows(std::integral_constant<int, TTS_KV8_E4M3>{}) : by_rows(std::integral_constant<int, TTS_KV8_INT8>{});
}

}  // namespace tts
