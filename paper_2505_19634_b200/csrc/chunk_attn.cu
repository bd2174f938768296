// Attention of ragged chunks of new tokens over the paged cache: prompts on their way in, a serving step's mix
// of prompt pieces and single tokens.
//
//   out[r] = sum_t p_t V_t / sum_t p_t,  p_t = exp(scale <q_r, K_t> - m_r),  lse[r] = m_r + log sum_t p_t,
//
// over the keys t below the row's limit (its own place in the sequence + 1), in one pass over the KV tiles with
// a running maximum and sum.  Scores, probabilities, sums and O are fp32; the probabilities are rounded to
// bf16 (2^-8 of each at most, averaging out over the keys) where they become an operand of the second contraction.
//
// Bound by the tensor cores for long chunks (4 x 128 operations per query row and key) and by HBM for single
// tokens.  One persistent CTA per SM takes pieces (chunk_attn.cuh) from a list.  A CTA has two *sides*, each
// with a 128-row score tile and a 128 x 128 fp32 accumulator in TMEM and a softmax warpgroup of its own, so
// that one side's exponentials run while the tensor pipe works for the other:
//   wide piece     side s holds row tile s; both go over the same KV tiles, which are loaded once for 256 rows
//   narrow piece   both sides hold the same rows; side s takes every second KV tile; side 0 joins the two
//
//   warps 0-3, 4-7  softmax of side 0, 1: one thread per row.  It reads its 128 scores from TMEM, writes the
//                   probabilities as bf16 pairs over the first half of its own score columns (the A operand of
//                   P V comes from TMEM), rescales O in TMEM only when the maximum has moved by more than 2^8
//                   (l carries the same reference, so the result is the same), and at the end divides and
//                   stores its row, or leaves (m, l, O) for the last piece of the entry to join.
//   warp 8          takes pieces, hands them to the other roles through a ring of two, loads Q
//   warp 9, 10      load the K and V tiles: one TMA box per 4 KiB page tile, rings of two and three slots (a V
//                   tile waits for its probabilities, a K tile does not)
//   warp 11         issues the MMAs.  Per side the order is S(0); then for each tile P V(j), S(j+1): the tensor
//                   pipe keeps issue order, so S(j+1) may overwrite the columns that held P(j), and when S(j+1)
//                   is complete P V(j) is as well -- the only wait on O that the softmax needs.
//
// Measured (B200 whose copy peak is 6538 GB/s and whose bf16 GEMMs reach 1663 TFLOP/s in a burst, 1394 sustained):
// 8192 tokens of 40 / 8 heads over 24576 keys 4.5 ms = 1070 TFLOP/s, 0.77 of the sustained rate; 64 single tokens
// over 1 k to 8 k keys 250 us = 5.65 TB/s, 0.86.  Both run into the card's power limit (1.5 GHz instead of 1.85): a
// tile of both sides takes 3300 clocks, of which the tensor pipe works 2050 and a softmax warp's chain (scores,
// maximum, exponentials at 8 clocks each, stores) fills about 2000, and changes that saved clocks alone
// (a second MMA warp, two threads per row, part of the exponentials as polynomials) did not save time.  Short pieces
// (24 prompts of up to 800 tokens: 53 us) wait for instructions as much as for anything else: two sides in different
// parts of the code miss the instruction cache at 22 % of its lookups, so code that is not the loop's is kept small.
//
// Page ids outside the pool and entries beyond the table row read as zeros (and are reported); tokens past the
// end of a branch never contribute: their scores are replaced before the maximum and their V rows are zeroed in
// shared memory, whatever the page holds there.  All waits between warps are bounded (umma_ptx.cuh), so a warp may leave
// at any of them: there is no barrier between the one where all begin and the one where all end.
#include <cuda.h>

#include <type_traits>

#include "chunk_attn.cuh"
#include "launch.cuh"
#include "packed.cuh"
#include "umma_ptx.cuh"

namespace tts {

namespace {

using namespace ptx;

constexpr int kTile = kChunkTile;
constexpr int kRows = 128;
constexpr int kSideThreads = 128;
constexpr int kThreadsChunk = 2 * kSideThreads + 128;
constexpr int kTakeWarp = 8, kKWarp = 9, kVWarp = 10, kMmaWarp = 11;
constexpr int kHalfBytes = kRows * 128;
constexpr int kOperandBytes = 2 * kHalfBytes;
constexpr int kRingK = 2, kRingV = 3, kRingPiece = 2;
constexpr uint32_t kTmemCols = 512;
// registers per thread: at launch, and after the softmax warpgroups have taken from the third one
constexpr int kLaunchRegs = 168, kSoftmaxRegs = 216, kHelperRegs = 72;
static_assert(2 * kSoftmaxRegs + kHelperRegs <= 3 * kLaunchRegs, "the split draws on what the block was launched with");

// The schedule of a call of up to kChunkSmall entries, made by every CTA for itself: smaller calls are one launch, and
// their time is latency (64 single tokens: 12 us less than with a launch of its own for the plan).
struct SmallTable {
    int pieces, part_rows;             // of one KV head
    int start[kChunkSmall + 1], keys[kChunkSmall];                                // rows and cached tokens of the branches
    unsigned short first[kChunkSmall + 1], at[kChunkSmall], cuts[kChunkSmall];    // first entry of a branch; an entry's first piece and their number
    int row[kChunkSmall];              // first partial-result row
};

constexpr int kOffQ = 0;                                       // two row tiles
constexpr int kOffK = kOffQ + 2 * kOperandBytes;
constexpr int kOffV = kOffK + kRingK * kOperandBytes;
constexpr int kOffBar = kOffV + kRingV * kOperandBytes;
enum Bar {
    K_FULL = 0, K_EMPTY = K_FULL + kRingK, V_FULL = K_EMPTY + kRingK, V_EMPTY = V_FULL + kRingV, V_TAIL = V_EMPTY + kRingV,
    Q_FULL, Q_EMPTY = Q_FULL + 2, S_FULL = Q_EMPTY + 2, P_HALF = S_FULL + 2, P_FULL = P_HALF + 2, O_FULL = P_FULL + 2, PIECE_FULL = O_FULL + 2,
    PIECE_EMPTY = PIECE_FULL + kRingPiece, JOIN_FULL = PIECE_EMPTY + kRingPiece, JOIN_EMPTY, PART_DONE, PART_LAST = PART_DONE + 2, DRAINED = PART_LAST + 2, kNumBars
};
constexpr int kOffMisc = kOffBar + ((kNumBars * 8 + 15) & ~15);   // [0] abort, [1] TMEM base, [2, 3] scratch of the K and V warps, [4, 5] last-piece flags, [6, 7] scratch of the taker and the MMA warp
constexpr int kOffPiece = kOffMisc + 32;                       // ring of pieces (+ their KV head)
constexpr int kPieceBytes = 64;
constexpr int kOffJoin = kOffPiece + kRingPiece * kPieceBytes; // side 1's (m, l) of a narrow piece
constexpr int kOffSmall = kOffJoin + kRows * 8;
constexpr int kSmemBytes = kOffSmall + ((sizeof(SmallTable) + 15) & ~15);     // the base is 1024-byte aligned: the kernel has no static shared memory
static_assert(kSmemBytes <= 227 * 1024, "shared memory");

// tcgen05.mma with descriptors as two words each; `accumulate` 0: the first step of a sum
__device__ __forceinline__ void umma_ss(uint32_t d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
        "mov.b64 a, {%1, %2};\n\tmov.b64 b, {%3, %4};\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %5, p;\n\t}"
        ::"r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a_tmem, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tmov.b64 b, {%2, %3};\n\tsetp.ne.b32 p, %5, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}"
        ::"r"(d), "r"(a_tmem), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate) : "memory");
}

// true in one lane of the warp; used right where it guards, which the compiler knows how to treat
__device__ __forceinline__ bool elect_one() {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok));
    return ok != 0;
}

__device__ __forceinline__ void warp_arrive(uint32_t bar, int lane) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
}

// A piece as every role sees it.
struct Work {
    ChunkPiece x;
    int kvh, part_rows;
    bool wide;
    int n0, n1;      // KV tiles of each side
    int loads;       // KV tiles to load
};

__device__ __forceinline__ void derive(Work& w, int T) {
    const ChunkPiece& x = w.x;
    w.wide = x.n_tok > T;
    const int tiles = x.tile_end - x.tile_begin;
    if (w.wide) {
        // side 0 stops at the tile of its last token's last key
        const int limit = min(x.keys, max(0, x.limit0 + T - 1));
        w.n0 = max(0, min(x.tile_end, ceil_div(limit, kTile)) - x.tile_begin);
        w.n1 = tiles;
    } else {
        w.n0 = (tiles + 1) >> 1;
        w.n1 = tiles >> 1;
    }
    w.loads = tiles;
}

// Next piece from the ring; false at the end of the list or when the CTA is aborting.  A role that keeps reading the
// ring's entry (kKeep) gives it back itself.
template <bool kKeep = false>
__device__ __forceinline__ bool next_piece(Work& w, int it, const unsigned char* smem, uint32_t bar0, int lane, int T, const Abort& ab) {
    const int slot = it % kRingPiece;
    const bool ok = __all_sync(0xffffffffu, mbar_wait(bar0 + 8u * (PIECE_FULL + slot), (it / kRingPiece) & 1, ab));
    if (!ok) return false;
    const int4* src = reinterpret_cast<const int4*>(smem + kOffPiece + slot * kPieceBytes);
    int4* dst = reinterpret_cast<int4*>(&w.x);
    dst[0] = src[0]; dst[1] = src[1]; dst[2] = src[2];
    w.kvh = src[3].x;
    if (!kKeep) warp_arrive(bar0 + 8u * (PIECE_EMPTY + slot), lane);
    if (w.kvh < 0) return false;
    derive(w, T);
    return true;
}

__device__ __forceinline__ int small_branch(const SmallTable& t, int n_branches, int e) {
    int lo = 0, hi = n_branches - 1;   // the last branch whose first entry is at or before e
    while (lo < hi) { const int mid = (lo + hi + 1) >> 1; if (t.first[mid] <= e) lo = mid; else hi = mid - 1; }
    return lo;
}

__device__ __forceinline__ ChunkEntry small_entry(const ChunkParams& p, const SmallTable& t, int e) {
    const int b = small_branch(t, p.n_branches, e);
    return chunk_entry(p.T, b, t.first[b + 1] - 1 - e, t.start[b], t.start[b + 1] - t.start[b], t.keys[b]);
}

__device__ __forceinline__ int warp_scan(int v, int lane, int* total) {        // exclusive
    int s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int n = __shfl_up_sync(0xffffffffu, s, o); if (lane >= o) s += n; }
    *total = __shfl_sync(0xffffffffu, s, 31);
    return s - v;
}

// One warp, two branches and two entries per lane.
__device__ void small_plan(const ChunkParams& p, SmallTable& t, int lane) {
    constexpr int kPer = kChunkSmall / 32;
    int count[kPer], mine = 0;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int b = kPer * lane + i;
        count[i] = 0;
        if (b < p.n_branches) {
            const int lo = p.row_start[b], hi = p.row_start[b + 1], len = p.branch_lens[b];
            bad |= !chunk_branch_ok(p, lo, hi, len);
            t.start[b] = lo; t.keys[b] = p.prefix_len + len;
            if (b == p.n_branches - 1) t.start[b + 1] = hi;
            count[i] = ceil_div(hi - lo, 2 * p.T);
        }
        mine += count[i];
    }
    bad = __any_sync(0xffffffffu, bad);
    if (bad && lane == 0) atomicMin(p.status, (int)TTS_ERR_DEVICE_BOUNDS);
    int n, first = warp_scan(bad ? 0 : mine, lane, &n);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int b = kPer * lane + i;
        if (b < p.n_branches) t.first[b] = (unsigned short)first;
        if (!bad) first += count[i];
        if (b == p.n_branches - 1) t.first[b + 1] = (unsigned short)n;
    }
    __syncwarp();
    ChunkEntry r[kPer];
    int cost[kPer], total = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int e = j * 32 + lane;
        cost[j] = -1;
        if (e < n) { r[j] = small_entry(p, t, e); cost[j] = chunk_cost(r[j], p.T); total += cost[j]; }
    }
    total = __reduce_add_sync(0xffffffffu, total);
    ChunkBound bound = chunk_bound(p, (float)total, n, (float)__reduce_max_sync(0xffffffffu, max(cost[0], cost[1])));
    int k[kPer], rows[kPer], at[kPer] = {}, row[kPer] = {}, pieces = 0, part_rows = 0;
    auto cut = [&](const int (&place)[kPer], const int (&after)[kPer]) {
        int sum = 0;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            k[j] = cost[j] >= 0 ? chunk_cuts(p, r[j], place[j], (float)after[j], (float)total, bound) : 0;
            rows[j] = k[j] > 1 ? k[j] * r[j].n_tok * p.G : 0;
            sum += rows[j];
        }
        part_rows = __reduce_add_sync(0xffffffffu, sum);
    };
    const int none[kPer] = {};
    if (bound.one_wave) cut(none, none);
    else part_rows = -1;
    if (part_rows >= 0 && (long)part_rows * p.Hkv <= p.part_rows) {
        // the bound alone says how entries are cut: their order does not matter
        int rows_so_far = 0;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            if (32 * j >= n) break;
            int sum_k, sum_rows = 0;
            at[j] = pieces + warp_scan(k[j], lane, &sum_k);
            if (part_rows > 0) row[j] = rows_so_far + warp_scan(rows[j], lane, &sum_rows);
            pieces += sum_k; rows_so_far += sum_rows;
        }
    } else {
        int after[kPer] = {};                          // cost of an entry and those handed out behind it
        unsigned long long ahead[kPer] = {};           // the entries handed out before it: costliest first, equal ones in their order
#pragma unroll
        for (int h = 0; h < kPer; ++h)
            for (int l = 0; l < min(32, n - 32 * h); ++l) {
                const int c = __shfl_sync(0xffffffffu, cost[h], l), i = 32 * h + l;
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    if (c > cost[j] || (c == cost[j] && i < j * 32 + lane)) ahead[j] |= 1ull << i;
                    else after[j] += c;
                }
            }
        int place[kPer];
#pragma unroll
        for (int j = 0; j < kPer; ++j) place[j] = __popcll(ahead[j]);
        for (;; bound = chunk_coarser(bound)) {
            cut(place, after);
            if (bound.narrow == kChunkNoBound || (long)part_rows * p.Hkv <= p.part_rows) break;    // else too much for the workspace
        }
#pragma unroll
        for (int h = 0; h < kPer; ++h)
            for (int l = 0; l < min(32, n - 32 * h); ++l) {
                const int k_i = __shfl_sync(0xffffffffu, k[h], l), rows_i = __shfl_sync(0xffffffffu, rows[h], l), i = 32 * h + l;
                pieces += k_i;
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    if (ahead[j] >> i & 1) { at[j] += k_i; row[j] += rows_i; }
            }
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int e = j * 32 + lane;
        if (e < n) { t.at[e] = (unsigned short)at[j]; t.cuts[e] = (unsigned short)k[j]; t.row[e] = row[j]; }
    }
    if (lane == 0) { t.pieces = pieces; t.part_rows = part_rows; }
    __syncwarp();
}
static_assert(kChunkSmall == 64, "two branches and two entries per lane, the order in 64 bits");

// One warp.
__device__ ChunkPiece small_piece(const ChunkParams& p, const SmallTable& t, int i, int lane) {
    const int n = t.first[p.n_branches];
    int e = 0;
    for (int j = 0; j < n; j += 32) {
        const bool here = j + lane < n && t.at[j + lane] <= i && i < t.at[j + lane] + t.cuts[j + lane];
        const unsigned found = __ballot_sync(0xffffffffu, here);
        if (found) e = j + __ffs(found) - 1;
    }
    return chunk_piece(small_entry(p, t, e), e, i - t.at[e], t.cuts[e], t.row[e]);
}

__device__ __forceinline__ void tma_load_rows(uint32_t dst, const CUtensorMap* map, int dim, int head, int row, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst), "l"(map), "r"(dim), "r"(head), "r"(row), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load_page_keep(uint32_t dst, const CUtensorMap* map, int page_head, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %2, %2, %2, %3}], [%4];"
        ::"r"(dst), "l"(map), "r"(0), "r"(page_head), "r"(bar) : "memory");
}

// 32 bytes per thread: whole sectors, although every thread writes a row of its own
__device__ __forceinline__ void st_global_32(void* to, const float* v) {
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(to), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]) : "memory");
}
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// 8 values of a result row from column `col` on
__device__ __forceinline__ void store_out8(const ChunkParams& p, size_t row_head, int col, const float* v) {
    if (p.out_dtype == TTS_OUT_FP32) {
        float4* to = reinterpret_cast<float4*>(static_cast<float*>(p.out) + row_head * kHeadDim + col);
        to[0] = make_float4(v[0], v[1], v[2], v[3]); to[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + row_head * kHeadDim + col) =
            make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
    }
}

__device__ __forceinline__ uint32_t bf16_pair2(uint64_t v) { const float2 f = unpack2(v); return bf16_pair(f.x, f.y); }

__device__ __forceinline__ uint64_t exp2_sfu2(uint64_t y) {
    const float2 f = unpack2(y);
    return pack2(ex2(f.x), ex2(f.y));
}
__global__ void __launch_bounds__(kThreadsChunk, 1)
chunk_attn_kernel(const __grid_constant__ ChunkParams p, const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_q1,
                  const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v) {
    extern __shared__ __align__(1024) unsigned char smem[];
    const uint32_t sbase = smem_u32(smem);
    const uint32_t bar0 = sbase + kOffBar;
    auto bar = [&](int i) { return bar0 + 8u * i; };
    volatile int* misc = reinterpret_cast<volatile int*>(smem + kOffMisc);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Abort ab{misc, p.status};

    // Rows of a single token's tile that hold no query: zeros cost the tensor cores less power than what they would find
    // there, and power is what bounds most calls of this kernel.
    for (int i = tid; i < kOperandBytes / 16; i += kThreadsChunk) *reinterpret_cast<uint4*>(smem + kOffQ + i * 16) = make_uint4(0, 0, 0, 0);
    fence_proxy_async();
    if (tid == 0) {
        misc[0] = 0;
        for (int i = 0; i < kRingK; ++i) { mbar_init(bar(K_FULL + i), 1); mbar_init(bar(K_EMPTY + i), 1); }
        for (int i = 0; i < kRingV; ++i) { mbar_init(bar(V_FULL + i), 1); mbar_init(bar(V_EMPTY + i), 1); }
        mbar_init(bar(V_TAIL), 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(Q_FULL + i), 1); mbar_init(bar(Q_EMPTY + i), 1); mbar_init(bar(S_FULL + i), 1);
            mbar_init(bar(P_HALF + i), kSideThreads / 32); mbar_init(bar(P_FULL + i), kSideThreads / 32); mbar_init(bar(O_FULL + i), 1);
            mbar_init(bar(PART_DONE + i), kSideThreads / 32); mbar_init(bar(PART_LAST + i), 1);
        }
        for (int i = 0; i < kRingPiece; ++i) { mbar_init(bar(PIECE_FULL + i), 1); mbar_init(bar(PIECE_EMPTY + i), 11); }   // all warps but the taker
        mbar_init(bar(JOIN_FULL), kSideThreads / 32); mbar_init(bar(JOIN_EMPTY), kSideThreads / 32); mbar_init(bar(DRAINED), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(sbase + kOffMisc + 4), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = (uint32_t)misc[1];
    grid_dependency_wait();
    grid_launch_dependents();

    if (warp >= 2 * kSideThreads / 32) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kHelperRegs));
        if (warp == kTakeWarp) {
            // =========================== takes pieces, loads Q ===========================
            SmallTable& small = *reinterpret_cast<SmallTable*>(smem + kOffSmall);
            if (p.small) small_plan(p, small, lane);
            // the first piece of a schedule made elsewhere, asked for together with their number
            int4 ahead[3];
            if (!p.small) {
                const int4* src = reinterpret_cast<const int4*>(p.pieces + min((int)blockIdx.x / p.Hkv, p.max_pieces - 1));
                ahead[0] = src[0]; ahead[1] = src[1]; ahead[2] = src[2];
            }
            const int total = (p.small ? small.pieces : p.head->pieces) * p.Hkv, part_rows = p.small ? small.part_rows : p.head->part_rows;
            int index = blockIdx.x, used[2] = {0, 0};
            bool alive = true;
            for (int it = 0; alive; ++it) {
                const int slot = it % kRingPiece;
                Work w;
                w.kvh = -1;
                if (index < total) {
                    const int i = index / p.Hkv;                            // all KV heads of a piece follow one another
                    w.kvh = index - i * p.Hkv;
                    if (!p.small) {
                        int4* dst = reinterpret_cast<int4*>(&w.x);
                        if (it > 0) {
                            const int4* src = reinterpret_cast<const int4*>(p.pieces + i);
                            ahead[0] = src[0]; ahead[1] = src[1]; ahead[2] = src[2];
                        }
                        dst[0] = ahead[0]; dst[1] = ahead[1]; dst[2] = ahead[2];
                    } else {
                        w.x = small_piece(p, small, i, lane);
                    }
                }
                if (lane == 0) {
                    alive = mbar_wait(bar(PIECE_EMPTY + slot), ((it / kRingPiece) & 1) ^ 1, ab);
                    if (alive) {
                        int4* ring = reinterpret_cast<int4*>(smem + kOffPiece + slot * kPieceBytes);
                        const int4* src = reinterpret_cast<const int4*>(&w.x);
                        ring[0] = src[0]; ring[1] = src[1]; ring[2] = src[2];
                        ring[3] = make_int4(w.kvh, part_rows, 0, 0);
                        mbar_arrive(bar(PIECE_FULL + slot));
                        if (w.kvh < 0) alive = false;
                    }
                    if (alive) {
                        index = p.grid + (int)atomicInc(&p.head->next, (unsigned)total - 1u);       // the next one; one for each piece, and back to 0
                        derive(w, p.T);
                        for (int s = 0; s < (w.wide ? 2 : 1) && alive; ++s) {
                            if ((s ? w.n1 : w.n0) == 0) continue;
                            alive = mbar_wait(bar(Q_EMPTY + s), (used[s] & 1) ^ 1, ab);
                            if (!alive) break;
                            ++used[s];
                            const bool single = w.x.n_tok == 1;
                            const CUtensorMap* tm = single ? &tm_q1 : &tm_q;
                            mbar_arrive_expect_tx(bar(Q_FULL + s), (uint32_t)(single ? p.G : p.T * p.G) * 256u);
                            const uint32_t dst = sbase + kOffQ + s * kOperandBytes;
                            tma_load_rows(dst, tm, 0, w.kvh * p.G, w.x.row0 + s * p.T, bar(Q_FULL + s));
                            tma_load_rows(dst + kHalfBytes, tm, 64, w.kvh * p.G, w.x.row0 + s * p.T, bar(Q_FULL + s));
                        }
                    }
                }
                alive = __shfl_sync(0xffffffffu, alive, 0);
                index = __shfl_sync(0xffffffffu, index, 0);
            }
            if (lane == 0) {
                // copies in flight land before the CTA may end: the consumers wait for them, unless they gave up
                if (*ab.flag)
                    for (int s = 0; s < 2; ++s)
                        if (used[s] > 0) {
                            const Abort quiet{misc + 6, p.status};
                            misc[6] = 0;
                            mbar_wait(bar(Q_FULL + s), (used[s] - 1) & 1, quiet);
                        }
            }
        } else if (warp == kKWarp || warp == kVWarp) {
            // =========================== K and V tiles ===========================
            const bool is_v = warp == kVWarp;
            const int ring_n = is_v ? kRingV : kRingK;
            const int full0 = is_v ? V_FULL : K_FULL, empty0 = is_v ? V_EMPTY : K_EMPTY;
            const int ring_off = is_v ? kOffV : kOffK;
            const CUtensorMap* tm = is_v ? &tm_v : &tm_k;
            const uint64_t once = l2_policy_evict_first();
            int slot = 0, round = 0, issued = 0, tails = 0;
            bool alive = true;
            Work w;
            for (int it = 0; alive && next_piece(w, it, smem, bar0, lane, p.T, ab); ++it) {
                const int32_t* bt = p.block_table + (size_t)w.x.branch * p.max_blocks;
                auto page_of = [&](int t) -> int {                          // this lane's page of KV tile t
                    const int blk = t * (kTile / kPage) + lane;
                    if (lane >= kTile / kPage || blk * kPage >= w.x.keys) return -2;
                    const int page = blk < p.max_blocks ? bt[blk] : -1;
                    if (page < 0 || page >= p.num_pages) { atomicMin(p.status, (int)TTS_ERR_DEVICE_BOUNDS); return -1; }
                    return page;
                };
                int page = w.loads > 0 ? page_of(w.x.tile_begin) : -2;
                for (int j = 0; j < w.loads; ++j) {
                    const int tok0 = (w.x.tile_begin + j) * kTile;
                    const int n_valid = min(kTile, w.x.keys - tok0), n_pages = ceil_div(n_valid, kPage);
                    const bool tail = is_v && n_valid < kTile;
                    const int full = tail ? (int)V_TAIL : full0 + slot;
                    const int next = j + 1 < w.loads ? page_of(w.x.tile_begin + j + 1) : -2;
                    if (lane == 0) {
                        alive = mbar_wait(bar(empty0 + slot), round ^ 1, ab);
                        if (alive) mbar_arrive_expect_tx(bar(full), (uint32_t)n_pages * 4096u);
                    }
                    alive = __shfl_sync(0xffffffffu, alive, 0);
                    if (!alive) break;
                    const uint32_t dst = sbase + ring_off + slot * kOperandBytes;
                    if (lane < n_pages) {
                        // a page outside the pool: a coordinate outside the map, which reads as zeros
                        const int page_head = page < 0 ? -1 : page * p.Hkv + w.kvh;
                        if (w.x.once) tma_load_page(dst + lane * 4096, tm, page_head, bar(full), once);
                        else tma_load_page_keep(dst + lane * 4096, tm, page_head, bar(full));
                    }
                    ++issued;
                    if (tail) {
                        // no row sees the tokens past the end, but 0 x NaN would be NaN: their V rows become zeros
                        alive = __all_sync(0xffffffffu, mbar_wait(bar(V_TAIL), tails & 1, ab));
                        ++tails;
                        if (!alive) break;
                        for (int i = lane; i < (kTile - n_valid) * 16; i += 32) {
                            const int row = n_valid + i / 16, c = i % 16;
                            *reinterpret_cast<uint4*>(smem + kOffV + slot * kOperandBytes + (row >> 4) * 4096 + ((row >> 3) & 1) * 2048 +
                                                      (c >> 3) * 1024 + (row & 7) * 128 + ((c & 7) << 4)) = make_uint4(0, 0, 0, 0);
                        }
                        fence_proxy_async();
                        warp_arrive(bar(full0 + slot), lane);
                    }
                    page = next;
                    if (++slot == ring_n) { slot = 0; round ^= 1; }
                }
            }
            if (*ab.flag && lane == 0) {
                const Abort quiet{misc + 2 + is_v, p.status};
                for (int back = 1; back <= ring_n && back <= issued; ++back) {
                    const int i = issued - back;
                    misc[2 + is_v] = 0;
                    mbar_wait(bar(full0 + i % ring_n), (i / ring_n) & 1, quiet);
                }
            }
        } else {
            // =========================== MMA issuer ===========================
            constexpr uint32_t idesc_qk = instr_desc(kRows, kTile, false, false), idesc_pv = instr_desc(kRows, kHeadDim, false, true);
            // The whole warp walks the loop and waits, so that addresses and descriptors stay in uniform registers; one
            // elected lane issues.  (With a single lane that does everything, 8192 new tokens over 24576 took 5.4 ms
            // instead of 4.85.)
            // low and high words of the operands' descriptors: addresses count in units of 16 bytes in the low word
            const uint64_t q_desc = smem_desc(sbase + kOffQ, 16, 1024), k_desc = smem_desc(sbase + kOffK, 16, 2048), v_desc = smem_desc(sbase + kOffV, 1024, 2048);
            const uint32_t q_lo = (uint32_t)q_desc, q_hi = (uint32_t)(q_desc >> 32), k_lo = (uint32_t)k_desc, k_hi = (uint32_t)(k_desc >> 32),
                           v_lo = (uint32_t)v_desc, v_hi = (uint32_t)(v_desc >> 32);
            const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);              // (a shuffle tells the compiler that the value is uniform)
            int k_slot = 0, k_round = 0, v_slot = 0, v_round = 0, q_phase[2] = {0, 0}, p_phase[2] = {0, 0};
            bool alive = true;
            Work w;
            for (int it = 0; alive && next_piece(w, it, smem, bar0, lane, p.T, ab); ++it) {
                const bool wide = __shfl_sync(0xffffffffu, (int)w.wide, 0) != 0;
                const int n0 = __shfl_sync(0xffffffffu, w.n0, 0), n1 = __shfl_sync(0xffffffffu, w.n1, 0), loads = __shfl_sync(0xffffffffu, w.loads, 0);
                const int n_max = max(n0, n1);
                const auto wait = [&](int i, int phase) { alive = alive && mbar_wait(bar(i), phase, ab); };
                // One turn of side s: O (+)= P V of its jj-th tile (jj >= 0), then S of the next one.  An issuing lane is held
                // back while the tensor pipe is busy, its queue being short; what is waited for between two groups of MMAs is
                // time the pipe stands still, so it is looked at while the first half of P V runs.  In a wide piece side 0
                // has waited for the tiles that both sides read.
                auto turn = [&](auto side, int jj) {
                    constexpr int s = decltype(side)::value;
                    const int n = s ? n1 : n0;
                    const bool own_q = wide || s == 0;                       // a narrow piece has one Q tile for both sides
                    const bool last_kv = s == 1 || !wide;                    // the last reader of a K or V tile gives it back
                    const bool more = jj + 1 < n, has_k = s == 1 && wide && jj + 1 < n0, has_v = s == 1 && wide && jj < n0;
                    if (jj >= 0) {
                        const uint32_t vd = v_lo + (uint32_t)(v_slot * (kOperandBytes / 16));     // one page (16 tokens) per step
                        if (!has_v) wait(V_FULL + v_slot, v_round);
                        wait(P_HALF + s, p_phase[s]);
                        alive = __all_sync(0xffffffffu, alive);
                        if (!alive) return;
                        tc_fence_after();
                        if (elect_one()) {
#pragma unroll
                            for (int ks = 0; ks < 4; ++ks)
                                umma_ts(tm + 256u + s * 128u, tm + s * 128u + ks * 8u, vd + ks * 4096 / 16, v_hi, idesc_pv, ks > 0 || jj > 0);
                        }
                        __syncwarp();
                        wait(P_FULL + s, p_phase[s]);
                        if (more && !has_k) wait(K_FULL + k_slot, k_round);
                        alive = __all_sync(0xffffffffu, alive);
                        if (!alive) return;
                        tc_fence_after();
                        if (elect_one()) {
#pragma unroll
                            for (int ks = 4; ks < 8; ++ks)
                                umma_ts(tm + 256u + s * 128u, tm + s * 128u + ks * 8u, vd + ks * 4096 / 16, v_hi, idesc_pv, 1u);
                            if (last_kv) umma_commit(bar(V_EMPTY + v_slot));
                            if (!more) umma_commit(bar(O_FULL + s));
                        }
                        __syncwarp();
                        p_phase[s] ^= 1;
                        if (last_kv && ++v_slot == kRingV) { v_slot = 0; v_round ^= 1; }
                    } else {
                        if (own_q && more) { wait(Q_FULL + s, q_phase[s]); q_phase[s] ^= 1; }
                        if (more && !has_k) wait(K_FULL + k_slot, k_round);
                        alive = __all_sync(0xffffffffu, alive);
                        if (!alive) return;
                        tc_fence_after();
                    }
                    if (!more) return;
                    // Q: two 64-dim blocks of 128 rows, K: dim halves 1 KiB apart inside a page
                    const uint32_t qd = q_lo + (own_q ? s * kOperandBytes / 16 : 0), kd = k_lo + (uint32_t)(k_slot * (kOperandBytes / 16));
                    const bool last_q = wide ? jj + 2 == n : 2 * (jj + 1) + s + 1 == loads;
                    if (elect_one()) {
#pragma unroll
                        for (int ks = 0; ks < 8; ++ks)
                            umma_ss(tm + s * 128u, qd + ((ks >> 2) * kHalfBytes + (ks & 3) * 32) / 16, q_hi, kd + ((ks >> 2) * 1024 + (ks & 3) * 32) / 16, k_hi, idesc_qk, ks > 0);
                        umma_commit(bar(S_FULL + s));
                        if (last_kv) umma_commit(bar(K_EMPTY + k_slot));
                        if (last_q) umma_commit(bar(Q_EMPTY + (own_q ? s : 0)));
                    }
                    __syncwarp();
                    if (last_kv && ++k_slot == kRingK) { k_slot = 0; k_round ^= 1; }
                };
                const std::integral_constant<int, 0> side0;
                const std::integral_constant<int, 1> side1;
#pragma unroll 1
                for (int jj = -1; jj < n_max && alive; ++jj) {
                    if (jj < n0) turn(side0, jj);
                    if (alive && jj < n1) turn(side1, jj);
                }
            }
            if (__any_sync(0xffffffffu, *ab.flag != 0)) {
                // products in flight end before their operands' shared memory and TMEM are someone else's
                if (elect_one()) {
                    misc[7] = 0;
                    umma_commit(bar(DRAINED));
                }
                __syncwarp();
                mbar_wait(bar(DRAINED), 0, Abort{misc + 7, p.status});
                __syncwarp();
            }
        }
    } else {
        // =========================== softmax ===========================
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        // What the loop over the tiles does not need stays in shared memory (the piece's record is given back at the
        // piece's end) or is worked out again: the loop's 128 scores leave few registers, and every spill is a stall.
        const int side = warp >> 2;
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t t_s = tmem + side * 128u + lane_base, t_o = t_s + 256u;
        uint32_t phases = 0;                                // bits: S_FULL, O_FULL of this side, O_FULL of the other, JOIN, a JOIN has been, PART
        enum { S_PHASE = 1, O_PHASE = 2, OTHER_PHASE = 4, JOIN_PHASE = 8, JOINED = 16, PART_PHASE = 32 };
        bool alive = true;
        for (int it = 0; alive; ++it) {
            int n, key0, step, limit, limit_min;
            bool idle, hollow;
            {
                Work w;
                if (!next_piece<true>(w, it, smem, bar0, lane, p.T, ab)) break;
                const int tok0 = w.wide ? side * p.T : 0;                           // first token of this side's rows
                const int tl = (int)(((warp & 3) * 32 + lane) * p.g_inv >> 16), last = min(p.T, w.x.n_tok - tok0) - 1;
                idle = (warp & 3) * 32 >= (last + 1) * p.G;                         // no row of this piece is this warp's
                hollow = tl > last;                                                 // nor is any this thread's: its weights are zeros
                n = side ? w.n1 : w.n0;
                step = w.wide ? kTile : 2 * kTile;
                key0 = w.x.tile_begin * kTile + (w.wide ? 0 : side * kTile);
                limit = min(w.x.keys, w.x.limit0 + tok0 + min(tl, last));           // keys this row sees (<= 0: none)
                limit_min = min(w.x.keys, w.x.limit0 + tok0);                       // the fewest that a row of the tile sees
            }
            if (side == 1 && n > 0 && (phases & JOINED)) {
                // side 0 has read what this side left of the last joined piece (O in TMEM, maxima and sums)
                alive = __all_sync(0xffffffffu, mbar_wait(bar(JOIN_EMPTY), phases & JOIN_PHASE ? 0 : 1, ab));
                if (!alive) break;
            }
            float m_ref = -INFINITY, l_sum = 0.f;
#pragma unroll 1
            for (int jj = 0; jj < n; ++jj, key0 += step) {
                alive = __all_sync(0xffffffffu, mbar_wait(bar(S_FULL + side), phases & S_PHASE ? 1 : 0, ab));
                if (!alive) break;
                phases ^= S_PHASE;
                tc_fence_after();
                if (idle) {                                 // (what its P rows hold reaches no row of the result)
                    warp_arrive(bar(P_HALF + side), lane);
                    warp_arrive(bar(P_FULL + side), lane);
                    continue;
                }
                const bool masked = key0 + kTile > limit_min;               // uniform over the side
                const int seen = limit - key0;
                if (masked) {
                    // In TMEM and in a loop: unrolled over the registers below, as a compare and a select per score, it is a
                    // third of this loop's code, and short pieces wait for code (24 prompts: 58.8 us instead of 56.2; long
                    // chunks, which hardly mask, are 1 % faster with it).
                    const int first = max(0, (int)__reduce_min_sync(0xffffffffu, seen)) >> 5;
#pragma unroll 1
                    for (int ch = first; ch < 4; ++ch) {
                        uint32_t v[32];
                        tmem_ld32(t_s + 32u * ch, v);
                        tmem_wait_ld();
                        const int left = seen - 32 * ch;
#pragma unroll
                        for (int c = 0; c < 32; ++c) if (c >= left) v[c] = 0xff800000u;       // -inf
                        tmem_st32(t_s + 32u * ch, v);
                    }
                    tmem_wait_st();
                }
                float sv[kTile];
                float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                tmem_ld32(t_s, reinterpret_cast<uint32_t*>(sv));
                tmem_ld32(t_s + 32u, reinterpret_cast<uint32_t*>(sv) + 32);
                tmem_wait_ld();
                tmem_ld32(t_s + 64u, reinterpret_cast<uint32_t*>(sv) + 64);  // on their way while the maximum of the first half is taken
                tmem_ld32(t_s + 96u, reinterpret_cast<uint32_t*>(sv) + 96);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    if (half) tmem_wait_ld();
#pragma unroll
                    for (int c = 32 * half; c < 32 * half + 32; ++c) mx4[c & 3] = max3(mx4[c & 3], sv[2 * c], sv[2 * c + 1]);
                }
                const float mx = max3(fmaxf(mx4[0], mx4[1]), mx4[2], mx4[3]) * p.scale_log2;
                const bool move = mx > m_ref + 8.f || (m_ref == -INFINITY && mx > -INFINITY);
                if (__any_sync(0xffffffffu, move)) {
                    const float factor = move && m_ref != -INFINITY ? ex2(m_ref - mx) : 1.f;
                    if (move) m_ref = mx;
                    l_sum *= factor;
                    if (jj > 0 && __any_sync(0xffffffffu, factor != 1.f))
                        // S of this tile is complete, so the previous P V is as well: O may be touched
#pragma unroll 1
                        for (int ch = 0; ch < 4; ++ch) {
                            uint32_t ov[32];
                            tmem_ld32(t_o + 32u * ch, ov);
                            tmem_wait_ld();
#pragma unroll
                            for (int c = 0; c < 32; ++c) ov[c] = __float_as_uint(__uint_as_float(ov[c]) * factor);
                            tmem_st32(t_o + 32u * ch, ov);
                        }
                }
                const float neg_m = hollow ? -INFINITY : m_ref == -INFINITY ? 0.f : -m_ref;
                const uint64_t scale2 = pack2(p.scale_log2, p.scale_log2), neg2 = pack2(neg_m, neg_m);
                uint64_t sum2[2] = {0, 0};
                uint32_t pw[kTile / 2];
                auto weights = [&](int c0, int c1) {                         // columns [2 c0, 2 c1)
#pragma unroll
                    for (int c = c0; c < c1; ++c) {
                        const uint64_t e = exp2_sfu2(fma2(pack2(sv[2 * c], sv[2 * c + 1]), scale2, neg2));
                        sum2[c & 1] = add2(sum2[c & 1], e);
                        pw[c] = bf16_pair2(e);
                    }
                };
                weights(0, 32);
                tmem_st32(t_s, pw);
                weights(32, 48);                                             // while the first half is stored
                tmem_wait_st();
                tc_fence_before();
                warp_arrive(bar(P_HALF + side), lane);
                weights(48, 64);
                tmem_st32(t_s + 32u, pw + 32);
                tmem_wait_st();
                tc_fence_before();
                warp_arrive(bar(P_FULL + side), lane);
                const float2 sum = unpack2(add2(sum2[0], sum2[1]));
                l_sum += sum.x + sum.y;
            }
            if (!alive) break;
            // ---- the piece's result ----
            Work w;
            {
                const int4* src = reinterpret_cast<const int4*>(smem + kOffPiece + (it % kRingPiece) * kPieceBytes);
                int4* dst = reinterpret_cast<int4*>(&w.x);
                dst[0] = src[0]; dst[1] = src[1]; dst[2] = src[2];
                w.kvh = src[3].x; w.part_rows = src[3].y;
                derive(w, p.T);
                warp_arrive(bar(PIECE_EMPTY + it % kRingPiece), lane);
            }
            const ChunkPiece& x = w.x;
            const int L = (warp & 3) * 32 + lane;           // row of the tile = TMEM lane
            const int tl = (int)(L * p.g_inv >> 16), gl = L - tl * p.G;      // token of the tile and head of the group
            const int tok0 = w.wide ? side * p.T : 0, n_tok = min(p.T, x.n_tok - tok0);
            const bool valid = tl < n_tok;                  // (L >= T G has tl >= T)
            const bool joined = !w.wide && w.n1 > 0;        // both sides hold a part of the same rows
            float2* join = reinterpret_cast<float2*>(smem + kOffJoin);
            if (!w.wide && side == 1) {
                if (joined) {
                    phases ^= O_PHASE;                      // side 0 waits for this side's O
                    join[L] = make_float2(m_ref, l_sum);
                    phases = (phases ^ JOIN_PHASE) | JOINED;
                    warp_arrive(bar(JOIN_FULL), lane);
                }
                continue;
            }
            if (n > 0) {
                alive = __all_sync(0xffffffffu, mbar_wait(bar(O_FULL + side), phases & O_PHASE ? 1 : 0, ab));
                phases ^= O_PHASE;
                if (!alive) break;
            }
            float f0 = 1.f, f1 = 0.f;                       // what each side's O counts
            if (joined) {
                alive = __all_sync(0xffffffffu, mbar_wait(bar(JOIN_FULL), phases & JOIN_PHASE ? 1 : 0, ab) &&
                                                mbar_wait(bar(O_FULL + 1), phases & OTHER_PHASE ? 1 : 0, ab));
                if (!alive) break;
                phases ^= JOIN_PHASE;
                const float2 o = join[L];
                const float m = fmaxf(m_ref, o.x);
                f0 = m_ref == -INFINITY ? 0.f : ex2(m_ref - m);
                f1 = o.x == -INFINITY ? 0.f : ex2(o.x - m);
                l_sum = l_sum * f0 + o.y * f1;
                m_ref = m;
            }
            if (w.n1 > 0) phases ^= OTHER_PHASE;
            tc_fence_after();
            const bool direct = x.parts == 1;
            const float inv = direct ? (l_sum > 0.f ? 1.f / l_sum : (l_sum == 0.f ? 0.f : l_sum)) : 1.f;
            f0 *= inv; f1 *= inv;
            const int rows = n_tok * p.G;                   // valid rows of this side
            // partial results of an entry: side 0's pieces, then side 1's
            const size_t part0 = (size_t)w.kvh * w.part_rows + x.part_row + (side == 1 ? (size_t)x.parts * p.T * p.G : 0);
            const size_t part_at = part0 + (size_t)x.part * rows + L;
            const size_t row_head = (size_t)(x.row0 + tok0 + tl) * p.Hq + w.kvh * p.G + gl;
            const uint32_t t_o1 = tmem + 384u + lane_base;  // side 1's O, which a joined piece adds
            // A thread writes its own row, whole sectors of 32 bytes at a time where the array's alignment allows it.  (Rows
            // gathered from neighbouring threads by shuffles make fuller lines, but take about 560 instructions per warp where this
            // takes about 240, and short pieces wait for instructions: 24 prompts 55.0 us, 54.4 this way.)
#pragma unroll 1
            for (int ch = 0; ch < 4 && !idle; ++ch) {
                float o[32], oj[32];                        // (both are read, if only to be dropped: a branch here cost more)
                tmem_ld32(t_o + 32u * ch, reinterpret_cast<uint32_t*>(o));
                tmem_ld32(t_o1 + 32u * ch, reinterpret_cast<uint32_t*>(oj));
                tmem_wait_ld();
#pragma unroll
                for (int c = 0; c < 32; ++c) {
                    o[c] = n > 0 && f0 != 0.f ? o[c] * f0 : 0.f;
                    o[c] = joined && f1 != 0.f ? fmaf(oj[c], f1, o[c]) : o[c];
                }
                if (valid) {
                    if (!direct) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) st_global_32(p.part_o + part_at * kHeadDim + 32 * ch + 8 * c, o + 8 * c);
                    } else if (p.out_dtype == TTS_OUT_BF16) {
                        float w2[16];
#pragma unroll
                        for (int c = 0; c < 16; ++c) w2[c] = __uint_as_float(bf16_pair(o[2 * c], o[2 * c + 1]));
                        __nv_bfloat16* to = static_cast<__nv_bfloat16*>(p.out) + row_head * kHeadDim + 32 * ch;
                        if (p.out_32) {
                            st_global_32(to, w2); st_global_32(to + 16, w2 + 8);
                        } else {
#pragma unroll
                            for (int c = 0; c < 4; ++c) reinterpret_cast<float4*>(to)[c] = make_float4(w2[4 * c], w2[4 * c + 1], w2[4 * c + 2], w2[4 * c + 3]);
                        }
                    } else {
#pragma unroll
                        for (int c = 0; c < 4; ++c) store_out8(p, row_head, 32 * ch + 8 * c, o + 8 * c);
                    }
                }
                __syncwarp();                           // TMEM is read by whole warps
            }
            tc_fence_before();
            if (joined) warp_arrive(bar(JOIN_EMPTY), lane);
            if (direct) {
                if (valid && p.lse) p.lse[row_head] = l_sum == 0.f ? -INFINITY : m_ref * 0.69314718055994530942f + logf(l_sum);
                continue;
            }
            if (valid) p.part_ml[part_at] = make_float2(m_ref, l_sum);
            // The last piece of the entry to arrive here joins all of them, in their order.  The side's warps meet through
            // waits that are bounded like all others, and not at a named barrier: when a wait has run out somewhere, one of
            // them may have left already while the others, whose waits came true at that moment, still arrive here.
            __threadfence();
            warp_arrive(bar(PART_DONE + side), lane);
            const bool leads = (warp & 3) == 0;             // counts the piece when all four have left their rows, and tells the others
            alive = __all_sync(0xffffffffu, mbar_wait(bar((leads ? PART_DONE : PART_LAST) + side), phases & PART_PHASE ? 1 : 0, ab));
            if (!alive) break;
            phases ^= PART_PHASE;
            if (leads) {
                if (lane == 0) {
                    unsigned* counter = p.arrived + ((size_t)x.entry * p.Hkv + w.kvh) * 2 + side;
                    misc[4 + side] = atomicInc(counter, (unsigned)x.parts - 1u) == (unsigned)x.parts - 1u;   // back to 0 for the next call
                    mbar_arrive(bar(PART_LAST + side));     // (the word is written again when all four are past the next PART_DONE)
                }
                __syncwarp();
            }
            if (misc[4 + side]) {
                __threadfence();
                // a unit is 8 columns of a row; four units and two parts at a time keep 16 loads in flight per thread
                const int units = rows * (kHeadDim / 8);
#pragma unroll 1
                for (int u0 = tid & (kSideThreads - 1); u0 < units; u0 += 4 * kSideThreads) {
                    float m[4], l[4], acc[4][8];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        m[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
                        for (int c = 0; c < 8; ++c) acc[i][c] = 0.f;
                    }
#pragma unroll 2
                    for (int k = 0; k < x.parts; ++k) {
                        float2 ml[4];
                        float4 va[4], vb[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int u = min(u0 + i * kSideThreads, units - 1);
                            const size_t at = part0 + (size_t)k * rows + u / (kHeadDim / 8);
                            const float4* src = reinterpret_cast<const float4*>(p.part_o + at * kHeadDim + (u % (kHeadDim / 8)) * 8);
                            ml[i] = __ldcg(p.part_ml + at); va[i] = __ldcg(src); vb[i] = __ldcg(src + 1);
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            // a piece without a key that this row sees counts 0 (and holds zeros); no branch, which would tear the loads apart
                            const float m_new = fmaxf(m[i], ml[i].x);
                            const float fa = m[i] == -INFINITY ? 0.f : ex2(m[i] - m_new), fb = ml[i].x == -INFINITY ? 0.f : ex2(ml[i].x - m_new);
                            const float v[8] = {va[i].x, va[i].y, va[i].z, va[i].w, vb[i].x, vb[i].y, vb[i].z, vb[i].w};
#pragma unroll
                            for (int c = 0; c < 8; ++c) acc[i][c] = acc[i][c] * fa + v[c] * fb;
                            l[i] = l[i] * fa + ml[i].y * fb;
                            m[i] = m_new;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int u = u0 + i * kSideThreads;
                        if (u >= units) continue;
                        const int row = u / (kHeadDim / 8), col = (u % (kHeadDim / 8)) * 8, t = (int)(row * p.g_inv >> 16);
                        const float scale = l[i] > 0.f ? 1.f / l[i] : (l[i] == 0.f ? 0.f : l[i]);
#pragma unroll
                        for (int c = 0; c < 8; ++c) acc[i][c] *= scale;
                        const size_t to = (size_t)(x.row0 + tok0 + t) * p.Hq + w.kvh * p.G + (row - t * p.G);
                        store_out8(p, to, col, acc[i]);
                        if (col == 0 && p.lse) p.lse[to] = l[i] == 0.f ? -INFINITY : m[i] * 0.69314718055994530942f + logf(l[i]);
                    }
                }
            }
        }
    }

    // ---- everyone arrives here, normally or after an abort ----
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
    static EncodeTiledFn fn = [] {
        void* sym = nullptr;
        cudaDriverEntryPointQueryResult res;
        return cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &res) == cudaSuccess && res == cudaDriverEntryPointSuccess
                   ? reinterpret_cast<EncodeTiledFn>(sym) : nullptr;
    }();
    return fn;
}

bool encode(CUtensorMap* map, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
    const cuuint32_t ones[5] = {1, 1, 1, 1, 1};
    const EncodeTiledFn fn = encode_fn();
    return fn && fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

cudaError_t launch_chunk_attn(const ChunkParams& p, const void* q, long q_stride, const void* k_pages, const void* v_pages, cudaStream_t st) {
    CUtensorMap tm_q, tm_q1, tm_k, tm_v;
    {
        // queries: (dim, head, row); a box is half the dims of G heads of T rows, or of one
        const cuuint64_t dims[3] = {(cuuint64_t)kHeadDim, (cuuint64_t)p.Hq, (cuuint64_t)p.total_rows};
        const cuuint64_t strides[2] = {kHeadDim * 2, (cuuint64_t)q_stride * 2};
        const cuuint32_t box[3] = {64, (cuuint32_t)p.G, (cuuint32_t)p.T}, box1[3] = {64, (cuuint32_t)p.G, 1};
        if (!encode(&tm_q, q, 3, dims, strides, box) || !encode(&tm_q1, q, 3, dims, strides, box1)) return cudaErrorInvalidValue;
    }
    {
        // pages: (64 dims, 8 tokens, dim half, token half, page-head); a box is one page of one head, laid out
        // [token half][dim half][8 tokens][128 bytes], so that a tile's pages form one MMA operand
        const cuuint64_t dims[5] = {64, 8, 2, 2, (cuuint64_t)p.num_pages * p.Hkv};
        const cuuint64_t strides[4] = {256, 128, 2048, 4096};
        const cuuint32_t box[5] = {64, 8, 2, 2, 1};
        if (!encode(&tm_k, k_pages, 5, dims, strides, box) || !encode(&tm_v, v_pages, 5, dims, strides, box)) return cudaErrorInvalidValue;
    }
    cudaError_t e = cudaFuncSetAttribute(chunk_attn_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
    if (e != cudaSuccess) return e;
    static const int regs = [] { cudaFuncAttributes a; return cudaFuncGetAttributes(&a, chunk_attn_kernel) == cudaSuccess ? a.numRegs : 0; }();
    if (regs < kLaunchRegs) return cudaErrorInvalidConfiguration;       // the register split needs what it was computed from
    return launch_dependent(chunk_attn_kernel, p.grid, kThreadsChunk, kSmemBytes, st, p, tm_q, tm_q1, tm_k, tm_v);
}

}  // namespace tts
