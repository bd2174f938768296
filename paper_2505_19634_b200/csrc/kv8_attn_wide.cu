// Attention of many rows per KV head (draft trees, long drafted chains with large head groups) over the 8-bit cache.
//
// The formula and the roundings of kv8_attn.cu, for which a row block is too much to hold in a warp's registers: there the codes of
// a page become operands once for 24 rows, here once for 128, and the products are the tensor cores' own.
//
// Two CTAs share an SM, so that one's exponentials run while the tensor cores work for the other.  64 tokens and 128 rows cost 512
// clocks of the tensor cores, 512 of the exponentials' unit and, in shared memory, about 1200: Q, K and V as operands (512), codes read,
// written in fp16 and fetched (512), scales, barriers.  Measured: about 1550 clocks, and a third of a call around them: 18000 clocks until the
// first product (cold instructions and TLBs), up to 35000 behind a piece's last (its rows, the fence, the join).  8 trees of 60 nodes,
// 300 rows to a KV head, over 7.9 k keys: 196 us = 389 TFLOP/s; the kernel for few rows took 410.  All of these took 190 to 200 us as well: Q in
// TMEM and one S; K's and V's conversion by warps of their own; a warp for each product; waits that sleep.  V's operand twice 229, codes
// loaded a tile ahead into registers 319.  In a CTA,
//   warps 0-7   softmax, two threads to a row, in warps w and w + 4: they lay out its query; per tile of 64 tokens each reads 32 of its
//               scores from TMEM and leaves p sv there, as the second product's A operand; O is touched only when the maximum moves
//               by more than 2^8 or the row's unit of p sv grows: the largest V scale that it sees.  At a piece's end they write the row.
//   warps 8-11  turn codes into fp16 operands (exact): [64 tokens][128 dims], two warps K with dims along the contraction, two V with
//               tokens.  One of K's leaves the tile's scales and the largest so far.
//   warp 12     issues the products: S = Q K^T (128 x 64 x 128) of the next tile, then O += P V (128 x 128 x 64) of this one.  The tensor
//               pipe keeps issue order, so S of a tile may overwrite the columns that held P two tiles before.
//   warp 13     fetches the records, by bulk copies: K with all scales into a ring of three tiles, V into one of two.
// TMEM columns of a CTA: two S of 64 (P in the first half of its S), O 128.
#include <cuda_fp16.h>

#include "kv8_run.cuh"
#include "launch.cuh"
#include "packed.cuh"
#include "umma_ptx.cuh"

namespace tts {

namespace {

using namespace ptx;

constexpr int kTile = 64, kTilePages = kTile / kPage;
constexpr int kRows = kKv8WideRows;
constexpr int kSoftmaxWarps = 8, kConvertWarps = 4, kMmaWarp = kSoftmaxWarps + kConvertWarps, kLoadWarp = kMmaWarp + 1;
constexpr int kThreads = (kLoadWarp + 1) * 32;
constexpr float kFar = -1e30f;                                      // "no key yet": finite, so that differences are never NaN
constexpr float kSlack = 8.f;                                       // log2 of how far a score may exceed the running maximum
constexpr int kRoom = 6;                                            // p sv is held times 2^kRoom
constexpr int kLeastUnit = 7;                                       // exponent field of the smallest unit of p sv: its reciprocal times 2^kRoom is a normal number
constexpr uint32_t kTmemCols = 256, kColS = 0, kColO = 128;
// An item's start and end take about as long as so many tiles (kv8_run.cuh).  64 (branch, KV head)s of 120 tiles: 93 us with 12, 97 with 4,
// 122 with 24 (125 rows); 197, 197 and 209 (300 rows, three blocks).
constexpr int kItemUnits = 12;
// Of a CTA's share of an item, where items are cut evenly.  100 rows of 40 / 8 heads over 8 k keys: 48.6 us with 16, 53.4 with 12, 51.7 with 24.
constexpr int kLeastTiles = 12, kMostTiles = 16;
using Walk = Kv8Walk<kTile, kItemUnits>;

constexpr int kOperand = kTile * kHeadDim * 2;                      // fp16 K, and V, of a tile: two blocks of 64 dims, rows of 128 bytes
constexpr int kBlock = kOperand / 2;
// a tile's records in shared memory: K codes and all scales, page after page; V codes
constexpr int kCodesTile = kTilePages * kKv8Codes, kScalesPage = kKv8Record - 2 * kKv8Codes;
constexpr int kRingK = 3, kRingV = 2;
constexpr int kRawK = kCodesTile + kTilePages * kScalesPage, kRawV = kCodesTile;
// what the softmax needs of a tile besides its scores
struct Scales {
    float k[kTile], v[kTile];                                       // (K's times the softmax's scale, in log2 units)
    int unit_exp;                                                   // exponent field of the largest power of two in V's scales so far
    int pad[3];
};
constexpr int kOffQ = 0;                                            // fp16 rows, laid out as K's
constexpr int kQBlock = kRows * 128;
constexpr int kOffK = kOffQ + 2 * kQBlock;
constexpr int kOffV = kOffK + kOperand;
constexpr int kOffRawK = kOffV + kOperand;
constexpr int kOffRawV = kOffRawK + kRingK * kRawK;
constexpr int kOffScales = kOffRawV + kRingV * kRawV;
constexpr int kScales = 4;                                          // tiles
constexpr int kOffCum = kOffQ;                                      // [branches + 1] units before each branch, until every role has found its first piece
constexpr int kOffSums = kOffScales + kScales * (int)sizeof(Scales);  // scratch of the scan
enum Bar { RAWK_FULL = 0, RAWK_EMPTY = RAWK_FULL + kRingK, RAWV_FULL = RAWK_EMPTY + kRingK, RAWV_EMPTY = RAWV_FULL + kRingV, S_FULL = RAWV_EMPTY + kRingV, P_FULL = S_FULL + 2, SCALES = P_FULL + 2, K_FULL = SCALES + kScales, K_EMPTY, V_FULL, V_EMPTY, Q_FULL, O_FULL, PART_DONE, PART_LAST, DRAINED, kNumBars };
static_assert((kMaxBranches + 1) * 8 <= 2 * kQBlock, "the branches' units lie where the queries will");
constexpr int kOffPair = kOffSums + (kThreads / 32) * 8;            // [2][2][rows] what the two threads of a row tell one another: maxima; units, then sums
constexpr int kOffBar = kOffPair + 4 * kRows * 4;
constexpr int kOffMisc = kOffBar + kNumBars * 8;                    // [0] abort, [1] TMEM base, [2] the last part, [3, 4] scratch of the copying and the MMA warp
constexpr int kSmemBytes = kOffMisc + 32;
static_assert(kOffBar % 8 == 0 && kOffRawK % 128 == 0 && kRawK % 128 == 0 && sizeof(Scales) % 16 == 0 && 2 * (kSmemBytes + 1024) <= 228 * 1024, "two CTAs to an SM");

// exponent field of a scale of V; a NaN or an infinity has no unit
__device__ __forceinline__ int unit_of(float v) { const int e = __float_as_int(v) >> 23 & 255; return e == 255 ? 0 : e; }
// 2^kRoom over the unit of this exponent field
__device__ __forceinline__ float up_of(int unit_exp) { return power_of_two(kRoom + 127 - unit_exp); }
__device__ __forceinline__ bool elect_one() {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok));
    return ok != 0;
}
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ void warp_arrive(uint32_t bar, int lane) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
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
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
constexpr uint32_t f16_desc(int m, int n, bool b_mn_major) { return instr_desc(m, n, false, b_mn_major) & ~(1u << 7 | 1u << 10); }   // fp16 operands

template <int kFormat>
__global__ void __launch_bounds__(kThreads, 2)
kv8_attn_wide_kernel(const __grid_constant__ Kv8AttnParams p) {
    extern __shared__ __align__(1024) unsigned char smem[];
    const uint32_t sbase = smem_u32(smem);
    auto bar = [&](int i) { return sbase + kOffBar + 8u * i; };
    long long* cum = reinterpret_cast<long long*>(smem + kOffCum);
    volatile int* misc = reinterpret_cast<volatile int*>(smem + kOffMisc);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Abort ab{misc, p.status};

    if (threadIdx.x == 0) {
        misc[0] = 0;
        for (int i = 0; i < kRingK; ++i) { mbar_init(bar(RAWK_FULL + i), 1); mbar_init(bar(RAWK_EMPTY + i), kConvertWarps); }
        for (int i = 0; i < kRingV; ++i) { mbar_init(bar(RAWV_FULL + i), 1); mbar_init(bar(RAWV_EMPTY + i), kConvertWarps); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(S_FULL + i), 1); mbar_init(bar(P_FULL + i), kSoftmaxWarps);
        }
        for (int i = 0; i < kScales; ++i) mbar_init(bar(SCALES + i), 1);
        mbar_init(bar(K_FULL), kConvertWarps); mbar_init(bar(V_FULL), kConvertWarps); mbar_init(bar(K_EMPTY), 1); mbar_init(bar(V_EMPTY), 1);
        mbar_init(bar(Q_FULL), kSoftmaxWarps); mbar_init(bar(O_FULL), 1);
        mbar_init(bar(PART_DONE), kSoftmaxWarps); mbar_init(bar(PART_LAST), 1); mbar_init(bar(DRAINED), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(sbase + kOffMisc + 4), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_proxy_async();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = (uint32_t)misc[1];
    grid_dependency_wait();
    grid_launch_dependents();
    kv8_scan_units<kThreads, kTile, kItemUnits>(p, cum, reinterpret_cast<long long*>(smem + kOffSums));
    const Kv8Run run = kv8_run<kThreads, kItemUnits>(p, cum, reinterpret_cast<int*>(smem + kOffSums), kLeastTiles, kMostTiles);
    Walk item;
    const bool work = run.n > 0 && item.init(p, cum, run.begin, run.n);   // every role walks over the pieces for itself
    bool alive = work;
    __syncthreads();

    if (warp >= kSoftmaxWarps && warp < kMmaWarp) {
        // =========================== records to operands ===========================
        // K of a tile before V of the one before it, which waits longer.
        const int w = warp - kSoftmaxWarps, ct = w * 32 + lane;
        // Eight lanes have a token's 128 codes; codes 16 c .. of a token become 16-byte chunks 2 c and 2 c + 1 of its row.
        // Lanes with c >= 4 write the second one first: eight different bank groups.
        auto convert = [&](const unsigned char* raw, unsigned char* operand, int left) {
            uint4 x[kTile / (kConvertWarps * 4)];
#pragma unroll
            for (int i = 0; i < kTile / (kConvertWarps * 4); ++i) x[i] = *reinterpret_cast<const uint4*>(raw + (i * kConvertWarps * 4 + (ct >> 3)) * kHeadDim + (ct & 7) * 16);
            if (left < kTile)                                           // what is not there: 0 x NaN would be NaN
#pragma unroll
                for (int i = 0; i < kTile / (kConvertWarps * 4); ++i)
                    if (i * kConvertWarps * 4 + (ct >> 3) >= left) x[i] = make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < kTile / (kConvertWarps * 4); ++i) {
                const int t = i * kConvertWarps * 4 + (ct >> 3), c = (ct & 7) ^ kv8_chunk_place(t & 15);
                const bool odd = c >= 4;
                unsigned char* to = operand + (c >> 2) * kBlock + t * 128;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const bool second = odd != (half == 1);
                    const uint32_t a = kv8_biased<kFormat>(second ? x[i].z : x[i].x), b = kv8_biased<kFormat>(second ? x[i].w : x[i].y);
                    *reinterpret_cast<uint4*>(to + ((((2 * c + (second ? 1 : 0)) & 7) ^ (t & 7)) << 4)) =
                        make_uint4(kv8_decode2<kFormat>(a, 0), kv8_decode2<kFormat>(a, 1), kv8_decode2<kFormat>(b, 0), kv8_decode2<kFormat>(b, 1));
                }
            }
            fence_proxy_async();                                        // the operand, for the tensor cores
            __syncwarp();
        };
        auto wait = [&](int i, uint32_t parity) { alive = __all_sync(0xffffffffu, alive && mbar_wait(bar(i), parity, ab)); };
        int tile = 0, before = 0, unit_exp = kLeastUnit;                // tile of the piece; tokens of the tile before
        int k_slot = 0, k_round = 0, v_slot = 0, v_round = 0;
        bool more = alive;
        for (int n = 0; alive && (more || n > 0); ++n) {                // tiles of the run
            int left = 0;
            const bool here = more;
            if (more) {
                left = min(kTile, item.tokens - (item.first + tile) * kTile);       // tokens here (may be 0)
                const unsigned char* raw = smem + kOffRawK + k_slot * kRawK;
                wait(RAWK_FULL + k_slot, k_round);
                wait(K_EMPTY, (n & 1) ^ 1);
                if (!alive) break;
                if (w == 1) {
                    // (S of the tile before is complete: P V of the third before was issued ahead of it, after its softmax)
                    Scales& to = *reinterpret_cast<Scales*>(smem + kOffScales + n % kScales * sizeof(Scales));
                    int top = 0;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int t = i * 32 + lane;
                        const float* s = reinterpret_cast<const float*>(raw + kCodesTile + (t >> 4) * kScalesPage) + (t & 15);
                        const float v = t < left ? s[kPage] : 0.f;
                        to.k[t] = t < left ? s[0] * p.scale_log2 : 0.f; to.v[t] = v;
                        top = max(top, unit_of(v));
                    }
                    unit_exp = max(tile == 0 ? kLeastUnit : unit_exp, __reduce_max_sync(0xffffffffu, top));
                    if (lane == 0) to.unit_exp = unit_exp;
                    warp_arrive(bar(SCALES + n % kScales), lane);
                }
                convert(raw, smem + kOffK, left);
                if (lane == 0) { mbar_arrive(bar(K_FULL)); mbar_arrive(bar(RAWK_EMPTY + k_slot)); }
                if (++k_slot == kRingK) { k_slot = 0; k_round ^= 1; }
                if (++tile >= item.n) { tile = 0; more = item.next(p); }
            }
            if (n > 0) {
                wait(RAWV_FULL + v_slot, v_round);
                wait(V_EMPTY, n & 1);
                if (!alive) break;
                convert(smem + kOffRawV + v_slot * kRawV, smem + kOffV, before);
                if (lane == 0) { mbar_arrive(bar(V_FULL)); mbar_arrive(bar(RAWV_EMPTY + v_slot)); }
                if (++v_slot == kRingV) { v_slot = 0; v_round ^= 1; }
            }
            before = left;
            if (!here) break;
        }
    } else if (warp == kLoadWarp) {
        // =========================== records ===========================
        // Half the lanes follow K's tiles, half V's, each as far ahead as their ring allows.
        const int kv = lane >> 4, sub = lane & 15, ring = kv ? kRingV : kRingK;
        const int full0 = kv ? RAWV_FULL : RAWK_FULL, empty0 = kv ? RAWV_EMPTY : RAWK_EMPTY;
        auto of_mine = [&](bool x) { return __ballot_sync(0xffffffffu, x) >> (16 * kv) & 0xffffu; };
        int tile = 0, slot = 0, round = 0, n = 0, page = -1;            // tile of the piece; the ring; tiles fetched
        bool more = alive;
        auto look_up = [&]() {                                          // the pages of the next tile
            const int first = (item.first + tile) * kTile;
            page = -1;
            if (sub < kTilePages && first + sub * kPage < item.tokens) page = p.block_table[(size_t)item.b * p.max_blocks + first / kPage + sub];
        };
        if (more) look_up();
        long long since = 0;                                            // of the last copy; this wait has its limit too
        for (int spin = 0; __any_sync(0xffffffffu, more); ++spin) {
            const bool go = of_mine(more && mbar_test(bar(empty0 + slot), round ^ 1)) == 0xffffu;
            if (!__any_sync(0xffffffffu, go)) {
                __nanosleep(100);                                       // (asking all the time was 40 % of all instructions)
                if ((spin & 63) == 63) {
                    const long long now = global_ns();
                    if (since == 0) since = now;
                    if (now - since > kWaitLimitNs) { *ab.flag = 1; atomicMin(p.status, (int)TTS_ERR_DEVICE_TIMEOUT); }
                    if (__any_sync(0xffffffffu, *ab.flag != 0)) break;
                }
                continue;
            }
            spin = 0; since = 0;
            const bool wanted = go && sub < kTilePages && (item.first + tile) * kTile + sub * kPage < item.tokens, there = wanted && page >= 0 && page < p.num_pages;
            const unsigned good = of_mine(there), bad = of_mine(wanted && !there);
            unsigned char* dst = smem + (kv ? kOffRawV + slot * kRawV : kOffRawK + slot * kRawK);
            if (__any_sync(0xffffffffu, bad != 0)) {                    // a page outside the pool counts as zeros
                if (bad && sub == 0) atomicMin(p.status, (int)TTS_ERR_DEVICE_BOUNDS);
                for (int pg = 0; pg < kTilePages; ++pg)
                    if (bad >> pg & 1) {
                        for (int i = sub; i < kKv8Codes / 16; i += 16) *reinterpret_cast<uint4*>(dst + pg * kKv8Codes + i * 16) = make_uint4(0, 0, 0, 0);
                        if (!kv && sub < kScalesPage / 16) *reinterpret_cast<uint4*>(dst + kCodesTile + pg * kScalesPage + sub * 16) = make_uint4(0, 0, 0, 0);
                    }
                fence_proxy_async();                                    // (before a later copy into the slot)
                __syncwarp();
            }
            const uint32_t full = bar(full0 + slot);
            if (go && sub == 0) { if (good) mbar_arrive_expect_tx(full, __popc(good) * (kv ? kKv8Codes : kKv8Codes + kScalesPage)); else mbar_arrive(full); }
            __syncwarp();
            if (there) {
                const unsigned char* src = p.pool + ((size_t)page * p.Hkv + item.item / p.n_rb) * kKv8Record;
                bulk_load(smem_u32(dst) + sub * kKv8Codes, src + kv * kKv8Codes, kKv8Codes, full);
                if (!kv) bulk_load(smem_u32(dst) + kCodesTile + sub * kScalesPage, src + 2 * kKv8Codes, kScalesPage, full);
            }
            if (go) {
                ++n;
                if (++slot == ring) { slot = 0; round ^= 1; }
                if (++tile >= item.n) { tile = 0; more = item.next(p); }
                if (more) look_up();
            }
        }
        // copies in flight land before the CTA ends, also where the warps that they are for have given up, or are about to
        const Abort quiet{misc + 3, p.status};
        for (int i = max(0, n - ring); i < n; ++i) { misc[3] = 0; mbar_wait(bar(full0 + i % ring), i / ring & 1, quiet); }
    } else if (warp == kMmaWarp) {
        // =========================== products ===========================
        constexpr uint32_t idesc_qk = f16_desc(kRows, kTile, false), idesc_pv = f16_desc(kRows, kHeadDim, true);
        const uint64_t q_desc = smem_desc(sbase + kOffQ, 16, 1024), k_desc = smem_desc(sbase + kOffK, 16, 1024), v_desc = smem_desc(sbase + kOffV, kBlock, 1024);
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);          // (a shuffle tells the compiler that the value is uniform)
        int n = 0, pieces = 0;
        auto wait = [&](int i, uint32_t parity) { alive = __all_sync(0xffffffffu, alive && mbar_wait(bar(i), parity, ab)); };
        auto scores = [&](int tile) {
            wait(K_FULL, tile & 1);
            if (!alive) return;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)
                    umma_bf16(tm + kColS + (tile & 1) * kTile, q_desc + ((ks >> 2) * kQBlock + (ks & 3) * 32) / 16, k_desc + ((ks >> 2) * kBlock + (ks & 3) * 32) / 16, idesc_qk, ks > 0);
                umma_commit(bar(S_FULL + (tile & 1)));
                umma_commit(bar(K_EMPTY));
            }
            __syncwarp();
        };
        for (bool more_items = alive; more_items && alive; more_items = item.next(p), ++pieces) {
            const int tiles = __shfl_sync(0xffffffffu, item.n, 0);
            wait(Q_FULL, pieces & 1);
            scores(n);
            for (int j = 0; alive && j < tiles; ++j, ++n) {
                if (j + 1 < tiles) scores(n + 1);
                wait(V_FULL, n & 1);
                wait(P_FULL + (n & 1), n >> 1 & 1);
                if (!alive) break;
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int ks = 0; ks < kTilePages; ++ks)
                        umma_bf16_tmem_a(tm + kColO, tm + kColS + (n & 1) * kTile + ks * 8u, v_desc + ks * 2048 / 16, idesc_pv, ks > 0 || j > 0);
                    umma_commit(bar(V_EMPTY));
                    if (j + 1 == tiles) umma_commit(bar(O_FULL));
                }
                __syncwarp();
            }
        }
        // products in flight end before their operands' shared memory and TMEM are someone else's, whoever has given up
        if (elect_one()) {
            misc[4] = 0;
            umma_commit(bar(DRAINED));
        }
        __syncwarp();
        mbar_wait(bar(DRAINED), 0, Abort{misc + 4, p.status});
        __syncwarp();
    } else if (warp < kSoftmaxWarps) {
        // =========================== softmax ===========================
        // The two warps of a row meet at barriers, so that neither leaves where a wait has run out: they go on, waiting no more, with
        // whatever is there.
        const int half = warp >> 2, meet = 1 + (warp & 3), r = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t t_o = tmem + lanes + kColO + 64u * half;
        float* mine = reinterpret_cast<float*>(smem + kOffPair) + half * kRows + r;
        const float* other = reinterpret_cast<float*>(smem + kOffPair) + (half ^ 1) * kRows + r;
        int n = 0, pieces = 0, parts_left = 0;
        auto wait = [&](int i, uint32_t parity) { alive = __all_sync(0xffffffffu, alive && mbar_wait(bar(i), parity, ab)); };
        for (bool more_items = work; more_items; more_items = item.next(p), ++pieces) {
            const int h = item.item / p.n_rb, row0 = (item.item - h * p.n_rb) * p.rb_rows, rows = min(p.rb_rows, p.nr - row0);
            const int stacked = row0 + min(r, rows - 1), i_row = stacked / p.G, head = h * p.G + stacked - i_row * p.G;
            const bool idle = (warp & 3) * 32 >= rows;                  // no row of the block is these warps'
            const int tail = item.tokens - p.R;                         // the first of the branch's last R tokens (may be negative)
            float factor = 0.f;
            unsigned long long mask = 0;                                // which of the branch's last R tokens the row sees
            if (!idle) {
                // ---- the query, scaled to fp16 by the power of two that puts its largest at 2^14; 64 dims to a thread
                const uint4* src = reinterpret_cast<const uint4*>(p.q + ((size_t)item.b * p.R + i_row) * p.q_stride + (size_t)head * kHeadDim + 64 * half);
                uint32_t x[32];
#pragma unroll
                for (int i = 0; i < 8; ++i) { const uint4 y = src[i]; x[4 * i] = y.x; x[4 * i + 1] = y.y; x[4 * i + 2] = y.z; x[4 * i + 3] = y.w; }
                uint32_t top = 0;                                       // the largest finite magnitude, as bits
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    const uint32_t lo = x[i] << 16 & 0x7fffffffu, hi = x[i] & 0x7fff0000u;
                    top = max(top, max(lo < 0x7f800000u ? lo : 0u, hi < 0x7f800000u ? hi : 0u));
                }
                *mine = __uint_as_float(top);
                bar_sync_id<64>(meet);
                const int e = max(-100, min(126, (int)(max(top, __float_as_uint(*other)) >> 23) - 127)) - 14;
                const float down = power_of_two(-e);
#pragma unroll
                for (int i = 0; i < 32; ++i) x[i] = pack_half2(__uint_as_float(x[i] << 16) * down, __uint_as_float(x[i] & 0xffff0000u) * down);
                unsigned char* to = smem + kOffQ + half * kQBlock + r * 128;
#pragma unroll
                for (int c = 0; c < 8; ++c) *reinterpret_cast<uint4*>(to + ((c ^ (r & 7)) << 4)) = make_uint4(x[4 * c], x[4 * c + 1], x[4 * c + 2], x[4 * c + 3]);
                fence_proxy_async();
                // (a power of two alone: the product with it is not rounded, so the maximum is what the fused multiply-add below takes it for, even
                // where it is so large that its own rounding would be more than an exponent that fp16 holds)
                factor = power_of_two(e);
                if (p.tree_parents == nullptr) mask = i_row >= 63 ? ~0ull : (2ull << i_row) - 1ull;
                else
                    for (int a = i_row, guard = 0; a >= 0 && guard < kMaxTreeRows; ++guard) {
                        mask |= 1ull << a;
                        const int parent = p.tree_parents[(size_t)item.b * p.R + a];
                        a = parent < a ? parent : -1;                   // malformed parents end the walk
                    }
            }
            warp_arrive(bar(Q_FULL), lane);
            float neg_m = -kFar, l = 0.f;
            int unit_exp = kLeastUnit;                                  // of the row: the largest V scale that it has seen
            const uint64_t factor2 = pack2(factor, factor);
#pragma unroll 1
            for (int j = 0; j < item.n; ++j, ++n) {
                const int st = n & 1;
                const uint32_t t_s = tmem + lanes + kColS + (uint32_t)st * kTile;
                wait(S_FULL + st, n >> 1 & 1);
                wait(SCALES + n % kScales, n / kScales & 1);
                tc_fence_after();
                if (idle) { warp_arrive(bar(P_FULL + st), lane); continue; }     // (what its rows hold reaches no row of the result)
                const Scales& sc = *reinterpret_cast<const Scales*>(smem + kOffScales + n % kScales * sizeof(Scales));
                const int first = (item.first + j) * kTile, left = item.tokens - first;
                const bool masked = first + kTile > tail || left < kTile;
                float s[32];
                tmem_ld32(t_s + 32u * half, reinterpret_cast<uint32_t*>(s));
                tmem_wait_ld();
#pragma unroll
                for (int c = 0; c < 32; c += 4) {
                    const float4 k = *reinterpret_cast<const float4*>(sc.k + 32 * half + c);
                    const float2 lo = unpack2(mul2(pack2(s[c], s[c + 1]), pack2(k.x, k.y))), hi = unpack2(mul2(pack2(s[c + 2], s[c + 3]), pack2(k.z, k.w)));
                    s[c] = lo.x; s[c + 1] = lo.y; s[c + 2] = hi.x; s[c + 3] = hi.y;
                }
                uint32_t seen = ~0u;                                    // of the thread's 32 tokens, those that the row sees
                if (masked) {
                    const int before = tail - first;                    // tokens of the tile ahead of the last R (may be negative, or all)
                    unsigned long long all = before >= kTile ? ~0ull : before >= 0 ? mask << before | ((1ull << before) - 1ull) : before > -kTile ? mask >> -before : 0ull;
                    if (left < kTile) all &= left <= 0 ? 0ull : (1ull << left) - 1ull;
                    seen = (uint32_t)(all >> (32 * half));
#pragma unroll
                    for (int c = 0; c < 32; ++c)
                        if (!(seen >> c & 1)) s[c] = -INFINITY;
                }
                float top4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < 32; c += 2) top4[c >> 1 & 3] = max3(top4[c >> 1 & 3], s[c], s[c + 1]);
                float top = max3(fmaxf(top4[0], top4[1]), top4[2], top4[3]) * factor;
                // (here both have their scores, so either may write P over them)
                if (bar_red_or<64>(meet, top + neg_m > kSlack || sc.unit_exp > unit_exp)) {
                    // ---- seldom: the maximum moves, or the unit (in a tile that the row does not see all of, by what it sees)
                    int unit = sc.unit_exp;
                    if (masked) {
                        unit = unit_exp;
#pragma unroll 4
                        for (int c = 0; c < 32; ++c)
                            if (seen >> c & 1) unit = max(unit, unit_of(sc.v[32 * half + c]));
                    }
                    *mine = top; mine[2 * kRows] = __int_as_float(unit);
                    bar_sync_id<64>(meet);
                    top = fmaxf(top, *other); unit = max(unit, __float_as_int(other[2 * kRows]));
                    const float was = neg_m;
                    neg_m = fminf(was, -top);
                    const float back = ex2(neg_m - was), both = unit_exp - unit < -126 ? 0.f : back * power_of_two(unit_exp - unit);
                    unit_exp = unit;
                    l *= back;
                    if (j > 0) {
                        wait(V_EMPTY, (n - 1) & 1);                     // the P V before this tile's
                        tc_fence_after();
#pragma unroll 1
                        for (int ch = 0; ch < 4; ++ch) {
                            uint32_t o[16];
                            tmem_ld16(t_o + 16u * ch, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * both);
                            tmem_st16(t_o + 16u * ch, o);
                        }
                    }
                }
                const uint64_t neg2 = pack2(neg_m, neg_m);
                uint64_t sum[2] = {0, 0};
                uint32_t w[16];
                const float up = up_of(unit_exp);
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const float4 v = *reinterpret_cast<const float4*>(sc.v + 32 * half + 4 * c);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const float2 d = unpack2(fma2(pack2(s[4 * c + 2 * k], s[4 * c + 2 * k + 1]), factor2, neg2));
                        const uint64_t e = pack2(ex2(d.x), ex2(d.y));
                        sum[k] = add2(sum[k], e);
                        const float2 y = unpack2(mul2(e, mul2(k ? pack2(v.z, v.w) : pack2(v.x, v.y), pack2(up, up))));
                        w[2 * c + k] = pack_half2(y.x, y.y);
                    }
                }
                if (masked)                                             // a hidden token's scale may be a NaN
#pragma unroll
                    for (int c = 0; c < 16; ++c)
                        w[c] &= (seen >> (2 * c) & 1 ? 0xffffu : 0u) | (seen >> (2 * c + 1) & 1 ? 0xffff0000u : 0u);
                tmem_st16(t_s + 16u * half, w);
                tmem_wait_st();
                tc_fence_before();
                warp_arrive(bar(P_FULL + st), lane);
                const float2 both = unpack2(add2(sum[0], sum[1]));
                l += both.x + both.y;
            }

            // ---- the piece's rows
            wait(O_FULL, pieces & 1);
            tc_fence_after();
            const bool whole = item.whole(), valid = r < rows;
            const Kv8Parts cut = kv8_parts(item, run);
            const size_t slot = 2 * (size_t)blockIdx.x + (item.nth == 0 ? 0 : 1);
            auto write_lse = [&](size_t row, float m, float sum) {      // natural logarithm
                p.lse[row] = sum == 0.f ? -INFINITY : (m + log2_approx(sum)) * 0.6931471805599453f;
            };
            if (!idle) {
                mine[2 * kRows] = l;
                bar_sync_id<64>(meet);
                l += other[2 * kRows];
                const float inv = l == 0.f ? 0.f : 1.f / l, unit = power_of_two(unit_exp - 127 - kRoom);     // (a row that saw nothing: zeros)
                const size_t at = ((size_t)item.b * p.R + i_row) * p.Hq + head;
#pragma unroll 1
                for (int ch = 0; ch < 4; ++ch) {
                    float o[16];
                    tmem_ld16(t_o + 16u * ch, reinterpret_cast<uint32_t*>(o));
                    tmem_wait_ld();
#pragma unroll
                    for (int c = 0; c < 16; ++c) o[c] = l == 0.f ? 0.f : o[c] * inv * unit;
                    if (!valid) continue;
                    const int dim = 64 * half + 16 * ch;
                    if (!whole || p.out_dtype == TTS_OUT_FP32) {
                        float* to = whole ? static_cast<float*>(p.out) + at * kHeadDim : p.part_o + (slot * kRows + r) * kHeadDim;
                        if (whole)
#pragma unroll
                            for (int c = 0; c < 16; c += 4) *reinterpret_cast<float4*>(to + dim + c) = make_float4(o[c], o[c + 1], o[c + 2], o[c + 3]);
                        else { st_global_32(to + dim, o); st_global_32(to + dim + 8, o + 8); }
                    } else {
                        uint4* to = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + at * kHeadDim + dim);
                        to[0] = make_uint4(bf16_pair(o[0], o[1]), bf16_pair(o[2], o[3]), bf16_pair(o[4], o[5]), bf16_pair(o[6], o[7]));
                        to[1] = make_uint4(bf16_pair(o[8], o[9]), bf16_pair(o[10], o[11]), bf16_pair(o[12], o[13]), bf16_pair(o[14], o[15]));
                    }
                }
                if (valid && half == 0) {
                    if (!whole) p.part_ml[slot * kRows + r] = make_float2(-neg_m, l);
                    else if (p.lse) write_lse(at, -neg_m, l);
                }
            }
            tc_fence_before();                                          // O and Q have been read, before the next piece's products
            if (!whole) {
                // ---- the last CTA to leave a part of the item joins them all
                const size_t id = ((size_t)item.b * p.Hkv + h) * p.n_rb + (item.item - h * p.n_rb);
                __threadfence();
                warp_arrive(bar(PART_DONE), lane);
                if (threadIdx.x == 0) {
                    int last = 0;
                    if (alive && mbar_wait(bar(PART_DONE), parts_left & 1, ab)) {
                        unsigned before;
                        asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(before) : "l"(p.arrived + id) : "memory");
                        last = before + 1 == (unsigned)cut.n;
                        if (last) p.arrived[id] = 0;                    // as the next call expects it
                    }
                    misc[2] = last;
                    __threadfence();
                    mbar_arrive(bar(PART_LAST));
                }
                __syncwarp();
                wait(PART_LAST, parts_left & 1);
                ++parts_left;
                if (alive && misc[2]) {
                    __threadfence();
                    // sixteen rows to a warp: a lane finds one's maximum and sum, then four rows at a time, four dims a lane
                    const int q = warp * 16 + (lane & 15);
                    float m = kFar, sum = 0.f;
                    if (q < rows)
#pragma unroll 2
                        for (int k = 0; k < cut.n; ++k) {
                            const float2 x = __ldcg(p.part_ml + (size_t)cut.slot(k) * kRows + q);
                            const float now = fmaxf(m, x.x);
                            sum = sum * ex2(m - now) + x.y * ex2(x.x - now);
                            m = now;
                        }
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;
                    auto place = [&](int row) { const int s = row0 + row, i = s / p.G; return ((size_t)item.b * p.R + i) * p.Hq + h * p.G + s - i * p.G; };
                    if (p.lse && lane < 16 && q < rows) write_lse(place(q), m, sum);
#pragma unroll 1
                    for (int g = 0; g < 16 && warp * 16 + g < rows; g += 4) {
                        float4 acc[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
                        for (int k = 0; k < cut.n; ++k) {
                            const size_t from = (size_t)cut.slot(k) * kRows + warp * 16;
                            const float2 x = __ldcg(p.part_ml + from + (lane & 15));
                            const float weight = x.y * ex2(x.x - m) * inv;
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                // (rows behind the last one: whatever lies in the workspace, not written anywhere)
                                const float4 y = __ldcg(reinterpret_cast<const float4*>(p.part_o + (from + g + i) * kHeadDim) + lane);
                                const float f = __shfl_sync(0xffffffffu, weight, g + i);
                                acc[i].x = fmaf(f, y.x, acc[i].x); acc[i].y = fmaf(f, y.y, acc[i].y); acc[i].z = fmaf(f, y.z, acc[i].z); acc[i].w = fmaf(f, y.w, acc[i].w);
                            }
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (warp * 16 + g + i >= rows) break;
                            const size_t to = place(warp * 16 + g + i) * kHeadDim + lane * 4;
                            const float v[4] = {acc[i].x, acc[i].y, acc[i].z, acc[i].w};
                            if (p.out_dtype == TTS_OUT_FP32) *reinterpret_cast<float4*>(static_cast<float*>(p.out) + to) = make_float4(v[0], v[1], v[2], v[3]);
                            else *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + to) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
                        }
                    }
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

}  // namespace

cudaError_t launch_kv8_attn_wide(const Kv8AttnParams& p, int format, cudaStream_t st) {
    auto launch = [&](auto kernel) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
        return e != cudaSuccess ? e : launch_dependent(kernel, p.grid, kThreads, kSmemBytes, st, p);
    };
    return format == TTS_KV8_E4M3 ? launch(kv8_attn_wide_kernel<TTS_KV8_E4M3>) : launch(kv8_attn_wide_kernel<TTS_KV8_INT8>);
}

}  // namespace tts
