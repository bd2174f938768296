// Attention of many rows per KV head (draft trees, long drafted chains with large head groups) over the 8-bit cache.
//
// The formula and the roundings of kv8_attn.cu, for which a row block is too much to hold in a warp's registers: there the codes of
// a page become operands once for 24 rows, here once for 128, and the products are the tensor cores' own.
//
// Bound by the tensor cores and the exponentials alike: 64 tokens and 128 rows take 512 clocks of either.  Two CTAs share an SM, so
// that one's exponentials run while the tensor cores work for the other.  In a CTA,
//   warps 0-3  softmax, a thread to a row: its query becomes the row's A operand in TMEM; per tile of 64 tokens it reads its scores
//              from TMEM and leaves p sv there, as the second product's A operand; O is touched only when the maximum moves by more
//              than 2^8 or the unit of p sv grows.  At a piece's end it writes its row.
//   warps 4-7  turn codes into fp16 operands (exact): [64 tokens][128 dims], K with dims along the contraction, V with tokens.  Warp 4
//              also fetches the records, by bulk copies into a ring of two tiles; warp 5 leaves the tile's scales and the unit.
//   warp 8     issues the products: S = Q K^T (128 x 64 x 128), then O += P V (128 x 128 x 64).  The tensor pipe keeps issue order, so
//              S of a tile may overwrite the columns that held P of the one before, and is complete no earlier than that one's P V.
// TMEM columns of a CTA: Q 64, S 64 (P in its first half), O 128.
#include <cuda_fp16.h>

#include "kv8_run.cuh"
#include "launch.cuh"
#include "umma_ptx.cuh"

namespace tts {

namespace {

using namespace ptx;

constexpr int kTile = 64, kTilePages = kTile / kPage;
constexpr int kRows = kKv8WideRows;
constexpr int kSoftmaxWarps = 4, kConvertWarps = 4, kMmaWarp = kSoftmaxWarps + kConvertWarps;
constexpr int kThreads = (kMmaWarp + 1) * 32;
// registers per thread: at launch (two CTAs of nine warps, five to a scheduler), and after the softmax has taken from the converting warps
constexpr int kLaunchRegs = 96, kSoftmaxRegs = 136, kConvertRegs = 56;
static_assert(kSoftmaxRegs + kConvertRegs <= 2 * kLaunchRegs, "the split draws on what the block was launched with");
constexpr float kFar = -1e30f;                                      // "no key yet": finite, so that differences are never NaN
constexpr float kSlack = 8.f;                                       // log2 of how far a score may exceed the running maximum
constexpr int kRoom = 6;                                            // p sv is held times 2^kRoom
constexpr uint32_t kTmemCols = 256, kColQ = 0, kColS = 64, kColO = 128;
// An item's start and end take about as long as so many tiles.
constexpr int kItemUnits = 4;
constexpr int kWholeTiles = 16;
using Walk = Kv8Walk<kTile, kItemUnits>;

constexpr int kOperand = kTile * kHeadDim * 2;                      // fp16 K, and V, of a tile: two blocks of 64 dims, rows of 128 bytes
constexpr int kBlock = kOperand / 2;
constexpr int kRawTile = kTilePages * kKv8Record;
// what the softmax needs of a tile besides its scores
struct Scales {
    float k[kTile], v[kTile];                                       // K's; V's in the unit, times 2^kRoom
    float unit_back;                                                // what O is multiplied by before the tile's P V: the unit has grown
    int unit_exp;                                                   // exponent field of the unit
    int pad[2];
};
constexpr int kOffK = 0;                                            // two stages
constexpr int kOffV = kOffK + 2 * kOperand;
constexpr int kOffRaw = kOffV + 2 * kOperand;                       // two stages
constexpr int kOffScales = kOffRaw + 2 * kRawTile;
constexpr int kOffCum = kOffScales + 2 * (int)sizeof(Scales);
constexpr int kOffSums = kOffCum + (kMaxBranches + 8) * 8;          // scratch of the scan
enum Bar { RAW_FULL = 0, RAW_EMPTY = 2, KV_FULL = 4, KV_EMPTY = 6, Q_FULL = 8, S_FULL, P_FULL, O_FULL, PART_DONE, PART_LAST, DRAINED, kNumBars };
constexpr int kOffBar = kOffSums + (kThreads / 32) * 8 + 8;
constexpr int kOffMisc = kOffBar + kNumBars * 8;                    // [0] abort, [1] TMEM base, [2] the last part, [3, 4] scratch of the copying and the MMA warp
constexpr int kSmemBytes = kOffMisc + 32;
static_assert(kOffBar % 8 == 0 && kOffRaw % 128 == 0 && sizeof(Scales) % 16 == 0 && 2 * (kSmemBytes + 1024) <= 228 * 1024, "two CTAs to an SM");

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
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
__device__ __forceinline__ float log2_approx(float x) { float y; asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ bool elect_one() {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok));
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
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(RAW_FULL + i), 1); mbar_init(bar(RAW_EMPTY + i), kConvertWarps);
            mbar_init(bar(KV_FULL + i), kConvertWarps); mbar_init(bar(KV_EMPTY + i), 1);
        }
        mbar_init(bar(Q_FULL), kSoftmaxWarps); mbar_init(bar(S_FULL), 1); mbar_init(bar(P_FULL), kSoftmaxWarps); mbar_init(bar(O_FULL), 1);
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
    const Kv8Run run = kv8_run<kThreads, kItemUnits>(p, cum, kItemUnits, kWholeTiles);
    Walk item;
    bool alive = run.n > 0 && item.init(p, cum, run.begin, run.n);      // every role walks over the pieces for itself

    if (warp >= kSoftmaxWarps && warp < kMmaWarp) {
        // =========================== records to operands ===========================
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kConvertRegs));
        const int w = warp - kSoftmaxWarps, ct = w * 32 + lane;
        // warp 0 of these: the copies, two tiles ahead
        Walk ahead = item;
        int ahead_tile = 0, copied = 0;
        bool more = alive;
        auto copy = [&]() {                                             // the next tile of the run into stage copied mod 2
            if (!more) return;
            const int first = (ahead.first + ahead_tile) * kTile;
            const uint32_t full = bar(RAW_FULL + (copied & 1));
            const bool wanted = lane < kTilePages && first + lane * kPage < ahead.tokens;
            const int page = wanted ? p.block_table[(size_t)ahead.b * p.max_blocks + first / kPage + lane] : 0;
            const bool there = wanted && page >= 0 && page < p.num_pages;
            const unsigned good = __ballot_sync(0xffffffffu, there), bad = __ballot_sync(0xffffffffu, wanted && !there);
            unsigned char* dst = smem + kOffRaw + (copied & 1) * kRawTile;
            if (bad) {                                                  // a page outside the pool counts as zeros
                if (lane == 0) atomicMin(p.status, (int)TTS_ERR_DEVICE_BOUNDS);
                for (int pg = 0; pg < kTilePages; ++pg)
                    if (bad >> pg & 1)
                        for (int i = lane; i < kKv8Record / 16; i += 32) *reinterpret_cast<uint4*>(dst + pg * kKv8Record + i * 16) = make_uint4(0, 0, 0, 0);
                fence_proxy_async();                                    // (before a later copy into the stage)
                __syncwarp();
            }
            if (lane == 0) { if (good) mbar_arrive_expect_tx(full, __popc(good) * kKv8Record); else mbar_arrive(full); }
            __syncwarp();
            if (there) bulk_load(smem_u32(dst) + lane * kKv8Record, p.pool + ((size_t)page * p.Hkv + ahead.item / p.n_rb) * kKv8Record, kKv8Record, full);
            ++copied;
            if (++ahead_tile >= ahead.n) { ahead_tile = 0; more = ahead.next(p); }
        };
        if (w == 0) { copy(); copy(); }
        int n = 0;                                                      // tiles of the run so far
        int unit_exp = 7;
        for (bool more_items = alive; more_items && alive; more_items = item.next(p)) {
            unit_exp = 7;
            for (int j = 0; j < item.n; ++j, ++n) {
                const int st = n & 1, round = n >> 1 & 1;
                const int left = min(kTile, item.tokens - (item.first + j) * kTile);       // tokens here (may be 0)
                const unsigned char* raw = smem + kOffRaw + st * kRawTile;
                alive = mbar_wait(bar(RAW_FULL + st), round, ab) && mbar_wait(bar(KV_EMPTY + st), round ^ 1, ab);
                alive = __all_sync(0xffffffffu, alive);
                if (!alive) break;
                if (w == 1) {
                    Scales& to = *reinterpret_cast<Scales*>(smem + kOffScales + st * sizeof(Scales));
                    float k[2], v[2];
                    int top = 0;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int t = i * 32 + lane;
                        const float* s = reinterpret_cast<const float*>(raw + (t >> 4) * kKv8Record + 2 * kKv8Codes) + (t & 15);
                        k[i] = t < left ? s[0] : 0.f; v[i] = t < left ? s[kPage] : 0.f;
                        const int e = __float_as_int(v[i]) >> 23 & 255;
                        top = max(top, e == 255 ? 0 : e);               // (a NaN or an infinity is not a unit)
                    }
                    const int e = max(unit_exp, __reduce_max_sync(0xffffffffu, top));
                    const float back = j == 0 ? 1.f : unit_exp - e < -126 ? 0.f : power_of_two(unit_exp - e), up = power_of_two(kRoom + 127 - e);
                    unit_exp = e;
#pragma unroll
                    for (int i = 0; i < 2; ++i) { to.k[i * 32 + lane] = k[i]; to.v[i * 32 + lane] = v[i] * up; }
                    if (lane == 0) { to.unit_back = back; to.unit_exp = e; }
                }
                // Eight lanes have a token's 128 codes; codes 16 c .. of a token become 16-byte chunks 2 c and 2 c + 1 of its row.
                // Lanes with c >= 4 write the second one first: eight different bank groups.
#pragma unroll
                for (int kv = 0; kv < 2; ++kv)
#pragma unroll
                    for (int i = 0; i < kTile * 8 / (kConvertWarps * 32); ++i) {
                        const int t = i * (kConvertWarps * 4) + (ct >> 3), c = (ct & 7) ^ kv8_chunk_place(t & 15);
                        uint4 x = *reinterpret_cast<const uint4*>(raw + (t >> 4) * kKv8Record + kv * kKv8Codes + (t & 15) * kHeadDim + (ct & 7) * 16);
                        if (kv == 1 && t >= left) x = make_uint4(0, 0, 0, 0);       // what is not there: 0 x NaN would be NaN (K's scores are replaced)
                        const bool odd = c >= 4;
                        unsigned char* to = smem + (kv ? kOffV : kOffK) + st * kOperand + (c >> 2) * kBlock + t * 128;
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            const bool second = odd != (half == 1);
                            const uint32_t a = kv8_biased<kFormat>(second ? x.z : x.x), b = kv8_biased<kFormat>(second ? x.w : x.y);
                            *reinterpret_cast<uint4*>(to + ((((2 * c + (second ? 1 : 0)) & 7) ^ (t & 7)) << 4)) =
                                make_uint4(kv8_decode2<kFormat>(a, 0), kv8_decode2<kFormat>(a, 1), kv8_decode2<kFormat>(b, 0), kv8_decode2<kFormat>(b, 1));
                        }
                    }
                fence_proxy_async();                                    // the operands, for the tensor cores
                __syncwarp();
                if (lane == 0) { mbar_arrive(bar(KV_FULL + st)); mbar_arrive(bar(RAW_EMPTY + st)); }
                if (w == 0 && more) {
                    alive = __all_sync(0xffffffffu, mbar_wait(bar(RAW_EMPTY + st), round, ab));
                    if (!alive) break;
                    copy();
                }
            }
        }
        if (w == 0 && *ab.flag) {
            // after a wait that ran out: copies in flight land before the CTA ends
            const Abort quiet{misc + 3, p.status};
            for (int i = max(0, copied - 2); i < copied; ++i) { misc[3] = 0; mbar_wait(bar(RAW_FULL + (i & 1)), i >> 1 & 1, quiet); }
        }
    } else if (warp == kMmaWarp) {
        // =========================== products ===========================
        constexpr uint32_t idesc_qk = f16_desc(kRows, kTile, false), idesc_pv = f16_desc(kRows, kHeadDim, true);
        const uint64_t k_desc = smem_desc(sbase + kOffK, 16, 1024), v_desc = smem_desc(sbase + kOffV, kBlock, 1024);
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);          // (a shuffle tells the compiler that the value is uniform)
        int n = 0, pieces = 0;
        for (bool more_items = alive; more_items && alive; more_items = item.next(p), ++pieces) {
            const int tiles = __shfl_sync(0xffffffffu, item.n, 0);
            alive = __all_sync(0xffffffffu, mbar_wait(bar(Q_FULL), pieces & 1, ab));
            for (int j = 0; alive && j < tiles; ++j, ++n) {
                const uint32_t st = n & 1;
                alive = __all_sync(0xffffffffu, mbar_wait(bar(KV_FULL + st), n >> 1 & 1, ab));
                if (!alive) break;
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks)
                        umma_bf16_tmem_a(tm + kColS, tm + kColQ + ks * 8u, k_desc + (st * kOperand + (ks >> 2) * kBlock + (ks & 3) * 32) / 16, idesc_qk, ks > 0);
                    umma_commit(bar(S_FULL));
                }
                __syncwarp();
                alive = __all_sync(0xffffffffu, mbar_wait(bar(P_FULL), n & 1, ab));
                if (!alive) break;
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int ks = 0; ks < kTilePages; ++ks)
                        umma_bf16_tmem_a(tm + kColO, tm + kColS + ks * 8u, v_desc + (st * kOperand + ks * 2048) / 16, idesc_pv, ks > 0 || j > 0);
                    umma_commit(bar(KV_EMPTY + st));
                    if (j + 1 == tiles) umma_commit(bar(O_FULL));
                }
                __syncwarp();
            }
        }
        if (__any_sync(0xffffffffu, *ab.flag != 0)) {
            // products in flight end before their operands' shared memory and TMEM are someone else's
            if (elect_one()) {
                misc[4] = 0;
                umma_commit(bar(DRAINED));
            }
            __syncwarp();
            mbar_wait(bar(DRAINED), 0, Abort{misc + 4, p.status});
            __syncwarp();
        }
    } else if (warp < kSoftmaxWarps) {
        // =========================== softmax ===========================
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        const uint32_t lanes = (uint32_t)(warp * 32) << 16;
        const uint32_t t_q = tmem + lanes + kColQ, t_s = tmem + lanes + kColS, t_o = tmem + lanes + kColO;
        int n = 0, pieces = 0, parts_left = 0;
        for (bool more_items = alive; more_items && alive; more_items = item.next(p), ++pieces) {
            const int h = item.item / p.n_rb, row0 = (item.item - h * p.n_rb) * p.rb_rows, rows = min(p.rb_rows, p.nr - row0);
            const int r = threadIdx.x, stacked = row0 + min(r, rows - 1), i_row = stacked / p.G, head = h * p.G + stacked - i_row * p.G;
            const bool idle = warp * 32 >= rows;                        // no row of the block is this warp's
            const int tail = item.tokens - p.R;                         // the first of the branch's last R tokens (may be negative)
            float factor = 0.f;
            unsigned long long mask = 0;                                // which of the branch's last R tokens the row sees
            if (!idle) {
                // ---- the query, scaled to fp16 by the power of two that puts its largest at 2^14
                const uint4* src = reinterpret_cast<const uint4*>(p.q + ((size_t)item.b * p.R + i_row) * p.q_stride + (size_t)head * kHeadDim);
                uint32_t x[64];
#pragma unroll
                for (int i = 0; i < 16; ++i) { const uint4 y = src[i]; x[4 * i] = y.x; x[4 * i + 1] = y.y; x[4 * i + 2] = y.z; x[4 * i + 3] = y.w; }
                uint32_t top = 0;                                       // the largest finite magnitude, as bits
#pragma unroll
                for (int i = 0; i < 64; ++i) {
                    const uint32_t lo = x[i] << 16 & 0x7fffffffu, hi = x[i] & 0x7fff0000u;
                    top = max(top, max(lo < 0x7f800000u ? lo : 0u, hi < 0x7f800000u ? hi : 0u));
                }
                const int e = max(-100, min(126, (int)(top >> 23) - 127)) - 14;
                const float down = power_of_two(-e);
#pragma unroll
                for (int i = 0; i < 64; ++i) x[i] = pack_half2(__uint_as_float(x[i] << 16) * down, __uint_as_float(x[i] & 0xffff0000u) * down);
                tmem_st32(t_q, x);
                tmem_st32(t_q + 32u, x + 32);
                tmem_wait_st();
                factor = power_of_two(e) * p.scale_log2;
                if (p.tree_parents == nullptr) mask = i_row >= 63 ? ~0ull : (2ull << i_row) - 1ull;
                else
                    for (int a = i_row, guard = 0; a >= 0 && guard < kMaxTreeRows; ++guard) {
                        mask |= 1ull << a;
                        const int parent = p.tree_parents[(size_t)item.b * p.R + a];
                        a = parent < a ? parent : -1;                   // malformed parents end the walk
                    }
            }
            tc_fence_before();
            warp_arrive(bar(Q_FULL), lane);
            float neg_m = -kFar, l = 0.f;
            int unit_exp = 7;
            const uint64_t factor2 = pack2(factor, factor);
#pragma unroll 1
            for (int j = 0; j < item.n; ++j, ++n) {
                const int st = n & 1;
                alive = __all_sync(0xffffffffu, mbar_wait(bar(S_FULL), n & 1, ab) && mbar_wait(bar(KV_FULL + st), n >> 1 & 1, ab));
                if (!alive) break;
                tc_fence_after();
                if (idle) { warp_arrive(bar(P_FULL), lane); continue; }     // (what its rows hold reaches no row of the result)
                const Scales& sc = *reinterpret_cast<const Scales*>(smem + kOffScales + st * sizeof(Scales));
                const int first = (item.first + j) * kTile, left = item.tokens - first;
                const bool masked = first + kTile > tail || left < kTile;
                float s[kTile];
                tmem_ld32(t_s, reinterpret_cast<uint32_t*>(s));
                tmem_ld32(t_s + 32u, reinterpret_cast<uint32_t*>(s) + 32);
                tmem_wait_ld();
#pragma unroll
                for (int c = 0; c < kTile; c += 4) {
                    const float4 k = *reinterpret_cast<const float4*>(sc.k + c);
                    const float2 lo = unpack2(mul2(pack2(s[c], s[c + 1]), pack2(k.x, k.y))), hi = unpack2(mul2(pack2(s[c + 2], s[c + 3]), pack2(k.z, k.w)));
                    s[c] = lo.x; s[c + 1] = lo.y; s[c + 2] = hi.x; s[c + 3] = hi.y;
                }
                unsigned long long seen = ~0ull;                        // tokens of the tile that the row sees
                if (masked) {
                    const int before = tail - first;                    // tokens of the tile ahead of the last R (may be negative, or all)
                    seen = before >= kTile ? ~0ull : before >= 0 ? mask << before | ((1ull << before) - 1ull) : before > -kTile ? mask >> -before : 0ull;
                    if (left < kTile) seen &= left <= 0 ? 0ull : (1ull << left) - 1ull;
#pragma unroll
                    for (int c = 0; c < kTile; ++c)
                        if (!(seen >> c & 1)) s[c] = -INFINITY;
                }
                float top4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < kTile; c += 2) top4[c >> 1 & 3] = fmaxf(top4[c >> 1 & 3], fmaxf(s[c], s[c + 1]));
                const float top = fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3])) * factor;
                const float unit_back = sc.unit_back;
                unit_exp = sc.unit_exp;
                if (__any_sync(0xffffffffu, top + neg_m > kSlack) || unit_back != 1.f) {
                    // ---- seldom: the maximum moves, or the unit
                    const float was = neg_m;
                    neg_m = fminf(was, -top);
                    const float back = ex2(neg_m - was);
                    l *= back;
                    const float both = back * unit_back;
                    if (j > 0)                                          // (S of this tile is complete, so the P V before it is as well)
#pragma unroll 1
                        for (int ch = 0; ch < 8; ++ch) {
                            uint32_t o[16];
                            tmem_ld16(t_o + 16u * ch, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * both);
                            tmem_st16(t_o + 16u * ch, o);
                        }
                }
                const uint64_t neg2 = pack2(neg_m, neg_m);
                uint64_t sum[2] = {0, 0};
                uint32_t w[kTile / 2];
#pragma unroll
                for (int c = 0; c < kTile / 4; ++c) {
                    const float4 v = *reinterpret_cast<const float4*>(sc.v + 4 * c);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const float2 d = unpack2(fma2(pack2(s[4 * c + 2 * k], s[4 * c + 2 * k + 1]), factor2, neg2));
                        const uint64_t e = pack2(ex2(d.x), ex2(d.y));
                        sum[k] = add2(sum[k], e);
                        const float2 y = unpack2(mul2(e, k ? pack2(v.z, v.w) : pack2(v.x, v.y)));
                        w[2 * c + k] = pack_half2(y.x, y.y);
                    }
                }
                if (masked)                                             // a hidden token's scale may be a NaN
#pragma unroll
                    for (int c = 0; c < kTile / 2; ++c)
                        w[c] &= (seen >> (2 * c) & 1 ? 0xffffu : 0u) | (seen >> (2 * c + 1) & 1 ? 0xffff0000u : 0u);
                tmem_st32(t_s, w);
                tmem_wait_st();
                tc_fence_before();
                warp_arrive(bar(P_FULL), lane);
                const float2 both = unpack2(add2(sum[0], sum[1]));
                l += both.x + both.y;
            }
            if (!alive) break;

            // ---- the piece's rows
            alive = __all_sync(0xffffffffu, mbar_wait(bar(O_FULL), pieces & 1, ab));
            if (!alive) break;
            tc_fence_after();
            const bool whole = item.whole(), mine = r < rows;
            const Kv8Parts cut = kv8_parts(item, run.begin + (run.n - item.left), run.per_cta);
            const size_t slot = 2 * (size_t)blockIdx.x + (item.nth == 0 ? 0 : 1);
            const size_t at = ((size_t)item.b * p.R + i_row) * p.Hq + head;
            auto write_out = [&](size_t row, int dim, const float* v) {         // 16 values
                if (p.out_dtype == TTS_OUT_FP32) {
                    float* to = static_cast<float*>(p.out) + row * kHeadDim + dim;
#pragma unroll
                    for (int c = 0; c < 16; c += 4) *reinterpret_cast<float4*>(to + c) = make_float4(v[c], v[c + 1], v[c + 2], v[c + 3]);
                } else {
                    uint4* to = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + row * kHeadDim + dim);
                    to[0] = make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
                    to[1] = make_uint4(bf16_pair(v[8], v[9]), bf16_pair(v[10], v[11]), bf16_pair(v[12], v[13]), bf16_pair(v[14], v[15]));
                }
            };
            auto write_lse = [&](size_t row, float m, float sum) {      // natural logarithm
                p.lse[row] = sum == 0.f ? -INFINITY : (m + log2_approx(sum)) * 0.6931471805599453f;
            };
            if (!idle) {
                const float inv = l == 0.f ? 0.f : 1.f / l, unit = power_of_two(unit_exp - 127 - kRoom);     // (a row that saw nothing: zeros)
#pragma unroll 1
                for (int ch = 0; ch < 8; ++ch) {
                    float o[16];
                    tmem_ld16(t_o + 16u * ch, reinterpret_cast<uint32_t*>(o));
                    tmem_wait_ld();
#pragma unroll
                    for (int c = 0; c < 16; ++c) o[c] = l == 0.f ? 0.f : o[c] * inv * unit;
                    if (mine && whole) write_out(at, 16 * ch, o);
                    else if (mine) {
                        float* to = p.part_o + (slot * kRows + r) * kHeadDim + 16 * ch;
                        st_global_32(to, o); st_global_32(to + 8, o + 8);
                    }
                }
                if (mine && !whole) p.part_ml[slot * kRows + r] = make_float2(-neg_m, l);
                if (mine && whole && p.lse) write_lse(at, -neg_m, l);
            }
            tc_fence_before();                                          // O and Q have been read, before the next piece's products
            if (!whole) {
                // ---- the last CTA to leave a part of the item joins them all
                const size_t id = ((size_t)item.b * p.Hkv + h) * p.n_rb + (item.item - h * p.n_rb);
                __threadfence();
                warp_arrive(bar(PART_DONE), lane);
                if (threadIdx.x == 0) {
                    int last = 0;
                    if (mbar_wait(bar(PART_DONE), parts_left & 1, ab)) {
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
                alive = __all_sync(0xffffffffu, mbar_wait(bar(PART_LAST), parts_left & 1, ab));
                ++parts_left;
                if (!alive) break;
                if (misc[2]) {
                    __threadfence();
                    // a warp to a row, four dims a lane
                    for (int q = warp; q < rows; q += kSoftmaxWarps) {
                        float m = kFar, sum = 0.f;
                        for (int k0 = 0; k0 < cut.n; k0 += 32) {
                            const float2 x = k0 + lane < cut.n ? __ldcg(p.part_ml + (size_t)cut.slot(k0 + lane) * kRows + q) : make_float2(kFar, 0.f);
                            float now = fmaxf(m, x.x);
#pragma unroll
                            for (int o = 1; o < 32; o <<= 1) now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, o));
                            float add = x.y * ex2(x.x - now);
#pragma unroll
                            for (int o = 1; o < 32; o <<= 1) add += __shfl_xor_sync(0xffffffffu, add, o);
                            sum = sum * ex2(m - now) + add;
                            m = now;
                        }
                        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
                        for (int k = 0; k < cut.n; ++k) {
                            const size_t from = (size_t)cut.slot(k) * kRows + q;
                            const float2 x = __ldcg(p.part_ml + from);
                            const float4 y = __ldcg(reinterpret_cast<const float4*>(p.part_o + from * kHeadDim) + lane);
                            const float f = x.y * ex2(x.x - m);
                            acc.x = fmaf(f, y.x, acc.x); acc.y = fmaf(f, y.y, acc.y); acc.z = fmaf(f, y.z, acc.z); acc.w = fmaf(f, y.w, acc.w);
                        }
                        const float inv = sum == 0.f ? 0.f : 1.f / sum;
                        const int s = row0 + q, i = s / p.G;
                        const size_t row = ((size_t)item.b * p.R + i) * p.Hq + h * p.G + s - i * p.G, to = row * kHeadDim + lane * 4;
                        if (p.out_dtype == TTS_OUT_FP32) *reinterpret_cast<float4*>(static_cast<float*>(p.out) + to) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
                        else *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + to) = make_uint2(bf16_pair(acc.x * inv, acc.y * inv), bf16_pair(acc.z * inv, acc.w * inv));
                        if (p.lse && lane == 0) write_lse(row, m, sum);
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
