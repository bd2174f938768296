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

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr int kStages = 4;                                          // pages of a warp in flight
constexpr int kMinUnits = kWarps;                                   // a CTA takes at least a page for each warp
constexpr float kFar = -1e30f;                                      // "no key yet": finite, so that differences are never NaN
constexpr float kSlack = 8.f;                                       // log2 of how far a score may exceed the running maximum
constexpr int kRoom = 6;                                            // p sv is held times 2^kRoom

// shared memory (bytes)
constexpr int kOffRing = 0;
constexpr int kOffQ = kOffRing + kWarps * kStages * kKv8Record;     // [rows][256]: fp16 rows, 16-byte chunks exchanged (q_place)
constexpr int kOffMask = kOffQ + kKv8MaxRows * kHeadDim * 2;        // [rows] which of the branch's last rows each row sees
constexpr int kOffFactor = kOffMask + kKv8MaxRows * 8;              // [rows] what a row's scores are multiplied by
constexpr int kOffMl = kOffFactor + kKv8MaxRows * 4;                // [warps][rows] (maximum, sum)
constexpr int kOffExp = kOffMl + kWarps * kKv8MaxRows * 8;          // [warps] exponent of the sums' unit; then flags
constexpr int kOffCum = kOffExp + 64;                               // [branches + 1] units before each branch
constexpr int kOffJoin = kOffCum + (kMaxBranches + 8) * 8;          // [warps][rows][64] floats
template <int kNB> constexpr int smem_bytes() { return kOffJoin + kWarps * kNB * 8 * 64 * 4; }
static_assert(smem_bytes<4>() <= 232448, "shared memory of a CTA");

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
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ float exp2_approx(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
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
        for (int w = 0; w < kWarps; ++w) {
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
    const long long within = unit - cum[lo];
    at.item = (int)(within / at.units);
    at.page = (int)(within - (long long)at.item * at.units);
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

template <int kFormat, int kNB>
__global__ void __launch_bounds__(kThreads, 1)
kv8_attn_kernel(const __grid_constant__ Kv8AttnParams p) {
    extern __shared__ __align__(128) unsigned char smem[];
    long long* cum = reinterpret_cast<long long*>(smem + kOffCum);
    unsigned long long* masks = reinterpret_cast<unsigned long long*>(smem + kOffMask);
    float* factors = reinterpret_cast<float*>(smem + kOffFactor);
    float2* ml = reinterpret_cast<float2*>(smem + kOffMl);
    int* exps = reinterpret_cast<int*>(smem + kOffExp);
    float* join = reinterpret_cast<float*>(smem + kOffJoin);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;

    grid_dependency_wait();
    grid_launch_dependents();
    scan_units(p, cum, reinterpret_cast<long long*>(smem + kOffMl));
    const long long total = cum[p.n_branches];
    const long long per_cta = max((long long)kMinUnits, (total + gridDim.x - 1) / gridDim.x);
    const long long begin = (long long)blockIdx.x * per_cta, end = min(total, begin + per_cta);
    if (begin >= end) return;

    // ---- the warp's own pages: begin + warp, + 8, ..; `next` runs kStages ahead of the work
    unsigned char* ring = smem + kOffRing + warp * kStages * kKv8Record;
    Place next = place_of(p, cum, min(begin + warp, end - 1));
    long long next_unit = begin + warp;
    int next_page = -1;                                             // of the pool, asked for one copy ahead
    auto look_up = [&]() {
        next_page = -1;
        if (next_unit < end && next.page * kPage < next.tokens) next_page = p.block_table[(size_t)next.b * p.max_blocks + next.page];
    };
    auto copy = [&](int stage) {                                    // the page that was looked up, and on to the one after it
        if (next_unit < end) {
            const bool there = next_page >= 0 && next_page < p.num_pages;
            if (!there && next.page * kPage < next.tokens && lane == 0) atomicMin(p.status, (int)TTS_ERR_DEVICE_BOUNDS);
            const unsigned char* src = p.pool + ((size_t)(there ? next_page : 0) * p.Hkv + next.item / p.n_rb) * kKv8Record + lane * 16;
            const uint32_t dst = smem_u32(ring + stage * kKv8Record) + lane * 16;
#pragma unroll
            for (int i = 0; i < kKv8Record / 512; ++i) copy16(dst + i * 512, src + i * 512, there);
            if (lane < (kKv8Record % 512) / 16) copy16(dst + kKv8Record / 512 * 512, src + kKv8Record / 512 * 512, there);
            next_unit += kWarps;
            if (next_unit < end) advance(p, next, kWarps);
            look_up();
        }
        copy_commit();
    };
    look_up();
#pragma unroll
    for (int i = 0; i < kStages; ++i) copy(i);
    int stage = 0;

    Place item = place_of(p, cum, begin);                           // the item that is worked on, at its first unit here
    long long unit = begin;
    for (int nth = 0; unit < end; ++nth) {
        const int h = item.item / p.n_rb, rb = item.item - h * p.n_rb, b = item.b;
        const int row0 = rb * p.rb_rows, rows = min(p.rb_rows, p.nr - row0);
        const long long item_begin = unit - item.page, item_end = item_begin + item.units, stop = min(end, item_end);
        const int tail = item.tokens - p.R;                         // the first of the branch's last R tokens (may be negative)

        // ---- Q: a warp takes rows warp, warp + 8, ..; scaled to fp16 by the power of two that puts the largest at 2^14
        for (int r = warp; r < kNB * 8; r += kWarps) {
            const int stacked = row0 + r, i = stacked / p.G, head = h * p.G + stacked - i * p.G;
            uint2 x = make_uint2(0, 0);
            if (r < rows) x = *reinterpret_cast<const uint2*>(p.q + ((size_t)b * p.R + i) * p.q_stride + (size_t)head * kHeadDim + lane * 4);
            float f[4] = {__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xffff0000u), __uint_as_float(x.y << 16), __uint_as_float(x.y & 0xffff0000u)};
            float top = 0.f;                                        // the largest finite magnitude
#pragma unroll
            for (int k = 0; k < 4; ++k) if (fabsf(f[k]) < INFINITY) top = fmaxf(top, fabsf(f[k]));
#pragma unroll
            for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            const int e = max(-100, min(126, ((__float_as_int(top) >> 23) & 255) - 127)) - 14;
            const float down = power_of_two(-e);
            uint2 y;
            y.x = pack_half2(f[0] * down, f[1] * down); y.y = pack_half2(f[2] * down, f[3] * down);
            // dims 4 lane ..: chunk (u, t) = ((lane / 2) mod 4, lane / 8), half lane mod 2
            *reinterpret_cast<uint2*>(smem + kOffQ + r * 256 + q_place((lane >> 1) & 3, lane >> 3, r) * 16 + (lane & 1) * 8) = y;
            if (lane == 0) {
                factors[r] = r < rows ? power_of_two(e) * p.scale_log2 : 0.f;
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

        float o[8][kNB][4], m[kNB][2], l[kNB][2], factor[kNB][2];
        int unit_exp = 7;                                           // exponent field of the power of two that p sv is held in units of
#pragma unroll
        for (int n = 0; n < kNB; ++n) {
#pragma unroll
            for (int j = 0; j < 2; ++j) { m[n][j] = kFar; l[n][j] = 0.f; factor[n][j] = factors[n * 8 + 2 * t + j]; }
#pragma unroll
            for (int d = 0; d < 8; ++d)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[d][n][j] = 0.f;
        }

        // ---- this warp's pages of the item
        const int skip = (int)((unit - begin) & (kWarps - 1));
        for (long long u = unit + ((warp - skip) & (kWarps - 1)); u < stop; u += kWarps) {
            const int first = (int)(u - item_begin) * kPage;        // the page's first token
            unsigned char* rec = ring + stage * kKv8Record;
            copy_wait<kStages - 1>();
            __syncwarp();
            const int left = item.tokens - first;                   // tokens here; the rest of the slots may hold anything
            float* scales = reinterpret_cast<float*>(rec + 2 * kKv8Codes);
            if (left < kPage) {
                if (left <= 0) goto done;                           // a branch of no tokens
                for (int r = left; r < kPage; ++r) {
                    if (lane < 8) *reinterpret_cast<uint4*>(rec + kKv8Codes + r * kHeadDim + lane * 16) = make_uint4(0, 0, 0, 0);
                    if (lane < 2) scales[lane * kPage + r] = 0.f;
                }
                __syncwarp();
            }
            {
                const int tok_a = 4 * (g >> 1) + (g & 1), tok_b = tok_a + 2;
                // S^T = K Q^T
                float s[kNB][4];
#pragma unroll
                for (int n = 0; n < kNB; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[n][j] = 0.f;
#pragma unroll
                for (int c = 0; c < 2; ++c) {                       // chunk 2 t + c of both tokens (both have chunk_place g)
                    const int place = ((2 * t + c) ^ g) * 16;
                    const uint4 xa = *reinterpret_cast<const uint4*>(rec + tok_a * kHeadDim + place), xb = *reinterpret_cast<const uint4*>(rec + tok_b * kHeadDim + place);
                    const uint32_t wa[4] = {xa.x, xa.y, xa.z, xa.w}, wb[4] = {xb.x, xb.y, xb.z, xb.w};
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
                            const uint4 q = *reinterpret_cast<const uint4*>(smem + kOffQ + (n * 8 + g) * 256 + q_place(2 * c + half, t, g) * 16);
                            mma(s[n], a[0][0], a[0][1], a[0][2], a[0][3], q.x, q.y);
                            mma(s[n], a[1][0], a[1][1], a[1][2], a[1][3], q.z, q.w);
                        }
                    }
                }
                // scores less the running maximum, in log2 units; j: (token a or b) * 2 + (row 2 t or 2 t + 1)
                const float ka = scales[tok_a], kb = scales[tok_b], va = scales[kPage + tok_a], vb = scales[kPage + tok_b];
#pragma unroll
                for (int n = 0; n < kNB; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[n][j] = s[n][j] * (j < 2 ? ka : kb) * factor[n][j & 1];
                if (first + kPage > tail) {
#pragma unroll
                    for (int n = 0; n < kNB; ++n)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int tok = j < 2 ? tok_a : tok_b, a = first + tok - tail;
                            const bool seen = tok < left && (a < 0 || (a < 64 && (masks[n * 8 + 2 * t + (j & 1)] >> a & 1)));
                            if (!seen) s[n][j] = -INFINITY;
                        }
                }
                float over = -INFINITY;
#pragma unroll
                for (int n = 0; n < kNB; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) over = fmaxf(over, s[n][j] - m[n][j & 1]);
                if (__any_sync(0xffffffffu, over > kSlack)) {
#pragma unroll
                    for (int n = 0; n < kNB; ++n)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            float top = fmaxf(s[n][j], s[n][2 + j]);
#pragma unroll
                            for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
                            top = fmaxf(top, m[n][j]);
                            const float back = exp2_approx(m[n][j] - top);
                            m[n][j] = top;
                            l[n][j] *= back;
#pragma unroll
                            for (int d = 0; d < 8; ++d) { o[d][n][j] *= back; o[d][n][2 + j] *= back; }
                        }
                }
                // the unit of p sv: the largest exponent in sv so far (a NaN or an infinity is not a unit)
                {
                    const int ea = __float_as_int(va) >> 23 & 255, eb = __float_as_int(vb) >> 23 & 255;
                    const int e = __reduce_max_sync(0xffffffffu, max(ea == 255 ? 0 : ea, eb == 255 ? 0 : eb));
                    if (e > unit_exp) {
                        const float back = unit_exp - e < -126 ? 0.f : power_of_two(unit_exp - e);
                        unit_exp = e;
#pragma unroll
                        for (int d = 0; d < 8; ++d)
#pragma unroll
                            for (int n = 0; n < kNB; ++n)
#pragma unroll
                                for (int j = 0; j < 4; ++j) o[d][n][j] *= back;
                    }
                }
                const float up = power_of_two(kRoom + 127 - unit_exp), fa = va * up, fb = vb * up;
                uint32_t pb[kNB][2];                                // P^T as the B operand: tokens 4 t, 4 t + 1 and 4 t + 2, 4 t + 3 of row g
#pragma unroll
                for (int n = 0; n < kNB; ++n) {
                    float w[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float e = exp2_approx(s[n][j] - m[n][j & 1]);
                        l[n][j & 1] += e;
                        w[j] = e * (j < 2 ? fa : fb);
                        if (e == 0.f) w[j] = 0.f;                   // a hidden token's scale may be a NaN
                    }
                    pb[n][0] = transpose8x8(pack_half2(w[0], w[1]));
                    pb[n][1] = transpose8x8(pack_half2(w[2], w[3]));
                }
                // O^T += V^T P^T: four bytes (tokens 4 t ..) of dims 2 d, 2 d + 1 of the lane's 16 make the A operand of tile d
                uint4 v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    v[j] = *reinterpret_cast<const uint4*>(rec + kKv8Codes + (4 * t + j) * kHeadDim + (g ^ ((j & 1) | 2 * t)) * 16);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t w[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = kv8_biased<kFormat>(q == 0 ? v[j].x : q == 1 ? v[j].y : q == 2 ? v[j].z : v[j].w);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t x = __byte_perm(w[0], w[1], half ? 0x7362 : 0x5140), y = __byte_perm(w[2], w[3], half ? 0x7362 : 0x5140);
                        const uint32_t a0 = kv8_decode2<kFormat>(x, 0), a1 = kv8_decode2<kFormat>(x, 1), a2 = kv8_decode2<kFormat>(y, 0), a3 = kv8_decode2<kFormat>(y, 1);
#pragma unroll
                        for (int n = 0; n < kNB; ++n) mma(o[2 * q + half][n], a0, a1, a2, a3, pb[n][0], pb[n][1]);
                    }
                }
            }
        done:
            __syncwarp();                                           // all lanes have read the page
            copy(stage);
            stage = stage + 1 == kStages ? 0 : stage + 1;
        }

        // ---- join the warps
#pragma unroll
        for (int n = 0; n < kNB; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) l[n][j] += __shfl_xor_sync(0xffffffffu, l[n][j], x);
                if (g == 0) ml[warp * kKv8MaxRows + n * 8 + 2 * t + j] = make_float2(m[n][j], l[n][j]);
            }
        if (lane == 0) exps[warp] = unit_exp;
        __syncthreads();
        int top_exp = exps[0];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) top_exp = max(top_exp, exps[w]);
        {
            const float unit_back = unit_exp - top_exp < -126 ? 0.f : power_of_two(unit_exp - top_exp);
#pragma unroll
            for (int n = 0; n < kNB; ++n)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float top = kFar, sum = 0.f;
#pragma unroll
                    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, ml[w * kKv8MaxRows + n * 8 + 2 * t + j].x);
#pragma unroll
                    for (int w = 0; w < kWarps; ++w) {
                        const float2 x = ml[w * kKv8MaxRows + n * 8 + 2 * t + j];
                        sum += x.y * exp2_approx(x.x - top);
                    }
                    // (a row that saw nothing has m = kFar and l = 0 everywhere: zeros)
                    const float back = sum == 0.f ? 0.f : exp2_approx(m[n][j] - top) * unit_back / sum;
#pragma unroll
                    for (int d = 0; d < 8; ++d) { o[d][n][j] *= back; o[d][n][2 + j] *= back; }
                    m[n][j] = top; l[n][j] = sum;
                }
        }
        const bool whole = unit == item_begin && stop == item_end;
        const float out_unit = power_of_two(min(127, max(-126, top_exp - 127 - kRoom)));
        const int slot = 2 * blockIdx.x + (nth == 0 ? 0 : 1);       // a CTA leaves parts of its first and of its last item only
        auto row_out = [&](int r, size_t& at) {                     // where row r of the block goes, in elements
            const int stacked = row0 + r, i = stacked / p.G, head = h * p.G + stacked - i * p.G;
            at = (((size_t)b * p.R + i) * p.Hq + head) * kHeadDim;
        };
        auto write_out = [&](int r, int dim, const float4& x) {
            size_t at;
            row_out(r, at);
            if (p.out_dtype == TTS_OUT_FP32) *reinterpret_cast<float4*>(static_cast<float*>(p.out) + at + dim) = x;
            else {
                const __nv_bfloat162 lo = __floats2bfloat162_rn(x.x, x.y), hi = __floats2bfloat162_rn(x.z, x.w);
                *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + at + dim) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
            }
        };
        auto write_lse = [&](int r, float top, float sum) {         // natural logarithm
            size_t at;
            row_out(r, at);
            p.lse[at / kHeadDim] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
        };
#pragma unroll
        for (int round = 0; round < 2; ++round) {                   // dims 16 g + 8 round .. + 7 of every g
#pragma unroll
            for (int n = 0; n < kNB; ++n)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float4* to = reinterpret_cast<float4*>(join + ((warp * kNB + n) * 8 + 2 * t + j) * 64 + g * 8);
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        to[k] = make_float4(o[4 * round + 2 * k][n][j], o[4 * round + 2 * k][n][2 + j], o[4 * round + 2 * k + 1][n][j], o[4 * round + 2 * k + 1][n][2 + j]);
                }
            __syncthreads();
            for (int i = threadIdx.x; i < rows * 16; i += kThreads) {
                const int r = i >> 4, c = i & 15;
                float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    const float4 x = *reinterpret_cast<const float4*>(join + (w * kNB * 8 + r) * 64 + c * 4);
                    sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
                }
                sum.x *= out_unit; sum.y *= out_unit; sum.z *= out_unit; sum.w *= out_unit;
                const int dim = (c >> 1) * 16 + round * 8 + (c & 1) * 4;
                if (whole) write_out(r, dim, sum);
                else *reinterpret_cast<float4*>(p.part_o + ((size_t)slot * kKv8MaxRows + r) * kHeadDim + dim) = sum;
            }
            __syncthreads();
        }
        if (warp == 0 && g == 0) {
#pragma unroll
            for (int n = 0; n < kNB; ++n)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int r = n * 8 + 2 * t + j;
                    if (r >= rows) continue;
                    if (!whole) p.part_ml[slot * kKv8MaxRows + r] = make_float2(m[n][j], l[n][j]);
                    else if (p.lse) write_lse(r, m[n][j], l[n][j]);
                }
        }
        if (!whole) {
            // ---- the last CTA to leave a part of the item joins them all
            __threadfence();
            __syncthreads();
            const int cta0 = (int)(item_begin / per_cta), parts = (int)((item_end - 1) / per_cta) - cta0 + 1;
            const size_t id = ((size_t)b * p.Hkv + h) * p.n_rb + rb;
            if (threadIdx.x == 0) {
                const bool last = atomicAdd(p.arrived + id, 1u) + 1 == (unsigned)parts;
                if (last) p.arrived[id] = 0;                        // as the next call expects it
                exps[kWarps] = last;
            }
            __syncthreads();
            if (exps[kWarps]) {
                __threadfence();
                // a part is the first item of its CTA unless it starts the item behind the CTA's first unit
                auto slot_of = [&](int k) { return 2 * (cta0 + k) + (k == 0 && item_begin != cta0 * per_cta ? 1 : 0); };
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
        }
        __syncthreads();                                            // Q, the masks and the sums are free again
        const int done_here = (int)(stop - unit);
        unit = stop;
        if (unit < end) advance(p, item, done_here);
    }
}

}  // namespace

cudaError_t launch_kv8_attn(const Kv8AttnParams& p, int format, cudaStream_t st) {
    auto launch = [&](auto fmt, auto nb) {
        constexpr int kFormat = decltype(fmt)::value, kNB = decltype(nb)::value;
        auto kernel = kv8_attn_kernel<kFormat, kNB>;
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes<kNB>());
        if (e != cudaSuccess) return e;
        return launch_dependent(kernel, p.grid, kThreads, smem_bytes<kNB>(), st, p);
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
