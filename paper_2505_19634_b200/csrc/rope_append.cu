// Rotary positions on the way into the cache: the queries and keys of ragged chunks of new tokens are
// rotated, the keys and values go to their page slots, the rotated queries to a dense array.
//
//   pair i of a head vector x is turned by angle a = positions[axis[i]][row] * inv_freq[i]:
//       (x_lo, x_hi) -> (x_lo cos a - x_hi sin a, x_lo sin a + x_hi cos a)
//
// The angle is formed in 64 bits as a number of whole turns, of which only the fraction is kept: far
// positions (2^20 and more) lose their phase in 32 bits.  Sine and cosine of the fraction and the rotation
// itself are fp32, with one rounding to bf16 at the end.
//
// Bound by HBM: q, k and v are read once, q, K and V written once; there is no reuse between rows.  Eight
// lanes handle one head vector, each two 16-byte chunks that hold both members of its pairs, so a rotation
// needs no exchange between lanes; a lane's eight sines and cosines serve all heads of the row that its
// warp walks through, sixteen at a time, whose loads are issued before the row's branch, page and angles are
// looked up.
#include "launch.cuh"
#include "tts_internal.cuh"

namespace tts {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kBatch = 4;                              // head vectors that a group of eight lanes has in flight

// Row starts that decrease or leave the rows make a call of which nothing is computed: a row taken for a branch's that
// starts behind it would have its key written before the branch's first token, or before the pool.
__device__ __forceinline__ bool bad_rows(const RopeParams& p, int lo, int hi) { return lo < 0 || hi < lo || hi > p.total_rows; }

// The last branch whose rows start at or before `row`, or -1, among more than 32: the whole warp looks at 32
// starts per step (two steps for up to 1024 branches).
__device__ __forceinline__ int branch_of_row(const int32_t* row_start, int n, int row, int lane) {
    const int lo = (__popc(__ballot_sync(0xffffffffu, lane * 32 < n && row_start[lane * 32] <= row)) - 1) * 32;      // 32 blocks of 32 starts
    if (lo < 0) return -1;
    const int at = lo + lane;
    return lo + __popc(__ballot_sync(0xffffffffu, at < n && row_start[at] <= row)) - 1;
}

__device__ __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ uint4 pack(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// kMode 0: all 64 pairs, pair i = dims (i, i + 64); 1: neighbours (2i, 2i+1), any number of pairs; 2: pair i =
// dims (i, i + n_pairs) with fewer than 64 pairs (partners fetched one by one).
// A warp takes one row and every parts-th group of four head vectors of it; with few rows several warps share
// a row, so that small calls still fill the GPU.
template <int kMode>
__global__ void __launch_bounds__(kThreads)
append_rope_kernel(const __grid_constant__ RopeParams p) {
    __shared__ double turns[kHeadDim / 2];              // inv_freq / (2 pi)
    __shared__ int axis_of[kHeadDim / 2];
    for (int i = threadIdx.x; i < kHeadDim / 2; i += kThreads) {
        turns[i] = i < p.n_pairs ? p.turns[i] : 0.0;
        axis_of[i] = i < p.n_pairs ? p.axis[i] : 0;
    }
    __syncthreads();
    grid_dependency_wait();
    grid_launch_dependents();
    const int lane = threadIdx.x & 31, sub = lane & 7, group = lane >> 3;
    const int vectors = p.Hq + 2 * p.Hkv;
    // up to 32 branches are checked by each warp with the starts that it looks the row up in, more by the block
    const bool few = p.n_branches <= 32;
    if (!few) {
        bool bad = false;
        for (int i = threadIdx.x; i < p.n_branches; i += kThreads) bad |= bad_rows(p, p.row_start[i], p.row_start[i + 1]);
        if (__syncthreads_or(bad)) {
            if (threadIdx.x == 0) atomicMin(p.status, (int)TTS_ERR_DEVICE_BOUNDS);
            return;
        }
    }
    for (long w = blockIdx.x * (long)kWarps + (threadIdx.x >> 5); w < (long)p.total_rows * p.parts; w += (long)gridDim.x * kWarps) {
        const int row = (int)(w / p.parts), part = (int)(w - (long)row * p.parts);
        const int step = p.parts * 4;
        auto source = [&](int h) -> const __nv_bfloat16* {
            return h < p.Hq ? p.q + (size_t)row * p.q_stride + (size_t)h * kHeadDim
                 : h < p.Hq + p.Hkv ? p.k + (size_t)row * p.kv_stride + (size_t)(h - p.Hq) * kHeadDim
                                    : p.v + (size_t)row * p.kv_stride + (size_t)(h - p.Hq - p.Hkv) * kHeadDim;
        };
        uint4 lo4[kBatch], hi4[kBatch];
        auto load = [&](int h0) {                       // kBatch head vectors per group of eight lanes, before anything else is waited for
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const int h = h0 + i * step + group;
                lo4[i] = hi4[i] = make_uint4(0, 0, 0, 0);
                if (h < vectors) {
                    const uint4* src = reinterpret_cast<const uint4*>(source(h));
                    lo4[i] = src[sub]; hi4[i] = src[sub + 8];
                }
            }
        };
        if (kMode != 2) load(part * 4);
        // where the row's key and value go
        int b, start, end;
        if (few) {
            const int lo = lane < p.n_branches ? p.row_start[lane] : p.total_rows, hi = lane < p.n_branches ? p.row_start[lane + 1] : p.total_rows;
            if (__any_sync(0xffffffffu, bad_rows(p, lo, hi))) {
                if (lane == 0) atomicMin(p.status, (int)TTS_ERR_DEVICE_BOUNDS);
                return;
            }
            b = __popc(__ballot_sync(0xffffffffu, lo <= row)) - 1;
            start = __shfl_sync(0xffffffffu, lo, b); end = __shfl_sync(0xffffffffu, hi, b);
        } else {
            b = branch_of_row(p.row_start, p.n_branches, row, lane);
            start = b < 0 ? 0 : p.row_start[b]; end = b < 0 ? 0 : p.row_start[b + 1];
        }
        if (b < 0 || row >= end) continue;              // a row of no branch: left as it is
        const int c = end - start, L = p.branch_lens[b];
        const long tok = (long)p.prefix_len + L - c + (row - start);
        int page = -1;
        if (L >= c && tok < (long)p.max_blocks * kPage) page = p.block_table[(size_t)b * p.max_blocks + tok / kPage];
        const bool store_kv = page >= 0 && page < p.num_pages;
        if (!store_kv && lane == 0) atomicMin(p.status, (int)TTS_ERR_DEVICE_BOUNDS);

        auto angle = [&](int pair, float& s, float& co) {
            double t = (double)p.positions[(size_t)axis_of[pair] * p.total_rows + row] * turns[pair];
            t -= rint(t);
            sincospif(2.f * (float)t, &s, &co);
        };
        // mode 0 and 2: chunk sub holds the low members of pairs 8 sub .. 8 sub + 7 (mode 2: where there are
        // such pairs); mode 1: chunk sub holds pairs 4 sub .. + 3 and chunk sub + 8 pairs 32 + 4 sub .. + 3.
        // The four groups of lanes need the same eight sines and cosines per `sub`: each works out two.
        float cs[8], sn[8];
        {
            float s2[2], c2[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int k = 2 * group + i;
                angle(kMode == 1 ? (k < 4 ? 4 * sub + k : 32 + 4 * sub + k - 4) : 8 * sub + k, s2[i], c2[i]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sn[i] = __shfl_sync(0xffffffffu, s2[i & 1], (i >> 1) * 8 + sub);
                cs[i] = __shfl_sync(0xffffffffu, c2[i & 1], (i >> 1) * 8 + sub);
            }
        }
        auto store = [&](int h, const uint4& lo, const uint4& hi) {
            const bool is_q = h < p.Hq, is_v = h >= p.Hq + p.Hkv;
            if (h >= vectors || (!is_q && !store_kv)) return;
            uint4* dst = is_q ? reinterpret_cast<uint4*>(p.q_out + ((size_t)row * p.Hq + h) * kHeadDim)
                              : reinterpret_cast<uint4*>((is_v ? p.v_pages : p.k_pages) +
                                                         ((((size_t)page * p.Hkv + h - p.Hq - (is_v ? p.Hkv : 0)) * kPage + (size_t)(tok % kPage)) * kHeadDim));
            dst[sub] = lo; dst[sub + 8] = hi;
        };
        if (kMode == 2) {
            for (int h0 = part * 4; h0 < vectors; h0 += step) {
                const int h = h0 + group;
                const bool live = h < vectors;
                const __nv_bfloat16* src = source(live ? h : 0);
                uint4 a4 = reinterpret_cast<const uint4*>(src)[sub], z4 = reinterpret_cast<const uint4*>(src)[sub + 8];
                if (live && h < p.Hq + p.Hkv) {
                    // this lane writes the same two chunks; each dim's partner is n_pairs away
                    float lo[8], hi[8];
                    unpack(a4, lo); unpack(z4, hi);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        float(&x)[8] = half ? hi : lo;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int dim = 8 * (sub + 8 * half) + i;
                            if (dim >= 2 * p.n_pairs) continue;
                            const bool low = dim < p.n_pairs;
                            const int pair = low ? dim : dim - p.n_pairs;
                            const float other = __bfloat162float(src[low ? dim + p.n_pairs : pair]);
                            float s = sn[i], co = cs[i];
                            if (pair != 8 * sub + i) angle(pair, s, co);        // not one of this lane's own angles
                            x[i] = low ? x[i] * co - other * s : other * s + x[i] * co;
                        }
                    }
                    a4 = pack(lo); z4 = pack(hi);
                }
                __syncwarp();                           // the partners have been read before anything is written in place
                store(h, a4, z4);
            }
            continue;
        }
        for (int h0 = part * 4; h0 < vectors; h0 += kBatch * step) {
            if (h0 > part * 4) load(h0);
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const int h = h0 + i * step + group;
                if (h < p.Hq + p.Hkv) {
                    float lo[8], hi[8];
                    unpack(lo4[i], lo); unpack(hi4[i], hi);
                    if (kMode == 0) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const float a = lo[k], z = hi[k];
                            lo[k] = a * cs[k] - z * sn[k];
                            hi[k] = a * sn[k] + z * cs[k];
                        }
                    } else {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const float a = lo[2 * k], z = lo[2 * k + 1], d = hi[2 * k], e = hi[2 * k + 1];
                            if (4 * sub + k < p.n_pairs) {
                                lo[2 * k] = a * cs[k] - z * sn[k];
                                lo[2 * k + 1] = a * sn[k] + z * cs[k];
                            }
                            if (32 + 4 * sub + k < p.n_pairs) {
                                hi[2 * k] = d * cs[4 + k] - e * sn[4 + k];
                                hi[2 * k + 1] = d * sn[4 + k] + e * cs[4 + k];
                            }
                        }
                    }
                    lo4[i] = pack(lo); hi4[i] = pack(hi);
                }
                store(h, lo4[i], hi4[i]);
            }
        }
    }
}

}  // namespace

cudaError_t launch_append_rope(RopeParams p, int n_sms, cudaStream_t st) {
    // rows x parts warps; parts grows until the GPU's 64 warps per SM have work or a warp has one group of heads
    const int groups = ceil_div(p.Hq + 2 * p.Hkv, 4);
    p.parts = 1;
    while (p.parts < groups && (long)p.total_rows * p.parts * 2 <= 64l * n_sms) p.parts *= 2;
    if (p.parts > groups) p.parts = groups;
    const long warps = (long)p.total_rows * p.parts;
    const long blocks = (warps + kWarps - 1) / kWarps;
    const int grid = (int)(blocks < 16l * n_sms ? blocks : 16l * n_sms);
    if (p.interleaved) return launch_dependent(append_rope_kernel<1>, grid, kThreads, 0, st, p);
    if (p.n_pairs == kHeadDim / 2) return launch_dependent(append_rope_kernel<0>, grid, kThreads, 0, st, p);
    return launch_dependent(append_rope_kernel<2>, grid, kThreads, 0, st, p);
}

}  // namespace tts
