// Reading the 8-bit cache back: whole pages, as bf16 pages of another pool (values code * scale, one rounding).
//
// Bound by HBM: 4224 bytes in and 8192 out per page and KV head, each touched once.  A warp takes one of them: K and V
// are 128 chunks of 16 codes each, so a lane has eight loads of 16 bytes and the scales of its tokens in flight before it
// stores; a lane's 16 values are one 32-byte sector, written by one instruction where the pools start on such a boundary
// (4128 pages of 8 KV heads: 69.4 us, 0.90 of the copy peak; in 16-byte stores 80.8).  One prompt's 47 pages of 2 heads: 4.4 to 4.8 us, a launch.
#include "kv8.cuh"
#include "launch.cuh"

namespace tts {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float2 half2_floats(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }

template <int kFormat>
__global__ void __launch_bounds__(kThreads)
kv8_read_kernel(const __grid_constant__ Kv8ReadParams p) {
    grid_dependency_wait();
    grid_launch_dependents();
    const int lane = threadIdx.x & 31;
    const bool wide = ((reinterpret_cast<uintptr_t>(p.k_pages) | reinterpret_cast<uintptr_t>(p.v_pages)) & 31) == 0;
    const long total = (long)p.n * p.Hkv;
    for (long w = (blockIdx.x * (long)kThreads + threadIdx.x) >> 5; w < total; w += (long)gridDim.x * (kThreads / 32)) {
        const int i = (int)(w / p.Hkv), h = (int)(w - (long)i * p.Hkv);
        const int s = p.src[i], d = p.dst[i];
        if (s < 0 || d < 0) continue;
        if (s >= p.num_pages || d >= p.num_dst) { if (lane == 0) atomicMin(p.status, (int)TTS_ERR_DEVICE_BOUNDS); continue; }
        const unsigned char* rec = p.pool + ((size_t)s * p.Hkv + h) * kKv8Record;
        const float* scales = reinterpret_cast<const float*>(rec + 2 * kKv8Codes);
        uint4 x[8];
        float sc[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = __ldcs(reinterpret_cast<const uint4*>(rec) + 32 * k + lane);
#pragma unroll
        for (int k = 0; k < 8; ++k) sc[k] = scales[4 * k + (lane >> 3)];          // (token 4 (k mod 4) + lane / 8 of K, then of V)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int t = (4 * k + (lane >> 3)) & (kPage - 1), c = (lane & 7) ^ kv8_chunk_place(t);
            const uint32_t in[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
            uint32_t out[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t b = kv8_biased<kFormat>(in[j]);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const float2 f = half2_floats(kv8_decode2<kFormat>(b, half));
                    const __nv_bfloat162 y = __floats2bfloat162_rn(f.x * sc[k], f.y * sc[k]);
                    out[2 * j + half] = *reinterpret_cast<const uint32_t*>(&y);
                }
            }
            uint4* to = reinterpret_cast<uint4*>((k < 4 ? p.k_pages : p.v_pages) + (((size_t)d * p.Hkv + h) * kPage + t) * kHeadDim + 16 * c);
            if (wide) {
                asm volatile("st.global.cs.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(out[0]), "r"(out[1]), "r"(out[2]), "r"(out[3]), "r"(out[4]),
                             "r"(out[5]), "r"(out[6]), "r"(out[7]) : "memory");
            } else {
                __stcs(to, make_uint4(out[0], out[1], out[2], out[3]));
                __stcs(to + 1, make_uint4(out[4], out[5], out[6], out[7]));
            }
        }
    }
}

}  // namespace

cudaError_t launch_kv8_read(const Kv8ReadParams& p, int format, int n_sms, cudaStream_t st) {
    const long blocks = ((long)p.n * p.Hkv + kThreads / 32 - 1) / (kThreads / 32);
    const int grid = (int)(blocks < 32l * n_sms ? blocks : 32l * n_sms);
    if (format == TTS_KV8_E4M3) return launch_dependent(kv8_read_kernel<TTS_KV8_E4M3>, grid, kThreads, 0, st, p);
    return launch_dependent(kv8_read_kernel<TTS_KV8_INT8>, grid, kThreads, 0, st, p);
}

}  // namespace tts
