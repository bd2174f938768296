// The 8-bit cache: layout of its pages, codes and scales.
//
// A pool holds, for every page and KV head, one record of 4224 bytes, so that all that attention needs of 16
// tokens lies in one run:
//     [16 tokens][128]  K codes    [16][128]  V codes    [16]  K scales, fp32    [16]  V scales, fp32
// value = code * scale, one scale for each token's K and V vector.  The eight 16-byte chunks of a token's codes
// are exchanged: chunk c of token t lies at place c ^ chunk_place(t).  With that exchange both contractions read
// their operands from shared memory as they lie, 16 bytes a lane, without a bank conflict (kv8_attn.cu); a
// token's codes stay one 128-byte line, so writing single tokens stays cheap.
#pragma once
#include "tts_internal.cuh"

namespace tts {

constexpr int kKv8Codes = kPage * kHeadDim;                              // bytes of K codes, and of V codes
constexpr int kKv8Record = 2 * kKv8Codes + 2 * kPage * 4;
constexpr float kKv8LeastScale = 7.52316384526264e-37f;                  // 2^-120: its reciprocal and its products with codes are finite, normal numbers

static_assert(kKv8Record == TTS_KV8_RECORD && kKv8Record % 128 == 0, "records are whole 128-byte lines");

__host__ __device__ constexpr int kv8_chunk_place(int t) { return (t & 1) | ((t >> 2) << 1); }

template <int kFormat>
__device__ __forceinline__ float kv8_largest() { return kFormat == TTS_KV8_E4M3 ? 448.f : 127.f; }

// Two floats to two codes, rounded to nearest (ties to even), the first in the low byte.  |x| is at most a rounding above
// the largest code.
template <int kFormat>
__device__ __forceinline__ uint32_t kv8_encode2(float a, float b) {
    if constexpr (kFormat == TTS_KV8_E4M3) {
        uint16_t r;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
        return r;
    } else {
        return (uint32_t)(uint8_t)(int8_t)max(-127, min(127, __float2int_rn(a))) | (uint32_t)(uint8_t)(int8_t)max(-127, min(127, __float2int_rn(b))) << 8;
    }
}

// The two codes in the low / high half of a word, as two halves of the same order (exact: e4m3 and int8 are subsets of fp16).
// int8: 0x6400 | u is 1024 + u in fp16, so with u = code + 128 (`w` has its sign bits turned, see kv8_biased) one subtraction
// of 1152 is left.
template <int kFormat>
__device__ __forceinline__ uint32_t kv8_decode2(uint32_t w, int half) {
    uint32_t r;
    if constexpr (kFormat == TTS_KV8_E4M3) {
        if (half) asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, hi;\n\t}" : "=r"(r) : "r"(w));
        else asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t}" : "=r"(r) : "r"(w));
    } else {
        const uint32_t x = __byte_perm(w, 0x64646464u, half ? 0x4342 : 0x4140), bias = 0x64806480u;
        asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(bias));
    }
    return r;
}
template <int kFormat>
__device__ __forceinline__ uint32_t kv8_biased(uint32_t w) { return kFormat == TTS_KV8_E4M3 ? w : w ^ 0x80808080u; }

struct Kv8AttnParams {
    const __nv_bfloat16* q;
    long q_stride;                     // elements from row to row
    const unsigned char* pool;
    const int32_t *block_table, *branch_lens, *tree_parents;
    void* out;
    float* lse;
    float* part_o;                     // [2 * grid][rb_rows, or 128 rows][128] normalised partial results
    float2* part_ml;                   // [2 * grid][rb_rows, or 128] their maximum (log2 units) and sum
    unsigned* arrived;                 // [branch][KV head][row block] parts written so far; zero between calls
    int32_t* status;
    int Hq, Hkv, G, R, nr, n_rb, rb_rows, prefix_len, n_branches, max_blocks, num_pages, out_dtype, grid;
    float scale_log2;
};
// Rows of one KV head that a block of kv8_attn.cu works on at a time: what a warp holds in registers.  (300 rows took 509 us in
// blocks of 16 and 410 in blocks of 24.)
constexpr int kKv8MaxRows = 24;
// kv8_attn_wide.cu works on up to 128 rows at a time, and takes over where the other would need more than two blocks: 64 (branch, KV head)s
// of 7.9 k keys take 79 us there with 25 to 48 rows and 109 with 60, here 78 with 40 and 82 with 60.  (Over 500 keys it is slower, 21 us
// against 17, but the host does not know how long the branches are.)
constexpr int kKv8WideRows = 128, kKv8WideFrom = 2 * kKv8MaxRows + 1;
// Rows of partial results of a context for up to nr rows per KV head: two parts for each CTA, of the first kernel one CTA to an SM, of the other two.
inline size_t kv8_part_rows(int nr, int n_sms) {
    const size_t few = 2 * (size_t)n_sms * (nr < kKv8MaxRows ? nr : kKv8MaxRows);
    return nr < kKv8WideFrom ? few : 4 * (size_t)n_sms * kKv8WideRows;
}
struct Kv8ReadParams {
    const unsigned char* pool;
    const int32_t *src, *dst;
    __nv_bfloat16 *k_pages, *v_pages;
    int32_t* status;
    int n, Hkv, num_pages, num_dst;
};
cudaError_t launch_kv8_attn(const Kv8AttnParams& p, int format, cudaStream_t st);
cudaError_t launch_kv8_attn_wide(const Kv8AttnParams& p, int format, cudaStream_t st);
cudaError_t launch_kv8_read(const Kv8ReadParams& p, int format, int n_sms, cudaStream_t st);

}  // namespace tts
