// What the C-ABI files share: checks of arguments and the end of a call.
#pragma once
#include <initializer_list>

#include "tts_internal.cuh"

namespace tts {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

inline int finish(Ctx* c, cudaError_t e, int launches) {
    if (e != cudaSuccess) { c->last_cuda_error = (int)e; return TTS_ERR_CUDA; }
    c->launches += launches;
    return TTS_OK;
}

constexpr int kMaxBlocks = 1 << 26;                    // 2^30 tokens per branch: token numbers and their sums fit 32 bits

inline bool branches_ok(const Ctx* c, const int32_t* block_table, int prefix_len, int n_branches) {
    const tts_config& f = c->cfg;
    return block_table && aligned4(block_table) && f.max_blocks_per_branch <= kMaxBlocks && n_branches >= 1 && n_branches <= f.max_branches && prefix_len >= 0 &&
           prefix_len % f.page_size == 0 && prefix_len / f.page_size <= f.max_blocks_per_branch;
}

// Both arrays as [p, p + bytes): do they share memory?
inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + nb && y < x + na;
}

struct Span { const void* at; size_t bytes; };
// Does `written` share memory with one of the others?
inline bool clash(const Span& written, std::initializer_list<Span> others) {
    for (const Span& o : others) if (overlap(written.at, written.bytes, o.at, o.bytes)) return true;
    return false;
}
inline size_t pool_bytes(const tts_config& f) { return (size_t)f.num_pages * f.n_kv_heads * kPage * kHeadDim * 2; }
inline size_t table_bytes(const tts_config& f, int n) { return (size_t)n * f.max_blocks_per_branch * 4; }

}  // namespace tts
