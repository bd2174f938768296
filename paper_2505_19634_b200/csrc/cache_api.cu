// C-ABI layer of the cache operators: argument checks, workspace, launches.  See include/tts.h.
#include <math.h>
#include <string.h>

#include <algorithm>
#include <functional>
#include <initializer_list>

#include "api_checks.cuh"
#include "chunk_attn.cuh"
#include "kv8.cuh"
#include "launch.cuh"
#include "tts_internal.cuh"

using namespace tts;

namespace {

// What the page calls copy: pools that overlap without being the same one, or that share memory with one of the arrays,
// would be read after they are written.
bool pools_clash(const tts_config& f, const PagePools& pools, std::initializer_list<Span> arrays) {
    const int n = pools.n_pools, half = n / 2;
    const size_t bytes = (size_t)f.num_pages * f.n_kv_heads * pools.tile_bytes;
    const std::less<const void*> before;
    const void* kv[2 * kMaxLayers], *at[2 * kMaxLayers];
    for (int i = 0; i < half; ++i) { kv[i] = pools.p[2 * i]; kv[half + i] = pools.p[2 * i + 1]; }
    if (n > 2 * half) kv[n - 1] = pools.p[n - 1];
    // (a program that allocates its layers in order has two runs in order: 128 pools take 0.3 us to merge, 2 to sort)
    if (!std::is_sorted(kv, kv + half, before)) std::sort(kv, kv + half, before);
    if (!std::is_sorted(kv + half, kv + n, before)) std::sort(kv + half, kv + n, before);
    std::merge(kv, kv + half, kv + half, kv + n, at, before);
    for (int i = 1; i < n; ++i)
        if (at[i] != at[i - 1] && overlap(at[i - 1], bytes, at[i], bytes)) return true;
    for (const Span& a : arrays) {
        const int i = (int)(std::upper_bound(at, at + n, a.at, before) - at);        // the first pool behind the array's start
        if ((i > 0 && overlap(at[i - 1], bytes, a.at, a.bytes)) || (i < n && overlap(at[i], bytes, a.at, a.bytes))) return true;
    }
    return false;
}

bool pools_from(int n_layers, void* const* k_pools, void* const* v_pools, PagePools* out) {
    if (n_layers < 1 || n_layers > kMaxLayers || !k_pools || !v_pools) return false;
    memset(out, 0, sizeof *out);
    out->n_pools = 2 * n_layers; out->tile_bytes = kPage * kHeadDim * 2;
    for (int i = 0; i < n_layers; ++i) {
        if (!k_pools[i] || !v_pools[i] || !aligned16(k_pools[i]) || !aligned16(v_pools[i])) return false;
        out->p[2 * i] = k_pools[i]; out->p[2 * i + 1] = v_pools[i];
    }
    return true;
}

bool pools_from_kv8(int n_layers, void* const* pools, PagePools* out) {
    if (n_layers < 1 || n_layers > kMaxLayers || !pools) return false;
    memset(out, 0, sizeof *out);
    out->n_pools = n_layers; out->tile_bytes = kKv8Record;
    for (int i = 0; i < n_layers; ++i) {
        if (!pools[i] || !aligned16(pools[i])) return false;
        out->p[i] = pools[i];
    }
    return true;
}

size_t align16(size_t n) { return (n + 15) & ~(size_t)15; }

PageWork page_work(const Ctx* c) {
    const size_t nb = c->cfg.max_branches, np = c->cfg.num_pages;
    char* p = reinterpret_cast<char*>(c->page_work);
    PageWork w;
    w.head = reinterpret_cast<int32_t*>(p); p += 16;
    w.child = reinterpret_cast<int4*>(p); p += nb * sizeof(int4);
    w.childless = reinterpret_cast<int32_t*>(p); p += align16(nb * 4);
    w.list_src = reinterpret_cast<int32_t*>(p); p += align16(np * 4);
    w.list_dst = reinterpret_cast<int32_t*>(p);
    return w;
}

// The page calls over whatever pools there are.
int copy_pages(Ctx* c, const PagePools& pools, const int32_t* src_pages, const int32_t* dst_pages, int n_copies) {
    if (!src_pages || !dst_pages || n_copies < 0 || !aligned4(src_pages) || !aligned4(dst_pages)) return TTS_ERR_INVALID;
    if (n_copies == 0) return TTS_OK;
    if (pools_clash(c->cfg, pools, {{src_pages, (size_t)n_copies * 4}, {dst_pages, (size_t)n_copies * 4}})) return TTS_ERR_INVALID;
    const OnDevice on(c->device);
    if (on.error() != cudaSuccess) return finish(c, on.error(), 0);
    return finish(c, launch_copy_pages(pools, src_pages, dst_pages, n_copies, c->cfg.n_kv_heads, c->cfg.num_pages, c->n_sms, c->d_status, c->stream), 1);
}

int fork_pages(Ctx* c, const PagePools& pools, const int32_t* block_table, int prefix_len, const int32_t* branch_lens, int n_branches,
               const int32_t* parents, int n_children, const int32_t* page_refs, int32_t* new_table, int32_t* new_lens, int32_t* new_refs) {
    if (!branch_lens || !parents || !page_refs || !new_table || !new_lens || !new_refs) return TTS_ERR_INVALID;
    if (!branches_ok(c, block_table, prefix_len, n_branches) || n_children < 1 || n_children > c->cfg.max_branches) return TTS_ERR_INVALID;
    if (!aligned4(branch_lens) || !aligned4(parents) || !aligned16(page_refs) || !aligned4(new_table) || !aligned4(new_lens) || !aligned16(new_refs))
        return TTS_ERR_INVALID;
    const tts_config& f = c->cfg;
    // children are written while their parents' rows are read
    const Span table{block_table, table_bytes(f, n_branches)}, lens{branch_lens, (size_t)n_branches * 4}, who{parents, (size_t)n_children * 4},
        refs{page_refs, (size_t)f.num_pages * 4}, out_table{new_table, table_bytes(f, n_children)}, out_lens{new_lens, (size_t)n_children * 4},
        out_refs{new_refs, refs.bytes};
    if (clash(out_table, {table, lens, who, refs, out_lens, out_refs}) || clash(out_lens, {table, lens, who, refs, out_refs}) ||
        clash(out_refs, {table, lens, who}) || (page_refs != new_refs && clash(out_refs, {refs})) ||
        pools_clash(f, pools, {table, lens, who, refs, out_table, out_lens, out_refs}))
        return TTS_ERR_INVALID;
    c->plan_explicit = 0;
    const OnDevice on(c->device);
    if (on.error() != cudaSuccess) return finish(c, on.error(), 0);
    return finish(c, launch_fork(pools, block_table, f.max_blocks_per_branch, prefix_len, branch_lens, n_branches, parents, n_children, page_refs,
                                 new_table, new_lens, new_refs, f.n_kv_heads, f.num_pages, c->n_sms, page_work(c), c->d_status, c->stream), 2);
}

int compact_pages(Ctx* c, const PagePools& pools, const int32_t* block_table, int n_branches, const int32_t* page_refs, int32_t* new_table,
                  int32_t* new_refs, int32_t* page_map, int32_t* n_used) {
    if (!page_refs || !new_table || !new_refs || !page_map || !n_used || !branches_ok(c, block_table, 0, n_branches)) return TTS_ERR_INVALID;
    if (!aligned16(page_refs) || !aligned4(new_table) || !aligned16(new_refs) || !aligned16(page_map) || !aligned4(n_used)) return TTS_ERR_INVALID;
    const tts_config& f = c->cfg;
    const Span table{block_table, table_bytes(f, n_branches)}, refs{page_refs, (size_t)f.num_pages * 4}, out_table{new_table, table.bytes},
        out_refs{new_refs, refs.bytes}, map{page_map, refs.bytes}, used{n_used, 4};
    if ((block_table != new_table && clash(out_table, {table})) || (page_refs != new_refs && clash(out_refs, {refs})) ||
        clash(out_table, {refs, out_refs}) || clash(out_refs, {table}) || clash(map, {table, refs, out_table, out_refs, used}) ||
        clash(used, {table, refs, out_table, out_refs}) || pools_clash(f, pools, {table, refs, out_table, out_refs, map, used}))
        return TTS_ERR_INVALID;
    c->plan_explicit = 0;
    const OnDevice on(c->device);
    if (on.error() != cudaSuccess) return finish(c, on.error(), 0);
    return finish(c, launch_compact(pools, block_table, f.max_blocks_per_branch, n_branches, page_refs, new_table, new_refs, page_map, n_used,
                                    f.n_kv_heads, f.num_pages, c->n_sms, page_work(c), c->d_status, c->stream), 2);
}

}  // namespace

namespace tts {

cudaError_t cache_alloc(Ctx* c) {
    const tts_config& f = c->cfg;
    const size_t nb = f.max_branches, np = f.num_pages, lists = align16(16 + nb * sizeof(int4) + align16(nb * 4) + 2 * align16(np * 4));
    // behind the page calls' lists, attention over the 8-bit cache: a counter for each (branch, KV head, row block)
    const int nr = f.max_rows_per_branch * (f.n_q_heads / f.n_kv_heads);
    c->kv8_arrived_bytes = nb * f.n_kv_heads * ceil_div(nr, kKv8MaxRows) * sizeof(unsigned);
    cudaError_t e = cudaMalloc(&c->page_work, lists + c->kv8_arrived_bytes);
    if (e != cudaSuccess) return e;
    c->kv8_arrived = reinterpret_cast<unsigned*>(reinterpret_cast<char*>(c->page_work) + lists);
    // zero before work on any stream, by one that waits for no other than the legacy stream's
    e = cudaMemsetAsync(c->kv8_arrived, 0, c->kv8_arrived_bytes, cudaStreamPerThread);
    if (e == cudaSuccess) e = cudaMemsetAsync(c->d_status, 0, 2 * sizeof(int32_t), cudaStreamPerThread);
    return e == cudaSuccess ? cudaStreamSynchronize(cudaStreamPerThread) : e;
}

cudaError_t cache_reset(Ctx* c) {
    cudaError_t e = cudaMemsetAsync(c->kv8_arrived, 0, c->kv8_arrived_bytes, c->stream);
    if (c->chunk_rows > 0) {
        if (e == cudaSuccess) e = cudaMemsetAsync(c->chunk_arrived, 0, c->chunk_arrived_bytes, c->stream);
        if (e == cudaSuccess) e = cudaMemsetAsync(c->chunk_head, 0, sizeof(ChunkHead), c->stream);
    }
    return e == cudaSuccess ? cudaStreamSynchronize(c->stream) : e;      // before work on another stream
}

cudaError_t cache_disturb(Ctx* c) {
    cudaError_t e = cudaMemsetAsync(c->kv8_arrived, 1, c->kv8_arrived_bytes, c->stream);
    if (e != cudaSuccess || c->chunk_rows == 0) return e;
    e = cudaMemsetAsync(c->chunk_arrived, 1, c->chunk_arrived_bytes, c->stream);
    return e == cudaSuccess ? cudaMemsetAsync(c->chunk_head, 1, sizeof(ChunkHead), c->stream) : e;
}

void cache_release(Ctx* c) {
    cudaFree(c->page_work);
    cudaFree(c->beam_work);
    c->kv8_arrived = nullptr; c->beam_work = nullptr; c->beam_rows = 0;
    cudaFree(c->chunk_head); cudaFree(c->chunk_pieces); cudaFree(c->chunk_arrived);
    cudaFree(c->chunk_part_o); cudaFree(c->chunk_part_ml);
    c->page_work = nullptr; c->chunk_head = nullptr; c->chunk_pieces = nullptr; c->chunk_arrived = nullptr;
    c->chunk_part_o = nullptr; c->chunk_part_ml = nullptr; c->chunk_rows = 0;
}

}  // namespace tts

extern "C" {

int tts_chunk_reserve(tts_ctx* ctx, int max_rows) {
    Ctx* c = reinterpret_cast<Ctx*>(ctx);
    if (!c || max_rows < 1 || max_rows > (1 << 24)) return TTS_ERR_INVALID;
    const tts_config& f = c->cfg;
    const int G = f.n_q_heads / f.n_kv_heads;
    if (G > 128) return TTS_ERR_UNSUPPORTED;
    if (c->chunk_rows > 0) return max_rows <= c->chunk_rows ? TTS_OK : TTS_ERR_INVALID;
    const OnDevice on(c->device);
    if (on.error() != cudaSuccess) return finish(c, on.error(), 0);
    const long entries = (long)max_rows / (2 * (128 / G)) + f.max_branches, pieces = entries + 2048;
    const long part_rows = (long)c->n_sms * kChunkPartsPerSm * 256;
    if (entries * f.n_kv_heads * 2 >= (1l << 31) || pieces * f.n_kv_heads >= (1l << 31)) return TTS_ERR_UNSUPPORTED;
    cudaError_t e = cudaMalloc(&c->chunk_head, sizeof(ChunkHead));
    if (e == cudaSuccess) e = cudaMalloc(&c->chunk_pieces, (size_t)pieces * sizeof(ChunkPiece));
    const size_t arrived = (size_t)entries * f.n_kv_heads * 2 * sizeof(unsigned);
    if (e == cudaSuccess) e = cudaMalloc(&c->chunk_arrived, arrived);
    if (e == cudaSuccess) e = cudaMemset(c->chunk_arrived, 0, arrived);
    if (e == cudaSuccess) e = cudaMemset(c->chunk_head, 0, sizeof(ChunkHead));
    if (e == cudaSuccess) e = cudaStreamSynchronize(cudaStreamLegacy);       // before work on a stream that does not wait for it
    if (e == cudaSuccess) e = cudaMalloc(&c->chunk_part_o, (size_t)part_rows * kHeadDim * sizeof(float));
    if (e == cudaSuccess) e = cudaMalloc(&c->chunk_part_ml, (size_t)part_rows * sizeof(float2));
    if (e != cudaSuccess) {
        cudaFree(c->chunk_head); cudaFree(c->chunk_pieces); cudaFree(c->chunk_arrived); cudaFree(c->chunk_part_o);
        c->chunk_head = nullptr; c->chunk_pieces = nullptr; c->chunk_arrived = nullptr; c->chunk_part_o = nullptr;
        return finish(c, e, 0);
    }
    c->chunk_rows = max_rows; c->chunk_arrived_bytes = arrived; c->chunk_max_pieces = (int)pieces; c->chunk_part_rows = part_rows;
    return TTS_OK;
}

int tts_chunk_attn(tts_ctx* ctx, const void* q, int64_t q_row_stride, const void* k_pages, const void* v_pages, const int32_t* block_table,
                   int prefix_len, const int32_t* branch_lens, const int32_t* row_start, int n_branches, int total_rows, void* out, float* lse) {
    Ctx* c = reinterpret_cast<Ctx*>(ctx);
    if (!c || !q || !k_pages || !v_pages || !branch_lens || !row_start || !out) return TTS_ERR_INVALID;
    if (!branches_ok(c, block_table, prefix_len, n_branches)) return TTS_ERR_INVALID;
    const tts_config& f = c->cfg;
    if (f.n_q_heads / f.n_kv_heads > 128) return TTS_ERR_UNSUPPORTED;
    if (total_rows < 0 || total_rows > c->chunk_rows) return TTS_ERR_INVALID;
    if (!aligned16(q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(out) || !aligned4(lse) || !aligned4(branch_lens) || !aligned4(row_start))
        return TTS_ERR_INVALID;
    if (q_row_stride < (int64_t)f.n_q_heads * kHeadDim || q_row_stride % 8 != 0 || q_row_stride >= (1ll << 38)) return TTS_ERR_INVALID;
    if (total_rows == 0) return TTS_OK;
    const size_t q_bytes = ((size_t)(total_rows - 1) * q_row_stride + (size_t)f.n_q_heads * kHeadDim) * 2;
    const size_t out_bytes = (size_t)total_rows * f.n_q_heads * kHeadDim * (f.out_dtype == TTS_OUT_FP32 ? 4 : 2);
    const size_t lse_bytes = lse ? (size_t)total_rows * f.n_q_heads * 4 : 0;
    const Span queries{q, q_bytes}, keys{k_pages, pool_bytes(f)}, values{v_pages, keys.bytes}, table{block_table, table_bytes(f, n_branches)},
        lens{branch_lens, (size_t)n_branches * 4}, starts{row_start, (size_t)(n_branches + 1) * 4}, result{out, out_bytes}, logs{lse, lse_bytes};
    if (clash(result, {queries, keys, values, table, lens, starts}) || (lse && clash(logs, {result, queries, keys, values, table, lens, starts})))
        return TTS_ERR_INVALID;
    const OnDevice on(c->device);
    if (on.error() != cudaSuccess) return finish(c, on.error(), 0);
    ChunkParams p;
    memset(&p, 0, sizeof p);
    p.block_table = block_table; p.branch_lens = branch_lens; p.row_start = row_start;
    p.out = out; p.lse = lse;
    // the entries of a call: at most one per branch and one per 2 T rows, and not more than rows
    const long entries = (long)total_rows / (2 * (128 / (f.n_q_heads / f.n_kv_heads))) + n_branches;
    const bool small = n_branches <= kChunkSmall && (entries <= kChunkSmall || total_rows <= kChunkSmall);
    p.small = small;
    p.head = c->chunk_head; p.pieces = c->chunk_pieces; p.arrived = c->chunk_arrived;
    p.part_o = c->chunk_part_o; p.part_ml = c->chunk_part_ml;
    p.status = c->d_status;
    p.Hq = f.n_q_heads; p.Hkv = f.n_kv_heads; p.G = p.Hq / p.Hkv; p.T = 128 / p.G;
    p.prefix_len = prefix_len; p.n_branches = n_branches; p.total_rows = total_rows; p.max_blocks = f.max_blocks_per_branch; p.num_pages = f.num_pages;
    p.max_pieces = c->chunk_max_pieces; p.part_rows = c->chunk_part_rows;
    p.grid = f.max_ctas > 0 && f.max_ctas < c->n_sms ? f.max_ctas : c->n_sms;
    p.g_inv = 65536u / (unsigned)p.G + 1u;
    p.heads_per_cta = (float)p.Hkv / p.grid; p.ctas_per_head = (float)p.grid / p.Hkv;
    p.out_dtype = f.out_dtype; p.out_32 = (reinterpret_cast<uintptr_t>(out) & 31u) == 0;
    p.scale_log2 = (f.softmax_scale > 0.f ? f.softmax_scale : 1.0f / sqrtf((float)f.head_dim)) * 1.4426950408889634f;
    cudaError_t e;
    if (!small) {
        e = launch_chunk_plan(p, c->stream);
        if (e != cudaSuccess) return finish(c, e, 0);
        c->launches += 1;
    }
    e = launch_chunk_attn(p, q, (long)q_row_stride, k_pages, v_pages, c->stream);
    return finish(c, e, 1);
}

int tts_kv_append_rope(tts_ctx* ctx, const tts_rope* rope, const void* q, int64_t q_row_stride, const void* k, const void* v, int64_t kv_row_stride,
                       const int32_t* positions, void* k_pages, void* v_pages, const int32_t* block_table, int prefix_len,
                       const int32_t* branch_lens, const int32_t* row_start, int n_branches, int total_rows, void* q_out) {
    Ctx* c = reinterpret_cast<Ctx*>(ctx);
    if (!c || !rope || !q || !k || !v || !positions || !k_pages || !v_pages || !branch_lens || !row_start || !q_out) return TTS_ERR_INVALID;
    if (!branches_ok(c, block_table, prefix_len, n_branches)) return TTS_ERR_INVALID;
    const tts_config& f = c->cfg;
    if (rope->n_pairs < 1 || rope->n_pairs > kHeadDim / 2 || rope->n_axes < 1 || rope->n_axes > 8) return TTS_ERR_INVALID;
    for (int i = 0; i < rope->n_pairs; ++i)
        if (rope->axis[i] >= rope->n_axes || !isfinite(rope->inv_freq[i])) return TTS_ERR_INVALID;
    if (total_rows < 0) return TTS_ERR_INVALID;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(q_out)) return TTS_ERR_INVALID;
    if (!aligned4(positions) || !aligned4(branch_lens) || !aligned4(row_start)) return TTS_ERR_INVALID;
    const int64_t q_row = (int64_t)f.n_q_heads * kHeadDim, kv_row = (int64_t)f.n_kv_heads * kHeadDim;
    if (q_row_stride < q_row || q_row_stride % 8 != 0 || kv_row_stride < kv_row || kv_row_stride % 8 != 0) return TTS_ERR_INVALID;
    if (total_rows == 0) return TTS_OK;
    // q_out may be q itself, when q is dense; any other overlap would be read after it is written
    const size_t kv_bytes = ((size_t)(total_rows - 1) * kv_row_stride + kv_row) * 2;
    const Span queries{q, ((size_t)(total_rows - 1) * q_row_stride + q_row) * 2}, new_k{k, kv_bytes}, new_v{v, kv_bytes},
        at{positions, (size_t)rope->n_axes * total_rows * 4}, turned{q_out, (size_t)total_rows * q_row * 2}, keys{k_pages, pool_bytes(f)},
        values{v_pages, keys.bytes}, table{block_table, table_bytes(f, n_branches)}, lens{branch_lens, (size_t)n_branches * 4},
        starts{row_start, (size_t)(n_branches + 1) * 4};
    if (clash(turned, {queries}) && !(q == q_out && q_row_stride == q_row)) return TTS_ERR_INVALID;
    if (clash(turned, {new_k, new_v, at, keys, values, table, lens, starts}) || clash(keys, {queries, new_k, new_v, at, values, table, lens, starts}) ||
        clash(values, {queries, new_k, new_v, at, table, lens, starts}))
        return TTS_ERR_INVALID;
    const OnDevice on(c->device);
    if (on.error() != cudaSuccess) return finish(c, on.error(), 0);
    RopeParams p;
    memset(&p, 0, sizeof p);
    p.q = static_cast<const __nv_bfloat16*>(q); p.k = static_cast<const __nv_bfloat16*>(k); p.v = static_cast<const __nv_bfloat16*>(v);
    p.q_stride = (long)q_row_stride; p.kv_stride = (long)kv_row_stride; p.positions = positions;
    p.q_out = static_cast<__nv_bfloat16*>(q_out); p.k_pages = static_cast<__nv_bfloat16*>(k_pages); p.v_pages = static_cast<__nv_bfloat16*>(v_pages);
    p.block_table = block_table; p.branch_lens = branch_lens; p.row_start = row_start; p.status = c->d_status;
    p.Hq = f.n_q_heads; p.Hkv = f.n_kv_heads; p.n_pairs = rope->n_pairs; p.interleaved = rope->interleaved != 0;
    p.prefix_len = prefix_len; p.n_branches = n_branches; p.total_rows = total_rows; p.max_blocks = f.max_blocks_per_branch; p.num_pages = f.num_pages;
    for (int i = 0; i < rope->n_pairs; ++i) { p.axis[i] = rope->axis[i]; p.turns[i] = rope->inv_freq[i] / 6.283185307179586476925; }
    return finish(c, launch_append_rope(p, c->n_sms, c->stream), 1);
}

int tts_kv_copy_pages(tts_ctx* ctx, int n_layers, void* const* k_pools, void* const* v_pools, const int32_t* src_pages, const int32_t* dst_pages,
                      int n_copies) {
    PagePools pools;
    if (!ctx || !pools_from(n_layers, k_pools, v_pools, &pools)) return TTS_ERR_INVALID;
    return copy_pages(reinterpret_cast<Ctx*>(ctx), pools, src_pages, dst_pages, n_copies);
}

int tts_kv_fork(tts_ctx* ctx, int n_layers, void* const* k_pools, void* const* v_pools, const int32_t* block_table, int prefix_len,
                const int32_t* branch_lens, int n_branches, const int32_t* parents, int n_children, const int32_t* page_refs,
                int32_t* new_table, int32_t* new_lens, int32_t* new_refs) {
    PagePools pools;
    if (!ctx || !pools_from(n_layers, k_pools, v_pools, &pools)) return TTS_ERR_INVALID;
    return fork_pages(reinterpret_cast<Ctx*>(ctx), pools, block_table, prefix_len, branch_lens, n_branches, parents, n_children, page_refs, new_table,
                      new_lens, new_refs);
}

int tts_kv_grow(tts_ctx* ctx, int32_t* block_table, int prefix_len, int32_t* branch_lens, const int32_t* n_new, int n_branches, int32_t* page_refs) {
    Ctx* c = reinterpret_cast<Ctx*>(ctx);
    if (!c || !branch_lens || !n_new || !page_refs || !branches_ok(c, block_table, prefix_len, n_branches)) return TTS_ERR_INVALID;
    if (!aligned4(branch_lens) || !aligned4(n_new) || !aligned16(page_refs)) return TTS_ERR_INVALID;
    const Span table{block_table, table_bytes(c->cfg, n_branches)}, lens{branch_lens, (size_t)n_branches * 4}, more{n_new, lens.bytes},
        refs{page_refs, (size_t)c->cfg.num_pages * 4};
    if (clash(table, {lens, more, refs}) || clash(lens, {more, refs}) || clash(refs, {more})) return TTS_ERR_INVALID;
    c->plan_explicit = 0;                               // the lengths and the table change
    const OnDevice on(c->device);
    if (on.error() != cudaSuccess) return finish(c, on.error(), 0);
    return finish(c, launch_grow(block_table, c->cfg.max_blocks_per_branch, prefix_len, branch_lens, n_new, n_branches, page_refs, c->cfg.num_pages,
                                 page_work(c), c->d_status, c->stream), 1);
}

int tts_kv_free(tts_ctx* ctx, int32_t* block_table, int32_t* branch_lens, const int32_t* freed, int n_branches, int32_t* page_refs) {
    Ctx* c = reinterpret_cast<Ctx*>(ctx);
    if (!c || !branch_lens || !freed || !page_refs || !branches_ok(c, block_table, 0, n_branches)) return TTS_ERR_INVALID;
    if (!aligned4(branch_lens) || !aligned4(freed) || !aligned16(page_refs)) return TTS_ERR_INVALID;
    const Span table{block_table, table_bytes(c->cfg, n_branches)}, lens{branch_lens, (size_t)n_branches * 4}, which{freed, lens.bytes},
        refs{page_refs, (size_t)c->cfg.num_pages * 4};
    if (clash(table, {lens, which, refs}) || clash(lens, {which, refs}) || clash(refs, {which})) return TTS_ERR_INVALID;
    c->plan_explicit = 0;
    const OnDevice on(c->device);
    if (on.error() != cudaSuccess) return finish(c, on.error(), 0);
    return finish(c, launch_free(block_table, c->cfg.max_blocks_per_branch, branch_lens, freed, n_branches, page_refs, c->cfg.num_pages, c->d_status,
                                 c->stream), 1);
}

int tts_kv_compact(tts_ctx* ctx, int n_layers, void* const* k_pools, void* const* v_pools, const int32_t* block_table, int n_branches,
                   const int32_t* page_refs, int32_t* new_table, int32_t* new_refs, int32_t* page_map, int32_t* n_used) {
    PagePools pools;
    if (!ctx || !pools_from(n_layers, k_pools, v_pools, &pools)) return TTS_ERR_INVALID;
    return compact_pages(reinterpret_cast<Ctx*>(ctx), pools, block_table, n_branches, page_refs, new_table, new_refs, page_map, n_used);
}

int tts_kv8_copy_pages(tts_ctx* ctx, int n_layers, void* const* kv8_pools, const int32_t* src_pages, const int32_t* dst_pages,
                      int n_copies) {
    PagePools pools;
    if (!ctx || !pools_from_kv8(n_layers, kv8_pools, &pools)) return TTS_ERR_INVALID;
    return copy_pages(reinterpret_cast<Ctx*>(ctx), pools, src_pages, dst_pages, n_copies);
}

int tts_kv8_fork(tts_ctx* ctx, int n_layers, void* const* kv8_pools, const int32_t* block_table, int prefix_len,
                const int32_t* branch_lens, int n_branches, const int32_t* parents, int n_children, const int32_t* page_refs,
                int32_t* new_table, int32_t* new_lens, int32_t* new_refs) {
    PagePools pools;
    if (!ctx || !pools_from_kv8(n_layers, kv8_pools, &pools)) return TTS_ERR_INVALID;
    return fork_pages(reinterpret_cast<Ctx*>(ctx), pools, block_table, prefix_len, branch_lens, n_branches, parents, n_children, page_refs, new_table,
                      new_lens, new_refs);
}

int tts_kv8_compact(tts_ctx* ctx, int n_layers, void* const* kv8_pools, const int32_t* block_table, int n_branches,
                   const int32_t* page_refs, int32_t* new_table, int32_t* new_refs, int32_t* page_map, int32_t* n_used) {
    PagePools pools;
    if (!ctx || !pools_from_kv8(n_layers, kv8_pools, &pools)) return TTS_ERR_INVALID;
    return compact_pages(reinterpret_cast<Ctx*>(ctx), pools, block_table, n_branches, page_refs, new_table, new_refs, page_map, n_used);
}

}  // extern "C"
