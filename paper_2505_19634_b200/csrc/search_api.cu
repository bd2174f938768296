// C-ABI layer of the search operators: the 8-bit cache, beam selection, reordering.  Argument checks, workspace, launches.
// See include/tts.h.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "api_checks.cuh"
#include "beam.cuh"
#include "kv8.cuh"
#include "launch.cuh"

using namespace tts;

namespace {

bool format_ok(int format) { return format == TTS_KV8_E4M3 || format == TTS_KV8_INT8; }
size_t kv8_bytes(const tts_config& f) { return (size_t)f.num_pages * f.n_kv_heads * kKv8Record; }

}  // namespace

extern "C" {

int tts_kv8_append(tts_ctx* ctx, int format, const tts_rope* rope, const void* q, int64_t q_row_stride, const void* k, const void* v,
                   int64_t kv_row_stride, const int32_t* positions, void* kv8_pages, const int32_t* block_table, int prefix_len,
                   const int32_t* branch_lens, const int32_t* row_start, int n_branches, int total_rows, void* q_out) {
    Ctx* c = reinterpret_cast<Ctx*>(ctx);
    if (!c || !k || !v || !kv8_pages || !branch_lens || !row_start) return TTS_ERR_INVALID;
    if (rope ? !q || !positions || !q_out : q || positions || q_out) return TTS_ERR_INVALID;
    if (!format_ok(format)) return TTS_ERR_UNSUPPORTED;
    if (!branches_ok(c, block_table, prefix_len, n_branches)) return TTS_ERR_INVALID;
    const tts_config& f = c->cfg;
    if (rope) {
        if (rope->n_pairs < 1 || rope->n_pairs > kHeadDim / 2 || rope->n_axes < 1 || rope->n_axes > 8) return TTS_ERR_INVALID;
        for (int i = 0; i < rope->n_pairs; ++i)
            if (rope->axis[i] >= rope->n_axes || !isfinite(rope->inv_freq[i])) return TTS_ERR_INVALID;
    }
    if (total_rows < 0) return TTS_ERR_INVALID;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(kv8_pages) || !aligned16(q_out)) return TTS_ERR_INVALID;
    if (!aligned4(positions) || !aligned4(branch_lens) || !aligned4(row_start)) return TTS_ERR_INVALID;
    const int64_t q_row = (int64_t)f.n_q_heads * kHeadDim, kv_row = (int64_t)f.n_kv_heads * kHeadDim;
    if (rope && (q_row_stride < q_row || q_row_stride % 8 != 0 || q_row_stride >= (1ll << 38))) return TTS_ERR_INVALID;
    if (kv_row_stride < kv_row || kv_row_stride % 8 != 0 || kv_row_stride >= (1ll << 38)) return TTS_ERR_INVALID;
    if (total_rows == 0) return TTS_OK;
    // q_out may be q itself, when q is dense; any other overlap would be read after it is written
    const size_t kv_bytes = ((size_t)(total_rows - 1) * kv_row_stride + kv_row) * 2;
    const Span new_k{k, kv_bytes}, new_v{v, kv_bytes}, pool{kv8_pages, kv8_bytes(f)}, table{block_table, table_bytes(f, n_branches)},
        lens{branch_lens, (size_t)n_branches * 4}, starts{row_start, (size_t)(n_branches + 1) * 4};
    if (clash(pool, {new_k, new_v, table, lens, starts})) return TTS_ERR_INVALID;
    if (rope) {
        const Span queries{q, ((size_t)(total_rows - 1) * q_row_stride + q_row) * 2}, at{positions, (size_t)rope->n_axes * total_rows * 4},
            turned{q_out, (size_t)total_rows * q_row * 2};
        if (clash(turned, {queries}) && !(q == q_out && q_row_stride == q_row)) return TTS_ERR_INVALID;
        if (clash(turned, {new_k, new_v, at, pool, table, lens, starts}) || clash(pool, {queries, at})) return TTS_ERR_INVALID;
    }
    const OnDevice on(c->device);
    if (on.error() != cudaSuccess) return finish(c, on.error(), 0);
    RopeParams p;
    memset(&p, 0, sizeof p);
    p.q = static_cast<const __nv_bfloat16*>(q); p.k = static_cast<const __nv_bfloat16*>(k); p.v = static_cast<const __nv_bfloat16*>(v);
    p.q_stride = (long)q_row_stride; p.kv_stride = (long)kv_row_stride; p.positions = positions;
    p.q_out = static_cast<__nv_bfloat16*>(q_out); p.kv8_pages = static_cast<unsigned char*>(kv8_pages); p.kv8_format = format;
    p.block_table = block_table; p.branch_lens = branch_lens; p.row_start = row_start; p.status = c->d_status;
    p.Hq = rope ? f.n_q_heads : 0; p.Hkv = f.n_kv_heads;
    p.prefix_len = prefix_len; p.n_branches = n_branches; p.total_rows = total_rows; p.max_blocks = f.max_blocks_per_branch; p.num_pages = f.num_pages;
    if (rope) {
        p.n_pairs = rope->n_pairs; p.interleaved = rope->interleaved != 0;
        for (int i = 0; i < rope->n_pairs; ++i) { p.axis[i] = rope->axis[i]; p.turns[i] = rope->inv_freq[i] / 6.283185307179586476925; }
    }
    return finish(c, launch_append_rope(p, c->n_sms, c->stream), 1);
}

int tts_kv8_read(tts_ctx* ctx, int format, const void* kv8_pages, const int32_t* src_pages, const int32_t* dst_pages, int n_pages, void* k_pages,
                 void* v_pages, int num_dst_pages) {
    Ctx* c = reinterpret_cast<Ctx*>(ctx);
    if (!c || !kv8_pages || !src_pages || !dst_pages || !k_pages || !v_pages || n_pages < 0 || num_dst_pages < 1) return TTS_ERR_INVALID;
    if (!format_ok(format)) return TTS_ERR_UNSUPPORTED;
    if (!aligned16(kv8_pages) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned4(src_pages) || !aligned4(dst_pages)) return TTS_ERR_INVALID;
    const tts_config& f = c->cfg;
    const size_t bytes = (size_t)num_dst_pages * f.n_kv_heads * kPage * kHeadDim * 2;
    const Span pool{kv8_pages, kv8_bytes(f)}, keys{k_pages, bytes}, values{v_pages, bytes}, src{src_pages, (size_t)n_pages * 4}, dst{dst_pages, (size_t)n_pages * 4};
    if (clash(keys, {pool, values, src, dst}) || clash(values, {pool, src, dst})) return TTS_ERR_INVALID;
    if (n_pages == 0) return TTS_OK;
    const OnDevice on(c->device);
    if (on.error() != cudaSuccess) return finish(c, on.error(), 0);
    Kv8ReadParams p;
    p.pool = static_cast<const unsigned char*>(kv8_pages); p.src = src_pages; p.dst = dst_pages;
    p.k_pages = static_cast<__nv_bfloat16*>(k_pages); p.v_pages = static_cast<__nv_bfloat16*>(v_pages);
    p.status = c->d_status; p.n = n_pages; p.Hkv = f.n_kv_heads; p.num_pages = f.num_pages; p.num_dst = num_dst_pages;
    return finish(c, launch_kv8_read(p, format, c->n_sms, c->stream), 1);
}

int tts_kv8_attn(tts_ctx* ctx, int format, const void* q, int64_t q_row_stride, const void* kv8_pages, const int32_t* block_table, int prefix_len,
                 const int32_t* branch_lens, const int32_t* tree_parents, int n_branches, int rows_per_branch, void* out, float* lse) {
    Ctx* c = reinterpret_cast<Ctx*>(ctx);
    if (!c || !q || !kv8_pages || !branch_lens || !out) return TTS_ERR_INVALID;
    if (!format_ok(format)) return TTS_ERR_UNSUPPORTED;
    if (!branches_ok(c, block_table, prefix_len, n_branches)) return TTS_ERR_INVALID;
    const tts_config& f = c->cfg;
    if (rows_per_branch < 1 || rows_per_branch > f.max_rows_per_branch) return TTS_ERR_INVALID;
    if (!aligned16(q) || !aligned16(kv8_pages) || !aligned16(out) || !aligned4(lse) || !aligned4(branch_lens) || !aligned4(tree_parents)) return TTS_ERR_INVALID;
    if (q_row_stride < (int64_t)f.n_q_heads * kHeadDim || q_row_stride % 8 != 0 || q_row_stride >= (1ll << 38)) return TTS_ERR_INVALID;
    const size_t rows = (size_t)n_branches * rows_per_branch;
    const Span queries{q, ((rows - 1) * q_row_stride + (size_t)f.n_q_heads * kHeadDim) * 2}, pool{kv8_pages, kv8_bytes(f)},
        table{block_table, table_bytes(f, n_branches)}, lens{branch_lens, (size_t)n_branches * 4}, parents{tree_parents, tree_parents ? rows * 4 : 0},
        result{out, rows * f.n_q_heads * kHeadDim * (f.out_dtype == TTS_OUT_FP32 ? 4 : 2)}, logs{lse, lse ? rows * f.n_q_heads * 4 : 0};
    const int nr = rows_per_branch * (f.n_q_heads / f.n_kv_heads);
    const bool wide = nr >= kKv8WideFrom;
    const int n_rb = ceil_div(nr, wide ? kKv8WideRows : kKv8MaxRows), most = wide ? 2 * c->n_sms : c->n_sms, grid = f.max_ctas > 0 && f.max_ctas < most ? f.max_ctas : most;
    // (units of a CTA, pages and at most 64 more for each item, are counted in 32 bits)
    if ((double)n_branches * (f.max_blocks_per_branch + 64.0) * f.n_kv_heads * n_rb / grid >= 2e9) return TTS_ERR_UNSUPPORTED;
    if (clash(result, {queries, pool, table, lens}) || (tree_parents && clash(result, {parents})) ||
        (lse && (clash(logs, {result, queries, pool, table, lens}) || (tree_parents && clash(logs, {parents})))))
        return TTS_ERR_INVALID;
    const OnDevice on(c->device);
    if (on.error() != cudaSuccess) return finish(c, on.error(), 0);
    Kv8AttnParams p;
    memset(&p, 0, sizeof p);
    p.q = static_cast<const __nv_bfloat16*>(q); p.q_stride = (long)q_row_stride; p.pool = static_cast<const unsigned char*>(kv8_pages);
    p.block_table = block_table; p.branch_lens = branch_lens; p.tree_parents = tree_parents; p.out = out; p.lse = lse;
    p.part_o = c->part_o_priv; p.part_ml = c->part_ml_priv; p.arrived = c->kv8_arrived; p.status = c->d_status;
    p.Hq = f.n_q_heads; p.Hkv = f.n_kv_heads; p.G = p.Hq / p.Hkv; p.R = rows_per_branch; p.nr = nr;
    p.n_rb = n_rb; p.rb_rows = ceil_div(p.nr, p.n_rb);
    p.prefix_len = prefix_len; p.n_branches = n_branches; p.max_blocks = f.max_blocks_per_branch; p.num_pages = f.num_pages; p.out_dtype = f.out_dtype;
    p.grid = grid;
    p.scale_log2 = (f.softmax_scale > 0.f ? f.softmax_scale : 1.0f / sqrtf((float)f.head_dim)) * 1.4426950408889634f;
    return finish(c, wide ? launch_kv8_attn_wide(p, format, c->stream) : launch_kv8_attn(p, format, c->stream), 1);
}

int tts_beam_reserve(tts_ctx* ctx, int max_rows, int max_select) {
    Ctx* c = reinterpret_cast<Ctx*>(ctx);
    if (!c || max_rows < 1 || max_rows > c->cfg.max_branches || max_select < 1) return TTS_ERR_INVALID;
    if (max_select > kMaxSelect) return TTS_ERR_UNSUPPORTED;
    if (c->beam_rows > 0) return max_rows <= c->beam_rows && max_select <= c->beam_select ? TTS_OK : TTS_ERR_INVALID;
    const OnDevice on(c->device);
    if (on.error() != cudaSuccess) return finish(c, on.error(), 0);
    // candidates, a sum and a maximum for every part of a row, two counters for every question
    const size_t bytes = (size_t)beam_max_parts(max_rows, c->n_sms) * ((8 << beam_cap_log2(max_select)) + 12) + (size_t)max_rows * 8;
    cudaError_t e = cudaMalloc(&c->beam_work, bytes);
    if (e != cudaSuccess) { c->beam_work = nullptr; return finish(c, e, 0); }
    e = cudaMemset(c->beam_work, 0, bytes);
    if (e == cudaSuccess) e = cudaStreamSynchronize(cudaStreamLegacy);       // before work on a stream that does not wait for it
    if (e != cudaSuccess) { cudaFree(c->beam_work); c->beam_work = nullptr; return finish(c, e, 0); }
    c->beam_rows = max_rows; c->beam_select = max_select;
    return TTS_OK;
}

int tts_beam_select(tts_ctx* ctx, const void* logits, int logits_dtype, int64_t row_stride, int vocab, const float* beam_scores,
                    const int32_t* finished, int pad_token, int n_groups, int n_beams, int n_select, int32_t* parents, int32_t* tokens, float* scores) {
    Ctx* c = reinterpret_cast<Ctx*>(ctx);
    if (!c || !logits || !beam_scores || !parents || !tokens || !scores) return TTS_ERR_INVALID;
    if (logits_dtype != TTS_LOGITS_BF16 && logits_dtype != TTS_LOGITS_FP32) return TTS_ERR_UNSUPPORTED;
    if (vocab < 1 || n_groups < 1 || n_beams < 1 || n_select < 1 || (long)n_groups * n_beams > c->beam_rows || n_select > c->beam_select) return TTS_ERR_INVALID;
    if ((long)n_beams * n_select > kMaxBeamCandidates || (long)n_beams * vocab >= (1l << 31) - (1l << 16)) return TTS_ERR_UNSUPPORTED;
    if (finished && (pad_token < 0 || pad_token >= vocab)) return TTS_ERR_INVALID;
    if (row_stride < vocab || row_stride >= (1ll << 38)) return TTS_ERR_INVALID;
    const size_t elt = logits_dtype == TTS_LOGITS_BF16 ? 2 : 4, rows = (size_t)n_groups * n_beams, picks = (size_t)n_groups * n_select * 4;
    if (reinterpret_cast<uintptr_t>(logits) % elt != 0 || !aligned4(beam_scores) || !aligned4(finished) || !aligned4(parents) || !aligned4(tokens) || !aligned4(scores))
        return TTS_ERR_INVALID;
    const Span in{logits, ((rows - 1) * row_stride + vocab) * elt}, before{beam_scores, rows * 4}, done{finished, finished ? rows * 4 : 0}, out_p{parents, picks},
        out_t{tokens, picks}, out_s{scores, picks};
    if (clash(out_p, {in, before, out_t, out_s}) || clash(out_t, {in, before, out_s}) || clash(out_s, {in, before})) return TTS_ERR_INVALID;
    if (finished && (clash(out_p, {done}) || clash(out_t, {done}) || clash(out_s, {done}))) return TTS_ERR_INVALID;
    const OnDevice on(c->device);
    if (on.error() != cudaSuccess) return finish(c, on.error(), 0);
    BeamParams p;
    memset(&p, 0, sizeof p);
    p.logits = logits; p.row_stride = (long)row_stride; p.beam_scores = beam_scores; p.finished = finished;
    const size_t parts = (size_t)beam_max_parts(c->beam_rows, c->n_sms);
    p.entries = static_cast<unsigned long long*>(c->beam_work);
    p.part_sum = reinterpret_cast<double*>(p.entries + (parts << beam_cap_log2(c->beam_select)));
    p.part_top = reinterpret_cast<float*>(p.part_sum + parts);
    p.n_entries = reinterpret_cast<int32_t*>(p.part_top + parts);
    p.arrived = p.n_entries + c->beam_rows;
    p.parents = parents; p.tokens = tokens; p.scores = scores;
    p.vocab = vocab; p.pad_token = pad_token; p.n_groups = n_groups; p.n_beams = n_beams; p.n_select = n_select;
    p.parts_log2 = beam_parts_log2(n_groups * n_beams, vocab, c->n_sms); p.cap_log2 = beam_cap_log2(n_select);
    return finish(c, launch_beam_select(p, logits_dtype, c->stream), 1);
}

int tts_beam_reorder(tts_ctx* ctx, int n_states, const void* const* src, void* const* dst, const int64_t* row_bytes, const int32_t* parents,
                     int n_rows, int n_children) {
    Ctx* c = reinterpret_cast<Ctx*>(ctx);
    if (!c || !src || !dst || !row_bytes || !parents || !aligned4(parents) || n_states < 1 || n_states > kMaxStates || n_rows < 1 || n_children < 1)
        return TTS_ERR_INVALID;
    ReorderParams p;
    memset(&p, 0, sizeof p);
    long blocks = 0;
    for (int i = 0; i < n_states; ++i) {
        if (!src[i] || !dst[i] || row_bytes[i] < 1 || row_bytes[i] >= (1ll << 40)) return TTS_ERR_INVALID;
        p.src[i] = static_cast<const unsigned char*>(src[i]); p.dst[i] = static_cast<unsigned char*>(dst[i]); p.row_bytes[i] = row_bytes[i];
        const long units = reorder_units(src[i], dst[i], row_bytes[i]);
        p.first[i] = (int)blocks;
        blocks += (units + kReorderUnits - 1) / kReorderUnits * n_children;
        if (blocks >= (1l << 31)) return TTS_ERR_UNSUPPORTED;
    }
    p.first[n_states] = (int)blocks;
    // rows are read in any order while others are written: in the order of their addresses, no written array may start before
    // the end of any other, nor a read one before the end of a written one
    struct Extent { uintptr_t begin, end; bool written; };
    Extent at[2 * kMaxStates + 1];
    for (int i = 0; i < n_states; ++i) {
        const uintptr_t from = reinterpret_cast<uintptr_t>(src[i]), to = reinterpret_cast<uintptr_t>(dst[i]);
        at[i] = {from, from + (size_t)n_rows * row_bytes[i], false};
        at[n_states + i] = {to, to + (size_t)n_children * row_bytes[i], true};
    }
    at[2 * n_states] = {reinterpret_cast<uintptr_t>(parents), reinterpret_cast<uintptr_t>(parents) + (size_t)n_children * 4, false};
    std::sort(at, at + 2 * n_states + 1, [](const Extent& x, const Extent& y) { return x.begin < y.begin; });
    uintptr_t any = 0, written = 0;
    for (int i = 0; i <= 2 * n_states; ++i) {
        if (at[i].begin < (at[i].written ? any : written)) return TTS_ERR_INVALID;
        any = std::max(any, at[i].end);
        if (at[i].written) written = std::max(written, at[i].end);
    }
    const OnDevice on(c->device);
    if (on.error() != cudaSuccess) return finish(c, on.error(), 0);
    p.parents = parents; p.status = c->d_status; p.n_states = n_states; p.n_in = n_rows; p.n_out = n_children;
    return finish(c, launch_beam_reorder(p, c->stream), 1);
}

}  // extern "C"
