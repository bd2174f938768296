// Schedule of the chunk attention (chunk_plan.cu writes it, chunk_attn.cu runs from it).
#pragma once
#include "tts_internal.cuh"

namespace tts {

// An *entry* is a run of up to 2 T new tokens of one branch, T = 128 / G being the tokens whose G query rows
// (the heads that share a KV head) fill one 128-row MMA tile.  An entry with more than T tokens is `wide`: its
// two row tiles walk the same KV tiles side by side.  A narrow one has one row tile and its even and odd KV
// tiles go to the two sides.  Every entry is worked on once per KV head, in one piece or in several runs of
// KV tiles (*pieces*) whose partial results the last one to finish puts together.
struct ChunkPiece {
    int branch;
    int row0;          // first row of the entry in q / out
    int n_tok;         // new tokens of the entry (1 .. 2 T)
    int limit0;        // keys that the entry's first token sees; may be <= 0 (sees nothing)
    int tile_begin, tile_end;
    int keys;          // cached tokens of the branch, the chunk included
    int parts;         // pieces of this entry (1: the piece writes the result itself)
    int part;          // which of them this is
    int part_row;      // first row of the entry's partial results, within its KV head's
    int entry;
    int once;          // the branch has no other entry in this call (a prefix that it shares with other branches is theirs as well)
};
static_assert(sizeof(ChunkPiece) == 48, "read as three 16-byte words");

constexpr int kChunkTile = 128;                       // KV tokens per tile
constexpr int kChunkPartsPerSm = 8;                   // wide pieces with partial results that the workspace has room for, per SM
constexpr int kChunkSmall = 64;                       // calls of up to so many entries are scheduled inside the attention kernel

struct ChunkHead {
    int pieces;        // per KV head
    unsigned next;     // pieces taken from the list, apart from each CTA's first; wraps to 0 with the last one
    int part_rows;     // partial-result rows of one KV head
    int pad;
};

struct ChunkParams {
    const int32_t* block_table;
    const int32_t* branch_lens;
    const int32_t* row_start;
    void* out;
    float* lse;                    // may be null
    ChunkHead* head;
    ChunkPiece* pieces;
    int small;                     // see kChunkSmall
    unsigned* arrived;             // [entries][Hkv][2] pieces that have left their partial result; the last one sets it back to 0
    float* part_o;                 // [part_rows][128]
    float2* part_ml;               // [part_rows] (max in log2 units, sum)
    int32_t* status;
    int Hq, Hkv, G, T;
    int prefix_len, n_branches, total_rows, max_blocks, num_pages;
    int max_pieces;                // capacity: pieces per KV head
    long part_rows;                // capacity: partial-result rows
    int grid;
    float heads_per_cta, ctas_per_head;   // Hkv / grid, grid / Hkv
    unsigned g_inv;                // x * g_inv >> 16 is x / G for x < 128: the error, x / 65536 at most, is below 1 / G
    int out_dtype;
    int out_32;                    // out is 32-byte aligned
    float scale_log2;
};

// ---- what both places that make a schedule share (the reasons are in chunk_plan.cu) ----
struct ChunkEntry { int b, row0, n_tok, limit0, keys, tiles, once; };

// The `index`-th entry of branch b, whose rows start at `start` (c of them) and which holds `keys` tokens.
__device__ __forceinline__ ChunkEntry chunk_entry(int T, int b, int index, int start, int c, int keys) {
    const int tok0 = index * 2 * T;
    ChunkEntry r;
    r.b = b; r.row0 = start + tok0; r.n_tok = min(2 * T, c - tok0); r.keys = keys;
    r.limit0 = keys - c + tok0 + 1;
    r.tiles = ceil_div(min(keys, max(0, r.limit0 + r.n_tok - 1)), kChunkTile);
    r.once = c <= 2 * T;
    return r;
}
__device__ __forceinline__ ChunkPiece chunk_piece(const ChunkEntry& r, int e, int part, int parts, int part_row) {
    ChunkPiece x;
    x.branch = r.b; x.row0 = r.row0; x.n_tok = r.n_tok; x.limit0 = r.limit0; x.keys = r.keys;
    // as even as whole tiles go, the longer ones first
    const int each = parts == 1 ? r.tiles : r.tiles / parts, longer = r.tiles - each * parts;
    x.tile_begin = part * each + min(part, longer); x.tile_end = x.tile_begin + each + (part < longer);
    x.parts = parts; x.part = part; x.part_row = part_row; x.entry = e; x.once = r.once;
    return x;
}
// A call whose row starts or lengths make no sense computes nothing.
__device__ __forceinline__ bool chunk_branch_ok(const ChunkParams& p, int lo, int hi, int len) {
    return lo >= 0 && hi >= lo && hi <= p.total_rows && len >= 0 && (long)p.prefix_len + len <= (long)p.max_blocks * kPage;
}
__device__ __forceinline__ int chunk_cost(const ChunkEntry& r, int T) { return r.tiles * (r.n_tok > T ? 2 : 1); }

constexpr float kChunkSlack = 10.f;                   // what the pieces of a call cost a CTA beside their tiles, about
constexpr int kChunkNoBound = 1 << 30;                // leaves every entry whole

// How small the pieces of a call may become.  `total`: the cost of its n entries per KV head, `largest` the costliest.
//   one wave   fewer entries than CTAs, and no piece of it much longer than a CTA's share: at most `narrow` = total /
//              (CTAs per KV head - n) per piece makes no more pieces than CTAs, whatever the entries are.  (200 tokens of
//              40 heads over 4000 keys: 44 us in one wave of 128 pieces, 82 us as 192 shorter ones.)
//   guided     otherwise pieces get smaller towards the end of the list (chunk_cuts), down to a sixteenth of a CTA's
//              share, but not below six tiles, whose time is several times what a piece costs by itself.  A wide piece's
//              partial result is 256 rows to write and to join: its bound is twice a narrow one's.
struct ChunkBound { int narrow, wide; bool one_wave; };
__device__ __forceinline__ ChunkBound chunk_bound(const ChunkParams& p, float total, int n, float largest) {
    const float share = total * p.heads_per_cta, spare = p.ctas_per_head - n, one = __fdividef(total, fmaxf(spare, 1.f));
    if (spare >= 1.f && fminf(one, largest) <= share + 12.f) {
        const int b = max(4, (int)ceilf(one));
        return {b, max(b, 8), true};
    }
    const int b = max(6, (int)(share / 16.f));
    return {b, 2 * b, false};
}
// larger pieces, when the partial results would not fit the workspace
__device__ __forceinline__ ChunkBound chunk_coarser(ChunkBound b) {
    const int n = b.narrow >= 4096 ? kChunkNoBound : b.narrow * 2;
    return {n, n == kChunkNoBound ? n : b.wide * 2, b.one_wave};
}
// Pieces of entry r, the `place`-th to be handed out, when `left` per KV head is still to be, its own cost included.
// Guided: a piece may cost what is left for each CTA, so that it ends with the others; those that every CTA starts with
// may cost a CTA's whole share.
__device__ __forceinline__ int chunk_cuts(const ChunkParams& p, const ChunkEntry& r, int place, float left, float total, ChunkBound bound) {
    if (bound.narrow == kChunkNoBound) return 1;
    const bool wide = r.n_tok > p.T, starts = (place + 1) * p.Hkv <= p.grid;
    float limit = (float)(wide ? bound.wide : bound.narrow);
    if (!bound.one_wave) limit = fmaxf(limit, (starts ? total : left) * p.heads_per_cta + kChunkSlack);
    return max(1, min(r.tiles, (int)ceilf(__fdividef((float)(wide ? 2 * r.tiles : r.tiles), limit))));
}

cudaError_t launch_chunk_plan(const ChunkParams& p, cudaStream_t st);
cudaError_t launch_chunk_attn(const ChunkParams& p, const void* q, long q_stride, const void* k_pages, const void* v_pages, cudaStream_t st);

}  // namespace tts
