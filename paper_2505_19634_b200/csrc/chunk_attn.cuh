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
    int once;          // the branch's keys are read by this entry alone
};
static_assert(sizeof(ChunkPiece) == 48, "read as three 16-byte words");

constexpr int kChunkTile = 128;                       // KV tokens per tile
constexpr int kChunkPartsPerSm = 4;                   // pieces with partial results that the workspace has room for, per SM

struct ChunkHead {
    int pieces_per_head;
    int next;          // the next piece that nobody has taken yet
    int rows_per_head; // partial-result rows of one KV head
    int entries;
};

struct ChunkParams {
    const int32_t* block_table;
    const int32_t* branch_lens;
    const int32_t* row_start;
    void* out;
    float* lse;                    // may be null
    ChunkHead* head;
    ChunkPiece* pieces;
    int2* entry_tiles;             // [entries] KV tiles and new tokens of each entry
    int* arrived;                  // [Hkv][entries][2] pieces that have left their partial result
    float* part_o;                 // [part_rows][128]
    float2* part_ml;               // [part_rows] (max in log2 units, sum)
    int32_t* status;
    int Hq, Hkv, G, T;
    int prefix_len, n_branches, total_rows, max_blocks, num_pages;
    int max_pieces;                // capacity: pieces per KV head
    long part_rows;                // capacity: partial-result rows
    int grid;
    int out_dtype;
    float scale_log2;
};

cudaError_t launch_chunk_plan(const ChunkParams& p, cudaStream_t st);
cudaError_t launch_chunk_attn(const ChunkParams& p, const void* q, long q_stride, const void* k_pages, const void* v_pages, cudaStream_t st);

}  // namespace tts
