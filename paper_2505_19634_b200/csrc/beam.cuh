// Beam selection and reordering of the beams' states.
#pragma once
#include "tts_internal.cuh"

namespace tts {

constexpr int kMaxSelect = 128;        // continuations that a question may keep
constexpr int kMaxBeamCandidates = 8192;   // beams of a question times continuations
// Candidates that a part of a row may leave for the question's last CTA, a power of two: more than the n best, for what the bound lets through.
__host__ __device__ constexpr int beam_cap_log2(int n) { return n <= 16 ? 6 : n <= 48 ? 7 : n <= 96 ? 8 : 9; }
// Parts of a row, 2^0 to 2^3: as long as the GPU takes all of them at once, four CTAs to an SM, and each has 4096 logits.
// (16 questions of 16 beams: 44.5 us in one part, 34.5 in two; one question of 4 beams: 19.7 in one, 16.0 in two, 10.9 in eight.)
inline int beam_parts_log2(int rows, int vocab, int n_sms) {
    int log2 = 0;
    while (log2 < 3 && (long)rows << (log2 + 1) <= 4l * n_sms && vocab >> (log2 + 1) >= 4096) ++log2;
    return log2;
}
inline long beam_max_parts(int rows, int n_sms) { return rows > 4 * n_sms ? rows : 4l * n_sms; }       // of all rows of a call

struct BeamParams {
    const void* logits;
    long row_stride;                   // elements
    const float* beam_scores;
    const int32_t* finished;           // or null
    double* part_sum;                  // of every part of a row: the sum of exp(logit - the largest),
    float* part_top;                   // the largest logit
    unsigned long long* entries;       // of every question: its parts' candidates (key of the logit, beam * vocab + token), in any order,
    int32_t* n_entries;                // their number,
    int32_t* arrived;                  // and the parts that have ended; the last two are zero between calls
    int32_t *parents, *tokens;
    float* scores;
    int vocab, pad_token, n_groups, n_beams, n_select, parts_log2, cap_log2, per_part;
};
constexpr int kMaxStates = 128;
struct ReorderParams {
    const unsigned char* src[kMaxStates];
    unsigned char* dst[kMaxStates];
    long row_bytes[kMaxStates];
    int first[kMaxStates + 1];         // blocks before each array
    const int32_t* parents;
    int32_t* status;
    int n_states, n_in, n_out;
};
constexpr int kReorderThreads = 256;
constexpr int kReorderUnits = 8 * kReorderThreads;             // 16-byte units of a row that a block moves
// all rows of an array start and end on 16-byte boundaries, in src and in dst
__host__ __device__ inline bool reorder_aligned(const void* src, const void* dst, long row_bytes) {
    return ((reinterpret_cast<uintptr_t>(src) | reinterpret_cast<uintptr_t>(dst) | (uintptr_t)row_bytes) & 15) == 0;
}
// units of a row; an unaligned one may start and end within a unit
inline long reorder_units(const void* src, const void* dst, long row_bytes) { return reorder_aligned(src, dst, row_bytes) ? row_bytes / 16 : (row_bytes + 30) / 16; }
cudaError_t launch_beam_select(BeamParams p, int logits_dtype, cudaStream_t st);
cudaError_t launch_beam_reorder(const ReorderParams& p, cudaStream_t st);

}  // namespace tts
