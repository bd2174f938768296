// Beam selection and reordering of the beams' states.
#pragma once
#include "tts_internal.cuh"

namespace tts {

constexpr int kMaxSelect = 128;        // continuations that a question may keep
constexpr int kMaxBeamCandidates = 8192;   // beams of a question times continuations: what the joining block sorts in shared memory

struct BeamParams {
    const void* logits;
    long row_stride;                   // elements
    const float* beam_scores;
    const int32_t* finished;           // or null
    double* lse;                       // [rows] logarithm of the sum of the row's exponentials
    int32_t* count;                    // [rows] entries of `best`
    unsigned long long* best;          // [rows][n_select] (key of the logit, 2^32 - 1 - token)
    int32_t *parents, *tokens;
    float* scores;
    int vocab, pad_token, n_groups, n_beams, n_select, per_cta;
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
constexpr int kReorderUnits = 8 * kReorderThreads;             // 16-byte (or 4-byte, or 1-byte) units of a row that a block moves
// bytes of the widest unit that all rows of an array start and end on
inline int reorder_unit(const void* src, const void* dst, long row_bytes) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(src) | reinterpret_cast<uintptr_t>(dst) | (uintptr_t)row_bytes;
    return x & 3 ? 1 : x & 15 ? 4 : 16;
}
cudaError_t launch_beam_select(BeamParams p, int logits_dtype, int n_sms, cudaStream_t st);
cudaError_t launch_beam_reorder(const ReorderParams& p, cudaStream_t st);

}  // namespace tts
