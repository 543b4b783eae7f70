// Beam search: internal declarations (kdn_beam*.hip).
#pragma once

#include "kdn_internal.h"

namespace kdn {

constexpr int BEAM_MAX = 64;  // beams of a batch element: one lane each

size_t beam_workspace_bytes(int N, int W, int V);
hipError_t launch_beam_select(const void* logits, const float* scores, const uint8_t* done, int N,
                              int W, int V, kdn_dtype_t dtype, int end_token, float* scores_out,
                              int32_t* token_out, int32_t* parent_out, uint8_t* done_out,
                              void* workspace, hipStream_t stream);
hipError_t launch_beam_reorder(const int32_t* parent, const int32_t* slot_idx, int32_t* slot_out,
                               int N, int W, int num_slots, void* S, size_t s_bytes, void* P,
                               size_t p_bytes, hipStream_t stream);

}  // namespace kdn
