// Gated delta rule: internal declarations (kdn_gdr*.hip).
#pragma once

#include "kdn_internal.h"

namespace kdn {

struct GdrCall {
    const void *q, *k, *v, *alpha, *beta;
    const float* S0;  // [N,H,dk,dv], or nullptr (0)
    void* o;
    float* S_T;  // or nullptr
    SeqArgs sa;
    int Hk, dk, dv;  // Hk key heads; value head h reads key head h / (H / Hk)
    kdn_dtype_t dtype;
    float scale;
    void* workspace;
};

// One token per row on a pool of states, or a few tokens per sequence, token by token (kdn_gdr.hip).
hipError_t launch_gdr_decode(const void* q, const void* k, const void* v, const void* alpha,
                             const void* beta, float* S, const int32_t* slot_idx, void* o, int R,
                             int num_slots, int H, int Hk, int dk, int dv, kdn_dtype_t dtype,
                             float scale, hipStream_t stream);
hipError_t launch_gdr_recurrent(const GdrCall& c, hipStream_t stream);

// Chunks of 64 tokens (kdn_gdr_chunk.hip).
size_t gdr_chunk_workspace_bytes(bool packed, int N, int B, int T, int H, kdn_dtype_t dtype);
hipError_t launch_gdr_chunked(const GdrCall& c, hipStream_t stream);

// Backward (kdn_gdr_bwd.hip): fwd.o and fwd.S_T are not read. Gradients in the call's type, dS0 float32.
struct GdrGradCall {
    GdrCall fwd;
    const void* dO;
    const float* dS_T;
    void *dq, *dk, *dv, *dalpha, *dbeta;
    float* dS0;
};
size_t gdr_backward_workspace_bytes(bool packed, int N, int B, int T, int H, int dk, int dv,
                                    kdn_dtype_t dtype);
hipError_t launch_gdr_backward(const GdrGradCall& b, hipStream_t stream);

}  // namespace kdn
