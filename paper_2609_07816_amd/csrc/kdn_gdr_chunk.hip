// Gated delta rule over chunks of 64 tokens on gfx950: the forward of long sequences. Every chunk's
// matrices in parallel (kdn_gdr_prep.hip), then the walk through the chunks (kdn_gdr_walk.h).
#include "kdn_gdr_walk.h"

namespace kdn {
namespace {

template <class T>
hipError_t launch_t(const GdrCall& c, hipStream_t stream)
{
    const SeqArgs& s = c.sa;
    const ChunkArgs<T> a = {(const T*)c.q, (const T*)c.k, (const T*)c.v, (const T*)c.alpha,
                            (const T*)c.beta, c.S0, (T*)c.o, c.S_T,
                            {s.cu_seqlens, s.N, s.T, s.B * s.T}, s.H, c.Hk, s.H / c.Hk,
                            gdr_max_chunks(s.cu_seqlens != nullptr, s.N, s.T, s.B * s.T), c.scale,
                            (char*)c.workspace};
    const hipError_t e = launch_gdr_prep(a, c.dk, false, stream);
    return e != hipSuccess ? e : launch_gdr_walk_dk(a, c.dk, c.dv, stream);
}

}  // namespace

size_t gdr_chunk_workspace_bytes(bool packed, int N, int B, int T, int H, kdn_dtype_t dtype)
{
    return (size_t)gdr_max_chunks(packed, N, T, B * T) * H *
           (dtype == KDN_F32 ? gdr_rec_bytes<float, false>() : gdr_rec_bytes<bf16, false>());
}

hipError_t launch_gdr_chunked(const GdrCall& c, hipStream_t stream)
{
    return c.dtype == KDN_F32 ? launch_t<float>(c, stream) : launch_t<bf16>(c, stream);
}

}  // namespace kdn
