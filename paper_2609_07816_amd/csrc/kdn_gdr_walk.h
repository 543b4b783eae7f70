// Gated delta rule over chunks of 64 tokens on gfx950: the walk that carries the state through a
// sequence's chunks (forward, and the backward's first pass).
//
//   X = V - 2^l K S, E = X - W (beta X), U = beta E
//   O = scale (2^l Q S + A U),  S <- 2^l_C S + K^T (2^(l_C - l) U)
//
// A workgroup has 16 NCW value columns of one (sequence, head). Its NCW chain waves carry 16 columns
// each, S in registers, and exchange nothing; NLW loader waves bring the next chunk's K and Q (scaled,
// f16, fragment order; K also transposed), matrices and factors into the other LDS buffer. One barrier
// per chunk. For the backward (BWD) it writes each chunk's entering S and E in place of O.
#pragma once

#include "kdn_gdr_device.h"

namespace kdn {

// What the backward keeps of every chunk and head, beside the records: the state S entering it and
// the adjoint dS of the state leaving it [dk][dvp], its innovations E and the adjoint Y of its writes
// [64][dvp] as f16 (float32 calls: a second plane with the low halves), each 16-column tile scaled by a
// power of two, whose inverses are in `scale` [4][dv / 16]. Columns stand in the order in which a lane
// of a fragment holds them (col_place), dvp = max(dv, 32).
struct GdrKeep {
    _Float16 *S, *dS, *E, *Y;
    float* scale;
};
enum { KEEP_S, KEEP_E, KEEP_DS, KEEP_Y, KEEP_COUNT };

__device__ __forceinline__ int col_place(int n)
{
    return (n & ~31) + ((n & 15) >> 2) * 8 + (n & 3) + ((n >> 4) & 1) * 4;
}

__device__ __forceinline__ float wave_max(float x)  // of values that are not negative
{
    unsigned u = __float_as_uint(x);
    auto step = [&](auto ctrl, auto rows) {
        u = max(u, (unsigned)__builtin_amdgcn_update_dpp(0, (int)u, decltype(ctrl)::value,
                                                         decltype(rows)::value, 0xf, false));
    };
    step(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});
    step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
    return __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)u, 63));
}

// A wave's 16 columns of a kept matrix (NB row blocks of result tiles), and their inverse scale.
template <int P, int DV, int NB>
__device__ __forceinline__ void keep_tile(_Float16* out, float* inv_out, const floatx4* x, int col,
                                          int gq)
{
    constexpr int DVP = DV < 32 ? 32 : DV;
    float m = 0.f, sc, inv;
#pragma unroll
    for (int b = 0; b < NB; ++b) m = max_abs4(m, x[b]);
    pow2_scale(wave_max(m), sc, inv);
    _Float16* at = out + 4 * gq * DVP + col_place(col);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float z = x[b][r] * sc;
            const _Float16 hi = (_Float16)z;
            _Float16* p = at + (16 * b + r) * DVP;
            p[0] = hi;
            if (DV == 16) p[4] = (_Float16)0.f;
            if (P == 2) {
                p[NB * 16 * DVP] = (_Float16)(z - (float)hi);
                if (DV == 16) p[NB * 16 * DVP + 4] = (_Float16)0.f;
            }
        }
    if ((threadIdx.x & 63) == 0) *inv_out = inv;
}

template <class T, int DK, bool BWD>
using WalkLds = ChunkLds<T, DK, true, true, !BWD, false, BWD ? 2 : 2 + gdr_parts<T>()>;

template <class T, int DK, int DV, int NCW, int NLW, bool BWD>
__global__ __launch_bounds__(64 * (NCW + NLW)) void gdr_walk_kernel(const ChunkArgs<T> a,
                                                                    const GdrKeep keep)
{
    using Sh = WalkLds<T, DK, BWD>;
    constexpr int REC = gdr_rec_bytes<T, BWD>();
    constexpr int TILES = DV / (16 * NCW);  // workgroups of a chain
    __shared__ __align__(16) char lds[Sh::NBUF * Sh::BYTES];
    // workgroups of one chain get indexes congruent modulo 8: one XCD, one L2 copy of K, Q and records
    const int chains = a.seq.N * a.H;
    const int chain = blockIdx.x / (8 * TILES) * 8 + blockIdx.x % 8, tile = blockIdx.x / 8 % TILES;
    if (chain >= chains) return;
    const int n = chain / a.H, h = chain % a.H, hk = h / a.rep;
    int t0, t1;
    gdr_span(a.seq, n, t0, t1);
    const int g0 = gdr_first_chunk(a.seq, n, t0);
    const int nch = min((t1 - t0 + GC - 1) / GC, a.maxch - g0);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, gq = lane >> 4, li = lane & 15;
    const char* rec0 = a.rec + ((size_t)g0 * a.H + h) * REC;
    const size_t rstep = (size_t)a.H * REC;

    if (DK == 16) {  // the upper half of the 32 contracted places stays 0
        for (int i = threadIdx.x; i < Sh::NBUF * Sh::BYTES / 16; i += 64 * (NCW + NLW))
            reinterpret_cast<uint4*>(lds)[i] = make_uint4(0, 0, 0, 0);
        __syncthreads();
    }

    if (wave >= NCW) {
        const int tid = threadIdx.x - 64 * NCW;
        Loader<T, DK, Sh, 64 * NLW, 0> ld;
        const size_t step = (size_t)a.Hk * DK;
        auto load = [&](int c) {
            const size_t at = ((size_t)(t0 + c * GC) * a.Hk + hk) * DK;
            ld.load(a.k + at, a.q + at, step, tid, t1 - t0 - c * GC, rec0 + (size_t)c * rstep);
        };
        if (nch > 0) {
            load(0);
            ld.store(lds, tid);
        }
        if (nch > 1) load(1);
        __syncthreads();
        for (int c = 0; c < nch; ++c) {
            if (Sh::NBUF == 1) __syncthreads();  // the chunk's last reads
            if (c + 1 < nch) {
                ld.store(lds + (c + 1) % Sh::NBUF * Sh::BYTES, tid);
                if (c + 2 < nch) load(c + 2);
            }
            __syncthreads();
        }
        return;
    }

    const int col = (tile * NCW + wave) * 16 + li;
    const size_t sbase = ((size_t)n * a.H + h) * DK * DV + (size_t)(4 * gq) * DV + col;
    floatx4 S[Sh::KT];
#pragma unroll
    for (int k = 0; k < Sh::KT; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            S[k][r] = a.S0 ? a.S0[sbase + (size_t)(16 * k + r) * DV] : 0.f;

    const size_t vstep = (size_t)a.H * DV;
    T vn[16];
    auto load_v = [&](int c) {
        load_tile(a.v + ((size_t)(t0 + c * GC) * a.H + h) * DV + col, vstep, gq,
                  min(GC, t1 - t0 - c * GC), vn);
    };
    if (nch > 0) load_v(0);
    __syncthreads();
    for (int c = 0; c < nch; ++c) {
        const char* buf = lds + c % Sh::NBUF * Sh::BYTES;
        const float* fac = reinterpret_cast<const float*>(buf + Sh::O_REC);
        const char* tri = buf + Sh::O_REC + REC_HEAD;
        const int len = min(GC, t1 - t0 - c * GC);
        auto factor = [&](int f, int b) { return ld4(fac + f * GC + 16 * b + 4 * gq); };
        float V[4][4];
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                V[b][r] = 16 * b + 4 * gq + r < len ? to_f32(vn[4 * b + r]) : 0.f;
        if (c + 1 < nch) load_v(c + 1);

        const size_t kept = (size_t)(g0 + c) * a.H + h;
        constexpr int DVP = DV < 32 ? 32 : DV;
        if (BWD)
            keep_tile<Sh::P, DV, Sh::KT>(keep.S + kept * DK * DVP * Sh::P,
                                         keep.scale + (kept * KEEP_COUNT + KEEP_S) * (DV / 16) + col / 16,
                                         S, col, gq);

        // S in halves
        float m = 0.f, sc, s_inv;
#pragma unroll
        for (int k = 0; k < Sh::KT; ++k) m = max_abs4(m, S[k]);
        pow2_scale(column_max(m), sc, s_inv);
        Split sp[Sh::KSTEPS];
#pragma unroll
        for (int s = 0; s < Sh::KSTEPS; ++s)
            sp[s] = split(S[2 * s], Sh::KT > 1 ? S[2 * s + 1] : zero4(), sc);

        // K S and Q S
        floatx4 x[4], o[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            x[b] = zero4();
            o[b] = zero4();
#pragma unroll
            for (int s = 0; s < Sh::KSTEPS; ++s) {
                const half8 kf = frag_ld(buf + Sh::O_K, b * Sh::KSTEPS + s, lane);
                x[b] = mma(kf, sp[s].hi, x[b]);
                x[b] = mma(kf, sp[s].lo, x[b]);
                if (Sh::P == 2)
                    x[b] = mma(frag_ld(buf + Sh::O_K + Sh::RB, b * Sh::KSTEPS + s, lane), sp[s].hi,
                               x[b]);
                if (!BWD) {
                    const half8 qf = frag_ld(buf + Sh::O_Q, b * Sh::KSTEPS + s, lane);
                    o[b] = mma(qf, sp[s].hi, o[b]);
                    if (Sh::P == 2) {
                        o[b] = mma(qf, sp[s].lo, o[b]);
                        o[b] = mma(frag_ld(buf + Sh::O_Q + Sh::RB, b * Sh::KSTEPS + s, lane),
                                   sp[s].hi, o[b]);
                    }
                }
            }
        }
        // X = V - 2^l K S, and beta X in halves
        floatx4 bx[4];
        m = 0.f;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            float g1[4], be[4];
            unpack4(factor(F_G1, b), g1);
            unpack4(factor(F_BE, b), be);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[b][r] = fmaf(-g1[r], x[b][r] * s_inv, V[b][r]);
                bx[b][r] = be[r] * x[b][r];
            }
            m = max_abs4(m, bx[b]);
        }
        float x_inv;
        pow2_scale(column_max(m), sc, x_inv);
        const Split xs[2] = {split(bx[0], bx[1], sc), split(bx[2], bx[3], sc)};
        // E = X - W (beta X), U = beta E
        floatx4 u[4], y[4];
        m = 0.f;
        float mw = 0.f;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            floatx4 d = zero4();
#pragma unroll
            for (int s = 0; s <= b / 2; ++s) {
                const half8 wh = frag_ld(tri, tri_frag(b, s), lane);
                d = mma(wh, xs[s].hi, d);
                d = mma(wh, xs[s].lo, d);
                d = mma(frag_ld(tri, TRI + tri_frag(b, s), lane), xs[s].hi, d);
            }
            float wr[4], w[4], be[4];
            unpack4(factor(F_WR, b), wr);
            unpack4(factor(F_W, b), w);
            unpack4(factor(F_BE, b), be);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[b][r] = fmaf(-wr[r], d[r] * x_inv, x[b][r]);
                u[b][r] = be[r] * x[b][r];
                y[b][r] = w[r] * u[b][r];
            }
            m = max_abs4(m, u[b]);
            mw = max_abs4(mw, y[b]);
        }
        if (BWD)
            keep_tile<Sh::P, DV, 4>(keep.E + kept * GC * DVP * Sh::P,
                                    keep.scale + (kept * KEEP_COUNT + KEEP_E) * (DV / 16) + col / 16, x,
                                    col, gq);
        // S <- 2^l_C S + K^T (2^(l_C - l) U)
        float y_inv;
        pow2_scale(column_max(mw), sc, y_inv);
        const Split ys[2] = {split(y[0], y[1], sc), split(y[2], y[3], sc)};
        const float gc = fac[REC_FACTORS];
#pragma unroll
        for (int k = 0; k < Sh::KT; ++k) {
            floatx4 d = zero4();
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const half8 kf = frag_ld(buf + Sh::O_KT, 2 * k + s, lane);
                d = mma(kf, ys[s].hi, d);
                d = mma(kf, ys[s].lo, d);
                if (Sh::P == 2)
                    d = mma(frag_ld(buf + Sh::O_KT + Sh::CB, 2 * k + s, lane), ys[s].hi, d);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) S[k][r] = fmaf(gc, S[k][r], d[r] * y_inv);
        }
        if (!BWD) {  // O = scale (2^l Q S + A U)
            float u_inv;
            pow2_scale(column_max(m), sc, u_inv);
            const Split us[2] = {split(u[0], u[1], sc), split(u[2], u[3], sc)};
            T* op = a.o + ((size_t)(t0 + c * GC) * a.H + h) * DV + col;
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                floatx4 d = zero4();
#pragma unroll
                for (int s = 0; s <= b / 2; ++s) {
                    const half8 af = frag_ld(tri, 2 * TRI + tri_frag(b, s), lane);
                    d = mma(af, us[s].hi, d);
                    if (Sh::P == 2) {
                        d = mma(af, us[s].lo, d);
                        d = mma(frag_ld(tri, 3 * TRI + tri_frag(b, s), lane), us[s].hi, d);
                    }
                }
                float gv[4], av[4];
                unpack4(factor(F_GQ, b), gv);
                unpack4(factor(F_AR, b), av);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int t = 16 * b + 4 * gq + r;
                    const float z = fmaf(gv[r], o[b][r] * s_inv, av[r] * (d[r] * u_inv));
                    if (t < len) op[(size_t)t * vstep] = from_f32<T>(z);
                }
            }
        }
        if (Sh::NBUF == 1) __syncthreads();
        __syncthreads();
    }
    if (a.S_T)
#pragma unroll
        for (int k = 0; k < Sh::KT; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r) a.S_T[sbase + (size_t)(16 * k + r) * DV] = S[k][r];
}

template <bool BWD, class T, int DK, int DV, int NCW, int NLW>
hipError_t launch_gdr_walk(const ChunkArgs<T>& a, const GdrKeep& keep, hipStream_t stream)
{
    constexpr int TILES = DV / (16 * NCW);
    const unsigned grid = (unsigned)((a.seq.N * a.H + 7) / 8 * 8 * TILES);
    hipLaunchKernelGGL((gdr_walk_kernel<T, DK, DV, NCW, NLW, BWD>), dim3(grid), dim3(64 * (NCW + NLW)), 0,
                       stream, a, keep);
    return hipGetLastError();
}

template <bool BWD, class T, int DK>
hipError_t launch_gdr_walk_dv(const ChunkArgs<T>& a, const GdrKeep& keep, int dv, hipStream_t stream)
{
    switch (dv) {
    case 16: return launch_gdr_walk<BWD, T, DK, 16, 1, 2>(a, keep, stream);
    case 32: return launch_gdr_walk<BWD, T, DK, 32, 2, 2>(a, keep, stream);
    case 64: return launch_gdr_walk<BWD, T, DK, 64, 2, 2>(a, keep, stream);
    case 128: return launch_gdr_walk<BWD, T, DK, 128, 2, 2>(a, keep, stream);
    }
    return hipErrorInvalidValue;
}

template <bool BWD, class T>
hipError_t launch_gdr_walk_dk(const ChunkArgs<T>& a, const GdrKeep& keep, int dk, int dv,
                              hipStream_t stream)
{
    switch (dk) {
    case 16: return launch_gdr_walk_dv<BWD, T, 16>(a, keep, dv, stream);
    case 32: return launch_gdr_walk_dv<BWD, T, 32>(a, keep, dv, stream);
    case 64: return launch_gdr_walk_dv<BWD, T, 64>(a, keep, dv, stream);
    case 128: return launch_gdr_walk_dv<BWD, T, 128>(a, keep, dv, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace kdn
