// Gated delta rule over chunks of 64 tokens on gfx950: the backward.
//
// Per chunk (kdn_gdr_prep.hip's matrices, kdn_gdr_walk.h's S, E and U = beta E; dS the adjoint of the
// state leaving the chunk, dO times the output scale):
//   D = A^T dO + 2^(l_C - l) K dS, Y = D - W^T (beta D) (the adjoint of U), dV = beta Y
//   dS_in = 2^l_C dS + (2^l Q)^T dO - (2^l K)^T dV
//   C = tril(R (dO U^T)), Z = -tril(beta R (Y U^T), -1)   (adjoints of A and of beta M, times R)
//   dQ = 2^l dO S^T + C K
//   dK = -2^l dV S^T + 2^(l_C - l) U dS^T + C^T Q + (Z + Z^T) K
//   dbeta = rowsum(Y E)
//   alpha_j dalpha_j: everything that crosses token j, from a state or write before it to a read, a
//   write's innovation or the state after it: sum over t >= j > s of (C (QK^T) + Z (KK^T))_ts, over t >= j
//   of the rows' S terms, over s < j of the rows' dS terms, and 2^l_C <S, dS>. No term stands in two sums
//   of opposite sign, so that a small alpha keeps the accuracy of its gradient.
// gdr_prep, gdr_walk (which keeps S and E), gdr_reverse (the walk in reverse, which keeps dS and Y and
// writes dV and dS0), gdr_grad (every chunk in parallel: the rest). The chains have float32 accuracy, as in
// the forward; products whose results are rounded to bf16 take operands of 11 bits (float32 calls: halves).
#include "kdn_gdr_walk.h"

namespace kdn {
namespace {

template <class T>
struct GradArgs {
    ChunkArgs<T> c;
    const T* dO;         // or nullptr (0)
    const float* dS_T;   // or nullptr (0)
    T *dq, *dk, *dv, *dalpha, *dbeta;
    float* dS0;  // or nullptr
    GdrKeep keep;
};

// ------------------------------------------------------------------------------------------
// gdr_reverse: as gdr_walk, the chunks in reverse and dS in registers.
// ------------------------------------------------------------------------------------------
template <class T, int DK, int DV, int NCW, int NLW>
__global__ __launch_bounds__(64 * (NCW + NLW)) void gdr_reverse_kernel(const GradArgs<T> ga)
{
    using Sh = ChunkLds<T, DK, true, true, false, true, 4>;
    const ChunkArgs<T>& a = ga.c;
    constexpr int REC = gdr_rec_bytes<T, true>();
    constexpr int TILES = DV / (16 * NCW);
    constexpr int DVP = DV < 32 ? 32 : DV;
    __shared__ __align__(16) char lds[Sh::NBUF * Sh::BYTES];
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
    // the i-th step handles chunk nch - 1 - i
    if (wave >= NCW) {
        const int tid = threadIdx.x - 64 * NCW;
        Loader<T, DK, Sh, 64 * NLW, 2 * TRI_BYTES> ld;
        const size_t step = (size_t)a.Hk * DK;
        auto load = [&](int i) {
            const int c = nch - 1 - i;
            const size_t at = ((size_t)(t0 + c * GC) * a.Hk + hk) * DK;
            ld.load(a.k + at, a.q + at, step, tid, t1 - t0 - c * GC, rec0 + (size_t)c * rstep);
        };
        if (nch > 0) {
            load(0);
            ld.store(lds, tid);
        }
        if (nch > 1) load(1);
        __syncthreads();
        for (int i = 0; i < nch; ++i) {
            if (Sh::NBUF == 1) __syncthreads();  // the chunk's last reads
            if (i + 1 < nch) {
                ld.store(lds + (i + 1) % Sh::NBUF * Sh::BYTES, tid);
                if (i + 2 < nch) load(i + 2);
            }
            __syncthreads();
        }
        return;
    }

    const int col = (tile * NCW + wave) * 16 + li;
    const size_t sbase = ((size_t)n * a.H + h) * DK * DV + (size_t)(4 * gq) * DV + col;
    floatx4 dS[Sh::KT];
#pragma unroll
    for (int k = 0; k < Sh::KT; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            dS[k][r] = ga.dS_T ? ga.dS_T[sbase + (size_t)(16 * k + r) * DV] : 0.f;

    const size_t vstep = (size_t)a.H * DV;
    T on[16];
    auto load_o = [&](int c) {
        if (ga.dO)
            load_tile(ga.dO + ((size_t)(t0 + c * GC) * a.H + h) * DV + col, vstep, gq,
                      min(GC, t1 - t0 - c * GC), on);
        else
#pragma unroll
            for (int i = 0; i < 16; ++i) on[i] = from_f32<T>(0.f);
    };
    if (nch > 0) load_o(nch - 1);
    __syncthreads();
    for (int i = 0; i < nch; ++i) {
        const int c = nch - 1 - i;
        const char* buf = lds + i % Sh::NBUF * Sh::BYTES;
        const float* fac = reinterpret_cast<const float*>(buf + Sh::O_REC);
        const char* tri = buf + Sh::O_REC + REC_HEAD;  // W^T hi, lo, A^T hi, lo
        const int len = min(GC, t1 - t0 - c * GC);
        auto factor = [&](int f, int b, float* x) { unpack4(ld4(fac + f * GC + 16 * b + 4 * gq), x); };
        floatx4 G[4];
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                G[b][r] = 16 * b + 4 * gq + r < len ? to_f32(on[4 * b + r]) : 0.f;
        if (c > 0) load_o(c - 1);
        const size_t kept = (size_t)(g0 + c) * a.H + h;
        float* kscale = ga.keep.scale + kept * KEEP_COUNT * (DV / 16) + col / 16;
        keep_tile<Sh::P, DV, Sh::KT>(ga.keep.dS + kept * DK * DVP * Sh::P, kscale + KEEP_DS * (DV / 16),
                                     dS, col, gq);

        // K dS and A^T dO
        float m = 0.f, sc, s_inv, g_inv;
#pragma unroll
        for (int k = 0; k < Sh::KT; ++k) m = max_abs4(m, dS[k]);
        pow2_scale(column_max(m), sc, s_inv);
        Split sp[Sh::KSTEPS];
#pragma unroll
        for (int s = 0; s < Sh::KSTEPS; ++s)
            sp[s] = split(dS[2 * s], Sh::KT > 1 ? dS[2 * s + 1] : zero4(), sc);
        m = 0.f;
#pragma unroll
        for (int b = 0; b < 4; ++b) m = max_abs4(m, G[b]);
        pow2_scale(column_max(m), sc, g_inv);
        const Split gs[2] = {split(G[0], G[1], sc), split(G[2], G[3], sc)};  // bf16: lo = 0
        floatx4 D[4], bd[4];
        m = 0.f;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            floatx4 x = zero4(), y = zero4();
#pragma unroll
            for (int s = 0; s < Sh::KSTEPS; ++s) {
                const half8 kf = frag_ld(buf + Sh::O_K, b * Sh::KSTEPS + s, lane);
                x = mma(kf, sp[s].hi, x);
                x = mma(kf, sp[s].lo, x);
                if (Sh::P == 2)
                    x = mma(frag_ld(buf + Sh::O_K + Sh::RB, b * Sh::KSTEPS + s, lane), sp[s].hi, x);
            }
#pragma unroll
            for (int s = b / 2; s < 2; ++s) {
                const half8 af = frag_ld(tri, 2 * TRI + tri_frag_t(b, s), lane);
                y = mma(af, gs[s].hi, y);
                if (Sh::P == 2) y = mma(af, gs[s].lo, y);
                y = mma(frag_ld(tri, 3 * TRI + tri_frag_t(b, s), lane), gs[s].hi, y);
            }
            float w[4], ar[4], be[4];
            factor(F_W, b, w);
            factor(F_ATR, b, ar);
            factor(F_BE, b, be);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                D[b][r] = fmaf(w[r], x[r] * s_inv, ar[r] * (y[r] * g_inv));
                bd[b][r] = be[r] * D[b][r];
            }
            m = max_abs4(m, bd[b]);
        }
        // Y = D - W^T (beta D)
        float d_inv;
        pow2_scale(column_max(m), sc, d_inv);
        const Split ds[2] = {split(bd[0], bd[1], sc), split(bd[2], bd[3], sc)};
        floatx4 z1[4], z2[4];
        float m1 = 0.f, m2 = 0.f;
        T* vp = ga.dv + ((size_t)(t0 + c * GC) * a.H + h) * DV + col;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            floatx4 y = zero4();
#pragma unroll
            for (int s = b / 2; s < 2; ++s) {
                const half8 wh = frag_ld(tri, tri_frag_t(b, s), lane);
                y = mma(wh, ds[s].hi, y);
                y = mma(wh, ds[s].lo, y);
                y = mma(frag_ld(tri, TRI + tri_frag_t(b, s), lane), ds[s].hi, y);
            }
            float wr[4], be[4], g1[4], g2[4];
            factor(F_WTR, b, wr);
            factor(F_BE, b, be);
            factor(F_G1, b, g1);
            factor(F_GQ, b, g2);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int t = 16 * b + 4 * gq + r;
                D[b][r] = fmaf(-wr[r], y[r] * d_inv, D[b][r]);
                const float dv = be[r] * D[b][r];
                if (t < len) vp[(size_t)t * vstep] = from_f32<T>(dv);
                z1[b][r] = g1[r] * dv;
                z2[b][r] = g2[r] * G[b][r];
            }
            m1 = max_abs4(m1, z1[b]);
            m2 = max_abs4(m2, z2[b]);
        }
        keep_tile<Sh::P, DV, 4>(ga.keep.Y + kept * GC * DVP * Sh::P, kscale + KEEP_Y * (DV / 16), D, col,
                                gq);
        // dS <- 2^l_C dS + (2^l Q)^T dO - (2^l K)^T dV
        float inv1, inv2, sc2;
        pow2_scale(column_max(m1), sc, inv1);
        pow2_scale(column_max(m2), sc2, inv2);
        const Split s1[2] = {split(z1[0], z1[1], sc), split(z1[2], z1[3], sc)};
        const Split s2[2] = {split(z2[0], z2[1], sc2), split(z2[2], z2[3], sc2)};
        const float gc = fac[REC_FACTORS];
#pragma unroll
        for (int k = 0; k < Sh::KT; ++k) {
            floatx4 x = zero4(), y = zero4();
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const half8 kf = frag_ld(buf + Sh::O_KT, 2 * k + s, lane);
                x = mma(kf, s1[s].hi, x);
                x = mma(kf, s1[s].lo, x);
                const half8 qf = frag_ld(buf + Sh::O_QT, 2 * k + s, lane);
                y = mma(qf, s2[s].hi, y);
                y = mma(qf, s2[s].lo, y);
                if (Sh::P == 2) {
                    x = mma(frag_ld(buf + Sh::O_KT + Sh::CB, 2 * k + s, lane), s1[s].hi, x);
                    y = mma(frag_ld(buf + Sh::O_QT + Sh::CB, 2 * k + s, lane), s2[s].hi, y);
                }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r)
                dS[k][r] = fmaf(gc, dS[k][r], fmaf(y[r], inv2, -(x[r] * inv1)));
        }
        if (Sh::NBUF == 1) __syncthreads();
        __syncthreads();
    }
    if (ga.dS0)
#pragma unroll
        for (int k = 0; k < Sh::KT; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r) ga.dS0[sbase + (size_t)(16 * k + r) * DV] = dS[k][r];
}

// ------------------------------------------------------------------------------------------
// gdr_grad: a workgroup per (chunk, key head), wave w has tokens 16w .. 16w+15; the value heads of the
// key head one after another, dQ and dK summed in registers in that order.
// ------------------------------------------------------------------------------------------
constexpr int CP = 68;  // floats of a row of the 64 x 64 matrices in LDS

__device__ __forceinline__ float pow2_inverse(float x)  // of a power of two in [2^-126, 2^126]
{
    return __uint_as_float(0x7f000000u - __float_as_uint(x));
}

// A fragment's slots of the two 16-value blocks times f0 and f1 (powers of two, at most 1).
__device__ __forceinline__ half8 fold(half8 x, float f0, float f1)
{
    const _Float16 a = (_Float16)f0, b = (_Float16)f1;
    return x * half8{a, a, a, a, b, b, b, b};
}

template <int P, int N>
struct Operand {
    half8 hi[N], lo[P == 2 ? N : 1];
};

// acc + A B with the parts that count
template <int P>
__device__ __forceinline__ floatx4 mma_parts(half8 ah, half8 al, half8 bh, half8 bl, floatx4 acc)
{
    acc = mma(ah, bh, acc);
    if (P == 2) {
        acc = mma(ah, bl, acc);
        acc = mma(al, bh, acc);
    }
    return acc;
}

template <class T, int DK, int DV>
__global__ __launch_bounds__(256, sizeof(T) == 4 ? 1 : 2) void gdr_grad_kernel(const GradArgs<T> ga)
{
    using Sh = ChunkLds<T, DK, false, true, false, true, -1>;
    using Fr = Frag<T, DK>;
    using V = typename Fr::V;
    constexpr int P = Sh::P, REC = gdr_rec_bytes<T, true>();
    constexpr int DVP = DV < 32 ? 32 : DV, VS = DVP / 32, NB = DV / 16;
    const ChunkArgs<T>& a = ga.c;
    __shared__ __align__(16) char lds[Sh::BYTES];
    __shared__ __align__(16) float sC[GC * CP];  // C on and below the diagonal, Z^T above it
    __shared__ __align__(16) float sP[GC * CP];  // the pairs' share of the log-decay's gradient
    __shared__ double s_l[GC];
    __shared__ float s_be[GC], s_ri[GC], s_reads[GC], s_writes[GC], s_dot[4];
    __shared__ float s_ic[GC], s_it[GC], s_iz[GC];  // inverse scales of the rows of C, C^T, Z + Z^T
    const int g = blockIdx.x / a.Hk, hk = blockIdx.x % a.Hk;
    int n, c0, c1;
    if (!gdr_locate(a.seq, g, n, c0, c1)) return;
    const int len = c1 - c0, tid = threadIdx.x, w = tid >> 6, lane = tid & 63, gq = lane >> 4,
              li = lane & 15, row = 16 * w + li;

    const T* kbase = a.k + ((size_t)c0 * a.Hk + hk) * DK;
    const T* qbase = a.q + ((size_t)c0 * a.Hk + hk) * DK;
    const size_t kstep = (size_t)a.Hk * DK;
    const char* rec = a.rec + ((size_t)g * a.H + (size_t)hk * a.rep) * REC;
    {
        Loader<T, DK, Sh, 256, 0> ld;
        ld.load(kbase, qbase, kstep, tid, len, rec);
        ld.store(lds, tid);
    }
    auto load_rows = [&](const T* base, int b, V* f) {
        const int t = 16 * b + li;
#pragma unroll
        for (int s = 0; s < Fr::NS; ++s) {
            f[s] = V{};
            if (t < len) f[s] = Fr::ld(base + t * kstep + gq * (Fr::KF / 4) + s * Fr::KF);
        }
    };
    floatx4 dq[Sh::KT], dk[Sh::KT];
#pragma unroll
    for (int k = 0; k < Sh::KT; ++k) dq[k] = dk[k] = zero4();

#pragma unroll 1
    for (int hv = 0; hv < a.rep; ++hv) {
        const int h = hk * a.rep + hv;
        const size_t kept = (size_t)g * a.H + h;
        rec = a.rec + kept * REC;
        const float* fac = reinterpret_cast<const float*>(rec);
        const float* ksc = ga.keep.scale + kept * KEEP_COUNT * NB;
        const float gamma = fac[REC_FACTORS];
        if (tid < GC) {
            s_l[tid] = reinterpret_cast<const double*>(fac + F_L * GC)[tid];
            s_be[tid] = fac[F_BE * GC + tid];
        }
        const _Float16* E = ga.keep.E + kept * GC * DVP * P;
        const _Float16* Y = ga.keep.Y + kept * GC * DVP * P;
        const _Float16* S = ga.keep.S + kept * DK * DVP * P;
        const _Float16* dS = ga.keep.dS + kept * DK * DVP * P;
        // this wave's rows of dO (scaled by row; the inverse scales to s_ri), and of E or Y
        auto load_dO = [&]() {
            Operand<P, VS> go;
            float x[VS][8], m = 0.f;
            const T* p = ga.dO + ((size_t)(c0 + row) * a.H + h) * DV + 4 * gq;
#pragma unroll
            for (int s = 0; s < VS; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[s][e] = 0.f;
                    if (ga.dO && row < len && (DV >= 32 || e < 4))
                        x[s][e] = to_f32(p[32 * s + (e & 3) + 16 * (e >> 2)]);
                    m = fmaxf(m, fabsf(x[s][e]));
                }
            float sc, inv;
            pow2_scale(column_max(m), sc, inv);
#pragma unroll
            for (int s = 0; s < VS; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float z = x[s][e] * sc;
                    go.hi[s][e] = (_Float16)z;
                    if (P == 2) go.lo[s][e] = (_Float16)(z - (float)go.hi[s][e]);
                }
            if (gq == 0) s_ri[row] = inv;
            return go;
        };
        auto kept_row = [&](const _Float16* x, int r, int s) {
            return *reinterpret_cast<const half8*>(x + r * DVP + 32 * s + 8 * gq);
        };
        auto load_kept = [&](const _Float16* x) {
            Operand<P, VS> y;
#pragma unroll
            for (int s = 0; s < VS; ++s) {
                y.hi[s] = kept_row(x, row, s);
                if (P == 2) y.lo[s] = kept_row(x + GC * DVP, row, s);
            }
            return y;
        };
        // the tiles' scales, and of the products over the value columns: the largest, and the others
        // over it (folded into the A side)
        float iS[2 * VS], iE[2 * VS], iD[2 * VS], iY[2 * VS];
#pragma unroll
        for (int j = 0; j < 2 * VS; ++j) {
            iS[j] = j < NB ? ksc[KEEP_S * NB + j] : 0.f;
            iE[j] = j < NB ? ksc[KEEP_E * NB + j] : 0.f;
            iD[j] = j < NB ? ksc[KEEP_DS * NB + j] : 0.f;
            iY[j] = j < NB ? ksc[KEEP_Y * NB + j] : 0.f;
        }
        auto operand = [&](const Operand<P, VS>& x, const float* f1, const float* f2, float& top) {
            Operand<P, VS> y;
            float f[2 * VS];
            top = 0x1p-126f;
#pragma unroll
            for (int j = 0; j < 2 * VS; ++j) {
                f[j] = f2 ? f1[j] * f2[j] : f1[j];
                top = fmaxf(top, f[j]);
            }
            const float r = pow2_inverse(top);
#pragma unroll
            for (int s = 0; s < VS; ++s) {
                y.hi[s] = fold(x.hi[s], f[2 * s] * r, f[2 * s + 1] * r);
                if (P == 2) y.lo[s] = fold(x.lo[s], f[2 * s] * r, f[2 * s + 1] * r);
            }
            return y;
        };
        // dbeta = rowsum(Y E); the A sides of the 64 x 64 products
        float top1, top2;
        Operand<P, VS> goE, yeE;
        {
            const Operand<P, VS> ye = load_kept(Y), ee = load_kept(E);
            float x = 0.f;
#pragma unroll
            for (int s = 0; s < VS; ++s) {
                float y0 = 0.f, y1 = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float p = (float)ye.hi[s][e], q = (float)ee.hi[s][e];
                    if (P == 2) {
                        p += (float)ye.lo[s][e];
                        q += (float)ee.lo[s][e];
                    }
                    (e < 4 ? y0 : y1) += p * q;
                }
                x += y0 * iY[2 * s] * iE[2 * s] + y1 * iY[2 * s + 1] * iE[2 * s + 1];
            }
            x = column_sum(x);
            if (gq == 0 && row < len) ga.dbeta[(size_t)(c0 + row) * a.H + h] = from_f32<T>(x);
            goE = operand(load_dO(), iE, nullptr, top1);
            yeE = operand(ye, iY, iE, top2);
        }
        __syncthreads();  // s_l, s_be, s_ri (and the K, Q fragments)

        // C, Z and the pairs' share of the log-decay's gradient
        {
            V fk[Fr::NS], fq[Fr::NS];
            load_rows(kbase, w, fk);
            load_rows(qbase, w, fq);
            double lr[4];
            float br[4], ri[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                lr[r] = s_l[16 * w + 4 * gq + r];
                br[r] = s_be[16 * w + 4 * gq + r];
                ri[r] = s_ri[16 * w + 4 * gq + r];
            }
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
                const int s = 16 * c + li;
                if (c > w) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) sP[(16 * w + 4 * gq + r) * CP + s] = 0.f;
                    continue;
                }
                V fc[Fr::NS];
                load_rows(kbase, c, fc);
                floatx4 kk = zero4(), qk = zero4(), d1 = zero4(), d2 = zero4();
#pragma unroll
                for (int i = 0; i < Fr::NS; ++i) {
                    kk = Fr::mma(kk, fk[i], fc[i]);
                    qk = Fr::mma(qk, fq[i], fc[i]);
                }
#pragma unroll
                for (int i = 0; i < VS; ++i) {
                    const half8 eh = kept_row(E, s, i);
                    half8 el = eh;
                    if (P == 2) el = kept_row(E + GC * DVP, s, i);
                    d1 = mma_parts<P>(goE.hi[i], goE.lo[P == 2 ? i : 0], eh, el, d1);
                    d2 = mma_parts<P>(yeE.hi[i], yeE.lo[P == 2 ? i : 0], eh, el, d2);
                }
                const double ls = s_l[s];
                const float bs = s_be[s];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int t = 16 * w + 4 * gq + r;
                    const float rho = t >= s ? bs * __builtin_amdgcn_exp2f((float)(lr[r] - ls)) : 0.f;
                    const float cc = t >= s ? a.scale * rho * (d1[r] * top1 * ri[r]) : 0.f;
                    const float zz = t > s ? -br[r] * rho * (d2[r] * top2) : 0.f;
                    if (t >= s) sC[t * CP + s] = cc;
                    if (t > s) sC[s * CP + t] = zz;
                    sP[t * CP + s] = cc * qk[r] + zz * kk[r];
                }
            }
        }
        __syncthreads();
        // C's rows, its columns and the rows of Z + Z^T as operands, over the scales of the K or Q rows
        // that they meet
        Operand<P, 2> opC, opT, opZ;
        {
            float x[3][2][8], m[3] = {0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int j = 32 * s + 4 * gq + (e & 3) + 16 * (e >> 2);
                    const float ki = pow2_inverse(fac[F_KS * GC + j]), qi = pow2_inverse(fac[F_QS * GC + j]);
                    const float y = sC[row * CP + j], z = sC[j * CP + row];
                    x[0][s][e] = j <= row ? y * ki : 0.f;
                    x[1][s][e] = j >= row ? z * qi : 0.f;
                    x[2][s][e] = j < row ? z * ki : j > row ? y * ki : 0.f;
#pragma unroll
                    for (int i = 0; i < 3; ++i) m[i] = fmaxf(m[i], fabsf(x[i][s][e]));
                }
            float sc[3], inv[3];
#pragma unroll
            for (int i = 0; i < 3; ++i) pow2_scale(column_max(m[i]), sc[i], inv[i]);
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float y0 = x[0][s][e] * sc[0], y1 = x[1][s][e] * sc[1], y2 = x[2][s][e] * sc[2];
                    opC.hi[s][e] = (_Float16)y0;
                    opT.hi[s][e] = (_Float16)y1;
                    opZ.hi[s][e] = (_Float16)y2;
                    if (P == 2) {
                        opC.lo[s][e] = (_Float16)(y0 - (float)opC.hi[s][e]);
                        opT.lo[s][e] = (_Float16)(y1 - (float)opT.hi[s][e]);
                        opZ.lo[s][e] = (_Float16)(y2 - (float)opZ.hi[s][e]);
                    }
                }
            if (gq == 0) {
                s_ic[row] = inv[0];
                s_it[row] = inv[1];
                s_iz[row] = inv[2];
            }
        }
        wave_lds_fence();

        // products over the value columns, and the small ones, per 16 key channels
        float topS, topY, topD;
        const Operand<P, VS> goS = operand(load_dO(), iS, nullptr, topS),
                             yeS = operand(load_kept(Y), iY, iS, topY),
                             eeD = operand(load_kept(E), iE, iD, topD);
        float rq[4], rk[4], rt[4], ic[4], it[4], iz[4], qi[4], ki[4];
        float reads[4] = {0.f, 0.f, 0.f, 0.f}, writes[4] = {0.f, 0.f, 0.f, 0.f}, dot = 0.f;
        const double l_end = s_l[GC - 1];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int t = 16 * w + 4 * gq + r;
            const float dec = __builtin_amdgcn_exp2f((float)s_l[t]);
            rq[r] = a.scale * dec * (s_ri[t] * topS);
            rk[r] = -dec * s_be[t] * topY;
            rt[r] = __builtin_amdgcn_exp2f((float)(l_end - s_l[t])) * s_be[t] * topD;
            ic[r] = s_ic[t];
            it[r] = s_it[t];
            iz[r] = s_iz[t];
            qi[r] = pow2_inverse(fac[F_QS * GC + t]);
            ki[r] = pow2_inverse(fac[F_KS * GC + t]);
        }
#pragma unroll
        for (int k = 0; k < Sh::KT; ++k) {
            floatx4 p1 = zero4(), p2 = zero4(), p3 = zero4();
#pragma unroll
            for (int s = 0; s < VS; ++s) {
                const half8 sh = kept_row(S, 16 * k + li, s), dh = kept_row(dS, 16 * k + li, s);
                half8 sl = sh, dl = dh;
                if (P == 2) {
                    sl = kept_row(S + DK * DVP, 16 * k + li, s);
                    dl = kept_row(dS + DK * DVP, 16 * k + li, s);
                }
                p1 = mma_parts<P>(goS.hi[s], goS.lo[P == 2 ? s : 0], sh, sl, p1);
                p2 = mma_parts<P>(yeS.hi[s], yeS.lo[P == 2 ? s : 0], sh, sl, p2);
                p3 = mma_parts<P>(eeD.hi[s], eeD.lo[P == 2 ? s : 0], dh, dl, p3);
                if (k % 4 == w) {  // <S, dS>
                    float y0 = 0.f, y1 = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float x = (float)sh[e], y = (float)dh[e];
                        if (P == 2) {
                            x += (float)sl[e];
                            y += (float)dl[e];
                        }
                        (e < 4 ? y0 : y1) += x * y;
                    }
                    dot += y0 * iS[2 * s] * iD[2 * s] + y1 * iS[2 * s + 1] * iD[2 * s + 1];
                }
            }
            floatx4 a1 = zero4(), a2 = zero4(), a3 = zero4();
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const half8 kh = frag_ld(lds + Sh::O_KT, 2 * k + s, lane);
                const half8 qh = frag_ld(lds + Sh::O_QT, 2 * k + s, lane);
                half8 kl = kh, ql = qh;
                if (P == 2) {
                    kl = frag_ld(lds + Sh::O_KT + Sh::CB, 2 * k + s, lane);
                    ql = frag_ld(lds + Sh::O_QT + Sh::CB, 2 * k + s, lane);
                }
                if (s <= w / 2) a1 = mma_parts<P>(opC.hi[s], opC.lo[P == 2 ? s : 0], kh, kl, a1);
                if (s >= w / 2) a2 = mma_parts<P>(opT.hi[s], opT.lo[P == 2 ? s : 0], qh, ql, a2);
                a3 = mma_parts<P>(opZ.hi[s], opZ.lo[P == 2 ? s : 0], kh, kl, a3);
            }
            // q and k of the result tile's places: four tokens of a channel
            const int at = frag_at(16 * k + li, 16 * w + 4 * gq, 2) * 2;
            const half4 qh = *reinterpret_cast<const half4*>(lds + Sh::O_QT + at);
            const half4 kh = *reinterpret_cast<const half4*>(lds + Sh::O_KT + at);
            half4 ql = qh, kl = kh;
            if (P == 2) {
                ql = *reinterpret_cast<const half4*>(lds + Sh::O_QT + Sh::CB + at);
                kl = *reinterpret_cast<const half4*>(lds + Sh::O_KT + Sh::CB + at);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float qv = ((float)qh[r] + (P == 2 ? (float)ql[r] : 0.f)) * qi[r];
                const float kv = ((float)kh[r] + (P == 2 ? (float)kl[r] : 0.f)) * ki[r];
                const float x1 = rq[r] * p1[r], x2 = rk[r] * p2[r], x3 = rt[r] * p3[r];
                reads[r] += qv * x1 + kv * x2;
                writes[r] += kv * x3;
                dq[k][r] += x1 + a1[r] * ic[r];
                dk[k][r] += (x2 + x3) + (a2[r] * it[r] + a3[r] * iz[r]);
            }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float x = row16_sum(reads[r]), y = row16_sum(writes[r]);
            if (li == 0) {
                s_reads[16 * w + 4 * gq + r] = x;
                s_writes[16 * w + 4 * gq + r] = y;
            }
        }
        dot = wave_sum(dot);
        if (lane == 0) s_dot[w] = dot;
        if (tid < GC) {  // sums along P's rows, of what stands before each place
            float f = 0.f;
            for (int s = 0; s < GC; ++s) {
                const float x = sP[tid * CP + s];
                sP[tid * CP + s] = f;
                f += x;
            }
        }
        __syncthreads();
        if (w == 0) {  // lane = token
            float after = s_reads[lane], before = s_writes[lane];
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const float x = __shfl_down(after, off, 64), y = __shfl_up(before, off, 64);
                if (lane + off < 64) after += x;
                if (lane >= off) before += y;
            }
            before = __shfl_up(before, 1, 64);  // of the tokens before this one
            if (lane == 0) before = 0.f;
            float cross = 0.f;  // down the columns, from the diagonal
            for (int t = 0; t < GC; ++t) cross += t >= lane ? sP[t * CP + lane] : 0.f;
            const float whole = gamma * ((s_dot[0] + s_dot[1]) + (s_dot[2] + s_dot[3]));
            const float dlog = cross + after + before + whole;
            if (lane < len) {
                const size_t at = (size_t)(c0 + lane) * a.H + h;
                ga.dalpha[at] = from_f32<T>(dlog / fmaxf(to_f32(a.alpha[at]), 0x1p-100f));
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < Sh::KT; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int t = 16 * w + 4 * gq + r;
            if (t < len) {
                const size_t at = ((size_t)(c0 + t) * a.Hk + hk) * DK + 16 * k + li;
                ga.dq[at] = from_f32<T>(dq[k][r]);
                ga.dk[at] = from_f32<T>(dk[k][r]);
            }
        }
}

template <class T, int DK, int DV, int NCW, int NLW>
hipError_t launch_rest(const GradArgs<T>& ga, hipStream_t stream)
{
    const ChunkArgs<T>& a = ga.c;
    constexpr int TILES = DV / (16 * NCW);
    const unsigned grid = (unsigned)((a.seq.N * a.H + 7) / 8 * 8 * TILES);
    hipLaunchKernelGGL((gdr_reverse_kernel<T, DK, DV, NCW, NLW>), dim3(grid), dim3(64 * (NCW + NLW)), 0,
                       stream, ga);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((gdr_grad_kernel<T, DK, DV>), dim3((unsigned)(a.maxch * a.Hk)), dim3(256), 0,
                       stream, ga);
    return hipGetLastError();
}

template <class T, int DK>
hipError_t launch_dv(const GradArgs<T>& ga, int dv, hipStream_t stream)
{
    switch (dv) {
    case 16: return launch_rest<T, DK, 16, 1, 2>(ga, stream);
    case 32: return launch_rest<T, DK, 32, 2, 2>(ga, stream);
    case 64: return launch_rest<T, DK, 64, 2, 2>(ga, stream);
    case 128: return launch_rest<T, DK, 128, 2, 2>(ga, stream);
    }
    return hipErrorInvalidValue;
}

// Parts of the workspace, each a multiple of 256 bytes.
struct Layout {
    size_t S, dS, E, Y, scale, total;
};
template <class T>
Layout layout(size_t units, int dk, int dv)
{
    const size_t dvp = dv < 32 ? 32 : dv, es = 2 * gdr_parts<T>();
    Layout l;
    l.S = al256(units * gdr_rec_bytes<T, true>());
    l.dS = l.S + al256(units * dk * dvp * es);
    l.E = l.dS + al256(units * dk * dvp * es);
    l.Y = l.E + al256(units * GC * dvp * es);
    l.scale = l.Y + al256(units * GC * dvp * es);
    l.total = l.scale + al256(units * KEEP_COUNT * (dv / 16) * 4);
    return l;
}

template <class T>
hipError_t launch_t(const GdrGradCall& b, hipStream_t stream)
{
    const GdrCall& c = b.fwd;
    const SeqArgs& s = c.sa;
    const int maxch = gdr_max_chunks(s.cu_seqlens != nullptr, s.N, s.T, s.B * s.T);
    const Layout l = layout<T>((size_t)maxch * s.H, c.dk, c.dv);
    char* ws = (char*)c.workspace;
    const GdrKeep keep = {(_Float16*)(ws + l.S), (_Float16*)(ws + l.dS), (_Float16*)(ws + l.E),
                          (_Float16*)(ws + l.Y), (float*)(ws + l.scale)};
    const ChunkArgs<T> a = {(const T*)c.q, (const T*)c.k, (const T*)c.v, (const T*)c.alpha,
                            (const T*)c.beta, c.S0, nullptr, nullptr,
                            {s.cu_seqlens, s.N, s.T, s.B * s.T}, s.H, c.Hk, s.H / c.Hk, maxch, c.scale,
                            ws};
    const GradArgs<T> ga = {a, (const T*)b.dO, b.dS_T, (T*)b.dq, (T*)b.dk, (T*)b.dv, (T*)b.dalpha,
                            (T*)b.dbeta, b.dS0, keep};
    hipError_t e = launch_gdr_prep(a, c.dk, true, stream);
    if (e == hipSuccess) e = launch_gdr_walk_dk<true>(a, keep, c.dk, c.dv, stream);
    if (e != hipSuccess) return e;
    switch (c.dk) {
    case 16: return launch_dv<T, 16>(ga, c.dv, stream);
    case 32: return launch_dv<T, 32>(ga, c.dv, stream);
    case 64: return launch_dv<T, 64>(ga, c.dv, stream);
    case 128: return launch_dv<T, 128>(ga, c.dv, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace

size_t gdr_backward_workspace_bytes(bool packed, int N, int B, int T, int H, int dk, int dv,
                                    kdn_dtype_t dtype)
{
    const size_t units = (size_t)gdr_max_chunks(packed, N, T, B * T) * H;
    return dtype == KDN_F32 ? layout<float>(units, dk, dv).total : layout<bf16>(units, dk, dv).total;
}

hipError_t launch_gdr_backward(const GdrGradCall& b, hipStream_t stream)
{
    return b.fwd.dtype == KDN_F32 ? launch_t<float>(b, stream) : launch_t<bf16>(b, stream);
}

}  // namespace kdn
