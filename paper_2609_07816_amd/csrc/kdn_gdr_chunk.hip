// Gated delta rule over chunks of 64 tokens on gfx950: the forward of long sequences.
//
// With l_t the cumulative log2 decay inside a chunk, R_ts = 2^(l_t - l_s), and S the state entering it:
//   L = tril(beta R (K K^T), -1), N = (I + L)^-1 - I, A = tril(R (Q K^T))
//   X = beta (V - 2^l K S), U = X + N X
//   O = scale (2^l Q S + A U),  S <- 2^l_C S + K^T (2^(l_C - l) U)
// gdr_prep (one workgroup per chunk and head, all in parallel) makes N and A; gdr_walk carries S
// through a sequence's chunks. Numbers and layouts: kdn_gdr_device.h.
#include "kdn_gdr_device.h"

namespace kdn {
namespace {

template <class T>
struct ChunkArgs {
    const T *q, *k, *v, *alpha, *beta;
    const float* S0;
    T* o;
    float* S_T;
    GdrSeq seq;
    int H, Hk, rep, maxch;
    float scale;
    char* rec;
};

// ------------------------------------------------------------------------------------------
// gdr_prep: wave w has rows 16w .. 16w+15 of the chunk. Products of the inputs as they are stored
// (bf16 or float32 instructions, exact operands), the decay ratios from float64 cumulative logarithms
// (a difference of two sums has the error of the difference), the inverse in float32: the diagonal
// 16 x 16 blocks by substitution (lane = column), the others by block products
// T_bc = -T_bb sum_m L_bm T_mc, wave = block column.
// ------------------------------------------------------------------------------------------
constexpr int LP = 20;  // floats of a tile's row in LDS
constexpr int MP = 68;  // floats of a matrix row in LDS

__device__ __forceinline__ float4 ld4(const float* p) { return *reinterpret_cast<const float4*>(p); }

template <class T, int DK>
__global__ __launch_bounds__(256) void gdr_prep_kernel(const ChunkArgs<T> a)
{
    using Fr = Frag<T, DK>;
    using V = typename Fr::V;
    __shared__ float sL[6][16 * LP];   // L's blocks below the diagonal ones: (b, c) at b (b - 1) / 2 + c
    __shared__ float sD[4][16 * LP];   // the diagonal blocks, then their inverses
    __shared__ float sM[GC * MP];      // A, then N
    __shared__ double s_l[GC];
    __shared__ float s_be[GC];
    const int g = blockIdx.x / a.H, h = blockIdx.x % a.H;
    int n, c0, c1;
    if (!gdr_locate(a.seq, g, n, c0, c1)) return;  // uniform across the workgroup
    const int len = c1 - c0;
    const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63, gq = lane >> 4, li = lane & 15;
    const int hk = h / a.rep;

    // cumulative decays: lane = token, in every wave (the values of tokens past the end change nothing)
    double l = 0.0;
    float be = 0.f;
    if (lane < len) {
        const size_t at = (size_t)(c0 + lane) * a.H + h;
        // a gate of 0 counts as 2^-100: what it lets through is lost against anything beside it
        l = log2((double)fmaxf(to_f32(a.alpha[at]), 0x1p-100f));
        be = to_f32(a.beta[at]);
    }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const double y = __shfl_up(l, off, 64);
        if (lane >= off) l += y;
    }
    if (w == 0) {
        s_l[lane] = l;
        s_be[lane] = be;
    }
    const double l_end = __shfl(l, 63, 64);

    // operands: this wave's rows of K and Q
    const T* kbase = a.k + ((size_t)c0 * a.Hk + hk) * DK + gq * (Fr::KF / 4);
    const T* qbase = a.q + ((size_t)c0 * a.Hk + hk) * DK + gq * (Fr::KF / 4);
    const size_t step = (size_t)a.Hk * DK;
    auto load_rows = [&](const T* base, int b, V* f) {
        const int t = 16 * b + li;
#pragma unroll
        for (int s = 0; s < Fr::NS; ++s) {
            f[s] = V{};
            if (t < len) f[s] = Fr::ld(base + t * step + s * Fr::KF);
        }
    };
    V fk[Fr::NS], fq[Fr::NS];
    load_rows(kbase, w, fk);
    load_rows(qbase, w, fq);
    // power-of-two scales of the rows
    float mk = 0.f, mq = 0.f;
#pragma unroll
    for (int s = 0; s < Fr::NS; ++s) {
        constexpr int E = Fr::KF / 4;
        T x[E], y[E];
        __builtin_memcpy(x, &fk[s], sizeof(V));
        __builtin_memcpy(y, &fq[s], sizeof(V));
#pragma unroll
        for (int e = 0; e < E; ++e) {
            mk = fmaxf(mk, fabsf(to_f32(x[e])));
            mq = fmaxf(mq, fabsf(to_f32(y[e])));
        }
    }
    mk = column_max(mk);
    mq = column_max(mq);
    __syncthreads();

    // products with the blocks c <= w; result lane (gq, li): rows 16w + 4gq + r, column 16c + li
    double lr[4];
    float br[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        lr[r] = s_l[16 * w + 4 * gq + r];
        br[r] = s_be[16 * w + 4 * gq + r];
    }
    for (int c = 0; c < 4; ++c) {
        float* am = sM + 16 * c + li;
        if (c > w) {  // above the diagonal
#pragma unroll
            for (int r = 0; r < 4; ++r) am[(16 * w + 4 * gq + r) * MP] = 0.f;
            continue;
        }
        V fc[Fr::NS];
        load_rows(kbase, c, fc);
        floatx4 kk = zero4(), qk = zero4();
#pragma unroll
        for (int s = 0; s < Fr::NS; ++s) {
            kk = Fr::mma(kk, fk[s], fc[s]);
            qk = Fr::mma(qk, fq[s], fc[s]);
        }
        const double ls = s_l[16 * c + li];
        float* lt = c == w ? sD[w] : sL[w * (w - 1) / 2 + c];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int t = 16 * w + 4 * gq + r, s = 16 * c + li;
            const float rho = t >= s ? __builtin_amdgcn_exp2f((float)(lr[r] - ls)) : 0.f;
            lt[(4 * gq + r) * LP + li] = t > s ? br[r] * rho * kk[r] : 0.f;
            am[t * MP] = t >= s ? rho * qk[r] : 0.f;
        }
    }
    wave_lds_fence();
    // inverse of this wave's diagonal block: column li by substitution
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        float y = i == li ? 1.f : 0.f;
#pragma unroll
        for (int j4 = 0; j4 < i; j4 += 4) {
            const float4 row = ld4(sD[w] + i * LP + j4);
            y = fmaf(-row.x, x[j4], y);
            if (j4 + 1 < i) y = fmaf(-row.y, x[j4 + 1], y);
            if (j4 + 2 < i) y = fmaf(-row.z, x[j4 + 2], y);
            if (j4 + 3 < i) y = fmaf(-row.w, x[j4 + 3], y);
        }
        x[i] = y;
    }
    wave_lds_fence();
    if (gq == 0)
#pragma unroll
        for (int i = 0; i < 16; ++i) sD[w][i * LP + li] = x[i];
    __syncthreads();

    // A's rows to the record: thread = (row, 16 columns)
    char* rec = a.rec + ((size_t)g * a.H + h) * gdr_rec_bytes<T>();
    float* fac = reinterpret_cast<float*>(rec);
    _Float16* frag = reinterpret_cast<_Float16*>(rec + REC_HEAD);
    const int row = tid >> 2, quarter = tid & 3;
    auto write_rows = [&](_Float16* hi, _Float16* lo) -> float {  // returns the row's inverse scale
        float4 y[4];
        float m = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            y[j] = ld4(sM + row * MP + 16 * quarter + 4 * j);
            m = fmaxf(m, fmaxf(fmaxf(fabsf(y[j].x), fabsf(y[j].y)), fmaxf(fabsf(y[j].z), fabsf(y[j].w))));
        }
        m = fmaxf(m, __shfl_xor(m, 1, 64));
        m = fmaxf(m, __shfl_xor(m, 2, 64));
        float sc, inv;
        pow2_scale(m, sc, inv);
        const int b = row >> 4;
        if (quarter / 2 <= b / 2) {
            _Float16* at = hi + tri_frag(b, quarter / 2) * 512 + (row & 15) * 8 + (quarter & 1) * 4;
            _Float16* at2 = lo + (at - hi);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float z[4] = {y[j].x * sc, y[j].y * sc, y[j].z * sc, y[j].w * sc};
                half4 p, q;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[e] = (_Float16)z[e];
                    q[e] = (_Float16)(z[e] - (float)p[e]);
                }
                *reinterpret_cast<half4*>(at + 16 * 8 * j) = p;
                if (lo) *reinterpret_cast<half4*>(at2 + 16 * 8 * j) = q;
            }
        }
        return inv;
    };
    constexpr int NH = TRI * 512;  // values of a triangular matrix
    const float a_inv = write_rows(frag + 2 * NH, gdr_parts<T>() == 2 ? frag + 3 * NH : nullptr);
    __syncthreads();  // sM is read

    // block column w of N: T_ww, then T_bw for b > w. A result tile is the B operand of the next product.
    {
        floatx4 t[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            t[0][r] = sD[w][(4 * gq + r) * LP + li];
            sM[(16 * w + 4 * gq + r) * MP + 16 * w + li] = 4 * gq + r == li ? 0.f : t[0][r];
        }
        for (int b = 0; b < w; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r) sM[(16 * b + 4 * gq + r) * MP + 16 * w + li] = 0.f;
#pragma unroll
        for (int d = 1; d < 4; ++d) {
            const int b = w + d;
            if (b < 4) {
                floatx4 y = zero4();
#pragma unroll
                for (int m = 0; m < d; ++m)
                    y = mma16_f32(y, ld4(sL[b * (b - 1) / 2 + w + m] + li * LP + 4 * gq), t[m]);
                t[d] = mma16_f32(zero4(), ld4(sD[b] + li * LP + 4 * gq), y);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    t[d][r] = -t[d][r];
                    sM[(16 * b + 4 * gq + r) * MP + 16 * w + li] = t[d][r];
                }
            }
        }
    }
    __syncthreads();
    const float n_inv = write_rows(frag, frag + NH);

    // factors
    if (quarter == 0) {
        fac[F_AR * GC + row] = a.scale * a_inv;
        fac[F_NR * GC + row] = n_inv;
        fac[F_BE * GC + row] = s_be[row];
    }
    if (gq == 0) {
        const int t = 16 * w + li;
        float ks, ki, qs, qi;
        pow2_scale(mk, ks, ki);
        pow2_scale(mq, qs, qi);
        const float dec = __builtin_amdgcn_exp2f((float)s_l[t]);
        fac[F_KS * GC + t] = ks;
        fac[F_QS * GC + t] = qs;
        fac[F_G1 * GC + t] = dec * ki;
        fac[F_W * GC + t] = __builtin_amdgcn_exp2f((float)(l_end - s_l[t])) * ki;
        fac[F_GQ * GC + t] = dec * a.scale * qi;
        if (t == 0) fac[REC_FACTORS] = __builtin_amdgcn_exp2f((float)l_end);
    }
}

// ------------------------------------------------------------------------------------------
// gdr_walk: a workgroup has 16 NCW value columns of one (sequence, head). Its NCW chain waves carry
// 16 columns each, S in registers, and exchange nothing; NLW loader waves bring the next chunk's K and
// Q (scaled, f16, fragment order; K also transposed), N, A and factors into the other LDS buffer. One
// barrier per chunk.
// ------------------------------------------------------------------------------------------
template <class T, int DK>
struct WalkShape {
    static constexpr int P = gdr_parts<T>();
    static constexpr int KSTEPS = DK < 32 ? 1 : DK / 32;
    static constexpr int KT = DK / 16;
    static constexpr int KB = 4 * KSTEPS * 1024;        // K or Q, one part
    static constexpr int KTB = KT * 2 * 1024;           // K transposed, one part
    static constexpr int REC = (int)gdr_rec_bytes<T>();
    static constexpr int O_K = 0, O_KT = O_K + P * KB, O_Q = O_KT + P * KTB, O_REC = O_Q + P * KB;
    static constexpr int BYTES = O_REC + REC;
    static constexpr int NBUF = 2 * BYTES <= 160 * 1024 ? 2 : 1;
};

// Four tokens x eight channels of K or Q as stored.
template <class T>
struct Raw8 {
    uint4 x[4][sizeof(T) / 2];
};

template <class T, int DK, int NLW>
struct Loader {
    using Sh = WalkShape<T, DK>;
    static constexpr int NT = 64 * NLW;
    static constexpr int TASKS = 2 * DK;  // (4 tokens, 8 channels) pieces of K, or of Q
    static constexpr int TPT = (TASKS + NT - 1) / NT;
    static constexpr int RECP = (Sh::REC / 16 + NT - 1) / NT;
    Raw8<T> k[TPT], q[TPT];
    float4 ks[TPT], qs[TPT];  // the rows' scales
    uint4 rec[RECP];

    __device__ void load(const ChunkArgs<T>& a, int tid, int c0, int len, int hk, const char* recp)
    {
#pragma unroll
        for (int j = 0; j < TPT; ++j) {
            const int task = tid + NT * j;
            const int tq = task / (DK / 8) % 16, m = task % (DK / 8);
            ks[j] = ld4(reinterpret_cast<const float*>(recp) + F_KS * GC + 4 * tq);
            qs[j] = ld4(reinterpret_cast<const float*>(recp) + F_QS * GC + 4 * tq);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int t = 4 * tq + r;
                const size_t at = ((size_t)(c0 + min(t, len - 1)) * a.Hk + hk) * DK + 8 * m;
#pragma unroll
                for (int u = 0; u < (int)sizeof(T) / 2; ++u) {
                    k[j].x[r][u] = q[j].x[r][u] = make_uint4(0, 0, 0, 0);
                    if (t < len && (TASKS % NT == 0 || task < TASKS)) {
                        k[j].x[r][u] = reinterpret_cast<const uint4*>(a.k + at)[u];
                        q[j].x[r][u] = reinterpret_cast<const uint4*>(a.q + at)[u];
                    }
                }
            }
        }
#pragma unroll
        for (int j = 0; j < RECP; ++j)
            if (tid + NT * j < Sh::REC / 16)
                rec[j] = reinterpret_cast<const uint4*>(recp)[tid + NT * j];
    }

    __device__ static float value(const Raw8<T>& x, int r, int e)
    {
        const uint4& y = x.x[r][e / (16 / sizeof(T))];
        if constexpr (sizeof(T) == 4) {
            const unsigned z[4] = {y.x, y.y, y.z, y.w};
            return __uint_as_float(z[e & 3]);
        } else {
            const unsigned z[4] = {y.x, y.y, y.z, y.w};
            const unsigned p = z[e / 2];
            return __uint_as_float(e & 1 ? p & 0xFFFF0000u : p << 16);
        }
    }

    __device__ void store(char* buf, int tid)
    {
#pragma unroll
        for (int j = 0; j < TPT; ++j) {
            const int task = tid + NT * j;
            if (TASKS % NT != 0 && task >= TASKS) break;
            const int tq = task / (DK / 8), m = task % (DK / 8);
            const float kf[4] = {ks[j].x, ks[j].y, ks[j].z, ks[j].w};
            const float qf[4] = {qs[j].x, qs[j].y, qs[j].z, qs[j].w};
#pragma unroll
            for (int p = 0; p < Sh::P; ++p) {
                _Float16* kd = reinterpret_cast<_Float16*>(buf + Sh::O_K + p * Sh::KB);
                _Float16* td = reinterpret_cast<_Float16*>(buf + Sh::O_KT + p * Sh::KTB);
                _Float16* qd = reinterpret_cast<_Float16*>(buf + Sh::O_Q + p * Sh::KB);
                _Float16 kv[4][8];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    _Float16 qv[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float x = value(k[j], r, e) * kf[r], y = value(q[j], r, e) * qf[r];
                        kv[r][e] = (_Float16)x;
                        qv[e] = (_Float16)y;
                        if (p == 1) {
                            kv[r][e] = (_Float16)(x - (float)kv[r][e]);
                            qv[e] = (_Float16)(y - (float)qv[e]);
                        }
                    }
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int at = frag_at(4 * tq + r, 8 * m + 4 * u, Sh::KSTEPS);
                        const half4 x = {kv[r][4 * u], kv[r][4 * u + 1], kv[r][4 * u + 2], kv[r][4 * u + 3]};
                        const half4 y = {qv[4 * u], qv[4 * u + 1], qv[4 * u + 2], qv[4 * u + 3]};
                        *reinterpret_cast<half4*>(kd + at) = x;
                        *reinterpret_cast<half4*>(qd + at) = y;
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const half4 x = {kv[0][e], kv[1][e], kv[2][e], kv[3][e]};
                    *reinterpret_cast<half4*>(td + frag_at(8 * m + e, 4 * tq, 2)) = x;
                }
            }
        }
#pragma unroll
        for (int j = 0; j < RECP; ++j)
            if (tid + NT * j < Sh::REC / 16)
                reinterpret_cast<uint4*>(buf + Sh::O_REC)[tid + NT * j] = rec[j];
    }
};

__device__ __forceinline__ half8 frag_ld(const char* base, int frag, int lane)
{
    return *reinterpret_cast<const half8*>(base + frag * 1024 + lane * 16);
}

template <class T, int DK, int DV, int NCW, int NLW>
__global__ __launch_bounds__(64 * (NCW + NLW)) void gdr_walk_kernel(const ChunkArgs<T> a)
{
    using Sh = WalkShape<T, DK>;
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
    const char* rec0 = a.rec + ((size_t)g0 * a.H + h) * Sh::REC;
    const size_t rstep = (size_t)a.H * Sh::REC;

    if (DK == 16) {  // the upper half of the 32 contracted places stays 0
        for (int i = threadIdx.x; i < Sh::NBUF * Sh::BYTES / 16; i += 64 * (NCW + NLW))
            reinterpret_cast<uint4*>(lds)[i] = make_uint4(0, 0, 0, 0);
        __syncthreads();
    }

    if (wave >= NCW) {
        const int tid = threadIdx.x - 64 * NCW;
        Loader<T, DK, NLW> ld;
        if (nch > 0) {
            ld.load(a, tid, t0, min(GC, t1 - t0), hk, rec0);
            ld.store(lds, tid);
        }
        if (nch > 1) ld.load(a, tid, t0 + GC, min(GC, t1 - t0 - GC), hk, rec0 + rstep);
        __syncthreads();
        for (int c = 0; c < nch; ++c) {
            if (Sh::NBUF == 1) __syncthreads();  // the chunk's last reads
            if (c + 1 < nch) {
                ld.store(lds + (c + 1) % Sh::NBUF * Sh::BYTES, tid);
                if (c + 2 < nch)
                    ld.load(a, tid, t0 + (c + 2) * GC, min(GC, t1 - t0 - (c + 2) * GC), hk,
                            rec0 + (size_t)(c + 2) * rstep);
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
        const int len = min(GC, t1 - t0 - c * GC);
        const T* p = a.v + ((size_t)(t0 + c * GC) * a.H + h) * DV + col;
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                vn[4 * b + r] = p[(size_t)min(16 * b + 4 * gq + r, len - 1) * vstep];
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
                const half8 qf = frag_ld(buf + Sh::O_Q, b * Sh::KSTEPS + s, lane);
                o[b] = mma(qf, sp[s].hi, o[b]);
                if (Sh::P == 2) {
                    x[b] = mma(frag_ld(buf + Sh::O_K + Sh::KB, b * Sh::KSTEPS + s, lane), sp[s].hi,
                               x[b]);
                    o[b] = mma(qf, sp[s].lo, o[b]);
                    o[b] = mma(frag_ld(buf + Sh::O_Q + Sh::KB, b * Sh::KSTEPS + s, lane), sp[s].hi,
                               o[b]);
                }
            }
        }
        // X = beta (V - 2^l K S)
        m = 0.f;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const float4 g1 = factor(F_G1, b), be = factor(F_BE, b);
            const float g1v[4] = {g1.x, g1.y, g1.z, g1.w}, bev[4] = {be.x, be.y, be.z, be.w};
#pragma unroll
            for (int r = 0; r < 4; ++r)
                x[b][r] = bev[r] * fmaf(-g1v[r], x[b][r] * s_inv, V[b][r]);
            m = max_abs4(m, x[b]);
        }
        // U = X + N X
        float x_inv;
        pow2_scale(column_max(m), sc, x_inv);
        Split xs[2] = {split(x[0], x[1], sc), split(x[2], x[3], sc)};
        floatx4 u[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            u[b] = zero4();
#pragma unroll
            for (int s = 0; s <= b / 2; ++s) {
                const half8 nh = frag_ld(tri, tri_frag(b, s), lane);
                u[b] = mma(nh, xs[s].hi, u[b]);
                u[b] = mma(nh, xs[s].lo, u[b]);
                u[b] = mma(frag_ld(tri, TRI + tri_frag(b, s), lane), xs[s].hi, u[b]);
            }
        }
        m = 0.f;
        float mw = 0.f;
        floatx4 y[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const float4 nr = factor(F_NR, b), w = factor(F_W, b);
            const float nrv[4] = {nr.x, nr.y, nr.z, nr.w}, wv[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                u[b][r] = fmaf(nrv[r], u[b][r] * x_inv, x[b][r]);
                y[b][r] = wv[r] * u[b][r];
            }
            m = max_abs4(m, u[b]);
            mw = max_abs4(mw, y[b]);
        }
        // S <- 2^l_C S + K^T (2^(l_C - l) U)
        float y_inv, u_inv;
        pow2_scale(column_max(mw), sc, y_inv);
        Split ys[2] = {split(y[0], y[1], sc), split(y[2], y[3], sc)};
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
                    d = mma(frag_ld(buf + Sh::O_KT + Sh::KTB, 2 * k + s, lane), ys[s].hi, d);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) S[k][r] = fmaf(gc, S[k][r], d[r] * y_inv);
        }
        // O = scale (2^l Q S + A U)
        pow2_scale(column_max(m), sc, u_inv);
        Split us[2] = {split(u[0], u[1], sc), split(u[2], u[3], sc)};
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
            const float4 gqf = factor(F_GQ, b), ar = factor(F_AR, b);
            const float gv[4] = {gqf.x, gqf.y, gqf.z, gqf.w}, av[4] = {ar.x, ar.y, ar.z, ar.w};
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int t = 16 * b + 4 * gq + r;
                const float z = fmaf(gv[r], o[b][r] * s_inv, av[r] * (d[r] * u_inv));
                if (t < len) op[(size_t)t * vstep] = from_f32<T>(z);
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

template <class T, int DK, int DV, int NCW, int NLW>
hipError_t launch_walk(const ChunkArgs<T>& a, hipStream_t stream)
{
    constexpr int TILES = DV / (16 * NCW);
    const unsigned grid = (unsigned)((a.seq.N * a.H + 7) / 8 * 8 * TILES);
    hipLaunchKernelGGL((gdr_walk_kernel<T, DK, DV, NCW, NLW>), dim3(grid), dim3(64 * (NCW + NLW)), 0,
                       stream, a);
    return hipGetLastError();
}

template <class T, int DK>
hipError_t launch_dk(const GdrCall& c, const ChunkArgs<T>& a, hipStream_t stream)
{
    hipLaunchKernelGGL((gdr_prep_kernel<T, DK>), dim3((unsigned)(a.maxch * a.H)), dim3(256), 0, stream,
                       a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    switch (c.dv) {
    case 16: return launch_walk<T, DK, 16, 1, 2>(a, stream);
    case 32: return launch_walk<T, DK, 32, 2, 2>(a, stream);
    case 64: return launch_walk<T, DK, 64, 2, 2>(a, stream);
    case 128: return launch_walk<T, DK, 128, 2, 2>(a, stream);
    }
    return hipErrorInvalidValue;
}

template <class T>
hipError_t launch_t(const GdrCall& c, hipStream_t stream)
{
    const SeqArgs& s = c.sa;
    const ChunkArgs<T> a = {(const T*)c.q, (const T*)c.k, (const T*)c.v, (const T*)c.alpha,
                            (const T*)c.beta, c.S0, (T*)c.o, c.S_T,
                            {s.cu_seqlens, s.N, s.T, s.B * s.T}, s.H, c.Hk, s.H / c.Hk,
                            gdr_max_chunks(s.cu_seqlens != nullptr, s.N, s.T, s.B * s.T), c.scale,
                            (char*)c.workspace};
    switch (c.dk) {
    case 16: return launch_dk<T, 16>(c, a, stream);
    case 32: return launch_dk<T, 32>(c, a, stream);
    case 64: return launch_dk<T, 64>(c, a, stream);
    case 128: return launch_dk<T, 128>(c, a, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace

size_t gdr_chunk_workspace_bytes(bool packed, int N, int B, int T, int H, kdn_dtype_t dtype)
{
    return (size_t)gdr_max_chunks(packed, N, T, B * T) * H *
           (dtype == KDN_F32 ? gdr_rec_bytes<float>() : gdr_rec_bytes<bf16>());
}

hipError_t launch_gdr_chunked(const GdrCall& c, hipStream_t stream)
{
    return c.dtype == KDN_F32 ? launch_t<float>(c, stream) : launch_t<bf16>(c, stream);
}

}  // namespace kdn
