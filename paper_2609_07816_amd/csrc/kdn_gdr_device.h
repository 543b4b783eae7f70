// Device helpers of the chunked gated delta rule: float16 operands in two halves, fragment order,
// chunk geometry without a table.
//
// Numbers. A product of float32 accuracy on the 16-bit matrix instructions: each float32 operand x is
// scaled by a power of two (exact) so that the largest value of its row or column lies in [2^14, 2^15),
// and split x = hi + lo with hi = f16(x), lo = f16(x - hi): 22 bits, and values down to 2^-29 of the
// largest keep all of them (f16 has subnormals down to 2^-24). hi hi + hi lo + lo hi then carries an
// error of about 2^-22 of the row's and column's largest. A bf16 input needs no second half: its 8 bits
// fit f16's 11 once its row is scaled. A float32 product of 16 columns costs 3 instructions of 16
// cycles per 16x16x32 (2 with a bf16 input on one side) instead of 8 of 32 cycles on float32
// instructions; bf16 halves would leave 2^-16.
//
// Fragments of v_mfma_f32_16x16x32_f16: lane (g, i) = (lane / 16, lane % 16) holds 8 values of row i
// (A) or column i (B); the result's lane (g, i) holds rows 4g .. 4g+3 of column i. The order of the 32
// contracted places is free as long as both sides use the same one: slot j < 4 of lane group g is place
// 4g + j, slot j >= 4 place 16 + 4g + j - 4. Two result tiles stacked along their rows are then the B
// fragment of the next product as they stand, lane by lane, and the chain of products over the chunks
// of a sequence never leaves a wavefront's registers.
#pragma once

#include "kdn_device.h"
#include "kdn_gdr.h"

namespace kdn {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));

constexpr int GC = 64;  // tokens of a chunk

__device__ __forceinline__ floatx4 mma(half8 a, half8 b, floatx4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Power of two that brings m (the largest magnitude) into [2^14, 2^15), and its inverse. Below 2^-112
// the scale stays at 2^126; infinities and NaN scale to themselves.
__device__ __forceinline__ void pow2_scale(float m, float& sc, float& inv)
{
    const unsigned e = max((__float_as_uint(m) >> 23) & 255u, 15u);
    sc = __uint_as_float((268u - e) << 23);
    inv = __uint_as_float((e - 14u) << 23);
}

// Largest over the lanes that hold other rows of the same column (lanes 16 apart).
__device__ __forceinline__ float column_max(float x)
{
    unsigned u = __float_as_uint(x);
    auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    x = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
    u = __float_as_uint(x);
    p = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float column_sum(float x)
{
    unsigned u = __float_as_uint(x);
    auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    x = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    u = __float_as_uint(x);
    p = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

__device__ __forceinline__ float max_abs4(float m, const floatx4& x)
{
    m = fmaxf(m, fmaxf(fabsf(x[0]), fabsf(x[1])));
    return fmaxf(m, fmaxf(fabsf(x[2]), fabsf(x[3])));
}

// B fragment (halves hi and lo) of two result tiles stacked, scaled by sc.
struct Split {
    half8 hi, lo;
};
__device__ __forceinline__ Split split(const floatx4& a, const floatx4& b, float sc)
{
    Split s;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float x = a[j] * sc, y = b[j] * sc;
        s.hi[j] = (_Float16)x;
        s.hi[4 + j] = (_Float16)y;
        s.lo[j] = (_Float16)(x - (float)s.hi[j]);
        s.lo[4 + j] = (_Float16)(y - (float)s.hi[4 + j]);
    }
    return s;
}
__device__ __forceinline__ half8 to_half(const floatx4& a, const floatx4& b, float sc)
{
    half8 s;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        s[j] = (_Float16)(a[j] * sc);
        s[4 + j] = (_Float16)(b[j] * sc);
    }
    return s;
}

// Place of element (row, col) of a matrix in fragment order, in values: fragments of 16 rows x 32
// columns, `steps` of them along the columns.
__device__ __forceinline__ int frag_at(int row, int col, int steps)
{
    const int c = col & 31;
    return ((row >> 4) * steps + (col >> 5)) * 512 + (((c & 15) >> 2) * 16 + (row & 15)) * 8 +
           (c & 3) + ((c >> 4) << 2);
}

// Chunks of 64 tokens restart at every sequence start. Sequence n's first chunk has the index
// n ceil(T / 64) (rows of one length) or t0 / 64 + n (packed): the latter leaves at least
// ceil(len / 64) indexes to every sequence, so no table is needed, and ntok / 64 + N in all.
struct GdrSeq {
    const int32_t* cu;
    int N, T, ntok;
};

__host__ __device__ inline int gdr_max_chunks(bool packed, int N, int T, int ntok)
{
    return packed ? ntok / GC + N : N * ((T + GC - 1) / GC);
}

__device__ __forceinline__ void gdr_span(const GdrSeq& s, int n, int& t0, int& t1)
{
    if (s.cu) {  // clamped: a broken table never leads outside the tensors
        t0 = min(max(s.cu[n], 0), s.ntok);
        t1 = min(max(s.cu[n + 1], t0), s.ntok);
    } else {
        t0 = n * s.T;
        t1 = t0 + s.T;
    }
}

__device__ __forceinline__ int gdr_first_chunk(const GdrSeq& s, int n, int t0)
{
    return s.cu ? t0 / GC + n : n * ((s.T + GC - 1) / GC);
}

// Chunk g -> its tokens [c0, c1) and sequence; false where the index is one that no sequence uses.
__device__ __forceinline__ bool gdr_locate(const GdrSeq& s, int g, int& n, int& c0, int& c1)
{
    if (s.cu) {
        int lo = 0, hi = s.N - 1;  // the last sequence whose first chunk is at most g
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            const int t = min(max(s.cu[mid], 0), s.ntok);
            if (t / GC + mid <= g) lo = mid; else hi = mid - 1;
        }
        n = lo;
    } else {
        n = g / ((s.T + GC - 1) / GC);
    }
    int t0, t1;
    gdr_span(s, n, t0, t1);
    const int m = g - gdr_first_chunk(s, n, t0);
    c0 = t0 + m * GC;
    c1 = min(c0 + GC, t1);
    return m >= 0 && c0 < c1;
}

// One chunk and head's record: per-token factors, then matrices in fragment order (f16, halves hi and
// lo). A strictly lower triangular matrix keeps the six fragments that hold it: (row block b, columns
// 32 s ..) with s <= b / 2; a transposed one those with s >= b / 2.
enum GdrFactor {
    F_KS,   // power of two that scales k's row
    F_QS,   // the same for q
    F_G1,   // decay since the chunk's start, over k's scale
    F_BE,   // beta
    F_WR,   // inverse scale of W's row
    F_W,    // decay to the chunk's end, over k's scale
    F_GQ,   // decay since the chunk's start times the output scale, over q's scale
    F_AR,   // output scale times the inverse scale of A's row
    F_WTR,  // the same of the transposed matrices (backward)
    F_ATR,
    F_L,    // float64 cumulative log2 decay (two rows)
    F_COUNT = F_L + 2
};
constexpr int REC_FACTORS = F_COUNT * GC;         // floats; then the chunk's whole decay
constexpr int REC_HEAD = (REC_FACTORS + 64) * 4;  // bytes
constexpr int TRI = 6;                            // fragments of a triangular matrix
constexpr int TRI_BYTES = TRI * 1024;
__device__ __forceinline__ int tri_frag(int b, int s) { return b < 2 ? b : 2 * b - 2 + s; }
__device__ __forceinline__ int tri_frag_t(int b, int s) { return b < 2 ? 2 * b + s : b + 2; }

template <class T> constexpr int gdr_parts() { return sizeof(T) == 4 ? 2 : 1; }

// Records of the forward (W hi, W lo, A hi (, A lo)) and of the backward (W, W^T, A^T, hi and lo).
template <class T, bool BWD> constexpr int gdr_rec_bytes()
{
    return REC_HEAD + (BWD ? 6 : 2 + gdr_parts<T>()) * TRI_BYTES;
}

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

__device__ __forceinline__ float4 ld4(const float* p) { return *reinterpret_cast<const float4*>(p); }

__device__ __forceinline__ half8 frag_ld(const char* base, int frag, int lane)
{
    return *reinterpret_cast<const half8*>(base + frag * 1024 + lane * 16);
}

// LDS of one chunk: fragment-order K, K transposed, Q, Q transposed (each if wanted, P parts), then the
// record's head and the part of its matrices that the kernel uses.
template <class T, int DK, bool KR, bool KC, bool QR, bool QC, int MATS>
struct ChunkLds {
    static constexpr int P = gdr_parts<T>();
    static constexpr int KSTEPS = DK < 32 ? 1 : DK / 32;
    static constexpr int KT = DK / 16;
    static constexpr int RB = 4 * KSTEPS * 1024;  // K or Q by rows, one part
    static constexpr int CB = KT * 2 * 1024;      // transposed, one part
    static constexpr int O_K = 0;
    static constexpr int O_KT = O_K + (KR ? P * RB : 0);
    static constexpr int O_Q = O_KT + (KC ? P * CB : 0);
    static constexpr int O_QT = O_Q + (QR ? P * RB : 0);
    static constexpr int O_REC = O_QT + (QC ? P * CB : 0);
    static constexpr int REC = MATS < 0 ? 0 : REC_HEAD + MATS * TRI_BYTES;
    static constexpr int BYTES = O_REC + REC;
    static constexpr int NBUF = 2 * BYTES <= 160 * 1024 ? 2 : 1;
    static constexpr bool kr = KR, kc = KC, qr = QR, qc = QC;
};

// Four tokens x eight channels of K or Q as stored.
template <class T>
struct Raw8 {
    uint4 x[4][sizeof(T) / 2];

    __device__ __forceinline__ void load(const T* base, size_t step, int t, int len, bool on)
    {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int u = 0; u < (int)sizeof(T) / 2; ++u) {
                x[r][u] = make_uint4(0, 0, 0, 0);
                if (on && t + r < len)
                    x[r][u] = reinterpret_cast<const uint4*>(base + (size_t)(t + r) * step)[u];
            }
    }
    __device__ __forceinline__ float value(int r, int e) const
    {
        const uint4& y = x[r][e / (16 / (int)sizeof(T))];
        const unsigned z[4] = {y.x, y.y, y.z, y.w};
        if constexpr (sizeof(T) == 4) {
            return __uint_as_float(z[e & 3]);
        } else {
            const unsigned p = z[e / 2];
            return __uint_as_float(e & 1 ? p & 0xFFFF0000u : p << 16);
        }
    }
    // Scaled by row, part p (0: hi, 1: lo), to the row fragments and the transposed ones.
    template <bool ROWS, bool COLS, int KSTEPS>
    __device__ __forceinline__ void store(const float4& sc, int p, int t, int c, _Float16* rows,
                                          _Float16* cols) const
    {
        const float f[4] = {sc.x, sc.y, sc.z, sc.w};
        _Float16 y[4][8];
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float z = value(r, e) * f[r];
                y[r][e] = (_Float16)z;
                if (p == 1) y[r][e] = (_Float16)(z - (float)y[r][e]);
            }
        if (ROWS)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    *reinterpret_cast<half4*>(rows + frag_at(t + r, c + 4 * u, KSTEPS)) =
                        half4{y[r][4 * u], y[r][4 * u + 1], y[r][4 * u + 2], y[r][4 * u + 3]};
        if (COLS)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                *reinterpret_cast<half4*>(cols + frag_at(c + e, t, 2)) =
                    half4{y[0][e], y[1][e], y[2][e], y[3][e]};
    }
};

// The loading side of a workgroup: NT threads bring a chunk from memory to registers, and from there
// to LDS. SKIP: bytes of the record between its head and the matrices wanted.
template <class T, int DK, class Lds, int NT, int SKIP>
struct Loader {
    static constexpr int TASKS = 2 * DK;  // (4 tokens, 8 channels) pieces of K, or of Q
    static constexpr int TPT = (TASKS + NT - 1) / NT;
    static constexpr int RECP = (Lds::REC / 16 + NT - 1) / NT;
    static constexpr bool useq = Lds::qr || Lds::qc;
    Raw8<T> k[TPT], q[useq ? TPT : 1];
    float4 ks[TPT], qs[useq ? TPT : 1];  // the rows' scales
    uint4 rec[RECP > 0 ? RECP : 1];

    __device__ __forceinline__ void load(const T* kbase, const T* qbase, size_t step, int tid, int len,
                                         const char* recp)
    {
#pragma unroll
        for (int j = 0; j < TPT; ++j) {
            const int task = tid + NT * j, t = 4 * (task / (DK / 8) % 16), c = 8 * (task % (DK / 8));
            const bool on = TASKS % NT == 0 || task < TASKS;
            const float* fac = reinterpret_cast<const float*>(recp);
            ks[j] = ld4(fac + F_KS * GC + t);
            k[j].load(kbase + c, step, t, len, on);
            if (useq) {
                qs[j] = ld4(fac + F_QS * GC + t);
                q[j].load(qbase + c, step, t, len, on);
            }
        }
#pragma unroll
        for (int j = 0; j < RECP; ++j) {
            const int at = tid + NT * j;
            if (at < Lds::REC / 16)
                rec[j] = reinterpret_cast<const uint4*>(
                    recp + (at < REC_HEAD / 16 ? 0 : SKIP))[at];
        }
    }

    __device__ __forceinline__ void store(char* buf, int tid)
    {
#pragma unroll
        for (int j = 0; j < TPT; ++j) {
            const int task = tid + NT * j, t = 4 * (task / (DK / 8)), c = 8 * (task % (DK / 8));
            if (TASKS % NT != 0 && task >= TASKS) break;
#pragma unroll
            for (int p = 0; p < Lds::P; ++p) {
                k[j].template store<Lds::kr, Lds::kc, Lds::KSTEPS>(
                    ks[j], p, t, c, reinterpret_cast<_Float16*>(buf + Lds::O_K + p * Lds::RB),
                    reinterpret_cast<_Float16*>(buf + Lds::O_KT + p * Lds::CB));
                if (useq)
                    q[j].template store<Lds::qr, Lds::qc, Lds::KSTEPS>(
                        qs[j], p, t, c, reinterpret_cast<_Float16*>(buf + Lds::O_Q + p * Lds::RB),
                        reinterpret_cast<_Float16*>(buf + Lds::O_QT + p * Lds::CB));
            }
        }
#pragma unroll
        for (int j = 0; j < RECP; ++j)
            if (tid + NT * j < Lds::REC / 16)
                reinterpret_cast<uint4*>(buf + Lds::O_REC)[tid + NT * j] = rec[j];
    }
};

// Column of 16 values x four row blocks of [tokens][H][DV] in the layout of result tiles, as stored.
template <class T>
__device__ __forceinline__ void load_tile(const T* p, size_t step, int gq, int len, T* x)
{
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            x[4 * b + r] = p[(size_t)min(16 * b + 4 * gq + r, len - 1) * step];
}

__device__ __forceinline__ void unpack4(const float4& x, float* y)
{
    y[0] = x.x; y[1] = x.y; y[2] = x.z; y[3] = x.w;
}

// Launchers of the kernels that forward and backward share (kdn_gdr_prep.hip).
template <class T>
hipError_t launch_gdr_prep(const ChunkArgs<T>& a, int dk, bool backward, hipStream_t stream);

}  // namespace kdn
