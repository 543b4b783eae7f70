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

// One chunk and head's record: per-token factors, then matrices in fragment order (f16). The strictly
// lower triangular matrices keep the six fragments that hold it: (row block b, columns 32 s ..) with
// s <= b / 2.
enum GdrFactor {
    F_KS,   // power of two that scales k's row
    F_QS,   // the same for q
    F_G1,   // decay since the chunk's start, over k's scale
    F_BE,   // beta
    F_NR,   // inverse scale of N's row
    F_W,    // decay to the chunk's end, over k's scale
    F_GQ,   // decay since the chunk's start times the output scale, over q's scale
    F_AR,   // output scale times the inverse scale of A's row
    F_COUNT
};
constexpr int REC_FACTORS = F_COUNT * GC;          // floats; then the chunk's whole decay
constexpr int REC_HEAD = (REC_FACTORS + 64) * 4;   // bytes
constexpr int TRI = 6;                             // fragments of a lower triangular matrix
constexpr int TRI_BYTES = TRI * 1024;
__device__ __forceinline__ int tri_frag(int b, int s) { return b < 2 ? b : 2 * b - 2 + s; }

// N hi, N lo, A hi (, A lo)
template <class T> constexpr int gdr_parts() { return sizeof(T) == 4 ? 2 : 1; }
template <class T> constexpr size_t gdr_rec_bytes()
{
    return REC_HEAD + (size_t)(2 + gdr_parts<T>()) * TRI_BYTES;
}

}  // namespace kdn
