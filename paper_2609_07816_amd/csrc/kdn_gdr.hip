// Gated delta rule, token by token, on gfx950: the decode step on a pool of states, and the forward
// of short sequences.
//
// Per token of a (row, head), with the state S [dk, dv] in float32 registers:
//   u = beta (v - alpha S^T k),  S <- alpha S + k u^T,  o = scale S^T q.
// The read is o = scale (alpha S^T q + (k.q) u) on the state before the write, so that S^T k, S^T q
// and k.q are summed across the lanes together: one exchange per token. A wavefront holds all dk
// rows of 32 value columns (16 at dv = 16) and no two wavefronts exchange anything: a lane has dk / 8
// rows of four adjacent columns, so a load of the state is 16 bytes per lane and whole 128-byte row
// pieces. A decode step is bound by HBM, which S crosses once in and once out: 256 rows of 16 heads of
// d 128 in 117 us, 4.6 TB/s, 96% of a large copy's rate; 4 rows in 9 us, a launch and one round trip.
#include "kdn_gdr.h"

namespace kdn {
namespace {

template <int DK, int DV>
struct RecShape {
    static constexpr int CW = DV < 32 ? DV : 32;  // columns of a wavefront
    static constexpr int NCG = CW / 4;            // lanes along the columns
    static constexpr int NRG = 64 / NCG;          // lanes along the rows
    static constexpr int RPT = DK / NRG;          // rows of a lane
};

template <class T, int N>
struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Vec {
    T v[N];
};

template <class T, int N>
__device__ __forceinline__ Vec<T, N> ldv(const T* p)
{
    return *reinterpret_cast<const Vec<T, N>*>(p);
}

// Sum over the lanes that hold other rows of the same columns (lanes NCG apart), to all of them.
template <int NCG>
__device__ __forceinline__ float rows_sum(float x)
{
    if (NCG == 4) x = dpp_add<0x124, 0xf>(x);  // row_ror:4 (a row of 16 lanes, rotated)
    x = dpp_add<0x128, 0xf>(x);                // row_ror:8
    unsigned u = __float_as_uint(x);
    auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);  // rows 0 and 1, 2 and 3
    x = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    u = __float_as_uint(x);
    p = __builtin_amdgcn_permlane32_swap(u, u, false, false);  // the wavefront's halves
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

template <class T>
struct RecArgs {
    const T *q, *k, *v, *alpha, *beta;
    const float* S_in;  // or nullptr (0)
    float* S_out;       // or nullptr
    T* o;
    const int32_t* cu;    // a packed batch's sequences, or nullptr: row n is tokens [n len, (n + 1) len)
    const int32_t* slot;  // the state of each row, or nullptr: row n has state n
    int rows, num_slots, len, ntok, H, rep;  // rep: value heads of a key head
    float scale;
};

template <class T, int DK, int DV>
__global__ __launch_bounds__(64) void gdr_recurrent_kernel(const RecArgs<T> a)
{
    using Sh = RecShape<DK, DV>;
    constexpr int NT = DV / Sh::CW, RPT = Sh::RPT;
    const int lane = threadIdx.x, cg = lane % Sh::NCG, rg = lane / Sh::NCG;
    const int tile = blockIdx.x % NT, rh = blockIdx.x / NT;
    const int h = rh % a.H, row = rh / a.H;
    if (row >= a.rows) return;
    const int slot = a.slot ? a.slot[row] : row;
    if (slot < 0 || slot >= a.num_slots) return;  // uniform across the wavefront
    int t0 = row * a.len, t1 = t0 + a.len;
    if (a.cu) {
        t0 = min(max(a.cu[row], 0), a.ntok);
        t1 = min(max(a.cu[row + 1], t0), a.ntok);
    }
    const size_t soff = ((size_t)slot * a.H + h) * DK * DV + (size_t)rg * RPT * DV +
                        tile * Sh::CW + 4 * cg;
    float4 s[RPT];
#pragma unroll
    for (int i = 0; i < RPT; ++i)
        s[i] = a.S_in ? *reinterpret_cast<const float4*>(a.S_in + soff + (size_t)i * DV)
                      : make_float4(0.f, 0.f, 0.f, 0.f);

    const int Hk = a.H / a.rep, hk = h / a.rep;
    const T* kp = a.k + ((size_t)t0 * Hk + hk) * DK + rg * RPT;
    const T* qp = a.q + ((size_t)t0 * Hk + hk) * DK + rg * RPT;
    const size_t vo = ((size_t)t0 * a.H + h) * DV + tile * Sh::CW + 4 * cg;
    const T* vp = a.v + vo;
    T* op = a.o + vo;
    const T* ap = a.alpha + (size_t)t0 * a.H + h;
    const T* bp = a.beta + (size_t)t0 * a.H + h;
    const size_t kstep = (size_t)Hk * DK, vstep = (size_t)a.H * DV;

    Vec<T, RPT> kn, qn;
    Vec<T, 4> vn;
    T an, bn;
    if (t0 < t1) {
        kn = ldv<T, RPT>(kp);
        qn = ldv<T, RPT>(qp);
        vn = ldv<T, 4>(vp);
        an = *ap;
        bn = *bp;
    }
    for (int t = t0; t < t1; ++t) {
        float kk[RPT], qq[RPT], vv[4];
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            kk[i] = to_f32(kn.v[i]);
            qq[i] = to_f32(qn.v[i]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) vv[j] = to_f32(vn.v[j]);
        const float al = to_f32(an), be = to_f32(bn);
        if (t + 1 < t1) {  // the next token's inputs, while this one is computed
            kp += kstep;
            qp += kstep;
            vp += vstep;
            ap += a.H;
            bp += a.H;
            kn = ldv<T, RPT>(kp);
            qn = ldv<T, RPT>(qp);
            vn = ldv<T, 4>(vp);
            an = *ap;
            bn = *bp;
        }
        float sk[4] = {0.f, 0.f, 0.f, 0.f}, sq[4] = {0.f, 0.f, 0.f, 0.f}, kq = 0.f;
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const float x[4] = {s[i].x, s[i].y, s[i].z, s[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sk[j] = fmaf(x[j], kk[i], sk[j]);
                sq[j] = fmaf(x[j], qq[i], sq[j]);
            }
            kq = fmaf(kk[i], qq[i], kq);
        }
        kq = rows_sum<Sh::NCG>(kq);
        float u[4];
        Vec<T, 4> out;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u[j] = be * (vv[j] - al * rows_sum<Sh::NCG>(sk[j]));
            out.v[j] = from_f32<T>(a.scale * (al * rows_sum<Sh::NCG>(sq[j]) + kq * u[j]));
        }
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            s[i].x = fmaf(al, s[i].x, kk[i] * u[0]);
            s[i].y = fmaf(al, s[i].y, kk[i] * u[1]);
            s[i].z = fmaf(al, s[i].z, kk[i] * u[2]);
            s[i].w = fmaf(al, s[i].w, kk[i] * u[3]);
        }
        if (rg == 0) *reinterpret_cast<Vec<T, 4>*>(op) = out;
        op += vstep;
    }
    if (a.S_out)
#pragma unroll
        for (int i = 0; i < RPT; ++i)
            *reinterpret_cast<float4*>(a.S_out + soff + (size_t)i * DV) = s[i];
}

template <class T>
hipError_t launch_t(const RecArgs<T>& a, int dk, int dv, hipStream_t stream)
{
    if (a.rows == 0) return hipSuccess;
    const unsigned tiles = dv <= 32 ? 1 : dv / 32;
    const dim3 grid((unsigned)a.rows * (unsigned)a.H * tiles), block(64);
#define KDN_GDR_CASE(DK, DV)                                                                \
    if (dk == DK && dv == DV) {                                                             \
        hipLaunchKernelGGL((gdr_recurrent_kernel<T, DK, DV>), grid, block, 0, stream, a);   \
        return hipGetLastError();                                                           \
    }
#define KDN_GDR_ROW(DK) \
    KDN_GDR_CASE(DK, 16) KDN_GDR_CASE(DK, 32) KDN_GDR_CASE(DK, 64) KDN_GDR_CASE(DK, 128)
    KDN_GDR_ROW(16) KDN_GDR_ROW(32) KDN_GDR_ROW(64) KDN_GDR_ROW(128)
#undef KDN_GDR_ROW
#undef KDN_GDR_CASE
    return hipErrorInvalidValue;
}

template <class T>
hipError_t decode_t(const void* q, const void* k, const void* v, const void* alpha,
                    const void* beta, float* S, const int32_t* slot_idx, void* o, int R,
                    int num_slots, int H, int Hk, int dk, int dv, float scale, hipStream_t stream)
{
    const RecArgs<T> a = {(const T*)q, (const T*)k, (const T*)v, (const T*)alpha, (const T*)beta,
                          S, S, (T*)o, nullptr, slot_idx, R, num_slots, 1, R, H, H / Hk, scale};
    return launch_t(a, dk, dv, stream);
}

template <class T>
hipError_t recurrent_t(const GdrCall& c, hipStream_t stream)
{
    const RecArgs<T> a = {(const T*)c.q, (const T*)c.k, (const T*)c.v, (const T*)c.alpha,
                          (const T*)c.beta, c.S0, c.S_T, (T*)c.o, c.sa.cu_seqlens, nullptr, c.sa.N,
                          c.sa.N, c.sa.T, c.sa.B * c.sa.T, c.sa.H, c.sa.H / c.Hk, c.scale};
    return launch_t(a, c.dk, c.dv, stream);
}

}  // namespace

hipError_t launch_gdr_decode(const void* q, const void* k, const void* v, const void* alpha,
                             const void* beta, float* S, const int32_t* slot_idx, void* o, int R,
                             int num_slots, int H, int Hk, int dk, int dv, kdn_dtype_t dtype,
                             float scale, hipStream_t stream)
{
    return dtype == KDN_F32 ? decode_t<float>(q, k, v, alpha, beta, S, slot_idx, o, R, num_slots,
                                              H, Hk, dk, dv, scale, stream)
                            : decode_t<bf16>(q, k, v, alpha, beta, S, slot_idx, o, R, num_slots, H,
                                             Hk, dk, dv, scale, stream);
}

hipError_t launch_gdr_recurrent(const GdrCall& c, hipStream_t stream)
{
    return c.dtype == KDN_F32 ? recurrent_t<float>(c, stream) : recurrent_t<bf16>(c, stream);
}

}  // namespace kdn
