// Beam search on gfx950: the selection of the W best of W x V candidates per batch element, and the
// reordering of the beams' recurrent states in their slot pool.
//
// Selection. A candidate (beam w, token y) has the score scores[w] + ((x_y - m) - log sum exp(x - m))
// with x the beam's logits and m the largest. Within a beam the order of scores is the order of
// logits, so nothing needs the sum before the end, and one pass reads the logits: each wavefront takes
// a piece of a row, keeps the running maximum and sum of its exponentials per lane, and the W largest
// logits in order, one per lane (entry i in lane i). Of a tile of 512 values only those above the W-th
// entry enter that list, one after another (taking the tile's largest first, round by round, took 34 us
// in place of 30 at 384 rows of 50,021; reading off the candidates lane by lane 49). The second kernel joins a row's pieces (lane = piece, each round takes the best head), then
// the rows (lane = beam). Values are compared as integers in the same order as the floats; 0 is below
// every value and marks places without one. The sums are float32 in a fixed order: no atomics.
#include "kdn_beam.h"
#include "kdn_device.h"

namespace kdn {
namespace {

constexpr int TILE = 512;       // values of a tile: eight per lane
constexpr int MAX_PIECES = 64;  // pieces of a row: one lane each when they are joined

// floats as integers of the same order; a NaN counts as -inf, +inf as the largest finite value and
// -0 as 0
__device__ __forceinline__ float counted(float x)
{
    return fminf(fmaxf(x, -INFINITY), 3.402823466e38f);
}
__device__ __forceinline__ unsigned bits_key(unsigned u)  // of a counted value's bits
{
    u = u == 0x80000000u ? 0u : u;
    return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ unsigned order_key(float x) { return bits_key(__float_as_uint(counted(x))); }
__device__ __forceinline__ float key_value(unsigned k)
{
    return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k);
}

template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned dpp_umax(unsigned x)
{
    return max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false));
}
// Largest value of the 64 lanes (same steps as wave_sum).
__device__ __forceinline__ unsigned wave_umax(unsigned x)
{
    x = dpp_umax<0x111, 0xf>(x);
    x = dpp_umax<0x112, 0xf>(x);
    x = dpp_umax<0x114, 0xf>(x);
    x = dpp_umax<0x118, 0xf>(x);
    x = dpp_umax<0x142, 0xa>(x);
    x = dpp_umax<0x143, 0xc>(x);
    return (unsigned)__builtin_amdgcn_readlane((int)x, 63);
}

__device__ __forceinline__ float exp_diff(float x, float m)  // e^(x - m)
{
    return __builtin_amdgcn_exp2f((x - m) * 1.44269504f);
}

struct Entry {
    unsigned key, token;
};

template <class T>
struct __attribute__((packed, aligned(sizeof(T)))) Values8 {
    T v[8];
};

// The list of a wavefront: entry i in lane i, in order of the keys, equal ones of the lowest token first;
// its W-th entry (uniform).
struct List {
    unsigned key = 0, token = 0, last_key = 0, last_token = 0;

    __device__ __forceinline__ void insert(unsigned k, unsigned tok, int lane, int W)
    {
        const unsigned long long above = __ballot(key > k), same = __ballot(key == k),
                                 lower = __ballot(token < tok);
        const int pos = __builtin_popcountll(above | (same & lower));  // sorted: a prefix
        const unsigned pk = lane_before(key), pt = lane_before(token);
        key = lane > pos ? pk : lane == pos ? k : key;
        token = lane > pos ? pt : lane == pos ? tok : token;
        if (lane >= W) key = 0;
        const unsigned lk = (unsigned)__builtin_amdgcn_readlane((int)key, W - 1);
        if (lk >= last_key && lk) {
            last_key = lk;
            last_token = (unsigned)__builtin_amdgcn_readlane((int)token, W - 1);
        }
    }
    __device__ static __forceinline__ unsigned lane_before(unsigned x)  // wave_shr 1
    {
        return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x138, 0xf, 0xf, false);
    }
};

// Grid: (pieces of a row, rows), 64 threads. stats [rows][pieces] (m, sum), best [rows][pieces][W].
// Bound by its own instructions, some 30 per value and wavefront (the exponential, the order of keys, the
// list), with every wavefront resident at once: 384 rows (a fifth of them finished) of 50,021 bf16 logits,
// W 8, take 30 us, 80 rows of 131,072 float32 ones, W 5, 19 us; reading them alone 6 and 8.5 us at the copy
// rate. Half and a quarter as many pieces measured the same and slower.
template <class T>
__global__ __launch_bounds__(64) void beam_piece_kernel(const T* __restrict__ logits,
                                                        const uint8_t* __restrict__ done, int W,
                                                        int V, int tiles, float2* __restrict__ stats,
                                                        Entry* __restrict__ best)
{
    const int lane = threadIdx.x, piece = blockIdx.x, pieces = gridDim.x;
    const size_t row = blockIdx.y;
    if (done && done[row]) return;
    const T* x0 = logits + row * (size_t)V;
    const int first = piece * tiles * TILE;
    List list;
    float m = -INFINITY, s = 0.f;
    // Eight values of a lane in one load whatever the row's alignment (rows of odd length start anywhere;
    // global loads need none): the places of a lane, and so the order of the sums, depend on the row
    // alone. The next tile is on its way while this one is worked on; places past the row's end are not
    // read.
    auto fetch = [&](int at) {
        Values8<T> y = {};
        if (at + 8 <= V) y = *reinterpret_cast<const Values8<T>*>(x0 + at);
        return y;
    };
    Values8<T> next = fetch(first + 8 * lane);
    for (int t = 0; t < tiles; ++t) {
        const int base = first + t * TILE, at = base + 8 * lane;
        if (base >= V) break;
        Values8<T> y = next;
        if (t + 1 < tiles) next = fetch(at + TILE);
        const bool whole = base + TILE <= V;  // uniform
        if (!whole && at + 8 > V)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (at + e < V) y.v[e] = x0[at + e];
        float x[8];
        unsigned key[8], b = 0;
        float mt = m;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = counted(to_f32(y.v[e]));
            if (!whole && at + e >= V) x[e] = -INFINITY;
            key[e] = bits_key(__float_as_uint(x[e]));
            if (!whole && at + e >= V) key[e] = 0;
            mt = fmaxf(mt, x[e]);
            b = max(b, key[e]);
        }
        const float ref = mt == -INFINITY ? 0.f : mt;
        s *= exp_diff(m, ref);
#pragma unroll
        for (int e = 0; e < 8; ++e) s += exp_diff(x[e], ref);
        m = mt;
        if (t == 0) {
            // the W-th of the lanes' largest: at least W values are no less, so none below it enters
            unsigned c = b, w_th = 0;
            for (int i = 0; i < W; ++i) {
                w_th = wave_umax(c);
                if (lane == __builtin_ctzll(__ballot(c == w_th))) c = 0;
            }
            list.last_key = w_th ? w_th - 1 : 0;
        }
        if (!__ballot(b > list.last_key)) continue;  // later tiles have higher tokens: no ties enter
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            // not in order of tokens: among equal values the lowest token counts
            unsigned long long todo = ~0ull;
            for (;;) {
                const unsigned long long in =
                    (__ballot(key[e] > list.last_key) |
                     (__ballot(key[e] == list.last_key) & __ballot((unsigned)(at + e) < list.last_token))) &
                    todo;
                if (!in) break;
                const int l = __builtin_ctzll(in);
                todo = l == 63 ? 0 : ~0ull << (l + 1);
                list.insert((unsigned)__builtin_amdgcn_readlane((int)key[e], l),
                            (unsigned)(base + 8 * l + e), lane, W);
            }
        }
    }
    const float M = key_value(wave_umax(order_key(m)));
    const float ref = M == -INFINITY ? 0.f : M;
    const float sum = wave_sum(s * exp_diff(m, ref));
    const size_t o = row * pieces + piece;
    if (lane == 0) stats[o] = make_float2(M, sum);
    if (lane < W) best[o * W + lane] = Entry{list.key, list.token};
}

// Grid: batch elements; `blockDim.x / 64` wavefronts take its rows in turn. Dynamic LDS: the rows'
// lists [W][W] (ordered score, token), then one piece table [pieces][W] per wavefront.
__global__ void beam_join_kernel(const float* __restrict__ scores, const uint8_t* __restrict__ done,
                                 int W, int V, int end_token, int pieces,
                                 const float2* __restrict__ stats, const Entry* __restrict__ best,
                                 float* __restrict__ scores_out, int32_t* __restrict__ token_out,
                                 int32_t* __restrict__ parent_out, uint8_t* __restrict__ done_out)
{
    extern __shared__ Entry lds[];
    Entry* lists = lds;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    Entry* mine = lds + W * W + wave * pieces * W;
    const size_t n = blockIdx.x;
    for (int w = wave; w < W; w += waves) {
        const size_t row = n * W + w;
        const float prev = scores[row];
        Entry* list = lists + w * W;
        if (done && done[row]) {  // its end token at its own score, then the others in order
            for (int i = lane; i < W; i += 64) {
                const int y = i == 0 ? end_token : (i <= end_token ? i - 1 : i);
                list[i] = i == 0 ? Entry{order_key(prev), (unsigned)y}
                                 : Entry{i < V ? order_key(-INFINITY) : 0u, (unsigned)y};
            }
            continue;
        }
        for (int i = lane; i < pieces * W; i += 64) mine[i] = best[row * pieces * W + i];
        float2 st = make_float2(-INFINITY, 0.f);
        if (lane < pieces) st = stats[row * pieces + lane];
        const float M = key_value(wave_umax(order_key(st.x)));
        const float ref = M == -INFINITY ? 0.f : M;
        const float norm = logf(wave_sum(st.y * exp_diff(st.x, ref)));
        wave_lds_fence();
        int at = 0;  // this lane's piece: entries taken so far
        Entry head = lane < pieces ? mine[lane * W] : Entry{0, 0};
        for (int i = 0; i < W; ++i) {
            const unsigned mx = wave_umax(head.key);
            unsigned long long tie = __ballot(head.key == mx);
            if (tie & (tie - 1)) {  // equal logits: the lowest token
                const unsigned low = ~wave_umax(head.key == mx ? ~head.token : 0u);
                tie = __ballot(head.key == mx && head.token == low);
            }
            const int win = __builtin_ctzll(tie);
            if (lane == win) {
                const float x = key_value(mx);
                // a masked logit has no score, whatever its row's sum is
                const float score = x == -INFINITY ? x : prev + ((x - M) - norm);
                list[i] = Entry{mx ? order_key(score) : 0u, head.token};
                ++at;
                head = lane < pieces && at < W ? mine[lane * W + at] : Entry{0, 0};
            }
        }
        wave_lds_fence();
    }
    __syncthreads();
    if (wave != 0) return;
    // the rows' lists: scores fall within each, equal ones go to the lowest beam
    int at = 0;
    Entry head = lane < W ? lists[lane * W] : Entry{0, 0};
    for (int i = 0; i < W; ++i) {
        const unsigned mx = wave_umax(head.key);
        const int win = __builtin_ctzll(__ballot(head.key == mx));
        if (lane == win) {
            const size_t o = n * W + i, row = n * W + lane;
            scores_out[o] = key_value(mx);
            token_out[o] = (int32_t)head.token;
            parent_out[o] = lane;
            if (done_out)
                done_out[o] = (int)head.token == end_token || (done && done[row]) ? 1 : 0;
            ++at;
            head = lane < W && at < W ? lists[lane * W + at] : Entry{0, 0};
        }
    }
}

// ------------------------------------------------------------------------------------------
// Reordering. A parent's first child keeps the parent's slot; every other child gets the slot of a
// beam without children (the i-th such child the i-th such beam) and a copy of its parent's state.
// Copies read slots that keep their content and write slots that nothing reads, so one kernel moves
// everything in place, and only what a fork needs: 2 bytes moved per byte forked. Every workgroup
// finds its child's slots from its batch element's W parents.
// ------------------------------------------------------------------------------------------
// Bound by memory: 240 forked states of 1 MB (500 MB moved) in 60 to 75 us, which the cache behind the L2s
// helps, 57 of them (120 MB) in 20 us. 16 KB a workgroup, all its loads in flight in registers: 32 KB
// measured the same, 8 KB 25 us more.
constexpr int COPY_UNROLL = 4;
constexpr size_t COPY_PIECE = 256 * 16 * COPY_UNROLL;  // bytes of a workgroup: 16 KB

__device__ __forceinline__ void copy_piece(const char* src, char* dst, size_t bytes)
{
    const int tid = threadIdx.x;
    if ((((uintptr_t)src | (uintptr_t)dst | bytes) & 15) == 0) {
        typedef unsigned u4 __attribute__((ext_vector_type(4)));
        const u4* s = reinterpret_cast<const u4*>(src);
        u4* d = reinterpret_cast<u4*>(dst);
        const int n = (int)(bytes / 16);
        u4 x[COPY_UNROLL];
#pragma unroll
        for (int i = 0; i < COPY_UNROLL; ++i) x[i] = s[min(tid + 256 * i, n - 1)];
#pragma unroll
        for (int i = 0; i < COPY_UNROLL; ++i)
            if (tid + 256 * i < n) d[tid + 256 * i] = x[i];
    } else {  // slots of an odd number of words (per-head variances)
        const unsigned* s = reinterpret_cast<const unsigned*>(src);
        unsigned* d = reinterpret_cast<unsigned*>(dst);
        for (int i = tid; i < (int)(bytes / 4); i += 256) d[i] = s[i];
    }
}

// Grid: (pieces of a slot of S, then of P; N * W), 256 threads.
__global__ __launch_bounds__(256) void beam_reorder_kernel(
    const int32_t* __restrict__ parent, const int32_t* __restrict__ slot_idx,
    int32_t* __restrict__ slot_out, int W, int num_slots, char* S, size_t s_bytes, int s_pieces,
    char* P, size_t p_bytes)
{
    const int lane = threadIdx.x & 63;
    const int n = blockIdx.y / W, w = blockIdx.y % W;
    int par = -1;
    if (lane < W) par = parent[(size_t)n * W + lane];
    unsigned long long seen = 0, extra = 0;  // beams with children; children without a slot yet
    for (int j = 0; j < W; ++j) {
        const int p = __builtin_amdgcn_readlane(par, j);
        const bool valid = p >= 0 && p < W;
        if (!valid || (seen >> p & 1)) extra |= 1ull << j;
        if (valid) seen |= 1ull << p;
    }
    const int p = __builtin_amdgcn_readlane(par, w);
    const bool valid = p >= 0 && p < W;
    int take = p;
    if (extra >> w & 1) {
        int rank = __builtin_popcountll(extra & ((1ull << w) - 1));
        unsigned long long free = ~seen;
        while (rank--) free &= free - 1;
        take = __builtin_ctzll(free);
    }
    const int dst = slot_idx[(size_t)n * W + take];
    if (blockIdx.x == 0 && threadIdx.x == 0) slot_out[(size_t)n * W + w] = dst;
    if (take == p || !valid) return;
    const int src = slot_idx[(size_t)n * W + p];
    if (src < 0 || src >= num_slots || dst < 0 || dst >= num_slots) return;
    const bool in_s = (int)blockIdx.x < s_pieces;
    char* pool = in_s ? S : P;
    const size_t bytes = in_s ? s_bytes : p_bytes;
    const size_t at = (size_t)(in_s ? blockIdx.x : blockIdx.x - s_pieces) * COPY_PIECE;
    copy_piece(pool + (size_t)src * bytes + at, pool + (size_t)dst * bytes + at,
               min(COPY_PIECE, bytes - at));
}

struct Plan {
    int pieces, tiles;
};

// Pieces of a row: one per tile, as long as a lane each suffices to join them and all rows together
// stay near 8192 wavefronts (32 per CU).
Plan plan(int rows, int V)
{
    const int all = (V + TILE - 1) / TILE;
    int pieces = 8192 / rows;
    pieces = pieces < 1 ? 1 : pieces > MAX_PIECES ? MAX_PIECES : pieces;
    pieces = pieces > all ? all : pieces;
    const int tiles = (all + pieces - 1) / pieces;
    return {(all + tiles - 1) / tiles, tiles};
}

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

size_t beam_workspace_bytes(int N, int W, int V)
{
    const Plan p = plan(N * W, V);
    const size_t lists = (size_t)N * W * p.pieces;
    return up256(lists * sizeof(float2)) + up256(lists * W * sizeof(Entry));
}

hipError_t launch_beam_select(const void* logits, const float* scores, const uint8_t* done, int N,
                              int W, int V, kdn_dtype_t dtype, int end_token, float* scores_out,
                              int32_t* token_out, int32_t* parent_out, uint8_t* done_out,
                              void* workspace, hipStream_t stream)
{
    const Plan p = plan(N * W, V);
    float2* stats = (float2*)workspace;
    Entry* best = (Entry*)((char*)workspace + up256((size_t)N * W * p.pieces * sizeof(float2)));
    const dim3 grid((unsigned)p.pieces, (unsigned)(N * W));
    if (dtype == KDN_F32)
        hipLaunchKernelGGL((beam_piece_kernel<float>), grid, dim3(64), 0, stream,
                           (const float*)logits, done, W, V, p.tiles, stats, best);
    else
        hipLaunchKernelGGL((beam_piece_kernel<bf16>), grid, dim3(64), 0, stream,
                           (const bf16*)logits, done, W, V, p.tiles, stats, best);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // as many wavefronts as rows, up to eight, while their piece tables fit beside the lists (at
    // most 32 KB each) in 64 KB
    const size_t table = (size_t)p.pieces * W * sizeof(Entry), lists = (size_t)W * W * sizeof(Entry);
    size_t waves = (65536 - lists) / table;
    waves = waves < 1 ? 1 : waves > 8 ? 8 : waves;
    waves = waves > (size_t)W ? W : waves;
    hipLaunchKernelGGL(beam_join_kernel, dim3((unsigned)N), dim3((unsigned)waves * 64),
                       lists + waves * table, stream, scores, done, W, V, end_token, p.pieces, stats,
                       best, scores_out, token_out, parent_out, done_out);
    return hipGetLastError();
}

hipError_t launch_beam_reorder(const int32_t* parent, const int32_t* slot_idx, int32_t* slot_out,
                               int N, int W, int num_slots, void* S, size_t s_bytes, void* P,
                               size_t p_bytes, hipStream_t stream)
{
    const size_t s_pieces = (s_bytes + COPY_PIECE - 1) / COPY_PIECE;
    const size_t p_pieces = P ? (p_bytes + COPY_PIECE - 1) / COPY_PIECE : 0;
    hipLaunchKernelGGL(beam_reorder_kernel, dim3((unsigned)(s_pieces + p_pieces), (unsigned)(N * W)),
                       dim3(256), 0, stream, parent, slot_idx, slot_out, W, num_slots, (char*)S,
                       s_bytes, (int)s_pieces, (char*)P, p_bytes);
    return hipGetLastError();
}

}  // namespace kdn
