// Tokens sorted by expert and back: the rows that the products by group take, made from tokens and the experts chosen for them.
//
// Slot s = t k + j is the j-th choice of token t.  A stable counting sort puts the slots in the order of their experts; row r of the
// sorted matrix belongs to slot order[r], and place[s] is the row of slot s, or its bitwise complement where the slot takes no
// part.  Everything after the sort goes by token: a token's row is read once and written k times on the way there, its k
// rows are read and summed in registers, in the order of the choices, on the way back.  No atomics on results: the same bits every time.
//
// What bounds them: the sort its launches, the others HBM (each row of either side is touched once).
#pragma once

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "cocod_grouped_sm100.cuh"

namespace cocod {
namespace lm {

constexpr int ERR_EXPERT = 102;              // error_flag: an expert's number beyond their count
constexpr int ERR_PLACE = 103;               // error_flag: a place beyond the rows

// ------------------------------------------------------------------------------------------ the sort
constexpr int SORT_WARPS = 16, SORT_THREADS = 32 * SORT_WARPS;

struct ExpertSlots {
    const int *experts;
    long long ld;                            // row stride
    int top, total, experts_n;               // slots of a token, all slots, experts
    int *error_flag;
};
// The bucket of slot s: its expert, or the one behind the last for slots that take no part.
__device__ __forceinline__ int bucket_of(const ExpertSlots &p, int s, bool tell)
{
    const long long at = p.ld == p.top ? (long long)s : (long long)(s / p.top) * p.ld + s % p.top;
    int e = p.experts[at];
    if (e >= p.experts_n && tell) atomicExch(p.error_flag, ERR_EXPERT);
    return e < 0 || e >= p.experts_n ? p.experts_n : e;
}

// Thread block b counts its slots b * span .. of each bucket.  before[b]: what the blocks before it in its cluster hold; totals[c]: what cluster c holds.
constexpr int SORT_CLUSTER = 8;
static __global__ void __cluster_dims__(SORT_CLUSTER, 1, 1) __launch_bounds__(SORT_THREADS)
expert_count(const ExpertSlots p, int span, int *before, int *totals)
{
    extern __shared__ int sums[];
    namespace cg = cooperative_groups;
    auto cluster = cg::this_cluster();
    pdl_launch_dependents();
    const int buckets = p.experts_n + 1;
    for (int e = threadIdx.x; e < buckets; e += SORT_THREADS) sums[e] = 0;
    pdl_wait();
    __syncthreads();
    const long long from = (long long)blockIdx.x * span, to = min(from + span, (long long)p.total);
    for (long long s = from + threadIdx.x; s < to; s += SORT_THREADS) atomicAdd(&sums[bucket_of(p, (int)s, false)], 1);
    cluster.sync();
    const int rank = blockIdx.x % SORT_CLUSTER;
    for (int e = threadIdx.x; e < buckets; e += SORT_THREADS) {
        int n[SORT_CLUSTER - 1], sum = 0;
#pragma unroll
        for (int r = 0; r < SORT_CLUSTER - 1; ++r) n[r] = r < rank ? cluster.map_shared_rank(sums, r)[e] : 0;
#pragma unroll
        for (int r = 0; r < SORT_CLUSTER - 1; ++r) sum += n[r];
        before[blockIdx.x * buckets + e] = sum;
        if (rank == SORT_CLUSTER - 1) totals[blockIdx.x / SORT_CLUSTER * buckets + e] = sum + sums[e];
    }
    cluster.sync();                          // (the others' counts are read until here)
}

// The lanes with the same bucket, by the bits of its number (64 experts: 7 votes).
__device__ __forceinline__ unsigned peers_of(int bucket, int bits)
{
    unsigned peers = ~0u;
    for (int b = 0; b < bits; ++b) {
        const bool one = bucket >> b & 1;
        const unsigned ones = __ballot_sync(~0u, one);
        peers &= one ? ones : ~ones;
    }
    return peers;
}

// Thread block b puts its slots into place.  A warp takes a stretch of them, 32 at a time; those of one bucket find each other,
// so that a slot's row is: the bucket's first row + what blocks, warps and tiles before hold of the bucket + how many lanes
// before it.  block_before, totals: expert_count's, not looked at where there is only one block.
static __global__ void __launch_bounds__(SORT_THREADS)
expert_place(const ExpertSlots p, int span, int bits, const int *block_before, const int *totals, int *offsets, int *per_expert, int *order, int *place)
{
    extern __shared__ int shared[];
    pdl_launch_dependents();
    const int buckets = p.experts_n + 1, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int *mine = shared + warp * buckets, *all = shared + SORT_WARPS * buckets, *before = all + buckets;
    for (int i = threadIdx.x; i < (SORT_WARPS + 2) * buckets; i += SORT_THREADS) shared[i] = 0;
    pdl_wait();
    __syncthreads();
    const int stretch = span / SORT_WARPS;
    const long long from = (long long)blockIdx.x * span + (long long)warp * stretch, to = min(from + stretch, (long long)p.total);
    constexpr int AT_ONCE = 4;
    for (long long s0 = from; s0 < to; s0 += 32 * AT_ONCE) {
        int e[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) e[u] = s0 + 32 * u + lane < to ? bucket_of(p, (int)(s0 + 32 * u + lane), true) : -1;
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u)
            if (e[u] >= 0) atomicAdd(&mine[e[u]], 1);
    }
    if (gridDim.x > 1) {                     // (all threads add up the clusters' counts)
        const int parts = max(1, SORT_THREADS / buckets), clusters = gridDim.x / SORT_CLUSTER, own = blockIdx.x / SORT_CLUSTER;
        for (int i = threadIdx.x; i < parts * buckets; i += SORT_THREADS) {
            const int e = i % buckets, part = i / buckets;
            int sum = 0, early = part == 0 ? block_before[blockIdx.x * buckets + e] : 0;
#pragma unroll 10
            for (int c = part; c < clusters; c += parts) {
                const int n = totals[c * buckets + e];
                sum += n;
                if (c < own) early += n;
            }
            atomicAdd(&all[e], sum);
            atomicAdd(&before[e], early);
        }
    }
    __syncthreads();
    if (gridDim.x == 1) {
        for (int e = threadIdx.x; e < buckets; e += SORT_THREADS) {
            int sum = 0;
            for (int w = 0; w < SORT_WARPS; ++w) sum += shared[w * buckets + e];
            all[e] = sum;
        }
        __syncthreads();
    }
    if (warp == 0) {                         // the buckets' first rows
        int carry = 0;
        for (int e0 = 0; e0 < buckets; e0 += 32) {
            const int e = e0 + lane, n = e < buckets ? all[e] : 0;
            int sum = n;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const int o = __shfl_up_sync(~0u, sum, d);
                if (lane >= d) sum += o;
            }
            const int first = carry + sum - n;
            if (e < buckets) before[e] += first;
            if (blockIdx.x == 0 && e < p.experts_n) {
                offsets[e] = first;
                per_expert[e] = n;
            }
            carry += __shfl_sync(~0u, sum, 31);
        }
        if (blockIdx.x == 0 && lane == 0) offsets[p.experts_n] = p.total;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < buckets; e += SORT_THREADS) {
        int at = before[e];
        for (int w = 0; w < SORT_WARPS; ++w) {
            const int n = shared[w * buckets + e];
            shared[w * buckets + e] = at;
            at += n;
        }
    }
    __syncthreads();
    for (long long s0 = from; s0 < to; s0 += 32 * AT_ONCE) {
        int e[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) e[u] = s0 + 32 * u + lane < to ? bucket_of(p, (int)(s0 + 32 * u + lane), false) : -1;
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const unsigned peers = peers_of(e[u] >= 0 ? e[u] : buckets, bits);        // (slots behind the end: a bucket of their own)
            const int s = (int)(s0 + 32 * u + lane);
            const int row = e[u] >= 0 ? mine[e[u]] + __popc(peers & ((1u << lane) - 1)) : 0;
            __syncwarp();
            if (e[u] >= 0 && row < p.total) {        // (always, unless the numbers change while they are sorted)
                if (lane == __ffs(peers) - 1) mine[e[u]] += __popc(peers);
                order[row] = s;
                place[s] = e[u] < p.experts_n ? row : ~row;
            }
            __syncwarp();
        }
    }
}

// ------------------------------------------------------------------------------------------ rows
// A piece is what a thread moves at once: 16 bytes where all rows start at multiples of 16 and hold a whole number of them, else one value.
template <typename T, bool WIDE> struct Piece;
template <typename T> struct Piece<T, true> {
    static constexpr int N = 16 / sizeof(T);
    uint4 raw;
};
template <typename T> struct Piece<T, false> {
    static constexpr int N = 1;
    T raw;
};
template <typename T, bool WIDE>
__device__ __forceinline__ Piece<T, WIDE> load_piece(const T *p)
{
    Piece<T, WIDE> r;
    r.raw = *reinterpret_cast<const decltype(r.raw) *>(p);      // (an ordinary load: a read-only one of bf16 is assembly that may be moved before its condition)
    return r;
}
template <typename T, bool WIDE>
__device__ __forceinline__ void store_piece(T *p, const Piece<T, WIDE> &r) { *reinterpret_cast<decltype(r.raw) *>(p) = r.raw; }
template <typename T, bool WIDE>
__device__ __forceinline__ Piece<T, WIDE> zero_piece()
{
    Piece<T, WIDE> r;
    memset(&r, 0, sizeof(r));
    return r;
}
__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T, bool WIDE>
__device__ __forceinline__ void widen(const Piece<T, WIDE> &r, float (&x)[Piece<T, WIDE>::N])
{
    if constexpr (!WIDE) {
        x[0] = as_float(r.raw);
    } else if constexpr (sizeof(T) == 4) {
        x[0] = __uint_as_float(r.raw.x); x[1] = __uint_as_float(r.raw.y); x[2] = __uint_as_float(r.raw.z); x[3] = __uint_as_float(r.raw.w);
    } else {
        const uint32_t w[4] = {r.raw.x, r.raw.y, r.raw.z, r.raw.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
}
// N values of fp32, rounded to T, to p (a multiple of N values' size where N > 1).
template <typename T, int N>
__device__ __forceinline__ void store_values(T *p, const float (&x)[N])
{
    if constexpr (sizeof(T) == 4) {
        if constexpr (N == 1) *p = x[0];
        else
#pragma unroll
            for (int i = 0; i < N; i += 4) *reinterpret_cast<float4 *>(p + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
    } else {
        if constexpr (N == 1) *p = __float2bfloat16_rn(x[0]);
        else if constexpr (N == 4) *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
        else
            *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
    }
}

constexpr int MAX_CHOICES = 32;              // of a token: a lane holds the place of each

struct ExpertRows {
    const int *place;                        // T x top, contiguous
    int tokens, top, rows;                   // rows = T * top
    int pieces;                              // of a row
    int *error_flag;
};
// Lane j's place, checked: whatever the tensor holds, nothing outside the rows is touched (row -1: nothing).
struct Slot {
    int row;
    bool there;
};
__device__ __forceinline__ Slot slot_of(const ExpertRows &p, int token, int lane)
{
    Slot s{-1, false};
    if (lane < p.top) {
        const int at = p.place[(long long)token * p.top + lane];
        s.there = at >= 0;
        s.row = at >= 0 ? at : ~at;
        if (s.row >= p.rows) {
            atomicExch(p.error_flag, ERR_PLACE);
            s = Slot{-1, false};
        }
    }
    return s;
}

// A warp takes ROW_PIECES x 32 pieces of a token's row and writes them to its k rows (zeros for a slot that takes no part).  With the sort before it, two pieces and
// four: 16384 x 4 of 2048 62.5 and 63.5 us, 100000 x 1 of 512 42.5 and 50.2, 64 x 8 of 2048 7.2 and 8.2; one piece 60.4 where two are 49.7 (65536 x 1 of 1024).
constexpr int ROW_PIECES = 2;
template <typename T, bool WIDE>
__global__ void __launch_bounds__(256)
expert_rows(const ExpertRows p, const T *x, long long ldx, T *out, long long ld_out)
{
    pdl_launch_dependents();
    pdl_wait();
    constexpr int N = Piece<T, WIDE>::N;
    const int lane = threadIdx.x & 31, parts = (p.pieces + 32 * ROW_PIECES - 1) / (32 * ROW_PIECES);
    const long long unit = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int token = (int)min(unit / parts, (long long)p.tokens);
    if (token >= p.tokens) return;
    const int first = (int)(unit - (long long)token * parts) * 32 * ROW_PIECES + lane;
    const Slot s = slot_of(p, token, lane);
    const T *row = x + (long long)token * ldx;
    Piece<T, WIDE> v[ROW_PIECES];
#pragma unroll
    for (int i = 0; i < ROW_PIECES; ++i)
        if (first + 32 * i < p.pieces) v[i] = load_piece<T, WIDE>(row + (long long)(first + 32 * i) * N);
    for (int j = 0; j < p.top; ++j) {
        const int r = __shfl_sync(~0u, s.row, j);
        const bool there = __shfl_sync(~0u, (int)s.there, j);
        if (r < 0) continue;
        T *to = out + (long long)r * ld_out;
#pragma unroll
        for (int i = 0; i < ROW_PIECES; ++i)
            if (first + 32 * i < p.pieces) store_piece<T, WIDE>(to + (long long)(first + 32 * i) * N, there ? v[i] : zero_piece<T, WIDE>());
    }
}

// The way back: y[t] = sum_j w[t][j] rows[place[t][j]] (weights == nullptr: the plain sum), fp32 in the order of j, in two forms with the same bits.  A warp takes
// PIECES x 32 pieces of one token, and U rows' pieces are under way together; BLOCKS of 256 threads share an SM (16384 x 8 of 2048, U = 4, two pieces: three blocks
// 95.8 us, four 91.7, one piece and six blocks 96.3, four 109; 65536 x 2 of 1024, U = 2: four blocks 78, five 73, six 77; 65536 x 1 of 1024, U = 1: eight blocks 50.7, four
// pieces and four blocks 49.1, but 54.8 against 39.4 at half the width; eight blocks of U = 1 spill 12 words with a bf16 result and 23 with fp32, and take 50.4 and 72.6, six 56.4 and 73.9 with two words).  A launch that leaves SMs idle takes one piece (64 x 8 of 2048, in a graph: 2.2 us instead of 2.6).
template <typename T, typename O, bool WIDE, int U, int PIECES, int BLOCKS>
__global__ void __launch_bounds__(256, BLOCKS)
expert_join_many(const ExpertRows p, const T *rows, long long ld, const float *weights, O *y, long long ldy)
{
    pdl_launch_dependents();
    pdl_wait();
    constexpr int N = Piece<T, WIDE>::N;
    const int lane = threadIdx.x & 31, parts = (p.pieces + 32 * PIECES - 1) / (32 * PIECES);
    const long long unit = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int token = (int)min(unit / parts, (long long)p.tokens);
    if (token >= p.tokens) return;
    const int first = (int)(unit - (long long)token * parts) * 32 * PIECES + lane;
    const Slot s = slot_of(p, token, lane);
    const float w = weights != nullptr && lane < p.top ? weights[(long long)token * p.top + lane] : 1.0f;
    float sum[PIECES][N];
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e) sum[i][e] = 0.0f;
    for (int j0 = 0; j0 < p.top; j0 += U) {
        Piece<T, WIDE> v[U][PIECES];
        bool there[U];
        float f[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = min(j0 + u, 31), r = __shfl_sync(~0u, s.row, j);
            there[u] = __shfl_sync(~0u, (int)s.there, j) && j0 + u < p.top;
            f[u] = __shfl_sync(~0u, w, j);
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
                if (there[u] && first + 32 * i < p.pieces) v[u][i] = load_piece<T, WIDE>(rows + (long long)r * ld + (long long)(first + 32 * i) * N);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!there[u]) continue;
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                float a[N];
                widen<T, WIDE>(v[u][i], a);
#pragma unroll
                for (int e = 0; e < N; ++e) sum[i][e] = fmaf(f[u], a[e], sum[i][e]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
        if (first + 32 * i < p.pieces) store_values<O, N>(y + (long long)token * ldy + (long long)(first + 32 * i) * N, sum[i]);
}

// One or two choices, where the rows' length would leave a quarter of those lanes idle: a thread takes PIECES pieces of tokens' rows, 256 apart, whatever the rows'
// length, and ROWS rows' pieces of each are under way together (30000 x 2 of 520: 21.5 us, the other form 28.2; of 1024 with 65536 tokens 81 and 73).
template <typename T, typename O, bool WIDE, int ROWS, int PIECES>
__global__ void __launch_bounds__(256, ROWS == 1 ? 6 : 8)
expert_join_few(const ExpertRows p, const T *rows, long long ld, const float *weights, O *y, long long ldy)
{
    pdl_launch_dependents();
    pdl_wait();
    constexpr int N = Piece<T, WIDE>::N;
    const long long first = (long long)blockIdx.x * (256 * PIECES), token0 = first / p.pieces;
    const unsigned begin = (unsigned)(first - token0 * p.pieces) + threadIdx.x;
    long long token[PIECES], at[PIECES];
    float sum[PIECES][N];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const unsigned local = begin + 256 * i, ahead = local / (unsigned)p.pieces;
        token[i] = token0 + ahead;
        at[i] = (long long)(local - ahead * p.pieces) * N;
#pragma unroll
        for (int e = 0; e < N; ++e) sum[i][e] = 0.0f;
    }
    for (int j0 = 0; j0 < p.top; j0 += ROWS) {
        int row[PIECES][ROWS];
        float f[PIECES][ROWS];
        Piece<T, WIDE> v[PIECES][ROWS];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
#pragma unroll
            for (int u = 0; u < ROWS; ++u) {
                const bool there = token[i] < p.tokens && j0 + u < p.top;
                row[i][u] = there ? p.place[token[i] * p.top + j0 + u] : -1;
                f[i][u] = there && weights != nullptr ? weights[token[i] * p.top + j0 + u] : 1.0f;
            }
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
#pragma unroll
            for (int u = 0; u < ROWS; ++u) {
                if (row[i][u] >= p.rows || ~row[i][u] >= p.rows) {
                    atomicExch(p.error_flag, ERR_PLACE);
                    row[i][u] = -1;
                }
                if (row[i][u] >= 0) v[i][u] = load_piece<T, WIDE>(rows + row[i][u] * ld + at[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
#pragma unroll
            for (int u = 0; u < ROWS; ++u) {
                if (row[i][u] < 0) continue;
                float a[N];
                widen<T, WIDE>(v[i][u], a);
#pragma unroll
                for (int e = 0; e < N; ++e) sum[i][e] = fmaf(f[i][u], a[e], sum[i][e]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
        if (token[i] < p.tokens) store_values<O, N>(y + token[i] * ldy + at[i], sum[i]);
}

// The gradient of that: back[place[t][j]] = w[t][j] dy[t] (0 where the slot takes no part), dw[t][j] = <dy[t], rows[place[t][j]]>.
// WARPS warps take a token; each sum runs over a thread's pieces, the lanes and the warps, always in the same order.
// The loads of a piece of U slots are under way together.  Blocks that share an SM: U = 4, four (16384 x 8 of 2048: 176 us, three 198, five 187); U = 2, of one or two
// choices, six, for which up to twelve words are spilled (100000 x 1 of 512: 65 us, with five blocks and two words 70, with U = 4 82).  U = 8 was behind at all sizes: 184.
template <typename T, bool WIDE, int WARPS, int U>
__global__ void __launch_bounds__(256, U == 2 ? 6 : 4)
expert_join_grad(const ExpertRows p, const T *dy, long long lddy, const T *rows, long long ld, const float *weights, T *back, long long ld_back, float *dw)
{
    pdl_launch_dependents();
    pdl_wait();
    constexpr int N = Piece<T, WIDE>::N;
    __shared__ float part[8][MAX_CHOICES];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, of = warp % WARPS;
    const int token = blockIdx.x * (8 / WARPS) + warp / WARPS;
    if (token < p.tokens) {
        const Slot s = slot_of(p, token, lane);
        const float w = lane < p.top ? weights[(long long)token * p.top + lane] : 0.0f;
        const T *d_row = dy + (long long)token * lddy;
        for (int j0 = 0; j0 < p.top; j0 += U) {
            float sum[U], f[U];
            int r[U];
            unsigned there = __ballot_sync(~0u, s.there) >> j0;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = min(j0 + u, 31);
                sum[u] = 0.0f;
                r[u] = __shfl_sync(~0u, s.row, j);
                if (j0 + u >= p.top) r[u] = -1;
                if (r[u] < 0) there &= ~(1u << u);
                f[u] = __shfl_sync(~0u, w, j);
            }
            for (int c = of * 32 + lane; c < p.pieces; c += 32 * WARPS) {
                const long long at = (long long)c * N;
                const Piece<T, WIDE> d = load_piece<T, WIDE>(d_row + at);
                Piece<T, WIDE> v[U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (there >> u & 1) v[u] = load_piece<T, WIDE>(rows + (long long)r[u] * ld + at);
                float g[N];
                widen<T, WIDE>(d, g);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (r[u] < 0) continue;
                    const bool here = there >> u & 1;
                    float out[N];
                    if (here) {
                        float a[N];
                        widen<T, WIDE>(v[u], a);
#pragma unroll
                        for (int e = 0; e < N; ++e) sum[u] = fmaf(g[e], a[e], sum[u]);
                    }
#pragma unroll
                    for (int e = 0; e < N; ++e) out[e] = here ? f[u] * g[e] : 0.0f;
                    store_values<T, N>(back + (long long)r[u] * ld_back + at, out);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
                for (int d = 16; d > 0; d /= 2) sum[u] += __shfl_xor_sync(~0u, sum[u], d);
                if (lane == 0 && j0 + u < p.top) part[warp][j0 + u] = sum[u];
            }
        }
    }
    __syncthreads();
    if (token < p.tokens && of == 0 && lane < p.top) {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < WARPS; ++i) sum += part[warp + i][lane];
        dw[(long long)token * p.top + lane] = sum;
    }
}

}  // namespace lm
}  // namespace cocod
