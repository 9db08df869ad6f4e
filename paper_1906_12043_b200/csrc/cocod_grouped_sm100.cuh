// Products of rows that belong to groups (the workers' mini-batches, of unequal sizes) with each group's own matrix, on
// the tensor cores of sm_100a.  Row m belongs to group g when offsets[g] <= m < offsets[g + 1]; the offsets live on the
// device, so a launch does not know how its rows are divided and finds its tiles itself.
//
//   rows form    out[m][n]    = sum_k A[m][k] B_g(n, k)      forward (B_g stored [n][k]) and input gradient (stored [k][n])
//   weight form  out_g[i][j]  = sum_{m in g} A[m][i] B[m][j] weight gradient; the reduction runs over the group's rows
//
// One persistent, warp-specialised kernel serves all forms:
//   * A tile is 256 x 256, computed by a PAIR of CTAs (cta_group::2): each holds 128 rows of A and 128 columns of B per
//     64-deep block of the reduction (32 KB a stage, six stages), so a pair moves 64 bytes per SM and clock for tensor
//     cores that need 512 clocks for the block.  Problems with few tiles use 128 x 128 tiles and single CTAs (CG = 1): twice
//     the bytes for a product, but more SMs take part.
//   * Two accumulators in tensor memory: the epilogue of a tile runs under the products of the next.
//   * Warps: 0 producer (TMA), 1 issuer of tcgen05.mma (leading CTA of the pair only), 2 tensor memory and groups' last blocks, 3 scheduler, 4..11 epilogue.
//     The scheduler reads the tile list (Walker) some tiles ahead and leaves them in shared memory; when every role found
//     its tiles itself, the producer's pause for it emptied the ring: 3000 clocks a tile.
//   * An epilogue warp owns 32 rows of its CTA's tile and half of the columns, stages them in shared memory of its own
//     (4 KB, TMA swizzle) and hands them to the store engine; rows behind the end of a group are some other group's, so a
//     warp whose rows end inside a group's last tile stores the valid ones itself.
// The tensor cores cut the accumulator's last bits off with every step they add: the sum of 2048 products came out 2.1e-6 too
// small, four times fp32's rounding error, and the loss grows with the length.  Where the result leaves as fp32, a reduction
// is therefore cut into parts of 768 (logits: 2048): each goes to the other accumulator, and the epilogue adds it, rounding to
// nearest, to sums that it holds in registers (half a tile row per thread; the epilogue warps take the registers that the
// others give up).  8192 x 8192 x 8192 in fp32: 774 us without, 788 in parts of 1024, 823 in parts of 512 (the epilogue's
// reads of tensor memory hold the products up for about 400 clocks a part); error 7e-7 at 768, 1.0e-6 at 1024.  A bf16 result does not show
// the difference below some 100000 products (1e-4 at that rate): its parts are of 32768, which cost nothing.
// Reductions end where the matrices do: TMA fills what lies outside with zeros.  In the weight form the reduction ends
// with the group, and behind its last row lie the next group's, which may hold anything: where a group's last block of 64 rows
// holds some, its copies complete at a barrier of their own CTA (rfull), warp 2 overwrites those rows with zeros as far as the last step of 16
// products reaches that the issuer takes of the block, and hands it on (rready).
// The weight gradient can take B as an 8-bit checkpoint (B_Q8): TMA brings the bytes, warp 2 their scales, and eight more warps write
// the bf16 operand tile, exactly (a whole number times a power of two), with zeros behind the group's end (and zeros into A there).
// The number of tiles is seldom a multiple of the CTA pairs.  The tiles of the last, incomplete wave (all of them when there are few)
// are cut along the reduction into as many parts as keep every pair busy; a part leaves as fp32 in scratch, at most one per
// pair, and join_parts adds the parts of a tile up in a fixed order.  5.2 waves of tiles take 5.2 and not 6 times a tile.
// Every wait is bounded, as in cocod_gemm_sm100.cuh.
//
// What bounds it.  Large products: the GPU's power limit.  8192 x 65536 x 2048 back to back takes 1650 us forward (1333 TFLOP/s; SM clock 1387
// MHz in the median, 993 W, the power cap active in every sample; cuBLAS in the same process 1644), 1803 as an input gradient, 1702 as a
// weight gradient.  All zeros, which switch less, take 1170 us at 1935 MHz: the same number of clocks.  Small ones: the launch, the pipeline's filling and the
// last wave (24 rows in 4 groups, 512 x 512: 6.8 us, of which 3.5 are a kernel without tiles).  Few rows with much to write: DRAM (16 workers
// of 16 to 128 rows, a 16777216-value gradient each: 125 us, 4.3 TB/s of writes).
#pragma once
#include "cocod_act8.cuh"
#include "cocod_gemm_sm100.cuh"

namespace cocod {
namespace lm {

using namespace cocod::gemm;

enum Operand { B_K = 0, B_MN = 1, B_Q8 = 2 };                       // B: reduction innermost; second; second and in 8 bits

constexpr int EPI_WARPS = 8, CONV_WARPS = 8;
__host__ __device__ constexpr int grouped_threads(int b) { return 128 + 32 * EPI_WARPS + (b == B_Q8 ? 32 * CONV_WARPS : 0); }
constexpr int Q_BYTES = 64 * 128;                                   // 8-bit values of a block of the reduction
__host__ __device__ constexpr int ring(int b) { return b == B_Q8 ? 4 : 6; }                  // stages
__host__ __device__ constexpr int stage_bytes(int b) { return STAGE_BYTES + (b == B_Q8 ? Q_BYTES : 0); }
constexpr int OUT_BYTES = 4096;                                     // staging of an epilogue warp: 32 rows of 128 bytes
constexpr int AHEAD = 4;                                            // tiles that the scheduler may be ahead
constexpr int GROUPED_SMEM = 6 * STAGE_BYTES + EPI_WARPS * OUT_BYTES + 1024 + 1024;
static_assert(ring(B_Q8) * stage_bytes(B_Q8) <= 6 * STAGE_BYTES, "the stages with 8-bit values take the same room");
// Registers per thread: what a launch holds, and what the warps 0..3, the epilogue and the converting warps keep of it.
__host__ __device__ constexpr int launch_registers(int b) { return b == B_Q8 ? 96 : 168; }
__host__ __device__ constexpr int few_registers(int b) { return b == B_Q8 ? 48 : 64; }
__host__ __device__ constexpr int epilogue_registers(int b) { return b == B_Q8 ? 160 : 216; }
constexpr int CONV_REGISTERS = 56;
static_assert(128 * few_registers(B_K) + 32 * EPI_WARPS * epilogue_registers(B_K) <= grouped_threads(B_K) * launch_registers(B_K), "a warp would wait for ever");
static_assert(128 * few_registers(B_Q8) + 32 * CONV_WARPS * CONV_REGISTERS + 32 * EPI_WARPS * epilogue_registers(B_Q8) <=
              grouped_threads(B_Q8) * launch_registers(B_Q8), "a warp would wait for ever");
constexpr int ERR_OFFSETS = 100;                                    // error_flag: the offsets do not rise from 0 to the number of rows
constexpr int ERR_LABEL = 101;                                      // error_flag: a label beyond the vocabulary

enum Out {
    OUT_BF16 = 0,
    OUT_F32 = 1,
    OUT_ADD_F32 = 2,       // added to what is there
    // rows form, the vocabulary's logits l = h w^T: nothing of l is written, but for every row r with reference c_r and label t_r
    OUT_VOCAB = 3,         // u[r][v] = exp(l - c_r) in bf16, 0 at v = t_r, and for each half of a tile sum_v u (in fp32) and max_v l, v != t_r
    OUT_VOCAB_SUMS = 4,    // only the sums and maxima
};
__host__ __device__ constexpr bool is_f32(int out) { return out == OUT_F32 || out == OUT_ADD_F32; }
__host__ __device__ constexpr bool is_vocab(int out) { return out == OUT_VOCAB || out == OUT_VOCAB_SUMS; }
// Blocks of 64 that the tensor cores sum at a time.
__host__ __device__ constexpr int part_blocks(int out) { return is_f32(out) ? 12 : is_vocab(out) ? 32 : 512; }

struct GroupedParams {
    const int *offsets;                // [groups + 1], device
    int groups;
    int total_rows;                    // offsets[groups] has to be this
    int row0, rows;                    // this launch takes rows row0 .. row0 + rows - 1; A and out start at row row0
    int n;                             // columns of out
    int kdim;                          // rows form: length of the reduction.  Weight form: rows of out_g
    int tiles_n;
    int band;                          // tile rows that are walked together, column by column
    int max_parts;                     // a tile of the last wave is cut into at most this many parts (1: none is)
    void *out;                         // for the rows of a partial tile, and for join_parts
    long long ld_out, out_stride;      // elements; out_stride (weight form): between groups
    const float *row_scale;            // rows form, optional: factor of every row (0: the row is 0 whatever the product is)
    const float *rest;                 // rows form with row_scale, optional: row r gets rest[r] B_g(., label[r]) added before the factor
    const __nv_bfloat16 *rest_b;       // with rest: B, stored [reduction][n]
    long long ld_b, b_stride;
    const int *order;                  // weight form: the groups, those with the most rows first; nullptr: a warp finds it (up to 32)
    const uint8_t *scales;             // B_Q8: [ceil(n / 128)][total_rows], exponents + 127
    // OUT_VOCAB, OUT_VOCAB_SUMS (rows counted from row0; label: also with rest)
    const float *ref;                  // c_r
    const int *label;                  // t_r; negative: the row takes no part (u = 0)
    float2 *sums;                      // [half tiles][ld_sums]: {sum, max}
    int ld_sums;
    const int *redo;                   // optional: only tiles with a row whose entry is not 0, and nothing at all if *redo_any is 0
    const int *redo_any;
    int *error_flag;
    unsigned long long wait_ns;        // 0 = WAIT_LIMIT_NS
    int debug_no_loads;                // self-test: the producer issues nothing
};

// ------------------------------------------------------------------------------------------ PTX wrappers
__device__ __forceinline__ void mbar_arrive_local(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t map_to_rank(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
// Arrive at a barrier of the pair, given by its shared::cluster address, when an accumulator has been read.  It orders this thread's
// accesses within the CTA only: what is handed over is tensor memory, whose reads are complete.  (Release at cluster scope took
// 1200 to 2000 clocks: it waits for the epilogue's global stores.)
__device__ __forceinline__ void mbar_arrive_accumulator(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Where the second CTA of a pair hands over shared memory that it wrote and the leading CTA's products read, the signal is a release at cluster
// scope, and the wait acquires at cluster scope.  The signal is an asynchronous store of a word that nobody reads, for the release that
// its completion at the barrier brings: the warp goes on at once.  (mbarrier.arrive.release.cluster waits for a round trip instead: a weight
// gradient of 2048 cubed from a checkpoint 41.7 us, this way 29.7.)
constexpr int SIGNAL_BYTES = 4;
__device__ __forceinline__ void signal_operand(uint32_t word, uint32_t bar)      // both: shared::cluster addresses in the leading CTA
{
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.u32 [%0], %1, [%2];" ::"r"(word), "r"(0), "r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try_operand(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool mbar_wait_operand(uint32_t bar, uint32_t parity, volatile int *abort, unsigned long long limit_ns)
{
    if (mbar_try_operand(bar, parity)) return true;
    const unsigned long long t0 = now_ns();
    for (unsigned it = 0;; ++it) {
        if (mbar_try_operand(bar, parity)) return true;
        if ((it & 63u) == 63u && (*abort || now_ns() - t0 > limit_ns)) return false;
    }
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// A tile load of one CTA of a pair; its bytes are counted at `bar` (a shared::cluster address: the leading CTA's barrier).
template <int CG>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y, int z)
{
    if (CG == 1)
        tma_load_3d(dst, map, bar, x, y, z);
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 "
                     "[%0], [%1, {%3, %4, %5}], [%2];"
                     ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void tma_add_3d(const CUtensorMap *map, uint32_t src, int x, int y, int z)
{
    asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.bulk_group [%0, {%2, %3, %4}], [%1];"
                 ::"l"(map), "r"(src), "r"(x), "r"(y), "r"(z) : "memory");
}
template <int CG> __device__ __forceinline__ void tmem_alloc_g(uint32_t slot, uint32_t cols)
{
    if (CG == 1) {
        tmem_alloc(slot, cols);
        tmem_relinquish();
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
}
template <int CG> __device__ __forceinline__ void tmem_dealloc_g(uint32_t taddr, uint32_t cols)
{
    if (CG == 1) tmem_dealloc(taddr, cols);
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(cols) : "memory");
}
template <int CG>
__device__ __forceinline__ void umma_g(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    if (CG == 1)
        umma_bf16(tmem_d, adesc, bdesc, idesc, accumulate);
    else
        asm volatile("{\n\t.reg .pred p;\n\t"
                     "setp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
// Arrive at the barrier (in both CTAs of a pair) once all products issued so far are complete.
template <int CG> __device__ __forceinline__ void umma_commit_g(uint32_t bar)
{
    if (CG == 1)
        umma_commit(bar);
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"((uint16_t)3) : "memory");
}
// Registers per thread from here on, for all warps of a warpgroup.
template <int N> __device__ __forceinline__ void give_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int CG> __device__ __forceinline__ uint32_t cta_rank()
{
    if (CG == 1) return 0;
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// Instruction descriptor: fp32 accumulator, bf16 operands, M = 128 per CTA, operand majors as given.
template <int CG, int TN, bool A_MN, bool B_MN> __host__ __device__ constexpr uint32_t grouped_idesc()
{
    return (1u << 4) | (1u << 7) | (1u << 10) | ((A_MN ? 1u : 0u) << 15) | ((B_MN ? 1u : 0u) << 16) |
           ((uint32_t)(TN >> 3) << 17) | ((uint32_t)(128 * CG >> 4) << 24);
}

// ------------------------------------------------------------------------------------------ tiles
struct __align__(16) Tile {
    int g;             // group; negative: there are no more tiles
    int m0, m1;        // rows form: first row of the tile, end of the group (both counted from row0).  Weight form: first row of out_g,
                       // end of the group
    int n0;            // first column
    int kb0, kb1;      // blocks of the reduction (64 each)
    int slot;          // negative: a whole tile; else a part of one, number `slot` in the scratch
    int lo;            // weight form: the group's first row
};

// Rows of group g within this launch, counted from row0; any content of offsets gives a range inside [0, rows].
__device__ __forceinline__ void group_range(const GroupedParams &p, int g, int &lo, int &hi)
{
    lo = min(max(p.offsets[g] - p.row0, 0), p.rows);
    hi = min(max(p.offsets[g + 1] - p.row0, lo), p.rows);
}

// Weight form: the end of the tile's blocks that hold rows of its group alone.  The next one, if it is in the tile, holds rows of the next
// group too (behind the batch's last row TMA writes zeros).
__device__ __forceinline__ int plain_blocks(const GroupedParams &p, const Tile &t)
{
    return t.m1 < p.rows ? min(t.kb1, (t.m1 - t.lo) / BK) : t.kb1;
}

// The place of group g when the groups are ordered by their rows, most first (one warp).
__device__ __forceinline__ int group_rank(const GroupedParams &p, int g)
{
    int lo, hi, rank = 0;
    group_range(p, g, lo, hi);
    const int mine = hi - lo;
    for (int j = threadIdx.x & 31; j < p.groups; j += 32) {
        group_range(p, j, lo, hi);
        rank += hi - lo > mine || (hi - lo == mine && j < g);
    }
    return __reduce_add_sync(0xffffffffu, rank);
}

// Within a group, tiles go in bands of tile rows, column by column: the CTAs that run at the same time share their operands
// through L2.
__device__ __forceinline__ void in_band(int i, int high, int tiles_m, int tiles_n, int &tm, int &tn)
{
    const int band = i / (high * tiles_n), r = i - band * high * tiles_n;
    const int here = min(high, tiles_m - band * high);
    tn = r / here;
    tm = band * high + r - tn * here;
}

// The list of a launch, read in rising order by a whole warp: first the tiles of the complete waves, then the parts of the last
// wave's tiles, then (weight form) the tiles of groups without rows.  In the rows form a group has as many tile rows as its rows
// fill; 32 groups are looked at together, one per lane.
template <int TM, int TN, bool WG> struct Walker {
    const GroupedParams &p;
    int lane, gb = 0, base = 0, lo = 0, hi = 0, cnt = 0, incl = 0, total = 0, rank = 0;
    int whole = 0x7fffffff, cut = 0, parts = 1;
    __device__ Walker(const GroupedParams &params, int lane_, int clusters) : p(params), lane(lane_)
    {
        int tiles = 0;
        bool loaded = false;
        if (WG) {
            for (int g0 = 0; g0 < p.groups; g0 += 32) {
                if (g0 + lane < p.groups) group_range(p, g0 + lane, lo, hi);
                tiles += __popc(__ballot_sync(0xffffffffu, g0 + lane < p.groups && hi > lo));
            }
            tiles *= (p.kdim + TM - 1) / TM * p.tiles_n;
            whole = tiles;
            if (p.order == nullptr) {                     // (group_rank with a group in each lane)
                const int mine = lane < p.groups ? hi - lo : -1;
                for (int j = 0; j < p.groups; ++j) {
                    const int rows = __shfl_sync(0xffffffffu, mine, j);
                    rank += rows > mine || (rows == mine && j < lane);
                }
            }
        } else if (p.max_parts > 1) {
            for (gb = 0; gb < p.groups; gb += 32) {
                load();
                tiles += total;
            }
            gb = 0;
            whole = tiles;
            loaded = p.groups <= 32;
        }
        if (p.max_parts > 1) {
            const int rest = tiles % clusters;
            parts = rest ? min(clusters / rest, p.max_parts) : 1;
            if (parts > 1) {
                cut = rest;
                whole = tiles - rest;
            }
        }
        if (!WG && !loaded) load();
    }
    __device__ void load()
    {
        const int g = gb + lane;
        lo = hi = cnt = 0;
        if (g < p.groups) {
            group_range(p, g, lo, hi);
            cnt = (hi - lo + TM - 1) / TM * p.tiles_n;
        }
        incl = cnt;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
        total = __shfl_sync(0xffffffffu, incl, 31);
    }
    __device__ bool find(int t, Tile &tile)
    {
        int part = 0, of = 1, tiles_m;
        tile.slot = -1;
        if (t >= whole) {
            const int u = t - whole;
            if (u < cut * parts) {
                part = u % parts;
                of = parts;
                tile.slot = u;
                t = whole + u / parts;
            } else if (WG) {
                t = whole + cut + u - cut * parts;
            } else {
                return false;
            }
        }
        if (WG) {
            tiles_m = (p.kdim + TM - 1) / TM;
            const int per = tiles_m * p.tiles_n, at = t / per;
            if (at >= p.groups) return false;
            tile.g = p.order != nullptr ? p.order[at] : __ffs(__ballot_sync(0xffffffffu, lane < p.groups && rank == at)) - 1;
            t -= at * per;
            group_range(p, tile.g, lo, hi);
        } else {
            while (t >= base + total) {
                base += total;
                gb += 32;
                if (gb >= p.groups) return false;
                load();
            }
            const int l = __ffs(__ballot_sync(0xffffffffu, t < base + incl)) - 1;
            tile.g = gb + l;
            t -= base + __shfl_sync(0xffffffffu, incl - cnt, l);
            tile.m0 = __shfl_sync(0xffffffffu, lo, l);
            tile.m1 = __shfl_sync(0xffffffffu, hi, l);
            tiles_m = (tile.m1 - tile.m0 + TM - 1) / TM;
        }
        int tm, tn;
        in_band(t, p.band, tiles_m, p.tiles_n, tm, tn);
        tile.n0 = tn * TN;
        int blocks;
        if (WG) {
            tile.m0 = tm * TM;
            tile.m1 = hi;
            tile.lo = lo;
            blocks = (hi - lo + BK - 1) / BK;
        } else {
            tile.m0 += tm * TM;
            blocks = (p.kdim + BK - 1) / BK;
        }
        tile.kb0 = (int)((long long)blocks * part / of);
        tile.kb1 = (int)((long long)blocks * (part + 1) / of);
        return true;
    }
};

// Whether a second pass over the logits takes this tile (all roles of both CTAs see the same).
template <int TM> __device__ __forceinline__ bool redo_tile(const GroupedParams &p, const Tile &t, int lane)
{
    bool any = false;
    for (int r = t.m0 + lane; r < min(t.m0 + TM, t.m1); r += 32) any |= p.redo[r] != 0;
    return __any_sync(0xffffffffu, any);
}

// Zeros into rows `first` .. end - 1 of each of BOXES boxes of 64 rows of 128 bytes, by `threads` threads.
template <int BOXES> __device__ __forceinline__ void zero_rows(uint8_t *boxes, int first, int end, int thread, int threads)
{
    const int pieces = (end - first) * 8;                      // of 16 bytes, in a box
    for (int i = thread; i < BOXES * pieces; i += threads) {
        const int box = i / pieces;
        *reinterpret_cast<uint4 *>(boxes + box * (BK * 128) + first * 128 + (i - box * pieces) * 16) = make_uint4(0, 0, 0, 0);
    }
}

__device__ __forceinline__ float exp2_approx(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// ------------------------------------------------------------------------------------------ kernel
// Tensor maps (all three-dimensional, innermost dimension contiguous, 128-byte swizzle):
//   A, B with the reduction innermost: boxes of 64 x 128 rows; A or B with it second: boxes of 64 x 64, two per operand; B in 8
//   bits: boxes of 128 x 64 rows, not swizzled.
//   out: boxes of 32 rows x 128 bytes; third index = group (weight form).  parts: the scratch as an fp32 matrix of TN columns, TM
//   rows for each part, boxes of 32 x 32.
template <int CG, int TN, bool WG, int B, int OUT>
__global__ void __launch_bounds__(grouped_threads(B), 1)
grouped_gemm(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
             const __grid_constant__ CUtensorMap map_out, const __grid_constant__ CUtensorMap map_parts, const GroupedParams p)
{
    constexpr int TM = 128 * CG, RING = ring(B), STAGE = stage_bytes(B);
    constexpr bool A_MN = WG, QB = B == B_Q8;
    static_assert(TN / CG == 128, "each CTA holds 128 columns of B");
    extern __shared__ uint8_t grouped_smem[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(grouped_smem) + 1023) & ~(uintptr_t)1023);
    uint8_t *outs = smem + RING * STAGE;
    uint64_t *bars = reinterpret_cast<uint64_t *>(outs + EPI_WARPS * OUT_BYTES);
    const uint32_t full0 = smem_u32(bars), empty0 = smem_u32(bars + RING), accf0 = smem_u32(bars + 2 * RING), acce0 = smem_u32(bars + 2 * RING + 2);
    const uint32_t tilef0 = smem_u32(bars + 2 * RING + 4), tilee0 = smem_u32(bars + 2 * RING + 4 + AHEAD);
    Tile *tiles = reinterpret_cast<Tile *>(bars + 2 * RING + 4 + 2 * AHEAD);
    uint64_t *bbars = reinterpret_cast<uint64_t *>(tiles + AHEAD);
    const uint32_t bfull0 = smem_u32(bbars), qfull0 = smem_u32(bbars + RING);      // B_Q8: the bf16 tile is written; bytes and scales are there
    const uint32_t rready0 = bfull0, rfull0 = qfull0;                              // else, weight form: the block is mended; its copies are there
    uint8_t *unit_bytes = reinterpret_cast<uint8_t *>(bbars + 2 * RING);           // B_Q8: scales of the 64 rows of every stage
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(unit_bytes + 64 * RING);
    volatile int *abort = reinterpret_cast<volatile int *>(tmem_slot + 1);
    uint32_t *words = tmem_slot + 2;                                               // weight form, pairs: where the other CTA's signals go
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cta_rank<CG>();
    const int cluster = blockIdx.x / CG, clusters = gridDim.x / CG;
    const uint32_t smem_base = smem_u32(smem);
    const unsigned long long limit = p.wait_ns ? p.wait_ns : WAIT_LIMIT_NS;

    if (is_vocab(OUT) && p.redo != nullptr) {     // a second pass over the logits that no row needs
        pdl_launch_dependents();
        pdl_wait();
        if (*p.redo_any == 0) return;
    }
    if (threadIdx.x == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_b) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_out) : "memory");
        for (int s = 0; s < RING; ++s) {
            mbar_init(full0 + 8 * s, 1);
            mbar_init(empty0 + 8 * s, 1);
            mbar_init(bfull0 + 8 * s, QB ? CONV_WARPS : 1);        // (and the signals of the other CTA of a pair)
            mbar_init(qfull0 + 8 * s, QB ? 2 : 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(accf0 + 8 * s, 1);
            mbar_init(acce0 + 8 * s, EPI_WARPS * CG);
        }
        for (int s = 0; s < AHEAD; ++s) {
            mbar_init(tilef0 + 8 * s, 1);
            mbar_init(tilee0 + 8 * s, 1 + (rank == 0 ? 1 : 0) + EPI_WARPS + (WG ? 1 : 0) + (QB ? CONV_WARPS : 0));      // producer, issuer, epilogue, warp 2, converters
        }
        *abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_smem();
    }
    if (warp == 2) tmem_alloc_g<CG>(smem_u32(tmem_slot), 2 * TN);
    tc_fence_before();
    __syncthreads();
    if (CG == 2) cluster_sync();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    pdl_launch_dependents();
    pdl_wait();

    int failed = 0;
    // The next tile in the scheduler's order, for one thread (the producer, the issuer) or a whole warp; false at the end of the
    // list (or when a wait gives up).
    unsigned turn = 0;
    auto read_tile = [&](Tile &t) {
        const int4 *src = reinterpret_cast<const int4 *>(tiles + turn++ % AHEAD);
        const int4 a = src[0], b = src[1];
        t.g = a.x; t.m0 = a.y; t.m1 = a.z; t.n0 = a.w;
        t.kb0 = b.x; t.kb1 = b.y; t.slot = b.z; t.lo = b.w;
    };
    auto next_tile = [&](Tile &t) {
        const unsigned s = turn % AHEAD;
        if (!mbar_wait(tilef0 + 8 * s, (turn / AHEAD) & 1, abort, limit)) { failed = 4; return false; }
        read_tile(t);
        mbar_arrive_local(tilee0 + 8 * s);
        return t.g >= 0;
    };
    auto next_tile_warp = [&](Tile &t) {
        const unsigned s = turn % AHEAD;
        if (!__all_sync(0xffffffffu, mbar_wait(tilef0 + 8 * s, (turn / AHEAD) & 1, abort, limit))) { failed = 4; return false; }
        read_tile(t);
        __syncwarp();
        if (lane == 0) mbar_arrive_local(tilee0 + 8 * s);
        return t.g >= 0;
    };
    if (warp >= 4 && warp < 4 + EPI_WARPS) {
        take_registers<epilogue_registers(B)>();
        // ---- epilogue: rows 32 (warp % 4) .. + 31 of the CTA's 128, columns of one half of the tile
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        uint8_t *staging = outs + (warp - 4) * OUT_BYTES;
        constexpr int HALF = TN / 2, CHUNK = is_f32(OUT) ? 32 : 64, CHUNKS = HALF / CHUNK;      // a chunk: 128 bytes of a row
        constexpr int ES = is_f32(OUT) ? 4 : 2, PER = 16 / ES;
        Tile t{};
        unsigned ai = 0;
        // A chunk at a time goes through the warp's staging.  (Room for two saved waits and cost a stage of the ring: 1 to 5 % slower.)
        auto staging_free = [&]() {
            if (lane == 0) tma_store_wait_read<0>();
            __syncwarp();
        };
        auto stage_f32 = [&](const uint32_t (&r)[32]) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                *reinterpret_cast<uint4 *>(staging + lane * 128 + ((j ^ (lane & 7)) << 4)) =
                    make_uint4(r[4 * j], r[4 * j + 1], r[4 * j + 2], r[4 * j + 3]);
        };
        auto stage_bf16 = [&](const uint32_t (&r)[64]) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                *reinterpret_cast<uint4 *>(staging + lane * 128 + ((j ^ (lane & 7)) << 4)) =
                    make_uint4(pack_bf16x2(__uint_as_float(r[8 * j]), __uint_as_float(r[8 * j + 1])), pack_bf16x2(__uint_as_float(r[8 * j + 2]), __uint_as_float(r[8 * j + 3])),
                               pack_bf16x2(__uint_as_float(r[8 * j + 4]), __uint_as_float(r[8 * j + 5])), pack_bf16x2(__uint_as_float(r[8 * j + 6]), __uint_as_float(r[8 * j + 7])));
        };
        // The staged chunk to out: row m, column col.
        auto store = [&](int col, int m, int valid) {
            if (WG || valid >= 32) {
                fence_async_smem();
                __syncwarp();
                if (lane == 0) {
                    if (OUT == OUT_ADD_F32) tma_add_3d(&map_out, smem_u32(staging), col, m, t.g);
                    else tma_store_3d(&map_out, smem_u32(staging), col, m, WG ? t.g : 0);
                    tma_store_commit();
                }
            } else {
                __syncwarp();
                uint8_t *dst = static_cast<uint8_t *>(p.out) + ((long long)m * p.ld_out + col) * ES;
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const int row = q * 4 + (lane >> 3), piece = lane & 7;
                    const uint4 v = *reinterpret_cast<const uint4 *>(staging + row * 128 + ((piece ^ (row & 7)) << 4));
                    if (row < valid && col + piece * PER < p.n) *reinterpret_cast<uint4 *>(dst + (long long)row * p.ld_out * ES + piece * 16) = v;
                }
                __syncwarp();
            }
        };
        auto release = [&](unsigned a) {          // this warp has read the accumulator
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (CG == 1) mbar_arrive_local(acce0 + 8 * a);
                else mbar_arrive_accumulator(map_to_rank(acce0 + 8 * a, 0));
            }
        };
        while (next_tile_warp(t)) {
            const int m = t.m0 + (int)rank * 128 + quarter * 32;            // first row of this warp
            const int valid = (WG ? p.kdim : t.m1) - m;                     // rows of the group (matrix) from there on
            const int col0 = t.n0 + half * HALF;
            const uint32_t tacc = tmem_base + ((uint32_t)(quarter * 32) << 16) + half * HALF;
            float scale = 1.0f;
            if (!WG && p.row_scale != nullptr && lane < valid) scale = p.row_scale[m + lane];
            float ref = 0.0f, sum = 0.0f, most = __uint_as_float(0xff800000u);
            int label = -1;
            if (is_vocab(OUT) && lane < valid) {
                label = p.label[m + lane];
                if (label >= 0) ref = p.ref[m + lane];
            }
            uint32_t acc[HALF];
            // The sums begin with the row's rest, fetched while the products run (added behind them it took 7 us a tile).
            const bool begun = !WG && B == B_MN && OUT == OUT_BF16 && p.rest != nullptr && t.kb0 == 0;
            if (begun) {
                const float rest = lane < valid ? p.rest[m + lane] : 0.0f;
                const uint4 *b = rest != 0.0f ? reinterpret_cast<const uint4 *>(p.rest_b + t.g * p.b_stride + p.label[m + lane] * p.ld_b + col0) : nullptr;
#pragma unroll
                for (int j = 0; j < HALF / 8; ++j) {
                    const uint4 v = b != nullptr && col0 + 8 * j < p.n ? b[j] : make_uint4(0, 0, 0, 0);
                    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        acc[8 * j + 2 * e] = __float_as_uint(rest * __uint_as_float(w[e] << 16));
                        acc[8 * j + 2 * e + 1] = __float_as_uint(rest * __uint_as_float(w[e] & 0xffff0000u));
                    }
                }
            }
            for (int k0 = t.kb0; k0 < t.kb1; k0 += part_blocks(OUT), ++ai) {
                const unsigned a = ai & 1;
                if (!__all_sync(0xffffffffu, mbar_wait(accf0 + 8 * a, (ai >> 1) & 1, abort, limit + limit / 2))) { failed = 3; break; }
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < HALF; c += 32) {
                    uint32_t(&sum)[32] = *reinterpret_cast<uint32_t (*)[32]>(&acc[c]);
                    if (k0 == t.kb0 && !begun) {
                        tmem_ld32(tacc + a * TN + c, sum);
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; e += 16) {
                            uint32_t r[16];
                            tmem_ld16(tacc + a * TN + c + e, r);
                            tmem_ld_wait();
#pragma unroll
                            for (int j = 0; j < 16; ++j) sum[e + j] = __float_as_uint(__uint_as_float(sum[e + j]) + __uint_as_float(r[j]));
                        }
                    }
                }
                tmem_ld_wait();
                release(a);
            }
            if (failed) break;
            if (valid <= 0 || (OUT == OUT_ADD_F32 && t.kb0 == t.kb1 && t.slot < 0)) continue;
            if (t.kb0 == t.kb1) {
#pragma unroll
                for (int j = 0; j < HALF; ++j) acc[j] = 0u;
            }
            if (!WG && !is_vocab(OUT) && p.row_scale != nullptr) {
#pragma unroll
                for (int j = 0; j < HALF; ++j) acc[j] = scale == 0.0f ? 0u : __float_as_uint(__uint_as_float(acc[j]) * scale);
            }
            if (!is_vocab(OUT) && t.slot >= 0) {         // a part: fp32, in the scratch
#pragma unroll
                for (int c = 0; c < HALF; c += 32) {
                    staging_free();
                    stage_f32(*reinterpret_cast<const uint32_t (*)[32]>(&acc[c]));
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_3d(&map_parts, smem_u32(staging), half * HALF + c, t.slot * TM + (int)rank * 128 + quarter * 32, 0);
                        tma_store_commit();
                    }
                }
                continue;
            }
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const int col = col0 + c * CHUNK;
                uint32_t (&r)[CHUNK] = *reinterpret_cast<uint32_t (*)[CHUNK]>(&acc[c * CHUNK]);
                if (is_vocab(OUT) && col < p.n) {
                    // logits that do not count become -inf: the label's, those behind the vocabulary, rows without a label
                    const int end = label < 0 ? 0 : p.n - col, at = label - col;
                    if (__any_sync(0xffffffffu, end < CHUNK || (at >= 0 && at < CHUNK))) {
#pragma unroll
                        for (int j = 0; j < CHUNK; ++j) if (j >= end || j == at) r[j] = 0xff800000u;
                    }
                    float s4[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int j = 0; j < CHUNK; ++j) {
                        const float l = __uint_as_float(r[j]);
                        most = fmaxf(most, l);
                        const float e = exp2_approx((l - ref) * 1.4426950408889634f);
                        s4[j & 3] += e;
                        r[j] = __float_as_uint(e);
                    }
                    sum += (s4[0] + s4[1]) + (s4[2] + s4[3]);
                }
                if (OUT == OUT_VOCAB_SUMS || col >= p.n) continue;
                staging_free();
                if constexpr (is_f32(OUT)) stage_f32(r);
                else stage_bf16(r);
                store(col, m, valid);
            }
            if (is_vocab(OUT) && col0 < p.n && lane < valid) p.sums[(long long)(col0 / HALF) * p.ld_sums + m + lane] = make_float2(sum, most);
        }
        if (lane == 0) tma_store_wait_read<0>();
    } else if (QB && warp >= 4 + EPI_WARPS) {
        // ---- converters: warp c takes rows 8 c .. + 7 of a block of the reduction.  A lane takes columns 8 j .. + 7 and 64 + 8 j .. + 7 of two of
        // them, the two halves of a row in turns by its parity, so that no two lanes meet in a bank.
        give_registers<CONV_REGISTERS>();
        constexpr int MINE = 64 / (4 * CONV_WARPS);            // rows of a lane
        const int first = (warp - 4 - EPI_WARPS) * (64 / CONV_WARPS) + (lane >> 3), j = lane & 7, odd = first & 1;
        Tile t;
        unsigned it = 0;
        while (next_tile_warp(t)) {
            const int plain = plain_blocks(p, t);
            for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
                const unsigned s = it % RING;
                if (!__all_sync(0xffffffffu, mbar_wait(qfull0 + 8 * s, (it / RING) & 1, abort, limit))) { failed = 6; break; }
                uint8_t *db = smem + s * STAGE + A_BYTES;
                if (kb == plain) zero_rows<2>(smem + s * STAGE, t.m1 - t.lo - kb * BK, BK, threadIdx.x - 32 * (4 + EPI_WARPS), 32 * CONV_WARPS);
                const uint8_t *q = db + B_BYTES;
                uint2 v[MINE][2];
                uint32_t scale[MINE];
#pragma unroll
                for (int i = 0; i < MINE; ++i) {
                    const int r = first + 4 * i;
                    v[i][0] = *reinterpret_cast<const uint2 *>(q + r * 128 + odd * 64 + j * 8);
                    v[i][1] = *reinterpret_cast<const uint2 *>(q + r * 128 + (1 - odd) * 64 + j * 8);
                    scale[i] = unit_bytes[s * 64 + r];
                }
#pragma unroll
                for (int i = 0; i < MINE; ++i) {
                    const int r = first + 4 * i;
                    const __nv_bfloat162 unit = unit_of(scale[i]);             // (0 behind the group: 0 times any whole number)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint4 w;
                        widen4(v[i][h].x, unit, unit, w.x, w.y);
                        widen4(v[i][h].y, unit, unit, w.z, w.w);
                        *reinterpret_cast<uint4 *>(db + (h ^ odd) * (BK * 128) + r * 128 + ((j ^ (r & 7)) << 4)) = w;
                    }
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) {
                    if (rank == 1) signal_operand(map_to_rank(smem_u32(words + warp - 4 - EPI_WARPS), 0), map_to_rank(bfull0 + 8 * s, 0));
                    else if (CG == 2 && warp == 4 + EPI_WARPS) mbar_expect_tx(bfull0 + 8 * s, CONV_WARPS * SIGNAL_BYTES);
                    else mbar_arrive_local(bfull0 + 8 * s);
                }
            }
            if (failed) break;
        }
    } else {
        give_registers<few_registers(B)>();
        if (warp == 0) {
            // ---- producer (one thread: a warp's own synchronisation at every tile cost the ring 300 clocks)
            Tile t;
            unsigned it = 0;
            while (lane == 0 && !failed && next_tile(t)) {
                if (p.debug_no_loads) continue;
                const int m0 = t.m0 + (int)rank * 128, n0 = t.n0 + (int)rank * 128, zb = WG ? 0 : t.g, r0 = WG ? t.lo : 0, plain = WG ? plain_blocks(p, t) : t.kb1;
                for (int kb = t.kb0; kb < plain; ++kb, ++it) {
                    const unsigned s = it % RING, use = it / RING;
                    if (use > 0 && !mbar_wait(empty0 + 8 * s, (use - 1) & 1, abort, limit)) { failed = 1; break; }
                    if (rank == 0) mbar_expect_tx(full0 + 8 * s, CG * (QB ? A_BYTES : STAGE_BYTES));
                    const uint32_t bar = CG == 1 ? full0 + 8 * s : map_to_rank(full0 + 8 * s, 0);
                    const uint32_t da = smem_base + s * STAGE, db = da + A_BYTES;
                    if (A_MN) {
                        load_tile<CG>(da, &map_a, bar, m0, r0 + kb * BK, 0);
                        load_tile<CG>(da + BK * 128, &map_a, bar, m0 + 64, r0 + kb * BK, 0);
                    } else {
                        load_tile<CG>(da, &map_a, bar, kb * BK, m0, 0);
                    }
                    if (QB) {
                        mbar_expect_tx(qfull0 + 8 * s, Q_BYTES);
                        tma_load_3d(db + B_BYTES, &map_b, qfull0 + 8 * s, n0, r0 + kb * BK, 0);
                    } else if (B == B_MN) {
                        load_tile<CG>(db, &map_b, bar, n0, r0 + kb * BK, zb);
                        load_tile<CG>(db + BK * 128, &map_b, bar, n0 + 64, r0 + kb * BK, zb);
                    } else {
                        load_tile<CG>(db, &map_b, bar, kb * BK, n0, zb);
                    }
                }
                if (WG && plain < t.kb1 && !failed) {          // a block shared with the next group: this CTA's barrier counts the bytes, `full` keeps step
                    const unsigned s = it % RING, use = it / RING;
                    if (use > 0 && !mbar_wait(empty0 + 8 * s, (use - 1) & 1, abort, limit)) { failed = 1; break; }
                    const uint32_t own = qfull0 + 8 * s, da = smem_base + s * STAGE, db = da + A_BYTES;
                    if (rank == 0) mbar_arrive_local(full0 + 8 * s);
                    mbar_expect_tx(own, QB ? A_BYTES + Q_BYTES : STAGE_BYTES);
                    tma_load_3d(da, &map_a, own, m0, r0 + plain * BK, 0);
                    tma_load_3d(da + BK * 128, &map_a, own, m0 + 64, r0 + plain * BK, 0);
                    if (QB) {
                        tma_load_3d(db + B_BYTES, &map_b, own, n0, r0 + plain * BK, 0);
                    } else {
                        tma_load_3d(db, &map_b, own, n0, r0 + plain * BK, 0);
                        tma_load_3d(db + BK * 128, &map_b, own, n0 + 64, r0 + plain * BK, 0);
                    }
                    ++it;
                }
            }
        } else if (warp == 1 && rank == 0) {
            // ---- issuer of the products (one thread)
            constexpr uint32_t idesc = grouped_idesc<CG, TN, A_MN, B != B_K>();
            constexpr uint32_t a_step = A_MN ? 2048u : 32u, b_step = B != B_K ? 2048u : 32u;
            Tile t;
            unsigned it = 0, ai = 0, mended = 0;               // mended: phases of rready, a bit for each stage
            while (lane == 0 && !failed && next_tile(t)) {
                const int plain = WG && !QB ? plain_blocks(p, t) : t.kb1;
                for (int k0 = t.kb0; k0 < t.kb1; ++ai) {
                    const int k1 = min(k0 + part_blocks(OUT), t.kb1);
                    const unsigned a = ai & 1, use = ai >> 1;
                    if (use > 0 && !mbar_wait(acce0 + 8 * a, (use - 1) & 1, abort, limit)) { failed = 2; break; }
                    tc_fence_after();
                    for (int kb = k0; kb < min(k1, plain); ++kb, ++it) {
                        const unsigned s = it % RING;
                        if (!mbar_wait(full0 + 8 * s, (it / RING) & 1, abort, limit)) { failed = 2; break; }
                        if (QB && !mbar_wait_operand(bfull0 + 8 * s, (it / RING) & 1, abort, limit)) { failed = 2; break; }
                        tc_fence_after();
                        const uint32_t da = smem_base + s * STAGE, db = da + A_BYTES;
#pragma unroll
                        for (int k = 0; k < BK / UMMA_K; ++k)
                            umma_g<CG>(tmem_base + a * TN, smem_desc(da + k * a_step, A_MN), smem_desc(db + k * b_step, B != B_K), idesc,
                                       (kb > k0 || k > 0) ? 1u : 0u);
                        umma_commit_g<CG>(empty0 + 8 * s);
                    }
                    if (WG && !QB && plain < k1 && !failed) {
                        const unsigned s = it % RING;
                        if (!mbar_wait(full0 + 8 * s, (it / RING) & 1, abort, limit) || !mbar_wait_operand(rready0 + 8 * s, (mended >> s) & 1, abort, limit)) { failed = 2; break; }
                        mended ^= 1u << s;
                        tc_fence_after();
                        const uint32_t da = smem_base + s * STAGE, db = da + A_BYTES;
                        const int steps = (t.m1 - t.lo - plain * BK + UMMA_K - 1) / UMMA_K;
                        for (int k = 0; k < steps; ++k)
                            umma_g<CG>(tmem_base + a * TN, smem_desc(da + k * a_step, A_MN), smem_desc(db + k * b_step, B != B_K), idesc,
                                       (plain > k0 || k > 0) ? 1u : 0u);
                        umma_commit_g<CG>(empty0 + 8 * s);
                        ++it;
                    }
                    if (failed) break;
                    umma_commit_g<CG>(accf0 + 8 * a);
                    k0 = k1;
                }
            }
        } else if (QB && warp == 2) {
            // ---- the scales of every block's 64 rows, 0 behind the group and behind the columns
            Tile t;
            unsigned it = 0;
            while (next_tile_warp(t)) {
                const int n0 = t.n0 + (int)rank * 128, rows = n0 < p.n ? t.m1 - t.lo : 0;
                const uint8_t *scale = p.scales + (long long)(n0 / ACT_BLOCK) * p.total_rows + t.lo;
                for (int kb = t.kb0; kb < t.kb1; ++kb, ++it) {
                    const unsigned s = it % RING, use = it / RING;
                    const int r = kb * BK + lane;
                    const uint8_t a = r < rows ? scale[r] : 0, b = r + 32 < rows ? scale[r + 32] : 0;
                    if (use > 0 && !__all_sync(0xffffffffu, mbar_wait(empty0 + 8 * s, (use - 1) & 1, abort, limit))) { failed = 7; break; }
                    unit_bytes[s * 64 + lane] = a;
                    unit_bytes[s * 64 + lane + 32] = b;
                    __syncwarp();
                    if (lane == 0) mbar_arrive_local(qfull0 + 8 * s);
                }
                if (failed) break;
            }
        } else if (WG && !QB && warp == 2) {
            // ---- the last blocks of groups: zeros behind the group's end
            Tile t;
            unsigned it = 0, there = 0;                        // there: phases of rfull, a bit for each stage
            while (next_tile_warp(t)) {
                it += t.kb1 - t.kb0;
                const int plain = plain_blocks(p, t);
                if (plain >= t.kb1) continue;
                const unsigned s = (it - 1) % RING;
                if (!__all_sync(0xffffffffu, mbar_wait(rfull0 + 8 * s, (there >> s) & 1, abort, limit))) { failed = 8; break; }
                there ^= 1u << s;
                const int rows = t.m1 - t.lo - plain * BK;     // (the issuer takes only the steps of 16 that hold some)
                zero_rows<4>(smem + s * STAGE, rows, (rows + UMMA_K - 1) / UMMA_K * UMMA_K, lane, 32);
                fence_async_smem();
                __syncwarp();
                if (lane == 0) {
                    if (rank == 1) signal_operand(map_to_rank(smem_u32(words), 0), map_to_rank(rready0 + 8 * s, 0));
                    else if (CG == 2) mbar_expect_tx(rready0 + 8 * s, SIGNAL_BYTES);
                    else mbar_arrive_local(rready0 + 8 * s);
                }
            }
        } else if (warp == 3) {
            // ---- scheduler
            if (blockIdx.x == 0 && p.error_flag != nullptr) {
                bool bad = false;
                for (int g = lane; g < p.groups; g += 32)
                    bad |= p.offsets[g + 1] < p.offsets[g] || (g == 0 && p.offsets[0] != 0) || (g == p.groups - 1 && p.offsets[p.groups] != p.total_rows);
                if (bad) atomicExch(p.error_flag, ERR_OFFSETS);
            }
            Walker<TM, TN, WG> walk(p, lane, clusters);
            for (int i = cluster;; i += clusters) {
                Tile t{};
                if (!walk.find(i, t)) t.g = -1;
                else if (is_vocab(OUT) && p.redo != nullptr && !redo_tile<TM>(p, t, lane)) continue;
                const unsigned s = turn % AHEAD;
                if (turn >= AHEAD && !__all_sync(0xffffffffu, mbar_wait(tilee0 + 8 * s, (turn / AHEAD - 1) & 1, abort, limit))) { failed = 5; break; }
                ++turn;
                if (lane == 0) {
                    reinterpret_cast<int4 *>(tiles + s)[0] = make_int4(t.g, t.m0, t.m1, t.n0);
                    reinterpret_cast<int4 *>(tiles + s)[1] = make_int4(t.kb0, t.kb1, t.slot, t.lo);
                    mbar_arrive_local(tilef0 + 8 * s);
                }
                if (t.g < 0) break;
            }
        }
    }
    if (failed) {
        *abort = 1;
        if (p.error_flag != nullptr) atomicExch(p.error_flag, 200 + failed);
        // copies in flight land within microseconds; this CTA's shared memory outlives them
        for (const unsigned long long t0 = now_ns(); now_ns() - t0 < 1000000ull;) { }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (CG == 2) cluster_sync();
    if (warp == 2) tmem_dealloc_g<CG>(tmem_base, 2 * TN);
}

// The tiles that were cut: block (x, y) adds the parts of the x-th of them up, for 256 groups of four results, and writes them to out.
template <int TM, int TN, bool WG, int OUT>
__global__ void __launch_bounds__(256)
join_parts(const GroupedParams p, const float *scratch, int clusters)
{
    pdl_launch_dependents();
    pdl_wait();
    Walker<TM, TN, WG> walk(p, threadIdx.x & 31, clusters);
    Tile t;
    if ((int)blockIdx.x >= walk.cut || !walk.find(walk.whole + blockIdx.x * walk.parts, t)) return;
    constexpr int QUADS = TN / 4;
    const int i = blockIdx.y * 256 + threadIdx.x, row = i / QUADS, c = (i % QUADS) * 4;
    if (t.m0 + row >= (WG ? p.kdim : t.m1) || t.n0 + c >= p.n) return;
    const float *src = scratch + (long long)t.slot * (TM * TN) + row * TN + c;
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    constexpr int AT_ONCE = 24;                           // loads under way together: most tiles have no more parts (a round trip takes 1 us)
    for (int k0 = 0; k0 < walk.parts; k0 += AT_ONCE) {
        float4 v[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k)
            if (k0 + k < walk.parts) v[k] = *reinterpret_cast<const float4 *>(src + (long long)(k0 + k) * (TM * TN));
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k)
            if (k0 + k < walk.parts) {
                s.x += v[k].x; s.y += v[k].y; s.z += v[k].z; s.w += v[k].w;
            }
    }
    const long long at = (WG ? t.g * p.out_stride : 0) + (t.m0 + row) * p.ld_out + t.n0 + c;
    if (OUT == OUT_BF16) {
        *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(p.out) + at) = make_uint2(pack_bf16x2(s.x, s.y), pack_bf16x2(s.z, s.w));
    } else {
        float4 *dst = reinterpret_cast<float4 *>(static_cast<float *>(p.out) + at);
        if (OUT == OUT_ADD_F32) {
            const float4 v = *dst;
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        *dst = s;
    }
}

}  // namespace lm
}  // namespace cocod
