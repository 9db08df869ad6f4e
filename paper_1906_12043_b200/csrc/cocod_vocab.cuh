// Softmax cross-entropy over a large vocabulary: what is left besides the three products.
//
// With c_r the reference of row r (its label's own logit, l[r][t]), S_r = sum_{v != t} exp(l - c_r) and D_r = S_r + exp(l[r][t] - c_r):
//     loss_r            = log D_r + c_r - l[r][t]            ( = log1p(S_r) for that reference)
//     d loss_r / d l    = softmax - onehot = u[r][v] / D_r   with u = exp(l - c_r) for v != t and u[r][t] = -S_r
// The row's factor rho_r = a_r / D_r (a_r: the row's share in the loss) is not needed before the sums are complete, and
// it is one number per row: it is the epilogue's factor in dh = rho (u w), and goes into h in dw = u^T (rho h).  So the
// exponentials are written once, next to the sums, and read by the two products as they are; no pass over them between.
// The label's own entry is the one whose value hangs on the sums; this file's vocab_finish puts it in.
// u in bf16 has 8 bits everywhere: -S_r is formed from the sum, not as a difference from one.  A row's largest entry of
// softmax - onehot is as a rule its label's, so its rounding is made good.  In dw by the factor that goes into h, rho_r S_r / bf16(S_r): the
// label's term carries one rounding (of rho h) and not two.  In dh by what the rounding left out, times the label's row of w, which
// the product's epilogue adds in fp32 (37 rows of 256 over 8191 entries: error against 64 bits 0.0024 -> 0.0016, a bf16 result's own).
// When loss_r > 50, exp(l - c_r) could leave bf16's range or rho_r fp32's, and with a small a_r (1e-25, loss 45) rho_r is gone earlier: such a
// row is done again relative to its largest logit.
#pragma once
#include "cocod_grouped_sm100.cuh"

namespace cocod {
namespace lm {

constexpr int FINISH_ROWS = 32, FINISH_WARPS = 16;
constexpr float SUM_LIMIT = 5.0e21f;         // about exp(50)
constexpr float RHO_LIMIT = 1.0e-30f;        // a smaller factor of a large sum is left to the second pass: it would near the end of fp32

struct VocabRows {
    const int *offsets;                // [groups + 1]
    int groups, total;                 // total: all rows
    int vocab, width;
    const int *labels;                 // [total], the caller's
    const float *row_weight;           // [total] or nullptr: 1 / (rows of the group that have a label)
    const __nv_bfloat16 *h;            // [total][ldh]
    long long ldh;
    const __nv_bfloat16 *w;            // [groups][vocab][ldw]
    long long ldw, w_stride;
    int *label;                        // [total]: negative where the row takes no part
    int *group;                        // [total]: the row's group
    float *own;                        // [total]: the label's logit
    float *ref;                        // [total]: c_r
    float *share;                      // [groups]: 1 / rows with a label
    int *redo_any;                     // whether a row needs the second pass; [1]: blocks of vocab_finish that are through
    int *error_flag;
};

// The group of row r, -1: in none (one warp, 32 groups at a time).
__device__ __forceinline__ int group_of(const int *offsets, int groups, int r)
{
    const int lane = threadIdx.x & 31;
    for (int g0 = 0; g0 < groups; g0 += 32) {
        const int g = g0 + lane;
        const uint32_t hit = __ballot_sync(0xffffffffu, g < groups && offsets[g] <= r && r < offsets[g + 1]);
        if (hit) return g0 + __ffs(hit) - 1;
    }
    return -1;
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// One warp per row: the label's logit.  The last `groups` blocks count the rows of a group that have a label, and, where it is
// wanted, write the group's place by size.
__global__ void __launch_bounds__(256)
vocab_begin(const GroupedParams window, int *order, const VocabRows p, int row_blocks)
{
    __shared__ int part[8];
    pdl_launch_dependents();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if ((int)blockIdx.x >= row_blocks) {
        const int g = blockIdx.x - row_blocks;
        if (g == 0 && threadIdx.x < 2) p.redo_any[threadIdx.x] = 0;
        if (order != nullptr && warp == 5) {
            const int rank = group_rank(window, g);
            if (lane == 0) order[rank] = g;
        }
        const int lo = min(max(p.offsets[g], 0), p.total), hi = min(max(p.offsets[g + 1], lo), p.total);
        int n = 0;
        for (int r = lo + threadIdx.x; r < hi; r += 256) {
            const int t = p.labels[r];
            n += t >= 0 && t < p.vocab && (p.row_weight == nullptr || p.row_weight[r] != 0.0f);
        }
        n = __reduce_add_sync(0xffffffffu, n);
        if (lane == 0) part[warp] = n;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int i = 1; i < 8; ++i) n += part[i];
            p.share[g] = 1.0f / (float)max(n, 1);
        }
        return;
    }
    const long long r = window.row0 + (long long)blockIdx.x * 8 + warp;
    if (r >= window.row0 + window.rows) return;
    int t = p.labels[r];
    const int g = group_of(p.offsets, p.groups, (int)r);
    if (t >= p.vocab) {
        if (lane == 0 && p.error_flag != nullptr) atomicExch(p.error_flag, ERR_LABEL);
        t = -1;
    }
    if (g < 0 || (p.row_weight != nullptr && p.row_weight[r] == 0.0f)) t = -1;
    float s = 0.0f;
    if (t >= 0) {
        const uint4 *a = reinterpret_cast<const uint4 *>(p.h + r * p.ldh);
        const uint4 *b = reinterpret_cast<const uint4 *>(p.w + g * p.w_stride + t * p.ldw);
#pragma unroll 4
        for (int i = lane; i < p.width / 8; i += 32) {
            const uint4 x = a[i], y = b[i];
            const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s = fmaf(__uint_as_float(xs[j] << 16), __uint_as_float(ys[j] << 16), s);
                s = fmaf(__uint_as_float(xs[j] & 0xffff0000u), __uint_as_float(ys[j] & 0xffff0000u), s);
            }
        }
    }
    s = warp_sum(s);
    if (lane == 0) {
        p.label[r] = t < 0 ? -1 : t;
        p.group[r] = max(g, 0);
        p.own[r] = s;
        p.ref[r] = s;
    }
}

struct FinishParams {
    VocabRows v;
    int row0, rows;                    // of this launch; u, sums, rho, redo and hs start at row0
    const float2 *sums;
    int n_sums, ld_sums;
    float *row_loss;                   // [total]
    float *rho;                        // [rows], nullptr: the loss alone is wanted
    float *rest;                       // [rows]: -S less its rounding to bf16 (with rho)
    __nv_bfloat16 *u;                  // [rows][ldu]
    long long ldu;
    __nv_bfloat16 *hs;                 // [rows][width]: rho h
    int *redo;                         // first pass: set
    float *loss;                       // [groups], second pass over the last rows: the means; else nullptr
    int second;                        // second pass: no row is looked at again if *v.redo_any is 0
};

// loss[g] = sum of the rows' losses with their shares, by one block in a fixed order: a group's rows are shared out over as many
// warps as there are for each group.
__device__ __forceinline__ void vocab_mean(const VocabRows &p, const float *row_loss, float *loss)
{
    __shared__ float part[FINISH_WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int per = p.groups >= FINISH_WARPS ? 1 : FINISH_WARPS / p.groups, at_once = FINISH_WARPS / per;
    for (int g0 = 0; g0 < p.groups; g0 += at_once) {
        const int g = g0 + warp / per;
        float s = 0.0f;
        if (g < p.groups && warp < at_once * per) {
            const int lo = min(max(p.offsets[g], 0), p.total), hi = min(max(p.offsets[g + 1], lo), p.total);
#pragma unroll 8
            for (int r = lo + (warp % per) * 32 + lane; r < hi; r += 32 * per) {
                const float v = __ldcg(row_loss + r);
                s += p.row_weight == nullptr ? v : v == 0.0f ? 0.0f : p.row_weight[r] * v;
            }
        }
        s = warp_sum(s);
        __syncthreads();
        if (lane == 0) part[warp] = s;
        __syncthreads();
        if (lane == 0 && warp % per == 0 && g < p.groups && warp < at_once * per) {
            for (int i = 1; i < per; ++i) s += part[warp + i];
            loss[g] = p.row_weight != nullptr ? s : s * p.share[g];
        }
    }
}

// 32 rows per CTA: their sums, losses and factors, the label's entry of u, and rho h.
__global__ void __launch_bounds__(32 * FINISH_WARPS)
vocab_finish(const FinishParams p)
{
    __shared__ float2 part[FINISH_WARPS][FINISH_ROWS];
    __shared__ float factor[FINISH_ROWS];
    pdl_launch_dependents();
    pdl_wait();
    if (p.second && *p.v.redo_any == 0) {          // (the losses are complete: the first block adds them up)
        if (blockIdx.x == 0 && p.loss != nullptr) vocab_mean(p.v, p.row_loss, p.loss);
        return;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int first = blockIdx.x * FINISH_ROWS, row = first + lane;        // counted from row0
    float s = 0.0f, most = __uint_as_float(0xff800000u);
    int t = -1;                        // what the first warp needs later is asked for now
    float own = 0.0f, ref = 0.0f, share = 0.0f;
    if (warp == 0 && row < p.rows) {
        t = p.v.label[p.row0 + row];
        own = p.v.own[p.row0 + row];
        ref = p.v.ref[p.row0 + row];
        if (p.rho != nullptr) share = p.v.row_weight != nullptr ? p.v.row_weight[p.row0 + row] : p.v.share[p.v.group[p.row0 + row]];
    }
    // The first values of h are under way before the sums are known.
    const int vecs = p.v.width / 8, rows = min(FINISH_ROWS, p.rows - first), all = p.rho != nullptr ? rows * vecs : 0;
    constexpr int BATCH = 4, THREADS = 32 * FINISH_WARPS;
    uint4 x[BATCH];
    auto fetch = [&](int i0) {
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int i = i0 + b * THREADS, rr = i / vecs;
            if (i < all) x[b] = reinterpret_cast<const uint4 *>(p.v.h + (long long)(p.row0 + first + rr) * p.v.ldh)[i - rr * vecs];
        }
    };
    fetch(threadIdx.x);
    if (row < p.rows) {
#pragma unroll 8
        for (int i = warp; i < p.n_sums; i += FINISH_WARPS) {
            const float2 v = p.sums[(long long)i * p.ld_sums + row];
            s += v.x;
            most = fmaxf(most, v.y);
        }
    }
    part[warp][lane] = make_float2(s, most);
    __syncthreads();
    if (warp == 0) {
        float rho = 0.0f, scale = 0.0f, rest = 0.0f;
        int again = 0;
        if (row < p.rows) {
            const int r = p.row0 + row;
            float loss = 0.0f;
            if (t >= 0) {
#pragma unroll
                for (int i = 1; i < FINISH_WARPS; ++i) {
                    s += part[i][lane].x;
                    most = fmaxf(most, part[i][lane].y);
                }
                const float et = own == ref ? 1.0f : expf(own - ref);
                loss = own == ref ? log1pf(s) : logf(s + et) + (ref - own);
                if (p.rho != nullptr) rho = share / (s + et);
                if (!p.second && (!(s <= SUM_LIMIT) || (s > 1.0f && p.rho != nullptr && fabsf(rho) < RHO_LIMIT))) {
                    again = 1;
                    p.v.ref[r] = most;
                    *p.v.redo_any = 1;
                }
                if (p.rho != nullptr) {
                    const __nv_bfloat16 entry = __float2bfloat16_rn(-s);
                    const float kept = -__bfloat162float(entry);
                    p.u[row * p.ldu + t] = entry;
                    scale = kept > 0.0f && kept <= 3.0e38f ? rho * (s / kept) : rho;
                    rest = kept - s;
                }
            }
            p.row_loss[r] = loss;
            if (!p.second) p.redo[row] = again;
            if (p.rho != nullptr) p.rho[row] = rho, p.rest[row] = rest;
        }
        factor[lane] = scale;
    }
    if (p.second && p.loss != nullptr) {           // the last block to get here adds the losses up
        __shared__ int last;
        if (warp == 0) {
            __threadfence();
            __syncwarp();              // every lane's loss is out before the block counts as through
            if (lane == 0) last = atomicAdd(p.v.redo_any + 1, 1) == (int)gridDim.x - 1;
        }
        __syncthreads();
        if (last) {
            __threadfence();
            vocab_mean(p.v, p.row_loss, p.loss);
        }
    }
    if (p.rho == nullptr) return;
    __syncthreads();
    for (int i0 = threadIdx.x; i0 < all; i0 += BATCH * THREADS) {
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int i = i0 + b * THREADS, rr = i / vecs;
            if (i >= all) break;
            const float f = factor[rr];
            uint4 o = make_uint4(0, 0, 0, 0);
            if (f != 0.0f) {           // (a row that takes no part is 0 whatever it holds)
                const uint32_t xs[4] = {x[b].x, x[b].y, x[b].z, x[b].w};
                uint32_t os[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) os[j] = pack_bf16x2(__uint_as_float(xs[j] << 16) * f, __uint_as_float(xs[j] & 0xffff0000u) * f);
                o = make_uint4(os[0], os[1], os[2], os[3]);
            }
            reinterpret_cast<uint4 *>(p.hs + (long long)(first + rr) * p.v.width)[i - rr * vecs] = o;
        }
        fetch(i0 + BATCH * THREADS);
    }
}

}  // namespace lm
}  // namespace cocod
