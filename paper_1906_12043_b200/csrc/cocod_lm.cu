// Operators for workers that train a language model: products of rows with their own group's weights, activations in
// 8 bits, softmax cross-entropy over a large vocabulary.  Declared in include/cocod_lm.h.
#include "cocod_lm.h"
#include "cocod_act8.cuh"
#include "cocod_grouped_sm100.cuh"
#include "cocod_vocab.cuh"
#include "cocod_lm_internal.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <utility>

namespace {

using namespace cocod;
using namespace cocod::lm;
using bf16 = __nv_bfloat16;

// A row-major matrix, or one per group.
struct Matrix {
    const void *data;
    int64_t ld, stride;                    // elements; stride: between groups
    int elem;                              // bytes of an element: 1 (8-bit checkpoint), 2 (bf16) or 4 (fp32)
};

// Three-dimensional map {columns, rows, groups}; a box is 128 bytes of `box_rows` rows.
bool encode(CUtensorMap *m, const Matrix &x, uint64_t cols, uint64_t rows, uint64_t groups, uint32_t box_rows)
{
    EncodeTiledFn enc = get_encoder();
    if (!enc) return false;
    const cuuint64_t dims[3] = {cols, rows, groups};
    const cuuint64_t strides[2] = {(cuuint64_t)x.ld * x.elem, (cuuint64_t)(groups > 1 ? x.stride : (int64_t)rows * x.ld) * x.elem};
    const cuuint32_t box[3] = {(cuuint32_t)(128 / x.elem), box_rows, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    const CUtensorMapDataType type = x.elem == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : x.elem == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32;
    return enc(m, type, 3, const_cast<void *>(x.data), dims,
               strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, x.elem == 1 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// ------------------------------------------------------------------------------------------ small kernels
// The groups by size, a warp for each.
__global__ void __launch_bounds__(256)
order_groups(const GroupedParams p, int *order)
{
    pdl_launch_dependents();
    pdl_wait();
    const int g = blockIdx.x * 8 + (threadIdx.x >> 5);
    if (g >= p.groups) return;
    const int rank = group_rank(p, g);
    if ((threadIdx.x & 31) == 0) order[rank] = g;
}
constexpr int WARP_GROUPS = 32;            // so many groups the product's warps order themselves

// out = bf16(sums), for `rows` rows of n columns (n a multiple of 4); row r of the result is row r % per_group of group r / per_group.
__global__ void __launch_bounds__(256)
round_sums(const float *sums, bf16 *out, long long ld, long long group_stride, long long per_group, long long rows, int n)
{
    pdl_launch_dependents();
    pdl_wait();
    const int quads = n / 4;
    const long long total = rows * quads;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (long long)gridDim.x * blockDim.x) {
        const long long r = i / quads, c = (i - r * quads) * 4;
        const float4 s = *reinterpret_cast<const float4 *>(sums + r * n + c);
        *reinterpret_cast<uint2 *>(out + (r / per_group) * group_stride + (r % per_group) * ld + c) =
            make_uint2(pack_bf16x2(s.x, s.y), pack_bf16x2(s.z, s.w));
    }
}

// ------------------------------------------------------------------------------------------ launching the products
enum Form { FORWARD, INPUT_GRAD, WEIGHT_GRAD };

// How a product is cut into tiles and parts.
struct Cut {
    bool pair;             // 256 x 256 tiles by pairs of CTAs, else 128 x 128 by single ones
    int max_parts;         // of a tile of the last wave
    int64_t tiles;         // at most
    int band;              // GroupedParams::band
};
// rows x cols results (rows form: `groups` groups share the rows; weight form: per group), reductions of `depth` (weight form: on
// average).  The choice minimises an estimate in microseconds, fitted to measurements: a launch 3.5 (pairs 4.5), a tile 1.5 (2.0)
// and for each block of 64 of its reduction 0.28 (0.33), or, when all SMs load at the same time, 0.34 (0.40): 4096 x 4096 x 4096
// takes 153 us in single tiles and 98 in pairs, 128 x 18944 x 512 7.4 and 10.0.  Joining the parts of tiles is another launch.
Cut choose_cut(Form form, int64_t groups, int64_t rows, int64_t cols, int64_t depth, bool parts_allowed)
{
    Cut best{};
    double best_cost = 1e300;
    const int sms = std::max(sm_count(), 2);
    for (int pair = 0; pair < 2; ++pair) {
        const int64_t t = pair ? 256 : 128, slots = pair ? sms / 2 : sms;
        // rows form: how the rows are divided is not known here; every group ends inside a tile, half a tile on average
        const int64_t most = form == WEIGHT_GRAD ? groups * ceil_div(rows, t) : std::min(rows, ceil_div(rows, t) + groups - 1);
        const double likely = form == WEIGHT_GRAD || groups == 1 ? (double)most
                                                                 : std::max((double)std::min(groups, rows), (double)rows / t + 0.5 * groups);
        const int64_t col_tiles = ceil_div(cols, t), blocks = std::max<int64_t>(1, ceil_div(depth, 64));
        const int64_t tiles = std::max<int64_t>(1, (int64_t)(likely * col_tiles)), full = tiles / slots, rest = tiles % slots;
        const double busy = std::min(1.0, (double)tiles / slots);
        const double block = pair ? std::max(0.33, 0.40 * busy) : std::max(0.28, 0.34 * busy), tile = pair ? 2.0 : 1.5;
        // A's tile rows of a band stay in L2 while B passes by; where all of B fits, or A's do not, eight are enough.  Never more
        // than there are: the kernel counts a band's tiles in 32 bits, which hold all tiles of a matrix.
        const int64_t row_bytes = t * depth * 2, tile_rows = std::max<int64_t>(1, ceil_div(rows, t));
        const bool b_fits = cols * depth * 2 <= (40 << 20);
        const int band = (int)std::min(tile_rows, std::max<int64_t>(8, b_fits ? 8 : (40 << 20) / std::max<int64_t>(row_bytes, 1)));
        // (joining takes about 0.09 us for each part: more parts than this cost more than they save)
        const int64_t sensible = (int64_t)std::sqrt(blocks * (pair ? 0.33 : 0.28) / 0.09) + 1, bound = std::min(blocks / 4, std::max<int64_t>(sensible, 2));
        const int64_t most_parts = rest > 0 && parts_allowed ? std::min(slots / rest, bound) : 1;
        for (int cut = 0; cut < 2; ++cut) {
            const int64_t parts = cut ? most_parts : 1;
            if (cut && parts < 2) break;
            const double busy_rest = std::min(1.0, (double)rest * parts / slots);
            const double block_rest = pair ? std::max(0.33, 0.40 * busy_rest) : std::max(0.28, 0.34 * busy_rest);
            const double cost = (pair ? 4.5 : 3.5) + full * (blocks * block + tile) + (rest ? ceil_div(blocks, parts) * block_rest + tile : 0.0) +
                                (parts > 1 ? 3.0 + parts * 0.09 + rest * parts * t * t * 4 / 8e6 : 0.0);
            // A cut has to promise a sixth: under load the GPU is at its power limit, where idle SMs leave the busy ones a higher clock
            // (4096 x 4096 x 4096: 3.5 instead of 4 waves, and 105 us instead of 101)
            if (cost * (parts > 1 ? 7.0 / 6.0 : 1.0) < best_cost) {
                best_cost = cost;
                // (the kernel counts the tiles itself and cuts by what it finds)
                best = Cut{pair != 0, cut ? (int)std::max<int64_t>(bound, 2) : 1, most * col_tiles, band};
            }
        }
    }
    return best;
}

template <int CG, int TN, bool WG, int B, int OUT>
int launch_tiles(cocod_lm *h, const CUtensorMap &a, const CUtensorMap &b, const CUtensorMap &out, const GroupedParams &p, int64_t tiles, cudaStream_t s)
{
    static bool configured[MAX_DEVICES] = {};
    const int dev = current_device(), sms = sm_count();
    if (dev < 0 || sms < 2) return COCOD_ERR_CUDA;
    auto kernel = grouped_gemm<CG, TN, WG, B, OUT>;
    if (!configured[dev]) {
        // The epilogue warps wait for the registers that the others give up: the launch has to hold their sum.
        cudaFuncAttributes attr{};
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, GROUPED_SMEM) != cudaSuccess ||
            cudaFuncGetAttributes(&attr, kernel) != cudaSuccess || attr.numRegs < launch_registers(B)) {
            cudaGetLastError();
            return COCOD_ERR_CUDA;
        }
        configured[dev] = true;
    }
    const int clusters = (int)(p.max_parts > 1 ? sms / CG : std::min<int64_t>(tiles, sms / CG));
    CUtensorMap parts = out;
    if (p.max_parts > 1 && !encode(&parts, Matrix{h->parts, TN, 0, 4}, TN, (uint64_t)clusters * 128 * CG, 1, 32)) return COCOD_ERR_CUDA;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)clusters * CG);
    cfg.blockDim = dim3(grouped_threads(B));
    cfg.dynamicSmemBytes = GROUPED_SMEM;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = CG;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    TRY_CUDA(cudaLaunchKernelEx(&cfg, kernel, a, b, out, parts, p));
    if constexpr (!is_vocab(OUT)) {
        // a wave has at most half its tiles cut, so that every one gets two parts
        if (p.max_parts > 1)
            TRY_CUDA(launch_dependent(true, join_parts<128 * CG, TN, WG, OUT>, dim3((unsigned)std::min<int64_t>(tiles, clusters / 2), 128 * CG * TN / 1024),
                                      dim3(256), 0, s, p, static_cast<const float *>(h->parts), clusters));
    }
    return COCOD_OK;
}

template <bool WG, int B, int OUT>
int launch_form(cocod_lm *h, const Cut &c, const CUtensorMap &a, const CUtensorMap &b, const CUtensorMap &o, const GroupedParams &p, cudaStream_t s)
{
    return c.pair ? launch_tiles<2, 256, WG, B, OUT>(h, a, b, o, p, c.tiles, s) : launch_tiles<1, 128, WG, B, OUT>(h, a, b, o, p, c.tiles, s);
}

// Which rows of the batch a call takes: row0 .. row0 + rows - 1 of total (A, out and row_scale start at row0).
struct Window {
    int64_t row0, rows, total;
};

// rows form: out (M x cols) = A (M x depth) times B_g (cols x depth for FORWARD, depth x cols for INPUT_GRAD)
// (row_scale, rest, label: see GroupedParams)
int run_rows(cocod_lm *h, Form form, int G, const int32_t *offsets, const Window &win, int64_t cols, int64_t depth, const Matrix &A, const Matrix &B,
             const Matrix &out, const float *row_scale, const float *rest, const int *label, cudaStream_t s)
{
    const int64_t M = win.rows;
    if (M == 0) return COCOD_OK;
    const Cut cut = choose_cut(form, G, M, cols, depth, true);
    CUtensorMap a, b, o;
    const bool ok = encode(&a, A, depth, M, 1, 128) &&
                    (form == FORWARD ? encode(&b, B, depth, cols, G, 128) : encode(&b, B, cols, depth, G, 64)) && encode(&o, out, cols, M, 1, 32);
    if (!ok) return COCOD_ERR_CUDA;
    GroupedParams p{};
    p.offsets = offsets; p.groups = G; p.total_rows = (int)win.total; p.row0 = (int)win.row0; p.rows = (int)M; p.n = (int)cols; p.kdim = (int)depth;
    p.tiles_n = (int)ceil_div(cols, cut.pair ? 256 : 128); p.band = cut.band; p.max_parts = cut.max_parts; p.row_scale = row_scale;
    p.rest = rest; p.label = label; p.rest_b = static_cast<const bf16 *>(B.data); p.ld_b = B.ld; p.b_stride = B.stride;
    p.out = const_cast<void *>(out.data); p.ld_out = out.ld;
    p.error_flag = h->flag;
    if (form == FORWARD)
        return out.elem == 2 ? launch_form<false, B_K, OUT_BF16>(h, cut, a, b, o, p, s) : launch_form<false, B_K, OUT_F32>(h, cut, a, b, o, p, s);
    return out.elem == 2 ? launch_form<false, B_MN, OUT_BF16>(h, cut, a, b, o, p, s) : launch_form<false, B_MN, OUT_F32>(h, cut, a, b, o, p, s);
}

// weight form: out_g (rows x cols) = sum over the group's rows m of A[m][.]^T B[m][.]
// (scales: B is an 8-bit checkpoint;  add: added to what out, fp32, holds;  ordered: a kernel before this one has
// written the groups' order, where there are more than WARP_GROUPS)
int run_weights(cocod_lm *h, int G, const int32_t *offsets, const Window &win, int64_t rows, int64_t cols, const Matrix &A, const Matrix &B,
                const uint8_t *scales, const Matrix &out, bool add, bool ordered, cudaStream_t s)
{
    const int64_t M = win.rows;
    const Cut cut = choose_cut(WEIGHT_GRAD, G, rows, cols, ceil_div(std::max<int64_t>(M, 1), G), true);
    Matrix a_rows = A, b_rows = B;
    if (M == 0) a_rows.data = b_rows.data = h->parts;           // nothing is read
    CUtensorMap a, b, o;
    if (!encode(&o, out, cols, rows, (uint64_t)G, 32) || !encode(&a, a_rows, rows, std::max<int64_t>(M, 1), 1, 64) ||
        !encode(&b, b_rows, cols, std::max<int64_t>(M, 1), 1, 64))
        return COCOD_ERR_CUDA;
    GroupedParams p{};
    p.offsets = offsets; p.groups = G; p.total_rows = (int)win.total; p.row0 = (int)win.row0; p.rows = (int)M; p.n = (int)cols; p.kdim = (int)rows;
    p.tiles_n = (int)ceil_div(cols, cut.pair ? 256 : 128); p.band = cut.band; p.max_parts = cut.max_parts;
    p.out = const_cast<void *>(out.data); p.ld_out = out.ld; p.out_stride = out.stride;
    p.order = G > WARP_GROUPS ? h->order : nullptr; p.scales = scales; p.error_flag = h->flag;
    if (G > WARP_GROUPS && !ordered) TRY_CUDA(launch_dependent(true, order_groups, dim3((unsigned)ceil_div(G, 8)), dim3(256), 0, s, p, h->order));
    if (scales)
        return out.elem == 2 ? launch_form<true, B_Q8, OUT_BF16>(h, cut, a, b, o, p, s) : launch_form<true, B_Q8, OUT_F32>(h, cut, a, b, o, p, s);
    if (add) return launch_form<true, B_MN, OUT_ADD_F32>(h, cut, a, b, o, p, s);
    return out.elem == 2 ? launch_form<true, B_MN, OUT_BF16>(h, cut, a, b, o, p, s) : launch_form<true, B_MN, OUT_F32>(h, cut, a, b, o, p, s);
}

// ------------------------------------------------------------------------------------------ vocabulary
// How a call's workspace is laid out when `at_once` rows are taken together.
struct VocabLayout {
    int64_t label, group, own, ref, share, any;       // whole batch: byte offsets
    int64_t rho, rest, redo, sums, u, hs;      // rows of one pass
    int64_t total32;                           // fp32 gradient of the weights, if it is summed over passes and wanted in bf16
    int64_t bytes, ldu, n_sums;
};
VocabLayout vocab_layout(int G, int64_t M, int64_t V, int64_t D, bool grad, int dw_elem, int64_t at_once)
{
    VocabLayout l{};
    int64_t at = 0;
    auto take = [&](int64_t bytes) { const int64_t here = at; at += ceil_div(bytes, 256) * 256; return here; };
    l.label = take(4 * M);
    l.group = take(4 * M);
    l.own = take(4 * M);
    l.ref = take(4 * M);
    l.share = take(4 * G);
    l.any = take(256);
    l.redo = take(4 * at_once);
    l.n_sums = ceil_div(V, 128) * 2;           // (as many as the smaller tiles give)
    l.sums = take(8 * at_once * l.n_sums);
    l.ldu = ceil_div(V, 64) * 64;
    if (grad) {
        l.rho = take(4 * at_once);
        l.rest = take(4 * at_once);
        l.u = take(2 * at_once * l.ldu);
        l.hs = take(2 * at_once * D);
        if (at_once < M && dw_elem == 2) l.total32 = take(4 * G * V * D);
    }
    l.bytes = at;
    return l;
}
// The most rows that fit, 0 if not even the fewest do.
int64_t vocab_rows(int G, int64_t M, int64_t V, int64_t D, bool grad, int dw_elem, int64_t bytes)
{
    if (vocab_layout(G, M, V, D, grad, dw_elem, M).bytes <= bytes) return M;
    int64_t lo = 0, hi = ceil_div(M, 256);     // in units of 256 rows: lo fits, hi does not
    while (hi - lo > 1) {
        const int64_t mid = (lo + hi) / 2;
        if (vocab_layout(G, M, V, D, grad, dw_elem, mid * 256).bytes <= bytes) lo = mid; else hi = mid;
    }
    return lo * 256;
}

struct VocabGrad {
    Matrix dh, dw;
};

int run_vocab(cocod_lm *h, int G, const int32_t *offsets, int64_t M, int64_t V, int64_t D, const Matrix &x, const Matrix &w, const int32_t *labels,
              const float *row_weight, float *loss, float *row_loss, const VocabGrad *grad, char *ws, int64_t workspace_bytes, cudaStream_t s)
{
    const int dw_elem = grad ? grad->dw.elem : 0;
    const int64_t at_once = M ? vocab_rows(G, M, V, D, grad != nullptr, dw_elem, workspace_bytes) : 0;
    if (M && at_once == 0) return COCOD_ERR_TOO_LARGE;
    const VocabLayout l = vocab_layout(G, M, V, D, grad != nullptr, dw_elem, at_once);
    if (l.bytes > workspace_bytes) return COCOD_ERR_TOO_LARGE;
    VocabRows v{};
    v.offsets = offsets; v.groups = G; v.total = (int)M; v.vocab = (int)V; v.width = (int)D; v.labels = labels; v.row_weight = row_weight;
    v.h = static_cast<const bf16 *>(x.data); v.ldh = x.ld;
    v.w = static_cast<const bf16 *>(w.data); v.ldw = w.ld; v.w_stride = w.stride;
    v.label = reinterpret_cast<int *>(ws + l.label); v.group = reinterpret_cast<int *>(ws + l.group); v.own = reinterpret_cast<float *>(ws + l.own);
    v.ref = reinterpret_cast<float *>(ws + l.ref); v.share = reinterpret_cast<float *>(ws + l.share);
    v.redo_any = reinterpret_cast<int *>(ws + l.any);
    v.error_flag = h->flag;
    const Cut cut = choose_cut(FORWARD, G, M, V, D, false);  // by the whole batch: the passes change no sum's order
    const bool several = at_once < M;
    int64_t row0 = 0;
    do {                                   // (no rows at all: one pass, for the results' zeros)
        const Window win{row0, std::min(at_once, M - row0), M};
        const int64_t rows = std::max<int64_t>(win.rows, 1);
        const Matrix hx{M ? static_cast<const bf16 *>(x.data) + row0 * x.ld : (const void *)h->parts, M ? x.ld : D, 0, 2};
        const Matrix u{ws + l.u, l.ldu, 0, 2}, hs{ws + l.hs, D, 0, 2};
        CUtensorMap a, b, o;
        if (!encode(&a, hx, D, rows, 1, 128) || !encode(&b, w, D, V, G, 128) || !encode(&o, grad ? u : hx, grad ? V : D, rows, 1, 32)) return COCOD_ERR_CUDA;
        GroupedParams p{};
        p.offsets = offsets; p.groups = G; p.total_rows = (int)M; p.row0 = (int)row0; p.rows = (int)win.rows; p.n = (int)V; p.kdim = (int)D;
        p.tiles_n = (int)ceil_div(V, cut.pair ? 256 : 128); p.max_parts = 1;
        p.band = (int)std::min<int64_t>(cut.band, ceil_div(rows, cut.pair ? 256 : 128));
        p.out = ws + l.u; p.ld_out = l.ldu; p.error_flag = h->flag;
        p.ref = v.ref + row0; p.label = v.label + row0; p.sums = reinterpret_cast<float2 *>(ws + l.sums); p.ld_sums = (int)win.rows;
        const int row_blocks = (int)ceil_div(win.rows, 8);
        TRY_CUDA(launch_dependent(true, vocab_begin, dim3(row_blocks + G), dim3(256), 0, s, p, grad && G > WARP_GROUPS ? h->order : (int *)nullptr, v, row_blocks));
        FinishParams f{};
        f.v = v; f.row0 = (int)row0; f.rows = (int)win.rows; f.sums = p.sums; f.ld_sums = p.ld_sums;
        f.n_sums = (int)ceil_div(V, cut.pair ? 128 : 64);
        f.row_loss = row_loss; f.redo = reinterpret_cast<int *>(ws + l.redo);
        f.loss = row0 + win.rows >= M ? loss : nullptr;
        if (grad) {
            f.rho = reinterpret_cast<float *>(ws + l.rho);
            f.rest = reinterpret_cast<float *>(ws + l.rest);
            f.u = reinterpret_cast<bf16 *>(ws + l.u); f.ldu = l.ldu;
            f.hs = reinterpret_cast<bf16 *>(ws + l.hs);
        }
        const dim3 finish_grid((unsigned)ceil_div(rows, FINISH_ROWS));
        for (int pass = 0; pass < 2; ++pass) {
            p.redo = pass ? f.redo : nullptr;
            p.redo_any = v.redo_any;
            f.second = pass;
            if (win.rows > 0) {
                if (int rc = grad ? launch_form<false, B_K, OUT_VOCAB>(h, cut, a, b, o, p, s) : launch_form<false, B_K, OUT_VOCAB_SUMS>(h, cut, a, b, o, p, s))
                    return rc;
            }
            TRY_CUDA(launch_dependent(true, vocab_finish, finish_grid, dim3(32 * FINISH_WARPS), 0, s, f));
        }
        if (grad) {
            const Matrix dh{static_cast<const bf16 *>(grad->dh.data) + row0 * grad->dh.ld, grad->dh.ld, 0, 2};
            if (int rc = run_rows(h, INPUT_GRAD, G, offsets, win, D, V, u, w, dh, f.rho, f.rest, p.label, s)) return rc;
            const Matrix dst = several && dw_elem == 2 ? Matrix{ws + l.total32, D, V * D, 4} : grad->dw;
            if (int rc = run_weights(h, G, offsets, win, V, D, u, hs, nullptr, dst, several && row0 > 0, true, s)) return rc;
        }
        row0 += win.rows;
    } while (row0 < M);
    if (grad && several && dw_elem == 2)
        TRY_CUDA(launch_dependent(true, round_sums, dim3((unsigned)std::min<int64_t>(ceil_div(G * V * D / 4, 256), 8 * (int64_t)sm_count())), dim3(256), 0, s,
                                  reinterpret_cast<const float *>(ws + l.total32), static_cast<bf16 *>(const_cast<void *>(grad->dw.data)),
                                  (long long)grad->dw.ld, (long long)grad->dw.stride, (long long)V, (long long)(G * V), (int)D));
    return COCOD_OK;
}

// ------------------------------------------------------------------------------------------ checks of arguments
bool good_rows(const void *p, int64_t ld, int64_t cols, int64_t M, int elem)
{
    return (M == 0 || p != nullptr) && aligned16(p) && ld >= cols && (ld * elem) % 16 == 0 && ld < (1ll << 36);
}
bool good_groups(const void *p, int64_t ld, int64_t stride, int64_t rows, int64_t cols, int G, int elem)
{
    return p != nullptr && aligned16(p) && ld >= cols && (ld * elem) % 16 == 0 && ld < (1ll << 36) &&
           (G == 1 || (stride >= (rows - 1) * ld + cols && (stride * elem) % 16 == 0 && stride < (1ll << 37)));
}
bool good_shape(const cocod_lm *h, int G, const int32_t *offsets, int64_t M, int64_t n, int64_t k)
{
    return h && G >= 1 && G <= COCOD_LM_MAX_GROUPS && offsets && (reinterpret_cast<uintptr_t>(offsets) & 3u) == 0 && M >= 0 && M <= MAX_DIM &&
           n >= 8 && n <= MAX_DIM && n % 8 == 0 && k >= 8 && k <= MAX_DIM && k % 8 == 0;
}
void lm_free(cocod_lm *h)
{
    void *ptrs[] = {h->order, h->parts, h->flag};
    for (void *p : ptrs) if (p) cudaFree(p);
    delete h;
}

}  // namespace

extern "C" {

int cocod_lm_create(cocod_lm_handle **out)
{
    if (!out) return COCOD_ERR_INVALID;
    if (!get_encoder()) return COCOD_ERR_CUDA;
    cocod_lm *h = new (std::nothrow) cocod_lm();
    if (!h) return COCOD_ERR_OOM;
    h->device = current_device();
    cudaError_t e = cudaMalloc((void **)&h->order, COCOD_LM_MAX_GROUPS * sizeof(int));
    if (e == cudaSuccess) e = cudaMalloc((void **)&h->parts, (size_t)(sm_count() / 2 + 1) * 256 * 256 * sizeof(float));
    if (e == cudaSuccess) e = cudaMalloc((void **)&h->flag, 256);
    // (calls come on any stream: the zeros have to be there, and need not wait for other work)
    cudaStream_t s = nullptr;
    if (e == cudaSuccess) e = cudaStreamCreateWithFlags(&s, cudaStreamNonBlocking);
    if (e == cudaSuccess) e = cudaMemsetAsync(h->flag, 0, 256, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (s) cudaStreamDestroy(s);
    if (e != cudaSuccess) {
        cudaGetLastError();
        lm_free(h);
        return e == cudaErrorMemoryAllocation ? COCOD_ERR_OOM : COCOD_ERR_CUDA;
    }
    *out = h;
    return COCOD_OK;
}

int cocod_lm_destroy(cocod_lm_handle *h)
{
    if (!h) return COCOD_OK;
    const int now = current_device();      // (another one may be current: it is this one whose work has to end)
    if (now != h->device) cudaSetDevice(h->device);
    cudaDeviceSynchronize();
    if (now != h->device && now >= 0) cudaSetDevice(now);
    lm_free(h);
    return COCOD_OK;
}

int cocod_lm_check(cocod_lm_handle *h, cocod_stream_t stream)
{
    if (!h) return COCOD_ERR_INVALID;
    cudaStream_t s = (cudaStream_t)stream;
    int f = 0;
    if (cudaMemcpyAsync(&f, h->flag, sizeof(int), cudaMemcpyDeviceToHost, s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess)
        return COCOD_ERR_CUDA;
    if (f == 0) return COCOD_OK;
    if (cudaMemsetAsync(h->flag, 0, sizeof(int), s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess) return COCOD_ERR_CUDA;
    return f >= ERR_OFFSETS && f < 200 ? COCOD_ERR_INVALID : COCOD_ERR_TIMEOUT;
}

int64_t cocod_lm_launch_count(const cocod_lm_handle *h) { return h ? h->launches : -1; }

int cocod_grouped_forward(cocod_lm_handle *h, int G, const int32_t *offsets, int64_t M, int64_t n, int64_t k, const void *x, int64_t ldx,
                          const void *w, int64_t ldw, int64_t w_stride, void *y, int64_t ldy, int out_type,
                          cocod_stream_t stream)
{
    const int es = size_of(out_type);
    if (!good_shape(h, G, offsets, M, n, k) || !es || !good_rows(x, ldx, k, M, 2) ||
        !good_groups(w, ldw, w_stride, n, k, G, 2) || !good_rows(y, ldy, n, M, es))
        return COCOD_ERR_INVALID;
    return run_rows(h, FORWARD, G, offsets, Window{0, M, M}, n, k, Matrix{x, ldx, 0, 2}, Matrix{w, ldw, w_stride, 2}, Matrix{y, ldy, 0, es}, nullptr, nullptr, nullptr,
                    (cudaStream_t)stream);
}

int cocod_grouped_input_grad(cocod_lm_handle *h, int G, const int32_t *offsets, int64_t M, int64_t n, int64_t k, const void *dy, int64_t lddy,
                             const void *w, int64_t ldw, int64_t w_stride, void *dx, int64_t lddx, int out_type,
                             cocod_stream_t stream)
{
    const int es = size_of(out_type);
    if (!good_shape(h, G, offsets, M, n, k) || !es || !good_rows(dy, lddy, n, M, 2) ||
        !good_groups(w, ldw, w_stride, n, k, G, 2) || !good_rows(dx, lddx, k, M, es))
        return COCOD_ERR_INVALID;
    return run_rows(h, INPUT_GRAD, G, offsets, Window{0, M, M}, k, n, Matrix{dy, lddy, 0, 2}, Matrix{w, ldw, w_stride, 2}, Matrix{dx, lddx, 0, es}, nullptr, nullptr, nullptr,
                    (cudaStream_t)stream);
}

int cocod_grouped_weight_grad(cocod_lm_handle *h, int G, const int32_t *offsets, int64_t M, int64_t n, int64_t k, const void *dy, int64_t lddy,
                              const void *x, int64_t ldx, void *dw, int64_t lddw, int64_t dw_stride, int out_type,
                              cocod_stream_t stream)
{
    const int es = size_of(out_type);
    if (!good_shape(h, G, offsets, M, n, k) || !es || !good_rows(dy, lddy, n, M, 2) || !good_rows(x, ldx, k, M, 2) ||
        !good_groups(dw, lddw, dw_stride, n, k, G, es))
        return COCOD_ERR_INVALID;
    return run_weights(h, G, offsets, Window{0, M, M}, n, k, Matrix{dy, lddy, 0, 2}, Matrix{x, ldx, 0, 2}, nullptr, Matrix{dw, lddw, dw_stride, es}, false, false,
                       (cudaStream_t)stream);
}

static bool good_act(const cocod_lm_handle *h, int64_t M, int64_t k, const int8_t *q, int64_t ldq)
{
    return h && M >= 0 && M <= MAX_DIM && k >= 1 && k <= 65535ll * ACT_BLOCK - 7 && (M == 0 || q) && aligned16(q) && ldq % 16 == 0 && ldq >= k &&
           ldq < (1ll << 36);
}
// Which form of the kernels below a call takes (cocod_act8.cuh): whether all rows start at multiples of so many bytes ...
static bool rows_aligned(const void *p, int64_t ld, int64_t M, int bytes)
{
    return reinterpret_cast<uintptr_t>(p) % bytes == 0 && (M == 1 || ld * 2 % bytes == 0);
}
// ... and how many rows a thread takes: one while all CTAs find a place at the same time (8192 x 512: packed in 3.8 us, two rows 4.3;
// 77 x 999: 2.1 and 2.8), two beyond that (32768 x 4095: 98 us, one row 104).
static int act_rows_at_once(int64_t M, int64_t k) { return ceil_div(M, ACT_ROWS) * ceil_div(k, ACT_BLOCK) <= 8 * (int64_t)sm_count() ? 1 : 2; }
static bool good_bf16(const void *p, int64_t ld, int64_t M, int64_t k)
{
    return (M == 0 || p) && (reinterpret_cast<uintptr_t>(p) & 1u) == 0 && ld >= k && ld < (1ll << 36);
}

int cocod_act_pack(cocod_lm_handle *h, int64_t M, int64_t k, const void *x, int64_t ldx, int8_t *q, int64_t ldq, uint8_t *scales,
                   cocod_stream_t stream)
{
    if (!good_act(h, M, k, q, ldq) || !good_bf16(x, ldx, M, k) || (M > 0 && !scales)) return COCOD_ERR_INVALID;
    if (M == 0) return COCOD_OK;
    const int at_once = act_rows_at_once(M, k);
    const dim3 grid((unsigned)ceil_div(M, at_once * ACT_ROWS), (unsigned)ceil_div(k, ACT_BLOCK));
    const auto kernels = rows_aligned(x, ldx, M, 16) ? std::make_pair(act_pack<16, 1>, act_pack<16, 2>)
                       : rows_aligned(x, ldx, M, 8)  ? std::make_pair(act_pack<8, 1>, act_pack<8, 2>)
                       : rows_aligned(x, ldx, M, 4)  ? std::make_pair(act_pack<4, 1>, act_pack<4, 2>)
                                                     : std::make_pair(act_pack<2, 1>, act_pack<2, 2>);
    const auto kernel = at_once == 1 ? kernels.first : kernels.second;
    TRY_CUDA(launch_dependent(true, kernel, grid, dim3(256), 0, (cudaStream_t)stream, static_cast<const bf16 *>(x), (long long)ldx, q,
                              (long long)ldq, scales, (long long)M, (int)k));
    return COCOD_OK;
}

int cocod_act_unpack(cocod_lm_handle *h, int64_t M, int64_t k, const int8_t *q, int64_t ldq, const uint8_t *scales, void *y, int64_t ldy,
                     cocod_stream_t stream)
{
    if (!good_act(h, M, k, q, ldq) || !good_bf16(y, ldy, M, k) || (M > 0 && !scales)) return COCOD_ERR_INVALID;
    if (M == 0) return COCOD_OK;
    const bool aligned = rows_aligned(y, ldy, M, 16);
    const int at_once = act_rows_at_once(M, k);
    const dim3 grid((unsigned)ceil_div(M, at_once * ACT_ROWS), (unsigned)ceil_div(aligned ? k : k + 7, ACT_BLOCK));     // (columns moved by up to 7)
    const auto kernel = at_once == 1 ? (aligned ? act_unpack<true, 1> : act_unpack<false, 1>) : (aligned ? act_unpack<true, 2> : act_unpack<false, 2>);
    TRY_CUDA(launch_dependent(true, kernel, grid, dim3(256), 0, (cudaStream_t)stream, q, (long long)ldq, scales, static_cast<bf16 *>(y),
                              (long long)ldy, (long long)M, (int)k));
    return COCOD_OK;
}

int cocod_act_relu_grad(cocod_lm_handle *h, int64_t M, int64_t k, const void *dh, int64_t lddh, const int8_t *q, int64_t ldq, void *dz,
                        int64_t lddz, cocod_stream_t stream)
{
    if (!good_act(h, M, k, q, ldq) || !good_bf16(dh, lddh, M, k) || !good_bf16(dz, lddz, M, k)) return COCOD_ERR_INVALID;
    if (M == 0) return COCOD_OK;
    const bool aligned = rows_aligned(dh, lddh, M, 16) && rows_aligned(dz, lddz, M, 16);
    const bool together = (reinterpret_cast<uintptr_t>(dh) - reinterpret_cast<uintptr_t>(dz)) % 16 == 0 && (M == 1 || (lddh - lddz) % 8 == 0);
    const int at_once = act_rows_at_once(M, k);
    const dim3 grid((unsigned)ceil_div(M, at_once * ACT_ROWS), (unsigned)ceil_div(aligned ? k : k + 7, ACT_BLOCK));
    const auto kernels = aligned    ? std::make_pair(act_relu_grad<true, true, 1>, act_relu_grad<true, true, 2>)
                         : together ? std::make_pair(act_relu_grad<false, true, 1>, act_relu_grad<false, true, 2>)
                                    : std::make_pair(act_relu_grad<false, false, 1>, act_relu_grad<false, false, 2>);
    const auto kernel = at_once == 1 ? kernels.first : kernels.second;
    TRY_CUDA(launch_dependent(true, kernel, grid, dim3(256), 0, (cudaStream_t)stream, static_cast<const bf16 *>(dh), (long long)lddh, q,
                              (long long)ldq, static_cast<bf16 *>(dz), (long long)lddz, (long long)M, (int)k));
    return COCOD_OK;
}

// Whether a checkpoint is better turned into bf16 once, by a kernel before the product, than inside it.  The conversion costs the
// product about 0.26 us for every block of 64 of a tile's reduction (4 groups of 8192 rows, 2048 x 4096 results: 523 us against
// 399 with the kernel before it; 2048 rows, 2048 x 2048: 26.0 and 19.7); the kernel costs a launch and 3 bytes a value at 5.4 TB/s (16
// groups of 128 rows, 1024 x 1024 results: 20.5 us against 18.8 with the conversion inside).
static bool widen_first(int G, int64_t M, int64_t n, int64_t k)
{
    const int64_t depth = ceil_div(std::max<int64_t>(M, 1), G);
    const Cut cut = choose_cut(WEIGHT_GRAD, G, n, k, depth, true);
    const double waves = std::ceil((double)cut.tiles / (cut.pair ? sm_count() / 2 : std::max(sm_count(), 1)));
    return waves * ceil_div(depth, 64) * 0.26 > 4.0 + 3.0 * M * k / 5.4e6;
}

int64_t cocod_grouped_packed_workspace(int G, int64_t M, int64_t n, int64_t k)
{
    if (G < 1 || G > COCOD_LM_MAX_GROUPS || M < 0 || M > MAX_DIM || n < 8 || n > MAX_DIM || k < 8 || k > MAX_DIM) return COCOD_ERR_INVALID;
    return sm_count() > 1 && widen_first(G, M, n, k) ? M * k * 2 : 0;
}

int cocod_grouped_weight_grad_packed(cocod_lm_handle *h, int G, const int32_t *offsets, int64_t M, int64_t n, int64_t k, const void *dy,
                                     int64_t lddy, const int8_t *q, int64_t ldq, const uint8_t *scales, void *dw, int64_t lddw,
                                     int64_t dw_stride, int out_type, void *workspace, int64_t workspace_bytes, cocod_stream_t stream)
{
    const int es = size_of(out_type);
    if (!good_shape(h, G, offsets, M, n, k) || !es || !good_rows(dy, lddy, n, M, 2) || !good_act(h, M, k, q, ldq) || (M > 0 && !scales) ||
        !good_groups(dw, lddw, dw_stride, n, k, G, es) || workspace_bytes < 0 || (workspace_bytes > 0 && (!workspace || !aligned16(workspace))))
        return COCOD_ERR_INVALID;
    const Matrix A{dy, lddy, 0, 2}, out{dw, lddw, dw_stride, es};
    if (M > 0 && workspace_bytes >= M * k * 2) {
        if (int rc = cocod_act_unpack(h, M, k, q, ldq, scales, workspace, k, stream)) return rc;
        return run_weights(h, G, offsets, Window{0, M, M}, n, k, A, Matrix{workspace, k, 0, 2}, nullptr, out, false, false, (cudaStream_t)stream);
    }
    const uint8_t *any = reinterpret_cast<const uint8_t *>(h->flag);      // (no rows: nothing is read)
    return run_weights(h, G, offsets, Window{0, M, M}, n, k, A, Matrix{q, ldq, 0, 1}, M > 0 ? scales : any, out, false, false, (cudaStream_t)stream);
}

int64_t cocod_vocab_workspace(int G, int64_t M, int64_t V, int64_t D, int with_grad, int dw_type, int64_t limit)
{
    const int es = with_grad ? size_of(dw_type) : 2;
    if (G < 1 || G > COCOD_LM_MAX_GROUPS || M < 0 || M > MAX_DIM || V < 1 || V > MAX_DIM || D < 8 || D > MAX_DIM || D % 8 || !es || limit < 0)
        return COCOD_ERR_INVALID;
    const int64_t all = vocab_layout(G, M, V, D, with_grad != 0, es, M).bytes;
    int64_t bytes = all;
    if (all > limit) {
        const int64_t rows = vocab_rows(G, M, V, D, with_grad != 0, es, limit);
        bytes = std::min(all, vocab_layout(G, M, V, D, with_grad != 0, es, std::max<int64_t>(rows, std::min<int64_t>(M, 256))).bytes);
    }
    return bytes;
}

static bool good_vocab(const cocod_lm_handle *h, int G, const int32_t *offsets, int64_t M, int64_t V, int64_t D, const void *x, int64_t ldx,
                       const void *w, int64_t ldw, int64_t w_stride, const int32_t *labels, const float *row_weights, const float *loss,
                       const float *row_loss, const void *workspace, int64_t workspace_bytes)
{
    return good_shape(h, G, offsets, M, 8, D) && workspace && (reinterpret_cast<uintptr_t>(workspace) & 255u) == 0 && workspace_bytes >= 0 && V >= 1 && V <= MAX_DIM && good_rows(x, ldx, D, M, 2) &&
           good_groups(w, ldw, w_stride, V, D, G, 2) && (M == 0 || (labels && row_loss)) && loss &&
           ((reinterpret_cast<uintptr_t>(labels) | reinterpret_cast<uintptr_t>(row_weights) | reinterpret_cast<uintptr_t>(loss) |
             reinterpret_cast<uintptr_t>(row_loss)) & 3u) == 0;
}

int cocod_vocab_loss(cocod_lm_handle *h, int G, const int32_t *offsets, int64_t M, int64_t V, int64_t D, const void *x, int64_t ldx,
                     const void *w, int64_t ldw, int64_t w_stride, const int32_t *labels, const float *row_weights, float *loss,
                     float *row_loss, void *workspace, int64_t workspace_bytes, cocod_stream_t stream)
{
    if (!good_vocab(h, G, offsets, M, V, D, x, ldx, w, ldw, w_stride, labels, row_weights, loss, row_loss, workspace, workspace_bytes))
        return COCOD_ERR_INVALID;
    return run_vocab(h, G, offsets, M, V, D, Matrix{x, ldx, 0, 2}, Matrix{w, ldw, w_stride, 2}, labels, row_weights, loss, row_loss, nullptr,
                     static_cast<char *>(workspace), workspace_bytes, (cudaStream_t)stream);
}

int cocod_vocab_loss_grad(cocod_lm_handle *h, int G, const int32_t *offsets, int64_t M, int64_t V, int64_t D, const void *x, int64_t ldx,
                          const void *w, int64_t ldw, int64_t w_stride, const int32_t *labels, const float *row_weights, float *loss,
                          float *row_loss, void *dx, int64_t lddx, void *dw, int64_t lddw, int64_t dw_stride, int dw_type, void *workspace,
                          int64_t workspace_bytes, cocod_stream_t stream)
{
    const int es = size_of(dw_type);
    if (!good_vocab(h, G, offsets, M, V, D, x, ldx, w, ldw, w_stride, labels, row_weights, loss, row_loss, workspace, workspace_bytes) || !es ||
        !good_rows(dx, lddx, D, M, 2) || !good_groups(dw, lddw, dw_stride, V, D, G, es))
        return COCOD_ERR_INVALID;
    const VocabGrad grad{Matrix{dx, lddx, 0, 2}, Matrix{dw, lddw, dw_stride, es}};
    return run_vocab(h, G, offsets, M, V, D, Matrix{x, ldx, 0, 2}, Matrix{w, ldw, w_stride, 2}, labels, row_weights, loss, row_loss, &grad,
                     static_cast<char *>(workspace), workspace_bytes, (cudaStream_t)stream);
}

int cocod_grouped_wait_selftest(int wait_ms, int pair, cocod_stream_t stream)
{
    if (wait_ms < 1 || wait_ms > 2000) return COCOD_ERR_INVALID;
    struct Scratch {                       // of this call only
        char *p = nullptr;
        ~Scratch() { if (p) cudaFree(p); }
    } sc;
    cudaStream_t s = (cudaStream_t)stream;
    constexpr size_t BYTES = 512 * 512 * 4;
    if (cudaMalloc((void **)&sc.p, BYTES + 512) != cudaSuccess) { cudaGetLastError(); return COCOD_ERR_OOM; }
    int *flag = reinterpret_cast<int *>(sc.p + BYTES), *offsets = flag + 32;
    const int32_t two[2] = {0, 512};
    if (cudaMemsetAsync(sc.p, 0, BYTES + 512, s) != cudaSuccess ||
        cudaMemcpyAsync(offsets, two, sizeof(two), cudaMemcpyHostToDevice, s) != cudaSuccess)
        return COCOD_ERR_CUDA;
    const Matrix m{sc.p, 512, 512 * 512, 2};
    CUtensorMap a, b, o;
    if (!encode(&a, m, 512, 512, 1, 128) || !encode(&b, m, 512, 512, 1, 128) || !encode(&o, m, 512, 512, 1, 32)) return COCOD_ERR_CUDA;
    GroupedParams p{};
    p.offsets = offsets; p.groups = 1; p.total_rows = 512; p.rows = 512; p.n = 512; p.kdim = 512; p.band = 8; p.max_parts = 1;
    p.tiles_n = pair ? 2 : 4; p.out = sc.p; p.ld_out = 512; p.error_flag = flag;
    p.wait_ns = (unsigned long long)wait_ms * 1000000ull;
    p.debug_no_loads = 1;
    // two CTAs (one pair), so that several tiles wait for each
    cocod_lm scratch;
    const int rc = pair ? launch_tiles<2, 256, false, B_K, OUT_BF16>(&scratch, a, b, o, p, 1, s) : launch_tiles<1, 128, false, B_K, OUT_BF16>(&scratch, a, b, o, p, 2, s);
    int f = 0;
    if (rc != COCOD_OK || cudaMemcpyAsync(&f, flag, sizeof(int), cudaMemcpyDeviceToHost, s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess) {
        cudaGetLastError();
        return COCOD_ERR_CUDA;
    }
    return f ? COCOD_ERR_TIMEOUT : COCOD_OK;
}

}  // extern "C"
