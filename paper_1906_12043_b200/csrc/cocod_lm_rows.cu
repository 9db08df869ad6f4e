// Operators that go by rows: tokens sorted by expert and back, log probabilities of given tokens.  Declared in include/cocod_lm.h.
#include "cocod_experts.cuh"
#include "cocod_logprobs.cuh"
#include "cocod_lm_internal.h"

#include <algorithm>

namespace {

using namespace cocod;
using namespace cocod::lm;
using bf16 = __nv_bfloat16;

template <typename P> bool aligned_to(const P *p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes == 0; }

// ------------------------------------------------------------------------------------------ experts
bool good_slots(const cocod_lm *h, int64_t T, int k, int64_t rows_at_most)
{
    return h && T >= 0 && k >= 1 && k <= MAX_CHOICES && T <= rows_at_most / k;
}
bool good_matrix(const void *p, int64_t ld, int64_t cols, int64_t M, int elem)
{
    return elem && (M == 0 || (p != nullptr && aligned_to(static_cast<const char *>(p), elem))) && ld >= cols && ld < (1ll << 36);
}
// Whether a matrix' rows start at multiples of 16 bytes (a single row: its address alone).
bool wide_rows(const void *p, int64_t ld, int64_t M, int elem) { return aligned16(p) && (M <= 1 || ld * elem % 16 == 0); }

ExpertRows expert_rows_of(const cocod_lm *h, int64_t T, int k, int64_t D, const int32_t *place, int per_piece)
{
    ExpertRows p{};
    p.place = place; p.tokens = (int)T; p.top = k; p.rows = (int)(T * k); p.pieces = (int)(D / per_piece); p.error_flag = h->flag;
    return p;
}
// Thread blocks of eight warps, a warp for `at_once` pieces of a token.
bool warp_blocks(int64_t T, int64_t pieces, int64_t at_once, unsigned *blocks)
{
    const int64_t n = ceil_div(T * ceil_div(pieces, at_once * 32), 8);
    *blocks = (unsigned)n;
    return n <= MAX_DIM;
}

template <typename T, bool WIDE>
int run_expert_rows(cocod_lm *h, int64_t tokens, int k, int64_t D, const void *x, int64_t ldx, const int32_t *place, void *out, int64_t ld, cudaStream_t s)
{
    const ExpertRows p = expert_rows_of(h, tokens, k, D, place, Piece<T, WIDE>::N);
    unsigned blocks;
    if (!warp_blocks(tokens, p.pieces, ROW_PIECES, &blocks)) return COCOD_ERR_TOO_LARGE;
    TRY_CUDA(launch_dependent(true, expert_rows<T, WIDE>, dim3(blocks), dim3(256), 0, s, p, static_cast<const T *>(x), (long long)ldx, static_cast<T *>(out),
                              (long long)ld));
    return COCOD_OK;
}
template <typename T, typename O, bool WIDE>
int run_expert_join(cocod_lm *h, int64_t tokens, int k, int64_t D, const void *rows, int64_t ld, const int32_t *place, const float *weights, void *y, int64_t ldy,
                    cudaStream_t s)
{
    const ExpertRows p = expert_rows_of(h, tokens, k, D, place, Piece<T, WIDE>::N);
    unsigned blocks;
    if (k > 2 || p.pieces * 4ll >= 3 * ceil_div(p.pieces, 64) * 64) {
        if (!warp_blocks(tokens, p.pieces, 2, &blocks)) return COCOD_ERR_TOO_LARGE;
        auto kernel = k > 2 ? expert_join_many<T, O, WIDE, 4, 2, 4> : k > 1 ? expert_join_many<T, O, WIDE, 2, 2, 5> : expert_join_many<T, O, WIDE, 1, 2, 8>;
        if (blocks < (unsigned)sm_count()) {
            warp_blocks(tokens, p.pieces, 1, &blocks);
            kernel = expert_join_many<T, O, WIDE, 4, 1, 4>;
        }
        TRY_CUDA(launch_dependent(true, kernel, dim3(blocks), dim3(256), 0, s, p, static_cast<const T *>(rows), (long long)ld, weights, static_cast<O *>(y),
                                  (long long)ldy));
        return COCOD_OK;
    }
    if (tokens > MAX_DIM * 256 / p.pieces) return COCOD_ERR_TOO_LARGE;
    blocks = (unsigned)ceil_div(tokens * p.pieces, k > 1 ? 256 : 512);
    TRY_CUDA(launch_dependent(true, k > 1 ? expert_join_few<T, O, WIDE, 2, 1> : expert_join_few<T, O, WIDE, 1, 2>, dim3(blocks), dim3(256), 0, s, p,
                              static_cast<const T *>(rows), (long long)ld, weights, static_cast<O *>(y), (long long)ldy));
    return COCOD_OK;
}
template <typename T, bool WIDE, int WARPS>
int run_join_grad(cocod_lm *h, const ExpertRows &p, const void *dy, int64_t lddy, const void *rows, int64_t ld, const float *weights, void *back, int64_t ld_back,
                  float *dw, cudaStream_t s)
{
    auto kernel = p.top <= 2 ? expert_join_grad<T, WIDE, WARPS, 2> : expert_join_grad<T, WIDE, WARPS, 4>;
    TRY_CUDA(launch_dependent(true, kernel, dim3((unsigned)ceil_div(p.tokens, 8 / WARPS)), dim3(256), 0, s, p, static_cast<const T *>(dy),
                              (long long)lddy, static_cast<const T *>(rows), (long long)ld, weights, static_cast<T *>(back), (long long)ld_back, dw));
    return COCOD_OK;
}
template <typename T, bool WIDE>
int run_expert_join_grad(cocod_lm *h, int64_t tokens, int k, int64_t D, const void *dy, int64_t lddy, const void *rows, int64_t ld, const int32_t *place,
                         const float *weights, void *back, int64_t ld_back, float *dw, cudaStream_t s)
{
    const ExpertRows p = expert_rows_of(h, tokens, k, D, place, Piece<T, WIDE>::N);
    // Warps of a token: as many as leave each lane two pieces, and more while there are SMs without a block and lanes would still have one.  16384 x 8 of 256 pieces: one,
    // two, four, eight warps 196, 183, 176, 185 us; 4999 x 6 of 129: 33.8, 31.7, 33.8, 41.0; 40000 x 6 of 64: 93, 99, 148, 246; 4096 x 12 of 512: 160, 148, 140, 133;
    // 64 x 8 of 256: 15.4, 9.2, 6.7, 5.1.
    int warps = p.pieces >= 512 ? 8 : p.pieces >= 256 ? 4 : p.pieces > 64 ? 2 : 1;
    while (warps < 8 && (int64_t)p.tokens * warps < 8 * (int64_t)sm_count() && p.pieces > 32 * warps) warps *= 2;
    if (warps == 1) return run_join_grad<T, WIDE, 1>(h, p, dy, lddy, rows, ld, weights, back, ld_back, dw, s);
    if (warps == 2) return run_join_grad<T, WIDE, 2>(h, p, dy, lddy, rows, ld, weights, back, ld_back, dw, s);
    if (warps == 4) return run_join_grad<T, WIDE, 4>(h, p, dy, lddy, rows, ld, weights, back, ld_back, dw, s);
    return run_join_grad<T, WIDE, 8>(h, p, dy, lddy, rows, ld, weights, back, ld_back, dw, s);
}

// How the slots are divided among thread blocks: a multiple of SORT_THREADS for each.  One block needs no count before it (2048 slots in 4.3 us, in several
// blocks 5); several come in whole clusters.
constexpr int64_t SORT_ALONE = 2048, SORT_LEAST = 1024;
struct SortPlan {
    int64_t blocks, span;
};
SortPlan sort_plan(int64_t N)
{
    if (N <= SORT_ALONE) return SortPlan{1, std::max<int64_t>(1, ceil_div(N, SORT_THREADS)) * SORT_THREADS};
    const int64_t most = std::max<int64_t>(1, sm_count() / SORT_CLUSTER), clusters = std::min(most, ceil_div(N, SORT_LEAST * SORT_CLUSTER));
    const int64_t blocks = clusters * SORT_CLUSTER;
    return SortPlan{blocks, ceil_div(ceil_div(N, blocks), SORT_THREADS) * SORT_THREADS};
}

// ------------------------------------------------------------------------------------------ log probabilities
constexpr int64_t SHORT_ROW = 256;

template <typename T, int LANES, int NR>
int launch_short(cocod_lm *h, const TokenRows &p, cudaStream_t s)
{
    TRY_CUDA(launch_dependent(true, token_logprobs_short<T, LANES, NR>, dim3((unsigned)ceil_div(p.rows, 256 / LANES)), dim3(256), 0, s, p));
    return COCOD_OK;
}
template <typename T>
int run_logprobs_short(cocod_lm *h, const TokenRows &p, cudaStream_t s)
{
    // (65536 x 64, two alternatives: half a warp 13.6 us, a whole one 18; 16384 x 64, four: 6.5 and 6.2)
    if (p.vocab <= 16) return launch_short<T, 8, 2>(h, p, s);
    if (p.vocab <= 32) return launch_short<T, 16, 2>(h, p, s);
    if (p.vocab <= 64) return p.top <= 2 ? launch_short<T, 16, 4>(h, p, s) : launch_short<T, 32, 2>(h, p, s);
    return p.vocab <= 128 ? launch_short<T, 32, 4>(h, p, s) : launch_short<T, 32, 8>(h, p, s);
}

// Thread blocks for a row: one while there are rows for every SM; for fewer rows up to eight, each with at least 2048 values.
int row_blocks(int64_t M, int64_t V)
{
    int blocks = 1;
    while (blocks < 8 && M * blocks * 2 <= 2 * (int64_t)sm_count() && V / (blocks * 2) >= 2048) blocks *= 2;
    return blocks;
}

template <typename T, int THREADS>
int run_logprobs_row(cocod_lm *h, const TokenRows &p, int blocks, cudaStream_t s)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(THREADS == 32 ? ceil_div(p.rows, ROW_BLOCK<32> / 32) : p.rows * blocks));
    cfg.blockDim = dim3(ROW_BLOCK<THREADS>);
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)blocks;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = blocks > 1 ? 2 : 1;
    auto kernel = p.top ? token_logprobs_row<T, THREADS, true> : token_logprobs_row<T, THREADS, false>;
    TRY_CUDA(cudaLaunchKernelEx(&cfg, kernel, p, blocks));
    return COCOD_OK;
}
template <typename T>
int run_logprobs(cocod_lm *h, const TokenRows &p, cudaStream_t s)
{
    if (p.vocab <= SHORT_ROW) return run_logprobs_short<T>(h, p, s);
    const int blocks = row_blocks(p.rows, p.vocab);
    if (p.rows > MAX_DIM / blocks) return COCOD_ERR_TOO_LARGE;
    if (blocks > 1) return run_logprobs_row<T, 512>(h, p, blocks, s);
    // A row's threads: what follows the pass over a row costs every one of them, and leaves HBM idle unless other rows are under way (32768 x 4000, five
    // alternatives: 84 us with 32 threads, 107 with 64; 16384 x 16000: 114 and 113, 133 with 128; 4096 x 50001 with twenty: 131 with 64, 99 and 100 with 128
    // and 256, whose threads have less to look at again).  Where few rows leave SMs without warps, more: 200 x 5000 with twenty: 12.9 us with 32, 8.5 with 256.
    int threads = p.vocab <= 12000 ? 32 : p.vocab <= 24000 ? 64 : p.vocab <= 48000 ? 128 : 256;
    while (threads < 256 && p.rows * (threads / 32) * 2 <= 16 * (int64_t)sm_count() && p.vocab >= 16 * threads) threads *= 2;
    return threads == 32 ? run_logprobs_row<T, 32>(h, p, 1, s) : threads == 64 ? run_logprobs_row<T, 64>(h, p, 1, s)
         : threads == 128 ? run_logprobs_row<T, 128>(h, p, 1, s) : run_logprobs_row<T, 256>(h, p, 1, s);
}

template <typename T>
int run_logprobs_grad(cocod_lm *h, const TokenGrads &p, cudaStream_t s)
{
    constexpr int N = Word<T>::N, STEP = GRAD_THREADS * GRAD_WORDS;
    const int64_t words = ((int64_t)p.vocab + 2 * N - 2) / N, steps = ceil_div(words, STEP);
    // a thread block takes up to eight steps of a row, as long as there are sixteen thread blocks for every SM
    int64_t at_once = std::min<int64_t>(steps, 8);
    while (at_once > 1 && p.rows * ceil_div(steps, at_once) < 16 * (int64_t)sm_count()) --at_once;
    const int64_t parts = ceil_div(steps, at_once);
    if (p.rows > MAX_DIM / parts) return COCOD_ERR_TOO_LARGE;
    const bool together = (reinterpret_cast<uintptr_t>(p.logits) - reinterpret_cast<uintptr_t>(p.out)) % 16 == 0 &&
                          (p.rows <= 1 || (p.ld - p.ld_out) * (int64_t)sizeof(T) % 16 == 0);
    TRY_CUDA(launch_dependent(true, together ? token_logprobs_grad<T, true> : token_logprobs_grad<T, false>, dim3((unsigned)(p.rows * parts)), dim3(GRAD_THREADS), 0,
                              s, p, (int)parts, (int)(at_once * STEP)));
    return COCOD_OK;
}

bool good_tokens(const cocod_lm *h, int64_t M, int64_t V, const void *logits, int64_t ld, int es, const int32_t *tokens, float scale, int top)
{
    return h && es && M >= 0 && M <= MAX_DIM && V >= 1 && V <= MAX_DIM && good_matrix(logits, ld, V, M, es) && aligned_to(tokens, 4) && scale >= 1.0e-30f &&
           scale <= 1.0e30f && top >= 0 && top <= MAX_ALTERNATIVES && top <= V;
}
bool words_aligned(std::initializer_list<const void *> all)
{
    for (const void *p : all)
        if (!aligned_to(static_cast<const char *>(p), 4)) return false;
    return true;
}

}  // namespace

extern "C" {

int64_t cocod_expert_workspace(int64_t T, int k, int E)
{
    if (T < 0 || k < 1 || k > MAX_CHOICES || T > MAX_DIM / k || E < 1 || E > COCOD_LM_MAX_GROUPS) return COCOD_ERR_INVALID;
    const int64_t blocks = sort_plan(T * k).blocks;
    return blocks > 1 ? (blocks + blocks / SORT_CLUSTER) * (E + 1) * 4 : 0;
}

int cocod_expert_sort(cocod_lm_handle *h, int64_t T, int k, int E, const int32_t *experts, int64_t ld, int32_t *offsets, int32_t *counts, int32_t *order,
                      int32_t *place, void *workspace, int64_t workspace_bytes, cocod_stream_t stream)
{
    if (!good_slots(h, T, k, MAX_DIM) || E < 1 || E > COCOD_LM_MAX_GROUPS || !offsets || !counts || (T > 0 && (!experts || !order || !place)) || ld < k ||
        ld >= (1ll << 36) || !words_aligned({experts, offsets, counts, order, place, workspace}))
        return COCOD_ERR_INVALID;
    const int64_t need = cocod_expert_workspace(T, k, E);
    if (need > 0 && (!workspace || workspace_bytes < need)) return COCOD_ERR_TOO_LARGE;
    static bool configured[MAX_DEVICES] = {};
    const int dev = current_device();
    if (dev < 0) return COCOD_ERR_CUDA;
    if (!configured[dev]) {
        if (cudaFuncSetAttribute(expert_place, cudaFuncAttributeMaxDynamicSharedMemorySize, (SORT_WARPS + 2) * (COCOD_LM_MAX_GROUPS + 1) * 4) != cudaSuccess) {
            cudaGetLastError();
            return COCOD_ERR_CUDA;
        }
        configured[dev] = true;
    }
    const int64_t N = T * k;
    const SortPlan plan = sort_plan(N);
    ExpertSlots p{};
    p.experts = experts; p.ld = T > 1 ? ld : k; p.top = k; p.total = (int)N; p.experts_n = E; p.error_flag = h->flag;
    int *before = static_cast<int *>(workspace), *totals = before + plan.blocks * (E + 1);
    const dim3 grid((unsigned)plan.blocks);
    const cudaStream_t s = (cudaStream_t)stream;
    if (plan.blocks > 1) TRY_CUDA(launch_dependent(true, expert_count, grid, dim3(SORT_THREADS), (E + 1) * 4, s, p, (int)plan.span, before, totals));
    TRY_CUDA(launch_dependent(true, expert_place, grid, dim3(SORT_THREADS), (SORT_WARPS + 2) * (E + 1) * 4, s, p, (int)plan.span,
                              32 - __builtin_clz((unsigned)E + 1), static_cast<const int *>(before), static_cast<const int *>(totals), offsets, counts, order, place));
    return COCOD_OK;
}

int cocod_expert_rows(cocod_lm_handle *h, int64_t T, int k, int64_t D, const void *x, int64_t ldx, const int32_t *place, void *rows, int64_t ld, int type,
                      cocod_stream_t stream)
{
    const int es = size_of(type);
    if (!good_slots(h, T, k, MAX_DIM) || D < 1 || D > MAX_DIM || !good_matrix(x, ldx, D, T, es) || !good_matrix(rows, ld, D, T, es) || (T > 0 && !place) ||
        !words_aligned({place}))
        return COCOD_ERR_INVALID;
    if (T == 0) return COCOD_OK;
    const bool wide = D * es % 16 == 0 && wide_rows(x, ldx, T, es) && wide_rows(rows, ld, T * k, es);
    auto f = es == 2 ? (wide ? run_expert_rows<bf16, true> : run_expert_rows<bf16, false>) : (wide ? run_expert_rows<float, true> : run_expert_rows<float, false>);
    return f(h, T, k, D, x, ldx, place, rows, ld, (cudaStream_t)stream);
}

int cocod_expert_join(cocod_lm_handle *h, int64_t T, int k, int64_t D, const void *rows, int64_t ld, int type, const int32_t *place, const float *weights, void *y,
                      int64_t ldy, int out_type, cocod_stream_t stream)
{
    const int es = size_of(type), os = size_of(out_type);
    if (!good_slots(h, T, k, MAX_DIM) || D < 1 || D > MAX_DIM || !good_matrix(rows, ld, D, T, es) || !good_matrix(y, ldy, D, T, os) || (T > 0 && !place) ||
        !words_aligned({place, weights}))
        return COCOD_ERR_INVALID;
    if (T == 0) return COCOD_OK;
    const bool wide = D * es % 16 == 0 && wide_rows(rows, ld, T * k, es) && wide_rows(y, ldy, T, os);
    auto f = es == 2 ? (os == 2 ? (wide ? run_expert_join<bf16, bf16, true> : run_expert_join<bf16, bf16, false>)
                                : (wide ? run_expert_join<bf16, float, true> : run_expert_join<bf16, float, false>))
                     : (os == 2 ? (wide ? run_expert_join<float, bf16, true> : run_expert_join<float, bf16, false>)
                                : (wide ? run_expert_join<float, float, true> : run_expert_join<float, float, false>));
    return f(h, T, k, D, rows, ld, place, weights, y, ldy, (cudaStream_t)stream);
}

int cocod_expert_join_grad(cocod_lm_handle *h, int64_t T, int k, int64_t D, const void *dy, int64_t lddy, const void *rows, int64_t ld, const int32_t *place,
                           const float *weights, void *drows, int64_t ld_drows, float *dweights, int type, cocod_stream_t stream)
{
    const int es = size_of(type);
    if (!good_slots(h, T, k, MAX_DIM) || D < 1 || D > MAX_DIM || !good_matrix(dy, lddy, D, T, es) || !good_matrix(rows, ld, D, T, es) ||
        !good_matrix(drows, ld_drows, D, T, es) || (T > 0 && (!place || !weights || !dweights)) || !words_aligned({place, weights, dweights}))
        return COCOD_ERR_INVALID;
    if (T == 0) return COCOD_OK;
    const bool wide = D * es % 16 == 0 && wide_rows(dy, lddy, T, es) && wide_rows(rows, ld, T * k, es) && wide_rows(drows, ld_drows, T * k, es);
    auto f = es == 2 ? (wide ? run_expert_join_grad<bf16, true> : run_expert_join_grad<bf16, false>)
                     : (wide ? run_expert_join_grad<float, true> : run_expert_join_grad<float, false>);
    return f(h, T, k, D, dy, lddy, rows, ld, place, weights, drows, ld_drows, dweights, (cudaStream_t)stream);
}

int cocod_token_logprobs(cocod_lm_handle *h, int64_t M, int64_t V, const void *logits, int64_t ld, int type, const int32_t *tokens, float scale, int top,
                         float *logp, float *entropy, float *log_sum, float *top_logp, int32_t *top_tokens, cocod_stream_t stream)
{
    const int es = size_of(type);
    if (!good_tokens(h, M, V, logits, ld, es, tokens, scale, top) ||
        (M > 0 && (!entropy || !log_sum || (tokens && !logp) || (top > 0 && (!top_logp || !top_tokens)))) ||
        !words_aligned({logp, entropy, log_sum, top_logp, top_tokens}))
        return COCOD_ERR_INVALID;
    if (M == 0) return COCOD_OK;
    TokenRows p{};
    p.logits = logits; p.ld = ld; p.rows = M; p.vocab = (int)V; p.top = top; p.scale = scale; p.tokens = tokens; p.logp = logp; p.entropy = entropy;
    p.log_sum = log_sum; p.top_logp = top_logp; p.top_tokens = top_tokens; p.error_flag = h->flag;
    const cudaStream_t s = (cudaStream_t)stream;
    return es == 2 ? run_logprobs<bf16>(h, p, s) : run_logprobs<float>(h, p, s);
}

int cocod_token_logprobs_grad(cocod_lm_handle *h, int64_t M, int64_t V, const void *logits, int64_t ld, int type, const int32_t *tokens, float scale, int top,
                              const int32_t *top_tokens, const float *log_sum, const float *entropy, const float *d_logp, const float *d_entropy,
                              const float *d_top, void *dlogits, int64_t ld_dlogits, cocod_stream_t stream)
{
    const int es = size_of(type);
    if (!good_tokens(h, M, V, logits, ld, es, tokens, scale, top) || !good_matrix(dlogits, ld_dlogits, V, M, es) ||
        (M > 0 && (!log_sum || (d_logp && !tokens) || (d_entropy && !entropy) || (top > 0 && (!top_tokens || !d_top)))) ||
        !words_aligned({top_tokens, log_sum, entropy, d_logp, d_entropy, d_top}))
        return COCOD_ERR_INVALID;
    if (M == 0) return COCOD_OK;
    TokenGrads p{};
    p.logits = logits; p.ld = ld; p.out = dlogits; p.ld_out = ld_dlogits; p.rows = M; p.vocab = (int)V; p.top = top; p.scale = scale; p.tokens = tokens;
    p.top_tokens = top_tokens; p.log_sum = log_sum; p.entropy = entropy; p.d_logp = d_logp; p.d_entropy = d_entropy; p.d_top = d_top; p.error_flag = h->flag;
    return es == 2 ? run_logprobs_grad<bf16>(h, p, (cudaStream_t)stream) : run_logprobs_grad<float>(h, p, (cudaStream_t)stream);
}

}  // extern "C"
