// Log probabilities of given tokens, with the entropy and the top alternatives, from logits that lie in memory; and their gradient.
//
// With y = scale * l, the row's reference m (its largest logit) and t = (l - m) * scale * log2(e):
//     S1 = sum 2^t,  S2 = sum 2^t t,   Z = scale m + ln S1,  log p_v = scale (l_v - m) - ln S1,  H = ln S1 - ln 2 * S2 / S1
// in one pass over the row: every thread holds a reference of its own, raised when a batch of its values exceeds it (S1' = c S1,
// S2' = c (S2 + d S1) with d = old - new reference in units of t, c = 2^d), and threads are joined by the same rule at the end.
//
// The top alternatives cost that pass nothing.  A thread's reference is its largest value, so that the k-th largest of 64 groups' maxima
// is a bound that at least k values reach and, as a rule, few more.  Only the threads that hold such a value look at their part of the row once
// more (it lies in L2), and the few values found are ranked by pairs: larger first, of equal ones the lower index, by whole numbers that are in
// the values' order (NaN above all, -0 equal to 0).
//
// Values that are not finite: a row with a NaN or +inf has NaN for its log probabilities and its entropy; -inf is a masked entry (p = 0); a
// row of nothing else has Z = -inf, log p = -inf, H = 0 and gradient 0.
//
// What bounds them: HBM, one reading (forward) or one reading and one writing (gradient) of the logits; the forward pass
// takes about seven issue slots a value of the eleven that bf16 leaves at the measured copy rate.
#pragma once
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "cocod_experts.cuh"

namespace cocod {
namespace lm {

constexpr int MAX_ALTERNATIVES = 32;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct TokenRows {
    const void *logits;
    long long ld;                            // row stride
    long long rows;
    int vocab, top;
    float scale;
    const int *tokens;                       // or nullptr: all rows take part, none has a token
    float *logp, *entropy, *log_sum;         // logp: not written without tokens
    float *top_logp;                         // rows x top
    int *top_tokens;
    int *error_flag;
};

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float minus_inf() { return __int_as_float(0xff800000); }

// Whole numbers in the order of the values; 0 is below every value's.
__device__ __forceinline__ uint32_t key_of(float x)
{
    if (x != x) return 0xffffffffu;
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key)
{
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
// ... and of value and index together: of equal values the lower index comes first.
__device__ __forceinline__ unsigned long long ranked(uint32_t key, int index) { return (unsigned long long)key << 32 | (0xffffffffu - (uint32_t)index); }
__device__ __forceinline__ int index_of(unsigned long long r) { return (int)(0xffffffffu - (uint32_t)r); }

// What is known of a part of a row: its reference and the two sums.
struct Sums {
    float most, s1, s2;
};
// The same sums relative to another reference that is not below (unit: scale * log2 e).
__device__ __forceinline__ Sums relative_to(const Sums &a, float most, float unit)
{
    if (a.most == minus_inf()) return Sums{most, 0.0f, 0.0f};
    const float d = (a.most - most) * unit, c = a.most == most ? 1.0f : exp2_fast(d);
    if (a.most == most || c == 0.0f) return Sums{most, c * a.s1, c * a.s2};
    return Sums{most, c * a.s1, c * fmaf(d, a.s1, a.s2)};
}

// The row's token: the label, -1 where the row takes no part (or has none).
struct RowToken {
    bool part;
    int token;
};
__device__ __forceinline__ RowToken row_token(const int *tokens, long long row, int vocab, int *error_flag, bool tell)
{
    if (tokens == nullptr) return RowToken{true, -1};
    const int t = tokens[row];
    if (t >= vocab && tell) atomicExch(error_flag, ERR_LABEL);
    return t < 0 || t >= vocab ? RowToken{false, -1} : RowToken{true, t};
}
template <typename T>
__device__ __forceinline__ float load_one(const T *p) { return as_float(*p); }

// A row that takes no part: `lane` of `lanes` threads write its zeros.
__device__ __forceinline__ void write_nothing(const TokenRows &p, long long row, int lane, int lanes)
{
    if (lane == 0) {
        p.logp[row] = 0.0f;
        p.entropy[row] = 0.0f;
        p.log_sum[row] = 0.0f;
    }
    for (int j = lane; j < p.top; j += lanes) {
        p.top_logp[row * p.top + j] = 0.0f;
        p.top_tokens[row * p.top + j] = -1;
    }
}
// (one thread)
__device__ __forceinline__ void write_row(const TokenRows &p, long long row, const Sums &a, float log_s1, float own)
{
    const bool empty = a.most == minus_inf();
    p.entropy[row] = empty ? 0.0f : log_s1 - LN2 * (a.s2 / a.s1);
    p.log_sum[row] = empty ? minus_inf() : fmaf(p.scale, a.most, log_s1);
    if (p.tokens != nullptr) p.logp[row] = empty ? minus_inf() : fmaf(p.scale, own - a.most, -log_s1);
}
__device__ __forceinline__ void write_top(const TokenRows &p, long long row, int j, unsigned long long r, const Sums &a, float log_s1)
{
    p.top_logp[row * p.top + j] = a.most == minus_inf() ? minus_inf() : fmaf(p.scale, value_of((uint32_t)(r >> 32)) - a.most, -log_s1);
    p.top_tokens[row * p.top + j] = index_of(r);
}

// ------------------------------------------------------------------------------------------ short rows: a warp for each
// The row (at most 32 * NR entries) lies in the lanes' registers: lane + 32 i is value i.
template <typename T, int NR>
__global__ void __launch_bounds__(256)
token_logprobs_warp(const TokenRows p)
{
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (row >= p.rows) return;
    const RowToken t = row_token(p.tokens, row, p.vocab, p.error_flag, lane == 0);
    if (!t.part) {
        write_nothing(p, row, lane, 32);
        return;
    }
    const T *x = static_cast<const T *>(p.logits) + row * p.ld;
    const float own = t.token >= 0 ? load_one(x + t.token) : 0.0f;
    float v[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) v[i] = lane + 32 * i < p.vocab ? load_one(x + lane + 32 * i) : minus_inf();
    uint32_t key[NR], best = 0;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        key[i] = lane + 32 * i < p.vocab ? key_of(v[i]) : 0;
        best = max(best, key[i]);
    }
    Sums a{0.0f, 0.0f, 0.0f};
    a.most = value_of(__reduce_max_sync(~0u, best));
    const float unit = p.scale * LOG2E, m = a.most == minus_inf() ? 0.0f : a.most;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const float d = (v[i] - m) * unit, e = exp2_fast(d);
        a.s1 += e;
        a.s2 = fmaf(e, fmaxf(d, -1.0e4f), a.s2);          // (0 * -inf)
    }
#pragma unroll
    for (int d = 16; d > 0; d /= 2) {
        a.s1 += __shfl_xor_sync(~0u, a.s1, d);
        a.s2 += __shfl_xor_sync(~0u, a.s2, d);
    }
    const float log_s1 = logf(a.s1);
    if (lane == 0) write_row(p, row, a, log_s1, own);
    // one after the other: the lanes' largest, the lowest index that has it, and its lane takes it out
    unsigned long long mine = 0;
    for (int j = 0; j < p.top; ++j) {
        const uint32_t most = __reduce_max_sync(~0u, best);
        int at = 0x7fffffff;
        if (best == most) {
#pragma unroll
            for (int i = NR - 1; i >= 0; --i)
                if (key[i] == most) at = lane + 32 * i;
        }
        const int first = (int)__reduce_min_sync(~0u, (unsigned)at);
        if (lane == j) mine = ranked(most, first);
        if (at == first) {
            best = 0;
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                if (lane + 32 * i == first) key[i] = 0;
                best = max(best, key[i]);
            }
        }
    }
    if (lane < p.top) write_top(p, row, lane, mine, a, log_s1);
}

// ------------------------------------------------------------------------------------------ long rows: one to eight thread blocks for each
__device__ __forceinline__ uint64_t pack2(float a, float b)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(uint64_t r, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b)        // NaN if one is
{
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// 16 bytes of logits: N values.
template <typename T> struct Word {
    static constexpr int N = 16 / sizeof(T);
};
template <typename T> __device__ __forceinline__ uint4 all_masked()
{
    const uint32_t w = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
    return make_uint4(w, w, w, w);
}
template <typename T, int U>
__device__ __forceinline__ float largest(const uint4 (&r)[U])
{
    if constexpr (sizeof(T) == 2) {
        uint32_t m = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t a = max_bf16x2(max_bf16x2(r[u].x, r[u].y), max_bf16x2(r[u].z, r[u].w));
            m = u ? max_bf16x2(m, a) : a;
        }
        return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
    } else {
        float m = 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float a = max_nan(max_nan(__uint_as_float(r[u].x), __uint_as_float(r[u].y)), max_nan(__uint_as_float(r[u].z), __uint_as_float(r[u].w)));
            m = u ? max_nan(m, a) : a;
        }
        return m;
    }
}
template <typename T>
__device__ __forceinline__ void values_of(const uint4 &r, float (&x)[Word<T>::N])
{
    Piece<T, true> q;
    q.raw = r;
    widen<T, true>(q, x);
}

// A row's words: 16 aligned bytes each.  The first and the last may hold values that are not the row's; those ("ends") go one by one.
struct RowWords {
    int lead;                                // values before the row in the first word
    int full_from, full_to;                  // words that are the row's alone
    int words;
};
template <typename T>
__device__ __forceinline__ RowWords row_words(const T *x, int vocab)
{
    constexpr int N = Word<T>::N;
    RowWords w;
    w.lead = (int)((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(T));
    w.words = (int)(((long long)w.lead + vocab + N - 1) / N);
    w.full_from = w.lead ? 1 : 0;
    w.full_to = (int)(((long long)w.lead + vocab) / N);
    return w;
}

constexpr int TOP_GROUPS = 64, TOP_FOUND = 512;

template <int THREADS>
struct LogprobsShared {
    uint32_t group[TOP_GROUPS];              // the largest key of each group of threads
    float s1[THREADS / 32], s2[THREADS / 32];
    Sums part;                               // this thread block's
    uint32_t bound;
    int found;
    int scan[THREADS / 32];
    unsigned long long list[TOP_FOUND];
    unsigned long long best[MAX_ALTERNATIVES];
    unsigned long long round[THREADS / 32];
};

// A value that reaches the bound (above: exceeds it) goes into the list, as long as there is room; all are counted.
__device__ __forceinline__ void note_found(unsigned long long *list, int *found, uint32_t key, uint32_t bound, bool above, int index)
{
    if (above ? key > bound : key >= bound) {
        const int at = atomicAdd(found, 1);
        if (at < TOP_FOUND) list[at] = ranked(key, index);
    }
}

// The slice of a row that a thread block works on.
template <typename T>
struct Slice {
    const T *x;
    RowWords w;
    int from, to;                            // words that are full: word from + thread + n * THREADS is the thread's
    long long first, last;                   // values
    int ends;                                // this thread's value of a word that is not full: its index, or -1
};

// The k best of a slice, in order, in sh.best (0 where there are fewer).  most: the thread's largest value's key (0: it had none).
template <typename T, int THREADS>
__device__ void find_top(LogprobsShared<THREADS> &sh, const Slice<T> &s, uint32_t most, int k)
{
    constexpr int N = Word<T>::N;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (warp == 0) {                         // the k-th largest of the groups' maxima
        const uint32_t a = sh.group[lane], b = sh.group[lane + 32];
        int before_a = 0, before_b = 0;
#pragma unroll 8
        for (int i = 0; i < TOP_GROUPS; ++i) {
            const uint32_t o = sh.group[i];
            before_a += o > a || (o == a && i < lane);
            before_b += o > b || (o == b && i < lane + 32);
        }
        if (before_a == k - 1) sh.bound = a;
        if (before_b == k - 1) sh.bound = b;
        if (lane == 0) sh.found = 0;
    }
    __syncthreads();
    const uint32_t bound = sh.bound;
    // Every value that reaches it (above: exceeds it), from the threads whose largest does: their warp reads their words together.
    auto collect = [&](bool above) {
        unsigned who = __ballot_sync(~0u, most != 0 && (above ? most > bound : most >= bound));
        if (s.ends >= 0) note_found(sh.list, &sh.found, key_of(load_one(s.x + s.ends)), bound, above, s.ends);
        while (who) {
            const int l = __ffs(who) - 1;
            who &= who - 1;
            for (int i = s.from + warp * 32 + l + lane * THREADS; i < s.to; i += 32 * THREADS) {
                const uint4 r = reinterpret_cast<const uint4 *>(s.x - s.w.lead)[i];
                float x[N];
                values_of<T>(r, x);
                const int at = i * N - s.w.lead;
#pragma unroll
                for (int e = 0; e < N; ++e) note_found(sh.list, &sh.found, key_of(x[e]), bound, above, at + e);
            }
        }
        __syncthreads();
    };
    collect(false);
    int n = sh.found;
    __syncthreads();
    if (n > TOP_FOUND) {                     // many equal values: those above the bound ...
        if (tid == 0) sh.found = 0;
        __syncthreads();
        collect(true);
        n = sh.found;
        __syncthreads();
        if (n <= TOP_FOUND - MAX_ALTERNATIVES) {
            // ... and of those equal to it the first ones, in the row's order
            const int need = max(0, k - n);
            int have = 0;
            for (long long i0 = s.first; i0 < s.last && have < need; i0 += THREADS * N) {
                const long long i = i0 + tid * N;
                unsigned equal = 0;
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (i + e < s.last && key_of(load_one(s.x + i + e)) == bound) equal |= 1u << e;
                int sum = __popc(equal);
                const int own = sum;
#pragma unroll
                for (int d = 1; d < 32; d *= 2) {
                    const int o = __shfl_up_sync(~0u, sum, d);
                    if (lane >= d) sum += o;
                }
                if (lane == 31) sh.scan[warp] = sum;
                __syncthreads();
                int at = have + sum - own, all = 0;
                for (int w = 0; w < THREADS / 32; ++w) {
                    if (w < warp) at += sh.scan[w];
                    all += sh.scan[w];
                }
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (equal >> e & 1) {
                        if (at < need) sh.list[n + at] = ranked(bound, (int)(i + e));
                        ++at;
                    }
                have += all;
                __syncthreads();
            }
            n += min(have, need);
        } else {
            n = -1;
        }
    }
    if (n >= 0) {                            // ranked by pairs (all are different)
        for (int i = tid; i < n; i += THREADS) {
            const unsigned long long r = sh.list[i];
            int before = 0;
            for (int o = 0; o < n; ++o) before += sh.list[o] > r;
            if (before < k) sh.best[before] = r;
        }
        for (int i = n + tid; i < k; i += THREADS) sh.best[i] = 0;
        __syncthreads();
        return;
    }
    // A row made so that many values lie above the bound: one after the other.
    unsigned long long last = ~0ull;
    for (int j = 0; j < k; ++j) {
        unsigned long long best = 0;
        if (s.ends >= 0) {
            const unsigned long long r = ranked(key_of(load_one(s.x + s.ends)), s.ends);
            if (r < last) best = r;
        }
        for (int i = s.from + tid; i < s.to; i += THREADS) {
            const uint4 raw = reinterpret_cast<const uint4 *>(s.x - s.w.lead)[i];
            float x[N];
            values_of<T>(raw, x);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const unsigned long long r = ranked(key_of(x[e]), i * N + e - s.w.lead);
                if (r < last && r > best) best = r;
            }
        }
#pragma unroll
        for (int d = 16; d > 0; d /= 2) {
            const unsigned long long o = __shfl_xor_sync(~0u, best, d);
            best = o > best ? o : best;
        }
        if (lane == 0) sh.round[warp] = best;
        __syncthreads();
        best = 0;
        for (int w = 0; w < THREADS / 32; ++w) best = sh.round[w] > best ? sh.round[w] : best;
        if (tid == 0) sh.best[j] = best;
        last = best;
        __syncthreads();
    }
}

// The two sums of U words' values relative to `most`.
template <typename T, int U>
__device__ __forceinline__ void add_words(const uint4 (&r)[U], float most, float unit, uint64_t &s1, uint64_t &s2)
{
    const float ref = most == minus_inf() ? 0.0f : -most;
    const uint64_t shift = pack2(ref, ref), factor = pack2(unit, unit);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float x[Word<T>::N];
        values_of<T>(r[u], x);
#pragma unroll
        for (int e = 0; e < Word<T>::N; e += 2) {
            float d0, d1;
            unpack2(mul2(add2(pack2(x[e], x[e + 1]), shift), factor), d0, d1);
            const uint64_t y = pack2(exp2_fast(d0), exp2_fast(d1));
            s1 = add2(s1, y);
            s2 = fma2(y, pack2(fmaxf(d0, -1.0e4f), fmaxf(d1, -1.0e4f)), s2);          // (0 * -inf)
        }
    }
}
// A thread's running sums (two of each, for the even and the odd values).
struct Running {
    float most;
    uint64_t s1, s2;
};
__device__ __forceinline__ void raise(Running &a, float most, float unit)
{
    const float next = max_nan(a.most, most);
    if (a.most != minus_inf()) {
        const float d = (a.most - next) * unit, c = exp2_fast(d), d_ = c == 0.0f ? 0.0f : d;
        a.s2 = mul2(pack2(c, c), fma2(pack2(d_, d_), a.s1, a.s2));
        a.s1 = mul2(pack2(c, c), a.s1);
    }
    a.most = next;
}

// `blocks` thread blocks (a cluster where there are more than one) take a row; each takes a stretch of its words.
template <typename T, int THREADS, bool TOP>
__global__ void __launch_bounds__(THREADS)
token_logprobs_row(const TokenRows p, int blocks)
{
    constexpr int N = Word<T>::N, U = 4;
    __shared__ LogprobsShared<THREADS> sh;
    namespace cg = cooperative_groups;
    pdl_launch_dependents();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = blockIdx.x % blocks;
    if (tid < TOP_GROUPS) sh.group[tid] = 0;
    pdl_wait();
    const long long row = blockIdx.x / blocks;
    const RowToken t = row_token(p.tokens, row, p.vocab, p.error_flag, tid == 0);
    if (!t.part) {                           // (the whole cluster)
        if (rank == 0) write_nothing(p, row, tid, THREADS);
        return;
    }
    Slice<T> s;
    s.x = static_cast<const T *>(p.logits) + row * p.ld;
    s.w = row_words(s.x, p.vocab);
    const int per = (s.w.words + blocks - 1) / blocks, lo = min(rank * per, s.w.words), hi = min(lo + per, s.w.words);
    s.from = max(lo, s.w.full_from);
    s.to = min(hi, s.w.full_to);
    s.first = max(0ll, (long long)lo * N - s.w.lead);
    s.last = min((long long)p.vocab, (long long)hi * N - s.w.lead);
    s.ends = -1;
    if (lo == 0 && lo < hi && tid >= s.w.lead && tid < N && s.w.lead > 0) s.ends = tid - s.w.lead;
    if (hi == s.w.words && lo < hi && s.w.full_to < s.w.words && tid >= 32 && tid < 32 + N) {
        const long long at = (long long)s.w.full_to * N - s.w.lead + (tid - 32);
        if (at < p.vocab) s.ends = (int)at;
    }
    const float own = tid == 0 && rank == 0 && t.token >= 0 ? load_one(s.x + t.token) : 0.0f;
    const float unit = p.scale * LOG2E;
    Running a{minus_inf(), 0, 0};
    const uint4 *words = reinterpret_cast<const uint4 *>(s.x - s.w.lead);
    for (int i = s.from + tid; i < s.to; i += U * THREADS) {
        uint4 r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) r[u] = i + u * THREADS < s.to ? words[i + u * THREADS] : all_masked<T>();
        const float most = largest<T, U>(r);
        if (!(most <= a.most)) raise(a, most, unit);
        add_words<T, U>(r, a.most, unit, a.s1, a.s2);
    }
    const bool any = s.from + tid < s.to || s.ends >= 0;
    if (s.ends >= 0) {
        const float x = load_one(s.x + s.ends);
        if (!(x <= a.most)) raise(a, x, unit);
        const float d = (x - (a.most == minus_inf() ? 0.0f : a.most)) * unit, e = exp2_fast(d);
        a.s1 = add2(a.s1, pack2(e, 0.0f));
        a.s2 = add2(a.s2, pack2(e * fmaxf(d, -1.0e4f), 0.0f));
    }
    // the threads' sums, relative to the largest of all
    const uint32_t most = any ? key_of(a.most) : 0;
    __syncthreads();                         // (the groups are zero)
    if (any) atomicMax(&sh.group[tid % TOP_GROUPS], most);
    __syncthreads();
    const uint32_t top = __reduce_max_sync(~0u, max(sh.group[lane], sh.group[lane + 32]));
    float lo1, hi1, lo2, hi2;
    unpack2(a.s1, lo1, hi1);
    unpack2(a.s2, lo2, hi2);
    Sums b = relative_to(Sums{a.most, lo1 + hi1, lo2 + hi2}, top ? value_of(top) : minus_inf(), unit);
#pragma unroll
    for (int d = 16; d > 0; d /= 2) {
        b.s1 += __shfl_xor_sync(~0u, b.s1, d);
        b.s2 += __shfl_xor_sync(~0u, b.s2, d);
    }
    if (lane == 0) {
        sh.s1[warp] = b.s1;
        sh.s2[warp] = b.s2;
    }
    __syncthreads();
    if (warp == 0) {
        float s1 = lane < THREADS / 32 ? sh.s1[lane] : 0.0f, s2 = lane < THREADS / 32 ? sh.s2[lane] : 0.0f;
#pragma unroll
        for (int d = 16; d > 0; d /= 2) {
            s1 += __shfl_xor_sync(~0u, s1, d);
            s2 += __shfl_xor_sync(~0u, s2, d);
        }
        b.s1 = s1;
        b.s2 = s2;
        if (lane == 0) sh.part = b;
    }
    if constexpr (TOP) find_top<T, THREADS>(sh, s, most, p.top);
    if (blocks == 1) {
        const float log_s1 = TOP || tid == 0 ? logf(TOP ? sh.part.s1 : b.s1) : 0.0f;      // (thread 0 wrote sh.part itself; find_top ends with a barrier)
        if (tid == 0) write_row(p, row, b, log_s1, own);
        if (TOP && tid < p.top) write_top(p, row, tid, sh.best[tid], sh.part, log_s1);
        return;
    }
    auto cluster = cg::this_cluster();
    cluster.sync();
    if (rank == 0) {
        Sums all{minus_inf(), 0.0f, 0.0f};
        uint32_t key = 0;
        for (int c = 0; c < blocks; ++c) key = max(key, key_of(cluster.map_shared_rank(&sh, c)->part.most));
        all.most = value_of(key);
        for (int c = 0; c < blocks; ++c) {
            const Sums o = relative_to(cluster.map_shared_rank(&sh, c)->part, all.most, unit);
            all.s1 += o.s1;
            all.s2 += o.s2;
        }
        const float log_s1 = logf(all.s1);
        if (tid == 0) write_row(p, row, all, log_s1, own);
        if constexpr (TOP) {
            const int n = blocks * p.top;    // (up to 8 * 32)
            for (int i = tid; i < n; i += THREADS) sh.list[i] = cluster.map_shared_rank(&sh, i / p.top)->best[i % p.top];
            __syncthreads();
            for (int i = tid; i < n; i += THREADS) {
                const unsigned long long r = sh.list[i];
                int before = 0;
                for (int o = 0; o < n; ++o) before += sh.list[o] > r;
                if (r != 0 && before < p.top) write_top(p, row, before, r, all, log_s1);
            }
        }
    }
    cluster.sync();                          // (the others' shared memory is read until here)
}

// ------------------------------------------------------------------------------------------ the gradient
// dl_v = scale * (sum of the given gradients at v - p_v (A + g_H (log p_v + H))), A: the sum of all given gradients of the row.  A thread block
// takes GRAD_WORDS words a thread of one row.  The few entries with a gradient of their own are written once more by one thread
// each, from the logit read before (the result may lie on the logits).
struct TokenGrads {
    const void *logits;
    long long ld;
    void *out;
    long long ld_out;
    long long rows;
    int vocab, top;
    float scale;
    const int *tokens, *top_tokens;
    const float *log_sum, *entropy, *d_logp, *d_entropy, *d_top;
    int *error_flag;
};
constexpr int GRAD_THREADS = 256, GRAD_WORDS = 4;

// TOGETHER: in every row the result lies at the same alignment as the logits.
template <typename T, bool TOGETHER>
__global__ void __launch_bounds__(GRAD_THREADS)
token_logprobs_grad(const TokenGrads p, int parts)
{
    constexpr int N = Word<T>::N;
    pdl_launch_dependents();
    pdl_wait();
    __shared__ int at[MAX_ALTERNATIVES + 1];
    __shared__ float given[MAX_ALTERNATIVES + 1];
    const int tid = threadIdx.x;
    const long long row = blockIdx.x / parts;
    const int part = (int)(blockIdx.x - row * parts);
    const T *x = static_cast<const T *>(p.logits) + row * p.ld;
    T *out = static_cast<T *>(p.out) + row * p.ld_out;
    const RowWords w = row_words(x, p.vocab);
    const int from = part * GRAD_THREADS * GRAD_WORDS, to = min(from + GRAD_THREADS * GRAD_WORDS, w.words);
    if (from >= to) return;
    const RowToken t = row_token(p.tokens, row, p.vocab, p.error_flag, tid == 0 && part == 0);
    const float z = p.log_sum[row];
    const bool nothing = !t.part || z == minus_inf();
    const uint4 *words = reinterpret_cast<const uint4 *>(x - w.lead);
    uint4 r[GRAD_WORDS];
#pragma unroll
    for (int u = 0; u < GRAD_WORDS; ++u) {
        const int i = from + tid + u * GRAD_THREADS;
        if (i < to && i >= w.full_from && i < w.full_to) {
            r[u] = words[i];
        } else if (i < to) {
            float v[N];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const long long c = (long long)i * N + e - w.lead;
                v[e] = c >= 0 && c < p.vocab ? load_one(x + c) : 0.0f;
            }
            if constexpr (sizeof(T) == 2) r[u] = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4 % N], v[5 % N]), pack_bf16x2(v[6 % N], v[7 % N]));
            else r[u] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        }
    }
    // the row's few entries of their own
    const int n = p.top + 1;
    if (tid < n) {
        int c = -1;
        float g = 0.0f;
        if (tid == 0 && t.token >= 0 && p.d_logp != nullptr) {
            c = t.token;
            g = p.d_logp[row];
        }
        if (tid > 0 && t.part) {
            c = p.top_tokens[row * p.top + tid - 1];
            g = p.d_top[row * p.top + tid - 1];
            if (c >= p.vocab && part == 0) atomicExch(p.error_flag, ERR_LABEL);
            if (c < 0 || c >= p.vocab) c = -1, g = 0.0f;
        }
        at[tid] = c;
        given[tid] = g;
    }
    __syncthreads();
    float every = 0.0f;
    for (int j = 0; j < n; ++j) every += given[j];
    const float gh = p.d_entropy != nullptr && t.part ? p.d_entropy[row] : 0.0f, h = gh != 0.0f ? p.entropy[row] : 0.0f;
    const float base = fmaf(gh, h, every);
    // (the entries' own: the first of equal ones takes them all; its logit is read before anything is written)
    const long long c0 = (long long)from * N - w.lead, c1 = (long long)to * N - w.lead;
    bool special = false;
    float special_x = 0.0f, special_g = 0.0f;
    if (tid < n && at[tid] >= 0 && at[tid] >= c0 && at[tid] < c1 && !nothing) {
        special = true;
        for (int j = 0; j < n; ++j) {
            if (at[j] != at[tid]) continue;
            special = special && j >= tid;
            special_g += given[j];
        }
        special_x = load_one(x + at[tid]);
    }
    __syncthreads();
    const uint64_t mul = pack2(p.scale, p.scale), sub = pack2(-z, -z), l2 = pack2(LOG2E, LOG2E), ghs = pack2(gh, gh), bases = pack2(base, base),
                   minus = pack2(-p.scale, -p.scale);
#pragma unroll
    for (int u = 0; u < GRAD_WORDS; ++u) {
        const int i = from + tid + u * GRAD_THREADS;
        if (i >= to) break;
        float v[N];
        values_of<T>(r[u], v);
#pragma unroll
        for (int e = 0; e < N; e += 2) {
            float d0, d1, e0, e1;
            const uint64_t lp = fma2(pack2(v[e], v[e + 1]), mul, sub);
            unpack2(lp, d0, d1);
            unpack2(mul2(lp, l2), e0, e1);
            const uint64_t prob = mul2(pack2(exp2_fast(e0), exp2_fast(e1)), minus);
            unpack2(mul2(prob, fma2(ghs, pack2(fmaxf(d0, -1.0e4f), fmaxf(d1, -1.0e4f)), bases)), v[e], v[e + 1]);
        }
        if (nothing)
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = 0.0f;
        if (TOGETHER && i >= w.full_from && i < w.full_to) {
            store_values<T, N>(out + ((long long)i * N - w.lead), v);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const long long c = (long long)i * N + e - w.lead;
                if (c >= 0 && c < p.vocab) store_values<T, 1>(out + c, reinterpret_cast<const float (&)[1]>(v[e]));
            }
        }
    }
    __syncthreads();
    if (special) {
        // c (1 - p) - p (the others' + g_H (log p + H)): as exact near p = 1 as 1 - p itself
        const float lp = fmaf(special_x, p.scale, -z), prob = exp2_fast(lp * LOG2E);
        const float g[1] = {p.scale * (special_g * -expm1f(lp) - prob * fmaf(gh, fmaxf(lp, -1.0e4f), base - special_g))};
        store_values<T, 1>(out + at[tid], g);
    }
}

}  // namespace lm
}  // namespace cocod
