// Log probabilities of given tokens, with the entropy and the top alternatives, from logits that lie in memory; and their gradient.
//
// With y = scale * l, the row's reference m (its largest logit) and t = (l - m) * scale * log2(e):
//     S1 = sum 2^t,  S2 = sum 2^t t,   Z = scale m + ln S1,  log p_v = scale (l_v - m) - ln S1,  H = ln S1 - ln 2 * S2 / S1
// in one pass over the row: a warp's threads share a reference, the largest logit that the warp has seen, and change it together when a batch exceeds it (S1' = c S1,
// S2' = c (S2 + d S1) with d = old - new reference in units of t, c = 2^d); warps are joined by the same rule at the end.  The largest logit's own term, (1, 0)
// exactly, is not in the thread's sums but counted beside them: S1 = n + (the others), so that ln S1 = log1p(n - 1 + the others) and what a confident row has beside its
// largest logit is not lost in rounding; no log p is above 0, and no entropy below.  (Rows of 4000 to 128256 entries with one 20 to 40 above
// the others: log p and H are off by up to 2.1e-7; with a thread's references, kept until a value was 2^64 times the reference's, by 3.1e-6 and 2.0e-5, of either sign.)
//
// The top alternatives cost that pass next to nothing.  The largest of each batch of 32 values is needed there anyway; every thread keeps those of its
// batches (up to eight, or of as many groups of batches).  The k-th largest of 64 groups' maxima is a bound that at least k values reach and, as a rule, few more.
// Only the batches that hold such a value are looked at once more (they lie in L2), a warp for each, and the few values found are ranked by
// pairs: larger first, of equal ones the lower index, by whole numbers that are in the values' order (NaN above all, -0 equal to 0).
//
// Values that are not finite: a row with a NaN or +inf has NaN for its log probabilities and its entropy; -inf is a masked entry (p = 0); a
// row of nothing else has Z = -inf, log p = -inf, H = 0 and gradient 0.
//
// What bounds them: HBM, one reading (forward) or one reading and one writing (gradient) of the logits, of long rows in bf16 (4096 x 65536, other logits every time: 97 us and
// 5.5 TB/s without alternatives, 108 with five; the gradient of 4096 x 50001 138 us, 5.9 TB/s): the forward pass takes eight issue slots a value of the eleven that the
// copy rate leaves.  Of short rows what follows the pass: its barriers, the second look and the ranking wait for one another, and a thread block has
// nothing else to do (32768 x 4000: 58 us without alternatives, 86 with five, 130 with twenty; one reading would take 40).
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
__device__ __forceinline__ float reciprocal_fast(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
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

// What is known of a part of a row: its reference and the two sums, of S1 without n terms that are the reference's own (1 each, and 0 in S2).
struct Sums {
    float most, s1, s2;
    int n;
};
// The same sums relative to another reference that is not below (unit: scale * log2 e).
__device__ __forceinline__ Sums relative_to(const Sums &a, float most, float unit)
{
    if (a.most == most) return a;
    if (a.most == minus_inf()) return Sums{most, 0.0f, 0.0f, 0};
    const float d = (a.most - most) * unit, c = exp2_fast(d), s1 = a.s1 + (float)a.n;
    return c == 0.0f ? Sums{most, 0.0f, 0.0f, 0} : Sums{most, c * s1, c * fmaf(d, s1, a.s2), 0};
}
// ln S1 of a whole row; then its S1 is the whole sum.  (S2 has no positive term: what roundings leave above 0 is 0.)
__device__ __forceinline__ float complete(Sums &a)
{
    const float log_s1 = log1pf((float)(a.n - 1) + a.s1);
    a.s1 += (float)a.n;
    a.s2 = a.s2 > 0.0f ? 0.0f : a.s2;
    return log_s1;
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

// ------------------------------------------------------------------------------------------ short rows: LANES lanes for each
// The row (at most LANES * NR entries) lies in the lanes' registers: lane + LANES * i is value i.
template <typename T, int LANES, int NR>
__global__ void __launch_bounds__(256)
token_logprobs_short(const TokenRows p)
{
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x % LANES;
    const unsigned mask = LANES == 32 ? ~0u : ((1u << (LANES % 32)) - 1) << ((threadIdx.x & 31) / LANES * LANES);
    const long long row = (long long)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    if (row >= p.rows) return;
    const T *x = static_cast<const T *>(p.logits) + row * p.ld;
    float v[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) v[i] = lane + LANES * i < p.vocab ? load_one(x + lane + LANES * i) : minus_inf();
    const RowToken t = row_token(p.tokens, row, p.vocab, p.error_flag, lane == 0);
    if (!t.part) {
        write_nothing(p, row, lane, LANES);
        return;
    }
    const float own = t.token >= 0 && lane == 0 ? load_one(x + t.token) : 0.0f;
    uint32_t key[NR], best = 0;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        key[i] = lane + LANES * i < p.vocab ? key_of(v[i]) : 0;
        best = max(best, key[i]);
    }
    Sums a{0.0f, 0.0f, 0.0f, 0};
    a.most = value_of(__reduce_max_sync(mask, best));
    const float unit = p.scale * LOG2E, m = a.most == minus_inf() ? 0.0f : a.most;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const float d = (v[i] - m) * unit, e = exp2_fast(d);
        a.s1 += e;
        a.s2 = fmaf(e, fmaxf(d, -1.0e4f), a.s2);          // (0 * -inf)
    }
#pragma unroll
    for (int d = LANES / 2; d > 0; d /= 2) {
        a.s1 += __shfl_xor_sync(mask, a.s1, d);
        a.s2 += __shfl_xor_sync(mask, a.s2, d);
    }
    const float log_s1 = logf(a.s1);
    if (lane == 0) write_row(p, row, a, log_s1, own);
    // one after the other: the lanes' largest, the lowest index that has it, and its lane takes it out
    for (int j = 0; j < p.top; ++j) {
        const uint32_t most = __reduce_max_sync(mask, best);
        unsigned at = 0x7fffffff;
        if (best == most) {
#pragma unroll
            for (int i = NR - 1; i >= 0; --i)
                if (key[i] == most) at = lane + LANES * i;
        }
        const unsigned first = __reduce_min_sync(mask, at);
        if (at == first) {
            write_top(p, row, j, ranked(most, (int)first), a, log_s1);
            best = 0;
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                if (lane + LANES * i == (int)first) key[i] = 0;
                best = max(best, key[i]);
            }
        }
    }
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
__device__ __forceinline__ float warp_max_nan(float x)
{
    float r;
    asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
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

constexpr int TOP_GROUPS = 64, TOP_SLOTS = 8, TOP_BATCHES = 256;
template <int THREADS> constexpr int TOP_FOUND = THREADS == 32 ? 256 : 512;

template <int THREADS>
struct LogprobsShared {
    __align__(16) uint32_t group[TOP_GROUPS];  // the largest key of each group of batches
    uint32_t slot[TOP_SLOTS][THREADS];       // the largest key of each batch (or group of batches) of a thread
    float s1[(THREADS + 31) / 32], s2[(THREADS + 31) / 32];
    int n[(THREADS + 31) / 32];
    Sums part;                               // this thread block's
    uint32_t bound;
    int batches, found;
    int scan[THREADS / 32];
    int batch[TOP_BATCHES];                  // the first words of those that reach the bound
    unsigned long long list[TOP_FOUND<THREADS>];
    unsigned long long best[MAX_ALTERNATIVES];
    unsigned long long round[THREADS / 32];
};

// The slice of a row that a thread block works on.
template <typename T>
struct Slice {
    const T *x;
    RowWords w;
    int from, to;                            // words that are full: word from + thread + n * THREADS is the thread's
    long long first, last;                   // values
    int ends;                                // this thread's value of a word that is not full: its index, or -1
    int per_slot;                            // a slot is so many batches of a thread
};
// A batch is what a thread takes at once: BATCH values.
constexpr int BATCH = 32;
template <typename T> constexpr int BATCH_WORDS = BATCH / Word<T>::N;

// A row's threads: the whole block, or, where 32 take it, one warp of a block that works on several rows.
template <int THREADS> __device__ __forceinline__ void team_sync()
{
    if constexpr (THREADS == 32) __syncwarp();
    else __syncthreads();
}

// Where the lanes of a warp that have something to put into a list put it, for N such things at a time (all lanes call; `count`: what the list holds,
// and would hold if it were longer).
template <int N>
__device__ __forceinline__ void places_in(const bool (&mine)[N], int (&at)[N], int *count, int lane)
{
    int total = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const unsigned who = __ballot_sync(~0u, mine[i]);
        at[i] = total + __popc(who & ((1u << lane) - 1));
        total += __popc(who);
    }
    if (total == 0) return;
    int first = 0;
    if (lane == 0) first = atomicAdd(count, total);
    first = __shfl_sync(~0u, first, 0);
#pragma unroll
    for (int i = 0; i < N; ++i) at[i] += first;
}

// The k best of a slice, in order, in sh.best (0 where there are fewer).  slots: of this thread.
template <typename T, int THREADS>
__device__ void find_top(LogprobsShared<THREADS> &sh, const Slice<T> &s, int slots, int k)
{
    constexpr int N = Word<T>::N, U = BATCH_WORDS<T>, WARPS = THREADS / 32;
    const int tid = threadIdx.x % THREADS, lane = tid & 31, warp = tid >> 5;
    if (warp == 0) {                         // the k-th largest of the groups' maxima
        const uint32_t a = sh.group[lane], b = sh.group[lane + 32];
        uint32_t more = max(a, b), less = min(a, b), most = 0;
        for (int n = 0; n < k;) {            // (a lane whose larger one is taken has its smaller one left; by pairs, k = 5 and 20, it took 5 us longer for 4096 x 65536)
            most = __reduce_max_sync(~0u, more);
            const bool taken = more == most;
            n += __popc(__ballot_sync(~0u, taken));
            more = taken ? less : more;
            less = taken ? 0 : less;
        }
        if (lane == 0) {
            sh.bound = most;
            sh.found = sh.batches = 0;
        }
    }
    team_sync<THREADS>();
    const uint32_t bound = sh.bound;
    const int my_word = lane / N * THREADS, my_value = lane % N - s.w.lead, slot_words = s.per_slot * U * THREADS;
    // Every value that reaches it (above: exceeds it): the batches that hold one are listed, and a warp reads each.
    auto collect = [&](bool above) {
        {
            bool mine[TOP_SLOTS];
            int at[TOP_SLOTS];
#pragma unroll
            for (int i = 0; i < TOP_SLOTS; ++i) {
                const uint32_t most = i < slots ? sh.slot[i][tid] : 0;
                mine[i] = i < slots && (above ? most > bound : most >= bound);
            }
            places_in<TOP_SLOTS>(mine, at, &sh.batches, lane);
#pragma unroll
            for (int i = 0; i < TOP_SLOTS; ++i)
                if (mine[i] && at[i] < TOP_BATCHES) sh.batch[at[i]] = s.from + tid + i * slot_words;
        }
        if (warp == 0) {                     // (the ends are its lanes')
            const uint32_t key = s.ends >= 0 ? key_of(load_one(s.x + s.ends)) : 0;
            const bool mine[1] = {s.ends >= 0 && (above ? key > bound : key >= bound)};
            int at[1];
            places_in<1>(mine, at, &sh.found, lane);
            if (mine[0] && at[0] < TOP_FOUND<THREADS>) sh.list[at[0]] = ranked(key, s.ends);
        }
        team_sync<THREADS>();
        const int n = min(sh.batches, TOP_BATCHES);
        constexpr int AT_ONCE = 4;
        for (int b0 = warp; b0 < n; b0 += AT_ONCE * WARPS) {
            for (int g = 0; g < s.per_slot; ++g) {
                uint32_t key[AT_ONCE];
                int value[AT_ONCE], at[AT_ONCE];
                bool mine[AT_ONCE];
#pragma unroll
                for (int a = 0; a < AT_ONCE; ++a) {
                    const int b = b0 + a * WARPS, word = sh.batch[min(b, n - 1)] + g * (U * THREADS) + my_word;
                    value[a] = word * N + my_value;
                    mine[a] = b < n && word < s.to;
                    key[a] = mine[a] ? key_of(load_one(s.x + value[a])) : 0;
                }
#pragma unroll
                for (int a = 0; a < AT_ONCE; ++a) mine[a] = mine[a] && (above ? key[a] > bound : key[a] >= bound);
                places_in<AT_ONCE>(mine, at, &sh.found, lane);
#pragma unroll
                for (int a = 0; a < AT_ONCE; ++a)
                    if (mine[a] && at[a] < TOP_FOUND<THREADS>) sh.list[at[a]] = ranked(key[a], value[a]);
            }
        }
        team_sync<THREADS>();
        return sh.batches <= TOP_BATCHES && sh.found <= TOP_FOUND<THREADS>;
    };
    bool fits = collect(false);
    int n = sh.found;
    team_sync<THREADS>();
    if (!fits) {                             // many equal values: those above the bound ...
        if (tid == 0) sh.found = sh.batches = 0;
        team_sync<THREADS>();
        fits = collect(true);
        n = sh.found;
        team_sync<THREADS>();
        if (fits && n <= TOP_FOUND<THREADS> - MAX_ALTERNATIVES) {
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
                team_sync<THREADS>();
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
                team_sync<THREADS>();
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
        team_sync<THREADS>();
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
        team_sync<THREADS>();
        best = 0;
        for (int w = 0; w < THREADS / 32; ++w) best = sh.round[w] > best ? sh.round[w] : best;
        if (tid == 0) sh.best[j] = best;
        last = best;
        team_sync<THREADS>();
    }
}

// A thread's running sums (two of each, for the even and the odd values), relative to its warp's reference.
//
// The exponent of a value is x * unit - R with R = ref * unit rounded: one instruction for two values.  What the rounding of R left out, rho = ref * unit
// - R, is the reference's own exponent, known exactly, and taken into account whenever the reference changes.  Values below `low` count as `low`, whose power is 0 as
// theirs, so that a masked entry adds 0 * (a finite number) to S2.  Both need R below 2^16 (rho below 2^-8); rows beyond that, or whose reference is no
// number, take (x - ref) * unit (`plain`).
struct Running {
    float ref, r, base;                      // base: 0, or (`plain`) the reference, and r = 0
    uint32_t low;                            // fp32, or two bf16
    bool own;                                // this thread has met the reference: that term is not in the sums
    uint64_t s1, s2;
};
constexpr float FUSED_LIMIT = 65536.0f, UNIT_LIMIT = 1.0e-30f;
// The value below which 2^(x unit - R) is 0 whatever the rounding to T: 256 below R, and a 64th of the reference for that rounding.
template <typename T>
__device__ __forceinline__ uint32_t low_of(float reference, float unit)
{
    const float low = reference - 256.0f * reciprocal_fast(unit) - fabsf(reference) * (1.0f / 64.0f);
    return sizeof(T) == 2 ? pack_bf16x2(low, low) : __float_as_uint(low);
}
template <typename T>
__device__ __forceinline__ uint4 not_below(const uint4 &w, uint32_t low)
{
    if constexpr (sizeof(T) == 2) {
        return make_uint4(max_bf16x2(w.x, low), max_bf16x2(w.y, low), max_bf16x2(w.z, low), max_bf16x2(w.w, low));
    } else {
        const float l = __uint_as_float(low);
        return make_uint4(__float_as_uint(max_nan(__uint_as_float(w.x), l)), __float_as_uint(max_nan(__uint_as_float(w.y), l)),
                          __float_as_uint(max_nan(__uint_as_float(w.z), l)), __float_as_uint(max_nan(__uint_as_float(w.w), l)));
    }
}
// The exponent of the value m under the present reference.
__device__ __forceinline__ float exponent_of(const Running &a, float m, float unit) { return fmaf(m - a.base, unit, -a.r); }
template <typename T>
__device__ __forceinline__ void refer_to(Running &a, float ref, float unit)
{
    a.ref = ref;
    const float m = ref == minus_inf() ? 0.0f : ref, r = m * unit;
    const bool fused = fabsf(r) <= FUSED_LIMIT;
    a.r = fused ? r : 0.0f;
    a.base = fused ? 0.0f : m;
    a.low = low_of<T>(m, unit);
}
// A term y with the exponent d, or 0, is added to the sums of the even or of the odd values.
__device__ __forceinline__ void add_one(Running &a, bool even, float y, float d)
{
    const uint64_t both = even ? pack2(y, 0.0f) : pack2(0.0f, y);
    a.s1 = add2(a.s1, both);
    a.s2 = fma2(both, pack2(d, d), a.s2);
}
// All lanes: the warp's largest is the reference now (NaN above all).
template <typename T>
__device__ __forceinline__ void raise(Running &a, float most, float unit)
{
    const Running old = a;
    refer_to<T>(a, warp_max_nan(max_nan(a.ref, most)), unit);
    // (the new reference's exponent under itself less the one that it has under the old one)
    const float d = old.ref == minus_inf() ? minus_inf() : exponent_of(a, a.ref, unit) - exponent_of(old, a.ref, unit), c = exp2_fast(d), d_ = c == 0.0f ? 0.0f : d;
    a.s2 = mul2(pack2(c, c), fma2(pack2(d_, d_), a.s1, a.s2));
    a.s1 = mul2(pack2(c, c), a.s1);
    const float before = fmaxf(exponent_of(a, old.ref, unit), -1.0e4f);      // (0 * -inf)
    add_one(a, true, old.own ? exp2_fast(before) : 0.0f, before);
}
template <typename T, int U>
__device__ __forceinline__ void add_words(Running &a, const uint4 (&r)[U], float unit)
{
    if (a.base == 0.0f) {
        const uint64_t units = pack2(unit, unit), minus = pack2(-a.r, -a.r);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float x[Word<T>::N];
            values_of<T>(not_below<T>(r[u], a.low), x);
#pragma unroll
            for (int e = 0; e < Word<T>::N; e += 2) {
                const uint64_t d = fma2(pack2(x[e], x[e + 1]), units, minus);
                float d0, d1;
                unpack2(d, d0, d1);
                const uint64_t y = pack2(exp2_fast(d0), exp2_fast(d1));
                a.s1 = add2(a.s1, y);
                a.s2 = fma2(y, d, a.s2);
            }
        }
        return;
    }
    const uint64_t shift = pack2(-a.base, -a.base), factor = pack2(unit, unit);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float x[Word<T>::N];
        values_of<T>(r[u], x);
#pragma unroll
        for (int e = 0; e < Word<T>::N; e += 2) {
            float d0, d1;
            unpack2(mul2(add2(pack2(x[e], x[e + 1]), shift), factor), d0, d1);
            const uint64_t y = pack2(exp2_fast(d0), exp2_fast(d1));
            a.s1 = add2(a.s1, y);
            a.s2 = fma2(y, pack2(fmaxf(d0, -1.0e4f), fmaxf(d1, -1.0e4f)), a.s2);          // (0 * -inf)
        }
    }
}
// (all lanes; the largest of the lane's words)
template <typename T, int U>
__device__ __forceinline__ float take_words(Running &a, const uint4 (&r)[U], float unit)
{
    const float most = largest<T, U>(r);
    const bool higher = __any_sync(~0u, !(most <= a.ref));
    if (higher) raise<T>(a, most, unit);
    add_words<T, U>(a, r, unit);
    if (higher) {                            // (the reference's term lies in the larger sum)
        float e, o;
        unpack2(a.s1, e, o);
        a.own = most == a.ref;
        const float d = exponent_of(a, a.ref, unit);
        add_one(a, e >= o, a.own ? -exp2_fast(d) : 0.0f, d);
    }
    return most;
}
// A thread's sums, relative to the row's (or the part's) largest.
__device__ __forceinline__ Sums sums_of(Running a, float most, float unit)
{
    if (a.ref == minus_inf()) return Sums{most, 0.0f, 0.0f, 0};
    const bool own = a.own && a.ref == most;
    if (a.own && !own) add_one(a, true, exp2_fast(exponent_of(a, a.ref, unit)), exponent_of(a, a.ref, unit));
    float e1, o1, e2, o2;
    unpack2(a.s1, e1, o1);
    unpack2(a.s2, e2, o2);
    const float d = exponent_of(a, most, unit), c = exp2_fast(-d), s1 = e1 + o1;
    return c == 0.0f ? Sums{most, 0.0f, 0.0f, own} : Sums{most, c * s1, c * fmaf(-d, s1, e2 + o2), own};
}

// `blocks` thread blocks (a cluster where there are more than one) take a row; each takes a stretch of its words.
// 32 warps an SM: 64 registers (4096 x 65536: 89 us; with 24 or 40 warps 94 and 106).  32 threads with alternatives spill three words for it.
template <int THREADS> constexpr int ROW_BLOCK = THREADS == 32 ? 128 : THREADS;
template <typename T, int THREADS, bool TOP>
__global__ void __launch_bounds__(ROW_BLOCK<THREADS>, 1024 / ROW_BLOCK<THREADS>)
token_logprobs_row(const TokenRows p, int blocks)
{
    constexpr int TEAMS = THREADS == 32 ? 4 : 1;
    constexpr int N = Word<T>::N, U = BATCH_WORDS<T>;
    __shared__ LogprobsShared<THREADS> shared[TEAMS];
    LogprobsShared<THREADS> &sh = shared[threadIdx.x / THREADS];
    namespace cg = cooperative_groups;
    pdl_launch_dependents();
    const int tid = threadIdx.x % THREADS, lane = tid & 31, warp = tid >> 5, rank = blockIdx.x % blocks;
    for (int g = tid; g < TOP_GROUPS; g += THREADS) sh.group[g] = 0;
    pdl_wait();
    const long long row = TEAMS > 1 ? (long long)blockIdx.x * TEAMS + threadIdx.x / THREADS : blockIdx.x / blocks;
    if (row >= p.rows) return;
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
    if (hi == s.w.words && lo < hi && s.w.full_to < s.w.words && tid >= 16 && tid < 16 + N) {
        const long long at = (long long)s.w.full_to * N - s.w.lead + (tid - 16);
        if (at < p.vocab) s.ends = (int)at;
    }
    const float own = tid == 0 && rank == 0 && t.token >= 0 ? load_one(s.x + t.token) : 0.0f;
    const float unit = p.scale * LOG2E;
    Running a{};
    refer_to<T>(a, minus_inf(), unit);
    const uint4 *words = reinterpret_cast<const uint4 *>(s.x - s.w.lead);
    // (a thread's batches: the same number for all but the last threads; groups of them where there are more than slots)
    const int batches = (max(0, s.to - s.from) + U * THREADS - 1) / (U * THREADS);
    s.per_slot = (batches + TOP_SLOTS - 1) / TOP_SLOTS;
    uint32_t even = 0, odd = 0;              // the largest keys of the even and the odd slots
    float most = minus_inf();                // (without alternatives: of all)
    int slots = 0;
    float slot_most = minus_inf();
    int i = s.from + tid, in_slot = 0;
    const auto note = [&](float batch_most) {
        if (i >= s.to) return;               // (the last lanes of the last batch)
        if constexpr (TOP) {
            slot_most = max_nan(slot_most, batch_most);
            if (++in_slot == s.per_slot || i + U * THREADS >= s.to) {
                const uint32_t key = key_of(slot_most);
                sh.slot[slots][tid] = key;
                if (slots & 1) odd = max(odd, key);
                else even = max(even, key);
                ++slots;
                in_slot = 0;
                slot_most = minus_inf();
            }
        } else {
            most = max_nan(most, batch_most);
        }
    };
    // bf16: the next batch is under way while one is taken (fp32, whose batches are twice the words, does without: 68 us, with it 126, for 2048 x 50001)
    constexpr bool AHEAD = sizeof(T) == 2;
    uint4 r[U];
    const auto fetch = [&](int from) {
        if (from + (U - 1) * THREADS < s.to) {
#pragma unroll
            for (int u = 0; u < U; ++u) r[u] = words[from + u * THREADS];
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) r[u] = from + u * THREADS < s.to ? words[from + u * THREADS] : all_masked<T>();
        }
    };
    if (AHEAD || TOP) fetch(i);              // (fp32: loads behind their use with alternatives, before it without: 8192 x 4000 34.4 us, the other way 36.0; 2048 x 50001 69.2 and 73.1)
    if (warp == 0 && __any_sync(~0u, s.ends >= 0)) {
        Piece<T, true> one;
        one.raw = all_masked<T>();
        if (s.ends >= 0) {
            const T x = s.x[s.ends];
            memcpy(&one.raw, &x, sizeof(T));
        }
        const uint4 word[1] = {one.raw};
        const float value = take_words<T, 1>(a, word, unit);
        if (s.ends >= 0) {
            even = max(even, key_of(value));
            most = max_nan(most, value);
        }
    }
    for (; i - lane < s.to; i += U * THREADS) {      // (all lanes of a warp)
        if constexpr (AHEAD) {
            uint4 now[U];
#pragma unroll
            for (int u = 0; u < U; ++u) now[u] = r[u];
            if (i - lane + U * THREADS < s.to) fetch(i + U * THREADS);
            note(take_words<T, U>(a, now, unit));
        } else {
            if (!TOP) fetch(i);
            note(take_words<T, U>(a, r, unit));
            if (TOP && i - lane + U * THREADS < s.to) fetch(i + U * THREADS);
        }
    }
    // the threads' sums, relative to the largest of all
    team_sync<THREADS>();                    // (the groups are zero)
    if constexpr (TOP) {
        if (even) atomicMax(&sh.group[tid % TOP_GROUPS], even);
        if (odd) atomicMax(&sh.group[(tid + 32) % TOP_GROUPS], odd);
    } else {
        if (s.from + tid < s.to || s.ends >= 0) atomicMax(&sh.group[tid % TOP_GROUPS], key_of(most));
    }
    team_sync<THREADS>();
    const uint32_t top = __reduce_max_sync(~0u, max(sh.group[lane], sh.group[lane + 32]));
    Sums b = sums_of(a, top ? value_of(top) : minus_inf(), unit);
    const int n = __popc(__ballot_sync(~0u, b.n != 0));
#pragma unroll
    for (int d = 16; d > 0; d /= 2) {
        b.s1 += __shfl_xor_sync(~0u, b.s1, d);
        b.s2 += __shfl_xor_sync(~0u, b.s2, d);
    }
    if (lane == 0) {
        sh.s1[warp] = b.s1;
        sh.s2[warp] = b.s2;
        sh.n[warp] = n;
    }
    team_sync<THREADS>();
    if (warp == 0) {
        float s1 = lane < THREADS / 32 ? sh.s1[lane] : 0.0f, s2 = lane < THREADS / 32 ? sh.s2[lane] : 0.0f;
        b.n = __reduce_add_sync(~0u, lane < THREADS / 32 ? sh.n[lane] : 0);
#pragma unroll
        for (int d = 16; d > 0; d /= 2) {
            s1 += __shfl_xor_sync(~0u, s1, d);
            s2 += __shfl_xor_sync(~0u, s2, d);
        }
        b.s1 = s1;
        b.s2 = s2;
        if (lane == 0) sh.part = b;
    }
    if constexpr (TOP) find_top<T, THREADS>(sh, s, slots, p.top);
    if (blocks == 1) {
        if (tid >= max(1, p.top)) return;
        if (TOP) b = sh.part;                // (thread 0 wrote it itself; find_top ends with a barrier)
        const float log_s1 = complete(b);
        if (tid == 0) write_row(p, row, b, log_s1, own);
        if (TOP && tid < p.top) write_top(p, row, tid, sh.best[tid], b, log_s1);
        return;
    }
    auto cluster = cg::this_cluster();
    cluster.sync();
    if (rank == 0) {
        // (every warp for itself, a lane for each block: their sums come together)
        Sums all{minus_inf(), 0.0f, 0.0f, 0};
        if (lane < blocks) all = cluster.map_shared_rank(&sh, lane)->part;
        all = relative_to(all, value_of(__reduce_max_sync(~0u, key_of(all.most))), unit);
#pragma unroll
        for (int d = 4; d > 0; d /= 2) {
            all.s1 += __shfl_xor_sync(~0u, all.s1, d);
            all.s2 += __shfl_xor_sync(~0u, all.s2, d);
            all.n += __shfl_xor_sync(~0u, all.n, d);
        }
        all.s1 = __shfl_sync(~0u, all.s1, 0);
        all.s2 = __shfl_sync(~0u, all.s2, 0);
        all.n = __shfl_sync(~0u, all.n, 0);
        const float log_s1 = complete(all);
        if (tid == 0) write_row(p, row, all, log_s1, own);
        if constexpr (TOP) {
            const int n = blocks * p.top;    // (up to 8 * 32)
            for (int i = tid; i < n; i += THREADS) sh.list[i] = cluster.map_shared_rank(&sh, i / p.top)->best[i % p.top];
            team_sync<THREADS>();
            for (int i = tid; i < n; i += THREADS) {      // (by pairs: a search in the blocks' ordered lists takes 1 us longer)
                const unsigned long long r = sh.list[i];
                int before = 0;
#pragma unroll 8
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

// Eight bf16 or four fp32 gradients from as many logits.  With q = x unit - zl (zl = z log2 e rounded, rho what that left out), out = 2^q (b + g q) with all the
// row's factors in b and g; as in the forward pass, values below `low` count as it, and `plain` rows take the formula as it stands.
struct GradRow {
    float scale, z, gh, base;                // plain
    float unit, zl, b, g;
    uint32_t low;
    bool plain, nothing;
};
template <typename T>
__device__ __forceinline__ void gradients_of(const GradRow &c, const uint4 &w, float (&v)[Word<T>::N])
{
    constexpr int N = Word<T>::N;
    if (c.nothing) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = 0.0f;
        return;
    }
    if (!c.plain) {
        values_of<T>(not_below<T>(w, c.low), v);
        const uint64_t unit = pack2(c.unit, c.unit), minus = pack2(-c.zl, -c.zl), b = pack2(c.b, c.b), g = pack2(c.g, c.g);
#pragma unroll
        for (int e = 0; e < N; e += 2) {
            const uint64_t q = fma2(pack2(v[e], v[e + 1]), unit, minus);
            float q0, q1;
            unpack2(q, q0, q1);
            unpack2(mul2(pack2(exp2_fast(q0), exp2_fast(q1)), fma2(q, g, b)), v[e], v[e + 1]);
        }
        return;
    }
    values_of<T>(w, v);
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float lp = fmaf(v[e], c.scale, -c.z);
        v[e] = -c.scale * exp2_fast(lp * LOG2E) * fmaf(c.gh, fmaxf(lp, -1.0e4f), c.base);
    }
}

// A thread block takes `chunk` words of one row.  TOGETHER: in every row the result lies at the same alignment as the logits.
template <typename T, bool TOGETHER>
__global__ void __launch_bounds__(GRAD_THREADS)
token_logprobs_grad(const TokenGrads p, int parts, int chunk)
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
    const int from = part * chunk, to = min(from + chunk, w.words);
    if (from >= to) return;
    const RowToken t = row_token(p.tokens, row, p.vocab, p.error_flag, tid == 0 && part == 0);
    GradRow c{};
    c.scale = p.scale;
    c.z = p.log_sum[row];
    c.nothing = !t.part || c.z == minus_inf();
    // the row's few entries of their own
    const int n = p.top + 1;
    if (tid < n) {
        int v = -1;
        float g = 0.0f;
        if (tid == 0 && t.token >= 0 && p.d_logp != nullptr) {
            v = t.token;
            g = p.d_logp[row];
        }
        if (tid > 0 && t.part) {
            v = p.top_tokens[row * p.top + tid - 1];
            g = p.d_top[row * p.top + tid - 1];
            if (v >= p.vocab && part == 0) atomicExch(p.error_flag, ERR_LABEL);
            if (v < 0 || v >= p.vocab) v = -1, g = 0.0f;
        }
        at[tid] = v;
        given[tid] = g;
    }
    c.gh = p.d_entropy != nullptr && t.part ? p.d_entropy[row] : 0.0f;
    const float h = c.gh != 0.0f ? p.entropy[row] : 0.0f;
    __syncthreads();
    float every = 0.0f;
    for (int j = 0; j < n; ++j) every += given[j];
    c.base = fmaf(c.gh, h, every);
    c.unit = p.scale * LOG2E;
    c.zl = c.z * LOG2E;
    c.plain = !(fabsf(c.zl) <= FUSED_LIMIT && c.unit >= UNIT_LIMIT && c.unit <= 1.0f / UNIT_LIMIT);
    c.low = low_of<T>(c.z / p.scale, c.unit);
    const float rho = fmaf(c.z, LOG2E, -c.zl), k = -p.scale * exp2_fast(-rho);
    c.g = k * c.gh * LN2;
    c.b = fmaf(k, c.base, -rho * c.g);
    // (the entries' own: the first of equal ones takes them all; its logit is read before anything is written)
    const long long c0 = (long long)from * N - w.lead, c1 = (long long)to * N - w.lead;
    bool special = false;
    float special_x = 0.0f, special_g = 0.0f;
    if (tid < n && at[tid] >= 0 && at[tid] >= c0 && at[tid] < c1 && !c.nothing) {
        special = true;
        for (int j = 0; j < n; ++j) {
            if (at[j] != at[tid]) continue;
            special = special && j >= tid;
            special_g += given[j];
        }
        special_x = load_one(x + at[tid]);
    }
    __syncthreads();
    const uint4 *words = reinterpret_cast<const uint4 *>(x - w.lead);
    uint4 *out_words = reinterpret_cast<uint4 *>(out - w.lead);
    for (int i0 = from; i0 < to; i0 += GRAD_THREADS * GRAD_WORDS) {
        if (TOGETHER && i0 >= w.full_from && i0 + GRAD_THREADS * GRAD_WORDS <= min(to, w.full_to)) {
            uint4 r[GRAD_WORDS];
#pragma unroll
            for (int u = 0; u < GRAD_WORDS; ++u) r[u] = words[i0 + tid + u * GRAD_THREADS];
#pragma unroll
            for (int u = 0; u < GRAD_WORDS; ++u) {
                float v[N];
                gradients_of<T>(c, r[u], v);
                store_values<T, N>(reinterpret_cast<T *>(out_words + i0 + tid + u * GRAD_THREADS), v);
            }
            continue;
        }
#pragma unroll 1
        for (int i = i0 + tid; i < min(i0 + GRAD_THREADS * GRAD_WORDS, to); i += GRAD_THREADS) {
            const bool full = i >= w.full_from && i < w.full_to;
            float v[N];
            uint4 r = make_uint4(0, 0, 0, 0);
            if (full) {
                r = words[i];
            } else {
                T one[N];
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const long long j = (long long)i * N + e - w.lead;
                    one[e] = j >= 0 && j < p.vocab ? x[j] : T(0.0f);
                }
                memcpy(&r, one, sizeof(r));
            }
            gradients_of<T>(c, r, v);
            if (TOGETHER && full) {
                store_values<T, N>(reinterpret_cast<T *>(out_words + i), v);
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const long long j = (long long)i * N + e - w.lead;
                    const float one[1] = {v[e]};
                    if (j >= 0 && j < p.vocab) store_values<T, 1>(out + j, one);
                }
            }
        }
    }
    __syncthreads();
    if (special) {
        // c (1 - p) - p (the others' + g_H (log p + H)): as exact near p = 1 as 1 - p itself
        const float lp = fmaf(special_x, p.scale, -c.z), prob = exp2_fast(lp * LOG2E);
        const float g[1] = {p.scale * (special_g * -expm1f(lp) - prob * fmaf(c.gh, fmaxf(lp, -1.0e4f), c.base - special_g))};
        store_values<T, 1>(out + at[tid], g);
    }
}

}  // namespace lm
}  // namespace cocod
