// AdamW over many tensors at once, moments in 32 or 8 bits.
//
// A thread block takes a chunk of a tensor's values, a thread eight at a time.  HBM bounds the 32-bit form: 28 bytes a value with fp32 parameters and
// gradients (187 M values in 770 us, 6.8 TB/s).  The 8-bit form moves 16.1 bytes; its codes are quadratic, value = c |c| unit, so that coding is a root and a
// rounding, decoding a product.  It takes 63 issue slots a value, as many as about 11 bytes leave, and is bound by them and by the chain of a block's
// maximum, division and codes (150 M values in 432 us, 5.6 TB/s; with bf16 parameters and gradients 397 us, 3.8 TB/s).
//
// The last thread block to finish (a ticket) counts the step and prepares the next one's factors, in fp64; nothing waits for another block.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "cocod_experts.cuh"

namespace cocod {
namespace adamw {

using lm::as_float;
using lm::store_values;
using gemm::pdl_launch_dependents;
using gemm::pdl_wait;

constexpr int BLOCK = 128, THREADS = 256;
constexpr int APART = THREADS * 4;         // values that a thread block takes four a thread
constexpr float EMPTY = 7.888609052210118e-31f;      // 2^-100: a block below it counts as zero

struct Tensor {
    long long size, start, state;          // start: in the flat buffers; state: first value in the moments
    int first_chunk;
    float decay;
};
struct Clock {
    double power1, power2;                 // beta^t of the steps done
    float lr, correct1, correct2;          // of the next step: 1 / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
    unsigned ticket;
    long long steps;
};
struct State {
    void *m, *v;
    float *m_units, *v_units;              // 8 bits
};
struct Step {
    const Tensor *tensors;
    const int *chunk_tensor;               // the tensor of each chunk
    Clock *clock;
    State state;
    const float *grad_scale;
    double beta1, beta2;
    float b1, rest1, b2, rest2, eps;
    int first_chunk, first_tensor;         // of this launch, a thread block for each of its chunks
    int quads;                             // a chunk is quads * APART values (8 bits: an even number)
    int advance;                           // the step's last launch
};
// Where the tensors lie: in flat buffers ...
struct Flat {
    const void *in;
    void *out;
    const void *grad;
    void *copy;
};
// ... or one by one (indexed from the launch's first tensor).
template <int CAPACITY> struct Lists {
    void *param[CAPACITY];
    const void *grad[CAPACITY];
    void *copy[CAPACITY];
};
template <typename P, typename G> struct Place {
    const P *in;
    P *out;
    const G *grad;
    __nv_bfloat16 *copy;
};
template <typename P, typename G>
__device__ __forceinline__ Place<P, G> place_of(const Flat &f, int, const Tensor &t)
{
    return Place<P, G>{static_cast<const P *>(f.in) + t.start, static_cast<P *>(f.out) + t.start, static_cast<const G *>(f.grad) + t.start,
                       f.copy ? static_cast<__nv_bfloat16 *>(f.copy) + t.start : nullptr};
}
template <typename P, typename G, int C>
__device__ __forceinline__ Place<P, G> place_of(const Lists<C> &l, int i, const Tensor &)
{
    return Place<P, G>{static_cast<const P *>(l.param[i]), static_cast<P *>(l.param[i]), static_cast<const G *>(l.grad[i]), static_cast<__nv_bfloat16 *>(l.copy[i])};
}

__device__ __forceinline__ void load4(const float *p, float (&x)[4])
{
    const float4 v = *reinterpret_cast<const float4 *>(p);
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
}
__device__ __forceinline__ void load4(const __nv_bfloat16 *p, float (&x)[4])
{
    const uint2 v = *reinterpret_cast<const uint2 *>(p);
    x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xffff0000u);
    x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xffff0000u);
}
template <typename T>
__device__ __forceinline__ bool whole_words(const T *p) { return (reinterpret_cast<uintptr_t>(p) & (4 * sizeof(T) - 1)) == 0; }

// Two products or sums of fp32 in one instruction.  The assembler joins a product and a sum of pairs to one that is rounded once, .rn or not; where
// both roundings are wanted, the sum is one of single values (add_apart).
struct Pair {
    uint64_t bits;
};
__device__ __forceinline__ Pair pair(float a, float b)
{
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.bits) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void split(Pair p, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p.bits)); }
__device__ __forceinline__ Pair mul(Pair a, Pair b)
{
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits));
    return r;
}
__device__ __forceinline__ Pair add(Pair a, Pair b)
{
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits));
    return r;
}
__device__ __forceinline__ Pair add_apart(Pair a, Pair b)
{
    float a0, a1, b0, b1;
    split(a, a0, a1);
    split(b, b0, b1);
    return pair(__fadd_rn(a0, b0), __fadd_rn(a1, b1));
}
__device__ __forceinline__ Pair fma(Pair a, Pair b, Pair c)
{
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits), "l"(c.bits));
    return r;
}
__device__ __forceinline__ float root_fast(float x)
{
    float y;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float reciprocal_fast(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// ------------------------------------------------------------------------------------------ 8 bits
// Bytes to fp32 and back by the bits of 2^23 (and 1.5 * 2^23, where the rounding is that of the addition: to nearest, half to even).
constexpr float WHOLE = 12582912.0f;
__device__ __forceinline__ void bytes_to_float(uint32_t w, float offset, Pair (&x)[2])
{
    const Pair o = pair(-offset, -offset);
#pragma unroll
    for (int i = 0; i < 2; ++i)
        x[i] = add(pair(__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7440 | 2 * i)), __uint_as_float(__byte_perm(w, 0x4b000000u, 0x7440 | (2 * i + 1)))), o);
}
__device__ __forceinline__ void decode_m(uint32_t w, float unit, Pair (&m)[2])
{
    bytes_to_float(w ^ 0x80808080u, 8388736.0f, m);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float a, b;
        split(m[i], a, b);
        m[i] = mul(mul(m[i], pair(fabsf(a), fabsf(b))), pair(unit, unit));
    }
}
__device__ __forceinline__ void decode_v(uint32_t w, float unit, Pair (&v)[2])
{
    bytes_to_float(w, 8388608.0f, v);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const Pair r = mul(mul(v[i], v[i]), pair(unit, unit));
        v[i] = mul(r, r);
    }
}
// Half a warp holds a block: lane l of it values 4 l .. + 3 and 64 + 4 l .. + 3, so that its accesses lie side by side.  (NaN is above all.)
// x: not negative.
__device__ __forceinline__ float block_max(const float (&x)[8], unsigned half)
{
    uint32_t m = __float_as_uint(x[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) m = max(m, __float_as_uint(x[i]));
    return __uint_as_float(__reduce_max_sync(half, m));
}
// The units of a block's m and r = sqrt v, and what its values are multiplied by for the codes' squares.  The root is monotonic when it is
// correctly rounded, so that max r is the root of max v.  One half of the lanes divides for m, the other for r.  A block with a value that is not finite has
// the unit NaN.
struct Units {
    float m, r, per_m, per_r;
};
__device__ __forceinline__ Units units_of(float most_m, float most_v, int lane, unsigned half)
{
    const float most_r = __fsqrt_rn(most_v);
    const bool first = (lane & 8) == 0;
    const float most = first ? most_m : most_r, squared = first ? 16129.0f : 65025.0f, part = first ? 1.0f / 16129.0f : 1.0f / 65025.0f;
    const bool zero = most < EMPTY;
    const float per = zero ? 0.0f : __fdiv_rn(squared, most);
    const float unit = zero ? 0.0f : most <= 3.402823466e38f ? __fmul_rn(most, part) : __int_as_float(0x7fffffff);
    const int at = lane & 16;
    return Units{__shfl_sync(half, unit, at), __shfl_sync(half, unit, at + 8), __shfl_sync(half, per, at), __shfl_sync(half, per, at + 8)};
}
// How far roots are from the nearest whole numbers, at most.
__device__ __forceinline__ float off_whole(const float (&c)[4])
{
    const Pair whole = pair(WHOLE, WHOLE), minus = pair(-WHOLE, -WHOLE), negative = pair(-1.0f, -1.0f);
    float off[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const Pair root = pair(c[2 * i], c[2 * i + 1]);
        split(fma(add(add(root, whole), minus), negative, root), off[2 * i], off[2 * i + 1]);
    }
    return fmaxf(fmaxf(fabsf(off[0]), fabsf(off[1])), fmaxf(fabsf(off[2]), fabsf(off[3])));
}
__device__ __forceinline__ uint32_t float_to_bytes(const float (&c)[4])
{
    const Pair whole = pair(WHOLE, WHOLE);
    float bits[4];
    split(add(pair(c[0], c[1]), whole), bits[0], bits[1]);
    split(add(pair(c[2], c[3]), whole), bits[2], bits[3]);
    return __byte_perm(__byte_perm(__float_as_uint(bits[0]), __float_as_uint(bits[1]), 0x0040), __byte_perm(__float_as_uint(bits[2]), __float_as_uint(bits[3]), 0x0040),
                       0x5410);
}
// Codes are the whole numbers nearest to correctly rounded roots of correctly rounded products.  Here roots come from the fast instruction, off by
// 2^-23 of themselves at most.  With 2^-23 from r, half of that and of a rounding's 2^-24 remaining under the root, another 2^-23 and the
// exact chain's own roundings (2^-24 each, halved under the root), a code's root (at most 255) differs by less than 255 * 3 * 2^-23 < 2^-13.  That matters only
// next to the middle of two whole numbers; there, once in thousands of values, all is computed again with exact roots.
constexpr float NEAR = 0.5f - 1.0f / 8192.0f;
__device__ __forceinline__ uint32_t encode_m(const float *m, const float *size, float per)
{
    const Pair f = pair(per, per);
    float q[4], c[4];
    split(mul(pair(size[0], size[1]), f), q[0], q[1]);
    split(mul(pair(size[2], size[3]), f), q[2], q[3]);
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = root_fast(q[i]);
    if (off_whole(c) > NEAR)
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = __fsqrt_rn(q[i]);
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = copysignf(c[i], m[i]);
    return float_to_bytes(c);
}
// (r: fast roots of v; the code is at least 1 where v > 0)
__device__ __forceinline__ uint32_t encode_v(const float *v, const float *r, float per)
{
    const Pair f = pair(per, per);
    float q[4], c[4];
    split(mul(pair(r[0], r[1]), f), q[0], q[1]);
    split(mul(pair(r[2], r[3]), f), q[2], q[3]);
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = root_fast(q[i]);
    if (off_whole(c) > NEAR || fminf(fminf(q[0], q[1]), fminf(q[2], q[3])) < 0.3f)
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = fmaxf(__fsqrt_rn(__fmul_rn(__fsqrt_rn(v[i]), per)), v[i] > 0.0f ? 1.0f : 0.0f);
    return float_to_bytes(c);
}

// ------------------------------------------------------------------------------------------ the step
struct Rates {
    float b1, rest1, b2, rest2, keep, rate, correct2, eps, scale;
};
// Where a thread's values of a chunk lie: two quads (32 bits: 1024 values apart; 8 bits: of its block, 64 apart).
template <typename P, typename G> struct Values {
    const P *in;
    P *out;
    const G *grad;
    __nv_bfloat16 *copy;
    void *m, *v;                           // fp32, or words of four codes
    float *m_unit, *v_unit;
    int left;                              // of the chunk, from the thread's first value on
};
template <typename T>
__device__ __forceinline__ void load_quad(const T *p, float (&x)[4], bool full, int left)
{
    if (full) {
        load4(p, x);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = e < left ? as_float(p[e]) : 0.0f;
    }
}
template <typename T>
__device__ __forceinline__ void store_quad(T *p, const float *x, bool full, int left)
{
    if (full) {
        store_values<T, 4>(p, *reinterpret_cast<const float (*)[4]>(x));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) store_values<T, 1>(p + e, *reinterpret_cast<const float (*)[1]>(x + e));
    }
}
// What a thread reads: two quads, their loads under way together.  words: they lie at multiples of their size; FULL: that, and they are all there.
struct Loaded {
    float p[2][4], g[2][4];
    float4 m32[2], v32[2];
    uint32_t m8[2], v8[2];
    float um, ur;
};
template <typename P, typename G, int BITS, bool FULL>
__device__ __forceinline__ void load(const Values<P, G> &at, bool words, Loaded &x)
{
    constexpr int NEXT = BITS == 8 ? BLOCK / 2 : APART;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        load_quad(at.in + u * NEXT, x.p[u], FULL || (words && at.left - u * NEXT >= 4), at.left - u * NEXT);
        load_quad(at.grad + u * NEXT, x.g[u], FULL || (words && at.left - u * NEXT >= 4), at.left - u * NEXT);
        if constexpr (BITS == 8) {
            x.m8[u] = static_cast<const uint32_t *>(at.m)[u * NEXT / 4];
            x.v8[u] = static_cast<const uint32_t *>(at.v)[u * NEXT / 4];
        } else if (FULL || at.left > u * NEXT) {
            x.m32[u] = static_cast<const float4 *>(at.m)[u * NEXT / 4];
            x.v32[u] = static_cast<const float4 *>(at.v)[u * NEXT / 4];
        }
    }
    if constexpr (BITS == 8) {
        x.um = *at.m_unit;
        x.ur = *at.v_unit;
    }
}
// The same on its way through shared memory (8 bits, FULL), a step ahead of its use; every thread reads what it has copied itself.
template <typename P, typename G> struct Stage {
    P p[2][THREADS][4];
    G g[2][THREADS][4];
    uint32_t m[2][THREADS], v[2][THREADS];
    float um[THREADS], ur[THREADS];
};
template <int BYTES>
__device__ __forceinline__ void copy_ahead(void *to, const void *from)
{
    const uint32_t at = (uint32_t)__cvta_generic_to_shared(to);
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(from), "n"(BYTES) : "memory");
}
template <typename P, typename G>
__device__ __forceinline__ void begin_load(const Values<P, G> &at, int offset, Stage<P, G> &to)
{
    const int t = threadIdx.x;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int k = offset + u * (BLOCK / 2);
        copy_ahead<4 * sizeof(P)>(to.p[u][t], at.in + k);
        copy_ahead<4 * sizeof(G)>(to.g[u][t], at.grad + k);
        copy_ahead<4>(&to.m[u][t], static_cast<const char *>(at.m) + k);
        copy_ahead<4>(&to.v[u][t], static_cast<const char *>(at.v) + k);
    }
    copy_ahead<4>(&to.um[t], at.m_unit + offset / BLOCK);
    copy_ahead<4>(&to.ur[t], at.v_unit + offset / BLOCK);
    asm volatile("cp.async.commit_group;" ::: "memory");
}
template <typename P, typename G>
__device__ __forceinline__ void end_load(const Stage<P, G> &from, bool last, Loaded &x)
{
    if (last) asm volatile("cp.async.wait_group 0;" ::: "memory");
    else asm volatile("cp.async.wait_group 1;" ::: "memory");
    const int t = threadIdx.x;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        load4(from.p[u][t], x.p[u]);
        load4(from.g[u][t], x.g[u]);
        x.m8[u] = from.m[u][t];
        x.v8[u] = from.v[u][t];
    }
    x.um = from.um[t];
    x.ur = from.ur[t];
}
template <typename P, typename G, int BITS, bool FULL>
__device__ __forceinline__ void update(const Values<P, G> &at, const Rates &s, int lane, bool words, Loaded &x)
{
    constexpr int NEXT = BITS == 8 ? BLOCK / 2 : APART;
    const unsigned half = lane < 16 ? 0x0000ffffu : 0xffff0000u;
    float m[8], v[8], r[8];
    float (&p)[2][4] = x.p, (&g)[2][4] = x.g;
    const float4 *m32 = x.m32, *v32 = x.v32;
    const uint32_t *m8 = x.m8, *v8 = x.v8;
    const float um = x.um, ur = x.ur;
    const Pair keeps = pair(s.keep, s.keep), rates = pair(-s.rate, -s.rate), corrections = pair(s.correct2, s.correct2), epsilons = pair(s.eps, s.eps),
               b1 = pair(s.b1, s.b1), rest1 = pair(s.rest1, s.rest1), b2 = pair(s.b2, s.b2), rest2 = pair(s.rest2, s.rest2), scales = pair(s.scale, s.scale);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        if (BITS == 32 && !FULL && at.left <= u * NEXT) break;
        Pair pm[2], pv[2];
        if constexpr (BITS == 8) {
            decode_m(m8[u], um, pm);
            decode_v(v8[u], ur, pv);
        } else {
            pm[0] = pair(m32[u].x, m32[u].y); pm[1] = pair(m32[u].z, m32[u].w);
            pv[0] = pair(v32[u].x, v32[u].y); pv[1] = pair(v32[u].z, v32[u].w);
        }
        float *mu = m + 4 * u, *vu = v + 4 * u, *ru = r + 4 * u;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            Pair d = pair(g[u][2 * i], g[u][2 * i + 1]);
            d = mul(d, scales);
            pm[i] = add_apart(mul(pm[i], b1), mul(d, rest1));
            pv[i] = add_apart(mul(pv[i], b2), mul(mul(d, d), rest2));
            split(pm[i], mu[2 * i], mu[2 * i + 1]);
            split(pv[i], vu[2 * i], vu[2 * i + 1]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) ru[e] = root_fast(vu[e]);
        // (the fast root takes numbers below 2^-126 for 0)
        if (fminf(fminf(vu[0], vu[1]), fminf(vu[2], vu[3])) < 1.2e-38f)
#pragma unroll
            for (int e = 0; e < 4; ++e) ru[e] = vu[e] < 1.2e-38f ? __fsqrt_rn(vu[e]) : ru[e];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float d0, d1;
            split(fma(pair(ru[2 * i], ru[2 * i + 1]), corrections, epsilons), d0, d1);
            const Pair step = mul(pm[i], pair(reciprocal_fast(d0), reciprocal_fast(d1)));
            split(fma(rates, step, mul(pair(p[u][2 * i], p[u][2 * i + 1]), keeps)), p[u][2 * i], p[u][2 * i + 1]);
        }
        store_quad(at.out + u * NEXT, p[u], FULL || (words && at.left - u * NEXT >= 4), at.left - u * NEXT);
        if (at.copy) store_quad(at.copy + u * NEXT, p[u], FULL || (words && at.left - u * NEXT >= 4), at.left - u * NEXT);
        if constexpr (BITS == 32) {
            store_quad(static_cast<float *>(at.m) + u * NEXT, mu, true, 0);
            store_quad(static_cast<float *>(at.v) + u * NEXT, vu, true, 0);
        }
    }
    if constexpr (BITS == 8) {
        float size[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) size[i] = fabsf(m[i]);
        const Units units = units_of(block_max(size, half), block_max(v, half), lane, half);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            static_cast<uint32_t *>(at.m)[u * NEXT / 4] = encode_m(m + 4 * u, size + 4 * u, units.per_m);
            static_cast<uint32_t *>(at.v)[u * NEXT / 4] = encode_v(v + 4 * u, r + 4 * u, units.per_r);
        }
        if ((lane & 15) == 0) {
            *at.m_unit = units.m;
            *at.v_unit = units.r;
        }
    }
}

// (32 bits: four blocks an SM, for which fp32 parameters spill up to seven words: 187 M values 775 us, three blocks without 787)
template <typename P, typename G, int BITS, typename W>
__global__ void __launch_bounds__(THREADS, BITS == 8 ? 3 : 4)
adamw_step(const Step s, const W where)
{
    __shared__ __align__(16) Stage<P, G> stage[BITS == 8 ? 2 : 1];
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    Rates rates{s.b1, s.rest1, s.b2, s.rest2, 1.0f, 0.0f, s.clock->correct2, s.eps, s.grad_scale ? *s.grad_scale : 1.0f};      // (a factor of one changes nothing)
    const float lr = s.clock->lr;
    rates.rate = lr * s.clock->correct1;
    const int chunk = s.first_chunk + blockIdx.x, i = s.chunk_tensor[chunk];
    const Tensor t = s.tensors[i];
    const Place<P, G> at = place_of<P, G>(where, i - s.first_tensor, t);
    if (at.grad != nullptr) {
        const long long from = (long long)(chunk - t.first_chunk) * s.quads * APART;
        const bool words = whole_words(at.in) && whole_words(at.out) && whole_words(at.grad) && whole_words(at.copy);
        rates.keep = fmaf(-lr, t.decay, 1.0f);
        constexpr int VALUE = BITS == 8 ? 1 : 4;
        const int mine = BITS == 8 ? (threadIdx.x >> 4) * BLOCK + 4 * (threadIdx.x & 15) : 4 * threadIdx.x;
        const long long k = from + mine, q = t.state + k;
        const int left = (int)min(t.size - from, (long long)s.quads * APART);
        Values<P, G> x{at.in + k, at.out + k, at.grad + k, at.copy ? at.copy + k : nullptr, static_cast<char *>(s.state.m) + q * VALUE,
                       static_cast<char *>(s.state.v) + q * VALUE, BITS == 8 ? s.state.m_units + q / BLOCK : nullptr,
                       BITS == 8 ? s.state.v_units + q / BLOCK : nullptr, left - mine};
        const auto next = [&] {
            x.in += 2 * APART; x.out += 2 * APART; x.grad += 2 * APART; x.left -= 2 * APART;
            if (x.copy) x.copy += 2 * APART;
            x.m = static_cast<char *>(x.m) + 2 * APART * VALUE;
            x.v = static_cast<char *>(x.v) + 2 * APART * VALUE;
            if constexpr (BITS == 8) x.m_unit += 2 * APART / BLOCK, x.v_unit += 2 * APART / BLOCK;
        };
        int u = 0;
        Loaded y;
        if constexpr (BITS == 8) {
            if (words && left >= 2 * APART) {
                begin_load(x, 0, stage[0]);
#pragma unroll 1
                for (; left - u >= 2 * APART; u += 2 * APART) {
                    const bool last = left - u < 4 * APART;
                    const int now = u / (2 * APART) & 1;
                    if (!last) begin_load(x, 2 * APART, stage[now ^ 1]);
                    end_load(stage[now], last, y);
                    update<P, G, BITS, true>(x, rates, lane, words, y);
                    next();
                }
            }
        }
#pragma unroll 1
        for (; u < left; u += 2 * APART) {
            if (BITS == 32 && words && left - u >= 2 * APART) {
                load<P, G, BITS, true>(x, words, y);
                update<P, G, BITS, true>(x, rates, lane, words, y);
            } else if (BITS == 32 || x.left > -4 * (int)(threadIdx.x & 15)) {      // (8 bits: where the half warp has a block)
                load<P, G, BITS, false>(x, words, y);
                update<P, G, BITS, false>(x, rates, lane, words, y);
            }
            next();
        }
    }
    if (!s.advance) return;
    __syncthreads();                       // (all threads have read the clock)
    if (threadIdx.x == 0) {
        __threadfence();
        if (atomicAdd(&s.clock->ticket, 1u) == gridDim.x - 1) {
            Clock *k = s.clock;
            k->power1 *= s.beta1;
            k->power2 *= s.beta2;
            k->correct1 = (float)(1.0 / (1.0 - k->power1 * s.beta1));
            k->correct2 = (float)(1.0 / sqrt(1.0 - k->power2 * s.beta2));
            k->steps += 1;
            k->ticket = 0;
        }
    }
}

static __global__ void adamw_set(Clock *k, int what, float lr, long long steps, double beta1, double beta2)
{
    pdl_wait();
    if (what == 0) {
        k->lr = lr;
        return;
    }
    k->power1 = pow(beta1, (double)steps);
    k->power2 = pow(beta2, (double)steps);
    k->correct1 = (float)(1.0 / (1.0 - k->power1 * beta1));
    k->correct2 = (float)(1.0 / sqrt(1.0 - k->power2 * beta2));
    k->steps = steps;
    k->ticket = 0;
}

// The moments in fp32 from the 8-bit state (READ), or the state from them; half a warp for a block.
template <bool READ>
static __global__ void __launch_bounds__(THREADS)
adamw_moments(const State s, long long blocks, float *m_out, float *v_out, const float *m_in, const float *v_in)
{
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const unsigned half = lane < 16 ? 0x0000ffffu : 0xffff0000u;
    for (long long b = (long long)blockIdx.x * (THREADS / 16) + (threadIdx.x >> 4); b < blocks; b += (long long)gridDim.x * (THREADS / 16)) {
        const long long q = b * BLOCK + 4 * (lane & 15);
        uint32_t *mw = static_cast<uint32_t *>(s.m) + q / 4, *vw = static_cast<uint32_t *>(s.v) + q / 4;
        if constexpr (READ) {
            const float um = s.m_units[b], ur = s.v_units[b];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                Pair pm[2], pv[2];
                decode_m(mw[16 * u], um, pm);
                decode_v(vw[16 * u], ur, pv);
                float m[4], v[4];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    split(pm[i], m[2 * i], m[2 * i + 1]);
                    split(pv[i], v[2 * i], v[2 * i + 1]);
                }
                store_values<float, 4>(m_out + q + 64 * u, m);
                store_values<float, 4>(v_out + q + 64 * u, v);
            }
        } else {
            float m[8], v[8], r[8], size[8];
            load4(m_in + q, *reinterpret_cast<float (*)[4]>(m));
            load4(m_in + q + 64, *reinterpret_cast<float (*)[4]>(m + 4));
            load4(v_in + q, *reinterpret_cast<float (*)[4]>(v));
            load4(v_in + q + 64, *reinterpret_cast<float (*)[4]>(v + 4));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                size[e] = fabsf(m[e]);
                v[e] += 0.0f;                // (-0 has the bits of a large number)
                r[e] = root_fast(v[e]);
            }
            const Units units = units_of(block_max(size, half), block_max(v, half), lane, half);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                mw[16 * u] = encode_m(m + 4 * u, size + 4 * u, units.per_m);
                vw[16 * u] = encode_v(v + 4 * u, r + 4 * u, units.per_r);
            }
            if ((lane & 15) == 0) {
                s.m_units[b] = units.m;
                s.v_units[b] = units.r;
            }
        }
    }
}

}  // namespace adamw
}  // namespace cocod
