// AdamW over many tensors at once, moments in 32 or 8 bits.
//
// A thread block takes chunks of 2048 values of a tensor, a warp 128 at a time (the block that shares a unit in the 8-bit state), four side by
// side for each lane.  HBM bounds the 32-bit form (28 bytes a value with fp32 parameters and gradients).  The 8-bit form moves 16.1 bytes and needs two
// more roots a value; its codes are quadratic, value = c |c| unit, so that coding is a root and a rounding, decoding a product.
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

constexpr int BLOCK = 128, CHUNK = 2048, THREADS = 256;
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
    int first_chunk, chunks, first_tensor; // of this launch
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

// ------------------------------------------------------------------------------------------ 8 bits
// Bytes to fp32 and back by the bits of 2^23 (and 1.5 * 2^23, where the rounding is that of the addition: to nearest, half to even).
__device__ __forceinline__ void bytes_to_float(uint32_t w, float offset, float (&x)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(__byte_perm(w, 0x4b000000u, 0x7440 | i)) - offset;
}
__device__ __forceinline__ uint32_t float_to_bytes(const float (&x)[4])
{
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = __float_as_uint(__fadd_rn(x[i], 12582912.0f));
    return __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
}
__device__ __forceinline__ void decode_m(uint32_t w, float unit, float (&m)[4])
{
    bytes_to_float(w ^ 0x80808080u, 8388736.0f, m);
#pragma unroll
    for (int i = 0; i < 4; ++i) m[i] = __fmul_rn(__fmul_rn(m[i], fabsf(m[i])), unit);
}
__device__ __forceinline__ void decode_root(uint32_t w, float unit, float (&r)[4])
{
    bytes_to_float(w, 8388608.0f, r);
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __fmul_rn(__fmul_rn(r[i], r[i]), unit);
}
// (the whole warp; NaN is above all)
__device__ __forceinline__ float block_max(const float (&x)[4])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
    return __uint_as_float(__reduce_max_sync(~0u, m));
}
// The unit of a block and its reciprocal.  A block with a value that is not finite has none: it reads as NaN.
__device__ __forceinline__ float unit_of(float most, float squared, float &per)
{
    const bool zero = most < EMPTY;
    per = zero ? 0.0f : __fdiv_rn(squared, most);
    return zero ? 0.0f : most <= 3.402823466e38f ? __fmul_rn(most, 1.0f / squared) : __int_as_float(0x7fffffff);
}
__device__ __forceinline__ uint32_t encode_m(const float (&m)[4], float &unit)
{
    float per;
    unit = unit_of(block_max(m), 16129.0f, per);
    float c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = copysignf(__fsqrt_rn(__fmul_rn(fabsf(m[i]), per)), m[i]);
    return float_to_bytes(c);
}
__device__ __forceinline__ uint32_t encode_root(const float (&r)[4], float &unit)
{
    float per;
    unit = unit_of(block_max(r), 65025.0f, per);
    float d[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) d[i] = fmaxf(__fsqrt_rn(__fmul_rn(r[i], per)), r[i] > 0.0f ? 1.0f : 0.0f);
    return float_to_bytes(d);
}

// ------------------------------------------------------------------------------------------ the step
template <typename P, typename G, int BITS, typename W>
__global__ void __launch_bounds__(THREADS)
adamw_step(const Step s, const W where)
{
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const float lr = s.clock->lr, rate = lr * s.clock->correct1, correct2 = s.clock->correct2, scale = s.grad_scale ? *s.grad_scale : 1.0f;
    for (int c = blockIdx.x; c < s.chunks; c += gridDim.x) {
        const int chunk = s.first_chunk + c, i = s.chunk_tensor[chunk];
        const Tensor t = s.tensors[i];
        const Place<P, G> at = place_of<P, G>(where, i - s.first_tensor, t);
        if (at.grad == nullptr) continue;
        const long long from = (long long)(chunk - t.first_chunk) * CHUNK;
        const bool words = whole_words(at.in) && whole_words(at.out) && whole_words(at.grad) && whole_words(at.copy);
        const float keep = fmaf(-lr, t.decay, 1.0f);
#pragma unroll
        for (int u = 0; u < CHUNK / THREADS / 4; ++u) {
            const long long first = from + (u * (THREADS / 32) + warp) * BLOCK, k = first + 4 * lane;
            if (first >= t.size) break;
            const bool full = words && first + BLOCK <= t.size;
            float p[4], g[4], m[4], v[4];
            if (full) {
                load4(at.in + k, p);
                load4(at.grad + k, g);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[e] = k + e < t.size ? as_float(at.in[k + e]) : 0.0f;
                    g[e] = k + e < t.size ? as_float(at.grad[k + e]) : 0.0f;
                }
            }
            const long long q = t.state + k;
            if constexpr (BITS == 8) {
                decode_m(reinterpret_cast<const uint32_t *>(s.state.m)[q / 4], s.state.m_units[q / BLOCK], m);
                decode_root(reinterpret_cast<const uint32_t *>(s.state.v)[q / 4], s.state.v_units[q / BLOCK], v);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = __fmul_rn(v[e], v[e]);
            } else {
                load4(static_cast<const float *>(s.state.m) + q, m);
                load4(static_cast<const float *>(s.state.v) + q, v);
            }
            float r[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (s.grad_scale) g[e] = __fmul_rn(g[e], scale);
                m[e] = __fadd_rn(__fmul_rn(m[e], s.b1), __fmul_rn(g[e], s.rest1));
                v[e] = __fadd_rn(__fmul_rn(v[e], s.b2), __fmul_rn(__fmul_rn(g[e], g[e]), s.rest2));
                r[e] = __fsqrt_rn(v[e]);
                p[e] = fmaf(-rate, __fdividef(m[e], fmaf(r[e], correct2, s.eps)), p[e] * keep);
            }
            if (full) {
                store_values<P, 4>(at.out + k, p);
                if (at.copy) store_values<__nv_bfloat16, 4>(at.copy + k, p);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (k + e < t.size) {
                        const float one[1] = {p[e]};
                        store_values<P, 1>(at.out + k + e, one);
                        if (at.copy) store_values<__nv_bfloat16, 1>(at.copy + k + e, one);
                    }
            }
            if constexpr (BITS == 8) {
                float um, ur;
                reinterpret_cast<uint32_t *>(s.state.m)[q / 4] = encode_m(m, um);
                reinterpret_cast<uint32_t *>(s.state.v)[q / 4] = encode_root(r, ur);
                if (lane == 0) {
                    s.state.m_units[q / BLOCK] = um;
                    s.state.v_units[q / BLOCK] = ur;
                }
            } else {
                store_values<float, 4>(static_cast<float *>(s.state.m) + q, m);
                store_values<float, 4>(static_cast<float *>(s.state.v) + q, v);
            }
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

// The moments in fp32 from the 8-bit state (READ), or the state from them; a warp for a block.
template <bool READ>
static __global__ void __launch_bounds__(THREADS)
adamw_moments(const State s, long long blocks, float *m_out, float *v_out, const float *m_in, const float *v_in)
{
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    for (long long b = (long long)blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5); b < blocks; b += (long long)gridDim.x * (THREADS / 32)) {
        const long long q = b * BLOCK + 4 * lane;
        uint32_t *mw = static_cast<uint32_t *>(s.m) + q / 4, *vw = static_cast<uint32_t *>(s.v) + q / 4;
        float m[4], v[4];
        if constexpr (READ) {
            decode_m(*mw, s.m_units[b], m);
            decode_root(*vw, s.v_units[b], v);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = __fmul_rn(v[e], v[e]);
            store_values<float, 4>(m_out + q, m);
            store_values<float, 4>(v_out + q, v);
        } else {
            load4(m_in + q, m);
            load4(v_in + q, v);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = __fsqrt_rn(v[e]);
            float um, ur;
            *mw = encode_m(m, um);
            *vw = encode_root(v, ur);
            if (lane == 0) {
                s.m_units[b] = um;
                s.v_units[b] = ur;
            }
        }
    }
}

}  // namespace adamw
}  // namespace cocod
