// Activations in 8 bits: whole numbers q with one power of two for each block of 128 columns of a row.
//
// All three kernels stream: a few instructions per byte, so HBM bounds them.  A thread takes 16 consecutive columns (one
// 16-byte access to q, two to a bf16 row), eight threads make a block of 128 columns and find its largest magnitude by
// shuffles; a CTA takes 32 rows of 128 columns, so that the scales, stored column block by column block, leave it as 32
// consecutive bytes.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "cocod_gemm_sm100.cuh"

namespace cocod {
namespace lm {

using namespace cocod::gemm;

constexpr int ACT_BLOCK = 128;         // columns that share a power of two
constexpr int ACT_ROWS = 32;           // rows of a CTA

// 16 bf16 of a row, starting at column c of k; what lies behind the row's end is 0.
__device__ __forceinline__ void load16(const __nv_bfloat16 *row, long long c, long long k, bool vec, uint32_t (&v)[8])
{
    if (vec && c + 16 <= k) {
        const uint4 a = *reinterpret_cast<const uint4 *>(row + c), b = *reinterpret_cast<const uint4 *>(row + c + 8);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
        const unsigned short *r = reinterpret_cast<const unsigned short *>(row);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t lo = c + 2 * j < k ? r[c + 2 * j] : 0, hi = c + 2 * j + 1 < k ? r[c + 2 * j + 1] : 0;
            v[j] = lo | hi << 16;
        }
    }
}
__device__ __forceinline__ void store16(__nv_bfloat16 *row, long long c, long long k, bool vec, const uint32_t (&v)[8])
{
    if (vec && c + 16 <= k) {
        *reinterpret_cast<uint4 *>(row + c) = make_uint4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<uint4 *>(row + c + 8) = make_uint4(v[4], v[5], v[6], v[7]);
    } else {
        unsigned short *r = reinterpret_cast<unsigned short *>(row);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (c + 2 * j < k) r[c + 2 * j] = (unsigned short)v[j];
            if (c + 2 * j + 1 < k) r[c + 2 * j + 1] = (unsigned short)(v[j] >> 16);
        }
    }
}

// e + 127 for the largest finite magnitude, given as bf16 bits: with amax = f 2^E, 1/2 <= f < 1, 127 * 2^(E - 7) reaches amax
// unless f = 255/256, the one bf16 significand above 127/128.
__device__ __forceinline__ int block_exponent(uint32_t amax)
{
    const int exponent = (int)(amax >> 7);                       // E + 126 for normal numbers
    const int e = exponent - 126 - 7 + ((amax & 0x7f) == 0x7f ? 1 : 0);
    return max(e, -126) + 127;
}
__device__ __forceinline__ float power_of_two(int biased) { return __uint_as_float((uint32_t)biased << 23); }

__global__ void __launch_bounds__(256)
act_pack(const __nv_bfloat16 *x, long long ldx, int8_t *q, long long ldq, uint8_t *scales, long long M, long long k, int vec)
{
    __shared__ uint8_t exps[ACT_ROWS];
    pdl_wait();
    const long long m = (long long)blockIdx.x * ACT_ROWS + (threadIdx.x >> 3);
    const long long c = (long long)blockIdx.y * ACT_BLOCK + (threadIdx.x & 7) * 16;
    uint32_t v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (m < M) load16(x + m * ldx, c, k, vec, v);
    uint32_t amax2 = 0;                 // bf16 magnitudes compare like whole numbers, two at a time
#pragma unroll
    for (int j = 0; j < 8; ++j) amax2 = __vmaxu2(amax2, v[j] & 0x7fff7fffu);
    uint32_t amax = max(amax2 & 0xffff, amax2 >> 16);
    const bool plain = amax < 0x7f80;   // none of this thread's values is infinite or NaN
    if (!plain) {
        amax = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t lo = v[j] & 0x7fff, hi = v[j] >> 16 & 0x7fff;
            amax = max(amax, max(lo < 0x7f80 ? lo : 0, hi < 0x7f80 ? hi : 0));
        }
    }
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    const int biased = block_exponent(amax);
    const float inv = power_of_two(254 - biased);       // 2^-e: exact from e = -126 up to the largest e, 122
    // With |y| = |x| 2^-e <= 127, y + 1.5 2^23 rounds y to a whole number, half to even, and holds it in its low byte; |y| below
    // 3/4 counts as 3/4, which rounds to 1, unless it is 0.
    uint32_t packed[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w = v[2 * j + (i >> 1)];
            const float a = __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
            const float y = copysignf(fmaxf(fabsf(a * inv), 0.75f), a);
            b[i] = a == 0.0f ? 0u : __float_as_uint(y + 12582912.0f);
        }
        packed[j] = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
    }
    if (!plain || biased == 122 + 127) {
        // The rare cases, value by value: the marker; and, where e is 122, the largest values would round up to 2^128, which bf16
        // does not hold: they stop at 63 units.
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const uint32_t bits = (v[j >> 1] >> (16 * (j & 1))) & 0xffff;
            int n = (int8_t)(packed[j >> 2] >> (8 * (j & 3)));
            if (biased == 122 + 127) n = min(max(n, -63), 63);
            if ((bits & 0x7fff) >= 0x7f80) n = -128;
            packed[j >> 2] = (packed[j >> 2] & ~(0xffu << (8 * (j & 3)))) | ((uint32_t)n & 0xff) << (8 * (j & 3));
        }
    }
    if (m < M && c < k) *reinterpret_cast<uint4 *>(q + m * ldq + c) = make_uint4(packed[0], packed[1], packed[2], packed[3]);
    const bool all_finite = __all_sync(0xffu << (threadIdx.x & 24), plain);      // of the eight threads of this block of columns
    if ((threadIdx.x & 7) == 0) exps[threadIdx.x >> 3] = all_finite ? (uint8_t)biased : 255;
    __syncthreads();
    const long long mm = (long long)blockIdx.x * ACT_ROWS + threadIdx.x;
    if (threadIdx.x < ACT_ROWS && mm < M) scales[(long long)blockIdx.y * M + mm] = exps[threadIdx.x];
}

// The bf16 pair that two 8-bit values stand for, without the power of two: with t = 128 + (b & 127) and s = 128 or 256 for
// b >= 0 or < 0, both exact in bf16, t - s = b.
__device__ __forceinline__ __nv_bfloat162 pair_of(uint32_t two)       // bytes 0 and 2 of `two`
{
    const uint32_t t = (two & 0x007f007fu) | 0x43004300u, s = (two & 0x00800080u) | 0x43004300u;
    return __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&t), *reinterpret_cast<const __nv_bfloat162 *>(&s));
}
// Four 8-bit values as two bf16 pairs, times the unit.
__device__ __forceinline__ void widen4(uint32_t b, __nv_bfloat162 unit, uint32_t &lo, uint32_t &hi)
{
    __nv_bfloat162 a = __hmul2(pair_of(__byte_perm(b, 0, 0x4140)), unit), c = __hmul2(pair_of(__byte_perm(b, 0, 0x4342)), unit);
    lo = *reinterpret_cast<uint32_t *>(&a);
    hi = *reinterpret_cast<uint32_t *>(&c);
}
// The unit that a scale byte stands for, twice: the exponent field of bf16 starts at bit 7; 255 is NaN (255 << 7 alone would be infinite).
__device__ __forceinline__ __nv_bfloat162 unit_of(uint32_t scale)
{
    const uint32_t bits = scale * 0x00800080u | (scale == 255u ? 0x00400040u : 0u);
    return *reinterpret_cast<const __nv_bfloat162 *>(&bits);
}

__global__ void __launch_bounds__(256)
act_unpack(const int8_t *q, long long ldq, const uint8_t *scales, __nv_bfloat16 *y, long long ldy, long long M, long long k, int vec)
{
    pdl_wait();
    const long long m = (long long)blockIdx.x * ACT_ROWS + (threadIdx.x >> 3);
    const long long c = (long long)blockIdx.y * ACT_BLOCK + (threadIdx.x & 7) * 16;
    if (m >= M || c >= k) return;
    const uint4 b = *reinterpret_cast<const uint4 *>(q + m * ldq + c);
    const __nv_bfloat162 unit = unit_of(scales[(long long)blockIdx.y * M + m]);
    uint32_t v[8];
    widen4(b.x, unit, v[0], v[1]);
    widen4(b.y, unit, v[2], v[3]);
    widen4(b.z, unit, v[4], v[5]);
    widen4(b.w, unit, v[6], v[7]);
    store16(y + m * ldy, c, k, vec, v);
}

__global__ void __launch_bounds__(256)
act_relu_grad(const __nv_bfloat16 *dh, long long lddh, const int8_t *q, long long ldq, __nv_bfloat16 *dz, long long lddz, long long M,
              long long k, int vec)
{
    pdl_wait();
    const long long m = (long long)blockIdx.x * ACT_ROWS + (threadIdx.x >> 3);
    const long long c = (long long)blockIdx.y * ACT_BLOCK + (threadIdx.x & 7) * 16;
    if (m >= M || c >= k) return;
    const uint4 b4 = *reinterpret_cast<const uint4 *>(q + m * ldq + c);
    uint32_t v[8];
    load16(dh + m * lddh, c, k, vec, v);
    const uint32_t b[4] = {b4.x, b4.y, b4.z, b4.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t open = __vcmpgts4(b[j], 0u), bad = __vcmpeq4(b[j], 0x80808080u);
        v[2 * j] &= __byte_perm(open, 0, 0x1100);
        v[2 * j + 1] &= __byte_perm(open, 0, 0x3322);
        if (bad) {
            v[2 * j] |= __byte_perm(bad, 0, 0x1100) & 0x7fff7fffu;
            v[2 * j + 1] |= __byte_perm(bad, 0, 0x3322) & 0x7fff7fffu;
        }
    }
    store16(dz + m * lddz, c, k, vec, v);
}

}  // namespace lm
}  // namespace cocod
