// Activations in 8 bits: whole numbers q with one power of two for each block of 128 columns of a row.
//
// All three kernels stream: a few instructions per byte, so HBM bounds them.  Eight threads make a block of 128 columns of a row; a thread
// takes columns 8 j .. + 7 and 64 + 8 j .. + 7, so that each of its 16-byte accesses to bf16 rows lies beside its neighbours', and two
// rows, whose loads are under way together.  A CTA takes 64 rows of 128 columns; the scales, stored column block by column block,
// leave it as 64 consecutive bytes.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "cocod_gemm_sm100.cuh"

namespace cocod {
namespace lm {

using namespace cocod::gemm;

constexpr int ACT_BLOCK = 128;         // columns that share a power of two
constexpr int ACT_ROWS = 64;           // rows of a CTA of 256 threads

// Eight bf16 of a row, starting at column c of k; what lies behind the row's end is 0.  A row may start at any even address (an odd
// number of columns, a view): the widest accesses that the address allows, at worst one value, three pairs and one value.
__device__ __forceinline__ uint4 load8(const __nv_bfloat16 *row, long long c, long long k)
{
    const unsigned short *r = reinterpret_cast<const unsigned short *>(row) + c;
    const unsigned at = (unsigned)reinterpret_cast<uintptr_t>(r);
    uint4 v;
    if (c + 8 > k) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t lo = c + 2 * j < k ? r[2 * j] : 0, hi = c + 2 * j + 1 < k ? r[2 * j + 1] : 0;
            w[j] = lo | hi << 16;
        }
        v = make_uint4(w[0], w[1], w[2], w[3]);
    } else if ((at & 15) == 0) {
        v = *reinterpret_cast<const uint4 *>(r);
    } else if ((at & 7) == 0) {
        const uint2 a = *reinterpret_cast<const uint2 *>(r), b = *reinterpret_cast<const uint2 *>(r + 4);
        v = make_uint4(a.x, a.y, b.x, b.y);
    } else if ((at & 3) == 0) {
        const uint32_t *w = reinterpret_cast<const uint32_t *>(r);
        v = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
        const uint32_t *w = reinterpret_cast<const uint32_t *>(r + 1);
        const uint32_t first = r[0], a = w[0], b = w[1], d = w[2], last = r[7];
        v = make_uint4(first | a << 16, __funnelshift_l(a, b, 16), __funnelshift_l(b, d, 16), d >> 16 | last << 16);
    }
    return v;
}
__device__ __forceinline__ void store8(__nv_bfloat16 *row, long long c, long long k, uint4 x)
{
    unsigned short *r = reinterpret_cast<unsigned short *>(row) + c;
    const unsigned at = (unsigned)reinterpret_cast<uintptr_t>(r);
    if (c + 8 > k) {
        const uint32_t v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (c + 2 * j < k) r[2 * j] = (unsigned short)v[j];
            if (c + 2 * j + 1 < k) r[2 * j + 1] = (unsigned short)(v[j] >> 16);
        }
    } else if ((at & 15) == 0) {
        *reinterpret_cast<uint4 *>(r) = x;
    } else if ((at & 7) == 0) {
        *reinterpret_cast<uint2 *>(r) = make_uint2(x.x, x.y);
        *reinterpret_cast<uint2 *>(r + 4) = make_uint2(x.z, x.w);
    } else if ((at & 3) == 0) {
        uint32_t *w = reinterpret_cast<uint32_t *>(r);
        w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
    } else {
        uint32_t *w = reinterpret_cast<uint32_t *>(r + 1);
        r[0] = (unsigned short)x.x;
        w[0] = __funnelshift_l(x.x, x.y, 16);
        w[1] = __funnelshift_l(x.y, x.z, 16);
        w[2] = __funnelshift_l(x.z, x.w, 16);
        r[7] = (unsigned short)(x.w >> 16);
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
act_pack(const __nv_bfloat16 *x, long long ldx, int8_t *q, long long ldq, uint8_t *scales, long long M, long long k)
{
    __shared__ uint8_t exps[ACT_ROWS];
    pdl_launch_dependents();
    pdl_wait();
    const long long c = (long long)blockIdx.y * ACT_BLOCK + (threadIdx.x & 7) * 8;
    uint4 in[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const long long m = (long long)blockIdx.x * ACT_ROWS + h * 32 + (threadIdx.x >> 3);
#pragma unroll
        for (int p = 0; p < 2; ++p) in[h][p] = m < M ? load8(x + m * ldx, c + 64 * p, k) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const long long m = (long long)blockIdx.x * ACT_ROWS + h * 32 + (threadIdx.x >> 3);
        const uint32_t v[8] = {in[h][0].x, in[h][0].y, in[h][0].z, in[h][0].w, in[h][1].x, in[h][1].y, in[h][1].z, in[h][1].w};
        uint32_t amax2 = 0;             // bf16 magnitudes compare like whole numbers, two at a time
#pragma unroll
        for (int j = 0; j < 8; ++j) amax2 = __vmaxu2(amax2, v[j] & 0x7fff7fffu);
        uint32_t amax = max(amax2 & 0xffff, amax2 >> 16);
        const bool plain = amax < 0x7f80;       // none of this thread's values is infinite or NaN
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
        const __nv_bfloat162 inv = __float2bfloat162_rn(power_of_two(254 - biased));   // 2^-e: exact from e = -126 up to the largest e, 122
        // Two at a time: y = x 2^-e is exact (what would underflow is far below 3/4); |y| below 3/4 counts as 3/4, which rounds to 1,
        // unless x is 0.  With |y| <= 127, y + 1.5 2^23 rounds y to a whole number, half to even, and holds it in its low byte.
        uint32_t packed[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t b[4], there[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t w = v[2 * j + i];
                const __nv_bfloat162 x2 = *reinterpret_cast<const __nv_bfloat162 *>(&w);
                const __nv_bfloat162 size = __hmax2(__habs2(__hmul2(x2, inv)), __float2bfloat162_rn(0.75f));
                const uint32_t y = (*reinterpret_cast<const uint32_t *>(&size) & 0x7fff7fffu) | (w & 0x80008000u);
                there[i] = __hne2_mask(x2, __float2bfloat162_rn(0.0f));
                b[2 * i] = __float_as_uint(__uint_as_float(y << 16) + 12582912.0f);
                b[2 * i + 1] = __float_as_uint(__uint_as_float(y & 0xffff0000u) + 12582912.0f);
            }
            packed[j] = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410) &
                        __byte_perm(there[0], there[1], 0x6420);
        }
        if (!plain || biased == 122 + 127) {
            // The rare cases, value by value: the marker; and, where e is 122, the largest values would round up to 2^128, which
            // bf16 does not hold: they stop at 63 units.
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const uint32_t bits = (v[j >> 1] >> (16 * (j & 1))) & 0xffff;
                int n = (int8_t)(packed[j >> 2] >> (8 * (j & 3)));
                if (biased == 122 + 127) n = min(max(n, -63), 63);
                if ((bits & 0x7fff) >= 0x7f80) n = -128;
                packed[j >> 2] = (packed[j >> 2] & ~(0xffu << (8 * (j & 3)))) | ((uint32_t)n & 0xff) << (8 * (j & 3));
            }
        }
        if (m < M) {
            int8_t *row = q + m * ldq;
            if (c < k) *reinterpret_cast<uint2 *>(row + c) = make_uint2(packed[0], packed[1]);
            if (c + 64 < k) *reinterpret_cast<uint2 *>(row + c + 64) = make_uint2(packed[2], packed[3]);
        }
        const uint32_t finite = __ballot_sync(0xffffffffu, plain) >> (threadIdx.x & 24) & 0xffu;      // of the eight threads of this block
        if ((threadIdx.x & 7) == 0) exps[h * 32 + (threadIdx.x >> 3)] = finite == 0xffu ? (uint8_t)biased : 255;
    }
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
act_unpack(const int8_t *q, long long ldq, const uint8_t *scales, __nv_bfloat16 *y, long long ldy, long long M, long long k)
{
    pdl_launch_dependents();
    pdl_wait();
    const long long c = (long long)blockIdx.y * ACT_BLOCK + (threadIdx.x & 7) * 8;
    uint2 b[2][2];
    uint32_t scale[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const long long m = (long long)blockIdx.x * ACT_ROWS + h * 32 + (threadIdx.x >> 3);
#pragma unroll
        for (int p = 0; p < 2; ++p)
            b[h][p] = m < M && c + 64 * p < k ? *reinterpret_cast<const uint2 *>(q + m * ldq + c + 64 * p) : make_uint2(0, 0);
        scale[h] = m < M ? scales[(long long)blockIdx.y * M + m] : 0;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const long long m = (long long)blockIdx.x * ACT_ROWS + h * 32 + (threadIdx.x >> 3);
        if (m >= M) return;
        const __nv_bfloat162 unit = unit_of(scale[h]);
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            uint4 v;
            widen4(b[h][p].x, unit, v.x, v.y);
            widen4(b[h][p].y, unit, v.z, v.w);
            if (c + 64 * p < k) store8(y + m * ldy, c + 64 * p, k, v);
        }
    }
}

__global__ void __launch_bounds__(256)
act_relu_grad(const __nv_bfloat16 *dh, long long lddh, const int8_t *q, long long ldq, __nv_bfloat16 *dz, long long lddz, long long M,
              long long k)
{
    pdl_launch_dependents();
    pdl_wait();
    const long long c = (long long)blockIdx.y * ACT_BLOCK + (threadIdx.x & 7) * 8;
    uint2 b[2][2];
    uint4 in[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const long long m = (long long)blockIdx.x * ACT_ROWS + h * 32 + (threadIdx.x >> 3);
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const bool there = m < M && c + 64 * p < k;
            b[h][p] = there ? *reinterpret_cast<const uint2 *>(q + m * ldq + c + 64 * p) : make_uint2(0, 0);
            in[h][p] = there ? load8(dh + m * lddh, c + 64 * p, k) : make_uint4(0, 0, 0, 0);
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const long long m = (long long)blockIdx.x * ACT_ROWS + h * 32 + (threadIdx.x >> 3);
        if (m >= M) return;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const uint32_t bytes[2] = {b[h][p].x, b[h][p].y};
            uint32_t v[4] = {in[h][p].x, in[h][p].y, in[h][p].z, in[h][p].w};
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t open = __vcmpgts4(bytes[j], 0u), bad = __vcmpeq4(bytes[j], 0x80808080u);
                v[2 * j] &= __byte_perm(open, 0, 0x1100);
                v[2 * j + 1] &= __byte_perm(open, 0, 0x3322);
                if (bad) {
                    v[2 * j] |= __byte_perm(bad, 0, 0x1100) & 0x7fff7fffu;
                    v[2 * j + 1] |= __byte_perm(bad, 0, 0x3322) & 0x7fff7fffu;
                }
            }
            if (c + 64 * p < k) store8(dz + m * lddz, c + 64 * p, k, make_uint4(v[0], v[1], v[2], v[3]));
        }
    }
}

}  // namespace lm
}  // namespace cocod
