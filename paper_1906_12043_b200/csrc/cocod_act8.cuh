// Activations in 8 bits: whole numbers q with one power of two for each block of 128 columns of a row.
//
// All three kernels stream, and HBM bounds them while rows start at multiples of 16 bytes.  Eight threads make a block of 128 columns of a
// row; a thread takes columns 8 j .. + 7 and 64 + 8 j .. + 7, so that each of its 16-byte accesses to bf16 rows lies beside its
// neighbours', and one or two rows, whose loads are under way together.  A CTA takes 32 or 64 rows of 128 columns; the scales, stored column
// block by column block, leave it side by side.  32768 rows of 4096: pack 76 us (5.3 TB/s; rounding and packing take about as many
// issue slots as the loads leave), unpack 72 (5.6), gate 111 (6.1).  Rows of 4095: 100, 98 and 120 us, bound by the
// instructions that shift the values; one by one at the widest access that each address allows they took 121, 143 and 186.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "cocod_gemm_sm100.cuh"

namespace cocod {
namespace lm {

using namespace cocod::gemm;

constexpr int ACT_BLOCK = 128;         // columns that share a power of two
constexpr int ACT_ROWS = 32;           // rows that a CTA of 256 threads takes at a time

// Rows of bf16 may start at any even address (an odd number of columns, a view).  Where all start at multiples of 16 bytes (ALIGNED),
// a thread's eight values are one access.  Otherwise a kernel that writes bf16 gives a thread the eight columns that one aligned access
// covers in its row (unpacking 32768 x 4092: 98 us; 106 with two accesses of 8 bytes).  What is read at another alignment comes in
// accesses of 8 or 4 bytes where all rows allow them (A = 8, 4: packing 32768 x 4092 79 us, x 4094 85), else (A = 2) as two aligned
// accesses of 16, the second of which the neighbour reads too, shifted into place (100 us; A = 2 for x 4092: 101).  A row's first
// and last values go one by one there, so that nothing outside the row is touched.
struct Raw8 {
    uint4 a, b;
    int shift;                         // values of `a` before the first wanted one; -1: not read yet
};
// Eight values from column c on, c < k; zeros behind the row's end, and before its start (c < 0 is possible).  The
// accesses are begun here (A: what the addresses of row + c are multiples of) ...
template <int A>
__device__ __forceinline__ Raw8 begin8(const __nv_bfloat16 *row, int c, int k)
{
    Raw8 r;
    r.a = r.b = make_uint4(0, 0, 0, 0);
    const int s = A == 2 ? ((int)(reinterpret_cast<uintptr_t>(row) >> 1) + c) & 7 : 0;
    const bool inner = c - s >= 0 && c - s + (s ? 16 : 8) <= k;
    const __nv_bfloat16 *from = row + (c - s);
    if (inner) {
        if (A == 8) {
            const uint2 x = reinterpret_cast<const uint2 *>(from)[0], y = reinterpret_cast<const uint2 *>(from)[1];
            r.a = make_uint4(x.x, x.y, y.x, y.y);
        } else if (A == 4) {
            const uint32_t *w = reinterpret_cast<const uint32_t *>(from);
            r.a = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            r.a = reinterpret_cast<const uint4 *>(from)[0];
        }
    }
    if (A == 2 && inner && s) r.b = reinterpret_cast<const uint4 *>(from)[1];
    r.shift = inner ? s : -1;
    return r;
}
// ... and put together here.
template <int A>
__device__ __forceinline__ uint4 end8(const Raw8 &r, const __nv_bfloat16 *row, int c, int k)
{
    if (r.shift < 0) {
        const unsigned short *p = reinterpret_cast<const unsigned short *>(row);
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = c + 2 * j;
            const uint32_t lo = i >= 0 && i < k ? p[i] : 0, hi = i + 1 >= 0 && i + 1 < k ? p[i + 1] : 0;
            w[j] = lo | hi << 16;
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    if (A != 2) return r.a;
    const uint32_t w[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
    uint32_t v[6], u[5];
#pragma unroll
    for (int j = 0; j < 6; ++j) v[j] = r.shift & 4 ? w[j + 2] : w[j];
#pragma unroll
    for (int j = 0; j < 5; ++j) u[j] = r.shift & 2 ? v[j + 1] : v[j];
    const uint32_t bits = (r.shift & 1) * 16;
    return make_uint4(__funnelshift_r(u[0], u[1], bits), __funnelshift_r(u[1], u[2], bits), __funnelshift_r(u[2], u[3], bits),
                      __funnelshift_r(u[3], u[4], bits));
}
// Eight values to columns c .. c + 7, as far as they are in the row.  The address of column c is a multiple of 16.
__device__ __forceinline__ void store8(__nv_bfloat16 *row, int c, int k, uint4 x)
{
    if (c >= 0 && c + 8 <= k) {
        *reinterpret_cast<uint4 *>(row + c) = x;
        return;
    }
    unsigned short *r = reinterpret_cast<unsigned short *>(row);
    const uint32_t v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (c + j >= 0 && c + j < k) r[c + j] = (unsigned short)(v[j >> 1] >> (16 * (j & 1)));
}
// How far before column c (a multiple of 8) the eight columns start whose address is a multiple of 16.
template <bool ALIGNED>
__device__ __forceinline__ int lead(const __nv_bfloat16 *row)
{
    return ALIGNED ? 0 : (int)(reinterpret_cast<uintptr_t>(row) >> 1) & 7;
}
// Eight 8-bit values to columns c .. c + 7, as far as they are in the row: what lies behind need not belong to the checkpoint (a view, the
// end of a buffer).
__device__ __forceinline__ void store8_q(int8_t *row, int c, int k, uint2 x)
{
    if (c + 8 <= k) {
        *reinterpret_cast<uint2 *>(row + c) = x;
        return;
    }
#pragma unroll 1
    for (; c < k; ++c) {
        row[c] = (int8_t)x.x;
        x.x = __funnelshift_r(x.x, x.y, 8);
        x.y >>= 8;
    }
}
// The 8-bit values of columns c - s .. c - s + 7 (c a multiple of 8, 0 <= s < 8; rows of q are 16-byte aligned, and the words that hold a
// row's last values may be read as a whole): the words that hold them, and how they come out of those.
template <bool ALIGNED>
__device__ __forceinline__ void begin_q(uint32_t (&w)[3], const int8_t *row, int c, int k, int s)
{
    w[2] = 0;
    if (ALIGNED) {
        const uint2 v = c < k ? *reinterpret_cast<const uint2 *>(row + c) : make_uint2(0, 0);
        w[0] = v.x, w[1] = v.y;
    } else {
        const int from = (c - s) & ~3;
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const int at = from + 4 * i;
            w[i] = at >= 0 && at < k ? *reinterpret_cast<const uint32_t *>(row + at) : 0;
        }
    }
}
template <bool ALIGNED>
__device__ __forceinline__ uint2 end_q(const uint32_t (&w)[3], int s)
{
    if (ALIGNED) return make_uint2(w[0], w[1]);
    const uint32_t bits = (uint32_t)(-s & 3) * 8;
    return make_uint2(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits));
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

template <int A, int H>
__global__ void __launch_bounds__(256)
act_pack(const __nv_bfloat16 *x, long long ldx, int8_t *q, long long ldq, uint8_t *scales, long long M, int k)
{
    __shared__ uint8_t exps[H * ACT_ROWS];
    pdl_launch_dependents();
    pdl_wait();
    const int c = (int)blockIdx.y * ACT_BLOCK + (threadIdx.x & 7) * 8;
    Raw8 raw[H][2];
#pragma unroll
    for (int h = 0; h < H; ++h) {
        const long long m = ((long long)blockIdx.x * H + h) * ACT_ROWS + (threadIdx.x >> 3);
#pragma unroll
        for (int p = 0; p < 2; ++p) raw[h][p] = begin8<A>(x + m * ldx, c + 64 * p, m < M ? k : 0);
    }
#pragma unroll
    for (int h = 0; h < H; ++h) {
        const long long m = ((long long)blockIdx.x * H + h) * ACT_ROWS + (threadIdx.x >> 3);
        uint4 in[2];
#pragma unroll
        for (int p = 0; p < 2; ++p) in[p] = end8<A>(raw[h][p], x + m * ldx, c + 64 * p, m < M ? k : 0);
        const uint32_t v[8] = {in[0].x, in[0].y, in[0].z, in[0].w, in[1].x, in[1].y, in[1].z, in[1].w};
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
            store8_q(row, c, k, make_uint2(packed[0], packed[1]));
            store8_q(row, c + 64, k, make_uint2(packed[2], packed[3]));
        }
        const uint32_t finite = __ballot_sync(0xffffffffu, plain) >> (threadIdx.x & 24) & 0xffu;      // of the eight threads of this block
        if ((threadIdx.x & 7) == 0) exps[h * 32 + (threadIdx.x >> 3)] = finite == 0xffu ? (uint8_t)biased : 255;
    }
    __syncthreads();
    const long long mm = (long long)blockIdx.x * (H * ACT_ROWS) + threadIdx.x;
    if (threadIdx.x < H * ACT_ROWS && mm < M) scales[(long long)blockIdx.y * M + mm] = exps[threadIdx.x];
}

// The bf16 pair that two 8-bit values stand for, without the power of two: with t = 128 + (b & 127) and s = 128 or 256 for
// b >= 0 or < 0, both exact in bf16, t - s = b.
__device__ __forceinline__ __nv_bfloat162 pair_of(uint32_t two)       // bytes 0 and 2 of `two`
{
    const uint32_t t = (two & 0x007f007fu) | 0x43004300u, s = (two & 0x00800080u) | 0x43004300u;
    return __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&t), *reinterpret_cast<const __nv_bfloat162 *>(&s));
}
// Four 8-bit values as two bf16 pairs, times their units.
__device__ __forceinline__ void widen4(uint32_t b, __nv_bfloat162 first, __nv_bfloat162 second, uint32_t &lo, uint32_t &hi)
{
    __nv_bfloat162 a = __hmul2(pair_of(__byte_perm(b, 0, 0x4140)), first), c = __hmul2(pair_of(__byte_perm(b, 0, 0x4342)), second);
    lo = *reinterpret_cast<uint32_t *>(&a);
    hi = *reinterpret_cast<uint32_t *>(&c);
}
// The unit that a scale byte stands for, twice: the exponent field of bf16 starts at bit 7; 255 is NaN (255 << 7 alone would be infinite).
__device__ __forceinline__ __nv_bfloat162 unit_of(uint32_t scale)
{
    const uint32_t bits = scale * 0x00800080u | (scale == 255u ? 0x00400040u : 0u);
    return *reinterpret_cast<const __nv_bfloat162 *>(&bits);
}

template <bool ALIGNED, int H>
__global__ void __launch_bounds__(256)
act_unpack(const int8_t *q, long long ldq, const uint8_t *scales, __nv_bfloat16 *y, long long ldy, long long M, int k)
{
    pdl_launch_dependents();
    pdl_wait();
    const int c = (int)blockIdx.y * ACT_BLOCK + (threadIdx.x & 7) * 8;
    uint32_t b[H][2][3];
    uint32_t scale[H], before[H];      // before: of the block before, where a thread's columns begin in that
#pragma unroll
    for (int h = 0; h < H; ++h) {
        const long long m = ((long long)blockIdx.x * H + h) * ACT_ROWS + (threadIdx.x >> 3);
        const int s = lead<ALIGNED>(y + m * ldy);
        const int valid = m < M ? k : 0;
#pragma unroll
        for (int p = 0; p < 2; ++p) begin_q<ALIGNED>(b[h][p], q + m * ldq, c + 64 * p, valid, s);
        scale[h] = (int)blockIdx.y * ACT_BLOCK < valid ? scales[(long long)blockIdx.y * M + m] : 0;
        before[h] = !ALIGNED && (threadIdx.x & 7) == 0 && blockIdx.y > 0 && m < M ? scales[((long long)blockIdx.y - 1) * M + m] : scale[h];
    }
#pragma unroll
    for (int h = 0; h < H; ++h) {
        const long long m = ((long long)blockIdx.x * H + h) * ACT_ROWS + (threadIdx.x >> 3);
        if (m >= M) return;
        const int s = lead<ALIGNED>(y + m * ldy);
        const __nv_bfloat162 unit = unit_of(scale[h]);
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const uint2 v8 = end_q<ALIGNED>(b[h][p], s);
            uint4 v;
            if (ALIGNED || p == 1) {
                widen4(v8.x, unit, unit, v.x, v.y);
                widen4(v8.y, unit, unit, v.z, v.w);
            } else {                   // the first s values have the unit of the block before
                const __nv_bfloat162 first = unit_of(before[h]);
                __nv_bfloat162 units[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) units[j] = __halves2bfloat162(2 * j < s ? first.x : unit.x, 2 * j + 1 < s ? first.y : unit.y);
                widen4(v8.x, units[0], units[1], v.x, v.y);
                widen4(v8.y, units[2], units[3], v.z, v.w);
            }
            if (c + 64 * p - s < k) store8(y + m * ldy, c + 64 * p - s, k, v);
        }
    }
}

// TOGETHER: the rows of dh start as far from a multiple of 16 bytes as those of dz, and are read as they are written (32768 x 4095:
// 120 us; 231 with the reading for any two addresses).
template <bool ALIGNED, bool TOGETHER, int H>
__global__ void __launch_bounds__(256)
act_relu_grad(const __nv_bfloat16 *dh, long long lddh, const int8_t *q, long long ldq, __nv_bfloat16 *dz, long long lddz, long long M,
              int k)
{
    pdl_launch_dependents();
    pdl_wait();
    const int c = (int)blockIdx.y * ACT_BLOCK + (threadIdx.x & 7) * 8;
    uint32_t b[H][2][3];
    Raw8 raw[H][2];
#pragma unroll
    for (int h = 0; h < H; ++h) {
        const long long m = ((long long)blockIdx.x * H + h) * ACT_ROWS + (threadIdx.x >> 3);
        const int s = lead<ALIGNED>(dz + m * lddz);
        const int valid = m < M ? k : 0;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            begin_q<ALIGNED>(b[h][p], q + m * ldq, c + 64 * p, valid, s);
            raw[h][p] = begin8<ALIGNED || TOGETHER ? 16 : 2>(dh + m * lddh, c + 64 * p - s, valid);
        }
    }
#pragma unroll
    for (int h = 0; h < H; ++h) {
        const long long m = ((long long)blockIdx.x * H + h) * ACT_ROWS + (threadIdx.x >> 3);
        if (m >= M) return;
        const int s = lead<ALIGNED>(dz + m * lddz);
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const uint2 v8 = end_q<ALIGNED>(b[h][p], s);
            const uint4 in = end8<ALIGNED || TOGETHER ? 16 : 2>(raw[h][p], dh + m * lddh, c + 64 * p - s, k);
            const uint32_t bytes[2] = {v8.x, v8.y};
            uint32_t v[4] = {in.x, in.y, in.z, in.w};
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
            if (c + 64 * p - s < k) store8(dz + m * lddz, c + 64 * p - s, k, make_uint4(v[0], v[1], v[2], v[3]));
        }
    }
}

}  // namespace lm
}  // namespace cocod
