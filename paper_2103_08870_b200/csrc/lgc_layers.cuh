// Internal declarations of the layer operators: the 8-bit matrix format on the device, row loads, the launchers.
#pragma once

#include <cuda_bf16.h>

#include "lgc_internal.cuh"

namespace lgc {

constexpr int kBlock = 128;            // entries of a row that share a scale (weights: 128 x 128 entries)
constexpr int kNormMaxCols = 16384;    // widest row the layer norm kernels hold in registers

// ---- the 8-bit format ---------------------------------------------------------------------------------------------
// The scale byte s of a block from the bits of its largest magnitude: the smallest power of two 2^(s - 127) that
// brings it to 448 = 1.75 * 2^8 or less.  Adding 0x1fffff carries into the exponent exactly when the mantissa is
// above 1.75.  The limits keep code * scale inside bf16 (7: 2^-9 * 2^-120 is a subnormal bf16) and below infinity
// (246: 448 * 2^119 < 2^128).
__device__ __forceinline__ uint32_t block_scale(uint32_t most_bits)
{
    if (most_bits >= 0x7f800000u) return 255u;                        // an entry is not finite
    const int s = (int)((most_bits + 0x1fffffu) >> 23) - 8;
    return (uint32_t)(s < 7 ? 7 : s > 246 ? 246 : s);
}
// 2^(127 - s), exact; not used for s = 255
__device__ __forceinline__ float block_inverse(uint32_t s) { return __uint_as_float((254u - s) << 23); }
// 2^(s - 127): s >= 7 keeps it normal; s = 255 gives NaN
__device__ __forceinline__ float block_factor(uint32_t s) { return s == 255u ? __uint_as_float(0x7fffffffu) : __uint_as_float(s << 23); }

// Four entries of a block to codes, first entry in the lowest byte.
__device__ __forceinline__ uint32_t codes4_bad(float a, float b, float c, float d)       // a block with s = 255: the signs stay
{
    return 0x7f7f7f7fu | (__float_as_uint(a) >> 31) << 7 | (__float_as_uint(b) >> 31) << 15 | (__float_as_uint(c) >> 31) << 23 |
           (__float_as_uint(d) >> 31) << 31;
}
__device__ __forceinline__ uint32_t codes4_scaled(float a, float b, float c, float d)    // entries times 2^(127 - s)
{
    uint32_t r;
    asm("{\n\t.reg .b16 l, h;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\t"
        "mov.b32 %0, {l, h};\n\t}"
        : "=r"(r)
        : "f"(a), "f"(b), "f"(c), "f"(d));
    return r;
}
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, uint32_t s)
{
    if (s == 255u) return codes4_bad(a, b, c, d);
    const float r = block_inverse(s);                                 // exact products: r is a power of two
    return codes4_scaled(__fmul_rn(a, r), __fmul_rn(b, r), __fmul_rn(c, r), __fmul_rn(d, r));
}
// Four codes to floats (without the scale).
__device__ __forceinline__ void codes_to_float4(uint32_t q, float (&v)[4])
{
    uint32_t a, b;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(a) : "h"((uint16_t)(q & 0xffffu)));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(b) : "h"((uint16_t)(q >> 16)));
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, h;\n\t}" : "=f"(v[0]), "=f"(v[1]) : "r"(a));
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, h;\n\t}" : "=f"(v[2]), "=f"(v[3]) : "r"(b));
}

// ---- eight neighbouring entries of a row ------------------------------------------------------------------------------
// VEC: the row starts 16-byte aligned and c is a multiple of 8.  Entries from `cols` on read as zero and are not written.
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T *row, int64_t c, int64_t cols, float (&v)[8])
{
    if (VEC && c + 8 <= cols) {
        if constexpr (sizeof(T) == 2) {
            const uint4 q = __ldg(reinterpret_cast<const uint4 *>(row + c));
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        } else {
            const float4 a = __ldg(reinterpret_cast<const float4 *>(row + c)), b = __ldg(reinterpret_cast<const float4 *>(row + c) + 1);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
            v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? (float)row[c + i] : 0.0f;
    }
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <typename T, bool VEC>
__device__ __forceinline__ void store8(T *row, int64_t c, int64_t cols, const float (&v)[8])
{
    if (VEC && c + 8 <= cols) {
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<uint4 *>(row + c) =
                make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
        } else {
            reinterpret_cast<float4 *>(row + c)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4 *>(row + c)[1] = make_float4(v[4], v[5], v[6], v[7]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < cols) row[c + i] = (T)v[i];
    }
}
// Codes of eight neighbouring entries; code rows always start 16-byte aligned.
__device__ __forceinline__ void store_codes8(uint8_t *row, int64_t c, int64_t cols, uint32_t lo, uint32_t hi)
{
    if (c + 8 <= cols) {
        *reinterpret_cast<uint2 *>(row + c) = make_uint2(lo, hi);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < cols) row[c + i] = (uint8_t)((i < 4 ? lo >> (8 * i) : hi >> (8 * (i - 4))) & 0xffu);
    }
}
// The first `cols - c` of eight codes of a row, zeros behind them.
__device__ __forceinline__ uint2 load_codes8(const uint8_t *row, int64_t c, int64_t cols)
{
    if (c + 8 <= cols) return __ldg(reinterpret_cast<const uint2 *>(row + c));
    uint2 q = make_uint2(0, 0);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c + i < cols) {
            if (i < 4) q.x |= (uint32_t)row[c + i] << (8 * i);
            else q.y |= (uint32_t)row[c + i] << (8 * (i - 4));
        }
    return q;
}
// The framework's activation; its derivative is known from the sign of its result.
__device__ __forceinline__ float leaky_slope(float x, float slope) { return x > 0.0f ? x : __fmul_rn(slope, x); }

// Bits of the largest magnitude of a block whose 128 entries lie in 16 consecutive lanes, eight each.  As integers the
// bits of infinities and NaNs are above those of every number.
__device__ __forceinline__ uint32_t most_of_block(const float (&v)[8])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    return m;
}

// ---- sixteen neighbouring entries of a row, as pairs ---------------------------------------------------------------------
// The streaming kernels fill half to two thirds of the issue slots, so they work on pairs of fp32 numbers in one instruction (add, mul,
// fma .f32x2), take the magnitude's maximum of two entries at a time, and give a lane 16 neighbours: eight lanes hold a
// block, three shuffles find its maximum, and a lane's codes are one 16-byte store.
typedef unsigned long long f2;          // (lower entry, upper entry)
__device__ __forceinline__ f2 f2_of(float lo, float hi)
{
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float f2_lo(f2 a) { return __uint_as_float((uint32_t)a); }
__device__ __forceinline__ float f2_hi(f2 a) { return __uint_as_float((uint32_t)(a >> 32)); }
__device__ __forceinline__ f2 f2_add(f2 a, f2 b) { f2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f2 f2_mul(f2 a, f2 b) { f2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f2 f2_fma(f2 a, f2 b, f2 c) { f2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
// The largest magnitude, NaN if there is one.
__device__ __forceinline__ float most2(f2 a, float m)
{
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(f2_lo(a)), "f"(f2_hi(a)), "f"(m));
    return r;
}

template <typename T>
struct Raw16 {                           // sixteen entries as they lie in memory
    uint32_t w[4 * sizeof(T)];
};
__device__ __forceinline__ f2 raw_pair(const Raw16<__nv_bfloat16> &q, int i)
{
    return f2_of(__uint_as_float(q.w[i] << 16), __uint_as_float(q.w[i] & 0xffff0000u));
}
__device__ __forceinline__ f2 raw_pair(const Raw16<float> &q, int i) { return f2_of(__uint_as_float(q.w[2 * i]), __uint_as_float(q.w[2 * i + 1])); }

// AL: the rows' alignment in bytes (32, 16; 0 = any), c a multiple of 16.  Entries from `cols` on read as zero.
template <int AL, typename T>
__device__ __forceinline__ void load16(const T *row, int c, int cols, Raw16<T> &q)
{
    constexpr int kWords = 4 * sizeof(T);
    if (AL > 0 && c + 16 <= cols) {
        const uint32_t *p = reinterpret_cast<const uint32_t *>(row + c);
        if (AL == 32) {
#pragma unroll
            for (int i = 0; i < kWords; i += 8)
                asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                             : "=r"(q.w[i]), "=r"(q.w[i + 1]), "=r"(q.w[i + 2]), "=r"(q.w[i + 3]), "=r"(q.w[i + 4]), "=r"(q.w[i + 5]),
                               "=r"(q.w[i + 6]), "=r"(q.w[i + 7])
                             : "l"(p + i));
        } else {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
                const uint4 a = __ldg(reinterpret_cast<const uint4 *>(p + i));
                q.w[i] = a.x, q.w[i + 1] = a.y, q.w[i + 2] = a.z, q.w[i + 3] = a.w;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const uint32_t x = c + i < cols ? (sizeof(T) == 2 ? (uint32_t)reinterpret_cast<const uint16_t *>(row)[c + i]
                                                              : reinterpret_cast<const uint32_t *>(row)[c + i])
                                            : 0u;
            if (sizeof(T) == 4) q.w[i % kWords] = x;
            else if (i & 1) q.w[i / 2] |= x << 16;
            else q.w[i / 2] = x;
        }
    }
}
template <int AL, typename T>
__device__ __forceinline__ void store16(T *row, int c, int cols, const f2 (&v)[8])
{
    if (AL > 0 && c + 16 <= cols) {
        uint32_t w[4 * sizeof(T)];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (sizeof(T) == 2) w[i] = bf16_pair(f2_lo(v[i]), f2_hi(v[i]));
            else w[(2 * i) % (4 * sizeof(T))] = (uint32_t)v[i], w[(2 * i + 1) % (4 * sizeof(T))] = (uint32_t)(v[i] >> 32);
        uint32_t *p = reinterpret_cast<uint32_t *>(row + c);
        if (AL == 32) {
#pragma unroll
            for (int i = 0; i < (int)(4 * sizeof(T)); i += 8)
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p + i), "r"(w[i]), "r"(w[i + 1]), "r"(w[i + 2]),
                             "r"(w[i + 3]), "r"(w[i + 4]), "r"(w[i + 5]), "r"(w[i + 6]), "r"(w[i + 7])
                             : "memory");
        } else {
#pragma unroll
            for (int i = 0; i < (int)(4 * sizeof(T)); i += 4) *reinterpret_cast<uint4 *>(p + i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (c + i < cols) row[c + i] = (T)((i & 1) ? f2_hi(v[i / 2]) : f2_lo(v[i / 2]));
    }
}
__device__ __forceinline__ void store_codes16(uint8_t *row, int c, int cols, const uint32_t (&q)[4])
{
    if (c + 16 <= cols) {
        *reinterpret_cast<uint4 *>(row + c) = make_uint4(q[0], q[1], q[2], q[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (c + i < cols) row[c + i] = (uint8_t)(q[i / 4] >> (8 * (i % 4)));
    }
}
__device__ __forceinline__ void load_codes16(const uint8_t *row, int c, int cols, uint32_t (&q)[4])
{
    if (c + 16 <= cols) {
        const uint4 a = __ldg(reinterpret_cast<const uint4 *>(row + c));
        q[0] = a.x, q[1] = a.y, q[2] = a.z, q[3] = a.w;
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (i % 4 == 0) q[i / 4] = 0;
            if (c + i < cols) q[i / 4] |= (uint32_t)row[c + i] << (8 * (i % 4));
        }
    }
}
// The scale byte of a block whose 128 entries lie in eight consecutive lanes, and this lane's sixteen codes.
__device__ __forceinline__ uint32_t codes16(const f2 (&v)[8], uint32_t (&q)[4])
{
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = most2(v[i], m);
    uint32_t most = __float_as_uint(m);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
    const uint32_t s = block_scale(most);
    if (s != 255u) {
        const float r = block_inverse(s);
        const f2 rr = f2_of(r, r);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f2 a = f2_mul(v[2 * i], rr), b = f2_mul(v[2 * i + 1], rr);
            q[i] = codes4_scaled(f2_lo(a), f2_hi(a), f2_lo(b), f2_hi(b));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = codes4_bad(f2_lo(v[2 * i]), f2_hi(v[2 * i]), f2_lo(v[2 * i + 1]), f2_hi(v[2 * i + 1]));
    }
    return s;
}

// Row at which node k starts: inside [0, rows] whatever the array holds.  start == nullptr: one node with every row.
__device__ __forceinline__ int64_t node_first_row(const int64_t *start, int k, int64_t rows)
{
    if (!start) return k == 0 ? 0 : rows;
    const int64_t r = start[k];
    return r < 0 ? 0 : r > rows ? rows : r;
}

// ---- launchers ----------------------------------------------------------------------------------------------------
struct Matrix {                // rows x cols of `type`, rows `ld` elements apart
    const void *p;
    int32_t type;
    int64_t ld;
};
bool matrix_rows_aligned(const void *p, int64_t ld, int elem_bytes);   // every row starts on a 16-byte boundary
int matrix_alignment(const void *p, int64_t ld, int elem_bytes);       // of every row: 32, 16 or 0 (less) bytes

cudaError_t launch_layer_norm(const Matrix &x, int64_t rows, int64_t cols, const float *gamma, const float *beta, float eps, void *y,
                              int64_t ldy, const lgc_packed *packed, float *mean, float *rstd, cudaStream_t s);
size_t layer_norm_backward_scratch(int64_t rows, int64_t cols, int32_t num_nodes);
cudaError_t launch_layer_norm_backward(const Matrix &dy, const Matrix &x, const lgc_packed *x_packed, int64_t rows, int64_t cols,
                                       const float *gamma, const float *mean, const float *rstd, const int64_t *node_start,
                                       int32_t num_nodes, void *dx, int64_t ld_dx, float *dgamma, float *dbeta, int64_t node_stride,
                                       void *scratch, int32_t *errword, cudaStream_t s);
cudaError_t launch_pack(const Matrix &x, int64_t rows, int64_t cols, int32_t block_rows, float slope, const lgc_packed *gate,
                        const lgc_packed &out, void *y, int64_t ldy, cudaStream_t s);
cudaError_t launch_unpack(const lgc_packed &src, int64_t rows, int64_t cols, int32_t block_rows, void *y, int32_t type, int64_t ldy,
                          cudaStream_t s);
cudaError_t launch_product(const lgc_packed &a, const lgc_packed &b, bool across, int64_t rows, int64_t cols, int64_t inner, float slope,
                           void *y, int32_t type, int64_t ldy, const lgc_packed *packed, int32_t *errword, cudaStream_t s);
size_t weight_gradient_scratch(int64_t rows, int64_t cols, int64_t inner, int32_t nodes);
cudaError_t launch_weight_gradient(const void *dy, int64_t ld_dy, const lgc_packed &x, int64_t rows, int64_t cols, int64_t inner,
                                   const int64_t *node_start, int32_t num_nodes, float *dw, int64_t node_stride, void *scratch,
                                   int32_t *errword, cudaStream_t s);

}  // namespace lgc
