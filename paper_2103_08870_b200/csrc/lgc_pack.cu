// 8-bit checkpoints: matrices to e4m3 codes with a power of two per block of 128 (or 128 x 128) entries, and back.
//
// Both directions only stream: an entry is read once and written once, with an exponent comparison and a conversion in
// between, so DRAM bounds them: 16384 x 8192 bf16 66 and 65 us (6.1 and 6.2 TB/s), the gated form 120 us (6.7 TB/s).
#include <type_traits>

#include "lgc_layers.cuh"

namespace lgc {

namespace {

// Blocks of one row: eight consecutive lanes hold a block, sixteen entries each.  Item = (row, block).
// AL, YAL: alignment of the rows of x and y.
template <typename T, int AL, bool GATE, int YAL>
__global__ void __launch_bounds__(256)
pack_rows_kernel(const T *__restrict__ x, int64_t ldx, int64_t rows, int cols, uint32_t blocks_per_row, float slope,
                 const uint8_t *__restrict__ gate, int64_t ld_gate, uint8_t *__restrict__ codes, int64_t ld_codes,
                 uint8_t *__restrict__ scales, int64_t ld_scales, __nv_bfloat16 *__restrict__ y, int64_t ldy)
{
    const int64_t items = rows * blocks_per_row;
    const int64_t item = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 3;
    const int part = threadIdx.x & 7;
    const bool live = item < items;                              // whole groups of eight lanes
    const int64_t row = live ? item / blocks_per_row : 0;
    const int block = live ? (int)(item - row * blocks_per_row) : 0;
    const int c = live ? block * kBlock + part * 16 : cols;      // (a dead group reads and writes nothing)
    Raw16<T> raw;
    load16<AL>(x + row * ldx, c, cols, raw);
    uint32_t g[4];
    if (GATE) load_codes16(gate + row * ld_gate, c, cols, g);
    f2 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = raw_pair(raw, i);
    if (GATE) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t w = g[i / 2] >> (16 * (i & 1));
            v[i] = f2_mul(v[i], f2_of(w & 0x80u ? slope : 1.0f, w & 0x8000u ? slope : 1.0f));
        }
    } else if (slope != 1.0f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = f2_mul(v[i], f2_of(f2_lo(v[i]) > 0.0f ? 1.0f : slope, f2_hi(v[i]) > 0.0f ? 1.0f : slope));
    }
    uint32_t q[4];
    const uint32_t s = codes16(v, q);
    if (y) store16<YAL>(y + row * ldy, c, cols, v);
    store_codes16(codes + row * ld_codes, c, cols, q);
    if (live && part == 0) scales[row * ld_scales + block] = (uint8_t)s;
}

// Blocks of 128 x 128: one CTA each.  The entries stay in registers (64 per thread) between the two passes.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256)
pack_square_kernel(const T *__restrict__ x, int64_t ldx, int64_t rows, int64_t cols, float slope, uint8_t *__restrict__ codes,
                   int64_t ld_codes, uint8_t *__restrict__ scales, int64_t ld_scales, __nv_bfloat16 *__restrict__ y, int64_t ldy, bool y_vec)
{
    __shared__ uint32_t most_of_warp[8];
    const int64_t c = (int64_t)blockIdx.x * kBlock + (threadIdx.x & 15) * 8;
    const int64_t r0 = (int64_t)blockIdx.y * kBlock + (threadIdx.x >> 4);
    float v[8][8];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t r = r0 + 16 * i;
        load8<T, VEC>(x + (r < rows ? r : 0) * ldx, r < rows ? c : cols, cols, v[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (slope != 1.0f) v[i][j] = leaky_slope(v[i][j], slope);
            most = max(most, __float_as_uint(v[i][j]) & 0x7fffffffu);
        }
    }
    most = __reduce_max_sync(0xffffffffu, most);
    if ((threadIdx.x & 31) == 0) most_of_warp[threadIdx.x >> 5] = most;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max(most, most_of_warp[i]);
    const uint32_t s = block_scale(most);
    if (threadIdx.x == 0) scales[blockIdx.y * ld_scales + blockIdx.x] = (uint8_t)s;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t r = r0 + 16 * i;
        if (r >= rows) continue;
        if (y) {
            if (y_vec) store8<__nv_bfloat16, true>(y + r * ldy, c, cols, v[i]);
            else store8<__nv_bfloat16, false>(y + r * ldy, c, cols, v[i]);
        }
        store_codes8(codes + r * ld_codes, c, cols, codes4(v[i][0], v[i][1], v[i][2], v[i][3], s), codes4(v[i][4], v[i][5], v[i][6], v[i][7], s));
    }
}

template <typename T, int AL>
__global__ void __launch_bounds__(256)
unpack_kernel(const uint8_t *__restrict__ codes, int64_t ld_codes, const uint8_t *__restrict__ scales, int64_t ld_scales, int64_t rows,
              int cols, uint32_t parts, int32_t block_rows, T *__restrict__ y, int64_t ldy)
{
    grid_release_dependents();                                   // (the weight gradient sets itself up meanwhile)
    const int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (item >= rows * parts) return;
    const int64_t row = item / parts;
    const int c = (int)(item - row * parts) * 16;
    uint32_t q[4];
    load_codes16(codes + row * ld_codes, c, cols, q);
    const float f = block_factor(__ldg(scales + row / block_rows * ld_scales + c / kBlock));
    const f2 ff = f2_of(f, f);
    f2 v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a[4];
        codes_to_float4(q[i], a);
        v[2 * i] = f2_mul(f2_of(a[0], a[1]), ff);
        v[2 * i + 1] = f2_mul(f2_of(a[2], a[3]), ff);
    }
    store16<AL>(y + row * ldy, c, cols, v);
}

template <typename T>
cudaError_t pack_type(const Matrix &x, int64_t rows, int64_t cols, int32_t block_rows, float slope, const lgc_packed *gate,
                      const lgc_packed &out, __nv_bfloat16 *y, int64_t ldy, cudaStream_t s)
{
    const T *p = static_cast<const T *>(x.p);
    const bool vec = matrix_rows_aligned(x.p, x.ld, sizeof(T)), y_vec = matrix_rows_aligned(y, ldy, 2);
    const int64_t blocks = (cols + kBlock - 1) / kBlock;
    if (block_rows == 1) {
        const int64_t ctas = (rows * blocks + 31) / 32;
        if (ctas > 0x7fffffff) return cudaErrorInvalidConfiguration;
        auto launch = [&](auto kern) {
            kern<<<(unsigned)ctas, 256, 0, s>>>(p, x.ld, rows, (int)cols, (uint32_t)blocks, slope, gate ? gate->codes : nullptr,
                                                gate ? gate->ld : 0, out.codes, out.ld, out.scales, out.ld_scales, y, ldy);
        };
        const int al = matrix_alignment(x.p, x.ld, sizeof(T)), yal = y ? matrix_alignment(y, ldy, 2) : 32;
        auto by_alignment = [&](auto gated) {
            constexpr bool G = decltype(gated)::value;
            if (al == 32 && yal == 32) launch(pack_rows_kernel<T, 32, G, 32>);
            else if (al >= 16) launch(pack_rows_kernel<T, 16, G, 0>);
            else launch(pack_rows_kernel<T, 0, G, 0>);
        };
        if (gate) by_alignment(std::true_type());
        else by_alignment(std::false_type());
    } else {
        const int64_t tall = (rows + kBlock - 1) / kBlock;
        if (tall > 65535 || blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
        auto kern = vec ? pack_square_kernel<T, true> : pack_square_kernel<T, false>;
        kern<<<dim3((unsigned)blocks, (unsigned)tall), 256, 0, s>>>(p, x.ld, rows, cols, slope, out.codes, out.ld, out.scales, out.ld_scales, y,
                                                                    ldy, y_vec);
    }
    ++g_kernel_launches;
    return cudaGetLastError();
}

template <typename T>
cudaError_t unpack_type(const lgc_packed &src, int64_t rows, int64_t cols, int32_t block_rows, T *y, int64_t ldy, cudaStream_t s)
{
    const int64_t parts = (cols + 15) / 16, ctas = (rows * parts + 255) / 256;
    if (ctas > 0x7fffffff) return cudaErrorInvalidConfiguration;
    const int al = matrix_alignment(y, ldy, sizeof(T));
    auto kern = al == 32 ? unpack_kernel<T, 32> : al == 16 ? unpack_kernel<T, 16> : unpack_kernel<T, 0>;
    kern<<<(unsigned)ctas, 256, 0, s>>>(src.codes, src.ld, src.scales, src.ld_scales, rows, (int)cols, (uint32_t)parts, block_rows, y, ldy);
    ++g_kernel_launches;
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_pack(const Matrix &x, int64_t rows, int64_t cols, int32_t block_rows, float slope, const lgc_packed *gate,
                        const lgc_packed &out, void *y, int64_t ldy, cudaStream_t s)
{
    __nv_bfloat16 *yb = static_cast<__nv_bfloat16 *>(y);
    return x.type == LGC_TYPE_FP32 ? pack_type<float>(x, rows, cols, block_rows, slope, gate, out, yb, ldy, s)
                                   : pack_type<__nv_bfloat16>(x, rows, cols, block_rows, slope, gate, out, yb, ldy, s);
}

cudaError_t launch_unpack(const lgc_packed &src, int64_t rows, int64_t cols, int32_t block_rows, void *y, int32_t type, int64_t ldy,
                          cudaStream_t s)
{
    return type == LGC_TYPE_FP32 ? unpack_type(src, rows, cols, block_rows, static_cast<float *>(y), ldy, s)
                                 : unpack_type(src, rows, cols, block_rows, static_cast<__nv_bfloat16 *>(y), ldy, s);
}

}  // namespace lgc
