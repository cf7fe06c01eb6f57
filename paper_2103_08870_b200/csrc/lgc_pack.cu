// 8-bit checkpoints: matrices to e4m3 codes with a power of two per block of 128 (or 128 x 128) entries, and back.
//
// Both directions only stream: an entry is read once and written once, with an exponent comparison and a conversion in
// between, so DRAM bounds them.
#include "lgc_layers.cuh"

namespace lgc {

namespace {

// Blocks of one row: 16 consecutive lanes hold a block of 128 entries, eight each, and find its largest magnitude with
// four shuffles.  Item = (row, block).
template <typename T, bool VEC, bool GATE>
__global__ void __launch_bounds__(256)
pack_rows_kernel(const T *__restrict__ x, int64_t ldx, int64_t rows, int64_t cols, uint32_t blocks_per_row, float slope,
                 const uint8_t *__restrict__ gate, int64_t ld_gate, uint8_t *__restrict__ codes, int64_t ld_codes,
                 uint8_t *__restrict__ scales, int64_t ld_scales, __nv_bfloat16 *__restrict__ y, int64_t ldy, bool y_vec)
{
    const int64_t items = rows * blocks_per_row;
    const int64_t item = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 4;
    const int part = threadIdx.x & 15;
    const bool live = item < items;                              // whole groups of 16 lanes
    const int64_t row = live ? item / blocks_per_row : 0;
    const int64_t block = live ? item - row * blocks_per_row : 0;
    const int64_t c = live ? block * kBlock + part * 8 : cols;   // (a dead group reads and writes nothing)
    float v[8];
    load8<T, VEC>(x + row * ldx, c, cols, v);
    if (GATE) {
        const uint2 q = load_codes8(gate + row * ld_gate, c, cols);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((i < 4 ? q.x >> (8 * i) : q.y >> (8 * (i - 4))) & 0x80u) v[i] = __fmul_rn(slope, v[i]);
    } else if (slope != 1.0f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = leaky_slope(v[i], slope);
    }
    const uint32_t s = block_scale(most_of_block(v));
    if (y) {
        if (y_vec) store8<__nv_bfloat16, true>(y + row * ldy, c, cols, v);
        else store8<__nv_bfloat16, false>(y + row * ldy, c, cols, v);
    }
    store_codes8(codes + row * ld_codes, c, cols, codes4(v[0], v[1], v[2], v[3], s), codes4(v[4], v[5], v[6], v[7], s));
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

template <typename T, bool VEC>
__global__ void __launch_bounds__(256)
unpack_kernel(const uint8_t *__restrict__ codes, int64_t ld_codes, const uint8_t *__restrict__ scales, int64_t ld_scales, int64_t rows,
              int64_t cols, uint32_t eighths, int32_t block_rows, T *__restrict__ y, int64_t ldy)
{
    const int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (item >= rows * eighths) return;
    const int64_t row = item / eighths;
    const int64_t c = (item - row * eighths) * 8;
    const uint2 q = load_codes8(codes + row * ld_codes, c, cols);
    const float f = block_factor(__ldg(scales + row / block_rows * ld_scales + c / kBlock));
    float a[4], b[4];
    codes_to_float4(q.x, a);
    codes_to_float4(q.y, b);
    const float v[8] = {__fmul_rn(a[0], f), __fmul_rn(a[1], f), __fmul_rn(a[2], f), __fmul_rn(a[3], f),
                        __fmul_rn(b[0], f), __fmul_rn(b[1], f), __fmul_rn(b[2], f), __fmul_rn(b[3], f)};
    store8<T, VEC>(y + row * ldy, c, cols, v);
}

template <typename T>
cudaError_t pack_type(const Matrix &x, int64_t rows, int64_t cols, int32_t block_rows, float slope, const lgc_packed *gate,
                      const lgc_packed &out, __nv_bfloat16 *y, int64_t ldy, cudaStream_t s)
{
    const T *p = static_cast<const T *>(x.p);
    const bool vec = matrix_rows_aligned(x.p, x.ld, sizeof(T)), y_vec = matrix_rows_aligned(y, ldy, 2);
    const int64_t blocks = (cols + kBlock - 1) / kBlock;
    if (block_rows == 1) {
        const int64_t ctas = (rows * blocks + 15) / 16;
        if (ctas > 0x7fffffff) return cudaErrorInvalidConfiguration;
        auto kern = gate ? (vec ? pack_rows_kernel<T, true, true> : pack_rows_kernel<T, false, true>)
                         : (vec ? pack_rows_kernel<T, true, false> : pack_rows_kernel<T, false, false>);
        kern<<<(unsigned)ctas, 256, 0, s>>>(p, x.ld, rows, cols, (uint32_t)blocks, slope, gate ? gate->codes : nullptr, gate ? gate->ld : 0,
                                            out.codes, out.ld, out.scales, out.ld_scales, y, ldy, y_vec);
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
    const int64_t eighths = (cols + 7) / 8, ctas = (rows * eighths + 255) / 256;
    if (ctas > 0x7fffffff) return cudaErrorInvalidConfiguration;
    auto kern = matrix_rows_aligned(y, ldy, sizeof(T)) ? unpack_kernel<T, true> : unpack_kernel<T, false>;
    kern<<<(unsigned)ctas, 256, 0, s>>>(src.codes, src.ld, src.scales, src.ld_scales, rows, cols, (uint32_t)eighths, block_rows, y, ldy);
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
