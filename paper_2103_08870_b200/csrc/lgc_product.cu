// Product of two 8-bit matrices with a power of two per block of 128: Y = act(A B^T) or act(A B), on the tensor cores.
//
// A's scale belongs to a row and 128 neighbours along the contraction, B's to 128 x 128 entries.  Both are powers of two
// in the tensor cores' own scale format, and the block-scaled instruction (kind::mxf8f6f4, one scale per row and 32 along
// the contraction) applies them itself: the four 32-wide steps of a block of 128 use one scale byte.  So the sums stay in
// tensor memory from the first block to the last, in fp32.  B is read in either order (the matrix descriptor says which
// dimension is contiguous): one set of weight bytes serves the forward product and the input gradient.
//
// Scales reach tensor memory as words of four bytes (four blocks of 128 along the contraction) per row: row r of a group
// of 128 sits in lane r % 32 of column r / 32, and tcgen05.cp spreads that over the four quarters of the lanes.
#include "lgc_layers.cuh"
#include "lgc_tensor_core.cuh"

namespace lgc {

namespace {

constexpr int kM = 128, kN = 128;                 // a CTA's tile
constexpr int kStageBytes = (kM + kN) * kBlock;   // one block of 128 along the contraction of both operands
constexpr int kStages = 5;
constexpr int kScaleBytes = (kM + kN) * 4;        // the scale words of four such blocks
constexpr int kSmemBytes = kStages * kStageBytes + 2 * kScaleBytes + 1024;
constexpr int kThreads = 256;                     // warp 0: TMA, 1: MMA, 2: scales, 3: tensor memory, 4..7: results
constexpr int kScaleCol = 2 * kN;                 // tensor memory: two accumulators, then two sets of A's and B's scale columns
constexpr int kScaleCols = (kM + kN) / 32;
constexpr int kTmemCols = 512;

__device__ __forceinline__ void mma_block_scaled(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, bool accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate ? 1u : 0u)
        : "memory");
}
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint32_t smem)
{
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(tc_desc_copy(smem)) : "memory");
}

struct ProductArgs {
    const uint8_t *a_scales, *b_scales;
    int64_t ld_as, ld_bs;
    int64_t rows, cols, inner;
    float slope;
    void *y;
    int32_t type;
    int64_t ldy;
    bool y_vec;
    uint8_t *codes, *scales;
    int64_t ld_codes, ld_scales;
    int32_t *errword;
    int tiles_m, tiles_n;
};

// Tiles in groups of 16 rows of tiles: the tiles that run at a time share their rows of A and B in L2.
__device__ __forceinline__ void tile_of(int64_t t, int tiles_m, int tiles_n, int &m, int &n)
{
    const int64_t per = (int64_t)16 * tiles_n;
    const int g = (int)(t / per);
    const int tall = min(16, tiles_m - g * 16);
    const int r = (int)(t - g * per);
    m = g * 16 + r % tall;
    n = r / tall;
}

template <bool ACROSS>
__global__ void __launch_bounds__(kThreads, 1)
product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ ProductArgs p)
{
    extern __shared__ uint8_t dyn_smem[];
    __shared__ __align__(8) uint64_t full_bar[kStages], empty_bar[kStages], sfull_bar[2], sempty_bar[2], tfull_bar[2], tempty_bar[2];
    __shared__ uint32_t tmem_base;
    __shared__ volatile int failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t tiles = (smem_addr(dyn_smem) + 1023u) & ~1023u;
    const uint32_t scales = tiles + kStages * kStageBytes;
    const int blocks = (int)((p.inner + kBlock - 1) / kBlock);
    const int64_t total = (int64_t)p.tiles_m * p.tiles_n;

    if (threadIdx.x == 0) {
        failed = 0;
        for (int s = 0; s < kStages; ++s) {
            bar_init(smem_addr(&full_bar[s]), 1);
            bar_init(smem_addr(&empty_bar[s]), 1);
        }
        for (int s = 0; s < 2; ++s) {
            bar_init(smem_addr(&sfull_bar[s]), 32);
            bar_init(smem_addr(&sempty_bar[s]), 1);
            bar_init(smem_addr(&tfull_bar[s]), 1);
            bar_init(smem_addr(&tempty_bar[s]), 4);
        }
        bar_init_fence();
    }
    if (warp == 3) tc_alloc(&tmem_base, kTmemCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base;

    if (threadIdx.x == 0) {
        int it = 0;
        for (int64_t tile = blockIdx.x; tile < total && !failed; tile += gridDim.x) {
            int m, n;
            tile_of(tile, p.tiles_m, p.tiles_n, m, n);
            for (int kb = 0; kb < blocks; ++kb, ++it) {
                const int s = it % kStages;
                if (it >= kStages && !bar_wait(smem_addr(&empty_bar[s]), ((it / kStages) & 1) ^ 1, &failed)) break;
                const uint32_t bar = smem_addr(&full_bar[s]), st = tiles + s * kStageBytes;
                bar_expect(bar, kStageBytes);
                tma_load(st, &map_a, bar, kb * kBlock, m * kM);
                if (ACROSS) tma_load(st + kM * kBlock, &map_b, bar, n * kN, kb * kBlock);
                else tma_load(st + kM * kBlock, &map_b, bar, kb * kBlock, n * kN);
            }
        }
    } else if (threadIdx.x == 32) {
        // e4m3 x e4m3, scales in e8m0; B K-major or (across) N-major
        constexpr uint32_t idesc = (ACROSS ? 1u << 16 : 0u) | (uint32_t)(kN >> 3) << 17 | 1u << 23 | (uint32_t)(kM >> 4) << 24;
        int it = 0, quads = 0, acc = 0;
        for (int64_t tile = blockIdx.x; tile < total && !failed; tile += gridDim.x, ++acc) {
            const int buf = acc & 1;
            if (acc >= 2 && !bar_wait(smem_addr(&tempty_bar[buf]), ((acc >> 1) & 1) ^ 1, &failed)) break;
            tc_fence_after();
            bool ok = true;
            for (int kb = 0; kb < blocks; ++kb, ++it) {
                const int s = it % kStages;
                const int q = quads & 1;
                const uint32_t sa = tmem + kScaleCol + q * kScaleCols, sb = sa + kM / 32;
                if ((kb & 3) == 0) {
                    // full means that the set's last user has finished: its shared memory and its columns are free
                    if (!bar_wait(smem_addr(&sfull_bar[q]), (quads >> 1) & 1, &failed)) { ok = false; break; }
                    tc_fence_after();
                    copy_scales(sa, scales + q * kScaleBytes);
                    copy_scales(sb, scales + q * kScaleBytes + kM * 4);
                }
                if (!bar_wait(smem_addr(&full_bar[s]), (it / kStages) & 1, &failed)) { ok = false; break; }
                tc_fence_after();
                const uint32_t st = tiles + s * kStageBytes;
                const uint32_t id = idesc | (uint32_t)(kb & 3) << 4 | (uint32_t)(kb & 3) << 29;    // which byte of the scale words
                const uint64_t a = tc_desc_k(st), b = ACROSS ? tc_desc(st + kM * kBlock, kN * kBlock) : tc_desc_k(st + kM * kBlock);
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)                     // 32 along the contraction: 32 bytes, or 32 rows of 128 bytes
                    mma_block_scaled(tmem + buf * kN, a + (uint64_t)(ks * 32 >> 4), b + (uint64_t)((ACROSS ? ks * 4096 : ks * 32) >> 4), id,
                                     sa, sb, kb > 0 || ks > 0);
                tc_commit(smem_addr(&empty_bar[s]));
                if ((kb & 3) == 3 || kb == blocks - 1) {
                    tc_commit(smem_addr(&sempty_bar[q]));
                    ++quads;
                }
            }
            if (!ok) break;
            tc_commit(smem_addr(&tfull_bar[buf]));
        }
    } else if (warp == 2) {
        // scale words of four blocks along the contraction: lane l serves rows l, l + 32, l + 64, l + 96 of the tile
        int quads = 0;
        bool ok = true;
        for (int64_t tile = blockIdx.x; tile < total && ok; tile += gridDim.x) {
            int m, n;
            tile_of(tile, p.tiles_m, p.tiles_n, m, n);
            for (int kb = 0; kb < blocks; kb += 4, ++quads) {
                const int q = quads & 1;
                uint32_t wa[4], wb = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    int64_t r = (int64_t)m * kM + 32 * j + lane;
                    if (r >= p.rows) r = p.rows - 1;               // (its codes arrive as zeros and its result is not written)
                    wa[j] = __ldg(reinterpret_cast<const uint32_t *>(p.a_scales + r * p.ld_as + kb));
                }
                if (ACROSS) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (kb + j < blocks) wb |= (uint32_t)__ldg(p.b_scales + (int64_t)(kb + j) * p.ld_bs + n) << (8 * j);
                } else {
                    wb = __ldg(reinterpret_cast<const uint32_t *>(p.b_scales + (int64_t)n * p.ld_bs + kb));
                }
                if (quads >= 2 && !bar_wait_warp(smem_addr(&sempty_bar[q]), ((quads >> 1) & 1) ^ 1, &failed)) { ok = false; break; }
                const uint32_t at = scales + q * kScaleBytes + lane * 16;
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(wa[0]), "r"(wa[1]), "r"(wa[2]), "r"(wa[3]) : "memory");
                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at + kM * 4), "r"(wb) : "memory");
                async_proxy_fence();
                bar_arrive(smem_addr(&sfull_bar[q]));
            }
        }
    } else if (warp >= 4) {
        const int q = warp & 3;
        int acc = 0;
        for (int64_t tile = blockIdx.x; tile < total; tile += gridDim.x, ++acc) {
            int m, n;
            tile_of(tile, p.tiles_m, p.tiles_n, m, n);
            const int buf = acc & 1;
            if (!bar_wait_warp(smem_addr(&tfull_bar[buf]), (acc >> 1) & 1, &failed)) break;
            tc_fence_after();
            const int64_t row = (int64_t)m * kM + q * 32 + lane, col0 = (int64_t)n * kN;
            const uint32_t at = tmem + buf * kN + ((uint32_t)(q * 32) << 16);
            float v[kN];
#pragma unroll
            for (int c = 0; c < kN; c += 32) {
                uint32_t r[32];
                tc_read32(at + c, r);
                tc_read_wait(r);
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    const float x = __uint_as_float(r[j]);
                    v[c + j] = p.slope != 1.0f ? leaky_slope(x, p.slope) : x;
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(smem_addr(&tempty_bar[buf]));      // the accumulator may be overwritten
            if (p.y && row < p.rows) {
#pragma unroll
                for (int c = 0; c < kN; c += 8) {
                    const float w[8] = {v[c], v[c + 1], v[c + 2], v[c + 3], v[c + 4], v[c + 5], v[c + 6], v[c + 7]};
                    if (p.type == LGC_TYPE_FP32) {
                        float *yr = static_cast<float *>(p.y) + row * p.ldy;
                        if (p.y_vec) store8<float, true>(yr, col0 + c, p.cols, w);
                        else store8<float, false>(yr, col0 + c, p.cols, w);
                    } else {
                        __nv_bfloat16 *yr = static_cast<__nv_bfloat16 *>(p.y) + row * p.ldy;
                        if (p.y_vec) store8<__nv_bfloat16, true>(yr, col0 + c, p.cols, w);
                        else store8<__nv_bfloat16, false>(yr, col0 + c, p.cols, w);
                    }
                }
            }
            if (p.codes && row < p.rows) {                               // a tile's 128 columns are one block of the result
                uint32_t most = 0;
#pragma unroll
                for (int c = 0; c < kN; ++c) most = max(most, __float_as_uint(v[c]) & 0x7fffffffu);
                const uint32_t s = block_scale(most);
                p.scales[row * p.ld_scales + n] = (uint8_t)s;
#pragma unroll
                for (int c = 0; c < kN; c += 8)
                    store_codes8(p.codes + row * p.ld_codes, col0 + c, p.cols, codes4(v[c], v[c + 1], v[c + 2], v[c + 3], s),
                                 codes4(v[c + 4], v[c + 5], v[c + 6], v[c + 7], s));
            }
            __syncwarp();
        }
    }
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && failed) atomicExch(p.errword, 1);
    if (warp == 3) tc_free(tmem, kTmemCols);
}

}  // namespace

cudaError_t launch_product(const lgc_packed &a, const lgc_packed &b, bool across, int64_t rows, int64_t cols, int64_t inner, float slope,
                           void *y, int32_t type, int64_t ldy, const lgc_packed *packed, int32_t *errword, cudaStream_t s)
{
    CUtensorMap map_a, map_b;
    cudaError_t e = make_matrix_map(&map_a, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, a.codes, inner, rows, a.ld, kBlock, kM, CU_TENSOR_MAP_SWIZZLE_128B);
    if (e != cudaSuccess) return e;
    e = across ? make_matrix_map(&map_b, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, b.codes, cols, inner, b.ld, kN, kBlock, CU_TENSOR_MAP_SWIZZLE_128B)
               : make_matrix_map(&map_b, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, b.codes, inner, cols, b.ld, kBlock, kN, CU_TENSOR_MAP_SWIZZLE_128B);
    if (e != cudaSuccess) return e;
    ProductArgs p{};
    p.a_scales = a.scales, p.b_scales = b.scales, p.ld_as = a.ld_scales, p.ld_bs = b.ld_scales;
    p.rows = rows, p.cols = cols, p.inner = inner, p.slope = slope;
    p.y = y, p.type = type, p.ldy = ldy, p.y_vec = matrix_rows_aligned(y, ldy, type == LGC_TYPE_FP32 ? 4 : 2);
    if (packed) p.codes = packed->codes, p.scales = packed->scales, p.ld_codes = packed->ld, p.ld_scales = packed->ld_scales;
    p.errword = errword;
    p.tiles_m = (int)((rows + kM - 1) / kM), p.tiles_n = (int)((cols + kN - 1) / kN);
    const int64_t total = (int64_t)p.tiles_m * p.tiles_n;
    auto kern = across ? product_kernel<true> : product_kernel<false>;
    static OncePerDevice configured;
    e = configured.run([&] {
        const cudaError_t f = cudaFuncSetAttribute(product_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
        return f != cudaSuccess ? f : cudaFuncSetAttribute(product_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
    });
    if (e != cudaSuccess) return e;
    kern<<<(unsigned)(total < sm_count() ? total : sm_count()), kThreads, kSmemBytes, s>>>(map_a, map_b, p);
    ++g_kernel_launches;
    return cudaGetLastError();
}

}  // namespace lgc
