// Weight gradients per node from 8-bit checkpoints: dW_k = dY_k^T X_k over node k's rows, on the tensor cores.
//
// The sum runs along the rows (tokens) of both operands, and the checkpoint's scale changes from row to row, so the
// 8-bit tensor-core form, whose scales cover 32 steps of the sum, cannot take X without rounding it a second time.
// Instead a code times its scale, exactly a bf16 number, is formed in shared memory by four warps between the TMA and the
// MMA; dY is bf16 and goes in as it is.  Both operands lie along their rows (MN-major): 128 bytes of columns per row.
//
// Rows of other nodes that a tile's last block of rows reaches are set to zero in both operands.
// Sums: the tensor cores add in fp32 in tensor memory over at most kFlushRows rows; then the accumulator is drained into
// registers and added to the total there, so that a long sum does not lose to the accumulator's rounding.
#include "lgc_layers.cuh"
#include "lgc_tensor_core.cuh"

namespace lgc {

namespace {

constexpr int kM = 128, kN = 128;                 // a CTA's tile: columns of dY x columns of X
constexpr int kRows = 64;                         // rows per stage
constexpr int kABytes = kM * kRows * 2, kCodeBytes = kN * kRows, kBBytes = kN * kRows * 2;
constexpr int kPiece = 64 * kRows * 2;            // 64 columns (128 bytes) of a stage's rows in bf16
constexpr int kStages = 4, kReady = 3;            // dY and codes as loaded; X as bf16
constexpr int kFlushRows = 1024;
constexpr int kPitch = 33;                        // floats per row of the result's staging blocks
constexpr int kOutBytes = 4 * 32 * kPitch * 4;
constexpr int kSmemBytes = kStages * (kABytes + kCodeBytes) + kReady * kBBytes + kOutBytes + 1024;
constexpr int kThreads = 320;                     // warp 0: TMA and tensor memory, 1: MMA, 2..5: X to bf16, 6..9: results
constexpr int kTmemCols = 2 * kN;

__device__ __forceinline__ void mma_bf16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate ? 1u : 0u)
        : "memory");
}

// Two codes (bytes 0 and 1 of q, or 2 and 3) as bf16 times a power of two, exact.  A code's exponent and mantissa bits
// moved to bf16's place read as the value times 2^-120 (subnormal codes as subnormal bf16), so factor = scale * 2^120.
__device__ __forceinline__ uint32_t codes_to_bf16(uint32_t q, uint32_t selector, uint32_t factor)
{
    const uint32_t w = __byte_perm(q, 0, selector);            // each code in the upper byte of a half
    const uint32_t x = (w & 0x80008000u) | ((w & 0x7f007f00u) >> 4);
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(factor));
    return r;
}

struct WeightArgs {
    const uint8_t *scales;
    int64_t ld_scales;
    int64_t rows, cols, inner;
    const int64_t *start;
    int nodes;
    float *dw;
    int64_t node_stride;
    int32_t *errword;
    int tiles_m, tiles_n;
};

struct Tile {
    int64_t begin, end;      // rows of the node
    int node, m, n;
    int steps;               // stages of kRows rows
};
__device__ __forceinline__ Tile tile_of(const WeightArgs &p, int64_t t)
{
    Tile w;
    const int64_t per = (int64_t)p.tiles_m * p.tiles_n;
    w.node = (int)(t / per);
    const int r = (int)(t - w.node * per);
    w.m = r % p.tiles_m;
    w.n = r / p.tiles_m;
    w.begin = node_first_row(p.start, w.node, p.rows);
    w.end = node_first_row(p.start, w.node + 1, p.rows);
    if (w.end < w.begin) w.end = w.begin;
    w.steps = (int)((w.end - w.begin + kRows - 1) / kRows);
    return w;
}

__global__ void __launch_bounds__(kThreads, 1)
weight_gradient_kernel(const __grid_constant__ CUtensorMap map_dy, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ WeightArgs p)
{
    extern __shared__ uint8_t dyn_smem[];
    __shared__ __align__(8) uint64_t full_bar[kStages], empty_bar[kStages], ready_bar[kReady], used_bar[kReady], tfull_bar[2], tempty_bar[2];
    __shared__ uint32_t tmem_base;
    __shared__ volatile int failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t base = (smem_addr(dyn_smem) + 1023u) & ~1023u;
    const uint32_t b_tiles = base + kStages * kABytes, codes = b_tiles + kReady * kBBytes;
    constexpr int kFlushSteps = kFlushRows / kRows;
    const int64_t total = (int64_t)p.tiles_m * p.tiles_n * p.nodes;

    if (threadIdx.x == 0) {
        failed = 0;
        for (int s = 0; s < kStages; ++s) {
            bar_init(smem_addr(&full_bar[s]), 1);
            bar_init(smem_addr(&empty_bar[s]), 1);
        }
        for (int s = 0; s < kReady; ++s) {
            bar_init(smem_addr(&ready_bar[s]), 4);
            bar_init(smem_addr(&used_bar[s]), 1);
        }
        for (int s = 0; s < 2; ++s) {
            bar_init(smem_addr(&tfull_bar[s]), 1);
            bar_init(smem_addr(&tempty_bar[s]), 4);
        }
        bar_init_fence();
    }
    if (warp == 0) tc_alloc(&tmem_base, kTmemCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base;

    if (threadIdx.x == 0) {
        int it = 0;
        for (int64_t t = blockIdx.x; t < total && !failed; t += gridDim.x) {
            const Tile w = tile_of(p, t);
            for (int i = 0; i < w.steps; ++i, ++it) {
                const int s = it % kStages;
                if (it >= kStages && !bar_wait(smem_addr(&empty_bar[s]), ((it / kStages) & 1) ^ 1, &failed)) break;
                const uint32_t bar = smem_addr(&full_bar[s]);
                const int row = (int)(w.begin + (int64_t)i * kRows);
                bar_expect(bar, kABytes + kCodeBytes);
#pragma unroll
                for (int j = 0; j < kM / 64; ++j) tma_load(base + s * kABytes + j * kPiece, &map_dy, bar, w.m * kM + 64 * j, row);
#pragma unroll
                for (int j = 0; j < kN / 64; ++j)
                    tma_load(codes + s * kCodeBytes + j * 64 * kRows, &map_x, bar, w.n * kN + 64 * j, row);
            }
        }
    } else if (threadIdx.x == 32) {
        // fp32 sums, bf16 x bf16, both operands MN-major
        constexpr uint32_t idesc = 1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | 1u << 16 | (uint32_t)(kN >> 3) << 17 | (uint32_t)(kM >> 4) << 24;
        int it = 0, acc = 0;
        for (int64_t t = blockIdx.x; t < total && !failed; t += gridDim.x) {
            const Tile w = tile_of(p, t);
            bool ok = true;
            for (int i = 0; i < w.steps; ++i, ++it) {
                const int s = it % kStages, b = it % kReady, buf = acc & 1;
                const bool first = i % kFlushSteps == 0;
                if (first && acc >= 2 && !bar_wait(smem_addr(&tempty_bar[buf]), ((acc >> 1) & 1) ^ 1, &failed)) { ok = false; break; }
                // the warps that make B have waited for the loads; this thread reads dY and waits for itself
                if (!bar_wait(smem_addr(&full_bar[s]), (it / kStages) & 1, &failed) ||
                    !bar_wait(smem_addr(&ready_bar[b]), (it / kReady) & 1, &failed)) { ok = false; break; }
                tc_fence_after();
#pragma unroll
                for (int ks = 0; ks < kRows / 16; ++ks)           // 16 rows of 128 bytes per step
                    mma_bf16(tmem + buf * kN, tc_desc(base + s * kABytes + ks * 2048, kPiece), tc_desc(b_tiles + b * kBBytes + ks * 2048, kPiece),
                             idesc, !first || ks > 0);
                tc_commit(smem_addr(&empty_bar[s]));
                tc_commit(smem_addr(&used_bar[b]));
                if (i % kFlushSteps == kFlushSteps - 1 || i == w.steps - 1) {
                    tc_commit(smem_addr(&tfull_bar[buf]));
                    ++acc;
                }
            }
            if (!ok) break;
        }
    } else if (warp >= 2 && warp < 6) {
        const int id = threadIdx.x - 64;
        int it = 0;
        bool ok = true;
        for (int64_t t = blockIdx.x; t < total && ok; t += gridDim.x) {
            const Tile w = tile_of(p, t);
            for (int i = 0; i < w.steps; ++i, ++it) {
                const int s = it % kStages, b = it % kReady;
                const int64_t row0 = w.begin + (int64_t)i * kRows;
                const int live = (int)min((int64_t)kRows, w.end - row0);          // rows of this node in the stage
                if (!bar_wait_warp(smem_addr(&full_bar[s]), (it / kStages) & 1, &failed) ||
                    (it >= kReady && !bar_wait_warp(smem_addr(&used_bar[b]), ((it / kReady) & 1) ^ 1, &failed))) { ok = false; break; }
                // unit: 16 neighbouring codes of a row; four lanes per row of 64 columns
#pragma unroll
                for (int u = id; u < kN * kRows / 16; u += 128) {
                    const int quarter = u & 3, r = (u >> 2) & (kRows - 1), piece = u >> 8;
                    uint32_t q[4], scale = 0;
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(q[0]), "=r"(q[1]), "=r"(q[2]), "=r"(q[3])
                                 : "r"(codes + s * kCodeBytes + piece * 64 * kRows + r * 64 + quarter * 16));
                    const int64_t block = ((int64_t)w.n * kN + piece * 64) / kBlock;
                    uint32_t f1 = 0, f2 = 0x3f803f80u;
                    if (r < live && block * kBlock < p.inner) {
                        scale = __ldg(p.scales + (row0 + r) * p.ld_scales + block);
                        // scale * 2^120 in two factors where one is beyond bf16's exponents
                        const uint32_t e1 = scale == 255u ? 255u : min(scale, 134u) + 120u, e2 = scale == 255u ? 127u : max(scale, 134u) - 7u;
                        f1 = scale == 255u ? 0x7fff7fffu : (e1 << 7) * 0x10001u;
                        f2 = (e2 << 7) * 0x10001u;
                    }
                    uint32_t x[8];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        x[2 * j] = codes_to_bf16(q[j], 0x1404, f1);
                        x[2 * j + 1] = codes_to_bf16(q[j], 0x3424, f1);
                    }
                    if (scale > 134u)
#pragma unroll
                        for (int j = 0; j < 8; ++j) asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(x[j]) : "r"(f2));
                    const uint32_t at = b_tiles + b * kBBytes + piece * kPiece + r * 128;
                    const int c0 = quarter * 2;                                    // 16-byte chunks, swizzled by the row
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + (((c0) ^ (r & 7)) << 4)), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]) : "memory");
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + (((c0 + 1) ^ (r & 7)) << 4)), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]) : "memory");
                    if (r >= live) {
                        // a row of another node: dY's part becomes zero as well (its chunks of 16 bytes, whatever their order)
                        const uint32_t a = base + s * kABytes + piece * kPiece + r * 128 + quarter * 32;
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(a), "r"(0) : "memory");
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(a + 16), "r"(0) : "memory");
                    }
                }
                async_proxy_fence();
                __syncwarp();
                if (lane == 0) bar_arrive(smem_addr(&ready_bar[b]));
            }
        }
    } else if (warp >= 6) {
        const int q = warp & 3;
        float *stage = reinterpret_cast<float *>(dyn_smem + (base - smem_addr(dyn_smem)) + kStages * (kABytes + kCodeBytes) + kReady * kBBytes) +
                       q * 32 * kPitch;
        int acc = 0;
        bool ok = true;
        for (int64_t t = blockIdx.x; t < total && ok; t += gridDim.x) {
            const Tile w = tile_of(p, t);
            float v[kN];
#pragma unroll
            for (int c = 0; c < kN; ++c) v[c] = 0.0f;
            for (int i = 0; i < w.steps; i += kFlushSteps, ++acc) {
                const int buf = acc & 1;
                if (!bar_wait_warp(smem_addr(&tfull_bar[buf]), (acc >> 1) & 1, &failed)) { ok = false; break; }
                tc_fence_after();
                const uint32_t at = tmem + buf * kN + ((uint32_t)(q * 32) << 16);
#pragma unroll
                for (int c = 0; c < kN; c += 32) {
                    uint32_t r[32];
                    tc_read32(at + c, r);
                    tc_read_wait(r);
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[c + j] = __fadd_rn(v[c + j], __uint_as_float(r[j]));
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(smem_addr(&tempty_bar[buf]));
            }
            if (!ok) break;
            // 32 x 32 entries at a time through shared memory: a warp writes 32 neighbours of a row, wherever the row starts
            float *out = p.dw + w.node * p.node_stride;
            const int64_t row0 = (int64_t)w.m * kM + q * 32;
#pragma unroll
            for (int c = 0; c < kN; c += 32) {
                __syncwarp();
#pragma unroll
                for (int j = 0; j < 32; ++j) stage[lane * kPitch + j] = v[c + j];
                __syncwarp();
                const int64_t col = (int64_t)w.n * kN + c + lane;
                if (col < p.inner)
#pragma unroll 8
                    for (int j = 0; j < 32; ++j)
                        if (row0 + j < p.cols) out[(row0 + j) * p.inner + col] = stage[j * kPitch + lane];
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && failed) atomicExch(p.errword, 2);
    if (warp == 0) tc_free(tmem, kTmemCols);
}

}  // namespace

cudaError_t launch_weight_gradient(const void *dy, int64_t ld_dy, const lgc_packed &x, int64_t rows, int64_t cols, int64_t inner,
                                   const int64_t *node_start, int32_t num_nodes, float *dw, int64_t node_stride, int32_t *errword,
                                   cudaStream_t s)
{
    WeightArgs p{x.scales, x.ld_scales, rows, cols, inner, node_start, num_nodes, dw, node_stride, errword, (int)((cols + kM - 1) / kM),
                 (int)((inner + kN - 1) / kN)};
    CUtensorMap map_dy, map_x;
    cudaError_t e = make_matrix_map(&map_dy, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, dy, cols, rows, ld_dy, 64, kRows, CU_TENSOR_MAP_SWIZZLE_128B);
    if (e != cudaSuccess) return e;
    e = make_matrix_map(&map_x, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, x.codes, inner, rows, x.ld, 64, kRows, CU_TENSOR_MAP_SWIZZLE_NONE);
    if (e != cudaSuccess) return e;
    static OncePerDevice configured;
    e = configured.run([&] { return cudaFuncSetAttribute(weight_gradient_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes); });
    if (e != cudaSuccess) return e;
    const int64_t total = (int64_t)p.tiles_m * p.tiles_n * num_nodes;
    weight_gradient_kernel<<<(unsigned)(total < sm_count() ? total : sm_count()), kThreads, kSmemBytes, s>>>(map_dy, map_x, p);
    ++g_kernel_launches;
    return cudaGetLastError();
}

}  // namespace lgc
