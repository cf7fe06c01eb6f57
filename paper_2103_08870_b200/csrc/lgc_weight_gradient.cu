// Weight gradients per node from 8-bit checkpoints: dW_k = dY_k^T X_k over node k's rows, on the tensor cores.
//
// The sum runs along the rows (tokens) of both operands, and the checkpoint's scale changes from row to row, so the
// 8-bit tensor-core form, whose scales cover 32 steps of the sum, cannot take X without rounding it a second time.
// Instead a code times its scale, exactly a bf16 number, is formed in shared memory by sixteen warps between the TMA and the
// MMA; dY is bf16 and goes in as it is.  Both operands lie along their rows (MN-major): 128 bytes of columns per row.
//
// Two CTAs make a tile of 256 x 256 together (cta_group::2): each loads, and converts, half of both operands, which halves
// what a tile of this size costs in loads and conversions per product.
//
// Rows of other nodes that a tile's last block of rows reaches are set to zero in both operands.
// Sums: the tensor cores add in fp32 in tensor memory over at most 64 * 64 rows; longer sums are added up in memory from
// there, so that they do not lose to the accumulator's rounding (it errs by about 2^-24 of the sum per 16 rows).
#include "lgc_layers.cuh"
#include "lgc_tensor_core.cuh"

namespace lgc {

namespace {

constexpr int kM = 256, kN = 256;                 // a pair's tile: columns of dY x columns of X; each CTA loads half of both
constexpr int kRows = 64;                         // rows per stage
constexpr int kHalf = 128;
constexpr int kABytes = kHalf * kRows * 2, kBBytes = kHalf * kRows * 2, kCodeBytes = kHalf * kRows;
constexpr int kStageBytes = kABytes + kBBytes + kCodeBytes;
constexpr int kPiece = 64 * kRows * 2;            // 64 columns (128 bytes) of a stage's rows in bf16
constexpr int kStages = 5;
constexpr int kFlushSteps = 64;                   // stages that the tensor cores add up before their sums go to memory
constexpr int kPitch = 33;                        // floats per row of the result's staging blocks
constexpr int kOutBytes = 4 * 32 * kPitch * 4;
constexpr int kSmemBytes = kStages * (kStageBytes + kRows * 4) + kOutBytes + 1024;
constexpr int kThreads = 768;                     // warp 0: TMA, 1: MMA, 2: scales, 3: tensor memory, 4..7: results, 8..23: X to bf16
constexpr int kTmemCols = 2 * kN;

__device__ __forceinline__ void mma_bf16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
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

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
weight_gradient_kernel(const __grid_constant__ CUtensorMap map_dy, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ WeightArgs p)
{
    extern __shared__ uint8_t dyn_smem[];
    // full: loads of a stage (both CTAs have their own); ready (CTA 0's): X of both halves is bf16; empty: the MMAs are through
    __shared__ __align__(8) uint64_t full_bar[kStages], ready_bar[kStages], empty_bar[kStages], tfull_bar[2], tempty_bar[2];
    __shared__ uint32_t tmem_base;
    __shared__ volatile int failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t base = (smem_addr(dyn_smem) + 1023u) & ~1023u;
    const uint32_t scale_words = base + kStages * kStageBytes;
    const int64_t total = (int64_t)p.tiles_m * p.tiles_n * p.nodes;
    const uint32_t rank = cluster_rank();
    const int64_t first = blockIdx.x >> 1, step = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        failed = 0;
        for (int s = 0; s < kStages; ++s) {
            bar_init(smem_addr(&full_bar[s]), 1 + 32);
            bar_init(smem_addr(&ready_bar[s]), 2 * 8);
            bar_init(smem_addr(&empty_bar[s]), 1);
        }
        for (int s = 0; s < 2; ++s) {
            bar_init(smem_addr(&tfull_bar[s]), 1);
            bar_init(smem_addr(&tempty_bar[s]), 2 * 4);
        }
        bar_init_fence();
    }
    if (warp == 3) tc_alloc_pair(&tmem_base, kTmemCols);
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem = tmem_base;

    if (threadIdx.x == 0) {
        int it = 0;
        for (int64_t t = first; t < total && !failed; t += step) {
            const Tile w = tile_of(p, t);
            const int mc = w.m * kM + (int)rank * kHalf, nc = w.n * kN + (int)rank * kHalf;
            for (int i = 0; i < w.steps; ++i, ++it) {
                const int s = it % kStages;
                if (it >= kStages && !bar_wait(smem_addr(&empty_bar[s]), ((it / kStages) & 1) ^ 1, &failed)) break;
                const uint32_t bar = smem_addr(&full_bar[s]), st = base + s * kStageBytes;
                const int row = (int)(w.begin + (int64_t)i * kRows);
                bar_expect(bar, kABytes + kCodeBytes);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    tma_load(st + j * kPiece, &map_dy, bar, mc + 64 * j, row);
                    tma_load(st + kABytes + kBBytes + j * 64 * kRows, &map_x, bar, nc + 64 * j, row);
                }
            }
        }
    } else if (warp == 1) {
        // fp32 sums, bf16 x bf16, both operands MN-major
        constexpr uint32_t idesc = 1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | 1u << 16 | (uint32_t)(kN >> 3) << 17 | (uint32_t)(kM >> 4) << 24;
        const bool issuer = elect_one();
        int s = 0, acc = 0;
        uint32_t phase = 0;
        bool ok = rank == 0;
        for (int64_t t = first; t < total && ok; t += step) {
            const int steps = __shfl_sync(0xffffffffu, tile_of(p, t).steps, 0);
            for (int i = 0; i < steps; ++i) {
                const int buf = acc & 1;
                const bool begin = i % kFlushSteps == 0, end = i % kFlushSteps == kFlushSteps - 1 || i == steps - 1;
                if (begin && acc >= 2 && !bar_wait_together(smem_addr(&tempty_bar[buf]), ((acc >> 1) & 1) ^ 1, &failed)) { ok = false; break; }
                // the warps that make B wait for the loads of their CTA, dY among them
                if (!bar_wait_together(smem_addr(&ready_bar[s]), phase, &failed)) { ok = false; break; }
                tc_fence_after();
                const uint32_t st = base + s * kStageBytes;
                const uint64_t a = tc_desc(st, kPiece), b = tc_desc(st + kABytes, kPiece);
                if (issuer) {
#pragma unroll
                    for (int ks = 0; ks < kRows / 16; ++ks)       // 16 rows of 128 bytes per step
                        mma_bf16(tmem + buf * kN, a + (uint64_t)(ks * 2048 >> 4), b + (uint64_t)(ks * 2048 >> 4), idesc, !begin || ks > 0);
                    tc_commit_pair(smem_addr(&empty_bar[s]));
                    if (end) tc_commit_pair(smem_addr(&tfull_bar[buf]));
                }
                __syncwarp();
                if (++s == kStages) s = 0, phase ^= 1;
                acc += end;
            }
        }
    } else if (warp == 2) {
        // scale words of the stage's rows (four blocks each; this CTA's columns are one of them)
        int it = 0;
        bool ok = true;
        for (int64_t t = first; t < total && ok; t += step) {
            const Tile w = tile_of(p, t);
            const int64_t block = (int64_t)w.n * 2 + rank;
            for (int i = 0; i < w.steps; ++i, ++it) {
                const int s = it % kStages;
                if (it >= kStages && !bar_wait_together(smem_addr(&empty_bar[s]), ((it / kStages) & 1) ^ 1, &failed)) { ok = false; break; }
#pragma unroll
                for (int j = 0; j < kRows / 32; ++j) {
                    const int64_t row = w.begin + (int64_t)i * kRows + 32 * j + lane;
                    if (row < w.end && block * kBlock < p.inner)
                        word_load(scale_words + (s * kRows + 32 * j + lane) * 4, p.scales + row * p.ld_scales + (block & ~(int64_t)3));
                }
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_addr(&full_bar[s])) : "memory");
            }
        }
    } else if (warp >= 8) {
        // Two groups of eight warps take the stages in turn.  A thread converts 16 neighbouring codes of one row in both
        // 64-column pieces; four lanes per row, so that eight lanes read and write 128 bytes without bank conflicts.
        const int group = (warp - 8) >> 3, id = threadIdx.x & 255, quarter = id & 3, r = id >> 2;
        const uint32_t from = kABytes + kBBytes + r * 64 + quarter * 16, to = kABytes + r * 128;
        const uint32_t c0 = ((quarter * 2) ^ (r & 7)) << 4, c1 = ((quarter * 2 + 1) ^ (r & 7)) << 4;    // 16-byte chunks, swizzled by the row
        int it = 0;
        bool ok = true;
        for (int64_t t = first; t < total && ok; t += step) {
            const Tile w = tile_of(p, t);
            const int64_t block = (int64_t)w.n * 2 + rank;
            const bool any = block * kBlock < p.inner;
            const int shift = (int)(block & 3) * 8;
            for (int i = 0; i < w.steps; ++i, ++it) {
                if ((it & 1) != group) continue;
                const int s = it % kStages;
                const uint32_t st = base + s * kStageBytes;
                const bool live = r < w.end - (w.begin + (int64_t)i * kRows);        // the row is this node's
                if (!bar_wait_together(smem_addr(&full_bar[s]), (it / kStages) & 1, &failed)) { ok = false; break; }
                uint32_t q[2][4], word;
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(q[j][0]), "=r"(q[j][1]), "=r"(q[j][2]), "=r"(q[j][3])
                                 : "r"(st + from + j * 64 * kRows));
                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(word) : "r"(scale_words + (s * kRows + r) * 4));
                const uint32_t scale = (word >> shift) & 255u;
                // scale * 2^120, in two factors where that is beyond bf16's exponents
                uint32_t f1 = ((min(scale, 134u) + 120u) << 7) * 0x10001u, f2 = 0;
                if (scale > 134u) {
                    if (scale == 255u) f1 = 0x7fff7fffu;
                    else f2 = ((scale - 7u) << 7) * 0x10001u;
                }
                if (!live || !any) f1 = f2 = 0;
                uint32_t x[2][8];
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        x[j][2 * k] = codes_to_bf16(q[j][k], 0x1404, f1);
                        x[j][2 * k + 1] = codes_to_bf16(q[j][k], 0x3424, f1);
                    }
                if (f2 != 0)
#pragma unroll
                    for (int j = 0; j < 16; ++j) asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(x[j >> 3][j & 7]) : "r"(f2));
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t at = st + to + j * kPiece;
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + c0), "r"(x[j][0]), "r"(x[j][1]), "r"(x[j][2]), "r"(x[j][3]) : "memory");
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + c1), "r"(x[j][4]), "r"(x[j][5]), "r"(x[j][6]), "r"(x[j][7]) : "memory");
                }
                if (!live) {
                    // a row of another node: dY's part becomes zero as well (its chunks of 16 bytes, whatever their order)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(st + (j >> 1) * kPiece + r * 128 + quarter * 32 + (j & 1) * 16), "r"(0)
                                     : "memory");
                }
                async_proxy_fence();
                __syncwarp();
                if (lane == 0) bar_arrive_cluster(cluster_addr(smem_addr(&ready_bar[s]), 0));
            }
        }
    } else if (warp >= 4) {
        const int q = warp & 3;
        float *stage = reinterpret_cast<float *>(dyn_smem + (scale_words - smem_addr(dyn_smem)) + kStages * kRows * 4) + q * 32 * kPitch;
        int acc = 0;
        bool ok = true;
        for (int64_t t = first; t < total && ok; t += step) {
            const Tile w = tile_of(p, t);
            float *out = p.dw + w.node * p.node_stride;
            const int64_t row0 = (int64_t)w.m * kM + rank * kHalf + q * 32;
            // (a node without rows: its gradient is zero)
            for (int i = 0; i == 0 || i < w.steps; i += kFlushSteps) {
                const int buf = acc & 1;
                if (w.steps > 0) {
                    if (!bar_wait_together(smem_addr(&tfull_bar[buf]), (acc >> 1) & 1, &failed)) { ok = false; break; }
                    tc_fence_after();
                    ++acc;
                }
                const uint32_t at = tmem + buf * kN + ((uint32_t)(q * 32) << 16);
#pragma unroll 1
                for (int c = 0; c < kN; c += 32) {
                    uint32_t v[32];
                    if (w.steps > 0) {
                        tc_read32(at + c, v);
                        tc_read_wait(v);
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = 0;
                    }
                    // 32 x 32 entries through shared memory: a warp writes 32 neighbours of a row, wherever the row starts
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < 32; ++j) stage[lane * kPitch + j] = __uint_as_float(v[j]);
                    __syncwarp();
                    const int64_t col = (int64_t)w.n * kN + c + lane;
                    if (col < p.inner)
#pragma unroll 8
                        for (int j = 0; j < 32; ++j)
                            if (row0 + j < p.cols) {
                                float *o = out + (row0 + j) * p.inner + col;
                                const float x = stage[j * kPitch + lane];
                                *o = i == 0 ? x : __fadd_rn(*o, x);
                            }
                }
                if (w.steps > 0) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive_cluster(cluster_addr(smem_addr(&tempty_bar[buf]), 0));
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();                       // the other CTA's MMAs read this one's shared memory
    if (threadIdx.x == 0 && failed) atomicExch(p.errword, 2);
    if (warp == 3) tc_free_pair(tmem, kTmemCols);
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
    const int64_t pairs = sm_count() / 2;
    weight_gradient_kernel<<<(unsigned)(2 * (total < pairs ? total : pairs)), kThreads, kSmemBytes, s>>>(map_dy, map_x, p);
    ++g_kernel_launches;
    return cudaGetLastError();
}

}  // namespace lgc
