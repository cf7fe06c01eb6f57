// Weight gradients per node from 8-bit checkpoints: dW_k = dY_k^T X_k over node k's rows, on the tensor cores.
//
// The sum runs along the rows (tokens) of both operands, and the checkpoint's scale changes from row to row, so the
// 8-bit tensor-core form, whose scales cover 32 steps of the sum, cannot take X without rounding it a second time.
// Instead X becomes bf16 first (exact: a code times its scale is a bf16 number), once, in scratch memory, and a bf16 product
// follows.  (Making the bf16 numbers inside the product, between the loads and the tensor cores, saves the 3 bytes an entry
// but repeats the conversion for every 256 columns of dY, and its shared memory and its delay are missing in the ring of
// loads: 626 us against 478 us for 16384 x 4096 x 4096.)
//
// Both operands lie along their rows (MN-major): 128 bytes of columns per row.  Two CTAs make a tile of 256 x 256 together
// (cta_group::2); each loads half of both operands.  Rows of other nodes that a tile's last stage reaches are set to zero in
// both operands, whatever they hold.
// Sums: the tensor cores' additions round towards zero (after 4096 rows a sum is 1.8e-6 of its size too small, and the error
// grows with the rows), so their accumulator takes only 8 * 64 rows at a time; eight warps add those sums up in registers
// while the other accumulator fills.  Where there are few tiles a node's rows are cut into parts, whose sums a last kernel
// adds in order.
//
// What bounds it (16384 x 4096 x 4096, eight nodes: 470 us, tensor pipe 59 %): of its 740,000 cycles the issuing warp waits 46 %
// for loads (boxes of 64 rows of 128 bytes that lie 8 KB apart; 32 KB per CTA and 512 cycles of products), 2 % for cleared
// rows and 10 % for an accumulator to be read.
#include "lgc_layers.cuh"
#include "lgc_tensor_core.cuh"

namespace lgc {

namespace {

constexpr int kM = 256, kN = 256;                 // a pair's tile: columns of dY x columns of X; each CTA loads half of both
constexpr int kRows = 64;                         // rows per stage
constexpr int kHalf = 128;
constexpr int kABytes = kHalf * kRows * 2, kStageBytes = 2 * kABytes;
constexpr int kPiece = 64 * kRows * 2;            // 64 columns (128 bytes) of a stage's rows
constexpr int kStages = 6;
constexpr int kFlushSteps = 8;                    // stages that the tensor cores add up before their sums go to registers
constexpr int kPitch = 33;                        // floats per row of the result's staging blocks
constexpr int kSmemBytes = kStages * kStageBytes + 8 * 32 * kPitch * 4 + 1024;
constexpr int kThreads = 384;                     // warp 0: TMA, 1: MMA, 2: rows of other nodes, 3: tensor memory, 4..11: results
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

struct WeightArgs {
    int64_t rows, cols, inner;
    const int64_t *start;
    int nodes, parts;        // parts of a node's rows
    float *dw;
    int64_t node_stride;
    float *partial;          // [parts][nodes * tiles][256][256] where parts > 1
    int32_t *errword;
    int tiles_m, tiles_n;
};

struct Tile {
    int64_t begin, end;      // rows: from the part's first to the node's end
    int node, m, n;
    int steps;               // stages of kRows rows
};
__device__ __forceinline__ Tile tile_of(const WeightArgs &p, int64_t t)
{
    Tile w;
    const int64_t per = (int64_t)p.tiles_m * p.tiles_n, all = per * p.nodes;
    const int part = (int)(t / all);
    const int64_t u = t - part * all;
    w.node = (int)(u / per);
    const int r = (int)(u - w.node * per);
    w.m = r % p.tiles_m;
    w.n = r / p.tiles_m;
    w.begin = node_first_row(p.start, w.node, p.rows);
    w.end = node_first_row(p.start, w.node + 1, p.rows);
    if (w.end < w.begin) w.end = w.begin;
    const int64_t steps = (w.end - w.begin + kRows - 1) / kRows;
    const int64_t from = steps * part / p.parts, to = steps * (part + 1) / p.parts;
    w.begin += from * kRows;
    w.steps = (int)(to - from);
    return w;
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
weight_gradient_kernel(const __grid_constant__ CUtensorMap map_dy, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ WeightArgs p)
{
    extern __shared__ uint8_t dyn_smem[];
    // full, cleared, tempty: CTA 0's count, for the pair; empty, tfull: arrive in both CTAs; loaded: this CTA's last stage of a tile
    __shared__ __align__(8) uint64_t full_bar[kStages], empty_bar[kStages], loaded_bar[kStages], cleared_bar[kStages], tfull_bar[2], tempty_bar[2];
    __shared__ uint32_t tmem_base;
    __shared__ volatile int failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t base = (smem_addr(dyn_smem) + 1023u) & ~1023u;
    const int64_t total = (int64_t)p.tiles_m * p.tiles_n * p.nodes * p.parts;
    const uint32_t rank = cluster_rank();
    const int64_t first = blockIdx.x >> 1, step = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        failed = 0;
        for (int s = 0; s < kStages; ++s) {
            bar_init(smem_addr(&full_bar[s]), 1);
            bar_init(smem_addr(&empty_bar[s]), 1);
            bar_init(smem_addr(&loaded_bar[s]), 1);
            bar_init(smem_addr(&cleared_bar[s]), 2);
        }
        for (int s = 0; s < 2; ++s) {
            bar_init(smem_addr(&tfull_bar[s]), 1);
            bar_init(smem_addr(&tempty_bar[s]), 2 * 8);
        }
        bar_init_fence();
    }
    if (warp == 3) tc_alloc_pair(&tmem_base, kTmemCols);
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem = tmem_base;
    grid_wait();                          // X in bf16 comes from the launch in front

    // A stage that reaches past its node's end completes at this CTA's own barrier `loaded`; warp 2 clears the rows that are
    // not the node's and reports to `cleared`.  Every other stage completes at CTA 0's `full`.
    if (threadIdx.x == 0) {
        int s = 0;
        uint32_t phase = 1;                                       // the first pass over the stages waits for nobody
        bool ok = true;
        for (int64_t t = first; t < total && ok; t += step) {
            const Tile w = tile_of(p, t);
            const int mc = w.m * kM + (int)rank * kHalf, nc = w.n * kN + (int)rank * kHalf;
            const int steps = w.steps;
            for (int i = 0; i < steps; ++i) {
                if (!bar_wait(smem_addr(&empty_bar[s]), phase, &failed)) { ok = false; break; }
                const int64_t row = w.begin + (int64_t)i * kRows;
                const bool ragged = row + kRows > w.end;
                const uint32_t st = base + s * kStageBytes;
                const uint32_t bar = ragged ? smem_addr(&loaded_bar[s]) : cluster_addr(smem_addr(&full_bar[s]), 0);
                if (ragged) bar_expect(smem_addr(&loaded_bar[s]), kStageBytes);
                else if (rank == 0) bar_expect(smem_addr(&full_bar[s]), 2 * kStageBytes);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    tma_load_pair(st + j * kPiece, &map_dy, bar, mc + 64 * j, (int)row);
                    tma_load_pair(st + kABytes + j * kPiece, &map_x, bar, nc + 64 * j, (int)row);
                }
                if (++s == kStages) s = 0, phase ^= 1;
            }
        }
    } else if (warp == 1) {
        // fp32 sums, bf16 x bf16, both operands MN-major
        constexpr uint32_t idesc = 1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | 1u << 16 | (uint32_t)(kN >> 3) << 17 | (uint32_t)(kM >> 4) << 24;
        const bool issuer = elect_one();
        int s = 0, acc = 0;
        uint32_t full = 0, cleared = 0;                           // a bit per stage: the phases of the two barriers to wait for next
        bool ok = rank == 0;
        for (int64_t t = first; t < total && ok; t += step) {
            const Tile w = tile_of(p, t);
            const int steps = __shfl_sync(0xffffffffu, w.steps, 0);
            const bool ragged_end = __all_sync(0xffffffffu, w.begin + (int64_t)w.steps * kRows > w.end);
            for (int i = 0; i < steps; ++i) {
                const int buf = acc & 1;
                const bool begin = i % kFlushSteps == 0, end = i % kFlushSteps == kFlushSteps - 1 || i == steps - 1;
                if (begin && acc >= 2 && !bar_wait_together(smem_addr(&tempty_bar[buf]), ((acc >> 1) & 1) ^ 1, &failed)) { ok = false; break; }
                if (ragged_end && i == steps - 1) {
                    if (!bar_wait_together(smem_addr(&cleared_bar[s]), (cleared >> s) & 1, &failed)) { ok = false; break; }
                    cleared ^= 1u << s;
                } else {
                    if (!bar_wait_together(smem_addr(&full_bar[s]), (full >> s) & 1, &failed)) { ok = false; break; }
                    full ^= 1u << s;
                }
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
                if (++s == kStages) s = 0;
                acc += end;
            }
        }
    } else if (warp == 2) {
        int s = 0;
        uint32_t phases = 0;                                      // a bit per stage: the phase of `loaded` to wait for next
        for (int64_t t = first; t < total; t += step) {
            const Tile w = tile_of(p, t);
            if (w.steps == 0) continue;
            s = (s + w.steps - 1) % kStages;                      // the tile's last stage
            const int live = (int)(w.end - (w.begin + (int64_t)(w.steps - 1) * kRows));
            if (live < kRows) {
                if (!bar_wait_together(smem_addr(&loaded_bar[s]), (phases >> s) & 1, &failed)) break;
                phases ^= 1u << s;
                // rows of 128 bytes, whose order inside does not matter: four pieces, eight lanes per row
                for (int r = live + (lane >> 3); r < kRows; r += 4)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(base + s * kStageBytes + j * kPiece + r * 128 + (lane & 7) * 16), "r"(0)
                                     : "memory");
                async_proxy_fence();
                __syncwarp();
                if (lane == 0) bar_arrive_cluster(cluster_addr(smem_addr(&cleared_bar[s]), 0));
            }
            s = s + 1 == kStages ? 0 : s + 1;
        }
    } else if (warp >= 4) {
        // a warp: 32 rows, half of the columns
        const int q = warp & 3, half = (warp - 4) >> 2;
        float *stage = reinterpret_cast<float *>(dyn_smem + (base - smem_addr(dyn_smem)) + kStages * kStageBytes) + (warp - 4) * 32 * kPitch;
        const uint32_t drained[2] = {cluster_addr(smem_addr(&tempty_bar[0]), 0), cluster_addr(smem_addr(&tempty_bar[1]), 0)};
        int acc = 0;
        bool ok = true;
        for (int64_t t = first; t < total && ok; t += step) {
            const Tile w = tile_of(p, t);
            float v[kHalf];                                       // (without rows: zeros)
#pragma unroll
            for (int c = 0; c < kHalf; ++c) v[c] = 0.0f;
            for (int i = 0; i < w.steps; i += kFlushSteps, ++acc) {
                const int buf = acc & 1;
                if (!bar_wait_together(smem_addr(&tfull_bar[buf]), (acc >> 1) & 1, &failed)) { ok = false; break; }
                tc_fence_after();
                const uint32_t at = tmem + buf * kN + half * kHalf + ((uint32_t)(q * 32) << 16);
#pragma unroll
                for (int c = 0; c < kHalf; c += 16) {
                    uint32_t r[16];
                    tc_read16(at + c, r);
#pragma unroll
                    for (int j = 0; j < 16; ++j) v[c + j] = __fadd_rn(v[c + j], __uint_as_float(r[j]));
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive_cluster(drained[buf]);
            }
            if (!ok) break;
            // where the tile's entry (0, 0) goes, and how much of the tile is written
            float *out = p.parts > 1 ? p.partial + t * (kM * kN) : p.dw + w.node * p.node_stride + (int64_t)w.m * kM * p.inner + (int64_t)w.n * kN;
            const int64_t ld = p.parts > 1 ? kN : p.inner;
            const int row0 = (int)rank * kHalf + q * 32;
            const int rows = p.parts > 1 ? 32 : (int)min((int64_t)32, p.cols - (int64_t)w.m * kM - row0);
            const int cols = p.parts > 1 ? kN : (int)min((int64_t)kN, p.inner - (int64_t)w.n * kN);
            // 32 x 32 entries at a time through shared memory: a warp writes 32 neighbours of a row, wherever the row starts
#pragma unroll
            for (int c = 0; c < kHalf; c += 32) {
                __syncwarp();
#pragma unroll
                for (int j = 0; j < 32; ++j) stage[lane * kPitch + j] = v[c + j];
                __syncwarp();
                if (half * kHalf + c + lane < cols) {
                    float *o = out + row0 * ld + half * kHalf + c + lane;
#pragma unroll 8
                    for (int j = 0; j < 32; ++j, o += ld)
                        if (j < rows) *o = stage[j * kPitch + lane];
                }
            }
        }
    }
    let_copies_land(&failed);
    tc_fence_before();
    __syncthreads();
    cluster_sync();                       // the other CTA's MMAs read this one's shared memory
    if (threadIdx.x == 0 && failed) atomicExch(p.errword, 2);
    if (warp == 3) tc_free_pair(tmem, kTmemCols);
}

// The parts of every tile, added in order.  A CTA: four rows of a tile; the loads of four parts are under way together.
constexpr int kSumRows = 4;
__global__ void __launch_bounds__(256)
weight_gradient_sum_kernel(const __grid_constant__ WeightArgs p)
{
    grid_wait();
    const int64_t per = (int64_t)p.tiles_m * p.tiles_n, step = per * p.nodes * (kM * kN), t = blockIdx.x;
    const int node = (int)(t / per), r = (int)(t - node * per);
    const int64_t row0 = (int64_t)(r % p.tiles_m) * kM + blockIdx.y * kSumRows, col = (int64_t)(r / p.tiles_m) * kN + threadIdx.x;
    if (col >= p.inner || row0 >= p.cols) return;
    const float *from = p.partial + t * (kM * kN) + blockIdx.y * kSumRows * kN + threadIdx.x;
    float sum[kSumRows] = {};
    for (int part = 0; part < p.parts; part += 4, from += 4 * step) {
        float v[4][kSumRows];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < kSumRows; ++j) v[i][j] = part + i < p.parts ? __ldcg(from + i * step + j * kN) : 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < kSumRows; ++j) sum[j] = __fadd_rn(sum[j], v[i][j]);
    }
    float *out = p.dw + node * p.node_stride + row0 * p.inner + col;
#pragma unroll
    for (int j = 0; j < kSumRows; ++j)
        if (row0 + j < p.cols) out[j * p.inner] = sum[j];
}

int64_t x_bytes(int64_t rows, int64_t inner) { return (rows * ((inner + 7) / 8 * 8) * 2 + 255) / 256 * 256; }
int64_t tiles_for(int64_t cols, int64_t inner, int32_t nodes) { return ((cols + kM - 1) / kM) * ((inner + kN - 1) / kN) * nodes; }

// Parts of a node's rows: as many as give every pair of SMs a tile, but at least eight stages to a part.
int parts_for(int64_t rows, int64_t cols, int64_t inner, int32_t nodes)
{
    const int64_t tiles = tiles_for(cols, inner, nodes), most = 148 / 2 / tiles, long_enough = rows / nodes / (8 * kRows);
    const int64_t parts = most < long_enough ? most : long_enough;
    return parts < 2 ? 1 : (int)parts;
}

}  // namespace

size_t weight_gradient_scratch(int64_t rows, int64_t cols, int64_t inner, int32_t nodes)
{
    const int parts = parts_for(rows, cols, inner, nodes);
    return (size_t)x_bytes(rows, inner) + (parts > 1 ? (size_t)parts * tiles_for(cols, inner, nodes) * kM * kN * 4 : 0);
}

cudaError_t launch_weight_gradient(const void *dy, int64_t ld_dy, const lgc_packed &x, int64_t rows, int64_t cols, int64_t inner,
                                   const int64_t *node_start, int32_t num_nodes, float *dw, int64_t node_stride, void *scratch,
                                   int32_t *errword, cudaStream_t s)
{
    const int64_t ld_x = (inner + 7) / 8 * 8;
    cudaError_t e = launch_unpack(x, rows, inner, 1, scratch, LGC_TYPE_BF16, ld_x, s);
    if (e != cudaSuccess) return e;
    WeightArgs p{rows, cols, inner, node_start, num_nodes, parts_for(rows, cols, inner, num_nodes), dw, node_stride,
                 reinterpret_cast<float *>(static_cast<char *>(scratch) + x_bytes(rows, inner)), errword, (int)((cols + kM - 1) / kM),
                 (int)((inner + kN - 1) / kN)};
    CUtensorMap map_dy, map_x;
    e = make_matrix_map(&map_dy, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, dy, cols, rows, ld_dy, 64, kRows, CU_TENSOR_MAP_SWIZZLE_128B);
    if (e != cudaSuccess) return e;
    e = make_matrix_map(&map_x, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, scratch, inner, rows, ld_x, 64, kRows, CU_TENSOR_MAP_SWIZZLE_128B);
    if (e != cudaSuccess) return e;
    static OncePerDevice configured;
    e = configured.run([&] { return cudaFuncSetAttribute(weight_gradient_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes); });
    if (e != cudaSuccess) return e;
    const int64_t tiles = tiles_for(cols, inner, num_nodes), total = tiles * p.parts, pairs = sm_count() / 2;
    e = launch_dependent_smem(weight_gradient_kernel, dim3((unsigned)(2 * (total < pairs ? total : pairs))), dim3(kThreads), kSmemBytes, s, map_dy,
                              map_x, p);
    if (e != cudaSuccess) return e;
    ++g_kernel_launches;
    if (p.parts > 1) {
        e = launch_dependent(weight_gradient_sum_kernel, dim3((unsigned)tiles, kM / kSumRows), dim3(256), s, p);
        if (e != cudaSuccess) return e;
        ++g_kernel_launches;
    }
    return cudaGetLastError();
}

}  // namespace lgc
