// Product of two 8-bit matrices with a power of two per block of 128: Y = act(A B^T) or act(A B), on the tensor cores.
//
// A's scale belongs to a row and 128 neighbours along the contraction, B's to 128 x 128 entries.  Both are powers of two
// in the tensor cores' own scale format, and the block-scaled instruction (kind::mxf8f6f4, one scale per row and 32 along
// the contraction) applies them itself: the four 32-wide steps of a block of 128 use one scale byte.  B is read in either
// order (the matrix descriptor says which dimension is contiguous): one set of weight bytes serves the forward product and
// the input gradient.
//
// Sums: the tensor cores' additions into tensor memory round towards zero, so a long sum ends too small by more than its
// rounding (terms of one sign: 4096 of them 1.4e-6, 16384 9.9e-6).  Their accumulator therefore takes only kFlushBlocks blocks
// at a time; the result warps add those sums up in fp32 registers, to nearest, while the other accumulator fills.
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
// Blocks that the tensor cores add up, a multiple of 4 (whole scale words).  128 x 4096 x 4096: 15.6 us with 4, 16.3 with 16;
// 16384 terms of one sign lose 7e-8 and 5e-7.
constexpr int kFlushBlocks = 4;
constexpr int kPiecePitch = 144;                  // bytes of a row in the results' staging: the lanes' 16-byte stores fall into different banks
constexpr int kPieceWarp = 32 * kPiecePitch;      // a result warp's staging
constexpr int kPieceBytes = 4 * kPieceWarp;
constexpr int kSmemBytes = kStages * kStageBytes + 2 * kScaleBytes + kPieceBytes + 1024;
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

// 32 rows of a tile in pieces of 128 bytes go through shared memory, STAGED rows at a time, so that eight lanes write a row's
// piece together: from registers, a lane per row, every 16 bytes would be a write of their own.  put: stores the lane's piece at
// the address it is given; at: where row 0's piece begins; bytes: how much of a piece lies inside the matrix; vec: rows and
// pieces start on 16-byte boundaries.
template <int STAGED, typename Put>
__device__ __forceinline__ void write_piece(uint8_t *stage, Put put, uint8_t *at, int64_t ld_bytes, int rows, int bytes, bool vec, int elem_bytes)
{
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (int h = 0; h < 32; h += STAGED, at += STAGED * ld_bytes, rows -= STAGED) {
        __syncwarp();
        if (STAGED == 32 || lane / STAGED * STAGED == h) put(stage + lane % STAGED * kPiecePitch);
        __syncwarp();
        if (vec && bytes >= 128) {
#pragma unroll
            for (int i = 0; i < STAGED / 4; ++i) {
                const int r = i * 4 + (lane >> 3), c = (lane & 7) * 16;
                if (r < rows) *reinterpret_cast<uint4 *>(at + r * ld_bytes + c) = *reinterpret_cast<const uint4 *>(stage + r * kPiecePitch + c);
            }
        } else {
            const int upto = min(STAGED, rows);
#pragma unroll 4
            for (int r = 0; r < upto; ++r)
                for (int c = lane * elem_bytes; c < bytes && c < 128; c += 32 * elem_bytes) {
                    const uint8_t *from = stage + r * kPiecePitch + c;
                    uint8_t *to = at + r * ld_bytes + c;
                    if (elem_bytes == 4) *reinterpret_cast<uint32_t *>(to) = *reinterpret_cast<const uint32_t *>(from);
                    else if (elem_bytes == 2) *reinterpret_cast<uint16_t *>(to) = *reinterpret_cast<const uint16_t *>(from);
                    else *to = *from;
                }
        }
    }
}

// A block of 128 columns of the result (number `block`), 32 rows from row0 on, a row per lane: 16- or 32-bit and / or 8-bit.
// v: the columns in pieces of 32, which stand in order (flip = 0) or the last one first (flip = 3).
template <int STAGED>
__device__ __forceinline__ void write_block(const ProductArgs &p, float (&v)[128], int flip, int64_t row0, int64_t block, uint8_t *stage)
{
    const int lane = threadIdx.x & 31;
    const int rows = (int)max((int64_t)0, min((int64_t)32, p.rows - row0));
    const int64_t col0 = block * kBlock;
    const int width = (int)max((int64_t)0, min((int64_t)kBlock, p.cols - col0));
    if (p.slope != 1.0f)
#pragma unroll
        for (int c = 0; c < kBlock; ++c) v[c] = leaky_slope(v[c], p.slope);
    if (p.y && p.type == LGC_TYPE_FP32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int first = 32 * (i ^ flip);
            write_piece<STAGED>(stage, [&](uint8_t *to) {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    reinterpret_cast<float4 *>(to)[k] = make_float4(v[32 * i + 4 * k], v[32 * i + 4 * k + 1], v[32 * i + 4 * k + 2], v[32 * i + 4 * k + 3]);
            }, reinterpret_cast<uint8_t *>(static_cast<float *>(p.y) + row0 * p.ldy + col0 + first), p.ldy * 4, rows, (width - first) * 4, p.y_vec, 4);
        }
    } else if (p.y) {
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            const int first = 32 * ((i ^ flip) & 2);
            write_piece<STAGED>(stage, [&](uint8_t *to) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float *e = v + 32 * i + 8 * k;
                    reinterpret_cast<uint4 *>(to)[k ^ (flip & 1) * 4] =
                        make_uint4(bf16_pair(e[0], e[1]), bf16_pair(e[2], e[3]), bf16_pair(e[4], e[5]), bf16_pair(e[6], e[7]));
                }
            }, reinterpret_cast<uint8_t *>(static_cast<__nv_bfloat16 *>(p.y) + row0 * p.ldy + col0 + first), p.ldy * 2, rows, (width - first) * 2, p.y_vec, 2);
        }
    }
    if (p.codes) {
        float most = 0.0f;
#pragma unroll
        for (int c = 0; c < kBlock; c += 2) most = most2(f2_of(v[c], v[c + 1]), most);
        const uint32_t s = block_scale(__float_as_uint(most));
        if (lane < rows && width > 0) p.scales[(row0 + lane) * p.ld_scales + block] = (uint8_t)s;
        uint32_t w[32];
        if (s != 255u) {
            const float r = block_inverse(s);
#pragma unroll
            for (int j = 0; j < 32; ++j)
                w[j] = codes4_scaled(__fmul_rn(v[4 * j], r), __fmul_rn(v[4 * j + 1], r), __fmul_rn(v[4 * j + 2], r), __fmul_rn(v[4 * j + 3], r));
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) w[j] = codes4_bad(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        }
        write_piece<STAGED>(stage, [&](uint8_t *to) {
#pragma unroll
            for (int k = 0; k < 8; ++k) reinterpret_cast<uint4 *>(to)[k ^ flip * 2] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
        }, p.codes + row0 * p.ld_codes + col0, p.ld_codes, rows, width, true, 1);
    }
}

// Adds 128 columns of an accumulator to a lane's sums, in pieces of 32 (piece i of v: the columns from 32 * (i ^ flip) on); a
// piece's reads are under way while the one in front is added.  first(): once the first piece has been read.
template <typename First>
__device__ __forceinline__ void add_columns(float (&v)[128], uint32_t at, int flip, First first)
{
    uint32_t r[2][32];
    tc_read32(at + 32 * flip, r[0]);
    tc_read_wait(r[0]);
    first();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i < 3) tc_read32(at + 32 * ((i + 1) ^ flip), r[(i + 1) & 1]);
#pragma unroll
        for (int j = 0; j < 32; ++j) v[32 * i + j] = __fadd_rn(v[32 * i + j], __uint_as_float(r[i & 1][j]));
        if (i < 3) tc_read_wait(r[(i + 1) & 1]);
    }
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
        int s = 0;
        uint32_t phase = 1;                                       // the first pass over the stages waits for nobody
        bool ok = true;
        for (int64_t tile = blockIdx.x; tile < total && ok; tile += gridDim.x) {
            int m, n;
            tile_of(tile, p.tiles_m, p.tiles_n, m, n);
            for (int kb = 0; kb < blocks; ++kb) {
                if (!bar_wait(smem_addr(&empty_bar[s]), phase, &failed)) { ok = false; break; }
                const uint32_t bar = smem_addr(&full_bar[s]), st = tiles + s * kStageBytes;
                bar_expect(bar, kStageBytes);
                tma_load(st, &map_a, bar, kb * kBlock, m * kM);
                if (ACROSS) tma_load(st + kM * kBlock, &map_b, bar, n * kN, kb * kBlock);
                else tma_load(st + kM * kBlock, &map_b, bar, kb * kBlock, n * kN);
                if (++s == kStages) s = 0, phase ^= 1;
            }
        }
    } else if (warp == 1) {
        // e4m3 x e4m3, scales in e8m0; B K-major or (across) N-major
        constexpr uint32_t idesc = (ACROSS ? 1u << 16 : 0u) | (uint32_t)(kN >> 3) << 17 | 1u << 23 | (uint32_t)(kM >> 4) << 24;
        const bool issuer = elect_one();
        int s = 0, quads = 0, acc = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int64_t tile = blockIdx.x; tile < total && ok; tile += gridDim.x) {
            for (int kb = 0; kb < blocks; ++kb) {
                const int q = quads & 1, buf = acc & 1;
                const bool begin = kb % kFlushBlocks == 0, end = kb % kFlushBlocks == kFlushBlocks - 1 || kb == blocks - 1;
                const uint32_t sa = tmem + kScaleCol + q * kScaleCols, sb = sa + kM / 32;
                if (begin && acc >= 2 && !bar_wait_together(smem_addr(&tempty_bar[buf]), ((acc >> 1) & 1) ^ 1, &failed)) { ok = false; break; }
                // full means that the set's last user has finished: its shared memory and its columns are free
                if ((kb & 3) == 0 && !bar_wait_together(smem_addr(&sfull_bar[q]), (quads >> 1) & 1, &failed)) { ok = false; break; }
                if (!bar_wait_together(smem_addr(&full_bar[s]), phase, &failed)) { ok = false; break; }
                tc_fence_after();
                const uint32_t st = tiles + s * kStageBytes;
                const uint32_t id = idesc | (uint32_t)(kb & 3) << 4 | (uint32_t)(kb & 3) << 29;    // which byte of the scale words
                const uint64_t a = tc_desc_k(st), b = ACROSS ? tc_desc(st + kM * kBlock, kN * kBlock) : tc_desc_k(st + kM * kBlock);
                const bool last = (kb & 3) == 3 || kb == blocks - 1;
                if (issuer) {
                    if ((kb & 3) == 0) {
                        copy_scales(sa, scales + q * kScaleBytes);
                        copy_scales(sb, scales + q * kScaleBytes + kM * 4);
                    }
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks)                 // 32 along the contraction: 32 bytes, or 32 rows of 128 bytes
                        mma_block_scaled(tmem + buf * kN, a + (uint64_t)(ks * 32 >> 4), b + (uint64_t)((ACROSS ? ks * 4096 : ks * 32) >> 4), id,
                                         sa, sb, !begin || ks > 0);
                    tc_commit(smem_addr(&empty_bar[s]));
                    if (last) tc_commit(smem_addr(&sempty_bar[q]));
                    if (end) tc_commit(smem_addr(&tfull_bar[buf]));
                }
                __syncwarp();
                if (++s == kStages) s = 0, phase ^= 1;
                quads += last, acc += end;
            }
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
                if (quads >= 2 && !bar_wait_together(smem_addr(&sempty_bar[q]), ((quads >> 1) & 1) ^ 1, &failed)) { ok = false; break; }
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
        bool ok = true;
        for (int64_t tile = blockIdx.x; tile < total && ok; tile += gridDim.x) {
            int m, n;
            tile_of(tile, p.tiles_m, p.tiles_n, m, n);
            float v[kN];
#pragma unroll
            for (int c = 0; c < kN; ++c) v[c] = -0.0f;            // (leaves the sign of a zero as it is)
            for (int kb = 0; kb < blocks; kb += kFlushBlocks, ++acc) {
                const int buf = acc & 1;
                if (!bar_wait_together(smem_addr(&tfull_bar[buf]), (acc >> 1) & 1, &failed)) { ok = false; break; }
                tc_fence_after();
                const uint32_t at = tmem + buf * kN + ((uint32_t)(q * 32) << 16);
                add_columns(v, at, 0, [] {});
                tc_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(smem_addr(&tempty_bar[buf]));      // the accumulator may be overwritten
            }
            if (!ok) break;
            write_block<32>(p, v, 0, (int64_t)m * kM + q * 32, n, dyn_smem + (scales - smem_addr(dyn_smem)) + 2 * kScaleBytes + q * kPieceWarp);
        }
    }
    let_copies_land(&failed);
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && failed) atomicExch(p.errword, 1);
    if (warp == 3) tc_free(tmem, kTmemCols);
}

// ---- pairs of CTAs: tiles of 256 x 256 ------------------------------------------------------------------------------------
// (16384 x 4096 x 8192 to 8 bits: 406 us in a burst, 2708 TFLOP/s; 427 us in a row, where the power cap holds the clock down.)
// Each CTA loads 128 rows of A and half of B's 256, and the pair's tensor cores share them: 32 KB per CTA and block of 128
// along the contraction for twice the products of the single CTA's tile, half of what its loads cost (which bound it: at
// 128 x 128 every SM takes 128 bytes a clock from L2).
//
// Tensor memory: two accumulators of 256 columns and the scales do not fit 512 columns, so the second accumulator begins 24
// columns before the first one's end.  Whoever reads an accumulator begins with the 32 columns that hold the shared ones, and
// the MMAs into the other accumulator wait for that alone.
namespace pair {

constexpr int kHalf = 128, kTile = 256;
constexpr int kStageBytes = 2 * kHalf * kBlock;
constexpr int kStages = 6;
constexpr int kScaleBytes = (kHalf + kTile) * 4;                 // A: this CTA's rows; B: all of the tile's
constexpr int kStaged = 16;                                      // rows that a result warp stages at a time
constexpr int kPieceWarp = kStaged * kPiecePitch;
// At the start of a segment the tensor cores wait for the shared columns, some 800 cycles for the way there and back between the
// CTAs.  16384 x 4096 x 8192 with segments of 4, 8, 16 blocks and without an end: 471, 406, 385 and 372 us in a burst; 300, 360, 490
// and 710 of its 134 million codes are not those of a 64-bit result (of a product in fp32: 370).  So 8: the sums are as exact as an
// fp32 product's, however long.
constexpr int kFlushBlocks = 8;                                  // blocks that the tensor cores add up
constexpr int kSmemBytes = kStages * kStageBytes + 2 * kScaleBytes + 8 * kPieceWarp + 1024;
constexpr int kThreads = 384;                                    // warp 0: TMA, 1: MMA, 2: scales, 3: tensor memory, 4..11: results
constexpr int kScaleCols = (kHalf + kTile) / 32;
constexpr int kScaleCol = 512 - 2 * kScaleCols;
constexpr int kSecond = kScaleCol - kTile;                       // first column of the second accumulator
static_assert(kSecond >= kTile - 32, "the shared columns are among the last 32 of the first accumulator and the first 32 of the second");

__device__ __forceinline__ void mma_block_scaled(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, bool accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate ? 1u : 0u)
        : "memory");
}
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint32_t smem)      // in both CTAs, each from its own shared memory
{
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(tc_desc_copy(smem)) : "memory");
}

__device__ __forceinline__ void tile_at(int64_t t, const ProductArgs &p, int &m, int &n)
{
    const int64_t per = (int64_t)8 * p.tiles_n;
    const int g = (int)(t / per);
    const int tall = min(8, p.tiles_m - g * 8);
    const int r = (int)(t - g * per);
    m = g * 8 + r % tall;
    n = r / tall;
}

template <bool ACROSS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
product_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ ProductArgs p)
{
    extern __shared__ uint8_t dyn_smem[];
    // full, sfull, tempty, shared: CTA 0's count, for the pair; empty, sempty, tfull: arrive in both CTAs
    __shared__ __align__(8) uint64_t full_bar[kStages], empty_bar[kStages], sfull_bar[2], sempty_bar[2], tfull_bar[2], tempty_bar[2], shared_bar;
    __shared__ uint32_t tmem_base;
    __shared__ volatile int failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t tiles = (smem_addr(dyn_smem) + 1023u) & ~1023u;
    const uint32_t scales = tiles + kStages * kStageBytes;
    const int blocks = (int)((p.inner + kBlock - 1) / kBlock);
    const int64_t total = (int64_t)p.tiles_m * p.tiles_n;
    const uint32_t rank = cluster_rank();
    const int64_t first = blockIdx.x >> 1, step = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        failed = 0;
        for (int s = 0; s < kStages; ++s) {
            bar_init(smem_addr(&full_bar[s]), 1);
            bar_init(smem_addr(&empty_bar[s]), 1);
        }
        for (int s = 0; s < 2; ++s) {
            bar_init(smem_addr(&sfull_bar[s]), 2);
            bar_init(smem_addr(&sempty_bar[s]), 1);
            bar_init(smem_addr(&tfull_bar[s]), 1);
            bar_init(smem_addr(&tempty_bar[s]), 2 * 8);
        }
        bar_init(smem_addr(&shared_bar), 2 * 4);
        bar_init_fence();
    }
    if (warp == 3) tc_alloc_pair(&tmem_base, 512);
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem = tmem_base;

    // Registers: 128 threads of 88 and 256 of 208 are the 384 of 168 that the CTA was launched with.  (A row's sums, a piece that is
    // being added and one under way take 192.)
    if (warp >= 4) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        // a warp: 32 rows, half of the columns
        const int q = warp & 3, half = (warp - 4) >> 2, flip = 3 * half;
        uint8_t *stage = dyn_smem + (scales - smem_addr(dyn_smem)) + 2 * kScaleBytes + (warp - 4) * kPieceWarp;
        const uint32_t shared = cluster_addr(smem_addr(&shared_bar), 0);
        const uint32_t drained = cluster_addr(smem_addr(&tempty_bar[0]), 0);
        int acc = 0;
        bool ok = true;
        for (int64_t tile = first; tile < total && ok; tile += step) {
            int m, n;
            tile_at(tile, p, m, n);
            float v[kBlock];
#pragma unroll
            for (int c = 0; c < kBlock; ++c) v[c] = -0.0f;        // (leaves the sign of a zero as it is)
            for (int kb = 0; kb < blocks; kb += kFlushBlocks, ++acc) {
                const int buf = acc & 1;
                if (!bar_wait_together(smem_addr(&tfull_bar[buf]), (acc >> 1) & 1, &failed)) { ok = false; break; }
                tc_fence_after();
                const uint32_t at = tmem + (buf ? kSecond : 0) + half * kBlock + ((uint32_t)(q * 32) << 16);
                // from the side of the shared columns: the first accumulator's last piece, the second one's first
                add_columns(v, at, flip, [&] {
                    if (half == buf) return;
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive_cluster(shared);
                });
                tc_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive_cluster(drained + buf * 8);
            }
            if (!ok) break;
            write_block<kStaged>(p, v, flip, (int64_t)m * kTile + rank * kHalf + q * 32, (int64_t)n * 2 + half, stage);
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        if (threadIdx.x == 0) {
            int s = 0;
            uint32_t phase = 1;                                       // the first pass over the stages waits for nobody
            bool ok = true;
            for (int64_t tile = first; tile < total && ok; tile += step) {
                int m, n;
                tile_at(tile, p, m, n);
                const int arow = m * kTile + (int)rank * kHalf, brow = n * kTile + (int)rank * kHalf;
                for (int kb = 0; kb < blocks; ++kb) {
                    if (!bar_wait(smem_addr(&empty_bar[s]), phase, &failed)) { ok = false; break; }
                    const uint32_t st = tiles + s * kStageBytes, bar0 = cluster_addr(smem_addr(&full_bar[s]), 0);
                    if (rank == 0) bar_expect(smem_addr(&full_bar[s]), 2 * kStageBytes);
                    tma_load_pair(st, &map_a, bar0, kb * kBlock, arow);
                    if (ACROSS) tma_load_pair(st + kHalf * kBlock, &map_b, bar0, brow, kb * kBlock);
                    else tma_load_pair(st + kHalf * kBlock, &map_b, bar0, kb * kBlock, brow);
                    if (++s == kStages) s = 0, phase ^= 1;
                }
            }
        } else if (warp == 1) {
            constexpr uint32_t idesc = (ACROSS ? 1u << 16 : 0u) | (uint32_t)(kTile >> 3) << 17 | 1u << 23 | (uint32_t)(kTile >> 4) << 24;
            const bool issuer = elect_one();
            int s = 0, quads = 0, acc = 0;
            uint32_t phase = 0;
            bool ok = rank == 0;
            for (int64_t tile = first; tile < total && ok; tile += step) {
                for (int kb = 0; kb < blocks; ++kb) {
                    const int q = quads & 1, buf = acc & 1;
                    const bool begin = kb % kFlushBlocks == 0, end = kb % kFlushBlocks == kFlushBlocks - 1 || kb == blocks - 1;
                    const uint32_t d = tmem + (buf ? kSecond : 0);
                    const uint32_t sa = tmem + kScaleCol + q * kScaleCols, sb = sa + kHalf / 32;
                    if ((kb & 3) == 0) {
                        // full means that the set's last user has finished: its shared memory and its columns are free
                        if (!bar_wait_together(smem_addr(&sfull_bar[q]), (quads >> 1) & 1, &failed)) { ok = false; break; }
                        tc_fence_after();
                        if (issuer) {
                            const uint32_t at = scales + q * kScaleBytes;
                            copy_scales(sa, at);
                            copy_scales(sb, at + kHalf * 4);
                            copy_scales(sb + 4, at + kHalf * 8);
                        }
                        __syncwarp();
                    }
                    if (!bar_wait_together(smem_addr(&full_bar[s]), phase, &failed)) { ok = false; break; }
                    if (begin) {                                      // this accumulator's last use and, what is waited for longest, the shared columns
                        if (acc >= 2 && !bar_wait_together(smem_addr(&tempty_bar[buf]), ((acc >> 1) & 1) ^ 1, &failed)) { ok = false; break; }
                        if (acc >= 1 && !bar_wait_together(smem_addr(&shared_bar), (acc - 1) & 1, &failed)) { ok = false; break; }
                    }
                    tc_fence_after();
                    const uint32_t st = tiles + s * kStageBytes;
                    const uint32_t id = idesc | (uint32_t)(kb & 3) << 4 | (uint32_t)(kb & 3) << 29;    // which byte of the scale words
                    const uint64_t a = tc_desc_k(st), b = ACROSS ? tc_desc(st + kHalf * kBlock, kHalf * kBlock) : tc_desc_k(st + kHalf * kBlock);
                    const bool last = (kb & 3) == 3 || kb == blocks - 1;
                    if (issuer) {
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks)                 // 32 along the contraction: 32 bytes, or 32 rows of 128 bytes
                            mma_block_scaled(d, a + (uint64_t)(ks * 32 >> 4), b + (uint64_t)((ACROSS ? ks * 4096 : ks * 32) >> 4), id, sa, sb,
                                             !begin || ks > 0);
                        if (end) tc_commit_pair(smem_addr(&tfull_bar[buf]));
                        tc_commit_pair(smem_addr(&empty_bar[s]));
                        if (last) tc_commit_pair(smem_addr(&sempty_bar[q]));
                    }
                    __syncwarp();
                    if (++s == kStages) s = 0, phase ^= 1;
                    quads += last, acc += end;
                }
            }
        } else if (warp == 2) {
            // scale words of four blocks along the contraction: lane l serves rows l, l + 32, l + 64, l + 96 of a group of 128
            int quads = 0;
            bool ok = true;
            const uint32_t to = cluster_addr(smem_addr(&sfull_bar[0]), 0);
            for (int64_t tile = first; tile < total && ok; tile += step) {
                int m, n;
                tile_at(tile, p, m, n);
                for (int kb = 0; kb < blocks; kb += 4, ++quads) {
                    const int q = quads & 1;
                    uint32_t wa[4], wb[2] = {0, 0};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        int64_t r = (int64_t)m * kTile + rank * kHalf + 32 * j + lane;
                        if (r >= p.rows) r = p.rows - 1;               // (its codes arrive as zeros and its result is not written)
                        wa[j] = __ldg(reinterpret_cast<const uint32_t *>(p.a_scales + r * p.ld_as + kb));
                    }
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        const int64_t group = (int64_t)n * 2 + g;
                        if (group * kBlock >= p.cols) continue;        // (columns that are not written)
                        if (ACROSS) {
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                if (kb + j < blocks) wb[g] |= (uint32_t)__ldg(p.b_scales + (int64_t)(kb + j) * p.ld_bs + group) << (8 * j);
                        } else {
                            wb[g] = __ldg(reinterpret_cast<const uint32_t *>(p.b_scales + group * p.ld_bs + kb));
                        }
                    }
                    if (quads >= 2 && !bar_wait_together(smem_addr(&sempty_bar[q]), ((quads >> 1) & 1) ^ 1, &failed)) { ok = false; break; }
                    const uint32_t at = scales + q * kScaleBytes + lane * 16;
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(wa[0]), "r"(wa[1]), "r"(wa[2]), "r"(wa[3]) : "memory");
                    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at + kHalf * 4), "r"(wb[0]) : "memory");
                    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at + kHalf * 8), "r"(wb[1]) : "memory");
                    async_proxy_fence();
                    __syncwarp();
                    if (lane == 0) bar_arrive_cluster(to + q * 8);
                }
            }
        }
    }
    let_copies_land(&failed);
    tc_fence_before();
    __syncthreads();
    cluster_sync();                       // the other CTA's MMAs read this one's shared memory
    if (threadIdx.x == 0 && failed) atomicExch(p.errword, 1);
    if (warp == 3) tc_free_pair(tmem, 512);
}

}  // namespace pair

// ---- one row (decoding) ---------------------------------------------------------------------------------------------------
// The weights are read once and that is all the work there is, so the products run on the fp32 pipes and everything is
// spread over the machine: a cluster of eight CTAs makes 128 columns (a block of the 8-bit result), a warp two columns, its
// lanes 16 neighbouring codes of the contraction each.  A lane has 16 pieces of the weights under way before A's row is
// ready.  1 x 4096 x 4096: 9.5 us, 14 us on the tensor cores (whose 32 tiles keep 32 SMs busy); read across, or with two
// rows and more, the tensor cores are as fast or faster.
namespace one_row {

constexpr int kThreadsOne = 256, kCtas = 8, kCols = kBlock / kCtas;
constexpr int kMaxInner = 8192;                    // A's row lies in shared memory as fp32

__device__ __forceinline__ float cluster_float(const float *p, uint32_t rank)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(cluster_addr(smem_addr(p), rank)) : "memory");
    return v;
}

// Where a[k] lies: in the order in which lanes of 16 neighbours read it, 16 bytes at a time, without bank conflicts.
__device__ __forceinline__ int a_place(int k) { return k / 512 * 512 + (k % 16 / 4) * 128 + k % 512 / 16 * 4 + k % 4; }

__global__ void __cluster_dims__(kCtas, 1, 1) __launch_bounds__(kThreadsOne)
product_one_row_kernel(const uint8_t *__restrict__ a, const uint8_t *__restrict__ b, int64_t ld_b, const __grid_constant__ ProductArgs p)
{
    extern __shared__ float shared[];              // A's row, up to the next multiple of 512
    __shared__ float result[kCols], most_of;
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const int rank = (int)cluster_rank(), block = blockIdx.x / kCtas;
    const int inner = (int)p.inner, wide = (inner + 511) / 512 * 512;
    const int64_t col0 = (int64_t)block * kBlock;

    auto load_a = [&]() {
        for (int k = t * 16; k < wide; k += kThreadsOne * 16) {
            uint32_t q[4] = {0, 0, 0, 0};
            float f = 0.0f;
            if (k < inner) {
                load_codes16(a, k, inner, q);
                f = block_factor(__ldg(p.a_scales + k / kBlock));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v[4];
                codes_to_float4(q[i], v);
                *reinterpret_cast<float4 *>(shared + a_place(k + 4 * i)) =
                    make_float4(__fmul_rn(v[0], f), __fmul_rn(v[1], f), __fmul_rn(v[2], f), __fmul_rn(v[3], f));
            }
        }
        __syncthreads();
    };

    static_assert(kCols == 2 * kThreadsOne / 32, "a warp makes two columns");
    constexpr int kAhead = 8;                  // 16-byte pieces of each column that a lane has under way
    const int64_t n0 = col0 + rank * kCols + warp;
    float acc[2] = {0.0f, 0.0f};
#pragma unroll 1
    for (int u0 = 0; u0 * 512 < wide; u0 += kAhead) {
        uint32_t q[kAhead][2][4];
        float f[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int k = (u0 + u) * 512 + lane * 16;
            f[u] = 0.0f;
            if (k < inner) f[u] = block_factor(__ldg(p.b_scales + (int64_t)block * p.ld_bs + k / kBlock));
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                q[u][h][0] = q[u][h][1] = q[u][h][2] = q[u][h][3] = 0;
                if (n0 + h * (kCols / 2) < p.cols && k < inner) load_codes16(b + (n0 + h * (kCols / 2)) * ld_b, k, inner, q[u][h]);
            }
        }
        if (u0 == 0) load_a();
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if ((u0 + u) * 512 >= inner) break;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float w[2][4];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    codes_to_float4(q[u][h][i], w[h]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[h][j] = __fmul_rn(w[h][j], f[u]);    // (exact, and nothing overflows that the result would not)
                }
                const float4 x = *reinterpret_cast<const float4 *>(shared + (u0 + u) * 512 + i * 128 + lane * 4);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    acc[h] = __fmaf_rn(x.x, w[h][0], acc[h]);
                    acc[h] = __fmaf_rn(x.y, w[h][1], acc[h]);
                    acc[h] = __fmaf_rn(x.z, w[h][2], acc[h]);
                    acc[h] = __fmaf_rn(x.w, w[h][3], acc[h]);
                }
            }
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) acc[h] = __fadd_rn(acc[h], __shfl_xor_sync(0xffffffffu, acc[h], o));
        if (lane == 0) result[warp + h * (kCols / 2)] = acc[h];
    }
    __syncthreads();

    // a thread per entry
    const int64_t n = col0 + rank * kCols + t;
    float v = 0.0f;
    if (t < kCols) {
        v = p.slope != 1.0f ? leaky_slope(result[t], p.slope) : result[t];
        if (n < p.cols && p.y) {
            if (p.type == LGC_TYPE_FP32) static_cast<float *>(p.y)[n] = v;
            else static_cast<__nv_bfloat16 *>(p.y)[n] = __float2bfloat16_rn(v);
        }
    }
    if (p.codes) {                                 // (the same for every CTA)
        uint32_t m = t < kCols && n < p.cols ? __float_as_uint(v) & 0x7fffffffu : 0u;
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
        if (t == 0) most_of = __uint_as_float(m);
        __syncthreads();
        cluster_sync();
        if (t < kCols) {
            uint32_t most = 0;
            for (int i = 0; i < kCtas; ++i) most = max(most, __float_as_uint(cluster_float(&most_of, i)));
            const uint32_t s = block_scale(most);
            if (n < p.cols) p.codes[n] = (uint8_t)codes4(v, 0.0f, 0.0f, 0.0f, s);
            if (t == 0 && rank == 0) p.scales[block] = (uint8_t)s;
        }
    }
    cluster_sync();                                // the others may still read this CTA's shared memory
}

cudaError_t launch(const lgc_packed &a, const lgc_packed &b, const ProductArgs &p, cudaStream_t s)
{
    const int a_bytes = (int)((p.inner + 511) / 512 * 512) * 4;       // at most 32 KB
    product_one_row_kernel<<<(unsigned)((p.cols + kBlock - 1) / kBlock * kCtas), kThreadsOne, a_bytes, s>>>(a.codes, b.codes, b.ld, p);
    ++g_kernel_launches;
    return cudaGetLastError();
}

}  // namespace one_row

}  // namespace

cudaError_t launch_product(const lgc_packed &a, const lgc_packed &b, bool across, int64_t rows, int64_t cols, int64_t inner, float slope,
                           void *y, int32_t type, int64_t ldy, const lgc_packed *packed, int32_t *errword, cudaStream_t s)
{
    ProductArgs p{};
    p.a_scales = a.scales, p.b_scales = b.scales, p.ld_as = a.ld_scales, p.ld_bs = b.ld_scales;
    p.rows = rows, p.cols = cols, p.inner = inner, p.slope = slope;
    p.y = y, p.type = type, p.ldy = ldy, p.y_vec = matrix_rows_aligned(y, ldy, type == LGC_TYPE_FP32 ? 4 : 2);
    if (packed) p.codes = packed->codes, p.scales = packed->scales, p.ld_codes = packed->ld, p.ld_scales = packed->ld_scales;
    p.errword = errword;
    if (rows == 1 && !across && inner <= one_row::kMaxInner) return one_row::launch(a, b, p, s);
    CUtensorMap map_a, map_b;
    cudaError_t e = make_matrix_map(&map_a, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, a.codes, inner, rows, a.ld, kBlock, kM, CU_TENSOR_MAP_SWIZZLE_128B);
    if (e != cudaSuccess) return e;
    e = across ? make_matrix_map(&map_b, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, b.codes, cols, inner, b.ld, kN, kBlock, CU_TENSOR_MAP_SWIZZLE_128B)
               : make_matrix_map(&map_b, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, b.codes, inner, cols, b.ld, kBlock, kN, CU_TENSOR_MAP_SWIZZLE_128B);
    if (e != cudaSuccess) return e;
    // Pairs where their tiles give at least half of the SMs work (16384 x 4096 x 8192: half the time of single CTAs, whose loads
    // bound them); below that, more and smaller tiles.
    const int64_t big = ((rows + pair::kTile - 1) / pair::kTile) * ((cols + pair::kTile - 1) / pair::kTile), pairs = sm_count() / 2;
    const bool two = 2 * big >= pairs && rows > kM;
    static OncePerDevice configured;
    e = configured.run([&] {
        cudaError_t f = cudaFuncSetAttribute(product_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
        if (f == cudaSuccess) f = cudaFuncSetAttribute(product_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
        if (f == cudaSuccess) f = cudaFuncSetAttribute(pair::product_pair_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, pair::kSmemBytes);
        if (f == cudaSuccess) f = cudaFuncSetAttribute(pair::product_pair_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, pair::kSmemBytes);
        return f;
    });
    if (e != cudaSuccess) return e;
    if (two) {
        p.tiles_m = (int)((rows + pair::kTile - 1) / pair::kTile), p.tiles_n = (int)((cols + pair::kTile - 1) / pair::kTile);
        auto kern = across ? pair::product_pair_kernel<true> : pair::product_pair_kernel<false>;
        kern<<<(unsigned)(2 * (big < pairs ? big : pairs)), pair::kThreads, pair::kSmemBytes, s>>>(map_a, map_b, p);
    } else {
        p.tiles_m = (int)((rows + kM - 1) / kM), p.tiles_n = (int)((cols + kN - 1) / kN);
        const int64_t total = (int64_t)p.tiles_m * p.tiles_n;
        auto kern = across ? product_kernel<true> : product_kernel<false>;
        kern<<<(unsigned)(total < sm_count() ? total : sm_count()), kThreads, kSmemBytes, s>>>(map_a, map_b, p);
    }
    ++g_kernel_launches;
    return cudaGetLastError();
}

}  // namespace lgc
