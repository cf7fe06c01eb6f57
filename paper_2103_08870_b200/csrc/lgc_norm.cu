// Layer norm over the rows of a matrix, and its backward pass with the weight's and bias's gradients per node.
//
// Forward: a row stays in registers between its three uses (sum, sum of squared deviations, result), so x is read once
// and y (and / or its 8-bit form) written once.  The variance is the mean of the squared deviations from
// the mean that was found, not a difference of squares.
// Backward: dx needs two sums per row, the weight's gradient a sum over rows per column.  A CTA walks down a chunk of
// consecutive rows of one node; a thread keeps its columns' gradients in registers on the way, so dy and x are read once;
// the chunks' partial sums (fp32) are added up per node, in chunk order, by a second small kernel.
#include "lgc_layers.cuh"
#include "lgc_tensor_core.cuh"

namespace lgc {

namespace {

__device__ __forceinline__ float sum8(const float (&p)[8])
{
    return __fadd_rn(__fadd_rn(__fadd_rn(p[0], p[1]), __fadd_rn(p[2], p[3])), __fadd_rn(__fadd_rn(p[4], p[5]), __fadd_rn(p[6], p[7])));
}

// Sums over the TPR threads that share a row (a warp, or the whole CTA); every thread gets the result.
template <int TPR, int COUNT>
__device__ __forceinline__ void row_sums(float (&v)[COUNT], float *shared)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] = __fadd_rn(v[i], __shfl_xor_sync(0xffffffffu, v[i], o));
    if (TPR > 32) {
        constexpr int kWarps = TPR / 32;
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < COUNT; ++i) shared[i * kWarps + warp] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            float t = lane < kWarps ? shared[i * kWarps + lane] : 0.0f;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) t = __fadd_rn(t, __shfl_xor_sync(0xffffffffu, t, o));
            v[i] = t;
        }
    }
}

// Few rows (less than four per SM), or rows that start anywhere: a CTA of TPR threads per row, NV vectors of eight
// entries each.  Lanes hold neighbouring vectors, so that 16 lanes hold a block of the 8-bit form.  One row of 4096: 8 us
// from cold caches.
template <typename T, bool VEC, int TPR, int NV>
__global__ void __launch_bounds__(TPR)
layer_norm_kernel(const T *__restrict__ x, int64_t ldx, int cols, const float *__restrict__ gamma,
                  const float *__restrict__ beta, float eps, T *__restrict__ y, int64_t ldy, bool y_vec, uint8_t *__restrict__ codes,
                  int64_t ld_codes, uint8_t *__restrict__ scales, int64_t ld_scales, float *__restrict__ mean_out,
                  float *__restrict__ rstd_out, bool gb_vec)
{
    __shared__ float shared[2][TPR / 32];
    const int64_t row = blockIdx.x;
    const int t = threadIdx.x;
    const T *xr = x + row * ldx;
    float v[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) load8<T, VEC>(xr, (i * TPR + t) * 8, cols, v[i]);
    float part[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) part[j] = __fadd_rn(part[j], v[i][j]);
    float sum[1] = {sum8(part)};
    row_sums<TPR>(sum, shared[0]);
    const float mean = __fdiv_rn(sum[0], (float)cols);
#pragma unroll
    for (int j = 0; j < 8; ++j) part[j] = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = __fsub_rn(v[i][j], mean);
        if (c + 8 <= cols) {
#pragma unroll
            for (int j = 0; j < 8; ++j) part[j] = __fmaf_rn(v[i][j], v[i][j], part[j]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c + j < cols) part[j] = __fmaf_rn(v[i][j], v[i][j], part[j]);
        }
    }
    float sq[1] = {sum8(part)};
    row_sums<TPR>(sq, shared[1]);
    const float rstd = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(__fdiv_rn(sq[0], (float)cols), eps)));
    if (t == 0) {
        mean_out[row] = mean;
        rstd_out[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * 8;
        if ((i * TPR + (t & ~31)) * 8 >= cols) break;            // the whole warp is past the row's end
        float g[8], b[8];
        if (gb_vec) {
            load8<float, true>(gamma, c, cols, g);
            load8<float, true>(beta, c, cols, b);
        } else {
            load8<float, false>(gamma, c, cols, g);
            load8<float, false>(beta, c, cols, b);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = __fmaf_rn(__fmul_rn(v[i][j], rstd), g[j], b[j]);
        if (c + 8 > cols)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c + j >= cols) v[i][j] = 0.0f;
        if (y) {
            if (y_vec) store8<T, true>(y + row * ldy, c, cols, v[i]);
            else store8<T, false>(y + row * ldy, c, cols, v[i]);
        }
        if (codes) {
            const uint32_t s = block_scale(most_of_block(v[i]));
            store_codes8(codes + row * ld_codes, c, cols, codes4(v[i][0], v[i][1], v[i][2], v[i][3], s),
                         codes4(v[i][4], v[i][5], v[i][6], v[i][7], s));
            if ((t & 15) == 0 && c < cols) scales[row * ld_scales + c / kBlock] = (uint8_t)s;
        }
    }
}

// Takes away the compiler's knowledge of the entries: it would keep them as fp32 numbers from one use to the next, which
// costs twice the registers and half the warps.
template <typename T, int UNITS>
__device__ __forceinline__ void keep_raw(Raw16<T> (&raw)[UNITS])
{
    if (sizeof(T) == 2)
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
#pragma unroll
            for (int i = 0; i < (int)(4 * sizeof(T)); ++i) asm volatile("" : "+r"(raw[u].w[i]));
}

// Many rows: WPR warps per row, walking from row to row.  The row stays as it was loaded (bf16: half the registers of fp32
// numbers), UNITS times 16 neighbouring entries per lane; gamma and beta lie in shared memory in the order in which lanes
// read them, one 16-byte piece per lane without bank conflicts.  16384 x 4096 bf16 to 8 bits: 59 us, 3.4 TB/s.  Nothing is full
// (issue slots 63 %, DRAM 35 %): a row's chain of load, two exchanges among its warps and store is long, and 32 warps per SM
// do not cover it; of the time between two instructions of a warp a quarter is waiting for the row's loads and a fifth for shuffles and
// shared memory.  One warp a row is slower (76 us), and the next row's loads, ahead in registers or in shared memory, gained
// nothing (61 and 73 us).
constexpr int kRowThreads = 256;

// A sum over the WPR warps of a row; the groups of a CTA have a named barrier each.
template <int WPR>
__device__ __forceinline__ float group_sum(const f2 (&p)[4], float *shared)
{
    const f2 t = f2_add(f2_add(p[0], p[1]), f2_add(p[2], p[3]));
    float v = __fadd_rn(f2_lo(t), f2_hi(t));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = __fadd_rn(v, __shfl_xor_sync(0xffffffffu, v, o));
    if (WPR > 1) {
        const int warp = threadIdx.x >> 5, group = warp / WPR;
        if ((threadIdx.x & 31) == 0) shared[warp] = v;
        asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(32 * WPR) : "memory");
        v = shared[group * WPR];
#pragma unroll
        for (int i = 1; i < WPR; ++i) v = __fadd_rn(v, shared[group * WPR + i]);
    }
    return v;
}

template <typename T, int UNITS>
constexpr int row_ctas()                 // CTAs per SM that the registers of a lane's raw entries and about 40 more allow
{
    constexpr int raw = 4 * UNITS * (int)sizeof(T);
    return raw <= 16 ? 4 : raw <= 32 ? 3 : raw <= 64 ? 2 : 1;
}
template <typename T, int AL, int YAL, int UNITS, int WPR>
__global__ void __launch_bounds__(kRowThreads, row_ctas<T, UNITS>())
layer_norm_rows_kernel(const T *__restrict__ x, int64_t ldx, int64_t rows, int cols, const float *__restrict__ gamma,
                       const float *__restrict__ beta, float eps, T *__restrict__ y, int64_t ldy, uint8_t *__restrict__ codes,
                       int64_t ld_codes, uint8_t *__restrict__ scales, int64_t ld_scales, float *__restrict__ mean_out,
                       float *__restrict__ rstd_out)
{
    extern __shared__ float4 gb[];                               // [gamma, beta][unit][piece][thread of the row]
    __shared__ float shared[2][kRowThreads / 32];
    constexpr int TPR = 32 * WPR, kWide = TPR * 16;              // threads of a row, entries of a unit
    const int t = threadIdx.x % TPR;
    for (int i = threadIdx.x; i < 2 * UNITS * kWide; i += kRowThreads) {
        const int c = i % (UNITS * kWide), unit = c / kWide, l = c % kWide / 16, piece = c % 16 / 4;
        const float *from = i < UNITS * kWide ? gamma : beta;
        reinterpret_cast<float *>(gb)[((i / (UNITS * kWide) * UNITS + unit) * 4 + piece) * TPR * 4 + l * 4 + c % 4] = c < cols ? __ldg(from + c) : 0.0f;
    }
    __syncthreads();
    const float inverse = __fdiv_rn(1.0f, (float)cols);
    constexpr int kGroups = kRowThreads / TPR;
    for (int64_t row = (int64_t)blockIdx.x * kGroups + threadIdx.x / TPR; row < rows; row += (int64_t)gridDim.x * kGroups) {
        const T *xr = x + row * ldx;
        Raw16<T> raw[UNITS];
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
            if (u * kWide < cols) load16<AL>(xr, u * kWide + t * 16, cols, raw[u]);
        f2 part[4] = {0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
            if (u * kWide < cols)
#pragma unroll
                for (int i = 0; i < 8; ++i) part[i & 3] = f2_add(part[i & 3], raw_pair(raw[u], i));
        const float mean = __fmul_rn(group_sum<WPR>(part, shared[0]), inverse);
        const f2 minus = f2_of(-mean, -mean);
        keep_raw(raw);
        part[0] = part[1] = part[2] = part[3] = 0;
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            if (u * kWide + ((t | 31) + 1) * 16 <= cols) {        // (the same for a warp)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const f2 d = f2_add(raw_pair(raw[u], i), minus);
                    part[i & 3] = f2_fma(d, d, part[i & 3]);
                }
            } else if (u * kWide < cols) {
                const int c = u * kWide + t * 16;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    f2 d = f2_add(raw_pair(raw[u], i), minus);
                    d = f2_of(c + 2 * i < cols ? f2_lo(d) : 0.0f, c + 2 * i + 1 < cols ? f2_hi(d) : 0.0f);
                    part[i & 3] = f2_fma(d, d, part[i & 3]);
                }
            }
        }
        const float rstd = __frsqrt_rn(__fmaf_rn(group_sum<WPR>(part, shared[1]), inverse, eps));
        if (t == 0) {
            mean_out[row] = mean;
            rstd_out[row] = rstd;
        }
        const f2 rr = f2_of(rstd, rstd);
        keep_raw(raw);
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const int c = u * kWide + t * 16;
            if (u * kWide + (t & ~31) * 16 >= cols) break;        // the whole warp is past the row's end
            const bool full = u * kWide + ((t | 31) + 1) * 16 <= cols;
            f2 v[8];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float4 g = gb[(u * 4 + k) * TPR + t], b = gb[((UNITS + u) * 4 + k) * TPR + t];
                v[2 * k] = f2_fma(f2_mul(f2_add(raw_pair(raw[u], 2 * k), minus), rr), f2_of(g.x, g.y), f2_of(b.x, b.y));
                v[2 * k + 1] = f2_fma(f2_mul(f2_add(raw_pair(raw[u], 2 * k + 1), minus), rr), f2_of(g.z, g.w), f2_of(b.z, b.w));
            }
            if (!full)                                            // (gamma = beta = 0 there, but rstd may be infinite or NaN)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = f2_of(c + 2 * i < cols ? f2_lo(v[i]) : 0.0f, c + 2 * i + 1 < cols ? f2_hi(v[i]) : 0.0f);
            const int upto = full ? c + 16 : cols;                // (a whole unit: no checks)
            if (y) store16<YAL>(y + row * ldy, c, upto, v);
            if (codes) {
                uint32_t q[4];
                const uint32_t s = codes16(v, q);
                store_codes16(codes + row * ld_codes, c, upto, q);
                if ((t & 7) == 0 && c < cols) scales[row * ld_scales + c / kBlock] = (uint8_t)s;
            }
        }
    }
}

// ---- backward ---------------------------------------------------------------------------------------------------------
// Chunk `want` of the nodes' rows, each node's rows cut into chunks of `chunk_rows`: its rows and its node.  After the last
// node's come the rows in front of the first node's run (as node `nodes`) and behind the last one's (`nodes` + 1), which have a
// dx like all others and no part in any node's sums.  Called by a whole warp; 32 nodes at a time.
struct Chunk {
    int64_t begin, end;
    int node;
};
__device__ __forceinline__ Chunk find_chunk(const int64_t *start, int nodes, int64_t rows, int64_t chunk_rows, int64_t want)
{
    const int lane = threadIdx.x & 31;
    for (int k0 = 0; k0 < nodes + 2; k0 += 32) {
        const int k = k0 + lane;
        // (both loads at once, whatever the lane: one latency in front of the CTA's work, not two)
        int64_t lo = node_first_row(start, min(k, nodes), rows), hi = node_first_row(start, k < nodes ? k + 1 : 0, rows);
        if (k == nodes) lo = 0;
        if (k > nodes) hi = k == nodes + 1 ? rows : lo;
        if (hi < lo) hi = lo;
        const int64_t mine = (hi - lo + chunk_rows - 1) / chunk_rows;
        int64_t upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t t = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += t;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, want < upto);
        if (hit) {
            const int src = __ffs(hit) - 1;
            const int64_t before = __shfl_sync(0xffffffffu, upto - mine, src);
            const int64_t l = __shfl_sync(0xffffffffu, lo, src), h = __shfl_sync(0xffffffffu, hi, src);
            const int64_t b = l + (want - before) * chunk_rows;
            return {b, b + chunk_rows < h ? b + chunk_rows : h, k0 + src};
        }
        want -= __shfl_sync(0xffffffffu, upto, 31);
    }
    return {0, 0, -1};
}

// Eight neighbouring entries of a row in shared memory, c a multiple of 8; what lies beyond the row's end reads as zero.
// whole: known to lie inside the row.
template <typename T>
__device__ __forceinline__ void slot8(const T *row, int c, int cols, bool whole, f2 (&v)[4])
{
    if (!whole && c >= cols) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = 0;
        return;
    }
    if constexpr (sizeof(T) == 1) {
        const uint2 q = *reinterpret_cast<const uint2 *>(row + c);
        float a[4], b[4];
        codes_to_float4(q.x, a);
        codes_to_float4(q.y, b);
        v[0] = f2_of(a[0], a[1]), v[1] = f2_of(a[2], a[3]), v[2] = f2_of(b[0], b[1]), v[3] = f2_of(b[2], b[3]);
    } else if constexpr (sizeof(T) == 2) {
        const uint4 q = *reinterpret_cast<const uint4 *>(row + c);
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = f2_of(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u));
    } else {
        const ulonglong2 a = *reinterpret_cast<const ulonglong2 *>(row + c), b = *reinterpret_cast<const ulonglong2 *>(row + c + 4);
        v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y;
    }
    if (!whole && c + 8 > cols)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = f2_of(c + 2 * j < cols ? f2_lo(v[j]) : 0.0f, c + 2 * j + 1 < cols ? f2_hi(v[j]) : 0.0f);
}

// x may be the 8-bit checkpoint (XT = uint8_t).
template <typename XT>
__device__ __forceinline__ void load_x8(const XT *x, int64_t ldx, const uint8_t *scales, int64_t ld_scales, int64_t row, int64_t c,
                                        int64_t cols, float (&v)[8])
{
    if constexpr (sizeof(XT) == 1) {
        const uint2 q = load_codes8(x + row * ldx, c, cols);
        const float f = c < cols ? block_factor(__ldg(scales + row * ld_scales + c / kBlock)) : 0.0f;
        float a[4], b[4];
        codes_to_float4(q.x, a);
        codes_to_float4(q.y, b);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = __fmul_rn(a[j], f);
            v[4 + j] = __fmul_rn(b[j], f);
        }
    } else {
        load8<XT, false>(x + row * ldx, c, cols, v);
    }
}

// partial: [chunks][2][cols], the weight's then the bias's gradient over the chunk's rows.
template <typename T, typename XT, int TPR, int NV>
__global__ void __launch_bounds__(TPR)
layer_norm_backward_kernel(const T *__restrict__ dy, int64_t ld_dy, const XT *__restrict__ x, int64_t ldx,
                           const uint8_t *__restrict__ x_scales, int64_t ld_scales, int64_t rows, int64_t cols,
                           const float *__restrict__ gamma, const float *__restrict__ mean, const float *__restrict__ rstd,
                           const int64_t *__restrict__ node_start, int nodes, int64_t chunk_rows, T *__restrict__ dx, int64_t ld_dx,
                           float *__restrict__ partial)
{
    __shared__ float shared[2][2 * (TPR / 32)];
    const int t = threadIdx.x;
    const int number = gridDim.x - 1 - blockIdx.x;               // (the first CTAs are those that may find no chunk: see max_chunks_for)
    const Chunk ch = find_chunk(node_start, nodes, rows, chunk_rows, number);
    if (ch.node < 0) return;
    float g[NV][8], dg[NV][8], db[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        load8<float, false>(gamma, (int64_t)(i * TPR + t) * 8, cols, g[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) dg[i][j] = db[i][j] = 0.0f;
    }
    const float count = (float)cols;
    for (int64_t row = ch.begin; row < ch.end; ++row) {
        float d[NV][8], h[NV][8];
        float sums[2] = {0.0f, 0.0f};
        const float mu = __ldg(mean + row), rs = __ldg(rstd + row);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t c = (int64_t)(i * TPR + t) * 8;
            load8<T, false>(dy + row * ld_dy, c, cols, d[i]);
            load_x8<XT>(x, ldx, x_scales, ld_scales, row, c, cols, h[i]);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                // entries beyond the row's end: d = g = 0, and their xh enters no sum
                h[i][j] = __fmul_rn(__fsub_rn(h[i][j], mu), rs);
                dg[i][j] = __fmaf_rn(d[i][j], h[i][j], dg[i][j]);
                db[i][j] = __fadd_rn(db[i][j], d[i][j]);
                d[i][j] = __fmul_rn(d[i][j], g[i][j]);
                sums[0] = __fadd_rn(sums[0], d[i][j]);
                sums[1] = __fmaf_rn(d[i][j], h[i][j], sums[1]);
            }
        row_sums<TPR>(sums, shared[row & 1]);                    // two sets: a fast warp may be a row ahead of a slow one
        const float m1 = __fdiv_rn(sums[0], count), m2 = __fdiv_rn(sums[1], count);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int j = 0; j < 8; ++j) d[i][j] = __fmul_rn(rs, __fsub_rn(__fsub_rn(d[i][j], m1), __fmul_rn(h[i][j], m2)));
            store8<T, false>(dx + row * ld_dx, (int64_t)(i * TPR + t) * 8, cols, d[i]);
        }
    }
    float *out = partial + (int64_t)number * 2 * cols;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        store8<float, false>(out, (int64_t)(i * TPR + t) * 8, cols, dg[i]);
        store8<float, false>(out + cols, (int64_t)(i * TPR + t) * 8, cols, db[i]);
    }
}

// The same for rows that start on 16-byte boundaries: whole rows of dy and x (and the 8-bit form's scales) come into a ring
// of shared-memory slots by bulk copies, so that the loads of the rows to come are always under way, whatever the registers
// hold (16384 x 4096 bf16, x in 8 bits: 100 us against 196 with plain loads; issue slots 44 %, DRAM 37 %: the 16 warps of an SM
// wait for one another at a barrier per row, and for the shuffles and shared-memory reads around it).  The barrier in the middle of a row's work says that every warp has read its slot, which a warp (another one each
// row) then gives to a row to come.  A thread owns NV vectors of 8 neighbouring columns.  A row's last bytes that do not
// fill 16 come in words of four, the last of them perhaps in part.
template <typename T, typename XT, int THREADS, int NV>
__global__ void __launch_bounds__(THREADS, (NV == 1 ? 1024 : 512) / THREADS)
layer_norm_backward_ring_kernel(const T *__restrict__ dy, int64_t ld_dy, const XT *__restrict__ x, int64_t ldx,
                                const uint8_t *__restrict__ x_scales, int64_t ld_scales, int64_t rows, int cols,
                                const float *__restrict__ gamma, const float *__restrict__ mean, const float *__restrict__ rstd,
                                const int64_t *__restrict__ node_start, int nodes, int64_t chunk_rows, T *__restrict__ dx, int64_t ld_dx,
                                float *__restrict__ partial, bool dx_vec, int slots, int slot_bytes, int32_t *__restrict__ errword)
{
    extern __shared__ __align__(16) uint8_t ring[];
    constexpr int kWarps = THREADS / 32, kMaxSlots = 8;
    __shared__ __align__(8) uint64_t full_bar[kMaxSlots];
    __shared__ float2 sums_of[2][kWarps];
    __shared__ __align__(16) T stage[kWarps][256];
    __shared__ volatile int failed;
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
    grid_release_dependents();                                   // the kernel that adds up the chunks waits for this one's end
    const int number = gridDim.x - 1 - blockIdx.x;               // (the first CTAs are those that may find no chunk: see max_chunks_for)
    const Chunk ch = find_chunk(node_start, nodes, rows, chunk_rows, number);
    if (ch.node < 0) return;
    if (t == 0) {
        failed = 0;
        for (int s = 0; s < slots; ++s) bar_init(smem_addr(&full_bar[s]), 1 + 32);
        bar_init_fence();
    }
    __syncthreads();
    // a slot: dy's row, x's row (each from a 16-byte boundary), then mean, rstd and the scale words
    const uint32_t dy_bytes = cols * (uint32_t)sizeof(T), x_bytes = cols * (uint32_t)sizeof(XT);
    const uint32_t x_at = (dy_bytes + 15u) & ~15u, more_at = x_at + ((x_bytes + 15u) & ~15u);
    const float inverse = __fdiv_rn(1.0f, (float)cols);
    const int count = (int)(ch.end - ch.begin);

    auto load_row = [&](int k, int s) {                          // by a whole warp
        const int64_t row = ch.begin + k;
        const uint32_t slot = smem_addr(ring) + s * slot_bytes, bar = smem_addr(&full_bar[s]);
        const uint8_t *d = reinterpret_cast<const uint8_t *>(dy + row * ld_dy), *xr = reinterpret_cast<const uint8_t *>(x + row * ldx);
        const uint32_t d16 = dy_bytes & ~15u, x16 = x_bytes & ~15u, words = lane * 4;
        if (lane == 0) {
            bar_expect(bar, d16 + x16);
            if (d16) bulk_load(slot, d, d16, bar);
            if (x16) bulk_load(slot + x_at, xr, x16, bar);
        }
        // at most four words; of the last one only what belongs to the row
        if (d16 + words < dy_bytes) word_load(slot + d16 + words, d + d16 + words, sizeof(T) == 4 ? 4u : 2u + (d16 + words + 2 < dy_bytes) * 2u);
        if (x16 + words < x_bytes)
            word_load(slot + x_at + x16 + words, xr + x16 + words,
                      sizeof(XT) == 4 ? 4u : sizeof(XT) == 2 ? 2u + (x16 + words + 2 < x_bytes) * 2u : min(4u, x_bytes - x16 - words));
        if (lane == 8) word_load(slot + more_at, mean + row);
        if (lane == 9) word_load(slot + more_at + 4, rstd + row);
        if (sizeof(XT) == 1 && lane < (cols + 4 * kBlock - 1) / (4 * kBlock))            // (at most 16 words: 8192 columns)
            word_load(slot + more_at + 8 + words, x_scales + row * ld_scales + words);
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
    };
    for (int k = warp; k < slots && k < count; k += kWarps) load_row(k, k);

    {
        f2 g[NV][4], dg[NV][4], db[NV][4];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float w[8];
            load8<float, false>(gamma, (int64_t)(i * THREADS + t) * 8, cols, w);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                g[i][j] = f2_of(w[2 * j], w[2 * j + 1]);
                dg[i][j] = db[i][j] = 0;
            }
        }
        int s = 0;
        uint32_t phase = 0, set = 0;
        int issuer = 0;                                          // the warp that loads into this row's slot
        T *to = dx + ch.begin * ld_dx;
        for (int k = 0; k < count; ++k, to += ld_dx, s = s + 1 == slots ? 0 : s + 1, phase ^= s == 0, set ^= 1) {
            // a wait that runs out is recorded; the warps stay together, and this one loads nothing more (a slot's barrier may still
            // count the copies of the row that it waited for)
            if (!bar_wait(smem_addr(&full_bar[s]), phase, &failed)) issuer = kWarps;
            __syncwarp();
            const uint8_t *slot = ring + s * slot_bytes;
            const float *more = reinterpret_cast<const float *>(slot + more_at);
            const float mu = more[0], rs = more[1];
            f2 d[NV][4], h[NV][4];
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (i * THREADS + t) * 8;
                const bool whole = (i * THREADS + (t | 31) + 1) * 8 <= cols;    // (the same for a warp)
                slot8(reinterpret_cast<const T *>(slot), c, cols, whole, d[i]);
                slot8(reinterpret_cast<const XT *>(slot + x_at), c, cols, whole, h[i]);
                if (sizeof(XT) == 1) {
                    const float f = whole || c < cols ? block_factor(reinterpret_cast<const uint8_t *>(more + 2)[c / kBlock]) : 0.0f;
#pragma unroll
                    for (int j = 0; j < 4; ++j) h[i][j] = f2_fma(h[i][j], f2_of(f, f), f2_of(-mu, -mu));      // (the product is exact)
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) h[i][j] = f2_add(h[i][j], f2_of(-mu, -mu));
                }
            }
            f2 s0 = 0, s1 = 0;
            const f2 rr = f2_of(rs, rs);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    // entries beyond the row's end: d = 0, and their xh enters no sum
                    h[i][j] = f2_mul(h[i][j], rr);
                    dg[i][j] = f2_fma(d[i][j], h[i][j], dg[i][j]);
                    db[i][j] = f2_add(db[i][j], d[i][j]);
                    d[i][j] = f2_mul(d[i][j], g[i][j]);
                    s0 = f2_add(s0, d[i][j]);
                    s1 = f2_fma(d[i][j], h[i][j], s1);
                }
            float sums[2] = {__fadd_rn(f2_lo(s0), f2_hi(s0)), __fadd_rn(f2_lo(s1), f2_hi(s1))};
            row_sums<32>(sums, nullptr);
            if (kWarps > 1) {
                float2 *part = sums_of[set];                  // two sets: a fast warp may be a row ahead of a slow one
                if (lane == 0) part[warp] = make_float2(sums[0], sums[1]);
                asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory");
                f2 total = reinterpret_cast<const f2 *>(part)[0];
#pragma unroll
                for (int i = 1; i < kWarps; ++i) total = f2_add(total, reinterpret_cast<const f2 *>(part)[i]);
                sums[0] = f2_lo(total), sums[1] = f2_hi(total);
            }
            if (warp == issuer && k + slots < count) load_row(k + slots, s);     // (one warp: row_sums' shuffles are its barrier)
            issuer = issuer + 1 == kWarps ? 0 : issuer + 1;
            const float m1 = __fmul_rn(sums[0], -inverse), m2 = __fmul_rn(sums[1], -inverse);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (i * THREADS + t) * 8;
#pragma unroll
                for (int j = 0; j < 4; ++j) d[i][j] = f2_mul(rr, f2_fma(h[i][j], f2_of(m2, m2), f2_add(d[i][j], f2_of(m1, m1))));
                const float w[8] = {f2_lo(d[i][0]), f2_hi(d[i][0]), f2_lo(d[i][1]), f2_hi(d[i][1]),
                                    f2_lo(d[i][2]), f2_hi(d[i][2]), f2_lo(d[i][3]), f2_hi(d[i][3])};
                if (dx_vec) {
                    store8<T, true>(to, c, (i * THREADS + (t | 31) + 1) * 8 <= cols ? c + 8 : cols, w);
                } else {                                          // rows that start anywhere: neighbouring lanes write neighbours
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < 8; ++j) stage[warp][lane * 8 + j] = (T)w[j];
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int at = (i * THREADS + warp * 32) * 8 + j * 32 + lane;
                        if (at < cols) to[at] = stage[warp][j * 32 + lane];
                    }
                }
            }
        }
        float *out = partial + (int64_t)number * 2 * cols;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * THREADS + t) * 8;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (c + 2 * j < cols) out[c + 2 * j] = f2_lo(dg[i][j]), out[cols + c + 2 * j] = f2_lo(db[i][j]);
                if (c + 2 * j + 1 < cols) out[c + 2 * j + 1] = f2_hi(dg[i][j]), out[cols + c + 2 * j + 1] = f2_hi(db[i][j]);
            }
        }
        let_copies_land(&failed);
        if (t == 0 && failed) atomicExch(errword, 3);
    }
}

// The chunks' sums of one node, 32 columns per CTA: 8 slices of the chunks side by side, each in chunk order, then the
// slices in order.
__global__ void __launch_bounds__(256)
layer_norm_gradient_kernel(const float *__restrict__ partial, int64_t rows, int64_t cols, const int64_t *__restrict__ node_start,
                           int64_t chunk_rows, int64_t max_chunks, float *__restrict__ dgamma, float *__restrict__ dbeta,
                           int64_t node_stride)
{
    __shared__ float part[2][8][33];
    const int node = blockIdx.y, lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
    // this node's chunks: those of the nodes in front come first
    int64_t first = 0;
    for (int k0 = 0; k0 < node; k0 += 32) {
        const int k = k0 + lane;
        int64_t mine = 0;
        if (k < node) {
            const int64_t lo = node_first_row(node_start, k, rows), hi = node_first_row(node_start, k + 1, rows);
            mine = hi > lo ? (hi - lo + chunk_rows - 1) / chunk_rows : 0;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
        first += mine;
    }
    const int64_t lo = node_first_row(node_start, node, rows), hi = node_first_row(node_start, node + 1, rows);
    int64_t count = hi > lo ? (hi - lo + chunk_rows - 1) / chunk_rows : 0;
    if (first + count > max_chunks) count = first < max_chunks ? max_chunks - first : 0;   // (only if node_start does not ascend)
    grid_wait();                                                 // the chunks' sums come from the launch in front
    const int64_t each = (count + 7) / 8;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    float g = 0.0f, b = 0.0f;
    if (c < cols) {
        const int64_t end = (slice + 1) * each < count ? (slice + 1) * each : count;
#pragma unroll 8
        for (int64_t i = slice * each; i < end; ++i) {
            const float *p = partial + (first + i) * 2 * cols + c;
            g = __fadd_rn(g, __ldcg(p));                          // (not __ldg: they are written while this kernel is under way)
            b = __fadd_rn(b, __ldcg(p + cols));
        }
    }
    part[0][slice][lane] = g;
    part[1][slice][lane] = b;
    __syncthreads();
    if (slice < 2 && c < cols) {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) t = __fadd_rn(t, part[slice][i][lane]);
        (slice == 0 ? dgamma : dbeta)[(int64_t)node * node_stride + c] = t;
    }
}

// Rows per chunk, at least four: as many chunks as there is room for CTAs at a time (one per SM for rows of more than 4096, two
// from 2049 on, up to sixteen for narrow ones), the nodes' rounding included, since a chunk too many costs a second round of CTAs.
// (The ring's slots leave no room for the last of them at about 470 to 510 columns, and of fp32 at about 990 to 1020: there 16384
// rows do take a second round.)  The chunks' 2 * cols partial sums stay small beside their rows.
int64_t chunk_rows_for(int64_t rows, int64_t cols, int32_t nodes)
{
    const int64_t per_sm = cols > 4096 ? 1 : cols > 2048 ? 2 : cols > 1024 ? 4 : cols > 512 ? 8 : 16;
    const int64_t room = per_sm * 148 - nodes, r = (rows + (room < 148 ? 148 : room) - 1) / (room < 148 ? 148 : room);
    return r < 4 ? 4 : r;
}
// Every run of rows, the two of no node among them, may end in part of a chunk.  The CTAs that find no chunk come first and
// make room at once: behind the others, one that found no room would hold up the launch of the kernel that adds up the chunks.
int64_t max_chunks_for(int64_t rows, int64_t cols, int32_t nodes)
{
    return rows / chunk_rows_for(rows, cols, nodes) + nodes + 2;
}

struct ForwardArgs {
    const Matrix &x;
    int64_t rows, cols;
    const float *gamma, *beta;
    float eps;
    void *y;
    int64_t ldy;
    const lgc_packed *p;
    float *mean, *rstd;
    cudaStream_t s;
};

template <typename T, bool VEC>
void forward_shared_rows(const ForwardArgs &a)
{
    const bool y_vec = matrix_rows_aligned(a.y, a.ldy, sizeof(T)), gb_vec = matrix_rows_aligned(a.gamma, 4, 4) && matrix_rows_aligned(a.beta, 4, 4);
    auto launch = [&](auto kern, int64_t ctas, int threads) {
        kern<<<(unsigned)ctas, threads, 0, a.s>>>(static_cast<const T *>(a.x.p), a.x.ld, (int)a.cols, a.gamma, a.beta, a.eps,
                                                  static_cast<T *>(a.y), a.ldy, y_vec, a.p ? a.p->codes : nullptr, a.p ? a.p->ld : 0,
                                                  a.p ? a.p->scales : nullptr, a.p ? a.p->ld_scales : 0, a.mean, a.rstd, gb_vec);
    };
    if (a.cols <= 1024) launch(layer_norm_kernel<T, VEC, 128, 1>, a.rows, 128);
    else if (a.cols <= 4096) launch(layer_norm_kernel<T, VEC, 128, 4>, a.rows, 128);
    else if (a.cols <= 8192) launch(layer_norm_kernel<T, VEC, 256, 4>, a.rows, 256);
    else launch(layer_norm_kernel<T, VEC, 512, 4>, a.rows, 512);
}

template <typename T, int AL, int YAL, int UNITS, int WPR>
cudaError_t forward_rows(const ForwardArgs &a)
{
    auto kern = layer_norm_rows_kernel<T, AL, YAL, UNITS, WPR>;
    constexpr int kSmem = 2 * UNITS * WPR * 512 * 4, kGroups = kRowThreads / 32 / WPR;
    static OncePerDevice configured;
    if (kSmem > 48 * 1024) {
        const cudaError_t e = configured.run([&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem); });
        if (e != cudaSuccess) return e;
    }
    const int64_t need = (a.rows + kGroups - 1) / kGroups, most = (int64_t)row_ctas<T, UNITS>() * sm_count();
    kern<<<(unsigned)(need < most ? need : most), kRowThreads, kSmem, a.s>>>(
        static_cast<const T *>(a.x.p), a.x.ld, a.rows, (int)a.cols, a.gamma, a.beta, a.eps, static_cast<T *>(a.y), a.ldy, a.p ? a.p->codes : nullptr,
        a.p ? a.p->ld : 0, a.p ? a.p->scales : nullptr, a.p ? a.p->ld_scales : 0, a.mean, a.rstd);
    return cudaSuccess;
}

template <typename T, int AL, int YAL>
cudaError_t forward_units(const ForwardArgs &a)
{
    if (a.cols <= 512) return forward_rows<T, AL, YAL, 1, 1>(a);
    if (a.cols <= 1024) return forward_rows<T, AL, YAL, 2, 1>(a);
    if (a.cols <= 2048) return forward_rows<T, AL, YAL, 1, 4>(a);
    if (a.cols <= 4096) return forward_rows<T, AL, YAL, 2, 4>(a);
    if (a.cols <= 8192) return forward_rows<T, AL, YAL, 4, 4>(a);
    return forward_rows<T, AL, YAL, 8, 4>(a);
}

template <typename T>
cudaError_t forward_type(const ForwardArgs &a)
{
    const int al = matrix_alignment(a.x.p, a.x.ld, sizeof(T)), yal = a.y ? matrix_alignment(a.y, a.ldy, sizeof(T)) : 32;
    cudaError_t e = cudaSuccess;
    if (al >= 16 && a.rows >= 4 * sm_count()) e = al == 32 && yal == 32 ? forward_units<T, 32, 32>(a) : forward_units<T, 16, 0>(a);
    else if (al >= 16) forward_shared_rows<T, true>(a);
    else forward_shared_rows<T, false>(a);
    ++g_kernel_launches;
    return e != cudaSuccess ? e : cudaGetLastError();
}

struct BackwardArgs {
    const Matrix &dy, &x;
    const lgc_packed *xp;
    int64_t rows, cols;
    const float *gamma, *mean, *rstd;
    const int64_t *node_start;
    int32_t nodes;
    void *dx;
    int64_t ld_dx;
    float *partial;
    int32_t *errword;
    cudaStream_t s;
};

// Rows that start anywhere, or wider than the ring kernel's threads can own (beyond 8192 columns 1024 threads of 64 registers
// spill up to 256 bytes each).
template <typename T, typename XT>
void backward_any(const BackwardArgs &a)
{
    const int64_t chunk = chunk_rows_for(a.rows, a.cols, a.nodes), ctas = max_chunks_for(a.rows, a.cols, a.nodes);
    auto launch = [&](auto kern, int threads) {
        kern<<<(unsigned)ctas, threads, 0, a.s>>>(static_cast<const T *>(a.dy.p), a.dy.ld,
                                                  static_cast<const XT *>(a.xp ? a.xp->codes : a.x.p), a.xp ? a.xp->ld : a.x.ld,
                                                  a.xp ? a.xp->scales : nullptr, a.xp ? a.xp->ld_scales : 0, a.rows, a.cols, a.gamma, a.mean,
                                                  a.rstd, a.node_start, a.nodes, chunk, static_cast<T *>(a.dx), a.ld_dx, a.partial);
    };
    if (a.cols <= 2048) launch(layer_norm_backward_kernel<T, XT, 128, 2>, 128);
    else if (a.cols <= 8192) launch(layer_norm_backward_kernel<T, XT, 512, 2>, 512);
    else launch(layer_norm_backward_kernel<T, XT, 1024, 2>, 1024);
}

template <typename T, typename XT, int THREADS, int NV>
cudaError_t backward_ring(const BackwardArgs &a)
{
    auto kern = layer_norm_backward_ring_kernel<T, XT, THREADS, NV>;
    const int64_t cols = a.cols;
    const int slot = (int)((cols * sizeof(T) + 15) / 16 * 16 + (cols * sizeof(XT) + 15) / 16 * 16 +
                           (8 + (sizeof(XT) == 1 ? (cols + 511) / 512 * 4 : 0) + 15) / 16 * 16);
    constexpr int kMost = 192 * 1024;
    // as many slots as leave room for the CTAs that the registers allow (narrow rows: more CTAs count for more than more slots)
    constexpr int kCtas = (NV == 1 ? 1024 : 512) / THREADS;
    int slots = kMost / kCtas / slot;
    if (slots < 2) slots = kMost / slot;
    slots = slots > 8 ? 8 : slots < 2 ? 2 : slots;
    static OncePerDevice configured;
    const cudaError_t e = configured.run([&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost); });
    if (e != cudaSuccess) return e;
    kern<<<(unsigned)max_chunks_for(a.rows, cols, a.nodes), THREADS, (size_t)slots * slot, a.s>>>(
        static_cast<const T *>(a.dy.p), a.dy.ld, static_cast<const XT *>(a.xp ? a.xp->codes : a.x.p), a.xp ? a.xp->ld : a.x.ld,
        a.xp ? a.xp->scales : nullptr, a.xp ? a.xp->ld_scales : 0, a.rows, (int)cols, a.gamma, a.mean, a.rstd, a.node_start, a.nodes,
        chunk_rows_for(a.rows, cols, a.nodes), static_cast<T *>(a.dx), a.ld_dx, a.partial, matrix_rows_aligned(a.dx, a.ld_dx, sizeof(T)), slots, slot, a.errword);
    return cudaSuccess;
}
template <typename T, typename XT>
cudaError_t backward_aligned(const BackwardArgs &a)
{
    const bool vec = matrix_rows_aligned(a.dy.p, a.dy.ld, sizeof(T)) && (sizeof(XT) == 1 || matrix_rows_aligned(a.x.p, a.x.ld, sizeof(XT)));
    if (!vec || a.cols > 8192) {
        backward_any<T, XT>(a);
        return cudaSuccess;
    }
    if (a.cols <= 512) return backward_ring<T, XT, 64, 1>(a);
    if (a.cols <= 1024) return backward_ring<T, XT, 128, 1>(a);
    if (a.cols <= 2048) return backward_ring<T, XT, 256, 1>(a);
    if (a.cols <= 4096) return backward_ring<T, XT, 256, 2>(a);
    return backward_ring<T, XT, 512, 2>(a);
}
template <typename T>
cudaError_t backward_type(const BackwardArgs &a)
{
    if (a.xp) return backward_aligned<T, uint8_t>(a);
    return a.x.type == LGC_TYPE_FP32 ? backward_aligned<T, float>(a) : backward_aligned<T, __nv_bfloat16>(a);
}

}  // namespace

cudaError_t launch_layer_norm(const Matrix &x, int64_t rows, int64_t cols, const float *gamma, const float *beta, float eps, void *y,
                              int64_t ldy, const lgc_packed *packed, float *mean, float *rstd, cudaStream_t s)
{
    const ForwardArgs a{x, rows, cols, gamma, beta, eps, y, ldy, packed, mean, rstd, s};
    return x.type == LGC_TYPE_FP32 ? forward_type<float>(a) : forward_type<__nv_bfloat16>(a);
}

size_t layer_norm_backward_scratch(int64_t rows, int64_t cols, int32_t num_nodes)
{
    return (size_t)max_chunks_for(rows, cols, num_nodes) * 2 * (size_t)cols * sizeof(float);
}

cudaError_t launch_layer_norm_backward(const Matrix &dy, const Matrix &x, const lgc_packed *x_packed, int64_t rows, int64_t cols,
                                       const float *gamma, const float *mean, const float *rstd, const int64_t *node_start,
                                       int32_t num_nodes, void *dx, int64_t ld_dx, float *dgamma, float *dbeta, int64_t node_stride,
                                       void *scratch, int32_t *errword, cudaStream_t s)
{
    const BackwardArgs a{dy, x, x_packed, rows, cols, gamma, mean, rstd, node_start, num_nodes, dx, ld_dx, static_cast<float *>(scratch),
                         errword, s};
    if (rows > 0) {
        cudaError_t e = dy.type == LGC_TYPE_FP32 ? backward_type<float>(a) : backward_type<__nv_bfloat16>(a);
        ++g_kernel_launches;
        if (e == cudaSuccess) e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    const cudaError_t e = launch_dependent(layer_norm_gradient_kernel, dim3((unsigned)((cols + 31) / 32), (unsigned)num_nodes), dim3(256), s, a.partial,
                                           rows, cols, node_start, chunk_rows_for(rows, cols, num_nodes), max_chunks_for(rows, cols, num_nodes),
                                           dgamma, dbeta, node_stride);
    if (e != cudaSuccess) return e;
    ++g_kernel_launches;
    return cudaGetLastError();
}

}  // namespace lgc
