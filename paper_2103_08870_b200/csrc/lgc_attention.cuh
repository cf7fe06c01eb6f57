// What attention's kernels share: the runs of rows, the units of work, tiles in shared memory.
//
// A tile of queries is 128 rows: kRows / group queries of every head that shares a head of k and v (row = query * group + head),
// so that a key is read once for all of them, a masked diagonal tile wastes few queries, and a sum over a tile's rows is
// already the sum over the heads that dk and dv want.  What a group that does not divide 128 leaves of the rows is not used.
#pragma once

#include "lgc_layers.cuh"
#include "lgc_tensor_core.cuh"

namespace lgc {
namespace attention {

constexpr int kRows = 128;             // rows of a tile of queries, keys of a tile of keys
constexpr int kPiece = kRows * 128;    // bytes of 64 columns of a tile: rows of 128 bytes, 128-byte swizzle
constexpr int kMostDim = 128;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Where a sequence's queries and keys lie; start == nullptr: one sequence with every row.
struct Runs {
    const int64_t *query_start, *key_start;
    int sequences;
    int64_t query_rows, key_rows;
};

// A run of queries, or of keys, of one sequence, and the sequence's rows on the other side.
struct __align__(16) Unit {
    int row, rows;             // first row, number of rows
    int pos;                   // of the first row in its sequence
    int other_row, other_len;  // the sequence's keys, or queries
    int shift;                 // number of keys - number of queries: causal: query i sees keys up to i + shift
    int pad[2];
};

struct Mask {
    int causal;
    int window;                // 0: none
};

// The units' table in scratch memory (where the runs are given): their number, then the units, those with most to do first.
struct Plan {
    int *count;
    Unit *units;
    int *prefix;               // [sequences + 1] units in front of a sequence's
    int per;                   // rows of a unit
    int64_t most;              // units that there is room for, and CTAs per head
};

inline int64_t most_units(const int64_t *start, int64_t rows, int per, int sequences) { return start ? rows / per + sequences : (rows + per - 1) / per; }
inline size_t plan_bytes(const int64_t *start, int64_t rows, int per, int sequences)
{
    return start ? 16 + (size_t)most_units(start, rows, per, sequences) * sizeof(Unit) + ((size_t)sequences + 1 + 3) / 4 * 16 : 0;
}
inline Plan plan_at(char *p, const int64_t *start, int64_t rows, int per, int sequences)
{
    const int64_t most = most_units(start, rows, per, sequences);
    Unit *units = reinterpret_cast<Unit *>(p + 16);
    return Plan{reinterpret_cast<int *>(p), units, reinterpret_cast<int *>(units + most), per, most};
}

// Writes the table of the queries' units and / or the keys' (nullptr: not wanted).
cudaError_t launch_plan(const Runs &runs, const Mask &mask, const Plan *queries, const Plan *keys, cudaStream_t s);

// The unit of a CTA; units with more to do come first (causal: the last queries, the first keys).  False: there is none.
__device__ __forceinline__ bool unit_of(const Runs &r, const Plan &plan, bool by_key, int64_t index, Unit &u)
{
    if (r.query_start) {
        if (index >= *plan.count) return false;
        u = plan.units[index];
        return true;
    }
    const int64_t rows = by_key ? r.key_rows : r.query_rows;
    if (index >= plan.most) return false;
    if (!by_key) index = plan.most - 1 - index;
    u.row = u.pos = (int)(index * plan.per);
    u.rows = (int)min((int64_t)plan.per, rows - index * plan.per);
    u.other_row = 0;
    u.other_len = (int)(by_key ? r.query_rows : r.key_rows);
    u.shift = (int)(r.key_rows - r.query_rows);
    return true;
}

// Keys [lo, hi) of the sequence that some of the queries pos .. pos + rows - 1 see.
__device__ __forceinline__ void keys_seen(const Mask &m, int pos, int rows, int shift, int keys, int &lo, int &hi)
{
    lo = 0;
    hi = keys;
    if (m.causal) {
        hi = min(keys, pos + rows + shift);
        if (m.window) lo = max(0, pos + shift - m.window + 1);
    }
    if (rows <= 0 || hi <= lo) lo = hi = 0;
}
// Queries [lo, hi) of the sequence that see some of the keys pos .. pos + rows - 1.
__device__ __forceinline__ void queries_seeing(const Mask &m, int pos, int rows, int shift, int queries, int &lo, int &hi)
{
    lo = 0;
    hi = queries;
    if (m.causal) {
        lo = max(0, pos - shift);
        if (m.window) hi = (int)min((int64_t)queries, (int64_t)pos + rows - 1 + m.window - shift);
    }
    if (rows <= 0 || hi <= lo) lo = hi = 0;
}

// Rows from `row` on of a tile of DP columns become zero: they belong to another sequence, and zero times what they hold might not
// be zero.  By a whole warp, in front of the products that sum over the rows.
template <int DP>
__device__ __forceinline__ void clear_rows(uint32_t tile, int row)
{
    const int lane = threadIdx.x & 31;
    for (int r = row + (lane >> 3); r < kRows; r += 4)
#pragma unroll
        for (int j = 0; j < DP / 64; ++j)
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(tile + j * kPiece + r * 128 + (lane & 7) * 16), "r"(0) : "memory");
    async_proxy_fence();
    __syncwarp();
}

// fp32 sums of bf16 products; M = 128 rows, N columns; b_rows: B lies with the summed index along its rows
__device__ __forceinline__ constexpr uint32_t idesc_of(int n, bool b_rows)
{
    return 1u << 4 | 1u << 7 | 1u << 10 | (b_rows ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 | (uint32_t)(kRows >> 4) << 24;
}
// D = A B^T over DP columns of two tiles in shared memory (128 x 128 results).
template <int DP>
__device__ __forceinline__ void product_of_tiles(uint32_t d, uint32_t a, uint32_t b)
{
    const uint64_t da = tc_desc_k(a), db = tc_desc_k(b);
#pragma unroll
    for (int ks = 0; ks < DP / 16; ++ks) {
        const uint64_t at = (uint64_t)((ks / 4 * kPiece + ks % 4 * 32) >> 4);
        tc_mma(d, da + at, db + at, idesc_of(kRows, false), ks > 0);
    }
}
// D (+)= A B: A 128 x 16 entries in tensor memory per step, B the 16 rows of a tile from `step` on.
template <int DP>
__device__ __forceinline__ void product_step(uint32_t d, uint32_t a, uint32_t b, int step, bool accumulate)
{
    tc_mma_tmem(d, a, tc_desc(b + step * 2048, kPiece), idesc_of(DP, true), accumulate);
}
template <int DP>
__device__ __forceinline__ void load_tile(uint32_t tile, const CUtensorMap *map, uint32_t bar, int head, int row)
{
#pragma unroll
    for (int j = 0; j < DP / 64; ++j) tma_load_heads(tile + j * kPiece, map, bar, 64 * j, head, row);
}
// By every warp of a group of four: gives back, or takes, registers of the block's launch (waits until there are as many).
template <int N>
__device__ __forceinline__ void give_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }

__device__ __forceinline__ float exp2_of(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Eight neighbours of a row as bf16; rows start 16-byte aligned.
__device__ __forceinline__ void store_bf16x8(__nv_bfloat16 *at, const float *v)
{
    *reinterpret_cast<uint4 *>(at) = make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
}

}  // namespace attention

// A [rows][heads][dim] operand as the C ABI gives it, with the strides that one row or one head may leave open filled in.
struct Heads {
    void *p;
    int64_t ld, head_stride;
};
struct AttentionShape {
    int64_t query_rows, key_rows;
    int heads, kv_heads, dim;
    const int64_t *query_start, *key_start;
    int sequences;
    int causal, window;
    float scale;
};
size_t attention_scratch(const AttentionShape &a);
size_t attention_backward_scratch(const AttentionShape &a);
bool attention_grid_fits(const AttentionShape &a);
cudaError_t launch_attention(const AttentionShape &a, const Heads &q, const Heads &k, const Heads &v, const Heads &y, float *lse, void *scratch,
                             int32_t *errword, cudaStream_t s);
cudaError_t launch_attention_backward(const AttentionShape &a, const Heads &dy, const Heads &q, const Heads &k, const Heads &v, const Heads &y,
                                      const float *lse, const Heads &dq, const Heads &dk, const Heads &dv, void *scratch, int32_t *errword,
                                      cudaStream_t s);
cudaError_t launch_rotary(const void *x, int32_t type, int64_t rows, int heads, int dim, int64_t ldx, int64_t head_stride_x, const int64_t *positions,
                          const double *frequencies, int pairs, bool interleaved, float amplitude, bool backward, void *y, int64_t ldy,
                          int64_t head_stride_y, cudaStream_t s);

}  // namespace lgc
