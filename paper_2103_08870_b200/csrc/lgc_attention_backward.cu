// Attention over sequences, backward: the probabilities are made again from q, k and lse, p = exp(scale q k^T - lse); then
//     dv = p^T dy,   ds = p (dy v^T - delta),   dq = scale ds k,   dk = scale ds^T q,   delta = sum(dy y) per row and head.
//
// Two kernels, so that every sum is taken on chip, in a fixed order, by one CTA: the first goes over the keys for a tile of queries
// (dq; three products a pair of tiles), the second over the queries for a tile of keys (dk and dv; four products).  One kernel
// with five products would have to add its parts of dq up in memory: in an order that changes, or as T / 128 copies.
// delta and lse (in powers of two) are left by the first kernel for the second, which reads them for every tile.
//
// P and dS never leave the SM's tensor memory: eight warps read S and dP there (a lane per row of the tile, half of the columns to
// each group of four), and write P and dS back as bf16 operands of the next product.  The other operands are tiles in
// shared memory, read along or across their rows as the product wants.  In the second kernel the keys are the lanes (S^T = K Q^T), so
// P^T and dS^T are such operands too.
//
// Precision: sums are fp32; P and dS are rounded to bf16 as operands; delta is a sum of bf16 products in fp32.
#include "lgc_attention.cuh"

namespace lgc {

using namespace attention;

namespace {

constexpr int kThreads = 384;           // warps 0..7: P and dS, 8: MMA, 9: TMA, 10 and 11 only give registers
constexpr int kRowRegisters = 208, kOtherRegisters = 88;      // 2 * 208 + 88 = 3 * 168 at the launch

struct BackwardArgs {
    Runs runs;
    Plan plan;
    Mask mask;
    int heads, kv_heads, group, dim;
    int queries;                        // of a tile
    float scale, scale_log2;            // scale_log2 = scale * log2(e)
    const __nv_bfloat16 *dy, *y;
    int64_t ld_dy, head_stride_dy, ld_y, head_stride_y;
    const float *lse;
    __nv_bfloat16 *dq, *dk, *dv;
    int64_t ld_dq, head_stride_dq, ld_dk, head_stride_dk, ld_dv, head_stride_dv;
    float *minus_lse2, *delta;          // [kv_heads][query rows][group]: -lse * log2(e), delta
    int32_t *errword;
};

template <int DP>
constexpr int kTileBytes = DP / 64 * kPiece;

// 32 columns times `by` to a row of bf16.
__device__ __forceinline__ void store_columns(__nv_bfloat16 *out, int column, int dim, uint32_t taddr, float by, bool live, bool any)
{
    uint32_t o[32];
    tc_read32(taddr, o);
    tc_read_wait(o);
#pragma unroll
    for (int n = 0; n < 32; n += 8)
        if (live && column + n < dim) {
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = any ? __fmul_rn(__uint_as_float(o[n + e]), by) : 0.0f;
            store_bf16x8(out + column + n, f);
        }
}

// ---- dq: a tile of queries goes over its keys --------------------------------------------------------------------------------
// Tensor memory: S of two tiles of keys in turn (columns 0 and 128; dS takes its place), dP (256), dQ (384).
// The tensor cores' order: dP(t + 1) once dP(t) has been read, dQ += dS(t) K(t), S(t + 2): the threads find the next S ready.
constexpr int kKeyStages = 3, kValueStages = 2;
template <int DP>
constexpr int kQuerySmem = (2 + kKeyStages + kValueStages) * kTileBytes<DP> + 1024;

template <int DP>
__global__ void __launch_bounds__(kThreads, 1)
attention_dq_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                    const __grid_constant__ CUtensorMap map_dy, const __grid_constant__ BackwardArgs p)
{
    constexpr int kTile = kTileBytes<DP>;
    extern __shared__ uint8_t dyn_smem[];
    __shared__ __align__(8) uint64_t q_full, k_full[kKeyStages], k_empty[kKeyStages], v_full[kValueStages], v_empty[kValueStages], s_full[2], dp_full,
        dp_taken, ds_full, done;
    __shared__ float delta_half[2][kRows];
    __shared__ uint32_t tmem_base;
    __shared__ volatile int failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t base = (smem_addr(dyn_smem) + 1023u) & ~1023u;
    const uint32_t q_tile = base, dy_tile = base + kTile, k_ring = base + 2 * kTile, v_ring = k_ring + kKeyStages * kTile;

    if (threadIdx.x == 0) {
        failed = 0;
        bar_init(smem_addr(&q_full), 1);
        for (int s = 0; s < kKeyStages; ++s) bar_init(smem_addr(&k_full[s]), 1), bar_init(smem_addr(&k_empty[s]), 1);
        for (int s = 0; s < kValueStages; ++s) bar_init(smem_addr(&v_full[s]), 1), bar_init(smem_addr(&v_empty[s]), 1);
        for (int s = 0; s < 2; ++s) bar_init(smem_addr(&s_full[s]), 1);
        bar_init(smem_addr(&dp_full), 1);
        bar_init(smem_addr(&dp_taken), 8);
        bar_init(smem_addr(&ds_full), 8);
        bar_init(smem_addr(&done), 1);
        bar_init_fence();
    }
    if (warp == 8) tc_alloc(&tmem_base, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base;
    grid_wait();
    const int kv_head = (int)(blockIdx.x % p.kv_heads), head0 = kv_head * p.group;
    Unit u;
    const bool any = unit_of(p.runs, p.plan, false, blockIdx.x / p.kv_heads, u);
    int key_lo = 0, key_hi = 0;
    if (any) keys_seen(p.mask, u.pos, u.rows, u.shift, u.other_len, key_lo, key_hi);
    const int tiles = (key_hi - key_lo + kRows - 1) / kRows;

    if (!any) {
    } else if (warp >= 8) {
        give_registers<kOtherRegisters>();
        if (warp == 9) {
            if (lane == 0 && tiles > 0) {
                const uint32_t q_bytes = (uint32_t)p.queries * p.group * (DP * 2);
                bar_expect(smem_addr(&q_full), 2 * q_bytes);
                load_tile<DP>(q_tile, &map_q, smem_addr(&q_full), head0, u.row);
                load_tile<DP>(dy_tile, &map_dy, smem_addr(&q_full), head0, u.row);
                int sk = 0, sv = 0;
                uint32_t ph_k = 1, ph_v = 1;
                for (int t = 0; t < tiles; ++t) {
                    const int row = u.other_row + key_lo + t * kRows;
                    if (!bar_wait(smem_addr(&k_empty[sk]), ph_k, &failed)) break;
                    bar_expect(smem_addr(&k_full[sk]), kTile);
                    load_tile<DP>(k_ring + sk * kTile, &map_k, smem_addr(&k_full[sk]), kv_head, row);
                    if (!bar_wait(smem_addr(&v_empty[sv]), ph_v, &failed)) break;
                    bar_expect(smem_addr(&v_full[sv]), kTile);
                    load_tile<DP>(v_ring + sv * kTile, &map_v, smem_addr(&v_full[sv]), kv_head, row);
                    if (++sk == kKeyStages) sk = 0, ph_k ^= 1;
                    if (++sv == kValueStages) sv = 0, ph_v ^= 1;
                }
            }
        } else if (warp == 8 && tiles > 0) {
            const bool issuer = elect_one();
            int sk = 0, sd = 0, sv = 0;                       // stages of S's K, of dQ's K, of V
            uint32_t ph_k = 0, ph_v = 0;
            // S(t): waits for K(t); its rows behind the sequence become zero, since dQ sums over them
            const auto make_s = [&](int t) {
                if (!bar_wait_together(smem_addr(&k_full[sk]), ph_k, &failed)) return false;
                const uint32_t tile = k_ring + sk * kTile;
                const int live = u.other_len - (key_lo + t * kRows);
                if (live < kRows) clear_rows<DP>(tile, live);
                tc_fence_after();
                if (issuer) {
                    product_of_tiles<DP>(tmem + (t & 1) * kRows, q_tile, tile);
                    tc_commit(smem_addr(&s_full[t & 1]));
                }
                __syncwarp();
                if (++sk == kKeyStages) sk = 0, ph_k ^= 1;
                return true;
            };
            const auto make_dp = [&]() {
                if (!bar_wait_together(smem_addr(&v_full[sv]), ph_v, &failed)) return false;
                tc_fence_after();
                if (issuer) {
                    product_of_tiles<DP>(tmem + 256, dy_tile, v_ring + sv * kTile);
                    tc_commit(smem_addr(&dp_full));
                    tc_commit(smem_addr(&v_empty[sv]));
                }
                __syncwarp();
                if (++sv == kValueStages) sv = 0, ph_v ^= 1;
                return true;
            };
            bool ok = bar_wait_together(smem_addr(&q_full), 0, &failed) && make_s(0) && make_dp() && (tiles < 2 || make_s(1));
            for (int t = 0; t < tiles && ok; ++t) {
                if (t + 1 < tiles && !(bar_wait_together(smem_addr(&dp_taken), t & 1, &failed) && make_dp())) break;
                if (!bar_wait_together(smem_addr(&ds_full), t & 1, &failed)) break;
                tc_fence_after();
                if (issuer) {
#pragma unroll
                    for (int ks = 0; ks < kRows / 16; ++ks)
                        product_step<DP>(tmem + 384, tmem + (t & 1) * kRows + ks / 4 * 64 + ks % 4 * 8, k_ring + sd * kTile, ks, t > 0 || ks > 0);
                    tc_commit(smem_addr(&k_empty[sd]));
                    if (t == tiles - 1) tc_commit(smem_addr(&done));
                }
                __syncwarp();
                if (++sd == kKeyStages) sd = 0;
                if (t + 2 < tiles && !make_s(t + 2)) break;      // (after the product that reads dS in the same columns)
            }
        }
    } else {
        take_registers<kRowRegisters>();
        const int half = warp >> 2;                              // of the columns
        const int row = (warp & 3) * 32 + lane;                  // of the tile
        const int query = row / p.group, head = head0 + row - query * p.group;
        const bool live = query < p.queries && query < u.rows;
        const int64_t q = (int64_t)u.row + query;
        int lo = 0, hi = 0x7fffffff;                             // (rows that nobody reads need no mask)
        if (live) keys_seen(p.mask, u.pos + query, 1, u.shift, u.other_len, lo, hi);
        // delta, half of the columns to each group of warps
        float part = 0.0f, minus_lse2 = 0.0f;
        if (live) {
            const __nv_bfloat16 *a = p.dy + q * p.ld_dy + head * p.head_stride_dy, *b = p.y + q * p.ld_y + head * p.head_stride_y;
            float sums[4] = {};
#pragma unroll 4
            for (int j = half * (DP / 2); j < (half + 1) * (DP / 2); j += 8)
                if (j < p.dim) {
                    float x[8], z[8];
                    load8<__nv_bfloat16, true>(a, j, p.dim, x);
                    load8<__nv_bfloat16, true>(b, j, p.dim, z);
#pragma unroll
                    for (int n = 0; n < 8; ++n) sums[n & 3] = __fmaf_rn(x[n], z[n], sums[n & 3]);
                }
            part = __fadd_rn(__fadd_rn(sums[0], sums[1]), __fadd_rn(sums[2], sums[3]));
            const float lse = p.lse[q * p.heads + head];
            minus_lse2 = lse == -INFINITY ? 0.0f : -__fmul_rn(lse, kLog2e);
        }
        delta_half[half][row] = part;
        asm volatile("bar.sync 1, 256;" ::: "memory");
        const float delta = __fadd_rn(delta_half[0][row], delta_half[1][row]);
        if (live && half == 0) {
            const int64_t at = ((int64_t)kv_head * p.runs.query_rows + u.row) * p.group + row;
            p.minus_lse2[at] = minus_lse2;
            p.delta[at] = delta;
        }
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const f2 cc = f2_of(p.scale_log2, p.scale_log2), mm = f2_of(minus_lse2, minus_lse2), dd = f2_of(-delta, -delta);
        bool ok = true;
        for (int t = 0; t < tiles; ++t) {
            const uint32_t s_at = tmem + lanes + (t & 1) * kRows + half * 64;
            if (!bar_wait_together(smem_addr(&s_full[t & 1]), (t >> 1) & 1, &failed)) { ok = false; break; }
            tc_fence_after();
            float v[64];
#pragma unroll
            for (int j = 0; j < 2; ++j) tc_read32(s_at + 32 * j, reinterpret_cast<uint32_t(&)[32]>(v[32 * j]));
#pragma unroll
            for (int j = 0; j < 2; ++j) tc_read_wait(reinterpret_cast<uint32_t(&)[32]>(v[32 * j]));
#pragma unroll
            for (int n = 0; n < 64; n += 2) {
                const f2 x = f2_fma(f2_of(v[n], v[n + 1]), cc, mm);
                v[n] = exp2_of(f2_lo(x));
                v[n + 1] = exp2_of(f2_hi(x));
            }
            if (!bar_wait_together(smem_addr(&dp_full), t & 1, &failed)) { ok = false; break; }
            tc_fence_after();
            float d[64];
#pragma unroll
            for (int j = 0; j < 2; ++j) tc_read32(tmem + lanes + 256 + half * 64 + 32 * j, reinterpret_cast<uint32_t(&)[32]>(d[32 * j]));
#pragma unroll
            for (int j = 0; j < 2; ++j) tc_read_wait(reinterpret_cast<uint32_t(&)[32]>(d[32 * j]));
            tc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(smem_addr(&dp_taken));
#pragma unroll
            for (int n = 0; n < 64; n += 2) {
                const f2 x = f2_mul(f2_of(v[n], v[n + 1]), f2_add(f2_of(d[n], d[n + 1]), dd));
                v[n] = f2_lo(x);
                v[n + 1] = f2_hi(x);
            }
            const int key0 = key_lo + t * kRows + half * 64, from = lo - key0, to = hi - key0;
            if (__any_sync(0xffffffffu, from > 0 || to < 64)) {
#pragma unroll
                for (int n = 0; n < 64; ++n) v[n] = n >= from && n < to ? v[n] : 0.0f;
            }
            uint32_t w[32];
#pragma unroll
            for (int n = 0; n < 64; n += 2) w[n >> 1] = bf16_pair(v[n], v[n + 1]);
            tc_write32(s_at, w);
            tc_write_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(smem_addr(&ds_full));
        }
        if (ok && tiles > 0 && !bar_wait_together(smem_addr(&done), 0, &failed)) ok = false;
        if (ok) {
            tc_fence_after();
            __nv_bfloat16 *out = p.dq + q * p.ld_dq + head * p.head_stride_dq;
#pragma unroll
            for (int j = 0; j < DP / 2; j += 32) {
                const int column = half * (DP / 2) + j;
                store_columns(out, column, p.dim, tmem + lanes + 384 + column, p.scale, live, tiles > 0);
            }
        }
    }
    let_copies_land(&failed);
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && failed) atomicExch(p.errword, 2);
    if (warp == 8) tc_free(tmem, 512);
}

// ---- dk and dv: a tile of keys goes over the queries that see it -----------------------------------------------------------------
// Tensor memory: S^T (columns 0; P^T takes its place), dP^T (128; dS^T takes its place), dV (256), dK (256 + DP).
// The tensor cores' order: dV += P(t) dY(t), S(t + 1), dK += dS(t) Q(t), dP(t + 1): while the threads are at P they have dK and dP
// to do, while they are at dS, dV and the next S.
constexpr int kPairStages = 2;          // of Q and dY
template <int DP>
constexpr int kKeySmem = (2 + 2 * kPairStages) * kTileBytes<DP> + kPairStages * kRows * 8 + 1024;

template <int DP>
__global__ void __launch_bounds__(kThreads, 1)
attention_dkv_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                     const __grid_constant__ CUtensorMap map_dy, const __grid_constant__ BackwardArgs p)
{
    constexpr int kTile = kTileBytes<DP>;
    extern __shared__ uint8_t dyn_smem[];
    __shared__ __align__(8) uint64_t kv_full, q_full[kPairStages], q_empty[kPairStages], dy_full[kPairStages], dy_empty[kPairStages],
        row_full[kPairStages], s_full, p_full, dp_full, ds_full, done;
    __shared__ uint32_t tmem_base;
    __shared__ volatile int failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t base = (smem_addr(dyn_smem) + 1023u) & ~1023u;
    const uint32_t k_tile = base, v_tile = base + kTile, q_ring = base + 2 * kTile, dy_ring = q_ring + kPairStages * kTile,
                   rows_at = dy_ring + kPairStages * kTile;       // [stage][-lse2 of 128 rows, delta of 128 rows]

    if (threadIdx.x == 0) {
        failed = 0;
        bar_init(smem_addr(&kv_full), 1);
        for (int s = 0; s < kPairStages; ++s) {
            bar_init(smem_addr(&q_full[s]), 1), bar_init(smem_addr(&q_empty[s]), 1);
            bar_init(smem_addr(&dy_full[s]), 1), bar_init(smem_addr(&dy_empty[s]), 1);
            bar_init(smem_addr(&row_full[s]), 1);
        }
        bar_init(smem_addr(&s_full), 1);
        bar_init(smem_addr(&p_full), 8);
        bar_init(smem_addr(&dp_full), 1);
        bar_init(smem_addr(&ds_full), 8);
        bar_init(smem_addr(&done), 1);
        bar_init_fence();
    }
    if (warp == 8) tc_alloc(&tmem_base, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base;
    grid_wait();
    const int kv_head = (int)(blockIdx.x % p.kv_heads), head0 = kv_head * p.group;
    Unit u;
    const bool any = unit_of(p.runs, p.plan, true, blockIdx.x / p.kv_heads, u);
    int query_lo = 0, query_hi = 0;
    if (any) queries_seeing(p.mask, u.pos, u.rows, u.shift, u.other_len, query_lo, query_hi);
    const int tiles = (query_hi - query_lo + p.queries - 1) / p.queries;

    if (!any) {
    } else if (warp >= 8) {
        give_registers<kOtherRegisters>();
        if (warp == 9) {
            const uint32_t q_bytes = (uint32_t)p.queries * p.group * (DP * 2);
            if (lane == 0 && tiles > 0) {
                bar_expect(smem_addr(&kv_full), 2 * kTile);
                load_tile<DP>(k_tile, &map_k, smem_addr(&kv_full), kv_head, u.row);
                load_tile<DP>(v_tile, &map_v, smem_addr(&kv_full), kv_head, u.row);
            }
            int s = 0;
            uint32_t phase = 1;
            for (int t = 0; t < tiles; ++t) {
                const int first = query_lo + t * p.queries;
                if (!bar_wait_together(smem_addr(&q_empty[s]), phase, &failed)) break;
                if (lane == 0) {
                    bar_expect(smem_addr(&q_full[s]), q_bytes);
                    load_tile<DP>(q_ring + s * kTile, &map_q, smem_addr(&q_full[s]), head0, u.other_row + first);
                }
                if (!bar_wait_together(smem_addr(&dy_empty[s]), phase, &failed)) break;
                if (lane == 0) {
                    bar_expect(smem_addr(&dy_full[s]), q_bytes);
                    load_tile<DP>(dy_ring + s * kTile, &map_dy, smem_addr(&dy_full[s]), head0, u.other_row + first);
                }
                // (dK(t - 2), which q_empty told of, came after the threads had read these rows)
                const int live = min(p.queries, u.other_len - first) * p.group;
                const int64_t at = ((int64_t)kv_head * p.runs.query_rows + u.other_row + first) * p.group;
                float a[4], b[4];
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const int r = n * 32 + lane;
                    a[n] = r < live ? p.minus_lse2[at + r] : 0.0f;
                    b[n] = r < live ? p.delta[at + r] : 0.0f;
                }
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const uint32_t to = rows_at + s * (kRows * 8) + (n * 32 + lane) * 4;
                    asm volatile("st.shared.f32 [%0], %1;" ::"r"(to), "f"(a[n]) : "memory");
                    asm volatile("st.shared.f32 [%0], %1;" ::"r"(to + kRows * 4), "f"(-b[n]) : "memory");
                }
                __syncwarp();
                if (lane == 0) bar_arrive(smem_addr(&row_full[s]));
                if (++s == kPairStages) s = 0, phase ^= 1;
            }
        } else if (warp == 8 && tiles > 0) {
            const bool issuer = elect_one();
            // Rows that are not the sequence's, or that the group leaves over, become zero: dV and dK sum over them.
            const auto make = [&](int t, uint64_t *full, uint32_t a, uint32_t ring, uint32_t d, uint64_t *ready) {
                const int s = t % kPairStages;
                if (!bar_wait_together(smem_addr(&full[s]), (t / kPairStages) & 1, &failed)) return false;
                const int live = min(p.queries, u.other_len - (query_lo + t * p.queries)) * p.group;
                if (live < kRows) clear_rows<DP>(ring + s * kTile, live);
                tc_fence_after();
                if (issuer) {
                    product_of_tiles<DP>(d, a, ring + s * kTile);
                    tc_commit(smem_addr(ready));
                }
                __syncwarp();
                return true;
            };
            const auto add = [&](int t, uint32_t d, uint32_t operand, uint32_t ring, uint64_t *empty) {
                const int s = t % kPairStages;
                tc_fence_after();
                if (issuer) {
#pragma unroll
                    for (int ks = 0; ks < kRows / 16; ++ks) product_step<DP>(d, operand + ks / 4 * 64 + ks % 4 * 8, ring + s * kTile, ks, t > 0 || ks > 0);
                    tc_commit(smem_addr(&empty[s]));
                }
                __syncwarp();
            };
            bool ok = bar_wait_together(smem_addr(&kv_full), 0, &failed) && make(0, q_full, k_tile, q_ring, tmem, &s_full) &&
                      make(0, dy_full, v_tile, dy_ring, tmem + 128, &dp_full);
            for (int t = 0; t < tiles && ok; ++t) {
                if (!bar_wait_together(smem_addr(&p_full), t & 1, &failed)) break;
                add(t, tmem + 256, tmem, dy_ring, dy_empty);
                // (the next S takes the columns of P, the next dP those of dS: the tensor cores work in order)
                if (t + 1 < tiles && !make(t + 1, q_full, k_tile, q_ring, tmem, &s_full)) break;
                if (!bar_wait_together(smem_addr(&ds_full), t & 1, &failed)) break;
                add(t, tmem + 256 + DP, tmem + 128, q_ring, q_empty);
                if (t + 1 < tiles && !make(t + 1, dy_full, v_tile, dy_ring, tmem + 128, &dp_full)) break;
                if (t == tiles - 1 && issuer) tc_commit(smem_addr(&done));
                __syncwarp();
            }
        }
    } else {
        take_registers<kRowRegisters>();
        const int half = warp >> 2;                              // of the columns
        const int row = (warp & 3) * 32 + lane;                  // the key
        const bool live = row < u.rows;
        int seen_lo = 0, seen_hi = u.other_len;                  // by these queries of the sequence (keys that nobody reads: by all)
        if (live) queries_seeing(p.mask, u.pos + row, 1, u.shift, u.other_len, seen_lo, seen_hi);
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_at = tmem + lanes + half * 64, d_at = s_at + 128;
        const f2 cc = f2_of(p.scale_log2, p.scale_log2);
        bool ok = true;
        for (int t = 0; t < tiles; ++t) {
            const int s = t % kPairStages;
            const uint32_t rows = rows_at + s * (kRows * 8) + half * 256;
            if (!bar_wait_together(smem_addr(&row_full[s]), (t / kPairStages) & 1, &failed) || !bar_wait_together(smem_addr(&s_full), t & 1, &failed)) {
                ok = false;
                break;
            }
            tc_fence_after();
            float v[64];
#pragma unroll
            for (int j = 0; j < 2; ++j) tc_read32(s_at + 32 * j, reinterpret_cast<uint32_t(&)[32]>(v[32 * j]));
#pragma unroll
            for (int j = 0; j < 2; ++j) tc_read_wait(reinterpret_cast<uint32_t(&)[32]>(v[32 * j]));
#pragma unroll
            for (int n = 0; n < 64; n += 4) {
                f2 m[2];
                asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(m[0]), "=l"(m[1]) : "r"(rows + n * 4));
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const f2 x = f2_fma(f2_of(v[n + 2 * e], v[n + 2 * e + 1]), cc, m[e]);
                    v[n + 2 * e] = exp2_of(f2_lo(x));
                    v[n + 2 * e + 1] = exp2_of(f2_hi(x));
                }
            }
            // of the tile's rows, those of the queries that see the key
            const int first = query_lo + t * p.queries;
            const int from = max(0, min(p.queries, seen_lo - first)) * p.group - half * 64, to = max(0, min(p.queries, seen_hi - first)) * p.group - half * 64;
            if (__any_sync(0xffffffffu, from > 0 || to < 64)) {
#pragma unroll
                for (int n = 0; n < 64; ++n) v[n] = n >= from && n < to ? v[n] : 0.0f;
            }
            uint32_t w[32];
#pragma unroll
            for (int n = 0; n < 64; n += 2) w[n >> 1] = bf16_pair(v[n], v[n + 1]);
            tc_write32(s_at, w);
            tc_write_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(smem_addr(&p_full));
            if (!bar_wait_together(smem_addr(&dp_full), t & 1, &failed)) { ok = false; break; }
            tc_fence_after();
            float d[64];
#pragma unroll
            for (int j = 0; j < 2; ++j) tc_read32(d_at + 32 * j, reinterpret_cast<uint32_t(&)[32]>(d[32 * j]));
#pragma unroll
            for (int j = 0; j < 2; ++j) tc_read_wait(reinterpret_cast<uint32_t(&)[32]>(d[32 * j]));
#pragma unroll
            for (int n = 0; n < 64; n += 4) {
                f2 m[2];
                asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(m[0]), "=l"(m[1]) : "r"(rows + kRows * 4 + n * 4));
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const f2 x = f2_mul(f2_of(v[n + 2 * e], v[n + 2 * e + 1]), f2_add(f2_of(d[n + 2 * e], d[n + 2 * e + 1]), m[e]));
                    w[(n >> 1) + e] = bf16_pair(f2_lo(x), f2_hi(x));
                }
            }
            tc_write32(d_at, w);
            tc_write_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(smem_addr(&ds_full));
        }
        if (ok && tiles > 0 && !bar_wait_together(smem_addr(&done), 0, &failed)) ok = false;
        if (ok) {
            tc_fence_after();
            // one group of warps writes dv, the other dk
            const int64_t key = (int64_t)u.row + row;
            __nv_bfloat16 *out = half ? p.dk + key * p.ld_dk + kv_head * p.head_stride_dk : p.dv + key * p.ld_dv + kv_head * p.head_stride_dv;
#pragma unroll
            for (int j = 0; j < DP; j += 32) store_columns(out, j, p.dim, tmem + lanes + 256 + half * DP + j, half ? p.scale : 1.0f, live, tiles > 0);
        }
    }
    let_copies_land(&failed);
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && failed) atomicExch(p.errword, 2);
    if (warp == 8) tc_free(tmem, 512);
}

struct Maps {
    CUtensorMap q, k, v, dy;
};
template <int DP>
cudaError_t launch_both(const Maps &m, const BackwardArgs &by_query, const BackwardArgs &by_key, bool dependent, cudaStream_t s)
{
    static OncePerDevice configured;
    cudaError_t e = configured.run([&] {
        const cudaError_t f = cudaFuncSetAttribute(attention_dq_kernel<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, kQuerySmem<DP>);
        return f != cudaSuccess ? f : cudaFuncSetAttribute(attention_dkv_kernel<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, kKeySmem<DP>);
    });
    if (e != cudaSuccess) return e;
    const dim3 grid_q((unsigned)(by_query.plan.most * by_query.kv_heads)), grid_k((unsigned)(by_key.plan.most * by_key.kv_heads));
    if (grid_q.x > 0) {
        if (dependent) {
            e = launch_dependent_smem(attention_dq_kernel<DP>, grid_q, dim3(kThreads), kQuerySmem<DP>, s, m.q, m.k, m.v, m.dy, by_query);
        } else {
            attention_dq_kernel<DP><<<grid_q, kThreads, kQuerySmem<DP>, s>>>(m.q, m.k, m.v, m.dy, by_query);
            e = cudaGetLastError();
        }
        if (e != cudaSuccess) return e;
        ++g_kernel_launches;
    }
    if (grid_k.x > 0) {
        e = launch_dependent_smem(attention_dkv_kernel<DP>, grid_k, dim3(kThreads), kKeySmem<DP>, s, m.q, m.k, m.v, m.dy, by_key);
        if (e == cudaSuccess) ++g_kernel_launches;
    }
    return e;
}

int queries_of_tile(const AttentionShape &a) { return kRows / (a.heads / a.kv_heads); }
size_t row_bytes(const AttentionShape &a) { return ((size_t)a.query_rows * a.heads * 4 + 15) / 16 * 16; }

}  // namespace

size_t attention_backward_scratch(const AttentionShape &a)
{
    return 2 * row_bytes(a) + plan_bytes(a.query_start, a.query_rows, queries_of_tile(a), a.sequences) +
           plan_bytes(a.key_start, a.key_rows, kRows, a.sequences) + 16;
}

cudaError_t launch_attention_backward(const AttentionShape &a, const Heads &dy, const Heads &q, const Heads &k, const Heads &v, const Heads &y,
                                      const float *lse, const Heads &dq, const Heads &dk, const Heads &dv, void *scratch, int32_t *errword,
                                      cudaStream_t s)
{
    const int group = a.heads / a.kv_heads, queries = queries_of_tile(a);
    char *at = static_cast<char *>(scratch);
    BackwardArgs p{};
    p.runs = Runs{a.query_start, a.key_start, a.sequences, a.query_rows, a.key_rows};
    p.mask = Mask{a.causal, a.window};
    p.heads = a.heads, p.kv_heads = a.kv_heads, p.group = group, p.dim = a.dim, p.queries = queries;
    p.scale = a.scale, p.scale_log2 = (float)((double)a.scale * 1.4426950408889634);
    p.dy = static_cast<const __nv_bfloat16 *>(dy.p), p.ld_dy = dy.ld, p.head_stride_dy = dy.head_stride;
    p.y = static_cast<const __nv_bfloat16 *>(y.p), p.ld_y = y.ld, p.head_stride_y = y.head_stride;
    p.lse = lse, p.errword = errword;
    p.dq = static_cast<__nv_bfloat16 *>(dq.p), p.ld_dq = dq.ld, p.head_stride_dq = dq.head_stride;
    p.dk = static_cast<__nv_bfloat16 *>(dk.p), p.ld_dk = dk.ld, p.head_stride_dk = dk.head_stride;
    p.dv = static_cast<__nv_bfloat16 *>(dv.p), p.ld_dv = dv.ld, p.head_stride_dv = dv.head_stride;
    p.minus_lse2 = reinterpret_cast<float *>(at), p.delta = reinterpret_cast<float *>(at + row_bytes(a));
    at += 2 * row_bytes(a);
    BackwardArgs by_key = p;
    p.plan = plan_at(at, a.query_start, a.query_rows, queries, a.sequences);
    at += plan_bytes(a.query_start, a.query_rows, queries, a.sequences);
    by_key.plan = plan_at(at, a.key_start, a.key_rows, kRows, a.sequences);
    Maps m;
    cudaError_t e = cudaSuccess;
    if (a.query_rows > 0) {
        e = make_heads_map(&m.q, q.p, a.dim, a.heads, a.query_rows, q.head_stride, q.ld, group, queries);
        if (e == cudaSuccess) e = make_heads_map(&m.dy, dy.p, a.dim, a.heads, a.query_rows, dy.head_stride, dy.ld, group, queries);
    }
    if (e == cudaSuccess && a.key_rows > 0) {
        e = make_heads_map(&m.k, k.p, a.dim, a.kv_heads, a.key_rows, k.head_stride, k.ld, 1, kRows);
        if (e == cudaSuccess) e = make_heads_map(&m.v, v.p, a.dim, a.kv_heads, a.key_rows, v.head_stride, v.ld, 1, kRows);
    }
    if (e == cudaSuccess && a.query_start) e = launch_plan(p.runs, p.mask, &p.plan, &by_key.plan, s);
    if (e != cudaSuccess) return e;
    return a.dim <= 64 ? launch_both<64>(m, p, by_key, a.query_start != nullptr, s) : launch_both<128>(m, p, by_key, a.query_start != nullptr, s);
}

}  // namespace lgc
