// Rotary positions: pairs of a head's entries turned by position * frequency, and the way back (the opposite angle).
//
// The kernel only streams: an entry is read once and written once, and DRAM bounds it.  The angles of a token are the same for
// all its heads, so a CTA makes the cosines and sines of a few tokens once, in shared memory, and goes over their heads with
// them.  Angles of far positions: position * frequency in turns is taken in 64 bits and brought to half a turn around zero
// before it becomes fp32 (2^22 positions of one radian: 32 bits would be off by a quarter of a radian).
#include "lgc_attention.cuh"

namespace lgc {

namespace {

constexpr int kThreads = 256;
constexpr int kTable = 512;            // cosines and sines of a CTA

struct RotaryArgs {
    const void *x;
    void *y;
    int64_t rows, ldx, hx, ldy, hy;    // distances of rows and heads, in elements
    int heads, dim, pairs;
    const int64_t *positions;
    const double *frequencies;
    float amplitude, sign;
    int tokens;                        // of a CTA
    bool in_place;
};

template <typename T, int V>
__device__ __forceinline__ void load(const T *at, float (&v)[V])
{
    if constexpr (V == 1) {
        v[0] = (float)*at;
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const float4 q = *reinterpret_cast<const float4 *>(at + i);
            v[i] = q.x, v[i + 1] = q.y, v[i + 2] = q.z, v[i + 3] = q.w;
        }
    } else {
        uint32_t w[V / 2];
        if constexpr (V == 8) {
            const uint4 q = *reinterpret_cast<const uint4 *>(at);
            w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
        } else {
            const uint2 q = *reinterpret_cast<const uint2 *>(at);
            w[0] = q.x, w[1] = q.y;
        }
#pragma unroll
        for (int i = 0; i < V / 2; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
template <typename T, int V>
__device__ __forceinline__ void store(T *at, const float (&v)[V])
{
    if constexpr (V == 1) {
        *at = (T)v[0];
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < V; i += 4) *reinterpret_cast<float4 *>(at + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    } else if constexpr (V == 8) {
        *reinterpret_cast<uint4 *>(at) = make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
    } else {
        *reinterpret_cast<uint2 *>(at) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
    }
}

// V pairs, or V entries that pass through, at a time; V divides both parts of a head.
template <typename T, int V, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads)
rotary_kernel(const __grid_constant__ RotaryArgs p)
{
    __shared__ float cosines[kTable], sines[kTable];
    const int64_t row0 = (int64_t)blockIdx.x * p.tokens;
    const int tokens = (int)min((int64_t)p.tokens, p.rows - row0);
    const int pieces = p.pairs / V, rest = p.in_place ? 0 : (p.dim - 2 * p.pairs) / V, per_head = pieces + rest, per_token = p.heads * per_head;
    // the pairs of a CTA's tokens, kTable at a time
    for (int pair0 = 0; pair0 < p.pairs || pair0 == 0; pair0 += kTable / p.tokens / 8 * 8) {
        const int width = min(kTable / p.tokens / 8 * 8, p.pairs - pair0);
        for (int i = threadIdx.x; i < tokens * width; i += kThreads) {
            const int token = i / width, pair = pair0 + i - token * width;
            const double turns = (double)p.positions[row0 + token] * (p.frequencies[pair] * 0.15915494309189535);
            float s, c;
            sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
            cosines[i] = __fmul_rn(c, p.amplitude);
            sines[i] = __fmul_rn(s, __fmul_rn(p.amplitude, p.sign));
        }
        __syncthreads();
        for (int token = 0; token < tokens; ++token) {
            const T *x = static_cast<const T *>(p.x) + (row0 + token) * p.ldx;
            T *y = static_cast<T *>(p.y) + (row0 + token) * p.ldy;
            for (int i = threadIdx.x; i < per_token; i += kThreads) {
                const int head = i / per_head, piece = i - head * per_head;
                const T *xh = x + head * p.hx;
                T *yh = y + head * p.hy;
                if (piece < pieces) {
                    const int pair = piece * V;
                    if (pair < pair0 || pair >= pair0 + width) continue;
                    const int at_a = INTERLEAVED ? 2 * pair : pair, at_b = INTERLEAVED ? 2 * pair + V : p.pairs + pair;
                    float a[V], b[V], u[V], v[V];
                    load<T, V>(xh + at_a, a);
                    load<T, V>(xh + at_b, b);
                    const float *c = cosines + token * width + pair - pair0, *s = sines + token * width + pair - pair0;
#pragma unroll
                    for (int n = 0; n < V; ++n) {
                        if (INTERLEAVED) {
                            // entries 2 n and 2 n + 1 of the 2 V that begin at a
                            const float first = 2 * n < V ? a[(2 * n) % V] : b[(2 * n) % V], second = 2 * n + 1 < V ? a[(2 * n + 1) % V] : b[(2 * n + 1) % V];
                            const float f = __fmaf_rn(first, c[n], -__fmul_rn(second, s[n])), g = __fmaf_rn(first, s[n], __fmul_rn(second, c[n]));
                            if (2 * n < V) u[(2 * n) % V] = f;
                            else v[(2 * n) % V] = f;
                            if (2 * n + 1 < V) u[(2 * n + 1) % V] = g;
                            else v[(2 * n + 1) % V] = g;
                        } else {
                            u[n] = __fmaf_rn(a[n], c[n], -__fmul_rn(b[n], s[n]));
                            v[n] = __fmaf_rn(a[n], s[n], __fmul_rn(b[n], c[n]));
                        }
                    }
                    store<T, V>(yh + at_a, u);
                    store<T, V>(yh + at_b, v);
                } else if (pair0 == 0) {
                    const int at = 2 * p.pairs + (piece - pieces) * V;
                    float a[V];
                    load<T, V>(xh + at, a);
                    store<T, V>(yh + at, a);
                }
            }
        }
        __syncthreads();
    }
}

template <typename T, int V>
void launch(const RotaryArgs &p, bool interleaved, unsigned ctas, cudaStream_t s)
{
    if (interleaved) rotary_kernel<T, V, true><<<ctas, kThreads, 0, s>>>(p);
    else rotary_kernel<T, V, false><<<ctas, kThreads, 0, s>>>(p);
}

}  // namespace

cudaError_t launch_rotary(const void *x, int32_t type, int64_t rows, int heads, int dim, int64_t ldx, int64_t head_stride_x, const int64_t *positions,
                          const double *frequencies, int pairs, bool interleaved, float amplitude, bool backward, void *y, int64_t ldy,
                          int64_t head_stride_y, cudaStream_t s)
{
    RotaryArgs p{x, y, rows, ldx, head_stride_x, ldy, head_stride_y, heads, dim, pairs, positions, frequencies, amplitude, backward ? -1.0f : 1.0f, 1,
                 x == y};
    // four tokens to a CTA where that leaves enough of them for every SM: their angles are one evaluation per thread
    p.tokens = rows >= 4 * 148 * 4 ? 4 : 1;
    const int size = type == LGC_TYPE_FP32 ? 4 : 2;
    // the widest step that divides both parts of a head and keeps every access on its boundary
    const uint64_t bits = reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(y) |
                          (uint64_t)((rows > 1 ? ldx | ldy : 0) | (heads > 1 ? head_stride_x | head_stride_y : 0)) * size;
    const uint64_t parts = (uint64_t)(pairs | (dim - 2 * pairs));
    const int v = parts % 8 == 0 && bits % 16 == 0 ? 8 : parts % 4 == 0 && bits % (4 * size) == 0 ? 4 : 1;
    const unsigned ctas = (unsigned)((rows + p.tokens - 1) / p.tokens);
    if (type == LGC_TYPE_FP32) {
        if (v == 8) launch<float, 8>(p, interleaved, ctas, s);
        else if (v == 4) launch<float, 4>(p, interleaved, ctas, s);
        else launch<float, 1>(p, interleaved, ctas, s);
    } else {
        if (v == 8) launch<__nv_bfloat16, 8>(p, interleaved, ctas, s);
        else if (v == 4) launch<__nv_bfloat16, 4>(p, interleaved, ctas, s);
        else launch<__nv_bfloat16, 1>(p, interleaved, ctas, s);
    }
    ++g_kernel_launches;
    return cudaGetLastError();
}

}  // namespace lgc
