// Rotary positions: pairs of a head's entries turned by position * frequency, and the way back (the opposite angle).
//
// The kernel only streams: an entry is read once and written once, and DRAM bounds it.  The angles of a token are the same for
// all its heads, so a warp makes the cosines and sines of a token once and goes over its heads with them; that takes it
// about a microsecond (two products and a rounding in 64 bits, a sine and a cosine per pair), in which the SM's other warps stream.
// (A CTA that does both in step: 68 to 119 us for 16384 tokens of 40 heads of 128.)  Angles of far positions: position * frequency in turns
// is taken in 64 bits and brought to half a turn around zero before it becomes fp32 (2^22 positions of one radian: 32 bits
// would be off by a quarter of a radian).
#include "lgc_attention.cuh"

namespace lgc {

namespace {

constexpr int kThreads = 128;
constexpr int kTable = 256;            // pairs whose cosines and sines a warp holds at a time
constexpr int kFlight = 3;             // heads whose pieces a lane has under way

struct RotaryArgs {
    const void *x;
    void *y;
    int64_t rows, ldx, hx, ldy, hy;    // distances of rows and heads, in elements
    int heads, dim, pairs;
    const int64_t *positions;
    const double *frequencies;
    float amplitude, sign;
    int span, spans;                   // heads of a warp, warps of a token
    bool in_place;
};

// V entries as they lie in memory: they stay packed while they are on their way.
template <typename T, int V>
struct Raw {
    uint32_t w[V * sizeof(T) < 4 ? 1 : V * sizeof(T) / 4];
};
template <typename T, int V>
__device__ __forceinline__ void load(const T *at, Raw<T, V> &q)
{
    constexpr int kBytes = V * sizeof(T);
    if constexpr (kBytes == 2) {
        q.w[0] = *reinterpret_cast<const uint16_t *>(at);
    } else if constexpr (kBytes == 4) {
        q.w[0] = *reinterpret_cast<const uint32_t *>(at);
    } else if constexpr (kBytes == 8) {
        const uint2 v = *reinterpret_cast<const uint2 *>(at);
        q.w[0] = v.x, q.w[1] = v.y;
    } else {
#pragma unroll
        for (int i = 0; i < kBytes / 4; i += 4) {
            const uint4 v = *(reinterpret_cast<const uint4 *>(at) + i / 4);
            q.w[i] = v.x, q.w[i + 1] = v.y, q.w[i + 2] = v.z, q.w[i + 3] = v.w;
        }
    }
}
template <typename T, int V>
__device__ __forceinline__ float entry(const Raw<T, V> &q, int i)
{
    if constexpr (sizeof(T) == 4) return __uint_as_float(q.w[i]);
    else return __uint_as_float(i & 1 ? q.w[i / 2] & 0xffff0000u : q.w[i / 2] << 16);
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

// V pairs, or V entries that pass through, at a time; V divides both parts of a head.  A lane keeps its piece of a head and goes over
// the heads, kFlight at a time under way.
template <typename T, int V, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads)
rotary_kernel(const __grid_constant__ RotaryArgs p)
{
    __shared__ float cosines[kThreads / 32][kTable], sines[kThreads / 32][kTable];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t number = (int64_t)blockIdx.x * (kThreads / 32) + warp, row = number / p.spans;
    if (row >= p.rows) return;
    const int head0 = (int)(number - row * p.spans) * p.span, heads = min(p.span, p.heads - head0);
    const int pieces = p.pairs / V, per_head = pieces + (p.in_place ? 0 : (p.dim - 2 * p.pairs) / V);
    const int side = min(per_head, 32), at_once = 32 / side, first = lane / side;
    const T *x = static_cast<const T *>(p.x) + row * p.ldx + head0 * p.hx;
    T *y = static_cast<T *>(p.y) + row * p.ldy + head0 * p.hy;
    const double position = (double)p.positions[row];
    float *cos_of = cosines[warp], *sin_of = sines[warp];
    for (int pair0 = 0; pair0 < p.pairs; pair0 += kTable) {
        const int width = min(kTable, p.pairs - pair0);
        __syncwarp();
        for (int i = lane; i < width; i += 32) {
            const double turns = position * (p.frequencies[pair0 + i] * 0.15915494309189535);
            float s, c;
            sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
            cos_of[i] = __fmul_rn(c, p.amplitude);
            sin_of[i] = __fmul_rn(s, __fmul_rn(p.amplitude, p.sign));
        }
        __syncwarp();
        for (int piece = lane - first * side; piece < per_head && first < at_once; piece += side) {
            const int pair = piece * V;
            if (piece >= pieces) {
                if (pair0 > 0) continue;
                const int at = 2 * p.pairs + (piece - pieces) * V;
                for (int head = first; head < heads; head += at_once) {
                    Raw<T, V> q;
                    float a[V];
                    load<T, V>(x + head * p.hx + at, q);
#pragma unroll
                    for (int n = 0; n < V; ++n) a[n] = entry(q, n);
                    store<T, V>(y + head * p.hy + at, a);
                }
                continue;
            }
            if (pair < pair0 || pair >= pair0 + width) continue;
            const int at_a = INTERLEAVED ? 2 * pair : pair, at_b = INTERLEAVED ? 2 * pair + V : p.pairs + pair;
            float c[V], s[V];
#pragma unroll
            for (int n = 0; n < V; ++n) c[n] = cos_of[pair - pair0 + n], s[n] = sin_of[pair - pair0 + n];
            for (int head = first; head < heads; head += kFlight * at_once) {
                Raw<T, V> a[kFlight], b[kFlight];
#pragma unroll
                for (int h = 0; h < kFlight; ++h)
                    if (head + h * at_once < heads) {
                        const T *from = x + (head + h * at_once) * p.hx;
                        load<T, V>(from + at_a, a[h]);
                        load<T, V>(from + at_b, b[h]);
                    }
#pragma unroll
                for (int h = 0; h < kFlight; ++h) {
                    if (head + h * at_once >= heads) break;
                    float u[V], v[V];
#pragma unroll
                    for (int n = 0; n < V; ++n) {
                        if (INTERLEAVED) {
                            // entries 2 n and 2 n + 1 of the 2 V that begin at a
                            const float one = 2 * n < V ? entry(a[h], (2 * n) % V) : entry(b[h], (2 * n) % V);
                            const float two = 2 * n + 1 < V ? entry(a[h], (2 * n + 1) % V) : entry(b[h], (2 * n + 1) % V);
                            const float f = __fmaf_rn(one, c[n], -__fmul_rn(two, s[n])), g = __fmaf_rn(one, s[n], __fmul_rn(two, c[n]));
                            if (2 * n < V) u[(2 * n) % V] = f;
                            else v[(2 * n) % V] = f;
                            if (2 * n + 1 < V) u[(2 * n + 1) % V] = g;
                            else v[(2 * n + 1) % V] = g;
                        } else {
                            u[n] = __fmaf_rn(entry(a[h], n), c[n], -__fmul_rn(entry(b[h], n), s[n]));
                            v[n] = __fmaf_rn(entry(a[h], n), s[n], __fmul_rn(entry(b[h], n), c[n]));
                        }
                    }
                    T *to = y + (head + h * at_once) * p.hy;
                    store<T, V>(to + at_a, u);
                    store<T, V>(to + at_b, v);
                }
            }
        }
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
    RotaryArgs p{x, y, rows, ldx, head_stride_x, ldy, head_stride_y, heads, dim, pairs, positions, frequencies, amplitude, backward ? -1.0f : 1.0f, heads, 1,
                 x == y};
    // a warp has all heads of a token where there are tokens for eight warps an SM, otherwise eight
    if (rows < 148 * 8 && heads > 8) p.span = 8, p.spans = (heads + 7) / 8;
    const int size = type == LGC_TYPE_FP32 ? 4 : 2;
    // the widest step that divides both parts of a head and keeps every access on its boundary
    const uint64_t bits = reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(y) |
                          (uint64_t)((rows > 1 ? ldx | ldy : 0) | (heads > 1 ? head_stride_x | head_stride_y : 0)) * size;
    const uint64_t parts = (uint64_t)(pairs | (dim - 2 * pairs));
    const int v = parts % 8 == 0 && bits % 16 == 0 ? 8 : parts % 4 == 0 && bits % (4 * size) == 0 ? 4 : 1;
    const unsigned ctas = (unsigned)((rows * p.spans + kThreads / 32 - 1) / (kThreads / 32));
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
