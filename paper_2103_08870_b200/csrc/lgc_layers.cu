// C ABI of the layer operators: argument checks and the word their kernels record failures in (see include/lgc.h for
// the contract of each).
#include <cmath>
#include <mutex>

#include "lgc_layers.cuh"
#include "lgc_tensor_core.cuh"

namespace lgc {

bool matrix_rows_aligned(const void *p, int64_t ld, int elem_bytes)
{
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (ld * elem_bytes) % 16 == 0;
}

int matrix_alignment(const void *p, int64_t ld, int elem_bytes)
{
    const uint64_t bits = reinterpret_cast<uintptr_t>(p) | (uint64_t)(ld * elem_bytes);
    return bits % 32 == 0 ? 32 : bits % 16 == 0 ? 16 : 0;
}

namespace {

static __device__ int32_t g_layers_record;      // a handle in host code: see record_address

// Device address of the record on the current device; looked up once per device.
cudaError_t record_address(int32_t **out)
{
    static std::mutex mu;
    static int32_t *cached[kMaxDevices] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    std::lock_guard<std::mutex> lock(mu);
    if (!cached[dev]) {
        void *p = nullptr;
        e = cudaGetSymbolAddress(&p, g_layers_record);
        if (e != cudaSuccess) return e;
        cached[dev] = static_cast<int32_t *>(p);
    }
    *out = cached[dev];
    return cudaSuccess;
}

lgc_status refuse(const char *where, const char *why, lgc_status status = LGC_ERR_INVALID_ARG)
{
    g_last_error = std::string(where) + ": " + why;
    return status;
}
lgc_status done(const char *where, cudaError_t e)
{
    if (e == cudaSuccess) return LGC_OK;
    g_last_error = std::string(where) + ": " + cudaGetErrorString(e);
    return LGC_ERR_CUDA;
}

constexpr int64_t kMaxRows = (int64_t)1 << 30;   // rows and columns are TMA coordinates (int32), a tile may reach past the end
constexpr int64_t kMaxCols = (int64_t)1 << 30;

const char *bad_sizes(int64_t rows, int64_t cols)
{
    if (rows < 0 || rows > kMaxRows) return "num_rows must be in [0, 2^30]";
    if (cols < 1 || cols > kMaxCols) return "sizes of a row must be in [1, 2^30]";
    return nullptr;
}
const char *bad_matrix(const void *p, int32_t type, int64_t cols, int64_t ld)
{
    if (type != LGC_TYPE_FP32 && type != LGC_TYPE_BF16) return "matrices are fp32 or bf16";
    if (!p) return "NULL matrix";
    if (reinterpret_cast<uintptr_t>(p) % (type == LGC_TYPE_FP32 ? 4 : 2) != 0) return "misaligned matrix";
    if (ld < cols) return "rows of a matrix overlap (ld below the number of columns)";
    if (ld > ((int64_t)1 << 40)) return "ld above 2^40";
    return nullptr;
}
const char *bad_packed(const lgc_packed *p, int64_t cols)
{
    if (!p || !p->codes || !p->scales) return "NULL 8-bit matrix";
    if ((reinterpret_cast<uintptr_t>(p->codes) & 15) != 0 || p->ld % 16 != 0 || p->ld < cols || p->ld > ((int64_t)1 << 39))
        return "codes must be 16-byte aligned, ld a multiple of 16 that holds a row";
    if ((reinterpret_cast<uintptr_t>(p->scales) & 3) != 0 || p->ld_scales % 4 != 0 || p->ld_scales < (cols + kBlock - 1) / kBlock ||
        p->ld_scales > ((int64_t)1 << 39))
        return "scales must be 4-byte aligned, ld_scales a multiple of 4 that holds a row's blocks";
    return nullptr;
}
bool aligned4(const void *p) { return p && (reinterpret_cast<uintptr_t>(p) & 3) == 0; }
const char *bad_nodes(const int64_t *node_start, int32_t num_nodes, int64_t per_node, int64_t node_stride)
{
    if (num_nodes < 1 || num_nodes > 65535) return "num_nodes must be in [1, 65535]";
    if (!node_start && num_nodes != 1) return "node_start is NULL with more than one node";
    if ((reinterpret_cast<uintptr_t>(node_start) & 7) != 0) return "misaligned node_start";
    if (num_nodes > 1 && node_stride < per_node) return "the nodes' gradients overlap (node_stride)";
    return nullptr;
}

}  // namespace

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// cuTensorMapEncodeTiled, fetched once through the runtime so that the library does not link the driver
static cudaError_t encode_fn(EncodeTiledFn *out)
{
    static std::mutex mu;
    static EncodeTiledFn found = nullptr;
    std::lock_guard<std::mutex> lock(mu);
    if (!found) {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult q;
        const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q);
        if (e != cudaSuccess) return e;
        if (q != cudaDriverEntryPointSuccess || !fn) return cudaErrorNotSupported;
        found = reinterpret_cast<EncodeTiledFn>(fn);
    }
    *out = found;
    return cudaSuccess;
}

cudaError_t make_matrix_map(CUtensorMap *m, CUtensorMapDataType type, int elem_bytes, const void *base, int64_t cols, int64_t rows,
                            int64_t ld, int box_cols, int box_rows, CUtensorMapSwizzle swizzle)
{
    EncodeTiledFn enc;
    const cudaError_t e = encode_fn(&enc);
    if (e != cudaSuccess) return e;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)ld * (cuuint64_t)elem_bytes};
    const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows};
    const cuuint32_t es[2] = {1, 1};
    return enc(m, type, 2, const_cast<void *>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? cudaSuccess
               : cudaErrorInvalidValue;
}

}  // namespace lgc

using namespace lgc;

extern "C" {

lgc_status lgc_pack(const void *x, int32_t type, int64_t num_rows, int64_t num_cols, int64_t ldx, int32_t block_rows, float slope,
                    const lgc_packed *gate, const lgc_packed *out, void *y, int64_t ldy, void *stream)
{
    const char *where = "lgc_pack", *why = bad_sizes(num_rows, num_cols);
    if (why) return refuse(where, why);
    if (num_rows == 0) return LGC_OK;
    if ((why = bad_matrix(x, type, num_cols, ldx)) || (why = bad_packed(out, num_cols)) ||
        (gate && (why = bad_packed(gate, num_cols))) || (y && (why = bad_matrix(y, LGC_TYPE_BF16, num_cols, ldy))))
        return refuse(where, why);
    if (block_rows != 1 && block_rows != kBlock) return refuse(where, "block_rows must be 1 or 128");
    if (gate && block_rows != 1) return refuse(where, "a gate goes with block_rows = 1");
    if (gate && (std::isnan(slope) || std::signbit(slope))) return refuse(where, "with a gate, slope must not be negative (nor -0)");
    if (block_rows != 1 && num_rows > 65535 * (int64_t)kBlock) return refuse(where, "too many rows for block_rows = 128", LGC_ERR_UNSUPPORTED);
    return done(where, launch_pack(Matrix{x, type, ldx}, num_rows, num_cols, block_rows, slope, gate, *out, y, ldy,
                                   static_cast<cudaStream_t>(stream)));
}

lgc_status lgc_unpack(const lgc_packed *src, int64_t num_rows, int64_t num_cols, int32_t block_rows, void *y, int32_t type, int64_t ldy,
                      void *stream)
{
    const char *where = "lgc_unpack", *why = bad_sizes(num_rows, num_cols);
    if (why) return refuse(where, why);
    if (num_rows == 0) return LGC_OK;
    if ((why = bad_packed(src, num_cols)) || (why = bad_matrix(y, type, num_cols, ldy)))
        return refuse(where, why);
    if (block_rows != 1 && block_rows != kBlock) return refuse(where, "block_rows must be 1 or 128");
    return done(where, launch_unpack(*src, num_rows, num_cols, block_rows, y, type, ldy, static_cast<cudaStream_t>(stream)));
}

lgc_status lgc_layer_norm(const void *x, int32_t type, int64_t num_rows, int64_t num_cols, int64_t ldx, const float *gamma,
                          const float *beta, float eps, void *y, int64_t ldy, const lgc_packed *packed, float *mean, float *rstd,
                          void *stream)
{
    const char *where = "lgc_layer_norm", *why = bad_sizes(num_rows, num_cols);
    if (why) return refuse(where, why);
    if (num_rows == 0) return LGC_OK;
    if ((why = bad_matrix(x, type, num_cols, ldx)) ||
        (y && (why = bad_matrix(y, type, num_cols, ldy))) || (packed && (why = bad_packed(packed, num_cols))))
        return refuse(where, why);
    if (num_cols > kNormMaxCols) return refuse(where, "more than 16384 columns", LGC_ERR_UNSUPPORTED);
    if (!y && !packed) return refuse(where, "neither y nor packed is given");
    if (!aligned4(gamma) || !aligned4(beta) || !aligned4(mean) || !aligned4(rstd)) return refuse(where, "NULL or misaligned vector");
    if (!(eps >= 0.0f)) return refuse(where, "eps must not be negative");
    return done(where, launch_layer_norm(Matrix{x, type, ldx}, num_rows, num_cols, gamma, beta, eps, y, ldy, packed, mean, rstd,
                                         static_cast<cudaStream_t>(stream)));
}

lgc_status lgc_layer_norm_backward_scratch(int64_t num_rows, int64_t num_cols, int32_t num_nodes, size_t *bytes)
{
    const char *where = "lgc_layer_norm_backward_scratch", *why = bad_sizes(num_rows, num_cols);
    if (why) return refuse(where, why);
    if (!bytes || num_nodes < 1 || num_nodes > 65535) return refuse(where, "NULL result or num_nodes outside [1, 65535]");
    *bytes = layer_norm_backward_scratch(num_rows, num_cols, num_nodes);
    return LGC_OK;
}

lgc_status lgc_layer_norm_backward(const void *dy, int32_t dy_type, int64_t ld_dy, const void *x, int32_t x_type, int64_t ldx,
                                   const lgc_packed *x_packed, int64_t num_rows, int64_t num_cols, const float *gamma, const float *mean,
                                   const float *rstd, const int64_t *node_start, int32_t num_nodes, void *dx, int64_t ld_dx, float *dgamma,
                                   float *dbeta, int64_t node_stride, void *scratch, size_t scratch_bytes, void *stream)
{
    const char *where = "lgc_layer_norm_backward", *why = nullptr;
    const bool kept = x_type == LGC_TYPE_PACKED;
    if ((why = bad_sizes(num_rows, num_cols)) || (why = bad_nodes(node_start, num_nodes, num_cols, node_stride))) return refuse(where, why);
    if (num_rows > 0 && ((why = bad_matrix(dy, dy_type, num_cols, ld_dy)) ||
                         (why = kept ? bad_packed(x_packed, num_cols) : bad_matrix(x, x_type, num_cols, ldx)) ||
                         (why = bad_matrix(dx, dy_type, num_cols, ld_dx))))
        return refuse(where, why);
    if (num_cols > kNormMaxCols) return refuse(where, "more than 16384 columns", LGC_ERR_UNSUPPORTED);
    if ((num_rows > 0 && (!aligned4(gamma) || !aligned4(mean) || !aligned4(rstd))) || !aligned4(dgamma) || !aligned4(dbeta))
        return refuse(where, "NULL or misaligned vector");
    if (!scratch || (reinterpret_cast<uintptr_t>(scratch) & 15) != 0) return refuse(where, "scratch is NULL or not 16-byte aligned");
    if (scratch_bytes < layer_norm_backward_scratch(num_rows, num_cols, num_nodes))
        return refuse(where, "scratch is smaller than lgc_layer_norm_backward_scratch says", LGC_ERR_WORKSPACE);
    int32_t *record = nullptr;
    cudaError_t e = record_address(&record);
    if (e == cudaSuccess)
        e = launch_layer_norm_backward(Matrix{dy, dy_type, ld_dy}, Matrix{x, x_type, ldx}, kept ? x_packed : nullptr, num_rows, num_cols, gamma,
                                       mean, rstd, node_start, num_nodes, dx, ld_dx, dgamma, dbeta, node_stride, scratch, record,
                                       static_cast<cudaStream_t>(stream));
    return done(where, e);
}

lgc_status lgc_product(const lgc_packed *a, const lgc_packed *b, int32_t across, int64_t num_rows, int64_t num_cols, int64_t inner,
                       float slope, void *y, int32_t type, int64_t ldy, const lgc_packed *packed, void *stream)
{
    const char *where = "lgc_product", *why = nullptr;
    if ((why = bad_sizes(num_rows, num_cols)) || (why = bad_sizes(0, inner))) return refuse(where, why);
    if (num_rows == 0) return LGC_OK;
    if ((why = bad_packed(a, inner)) || (why = bad_packed(b, across ? num_cols : inner)) || (y && (why = bad_matrix(y, type, num_cols, ldy))) ||
        (packed && (why = bad_packed(packed, num_cols))))
        return refuse(where, why);
    if (across != 0 && across != 1) return refuse(where, "across must be 0 or 1");
    if (!y && !packed) return refuse(where, "neither y nor packed is given");
    int32_t *record = nullptr;
    cudaError_t e = record_address(&record);
    if (e == cudaSuccess)
        e = launch_product(*a, *b, across != 0, num_rows, num_cols, inner, slope, y, type, ldy, packed, record,
                           static_cast<cudaStream_t>(stream));
    return done(where, e);
}

lgc_status lgc_weight_gradient_scratch(int64_t num_rows, int64_t num_cols, int64_t inner, int32_t num_nodes, size_t *bytes)
{
    const char *where = "lgc_weight_gradient_scratch", *why = bad_sizes(num_rows, num_cols);
    if (why || (why = bad_sizes(0, inner))) return refuse(where, why);
    if (!bytes || num_nodes < 1 || num_nodes > 65535) return refuse(where, "NULL result or num_nodes outside [1, 65535]");
    *bytes = weight_gradient_scratch(num_rows, num_cols, inner, num_nodes);
    return LGC_OK;
}

lgc_status lgc_weight_gradient(const void *dy, int64_t ld_dy, const lgc_packed *x, int64_t num_rows, int64_t num_cols, int64_t inner,
                               const int64_t *node_start, int32_t num_nodes, float *dw, int64_t node_stride, void *scratch,
                               size_t scratch_bytes, void *stream)
{
    const char *where = "lgc_weight_gradient", *why = nullptr;
    if ((why = bad_sizes(num_rows, num_cols)) || (why = bad_sizes(0, inner))) return refuse(where, why);
    if (num_rows > 0 && ((why = bad_packed(x, inner)) || (why = bad_matrix(dy, LGC_TYPE_BF16, num_cols, ld_dy)))) return refuse(where, why);
    if (num_cols > ((int64_t)1 << 40) / inner) return refuse(where, "num_cols * inner above 2^40");
    if ((why = bad_nodes(node_start, num_nodes, num_cols * inner, node_stride))) return refuse(where, why);
    if (num_rows > 0 && !matrix_rows_aligned(dy, ld_dy, 2)) return refuse(where, "dy must be 16-byte aligned, ld_dy a multiple of 8");
    if (!aligned4(dw)) return refuse(where, "NULL or misaligned dw");
    if (num_rows == 0)                            // no node has a row: every gradient is zero
        return done(where, cudaMemset2DAsync(dw, (size_t)(num_nodes > 1 ? node_stride : num_cols * inner) * 4, 0,
                                             (size_t)(num_cols * inner) * 4, (size_t)num_nodes, static_cast<cudaStream_t>(stream)));
    if (!scratch || (reinterpret_cast<uintptr_t>(scratch) & 15) != 0) return refuse(where, "scratch is NULL or not 16-byte aligned");
    if (scratch_bytes < weight_gradient_scratch(num_rows, num_cols, inner, num_nodes))
        return refuse(where, "scratch is smaller than lgc_weight_gradient_scratch says", LGC_ERR_WORKSPACE);
    int32_t *record = nullptr;
    cudaError_t e = record_address(&record);
    if (e == cudaSuccess)
        e = launch_weight_gradient(dy, ld_dy, *x, num_rows, num_cols, inner, node_start, num_nodes, dw, node_stride, scratch, record,
                                   static_cast<cudaStream_t>(stream));
    return done(where, e);
}

lgc_status lgc_layers_check(void *stream)
{
    const char *where = "lgc_layers_check";
    int32_t *record = nullptr, word = 0;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = record_address(&record);
    if (e == cudaSuccess) e = cudaMemcpyAsync(&word, record, sizeof word, cudaMemcpyDeviceToHost, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (e == cudaSuccess && word != 0) e = cudaMemsetAsync(record, 0, sizeof word, s);
    if (e != cudaSuccess) return done(where, e);
    if (word == 0) return LGC_OK;
    return refuse(where, "a wait inside a kernel ran out", LGC_ERR_DEVICE_CHECK);
}

}  // extern "C"
