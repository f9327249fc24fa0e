// Microscaled numbers for gfx950 (wave64): rows in 4 or 8 bits with a scale per 32 columns, the product of a dense layer on
// the pooled output in 4 bits, and its weights' gradient from the pooled output's 8-bit checkpoint.  (The lookup from 4-bit
// tables is with the layer's other kernels, in pk_device.hip.)  No call here needs a plan; none allocates.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <string>
#include <type_traits>

#include "pk_internal.h"

using namespace pk;

namespace {

#include "dev_common.h"
#include "dev_rows.h"
#include "dev_mx.h"
#include "dev_mx_rows.h"
#include "dev_mx_linear.h"
#include "dev_mx_grad.h"

#define MX_LAUNCH(name, kernel, grid, block, ...)                                                       \
    do {                                                                                                \
        kernel<<<grid, block, 0, stream>>>(__VA_ARGS__);                                                \
        const hipError_t e_ = hipGetLastError();                                                        \
        if (e_ != hipSuccess) return fail(PK_EHIP, std::string("launch of " name ": ") + hipGetErrorString(e_)); \
    } while (0)

bool misaligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

// a matrix of fp32 or bf16: what is wrong with it, or nullptr
const char* bad_matrix(const void* p, int32_t dtype, int64_t stride, int64_t n_rows, int64_t cols)
{
    if (dtype != PK_F32 && dtype != PK_BF16) return "dtype is neither PK_F32 nor PK_BF16";
    if (n_rows == 0) return nullptr;
    if (!p) return "NULL matrix";
    if (misaligned(p, dtype == PK_F32 ? 4 : 2)) return "matrix is not aligned to its elements";
    if (n_rows > 1 && stride < cols) return "row stride is smaller than the columns";
    return nullptr;
}
const char* bad_rows(const void* p, int32_t format, int64_t stride, int64_t n_rows, int64_t cols)
{
    if (n_rows == 0) return nullptr;
    if (!p) return "NULL rows";
    if (misaligned(p, 4) || stride % 4) return "rows and their stride must be multiples of 4 bytes";
    if (stride < mx_row_bytes(format, cols)) return "row stride is smaller than pk_mx_row_bytes";
    return nullptr;
}
pk_status bad_shape(const char* who, const char* what) { return fail(PK_ESHAPE, std::string(who) + ": " + what); }

constexpr int64_t kMxMax = ((int64_t)1 << 31) - 1;      // rows, columns
// Products: rows and columns of the result (whole tiles of them are counted in 32 bits); columns of microscaled rows and bytes
// between them (a tile's 128 rows are addressed in 32 bits).
constexpr int64_t kMxProductMax = (int64_t)1 << 30, kMxDepthMax = (int64_t)1 << 23;
constexpr int64_t kMxGradStrideMax = (int64_t)1 << 24;   // elements between rows of dY (16 rows are addressed in 31 bits)

template <int FMT, bool BF16>
pk_status quantize_launch(const void* src, int64_t src_stride, int64_t n_rows, int64_t cols, void* rows, int64_t row_stride, hipStream_t stream)
{
    const RowGroups g(cols);
    const int64_t items = n_rows * g.n;
    MX_LAUNCH("mx_quantize", (mx_quantize_kernel<FMT, BF16>), dim3(mx_blocks_for(items)), dim3(NT), static_cast<const char*>(src),
              src_stride * (BF16 ? 2 : 4), (uint32_t)cols, g, static_cast<uint8_t*>(rows), row_stride, items);
    return PK_OK;
}
template <int FMT, bool BF16>
pk_status dequantize_launch(const void* rows, int64_t row_stride, int64_t n_rows, int64_t cols, void* dst, int64_t dst_stride, hipStream_t stream)
{
    const RowGroups g(cols);
    const int64_t items = n_rows * g.n;
    MX_LAUNCH("mx_dequantize", (mx_dequantize_kernel<FMT, BF16>), dim3(mx_blocks_for(items)), dim3(NT), static_cast<const uint8_t*>(rows),
              row_stride, (uint32_t)cols, g, static_cast<char*>(dst), dst_stride * (BF16 ? 2 : 4), items);
    return PK_OK;
}

// No call throws: what is thrown while an error's text is made ends here.
template <typename Fn>
pk_status guarded(Fn&& fn) noexcept
{
    try { return fn(); } catch (...) { return PK_ENOMEM; }
}

pk_status check_matrix_shape(const char* who, int64_t n_rows, int64_t cols)
{
    if (n_rows < 0 || cols <= 0) return bad_shape(who, "sizes must be positive (rows may be 0)");
    if (n_rows > kMxMax || cols > kMxMax) return fail(PK_EOVERFLOW, std::string(who) + ": sizes must be below 2^31");
    return PK_OK;
}
pk_status check_product(const char* who, int64_t rows, int64_t N, int64_t K, int64_t row_stride)
{
    if (rows < 0 || N <= 0 || K <= 0) return bad_shape(who, "sizes must be positive (rows of the input may be 0)");
    if (rows > kMxProductMax || N > kMxProductMax) return fail(PK_EOVERFLOW, std::string(who) + ": rows and N must be at most 2^30");
    if (K > kMxDepthMax || row_stride > kMxDepthMax * 2) return fail(PK_EOVERFLOW, std::string(who) + ": K must be at most 2^23, microscaled rows at most 2^24 bytes apart");
    return PK_OK;
}
bool bad_product(int64_t rows, int64_t N, int64_t K)
{
    return rows < 0 || N <= 0 || K <= 0 || rows > kMxProductMax || N > kMxProductMax || K > kMxDepthMax;
}

}  // namespace

extern "C" {

size_t pk_mx_row_bytes(int32_t format, int64_t cols)
{
    if ((format != PK_MXFP4 && format != PK_MXFP8) || cols <= 0 || cols > kMxMax) return 0;
    return (size_t)mx_row_bytes(format, cols);
}

pk_status pk_mx_quantize(const void* src, int32_t src_dtype, int64_t src_row_stride, int64_t n_rows, int64_t cols, int32_t format,
                         void* rows, int64_t row_stride, void* hip_stream)
{
    return guarded([&]() -> pk_status {
        const char* who = "pk_mx_quantize";
        if (format != PK_MXFP4 && format != PK_MXFP8) return fail(PK_EINVAL, std::string(who) + ": unknown format");
        pk_status rc = check_matrix_shape(who, n_rows, cols);
        if (rc != PK_OK) return rc;
        const char* bad = bad_matrix(src, src_dtype, src_row_stride, n_rows, cols);
        if (!bad) bad = bad_rows(rows, format, row_stride, n_rows, cols);
        if (bad) return fail(PK_EINVAL, std::string(who) + ": " + bad);
        if (n_rows == 0) return PK_OK;
        const auto run = format == PK_MXFP4 ? (src_dtype == PK_BF16 ? quantize_launch<PK_MXFP4, true> : quantize_launch<PK_MXFP4, false>)
                                            : (src_dtype == PK_BF16 ? quantize_launch<PK_MXFP8, true> : quantize_launch<PK_MXFP8, false>);
        return run(src, src_row_stride, n_rows, cols, rows, row_stride, static_cast<hipStream_t>(hip_stream));
    });
}

pk_status pk_mx_dequantize(const void* rows, int64_t row_stride, int64_t n_rows, int64_t cols, int32_t format,
                           void* dst, int32_t dst_dtype, int64_t dst_row_stride, void* hip_stream)
{
    return guarded([&]() -> pk_status {
        const char* who = "pk_mx_dequantize";
        if (format != PK_MXFP4 && format != PK_MXFP8) return fail(PK_EINVAL, std::string(who) + ": unknown format");
        pk_status rc = check_matrix_shape(who, n_rows, cols);
        if (rc != PK_OK) return rc;
        const char* bad = bad_matrix(dst, dst_dtype, dst_row_stride, n_rows, cols);
        if (!bad) bad = bad_rows(rows, format, row_stride, n_rows, cols);
        if (bad) return fail(PK_EINVAL, std::string(who) + ": " + bad);
        if (n_rows == 0) return PK_OK;
        const auto run = format == PK_MXFP4 ? (dst_dtype == PK_BF16 ? dequantize_launch<PK_MXFP4, true> : dequantize_launch<PK_MXFP4, false>)
                                            : (dst_dtype == PK_BF16 ? dequantize_launch<PK_MXFP8, true> : dequantize_launch<PK_MXFP8, false>);
        return run(rows, row_stride, n_rows, cols, dst, dst_row_stride, static_cast<hipStream_t>(hip_stream));
    });
}

size_t pk_mx_linear_workspace_bytes(int64_t M, int64_t N, int64_t K)
{
    if (bad_product(M, N, K)) { set_error("pk_mx_linear_workspace_bytes: bad sizes"); return 0; }
    return linear_layout(M, N, K).total;
}

pk_status pk_mx_linear(const void* x, int32_t x_dtype, int64_t x_row_stride, int64_t M, const void* w_rows, int64_t w_row_stride,
                       int64_t N, int64_t K, const float* bias, void* y, int32_t y_dtype, int64_t y_row_stride,
                       void* workspace, size_t ws_bytes, void* hip_stream)
{
    return guarded([&]() -> pk_status {
        const char* who = "pk_mx_linear";
        pk_status rc = check_product(who, M, N, K, w_row_stride);
        if (rc != PK_OK) return rc;
        const char* bad = bad_matrix(x, x_dtype, x_row_stride, M, K);
        if (!bad) bad = bad_matrix(y, y_dtype, y_row_stride, M, N);
        if (!bad) bad = bad_rows(w_rows, PK_MXFP4, w_row_stride, N, K);
        if (!bad && misaligned(bias, 4)) bad = "bias is not aligned to its elements";
        if (bad) return fail(PK_EINVAL, std::string(who) + ": " + bad);
        if (M == 0) return PK_OK;
        const LinearLayout L = linear_layout(M, N, K);
        if (!workspace) return fail(PK_EINVAL, std::string(who) + ": workspace is NULL");
        if (misaligned(workspace, kAlign)) return fail(PK_EWORKSPACE, std::string(who) + ": workspace must be 256-byte aligned");
        if (ws_bytes < L.total) return fail(PK_EWORKSPACE, std::string(who) + ": workspace is smaller than pk_mx_linear_workspace_bytes");
        hipStream_t stream = static_cast<hipStream_t>(hip_stream);
        const int64_t x_bytes = x_row_stride * (x_dtype == PK_BF16 ? 2 : 4);
        if (linear_few(M, N, K)) {
            const int waves = linear_few_waves(K);
            const auto few = x_dtype == PK_BF16 ? (y_dtype == PK_BF16 ? mx_linear_few_kernel<true, true> : mx_linear_few_kernel<true, false>)
                                                : (y_dtype == PK_BF16 ? mx_linear_few_kernel<false, true> : mx_linear_few_kernel<false, false>);
            MX_LAUNCH("mx_linear_few", few, dim3((unsigned)((N + 15) / 16)), dim3(64 * waves), static_cast<const char*>(x), x_bytes, (int)M,
                      static_cast<const uint8_t*>(w_rows), w_row_stride, (int)N, (int)K, bias, static_cast<char*>(y), y_row_stride);
            return PK_OK;
        }
        char* ws = static_cast<char*>(workspace);
        const RowGroups g(L.kp);
        const int64_t items = M * g.n, tiles = L.tiles_m * L.tiles_n;
        if (tiles * L.splits > kLaunchBlocks) return fail(PK_EOVERFLOW, std::string(who) + ": M * N is too large");
        uint32_t* codes = reinterpret_cast<uint32_t*>(ws);
        uint8_t* scales = reinterpret_cast<uint8_t*>(ws + L.scales);
        const auto round = x_dtype == PK_BF16 ? mx_linear_round_kernel<true> : mx_linear_round_kernel<false>;
        MX_LAUNCH("mx_linear_round", round, dim3(mx_blocks_for(items)), dim3(NT), static_cast<const char*>(x), x_bytes, (uint32_t)K,
                  g, codes, scales, items);
        const bool join = L.splits > 1;
        char* parts = ws + L.parts;
        const auto kernel = y_dtype == PK_BF16 && !join ? mx_linear_kernel<true> : mx_linear_kernel<false>;
        MX_LAUNCH("mx_linear", kernel, dim3((unsigned)((tiles * L.splits + 7) / 8 * 8)), dim3(256), reinterpret_cast<const uint8_t*>(codes), scales,
                  static_cast<const uint8_t*>(w_rows), w_row_stride, (int)M, (int)N, (int)K, (int)L.tiles_n, (int)tiles, (int)L.steps, (int)L.splits,
                  join ? nullptr : bias, join ? parts : static_cast<char*>(y), join ? L.ld : y_row_stride, M * L.ld * 4);
        if (join) {
            const int64_t n = M * (L.ld / 4);
            const auto sum = y_dtype == PK_BF16 ? mx_linear_join_kernel<true> : mx_linear_join_kernel<false>;
            MX_LAUNCH("mx_linear_join", sum, dim3(mx_blocks_for(n)), dim3(NT), reinterpret_cast<const float*>(parts), L.ld, M * L.ld, (int)L.splits, (int)N, n,
                      bias, static_cast<char*>(y), y_row_stride);
        }
        return PK_OK;
    });
}

size_t pk_mx_weight_grad_workspace_bytes(int64_t B, int64_t N, int64_t K)
{
    if (bad_product(B, N, K)) { set_error("pk_mx_weight_grad_workspace_bytes: bad sizes"); return 0; }
    return grad_layout(B, N, K).total;
}

pk_status pk_mx_weight_grad(const void* dy, int32_t dy_dtype, int64_t dy_row_stride, const void* x_rows, int64_t x_row_stride,
                            int64_t B, int64_t N, int64_t K, float* dw, int64_t dw_row_stride, int32_t accumulate,
                            void* workspace, size_t ws_bytes, void* hip_stream)
{
    return guarded([&]() -> pk_status {
        const char* who = "pk_mx_weight_grad";
        const pk_status rc = check_product(who, B, N, K, x_row_stride);
        if (rc != PK_OK) return rc;
        if (N > kMxGradStrideMax || (B > 1 && dy_row_stride > kMxGradStrideMax)) return fail(PK_EOVERFLOW, std::string(who) + ": N and the distance of dy's rows must be at most 2^24");
        const char* bad = bad_matrix(dy, dy_dtype, dy_row_stride, B, N);
        if (!bad) bad = bad_rows(x_rows, PK_MXFP8, x_row_stride, B, K);
        if (!bad) bad = bad_matrix(dw, PK_F32, dw_row_stride, N, K);
        if (bad) return fail(PK_EINVAL, std::string(who) + ": " + bad);
        if (!workspace) return fail(PK_EINVAL, std::string(who) + ": workspace is NULL");
        if (misaligned(workspace, kAlign)) return fail(PK_EWORKSPACE, std::string(who) + ": workspace must be 256-byte aligned");
        if (ws_bytes < pk_mx_weight_grad_workspace_bytes(B, N, K)) return fail(PK_EWORKSPACE, std::string(who) + ": workspace is smaller than pk_mx_weight_grad_workspace_bytes");
        hipStream_t stream = static_cast<hipStream_t>(hip_stream);
        const GradLayout L = grad_layout(B, N, K);
        const int64_t tiles = L.tiles;
        if (tiles * L.splits > kLaunchBlocks) return fail(PK_EOVERFLOW, std::string(who) + ": N * K is too large");
        const bool join = L.splits > 1;
        const GradJob job{static_cast<const char*>(dy), (B > 1 ? dy_row_stride : N) * (dy_dtype == PK_BF16 ? 2 : 4), static_cast<const uint8_t*>(x_rows), x_row_stride, B,
                          (int)N, (int)K, (int)L.tiles_n, (int)tiles, (int)L.steps, (int)L.splits, join ? static_cast<float*>(workspace) : dw,
                          join ? L.ld : dw_row_stride, N * L.ld, join ? 0 : accumulate};
        const auto kernel = dy_dtype == PK_BF16 ? mx_grad_bf16_kernel : mx_grad_f32_kernel;
        MX_LAUNCH("mx_grad", kernel, dim3((unsigned)((tiles * L.splits + 7) / 8 * 8)), dim3(256), job);
        if (join) {
            const int64_t items = N * (L.ld / 4);
            MX_LAUNCH("mx_grad_join", mx_grad_join_kernel, dim3(mx_blocks_for(items)), dim3(NT), static_cast<const float*>(workspace), L.ld, N * L.ld,
                      (int)L.splits, (int)K, items, dw, dw_row_stride, accumulate);
        }
        return PK_OK;
    });
}

}  // extern "C"
