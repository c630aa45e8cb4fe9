// Matrices in microscaled 4-bit floating point, and the product with them: argument checks and launches; the kernels are in kernels_mx4.hpp.
#include "operators_host.hpp"

#include "kernels_mx4.hpp"

namespace {

int64_t blocks_of(int32_t cols) { return ((int64_t)cols + mlda::kMxBlock - 1) / mlda::kMxBlock; }

int check_mx4(int64_t rows, int32_t cols, int32_t type) {
    if (rows < 0 || cols < 1 || cols > kMostCols) return refuse("4-bit matrix: need rows >= 0 and 1 <= cols <= 2^30");
    if (!known_type(type)) return refuse("4-bit matrix: unknown type");
    return MLDA_OK;
}

int check_codes(const void* codes, const void* scales) {
    if (!codes || !scales) return refuse("4-bit matrix: codes or scales are null");
    if (!aligned(codes, 16)) return refuse("4-bit matrix: codes are not aligned to 16 bytes");
    return MLDA_OK;
}

// Calls f(args, grid) for stretches of rows whose pieces have 32-bit numbers.
template <class F>
int for_pieces(const void* x, int64_t x_stride, const uint8_t* codes, const uint8_t* scales, int64_t rows, int32_t cols, int32_t type, F&& f) {
    const int64_t blocks = blocks_of(cols), per_row = blocks * mlda::kMxBlock * (int64_t)type_bytes(type) / 16;
    const int64_t most = std::max<int64_t>(1, ((int64_t)1 << 30) / per_row);
    for (int64_t row = 0; row < rows; row += most) {
        const int64_t n = std::min(most, rows - row);
        const mlda::MxArgs a{static_cast<const char*>(x) + row * x_stride * (int64_t)type_bytes(type), x_stride,
                             const_cast<uint8_t*>(codes) + row * blocks * mlda::kMxBytes, const_cast<uint8_t*>(scales) + row * blocks,
                             (uint32_t)(n * per_row), cols, mlda::divisor((uint32_t)per_row),
                             passes_caches((double)rows * cols * ((double)type_bytes(type) + 0.53))};
        constexpr int64_t kEach = mlda::kMxThreads * mlda::kMxPieces;
        RC_TRY(f(a, dim3((unsigned)((n * per_row + kEach - 1) / kEach))));
    }
    return MLDA_OK;
}

int quantize(const void* x, int64_t x_stride, uint8_t* codes, uint8_t* scales, int64_t rows, int32_t cols, int32_t type, hipStream_t stream) {
    return for_pieces(x, x_stride, codes, scales, rows, cols, type, [&](const mlda::MxArgs& a, dim3 grid) {
        return with_type(type, [&](auto t) {
            hipLaunchKernelGGL((mlda::mx4_quantize_kernel<decltype(t)>), grid, dim3(mlda::kMxThreads), 0, stream, a);
            return launched("mx4_quantize_kernel");
        });
    });
}

}  // namespace

extern "C" {

int mlda_mx_quantize(const void* x, int64_t x_stride, uint8_t* codes, uint8_t* scales, int64_t rows, int32_t cols, int32_t type,
                      void* hip_stream) {
    RC_TRY(check_mx4(rows, cols, type));
    if (rows == 0) return MLDA_OK;
    RC_TRY(check_rows(x, x_stride, rows, cols, type, "4-bit matrix: x is null", "4-bit matrix: rows of x overlap or are not aligned to their type"));
    RC_TRY(check_codes(codes, scales));
    return quantize(x, x_stride, codes, scales, rows, cols, type, (hipStream_t)hip_stream);
}

int mlda_mx_dequantize(const uint8_t* codes, const uint8_t* scales, void* x, int64_t x_stride, int64_t rows, int32_t cols, int32_t type,
                        void* hip_stream) {
    RC_TRY(check_mx4(rows, cols, type));
    if (rows == 0) return MLDA_OK;
    RC_TRY(check_rows(x, x_stride, rows, cols, type, "4-bit matrix: x is null", "4-bit matrix: rows of x overlap or are not aligned to their type"));
    RC_TRY(check_codes(codes, scales));
    return for_pieces(x, x_stride, codes, scales, rows, cols, type, [&](const mlda::MxArgs& a, dim3 grid) {
        return with_type(type, [&](auto t) {
            hipLaunchKernelGGL((mlda::mx4_dequantize_kernel<decltype(t)>), grid, dim3(mlda::kMxThreads), 0, (hipStream_t)hip_stream, a);
            return launched("mx4_dequantize_kernel");
        });
    });
}

int mlda_mx_linear_workspace_bytes(int64_t rows, int32_t cols, size_t* bytes) {
    if (!bytes) return refuse("bytes is null");
    RC_TRY(check_mx4(rows, cols, MLDA_FP32));
    *bytes = (size_t)rows * (size_t)blocks_of(cols) * (mlda::kMxBytes + 1);
    return MLDA_OK;
}

int mlda_mx_linear(const void* x, int64_t x_stride, const uint8_t* codes, const uint8_t* scales, const void* bias, void* y, int64_t y_stride,
                    int64_t rows, int32_t cols, int32_t words, int32_t type, int32_t out_type, int32_t bias_type, void* dev_workspace,
                    size_t workspace_bytes, void* hip_stream) {
    RC_TRY(check_mx4(rows, cols, type));
    if (words < 1 || words > kMostCols) return refuse("4-bit product: need 1 <= words <= 2^30");
    if (!known_type(out_type)) return refuse("4-bit product: unknown type of y");
    if (bias_type != out_type && bias_type != MLDA_FP32) return refuse("4-bit product: the bias has the type of y, or fp32");
    if (rows == 0) return MLDA_OK;
    RC_TRY(check_rows(x, x_stride, rows, cols, type, "4-bit product: x is null", "4-bit product: rows of x overlap or are not aligned to their type"));
    RC_TRY(check_rows(y, y_stride, rows, words, out_type, "4-bit product: y is null", "4-bit product: rows of y overlap or are not aligned to their type"));
    if (x == y) return refuse("4-bit product: y cannot be in the place of x");
    RC_TRY(check_codes(codes, scales));
    if (!aligned(bias, type_bytes(bias_type))) return refuse("4-bit product: the bias is not aligned to its type");
    const size_t blocks = (size_t)blocks_of(cols), need = (size_t)rows * blocks * (mlda::kMxBytes + 1);
    if (!dev_workspace || !aligned(dev_workspace, 16)) return refuse("4-bit product: the workspace is null or not aligned");
    if (workspace_bytes < need) return set_error(MLDA_ENOMEM, "4-bit product: the workspace is smaller than mlda_mx_linear_workspace_bytes");
    uint8_t* x_codes = static_cast<uint8_t*>(dev_workspace);
    uint8_t* x_scales = x_codes + (size_t)rows * blocks * mlda::kMxBytes;
    const hipStream_t stream = (hipStream_t)hip_stream;
    RC_TRY(quantize(x, x_stride, x_codes, x_scales, rows, cols, type, stream));
    return with_type(out_type, [&](auto t) {
        typedef decltype(t) T;
        constexpr int kTiles = 4;
        constexpr int64_t kMostRows = 65535 * 16 * kTiles;       // of a launch
        for (int64_t row = 0; row < rows; row += kMostRows) {
            const int64_t n = std::min(kMostRows, rows - row);
            const mlda::MxLinearArgs a{x_codes + (size_t)row * blocks * mlda::kMxBytes, x_scales + (size_t)row * blocks, codes, scales, bias,
                                       bias_type == MLDA_FP32, static_cast<T*>(y) + row * y_stride, y_stride, n, words, (int32_t)blocks};
            hipLaunchKernelGGL((mlda::mx4_linear_kernel<T, kTiles>), dim3((unsigned)((words + 63) / 64), (unsigned)((n + 16 * kTiles - 1) / (16 * kTiles))),
                               dim3(256), 0, stream, a);
            RC_TRY(launched("mx4_linear_kernel"));
        }
        return MLDA_OK;
    });
}

}  // extern "C"
