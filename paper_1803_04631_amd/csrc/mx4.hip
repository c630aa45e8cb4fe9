// Matrices in microscaled 4-bit floating point, and the product with them: argument checks and launches; the kernels are in kernels_mx4.hpp.
#include "operators_host.hpp"

#include "kernels_mx4.hpp"

namespace {

int64_t blocks_of(int32_t cols) { return ((int64_t)cols + mlda::kMxBlock - 1) / mlda::kMxBlock; }

constexpr int32_t kMostProductCols = 1 << 24;    // tiles of rows have 32-bit numbers of pieces

// How a product's rows are held in 4 bits: few, and short ones of a small product, by each workgroup for itself, others in the workspace, in whole tiles of rows
// and whole stretches of steps.  With a launch for the rows, and so, us.  Up to 16 rows and 512 blocks (rows x columns x words, bf16): 1 x 1,000 x 141,000 24.3, 17.9;
// 8 x 1,000 x 40,009 10.8, 9.5; 16 x 500 x 40,009 8.6, 8.1; 16 x 1,000 x 3,000 8.5, 8.2, x 40,009 11.4, 12.0, x 141,000 27.9, 27.8; 1 x 16,384 x 3,000 16.0, 16.0.  But with
// more blocks 16 x 1,537 x 40,009 16.1, 18.8; 16 x 2,048 x 40,009 15.6, 19.4; 4 x 8,192 x 3,000 11.4, 14.8; 1 x 32,768 x 2,000 24.7, 27.8; with more rows 17 x 500 x 3,000 7.5, 8.1;
// 24 x 500 x 3,000 7.8, 9.4, x 40,009 9.3, 9.6; 32 x 500 x 40,009 10.1, 11.2.  Short rows: 24 x 256 x 40,009 7.6, 6.2; 1,000 x 32 x 5,000 fp32 12.6, 8.4; 65 x 128 x 64,000 bf16
// 9.8, 9.3; 1,000 x 128 x 4,000 bf16 9.3, 8.2; 1,000 x 224 x 2,300 bf16 9.3, 8.3; 250 x 256 x 8,000 fp16 8.6, 7.1.  But 1,000 x 32 x 16,000 bf16 15.6, 19.3;
// 2,000 x 128 x 4,000 bf16 11.4, 13.7; 2,000 x 200 x 4,000 bf16 12.1, 16.8; 300 x 500 x 3,000 bf16 9.4, 10.5.
bool few_rows(int64_t rows, int32_t cols) { return rows <= 16 && rows * blocks_of(cols) <= 512; }
bool short_rows(int64_t rows, int32_t cols, int32_t words) {
    return blocks_of(cols) <= 8 && rows <= ((int64_t)1 << 24) / std::max(blocks_of(cols), (int64_t)2) / words;
}
// Which products are few enough for a wave for each 32 x 32 of them; the others take tiles of 128 words and as many rows as a workgroup's waves have: 128, or
// 256 where there are that many tiles and rows.  1,000 columns, bf16, us, a wave for each, 128: 17 x 40,009 11.7, 14.0; 17 x 141,000 28.2, 34.2; 32 x 3,000 9.2, 9.2; 32 x 40,009 12.9, 13.7;
// 32 x 141,000 31.4, 32.1 (32 x 3,000 of 500 columns 8.4, 8.2, of 4,096 9.8, 17.9).  A wave for each, 128, 256: 300 x 3,000: 9.9, 10.1, -; 100 x 8,516: 10.0, 9.5, -; 300 x 5,000: 11.4, 10.5,
// 11.0; 65 x 141,000: 55, 29, 41; 500 x 141,000: 246, 66, 70; 2,048 x 141,000: 958, 246, 232; 2,932 x 1,120 of 9,205 columns: 85, 62, 63.
bool few_products(int64_t rows, int32_t words) { return rows <= 32 || words < mlda::kTileWords || (rows + 31) / 32 <= 1024 / (((int64_t)words + 31) / 32); }
bool many_products(int64_t rows, int32_t words) {
    return rows > 512 && (rows + 255) / 256 * (((int64_t)words + mlda::kTileWords - 1) / mlda::kTileWords) >= 4 * kCus;
}
int64_t held_rows(int64_t rows) { return (rows + 31) / 32 * 32; }
int64_t held_blocks(int32_t cols) {
    constexpr int64_t kEach = 2 * mlda::kAhead;
    return (blocks_of(cols) + kEach - 1) / kEach * kEach;
}
size_t held_bytes(int64_t rows, int32_t cols) {
    return few_rows(rows, cols) ? 0 : (size_t)held_rows(rows) * (size_t)held_blocks(cols) * (mlda::kMxBytes + 1);
}

int check_mx4(int64_t rows, int32_t cols, int32_t type) {
    if (rows < 0 || cols < 1 || cols > kMostCols) return refuse("4-bit matrix: need rows >= 0 and 1 <= cols <= 2^30");
    if (rows > ((int64_t)1 << 54) / cols) return refuse("4-bit matrix: need rows * cols <= 2^54");            // (whose bytes 64 bits count)
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

// A product's rows, in steps of two blocks.
int lay_out(const void* x, int64_t x_stride, uint8_t* codes, uint8_t* scales, int64_t rows, int32_t cols, int32_t type, int32_t steps, hipStream_t stream) {
    const int64_t most = std::max<int64_t>(1, 4 * kMostGroups / steps) * 32;         // of a launch
    for (int64_t row = 0; row < rows; row += most) {
        const int64_t n = std::min(most, rows - row), units = (n + 31) / 32 * steps;
        const mlda::MxArgs a{static_cast<const char*>(x) + row * x_stride * (int64_t)type_bytes(type), x_stride, codes + row * steps * 2 * mlda::kMxBytes,
                             scales + row * steps * 2, 0, cols, mlda::Divisor{}, false};
        constexpr int64_t kEach = mlda::kMxThreads / mlda::kWave;
        RC_TRY(with_type(type, [&](auto t) {
            hipLaunchKernelGGL((mlda::mx4_fragments_kernel<decltype(t)>), dim3((unsigned)((units + kEach - 1) / kEach)), dim3(mlda::kMxThreads), 0, stream, a, n,
                               mlda::divisor((uint32_t)steps));
            return launched("mx4_fragments_kernel");
        }));
    }
    return MLDA_OK;
}

template <class T, class X>
int multiply_few_of(mlda::MxLinearArgs a, mlda::MxArgs q, int32_t steps, hipStream_t stream) {
    constexpr bool kOwn = !std::is_void_v<X>;
    const unsigned lds = kOwn ? (unsigned)(std::min<int64_t>(a.rows, 32) * a.blocks * (mlda::kMxBytes + 1)) : 0;
    const int64_t waves = ((int64_t)a.words + mlda::kFewWords - 1) / mlda::kFewWords;
    // With fewer waves than SIMDs, and more slabs than a wave has on their way, four share their words.
    const bool split = waves * ((a.rows + 31) / 32) < 4 * kCus && a.blocks > 4 * mlda::kFewBlocks;
    const unsigned groups = (unsigned)(split ? waves : (waves + mlda::kFewWaves - 1) / mlda::kFewWaves);
    constexpr int64_t kMost = 65535 * 32;                    // rows of a launch
    const int64_t rows = a.rows;
    for (int64_t row = 0; row < rows; row += kMost) {
        a.rows = std::min(kMost, rows - row);
        const dim3 grid(groups, (unsigned)((a.rows + 31) / 32)), threads(mlda::kFewWaves * mlda::kWave);
        if (split) hipLaunchKernelGGL((mlda::mx4_few_kernel<T, X, true, 4>), grid, threads, lds, stream, a, q, steps);
        else if (kOwn && a.blocks <= mlda::kFewBlocks) hipLaunchKernelGGL((mlda::mx4_few_kernel<T, X, false, kOwn ? 1 : 4>), grid, threads, lds, stream, a, q, steps);
        else hipLaunchKernelGGL((mlda::mx4_few_kernel<T, X, false, 4>), grid, threads, lds, stream, a, q, steps);
        RC_TRY(launched("mx4_few_kernel"));
        if constexpr (kOwn) q.x = static_cast<const X*>(q.x) + a.rows * q.stride;
        a.x_codes += a.rows * steps * 2 * mlda::kMxBytes;
        a.x_scales += a.rows * steps * 2;
        a.y = static_cast<T*>(a.y) + a.rows * a.y_stride;
    }
    return MLDA_OK;
}

template <class T, int kWaves, int kChunk>
int multiply_tiles_of(const mlda::MxLinearArgs& m, int32_t steps, hipStream_t stream) {
    mlda::MxTilesArgs a{};
    a.m = m;
    a.steps = steps;
    a.once = passes_caches((double)m.rows * m.words * (double)sizeof(T));
    constexpr int kRows = kWaves * 32, kStepBytes = mlda::kTileWords * 2 * (mlda::kMxBytes + 1);
    const int64_t tiles = ((int64_t)m.words + mlda::kTileWords - 1) / mlda::kTileWords;
    a.passes = (uint32_t)((m.rows + kRows - 1) / kRows);
    if ((m.rows + kRows - 1) / kRows > ((int64_t)1 << 30) / tiles) return refuse("4-bit product: more than 2^30 tiles of rows and words");
    a.pass = mlda::divisor(a.passes);
    a.units = (uint32_t)(tiles * a.passes);
    const unsigned lds = (unsigned)(2 * std::min(kChunk, steps) * kStepBytes);
    const auto kernel = mlda::mx4_tiles_kernel<T, kWaves, kChunk>;
    if (lds > 48 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return set_error(MLDA_EHIP, "mx4_tiles_kernel's LDS", hipGetErrorString(e));
    }
    constexpr int64_t kFits = kCus * (8 / kWaves);           // workgroups that the registers of the chip hold
    hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>(a.units, kFits)), dim3(kWaves * mlda::kWave), lds, stream, a);
    return launched("mx4_tiles_kernel");
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
    if (cols > kMostProductCols) return refuse("4-bit product: need cols <= 2^24");
    *bytes = held_bytes(rows, cols);
    return MLDA_OK;
}

int mlda_mx_linear(const void* x, int64_t x_stride, const uint8_t* codes, const uint8_t* scales, const void* bias, void* y, int64_t y_stride,
                    int64_t rows, int32_t cols, int32_t words, int32_t type, int32_t out_type, int32_t bias_type, void* dev_workspace,
                    size_t workspace_bytes, void* hip_stream) {
    RC_TRY(check_mx4(rows, cols, type));
    if (words < 1 || words > kMostCols) return refuse("4-bit product: need 1 <= words <= 2^30");
    if (cols > kMostProductCols) return refuse("4-bit product: need cols <= 2^24");
    if (!known_type(out_type)) return refuse("4-bit product: unknown type of y");
    if (bias_type != out_type && bias_type != MLDA_FP32) return refuse("4-bit product: the bias has the type of y, or fp32");
    if (rows == 0) return MLDA_OK;
    RC_TRY(check_rows(x, x_stride, rows, cols, type, "4-bit product: x is null", "4-bit product: rows of x overlap or are not aligned to their type"));
    RC_TRY(check_rows(y, y_stride, rows, words, out_type, "4-bit product: y is null", "4-bit product: rows of y overlap or are not aligned to their type"));
    if (x == y) return refuse("4-bit product: y cannot be in the place of x");
    RC_TRY(check_codes(codes, scales));
    if (!aligned(bias, type_bytes(bias_type))) return refuse("4-bit product: the bias is not aligned to its type");
    const size_t need = held_bytes(rows, cols);
    if (need && (!dev_workspace || !aligned(dev_workspace, 16))) return refuse("4-bit product: the workspace is null or not aligned");
    if (workspace_bytes < need) return set_error(MLDA_ENOMEM, "4-bit product: the workspace is smaller than mlda_mx_linear_workspace_bytes");
    const hipStream_t stream = (hipStream_t)hip_stream;
    mlda::MxLinearArgs a{nullptr, nullptr, codes, scales, bias, bias_type == MLDA_FP32, y, y_stride, rows, words, (int32_t)blocks_of(cols)};
    if (!need || short_rows(rows, cols, words)) {
        const mlda::MxArgs q{x, x_stride, nullptr, nullptr, 0, cols, mlda::divisor((uint32_t)(blocks_of(cols) * mlda::kMxBlock * (int64_t)type_bytes(type) / 16)), false};
        return with_type(out_type, [&](auto t) {
            return with_type(type, [&](auto u) { return multiply_few_of<decltype(t), decltype(u)>(a, q, 0, stream); });
        });
    }
    const int64_t blocks = held_blocks(cols);
    uint8_t* x_codes = static_cast<uint8_t*>(dev_workspace);
    uint8_t* x_scales = x_codes + held_rows(rows) * blocks * mlda::kMxBytes;
    const int32_t steps = (int32_t)(blocks / 2);
    RC_TRY(lay_out(x, x_stride, x_codes, x_scales, rows, cols, type, steps, stream));
    a.x_codes = x_codes;
    a.x_scales = x_scales;
    return with_type(out_type, [&](auto t) {
        typedef decltype(t) T;
        if (few_products(rows, words)) return multiply_few_of<T, void>(a, mlda::MxArgs{}, steps, stream);
        if (many_products(rows, words)) return multiply_tiles_of<T, 8, 16>(a, steps, stream);
        return multiply_tiles_of<T, 4, 8>(a, steps, stream);
    });
}

}  // extern "C"
