// Matrices in microscaled 4-bit floating point, and the product with them.
//
// A row is cut into blocks of 32 columns.  A block's scale is the least 2^s, s >= -127, of which 7 exceed the block's greatest magnitude (what is
// below 7 rounds to 6 at most, the greatest number held; with the exponent of the greatest magnitude alone the error of normal numbers is
// 11.5% instead of 11.2, of evenly spread ones 14.4 instead of 9.9), and an element is x / 2^s, rounded to nearest even among 0, 1/2, 1, 3/2, 2,
// 3, 4, 6 with a sign: 2 bits of exponent and one of mantissa.  Scales are held as the byte s + 127; 255 stands for NaN, for a block
// with NaN or infinity in it.
#pragma once
#include "divisor.hpp"
#include "vec_io.hpp"

namespace mlda {

constexpr int kMxBlock = 32;             // columns that share a scale
constexpr int kMxBytes = kMxBlock / 2;   // of a block's codes

constexpr int kMxThreads = 256;
constexpr int kMxPieces = 4;             // 16-byte pieces that a thread has in flight

struct MxArgs {
    const void* x;
    int64_t stride;
    uint8_t* codes;
    uint8_t* scales;
    uint32_t pieces;                     // of all rows, below 2^31
    int32_t cols;
    Divisor per_row;                     // pieces to a row of whole blocks
    bool once;
};

// The greatest of 32 columns' numbers: `kLanes` (4 or 8) neighbouring lanes have a block.
template <int kLanes>
__device__ __forceinline__ uint32_t block_max(uint32_t v) {
    auto with = [&](auto ctrl) {
        v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xf, 0xf, false));
    };
    with(std::integral_constant<int, 0xb1>());                             // quad_perm: 1 0 3 2
    with(std::integral_constant<int, 0x4e>());                             // 2 3 0 1
    if constexpr (kLanes == 8) with(std::integral_constant<int, 0x141>()); // row_half_mirror
    return v;
}

// The scale's byte for the bits of the greatest magnitude (NaN's are above infinity's, and those above every number's).
__device__ __forceinline__ uint32_t mx_scale(uint32_t most) {
    if (most >= 0x7f800000u) return 255;
    return (uint32_t)max((int)(most >> 23) - 2 + (int)((most & 0x7fffffu) >= 0x600000u), 0);
}

// A scale as fp32; the conversions take only its exponent (2^-127 is no normal number, its exponent's bits are 0 too).
__device__ __forceinline__ float mx_factor(uint32_t scale) { return __uint_as_float(scale ? scale << 23 : 0x400000u); }

// Bound by memory: read once, a quarter or less of it written.  A lane has the 16 bytes of a piece, so that a wave reads whole lines.
template <class T>
__global__ __launch_bounds__(kMxThreads) void mx4_quantize_kernel(MxArgs a) {
    constexpr int P = kPack<T>, kLanes = kMxBlock / P;
    const uint32_t first = blockIdx.x * (uint32_t)(kMxThreads * kMxPieces) + threadIdx.x;
    Raw r[kMxPieces];
#pragma unroll
    for (int j = 0; j < kMxPieces; ++j) {
        const uint32_t piece = first + j * kMxThreads;
        if (piece >= a.pieces) continue;                                   // (whole blocks: their lanes are all there, or none)
        const uint32_t row = a.per_row(piece);
        const int32_t col = (int32_t)(piece - row * a.per_row.by) * P;
        r[j] = load_piece(static_cast<const T*>(a.x) + (int64_t)row * a.stride, col, 0, a.cols, 0.0f, a.once);
    }
#pragma unroll
    for (int j = 0; j < kMxPieces; ++j) {
        const uint32_t piece = first + j * kMxThreads;
        if (piece >= a.pieces) continue;
        float v[P];
        unpack(r[j], v, T());
        uint32_t most = 0;
#pragma unroll
        for (int e = 0; e < P; ++e) most = max(most, __float_as_uint(v[e]) & 0x7fffffffu);
        const uint32_t scale = mx_scale(block_max<kLanes>(most));
        const float f = mx_factor(scale);
        uint32_t code = 0;
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[0], v[1], f, 0);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[2], v[3], f, 1);
        if constexpr (P == 8) {
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[4], v[5], f, 2);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[6], v[7], f, 3);
        }
        if (scale == 255) code = 0;
        if constexpr (P == 8) reinterpret_cast<uint32_t*>(a.codes)[piece] = code;
        else reinterpret_cast<uint16_t*>(a.codes)[piece] = (uint16_t)code;
        if (piece % kLanes == 0) a.scales[piece / kLanes] = (uint8_t)scale;
    }
}

// The numbers that codes and scales stand for.  Bound by memory: what is written.
template <class T>
__global__ __launch_bounds__(kMxThreads) void mx4_dequantize_kernel(MxArgs a) {
    constexpr int P = kPack<T>, kLanes = kMxBlock / P;
    typedef float F2 __attribute__((ext_vector_type(2)));
    const uint32_t first = blockIdx.x * (uint32_t)(kMxThreads * kMxPieces) + threadIdx.x;
    uint32_t code[kMxPieces], scale[kMxPieces];
#pragma unroll
    for (int j = 0; j < kMxPieces; ++j) {
        const uint32_t piece = first + j * kMxThreads;
        if (piece >= a.pieces) continue;
        if constexpr (P == 8) code[j] = reinterpret_cast<const uint32_t*>(a.codes)[piece];
        else code[j] = reinterpret_cast<const uint16_t*>(a.codes)[piece];
        scale[j] = a.scales[piece / kLanes];
    }
#pragma unroll
    for (int j = 0; j < kMxPieces; ++j) {
        const uint32_t piece = first + j * kMxThreads;
        if (piece >= a.pieces) continue;
        const uint32_t row = a.per_row(piece);
        const int32_t col = (int32_t)(piece - row * a.per_row.by) * P;
        const float f = mx_factor(scale[j]);
        float v[P];
        auto pair = [&](auto which) {
            constexpr int k = decltype(which)::value;
            const F2 two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[j], f, k);
            v[2 * k] = two[0];
            v[2 * k + 1] = two[1];
        };
        pair(std::integral_constant<int, 0>());
        pair(std::integral_constant<int, 1>());
        if constexpr (P == 8) {
            pair(std::integral_constant<int, 2>());
            pair(std::integral_constant<int, 3>());
        }
        T* x = static_cast<T*>(const_cast<void*>(a.x)) + (int64_t)row * a.stride;
        store_piece(x, col, 0, a.cols, pack(v, T()), a.once);
    }
}

// ---------------------------------------------------------------- product
typedef int Codes __attribute__((ext_vector_type(4)));      // a block's
typedef float Acc __attribute__((ext_vector_type(4)));

struct MxLinearArgs {
    const uint8_t* x_codes;
    const uint8_t* x_scales;
    const uint8_t* codes;
    const uint8_t* scales;
    const void* bias;
    bool bias_fp32;
    void* y;
    int64_t y_stride;
    int64_t rows;
    int32_t words;
    int32_t blocks;                      // to a row
};

// acc += the products of 16 words (a) and 16 rows (b) over four blocks: lane l has the block l / 16 of word or row l % 16, and gets words
// 4 (l / 16) .. + 3 of row l % 16.  Products are exact, their sum is rounded once to fp32 (within 0.7 units of roundoff of the sum of magnitudes, as measured).
__device__ __forceinline__ Acc mx4_mfma(Codes a, uint32_t a_scale, Codes b, uint32_t b_scale, Acc acc) {
    typedef int Wide __attribute__((ext_vector_type(8)));
    const Wide x = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, y = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, acc, 4, 4, 0, (int)a_scale, 0, (int)b_scale);
}

template <class T>
__device__ __forceinline__ float bias_at(const MxLinearArgs& a, int32_t word) {
    if (!a.bias) return 0.0f;
    return a.bias_fp32 ? static_cast<const float*>(a.bias)[word] : (float)static_cast<const T*>(a.bias)[word];
}

// A wave has 16 words and 16 kTiles rows.
template <class T, int kTiles>
__global__ __launch_bounds__(256) void mx4_linear_kernel(MxLinearArgs a) {
    const int lane = lane_id(), at = lane % 16, part = lane / 16;
    const int64_t word0 = ((int64_t)blockIdx.x * 4 + threadIdx.x / kWave) * 16;
    if (word0 >= a.words) return;
    const int64_t row0 = (int64_t)blockIdx.y * 16 * kTiles;
    const int64_t word = min(word0 + at, (int64_t)a.words - 1);            // (what comes of the lanes past the end is not stored)
    Acc acc[kTiles] = {};
    for (int32_t b = part; b - part < a.blocks; b += 4) {
        const bool there = b < a.blocks;
        auto load = [&](const uint8_t* codes, int64_t row, Codes& c) {
            c = there ? *reinterpret_cast<const Codes*>(codes + (row * a.blocks + b) * kMxBytes) : Codes{0, 0, 0, 0};
        };
        Codes w, x;
        load(a.codes, word, w);
        const uint32_t ws = there ? a.scales[word * a.blocks + b] : 127;
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const int64_t row = min(row0 + 16 * t + at, a.rows - 1);
            load(a.x_codes, row, x);
            const uint32_t xs = there ? a.x_scales[row * a.blocks + b] : 127;
            acc[t] = mx4_mfma(w, ws, x, xs, acc[t]);
        }
    }
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        const int64_t row = row0 + 16 * t + at;
        if (row >= a.rows) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t n = word0 + 4 * part + i;
            if (n < a.words) static_cast<T*>(a.y)[row * a.y_stride + n] = (T)(acc[t][i] + bias_at<T>(a, (int32_t)n));
        }
    }
}

}  // namespace mlda
