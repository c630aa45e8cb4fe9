// Dropout of the elements of a matrix, whose mask is drawn from a counter and never stored.
//
//   y = x / (1 - p) where u >= p 2^32, else 0   (+ residual)
//
// u is a 32-bit number of the element: 16 bits of Philox4x32-10 with the seed as key and the counter (column / 8, row, step, 1) as its
// upper half, of (column / 8, row, step, 2) as its lower.  The sampler's counters end in 0.  The upper half decides but for one element in 65,536, so the lower is drawn
// only where a wave has such an element: ten rounds serve eight elements, and p is exact to 2^-32 all the same.
#pragma once
#include "divisor.hpp"
#include "vec_io.hpp"

namespace mlda {

constexpr int kDropThreads = 256;
constexpr int kDropCols = 8;             // of one generator's call

struct DropoutArgs {
    const void* x;
    int64_t x_stride;
    const void* residual;                // null: none
    int64_t residual_stride;
    void* y;
    int64_t y_stride;
    uint32_t units;                      // of kDropCols columns, of all rows, below 2^31
    int32_t cols;
    Divisor per_row;
    uint64_t threshold;                  // 0 .. 2^32
    float scale;
    uint32_t key0, key1, step, first_row;
    const int64_t* more_steps;           // null: none
    bool once;
};

// The four words of Philox4x32-10.
__device__ __forceinline__ void philox_words(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1, uint32_t (&out)[4]) {
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    out[0] = c0;
    out[1] = c1;
    out[2] = c2;
    out[3] = c3;
}

// Bound by memory: 300,000 x 1,000 bf16 with residual 284 us, 6.3 TB/s; ten rounds take some 100 instructions, 13 an element.  A lane draws for eight
// neighbouring columns; where those are two pieces of 16 bytes (fp32) the lanes change them, so that a wave's loads and stores are whole lines
// (5,682 x 9,236 fp32 133 us without, so 72).
template <class T, bool kResidual>
__global__ __launch_bounds__(kDropThreads) void dropout_kernel(DropoutArgs a) {
    constexpr int P = kPack<T>, kPieces = kDropCols / P;
    const uint32_t wave_unit = blockIdx.x * (uint32_t)kDropThreads + threadIdx.x / kWave * kWave, unit = wave_unit + lane_id();
    // piece j of a lane: of unit j 64 / kPieces + lane / kPieces of the wave
    uint32_t row[kPieces];
    int32_t col[kPieces];
    bool there[kPieces];
    Raw rx[kPieces], rr[kPieces];
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
        const uint32_t of = wave_unit + j * (kWave / kPieces) + lane_id() / kPieces;
        there[j] = of < a.units;
        row[j] = a.per_row(min(of, a.units - 1));
        col[j] = (int32_t)(of - row[j] * a.per_row.by) * kDropCols + lane_id() % kPieces * P;
        if (!there[j]) continue;
        rx[j] = load_piece(static_cast<const T*>(a.x) + (int64_t)row[j] * a.x_stride, col[j], 0, a.cols, 0.0f, a.once);
        if (kResidual) rr[j] = load_piece(static_cast<const T*>(a.residual) + (int64_t)row[j] * a.residual_stride, col[j], 0, a.cols, 0.0f, a.once);
    }
    const uint32_t step = a.step + (a.more_steps ? (uint32_t)*a.more_steps : 0);
    const uint32_t upper = (uint32_t)(a.threshold >> 16), lower = (uint32_t)a.threshold & 0xffffu;
    const uint32_t drawn_row = a.per_row(min(unit, a.units - 1)), group = unit - drawn_row * a.per_row.by;
    uint32_t bits[4], number[kDropCols];
    philox_words(group, a.first_row + drawn_row, step, 1, a.key0, a.key1, bits);
    bool drawn = false;
    uint32_t kept = 0;
#pragma unroll
    for (int e = 0; e < kDropCols; ++e) {
        number[e] = e % 2 ? bits[e / 2] >> 16 : bits[e / 2] & 0xffffu;
        drawn |= number[e] == upper;
        kept |= (uint32_t)(number[e] >= upper) << e;
    }
    if (drawn) {
        philox_words(group, a.first_row + drawn_row, step, 2, a.key0, a.key1, bits);
#pragma unroll
        for (int e = 0; e < kDropCols; ++e) {
            const uint32_t low = e % 2 ? bits[e / 2] >> 16 : bits[e / 2] & 0xffffu;
            if (number[e] == upper && low < lower) kept &= ~(1u << e);
        }
    }
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
        uint32_t mine = kept;
        if constexpr (kPieces > 1) mine = (uint32_t)__shfl((int)kept, j * (kWave / kPieces) + lane_id() / kPieces, kWave) >> lane_id() % kPieces * P;
        if (!there[j]) continue;
        float v[P], w[P];
        unpack(rx[j], v, T());
        if (kResidual) unpack(rr[j], w, T());
#pragma unroll
        for (int e = 0; e < P; ++e) {
            v[e] = mine >> e & 1 ? v[e] * a.scale : 0.0f;                 // (whatever is dropped, NaN too, is 0)
            if (kResidual) v[e] += w[e];
        }
        store_piece(static_cast<T*>(a.y) + (int64_t)row[j] * a.y_stride, col[j], 0, a.cols, pack(v, T()), a.once);
    }
}

}  // namespace mlda
