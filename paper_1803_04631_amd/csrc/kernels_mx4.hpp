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

// The codes of the 16 bytes of a block that a lane has, and the block's scale.
template <class T>
__device__ __forceinline__ uint32_t mx4_codes(const float (&v)[kPack<T>], uint32_t& scale) {
    constexpr int P = kPack<T>;
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < P; ++e) most = max(most, __float_as_uint(v[e]) & 0x7fffffffu);
    scale = mx_scale(block_max<kMxBlock / P>(most));
    const float f = mx_factor(scale);
    uint32_t code = 0;
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[0], v[1], f, 0);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[2], v[3], f, 1);
    if constexpr (P == 8) {
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[4], v[5], f, 2);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[6], v[7], f, 3);
    }
    return scale == 255 ? 0 : code;
}

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
        uint32_t scale;
        const uint32_t code = mx4_codes<T>(v, scale);
        if constexpr (P == 8) reinterpret_cast<uint32_t*>(a.codes)[piece] = code;
        else reinterpret_cast<uint16_t*>(a.codes)[piece] = (uint16_t)code;
        if (piece % kLanes == 0) a.scales[piece / kLanes] = (uint8_t)scale;
    }
}

// The same for a product's rows, in the order in which the matrix instructions want them: of 32 rows and two blocks (a step) 1,024 bytes, lane by lane,
// and of four steps a word of scales for each lane.  Steps behind the row's end are zeros.  A wave has 32 rows of a step, so that it writes whole lines.
template <class T>
__global__ __launch_bounds__(kMxThreads) void mx4_fragments_kernel(MxArgs a, int64_t rows, Divisor steps) {
    constexpr int P = kPack<T>, kLanes = kMxBlock / P, kRows = kWave / (2 * kLanes);       // rows of a load
    const uint32_t unit = blockIdx.x * (uint32_t)(kMxThreads / kWave) + threadIdx.x / kWave, tile = steps(unit), step = unit - tile * steps.by;
    const int lane = lane_id(), in = lane % (2 * kLanes);
    const int64_t row0 = (int64_t)tile * 32 + lane / (2 * kLanes);
    if ((int64_t)tile * 32 >= rows) return;
    Raw r[32 / kRows];
#pragma unroll
    for (int j = 0; j < 32 / kRows; ++j)
        r[j] = load_piece(static_cast<const T*>(a.x) + min(row0 + j * kRows, rows - 1) * a.stride, (int64_t)step * 2 * kMxBlock + in * P, 0, a.cols, 0.0f, false);
#pragma unroll
    for (int j = 0; j < 32 / kRows; ++j) {
        float v[P];
        unpack(r[j], v, T());
        uint32_t scale;
        const uint32_t code = mx4_codes<T>(v, scale);
        const int lane_of = in / kLanes * 32 + lane / (2 * kLanes) + j * kRows;
        const int64_t to = ((int64_t)unit * kWave + lane_of) * kLanes + in % kLanes;
        if constexpr (P == 8) reinterpret_cast<uint32_t*>(a.codes)[to] = code;
        else reinterpret_cast<uint16_t*>(a.codes)[to] = (uint16_t)code;
        if (in % kLanes == 0) a.scales[(((int64_t)tile * (steps.by / 4) + step / 4) * kWave + lane_of) * 4 + step % 4] = (uint8_t)scale;
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

template <class T>
__device__ __forceinline__ float bias_at(const MxLinearArgs& a, int32_t word) {
    if (!a.bias) return 0.0f;
    return a.bias_fp32 ? static_cast<const float*>(a.bias)[word] : (float)static_cast<const T*>(a.bias)[word];
}

// acc += the products of 32 rows (a) and 32 words (b) over two blocks: lane l has the block l / 32 of row or word l % 32, and gets, in element j,
// row 8 (j / 4) + 4 (l / 32) + j % 4 of word l % 32.  Scales: the bytes kA and kB.  Products are exact; a sum of 64 and what was there is rounded once (within 0.7
// units of roundoff of the sum of magnitudes, as measured).  (7,500 TFLOP/s of equal numbers, 6,600 of random ones; the form for 16 x 16 x 128 4,190.)
typedef float Acc __attribute__((ext_vector_type(16)));
template <int kA, int kB>
__device__ __forceinline__ Acc mx4_mfma(Codes a, uint32_t a_scales, Codes b, uint32_t b_scales, Acc acc) {
    typedef int Wide __attribute__((ext_vector_type(8)));
    const Wide x = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, y = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, acc, 4, 4, kA, (int)a_scales, kB, (int)b_scales);
}

// A row's scales from a block on, eight, as they lie there: of a last eight that are short those that end with the row.
__device__ __forceinline__ uint64_t load_scales(const uint8_t* row, int32_t first, int32_t blocks) {
    typedef uint64_t Anywhere __attribute__((aligned(1), may_alias));
    uint64_t s = 0;
    if (blocks >= 8) {
        s = *reinterpret_cast<const Anywhere*>(row + min(first, blocks - 8));
    } else {
        for (int c = blocks; c-- > 0;) s = s << 8 | row[c];
        s <<= 8 * (8 - blocks);
    }
    return s;
}
// Moves those of a short eight to where the others' are; ones behind them (NaN times zero would be NaN).
__device__ __forceinline__ uint64_t placed_scales(uint64_t s, int32_t first, int32_t blocks) {
    const int short_by = min(max(first + 8 - blocks, 0), 8) * 8;
    return short_by == 0 ? s : short_by == 64 ? 0x7f7f7f7f7f7f7f7full : s >> short_by | 0x7f7f7f7f7f7f7f7full << (64 - short_by);
}

// Few rows (or words).  A wave has 32 words and 32 rows.  Its words' codes come straight from memory, 128 bytes of a word at a time (a line, or two that
// the next slab meets again) and kFewAhead such slabs on their way, and through LDS into the instructions' order: bound by reading them.  Rows that are few or short enough are put into 4 bits by each workgroup for itself, while its words' codes are on their way (X: their type); others
// (X = void) are laid out by mx4_fragments_kernel and come from the L2 cache.  With kSplit the four waves of a workgroup share their words'
// slabs, and their sums are joined in a fixed order.
constexpr int kFewBlocks = 8;            // of a slab
constexpr int kFewWaves = 4;
constexpr int kFewWords = 32;            // of a wave

template <class T, class X, bool kSplit, int kFewAhead>
__global__ __launch_bounds__(kFewWaves * kWave) void mx4_few_kernel(MxLinearArgs a, MxArgs q, int32_t steps) {
    constexpr bool kOwn = !std::is_void_v<X>;
    extern __shared__ Codes few_room[];                    // own rows: [block][row], then their scales; the parts of the sums
    __shared__ Codes turned[kFewWaves][kFewWords * kFewBlocks];            // a word's blocks turned by its number, so that eight lanes that read a block of eight words meet all banks
    __shared__ Acc sums[kSplit ? kFewWaves - 1 : 1][kWave];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), col = lane % 32, part = lane / 32;
    const int64_t row0 = (int64_t)blockIdx.y * 32;
    const int rows = (int)min((int64_t)32, a.rows - row0);
    const int64_t word0 = ((int64_t)blockIdx.x * (kSplit ? 1 : kFewWaves) + (kSplit ? 0 : wave)) * kFewWords;
    const int64_t word = min(word0 + col, (int64_t)a.words - 1);           // (what comes of the lanes past the end is not stored)
    const uint8_t* scales = a.scales + word * a.blocks;
    const int32_t slabs = (a.blocks + kFewBlocks - 1) / kFewBlocks, begin = kSplit ? wave : 0, stride = kSplit ? kFewWaves : 1, block = lane % kFewBlocks;
    const uint8_t* from[4];                                // of the lane's four words
#pragma unroll
    for (int i = 0; i < 4; ++i) from[i] = a.codes + min(word0 + 8 * i + lane / kFewBlocks, (int64_t)a.words - 1) * a.blocks * kMxBytes;
    Codes x[2][4];                                         // rows that are laid out: of this slab and the next
    uint32_t xs[2];
    auto fetch_rows = [&](int buffer, int32_t slab) {
        if (kOwn || slab >= slabs) return;
        const Codes* const from_rows = reinterpret_cast<const Codes*>(a.x_codes) + ((int64_t)blockIdx.y * steps + slab * 4) * kWave + lane;
#pragma unroll
        for (int s = 0; s < 4; ++s) x[buffer][s] = from_rows[s * kWave];
        xs[buffer] = reinterpret_cast<const uint32_t*>(a.x_scales)[((int64_t)blockIdx.y * (steps / 4) + slab) * kWave + lane];
    };
    static_assert(kFewAhead % 2 == 0 || kOwn, "rows that are laid out take turns in two places");
    fetch_rows(0, begin);
    fetch_rows(1, begin + stride);
    Codes w[kFewAhead][4];
    uint64_t ws[kFewAhead];
    auto fetch = [&](int buffer, int32_t slab) {
        if (slab >= slabs) return;
        const int64_t at = (int64_t)min(slab * kFewBlocks + block, a.blocks - 1) * kMxBytes;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[buffer][i] = *reinterpret_cast<const Codes*>(from[i] + at);
        ws[buffer] = load_scales(scales, slab * kFewBlocks, a.blocks);
    };
#pragma unroll
    for (int k = 0; k < kFewAhead; ++k) fetch(k, begin + k * stride);

    uint8_t* const own_scales = reinterpret_cast<uint8_t*>(few_room + a.blocks * rows);
    if constexpr (kOwn) {
        constexpr int P = kPack<X>, kLanes = kMxBlock / P;
        for (uint32_t piece = threadIdx.x; piece < q.per_row.by * (uint32_t)rows; piece += kFewWaves * kWave) {
            const uint32_t row = q.per_row(piece), in = piece - row * q.per_row.by, block = in / kLanes;
            float v[P];
            unpack(load_piece(static_cast<const X*>(q.x) + (row0 + row) * q.stride, (int64_t)in * P, 0, q.cols, 0.0f, false), v, X());
            uint32_t scale;
            const uint32_t code = mx4_codes<X>(v, scale);
            const uint32_t to = (block * (uint32_t)rows + row) * kLanes + in % kLanes;
            if constexpr (P == 8) reinterpret_cast<uint32_t*>(few_room)[to] = code;
            else reinterpret_cast<uint16_t*>(few_room)[to] = (uint16_t)code;
            if (in % kLanes == 0) own_scales[block * (uint32_t)rows + row] = (uint8_t)scale;
        }
        __syncthreads();
    }

    Acc acc = {};
    auto use = [&](int buffer, int32_t slab) {
        if (slab >= slabs) return;
        const int32_t first = slab * kFewBlocks;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            turned[wave][(8 * i + lane / kFewBlocks) * kFewBlocks + (block ^ (lane / kFewBlocks))] = first + block < a.blocks ? w[buffer][i] : Codes{0, 0, 0, 0};
        const uint64_t word_scales = placed_scales(ws[buffer], first, a.blocks) >> 8 * part;
        __builtin_amdgcn_wave_barrier();                   // (a wave's own room: its reads and writes are in order)
        auto step = [&](auto which) {
            constexpr int s = decltype(which)::value;
            if (first + 2 * s >= a.blocks) return;
            const Codes wc = turned[wave][col * kFewBlocks + ((2 * s + part) ^ (col & 7))];
            Codes xc;
            uint32_t row_scale;
            if constexpr (kOwn) {
                const int at = min(first + 2 * s + part, a.blocks - 1) * rows + min(col, rows - 1);
                xc = few_room[at];
                row_scale = own_scales[at];
            } else {
                xc = x[buffer % 2][s];
                row_scale = xs[buffer % 2];
            }
            acc = mx4_mfma<kOwn ? 0 : s, s % 2 * 2>(xc, row_scale, wc, (uint32_t)(word_scales >> s / 2 * 32), acc);
        };
        step(std::integral_constant<int, 0>());
        step(std::integral_constant<int, 1>());
        step(std::integral_constant<int, 2>());
        step(std::integral_constant<int, 3>());
        __builtin_amdgcn_wave_barrier();
    };
    for (int32_t slab = begin; slab < slabs; slab += kFewAhead * stride) {
#pragma unroll
        for (int k = 0; k < kFewAhead; ++k) {
            use(k, slab + k * stride);
            fetch_rows(k % 2, slab + (k + 2) * stride);
            fetch(k, slab + (k + kFewAhead) * stride);
        }
    }
    if constexpr (kSplit) {
        if (wave > 0) sums[wave - 1][lane] = acc;
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int k = 0; k < kFewWaves - 1; ++k) acc += sums[k][lane];
    }
    if (word0 + col >= a.words) return;
    const float bias = bias_at<T>(a, (int32_t)word);
    T* const y = static_cast<T*>(a.y) + row0 * a.y_stride + word0 + col;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const int row = 8 * (j / 4) + 4 * part + j % 4;
        if (row < rows) y[row * a.y_stride] = (T)(acc[j] + bias);
    }
}

// Many rows.  A workgroup holds the codes of 128 words in LDS, as the matrix instructions want them, and goes through the rows: a wave has 32 of them at a
// time, whose codes (laid out by mx4_fragments_kernel) come straight from the L2 cache, three steps ahead.  So the waves wait for each other only where
// the words change, and the next words are on their way before.  (Words and rows both through LDS, 256 x 128 a workgroup: 2,048 x 141,000 x 1,000 bf16 took 270 us,
// LDS and matrix instructions in turn; words held, 239, or 229 with the next ones sent for.)
//
// The columns of an instruction's result are the words 4 c + i of its four matrices i: a lane has four neighbouring words of a row, and a
// wave stores 256 bytes or more of it at once.
//
// Bound, at 1,000 columns, by products and stores that overlap only in part: 2,048 x 141,000 bf16 takes 233 us (212 with weights that are all zeros, for which the clock stays
// higher), the products without stores 176, stores alone 169, matrix instructions alone 90.  At 100 columns by writing: a line that two workgroups write a part of
// costs memory more than two lines do, so that rows of 141,000 words, each 16 bytes further off a line than the one before, take 169 us and rows of 140,928, which are
// whole lines, 129.  (Rows held in registers by waves that go along the words and write whole lines only, as what is left of a line is kept in LDS, write at 110, but
// with the products it took 284 .. 318: what the lines cost in instructions is more than they save.  Rows' codes 7 steps ahead: no difference.)
//
// At thousands of columns no unit is used up: 3,822 x 7,232 x 8,628 bf16, 199 us, has its matrix instructions busy for 32% of the cycles and LDS for 31 (both would be at
// the full rate: a wave's step is 128 cycles of matrix instructions and 4,352 bytes of LDS, 34 cycles, and four SIMDs share the LDS).  Its waves wait 45% of their
// time to issue and 26% for data.  195 registers, two waves to a SIMD; 31 to 34 scalar registers are kept in lanes of a vector register.
constexpr int kAhead = 4;                // steps of two blocks, which share a word of scales
constexpr int kTileWords = 128;

// Four neighbouring elements, wherever they lie.
template <class T>
__device__ __forceinline__ void store_four(T* p, const float (&v)[4], bool once) {
    typedef T Four __attribute__((ext_vector_type(4)));
    typedef Four Anywhere __attribute__((aligned(sizeof(T)), may_alias));
    const Four four = {(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
    if (once) __builtin_nontemporal_store(four, reinterpret_cast<Anywhere*>(p));
    else *reinterpret_cast<Anywhere*>(p) = four;
}

struct MxTilesArgs {
    MxLinearArgs m;                      // x in the order above, kTileWords words at least
    int32_t steps;                       // of two blocks, a multiple of kAhead
    uint32_t passes;                     // through all rows
    uint32_t units;                      // word tiles times passes
    Divisor pass;                        // by passes
    bool once;
};

// kChunk: steps that are held at a time, twice: those that are multiplied, and those that were before or will be next.
template <class T, int kWaves, int kChunk>
__global__ __launch_bounds__(kWaves * kWave, 2) void mx4_tiles_kernel(MxTilesArgs a) {
    constexpr int kThreads = kWaves * kWave, kPieces = kTileWords * 2 * kChunk / kThreads;
    static_assert(kTileWords * kChunk / 4 == kThreads, "a thread has the scales of eight blocks");
    // [slot][step][i][lane]; a lane's place is turned by its block's number, so that neighbouring blocks of a word do not meet in a bank
    extern __shared__ Codes held[];
    const MxLinearArgs& m = a.m;
    const int32_t slot_steps = min(kChunk, a.steps), chunks = (a.steps + kChunk - 1) / kChunk;
    uint32_t* const held_scales = reinterpret_cast<uint32_t*>(held + 2 * slot_steps * 4 * kWave);        // [slot][step][lane], a byte for each i
    const int thread = (int)threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(thread / kWave), col = lane % 32, part = lane / 32;
    // Whole rounds of tiles first, neighbouring tiles in neighbouring workgroups of an XCD, so that all that is written at a time is long runs of the same
    // rows; what is left of the tiles is cut into equal parts.
    const uint32_t groups = gridDim.x, group = groups % 8 ? blockIdx.x : blockIdx.x % 8 * (groups / 8) + blockIdx.x / 8;
    const uint32_t rounds = a.units / a.passes / groups, whole = rounds * a.passes, left = a.units - whole * groups;
    const uint32_t begin = (uint32_t)((uint64_t)left * group / groups), end = (uint32_t)((uint64_t)left * (group + 1) / groups), count = whole + (end - begin);
    if (count == 0) return;
    auto tile_of = [&](uint32_t n, uint32_t& pass) {
        const uint32_t unit = n < whole ? n : begin + (n - whole), in_round = a.pass(unit);
        pass = unit - in_round * a.passes;
        return (int32_t)(n < whole ? in_round * groups + group : rounds * groups + in_round);
    };

    // The last tile ends with the words, and does some of the one before again, the same bits: the workgroup that has it is what a launch waits for (2,048 x
    // 20,095 words of 100 columns bf16 41 us with a question for each row's last words, so 28).
    auto first_word = [&](int32_t tile) { return min((int64_t)tile * kTileWords, (int64_t)m.words - kTileWords); };

    // The words' codes and scales of a chunk: on their way, then held.  A thread has block thread % kIn of the words thread / kIn + 16 j; places in a
    // tile fit 32 bits, and what can be is worked out beforehand (2,932 x 9,205 x 1,120 fp32 68.8 us with all of it worked out for each chunk, so 64.8).
    constexpr int kIn = 2 * kChunk;
    static_assert(kThreads / kIn == 16 && kPieces * 16 == kTileWords, "words of a thread are 16 apart");
    Codes way[kPieces];
    uint64_t way_scales;
    const int scale_word = thread % kTileWords, scale_block = thread / kTileWords * 8, in = thread % kIn;
    const uint32_t first_code = (uint32_t)(thread / kIn) * (uint32_t)m.blocks * kMxBytes, first_scale = (uint32_t)scale_word * (uint32_t)m.blocks;
    auto send_for = [&](int32_t tile, int32_t chunk) {
        const int64_t word0 = first_word(tile);
        const uint8_t* const codes = m.codes + (word0 * m.blocks + chunk * kIn) * kMxBytes;
        const uint32_t at = first_code + (uint32_t)min(in, m.blocks - 1 - chunk * kIn) * kMxBytes;
#pragma unroll
        for (int j = 0; j < kPieces; ++j) way[j] = *reinterpret_cast<const Codes*>(codes + (int64_t)(16 * j) * m.blocks * kMxBytes + at);
        way_scales = load_scales(m.scales + word0 * m.blocks + first_scale, chunk * kIn + scale_block, m.blocks);
    };
    // The place of word 16 j + 4 k + i is 4 j + k, turned by n: 8 (j / 2) + (k ^ n), or that with its third bit turned.
    const int place = thread / kIn / 4 ^ (in & 7), other_place = 4 - 2 * (place & 4);
    Codes* const to_even = held + (in / 2 * 4 + thread / kIn % 4) * kWave + in % 2 * 32 + place;
    uint8_t* const to_scales = reinterpret_cast<uint8_t*>(held_scales + scale_block / 2 * kWave + scale_word / 4) + scale_word % 4;
    auto hold = [&](int slot, int32_t chunk) {             // (rows are zeros behind their end: codes there may be any)
        Codes* const to = to_even + slot * slot_steps * 4 * kWave;
        if (in / 2 < slot_steps) {
#pragma unroll
            for (int j = 0; j < kPieces; ++j) to[j / 2 * 8 + (j % 2 ? other_place : 0)] = way[j];
        }
        uint64_t s = way_scales;
        if ((chunk + 1) * kIn > m.blocks) s = placed_scales(s, chunk * kIn + scale_block, m.blocks);
        if (scale_block / 2 < slot_steps) {
            uint8_t* const scales_to = to_scales + slot * slot_steps * kWave * 4;
#pragma unroll
            for (int c = 0; c < 8; ++c) scales_to[(c / 2 * kWave + c % 2 * 32) * 4] = (uint8_t)(s >> 8 * c);
        }
    };

    const int64_t last_tile = (m.rows - 1) / 32;
    const Codes* x = nullptr;
    const uint32_t* x_scales = nullptr;
    Codes next[kAhead];                                    // of the next three steps
    uint32_t next_scales = 0;                              // of the next four
    auto fetch = [&](int s, int32_t step) { next[s] = x[step * kWave + lane]; };
    auto fetch_first = [&](uint32_t pass) {
        const int64_t at = min((int64_t)pass * kWaves + wave, last_tile);
        x = reinterpret_cast<const Codes*>(m.x_codes) + at * a.steps * kWave;
        x_scales = reinterpret_cast<const uint32_t*>(m.x_scales) + at * (a.steps / 4) * kWave;
        next_scales = x_scales[lane];
#pragma unroll
        for (int s = 0; s < kAhead - 1; ++s) fetch(s, s);
    };

    uint32_t pass;
    int32_t tile = tile_of(0, pass), slot = 0;
    int32_t other_tile = -1, other_chunk = -1;             // what the other slot holds
    send_for(tile, 0);
    fetch_first(pass);
    hold(0, 0);
    __syncthreads();
    float bias[4];
    int32_t bias_of = -1;
    for (uint32_t n = 0; n < count; ++n) {
        const int64_t word = first_word(tile) + 4 * col;
        if (bias_of != tile) {
            bias_of = tile;
#pragma unroll
            for (int i = 0; i < 4; ++i) bias[i] = bias_at<T>(m, (int32_t)(word + i));
        }
        uint32_t next_pass = pass;
        const int32_t next_tile = n + 1 < count ? tile_of(n + 1, next_pass) : tile;
        Acc acc[4] = {};
        for (int32_t chunk = 0; chunk < chunks; ++chunk) {
            // what comes after this chunk, and whether it has to be sent for
            const bool last = chunk + 1 == chunks;
            const int32_t after_tile = last ? next_tile : tile, after_chunk = last ? 0 : chunk + 1;
            const bool stay = after_tile == tile && after_chunk == chunk, there = after_tile == other_tile && after_chunk == other_chunk;
            const bool send = !stay && !there && !(last && n + 1 == count);
            if (send) send_for(after_tile, after_chunk);
            const int32_t first = chunk * kChunk, steps = min(kChunk, a.steps - first);
            const Codes* const mine = held + slot * slot_steps * 4 * kWave + part * 32;
            const uint32_t* const mine_scales = held_scales + slot * slot_steps * kWave + lane;
            Codes w[2][4];                                 // of this step and the next
            uint32_t ws[2];
            auto read = [&](int buffer, int s, int32_t step) {     // s: step % 4
                const Codes* at = mine + step * 4 * kWave + (col ^ ((2 * s + part) & 7));
#pragma unroll
                for (int i = 0; i < 4; ++i) w[buffer][i] = at[i * kWave];
                ws[buffer] = mine_scales[step * kWave];
            };
            read(0, 0, 0);
            for (int32_t in = 0; in < steps; in += kAhead) {
                const int32_t ahead = min(first + in + kAhead, a.steps - kAhead);          // (the last ones are loaded again)
                const uint32_t xs = next_scales;
                next_scales = x_scales[ahead / 4 * kWave + lane];
                auto step = [&](auto which) {
                    constexpr int s = decltype(which)::value;
                    read((s + 1) & 1, (s + 1) % 4, min(in + s + 1, steps - 1));
                    fetch((s + 3) % 4, s ? ahead + s - 1 : min(first + in + 3, a.steps - 1));
                    __builtin_amdgcn_sched_barrier(0);     // (or the loads are moved to where they are needed)
                    acc[0] = mx4_mfma<s, 0>(next[s], xs, w[s & 1][0], ws[s & 1], acc[0]);
                    acc[1] = mx4_mfma<s, 1>(next[s], xs, w[s & 1][1], ws[s & 1], acc[1]);
                    acc[2] = mx4_mfma<s, 2>(next[s], xs, w[s & 1][2], ws[s & 1], acc[2]);
                    acc[3] = mx4_mfma<s, 3>(next[s], xs, w[s & 1][3], ws[s & 1], acc[3]);
                    __builtin_amdgcn_sched_barrier(0);
                };
                step(std::integral_constant<int, 0>());
                step(std::integral_constant<int, 1>());
                step(std::integral_constant<int, 2>());
                step(std::integral_constant<int, 3>());
            }
            if (last && n + 1 < count) fetch_first(next_pass);
            if (send) {
                __syncthreads();                           // (the other slot's readers are done)
                hold(1 - slot, after_chunk);
                __syncthreads();
            }
            if (!stay) {
                other_tile = tile;
                other_chunk = chunk;
                slot = 1 - slot;
            }
        }
        __builtin_amdgcn_sched_barrier(0);                 // (the next rows' loads before the stores: they are waited for in order)
        const int64_t row0 = ((int64_t)pass * kWaves + wave) * 32 + 4 * part;
        T* const y = static_cast<T*>(m.y) + row0 * m.y_stride + word;
        const int64_t rows_here = m.rows - row0;
        auto store = [&](bool all) {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int down = 8 * (j / 4) + j % 4;
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = acc[i][j] + bias[i];
                if (all || down < rows_here) store_four(y + down * m.y_stride, v, a.once);
            }
        };
        if (((int64_t)pass * kWaves + wave + 1) * 32 <= m.rows) store(true);
        else store(false);
        tile = next_tile;
        pass = next_pass;
    }
}

}  // namespace mlda
