// Layer norm over the columns of a row, and its gradients.
//
//   mean = sum x / C,  var = sum (x - mean)^2 / C,  rstd = 1 / sqrt(var + eps),  y = (x - mean) rstd w + b
//   u = (x - mean) rstd,  h = g w:   dx = rstd (h - sum h / C - u sum(h u) / C),  dw = sum_rows g u,  db = sum_rows g
//
// Bound by memory (7 and 13 operations an element).  A row is held by a team of lanes, so many 16-byte pieces each, from its one read
// to its one write: four or sixteen lanes, a wave, or a workgroup, by the bytes of a row.  Teams take row after row, so that
// weight and bias are read once and the weight's gradient is summed in registers; the next row's loads are on their way
// while a row is worked on.  Sums are in a fixed order, fp32 where a lane adds up 64 columns at the most, fp64 in longer rows; the
// deviations' squares are taken after the mean is known.
#pragma once
#include "vec_io.hpp"

namespace mlda {

struct LayerNormArgs {
    const void* x;
    int64_t x_stride;
    const void* weight;          // null: ones
    const void* bias;            // null: zeros
    void* y;
    int64_t y_stride;
    float* mean;                 // null: not wanted
    float* rstd;
    int64_t rows;
    int32_t cols;
    float eps;
    bool once;                   // x and y are more than the caches hold
};

struct LayerNormGradArgs {
    const void* grad;
    int64_t grad_stride;
    const void* x;
    int64_t x_stride;
    const float* mean;
    const float* rstd;
    const void* weight;          // null: ones
    void* grad_x;                // null: not wanted
    int64_t grad_x_stride;
    float* partial;              // [workgroups][2][cols]; null: the sums over rows are not wanted, or the one workgroup's are the whole
    void* grad_weight;           // then: null: not wanted
    void* grad_bias;
    int64_t rows;
    int32_t cols;
    bool once;                   // x, grad and grad_x are more than the caches hold
};

// P columns of a vector of type W, as they are loaded: P elements of another type make up 16 bytes.
template <class W, int P>
struct Columns {
    static constexpr int kRaw = P / kPack<W>;
    Raw raw[kRaw];

    // `fill` past the end, and everywhere where there is no vector
    __device__ __forceinline__ void load(const void* at, int32_t c, int32_t cols, float fill) {
        const W* p = static_cast<const W*>(at);
#pragma unroll
        for (int i = 0; i < kRaw; ++i) raw[i] = load_some(p + c + i * kPack<W>, p ? cols - c - i * kPack<W> : 0, fill, c + i * kPack<W>);
    }
    __device__ __forceinline__ void get(float (&out)[P]) const {
#pragma unroll
        for (int i = 0; i < kRaw; ++i) {
            float v[kPack<W>];
            unpack(raw[i], v, W());
#pragma unroll
            for (int e = 0; e < kPack<W>; ++e) out[i * kPack<W> + e] = v[e];
        }
    }
};

constexpr int team_threads(int team) { return team < 256 ? 256 : team; }

// kHeld: weight and bias are kept, and the next row's pieces are loaded ahead.  300,000 x 1,000 bf16 254 us (4.7 TB/s; a copy does 5.2),
// 8,009 x 10,000 fp32 106 us (6.1 TB/s), one row of 1,000 fp32 2.7 us.
template <class T, class W, int kTeam, int kPieces, bool kHeld>
__global__ __launch_bounds__(team_threads(kTeam)) void layer_norm_kernel(LayerNormArgs a) {
    constexpr int P = kPack<T>, kThreads = team_threads(kTeam), kTeams = kThreads / kTeam;
    __shared__ float slots[2][kThreads / kWave];
    const int lane = (int)threadIdx.x % kTeam;
    const int32_t cols = a.cols;
    const float n_cols = (float)cols;              // (a quotient is right where the sum is)
    Columns<W, P> w[kHeld ? kPieces : 1], b[kHeld ? kPieces : 1];
    if constexpr (kHeld) {
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            w[j].load(a.weight, (j * kTeam + lane) * P, cols, 1.0f);
            b[j].load(a.bias, (j * kTeam + lane) * P, cols, 0.0f);
        }
    }
    const int64_t step = (int64_t)gridDim.x * kTeams;
    int64_t row = (int64_t)blockIdx.x * kTeams + (int)threadIdx.x / kTeam;
    // (the sums want every lane of a wave: teams of fewer whose rows have run out go on beside the others with a row of zeros)
    const int64_t rounds = (a.rows - (int64_t)blockIdx.x * kTeams + step - 1) / step;
    auto load_row = [&](int64_t r, Raw (&to)[kPieces]) {
        const T* x = static_cast<const T*>(a.x) + r * a.x_stride;
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const int32_t c = (j * kTeam + lane) * P;
            to[j] = load_some(x + c, r < a.rows ? cols - c : 0, 0.0f, c);
        }
    };
    Raw x[kPieces], next[kPieces];
    if (kHeld) load_row(row, next);
    for (int64_t i = 0; i < rounds; ++i, row += step) {
        if constexpr (kHeld) {
#pragma unroll
            for (int j = 0; j < kPieces; ++j) x[j] = next[j];
            if (i + 1 < rounds) load_row(row + step, next);
        } else {
            load_row(row, x);
        }
        // (where they are not held, the loads of weight and bias are to stay in the loop: outside it they are held after all)
        const void* weight = a.weight;
        const void* bias = a.bias;
        if constexpr (!kHeld) asm volatile("" : "+s"(weight), "+s"(bias));
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            float v[P];
            unpack(x[j], v, T());
#pragma unroll
            for (int e = 0; e < P; ++e) sum += v[e];
        }
        const float mean = team_sum<kTeam>(sum, slots[0]) / n_cols;
        forget(x);
        float squares = 0.0f;
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const int32_t c = (j * kTeam + lane) * P;
            float v[P];
            unpack(x[j], v, T());
            if (c + P <= cols) {
#pragma unroll
                for (int e = 0; e < P; ++e) squares = __builtin_fmaf(v[e] - mean, v[e] - mean, squares);
            } else {
#pragma unroll
                for (int e = 0; e < P; ++e) squares += c + e < cols ? (v[e] - mean) * (v[e] - mean) : 0.0f;
            }
        }
        const float rstd = 1.0f / sqrtf(team_sum<kTeam>(squares, slots[1]) / n_cols + a.eps);
        forget(x);
        if (row < a.rows) {
            T* y = static_cast<T*>(a.y) + row * a.y_stride;
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
                const int32_t c = (j * kTeam + lane) * P;
                if constexpr (!kHeld) {
                    w[0].load(weight, c, cols, 1.0f);
                    b[0].load(bias, c, cols, 0.0f);
                }
                float v[P], vw[P], vb[P];
                unpack(x[j], v, T());
                forget(w[kHeld ? j : 0].raw);
                forget(b[kHeld ? j : 0].raw);
                w[kHeld ? j : 0].get(vw);
                b[kHeld ? j : 0].get(vb);
#pragma unroll
                for (int e = 0; e < P; ++e) v[e] = __builtin_fmaf((v[e] - mean) * rstd, vw[e], vb[e]);
                store_piece(y, c, 0, cols, pack(v, T()), a.once);
                if constexpr (!kHeld) __builtin_amdgcn_sched_barrier(0);      // (a piece at a time: more have no registers)
            }
            if (lane == 0) {
                if (a.mean) a.mean[row] = mean;
                if (a.rstd) a.rstd[row] = rstd;
            }
        }
    }
}

// Rows that no team has the registers for: a workgroup reads them three times, the second and third time from the caches (2,003 x 40,000
// fp32 174 us, 3.7 TB/s of the row once in and once out).  A thread adds up any number of columns, so in fp64, which the reads leave time for: the
// sum of equal numbers is exact, whatever their number.
template <class T, class W>
__global__ __launch_bounds__(1024) void layer_norm_long_kernel(LayerNormArgs a) {
    constexpr int P = kPack<T>;
    __shared__ double slots[2][16];
    const int32_t cols = a.cols;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        T* y = static_cast<T*>(a.y) + row * a.y_stride;
        double sum = 0.0;
        for (int64_t c = (int64_t)threadIdx.x * P; c < cols; c += 1024 * P) {
            float v[P];
            unpack(load_some(x + c, (int)min((int64_t)P, cols - c), 0.0f, c), v, T());
#pragma unroll
            for (int e = 0; e < P; ++e) sum += (double)v[e];
        }
        const float mean = (float)(group_sum<1024>(sum, slots[0]) / cols);
        double squares = 0.0;
        for (int64_t c = (int64_t)threadIdx.x * P; c < cols; c += 1024 * P) {
            const int n = (int)min((int64_t)P, cols - c);
            float v[P];
            unpack(load_some(x + c, n, 0.0f, c), v, T());
#pragma unroll
            for (int e = 0; e < P; ++e) {
                const double d = e < n ? (double)(v[e] - mean) : 0.0;
                squares = __builtin_fma(d, d, squares);
            }
        }
        const float rstd = 1.0f / sqrtf((float)(group_sum<1024>(squares, slots[1]) / cols) + a.eps);
        // (x and y may be the same rows: what is written below is read by the same thread only)
        for (int64_t c = (int64_t)threadIdx.x * P; c < cols; c += 1024 * P) {
            const int n = (int)min((int64_t)P, cols - c);
            float v[P], vw[P], vb[P];
            Columns<W, P> w, b;
            unpack(load_some(x + c, n, 0.0f, c), v, T());
            w.load(a.weight, (int32_t)c, cols, 1.0f);
            b.load(a.bias, (int32_t)c, cols, 0.0f);
            w.get(vw);
            b.get(vb);
#pragma unroll
            for (int e = 0; e < P; ++e) v[e] = __builtin_fmaf((v[e] - mean) * rstd, vw[e], vb[e]);
            store_piece(y, c, 0, cols, pack(v, T()), a.once);
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// One row's part in the gradient: u and h of a piece.
template <class T, class W>
__device__ __forceinline__ void grad_piece(Raw x, Raw g, const Columns<W, kPack<T>>& w, float mean, float rstd, float (&u)[kPack<T>],
                                           float (&h)[kPack<T>], float (&grad)[kPack<T>]) {
    unpack(x, u, T());
    unpack(g, grad, T());
    w.get(h);
#pragma unroll
    for (int e = 0; e < kPack<T>; ++e) {
        u[e] = (u[e] - mean) * rstd;
        h[e] *= grad[e];
    }
}

// kSums: the weight's and bias' gradients are summed here, and the weight is kept.  kAhead: the next row's pieces are loaded ahead.
// 300,000 x 1,000 bf16 374 us (4.8 TB/s), fp32 712 (5.1); 30,011 x 1,537 bf16, rows at odd addresses, 59 us (4.7; the vector units work in 93%
// of the cycles); 8,009 x 10,000 fp32, whose sums and weights take three eighths of the registers, 209 (4.6).  Four waves a SIMD are worth
// more than the few registers of a lane that 16-bit rows with fp32 weights keep in memory for it (5 to 11 of 128): 30,011 x 1,537 66 us,
// with three waves and none 77; 300,000 x 1,000 339 and 389.
template <class T, class W, int kTeam, int kPieces, bool kSums, bool kAhead = kSums>
__global__ __launch_bounds__(team_threads(kTeam), kTeam <= 512 && kPieces == 2 ? 4 : 1) void layer_norm_grad_kernel(LayerNormGradArgs a) {
    constexpr int P = kPack<T>, kThreads = team_threads(kTeam), kTeams = kThreads / kTeam;
    __shared__ float slots[2][2 * (kThreads / kWave)];
    // sums over the workgroup's teams: [dw or db][column]
    __shared__ float joined[kSums && kTeams > 1 ? 2 * kTeam * kPieces * P : 1];
    const int lane = (int)threadIdx.x % kTeam;
    const int32_t cols = a.cols;
    const float n_cols = (float)cols;
    Columns<W, P> w[kSums ? kPieces : 1];
    float dw[kSums ? kPieces * P : 1], db[kSums ? kPieces * P : 1];
    if constexpr (kSums) {
#pragma unroll
        for (int j = 0; j < kPieces; ++j) w[j].load(a.weight, (j * kTeam + lane) * P, cols, 1.0f);
#pragma unroll
        for (int k = 0; k < kPieces * P; ++k) dw[k] = db[k] = 0.0f;
    }
    const int64_t step = (int64_t)gridDim.x * kTeams;
    int64_t row = (int64_t)blockIdx.x * kTeams + (int)threadIdx.x / kTeam;
    const int64_t rounds = (a.rows - (int64_t)blockIdx.x * kTeams + step - 1) / step;
    Raw x[kPieces], g[kPieces], next_x[kPieces], next_g[kPieces];
    float mean, rstd, next_mean, next_rstd;
    // (columns past the end: the gradient is zero there, and what comes out is not stored)
    auto load_row = [&](int64_t r, Raw (&to_x)[kPieces], Raw (&to_g)[kPieces], float& to_mean, float& to_rstd) {
        const T* at_x = static_cast<const T*>(a.x) + r * a.x_stride;
        const T* at_g = static_cast<const T*>(a.grad) + r * a.grad_stride;
        const bool there = r < a.rows;
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const int32_t c = (j * kTeam + lane) * P;
            const int n = there ? cols - c : 0;
            to_x[j] = load_some(at_x + c, n, 0.0f, c);
            to_g[j] = load_some(at_g + c, n, 0.0f, c);
        }
        to_mean = there ? a.mean[r] : 0.0f;
        to_rstd = there ? a.rstd[r] : 0.0f;
    };
    if (kAhead) load_row(row, next_x, next_g, next_mean, next_rstd);
    for (int64_t i = 0; i < rounds; ++i, row += step) {
        if constexpr (kAhead) {
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
                x[j] = next_x[j];
                g[j] = next_g[j];
            }
            mean = next_mean;
            rstd = next_rstd;
            if (i + 1 < rounds) load_row(row + step, next_x, next_g, next_mean, next_rstd);
        } else {
            load_row(row, x, g, mean, rstd);
        }
        const void* weight = a.weight;             // (as in layer_norm_kernel)
        if constexpr (!kSums) asm volatile("" : "+s"(weight));
        float sum_h = 0.0f, sum_hu = 0.0f;
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            float u[P], h[P], grad[P];
            if constexpr (!kSums) w[0].load(weight, (j * kTeam + lane) * P, cols, 1.0f);
            forget(w[kSums ? j : 0].raw);
            grad_piece<T, W>(x[j], g[j], w[kSums ? j : 0], mean, rstd, u, h, grad);
#pragma unroll
            for (int e = 0; e < P; ++e) {
                sum_h += h[e];
                sum_hu = __builtin_fmaf(h[e], u[e], sum_hu);
            }
        }
        team_sums<kTeam>(sum_h, sum_hu, slots[i & 1]);
        const float mean_h = sum_h / n_cols, mean_hu = sum_hu / n_cols;
        forget(x);
        forget(g);
        T* dx = row < a.rows && a.grad_x ? static_cast<T*>(a.grad_x) + row * a.grad_x_stride : nullptr;
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const int32_t c = (j * kTeam + lane) * P;
            float u[P], h[P], v[P];
            if constexpr (!kSums) w[0].load(weight, c, cols, 1.0f);
            forget(w[kSums ? j : 0].raw);
            grad_piece<T, W>(x[j], g[j], w[kSums ? j : 0], mean, rstd, u, h, v);
            if constexpr (kSums) {                 // (not beside the sums above: what that needs would be kept until here)
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    dw[j * P + e] = __builtin_fmaf(v[e], u[e], dw[j * P + e]);
                    db[j * P + e] += v[e];
                }
            }
#pragma unroll
            for (int e = 0; e < P; ++e) v[e] = rstd * ((h[e] - mean_h) - u[e] * mean_hu);
            // (a team that its sums fill has no registers for two kinds of stores: 8,009 x 10,000 fp32 209 us, with both 223)
            if constexpr (kSums && !kAhead) {
                if (dx) store_some(dx + c, pack(v, T()), min(max(cols - c, 0), P));
            } else {
                if (dx) store_piece(dx, c, 0, cols, pack(v, T()), a.once);
            }
        }
    }
    if constexpr (kSums) {
        if (!a.partial && !a.grad_weight && !a.grad_bias) return;
        // a sum of this thread's: to the workgroup's, or, where there is only one, to where it is wanted
        auto put = [&](int c, float w_sum, float b_sum) {
            if (c >= cols) return;
            if (a.partial) {
                float* out = a.partial + (int64_t)blockIdx.x * 2 * cols;
                out[c] = w_sum;
                out[cols + c] = b_sum;
            } else {
                if (a.grad_weight) static_cast<W*>(a.grad_weight)[c] = (W)w_sum;
                if (a.grad_bias) static_cast<W*>(a.grad_bias)[c] = (W)b_sum;
            }
        };
        if constexpr (kTeams > 1) {
            // the teams of a wave by its lanes, then one wave or team after the other: the order of the additions is fixed
            constexpr int kCols = kTeam * kPieces * P, kLanes = kTeam < kWave ? kWave : kTeam;
#pragma unroll
            for (int k = 0; k < kPieces * P; ++k)
#pragma unroll
                for (int off = kTeam; off < kWave; off *= 2) {
                    dw[k] += __shfl_xor(dw[k], off, kWave);
                    db[k] += __shfl_xor(db[k], off, kWave);
                }
            for (int t = 0; t < kThreads / kLanes; ++t) {
                if ((int)threadIdx.x / kLanes == t && (int)threadIdx.x % kLanes < kTeam) {
#pragma unroll
                    for (int j = 0; j < kPieces; ++j)
#pragma unroll
                        for (int e = 0; e < P; ++e) {
                            const int c = (j * kTeam + lane) * P + e, k = j * P + e;
                            joined[c] = t ? joined[c] + dw[k] : dw[k];
                            joined[kCols + c] = t ? joined[kCols + c] + db[k] : db[k];
                        }
                }
                __syncthreads();
            }
            for (int c = (int)threadIdx.x; c < min(cols, kCols); c += kThreads) put(c, joined[c], joined[kCols + c]);
        } else {
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
                const int c = (j * kTeam + lane) * P;
                if (a.partial && c + P <= cols) {
                    float* out = a.partial + (int64_t)blockIdx.x * 2 * cols + c;
#pragma unroll
                    for (int e = 0; e < P; e += 4) {
                        const int k = j * P + e;
                        store_raw(out + e, pack({dw[k], dw[k + 1], dw[k + 2], dw[k + 3]}, 0.0f));
                        store_raw(out + cols + e, pack({db[k], db[k + 1], db[k + 2], db[k + 3]}, 0.0f));
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < P; ++e) put(c + e, dw[j * P + e], db[j * P + e]);
                }
            }
        }
    }
}

// Rows without room in registers: the gradient of x by a workgroup a row, which reads the row twice (2,003 x 40,000 fp32 with the sums
// below 366 us, 2.6 TB/s of everything once).  Sums over columns in fp64, as above.
template <class T, class W>
__global__ __launch_bounds__(1024) void layer_norm_grad_long_kernel(LayerNormGradArgs a) {
    constexpr int P = kPack<T>;
    __shared__ double slots[2][2][16];
    const int32_t cols = a.cols;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        const T* grad = static_cast<const T*>(a.grad) + row * a.grad_stride;
        T* dx = static_cast<T*>(a.grad_x) + row * a.grad_x_stride;
        const float mean = a.mean[row], rstd = a.rstd[row];
        double sum_h = 0.0, sum_hu = 0.0;
        auto piece = [&](int64_t c, float (&u)[P], float (&h)[P]) {
            const int n = (int)min((int64_t)P, cols - c);
            Columns<W, P> w;
            float unused[P];
            w.load(a.weight, (int32_t)c, cols, 1.0f);
            grad_piece<T, W>(load_some(x + c, n, 0.0f, c), load_some(grad + c, n, 0.0f, c), w, mean, rstd, u, h, unused);
        };
        for (int64_t c = (int64_t)threadIdx.x * P; c < cols; c += 1024 * P) {
            float u[P], h[P];
            piece(c, u, h);
#pragma unroll
            for (int e = 0; e < P; ++e) {
                sum_h += (double)h[e];
                sum_hu = __builtin_fma((double)h[e], (double)u[e], sum_hu);
            }
        }
        const float mean_h = (float)(group_sum<1024>(sum_h, slots[turn][0]) / cols), mean_hu = (float)(group_sum<1024>(sum_hu, slots[turn][1]) / cols);
        for (int64_t c = (int64_t)threadIdx.x * P; c < cols; c += 1024 * P) {
            float u[P], h[P], v[P];
            piece(c, u, h);
#pragma unroll
            for (int e = 0; e < P; ++e) v[e] = rstd * ((h[e] - mean_h) - u[e] * mean_hu);
            store_piece(dx, c, 0, cols, pack(v, T()), a.once);
        }
    }
}

// The sums over rows on their own, by tiles of 64 x kPack columns: workgroup (tile, slab) sums its slab's rows, four to a wave at
// once.
template <class T>
__global__ __launch_bounds__(256) void layer_norm_grad_columns_kernel(LayerNormGradArgs a) {
    constexpr int P = kPack<T>, kAtOnce = 4;
    __shared__ float joined[4][2 * kWave * P];
    const int wave = (int)threadIdx.x / kWave, lane = lane_id();
    const int32_t c = ((int32_t)blockIdx.x * kWave + lane) * P;
    const int n = min(max(a.cols - c, 0), P);
    float dw[P], db[P];
#pragma unroll
    for (int e = 0; e < P; ++e) dw[e] = db[e] = 0.0f;
    for (int64_t first = ((int64_t)blockIdx.y * 4 + wave) * kAtOnce; first < a.rows; first += (int64_t)gridDim.y * 4 * kAtOnce) {
        Raw x[kAtOnce], g[kAtOnce];
        float mean[kAtOnce], rstd[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int64_t row = first + k;
            const int there = row < a.rows ? n : 0;
            x[k] = load_some(static_cast<const T*>(a.x) + row * a.x_stride + c, there, 0.0f, c);
            g[k] = load_some(static_cast<const T*>(a.grad) + row * a.grad_stride + c, there, 0.0f, c);
            mean[k] = row < a.rows ? a.mean[row] : 0.0f;
            rstd[k] = row < a.rows ? a.rstd[row] : 0.0f;
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            float vx[P], vg[P];
            unpack(x[k], vx, T());
            unpack(g[k], vg, T());
#pragma unroll
            for (int e = 0; e < P; ++e) {
                dw[e] = __builtin_fmaf(vg[e], (vx[e] - mean[k]) * rstd[k], dw[e]);
                db[e] += vg[e];
            }
        }
    }
#pragma unroll
    for (int e = 0; e < P; ++e) {
        joined[wave][lane * P + e] = dw[e];
        joined[wave][(kWave + lane) * P + e] = db[e];
    }
    __syncthreads();
    float* out = a.partial + (int64_t)blockIdx.y * 2 * a.cols;
    for (int i = (int)threadIdx.x; i < 2 * kWave * P; i += 256) {
        const int64_t col = (int64_t)blockIdx.x * kWave * P + i % (kWave * P);
        if (col < a.cols)
            out[(i / (kWave * P)) * (int64_t)a.cols + col] = (joined[0][i] + joined[1][i]) + (joined[2][i] + joined[3][i]);
    }
}

// The workgroups' sums added up, in their order, and rounded to the weight's type: 16 columns of [dw, db] a workgroup at a time, by 64
// slices of the workgroups.
constexpr int kFinalCols = 16;
template <class W>
__global__ __launch_bounds__(1024) void layer_norm_grad_final_kernel(const float* partial, int32_t partials, int32_t cols,
                                                                     W* grad_weight, W* grad_bias) {
    constexpr int kSlices = 64;
    __shared__ float joined[2][kSlices][kFinalCols + 1];
    const int slice = (int)threadIdx.x / kFinalCols, lane = (int)threadIdx.x % kFinalCols;
    int turn = 0;
    for (int64_t first = (int64_t)blockIdx.x * kFinalCols; first < 2 * (int64_t)cols; first += (int64_t)gridDim.x * kFinalCols, turn ^= 1) {
        const int64_t i = first + lane;
        float sum = 0.0f;
        if (i < 2 * (int64_t)cols)
#pragma unroll 4
            for (int p = slice; p < partials; p += kSlices) sum += partial[(int64_t)p * 2 * cols + i];
        joined[turn][slice][lane] = sum;
        __syncthreads();
        // a column to each group of 16 lanes: four slices a lane, then the lanes
        const int column = (int)threadIdx.x / 16, part = (int)threadIdx.x % 16;
        if (threadIdx.x >= kFinalCols * 16) continue;
        const float(&from)[kSlices][kFinalCols + 1] = joined[turn];
        sum = (from[part][column] + from[part + 16][column]) + (from[part + 32][column] + from[part + 48][column]);
        sum = row16_sum(sum);
        const int64_t at = first + column;
        if (part != 0 || at >= 2 * (int64_t)cols) continue;
        if (at < cols) {
            if (grad_weight) grad_weight[at] = (W)sum;
        } else if (grad_bias) {
            grad_bias[at - cols] = (W)sum;
        }
    }
}

}  // namespace mlda
