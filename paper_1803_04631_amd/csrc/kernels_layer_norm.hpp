// Layer norm over the columns of a row, and its gradients.
//
//   mean = sum x / C,  var = sum (x - mean)^2 / C,  rstd = 1 / sqrt(var + eps),  y = (x - mean) rstd w + b
//   u = (x - mean) rstd,  h = g w:   dx = rstd (h - sum h / C - u sum(h u) / C),  dw = sum_rows g u,  db = sum_rows g
//
// Bound by memory (7 and 13 operations an element).  Up to 16,384 columns a row stays in the registers of a team of lanes
// from its one read to its one write: 16 lanes, a wave, or a workgroup, by the number of columns.  Teams take row after row, so
// that weight and bias are read once and the weight's gradient is summed in registers; the next row's loads are
// on their way while a row is worked on.  Sums are fp32 in a fixed order, the deviations' squares are taken
// after the mean is known.
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
    float* partial;              // [workgroups][2][cols], null: the sums over rows are not wanted
    int64_t rows;
    int32_t cols;
};

// P elements of a vector of type W (P of another type make up 16 bytes) from column c on; `fill` past the end.
template <class W, int P>
__device__ __forceinline__ void load_columns(const void* at, int32_t c, int32_t cols, float fill, float (&out)[P]) {
    const W* p = static_cast<const W*>(at);
#pragma unroll
    for (int e = 0; e < P; ++e) out[e] = p && c + e < cols ? (float)p[c + e] : fill;
}

template <class T, class W, int kTeam, int kE>
__global__ __launch_bounds__(kTeam < 256 ? 256 : kTeam) void layer_norm_kernel(LayerNormArgs a) {
    constexpr int P = kPack<T>, kPieces = kE / P, kThreads = kTeam < 256 ? 256 : kTeam, kTeams = kThreads / kTeam;
    __shared__ float slots[2][kThreads / kWave];
    const int lane = (int)threadIdx.x % kTeam;
    const int32_t cols = a.cols;
    const float n_cols = (float)cols;              // (a quotient is right where the sum is: a row of equal numbers has no variance)
    float w[kE], b[kE];
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
        float v[P];
        load_columns<W, P>(a.weight, (j * kTeam + lane) * P, cols, 1.0f, v);
#pragma unroll
        for (int e = 0; e < P; ++e) w[j * P + e] = v[e];
        load_columns<W, P>(a.bias, (j * kTeam + lane) * P, cols, 0.0f, v);
#pragma unroll
        for (int e = 0; e < P; ++e) b[j * P + e] = v[e];
    }
    const int64_t step = (int64_t)gridDim.x * kTeams;
    int64_t row = (int64_t)blockIdx.x * kTeams + (int)threadIdx.x / kTeam;
    // (the sums want every lane of a wave: teams of 16 whose rows have run out go on beside the others with a row of zeros)
    const int64_t rounds = (a.rows - (int64_t)blockIdx.x * kTeams + step - 1) / step;
    Raw next[kPieces];
    auto load_row = [&](int64_t r) {
        const T* x = static_cast<const T*>(a.x) + r * a.x_stride;
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const int32_t c = (j * kTeam + lane) * P;
            next[j] = r < a.rows ? load_some(x + c, min(max(cols - c, 0), P), 0.0f) : Raw{0, 0, 0, 0};
        }
    };
    load_row(row);
    for (int64_t i = 0; i < rounds; ++i, row += step) {
        float x[kE];
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            float v[P];
            unpack(next[j], v, T());
#pragma unroll
            for (int e = 0; e < P; ++e) { x[j * P + e] = v[e]; sum += v[e]; }
        }
        if (i + 1 < rounds) load_row(row + step);
        const float mean = team_sum<kTeam>(sum, slots[0]) / n_cols;
        float squares = 0.0f;
#pragma unroll
        for (int j = 0; j < kPieces; ++j)
#pragma unroll
            for (int e = 0; e < P; ++e) {
                const float d = x[j * P + e] - mean;
                x[j * P + e] = d;
                squares += (j * kTeam + lane) * P + e < cols ? d * d : 0.0f;
            }
        const float rstd = 1.0f / sqrtf(team_sum<kTeam>(squares, slots[1]) / n_cols + a.eps);
        if (row < a.rows) {
            T* y = static_cast<T*>(a.y) + row * a.y_stride;
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
                float v[P];
#pragma unroll
                for (int e = 0; e < P; ++e) v[e] = __builtin_fmaf(x[j * P + e] * rstd, w[j * P + e], b[j * P + e]);
                const int32_t c = (j * kTeam + lane) * P;
                store_some(y + c, pack(v, T()), min(max(cols - c, 0), P));
            }
            if (lane == 0) {
                if (a.mean) a.mean[row] = mean;
                if (a.rstd) a.rstd[row] = rstd;
            }
        }
    }
}

// Rows that no team has the registers for: a workgroup reads them three times, the second and third time from the caches.
template <class T, class W>
__global__ __launch_bounds__(1024) void layer_norm_long_kernel(LayerNormArgs a) {
    constexpr int P = kPack<T>;
    __shared__ float slots[2][16];
    const int32_t cols = a.cols;
    const float n_cols = (float)cols;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        T* y = static_cast<T*>(a.y) + row * a.y_stride;
        float sum = 0.0f;
        for (int64_t c = (int64_t)threadIdx.x * P; c < cols; c += 1024 * P) {
            float v[P];
            unpack(load_some(x + c, (int)min((int64_t)P, cols - c), 0.0f), v, T());
#pragma unroll
            for (int e = 0; e < P; ++e) sum += v[e];
        }
        const float mean = team_sum<1024>(sum, slots[0]) / n_cols;
        float squares = 0.0f;
        for (int64_t c = (int64_t)threadIdx.x * P; c < cols; c += 1024 * P) {
            const int n = (int)min((int64_t)P, cols - c);
            float v[P];
            unpack(load_some(x + c, n, 0.0f), v, T());
#pragma unroll
            for (int e = 0; e < P; ++e) squares += e < n ? (v[e] - mean) * (v[e] - mean) : 0.0f;
        }
        const float rstd = 1.0f / sqrtf(team_sum<1024>(squares, slots[1]) / n_cols + a.eps);
        // (x and y may be the same rows: what is written below is read by the same thread only)
        for (int64_t c = (int64_t)threadIdx.x * P; c < cols; c += 1024 * P) {
            const int n = (int)min((int64_t)P, cols - c);
            float v[P], w[P], b[P];
            unpack(load_some(x + c, n, 0.0f), v, T());
            load_columns<W, P>(a.weight, (int32_t)c, cols, 1.0f, w);
            load_columns<W, P>(a.bias, (int32_t)c, cols, 0.0f, b);
#pragma unroll
            for (int e = 0; e < P; ++e) v[e] = __builtin_fmaf((v[e] - mean) * rstd, w[e], b[e]);
            store_some(y + c, pack(v, T()), n);
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

template <class T, class W, int kTeam, int kE>
__global__ __launch_bounds__(kTeam < 256 ? 256 : kTeam) void layer_norm_grad_kernel(LayerNormGradArgs a) {
    constexpr int P = kPack<T>, kPieces = kE / P, kThreads = kTeam < 256 ? 256 : kTeam, kTeams = kThreads / kTeam;
    __shared__ float slots[4][kThreads / kWave];
    // sums over the workgroup's teams: [dw or db][column]
    __shared__ float joined[kTeams > 1 ? 2 * kTeam * kE : 1];
    const int lane = (int)threadIdx.x % kTeam;
    const int32_t cols = a.cols;
    const float n_cols = (float)cols;
    // (a thousand threads of sixteen columns have no registers left for the weight and the next row)
    constexpr bool kTight = kTeam == 1024 && kE > 8;
    float w[kTight ? 1 : kE], dw[kE], db[kE];
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
        float v[P];
        if constexpr (!kTight) load_columns<W, P>(a.weight, (j * kTeam + lane) * P, cols, 1.0f, v);
#pragma unroll
        for (int e = 0; e < P; ++e) {
            if constexpr (!kTight) w[j * P + e] = v[e];
            dw[j * P + e] = db[j * P + e] = 0.0f;
        }
    }
    const int64_t step = (int64_t)gridDim.x * kTeams;
    int64_t row = (int64_t)blockIdx.x * kTeams + (int)threadIdx.x / kTeam;
    const int64_t rounds = (a.rows - (int64_t)blockIdx.x * kTeams + step - 1) / step;
    Raw next_x[kPieces], next_g[kPieces];
    float next_mean, next_rstd;
    auto load_row = [&](int64_t r) {
        const T* x = static_cast<const T*>(a.x) + r * a.x_stride;
        const T* g = static_cast<const T*>(a.grad) + r * a.grad_stride;
        const bool there = r < a.rows;
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const int32_t c = (j * kTeam + lane) * P;
            const int n = min(max(cols - c, 0), P);
            next_x[j] = there ? load_some(x + c, n, 0.0f) : Raw{0, 0, 0, 0};
            next_g[j] = there ? load_some(g + c, n, 0.0f) : Raw{0, 0, 0, 0};
        }
        next_mean = there ? a.mean[r] : 0.0f;
        next_rstd = there ? a.rstd[r] : 0.0f;
    };
    if (!kTight) load_row(row);
    for (int64_t i = 0; i < rounds; ++i, row += step) {
        if (kTight) load_row(row);
        float u[kE], h[kE];
        const float mean = next_mean, rstd = next_rstd;
        float sum_h = 0.0f, sum_hu = 0.0f;
        // (columns past the end: the gradient is zero there, and what comes out is not stored)
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            float x[P], g[P], here[P];
            unpack(next_x[j], x, T());
            unpack(next_g[j], g, T());
            if constexpr (kTight) load_columns<W, P>(a.weight, (j * kTeam + lane) * P, cols, 1.0f, here);
#pragma unroll
            for (int e = 0; e < P; ++e) {
                const int k = j * P + e;
                u[k] = (x[e] - mean) * rstd;
                h[k] = g[e] * (kTight ? here[e] : w[kTight ? 0 : k]);
                dw[k] = __builtin_fmaf(g[e], u[k], dw[k]);
                db[k] += g[e];
                sum_h += h[k];
                sum_hu = __builtin_fmaf(h[k], u[k], sum_hu);
            }
        }
        if (!kTight && i + 1 < rounds) load_row(row + step);
        if (a.grad_x) {
            // two sums a row, and the barrier of the second parts the first's readers from the next row's writers
            const float mean_h = team_sum<kTeam>(sum_h, slots[0]) / n_cols;
            const float mean_hu = team_sum<kTeam>(sum_hu, slots[1]) / n_cols;
            if (row < a.rows) {
                T* dx = static_cast<T*>(a.grad_x) + row * a.grad_x_stride;
#pragma unroll
                for (int j = 0; j < kPieces; ++j) {
                    float v[P];
#pragma unroll
                    for (int e = 0; e < P; ++e) {
                        const int k = j * P + e;
                        v[e] = rstd * (h[k] - mean_h - u[k] * mean_hu);
                    }
                    const int32_t c = (j * kTeam + lane) * P;
                    store_some(dx + c, pack(v, T()), min(max(cols - c, 0), P));
                }
            }
        }
    }
    if (!a.partial) return;
    float* out = a.partial + (int64_t)blockIdx.x * 2 * cols;
    if constexpr (kTeams > 1) {
        // one team after the other, so that the order of the additions is fixed
        for (int t = 0; t < kTeams; ++t) {
            if ((int)threadIdx.x / kTeam == t) {
#pragma unroll
                for (int j = 0; j < kPieces; ++j)
#pragma unroll
                    for (int e = 0; e < P; ++e) {
                        const int c = (j * kTeam + lane) * P + e, k = j * P + e;
                        joined[c] = t ? joined[c] + dw[k] : dw[k];
                        joined[kTeam * kE + c] = t ? joined[kTeam * kE + c] + db[k] : db[k];
                    }
            }
            __syncthreads();
        }
        for (int c = (int)threadIdx.x; c < cols; c += kThreads) {
            out[c] = joined[c];
            out[cols + c] = joined[kTeam * kE + c];
        }
    } else {
#pragma unroll
        for (int j = 0; j < kPieces; ++j)
#pragma unroll
            for (int e = 0; e < P; ++e) {
                const int c = (j * kTeam + lane) * P + e, k = j * P + e;
                if (c < cols) {
                    out[c] = dw[k];
                    out[cols + c] = db[k];
                }
            }
    }
}

// Rows without room in registers: the gradient of x by a workgroup a row, which reads the row twice ...
template <class T, class W>
__global__ __launch_bounds__(1024) void layer_norm_grad_long_kernel(LayerNormGradArgs a) {
    constexpr int P = kPack<T>;
    __shared__ float slots[2][16];
    const int32_t cols = a.cols;
    const float n_cols = (float)cols;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        const T* grad = static_cast<const T*>(a.grad) + row * a.grad_stride;
        T* dx = static_cast<T*>(a.grad_x) + row * a.grad_x_stride;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float sum_h = 0.0f, sum_hu = 0.0f;
        auto piece = [&](int64_t c, float (&u)[P], float (&h)[P]) {
            const int n = (int)min((int64_t)P, cols - c);
            float w[P];
            unpack(load_some(x + c, n, 0.0f), u, T());
            unpack(load_some(grad + c, n, 0.0f), h, T());
            load_columns<W, P>(a.weight, (int32_t)c, cols, 1.0f, w);
#pragma unroll
            for (int e = 0; e < P; ++e) {
                u[e] = (u[e] - mean) * rstd;
                h[e] *= w[e];
            }
            return n;
        };
        for (int64_t c = (int64_t)threadIdx.x * P; c < cols; c += 1024 * P) {
            float u[P], h[P];
            piece(c, u, h);
#pragma unroll
            for (int e = 0; e < P; ++e) {
                sum_h += h[e];
                sum_hu = __builtin_fmaf(h[e], u[e], sum_hu);
            }
        }
        const float mean_h = team_sum<1024>(sum_h, slots[0]) / n_cols;
        const float mean_hu = team_sum<1024>(sum_hu, slots[1]) / n_cols;
        for (int64_t c = (int64_t)threadIdx.x * P; c < cols; c += 1024 * P) {
            float u[P], h[P], v[P];
            const int n = piece(c, u, h);
#pragma unroll
            for (int e = 0; e < P; ++e) v[e] = rstd * (h[e] - mean_h - u[e] * mean_hu);
            store_some(dx + c, pack(v, T()), n);
        }
    }
}

// ... and the sums over rows by tiles of 64 x kPack columns: workgroup (tile, slab) sums its slab's rows, wave by wave.
template <class T>
__global__ __launch_bounds__(256) void layer_norm_grad_columns_kernel(LayerNormGradArgs a) {
    constexpr int P = kPack<T>;
    __shared__ float joined[4][2 * kWave * P];
    const int wave = (int)threadIdx.x / kWave, lane = lane_id();
    const int32_t c = ((int32_t)blockIdx.x * kWave + lane) * P;
    const int n = min(max(a.cols - c, 0), P);
    float dw[P], db[P];
#pragma unroll
    for (int e = 0; e < P; ++e) dw[e] = db[e] = 0.0f;
    for (int64_t row = (int64_t)blockIdx.y * 4 + wave; row < a.rows; row += (int64_t)gridDim.y * 4) {
        float x[P], g[P];
        unpack(load_some(static_cast<const T*>(a.x) + row * a.x_stride + c, n, 0.0f), x, T());
        unpack(load_some(static_cast<const T*>(a.grad) + row * a.grad_stride + c, n, 0.0f), g, T());
        const float mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
        for (int e = 0; e < P; ++e) {
            dw[e] = __builtin_fmaf(g[e], (x[e] - mean) * rstd, dw[e]);
            db[e] += g[e];
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

// The workgroups' sums added up, in their order, and rounded to the weight's type: 64 columns of [dw, db] a workgroup.
template <class W>
__global__ __launch_bounds__(1024) void layer_norm_grad_final_kernel(const float* partial, int32_t partials, int32_t cols,
                                                                     W* grad_weight, W* grad_bias) {
    __shared__ float joined[16][kWave];
    const int slice = (int)threadIdx.x / kWave, lane = lane_id();
    const int64_t i = (int64_t)blockIdx.x * kWave + lane;
    float sum = 0.0f;
    if (i < 2 * (int64_t)cols)
#pragma unroll 4
        for (int p = slice; p < partials; p += 16) sum += partial[(int64_t)p * 2 * cols + i];
    joined[slice][lane] = sum;
    __syncthreads();
    if (slice != 0 || i >= 2 * (int64_t)cols) return;
    sum = 0.0f;
#pragma unroll
    for (int s = 0; s < 16; ++s) sum += joined[s][lane];
    if (i < cols) {
        if (grad_weight) grad_weight[i] = (W)sum;
    } else if (grad_bias) {
        grad_bias[i - cols] = (W)sum;
    }
}

}  // namespace mlda
