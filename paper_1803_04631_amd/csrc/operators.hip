// Operators on device tensors for models next to the sampled topics: layer norm, log-probabilities of words, gradient clipping.
// Argument checks and launches; the kernels are in kernels_layer_norm.hpp, kernels_logprobs.hpp and kernels_clip.hpp.
#include "operators_host.hpp"

#include <math.h>

#include "kernels_clip.hpp"
#include "kernels_layer_norm.hpp"
#include "kernels_logprobs.hpp"

namespace {

constexpr int64_t kWaveRowBytes = 16384, kGroupRowBytes = 65536;

// f(tag of x, tag of the weight): the same type, or a weight in fp32.
template <class F>
int with_types(int32_t type, int32_t weight_type, F&& f) {
    return with_type(type, [&](auto t) { return weight_type == type ? f(t, t) : f(t, float()); });
}

// ---------------------------------------------------------------- layer norm
int check_layer_norm(int64_t rows, int32_t cols, int32_t type, int32_t weight_type) {
    if (rows < 0 || cols < 1 || cols > kMostCols) return refuse("layer norm: need rows >= 0 and 1 <= cols <= 2^30");
    if (!known_type(type)) return refuse("layer norm: unknown type");
    if (weight_type != type && weight_type != MLDA_FP32) return refuse("layer norm: the weight has the type of x, or fp32");
    return MLDA_OK;
}

template <int kTeam, int kPieces>
struct Team {
    static constexpr int team = kTeam, pieces = kPieces;
};

// f(team) for the lanes that share a row and the 16-byte pieces that each holds: as few lanes as have the registers.  300,000 x 1,000 bf16
// by a wave a row 253 us, by four 585; 30,011 x 1,537 38 and 66.
template <class F>
void with_team(int64_t row_bytes, F&& f) {
    if (row_bytes <= 64) f(Team<4, 1>());
    else if (row_bytes <= 256) f(Team<16, 1>());
    else if (row_bytes <= 1024) f(Team<64, 1>());
    else if (row_bytes <= 2048) f(Team<64, 2>());
    else if (row_bytes <= 4096) f(Team<64, 4>());
    else if (row_bytes <= 8192) f(Team<256, 2>());
    else if (row_bytes <= 16384) f(Team<256, 4>());
    else if (row_bytes <= 32768) f(Team<1024, 2>());
    else if (row_bytes <= 65536) f(Team<1024, 4>());
    else f(Team<1024, 8>());
}
constexpr int64_t kHeldBytes = 131072;            // of a row that a team holds
// of one beside whose gradient there is room for the weight's (two sums a column; 8,009 x 10,000 fp32 with the sums on their own 315 us, so 209)
constexpr int64_t summed_bytes(int64_t type_bytes) { return type_bytes == 4 ? 65536 : 32768; }

// The same for the gradient, where a column takes four times the registers; f(team, workgroups that fit a CU).
template <class F>
void with_grad_team(int64_t row_bytes, F&& f) {
    if (row_bytes <= 64) f(Team<4, 1>(), 4);
    else if (row_bytes <= 256) f(Team<16, 1>(), 4);
    else if (row_bytes <= 1024) f(Team<64, 1>(), 4);
    else if (row_bytes <= 2048) f(Team<64, 2>(), 4);
    else if (row_bytes <= 4096) f(Team<128, 2>(), 4);
    else if (row_bytes <= 8192) f(Team<256, 2>(), 4);
    else if (row_bytes <= 16384) f(Team<512, 2>(), 2);
    else if (row_bytes <= 32768) f(Team<1024, 2>(), 1);
    else f(Team<1024, 4>(), 1);
}

// Workgroups of the gradient's kernel, each of which leaves sums over its rows.
int32_t norm_grad_groups(int64_t rows, int32_t cols, int32_t type) {
    const int64_t bytes = cols * (int64_t)type_bytes(type);
    if (bytes > summed_bytes((int64_t)type_bytes(type))) return (int32_t)std::max<int64_t>(1, std::min<int64_t>((rows + 15) / 16, 64));      // slabs
    int64_t groups = 1;
    with_grad_team(bytes, [&](auto t, int per_cu) {
        constexpr int kThreads = mlda::team_threads(t.team), kTeams = kThreads / t.team;
        groups = std::min<int64_t>((rows + kTeams - 1) / kTeams, per_cu * kCus);
    });
    // their sums, written and read, are to be no more than what the rows are, unless they are less than 1 MB: 247 x 14,375 bf16 with a
    // workgroup a row 31 us, so 28
    groups = std::min(groups, std::max<int64_t>(rows * (int64_t)type_bytes(type) * 3 / 16, (1 << 20) / (8 * (int64_t)cols)));
    return (int32_t)std::max<int64_t>(1, groups);
}

// ---------------------------------------------------------------- log-probabilities
int check_logits(const void* logits, int64_t stride, int64_t rows, int32_t vocab, int32_t type, const int32_t* tokens,
                 const int64_t* row_ptr, int64_t n_tokens) {
    if (rows < 0 || vocab < 1 || vocab > kMostCols) return refuse("log-probabilities: need rows >= 0 and 1 <= vocab <= 2^30");
    if (!known_type(type)) return refuse("log-probabilities: unknown type");
    if (n_tokens < 0 || n_tokens >= ((int64_t)1 << 31)) return refuse("log-probabilities: need 0 <= n_tokens < 2^31");
    if (!row_ptr && n_tokens != rows) return refuse("log-probabilities: without row_ptr every row has one word");
    if (rows == 0) return MLDA_OK;
    RC_TRY(check_rows(logits, stride, rows, vocab, type, "log-probabilities: logits are null",
                      "log-probabilities: rows of logits overlap or are not aligned to their type"));
    if (n_tokens > 0 && !tokens) return refuse("log-probabilities: tokens are null");
    return MLDA_OK;
}

// Few rows are cut into segments, so that there is work for the whole chip; a workgroup has at least a tile for each wave, and
// segments are no more than the lanes that join them.  From twice as many rows as CUs on, rows are worked on whole.
void segments_of(int64_t rows, int32_t vocab, int32_t unit, int32_t* segments, int32_t* cols) {
    int64_t n = 1;
    if (rows < 2 * kCus) {
        n = std::min<int64_t>((4 * kCus + rows - 1) / std::max<int64_t>(rows, 1), ((int64_t)vocab + unit - 1) / unit);
        n = std::max<int64_t>(1, std::min<int64_t>(n, 64));
    }
    const int64_t per = ((int64_t)vocab + n - 1) / n;
    *cols = (int32_t)std::min<int64_t>((per + unit - 1) / unit * unit, kMostCols);
    *segments = (int32_t)(((int64_t)vocab + *cols - 1) / *cols);
}

// Where documents are this long on average, their words are looked up by more workgroups than there are rows.
constexpr int64_t kLongDocument = 2048;

// Many short rows have a wave each instead of a workgroup of four: 4,096 rows of 12,000 bf16 with the 20 likeliest words 29 us against
// 40, 20,000 of 3,001 54 against 126; but 4,096 of 100,000 fp32 318 against 301, and 1,024 of 48,001 bf16 35 against 27.
bool wave_rows(int64_t rows, int32_t vocab, int32_t type) {
    const int64_t bytes = (int64_t)vocab * (int64_t)type_bytes(type);
    return bytes <= 4096 || (bytes <= 49152 && rows >= 8 * kCus);
}

template <class T> constexpr int32_t kLogprobUnit = mlda::kLogprobWaves * mlda::kTileCols<T>;

int32_t logprob_unit(int32_t type) { return type == MLDA_FP32 ? kLogprobUnit<float> : kLogprobUnit<Bf16>; }

size_t logprob_workspace(int64_t rows, int32_t vocab, int32_t top, int32_t type) {
    int32_t segments, cols;
    segments_of(rows, vocab, logprob_unit(type), &segments, &cols);
    if (segments == 1) return 0;
    return (size_t)rows * (size_t)segments * (sizeof(mlda::RowPart) + (size_t)top * 8);
}

int run_logprobs(mlda::LogprobArgs a, int32_t type, void* workspace, hipStream_t stream) {
    const int64_t mean_len = a.n_tokens / a.rows;
    a.words_apart = a.stats && mean_len >= kLongDocument && a.rows < 4 * kCus;
    segments_of(a.rows, a.vocab, logprob_unit(type), &a.segments, &a.segment_cols);
    a.parts = static_cast<mlda::RowPart*>(workspace);
    a.part_top = reinterpret_cast<uint64_t*>(a.parts + a.rows * a.segments);
    const dim3 grid((unsigned)std::min(a.rows * a.segments, kMostGroups)), threads(mlda::kLogprobWaves * mlda::kWave);
    return with_type(type, [&](auto t) {
        typedef decltype(t) T;
        auto launch = [&](auto waves) {
            constexpr int kWaves = decltype(waves)::value;
            if (a.top) hipLaunchKernelGGL((mlda::logprob_kernel<T, true, true, kWaves>), grid, dim3(kWaves * mlda::kWave), 0, stream, a);
            else if (a.entropy) hipLaunchKernelGGL((mlda::logprob_kernel<T, true, false, kWaves>), grid, dim3(kWaves * mlda::kWave), 0, stream, a);
            else hipLaunchKernelGGL((mlda::logprob_kernel<T, false, false, kWaves>), grid, dim3(kWaves * mlda::kWave), 0, stream, a);
        };
        if (wave_rows(a.rows, a.vocab, type) && (mean_len < 512 || a.words_apart)) launch(std::integral_constant<int, 1>());
        else launch(std::integral_constant<int, mlda::kLogprobWaves>());
        RC_TRY(launched("logprob_kernel"));
        if (a.segments > 1) {
            hipLaunchKernelGGL((mlda::logprob_join_kernel<T>), dim3((unsigned)std::min(a.rows, kMostGroups)), threads, 0, stream, a);
            RC_TRY(launched("logprob_join_kernel"));
        }
        if (!a.words_apart) return MLDA_OK;
        const int split = (int)std::min<int64_t>(mean_len / 1024, 64);
        hipLaunchKernelGGL((mlda::logprob_words_kernel<T>), dim3((unsigned)std::min(a.rows * split, kMostGroups)), threads, 0, stream, a, split);
        return launched("logprob_words_kernel");
    });
}

// The words' table has eight slots for each word of a document of mean length (longer ones fit up to seven times that), and so many that
// a document of more words, done by ranges of columns, has at most 64 ranges, up to 786,432 columns; beyond, the table has its most slots, and there
// is a range for every 12,288 columns.  Where sums for all columns take no more room there is no table (0 slots); *columns: of a
// range.  (With four slots a word 1,000 documents of 100 words over 5,000 columns, with the loss, took 21 us, as the few that were
// too long held up the end; so 15.  14,235 of 22 over 400 28 and 27.)
int32_t table_slots(int64_t rows, int64_t n_tokens, int32_t cols, int32_t* columns) {
    constexpr int32_t kMostSlots = 8192;
    int32_t slots = 64;
    while (slots < kMostSlots && ((int64_t)slots * rows < 8 * n_tokens || slots < cols / 96)) slots *= 2;
    *columns = slots * mlda::kSlotBytes / 8;
    if (cols > *columns) return slots;
    *columns = cols;
    return 0;
}

// Threads that share a row, by its bytes.  Loss and gradient with 64, 256 and 512 threads: 20,000 x 3,001 bf16 62, 109 and 190 us,
// 1,000 x 5,000 fp32 30, 15 and 19, 8,000 x 12,000 fp32 193, 151 and 176, 1,024 x 102,000 bf16 346, 142 and 109.
int grad_threads(int64_t cols, int32_t type) {
    const int64_t bytes = cols * (int64_t)type_bytes(type);
    return bytes <= kWaveRowBytes ? 64 : bytes <= kGroupRowBytes ? 256 : 512;
}

template <bool kLoss>
int run_grad(mlda::LogprobGradArgs a, int32_t type, hipStream_t stream) {
    const bool single = !a.row_ptr;
    a.slots = a.columns = 0;
    a.once = passes_caches(2.0 * a.rows * a.vocab * type_bytes(type));
    if (!single) a.slots = table_slots(a.rows, a.n_tokens, a.segment_cols, &a.columns);
    const unsigned lds = (unsigned)std::max(a.slots * mlda::kSlotBytes, a.columns * 8);
    const dim3 grid((unsigned)std::min(a.rows * a.segments, kMostGroups));
    return with_type(type, [&](auto t) {
        typedef decltype(t) T;
        auto launch = [&](auto threads) {
            constexpr int kThreads = decltype(threads)::value;
            void (*kernel)(mlda::LogprobGradArgs);
            if (kLoss || !a.grad_entropy)
                kernel = single ? mlda::logprob_grad_kernel<T, kThreads, kLoss, false, true> : mlda::logprob_grad_kernel<T, kThreads, kLoss, false, false>;
            else
                kernel = single ? mlda::logprob_grad_kernel<T, kThreads, false, true, true> : mlda::logprob_grad_kernel<T, kThreads, false, true, false>;
            if (lds > 48 * 1024) {
                const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
                if (e != hipSuccess) return set_error(MLDA_EHIP, "logprob_grad_kernel's LDS", hipGetErrorString(e));
            }
            hipLaunchKernelGGL(kernel, grid, dim3(kThreads), lds, stream, a);
            return launched("logprob_grad_kernel");
        };
        switch (a.n_tokens / a.rows > 512 ? 512 : grad_threads(a.segment_cols, type)) {
        case 64: return launch(std::integral_constant<int, 64>());
        case 256: return launch(std::integral_constant<int, 256>());
        default: return launch(std::integral_constant<int, 512>());
        }
    });
}

int check_grad_out(const void* out, int64_t out_stride, const void* logits, int64_t stride, int64_t rows, int32_t vocab, int32_t type) {
    RC_TRY(check_rows(out, out_stride, rows, vocab, type, "log-probabilities: grad_logits are null",
                      "log-probabilities: rows of grad_logits overlap or are not aligned to their type"));
    if (out == logits && out_stride != stride && rows > 1)
        return refuse("log-probabilities: a gradient in the place of the logits has their stride");
    return MLDA_OK;
}

// ---------------------------------------------------------------- clipping
int check_tensors(const void* const* tensors, const int64_t* sizes, const int32_t* types, int32_t n) {
    if (n < 0) return refuse("gradients: n_tensors must be >= 0");
    if (n == 0) return MLDA_OK;
    if (!tensors || !sizes || !types) return refuse("gradients: the list of tensors, sizes or types is null");
    for (int32_t i = 0; i < n; ++i) {
        if (sizes[i] < 0 || sizes[i] > ((int64_t)1 << 40)) return refuse("gradients: a tensor's size is outside 0 .. 2^40");
        if (!known_type(types[i])) return refuse("gradients: unknown type");
        if (sizes[i] > 0 && (!tensors[i] || !aligned(tensors[i], type_bytes(types[i]))))
            return refuse("gradients: a tensor is null or not aligned to its type");
    }
    return MLDA_OK;
}

int32_t clip_launches(int32_t n) { return std::max(1, (n + mlda::kClipTensors - 1) / mlda::kClipTensors); }

// Calls f(args, grid, launch) for each launch's share of the tensors.
template <class F>
int for_launches(const void* const* in, void* const* out, const int64_t* sizes, const int32_t* types, int32_t n, F&& f) {
    for (int32_t l = 0; l < clip_launches(n); ++l) {
        mlda::ClipArgs a;
        a.partial = nullptr;
        const int32_t first = l * mlda::kClipTensors;
        a.tensors = std::min(n - first, mlda::kClipTensors);
        uint64_t units = 0;
        for (int32_t i = 0; i < a.tensors; ++i) {
            a.tensor[i] = mlda::ClipTensor{in[first + i], out ? out[first + i] : nullptr, sizes[first + i]};
            a.type[i] = (uint8_t)types[first + i];
            a.first_unit[i] = (uint32_t)units;
            units += (uint64_t)((sizes[first + i] + mlda::kClipUnit - 1) / mlda::kClipUnit);
        }
        if (units > 0xffffffffull) return refuse("gradients: more than 2^32 units of elements in one launch's tensors");
        a.first_unit[a.tensors] = (uint32_t)units;
        RC_TRY(f(a, units));
    }
    return MLDA_OK;
}

}  // namespace

extern "C" {

int mlda_layer_norm(const void* x, int64_t x_stride, const void* weight, const void* bias, void* y, int64_t y_stride,
                    float* mean, float* rstd, int64_t rows, int32_t cols, double eps, int32_t type, int32_t weight_type,
                    void* hip_stream) {
    RC_TRY(check_layer_norm(rows, cols, type, weight_type));
    if (!(eps >= 0.0) || !(eps <= 3.4e38)) return refuse("layer norm: eps must be finite and >= 0");
    if (rows == 0) return MLDA_OK;
    RC_TRY(check_rows(x, x_stride, rows, cols, type, "layer norm: x is null", "layer norm: rows of x overlap or are not aligned to their type"));
    RC_TRY(check_rows(y, y_stride, rows, cols, type, "layer norm: y is null", "layer norm: rows of y overlap or are not aligned to their type"));
    if (x == y && x_stride != y_stride && rows > 1) return refuse("layer norm: y in the place of x has its stride");
    if (!aligned(weight, type_bytes(weight_type)) || !aligned(bias, type_bytes(weight_type)) || !aligned(mean, 4) || !aligned(rstd, 4))
        return refuse("layer norm: weight, bias, mean or rstd is not aligned to its type");
    const mlda::LayerNormArgs a{x, x_stride, weight, bias, y, y_stride, mean, rstd, rows, cols, (float)eps,
                                passes_caches(2.0 * rows * cols * type_bytes(type))};
    const hipStream_t stream = (hipStream_t)hip_stream;
    return with_types(type, weight_type, [&](auto t, auto w) {
        typedef decltype(t) T;
        typedef decltype(w) W;
        const int64_t bytes = cols * (int64_t)sizeof(T);
        if (bytes > kHeldBytes) {
            hipLaunchKernelGGL((mlda::layer_norm_long_kernel<T, W>), dim3((unsigned)std::min(rows, kMostGroups)), dim3(1024), 0, stream, a);
        } else {
            with_team(bytes, [&](auto t) {
                constexpr int kThreads = mlda::team_threads(t.team), kTeams = kThreads / t.team;
                // (3,001 x 30,000 bf16 with fp32 weights, which fill the registers, 74 us, held 77)
                constexpr bool kHeld = t.pieces * t.team < (sizeof(W) > sizeof(T) ? 4096 : 8192);
                const int64_t groups = std::min<int64_t>((rows + kTeams - 1) / kTeams, kThreads == 256 ? 8 * kCus : 2 * kCus);
                hipLaunchKernelGGL((mlda::layer_norm_kernel<T, W, t.team, t.pieces, kHeld>), dim3((unsigned)groups), dim3(kThreads), 0, stream, a);
            });
        }
        return launched("layer_norm_kernel");
    });
}

int mlda_layer_norm_workspace_bytes(int64_t rows, int32_t cols, size_t* bytes) {
    if (!bytes) return refuse("bytes is null");
    RC_TRY(check_layer_norm(rows, cols, MLDA_FP32, MLDA_FP32));
    *bytes = rows == 0 ? 0 : (size_t)std::max(norm_grad_groups(rows, cols, MLDA_FP32), norm_grad_groups(rows, cols, MLDA_BF16)) * 2 * (size_t)cols * 4;
    return MLDA_OK;
}

int mlda_layer_norm_backward(const void* grad_y, int64_t grad_y_stride, const void* x, int64_t x_stride, const float* mean,
                             const float* rstd, const void* weight, void* grad_x, int64_t grad_x_stride, void* grad_weight,
                             void* grad_bias, int64_t rows, int32_t cols, int32_t type, int32_t weight_type,
                             void* dev_workspace, size_t workspace_bytes, void* hip_stream) {
    RC_TRY(check_layer_norm(rows, cols, type, weight_type));
    const bool sums = grad_weight || grad_bias;
    if (!aligned(weight, type_bytes(weight_type)) || !aligned(grad_weight, type_bytes(weight_type)) || !aligned(grad_bias, type_bytes(weight_type)))
        return refuse("layer norm: weight or its gradient is not aligned to its type");
    mlda::LayerNormGradArgs a{grad_y, grad_y_stride, x, x_stride, mean, rstd, weight, grad_x, grad_x_stride, nullptr, nullptr, nullptr, rows, cols,
                              passes_caches(3.0 * rows * cols * type_bytes(type))};
    const int32_t groups = norm_grad_groups(rows, cols, type);
    if (rows > 0) {
        RC_TRY(check_rows(x, x_stride, rows, cols, type, "layer norm: x is null", "layer norm: rows of x overlap or are not aligned to their type"));
        RC_TRY(check_rows(grad_y, grad_y_stride, rows, cols, type, "layer norm: grad_y is null", "layer norm: rows of grad_y overlap or are not aligned to their type"));
        if (!mean || !rstd || !aligned(mean, 4) || !aligned(rstd, 4)) return refuse("layer norm: mean or rstd is null or not aligned to its type");
        if (grad_x) {
            RC_TRY(check_rows(grad_x, grad_x_stride, rows, cols, type, "", "layer norm: rows of grad_x overlap or are not aligned to their type"));
            if (((grad_x == x && grad_x_stride != x_stride) || (grad_x == grad_y && grad_x_stride != grad_y_stride)) && rows > 1)
                return refuse("layer norm: grad_x in the place of an input has its stride");
        }
        if (sums) {
            if (!dev_workspace || !aligned(dev_workspace, 4)) return refuse("layer norm: the workspace is null or not aligned");
            if (workspace_bytes < (size_t)groups * 2 * (size_t)cols * 4)
                return set_error(MLDA_ENOMEM, "layer norm: the workspace is smaller than mlda_layer_norm_workspace_bytes");
            if (groups > 1 || cols * (int64_t)type_bytes(type) > summed_bytes((int64_t)type_bytes(type))) {
                a.partial = static_cast<float*>(dev_workspace);
            } else {
                a.grad_weight = grad_weight;
                a.grad_bias = grad_bias;
            }
        }
    }
    if (!sums && (!grad_x || rows == 0)) return MLDA_OK;
    const hipStream_t stream = (hipStream_t)hip_stream;
    return with_types(type, weight_type, [&](auto t, auto w) {
        typedef decltype(t) T;
        typedef decltype(w) W;
        const int64_t bytes = cols * (int64_t)sizeof(T);
        if (rows > 0 && bytes > summed_bytes(sizeof(T))) {
            // (the sums first: grad_x may be written over what they read)
            if (a.partial) {
                const int32_t tile = mlda::kWave * mlda::kPack<T>;
                hipLaunchKernelGGL((mlda::layer_norm_grad_columns_kernel<T>), dim3((unsigned)((cols + tile - 1) / tile), (unsigned)groups),
                                   dim3(256), 0, stream, a);
                RC_TRY(launched("layer_norm_grad_columns_kernel"));
            }
            const dim3 grid((unsigned)std::min(rows, kMostGroups));
            if (!grad_x) {}
            else if (bytes <= 65536) hipLaunchKernelGGL((mlda::layer_norm_grad_kernel<T, W, 1024, 4, false>), grid, dim3(1024), 0, stream, a);
            else hipLaunchKernelGGL((mlda::layer_norm_grad_long_kernel<T, W>), grid, dim3(1024), 0, stream, a);
        } else if (rows > 0) {
            with_grad_team(bytes, [&](auto t, int) {
                constexpr int kThreads = mlda::team_threads(t.team);
                if constexpr (sizeof(T) == 4 || t.pieces < 4)
                    hipLaunchKernelGGL((mlda::layer_norm_grad_kernel<T, W, t.team, t.pieces, true, (t.pieces < 4)>), dim3((unsigned)groups), dim3(kThreads), 0, stream, a);
            });
        }
        RC_TRY(launched("layer_norm_grad_kernel"));
        if (!sums || (rows > 0 && !a.partial)) return MLDA_OK;
        const int64_t finals = std::min((2 * (int64_t)cols + mlda::kFinalCols - 1) / mlda::kFinalCols, kMostGroups);
        hipLaunchKernelGGL((mlda::layer_norm_grad_final_kernel<W>), dim3((unsigned)finals), dim3(1024), 0, stream, a.partial,
                           rows > 0 ? groups : 0, cols, static_cast<W*>(grad_weight), static_cast<W*>(grad_bias));
        return launched("layer_norm_grad_final_kernel");
    });
}

int mlda_token_logprobs_workspace_bytes(int64_t rows, int32_t vocab, int32_t alternatives, int32_t type, size_t* bytes) {
    if (!bytes) return refuse("bytes is null");
    if (rows < 0 || vocab < 1 || vocab > kMostCols) return refuse("log-probabilities: need rows >= 0 and 1 <= vocab <= 2^30");
    if (!known_type(type)) return refuse("log-probabilities: unknown type");
    if (alternatives < 0 || alternatives > MLDA_MAX_ALTERNATIVES || alternatives > vocab)
        return refuse("log-probabilities: need 0 <= alternatives <= 32, and no more than there are words");
    // (the statistics that mlda_token_logprobs_grad keeps where it works in two steps come on top)
    const size_t parts = logprob_workspace(rows, vocab, alternatives, type);
    *bytes = parts ? parts + (size_t)rows * 8 : 0;
    return MLDA_OK;
}

int mlda_token_logprobs(const void* logits, int64_t stride, int64_t rows, int32_t vocab, int32_t type, const int32_t* tokens,
                        const int64_t* row_ptr, int64_t n_tokens, int32_t alternatives, float* logprobs, float* stats,
                        float* entropy, int32_t* top_ids, float* top_logprobs, void* dev_workspace, size_t workspace_bytes,
                        void* hip_stream) {
    RC_TRY(check_logits(logits, stride, rows, vocab, type, tokens, row_ptr, n_tokens));
    if (alternatives < 0 || alternatives > MLDA_MAX_ALTERNATIVES || alternatives > vocab)
        return refuse("log-probabilities: need 0 <= alternatives <= 32, and no more than there are words");
    if (rows == 0) return MLDA_OK;
    if (n_tokens > 0 && !logprobs) return refuse("log-probabilities: logprobs are null");
    if (alternatives > 0 && (!top_ids || !top_logprobs)) return refuse("log-probabilities: top_ids or top_logprobs is null");
    const size_t need = logprob_workspace(rows, vocab, alternatives, type);
    if (need && (!dev_workspace || !aligned(dev_workspace, 8))) return refuse("log-probabilities: the workspace is null or not aligned");
    if (workspace_bytes < need) return set_error(MLDA_ENOMEM, "log-probabilities: the workspace is smaller than mlda_token_logprobs_workspace_bytes");
    const mlda::LogprobArgs a{logits, stride, rows, vocab, tokens, row_ptr, n_tokens, alternatives, logprobs, stats, entropy,
                              top_ids, top_logprobs, 1, vocab, false, nullptr, nullptr};
    return run_logprobs(a, type, dev_workspace, (hipStream_t)hip_stream);
}

int mlda_token_logprobs_backward(const void* logits, int64_t stride, int64_t rows, int32_t vocab, int32_t type, const int32_t* tokens,
                                 const int64_t* row_ptr, int64_t n_tokens, const float* stats, const float* grad_logprobs,
                                 const float* entropy, const float* grad_entropy, void* grad_logits, int64_t grad_stride,
                                 void* hip_stream) {
    RC_TRY(check_logits(logits, stride, rows, vocab, type, tokens, row_ptr, n_tokens));
    if (rows == 0) return MLDA_OK;
    RC_TRY(check_grad_out(grad_logits, grad_stride, logits, stride, rows, vocab, type));
    if (!stats || (n_tokens > 0 && !grad_logprobs)) return refuse("log-probabilities: stats or grad_logprobs are null");
    if (grad_entropy && !entropy) return refuse("log-probabilities: a gradient of the entropy needs the entropy");
    mlda::LogprobGradArgs a{logits, stride, rows, vocab, tokens, row_ptr, n_tokens, grad_logprobs, stats, entropy,
                            grad_entropy, nullptr, grad_logits, grad_stride, 1, vocab, 0, 0, false};
    segments_of(rows, vocab, 1024 * (int32_t)(16 / type_bytes(type)), &a.segments, &a.segment_cols);
    return run_grad<false>(a, type, (hipStream_t)hip_stream);
}

int mlda_token_logprobs_grad(const void* logits, int64_t stride, int64_t rows, int32_t vocab, int32_t type, const int32_t* tokens,
                             const int64_t* row_ptr, int64_t n_tokens, const float* weights, float* logprobs, void* grad_logits,
                             int64_t grad_stride, void* dev_workspace, size_t workspace_bytes, void* hip_stream) {
    RC_TRY(check_logits(logits, stride, rows, vocab, type, tokens, row_ptr, n_tokens));
    if (rows == 0) return MLDA_OK;
    RC_TRY(check_grad_out(grad_logits, grad_stride, logits, stride, rows, vocab, type));
    if (n_tokens > 0 && (!weights || !logprobs)) return refuse("log-probabilities: weights or logprobs are null");
    const size_t parts = logprob_workspace(rows, vocab, 0, type);
    const hipStream_t stream = (hipStream_t)hip_stream;
    if (parts) {
        // few rows: the statistics by segments, then the gradient by segments
        if (!dev_workspace || !aligned(dev_workspace, 8)) return refuse("log-probabilities: the workspace is null or not aligned");
        if (workspace_bytes < parts + (size_t)rows * 8)
            return set_error(MLDA_ENOMEM, "log-probabilities: the workspace is smaller than mlda_token_logprobs_workspace_bytes");
        float* stats = reinterpret_cast<float*>(static_cast<char*>(dev_workspace) + parts);
        const mlda::LogprobArgs f{logits, stride, rows, vocab, tokens, row_ptr, n_tokens, 0, logprobs, stats, nullptr,
                                  nullptr, nullptr, 1, vocab, false, nullptr, nullptr};
        RC_TRY(run_logprobs(f, type, dev_workspace, stream));
        return mlda_token_logprobs_backward(logits, stride, rows, vocab, type, tokens, row_ptr, n_tokens, stats, weights, nullptr,
                                            nullptr, grad_logits, grad_stride, hip_stream);
    }
    const mlda::LogprobGradArgs a{logits, stride, rows, vocab, tokens, row_ptr, n_tokens, weights, nullptr, nullptr, nullptr, logprobs,
                                  grad_logits, grad_stride, 1, vocab, 0, 0, false};
    return run_grad<true>(a, type, stream);
}

int mlda_grad_norm_workspace_bytes(int32_t n_tensors, size_t* bytes) {
    if (!bytes) return refuse("bytes is null");
    if (n_tensors < 0) return refuse("gradients: n_tensors must be >= 0");
    *bytes = (size_t)clip_launches(n_tensors) * mlda::kClipGroups * 8;
    return MLDA_OK;
}

}  // extern "C"

namespace {

unsigned clip_groups(uint64_t units) { return (unsigned)std::max<uint64_t>(1, std::min<uint64_t>(units, mlda::kClipGroups)); }

// The workgroups' sums of squares, packed: the number of them is returned in *partials.
int sum_squares(const void* const* tensors, const int64_t* sizes, const int32_t* types, int32_t n, double* partial, int32_t* partials, hipStream_t stream) {
    *partials = 0;
    return for_launches(tensors, nullptr, sizes, types, n, [&](mlda::ClipArgs& a, uint64_t units) {
        const unsigned groups = clip_groups(units);
        a.partial = partial + *partials;
        *partials += (int32_t)groups;
        hipLaunchKernelGGL(mlda::square_sums_kernel, dim3(groups), dim3(mlda::kClipThreads), 0, stream, a);
        return launched("square_sums_kernel");
    });
}

int check_clip(const void* const* tensors, const int64_t* sizes, const int32_t* types, int32_t n, const float* norm, const void* workspace, size_t bytes) {
    RC_TRY(check_tensors(tensors, sizes, types, n));
    if (!norm || !aligned(norm, 4)) return refuse("gradients: norm is null or not aligned");
    if (!workspace || !aligned(workspace, 8)) return refuse("gradients: the workspace is null or not aligned");
    if (bytes < (size_t)clip_launches(n) * mlda::kClipGroups * 8)
        return set_error(MLDA_ENOMEM, "gradients: the workspace is smaller than mlda_grad_norm_workspace_bytes");
    return MLDA_OK;
}

}  // namespace

extern "C" {

int mlda_grad_norm(const void* const* tensors, const int64_t* sizes, const int32_t* types, int32_t n_tensors, float* norm,
                   void* dev_workspace, size_t workspace_bytes, void* hip_stream) {
    RC_TRY(check_clip(tensors, sizes, types, n_tensors, norm, dev_workspace, workspace_bytes));
    double* partial = static_cast<double*>(dev_workspace);
    int32_t partials = 0;
    RC_TRY(sum_squares(tensors, sizes, types, n_tensors, partial, &partials, (hipStream_t)hip_stream));
    hipLaunchKernelGGL(mlda::norm_kernel, dim3(1), dim3(mlda::kClipThreads), 0, (hipStream_t)hip_stream, partial, partials, norm);
    return launched("norm_kernel");
}

int mlda_clip_grads(const void* const* tensors, void* const* out, const int64_t* sizes, const int32_t* types, int32_t n_tensors,
                    double max_norm, float* norm, void* dev_workspace, size_t workspace_bytes, void* hip_stream) {
    RC_TRY(check_clip(tensors, sizes, types, n_tensors, norm, dev_workspace, workspace_bytes));
    if (!(max_norm >= 0.0)) return refuse("gradients: max_norm must be >= 0");
    if (n_tensors > 0 && !out) return refuse("gradients: the list of outputs is null");
    for (int32_t i = 0; i < n_tensors; ++i)
        if (sizes[i] > 0 && (!out[i] || !aligned(out[i], type_bytes(types[i])))) return refuse("gradients: an output is null or not aligned to its type");
    double* partial = static_cast<double*>(dev_workspace);
    int32_t partials = 0;
    const hipStream_t stream = (hipStream_t)hip_stream;
    RC_TRY(sum_squares(tensors, sizes, types, n_tensors, partial, &partials, stream));
    return for_launches(tensors, out, sizes, types, n_tensors, [&](mlda::ClipArgs& a, uint64_t units) {
        hipLaunchKernelGGL(mlda::clip_kernel, dim3(clip_groups(units)), dim3(mlda::kClipThreads), 0, stream, a, partial, partials, max_norm, norm);
        return launched("clip_kernel");
    });
}

}  // extern "C"
