// Log-probabilities of given words out of rows of logits, the distributions' entropies, the likeliest
// words, and the gradient with respect to the logits.
//
// With m = max_v x_v, s = sum_v exp(x_v - m), p_v = exp(x_v - m) / s of a row:
//   log p(word) = x_word - m - ln s
//   H           = -sum_v p_v ln p_v = ln s - sum_v exp(x_v - m) (x_v - m) / s
//   d/dx_v of  sum_t g_t log p(word_t) + h H  =  sum_{t: word_t = v} g_t  -  p_v (G + h (x_v - m - ln s + H)),  G = sum_t g_t
//
// One pass over a row has the maximum, both sums and the likeliest words: each lane keeps a running maximum and rescales
// its sums when it grows; lanes, waves and segments of a row are joined at the end.  Bound by memory where the logits have 4 bytes;
// with 2 by the vector instructions issued (with entropies and likeliest words 11 to 15 an element).
//
// The statistics of a row are kept as the pair (m, ln s): their sum is the logarithm of the sum of exponentials, and
// differences to m lose nothing where m is large.  A row whose logits are all minus infinity has (-inf, 0).
#pragma once
#include "vec_io.hpp"

namespace mlda {

constexpr int kMaxAlternatives = 32;
constexpr int kHeld = 128;                       // candidates a wave holds before it sorts them: two a lane
constexpr int kTilePieces = 2;                   // 16-byte pieces of a row that a lane has on their way
constexpr float kLog2E = 1.44269504088896340736f;
constexpr float kLowest = -3.402823466e+38f;
constexpr float kVanished = -200.0f;             // exponentials of less are 0 in fp32: what they are multiplied with may stay finite
constexpr int kLogprobWaves = 4;                 // of a workgroup with a row, or a segment of one; one wave for a short row

template <class T> constexpr int kTileCols = kWave * kTilePieces * kPack<T>;    // columns of a wave's tile

struct RowPart {          // what a segment of a row comes to
    double s, u;          // sums of exp(x - m) and of exp(x - m) (x - m)
    float m;
    int32_t n;            // candidates
};

struct LogprobArgs {
    const void* logits;
    int64_t stride, rows;
    int32_t vocab;
    const int32_t* tokens;       // words; below zero: none
    const int64_t* row_ptr;      // null: one word to a row
    int64_t n_tokens;
    int32_t top;
    float* logprobs;
    float* stats;                // [rows][2]
    float* entropy;              // null: not wanted
    int32_t* top_ids;
    float* top_logprobs;
    int32_t segments;            // of a row, at most a wave's lanes, of segment_cols columns each (a multiple of the workgroup's tiles)
    int32_t segment_cols;
    bool words_apart;            // the words' log-probabilities are left to logprob_words_kernel
    RowPart* parts;              // [rows][segments]
    uint64_t* part_top;          // [rows][segments][top]
};

// A stretch of a row as sums over it are taken.  (Its pieces begin at its first column, wherever that lies: what a row comes to does
// not depend on its address.)
template <class T>
struct Span {
    const T* row;
    int32_t first, end;
    __device__ __forceinline__ Raw load(int64_t c, float fill) const { return load_some(row + c, (int)max((int64_t)0, min((int64_t)kPack<T>, end - c)), fill, c - first); }
};

// ---------------------------------------------------------------- the order of the alternatives
// Greater logits first, then lower words; NaN after every number.  A logit's key is a whole number in that order; 0 is kept
// for "no word".
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);                  // (minus zero is zero)
    const uint32_t k = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
    return x == x ? k : 1u;
}
__device__ __forceinline__ float key_logit(uint32_t k) {
    if (k == 1u) return __uint_as_float(0x7fc00000u);
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
__device__ __forceinline__ uint64_t candidate(uint32_t key, int32_t word) { return (uint64_t)key << 32 | (uint32_t)~word; }
__device__ __forceinline__ int32_t candidate_word(uint64_t c) { return (int32_t)~(uint32_t)c; }

// LDS of a wave that other lanes of the same wave have written: the hardware keeps a wave's LDS accesses in order, the compiler must, too.
__device__ __forceinline__ void wave_lds_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Puts the `n` greatest of held[0 .. count) (count <= kHeld, all different) first, in descending order.  By one wave; every lane takes
// part.  Returns how many there are now.
__device__ __forceinline__ int keep_greatest(uint64_t* held, int count, int n) {
    const int lane = lane_id();
    wave_lds_fence();
    const uint64_t a = lane < count ? held[lane] : 0, b = lane + kWave < count ? held[lane + kWave] : 0;
    int rank_a = 0, rank_b = 0;
    if (count <= kWave) {
#pragma unroll 8
        for (int i = 0; i < count; ++i) rank_a += held[i] > a ? 1 : 0;
    } else {
#pragma unroll 8
        for (int i = 0; i < count; ++i) {
            const uint64_t c = held[i];
            rank_a += c > a ? 1 : 0;
            rank_b += c > b ? 1 : 0;
        }
    }
    wave_lds_fence();
    if (lane < count && rank_a < n) held[rank_a] = a;
    if (lane + kWave < count && rank_b < n) held[rank_b] = b;
    wave_lds_fence();
    return min(count, n);
}

// The greatest key, of those that end in sixteen zeros, that at least n lanes' keys reach (0 if fewer than n have one).
__device__ __forceinline__ uint32_t nth_key(uint32_t key, int n) {
    uint32_t found = 0;
#pragma unroll 4
    for (int bit = 31; bit >= 16; --bit) {
        const uint32_t with = found | 1u << bit;
        if (__popcll(__ballot(key >= with)) >= n) found = with;
    }
    return found;
}

// A wave's candidates for the alternatives of a row.
struct Candidates {
    uint64_t* held;        // LDS, kHeld of them
    int n, count = 0;      // wanted; held
    uint64_t least = 0;    // the n-th greatest so far, if there are n
    float bar = 0.0f;      // its logit

    __device__ __forceinline__ void sort() {
        count = keep_greatest(held, count, n);
        if (count == n) {
            const uint64_t c = held[n - 1];
            least = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(c >> 32)) << 32 |
                    (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)c);
            bar = key_logit((uint32_t)(least >> 32));
        }
    }
    // Whether a tile may have something to add, by each lane's maximum of it.  Columns ascend from tile to tile, so an equal logit
    // of a later tile comes after those held.  (A bar that is NaN lets everything through.)
    __device__ __forceinline__ bool wants(float lane_max) const { return count < n || __ballot(!(lane_max <= bar)) != 0; }

    // The tile of columns [first, first + kTileCols) of a row, read once more (from the caches).  At least n of its logits reach the n-th
    // greatest of the lanes' maxima, so only those can be among the n greatest.
    template <class T>
    __device__ __forceinline__ void add(const Span<T>& span, int64_t first) {
        constexpr int P = kPack<T>;
        auto piece = [&](int j, float (&v)[P]) {
            const int64_t c = first + (j * kWave + lane_id()) * P;
            unpack(span.load(c, 0.0f), v, T());
            return c;
        };
        uint32_t most = 0;
#pragma unroll 1
        for (int j = 0; j < kTilePieces; ++j) {
            float v[P];
            const int64_t c = piece(j, v);
#pragma unroll
            for (int e = 0; e < P; ++e) most = max(most, c + e < span.end ? order_key(v[e]) : 0u);
        }
        const uint32_t floor = max(nth_key(most, n), 1u);
#pragma unroll 1
        for (int j = 0; j < kTilePieces; ++j) {
            float v[P];
            const int64_t c = piece(j, v);
#pragma unroll
            for (int e = 0; e < P; ++e) {
                const uint32_t key = c + e < span.end ? order_key(v[e]) : 0u;
                const uint64_t mine = candidate(key, (int32_t)(c + e));
                uint64_t mask = __ballot(key >= floor && mine > least);
                if (mask) {
                    if (count + __popcll(mask) > kHeld) {
                        sort();
                        mask = __ballot(key >= floor && mine > least);
                    }
                    if (key >= floor && mine > least) held[count + __popcll(mask & lanes_below())] = mine;
                    count += __popcll(mask);
                }
            }
        }
        if (count >= n) sort();
    }
};

// ---------------------------------------------------------------- one pass over a row, or a segment
// x - m for a bound m of x, and its exponential.  The product t = d log2(e) alone, rounded, would leave an exponential with |d| units of
// roundoff: w = d - t ln(2) is what it leaves out, and 2^t + 2^t w is within three units at any distance (2,400 x 102,000 fp32 176 us,
// 174 without).  Logits of 16 bits have 2^-9 or 2^-12 of themselves for an error, and their kernels are held up by instructions: there the
// product is taken as it is (1,024 x 102,000 bf16 40 us, with w 50; 6,007 x 40,009 with the 20 likeliest words 131, with w 142).
constexpr float kLn2 = 0.693147182464599609375f, kLn2Low = -1.904654299957768e-9f;      // ln(2) as fp32 has it, and the rest
template <class T>
constexpr bool kExact = sizeof(T) == 4;

template <class T>
__device__ __forceinline__ float below(float x, float m) {
    if constexpr (kExact<T>) return __builtin_elementwise_maximum(x - m, kVanished);     // (NaN stays NaN; t - t is none at infinity)
    return x - m;
}
template <class T>
__device__ __forceinline__ float exp_of(float d) {
    const float t = d * kLog2E, e = __builtin_amdgcn_exp2f(t);       // (a product may overflow to minus infinity, which is meant)
    if constexpr (!kExact<T>) return e;
    return __builtin_fmaf(e, __builtin_fmaf(-t, kLn2Low, __builtin_fmaf(-t, kLn2, d)), e);
}

struct LaneSums {
    float m = kLowest;        // (a finite bound: minus infinity minus it is minus infinity, whose exponential is 0)
    float s = 0.0f, u = 0.0f;

    __device__ __forceinline__ void raise(float to) {
        if (to > m) {
            const float d = below<float>(m, to);
            const float f = exp_of<float>(d);
            u = f * __builtin_fmaf(d, s, u);
            s *= f;
            m = to;
        }
    }
    template <class T, bool kEntropy>
    __device__ __forceinline__ void add(float x) {
        const float d = below<T>(x, m), e = exp_of<T>(d);
        s += e;
        if constexpr (kEntropy) u = __builtin_fmaf(e, fmaxf(d, kVanished), u);
    }
};

// A lane's sums over all of its tiles.
struct RowSums {
    float m;
    double s, u;
};

// The fp32 sums of a lane lose more the more terms have been added one after the other, so that after so many tiles (256 terms) they
// go into sums in fp64.  Few rows have more, and a lane's registers decide how many rows a CU has: these sums are in LDS, each read and
// written by its own thread only.
template <class T> constexpr int kFoldTiles = 256 / (kTilePieces * kPack<T>);

template <int kThreads>
struct FoldLds {
    double s[kThreads], u[kThreads];
    float m[kThreads];
};

struct Fold {
    double *s, *u;                                   // of this thread, in LDS
    float* m;                                        // the bound they are relative to
    bool empty = true;

    template <int kThreads>
    __device__ __forceinline__ explicit Fold(FoldLds<kThreads>& lds) : s(&lds.s[threadIdx.x]), u(&lds.u[threadIdx.x]), m(&lds.m[threadIdx.x]) {}
    __device__ __forceinline__ Fold(double* s_at, double* u_at, float* m_at) : s(s_at), u(u_at), m(m_at) {}

    // (a lane's bound only grows)
    __device__ __forceinline__ RowSums with(const LaneSums& l) const {
        if (empty) return RowSums{l.m, (double)l.s, (double)l.u};
        const float d = below<float>(*m, l.m);
        const double f = exp_of<float>(d);
        return RowSums{l.m, f * *s + (double)l.s, f * __builtin_fma((double)d, *s, *u) + (double)l.u};
    }
    __device__ __forceinline__ void take(LaneSums& l) {
        const RowSums r = with(l);
        *s = r.s;
        *u = r.u;
        *m = r.m;
        l.s = l.u = 0.0f;
        empty = false;
    }
};

// The sums of all lanes of a wave, each relative to its own bound, as one, relative to the greatest.
__device__ __forceinline__ void join_lanes(float& m, double& s, double& u) {
    const float most = wave_max(m), d = below<float>(m, most);
    const double f = s != 0.0 ? (double)exp_of<float>(d) : 0.0;
    u = wave_sum(f != 0.0 ? f * (u + (double)d * s) : 0.0);
    s = wave_sum(f * s);
    m = most;
}

// The parts that the waves of a workgroup have left, as one; every wave gets it.
__device__ __forceinline__ void join_parts(const RowPart* part, int n, float& m, double& s, double& u) {
    const int lane = lane_id();
    m = lane < n ? part[lane].m : kLowest;
    s = lane < n ? part[lane].s : 0.0;
    u = lane < n ? part[lane].u : 0.0;
    join_lanes(m, s, u);
}

// f(raw pieces, first column) for the tiles of a span that are this wave's, where `waves` take them in turn; the next tile's loads
// are on their way meanwhile.  Past the end there is minus infinity.
template <class T, class F>
__device__ __forceinline__ void for_tiles(const Span<T>& span, int wave, int waves, F&& f) {
    constexpr int P = kPack<T>, kCols = kTileCols<T>;
    const int lane = lane_id();
    Raw next[kTilePieces];
    auto load = [&](int64_t first) {
        if (first + kCols <= span.end) {
#pragma unroll
            for (int j = 0; j < kTilePieces; ++j) next[j] = load_raw(span.row + first + (j * kWave + lane) * P);
        } else {
#pragma unroll
            for (int j = 0; j < kTilePieces; ++j) next[j] = span.load(first + (j * kWave + lane) * P, -INFINITY);
        }
    };
    // (the first round only loads)
    const int64_t start = span.first + (int64_t)wave * kCols, step = (int64_t)waves * kCols;
    for (int64_t first = start - step; first < span.end; first += step) {
        Raw now[kTilePieces];
#pragma unroll
        for (int j = 0; j < kTilePieces; ++j) now[j] = next[j];
        if (first + step < span.end) load(first + step);
        if (first >= start) f(now, first);
    }
}

template <class T>
__device__ __forceinline__ float tile_max(const Raw (&now)[kTilePieces]) {
    constexpr int P = kPack<T>;
    float most = -INFINITY;
#pragma unroll
    for (int j = 0; j < kTilePieces; ++j) {
        float v[P];
        unpack(now[j], v, T());
#pragma unroll
        for (int e = 0; e < P; ++e) most = fmaxf(most, v[e]);
    }
    return most;
}

// `seen(greatest logit of the tile)` is called for each tile of the wave.
template <class T, bool kEntropy, class Seen>
__device__ __forceinline__ RowSums walk_row(const Span<T>& span, int wave, int waves, Fold folded, Seen&& seen) {
    constexpr int P = kPack<T>;
    LaneSums sums;
    int tiles = 0;
    for_tiles(span, wave, waves, [&](const Raw (&now)[kTilePieces], int64_t) {
        const float most = tile_max<T>(now);
        seen(most);
        sums.raise(most);
#pragma unroll
        for (int j = 0; j < kTilePieces; ++j) {
            float v[P];
            unpack(now[j], v, T());
#pragma unroll
            for (int e = 0; e < P; ++e) sums.add<T, kEntropy>(v[e]);
        }
        if (++tiles == kFoldTiles<T>) {
            folded.take(sums);
            tiles = 0;
        }
    });
    return folded.with(sums);
}

// The log-probability of a word of that logit: NaN for one outside the vocabulary, 0 for none.
__device__ __forceinline__ float logprob_of(float logit, int32_t word, int32_t vocab, float m, float log_s) {
    if (word < 0) return 0.0f;
    if (word >= vocab) return __uint_as_float(0x7fc00000u);
    if (m == -INFINITY) return -INFINITY;
    return (logit - m) - log_s;
}
template <class T>
__device__ __forceinline__ float word_logprob(const T* row, int32_t word, int32_t vocab, float m, float log_s) {
    return logprob_of(word >= 0 && word < vocab ? (float)row[word] : 0.0f, word, vocab, m, log_s);
}

// The words of a row: [begin, end) of the tokens, whatever the bounds say.
__device__ __forceinline__ void row_tokens(const int64_t* row_ptr, int64_t n_tokens, int64_t row, int64_t& begin, int64_t& end) {
    if (row_ptr) {
        begin = min(max(row_ptr[row], (int64_t)0), n_tokens);
        end = min(max(row_ptr[row + 1], begin), n_tokens);
    } else {
        begin = row;
        end = row + 1;
    }
}

// Tokens before the first row's and behind the last row's are no row's words: their log-probability is 0, as a word's below zero.  Every
// kRestRows-th row clears a share of them: a batch out of a long list of tokens does not leave them all to one workgroup, and few
// rows look for the bounds (with all of them 14,235 x 400 took 6% longer).
constexpr int kRestRows = 64;
template <int kThreads>
__device__ __forceinline__ void clear_rest(const int64_t* row_ptr, int64_t rows, int64_t n_tokens, int64_t row, float* logprobs) {
    if (!row_ptr || row % kRestRows != 0) return;
    const int64_t head = min(max(row_ptr[0], (int64_t)0), n_tokens), tail = min(max(row_ptr[rows], head), n_tokens);
    const int64_t n = head + (n_tokens - tail), part = row / kRestRows, parts = (rows + kRestRows - 1) / kRestRows;
    if (n == 0) return;
    const int64_t last = n * (part + 1) / parts;
    for (int64_t i = n * part / parts + threadIdx.x; i < last; i += kThreads) logprobs[i < head ? i : tail + (i - head)] = 0.0f;
}

constexpr int kWordBatch = 4;                     // words that a thread has on their way

// f(token's number, word, is there one) for the tokens [begin, end), `threads` threads side by side; every thread calls it as often.
template <int kThreads, class F>
__device__ __forceinline__ void for_words(const int32_t* tokens, int64_t begin, int64_t end, int tid, F&& f) {
    for (int64_t first = begin; first < end; first += kThreads * kWordBatch) {
        int64_t t[kWordBatch];
        int32_t word[kWordBatch];
        bool there[kWordBatch];
#pragma unroll
        for (int k = 0; k < kWordBatch; ++k) {
            t[k] = first + k * kThreads + tid;
            there[k] = t[k] < end;
            word[k] = there[k] ? tokens[t[k]] : -1;
        }
        f(t, word, there);
    }
}

// Their log-probabilities.
template <class T, int kThreads>
__device__ __forceinline__ void word_logprobs(const T* row, const int32_t* tokens, int64_t begin, int64_t end, int tid, int32_t vocab, float m,
                                              float log_s, float* logprobs) {
    for_words<kThreads>(tokens, begin, end, tid, [&](const int64_t (&t)[kWordBatch], const int32_t (&word)[kWordBatch], const bool (&there)[kWordBatch]) {
        float l[kWordBatch];
#pragma unroll
        for (int k = 0; k < kWordBatch; ++k) l[k] = word_logprob(row, word[k], vocab, m, log_s);
#pragma unroll
        for (int k = 0; k < kWordBatch; ++k)
            if (there[k]) logprobs[t[k]] = l[k];
    });
}

// A row's statistics out of its sums.  No logit above minus infinity: (-inf, 0), entropy 0.
struct RowStats {
    float m, log_s, entropy;
    __device__ __forceinline__ RowStats(float max, double s, double u) {
        if (s == 0.0) {
            m = -INFINITY;
            log_s = entropy = 0.0f;
        } else {
            const double l = log(s);
            m = max;
            log_s = (float)l;
            entropy = (float)(l - u / s);
        }
    }
};

// What a row comes to is written, with its words from the `done`-th on.
template <class T, int kThreads>
__device__ __forceinline__ void finish_row(const LogprobArgs& a, int64_t row, const RowStats& st, const uint64_t* top, int done = 0) {
    if (!a.words_apart) {
        int64_t begin, end;
        row_tokens(a.row_ptr, a.n_tokens, row, begin, end);
        word_logprobs<T, kThreads>(static_cast<const T*>(a.logits) + row * a.stride, a.tokens, min(begin + done, end), end, (int)threadIdx.x, a.vocab, st.m, st.log_s,
                                   a.logprobs);
        clear_rest<kThreads>(a.row_ptr, a.rows, a.n_tokens, row, a.logprobs);
    }
    if (threadIdx.x == 0) {
        if (a.stats) {
            a.stats[2 * row] = st.m;
            a.stats[2 * row + 1] = st.log_s;
        }
        if (a.entropy) a.entropy[row] = st.entropy;
    }
    if ((int)threadIdx.x < a.top) {
        const uint64_t c = top[threadIdx.x];
        const float x = key_logit((uint32_t)(c >> 32));
        a.top_ids[row * a.top + threadIdx.x] = candidate_word(c);
        a.top_logprobs[row * a.top + threadIdx.x] = st.m == -INFINITY ? -INFINITY : (x - st.m) - st.log_s;
    }
}

// The words of long documents, whose rows' statistics are known: `split` workgroups a row.
template <class T>
__global__ __launch_bounds__(kLogprobWaves * kWave) void logprob_words_kernel(LogprobArgs a, int split) {
    constexpr int kThreads = kLogprobWaves * kWave;
    for (int64_t item = blockIdx.x; item < a.rows * split; item += gridDim.x) {
        const int64_t row = item / split;
        int64_t begin, end;
        row_tokens(a.row_ptr, a.n_tokens, row, begin, end);
        const int64_t each = (end - begin + split - 1) / split;
        begin = min(begin + item % split * each, end);
        word_logprobs<T, kThreads>(static_cast<const T*>(a.logits) + row * a.stride, a.tokens, begin, min(begin + each, end), (int)threadIdx.x,
                                   a.vocab, a.stats[2 * row], a.stats[2 * row + 1], a.logprobs);
        if (item % split == 0) clear_rest<kThreads>(a.row_ptr, a.rows, a.n_tokens, row, a.logprobs);
    }
}

// LDS of the search for the likeliest words.
constexpr int kStretches = 16;                    // a wave's tiles are grouped into as many stretches, at most
template <int kWaves>
struct TopLds {
    static constexpr int kLanes = kWaves * kWave;
    float stretch[kStretches][kLanes];            // each lane's greatest logit of each stretch
    float most[kLanes];                           // and of all
    uint64_t best[kHeld];                         // candidates, then the answer
    union {
        uint64_t held[kWaves][kHeld];             // of the waves, where every logit is looked at
        double folded[kWaves][2][kWave];          // before that, with `most`: the lanes' sums so far
    };
    int32_t chosen[kLanes];                       // lane and stretch
    int chosen_n, n, counts[kWaves];
};

// Keeps a lane's maxima by stretches of `tiles` tiles.
template <int kWaves>
struct StretchMost {
    TopLds<kWaves>& lds;
    int tiles, in = 0, at = 0;
    float most = -INFINITY;

    __device__ __forceinline__ void operator()(float tile) {
        most = in ? fmaxf(most, tile) : tile;
        lds.stretch[at][threadIdx.x] = most;
        if (++in == tiles) {
            in = 0;
            ++at;
        }
    }
};

template <class T, int kWaves>
__device__ __forceinline__ int stretch_tiles(const Span<T>& span) {
    constexpr int64_t kGroupCols = (int64_t)kWaves * kTileCols<T>;
    const int64_t tiles = (span.end - span.first + kGroupCols - 1) / kGroupCols;
    return (int)((tiles + kStretches - 1) / kStretches);
}

// The `n` greatest of a span, in order, into lds.best; returns how many there are (to wave 0).  `most`: this
// lane's greatest logit of those that walk_row gave it; lds.stretch is written.  The n-th greatest of the maxima of 64 groups of lanes is
// a bound that n logits reach: the few stretches of few lanes that reach it (about n of some thousand) are looked through once
// more, by everyone, and what reaches the bound is put in order.  Where that is more than the lists have room for (ties), or
// fewer than n lanes have a number, the row is looked through from the start.  By a whole workgroup.
template <class T, int kWaves>
__device__ __forceinline__ int find_top(const Span<T>& span, float most, int n, TopLds<kWaves>& lds) {
    constexpr int P = kPack<T>, kCols = kTileCols<T>, kLanes = kWaves * kWave;
    const int tid = (int)threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave), lane = lane_id();
    lds.most[tid] = most;
    if (tid == 0) lds.chosen_n = lds.n = 0;
    __syncthreads();
    float group = lds.most[lane];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) group = fmaxf(group, lds.most[w * kWave + lane]);
    const uint32_t bound = nth_key(order_key(group), n);
    bool all = bound <= order_key(kLowest);        // (a lane without a number starts from the lowest)
    if (!all) {
        const int tiles = stretch_tiles<T, kWaves>(span);
        if (order_key(most) >= bound) {
            const int64_t first = span.first + (int64_t)wave * kCols, step = (int64_t)kWaves * kCols * tiles;
            for (int i = 0; first + i * step < span.end; ++i)
                if (order_key(lds.stretch[i][tid]) >= bound) {
                    const int at = atomicAdd(&lds.chosen_n, 1);
                    if (at < kLanes) lds.chosen[at] = i * kLanes + tid;
                }
        }
        __syncthreads();
        const int pieces = tiles * kTilePieces, chosen = min(lds.chosen_n, kLanes), items = chosen * pieces;
        for (int i = tid; i < items; i += kLanes) {
            const int which = lds.chosen[i / pieces], piece = i % pieces, who = which % kLanes;
            const int64_t tile = (int64_t)(which / kLanes) * tiles + piece / kTilePieces;
            const int64_t c = span.first + (tile * kWaves + who / kWave) * kCols + ((piece % kTilePieces) * kWave + who % kWave) * P;
            float v[P];
            unpack(span.load(c, 0.0f), v, T());
#pragma unroll
            for (int e = 0; e < P; ++e) {
                const uint32_t key = order_key(v[e]);
                if (key >= bound && c + e < span.end) {
                    const int at = atomicAdd(&lds.n, 1);
                    if (at < kHeld) lds.best[at] = candidate(key, (int32_t)(c + e));
                }
            }
        }
        __syncthreads();
        all = lds.n > kHeld || lds.chosen_n > kLanes;
    }
    int count = lds.n;
    if (all) {
        Candidates top{lds.held[wave], n};
        for (int64_t first = span.first + (int64_t)wave * kCols; first < span.end; first += (int64_t)kWaves * kCols) {
            float tile = -INFINITY;
#pragma unroll 1
            for (int j = 0; j < kTilePieces; ++j) {
                float v[P];
                unpack(span.load(first + (j * kWave + lane) * P, -INFINITY), v, T());
#pragma unroll
                for (int e = 0; e < P; ++e) tile = fmaxf(tile, v[e]);
            }
            if (top.wants(tile)) top.add(span, first);
        }
        if (top.count < n) top.sort();
        if (lane == 0) lds.counts[wave] = top.count;
        __syncthreads();
        count = 0;
        if (wave == 0)                             // the waves' lists, of kMaxAlternatives each at most, one after the other
            for (int w = 0; w < kWaves; ++w) {
                const int held = lds.counts[w];
                if (lane < held) lds.best[count + lane] = lds.held[w][lane];
                count += held;
            }
    }
    return wave == 0 ? keep_greatest(lds.best, count, n) : 0;
}

// Workgroup by workgroup a row, or a segment of one: with one segment all is done, else logprob_join_kernel goes on.  2,400 x 102,000 fp32
// 176 us (5.6 TB/s), bf16 91; 2,048 x 141,000 fp16 with entropy and the 5 likeliest words 115 us (5.0), 6,007 x 40,009 bf16 with 20
// 122 (3.9): the vector units work in 91 and 92% of the cycles of both; one row of 102,000 bf16 in 25 segments 6.9 us, and 5.5 to join them.
template <class T, bool kEntropy, bool kTop, int kWaves>
__global__ __launch_bounds__(kWaves * kWave) void logprob_kernel(LogprobArgs a) {
    __shared__ std::conditional_t<kTop, TopLds<kWaves>, FoldLds<kWaves * kWave>> lds;
    __shared__ RowPart part[kWaves];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), lane = lane_id();
    const int64_t items = a.rows * a.segments;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t row = item / a.segments;
        const int32_t begin = (int32_t)(item % a.segments) * a.segment_cols;
        const int32_t end = min(a.vocab - begin, a.segment_cols) + begin;
        const Span<T> span{static_cast<const T*>(a.logits) + row * a.stride, begin, end};
        RowSums sums;
        if constexpr (kTop) {
            StretchMost<kWaves> seen{lds, stretch_tiles<T, kWaves>(span)};
            sums = walk_row<T, kEntropy>(span, wave, kWaves, Fold(&lds.folded[wave][0][lane], &lds.folded[wave][1][lane], &lds.most[threadIdx.x]), seen);
        } else {
            sums = walk_row<T, kEntropy>(span, wave, kWaves, Fold(lds), [](float) {});
        }
        float m = sums.m;
        double s = sums.s, u = sums.u;
        join_lanes(m, s, u);
        if (lane == 0) part[wave] = RowPart{s, u, m, 0};
        int count = 0;
        const uint64_t* best = nullptr;
        if constexpr (kTop) {
            count = find_top(span, sums.m, a.top, lds);
            best = lds.best;
        }
        __syncthreads();
        join_parts(part, kWaves, m, s, u);
        if (a.segments == 1) {
            finish_row<T, kWaves * kWave>(a, row, RowStats(m, s, u), best);
        } else {
            if (threadIdx.x == 0) a.parts[item] = RowPart{s, u, m, count};
            if (kTop && wave == 0 && lane < a.top) a.part_top[item * a.top + lane] = lane < count ? best[lane] : 0;
        }
        __syncthreads();                           // (the next row's parts and candidates)
    }
}

// Joins the segments of a row.
template <class T>
__global__ __launch_bounds__(kLogprobWaves * kWave) void logprob_join_kernel(LogprobArgs a) {
    __shared__ uint64_t held[kLogprobWaves][kHeld];
    __shared__ uint64_t best[kHeld];
    __shared__ uint32_t most[kLogprobWaves * kWave];
    __shared__ int found, counts[kLogprobWaves];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), lane = lane_id();
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const RowPart* parts = a.parts + row * a.segments;
        // the first words' logits are on their way meanwhile
        const T* logits = static_cast<const T*>(a.logits) + row * a.stride;
        int64_t begin = 0, end = 0;
        if (!a.words_apart) row_tokens(a.row_ptr, a.n_tokens, row, begin, end);
        const int64_t t = begin + threadIdx.x;
        const int32_t word = t < end ? a.tokens[t] : -1;
        const float logit = word >= 0 && word < a.vocab ? (float)logits[word] : 0.0f;
        // every wave the sums of all segments, of which there are at most as many as lanes
        float m = lane < a.segments ? parts[lane].m : kLowest;
        double s = lane < a.segments ? parts[lane].s : 0.0, u = lane < a.segments ? parts[lane].u : 0.0;
        join_lanes(m, s, u);
        if (a.top) {
            // the segments' lists, a few entries a thread; as in find_top a bound that enough of them reach leaves few to put in order
            constexpr int kThreads = kLogprobWaves * kWave, kMine = kWave * kMaxAlternatives / kThreads;
            const uint64_t* lists = a.part_top + row * a.segments * a.top;
            uint64_t mine[kMine], greatest = 0;
#pragma unroll
            for (int k = 0; k < kMine; ++k) {
                const int i = k * kThreads + (int)threadIdx.x;
                mine[k] = i < a.segments * a.top ? lists[i] : 0;
                greatest = max(greatest, mine[k]);
            }
            most[threadIdx.x] = (uint32_t)(greatest >> 32);
            if (threadIdx.x == 0) found = 0;
            __syncthreads();
            uint32_t group = most[lane];
#pragma unroll
            for (int w = 1; w < kLogprobWaves; ++w) group = max(group, most[w * kWave + lane]);
            const uint32_t bound = max(nth_key(group, a.top), 1u);
#pragma unroll
            for (int k = 0; k < kMine; ++k)
                if ((uint32_t)(mine[k] >> 32) >= bound) {
                    const int at = atomicAdd(&found, 1);
                    if (at < kHeld) best[at] = mine[k];
                }
            __syncthreads();
            int count = found;
            if (count > kHeld) {
                // many equal ones: a wave's share of the lists; full buffers are cut down to the wanted number
                count = 0;
                for (int i = wave; i < a.segments; i += kLogprobWaves) {
                    const int n = min(__builtin_amdgcn_readfirstlane(parts[i].n), a.top);
                    if (count + n > kHeld) count = keep_greatest(held[wave], count, a.top);
                    if (lane < n) held[wave][count + lane] = lists[i * a.top + lane];
                    count += n;
                }
                count = keep_greatest(held[wave], count, a.top);
                if (lane == 0) counts[wave] = count;
                __syncthreads();
                count = 0;
                if (wave == 0)
                    for (int w = 0; w < kLogprobWaves; ++w) {
                        const int n = counts[w];
                        if (lane < n) best[count + lane] = held[w][lane];
                        count += n;
                    }
            }
            if (wave == 0) keep_greatest(best, count, a.top);
            __syncthreads();
        }
        const RowStats st(m, s, u);
        if (t < end) a.logprobs[t] = logprob_of(logit, word, a.vocab, st.m, st.log_s);
        finish_row<T, kLogprobWaves * kWave>(a, row, st, best, kLogprobWaves * kWave);
        __syncthreads();
    }
}

// ---------------------------------------------------------------- gradient
struct LogprobGradArgs {
    const void* logits;
    int64_t stride, rows;
    int32_t vocab;
    const int32_t* tokens;
    const int64_t* row_ptr;
    int64_t n_tokens;
    const float* grad;           // of each word's log-probability
    const float* stats;          // (with kLoss they are found)
    const float* entropy;        // both null: no gradient of the entropy
    const float* grad_entropy;
    float* logprobs;             // kLoss
    void* out;
    int64_t out_stride;
    int32_t segments;
    int32_t segment_cols;
    int32_t slots;               // of the words' table, a power of two, or 0
    int32_t columns;             // of a range, where each column has a sum (a multiple of a piece, or all)
    bool once;                   // logits and gradient are more than the caches hold
};

constexpr int kSlotBytes = 12;

// The words' gradients of a row are summed in LDS, as whole numbers: a unit is so small that n of them of the greatest magnitude stay
// below 2^62, and whole numbers add up to the same in any order.  A word's slot is the next free one from the one that its
// hash says (at most seven of eight are taken); a row of more words has a sum for each column, range by range.
struct WordTable {
    unsigned long long* sums;    // [slots]; a column each: [columns]
    int32_t* words;              // [slots], -1: free
    int32_t slots, shift;

    __device__ __forceinline__ WordTable(unsigned long long* lds, int32_t n)
        : sums(lds), words(reinterpret_cast<int32_t*>(lds + n)), slots(n), shift(__clz(n) + 1) {}

    template <int kThreads>
    __device__ __forceinline__ void clear(int tid) const {
        for (int i = tid; i < slots; i += kThreads) {
            sums[i] = 0;
            words[i] = -1;
        }
    }
    // The slot, if the word is new to the table, else -1.
    __device__ __forceinline__ int add(int32_t word, long long units) const {
        int i = (int)(((uint32_t)word * 0x9E3779B1u) >> shift), was;
        for (;;) {
            was = atomicCAS(&words[i], -1, word);
            if (was == -1 || was == word) break;
            i = (i + 1) & (slots - 1);
        }
        atomicAdd(&sums[i], (unsigned long long)units);
        return was == -1 ? i : -1;
    }
};

// What a row's gradient needs besides its logits.
struct RowGrad {
    float m, log_s, inv_s;       // of the row
    float total, h, entropy;     // G, gradient of the entropy, entropy
    // of one logit, without its own words' gradients
    template <class T, bool kEntropy>
    __device__ __forceinline__ float of(float x) const {
        const float d = below<T>(x, m), p = exp_of<T>(d) * inv_s;
        if constexpr (kEntropy) return -p * (total + h * (fmaxf(d, kVanished) - log_s + entropy));
        return -p * total;
    }
};

// The gradient of a span's columns; own(values, first column) adds what a column's own words give.  `once`: neither the logits (kLoss:
// they have been read before) nor the gradient are kept in the caches.
template <class T, int kThreads, bool kLoss, bool kEntropy, class Own>
__device__ __forceinline__ void stream_grad(const T* row, T* out, int32_t begin, int32_t end, const RowGrad& g, bool once, Own&& own) {
    // a column's place is its number plus `shift`: all pieces but the first and the last lie at 16-byte boundaries, wherever rows begin
    // (6,007 x 40,009 bf16, one word a row: at the row's own 202 us, so 190)
    constexpr int P = kPack<T>;
    const int shift = (int)(reinterpret_cast<uintptr_t>(row) / sizeof(T) % P);
    const int64_t lo = (int64_t)begin + shift, hi = (int64_t)end + shift;
    for (int64_t c = begin + (int64_t)threadIdx.x * P; c < hi; c += kThreads * P) {
        float v[P];
        unpack(load_piece(row - shift, c, lo, hi, -INFINITY, kLoss && once), v, T());
#pragma unroll
        for (int e = 0; e < P; ++e) v[e] = g.template of<T, kEntropy>(v[e]);
        own(v, (int32_t)(c - shift));
        store_piece(out - shift, c, lo, hi, pack(v, T()), once);
    }
}

// Rows, or segments of rows.  kLoss: the statistics and the words' log-probabilities are found first, by the same workgroup
// (one segment); the row is read twice then, and the last cache gives it no faster than memory does.  1,024 x 102,000 bf16, 330 words a
// row: 72 us for the gradient alone (5.8 TB/s), 109 with the loss; 8,000 x 12,000 fp32, one word a row, 143 and 151.  Table: a word's
// slot costs 12 bytes of LDS, against 8 bytes a column.  kSingle: one word to a row.  The logits' rows may be the gradient's.
template <class T, int kThreads, bool kLoss, bool kEntropy, bool kSingle>
__global__ __launch_bounds__(kThreads) void logprob_grad_kernel(LogprobGradArgs a) {
    constexpr int P = kPack<T>, kWaves = kThreads / kWave;
    extern __shared__ unsigned long long table_lds[];
    __shared__ RowPart part[kWaves];
    __shared__ double totals[kWaves];
    __shared__ float largest[kWaves];
    __shared__ std::conditional_t<kLoss, FoldLds<kThreads>, int> folded;
    const int tid = (int)threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave), lane = lane_id();
    const int64_t items = a.rows * a.segments;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t row = item / a.segments;
        const int32_t begin = (int32_t)(item % a.segments) * a.segment_cols;
        const int32_t end = min(a.vocab - begin, a.segment_cols) + begin;
        const T* logits = static_cast<const T*>(a.logits) + row * a.stride;
        T* out = static_cast<T*>(a.out) + row * a.out_stride;
        int64_t t0, t1;
        row_tokens(a.row_ptr, a.n_tokens, row, t0, t1);
        RowGrad g;
        g.h = kEntropy ? a.grad_entropy[row] : 0.0f;
        g.entropy = kEntropy ? a.entropy[row] : 0.0f;
        // the row's total and the greatest magnitude of its words' gradients; of a document that is no longer than the workgroup has
        // room for, words, gradients and logits stay in registers
        const int64_t n = t1 - t0;
        const bool brief = !kSingle && n <= min(kThreads * kWordBatch, a.slots / 8 * 7);
        int32_t words[kWordBatch];
        float owns[kWordBatch], xs[kWordBatch];
        double total = 0.0;
        float most = 0.0f;
        int32_t word = -1;
        if (kSingle) {
            word = a.tokens[row];
            if (word >= 0 && word < a.vocab) {
                total = (double)a.grad[row];
                most = fabsf(a.grad[row]);
            }
        } else {
            if (brief) {
#pragma unroll
                for (int k = 0; k < kWordBatch; ++k) {
                    const int64_t t = t0 + k * kThreads + tid;
                    words[k] = t < t1 ? a.tokens[t] : -1;
                }
                WordTable(table_lds, a.slots).template clear<kThreads>(tid);
#pragma unroll
                for (int k = 0; k < kWordBatch; ++k) {
                    const bool known = words[k] >= 0 && words[k] < a.vocab;
                    owns[k] = known ? a.grad[t0 + k * kThreads + tid] : 0.0f;
                    xs[k] = known ? (float)logits[words[k]] : 0.0f;
                    total += (double)owns[k];
                    most = fmaxf(most, fabsf(owns[k]));
                }
            } else {
                for_words<kThreads>(a.tokens, t0, t1, tid, [&](const int64_t (&t)[kWordBatch], const int32_t (&w)[kWordBatch], const bool (&)[kWordBatch]) {
                    float own[kWordBatch];
#pragma unroll
                    for (int k = 0; k < kWordBatch; ++k) own[k] = w[k] >= 0 && w[k] < a.vocab ? a.grad[t[k]] : 0.0f;
#pragma unroll
                    for (int k = 0; k < kWordBatch; ++k) {
                        total += (double)own[k];
                        most = fmaxf(most, fabsf(own[k]));
                    }
                });
            }
            total = wave_sum(total);
            most = wave_max(most);
            if (lane == 0) {
                totals[wave] = total;
                largest[wave] = most;
            }
        }
        const bool walked = kLoss && n > 0;        // (a row without words: nothing to read it for)
        float m = -INFINITY;
        double s = 0.0, u = 0.0;
        if constexpr (kLoss) {
            if (walked) {
                const RowSums sums = walk_row<T, false>(Span<T>{logits, begin, end}, wave, kWaves, Fold(folded), [](float) {});
                m = sums.m;
                s = sums.s;
                join_lanes(m, s, u);
                if (lane == 0) part[wave] = RowPart{s, u, m, 0};
            }
        }
        if (kLoss || !kSingle) __syncthreads();
        if (!kSingle) {
            total = 0.0;
            most = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                total += totals[w];
                most = fmaxf(most, largest[w]);
            }
        }
        if (kLoss) {
            if (walked && kWaves > 1) join_parts(part, kWaves, m, s, u);
            const RowStats st(m, s, u);
            g.m = st.m;
            g.log_s = st.log_s;
            g.inv_s = (float)(1.0 / s);
            if (kSingle) {
                if (tid == 0) a.logprobs[row] = word_logprob(logits, word, a.vocab, g.m, g.log_s);
            } else if (brief) {
#pragma unroll
                for (int k = 0; k < kWordBatch; ++k) {
                    const int64_t t = t0 + k * kThreads + tid;
                    if (t < t1) a.logprobs[t] = logprob_of(xs[k], words[k], a.vocab, g.m, g.log_s);
                }
            } else {
                word_logprobs<T, kThreads>(logits, a.tokens, t0, t1, tid, a.vocab, g.m, g.log_s, a.logprobs);
            }
            clear_rest<kThreads>(a.row_ptr, a.rows, a.n_tokens, row, a.logprobs);
        } else {
            g.m = a.stats[2 * row];
            g.log_s = a.stats[2 * row + 1];
            g.inv_s = (float)exp(-(double)g.log_s);
        }
        g.total = (float)total;
        const bool finite = most < INFINITY && total == total;
        if (!finite) g.total = __uint_as_float(0x7fc00000u);       // the whole row's gradient is NaN
        if (g.m == -INFINITY || (most == 0.0f && total == 0.0 && g.h == 0.0f)) {
            // nothing is allowed, or nothing is wanted: zeros
            if (kLoss) __syncthreads();                            // (logits read above may be written here)
            for (int64_t c = begin + (int64_t)tid * P; c < end; c += kThreads * P) store_some(out + c, Raw{0, 0, 0, 0}, (int)min((int64_t)P, end - c));
        } else if (kSingle) {
            if (kLoss) __syncthreads();
            stream_grad<T, kThreads, kLoss, kEntropy>(logits, out, begin, end, g, a.once, [&](float (&v)[P], int32_t c) {
                if (word >= 0 && word < a.vocab && (uint32_t)(word - c) < (uint32_t)P) {
#pragma unroll
                    for (int e = 0; e < P; ++e) v[e] += c + e == word ? (float)total : 0.0f;
                }
            });
        } else {
            const WordTable table(table_lds, a.slots);
            const int unit = 62 - (n > 1 ? 64 - __clzll(n - 1) : 0) - (finite && most > 0.0f ? ilogbf(most) + 1 : 0);
            const double units = ldexp(1.0, unit), per_unit = ldexp(1.0, -unit);
            auto value = [&](unsigned long long sum) { return (float)((double)(long long)sum * per_unit); };
            // put(word, units) for the words of the columns [first, last)
            auto each = [&](int32_t first, int32_t last, auto&& put) {
                if (!finite) return;
                for_words<kThreads>(a.tokens, t0, t1, tid, [&](const int64_t (&t)[kWordBatch], const int32_t (&w)[kWordBatch], const bool (&)[kWordBatch]) {
                    float own[kWordBatch];
#pragma unroll
                    for (int k = 0; k < kWordBatch; ++k) own[k] = w[k] >= first && w[k] < last ? a.grad[t[k]] : 0.0f;
#pragma unroll
                    for (int k = 0; k < kWordBatch; ++k)
                        if (w[k] >= first && w[k] < last) put(w[k], (long long)rint((double)own[k] * units));
                });
            };
            if (brief) {
                // the thread that brings a word first works out its column, and writes it last
                int slot[kWordBatch];
#pragma unroll
                for (int k = 0; k < kWordBatch; ++k)
                    slot[k] = finite && words[k] >= begin && words[k] < end ? table.add(words[k], (long long)rint((double)owns[k] * units)) : -1;
                __syncthreads();
#pragma unroll
                for (int k = 0; k < kWordBatch; ++k)
                    if (slot[k] >= 0) xs[k] = value(table.sums[slot[k]]) + g.template of<T, kEntropy>(xs[k]);
                stream_grad<T, kThreads, kLoss, kEntropy>(logits, out, begin, end, g, a.once, [](float (&)[P], int32_t) {});
                __syncthreads();
#pragma unroll
                for (int k = 0; k < kWordBatch; ++k)
                    if (slot[k] >= 0) out[words[k]] = (T)xs[k];
            } else if (n <= table.slots / 8 * 7) {
                table.template clear<kThreads>(tid);
                __syncthreads();
                each(begin, end, [&](int32_t w, long long v) { table.add(w, v); });
                __syncthreads();
                // the words' columns are worked out before the row is written over, and written last
                for (int i = tid; i < table.slots; i += kThreads) {
                    const int32_t w = table.words[i];
                    if (w >= 0) table.sums[i] = (unsigned long long)__float_as_uint(value(table.sums[i]) + g.template of<T, kEntropy>((float)logits[w]));
                }
                __syncthreads();
                stream_grad<T, kThreads, kLoss, kEntropy>(logits, out, begin, end, g, a.once, [](float (&)[P], int32_t) {});
                __syncthreads();
                for (int i = tid; i < table.slots; i += kThreads)
                    if (table.words[i] >= 0) out[table.words[i]] = (T)__uint_as_float((uint32_t)table.sums[i]);
            } else {
                for (int32_t first = begin; first < end; first += a.columns) {
                    const int32_t last = min(end - first, a.columns) + first;
                    for (int i = tid; i < last - first; i += kThreads) table.sums[i] = 0;
                    __syncthreads();
                    each(first, last, [&](int32_t w, long long v) { atomicAdd(&table.sums[w - first], (unsigned long long)v); });
                    __syncthreads();
                    stream_grad<T, kThreads, kLoss, kEntropy>(logits, out, first, last, g, a.once, [&](float (&v)[P], int32_t c) {
#pragma unroll
                        for (int e = 0; e < P; ++e)
                            if (c + e >= first && c + e < last) v[e] += value(table.sums[c + e - first]);
                    });
                    __syncthreads();
                }
            }
        }
        __syncthreads();
    }
}

}  // namespace mlda
