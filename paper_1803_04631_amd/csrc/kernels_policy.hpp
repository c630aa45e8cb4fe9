// The clipped policy loss with a KL term, and its gradient with respect to the words' log-probabilities.
//
// With l a word's log-probability, o the one it was drawn with, f that of a reference model, A its advantage, w its weight and d = l - o:
//   the word is clipped where A > 0 and d > ln(1 + high), or A < 0 and d < ln(1 - low)
//   loss = sum of w (kl (exp(f - l) - (f - l) - 1) - A (its bound, 1 + high or 1 - low, where clipped, else exp(d)))
//   grad = w (kl (1 - exp(f - l)) - A (0 where clipped, else exp(d)))
// A word of weight 0 is none: nothing of it counts, whatever its numbers are.  One whose advantage is 0 has no policy part, however large its ratio is.
//
// All of it is in fp64 and rounded once: the border is then the same for every way of computing it, sums of millions of words keep their bits, and a ratio that fp32
// cannot hold does no harm under a weight that makes it small again.  Exponentials are a series, within 2^-40 of themselves, and the KL term, a difference of nearly
// equal numbers, within 2^-36.  (With fp32's exponentials, which end at exp(88.7), it takes as long: 26,154 documents of 113 words with a KL term 26.7 us, so 26.5; 50e6 words 190 and 191,
// with a KL term 242 and 233.)  Many words are bound by memory: 50e6 words, 20 bytes each, 5.2 TB/s (one word to a thread at a time 277 us).  In between it is instructions: 26,154
// documents with a KL term take 220 for each word, 50 of them for its row, which keep the vector units busy for 71% of the time.  Few words are one workgroup's and one launch; more
// leave partial sums, which a second launch joins in a fixed order.
#pragma once
#include "vec_io.hpp"

namespace mlda {

constexpr int kPolicyGroups = 4096;      // of a launch at most, each of which leaves three sums

struct PolicyArgs {
    const float* logprobs;
    const float* old;
    const float* reference;              // null: none
    const float* advantages;             // a word's, or with row_ptr a row's
    const float* weights;                // null: 1 / n each
    const int64_t* row_ptr;              // null: none
    int64_t rows, n;
    double low, high;                    // ln(1 - low), ln(1 + high)
    double at_low, at_high;              // 1 - low, 1 + high
    double kl, weight;
    float* grad;
    float* sums;                         // loss, KL term, clipped weight; null: partial sums
    double* partial;
    bool once;
};

// The rows of two words, by a wave: the last that begins at or before each.  64 bounds are looked at at a time.
__device__ __forceinline__ void rows_of_wave(const int64_t* row_ptr, int64_t rows, int64_t first, int64_t last, int64_t& lo, int64_t& hi) {
    int64_t a0 = 0, a1 = rows, b0 = 0, b1 = rows;
    while (a1 - a0 > 1 || b1 - b0 > 1) {
        const int64_t a_step = (a1 - a0 + kWave - 1) / kWave, b_step = (b1 - b0 + kWave - 1) / kWave;
        const int64_t a = a0 + lane_id() * a_step, b = b0 + lane_id() * b_step;
        const int64_t at_a = row_ptr[min(a, rows)], at_b = row_ptr[min(b, rows)];
        const int a_n = max(__popcll(__ballot(a < a1 && at_a <= first)), 1), b_n = max(__popcll(__ballot(b < b1 && at_b <= last)), 1);
        a0 += (a_n - 1) * a_step;
        a1 = min(a1, a0 + a_step);
        b0 += (b_n - 1) * b_step;
        b1 = min(b1, b0 + b_step);
    }
    lo = a0;
    hi = max(a0, b0);
}

// exp(x) of any x in fp64 as 2^k (1 + r + far), k whole and |r| <= ln 2 / 2.  The series of exp(r) ends with r^10 / 10!: what is left out is below 2^-42 of exp(r), and so is what
// the terms from r^6 on lose in fp32; of `far`, exp(r) - 1 - r, both are below 2^-37.  Up to ln 2 / 2 k is 0, and `far` there exp(x) - 1 - x, whose difference would lose bits.
struct Exp {
    double value, far, most;                               // most: x, or about 720 where x is more: exp(x) is infinite there
    bool near;
};
__device__ __forceinline__ Exp exp_of(double x) {
    // Limits, 720 and -800 (exp(x) is 0 there), by the upper words, whose order is that of numbers of one sign (comparisons of fp64 numbers: 50e6 words 283 us with rows, so 277).
    const uint64_t bits = __builtin_bit_cast(uint64_t, x);
    const uint32_t most = (uint32_t)min((int32_t)(bits >> 32), 0x40868000), within = x == x ? min(most, 0xc0890000u) : 0x7ff80000u;
    const double c = __builtin_bit_cast(double, (uint64_t)within << 32 | (uint32_t)bits);
    // 1.5 x 2^52 more, and a number is whole, with itself in the lower bits
    const double whole = __builtin_fma(c, 1.4426950408889634, 6755399441055744.0), k = whole - 6755399441055744.0, r = __builtin_fma(-k, 0.6931471805599453, c);
    const float q = (float)r;
    float h = __builtin_fmaf(q, 1.0f / 3628800.0f, 1.0f / 362880.0f);
    h = __builtin_fmaf(q, h, 1.0f / 40320.0f);
    h = __builtin_fmaf(q, h, 1.0f / 5040.0f);
    h = __builtin_fmaf(q, h, 1.0f / 720.0f);
    double s = __builtin_fma(r, (double)h, 1.0 / 120.0);
    s = __builtin_fma(r, s, 1.0 / 24.0);
    s = __builtin_fma(r, s, 1.0 / 6.0);
    s = __builtin_fma(r, s, 0.5);
    const double e = __builtin_fma(r, __builtin_fma(r, s, 1.0), 1.0);
    return {__builtin_amdgcn_ldexp(e, (int)(uint32_t)__builtin_bit_cast(uint64_t, whole)), r * r * s,
            __builtin_bit_cast(double, (uint64_t)most << 32 | (uint32_t)bits), k == 0.0};
}

// kPolicyEach: neighbouring words of a thread.  A word is a long chain of instructions: those of a single workgroup have a thread each if they can (405 of them with
// a KL term 4.6 us by four, 2.9 apart).
template <int kThreads, int kPolicyEach, bool kReference>
__global__ __launch_bounds__(kThreads) void policy_kernel(PolicyArgs a) {
    constexpr int kChunk = kThreads * kPolicyEach;
    __shared__ double slots[3][kThreads / kWave];
    double loss = 0.0, kl = 0.0, clipped = 0.0;
    const int64_t chunks = (a.n + kChunk - 1) / kChunk;
    const int64_t begin = chunks * blockIdx.x / gridDim.x, end = chunks * (blockIdx.x + 1) / gridDim.x;
    for (int64_t chunk = begin; chunk < end; ++chunk) {
        const int64_t i = chunk * kChunk + threadIdx.x * kPolicyEach;
        const int64_t wave_first = chunk * kChunk + (int)threadIdx.x / kWave * kWave * kPolicyEach;
        if (wave_first >= a.n) break;
        auto load = [&](const float* p, float (&v)[kPolicyEach]) {
            if constexpr (kPolicyEach == 4) unpack(load_piece(p, i, 0, a.n, 0.0f, a.once), v, float());
            else v[0] = i < a.n ? p[i] : 0.0f;
        };
        float l[kPolicyEach], old[kPolicyEach], ref[kPolicyEach], w32[kPolicyEach], adv[kPolicyEach];
        bool used[kPolicyEach];
        load(a.logprobs, l);
        load(a.old, old);
        if (kReference) load(a.reference, ref);
        if (a.weights) load(a.weights, w32);
        if (a.row_ptr) {
            const int64_t first = a.rows ? a.row_ptr[0] : 0, last = a.rows ? a.row_ptr[a.rows] : 0;
            int64_t lo = 0, hi = 0;
            if (a.rows) rows_of_wave(a.row_ptr, a.rows, wave_first, min(wave_first + kWave * kPolicyEach, a.n) - 1, lo, hi);
#pragma unroll
            for (int e = 0; e < kPolicyEach; ++e) used[e] = i + e >= first && i + e < last;
            if (hi - lo < kWave) {
                // a lane has the end and the advantage of a row, and every word meets all of them
                const int64_t mine = lo + min((int64_t)lane_id(), hi - lo);
                const int64_t ends = a.rows ? a.row_ptr[mine + 1] : 0;
                const float advantages = a.rows ? a.advantages[mine] : 0.0f;
                const float at_first = read_lane(advantages, 0);
#pragma unroll
                for (int e = 0; e < kPolicyEach; ++e) adv[e] = at_first;
                const int more = __builtin_amdgcn_readfirstlane((int)(hi - lo));
                for (int k = 0; k < more; ++k) {
                    const int64_t bound = (int64_t)(uint32_t)read_lane((int)ends, k) | (int64_t)read_lane((int)(ends >> 32), k) << 32;
                    const float next = read_lane(advantages, k + 1);
#pragma unroll
                    for (int e = 0; e < kPolicyEach; ++e) adv[e] = i + e >= bound ? next : adv[e];
                }
            } else {
#pragma unroll
                for (int e = 0; e < kPolicyEach; ++e) {
                    int64_t most = hi;
                    while (lo < most) {
                        const int64_t mid = (lo + most + 1) >> 1;
                        if (a.row_ptr[mid] <= i + e) lo = mid;
                        else most = mid - 1;
                    }
                    adv[e] = a.advantages[lo];
                }
            }
        } else {
            load(a.advantages, adv);
#pragma unroll
            for (int e = 0; e < kPolicyEach; ++e) used[e] = i + e < a.n;
        }
        float grads[kPolicyEach];
#pragma unroll
        for (int e = 0; e < kPolicyEach; ++e) {
            // (without branches, so that the words' chains of instructions go side by side)
            const double w = a.weights ? (double)w32[e] : a.weight;
            const bool counts = used[e] && w != 0.0;
            const double d = (double)l[e] - (double)old[e], advantage = adv[e];
            const bool over = advantage > 0.0 && d > a.high, under = advantage < 0.0 && d < a.low;
            const double ratio = exp_of(d).value;
            // (an advantage of 0 makes 0 of an infinite ratio too, not NaN: the word tells nothing)
            const double gain = advantage == 0.0 && ratio == INFINITY ? 0.0 : ratio * advantage;
            double term = over ? -a.at_high * advantage : under ? -a.at_low * advantage : -gain;
            double grad = over || under ? 0.0 : -gain;
            clipped += counts && (over || under) ? w : 0.0;
            if (kReference) {
                const double x = (double)ref[e] - (double)l[e];
                const Exp f = exp_of(x);
                const double more = f.near ? x + f.far : f.value - 1.0;    // exp(x) - 1
                const double part = f.near ? f.far : more - f.most;
                kl += counts ? w * part : 0.0;
                if (a.kl != 0.0) {                                         // (only watched, it is no part of them, infinite or NaN)
                    term += a.kl * part;
                    grad -= a.kl * more;
                }
            }
            loss += counts ? w * term : 0.0;
            grad = counts ? w * grad : 0.0;
            grads[e] = (float)grad;
        }
        if constexpr (kPolicyEach == 4) store_piece(a.grad, i, 0, a.n, pack(grads, float()), a.once);
        else if (i < a.n) a.grad[i] = grads[0];
    }
    loss = wave_sum(loss);
    kl = wave_sum(kl);
    clipped = wave_sum(clipped);
    if (lane_id() == 0) {
        slots[0][threadIdx.x / kWave] = loss;
        slots[1][threadIdx.x / kWave] = kl;
        slots[2][threadIdx.x / kWave] = clipped;
    }
    __syncthreads();
    const int k = threadIdx.x / kWave;
    if (k < 3) {
        const double sum = wave_sum(lane_id() < kThreads / kWave ? slots[k][lane_id()] : 0.0);
        if (lane_id() > 0) return;
        if (a.sums) a.sums[k] = (float)sum;
        else a.partial[k * kPolicyGroups + blockIdx.x] = sum;
    }
}

constexpr int kPolicySumThreads = 1024;

// A workgroup for each sum.
__global__ __launch_bounds__(kPolicySumThreads) void policy_sums_kernel(const double* partial, int32_t groups, float* sums) {
    constexpr int kEach = kPolicyGroups / kPolicySumThreads;
    __shared__ double slots[kPolicySumThreads / kWave];
    const double* const mine = partial + blockIdx.x * kPolicyGroups;
    double part[kEach], v = 0.0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) part[i] = mine[min(i * kPolicySumThreads + (int)threadIdx.x, groups - 1)];
#pragma unroll
    for (int i = 0; i < kEach; ++i) v += i * kPolicySumThreads + (int)threadIdx.x < groups ? part[i] : 0.0;
    v = wave_sum(v);
    if (lane_id() == 0) slots[threadIdx.x / kWave] = v;
    __syncthreads();
    if (threadIdx.x >= kWave) return;
    v = wave_sum(lane_id() < kPolicySumThreads / kWave ? slots[lane_id()] : 0.0);
    if (lane_id() == 0) sums[blockIdx.x] = (float)v;
}

}  // namespace mlda
