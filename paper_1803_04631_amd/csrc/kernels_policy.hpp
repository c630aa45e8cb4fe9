// The clipped policy loss with a KL term, and its gradient with respect to the words' log-probabilities.
//
// With l a word's log-probability, o the one it was drawn with, f that of a reference model, A its advantage, w its weight and d = l - o:
//   the word is clipped where A > 0 and d > ln(1 + high), or A < 0 and d < ln(1 - low)
//   loss = sum of w (kl (exp(f - l) - (f - l) - 1) - A (its bound, 1 + high or 1 - low, where clipped, else exp(d)))
//   grad = w (kl (1 - exp(f - l)) - A (0 where clipped, else exp(d)))
// A word of weight 0 is none: nothing of it counts, whatever its numbers are.
//
// Everything is in fp64: the border is then the same for every way of computing it, the KL term, a difference of nearly equal numbers, keeps
// its bits, and sums of millions of words theirs.
#pragma once
#include "vec_io.hpp"

namespace mlda {

constexpr int kPolicyThreads = 256;
constexpr int kPolicyGroups = 1024;      // of a launch at most, each of which leaves three sums

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
};

// The row of a word: the last that begins at or before it.  -1: none.
__device__ __forceinline__ int64_t row_of(const PolicyArgs& a, int64_t word) {
    if (a.rows == 0 || word < a.row_ptr[0] || word >= a.row_ptr[a.rows]) return -1;
    int64_t lo = 0, hi = a.rows - 1;
    while (lo < hi) {
        const int64_t mid = (lo + hi + 1) >> 1;
        if (a.row_ptr[mid] <= word) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

template <bool kReference>
__global__ __launch_bounds__(kPolicyThreads) void policy_kernel(PolicyArgs a) {
    __shared__ double slots[3][kPolicyThreads / kWave];
    double loss = 0.0, kl = 0.0, clipped = 0.0;
    for (int64_t i = (int64_t)blockIdx.x * kPolicyThreads + threadIdx.x; i < a.n; i += (int64_t)gridDim.x * kPolicyThreads) {
        int64_t at = i;
        if (a.row_ptr) at = row_of(a, i);
        const double w = a.weights ? (double)a.weights[i] : a.weight;
        double grad = 0.0;
        if (at >= 0 && w != 0.0) {
            const double l = a.logprobs[i], d = l - (double)a.old[i], advantage = a.advantages[at];
            const bool over = advantage > 0.0 && d > a.high, under = advantage < 0.0 && d < a.low;
            const double ratio = exp(d);
            double term = -(over ? a.at_high : under ? a.at_low : ratio) * advantage;
            grad = over || under ? 0.0 : -ratio * advantage;
            if (over || under) clipped += w;
            if (kReference) {
                const double e = (double)a.reference[i] - l, more = expm1(e);
                kl += w * (more - e);
                term += a.kl * (more - e);
                grad -= a.kl * more;
            }
            loss += w * term;
            grad *= w;
        }
        a.grad[i] = (float)grad;
    }
    loss = group_sum<kPolicyThreads>(loss, slots[0]);
    kl = group_sum<kPolicyThreads>(kl, slots[1]);
    clipped = group_sum<kPolicyThreads>(clipped, slots[2]);
    if (threadIdx.x == 0) {
        const double all[3] = {loss, kl, clipped};
        for (int k = 0; k < 3; ++k) {
            if (a.sums) a.sums[k] = (float)all[k];
            else a.partial[3 * blockIdx.x + k] = all[k];
        }
    }
}

__global__ __launch_bounds__(kPolicyThreads) void policy_sums_kernel(const double* partial, int32_t groups, float* sums) {
    __shared__ double slots[3][kPolicyThreads / kWave];
    for (int k = 0; k < 3; ++k) {
        double sum = 0.0;
        for (int i = (int)threadIdx.x; i < groups; i += kPolicyThreads) sum += partial[3 * i + k];
        sum = group_sum<kPolicyThreads>(sum, slots[k]);
        if (threadIdx.x == 0) sums[k] = (float)sum;
    }
}

}  // namespace mlda
