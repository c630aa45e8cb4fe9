// The clipped policy loss with a KL term, and its gradient with respect to the words' log-probabilities.
//
// With l a word's log-probability, o the one it was drawn with, f that of a reference model, A its advantage, w its weight and d = l - o:
//   the word is clipped where A > 0 and d > ln(1 + high), or A < 0 and d < ln(1 - low)
//   loss = sum of w (kl (exp(f - l) - (f - l) - 1) - A (its bound, 1 + high or 1 - low, where clipped, else exp(d)))
//   grad = w (kl (1 - exp(f - l)) - A (0 where clipped, else exp(d)))
// A word of weight 0 is none: nothing of it counts, whatever its numbers are.
//
// Differences, products and sums are in fp64: the border is then the same for every way of computing it, and sums of millions of words keep their bits.
// The exponentials are fp32's, corrected for what the difference has beyond fp32: within 3 units of roundoff (2^-24); the KL term, a difference of nearly equal
// numbers, is a series near 0: within 12.  (In fp64 they bound the kernel: 26,154 documents of 113 words with a KL term 28.5 us, so 26.)  Bound by memory: 50e6
// words, 20 bytes each, 197 us (one word to a thread at a time 277).  Few words are one workgroup's and one launch; more leave partial sums, which a second launch
// joins in a fixed order.
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

// exp(d), for a d of more bits than fp32 has.
__device__ __forceinline__ float exp_of(double d) {
    const float high = (float)d, e = expf(high);
    // (an infinite difference has no remainder, and an infinite exponential nothing to correct)
    return e < INFINITY && high > -200.0f ? __builtin_fmaf(e, (float)(d - (double)high), e) : e;
}

// exp(x) - x - 1 up to 1, where the difference would lose bits: ten terms of x^2 / 2 + x^3 / 6 + ..; what is left out is below 2^-27 of it.
__device__ __forceinline__ float kl_near(float x) {
    float s = __builtin_fmaf(x, 1.0f / 39916800.0f, 1.0f / 3628800.0f);
    s = __builtin_fmaf(x, s, 1.0f / 362880.0f);
    s = __builtin_fmaf(x, s, 1.0f / 40320.0f);
    s = __builtin_fmaf(x, s, 1.0f / 5040.0f);
    s = __builtin_fmaf(x, s, 1.0f / 720.0f);
    s = __builtin_fmaf(x, s, 1.0f / 120.0f);
    s = __builtin_fmaf(x, s, 1.0f / 24.0f);
    s = __builtin_fmaf(x, s, 1.0f / 6.0f);
    s = __builtin_fmaf(x, s, 0.5f);
    return x * x * s;
}

// kPolicyEach: neighbouring words of a thread.  A word is a long chain of instructions: those of a single workgroup have a thread each if they can (330 of them, in fp64
// with a KL term, 4.9 us by four, 2.8 apart).
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
            const double ratio = exp_of(d);
            double term = -(over ? a.at_high : under ? a.at_low : ratio) * advantage;
            double grad = over || under ? 0.0 : -ratio * advantage;
            clipped += counts && (over || under) ? w : 0.0;
            if (kReference) {
                const double x = (double)ref[e] - (double)l[e], near = kl_near((float)x), much = (double)exp_of(x) - 1.0;
                const bool is_near = fabs(x) < 1.0;
                const double part = is_near ? near : much < INFINITY ? much - x : much;     // (infinity also where both are)
                kl += counts ? w * part : 0.0;
                term += a.kl * part;
                grad -= a.kl * (is_near ? x + near : much);
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
