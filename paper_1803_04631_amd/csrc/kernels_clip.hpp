// The norm over all tensors of a gradient, and the tensors scaled down to a greatest norm.
//
//   norm = sqrt(sum over all tensors of g^2),   g' = g most / norm  where norm > most, else g
//
// Bound by memory: a read of everything, and, where it is scaled, another read and a write.  The tensors are taken as one long
// line of units of kClipUnit elements (a tensor's last unit may be short), cut into equal runs, one for
// each workgroup, whatever tensors it crosses.  Squares are summed in fp64: no gradient that fp32 holds overflows it,
// and the order is fixed: by thread, by workgroup, then over the workgroups.  The scaling goes over each run
// from its end to its start, where what was read last is still in the caches, and keeps what it reads and writes out of them:
// 142e6 fp32 elements 281 us, without the latter 318 (98 us of it the first read, 5.8 TB/s).
#pragma once
#include "vec_io.hpp"

namespace mlda {

constexpr int kClipThreads = 256;
constexpr int kClipUnit = 8192;              // elements
constexpr int kClipTensors = 120;            // of one launch: their table is a kernel argument
constexpr int kClipGroups = 1024;            // workgroups of one launch at most: four to a CU (142e6 bf16 elements read in 47 us, with twice as many of half the unit 54)

struct ClipTensor {
    const void* in;
    void* out;
    int64_t n;
};

struct ClipArgs {
    ClipTensor tensor[kClipTensors];
    uint32_t first_unit[kClipTensors + 1];   // of each tensor; the last entry is the number of units
    uint8_t type[kClipTensors];
    int32_t tensors;
    double* partial;                         // where the sums of squares go, one of each workgroup (launch after launch, without gaps)
};

// f(type tag, tensor's number, unit) for the units of this workgroup's run, first to last or last to first.
template <bool kBackwards, class F>
__device__ __forceinline__ void for_units(const ClipArgs& a, F&& f) {
    const uint64_t units = a.first_unit[a.tensors];
    const uint32_t begin = (uint32_t)(units * blockIdx.x / gridDim.x), end = (uint32_t)(units * (blockIdx.x + 1) / gridDim.x);
    if (begin == end) return;
    const uint32_t at = kBackwards ? end - 1 : begin;
    int lo = 0, hi = a.tensors - 1;          // the last tensor that begins at or before `at` (empty ones have no unit)
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (a.first_unit[mid] <= at) lo = mid;
        else hi = mid - 1;
    }
    auto unit = [&](uint32_t u) {
        const int type = a.type[lo];
        if (type == 0) f(float(), lo, u - a.first_unit[lo]);
        else if (type == 1) f(Bf16(), lo, u - a.first_unit[lo]);
        else f(Fp16(), lo, u - a.first_unit[lo]);
    };
    if (kBackwards) {
        for (uint32_t u = end; u-- > begin;) {
            while (a.first_unit[lo] > u) --lo;
            unit(u);
        }
    } else {
        for (uint32_t u = begin; u < end; ++u) {
            while (a.first_unit[lo + 1] <= u) ++lo;
            unit(u);
        }
    }
}

// Sum over the workgroup; every thread gets it.
__device__ __forceinline__ double clip_group_sum(double v, double* slots) {
    v = wave_sum(v);
    if (lane_id() == 0) slots[threadIdx.x / kWave] = v;
    __syncthreads();
    return (slots[0] + slots[1]) + (slots[2] + slots[3]);
}

__global__ __launch_bounds__(kClipThreads) void square_sums_kernel(ClipArgs a) {
    __shared__ double slots[kClipThreads / kWave];
    double sum = 0.0;
    for_units<false>(a, [&](auto tag, int i, uint32_t unit) {
        typedef decltype(tag) T;
        constexpr int P = kPack<T>;
        const T* in = static_cast<const T*>(a.tensor[i].in) + (int64_t)unit * kClipUnit;
        const int n = (int)min((int64_t)kClipUnit, a.tensor[i].n - (int64_t)unit * kClipUnit);
        auto take = [&](Raw r) {
            float v[P];
            unpack(r, v, T());
#pragma unroll
            for (int e = 0; e < P; ++e) sum = __builtin_fma((double)v[e], (double)v[e], sum);
        };
        if (n == kClipUnit) {
            Raw r[kClipUnit / (kClipThreads * P)];
#pragma unroll
            for (int j = 0; j < kClipUnit / (kClipThreads * P); ++j) r[j] = load_raw(in + (j * kClipThreads + (int)threadIdx.x) * P);
#pragma unroll
            for (int j = 0; j < kClipUnit / (kClipThreads * P); ++j) take(r[j]);
        } else {
            for (int c = (int)threadIdx.x * P; c < n; c += kClipThreads * P) take(load_some(in + c, min(P, n - c), 0.0f, c));
        }
    });
    sum = clip_group_sum(sum, slots);
    if (threadIdx.x == 0) a.partial[blockIdx.x] = sum;
}

// The norm out of all workgroups' sums, by every thread of a workgroup in the same order.
__device__ __forceinline__ double norm_of(const double* partial, int32_t partials, double* slots) {
    double sum = 0.0;
    for (int i = (int)threadIdx.x; i < partials; i += kClipThreads) sum += partial[i];
    return sqrt(clip_group_sum(sum, slots));
}

__global__ __launch_bounds__(kClipThreads) void norm_kernel(const double* partial, int32_t partials, float* norm) {
    __shared__ double slots[kClipThreads / kWave];
    const double n = norm_of(partial, partials, slots);
    if (threadIdx.x == 0) *norm = (float)n;
}

// A norm that is not finite scales nothing: the caller sees it and leaves the step out.
__global__ __launch_bounds__(kClipThreads) void clip_kernel(ClipArgs a, const double* partial, int32_t partials, double most, float* norm) {
    __shared__ double slots[kClipThreads / kWave];
    const double n = norm_of(partial, partials, slots);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
    const bool scaled = n > most && n < INFINITY;
    const double factor = scaled ? most / n : 1.0;
    const float scale = (float)factor;
    const bool tiny = factor < 0x1p-126;     // (where fp32 has fewer bits for it, or none, though the largest gradients times it are not that small)
    for_units<true>(a, [&](auto tag, int i, uint32_t unit) {
        typedef decltype(tag) T;
        constexpr int P = kPack<T>;
        const T* in = static_cast<const T*>(a.tensor[i].in) + (int64_t)unit * kClipUnit;
        T* out = static_cast<T*>(a.tensor[i].out) + (int64_t)unit * kClipUnit;
        if (!scaled && in == out) return;
        const int n = (int)min((int64_t)kClipUnit, a.tensor[i].n - (int64_t)unit * kClipUnit);
        auto times = [&](Raw r) {
            if (!scaled) return r;           // (bit by bit, NaN too)
            float v[P];
            unpack(r, v, T());
#pragma unroll
            for (int e = 0; e < P; ++e) v[e] = tiny ? (float)((double)v[e] * factor) : v[e] * scale;
            return pack(v, T());
        };
        if (n == kClipUnit) {
            Raw r[kClipUnit / (kClipThreads * P)];
#pragma unroll
            for (int j = 0; j < kClipUnit / (kClipThreads * P); ++j) r[j] = load_raw_once(in + (j * kClipThreads + (int)threadIdx.x) * P);
#pragma unroll
            for (int j = 0; j < kClipUnit / (kClipThreads * P); ++j) store_raw_once(out + (j * kClipThreads + (int)threadIdx.x) * P, times(r[j]));
        } else {
            for (int c = (int)threadIdx.x * P; c < n; c += kClipThreads * P)
                store_some(out + c, times(load_some(in + c, min(P, n - c), 0.0f, c)), min(P, n - c));
        }
    });
}

}  // namespace mlda
