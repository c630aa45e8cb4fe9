// Typed rows in 16-byte pieces, and sums and maxima over teams of lanes, for the operators on tensors.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include "device_util.hpp"

namespace mlda {

typedef uint32_t Raw __attribute__((ext_vector_type(4)));                         // 16 bytes as loaded
typedef Raw RawAnywhere __attribute__((aligned(2), may_alias));                   // at any element of a row
typedef __bf16 Bf16;
typedef _Float16 Fp16;

template <class T> constexpr int kPack = 16 / (int)sizeof(T);                      // elements of 16 bytes

// Rows start wherever their stride puts them: 16 bytes are read and written at the alignment of an element.
template <class T> __device__ __forceinline__ Raw load_raw(const T* p) { return *reinterpret_cast<const RawAnywhere*>(p); }
template <class T> __device__ __forceinline__ void store_raw(T* p, Raw r) { *reinterpret_cast<RawAnywhere*>(p) = r; }

__device__ __forceinline__ void unpack(Raw r, float (&out)[4], float) {
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void unpack(Raw r, float (&out)[8], Bf16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        out[2 * i] = __uint_as_float(r[i] << 16);
        out[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack(Raw r, float (&out)[8], Fp16) {
    typedef Fp16 H8 __attribute__((ext_vector_type(8)));
    const H8 h = __builtin_bit_cast(H8, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) out[i] = (float)h[i];
}

// Rounded to nearest, ties to even: the one rounding of a result.
__device__ __forceinline__ Raw pack(const float (&in)[4], float) {
    Raw r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(in[i]);
    return r;
}
template <class H>
__device__ __forceinline__ Raw pack(const float (&in)[8], H) {
    typedef H H8 __attribute__((ext_vector_type(8)));
    typedef float F8 __attribute__((ext_vector_type(8)));
    F8 f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = in[i];
    const H8 h = __builtin_convertvector(f, H8);
    return __builtin_bit_cast(Raw, h);
}

// `n` (0 .. kPack) elements from p on, `fill` behind them; never reads past the n-th.
template <class T>
__device__ __forceinline__ Raw load_some(const T* p, int n, float fill) {
    if (n >= kPack<T>) return load_raw(p);
    float v[kPack<T>];
#pragma unroll
    for (int e = 0; e < kPack<T>; ++e) v[e] = e < n ? (float)p[e] : fill;
    return pack(v, T());
}

template <class T>
__device__ __forceinline__ void store_some(T* p, Raw r, int n) {
    if (n >= kPack<T>) { store_raw(p, r); return; }
    float v[kPack<T>];
    unpack(r, v, T());
#pragma unroll
    for (int e = 0; e < kPack<T>; ++e)
        if (e < n) p[e] = (T)v[e];
}

template <int kCtrl>
__device__ __forceinline__ float dpp_all(float v) {          // a permutation of lanes: every lane has a source
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), kCtrl, 0xf, 0xf, false));
}

// Sum over the 16 lanes of a row; every lane gets it.  Every lane must be active.
__device__ __forceinline__ float row16_sum(float v) {
    v += dpp_all<0x128>(v);          // row_ror:8, 4, 2, 1
    v += dpp_all<0x124>(v);
    v += dpp_all<0x122>(v);
    v += dpp_all<0x121>(v);
    return v;
}

__device__ __forceinline__ float wave_sum(float v) {
    v = row16_sum(v);
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x142, 0xa, 0xf, false));   // row_bcast:15
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x143, 0xc, 0xf, false));   // row_bcast:31
    return read_lane(v, kWave - 1);
}

// (NaN counts for nothing in a maximum)
__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, dpp_all<0x128>(v));
    v = fmaxf(v, dpp_all<0x124>(v));
    v = fmaxf(v, dpp_all<0x122>(v));
    v = fmaxf(v, dpp_all<0x121>(v));
    const float a = fmaxf(read_lane(v, 15), read_lane(v, 31)), b = fmaxf(read_lane(v, 47), read_lane(v, 63));
    return fmaxf(a, b);
}

// Sum over a team of kTeam lanes (16, 64, or a whole workgroup of more), which every lane of the team gets.  `slots`: LDS of
// kTeam / 64 floats that no earlier sum uses whose readers may still be reading: two taken in turn do, as each sum has one
// barrier.  The order of the additions is fixed.
template <int kTeam>
__device__ __forceinline__ float team_sum(float v, float* slots) {
    if constexpr (kTeam == 16) return row16_sum(v);
    v = wave_sum(v);
    if constexpr (kTeam > kWave) {
        constexpr int kWaves = kTeam / kWave;
        if (lane_id() == 0) slots[threadIdx.x / kWave] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v += slots[w];
    }
    return v;
}

}  // namespace mlda
