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
// The same for what is not read again soon: it does not take the place in the caches of what is.
template <class T> __device__ __forceinline__ Raw load_raw_once(const T* p) { return __builtin_nontemporal_load(reinterpret_cast<const RawAnywhere*>(p)); }
template <class T> __device__ __forceinline__ void store_raw_once(T* p, Raw r) { __builtin_nontemporal_store(r, reinterpret_cast<RawAnywhere*>(p)); }

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

// What was made of these pieces before is not kept in registers for what is made of them next: unpacking again takes one
// instruction an element, keeping it a register.
template <int N>
__device__ __forceinline__ void forget(Raw (&r)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(r[i]));
}

// Moves a piece's elements `by` (0 .. kPack - 1) places down, and puts `fill` behind the first `n` of what results.
template <class T>
__device__ __forceinline__ Raw move_down(Raw r, int by, int n, T fill) {
    if constexpr (sizeof(T) == 4) {
        const uint32_t f = __builtin_bit_cast(uint32_t, fill);
        if (by & 2) { r[0] = r[2]; r[1] = r[3]; }
        if (by & 1) { r[0] = r[1]; r[1] = r[2]; r[2] = r[3]; }
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = i < n ? r[i] : f;
    } else {
        const uint32_t f = __builtin_bit_cast(uint16_t, fill);
        if (by & 4) { r[0] = r[2]; r[1] = r[3]; }
        if (by & 2) { r[0] = r[1]; r[1] = r[2]; r[2] = r[3]; }
        if (by & 1) {
            r[0] = r[0] >> 16 | r[1] << 16;
            r[1] = r[1] >> 16 | r[2] << 16;
            r[2] = r[2] >> 16 | r[3] << 16;
            r[3] = r[3] >> 16;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = 2 * i + 1 < n ? r[i] : 2 * i < n ? (r[i] & 0xffffu) | f << 16 : f << 16 | f;
    }
    return r;
}

// Moves a piece's elements `by` (0 .. kPack - 1) places up.
template <class T>
__device__ __forceinline__ Raw move_up(Raw r, int by) {
    if constexpr (sizeof(T) == 4) {
        if (by & 2) { r[3] = r[1]; r[2] = r[0]; }
        if (by & 1) { r[3] = r[2]; r[2] = r[1]; r[1] = r[0]; }
    } else {
        if (by & 4) { r[3] = r[1]; r[2] = r[0]; }
        if (by & 2) { r[3] = r[2]; r[2] = r[1]; r[1] = r[0]; }
        if (by & 1) {
            r[3] = r[3] << 16 | r[2] >> 16;
            r[2] = r[2] << 16 | r[1] >> 16;
            r[1] = r[1] << 16 | r[0] >> 16;
            r[0] = r[0] << 16;
        }
    }
    return r;
}

// The elements [from, to) of a piece, `fill` in the others' places.
template <class T>
__device__ __forceinline__ Raw keep(Raw r, int from, int to, T fill) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            r[i] = i >= from && i < to ? r[i] : __builtin_bit_cast(uint32_t, fill);
        } else {
            const uint32_t f = __builtin_bit_cast(uint16_t, fill);
            const uint32_t mask = (2 * i >= from && 2 * i < to ? 0xffffu : 0u) | (2 * i + 1 >= from && 2 * i + 1 < to ? 0xffff0000u : 0u);
            r[i] = (r[i] & mask) | ((f << 16 | f) & ~mask);
        }
    }
    return r;
}

// The piece of columns [c, c + kPack) of which [lo, hi) are there, `fill` in the others' places; reads nothing outside [lo, hi).
template <class T>
__device__ __forceinline__ Raw load_piece(const T* base, int64_t c, int64_t lo, int64_t hi, float fill, bool once) {
    constexpr int P = kPack<T>;
    if (c >= lo && c + P <= hi) {
        Raw r;
        if (once) {
            asm volatile("" ::: "memory");              // (or both loads become one, the second)
            r = load_raw_once(base + c);
            asm volatile("" ::: "memory");
        } else {
            r = load_raw(base + c);
        }
        return r;
    }
    const int from = (int)max((int64_t)0, min((int64_t)P, lo - c)), to = (int)max((int64_t)0, min((int64_t)P, hi - c));
    Raw r = {0, 0, 0, 0};
    if (from >= to) return keep(r, 0, 0, (T)fill);
    if (hi - lo >= P) {
        const int64_t at = max(lo, min(c, hi - P));     // a whole piece nearby
        r = load_raw(base + at);
        r = at > c ? move_up<T>(r, (int)(at - c)) : move_down(r, (int)(c - at), P, (T)fill);
    } else {
        typedef std::conditional_t<sizeof(T) == 4, uint32_t, uint16_t> Bits;
#pragma unroll 1
        for (int e = to; e-- > 0;) {                    // a row shorter than a piece
            const uint32_t bits = e >= from ? *reinterpret_cast<const Bits*>(base + c + e) : 0;
            if constexpr (sizeof(T) == 4) r = Raw{bits, r[0], r[1], r[2]};
            else r = Raw{r[0] << 16 | bits, r[1] << 16 | r[0] >> 16, r[2] << 16 | r[1] >> 16, r[3] << 16 | r[2] >> 16};
        }
    }
    return keep(r, from, to, (T)fill);
}

template <class T>
__device__ __forceinline__ void store_piece(T* base, int64_t c, int64_t lo, int64_t hi, Raw r, bool once) {
    constexpr int P = kPack<T>;
    if (c >= lo && c + P <= hi) {
        if (once) {
            asm volatile("" ::: "memory");              // (or both stores become one, the second)
            store_raw_once(base + c, r);
            asm volatile("" ::: "memory");
        } else {
            store_raw(base + c, r);
        }
        return;
    }
    typedef std::conditional_t<sizeof(T) == 4, uint32_t, uint16_t> Bits;
#pragma unroll
    for (int e = 0; e < P; ++e) {
        const uint32_t bits = sizeof(T) == 4 ? r[e % 4] : r[e / 2] >> (e % 2 * 16);
        if (c + e >= lo && c + e < hi) *reinterpret_cast<Bits*>(base + c + e) = (Bits)bits;
    }
}

// `n` (at most kPack) elements from p on, `fill` behind them; never reads past the n-th, nor more than `before` elements before
// p.  The end of a row is the piece that ends there, moved down: one load, whatever is left.
template <class T>
__device__ __forceinline__ Raw load_some(const T* p, int n, float fill, int64_t before) {
    constexpr int P = kPack<T>;
    if (n >= P) return load_raw(p);
    Raw r = {0, 0, 0, 0};
    if (n <= 0) return move_down(r, 0, 0, (T)fill);
    if (before >= P - n) return move_down(load_raw(p - (P - n)), P - n, n, (T)fill);
#pragma unroll 1
    for (int e = n; e-- > 0;) {                       // a row shorter than a piece
        typedef std::conditional_t<sizeof(T) == 4, uint32_t, uint16_t> Bits;
        const uint32_t bits = *reinterpret_cast<const Bits*>(p + e);
        if constexpr (sizeof(T) == 4) r = Raw{bits, r[0], r[1], r[2]};
        else r = Raw{r[0] << 16 | bits, r[1] << 16 | r[0] >> 16, r[2] << 16 | r[1] >> 16, r[3] << 16 | r[2] >> 16};
    }
    return move_down(r, 0, n, (T)fill);
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

// Sum over a team of kTeam lanes (4, 16, or whole waves: then all of the workgroup's teams take part at once), which every lane of the
// team gets.  `slots`: LDS of a float for each of the workgroup's waves that no earlier sum uses whose readers may still be
// reading: two taken in turn do, as each sum has one barrier.  The order of the additions is fixed.
template <int kTeam>
__device__ __forceinline__ float lanes_sum(float v) {
    if constexpr (kTeam == 4) {
        v += dpp_all<0xb1>(v);       // quad_perm: 1 0 3 2, then 2 3 0 1
        return v + dpp_all<0x4e>(v);
    }
    return kTeam == 16 ? row16_sum(v) : wave_sum(v);
}

template <int kTeam>
__device__ __forceinline__ float team_sum(float v, float* slots) {
    v = lanes_sum<kTeam>(v);
    if constexpr (kTeam > kWave) {
        constexpr int kWaves = kTeam / kWave;
        slots += (int)threadIdx.x / kTeam * kWaves;
        if (lane_id() == 0) slots[(int)threadIdx.x % kTeam / kWave] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v += slots[w];
    }
    return v;
}

// The same in fp64 over a workgroup.
template <int kThreads>
__device__ __forceinline__ double group_sum(double v, double* slots) {
    v = wave_sum(v);
    if (lane_id() == 0) slots[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / kWave; ++w) v += slots[w];
    return v;
}

// Two sums with one barrier; slots of twice the size.
template <int kTeam>
__device__ __forceinline__ void team_sums(float& a, float& b, float* slots) {
    a = lanes_sum<kTeam>(a);
    b = lanes_sum<kTeam>(b);
    if constexpr (kTeam > kWave) {
        constexpr int kWaves = kTeam / kWave;
        slots += (int)threadIdx.x / kTeam * 2 * kWaves;
        if (lane_id() == 0) {
            slots[(int)threadIdx.x % kTeam / kWave] = a;
            slots[kWaves + (int)threadIdx.x % kTeam / kWave] = b;
        }
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            a += slots[w];
            b += slots[kWaves + w];
        }
    }
}

}  // namespace mlda
