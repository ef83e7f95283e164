// Values of the three element types (include/rocket.h, ROCKET_F32 ...) as the kernels load and store them: 16 bytes per
// lane at any element's address, arithmetic in fp32.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "rocket.h"

typedef __bf16 rk_bf16;
typedef _Float16 rk_f16;

inline size_t rk_type_bytes(int32_t dtype) { return dtype == ROCKET_F32 ? 4 : 2; }
inline bool rk_type_known(int32_t dtype) { return dtype == ROCKET_F32 || dtype == ROCKET_BF16 || dtype == ROCKET_F16; }

template <class T>
constexpr int kPerLoad = 16 / static_cast<int>(sizeof(T));

// 16 bytes that start at any element (the hardware takes such addresses; whole, aligned lines are faster)
template <class T>
struct RkSlot {
    typedef T V __attribute__((ext_vector_type(kPerLoad<T>), aligned(sizeof(T))));
    V v;
};

// Loads and stores of what a kernel passes once (`STREAM`) are marked as not to be kept: 800 MB read by 2,048 workgroups 125 us, so
// 115 (7.0 TB/s); 800 MB to 800 MB 283 us, so 256 (6.3 TB/s).
template <class T, bool STREAM>
__device__ __forceinline__ typename RkSlot<T>::V rk_load_slot(const T *p)
{
    if constexpr (STREAM) return __builtin_nontemporal_load(&reinterpret_cast<const RkSlot<T> *>(p)->v);
    else return reinterpret_cast<const RkSlot<T> *>(p)->v;
}

template <class T, bool STREAM>
__device__ __forceinline__ void rk_store_slot(T *p, typename RkSlot<T>::V v)
{
    if constexpr (STREAM) __builtin_nontemporal_store(v, &reinterpret_cast<RkSlot<T> *>(p)->v);
    else reinterpret_cast<RkSlot<T> *>(p)->v = v;
}

// The slot of values i .. i + N - 1 of a run of n that starts at p, zeros for those beyond its end.  No lane takes a way of its own
// (a lane that loads the last values one by one keeps its wavefront waiting for each): the slot is read where it still lies inside
// the run and shifted.  TINY: the run may be shorter than a slot.
template <class T, bool STREAM, bool TINY>
__device__ __forceinline__ typename RkSlot<T>::V rk_load_edge(const T *p, int i, int n)
{
    constexpr int N = kPerLoad<T>;
    if (TINY && n < N) {
        typename RkSlot<T>::V v;
        T each[N];
#pragma unroll
        for (int q = 0; q < N; ++q) each[q] = p[min(i + q, n - 1)];
#pragma unroll
        for (int q = 0; q < N; ++q) v[q] = i + q < n ? each[q] : static_cast<T>(0.f);
        return v;
    }
    const int at = min(i, n - N);
    const int bits = min(i - at, N) * static_cast<int>(8 * sizeof(T));
    const uint4 w = __builtin_bit_cast(uint4, rk_load_slot<T, STREAM>(p + at));
    uint64_t lo = (static_cast<uint64_t>(w.y) << 32) | w.x, hi = (static_cast<uint64_t>(w.w) << 32) | w.z;
    lo = (bits & 64) ? hi : lo;
    hi = (bits & 64) ? 0 : hi;
    const int some = bits & 63;       // lo of a shift by 64 - 0 would be undefined: in two steps
    lo = (lo >> some) | (hi << 1 << (63 - some));
    hi >>= some;
    const bool none = bits >= 128;
    const uint4 u = make_uint4(none ? 0 : static_cast<uint32_t>(lo), none ? 0 : static_cast<uint32_t>(lo >> 32), none ? 0 : static_cast<uint32_t>(hi),
                               none ? 0 : static_cast<uint32_t>(hi >> 32));
    return __builtin_bit_cast(typename RkSlot<T>::V, u);
}

// N fp32 values from p on
template <int N>
__device__ __forceinline__ void rk_load_f32(const float *p, float (&v)[N])
{
#pragma unroll
    for (int k = 0; k < N; k += 4) {
        const RkSlot<float>::V q = rk_load_slot<float, false>(p + k);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[k + j] = q[j];
    }
}

// values i .. i + N - 1 of a run of n, four at least, that starts at p, zeros beyond its end
template <int N>
__device__ __forceinline__ void rk_load_f32_edge(const float *p, int i, int n, float (&v)[N])
{
#pragma unroll
    for (int k = 0; k < N; k += 4) {
        const RkSlot<float>::V q = rk_load_edge<float, false, false>(p, i + k, n);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[k + j] = q[j];
    }
}

template <class T, bool STREAM>
__device__ __forceinline__ void rk_store(T *p, int left, const float (&v)[kPerLoad<T>])
{
    constexpr int N = kPerLoad<T>;
    if (left >= N) {
        typename RkSlot<T>::V q;
#pragma unroll
        for (int i = 0; i < N; ++i) q[i] = static_cast<T>(v[i]);
        rk_store_slot<T, STREAM>(p, q);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) p[i] = static_cast<T>(v[i]);
    }
}

template <int N, bool STREAM = false>
__device__ __forceinline__ void rk_store_f32(float *p, int left, const float (&v)[N])
{
#pragma unroll
    for (int k = 0; k < N; k += 4) {
        const float some[4] = {v[k], v[k + 1], v[k + 2], v[k + 3]};
        rk_store<float, STREAM>(p + k, left - k, some);
    }
}
