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

// N = kPerLoad<T> values from p on, as far as the first `left` of them exist (zeros beyond)
template <class T>
__device__ __forceinline__ void rk_load(const T *p, int64_t left, float (&v)[kPerLoad<T>])
{
    constexpr int N = kPerLoad<T>;
    if (left >= N) {
        const auto q = reinterpret_cast<const RkSlot<T> *>(p)->v;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = static_cast<float>(q[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = i < left ? static_cast<float>(p[i]) : 0.f;
    }
}

template <class T>
__device__ __forceinline__ void rk_store(T *p, int64_t left, const float (&v)[kPerLoad<T>])
{
    constexpr int N = kPerLoad<T>;
    if (left >= N) {
        typename RkSlot<T>::V q;
#pragma unroll
        for (int i = 0; i < N; ++i) q[i] = static_cast<T>(v[i]);
        reinterpret_cast<RkSlot<T> *>(p)->v = q;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) p[i] = static_cast<T>(v[i]);
    }
}

// N fp32 values from p on, as far as the first `left` of them exist (the others stay as they are)
template <int N>
__device__ __forceinline__ void rk_load_f32(const float *p, int64_t left, float (&v)[N])
{
    if (left >= N) {
#pragma unroll
        for (int k = 0; k < N; k += 4) {
            const auto q = reinterpret_cast<const RkSlot<float> *>(p + k)->v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[k + i] = q[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) v[i] = p[i];
    }
}

template <int N>
__device__ __forceinline__ void rk_store_f32(float *p, int64_t left, const float (&v)[N])
{
    if (left >= N) {
#pragma unroll
        for (int k = 0; k < N; k += 4) {
            RkSlot<float>::V q;
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = v[k + i];
            reinterpret_cast<RkSlot<float> *>(p + k)->v = q;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) p[i] = v[i];
    }
}
