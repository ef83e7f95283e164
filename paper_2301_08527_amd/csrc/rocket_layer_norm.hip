// Layer norm of feature planes for MI355X (gfx950), forward and backward.  See include/rocket.h for the contract.
//
// A row is one plane of one example: R = rows * planes rows of n values, row i has the weights of plane i % planes.
//   forward   m = mean x, v = mean (x - m)^2, r = 1/sqrt(v + eps), y = (x - m) r w + b
//   backward  g = dy w, h = (x - m) r:  dx = r (g - mean g - h mean(g h)),  dw = sum dy h,  db = sum dy (over the rows of a plane)
// Both are bound by memory, with some ten vector instructions a value and more; of 16-bit values, where those fill the issue slots at the
// same time, each counts.
//
// The mean that the backward pass is given is rounded to 32 bits, an error of (x - m) that all values of a row share.  With
// h' = (x - m') r and e = mean h' (0 but for that rounding), h = h' - e: one more sum, and rows whose mean is a million times
// their spread keep all their digits.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>
#include <type_traits>

#include "rocket_elements.hpp"
#include "rocket_internal.hpp"

namespace {

constexpr int kNormThreads = 256;

// ------------------------------------------------------------------ sums over lanes

template <int CTRL, int ROWS>
__device__ __forceinline__ float rn_dpp(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
}

// Sum over LANES neighbouring lanes, the same bits on each of them: within quads, then by reflections within eight and sixteen
// lanes, then across the rows of sixteen.
template <int LANES>
__device__ __forceinline__ float rn_lanes_sum(float v)
{
    static_assert(LANES == 4 || LANES == 8 || LANES == 16 || LANES == 32 || LANES == 64, "lanes that meet without LDS");
    v += rn_dpp<0xB1, 0xf>(v);        // quad_perm 1,0,3,2 and 2,3,0,1
    v += rn_dpp<0x4E, 0xf>(v);
    if constexpr (LANES >= 8) v += rn_dpp<0x141, 0xf>(v);      // row_half_mirror
    if constexpr (LANES >= 16) v += rn_dpp<0x140, 0xf>(v);     // row_mirror
    if constexpr (LANES == 32) v += __shfl_xor(v, 16, 64);
    if constexpr (LANES == 64) {
        v += rn_dpp<0x142, 0xa>(v);   // row_bcast:15 into rows 1 and 3, row_bcast:31 into rows 2 and 3
        v += rn_dpp<0x143, 0xc>(v);
        v = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
    }
    return v;
}

// Count, mean and sum of squared distances from it of some values of a row, the mean as shift + rest: two parts whose sum has
// more than 32 bits, so that x - shift - rest is right to the last bits however far from zero the row lies.
struct Moments {
    float count, shift, rest, m2;
};

// A row in the registers of its lanes, as it was loaded: slot k of LANES lanes together is values k * step .. (k + 1) * step - 1, and all
// slots but the last are whole.  In the last one the lane that reaches over the end has the row's last N values instead, and so
// have the lanes beyond it: no lane takes a way of its own (one that loads its values one by one keeps its wavefront waiting
// for each).  Values that an earlier lane has too count in no sum; what is stored for them is the same bits twice.  Only rows
// shorter than a slot (TINY) are loaded and stored value by value.
template <class T, int SLOTS>
using Held = typename RkSlot<T>::V[SLOTS];

template <class T, int LANES, int SLOTS>
struct Place {
    static constexpr int N = kPerLoad<T>, kStep = LANES * N;
    static constexpr bool kTiny = LANES == 4;
    int n, first, last, skip;      // values of the row; places of slots 0 and SLOTS - 1; values of the last one that do not count
    bool tiny, some, mixed;        // some: the last slot has values that count; mixed: the wavefront has values that do not
    __device__ __forceinline__ Place(int n, int lane) : n(n)
    {
        const int i = lane * N + (SLOTS - 1) * kStep;
        tiny = kTiny && n < N;
        last = max(min(i, n - N), 0);
        first = SLOTS > 1 ? lane * N : last;
        skip = min(i - last, N);
        some = tiny ? lane == 0 : skip < N;
        mixed = __any(tiny || skip > 0);
    }
    __device__ __forceinline__ int at(int k) const { return k < SLOTS - 1 ? first + k * kStep : last; }
    // whether value q of slot k counts
    __device__ __forceinline__ bool counts(int k, int q) const { return k < SLOTS - 1 || (kTiny && tiny ? some && q < n : q >= skip); }
};

template <class T, int LANES, int SLOTS, bool STREAM>
__device__ __forceinline__ void rn_hold(Held<T, SLOTS> &raw, const T *src, const Place<T, LANES, SLOTS> &place)
{
    constexpr int N = kPerLoad<T>;
    if (place.kTiny && place.tiny) {
#pragma unroll
        for (int q = 0; q < N; ++q) raw[0][q] = src[min(q, place.n - 1)];
        return;
    }
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) raw[k] = rk_load_slot<T, STREAM>(src + place.at(k));
}

// N values of a plane's weights or biases beside those of slot k
template <class T, int LANES, int SLOTS>
__device__ __forceinline__ void rn_beside(const float *from, const Place<T, LANES, SLOTS> &place, int k, float (&v)[kPerLoad<T>])
{
    if (place.kTiny && place.tiny) {
#pragma unroll
        for (int q = 0; q < kPerLoad<T>; ++q) v[q] = from[min(q, place.n - 1)];
        return;
    }
    rk_load_f32<kPerLoad<T>>(from + place.at(k), v);
}

template <class T, int LANES, int SLOTS, bool STREAM>
__device__ __forceinline__ void rn_put(T *dst, const Place<T, LANES, SLOTS> &place, int k, const float (&v)[kPerLoad<T>])
{
    if (k == SLOTS - 1 && !place.some) return;
    rk_store<T, STREAM>(dst + place.at(k), place.kTiny && place.tiny ? place.n : kPerLoad<T>, v);
}

// Keeps the compiler from carrying what it made of the slots (their values as floats, twice the registers of 16-bit ones) from one
// pass over them to the next: made again, they cost an instruction or two.
template <class T, int SLOTS>
__device__ __forceinline__ void rn_forget(Held<T, SLOTS> &raw)
{
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
        uint4 u = __builtin_bit_cast(uint4, raw[k]);
        asm volatile("" : "+v"(u.x), "+v"(u.y), "+v"(u.z), "+v"(u.w));
        raw[k] = __builtin_bit_cast(typename RkSlot<T>::V, u);
    }
}

// Moments of what LANES lanes hold of a row, `count` values; counts(k, q): whether value q of slot k does.  (Whole slots by a branch of their
// own: 65,536 x 2,048 bf16 98 us, then 106.)  More than 64 values a lane adds in two halves, so that no sum has more than 80 numbers one after
// the other (64, 6 exchanges of lanes and 4 of wavefronts); 500 x 125,000 bf16 55.3 us, with it 56.2.
template <class T, int LANES, int SLOTS, class F>
__device__ __forceinline__ Moments rn_moments(const Held<T, SLOTS> &raw, float count, F counts)
{
    constexpr int N = kPerLoad<T>, kSums = SLOTS * N > 64 ? 2 : 1;
    const auto halves = [](const float (&v)[kSums]) { return kSums > 1 ? v[0] + v[kSums - 1] : v[0]; };
    float s[kSums] = {}, d1s[kSums] = {}, d2s[kSums] = {};
#pragma unroll
    for (int k = 0; k < SLOTS; ++k)
#pragma unroll
        for (int q = 0; q < N; ++q) s[k * kSums / SLOTS] += counts(k, q) ? static_cast<float>(raw[k][q]) : 0.f;
    const float shift = rn_lanes_sum<LANES>(halves(s)) / count;
#pragma unroll
    for (int k = 0; k < SLOTS; ++k)
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const float d = counts(k, q) ? static_cast<float>(raw[k][q]) - shift : 0.f;
            d1s[k * kSums / SLOTS] += d;
            d2s[k * kSums / SLOTS] = fmaf(d, d, d2s[k * kSums / SLOTS]);
        }
    const float d1 = rn_lanes_sum<LANES>(halves(d1s)), d2 = rn_lanes_sum<LANES>(halves(d2s));
    const float rest = d1 / count;
    const float m2 = fmaf(-rest, d1, d2);
    return {count, shift, rest, m2 < 0.f ? 0.f : m2};      // NaN stays
}

// Moments of the values of up to 16 parts, of which lane l of every row of 16 lanes holds part l (count 0: none): distances of
// the parts' means from the first one's, weighted by their counts.
__device__ __forceinline__ Moments rn_join(const Moments &part, float n)
{
    const float shift = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, part.shift), 0));
    const bool some = part.count > 0.f;
    const float off = some ? (part.shift - shift) + part.rest : 0.f;
    const float rest = rn_lanes_sum<16>(part.count * off) / n;
    const float apart = off - rest;
    return {n, shift, rest, rn_lanes_sum<16>(some ? fmaf(part.count * apart, apart, part.m2) : 0.f)};
}

// The rest of the mean is a rounding or so of x - shift: its product with r loses nothing that counts.
template <int N>
__device__ __forceinline__ void rn_normal(const float (&x)[N], const Moments &m, float r, const float (&w)[N], const float (&b)[N], float (&y)[N])
{
    const float rest = -m.rest * r;
#pragma unroll
    for (int q = 0; q < N; ++q) y[q] = fmaf(fmaf(x[q] - m.shift, r, rest), w[q], b[q]);
}

// n as a float: exact up to 2^24, and a rounding of 2^-25 of the mean of squares beyond
__device__ __forceinline__ float rn_rstd(const Moments &m, float eps) { return 1.f / sqrtf(m.m2 / m.count + eps); }

// A row lies in the registers of LANES lanes, SLOTS loads of 16 bytes in each (as loaded: 16-bit values take half the registers),
// so x is read once.  Two passes over the registers give the mean and the distances from it; up to 64 lanes meet by lane
// exchanges alone, more lanes once through LDS, where the wavefronts' own means and sums of squares are joined.  A group of lanes has one
// plane of ROWS examples, whose weights it loads once.  Groups of neighbouring planes lie side by side; examples
// `first` .. `end` - 1 (the last workgroup may have groups left over: what lies behind `end` is another launch's).
template <class T, int LANES, int SLOTS, int ROWS, bool STREAM>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void rn_forward(const T *x, int first, int end, int planes, int n,
                                                                        const float *__restrict__ weight, const float *__restrict__ bias, float eps,
                                                                        T *y, float *__restrict__ mean, float *__restrict__ rstd)
{
    constexpr int N = kPerLoad<T>, kGroups = LANES < 256 ? 256 / LANES : 1;
    constexpr bool kEarly = SLOTS * N * (ROWS > 2 ? 2 : ROWS) <= 16;       // weights and biases are on their way while the lanes meet
    static_assert(LANES <= 64 || LANES >= 256, "a row of several wavefronts has the workgroup to itself");
    __shared__ float4 meet[LANES > 64 ? ROWS : 1][LANES > 64 ? 16 : 1];
    const int lane = static_cast<int>(threadIdx.x) & (LANES - 1), wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
    const unsigned group = blockIdx.x * kGroups + threadIdx.x / LANES, block = group / static_cast<unsigned>(planes);
    const int plane = static_cast<int>(group - block * static_cast<unsigned>(planes));
    const int64_t b0 = first + static_cast<int64_t>(block) * ROWS;
    if (LANES <= 64 && b0 >= end) return;
    const Place<T, LANES, SLOTS> place(n, lane);
    Held<T, SLOTS> raw[ROWS];
    float w[kEarly ? SLOTS : 1][N], b[kEarly ? SLOTS : 1][N];
    const int64_t w0 = static_cast<int64_t>(plane) * n;
    const auto load_beside = [&](int k, float (&ww)[N], float (&bb)[N]) {
#pragma unroll
        for (int q = 0; q < N; ++q) ww[q] = 1.f, bb[q] = 0.f;
        if (weight) rn_beside(weight + w0, place, k, ww);
        if (bias) rn_beside(bias + w0, place, k, bb);
    };
    const auto row_of = [&](int j) { return min(b0 + j, static_cast<int64_t>(end) - 1) * planes + plane; };       // beyond the last: the last once more
#pragma unroll
    for (int j = 0; j < ROWS; ++j) rn_hold<T, LANES, SLOTS, STREAM>(raw[j], x + row_of(j) * n, place);
    if constexpr (kEarly)
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) load_beside(k, w[k], b[k]);
    const auto counts = [&](int k, int q) { return place.counts(k, q); };
    Moments m[ROWS];
    float r[ROWS];
    if constexpr (LANES <= 64) {
#pragma unroll
        for (int j = 0; j < ROWS; ++j) m[j] = rn_moments<T, LANES, SLOTS>(raw[j], static_cast<float>(n), counts);
    } else {
        const int count = (SLOTS - 1) * 64 * N + min(max(n - ((SLOTS - 1) * place.kStep + wave * 64 * N), 0), 64 * N);
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
            const Moments own = rn_moments<T, 64, SLOTS>(raw[j], static_cast<float>(max(count, 1)), counts);
            if ((threadIdx.x & 63) == 0) meet[j][wave] = make_float4(static_cast<float>(count), own.shift, own.rest, own.m2);
            if (static_cast<int>(threadIdx.x) >= LANES - 64 && static_cast<int>(threadIdx.x & 63) > 0 && wave + static_cast<int>(threadIdx.x & 63) < 16)
                meet[j][wave + (threadIdx.x & 63)] = make_float4(0.f, 0.f, 0.f, 0.f);        // places that no wavefront has
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
            const float4 part = meet[j][threadIdx.x & 15];
            m[j] = rn_join({part.x, part.y, part.z, part.w}, static_cast<float>(n));
        }
    }
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        r[j] = rn_rstd(m[j], eps);
        if constexpr (sizeof(T) == 2) rn_forget<T, SLOTS>(raw[j]);
        if (mean && lane == 0 && b0 + j < end) {
            mean[row_of(j)] = m[j].shift + m[j].rest;
            rstd[row_of(j)] = r[j];
        }
    }
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
        if constexpr (!kEarly) load_beside(k, w[0], b[0]);
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
            float v[N], out[N];
#pragma unroll
            for (int q = 0; q < N; ++q) v[q] = static_cast<float>(raw[j][k][q]);
            rn_normal(v, m[j], r[j], w[kEarly ? k : 0], b[kEarly ? k : 0], out);
            if (ROWS == 1 || b0 + j < end) rn_put<T, LANES, SLOTS, STREAM>(y + row_of(j) * n, place, k, out);
        }
    }
}

// Longer rows: moments of parts of a row, one workgroup each, then each part again with those of its row joined.  At most kMostParts
// parts to a row; a part is `length` values, in pieces of kPart that a workgroup holds.  grid (parts, R up to 2^15 and on)
constexpr int kMostParts = 64, kPartSlots = 4;
template <class T>
constexpr int kPart = kNormThreads * kPartSlots * kPerLoad<T>;

// The slots of a piece from value `from` of a row of n on; whole: the row has all of them (else zeros beyond its end)
template <class T, bool STREAM, class F>
__device__ __forceinline__ void rn_piece(Held<T, kPartSlots> &raw, const T *src, int from, int n, F whole)
{
    constexpr int N = kPerLoad<T>;
#pragma unroll
    for (int k = 0; k < kPartSlots; ++k) {
        const int i = from + (k * kNormThreads + static_cast<int>(threadIdx.x)) * N;
        raw[k] = whole ? rk_load_slot<T, STREAM>(src + i) : rk_load_edge<T, STREAM, false>(src, i, n);
    }
}

// f(true_type) or f(false_type): one copy of the code for whole pieces, one for the last
template <class F>
__device__ __forceinline__ void rn_by_whole(bool whole, F f)
{
    if (whole) f(std::true_type());
    else f(std::false_type());
}

template <class T>
__global__ __launch_bounds__(kNormThreads) void rn_forward_parts(const T *x, int64_t R, int n, int length, float4 *__restrict__ moments)
{
    constexpr int N = kPerLoad<T>;
    __shared__ float4 lds[16];
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
    for (int64_t row = blockIdx.y; row < R; row += gridDim.y) {
        const int from = static_cast<int>(blockIdx.x) * length, to = from + min(n - from, length);
        Moments m = {0.f, 0.f, 0.f, 0.f};
        for (int at = from; at < to; at += kPart<T>) {
            const int some = min(to - at, kPart<T>);
            int count = 0;
            Moments own;
            rn_by_whole(some == kPart<T>, [&](auto whole) {
                Held<T, kPartSlots> raw;
                rn_piece<T, false>(raw, x + row * n, at, n, whole);
#pragma unroll
                for (int k = 0; k < kPartSlots; ++k) count += whole ? 64 * N : min(max(some - (k * kNormThreads * N + wave * 64 * N), 0), 64 * N);
                own = rn_moments<T, 64, kPartSlots>(raw, static_cast<float>(max(count, 1)), [&](int k, int q) {
                    return whole || (k * kNormThreads + static_cast<int>(threadIdx.x)) * N + q < some;
                });
            });
            __syncthreads();      // the last piece has been read
            if (static_cast<int>(threadIdx.x) < 16) lds[threadIdx.x] = make_float4(0.f, 0.f, 0.f, 0.f);
            __syncthreads();
            if ((threadIdx.x & 63) == 0) lds[wave] = make_float4(static_cast<float>(count), own.shift, own.rest, own.m2);
            if (threadIdx.x == 0) lds[4] = make_float4(m.count, m.shift, m.rest, m.m2);      // what came before
            __syncthreads();
            const float4 part = lds[threadIdx.x & 15];
            m = rn_join({part.x, part.y, part.z, part.w}, m.count + static_cast<float>(some));
        }
        if (threadIdx.x == 0) moments[row * gridDim.x + blockIdx.x] = make_float4(m.count, m.shift, m.rest, m.m2);
    }
}

// The moments of a row from those of its parts, 16 at a time.
__device__ __forceinline__ Moments rn_row_moments(const float4 *moments, int parts)
{
    Moments m = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < parts; p += 15) {
        const int l = static_cast<int>(threadIdx.x) & 15;
        const bool some = l > 0 && p + l - 1 < parts;
        const float4 part = some ? moments[p + l - 1] : make_float4(l == 0 ? m.count : 0.f, m.shift, m.rest, m.m2);
        const float count = rn_lanes_sum<16>(part.x);
        if (p == 0) {       // nothing before: the first part takes its place, so that the shift is one of the row's means
            const float4 first = moments[0];
            const Moments mine = {l == 0 ? 0.f : part.x, l == 0 ? first.y : part.y, l == 0 ? 0.f : part.z, l == 0 ? 0.f : part.w};
            m = rn_join(mine, count);
        } else {
            m = rn_join({part.x, part.y, part.z, part.w}, count);
        }
    }
    return m;
}

// What is written is never kept for the next kernel at the cost of what the caches hold, what is read for the last time (ONCE) neither where
// they did not keep it anyway: 1,000 x 50,000 fp32 128 us, so 108; 1,000 x 150,000 347, so 313.
template <class T, bool ONCE>
__global__ __launch_bounds__(kNormThreads) void rn_forward_apply(const T *x, int64_t R, int planes, int n, int parts,
                                                                 const float4 *__restrict__ moments, const float *__restrict__ weight,
                                                                 const float *__restrict__ bias, float eps, T *y, float *__restrict__ mean,
                                                                 float *__restrict__ rstd)
{
    constexpr int N = kPerLoad<T>;
    for (int64_t row = blockIdx.y; row < R; row += gridDim.y) {
        const Moments m = rn_row_moments(moments + row * parts, parts);
        const float r = rn_rstd(m, eps);
        const int64_t w0 = row % planes * n;
        const int from = static_cast<int>(blockIdx.x) * kPart<T>;
        rn_by_whole(from + kPart<T> <= n, [&](auto whole) {
            Held<T, kPartSlots> raw;
            rn_piece<T, ONCE>(raw, x + row * n, from, n, whole);
#pragma unroll
            for (int k = 0; k < kPartSlots; ++k) {
                const int i = from + (k * kNormThreads + static_cast<int>(threadIdx.x)) * N;
                float v[N], w[N], b[N], out[N];
#pragma unroll
                for (int q = 0; q < N; ++q) v[q] = static_cast<float>(raw[k][q]), w[q] = 1.f, b[q] = 0.f;
                if (weight) {
                    if constexpr (whole) rk_load_f32<N>(weight + w0 + i, w);
                    else rk_load_f32_edge<N>(weight + w0, i, n, w);
                }
                if (bias) {
                    if constexpr (whole) rk_load_f32<N>(bias + w0 + i, b);
                    else rk_load_f32_edge<N>(bias + w0, i, n, b);
                }
                rn_normal(v, m, r, w, b, out);
                if (whole || i < n) rk_store<T, true>(y + row * n + i, whole ? N : n - i, out);
            }
        });
        if (mean && blockIdx.x == 0 && threadIdx.x == 0) {
            mean[row] = m.shift + m.rest;
            rstd[row] = r;
        }
    }
}

// ------------------------------------------------------------------ backward

// The partial sums of the weight's and the bias's gradient: one row of 2 * stride floats for each part of the rows, wide = planes * n
// of each used.
__device__ __host__ __forceinline__ int64_t rn_stride(int64_t wide) { return (wide + 3) / 4 * 4; }

// A row of x and one of dy lie in the registers of LANES lanes as in the forward pass; the lanes go on to further rows of the same
// plane and keep the sums of their columns, so x and dy are read once.  GROUPS rows at a time, whose sums meet in LDS at the end.
// grid (parts of the rows, planes).  With one part the sums are the gradients.
template <class T, int LANES, int SLOTS, int GROUPS, bool STREAM>
__global__ __launch_bounds__(LANES * GROUPS) void rn_backward(const T *x, const T *dy, int rows, int planes, int n, const float *__restrict__ weight,
                                                              const float *__restrict__ mean, const float *__restrict__ rstd, T *dx,
                                                              float *__restrict__ part, float *__restrict__ grad_w, float *__restrict__ grad_b)
{
    constexpr int N = kPerLoad<T>, kWaves = LANES > 64 ? LANES / 64 : 1, kWide = SLOTS * N * LANES;
    constexpr bool kAhead = sizeof(T) == 2 && SLOTS == 1 && LANES >= 512;       // the next row is loaded before the last one is done with
    static_assert(LANES <= 64 || GROUPS == 1, "a row of several wavefronts has the workgroup to itself");
    __shared__ float meet[2][3][kWaves];
    __shared__ float4 total[GROUPS > 1 ? 2 * kWide / 4 : 1];
    const int lane = static_cast<int>(threadIdx.x) & (LANES - 1), group = static_cast<int>(threadIdx.x) / LANES;
    const int plane = static_cast<int>(blockIdx.y), wave = static_cast<int>(threadIdx.x) >> 6;
    const int64_t w0 = static_cast<int64_t>(plane) * n;
    const Place<T, LANES, SLOTS> place(n, lane);
    const float per = 1.f / static_cast<float>(n);
    constexpr bool kKeep = SLOTS * N <= 16 && SLOTS < 4;       // the weights stay in registers, where there is room for them
    float kept[kKeep ? SLOTS : 1][N], dw[SLOTS][N] = {}, db[SLOTS][N] = {};
    const auto load_weights = [&](const float *from, int k, float (&w)[N]) {
#pragma unroll
        for (int q = 0; q < N; ++q) w[q] = 1.f;
        if (from) rn_beside(from + w0, place, k, w);
    };
    if constexpr (kKeep)
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) load_weights(weight, k, kept[k]);
    constexpr bool kFloats = sizeof(T) == 4 || SLOTS == 1;     // the slots as floats from the first pass to the second, where there is room for them
    struct Row {
        Held<T, SLOTS> xs, ds;
        float m, r;
    };
    int turn = 0;
    const auto load_row = [&](Row &row, int64_t b) {       // beyond the last: the last once more
        const int64_t at = min(b, static_cast<int64_t>(rows) - 1) * planes + plane;
        rn_hold<T, LANES, SLOTS, STREAM>(row.xs, x + at * n, place);
        rn_hold<T, LANES, SLOTS, STREAM>(row.ds, dy + at * n, place);
        row.m = mean[at];
        row.r = rstd[at];
    };
    const auto use_row = [&](Row &row, int64_t b) {
        const float m = row.m, r = row.r;
        const float *again = weight;
        if constexpr (!kKeep) asm volatile("" : "+s"(again));       // or the loads are moved out of the loop, into registers that are not there
        float xf[SLOTS][N], df[SLOTS][N];                           // x - m and dy
        const auto widen = [&] {
#pragma unroll
            for (int k = 0; k < SLOTS; ++k)
#pragma unroll
                for (int q = 0; q < N; ++q) {
                    xf[k][q] = static_cast<float>(row.xs[k][q]) - m;
                    df[k][q] = static_cast<float>(row.ds[k][q]);
                }
        };
        widen();
        float s[3] = {0.f, 0.f, 0.f};       // of g, g (x - m), x - m
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) {
            if constexpr (!kKeep) load_weights(again, k, kept[0]);
            const float (&w)[N] = kept[kKeep ? k : 0];
            if (k == SLOTS - 1 && (LANES == 4 || place.mixed)) {
#pragma unroll
                for (int q = 0; q < N; ++q) {
                    const bool count = place.counts(k, q);
                    const float g = count ? df[k][q] * w[q] : 0.f, d = count ? xf[k][q] : 0.f;
                    s[0] += g;
                    s[1] = fmaf(g, d, s[1]);
                    s[2] += d;
                }
            } else {
#pragma unroll
                for (int q = 0; q < N; ++q) {
                    const float g = df[k][q] * w[q];
                    s[0] += g;
                    s[1] = fmaf(g, xf[k][q], s[1]);
                    s[2] += xf[k][q];
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 3; ++i) s[i] = rn_lanes_sum<(LANES < 64 ? LANES : 64)>(s[i]);
        if constexpr (LANES > 64) {
            // two sets of places by turns: one barrier to a row
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int i = 0; i < 3; ++i) meet[turn][i][wave] = s[i];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 3; ++i) s[i] = rn_lanes_sum<16>(static_cast<int>(threadIdx.x & 15) < kWaves ? meet[turn][i][threadIdx.x & 15] : 0.f);
            turn ^= 1;
        }
        // dx = r (g - c1 - h c2)
        const float e = s[2] * r * per, c2 = r * fmaf(-e, s[0], s[1] * r) * per, c1 = r * s[0] * per;
        if constexpr (!kFloats) {
            rn_forget<T, SLOTS>(row.xs);
            rn_forget<T, SLOTS>(row.ds);
            widen();
        }
        T *to = dx + (b * planes + plane) * n;
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) {
            if constexpr (!kKeep) load_weights(again, k, kept[0]);
            const float (&w)[N] = kept[kKeep ? k : 0];
            float v[N];
#pragma unroll
            for (int q = 0; q < N; ++q) {
                const float h = fmaf(xf[k][q], r, -e);
                dw[k][q] = fmaf(df[k][q], h, dw[k][q]);
                db[k][q] += df[k][q];
                v[q] = fmaf(df[k][q] * r, w[q], fmaf(-h, c2, -c1));
            }
            rn_put<T, LANES, SLOTS, STREAM>(to, place, k, v);
        }
    };
    int64_t b = static_cast<int64_t>(blockIdx.x) * GROUPS + group;
    const int64_t stride = static_cast<int64_t>(gridDim.x) * GROUPS;
    if constexpr (kAhead) {
        Row one, two;
        if (b < rows) load_row(one, b);
        while (b < rows) {
            load_row(two, b + stride);
            use_row(one, b);
            b += stride;
            if (b >= rows) break;
            load_row(one, b + stride);
            use_row(two, b);
            b += stride;
        }
    } else {
        for (; b < rows; b += stride) {
            Row one;
            load_row(one, b);
            use_row(one, b);
        }
    }
    if (!part && !grad_w && !grad_b) return;
    if constexpr (GROUPS > 1) {
        // the groups add their sums in turn, each lane's own four at a time
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            if (group == g) {
#pragma unroll
                for (int k = 0; k < SLOTS; ++k)
#pragma unroll
                    for (int q = 0; q < N; q += 4) {
                        float4 &tw = total[((k * 2) * (N / 4) + q / 4) * LANES + lane], &tb = total[((k * 2 + 1) * (N / 4) + q / 4) * LANES + lane];
                        float4 aw = make_float4(dw[k][q], dw[k][q + 1], dw[k][q + 2], dw[k][q + 3]);
                        float4 ab = make_float4(db[k][q], db[k][q + 1], db[k][q + 2], db[k][q + 3]);
                        if (g > 0) {
                            const float4 ow = tw, ob = tb;
                            aw = make_float4(ow.x + aw.x, ow.y + aw.y, ow.z + aw.z, ow.w + aw.w);
                            ab = make_float4(ob.x + ab.x, ob.y + ab.y, ob.z + ab.z, ob.w + ab.w);
                        }
                        if (g < GROUPS - 1) {
                            tw = aw;
                            tb = ab;
                        } else {
                            dw[k][q] = aw.x; dw[k][q + 1] = aw.y; dw[k][q + 2] = aw.z; dw[k][q + 3] = aw.w;
                            db[k][q] = ab.x; db[k][q + 1] = ab.y; db[k][q + 2] = ab.z; db[k][q + 3] = ab.w;
                        }
                    }
            }
            __syncthreads();
        }
        if (group != GROUPS - 1) return;
    }
    const int64_t wide = rn_stride(static_cast<int64_t>(planes) * n);
    float *to_w = part ? part + 2 * wide * blockIdx.x + w0 : grad_w ? grad_w + w0 : nullptr;
    float *to_b = part ? part + 2 * wide * blockIdx.x + wide + w0 : grad_b ? grad_b + w0 : nullptr;
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
        if (k == SLOTS - 1 && !place.some) break;
        const int left = place.kTiny && place.tiny ? n : N;
        if (to_w) rk_store_f32<N>(to_w + place.at(k), left, dw[k]);
        if (to_b) rk_store_f32<N>(to_b + place.at(k), left, db[k]);
    }
}

// Rows too long for that: sums {sum g, sum g h', sum h'} of parts of a row first.  Pieces of kPart values in fp32, joined in fp64.
// grid (parts, R up to 2^15 and on)
template <class T>
__global__ __launch_bounds__(kNormThreads) void rn_backward_parts(const T *x, const T *dy, int64_t R, int planes, int n, int length,
                                                                  const float *__restrict__ weight, const float *__restrict__ mean,
                                                                  const float *__restrict__ rstd, float4 *__restrict__ sums)
{
    constexpr int N = kPerLoad<T>;
    __shared__ float meet[3][kNormThreads / 64];
    for (int64_t row = blockIdx.y; row < R; row += gridDim.y) {
        const float m = mean[row], r = rstd[row];
        const int64_t w0 = row % planes * n;
        const int from = static_cast<int>(blockIdx.x) * length, to = from + min(n - from, length);
        double total[3] = {0.0, 0.0, 0.0};
        for (int at = from; at < to; at += kPart<T>) {
            float s[3] = {0.f, 0.f, 0.f};
            rn_by_whole(at + kPart<T> <= n, [&](auto whole) {
                Held<T, kPartSlots> xs, ds;
                rn_piece<T, false>(xs, x + row * n, at, n, whole);
                rn_piece<T, false>(ds, dy + row * n, at, n, whole);
#pragma unroll
                for (int k = 0; k < kPartSlots; ++k) {
                    const int i = at + (k * kNormThreads + static_cast<int>(threadIdx.x)) * N;
                    float w[N];
#pragma unroll
                    for (int q = 0; q < N; ++q) w[q] = 1.f;
                    if (weight) {
                        if constexpr (whole) rk_load_f32<N>(weight + w0 + i, w);
                        else rk_load_f32_edge<N>(weight + w0, i, n, w);
                    }
#pragma unroll
                    for (int q = 0; q < N; ++q) {
                        // (beyond the row's end x is 0 and -m r may be infinite, its product with g = 0 a NaN)
                        const float h = whole || i + q < n ? (static_cast<float>(xs[k][q]) - m) * r : 0.f, g = static_cast<float>(ds[k][q]) * w[q];
                        s[0] += g;
                        s[1] = fmaf(g, h, s[1]);
                        s[2] += h;
                    }
                }
            });
            __syncthreads();        // the last piece's sums have been read
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                s[i] = rn_lanes_sum<64>(s[i]);
                if ((threadIdx.x & 63) == 0) meet[i][threadIdx.x >> 6] = s[i];
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 3; ++i)
#pragma unroll
                for (int v = 0; v < kNormThreads / 64; ++v) total[i] += static_cast<double>(meet[i][v]);
        }
        if (threadIdx.x == 0)
            sums[row * gridDim.x + blockIdx.x] = make_float4(static_cast<float>(total[0]), static_cast<float>(total[1]), static_cast<float>(total[2]), 0.f);
    }
}

// Then a workgroup has kNormThreads * N columns of a plane and `per` of its rows: dx there, and the columns' sums over those rows.
// grid (column tiles, planes, parts of the rows), the last rows first: they were read last
// (loads and stores as in rn_forward_apply: 4,000 x 30,000 fp32 472 us, so 421; 256 x 30,000 34, and would be 38 if x and dy were not kept)
constexpr int kRowsAtOnce = kNormThreads / 4;
template <class T, bool ONCE>
__global__ __launch_bounds__(kNormThreads) void rn_backward_columns(const T *x, const T *dy, int rows, int planes, int n, int per, int parts,
                                                                    const float *__restrict__ weight, const float *__restrict__ mean,
                                                                    const float *__restrict__ rstd, const float4 *__restrict__ sums, T *dx,
                                                                    float *__restrict__ part)
{
    constexpr int N = kPerLoad<T>;
    __shared__ float4 rs[kRowsAtOnce];      // m, r, e, c2
    __shared__ float c1s[kRowsAtOnce];
    const int plane = blockIdx.y, z = static_cast<int>(gridDim.z - 1 - blockIdx.z);
    const int i = (static_cast<int>(blockIdx.x) * kNormThreads + static_cast<int>(threadIdx.x)) * N;
    const bool all = static_cast<int>(blockIdx.x + 1) * (kNormThreads * N) <= n;      // columns of the workgroup exist
    float w[N], dw[N] = {}, db[N] = {}, v[N];
#pragma unroll
    for (int q = 0; q < N; ++q) w[q] = 1.f;
    if (weight) rk_load_f32_edge<N>(weight + static_cast<int64_t>(plane) * n, i, n, w);
    const int from = z * per, to = static_cast<int>(min(static_cast<int64_t>(rows), static_cast<int64_t>(from) + per));
    for (int at = from; at < to; at += kRowsAtOnce) {
        const int some = min(to - at, kRowsAtOnce);
        __syncthreads();        // the last rows are done with
        {
            // four lanes to a row add the sums of its parts
            const int l = static_cast<int>(threadIdx.x) >> 2;
            double s[3] = {0.0, 0.0, 0.0};
            const int64_t row = (at + static_cast<int64_t>(min(l, some - 1))) * planes + plane;
            for (int p = static_cast<int>(threadIdx.x) & 3; p < parts; p += 4) {
                const float4 one = sums[row * parts + p];
                s[0] += static_cast<double>(one.x);
                s[1] += static_cast<double>(one.y);
                s[2] += static_cast<double>(one.z);
            }
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                s[k] += __shfl_xor(s[k], 1, 64);
                s[k] += __shfl_xor(s[k], 2, 64);
            }
            if (l < some && (threadIdx.x & 3) == 0) {
                const double e = s[2] / n;
                rs[l] = make_float4(mean[row], rstd[row], static_cast<float>(e), static_cast<float>((s[1] - e * s[0]) / n));
                c1s[l] = static_cast<float>(s[0] / n);
            }
        }
        __syncthreads();
        rn_by_whole(all, [&](auto whole) {
            for (int b = 0; b < some; ++b) {
                const float4 c = rs[b];
                const float c1 = c1s[b];
                const int64_t place = ((at + static_cast<int64_t>(b)) * planes + plane) * n;
                const auto xs = whole ? rk_load_slot<T, ONCE>(x + place + i) : rk_load_edge<T, ONCE, false>(x + place, i, n);
                const auto ds = whole ? rk_load_slot<T, ONCE>(dy + place + i) : rk_load_edge<T, ONCE, false>(dy + place, i, n);
#pragma unroll
                for (int q = 0; q < N; ++q) {
                    const float h = fmaf(static_cast<float>(xs[q]) - c.x, c.y, -c.z), d = static_cast<float>(ds[q]);
                    dw[q] = fmaf(d, h, dw[q]);
                    db[q] += d;
                    v[q] = c.y * (fmaf(-h, c.w, d * w[q]) - c1);
                }
                if (whole || i < n) rk_store<T, true>(dx + place + i, whole ? N : n - i, v);
            }
        });
    }
    if (!part || i >= n) return;
    const int64_t stride = rn_stride(static_cast<int64_t>(planes) * n);
    float *to_w = part + 2 * stride * z + static_cast<int64_t>(plane) * n + i;
    rk_store_f32<N>(to_w, n - i, dw);
    rk_store_f32<N>(to_w + stride, n - i, db);
}

// The gradients from the parts' sums, in their order: COLUMNS columns to a workgroup, 4 a lane, the parts dealt out to the
// kNormThreads / (COLUMNS / 4) lanes that a column then has; joined in fp64.
template <int COLUMNS>
__global__ __launch_bounds__(kNormThreads) void rn_backward_finish(const float *__restrict__ part, int parts, int64_t wide, float *__restrict__ dw,
                                                                   float *__restrict__ db)
{
    constexpr int kAcross = COLUMNS / 4, kDown = kNormThreads / kAcross;
    __shared__ double4 lds[kDown][kAcross];
    const int64_t stride = rn_stride(wide);
    const int down = threadIdx.x / kAcross;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * COLUMNS; first < 2 * stride; first += static_cast<int64_t>(gridDim.x) * COLUMNS) {
        const int64_t i = first + (threadIdx.x % kAcross) * 4;
        double4 s = {0.0, 0.0, 0.0, 0.0};
        if (i < 2 * stride)
#pragma unroll 4
            for (int p = down; p < parts; p += kDown) {
                const float4 v = *reinterpret_cast<const float4 *>(part + 2 * stride * p + i);
                s.x += static_cast<double>(v.x); s.y += static_cast<double>(v.y); s.z += static_cast<double>(v.z); s.w += static_cast<double>(v.w);
            }
        __syncthreads();        // the last columns have been read
        lds[down][threadIdx.x % kAcross] = s;
        __syncthreads();
        if (threadIdx.x >= COLUMNS) continue;
        const int64_t at = first + threadIdx.x;
        double t = 0.0;
#pragma unroll
        for (int k = 0; k < kDown; ++k) t += reinterpret_cast<const double *>(&lds[k][threadIdx.x / 4])[threadIdx.x % 4];
        if (at < wide) {
            if (dw) dw[at] = static_cast<float>(t);
        } else if (at >= stride && at < stride + wide) {
            if (db) db[at - stride] = static_cast<float>(t);
        }
    }
}

inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }

constexpr int32_t kMostPlanes = 65535;        // a launch's second dimension
constexpr int32_t kMostValues = 1 << 30;      // of a row: its slots' numbers stay within 32 bits
constexpr int64_t kMostGroups = 1 << 20;      // of a launch (its lanes must be fewer than 2^32)

template <int V>
using Int = std::integral_constant<int, V>;

// x and y are streamed, not kept by the caches, where they are more than those hold and their rows are whole cache lines but
// for a few: 65,536 x 2,048 bf16 102 us, so 97; 1,000,000 x 64 bf16 49, so 46; but 256 x 3 x 10,000 fp32 (62 MB) 13.3, and would be 15.7;
// 2,000,000 x 3 x 16 fp32 138, and 147.  Fewer than kTwoRows rows of 65 loads to 4,096 are kept whatever their bytes (2,000 x 16,384 fp32 51.4 us,
// streamed 50.6; 1,900 x 32,768 bf16 50.5 and 48.8).
constexpr double kKeptBytes = 192 << 20;
// From so many rows on, those of all planes counted, a group of lanes takes two examples of a plane, whose weights it then loads once:
// 60,001 x 3 x 1,537 bf16 297 us, so 240; 16,384 x 2 x 10,000 fp32 508, so 482.  Fewer rows are taken one by one (700 x 3 x 1,000 fp32, 2,100 rows of 700
// examples: 5.4 us, one by one 4.5).  Rows of up to 64 loads are taken four examples at a time however few they are (1,000 x 256 fp32
// 3.2 us, one by one 2.3).
constexpr int64_t kTwoRows = 2048;
// How a row is held: in registers as long as kMostSlots loads of 1,024 lanes hold it, else in parts.  Of more than kFewSlots only if there
// is a row for each CU: 500 x 125,000 bf16 74.5 us in parts, 57 so; 1,000 x 65,000 fp32 142 and 114; but 64 x 100,000 f16 16 and 19.6.
constexpr int kMostSlots = 16, kFewSlots = 8, kCus = 256;
struct ForwardPlan {
    int64_t R;
    int parts = 0, length = 0;
    bool once = false;
    ForwardPlan(int32_t rows, int32_t planes, int32_t n, int32_t dtype) : R(static_cast<int64_t>(rows) * planes)
    {
        const int64_t size = static_cast<int64_t>(rk_type_bytes(dtype)), per = 16 / size, row = n * size;
        once = 2.0 * static_cast<double>(R) * static_cast<double>(row) > kKeptBytes && (row % 128 == 0 || row >= 16384);
        if (n <= (R < kCus ? kFewSlots : kMostSlots) * 1024 * per) return;
        const int64_t piece = kNormThreads * kPartSlots * per;
        const int64_t pieces = (n + piece - 1) / piece, each = (pieces + kMostParts - 1) / kMostParts;
        parts = static_cast<int>((pieces + each - 1) / each);
        length = static_cast<int>(each * piece);
    }
    size_t bytes() const { return up256(static_cast<size_t>(R) * static_cast<size_t>(parts) * sizeof(float4)); }
};

// One pass of the backward pass streams x, dy and dx where they are more than this: 677 x 2 x 10,000 fp32 (162 MB) 43 us, so 40.5, 65,536 x 2,048
// bf16 159 and 149, but 400 x 10,000 fp32 (48 MB) 19.6, and would be 22, 5,000 x 1,000 18.3 and 20.5.  Rows of four lanes are never streamed: several
// share a cache line, and where planes lie between them that costs (3,000,000 x 2 x 13 fp32 309 us, streamed 439; 3,000,000 x 16 114 and 106).
constexpr double kHeldKeptBytes = 128 << 20;

// The backward pass.  `lanes` x `slots` hold a row (0: rows are too long and go in two passes); the rows of a plane are dealt out
// to `parts` workgroups.
struct BackwardPlan {
    int64_t R, wide;
    int lanes = 0, slots = 0, parts = 1;
    int most_parts = 1;                           // of as many rows or fewer
    int row_parts = 0, length = 0, per = 0;       // two passes: parts of a row, their length; rows of a part
    bool once = false;                            // nothing is kept by the caches; of two passes: for the second
    BackwardPlan(int32_t rows, int32_t planes, int32_t n, int32_t dtype) : R(static_cast<int64_t>(rows) * planes), wide(static_cast<int64_t>(planes) * n)
    {
        const int64_t per_load = 16 / static_cast<int64_t>(rk_type_bytes(dtype)), loads = (n + per_load - 1) / per_load;
        const auto take = [&](int l, int s) { lanes = l, slots = s; };
        if (loads <= 4) take(4, 1);
        else if (loads <= 8) take(8, 1);
        else if (loads <= 16) take(16, 1);
        else if (loads <= 32) take(32, 1);
        else if (loads <= 64) take(64, 1);
        else if (loads <= 128) take(64, 2);
        else if (loads <= 256) take(256, 1);
        else if (loads <= 512) take(512, 1);
        else if (loads <= 1024) take(1024, 1);
        else if (loads <= 2048) take(1024, 2);
        else if (loads <= 5 * 1024 && dtype == ROCKET_F32) take(1024, static_cast<int>((loads + 1023) / 1024));
        const double bytes = static_cast<double>(R) * n * static_cast<double>(rk_type_bytes(dtype));
        if (lanes > 0) {
            once = 3.0 * bytes > kHeldKeptBytes;
            const int groups = lanes < 256 ? 256 / lanes : 1, threads = lanes < 256 ? 256 : lanes;
            const int64_t turns = (static_cast<int64_t>(rows) + groups - 1) / groups;      // of all groups together
            // a workgroup of 1,024 lanes to a CU, or four of 256; fewer where a wavefront has two slots of each row in flight: 100,000 x 2 x 500
            // fp32 257 us, so 215
            const int64_t most = std::max<int64_t>(1, (lanes <= 64 ? 256 / slots : 256) * 1024 / threads / planes);
            // a few turns of one workgroup take less than the second launch (2 x 500 fp32, 32 examples: 10.3 us, with it 12.3; 64: 17.4 and 12.2;
            // 2 x 10,000, 4 examples: 11 and 13.5, 16: 45 and 13)
            parts = most_parts = static_cast<int>(std::min(most, turns <= (lanes <= 64 || slots == 1 ? 8 : 4) ? 1 : turns));
            if (parts > 1) parts = static_cast<int>((turns + (turns + parts - 1) / parts - 1) / ((turns + parts - 1) / parts));     // all take as many turns
            return;
        }
        once = 2.0 * bytes > kKeptBytes;
        const int64_t piece = kNormThreads * kPartSlots * per_load, pieces = (n + piece - 1) / piece, each = (pieces + kMostParts - 1) / kMostParts;
        row_parts = static_cast<int>((pieces + each - 1) / each);
        length = static_cast<int>(each * piece);
        const int64_t tiles = (n + kNormThreads * per_load - 1) / (kNormThreads * per_load) * planes;
        const int64_t want = std::min<int64_t>(std::max<int64_t>(1, 2048 / tiles), 4096);
        per = static_cast<int>(std::max<int64_t>(8, (rows + want - 1) / want));
        parts = static_cast<int>((static_cast<int64_t>(rows) + per - 1) / per);
        most_parts = static_cast<int>(std::min(want, (static_cast<int64_t>(rows) + 7) / 8));
    }
    size_t sums_bytes() const { return up256(static_cast<size_t>(R) * static_cast<size_t>(row_parts) * sizeof(float4)); }
    size_t part_bytes(int count) const { return row_parts == 0 && count == 1 ? 0 : up256(static_cast<size_t>(2 * count) * static_cast<size_t>(rn_stride(wide)) * 4); }
    size_t bytes() const { return std::max<size_t>(256, sums_bytes() + part_bytes(parts)); }
    size_t most_bytes() const { return std::max<size_t>(256, sums_bytes() + part_bytes(most_parts)); }
};

// f(Int<v>) where v is one of FROM .. TO
template <int FROM, int TO, class F>
void by_number(int v, F f)
{
    if (v == FROM) f(Int<FROM>());
    else if constexpr (FROM < TO) by_number<FROM + 1, TO>(v, f);
}

template <class F>
void by_kept(bool once, F f)
{
    if (once) f(std::true_type());
    else f(std::false_type());
}

template <class F>
void by_type(int32_t dtype, F f)
{
    if (dtype == ROCKET_F32) f(float());
    else if (dtype == ROCKET_BF16) f(rk_bf16());
    else f(rk_f16());
}

bool misaligned(const void *p, int32_t dtype) { return reinterpret_cast<uintptr_t>(p) % rk_type_bytes(dtype) != 0; }

}  // namespace

extern "C" size_t rocket_layer_norm_workspace_bytes(int32_t rows, int32_t planes, int32_t n, int backward)
{
    if (rows < 1 || planes < 1 || n < 1 || planes > kMostPlanes || n > kMostValues) return 0;
    // the call's element type is not known here (fp32 rows take the most parts), and its rows may be fewer: the last batch of many
    if (backward) return std::max(BackwardPlan(rows, planes, n, ROCKET_F32).most_bytes(), BackwardPlan(rows, planes, n, ROCKET_BF16).most_bytes());
    const int32_t few = std::min(rows, (kCus - 1) / planes);      // that leave CUs without a row may go in parts where more do not
    return std::max(ForwardPlan(rows, planes, n, ROCKET_F32).bytes(), few > 0 ? ForwardPlan(few, planes, n, ROCKET_F32).bytes() : 0);
}

extern "C" int rocket_layer_norm(const void *x_dev, int32_t dtype, int32_t rows, int32_t planes, int32_t n, const float *weight_dev,
                                 const float *bias_dev, float eps, void *y_dev, float *mean_dev, float *rstd_dev, void *ws,
                                 size_t ws_bytes, void *hip_stream)
{
    if (!x_dev || !y_dev) return rk_fail(ROCKET_EINVAL, "rocket_layer_norm: NULL pointer");
    if (!rk_type_known(dtype)) return rk_fail(ROCKET_EINVAL, "rocket_layer_norm: unknown element type");
    if (rows < 1 || planes < 1 || n < 1 || planes > kMostPlanes || n > kMostValues)
        return rk_fail(ROCKET_EINVAL, "rocket_layer_norm: rows, planes and n must be >= 1, planes <= 65535, n <= 2^30");
    if (!std::isfinite(eps) || !(eps > 0.f)) return rk_fail(ROCKET_EINVAL, "rocket_layer_norm: eps must be positive and finite");
    if (!mean_dev != !rstd_dev) return rk_fail(ROCKET_EINVAL, "rocket_layer_norm: mean and rstd go together");
    if (misaligned(x_dev, dtype) || misaligned(y_dev, dtype)) return rk_fail(ROCKET_EINVAL, "rocket_layer_norm: x or y is not at an element's address");
    const ForwardPlan plan(rows, planes, n, dtype);
    if (plan.parts > 0 && (!ws || ws_bytes < plan.bytes() || reinterpret_cast<uintptr_t>(ws) % 16 != 0))
        return rk_fail(ROCKET_EWORKSPACE, "rocket_layer_norm: an aligned workspace of " + std::to_string(plan.bytes()) + " bytes required");
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    by_type(dtype, [&](auto t) {
        using T = decltype(t);
        const T *x = static_cast<const T *>(x_dev);
        T *y = static_cast<T *>(y_dev);
        const auto launch = [&](auto lanes, auto slots, auto rows_at_once, auto once) {
            constexpr int L = decltype(lanes)::value, S = decltype(slots)::value, J = decltype(rows_at_once)::value, kGroups = L < 256 ? 256 / L : 1;
            // examples of a launch: its groups of lanes are fewer than 2^32, and so are its lanes
            const int64_t most = kMostGroups * kGroups / planes * J;
            for (int64_t first = 0; first < rows; first += most) {
                const int64_t end = std::min<int64_t>(rows, first + most), groups = (end - first + J - 1) / J * planes;
                hipLaunchKernelGGL((rn_forward<T, L, S, J, decltype(once)::value>), dim3(static_cast<unsigned>((groups + kGroups - 1) / kGroups)), dim3(L < 256 ? 256 : L), 0,
                                   stream, x, static_cast<int>(first), static_cast<int>(end), planes, n, weight_dev, bias_dev, eps, y, mean_dev, rstd_dev);
            }
        };
        const int64_t loads = (n + kPerLoad<T> - 1) / kPerLoad<T>;      // of 16 bytes in a row
        if (plan.parts == 0) {
            // lanes to a row, slots, rows at a time: with one slot fewer, or fewer lanes, the row would not fit
            const int s64 = static_cast<int>((loads + 63) / 64), s256 = static_cast<int>((loads + 255) / 256), s1024 = static_cast<int>((loads + 1023) / 1024);
            const auto held = [&](auto lanes, auto slots, auto rows_at_once) {
                if constexpr (decltype(lanes)::value > 4) by_kept(plan.once, [&](auto once) { launch(lanes, slots, rows_at_once, once); });
                else launch(lanes, slots, rows_at_once, std::false_type());       // such rows are no whole lines
            };
            const auto pick = [&](auto lanes, auto slots) {
                plan.R >= kTwoRows ? held(lanes, slots, Int<2>()) : launch(lanes, slots, Int<1>(), std::false_type());
            };
            if (loads <= 4) held(Int<4>(), Int<1>(), Int<4>());
            else if (loads <= 8) held(Int<8>(), Int<1>(), Int<4>());
            else if (loads <= 16) held(Int<16>(), Int<1>(), Int<4>());
            else if (loads <= 32) held(Int<32>(), Int<1>(), Int<4>());
            else if (s64 == 1) held(Int<64>(), Int<1>(), Int<4>());
            else if (s64 <= 4) by_number<2, 4>(s64, [&](auto slots) { pick(Int<64>(), slots); });
            else if (s256 <= 4) by_number<2, 4>(s256, [&](auto slots) { pick(Int<256>(), slots); });
            else if (s1024 <= 4) by_number<2, 4>(s1024, [&](auto slots) { pick(Int<1024>(), slots); });
            else by_number<5, kMostSlots>(s1024, [&](auto slots) { held(Int<1024>(), slots, Int<1>()); });
        } else {
            float4 *moments = static_cast<float4 *>(ws);
            const unsigned tall = static_cast<unsigned>(std::min<int64_t>(plan.R, 32768));
            hipLaunchKernelGGL(rn_forward_parts<T>, dim3(static_cast<unsigned>(plan.parts), tall), dim3(kNormThreads), 0, stream, x, plan.R, n, plan.length,
                               moments);
            by_kept(plan.once, [&](auto once) {
                hipLaunchKernelGGL((rn_forward_apply<T, decltype(once)::value>), dim3(static_cast<unsigned>((n + int64_t{kPart<T>} - 1) / kPart<T>), tall),
                                   dim3(kNormThreads), 0, stream, x, plan.R, planes, n, plan.parts, moments, weight_dev, bias_dev, eps, y,
                                   mean_dev, rstd_dev);
            });
        }
    });
    return hipGetLastError() == hipSuccess ? ROCKET_OK : rk_fail(ROCKET_EHIP, "launch of the layer norm kernel failed");
}

extern "C" int rocket_layer_norm_backward(const void *x_dev, const void *grad_y_dev, int32_t dtype, int32_t rows, int32_t planes, int32_t n,
                                          const float *weight_dev, const float *mean_dev, const float *rstd_dev, void *grad_x_dev,
                                          float *grad_weight_dev, float *grad_bias_dev, void *ws, size_t ws_bytes, void *hip_stream)
{
    if (!x_dev || !grad_y_dev || !mean_dev || !rstd_dev || !grad_x_dev) return rk_fail(ROCKET_EINVAL, "rocket_layer_norm_backward: NULL pointer");
    if (!rk_type_known(dtype)) return rk_fail(ROCKET_EINVAL, "rocket_layer_norm_backward: unknown element type");
    if (rows < 1 || planes < 1 || n < 1 || planes > kMostPlanes || n > kMostValues)
        return rk_fail(ROCKET_EINVAL, "rocket_layer_norm_backward: rows, planes and n must be >= 1, planes <= 65535, n <= 2^30");
    if (misaligned(x_dev, dtype) || misaligned(grad_y_dev, dtype) || misaligned(grad_x_dev, dtype))
        return rk_fail(ROCKET_EINVAL, "rocket_layer_norm_backward: x, grad_y or grad_x is not at an element's address");
    const BackwardPlan plan(rows, planes, n, dtype);
    if (!ws || ws_bytes < plan.bytes() || reinterpret_cast<uintptr_t>(ws) % 16 != 0)
        return rk_fail(ROCKET_EWORKSPACE, "rocket_layer_norm_backward: an aligned workspace of " + std::to_string(plan.bytes()) + " bytes required");
    const bool sums_wanted = grad_weight_dev || grad_bias_dev;
    float4 *sums = static_cast<float4 *>(ws);
    float *part = sums_wanted && plan.part_bytes(plan.parts) > 0 ? reinterpret_cast<float *>(static_cast<char *>(ws) + plan.sums_bytes()) : nullptr;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    by_type(dtype, [&](auto t) {
        using T = decltype(t);
        const T *x = static_cast<const T *>(x_dev), *dy = static_cast<const T *>(grad_y_dev);
        T *dx = static_cast<T *>(grad_x_dev);
        const auto held = [&](auto lanes, auto slots) {
            constexpr int L = decltype(lanes)::value, S = decltype(slots)::value, G = L < 256 ? 256 / L : 1;
            if (plan.lanes != L || plan.slots != S) return;
            const auto run = [&](auto once) {
                hipLaunchKernelGGL((rn_backward<T, L, S, G, decltype(once)::value>), dim3(static_cast<unsigned>(plan.parts), static_cast<unsigned>(planes)),
                                   dim3(L * G), 0, stream, x, dy, rows, planes, n, weight_dev, mean_dev, rstd_dev, dx, part, grad_weight_dev, grad_bias_dev);
            };
            if constexpr (L > 4) by_kept(plan.once, run);
            else run(std::false_type());
        };
        held(Int<4>(), Int<1>());
        held(Int<8>(), Int<1>());
        held(Int<16>(), Int<1>());
        held(Int<32>(), Int<1>());
        held(Int<64>(), Int<1>());
        held(Int<64>(), Int<2>());
        held(Int<256>(), Int<1>());
        held(Int<512>(), Int<1>());
        held(Int<1024>(), Int<1>());
        held(Int<1024>(), Int<2>());
        if constexpr (sizeof(T) == 4) {
            held(Int<1024>(), Int<3>());
            held(Int<1024>(), Int<4>());
            held(Int<1024>(), Int<5>());
        }
        if (plan.row_parts > 0) {
            hipLaunchKernelGGL(rn_backward_parts<T>, dim3(static_cast<unsigned>(plan.row_parts), static_cast<unsigned>(std::min<int64_t>(plan.R, 32768))),
                               dim3(kNormThreads), 0, stream, x, dy, plan.R, planes, n, plan.length, weight_dev, mean_dev, rstd_dev, sums);
            const unsigned tiles = static_cast<unsigned>((n + int64_t{kNormThreads * kPerLoad<T>} - 1) / (kNormThreads * kPerLoad<T>));
            by_kept(plan.once, [&](auto once) {
                hipLaunchKernelGGL((rn_backward_columns<T, decltype(once)::value>), dim3(tiles, static_cast<unsigned>(planes), static_cast<unsigned>(plan.parts)),
                                   dim3(kNormThreads), 0, stream, x, dy, rows, planes, n, plan.per, plan.row_parts, weight_dev, mean_dev, rstd_dev, sums, dx,
                                   part);
            });
        }
        if (part) {
            const int64_t floats = 2 * rn_stride(plan.wide);
            if (floats >= 64 * 512)
                hipLaunchKernelGGL(rn_backward_finish<64>, dim3(static_cast<unsigned>(std::min(kMostGroups, (floats + 63) / 64))), dim3(kNormThreads), 0, stream, part, plan.parts,
                                   plan.wide, grad_weight_dev, grad_bias_dev);
            else
                hipLaunchKernelGGL(rn_backward_finish<16>, dim3(static_cast<unsigned>((floats + 15) / 16)), dim3(kNormThreads), 0, stream, part, plan.parts,
                                   plan.wide, grad_weight_dev, grad_bias_dev);
        }
    });
    return hipGetLastError() == hipSuccess ? ROCKET_OK : rk_fail(ROCKET_EHIP, "launch of the layer norm's backward kernels failed");
}
