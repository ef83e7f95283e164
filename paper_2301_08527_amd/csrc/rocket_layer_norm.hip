// Layer norm of feature planes for MI355X (gfx950), forward and backward.  See include/rocket.h for the contract.
//
// A row is one plane of one example: R = rows * planes rows of n values, row i has the weights of plane i % planes.
//   forward   m = mean x, v = mean (x - m)^2, r = 1/sqrt(v + eps), y = (x - m) r w + b
//   backward  g = dy w, h = (x - m) r:  dx = r (g - mean g - h mean(g h)),  dw = sum dy h,  db = sum dy (over the rows of a plane)
// Both are bound by memory: some ten operations a value.
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

// Sum over 16 or 64 neighbouring lanes, the same bits on each of them: rotations within the rows of 16 lanes, then the
// rows' sums one after the other into the last row.
template <int LANES>
__device__ __forceinline__ float rn_lanes_sum(float v)
{
    static_assert(LANES == 16 || LANES == 64, "a row of lanes or a wavefront");
    v += rn_dpp<0x128, 0xf>(v);       // row_ror:8, 4, 2, 1
    v += rn_dpp<0x124, 0xf>(v);
    v += rn_dpp<0x122, 0xf>(v);
    v += rn_dpp<0x121, 0xf>(v);
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

// Of all values that the LANES lanes of a row hold in `raw`.  `left[s]` values of slot s exist, `n` of all lanes.
template <class T, int SLOTS>
using Held = typename RkSlot<T>::V[SLOTS];

template <class T, int LANES, int SLOTS>
__device__ __forceinline__ Moments rn_moments(const Held<T, SLOTS> &raw, int i0, int step, int n, float count)
{
    constexpr int N = kPerLoad<T>;
    float s = 0.f;        // values that do not exist are zeros
#pragma unroll
    for (int k = 0; k < SLOTS; ++k)
#pragma unroll
        for (int q = 0; q < N; ++q) s += static_cast<float>(raw[k][q]);
    const float shift = rn_lanes_sum<LANES>(s) / count;
    float d1 = 0.f, d2 = 0.f;
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
        const int left = n - (i0 + k * step);
        if (left >= N) {
#pragma unroll
            for (int q = 0; q < N; ++q) {
                const float d = static_cast<float>(raw[k][q]) - shift;
                d1 += d;
                d2 = fmaf(d, d, d2);
            }
        } else if (left > 0) {
#pragma unroll
            for (int q = 0; q < N; ++q) {
                const float d = q < left ? static_cast<float>(raw[k][q]) - shift : 0.f;
                d1 += d;
                d2 = fmaf(d, d, d2);
            }
        }
    }
    d1 = rn_lanes_sum<LANES>(d1);
    d2 = rn_lanes_sum<LANES>(d2);
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

template <class T, int SLOTS>
__device__ __forceinline__ void rn_hold(Held<T, SLOTS> &raw, const T *src, int i0, int step, int n)
{
    constexpr int N = kPerLoad<T>;
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
        const int i = i0 + k * step;
        if (i + N <= n) {
            raw[k] = reinterpret_cast<const RkSlot<T> *>(src + i)->v;
        } else {
#pragma unroll
            for (int q = 0; q < N; ++q) raw[k][q] = i + q < n ? src[i + q] : static_cast<T>(0.f);
        }
    }
}

template <class T, int SLOTS>
__device__ __forceinline__ void rn_write(const Held<T, SLOTS> &raw, T *dst, int i0, int step, int n, const Moments &m, float r, const float *weight,
                                         const float *bias)
{
    constexpr int N = kPerLoad<T>;
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
        const int i = i0 + k * step;
        if (i >= n) break;
        float v[N], w[N], b[N];
#pragma unroll
        for (int q = 0; q < N; ++q) w[q] = 1.f, b[q] = 0.f;
        if (weight) rk_load_f32<N>(weight + i, n - i, w);
        if (bias) rk_load_f32<N>(bias + i, n - i, b);
#pragma unroll
        for (int q = 0; q < N; ++q) v[q] = fmaf(((static_cast<float>(raw[k][q]) - m.shift) - m.rest) * r, w[q], b[q]);
        rk_store(dst + i, n - i, v);
    }
}

// n as a float: exact up to 2^24, and a rounding of 2^-25 of the mean of squares beyond
__device__ __forceinline__ float rn_rstd(const Moments &m, float eps) { return 1.f / sqrtf(m.m2 / m.count + eps); }

// A row lies in the registers of LANES lanes, SLOTS loads of 16 bytes in each (as loaded: 16-bit values take half the registers),
// so x is read once.  Two passes over the registers give the mean and the distances from it; up to 64 lanes meet by lane
// rotations alone, more lanes once through LDS, where the wavefronts' own means and sums of squares are joined.
template <class T, int LANES, int SLOTS>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void rn_forward(const T *x, int64_t R, int planes, int n, const float *__restrict__ weight,
                                                                        const float *__restrict__ bias, float eps, T *y,
                                                                        float *__restrict__ mean, float *__restrict__ rstd)
{
    constexpr int N = kPerLoad<T>, kRows = LANES < 256 ? 256 / LANES : 1;
    __shared__ float4 lds[LANES > 64 ? 16 : 1];
    const int lane = static_cast<int>(threadIdx.x) & (LANES - 1), i0 = lane * N, step = LANES * N;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / LANES;
    if (row >= R) return;
    Held<T, SLOTS> raw;
    rn_hold<T, SLOTS>(raw, x + row * n, i0, step, n);
    Moments m;
    if constexpr (LANES <= 64) {
        m = rn_moments<T, LANES, SLOTS>(raw, i0, step, n, static_cast<float>(n));
    } else {
        const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
        int count = 0;
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) count += min(max(n - (k * step + wave * 64 * N), 0), 64 * N);
        const Moments own = rn_moments<T, 64, SLOTS>(raw, i0, step, n, static_cast<float>(max(count, 1)));
        if (static_cast<int>(threadIdx.x) < 16) lds[threadIdx.x] = make_float4(0.f, 0.f, 0.f, 0.f);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) lds[wave] = make_float4(static_cast<float>(count), own.shift, own.rest, own.m2);
        __syncthreads();
        const float4 part = lds[threadIdx.x & 15];
        m = rn_join({part.x, part.y, part.z, part.w}, static_cast<float>(n));
    }
    const float r = rn_rstd(m, eps);
    const int64_t w0 = row % planes * n;
    rn_write<T, SLOTS>(raw, y + row * n, i0, step, n, m, r, weight ? weight + w0 : nullptr, bias ? bias + w0 : nullptr);
    if (mean && lane == 0) {
        mean[row] = m.shift + m.rest;
        rstd[row] = r;
    }
}

// Longer rows: moments of parts of a row, one workgroup each, then each part again with those of its row joined.  At most kMostParts
// parts to a row; a part is `length` values, in pieces of kPart that a workgroup holds.  grid (parts, R up to 2^15 and on)
constexpr int kMostParts = 64, kPartSlots = 4;
template <class T>
constexpr int kPart = kNormThreads * kPartSlots * kPerLoad<T>;

template <class T>
__global__ __launch_bounds__(kNormThreads) void rn_forward_parts(const T *x, int64_t R, int n, int length, float4 *__restrict__ moments)
{
    constexpr int N = kPerLoad<T>;
    __shared__ float4 lds[16];
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
    for (int64_t row = blockIdx.y; row < R; row += gridDim.y) {
        const int from = static_cast<int>(blockIdx.x) * length, to = min(n - from, length) + from;
        Moments m = {0.f, 0.f, 0.f, 0.f};
        for (int64_t at = from; at < to; at += kPart<T>) {
            const int some = static_cast<int>(min(static_cast<int64_t>(to) - at, static_cast<int64_t>(kPart<T>)));
            Held<T, kPartSlots> raw;
            rn_hold<T, kPartSlots>(raw, x + row * n + at, static_cast<int>(threadIdx.x) * N, kNormThreads * N, some);
            int count = 0;
#pragma unroll
            for (int k = 0; k < kPartSlots; ++k) count += min(max(some - (k * kNormThreads * N + wave * 64 * N), 0), 64 * N);
            const Moments own = rn_moments<T, 64, kPartSlots>(raw, static_cast<int>(threadIdx.x) * N, kNormThreads * N, some, static_cast<float>(max(count, 1)));
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

template <class T>
__global__ __launch_bounds__(kNormThreads) void rn_forward_apply(const T *x, int64_t R, int planes, int n, int length, int parts,
                                                                 const float4 *__restrict__ moments, const float *__restrict__ weight,
                                                                 const float *__restrict__ bias, float eps, T *y, float *__restrict__ mean,
                                                                 float *__restrict__ rstd)
{
    constexpr int N = kPerLoad<T>;
    for (int64_t row = blockIdx.y; row < R; row += gridDim.y) {
        const Moments m = rn_row_moments(moments + row * parts, parts);
        const float r = rn_rstd(m, eps);
        const int64_t w0 = row % planes * n;
        const int64_t from = static_cast<int64_t>(blockIdx.x) * kPart<T>;
        const int some = static_cast<int>(min(static_cast<int64_t>(n) - from, static_cast<int64_t>(kPart<T>)));
        Held<T, kPartSlots> raw;
        rn_hold<T, kPartSlots>(raw, x + row * n + from, static_cast<int>(threadIdx.x) * N, kNormThreads * N, some);
        rn_write<T, kPartSlots>(raw, y + row * n + from, static_cast<int>(threadIdx.x) * N, kNormThreads * N, some, m, r,
                                weight ? weight + w0 + from : nullptr, bias ? bias + w0 + from : nullptr);
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
template <class T, int LANES, int SLOTS, int GROUPS>
__global__ __launch_bounds__(LANES * GROUPS) void rn_backward(const T *x, const T *dy, int rows, int planes, int n, const float *__restrict__ weight,
                                                              const float *__restrict__ mean, const float *__restrict__ rstd, T *dx,
                                                              float *__restrict__ part, float *__restrict__ grad_w, float *__restrict__ grad_b)
{
    constexpr int N = kPerLoad<T>, kWaves = LANES > 64 ? LANES / 64 : 1, kWide = SLOTS * N * LANES;
    static_assert(LANES <= 64 || GROUPS == 1, "a row of several wavefronts has the workgroup to itself");
    __shared__ float meet[2][3][kWaves];
    __shared__ float4 total[GROUPS > 1 ? 2 * kWide / 4 : 1];
    const int lane = static_cast<int>(threadIdx.x) & (LANES - 1), group = static_cast<int>(threadIdx.x) / LANES, i0 = lane * N, step = LANES * N;
    const int plane = static_cast<int>(blockIdx.y), wave = static_cast<int>(threadIdx.x) >> 6;
    const float per = 1.f / static_cast<float>(n);
    constexpr bool kKeep = SLOTS < 5;       // the weights stay in registers, where there is room for them
    float kept[kKeep ? SLOTS : 1][N], dw[SLOTS][N] = {}, db[SLOTS][N] = {};
    const auto load_weights = [&](int i, float (&w)[N]) {
#pragma unroll
        for (int q = 0; q < N; ++q) w[q] = 1.f;
        if (weight && i < n) rk_load_f32<N>(weight + static_cast<int64_t>(plane) * n + i, n - i, w);
    };
    if constexpr (kKeep)
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) load_weights(i0 + k * step, kept[k]);
    int turn = 0;
    for (int64_t b = static_cast<int64_t>(blockIdx.x) * GROUPS + group; b < rows; b += static_cast<int64_t>(gridDim.x) * GROUPS, turn ^= 1) {
        const int64_t row = b * planes + plane;
        Held<T, SLOTS> xs, ds;
        rn_hold<T, SLOTS>(xs, x + row * n, i0, step, n);
        rn_hold<T, SLOTS>(ds, dy + row * n, i0, step, n);
        const float m = mean[row], r = rstd[row];
        float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) {
            const int left = n - (i0 + k * step);
            if constexpr (!kKeep) load_weights(i0 + k * step, kept[0]);
            const float (&w)[N] = kept[kKeep ? k : 0];
#pragma unroll
            for (int q = 0; q < N; ++q) {
                const float h = (static_cast<float>(xs[k][q]) - m) * r, g = static_cast<float>(ds[k][q]) * w[q];
                s[0] += g;
                s[1] = fmaf(g, h, s[1]);
                s[2] += q < left ? h : 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < 3; ++i) s[i] = rn_lanes_sum<LANES < 64 ? LANES : 64>(s[i]);
        if constexpr (LANES > 64) {
            // two sets of places by turns: one barrier to a row
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int i = 0; i < 3; ++i) meet[turn][i][wave] = s[i];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 3; ++i) s[i] = rn_lanes_sum<16>(static_cast<int>(threadIdx.x & 15) < kWaves ? meet[turn][i][threadIdx.x & 15] : 0.f);
        }
        const float c1 = s[0] * per, e = s[2] * per, c2 = fmaf(-e, s[0], s[1]) * per;
#pragma unroll
        for (int k = 0; k < SLOTS; ++k) {
            const int i = i0 + k * step;
            if constexpr (!kKeep) load_weights(i, kept[0]);
            const float (&w)[N] = kept[kKeep ? k : 0];
            float v[N];
#pragma unroll
            for (int q = 0; q < N; ++q) {
                const float h = fmaf(static_cast<float>(xs[k][q]) - m, r, -e), d = static_cast<float>(ds[k][q]);
                dw[k][q] = fmaf(d, h, dw[k][q]);
                db[k][q] += d;
                v[q] = r * (fmaf(-h, c2, d * w[q]) - c1);
            }
            if (i < n) rk_store(dx + row * n + i, n - i, v);
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
    const int64_t wide = static_cast<int64_t>(planes) * n, w0 = static_cast<int64_t>(plane) * n;
    float *to_w = part ? part + 2 * rn_stride(wide) * blockIdx.x + w0 : grad_w ? grad_w + w0 : nullptr;
    float *to_b = part ? part + 2 * rn_stride(wide) * blockIdx.x + rn_stride(wide) + w0 : grad_b ? grad_b + w0 : nullptr;
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
        const int i = i0 + k * step;
        if (i >= n) break;
        if (to_w) rk_store_f32<N>(to_w + i, n - i, dw[k]);
        if (to_b) rk_store_f32<N>(to_b + i, n - i, db[k]);
    }
}

// Rows too long for that: sums {sum g, sum g h', sum h'} of parts of a row first.  Pieces of kPart values in fp32, joined in fp64.
// grid (parts, R up to 2^15 and on)
template <class T>
__global__ __launch_bounds__(kNormThreads) void rn_backward_parts(const T *x, const T *dy, int64_t R, int planes, int n, int length,
                                                                  const float *__restrict__ weight, const float *__restrict__ mean,
                                                                  const float *__restrict__ rstd, float4 *__restrict__ sums)
{
    constexpr int N = kPerLoad<T>, kStep = kNormThreads * N;
    __shared__ float meet[3][kNormThreads / 64];
    for (int64_t row = blockIdx.y; row < R; row += gridDim.y) {
        const float m = mean[row], r = rstd[row];
        const int64_t w0 = row % planes * n;
        const int64_t from = static_cast<int64_t>(blockIdx.x) * length, to = min(static_cast<int64_t>(n), from + length);
        double total[3] = {0.0, 0.0, 0.0};
        for (int64_t at = from; at < to; at += kPart<T>) {
            const int some = static_cast<int>(min(to - at, static_cast<int64_t>(kPart<T>))), i0 = static_cast<int>(threadIdx.x) * N;
            Held<T, kPartSlots> xs, ds;
            rn_hold<T, kPartSlots>(xs, x + row * n + at, i0, kStep, some);
            rn_hold<T, kPartSlots>(ds, dy + row * n + at, i0, kStep, some);
            float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < kPartSlots; ++k) {
                const int i = i0 + k * kStep, left = some - i;
                float w[N];
#pragma unroll
                for (int q = 0; q < N; ++q) w[q] = 1.f;
                if (weight && left > 0) rk_load_f32<N>(weight + w0 + at + i, left, w);
#pragma unroll
                for (int q = 0; q < N; ++q) {
                    const float h = (static_cast<float>(xs[k][q]) - m) * r, g = static_cast<float>(ds[k][q]) * w[q];
                    s[0] += g;
                    s[1] = fmaf(g, h, s[1]);
                    s[2] += q < left ? h : 0.f;
                }
            }
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
constexpr int kRowsAtOnce = kNormThreads / 4;
template <class T>
__global__ __launch_bounds__(kNormThreads) void rn_backward_columns(const T *x, const T *dy, int rows, int planes, int n, int per, int parts,
                                                                    const float *__restrict__ weight, const float *__restrict__ mean,
                                                                    const float *__restrict__ rstd, const float4 *__restrict__ sums, T *dx,
                                                                    float *__restrict__ part)
{
    constexpr int N = kPerLoad<T>;
    __shared__ float4 rs[kRowsAtOnce];      // m, r, e, c2
    __shared__ float c1s[kRowsAtOnce];
    const int plane = blockIdx.y, z = static_cast<int>(gridDim.z - 1 - blockIdx.z);
    const int64_t i = (static_cast<int64_t>(blockIdx.x) * kNormThreads + static_cast<int>(threadIdx.x)) * N;
    float w[N], dw[N] = {}, db[N] = {}, v[N], d[N];
#pragma unroll
    for (int q = 0; q < N; ++q) w[q] = 1.f;
    if (weight && i < n) rk_load_f32<N>(weight + static_cast<int64_t>(plane) * n + i, n - i, w);
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
        if (i >= n) continue;
        for (int b = 0; b < some; ++b) {
            const float4 c = rs[b];
            const float c1 = c1s[b];
            const int64_t place = ((at + static_cast<int64_t>(b)) * planes + plane) * n + i;
            rk_load(x + place, n - i, v);
            rk_load(dy + place, n - i, d);
#pragma unroll
            for (int q = 0; q < N; ++q) {
                const float h = fmaf(v[q] - c.x, c.y, -c.z);
                dw[q] = fmaf(d[q], h, dw[q]);
                db[q] += d[q];
                v[q] = c.y * (fmaf(-h, c.w, d[q] * w[q]) - c1);
            }
            rk_store(dx + place, n - i, v);
        }
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
    const int64_t stride = rn_stride(wide), i = static_cast<int64_t>(blockIdx.x) * COLUMNS + (threadIdx.x % kAcross) * 4;
    const int down = threadIdx.x / kAcross;
    double4 s = {0.0, 0.0, 0.0, 0.0};
    if (i < 2 * stride)
#pragma unroll 4
        for (int p = down; p < parts; p += kDown) {
            const float4 v = *reinterpret_cast<const float4 *>(part + 2 * stride * p + i);
            s.x += static_cast<double>(v.x); s.y += static_cast<double>(v.y); s.z += static_cast<double>(v.z); s.w += static_cast<double>(v.w);
        }
    lds[down][threadIdx.x % kAcross] = s;
    __syncthreads();
    if (threadIdx.x >= COLUMNS) return;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * COLUMNS + threadIdx.x;
    double t = 0.0;
#pragma unroll
    for (int k = 0; k < kDown; ++k) t += reinterpret_cast<const double *>(&lds[k][threadIdx.x / 4])[threadIdx.x % 4];
    if (at < wide) {
        if (dw) dw[at] = static_cast<float>(t);
    } else if (at >= stride && at < stride + wide) {
        if (db) db[at - stride] = static_cast<float>(t);
    }
}

inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }

template <int V>
using Int = std::integral_constant<int, V>;

// How a row is held: in registers as long as 8 loads of 1,024 lanes hold it, else in parts.
struct ForwardPlan {
    int64_t R;
    int parts = 0, length = 0;
    ForwardPlan(int32_t rows, int32_t planes, int32_t n, int32_t dtype) : R(static_cast<int64_t>(rows) * planes)
    {
        const int64_t per = 16 / static_cast<int64_t>(rk_type_bytes(dtype));
        if (n <= 8 * 1024 * per) return;
        const int64_t piece = kNormThreads * kPartSlots * per;
        const int64_t pieces = (n + piece - 1) / piece, each = (pieces + kMostParts - 1) / kMostParts;
        parts = static_cast<int>((pieces + each - 1) / each);
        length = static_cast<int>(each * piece);
    }
    size_t bytes() const { return up256(static_cast<size_t>(R) * static_cast<size_t>(parts) * sizeof(float4)); }
};

// The backward pass.  `lanes` x `slots` hold a row (0: rows are too long and go in two passes); the rows of a plane are dealt out
// to `parts` workgroups.
struct BackwardPlan {
    int64_t R, wide;
    int lanes = 0, slots = 0, parts = 1;
    int row_parts = 0, length = 0, per = 0;       // two passes: parts of a row, their length; rows of a part
    BackwardPlan(int32_t rows, int32_t planes, int32_t n, int32_t dtype) : R(static_cast<int64_t>(rows) * planes), wide(static_cast<int64_t>(planes) * n)
    {
        const int64_t per_load = 16 / static_cast<int64_t>(rk_type_bytes(dtype)), loads = (n + per_load - 1) / per_load;
        const auto take = [&](int l, int s) { lanes = l, slots = s; };
        if (loads <= 16) take(16, 1);
        else if (loads <= 64) take(64, 1);
        else if (loads <= 128) take(64, 2);
        else if (loads <= 256) take(256, 1);
        else if (loads <= 512) take(256, 2);
        else if (loads <= 1024) take(512, 2);
        else if (loads <= 2048) take(1024, 2);
        else if (loads <= 4096 && dtype == ROCKET_F32) take(1024, 4);
        else if (loads <= 5120 && dtype == ROCKET_F32) take(1024, 5);
        if (lanes > 0) {
            const int groups = lanes < 256 ? 256 / lanes : 1, threads = lanes < 256 ? 256 : lanes;
            const int64_t turns = (static_cast<int64_t>(rows) + groups - 1) / groups;      // of all groups together
            const int64_t most = std::max<int64_t>(1, 256 * 1024 / threads / planes);
            parts = static_cast<int>(std::min(most, turns <= 16 ? 1 : turns));
            if (parts > 1) parts = static_cast<int>((turns + (turns + parts - 1) / parts - 1) / ((turns + parts - 1) / parts));     // all take as many turns
            return;
        }
        const int64_t piece = kNormThreads * kPartSlots * per_load, pieces = (n + piece - 1) / piece, each = (pieces + kMostParts - 1) / kMostParts;
        row_parts = static_cast<int>((pieces + each - 1) / each);
        length = static_cast<int>(each * piece);
        const int64_t tiles = (n + kNormThreads * per_load - 1) / (kNormThreads * per_load) * planes;
        const int64_t want = std::min<int64_t>(std::max<int64_t>(1, 2048 / tiles), 4096);
        per = static_cast<int>(std::max<int64_t>(8, (rows + want - 1) / want));
        parts = (rows + per - 1) / per;
    }
    size_t sums_bytes() const { return up256(static_cast<size_t>(R) * static_cast<size_t>(row_parts) * sizeof(float4)); }
    size_t part_bytes() const { return row_parts == 0 && parts == 1 ? 0 : up256(static_cast<size_t>(2 * parts) * static_cast<size_t>(rn_stride(wide)) * 4); }
    size_t bytes() const { return std::max<size_t>(256, sums_bytes() + part_bytes()); }
};

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
    if (rows < 1 || planes < 1 || n < 1) return 0;
    // the call's element type is not known here: fp32 rows take the most parts
    return backward ? std::max(BackwardPlan(rows, planes, n, ROCKET_F32).bytes(), BackwardPlan(rows, planes, n, ROCKET_BF16).bytes())
                    : ForwardPlan(rows, planes, n, ROCKET_F32).bytes();
}

extern "C" int rocket_layer_norm(const void *x_dev, int32_t dtype, int32_t rows, int32_t planes, int32_t n, const float *weight_dev,
                                 const float *bias_dev, float eps, void *y_dev, float *mean_dev, float *rstd_dev, void *ws,
                                 size_t ws_bytes, void *hip_stream)
{
    if (!x_dev || !y_dev) return rk_fail(ROCKET_EINVAL, "rocket_layer_norm: NULL pointer");
    if (!rk_type_known(dtype)) return rk_fail(ROCKET_EINVAL, "rocket_layer_norm: unknown element type");
    if (rows < 1 || planes < 1 || n < 1) return rk_fail(ROCKET_EINVAL, "rocket_layer_norm: rows, planes and n must be >= 1");
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
        const auto held = [&](auto lanes, auto slots) {
            constexpr int L = decltype(lanes)::value, S = decltype(slots)::value, kRows = L < 256 ? 256 / L : 1;
            hipLaunchKernelGGL((rn_forward<T, L, S>), dim3(static_cast<unsigned>((plan.R + kRows - 1) / kRows)), dim3(L < 256 ? 256 : L), 0, stream, x,
                               plan.R, planes, n, weight_dev, bias_dev, eps, y, mean_dev, rstd_dev);
        };
        const int64_t loads = (n + kPerLoad<T> - 1) / kPerLoad<T>;      // of 16 bytes in a row
        if (plan.parts == 0) {
            if (loads <= 16) held(Int<16>(), Int<1>());
            else if (loads <= 64) held(Int<64>(), Int<1>());
            else if (loads <= 128) held(Int<64>(), Int<2>());
            else if (loads <= 256) held(Int<64>(), Int<4>());
            else if (loads <= 512) held(Int<64>(), Int<8>());
            else if (loads <= 1024) held(Int<256>(), Int<4>());
            else if (loads <= 2048) held(Int<256>(), Int<8>());
            else if (loads <= 4096) held(Int<1024>(), Int<4>());
            else held(Int<1024>(), Int<8>());
        } else {
            float4 *moments = static_cast<float4 *>(ws);
            const unsigned tall = static_cast<unsigned>(std::min<int64_t>(plan.R, 32768));
            hipLaunchKernelGGL(rn_forward_parts<T>, dim3(static_cast<unsigned>(plan.parts), tall), dim3(kNormThreads), 0, stream, x, plan.R, n, plan.length,
                               moments);
            hipLaunchKernelGGL(rn_forward_apply<T>, dim3(static_cast<unsigned>((n + int64_t{kPart<T>} - 1) / kPart<T>), tall), dim3(kNormThreads), 0, stream, x,
                               plan.R, planes, n, plan.length, plan.parts, moments, weight_dev, bias_dev, eps, y, mean_dev, rstd_dev);
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
    if (rows < 1 || planes < 1 || n < 1) return rk_fail(ROCKET_EINVAL, "rocket_layer_norm_backward: rows, planes and n must be >= 1");
    if (misaligned(x_dev, dtype) || misaligned(grad_y_dev, dtype) || misaligned(grad_x_dev, dtype))
        return rk_fail(ROCKET_EINVAL, "rocket_layer_norm_backward: x, grad_y or grad_x is not at an element's address");
    if (planes > 65535) return rk_fail(ROCKET_EINVAL, "rocket_layer_norm_backward: more than 65535 planes");
    const BackwardPlan plan(rows, planes, n, dtype);
    if (!ws || ws_bytes < plan.bytes() || reinterpret_cast<uintptr_t>(ws) % 16 != 0)
        return rk_fail(ROCKET_EWORKSPACE, "rocket_layer_norm_backward: an aligned workspace of " + std::to_string(plan.bytes()) + " bytes required");
    const bool sums_wanted = grad_weight_dev || grad_bias_dev;
    float4 *sums = static_cast<float4 *>(ws);
    float *part = sums_wanted && plan.part_bytes() > 0 ? reinterpret_cast<float *>(static_cast<char *>(ws) + plan.sums_bytes()) : nullptr;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    by_type(dtype, [&](auto t) {
        using T = decltype(t);
        const T *x = static_cast<const T *>(x_dev), *dy = static_cast<const T *>(grad_y_dev);
        T *dx = static_cast<T *>(grad_x_dev);
        const auto held = [&](auto lanes, auto slots) {
            constexpr int L = decltype(lanes)::value, S = decltype(slots)::value, G = L < 256 ? 256 / L : 1;
            if (plan.lanes != L || plan.slots != S) return;
            hipLaunchKernelGGL((rn_backward<T, L, S, G>), dim3(static_cast<unsigned>(plan.parts), static_cast<unsigned>(planes)), dim3(L * G), 0, stream, x, dy,
                               rows, planes, n, weight_dev, mean_dev, rstd_dev, dx, part, grad_weight_dev, grad_bias_dev);
        };
        held(Int<16>(), Int<1>());
        held(Int<64>(), Int<1>());
        held(Int<64>(), Int<2>());
        held(Int<256>(), Int<1>());
        held(Int<256>(), Int<2>());
        held(Int<512>(), Int<2>());
        held(Int<1024>(), Int<2>());
        if constexpr (sizeof(T) == 4) {
            held(Int<1024>(), Int<4>());
            held(Int<1024>(), Int<5>());
        }
        if (plan.row_parts > 0) {
            hipLaunchKernelGGL(rn_backward_parts<T>, dim3(static_cast<unsigned>(plan.row_parts), static_cast<unsigned>(std::min<int64_t>(plan.R, 32768))),
                               dim3(kNormThreads), 0, stream, x, dy, plan.R, planes, n, plan.length, weight_dev, mean_dev, rstd_dev, sums);
            const unsigned tiles = static_cast<unsigned>((n + int64_t{kNormThreads * kPerLoad<T>} - 1) / (kNormThreads * kPerLoad<T>));
            hipLaunchKernelGGL(rn_backward_columns<T>, dim3(tiles, static_cast<unsigned>(planes), static_cast<unsigned>(plan.parts)), dim3(kNormThreads), 0,
                               stream, x, dy, rows, planes, n, plan.per, plan.row_parts, weight_dev, mean_dev, rstd_dev, sums, dx, part);
        }
        if (part) {
            const int64_t floats = 2 * rn_stride(plan.wide);
            if (floats >= 64 * 512)
                hipLaunchKernelGGL(rn_backward_finish<64>, dim3(static_cast<unsigned>((floats + 63) / 64)), dim3(kNormThreads), 0, stream, part, plan.parts,
                                   plan.wide, grad_weight_dev, grad_bias_dev);
            else
                hipLaunchKernelGGL(rn_backward_finish<16>, dim3(static_cast<unsigned>((floats + 15) / 16)), dim3(kNormThreads), 0, stream, part, plan.parts,
                                   plan.wide, grad_weight_dev, grad_bias_dev);
        }
    });
    return hipGetLastError() == hipSuccess ? ROCKET_OK : rk_fail(ROCKET_EHIP, "launch of the layer norm's backward kernels failed");
}
