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

#include "rocket_elements.hpp"
#include "rocket_internal.hpp"

namespace {

constexpr int kNormThreads = 256;

// Sums of N values over the workgroup, the same on every lane.
template <int N, class S>
__device__ __forceinline__ void rn_sum(S (&v)[N], S *lds)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
        for (int off = 32; off > 0; off >>= 1) v[i] += __shfl_xor(v[i], off, 64);
    const int wave = static_cast<int>(threadIdx.x) >> 6;
    __syncthreads();        // the last sums have been read
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) lds[wave * N + i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        S s = 0;
        for (int w = 0; w < kNormThreads / 64; ++w) s += lds[w * N + i];
        v[i] = s;
    }
}

// One workgroup per row, three passes over it.
template <class T>
__global__ __launch_bounds__(kNormThreads) void rn_forward(const T *x, int64_t R, int planes, int n, const float *__restrict__ weight,
                                                           const float *__restrict__ bias, float eps, T *y, float *__restrict__ mean,
                                                           float *__restrict__ rstd)
{
    constexpr int N = kPerLoad<T>;
    __shared__ double lds[kNormThreads / 64];
    for (int64_t row = blockIdx.x; row < R; row += gridDim.x) {
        const T *src = x + row * n;
        T *dst = y + row * n;
        const int64_t w0 = row % planes * n;
        float v[N], wt[N], bs[N];
        double s[1] = {0.0};
        for (int i = static_cast<int>(threadIdx.x) * N; i < n; i += kNormThreads * N) {
            rk_load(src + i, n - i, v);
#pragma unroll
            for (int q = 0; q < N; ++q) s[0] += static_cast<double>(v[q]);
        }
        rn_sum(s, lds);
        const double m = s[0] / n;
        s[0] = 0.0;
        for (int i = static_cast<int>(threadIdx.x) * N; i < n; i += kNormThreads * N) {
            rk_load(src + i, n - i, v);
#pragma unroll
            for (int q = 0; q < N; ++q) {
                const double d = i + q < n ? static_cast<double>(v[q]) - m : 0.0;
                s[0] += d * d;
            }
        }
        rn_sum(s, lds);
        const float hi = static_cast<float>(m), lo = static_cast<float>(m - static_cast<double>(hi));
        const float r = static_cast<float>(1.0 / sqrt(s[0] / n + static_cast<double>(eps)));
        for (int i = static_cast<int>(threadIdx.x) * N; i < n; i += kNormThreads * N) {
            rk_load(src + i, n - i, v);
#pragma unroll
            for (int q = 0; q < N; ++q) wt[q] = 1.f, bs[q] = 0.f;
            for (int q = 0; q < N; ++q) {
                if (weight && i + q < n) wt[q] = weight[w0 + i + q];
                if (bias && i + q < n) bs[q] = bias[w0 + i + q];
            }
#pragma unroll
            for (int q = 0; q < N; ++q) v[q] = fmaf(((v[q] - hi) - lo) * r, wt[q], bs[q]);
            rk_store(dst + i, n - i, v);
        }
        if (mean && threadIdx.x == 0) {
            mean[row] = hi;
            rstd[row] = r;
        }
    }
}

// Row sums of the backward pass: {mean g, mean(g h), e, r} of every row.
template <class T>
__global__ __launch_bounds__(kNormThreads) void rn_backward_rows(const T *x, const T *dy, int64_t R, int planes, int n,
                                                                 const float *__restrict__ weight, const float *__restrict__ mean,
                                                                 const float *__restrict__ rstd, float4 *__restrict__ sums)
{
    constexpr int N = kPerLoad<T>;
    __shared__ double lds[3 * kNormThreads / 64];
    for (int64_t row = blockIdx.x; row < R; row += gridDim.x) {
        const float m = mean[row], r = rstd[row];
        const int64_t w0 = row % planes * n;
        float v[N], d[N];
        double s[3] = {0.0, 0.0, 0.0};
        for (int i = static_cast<int>(threadIdx.x) * N; i < n; i += kNormThreads * N) {
            rk_load(x + row * n + i, n - i, v);
            rk_load(dy + row * n + i, n - i, d);
            for (int q = 0; q < N; ++q) {
                const float g = weight && i + q < n ? d[q] * weight[w0 + i + q] : d[q];
                const float h = i + q < n ? (v[q] - m) * r : 0.f;
                s[0] += static_cast<double>(g);
                s[1] += static_cast<double>(g) * static_cast<double>(h);
                s[2] += static_cast<double>(h);
            }
        }
        rn_sum(s, lds);
        const double e = s[2] / n;
        if (threadIdx.x == 0)
            sums[row] = make_float4(static_cast<float>(s[0] / n), static_cast<float>((s[1] - e * s[0]) / n), static_cast<float>(e), r);
    }
}

// A workgroup has kNormThreads * N columns of a plane and `per` of its rows: dx there, and the columns' partial sums of those rows.
// grid (column tiles, planes, row groups)
template <class T>
__global__ __launch_bounds__(kNormThreads) void rn_backward_columns(const T *x, const T *dy, int rows, int planes, int n, int per,
                                                                    const float *__restrict__ weight, const float *__restrict__ mean,
                                                                    const float4 *__restrict__ sums, T *dx, float *__restrict__ part)
{
    constexpr int N = kPerLoad<T>;
    const int plane = blockIdx.y, i = (static_cast<int>(blockIdx.x) * kNormThreads + static_cast<int>(threadIdx.x)) * N;
    if (i >= n) return;
    float wt[N], dw[N] = {}, db[N] = {}, v[N], d[N];
    for (int q = 0; q < N; ++q) wt[q] = weight && i + q < n ? weight[static_cast<int64_t>(plane) * n + i + q] : 1.f;
    const int from = static_cast<int>(blockIdx.z) * per, to = min(rows, from + per);
    for (int b = from; b < to; ++b) {
        const int64_t row = static_cast<int64_t>(b) * planes + plane;
        const float4 s = sums[row];
        const float m = mean[row];
        rk_load(x + row * n + i, n - i, v);
        rk_load(dy + row * n + i, n - i, d);
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const float h = (v[q] - m) * s.w - s.z;
            dw[q] = fmaf(d[q], h, dw[q]);
            db[q] += d[q];
            v[q] = s.w * (fmaf(-h, s.y, d[q] * wt[q]) - s.x);
        }
        rk_store(dx + row * n + i, n - i, v);
    }
    const int64_t wide = static_cast<int64_t>(planes) * n;
    float *to_w = part + 2 * static_cast<int64_t>(blockIdx.z) * wide + static_cast<int64_t>(plane) * n + i;
    rk_store(to_w, n - i, *reinterpret_cast<float (*)[4]>(&dw[0]));
    rk_store(to_w + wide, n - i, *reinterpret_cast<float (*)[4]>(&db[0]));
    if constexpr (N == 8) {
        rk_store(to_w + 4, n - i - 4, *reinterpret_cast<float (*)[4]>(&dw[4]));
        rk_store(to_w + wide + 4, n - i - 4, *reinterpret_cast<float (*)[4]>(&db[4]));
    }
}

// Sums of the row groups' partial sums, in their order.
__global__ __launch_bounds__(kNormThreads) void rn_backward_finish(const float *__restrict__ part, int groups, int64_t wide,
                                                                   float *__restrict__ dw, float *__restrict__ db)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kNormThreads + threadIdx.x;
    if (i >= wide) return;
    double a = 0.0, b = 0.0;
    for (int g = 0; g < groups; ++g) {
        a += static_cast<double>(part[2 * g * wide + i]);
        b += static_cast<double>(part[(2 * g + 1) * wide + i]);
    }
    if (dw) dw[i] = static_cast<float>(a);
    if (db) db[i] = static_cast<float>(b);
}

inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// Row groups of the backward pass: enough workgroups to fill the chip, eight rows to a group at least (its partial sums are
// then a small part of what it reads).
struct NormPlan {
    int64_t R, wide;
    int per, groups;
    NormPlan(int32_t rows, int32_t planes, int32_t n) : R(static_cast<int64_t>(rows) * planes), wide(static_cast<int64_t>(planes) * n)
    {
        const int64_t tiles = (n + kNormThreads * 4 - 1) / (kNormThreads * 4) * planes;
        const int64_t want = std::min<int64_t>(std::max<int64_t>(1, 2048 / tiles), 4096);
        per = static_cast<int>(std::max<int64_t>(8, (rows + want - 1) / want));
        groups = (rows + per - 1) / per;
    }
    size_t sums_bytes() const { return up256(static_cast<size_t>(R) * sizeof(float4)); }
    size_t bytes() const { return sums_bytes() + up256(static_cast<size_t>(2 * groups) * static_cast<size_t>(wide) * 4); }
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
    if (rows < 1 || planes < 1 || n < 1 || !backward) return 0;
    return NormPlan(rows, planes, n).bytes();
}

extern "C" int rocket_layer_norm(const void *x_dev, int32_t dtype, int32_t rows, int32_t planes, int32_t n, const float *weight_dev,
                                 const float *bias_dev, float eps, void *y_dev, float *mean_dev, float *rstd_dev, void *, size_t,
                                 void *hip_stream)
{
    if (!x_dev || !y_dev) return rk_fail(ROCKET_EINVAL, "rocket_layer_norm: NULL pointer");
    if (!rk_type_known(dtype)) return rk_fail(ROCKET_EINVAL, "rocket_layer_norm: unknown element type");
    if (rows < 1 || planes < 1 || n < 1) return rk_fail(ROCKET_EINVAL, "rocket_layer_norm: rows, planes and n must be >= 1");
    if (!std::isfinite(eps) || !(eps > 0.f)) return rk_fail(ROCKET_EINVAL, "rocket_layer_norm: eps must be positive and finite");
    if (!mean_dev != !rstd_dev) return rk_fail(ROCKET_EINVAL, "rocket_layer_norm: mean and rstd go together");
    if (misaligned(x_dev, dtype) || misaligned(y_dev, dtype)) return rk_fail(ROCKET_EINVAL, "rocket_layer_norm: x or y is not at an element's address");
    const int64_t R = static_cast<int64_t>(rows) * planes;
    by_type(dtype, [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL(rn_forward<T>, dim3(static_cast<unsigned>(std::min<int64_t>(R, 1 << 20))), dim3(kNormThreads), 0,
                           static_cast<hipStream_t>(hip_stream), static_cast<const T *>(x_dev), R, planes, n, weight_dev, bias_dev, eps,
                           static_cast<T *>(y_dev), mean_dev, rstd_dev);
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
    const NormPlan plan(rows, planes, n);
    if (!ws || ws_bytes < plan.bytes() || reinterpret_cast<uintptr_t>(ws) % 16 != 0)
        return rk_fail(ROCKET_EWORKSPACE, "rocket_layer_norm_backward: an aligned workspace of " + std::to_string(plan.bytes()) + " bytes required");
    float4 *sums = static_cast<float4 *>(ws);
    float *part = reinterpret_cast<float *>(static_cast<char *>(ws) + plan.sums_bytes());
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    by_type(dtype, [&](auto t) {
        using T = decltype(t);
        const T *x = static_cast<const T *>(x_dev), *dy = static_cast<const T *>(grad_y_dev);
        hipLaunchKernelGGL(rn_backward_rows<T>, dim3(static_cast<unsigned>(std::min<int64_t>(plan.R, 1 << 20))), dim3(kNormThreads), 0, stream, x, dy,
                           plan.R, planes, n, weight_dev, mean_dev, rstd_dev, sums);
        const unsigned tiles = static_cast<unsigned>((n + kNormThreads * kPerLoad<T> - 1) / (kNormThreads * kPerLoad<T>));
        hipLaunchKernelGGL(rn_backward_columns<T>, dim3(tiles, static_cast<unsigned>(planes), static_cast<unsigned>(plan.groups)), dim3(kNormThreads), 0,
                           stream, x, dy, rows, planes, n, plan.per, weight_dev, mean_dev, sums, static_cast<T *>(grad_x_dev), part);
        if (grad_weight_dev || grad_bias_dev)
            hipLaunchKernelGGL(rn_backward_finish, dim3(static_cast<unsigned>((plan.wide + kNormThreads - 1) / kNormThreads)), dim3(kNormThreads), 0, stream,
                               part, plan.groups, plan.wide, grad_weight_dev, grad_bias_dev);
    });
    return hipGetLastError() == hipSuccess ? ROCKET_OK : rk_fail(ROCKET_EHIP, "launch of the layer norm's backward kernels failed");
}
