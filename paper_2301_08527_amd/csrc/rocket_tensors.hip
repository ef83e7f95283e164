// Many tensors at once for MI355X (gfx950): the global norm of all gradients, clipping, and the update that clips on the way.
// See include/rocket.h for the contract.
//
// The tensors of a list are cut into chunks of equal size; the records of up to kPerLaunch tensors travel in a launch's
// arguments, so nothing is copied to the device beforehand.  A workgroup finds a chunk's tensor by comparing the
// chunk's number with the first chunks of all tensors, one per lane.
//   rt_squares   sums of squares of the chunks, fp64: a partial sum per workgroup
//   rt_finish    norm = sqrt(sum of the partial sums), coefficient = norm <= max ? 1 : max / norm
//   rt_scale     out = grad * coefficient
//   rt_sgd       out = param - lr * coefficient * grad
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>

#include "rocket_elements.hpp"
#include "rocket_internal.hpp"

namespace {

constexpr int kThreads_ = 256;
constexpr int kPerLaunch = 96;            // records of a launch: under 4 KB of arguments with three addresses each
constexpr int kMostGroups = 2048;         // workgroups of a launch, eight to a CU

// Up to kPerLaunch tensors, POINTERS addresses each.
template <int POINTERS>
struct Records {
    int64_t count[kPerLaunch];
    void *data[POINTERS][kPerLaunch];
    int32_t first[kPerLaunch + 1];        // chunk of the launch that a tensor begins with; first[tensors]: chunks of the launch
    uint8_t dtype[kPerLaunch];
    int32_t tensors, chunk;               // chunk: values of a chunk, a multiple of 8 * kThreads_
};

// The tensor of chunk c: as many lanes as have a tensor that starts at or before c.
template <int P>
__device__ __forceinline__ int tensor_of(const Records<P> &r, int c)
{
    int found = 0;
    for (int i = 0; i < r.tensors; i += 64) {
        const int at = i + static_cast<int>(threadIdx.x & 63);
        found += __popcll(__ballot(at < r.tensors && r.first[min(at, kPerLaunch)] <= c));
    }
    return __builtin_amdgcn_readfirstlane(found - 1);
}

template <class T>
__device__ double chunk_squares(const T *g, int64_t count)
{
    constexpr int N = kPerLoad<T>;
    double s = 0.0;
    for (int64_t i = static_cast<int64_t>(threadIdx.x) * N; i < count; i += kThreads_ * N) {
        float v[N];
        rk_load(g + i, count - i, v);
#pragma unroll
        for (int q = 0; q < N; ++q) s = fma(static_cast<double>(v[q]), static_cast<double>(v[q]), s);
    }
    return s;
}

__device__ __forceinline__ double group_sum(double v, double *lds)
{
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
    for (int w = 0; w < kThreads_ / 64; ++w) v += lds[w];
    return v;
}

__global__ __launch_bounds__(kThreads_) void rt_squares(const Records<1> r, double *__restrict__ partial)
{
    __shared__ double lds[kThreads_ / 64];
    double s = 0.0;
    for (int c = blockIdx.x; c < r.first[r.tensors]; c += gridDim.x) {
        const int t = tensor_of(r, c);
        const int64_t at = static_cast<int64_t>(c - r.first[t]) * r.chunk, left = min(r.count[t] - at, static_cast<int64_t>(r.chunk));
        if (r.dtype[t] == ROCKET_F32) s += chunk_squares(static_cast<const float *>(r.data[0][t]) + at, left);
        else if (r.dtype[t] == ROCKET_BF16) s += chunk_squares(static_cast<const rk_bf16 *>(r.data[0][t]) + at, left);
        else s += chunk_squares(static_cast<const rk_f16 *>(r.data[0][t]) + at, left);
    }
    s = group_sum(s, lds);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__global__ __launch_bounds__(kThreads_) void rt_finish(const double *__restrict__ partial, int count, double max_norm, double *__restrict__ out)
{
    __shared__ double lds[kThreads_ / 64];
    double s = 0.0;
    for (int i = threadIdx.x; i < count; i += kThreads_) s += partial[i];
    s = group_sum(s, lds);
    if (threadIdx.x == 0) {
        const double norm = sqrt(s);
        out[0] = norm;
        out[1] = norm <= max_norm ? 1.0 : max_norm / norm;     // NaN stays NaN
    }
}

template <class T>
__device__ void chunk_scale(const T *g, T *out, int64_t count, double c)
{
    constexpr int N = kPerLoad<T>;
    for (int64_t i = static_cast<int64_t>(threadIdx.x) * N; i < count; i += kThreads_ * N) {
        float v[N];
        rk_load(g + i, count - i, v);
        // the product in fp64: the coefficient of a norm beyond 1e38 would lose its digits in fp32
#pragma unroll
        for (int q = 0; q < N; ++q) v[q] = static_cast<float>(static_cast<double>(v[q]) * c);
        rk_store(out + i, count - i, v);
    }
}

// r.data: gradients, results
__global__ __launch_bounds__(kThreads_) void rt_scale(const Records<2> r, const double *__restrict__ norm, int in_place)
{
    const double k = norm[1];
    if (in_place && k == 1.0) return;
    for (int c = blockIdx.x; c < r.first[r.tensors]; c += gridDim.x) {
        const int t = tensor_of(r, c);
        const int64_t at = static_cast<int64_t>(c - r.first[t]) * r.chunk, left = min(r.count[t] - at, static_cast<int64_t>(r.chunk));
        if (r.dtype[t] == ROCKET_F32) chunk_scale(static_cast<const float *>(r.data[0][t]) + at, static_cast<float *>(r.data[1][t]) + at, left, k);
        else if (r.dtype[t] == ROCKET_BF16) chunk_scale(static_cast<const rk_bf16 *>(r.data[0][t]) + at, static_cast<rk_bf16 *>(r.data[1][t]) + at, left, k);
        else chunk_scale(static_cast<const rk_f16 *>(r.data[0][t]) + at, static_cast<rk_f16 *>(r.data[1][t]) + at, left, k);
    }
}

template <class T>
__device__ void chunk_sgd(const float *p, const T *g, float *out, int64_t count, double rate)
{
    constexpr int N = 4;
    for (int64_t i = static_cast<int64_t>(threadIdx.x) * N; i < count; i += kThreads_ * N) {
        float v[N], w[N];
        rk_load(p + i, count - i, v);
        for (int q = 0; q < N; ++q) w[q] = i + q < count ? static_cast<float>(g[i + q]) : 0.f;
#pragma unroll
        for (int q = 0; q < N; ++q) v[q] = static_cast<float>(fma(-rate, static_cast<double>(w[q]), static_cast<double>(v[q])));
        rk_store(out + i, count - i, v);
    }
}

// r.data: gradients, parameters, results
__global__ __launch_bounds__(kThreads_) void rt_sgd(const Records<3> r, double lr, const double *__restrict__ norm)
{
    const double rate = norm ? lr * norm[1] : lr;
    for (int c = blockIdx.x; c < r.first[r.tensors]; c += gridDim.x) {
        const int t = tensor_of(r, c);
        const int64_t at = static_cast<int64_t>(c - r.first[t]) * r.chunk, left = min(r.count[t] - at, static_cast<int64_t>(r.chunk));
        const float *p = static_cast<const float *>(r.data[1][t]) + at;
        float *out = static_cast<float *>(r.data[2][t]) + at;
        if (r.dtype[t] == ROCKET_F32) chunk_sgd(p, static_cast<const float *>(r.data[0][t]) + at, out, left, rate);
        else if (r.dtype[t] == ROCKET_BF16) chunk_sgd(p, static_cast<const rk_bf16 *>(r.data[0][t]) + at, out, left, rate);
        else chunk_sgd(p, static_cast<const rk_f16 *>(r.data[0][t]) + at, out, left, rate);
    }
}

constexpr int64_t kMostValues = int64_t{1} << 42;      // of one tensor: chunk numbers stay below 2^31 with room for a launch's tensors

// "" or what is wrong with a list
std::string list_fault(const rocket_tensor *t, int32_t tensors, bool f32_only)
{
    if (!t) return "NULL list";
    if (tensors < 1) return "a list holds one tensor at least";
    for (int32_t i = 0; i < tensors; ++i) {
        const char *what = nullptr;
        if (!rk_type_known(t[i].dtype) || (f32_only && t[i].dtype != ROCKET_F32)) what = f32_only ? "ROCKET_F32 required" : "unknown element type";
        else if (t[i].count < 0 || t[i].count > kMostValues) what = "a count outside [0, 2^42]";
        else if (t[i].count > 0 && !t[i].data) what = "NULL data";
        else if (t[i].count > 0 && reinterpret_cast<uintptr_t>(t[i].data) % rk_type_bytes(t[i].dtype) != 0) what = "not at an element's address";
        if (what) return "tensor " + std::to_string(i) + ": " + what;
    }
    return "";
}

std::string pair_fault(const rocket_tensor *a, const rocket_tensor *b, int32_t tensors, bool types)
{
    for (int32_t i = 0; i < tensors; ++i)
        if (a[i].count != b[i].count || (types && a[i].dtype != b[i].dtype))
            return "tensor " + std::to_string(i) + ": the lists differ in " + (a[i].count != b[i].count ? "count" : "type");
    return "";
}

// Chunks so large that all tensors together make about kMostGroups of them, between 2,048 and 16,384 values; the chunks of a
// launch must fit 31 bits (larger ones where they would not).
struct ListPlan {
    int32_t chunk = 0, launches = 0;
    int64_t groups = 0;      // workgroups of all launches
    ListPlan(const rocket_tensor *t, int32_t tensors)
    {
        int64_t values = 0;
        for (int32_t i = 0; i < tensors; ++i) values += t[i].count;
        int64_t c = std::min<int64_t>(std::max<int64_t>(values / kMostGroups, 2048), 16384) / 2048 * 2048;
        while (values / c > (int64_t{1} << 30)) c *= 2;
        chunk = static_cast<int32_t>(std::min<int64_t>(c, 1 << 30));
        each(t, tensors, [&](int32_t, int32_t, int64_t chunks) {
            ++launches;
            groups += std::min<int64_t>(chunks, kMostGroups);
            return ROCKET_OK;
        });
    }
    int64_t chunks_of(int64_t count) const { return (count + chunk - 1) / chunk; }
    // f(first tensor, one past the last, chunks) for the tensors of each launch
    template <class F>
    int each(const rocket_tensor *t, int32_t tensors, F f) const
    {
        for (int32_t a = 0; a < tensors;) {
            int64_t chunks = 0;
            int32_t b = a;
            int filled = 0;
            for (; b < tensors && filled < kPerLaunch; ++b) {
                const int64_t more = chunks_of(t[b].count);
                if (chunks + more > INT32_MAX - kMostGroups && chunks > 0) break;
                chunks += more;
                filled += more > 0;
            }
            if (chunks > 0)
                if (const int rc = f(a, b, chunks); rc != ROCKET_OK) return rc;
            a = b;
        }
        return ROCKET_OK;
    }
};

template <int P>
void fill(Records<P> &r, const ListPlan &plan, int32_t a, int32_t b, const rocket_tensor *const (&lists)[P])
{
    int k = 0;
    int64_t first = 0;
    for (int32_t i = a; i < b; ++i) {
        const int64_t count = lists[0][i].count;
        if (count == 0) continue;
        r.count[k] = count;
        r.dtype[k] = static_cast<uint8_t>(lists[0][i].dtype);
        for (int p = 0; p < P; ++p) r.data[p][k] = lists[p][i].data;
        r.first[k++] = static_cast<int32_t>(first);
        first += plan.chunks_of(count);
    }
    r.first[k] = static_cast<int32_t>(first);
    r.tensors = k;
    r.chunk = plan.chunk;
}

int checked_launch(const char *who)
{
    return hipGetLastError() == hipSuccess ? ROCKET_OK : rk_fail(ROCKET_EHIP, std::string(who) + ": launch of a kernel failed");
}

int norm_impl(const char *who, const rocket_tensor *grads, int32_t tensors, double max_norm, double *norm_dev, void *ws, size_t ws_bytes,
              hipStream_t stream, const ListPlan &plan)
{
    double *partial = static_cast<double *>(ws);
    int64_t at = 0;
    const int rc = plan.each(grads, tensors, [&](int32_t a, int32_t b, int64_t chunks) {
        Records<1> r;
        fill<1>(r, plan, a, b, {grads});
        const unsigned groups = static_cast<unsigned>(std::min<int64_t>(chunks, kMostGroups));
        hipLaunchKernelGGL(rt_squares, dim3(groups), dim3(kThreads_), 0, stream, r, partial + at);
        at += groups;
        return checked_launch(who);
    });
    if (rc != ROCKET_OK) return rc;
    hipLaunchKernelGGL(rt_finish, dim3(1), dim3(kThreads_), 0, stream, partial, static_cast<int>(at), max_norm, norm_dev);
    return checked_launch(who);
}

int check_norm(const char *fn, const rocket_tensor *grads, int32_t tensors, double max_norm, const double *norm_dev, const void *ws, size_t ws_bytes)
{
    const std::string who = std::string(fn) + ": ";
    const std::string fault = list_fault(grads, tensors, false);
    if (!fault.empty()) return rk_fail(ROCKET_EINVAL, who + fault);
    if (!(max_norm > 0.0)) return rk_fail(ROCKET_EINVAL, who + "max_norm must be positive");
    if (!norm_dev) return rk_fail(ROCKET_EINVAL, who + "NULL norm");
    const size_t need = rocket_grad_workspace_bytes(grads, tensors);
    if (!ws || ws_bytes < need || reinterpret_cast<uintptr_t>(ws) % 16 != 0)
        return rk_fail(ROCKET_EWORKSPACE, who + "an aligned workspace of " + std::to_string(need) + " bytes required");
    return ROCKET_OK;
}

}  // namespace

extern "C" size_t rocket_grad_workspace_bytes(const rocket_tensor *grads, int32_t tensors)
{
    if (!list_fault(grads, tensors, false).empty()) return 0;
    const ListPlan plan(grads, tensors);
    return static_cast<size_t>((plan.groups * 8 + 255) / 256 * 256 + 256);
}

extern "C" int rocket_grad_norm(const rocket_tensor *grads, int32_t tensors, double max_norm, double *norm_dev, void *ws, size_t ws_bytes,
                                void *hip_stream)
{
    if (const int rc = check_norm("rocket_grad_norm", grads, tensors, max_norm, norm_dev, ws, ws_bytes); rc != ROCKET_OK) return rc;
    return norm_impl("rocket_grad_norm", grads, tensors, max_norm, norm_dev, ws, ws_bytes, static_cast<hipStream_t>(hip_stream),
                     ListPlan(grads, tensors));
}

extern "C" int rocket_grad_clip(const rocket_tensor *grads, const rocket_tensor *out, int32_t tensors, double max_norm, double *norm_dev, void *ws,
                                size_t ws_bytes, void *hip_stream)
{
    const char *who = "rocket_grad_clip";
    if (const int rc = check_norm(who, grads, tensors, max_norm, norm_dev, ws, ws_bytes); rc != ROCKET_OK) return rc;
    if (out) {
        std::string fault = list_fault(out, tensors, false);
        if (fault.empty()) fault = pair_fault(grads, out, tensors, true);
        if (!fault.empty()) return rk_fail(ROCKET_EINVAL, std::string(who) + ": out: " + fault);
    }
    const ListPlan plan(grads, tensors);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (const int rc = norm_impl(who, grads, tensors, max_norm, norm_dev, ws, ws_bytes, stream, plan); rc != ROCKET_OK) return rc;
    return plan.each(grads, tensors, [&](int32_t a, int32_t b, int64_t chunks) {
        Records<2> r;
        fill<2>(r, plan, a, b, {grads, out ? out : grads});
        hipLaunchKernelGGL(rt_scale, dim3(static_cast<unsigned>(std::min<int64_t>(chunks, kMostGroups))), dim3(kThreads_), 0, stream, r, norm_dev,
                           out ? 0 : 1);
        return checked_launch(who);
    });
}

extern "C" int rocket_sgd_tensors(const rocket_tensor *params, const rocket_tensor *grads, const rocket_tensor *out, int32_t tensors, double lr,
                                  const double *norm_dev, void *hip_stream)
{
    const std::string who = "rocket_sgd_tensors: ";
    std::string fault = list_fault(grads, tensors, false);
    if (fault.empty()) fault = list_fault(params, tensors, true);
    if (fault.empty()) fault = pair_fault(grads, params, tensors, false);
    if (fault.empty() && out) fault = list_fault(out, tensors, true);
    if (fault.empty() && out) fault = pair_fault(grads, out, tensors, false);
    if (!fault.empty()) return rk_fail(ROCKET_EINVAL, who + fault);
    if (!std::isfinite(lr)) return rk_fail(ROCKET_EINVAL, who + "lr must be finite");
    const ListPlan plan(grads, tensors);
    return plan.each(grads, tensors, [&](int32_t a, int32_t b, int64_t chunks) {
        Records<3> r;
        fill<3>(r, plan, a, b, {grads, params, out ? out : params});
        hipLaunchKernelGGL(rt_sgd, dim3(static_cast<unsigned>(std::min<int64_t>(chunks, kMostGroups))), dim3(kThreads_), 0,
                           static_cast<hipStream_t>(hip_stream), r, lr, norm_dev);
        return checked_launch("rocket_sgd_tensors");
    });
}
