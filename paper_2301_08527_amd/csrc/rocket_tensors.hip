// Many tensors at once for MI355X (gfx950): the global norm of all gradients, clipping, and the update that clips on the way.
// See include/rocket.h for the contract.
//
// The values of a list are counted in units of kUnit, each tensor beginning a new one; the workgroups of a launch take every
// gridDim.x-th unit.  The records of the tensors travel in a launch's arguments, as many as fit 4 KB, so nothing is copied to the
// device beforehand; a workgroup finds a unit's tensor by comparing its number with the first units of all tensors, one per lane.
//   rt_squares   sums of squares, fp64: a partial sum per workgroup
//   rt_finish    norm = sqrt(sum of the partial sums), coefficient = norm <= max ? 1 : max / norm
//   rt_scale     out = grad * coefficient
//   rt_few       all of these, for a list that one workgroup goes through sooner than two launches do
//   rt_sgd       out = param - lr * coefficient * grad
// All are bound by memory.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <string>
#include <type_traits>
#include <vector>

#include "rocket_elements.hpp"
#include "rocket_internal.hpp"

namespace {

constexpr int kListThreads = 256;
// Values of a unit: of the norm and the scaling 16 KB, four loads of a lane (16-bit values in units of 8 KB: 100 million in 56 us, so in 43);
// of the update as many as there are fp32 parameters in 16 KB.
constexpr int kUnitBytes = 16384;
template <class T>
constexpr int kUnit = kUnitBytes / static_cast<int>(sizeof(T));
constexpr int kSgdUnit = kUnit<float>;
constexpr int kMostSums = 2048;           // workgroups of all rt_squares over a list together, eight to a CU (four: 200 million fp32 387 us, then 446)
constexpr int kMostGroups = 1 << 20;      // of another launch (its lanes must be fewer than 2^32)
// A list of so few units is one workgroup's: rt_few goes through 16 of them in the time of rt_squares, and no rt_finish follows (norm and
// update of 48,000 values 18.4 us, so 14.6).  Scaling them too it beats a launch for that up to 6 (8,000 values 13.3 us, so 9.0; 64,000 would
// be 14.5 against 12.6).
constexpr int kFewUnits = 16, kFewScaled = 6;
constexpr int kJoinedSums = 1024;         // partial sums up to which every workgroup of rt_scale adds them up itself: no rt_finish

// Tensors of a launch, with POINTERS addresses of 48 bits each: a few (4 tensors with the large records 15.9 us, so 13), or as many as the
// arguments may hold: 330, 220, 165 (addresses of 64 bits, 264, 172 and 128: 300 tensors scaled 56.5 us, so 48; 150 updated 223, so 216; at 48
// tensors of 17 MB 399 us, so 403).  The first address shares its 64 bits with what else a unit begins with, so that its loads wait for one
// scalar load (150 tensors: 217.5 us without); the others take 32 and 16 bits, those two to a word, as no scalar load reads 16 bits (231 us).
constexpr int kFew = 16;
constexpr int kAddressBits = 48;
constexpr int most_records(int pointers) { return (4096 - 128) / (6 * pointers + 4 + 2); }
template <int POINTERS, int MOST>
struct Records {
    static constexpr int kMost = MOST;
    uint64_t head[MOST];                  // the first address; above it 14 bits: values of the tensor's last unit, less one; and 2: the type
    int32_t first[MOST + 1];              // unit of the launch that a tensor begins with; first[tensors]: units of the launch
    int32_t tensors;
    uint32_t low[POINTERS > 1 ? POINTERS - 1 : 1][POINTERS > 1 ? MOST : 1];
    uint32_t high[POINTERS > 1 ? POINTERS - 1 : 1][POINTERS > 1 ? (MOST + 1) / 2 : 1];

    // device memory, said to the compiler: for an address out of a number it takes flat loads and stores (48 tensors of 17 MB 409 us)
    template <class T>
    __device__ __forceinline__ T *at(int p, int t) const
    {
        uint64_t a = head[t] & ((uint64_t{1} << kAddressBits) - 1);
        if (p > 0) a = static_cast<uint64_t>(high[p - 1][t >> 1] >> (t & 1) * 16 & 0xffff) << 32 | low[p - 1][t];
        return (T *)(__attribute__((address_space(1))) T *)a;
    }
    __device__ __forceinline__ int type(int t) const { return static_cast<int>(head[t] >> 62); }
    __device__ __forceinline__ int last(int t) const { return (static_cast<int>(head[t] >> kAddressBits) & 0x3fff) + 1; }
    // t: 0, 1, ... in order
    void set(int t, int64_t unit, const rocket_tensor &tensor, int last)
    {
        first[t] = static_cast<int32_t>(unit);
        head[t] = reinterpret_cast<uintptr_t>(tensor.data) | static_cast<uint64_t>(tensor.dtype << 14 | (last - 1)) << kAddressBits;
    }
    void point(int p, int t, const void *data)
    {
        const uint64_t a = reinterpret_cast<uintptr_t>(data);
        uint32_t &above = high[p - 1][t >> 1];
        low[p - 1][t] = static_cast<uint32_t>(a);
        above = t & 1 ? above | static_cast<uint32_t>(a >> 32) << 16 : static_cast<uint32_t>(a >> 32);
    }
};
static_assert(kUnitBytes / 2 <= 1 << 14 && ROCKET_F16 < 4, "a tail and a type in 16 bits");
template <int P>
using Many = Records<P, most_records(P)>;
static_assert(sizeof(Many<1>) <= 4000 && sizeof(Many<2>) <= 4000 && sizeof(Many<3>) <= 4000, "beside the other arguments");

// The tensor of unit u: as many lanes as have a tensor that starts at or before u.
template <int P, int M>
__device__ __forceinline__ int tensor_of(const Records<P, M> &r, int u)
{
    int found = 0;
    for (int i = 0; i < r.tensors; i += 64) {
        const int at = i + static_cast<int>(threadIdx.x & 63);
        found += __popcll(__ballot(at < r.tensors && r.first[min(at, M)] <= u));
    }
    return __builtin_amdgcn_readfirstlane(found - 1);
}

// Which units kListThreads lanes work on, first, first + stride, ...: those of a workgroup by default.
struct Turn {
    int first = static_cast<int>(blockIdx.x), stride = static_cast<int>(gridDim.x), lane = static_cast<int>(threadIdx.x);
};

// f(type, whole, tensor, first value, values) for these units.  UNIT: values of a unit, 0: kUnit of the type
template <int UNIT, int P, int M, class F>
__device__ __forceinline__ void each_unit(const Records<P, M> &r, const Turn &turn, F f)
{
    const int units = r.first[r.tensors];
    int t = 0, begin = 0, end = 0;
    for (int u = turn.first; u < units; u += turn.stride) {
        if (u < begin || u >= end) {
            t = tensor_of(r, u);
            begin = r.first[t];
            end = r.first[t + 1];
        }
        const auto one = [&](auto type) {
            constexpr int kValues = UNIT > 0 ? UNIT : kUnit<decltype(type)>;
            const int values = u + 1 == end ? r.last(t) : kValues;
            if (values == kValues) f(type, std::true_type(), t, static_cast<int64_t>(u - begin) * kValues, kValues);
            else f(type, std::false_type(), t, static_cast<int64_t>(u - begin) * kValues, values);
        };
        const int type = r.type(t);
        if (type == ROCKET_F32) one(float());
        else if (type == ROCKET_BF16) one(rk_bf16());
        else one(rk_f16());
    }
}

template <int THREADS = kListThreads>
__device__ __forceinline__ double group_sum(double v, double *lds)
{
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
    for (int w = 0; w < THREADS / 64; ++w) v += lds[w];
    return v;
}

// A unit's values from p on; i: this lane's first.  whole: a true_type or a false_type, so that whole units and the last of a tensor
// have code of their own (where their ways meet again, loads would be waited for).
template <class T, bool STREAM, int LOADS, class F>
__device__ __forceinline__ void load_unit(const T *p, int i, int step, int values, F whole, typename RkSlot<T>::V (&v)[LOADS])
{
#pragma unroll
    for (int k = 0; k < LOADS; ++k) v[k] = whole ? rk_load_slot<T, STREAM>(p + i + k * step) : rk_load_edge<T, STREAM, true>(p, i + k * step, values);
}

// STREAM: the list is too long for the caches to keep until the next pass over it
template <bool STREAM, class R>
__device__ __forceinline__ double squares_of(const R &r, const Turn &turn)
{
    double s = 0.0;
    each_unit<0>(r, turn, [&](auto type, auto whole, int t, int64_t at, int values) {
        using T = decltype(type);
        constexpr int N = kPerLoad<T>, kStep = kListThreads * N, kLoads = kUnit<T> / kStep;
        const T *g = r.template at<const T>(0, t) + at;
        const int i = turn.lane * N;
        typename RkSlot<T>::V v[kLoads];
        load_unit<T, STREAM, kLoads>(g, i, kStep, values, whole, v);
#pragma unroll
        for (int k = 0; k < kLoads; ++k)
#pragma unroll
            for (int q = 0; q < N; ++q) {
                const double d = static_cast<double>(static_cast<float>(v[k][q]));
                s = fma(d, d, s);
            }
    });
    return s;
}

template <bool STREAM, class R>
__global__ __launch_bounds__(kListThreads) void rt_squares(const R r, double *__restrict__ partial)
{
    __shared__ double lds[kListThreads / 64];
    const double s = group_sum(squares_of<STREAM>(r, Turn()), lds);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// {norm, coefficient}
__device__ __forceinline__ double2 norm_and_coefficient(double squares, double max_norm)
{
    const double norm = sqrt(squares);
    return make_double2(norm, norm <= max_norm ? 1.0 : max_norm / norm);       // NaN stays NaN
}

// from the partial sums, in a fixed order
__device__ __forceinline__ double2 norm_of(const double *partial, int count, double max_norm, double *lds)
{
    double s = 0.0;
#pragma unroll 8
    for (int i = threadIdx.x; i < count; i += kListThreads) s += partial[i];
    return norm_and_coefficient(group_sum(s, lds), max_norm);
}

__global__ __launch_bounds__(kListThreads) void rt_finish(const double *__restrict__ partial, int count, double max_norm, double *__restrict__ out)
{
    __shared__ double lds[kListThreads / 64];
    const double2 n = norm_of(partial, count, max_norm, lds);
    if (threadIdx.x == 0) {
        out[0] = n.x;
        out[1] = n.y;
    }
}

// r: gradients, results
template <bool STREAM, class R>
__device__ __forceinline__ void scale_units(const R &r, const Turn &turn, double c)
{
    each_unit<0>(r, turn, [&](auto type, auto whole, int t, int64_t at, int values) {
        using T = decltype(type);
        constexpr int N = kPerLoad<T>, kStep = kListThreads * N, kLoads = kUnit<T> / kStep;
        const T *g = r.template at<const T>(0, t) + at;
        T *o = r.template at<T>(1, t) + at;
        const int i = turn.lane * N;
        typename RkSlot<T>::V v[kLoads];
        load_unit<T, STREAM, kLoads>(g, i, kStep, values, whole, v);
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            // the product in fp64: the coefficient of a norm beyond 1e38 would lose its digits in fp32
            float u[N];
#pragma unroll
            for (int q = 0; q < N; ++q) u[q] = static_cast<float>(static_cast<double>(static_cast<float>(v[k][q])) * c);
            rk_store<T, true>(o + i + k * kStep, whole ? N : values - i - k * kStep, u);
        }
    });
}

// count > 0: the norm is still in `count` partial sums, which every workgroup adds up; workgroup 0 writes it.
template <bool STREAM, class R>
__global__ __launch_bounds__(kListThreads) void rt_scale(const R r, const double *__restrict__ partial, int count, double max_norm, double *__restrict__ norm,
                                                      int in_place)
{
    __shared__ double lds[kListThreads / 64];
    double c;
    if (count > 0) {
        const double2 n = norm_of(partial, count, max_norm, lds);
        if (blockIdx.x == 0 && threadIdx.x == 0) {
            norm[0] = n.x;
            norm[1] = n.y;
        }
        c = n.y;
    } else {
        c = norm[1];
    }
    if (in_place && c == 1.0) return;
    scale_units<STREAM>(r, Turn(), c);
}

// A list of few units by one workgroup of kQuarters times kListThreads lanes: the norm and, SCALE, the scaling too (every square was
// added before the first value is written).
constexpr int kQuarters = 4;
template <bool SCALE, class R>
__global__ __launch_bounds__(kQuarters * kListThreads) void rt_few(const R r, double max_norm, double *__restrict__ norm, int in_place)
{
    __shared__ double lds[kQuarters * kListThreads / 64];
    Turn turn;
    turn.first = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kListThreads);
    turn.stride = kQuarters;
    turn.lane = static_cast<int>(threadIdx.x) % kListThreads;
    const double2 n = norm_and_coefficient(group_sum<kQuarters * kListThreads>(squares_of<false>(r, turn), lds), max_norm);
    if (threadIdx.x == 0) {
        norm[0] = n.x;
        norm[1] = n.y;
    }
    if constexpr (SCALE)
        if (!in_place || n.y != 1.0) scale_units<false>(r, turn, n.y);
}

// r: gradients, parameters, results
template <bool STREAM, class R>
__global__ __launch_bounds__(kListThreads) void rt_sgd(const R r, double lr, const double *__restrict__ norm)
{
    const double rate = norm ? lr * norm[1] : lr;
    const Turn turn;
    each_unit<kSgdUnit>(r, turn, [&](auto type, auto whole, int t, int64_t at, int values) {
        using T = decltype(type);
        constexpr int N = kPerLoad<T>, kStep = kListThreads * N, kLoads = kSgdUnit / kStep;
        const T *g = r.template at<const T>(0, t) + at;
        const float *p = r.template at<const float>(1, t) + at;
        float *o = r.template at<float>(2, t) + at;
        const int i = turn.lane * N;
        typename RkSlot<T>::V v[kLoads];
        RkSlot<float>::V w[kLoads * N / 4];
        load_unit<T, STREAM, kLoads>(g, i, kStep, values, whole, v);
        // the parameters of a lane's values: N of them from i + k * kStep on
#pragma unroll
        for (int k = 0; k < kLoads; ++k)
#pragma unroll
            for (int q = 0; q < N; q += 4) {
                const int j = i + k * kStep + q;
                w[(k * N + q) / 4] = whole ? rk_load_slot<float, true>(p + j) : rk_load_edge<float, true, true>(p, j, values);
            }
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            float u[N];
#pragma unroll
            for (int q = 0; q < N; ++q)
                u[q] = static_cast<float>(fma(-rate, static_cast<double>(static_cast<float>(v[k][q])), static_cast<double>(w[(k * N + q) / 4][q % 4])));
            rk_store_f32<N, true>(o + i + k * kStep, whole ? N : values - i - k * kStep, u);
        }
    });
}

constexpr int64_t kMostValues = int64_t{1} << 40;      // of a list: units stay below 2^30

// "" or what is wrong with a list
std::string list_fault(const rocket_tensor *t, int32_t tensors, bool f32_only)
{
    if (!t) return "NULL list";
    if (tensors < 1) return "a list holds one tensor at least";
    int64_t values = 0;
    for (int32_t i = 0; i < tensors; ++i) {
        const char *what = nullptr;
        if (!rk_type_known(t[i].dtype) || (f32_only && t[i].dtype != ROCKET_F32)) what = f32_only ? "ROCKET_F32 required" : "unknown element type";
        else if (t[i].count < 0 || t[i].count > kMostValues || (values += t[i].count) > kMostValues) what = "a negative count, or more than 2^40 values";
        else if (t[i].count > 0 && !t[i].data) what = "NULL data";
        else if (t[i].count > 0 && reinterpret_cast<uintptr_t>(t[i].data) % rk_type_bytes(t[i].dtype) != 0) what = "not at an element's address";
        else if (t[i].count > 0 && reinterpret_cast<uintptr_t>(t[i].data) >> kAddressBits != 0) what = "an address of more than 48 bits";
        else if (t[i].reserved != 0) what = "reserved must be 0";
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

// Whether memory that a call writes (`out`) is written twice or read as something else: every tensor of `out` may be the tensor of
// `in` that has its place, else it overlaps none of `out`, `in` and `other`.
bool overlapping(const rocket_tensor *out, const rocket_tensor *in, const rocket_tensor *other, int32_t tensors)
{
    struct Span {
        uintptr_t from, to;
        bool written;
    };
    Span few[3 * kFew];
    std::vector<Span> many;
    int32_t k = 0;
    Span *spans = few;
    if (tensors > kFew) {
        many.resize(static_cast<size_t>(tensors) * 3);
        spans = many.data();
    }
    const auto add = [&](const rocket_tensor &t, bool written) {
        const uintptr_t from = reinterpret_cast<uintptr_t>(t.data);
        spans[k++] = {from, from + static_cast<uintptr_t>(t.count) * rk_type_bytes(t.dtype), written};
    };
    for (int32_t i = 0; i < tensors; ++i) {
        if (out[i].count == 0) continue;
        add(out[i], true);
        if (in[i].data != out[i].data) add(in[i], false);
        if (other) add(other[i], false);
    }
    std::sort(spans, spans + k, [](const Span &a, const Span &b) { return a.from < b.from; });
    uintptr_t written = 0, read = 0;      // ends of what lies before
    for (int32_t i = 0; i < k; ++i) {
        if (spans[i].from < written || (spans[i].written && spans[i].from < read)) return true;
        uintptr_t &end = spans[i].written ? written : read;
        end = std::max(end, spans[i].to);
    }
    return false;
}

int check_written(const char *who, const rocket_tensor *out, const rocket_tensor *in, const rocket_tensor *other, int32_t tensors)
{
    try {
        if (overlapping(out, in, other, tensors)) return rk_fail(ROCKET_EINVAL, std::string(who) + ": tensors that are written overlap others");
    } catch (const std::bad_alloc &) {
        return rk_fail(ROCKET_ENOMEM, std::string(who) + ": no memory for the list");
    }
    return ROCKET_OK;
}

inline int64_t unit_of(int32_t dtype) { return kUnitBytes / static_cast<int64_t>(rk_type_bytes(dtype)); }

// A list's launches.
struct ListPlan {
    int64_t units = 0, bytes = 0, unit;
    // unit: values of one, 0: kUnit of each tensor's type
    ListPlan(const rocket_tensor *t, int32_t tensors, int64_t unit = 0) : unit(unit)
    {
        for (int32_t i = 0; i < tensors; ++i) {
            units += units_of(t[i]);
            bytes += t[i].count * static_cast<int64_t>(rk_type_bytes(t[i].dtype));
        }
    }
    int64_t values(const rocket_tensor &t) const { return unit > 0 ? unit : unit_of(t.dtype); }
    int64_t units_of(const rocket_tensor &t) const { return (t.count + values(t) - 1) / values(t); }
    // f(records, units) for each launch of tensors with P addresses each; a list without values has none
    template <int P, class F>
    int each(const rocket_tensor *const (&lists)[P], int32_t tensors, F f) const
    {
        return tensors <= kFew ? each_of<Records<P, kFew>>(lists, tensors, f) : each_of<Many<P>>(lists, tensors, f);
    }
    template <class R, int P, class F>
    int each_of(const rocket_tensor *const (&lists)[P], int32_t tensors, F f) const
    {
        for (int32_t i = 0; i < tensors;) {
            R r;
            int k = 0;
            int64_t some = 0;
            for (; i < tensors && k < R::kMost; ++i) {
                const int64_t count = lists[0][i].count;
                if (count == 0) continue;
                for (int p = 1; p < P; ++p) r.point(p, k, lists[p][i].data);
                r.set(k++, some, lists[0][i], static_cast<int>((count - 1) % values(lists[0][i])) + 1);
                some += units_of(lists[0][i]);
            }
            if (k == 0) break;
            r.first[k] = static_cast<int32_t>(some);
            r.tensors = k;
            const int rc = f(r, some);
            if (rc != ROCKET_OK) return rc;
        }
        return ROCKET_OK;
    }
    bool few() const { return units > 0 && units <= kFewUnits; }       // one launch: no tensor without a unit is in it
    // partial sums of a launch of a norm: of kMostSums as many as it has of the units
    int64_t sums(int64_t some) const { return std::min(some, std::max<int64_t>(1, kMostSums * some / units)); }
    size_t workspace(int32_t tensors) const
    {
        const int64_t most = std::min<int64_t>(units, kMostSums + tensors / Many<1>::kMost + 1);
        return static_cast<size_t>((most * 8 + 255) / 256 * 256 + 256);
    }
};

int checked_launch(const char *who)
{
    return hipGetLastError() == hipSuccess ? ROCKET_OK : rk_fail(ROCKET_EHIP, std::string(who) + ": launch of a kernel failed");
}

unsigned groups_of(int64_t units) { return static_cast<unsigned>(std::min<int64_t>(units, kMostGroups)); }

// What a pass leaves for the next one is kept by the caches up to here (256 MB on the memory's side); beyond, it only displaces, and so do
// results: 300 tensors (67 MB) streamed 73 us, kept 58, their results kept too 72; 200 million fp32 (800 MB) kept 414, streamed 387.
constexpr int64_t kKeptBytes = 192 << 20;
template <class F>
void by_length(bool stream, F f)
{
    if (stream) f(std::true_type());
    else f(std::false_type());
}

// the partial sums of a norm; *count receives their number
int squares(const char *who, const rocket_tensor *grads, int32_t tensors, double *partial, hipStream_t stream, const ListPlan &plan, int *count)
{
    *count = 0;
    return plan.each<1>({grads}, tensors, [&](const auto &r, int64_t units) {
        const int sums = static_cast<int>(plan.sums(units));
        by_length(plan.bytes > kKeptBytes, [&](auto once) {
            hipLaunchKernelGGL((rt_squares<decltype(once)::value>), dim3(static_cast<unsigned>(sums)), dim3(kListThreads), 0, stream, r, partial + *count);
        });
        *count += sums;
        return checked_launch(who);
    });
}

int finish(const char *who, const double *partial, int count, double max_norm, double *norm_dev, hipStream_t stream)
{
    hipLaunchKernelGGL(rt_finish, dim3(1), dim3(kListThreads), 0, stream, partial, count, max_norm, norm_dev);
    return checked_launch(who);
}

int few_norm(const char *who, const rocket_tensor *grads, int32_t tensors, double max_norm, double *norm_dev, hipStream_t stream, const ListPlan &plan)
{
    return plan.each<1>({grads}, tensors, [&](const auto &r, int64_t) {
        hipLaunchKernelGGL((rt_few<false>), dim3(1), dim3(kQuarters * kListThreads), 0, stream, r, max_norm, norm_dev, 0);
        return checked_launch(who);
    });
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
    return list_fault(grads, tensors, false).empty() ? ListPlan(grads, tensors).workspace(tensors) : 0;
}

extern "C" int rocket_grad_norm(const rocket_tensor *grads, int32_t tensors, double max_norm, double *norm_dev, void *ws, size_t ws_bytes,
                                void *hip_stream)
{
    const char *who = "rocket_grad_norm";
    if (const int rc = check_norm(who, grads, tensors, max_norm, norm_dev, ws, ws_bytes); rc != ROCKET_OK) return rc;
    const ListPlan plan(grads, tensors);
    if (plan.few()) return few_norm(who, grads, tensors, max_norm, norm_dev, static_cast<hipStream_t>(hip_stream), plan);
    double *partial = static_cast<double *>(ws);
    int count = 0;
    if (const int rc = squares(who, grads, tensors, partial, static_cast<hipStream_t>(hip_stream), plan, &count); rc != ROCKET_OK) return rc;
    return finish(who, partial, count, max_norm, norm_dev, static_cast<hipStream_t>(hip_stream));
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
    if (const int rc = check_written(who, out ? out : grads, grads, nullptr, tensors); rc != ROCKET_OK) return rc;
    const ListPlan plan(grads, tensors);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (plan.few() && plan.units <= kFewScaled)
        return plan.each<2>({grads, out ? out : grads}, tensors, [&](const auto &r, int64_t) {
            hipLaunchKernelGGL((rt_few<true>), dim3(1), dim3(kQuarters * kListThreads), 0, stream, r, max_norm, norm_dev, out ? 0 : 1);
            return checked_launch(who);
        });
    double *partial = static_cast<double *>(ws);
    int count = 0;
    int rc = plan.few() ? few_norm(who, grads, tensors, max_norm, norm_dev, stream, plan) : squares(who, grads, tensors, partial, stream, plan, &count);
    const bool joined = count > 0 && count <= kJoinedSums;
    if (rc == ROCKET_OK && !joined && !plan.few()) rc = finish(who, partial, count, max_norm, norm_dev, stream);
    if (rc != ROCKET_OK) return rc;
    return plan.each<2>({grads, out ? out : grads}, tensors, [&](const auto &r, int64_t units) {
        by_length(plan.bytes > kKeptBytes, [&](auto once) {
            hipLaunchKernelGGL((rt_scale<decltype(once)::value>), dim3(groups_of(units)), dim3(kListThreads), 0, stream, r, partial, joined ? count : 0, max_norm,
                               norm_dev, out ? 0 : 1);
        });
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
    if (const int rc = check_written("rocket_sgd_tensors", out ? out : params, params, grads, tensors); rc != ROCKET_OK) return rc;
    const ListPlan plan(grads, tensors, kSgdUnit);
    return plan.each<3>({grads, params, out ? out : params}, tensors, [&](const auto &r, int64_t units) {
        by_length(plan.bytes > kKeptBytes, [&](auto once) {
            hipLaunchKernelGGL((rt_sgd<decltype(once)::value>), dim3(groups_of(units)), dim3(kListThreads), 0, static_cast<hipStream_t>(hip_stream), r, lr, norm_dev);
        });
        return checked_launch("rocket_sgd_tensors");
    });
}
