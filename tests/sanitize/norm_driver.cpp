// The layer norm's sizes up to their limits, and which rows the launches of its forward pass cover, under AddressSanitizer and
// UndefinedBehaviorSanitizer without a GPU: a call of more rows than a launch holds is several launches, and each row belongs to one of them alone (in place, a row that
// two launches normalise is normalised twice).  Launches are replaced by a stub that reads their arguments.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <string>

#include "rocket_internal.hpp"

static std::string g_error;
void rk_set_error(const std::string &msg) { g_error = msg; }
int rk_fail(int code, const std::string &msg)
{
    g_error = msg;
    return code;
}

// kernels' names by their host address; the first is entered before this file's own variables are made
static std::map<const void *, std::string> &names()
{
    static std::map<const void *, std::string> all;
    return all;
}
static dim3 g_grid, g_block;
static int64_t g_next = 0, g_rows = 0, g_launches = 0, g_calls = 0;      // examples covered so far, of a call; launches
static int32_t g_planes = 0;

// the number after the i-th "Li" of a mangled name
static int number(const std::string &name, int i)
{
    size_t at = 0;
    for (; i >= 0; --i) at = name.find("Li", at) + 2;
    return std::atoi(name.c_str() + at);
}

static void fail(const char *what, const std::string &name)
{
    std::printf("%s: %s, rows %lld planes %d, launch from %lld\n", what, name.c_str(), static_cast<long long>(g_rows), g_planes, static_cast<long long>(g_next));
    std::exit(1);
}

extern "C" {
void **__hipRegisterFatBinary(const void *)
{
    static void *none = nullptr;
    return &none;
}
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *device, unsigned, void *, void *, void *, void *, int *)
{
    names()[host] = device;
}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t)
{
    g_grid = grid;
    g_block = block;
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *shared, hipStream_t *stream)
{
    *grid = g_grid;
    *block = g_block;
    *shared = 0;
    *stream = nullptr;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *kernel, dim3 grid, dim3 block, void **args, size_t, hipStream_t)
{
    const std::string &name = names()[kernel];
    if (name.find("10rn_forwardI") == std::string::npos) return hipSuccess;
    // rn_forward<T, lanes, slots, examples of a group, streamed>(x, first, end, planes, ...)
    const int lanes = number(name, 0), at_once = number(name, 2);
    const int64_t first = *static_cast<int *>(args[1]), end = *static_cast<int *>(args[2]), planes = *static_cast<int *>(args[3]);
    const int64_t groups = static_cast<int64_t>(grid.x) * (static_cast<int>(block.x) / lanes);
    ++g_launches;
    if (first != g_next) fail("a launch does not begin where the last one ended", name);
    if (planes != g_planes || end > g_rows || end <= first) fail("bad arguments", name);
    // group g has plane g % planes of the examples from first + g / planes * at_once on, and stops at `end`; one of up to 64 lanes
    // that begins there has nothing to do
    const int64_t last = first + (groups - 1) / planes * at_once;
    if (lanes > 64 && (last >= end || groups % planes != 0)) fail("a group without an example", name);
    const int64_t whole = first + groups / planes * at_once;       // examples before this one are covered in all planes
    const int64_t reach = std::min(last + at_once, end);           // examples from this one on in none
    if (whole < reach && groups % planes != 0) fail("examples of which only some planes are covered", name);
    g_next = reach;
    return hipSuccess;
}
hipError_t hipGetLastError(void) { return hipSuccess; }
}

static void *at(uint64_t a) { return reinterpret_cast<void *>(a); }

int main()
{
    // workspace sizes are told for every size that the calls take, also for what no card holds; more rows never need less
    for (int32_t n : {1, 17, 4097, 20481, 33000, 131073, 1000003, 1 << 30})
        for (int32_t planes : {1, 3, 2048, 65535})
            for (int backward : {0, 1}) {
                size_t before = 0;
                for (int32_t rows : {1, 300, 1 << 20, 1 << 30, (1 << 30) + 1, 2147483646, 2147483647}) {
                    const size_t need = rocket_layer_norm_workspace_bytes(rows, planes, n, backward);
                    if (need % 256 != 0 || (backward && need < 256) || (rows > 300 && need < before)) fail("bad workspace size", std::to_string(rows) + " " + std::to_string(planes) + " " + std::to_string(n));
                    before = need;
                }
            }
    float *f = static_cast<float *>(at(1 << 25));
    for (int32_t type : {ROCKET_F32, ROCKET_BF16})
        for (int32_t n : {2, 16, 17, 40, 100, 200, 500, 700, 1000, 2000, 3001, 5000, 10000, 30000})
            for (int32_t planes : {1, 2, 3, 5, 7, 1000, 65535})
                for (int32_t rows : {1, 9, 4097, 1048577, 22369621, 22369622, 89478485, 89478486, 300000001, 2147483647}) {
                    if (static_cast<double>(rows) * planes > 3e10) continue;       // thousands of launches
                    g_rows = rows;
                    g_planes = planes;
                    g_next = 0;
                    if (rocket_layer_norm(at(1 << 20), type, rows, planes, n, f, f, 1e-5f, at(1 << 20), f, f, nullptr, 0, nullptr) != ROCKET_OK) {
                        if (n == 30000) continue;       // few of them go in parts, which needs a workspace
                        fail(g_error.c_str(), "refused");
                    }
                    ++g_calls;
                    if (g_next != rows) fail("examples are left over", "call");
                }
    if (g_calls < 500 || g_launches < 5 * g_calls) fail("too few launches", "all");
    std::printf("norm driver: ok\n");
    return 0;
}
