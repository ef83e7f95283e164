// Drives the host side of the layer norm and of the lists of tensors under AddressSanitizer and UndefinedBehaviorSanitizer
// without a GPU: plans, records, checks and workspace sizes at sizes from one value to the limits.  Launches are replaced by a
// stub that looks at the grid.
#include <hip/hip_runtime.h>

#include <cstdio>
#include <cstdlib>
#include <string>
#include <vector>

#include "rocket_internal.hpp"

static int64_t g_launches = 0, g_lanes = 0;
static std::string g_error;
void rk_set_error(const std::string &msg) { g_error = msg; }
int rk_fail(int code, const std::string &msg)
{
    g_error = msg;
    return code;
}

static dim3 g_grid, g_block;
extern "C" hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t)
{
    g_grid = grid;
    g_block = block;
    return hipSuccess;
}
extern "C" hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *shared, hipStream_t *stream)
{
    *grid = g_grid;
    *block = g_block;
    *shared = 0;
    *stream = nullptr;
    return hipSuccess;
}
extern "C" hipError_t hipLaunchKernel(const void *, dim3 grid, dim3 block, void **, size_t, hipStream_t)
{
    const uint64_t lanes = static_cast<uint64_t>(grid.x) * block.x;
    if (grid.x == 0 || grid.y == 0 || grid.z == 0 || lanes >= (1ull << 32) || grid.y > 65535 || grid.z > 65535 || block.x > 1024) {
        std::printf("bad grid %u %u %u x %u\n", grid.x, grid.y, grid.z, block.x);
        std::exit(1);
    }
    ++g_launches;
    g_lanes += static_cast<int64_t>(lanes);
    return hipSuccess;
}
extern "C" hipError_t hipGetLastError(void) { return hipSuccess; }

#define CHECK(x)                                                                \
    do {                                                                        \
        if (!(x)) {                                                             \
            std::printf("line %d: %s (%s)\n", __LINE__, #x, g_error.c_str());   \
            return 1;                                                           \
        }                                                                       \
    } while (0)

static void *at(uint64_t a) { return reinterpret_cast<void *>(a); }

int main()
{
    double *norm = static_cast<double *>(at(4096));
    // lists of any length, with empty tensors, one value, whole units and one more
    for (int32_t n : {1, 2, 15, 16, 17, 164, 165, 166, 219, 220, 221, 329, 330, 331, 662, 5000}) {
        std::vector<rocket_tensor> g(n), o(n), p(n), q(n);
        uint64_t next = 1 << 20;
        for (int32_t i = 0; i < n; ++i) {
            const int64_t counts[] = {0, 1, 4095, 4096, 4097, 8192, 8193, 100003, 7};
            const int64_t count = counts[(i * 7 + n) % 9];
            const int32_t type = i % 3;
            for (rocket_tensor *t : {&g[i], &o[i], &p[i], &q[i]}) {
                *t = {at(next), count, t == &p[i] || t == &q[i] ? ROCKET_F32 : type, 0};
                next += (static_cast<uint64_t>(count) * 4 + 255) / 256 * 256;
            }
        }
        const size_t need = rocket_grad_workspace_bytes(g.data(), n);
        CHECK(need >= 256 && need % 256 == 0);
        CHECK(rocket_grad_norm(g.data(), n, 1.0, norm, at(8192), need, nullptr) == ROCKET_OK);
        CHECK(rocket_grad_norm(g.data(), n, 1.0, norm, at(8192), need - 1, nullptr) == ROCKET_EWORKSPACE);
        CHECK(rocket_grad_clip(g.data(), o.data(), n, 1.0, norm, at(8192), need, nullptr) == ROCKET_OK);
        CHECK(rocket_grad_clip(g.data(), nullptr, n, 1.0, norm, at(8192), need, nullptr) == ROCKET_OK);
        CHECK(rocket_sgd_tensors(p.data(), g.data(), q.data(), n, 0.1, norm, nullptr) == ROCKET_OK);
        CHECK(rocket_sgd_tensors(p.data(), g.data(), nullptr, n, 0.1, nullptr, nullptr) == ROCKET_OK);
        if (n > 16) {
            int32_t i = 3, j = n - 2;
            while (g[i].count == 0) ++i;
            while (g[j].count == 0) --j;
            if (i < j) {
                o[j].data = o[i].data;
                CHECK(rocket_grad_clip(g.data(), o.data(), n, 1.0, norm, at(8192), need, nullptr) == ROCKET_EINVAL);
            }
        }
    }
    // the largest lists: 2^40 values, and one more
    rocket_tensor big[2] = {{at(1 << 20), (int64_t{1} << 40) - 5, ROCKET_BF16, 0}, {at(uint64_t{1} << 47), 5, ROCKET_F32, 0}};
    CHECK(rocket_grad_norm(big, 2, 1.0, norm, at(8192), size_t{1} << 30, nullptr) == ROCKET_OK);
    CHECK(rocket_grad_clip(big, nullptr, 2, 1.0, norm, at(8192), size_t{1} << 30, nullptr) == ROCKET_OK);
    big[1].count = 6;
    CHECK(rocket_grad_norm(big, 2, 1.0, norm, at(8192), size_t{1} << 30, nullptr) == ROCKET_EINVAL);
    big[1] = {at(uint64_t{1} << 48), 5, ROCKET_F32, 0};
    CHECK(rocket_grad_norm(big, 2, 1.0, norm, at(8192), size_t{1} << 30, nullptr) == ROCKET_EINVAL);
    big[1].count = 0;
    CHECK(rocket_grad_norm(big, 2, 1.0, norm, at(8192), size_t{1} << 30, nullptr) == ROCKET_OK);
    // the layer norm: every way a row is held, and the limits
    const void *x = at(1 << 20);
    const float *w = static_cast<const float *>(at(1 << 24));
    float *f = static_cast<float *>(at(1 << 25));
    for (int32_t type : {ROCKET_F32, ROCKET_BF16, ROCKET_F16})
        for (int32_t n : {1, 3, 4, 16, 17, 33, 65, 257, 500, 1025, 2049, 4097, 10000, 16385, 20480, 20481, 33000, 65537, 131073, 1000003, 1 << 30})
            for (int32_t rows : {1, 7, 16, 300, 4099, 1 << 30, 2147483647})
                for (int32_t planes : {1, 3, 65535}) {
                    if (static_cast<double>(rows) * planes * n > 3e11) continue;       // more than the card holds
                    const size_t fw = rocket_layer_norm_workspace_bytes(rows, planes, n, 0), bw = rocket_layer_norm_workspace_bytes(rows, planes, n, 1);
                    CHECK(bw >= 256 && bw % 256 == 0 && fw % 256 == 0);
                    CHECK(rocket_layer_norm(x, type, rows, planes, n, w, w, 1e-5f, at(1 << 26), f, f, fw ? at(1 << 27) : nullptr, fw, nullptr) == ROCKET_OK);
                    CHECK(rocket_layer_norm_backward(x, x, type, rows, planes, n, w, w, w, at(1 << 26), f, f, at(1 << 27), bw, nullptr) == ROCKET_OK);
                }
    CHECK(g_launches > 1000 && g_lanes > 0);
    std::printf("lists driver: ok\n");
    return 0;
}
