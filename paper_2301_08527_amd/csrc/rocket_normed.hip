// ROCKET transform for MI355X (gfx950): inference and training with a layer norm between the features and the linear head.
// Sequences of the library's own calls on one stream; the contract is in include/rocket.h.
#include <algorithm>
#include <cmath>
#include <string>

#include "rocket_internal.hpp"

namespace {

size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// The parts of the workspace, each on a multiple of 256 bytes.  `inner` is the scratch memory of one call at a time: transform,
// layer norm, backward pass, gradient norm.
struct Layout {
    size_t inner = 0, feats = 0, gout = 0, pred = 0, mean = 0, rstd = 0, gw = 0, gb = 0, gnw = 0, gnb = 0, norm = 0, total = 0;
    int32_t F = 0;
    rocket_tensor grads[4] = {};

    Layout(const rocket_kernels *h, int32_t B, uint32_t mask, bool training)
    {
        F = rocket_num_features(mask);
        const size_t p = static_cast<size_t>(F) * h->K, b = static_cast<size_t>(B);
        inner = std::max(rocket_workspace_bytes(h, B, mask, 0), rocket_layer_norm_workspace_bytes(B, F, h->K, 0));
        feats = up256(inner);
        if (!training) {
            total = feats + up256(b * p * 4);
            return;
        }
        grads[0].count = h->w_off[h->K];
        grads[1].count = h->K;
        grads[2].count = grads[3].count = static_cast<int64_t>(p);
        // (the addresses play no part in the size)
        for (rocket_tensor &t : grads) t.data = &t, t.dtype = ROCKET_F32;
        inner = std::max({inner, rocket_workspace_bytes(h, B, mask, 1), rocket_layer_norm_workspace_bytes(B, F, h->K, 1),
                          rocket_grad_workspace_bytes(grads, 4)});
        feats = up256(inner);
        gout = feats + up256(b * p * 4);
        pred = gout + up256(b * p * 4);
        mean = pred + up256(b * 8);
        rstd = mean + up256(b * F * 4);
        gw = rstd + up256(b * F * 4);
        gb = gw + up256(static_cast<size_t>(h->w_off[h->K]) * 4);
        gnw = gb + up256(static_cast<size_t>(h->K) * 4);
        gnb = gnw + up256(p * 4);
        norm = gnb + up256(p * 4);
        total = norm + 256;
    }
};

bool sizes_fit(const rocket_kernels *h, int32_t B, uint32_t mask) { return h && B >= 1 && rocket_num_features(mask) > 0; }

int check_workspace(const char *fn, size_t need, const void *ws, size_t ws_bytes)
{
    if (ws && ws_bytes >= need && reinterpret_cast<uintptr_t>(ws) % 16 == 0) return ROCKET_OK;
    return rk_fail(ROCKET_EWORKSPACE, std::string(fn) + ": an aligned workspace of " + std::to_string(need) + " bytes required");
}

int transform(rocket_kernels *h, const void *x, int x_is_u8, int32_t B, uint32_t mask, float lambda, float shift, float *out, void *ws, size_t bytes,
              void *stream)
{
    return x_is_u8 ? rocket_transform_u8(h, static_cast<const uint8_t *>(x), B, mask, lambda, shift, out, ws, bytes, stream)
                   : rocket_transform(h, static_cast<const float *>(x), B, mask, lambda, shift, out, ws, bytes, stream);
}

bool usable_eps(float eps) { return std::isfinite(eps) && eps > 0.f; }

}  // namespace

extern "C" size_t rocket_infer_normed_workspace_bytes(const rocket_kernels *h, int32_t B, uint32_t mask)
{
    return sizes_fit(h, B, mask) ? Layout(h, B, mask, false).total : 0;
}

extern "C" int rocket_infer_normed(rocket_kernels *h, const void *x_dev, int x_is_u8, int32_t B, uint32_t mask, float lambda, float shift,
                                   const float *norm_weight_dev, const float *norm_bias_dev, float eps, const double *coef_dev,
                                   const double *intercept_dev, float *features_dev, double *pred_dev, void *ws, size_t ws_bytes,
                                   void *hip_stream)
{
    const char *fn = "rocket_infer_normed";
    if (!sizes_fit(h, B, mask)) return rk_fail(ROCKET_EINVAL, std::string(fn) + ": a handle, B >= 1 and a feature mask required");
    if (!x_dev || !coef_dev || !intercept_dev || !features_dev || !pred_dev) return rk_fail(ROCKET_EINVAL, std::string(fn) + ": NULL pointer");
    if (!usable_eps(eps)) return rk_fail(ROCKET_EINVAL, std::string(fn) + ": eps must be positive and finite");
    const Layout t(h, B, mask, false);
    int rc = check_workspace(fn, t.total, ws, ws_bytes);
    if (rc != ROCKET_OK) return rc;
    float *feats = reinterpret_cast<float *>(static_cast<char *>(ws) + t.feats);
    rc = transform(h, x_dev, x_is_u8, B, mask, lambda, shift, feats, ws, t.inner, hip_stream);
    if (rc != ROCKET_OK) return rc;
    rc = rocket_layer_norm(feats, ROCKET_F32, B, t.F, h->K, norm_weight_dev, norm_bias_dev, eps, features_dev, nullptr, nullptr, ws, t.inner, hip_stream);
    if (rc != ROCKET_OK) return rc;
    return rocket_ridge_predict(features_dev, B, t.F * h->K, coef_dev, intercept_dev, pred_dev, hip_stream);
}

extern "C" size_t rocket_train_normed_workspace_bytes(const rocket_kernels *h, int32_t B, uint32_t mask)
{
    return sizes_fit(h, B, mask) ? Layout(h, B, mask, true).total : 0;
}

extern "C" int rocket_train_step_normed(rocket_kernels *h, const void *x_dev, int x_is_u8, int32_t B, uint32_t mask, float lambda, float shift,
                                        float *norm_weight_dev, float *norm_bias_dev, float eps, const double *coef_dev,
                                        const double *intercept_dev, const float *targets_dev, float lr, int recentre, double max_norm,
                                        double *loss_dev, double *norm_dev, void *ws, size_t ws_bytes, void *hip_stream)
{
    const std::string who = "rocket_train_step_normed: ";
    if (!sizes_fit(h, B, mask) || !(mask & ROCKET_F_SOFTPPV) || B > 65535)
        return rk_fail(ROCKET_EINVAL, who + "a handle, B in [1, 65535] and a feature mask that contains ROCKET_F_SOFTPPV required");
    if (!x_dev || !norm_weight_dev || !norm_bias_dev || !coef_dev || !intercept_dev || !targets_dev) return rk_fail(ROCKET_EINVAL, who + "NULL pointer");
    if (!usable_eps(eps)) return rk_fail(ROCKET_EINVAL, who + "eps must be positive and finite");
    if (!std::isfinite(lr)) return rk_fail(ROCKET_EINVAL, who + "lr must be finite");
    if (!(max_norm > 0.0)) return rk_fail(ROCKET_EINVAL, who + "max_norm must be positive");
    Layout t(h, B, mask, true);
    int rc = check_workspace("rocket_train_step_normed", t.total, ws, ws_bytes);
    if (rc != ROCKET_OK) return rc;
    char *base = static_cast<char *>(ws);
    const auto f32 = [&](size_t at) { return reinterpret_cast<float *>(base + at); };
    double *pred = reinterpret_cast<double *>(base + t.pred);
    double *norm = norm_dev ? norm_dev : reinterpret_cast<double *>(base + t.norm);
    const int32_t p = t.F * h->K;
    // `gout` holds the normalised features until they are predicted from, then their gradient, then the features' gradient
    rc = transform(h, x_dev, x_is_u8, B, mask, lambda, shift, f32(t.feats), ws, t.inner, hip_stream);
    if (rc == ROCKET_OK)
        rc = rocket_layer_norm(f32(t.feats), ROCKET_F32, B, t.F, h->K, norm_weight_dev, norm_bias_dev, eps, f32(t.gout), f32(t.mean), f32(t.rstd), ws, t.inner,
                               hip_stream);
    if (rc == ROCKET_OK) rc = rocket_ridge_predict(f32(t.gout), B, p, coef_dev, intercept_dev, pred, hip_stream);
    if (rc == ROCKET_OK) rc = rocket_mse_grad(pred, targets_dev, coef_dev, B, p, f32(t.gout), loss_dev, hip_stream);
    if (rc == ROCKET_OK)
        rc = rocket_layer_norm_backward(f32(t.feats), f32(t.gout), ROCKET_F32, B, t.F, h->K, norm_weight_dev, f32(t.mean), f32(t.rstd), f32(t.gout),
                                        f32(t.gnw), f32(t.gnb), ws, t.inner, hip_stream);
    const int include_max = (mask & ROCKET_F_MAX) ? 1 : 0;
    if (rc == ROCKET_OK)
        rc = x_is_u8 ? rocket_soft_ppv_backward_u8(h, static_cast<const uint8_t *>(x_dev), B, mask, f32(t.gout), lambda, shift, include_max, f32(t.gw),
                                                   f32(t.gb), ws, t.inner, hip_stream)
                     : rocket_soft_ppv_backward(h, static_cast<const float *>(x_dev), B, mask, f32(t.gout), lambda, shift, include_max, f32(t.gw),
                                                f32(t.gb), ws, t.inner, hip_stream);
    t.grads[0].data = f32(t.gw);
    t.grads[1].data = f32(t.gb);
    t.grads[2].data = f32(t.gnw);
    t.grads[3].data = f32(t.gnb);
    if (rc == ROCKET_OK) rc = rocket_grad_norm(t.grads, 4, max_norm, norm, ws, t.inner, hip_stream);
    rocket_tensor params[2] = {t.grads[2], t.grads[3]};
    params[0].data = norm_weight_dev;
    params[1].data = norm_bias_dev;
    // first the update that may still refuse its arguments (weights that overlap)
    if (rc == ROCKET_OK) rc = rocket_sgd_tensors(params, t.grads + 2, nullptr, 2, lr, norm, hip_stream);
    if (rc == ROCKET_OK) rc = rocket_sgd_update_clipped(h, f32(t.gw), f32(t.gb), lr, recentre, norm, hip_stream);
    return rc;
}
