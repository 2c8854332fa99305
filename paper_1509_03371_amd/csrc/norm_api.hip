// Host side of the operators on a caller's tensors: dropout and layer norm.  See include/sknet.h for the contract.
#include <cmath>
#include <utility>

#include "operand_checks.h"

namespace {

bool same_strides(const sk_extent &e, const sk_view &a, const sk_view &b)
{
    return (e.n == 1 || a.stride_n == b.stride_n) && (e.layout == SK_ROWS || e.c == 1 || a.stride_c == b.stride_c);
}

// Do two views share no element?  True where their ranges of memory are apart, and with equal strides where no difference i stride_n + j stride_c of two
// places brings their lines together.  With equal strides one of the two must have elements apart (an output).
bool disjoint(const sk_extent &e, const sk_view &a, const sk_view &b)
{
    const int64_t size = element_bytes(e);
    const __int128 a0 = reinterpret_cast<uintptr_t>(a.data), b0 = reinterpret_cast<uintptr_t>(b.data);
    const __int128 a1 = a0 + (last_element(e, a) + 1) * size, b1 = b0 + (last_element(e, b) + 1) * size;
    if (a1 <= b0 || b1 <= a0) return true;
    if (!same_strides(e, a, b)) return false;
    const bool rows = e.layout == SK_ROWS;
    const __int128 line = (rows ? e.c : e.plane) * (__int128)size;
    Steps images = {e.n, e.n == 1 ? 0 : (__int128)a.stride_n * size}, maps = {rows || e.c == 1 ? 1 : e.c, rows || e.c == 1 ? 0 : (__int128)a.stride_c * size};
    if (images.stride < maps.stride) std::swap(images, maps);       // the wider step first: it spans all of the other's
    return !some_step(b0 - a0, images, [&](__int128 r) { return some_step(r, maps, [&](__int128 d) { return d > -line && d < line; }); });
}

// an output may be an input's buffer, element for element; any other overlap is refused
sk_status check_in_place(const char *who, const sk_extent &e, const char *out_name, const sk_view *out, const char *in_name, const sk_view *in)
{
    if (!out || !in) return SK_OK;
    if (out->data == in->data && same_strides(e, *out, *in)) return SK_OK;
    if (!disjoint(e, *out, *in)) return fail(SK_EINVAL, "%s: %s overlaps %s without being the same tensor", who, out_name, in_name);
    return SK_OK;
}

sk_status check_apart(const char *who, const sk_extent &e, const char *a_name, const sk_view *a, const char *b_name, const sk_view *b)
{
    if (!a || !b || disjoint(e, *a, *b)) return SK_OK;
    return fail(SK_EINVAL, "%s: %s and %s overlap", who, a_name, b_name);
}

// fp32 values beside the views: parameters, statistics, their gradients
struct Values {
    const char *name;
    const void *p;
    int64_t bytes;
    bool output;
};

// aligned to their elements, and what is written shares no place with the others
template <int N>
sk_status check_values(const char *who, const Values (&v)[N])
{
    for (const Values &a : v) {
        if (reinterpret_cast<uintptr_t>(a.p) % 4) return fail(SK_EINVAL, "%s: %s is not aligned to its elements", who, a.name);
        if (!a.p || !a.output) continue;
        const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p);
        for (const Values &b : v) {
            const uintptr_t b0 = reinterpret_cast<uintptr_t>(b.p);
            if (&a != &b && b.p && a0 < b0 + b.bytes && b0 < a0 + a.bytes) return fail(SK_EINVAL, "%s: %s and %s overlap", who, a.name, b.name);
        }
    }
    return SK_OK;
}

sk_status take_mask(const char *who, const sk_drop *d, sk::DropMask *m)
{
    if (!d) return SK_OK;
    if (!(d->p >= 0.0 && d->p <= 1.0)) return fail(SK_EINVAL, "%s: the rate must be in [0, 1]", who);
    if (reinterpret_cast<uintptr_t>(d->step_dev) % 8) return fail(SK_EINVAL, "%s: step_dev is not aligned to 8 bytes", who);
    m->thresh = (uint32_t)(d->p * 65536.0 + 0.5);
    m->scale = m->thresh >= 65536 ? 0.f : (float)(65536.0 / (65536.0 - m->thresh));
    m->seed = d->seed; m->offset = d->offset; m->step = d->step_dev;
    return SK_OK;
}

}  // namespace

extern "C" {

sk_status sknet_dropout(const sk_extent *extent, const sk_view *x, const sk_view *y, const sk_drop *drop, void *hip_stream)
{
    const char *who = "dropout";
    bool empty = false;
    SK_TRY(check_extent(who, extent, &empty));
    if (!x || !y || !drop) return fail(SK_EINVAL, "%s: null argument", who);
    sk::DropoutArgs a{};
    SK_TRY(take_mask(who, drop, &a.drop));
    if (empty) return SK_OK;
    SK_TRY(check_view(who, "x", *extent, x, false));
    SK_TRY(check_view(who, "y", *extent, y, true));
    SK_TRY(check_in_place(who, *extent, "y", y, "x", x));
    take_span(*extent, &a);
    a.x = take_view(x);
    a.y = take_view(y);
    SK_HIP(sk::launch_dropout(a, static_cast<hipStream_t>(hip_stream)));
    return SK_OK;
}

sk_status sknet_layer_norm(const sk_extent *extent, const sk_view *x, const sk_view *residual, const sk_drop *drop, const float *gamma_dev,
                           const float *beta_dev, float eps, const sk_view *sum, const sk_view *y, float *mean_dev, float *rstd_dev,
                           void *hip_stream)
{
    const char *who = "layer_norm";
    bool empty = false;
    SK_TRY(check_extent(who, extent, &empty));
    if (!x || !y) return fail(SK_EINVAL, "%s: null argument", who);
    if (!(eps > 0.f) || !std::isfinite(eps)) return fail(SK_EINVAL, "%s: eps must be positive and finite", who);
    sk::NormArgs a{};
    SK_TRY(take_mask(who, drop, &a.drop));
    if (empty) return SK_OK;
    const sk_extent &e = *extent;
    SK_TRY(check_view(who, "x", e, x, false));
    if (residual) SK_TRY(check_view(who, "residual", e, residual, false));
    if (sum) SK_TRY(check_view(who, "sum", e, sum, true));
    SK_TRY(check_view(who, "y", e, y, true));
    SK_TRY(check_apart(who, e, "y", y, "sum", sum));
    SK_TRY(check_in_place(who, e, "y", y, "x", x));
    SK_TRY(check_in_place(who, e, "y", y, "residual", residual));
    SK_TRY(check_in_place(who, e, "sum", sum, "x", x));
    SK_TRY(check_in_place(who, e, "sum", sum, "residual", residual));
    const int64_t line = 4 * e.c, positions = 4 * e.n * e.plane;
    const Values values[] = {{"gamma", gamma_dev, line, false}, {"beta", beta_dev, line, false}, {"mean", mean_dev, positions, true}, {"rstd", rstd_dev, positions, true}};
    SK_TRY(check_values(who, values));
    take_span(e, &a);
    a.x = take_view(x);
    a.residual = take_view(residual);
    a.sum = take_view(sum);
    a.y = take_view(y);
    a.gamma = gamma_dev; a.beta = beta_dev; a.mean = mean_dev; a.rstd = rstd_dev;
    a.eps = eps;
    SK_HIP(sk::launch_layer_norm(a, static_cast<hipStream_t>(hip_stream)));
    return SK_OK;
}

sk_status sknet_layer_norm_workspace(const sk_extent *extent, uint64_t *bytes)
{
    bool empty = false;
    if (!bytes) return fail(SK_EINVAL, "layer_norm_workspace: bytes is null");
    SK_TRY(check_extent("layer_norm_workspace", extent, &empty));
    sk::NormSpan s{};
    take_span(*extent, &s);
    *bytes = empty ? 0 : sizeof(float) * (uint64_t)sk::norm_bwd_scratch_floats(s);
    return SK_OK;
}

sk_status sknet_layer_norm_backward(const sk_extent *extent, const sk_view *dy, const sk_view *s, const float *mean_dev, const float *rstd_dev,
                                    const float *gamma_dev, const sk_view *dsum, const sk_drop *drop, const sk_view *dx, const sk_view *dresidual,
                                    float *dgamma_dev, float *dbeta_dev, void *workspace_dev, uint64_t workspace_bytes, void *hip_stream)
{
    const char *who = "layer_norm_backward";
    bool empty = false;
    SK_TRY(check_extent(who, extent, &empty));
    if (!dy || !s) return fail(SK_EINVAL, "%s: null argument", who);
    sk::NormBwdArgs a{};
    SK_TRY(take_mask(who, drop, &a.drop));
    const sk_extent &e = *extent;
    take_span(e, &a);
    a.dgamma = dgamma_dev; a.dbeta = dbeta_dev;
    if (!empty) {
        if (!mean_dev || !rstd_dev) return fail(SK_EINVAL, "%s: needs the forward pass's mean and rstd", who);
        SK_TRY(check_view(who, "dy", e, dy, false));
        SK_TRY(check_view(who, "s", e, s, false));
        if (dsum) SK_TRY(check_view(who, "dsum", e, dsum, false));
        if (dx) SK_TRY(check_view(who, "dx", e, dx, true));
        if (dresidual) SK_TRY(check_view(who, "dresidual", e, dresidual, true));
        SK_TRY(check_apart(who, e, "dx", dx, "dresidual", dresidual));
        const struct { const char *name; const sk_view *v; } outs[] = {{"dx", dx}, {"dresidual", dresidual}}, ins[] = {{"dy", dy}, {"s", s}, {"dsum", dsum}};
        for (const auto &o : outs)
            for (const auto &i : ins) SK_TRY(check_in_place(who, e, o.name, o.v, i.name, i.v));
        const bool wants_sums = dgamma_dev || dbeta_dev;
        const uint64_t need = wants_sums ? sizeof(float) * (uint64_t)sk::norm_bwd_scratch_floats(a) : 0;
        if (need && (!workspace_dev || workspace_bytes < need))
            return fail(SK_EINVAL, "%s: needs a workspace of %llu bytes", who, (unsigned long long)need);
        if (reinterpret_cast<uintptr_t>(workspace_dev) % 16) return fail(SK_EINVAL, "%s: the workspace is not aligned to 16 bytes", who);
        const int64_t line = 4 * e.c, positions = 4 * e.n * e.plane;
        const Values values[] = {{"mean", mean_dev, positions, false}, {"rstd", rstd_dev, positions, false}, {"gamma", gamma_dev, line, false},
                                 {"dgamma", dgamma_dev, line, true}, {"dbeta", dbeta_dev, line, true}, {"the workspace", workspace_dev, (int64_t)need, true}};
        SK_TRY(check_values(who, values));
        a.dy = take_view(dy);
        a.s = take_view(s);
        a.dsum = take_view(dsum);
        a.dx = take_view(dx);
        a.dresidual = take_view(dresidual);
        a.mean = mean_dev; a.rstd = rstd_dev; a.gamma = gamma_dev;
        a.scratch = static_cast<float *>(workspace_dev);
        a.scratch_floats = (size_t)(need / sizeof(float));
    }
    SK_HIP(sk::launch_layer_norm_bwd(a, static_cast<hipStream_t>(hip_stream)));
    return SK_OK;
}

}  // extern "C"
