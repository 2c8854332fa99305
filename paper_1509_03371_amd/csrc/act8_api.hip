// Host side of activations in 8 bits, root-mean-square norm and the weight gradient over inputs in 8 bits.  See include/sknet.h for the contract.
#include <cmath>
#include <utility>

#include "act8.h"
#include "operand_checks.h"

namespace {

// What a call reads or writes: lines of `line` bytes, `images` times `maps` of them.
struct Operand {
    const char *name;
    const void *p;
    __int128 line;
    Steps images, maps;
    bool result;
    const sk_view *view;
    __int128 at() const { return reinterpret_cast<uintptr_t>(p); }
    __int128 end() const { return at() + (images.len - 1) * images.stride + (maps.len - 1) * maps.stride + line; }
    bool same(const Operand &o) const
    {
        return images.len == o.images.len && maps.len == o.maps.len && images.stride == o.images.stride && maps.stride == o.maps.stride;
    }
    // no two lines of `span` bytes at these places share one
    bool apart(__int128 span) const
    {
        const Steps &wide = images.stride >= maps.stride ? images : maps, &narrow = images.stride >= maps.stride ? maps : images;
        return (narrow.len == 1 || narrow.stride >= span) && (wide.len == 1 || wide.stride >= (narrow.len - 1) * narrow.stride + span);
    }
};

Steps steps(int64_t len, __int128 stride) { return {len, len == 1 ? 0 : stride}; }

Operand lines(const char *name, const void *p, const sk_extent &e, int64_t c, int64_t stride_n, int64_t stride_c, int64_t size, bool blocks, bool result)
{
    const bool rows = e.layout == SK_ROWS;
    const int64_t length = rows ? c : e.plane;
    return {name, p, (__int128)(blocks ? (length + 31) / 32 : length) * size, steps(e.n, (__int128)stride_n * size), steps(rows ? 1 : c, rows ? 0 : (__int128)stride_c * size), result, nullptr};
}

Operand flat(const char *name, const void *p, __int128 bytes, bool result) { return {name, p, bytes, {1, 0}, {1, 0}, result, nullptr}; }

// Do two operands share no byte?  Exact for lines at equal distances, else by ranges.
bool disjoint(const Operand &a, const Operand &b)
{
    if (a.end() <= b.at() || b.end() <= a.at()) return true;
    const __int128 span = a.line > b.line ? a.line : b.line;
    if (!a.same(b) || !a.apart(span)) return false;
    Steps wide = a.images, narrow = a.maps;
    if (wide.stride < narrow.stride) std::swap(wide, narrow);
    return !some_step(b.at() - a.at(), wide, [&](__int128 r) { return some_step(r, narrow, [&](__int128 d) { return d > -b.line && d < a.line; }); });
}

// The operands of a call; results share nothing with the others, but where one may take another's place.
class Operands {
public:
    explicit Operands(const char *who, const sk_extent &e) : who_(who), e_(e) {}
    sk_status view(const char *name, const sk_view *v, bool result, int64_t c = 0)
    {
        if (!v) return SK_OK;
        sk_extent e = e_;
        if (c) e.c = c;
        SK_TRY(check_view(who_, name, e, v, result));
        add(lines(name, v->data, e, e.c, v->stride_n, v->stride_c, element_bytes(e), false, result));
        all_[count_ - 1].view = v;
        return SK_OK;
    }
    sk_status packed(const char *name, const sk_packed *p, bool result)
    {
        if (!p) return SK_OK;
        if (p->code != SK_E4M3 && p->code != SK_I8) return fail(SK_EINVAL, "%s: %s: bad code", who_, name);
        if (!p->codes || !p->scales) return fail(SK_EINVAL, "%s: %s has no data", who_, name);
        const struct { const void *p; int64_t sn, sc; bool blocks; } both[] = {{p->codes, p->stride_n, p->stride_c, false}, {p->scales, p->scale_stride_n, p->scale_stride_c, true}};
        for (const auto &o : both) {
            if (o.sn < 0 || (e_.layout == SK_MAPS && o.sc < 0)) return fail(SK_ESHAPE, "%s: %s has a negative stride", who_, name);
            const Operand l = lines(name, o.p, e_, e_.c, o.sn, o.sc, 1, o.blocks, result);
            if (l.end() - l.at() > kMaxElements) return fail(SK_EUNSUPPORTED, "%s: %s reaches over more than 2^46 bytes", who_, name);
            if (result && !l.apart(l.line)) return fail(SK_ESHAPE, "%s: lines of %s overlap", who_, name);
            add(l);
        }
        return SK_OK;
    }
    sk_status values(const char *name, const float *p, __int128 count, bool result)
    {
        if (!p) return SK_OK;
        if (reinterpret_cast<uintptr_t>(p) % 4) return fail(SK_EINVAL, "%s: %s is not aligned to its elements", who_, name);
        add(flat(name, p, 4 * count, result));
        return SK_OK;
    }
    sk_status workspace(const void *p, uint64_t bytes, uint64_t need)
    {
        if (need && (!p || bytes < need)) return fail(SK_EINVAL, "%s: needs a workspace of %llu bytes", who_, (unsigned long long)need);
        if (reinterpret_cast<uintptr_t>(p) % 16) return fail(SK_EINVAL, "%s: the workspace is not aligned to 16 bytes", who_);
        if (need) add(flat("the workspace", p, need, true));
        return SK_OK;
    }
    // places: views that an input may give to a result, element for element
    sk_status settle(std::initializer_list<const sk_view *> places = {}) const
    {
        for (int i = 0; i < count_; ++i)
            for (int j = 0; j < count_; ++j) {
                const Operand &a = all_[i], &b = all_[j];
                if (i == j || !a.result || (b.result && j < i) || disjoint(a, b)) continue;
                bool place = false;
                if (a.view && !b.result && a.p == b.p && a.line == b.line && a.same(b))
                    for (const sk_view *v : places) place |= v && v == b.view;
                if (!place) return fail(SK_EINVAL, "%s: %s overlaps %s", who_, a.name, b.name);
            }
        return SK_OK;
    }

private:
    const char *who_;
    const sk_extent &e_;
    static constexpr int kMost = 16;                    // a call has no more operands than this, codes and scales apart
    Operand all_[kMost];
    int count_ = 0;
    void add(const Operand &o) { all_[count_++] = o; }
};

sk::PackedView take_packed(const sk_packed *p)
{
    sk::PackedView o;
    if (p) {
        o.codes = p->codes; o.scales = p->scales;
        o.sn = p->stride_n; o.sc = p->stride_c;
        o.ssn = p->scale_stride_n; o.ssc = p->scale_stride_c;
        o.code = p->code == SK_E4M3 ? sk::E4M3 : sk::I8;
    }
    return o;
}

sk_status check_c_out(const char *who, const sk_extent &e, int64_t c_out)
{
    if (c_out < 1) return fail(SK_ESHAPE, "%s: needs at least one output channel", who);
    if (c_out > kMaxChannels || (__int128)e.c * c_out > kMaxPositions) return fail(SK_EUNSUPPORTED, "%s: more than 2^27 output channels or 2^40 weights", who);
    if ((__int128)e.n * e.plane * c_out > kMaxElements) return fail(SK_EUNSUPPORTED, "%s: more than 2^46 elements", who);
    return SK_OK;
}

sk_status change8(const char *who, const sk_extent *extent, const sk_view *x, const sk_packed *packed, bool pack, void *hip_stream)
{
    bool empty = false;
    SK_TRY(check_extent(who, extent, &empty));
    if (!x || !packed) return fail(SK_EINVAL, "%s: null argument", who);
    if (packed->code != SK_E4M3 && packed->code != SK_I8) return fail(SK_EINVAL, "%s: bad code", who);
    if (empty) return SK_OK;
    Operands all(who, *extent);
    SK_TRY(all.view(pack ? "x" : "y", x, !pack));
    SK_TRY(all.packed("packed", packed, pack));
    SK_TRY(all.settle());
    sk::Pack8Args a{};
    take_span(*extent, &a);
    a.x = take_view(x);
    a.packed = take_packed(packed);
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    SK_HIP(pack ? sk::launch_pack8(a, stream) : sk::launch_unpack8(a, stream));
    return SK_OK;
}

}  // namespace

extern "C" {

sk_status sknet_pack8(const sk_extent *extent, const sk_view *x, const sk_packed *packed, void *hip_stream)
{
    return change8("pack8", extent, x, packed, true, hip_stream);
}

sk_status sknet_unpack8(const sk_extent *extent, const sk_packed *packed, const sk_view *y, void *hip_stream)
{
    return change8("unpack8", extent, y, packed, false, hip_stream);
}

sk_status sknet_rms_norm(const sk_extent *extent, const sk_view *x, const sk_view *residual, const float *gamma_dev, float eps, const sk_view *sum,
                         const sk_packed *sum8, const sk_view *y, const sk_packed *y8, float *rstd_dev, void *hip_stream)
{
    const char *who = "rms_norm";
    bool empty = false;
    SK_TRY(check_extent(who, extent, &empty));
    if (!x) return fail(SK_EINVAL, "%s: null argument", who);
    if (!sum && !sum8 && !y && !y8 && !rstd_dev) return fail(SK_EINVAL, "%s: no result is asked for", who);
    if (!(eps > 0.f) || !std::isfinite(eps)) return fail(SK_EINVAL, "%s: eps must be positive and finite", who);
    if (empty) return SK_OK;
    const sk_extent &e = *extent;
    Operands all(who, e);
    SK_TRY(all.view("x", x, false));
    SK_TRY(all.view("residual", residual, false));
    SK_TRY(all.view("sum", sum, true));
    SK_TRY(all.packed("sum8", sum8, true));
    SK_TRY(all.view("y", y, true));
    SK_TRY(all.packed("y8", y8, true));
    SK_TRY(all.values("gamma", gamma_dev, e.c, false));
    SK_TRY(all.values("rstd", rstd_dev, (__int128)e.n * e.plane, true));
    SK_TRY(all.settle({x, residual}));
    sk::RmsArgs a{};
    take_span(e, &a);
    a.x = take_view(x);
    a.residual = take_view(residual);
    a.sum = take_view(sum);
    a.sum8 = take_packed(sum8);
    a.y = take_view(y);
    a.y8 = take_packed(y8);
    a.gamma = gamma_dev; a.rstd = rstd_dev; a.eps = eps;
    SK_HIP(sk::launch_rms_norm(a, static_cast<hipStream_t>(hip_stream)));
    return SK_OK;
}

sk_status sknet_rms_norm_workspace(const sk_extent *extent, uint64_t *bytes)
{
    bool empty = false;
    if (!bytes) return fail(SK_EINVAL, "rms_norm_workspace: bytes is null");
    SK_TRY(check_extent("rms_norm_workspace", extent, &empty));
    sk::NormSpan s{};
    take_span(*extent, &s);
    *bytes = empty ? 0 : sizeof(float) * (uint64_t)sk::rms_bwd_scratch_floats(s);
    return SK_OK;
}

sk_status sknet_rms_norm_backward(const sk_extent *extent, const sk_view *dy, const sk_view *s, const sk_packed *s8, const float *rstd_dev,
                                  const float *gamma_dev, const sk_view *dsum, const sk_view *dx, float *dgamma_dev, void *workspace_dev,
                                  uint64_t workspace_bytes, void *hip_stream)
{
    const char *who = "rms_norm_backward";
    bool empty = false;
    SK_TRY(check_extent(who, extent, &empty));
    if (!dy || !s == !s8) return fail(SK_EINVAL, "%s: needs dy, and either s or s8", who);
    const sk_extent &e = *extent;
    sk::RmsBwdArgs a{};
    take_span(e, &a);
    Operands all(who, e);
    SK_TRY(all.values("dgamma", dgamma_dev, e.c, true));
    SK_TRY(all.values("gamma", gamma_dev, e.c, false));
    if (!empty) {
        if (!rstd_dev) return fail(SK_EINVAL, "%s: needs the forward pass's rstd", who);
        SK_TRY(all.view("dy", dy, false));
        SK_TRY(all.view("s", s, false));
        SK_TRY(all.packed("s8", s8, false));
        SK_TRY(all.view("dsum", dsum, false));
        SK_TRY(all.view("dx", dx, true));
        SK_TRY(all.values("rstd", rstd_dev, (__int128)e.n * e.plane, false));
        const uint64_t need = dgamma_dev ? sizeof(float) * (uint64_t)sk::rms_bwd_scratch_floats(a) : 0;
        SK_TRY(all.workspace(workspace_dev, workspace_bytes, need));
        a.dy = take_view(dy);
        a.s = take_view(s);
        a.s8 = take_packed(s8);
        a.dsum = take_view(dsum);
        a.dx = take_view(dx);
        a.rstd = rstd_dev;
        a.scratch = static_cast<float *>(workspace_dev);
    }
    SK_TRY(all.settle({dy, s, dsum}));
    a.gamma = gamma_dev;
    a.dgamma = dgamma_dev;
    SK_HIP(sk::launch_rms_norm_bwd(a, static_cast<hipStream_t>(hip_stream)));
    return SK_OK;
}

sk_status sknet_weight_gradient8_workspace(const sk_extent *extent, int64_t c_out, uint64_t *bytes)
{
    const char *who = "weight_gradient8_workspace";
    bool empty = false;
    if (!bytes) return fail(SK_EINVAL, "%s: bytes is null", who);
    SK_TRY(check_extent(who, extent, &empty));
    SK_TRY(check_c_out(who, *extent, c_out));
    sk::NormSpan s{};
    take_span(*extent, &s);
    *bytes = empty ? 0 : sizeof(float) * (uint64_t)sk::wgrad8_scratch_floats(s, c_out);
    return SK_OK;
}

sk_status sknet_weight_gradient8(const sk_extent *extent, int64_t c_out, const sk_view *dy, const sk_packed *x, int32_t accumulate, float *dw_dev,
                                 float *db_dev, void *workspace_dev, uint64_t workspace_bytes, void *hip_stream)
{
    const char *who = "weight_gradient8";
    bool empty = false;
    SK_TRY(check_extent(who, extent, &empty));
    if (!dy || !x || !dw_dev) return fail(SK_EINVAL, "%s: null argument", who);
    const sk_extent &e = *extent;
    SK_TRY(check_c_out(who, e, c_out));
    sk::Wgrad8Args a{};
    take_span(e, &a);
    Operands all(who, e);
    SK_TRY(all.values("dw", dw_dev, (__int128)c_out * e.c, true));
    SK_TRY(all.values("db", db_dev, c_out, true));
    if (!empty) {
        SK_TRY(all.view("dy", dy, false, c_out));
        SK_TRY(all.packed("x", x, false));
        const uint64_t need = sizeof(float) * (uint64_t)sk::wgrad8_scratch_floats(a, c_out);
        SK_TRY(all.workspace(workspace_dev, workspace_bytes, need));
        a.dy = take_view(dy);
        a.x = take_packed(x);
        a.scratch = static_cast<float *>(workspace_dev);
    }
    SK_TRY(all.settle());
    a.c_out = c_out;
    a.accumulate = accumulate != 0;
    a.dw = dw_dev; a.db = db_dev;
    SK_HIP(sk::launch_wgrad8(a, static_cast<hipStream_t>(hip_stream)));
    return SK_OK;
}

}  // extern "C"
