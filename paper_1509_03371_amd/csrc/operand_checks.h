// Checks of the operators' arguments: extents, views of a caller's tensors and how they lie to one another (host side, internal to libsknet).
#pragma once
#include "norm.h"
#include "sk_host.h"

namespace {

using namespace skh;

constexpr int64_t kMaxChannels = (int64_t)1 << 27;       // what the counter of the generator has room for
constexpr int64_t kMaxPositions = (int64_t)1 << 40;
constexpr int64_t kMaxElements = (int64_t)1 << 46;       // byte offsets then stay far from 2^63

// a positions-by-channels range of memory, in elements from the view's first
__int128 last_element(const sk_extent &e, const sk_view &v)
{
    __int128 last = (__int128)(e.n - 1) * v.stride_n;
    if (e.layout == SK_ROWS) return last + e.c - 1;
    return last + (__int128)(e.c - 1) * v.stride_c + e.plane - 1;
}

int64_t element_bytes(const sk_extent &e) { return e.dtype == SK_F32 ? 4 : 2; }

sk_status check_extent(const char *who, const sk_extent *e, bool *empty)
{
    if (!e) return fail(SK_EINVAL, "%s: null extent", who);
    if (e->dtype != SK_F32 && e->dtype != SK_BF16 && e->dtype != SK_F16) return fail(SK_EINVAL, "%s: bad dtype", who);
    if (e->layout != SK_ROWS && e->layout != SK_MAPS) return fail(SK_EINVAL, "%s: layout must be SK_ROWS or SK_MAPS", who);
    if (e->n < 0 || e->plane < 0) return fail(SK_ESHAPE, "%s: negative size", who);
    if (e->c < 1) return fail(SK_ESHAPE, "%s: needs at least one channel", who);
    if (e->layout == SK_ROWS && e->plane != 1) return fail(SK_ESHAPE, "%s: rows have plane = 1", who);
    if (e->c > kMaxChannels) return fail(SK_EUNSUPPORTED, "%s: more than 2^27 channels", who);
    if ((__int128)e->n * e->plane > kMaxPositions || (__int128)e->n * e->plane * e->c > kMaxElements)
        return fail(SK_EUNSUPPORTED, "%s: more than 2^40 positions or 2^46 elements", who);
    *empty = e->n == 0 || e->plane == 0;
    return SK_OK;
}

// strides that reach every element in range; of an output, each element at a place of its own
sk_status check_view(const char *who, const char *what, const sk_extent &e, const sk_view *v, bool output)
{
    if (!v->data) return fail(SK_EINVAL, "%s: %s has no data", who, what);
    if (reinterpret_cast<uintptr_t>(v->data) % element_bytes(e)) return fail(SK_EINVAL, "%s: %s is not aligned to its elements", who, what);
    if (v->stride_n < 0 || (e.layout == SK_MAPS && v->stride_c < 0)) return fail(SK_ESHAPE, "%s: %s has a negative stride", who, what);
    if (last_element(e, *v) > kMaxElements) return fail(SK_EUNSUPPORTED, "%s: %s reaches over more than 2^46 elements", who, what);
    if (!output) return SK_OK;
    bool apart;
    if (e.layout == SK_ROWS) {
        apart = e.n == 1 || v->stride_n >= e.c;
    } else {
        const bool images_outside = (e.c == 1 || v->stride_c >= e.plane) && (e.n == 1 || v->stride_n >= (__int128)(e.c - 1) * v->stride_c + e.plane);
        const bool maps_outside = (e.n == 1 || v->stride_n >= e.plane) && (e.c == 1 || v->stride_c >= (__int128)(e.n - 1) * v->stride_n + e.plane);
        apart = images_outside || maps_outside;
    }
    if (!apart) return fail(SK_ESHAPE, "%s: elements of %s overlap", who, what);
    return SK_OK;
}

// `len` places, `stride` bytes apart
struct Steps {
    __int128 len, stride;
};

// Is there an i of -(len - 1) .. len - 1 with f(far - i stride), which can hold only where its argument lies within (-reach, reach)?  Two at
// most come into question: the places of a step lie at least `reach` apart.
template <class F> bool some_step(__int128 far, const Steps &s, F f)
{
    if (s.len == 1) return f(far);
    const __int128 down = far >= 0 ? far / s.stride : -((-far + s.stride - 1) / s.stride);
    for (__int128 i = down; i <= down + 1; ++i)
        if (i > -s.len && i < s.len && f(far - i * s.stride)) return true;
    return false;
}

void take_span(const sk_extent &e, sk::NormSpan *s)
{
    s->dtype = e.dtype;
    s->layout = e.layout == SK_ROWS ? sk::ROWS : sk::MAPS;
    s->n = e.n; s->plane = e.plane; s->c = (int)e.c;
}

sk::NormView take_view(const sk_view *v)
{
    sk::NormView o;
    if (v) { o.p = v->data; o.sn = v->stride_n; o.sc = v->stride_c; }
    return o;
}

}  // namespace
