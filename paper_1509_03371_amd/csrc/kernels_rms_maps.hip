// Root-mean-square norm of maps: the channels of a pixel a plane apart.
#include "rms_maps.h"

namespace sk {

namespace {

// s of an octet, zeros where there is nothing
template <int DT, int P, int V, bool FAR> __device__ __forceinline__ void sums_of(const Spot<DT, P, V, FAR> &t, const RmsArgs &a, int o, float (&s)[8][V])
{
    Words<DT, V> x[8], u[8];
    t.load(a.x, o, x);
    if (a.residual.p) t.load(a.residual, o, u);
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) s[j][i] = x[j][i];
    if (a.residual.p)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) s[j][i] += u[j][i];
}
template <int DT, int P, int V, bool FAR> __device__ __forceinline__ void put_maps(const Spot<DT, P, V, FAR> &t, const RmsArgs &a, int o, const float (&rstd)[V], float (&s)[8][V])
{
    // s, then y: one piece of code for both
#pragma unroll 1
    for (int last = 0; last < 2; ++last) {
        // (field by field: chosen as a whole, the arguments would be copied to memory first)
        const NormView view = {last ? a.y.p : a.sum.p, last ? a.y.sn : a.sum.sn, last ? a.y.sc : a.sum.sc};
        const PackedView packed = {last ? a.y8.codes : a.sum8.codes, last ? a.y8.scales : a.sum8.scales, last ? a.y8.sn : a.sum8.sn, last ? a.y8.sc : a.sum8.sc,
                                   last ? a.y8.ssn : a.sum8.ssn, last ? a.y8.ssc : a.sum8.ssc, last ? a.y8.code : a.sum8.code};
        if (last) {
            if (!a.y.p && !a.y8.codes) return;
            float g[8];
            t.gamma(a.gamma, o, g);
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) s[j][i] = s[j][i] * rstd[i] * g[j];
        }
        if (view.p) t.store(view, o, s);
        if (packed.codes) {
            float f[8][V];
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) f[j][i] = s[j][i];
            t.pack(packed, o, f);
        }
    }
}

// K octets a thread stay in registers; K = 0: more than fit, read twice.  HBM, and for results in 8 bits the operations of packing, bound it: 48 x 527^2 fp32, 107 MB
// in 24 us = 4.5 TB/s (planes of whole cache lines 5.4), with its values in int8 besides 121 MB in 29 = 4.2.  Held to 128 registers the kernels spill and take 8 to 30 %
// longer.
template <int DT, int P, int V, int K, int T> __global__ __launch_bounds__(T) void rms_maps_kernel(RmsArgs a, long tiles, long tiles_of_image)
{
    __shared__ float part[T > 64 ? 2 * (T / 64) * P * V : 1];
    Spot<DT, P, V, K == 0> t(a);
    int half = 0;
    for (long tile = neighbour(); tile < tiles; tile += gridDim.x) {       // (every thread alike)
        t.go(tile, tiles_of_image);
        float s[K ? K : 1][8][V], q[V] = {};
        if (K) {
#pragma unroll
            for (int k = 0; k < K; ++k) sums_of(t, a, t.octet0 + k * t.octets, s[k]);
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) q[i] += s[k][j][i] * s[k][j][i];
        } else {
            for (int o = t.octet0; t.channels(o) > 0; o += t.octets) {
                sums_of(t, a, o, s[0]);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float v = 0.f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) v += s[0][j][i] * s[0][j][i];
                    q[i] += v;
                }
            }
        }
        t.total(q, part, half);
        float rstd[V];
#pragma unroll
        for (int i = 0; i < V; ++i) rstd[i] = inverse_root(q[i] / (float)a.c + a.eps);
        if (K) {
#pragma unroll
            for (int k = 0; k < K; ++k) put_maps(t, a, t.octet0 + k * t.octets, rstd, s[k]);
        } else {
            for (int o0 = 0; 8 * o0 < a.c; o0 += t.octets) {                // (every thread alike: lanes work together on blocks)
                const int o = o0 + t.octet0;
                sums_of(t, a, o, s[0]);
                put_maps(t, a, o, rstd, s[0]);
            }
        }
        if (a.rstd && t.octet0 == 0)
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < t.left) a.rstd[t.position(i)] = rstd[i];
    }
}

}  // namespace

hipError_t launch_rms_maps(const RmsArgs &a, hipStream_t stream)
{
    const bool far = far_maps(a, {&a.x, &a.residual, &a.sum, &a.y}, {&a.sum8, &a.y8});
    pick_maps(a, far, [&](auto p, auto v, auto k, auto t) {
        const long per = tiles_per_image(a, p() * v()), tiles = a.n * per;
        const int threads = threads_of(a, p());
        pick_dtype(a.dtype, [&](auto dt) { rms_maps_kernel<dt(), p(), v(), k(), t()><<<norm_blocks(tiles, 1), threads, 0, stream>>>(a, tiles, per); });
    });
    return hipGetLastError();
}

}  // namespace sk
