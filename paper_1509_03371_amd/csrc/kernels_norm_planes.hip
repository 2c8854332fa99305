// Layer norm of maps: planes of pixels, one after the other (MAPS) or in octets of channels (OCTETS).
#include "norm_tile.h"

namespace sk {

namespace {

// One octet a thread: every input is read once and every output written once, and the variance is taken from the values themselves about their mean.
// ADD: what is normalised is residual + dropout(x), or is wanted as an output (the rest is not compiled in: at the speed of the memory 16-bit maps leave 26
// instructions an element).  HBM bounds it: 48 x 527^2 fp32 109 MB in 22.8 us = 4.8 TB/s, 1024 x 128^2 fp32 with residual, dropout and sum 269 MB in 57 us = 4.7.
// Segments of a plane shorter than 128 bytes cost: two pixels a thread took 28 and 88 us instead of 27 and 67 (before results were stored past the L2);
// a wave for all channels, without a barrier, 28.5, and 64 pixel lanes 29.
template <int DT, int LAYOUT, int P, int T, bool ADD> __global__ __launch_bounds__(T, 4) void norm_planes_kernel(NormArgs a, long tiles, long row)
{
    constexpr int V = 4;
    extern __shared__ __align__(16) float part[];
    Tile<DT, LAYOUT, P, V> t(a.plane, row, tiles, a.c);
    const uint64_t counter = ADD ? a.drop.base() : 0;
    int half = 0;
    for (long tile = neighbour(); tile < tiles; tile += gridDim.x) {
        t.go(tile);
        float s[8][V], sum[1][V] = {}, var[1][V] = {}, mean[V], rstd[V];
        t.template values<ADD>(a, counter, t.oct0, s);
        t.add_channels(t.oct0, s, sum[0]);
        t.template total<1>(sum, part, half);
#pragma unroll
        for (int v = 0; v < V; ++v) mean[v] = sum[0][v] / (float)a.c;
        t.add_squares(t.oct0, s, mean, var[0]);
        t.template total<1>(var, part, half);
#pragma unroll
        for (int v = 0; v < V; ++v) rstd[v] = 1.f / sqrtf(var[0][v] / (float)a.c + a.eps);
        t.put_statistics(a, mean, rstd);
        t.template put<ADD>(a, t.oct0, s, mean, rstd);
    }
}

// More channels than a workgroup has threads for, planes of fewer than four pixels (V = 1), or strides between maps that 32 bits do not span (P = 64):
// octets in turn, read three times.
template <int DT, int LAYOUT, int P, int V> __global__ __launch_bounds__(1024) void norm_deep_planes_kernel(NormArgs a, long tiles, long row)
{
    extern __shared__ __align__(16) float part[];
    Tile<DT, LAYOUT, P, V> t(a.plane, row, tiles, a.c);
    const uint64_t counter = a.drop.base();
    const int last = (a.c + 7) / 8, octs = blockDim.x / P;
    int half = 0;
    for (long tile = neighbour(); tile < tiles; tile += gridDim.x) {
        t.go(tile);
        float s[8][V], sum[1][V] = {}, var[1][V] = {}, mean[V], rstd[V];
        for (int o0 = t.oct0; o0 < last; o0 += octs) {
            t.template values<true>(a, counter, o0, s);
            t.add_channels(o0, s, sum[0]);
        }
        t.template total<1>(sum, part, half);
#pragma unroll
        for (int v = 0; v < V; ++v) mean[v] = sum[0][v] / (float)a.c;
        for (int o0 = t.oct0; o0 < last; o0 += octs) {
            t.template values<true>(a, counter, o0, s);
            t.add_squares(o0, s, mean, var[0]);
        }
        t.template total<1>(var, part, half);
#pragma unroll
        for (int v = 0; v < V; ++v) rstd[v] = 1.f / sqrtf(var[0][v] / (float)a.c + a.eps);
        t.put_statistics(a, mean, rstd);
        for (int o0 = t.oct0; o0 < last; o0 += octs) {
            t.template values<true>(a, counter, o0, s);
            t.template put<true>(a, o0, s, mean, rstd);
        }
    }
}

}  // namespace

hipError_t launch_norm_planes(const NormArgs &a, hipStream_t stream)
{
    auto fits = [&](int p) { return spans(a, p, {&a.x, &a.residual, &a.sum, &a.y}); };
    const bool adds = a.residual.p || a.sum.p || a.drop.thresh;
    pick_type(a, [&](auto dt, auto layout) {
        bool done = false;
        if (layout() == OCTETS || a.plane >= 4)
            pick_planes<false>(a.c, [&](auto p, auto t, int threads) {
                if (!fits(p())) return;
                const long row = tiles_of_image(a, p() * 4), tiles = a.n * row;
                const size_t lds = part_bytes(1, p(), 4, threads);
                if (adds) norm_planes_kernel<dt(), layout(), p(), t(), true><<<norm_blocks(tiles, 1), threads, lds, stream>>>(a, tiles, row);
                else norm_planes_kernel<dt(), layout(), p(), t(), false><<<norm_blocks(tiles, 1), threads, lds, stream>>>(a, tiles, row);
                done = true;
            });
        if (done) return;
        pick_deep(a, !fits(4), [&](auto p, auto v) {
            const long row = tiles_of_image(a, p() * v()), tiles = a.n * row;
            const int threads = deep_threads(a.c, p());
            norm_deep_planes_kernel<dt(), layout(), p(), v()><<<norm_blocks(tiles, 1), threads, part_bytes(1, p(), v(), threads), stream>>>(a, tiles, row);
        });
    });
    return hipGetLastError();
}

}  // namespace sk
