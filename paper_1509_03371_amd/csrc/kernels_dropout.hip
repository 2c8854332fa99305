// Dropout of rows, maps and octets, and the counter of a net's training passes.
#include "norm_device.h"

namespace sk {

namespace {

// One call of the generator, some sixty instructions of which twenty are products at a quarter of the rate, serves the eight channels of an octet: about half of the time
// that 16-bit elements take to come and go.  HBM bounds it: 200 maps of 512^2 fp32 419 MB in 72 us = 5.8 TB/s, 64 x 388^2 bf16 of four images 154 MB in 30 us = 5.1.
// (One call and one element a thread took 216 us for the first.)

// A thread takes the eight channels of an octet that one call of the generator serves; 1 << shift octets of a row lie side by side in a workgroup.
template <int DT> __global__ __launch_bounds__(256) void dropout_rows_kernel(DropoutArgs a, int shift, int parts)
{
    typedef elem_t<DT> E;
    const uint64_t counter = a.drop.base();
    const int down = 256 >> shift, c0 = 8 * (((blockIdx.x % parts) << shift) + (threadIdx.x & ((1 << shift) - 1))), left = a.c - c0;
    if (left <= 0) return;
    const long step = gridDim.x / parts * (long)down;
    for (long row = blockIdx.x / parts * (long)down + (threadIdx.x >> shift); row < a.n; row += step) {
        const E *x = static_cast<const E *>(a.x.p) + row * a.x.sn + c0;
        E *y = static_cast<E *>(a.y.p) + row * a.y.sn + c0;
        uint32_t w[4];
        if (left >= 8) {
            Words<DT, 8> v;
            v.load(reinterpret_cast<src_t>(x), 0);
            mask_words(w, a.drop, counter, (uint64_t)row, c0 / 8);
            float f[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = dropped(v[j], w, j, a.drop);
            store_at<DT, 8>(reinterpret_cast<dst_t>(y), 0, f);
        } else {
            mask_words(w, a.drop, counter, (uint64_t)row, c0 / 8);
#pragma unroll
            for (int j = 0; j < 7; ++j)
                if (j < left) y[j] = static_cast<E>(dropped((float)x[j], w, j, a.drop));
        }
    }
}

// Maps: a thread takes an octet of channels of V pixels side by side, a wave a stretch of 64 V.
template <int DT, int V> __global__ __launch_bounds__(256) void dropout_maps_kernel(DropoutArgs a, long tiles, int octs, long parts)
{
    typedef elem_t<DT> E;
    const uint64_t counter = a.drop.base();
    const uint32_t mine = V * (threadIdx.x & 63);
    for (long t = blockIdx.x; t < tiles; t += gridDim.x) {          // tile: (image, octet, part of the plane), the last fastest
        const long line = t / parts, b = line / octs, first = (t % parts * 4 + uniform(threadIdx.x >> 6)) * (64L * V);
        const int o = (int)(line % octs), left = a.c - 8 * o;
        if (first >= a.plane) continue;
        const Stretch<V> run(first, 64 * V, a.plane, mine);
        if (run.empty(mine)) continue;
        const long from = run.start;
        const uint32_t px = run.at, off = px * sizeof(E);
        src_t x = reinterpret_cast<src_t>(static_cast<const E *>(a.x.p) + b * a.x.sn + 8L * o * a.x.sc + from);
        dst_t y = reinterpret_cast<dst_t>(static_cast<E *>(a.y.p) + b * a.y.sn + 8L * o * a.y.sc + from);
        const long up_x = a.x.sc * sizeof(E), up_y = a.y.sc * sizeof(E), up_r = a.relu_src.sc * sizeof(E);
        Words<DT, V> v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j].load(x + std::min(j, left - 1) * up_x, off);        // (channels behind the last repeat it)
        uint32_t w[V][4];
#pragma unroll
        for (int i = 0; i < V; ++i) mask_words(w[i], a.drop, counter, (uint64_t)(b * a.plane + from + px + i), o);
        src_t r = reinterpret_cast<src_t>(static_cast<const E *>(a.relu_src.p) + b * a.relu_src.sn + 8L * o * a.relu_src.sc + from);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < left) {
                float f[V];
#pragma unroll
                for (int i = 0; i < V; ++i) f[i] = dropped(v[j][i], w[i], j, a.drop);
                if (a.relu_src.p) {
                    Words<DT, V> u;
                    u.load(r + j * up_r, off);
#pragma unroll
                    for (int i = 0; i < V; ++i) f[i] = u[i] > 0.f ? f[i] : 0.f;
                }
                store_at<DT, V>(y + j * up_y, off, f);
            }
    }
}

// Octets: a thread takes the octet of a pixel; channels behind the last are written as zeros.
template <int DT> __global__ __launch_bounds__(256) void dropout_octets_kernel(DropoutArgs a, long tiles, int octs, long parts)
{
    typedef elem_t<DT> E;
    const uint64_t counter = a.drop.base();
    for (long t = blockIdx.x; t < tiles; t += gridDim.x) {
        const long line = t / parts, b = line / octs, first = t % parts * 256L;
        const int o = (int)(line % octs), left = a.c - 8 * o;
        if (first + threadIdx.x >= a.plane) continue;
        const uint32_t off = threadIdx.x * 8 * sizeof(E);
        Words<DT, 8> x;
        x.load(reinterpret_cast<src_t>(static_cast<const E *>(a.x.p) + b * a.x.sn + o * a.x.sc + 8 * first), off);
        uint32_t w[4];
        mask_words(w, a.drop, counter, (uint64_t)(b * a.plane + first + threadIdx.x), o);
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = dropped(x[j], w, j, a.drop);
        if (left < 8)
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = j < left ? y[j] : 0.f;
        if (a.relu_src.p) {
            x.load(reinterpret_cast<src_t>(static_cast<const E *>(a.relu_src.p) + b * a.relu_src.sn + o * a.relu_src.sc + 8 * first), off);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = x[j] > 0.f ? y[j] : 0.f;
        }
        store_at<DT, 8>(reinterpret_cast<dst_t>(static_cast<E *>(a.y.p) + b * a.y.sn + o * a.y.sc + 8 * first), off, y);
    }
}

__global__ void step_add_kernel(uint64_t *step) { step[1] = step[0] += 1; }

template <int DT> hipError_t launch(const DropoutArgs &a, hipStream_t stream)
{
    const int octs = (a.c + 7) / 8;
    if (a.layout == ROWS) {
        int shift = 0;                                  // the narrowest power of two of octets that wastes no more of a row than a wider one
        while (shift < 8 && (1 << shift) < octs) ++shift;
        const auto idle = [&](int s) { return (octs + (1 << s) - 1) / (1 << s) * (1 << s) - octs; };
        while (shift > 5 && idle(shift - 1) < idle(shift)) --shift;
        const int parts = (octs + (1 << shift) - 1) >> shift;
        const long rows = (a.n + (256 >> shift) - 1) / (256 >> shift);
        const long most = std::max(1L, (1L << 21) / parts);
        dropout_rows_kernel<DT><<<(unsigned)(std::min(rows, most) * parts), 256, 0, stream>>>(a, shift, parts);
    } else {
        const int v = a.layout == MAPS && a.plane >= 4 ? 4 : 1;
        const long parts = (a.plane + 256 * v - 1) / (256 * v), tiles = a.n * octs * parts;
        if (a.layout == MAPS && v == 4) dropout_maps_kernel<DT, 4><<<norm_blocks(tiles, 1), 256, 0, stream>>>(a, tiles, octs, parts);
        else if (a.layout == MAPS) dropout_maps_kernel<DT, 1><<<norm_blocks(tiles, 1), 256, 0, stream>>>(a, tiles, octs, parts);
        else if constexpr (DT != 0) dropout_octets_kernel<DT><<<norm_blocks(tiles, 1), 256, 0, stream>>>(a, tiles, octs, parts);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs &a, hipStream_t stream)
{
    if (a.n * a.plane == 0) return hipSuccess;
    return a.dtype == 0 ? launch<0>(a, stream) : a.dtype == 1 ? launch<1>(a, stream) : launch<2>(a, stream);
}

hipError_t launch_step_add(uint64_t *step, hipStream_t stream)
{
    step_add_kernel<<<1, 1, 0, stream>>>(step);
    return hipGetLastError();
}

}  // namespace sk
