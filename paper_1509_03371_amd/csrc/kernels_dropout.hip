// Dropout of rows, maps and octets, and the counter of a net's training passes.
#include "norm_device.h"

namespace sk {

namespace {

// A thread takes the eight channels of an octet that one call of the generator serves; bx (a power of two) octets of a row lie side by side
// in a workgroup.
template <int DT> __global__ __launch_bounds__(256) void dropout_rows_kernel(DropoutArgs a, int shift, int parts)
{
    typedef elem_t<DT> E;
    const uint64_t base = a.drop.base();
    const int across = 1 << shift, down = 256 >> shift;
    const int o = (blockIdx.x % parts) * across + (threadIdx.x & (across - 1));
    if (8 * o >= a.c) return;
    const long step = gridDim.x / parts * (long)down;
    for (long row = blockIdx.x / parts * (long)down + (threadIdx.x >> shift); row < a.n; row += step) {
        const line_t<DT, 8> x = load_line<DT, 8>(static_cast<const E *>(a.x.p) + row * a.x.sn, 8 * o, a.c);
        uint32_t w[4];
        mask_words(w, a.drop, base, (uint64_t)row, o);
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = dropped((float)x[j], w, j, a.drop);
        store_line<DT, 8>(static_cast<E *>(a.y.p) + row * a.y.sn, 8 * o, a.c, y);
    }
}

// Maps: a thread takes an octet of channels of four pixels side by side.
template <int DT> __global__ __launch_bounds__(256) void dropout_maps_kernel(DropoutArgs a, long tiles, int octs, long parts)
{
    typedef elem_t<DT> E;
    constexpr int V = 4;
    const uint64_t base = a.drop.base();
    for (long t = blockIdx.x; t < tiles; t += gridDim.x) {          // tile: (image, octet, part of the plane), the last fastest
        const long line = t / parts, b = line / octs, pixel = (t % parts * 256L + threadIdx.x) * V;
        const int o = (int)(line % octs);
        if (pixel >= a.plane) continue;
        const E *x = static_cast<const E *>(a.x.p) + b * a.x.sn + 8L * o * a.x.sc;
        E *y = static_cast<E *>(a.y.p) + b * a.y.sn + 8L * o * a.y.sc;
        line_t<DT, V> v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 8 * o + j < a.c ? load_line<DT, V>(x + j * a.x.sc, pixel, a.plane) : line_t<DT, V>{};
        float f[8][V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            uint32_t w[4];
            mask_words(w, a.drop, base, (uint64_t)(b * a.plane + pixel + i), o);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j][i] = dropped((float)v[j][i], w, j, a.drop);
        }
        const E *r = static_cast<const E *>(a.relu_src.p) + b * a.relu_src.sn + 8L * o * a.relu_src.sc;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (8 * o + j >= a.c) break;
            if (a.relu_src.p) {
                const line_t<DT, V> u = load_line<DT, V>(r + j * a.relu_src.sc, pixel, a.plane);
#pragma unroll
                for (int i = 0; i < V; ++i) f[j][i] = (float)u[i] > 0.f ? f[j][i] : 0.f;
            }
            store_line<DT, V>(y + j * a.y.sc, pixel, a.plane, f[j]);
        }
    }
}

// Octets: a thread takes the octet of a pixel; channels behind the last are written as zeros.
template <int DT> __global__ __launch_bounds__(256) void dropout_octets_kernel(DropoutArgs a, long tiles, int octs, long parts)
{
    typedef elem_t<DT> E;
    const uint64_t base = a.drop.base();
    for (long t = blockIdx.x; t < tiles; t += gridDim.x) {
        const long line = t / parts, b = line / octs, pixel = t % parts * 256L + threadIdx.x;
        const int o = (int)(line % octs);
        if (pixel >= a.plane) continue;
        const line_t<DT, 8> x = *reinterpret_cast<const line_t<DT, 8> *>(static_cast<const E *>(a.x.p) + b * a.x.sn + o * a.x.sc + 8 * pixel);
        line_t<DT, 8> r{};
        if (a.relu_src.p) r = *reinterpret_cast<const line_t<DT, 8> *>(static_cast<const E *>(a.relu_src.p) + b * a.relu_src.sn + o * a.relu_src.sc + 8 * pixel);
        uint32_t w[4];
        mask_words(w, a.drop, base, (uint64_t)(b * a.plane + pixel), o);
        line_t<DT, 8> y;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float v = dropped((float)x[j], w, j, a.drop);
            if (8 * o + j >= a.c || (a.relu_src.p && !((float)r[j] > 0.f))) v = 0.f;
            y[j] = static_cast<E>(v);
        }
        *reinterpret_cast<line_t<DT, 8> *>(static_cast<E *>(a.y.p) + b * a.y.sn + o * a.y.sc + 8 * pixel) = y;
    }
}

__global__ void step_add_kernel(uint64_t *step) { *step += 1; }

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
        const int pixels = a.layout == MAPS ? 1024 : 256;
        const long parts = (a.plane + pixels - 1) / pixels, tiles = a.n * octs * parts;
        if (a.layout == MAPS) dropout_maps_kernel<DT><<<norm_blocks(tiles, 1), 256, 0, stream>>>(a, tiles, octs, parts);
        else if (DT != 0) dropout_octets_kernel<DT><<<norm_blocks(tiles, 1), 256, 0, stream>>>(a, tiles, octs, parts);
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
