// Tensors into 8 bits and back.
#include "act8_device.h"

namespace sk {

namespace {

// A line and the block of it that a thread takes.
struct Block8 {
    long b, k, first;            // image or row, map, first element
    int count;
    __device__ __forceinline__ Block8(const NormSpan &s, long i)
    {
        const long length = s.layout == ROWS ? s.c : s.plane, nb = blocks_of(length), line = i / nb;
        first = 32 * (i - line * nb);
        count = (int)(length - first < 32 ? length - first : 32);
        b = s.layout == ROWS ? line : line / s.c;
        k = s.layout == ROWS ? 0 : line - b * s.c;
    }
};
long all_blocks(const NormSpan &s) { return s.layout == ROWS ? s.n * blocks_of(s.c) : s.n * s.c * blocks_of(s.plane); }

template <int DT, int CODE> __global__ __launch_bounds__(256) void pack8_kernel(Pack8Args a, long blocks)
{
    typedef elem_t<DT> E;
    constexpr uint32_t limit = Code8<CODE>::limit(DT);
    for (long i = blockIdx.x * 256L + threadIdx.x; i < blocks; i += gridDim.x * 256L) {
        const Block8 l(a, i);
        const E *x = static_cast<const E *>(a.x.p) + l.b * a.x.sn + l.k * a.x.sc + l.first;
        uint32_t most = 0;
        for (int j = 0; j < l.count; ++j) most = max(most, counted((float)x[j], limit));
        const uint32_t byte = Code8<CODE>::scale_byte(most);
        a.packed.scales[l.b * a.packed.ssn + l.k * a.packed.ssc + l.first / 32] = (uint8_t)byte;
        uint8_t *to = a.packed.codes + l.b * a.packed.sn + l.k * a.packed.sc + l.first;
        for (int j = 0; j < l.count; ++j) to[j] = (uint8_t)any_code<CODE>((float)x[j], Code8<CODE>::inverse(byte), limit);
    }
}

template <int DT, int CODE> __global__ __launch_bounds__(256) void unpack8_kernel(Pack8Args a, long blocks)
{
    typedef elem_t<DT> E;
    for (long i = blockIdx.x * 256L + threadIdx.x; i < blocks; i += gridDim.x * 256L) {
        const Block8 l(a, i);
        const float scale = Code8<CODE>::scale(a.packed.scales[l.b * a.packed.ssn + l.k * a.packed.ssc + l.first / 32]);
        const uint8_t *from = a.packed.codes + l.b * a.packed.sn + l.k * a.packed.sc + l.first;
        E *y = static_cast<E *>(a.x.p) + l.b * a.x.sn + l.k * a.x.sc + l.first;
        for (int j = 0; j < l.count; ++j) y[j] = static_cast<E>(Code8<CODE>::value(from[j], scale));
    }
}

template <class F> void pick_dtype(int dtype, F f)
{
    if (dtype == 0) return f(std::integral_constant<int, 0>{});
    if (dtype == 1) return f(std::integral_constant<int, 1>{});
    return f(std::integral_constant<int, 2>{});
}

}  // namespace

hipError_t launch_pack8(const Pack8Args &a, hipStream_t stream)
{
    const long blocks = all_blocks(a);
    pick_dtype(a.dtype, [&](auto dt) { pick_code(a.packed.code, [&](auto code) { pack8_kernel<dt(), code()><<<norm_blocks(blocks, 256), 256, 0, stream>>>(a, blocks); }); });
    return hipGetLastError();
}

hipError_t launch_unpack8(const Pack8Args &a, hipStream_t stream)
{
    const long blocks = all_blocks(a);
    pick_dtype(a.dtype, [&](auto dt) { pick_code(a.packed.code, [&](auto code) { unpack8_kernel<dt(), code()><<<norm_blocks(blocks, 256), 256, 0, stream>>>(a, blocks); }); });
    return hipGetLastError();
}

}  // namespace sk
