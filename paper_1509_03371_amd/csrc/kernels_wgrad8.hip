// Weight gradient of an inner product over inputs held in 8 bits.
#include "act8_device.h"

namespace sk {

namespace {

// a thread an element of the gradient
template <int DT, int CODE> __global__ __launch_bounds__(256) void wgrad8_kernel(Wgrad8Args a)
{
    const bool rows = a.layout == ROWS;
    const long all = a.c_out * (a.c + (a.db ? 1L : 0L));
    for (long i = blockIdx.x * 256L + threadIdx.x; i < all; i += gridDim.x * 256L) {
        const bool bias = i >= a.c_out * a.c;
        const long o = bias ? i - a.c_out * a.c : i / a.c, k = bias ? 0 : i - o * a.c;
        const long positions = a.n * a.plane;
        float sum = 0.f;
        for (long q0 = 0; q0 < positions; q0 += 32) {
            float part = 0.f;
            for (long q = q0; q < q0 + 32 && q < positions; ++q) {
                const long b = q / a.plane, m = q - b * a.plane;
                const float dy = (float)static_cast<const elem_t<DT> *>(a.dy.p)[b * a.dy.sn + (rows ? o : o * a.dy.sc + m)];
                if (bias) {
                    part += dy;
                } else {
                    const float scale = Code8<CODE>::scale(a.x.scales[b * a.x.ssn + (rows ? k / 32 : k * a.x.ssc + m / 32)]);
                    part = fmaf(dy, Code8<CODE>::value(a.x.codes[b * a.x.sn + (rows ? k : k * a.x.sc + m)], scale), part);
                }
            }
            sum += part;
        }
        float *out = bias ? a.db + o : a.dw + i;
        *out = a.accumulate ? *out + sum : sum;
    }
}

}  // namespace

size_t wgrad8_scratch_floats(const NormSpan &, long) { return 0; }

hipError_t launch_wgrad8(const Wgrad8Args &a, hipStream_t stream)
{
    const unsigned blocks = norm_blocks(a.c_out * (a.c + 1), 256);
    pick_code(a.x.code, [&](auto code) {
        if (a.dtype == 0) wgrad8_kernel<0, code()><<<blocks, 256, 0, stream>>>(a);
        else if (a.dtype == 1) wgrad8_kernel<1, code()><<<blocks, 256, 0, stream>>>(a);
        else wgrad8_kernel<2, code()><<<blocks, 256, 0, stream>>>(a);
    });
    return hipGetLastError();
}

}  // namespace sk
