// Root-mean-square norm: what its kernels share (internal device code).
#pragma once
#include "act8_block.h"

namespace sk {

template <int N> using num = std::integral_constant<int, N>;

template <class F> void pick_dtype(int dtype, F f)
{
    if (dtype == 0) return f(num<0>{});
    if (dtype == 1) return f(num<1>{});
    return f(num<2>{});
}

// eight values of a block of LANES lanes, in the form that the view asks for; the same code in all lanes
template <int DT, int LANES> __device__ __forceinline__ void put_packed(const PackedView &v, const float (&f)[8], int left, uint8_t *codes, uint8_t *scale)
{
    if (v.code == E4M3) put_octet<DT, E4M3, LANES>(f, left, codes, scale);
    else put_octet<DT, I8, LANES>(f, left, codes, scale);
}
__device__ __forceinline__ void held_octet(const PackedView &v, const uint32_t (&c)[2], uint32_t byte, float (&f)[8])
{
    if (v.code == E4M3) octet_of_codes<E4M3>(c, byte, f);
    else octet_of_codes<I8>(c, byte, f);
}

// 1 / sqrt(v), rounded once: the root and the division, rounded each, are up to three half steps off (more than one for a quarter of all v), and what they are off goes into every
// value of the position.  r = (1 / sqrt v)(1 + d) has 1 - v r^2 = -2 d but for d^2, taken from the whole product v r = h + l.  Infinite v: 0.
__device__ __forceinline__ float inverse_root(float v)
{
    const float r = 1.f / sqrtf(v), h = v * r, l = fmaf(v, r, -h);
    const float e = fmaf(-h, r, 1.f) - l * r;
    return r > 0.f ? fmaf(0.5f * r, e, r) : r;
}

// dgamma from the `copies` copies of its sums, each of c rounded up to 4
__host__ __device__ inline long rms_copy_floats(long c) { return (c + 3) / 4 * 4; }
hipError_t launch_rms_reduce(const float *scratch, int copies, float *dgamma, int c, hipStream_t stream);

hipError_t launch_rms_rows(const RmsArgs &a, hipStream_t stream);
hipError_t launch_rms_maps(const RmsArgs &a, hipStream_t stream);
// the most copies that a gradient of these sizes writes, whatever its strides
int rms_rows_bwd_copies(const NormSpan &s);
int rms_maps_bwd_copies(const NormSpan &s);
hipError_t launch_rms_rows_bwd(const RmsBwdArgs &a, hipStream_t stream);
hipError_t launch_rms_maps_bwd(const RmsBwdArgs &a, hipStream_t stream);

}  // namespace sk
