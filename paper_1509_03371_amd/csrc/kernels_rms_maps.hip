// Root-mean-square norm over the channels of a position, forwards and backwards.
#include "rms.h"

namespace sk {

namespace {

// A workgroup takes a row, or 32 pixels of an image (a block of every map), and reads the values once for each thing that it makes of them.
constexpr int T = 256;

struct Place {
    long b, first;
    int pixels;                  // positions of the workgroup
    __device__ __forceinline__ Place(const NormSpan &s, long i)
    {
        const long nb = s.layout == ROWS ? 1 : blocks_of(s.plane);
        b = i / nb;
        first = 32 * (i - b * nb);
        pixels = s.layout == ROWS ? 1 : (int)(s.plane - first < 32 ? s.plane - first : 32);
    }
};
long all_places(const NormSpan &s) { return s.layout == ROWS ? s.n : s.n * blocks_of(s.plane); }

template <int DT> __device__ __forceinline__ float read(const NormView &v, const NormSpan &s, long b, long k, long m)
{
    const long at = b * v.sn + (s.layout == ROWS ? k : k * v.sc + m);
    return (float)static_cast<const elem_t<DT> *>(v.p)[at];
}
template <int DT> __device__ __forceinline__ void write(const NormView &v, const NormSpan &s, long b, long k, long m, float f)
{
    const long at = b * v.sn + (s.layout == ROWS ? k : k * v.sc + m);
    static_cast<elem_t<DT> *>(v.p)[at] = static_cast<elem_t<DT>>(f);
}
__device__ __forceinline__ float held(const PackedView &p, const NormSpan &s, long b, long k, long m)
{
    const bool rows = s.layout == ROWS;
    const uint32_t code = p.codes[b * p.sn + (rows ? k : k * p.sc + m)];
    const float scale = Code8<0>::scale(p.scales[b * p.ssn + (rows ? k / 32 : k * p.ssc + m / 32)]);
    return p.code == E4M3 ? Code8<E4M3>::value(code, scale) : Code8<I8>::value(code, scale);
}

// sums over threads with equal number modulo 32 (MAPS) or all (ROWS)
__device__ __forceinline__ float total(const NormSpan &s, float v, float *part)
{
    __syncthreads();
    part[threadIdx.x] = v;
    __syncthreads();
    float t = 0.f;
    for (int i = s.layout == ROWS ? 0 : threadIdx.x % 32; i < T; i += s.layout == ROWS ? 1 : 32) t += part[i];
    return t;
}

template <int DT, class F> __device__ void pack_block(const PackedView &p, const NormSpan &s, long b, long k, long m, int count, F value)
{
    const bool rows = s.layout == ROWS;
    uint8_t *codes = p.codes + b * p.sn + (rows ? k : k * p.sc + m), *scale = p.scales + b * p.ssn + (rows ? k / 32 : k * p.ssc + m / 32);
    auto go = [&](auto code) {
        constexpr uint32_t limit = Code8<code()>::limit(DT);
        uint32_t most = 0;
        for (int j = 0; j < count; ++j) most = max(most, counted(value(j), limit));
        const uint32_t byte = Code8<code()>::scale_byte(most);
        *scale = (uint8_t)byte;
        for (int j = 0; j < count; ++j) codes[j] = (uint8_t)any_code<code()>(value(j), Code8<code()>::inverse(byte), limit);
    };
    if (p.code == E4M3) go(std::integral_constant<int, E4M3>{});
    else go(std::integral_constant<int, I8>{});
}

template <int DT> __global__ __launch_bounds__(T) void rms_kernel(RmsArgs a, long places)
{
    __shared__ float part[T], rs[32];
    const bool rows = a.layout == ROWS;
    for (long i = blockIdx.x; i < places; i += gridDim.x) {
        const Place at(a, i);
        auto sum = [&](long k, long m) {
            const float x = read<DT>(a.x, a, at.b, k, m);
            return a.residual.p ? x + read<DT>(a.residual, a, at.b, k, m) : x;
        };
        const int px = rows ? 0 : threadIdx.x % 32, k0 = rows ? threadIdx.x : threadIdx.x / 32, step = rows ? T : T / 32;
        float q = 0.f;
        if (px < at.pixels)
            for (long k = k0; k < a.c; k += step) {
                const float v = sum(k, at.first + px);
                q += v * v;
            }
        const float rstd = 1.f / sqrtf(total(a, q, part) / (float)a.c + a.eps);
        if (threadIdx.x < 32) rs[threadIdx.x] = rstd;
        if ((rows ? threadIdx.x == 0 : threadIdx.x < at.pixels) && a.rstd) a.rstd[at.b * a.plane + at.first + px] = rstd;
        __syncthreads();
        // blocks in 8 bits first: y and sum may go to the operands' place
        const long lines = rows ? blocks_of(a.c) : a.c;
        for (long l = threadIdx.x; l < lines; l += T) {
            const long k = rows ? 32 * l : l;
            const int count = rows ? (int)std::min<long>(32, a.c - k) : at.pixels;
            if (a.sum8.codes) pack_block<DT>(a.sum8, a, at.b, k, at.first, count, [&](int j) { return rows ? sum(k + j, 0) : sum(k, at.first + j); });
            if (a.y8.codes)
                pack_block<DT>(a.y8, a, at.b, k, at.first, count, [&](int j) {
                    const float g = a.gamma ? a.gamma[rows ? k + j : k] : 1.f;
                    return (rows ? sum(k + j, 0) : sum(k, at.first + j)) * rs[rows ? 0 : j] * g;
                });
        }
        __syncthreads();
        if (px < at.pixels)
            for (long k = k0; k < a.c; k += step) {
                const float v = sum(k, at.first + px);
                if (a.sum.p) write<DT>(a.sum, a, at.b, k, at.first + px, v);
                if (a.y.p) write<DT>(a.y, a, at.b, k, at.first + px, v * rstd * (a.gamma ? a.gamma[k] : 1.f));
            }
        __syncthreads();
    }
}

template <int DT> __global__ __launch_bounds__(T) void rms_bwd_kernel(RmsBwdArgs a, long places)
{
    __shared__ float part[T];
    const bool rows = a.layout == ROWS;
    for (long i = blockIdx.x; i < places; i += gridDim.x) {
        const Place at(a, i);
        const int px = rows ? 0 : threadIdx.x % 32, k0 = rows ? threadIdx.x : threadIdx.x / 32, step = rows ? T : T / 32;
        const bool mine = px < at.pixels;
        const long m = at.first + px;
        const float rstd = mine ? a.rstd[at.b * a.plane + m] : 0.f;
        auto value = [&](long k) { return a.s8.codes ? held(a.s8, a, at.b, k, m) : read<DT>(a.s, a, at.b, k, m); };
        float q = 0.f;
        if (mine)
            for (long k = k0; k < a.c; k += step) q += read<DT>(a.dy, a, at.b, k, m) * (a.gamma ? a.gamma[k] : 1.f) * (value(k) * rstd);
        const float mean = total(a, q, part) / (float)a.c;
        if (mine)
            for (long k = k0; k < a.c; k += step) {
                float t = rstd * (read<DT>(a.dy, a, at.b, k, m) * (a.gamma ? a.gamma[k] : 1.f) - value(k) * rstd * mean);
                if (a.dsum.p) t += read<DT>(a.dsum, a, at.b, k, m);
                write<DT>(a.dx, a, at.b, k, m, t);
            }
    }
}

template <int DT> __global__ __launch_bounds__(T) void rms_dgamma_kernel(RmsBwdArgs a)
{
    __shared__ float part[T];
    for (long k = blockIdx.x; k < a.c; k += gridDim.x) {
        float q = 0.f;
        for (long i = threadIdx.x; i < a.n * a.plane; i += T) {
            const long b = i / a.plane, m = i - b * a.plane;
            const float s = a.s8.codes ? held(a.s8, a, b, k, m) : read<DT>(a.s, a, b, k, m);
            q += read<DT>(a.dy, a, b, k, m) * (s * a.rstd[i]);
        }
        __syncthreads();
        part[threadIdx.x] = q;
        __syncthreads();
        if (threadIdx.x == 0) {
            float t = 0.f;
            for (int i = 0; i < T; ++i) t += part[i];
            a.dgamma[k] = t;
        }
    }
}

}  // namespace

hipError_t launch_rms_maps(const RmsArgs &a, hipStream_t stream)
{
    const long places = all_places(a);
    pick_dtype(a.dtype, [&](auto dt) { rms_kernel<dt()><<<norm_blocks(places, 1), T, 0, stream>>>(a, places); });
    return hipGetLastError();
}

int rms_maps_bwd_copies(const NormSpan &) { return 1; }

hipError_t launch_rms_maps_bwd(const RmsBwdArgs &a, int, hipStream_t stream)
{
    const long places = all_places(a);
    Launches done;
    pick_dtype(a.dtype, [&](auto dt) {
        // the sums first: dx may go to the place of dy or s
        if (a.dgamma) rms_dgamma_kernel<dt()><<<norm_blocks(a.c, 1), T, 0, stream>>>(a);
        if (done.failed() || !a.dx.p || !places) return;
        rms_bwd_kernel<dt()><<<norm_blocks(places, 1), T, 0, stream>>>(a, places);
    });
    return done.status();
}

}  // namespace sk
