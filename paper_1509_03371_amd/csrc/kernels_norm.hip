// Layer norm over the channels of a position and dropout, forwards and backwards (internal).
// Sums, statistics and parameters are fp32; a 16-bit tensor is rounded once, when it is stored.
#include "norm.h"

namespace sk {

namespace {

template <int DT> struct Elem;
template <> struct Elem<0> { typedef float type; };
template <> struct Elem<1> { typedef __bf16 type; };
template <> struct Elem<2> { typedef _Float16 type; };

template <int LAYOUT> __device__ __forceinline__ long at(const NormView &v, long b, int c, long m)
{
    if (LAYOUT == ROWS) return b * v.sn + c;
    if (LAYOUT == MAPS) return b * v.sn + (long)c * v.sc + m;
    return b * v.sn + (long)(c >> 3) * v.sc + 8 * m + (c & 7);
}

template <int DT, int LAYOUT> __device__ __forceinline__ float load(const NormView &v, long b, int c, long m)
{
    return (float)static_cast<const typename Elem<DT>::type *>(v.p)[at<LAYOUT>(v, b, c, m)];
}

template <int DT, int LAYOUT> __device__ __forceinline__ void store(const NormView &v, long b, int c, long m, float f)
{
    static_cast<typename Elem<DT>::type *>(v.p)[at<LAYOUT>(v, b, c, m)] = static_cast<typename Elem<DT>::type>(f);
}

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int i = 32; i >= 1; i >>= 1) v += __shfl_xor(v, i);
    return v;
}

__device__ __forceinline__ float drop_one(float v, const DropMask &d, uint64_t base, long q, int c)
{
    uint32_t w[4];
    mask_words(w, d, base, (uint64_t)q, (uint32_t)c >> 3);
    return dropped(v, w, c & 7, d);
}

// one thread an element (the octets' tail channels among them, which are zeros)
template <int DT, int LAYOUT> __global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a)
{
    const int cs = LAYOUT == OCTETS ? (a.c + 7) / 8 * 8 : a.c;
    const long total = a.n * a.plane * cs;
    const uint64_t base = a.drop.base();
    for (long i = blockIdx.x * 256L + threadIdx.x; i < total; i += gridDim.x * 256L) {
        long b, m;
        int c;
        if (LAYOUT == ROWS) { b = i / cs; c = (int)(i % cs); m = 0; }
        else { m = i % a.plane; const long t = i / a.plane; c = (int)(t % cs); b = t / cs; }
        float v = 0.f;
        if (c < a.c) {
            v = load<DT, LAYOUT>(a.x, b, c, m);
            if (a.drop.thresh) v = drop_one(v, a.drop, base, b * a.plane + m, c);
            if (a.relu_src.p && !(load<DT, LAYOUT>(a.relu_src, b, c, m) > 0.f)) v = 0.f;
        }
        store<DT, LAYOUT>(a.y, b, c, m, v);
    }
}

// one wave a position
template <int DT, int LAYOUT> __global__ __launch_bounds__(256) void layer_norm_kernel(NormArgs a)
{
    const int lane = threadIdx.x & 63;
    const long positions = a.n * a.plane;
    const uint64_t base = a.drop.base();
    for (long q = blockIdx.x * 4L + (threadIdx.x >> 6); q < positions; q += gridDim.x * 4L) {
        const long b = q / a.plane, m = q % a.plane;
        auto value = [&](int c) {
            float v = load<DT, LAYOUT>(a.x, b, c, m);
            if (a.drop.thresh) v = drop_one(v, a.drop, base, q, c);
            return a.residual.p ? load<DT, LAYOUT>(a.residual, b, c, m) + v : v;
        };
        float s = 0.f, ss = 0.f;
        for (int c = lane; c < a.c; c += 64) s += value(c);
        const float mean = wave_sum(s) / (float)a.c;
        for (int c = lane; c < a.c; c += 64) {
            const float d = value(c) - mean;
            ss += d * d;
        }
        const float rstd = 1.f / sqrtf(wave_sum(ss) / (float)a.c + a.eps);
        const int cs = LAYOUT == OCTETS ? (a.c + 7) / 8 * 8 : a.c;
        for (int c = lane; c < cs; c += 64) {
            float y = 0.f, v = 0.f;
            if (c < a.c) {
                v = value(c);
                y = (v - mean) * rstd;
                if (a.gamma) y *= a.gamma[c];
                if (a.beta) y += a.beta[c];
                if (a.relu && y < 0.f) y = 0.f;
            }
            if (a.sum.p) store<DT, LAYOUT>(a.sum, b, c, m, v);
            store<DT, LAYOUT>(a.y, b, c, m, y);
        }
        if (lane == 0) {
            if (a.mean) a.mean[q] = mean;
            if (a.rstd) a.rstd[q] = rstd;
        }
    }
}

// one wave a position: the gradient of what was normalised
template <int DT, int LAYOUT> __global__ __launch_bounds__(256) void layer_norm_bwd_kernel(NormBwdArgs a)
{
    const int lane = threadIdx.x & 63;
    const long positions = a.n * a.plane;
    const uint64_t base = a.drop.base();
    for (long q = blockIdx.x * 4L + (threadIdx.x >> 6); q < positions; q += gridDim.x * 4L) {
        const long b = q / a.plane, m = q % a.plane;
        const float mean = a.mean[q], rstd = a.rstd[q];
        float sg = 0.f, sgh = 0.f;
        for (int c = lane; c < a.c; c += 64) {
            float g = load<DT, LAYOUT>(a.dy, b, c, m);
            if (a.gamma) g *= a.gamma[c];
            sg += g;
            sgh += g * ((load<DT, LAYOUT>(a.s, b, c, m) - mean) * rstd);
        }
        const float mg = wave_sum(sg) / (float)a.c, mgh = wave_sum(sgh) / (float)a.c;
        const int cs = LAYOUT == OCTETS ? (a.c + 7) / 8 * 8 : a.c;
        for (int c = lane; c < cs; c += 64) {
            float t = 0.f, dx = 0.f;
            if (c < a.c) {
                const float s = load<DT, LAYOUT>(a.s, b, c, m);
                float g = load<DT, LAYOUT>(a.dy, b, c, m);
                if (a.gamma) g *= a.gamma[c];
                t = rstd * (g - mg - (s - mean) * rstd * mgh);
                if (a.dsum.p) t += load<DT, LAYOUT>(a.dsum, b, c, m);
                dx = a.drop.thresh ? drop_one(t, a.drop, base, q, c) : t;
                if (a.relu_x && !(s > 0.f)) dx = 0.f;
            }
            if (a.dresidual.p) store<DT, LAYOUT>(a.dresidual, b, c, m, t);
            if (a.dx.p) store<DT, LAYOUT>(a.dx, b, c, m, dx);
        }
    }
}

// one workgroup a channel
template <int DT, int LAYOUT> __global__ __launch_bounds__(256) void layer_norm_wgrad_kernel(NormBwdArgs a)
{
    __shared__ float part[2][4];
    const long positions = a.n * a.plane;
    for (int c = blockIdx.x; c < a.c; c += gridDim.x) {
        float dg = 0.f, db = 0.f;
        for (long q = threadIdx.x; q < positions; q += 256) {
            const long b = q / a.plane, m = q % a.plane;
            const float dy = load<DT, LAYOUT>(a.dy, b, c, m);
            db += dy;
            dg += dy * ((load<DT, LAYOUT>(a.s, b, c, m) - a.mean[q]) * a.rstd[q]);
        }
        dg = wave_sum(dg);
        db = wave_sum(db);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) {
            part[0][threadIdx.x >> 6] = dg;
            part[1][threadIdx.x >> 6] = db;
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            if (a.dgamma) a.dgamma[c] = (part[0][0] + part[0][1]) + (part[0][2] + part[0][3]);
            if (a.dbeta) a.dbeta[c] = (part[1][0] + part[1][1]) + (part[1][2] + part[1][3]);
        }
    }
}

__global__ void step_add_kernel(uint64_t *step) { *step += 1; }

unsigned blocks_for(long work, long each)
{
    const long b = (work + each - 1) / each;
    return (unsigned)(b < 65536 ? b : 65536);
}

// f(type, layout) with both as compile-time numbers
template <class F> hipError_t pick(const NormSpan &s, F f)
{
    auto by_layout = [&](auto dt) {
        if (s.layout == ROWS) return f(dt, std::integral_constant<int, ROWS>{});
        if (s.layout == MAPS) return f(dt, std::integral_constant<int, MAPS>{});
        return f(dt, std::integral_constant<int, OCTETS>{});
    };
    if (s.dtype == 0) return by_layout(std::integral_constant<int, 0>{});
    if (s.dtype == 1) return by_layout(std::integral_constant<int, 1>{});
    return by_layout(std::integral_constant<int, 2>{});
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs &a, hipStream_t stream)
{
    const long total = a.n * a.plane * (a.layout == OCTETS ? (a.c + 7) / 8 * 8 : a.c);
    if (total == 0) return hipSuccess;
    return pick(a, [&](auto dt, auto layout) {
        dropout_kernel<dt(), layout()><<<blocks_for(total, 256), 256, 0, stream>>>(a);
        return hipGetLastError();
    });
}

hipError_t launch_layer_norm(const NormArgs &a, hipStream_t stream)
{
    if (a.n * a.plane == 0) return hipSuccess;
    return pick(a, [&](auto dt, auto layout) {
        layer_norm_kernel<dt(), layout()><<<blocks_for(a.n * a.plane, 4), 256, 0, stream>>>(a);
        return hipGetLastError();
    });
}

size_t norm_bwd_scratch_floats(const NormSpan &) { return 0; }
size_t norm_bwd_min_scratch_floats(const NormSpan &) { return 0; }

hipError_t launch_layer_norm_bwd(const NormBwdArgs &a, hipStream_t stream)
{
    return pick(a, [&](auto dt, auto layout) {
        if (a.dgamma || a.dbeta) layer_norm_wgrad_kernel<dt(), layout()><<<(unsigned)(a.c < 65536 ? a.c : 65536), 256, 0, stream>>>(a);
        if (a.n * a.plane > 0 && (a.dx.p || a.dresidual.p))
            layer_norm_bwd_kernel<dt(), layout()><<<blocks_for(a.n * a.plane, 4), 256, 0, stream>>>(a);
        return hipGetLastError();
    });
}

hipError_t launch_step_add(uint64_t *step, hipStream_t stream)
{
    step_add_kernel<<<1, 1, 0, stream>>>(step);
    return hipGetLastError();
}

}  // namespace sk
