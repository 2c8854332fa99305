// Root-mean-square norm of maps, backwards.
#include "rms_maps.h"

namespace sk {

namespace {

// An octet of what was normalised, kept as it was read.
template <int DT, int P, int V, bool FAR, bool HELD> struct NormedMaps;
template <int DT, int P, int V, bool FAR> struct NormedMaps<DT, P, V, FAR, false> {
    Words<DT, V> w[8];
    __device__ __forceinline__ void load(const Spot<DT, P, V, FAR> &t, const RmsBwdArgs &a, int o) { t.load(a.s, o, w); }
    __device__ __forceinline__ void values(const RmsBwdArgs &, int j, float (&f)[V]) const
    {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = w[j][i];
    }
    __device__ __forceinline__ void forget()
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j].forget();
    }
};
template <int DT, int P, int V, bool FAR> struct NormedMaps<DT, P, V, FAR, true> {
    uint32_t c[8], bytes[2];                            // four scales a word
    __device__ __forceinline__ void load(const Spot<DT, P, V, FAR> &t, const RmsBwdArgs &a, int o)
    {
        typedef typename Spot<DT, P, V, FAR>::Off Off;
        const PackedView &v = a.s8;
        const int n = t.left > 0 ? t.channels(o) : 0;
        const uint8_t *scale = v.scales + t.b * v.ssn + t.first / 32 + (Off)(8 * o) * (Off)v.ssc + V * t.lane / 32;
        const uint8_t *early = v.codes - V;            // (as Spot::load)
        const Off off = t.offset(v.sc, 1, o) + (V - t.back);
        uint32_t byte[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            c[j] = 0;
            byte[j] = 127;
        }
        if (n >= 8) {
#pragma unroll
            for (int j = 0; j < 8; ++j) c[j] = load_codes_of<V>(early + t.base(v.sn, v.sc, 1, j) + off);
#pragma unroll
            for (int j = 0; j < 8; ++j) byte[j] = scale[j * v.ssc];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < n) {
                    c[j] = load_codes_of<V>(early + t.base(v.sn, v.sc, 1, j) + off);
                    byte[j] = scale[j * v.ssc];
                }
        }
        if (t.back)
#pragma unroll
            for (int j = 0; j < 8; ++j) c[j] >>= 8 * t.back;
#pragma unroll
        for (int j = 0; j < 2; ++j) bytes[j] = byte[4 * j] | byte[4 * j + 1] << 8 | byte[4 * j + 2] << 16 | byte[4 * j + 3] << 24;
    }
    __device__ __forceinline__ void values(const RmsBwdArgs &a, int j, float (&f)[V]) const
    {
        const float scale = Code8<E4M3>::scale((bytes[j / 4] >> 8 * (j & 3)) & 0xff);
        float four[4];
        if (a.s8.code == E4M3) Code8<E4M3>::values(c[j], scale, four);
        else Code8<I8>::values(c[j], scale, four);
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = four[i];
    }
    __device__ __forceinline__ void forget()
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) asm volatile("" : "+v"(c[j]));
    }
};

template <int DT, int P, int V, bool FAR> __device__ __forceinline__ void rstd_of(const Spot<DT, P, V, FAR> &t, const RmsBwdArgs &a, float (&rstd)[V])
{
    Words<0, V> w;
    w.clear();
    if (t.left > 0) {
        w.load(reinterpret_cast<src_t>(a.rstd + t.position(0) - t.back), 0);
        if (t.back) move_down<0, V>(w, t.back);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) rstd[i] = w[i];
}

// gamma dy h, added up over the octet's channels for each pixel; dy h over the pixels for each channel
template <int DT, int P, int V, bool FAR, bool HELD>
__device__ __forceinline__ void add_products(const RmsBwdArgs &a, const Words<DT, V> (&dy)[8], const NormedMaps<DT, P, V, FAR, HELD> &vs, const float (&gamma)[8], const float (&rstd)[V],
                                             float (&q)[V], float (&dg)[8])
{
    float sum[V] = {};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float s[V];
        vs.values(a, j, s);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float p = dy[j][i] * (s[i] * rstd[i]);
            sum[i] += p * gamma[j];
            dg[j] += p;
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) q[i] += sum[i];
}
template <int DT, int P, int V, bool FAR, bool HELD>
__device__ __forceinline__ void put_gradients(const Spot<DT, P, V, FAR> &t, const RmsBwdArgs &a, int o, const Words<DT, V> (&dy)[8], const NormedMaps<DT, P, V, FAR, HELD> &vs,
                                              const float (&gamma)[8], const float (&rstd)[V], const float (&mean)[V])
{
    float f[8][V];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float s[V];
        vs.values(a, j, s);
#pragma unroll
        for (int i = 0; i < V; ++i) f[j][i] = rstd[i] * (dy[j][i] * gamma[j] - s[i] * rstd[i] * mean[i]);
    }
    if (a.dsum.p) {
        Words<DT, V> d[8];
        t.load(a.dsum, o, d);
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) f[j][i] += d[j][i];
    }
    t.store(a.dx, o, f);
}

// Backwards; a workgroup keeps its threads' sums for dgamma in registers over its tiles, adds them up over its pixels' lanes at the end and writes a copy of them.
// 4 x 64 x 388^2 bf16 from int8, 193 MB in 62 us = 3.1 TB/s, and the copies' sum 5: a tile's loads, sums and stores follow one another, and the four workgroups of a CU do
// not cover all of that.  In 16 bits 128 registers (four workgroups; some spilled) or 200 (two): 62 and 64 us; fp32 spills too many.  With the copies' sum: from a tensor 62 us = 3.8
// TB/s, fp32 100 = 4.6, from int8 85 = 4.1.  (The next tile's loads at 200 registers: not tried.)
template <int DT, int P, int V, int K, int T, bool HELD> __global__ __launch_bounds__(T, DT == 0 ? 2 : 4) void rms_maps_bwd_kernel(RmsBwdArgs a, long tiles, long tiles_of_image)
{
    __shared__ float part[T > 64 ? 2 * (T / 64) * P * V : 1];
    constexpr bool FAR = K == 0;
    Spot<DT, P, V, FAR> t(a);
    int half = 0;
    float dg[K ? K : 1][8] = {};
    for (long tile = neighbour(); tile < tiles; tile += gridDim.x) {       // (every thread alike)
        t.go(tile, tiles_of_image);
        Words<DT, V> dy[K ? K : 1][8];
        NormedMaps<DT, P, V, FAR, HELD> vs[K ? K : 1];
        float rstd[V], q[V] = {}, gamma[8];
        rstd_of(t, a, rstd);
        if (K) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                t.load(a.dy, t.octet0 + k * t.octets, dy[k]);
                vs[k].load(t, a, t.octet0 + k * t.octets);
            }
#pragma unroll
            for (int k = 0; k < K; ++k) {
                t.gamma(a.gamma, t.octet0 + k * t.octets, gamma);
                add_products(a, dy[k], vs[k], gamma, rstd, q, dg[k]);
            }
        } else {
            for (int o = t.octet0; t.channels(o) > 0; o += t.octets) {
                float none[8];
                t.load(a.dy, o, dy[0]);
                vs[0].load(t, a, o);
                t.gamma(a.gamma, o, gamma);
                add_products(a, dy[0], vs[0], gamma, rstd, q, none);
            }
        }
        t.total(q, part, half);
        if (!a.dx.p) continue;
#pragma unroll
        for (int i = 0; i < V; ++i) q[i] /= (float)a.c;
        if (K) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int o = t.octet0 + k * t.octets;
#pragma unroll
                for (int j = 0; j < 8; ++j) dy[k][j].forget();
                vs[k].forget();
                t.gamma(a.gamma, o, gamma);
                put_gradients(t, a, o, dy[k], vs[k], gamma, rstd, q);
            }
        } else {
            for (int o = t.octet0; t.channels(o) > 0; o += t.octets) {
                t.load(a.dy, o, dy[0]);
                vs[0].load(t, a, o);
                t.gamma(a.gamma, o, gamma);
                put_gradients(t, a, o, dy[0], vs[0], gamma, rstd, q);
            }
        }
    }
    if (!K || !a.dgamma) return;
    float *out = gridDim.x == 1 ? a.dgamma : a.scratch + blockIdx.x * rms_copy_floats(a.c);
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float v = sum_lanes<P>(dg[k][j]);
            const int c = 8 * (t.octet0 + k * t.octets) + j;
            if (t.lane == 0 && c < a.c) out[c] = v;
        }
}

// dgamma where no workgroup keeps all channels: eight of them a workgroup, a position a lane, blockIdx.y a share of the positions.
template <int DT, bool HELD> __global__ __launch_bounds__(256) void rms_deep_dgamma_kernel(RmsBwdArgs a)
{
    typedef elem_t<DT> E;
    __shared__ float part[4][8];
    float *out = gridDim.y == 1 ? a.dgamma : a.scratch + blockIdx.y * rms_copy_floats(a.c);
    const long positions = a.n * a.plane;
    for (long c0 = 8L * blockIdx.x; c0 < a.c; c0 += 8L * gridDim.x) {
        float dg[8] = {};
        for (long q = blockIdx.y * 256L + threadIdx.x; q < positions; q += gridDim.y * 256L) {
            const long b = positions < (1L << 32) ? (long)((uint32_t)q / (uint32_t)a.plane) : q / a.plane, m = q - b * a.plane;
            const float rstd = a.rstd[q];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const long c = std::min<long>(c0 + j, a.c - 1);
                const float dy = (float)static_cast<const E *>(a.dy.p)[b * a.dy.sn + c * a.dy.sc + m];
                float s;
                if constexpr (HELD) {
                    const uint32_t code = a.s8.codes[b * a.s8.sn + c * a.s8.sc + m];
                    const float scale = Code8<E4M3>::scale(a.s8.scales[b * a.s8.ssn + c * a.s8.ssc + m / 32]);
                    s = a.s8.code == E4M3 ? Code8<E4M3>::value(code, scale) : Code8<I8>::value(code, scale);
                } else {
                    s = (float)static_cast<const E *>(a.s.p)[b * a.s.sn + c * a.s.sc + m];
                }
                dg[j] += dy * (s * rstd);
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float v = sum_lanes<64>(dg[j]);
            if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6][j] = v;
        }
        __syncthreads();
        if (threadIdx.x < 8 && c0 + threadIdx.x < a.c)
            out[c0 + threadIdx.x] = (part[0][threadIdx.x] + part[1][threadIdx.x]) + (part[2][threadIdx.x] + part[3][threadIdx.x]);
        __syncthreads();
    }
}

// copies of dgamma's sums: one a workgroup that keeps them, or the shares of the positions
int copies_of(const NormSpan &s, int p, int v, int k, int threads)
{
    if (!k) return (int)std::min<long>((s.n * s.plane + 1023) / 1024, 64);
    // up to four tiles are one workgroup's: no second launch, whose 4 us are two tiles' time
    const long tiles = s.n * tiles_per_image(s, p * v);
    return tiles <= 4 ? 1 : (int)std::min<long>(tiles, std::max(1, 256 * 1024 / threads));
}

}  // namespace

// (maps far apart have fewer)
int rms_maps_bwd_copies(const NormSpan &s)
{
    int copies = 1;
    for (bool far : {false, true})
        pick_maps(s, far, [&](auto p, auto v, auto k, auto) { copies = std::max(copies, copies_of(s, p(), v(), k(), threads_of(s, p()))); });
    return copies;
}

hipError_t launch_rms_maps_bwd(const RmsBwdArgs &a, hipStream_t stream)
{
    const bool far = far_maps(a, {&a.dy, &a.s, &a.dsum, &a.dx}, {&a.s8});
    Launches done;
    auto go = [&](auto dt, auto held) {
        pick_maps(a, far, [&](auto p, auto v, auto k, auto t) {
            const long per = tiles_per_image(a, p() * v()), tiles = a.n * per;
            const int threads = threads_of(a, p()), copies = copies_of(a, p(), v(), k(), threads);
            if (!k() && a.dgamma) {                     // first: dx may go to the place of dy or s
                rms_deep_dgamma_kernel<dt(), held()><<<dim3((unsigned)std::min((a.c + 7) / 8, 65536), copies), 256, 0, stream>>>(a);
                if (done.failed() || (copies > 1 && done.failed(launch_rms_reduce(a.scratch, copies, a.dgamma, a.c, stream)))) return;
            }
            if (!k() && !a.dx.p) return;
            rms_maps_bwd_kernel<dt(), p(), v(), k(), t(), held()><<<k() ? (unsigned)copies : norm_blocks(tiles, 1), threads, 0, stream>>>(a, tiles, per);
            if (done.failed() || !k() || !a.dgamma || copies == 1) return;
            done.failed(launch_rms_reduce(a.scratch, copies, a.dgamma, a.c, stream));
        });
    };
    pick_dtype(a.dtype, [&](auto dt) {
        if (a.s8.codes) go(dt, std::true_type{});
        else go(dt, std::false_type{});
    });
    return done.status();
}

}  // namespace sk
