// Layer norm of maps: planes of pixels, one after the other (MAPS) or in octets of channels (OCTETS).
#include "norm_device.h"

namespace sk {

namespace {

constexpr int V = 4;                                    // pixels of a thread

// A workgroup takes P * 4 pixels of one image and all channels: thread t holds the pixels of lane t % P in the channels of octet t / P, in registers:
// one read of every input and one write of every output.  Sums over the channels: a thread's own, the
// wave's, then the waves' through LDS.
template <int DT, int LAYOUT, int P> struct Tile {
    typedef elem_t<DT> E;
    long b, pixel;                                      // image; first pixel of the tile
    int lane, oct, octs;                                // octs: octets of the workgroup
    long plane;
    int c;
    // pixel number v of this thread inside the plane: four in a row where a plane's are neighbours, P apart where an octet's are
    __device__ __forceinline__ long at(int v) const { return LAYOUT == MAPS ? pixel + V * lane + v : pixel + v * P + lane; }
    __device__ __forceinline__ int slot(int v) const { return LAYOUT == MAPS ? V * lane + v : v * P + lane; }
    // 8 channels x 4 pixels of octet o, zeros outside
    __device__ __forceinline__ void load(const NormView &w, int o, line_t<DT, V> (&raw)[8]) const
    {
        const E *p = static_cast<const E *>(w.p) + b * w.sn;
        if (LAYOUT == MAPS) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                raw[j] = 8 * o + j < c ? load_line<DT, V>(p + (8L * o + j) * w.sc, pixel + V * lane, plane) : line_t<DT, V>{};
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                line_t<DT, 8> u{};
                if (8 * o < c && at(v) < plane) u = *reinterpret_cast<const line_t<DT, 8> *>(p + o * w.sc + 8 * at(v));
#pragma unroll
                for (int j = 0; j < 8; ++j) raw[j][v] = u[j];
            }
        }
    }
    __device__ __forceinline__ void store(const NormView &w, int o, const float (&f)[8][V]) const
    {
        E *p = static_cast<E *>(w.p) + b * w.sn;
        if (LAYOUT == MAPS) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (8 * o + j < c) store_line<DT, V>(p + (8L * o + j) * w.sc, pixel + V * lane, plane, f[j]);
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (8 * o < c && at(v) < plane) {
                    line_t<DT, 8> u;
#pragma unroll
                    for (int j = 0; j < 8; ++j) u[j] = static_cast<E>(8 * o + j < c ? f[j][v] : 0.f);
                    *reinterpret_cast<line_t<DT, 8> *>(p + o * w.sc + 8 * at(v)) = u;
                }
        }
    }
    __device__ __forceinline__ long position(int v) const { return b * plane + at(v); }
    // f, 0 where the mask drops
    __device__ __forceinline__ void drop(const DropMask &d, uint64_t base, int o, float (&f)[8][V]) const
    {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            uint32_t w[4];
            mask_words(w, d, base, (uint64_t)position(v), o);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j][v] = dropped(f[j][v], w, j, d);
        }
    }
    __device__ __forceinline__ void statistics(const float *p, float (&f)[V]) const
    {
        if (LAYOUT == MAPS) {
            const line_t<0, V> u = load_line<0, V>(p + b * plane, pixel + V * lane, plane);
#pragma unroll
            for (int v = 0; v < V; ++v) f[v] = u[v];
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) f[v] = at(v) < plane ? p[position(v)] : 0.f;
        }
    }
    // N sums over all channels of each pixel; part: two halves of [N][waves][P * 4], taken in turn (one barrier a call)
    template <int N> __device__ __forceinline__ void total(float (&s)[N][V], float *part, int &half) const
    {
        const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
        float *p = part + half * N * waves * P * V;
        half ^= 1;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int v = 0; v < V; ++v) s[n][v] = sum_over_groups<P>(s[n][v]);
        if (waves == 1) return;
        if ((threadIdx.x & 63) < P)
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int v = 0; v < V; ++v) p[(n * waves + wave) * P * V + v * P + lane] = s[n][v];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int v = 0; v < V; ++v) s[n][v] = 0.f;
        for (int i = 0; i < waves; ++i)
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int v = 0; v < V; ++v) s[n][v] += p[(n * waves + i) * P * V + v * P + lane];
    }
};

template <int DT, int LAYOUT, int P, int T> __global__ __launch_bounds__(T) void norm_planes_kernel(NormArgs a, long tiles, long row)
{
    extern __shared__ float part[];
    Tile<DT, LAYOUT, P> t;
    t.lane = threadIdx.x % P;
    t.oct = threadIdx.x / P;
    t.octs = blockDim.x / P;
    t.plane = a.plane;
    t.c = a.c;
    const uint64_t base = a.drop.base();
    int half = 0;
    for (long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        t.b = tile / row;                               // row: tiles of an image
        t.pixel = tile % row * (P * V);
        float s[8][V], sum[1][V] = {};
        {
            line_t<DT, V> x[8];
            t.load(a.x, t.oct, x);
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int v = 0; v < V; ++v) s[j][v] = (float)x[j][v];
        }
        if (a.drop.thresh)
            t.drop(a.drop, base, t.oct, s);
        if (a.residual.p) {
            line_t<DT, V> r[8];
            t.load(a.residual, t.oct, r);
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int v = 0; v < V; ++v) s[j][v] += (float)r[j][v];
        }
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) sum[0][v] += s[j][v];
        t.template total<1>(sum, part, half);
        float mean[V], rstd[V], var[1][V] = {};
#pragma unroll
        for (int v = 0; v < V; ++v) mean[v] = sum[0][v] / (float)a.c;
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float d = 8 * t.oct + j < a.c ? s[j][v] - mean[v] : 0.f;
                    var[0][v] += d * d;
                }
        t.template total<1>(var, part, half);
#pragma unroll
        for (int v = 0; v < V; ++v) rstd[v] = 1.f / sqrtf(var[0][v] / (float)a.c + a.eps);
        const int o = t.oct;
        if (8 * o < a.c) {
            if (a.sum.p) t.store(a.sum, o, s);
            const line_t<0, 8> g = a.gamma ? load_line<0, 8>(a.gamma, 8 * o, a.c) : line_t<0, 8>{}, be = a.beta ? load_line<0, 8>(a.beta, 8 * o, a.c) : line_t<0, 8>{};
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    float y = (s[j][v] - mean[v]) * rstd[v];
                    if (a.gamma) y *= g[j];
                    y += be[j];
                    s[j][v] = a.relu && y < 0.f ? 0.f : y;
                }
            t.store(a.y, o, s);
        }
        if (t.oct == 0)
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (t.at(v) < a.plane) {
                    if (a.mean) a.mean[t.position(v)] = mean[v];
                    if (a.rstd) a.rstd[t.position(v)] = rstd[v];
                }
    }
}

// More channels than the threads of a workgroup hold: read three times.
template <int DT, int LAYOUT> __global__ __launch_bounds__(1024) void norm_deep_planes_kernel(NormArgs a, long tiles, long row)
{
    constexpr int P = 16;
    extern __shared__ float part[];
    Tile<DT, LAYOUT, P> t;
    t.lane = threadIdx.x % P;
    t.oct = threadIdx.x / P;
    t.octs = blockDim.x / P;
    t.plane = a.plane;
    t.c = a.c;
    const uint64_t base = a.drop.base();
    const int last = (a.c + 7) / 8;
    int half = 0;
    auto values = [&](int o, float (&s)[8][V]) {
        line_t<DT, V> x[8];
        t.load(a.x, o, x);
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int v = 0; v < V; ++v) s[j][v] = (float)x[j][v];
        if (a.drop.thresh) t.drop(a.drop, base, o, s);
        if (a.residual.p) {
            t.load(a.residual, o, x);
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) s[j][v] += (float)x[j][v];
        }
    };
    for (long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        t.b = tile / row;
        t.pixel = tile % row * (P * V);
        float s[8][V], sum[1][V] = {}, var[1][V] = {}, mean[V], rstd[V];
        for (int o = t.oct; o < last; o += t.octs) {
            values(o, s);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float q = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) q += s[j][v];
                sum[0][v] += q;
            }
        }
        t.template total<1>(sum, part, half);
#pragma unroll
        for (int v = 0; v < V; ++v) mean[v] = sum[0][v] / (float)a.c;
        for (int o = t.oct; o < last; o += t.octs) {
            values(o, s);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float q = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float d = 8 * o + j < a.c ? s[j][v] - mean[v] : 0.f;
                    q += d * d;
                }
                var[0][v] += q;
            }
        }
        t.template total<1>(var, part, half);
#pragma unroll
        for (int v = 0; v < V; ++v) rstd[v] = 1.f / sqrtf(var[0][v] / (float)a.c + a.eps);
        for (int o = t.oct; o < last; o += t.octs) {
            values(o, s);
            if (a.sum.p) t.store(a.sum, o, s);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool in = 8 * o + j < a.c;
                const float g = a.gamma && in ? a.gamma[8 * o + j] : 1.f, be = a.beta && in ? a.beta[8 * o + j] : 0.f;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float y = (s[j][v] - mean[v]) * rstd[v] * g + be;
                    s[j][v] = a.relu && y < 0.f ? 0.f : y;
                }
            }
            t.store(a.y, o, s);
        }
        if (t.oct == 0)
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (t.at(v) < a.plane) {
                    if (a.mean) a.mean[t.position(v)] = mean[v];
                    if (a.rstd) a.rstd[t.position(v)] = rstd[v];
                }
    }
}

// Backwards: a workgroup walks the tiles gridDim.x apart and keeps its threads' sums for dgamma and dbeta in registers until the end, where they go to the
// workgroup's copy of the scratch, or to dgamma and dbeta themselves if there is one workgroup.
template <int DT, int LAYOUT, int P, int T> __global__ __launch_bounds__(T) void norm_planes_bwd_kernel(NormBwdArgs a, long tiles, long row)
{
    extern __shared__ float part[];
    Tile<DT, LAYOUT, P> t;
    t.lane = threadIdx.x % P;
    t.oct = threadIdx.x / P;
    t.octs = blockDim.x / P;
    t.plane = a.plane;
    t.c = a.c;
    const uint64_t base = a.drop.base();
    float gamma[8], dg[8], db[8];
    const line_t<0, 8> g8 = a.gamma ? load_line<0, 8>(a.gamma, 8 * t.oct, a.c) : line_t<0, 8>{};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        gamma[j] = a.gamma ? g8[j] : 1.f;
        dg[j] = db[j] = 0.f;
    }
    int half = 0;
    for (long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        t.b = tile / row;
        t.pixel = tile % row * (P * V);
        line_t<DT, V> vy[8], vs[8];
        t.load(a.dy, t.oct, vy);
        t.load(a.s, t.oct, vs);
        float mean[V], rstd[V], sums[2][V] = {};
        t.statistics(a.mean, mean);
        t.statistics(a.rstd, rstd);
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) {           // outside the tensor y is zero
                    const float h = ((float)vs[j][v] - mean[v]) * rstd[v], y = (float)vy[j][v], g = y * gamma[j];
                    sums[0][v] += g;
                    sums[1][v] += g * h;
                    dg[j] += y * h;
                    db[j] += y;
                }
        t.template total<2>(sums, part, half);
        if (!a.dx.p && !a.dresidual.p) continue;
        float mg[V], mgh[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            mg[v] = sums[0][v] / (float)a.c;
            mgh[v] = sums[1][v] / (float)a.c;
        }
        const int o = t.oct;
        if (8 * o < a.c) {
            float f[8][V];
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float h = ((float)vs[j][v] - mean[v]) * rstd[v];
                    f[j][v] = rstd[v] * ((float)vy[j][v] * gamma[j] - mg[v] - h * mgh[v]);
                }
            if (a.dsum.p) {
                line_t<DT, V> d[8];
                t.load(a.dsum, o, d);
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int v = 0; v < V; ++v) f[j][v] += (float)d[j][v];
            }
            if (a.dresidual.p) t.store(a.dresidual, o, f);
            if (!a.dx.p) continue;
            if (a.drop.thresh) t.drop(a.drop, base, o, f);
            if (a.relu_x)
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int v = 0; v < V; ++v) f[j][v] = (float)vs[j][v] > 0.f ? f[j][v] : 0.f;
            t.store(a.dx, o, f);
        }
    }
    if (!a.dgamma && !a.dbeta) return;
    // an octet belongs to the P lanes that hold its pixels
    const bool alone = gridDim.x == 1;
    const long cp = norm_copy_floats(a.c) / 2;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float *out = alone ? (which ? a.dbeta : a.dgamma) : a.scratch + (blockIdx.x * 2L + which) * cp;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = sum_lanes<P>(which ? db[j] : dg[j]);
        if (out && t.lane == 0 && 8 * t.oct < a.c) store_line<0, 8>(out, 8 * t.oct, a.c, v);
    }
}

// More channels than that: read twice, and once more for the sums of dgamma and dbeta.
template <int DT, int LAYOUT> __global__ __launch_bounds__(1024) void norm_deep_planes_bwd_kernel(NormBwdArgs a, long tiles, long row)
{
    constexpr int P = 16;
    extern __shared__ float part[];
    Tile<DT, LAYOUT, P> t;
    t.lane = threadIdx.x % P;
    t.oct = threadIdx.x / P;
    t.octs = blockDim.x / P;
    t.plane = a.plane;
    t.c = a.c;
    const uint64_t base = a.drop.base();
    const int last = (a.c + 7) / 8;
    int half = 0;
    for (long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        t.b = tile / row;
        t.pixel = tile % row * (P * V);
        float mean[V], rstd[V], sums[2][V] = {}, f[8][V];
        t.statistics(a.mean, mean);
        t.statistics(a.rstd, rstd);
        line_t<DT, V> vy[8], vs[8];
        for (int o = t.oct; o < last; o += t.octs) {
            t.load(a.dy, o, vy);
            t.load(a.s, o, vs);
            float q[2][V] = {};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float gamma = a.gamma && 8 * o + j < a.c ? a.gamma[8 * o + j] : 1.f;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float g = (float)vy[j][v] * gamma;
                    q[0][v] += g;
                    q[1][v] += g * (((float)vs[j][v] - mean[v]) * rstd[v]);
                }
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                sums[0][v] += q[0][v];
                sums[1][v] += q[1][v];
            }
        }
        t.template total<2>(sums, part, half);
        for (int o = t.oct; o < last; o += t.octs) {
            t.load(a.dy, o, vy);
            t.load(a.s, o, vs);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float gamma = a.gamma && 8 * o + j < a.c ? a.gamma[8 * o + j] : 1.f;
#pragma unroll
                for (int v = 0; v < V; ++v)
                    f[j][v] = rstd[v] * ((float)vy[j][v] * gamma - sums[0][v] / (float)a.c - ((float)vs[j][v] - mean[v]) * rstd[v] * (sums[1][v] / (float)a.c));
            }
            if (a.dsum.p) {
                t.load(a.dsum, o, vy);
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int v = 0; v < V; ++v) f[j][v] += (float)vy[j][v];
            }
            if (a.dresidual.p) t.store(a.dresidual, o, f);
            if (!a.dx.p) continue;
            if (a.drop.thresh) t.drop(a.drop, base, o, f);
            if (a.relu_x)
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int v = 0; v < V; ++v) f[j][v] = (float)vs[j][v] > 0.f ? f[j][v] : 0.f;
            t.store(a.dx, o, f);
        }
    }
}

// ... a wave an octet of channels, blockIdx.y a share of the tiles of 256 pixels
template <int DT, int LAYOUT> __global__ __launch_bounds__(64) void norm_deep_planes_wgrad_kernel(NormBwdArgs a, long tiles, long row)
{
    Tile<DT, LAYOUT, 64> t;
    t.lane = threadIdx.x;
    t.plane = a.plane;
    t.c = a.c;
    const long cp = norm_copy_floats(a.c) / 2;
    const int o = blockIdx.x;
    float dg[8] = {}, db[8] = {};
    for (long tile = blockIdx.y; tile < tiles; tile += gridDim.y) {
        t.b = tile / row;
        t.pixel = tile % row * (64 * V);
        line_t<DT, V> vy[8], vs[8];
        float mean[V], rstd[V];
        t.load(a.dy, o, vy);
        t.load(a.s, o, vs);
        t.statistics(a.mean, mean);
        t.statistics(a.rstd, rstd);
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                dg[j] += (float)vy[j][v] * (((float)vs[j][v] - mean[v]) * rstd[v]);
                db[j] += (float)vy[j][v];
            }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        dg[j] = sum_lanes<64>(dg[j]);
        db[j] = sum_lanes<64>(db[j]);
    }
    if (t.lane == 0) {
        store_line<0, 8>(a.scratch + blockIdx.y * 2L * cp, 8 * o, a.c, dg);
        store_line<0, 8>(a.scratch + (blockIdx.y * 2L + 1) * cp, 8 * o, a.c, db);
    }
}

constexpr int kDeep = 2048;                             // channels that the registers of a workgroup hold

// f(P, T) and the threads of a workgroup for c channels
template <class F> hipError_t pick_planes(int c, F f)
{
    const int octs = (c + 7) / 8;
    auto go = [&](auto p, auto t) { return f(p, t, (octs * p() + 63) / 64 * 64); };
    typedef std::integral_constant<int, 256> small;
    typedef std::integral_constant<int, 1024> large;
    if (octs <= 4) return go(std::integral_constant<int, 64>{}, small{});
    if (octs <= 8) return go(std::integral_constant<int, 32>{}, small{});
    if (octs <= 16) return go(std::integral_constant<int, 16>{}, small{});
    if (octs <= 64) return go(std::integral_constant<int, 16>{}, large{});
    if (octs <= 128) return go(std::integral_constant<int, 8>{}, large{});
    return go(std::integral_constant<int, 4>{}, large{});
}

template <class F> hipError_t pick_type(const NormSpan &s, F f)
{
    typedef std::integral_constant<int, MAPS> maps;
    typedef std::integral_constant<int, OCTETS> octets;
    if (s.dtype == 0) return f(std::integral_constant<int, 0>{}, maps{});
    if (s.dtype == 1) return s.layout == MAPS ? f(std::integral_constant<int, 1>{}, maps{}) : f(std::integral_constant<int, 1>{}, octets{});
    return s.layout == MAPS ? f(std::integral_constant<int, 2>{}, maps{}) : f(std::integral_constant<int, 2>{}, octets{});
}

size_t part_bytes(int sums, int p, int threads) { return threads > 64 ? sizeof(float) * 2 * sums * (threads / 64) * p * V : 0; }

}  // namespace

hipError_t launch_norm_planes(const NormArgs &a, hipStream_t stream)
{
    return pick_type(a, [&](auto dt, auto layout) {
        if (a.c > kDeep) {
            const long row = (a.plane + 63) / 64;
            norm_deep_planes_kernel<dt(), layout()><<<norm_blocks(a.n * row, 1), 1024, part_bytes(1, 16, 1024), stream>>>(a, a.n * row, row);
            return hipGetLastError();
        }
        return pick_planes(a.c, [&](auto p, auto t, int threads) {
            const long row = (a.plane + p() * V - 1) / (p() * V);
            norm_planes_kernel<dt(), layout(), p(), t()><<<norm_blocks(a.n * row, 1), threads, part_bytes(1, p(), threads), stream>>>(a, a.n * row, row);
            return hipGetLastError();
        });
    });
}

int norm_planes_bwd_copies(const NormSpan &s)
{
    if (s.c > kDeep) return (int)std::min<long>(s.n * ((s.plane + 255) / 256), 16);
    int copies = 1;
    (void)pick_planes(s.c, [&](auto p, auto, int threads) {
        copies = (int)std::min<long>(s.n * ((s.plane + p() * V - 1) / (p() * V)), 256 * std::max(1, 1024 / threads));
        return hipSuccess;
    });
    return copies;
}

hipError_t launch_norm_planes_bwd(const NormBwdArgs &a, int copies, hipStream_t stream)
{
    return pick_type(a, [&](auto dt, auto layout) {
        if (a.c > kDeep) {
            if (a.dgamma || a.dbeta) {
                const long row = (a.plane + 255) / 256;
                norm_deep_planes_wgrad_kernel<dt(), layout()><<<dim3((unsigned)((a.c + 7) / 8), copies), 64, 0, stream>>>(a, a.n * row, row);
                if (hipError_t e = launch_norm_reduce(a.scratch, copies, a.dgamma, a.dbeta, a.c, stream)) return e;
            }
            const long row = (a.plane + 63) / 64;
            if (a.dx.p || a.dresidual.p)
                norm_deep_planes_bwd_kernel<dt(), layout()><<<norm_blocks(a.n * row, 1), 1024, part_bytes(2, 16, 1024), stream>>>(a, a.n * row, row);
            return hipGetLastError();
        }
        return pick_planes(a.c, [&](auto p, auto t, int threads) {
            const long row = (a.plane + p() * V - 1) / (p() * V);
            norm_planes_bwd_kernel<dt(), layout(), p(), t()><<<copies, threads, part_bytes(2, p(), threads), stream>>>(a, a.n * row, row);
            if ((a.dgamma || a.dbeta) && copies > 1) return launch_norm_reduce(a.scratch, copies, a.dgamma, a.dbeta, a.c, stream);
            return hipGetLastError();
        });
    });
}

}  // namespace sk
