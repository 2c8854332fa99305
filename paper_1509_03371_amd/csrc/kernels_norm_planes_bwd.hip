// Layer norm of maps, backwards (see norm_tile.h).
#include "norm_tile.h"

namespace sk {

namespace {

// The gradients of an octet from its dy and s (both kept as they were read) and the four numbers of each pixel.
// ADD: with dropout, dsum or dresidual.
template <bool ADD, int DT, int LAYOUT, int P, int V>
__device__ __forceinline__ void put_gradients(const Tile<DT, LAYOUT, P, V> &t, const NormBwdArgs &a, uint64_t counter, int o0,
                                              typename Tile<DT, LAYOUT, P, V>::Octet &vy, typename Tile<DT, LAYOUT, P, V>::Octet &vs, const float (&gamma)[8],
                                              const float (&mean)[V], const float (&rstd)[V], const float (&mg)[V], const float (&mgh)[V])
{
    const int left = t.channels(o0);
    if (left <= 0 || !t.stores()) return;
    const bool drops = ADD && a.drop.thresh && a.dx.p;
    uint32_t w[V][4];
    if (drops) t.draw(a.drop, counter, o0 + t.delta, w);
    float mr[V];                                        // rstd (gamma dy - mg - h mgh) with h = (s - mean) rstd
#pragma unroll
    for (int v = 0; v < V; ++v) mr[v] = mgh[v] * rstd[v];
    auto gradient = [&](int j, int v) { return rstd[v] * (product(vy.at(j, v), gamma[j]) - mg[v] - (vs.at(j, v) - mean[v]) * mr[v]); };
    auto to_x = [&](int j, int v, float f) {
        if (drops) f = dropped(f, w[v], j, a.drop);
        if (a.relu_x) f = vs.at(j, v) > 0.f ? f : 0.f;
        return f;
    };
    // a line at a time, each behind a branch of its own: together the values of all lines are more than the registers hold
    typedef typename Tile<DT, LAYOUT, P, V>::Lines Lines;
    const Lines sum = ADD ? t.lines(a.dsum, o0) : Lines{}, residual = ADD ? t.lines(a.dresidual, o0) : Lines{}, x = t.lines(a.dx, o0);
    constexpr bool maps = LAYOUT == MAPS;
    constexpr int L = maps ? 8 : V, N = maps ? V : 8;   // lines, and elements of one
#pragma unroll
    for (int i = 0; i < L; ++i) {
        if (maps ? i >= left : !t.inside(i)) continue;
        float f[N];
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = maps ? gradient(i, e) : e < left ? gradient(e, i) : 0.f;
        if (ADD && a.dsum.p) {
            Words<DT, N> d;
            d.load(sum.base(i), sum.offset(i));
#pragma unroll
            for (int e = 0; e < N; ++e) f[e] += d[e];
        }
        if (ADD && a.dresidual.p) store_at<DT, N>(residual.base(i), residual.offset(i), f);
        if (ADD && !a.dx.p) continue;
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = maps ? to_x(i, e, f[e]) : to_x(e, i, f[e]);
        store_at<DT, N>(x.base(i), x.offset(i), f);
    }
}

// dgamma and dbeta of octet o by a wave, over the tiles first, first + step, ... of its 64 * V pixels; the sums in every lane
template <int DT, int LAYOUT, int V>
__device__ __forceinline__ void norm_planes_sums(const NormBwdArgs &a, int o, long first, long step, long tiles, long row, float (&g)[8], float (&s)[8])
{
    Tile<DT, LAYOUT, 64, V> t(a.plane, row, tiles, a.c);
    float dg[8] = {}, db[8] = {};
    for (long tile = first; tile < tiles; tile += step) {
        t.go(tile);
        typename Tile<DT, LAYOUT, 64, V>::Octet vy, vs;
        float mean[V], rstd[V];
        t.load(a.dy, o, vy);
        t.load(a.s, o, vs);
        t.statistics(a.mean, mean);
        t.statistics(a.rstd, rstd);
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float mine = t.own(v) ? vy.at(j, v) : 0.f;
                dg[j] += mine * ((vs.at(j, v) - mean[v]) * rstd[v]);
                db[j] += mine;
            }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        g[j] = sum_lanes<64>(dg[j]);
        s[j] = sum_lanes<64>(db[j]);
    }
}

// pixels of a thread: four while it may have 256 registers, else two
constexpr int bwd_pixels(int threads) { return threads == 1024 ? 2 : 4; }

// Backwards: a workgroup walks the tiles gridDim.x apart and keeps its threads' sums for dgamma and dbeta in registers until the end, where they go to the
// workgroup's copy of the scratch, or to dgamma and dbeta themselves if there is one workgroup.  The grid is what fits the registers at once.
// 4 x 64 x 388^2 bf16: 236 MB in 60 us, the sums of 512 copies (4.7 us) with it = 3.9 TB/s; planes of 128-byte multiples 43 us + 4.7, these begin at any
// multiple of 32, and their segments touch a fifth line in four.  What did not help: the next tile's loads in flight (57.5 us for 57.1), 64-pixel
// segments without a barrier (68), 512-byte segments (68: one workgroup a CU).
// fp32 of 513 to 2048 channels with residual or dropout spills 19 to 20 registers (1000 x 10001: 200 MB in 98 us); 16 bits of these widths fit (60 us).
//
// ROLES, for few pixels: the first `walkers` workgroups leave the sums alone, and each of the others takes them for an octet over all pixels, which are
// read twice (from the L2): one launch and no workspace.

template <int DT, int LAYOUT, int P, int T, bool ADD, bool ROLES>
__global__ __launch_bounds__(T, T == 1024 ? 4 : 2) void norm_planes_bwd_kernel(NormBwdArgs a, long tiles, long row, int walkers)
{
    if (ROLES && blockIdx.x >= (unsigned)walkers) {
        __shared__ float sums[T / 64][16];
        const long wide = (a.plane + 255) / 256;        // tiles of a wave's 64 * 4 pixels
        const int o = blockIdx.x - walkers, wave = uniform(threadIdx.x >> 6), waves = blockDim.x >> 6;
        float g[8], s[8];
        norm_planes_sums<DT, LAYOUT, 4>(a, o, wave, waves, a.n * wide, wide, g, s);
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sums[wave][j] = g[j];
                sums[wave][8 + j] = s[j];
            }
        __syncthreads();
        const int c = 8 * o + (threadIdx.x & 7);
        float *out = threadIdx.x < 8 ? a.dgamma : a.dbeta;
        if (threadIdx.x >= 16 || c >= a.c || !out) return;
        float v = 0.f;
        for (int i = 0; i < waves; ++i) v += sums[i][threadIdx.x];
        out[c] = v;
        return;
    }
    constexpr int V = bwd_pixels(T);
    extern __shared__ __align__(16) float part[];
    Tile<DT, LAYOUT, P, V> t(a.plane, row, tiles, a.c);
    const uint64_t counter = ADD ? a.drop.base() : 0;
    const int c0 = 8 * t.octet(), left = a.c - c0;
    float gamma[8], dg[8], db[8];
    octet_values(a.gamma, c0, left, 1.f, gamma);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        gamma[j] = j < left ? gamma[j] : 0.f;           // what does not count adds nothing to the sums over channels
        dg[j] = db[j] = 0.f;
    }
    int half = 0;
    for (long tile = ROLES ? blockIdx.x : neighbour(); tile < tiles; tile += walkers) {
        t.go(tile);
        typename Tile<DT, LAYOUT, P, V>::Octet vy, vs;
        t.load(a.dy, t.oct0, vy);
        t.load(a.s, t.oct0, vs);
        t.blank(t.oct0, vy);
        float mean[V], rstd[V], sums[2][V] = {};
        t.statistics(a.mean, mean);
        t.statistics(a.rstd, rstd);
        uint32_t counts[V];                             // zeros where another lane counts the pixel (a factor of zero would make NaN of an infinite y)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            counts[v] = t.own(v) ? ~0u : 0u;
            if (T != 1024) asm volatile("" : "+v"(counts[v]));  // a word a pixel; where registers are short the compiler's select by the scalar unit
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float d = vs.at(j, v) - mean[v], y = vy.at(j, v), g = product(y, gamma[j]);
                sums[0][v] += g;
                sums[1][v] += g * d;
                if (ROLES) continue;
                const float mine = __uint_as_float(__float_as_uint(y) & counts[v]);
                dg[j] += mine * rstd[v] * d;
                db[j] += mine;
            }
        t.template total<2>(sums, part, half);
        if (!a.dx.p && !a.dresidual.p) continue;
        float mg[V], mgh[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            mg[v] = sums[0][v] / (float)a.c;
            mgh[v] = sums[1][v] * rstd[v] / (float)a.c;
        }
        if (T == 1024) {
            vy.forget();
            vs.forget();
        }
        put_gradients<ADD>(t, a, counter, t.oct0, vy, vs, gamma, mean, rstd, mg, mgh);
    }
    if (ROLES || (!a.dgamma && !a.dbeta)) return;
    // an octet belongs to the P lanes that hold its pixels
    const bool alone = gridDim.x == 1;
    const long cp = norm_copy_floats(a.c) / 2;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float *out = alone ? (which ? a.dbeta : a.dgamma) : a.scratch + (blockIdx.x * 2L + which) * cp;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = sum_lanes<P>(which ? +db[j] : +dg[j]);
        if (!out || t.lane != 0) continue;
        if (left >= 8) {
            *reinterpret_cast<line_t<0, 8> *>(out + c0) = packed<0, 8>(v);
        } else {
#pragma unroll
            for (int j = 0; j < 7; ++j)
                if (j < left) out[c0 + j] = v[j];
        }
    }
}

// As norm_deep_planes_kernel: read twice, and once more for the sums of dgamma and dbeta.
template <int DT, int LAYOUT, int P, int V> __global__ __launch_bounds__(1024) void norm_deep_planes_bwd_kernel(NormBwdArgs a, long tiles, long row)
{
    extern __shared__ __align__(16) float part[];
    Tile<DT, LAYOUT, P, V> t(a.plane, row, tiles, a.c);
    const uint64_t counter = a.drop.base();
    const int last = (a.c + 7) / 8, octs = blockDim.x / P;
    int half = 0;
    for (long tile = neighbour(); tile < tiles; tile += gridDim.x) {
        t.go(tile);
        float mean[V], rstd[V], sums[2][V] = {}, mg[V], mgh[V], gamma[8];
        t.statistics(a.mean, mean);
        t.statistics(a.rstd, rstd);
        typename Tile<DT, LAYOUT, P, V>::Octet vy, vs;
        auto take = [&](int o0) {
            t.load(a.dy, o0, vy);
            t.load(a.s, o0, vs);
            t.blank(o0, vy);
            const int c0 = 8 * (o0 + t.delta);
            octet_values(a.gamma, c0, a.c - c0, 1.f, gamma);
#pragma unroll
            for (int j = 0; j < 8; ++j) gamma[j] = c0 + j < a.c ? gamma[j] : 0.f;
        };
        for (int o0 = t.oct0; o0 < last; o0 += octs) {
            take(o0);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float q = 0.f, r = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float g = product(vy.at(j, v), gamma[j]);
                    q += g;
                    r += g * ((vs.at(j, v) - mean[v]) * rstd[v]);
                }
                sums[0][v] += q;
                sums[1][v] += r;
            }
        }
        t.template total<2>(sums, part, half);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            mg[v] = sums[0][v] / (float)a.c;
            mgh[v] = sums[1][v] / (float)a.c;
        }
        for (int o0 = t.oct0; o0 < last; o0 += octs) {
            take(o0);
            put_gradients<true>(t, a, counter, o0, vy, vs, gamma, mean, rstd, mg, mgh);
        }
    }
}

// The sums of planes of fewer than four pixels, as norm_planes_sums: a wave's lanes take positions side by side, of as many images as they reach over
// (a wave an image and sixteen shares of them: 100000 x 20 x 3 fp32 4307 us with the results, so 146; 200000 x 64 x 2 bf16 9449 and 353).
template <int DT>
__device__ __forceinline__ void norm_small_planes_sums(const NormBwdArgs &a, int o, long first, long step, float (&g)[8], float (&s)[8])
{
    constexpr int S = sizeof(elem_t<DT>);
    const int last = std::min(7, a.c - 8 * o - 1);
    float dg[8] = {}, db[8] = {};
    for (long q = first * 64 + threadIdx.x; q < a.n * a.plane; q += step * 64) {
        const long b = a.plane == 1 ? q : a.plane == 2 ? q / 2 : q / 3, m = q - b * a.plane;
        const src_t y = static_cast<src_t>(a.dy.p) + S * (b * a.dy.sn + 8L * o * a.dy.sc + m), x = static_cast<src_t>(a.s.p) + S * (b * a.s.sn + 8L * o * a.s.sc + m);
        Words<DT, 1> vy[8], vs[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {                   // (channels behind the last repeat it, and are not written)
            vy[j].load(y + S * a.dy.sc * std::min(j, last), 0);
            vs[j].load(x + S * a.s.sc * std::min(j, last), 0);
        }
        const float mean = a.mean[q], rstd = a.rstd[q];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            dg[j] += vy[j][0] * ((vs[j][0] - mean) * rstd);
            db[j] += vy[j][0];
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        g[j] = sum_lanes<64>(dg[j]);
        s[j] = sum_lanes<64>(db[j]);
    }
}

// ... a wave an octet of channels, blockIdx.y a share of the tiles
template <int DT, int LAYOUT, int V> __global__ __launch_bounds__(64) void norm_deep_planes_wgrad_kernel(NormBwdArgs a, long tiles, long row)
{
    const long cp = norm_copy_floats(a.c) / 2;
    float *dgamma = gridDim.y == 1 ? a.dgamma : a.scratch + blockIdx.y * 2L * cp;
    float *dbeta = gridDim.y == 1 ? a.dbeta : a.scratch + (blockIdx.y * 2L + 1) * cp;
    for (int o = blockIdx.x; 8 * o < a.c; o += gridDim.x) {
        float g[8], s[8];
        if constexpr (V == 1) norm_small_planes_sums<DT>(a, o, blockIdx.y, gridDim.y, g, s);
        else norm_planes_sums<DT, LAYOUT, V>(a, o, blockIdx.y, gridDim.y, tiles, row, g, s);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (threadIdx.x == 0 && 8 * o + j < a.c) {
                if (dgamma) dgamma[8 * o + j] = g[j];
                if (dbeta) dbeta[8 * o + j] = s[j];
            }
    }
}

}  // namespace

// Where ROLES take the work: up to sixteen tiles of 256 pixels and 2^21 elements.  With roles and with copies and a second launch, us, bf16: 64 x 128 4.1 and 4.9,
// 1024 x 784 6.0 and 9.6, 64 x 4096 6.4 and 7.4, 256 x 4096 6.5 and 8.2, 1024 x 2000 9.6 and 10.5; 64 x 8192 10.2 and 7.5, 256 x 8192 11.1 and 9.1,
// 1024 x 4096 20.5 and 13.3.
static bool takes_roles(const NormSpan &s)
{
    return (s.layout == OCTETS || s.plane >= 4) && (s.c + 7) / 8 <= 256 && s.n * tiles_of_image(s, 256) <= 16 && s.n * s.plane * s.c <= 1L << 21;
}
// workgroups that the registers hold at once
static int resident(int t, int threads) { return 256 * std::max(1, (t == 1024 ? 16 : 8) / (threads / 64)); }

// planes of fewer than four pixels: shares of 64 positions, as many as make some 2048 waves with the octets
static bool small_planes(const NormSpan &s) { return s.layout == MAPS && s.plane < 4; }
static int small_planes_shares(const NormSpan &s)
{
    return (int)std::min<long>((s.n * s.plane + 63) / 64, std::max(16, 2048 / ((s.c + 7) / 8)));
}

// (a call whose strides 32 bits do not span takes fewer: it walks octets, whose copies are at most 16)
int norm_planes_bwd_copies(const NormSpan &s)
{
    int copies = 16;
    if (takes_roles(s)) return 1;
    if (small_planes(s)) return small_planes_shares(s);
    pick_planes<true>(s.c, [&](auto p, auto t, int threads) {
        copies = (int)std::min<long>(s.n * tiles_of_image(s, p() * bwd_pixels(t())), resident(t(), threads));
    });
    return copies;
}

hipError_t launch_norm_planes_bwd(const NormBwdArgs &a, int copies, hipStream_t stream)
{
    auto fits = [&](int p) { return spans(a, p, {&a.dy, &a.s, &a.dsum, &a.dx, &a.dresidual}); };
    const bool sums = a.dgamma || a.dbeta, results = a.dx.p || a.dresidual.p, adds = a.dsum.p || a.dresidual.p || a.drop.thresh;
    Launches done;
    pick_type(a, [&](auto dt, auto layout) {
        bool taken = false;
        if (layout() == OCTETS || a.plane >= 4)
            pick_planes<true>(a.c, [&](auto p, auto t, int threads) {
                if (!fits(p())) return;
                const long row = tiles_of_image(a, p() * bwd_pixels(t())), tiles = a.n * row;
                const size_t lds = part_bytes(2, p(), bwd_pixels(t()), threads);
                taken = true;
                const int all = (int)std::min<long>(tiles, resident(t(), threads));
                const bool roles = sums && takes_roles(a);
                if (roles) {
                    const int walkers = results && !a.in_place() ? all : 0, blocks = walkers + (a.c + 7) / 8;
                    if (adds) norm_planes_bwd_kernel<dt(), layout(), p(), t(), true, true><<<blocks, threads, lds, stream>>>(a, tiles, row, walkers);
                    else norm_planes_bwd_kernel<dt(), layout(), p(), t(), false, true><<<blocks, threads, lds, stream>>>(a, tiles, row, walkers);
                    if (done.failed() || walkers || !results) return;
                }
                NormBwdArgs b = a;
                if (roles) b.dgamma = b.dbeta = nullptr;
                if (roles || !sums) copies = all;
                if (adds) norm_planes_bwd_kernel<dt(), layout(), p(), t(), true, false><<<copies, threads, lds, stream>>>(b, tiles, row, copies);
                else norm_planes_bwd_kernel<dt(), layout(), p(), t(), false, false><<<copies, threads, lds, stream>>>(b, tiles, row, copies);
                if (!done.failed() && sums && !roles && copies > 1) done.failed(launch_norm_reduce(a.scratch, copies, a.dgamma, a.dbeta, a.c, stream));
            });
        if (taken) return;
        pick_deep(a, !fits(4), [&](auto p, auto v) {
            if (sums) {
                const long row = tiles_of_image(a, 64 * v()), tiles = a.n * row;
                const int shares = small_planes(a) ? std::min(copies, small_planes_shares(a)) : (int)std::min<long>(std::min(copies, 16), tiles);
                norm_deep_planes_wgrad_kernel<dt(), layout(), v()><<<dim3(std::min((a.c + 7) / 8, 65536), shares), 64, 0, stream>>>(a, tiles, row);
                if (done.failed() || (shares > 1 && done.failed(launch_norm_reduce(a.scratch, shares, a.dgamma, a.dbeta, a.c, stream)))) return;
            }
            if (!results) return;
            const long row = tiles_of_image(a, p() * v()), tiles = a.n * row;
            const int threads = deep_threads(a.c, p());
            norm_deep_planes_bwd_kernel<dt(), layout(), p(), v()><<<norm_blocks(tiles, 1), threads, part_bytes(2, p(), v(), threads), stream>>>(a, tiles, row);
        });
    });
    return done.status();
}

}  // namespace sk
