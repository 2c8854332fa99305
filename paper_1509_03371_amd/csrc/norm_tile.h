// Layer norm of maps: how a workgroup shares out pixels and channels (internal device code).
#pragma once
#include <initializer_list>

#include "norm_device.h"

namespace sk {

// the values of channels c0 .. c0 + 7 (left: how many there are; the others, and all of a null pointer, are `without`)
__device__ __forceinline__ void octet_values(const float *p, int c0, int left, float without, float (&f)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = without;
    if (!p) return;
    if (left >= 8) {
        const line_t<0, 8> v = *reinterpret_cast<const line_t<0, 8> *>(p + c0);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = v[j];
    } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < left) f[j] = p[c0 + j];
    }
}

// Where a thread stands.  A workgroup takes P * V pixels of one image and all channels (or as many octets at a time as it has threads / P): thread t the
// V pixels of lane t % P in the eight channels of octet t / P.
template <int DT, int LAYOUT, int P, int V> struct Tile {
    typedef elem_t<DT> E;
    static constexpr int S = sizeof(E);
    // eight channels of V pixels, as read
    struct Octet {
        Words<DT, V> line[LAYOUT == MAPS ? 8 : 1];      // MAPS: a channel's pixels
        Words<DT, 8> unit[LAYOUT == MAPS ? 1 : V];      // OCTETS: a pixel's channels
        __device__ __forceinline__ float at(int j, int v) const { return LAYOUT == MAPS ? line[j][v] : unit[v][j]; }
        __device__ __forceinline__ void forget()
        {
            if (LAYOUT == MAPS)
#pragma unroll
                for (int j = 0; j < 8; ++j) line[LAYOUT == MAPS ? j : 0].forget();
            else
#pragma unroll
                for (int v = 0; v < V; ++v) unit[LAYOUT == MAPS ? 0 : v].forget();
        }
    };
    const long plane, row;                              // row: tiles of an image
    const bool narrow;                                  // the number of tiles has 32 bits
    const int c;
    const int lane, delta, oct0;                        // octet: oct0 of the wave's first lane + delta
    long b, start;                                      // image, first pixel of the tile
    uint32_t length, px;                                // MAPS: its pixels, and where this lane's begin

    __device__ __forceinline__ Tile(long plane_, long row_, long tiles, int c_)
        : plane(plane_), row(row_), narrow(tiles < (1L << 32)), c(c_), lane(threadIdx.x % P), delta((threadIdx.x & 63) / P),
          oct0(uniform(threadIdx.x >> 6) * (64 / P))
    {
    }
    __device__ __forceinline__ int octet() const { return oct0 + delta; }
    __device__ __forceinline__ void go(long tile)
    {
        b = narrow ? (long)((uint32_t)tile / (uint32_t)row) : tile / row;
        start = (tile - b * row) * (P * V);
        if (LAYOUT == MAPS) {
            const Stretch<V> s(start, P * V, plane, V * lane);
            start = s.start;
            length = s.length;
            px = s.at;
        } else {
            px = lane;
        }
    }
    // number of pixel v inside the plane: V in a row where a plane's are neighbours, P apart where an octet's are (there the last for those behind it)
    __device__ __forceinline__ uint32_t behind(int v) const
    {
        if (LAYOUT == MAPS) return px + v;
        const uint32_t last = (uint32_t)std::min<long>(plane - 1 - start, P * V);
        return std::min<uint32_t>(v * P + lane, last);
    }
    __device__ __forceinline__ long pixel(int v) const { return start + behind(v); }
    __device__ __forceinline__ long position(int v) const { return b * plane + pixel(v); }
    __device__ __forceinline__ bool inside(int v) const { return LAYOUT == MAPS || start + v * P + lane < plane; }
    // ... and does it count here in sums over pixels?
    __device__ __forceinline__ bool own(int v) const { return LAYOUT == MAPS ? px + v >= (uint32_t)(V * lane) : inside(v); }
    __device__ __forceinline__ bool stores() const { return LAYOUT != MAPS || (uint32_t)(V * lane) < length; }
    // Every thread loads, whole vectors and without a branch.  Channels behind the last repeat the last one's address, threads without an octet the first
    // of their wave; what they hold must not count.  o0: the wave's first octet, which has channels.
    __device__ __forceinline__ int channels(int o0) const { return c - 8 * (o0 + delta); }       // of this thread's octet: 8 and more = all
    __device__ __forceinline__ long base(const NormView &w, int o0) const
    {
        return S * (LAYOUT == MAPS ? b * w.sn + 8L * o0 * w.sc + start : b * w.sn + o0 * w.sc + 8 * start);
    }
    // from one channel (MAPS) or octet to the next, in bytes.  Opaque, or the compiler keeps eight multiples of it for every operand across the loop
    // over tiles, in more registers than the scalar unit has.
    // FAR: a wave's lanes are all in one octet, and the steps are added to the base, in 64 bits; else to the lanes' offsets, in 32.
    static constexpr bool FAR = LAYOUT == MAPS && P == 64;
    typedef typename std::conditional<FAR, long, uint32_t>::type Step;
    __device__ __forceinline__ Step step(const NormView &w) const
    {
        Step v = S * (Step)w.sc;
        asm volatile("" : "+s"(v));
        return v;
    }
    __device__ __forceinline__ void load(const NormView &w, int o0, Octet &raw) const
    {
        const int left = channels(o0);
        const src_t p = static_cast<src_t>(w.p) + base(w, o0);
        const Step up = step(w);
        if constexpr (FAR) {
            const int last = std::max(0, std::min(7, left - 1));
#pragma unroll
            for (int j = 0; j < 8; ++j) raw.line[j].load(p + up * std::min(j, last), S * px);
        } else if constexpr (LAYOUT == MAPS) {
            const uint32_t off = (left > 0 ? 8 * up * delta : 0) + S * px, last = up * std::max(0, std::min(7, left - 1));
#pragma unroll
            for (int j = 0; j < 8; ++j) raw.line[j].load(p, off + std::min(up * j, last));
        } else {
            const uint32_t off = left > 0 ? up * delta : 0;
#pragma unroll
            for (int v = 0; v < V; ++v) raw.unit[v].load(p, off + 8 * S * behind(v));
        }
    }
    // zeros for values that stand in for none (repeats of the last channel, of the wave's first octet): a factor of zero would make NaN of infinite ones.
    // Behind the last channel of OCTETS there are none in memory.
    __device__ __forceinline__ void blank(int o0, Octet &raw) const
    {
        const int left = channels(o0);
        if (left >= 8) return;
        if (LAYOUT == MAPS) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j >= left) raw.line[LAYOUT == MAPS ? j : 0].clear();
        } else if (left <= 0) {
#pragma unroll
            for (int v = 0; v < V; ++v) raw.unit[LAYOUT == MAPS ? 0 : v].clear();
        }
    }
    // where line i of an octet that has channels lies: a channel's (MAPS) or a pixel's unit (OCTETS)
    struct Lines {
        dst_t p;
        uint32_t off;
        Step up;
        __device__ __forceinline__ dst_t base(int i) const { return FAR ? p + i * up : p; }
        __device__ __forceinline__ uint32_t offset(int i) const { return FAR ? off : off + i * (LAYOUT == MAPS ? (uint32_t)up : 8 * S * P); }
    };
    __device__ __forceinline__ Lines lines(const NormView &w, int o0) const
    {
        const Step up = step(w);
        const uint32_t first = FAR ? S * px : LAYOUT == MAPS ? 8 * (uint32_t)up * delta + S * px : (uint32_t)up * delta + 8 * S * lane;
        return {static_cast<dst_t>(w.p) + base(w, o0), first, up};
    }
    __device__ __forceinline__ void store(const NormView &w, int o0, const float (&f)[8][V]) const
    {
        const int left = channels(o0);
        if (left <= 0 || !stores()) return;
        const Lines at = lines(w, o0);
        if (LAYOUT == MAPS) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < left) store_at<DT, V>(at.base(j), at.offset(j), f[j]);
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (inside(v)) {
                    float u[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) u[j] = j < left ? f[j][v] : 0.f;
                    store_at<DT, 8>(at.base(v), at.offset(v), u);
                }
        }
    }
    // the numbers of an octet's channels at each pixel
    __device__ __forceinline__ void draw(const DropMask &d, uint64_t counter, int o, uint32_t (&w)[V][4]) const
    {
#pragma unroll
        for (int v = 0; v < V; ++v) mask_words(w[v], d, counter, (uint64_t)position(v), o);
    }
    // s = x, or residual + dropout(x), of an octet
    template <bool ADD> __device__ __forceinline__ void values(const NormArgs &a, uint64_t counter, int o0, float (&s)[8][V]) const
    {
        Octet x, r;
        load(a.x, o0, x);
        if (ADD && a.residual.p) load(a.residual, o0, r);
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int v = 0; v < V; ++v) s[j][v] = x.at(j, v);
        if (ADD && a.drop.thresh) {
            uint32_t w[V][4];
            draw(a.drop, counter, o0 + delta, w);
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) s[j][v] = dropped(s[j][v], w[v], j, a.drop);
        }
        if (ADD && a.residual.p)
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) s[j][v] += r.at(j, v);
    }
    // sum over the octet's channels
    __device__ __forceinline__ void add_channels(int o0, const float (&s)[8][V], float (&sum)[V]) const
    {
        const int left = channels(o0);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float q = 0.f;
            if (c % 8 == 0) {                           // every octet is whole
#pragma unroll
                for (int j = 0; j < 8; ++j) q += s[j][v];
                q = left > 0 ? q : 0.f;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) q += j < left ? s[j][v] : 0.f;
            }
            sum[v] += q;
        }
    }
    // sum over the octet's channels of (s - mean)^2
    __device__ __forceinline__ void add_squares(int o0, const float (&s)[8][V], const float (&mean)[V], float (&var)[V]) const
    {
        const int left = c - 8 * (o0 + delta);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float q = 0.f;
            if (c % 8 == 0) {
#pragma unroll
                for (int j = 0; j < 8; ++j) q += (s[j][v] - mean[v]) * (s[j][v] - mean[v]);
                q = left > 0 ? q : 0.f;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) q += j < left ? (s[j][v] - mean[v]) * (s[j][v] - mean[v]) : 0.f;
            }
            var[v] += q;
        }
    }
    // y from s, and s itself where it is asked for
    template <bool ADD> __device__ __forceinline__ void put(const NormArgs &a, int o0, float (&s)[8][V], const float (&mean)[V], const float (&rstd)[V]) const
    {
        const int c0 = 8 * (o0 + delta), left = c - c0;
        if (left <= 0) return;
        if (ADD && a.sum.p) store(a.sum, o0, s);
        float gamma[8], beta[8];
        octet_values(a.gamma, c0, left, 1.f, gamma);
        octet_values(a.beta, c0, left, 0.f, beta);
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int v = 0; v < V; ++v) s[j][v] = (s[j][v] - mean[v]) * rstd[v] * gamma[j] + beta[j];
        if (a.relu)
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) s[j][v] = s[j][v] < 0.f ? 0.f : s[j][v];
        store(a.y, o0, s);
    }
    __device__ __forceinline__ void statistics(const float *p, float (&f)[V]) const
    {
        if (LAYOUT == MAPS) {
            Words<0, V> u;
            u.load(reinterpret_cast<src_t>(p + b * plane + start), 4 * px);
#pragma unroll
            for (int v = 0; v < V; ++v) f[v] = u[v];
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) f[v] = p[position(v)];
        }
    }
    __device__ __forceinline__ void put_statistics(const NormArgs &a, const float (&mean)[V], const float (&rstd)[V]) const
    {
        if (octet() == 0 && stores())
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (inside(v)) {
                    if (a.mean) a.mean[position(v)] = mean[v];
                    if (a.rstd) a.rstd[position(v)] = rstd[v];
                }
    }
    // N sums over all channels of each pixel; part: two halves of [N][waves][P * V], taken in turn (one barrier a call)
    template <int N> __device__ __forceinline__ void total(float (&s)[N][V], float *part, int &half) const
    {
        typedef float Sums __attribute__((ext_vector_type(V)));
        const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int v = 0; v < V; ++v) s[n][v] = sum_over_groups<P>(s[n][v]);
        if (waves == 1) return;
        Sums *p = reinterpret_cast<Sums *>(part) + half * N * waves * P;
        half ^= 1;
        if (delta == 0)
#pragma unroll
            for (int n = 0; n < N; ++n) {
                Sums u;
#pragma unroll
                for (int v = 0; v < V; ++v) u[v] = s[n][v];
                p[(n * waves + wave) * P + lane] = u;
            }
        __syncthreads();
        // the 64 / P octets of a wave share the waves' sums out among them
#pragma unroll
        for (int n = 0; n < N; ++n) {
            Sums u{};
            for (int i = delta; i < waves; i += 64 / P) u += p[(n * waves + i) * P + lane];
#pragma unroll
            for (int v = 0; v < V; ++v) s[n][v] = sum_over_groups<P>(u[v]);
        }
    }
};

template <int N> using num = std::integral_constant<int, N>;

// f(P, T) and the threads of a workgroup that holds c channels; false: more than it can.  BACK: backwards
template <bool BACK, class F> bool pick_planes(int c, F f)
{
    const int octs = (c + 7) / 8;
    auto go = [&](auto p, auto t) {
        f(p, t, (octs * p() + 63) / 64 * 64);
        return true;
    };
    if (octs <= 4) return go(num<64>{}, num<256>{});
    if (octs <= 8) return go(num<32>{}, num<256>{});
    if (octs <= 16) return go(num<16>{}, num<256>{});
    if (octs <= 64) return go(num<BACK ? 8 : 16>{}, num<BACK ? 512 : 1024>{});
    if (octs <= 128) return go(num<8>{}, num<1024>{});
    if (octs <= 256) return go(num<4>{}, num<1024>{});
    return false;
}

// the views' strides between octets that a wave of P pixel lanes spans have 32 bits of bytes
inline bool spans(const NormSpan &s, int p, std::initializer_list<const NormView *> views)
{
    for (const NormView *v : views)
        if (p < 64 && v->p && (64 / p) * (s.layout == MAPS ? 8 : 1) * v->sc >= (1L << 30)) return false;      // elements of at most four bytes
    return true;
}

template <class F> void pick_type(const NormSpan &s, F f)
{
    if (s.dtype == 0) return f(num<0>{}, num<MAPS>{});
    if (s.dtype == 1) return s.layout == MAPS ? f(num<1>{}, num<MAPS>{}) : f(num<1>{}, num<OCTETS>{});
    return s.layout == MAPS ? f(num<2>{}, num<MAPS>{}) : f(num<2>{}, num<OCTETS>{});
}

// f(P, V) of the kernels that take octets in turn
template <class F> void pick_deep(const NormSpan &s, bool far, F f)
{
    if (s.layout == MAPS && s.plane < 4) return far ? f(num<64>{}, num<1>{}) : f(num<4>{}, num<1>{});
    return far ? f(num<64>{}, num<4>{}) : f(num<16>{}, num<4>{});
}

inline int deep_threads(int c, int p) { return std::min(1024, ((c + 7) / 8 * p + 63) / 64 * 64); }
inline size_t part_bytes(int sums, int p, int v, int threads) { return threads > 64 ? sizeof(float) * 2 * sums * (threads / 64) * p * v : 0; }
inline long tiles_of_image(const NormSpan &s, int pixels) { return (s.plane + pixels - 1) / pixels; }

}  // namespace sk
