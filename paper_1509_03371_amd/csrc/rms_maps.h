// Root-mean-square norm of maps: how a workgroup shares out pixels and channels (internal device code).
#pragma once
#include "rms.h"

namespace sk {

// V elements of a line that were read `back` elements early, because the line ends: moved down, zeros behind them
template <int DT, int V> __device__ __forceinline__ void move_down(Words<DT, V> &w, int back)
{
    if constexpr (V == 4 && DT == 0) {
        if (back & 2) { w.w[0] = w.w[2]; w.w[1] = w.w[3]; w.w[2] = w.w[3] = 0; }
        if (back & 1) { w.w[0] = w.w[1]; w.w[1] = w.w[2]; w.w[2] = w.w[3]; w.w[3] = 0; }
    } else if constexpr (V == 4) {
        const uint64_t v = ((uint64_t)w.w[1] << 32 | w.w[0]) >> 16 * back;
        w.w[0] = (uint32_t)v;
        w.w[1] = (uint32_t)(v >> 32);
    }
}
// the first 1 to 3 of four elements
template <int DT> __device__ __forceinline__ void store_some(dst_t p, int left, const float (&f)[4])
{
    const float first = f[0], third = f[2];             // (values: a choice of places would put f into memory)
    if (left & 2) store_at<DT, 2>(p, 0, {f[0], f[1]});
    if (left & 1) store_at<DT, 1>(p, sizeof(elem_t<DT>) * (left & 2), {left & 2 ? third : first});
}
typedef uint32_t code_word __attribute__((ext_vector_type(1), aligned(1)));
template <int V> __device__ __forceinline__ uint32_t load_codes_of(const uint8_t *p)
{
    if (V == 1) return *p;
    return (*reinterpret_cast<const code_word *>(p))[0];
}

// the largest of the lanes that hold a block's pixels: eight of four each, or four of one each
template <int V> __device__ __forceinline__ uint32_t max_of_pixels(uint32_t v)
{
    v = max_across<2>(max_across<1>(v));
    if (V == 1) return v;
    const uint32_t o = __builtin_amdgcn_mov_dpp(v, 0x141, 0xF, 0xF, true);     // eight lanes mirrored
    return v > o ? v : o;
}

// Where a thread stands.  A workgroup takes P * V pixels of one image from a block's beginning on, and as many octets of channels at a time as it has threads / P:
// thread t the V pixels of lane t % P in the eight channels of octet t / P.
// FAR: the channels of a wave's octets are further apart than 32 bits of bytes span.
template <int DT, int P, int V, bool FAR> struct Spot {
    static constexpr int S = sizeof(elem_t<DT>);
    typedef typename std::conditional<FAR, long, uint32_t>::type Off;
    const NormSpan &s;
    const int lane, octet0, octets;                     // octets: of the workgroup at a time
    long b, first;                                      // image, first pixel of the tile
    int left, back;                                     // of this lane's pixels (0: none); how much earlier it reads, so as not to read behind the line
    __device__ __forceinline__ explicit Spot(const NormSpan &s_) : s(s_), lane(threadIdx.x % P), octet0(threadIdx.x / P), octets(blockDim.x / P) {}
    __device__ __forceinline__ void go(long tile, long tiles_of_image)
    {
        b = tile < (1L << 32) ? (long)((uint32_t)tile / (uint32_t)tiles_of_image) : tile / tiles_of_image;
        first = (tile - b * tiles_of_image) * (P * V);
        const long n = s.plane - first - V * lane;
        left = n >= V ? V : n > 0 ? (int)n : 0;
        back = left > 0 ? V - left : 0;
    }
    // of an octet's channels: 8 and more = all, 0 and less = none
    __device__ __forceinline__ int channels(int o) const { return s.c - 8 * o; }
    // the lane's pixels in channel 8 o + j; `size` bytes an element
    __device__ __forceinline__ long base(long sn, long sc, int size, int j) const { return size * (b * sn + j * sc + first); }        // equal in all lanes
    __device__ __forceinline__ Off offset(long sc, int size, int o) const { return (Off)(8 * o) * (Off)(size * sc) + (Off)(size * V * lane); }
    // zeros where there is nothing
    __device__ __forceinline__ void load(const NormView &v, int o, Words<DT, V> (&w)[8]) const
    {
        const int n = channels(o);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j].clear();
        if (left <= 0 || n <= 0) return;
        // V elements early and V - back on again: offsets of 32 bits are none below zero
        const src_t early = static_cast<src_t>(v.p) - S * V;
        const Off off = offset(v.sc, S, o) + S * (V - back);
        if (n >= 8) {
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j].load(early + base(v.sn, v.sc, S, j) + off, 0);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < n) w[j].load(early + base(v.sn, v.sc, S, j) + off, 0);
        }
        if (back)
#pragma unroll
            for (int j = 0; j < 8; ++j) move_down<DT, V>(w[j], back);
    }
    __device__ __forceinline__ void store(const NormView &v, int o, const float (&f)[8][V]) const
    {
        const int n = channels(o);
        const Off off = offset(v.sc, S, o);
        if (left >= V && n >= 8) {
#pragma unroll
            for (int j = 0; j < 8; ++j) store_at<DT, V>(static_cast<dst_t>(v.p) + base(v.sn, v.sc, S, j) + off, 0, f[j]);
            return;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) {
                const dst_t p = static_cast<dst_t>(v.p) + base(v.sn, v.sc, S, j) + off;
                if (left >= V) store_at<DT, V>(p, 0, f[j]);
                else if constexpr (V == 4) store_some<DT>(p, left, f[j]);
            }
    }
    // f in 8 bits.  All threads of the workgroup come here, with zeros where there is nothing; f does not outlive it.
    __device__ __forceinline__ void pack(const PackedView &v, int o, float (&f)[8][V]) const
    {
        const int n = channels(o);
        const bool is_e4m3 = v.code == E4M3;            // (the same in all lanes)
        const uint32_t limit = is_e4m3 ? Code8<E4M3>::limit(DT) : Code8<I8>::limit(DT);
        uint32_t most[8], all = 0, odd = 0;             // odd: the values that are no numbers
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const uint32_t a = magnitude(f[j][i]);
                m = m > a ? m : a;
            }
            most[j] = max_of_pixels<V>(m);
            all = all > most[j] ? all : most[j];
        }
        if (all > limit)                                // (in all lanes of a block or in none)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t m = 0;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const uint32_t a = counted(f[j][i], limit);
                    odd |= (magnitude(f[j][i]) >= 0x7f800000u ? 1u : 0u) << (V * j + i);
                    f[j][i] = __uint_as_float(a | (__float_as_uint(f[j][i]) & 0x80000000u));
                    m = m > a ? m : a;
                }
                most[j] = max_of_pixels<V>(m);
            }
        uint32_t c[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            most[j] = is_e4m3 ? Code8<E4M3>::scale_byte(most[j]) : Code8<I8>::scale_byte(most[j]);
            const float inverse = Code8<E4M3>::inverse(most[j]);
            const float f1 = V > 1 ? f[j][V > 1 ? 1 : 0] : 0.f, f2 = V > 1 ? f[j][V > 1 ? 2 : 0] : 0.f, f3 = V > 1 ? f[j][V > 1 ? 3 : 0] : 0.f;
            c[j] = is_e4m3 ? Code8<E4M3>::four(f[j][0], f1, f2, f3, inverse) : Code8<I8>::four(f[j][0], f1, f2, f3, inverse);
        }
        if (odd) {
            const uint32_t nan = is_e4m3 ? Code8<E4M3>::nan : Code8<I8>::nan;
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (odd >> (V * j + i) & 1) c[j] = (c[j] & ~(0xffu << 8 * i)) | nan << 8 * i;
        }
        const Off at = offset(v.sc, 1, o);
        uint8_t *scale = v.scales + b * v.ssn + first / 32 + (Off)(8 * o) * (Off)v.ssc + V * lane / 32;
        const bool leads = V * lane % 32 == 0;
        if (left >= V && n >= 8) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint8_t *p = v.codes + base(v.sn, v.sc, 1, j) + at;
                if (V == 1) *p = (uint8_t)c[j];
                else __builtin_nontemporal_store(code_word{c[j]}, reinterpret_cast<code_word *>(p));
            }
            if (leads)
#pragma unroll
                for (int j = 0; j < 8; ++j) scale[j * v.ssc] = (uint8_t)most[j];
            return;
        }
        if (left <= 0) return;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) {
                uint8_t *p = v.codes + base(v.sn, v.sc, 1, j) + at;
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (i < left) p[i] = (uint8_t)(c[j] >> 8 * i);
                if (leads) scale[j * v.ssc] = (uint8_t)most[j];
            }
    }
    // gamma of an octet's channels; behind the last, 0
    __device__ __forceinline__ void gamma(const float *p, int o, float (&g)[8]) const
    {
        const int n = channels(o);
        if (!p) {
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = 1.f;
        } else if (n >= 8) {
            const line_t<0, 8> v = *reinterpret_cast<const line_t<0, 8> *>(p + 8 * o);
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = v[j];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = j < n ? p[8 * o + j] : 0.f;
        }
    }
    // sums over all channels of each pixel; part: two halves of [waves][P * V], taken in turn (one barrier a call)
    __device__ __forceinline__ void total(float (&q)[V], float *part, int &half) const
    {
        typedef float Sums __attribute__((ext_vector_type(V)));
        const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
#pragma unroll
        for (int i = 0; i < V; ++i) q[i] = sum_over_groups<P>(q[i]);
        if (waves == 1) return;
        Sums *p = reinterpret_cast<Sums *>(part) + half * waves * P;
        half ^= 1;
        const int group = (threadIdx.x & 63) / P;
        if (group == 0) {
            Sums u;
#pragma unroll
            for (int i = 0; i < V; ++i) u[i] = q[i];
            p[wave * P + lane] = u;
        }
        __syncthreads();
        Sums u{};
        for (int i = group; i < waves; i += 64 / P) u += p[i * P + lane];
#pragma unroll
        for (int i = 0; i < V; ++i) q[i] = sum_over_groups<P>(u[i]);
    }
    __device__ __forceinline__ long position(int i) const { return b * s.plane + first + V * lane + i; }
};

// f(P, V, K, T): pixel lanes, pixels a lane, octets a thread (0: more than fit the registers, or strides that 32 bits do not span; read twice), most threads.  Wide tiles
// make long lines.
template <class F> void pick_maps(const NormSpan &s, bool far, F f)
{
    const int octs = (s.c + 7) / 8;
    if (s.plane < 4) return f(num<4>{}, num<1>{}, num<0>{}, num<1024>{});
    if (far || octs > 128) return f(num<8>{}, num<4>{}, num<0>{}, num<1024>{});
    if (octs <= 4 && s.plane > 128) return f(num<64>{}, num<4>{}, num<1>{}, num<256>{});
    if (octs <= 8 && s.plane > 64) return f(num<32>{}, num<4>{}, num<1>{}, num<256>{});
    if (octs <= 16 && s.plane > 32) return f(num<16>{}, num<4>{}, num<1>{}, num<256>{});
    if (octs <= 32) return f(num<8>{}, num<4>{}, num<1>{}, num<256>{});
    f(num<8>{}, num<4>{}, num<1>{}, num<1024>{});
}
inline int threads_of(const NormSpan &s, int p) { return (int)std::min<long>(1024, ((s.c + 7L) / 8 * p + 63) / 64 * 64); }
inline long tiles_per_image(const NormSpan &s, int pixels) { return (s.plane + pixels - 1) / pixels; }

// the strides between the first and the last channel of a wave span 32 bits of bytes, of elements of at most four
inline bool far_maps(const NormSpan &s, std::initializer_list<const NormView *> views, std::initializer_list<const PackedView *> packed)
{
    for (const NormView *v : views)
        if (v->p && (s.c + 8) * v->sc >= (1L << 29)) return true;
    for (const PackedView *v : packed)
        if (v->codes && ((s.c + 8) * v->sc >= (1L << 31) || (s.c + 8) * v->ssc >= (1L << 31))) return true;
    return false;
}

}  // namespace sk
